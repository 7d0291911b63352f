// mx.hip -- quantisation to and from microscaled 4-bit values (format: mx.hpp).
//
// Bound by HBM in both directions: 2 (or 4) bytes of a value in or out, 17/32 of a byte
// for its code and its share of the scale. In a row-major [R, K] array quantised along K
// the blocks of 32 follow each other through memory, whatever R and K are, so those
// kernels see one long run of blocks; the transposed form reads a [K, N] matrix (the
// layout of the layer's expert weights) and writes [N, K], the layout that the grouped
// products read.
#include "launch.hpp"
#include "mx.hpp"
#include "probe.hpp"

namespace moe {
namespace {

constexpr int QT = 256;

template <bool F32>
__device__ __forceinline__ void load8(const void* p, int64_t i, float (&v)[8]) {
    if constexpr (F32) {
        const uint4* q = reinterpret_cast<const uint4*>(static_cast<const float*>(p) + i);
        const uint4 a = q[0], b = q[1];
        v[0] = __uint_as_float(a.x); v[1] = __uint_as_float(a.y); v[2] = __uint_as_float(a.z); v[3] = __uint_as_float(a.w);
        v[4] = __uint_as_float(b.x); v[5] = __uint_as_float(b.y); v[6] = __uint_as_float(b.z); v[7] = __uint_as_float(b.w);
    } else {
        unpack8(ld16(static_cast<const bf16_t*>(p) + i), v);
    }
}

// largest magnitude as float bits: magnitudes order like their bit patterns, NaN above all
__device__ __forceinline__ uint32_t top8(const float (&v)[8]) {
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) t = max(t, __float_as_uint(v[i]) & 0x7fffffffu);
    return t;
}

// Four lanes a block, eight values a lane: each wave reads and writes consecutive bytes.
// UN groups a thread, all loads ahead.
template <bool F32, int UN>
__global__ void __launch_bounds__(QT)
mx_quantize_rows(const void* __restrict__ src, int64_t groups, uint32_t* __restrict__ codes,
                 uint8_t* __restrict__ scales) {
    const int64_t g0 = (int64_t)blockIdx.x * (QT * UN) + threadIdx.x;
    float v[UN][8];
#pragma unroll
    for (int u = 0; u < UN; ++u) {
        const int64_t g = g0 + u * QT;
        if (g < groups) load8<F32>(src, g * 8, v[u]);
    }
#pragma unroll
    for (int u = 0; u < UN; ++u) {
        const int64_t g = g0 + u * QT;
        uint32_t t = g < groups ? top8(v[u]) : 0u;
        t = max(t, (uint32_t)__shfl_xor((int)t, 1, 64));
        t = max(t, (uint32_t)__shfl_xor((int)t, 2, 64));
        const uint32_t s = mx::scale_byte(t);
        if (g >= groups) continue;
        codes[g] = mx::encode8(v[u], mx::scale_value(s));
        if ((g & 3) == 0) scales[g >> 2] = (uint8_t)s;
    }
}

// [K, R] to codes [R, K / 2]: a workgroup takes 256 values of K by 128 columns, a wave one
// block of 32 of K, a lane two columns: a block's 32 values never leave their lane, and the
// 16 bytes of its codes go through LDS so that whole 128-byte lines of a column are written.
constexpr int TR_WAVES = 8, TR_COLS = 128;
template <bool F32>
__global__ void __launch_bounds__(64 * TR_WAVES)
mx_quantize_transposed(const void* __restrict__ src_, int64_t R, int K, uint8_t* __restrict__ codes,
                       uint8_t* __restrict__ scales) {
    __shared__ uint4 lds[TR_COLS][TR_WAVES + 1];
    __shared__ uint8_t sl[TR_COLS][TR_WAVES];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int64_t n = (int64_t)blockIdx.x * TR_COLS + lane * 2;   // R is even: both columns or none
    const int kb0 = blockIdx.y * TR_WAVES, nkb = K / mx::BLOCK;
    const int64_t b = blockIdx.z;
    const int kb = kb0 + wv;
    if (n < R && kb < nkb) {
        const int64_t at = (b * K + (int64_t)kb * mx::BLOCK) * R + n;
        uint32_t raw[F32 ? 1 : 32];
        float2 rawf[F32 ? 32 : 1];
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            if constexpr (F32) rawf[i] = *reinterpret_cast<const float2*>(static_cast<const float*>(src_) + at + i * R);
            else raw[i] = *reinterpret_cast<const uint32_t*>(static_cast<const bf16_t*>(src_) + at + i * R);
        }
        auto val = [&](int c, int i) -> float {
            if constexpr (F32) return c ? rawf[i].y : rawf[i].x;
            else return c ? bf_hi(raw[i]) : bf_lo(raw[i]);
        };
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            uint32_t t = 0;
#pragma unroll
            for (int i = 0; i < 32; ++i) t = max(t, __float_as_uint(val(c, i)) & 0x7fffffffu);
            const uint32_t s = mx::scale_byte(t);
            const float sv = mx::scale_value(s);
            uint32_t o[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = val(c, q * 8 + i);
                o[q] = mx::encode8(v, sv);
            }
            lds[lane * 2 + c][wv] = make_uint4(o[0], o[1], o[2], o[3]);
            sl[lane * 2 + c][wv] = (uint8_t)s;
        }
    }
    __syncthreads();
    const int have = min(TR_WAVES, nkb - kb0);
#pragma unroll
    for (int p = 0; p < TR_COLS * TR_WAVES / (64 * TR_WAVES); ++p) {
        const int i = threadIdx.x + p * 64 * TR_WAVES;
        const int col = i / TR_WAVES, q = i % TR_WAVES;
        const int64_t row = (int64_t)blockIdx.x * TR_COLS + col;
        if (row >= R || q >= have) continue;
        const int64_t blk = (b * R + row) * nkb + kb0 + q;
        st16(codes + blk * 16, lds[col][q]);
        scales[blk] = sl[col][q];
    }
}

template <bool F32, int UN>
__global__ void __launch_bounds__(QT)
mx_dequantize_rows(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                   int64_t groups, void* __restrict__ out) {
    const int64_t g0 = (int64_t)blockIdx.x * (QT * UN) + threadIdx.x;
    uint32_t c[UN], s[UN];
#pragma unroll
    for (int u = 0; u < UN; ++u) {
        const int64_t g = g0 + u * QT;
        if (g < groups) { c[u] = codes[g]; s[u] = scales[g >> 2]; }
    }
#pragma unroll
    for (int u = 0; u < UN; ++u) {
        const int64_t g = g0 + u * QT;
        if (g >= groups) continue;
        // the codes alone are exact in bfloat16; scaling them in float32 rounds nothing
        // but results below its subnormals
        float v[8];
        unpack8(mx::decode8(c[u], 1.0f), v);
        const float sv = mx::scale_value(s[u]);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= sv;
        if constexpr (F32) {
            float* o = static_cast<float*>(out) + g * 8;
            st16(o, make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])));
            st16(o + 4, make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])));
        } else {
            st16(static_cast<bf16_t*>(out) + g * 8, pack8(v));
        }
    }
}

}  // namespace

hipError_t mx_quantize(const void* src, int64_t batch, int64_t R, int K, bool f32, bool transposed,
                       void* codes, void* scales, hipStream_t st) {
    if (transposed) {
        const dim3 grid((unsigned)((R + TR_COLS - 1) / TR_COLS),
                        (unsigned)((K / mx::BLOCK + TR_WAVES - 1) / TR_WAVES), (unsigned)batch);
        if (f32)
            hipLaunchKernelGGL(mx_quantize_transposed<true>, grid, dim3(64 * TR_WAVES), 0, st, src, R, K,
                               static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scales));
        else
            hipLaunchKernelGGL(mx_quantize_transposed<false>, grid, dim3(64 * TR_WAVES), 0, st, src, R, K,
                               static_cast<uint8_t*>(codes), static_cast<uint8_t*>(scales));
        probe::mark("mx_quantize_transposed", st);
        return hipGetLastError();
    }
    const int64_t groups = batch * R * (K / 8);
    constexpr int UN = 2;
    const dim3 grid((unsigned)((groups + QT * UN - 1) / (QT * UN)));
    if (f32)
        hipLaunchKernelGGL((mx_quantize_rows<true, UN>), grid, dim3(QT), 0, st, src, groups,
                           static_cast<uint32_t*>(codes), static_cast<uint8_t*>(scales));
    else
        hipLaunchKernelGGL((mx_quantize_rows<false, UN>), grid, dim3(QT), 0, st, src, groups,
                           static_cast<uint32_t*>(codes), static_cast<uint8_t*>(scales));
    probe::mark("mx_quantize", st);
    return hipGetLastError();
}

hipError_t mx_dequantize(const void* codes, const void* scales, int64_t n, bool f32, void* out,
                         hipStream_t st) {
    const int64_t groups = n / 8;
    constexpr int UN = 4;
    const dim3 grid((unsigned)((groups + QT * UN - 1) / (QT * UN)));
    if (f32)
        hipLaunchKernelGGL((mx_dequantize_rows<true, UN>), grid, dim3(QT), 0, st,
                           static_cast<const uint32_t*>(codes), static_cast<const uint8_t*>(scales), groups, out);
    else
        hipLaunchKernelGGL((mx_dequantize_rows<false, UN>), grid, dim3(QT), 0, st,
                           static_cast<const uint32_t*>(codes), static_cast<const uint8_t*>(scales), groups, out);
    probe::mark("mx_dequantize", st);
    return hipGetLastError();
}

}  // namespace moe
