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

#include <type_traits>

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
// UN groups a thread, all loads ahead. 64 x 2048 x 1408 bfloat16 77 us, 6.1 TB/s (four fifths
// of the bytes are reads); float32 153, 5.5.
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

// [K, R] to codes [R, K / 2]: a workgroup takes 512 values of K by 128 columns, a wave one
// block of 32 of K, half a wave half of it, a lane four columns: 16 loads ahead of 8 (16)
// bytes a lane, whole lines of two rows each. The halves exchange their largest magnitudes;
// codes go through LDS, so that 256 consecutive bytes of a column and 16 of its scales are
// written at once, whatever line they start in. Against 8 waves and two columns a lane (128
// and 8 bytes), bfloat16: 64 x 2048 x 1408 91.4 and 88.5 us (5.1 and 5.3 TB/s, a copy's
// rate), 64 x 1408 x 2048 86.6 and 98.5, 128 x 2880 x 2880, where columns start and end
// inside lines, 562 and 690. Workgroups that walk along K with the next block's loads
// ahead: no faster than that on any of them. (Call after call; behind another kernel, whose
// 370 MB of results still leave the caches, 64 x 2048 x 1408 takes 112. float32: 189, 4.4 TB/s.)
constexpr int TR_WAVES = 16, TR_COLS = 128;
template <bool F32>
__global__ void __launch_bounds__(64 * TR_WAVES)
mx_quantize_transposed(const void* __restrict__ src_, int64_t R, int K, uint8_t* __restrict__ codes,
                       uint8_t* __restrict__ scales) {
    __shared__ uint4 lds[TR_COLS][TR_WAVES + 1];
    __shared__ uint8_t sl[TR_COLS][TR_WAVES];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int half = lane >> 5, cl = (lane & 31) * 4;
    const int64_t n0 = (int64_t)blockIdx.x * TR_COLS, n = n0 + cl;   // R is even: all four columns, two or none
    const int kb0 = blockIdx.y * TR_WAVES, nkb = K / mx::BLOCK;
    const int64_t b = blockIdx.z;
    const int kb = kb0 + wv;
    if (n < R && kb < nkb) {
        using E = std::conditional_t<F32, float, bf16_t>;
        const E* p = static_cast<const E*>(src_) + (b * K + (int64_t)kb * mx::BLOCK + half * 16) * R + n;
        E raw[16][4];   // rows of an even number of elements: 4 bytes of alignment
        if (n + 4 <= R) {
#pragma unroll
            for (int i = 0; i < 16; ++i) __builtin_memcpy(raw[i], p + i * R, sizeof raw[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                __builtin_memcpy(raw[i], p + i * R, sizeof raw[i] / 2);
                raw[i][2] = raw[i][3] = E(0);
            }
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            float v[2][8];
            uint32_t t = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if constexpr (F32) v[i / 8][i % 8] = raw[i][c];
                else v[i / 8][i % 8] = bf2f(raw[i][c]);
                t = max(t, __float_as_uint(v[i / 8][i % 8]) & 0x7fffffffu);
            }
            t = max(t, (uint32_t)__shfl_xor((int)t, 32, 64));
            const uint32_t s = mx::scale_byte(t);
            const float sv = mx::scale_value(s);
            reinterpret_cast<uint2*>(&lds[cl + c][wv])[half] = make_uint2(mx::encode8(v[0], sv), mx::encode8(v[1], sv));
            if (half == (c & 1)) sl[cl + c][wv] = (uint8_t)s;
        }
    }
    __syncthreads();
    const int have = min(TR_WAVES, nkb - kb0);
#pragma unroll
    for (int p = 0; p < TR_COLS / 64; ++p) {
        const int i = threadIdx.x + p * 64 * TR_WAVES;
        const int col = i / TR_WAVES, q = i % TR_WAVES;
        if (n0 + col >= R || q >= have) continue;
        const int64_t blk = (b * R + n0 + col) * nkb + kb0 + q;
        st16(codes + blk * 16, lds[col][q]);
        scales[blk] = sl[col][q];
    }
}

// 16 bytes of values a lane, UN times: 8 or, in float32, 4 codes. 64 x 2048 x 1408 to bfloat16
// 81 us, 5.8 TB/s, to float32 156, 5.3, mostly writes either way. (Eight float32 values, two
// stores a lane 32 bytes apart from its neighbours': 4.0 TB/s, half lines a store.)
template <bool F32, int UN>
__global__ void __launch_bounds__(QT)
mx_dequantize_rows(const void* __restrict__ codes, const uint8_t* __restrict__ scales,
                   int64_t groups, uint4* __restrict__ out) {
    using Code = std::conditional_t<F32, uint16_t, uint32_t>;
    constexpr int N = F32 ? 4 : 8;
    const int64_t g0 = (int64_t)blockIdx.x * (QT * UN) + threadIdx.x;
    uint32_t c[UN], s[UN];
#pragma unroll
    for (int u = 0; u < UN; ++u) {
        const int64_t g = g0 + u * QT;
        if (g < groups) { c[u] = static_cast<const Code*>(codes)[g]; s[u] = scales[g / (mx::BLOCK / N)]; }
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
        for (int i = 0; i < N; ++i) v[i] *= sv;
        if constexpr (F32)
            st16(out + g, make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])));
        else
            st16(out + g, pack8(v));
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
    constexpr int UN = 4;
    const int64_t groups = n / (f32 ? 4 : 8);
    const dim3 grid((unsigned)((groups + QT * UN - 1) / (QT * UN)));
    const auto kernel = f32 ? &mx_dequantize_rows<true, UN> : &mx_dequantize_rows<false, UN>;
    hipLaunchKernelGGL(kernel, grid, dim3(QT), 0, st, codes, static_cast<const uint8_t*>(scales), groups,
                       static_cast<uint4*>(out));
    probe::mark("mx_dequantize", st);
    return hipGetLastError();
}

}  // namespace moe
