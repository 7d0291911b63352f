// mx_gemm.hip -- products grouped by expert over weights in microscaled 4 bits (mx.hpp).
//
// out[s] = act(x[row(s)] w[e]^T), for SwiGLU SiLU(x w^T) * (x w3^T), for the slots s of
// each expert e; x in bfloat16, or in microscaled 4 bits too. Two cores:
//  * stream (few rows per expert, 16 or 32 a tile): bound by reading the weights once,
//    17/32 of a byte each;
//  * tiles (more rows): bound by the matrix cores.
// In both, the operands come by direct-to-LDS copies into a ring of slices. The weights
// stay 4-bit in LDS, a quarter of bfloat16's LDS traffic, and are converted as fragments.
// With bfloat16 rows the weights are converted exactly (v_cvt_scalef32_pk_bf16_fp4) and
// multiplied by the bfloat16 matrix instructions; with 4-bit rows both operands go to the
// scaled matrix instructions as they are. Sums are float32, and each output is rounded once.
//
// The order of K inside a matrix instruction is free as long as both operands agree: the
// layouts below give every lane whole blocks of 32 values, so that it needs one scale.
#include <algorithm>
#include <cmath>

#include "gemm.hpp"
#include "launch.hpp"
#include "mx.hpp"
#include "probe.hpp"

namespace moe {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ i32x8 fp4_operand(const uint4& c) {
    return i32x8{(int)c.x, (int)c.y, (int)c.z, (int)c.w, 0, 0, 0, 0};
}
// Operand format 4 is e2m1. Lane L supplies row (column) L % 16 of block L / 16 (16x16x128),
// or L % 32 of block L / 32 (32x32x64), and that block's scale in the low (or another) byte
// of its scale register; results as for the bfloat16 instructions (all checked on the device).
__device__ __forceinline__ f32x4 mfma_mx16(const uint4& p, uint32_t sp, const uint4& q, uint32_t sq, const f32x4& c) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fp4_operand(p), fp4_operand(q), c, 4, 4, 0, (int)sp, 0, (int)sq);
}
template <int BYTE>   // of the scale registers
__device__ __forceinline__ f32x16 mfma_mx32(const uint4& p, uint32_t sp, const uint4& q, uint32_t sq, const f32x16& c) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fp4_operand(p), fp4_operand(q), c, 4, 4, BYTE, (int)sp, BYTE, (int)sq);
}

// the activation of one sum (a pair of sums for SwiGLU), in float32. A NaN sum stays NaN, also
// under ReLU, where fmaxf would give zero: a weight block that held an infinity has the NaN scale.
template <int NB>
__device__ __forceinline__ float activate(float a, float b, int act) {
    if constexpr (NB == 2) return a * sigmoidf_(a) * b;
    return act == 1 ? a * sigmoidf_(a) : act == 2 ? (a <= 0.f ? 0.f : a) : a;
}

struct Args {
    const void* x;
    const uint8_t* xs;
    const uint8_t *w[2], *ws[2];
    const int32_t *offsets, *rows;
    int64_t T;
    int S, N, K, E, act;
    bf16_t* out;
};

// row of x of a slot; an index outside x, which no index build writes, reads its last row
__device__ __forceinline__ int64_t x_row(const Args& a, int slot) {
    const uint32_t r = a.rows ? (uint32_t)a.rows[slot] : (uint32_t)slot;
    return min((int64_t)r, a.T - 1);
}

// Whether a tile has anything to compute. Its rows end with the result's: offsets are a caller's
// data, and whatever they hold, no slot outside [0, S) and no weight outside w is touched.
__device__ __forceinline__ bool inside(const Args& a, SlotTile& t) {
    const uint32_t slot = (uint32_t)t.off + (uint32_t)t.m0;
    if ((t.off | t.m0) < 0 || slot >= (uint32_t)a.S || (uint32_t)t.n0 >= (uint32_t)a.N ||
        (uint32_t)t.e >= (uint32_t)a.E)
        return false;
    t.mrows = min(t.mrows, a.S - (int)slot);
    return t.mrows > 0;
}

// ---- stream core ------------------------------------------------------------------------
// A tile of up to 16 MT rows by BN columns of NB weights, in slices of 128 GROUPS values of
// K. WN waves take different columns, WK waves different blocks of a slice, whose sums are
// added through LDS at the end.
// Loads straight into registers in the layout of the matrix instructions, 16 rows a load
// and a scale byte with each, reached 3.3 TB/s: the address unit takes a cycle for every
// line that four neighbouring lanes touch. Copies into LDS with eight lanes to a line cut
// that to a quarter, and the scales come for CHUNK blocks of K at a time, 16 bytes a load
// (one token's gated product at K = 4096, N = 14336, two experts: 41 -> 24 us, of it 22.4 in
// the kernel with the same 125 MB of weights pass after pass, which the last-level cache
// holds; behind other layers' weights, from HBM, 25.2, 5.0 TB/s).
__device__ __constant__ uint4 g_zero16 = {0u, 0u, 0u, 0u};

template <int BM_, int BN_, int WN_, int WK_, int GROUPS_, int NB_, bool X4_, int NST_, int CHUNK_>
struct SCfg {
    static constexpr int BM = BM_, MT = (BM + 15) / 16, BN = BN_, WN = WN_, WK = WK_, NB = NB_, NST = NST_;
    static constexpr bool X4 = X4_;
    static constexpr int NW = WN * WK, THREADS = 64 * NW;
    static constexpr int NT = BN / 16 / WN;                  // column fragments of a wave
    static constexpr int GROUPS = GROUPS_, KS = 128 * GROUPS, BLOCKS = 4 * GROUPS;   // of a slice
    static constexpr int GPW = GROUPS / WK;                  // groups of four blocks of a wave
    static constexpr int XROW = X4 ? KS / 2 : KS * 2;
    static constexpr int WR = NB * BN, SR = WR + (X4 ? BM : 0);
    static constexpr int X_BYTES = BM * XROW, WROW = KS / 2, W_BYTES = WR * WROW;
    static constexpr int XCOPIES = (X_BYTES + 1023) / 1024, WCOPIES = W_BYTES / 1024;
    static constexpr int NCX = (XCOPIES + NW - 1) / NW, NCW = WCOPIES / NW;
    static constexpr int XSPACE = XCOPIES * 1024, STAGE = XSPACE + W_BYTES, PER = NCX + NCW;
    static constexpr int CHUNK = CHUNK_;                      // blocks whose scales LDS holds
    static constexpr int SPITCH = CHUNK + 4;
    static constexpr int PIECES = SR * (CHUNK / 16), NP = (PIECES + THREADS - 1) / THREADS;
    static constexpr int RING = NST * STAGE, LDS = RING + SR * SPITCH;
    static constexpr int PITCH = WR + 4;                     // floats of a row of partial sums
    static_assert(NT >= 1 && GPW >= 1 && WCOPIES % NW == 0 && LDS <= 160 * 1024, "tile");
    static_assert(BM == 16 * MT || (BM < 16 && 16 % BM == 0), "rows");
    static_assert(WK * 16 * MT * PITCH * 4 <= RING && PER * (NST - 2) < 64, "epilogue, wait count");
};

// 16 bytes from an address that need not be aligned
__device__ __forceinline__ uint4 ld16_any(const uint8_t* p) {
    uint4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}

template <class C>
__global__ void __launch_bounds__(C::THREADS)
mx_stream(const Args a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    SlotTile t;
    if (!find_slot_tile<C::THREADS>(reinterpret_cast<int*>(lds), a.offsets, a.E, C::BM,
                                    (a.N + C::BN - 1) / C::BN, blockIdx.x, C::BN, t) ||
        !inside(a, t))
        return;
    const int lane = threadIdx.x & 63, wv = wave_id();
    const int r16 = lane & 15, g = lane >> 4, wn = wv % C::WN, wk = wv / C::WN;
    const int nkb = a.K / mx::BLOCK, nk = (nkb + C::BLOCKS - 1) / C::BLOCKS;
    auto column = [&](int r) { return (int64_t)t.e * a.N + min(t.n0 + r % C::BN, a.N - 1); };   // of weight row r
    // this lane's sources: of place q of the x tile (rows of XROW bytes) and of the weights'
    const uint8_t *px[C::NCX], *pw[C::NCW];
    int bx[C::NCX], bw[C::NCW];   // block inside the slice
#pragma unroll
    for (int i = 0; i < C::NCX; ++i) {
        const int q = (wv + i * C::NW) % C::XCOPIES * 64 + lane;   // waves left over copy the same again
        constexpr int CPR = C::XROW / 16;
        const int r = q / CPR, c = (q % CPR & ~7) | ((q & 7) ^ (C::X4 ? (r >> 1) & 7 : r & 7));
        bx[i] = C::X4 ? c : c >> 2;
        px[i] = static_cast<const uint8_t*>(a.x) +
                x_row(a, t.off + t.m0 + min(r, t.mrows - 1)) * (C::X4 ? a.K / 2 : 2 * a.K) + c * 16;
    }
#pragma unroll
    for (int i = 0; i < C::NCW; ++i) {
        const int q = (wv + i * C::NW) * 64 + lane;
        constexpr int CPR = C::WROW / 16;
        const int r = q / CPR;
        bw[i] = (q % CPR & ~7) | ((q & 7) ^ ((r >> 1) & 7));
        pw[i] = a.w[C::NB == 2 ? r / C::BN : 0] + column(r) * (a.K / 2) + bw[i] * 16;
    }
    const uint32_t base = lds_offset(lds);
    auto issue = [&](int s, uint32_t dst) __attribute__((always_inline)) {
        const int left = nkb - s * C::BLOCKS;   // past K: zeros
#pragma unroll
        for (int i = 0; i < C::NCX; ++i) {
            const void* p = px[i] + (int64_t)s * C::XROW;
            dma16(bx[i] < left ? p : &g_zero16, dst + (wv + i * C::NW) % C::XCOPIES * 1024);
        }
#pragma unroll
        for (int i = 0; i < C::NCW; ++i) {
            const void* p = pw[i] + (int64_t)s * C::WROW;
            dma16(bw[i] < left ? p : &g_zero16, dst + C::XSPACE + (wv + i * C::NW) * 1024);
        }
    };
    // scales of chunk c: loaded 16 bytes a piece, then written to LDS; past K the byte of 1.0
    uint8_t* const sl = reinterpret_cast<uint8_t*>(lds) + C::RING;
    uint4 sc[C::NP];
    auto load_scales = [&](int chunk) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < C::NP; ++i) {
            const int p = threadIdx.x + i * C::THREADS, r = p / (C::CHUNK / 16);
            const int b0 = chunk * C::CHUNK + p % (C::CHUNK / 16) * 16, n = nkb - b0;
            if (p >= C::PIECES || n <= 0) continue;
            const uint8_t* src = r < C::WR ? a.ws[C::NB == 2 ? r / C::BN : 0] + column(r) * nkb
                                           : a.xs + x_row(a, t.off + t.m0 + min(r - C::WR, t.mrows - 1)) * nkb;
            src += b0;
            if (n >= 16) {
                sc[i] = ld16_any(src);
            } else {   // the row's end: nkb is even
                uint32_t v[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t lo = 4 * q < n ? src[4 * q] | (uint32_t)src[4 * q + 1] << 8 : 0x7f7fu;
                    const uint32_t hi = 4 * q + 2 < n ? src[4 * q + 2] | (uint32_t)src[4 * q + 3] << 8 : 0x7f7fu;
                    v[q] = lo | hi << 16;
                }
                sc[i] = make_uint4(v[0], v[1], v[2], v[3]);
            }
        }
    };
    auto store_scales = [&](int chunk) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < C::NP; ++i) {
            const int p = threadIdx.x + i * C::THREADS, r = p / (C::CHUNK / 16), c = p % (C::CHUNK / 16);
            if (p >= C::PIECES) continue;
            const bool in = nkb - (chunk * C::CHUNK + c * 16) > 0;
            uint32_t* d = reinterpret_cast<uint32_t*>(sl + r * C::SPITCH + c * 16);
            d[0] = in ? sc[i].x : 0x7f7f7f7fu; d[1] = in ? sc[i].y : 0x7f7f7f7fu;
            d[2] = in ? sc[i].z : 0x7f7f7f7fu; d[3] = in ? sc[i].w : 0x7f7f7f7fu;
        }
    };
    f32x4 acc[C::NB][C::MT][C::NT];
#pragma unroll
    for (int b = 0; b < C::NB; ++b)
#pragma unroll
        for (int i = 0; i < C::MT; ++i)
#pragma unroll
            for (int j = 0; j < C::NT; ++j) acc[b][i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    __syncthreads();                       // the tile lookup's words are free
    load_scales(0);
    for (int s = 0; s < C::NST - 1 && s < nk; ++s) issue(s, base + s * C::STAGE);
    store_scales(0);
    int cur = 0, nxt = C::NST - 1;
    for (int s = 0; s < nk; ++s) {
        constexpr int SPC = C::CHUNK / C::BLOCKS;   // slices a chunk of scales
        if (s % SPC == 0 && s) {
            load_scales(s / SPC);
            __syncthreads();
            store_scales(s / SPC);
        }
        if (s + C::NST - 2 < nk) wait_vmcnt<C::PER * (C::NST - 2)>();
        else wait_vmcnt<0>();
        lds_barrier();   // slice s is there for all waves, and slice s - 1 has been read by all
        if (s + C::NST - 1 < nk) issue(s + C::NST - 1, base + nxt * C::STAGE);
        const char* X = lds + cur * C::STAGE;
        const char* Wt = X + C::XSPACE;
#pragma unroll
        for (int u = 0; u < C::GPW; ++u) {
            const int kb = (wk + u * C::WK) * 4 + g;   // this lane's block of the slice
            const uint8_t* sk = sl + s % SPC * C::BLOCKS + kb;
            uint4 x[C::MT][C::X4 ? 1 : 4];
            uint32_t xs[C::MT];
#pragma unroll
            for (int i = 0; i < C::MT; ++i) {
                const int m = (i * 16 + r16) % C::BM;   // fragment rows past BM: any of the tile's
                if constexpr (C::X4) {
                    x[i][0] = ld16(X + m * C::XROW + (((kb & ~7) | ((kb & 7) ^ ((m >> 1) & 7))) << 4));
                    xs[i] = sk[(C::WR + m) * C::SPITCH];
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        x[i][q] = ld16(X + m * C::XROW + (kb >> 1) * 128 + ((((kb & 1) * 4 + q) ^ (m & 7)) << 4));
                }
            }
#pragma unroll
            for (int b = 0; b < C::NB; ++b)
#pragma unroll
                for (int j = 0; j < C::NT; ++j) {
                    const int n = b * C::BN + (wn * C::NT + j) * 16 + r16;
                    const uint4 w = ld16(Wt + n * C::WROW + (((kb & ~7) | ((kb & 7) ^ ((n >> 1) & 7))) << 4));
                    const uint32_t ws = sk[n * C::SPITCH];
                    if constexpr (C::X4) {
#pragma unroll
                        for (int i = 0; i < C::MT; ++i)
                            acc[b][i][j] = mfma_mx16(w, ws, x[i][0], xs[i], acc[b][i][j]);
                    } else {
                        const float f = mx::scale_value(ws);
                        const uint32_t c[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const bf16x8 v = __builtin_bit_cast(bf16x8, mx::decode8(c[q], f));
#pragma unroll
                            for (int i = 0; i < C::MT; ++i)
                                acc[b][i][j] = mfma16x16x32(v, __builtin_bit_cast(bf16x8, x[i][q]), acc[b][i][j]);
                        }
                    }
                }
        }
        cur = cur + 1 == C::NST ? 0 : cur + 1;
        nxt = nxt + 1 == C::NST ? 0 : nxt + 1;
    }
    __syncthreads();   // the ring is free
    // lane L holds row L % 16, columns 4 (L / 16) + 0..3 of every 16 x 16 fragment
    float* red = reinterpret_cast<float*>(lds);   // [WK][16 MT][PITCH]
#pragma unroll
    for (int b = 0; b < C::NB; ++b)
#pragma unroll
        for (int i = 0; i < C::MT; ++i)
#pragma unroll
            for (int j = 0; j < C::NT; ++j)
                *reinterpret_cast<f32x4*>(red + ((wk * C::MT + i) * 16 + r16) * C::PITCH + b * C::BN +
                                          (wn * C::NT + j) * 16 + g * 4) = acc[b][i][j];
    __syncthreads();
    for (int o = threadIdx.x; o < C::BM * C::BN / 4; o += C::THREADS) {
        const int m = o / (C::BN / 4), c = o % (C::BN / 4) * 4;
        if (m >= t.mrows || t.n0 + c >= a.N) continue;
        f32x4 v[C::NB];
#pragma unroll
        for (int b = 0; b < C::NB; ++b) {
            v[b] = *reinterpret_cast<const f32x4*>(red + m * C::PITCH + b * C::BN + c);
#pragma unroll
            for (int w = 1; w < C::WK; ++w)
                v[b] += *reinterpret_cast<const f32x4*>(red + (w * C::MT * 16 + m) * C::PITCH + b * C::BN + c);
        }
        float h[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) h[r] = activate<C::NB>(v[0][r], v[C::NB - 1][r], a.act);
        *reinterpret_cast<uint2*>(a.out + (int64_t)(t.off + t.m0 + m) * a.N + t.n0 + c) =
            make_uint2(pack_bf2(h[0], h[1]), pack_bf2(h[2], h[3]));
    }
}

// ---- tile core --------------------------------------------------------------------------
// Measured: 4-bit rows 4096 -> 14336 gated, eight experts, 3554 slots (444 rows each in tiles
// of 256) 287 to 291 us, 2.9 PFLOP/s; 16384 slots 1137, 3.38, where a loop of the scaled
// instruction alone reaches 7.0 on random values (9.6 on zeros: power bounds it). bfloat16 rows
// 2048 -> 1408 gated, 64 experts, 98304 slots 975 to 1030 us, 1.1 to 1.16 PFLOP/s;
// 8192 x 8192 x 8192 1.28, a loop of its instruction 1.8 (2.5). About 12 (8) us of a tile's
// time, its first copies and its results, run beside no matrix instruction: one workgroup a CU.
// BM x BN outputs of NB weights, WM x WN waves of 32 x 32 fragments. A slice is 64 values of
// K with bfloat16 rows (128-byte rows of x, 32-byte rows of codes), 256 with 4-bit rows
// (128-byte rows of either: whole lines take 40% fewer requests to L2 than slices of 128 do).
// Each 64 values are two blocks; lane half h = L / 32 takes block h of them, one 16-byte LDS
// read of codes, which four 32x32x16 bfloat16 or one 32x32x64 scaled instruction use up. With bfloat16 rows instruction q takes values 8q .. 8q + 7 of
// both blocks, so x comes as the chunks at bytes 64 h + 16 q of its row.
// Scales come for 512 values of K at a time, 16 bytes of each row as aligned dwords, four
// lanes to a row, into one of three buffers: a piece of chunk c + 1 goes out with each slice
// of chunk c, while slices of chunk c - 1 may still be read. (One 16-bit copy a lane for
// each two blocks, every lane in a row of its own, cost 14% with bfloat16 rows and 25% with
// 4-bit ones.) Where a row has an odd number of pairs of blocks, odd rows start in the
// middle of a dword: their chunks begin two bytes early. (The last dword of all may end two
// bytes behind the last scale of x; those bytes are not used.)

// 16-byte global -> LDS copy as dma16 (gemm.hpp), from a base of the whole wave's and a lane's
// offset
__device__ __forceinline__ void dma16_at(const void* base, uint32_t off, uint32_t lds_off) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                 ::"v"(off), "s"(base), "s"(lds_off) : "memory", "m0");
}
// 4-byte global -> LDS copy: lane l writes the dword at lds_off + 4 l
__device__ __forceinline__ void dma4(const void* g, uint32_t lds_off) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off"
                 ::"v"(g), "s"(lds_off) : "memory", "m0");
}

template <int BM_, int BN_, int WM_, int WN_, int NB_, bool X4_, int NST_>
struct TCfg {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NB = NB_, NST = NST_;
    static constexpr bool X4 = X4_;
    static constexpr int NW = WM * WN, THREADS = 64 * NW;
    static constexpr int WTM = BM / WM, WTN = BN / WN, FM = WTM / 32, FN = WTN / 32;
    static constexpr int KS = X4 ? 256 : 64;              // values of a slice
    static constexpr int KP = KS / 64;                    // pairs of blocks
    static constexpr int XROW = 128, WROW = KS / 2;
    static constexpr int X_BYTES = BM * XROW, W_BYTES = NB * BN * WROW;
    static constexpr int NCX = X_BYTES / 1024 / NW, NCW = W_BYTES / 1024 / NW;
    // scale rows: the weights' NB * BN, then (4-bit rows) x's BM; chunks of 16 bytes each
    static constexpr int SROWS = NB * BN + (X4 ? BM : 0), S_BYTES = SROWS * 16;
    static constexpr int SPC = 512 / KS;                       // slices of a chunk
    static constexpr int NCS = SROWS / 16 / NW;                // copies of a chunk, for each wave
    static constexpr int NCP = (NCS + SPC - 1) / SPC;          // ... that go out with a slice
    static constexpr int STAGE = X_BYTES + W_BYTES, RING = NST * STAGE;
    static constexpr int LDS = RING + 3 * S_BYTES;
    static constexpr int PER = NCX + NCW + NCP;
    static constexpr int AHEAD = X4 ? (PER + 2) / 3 : 0;       // copies of a slice that go out two slices ahead
    static_assert(SROWS % (16 * NW) == 0 && NST <= SPC + 1, "scale rows, buffers");
    static_assert(X_BYTES % (1024 * NW) == 0 && W_BYTES % (1024 * NW) == 0 && NCX >= 1 && NCW >= 1, "copies");
    static_assert(FM >= 1 && FN >= 1 && LDS <= 160 * 1024 && PER * (NST - 1) < 64, "tile");
};

// 16-byte chunk c of row r in an LDS tile of ROW-byte rows: 128 / ROW rows share a line of
// eight chunks, and a chunk's place in its line is XORed with half the line's number (two
// lines are the width of the banks), so that a fragment read, one chunk of 32 consecutive
// rows, spreads over all banks.
template <int ROW>
struct Place {
    static constexpr int CPR = ROW / 16, RPL = 8 / CPR;   // chunks a row, rows a line
    __device__ static __forceinline__ int swz(int line) { return (line >> 1) & (ROW == 128 ? 7 : ROW == 64 ? 3 : 1); }
    __device__ static __forceinline__ int byte(int r, int c) {
        const int line = r / RPL;
        return line * 128 + ((((r % RPL) * CPR + c) ^ swz(line)) << 4);
    }
    // row and chunk of the tile's 16-byte place q
    __device__ static __forceinline__ void at(int q, int& r, int& c) {
        const int line = q >> 3, p = (q & 7) ^ swz(line);
        r = line * RPL + p / CPR;
        c = p % CPR;
    }
};

// ODD (4-bit rows): rows have an odd number of pairs of blocks, K / 64.
template <class C, bool ODD>
__global__ void __launch_bounds__(C::THREADS)
mx_tile(const Args a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    SlotTile t;
    if (!find_slot_tile<C::THREADS>(reinterpret_cast<int*>(lds), a.offsets, a.E, C::BM,
                                    (a.N + C::BN - 1) / C::BN, blockIdx.x, C::BN, t, 4) ||
        !inside(a, t))
        return;
    const int lane = threadIdx.x & 63, wv = wave_id();
    const int wm = wv / C::WN, wn = wv % C::WN;
    const int nkb = a.K / mx::BLOCK, nk = (a.K + C::KS - 1) / C::KS;
    using PX = Place<C::XROW>;
    using PW = Place<C::WROW>;
    // this lane's sources, one for each copy
    const uint8_t *px[C::NCX], *ps[C::NCS];
    // four bits for each scale copy: this lane's dword of a chunk, and whether the row starts in
    // the middle of a dword. Dword d of row r lies in place d ^ (r / 8) % 4 of the row's four.
    int pd = 0;
    uint32_t ow[C::NCW];          // offsets into the expert's matrix (below 4 GB: N K < 2^33)
    const uint8_t* bw[C::NB];     // and its start, moved on with the slices
    auto chunk_x = [&](int i, int& r) { int c; PX::at((wv + i * C::NW) * 64 + lane, r, c); return c; };
    auto chunk_w = [&](int i, int& r) { int c; PW::at((wv + i * C::NW) * 64 + lane, r, c); return c; };
#pragma unroll
    for (int i = 0; i < C::NCX; ++i) {
        int r;
        const int c = chunk_x(i, r);
        const int64_t row = x_row(a, t.off + t.m0 + min(r, t.mrows - 1));
        px[i] = static_cast<const uint8_t*>(a.x) + row * (C::X4 ? a.K / 2 : 2 * a.K) + c * 16;
    }
    auto column = [&](int n) { return min(t.n0 + n % C::BN, a.N - 1); };   // of weight row n of the tile
#pragma unroll
    for (int b = 0; b < C::NB; ++b) bw[b] = a.w[b] + (int64_t)t.e * a.N * (a.K / 2);
#pragma unroll
    for (int i = 0; i < C::NCW; ++i) {
        int r;
        const int c = chunk_w(i, r);
        ow[i] = (uint32_t)column(r) * (uint32_t)(a.K / 2) + c * 16;
    }
    // the start of the weight that copy i of this wave belongs to
    auto weight = [&](int i) __attribute__((always_inline)) {
        if constexpr (C::NB == 1) return bw[0];
        else return (wv + i * C::NW) * 1024 >= C::BN * C::WROW ? bw[1] : bw[0];
    };
    const int half_pair = nkb & 2;   // rows start in the middle of a dword every other time
#pragma unroll
    for (int i = 0; i < C::NCS; ++i) {
        const int r = (wv * C::NCS + i) * 16 + (lane >> 2);
        const uint8_t* p;
        if (r < C::NB * C::BN) p = a.ws[C::NB == 2 ? r / C::BN : 0] + ((int64_t)t.e * a.N + column(r)) * nkb;
        else p = a.xs + x_row(a, t.off + t.m0 + min(r - C::NB * C::BN, t.mrows - 1)) * nkb;
        const int lead = (int)(reinterpret_cast<uintptr_t>(p) & 2), d = (lane ^ (r >> 3)) & 3;
        ps[i] = p - lead + d * 4;
        pd |= (lead * 2 | d) << (4 * i);
    }
    const uint32_t base = lds_offset(lds), sbase = base + C::RING;
    // copy i of this wave's of scale chunk c into the buffer at `dst` (past the row: its last
    // dword again; a select among array elements would go to memory, hence the sums)
    auto copy_scales = [&](int i, int c, uint32_t dst) __attribute__((always_inline)) {
        const uint8_t* p = ps[0];
#pragma unroll
        for (int q = 1; q < C::NCS; ++q) p += i == q ? ps[q] - ps[0] : 0;
        const int e = pd >> (4 * i);
        const int last = ((nkb + (e >> 1 & 2) - 1) & ~3) - 4 * (e & 3);   // dword of the row
        dma4(p + min(c * 16, last), dst + (wv * C::NCS + i) * 256);
    };
    int sbuf = 1;   // buffer of the chunk after the one that the slices being issued are in
    // Before the first copies of slice s of x's places [x0, x1) and, with W, of the weights: where
    // K cuts the slice short, chunk 0 stands in for the chunks behind K, which are not used; where
    // there is no such slice, the last one does. (4-bit rows; with bfloat16 ones slices are whole
    // and none is copied that does not exist.)
    auto edge = [&](int s, int x0, int x1, bool W) __attribute__((always_inline)) {
        const int left = nkb - s * (C::KS / 32);
        if (left >= C::KS / 32) return;
        int r, l = lane;
        asm volatile("" : "+v"(l));   // or the places below would be held in registers all along
#pragma unroll
        for (int i = 0; i < C::NCX; ++i) {
            if (i < x0 || i >= x1) continue;
            int c;
            PX::at((wv + i * C::NW) * 64 + l, r, c);
            px[i] -= left <= 0 ? C::XROW : c >= left ? c * 16 : 0;
        }
        if (!W) return;
        if (left <= 0)
#pragma unroll
            for (int b = 0; b < C::NB; ++b) bw[b] -= C::WROW;
        else
#pragma unroll
            for (int i = 0; i < C::NCW; ++i) {
                int c;
                PW::at((wv + i * C::NW) * 64 + l, r, c);
                ow[i] -= c >= left ? c * 16 : 0;
            }
    };
    // copy u of this wave's C::PER of slice s, slices in order
    auto issue = [&](int s, uint32_t dst, int u) __attribute__((always_inline)) {
        if (u < C::NCP) {
            copy_scales((s % C::SPC * C::NCP + u) * C::NCS / (C::SPC * C::NCP), s / C::SPC + 1, sbase + sbuf * C::S_BYTES);
            if (u == C::NCP - 1 && (s + 1) % C::SPC == 0) sbuf = sbuf == 2 ? 0 : sbuf + 1;
        } else if (u < C::NCP + C::NCX) {
            const int i = u - C::NCP;
            dma16(px[i], dst + (wv + i * C::NW) * 1024);
            px[i] += C::XROW;
        } else {
            const int i = u - C::NCP - C::NCX;
            dma16_at(weight(i), ow[i], dst + C::X_BYTES + (wv + i * C::NW) * 1024);
            if (u == C::PER - 1)
#pragma unroll
                for (int b = 0; b < C::NB; ++b) bw[b] += C::WROW;
        }
    };
    f32x16 acc[C::NB][C::FM][C::FN];
#pragma unroll
    for (int b = 0; b < C::NB; ++b)
#pragma unroll
        for (int i = 0; i < C::FM; ++i)
#pragma unroll
            for (int j = 0; j < C::FN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[b][i][j][r] = 0.f;
    __syncthreads();                       // the tile lookup's words are free
    __builtin_amdgcn_s_waitcnt(0x0F70);    // vmcnt(0): only copies are outstanding from here on
#pragma unroll
    for (int i = 0; i < C::NCS; ++i) copy_scales(i, 0, sbase);
    if constexpr (C::X4) edge(0, 0, C::NCX, true);
    for (int s = 0; s < C::NST - 1 && s < nk; ++s)
#pragma unroll
        for (int u = 0; u < C::PER; ++u) issue(s, base + s * C::STAGE, u);
    const int h = lane >> 5, l32 = lane & 31;
    // whether the scales of x's fragment rows start in the middle of a dword
    bool odd[C::X4 ? C::FM : 1] = {};
    if constexpr (C::X4)
#pragma unroll
        for (int i = 0; i < C::FM; ++i)
            odd[i] = half_pair && (x_row(a, t.off + t.m0 + min(wm * C::WTM + i * 32 + l32, t.mrows - 1)) & 1);
    int rbuf = 0;      // buffer of the scale chunk that the slice being read is in
    int cur = 0;       // ring position of the slice being read
    // LDS place of the scale of block h of pair s KP + k, for a row l32 of 32 whose first is
    // row 0 (others: 16 bytes a row further on); odd: of a row that starts in mid-dword, whose
    // last pair lies in the next chunk
    auto scale_at = [&](int s, int k, int odd) __attribute__((always_inline)) {
        const int q = s % C::SPC * C::KP + k + odd;
        const int b = q < 8 ? rbuf : rbuf == 2 ? 0 : rbuf + 1;
        return C::RING + b * C::S_BYTES + l32 * 16 + (((q & 7) >> 1 ^ ((l32 >> 3) & 3)) << 2) + (q & 1) * 2 + h;
    };
    auto byte = [&](int at) __attribute__((always_inline)) {
        return (uint32_t)*reinterpret_cast<const uint8_t*>(lds + at);
    };
    constexpr int NW = C::NB * C::FN, NM = NW * C::FM;   // weight fragments, matrix instructions a step
    // weight fragment f = b FN + j of pair k; columns of even number (e N and the tile's first
    // are) start on a dword
    auto read_w = [&](int s, int k, int f, uint4& w, uint32_t& sw) __attribute__((always_inline)) {
        const int n = f / C::FN * C::BN + f % C::FN * 32;
        w = ld16(lds + cur * C::STAGE + C::X_BYTES + PW::byte(wn * C::WTN + l32, 2 * k + h) + n * C::WROW);
        sw = byte(scale_at(s, k, half_pair ? l32 & 1 : 0) + wn * C::WTN * 16 + n * 16);
    };
    auto read_x = [&](int c, int i) __attribute__((always_inline)) {
        return ld16(lds + cur * C::STAGE + PX::byte(wm * C::WTM + l32, c) + i * 32 * C::XROW);
    };
    // A step is NM matrix instructions, each followed by its share of `n` other actions: the
    // fragment reads of the next step and the copies of a later slice. Both run beside the
    // matrix instructions then (with all of a slice's copies issued behind its barrier, every
    // wave at once, the matrix cores waited for some 400 of 2500 cycles a slice).
    auto step = [&](auto&& mma, int n, auto&& act) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < NM; ++t) {
            mma(t / (C::FM * C::FN), t / C::FN % C::FM, t % C::FN);
#pragma unroll
            for (int u = t * n / NM; u < (t + 1) * n / NM; ++u) act(u);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // between the last fragment reads of slice s and their use: every wave has read slice s,
    // whose place later copies take, and slice s + 1 is there for all
    auto next = [&](int s, auto MORE) __attribute__((always_inline)) {
        if constexpr (decltype(MORE)::value) wait_vmcnt<C::PER * (C::NST - 2)>();
        else wait_vmcnt<0>();
        lds_barrier();
        cur = cur + 1 == C::NST ? 0 : cur + 1;
        if ((s + 1) % C::SPC == 0) rbuf = rbuf == 2 ? 0 : rbuf + 1;
    };
    // copy u of slice s + NST - 1, into the place of slice s - 1
    auto copy = [&](int s, int u) __attribute__((always_inline)) {
        issue(s + C::NST - 1, base + (cur == 0 ? C::NST - 1 : cur - 1) * C::STAGE, u);
    };
    if (nk >= C::NST - 1) wait_vmcnt<C::PER * (C::NST - 2)>();
    else wait_vmcnt<0>();
    lds_barrier();
    if constexpr (C::X4) {
        constexpr int NR = NW + C::FM;
        struct Frag { uint4 w[NW], x[C::FM]; } f0, f1;        // of a slice's first and second pair
        // scales of a slice for this lane's half: bytes 0 and 2 of each fragment's word
        uint32_t sa[NR], sb[NR];
        const int swz = ((l32 >> 3) & 3) << 2;
        const int lw = (wn * C::WTN + l32) * 16 + swz, lx = (C::NB * C::BN + wm * C::WTM + l32) * 16 + swz;
        auto read = [&](int pos, int k, Frag& f, int u) __attribute__((always_inline)) {
            if (u < NW)
                f.w[u] = ld16(lds + pos * C::STAGE + C::X_BYTES + PW::byte(wn * C::WTN + l32, 2 * k + h) +
                              (u / C::FN * C::BN + u % C::FN * 32) * C::WROW);
            else
                f.x[u - NW] = ld16(lds + pos * C::STAGE + PX::byte(wm * C::WTM + l32, 2 * k + h) +
                                   (u - NW) * 32 * C::XROW);
        };
        // scales of fragment u of slice q of the chunk at r (the next chunk's at rn). Rows that
        // start in mid-dword: the upper half of this dword and the lower of the next.
        auto read_scale = [&](int r, int rn, int q, int u) __attribute__((always_inline)) {
            const int l = u < NW ? lw : lx;
            const int n = (u < NW ? u / C::FN * C::BN + u % C::FN * 32 : (u - NW) * 32) * 16;
            const char* p = lds + ((r + l) ^ (q << 2)) + n;
            if constexpr (!ODD) {
                return *reinterpret_cast<const uint32_t*>(p) >> (8 * h);
            } else {
                const bool mid = u < NW ? l32 & 1 : odd[u < NW ? 0 : u - NW];
                const char* pn = lds + (q == 3 ? rn + l : (r + l) ^ ((q + 1) << 2)) + n;
                const uint32_t lo = *reinterpret_cast<const uint16_t*>(mid ? p + 2 : p);
                const uint32_t hi = *reinterpret_cast<const uint16_t*>(mid ? pn : p + 2);
                return (lo | hi << 16) >> (8 * h);
            }
        };
        int r0 = C::RING, r1 = C::RING + C::S_BYTES, r2 = C::RING + 2 * C::S_BYTES;   // this chunk's scales, ...
        auto turn = [&] { const int r = r0; r0 = r1; r1 = r2; r2 = r; };
        auto mma = [&](const Frag& f, const uint32_t (&sc)[NR], auto BYTE) __attribute__((always_inline)) {
            return [&](int b, int i, int j) __attribute__((always_inline)) {
                acc[b][i][j] = mfma_mx32<decltype(BYTE)::value>(f.w[b * C::FN + j], sc[b * C::FN + j], f.x[i],
                                                                sc[NW + i], acc[b][i][j]);
            };
        };
        constexpr std::integral_constant<int, 0> LO{};
        constexpr std::integral_constant<int, 2> HI{};
        static_assert(C::NST == 2 && C::SPC == 2 && C::KP == 4, "ring places and scale words of a slice");
        int s = 0;
        constexpr int XA = C::AHEAD > C::NCP ? C::AHEAD - C::NCP : 0;   // copies of x among those two ahead
        static_assert(XA <= C::NCX, "copies ahead");
        // copy u of slice s + d (Q: of slice s, below)
        auto copy = [&](auto Q, int d, int u) __attribute__((always_inline)) {
            const int q = Q, place = d == 1 ? 1 - q : q;
            if (u < C::NCP) {
                copy_scales((place * C::NCP + u) * C::NCS / (2 * C::NCP), (s + d) / 2 + 1,
                            base + (d == 2 || q ? r2 : r1));
            } else if (u < C::NCP + C::NCX) {
                const int i = u - C::NCP;
                dma16(px[i], base + place * C::STAGE + (wv + i * C::NW) * 1024);
                px[i] += C::XROW;
            } else {
                const int i = u - C::NCP - C::NCX;
                dma16_at(weight(i), ow[i], base + place * C::STAGE + C::X_BYTES + (wv + i * C::NW) * 1024);
                if (u == C::PER - 1)
#pragma unroll
                    for (int b = 0; b < C::NB; ++b) bw[b] += C::WROW;
            }
        };
        // Slice s, number q = s % 2 of its scale chunk and in ring place q: four steps, the arrival
        // of slice s + 1 before the last. Its copies go out beside the first two and the step
        // behind the barrier before those: spread out, for a wave whose copy waits for the
        // address unit issues no matrix instructions either. A scale word holds
        // two pairs; words are read when those before them are used up. CUT: K may end inside the
        // slice, with codes of zero and scales of 1.0 behind it then.
        auto slice = [&](auto Q, auto CUT) __attribute__((always_inline)) {
            const int q = Q, t = 1 - q;
            constexpr bool CUTS = decltype(CUT)::value;
            auto cut = [&](int k, Frag& f, uint32_t (&sc)[NR]) __attribute__((always_inline)) {
                if constexpr (CUTS) {
                    const bool past = s * 8 + k * 2 >= nkb;
#pragma unroll
                    for (int u = 0; u < NW; ++u) f.w[u] = past ? zero16() : f.w[u];
#pragma unroll
                    for (int u = 0; u < NR; ++u) sc[u] = past ? 0x007f007fu : sc[u];
                }
            };
            // (the sums are pinned to this side of the branches, or their instructions would sink
            // behind them and spill)
#pragma unroll
            for (int u = 0; u < C::NB * C::FM * C::FN; ++u)
                asm volatile("" : "+v"(acc[u / (C::FM * C::FN)][u / C::FN % C::FM][u % C::FN]));
            edge(s + 1, XA, C::NCX, true);
            edge(s + 2, 0, XA, false);
            constexpr int P0 = C::AHEAD, P1 = P0 + (C::PER - P0 + 1) / 2;
            step(mma(f0, sa, LO), NR + P1 - P0, [&](int u) __attribute__((always_inline)) {
                if (u < NR) read(q, 1, f1, u);
                else copy(Q, 1, u - NR + P0);
            });
            cut(1, f1, sa);
            constexpr int P2 = C::PER - P1;
            step(mma(f1, sa, HI), 2 * NR + P2, [&](int u) __attribute__((always_inline)) {
                if (u < NR) read(q, 2, f0, u);
                else if (u < NR + P2) copy(Q, 1, u - NR + P1);
                else sb[u - NR - P2] = read_scale(r0, r1, 2 * q + 1, u - NR - P2);
            });
            cut(2, f0, sb);
            step(mma(f0, sb, LO), NR, [&](int u) __attribute__((always_inline)) { read(q, 3, f1, u); });
            cut(3, f1, sb);
            wait_vmcnt<0>();
            lds_barrier();   // all waves have read slice s, and slice s + 1 is there for all
            step(mma(f1, sb, HI), 2 * NR + P0, [&](int u) __attribute__((always_inline)) {
                if (u < NR) read(t, 0, f0, u);
                else if (u < 2 * NR) sa[u - NR] = read_scale(q ? r1 : r0, q ? r2 : r1, 2 * t, u - NR);
                else copy(Q, 2, u - 2 * NR);
            });
        };
#pragma unroll
        for (int u = 0; u < NR; ++u) {
            sa[u] = read_scale(r0, r1, 0, u);
            read(0, 0, f0, u);
        }
        constexpr std::integral_constant<int, 0> Q0{};
        constexpr std::integral_constant<int, 1> Q1{};
        edge(1, 0, XA, false);
#pragma unroll
        for (int u = 0; u < C::AHEAD; ++u) copy(Q0, 1, u);
        // Whole slices in pairs, then what is left: ring places are known at compile time (a loop
        // that finds them out slice by slice issues twice as many instructions beside the matrix
        // instructions, more than those hide).
        for (; (s + 2) * 8 <= nkb; turn()) {
            slice(Q0, std::false_type{});
            ++s;
            slice(Q1, std::false_type{});
            ++s;
        }
        if (s < nk) {
            slice(Q0, std::true_type{});
            if (++s < nk) slice(Q1, std::true_type{});
        }
        wait_vmcnt<0>();   // no copy may land behind the workgroup's end
    } else {
        constexpr std::true_type MORE{};
        constexpr std::false_type REST{};
        uint4 w[NW], wnext[NW], x0[C::FM], x1[C::FM];
        uint32_t snext[NW];
        float sc[NW];
        // instruction q of the slice: values 8 q .. 8 q + 7 of both blocks
        auto mma = [&](int q, const uint4 (&x)[C::FM]) __attribute__((always_inline)) {
            return [&, q](int b, int i, int j) __attribute__((always_inline)) {
                const uint4& v = w[b * C::FN + j];
                const uint32_t c = q == 0 ? v.x : q == 1 ? v.y : q == 2 ? v.z : v.w;
                acc[b][i][j] = mfma32x32x16(__builtin_bit_cast(bf16x8, mx::decode8(c, sc[b * C::FN + j])),
                                            __builtin_bit_cast(bf16x8, x[i]), acc[b][i][j]);
            };
        };
        auto read = [&](int s, int u) __attribute__((always_inline)) {   // of slice s: weights, first x
            if (u < NW) read_w(s, 0, u, wnext[u], snext[u]);
            else x0[u - NW] = read_x(4 * h, u - NW);
        };
        auto slice = [&](int s, auto more) __attribute__((always_inline)) {
#pragma unroll
            for (int f = 0; f < NW; ++f) {   // the weights read ahead come into use
                w[f] = wnext[f];
                sc[f] = mx::scale_value(snext[f]);
            }
            constexpr int P = decltype(more)::value ? C::PER : 0, P0 = P / 2;
            step(mma(0, x0), C::FM + P0, [&](int u) __attribute__((always_inline)) {
                if (u < C::FM) x1[u] = read_x(4 * h + 1, u);
                else copy(s, u - C::FM);
            });
            step(mma(1, x1), C::FM + P - P0, [&](int u) __attribute__((always_inline)) {
                if (u < C::FM) x0[u] = read_x(4 * h + 2, u);
                else copy(s, u - C::FM + P0);
            });
            step(mma(2, x0), C::FM, [&](int u) __attribute__((always_inline)) { x1[u] = read_x(4 * h + 3, u); });
            next(s, more);   // behind the last slice: reads that nothing uses
            step(mma(3, x1), NW + C::FM, [&](int u) __attribute__((always_inline)) { read(s + 1, u); });
        };
#pragma unroll
        for (int u = 0; u < NW + C::FM; ++u) read(0, u);
        int s = 0;
        for (; s + C::NST - 1 < nk; ++s) slice(s, MORE);
        for (; s < nk; ++s) slice(s, REST);
    }
    const WaveCoord<C> wc;
#pragma unroll
    for (int i = 0; i < C::FM; ++i) {
        const int m = wc.row(i);
        if (m >= t.mrows) continue;
        bf16_t* o = a.out + (int64_t)(t.off + t.m0 + m) * a.N + t.n0;
#pragma unroll
        for (int j = 0; j < C::FN; ++j) {
            float v[C::NB][2][8];
#pragma unroll
            for (int b = 0; b < C::NB; ++b) frag_cols8(acc[b][i][j], v[b]);
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const int c = wc.col8(j, p);
                if (t.n0 + c >= a.N) continue;
                float y[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) y[r] = activate<C::NB>(v[0][p][r], v[C::NB - 1][p][r], a.act);
                st16(o + c, pack8(y));
            }
        }
    }
}

// ---- launch -----------------------------------------------------------------------------
// the worst case of ceil(rows / BM) over the experts
int64_t row_tiles(int64_t S, int E, int BM) {
    const int64_t active = std::min<int64_t>(S, E);
    return active + (S - active) / BM;
}

template <class C>
hipError_t stream(const MxArgs& m, const Args& a, hipStream_t st) {
    const int64_t grid = row_tiles(m.S, m.E, C::BM) * ((m.N + C::BN - 1) / C::BN);
    static const hipError_t attr = hipFuncSetAttribute(
        reinterpret_cast<const void*>(&mx_stream<C>), hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS);
    if (attr != hipSuccess) return attr;
    if (grid > INT32_MAX / C::THREADS) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(mx_stream<C>, dim3((unsigned)grid), dim3(C::THREADS), C::LDS, st, a);
    probe::mark("mx_stream", st);
    return hipGetLastError();
}

template <class C>
hipError_t tile(const MxArgs& m, const Args& a, hipStream_t st) {
    const int64_t grid = row_tiles(m.S, m.E, C::BM) * ((m.N + C::BN - 1) / C::BN);
    if (grid > INT32_MAX / C::THREADS) return hipErrorInvalidConfiguration;
    auto go = [&](auto odd) {
        constexpr bool ODD = decltype(odd)::value;
        static const hipError_t attr = hipFuncSetAttribute(
            reinterpret_cast<const void*>(&mx_tile<C, ODD>), hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS);
        if (attr != hipSuccess) return attr;
        hipLaunchKernelGGL((mx_tile<C, ODD>), dim3((unsigned)grid), dim3(C::THREADS), C::LDS, st, a);
        probe::mark("mx_tile", st);
        return hipGetLastError();
    };
    if constexpr (C::X4)
        if (m.K / 64 % 2) return go(std::true_type{});
    return go(std::false_type{});
}

// Times in us, the alternatives on the same data.
template <bool X4, int NB>
hipError_t pick(const MxArgs& m, const Args& a, hipStream_t st) {
    // rows of an expert that has any, about, and workgroups of 64 columns
    const int64_t active = std::min<int64_t>(m.S, m.E);
    const double rows = (double)m.S / (double)active;
    const int64_t blocks = row_tiles(m.S, m.E, 16) * (m.N / 64);
    constexpr int BN = NB == 2 ? 128 : 256, NST = X4 ? 2 : 3;
    // Fewer workgroups than CUs, a row or so each (single tokens): 16 columns, and slices of
    // 1024 values, four waves deep. d = 14336 -> 4096, two experts: 13.9 against 22.8;
    // 2880 -> 2880 gated, four experts: 11.0, 12.2.
    if (m.S <= m.E && blocks < 256) return stream<SCfg<4, 16, 1, 4, 8, NB, X4, 2, 128>>(m, a, st);
    // The largest tile that the rows fill and that still gives two thirds of the CUs one: its
    // operands are used most often, but a workgroup takes as long on an idle chip as on a full
    // one (K = 4096, bfloat16 rows, one weight, tiles of 256, 128, 64 and 32 rows: 79, 49, 38, 16).
    // 256, 128, 64, 32 rows a tile, K -> N, E experts of so many rows:
    //                              bfloat16 rows: one weight,       gated         4-bit rows: one weight,         gated
    //   4096 -> 14336  8 x  32   168  108 68.1 46.5   360  239  154  110   60.3 46.3 42.8 44.1    143  115  104 97.5
    //                  8 x  64   177  116 78.5 80.9   368  247  165  178   68.8 55.2 48.7 52.6    140  119  114  124
    //                  8 x 128   200  132  143  158   390  258  270  318   80.3 66.4 91.3 97.2    152  136  174  199
    //                  8 x 512   422  465  524  628   754  918 1024 1223    174  215  330  360    292  400  626  685
    //   14336 -> 4096  8 x 128   265  222  156  158   349  254  273  309   91.3 76.4 67.4 94.5    127  121  163  215
    //                  8 x 256   298  238  257  300   373  470  505  586    118 94.5  143  177    148  191  289  385
    //   4096 -> 4096   2 x 128  79.1 49.7 38.8 16.0  75.7 50.3 37.3 23.4   28.4 18.2 14.5 10.6   25.8 21.9 17.8 15.0
    //                  2 x 256  79.8 50.4 39.4 23.9  77.2 50.9 41.4 43.2   28.9 18.8 15.2 14.5   28.3 22.2 19.6 27.4
    //                  2 x 1024 83.4 66.3 73.5 90.7   108  126  139  174   32.9 27.5 38.9 43.8   39.3 48.9 73.2 81.0
    //   2880 -> 2880   4 x 512  60.4 41.8 45.6 51.5  62.8 80.3 76.0  102   29.0 22.0 31.3 32.1   30.2 41.3 48.1 60.2
    //   2048 -> 1408   64 x 48  89.1 59.7 36.1 37.7   135 90.0 58.0 66.1   37.6 30.6 25.3 22.6   52.7 41.5 37.4 38.4
    //                  64 x 96  93.6 61.7 57.8 54.6   141 94.6  100 99.8   41.8 31.6 34.6 31.1   55.8 44.9 60.7 52.2
    //                  64 x 192  101  103 89.5  106   161  195  160  211   46.5 48.1 55.1 56.4   65.0 82.5 90.8 96.1
    // The rule takes the fastest of these, or one within 5% of it, in 47 of the 52; in the others
    // it loses 8 to 17% (2 x 128 rows, 4-bit gated: 17.6 of 64 rows against 15.0 of 32). The host
    // knows the experts' mean alone, and under a skewed routing no expert may have it: gated
    // products of 16 to 8192 tokens by four layers' shapes, experts drawn by a Zipf law of 1.2,
    // lose more than 6% in 5 of 40 cases, the most in 2048 -> 1408, bfloat16, 1777 tokens of 64
    // experts (mean 167, largest 1632): 204 of 256 rows against 158 of 64.
    auto fills = [&](int bm, int bn) {
        return (double)active * std::ceil(rows / bm) * ((m.N + bn - 1) / bn) * 3.0 >= 2.0 * 256.0;
    };
    if (rows > 128 && fills(256, BN)) return tile<TCfg<256, BN, 2, 4, NB, X4, NST>>(m, a, st);
    if (rows > 64 && fills(128, BN)) return tile<TCfg<128, BN, 2, 4, NB, X4, NST>>(m, a, st);
    // With 4-bit rows half as many columns, twice the workgroups, where 64 rows: 4096 -> 14336,
    // 8 x 48 rows 48.4, 57.0; 2048 -> 1408 gated, 64 x 48 rows 37.7, 43.7. bfloat16 rows, for
    // which four waves side by side convert the weights once each: 93.4, 79.7; 63.6, 60.2.
    constexpr int BN64 = X4 ? BN / 2 : BN;
    if (rows > 32 && fills(64, BN64)) {
        if constexpr (X4) return tile<TCfg<64, BN64, 2, 2, NB, X4, NST>>(m, a, st);
        else return tile<TCfg<64, BN64, 1, 4, NB, X4, NST>>(m, a, st);
    }
    // 16 and 32 rows a tile: 9.4 rows an expert (2880 -> 2880) 276, 287; 24 rows (4096 ->
    // 14336 gated) 145, 105
    if (rows > 12) {
        if constexpr (NB == 2) return stream<SCfg<32, 64, 2, 2, 2, NB, X4, 2, 64>>(m, a, st);
        else return stream<SCfg<32, 128, 4, 2, 2, NB, X4, 2, 64>>(m, a, st);
    }
    // A long K on few workgroups is bound by the steps of each one's loop: 16 waves, 512
    // values a step. 14336 -> 4096, 8 experts, 32 tokens: 47.9, 56.2; the other way round
    // with many workgroups (2880 -> 2880, 300 tokens, 128 experts): 150.8, 137.2.
    if constexpr (NB == 1)
        if (m.K >= 4096 && blocks <= 1024) return stream<SCfg<16, 64, 4, 4, 4, NB, X4, 2, 128>>(m, a, st);
    // bfloat16 rows cost LDS and L2 as much as the weights of 64 columns do: 192 columns, two
    // workgroups a CU, where they fill their rounds over the chip as well as 64 columns, four
    // workgroups a CU, do. 9 rows an expert, 128 x 2880 -> 2880 (3.75 rounds of 4; 5.6 of 6) 128.5,
    // 136.3; 64 x 2048 -> 1408 (1 of 1; 1.4 of 2) 20.2, 24.3; 64 x 1408 -> 2048 (1.4 of 2; 2 of 2)
    // 30.3, 26.0. With 4-bit rows no faster: 124.1, 124.5; 19.6, 20.1; 29.5, 25.8.
    if constexpr (NB == 1 && !X4) {
        auto rounds = [&](int bn, int wgs) {
            return (double)active * std::ceil(rows / 16) * ((m.N + bn - 1) / bn) / wgs;
        };
        const double wide = rounds(192, 512), narrow = rounds(64, 1024);
        if (wide >= 1 && wide / std::ceil(wide) >= narrow / std::ceil(narrow))
            return stream<SCfg<16, 192, 4, 2, 2, NB, X4, 2, 64>>(m, a, st);
    }
    return stream<SCfg<16, 64, 2, 2, 2, NB, X4, 2, 64>>(m, a, st);
}

}  // namespace

hipError_t mx_gemm(const MxArgs& m, hipStream_t st) {
    const Args a{m.x, m.xs, {m.w, m.w3}, {m.ws, m.ws3}, m.offsets, m.rows, m.T, (int)m.S, m.N, m.K, m.E,
                 m.act, static_cast<bf16_t*>(m.out)};
    if (m.xs) return m.w3 ? pick<true, 2>(m, a, st) : pick<true, 1>(m, a, st);
    return m.w3 ? pick<false, 2>(m, a, st) : pick<false, 1>(m, a, st);
}

}  // namespace moe
