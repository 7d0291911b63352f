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
// or L % 32 of block L / 32 (32x32x64), and that block's scale byte in the low byte of its
// scale register; results as for the bfloat16 instructions (all checked on the device).
__device__ __forceinline__ f32x4 mfma_mx16(const uint4& p, uint32_t sp, const uint4& q, uint32_t sq, const f32x4& c) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fp4_operand(p), fp4_operand(q), c, 4, 4, 0, (int)sp, 0, (int)sq);
}
__device__ __forceinline__ f32x16 mfma_mx32(const uint4& p, uint32_t sp, const uint4& q, uint32_t sq, const f32x16& c) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fp4_operand(p), fp4_operand(q), c, 4, 4, 0, (int)sp, 0, (int)sq);
}

// the activation of one sum (a pair of sums for SwiGLU), in float32
template <int NB>
__device__ __forceinline__ float activate(float a, float b, int act) {
    if constexpr (NB == 2) return a * sigmoidf_(a) * b;
    return act == 1 ? a * sigmoidf_(a) : act == 2 ? fmaxf(a, 0.f) : a;
}

struct Args {
    const void* x;
    const uint8_t* xs;
    const uint8_t *w[2], *ws[2];
    const int32_t *offsets, *rows;
    int64_t T;
    int N, K, E, act;
    bf16_t* out;
};

// row of x of a slot; an index outside x, which no index build writes, reads its last row
__device__ __forceinline__ int64_t x_row(const Args& a, int slot) {
    const uint32_t r = a.rows ? (uint32_t)a.rows[slot] : (uint32_t)slot;
    return min((int64_t)r, a.T - 1);
}

// ---- stream core ------------------------------------------------------------------------
// A tile of up to 16 MT rows by BN columns of NB weights, in slices of 128 GROUPS values of
// K. WN waves take different columns, WK waves different blocks of a slice, whose sums are
// added through LDS at the end.
// Loads straight into registers in the layout of the matrix instructions, 16 rows a load
// and a scale byte with each, reached 3.3 TB/s: the address unit takes a cycle for every
// line that four neighbouring lanes touch. Copies into LDS with eight lanes to a line cut
// that to a quarter, and the scales come for CHUNK blocks of K at a time, 16 bytes a load:
// 5.2 TB/s (one token's gated product at K = 4096, N = 14336, two experts: 41 -> 24 us).
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
                                    (a.N + C::BN - 1) / C::BN, blockIdx.x, C::BN, t))
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
// BM x BN outputs of NB weights, WM x WN waves of 32 x 32 fragments. A slice is 64 values of
// K with bfloat16 rows (128-byte rows of x, 32-byte rows of codes), 128 with 4-bit rows
// (64-byte rows of either). Each 64 values are two blocks; lane half h = L / 32 takes block h
// of them, one 16-byte LDS read of codes, which four 32x32x16 bfloat16 or one 32x32x64
// scaled instruction use up. With bfloat16 rows instruction q takes values 8q .. 8q + 7 of
// both blocks, so x comes as the chunks at bytes 64 h + 16 q of its row.
// Scales come for 512 values of K at a time, 16 bytes of each row as aligned dwords, four
// lanes to a row, into one of three buffers: a piece of chunk c + 1 goes out with each slice
// of chunk c, while slices of chunk c - 1 may still be read. (One 16-bit copy a lane for
// each two blocks, every lane in a row of its own, cost 14% with bfloat16 rows and 25% with
// 4-bit ones.) Where a row has an odd number of pairs of blocks, odd rows start in the
// middle of a dword: their chunks begin two bytes early, and `odd` is added to the pair.

// 4-byte and 2-byte global -> LDS copies: lane l writes the dword at lds_off + 4 l
__device__ __forceinline__ void dma4(const void* g, uint32_t lds_off) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off"
                 ::"v"(g), "s"(lds_off) : "memory", "m0");
}
__device__ __forceinline__ void dma2(const void* g, uint32_t lds_off) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_ushort %0, off"
                 ::"v"(g), "s"(lds_off) : "memory", "m0");
}

template <int BM_, int BN_, int WM_, int WN_, int NB_, bool X4_, int NST_>
struct TCfg {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NB = NB_, NST = NST_;
    static constexpr bool X4 = X4_;
    static constexpr int NW = WM * WN, THREADS = 64 * NW;
    static constexpr int WTM = BM / WM, WTN = BN / WN, FM = WTM / 32, FN = WTN / 32;
    static constexpr int KS = X4 ? 128 : 64;              // values of a slice
    static constexpr int KP = KS / 64;                    // pairs of blocks
    static constexpr int XROW = X4 ? 64 : 128, WROW = KS / 2;
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
    static_assert(SROWS % (16 * NW) == 0, "scale rows");
    static_assert(X_BYTES % (1024 * NW) == 0 && W_BYTES % (1024 * NW) == 0 && NCX >= 1 && NCW >= 1, "copies");
    static_assert(FM >= 1 && FN >= 1 && LDS <= 160 * 1024 && PER * (NST - 2) < 64, "tile");
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

template <class C>
__global__ void __launch_bounds__(C::THREADS)
mx_tile(const Args a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    SlotTile t;
    if (!find_slot_tile<C::THREADS>(reinterpret_cast<int*>(lds), a.offsets, a.E, C::BM,
                                    (a.N + C::BN - 1) / C::BN, blockIdx.x, C::BN, t, 4))
        return;
    const int lane = threadIdx.x & 63, wv = wave_id();
    const int wm = wv / C::WN, wn = wv % C::WN;
    const int nkb = a.K / mx::BLOCK, nk = (a.K + C::KS - 1) / C::KS;
    using PX = Place<C::XROW>;
    using PW = Place<C::WROW>;
    // this lane's sources, one for each copy
    const uint8_t *px[C::NCX], *pw[C::NCW], *ps[C::NCS];
    int smax[C::NCS];             // last dword of the scale row that this lane copies of
    int cx[C::NCX], cw[C::NCW];   // chunk inside the slice
#pragma unroll
    for (int i = 0; i < C::NCX; ++i) {
        int r;
        PX::at((wv + i * C::NW) * 64 + lane, r, cx[i]);
        const int64_t row = x_row(a, t.off + t.m0 + min(r, t.mrows - 1));
        px[i] = static_cast<const uint8_t*>(a.x) + row * (C::X4 ? a.K / 2 : 2 * a.K) + cx[i] * 16;
    }
    auto column = [&](int n) {   // of tile column n over the NB weights, clamped
        return (int64_t)t.e * a.N + min(t.n0 + n % C::BN, a.N - 1);
    };
#pragma unroll
    for (int i = 0; i < C::NCW; ++i) {
        int r;
        PW::at((wv + i * C::NW) * 64 + lane, r, cw[i]);
        pw[i] = a.w[C::NB == 2 ? r / C::BN : 0] + column(r) * (a.K / 2) + cw[i] * 16;
    }
    const int half_pair = nkb & 2;   // rows start in the middle of a dword every other time
#pragma unroll
    for (int i = 0; i < C::NCS; ++i) {
        const int r = (wv * C::NCS + i) * 16 + (lane >> 2);
        const uint8_t* p;
        if (r < C::NB * C::BN) p = a.ws[C::NB == 2 ? r / C::BN : 0] + column(r) * nkb;
        else p = a.xs + x_row(a, t.off + t.m0 + min(r - C::NB * C::BN, t.mrows - 1)) * nkb;
        const int lead = (int)(reinterpret_cast<uintptr_t>(p) & 2);
        ps[i] = p - lead;
        smax[i] = (nkb + lead - 1) & ~3;
    }
    const uint8_t* const xs_end = C::X4 ? a.xs + a.T * nkb : nullptr;
    const uint32_t base = lds_offset(lds);
    // all of this wave's copies of slice s; with 4-bit rows the last slice may be half a slice
    const uint32_t sbase = base + C::RING;
    // copy i of this wave's of scale chunk c (past the row: its last dword again)
    auto issue_scales = [&](int i, int c, int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < C::NCS; ++q) {
            if (q != i) continue;
            const uint8_t* p = ps[q] + min(c * 16 + (lane & 3) * 4, smax[q]);
            const uint32_t dst = sbase + buf * C::S_BYTES + (wv * C::NCS + q) * 256;
            // an odd number of pairs in all of x's rows: the last dword is half outside
            if (C::X4 && p + 4 == xs_end + 2) dma2(p, dst);
            else dma4(p, dst);
        }
    };
    int sbuf = 1;   // buffer of the chunk after the one that the slices being issued are in
    auto issue = [&](int s, uint32_t dst) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < C::NCP; ++u)
            issue_scales((s % C::SPC * C::NCP + u) * C::NCS / (C::SPC * C::NCP), s / C::SPC + 1, sbuf);
        if ((s + 1) % C::SPC == 0) sbuf = sbuf == 2 ? 0 : sbuf + 1;
        const bool cut = C::KP == 2 && s * 4 + 4 > nkb;
#pragma unroll
        for (int i = 0; i < C::NCX; ++i) {
            const void* p = px[i] + (int64_t)s * C::XROW;
            if (cut && cx[i] >= 2) p = &g_zero16;
            dma16(p, dst + (wv + i * C::NW) * 1024);
        }
#pragma unroll
        for (int i = 0; i < C::NCW; ++i) {
            const void* p = pw[i] + (int64_t)s * C::WROW;
            if (cut && cw[i] >= 2) p = &g_zero16;
            dma16(p, dst + C::X_BYTES + (wv + i * C::NW) * 1024);
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
    for (int i = 0; i < C::NCS; ++i) issue_scales(i, 0, 0);
    for (int s = 0; s < C::NST - 1 && s < nk; ++s) issue(s, base + s * C::STAGE);
    const int h = lane >> 5, l32 = lane & 31;
    // 1 for the fragment rows whose scales start in the middle of a dword (e N is even)
    int wodd[C::FN], xodd[C::X4 ? C::FM : 1];
#pragma unroll
    for (int j = 0; j < C::FN; ++j)
        wodd[j] = half_pair ? min(t.n0 + wn * C::WTN + j * 32 + l32, a.N - 1) & 1 : 0;
    if constexpr (C::X4)
#pragma unroll
        for (int i = 0; i < C::FM; ++i)
            xodd[i] = half_pair ? (int)(x_row(a, t.off + t.m0 + min(wm * C::WTM + i * 32 + l32, t.mrows - 1)) & 1) : 0;
    int rbuf = 0;   // buffer of the chunk that slice s is in
    int cur = 0, nxt = C::NST - 1;
    for (int s = 0; s < nk; ++s) {
        if (s + C::NST - 2 < nk) wait_vmcnt<C::PER * (C::NST - 2)>();
        else wait_vmcnt<0>();
        lds_barrier();   // slice s is there for all waves, and slice s - 1 has been read by all
        if (s + C::NST - 1 < nk) issue(s + C::NST - 1, base + nxt * C::STAGE);
        const char* X = lds + cur * C::STAGE;
        const char* Wt = X + C::X_BYTES;
        // the scale byte of this lane's block of pair s KP + k, row r; past K, where the codes
        // are zeros and LDS may hold the next row's scales (a NaN's), that of 1.0
        auto scale = [&](int r, int k, int odd) __attribute__((always_inline)) {
            if (C::KP == 2 && k == 1 && s * 4 + 4 > nkb) return 127u;
            const int q = s % C::SPC * C::KP + k + odd;       // pair inside the chunk; 8: in the next
            const int b = q < 8 ? rbuf : rbuf == 2 ? 0 : rbuf + 1;
            return (uint32_t)*reinterpret_cast<const uint8_t*>(lds + C::RING + b * C::S_BYTES + r * 16 + (q & 7) * 2 + h);
        };
#pragma unroll
        for (int k = 0; k < C::KP; ++k) {
            uint4 w[C::NB][C::FN];
            uint32_t sw[C::NB][C::FN];
#pragma unroll
            for (int b = 0; b < C::NB; ++b)
#pragma unroll
                for (int j = 0; j < C::FN; ++j) {
                    const int n = b * C::BN + wn * C::WTN + j * 32 + l32;
                    w[b][j] = ld16(Wt + PW::byte(n, 2 * k + h));
                    sw[b][j] = scale(n, k, wodd[j]);
                }
            if constexpr (C::X4) {
                uint4 xf[C::FM];
                uint32_t sx[C::FM];
#pragma unroll
                for (int i = 0; i < C::FM; ++i) {
                    const int m = wm * C::WTM + i * 32 + l32;
                    xf[i] = ld16(X + PX::byte(m, 2 * k + h));
                    sx[i] = scale(C::NB * C::BN + m, k, xodd[i]);
                }
#pragma unroll
                for (int b = 0; b < C::NB; ++b)
#pragma unroll
                    for (int i = 0; i < C::FM; ++i)
#pragma unroll
                        for (int j = 0; j < C::FN; ++j)
                            acc[b][i][j] = mfma_mx32(w[b][j], sw[b][j], xf[i], sx[i], acc[b][i][j]);
            } else {
                float sc[C::NB][C::FN];
#pragma unroll
                for (int b = 0; b < C::NB; ++b)
#pragma unroll
                    for (int j = 0; j < C::FN; ++j) sc[b][j] = mx::scale_value(sw[b][j]);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    bf16x8 xf[C::FM];
#pragma unroll
                    for (int i = 0; i < C::FM; ++i)
                        xf[i] = __builtin_bit_cast(bf16x8, ld16(X + PX::byte(wm * C::WTM + i * 32 + l32, 4 * h + q)));
#pragma unroll
                    for (int b = 0; b < C::NB; ++b)
#pragma unroll
                        for (int j = 0; j < C::FN; ++j) {
                            const uint32_t c = q == 0 ? w[b][j].x : q == 1 ? w[b][j].y : q == 2 ? w[b][j].z : w[b][j].w;
                            const bf16x8 wf = __builtin_bit_cast(bf16x8, mx::decode8(c, sc[b][j]));
#pragma unroll
                            for (int i = 0; i < C::FM; ++i)
                                acc[b][i][j] = mfma32x32x16(wf, xf[i], acc[b][i][j]);
                        }
                }
            }
        }
        cur = cur + 1 == C::NST ? 0 : cur + 1;
        nxt = nxt + 1 == C::NST ? 0 : nxt + 1;
        if ((s + 1) % C::SPC == 0) rbuf = rbuf == 2 ? 0 : rbuf + 1;
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
    static const hipError_t attr = hipFuncSetAttribute(
        reinterpret_cast<const void*>(&mx_tile<C>), hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS);
    if (attr != hipSuccess) return attr;
    if (grid > INT32_MAX / C::THREADS) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(mx_tile<C>, dim3((unsigned)grid), dim3(C::THREADS), C::LDS, st, a);
    probe::mark("mx_tile", st);
    return hipGetLastError();
}

// Times in us, bfloat16 rows, the alternatives on the same data.
template <bool X4, int NB>
hipError_t pick(const MxArgs& m, const Args& a, hipStream_t st) {
    // rows of an expert that has any, about, and workgroups of 64 columns
    const double rows = (double)m.S / (double)std::min<int64_t>(m.S, m.E);
    const int64_t blocks = row_tiles(m.S, m.E, 16) * (m.N / 64);
    constexpr int BN = NB == 2 ? 128 : 256;
    constexpr int NST = X4 ? 4 : 3;
    // Fewer workgroups than CUs, a row or so each (single tokens): 16 columns, and slices of
    // 1024 values, four waves deep. d = 14336 -> 4096, two experts: 13.9 against 22.8;
    // 2880 -> 2880 gated, four experts: 11.0, 12.2.
    if (m.S <= m.E && blocks < 256) return stream<SCfg<4, 16, 1, 4, 8, NB, X4, 2, 128>>(m, a, st);
    if (rows <= 12) {
        // A long K on few workgroups is bound by the steps of each one's loop: 16 waves, 512
        // values a step. 14336 -> 4096, 8 experts, 32 tokens: 47.9, 56.2; the other way round
        // with many workgroups (2880 -> 2880, 300 tokens, 128 experts): 150.8, 137.2.
        if constexpr (NB == 1)
            if (m.K >= 4096 && blocks <= 1024) return stream<SCfg<16, 64, 4, 4, 4, NB, X4, 2, 128>>(m, a, st);
        return stream<SCfg<16, 64, 2, 2, 2, NB, X4, 2, 64>>(m, a, st);
    }
    // 16 and 32 rows a tile: 9.4 rows an expert (2880 -> 2880) 276, 287; 24 rows (4096 ->
    // 14336 gated) 144, 111
    if (rows <= 24) {
        if constexpr (NB == 2) return stream<SCfg<32, 64, 2, 2, 2, NB, X4, 2, 64>>(m, a, st);
        else return stream<SCfg<32, 128, 4, 2, 2, NB, X4, 2, 64>>(m, a, st);
    }
    if (rows <= 64) return tile<TCfg<64, BN, 1, 4, NB, X4, 3>>(m, a, st);
    if (rows <= 128) return tile<TCfg<128, BN, 2, 4, NB, X4, NST>>(m, a, st);
    return tile<TCfg<256, BN, 2, 4, NB, X4, NST>>(m, a, st);
}

}  // namespace

hipError_t mx_gemm(const MxArgs& m, hipStream_t st) {
    const Args a{m.x, m.xs, {m.w, m.w3}, {m.ws, m.ws3}, m.offsets, m.rows, m.T, m.N, m.K, m.E, m.act,
                 static_cast<bf16_t*>(m.out)};
    if (m.xs) return m.w3 ? pick<true, 2>(m, a, st) : pick<true, 1>(m, a, st);
    return m.w3 ? pick<false, 2>(m, a, st) : pick<false, 1>(m, a, st);
}

}  // namespace moe
