// mx_gemm.hip -- products grouped by expert over weights in microscaled 4 bits (mx.hpp).
//
// out[s] = act(x[row(s)] w[e]^T), for SwiGLU SiLU(x w^T) * (x w3^T), for the slots s of
// each expert e; x in bfloat16, or in microscaled 4 bits too. Two cores:
//  * stream (few rows per expert, 16 or 32 a tile): bound by reading the weights once,
//    17/32 of a byte each. Weights go from HBM straight into registers, a lane holding
//    whole blocks of 32 with their one scale; the waves of a workgroup take the same
//    columns and different parts of K, and add their sums through LDS at the end.
//  * tiles (more rows): bound by the matrix cores. Both operands come by direct-to-LDS
//    copies into a ring of slices. The weights stay 4-bit in LDS, a quarter of bfloat16's
//    LDS traffic, and are converted as fragments.
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
// A tile of MT * 16 rows by NT * 16 columns of NB weights; W waves split K, 128 values (four
// blocks, one for each 16 lanes) at a time. A step's loads are issued one step ahead.
template <int MT_, int NT_, int NB_, bool X4_, int W_>
struct SCfg {
    static constexpr int MT = MT_, NT = NT_, NB = NB_, W = W_;
    static constexpr bool X4 = X4_;
    static constexpr int BM = 16 * MT, BN = 16 * NT, THREADS = 64 * W;
    static constexpr int PITCH = NB * BN + 4;   // floats of a row of partial sums
};

template <class C>
struct Step {
    uint4 w[C::NB][C::NT];
    uint32_t ws[C::NB][C::NT];
    uint4 x[C::MT][C::X4 ? 1 : 4];
    uint32_t xs[C::X4 ? C::MT : 1];
};

template <class C>
__global__ void __launch_bounds__(C::THREADS)
mx_stream(const Args a) {
    __shared__ int sh[8];
    __shared__ float red[C::W][C::BM][C::PITCH];
    SlotTile t;
    if (!find_slot_tile<C::THREADS>(sh, a.offsets, a.E, C::BM, a.N / C::BN, blockIdx.x, C::BN, t)) return;
    const int lane = threadIdx.x & 63, wv = wave_id();
    const int r16 = lane & 15, g = lane >> 4;
    const int nkb = a.K / mx::BLOCK, steps = (nkb + 3) / 4;
    const int64_t col0 = (int64_t)t.e * a.N + t.n0;
    const uint8_t *wp[C::NB], *sp[C::NB];
#pragma unroll
    for (int b = 0; b < C::NB; ++b) {
        wp[b] = a.w[b] + col0 * (a.K / 2);
        sp[b] = a.ws[b] + col0 * nkb;
    }
    const uint8_t *xp[C::MT], *xsp[C::MT];
#pragma unroll
    for (int i = 0; i < C::MT; ++i) {
        const int64_t row = x_row(a, t.off + t.m0 + min(i * 16 + r16, t.mrows - 1));
        xp[i] = static_cast<const uint8_t*>(a.x) + row * (C::X4 ? a.K / 2 : 2 * a.K);
        if constexpr (C::X4) xsp[i] = a.xs + row * nkb;
    }
    auto load = [&](Step<C>& s, int step) __attribute__((always_inline)) {
        const int kb = step * 4 + g;
        const bool in = kb < nkb;
        const int k = in ? kb : nkb - 1;    // past K: rows of zeros
#pragma unroll
        for (int b = 0; b < C::NB; ++b)
#pragma unroll
            for (int j = 0; j < C::NT; ++j) {
                const uint32_t row = j * 16 + r16;
                s.w[b][j] = ld16(wp[b] + (row * (uint32_t)(a.K / 2) + k * 16));
                s.ws[b][j] = sp[b][row * (uint32_t)nkb + k];
            }
#pragma unroll
        for (int i = 0; i < C::MT; ++i) {
            if constexpr (C::X4) {
                s.x[i][0] = ld16(xp[i] + k * 16);
                s.xs[i] = xsp[i][k];
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q) s.x[i][q] = ld16(xp[i] + k * 64 + q * 16);
            }
        }
        if (!in) {
#pragma unroll
            for (int b = 0; b < C::NB; ++b)
#pragma unroll
                for (int j = 0; j < C::NT; ++j) s.ws[b][j] = 127u;
#pragma unroll
            for (int i = 0; i < C::MT; ++i) {
#pragma unroll
                for (int q = 0; q < (C::X4 ? 1 : 4); ++q) s.x[i][q] = zero16();
                if constexpr (C::X4) s.xs[i] = 127u;
            }
        }
    };
    f32x4 acc[C::NB][C::MT][C::NT];
#pragma unroll
    for (int b = 0; b < C::NB; ++b)
#pragma unroll
        for (int i = 0; i < C::MT; ++i)
#pragma unroll
            for (int j = 0; j < C::NT; ++j) acc[b][i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto compute = [&](const Step<C>& s) __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < C::NB; ++b)
#pragma unroll
            for (int j = 0; j < C::NT; ++j) {
                if constexpr (C::X4) {
#pragma unroll
                    for (int i = 0; i < C::MT; ++i)
                        acc[b][i][j] = mfma_mx16(s.w[b][j], s.ws[b][j], s.x[i][0], s.xs[i], acc[b][i][j]);
                } else {
                    const float sc = mx::scale_value(s.ws[b][j]);
                    const uint32_t c[4] = {s.w[b][j].x, s.w[b][j].y, s.w[b][j].z, s.w[b][j].w};
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const bf16x8 f = __builtin_bit_cast(bf16x8, mx::decode8(c[q], sc));
#pragma unroll
                        for (int i = 0; i < C::MT; ++i)
                            acc[b][i][j] = mfma16x16x32(f, __builtin_bit_cast(bf16x8, s.x[i][q]), acc[b][i][j]);
                    }
                }
            }
    };
    if (wv < steps) {
        Step<C> s0, s1;
        load(s0, wv);
        for (int st = wv; st < steps; st += 2 * C::W) {
            const bool more = st + C::W < steps;
            if (more) load(s1, st + C::W);
            compute(s0);
            if (!more) break;
            if (st + 2 * C::W < steps) load(s0, st + 2 * C::W);
            compute(s1);
        }
    }
    // lane L holds row L % 16, columns 4 (L / 16) + 0..3 of every 16 x 16 fragment
#pragma unroll
    for (int b = 0; b < C::NB; ++b)
#pragma unroll
        for (int i = 0; i < C::MT; ++i)
#pragma unroll
            for (int j = 0; j < C::NT; ++j)
                *reinterpret_cast<f32x4*>(&red[wv][i * 16 + r16][b * C::BN + j * 16 + g * 4]) = acc[b][i][j];
    __syncthreads();
    for (int o = threadIdx.x; o < C::BM * C::BN / 4; o += C::THREADS) {
        const int m = o / (C::BN / 4), c = o % (C::BN / 4) * 4;
        if (m >= t.mrows) continue;
        f32x4 v[C::NB];
#pragma unroll
        for (int b = 0; b < C::NB; ++b) {
            v[b] = *reinterpret_cast<const f32x4*>(&red[0][m][b * C::BN + c]);
#pragma unroll
            for (int w = 1; w < C::W; ++w) v[b] += *reinterpret_cast<const f32x4*>(&red[w][m][b * C::BN + c]);
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
// The scale bytes of two blocks are one 16-bit copy, which leaves a zero-extended dword.
__device__ __constant__ uint4 g_zero16 = {0u, 0u, 0u, 0u};

// 2-byte global -> LDS copy: lane l writes the dword at lds_off + 4 l
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
    // scale rows: the weights' NB * BN, then (4-bit rows) x's BM; one dword each and pair
    static constexpr int SROWS = NB * BN + (X4 ? BM : 0);
    static constexpr int NCS = (SROWS + THREADS - 1) / THREADS;   // copies per wave and pair
    static constexpr int S_BYTES = KP * NCS * THREADS * 4;
    static constexpr int STAGE = X_BYTES + W_BYTES + S_BYTES;
    static constexpr int LDS = NST * STAGE;
    static constexpr int PER = NCX + NCW + KP * NCS;
    static_assert(X_BYTES % (1024 * NW) == 0 && W_BYTES % (1024 * NW) == 0 && NCX >= 1 && NCW >= 1, "copies");
    static_assert(FM >= 1 && FN >= 1 && LDS <= 160 * 1024 && PER * (NST - 2) < 64, "tile");
};

// 16-byte chunk c of row r in an LDS tile of ROW-byte rows: 128 / ROW rows share a line of
// eight chunks, and the chunk's place in its line is XORed with the line's number, so that
// the rows of a fragment read (one chunk of 32 consecutive rows) spread over the banks.
template <int ROW>
struct Place {
    static constexpr int CPR = ROW / 16, RPL = 8 / CPR;   // chunks a row, rows a line
    __device__ static __forceinline__ int swz(int line) { return ROW == 128 ? (line >> 1) & 7 : ROW == 64 ? line & 3 : line & 1; }
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
#pragma unroll
    for (int i = 0; i < C::NCS; ++i) {
        const int r = (i * C::NW + wv) * 64 + lane;
        if (r < C::NB * C::BN || !C::X4) {
            const int n = r % (C::NB * C::BN);
            ps[i] = a.ws[C::NB == 2 ? n / C::BN : 0] + column(n) * nkb;
        } else {
            const int m = min(r - C::NB * C::BN, t.mrows - 1);
            ps[i] = a.xs + x_row(a, t.off + t.m0 + m) * nkb;
        }
    }
    const uint32_t base = lds_offset(lds);
    // all of this wave's copies of slice s; with 4-bit rows the last slice may be half a slice
    auto issue = [&](int s, uint32_t dst) __attribute__((always_inline)) {
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
#pragma unroll
        for (int k = 0; k < C::KP; ++k)
#pragma unroll
            for (int i = 0; i < C::NCS; ++i)   // past K: the row's last scales, over codes of zero
                dma2(ps[i] + 2 * min(s * C::KP + k, nkb / 2 - 1),
                     dst + C::X_BYTES + C::W_BYTES + (k * C::NCS + i) * C::THREADS * 4 + wv * 256);
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
    for (int s = 0; s < C::NST - 1 && s < nk; ++s) issue(s, base + s * C::STAGE);
    const int h = lane >> 5, l32 = lane & 31;
    int cur = 0, nxt = C::NST - 1;
    for (int s = 0; s < nk; ++s) {
        if (s + C::NST - 2 < nk) wait_vmcnt<C::PER * (C::NST - 2)>();
        else wait_vmcnt<0>();
        lds_barrier();   // slice s is there for all waves, and slice s - 1 has been read by all
        if (s + C::NST - 1 < nk) issue(s + C::NST - 1, base + nxt * C::STAGE);
        const char* X = lds + cur * C::STAGE;
        const char* Wt = X + C::X_BYTES;
        const uint32_t* Sc = reinterpret_cast<const uint32_t*>(Wt + C::W_BYTES);
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
                    sw[b][j] = (Sc[k * C::NCS * C::THREADS + n] >> (8 * h)) & 255u;
                }
            if constexpr (C::X4) {
                uint4 xf[C::FM];
                uint32_t sx[C::FM];
#pragma unroll
                for (int i = 0; i < C::FM; ++i) {
                    const int m = wm * C::WTM + i * 32 + l32;
                    xf[i] = ld16(X + PX::byte(m, 2 * k + h));
                    sx[i] = Sc[k * C::NCS * C::THREADS + C::NB * C::BN + m] >> (8 * h);
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
    const int64_t grid = row_tiles(m.S, m.E, C::BM) * (m.N / C::BN);
    if (grid > INT32_MAX / C::THREADS) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(mx_stream<C>, dim3((unsigned)grid), dim3(C::THREADS), 0, st, a);
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

template <bool X4, int NB>
hipError_t pick(const MxArgs& m, const Args& a, hipStream_t st) {
    // rows of an expert that has any, about
    const double rows = (double)m.S / (double)std::min<int64_t>(m.S, m.E);
    constexpr int BN = NB == 2 ? 128 : 256;
    constexpr int NST = X4 ? 4 : 3;
    if (rows <= 12) return stream<SCfg<1, 4, NB, X4, 4>>(m, a, st);
    if (rows <= 24) return stream<SCfg<2, 4, NB, X4, 4>>(m, a, st);
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
