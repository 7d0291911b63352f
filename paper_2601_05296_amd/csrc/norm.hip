// norm.hip -- the norms of a residual block around the MoE layer, fused with the
// block's gate, its residual scale and the residual addition.
//
// Forward, per row of d elements (res: residual stream, y: block output):
//   p = y * rstd_post * w_post,  rstd_post = 1 / sqrt(mean(y^2) + eps)   (or p = y)
//   r = res_scale * res + gate * p
//   n = r * rstd_pre * w_pre,    rstd_pre = 1 / sqrt(mean(r^2) + eps)    (the next block's input)
// Backward, with rhat = r * rstd_pre, yhat = y * rstd_post:
//   G      = dr + rstd_pre * (w_pre dn - rhat * m),   m = mean(w_pre dn rhat)
//   dres   = res_scale * G,      dw_pre = sum_t dn rhat
//   dgate  = G p (summed over rows or columns),  dw_post = sum_t gate G yhat
//   dy     = rstd_post * (c G - yhat * mean(c G yhat)),  c = w_post gate
// Both move each tensor once: the row lives in registers between its loads and its
// stores, all arithmetic is float32, and outputs are rounded once.
#include "common.hpp"
#include "launch.hpp"
#include "probe.hpp"

namespace moe {
namespace {

enum : int { GATE_NONE = 0, GATE_CHANNEL = 1, GATE_TOKEN = 2, GATE_FULL = 3 };

// 16 bytes of elements as floats and back
template <bool F32>
struct Vec {
    static constexpr int N = F32 ? 4 : 8;
    static __device__ __forceinline__ void get(const uint4& v, float (&o)[N]) {
        if constexpr (F32) {
            o[0] = __uint_as_float(v.x); o[1] = __uint_as_float(v.y);
            o[2] = __uint_as_float(v.z); o[3] = __uint_as_float(v.w);
        } else {
            unpack8(v, o);
        }
    }
    static __device__ __forceinline__ uint4 put(const float (&o)[N]) {
        if constexpr (F32)
            return make_uint4(__float_as_uint(o[0]), __float_as_uint(o[1]), __float_as_uint(o[2]),
                              __float_as_uint(o[3]));
        else
            return pack8(o);
    }
    // one element as it lies in memory, and as a float: converting it where it is loaded would
    // wait for it, and with it for all loads of a row ahead
    static __device__ __forceinline__ uint32_t raw(const void* p, int64_t i) {
        if constexpr (F32) return static_cast<const uint32_t*>(p)[i];
        else return static_cast<const uint16_t*>(p)[i];
    }
    static __device__ __forceinline__ float one(uint32_t raw) { return __uint_as_float(F32 ? raw : raw << 16); }
};

// A row is held by WPR waves, NV vectors a lane: lane l of the row's wave w holds
// the vectors (i * WPR + w) * 64 + l. RPB rows per workgroup at a time.
template <bool F32_, int WPR_, int NV_, int RPB_>
struct Shape {
    static constexpr bool F32 = F32_;
    static constexpr int WPR = WPR_, NV = NV_, RPB = RPB_;
    static constexpr int THREADS = 64 * WPR * RPB;
    static constexpr int EPV = Vec<F32>::N;
};

// Sums over the waves of each row, the same in all of its lanes and always added in the
// same order. LDS is used alternately in two halves, so that one barrier per call does.
template <class S, int NS>
struct RowSum {
    float* lds;   // [2][RPB][WPR][NS]
    int half = 0;
    __device__ explicit RowSum(float* p) : lds(p) {}
    __device__ __forceinline__ void operator()(float (&v)[NS]) {
#pragma unroll
        for (int i = 0; i < NS; ++i) v[i] = wave_sum(v[i]);
        if constexpr (S::WPR > 1) {
            const int wv = threadIdx.x / 64, grp = wv / S::WPR, w = wv % S::WPR;
            float* p = lds + (half * S::RPB + grp) * S::WPR * NS;
            half ^= 1;
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int i = 0; i < NS; ++i) p[w * NS + i] = v[i];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NS; ++i) v[i] = 0.f;
#pragma unroll
            for (int j = 0; j < S::WPR; ++j)
#pragma unroll
                for (int i = 0; i < NS; ++i) v[i] += p[j * NS + i];
        }
    }
};

struct FwdArgs {
    const void *res, *y, *gate, *w_post, *w_pre;
    void *r, *n;
    float *rstd_post, *rstd_pre;
    float res_scale, eps;
    int64_t T;
    int d, kind;
};

// Bound by HBM: res, y in, r, n out, 5.2 to 5.4 TB/s (32768 x 4096 bfloat16 197 to 206 us, a
// copy's rate). The gate's kind is a template argument: as one of the launch it took 16383 x
// 2880 from 70-77 us to 85-99.
// Workgroups walk over the rows with the weights in registers and the next row's loads
// issued before the present row's sums. r may take the place of res (or y), and n that
// of y: a row's stores follow its loads, and no other workgroup touches the row.
template <class S, int KIND>
__global__ void __launch_bounds__(S::THREADS)
norm_fwd_kernel(const FwdArgs a) {
    using V = Vec<S::F32>;
    constexpr int NV = S::NV, EPV = S::EPV;
    __shared__ float lds[2 * S::RPB * S::WPR];
    RowSum<S, 1> sum(lds);
    const int wv = threadIdx.x / 64, grp = wv / S::WPR;
    const int c0 = (wv % S::WPR) * 64 + (threadIdx.x & 63);
    const int nvec = a.d / EPV;
    const bool block = a.y != nullptr, post = a.w_post != nullptr, pre = a.w_pre != nullptr;
    constexpr bool full = KIND == GATE_FULL;
    const float inv_d = 1.0f / (float)a.d;
    auto vec = [&](const void* p, int64_t row, int i) {
        return static_cast<const uint4*>(p) + row * nvec + c0 + i * S::WPR * 64;
    };
    auto in = [&](int i) { return c0 + i * S::WPR * 64 < nvec; };
    uint4 wpo[NV], wpr[NV], gc[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (!in(i)) continue;
        if (post) wpo[i] = *vec(a.w_post, 0, i);
        if (pre) wpr[i] = *vec(a.w_pre, 0, i);
        if (KIND == GATE_CHANNEL) gc[i] = *vec(a.gate, 0, i);
    }
    uint4 y[NV], x[NV], g[NV];
    uint32_t gt = 0;
    auto load = [&](int64_t t) {
        if (t >= a.T) return;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (!in(i)) continue;
            x[i] = *vec(a.res, t, i);
            if (block) y[i] = *vec(a.y, t, i);
            if (full) g[i] = *vec(a.gate, t, i);
        }
        if (KIND == GATE_TOKEN) gt = V::raw(a.gate, t);
    };
    const int64_t step = (int64_t)gridDim.x * S::RPB;
    load((int64_t)blockIdx.x * S::RPB + grp);
    for (int64_t t0 = (int64_t)blockIdx.x * S::RPB; t0 < a.T; t0 += step) {
        const int64_t t = t0 + grp;
        const bool row = t < a.T;
        float p[NV][EPV], r[NV][EPV];
        float s[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (in(i) && row) {
                V::get(x[i], r[i]);
                if (block) V::get(y[i], p[i]);
            }
            if (!(in(i) && row))
#pragma unroll
                for (int e = 0; e < EPV; ++e) r[i][e] = p[i][e] = 0.f;
        }
        float gv[NV][EPV];
        if (full)
#pragma unroll
            for (int i = 0; i < NV; ++i) V::get(g[i], gv[i]);
        const float gtok = V::one(gt);
        load(t + step);
        if (post) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < EPV; ++e) s[0] = fmaf(p[i][e], p[i][e], s[0]);
            sum(s);
            const float rs = rsqrtf(s[0] * inv_d + a.eps);
            if (row && a.rstd_post && c0 == 0) a.rstd_post[t] = rs;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float w[EPV];
                V::get(wpo[i], w);
#pragma unroll
                for (int e = 0; e < EPV; ++e) p[i][e] *= rs * w[e];
            }
        }
        if (block) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (KIND == GATE_CHANNEL) V::get(gc[i], gv[i]);
#pragma unroll
                for (int e = 0; e < EPV; ++e) {
                    const float ge = KIND == GATE_NONE ? 1.0f : KIND == GATE_TOKEN ? gtok : gv[i][e];
                    r[i][e] = fmaf(a.res_scale, r[i][e], ge * p[i][e]);
                }
                if (in(i) && row) *const_cast<uint4*>(vec(a.r, t, i)) = V::put(r[i]);
            }
        }
        if (pre) {
            s[0] = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (in(i))
#pragma unroll
                    for (int e = 0; e < EPV; ++e) s[0] = fmaf(r[i][e], r[i][e], s[0]);
            sum(s);
            const float rs = rsqrtf(s[0] * inv_d + a.eps);
            if (row && a.rstd_pre && c0 == 0) a.rstd_pre[t] = rs;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (!(in(i) && row)) continue;
                float w[EPV];
                V::get(wpr[i], w);
#pragma unroll
                for (int e = 0; e < EPV; ++e) w[e] *= r[i][e] * rs;
                *const_cast<uint4*>(vec(a.n, t, i)) = V::put(w);
            }
        }
    }
}

struct BwdArgs {
    const void *dr, *dn, *y, *r, *gate, *w_post, *w_pre;
    const float *rstd_post, *rstd_pre;
    void *dres, *dy, *dgate;
    float* part;   // [gridDim][3][d]: dw_pre, dw_post, dgate (channel)
    float res_scale;
    int64_t T;
    int d, kind;
};

// The row sums of G's own projection and of dy's are taken in one pass: with q = c yhat,
//   sum(c G yhat) = sum(q (dr + rstd_pre w_pre dn)) - rstd_pre m sum(q rhat),
// so a row takes one exchange between its waves instead of two. Column sums stay in
// registers over all of a workgroup's rows; the workgroups' sums are added in
// norm_bwd_sum, always in the same order. (The difference of two float32 sums is off by a few
// half steps of either, where summing differences is off by as many of theirs: against 64
// bits float32 gradients 1021 x 2880 1.4e-7, a sum of differences 1.2e-7.)
// Bound by HBM: dr, dn, y, r in, dres, dy out, 5.5 TB/s (16383 x 4096 bfloat16 147 us, 5 of
// them the sums' launch; a copy reaches 4.7 to 5.2, half of its bytes being writes, here a
// third). The gate's kind is a template argument: one kernel for all kinds spilled (184 us). Row
// groups that share a workgroup add their sums in LDS first: 60000 x 512 84 to 73 us.
template <class S, int KIND>
__global__ void __launch_bounds__(S::THREADS)
norm_bwd_kernel(const BwdArgs a) {
    using V = Vec<S::F32>;
    constexpr int NV = S::NV, EPV = S::EPV;
    constexpr int NS = 3;
    __shared__ float lds[2 * S::RPB * S::WPR * NS];
    RowSum<S, NS> sum(lds);
    const int wv = threadIdx.x / 64, grp = wv / S::WPR;
    const int c0 = (wv % S::WPR) * 64 + (threadIdx.x & 63);
    const int nvec = a.d / EPV;
    const bool post = a.w_post != nullptr, pre = a.w_pre != nullptr;
    const bool block = a.dy != nullptr, need_y = block && (post || KIND != GATE_NONE);
    const bool has_dr = a.dr != nullptr;
    constexpr bool full = KIND == GATE_FULL;
    const float inv_d = 1.0f / (float)a.d;
    auto vec = [&](const void* p, int64_t row, int i) {
        return static_cast<const uint4*>(p) + row * nvec + c0 + i * S::WPR * 64;
    };
    auto in = [&](int i) { return c0 + i * S::WPR * 64 < nvec; };
    uint4 wpo[NV], wpr[NV], gc[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        wpo[i] = wpr[i] = gc[i] = zero16();
        if (!in(i)) continue;
        if (post) wpo[i] = *vec(a.w_post, 0, i);
        if (pre) wpr[i] = *vec(a.w_pre, 0, i);
        if (KIND == GATE_CHANNEL) gc[i] = *vec(a.gate, 0, i);
    }
    float awpr[NV][EPV] = {}, awpo[NV][EPV] = {}, agc[NV][EPV] = {};
    uint4 ldr[NV], ldn[NV], lr[NV], ly[NV], lg[NV];
    float rpo = 1.f, rpr = 0.f;
    uint32_t gt = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) ldr[i] = ldn[i] = lr[i] = ly[i] = lg[i] = zero16();
    auto load = [&](int64_t t) {
        if (t >= a.T) return;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (!in(i)) continue;
            if (has_dr) ldr[i] = *vec(a.dr, t, i);
            if (pre) { ldn[i] = *vec(a.dn, t, i); lr[i] = *vec(a.r, t, i); }
            if (need_y) ly[i] = *vec(a.y, t, i);
            if (full) lg[i] = *vec(a.gate, t, i);
        }
        if (post) rpo = a.rstd_post[t];
        if (pre) rpr = a.rstd_pre[t];
        if (KIND == GATE_TOKEN) gt = V::raw(a.gate, t);
    };
    const int64_t step = (int64_t)gridDim.x * S::RPB;
    // four vectors of everything twice would not fit the registers (8192 float32, channel gate:
    // 8192 rows: 474 us with spills, 345 without a row ahead)
    constexpr bool AHEAD = NV < 4;
    if (AHEAD) load((int64_t)blockIdx.x * S::RPB + grp);
    for (int64_t t0 = (int64_t)blockIdx.x * S::RPB; t0 < a.T; t0 += step) {
        const int64_t t = t0 + grp;
        const bool row = t < a.T;
        if (!AHEAD) load(t);
        uint4 cdr[NV], cdn[NV], cr[NV], cy[NV], cg[NV];
        const float rp = rpr, ro = rpo, gtok = KIND == GATE_TOKEN ? V::one(gt) : 1.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            cdr[i] = ldr[i]; cdn[i] = ldn[i]; cr[i] = lr[i]; cy[i] = ly[i];
            cg[i] = full ? lg[i] : gc[i];
        }
        if (AHEAD) load(t + step);
        auto gate = [&](int i, float (&g)[EPV]) {
            if (KIND == GATE_CHANNEL || full) V::get(cg[i], g);
            else
#pragma unroll
                for (int e = 0; e < EPV; ++e) g[e] = gtok;   // 1 without a gate
        };
        float s[NS] = {0.f, 0.f, 0.f};
        if (row)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float vdr[EPV], vdn[EPV], vr[EPV], vy[EPV], g[EPV], wo[EPV], wr[EPV];
                V::get(cdr[i], vdr); V::get(cdn[i], vdn); V::get(cr[i], vr); V::get(cy[i], vy);
                gate(i, g); V::get(wpo[i], wo); V::get(wpr[i], wr);
#pragma unroll
                for (int e = 0; e < EPV; ++e) {
                    const float rhat = vr[e] * rp, wdn = wr[e] * vdn[e];
                    awpr[i][e] = fmaf(vdn[e], rhat, awpr[i][e]);
                    const float u = fmaf(rp, wdn, vdr[e]);
                    const float pn = post ? wo[e] * (vy[e] * ro) : vy[e];   // p
                    s[0] = fmaf(wdn, rhat, s[0]);
                    const float q = KIND == GATE_TOKEN ? pn : g[e] * pn;
                    s[1] = fmaf(q, u, s[1]);
                    s[2] = fmaf(q, rhat, s[2]);
                }
            }
        sum(s);
        if (!row) continue;
        const float m = s[0] * inv_d;
        // sum(p G) for a token's gate, which may be zero and comes in afterwards, else sum(gate p G)
        const float pG = s[1] - rp * m * s[2];
        const float m2 = (KIND == GATE_TOKEN ? gtok * pG : pG) * inv_d;
        if (KIND == GATE_TOKEN && c0 == 0) static_cast<float*>(a.dgate)[t] = pG;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (!in(i)) continue;
            float vdr[EPV], vdn[EPV], vr[EPV], vy[EPV], g[EPV], wo[EPV], wr[EPV], o[EPV], dg[EPV];
            V::get(cdr[i], vdr); V::get(cdn[i], vdn); V::get(cr[i], vr); V::get(cy[i], vy);
            gate(i, g); V::get(wpo[i], wo); V::get(wpr[i], wr);
            float G[EPV];
#pragma unroll
            for (int e = 0; e < EPV; ++e) {
                const float rhat = vr[e] * rp;
                G[e] = vdr[e] + rp * (wr[e] * vdn[e] - rhat * m);
                o[e] = a.res_scale * G[e];
            }
            *const_cast<uint4*>(vec(a.dres, t, i)) = V::put(o);
            if (!block) continue;
#pragma unroll
            for (int e = 0; e < EPV; ++e) {
                const float yhat = vy[e] * ro;
                const float gG = g[e] * G[e];
                if (post) {
                    awpo[i][e] = fmaf(gG, yhat, awpo[i][e]);
                    dg[e] = G[e] * (wo[e] * yhat);
                    o[e] = ro * (wo[e] * gG - yhat * m2);
                } else {
                    dg[e] = G[e] * vy[e];
                    o[e] = gG;
                }
                agc[i][e] += dg[e];
            }
            *const_cast<uint4*>(vec(a.dy, t, i)) = V::put(o);
            if (full) *const_cast<uint4*>(vec(a.dgate, t, i)) = V::put(dg);
        }
    }
    // the workgroup's column sums, its row groups' added in order
    float* part = a.part + (int64_t)blockIdx.x * 3 * a.d;
    __shared__ f32x4 cols[S::RPB > 1 ? S::RPB : 1][S::RPB > 1 ? S::WPR * 64 * NV * EPV / 4 : 1];
    auto put = [&](const float (&acc)[NV][EPV], float* out) __attribute__((always_inline)) {
        if constexpr (S::RPB > 1) __syncthreads();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (!in(i)) continue;
            const int c = (c0 + i * S::WPR * 64) * EPV;
#pragma unroll
            for (int e = 0; e < EPV; e += 4) {
                const f32x4 v{acc[i][e], acc[i][e + 1], acc[i][e + 2], acc[i][e + 3]};
                if constexpr (S::RPB > 1) cols[grp][(c + e) / 4] = v;
                else *reinterpret_cast<f32x4*>(out + c + e) = v;
            }
        }
        if constexpr (S::RPB > 1) {
            __syncthreads();
            for (int c = threadIdx.x; c < a.d / 4; c += S::THREADS) {
                f32x4 v = cols[0][c];
#pragma unroll
                for (int g = 1; g < S::RPB; ++g) v += cols[g][c];
                *reinterpret_cast<f32x4*>(out + c * 4) = v;
            }
        }
    };
    if (pre) put(awpr, part);
    if (post) put(awpo, part + a.d);
    if constexpr (KIND == GATE_CHANNEL) put(agc, part + 2 * a.d);
}

// out[c] = sum over the P partial sums of column c: 32 lanes of four columns by 32
// slices of the partials, the slices' sums added in order. blockIdx.y picks the output.
constexpr int SUM_COLS = 32, SUM_SLICES = 32;
__global__ void __launch_bounds__(SUM_COLS * SUM_SLICES)
norm_bwd_sum(const float* __restrict__ part, int P, int d, float* dw_pre, float* dw_post, float* dgate) {
    float* out = blockIdx.y == 0 ? dw_pre : blockIdx.y == 1 ? dw_post : dgate;
    if (!out) return;
    __shared__ f32x4 lds[SUM_SLICES][SUM_COLS];
    const int lane = threadIdx.x % SUM_COLS, slice = threadIdx.x / SUM_COLS;
    const int c = (blockIdx.x * SUM_COLS + lane) * 4;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (c < d)
#pragma unroll 4
        for (int p = slice; p < P; p += SUM_SLICES)
            v += *reinterpret_cast<const f32x4*>(part + ((int64_t)p * 3 + blockIdx.y) * d + c);
    lds[slice][lane] = v;
    __syncthreads();
    if (slice || c >= d) return;
    for (int i = 1; i < SUM_SLICES; ++i) v += lds[i][lane];
    *reinterpret_cast<f32x4*>(out + c) = v;
}

// Rows are spread over the fewest workgroups that need the same number of passes. The forward
// allows 32 waves a CU (16383 x 4096, no gate: 102 us; 16 waves 119, 8 110).
int row_blocks(int64_t T, int rpb, int most) {
    const int64_t n = (T + rpb - 1) / rpb;
    if (n <= most) return (int)n;
    const int64_t passes = (n + most - 1) / most;
    return (int)((n + passes - 1) / passes);
}

// f(Shape) for rows of d elements. The backward holds three column sums a lane beside its
// rows, so it takes one vector a lane up to 512 of them, and six waves where those hold the
// row; the forward fewer waves of two. us, forward and backward, bfloat16, channel gate:
//   16383 x 4096   4 waves of 2: 99, 163   8 of 1: 107, 147
//   16383 x 2880   4 waves of 2: 77, 117   6 of 1:  -, 109   8 of 1: 83, 121
//   60000 x 1024   1 wave of 2:  97, 148   2 of 1: 97, 137
//   8192 x 8192    8 waves of 2: 96, 159   16 of 1: 98, 665 (spills)
template <bool F32, bool BWD, class F>
void with_shape(int d, F&& f) {
    const int nvec = d / Vec<F32>::N;
    if (nvec <= 64) f(Shape<F32, 1, 1, 4>{});
    else if (BWD && nvec <= 128) f(Shape<F32, 2, 1, 2>{});
    else if (nvec <= 128) f(Shape<F32, 1, 2, 4>{});
    else if (nvec <= 256) f(Shape<F32, 4, 1, 1>{});
    else if (BWD && nvec <= 384) f(Shape<F32, 6, 1, 1>{});
    else if (BWD && nvec <= 512) f(Shape<F32, 8, 1, 1>{});
    else if (nvec <= 512) f(Shape<F32, 4, 2, 1>{});
    else if (nvec <= 1024) f(Shape<F32, 8, 2, 1>{});
    else if constexpr (F32) f(Shape<F32, 8, 4, 1>{});   // d <= 8192
}

// Workgroups of the backward: 8 waves (or one workgroup of 6) a CU hold enough loads in flight,
// and each more would write another 3 d partial sums. 16383 x 4096 in workgroups of 4 waves,
// channel gate: 8 waves a CU 163 us, 12 178, 16 175; 16383 x 2880 in workgroups of 6: one a CU
// 109, two 116; 4 waves are too few, 60000 x 512: 8 73, 4 105.
template <class S>
int bwd_blocks(int64_t T) {
    constexpr int W = S::THREADS / 64;
    return row_blocks(T, S::RPB, 256 * (8 / W));   // the same on every CU
}

// partial sums of a column: one a workgroup
int bwd_parts(int64_t T, int d, bool f32) {
    int P = 0;
    auto count = [&](auto s) { P = bwd_blocks<decltype(s)>(T); };
    if (f32) with_shape<true, true>(d, count);
    else with_shape<false, true>(d, count);
    return P;
}

template <bool F32>
void launch_fwd(const FwdArgs& a, hipStream_t st) {
    with_shape<F32, false>(a.d, [&](auto s) {
        using S = decltype(s);
        const int grid = row_blocks(a.T, S::RPB, 256 * 32 / (S::THREADS / 64));
        const auto kernel = a.kind == GATE_NONE ? &norm_fwd_kernel<S, GATE_NONE> : a.kind == GATE_CHANNEL ? &norm_fwd_kernel<S, GATE_CHANNEL>
                          : a.kind == GATE_TOKEN ? &norm_fwd_kernel<S, GATE_TOKEN> : &norm_fwd_kernel<S, GATE_FULL>;
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(S::THREADS), 0, st, a);
    });
    probe::mark("norm_fwd", st);
}

template <bool F32>
void launch_bwd(const BwdArgs& a, hipStream_t st) {
    with_shape<F32, true>(a.d, [&](auto s) {
        using S = decltype(s);
        const auto kernel = a.kind == GATE_NONE ? &norm_bwd_kernel<S, GATE_NONE> : a.kind == GATE_CHANNEL ? &norm_bwd_kernel<S, GATE_CHANNEL>
                          : a.kind == GATE_TOKEN ? &norm_bwd_kernel<S, GATE_TOKEN> : &norm_bwd_kernel<S, GATE_FULL>;
        hipLaunchKernelGGL(kernel, dim3(bwd_blocks<S>(a.T)), dim3(S::THREADS), 0, st, a);
    });
    probe::mark("norm_bwd", st);
}

}  // namespace

hipError_t norm_fwd(const NormArgs& a, hipStream_t st) {
    const FwdArgs k{a.res, a.y, a.gate, a.w_post, a.w_pre, a.r, a.n, a.rstd_post, a.rstd_pre,
                    a.res_scale, a.eps, a.T, a.d, a.gate_kind};
    if (a.f32) launch_fwd<true>(k, st);
    else launch_fwd<false>(k, st);
    return hipGetLastError();
}

size_t norm_bwd_workspace(int64_t T, int d, bool f32) {
    return (size_t)bwd_parts(T, d, f32) * 3 * d * sizeof(float);
}

hipError_t norm_bwd(const NormArgs& a, hipStream_t st) {
    const BwdArgs k{a.dr, a.dn, a.y, a.r, a.gate, a.w_post, a.w_pre, a.rstd_post, a.rstd_pre,
                    a.dres, a.dy, a.dgate, a.part, a.res_scale, a.T, a.d, a.gate_kind};
    const bool sums = a.w_pre || a.w_post || a.gate_kind == GATE_CHANNEL;
    if (a.T == 0 && !sums) return hipSuccess;
    if (a.T > 0) {
        if (a.f32) launch_bwd<true>(k, st);
        else launch_bwd<false>(k, st);
    }
    if (sums) {
        hipLaunchKernelGGL(norm_bwd_sum, dim3((a.d + 4 * SUM_COLS - 1) / (4 * SUM_COLS), 3),
                           dim3(SUM_COLS * SUM_SLICES), 0, st, a.part,
                           a.T > 0 ? bwd_parts(a.T, a.d, a.f32) : 0, a.d, a.w_pre ? a.dw_pre : nullptr,
                           a.w_post ? a.dw_post : nullptr,
                           a.gate_kind == GATE_CHANNEL ? static_cast<float*>(a.dgate) : nullptr);
        probe::mark("norm_bwd_sum", st);
    }
    return hipGetLastError();
}

}  // namespace moe
