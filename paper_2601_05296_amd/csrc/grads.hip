// grads.hip -- the global norm of a list of gradients, and clipping by it.
//
//   sumsq = sum over all tensors of g^2,  c = min(1, max_norm / (sqrt(sumsq) + 1e-6)),
//   out = c g
// The layer's own gradients are the reason: 2.2 GB of float32 for 64 experts of
// 2048 x 1408, far beyond any cache, so each pass is one stream over HBM. Squares and
// sums are 64-bit (a float32 square overflows past 1.8e19 and loses values below 1e-19;
// one convert and one fused multiply-add per element take a quarter of the time that
// reading the element does), so the sum of several devices' or calls' results is exact
// enough to add up. Partial sums are added in one fixed order: no atomics.
// 554 million float32 values: the norm 365 us, 6.1 TB/s, the highest rate reached for reading;
// scaling them into other tensors 890 us, 5.0 TB/s, a copy's. (Scaling them from the last
// piece to the first, which a cache might still hold: no faster.)
#include "common.hpp"
#include "launch.hpp"
#include "probe.hpp"

#include <algorithm>

namespace moe {
namespace {

constexpr int GT = 256;              // threads
constexpr int TABLE = 96;            // tensors a launch: the table travels with the launch
constexpr int CHUNK_VECS = 4096;     // 16-byte vectors of one piece of work
constexpr int BLOCKS = 2048;         // partial sums of a launch

struct Entry {
    const void* g;
    void* out;
    int64_t n;
};
struct Table {
    Entry t[TABLE];
    int64_t first[TABLE + 1];        // first chunk of each tensor
    unsigned f32[(TABLE + 31) / 32];
    int n;
};
__device__ __forceinline__ bool is_f32(const Table& t, int i) { return t.f32[i >> 5] >> (i & 31) & 1; }

// the tensor that holds chunk c
__device__ __forceinline__ int find(const Table& t, int64_t c) {
    int lo = 0, hi = t.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= c) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ void add_sq(double& s, float v) { s = fma((double)v, (double)v, s); }

// s += the squares of one 16-byte vector
template <bool F32>
__device__ __forceinline__ void add_vec(double& s, const uint4& v) {
    if constexpr (F32) {
        add_sq(s, __uint_as_float(v.x)); add_sq(s, __uint_as_float(v.y));
        add_sq(s, __uint_as_float(v.z)); add_sq(s, __uint_as_float(v.w));
    } else {
        float f[8];
        unpack8(v, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) add_sq(s, f[i]);
    }
}

template <bool F32>
__device__ __forceinline__ float load1(const void* p, int64_t i) {
    if constexpr (F32) return static_cast<const float*>(p)[i];
    else return bf2f(static_cast<const bf16_t*>(p)[i]);
}

template <bool F32>
__device__ __forceinline__ double chunk_sq(const Entry& e, int64_t c) {
    constexpr int EPV = F32 ? 4 : 8;
    const int64_t e0 = c * CHUNK_VECS * EPV;
    double s = 0.0;
    if (reinterpret_cast<uintptr_t>(e.g) & 15) {   // a view that starts inside a vector
        const int64_t e1 = min(e.n, e0 + (int64_t)CHUNK_VECS * EPV);
        for (int64_t i = e0 + threadIdx.x; i < e1; i += GT) add_sq(s, load1<F32>(e.g, i));
        return s;
    }
    const int64_t nv = e.n / EPV;
    const int64_t v0 = c * CHUNK_VECS;
    const uint4* p = static_cast<const uint4*>(e.g) + v0;
    const int m = (int)min((int64_t)CHUNK_VECS, nv - v0);
    int i = threadIdx.x;
    for (; i + 7 * GT < m; i += 8 * GT) {
        uint4 v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = p[i + u * GT];
#pragma unroll
        for (int u = 0; u < 8; ++u) add_vec<F32>(s, v[u]);
    }
    for (; i < m; i += GT) add_vec<F32>(s, p[i]);
    // the last elements, fewer than a vector, go with the chunk that ends the tensor
    const int64_t rest = nv * EPV + threadIdx.x;
    if (e0 + (int64_t)CHUNK_VECS * EPV >= e.n && rest < e.n) add_sq(s, load1<F32>(e.g, rest));
    return s;
}

__device__ __forceinline__ double block_sum(double s) {
    __shared__ double lds[GT / 64];
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int i = 0; i < GT / 64; ++i) s += lds[i];
    return s;
}

// part: this launch's BLOCKS partial sums; with `one`, the only workgroup's sum is the result
__global__ void __launch_bounds__(GT)
grad_sumsq(const Table t, double* __restrict__ part, double* sumsq, float* norm) {
    double s = 0.0;
    for (int64_t c = blockIdx.x; c < t.first[t.n]; c += gridDim.x) {
        const int i = find(t, c);
        const Entry e = t.t[i];
        s += is_f32(t, i) ? chunk_sq<true>(e, c - t.first[i]) : chunk_sq<false>(e, c - t.first[i]);
    }
    s = block_sum(s);
    if (threadIdx.x) return;
    if (sumsq) {
        *sumsq = s;
        *norm = (float)sqrt(s);
    } else {
        part[blockIdx.x] = s;
    }
}

__global__ void __launch_bounds__(GT)
grad_sum_parts(const double* __restrict__ part, int n, double* __restrict__ sumsq, float* __restrict__ norm) {
    double s = 0.0;
    for (int i = threadIdx.x; i < n; i += GT) s += part[i];
    s = block_sum(s);
    if (threadIdx.x) return;
    *sumsq = s;
    *norm = (float)sqrt(s);
}

template <bool F32>
__device__ __forceinline__ uint4 scaled(const uint4& v, float c) {
    if constexpr (F32) {
        return make_uint4(__float_as_uint(c * __uint_as_float(v.x)), __float_as_uint(c * __uint_as_float(v.y)),
                          __float_as_uint(c * __uint_as_float(v.z)), __float_as_uint(c * __uint_as_float(v.w)));
    } else {
        float f[8];
        unpack8(v, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] *= c;
        return pack8(f);
    }
}

template <bool F32>
__device__ __forceinline__ void chunk_scale(const Entry& e, int64_t c, float k) {
    constexpr int EPV = F32 ? 4 : 8;
    const int64_t e0 = c * CHUNK_VECS * EPV;
    auto one = [&](int64_t i) {
        const float v = k * load1<F32>(e.g, i);
        if constexpr (F32) static_cast<float*>(e.out)[i] = v;
        else static_cast<bf16_t*>(e.out)[i] = (bf16_t)f2bf(v);
    };
    if ((reinterpret_cast<uintptr_t>(e.g) | reinterpret_cast<uintptr_t>(e.out)) & 15) {
        const int64_t e1 = min(e.n, e0 + (int64_t)CHUNK_VECS * EPV);
        for (int64_t i = e0 + threadIdx.x; i < e1; i += GT) one(i);
        return;
    }
    const int64_t nv = e.n / EPV;
    const int64_t v0 = c * CHUNK_VECS;
    const uint4* p = static_cast<const uint4*>(e.g) + v0;
    uint4* q = static_cast<uint4*>(e.out) + v0;
    const int m = (int)min((int64_t)CHUNK_VECS, nv - v0);
    int i = threadIdx.x;
    for (; i + 7 * GT < m; i += 8 * GT) {
        uint4 v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = p[i + u * GT];
#pragma unroll
        for (int u = 0; u < 8; ++u) st16_nt(q + i + u * GT, scaled<F32>(v[u], k));
    }
    for (; i < m; i += GT) q[i] = scaled<F32>(p[i], k);
    const int64_t rest = nv * EPV + threadIdx.x;
    if (e0 + (int64_t)CHUNK_VECS * EPV >= e.n && rest < e.n) one(rest);
}

__global__ void __launch_bounds__(GT)
grad_scale(const Table t, const double* __restrict__ sumsq, double max_norm) {
    // a norm up to the limit, an infinite one up to an infinite limit: unchanged; NaN stays
    const double norm = sqrt(*sumsq) + 1e-6;
    const float k = norm <= max_norm ? 1.0f : (float)(max_norm / norm);
    for (int64_t c = blockIdx.x; c < t.first[t.n]; c += gridDim.x) {
        const int i = find(t, c);
        const Entry e = t.t[i];
        if (e.g == e.out && k == 1.0f) continue;   // in place and nothing to clip
        if (is_f32(t, i)) chunk_scale<true>(e, c - t.first[i], k);
        else chunk_scale<false>(e, c - t.first[i], k);
    }
}

// The tables of tensors [i0, i0 + TABLE): empty ones are left out.
Table make_table(const void* const* g, void* const* out, const int64_t* sizes, const unsigned* types,
                 int i0, int n) {
    Table t{};
    for (int i = i0; i < n && i < i0 + TABLE; ++i) {
        if (sizes[i] == 0) continue;
        const int64_t per = (types[i] & 1u) ? (int64_t)CHUNK_VECS * 4 : (int64_t)CHUNK_VECS * 8;
        t.t[t.n] = Entry{g[i], out ? out[i] : nullptr, sizes[i]};
        if (types[i] & 1u) t.f32[t.n >> 5] |= 1u << (t.n & 31);
        t.first[t.n + 1] = t.first[t.n] + (sizes[i] + per - 1) / per;
        ++t.n;
    }
    return t;
}

int grid_of(const Table& t) { return (int)std::min<int64_t>(BLOCKS, t.first[t.n]); }

}  // namespace

size_t grad_norm_workspace(int n) { return (size_t)((n + TABLE - 1) / TABLE) * BLOCKS * sizeof(double); }

hipError_t grad_norm(const void* const* g, const int64_t* sizes, const unsigned* types, int n,
                     double* sumsq, float* norm, void* ws, hipStream_t st) {
    double* part = static_cast<double*>(ws);
    int parts = 0;
    for (int i0 = 0; i0 < n; i0 += TABLE) {
        const Table t = make_table(g, nullptr, sizes, types, i0, n);
        const int grid = grid_of(t);
        if (grid == 0) continue;
        const bool only = grid == 1 && n <= TABLE;   // one launch does
        hipLaunchKernelGGL(grad_sumsq, dim3(grid), dim3(GT), 0, st, t, part + parts,
                           only ? sumsq : nullptr, only ? norm : nullptr);
        probe::mark("grad_sumsq", st);
        if (only) return hipGetLastError();
        parts += grid;
    }
    hipLaunchKernelGGL(grad_sum_parts, dim3(1), dim3(GT), 0, st, part, parts, sumsq, norm);
    probe::mark("grad_sum_parts", st);
    return hipGetLastError();
}

hipError_t grad_clip(const void* const* g, void* const* out, const int64_t* sizes,
                     const unsigned* types, int n, const double* sumsq, double max_norm,
                     hipStream_t st) {
    bool any = false;
    for (int i0 = 0; i0 < n; i0 += TABLE) {
        const Table t = make_table(g, out, sizes, types, i0, n);
        const int grid = grid_of(t);
        if (grid == 0) continue;
        hipLaunchKernelGGL(grad_scale, dim3(grid), dim3(GT), 0, st, t, sumsq, max_norm);
        probe::mark("grad_scale", st);
        any = true;
    }
    return any ? hipGetLastError() : hipSuccess;
}

}  // namespace moe
