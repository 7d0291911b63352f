// api.cpp -- the extern "C" entry points of libmoeblaze.so: argument
// validation (before anything is enqueued), then the internal launchers.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include <algorithm>
#include <new>
#include <vector>

#include "../../include/moeblaze.h"
#include "launch.hpp"
#include "probe.hpp"

namespace {

thread_local char g_err[512] = "";

int fail(int code, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
    return code;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

#define REQUIRE_PTR(p)                                                                 \
    do {                                                                               \
        if (!(p)) return fail(MOE_ERR_INVALID_ARG, "%s: %s is NULL", fn, #p);          \
        if (!aligned16(p)) return fail(MOE_ERR_INVALID_ARG, "%s: %s is not 16-byte aligned", fn, #p); \
    } while (0)
#define OPT_PTR(p)                                                                     \
    do {                                                                               \
        if ((p) && !aligned16(p))                                                      \
            return fail(MOE_ERR_INVALID_ARG, "%s: %s is not 16-byte aligned", fn, #p); \
    } while (0)

const unsigned KNOWN_FLAGS = MOE_F32 | MOE_RENORM | MOE_ACCUMULATE | MOE_ACT_SILU |
                             MOE_ACT_RELU | MOE_H_ON_LOAD | MOE_ACCUMULATE_DW |
                             MOE_ATOMIC_COMBINE;
const unsigned ACT_FLAGS = MOE_ACT_SILU | MOE_ACT_RELU;
// meaningful to the FFN calls only
const unsigned FFN_ONLY = ACT_FLAGS | MOE_H_ON_LOAD | MOE_ACCUMULATE_DW | MOE_ATOMIC_COMBINE;

// MOE_ATOMIC_COMBINE: combined bf16 calls only
int check_scatter(const char* fn, bool combined, unsigned flags) {
    if (!(flags & MOE_ATOMIC_COMBINE)) return MOE_OK;
    if (!combined)
        return fail(MOE_ERR_INVALID_ARG, "%s: MOE_ATOMIC_COMBINE applies to the combined calls only", fn);
    if (flags & MOE_F32)
        return fail(MOE_ERR_UNSUPPORTED, "%s: MOE_ATOMIC_COMBINE is bfloat16 only", fn);
    return MOE_OK;
}

// expert activation code of the FFN calls (0 SwiGLU, 1 SiLU, 2 ReLU), or -1
int act_of(unsigned flags) {
    const unsigned a = flags & ACT_FLAGS;
    return a == 0 ? 0 : a == MOE_ACT_SILU ? 1 : a == MOE_ACT_RELU ? 2 : -1;
}

int check_common(const char* fn, int64_t T, int E, int k, unsigned flags) {
    if (T < 0) return fail(MOE_ERR_INVALID_ARG, "%s: T = %lld < 0", fn, (long long)T);
    if (E < 1) return fail(MOE_ERR_INVALID_ARG, "%s: E = %d < 1", fn, E);
    if (k < 1) return fail(MOE_ERR_INVALID_ARG, "%s: k = %d < 1", fn, k);
    if (k > E) return fail(MOE_ERR_INVALID_ARG, "%s: k = %d > E = %d", fn, k, E);
    if (flags & ~KNOWN_FLAGS) return fail(MOE_ERR_INVALID_ARG, "%s: unknown flag bits 0x%x", fn, flags);
    if (E > 256) return fail(MOE_ERR_UNSUPPORTED, "%s: E = %d > 256", fn, E);
    if (k > 16) return fail(MOE_ERR_UNSUPPORTED, "%s: k = %d > 16", fn, k);
    if (T * (int64_t)k >= (int64_t(1) << 31))
        return fail(MOE_ERR_UNSUPPORTED, "%s: T*k = %lld does not fit int32 slots", fn,
                    (long long)(T * k));
    return MOE_OK;
}

int check_dim(const char* fn, const char* name, int v) {
    if (v < 1) return fail(MOE_ERR_INVALID_ARG, "%s: %s = %d < 1", fn, name, v);
    if (v % 64) return fail(MOE_ERR_UNSUPPORTED, "%s: %s = %d is not a multiple of 64", fn, name, v);
    return MOE_OK;
}

int hip_status(const char* fn, hipError_t e) {
    if (e != hipSuccess) return fail(MOE_ERR_HIP, "%s: %s", fn, hipGetErrorString(e));
    return MOE_OK;
}

}  // namespace

namespace {

// moe_ffn_fwd and moe_ffn_fwd_combine: O (plain) or y via gates and
// token_index_map (combined)
int ffn_fwd_impl(const char* fn, bool combined, const void* x, const void* w1, const void* w3,
                 const void* w2, const int32_t* offsets, const int32_t* expert_token_indices,
                 const float* gates, const int32_t* token_index_map, int64_t T, int d, int f,
                 int E, int k, unsigned flags, void* A, void* B, void* out, void* workspace,
                 size_t workspace_bytes, hipStream_t stream) {
    int r;
    if ((r = check_common(fn, T, E, k, flags)) || (r = check_dim(fn, "d", d)) ||
        (r = check_dim(fn, "f", f)))
        return r;
    if (flags & (MOE_RENORM | MOE_ACCUMULATE | MOE_ACCUMULATE_DW))
        return fail(MOE_ERR_INVALID_ARG, "%s: only MOE_F32 / MOE_BF16, an activation flag, MOE_H_ON_LOAD and (combined) MOE_ATOMIC_COMBINE are valid", fn);
    if ((r = check_scatter(fn, combined, flags))) return r;
    const int act = act_of(flags);
    if (act < 0) return fail(MOE_ERR_INVALID_ARG, "%s: MOE_ACT_SILU and MOE_ACT_RELU both set", fn);
    if (T == 0) return MOE_OK;
    REQUIRE_PTR(x); REQUIRE_PTR(w1); REQUIRE_PTR(w2); REQUIRE_PTR(offsets);
    REQUIRE_PTR(expert_token_indices); REQUIRE_PTR(A);
    if (combined) {
        const void* y = out;
        REQUIRE_PTR(gates); REQUIRE_PTR(token_index_map); REQUIRE_PTR(y);
    } else {
        const void* O = out;
        REQUIRE_PTR(O);
    }
    if (act == 0) { REQUIRE_PTR(w3); REQUIRE_PTR(B); }
    else { OPT_PTR(w3); OPT_PTR(B); }
    const size_t need =
        moe::ffn_fwd_workspace(T, d, f, E, k, flags & MOE_F32, combined, flags & MOE_H_ON_LOAD,
                               flags & MOE_ATOMIC_COMBINE);
    if (need && (!workspace || workspace_bytes < need))
        return fail(MOE_ERR_WORKSPACE, "%s: workspace %zu bytes < %zu needed", fn, workspace_bytes, need);
    OPT_PTR(workspace);
    moe::FfnArgs a{};
    a.x = x; a.w1 = w1; a.w3 = w3; a.w2 = w2; a.offsets = offsets; a.eti = expert_token_indices;
    a.A = A; a.B = B; a.T = T; a.d = d; a.f = f; a.E = E; a.k = k; a.ws = workspace;
    a.act = act;
    a.h_on_load = flags & MOE_H_ON_LOAD;
    a.scatter = flags & MOE_ATOMIC_COMBINE;
    if (combined) { a.y = out; a.gates = gates; a.tim = token_index_map; }
    else a.O = out;
    moe::probe::begin(stream);
    return hip_status(fn, moe::ffn_fwd(a, flags & MOE_F32, stream));
}

}  // namespace

namespace {

// moe_ffn_bwd and moe_ffn_bwd_combine: dX_slot (plain) or dx through
// token_index_map (combined; MOE_ACCUMULATE adds into dx)
int ffn_bwd_impl(const char* fn, bool combined, const void* dy, const void* x, const void* w1,
                 const void* w3, const void* w2, const float* gates, const int32_t* offsets,
                 const int32_t* expert_token_indices, const int32_t* slot_src,
                 const int32_t* token_index_map, void* A, void* B, int64_t T, int d, int f,
                 int E, int k, unsigned flags, float* dw1, float* dw3, float* dw2,
                 float* d_gates, void* out, void* workspace, size_t workspace_bytes,
                 hipStream_t stream) {
    int r;
    if ((r = check_common(fn, T, E, k, flags)) || (r = check_dim(fn, "d", d)) ||
        (r = check_dim(fn, "f", f)))
        return r;
    if ((flags & MOE_RENORM) || (!combined && (flags & MOE_ACCUMULATE)))
        return fail(MOE_ERR_INVALID_ARG, "%s: flag not valid here", fn);
    if ((r = check_scatter(fn, combined, flags))) return r;
    const int act = act_of(flags);
    if (act < 0) return fail(MOE_ERR_INVALID_ARG, "%s: MOE_ACT_SILU and MOE_ACT_RELU both set", fn);
    if (T == 0) return MOE_OK;
    REQUIRE_PTR(dy); REQUIRE_PTR(x); REQUIRE_PTR(w1); REQUIRE_PTR(w2);
    REQUIRE_PTR(gates); REQUIRE_PTR(offsets); REQUIRE_PTR(expert_token_indices);
    REQUIRE_PTR(slot_src); REQUIRE_PTR(A); REQUIRE_PTR(dw1);
    REQUIRE_PTR(dw2); REQUIRE_PTR(d_gates);
    if (combined) {
        const void* dx = out;
        REQUIRE_PTR(token_index_map); REQUIRE_PTR(dx);
    } else {
        const void* dX_slot = out;
        REQUIRE_PTR(dX_slot);
    }
    if (act == 0) { REQUIRE_PTR(w3); REQUIRE_PTR(B); REQUIRE_PTR(dw3); }
    else { OPT_PTR(w3); OPT_PTR(B); OPT_PTR(dw3); }
    const size_t need =
        moe::ffn_bwd_workspace(T, d, f, E, k, flags & MOE_F32, combined, flags & MOE_H_ON_LOAD,
                               flags & MOE_ATOMIC_COMBINE);
    if (need && (!workspace || workspace_bytes < need))
        return fail(MOE_ERR_WORKSPACE, "%s: workspace %zu bytes < %zu needed", fn, workspace_bytes, need);
    OPT_PTR(workspace);
    moe::FfnArgs a{};
    a.x = x; a.w1 = w1; a.w3 = w3; a.w2 = w2; a.offsets = offsets; a.eti = expert_token_indices;
    a.slot_src = slot_src; a.gates = gates; a.dy = dy; a.A = A; a.B = B;
    a.dw1 = dw1; a.dw3 = dw3; a.dw2 = dw2; a.dgates = d_gates; a.T = T; a.d = d; a.f = f;
    a.E = E; a.k = k; a.ws = workspace; a.act = act;
    a.h_on_load = flags & MOE_H_ON_LOAD;
    a.accumulate_dw = flags & MOE_ACCUMULATE_DW;
    a.scatter = flags & MOE_ATOMIC_COMBINE;
    if (combined) { a.y = out; a.tim = token_index_map; a.accumulate = flags & MOE_ACCUMULATE; }
    else a.dX = out;
    moe::probe::begin(stream);
    return hip_status(fn, moe::ffn_bwd(a, flags & MOE_F32, stream));
}

}  // namespace

extern "C" {

const char* moe_strerror(int status) {
    switch (status) {
        case MOE_OK: return "MOE_OK";
        case MOE_ERR_INVALID_ARG: return "MOE_ERR_INVALID_ARG";
        case MOE_ERR_UNSUPPORTED: return "MOE_ERR_UNSUPPORTED";
        case MOE_ERR_WORKSPACE: return "MOE_ERR_WORKSPACE";
        case MOE_ERR_HIP: return "MOE_ERR_HIP";
        default: return "unknown status";
    }
}

const char* moe_last_error(void) { return g_err; }

int moe_probe_enable(int capacity) {
    if (capacity < 1) return fail(MOE_ERR_INVALID_ARG, "moe_probe_enable: capacity %d < 1", capacity);
    if (moe::probe::enable(capacity) != 0)
        return fail(MOE_ERR_HIP, "moe_probe_enable: hipEventCreate failed");
    return MOE_OK;
}

void moe_probe_disable(void) { moe::probe::disable(); }

int moe_probe_count(void) { return moe::probe::count(); }

int moe_probe_dropped(void) { return moe::probe::dropped(); }

int moe_probe_get(int index, const char** kernel_name, float* ms) {
    if (!kernel_name || !ms) return fail(MOE_ERR_INVALID_ARG, "moe_probe_get: NULL output");
    if (moe::probe::get(index, kernel_name, ms) != 0)
        return fail(MOE_ERR_INVALID_ARG, "moe_probe_get: no record %d", index);
    return MOE_OK;
}

int moe_route(const void* x, const void* w_gate, const float* bias, int64_t T, int d, int E,
              int k, unsigned flags, int32_t* topk_ids, float* gates, float* logits,
              hipStream_t stream) {
    const char* fn = "moe_route";
    int r;
    if ((r = check_common(fn, T, E, k, flags)) || (r = check_dim(fn, "d", d))) return r;
    if (flags & FFN_ONLY) return fail(MOE_ERR_INVALID_ARG, "%s: activation, h-on-load and weight-gradient accumulation flags apply to the FFN calls only", fn);
    if (flags & MOE_ACCUMULATE) return fail(MOE_ERR_INVALID_ARG, "%s: MOE_ACCUMULATE not valid here", fn);
    if (T == 0) return MOE_OK;
    REQUIRE_PTR(x); REQUIRE_PTR(w_gate); OPT_PTR(bias); REQUIRE_PTR(topk_ids); REQUIRE_PTR(gates);
    OPT_PTR(logits);
    moe::probe::begin(stream);
    return hip_status(fn, moe::route(x, w_gate, bias, T, d, E, k, flags & MOE_F32,
                                     flags & MOE_RENORM, topk_ids, gates, logits, stream));
}

size_t moe_build_index_workspace_size(int64_t T, int E, int k) {
    if (T <= 0 || E < 1 || k < 1) return 0;
    return moe::build_index_workspace(T, E, k);
}

int moe_build_index(const int32_t* topk_ids, int64_t T, int E, int k, int32_t* counts,
                    int32_t* offsets, int32_t* expert_token_indices, int32_t* token_index_map,
                    int32_t* slot_src, void* workspace, size_t workspace_bytes,
                    hipStream_t stream) {
    const char* fn = "moe_build_index";
    int r;
    if ((r = check_common(fn, T, E, k, 0))) return r;
    if (T == 0) return MOE_OK;
    REQUIRE_PTR(topk_ids); REQUIRE_PTR(counts); REQUIRE_PTR(offsets);
    REQUIRE_PTR(expert_token_indices); REQUIRE_PTR(token_index_map); REQUIRE_PTR(slot_src);
    const size_t need = moe::build_index_workspace(T, E, k);
    if (!workspace || workspace_bytes < need)
        return fail(MOE_ERR_WORKSPACE, "%s: workspace %zu bytes < %zu needed", fn, workspace_bytes, need);
    REQUIRE_PTR(workspace);
    moe::probe::begin(stream);
    return hip_status(fn, moe::build_index(topk_ids, T, E, k, counts, offsets, expert_token_indices,
                                           token_index_map, slot_src, workspace, stream));
}

int moe_build_index_noalloc(const int32_t* topk_ids, int64_t T, int E, int k, int32_t* counts,
                            int32_t* offsets, int32_t* expert_token_indices,
                            int32_t* token_index_map, int32_t* slot_src, hipStream_t stream) {
    const char* fn = "moe_build_index_noalloc";
    int r;
    if ((r = check_common(fn, T, E, k, 0))) return r;
    if (T == 0) return MOE_OK;
    REQUIRE_PTR(topk_ids); REQUIRE_PTR(counts); REQUIRE_PTR(offsets);
    REQUIRE_PTR(expert_token_indices); REQUIRE_PTR(token_index_map); REQUIRE_PTR(slot_src);
    void* ws = nullptr;
    size_t have = 0;
    if (hipError_t e = moe::noalloc_scratch(&ws, &have); e != hipSuccess)
        return fail(MOE_ERR_HIP, "%s: scratch address lookup failed: %s", fn, hipGetErrorString(e));
    const size_t need = moe::build_index_workspace(T, E, k);
    if (need > have)
        return fail(MOE_ERR_UNSUPPORTED, "%s: needs %zu bytes of scratch, the static scratch holds %zu",
                    fn, need, have);
    moe::probe::begin(stream);
    return hip_status(fn, moe::build_index(topk_ids, T, E, k, counts, offsets, expert_token_indices,
                                           token_index_map, slot_src, ws, stream));
}

size_t moe_ffn_fwd_workspace_size(int64_t T, int d, int f, int E, int k, unsigned flags) {
    if (T <= 0 || d < 1 || f < 1 || E < 1 || k < 1) return 0;
    return moe::ffn_fwd_workspace(T, d, f, E, k, flags & MOE_F32, false, flags & MOE_H_ON_LOAD,
                                  false);
}

int moe_ffn_fwd(const void* x, const void* w1, const void* w3, const void* w2,
                const int32_t* offsets, const int32_t* expert_token_indices, int64_t T, int d,
                int f, int E, int k, unsigned flags, void* A, void* B, void* O, void* workspace,
                size_t workspace_bytes, hipStream_t stream) {
    return ffn_fwd_impl("moe_ffn_fwd", false, x, w1, w3, w2, offsets, expert_token_indices,
                        nullptr, nullptr, T, d, f, E, k, flags, A, B, O, workspace,
                        workspace_bytes, stream);
}

int moe_ffn_recompute(const void* x, const void* w1, const void* w3,
                      const int32_t* offsets, const int32_t* expert_token_indices, int64_t T,
                      int d, int f, int E, int k, unsigned flags, void* A, void* B,
                      hipStream_t stream) {
    const char* fn = "moe_ffn_recompute";
    int r;
    if ((r = check_common(fn, T, E, k, flags)) || (r = check_dim(fn, "d", d)) ||
        (r = check_dim(fn, "f", f)))
        return r;
    if (flags & (MOE_RENORM | MOE_ACCUMULATE | MOE_ACCUMULATE_DW | MOE_ATOMIC_COMBINE))
        return fail(MOE_ERR_INVALID_ARG, "%s: only MOE_F32 / MOE_BF16, an activation flag and MOE_H_ON_LOAD are valid", fn);
    const int act = act_of(flags);
    if (act < 0) return fail(MOE_ERR_INVALID_ARG, "%s: MOE_ACT_SILU and MOE_ACT_RELU both set", fn);
    if (T == 0) return MOE_OK;
    REQUIRE_PTR(x); REQUIRE_PTR(w1); REQUIRE_PTR(offsets); REQUIRE_PTR(expert_token_indices);
    REQUIRE_PTR(A);
    if (act == 0) { REQUIRE_PTR(w3); REQUIRE_PTR(B); }
    else { OPT_PTR(w3); OPT_PTR(B); }
    moe::FfnArgs a{};
    a.x = x; a.w1 = w1; a.w3 = w3; a.offsets = offsets; a.eti = expert_token_indices;
    a.A = A; a.B = B; a.T = T; a.d = d; a.f = f; a.E = E; a.k = k; a.act = act;
    moe::probe::begin(stream);
    return hip_status(fn, moe::ffn_first(a, flags & MOE_F32, stream));
}

size_t moe_ffn_fwd_combine_workspace_size(int64_t T, int d, int f, int E, int k, unsigned flags) {
    if (T <= 0 || d < 1 || f < 1 || E < 1 || k < 1) return 0;
    return moe::ffn_fwd_workspace(T, d, f, E, k, flags & MOE_F32, true, flags & MOE_H_ON_LOAD,
                                  flags & MOE_ATOMIC_COMBINE);
}

int moe_ffn_fwd_combine(const void* x, const void* w1, const void* w3, const void* w2,
                        const int32_t* offsets, const int32_t* expert_token_indices,
                        const float* gates, const int32_t* token_index_map, int64_t T, int d,
                        int f, int E, int k, unsigned flags, void* A, void* B, void* y,
                        void* workspace, size_t workspace_bytes, hipStream_t stream) {
    return ffn_fwd_impl("moe_ffn_fwd_combine", true, x, w1, w3, w2, offsets,
                        expert_token_indices, gates, token_index_map, T, d, f, E, k, flags, A, B,
                        y, workspace, workspace_bytes, stream);
}

int moe_combine(const void* src, const float* weights, const int32_t* token_index_map,
                int64_t T, int d, int k, unsigned flags, void* out, hipStream_t stream) {
    const char* fn = "moe_combine";
    int r;
    if ((r = check_common(fn, T, k, k, flags)) || (r = check_dim(fn, "d", d))) return r;
    if (flags & FFN_ONLY) return fail(MOE_ERR_INVALID_ARG, "%s: activation, h-on-load and weight-gradient accumulation flags apply to the FFN calls only", fn);
    if (flags & MOE_RENORM) return fail(MOE_ERR_INVALID_ARG, "%s: MOE_RENORM not valid here", fn);
    if (T == 0) return MOE_OK;
    REQUIRE_PTR(src); OPT_PTR(weights); REQUIRE_PTR(token_index_map); REQUIRE_PTR(out);
    moe::probe::begin(stream);
    return hip_status(fn, moe::combine(src, weights, token_index_map, T, d, k, flags & MOE_F32,
                                       flags & MOE_ACCUMULATE, out, stream));
}


size_t moe_ffn_bwd_workspace_size(int64_t T, int d, int f, int E, int k, unsigned flags) {
    if (T <= 0 || d < 1 || f < 1 || E < 1 || k < 1) return 0;
    return moe::ffn_bwd_workspace(T, d, f, E, k, flags & MOE_F32, false, flags & MOE_H_ON_LOAD,
                                  false);
}

int moe_ffn_bwd(const void* dy, const void* x, const void* w1, const void* w3, const void* w2,
                const float* gates, const int32_t* offsets, const int32_t* expert_token_indices,
                const int32_t* slot_src, void* A, void* B, int64_t T, int d, int f, int E, int k,
                unsigned flags, float* dw1, float* dw3, float* dw2, float* d_gates,
                void* dX_slot, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    return ffn_bwd_impl("moe_ffn_bwd", false, dy, x, w1, w3, w2, gates, offsets,
                        expert_token_indices, slot_src, nullptr, A, B, T, d, f, E, k, flags, dw1,
                        dw3, dw2, d_gates, dX_slot, workspace, workspace_bytes, stream);
}

size_t moe_ffn_bwd_combine_workspace_size(int64_t T, int d, int f, int E, int k, unsigned flags) {
    if (T <= 0 || d < 1 || f < 1 || E < 1 || k < 1) return 0;
    return moe::ffn_bwd_workspace(T, d, f, E, k, flags & MOE_F32, true, flags & MOE_H_ON_LOAD,
                                  flags & MOE_ATOMIC_COMBINE);
}

int moe_ffn_bwd_combine(const void* dy, const void* x, const void* w1, const void* w3,
                        const void* w2, const float* gates, const int32_t* offsets,
                        const int32_t* expert_token_indices, const int32_t* slot_src,
                        const int32_t* token_index_map, void* A, void* B, int64_t T, int d,
                        int f, int E, int k, unsigned flags, float* dw1, float* dw3, float* dw2,
                        float* d_gates, void* dx, void* workspace, size_t workspace_bytes,
                        hipStream_t stream) {
    return ffn_bwd_impl("moe_ffn_bwd_combine", true, dy, x, w1, w3, w2, gates, offsets,
                        expert_token_indices, slot_src, token_index_map, A, B, T, d, f, E, k,
                        flags, dw1, dw3, dw2, d_gates, dx, workspace, workspace_bytes, stream);
}

size_t moe_route_bwd_workspace_size(int64_t T, int d, int E, int k, unsigned flags) {
    if (T <= 0 || d < 1 || E < 1 || k < 1) return 0;
    return moe::route_bwd_workspace(T, d, E, k, flags & MOE_F32);
}

int moe_route_bwd(const float* d_gates, const float* logits, const int32_t* topk_ids,
                  const float* gates, const void* x, const void* w_gate, int64_t T, int d, int E,
                  int k, unsigned flags, float* dw_gate, void* dx, void* workspace,
                  size_t workspace_bytes, hipStream_t stream) {
    const char* fn = "moe_route_bwd";
    int r;
    if ((r = check_common(fn, T, E, k, flags)) || (r = check_dim(fn, "d", d))) return r;
    if (flags & FFN_ONLY) return fail(MOE_ERR_INVALID_ARG, "%s: activation, h-on-load and weight-gradient accumulation flags apply to the FFN calls only", fn);
    if (T == 0) return MOE_OK;
    REQUIRE_PTR(d_gates); REQUIRE_PTR(logits); REQUIRE_PTR(topk_ids); REQUIRE_PTR(gates);
    REQUIRE_PTR(x); REQUIRE_PTR(w_gate); REQUIRE_PTR(dw_gate); REQUIRE_PTR(dx);
    const size_t need = moe::route_bwd_workspace(T, d, E, k, flags & MOE_F32);
    if (!workspace || workspace_bytes < need)
        return fail(MOE_ERR_WORKSPACE, "%s: workspace %zu bytes < %zu needed", fn, workspace_bytes, need);
    REQUIRE_PTR(workspace);
    moe::probe::begin(stream);
    return hip_status(fn, moe::route_bwd(d_gates, logits, topk_ids, gates, x, w_gate, T, d, E, k,
                                         flags & MOE_F32, flags & MOE_RENORM,
                                         flags & MOE_ACCUMULATE, dw_gate, dx, workspace, stream));
}

// ---- norms of a residual block ----

}  // extern "C"

namespace {

// flags and sizes of the norm calls; `gate_kind`: 0 none, 1 [d], 2 [T], 3 [T, d]
int check_norm(const char* fn, int64_t T, int d, float res_scale, unsigned flags, int* gate_kind) {
    const unsigned known = MOE_F32 | MOE_NORM_POST | MOE_NORM_PRE | MOE_GATE_CHANNEL | MOE_GATE_TOKEN;
    if (flags & ~known) return fail(MOE_ERR_INVALID_ARG, "%s: unknown flag bits 0x%x", fn, flags & ~known);
    if (T < 0) return fail(MOE_ERR_INVALID_ARG, "%s: T = %lld < 0", fn, (long long)T);
    if (d < 1) return fail(MOE_ERR_INVALID_ARG, "%s: d = %d < 1", fn, d);
    if (d % 8) return fail(MOE_ERR_UNSUPPORTED, "%s: d = %d is not a multiple of 8", fn, d);
    if (d > 8192) return fail(MOE_ERR_UNSUPPORTED, "%s: d = %d > 8192", fn, d);
    if (!isfinite(res_scale)) return fail(MOE_ERR_INVALID_ARG, "%s: res_scale is not finite", fn);
    *gate_kind = (flags & MOE_GATE_CHANNEL ? 1 : 0) + (flags & MOE_GATE_TOKEN ? 2 : 0);
    return MOE_OK;
}

// what a call without a block output may not ask for
int check_no_block(const char* fn, float res_scale, unsigned flags) {
    if (flags & (MOE_NORM_POST | MOE_GATE_CHANNEL | MOE_GATE_TOKEN))
        return fail(MOE_ERR_INVALID_ARG, "%s: a post-norm or a gate without a block output", fn);
    if (!(flags & MOE_NORM_PRE))
        return fail(MOE_ERR_INVALID_ARG, "%s: neither a block output nor MOE_NORM_PRE: nothing to do", fn);
    if (res_scale != 1.0f)
        return fail(MOE_ERR_INVALID_ARG, "%s: res_scale must be 1 without a block output", fn);
    return MOE_OK;
}

// a pointer that a flag asks for, and that must be NULL without it
#define FLAG_PTR(p, on, why)                                                                   \
    do {                                                                                       \
        if (on) REQUIRE_PTR(p);                                                                \
        else if (p) return fail(MOE_ERR_INVALID_ARG, "%s: %s without %s", fn, #p, why);        \
    } while (0)

struct Span {
    uintptr_t lo, hi;
    bool written;
    int tensor;   // a gradient and its own output share a number
};

}  // namespace

extern "C" {

int moe_norm_fwd(const void* res, const void* y, const void* gate, const void* w_post,
                 const void* w_pre, float res_scale, float eps, int64_t T, int d, unsigned flags,
                 void* r, void* n, float* rstd_post, float* rstd_pre, hipStream_t stream) {
    const char* fn = "moe_norm_fwd";
    int e, kind;
    if ((e = check_norm(fn, T, d, res_scale, flags, &kind))) return e;
    if (!(eps > 0.0f) || !isfinite(eps)) return fail(MOE_ERR_INVALID_ARG, "%s: eps must be positive and finite", fn);
    if (T == 0) return MOE_OK;
    if (!y && (e = check_no_block(fn, res_scale, flags))) return e;
    REQUIRE_PTR(res); OPT_PTR(y); OPT_PTR(rstd_post); OPT_PTR(rstd_pre);
    FLAG_PTR(r, y != nullptr, "a block output");
    FLAG_PTR(gate, kind, "a gate flag");
    FLAG_PTR(w_post, flags & MOE_NORM_POST, "MOE_NORM_POST");
    FLAG_PTR(w_pre, flags & MOE_NORM_PRE, "MOE_NORM_PRE");
    FLAG_PTR(n, flags & MOE_NORM_PRE, "MOE_NORM_PRE");
    if (r && r == n) return fail(MOE_ERR_INVALID_ARG, "%s: r and n are the same", fn);
    moe::NormArgs a{};
    a.res = res; a.y = y; a.gate = gate; a.w_post = w_post; a.w_pre = w_pre; a.r = r; a.n = n;
    a.rstd_post = rstd_post; a.rstd_pre = rstd_pre; a.res_scale = res_scale; a.eps = eps;
    a.T = T; a.d = d; a.gate_kind = kind; a.f32 = flags & MOE_F32;
    moe::probe::begin(stream);
    return hip_status(fn, moe::norm_fwd(a, stream));
}

size_t moe_norm_bwd_workspace_size(int64_t T, int d, unsigned flags) {
    if (T <= 0 || d < 1 || d > 8192) return 0;
    return moe::norm_bwd_workspace(T, d, flags & MOE_F32);
}

int moe_norm_bwd(const void* dr, const void* dn, const void* y, const void* r, const void* gate,
                 const void* w_post, const void* w_pre, const float* rstd_post,
                 const float* rstd_pre, float res_scale, int64_t T, int d, unsigned flags,
                 void* dres, void* dy, void* dgate, float* dw_post, float* dw_pre, void* workspace,
                 size_t workspace_bytes, hipStream_t stream) {
    const char* fn = "moe_norm_bwd";
    int e, kind;
    if ((e = check_norm(fn, T, d, res_scale, flags, &kind))) return e;
    const bool post = flags & MOE_NORM_POST, pre = flags & MOE_NORM_PRE;
    FLAG_PTR(w_post, post, "MOE_NORM_POST"); FLAG_PTR(dw_post, post, "MOE_NORM_POST");
    FLAG_PTR(w_pre, pre, "MOE_NORM_PRE"); FLAG_PTR(dw_pre, pre, "MOE_NORM_PRE");
    // without rows a token's or a full gate has no element, and its address may be NULL
    if (T > 0 || kind < 2) FLAG_PTR(dgate, kind, "a gate flag");
    if (T > 0) {
        if (!dy && (e = check_no_block(fn, res_scale, flags))) return e;
        if (!dr && !pre) return fail(MOE_ERR_INVALID_ARG, "%s: neither dr nor MOE_NORM_PRE: no gradient comes in", fn);
        REQUIRE_PTR(dres); OPT_PTR(dr); OPT_PTR(dy); OPT_PTR(y); OPT_PTR(r);
        FLAG_PTR(gate, kind, "a gate flag");
        FLAG_PTR(dn, pre, "MOE_NORM_PRE");
        if (pre) { REQUIRE_PTR(r); REQUIRE_PTR(rstd_pre); }
        if (post) REQUIRE_PTR(rstd_post);
        if (post || kind) REQUIRE_PTR(y);
        if (dres == dy) return fail(MOE_ERR_INVALID_ARG, "%s: dres and dy are the same", fn);
        const size_t need = moe::norm_bwd_workspace(T, d, flags & MOE_F32);
        if (!workspace || workspace_bytes < need)
            return fail(MOE_ERR_WORKSPACE, "%s: workspace %zu bytes < %zu needed", fn, workspace_bytes, need);
        REQUIRE_PTR(workspace);
    }
    moe::NormArgs a{};
    a.dr = dr; a.dn = dn; a.y = y; a.r = const_cast<void*>(r); a.gate = gate; a.w_post = w_post;
    a.w_pre = w_pre; a.rstd_post = const_cast<float*>(rstd_post);
    a.rstd_pre = const_cast<float*>(rstd_pre); a.res_scale = res_scale; a.T = T; a.d = d;
    a.gate_kind = kind; a.f32 = flags & MOE_F32; a.dres = dres; a.dy = dy; a.dgate = dgate;
    a.dw_post = dw_post; a.dw_pre = dw_pre; a.part = static_cast<float*>(workspace);
    moe::probe::begin(stream);
    return hip_status(fn, moe::norm_bwd(a, stream));
}

// ---- gradient norm and clipping ----

}  // extern "C"

namespace {

int check_grads(const char* fn, const void* const* grads, const int64_t* sizes, const unsigned* types,
                int n) {
    if (n < 0) return fail(MOE_ERR_INVALID_ARG, "%s: n = %d < 0", fn, n);
    if (n > (1 << 20)) return fail(MOE_ERR_UNSUPPORTED, "%s: n = %d > 2^20 tensors", fn, n);
    if (n && (!grads || !sizes || !types)) return fail(MOE_ERR_INVALID_ARG, "%s: a NULL list", fn);
    for (int i = 0; i < n; ++i) {
        if (sizes[i] < 0) return fail(MOE_ERR_INVALID_ARG, "%s: sizes[%d] = %lld < 0", fn, i, (long long)sizes[i]);
        if (sizes[i] > (int64_t(1) << 44)) return fail(MOE_ERR_UNSUPPORTED, "%s: sizes[%d] > 2^44", fn, i);
        if (types[i] != MOE_BF16 && types[i] != MOE_F32)
            return fail(MOE_ERR_INVALID_ARG, "%s: types[%d] = 0x%x is neither MOE_BF16 nor MOE_F32", fn, i, types[i]);
        if (sizes[i] && !grads[i]) return fail(MOE_ERR_INVALID_ARG, "%s: grads[%d] is NULL", fn, i);
        if (sizes[i] && reinterpret_cast<uintptr_t>(grads[i]) % (types[i] == MOE_F32 ? 4 : 2))
            return fail(MOE_ERR_INVALID_ARG, "%s: grads[%d] is not aligned to its elements", fn, i);
    }
    return MOE_OK;
}

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
    return p < q + nb && q < p + na;
}

// Among the tensors that a clip reads and writes, no written one may share memory with
// another. O(n log n) on the host.
int check_overlap(const char* fn, const void* const* grads, void* const* outs, const int64_t* sizes,
                  const unsigned* types, int n) {
    std::vector<Span> v;
    v.reserve(2 * (size_t)n);
    for (int i = 0; i < n; ++i) {
        if (sizes[i] == 0) continue;
        const uintptr_t bytes = (uintptr_t)sizes[i] * (types[i] == MOE_F32 ? 4 : 2);
        const uintptr_t g = reinterpret_cast<uintptr_t>(grads[i]);
        const uintptr_t o = outs ? reinterpret_cast<uintptr_t>(outs[i]) : g;
        if (o == g) {
            v.push_back({g, g + bytes, true, i});
        } else {
            v.push_back({g, g + bytes, false, i});
            v.push_back({o, o + bytes, true, i});
        }
    }
    std::sort(v.begin(), v.end(), [](const Span& a, const Span& b) { return a.lo < b.lo; });
    // the furthest end so far, of all spans and of the written ones
    uintptr_t end = 0, wend = 0;
    int who = 0, wwho = 0;
    for (const Span& s : v) {
        if (s.written && s.lo < end)
            return fail(MOE_ERR_INVALID_ARG, "%s: tensors %d and %d overlap, and one of them is written", fn, who, s.tensor);
        if (s.lo < wend)
            return fail(MOE_ERR_INVALID_ARG, "%s: tensors %d and %d overlap, and one of them is written", fn, wwho, s.tensor);
        if (s.hi > end) { end = s.hi; who = s.tensor; }
        if (s.written && s.hi > wend) { wend = s.hi; wwho = s.tensor; }
    }
    return MOE_OK;
}

}  // namespace

extern "C" {

size_t moe_grad_norm_workspace_size(int n) { return n < 1 ? 0 : moe::grad_norm_workspace(n); }

int moe_grad_norm(const void* const* grads, const int64_t* sizes, const unsigned* types, int n,
                  double* sumsq, float* norm, void* workspace, size_t workspace_bytes,
                  hipStream_t stream) {
    const char* fn = "moe_grad_norm";
    int e;
    if ((e = check_grads(fn, grads, sizes, types, n))) return e;
    if (!sumsq || reinterpret_cast<uintptr_t>(sumsq) % 8) return fail(MOE_ERR_INVALID_ARG, "%s: sumsq is NULL or not aligned", fn);
    if (!norm || reinterpret_cast<uintptr_t>(norm) % 4) return fail(MOE_ERR_INVALID_ARG, "%s: norm is NULL or not aligned", fn);
    const size_t need = moe_grad_norm_workspace_size(n);
    if (need && (!workspace || workspace_bytes < need))
        return fail(MOE_ERR_WORKSPACE, "%s: workspace %zu bytes < %zu needed", fn, workspace_bytes, need);
    OPT_PTR(workspace);
    moe::probe::begin(stream);
    return hip_status(fn, moe::grad_norm(grads, sizes, types, n, sumsq, norm, workspace, stream));
}

int moe_grad_clip(const void* const* grads, void* const* outs, const int64_t* sizes,
                  const unsigned* types, int n, const double* sumsq, double max_norm,
                  hipStream_t stream) {
    const char* fn = "moe_grad_clip";
    int e;
    if ((e = check_grads(fn, grads, sizes, types, n))) return e;
    if (!(max_norm >= 0.0)) return fail(MOE_ERR_INVALID_ARG, "%s: max_norm must be zero or more", fn);
    if (!sumsq || reinterpret_cast<uintptr_t>(sumsq) % 8) return fail(MOE_ERR_INVALID_ARG, "%s: sumsq is NULL or not aligned", fn);
    for (int i = 0; outs && i < n; ++i)
        if (sizes[i] && (!outs[i] || reinterpret_cast<uintptr_t>(outs[i]) % (types[i] == MOE_F32 ? 4 : 2)))
            return fail(MOE_ERR_INVALID_ARG, "%s: outs[%d] is NULL or not aligned to its elements", fn, i);
    try {
        if ((e = check_overlap(fn, grads, outs, sizes, types, n))) return e;
    } catch (const std::bad_alloc&) {
        return fail(MOE_ERR_INVALID_ARG, "%s: no host memory for %d tensors", fn, n);
    }
    moe::probe::begin(stream);
    return hip_status(fn, moe::grad_clip(grads, outs ? outs : const_cast<void* const*>(grads), sizes,
                                         types, n, sumsq, max_norm, stream));
}

// ---- microscaled 4-bit values and the products over them ----

int moe_mx_quantize(const void* src, int64_t batch, int64_t R, int K, unsigned flags, void* codes,
                    void* scales, hipStream_t stream) {
    const char* fn = "moe_mx_quantize";
    const unsigned known = MOE_F32 | MOE_TRANSPOSED;
    if (flags & ~known) return fail(MOE_ERR_INVALID_ARG, "%s: unknown flag bits 0x%x", fn, flags & ~known);
    if (batch < 0 || R < 0) return fail(MOE_ERR_INVALID_ARG, "%s: batch = %lld, R = %lld", fn, (long long)batch, (long long)R);
    if (K < 1) return fail(MOE_ERR_INVALID_ARG, "%s: K = %d < 1", fn, K);
    if (K % 32) return fail(MOE_ERR_UNSUPPORTED, "%s: K = %d is not a multiple of 32", fn, K);
    // a launch has fewer than 2^32 threads: 16 values each, 256 a workgroup
    if ((double)batch * (double)R * K > 68719476736.0 - 4096.0)
        return fail(MOE_ERR_UNSUPPORTED, "%s: more than 2^36 - 4096 values", fn);
    if (flags & MOE_TRANSPOSED) {
        if (R % 2) return fail(MOE_ERR_UNSUPPORTED, "%s: R = %lld is odd (MOE_TRANSPOSED)", fn, (long long)R);
        if (batch > 65535) return fail(MOE_ERR_UNSUPPORTED, "%s: batch = %lld > 65535 (MOE_TRANSPOSED)", fn, (long long)batch);
        // 1024 threads for 128 columns
        if (R > (1 << 29) - 128) return fail(MOE_ERR_UNSUPPORTED, "%s: R = %lld > 2^29 - 128 (MOE_TRANSPOSED)", fn, (long long)R);
        if (K > (1 << 24)) return fail(MOE_ERR_UNSUPPORTED, "%s: K = %d > 2^24 (MOE_TRANSPOSED)", fn, K);
    }
    if (batch == 0 || R == 0) return MOE_OK;
    REQUIRE_PTR(src); REQUIRE_PTR(codes); REQUIRE_PTR(scales);
    moe::probe::begin(stream);
    return hip_status(fn, moe::mx_quantize(src, batch, R, K, flags & MOE_F32, flags & MOE_TRANSPOSED,
                                           codes, scales, stream));
}

int moe_mx_dequantize(const void* codes, const void* scales, int64_t R, int K, unsigned flags,
                      void* out, hipStream_t stream) {
    const char* fn = "moe_mx_dequantize";
    if (flags & ~MOE_F32) return fail(MOE_ERR_INVALID_ARG, "%s: unknown flag bits 0x%x", fn, flags & ~MOE_F32);
    if (R < 0) return fail(MOE_ERR_INVALID_ARG, "%s: R = %lld < 0", fn, (long long)R);
    if (K < 1) return fail(MOE_ERR_INVALID_ARG, "%s: K = %d < 1", fn, K);
    if (K % 32) return fail(MOE_ERR_UNSUPPORTED, "%s: K = %d is not a multiple of 32", fn, K);
    if ((double)R * K >= 68719476736.0) return fail(MOE_ERR_UNSUPPORTED, "%s: 2^36 values or more", fn);
    if (R == 0) return MOE_OK;
    REQUIRE_PTR(codes); REQUIRE_PTR(scales); REQUIRE_PTR(out);
    moe::probe::begin(stream);
    return hip_status(fn, moe::mx_dequantize(codes, scales, R * K, flags & MOE_F32, out, stream));
}

int moe_mx_gemm(const void* x, const void* x_scales, const void* w, const void* w_scales,
                const void* w3, const void* w3_scales, const int32_t* offsets, const int32_t* rows,
                int64_t T, int64_t S, int K, int N, int E, unsigned flags, void* out,
                hipStream_t stream) {
    const char* fn = "moe_mx_gemm";
    const unsigned known = MOE_F32 | ACT_FLAGS | MOE_GATED;
    int r;
    if (flags & ~known) return fail(MOE_ERR_INVALID_ARG, "%s: unknown flag bits 0x%x", fn, flags & ~known);
    if (flags & MOE_F32) return fail(MOE_ERR_UNSUPPORTED, "%s: bfloat16 only", fn);
    const unsigned act = flags & (ACT_FLAGS | MOE_GATED);
    if (act & (act - 1)) return fail(MOE_ERR_INVALID_ARG, "%s: at most one of MOE_GATED, MOE_ACT_SILU, MOE_ACT_RELU", fn);
    if (T < 0 || S < 0) return fail(MOE_ERR_INVALID_ARG, "%s: T = %lld, S = %lld", fn, (long long)T, (long long)S);
    if (E < 1) return fail(MOE_ERR_INVALID_ARG, "%s: E = %d < 1", fn, E);
    if (E > 256) return fail(MOE_ERR_UNSUPPORTED, "%s: E = %d > 256", fn, E);
    if ((r = check_dim(fn, "K", K)) || (r = check_dim(fn, "N", N))) return r;
    if (S >= (int64_t(1) << 31) || T >= (int64_t(1) << 31))
        return fail(MOE_ERR_UNSUPPORTED, "%s: T = %lld, S = %lld do not fit int32", fn, (long long)T, (long long)S);
    if ((int64_t)N * K >= (int64_t(1) << 33))
        return fail(MOE_ERR_UNSUPPORTED, "%s: N * K = %lld, 2^33 or more", fn, (long long)N * K);
    if (!rows && S != T) return fail(MOE_ERR_INVALID_ARG, "%s: rows is NULL and T = %lld is not S = %lld", fn, (long long)T, (long long)S);
    if (S > 0 && T == 0) return fail(MOE_ERR_INVALID_ARG, "%s: T = 0 with S = %lld slots", fn, (long long)S);
    if (S == 0) return MOE_OK;
    REQUIRE_PTR(x); REQUIRE_PTR(w); REQUIRE_PTR(w_scales); REQUIRE_PTR(offsets); REQUIRE_PTR(out);
    OPT_PTR(x_scales); OPT_PTR(rows);
    FLAG_PTR(w3, flags & MOE_GATED, "MOE_GATED");
    FLAG_PTR(w3_scales, flags & MOE_GATED, "MOE_GATED");
    // workgroups read x and the weights while others write
    const size_t row = x_scales ? K / 2 : 2 * (size_t)K, mat = (size_t)E * N * (K / 2);
    const struct { const void* p; size_t bytes; const char* name; } in[] = {
        {x, T * row, "x"}, {x_scales, T * (size_t)(K / 32), "x_scales"}, {w, mat, "w"},
        {w_scales, mat / 16, "w_scales"}, {w3, mat, "w3"}, {w3_scales, mat / 16, "w3_scales"},
        {offsets, (E + 1) * sizeof *offsets, "offsets"}, {rows, S * sizeof *rows, "rows"}};
    for (const auto& i : in)
        if (i.p && overlap(i.p, i.bytes, out, (size_t)S * N * 2))
            return fail(MOE_ERR_INVALID_ARG, "%s: out overlaps %s", fn, i.name);
    moe::MxArgs a{};
    a.x = x; a.xs = static_cast<const uint8_t*>(x_scales);
    a.w = static_cast<const uint8_t*>(w); a.ws = static_cast<const uint8_t*>(w_scales);
    a.w3 = static_cast<const uint8_t*>(w3); a.ws3 = static_cast<const uint8_t*>(w3_scales);
    a.offsets = offsets; a.rows = rows; a.T = T; a.S = S; a.N = N; a.K = K; a.E = E;
    a.act = act_of(flags); a.out = out;
    moe::probe::begin(stream);
    return hip_status(fn, moe::mx_gemm(a, stream));
}

}  // extern "C"
