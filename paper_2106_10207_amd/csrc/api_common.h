// What the files of the C-ABI layer share: the calling thread's last error,
// the per-kernel event profiler and small checks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

#include <mutex>
#include <string>
#include <vector>

#include "../../include/dedloc.h"

namespace dedloc {

inline thread_local std::string g_err;

inline int fail(int code, const char *fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    g_err = buf;
    return code;
}

inline int hip_fail(hipError_t e, const char *what) {
    return fail(DEDLOC_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }

// ------------------------------------------------------------ profiling
enum Kind {
    K_ENCODE_FP16, K_DECODE_FP16, K_ENCODE_I8, K_DECODE_I8, K_REDUCE_FP16, K_REDUCE_I8,
    K_LAMB_A_F32, K_LAMB_A_FP16, K_LAMB_A_I8, K_LAMB_A_FUSED_FP16, K_LAMB_B,
    K_LARS_A_F32, K_LARS_A_FP16, K_LARS_A_I8, K_LARS_A_FUSED_FP16, K_LARS_B,
    K_ACCUMULATE, K_FINALIZE_FP16, K_FINALIZE_I8, K_FILL,
    K_NS_SUM, K_NS_PREPARE, K_NS_PRODUCT, K_NS_JOIN, K_NS_NARROW, K_MUON_SUM,
    K_EMBED, K_EMBED_SORT, K_EMBED_MERGE, K_EMBED_COUNT, K_EMBED_SCATTER, K_EMBED_SUM, K_EMBED_JOIN,
    K_DROPOUT, K_RESIDUAL, K_RESIDUAL_GRAD, K_RESIDUAL_JOIN, K_GATE_JOIN, K_COUNT
};
inline const char *const kKindNames[K_COUNT] = {
    "encode_fp16", "decode_fp16", "encode_i8", "decode_i8", "reduce_fp16", "reduce_i8",
    "lamb_a_f32", "lamb_a_fp16", "lamb_a_i8", "lamb_a_fused_fp16", "lamb_b",
    "lars_a_f32", "lars_a_fp16", "lars_a_i8", "lars_a_fused_fp16", "lars_b",
    "accumulate", "finalize_fp16", "finalize_i8", "fill_zero",
    "ns_sum", "ns_prepare", "ns_product", "ns_join", "ns_narrow", "muon_sum",
    "embed", "embed_sort", "embed_merge", "embed_count", "embed_scatter", "embed_sum", "embed_join",
    "dropout", "residual", "residual_grad", "residual_join", "gate_join"};

struct Profiler {
    std::mutex mu;
    bool on = false;
    uint32_t cap = 0;
    std::vector<hipEvent_t> ev;     // 2 per recorded launch
    std::vector<int> kind;
    size_t used = 0;
};
inline Profiler g_prof;

// Run `launch` (returning hipError_t), bracketed by events when profiling.
template <typename F>
hipError_t timed(int kind, hipStream_t s, F launch) {
    std::unique_lock<std::mutex> lk(g_prof.mu);
    if (!g_prof.on || g_prof.used >= g_prof.cap) {
        lk.unlock();
        return launch();
    }
    const size_t i = g_prof.used++;
    while (g_prof.ev.size() < 2 * g_prof.used) {
        hipEvent_t e;
        hipError_t r = hipEventCreate(&e);
        if (r != hipSuccess) return r;
        g_prof.ev.push_back(e);
    }
    g_prof.kind.resize(g_prof.used);
    g_prof.kind[i] = kind;
    hipError_t r = hipEventRecord(g_prof.ev[2 * i], s);
    if (r != hipSuccess) return r;
    r = launch();
    if (r != hipSuccess) return r;
    return hipEventRecord(g_prof.ev[2 * i + 1], s);
}

inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

}  // namespace dedloc
