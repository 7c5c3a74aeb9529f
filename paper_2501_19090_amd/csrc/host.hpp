// Host-side helpers that the library's translation units share: status macros,
// device checks, overlap checks, and the timing of launches.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <mutex>
#include <vector>

#include "../../include/pifa.h"
#include "common.hpp"

namespace pifa {

constexpr int64_t kCus = 256;

#define PIFA_HIP(call)                                  \
    do {                                                \
        if ((call) != hipSuccess) return PIFA_ERR_HIP;  \
    } while (0)

inline hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// A handle's memory lives on the device current at its creation; launching
// its kernels with another device current would touch that memory from the
// wrong GPU, so such calls are refused.
inline pifa_status check_device(int dev) {
    int cur = -1;
    if (hipGetDevice(&cur) != hipSuccess) return PIFA_ERR_HIP;
    return cur == dev ? PIFA_OK : PIFA_ERR_WRONG_DEVICE;
}

#define PIFA_ON_DEVICE(dev)                      \
    do {                                         \
        const pifa_status s_ = check_device(dev); \
        if (s_ != PIFA_OK) return s_;            \
    } while (0)
inline size_t esize(pifa_dtype dt) { return dt == PIFA_BF16 ? 2 : 4; }
inline bool valid_dtype(pifa_dtype dt) { return dt == PIFA_BF16 || dt == PIFA_F32; }

inline unsigned grid_for(int64_t work) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(ceil_div(work, 256), 65536)); }

inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && x < y + nb && y < x + na;
}

// An output of n bytes over one of these inputs, other than in its place.
inline bool overlap_part(const void* out, size_t n, std::initializer_list<const void*> in) {
    for (const void* p : in)
        if (out != p && overlap(out, n, p, n)) return true;
    return false;
}
// An output over any of these buffers.
struct Buffer {
    const void* p;
    size_t n;
};
inline bool overlap_any(const void* out, size_t n, std::initializer_list<Buffer> others) {
    for (const Buffer& b : others)
        if (overlap(out, n, b.p, b.n)) return true;
    return false;
}

// ------------------------------------------------------------------ norms
// A launch may not pass 2^32 threads: columns of a row in one launch (64 columns
// of dgain take 1024 threads), rows of one launch (1024 threads at most each).
constexpr int64_t kNormMaxD = 1ll << 27, kNormMaxRows = 1ll << 21;

inline pifa_status check_norm(int64_t M, int64_t d, pifa_dtype dtype, float eps) {
    if (!valid_dtype(dtype) || M < 0 || d < 1 || !(eps > 0.f) || std::isinf(eps)) return PIFA_ERR_INVALID_ARG;
    if (d > kNormMaxD || M > INT32_MAX) return PIFA_ERR_UNSUPPORTED;
    return PIFA_OK;
}

// ------------------------------------------------------------------ kernel timing
enum Site {
    kSitePifaGemm1 = 0,
    kSitePifaGemm2,
    kSitePifaGemv1,
    kSitePifaGemv2,
    kSitePifaF32Gemm1,
    kSitePifaF32Gemm2,
    kSiteDenseGemm,
    kSiteDenseGemv,
    kSiteDenseF32,
    kSiteLowrankGemm1,
    kSiteLowrankGemm2,
    kSiteLowrankGemv1,
    kSiteLowrankGemv2,
    kSiteLowrankF32,
    kSiteGroupGemm1,
    kSiteGroupGemm2,
    kSiteGroupGemv1,
    kSiteGroupGemv2,
    kSiteBwdData,
    kSiteBwdGp,
    kSiteBwdDx,
    kSiteBwdDwp,
    kSiteBwdDc,
    kSiteBwdRows,
    kSiteCalibGather,
    kSiteCalibGram,
    kSiteCalibSolve,
    kSiteNorm,
    kSiteNormBwd,
    kSiteNormDgain,
    kSiteQ4,
    kSiteQ4Norm,
    kSiteLayerNorm,
    kSiteLayerNormBwd,
    kSiteLayerNormSums,
    kSiteAdapterPlan,
    kSiteAdapterShrink,
    kSiteAdapterExpand,
    kSiteAdapterGrads,
    kSiteAdapterSums,
    kSiteAdamw,
    kSiteCount
};

inline const char* const kSiteNames[kSiteCount] = {
    "pifa_gemm1_xwp",      "pifa_gemm2_ypc",      "pifa_gemv1_xwp",      "pifa_gemv2_ypc",
    "pifa_f32_gemm1",      "pifa_f32_gemm2",      "dense_gemm",          "dense_gemv",
    "dense_f32",           "lowrank_gemm1_xv",    "lowrank_gemm2_tu",    "lowrank_gemv1_xv",
    "lowrank_gemv2_tu",    "lowrank_f32",         "pifa_group_gemm1",    "pifa_group_gemm2",
    "pifa_group_gemv1",    "pifa_group_gemv2",    "pifa_bwd_gather",     "pifa_bwd_gp",
    "pifa_bwd_dx",         "pifa_bwd_dwp",        "pifa_bwd_dc",         "pifa_bwd_rows_f16",
    "pifa_calib_gather",   "pifa_calib_gram",     "pifa_calib_solve",
    "rms_norm",            "rms_norm_bwd",        "rms_norm_dgain",      "q4_product",
    "q4_norm_product",     "layer_norm",          "layer_norm_bwd",      "layer_norm_sums",
    "adapter_plan",        "adapter_shrink",      "adapter_expand",      "adapter_grads",
    "adapter_sums",        "adamw"};

struct Profiler {
    std::mutex mu;
    bool on = false;
    struct Rec {
        int site;
        hipEvent_t start, stop;
    };
    std::vector<Rec> pending;
    std::vector<hipEvent_t> pool;
    int64_t launches[kSiteCount] = {};
    double ms[kSiteCount] = {};

    hipEvent_t get() {
        if (!pool.empty()) {
            hipEvent_t e = pool.back();
            pool.pop_back();
            return e;
        }
        hipEvent_t e = nullptr;
        if (hipEventCreate(&e) != hipSuccess) return nullptr;
        return e;
    }
};

inline Profiler& profiler() {
    static Profiler p;
    return p;
}

// Set while a call runs that must create nothing (pifa_forward_noalloc):
// its launches are never bracketed by profiling events.
inline thread_local bool t_untimed = false;

// Brackets one launch with events when profiling is on.
struct TimedLaunch {
    int site;
    hipStream_t st;
    hipEvent_t start = nullptr, stop = nullptr;
    TimedLaunch(int s, hipStream_t stream) : site(s), st(stream) {
        Profiler& p = profiler();
        if (!p.on || t_untimed) return;
        std::lock_guard<std::mutex> g(p.mu);
        start = p.get();
        stop = p.get();
        if (start) (void)hipEventRecord(start, st);
    }
    ~TimedLaunch() {
        if (!start || !stop) return;
        Profiler& p = profiler();
        (void)hipEventRecord(stop, st);
        std::lock_guard<std::mutex> g(p.mu);
        p.pending.push_back({site, start, stop});
    }
};

}  // namespace pifa
