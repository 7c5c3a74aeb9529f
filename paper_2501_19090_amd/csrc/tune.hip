// libpifa: what fine-tuning a compressed model, and serving what came of it,
// needs around its layers: layer norms, low-rank adapters, AdamW.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <new>
#include <vector>

#include "../../include/pifa.h"
#include "adamw.hpp"
#include "adapter.hpp"
#include "common.hpp"
#include "host.hpp"
#include "layer_norm.hpp"
#include "norm.hpp"

using namespace pifa;

// ===================================================================== layer norms
namespace {

template <typename T, int TPR, int V, int ROWS>
void layer_norm_fwd_launch(const LayerNormFwd<T>& p, hipStream_t st) {
    hipLaunchKernelGGL((layer_norm_fwd<T, TPR, V, ROWS>), dim3((unsigned)ceil_div(p.M, ROWS)), dim3(TPR * ROWS), 0, st,
                       p);
}

// Threads of a row x its chunks each, by the row's full chunks, as for the
// root-mean-square norm.
template <typename T>
hipError_t launch_layer_norm(const LayerNormFwd<T>& p, hipStream_t st) {
    TimedLaunch timed(kSiteLayerNorm, st);
    const int64_t chunks = p.d / NormChunk<T>::N;  // full ones
    if (chunks <= 64) layer_norm_fwd_launch<T, 64, 1, 4>(p, st);
    else if (chunks <= 256) layer_norm_fwd_launch<T, 256, 1, 1>(p, st);
    else if (chunks <= 512 && p.M > kCus) layer_norm_fwd_launch<T, 256, 2, 1>(p, st);
    else if (chunks <= 1024 && p.M > kCus) layer_norm_fwd_launch<T, 256, 4, 1>(p, st);
    else if (chunks <= 1024) layer_norm_fwd_launch<T, 1024, 1, 1>(p, st);
    else if (chunks <= 2048) layer_norm_fwd_launch<T, 1024, 2, 1>(p, st);
    else if (chunks <= 4096) layer_norm_fwd_launch<T, 1024, 4, 1>(p, st);
    else hipLaunchKernelGGL((layer_norm_fwd_long<T>), dim3((unsigned)p.M), dim3(kNormThreads), 0, st, p);
    return hipGetLastError();
}

template <typename T>
hipError_t layer_norm_forward_run(const void* X, const void* R, const void* gain, const void* bias, float eps, void* H,
                                  void* Y, int64_t M, int64_t d, hipStream_t st) {
    for (int64_t m = 0; m < M; m += kNormMaxRows) {
        const int64_t at = m * d;
        auto from = [&](auto* p) { return p ? p + at : p; };
        const LayerNormFwd<T> p{from((const T*)X), from((const T*)R), (const T*)gain, (const T*)bias, from((T*)H),
                                from((T*)Y), std::min(kNormMaxRows, M - m), d, eps};
        const hipError_t e = launch_layer_norm<T>(p, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Backward: rows a workgroup takes at a time, a thread of its 1024 for each of a
// row's full chunks; at most one workgroup per CU, so that there are few partial
// sums.
int64_t layer_norm_bwd_rows(int64_t d, int64_t n) {
    const int64_t chunks = d / n;
    return chunks <= 64 ? 16 : chunks <= 128 ? 8 : chunks <= 256 ? 4 : chunks <= 512 ? 2 : 1;
}
int64_t layer_norm_bwd_groups(int64_t M, int64_t d, int64_t n) {
    return std::min<int64_t>({kCus, kNormMaxGroups, ceil_div(M, layer_norm_bwd_rows(d, n))});
}

template <typename T>
pifa_status layer_norm_backward_run(const void* H, const void* gain, const void* dY, const void* dR, float eps, void* dX,
                                    float* dgain, float* dbias, int64_t M, int64_t d, float* work, hipStream_t st) {
    constexpr int64_t N = NormChunk<T>::N;
    const int64_t chunks = d / N, groups = layer_norm_bwd_groups(M, d, N);
    const bool sums = groups > 1 && (dgain || dbias);
    const LayerNormBwd<T> p{(const T*)H, (const T*)gain, (const T*)dY, (const T*)dR, (T*)dX,
                            dgain && sums ? work : dgain, dbias && sums ? work + d : dbias, 2 * d, M, d, eps};
    {
        TimedLaunch timed(kSiteLayerNormBwd, st);
        const dim3 grid((unsigned)groups), block(kNormThreads);
        const bool whole = d % N == 0 && dR && dX;
        auto launch = [&](auto tpr, auto v) {
            constexpr int TPR = decltype(tpr)::value, V = decltype(v)::value;
            if (whole && chunks == TPR * V) hipLaunchKernelGGL((layer_norm_bwd<T, TPR, V, true>), grid, block, 0, st, p);
            else hipLaunchKernelGGL((layer_norm_bwd<T, TPR, V, false>), grid, block, 0, st, p);
        };
        using std::integral_constant;
        if (chunks <= 64) launch(integral_constant<int, 64>{}, integral_constant<int, 1>{});
        else if (chunks <= 128) launch(integral_constant<int, 128>{}, integral_constant<int, 1>{});
        else if (chunks <= 256) launch(integral_constant<int, 256>{}, integral_constant<int, 1>{});
        else if (chunks <= 512) launch(integral_constant<int, 512>{}, integral_constant<int, 1>{});
        else if (chunks <= 1024) launch(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
        else if (chunks <= 2048) launch(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
        else if (sizeof(T) == 4 && chunks <= 4096) launch(integral_constant<int, 1024>{}, integral_constant<int, sizeof(T) == 4 ? 4 : 2>{});
        else hipLaunchKernelGGL((layer_norm_bwd_long<T>), grid, block, 0, st, p);
        if (hipGetLastError() != hipSuccess) return PIFA_ERR_HIP;
    }
    if (sums) {
        TimedLaunch timed(kSiteLayerNormSums, st);
        hipLaunchKernelGGL(norm_dgain, dim3((unsigned)ceil_div(d, kWave), 2), dim3(kNormThreads), 0, st, work,
                           (int)groups, d, dgain, dbias);
        if (hipGetLastError() != hipSuccess) return PIFA_ERR_HIP;
    }
    return PIFA_OK;
}

}  // namespace

// ===================================================================== adapters
namespace {

constexpr int64_t kAdMaxD = 1 << 19, kAdMaxRank = 1024;
// Workgroups of shrink that the chip holds at once, three or two a CU, for one or two
// jobs and by their blocks of columns of t.
int adapter_target(int64_t r, int jobs) {
    return (int)((r <= 16 ? 3 : 2) * kCus / (jobs * ceil_div(adapter_rp(r), 64)));
}

pifa_status check_plan(int64_t M, int64_t n) {
    if (M < 0 || n < 1) return PIFA_ERR_INVALID_ARG;
    return M > kAdMaxRows || n > kAdMaxSlots ? PIFA_ERR_UNSUPPORTED : PIFA_OK;
}
pifa_status check_adapter(int64_t M, int64_t d_in, int64_t d_out, int64_t r, int64_t n) {
    const pifa_status s = check_plan(M, n);
    if (s == PIFA_ERR_INVALID_ARG || d_in < 1 || d_out < 1 || r < 1) return PIFA_ERR_INVALID_ARG;
    return s != PIFA_OK || d_in > kAdMaxD || d_out > kAdMaxD || r > kAdMaxRank ? PIFA_ERR_UNSUPPORTED : PIFA_OK;
}
bool aligned(std::initializer_list<const void*> p, uintptr_t to) {
    for (const void* x : p)
        if ((uintptr_t)x % to != 0) return false;
    return true;
}

// Up to as many rows t stays in parts, which each workgroup of expand adds up itself,
// without finish between.  us of 4096 -> 12288 so, and with finish: 16 rows of rank 16
// 7.5 and 9.2, of rank 64 11.3 and 11.3, of rank 128 14.7 and 13.2; 256 rows 10.4 and
// 12.0, 20.7 and 17.0, 35.9 and 20.6; 512 rows of rank 16 13.5 and 14.7, of rank 64
// 31.5 and 20.3.  So the rows alone decide well up to rank 32, and cost up to 1.8 times
// the call above.
constexpr int64_t kAdFewRows = 256;

// Bytes of t (or u): at most 8 parts of K of every tile, and where K is cut at all,
// no more parts than its target; of its forms for expand and for grads.
size_t adapter_t_bytes(int64_t M, int64_t r, int64_t n) {
    const int64_t tiles = adapter_max_tiles(M, n);
    const int64_t parts = std::min<int64_t>(kAdMaxSplit * tiles, std::max<int64_t>(tiles, adapter_target(r, 1)));
    return (size_t)(parts * kAdTile * adapter_rp(r) * 4);
}
size_t adapter_halves_bytes(int64_t M, int64_t r, int64_t n) {
    return (size_t)(adapter_max_tiles(M, n) * kAdTile * 2 * adapter_rp(r) * 2);
}
size_t adapter_turned_bytes(int64_t M, int64_t r, int64_t n) {
    return (size_t)(adapter_max_tiles(M, n) * kAdTile * 3 * adapter_rp(r) * 2);
}
size_t adapter_partial_bytes(int64_t M, int64_t r, int64_t d) {
    return (size_t)round_up(2 * (M / kAdPiece) * r * d * 4, 256);
}

AdapterPlan adapter_read_plan(const void* plan, int64_t M, int64_t n) {
    AdapterPlan p;
    (void)adapter_layout(const_cast<void*>(plan), M, n, &p);
    return p;
}

// One or two shrinks in a launch.
hipError_t launch_shrink(const AdapterShrink& a, const AdapterShrink* b, const AdapterPlan& p, int64_t M, int64_t n,
                         int64_t r, int target, hipStream_t st) {
    TimedLaunch timed(kSiteAdapterShrink, st);
    const int64_t rp = adapter_rp(r), jb = std::min<int64_t>(4, rp / 16), most = std::max(a.K, b ? b->K : 0);
    const dim3 grid((unsigned)adapter_max_tiles(M, n), (unsigned)adapter_splits(1, most, target),
                    (unsigned)(ceil_div(rp, 16 * jb) * (b ? 2 : 1)));
    const dim3 block(kAdWaves * kWave);
    const AdapterShrink& second = b ? *b : a;
    if (jb == 1) hipLaunchKernelGGL((adapter_shrink<1>), grid, block, 0, st, a, second, p, M, (int)n, r, target);
    else if (jb == 2) hipLaunchKernelGGL((adapter_shrink<2>), grid, block, 0, st, a, second, p, M, (int)n, r, target);
    else hipLaunchKernelGGL((adapter_shrink<4>), grid, block, 0, st, a, second, p, M, (int)n, r, target);
    return hipGetLastError();
}

hipError_t launch_finish(const AdapterFinish& a, const AdapterFinish* b, const AdapterPlan& p, int64_t M, int64_t n,
                         int64_t r, int target, hipStream_t st) {
    TimedLaunch timed(kSiteAdapterShrink, st);
    const int64_t tiles = adapter_max_tiles(M, n);
    hipLaunchKernelGGL(adapter_finish, dim3((unsigned)tiles, (unsigned)(adapter_rp(r) / 16), b ? 2 : 1), dim3(256), 0, st, a,
                       b ? *b : a, p, M, (int)n, r, target);
    return hipGetLastError();
}

template <bool SUM, bool COL>
hipError_t launch_expand(const AdapterExpand& a, const AdapterPlan& p, int64_t M, int64_t n, int64_t r, int target,
                         hipStream_t st) {
    TimedLaunch timed(kSiteAdapterExpand, st);
    // columns keep to their XCD over the tiles, so that it reads only its part of W
    const int64_t blocks = ceil_div(a.d, kAdWide);
    const dim3 grid((unsigned)(blocks > 8 ? round_up(blocks, 8) : blocks), (unsigned)adapter_max_tiles(M, n));
    auto launch = [&](auto kb, auto one) {
        constexpr int KB = decltype(kb)::value;
        constexpr bool ONE = decltype(one)::value;
        hipLaunchKernelGGL((adapter_expand<KB, ONE, SUM, COL>), grid, dim3(kAdThreads), 0, st, a, p, M, (int)n, r, target);
    };
    using std::integral_constant;
    if (r <= 16) launch(integral_constant<int, 0>{}, std::true_type{});
    else if (r <= 32) launch(integral_constant<int, 1>{}, std::true_type{});
    else if (r <= 64) launch(integral_constant<int, 2>{}, std::true_type{});
    else launch(integral_constant<int, 2>{}, std::false_type{});
    return hipGetLastError();
}

}  // namespace

// ===================================================================== AdamW
struct adamw_state {
    int device = 0;
    int bits = 32;
    pifa_dtype g_dtype = PIFA_F32;
    uint32_t seed = 0;
    int64_t chunks = 0;
    void* memory = nullptr;  // the tables and the count, one allocation
    AdamwTensor* tensors = nullptr;
    AdamwChunk* table = nullptr;
    AdamwStep* count = nullptr;
};

namespace {

constexpr int64_t kAdamwMaxChunks = 1ll << 23;  // of one launch: its threads stay below 2^32

void free_adamw(adamw_state* h) {
    if (!h) return;
    if (h->memory) (void)hipFree(h->memory);
    delete h;
}

struct Span {
    uintptr_t from, to;
    bool out;
};

// No two outputs, and no output and gradient, share a byte.
bool adamw_overlap(std::vector<Span>& spans) {
    std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.from < b.from; });
    uintptr_t end_out = 0, end_any = 0;  // of those seen so far
    for (const Span& s : spans) {
        if (s.from < end_out || (s.out && s.from < end_any)) return true;
        end_any = std::max(end_any, s.to);
        if (s.out) end_out = std::max(end_out, s.to);
    }
    return false;
}

pifa_status adamw_check(const adamw_tensor* tensors, int64_t count, int bits, pifa_dtype g_dtype, int64_t* chunks) {
    if (!tensors || count < 1 || (bits != 8 && bits != 32) || !valid_dtype(g_dtype)) return PIFA_ERR_INVALID_ARG;
    if (count > INT32_MAX) return PIFA_ERR_UNSUPPORTED;
    const size_t ms = bits == 8 ? 1 : 4;
    std::vector<Span> spans;
    *chunks = 0;
    bool aligned = true;
    for (int64_t i = 0; i < count; ++i) {
        const adamw_tensor& t = tensors[i];
        if (t.n < 0 || !(t.weight_decay >= 0.0) || std::isinf(t.weight_decay)) return PIFA_ERR_INVALID_ARG;
        if (t.n == 0) continue;
        if (!t.p || !t.g || !t.m || !t.v || (bits == 8 && (!t.m_scale || !t.v_scale))) return PIFA_ERR_INVALID_ARG;
        if (t.n > kAdamwMaxChunks * kAdamwChunk) return PIFA_ERR_UNSUPPORTED;
        auto add = [&](const void* p, size_t bytes, bool out) {
            if (p) spans.push_back({(uintptr_t)p, (uintptr_t)p + bytes, out});
        };
        const size_t n = (size_t)t.n, groups = (size_t)ceil_div(t.n, kAdamwGroup);
        add(t.p, 4 * n, true);
        add(t.m, ms * n, true);
        add(t.v, ms * n, true);
        if (bits == 8) {
            add(t.m_scale, groups, true);
            add(t.v_scale, groups, true);
        }
        add(t.p_bf16, 2 * n, true);
        add(t.g, esize(g_dtype) * n, false);
        aligned = aligned && (uintptr_t)t.p % 4 == 0 && (uintptr_t)t.m % ms == 0 && (uintptr_t)t.v % ms == 0 &&
                  (uintptr_t)t.p_bf16 % 2 == 0 && (uintptr_t)t.g % esize(g_dtype) == 0;
        *chunks += ceil_div(t.n, kAdamwChunk);
        if (*chunks > kAdamwMaxChunks) return PIFA_ERR_UNSUPPORTED;
    }
    if (adamw_overlap(spans)) return PIFA_ERR_INVALID_ARG;
    return aligned ? PIFA_OK : PIFA_ERR_UNSUPPORTED;
}

}  // namespace

extern "C" {

pifa_status layer_norm_forward(const void* X, const void* R, const void* gain, const void* bias, float eps, void* H,
                               void* Y, int64_t M, int64_t d, pifa_dtype dtype, void* stream) {
    const pifa_status s = check_norm(M, d, dtype, eps);
    if (s != PIFA_OK) return s;
    if (M == 0) return PIFA_OK;
    if (!X || !Y) return PIFA_ERR_INVALID_ARG;
    const size_t n = (size_t)M * (size_t)d * esize(dtype), row = (size_t)d * esize(dtype);
    if (overlap_part(H, n, {X, R}) || overlap_part(Y, n, {X, R}) ||
        overlap_any(H, n, {{gain, row}, {bias, row}, {Y, n}}) || overlap_any(Y, n, {{gain, row}, {bias, row}}))
        return PIFA_ERR_INVALID_ARG;
    const hipStream_t st = as_stream(stream);
    const hipError_t e = dtype == PIFA_BF16 ? layer_norm_forward_run<bf16>(X, R, gain, bias, eps, H, Y, M, d, st)
                                            : layer_norm_forward_run<float>(X, R, gain, bias, eps, H, Y, M, d, st);
    return e == hipSuccess ? PIFA_OK : PIFA_ERR_HIP;
}

size_t layer_norm_backward_bytes(int64_t M, int64_t d) {
    if (M < 1 || d < 1 || d > kNormMaxD || M > INT32_MAX) return 0;
    const int64_t groups =
        std::max(layer_norm_bwd_groups(M, d, NormChunk<bf16>::N), layer_norm_bwd_groups(M, d, NormChunk<float>::N));
    return groups > 1 ? (size_t)groups * (size_t)d * 2 * sizeof(float) : 0;
}

pifa_status layer_norm_backward(const void* H, const void* gain, const void* dY, const void* dR, float eps, void* dX,
                                float* dgain, float* dbias, int64_t M, int64_t d, pifa_dtype dtype, void* work,
                                size_t work_bytes, void* stream) {
    const pifa_status s = check_norm(M, d, dtype, eps);
    if (s != PIFA_OK) return s;
    const hipStream_t st = as_stream(stream);
    const size_t ng = (size_t)d * sizeof(float);
    if (overlap(dgain, ng, dbias, ng)) return PIFA_ERR_INVALID_ARG;
    if (M == 0) {
        for (float* p : {dgain, dbias})
            if (p) hipLaunchKernelGGL(norm_zero, dim3(grid_for(d)), dim3(256), 0, st, p, d);
        return (dgain || dbias) && hipGetLastError() != hipSuccess ? PIFA_ERR_HIP : PIFA_OK;
    }
    if (!H || !dY) return PIFA_ERR_INVALID_ARG;
    if (!dX && !dgain && !dbias) return PIFA_OK;
    const size_t need = dgain || dbias ? layer_norm_backward_bytes(M, d) : 0;
    if (need > 0 && (!work || work_bytes < need)) return PIFA_ERR_INVALID_ARG;
    const size_t n = (size_t)M * (size_t)d * esize(dtype), row = (size_t)d * esize(dtype);
    const Buffer part{need > 0 ? work : nullptr, need};
    if (overlap_part(dX, n, {H, dY, dR}) || overlap_any(dX, n, {{gain, row}, {dgain, ng}, {dbias, ng}, part}))
        return PIFA_ERR_INVALID_ARG;
    for (const Buffer& b : {Buffer{dgain, ng}, Buffer{dbias, ng}, part})
        if (overlap_any(b.p, b.n, {{H, n}, {gain, row}, {dY, n}, {dR, n}})) return PIFA_ERR_INVALID_ARG;
    if (overlap(part.p, part.n, dgain, ng) || overlap(part.p, part.n, dbias, ng)) return PIFA_ERR_INVALID_ARG;
    if (need > 0 && ((uintptr_t)work & 3) != 0) return PIFA_ERR_UNSUPPORTED;
    return dtype == PIFA_BF16
               ? layer_norm_backward_run<bf16>(H, gain, dY, dR, eps, dX, dgain, dbias, M, d, (float*)work, st)
               : layer_norm_backward_run<float>(H, gain, dY, dR, eps, dX, dgain, dbias, M, d, (float*)work, st);
}

size_t adapter_plan_bytes(int64_t M, int64_t n) {
    if (check_plan(M, n) != PIFA_OK) return 0;
    AdapterPlan p;
    return adapter_layout(nullptr, M, n, &p);
}

pifa_status adapter_plan(const int32_t* ids, int64_t M, int64_t n, void* plan, size_t plan_bytes, void* stream) {
    const pifa_status s = check_plan(M, n);
    if (s != PIFA_OK) return s;
    const size_t need = adapter_plan_bytes(M, n);
    if ((M > 0 && !ids) || !plan || plan_bytes < need || overlap(plan, need, ids, (size_t)M * 4))
        return PIFA_ERR_INVALID_ARG;
    if (!aligned({ids}, 4) || !aligned({plan}, 16)) return PIFA_ERR_UNSUPPORTED;
    const hipStream_t st = as_stream(stream);
    const AdapterPlan p = adapter_read_plan(plan, M, n);
    const unsigned blocks = (unsigned)std::max<int64_t>(1, adapter_blocks(M));
    TimedLaunch timed(kSiteAdapterPlan, st);
    if (blocks > 1) hipLaunchKernelGGL(adapter_hist, dim3(blocks), dim3(1024), 0, st, ids, M, (int)n, p);
    hipLaunchKernelGGL(adapter_place, dim3(blocks), dim3(1024), 0, st, ids, M, (int)n, p);
    return hipGetLastError() == hipSuccess ? PIFA_OK : PIFA_ERR_HIP;
}

size_t adapter_forward_bytes(int64_t M, int64_t d_in, int64_t d_out, int64_t r, int64_t n) {
    if (check_adapter(M, d_in, d_out, r, n) != PIFA_OK) return 0;
    return adapter_t_bytes(M, r, n) + (M > kAdFewRows ? adapter_halves_bytes(M, r, n) : 0);
}

pifa_status adapter_forward(const void* X, const void* A, const void* B, const float* scale, const void* plan,
                            const void* Y0, void* Y, int64_t M, int64_t d_in, int64_t d_out, int64_t r, int64_t n,
                            void* work, size_t work_bytes, void* stream) {
    const pifa_status s = check_adapter(M, d_in, d_out, r, n);
    if (s != PIFA_OK) return s;
    if (M == 0) return PIFA_OK;
    const size_t need = adapter_forward_bytes(M, d_in, d_out, r, n);
    if (!X || !A || !B || !plan || !Y || !work || work_bytes < need) return PIFA_ERR_INVALID_ARG;
    const Buffer in[] = {{X, (size_t)(2 * M * d_in)}, {A, (size_t)(2 * n * r * d_in)}, {B, (size_t)(2 * n * r * d_out)},
                         {scale, (size_t)(4 * n)}, {plan, adapter_plan_bytes(M, n)}};
    const Buffer y{Y, (size_t)(2 * M * d_out)}, y0{Y0, y.n}, w{work, need};
    for (const Buffer& b : in)
        if (overlap(y.p, y.n, b.p, b.n) || overlap(w.p, w.n, b.p, b.n)) return PIFA_ERR_INVALID_ARG;
    if (overlap_part(Y, y.n, {Y0}) || overlap(w.p, w.n, y.p, y.n) || overlap(w.p, w.n, y0.p, y0.n))
        return PIFA_ERR_INVALID_ARG;
    if (!aligned({X, A, B, Y0, Y}, 2) || !aligned({scale}, 4) || !aligned({plan, work}, 16)) return PIFA_ERR_UNSUPPORTED;
    const hipStream_t st = as_stream(stream);
    const AdapterPlan p = adapter_read_plan(plan, M, n);
    const int target = adapter_target(r, 1);
    float* T = (float*)work;
    u32x4* halves = (u32x4*)((uint8_t*)work + adapter_t_bytes(M, r, n));
    if (launch_shrink({(const bf16*)X, (const bf16*)A, false, scale, T, d_in}, nullptr, p, M, n, r, target, st) != hipSuccess)
        return PIFA_ERR_HIP;
    const AdapterExpand expand{T, halves, (const bf16*)B, (const bf16*)Y0, (bf16*)Y, d_out, d_in};
    if (M <= kAdFewRows) return launch_expand<true, false>(expand, p, M, n, r, target, st) == hipSuccess ? PIFA_OK : PIFA_ERR_HIP;
    if (launch_finish({T, halves, nullptr, d_in}, nullptr, p, M, n, r, target, st) != hipSuccess ||
        launch_expand<false, false>(expand, p, M, n, r, target, st) != hipSuccess)
        return PIFA_ERR_HIP;
    return PIFA_OK;
}

size_t adapter_backward_bytes(int64_t M, int64_t d_in, int64_t d_out, int64_t r, int64_t n) {
    if (check_adapter(M, d_in, d_out, r, n) != PIFA_OK) return 0;
    return 2 * adapter_t_bytes(M, r, n) + adapter_halves_bytes(M, r, n) + 2 * adapter_turned_bytes(M, r, n) +
           adapter_partial_bytes(M, r, d_in) + adapter_partial_bytes(M, r, d_out);
}

pifa_status adapter_backward(const void* X, const void* A, const void* B, const float* scale, const void* plan,
                             const void* dY, const void* dX0, void* dX, float* dA, float* dB, int64_t M, int64_t d_in,
                             int64_t d_out, int64_t r, int64_t n, void* work, size_t work_bytes, void* stream) {
    const pifa_status s = check_adapter(M, d_in, d_out, r, n);
    if (s != PIFA_OK) return s;
    const size_t na = (size_t)(4 * n * r * d_in), nb = (size_t)(4 * n * r * d_out);
    if (overlap(dA, na, dB, nb)) return PIFA_ERR_INVALID_ARG;
    const hipStream_t st = as_stream(stream);
    if (M == 0) {
        if (dA) hipLaunchKernelGGL(norm_zero, dim3(grid_for(n * r * d_in)), dim3(256), 0, st, dA, n * r * d_in);
        if (dB) hipLaunchKernelGGL(norm_zero, dim3(grid_for(n * r * d_out)), dim3(256), 0, st, dB, n * r * d_out);
        return (dA || dB) && hipGetLastError() != hipSuccess ? PIFA_ERR_HIP : PIFA_OK;
    }
    if (!dX && !dA && !dB) return PIFA_OK;
    const size_t need = adapter_backward_bytes(M, d_in, d_out, r, n);
    if (!X || !A || !B || !plan || !dY || !work || work_bytes < need) return PIFA_ERR_INVALID_ARG;
    const Buffer in[] = {{X, (size_t)(2 * M * d_in)}, {A, na / 2}, {B, nb / 2}, {scale, (size_t)(4 * n)},
                         {plan, adapter_plan_bytes(M, n)}, {dY, (size_t)(2 * M * d_out)}};
    const Buffer dx{dX, (size_t)(2 * M * d_in)}, dx0{dX0, dx.n}, w{work, need};
    const Buffer out[] = {dx, {dA, na}, {dB, nb}, w};
    for (const Buffer& o : out)
        for (const Buffer& b : in)
            if (overlap(o.p, o.n, b.p, b.n)) return PIFA_ERR_INVALID_ARG;
    if (overlap_part(dX, dx.n, {dX0}) || overlap_any(dA, na, {dx, dx0, w}) || overlap_any(dB, nb, {dx, dx0, w}) ||
        overlap_any(work, need, {dx, dx0}))
        return PIFA_ERR_INVALID_ARG;
    if (!aligned({X, A, B, dY, dX0, dX}, 2) || !aligned({scale, dA, dB}, 4) || !aligned({plan, work}, 16))
        return PIFA_ERR_UNSUPPORTED;
    const AdapterPlan p = adapter_read_plan(plan, M, n);
    uint8_t* at = (uint8_t*)work;
    auto take = [&](size_t bytes) {
        uint8_t* r = at;
        at += bytes;
        return r;
    };
    float* T = (float*)take(adapter_t_bytes(M, r, n));
    float* U = (float*)take(adapter_t_bytes(M, r, n));
    u32x4* halves = (u32x4*)take(adapter_halves_bytes(M, r, n));
    u32x4* turned_u = (u32x4*)take(adapter_turned_bytes(M, r, n));
    u32x4* turned_t = (u32x4*)take(adapter_turned_bytes(M, r, n));
    float* part_a = (float*)take(adapter_partial_bytes(M, r, d_in));
    float* part_b = (float*)take(adapter_partial_bytes(M, r, d_out));
    const int target = adapter_target(r, 2);  // also without dB: a gradient has the same bits whichever others are asked for
    const AdapterShrink t{(const bf16*)X, (const bf16*)A, false, scale, T, d_in};
    const AdapterShrink u{(const bf16*)dY, (const bf16*)B, true, scale, U, d_out};
    const AdapterFinish done_u{U, dX ? halves : nullptr, dA ? turned_u : nullptr, d_out}, done_t{T, nullptr, turned_t, d_in};
    if (launch_shrink(u, dB ? &t : nullptr, p, M, n, r, target, st) != hipSuccess ||
        launch_finish(done_u, dB ? &done_t : nullptr, p, M, n, r, target, st) != hipSuccess)
        return PIFA_ERR_HIP;
    if (dX && launch_expand<false, true>({U, halves, (const bf16*)A, (const bf16*)dX0, (bf16*)dX, d_in, d_out}, p, M, n, r, target, st) != hipSuccess)
        return PIFA_ERR_HIP;
    if (!dA && !dB) return PIFA_OK;
    const AdapterGrads ga{(const bf16*)X, turned_u, dA, part_a, d_in, false};
    const AdapterGrads gb{(const bf16*)dY, turned_t, dB, part_b, d_out, true};
    {
        TimedLaunch timed(kSiteAdapterGrads, st);
        const int64_t rp = adapter_rp(r), jb = std::min<int64_t>(4, rp / 16);
        const int64_t b0 = dA ? ceil_div(d_in, kAdCols) : 0, b1 = dB ? ceil_div(d_out, kAdCols) : 0;
        const dim3 grid((unsigned)(b0 + b1), (unsigned)adapter_max_pieces(M, n), (unsigned)ceil_div(rp, 16 * jb));
        if (jb == 1) hipLaunchKernelGGL((adapter_grads<1>), grid, dim3(kAdGradThreads), 0, st, ga, gb, (int)b0, p, M, (int)n, r);
        else if (jb == 2) hipLaunchKernelGGL((adapter_grads<2>), grid, dim3(kAdGradThreads), 0, st, ga, gb, (int)b0, p, M, (int)n, r);
        else hipLaunchKernelGGL((adapter_grads<4>), grid, dim3(kAdGradThreads), 0, st, ga, gb, (int)b0, p, M, (int)n, r);
        if (hipGetLastError() != hipSuccess) return PIFA_ERR_HIP;
    }
    if (M > kAdPiece) {
        TimedLaunch timed(kSiteAdapterSums, st);
        const int64_t n0 = dA ? r * d_in : 0, n1 = dB ? r * d_out : 0, b0 = ceil_div(n0, 1024);
        hipLaunchKernelGGL(adapter_sum, dim3((unsigned)(b0 + ceil_div(n1, 1024)), (unsigned)std::min(n, M / kAdPiece)),
                           dim3(256), 0, st, part_a, dA, n0, (int)b0, part_b, dB, n1, p, M, (int)n);
        if (hipGetLastError() != hipSuccess) return PIFA_ERR_HIP;
    }
    return PIFA_OK;
}

pifa_status adamw_create(const adamw_tensor* tensors, int64_t count, int state_bits, pifa_dtype g_dtype, uint32_t seed,
                         adamw_handle* out) {
    if (!out) return PIFA_ERR_INVALID_ARG;
    *out = nullptr;
    try {
        int64_t chunks = 0;
        const pifa_status s = adamw_check(tensors, count, state_bits, g_dtype, &chunks);
        if (s != PIFA_OK) return s;
        // count, tensors, chunks
        const size_t at_tensors = 256, at_chunks = (size_t)round_up(at_tensors + count * (int64_t)sizeof(AdamwTensor), 256);
        std::vector<uint8_t> image(at_chunks + (size_t)chunks * sizeof(AdamwChunk), 0);
        AdamwTensor* T = reinterpret_cast<AdamwTensor*>(image.data() + at_tensors);
        AdamwChunk* C = reinterpret_cast<AdamwChunk*>(image.data() + at_chunks);
        for (int64_t i = 0; i < count; ++i) {
            const adamw_tensor& t = tensors[i];
            T[i] = AdamwTensor{t.p, t.g, t.m, t.v, t.m_scale, t.v_scale, (bf16*)t.p_bf16, t.n, t.weight_decay};
            for (int64_t k = 0; k < ceil_div(t.n, kAdamwChunk); ++k) *C++ = AdamwChunk{(int32_t)i, (uint32_t)k};
        }
        adamw_state* h = new (std::nothrow) adamw_state();
        if (!h) return PIFA_ERR_OOM;
        h->bits = state_bits;
        h->g_dtype = g_dtype;
        h->seed = seed;
        h->chunks = chunks;
        pifa_status e = PIFA_OK;
        if (hipGetDevice(&h->device) != hipSuccess || hipDeviceSynchronize() != hipSuccess) e = PIFA_ERR_HIP;
        else if (hipMalloc(&h->memory, image.size()) != hipSuccess) {
            (void)hipGetLastError();
            e = PIFA_ERR_OOM;
        } else if (hipMemcpy(h->memory, image.data(), image.size(), hipMemcpyHostToDevice) != hipSuccess) {
            e = PIFA_ERR_HIP;
        }
        if (e != PIFA_OK) {
            free_adamw(h);
            return e;
        }
        h->count = (AdamwStep*)h->memory;
        h->tensors = (AdamwTensor*)((uint8_t*)h->memory + at_tensors);
        h->table = (AdamwChunk*)((uint8_t*)h->memory + at_chunks);
        *out = h;
        return PIFA_OK;
    } catch (const std::bad_alloc&) {
        return PIFA_ERR_OOM;
    }
}

pifa_status adamw_destroy(adamw_handle h) {
    if (!h) return PIFA_OK;
    (void)hipDeviceSynchronize();
    free_adamw(h);
    return PIFA_OK;
}

pifa_status adamw_count(adamw_handle h, int64_t* steps) {
    if (!h || !steps) return PIFA_ERR_INVALID_ARG;
    PIFA_ON_DEVICE(h->device);
    PIFA_HIP(hipDeviceSynchronize());
    PIFA_HIP(hipMemcpy(steps, &h->count->t, sizeof(int64_t), hipMemcpyDeviceToHost));
    return PIFA_OK;
}

pifa_status adamw_step(adamw_handle h, double lr, double beta1, double beta2, double eps, int64_t step,
                       const float* grad_scale, void* stream) {
    if (!h || !(lr >= 0.0) || std::isinf(lr) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) ||
        !((float)eps >= 0x1p-126f) || std::isinf((float)eps) || step < 0)
        return PIFA_ERR_INVALID_ARG;
    if ((uintptr_t)grad_scale % 4 != 0) return PIFA_ERR_UNSUPPORTED;
    PIFA_ON_DEVICE(h->device);
    const hipStream_t st = as_stream(stream);
    if (step == 0 || h->chunks == 0) {
        hipLaunchKernelGGL(adamw_tick, dim3(1), dim3(1), 0, st, h->count, step, lr, beta1, beta2);
        if (hipGetLastError() != hipSuccess) return PIFA_ERR_HIP;
    }
    if (h->chunks == 0) return PIFA_OK;
    AdamwArgs a{};
    a.tensors = h->tensors;
    a.chunks = h->table;
    a.count = h->count;
    a.step.t = step;
    if (step > 0) {
        a.step.rate = (float)(lr / (1.0 - std::pow(beta1, (double)step)));
        a.step.root = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
    }
    a.grad_scale = grad_scale;
    a.lr = lr;
    a.b1 = (float)beta1;
    a.c1 = (float)(1.0 - beta1);
    a.b2 = (float)beta2;
    a.c2 = (float)(1.0 - beta2);
    a.eps = (float)eps;
    a.seed = h->seed;
    TimedLaunch timed(kSiteAdamw, st);
    const dim3 grid((unsigned)h->chunks), block(kAdamwThreads);
    if (h->bits == 8) {
        if (h->g_dtype == PIFA_BF16) hipLaunchKernelGGL((adamw_update<true, bf16>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((adamw_update<true, float>), grid, block, 0, st, a);
    } else {
        if (h->g_dtype == PIFA_BF16) hipLaunchKernelGGL((adamw_update<false, bf16>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((adamw_update<false, float>), grid, block, 0, st, a);
    }
    return hipGetLastError() == hipSuccess ? PIFA_OK : PIFA_ERR_HIP;
}

}  // extern "C"
