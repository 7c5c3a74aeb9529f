// Root-mean-square norm of the rows a layer reads, with the residual's
// addition, and its gradients.
//
//   h = x + r,   rho = (mean_k h_k^2 + eps)^-1/2,   y_k = h_k rho g_k
//   u = g dy,    dx = rho u - h rho^3 mean_k(u_k h_k) + dr,   dg = sum over rows of dy h rho
//
// Both are bound by memory: every operand is read once and every result
// written once, in 16-byte pieces ("chunks"; rows of any length and alignment,
// the hardware takes unaligned ones), and a row stays in registers between its
// sums and its results.  TPR threads share a row, V chunks each, dealt so that
// neighbouring threads hold neighbouring chunks.  Sums, rho and the quotient
// are fp32; each result is rounded once, from the unrounded h.
//
// Measured, calls in a row, both launches of the gradients: X, R, H and Y of 4096
// rows of 8192 in bf16 47 to 48 us, 5.6 TB/s (a copy of 1 GiB: 5.2), in fp32 97
// us, 5.5 TB/s.  The gradients of 4096 x 4096 31 us (4.3 TB/s), of 8192 x 8192
// 103 us (5.2 TB/s).  One row of 4096 takes 2.7 us, one of 64 2.3: a launch (in a
// trace the kernel of the former is 2.2).
#pragma once

#include <type_traits>

#include "common.hpp"

namespace pifa {

constexpr int kNormThreads = 1024;     // of a workgroup in the wide forms
constexpr float kE4m3Max = 448.f;      // largest e4m3 value
constexpr float kE4m3Tiny = 0x1p-126f; // smallest row scale: its inverse is finite

// The full chunks of a row; the d % N elements behind them are handled one
// per thread, which costs rows of whole chunks a uniform branch.
template <typename T>
struct NormChunk {
    static constexpr int N = 16 / (int)sizeof(T);
    struct __attribute__((packed, aligned(sizeof(T)))) Any {
        u32x4 v;
    };
    __device__ __forceinline__ static u32x4 load(const T* row, int64_t c, int64_t full) {
        u32x4 v = zero16();
        if (c < full) v = reinterpret_cast<const Any*>(row + c * N)->v;
        return v;
    }
    __device__ __forceinline__ static float one(u32x4 raw, int e) {
        const uint32_t w = raw[sizeof(T) == 4 ? e : e / 2];
        if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, w);
        else return bf16_bits_to_f32((uint16_t)(w >> (16 * (e & 1))));
    }
    __device__ __forceinline__ static void floats(u32x4 raw, float (&v)[N]) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = one(raw, e);
    }
    __device__ __forceinline__ static void store(T* row, int64_t c, int64_t full, const float (&v)[N]) {
        T out[N];
#pragma unroll
        for (int e = 0; e < N; ++e) out[e] = (T)v[e];
        if (c < full) reinterpret_cast<Any*>(row + c * N)->v = __builtin_bit_cast(u32x4, out);
    }
    // N e4m3 bytes
    __device__ __forceinline__ static void store_e4m3(uint8_t* row, int64_t c, int64_t full, const float (&v)[N]) {
        struct __attribute__((packed, aligned(1))) Bytes {
            uint32_t w[N / 4];
        };
        Bytes b;
#pragma unroll
        for (int e = 0; e < N; e += 4) {
            const int q = __builtin_amdgcn_cvt_pk_fp8_f32(v[e], v[e + 1], 0, false);
            b.w[e / 4] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[e + 2], v[e + 3], q, true);
        }
        if (c < full) *reinterpret_cast<Bytes*>(row + c * N) = b;
    }
};
// Quotients by a row's scale: the product with its reciprocal, corrected by what
// that leaves.  Before its rounding to fp32 it is within 2^-46 of the quotient, so
// that midpoints of two e4m3 values are met as a division meets them (1999 rows
// of 4096: divided 13.6 us, corrected 12.2, the product alone 11.8).
struct E4m3Scale {
    float s, inv;
    __device__ __forceinline__ explicit E4m3Scale(float scale)
        : s(scale <= 3.402823466e38f ? scale : 0.f), inv(1.f / scale) {}  // an infinite one: y * 0
    __device__ __forceinline__ float operator()(float y) const {
        const float q = y * inv;
        return __builtin_fmaf(__builtin_fmaf(-q, s, y), inv, q);
    }
};
__device__ __forceinline__ uint8_t to_e4m3(float v) {
    return (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(v, v, 0, false);
}

// a > b or NaN: a maximum that a NaN survives
__device__ __forceinline__ float max_or_nan(float a, float b) { return (a > b || a != a) ? a : b; }

// Sum (or maximum) of one value over the TPR threads of each row, in a fixed
// order.  `red` holds one float per wave; two calls in a row need two arrays.
template <int TPR, bool MAX = false>
__device__ __forceinline__ float row_reduce(float v, float* red) {
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) {
        const float o = __shfl_xor(v, s);
        v = MAX ? max_or_nan(v, o) : v + o;
    }
    if constexpr (TPR > kWave) {
        constexpr int W = TPR / kWave;
        const int wave = threadIdx.x / kWave;
        if ((threadIdx.x & (kWave - 1)) == 0) red[wave] = v;
        __syncthreads();
        const int w0 = wave / W * W;
        v = red[w0];
#pragma unroll
        for (int w = 1; w < W; ++w) v = MAX ? max_or_nan(v, red[w0 + w]) : v + red[w0 + w];
    }
    return v;
}

// What the forward writes: rows of T, e4m3 rows with scales, or rows of T with
// what their rounding left in rows of their own (a product that adds both
// loses nothing).
enum NormOut : int { kNormSame = 0, kNormE4m3 = 1, kNormSplit = 2 };

template <typename T>
struct NormFwd {
    const T* X;
    const T* R;     // or null
    const T* gain;  // or null: ones
    T* H;           // or null; may be X or R
    T* Y;           // bf16 / fp32 rows (may be X or R), or
    uint8_t* Q;     // e4m3 rows with
    float* scale;   // a scale each
    T* left;        // kNormSplit: Y less its rounded values
    int64_t M, d;
    float eps;
};

// y as two bf16 values: hi next to it (at most the largest bf16, so that a y that
// would round to infinity is not one), lo next to what that leaves: an infinity
// or a NaN is in lo.
struct NormPair {
    bf16 hi, lo;
    __device__ __forceinline__ explicit NormPair(float y)
        : hi((bf16)__builtin_amdgcn_fmed3f(y, -0x1.FEp127f, 0x1.FEp127f)), lo((bf16)(y - (float)hi)) {}
};

// A chunk of both rows of kNormSplit.
template <typename T>
__device__ __forceinline__ void norm_store_pairs(const NormFwd<T>& p, int64_t row, int64_t c, int64_t full,
                                                 float (&y)[NormChunk<T>::N]) {
    float lo[NormChunk<T>::N];
#pragma unroll
    for (int e = 0; e < NormChunk<T>::N; ++e) {
        const NormPair v(y[e]);
        y[e] = (float)v.hi;
        lo[e] = (float)v.lo;
    }
    NormChunk<T>::store(p.Y + row, c, full, y);
    NormChunk<T>::store(p.left + row, c, full, lo);
}

// ROWS rows of at most TPR * V full chunks per workgroup.
template <typename T, int OUT, int TPR, int V, int ROWS>
__global__ __launch_bounds__(TPR* ROWS) void norm_fwd(NormFwd<T> p) {
    using C = NormChunk<T>;
    constexpr int N = C::N;
    constexpr bool E4M3 = OUT == kNormE4m3;
    __shared__ float red[2][TPR * ROWS / kWave];
    const int t = threadIdx.x % TPR;
    const int64_t m = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR;
    const bool live = m < p.M;
    const int64_t row = (live ? m : 0) * p.d;
    const int64_t full = live ? p.d / N : 0;  // rows past M: nothing is loaded or stored
    const int64_t kt = p.d / N * N + t;       // this thread's element behind the full chunks
    const bool tail = live && t < N && kt < p.d;

    float h[V][N], ht = 0.f, gt = 1.f;
    u32x4 x[V], r[V], g[V];
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = C::load(p.X + row, t + i * TPR, full);
    if (p.R) {
#pragma unroll
        for (int i = 0; i < V; ++i) r[i] = C::load(p.R + row, t + i * TPR, full);
    }
    if (p.gain) {
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = C::load(p.gain, t + i * TPR, full);
    }
    if (tail) {
        ht = (float)p.X[row + kt];
        if (p.R) ht += (float)p.R[row + kt];
        if (p.gain) gt = (float)p.gain[kt];
    }
    float ss = ht * ht;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        C::floats(x[i], h[i]);
        if (p.R) {
#pragma unroll
            for (int e = 0; e < N; ++e) h[i][e] += C::one(r[i], e);
        }
#pragma unroll
        for (int e = 0; e < N; ++e) ss += h[i][e] * h[i][e];
    }
    if (p.H) {
#pragma unroll
        for (int i = 0; i < V; ++i) C::store(p.H + row, t + i * TPR, full, h[i]);
        if (tail) p.H[row + kt] = (T)ht;
    }
    const float rho = rsqrtf(row_reduce<TPR>(ss, red[0]) / (float)p.d + p.eps);
    ht *= rho * gt;
    float amax = fabsf(ht);
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            h[i][e] *= rho;
            if (p.gain) h[i][e] *= C::one(g[i], e);
            if constexpr (E4M3) amax = max_or_nan(fabsf(h[i][e]), amax);
        }
        if constexpr (OUT == kNormSame) C::store(p.Y + row, t + i * TPR, full, h[i]);
        if constexpr (OUT == kNormSplit) norm_store_pairs<T>(p, row, t + i * TPR, full, h[i]);
    }
    if constexpr (OUT == kNormSame) {
        if (tail) p.Y[row + kt] = (T)ht;
    } else if constexpr (OUT == kNormSplit) {
        if (tail) {
            const NormPair y(ht);
            p.Y[row + kt] = y.hi;
            p.left[row + kt] = y.lo;
        }
    } else {
        const float s = max_or_nan(row_reduce<TPR, true>(amax, red[1]) / kE4m3Max, kE4m3Tiny);
        const E4m3Scale by(s);
#pragma unroll
        for (int i = 0; i < V; ++i) {
#pragma unroll
            for (int e = 0; e < N; ++e) h[i][e] = by(h[i][e]);
            C::store_e4m3(p.Q + row, t + i * TPR, full, h[i]);
        }
        if (tail) p.Q[row + kt] = to_e4m3(by(ht));
        if (live && t == 0) p.scale[m] = s;
    }
}

// Rows too long for a workgroup's registers are read again for the results
// (and for the maximum of 8-bit rows).  H or Y may be X or R: a thread stores
// only elements that it alone reads, after its last read of them.
template <typename T, int OUT>
__global__ __launch_bounds__(kNormThreads) void norm_fwd_long(NormFwd<T> p) {
    using C = NormChunk<T>;
    constexpr int N = C::N;
    constexpr bool E4M3 = OUT == kNormE4m3;
    __shared__ float red[2][kNormThreads / kWave];
    const int64_t row = (int64_t)blockIdx.x * p.d;
    const int64_t full = p.d / N, kt = full * N + threadIdx.x;
    const bool tail = threadIdx.x < N && kt < p.d;
    auto sum = [&](int64_t c, float(&h)[N]) {
        C::floats(C::load(p.X + row, c, full), h);
        if (p.R) {
            const u32x4 r = C::load(p.R + row, c, full);
#pragma unroll
            for (int e = 0; e < N; ++e) h[e] += C::one(r, e);
        }
    };
    float ht = 0.f;
    if (tail) ht = (float)p.X[row + kt] + (p.R ? (float)p.R[row + kt] : 0.f);
    float ss = ht * ht;
    for (int64_t c = threadIdx.x; c < full; c += kNormThreads) {
        float h[N];
        sum(c, h);
#pragma unroll
        for (int e = 0; e < N; ++e) ss += h[e] * h[e];
    }
    const float rho = rsqrtf(row_reduce<kNormThreads>(ss, red[0]) / (float)p.d + p.eps);
    if (tail && p.H) p.H[row + kt] = (T)ht;
    ht *= rho * (tail && p.gain ? (float)p.gain[kt] : 1.f);
    auto norm = [&](int64_t c, const float(&h)[N], float(&y)[N]) {
        u32x4 g = zero16();
        if (p.gain) g = C::load(p.gain, c, full);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            y[e] = h[e] * rho;
            if (p.gain) y[e] *= C::one(g, e);
        }
    };
    E4m3Scale by(1.f);
    if constexpr (E4M3) {
        float amax = fabsf(ht);
        for (int64_t c = threadIdx.x; c < full; c += kNormThreads) {
            float h[N], y[N];
            sum(c, h);
            norm(c, h, y);
#pragma unroll
            for (int e = 0; e < N; ++e) amax = max_or_nan(fabsf(y[e]), amax);
        }
        const float s = max_or_nan(row_reduce<kNormThreads, true>(amax, red[1]) / kE4m3Max, kE4m3Tiny);
        by = E4m3Scale(s);
        if (threadIdx.x == 0) p.scale[blockIdx.x] = s;
        if (tail) p.Q[row + kt] = to_e4m3(by(ht));
    } else {
        if constexpr (OUT == kNormSplit) {
            if (tail) {
                const NormPair y(ht);
                p.Y[row + kt] = y.hi;
                p.left[row + kt] = y.lo;
            }
        } else if (tail) {
            p.Y[row + kt] = (T)ht;
        }
    }
    for (int64_t c = threadIdx.x; c < full; c += kNormThreads) {
        float h[N], y[N];
        sum(c, h);
        norm(c, h, y);
        if (p.H) C::store(p.H + row, c, full, h);
        if constexpr (E4M3) {
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] = by(y[e]);
            C::store_e4m3(p.Q + row, c, full, y);
        } else {
            if constexpr (OUT == kNormSplit) norm_store_pairs<T>(p, row, c, full, y);
            else C::store(p.Y + row, c, full, y);
        }
    }
}

template <typename T>
struct NormBwd {
    const T* H;
    const T* gain;  // or null: ones
    const T* dY;
    const T* dR;    // or null: nothing flows in beside the norm
    T* dX;          // or null; may be H, dY or dR
    float* dgain;   // or null: per workgroup partial sums at dgain + blockIdx.x * d
    int64_t M, d;
    float eps;
};

// rho^2 mean(u h): rho^2 alone may leave fp32's range, and u h may where rho is 0
// (a row whose squares overflow).
__device__ __forceinline__ float norm_back(float rho, float uh, float d) {
    float q = rho * (uh / d);
    asm volatile("" : "+v"(q));  // a select, not a branch around the division (rows of 16384: 2%)
    return rho * (rho == 0.f ? 0.f : q);
}

// Sums of two values over the TPR threads of each row, one barrier for both.
template <int TPR>
__device__ __forceinline__ float2 row_sum2(float a, float b, float2* red) {
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) {
        a += __shfl_xor(a, s);
        b += __shfl_xor(b, s);
    }
    if constexpr (TPR > kWave) {
        constexpr int W = TPR / kWave;
        const int wave = threadIdx.x / kWave;
        if ((threadIdx.x & (kWave - 1)) == 0) red[wave] = float2{a, b};
        __syncthreads();
        const int w0 = wave / W * W;
        a = red[w0].x;
        b = red[w0].y;
#pragma unroll
        for (int w = 1; w < W; ++w) {
            a += red[w0 + w].x;
            b += red[w0 + w].y;
        }
    }
    return float2{a, b};
}

// A workgroup takes ROWS rows at a time, rows ROWS * blockIdx.x + i * ROWS *
// gridDim.x, and keeps the gain's gradient of the columns its threads hold in
// registers over all of them; at the end the ROWS sums of a column are added
// in LDS, so that only gridDim.x partial sums per column go to memory.  The
// next rows' operands are loaded before the current ones' sums are reduced, in
// two sets of registers in turn.
// EXACT: rows are TPR * V full chunks and have a residual gradient and a dX, so
// that no load or store stands under a condition (behind one, the wait for a
// row's operands would be a wait for its successor's too).
template <typename T, int TPR, int V, bool EXACT>
__global__ __launch_bounds__(kNormThreads) void norm_bwd(NormBwd<T> p) {
    using C = NormChunk<T>;
    constexpr int N = C::N;
    constexpr int ROWS = kNormThreads / TPR;
    __shared__ float2 red[2][kNormThreads / kWave];
    __shared__ float cols[ROWS > 1 ? kNormThreads * (V * N + 1) : 1];
    const int t = threadIdx.x % TPR, rg = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
    const int64_t step = (int64_t)gridDim.x * ROWS, nfull = EXACT ? TPR * V : p.d / N, kt = nfull * N + t;
    const bool has_tail = !EXACT && t < N && kt < p.d, add = EXACT || (p.dR && p.dX);

    float dg[V][N], dgt = 0.f;
    u32x4 g[V];
    float gt = 1.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        g[i] = zero16();
        if (p.gain) g[i] = C::load(p.gain, t + i * TPR, nfull);
#pragma unroll
        for (int e = 0; e < N; ++e) dg[i][e] = 0.f;
    }
    if (p.gain && has_tail) gt = (float)p.gain[kt];
    auto gain = [&](int i, int e) { return p.gain ? C::one(g[i], e) : 1.f; };

    struct Rows {
        u32x4 h[V], y[V], r[V];
        float ht, yt, rt;
    };
    // ALL: no row past M is among them (where a workgroup takes one row at a
    // time, none ever is).  A row past M is zeros and reads nothing: the rows
    // before it may be other waves', which store dX over them meanwhile.
    auto fetch = [&](auto all, int64_t m, Rows& f) {
        constexpr bool ALL = EXACT && (ROWS == 1 || decltype(all)::value);
        const bool live = ALL || m < p.M;
        const int64_t row = (live ? m : 0) * p.d, full = live ? nfull : 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int64_t c = t + i * TPR;
            if constexpr (ALL) {  // c < nfull is known
                f.h[i] = reinterpret_cast<const typename C::Any*>(p.H + row + c * N)->v;
                f.y[i] = reinterpret_cast<const typename C::Any*>(p.dY + row + c * N)->v;
                f.r[i] = reinterpret_cast<const typename C::Any*>(p.dR + row + c * N)->v;
            } else {
                f.h[i] = C::load(p.H + row, c, full);
                f.y[i] = C::load(p.dY + row, c, full);
                if (add) f.r[i] = C::load(p.dR + row, c, full);
            }
        }
        f.ht = f.yt = f.rt = 0.f;
        if (live && has_tail) {
            f.ht = (float)p.H[row + kt];
            f.yt = (float)p.dY[row + kt];
            if (add) f.rt = (float)p.dR[row + kt];
        }
    };
    int par = 0;
    // LAST: rows past M may be among them
    auto rows = [&](auto last, int64_t m, Rows& cur) {
        constexpr bool LAST = decltype(last)::value || !EXACT;
        const bool live = !LAST || m < p.M;
        float ss = cur.ht * cur.ht, uh = gt * cur.yt * cur.ht;
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                // written-out fused steps: every form of this kernel gives the same bits
                const float h = C::one(cur.h[i], e);
                ss = __builtin_fmaf(h, h, ss);
                uh = __builtin_fmaf(gain(i, e) * C::one(cur.y[i], e), h, uh);
            }
        const float2 sums = row_sum2<TPR>(ss, uh, red[par]);
        par ^= 1;
        const float rho = rsqrtf(sums.x / (float)p.d + p.eps);
        const float back = norm_back(rho, sums.y, (float)p.d);
        const int64_t row = live ? m * p.d : 0, full = live ? nfull : 0;
        // the second reading of the row's registers converts them again: kept
        // from the first one, the fp32 values do not fit 128 registers (of bf16
        // rows of two chunks a thread 8 to 14 are spilled all the same)
#pragma unroll
        for (int i = 0; i < V; ++i) asm volatile("" : "+v"(cur.h[i]), "+v"(cur.y[i]), "+v"(g[i]));
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float dx[N];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float h = C::one(cur.h[i], e), y = C::one(cur.y[i], e);
                dg[i][e] = __builtin_fmaf(h * rho, y, dg[i][e]);
                dx[e] = rho * (gain(i, e) * y - h * back);
                if (add) dx[e] += C::one(cur.r[i], e);
            }
            if constexpr (EXACT && !LAST) C::store(p.dX + row, t + i * TPR, TPR * V, dx);
            else if (p.dX) C::store(p.dX + row, t + i * TPR, full, dx);
        }
        dgt = __builtin_fmaf(cur.ht * rho, cur.yt, dgt);
        if (live && has_tail && p.dX) p.dX[row + kt] = (T)(rho * (gt * cur.yt - cur.ht * back) + cur.rt);
    };
    const int64_t first = (int64_t)blockIdx.x * ROWS;
    Rows even, odd;
    fetch(std::false_type{}, first + rg, even);
    int64_t m0 = first;  // uniform over the workgroup
    for (; EXACT && m0 + 2 * step + ROWS <= p.M; m0 += 2 * step) {
        fetch(std::true_type{}, m0 + step + rg, odd);
        __builtin_amdgcn_sched_barrier(0);
        rows(std::false_type{}, m0 + rg, even);
        fetch(std::true_type{}, m0 + 2 * step + rg, even);
        __builtin_amdgcn_sched_barrier(0);
        rows(std::false_type{}, m0 + step + rg, odd);
    }
    for (; m0 < p.M; m0 += step) {  // EXACT: at most three, the last of them perhaps cut
        const bool more = m0 + step < p.M;
        if (more) fetch(std::false_type{}, m0 + step + rg, odd);
        rows(std::true_type{}, m0 + rg, even);
        if (more) even = odd;
    }
    if (!p.dgain) return;
    float* out = p.dgain + (int64_t)blockIdx.x * p.d;
    if constexpr (ROWS > 1) {
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) cols[(i * N + e) * kNormThreads + threadIdx.x] = dg[i][e];
        cols[V * N * kNormThreads + threadIdx.x] = dgt;
        __syncthreads();
        // column j: element j % N of chunk j / N, or a tail element
        for (int j = threadIdx.x; j < p.d; j += kNormThreads) {
            const int c = j / N;
            const float* from = c < nfull ? cols + ((c / TPR) * N + j % N) * kNormThreads + c % TPR
                                          : cols + V * N * kNormThreads + j % N;
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < ROWS; ++w) s += from[w * TPR];
            out[j] = s;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int64_t c = t + i * TPR;
                if (c < nfull) out[c * N + e] = dg[i][e];
            }
        if (has_tail) out[kt] = dgt;
    }
}

// Rows too long for registers: a second pass over each row, and the partial
// sums of the gain's gradient kept in memory (each thread reads and writes
// its own columns only).
template <typename T>
__global__ __launch_bounds__(kNormThreads) void norm_bwd_long(NormBwd<T> p) {
    using C = NormChunk<T>;
    constexpr int N = C::N;
    __shared__ float red[2][2][kNormThreads / kWave];
    const int64_t full = p.d / N, kt = full * N + threadIdx.x;
    const bool tail = threadIdx.x < N && kt < p.d;
    float* out = p.dgain ? p.dgain + (int64_t)blockIdx.x * p.d : nullptr;
    const float gt = tail && p.gain ? (float)p.gain[kt] : 1.f;
    auto load = [&](int64_t row, int64_t c, float(&h)[N], float(&y)[N], float(&g)[N]) {
        C::floats(C::load(p.H + row, c, full), h);
        C::floats(C::load(p.dY + row, c, full), y);
        if (p.gain) C::floats(C::load(p.gain, c, full), g);
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (!p.gain) g[e] = 1.f;
    };
    int par = 0;
    for (int64_t m = blockIdx.x; m < p.M; m += gridDim.x, par ^= 1) {
        const int64_t row = m * p.d;
        const float ht = tail ? (float)p.H[row + kt] : 0.f, yt = tail ? (float)p.dY[row + kt] : 0.f;
        float ss = ht * ht, uh = gt * yt * ht;
        for (int64_t c = threadIdx.x; c < full; c += kNormThreads) {
            float h[N], y[N], g[N];
            load(row, c, h, y, g);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                ss += h[e] * h[e];
                uh += g[e] * y[e] * h[e];
            }
        }
        ss = row_reduce<kNormThreads>(ss, red[par][0]);
        uh = row_reduce<kNormThreads>(uh, red[par][1]);
        const float rho = rsqrtf(ss / (float)p.d + p.eps);
        const float back = norm_back(rho, uh, (float)p.d);
        const bool begun = m != blockIdx.x;
        for (int64_t c = threadIdx.x; c < full; c += kNormThreads) {
            float h[N], y[N], g[N], dx[N];
            load(row, c, h, y, g);
            if (out) {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float v = h[e] * rho * y[e];
                    out[c * N + e] = begun ? out[c * N + e] + v : v;
                }
            }
            if (p.dX) {
                u32x4 r = zero16();
                if (p.dR) r = C::load(p.dR + row, c, full);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    dx[e] = rho * (g[e] * y[e] - h[e] * back);
                    if (p.dR) dx[e] += C::one(r, e);
                }
                C::store(p.dX + row, c, full, dx);
            }
        }
        if (tail) {
            if (out) out[kt] = begun ? out[kt] + ht * rho * yt : ht * rho * yt;
            if (p.dX) p.dX[row + kt] = (T)(rho * (gt * yt - ht * back) + (p.dR ? (float)p.dR[row + kt] : 0.f));
        }
    }
}

// dgain = the sum of P <= 256 partial rows of d, in a fixed order: a workgroup
// of 16 x 64 threads takes 64 columns; a thread's loads are all in flight.
constexpr int kNormMaxGroups = 256;
__global__ __launch_bounds__(kNormThreads) void norm_dgain(const float* __restrict__ part, int P, int64_t d,
                                                          float* __restrict__ dgain) {
    constexpr int SLICES = kNormThreads / kWave, EACH = kNormMaxGroups / SLICES;
    __shared__ float red[kNormThreads];
    const int64_t k = (int64_t)blockIdx.x * kWave + (threadIdx.x & (kWave - 1));
    const int slice = threadIdx.x / kWave;
    float v[EACH], s = 0.f;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int q = slice + i * SLICES;
        v[i] = part[(int64_t)(q < P ? q : 0) * d + (k < d ? k : 0)];
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) s += slice + i * SLICES < P ? v[i] : 0.f;
    red[threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.x < kWave && k < d) {
#pragma unroll
        for (int w = 1; w < SLICES; ++w) s += red[w * kWave + threadIdx.x];
        dgain[k] = s;
    }
}

// dgain of no rows (a fill kernel: a captured graph may hold it)
__global__ void norm_zero(float* p, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) p[i] = 0.f;
}

}  // namespace pifa
