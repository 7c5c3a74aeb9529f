// Layer norm of the rows a layer reads, with the residual's addition, and its
// gradients.
//
//   h = x + r,   c_k = h_k - mean(h),   rho = (mean_k c_k^2 + eps)^-1/2,   y_k = c_k rho g_k + b_k
//   u = g dy,    hat = c rho,   dx = rho (u - mean(u) - hat mean(u hat)) + dr
//   dg = sum over rows of dy hat,   db = sum over rows of dy
//
// Bound by memory, and laid out like the root-mean-square norm: a row stays in
// the registers of TPR threads, V 16-byte chunks each, between its sums and its
// results.  The squares are summed after the mean is taken off, in a second
// reduction: a sum of squares less the squared mean would lose the digits that
// rows far from zero share.  A rounded mean is itself off by the last bits of the
// row's size, which rho makes large where a row hardly varies (4096 values of 1000.1:
// hat up to 0.04 in place of 0).  So the second reduction also sums the c_k, whose
// mean is what the first one missed: it is taken off c, and its square off the mean
// of the squares.  Sums, mean and rho are fp32; each result is rounded once, from
// the unrounded h.
#pragma once

#include "norm.hpp"
#include "streamed.hpp"

namespace pifa {

// Of c with a mean of `off` that is still in it; NaN stays NaN.
__device__ __forceinline__ float layer_norm_rho(float ss, float off, float d, float eps) {
    const float var = __builtin_fmaf(-off, off, ss / d);
    return rsqrtf((var < 0.f ? 0.f : var) + eps);
}

// The value of another lane of the 16 around this one.
template <int CTRL>
__device__ __forceinline__ float layer_norm_dpp(float v) {
    const int i = __builtin_bit_cast(int, v);
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, CTRL, 0xF, 0xF, false));
}

// Sums of up to four values over the TPR threads of each row, in a fixed order.  The
// four lanes of a quad take a value each, so that adding up over the wave, and
// then over the row's waves, is adding up one value.  `red` holds four floats a wave;
// two calls in a row need two arrays.
template <int TPR>
__device__ __forceinline__ float4 row_sum4(float a, float b, float c, float d, float* red) {
    constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kTurn4 = 0x124, kTurn8 = 0x128;  // quad_perm, row_ror
    constexpr int W = TPR / kWave;
    const int lane = threadIdx.x & (kWave - 1);
    const bool odd = lane & 1, high = lane & 2;
    const float ab = (odd ? b : a) + layer_norm_dpp<kSwap1>(odd ? a : b);
    const float cd = (odd ? d : c) + layer_norm_dpp<kSwap1>(odd ? c : d);
    float v = (high ? cd : ab) + layer_norm_dpp<kSwap2>(high ? ab : cd);
    v += layer_norm_dpp<kTurn4>(v);
    v += layer_norm_dpp<kTurn8>(v);
    v += __shfl_xor(v, 16);
    v += __shfl_xor(v, 32);
    if constexpr (W > 1) {
        const int wave = threadIdx.x / kWave;
        if (lane < 4) red[4 * wave + lane] = v;
        __syncthreads();
        v = red[4 * (wave / W * W + lane / 4 % W) + lane % 4];
        v += layer_norm_dpp<kTurn4>(v);
        if constexpr (W > 2) v += layer_norm_dpp<kTurn8>(v);
        if constexpr (W > 4) v += __shfl_xor(v, 16);
        if constexpr (W > 8) v += __shfl_xor(v, 32);
    }
    // the first four lanes': the others added up in another order
    auto of = [&](int k) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), k)); };
    return float4{of(0), of(1), of(2), of(3)};
}

template <typename T>
struct LayerNormFwd {
    const T* X;
    const T* R;     // or null
    const T* gain;  // or null: ones
    const T* bias;  // or null: zeros
    T* H;           // or null; may be X or R
    T* Y;           // may be X or R
    int64_t M, d;
    float eps;
};

// ROWS rows of at most TPR * V full chunks per workgroup.  4096 x 8192 bf16 with the
// residual 50.1 us, 5.4 TB/s.
template <typename T, int TPR, int V, int ROWS>
__global__ __launch_bounds__(TPR* ROWS) void layer_norm_fwd(LayerNormFwd<T> p) {
    using C = NormChunk<T>;
    constexpr int N = C::N;
    __shared__ float red[2][4 * TPR * ROWS / kWave];
    const int t = threadIdx.x % TPR;
    const int64_t m = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR;
    const bool live = m < p.M;
    const int64_t row = (live ? m : 0) * p.d;
    const int64_t full = live ? p.d / N : 0;  // rows past M: nothing is loaded or stored
    const int64_t kt = p.d / N * N + t;       // this thread's element behind the full chunks
    const bool tail = live && t < N && kt < p.d;

    float h[V][N], ht = 0.f, gt = 1.f, bt = 0.f;
    u32x4 x[V], r[V], g[V], b[V];
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
    if (p.bias) {
#pragma unroll
        for (int i = 0; i < V; ++i) b[i] = C::load(p.bias, t + i * TPR, full);
    }
    if (tail) {
        ht = (float)p.X[row + kt];
        if (p.R) ht += (float)p.R[row + kt];
        if (p.gain) gt = (float)p.gain[kt];
        if (p.bias) bt = (float)p.bias[kt];
    }
    float sum = ht;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        C::floats(x[i], h[i]);
        if (p.R) {
#pragma unroll
            for (int e = 0; e < N; ++e) h[i][e] += C::one(r[i], e);
        }
#pragma unroll
        for (int e = 0; e < N; ++e) sum += h[i][e];
    }
    if (p.H) {
#pragma unroll
        for (int i = 0; i < V; ++i) C::store(p.H + row, t + i * TPR, full, h[i]);
        if (tail) p.H[row + kt] = (T)ht;
    }
    const float mean = row_sum4<TPR>(sum, 0.f, 0.f, 0.f, red[0]).x / (float)p.d;
    ht = tail ? ht - mean : 0.f;
    float ss = ht * ht, sc = ht;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const bool in = t + i * TPR < full;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            h[i][e] = in ? h[i][e] - mean : 0.f;
            ss += h[i][e] * h[i][e];
            sc += h[i][e];
        }
    }
    const float4 again = row_sum4<TPR>(ss, sc, 0.f, 0.f, red[1]);
    const float off = again.y / (float)p.d, rho = layer_norm_rho(again.x, off, (float)p.d, p.eps);
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            h[i][e] = __builtin_fmaf(h[i][e], rho, -off * rho);
            if (p.gain) h[i][e] *= C::one(g[i], e);
            if (p.bias) h[i][e] += C::one(b[i], e);
        }
        C::store(p.Y + row, t + i * TPR, full, h[i]);
    }
    if (tail) p.Y[row + kt] = (T)((ht - off) * rho * gt + bt);
}

// Rows too long for a workgroup's registers are read again for each sum and for
// the results.  H or Y may be X or R: a thread stores only elements that it
// alone reads, after its last read of them.
template <typename T>
__global__ __launch_bounds__(kNormThreads) void layer_norm_fwd_long(LayerNormFwd<T> p) {
    using C = NormChunk<T>;
    constexpr int N = C::N;
    __shared__ float red[2][4 * kNormThreads / kWave];
    const int64_t row = (int64_t)blockIdx.x * p.d;
    const int64_t full = p.d / N, kt = full * N + threadIdx.x;
    const bool tail = threadIdx.x < N && kt < p.d;
    auto load = [&](int64_t c, float(&h)[N]) {
        C::floats(C::load(p.X + row, c, full), h);
        if (p.R) {
            const u32x4 r = C::load(p.R + row, c, full);
#pragma unroll
            for (int e = 0; e < N; ++e) h[e] += C::one(r, e);
        }
    };
    const float ht = tail ? (float)p.X[row + kt] + (p.R ? (float)p.R[row + kt] : 0.f) : 0.f;
    float sum = ht;
    for (int64_t c = threadIdx.x; c < full; c += kNormThreads) {
        float h[N];
        load(c, h);
#pragma unroll
        for (int e = 0; e < N; ++e) sum += h[e];
    }
    const float mean = row_sum4<kNormThreads>(sum, 0.f, 0.f, 0.f, red[0]).x / (float)p.d;
    const float ct = tail ? ht - mean : 0.f;
    float ss = ct * ct, sc = ct;
    for (int64_t c = threadIdx.x; c < full; c += kNormThreads) {
        float h[N];
        load(c, h);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float k = h[e] - mean;
            ss += k * k;
            sc += k;
        }
    }
    const float4 again = row_sum4<kNormThreads>(ss, sc, 0.f, 0.f, red[1]);
    const float off = again.y / (float)p.d, rho = layer_norm_rho(again.x, off, (float)p.d, p.eps);
    for (int64_t c = threadIdx.x; c < full; c += kNormThreads) {
        float h[N], y[N];
        load(c, h);
        u32x4 g = zero16(), b = zero16();
        if (p.gain) g = C::load(p.gain, c, full);
        if (p.bias) b = C::load(p.bias, c, full);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            y[e] = (h[e] - mean - off) * rho;
            if (p.gain) y[e] *= C::one(g, e);
            if (p.bias) y[e] += C::one(b, e);
        }
        if (p.H) C::store(p.H + row, c, full, h);
        C::store(p.Y + row, c, full, y);
    }
    if (tail) {
        if (p.H) p.H[row + kt] = (T)ht;
        p.Y[row + kt] = (T)((ct - off) * rho * (p.gain ? (float)p.gain[kt] : 1.f) + (p.bias ? (float)p.bias[kt] : 0.f));
    }
}

template <typename T>
struct LayerNormBwd {
    const T* H;
    const T* gain;  // or null: ones
    const T* dY;
    const T* dR;    // or null: nothing flows in beside the norm
    T* dX;          // or null; may be H, dY or dR
    float* dgain;   // or null: a workgroup's sums at dgain + blockIdx.x * stride
    float* dbias;   // or null, likewise
    int64_t stride;
    int64_t M, d;
    float eps;
};

// Adds a chunk's h to sh and its u = g y to su; of bf16 values two at a time, their
// products exact.
template <typename T>
__device__ __forceinline__ void layer_norm_sums_of(u32x4 h, u32x4 y, u32x4 g, bool gain, float& sh, float& su) {
    if constexpr (sizeof(T) == 2) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        const auto pair = [](uint32_t w) { return __builtin_bit_cast(bf16x2, w); };
        constexpr uint32_t ones = 0x3F803F80u;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            sh = __builtin_amdgcn_fdot2_f32_bf16(pair(h[k]), pair(ones), sh, false);
            su = __builtin_amdgcn_fdot2_f32_bf16(pair(y[k]), pair(gain ? g[k] : ones), su, false);
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            sh += NormChunk<T>::one(h, k);
            su = __builtin_fmaf(gain ? NormChunk<T>::one(g, k) : 1.f, NormChunk<T>::one(y, k), su);
        }
    }
}

// mean(u hat), where rho is 0 (a row whose squares sum past fp32) and the sum of
// u c may be infinite: 0.
__device__ __forceinline__ float layer_norm_back(float rho, float uc, float d) {
    float q = rho * (uc / d);
    asm volatile("" : "+v"(q));  // a select, not a branch around the division
    return rho == 0.f ? 0.f : q;
}

// A workgroup takes ROWS rows at a time, rows ROWS * blockIdx.x + i * ROWS *
// gridDim.x, and keeps the sums of dgain and dbias for the columns its threads
// hold in registers over all of them; at the end the ROWS sums of a column are
// added in LDS, so that only gridDim.x partial sums a column go to memory.
// 4096 x 4096 bf16 27.9 us (4.8 TB/s) and 4.6 for the partial sums; 333 x 2867 fp32,
// one or two rows a CU, 8.2 and 3.5: a row's loads and two reductions one after the
// other.
// EXACT: rows are TPR * V full chunks and have a residual gradient and a dX, so
// that no load or store stands under a condition.  With four chunks a thread (fp32
// rows past 8195 values) only H and dY are held beside the sums: gain and dR are
// loaded where they are used, chunk by chunk so that the registers suffice (2048 x
// 16384 in fp32 123 us, by the long form below 270; 1140 x 14704 without dR 58, 119;
// 300 x 10007 26, 40).
template <typename T, int TPR, int V, bool EXACT>
__global__ __launch_bounds__(kNormThreads) void layer_norm_bwd(LayerNormBwd<T> p) {
    using C = NormChunk<T>;
    constexpr int N = C::N;
    constexpr int ROWS = kNormThreads / TPR;
    constexpr bool HELD = V <= 2;  // gain and dR
    __shared__ float red[2][4 * kNormThreads / kWave];
    __shared__ float cols[ROWS > 1 ? kNormThreads * (V * N + 1) : 1];
    const int t = threadIdx.x % TPR, rg = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);
    const int64_t step = (int64_t)gridDim.x * ROWS, nfull = EXACT ? TPR * V : p.d / N, kt = nfull * N + t;
    const bool has_tail = !EXACT && t < N && kt < p.d, add = EXACT || (p.dR && p.dX);

    float mine = has_tail ? 1.f : 0.f;  // values of a row that this thread holds
#pragma unroll
    for (int i = 0; i < V; ++i) mine += EXACT || t + i * TPR < nfull ? (float)N : 0.f;
    float dg[V][N], db[V][N], dgt = 0.f, dbt = 0.f;
    u32x4 g[HELD ? V : 1];
    float gt = 1.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if constexpr (HELD) {
            g[i] = zero16();
            if (p.gain) g[i] = C::load(p.gain, t + i * TPR, nfull);
        }
#pragma unroll
        for (int e = 0; e < N; ++e) dg[i][e] = db[i][e] = 0.f;
    }
    if (p.gain && has_tail) gt = (float)p.gain[kt];
    auto gains = [&](int i) {
        if constexpr (HELD) return g[i];
        else __builtin_amdgcn_sched_barrier(0);
        return p.gain ? C::load(p.gain, t + i * TPR, nfull) : zero16();
    };

    struct Rows {
        u32x4 h[V], y[V], r[HELD ? V : 1];
        float ht, yt, rt;
    };
    // ALL: no row past M is among them.  A row past M is zeros and reads nothing:
    // the rows before it may be other waves', which store dX over them meanwhile.
    auto fetch = [&](auto all, int64_t m, Rows& f) {
        constexpr bool ALL = EXACT && (ROWS == 1 || decltype(all)::value);
        const bool live = ALL || m < p.M;
        const int64_t row = (live ? m : 0) * p.d, full = live ? nfull : 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int64_t c = t + i * TPR;
            if constexpr (ALL) {  // c < nfull is known; streamed, 4096 x 4096 takes 30.5 us instead of 32.8
                f.h[i] = load_streamed<u32x4>(p.H + row + c * N);
                f.y[i] = load_streamed<u32x4>(p.dY + row + c * N);
                if constexpr (HELD) f.r[i] = load_streamed<u32x4>(p.dR + row + c * N);
            } else {
                f.h[i] = C::load(p.H + row, c, full);
                f.y[i] = C::load(p.dY + row, c, full);
                if constexpr (HELD) {
                    if (add) f.r[i] = C::load(p.dR + row, c, full);
                }
            }
        }
        f.ht = f.yt = f.rt = 0.f;
        if (live && has_tail) {
            f.ht = (float)p.H[row + kt];
            f.yt = (float)p.dY[row + kt];
            if (add) f.rt = (float)p.dR[row + kt];
        }
    };
    // LAST: rows past M may be among them
    auto rows = [&](auto last, int64_t m, Rows& cur) {
        constexpr bool LAST = decltype(last)::value || !EXACT;
        const bool live = !LAST || m < p.M;
        float sh = cur.ht, su = gt * cur.yt;
#pragma unroll
        for (int i = 0; i < V; ++i) layer_norm_sums_of<T>(cur.h[i], cur.y[i], gains(i), p.gain != nullptr, sh, su);
        const float4 sums = row_sum4<TPR>(sh, su, 0.f, 0.f, red[0]);
        const float mean = sums.x / (float)p.d, ubar = sums.y / (float)p.d;
        float ct = has_tail ? cur.ht - mean : 0.f;
        float ss = ct * ct, uc = (gt * cur.yt - ubar) * ct;
        // a thread's sum of bf16 values that lie close together is exact, so what the
        // mean leaves of it is their c's sum
        float sc = sizeof(T) == 2 ? __builtin_fmaf(-mine, mean, sh) : ct;
        // h and u less their means, kept for the results where the registers hold them;
        // written-out fused steps: every form of this kernel gives the same bits
        float c[V == 1 ? N : 1], v[V == 1 ? N : 1];
        auto centre = [&](int i, int e, u32x4 gi, float& ce, float& ve) {
            ce = EXACT || t + i * TPR < nfull ? C::one(cur.h[i], e) - mean : 0.f;
            ve = __builtin_fmaf(p.gain ? C::one(gi, e) : 1.f, C::one(cur.y[i], e), -ubar);
        };
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const u32x4 gi = gains(i);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                float ce, ve;
                centre(i, e, gi, ce, ve);
                ss = __builtin_fmaf(ce, ce, ss);
                uc = __builtin_fmaf(ve, ce, uc);  // u - ubar adds up to nothing: c's mean need not be off it
                if constexpr (sizeof(T) == 4) sc += ce;
                if constexpr (V == 1) c[e] = ce, v[e] = ve;
            }
        }
        const float4 again = row_sum4<TPR>(ss, uc, sc, 0.f, red[1]);
        const float off = again.z / (float)p.d, rho = layer_norm_rho(again.x, off, (float)p.d, p.eps), left = -off * rho;
        const float back = layer_norm_back(rho, again.y, (float)p.d);
        ct -= off;
        const int64_t row = live ? m * p.d : 0, full = live ? nfull : 0;
        if constexpr (V > 1) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                asm volatile("" : "+v"(cur.h[i]), "+v"(cur.y[i]));
                if constexpr (HELD) asm volatile("" : "+v"(g[i]));
            }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const u32x4 gi = gains(i);
            u32x4 ri = zero16();
            if constexpr (HELD) ri = cur.r[i];
            else if (add) ri = C::load(p.dR + row, t + i * TPR, full);
            float dx[N];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                float ce, ve;
                if constexpr (V == 1) ce = c[e], ve = v[e];
                else centre(i, e, gi, ce, ve);
                const float hat = __builtin_fmaf(ce, rho, left), y = C::one(cur.y[i], e);
                dg[i][e] = __builtin_fmaf(hat, y, dg[i][e]);
                db[i][e] += y;
                dx[e] = __builtin_fmaf(-hat, back, ve);
                dx[e] = add ? __builtin_fmaf(rho, dx[e], C::one(ri, e)) : rho * dx[e];
            }
            if constexpr (EXACT && !LAST) C::store(p.dX + row, t + i * TPR, TPR * V, dx);
            else if (p.dX) C::store(p.dX + row, t + i * TPR, full, dx);
        }
        dgt = __builtin_fmaf(ct * rho, cur.yt, dgt);
        dbt += cur.yt;
        if (live && has_tail && p.dX) p.dX[row + kt] = (T)(rho * (gt * cur.yt - ubar - ct * rho * back) + cur.rt);
    };
    const int64_t first = (int64_t)blockIdx.x * ROWS;
    if constexpr (V == 1) {
        // the next rows' operands are loaded before the current ones' sums are
        // reduced, in two sets of registers in turn
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
    } else {  // a second set does not fit
        for (int64_t m0 = first; m0 < p.M; m0 += step) {
            Rows cur;
            fetch(std::false_type{}, m0 + rg, cur);
            rows(std::true_type{}, m0 + rg, cur);
        }
    }
    auto write = [&](float* to, const float(&s)[V][N], float st) {
        if (!to) return;
        float* out = to + (int64_t)blockIdx.x * p.stride;
        if constexpr (ROWS > 1) {
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) cols[(i * N + e) * kNormThreads + threadIdx.x] = s[i][e];
            cols[V * N * kNormThreads + threadIdx.x] = st;
            __syncthreads();
            // column j: element j % N of chunk j / N, or a tail element
            for (int j = threadIdx.x; j < p.d; j += kNormThreads) {
                const int c = j / N;
                const float* from = c < nfull ? cols + ((c / TPR) * N + j % N) * kNormThreads + c % TPR
                                              : cols + V * N * kNormThreads + j % N;
                float a = 0.f;
#pragma unroll
                for (int w = 0; w < ROWS; ++w) a += from[w * TPR];
                out[j] = a;
            }
            __syncthreads();
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const int64_t c = t + i * TPR;
                    if (c < nfull) out[c * N + e] = s[i][e];
                }
            if (has_tail) out[kt] = st;
        }
    };
    write(p.dgain, dg, dgt);
    write(p.dbias, db, dbt);
}

// Rows too long for registers: two more passes over each row, and the partial
// sums kept in memory (each thread reads and writes its own columns only).
template <typename T>
__global__ __launch_bounds__(kNormThreads) void layer_norm_bwd_long(LayerNormBwd<T> p) {
    using C = NormChunk<T>;
    constexpr int N = C::N;
    __shared__ float red[2][4 * kNormThreads / kWave];
    const int64_t full = p.d / N, kt = full * N + threadIdx.x;
    const bool tail = threadIdx.x < N && kt < p.d;
    float* dg = p.dgain ? p.dgain + (int64_t)blockIdx.x * p.stride : nullptr;
    float* db = p.dbias ? p.dbias + (int64_t)blockIdx.x * p.stride : nullptr;
    const float gt = tail && p.gain ? (float)p.gain[kt] : 1.f;
    auto load = [&](int64_t row, int64_t c, float(&h)[N], float(&y)[N], float(&u)[N]) {
        C::floats(C::load(p.H + row, c, full), h);
        C::floats(C::load(p.dY + row, c, full), y);
        u32x4 g = zero16();
        if (p.gain) g = C::load(p.gain, c, full);
#pragma unroll
        for (int e = 0; e < N; ++e) u[e] = p.gain ? C::one(g, e) * y[e] : y[e];
    };
    for (int64_t m = blockIdx.x; m < p.M; m += gridDim.x) {
        const int64_t row = m * p.d;
        const float ht = tail ? (float)p.H[row + kt] : 0.f, yt = tail ? (float)p.dY[row + kt] : 0.f;
        float sh = ht, su = gt * yt;
        for (int64_t c = threadIdx.x; c < full; c += kNormThreads) {
            float h[N], y[N], u[N];
            load(row, c, h, y, u);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                sh += h[e];
                su += u[e];
            }
        }
        const float4 sums = row_sum4<kNormThreads>(sh, su, 0.f, 0.f, red[0]);
        const float mean = sums.x / (float)p.d, ubar = sums.y / (float)p.d;
        float ct = tail ? ht - mean : 0.f;
        float ss = ct * ct, uc = (gt * yt - ubar) * ct, sc = ct;
        for (int64_t c = threadIdx.x; c < full; c += kNormThreads) {
            float h[N], y[N], u[N];
            load(row, c, h, y, u);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float k = h[e] - mean;
                ss += k * k;
                uc += (u[e] - ubar) * k;
                sc += k;
            }
        }
        const float4 again = row_sum4<kNormThreads>(ss, uc, sc, 0.f, red[1]);
        const float off = again.z / (float)p.d, rho = layer_norm_rho(again.x, off, (float)p.d, p.eps);
        const float back = layer_norm_back(rho, again.y, (float)p.d);
        ct -= off;
        const bool begun = m != blockIdx.x;
        for (int64_t c = threadIdx.x; c < full; c += kNormThreads) {
            float h[N], y[N], u[N], dx[N];
            load(row, c, h, y, u);
#pragma unroll
            for (int e = 0; e < N; ++e) h[e] = (h[e] - mean - off) * rho;
            if (dg) {
#pragma unroll
                for (int e = 0; e < N; ++e) dg[c * N + e] = (begun ? dg[c * N + e] : 0.f) + h[e] * y[e];
            }
            if (db) {
#pragma unroll
                for (int e = 0; e < N; ++e) db[c * N + e] = (begun ? db[c * N + e] : 0.f) + y[e];
            }
            if (p.dX) {
                u32x4 r = zero16();
                if (p.dR) r = C::load(p.dR + row, c, full);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    dx[e] = rho * (u[e] - ubar - h[e] * back);
                    if (p.dR) dx[e] += C::one(r, e);
                }
                C::store(p.dX + row, c, full, dx);
            }
        }
        if (tail) {
            if (dg) dg[kt] = (begun ? dg[kt] : 0.f) + ct * rho * yt;
            if (db) db[kt] = (begun ? db[kt] : 0.f) + yt;
            if (p.dX) p.dX[row + kt] = (T)(rho * (gt * yt - ubar - ct * rho * back) + (p.dR ? (float)p.dR[row + kt] : 0.f));
        }
    }
}

}  // namespace pifa
