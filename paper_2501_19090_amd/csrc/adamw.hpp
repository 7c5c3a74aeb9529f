// AdamW over many tensors at once, moments in fp32 or in 8 bits.
//
//   g' = g c,   m = b1 m + (1 - b1) g',   v = b2 v + (1 - b2) g'^2
//   p = p (1 - lr decay) - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)
//
// Bound by memory: each operand is read once and written once, 28 bytes a value
// with fp32 moments and gradients, 16.1 with moments in 8 bits, 2 more with a
// bf16 copy.  The tensors are cut into chunks of 4096 values, a workgroup each,
// by a table that the handle holds, so that any number of tensors is one launch.
//
// Moments in 8 bits are e4m3 codes in groups of 32 values with a power of two
// each (byte - 127; 255: the group is NaN).  A step moves a moment by less than
// half a step of e4m3 (b2 = 0.999: 0.1%, half a step is 3 to 6%), so rounding to
// nearest would leave it where it is for good.  It is rounded up or down by
// chance instead, up with the probability of what is left over the lower
// neighbour, which keeps the moment right on average: a step spreads v by about
// (0.09 (1 - b2))^1/2 of it, and over its memory of 1 / (1 - b2) steps that comes to
// a deviation of 0.2 v, 0.1 of its root.  That holds for a v of some units or more (a
// unit: the smallest code of its group, 2^-17 to 2^-18 of the largest v in it).  One
// of 1.3 units is 15% too large on average, and one below a unit stays at about a
// unit, because above zero it gets the smallest code at least: a value whose gradients
// are 5000 times smaller than its group's largest moves by about a tenth of
// what it should for as long as that one is there.  The update takes m and v before
// they are rounded; a v below fp32's normal range counts as zero in it.
#pragma once

#include "common.hpp"
#include "streamed.hpp"

namespace pifa {

constexpr int kAdamwThreads = 256;
constexpr int kAdamwChunk = 4096;  // values of a workgroup, and of one key of the random bits
constexpr int kAdamwGroup = 32;    // values that share a scale

struct AdamwTensor {
    float* p;
    const void* g;
    void* m;
    void* v;
    uint8_t* m_scale;
    uint8_t* v_scale;
    bf16* copy;  // or null
    int64_t n;
    double decay;
};
struct AdamwChunk {
    int32_t tensor;
    uint32_t index;  // of the tensor's chunks
};
// What depends on the number of the step.
struct AdamwStep {
    int64_t t;
    float rate, root;  // lr / (1 - b1^t), (1 - b2^t)^-1/2
};
struct AdamwArgs {
    const AdamwTensor* tensors;
    const AdamwChunk* chunks;
    AdamwStep* count;   // the handle's
    AdamwStep step;     // t = 0: *count holds it
    const float* grad_scale;  // or null
    double lr;
    float b1, c1, b2, c2, eps;  // c = 1 - b
    uint32_t seed;
};

// 32 bits that look random: two rounds of multiplication (by the fractions of the
// square roots of 2 and 3) and shift.
__device__ __forceinline__ uint32_t adamw_mix(uint32_t x) {
    x = (x ^ (x >> 16)) * 0x6A09E667u;
    x = (x ^ (x >> 15)) * 0xBB67AE85u;
    return x ^ (x >> 16);
}

// 2^(byte - 127)
__device__ __forceinline__ float adamw_scale(uint32_t byte) {
    const uint32_t bits = byte == 0 ? 0x00400000u : byte == 255 ? 0x7FC00000u : byte << 23;
    return __builtin_bit_cast(float, bits);
}

// Code of x >= 0, given in steps of the smallest e4m3 value (2^-9) and at most 448 *
// 512.  From 8 steps on a code is the value's exponent and its upper 3 bits, below it
// is the number of steps; both with 20 more bits behind them, to which the random
// ones and half of their last are added.  rnd: 16 bits, times 16, and 8.
__device__ __forceinline__ uint32_t adamw_e4m3(float x, uint32_t rnd) {
    const uint32_t large = __builtin_bit_cast(uint32_t, x) - (1032u << 20), small = (uint32_t)(x * 0x1p20f);
    return ((x >= 8.f ? large : small) + rnd) >> 20;
}

// The number of a step that the handle counts itself.
static __global__ void adamw_tick(AdamwStep* count, int64_t t, double lr, double b1, double b2) {
    if (t == 0) t = count->t + 1;
    count->t = t;
    count->rate = (float)(lr / (1.0 - pow(b1, (double)t)));
    count->root = (float)(1.0 / sqrt(1.0 - pow(b2, (double)t)));
}

// Groups of four values; EIGHT: eight neighbouring lanes hold a group of 32.  All
// but the bf16 copy, which the next forward reads, is streamed: 50.3 M values in
// fp32 take 253 us instead of 279.
template <typename T>
struct AdamwQuad {
    struct Four {
        T v[4];
    };
    __device__ __forceinline__ static void load(const void* base, int64_t at, float (&v)[4]) {
        const Four a = load_streamed<Four>((const T*)base + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (float)a.v[e];
    }
    __device__ __forceinline__ static void store(void* base, int64_t at, const float (&v)[4], bool streamed = true) {
        struct __attribute__((packed, aligned(sizeof(T)))) Any {
            Four f;
        } a;
#pragma unroll
        for (int e = 0; e < 4; ++e) a.f.v[e] = (T)v[e];
        if (streamed) store_streamed((T*)base + at, a.f);
        else *reinterpret_cast<Any*>((T*)base + at) = a;
    }
};

// Largest magnitude over the eight lanes of a group; a NaN survives.
__device__ __forceinline__ float adamw_top(float v) {
#pragma unroll
    for (int s = 1; s < 8; s <<= 1) {
        const float o = __shfl_xor(v, s);
        v = (v > o || v != v) ? v : o;
    }
    return v;
}

// Four codes of a group whose largest magnitude is `top`, and the scale's byte.
// LEAST: no value is below zero, and one above it has the smallest code at least.
template <bool LEAST>
__device__ __forceinline__ uint32_t adamw_pack(const float (&x)[4], float top, const uint32_t (&rnd)[4], uint32_t* byte) {
    const uint32_t t = __builtin_bit_cast(uint32_t, top) & 0x7FFFFFFFu;
    const bool bad = t >= 0x7F800000u;
    // the smallest k with top <= 448 2^k; 448 is 1.75 * 2^8
    const int k = max(-126, (int)(t >> 23) - 127 - 8 + ((t & 0x7FFFFFu) > 0x600000u ? 1 : 0));
    *byte = bad ? 255u : (uint32_t)(k + 127);
    uint32_t out = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float a = __builtin_amdgcn_ldexpf(fabsf(x[e]), 9 - k);
        uint32_t c = adamw_e4m3(a, rnd[e]);
        if constexpr (LEAST) c = max(c, min(__builtin_bit_cast(uint32_t, a), 1u));
        else c |= __builtin_bit_cast(uint32_t, x[e]) >> 24 & 0x80u;
        out |= c << (8 * e);
    }
    if (LEAST && k > 9) {  // the units are so large that an a may have vanished
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (x[e] > 0.f && (out >> (8 * e) & 0xFF) == 0) out |= 1u << (8 * e);
    }
    return bad ? 0x7F7F7F7Fu : out;
}

// m / d, rounded as a division rounds it but for one in some thousands: the product
// with the reciprocal, corrected by what that leaves; uncorrected where that is no
// number (an infinite d or quotient).
__device__ __forceinline__ float adamw_quotient(float m, float d) {
    const float y = __builtin_amdgcn_rcpf(d), q = m * y;
    const float c = __builtin_fmaf(__builtin_fmaf(-q, d, m), y, q);
    return c == c ? c : q;
}

// A workgroup for each chunk; a thread has four groups of four values, all of whose
// loads are on their way before the first is used.  50.3 M values in 8 tensors with
// fp32 gradients and a copy 253 us (6.0 TB/s), in 8 bits 158 us (5.8 TB/s), 29.4 M in
// 448 tensors of odd sizes in 8 bits with bf16 gradients 98 us.
template <bool EIGHT, typename G>
__global__ __launch_bounds__(kAdamwThreads) void adamw_update(AdamwArgs h) {
    constexpr int QUADS = kAdamwChunk / 4 / kAdamwThreads;  // of a thread
    const AdamwChunk chunk = h.chunks[blockIdx.x];
    const AdamwTensor T = h.tensors[chunk.tensor];
    const int64_t first = (int64_t)chunk.index * kAdamwChunk;
    const int left = (int)min((int64_t)kAdamwChunk, T.n - first);
    const AdamwStep step = h.step.t ? h.step : *h.count;
    const float c = h.grad_scale ? *h.grad_scale : 1.f;
    const float fall = (float)(h.lr * T.decay);
    uint32_t key = 0;
    if constexpr (EIGHT) {
        key = adamw_mix(adamw_mix(h.seed) + (uint32_t)step.t);
        key = adamw_mix(adamw_mix(key + (uint32_t)chunk.tensor) + chunk.index);
    }
    float p[QUADS][4], g[QUADS][4], m[QUADS][4], v[QUADS][4];
    uint32_t mc[QUADS], vc[QUADS];
    float ms[QUADS], vs[QUADS];
#pragma unroll
    for (int i = 0; i < QUADS; ++i) {
        const int at = 4 * (threadIdx.x + i * kAdamwThreads);
        const int64_t e0 = first + at;
        mc[i] = vc[i] = 0;
        ms[i] = vs[i] = 1.f;
        if (at + 4 <= left) {
            AdamwQuad<float>::load(T.p, e0, p[i]);
            AdamwQuad<G>::load(T.g, e0, g[i]);
            if constexpr (EIGHT) {
                mc[i] = load_streamed<uint32_t>((const uint8_t*)T.m + e0);
                vc[i] = load_streamed<uint32_t>((const uint8_t*)T.v + e0);
            } else {
                AdamwQuad<float>::load(T.m, e0, m[i]);
                AdamwQuad<float>::load(T.v, e0, v[i]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool in = at + e < left;
                p[i][e] = in ? T.p[e0 + e] : 0.f;
                g[i][e] = in ? (float)((const G*)T.g)[e0 + e] : 0.f;
                if constexpr (EIGHT) {
                    mc[i] |= in ? (uint32_t)((const uint8_t*)T.m)[e0 + e] << (8 * e) : 0u;
                    vc[i] |= in ? (uint32_t)((const uint8_t*)T.v)[e0 + e] << (8 * e) : 0u;
                } else {
                    m[i][e] = in ? ((const float*)T.m)[e0 + e] : 0.f;
                    v[i][e] = in ? ((const float*)T.v)[e0 + e] : 0.f;
                }
            }
        }
        if (EIGHT && at < left) {
            ms[i] = adamw_scale(T.m_scale[e0 / kAdamwGroup]);
            vs[i] = adamw_scale(T.v_scale[e0 / kAdamwGroup]);
        }
    }
#pragma unroll
    for (int i = 0; i < QUADS; ++i) {
        const int at = 4 * (threadIdx.x + i * kAdamwThreads);
        const int64_t e0 = first + at;
        if constexpr (EIGHT) {
            const auto m01 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mc[i], false), m23 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mc[i], true);
            const auto v01 = __builtin_amdgcn_cvt_pk_f32_fp8((int)vc[i], false), v23 = __builtin_amdgcn_cvt_pk_f32_fp8((int)vc[i], true);
            m[i][0] = m01[0] * ms[i], m[i][1] = m01[1] * ms[i], m[i][2] = m23[0] * ms[i], m[i][3] = m23[1] * ms[i];
            v[i][0] = v01[0] * vs[i], v[i][1] = v01[1] * vs[i], v[i][2] = v23[0] * vs[i], v[i][3] = v23[1] * vs[i];
        }
        {
            // each operation is rounded by itself, so that what the moments are
            // rounded from follows from the formula alone
#pragma clang fp contract(off)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float gs = g[i][e] * c;
                m[i][e] = m[i][e] * h.b1 + gs * h.c1;
                v[i][e] = v[i][e] * h.b2 + (gs * gs) * h.c2;
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            // the decay is added to the update before both meet p: 1 - lr decay, rounded to
            // fp32 first, would make 1.2e-7 of 1e-7 and nothing of 1e-8 for every value in
            // every step.  An infinite p stays infinite.
            const float q = adamw_quotient(step.rate * m[i][e], __builtin_amdgcn_sqrtf(v[i][e]) * step.root + h.eps);
            p[i][e] -= __builtin_fmaf(fall, __builtin_amdgcn_fmed3f(p[i][e], -0x1.FFFFFEp127f, 0x1.FFFFFEp127f), q);
        }
        uint32_t mb = 0, vb = 0;
        if constexpr (EIGHT) {
            uint32_t rm[4], rv[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t rnd = adamw_mix(key + (uint32_t)(at + e));
                rm[e] = (rnd >> 12 & 0xFFFF0u) | 8u;
                rv[e] = (rnd << 4 & 0xFFFF0u) | 8u;
                if (at + e >= left) m[i][e] = v[i][e] = 0.f;
            }
            auto top = [](const float(&x)[4]) {
                float t = fabsf(x[0]);
#pragma unroll
                for (int e = 1; e < 4; ++e) t = (t > fabsf(x[e]) || t != t) ? t : fabsf(x[e]);
                return adamw_top(t);
            };
            mc[i] = adamw_pack<false>(m[i], top(m[i]), rm, &mb);
            vc[i] = adamw_pack<true>(v[i], top(v[i]), rv, &vb);
            if (at < left && at % kAdamwGroup == 0) {
                T.m_scale[e0 / kAdamwGroup] = (uint8_t)mb;
                T.v_scale[e0 / kAdamwGroup] = (uint8_t)vb;
            }
        }
        if (at + 4 <= left) {
            AdamwQuad<float>::store(T.p, e0, p[i]);
            if constexpr (EIGHT) {
                store_streamed((uint8_t*)T.m + e0, mc[i]);
                store_streamed((uint8_t*)T.v + e0, vc[i]);
            } else {
                AdamwQuad<float>::store(T.m, e0, m[i]);
                AdamwQuad<float>::store(T.v, e0, v[i]);
            }
            if (T.copy) AdamwQuad<bf16>::store(T.copy, e0, p[i], false);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (at + e >= left) continue;
                T.p[e0 + e] = p[i][e];
                if constexpr (EIGHT) {
                    ((uint8_t*)T.m)[e0 + e] = (uint8_t)(mc[i] >> (8 * e));
                    ((uint8_t*)T.v)[e0 + e] = (uint8_t)(vc[i] >> (8 * e));
                } else {
                    ((float*)T.m)[e0 + e] = m[i][e];
                    ((float*)T.v)[e0 + e] = v[i][e];
                }
                if (T.copy) T.copy[e0 + e] = (bf16)p[i][e];
            }
        }
    }
    if (blockIdx.x == 0 && threadIdx.x == 0 && h.step.t) *h.count = h.step;
}

}  // namespace pifa
