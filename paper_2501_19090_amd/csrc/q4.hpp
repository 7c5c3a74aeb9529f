// Layers with 4-bit weights: Y = X W^T with
//   W[n, k] = e2m1(code[n, k]) * 2^(scale[n, k / 32] - 127)
// (OCP microscaling: 4-bit elements of value 0, 0.5, 1, 1.5, 2, 3, 4, 6 and
// their negatives, and one 8-bit power of two per 32 of a row; scale 255 is
// NaN).
//
// Two forms of the product, both on the instructions gfx950 has for the format:
//   bf16 rows   the codes become bf16 in registers, two per instruction and
//               scaled by it (v_cvt_scalef32_pk_bf16_fp4, exact except where
//               bf16 ends), and feed 16x16x32 MFMAs;
//   e4m3 rows   the codes feed the 16x16x128 MFMA as they are, which scales
//               each 32 of a row itself; the row's own scale is a factor of
//               the output.
//
// Packed layout: blocks of 16 rows x 128 columns, block (g, b) at ((g * KB) +
// b) * 1088 bytes (KB = ceil(K / 128)).  Chunk l (16 bytes, l = 0..63) holds
// the 32 codes of row 16g + l % 16, columns 128b + 32 (l / 16) .. + 31, lower
// column in the lower half of a byte, and byte 1024 + l their scale: what lane
// l of a wave feeds as an MFMA operand.  Rows past N and columns past K hold
// zero codes under scale 127 (1.0), so a block is a kilobyte and 64 bytes of
// one stream.
#pragma once

#include "common.hpp"
#include "gemm_mfma.hpp"
#include "layout.hpp"
#include "norm.hpp"

namespace pifa {

constexpr int kQ4Group = 32;
constexpr int kQ4Block = 1088;
constexpr int kQ4NanScale = 255;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

__host__ __device__ inline int64_t q4_packed_bytes(int64_t N, int64_t K) {
    return packed_groups(N) * packed_kblocks(K) * kQ4Block;
}
// byte of the packed image that holds the codes of (n, 32 * grp ...), and their scale
__device__ __forceinline__ int64_t q4_chunk(int64_t n, int64_t grp, int64_t KB) {
    return ((n / 16) * KB + grp / 4) * kQ4Block + ((n % 16) + 16 * (grp % 4)) * 16;
}
__device__ __forceinline__ int64_t q4_scale_at(int64_t n, int64_t grp, int64_t KB) {
    return ((n / 16) * KB + grp / 4) * kQ4Block + 1024 + (n % 16) + 16 * (grp % 4);
}

// ------------------------------------------------------------------ making weights
// Code of the e2m1 value next to |a| (ties to the even code; past 6: 6).
__device__ __forceinline__ uint32_t e2m1_code(float a) {
    // the midpoints belong to the code with an even mantissa bit: 0.25 -> 0,
    // 0.75 -> 1, 1.25 -> 1, 1.75 -> 2, 2.5 -> 2, 3.5 -> 4, 5 -> 4
    return (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.f);
}
__device__ __forceinline__ float e2m1_value(uint32_t c) {  // c = 0..7
    return c < 2 ? 0.5f * (float)c : __builtin_ldexpf(1.f + 0.5f * (float)(c & 1), (int)(c >> 1) - 1);
}

// One thread per 32 weights of a row (padding rows and groups included).  Of
// the two scales that put the largest magnitude into the elements' range, the
// one that makes it 4 to 8 (values past 6 become 6) and the one that makes it 2
// to 4, the one with the smaller squared error is taken, the first on a tie.
// A group with an infinity or a NaN gets the NaN scale.
template <typename T>
__global__ void q4_quantize(const T* __restrict__ W, int64_t N, int64_t K, uint8_t* __restrict__ packed) {
    const int64_t KB = packed_kblocks(K), groups = KB * 4;
    const int64_t total = packed_groups(N) * 16 * groups;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t n = i / groups, grp = i % groups;
        uint32_t codes[4] = {0, 0, 0, 0}, scale = 127;
        if (n < N && grp * kQ4Group < K) {  // K is a multiple of 32
            const T* w = W + n * K + grp * kQ4Group;
            float v[kQ4Group], amax = 0.f;
            bool bad = false;
#pragma unroll
            for (int e = 0; e < kQ4Group; ++e) {
                if constexpr (sizeof(T) == 2) v[e] = bf16_bits_to_f32(__builtin_bit_cast(uint16_t, w[e]));
                else v[e] = w[e];
                bad |= !(fabsf(v[e]) <= 3.402823466e38f);
                amax = fmaxf(amax, fabsf(v[e]));
            }
            if (bad) {
                scale = kQ4NanScale;
            } else if (amax > 0.f) {
                int e2;
                (void)frexpf(amax, &e2);  // amax = f * 2^e2, f in [0.5, 1)
                float best = 0.f;
                for (int c = 0; c < 2; ++c) {
                    // exponents from -127 up; 2^-s is finite for all of them but the last few, where ldexp steps twice
                    int s = e2 - 3 + c;
                    s = s < -127 ? -127 : s > 126 ? 126 : s;
                    float err = 0.f;
                    uint32_t q[4] = {0, 0, 0, 0};
#pragma unroll
                    for (int e = 0; e < kQ4Group; ++e) {
                        const float a = __builtin_ldexpf(v[e], -s);
                        const uint32_t code = e2m1_code(fabsf(a));
                        const float off = fabsf(a) - e2m1_value(code);
                        err += off * off;
                        q[e / 8] |= (code | (signbit(v[e]) ? 8u : 0u)) << (4 * (e & 7));
                    }
                    err = __builtin_ldexpf(err, 2 * c);  // in units of the first scale
                    if (c == 0 || err < best) {
                        best = err;
                        scale = (uint32_t)(s + 127);
#pragma unroll
                        for (int x = 0; x < 4; ++x) codes[x] = q[x];
                    }
                }
            }
        }
        *reinterpret_cast<u32x4*>(packed + q4_chunk(n, grp, KB)) = u32x4{codes[0], codes[1], codes[2], codes[3]};
        packed[q4_scale_at(n, grp, KB)] = (uint8_t)scale;
    }
}

// Row-major codes (N x K / 2 bytes) and scales (N x K / 32 bytes) to and from
// the packed image; any alignment.  TO_PACKED writes the padding too.
template <bool TO_PACKED>
__global__ void q4_convert(uint8_t* __restrict__ codes, uint8_t* __restrict__ scales, int64_t N, int64_t K,
                           uint8_t* __restrict__ packed) {
    const int64_t KB = packed_kblocks(K), groups = KB * 4;
    const int64_t total = packed_groups(N) * 16 * groups;
    struct __attribute__((packed, aligned(1))) Any16 {
        u32x4 v;
    };
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (int64_t)gridDim.x * blockDim.x) {
        const int64_t n = i / groups, grp = i % groups;
        const bool in = n < N && grp * kQ4Group < K;
        u32x4* chunk = reinterpret_cast<u32x4*>(packed + q4_chunk(n, grp, KB));
        uint8_t* scale = packed + q4_scale_at(n, grp, KB);
        Any16* row = reinterpret_cast<Any16*>(codes + n * (K / 2) + grp * 16);
        if constexpr (TO_PACKED) {
            *chunk = in ? row->v : zero16();
            *scale = in ? scales[n * (K / kQ4Group) + grp] : 127;
        } else if (in) {
            if (codes) row->v = *chunk;
            if (scales) scales[n * (K / kQ4Group) + grp] = *scale;
        }
    }
}

// ------------------------------------------------------------------ products of few rows
// acc(n, m): the weights are the first MFMA operand, so a lane holds four
// consecutive columns n of Y of one row m (row l % 16, columns 4 (l / 16) ..).

// 8 codes -> 8 bf16, times the scale (an fp32 power of two)
__device__ __forceinline__ u32x4 q4_to_bf16(uint32_t w, float scale) {
    bf16x2 p[4];
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    return __builtin_bit_cast(u32x4, p);
}
__device__ __forceinline__ f32x4 q4_mfma_bf16(u32x4 w, u32x4 x, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), c, 0,
                                                   0, 0);
}
// 16 x 16 x 128, e2m1 codes under their scales by e4m3 values.  Lane l brings
// 32 codes of row l % 16, columns 32 (l / 16) ..; of the e4m3 row l % 16 it
// brings columns 16 (l / 16) .. + 15 in x0 and 64 + 16 (l / 16) .. in x1.
__device__ __forceinline__ f32x4 q4_mfma_e4m3(u32x4 w, uint32_t scale, u32x4 x0, u32x4 x1, f32x4 c) {
    const i32x8 a = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
    const i32x8 b = {(int)x0[0], (int)x0[1], (int)x0[2], (int)x0[3], (int)x1[0], (int)x1[1], (int)x1[2], (int)x1[3]};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 4 /* e2m1 */, 0 /* e4m3 */, 0, (int)scale, 0,
                                                            0x7F7F7F7F);
}

enum Q4Act : int { kQ4Bf16 = 0, kQ4E4m3 = 1 };

struct Q4Args {
    const uint8_t* W;      // packed
    const void* X;         // M x K, bf16 or e4m3
    const float* x_scale;  // e4m3: a scale per row
    bf16* Y;               // M x N
    int64_t M, N, K;
    // the norm's form: rows X + R, normed with gain
    const bf16* R;     // or null
    const bf16* gain;  // or null
    bf16* H;           // or null; X + R, written by the first workgroup
    float eps;
};

// Columns 4 * q .. + 3 of row m from v.
__device__ __forceinline__ void q4_store4(const Q4Args& p, int64_t m, int64_t n, const f32x4& v, float factor) {
    if (m >= p.M || n >= p.N) return;
    bf16* y = p.Y + m * p.N + n;
    uint16_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = f32_to_bf16_bits(v[i] * factor);
    struct __attribute__((packed, aligned(2))) Any8 {
        uint16_t h[4];
    };
    if (n + 4 <= p.N) {
        *reinterpret_cast<Any8*>(y) = Any8{{h[0], h[1], h[2], h[3]}};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < p.N) reinterpret_cast<uint16_t*>(y)[i] = h[i];
    }
}

// A workgroup owns NG groups of 16 weight rows (columns of Y) and 16 MT rows of
// X (blockIdx.y picks them); its waves take the 128-wide blocks of K in turn,
// each on registers alone, and are summed in LDS at the end.  The loads of a
// wave's next U blocks are issued before the MFMAs of the current ones.
template <int ACT, bool NORM, int MT, int NG, int WAVES, int U>
__global__ __launch_bounds__(WAVES* kWave) void q4_few(Q4Args p) {
    static_assert(!NORM || (MT == 1 && ACT == kQ4Bf16), "the norm's form has one tile of bf16 rows");
    constexpr int XC = ACT == kQ4Bf16 ? 4 : 2;  // 16-byte pieces of a row's 32 values
    constexpr int ES = ACT == kQ4Bf16 ? 2 : 1;
    __shared__ f32x4 red[WAVES][MT * NG][kWave];
    __shared__ float reds[NORM ? WAVES : 1][16];
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int row = lane & 15, q = lane >> 4;
    const int KB = (int)packed_kblocks(p.K), K = (int)p.K;
    const int64_t g0 = (int64_t)blockIdx.x * NG, m0 = (int64_t)blockIdx.y * (16 * MT);
    const int64_t left = p.M - m0;
    const int rows = left < 16 * MT ? (int)left : 16 * MT;

    // streams: buffer ranges end with the data, so masked lanes read zeros
    const auto xrs = make_rsrc31((const char*)p.X + m0 * p.K * ES, (int64_t)rows * p.K * ES);
    __amdgpu_buffer_rsrc_t rrs, grs;
    if constexpr (NORM) {
        rrs = make_rsrc31(p.R, p.R ? (int64_t)rows * p.K * 2 : 0);
        grs = make_rsrc31(p.gain, p.gain ? p.K * 2 : 0);
    }
    const uint8_t* wp[NG];
    const int64_t groups = packed_groups(p.N);
#pragma unroll
    for (int j = 0; j < NG; ++j) wp[j] = p.W + (g0 + j < groups ? g0 + j : groups - 1) * KB * kQ4Block;

    f32x4 acc[MT][NG];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int j = 0; j < NG; ++j) acc[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    float ss = 0.f;

    struct Blk {
        u32x4 w[NG];
        uint32_t s[NG];
        u32x4 x[MT][XC];
        u32x4 r[NORM ? XC : 1], g[NORM ? XC : 1];
    };
    // first column of piece c of this lane's 32 values of block b
    auto col = [&](int b, int c) { return ACT == kQ4Bf16 ? 128 * b + 32 * q + 8 * c : 128 * b + 64 * c + 16 * q; };
    auto fetch = [&](int b, Blk& f) {
        const bool in = b < KB;  // uniform
        const int bb = in ? b : KB - 1;
#pragma unroll
        for (int j = 0; j < NG; ++j) {
            const uint8_t* blk = wp[j] + (int64_t)bb * kQ4Block;
            f.w[j] = *reinterpret_cast<const u32x4*>(blk + lane * 16);
            f.s[j] = blk[1024 + lane];
        }
#pragma unroll
        for (int c = 0; c < XC; ++c) {
            const int k = col(b, c);
#pragma unroll
            for (int t = 0; t < MT; ++t)
                f.x[t][c] = load16(xrs, row + 16 * t < rows && k < K ? (uint32_t)(((row + 16 * t) * K + k) * ES)
                                                                     : kMaskedOffset);
            if constexpr (NORM) {
                f.r[c] = load16(rrs, row < rows && k < K ? (uint32_t)((row * K + k) * 2) : kMaskedOffset);
                f.g[c] = load16(grs, row < rows && k < K ? (uint32_t)(k * 2) : kMaskedOffset);
            }
        }
    };
    auto step = [&](int b, Blk& f) {
        if (b >= KB) return;  // uniform
        if constexpr (NORM) {
            typedef NormChunk<bf16> C;
#pragma unroll
            for (int c = 0; c < XC; ++c) {
                float h[8], r[8], g[8];
                C::floats(f.x[0][c], h);
                C::floats(f.r[c], r);
                C::floats(f.g[c], g);
                bf16 v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    h[e] += r[e];
                    ss += h[e] * h[e];
                    v[e] = (bf16)(p.gain ? h[e] * g[e] : h[e]);
                }
                const int k = col(b, c);
                if (p.H && blockIdx.x == 0 && row < rows && k < K) C::store(p.H + row * p.K, k / 8, p.K / 8, h);
                f.x[0][c] = __builtin_bit_cast(u32x4, v);
            }
        }
        if constexpr (ACT == kQ4Bf16) {
#pragma unroll
            for (int j = 0; j < NG; ++j) {
                const float s = __builtin_bit_cast(float, f.s[j] << 23);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const u32x4 w = q4_to_bf16(f.w[j][c], s);
#pragma unroll
                    for (int t = 0; t < MT; ++t) acc[t][j] = q4_mfma_bf16(w, f.x[t][c], acc[t][j]);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < NG; ++j)
#pragma unroll
                for (int t = 0; t < MT; ++t)
                    acc[t][j] = q4_mfma_e4m3(f.w[j], f.s[j], f.x[t][0], f.x[t][1], acc[t][j]);
        }
    };
    Blk cur[U], nxt[U];
#pragma unroll
    for (int u = 0; u < U; ++u) fetch(wave + u * WAVES, cur[u]);
    for (int b = wave; b < KB; b += U * WAVES) {
        const bool more = b + U * WAVES < KB;  // uniform
        if (more) {
#pragma unroll
            for (int u = 0; u < U; ++u) fetch(b + (U + u) * WAVES, nxt[u]);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < U; ++u) step(b + u * WAVES, cur[u]);
        if (more) {
#pragma unroll
            for (int u = 0; u < U; ++u) cur[u] = nxt[u];
        }
    }

#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int j = 0; j < NG; ++j) red[wave][t * NG + j][lane] = acc[t][j];
    if constexpr (NORM) {
        ss += __shfl_xor(ss, 16);
        ss += __shfl_xor(ss, 32);
        if (lane < 16) reds[wave][lane] = ss;
    }
    __syncthreads();
    for (int i = wave; i < MT * NG; i += WAVES) {
        const int t = i / NG, j = i % NG;
        f32x4 tot = red[0][i][lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) tot += red[w][i][lane];
        const int64_t m = m0 + 16 * t + row;
        float factor = 1.f;
        if constexpr (NORM) {
            float s = reds[0][row];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) s += reds[w][row];
            factor = rsqrtf(s / (float)p.K + p.eps);
        }
        if constexpr (ACT == kQ4E4m3) factor = m < p.M ? p.x_scale[m] : 0.f;
        if (g0 + j < groups) q4_store4(p, m, (g0 + j) * 16 + 4 * q, tot, factor);
    }
}

}  // namespace pifa
