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
//
// Few rows are bound by that stream: one row of 8192 -> 28672 (125 MB) 22.9 us,
// 5.4 TB/s, where plain reads of 1 GiB reach 6.6; of 4096 -> 11008 (24 MB) 6.2
// us, of which reading at that rate is 3.7 and a launch about 2.
#pragma once

#include "common.hpp"
#include "gemm_dma.hpp"
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
__global__ __launch_bounds__(256) void q4_quantize(const T* __restrict__ W, int64_t N, int64_t K, uint8_t* __restrict__ packed) {
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

// The largest scale of any group, NaN aside (*top starts as 0).
__global__ __launch_bounds__(256) void q4_top_scale(const uint8_t* __restrict__ packed, int64_t blocks, int* top) {
    int most = 0;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < blocks * 4; i += (int64_t)gridDim.x * blockDim.x) {
        const u32x4 s = *reinterpret_cast<const u32x4*>(packed + i / 4 * kQ4Block + 1024 + i % 4 * 16);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int v = (int)((s[e / 4] >> (8 * (e & 3))) & 255);
            most = max(most, v == kQ4NanScale ? 0 : v);
        }
    }
#pragma unroll
    for (int s = 1; s < kWave; s <<= 1) most = max(most, __shfl_xor(most, s));
    if ((threadIdx.x & (kWave - 1)) == 0) atomicMax(top, most);
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

// 4 x 4 transpose of 16-byte pieces over the lane groups q = lane / 16: piece c
// of group q goes to piece q of group c.
__device__ __forceinline__ void q4_turn(u32x4 (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t a = x[0][i], b = x[1][i], c = x[2][i], d = x[3][i];
        auto s = __builtin_amdgcn_permlane32_swap(a, c, false, false);
        a = s[0]; c = s[1];
        s = __builtin_amdgcn_permlane32_swap(b, d, false, false);
        b = s[0]; d = s[1];
        s = __builtin_amdgcn_permlane16_swap(a, b, false, false);
        x[0][i] = s[0]; x[1][i] = s[1];
        s = __builtin_amdgcn_permlane16_swap(c, d, false, false);
        x[2][i] = s[0]; x[3][i] = s[1];
    }
}

// Lane l's codes and scale of block b of a group's stream (zeros if not `in`).
__device__ __forceinline__ void q4_load(__amdgpu_buffer_rsrc_t rs, bool in, int b, int lane, u32x4& w, uint32_t& s) {
    const uint32_t at = in ? (uint32_t)b * kQ4Block : kMaskedOffset;
    w = load16(rs, at + lane * 16);
    s = __builtin_amdgcn_raw_buffer_load_b8(rs, (int)(at + 1024 + lane), 0, 0);
}

// The steps of one wave (blocks wave, wave + WAVES, ... below KB, U of them a
// step; step 0 is in `even` already): the loads of a step are issued before the
// products of the one before it, in two sets of registers in turn.  No load
// stands under a condition, or the wait for the one set would be a wait for
// both.
template <int U, int WAVES, typename Blk, typename Fetch, typename Step>
__device__ __forceinline__ void q4_pipeline(int wave, int KB, Blk (&even)[U], Blk (&odd)[U], const Fetch& fetch,
                                            const Step& step) {
    const int n = wave < KB ? (KB - wave + U * WAVES - 1) / (U * WAVES) : 0;
    auto products = [&](int s, Blk(&f)[U]) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int b = wave + (s * U + u) * WAVES;
            if (u == 0 || b < KB) step(b, f[u]);  // uniform
        }
    };
    int i = 0;
    for (; i + 2 < n; i += 2) {
        fetch(i + 1, odd);
        products(i, even);
        fetch(i + 2, even);
        products(i + 1, odd);
    }
    if (i + 1 < n) {
        fetch(i + 1, odd);
        products(i, even);
        products(i + 1, odd);
    } else if (i < n) {
        products(i, even);
    }
}

constexpr int kQ4NormRows = 8;  // rows that come as two bf16 values each
// The norm's form in one launch: most elements of X; values of (X + R) gain
// beyond which a row (512 of it, for the lower bound) counts as far from 1; the
// largest group scale of the weights, as a power of two.
constexpr int64_t kQ4NormElems = 12288;
constexpr float kQ4NormBig = 0x1p40f, kQ4NormSmall = 0x1p-30f;
constexpr int kQ4NormTop = 60;

// At most 16 rows.  A workgroup owns NG groups of 16 weight rows (columns of Y);
// its waves take the 128-wide blocks of K in turn, each on registers alone, and
// are summed in LDS at the end.  The rows come from the caches again for every
// workgroup: NG grows with the number of groups (see the dispatch).  A bf16
// lane multiplies 64 consecutive bytes of a row; the four lanes of a row load
// them as 64 bytes side by side per instruction and turn them (16 rows of 8192
// -> 28672 33 us, loaded as they are multiplied 38 us).
// SPLIT: X is at most 8 rows and behind them what their rounding left, which
// take rows 8 + m of the MFMA; both sums are added at the end.
template <int ACT, int NG, int WAVES, int U, bool SPLIT>
__global__ __launch_bounds__(WAVES* kWave) void q4_few(Q4Args p) {
    constexpr int XC = ACT == kQ4Bf16 ? 4 : 2;  // 16-byte pieces of a lane's 32 values
    constexpr int ES = ACT == kQ4Bf16 ? 2 : 1;
    static_assert(NG <= WAVES, "a wave adds up a group");
    __shared__ f32x4 red[WAVES][NG][kWave];
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int row = lane & 15, q = lane >> 4;
    const int KB = (int)packed_kblocks(p.K), K = (int)p.K, rows = (int)p.M;
    const int64_t groups = packed_groups(p.N), g0 = (int64_t)blockIdx.x * NG;

    // the range ends with the last row; masked lanes read zeros
    const auto xrs = make_rsrc31(p.X, (int64_t)rows * (SPLIT ? 2 : 1) * K * ES);
    const bool second = SPLIT && row >= kQ4NormRows;
    const bool held = second ? row - kQ4NormRows < rows : row < rows;
    const int slot = second ? row - kQ4NormRows + rows : row;
    __amdgpu_buffer_rsrc_t wrs[NG];
#pragma unroll
    for (int j = 0; j < NG; ++j)
        wrs[j] = make_rsrc31(p.W + (g0 + j < groups ? g0 + j : 0) * KB * kQ4Block,
                             g0 + j < groups ? (int64_t)KB * kQ4Block : 0);
    f32x4 acc[NG];
#pragma unroll
    for (int j = 0; j < NG; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};

    struct Blk {
        u32x4 w[NG];
        uint32_t s[NG];
        u32x4 x[XC];
    };
    auto fetch_step = [&](int s, Blk(&f)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int b = wave + (s * U + u) * WAVES;
#pragma unroll
            for (int j = 0; j < NG; ++j) q4_load(wrs[j], b < KB, b, lane, f[u].w[j], f[u].s[j]);
#pragma unroll
            for (int c = 0; c < XC; ++c) {
                // 64 bytes in a row of the four lane groups; bf16 is turned in step()
                const int k = 128 * b + (64 / ES) * c + (16 / ES) * q;
                f[u].x[c] = load16(xrs, held && k < K ? (uint32_t)((slot * K + k) * ES) : kMaskedOffset);
            }
        }
    };
    auto step = [&](int, Blk& f) {
        if constexpr (ACT == kQ4Bf16) q4_turn(f.x);
#pragma unroll
        for (int j = 0; j < NG; ++j) {
            if constexpr (ACT == kQ4Bf16) {
                const float s = __builtin_bit_cast(float, f.s[j] << 23);
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[j] = q4_mfma_bf16(q4_to_bf16(f.w[j][c], s), f.x[c], acc[j]);
            } else {
                acc[j] = q4_mfma_e4m3(f.w[j], f.s[j], f.x[0], f.x[1], acc[j]);
            }
        }
    };
    Blk even[U], odd[U];
    fetch_step(0, even);
    q4_pipeline<U, WAVES>(wave, KB, even, odd, fetch_step, step);

#pragma unroll
    for (int j = 0; j < NG; ++j) red[wave][j][lane] = acc[j];
    __syncthreads();
    if (wave < NG && g0 + wave < groups) {
        f32x4 tot = red[0][wave][lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) tot += red[w][wave][lane];
        if constexpr (SPLIT) {
#pragma unroll
            for (int i = 0; i < 4; ++i) tot[i] += __shfl(tot[i], lane ^ kQ4NormRows);
        }
        const float factor = ACT == kQ4E4m3 ? (row < rows ? p.x_scale[row] : 0.f) : 1.f;
        q4_store4(p, row, (g0 + wave) * 16 + 4 * q, tot, factor);
    }
}

// ------------------------------------------------------------------ few rows, staged
// As q4_few for bf16 rows, with them in LDS, which each workgroup stages while its first
// weights are on their way; the norm's form norms them on the way there: the
// product is of (X + R) gain, and rho, a factor of the row, is applied to the
// sums.  Rounded to bf16 alone, (X + R) gain would add as much error as the
// output's rounding (more where a few columns carry a row), so at most 8 rows
// take the MFMA's 16: row m is the rounded values, row 8 + m what the rounding
// left, and their sums are added at the end.  The staged rows leave the loop
// nothing to load but weights.
// The sums of unscaled products could leave fp32's range where those of the
// normed row do not, so a row with values far from 1 is staged again with rho
// (no row of a model's; the check for it costs up to 0.2 us of 6), and
// layers with weights past 2^kQ4NormTop take norm and product in two launches:
// sums stay below 12288 2^40 6 2^60 < 2^117.
//
// LDS: for each block of K, its pieces (column chunk c, lane group q, row slot r
// of S) at ((c * 4 + q) * S + r) * 16 bytes (S = M, the norm's form 2 M); 16 zero
// bytes, which the lanes of rows past M read; over both, after the loop, the
// sums of the waves.  Then rho and the partial sums of squares (512 columns each).
__host__ __device__ inline int64_t q4_staged_rows_lds(int64_t M, int64_t K, bool norm, int red_kb) {
    const int64_t x = (norm ? 2 : 1) * M * packed_kblocks(K) * 256 + 16;
    return x > red_kb * 1024 ? x : red_kb * 1024;
}
__host__ __device__ inline int64_t q4_staged_lds(int64_t M, int64_t K, bool norm, int red_kb) {
    return q4_staged_rows_lds(M, K, norm, red_kb) + (norm ? (M * ceil_div(K, 512) + 16) * 4 : 0);
}

template <bool NORM, int NG, int WAVES, int U>
__global__ __launch_bounds__(WAVES* kWave) void q4_staged(Q4Args p) {
    extern __shared__ __attribute__((aligned(1024))) char dyn[];
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int row = lane & 15, q = lane >> 4;
    const int K = (int)p.K, KB = (int)packed_kblocks(p.K), M = (int)p.M;
    const int S = NORM ? 2 * M : M, xbytes = S * KB * 256;
    f32x4* red = reinterpret_cast<f32x4*>(dyn);  // WAVES x NG x 64, after the loop
    char* xs = dyn;
    float* rho = reinterpret_cast<float*>(dyn + q4_staged_rows_lds(M, K, NORM, WAVES * NG));
    float* sums = rho + 16;

    const int64_t groups = packed_groups(p.N), g0 = (int64_t)blockIdx.x * NG;
    struct Blk {
        u32x4 w[NG];
        uint32_t s[NG];
    };
    __amdgpu_buffer_rsrc_t wrs[NG];
#pragma unroll
    for (int j = 0; j < NG; ++j)
        wrs[j] = make_rsrc31(p.W + (g0 + j < groups ? g0 + j : 0) * KB * kQ4Block,
                             g0 + j < groups ? (int64_t)KB * kQ4Block : 0);
    auto fetch_step = [&](int s, Blk(&f)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int b = wave + (s * U + u) * WAVES;
#pragma unroll
            for (int j = 0; j < NG; ++j) q4_load(wrs[j], b < KB, b, lane, f[u].w[j], f[u].s[j]);
        }
    };
    Blk even[U], odd[U];
    fetch_step(0, even);

    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)xs;
    if (threadIdx.x < 4) reinterpret_cast<uint32_t*>(xs + xbytes)[threadIdx.x] = 0;
    if constexpr (NORM) {
        typedef NormChunk<bf16> C;
        // a wave takes 512 columns of a row at a time, four such units in flight
        const int segs = (K + 511) / 512, units = M * segs, full = K / 8;
        constexpr int UN = 4;
        static_assert(kQ4NormElems / 512 + kQ4NormRows <= kWave, "a bit and a lane for each unit");
        // AGAIN: the units of `which` once more, with rho
        auto stage = [&](auto again, uint64_t which) {
            constexpr bool AGAIN = decltype(again)::value;
            for (int u0 = wave; u0 < units; u0 += UN * WAVES) {
                u32x4 x[UN], r[UN], g[UN];
#pragma unroll
                for (int i = 0; i < UN; ++i) {
                    const int u = u0 + i * WAVES, m = u / segs, c = (u - m * segs) * 64 + lane;
                    const int in = u < units && (!AGAIN || ((which >> u) & 1)) ? full : 0;
                    x[i] = C::load((const bf16*)p.X + (int64_t)m * K, c, in);
                    r[i] = zero16();
                    g[i] = zero16();
                    if (p.R) r[i] = C::load(p.R + (int64_t)m * K, c, in);
                    if (p.gain) g[i] = C::load(p.gain, c, in);
                }
#pragma unroll
                for (int i = 0; i < UN; ++i) {
                    const int u = u0 + i * WAVES, m = u / segs, c = (u - m * segs) * 64 + lane;
                    if (u >= units) break;  // uniform
                    if (AGAIN && !((which >> u) & 1)) continue;
                    const float f = AGAIN ? rho[m] : 1.f;
                    float h[8], ss = 0.f, top = 0.f;
                    bf16 v[8], left[8];
                    C::floats(x[i], h);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        h[e] += C::one(r[i], e);
                        ss += h[e] * h[e];
                        const float k = AGAIN ? h[e] * f : h[e], y = p.gain ? k * C::one(g[i], e) : k;
                        top = fmaxf(top, fabsf(y));
                        const NormPair pair(y);
                        v[e] = pair.hi;
                        left[e] = pair.lo;
                    }
                    if (!AGAIN && p.H && blockIdx.x == 0) C::store(p.H + (int64_t)m * K, c, full, h);
                    // columns 8c .. 8c + 7: block c / 16, lane group (c / 4) % 4, piece c % 4
                    if (c < KB * 16) {
                        char* at = xs + (((c >> 4) * 16 + (c & 3) * 4 + ((c >> 2) & 3)) * S + m) * 16;
                        *reinterpret_cast<u32x4*>(at) = __builtin_bit_cast(u32x4, v);
                        *reinterpret_cast<u32x4*>(at + M * 16) = __builtin_bit_cast(u32x4, left);
                    }
                    if constexpr (!AGAIN) {
#pragma unroll
                        for (int s = 1; s < kWave; s <<= 1) ss += __shfl_xor(ss, s);
                        // the sign says whether the unit's values are far from 1
                        const bool far = __any(top > kQ4NormBig) || (__any(top > 0.f) && !__any(top >= kQ4NormSmall));
                        if (lane == 0) sums[u] = copysignf(ss, far ? -1.f : 1.f);
                    }
                }
            }
        };
        stage(std::false_type{}, 0);
        __syncthreads();
        const uint64_t far = __ballot(lane < units && signbit(sums[lane < units ? lane : 0]));
        for (int m = wave; m < M; m += WAVES) {  // read after the barrier behind the products
            float ss = 0.f;
            for (int s = lane; s < segs; s += kWave) ss += fabsf(sums[m * segs + s]);
#pragma unroll
            for (int s = 1; s < kWave; s <<= 1) ss += __shfl_xor(ss, s);
            if (lane == 0) rho[m] = rsqrtf(ss / (float)K + p.eps);
        }
        if (far) {  // the same in all waves
            uint64_t which = 0;
            for (int m = 0; m < M; ++m) {
                const uint64_t row_units = ((1ull << segs) - 1) << (m * segs);
                if (far & row_units) which |= row_units;
            }
            __syncthreads();
            stage(std::true_type{}, which);
            __syncthreads();
            if ((int)threadIdx.x < M && ((which >> (threadIdx.x * segs)) & 1)) rho[threadIdx.x] = 1.f;
        }
    } else {
        const u32x4 xrs = raw_rsrc31(p.X, (int64_t)M * K * 2);
        const int pieces = xbytes / 16;
        for (int i0 = wave * kWave; i0 < pieces; i0 += WAVES * kWave) {
            const int i = i0 + lane, r = i % M, at = i / M;
            const int b = at / 16, c = (at >> 2) & 3, qq = at & 3, k = 128 * b + 32 * qq + 8 * c;
            if (i < pieces) dma16(xrs, k < K ? (uint32_t)((r * K + k) * 2) : kMaskedOffset, lds0 + i0 * 16);
        }
        wait_vm<0>();
        __syncthreads();
    }
    const bool live = row < M;
    const int slot = NORM && row >= kQ4NormRows ? row - kQ4NormRows + M : row;
    const bool held = NORM && row >= kQ4NormRows ? row - kQ4NormRows < M : live;
    uint32_t xat[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) xat[c] = held ? (uint32_t)(((c * 4 + q) * S + slot) * 16) : (uint32_t)xbytes;
    const uint32_t xstep = held ? (uint32_t)(256 * S) : 0u;
    f32x4 acc[NG];
#pragma unroll
    for (int j = 0; j < NG; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto step = [&](int b, Blk& f) {
        u32x4 x[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) x[c] = *reinterpret_cast<const u32x4*>(xs + xat[c] + (uint32_t)b * xstep);
#pragma unroll
        for (int j = 0; j < NG; ++j) {
            const float s = __builtin_bit_cast(float, f.s[j] << 23);
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[j] = q4_mfma_bf16(q4_to_bf16(f.w[j][c], s), x[c], acc[j]);
        }
    };
    q4_pipeline<U, WAVES>(wave, KB, even, odd, fetch_step, step);
    __syncthreads();  // the sums take the rows' place
#pragma unroll
    for (int j = 0; j < NG; ++j) red[(wave * NG + j) * kWave + lane] = acc[j];
    __syncthreads();
    if (wave < NG && g0 + wave < groups) {
        f32x4 tot = red[wave * kWave + lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) tot += red[(w * NG + wave) * kWave + lane];
        float f = 1.f;
        if constexpr (NORM) {
#pragma unroll
            for (int i = 0; i < 4; ++i) tot[i] += __shfl(tot[i], lane ^ kQ4NormRows);
            f = live ? rho[row] : 0.f;
        }
        q4_store4(p, row, (g0 + wave) * 16 + 4 * q, tot, f);
    }
}

}  // namespace pifa
