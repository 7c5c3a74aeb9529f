// Low-rank adapters of many requests beside one shared projection, forward and
// backward.  Row m has adapter a = ids[m], or none:
//
//   t = s_a (X A_a^T)      Y  = Y0 + t B_a^T
//   u = s_a (dY B_a)       dX = dX0 + u A_a,   dA_a = sum over its rows of u^T X,   dB_a = sum of dY^T t
//
// A plan sorts the rows by adapter, once a batch; every layer's call goes by it.
// Each product then runs over tiles of up to 64 rows of one adapter, wherever
// they stand in X and Y, on matrix instructions of 16 x 16 x 32 bf16 values; the
// ranks are small, so all of them are bound by the rows that they stream.
//   shrink: rows times A^T (or B), over K, in waves that take 32 columns in turn;
//           with few tiles K is cut over workgroups too.  t and u stay fp32.
//   expand: t times B^T (or u times A) onto the rows of Y0.
//   grads:  sums over rows; a lane holds 8 rows of 8 columns and turns them round
//           in its registers, so that the rows become the instruction's K.
// t and u reach the matrix cores as two bf16 values each (16 bits) where the
// result is bf16, as three (24 bits) where it is fp32.  All sums are fp32 and in a
// fixed order.
#pragma once

#include "common.hpp"

namespace pifa {

constexpr int kAdTile = 64;      // rows of a tile
constexpr int kAdPiece = 512;    // rows of an adapter that one workgroup of grads sums over
constexpr int kAdMaxSlots = 4096;
constexpr int64_t kAdMaxRows = 1 << 20;
constexpr int kAdMaxSplit = 8;   // of K
constexpr int kAdThreads = 512;
constexpr int kAdWaves = kAdThreads / kWave;

// ------------------------------------------------------------------ plan
// A plan in memory: a header, then arrays of int32.  Tiles and pieces are found
// by a binary search in their prefix sums; rows without an adapter are bucket n.
struct AdapterHeader {
    int32_t M, n;      // of the call that wrote it
    int32_t tiles;     // of rows with an adapter
    int32_t tiles_all; // with those of rows without
    int32_t active;    // rows with an adapter
    int32_t pieces;    // of all adapters; one without rows has an empty one
    int32_t multi;     // adapters of more than one piece
    int32_t pad[9];
};
struct AdapterTile {
    int32_t adapter, first;  // n: none
};
struct AdapterMulti {
    int32_t adapter, slot, pieces;  // its partial sums
};

struct AdapterPlan {
    AdapterHeader* head;
    int32_t* seg;         // n + 2: first sorted row of each adapter, of the rows without, M
    int32_t* perm;        // M: rows in the order of their adapters
    AdapterTile* tiles;   // M / 64 + min(n, M) + 1
    AdapterTile* pieces;  // M / 512 + n
    int32_t* slots;       // for each piece: its partial sums, or -1 where it is its adapter's only one
    AdapterMulti* multi;  // M / 512
    int32_t* hist;        // for each block of 1024 rows: its rows of each bucket (n + 1)
};

__host__ __device__ inline int64_t adapter_max_tiles(int64_t M, int64_t n) { return M / kAdTile + (n < M ? n : M) + 1; }
__host__ __device__ inline int64_t adapter_max_pieces(int64_t M, int64_t n) { return M / kAdPiece + n; }
__host__ __device__ inline int64_t adapter_blocks(int64_t M) { return ceil_div(M, 1024); }

// Places of a plan's arrays; returns its size in bytes.
__host__ __device__ inline size_t adapter_layout(void* base, int64_t M, int64_t n, AdapterPlan* p) {
    uint8_t* at = (uint8_t*)base;
    auto take = [&](int64_t words) {
        uint8_t* r = at;
        at += round_up(4 * words, 64);
        return (int32_t*)r;
    };
    p->head = (AdapterHeader*)take(16);
    p->seg = take(n + 2);
    p->perm = take(M);
    p->tiles = (AdapterTile*)take(2 * adapter_max_tiles(M, n));
    p->pieces = (AdapterTile*)take(2 * adapter_max_pieces(M, n));
    p->slots = take(adapter_max_pieces(M, n));
    p->multi = (AdapterMulti*)take(3 * (M / kAdPiece + 1));
    p->hist = take(adapter_blocks(M) > 1 ? adapter_blocks(M) * (n + 1) : 0);
    return (size_t)(at - (uint8_t*)base);
}

__device__ __forceinline__ int adapter_bucket(const int32_t* ids, int64_t m, int64_t M, int n) {
    const int a = m < M ? ids[m] : -1;
    return a >= 0 && a < n ? a : n;
}

static __global__ __launch_bounds__(1024) void adapter_hist(const int32_t* ids, int64_t M, int n, AdapterPlan p) {
    __shared__ int count[kAdMaxSlots + 1];
    for (int a = threadIdx.x; a <= n; a += 1024) count[a] = 0;
    __syncthreads();
    const int64_t m = (int64_t)blockIdx.x * 1024 + threadIdx.x;
    if (m < M) atomicAdd(&count[adapter_bucket(ids, m, M, n)], 1);
    __syncthreads();
    for (int a = threadIdx.x; a <= n; a += 1024) p.hist[(int64_t)blockIdx.x * (n + 1) + a] = count[a];
}

// v[i] becomes the sum of those before it, v[len] the sum of all (len + 1 <= 4 * 1024 + 2 words).
__device__ __forceinline__ void adapter_scan(int* v, int len, int* red) {
    constexpr int EACH = (kAdMaxSlots + 2 + 1023) / 1024;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    int mine[EACH], sum = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int k = t * EACH + i;
        mine[i] = k < len ? v[k] : 0;
        sum += mine[i];
    }
    int up = sum;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const int o = __shfl_up(up, s);
        up += lane >= s ? o : 0;
    }
    __syncthreads();
    if (lane == 63) red[wave] = up;
    __syncthreads();
    int base = up - sum;
    for (int w = 0; w < wave; ++w) base += red[w];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int k = t * EACH + i;
        if (k <= len) v[k] = base;
        base += mine[i];
    }
    __syncthreads();
}

// The last i with v[i] <= x, of v[0] = 0 <= ... <= v[len] and x < v[len].
__device__ __forceinline__ int adapter_find(const int* v, int len, int x) {
    int lo = 0, hi = len;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (v[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// A block of 1024 rows goes to its places: those of its adapter in the blocks
// before it, then those in the waves before, then in the lanes before.  Block 0
// also writes the header and the lists.
static __global__ __launch_bounds__(1024) void adapter_place(const int32_t* ids, int64_t M, int n, AdapterPlan p) {
    __shared__ int at[kAdMaxSlots + 2], total[kAdMaxSlots + 2], list[kAdMaxSlots + 2];
    __shared__ int red[16];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, nb = gridDim.x;
    const int64_t m = (int64_t)blockIdx.x * 1024 + t;
    const int mine = adapter_bucket(ids, m, M, n);
    for (int a = t; a <= n + 1; a += 1024) at[a] = total[a] = 0;
    __syncthreads();
    if (nb == 1) {
        if (m < M) atomicAdd(&total[mine], 1);
    } else {
        for (int a = t; a <= n; a += 1024) {
            int before = 0, all = 0;
            for (int b = 0; b < nb; ++b) {
                const int c = p.hist[(int64_t)b * (n + 1) + a];
                before += b < (int)blockIdx.x ? c : 0;
                all += c;
            }
            at[a] = before;
            total[a] = all;
        }
    }
    __syncthreads();
    for (int a = t; a <= n; a += 1024) list[a] = total[a];
    __syncthreads();
    adapter_scan(list, n + 1, red);  // first sorted row of each bucket
    for (int a = t; a <= n; a += 1024) at[a] += list[a];
    if (blockIdx.x == 0)
        for (int a = t; a <= n + 1; a += 1024) p.seg[a] = list[a];
    __syncthreads();
    for (int w = 0; w < 16 && (int64_t)blockIdx.x * 1024 + 64 * w < M; ++w) {
        if (wave == w) {
            const bool live = m < M;
            uint64_t same = __ballot(live);
            for (int b = 0; (n >> b) != 0; ++b) {
                const uint64_t set = __ballot((mine >> b) & 1);
                same &= (mine >> b) & 1 ? set : ~set;
            }
            const int rank = __popcll(same & ((1ull << lane) - 1));
            if (live) p.perm[at[mine] + rank] = (int32_t)m;
            __builtin_amdgcn_wave_barrier();
            if (live && rank == 0) at[mine] += __popcll(same);
        }
        __syncthreads();
    }
    if (blockIdx.x != 0) return;
    const int active = list[n];
    // tiles: at[] is free now
    for (int a = t; a <= n; a += 1024) at[a] = (total[a] + kAdTile - 1) / kAdTile;
    __syncthreads();
    adapter_scan(at, n + 1, red);
    const int tiles = at[n], tiles_all = at[n + 1];
    for (int i = t; i < tiles_all; i += 1024) {
        const int a = adapter_find(at, n + 1, i);
        p.tiles[i] = AdapterTile{a, list[a] + (i - at[a]) * kAdTile};
    }
    __syncthreads();
    for (int a = t; a < n; a += 1024) at[a] = max(1, (total[a] + kAdPiece - 1) / kAdPiece);
    __syncthreads();
    adapter_scan(at, n, red);
    const int pieces = at[n];
    for (int i = t; i < pieces; i += 1024) {
        const int a = adapter_find(at, n, i);
        p.pieces[i] = AdapterTile{a, list[a] + (i - at[a]) * kAdPiece};
    }
    __syncthreads();
    // adapters of more than one piece, and places for their partial sums
    __shared__ int nmulti;
    int* where = list;  // free now
    for (int a = t; a < n; a += 1024) where[a] = at[a + 1] - at[a] > 1 ? at[a + 1] - at[a] : 0;
    __syncthreads();
    adapter_scan(where, n, red);
    for (int i = t; i < pieces; i += 1024) {
        const int a = adapter_find(at, n, i);
        p.slots[i] = at[a + 1] - at[a] > 1 ? where[a] + i - at[a] : -1;
    }
    for (int a = t; a < n; a += 1024) total[a] = at[a + 1] - at[a] > 1 ? 1 : 0;
    __syncthreads();
    adapter_scan(total, n, red);
    for (int a = t; a < n; a += 1024)
        if (total[a + 1] != total[a]) p.multi[total[a]] = AdapterMulti{a, where[a], at[a + 1] - at[a]};
    if (t == 0) {
        nmulti = total[n];
        *p.head = AdapterHeader{(int32_t)M, n, tiles, tiles_all, active, pieces, nmulti, {}};
    }
}

// ------------------------------------------------------------------ shared pieces
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

struct __attribute__((packed, aligned(2))) AdapterAny16 {
    u32x4 v;
};
struct __attribute__((packed, aligned(4))) AdapterAnyF4 {
    f32x4 v;
};

// Eight values from k on of a row of K, zeros behind its end.
__device__ __forceinline__ u32x4 adapter_load8(const bf16* row, int64_t k, int64_t K) {
    if (k + 8 <= K) return reinterpret_cast<const AdapterAny16*>(row + k)->v;
    u32x4 v = zero16();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t b = k + e < K ? (uint32_t) reinterpret_cast<const uint16_t*>(row)[k + e] : 0u;
        v[e / 2] |= b << (16 * (e & 1));
    }
    return v;
}

__device__ __forceinline__ f32x4 adapter_mfma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// How many workgroups share a tile's K: as many as bring `tiles` to `target`.
__host__ __device__ inline int adapter_splits(int tiles, int64_t slices, int target) {
    int s = tiles > 0 ? (target + tiles - 1) / tiles : 1;
    if (s > kAdMaxSplit) s = kAdMaxSplit;
    const int64_t most = slices / kAdWaves;  // a slice for every wave
    if (s > most) s = (int)most;
    return s < 1 ? 1 : s;
}

// Columns of t and u in memory.
__host__ __device__ inline int64_t adapter_rp(int64_t r) { return r <= 16 ? 16 : r <= 32 ? 32 : round_up(r, 64); }

// ------------------------------------------------------------------ shrink
struct AdapterShrink {
    const bf16* P;       // rows (M x K)
    const bf16* W;       // n x r x K
    const float* scale;  // or null: ones
    float* T;            // splits x active x rp
    int64_t K;
};

template <int JB, int RG>
__device__ __forceinline__ void adapter_shrink_tile(const AdapterShrink& j, const AdapterPlan& p, const AdapterTile tile,
                                                    int rows, int64_t r, int j0, int64_t s0, int64_t s1, int64_t rp,
                                                    float* out, float* lds) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
    const bf16* x[RG];
    const bf16* w[JB];
#pragma unroll
    for (int g = 0; g < RG; ++g) x[g] = j.P + (int64_t)p.perm[tile.first + min(16 * g + i, rows - 1)] * j.K;
#pragma unroll
    for (int b = 0; b < JB; ++b)
        w[b] = j.W + ((int64_t)tile.adapter * r + min((int64_t)(j0 + 16 * b + i), r - 1)) * j.K;
    f32x4 acc[RG][JB];
#pragma unroll
    for (int g = 0; g < RG; ++g)
#pragma unroll
        for (int b = 0; b < JB; ++b) acc[g][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int64_t whole = j.K / 32;  // slices of 32 full columns
    int64_t s = s0 + wave;
    for (; s < min(s1, whole); s += kAdWaves) {
        const int64_t k = 32 * s + 8 * q;
        u32x4 xv[RG], wv[JB];
#pragma unroll
        for (int g = 0; g < RG; ++g) xv[g] = reinterpret_cast<const AdapterAny16*>(x[g] + k)->v;
#pragma unroll
        for (int b = 0; b < JB; ++b) wv[b] = reinterpret_cast<const AdapterAny16*>(w[b] + k)->v;
#pragma unroll
        for (int g = 0; g < RG; ++g)
#pragma unroll
            for (int b = 0; b < JB; ++b) acc[g][b] = adapter_mfma(xv[g], wv[b], acc[g][b]);
    }
    if (s < s1) {  // the row's last columns
        const int64_t k = 32 * s + 8 * q;
        u32x4 xv[RG], wv[JB];
#pragma unroll
        for (int g = 0; g < RG; ++g) xv[g] = adapter_load8(x[g], k, j.K);
#pragma unroll
        for (int b = 0; b < JB; ++b) wv[b] = adapter_load8(w[b], k, j.K);
#pragma unroll
        for (int g = 0; g < RG; ++g)
#pragma unroll
            for (int b = 0; b < JB; ++b) acc[g][b] = adapter_mfma(xv[g], wv[b], acc[g][b]);
    }
    // the waves' sums, 16 rows at a time, in two halves of LDS in turn
    constexpr int COLS = 16 * JB;
    const float scale = j.scale ? j.scale[tile.adapter] : 1.f;
#pragma unroll
    for (int g = 0; g < RG; ++g) {
        float* part = lds + (g & 1) * kAdWaves * 16 * COLS;
#pragma unroll
        for (int b = 0; b < JB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) part[(wave * 16 + 4 * q + e) * COLS + 16 * b + i] = acc[g][b][e];
        __syncthreads();
        for (int at = threadIdx.x; at < 16 * COLS; at += kAdThreads) {
            const int row = 16 * g + at / COLS, col = j0 + at % COLS;
            float v = 0.f;
#pragma unroll
            for (int u = 0; u < kAdWaves; ++u) v += part[u * 16 * COLS + at];
            if (row < rows) out[(int64_t)(tile.first + row) * rp + col] = col < r ? v * scale : 0.f;
        }
    }
}

// Workgroups: x: tiles, y: splits of K, z: blocks of 16 JB columns of t, jobs outermost.
template <int JB>
__global__ __launch_bounds__(kAdThreads) void adapter_shrink(AdapterShrink j0, AdapterShrink j1, AdapterPlan p, int64_t M,
                                                             int n, int64_t r, int target) {
    __shared__ float lds[2 * kAdWaves * 16 * 16 * JB];
    const AdapterHeader& h = *p.head;
    if (h.M != M || h.n != n || (int)blockIdx.x >= h.tiles) return;
    const int64_t rp = adapter_rp(r);
    const int cols = (int)ceil_div(rp, 16 * JB), job = blockIdx.z / cols, c0 = (blockIdx.z % cols) * 16 * JB;
    const AdapterShrink j = job ? j1 : j0;
    const int64_t slices = ceil_div(j.K, 32);
    const int splits = adapter_splits(h.tiles, slices, target);
    if ((int)blockIdx.y >= splits) return;
    const int64_t each = ceil_div(slices, splits), s0 = each * blockIdx.y, s1 = min(s0 + each, slices);
    const AdapterTile tile = p.tiles[blockIdx.x];
    const int rows = min(kAdTile, p.seg[tile.adapter + 1] - tile.first);
    float* out = j.T + (int64_t)blockIdx.y * h.active * rp;
    if (rows <= 16) adapter_shrink_tile<JB, 1>(j, p, tile, rows, r, c0, s0, s1, rp, out, lds);
    else adapter_shrink_tile<JB, 4>(j, p, tile, rows, r, c0, s0, s1, rp, out, lds);
}

// ------------------------------------------------------------------ expand
struct AdapterExpand {
    const float* T;    // splits x active x rp
    const bf16* W;     // n x d x r
    const bf16* base;  // or null: zeros
    bf16* out;         // M x d; may be base
    int64_t d;
    int64_t K;         // that t was summed over
};

// Eight columns from k on of a row of t, the splits' sums added.
__device__ __forceinline__ void adapter_t8(const float* t, int splits, int64_t stride, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
    for (int s = 0; s < splits; ++s) {
        const f32x4 a = reinterpret_cast<const AdapterAnyF4*>(t + s * stride)->v;
        const f32x4 b = reinterpret_cast<const AdapterAnyF4*>(t + s * stride + 4)->v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] += a[e];
            v[4 + e] += b[e];
        }
    }
}
// The nearest bf16 values, and those nearest to what they leave.
__device__ __forceinline__ void adapter_split8(const float (&v)[8], u32x4& hi, u32x4& lo) {
    bf16x8 h, l;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        h[e] = (bf16)v[e];
        l[e] = (bf16)(v[e] - (float)h[e]);
    }
    hi = __builtin_bit_cast(u32x4, h);
    lo = __builtin_bit_cast(u32x4, l);
}

// The 64 columns of W that a wave takes as operands: instruction u's row i is column
// c0 + 32 (u / 2) + 8 (i / 4) + 4 (u % 2) + i % 4, so that two instructions leave
// a lane with 8 columns in a row.
__device__ __forceinline__ u32x4 adapter_w8(const bf16* W, int64_t c0, int u, int i, int64_t d, int64_t k, int64_t r) {
    return adapter_load8(W + min(c0 + 32 * (u / 2) + 8 * (i / 4) + 4 * (u % 2) + i % 4, d - 1) * r, k, r);
}

// Workgroups: x: 64 columns a wave, y: tiles (those of rows without an adapter
// last, which are copied).  KB: blocks of 32 columns of t, whose operands of W
// stay in registers over the tile's rows; 0: up to 16 columns, both halves of t
// in one instruction; -1: any number, read again for every 16 rows.
template <int KB>
__global__ __launch_bounds__(256) void adapter_expand(AdapterExpand j, AdapterPlan p, int64_t M, int n, int64_t r,
                                                      int target) {
    const AdapterHeader& h = *p.head;
    if (h.M != M || h.n != n || (int)blockIdx.y >= h.tiles_all) return;
    const AdapterTile tile = p.tiles[blockIdx.y];
    const bool none = tile.adapter >= n;
    if (none && j.out == j.base) return;
    const int rows = min(kAdTile, p.seg[tile.adapter + 1] - tile.first);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
    const int64_t c0 = ((int64_t)blockIdx.x * 4 + wave) * 64;
    if (c0 >= j.d) return;
    const int groups = (rows + 15) / 16;
    const int64_t rp = adapter_rp(r), stride = (int64_t)h.active * rp;
    const int splits = none ? 0 : adapter_splits(h.tiles, ceil_div(j.K, 32), target);
    const bf16* W = j.W + (int64_t)(none ? 0 : tile.adapter) * j.d * r;
    constexpr int KW = KB > 0 ? KB : 1;
    u32x4 w[KW][4];
    if (KB >= 0 && !none) {
#pragma unroll
        for (int b = 0; b < KW; ++b)
#pragma unroll
            for (int u = 0; u < 4; ++u) w[b][u] = adapter_w8(W, c0, u, i, j.d, KB == 0 ? 8 * (q & 1) : 32 * b + 8 * q, r);
    }
    for (int g = 0; g < groups; ++g) {
        const int pos = tile.first + min(16 * g + i, rows - 1);
        const int64_t row = (int64_t)p.perm[pos] * j.d;
        u32x4 base[2] = {zero16(), zero16()};
        if (j.base) {
#pragma unroll
            for (int u = 0; u < 2; ++u) base[u] = adapter_load8(j.base + row, min(c0 + 32 * u + 8 * q, j.d), j.d);
        }
        f32x4 acc[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) acc[u] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (!none) {
            const float* t = j.T + (int64_t)pos * rp;
            float v[8];
            u32x4 hi, lo;
            if constexpr (KB == 0) {
                adapter_t8(t + 8 * (q & 1), splits, stride, v);
                adapter_split8(v, hi, lo);
#pragma unroll
                for (int u = 0; u < 4; ++u) acc[u] = adapter_mfma(w[0][u], q < 2 ? hi : lo, acc[u]);
            } else {
                auto block = [&](int64_t k, const u32x4(&wk)[4]) {
                    adapter_t8(t + k, splits, stride, v);
                    adapter_split8(v, hi, lo);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        acc[u] = adapter_mfma(wk[u], hi, acc[u]);
                        acc[u] = adapter_mfma(wk[u], lo, acc[u]);
                    }
                };
                if constexpr (KB > 0) {
#pragma unroll
                    for (int b = 0; b < KB; ++b) block(32 * b + 8 * q, w[b]);
                } else {
                    for (int64_t k = 8 * q; k < rp; k += 32) {
#pragma unroll
                        for (int u = 0; u < 4; ++u) w[0][u] = adapter_w8(W, c0, u, i, j.d, k, r);
                        block(k, w[0]);
                    }
                }
            }
        }
        if (16 * g + i < rows) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int64_t c = c0 + 32 * u + 8 * q;
                bf16x8 y, b = __builtin_bit_cast(bf16x8, base[u]);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = none ? b[e] : (bf16)((float)b[e] + acc[2 * u + e / 4][e % 4]);
                if (c + 8 <= j.d) {
                    reinterpret_cast<AdapterAny16*>(j.out + row + c)->v = __builtin_bit_cast(u32x4, y);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (c + e < j.d) j.out[row + c + e] = y[e];
                }
            }
        }
    }
}

// ------------------------------------------------------------------ backward
// W (n x rows x cols) to its transpose (n x cols x rows), of adapters that have rows.
static __global__ __launch_bounds__(256) void adapter_transpose(const bf16* A, bf16* At, int64_t ar, int64_t ac,
                                                               const bf16* B, bf16* Bt, int64_t br, int64_t bc,
                                                               AdapterPlan p, int64_t M, int n) {
    __shared__ uint16_t tile[64][66];
    if (p.head->M != M || p.head->n != n) return;
    const int a = blockIdx.y;
    if (p.seg[a] == p.seg[a + 1]) return;
    const int64_t ta = ceil_div(ar, 64) * ceil_div(ac, 64);
    const bool second = (int64_t)blockIdx.x >= ta;
    const int64_t t = second ? blockIdx.x - ta : blockIdx.x, rows = second ? br : ar, cols = second ? bc : ac;
    const uint16_t* from = (const uint16_t*)(second ? B : A) + a * rows * cols;
    uint16_t* to = (uint16_t*)(second ? Bt : At) + a * rows * cols;
    const int64_t r0 = t / ceil_div(cols, 64) * 64, c0 = t % ceil_div(cols, 64) * 64;
    for (int k = threadIdx.x; k < 64 * 64; k += 256) {
        const int64_t row = r0 + k / 64, col = c0 + k % 64;
        if (row < rows && col < cols) tile[k / 64][k % 64] = from[row * cols + col];
    }
    __syncthreads();
    for (int k = threadIdx.x; k < 64 * 64; k += 256) {
        const int64_t col = c0 + k / 64, row = r0 + k % 64;
        if (row < rows && col < cols) to[col * rows + row] = tile[k % 64][k / 64];
    }
}

struct AdapterGrads {
    const bf16* P;    // rows (M x d)
    const float* T;   // splits x active x rp
    float* out;       // n x r x d (by_column: n x d x r)
    float* part;      // the same of one adapter for each slot
    int64_t d;
    int64_t K;        // that t was summed over
    bool by_column;
};

// v as three bf16 values that add up to all its bits.
__device__ __forceinline__ void adapter_split3(float v, bf16 (&s)[3]) {
    s[0] = (bf16)v;
    v -= (float)s[0];
    s[1] = (bf16)v;
    s[2] = (bf16)(v - (float)s[1]);
}

constexpr int kAdCols = 128;  // columns of P that a workgroup of grads takes

// Workgroups: x: columns of both jobs, y: pieces, z: blocks of 16 JB columns of t.
// Each wave takes 32 rows at a time: 8 loads of 8 columns a lane, 8 rows apart
// from lane group to lane group, turned round to 8 operands of 8 rows each.
template <int JB>
__global__ __launch_bounds__(kAdThreads) void adapter_grads(AdapterGrads j0, AdapterGrads j1, int blocks0, AdapterPlan p,
                                                            int64_t M, int n, int64_t r, int target) {
    constexpr int COLS = 16 * JB;
    constexpr int kPitch = 32 + 8;  // rows of a column of t in LDS, padded
    union alignas(16) Shared {
        uint16_t t[kAdWaves][3][COLS][kPitch];
        struct {
            float part[2][kAdWaves][16 * COLS];
            float out[COLS][kAdCols + 1];
        } sum;
    };
    __shared__ Shared lds;
    const AdapterHeader& h = *p.head;
    if (h.M != M || h.n != n || (int)blockIdx.y >= h.pieces) return;
    const bool second = (int)blockIdx.x >= blocks0;
    const AdapterGrads j = second ? j1 : j0;
    const int64_t c0 = (int64_t)(second ? blockIdx.x - blocks0 : blockIdx.x) * kAdCols;
    const int b0 = blockIdx.z * COLS;
    const AdapterTile piece = p.pieces[blockIdx.y];
    const int slot = p.slots[blockIdx.y];
    const int rows = min(kAdPiece, p.seg[piece.adapter + 1] - piece.first);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
    const int64_t rp = adapter_rp(r), stride = (int64_t)h.active * rp;
    const int splits = adapter_splits(h.tiles, ceil_div(j.K, 32), target);

    f32x4 acc[8][JB];
#pragma unroll
    for (int c = 0; c < 8; ++c)
#pragma unroll
        for (int b = 0; b < JB; ++b) acc[c][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int m0 = 32 * wave; m0 < rows; m0 += 32 * kAdWaves) {
        u32x4 x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int m = m0 + 8 * q + e;
            x[e] = zero16();
            if (m < rows) x[e] = adapter_load8(j.P + (int64_t)p.perm[piece.first + m] * j.d, min(c0 + 8 * i, j.d), j.d);
        }
        // t of these rows, as three bf16 values, with the rows of a column in a row
        for (int k = lane; k < 32 * COLS / 4; k += kWave) {
            const int m = k / (COLS / 4), col = k % (COLS / 4) * 4;
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
            if (m0 + m < rows) {
                const float* from = j.T + (int64_t)(piece.first + m0 + m) * rp + b0 + col;
                for (int s = 0; s < splits; ++s) v += reinterpret_cast<const AdapterAnyF4*>(from + s * stride)->v;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                bf16 s[3];
                adapter_split3(v[e], s);
#pragma unroll
                for (int u = 0; u < 3; ++u) lds.t[wave][u][col + e][m] = __builtin_bit_cast(uint16_t, s[u]);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        u32x4 turned[8];
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e)  // rows 2e, 2e + 1 of column 8 i + c
                turned[c][e] = __builtin_amdgcn_perm(x[2 * e + 1][c / 2], x[2 * e][c / 2], c & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int u = 0; u < 3; ++u)
#pragma unroll
            for (int b = 0; b < JB; ++b) {
                const u32x4 tv = *reinterpret_cast<const u32x4*>(&lds.t[wave][u][16 * b + i][8 * q]);
#pragma unroll
                for (int c = 0; c < 8; ++c) acc[c][b] = adapter_mfma(turned[c], tv, acc[c][b]);
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    // the waves' sums: acc[c][b], row 4 q + e is column 8 (4 q + e) + c of P, column i is column 16 b + i of t
#pragma unroll
    for (int c = 0; c < 8; ++c) {
#pragma unroll
        for (int b = 0; b < JB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) lds.sum.part[c & 1][wave][(4 * q + e) * COLS + 16 * b + i] = acc[c][b][e];
        __syncthreads();
        for (int at = threadIdx.x; at < 16 * COLS; at += kAdThreads) {
            float v = 0.f;
#pragma unroll
            for (int u = 0; u < kAdWaves; ++u) v += lds.sum.part[c & 1][u][at];
            lds.sum.out[at % COLS][8 * (at / COLS) + c] = v;
        }
    }
    __syncthreads();
    float* out = slot < 0 ? j.out + piece.adapter * r * j.d : j.part + slot * r * j.d;
    const int cols = (int)min((int64_t)kAdCols, j.d - c0), js = (int)min((int64_t)COLS, r - b0);
    for (int at = threadIdx.x; at < COLS * kAdCols; at += kAdThreads) {
        const int a = j.by_column ? at % COLS : at / kAdCols, c = j.by_column ? at / COLS : at % kAdCols;
        if (a >= js || c >= cols) continue;
        out[j.by_column ? (c0 + c) * r + b0 + a : (b0 + a) * j.d + c0 + c] = lds.sum.out[a][c];
    }
}

// Gradients of adapters of more than one piece: their partial sums, in order.
// Workgroups: x: values of both gradients, 1024 each, y: adapters.
static __global__ __launch_bounds__(256) void adapter_sum(const float* part0, float* out0, int64_t n0, int blocks0,
                                                         const float* part1, float* out1, int64_t n1, AdapterPlan p,
                                                         int64_t M, int n) {
    if (p.head->M != M || p.head->n != n || (int)blockIdx.y >= p.head->multi) return;
    const AdapterMulti a = p.multi[blockIdx.y];
    const bool second = (int)blockIdx.x >= blocks0;
    const int64_t count = second ? n1 : n0;
    const float* from = (second ? part1 : part0) + a.slot * count;
    float* to = (second ? out1 : out0) + a.adapter * count;
    const int64_t first = (int64_t)(second ? blockIdx.x - blocks0 : blockIdx.x) * 1024;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int64_t k = first + e * 256 + threadIdx.x;
        if (k >= count) continue;
        float v = from[k];
        for (int s = 1; s < a.pieces; ++s) v += from[s * count + k];
        to[k] = v;
    }
}

}  // namespace pifa
