// Low-rank adapters of many requests beside one shared projection, forward and
// backward.  Row m has adapter a = ids[m], or none:
//
//   t = s_a (X A_a^T)      Y  = Y0 + t B_a^T
//   u = s_a (dY B_a)       dX = dX0 + u A_a,   dA_a = sum over its rows of u^T X,   dB_a = sum of dY^T t
//
// A plan deals the rows to tiles of up to 64 rows of one adapter, once a batch;
// every layer's call goes by it.  The products run on matrix instructions of 16 x
// 16 x 32 bf16 values; the ranks are small, so that all of them are bound by the
// rows that they stream, wherever these stand in X and Y.
//   shrink: rows times A^T (or B), in waves that take 64 columns in turn; K is cut
//           over workgroups too, as far as the chip is not full of tiles.
//   finish: the parts' sums, rounded as the next products read them.
//   expand: t times B^T (or u times A) onto the rows of Y0.
//   grads:  sums over rows; a lane holds 8 rows of 8 columns and turns them round
//           in its registers, so that the rows become the instruction's K.
// t and u are fp32 sums; they reach the matrix cores as two bf16 values each (16
// bits) where the result is bf16, as three (24 bits) where it is fp32.  The parts
// behind the first have either sign or none, and beside an infinite operand would
// make no number of an infinity; so their products are summed first and kept finite,
// and what the first part, of t's own sign, adds decides.  All sums are fp32 and in a
// fixed order.
// us of each kernel: 1999 rows of 4096 -> 11008, rank 64: shrink 12, finish 4,
// expand 21 to 23; gradients of 4096 rows of 4096 x 4096, rank 16: shrink of both
// jobs 17 (67 MB), finish 4, expand 14 to 17 (67 MB), grads 15 (67 MB), sum 4; of 333
// rows of 1024 -> 1536, rank 24: 6, 4, 4, 8.  Small calls are chains of launches,
// each of which waits for the header, then rows, then their data.
#pragma once

#include "common.hpp"
#include "streamed.hpp"

namespace pifa {

constexpr int kAdTile = 64;        // rows of a tile
// Tiles of an adapter that one workgroup of grads sums over (32: 4096 rows of 4 adapters
// 55.0 us instead of 55.5, 2565 rows of one, 2102 -> 531, 53.3 instead of 39.7).
constexpr int kAdPieceTiles = 8;
constexpr int kAdPiece = kAdTile * kAdPieceTiles;
constexpr int kAdMaxSlots = 4096;
constexpr int64_t kAdMaxRows = 1 << 20;
constexpr int kAdMaxSplit = 8;     // of K
constexpr int kAdThreads = 256;    // of expand
constexpr int kAdWaves = 4;        // of shrink
constexpr int kAdSlice = 64;       // columns that a wave of shrink takes at a time

// ------------------------------------------------------------------ plan
// A plan in memory: a header, then arrays of int32.  Rows without an adapter are
// bucket n, whose tiles come last.
struct AdapterHeader {
    int32_t M, n;       // of the call that wrote it
    int32_t tiles;      // of rows with an adapter
    int32_t tiles_all;  // with those of rows without
    int32_t pieces;     // of all adapters; one without rows has one of no tiles
    int32_t multi;      // adapters of more than one piece
    int32_t pad[10];
};
struct AdapterTile {
    int32_t adapter, count;  // of its 64 rows, those that are there
};
struct AdapterPiece {
    int32_t adapter, first, tiles;
    int32_t slot;  // its partial sums, or -1 where it is its adapter's only one
};
struct AdapterMulti {
    int32_t adapter, slot, pieces;
};

struct AdapterPlan {
    AdapterHeader* head;
    AdapterTile* tiles;    // M / 64 + min(n, M) + 1
    int32_t* rows;         // 64 of each tile, -1 behind the last one
    AdapterPiece* pieces;  // M / 512 + n
    AdapterMulti* multi;   // M / 512
    int32_t* hist;         // for each block of 1024 rows: its rows of each bucket (n + 1)
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
    p->tiles = (AdapterTile*)take(2 * adapter_max_tiles(M, n));
    p->rows = take(kAdTile * adapter_max_tiles(M, n));
    p->pieces = (AdapterPiece*)take(4 * adapter_max_pieces(M, n));
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

// v[i] becomes the sum of those before it, v[len] the sum of all (len <= kAdMaxSlots + 1).
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

// Once a batch.  Bound by its own steps, scans of n + 1 places and their barriers:
// 48 rows 8 us, 4096 rows 13.  Every block adds up the counts of all blocks, which
// grows with their number squared and with n: both launches of 65536 rows of 16
// adapters take 27 us, of 2^20 rows 450; of 4096 adapters 125 and 4600.
// A block of 1024 rows goes to its places: those of its adapter in the blocks
// before it, then those in the waves before, then in the lanes before.  Block 0
// also writes the header and the lists.
static __global__ __launch_bounds__(1024) void adapter_place(const int32_t* ids, int64_t M, int n, AdapterPlan p) {
    __shared__ int at[kAdMaxSlots + 2], total[kAdMaxSlots + 2], tile0[kAdMaxSlots + 2];
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
    for (int a = t; a <= n; a += 1024) tile0[a] = (total[a] + kAdTile - 1) / kAdTile;
    __syncthreads();
    adapter_scan(tile0, n + 1, red);  // first tile of each bucket
    for (int w = 0; w < 16 && (int64_t)blockIdx.x * 1024 + 64 * w < M; ++w) {
        if (wave == w) {
            const bool live = m < M;
            uint64_t same = __ballot(live);
            for (int b = 0; (n >> b) != 0; ++b) {
                const uint64_t set = __ballot((mine >> b) & 1);
                same &= (mine >> b) & 1 ? set : ~set;
            }
            const int rank = __popcll(same & ((1ull << lane) - 1));
            if (live) p.rows[(int64_t)tile0[mine] * kAdTile + at[mine] + rank] = (int32_t)m;
            __builtin_amdgcn_wave_barrier();
            if (live && rank == 0) at[mine] += __popcll(same);
        }
        __syncthreads();
    }
    if (blockIdx.x != 0) return;
    const int tiles = tile0[n], tiles_all = tile0[n + 1];
    for (int i = t; i < tiles_all; i += 1024) {
        const int a = adapter_find(tile0, n + 1, i);
        p.tiles[i] = AdapterTile{a, min(kAdTile, total[a] - (i - tile0[a]) * kAdTile)};
    }
    for (int a = wave; a <= n; a += 16) {  // a wave each: the last tile's rows that are not there
        const int64_t last = (int64_t)tile0[a + 1] * kAdTile, end = (int64_t)tile0[a] * kAdTile + total[a];
        if (end + lane < last) p.rows[end + lane] = -1;
    }
    __syncthreads();
    auto piece_count = [&](int a) { return max(1, (total[a] + kAdPiece - 1) / kAdPiece); };
    for (int a = t; a < n; a += 1024) at[a] = piece_count(a);
    __syncthreads();
    adapter_scan(at, n, red);  // first piece of each adapter
    // places for the partial sums of adapters of more than one piece, behind the first pieces' LDS
    __shared__ int slot0[kAdMaxSlots + 2], multi0[kAdMaxSlots + 2];
    for (int a = t; a < n; a += 1024) {
        const int k = piece_count(a);
        slot0[a] = k > 1 ? k : 0;
        multi0[a] = k > 1 ? 1 : 0;
    }
    __syncthreads();
    adapter_scan(slot0, n, red);
    adapter_scan(multi0, n, red);
    const int pieces = at[n];
    for (int i = t; i < pieces; i += 1024) {
        const int a = adapter_find(at, n, i), first = tile0[a] + (i - at[a]) * kAdPieceTiles;
        p.pieces[i] = AdapterPiece{a, first, min(kAdPieceTiles, tile0[a + 1] - first),
                                   at[a + 1] - at[a] > 1 ? slot0[a] + i - at[a] : -1};
    }
    for (int a = t; a < n; a += 1024)
        if (multi0[a + 1] != multi0[a]) p.multi[multi0[a]] = AdapterMulti{a, slot0[a], at[a + 1] - at[a]};
    if (t == 0) *p.head = AdapterHeader{(int32_t)M, n, tiles, tiles_all, pieces, multi0[n], {}};
}

// ------------------------------------------------------------------ shared pieces
struct __attribute__((packed, aligned(2))) AdapterAny16 {
    u32x4 v;
};

__device__ __forceinline__ u32x4 adapter_load(const bf16* p) { return reinterpret_cast<const AdapterAny16*>(p)->v; }

// Eight values from k on of a row of K, zeros behind its end.
__device__ __forceinline__ u32x4 adapter_load8(const bf16* row, int64_t k, int64_t K) {
    if (k + 8 <= K) return adapter_load(row + k);
    u32x4 v = zero16();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t b = k + e < K ? (uint32_t) reinterpret_cast<const uint16_t*>(row)[k + e] : 0u;
        v[e / 2] |= b << (16 * (e & 1));
    }
    return v;
}

// The same of rows of at least 8 values, without a branch (whose end would wait for
// all loads): the row's last eight, moved down.
__device__ __forceinline__ u32x4 adapter_edge8(const bf16* row, int64_t k, int64_t K) {
    const int64_t at = min(k, K - 8);
    u32x4 v = adapter_load(row + at);
    const int s = (int)min(k - at, (int64_t)8);  // values to move
    const u32x4 z = zero16();
    if (s & 4) v = u32x4{v[2], v[3], 0u, 0u};
    if (s & 2) v = u32x4{v[1], v[2], v[3], 0u};
    const uint32_t odd = (s & 1) ? 16 : 0;
    v = u32x4{__builtin_amdgcn_alignbit(v[1], v[0], odd), __builtin_amdgcn_alignbit(v[2], v[1], odd),
              __builtin_amdgcn_alignbit(v[3], v[2], odd), v[3] >> odd};
    return s == 8 ? z : v;
}

__device__ __forceinline__ f32x4 adapter_mfma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Of 16 columns: a lane has four values of each.
__device__ __forceinline__ f32x4 adapter_mfma16(uint2 a, uint2 b, f32x4 c) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, a), __builtin_bit_cast(s16x4, b), c, 0, 0, 0);
}

// Infinities and what is no number made finite.
__device__ __forceinline__ f32x4 adapter_finite(f32x4 v) {
    constexpr float most = 0x1.FFFFFEp127f;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __builtin_amdgcn_fmed3f(v[e], -most, most);
    return v;
}

// Two rows' values in a register each: the lower or the upper ones of both.
__device__ __forceinline__ uint32_t adapter_pair(uint32_t even, uint32_t odd, int half) {
    return __builtin_amdgcn_perm(odd, even, half ? 0x07060302u : 0x05040100u);
}

// How many workgroups share a tile's K: as many as leave all of them, `target` at
// most, on the chip at once.
__host__ __device__ inline int adapter_splits(int tiles, int64_t K, int target) {
    int s = tiles > 0 ? target / tiles : 1;
    if (s > kAdMaxSplit) s = kAdMaxSplit;
    const int64_t most = ceil_div(K, kAdSlice) / kAdWaves;  // a slice for every wave
    if (s > most) s = (int)most;
    return s < 1 ? 1 : s;
}

// Columns of t and u in memory.
__host__ __device__ inline int64_t adapter_rp(int64_t r) { return r <= 16 ? 16 : r <= 32 ? 32 : round_up(r, 64); }

// ------------------------------------------------------------------ shrink
struct AdapterShrink {
    const bf16* P;       // rows (M x K)
    const bf16* W;       // n x r x K, or
    bool by_column;      // n x K x r
    const float* scale;  // or null: ones
    float* T;            // splits x 64 tiles x rp
    int64_t K;
};

// A tile's rows (RG groups of 16) times 16 JB of an adapter's; slices s0 to s1 of
// 64 columns, the waves taking them in turn.  The matrix instruction's operands have a
// row in each of 16 neighbouring lanes, which the caches would serve one by one; so
// a wave loads lines of 128 bytes, eight neighbouring lanes each, and turns them in
// LDS of its own (16-byte places of a row exchanged by its number, so that
// neighbouring rows' are in other banks).  The next slice is on its way meanwhile.
// COL: the adapter's columns lie in the rows of W; a lane takes eight of them from
// 2 JB neighbouring rows and turns these round first.  Columns past the rank are left
// out of t; where the rank is no multiple of 8 they come from the rows behind, and
// slices whose rows have not enough rows behind them end the loop like those of the
// last columns.
template <int JB, int RG, bool COL>
__device__ __forceinline__ void adapter_shrink_tile(const AdapterShrink& j, const int32_t* rows, const AdapterTile tile,
                                                    int64_t r, int j0, int64_t s0, int64_t s1, int64_t rp, float* out,
                                                    u32x4* lds) {
    constexpr int NX = 2 * RG, NW = 2 * JB;  // loads of a slice: 8 rows each
    constexpr int WAVES = kAdWaves;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
    const int row8 = lane >> 3, c8 = lane & 7;
    const bf16* x[NX];
    const bf16* w[NW];
#pragma unroll
    for (int k = 0; k < NX; ++k) x[k] = j.P + (int64_t)rows[min(8 * k + row8, tile.count - 1)] * j.K + 8 * c8;
    const int piece = lane % NW, group = lane / NW;  // COL: columns 8 piece on, of rows NW group on
    const int col = j0 + 8 * piece;
#pragma unroll
    for (int k = 0; k < NW; ++k)
        w[k] = j.W + (COL ? ((int64_t)tile.adapter * j.K + NW * group + k) * r + (r % 8 != 0 || col < r ? col : 0)
                          : ((int64_t)tile.adapter * r + min((int64_t)(j0 + 8 * k + row8), r - 1)) * j.K + 8 * c8);
    f32x4 acc[RG][JB];
#pragma unroll
    for (int g = 0; g < RG; ++g)
#pragma unroll
        for (int b = 0; b < JB; ++b) acc[g][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    u32x4* mine = lds + wave * (NX + NW) * kWave;
    u32x4 f[NX + NW];
    auto load = [&](int64_t s) {
#pragma unroll
        for (int k = 0; k < NX; ++k) f[k] = adapter_load(x[k] + kAdSlice * s);
#pragma unroll
        for (int k = 0; k < NW; ++k) f[NX + k] = adapter_load(w[k] + kAdSlice * s * (COL ? r : 1));
    };
    auto turn = [&] {
#pragma unroll
        for (int k = 0; k < (COL ? NX : NX + NW); ++k) {
            const int row = 8 * k + row8;
            mine[row * 8 + (c8 ^ (row >> 1 & 7))] = f[k];
        }
        if constexpr (COL) {
            struct alignas(2 * NW) Run {  // of a column, NW rows
                uint32_t v[NW / 2];
            };
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                Run v;
#pragma unroll
                for (int k = 0; k < NW / 2; ++k) v.v[k] = adapter_pair(f[NX + 2 * k][e / 2], f[NX + 2 * k + 1][e / 2], e & 1);
                const int row = 8 * piece + e, at = NW * group;
                *((Run*)(mine + (8 * NX + row) * 8 + ((at / 8) ^ (row >> 1 & 7))) + at % 8 / NW) = v;
            }
        }
    };
    auto multiply = [&] {
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // 32 columns each
            u32x4 a[RG], b[JB];
#pragma unroll
            for (int g = 0; g < RG; ++g) a[g] = mine[(16 * g + i) * 8 + ((4 * h + q) ^ (i >> 1 & 7))];
#pragma unroll
            for (int k = 0; k < JB; ++k) b[k] = mine[(8 * NX + 16 * k + i) * 8 + ((4 * h + q) ^ (i >> 1 & 7))];
#pragma unroll
            for (int g = 0; g < RG; ++g)
#pragma unroll
                for (int k = 0; k < JB; ++k) acc[g][k] = adapter_mfma(a[g], b[k], acc[g][k]);
        }
    };
    // slices of 64 full columns; behind them one or two, for different waves
    const int64_t behind = COL && r % 8 != 0 ? max((int64_t)0, ceil_div(j0 + 16 * JB, r) - 1) : 0;
    const int64_t whole = min(s1, max((int64_t)0, j.K - behind) / kAdSlice);
    const int64_t first = s0 + wave, count = first < whole ? (whole - first + WAVES - 1) / WAVES : 0;
    if (count > 0) {
        const int64_t last = first + (count - 1) * WAVES;
        load(first);
        for (int64_t c = 0; c < count; ++c) {
            turn();
            load(min(first + (c + 1) * WAVES, last));
            __builtin_amdgcn_sched_barrier(0);
            multiply();
        }
    }
    if (const int64_t s = first + count * WAVES; s < s1) {
        auto rest = [&](auto load8) {
#pragma unroll
            for (int k = 0; k < NX; ++k) f[k] = load8(x[k] - 8 * c8, kAdSlice * s + 8 * c8, j.K);
#pragma unroll
            for (int k = 0; k < NW; ++k) {
                if constexpr (COL) {
                    const int64_t at = kAdSlice * s + NW * group + k;  // row of W
                    f[NX + k] = load8(j.W + ((int64_t)tile.adapter * j.K + min(at, j.K - 1)) * r, (int64_t)col, r);
                    f[NX + k] = at < j.K ? f[NX + k] : zero16();
                } else {
                    f[NX + k] = load8(w[k] - 8 * c8, kAdSlice * s + 8 * c8, j.K);
                }
            }
        };
        if (j.K >= 8 && r >= 8) rest([](const bf16* row, int64_t k, int64_t K) { return adapter_edge8(row, k, K); });
        else rest([](const bf16* row, int64_t k, int64_t K) { return adapter_load8(row, k, K); });
        turn();
        multiply();
    }
    // the waves' sums
    constexpr int COLS = 16 * JB, PITCH = COLS + 4;  // the lanes of an instruction's four rows in other banks
    const float scale = j.scale ? j.scale[tile.adapter] : 1.f;
    float* part = (float*)lds;
    __syncthreads();
#pragma unroll
    for (int g = 0; g < RG; ++g)
#pragma unroll
        for (int b = 0; b < JB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) part[((wave * RG + g) * 16 + 4 * q + e) * PITCH + 16 * b + i] = acc[g][b][e];
    __syncthreads();
    for (int at = threadIdx.x; at < 16 * RG * COLS; at += WAVES * kWave) {
        const int row = at / COLS, c = at % COLS;
        float v = 0.f;
#pragma unroll
        for (int u = 0; u < WAVES; ++u) v += part[(u * 16 * RG + row) * PITCH + c];
        if (row < tile.count) out[(int64_t)row * rp + j0 + c] = j0 + c < r ? v * scale : 0.f;
    }
}

// Workgroups: x: tiles, y: parts of K, z: blocks of 16 JB columns of t, jobs outermost.
// Four waves, so that registers (146 for up to 16 columns, 240 for 64) and LDS hold
// three or two workgroups on a CU (4096 rows of 4096 twice, rank 16: 17.2 us; eight
// waves, one workgroup a CU, 18.4).
template <int JB>
__global__ __launch_bounds__(kAdWaves * kWave, JB == 1 ? 3 : 2) void adapter_shrink(AdapterShrink j0, AdapterShrink j1, AdapterPlan p,
                                                                                   int64_t M, int n, int64_t r, int target) {
    constexpr int WAVES = kAdWaves, SLICES = WAVES * (8 + 2 * JB) * kWave,
                  SUMS = WAVES * kAdTile * (16 * JB + 4) / 4;  // of 16 bytes
    __shared__ u32x4 lds[SLICES > SUMS ? SLICES : SUMS];
    const AdapterHeader h = *p.head;
    const AdapterTile tile = p.tiles[blockIdx.x];
    if (h.M != M || h.n != n || (int)blockIdx.x >= h.tiles) return;
    const int64_t rp = adapter_rp(r);
    const int cols = (int)ceil_div(rp, 16 * JB), job = blockIdx.z / cols, c0 = (blockIdx.z % cols) * 16 * JB;
    const AdapterShrink j = job ? j1 : j0;
    const int splits = adapter_splits(h.tiles, j.K, target);
    if ((int)blockIdx.y >= splits) return;
    const int64_t slices = ceil_div(j.K, kAdSlice);
    const int64_t each = ceil_div(slices, splits), s0 = each * blockIdx.y, s1 = min(s0 + each, slices);
    const int32_t* rows = p.rows + (int64_t)blockIdx.x * kAdTile;
    float* out = j.T + ((int64_t)blockIdx.y * h.tiles + blockIdx.x) * kAdTile * rp;
    if (j.by_column) {
        if (tile.count <= 16) adapter_shrink_tile<JB, 1, true>(j, rows, tile, r, c0, s0, s1, rp, out, lds);
        else adapter_shrink_tile<JB, 4, true>(j, rows, tile, r, c0, s0, s1, rp, out, lds);
    } else {
        if (tile.count <= 16) adapter_shrink_tile<JB, 1, false>(j, rows, tile, r, c0, s0, s1, rp, out, lds);
        else adapter_shrink_tile<JB, 4, false>(j, rows, tile, r, c0, s0, s1, rp, out, lds);
    }
}

// ------------------------------------------------------------------ finish
// What is left over a part; nothing over an infinite one or no number.
__device__ __forceinline__ float adapter_rest(float v, bf16 part) {
    const float rest = v - (float)part;
    return fabsf(rest) <= 3.402823466e38f ? rest : 0.f;
}
// The nearest bf16 value, and that nearest to what it leaves.
__device__ __forceinline__ void adapter_split2(float v, bf16& hi, bf16& lo) {
    hi = (bf16)v;
    lo = (bf16)adapter_rest(v, hi);
}
// v as three bf16 values that add up to all its bits.
__device__ __forceinline__ void adapter_split3(float v, bf16 (&s)[3]) {
    adapter_split2(v, s[0], s[1]);
    s[2] = (bf16)(adapter_rest(v, s[0]) - (float)s[1]);
}

// t as operands in the order of a wave's lanes, 16 bytes each:
//   halves: for each group of 16 rows and 32 columns, the values' and what they
//           leave (up to 16 columns: four values and four of what they leave in one);
//   turned: for 32 rows and 16 columns, three parts, K along the rows.
struct AdapterFinish {
    const float* T;  // splits x 64 tiles x rp
    u32x4* halves;   // or null
    u32x4* turned;   // or null
    int64_t K;       // that t was summed over
};
__device__ __forceinline__ int64_t adapter_half_at(int64_t group, int64_t rp, int64_t k32, int lo) {
    return (rp == 16 ? group : (group * (rp / 32) + k32) * 2 + lo) * kWave;
}
__device__ __forceinline__ int64_t adapter_turned_at(int64_t step, int64_t rp, int part, int64_t c16) {
    return ((step * 3 + part) * (rp / 16) + c16) * kWave;
}

// Four columns of a row of t, the parts' sums added, all parts' loads in flight.
__device__ __forceinline__ f32x4 adapter_t4(const float* t, int splits, int64_t stride) {
    f32x4 part[kAdMaxSplit], v;
#pragma unroll
    for (int s = 0; s < kAdMaxSplit; ++s) part[s] = *reinterpret_cast<const f32x4*>(t + (s < splits ? s : 0) * stride);
    v = part[0];
#pragma unroll
    for (int s = 1; s < kAdMaxSplit; ++s)
        if (s < splits) v += part[s];
    return v;
}

// A launch of its own, so that each part is added up and rounded once, not by every
// workgroup that reads it (which, up to 256 rows, the forward's expand does instead).
// Workgroups: x: tiles, y: blocks of 16 columns, z: jobs.
static __global__ __launch_bounds__(256) void adapter_finish(AdapterFinish j0, AdapterFinish j1, AdapterPlan p, int64_t M,
                                                            int n, int64_t r, int target) {
    __shared__ float lds[kAdTile][17];
    const AdapterHeader h = *p.head;
    const AdapterTile tile = p.tiles[blockIdx.x];
    if (h.M != M || h.n != n || (int)blockIdx.x >= h.tiles) return;
    const AdapterFinish j = blockIdx.z ? j1 : j0;
    const int64_t rp = adapter_rp(r), x = blockIdx.x;
    const int t = threadIdx.x, y = blockIdx.y;
    {
        const int row = t >> 2, c = (t & 3) * 4;
        f32x4 v = adapter_t4(j.T + (x * kAdTile + row) * rp + 16 * y + c, adapter_splits(h.tiles, j.K, target),
                             (int64_t)h.tiles * kAdTile * rp);
#pragma unroll
        for (int e = 0; e < 4; ++e) lds[row][c + e] = row < tile.count ? v[e] : 0.f;
    }
    __syncthreads();
    if (j.halves && t < 128) {  // 64 rows x 2 of 8 columns
        const int row = t & 63, c = t >> 6, lane = row & 15;
        bf16x8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            bf16 a, b;
            adapter_split2(lds[row][8 * c + e], a, b);
            hi[e] = a;
            lo[e] = b;
        }
        const int64_t group = x * 4 + row / 16;
        const u32x4 h = __builtin_bit_cast(u32x4, hi), l = __builtin_bit_cast(u32x4, lo);
        u32x4* at = j.halves + adapter_half_at(group, rp, y / 2, 0) + lane;
        if (rp == 16) {
            at[16 * (2 * c)] = u32x4{h[0], h[1], l[0], l[1]};
            at[16 * (2 * c + 1)] = u32x4{h[2], h[3], l[2], l[3]};
        } else {
            at[16 * (2 * (y & 1) + c)] = h;
            j.halves[adapter_half_at(group, rp, y / 2, 1) + lane + 16 * (2 * (y & 1) + c)] = l;
        }
    }
    if (j.turned && t >= 128) {  // 16 columns x 8 of 8 rows
        const int col = t & 15, r8 = (t >> 4) & 7;
        bf16x8 s[3];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            bf16 v[3];
            adapter_split3(lds[8 * r8 + e][col], v);
#pragma unroll
            for (int u = 0; u < 3; ++u) s[u][e] = v[u];
        }
#pragma unroll
        for (int u = 0; u < 3; ++u)
            j.turned[adapter_turned_at(2 * x + r8 / 4, rp, u, y) + 16 * (r8 & 3) + col] = __builtin_bit_cast(u32x4, s[u]);
    }
}

// ------------------------------------------------------------------ expand
struct AdapterExpand {
    const float* T;       // splits x 64 tiles x rp, or
    const u32x4* halves;  // as finish leaves them
    const bf16* W;        // n x d x r (COL: n x r x d)
    const bf16* base;     // or null: zeros
    bf16* out;            // M x d; may be base
    int64_t d;
    int64_t K;            // that t was summed over
};

constexpr int kAdWide = 128;  // columns that a workgroup of expand takes

// Workgroups: x: 128 columns, y: tiles (those of rows without an adapter last, which
// are copied); a wave for each of the tile's groups of 16 rows.  Instruction u's
// column i is c0 + 8 i + u, so that a lane ends up with 8 columns in a row and 16
// neighbouring lanes with 256 bytes of each row of Y.  The waves share W's rows of
// these columns, which go through LDS in the order of the operands, KB blocks of 32
// columns of t at a time; 0: up to 16 columns, instructions of 16.
// (W in registers, 64 rows a wave: eight waves a CU instead of twenty, and 1999 rows
// of 11008 with rank 64 take 30 us.)  ONE: those blocks are all.  SUM: t is still in
// parts.  COL: W's rows are the columns of t; a thread takes 8 columns of 8 of them
// and turns them round.  FULL: all columns of the workgroup are there.
template <int KB, bool ONE, bool SUM, bool COL, bool FULL>
__device__ __forceinline__ void adapter_expand_tile(const AdapterExpand& j, const AdapterHeader& h, const AdapterTile tile,
                                                    const int32_t* rows, int64_t c0, int64_t r, int target, u32x4* lds) {
    constexpr int NB = KB > 0 ? KB : 1, CH = KB > 0 ? 4 * KB : 2;  // pieces of 8 columns of t in a row of LDS
    constexpr int PITCH = CH + 1, PIECES = COL ? 8 : kAdWide * CH / kAdThreads;
    const int lane = threadIdx.x & 63, g = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
    const int64_t rp = adapter_rp(r), c = c0 + 8 * i;
    const bool live = 16 * g < tile.count;  // of the wave
    const bool add = j.base != nullptr;
    const bf16* from = add ? j.base : j.out;
    int row[4];
    {
        const int4 four = *reinterpret_cast<const int4*>(rows + 16 * g + 4 * q);
        row[0] = four.x, row[1] = four.y, row[2] = four.z, row[3] = four.w;
    }
    // t's operands
    const int splits = SUM ? adapter_splits(h.tiles, j.K, target) : 1;
    const int64_t group = 4 * (int64_t)blockIdx.y + g;
    u32x4 hi[NB], lo[NB];
    auto operands = [&](int64_t k0) {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            if constexpr (SUM) {
                const float* t = j.T + (16 * group + min(i, max(0, tile.count - 1 - 16 * g))) * rp + k0 +
                                 (KB == 0 ? 4 * q : 32 * b + 8 * q);
                const int64_t stride = (int64_t)h.tiles * kAdTile * rp;
                const f32x4 x = adapter_t4(t, splits, stride);
                f32x4 y = x;
                if constexpr (KB != 0) y = adapter_t4(t + 4, splits, stride);
                bf16x8 v[2];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    bf16 s[2];
                    adapter_split2(e < 4 ? x[e % 4] : y[e % 4], s[0], s[1]);
                    v[0][e] = s[0];
                    v[1][e] = s[1];
                }
                hi[b] = __builtin_bit_cast(u32x4, v[0]);
                lo[b] = __builtin_bit_cast(u32x4, v[1]);
                if constexpr (KB == 0) hi[0] = u32x4{hi[0][0], hi[0][1], lo[0][0], lo[0][1]};
            } else {
                hi[b] = j.halves[adapter_half_at(group, rp, k0 / 32 + b, 0) + lane];
                if constexpr (KB != 0) lo[b] = j.halves[adapter_half_at(group, rp, k0 / 32 + b, 1) + lane];
            }
        }
    };
    // W's values for the workgroup's columns: thread's piece k is 8 columns of t of one
    // of them (COL: 8 of them, of one column of t)
    const bf16* W = j.W + (int64_t)tile.adapter * j.d * r;
    u32x4 piece[PIECES];
    const int tc = threadIdx.x / CH, th = threadIdx.x % CH;
    auto pieces = [&](int64_t k0) {
        const int64_t at = k0 + 8 * th;
        if constexpr (COL) {
            if (tc >= 16) return;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const bf16* row = W + min(at + k, r - 1) * j.d;
                if constexpr (FULL) piece[k] = adapter_load(row + c0 + 8 * tc);
                else if (j.d >= 8) piece[k] = adapter_edge8(row, c0 + 8 * tc, j.d);
                else piece[k] = adapter_load8(row, min(c0 + 8 * tc, j.d), j.d);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) piece[k] = at + k < r ? piece[k] : zero16();
        } else {
            const bf16* row[PIECES];
#pragma unroll
            for (int k = 0; k < PIECES; ++k) row[k] = W + min(c0 + k * (kAdThreads / CH) + tc, j.d - 1) * r;
            if (r % 8 == 0) {
#pragma unroll
                for (int k = 0; k < PIECES; ++k) piece[k] = adapter_load(row[k] + (at < r ? at : 0));
            } else if (r >= 8) {
#pragma unroll
                for (int k = 0; k < PIECES; ++k) piece[k] = adapter_edge8(row[k], at, r);
            } else {
#pragma unroll
                for (int k = 0; k < PIECES; ++k) piece[k] = adapter_load8(row[k], at, r);
            }
#pragma unroll
            for (int k = 0; k < PIECES; ++k) piece[k] = at < r ? piece[k] : zero16();
        }
    };
    auto place = [&] {
        if constexpr (COL) {
            if (tc >= 16) return;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                u32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = adapter_pair(piece[2 * e][u / 2], piece[2 * e + 1][u / 2], u & 1);
                lds[(u * 16 + tc) * PITCH + th] = v;
            }
        } else {
#pragma unroll
            for (int k = 0; k < PIECES; ++k) {
                const int col = k * (kAdThreads / CH) + tc;
                lds[(col % 8 * 16 + col / 8) * PITCH + th] = piece[k];
            }
        }
    };
    operands(0);
    u32x4 base[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const bf16* at = from + (int64_t)max(row[e], 0) * j.d;
        // its last reader (1999 rows of 11008: 38.2 us a call, 40.8 through the caches)
        if constexpr (FULL) base[e] = load_streamed<u32x4>(at + c);
        else if (j.d >= 8) base[e] = adapter_edge8(at, c, j.d);
        else base[e] = adapter_load8(at, min(c, j.d), j.d);
    }
    pieces(0);
    f32x4 acc[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) acc[u] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int64_t k0 = 0;;) {
        place();
        __syncthreads();
        if (live) {
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const u32x4* row = lds + (u * 16 + i) * PITCH;
                f32x4 left{0.f, 0.f, 0.f, 0.f};
                if constexpr (KB == 0) {
                    const uint2 w = reinterpret_cast<const uint2*>(row)[q];
                    left = adapter_finite(adapter_mfma16(uint2{hi[0][2], hi[0][3]}, w, left));
                    acc[u] = adapter_mfma16(uint2{hi[0][0], hi[0][1]}, w, left);
                } else {
                    u32x4 w[NB];
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        w[b] = row[4 * b + q];
                        left = adapter_mfma(lo[b], w[b], left);
                    }
                    left = adapter_finite(left);
                    acc[u] = ONE ? left : acc[u] + left;
#pragma unroll
                    for (int b = 0; b < NB; ++b) acc[u] = adapter_mfma(hi[b], w[b], acc[u]);
                }
            }
        }
        if constexpr (ONE) break;
        k0 += 8 * CH;
        if (k0 >= rp) break;
        operands(k0);
        pieces(k0);
        __syncthreads();
    }
    if (!live) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const bf16x8 b = __builtin_bit_cast(bf16x8, base[e]);
        bf16x8 y;
#pragma unroll
        for (int u = 0; u < 8; ++u) y[u] = (bf16)((add ? (float)b[u] : 0.f) + acc[u][e]);
        if (row[e] < 0) continue;
        bf16* to = j.out + (int64_t)row[e] * j.d + c;
        if (FULL || c + 8 <= j.d) {
            reinterpret_cast<AdapterAny16*>(to)->v = __builtin_bit_cast(u32x4, y);
        } else {
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (c + u < j.d) to[u] = y[u];
        }
    }
}

template <int KB, bool ONE, bool SUM, bool COL>
__global__ __launch_bounds__(kAdThreads, SUM ? 2 : ONE ? 4 : 3) void adapter_expand(AdapterExpand j, AdapterPlan p, int64_t M, int n,
                                                                          int64_t r, int target) {
    __shared__ u32x4 lds[kAdWide * (KB > 0 ? 4 * KB + 1 : 3)];
    const AdapterHeader h = *p.head;
    const AdapterTile tile = p.tiles[blockIdx.y];
    if (h.M != M || h.n != n || (int)blockIdx.y >= h.tiles_all) return;
    const int64_t c0 = (int64_t)blockIdx.x * kAdWide;
    if (c0 >= j.d) return;
    const int32_t* rows = p.rows + (int64_t)blockIdx.y * kAdTile;
    if (tile.adapter >= n) {
        // rows without an adapter, 8 columns a lane
        if (j.out == j.base) return;
        const int64_t c = c0 + 8 * (threadIdx.x & 15);
        const bool inside = c + 8 <= j.d;
        int row[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) row[e] = rows[16 * e + (threadIdx.x >> 4)];
        u32x4 v[4] = {zero16(), zero16(), zero16(), zero16()};
        if (j.base && inside) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = load_streamed<u32x4>(j.base + max(row[e], 0) * j.d + c);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (row[e] < 0) continue;
            if (inside) store_streamed(j.out + row[e] * j.d + c, v[e]);
            else for (int64_t at = row[e] * j.d + c; at < (row[e] + 1) * j.d; ++at)
                ((uint16_t*)j.out)[at] = j.base ? ((const uint16_t*)j.base)[at] : (uint16_t)0;
        }
        return;
    }
    if (c0 + kAdWide <= j.d) adapter_expand_tile<KB, ONE, SUM, COL, true>(j, h, tile, rows, c0, r, target, lds);
    else adapter_expand_tile<KB, ONE, SUM, COL, false>(j, h, tile, rows, c0, r, target, lds);
}

// ------------------------------------------------------------------ backward
struct AdapterGrads {
    const bf16* P;        // rows (M x d)
    const u32x4* turned;  // as finish leaves it
    float* out;           // n x r x d (by_column: n x d x r)
    float* part;          // the same of one adapter for each slot
    int64_t d;
    bool by_column;
};

constexpr int kAdCols = 128;  // columns of P that a workgroup of grads takes
constexpr int kAdGradThreads = 512, kAdGradWaves = kAdGradThreads / kWave;

// Workgroups: x: columns of both jobs, y: pieces, z: blocks of 16 JB columns of t: 64
// at most, whose sums take half of a CU's registers and 98 KB of its LDS (waves that
// share the columns of t instead load and turn P's rows once for each share: 2125
// rows of rank 92 42 us, 40 so).
// Each wave takes 32 rows at a time, every eighth such step: 8 loads of 8 columns
// a lane, 8 rows apart from lane group to lane group, turned round to 8 operands
// of 8 rows each.
template <int JB>
__global__ __launch_bounds__(kAdGradThreads) void adapter_grads(AdapterGrads j0, AdapterGrads j1, int blocks0, AdapterPlan p,
                                                            int64_t M, int n, int64_t r) {
    constexpr int COLS = 16 * JB, ROUND = 8 / JB;  // operands whose sums LDS holds at once
    __shared__ float part[ROUND][kAdGradWaves][16 * COLS];
    __shared__ float sums[COLS][kAdCols + 1];
    const AdapterHeader h = *p.head;
    const AdapterPiece piece = p.pieces[blockIdx.y];
    if (h.M != M || h.n != n || (int)blockIdx.y >= h.pieces) return;
    const bool second = (int)blockIdx.x >= blocks0;
    const AdapterGrads j = second ? j1 : j0;
    const int64_t c0 = (int64_t)(second ? blockIdx.x - blocks0 : blockIdx.x) * kAdCols;
    const int b0 = blockIdx.z * COLS;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
    const int64_t rp = adapter_rp(r), c = c0 + 8 * i;
    const bool full = c0 + kAdCols <= j.d;

    f32x4 acc[8][JB];
#pragma unroll
    for (int u = 0; u < 8; ++u)
#pragma unroll
        for (int b = 0; b < JB; ++b) acc[u][b] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int64_t first = (int64_t)piece.first * kAdTile;
    for (int s = wave; s < 2 * piece.tiles; s += kAdGradWaves) {
        const int64_t at = first + 32 * s + 8 * q;
        int32_t row[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) row[e] = p.rows[at + e];
        u32x4 t[3][JB];
#pragma unroll
        for (int u = 0; u < 3; ++u)
#pragma unroll
            for (int b = 0; b < JB; ++b)
                t[u][b] = j.turned[adapter_turned_at(2 * piece.first + s, rp, u, b0 / 16 + b) + lane];
        u32x4 x[8];
        if (full) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = load_streamed<u32x4>(j.P + (int64_t)max(row[e], 0) * j.d + c);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = row[e] >= 0 ? x[e] : zero16();
        } else if (j.d >= 8) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = adapter_edge8(j.P + (int64_t)max(row[e], 0) * j.d, c, j.d);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = row[e] >= 0 ? x[e] : zero16();
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = zero16();
                if (row[e] >= 0) x[e] = adapter_load8(j.P + (int64_t)row[e] * j.d, min(c, j.d), j.d);
            }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            u32x4 turned;
#pragma unroll
            for (int e = 0; e < 4; ++e) turned[e] = adapter_pair(x[2 * e][k / 2], x[2 * e + 1][k / 2], k & 1);
#pragma unroll
            for (int b = 0; b < JB; ++b) {
                const f32x4 left = adapter_mfma(turned, t[1][b], adapter_mfma(turned, t[2][b], f32x4{0.f, 0.f, 0.f, 0.f}));
                acc[k][b] = adapter_mfma(turned, t[0][b], acc[k][b]) + adapter_finite(left);
            }
        }
    }
    if (piece.tiles > 0) {  // the same for all
        // the waves' sums: acc[k][b], row 4 q + e is column 8 (4 q + e) + k of P, column i is
        // column 16 b + i of t.  In LDS the rows lie as 4 e + q and their columns are moved on, so
        // that the lanes of a store are in different banks.
#pragma unroll
        for (int k0 = 0; k0 < 8; k0 += ROUND) {
            if (k0 > 0) __syncthreads();
#pragma unroll
            for (int k = 0; k < ROUND; ++k)
#pragma unroll
                for (int b = 0; b < JB; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        part[k][wave][(4 * e + q) * COLS + (16 * (b + q * JB / 4) + i) % COLS] = acc[k0 + k][b][e];
            __syncthreads();
            for (int at = threadIdx.x; at < ROUND * 16 * COLS; at += kAdGradThreads) {
                const int k = at / (16 * COLS), cell = at % (16 * COLS), e = cell / (4 * COLS), u4 = cell / COLS % 4;
                float v = 0.f;
#pragma unroll
                for (int u = 0; u < kAdGradWaves; ++u) v += part[k][u][cell];
                sums[(cell + COLS - 16 * (u4 * JB / 4)) % COLS][8 * (4 * u4 + e) + k0 + k] = v;
            }
        }
        __syncthreads();
    }
    // 4 neighbouring values a lane
    float* out = piece.slot < 0 ? j.out + piece.adapter * r * j.d : j.part + piece.slot * r * j.d;
    const int cols = (int)min((int64_t)kAdCols, j.d - c0), js = (int)min((int64_t)COLS, r - b0);
#pragma unroll
    for (int u = 0; u < COLS * kAdCols / 4 / kAdGradThreads; ++u) {
        const int at = u * kAdGradThreads + threadIdx.x;
        const int a = j.by_column ? 4 * (at % (COLS / 4)) : at / (kAdCols / 4);
        const int k = j.by_column ? at / (COLS / 4) : 4 * (at % (kAdCols / 4));
        const int left = j.by_column ? (k < cols ? js - a : 0) : a < js ? cols - k : 0;
        if (left <= 0) continue;
        float* to = out + (j.by_column ? (c0 + k) * r + b0 + a : (b0 + a) * j.d + c0 + k);
        f32x4 v{0.f, 0.f, 0.f, 0.f};
        if (piece.tiles > 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = j.by_column ? sums[a + e][k] : sums[a][k + e];
        }
        if (left >= 4) store_streamed(to, v);
        else for (int e = 0; e < left; ++e) to[e] = v[e];
    }
}

// Gradients of adapters of more than one piece: their partial sums, in order.
// Workgroups: x: values of both gradients, 1024 each, y: adapters.
static __global__ __launch_bounds__(256) void adapter_sum(const float* part0, float* out0, int64_t n0, int blocks0,
                                                         const float* part1, float* out1, int64_t n1, AdapterPlan p,
                                                         int64_t M, int n) {
    const AdapterHeader h = *p.head;
    const AdapterMulti a = p.multi[blockIdx.y];
    if (h.M != M || h.n != n || (int)blockIdx.y >= h.multi) return;
    const bool second = (int)blockIdx.x >= blocks0;
    const int64_t count = second ? n1 : n0;
    const float* from = (second ? part1 : part0) + a.slot * count;
    float* to = (second ? out1 : out0) + a.adapter * count;
    const int64_t first = (int64_t)(second ? blockIdx.x - blocks0 : blockIdx.x) * 1024 + threadIdx.x;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.pieces; s += 4) {
        float x[4][4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t k = first + 256 * e;
                x[u][e] = from[min(s + u, a.pieces - 1) * count + (k < count ? k : 0)];
            }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += s + u < a.pieces ? x[u][e] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (first + 256 * e < count) to[first + 256 * e] = v[e];
}

}  // namespace pifa
