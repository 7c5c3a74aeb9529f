// Products of 4-bit layers with many rows: tiles of Y = X W^T on matrix cores.
//
// One workgroup of eight waves per BM x BN tile.  A K tile is 128 bytes of each
// row of X (64 bf16 or 128 e4m3 values) and the packed codes and scales that
// meet them; all of it goes from memory straight into LDS, S tiles in flight,
// and the codes stay 4-bit up to the registers: the weights' share of the LDS
// traffic is a quarter of what bf16 weights would take.
//   bf16 rows: a step of 32 K values is one group of 32 for every weight row,
//              so its codes become bf16 under one scale (two per instruction)
//              between the LDS read and the 16x16x32 MFMA;
//   e4m3 rows: codes, scales and values feed the 16x16x128 MFMA as they are.
//
// Two groups of four waves alternate as in the prefill products of bf16
// layers: in a slot one reads (and converts) the operands of its next segment,
// the other runs its MFMAs, and a barrier ends the slot.  A K tile is two
// segments: its two steps (bf16), or the upper and lower half of the wave's
// rows (e4m3).  Group 0 reads segment p of tile t in slot 4 t + 2 p and
// multiplies it in the next, group 1 is one slot behind.  Tile t's stage is
// free from slot 4 (t + 1): group 0 issues tile t + S - 1 between the MFMAs of
// its first segment of tile t, group 1 tile t + S between those of its last.
// Each wave waits for its own loads of tile t + 1 before the barrier that ends
// slot 4 (t + 1) - 1; S - 2 later tiles may still be in flight then.
//
// The weights are the first MFMA operand and their rows are dealt over the TN
// fragments so that a lane's accumulators are 4 TN consecutive columns of a
// row of Y: row i of fragment j is column (i / 4) * 4 TN + 4 j + i % 4.
//
// Measured on several boards, calls in a row: 4096 rows of 4096 -> 11008 in bf16
// 279 to 292 us, 1.32 to 1.26 PFLOP/s (a library product of 8192^3: 1.40); 1999
// rows of 11008 -> 4096 in e4m3 79 to 83 us, 2.29 to 2.17 PFLOP/s (library: 2.64).
// Under the profiler the kernels take 296 to 326 and 81 to 84 us, with the matrix
// cores busy in 65% and 56% of the cycles CUs work.
#pragma once

#include "common.hpp"
#include "gemm_dma.hpp"
#include "gemm_f32.hpp"
#include "gemm_mfma.hpp"
#include "q4.hpp"

namespace pifa {

// A lane's 4 TN consecutive columns n .. of its rows m, m + 16, ...
template <bool E4, int TM, int TN>
__device__ __forceinline__ void q4_store_rows(const Q4Args& p, const f32x4 (&acc)[TM][TN], int64_t m, int64_t n) {
    constexpr int W = 4 * TN, C = W < 8 ? W : 8;  // columns of a store
    struct __attribute__((packed, aligned(2))) Run {
        uint16_t h[C];
    };
#pragma unroll
    for (int i = 0; i < TM; ++i, m += 16) {
        if (m >= p.M) continue;
        const float f = E4 ? p.x_scale[m] : 1.f;
        uint16_t* y = reinterpret_cast<uint16_t*>(p.Y) + m * p.N + n;
#pragma unroll
        for (int x = 0; x < W; x += C) {
            Run r;
#pragma unroll
            for (int e = 0; e < C; ++e) {
                const float v = acc[i][(x + e) / 4][(x + e) & 3];
                r.h[e] = f32_to_bf16_bits(E4 ? v * f : v);
            }
            if (n + x + C <= p.N) {
                *reinterpret_cast<Run*>(y + x) = r;
            } else {
#pragma unroll
                for (int e = 0; e < C; ++e)
                    if (n + x + e < p.N) y[x + e] = r.h[e];
            }
        }
    }
}

// The K tiles of one group of NW waves, WN of them along N, and what a lane
// reads of them.  X rows lie in 16-byte slots, slot = chunk ^ ((row / 2) % 8),
// so that the 16 rows a fragment read covers fall on different banks; the rows
// of weight group gl have their slots swapped (row ^ swap(gl)) for the same
// reason.  The scales are a piece of their own, 64 bytes a group.  A wave loads
// pieces w, w + NW, ...: first the XPIECES of X, then those of the codes, then
// the scales; which of them its j-th is does not change, so its buffer, its
// step along K and its place are chosen once (and where it is the same for all
// waves, known to the compiler).  Waves without a last piece of their own load
// the scales again, so that all wait for the same number of loads.
template <int ACT, int BM, int BN, int NW, int WN, int TN>
struct Q4Stage {
    static constexpr bool E4 = ACT == kQ4E4m3;
    static constexpr int ES = E4 ? 1 : 2, BK = E4 ? 128 : 64;
    static constexpr int GB = E4 ? 1024 : 512;  // bytes of codes of a 16-row group per K tile
    static constexpr int XPIECES = BM / 8, WPIECES = BN / 16 * GB / 1024, PIECES = XPIECES + WPIECES + 1;
    static constexpr int kBytes = PIECES * 1024;
    static constexpr int kLoads = (PIECES + NW - 1) / NW;
    static_assert(BM % 16 == 0 && BN % 32 == 0 && BN <= 256, "pieces");
    static_assert(TN == 1 || TN == 2 || TN == 4, "fragments of a wave");

    // 0 X, 1 codes, 2 scales
    __device__ __forceinline__ static constexpr int kind_of(int piece) {
        return piece < XPIECES ? 0 : piece < XPIECES + WPIECES ? 1 : 2;
    }
    __device__ __forceinline__ static constexpr bool same_kind(int j) { return kind_of(NW * j) == kind_of(NW * j + NW - 1); }
    __device__ __forceinline__ int kind(int j) const { return same_kind(j) ? kind_of(NW * j) : kinds[j]; }

    int nk, w;
    const char *xbase, *wbase;
    int xbytes, wbytes;  // of the buffers behind them
    int kinds[kLoads];
    uint32_t off[kLoads], last[kLoads], place[kLoads];
    uint32_t rx[2], rw[TN], rs;  // a lane's places in a stage

    __device__ __forceinline__ static int swap(int gl) { return TN == 4 ? 4 * (gl & 3) : TN == 2 ? 4 * (gl & 1) : 0; }
    __device__ __forceinline__ static int clip(int64_t n) { return n > 0x7FFFFFFF ? 0x7FFFFFFF : (int)n; }

    // wrow: the wave's first row of the tile, wn: its place along N
    __device__ __forceinline__ void init(const Q4Args& p, int64_t m0, int64_t n0, int wave, int wrow, int wn, int lane) {
        const int64_t KB = packed_kblocks(p.K);
        const int K = (int)p.K, li = lane & 15, lg = lane >> 4;
        w = wave;
        nk = (K + BK - 1) / BK;
        xbase = (const char*)p.X + m0 * p.K * ES;
        wbase = (const char*)p.W + n0 / 16 * KB * kQ4Block;
        xbytes = clip((p.M - m0) * p.K * ES);
        wbytes = clip((packed_groups(p.N) - n0 / 16) * KB * kQ4Block);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            int piece = w + NW * j;
            if (piece >= PIECES) piece = PIECES - 1;
            place[j] = (uint32_t)__builtin_amdgcn_readfirstlane(piece * 1024);
            kinds[j] = __builtin_amdgcn_readfirstlane(kind_of(piece));
            if (kind(j) == 0) {  // 8 rows x 128 bytes
                const int row = 8 * piece + (lane >> 3), c = (lane & 7) ^ ((row >> 1) & 7);
                off[j] = (uint32_t)(row * K * ES + 16 * c);
                last[j] = (nk - 1) * BK + (16 / ES) * c < K ? off[j] : kMaskedOffset;
            } else {
                if (kind(j) == 1) {  // e4m3: a group's 128 columns; bf16: 64 columns of two groups
                    const int q = piece - XPIECES, gl = E4 ? q : 2 * q + (lane >> 5);
                    off[j] = (uint32_t)(gl * KB * kQ4Block + ((li ^ swap(gl)) + 16 * (E4 ? lg : lg & 1)) * 16);
                } else {  // 64 bytes of each group
                    const int gl = lane >> 2;
                    off[j] = gl < BN / 16 ? (uint32_t)(gl * KB * kQ4Block + 1024 + (lane & 3) * 16) : kMaskedOffset;
                }
                last[j] = off[j];
            }
        }
        const int row = wrow + li;
#pragma unroll
        for (int h = 0; h < 2; ++h) rx[h] = (uint32_t)(row * 128 + (((4 * h + lg) ^ ((row >> 1) & 7)) << 4));
        const int n = (li >> 2) * 4 * TN + (li & 3), gw = n >> 4, gl = wn * TN + gw;  // n + 4 j: same group
#pragma unroll
        for (int j = 0; j < TN; ++j)
            rw[j] = (uint32_t)(XPIECES * 1024 + gl * GB + ((((n & 15) + 4 * j) ^ swap(gl)) << 4) +
                               (E4 ? lg * 256 : lg * 4));
        rs = (uint32_t)((XPIECES + WPIECES) * 1024 + gl * 64 + (n & 15) + (E4 ? 16 * lg : 0));
    }
    // the wave's j-th load of K tile t into the stage at lds.  A tile past the
    // last is not multiplied; its loads stay inside the buffers.
    __device__ __forceinline__ void issue(int t, uint32_t lds, int j) const {
        const int blk = (E4 ? t : t >> 1) * kQ4Block, k = kind(j);
        const int at = k == 0 ? t * 128 : k == 1 && !E4 ? blk + (t & 1) * 512 : blk;
        const uint64_t b = reinterpret_cast<uint64_t>(k == 0 ? xbase : wbase) + (uint32_t)at;
        const int n = (k == 0 ? xbytes : wbytes) - at;
        const u32x4 rs = {(uint32_t)b, (uint32_t)(b >> 32), (uint32_t)(n > 0 ? n : 0), 0x00020000u};
        const bool ends = same_kind(j) && k != 0;  // no tail of their own: padded
        dma16(rs, !ends && t == nk - 1 ? last[j] : off[j], lds + place[j]);
    }
    __device__ __forceinline__ u32x4 x(const char* st, int h, int i) const {
        return *reinterpret_cast<const u32x4*>(st + rx[h] + i * 2048);
    }
    __device__ __forceinline__ u32x4 codes(const char* st, int j) const {  // e4m3
        return *reinterpret_cast<const u32x4*>(st + rw[j]);
    }
    __device__ __forceinline__ uint32_t codes(const char* st, int j, int h) const {  // bf16, step h
        return *reinterpret_cast<const uint32_t*>(st + rw[j] + h * 256);
    }
    // e4m3: the scale of fragment j; bf16: of step `sub` (0..3) of the block
    __device__ __forceinline__ uint32_t scale(const char* st, int j, int sub) const {
        return *reinterpret_cast<const uint8_t*>(st + rs + 4 * j + 16 * sub);
    }
};

template <int ACT, int BM, int BN, int WM, int WN, int S, int OCC>
__global__ __launch_bounds__(8 * kWave, OCC) void q4_tiles(Q4Args p) {
    constexpr bool E4 = ACT == kQ4E4m3;
    constexpr int NW = 8;
    static_assert(WM * WN == NW, "eight waves");
    constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 16, TN = WTN / 16;
    static_assert(TM % 2 == 0, "fragments of a wave");
    using Stage = Q4Stage<ACT, BM, BN, NW, WN, TN>;
    constexpr int STAGE = Stage::kBytes, DPW = Stage::kLoads;
    static_assert(S >= 2 && S * STAGE <= 163840, "160 KB of LDS");
    __shared__ __attribute__((aligned(1024))) char smem[S * STAGE];

    int64_t tm, tn;
    tile_coords<BM, BN>(blockIdx.x, ceil_div(p.M, BM), ceil_div(p.N, BN), tm, tn);
    const int64_t m0 = tm * BM, n0 = tn * BN;
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wm = wave / WN, wn = wave % WN, grp = wave >= NW / 2 ? 1 : 0;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;
    Stage sg;
    sg.init(p, m0, n0, wave, wm * WTM, wn, lane);
    const int nk = sg.nk;

    // ---- operands of a segment
    constexpr int FA = E4 ? TM / 2 : TM;  // row fragments
    u32x4 fa[E4 ? 2 : 1][FA], fb[TN];
    uint32_t fs[TN];
    auto frags = [&](int t, const char* st, int seg) {
        if constexpr (E4) {
            if (seg == 0) {
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    fb[j] = sg.codes(st, j);
                    fs[j] = sg.scale(st, j, 0);
                }
            }
#pragma unroll
            for (int i = 0; i < FA; ++i) {
                fa[0][i] = sg.x(st, 0, seg * FA + i);
                fa[1][i] = sg.x(st, 1, seg * FA + i);
            }
        } else {
            uint32_t codes[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                codes[j] = sg.codes(st, j, seg);
                fs[j] = sg.scale(st, j, 2 * (t & 1) + seg);
            }
#pragma unroll
            for (int i = 0; i < FA; ++i) fa[0][i] = sg.x(st, seg, i);
#pragma unroll
            for (int j = 0; j < TN; ++j) fb[j] = q4_to_bf16(codes[j], __builtin_bit_cast(float, fs[j] << 23));
        }
    };
    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // a segment's MFMAs, with tile t's loads between them (ISSUE)
    auto mma = [&](auto with, auto which, int t, uint32_t lds) {
        constexpr bool ISSUE = decltype(with)::value;
        constexpr int seg = decltype(which)::value;
        constexpr int GAP = FA * TN / DPW > 0 ? FA * TN / DPW : 1;
        int n = 0, d = 0;
#pragma unroll
        for (int i = 0; i < FA; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                f32x4& a = acc[E4 ? seg * FA + i : i][j];
                if constexpr (E4) a = q4_mfma_e4m3(fb[j], fs[j], fa[0][i], fa[E4 ? 1 : 0][i], a);
                else a = q4_mfma_bf16(fb[j], fa[0][i], a);
                if constexpr (ISSUE) {
                    if (n % GAP == GAP / 2 && d < DPW) {
                        __builtin_amdgcn_sched_barrier(0);
                        sg.issue(t, lds, d++);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                ++n;
            }
        if constexpr (ISSUE) {
#pragma unroll
            for (; d < DPW; ++d) sg.issue(t, lds, d);
        }
    };

#pragma unroll
    for (int s = 0; s < S; ++s) {
        if (s < S - 1 || grp) {
#pragma unroll
            for (int d = 0; d < DPW; ++d) sg.issue(s, lds0 + s * STAGE, d);
        }
    }
    if (grp) wait_vm<(S - 1) * DPW>();
    else wait_vm<(S - 2) * DPW>();
    slot_barrier();
    auto loop = [&](auto second) {
        constexpr bool G1 = decltype(second)::value;
        int at = 0;  // tile t's stage
        for (int t = 0; t < nk; ++t) {
            const char* st = smem + at * STAGE;
            const int next = at + 1 == S ? 0 : at + 1, prev = at == 0 ? S - 1 : at - 1;
            auto segment = [&](auto which) {
                constexpr int seg = decltype(which)::value;
                frags(t, st, seg);
                wait_lgkm0();
                if (G1 && seg == 1) wait_vm<(S - 2) * DPW>();
                slot_barrier();
                __builtin_amdgcn_s_setprio(1);
                if constexpr (seg == (G1 ? 1 : 0))
                    mma(std::true_type{}, which, t + (G1 ? S : S - 1), lds0 + (G1 ? at : prev) * STAGE);
                else mma(std::false_type{}, which, 0, 0);
                __builtin_amdgcn_s_setprio(0);
                if (!G1 && seg == 1) wait_vm<(S - 2) * DPW>();
                slot_barrier();
            };
            segment(std::integral_constant<int, 0>{});
            segment(std::integral_constant<int, 1>{});
            at = next;
        }
    };
    if (grp) {
        slot_barrier();
        loop(std::true_type{});
        wait_vm<0>();
    } else {
        loop(std::false_type{});
        wait_vm<0>();
        slot_barrier();
    }
    q4_store_rows<E4, TM, TN>(p, acc, m0 + wm * WTM + (lane & 15), n0 + wn * WTN + (lane >> 4) * 4 * TN);
}

// Middling numbers of rows.  A slot of the form above costs a barrier and an
// LDS round trip, which the few MFMAs of a small tile do not cover, so here a
// wave reads the operands of its next K tile while it multiplies the current
// one, and a K tile costs one barrier.  KG groups of WM x WN waves take every
// KG-th K tile each (their sums meet in LDS at the end), so a long K is a
// short loop also where there are few tiles.
// Step s's stage is read (into registers) before the barrier of step s, and
// loaded again with step s + S after it.
// S: stages of each group's ring, as many as fit LDS up to SMAX.
// Bound by those steps, not by memory: 57 rows of 4096 -> 11008 14.1 us, of which
// reading 26 MB takes 4; deeper rings (4 to 7 stages) gained nothing.
template <int ACT, int BM, int BN, int WM, int WN, int KG, int SMAX, int OCC>
__global__ __launch_bounds__(WM* WN* KG* kWave, OCC) void q4_mid(Q4Args p) {
    constexpr bool E4 = ACT == kQ4E4m3;
    constexpr int NW = WM * WN;
    constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 16, TN = WTN / 16;
    using Stage = Q4Stage<ACT, BM, BN, NW, WN, TN>;
    constexpr int STAGE = Stage::kBytes, DPW = Stage::kLoads;
    constexpr int FIT = 163840 / (KG * STAGE), S = FIT < SMAX ? FIT : SMAX;
    constexpr int LOOP = KG * S * STAGE, RED = (KG - 1) * BM * BN * 4;
    static_assert(S >= 2 && LOOP <= 163840 && RED <= 163840, "160 KB of LDS");
    __shared__ __attribute__((aligned(1024))) char smem[LOOP > RED ? LOOP : RED];

    int64_t tm, tn;
    tile_coords<BM, BN>(blockIdx.x, ceil_div(p.M, BM), ceil_div(p.N, BN), tm, tn);
    const int64_t m0 = tm * BM, n0 = tn * BN;
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int kg = wave / NW, w = wave % NW, wm = w / WN, wn = w % WN;
    char* ring = smem + kg * S * STAGE;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)ring;
    Stage sg;
    sg.init(p, m0, n0, w, wm * WTM, wn, lane);
    const int steps = (sg.nk + KG - 1) / KG;

    auto issue = [&](int s, int at) {
#pragma unroll
        for (int d = 0; d < DPW; ++d) sg.issue(s * KG + kg, lds0 + at * STAGE, d);
    };
    struct Ops {
        u32x4 x[2][TM];
        u32x4 w[E4 ? TN : 1];        // e4m3: codes of a K tile
        uint32_t c[E4 ? 1 : 2][TN];  // bf16: codes of its two steps
        uint32_t s[E4 ? 1 : 2][TN];
    };
    auto read = [&](int s, int at, Ops& o) {
        const char* st = ring + at * STAGE;
        const int t = s * KG + kg;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            if constexpr (E4) {
                o.w[j] = sg.codes(st, j);
                o.s[0][j] = sg.scale(st, j, 0);
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    o.c[h][j] = sg.codes(st, j, h);
                    o.s[h][j] = sg.scale(st, j, 2 * (t & 1) + h);
                }
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < TM; ++i) o.x[h][i] = sg.x(st, h, i);
    };
    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto mma = [&](const Ops& o) {
        if constexpr (E4) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = q4_mfma_e4m3(o.w[j], o.s[0][j], o.x[0][i], o.x[1][i], acc[i][j]);
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 wj[TN];
#pragma unroll
                for (int j = 0; j < TN; ++j) wj[j] = q4_to_bf16(o.c[h][j], __builtin_bit_cast(float, o.s[h][j] << 23));
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j] = q4_mfma_bf16(wj[j], o.x[h][i], acc[i][j]);
            }
        }
    };

#pragma unroll
    for (int s = 0; s < S; ++s) issue(s, s);
    wait_vm<(S - 1) * DPW>();
    slot_barrier();
    Ops even, odd;
    read(0, 0, even);
    int at = 0;  // step s's stage
    auto step = [&](int s, const Ops& cur, Ops& nxt) {
        const int next = at + 1 == S ? 0 : at + 1;
        wait_lgkm0();
        wait_vm<(S - 2) * DPW>();  // step s + 1's loads
        slot_barrier();
        issue(s + S, at);
        read(s + 1, next, nxt);
        __builtin_amdgcn_sched_barrier(0);
        if (KG == 1 || s * KG + kg < sg.nk) mma(cur);  // uniform
        __builtin_amdgcn_sched_barrier(0);
        at = next;
    };
    int s = 0;
    for (; s + 1 < steps; s += 2) {
        step(s, even, odd);
        step(s + 1, odd, even);
    }
    if (s * KG + kg < sg.nk) mma(even);  // the last of an odd number: its operands are read
    wait_vm<0>();
    if constexpr (KG > 1) {
        wait_lgkm0();
        slot_barrier();  // the ring's memory takes the sums
        f32x4* red = reinterpret_cast<f32x4*>(smem);
        if (kg > 0) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) red[(((kg - 1) * NW + w) * TM * TN + i * TN + j) * kWave + lane] = acc[i][j];
        }
        __syncthreads();
        if (kg > 0) return;
#pragma unroll
        for (int g = 0; g < KG - 1; ++g)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] += red[((g * NW + w) * TM * TN + i * TN + j) * kWave + lane];
    }
    q4_store_rows<E4, TM, TN>(p, acc, m0 + wm * WTM + (lane & 15), n0 + wn * WTN + (lane >> 4) * 4 * TN);
}

}  // namespace pifa
