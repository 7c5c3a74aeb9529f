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
#pragma once

#include "common.hpp"
#include "gemm_dma.hpp"
#include "gemm_f32.hpp"
#include "gemm_mfma.hpp"
#include "q4.hpp"

namespace pifa {

template <int ACT, int BM, int BN, int WM, int WN, int S, int OCC>
__global__ __launch_bounds__(8 * kWave, OCC) void q4_tiles(Q4Args p) {
    constexpr bool E4 = ACT == kQ4E4m3;
    constexpr int NW = 8;
    static_assert(WM * WN == NW, "eight waves");
    constexpr int WTM = BM / WM, WTN = BN / WN, TM = WTM / 16, TN = WTN / 16;
    static_assert(TM % 2 == 0 && (TN == 2 || TN == 4), "fragments of a wave");
    constexpr int BK = E4 ? 128 : 64;
    constexpr int GB = E4 ? 1024 : 512;  // bytes of codes of a 16-row group per K tile
    constexpr int XB = BM * 128, WB = BN / 16 * GB, SB = NW * 256;
    constexpr int STAGE = XB + WB + SB;
    static_assert(S >= 2 && S * STAGE <= 163840, "160 KB of LDS");
    constexpr int XP = BM / 8 / NW;                              // 1 KB pieces of X a wave loads per K tile
    constexpr int WPIECES = WB / 1024, WP = (WPIECES + NW - 1) / NW;  // with fewer pieces than waves, some load one twice
    static_assert(BM % 64 == 0 && (WPIECES % NW == 0 || NW % WPIECES == 0), "pieces do not split over the waves");
    constexpr int DPW = XP + WP + 1;
    __shared__ __attribute__((aligned(1024))) char smem[S * STAGE];

    const int64_t K = p.K, KB = packed_kblocks(K), nk = ceil_div(K, BK);
    int64_t tm, tn;
    tile_coords<BM, BN>(blockIdx.x, ceil_div(p.M, BM), ceil_div(p.N, BN), tm, tn);
    const int64_t m0 = tm * BM, n0 = tn * BN;
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wm = wave / WN, wn = wave % WN, grp = wave >= NW / 2 ? 1 : 0;
    const int li = lane & 15, lg = lane >> 4;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)smem;

    // ---- loads.  X rows in 16-byte slots, slot = chunk ^ ((row / 2) % 8), so
    // that the 16 rows a fragment read covers fall on different banks; weight
    // groups with their rows' slots swapped by 4 (gl % 4), for the same reason.
    constexpr int ES = E4 ? 1 : 2;
    const u32x4 xrs = raw_rsrc31((const char*)p.X + m0 * K * ES, (p.M - m0) * K * ES);
    const u32x4 wrs = raw_rsrc31(p.W + n0 / 16 * KB * kQ4Block, (packed_groups(p.N) - n0 / 16) * KB * kQ4Block);
    auto w_swap = [](int gl) { return TN == 4 ? 4 * (gl & 3) : 4 * (gl & 1); };
    uint32_t xoff[XP], woff[WP], soff;
    int xc[XP];
#pragma unroll
    for (int j = 0; j < XP; ++j) {  // piece: 8 rows x 128 bytes
        const int row = 8 * (wave + NW * j) + (lane >> 3);
        xc[j] = (lane & 7) ^ ((row >> 1) & 7);
        xoff[j] = (uint32_t)(row * K * ES + 16 * xc[j]);
    }
#pragma unroll
    for (int j = 0; j < WP; ++j) {
        const int piece = (wave + NW * j) % WPIECES;
        if constexpr (E4) {  // a group's 128 columns
            woff[j] = (uint32_t)(piece * KB * kQ4Block + ((li ^ w_swap(piece)) + 16 * lg) * 16);
        } else {  // 64 columns of two groups
            const int gl = 2 * piece + (lane >> 5);
            woff[j] = (uint32_t)(gl * KB * kQ4Block + ((li ^ w_swap(gl)) + 16 * (lg & 1)) * 16);
        }
    }
    // the scales of the wave's own TN groups, 64 bytes each
    soff = lg < TN ? (uint32_t)((wn * TN + lg) * KB * kQ4Block + 1024 + 4 * li) : kMaskedOffset;
    auto issue1 = [&](int64_t t, int d) {
        const uint32_t st = lds0 + (uint32_t)(t % S) * STAGE;
        const int64_t k0 = t * BK;
        if (d < XP) {
            const int j = d < XP ? d : 0;
            dma16(xrs, k0 + (16 / ES) * xc[j] < K ? xoff[j] + (uint32_t)(t * 128) : kMaskedOffset,
                  st + (wave + NW * j) * 1024);
        } else if (d < XP + WP) {
            const int j = d < XP + WP && d >= XP ? d - XP : 0;
            const uint32_t add = E4 ? (uint32_t)(t * kQ4Block) : (uint32_t)((t >> 1) * kQ4Block + (t & 1) * 512);
            dma16(wrs, k0 < K ? woff[j] + add : kMaskedOffset, st + XB + (wave + NW * j) % WPIECES * 1024);
        } else {
            const uint32_t add = (uint32_t)((E4 ? t : t >> 1) * kQ4Block);
            dma4(wrs, k0 < K ? soff + add : kMaskedOffset, st + XB + WB + wave * 256);
        }
    };
    auto issue = [&](int64_t t) {
#pragma unroll
        for (int d = 0; d < DPW; ++d) issue1(t, d);
    };

    // ---- operands of a segment
    constexpr int FA = E4 ? TM / 2 : TM;  // row fragments
    u32x4 fa[E4 ? 2 : 1][FA], fb[TN];
    uint32_t fs[TN];
    auto frags = [&](int64_t t, int seg) {
        const char* st = smem + (t % S) * STAGE;
        auto x_at = [&](int i, int step) {
            const int row = wm * WTM + 16 * i + li;
            return *reinterpret_cast<const u32x4*>(st + row * 128 + (((4 * step + lg) ^ ((row >> 1) & 7)) << 4));
        };
        const char* wst = st + XB;
        const uint8_t* sst = reinterpret_cast<const uint8_t*>(st) + XB + WB + wave * 256;
        if (!E4 || seg == 0) {
            uint32_t codes[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int n = (li >> 2) * 4 * TN + 4 * j + (li & 3);  // column within the wave's
                const int gw = n >> 4, gl = wn * TN + gw, row = n & 15;
                const char* at = wst + gl * GB + ((row ^ w_swap(gl)) << 4);
                if constexpr (E4) {
                    fb[j] = *reinterpret_cast<const u32x4*>(at + lg * 256);
                    fs[j] = sst[gw * 64 + 16 * lg + row];
                } else {
                    codes[j] = *reinterpret_cast<const uint32_t*>(at + seg * 256 + 4 * lg);
                    fs[j] = sst[gw * 64 + 16 * (2 * (int)(t & 1) + seg) + row];
                }
            }
            if constexpr (!E4) {
#pragma unroll
                for (int i = 0; i < FA; ++i) fa[0][i] = x_at(i, seg);
#pragma unroll
                for (int j = 0; j < TN; ++j) fb[j] = q4_to_bf16(codes[j], __builtin_bit_cast(float, fs[j] << 23));
            }
        }
        if constexpr (E4) {
#pragma unroll
            for (int i = 0; i < FA; ++i) {
                fa[0][i] = x_at(seg * FA + i, 0);
                fa[1][i] = x_at(seg * FA + i, 1);
            }
        }
    };
    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // a segment's MFMAs, with tile t's loads between them (ISSUE)
    auto mma = [&](auto with, auto which, int64_t t) {
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
                        issue1(t, d++);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                ++n;
            }
        if constexpr (ISSUE) {
#pragma unroll
            for (; d < DPW; ++d) issue1(t, d);
        }
    };

#pragma unroll
    for (int s = 0; s < S - 1; ++s) issue(s);
    if (grp) {
        issue(S - 1);
        wait_vm<(S - 1) * DPW>();
    } else {
        wait_vm<(S - 2) * DPW>();
    }
    slot_barrier();
    auto loop = [&](auto second) {
        constexpr bool G1 = decltype(second)::value;
        auto segment = [&](auto which, int64_t t) {
            constexpr int seg = decltype(which)::value;
            frags(t, seg);
            wait_lgkm0();
            if (G1 && seg == 1) wait_vm<(S - 2) * DPW>();
            slot_barrier();
            __builtin_amdgcn_s_setprio(1);
            if constexpr (seg == (G1 ? 1 : 0)) mma(std::true_type{}, which, t + (G1 ? S : S - 1));
            else mma(std::false_type{}, which, 0);
            __builtin_amdgcn_s_setprio(0);
            if (!G1 && seg == 1) wait_vm<(S - 2) * DPW>();
            slot_barrier();
        };
        for (int64_t t = 0; t < nk; ++t) {
            segment(std::integral_constant<int, 0>{}, t);
            segment(std::integral_constant<int, 1>{}, t);
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

    // ---- a lane's 4 TN consecutive columns of each of its TM rows
    const int64_t n = n0 + wn * WTN + lg * 4 * TN;
    struct __attribute__((packed, aligned(2))) Any16 {
        u32x4 v;
    };
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t m = m0 + wm * WTM + 16 * i + li;
        if (m >= p.M) continue;
        const float f = E4 ? p.x_scale[m] : 1.f;
        uint16_t h[4 * TN];
#pragma unroll
        for (int x = 0; x < 4 * TN; ++x) h[x] = f32_to_bf16_bits(E4 ? acc[i][x / 4][x & 3] * f : acc[i][x / 4][x & 3]);
        uint16_t* y = reinterpret_cast<uint16_t*>(p.Y) + m * p.N + n;
#pragma unroll
        for (int x = 0; x < 4 * TN; x += 8) {
            if (n + x + 8 <= p.N) {
                uint16_t c[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) c[e] = h[x + e];
                reinterpret_cast<Any16*>(y + x)->v = __builtin_bit_cast(u32x4, c);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (n + x + e < p.N) y[x + e] = h[x + e];
            }
        }
    }
}

}  // namespace pifa
