// Grouped products in microscaled 4-bit floating point for many rows: 256 rows of weights by 256, 128 or 64 rows of
// activations on eight waves, operands fetched from memory straight into LDS.
//
// A unit of 256 columns of both operands is, in bytes and in clocks of the matrix units, what 64 columns of bf16 are:
// v_mfma_scale_f32_16x16x128_f8f6f4 takes 16 bytes of a lane and 16 clocks.  What bounds a tile of 256 by 256 is
// therefore what bounds it in bf16: 2048 clocks of products a unit and SIMD, 192 KB of fragment reads (128 B a clock) and
// 68 KB of fills; but there are a quarter as many units, so that a tile's way to its first fill and its epilogue
// weigh four times as much.  The layout of mxfp4.h makes every fill and every fragment read a run of 1 KB, lane
// after lane, free of bank conflicts without a swizzle.
//
// The eight waves are two groups, one wave of each on every SIMD, half a unit apart: while one multiplies out of
// registers, the other reads the fragments of its next unit.  Group 1 fetches, between its products.
// Measured on 2048 / 5632, Zipf loads, us (products of a wave for itself straight from memory / this): gate/up 105 / 72 and down 69 / 38 at 2048 tokens,
// 699 / 440 and 500 / 205 at 16384 (a loop of these instructions on random operands and nothing else reaches 7.1 PFLOP/s, the clock at 1.7 GHz
// under the board's power limit).  Down's figures, here and below, are of rows stored in bf16; in fp32, as now, it takes 42 and 236: 3.3 PFLOP/s over both products.
// The matrix units are busy 42 % of gate/up's clocks and 37 % of down's, at 2.0-2.1 GHz, so that it is not the power limit that holds them: a
// tile of 256 by 256 takes 3200 clocks a unit and 14000 beside them, of which 7000 are the activation's exponentials and reciprocals, with one workgroup
// a CU and so nothing under them.
// Measured and not adopted: tiles one after the other in a workgroup, the fills running on into the next (447 and 204, 477 with a wait behind the stores); fills by the
// group that reads (486 and 237: they stand before the reads); four waves of 128 by 128 and 256 accumulators, two thirds of the fragment reads
// but one wave to a SIMD (607 and 251); fills every second product, column tiles in blocks of one, two or eight: none.
#include "gemm.h"
#include "lds_fill.h"
#include "mxfp4.h"
#include "mxfp4_plan.h"

namespace moe {

namespace {

#define INLINE __attribute__((always_inline))

constexpr int kThreads = 512;

struct MxGemmArgs {
    const char *w0, *w1;  // packed weights (w1: up, with SWIGLU)
    const char* a;        // rows of activations in the layout of mxfp4.h: codes, then scales
    char* out;            // SWIGLU: rows of the next product in that layout; else rows [.., N] in fp32
    const int32_t* starts;  // [E + 1] first block of 32 rows of every expert
    int E, all_blocks, N, K;
};

// Bytes of a stage: a unit of eight blocks of weights and of `blocks` of activations, and their scales, in whole KB
constexpr int mx_stage(int blocks) { return (8 + blocks) * kMxCodes + (8 + (blocks + 3) / 4 * 4) * kMxScales; }

// BS: rows of activations of a tile; NST: units in LDS
template <int BS, int NST, bool SWIGLU>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void mx_gemm_kernel(const MxGemmArgs g) {
    constexpr int WM = BS == 256 ? 2 : 4, WS = 8 / WM;  // waves along the weights, along the activations
    constexpr int WB = 8 / WM, SB = BS / 32 / WS;       // blocks of 32 rows of a wave
    constexpr int SBLK = BS / 32;
    constexpr int W_BYTES = 8 * kMxCodes, S_BYTES = SBLK * kMxCodes;
    constexpr int SC_AT = W_BYTES + S_BYTES, STAGE = mx_stage(SBLK);
    constexpr int OUT_BLOCKS = mx_tile_blocks(SWIGLU);  // blocks of 32 output columns of a tile
    constexpr int NF = 8 + SBLK + 1;                    // fill instructions of a wave of group 1 a unit
    static_assert(WB >= 2 && SB >= 1, "a gate block and its up block are one wave's");
    extern __shared__ __align__(16) char smem[];

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int units = mx_units(g.K), fbs = mx_blocks(g.N), out_units = mx_units(g.N);
    const int out_blocks = SWIGLU ? out_units * (kMxUnit / 32) : fbs;
    int lo = 0, hi = 0, e, row0, row_end, nt;
    if (lane < g.E) {
        lo = g.starts[lane] * 32;
        hi = g.starts[lane + 1] * 32;
    }
    auto n_tiles_of = [&](int) INLINE { return mx_column_tiles(SWIGLU, g.N); };
    // (blocks of four column tiles, and the tiles of a last round that is half full at most in two: 16384 tokens of 2048 / 5632, down 209 -> 203 us)
    if (!find_tile<4, kMxSplitSlots>(lo, hi, g.E, BS, n_tiles_of, e, row0, row_end, nt)) return;
    const int sb0 = row0 >> 5, live_blocks = min(SBLK, (row_end - row0) >> 5);
    const int fb0 = nt * OUT_BLOCKS;
    const int grp = wave >> 2, wm = (wave % (2 * WM)) % WM, ws = wave / WM;

    // ---- fills, by the four waves of group 1: wave w takes the w-th KB of every block's unit
    const int fw = wave & 3;
    const size_t w_stride = (size_t)units * kMxCodes, w_first = (size_t)e * fbs, w_scales = (size_t)g.E * fbs * units * kMxCodes;
    const unsigned lds0 = (unsigned)(uintptr_t)(lds_char*)smem;
    const unsigned off = lane * 16;
    // the scales: KB w of the unit's (weights 8 blocks, activations SBLK), a block 16 lanes (the last one again where there is none)
    const char* sc_src;
    unsigned sc_off, sc_lds;
    {
        constexpr int S_INSTR = (SBLK + 3) / 4;
        const int part = min(fw, 1 + S_INSTR), b = (part < 2 ? part : part - 2) * 4 + (lane >> 4);
        if (part < 2) {
            const bool up = SWIGLU && part == 1;
            const int blk = min(fb0 + (SWIGLU ? b & 3 : b), fbs - 1);
            sc_src = (up ? g.w1 : g.w0) + w_scales + w_first * units * kMxScales;
            sc_off = (unsigned)blk * units * kMxScales + (lane & 15) * 16;
        } else {
            sc_src = g.a + ((size_t)g.all_blocks * units) * kMxCodes + (size_t)sb0 * units * kMxScales;
            sc_off = (unsigned)min(min(b, SBLK - 1), live_blocks - 1) * units * kMxScales + (lane & 15) * 16;
        }
        sc_lds = SC_AT + part * 1024;
    }
    auto fill = [&](int v, int p) INLINE {
        const unsigned stage = lds0 + v % NST * STAGE;
        if (p < 8) {  // block p of the weights
            const bool up = SWIGLU && p >= 4;
            const int blk = min(fb0 + (SWIGLU ? p & 3 : p), fbs - 1);
            dma16<false>(stage + p * kMxCodes + fw * 1024, (up ? g.w1 : g.w0) + (w_first + blk) * w_stride + (size_t)v * kMxCodes + fw * 1024, off);
        } else if (p < 8 + SBLK) {
            const int blk = sb0 + min(p - 8, live_blocks - 1);
            dma16<false>(stage + W_BYTES + (p - 8) * kMxCodes + fw * 1024, g.a + (size_t)blk * w_stride + (size_t)v * kMxCodes + fw * 1024, off);
        } else {
            dma16<false>(stage + sc_lds, sc_src + (size_t)v * kMxScales, sc_off);
        }
    };

    f32x4 acc[WB][SB][2][2];
#pragma unroll
    for (int i = 0; i < WB * SB * 4; ++i) acc[i / (SB * 4)][i / 4 % SB][i / 2 % 2][i % 2] = f32x4{0.f, 0.f, 0.f, 0.f};
    // the wave's blocks of rows are ws, ws + WS, ...
    const int live = max(0, min(SB, (live_blocks - ws + WS - 1) / WS));

    auto k_loop = [&](auto live_c, auto gc) INLINE {
        constexpr int L = decltype(live_c)::value, GRP = decltype(gc)::value, LR = L > 0 ? L : 1;
        i32x4 fw_[2][WB][2], fs[2][LR][2];
        int sw[WB], ss[LR];
        // SWIGLU: the wave's blocks are WB / 2 of gate and as many of up
        auto w_block = [&](int b) INLINE { return SWIGLU ? (b < WB / 2 ? wm * (WB / 2) + b : 4 + wm * (WB / 2) + b - WB / 2) : wm * WB + b; };
        auto read = [&](int v) INLINE {
            const char* st = smem + v % NST * STAGE;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int b = 0; b < WB; ++b)
#pragma unroll
                    for (int t = 0; t < 2; ++t) fw_[c][b][t] = *reinterpret_cast<const i32x4*>(st + w_block(b) * kMxCodes + (c * 2 + t) * 1024 + lane * 16);
#pragma unroll
                for (int i = 0; i < L; ++i)
#pragma unroll
                    for (int t = 0; t < 2; ++t)
                        fs[c][i][t] = *reinterpret_cast<const i32x4*>(st + W_BYTES + (ws + i * WS) * kMxCodes + (c * 2 + t) * 1024 + lane * 16);
            }
#pragma unroll
            for (int b = 0; b < WB; ++b) sw[b] = *reinterpret_cast<const int*>(st + SC_AT + w_block(b) * kMxScales + lane * 4);
#pragma unroll
            for (int i = 0; i < L; ++i) ss[i] = *reinterpret_cast<const int*>(st + SC_AT + (8 + ws + i * WS) * kMxScales + lane * 4);
        };
        auto multiply = [&](auto filling, int vf) INLINE {
            constexpr bool FILL = decltype(filling)::value;
            constexpr int NM = L * WB * 8, GAP = NM / NF > 0 ? NM / NF : 1;
            int p = 0, n = 0;
            auto between = [&]() INLINE {
                if (FILL && n % GAP == GAP - 1 && p < NF) {
                    __builtin_amdgcn_sched_barrier(0);
                    fill(vf, p);
                    ++p;
                    __builtin_amdgcn_sched_barrier(0);
                }
                ++n;
            };
#pragma unroll
            for (int b = 0; b < WB; ++b)
#pragma unroll
                for (int i = 0; i < L; ++i) {
                    auto& A = acc[b][i];
                    A[0][0] = mx_mfma<0, 0>(fw_[0][b][0], fs[0][i][0], A[0][0], sw[b], ss[i]), between();
                    A[0][1] = mx_mfma<0, 1>(fw_[0][b][0], fs[0][i][1], A[0][1], sw[b], ss[i]), between();
                    A[1][0] = mx_mfma<1, 0>(fw_[0][b][1], fs[0][i][0], A[1][0], sw[b], ss[i]), between();
                    A[1][1] = mx_mfma<1, 1>(fw_[0][b][1], fs[0][i][1], A[1][1], sw[b], ss[i]), between();
                }
#pragma unroll
            for (int b = 0; b < WB; ++b)
#pragma unroll
                for (int i = 0; i < L; ++i) {
                    auto& A = acc[b][i];
                    A[0][0] = mx_mfma<2, 2>(fw_[1][b][0], fs[1][i][0], A[0][0], sw[b], ss[i]), between();
                    A[0][1] = mx_mfma<2, 3>(fw_[1][b][0], fs[1][i][1], A[0][1], sw[b], ss[i]), between();
                    A[1][0] = mx_mfma<3, 2>(fw_[1][b][1], fs[1][i][0], A[1][0], sw[b], ss[i]), between();
                    A[1][1] = mx_mfma<3, 3>(fw_[1][b][1], fs[1][i][1], A[1][1], sw[b], ss[i]), between();
                }
            if (FILL) {
#pragma unroll
                for (; p < NF; ++p) fill(vf, p);
            }
        };
        // Group 0 reads unit v in phase 2 v and multiplies in phase 2 v + 1, group 1 a phase later.  The stage of unit v is free
        // from the end of phase 2 v + 1 on: group 1, multiplying unit v in phase 2 v + 2, fetches unit v + NST into it.  Unit
        // v + 1 has to have landed when phase 2 v + 2 begins: group 1 waits for it in phase 2 v + 1.
        if constexpr (GRP == 1) {
#pragma unroll
            for (int u = 0; u < NST; ++u)
                if (u < units) {
#pragma unroll
                    for (int p = 0; p < NF; ++p) fill(u, p);
                }
            if (units >= NST) wait_vm<(NST - 1) * NF>();
            else wait_vm<0>();
            phase_end();
        }
        phase_end();
        int v = 0;
        for (; v + NST < units; ++v) {
            if (L > 0) read(v);
            if (GRP == 1) wait_vm<(NST - 2) * NF>();
            phase_end();
            multiply(std::integral_constant<bool, GRP == 1>{}, v + NST);
            phase_end();
        }
        for (; v < units; ++v) {
            if (L > 0) read(v);
            if (GRP == 1) wait_vm<0>();
            phase_end();
            multiply(std::false_type{}, 0);
            phase_end();
        }
        if constexpr (GRP == 0) phase_end();
    };
    auto loops = [&](auto live_c) INLINE {
        if (grp == 0) k_loop(live_c, std::integral_constant<int, 0>{});
        else k_loop(live_c, std::integral_constant<int, 1>{});
    };
    if (live == SB) loops(std::integral_constant<int, SB>{});
    else if (live == 0) loops(std::integral_constant<int, 0>{});
    else loops(std::integral_constant<int, 1>{});

    // ---- epilogue: a lane holds columns 32 fb + 8 (lane / 16) .. + 8 of rows lane % 16 of both tiles of a block of rows
    char* const out_scales = g.out + (size_t)g.all_blocks * out_units * kMxCodes;
#pragma unroll
    for (int i = 0; i < SB; ++i) {
        if (i >= live) continue;
        const int sb = sb0 + ws + i * WS;
#pragma unroll
        for (int b = 0; b < (SWIGLU ? WB / 2 : WB); ++b) {
            const int fb = fb0 + (SWIGLU ? wm * (WB / 2) + b : wm * WB + b);
            if (fb >= out_blocks) continue;
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float z = acc[b][i][j / 4][n][j % 4];
                    f[j] = SWIGLU ? (fb < fbs ? silu_f32(z) * acc[(b + WB / 2) % WB][i][j / 4][n][j % 4] : 0.f) : z;  // (beyond: the last block's again)
                }
                if constexpr (SWIGLU) mx_store_hidden(f, g.out, out_scales, out_units, sb, n, fb, lane);
                else mx_store_rows(f, g.out, g.N, sb, n, fb, lane);
            }
        }
    }
}

template <int BS, int NST, bool SWIGLU>
int launch_tile(const MxGemmArgs& g, int P, hipStream_t st) {
    constexpr int SBLK = BS / 32;
    constexpr size_t lds = (size_t)NST * mx_stage(SBLK);
    static_assert(lds <= 160 * 1024, "of a CU");
    const int tiles = (int)mx_tiles(SWIGLU, P, g.E, g.N, BS);
    auto kern = mx_gemm_kernel<BS, NST, SWIGLU>;
    static std::atomic<uint64_t> allowed{0};
    if (allow_dynamic_lds(reinterpret_cast<const void*>(kern), lds, allowed) != MOE_OK) return MOE_ERR_LAUNCH;
    hipLaunchKernelGGL(kern, dim3(find_tile_grid(tiles, kMxSplitSlots)), dim3(kThreads), lds, st, g);
    return launch_status();
}

template <bool SWIGLU>
int launch_product(const MxGemmArgs& g, int P, int bs, hipStream_t st) {
    if (bs == 256) return launch_tile<256, 2, SWIGLU>(g, P, st);
    if (bs == 128) return launch_tile<128, 3, SWIGLU>(g, P, st);
    return launch_tile<64, 3, SWIGLU>(g, P, st);
}

}  // namespace

int launch_mx_gemm(bool swiglu, const void* w0, const void* w1, const char* a, char* out, const int32_t* starts, int P, int E,
                   int all_blocks, int N, int K, int bs, hipStream_t st) {
    const MxGemmArgs g{static_cast<const char*>(w0), static_cast<const char*>(w1), a, out, starts, E, all_blocks, N, K};
    return swiglu ? launch_product<true>(g, P, bs, st) : launch_product<false>(g, P, bs, st);
}

}  // namespace moe
