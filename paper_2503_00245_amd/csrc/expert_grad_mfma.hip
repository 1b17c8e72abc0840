// Gradient of bf16 experts on tiles of 256 (or 128) rows, operands fetched from memory straight into LDS (expert_grad.h names the
// products).
//
// What bounds it: matrix operations for many rows (16 P d F of them), weights and their gradients for few.
//
// Layouts.  An operand whose k-values are neighbours in memory (rows of x, gy, da, db; W_gate and W_up where k runs along
// d) lies in LDS as rows of 128 bytes, a k-step, and a lane's eight k-values are one 16-byte read.  The other operands (W_down under dh,
// W_gate and W_up under gx, and both operands of the gradients of weights, where k runs along the tokens) lie as they come,
// 64 rows of k by the tile's columns, and are transposed on their way out of LDS: ds_read_b64_tr_b16 hands a lane four k-values of its
// column, from four rows of which each of 16 lanes names 8 bytes.  No transposed copy of anything is made.  Both kinds of rows are swizzled
// on the memory side so that reads meet no bank conflict: chunks of 16 bytes by half the row's number, and, in rows read transposed,
// units of 32 bytes (16 columns) by bits 0, 1 and 3 of the row's (two groups of 16 lanes read rows r .. r + 3 and r + 8 .. r + 11).
//
// Schedule: that of expert_gemm_pp.hip.  Eight waves in two groups half a k-step apart: one multiplies out of registers while the
// other reads the fragments of its whole next step; fills go between the products, B by group 0, A by group 1.
//
// The activation's gradient needs a, b and dh of the same place: one workgroup forms all three for 128 columns (192
// accumulator registers a lane) or 96 (144), a and b in a first pass over d, dh in a second one.  dh then is never rounded nor
// stored: as a tensor of its own in bf16 it raised the error of the gradients from 2.3e-3 to 2.9e-3.
//
// Measured, 16384 tokens of 2048 / 5632, Zipf loads: a, b, dh 2135 us (1.06 PFLOP/s), weights 1758 (1.29), rows 1222 (1.24); a library product of 8192^3 runs at
// 1.44.  What is left out in turn (a copy, for timing): without fills 1640 / 1470 / 950 us, without products 1890 / 1513 / 1040.  Fills come at 46 GB/s a CU,
// bound by how far ahead LDS lets them be asked for (98 GB/s for the same pattern without the schedule), so bytes of fill a
// product count: a, b, dh of 128 columns at a time need a fifth less of them than of 96 (2370 -> 2140 us).
#include "expert_grad.h"
#include "expert_grad_plan.h"
#include "lds_fill.h"

#include <algorithm>

namespace moe {

namespace {

#define INLINE __attribute__((always_inline))

constexpr int BK = 64, kThreads = 512;
constexpr int kSplitSlots = 32;  // one workgroup per CU

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Gradients of weights are written past the caches: they are not read again here, and the weights and rows that are stay there (24 tokens of 1024 / 2816,
// 4 of 16 experts: gx, whose weights the product before has read, 55 -> 31 us, a and b and dh 79 -> 70)
__device__ __forceinline__ void store_past(void* p, uint4 v) {
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), reinterpret_cast<u32x4*>(p));
}

// Four k-values of the lane's column, twice: rows at and at + rows4 of LDS
__device__ __forceinline__ bf16x8 read_transposed(unsigned at, unsigned rows4) {
#if defined(__HIP_DEVICE_COMPILE__)
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4*>((uintptr_t)at));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4*>((uintptr_t)(at + rows4)));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
#else
    return bf16x8{};
#endif
}

// A fragment's eight k-values from k on, those from `left` on as zeros.  (Two to a register: value by value it was a third of all vector
// instructions of a tile of few steps.)
__device__ __forceinline__ bf16x8 first_of(bf16x8 v, int k, int left) {
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    u32x4 u = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int j = 0; j < 4; ++j) u[j] &= k + 2 * j + 1 < left ? ~0u : k + 2 * j < left ? 0xFFFFu : 0u;
    return __builtin_bit_cast(bf16x8, u);
}

// BM, COLS: rows and output columns of a tile (DX, WEIGHTS: 256 columns)
template <int OP, int BM, int COLS>
struct Form {
    static constexpr bool ACT = OP == GRAD_ACT, WGT = OP == GRAD_WEIGHTS;
    static constexpr int WAVES_M = ACT && BM == 256 ? 4 : 2, WAVES_N = 8 / WAVES_M;
    static constexpr int MB = BM / 32 / WAVES_M;     // 32-row blocks of a wave: wm, wm + WAVES_M, ...
    static constexpr int NI = (ACT ? 2 : 1) * COLS / WAVES_N / 16;  // 16-column blocks of a wave (ACT: half of them a, half b; then half as many dh)
    static constexpr int KS = ACT && BM == 256 && COLS == 128 ? 2 : 1;  // phases that a k-step is multiplied in: with 192 accumulators a lane, half a step's fragments at a time
    static constexpr int SA = BM == 128 ? 4 : 2, SB = COLS == 96 ? 4 : 3;  // k-steps in LDS
    static constexpr int A_BYTES = BM * BK * 2, B_BYTES = (ACT ? 2 : 1) * COLS * BK * 2;
    static constexpr int LDS = SA * A_BYTES + SB * B_BYTES;
    static_assert(LDS <= 160 * 1024, "LDS of a CU");
};

// Sizes of a group in descending order: the expert of each rank in lane `rank`.  (The gradients of weights take as long as an expert has
// rows: long ones go first.)
__device__ __forceinline__ int by_size(int count, int E) {
    const int lane = threadIdx.x & (kWave - 1);
    int rank = 0;
    for (int e = 0; e < E; ++e) {
        const int c = MOE_READLANE(count, e);
        rank += c > count || (c == count && e < lane) ? 1 : 0;
    }
    // lane r: the lane whose rank is r
    return __builtin_amdgcn_ds_permute((lane < E ? rank : lane) << 2, lane);
}

// PARTS (DX): the k-steps of a tile are cut into g.k_parts runs, each stored in fp32 to an output of its own
template <int OP, int BM, int COLS, bool PARTS>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void grad_kernel(const GradArgs g) {
    typedef Form<OP, BM, COLS> F;
    constexpr bool ACT = F::ACT, WGT = F::WGT;
    constexpr int WAVES_M = F::WAVES_M, WAVES_N = F::WAVES_N, MB = F::MB, BN = COLS, NI = F::NI, SA = F::SA, SB = F::SB, KS = F::KS;
    constexpr int A_BYTES = F::A_BYTES, B_BYTES = F::B_BYTES, B_AT = SA * A_BYTES;
    extern __shared__ __align__(16) char smem[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int grp = wave >> 2, fw = wave & 3;
    const int wm = wave / WAVES_N, wn = wave % WAVES_N;

    // ---- the tile
    int lo, hi, e, m0, m_end, n0, part = 0, which = 0;
    int M_pitch, N, K;  // A's row pitch (transposed: its columns), output columns, k-values (of a pass)
    group_bounds(g.offsets, g.E, g.P, lo, hi);
    lo = min(max(lo, 0), g.P), hi = min(max(hi, lo), g.P);
    const char *A0, *A1, *B0, *B1, *B2 = nullptr;
    const size_t at_w = (size_t)g.d * g.F * 2;
    if constexpr (WGT) {
        // Strips of 256 hidden columns of an expert's three matrices, by all tiles across d; strips are dealt to the XCDs in turn.
        const int dt = (g.d + 255) / 256, ft = (g.F + 255) / 256, slot = blockIdx.x >> 3;
        const int strip = uniform_div(slot, dt) * 8 + (blockIdx.x & 7), across = slot - uniform_div(slot, dt) * dt;
        const int rank = uniform_div(strip, 3 * ft), in = strip - rank * 3 * ft;
        if (rank >= g.E) return;
        e = MOE_READLANE(by_size(hi - lo, g.E), rank);
        which = uniform_div(in, ft);
        const int hidden = in - which * ft;
        if (!(which == 0 ? g.gw_gate : which == 1 ? g.gw_up : g.gw_down)) return;
        M_pitch = which == 2 ? g.d : g.F, N = which == 2 ? g.F : g.d;
        m0 = (which == 2 ? across : hidden) * BM, n0 = (which == 2 ? hidden : across) * BN, m_end = M_pitch;
        const int first = MOE_READLANE(lo, e);
        K = MOE_READLANE(hi, e) - first;
        A0 = A1 = static_cast<const char*>(which == 0 ? g.da : which == 1 ? g.db : g.gy) + (size_t)first * M_pitch * 2;
        B0 = B1 = static_cast<const char*>(which == 2 ? g.h : g.x) + (size_t)first * N * 2;
    } else {
        N = ACT ? g.F : g.d, K = M_pitch = ACT ? g.d : g.F;
        int nt;
        const int n_tiles = (N + BN - 1) / BN, copies = PARTS ? g.k_parts : 1;
        if (!find_tile<ACT ? 4 : kHiddenOperandBlock, kSplitSlots>(lo, hi, g.E, BM, [&](int) INLINE { return n_tiles * copies; }, e, m0, m_end, nt)) return;
        if (PARTS) {
            part = uniform_div(nt, n_tiles);
            nt -= part * n_tiles;
        }
        n0 = nt * BN;
        const size_t at_row = (size_t)m0 * M_pitch * 2, at_col = ACT ? (size_t)n0 * K * 2 : 0;  // (rows of 128 bytes: from the tile's first on)
        A0 = static_cast<const char*>(ACT ? g.x : g.da) + at_row, A1 = static_cast<const char*>(ACT ? g.gy : g.db) + at_row;
        B0 = static_cast<const char*>(g.w_gate) + e * at_w + at_col, B1 = static_cast<const char*>(g.w_up) + e * at_w + at_col;
        if (ACT) B2 = static_cast<const char*>(g.w_down) + e * at_w;
    }
    const int nk = (K + BK - 1) / BK;              // k-steps of a pass
    int v0 = 0, v_end = WGT ? nk : 2 * nk;         // those of this workgroup (ACT, DX: steps of the second pass from nk on)
    if (PARTS) v0 = uniform_div(2 * nk * part, g.k_parts), v_end = uniform_div(2 * nk * (part + 1), g.k_parts);
    const int rows_here = m_end - m0;
    const unsigned pitch_a = (unsigned)M_pitch * 2, pitch_b = (unsigned)N * 2;  // bytes (pitch_b: operands read transposed)

    // ---- fills.  Instruction p of wave w % 4 = fw writes the KB 4 p + fw of its operand's step; lane l the l-th 16 bytes of it.
    const unsigned lds0 = (unsigned)(uintptr_t)(lds_char*)smem;
    constexpr int PA = BM / 32;
    constexpr int PB0 = F::B_BYTES / 4096, PB1 = ACT ? 4 : 8;  // of B in the first and in the second pass
    // rows of 128 bytes: row 8 (4 p + fw) + l / 8, slot l % 8 = chunk ^ (row / 2) % 8
    const int k_row = fw * 8 + (lane >> 3);
    const unsigned k_chunk = ((lane & 7) ^ (((fw & 1) << 2) | (lane >> 4))) * 16;
    // rows of 512 bytes: row 2 (4 p + fw) + l / 32, slot l % 32 = chunk ^ 2 f, f = bits 0, 1 and 3 of the row
    const int t_row = fw * 2 + (lane >> 5);
    const int t_chunk = (lane & 31) ^ ((t_row & 3) << 1);  // (p odd: ^ 8)
    // Lane offsets are kept whole: beside them a fill takes scalar operations only.  The last step of ACT and DX is fetched as the last 64
    // k-values; those that it shares with the step before are taken out of A's fragments.
    unsigned off[8], col[2] = {};
    if (grp == 1 && !WGT) {
#pragma unroll
        for (int p = 0; p < PA; ++p) off[p] = (unsigned)min(k_row + 32 * p, m_end - 1 - m0) * pitch_a + k_chunk;
    } else if (grp == 1) {
#pragma unroll
        for (int p = 0; p < 2; ++p) col[p] = (unsigned)min(m0 + (t_chunk ^ (p << 3)) * 8, M_pitch - 8) * 2;
    } else if (ACT) {
#pragma unroll
        for (int p = 0; p < BN / 32; ++p) off[p] = (unsigned)min(k_row + 32 * p, N - 1 - n0) * ((unsigned)K * 2) + k_chunk;
        // rows of 256 bytes (16 chunks; of 96 columns they are 12): row 4 (4 p + fw) + l / 16
        const int f = (lane >> 4) | (fw >> 1) << 2;
        col[0] = (unsigned)min(n0 + min((lane & 15) ^ (f << 1), BN / 8 - 1) * 8, N - 8) * 2 + (unsigned)(4 * fw + (lane >> 4)) * pitch_b;
    } else {
#pragma unroll
        for (int p = 0; p < 2; ++p) col[p] = (unsigned)min(n0 + (t_chunk ^ (p << 3)) * 8, N - 8) * 2;
    }
    if (!(ACT || (grp == 1 && !WGT))) {
#pragma unroll
        for (int p = 0; p < 2; ++p) col[p] += (unsigned)t_row * (grp == 1 ? pitch_a : pitch_b);
    }
    // instruction p of step v (of pass S: ACT's differ; WGT: 2 is a last step of fewer than 64 rows, the others of which are the last again)
    auto fill = [&](auto gc, auto sc, int v, int p) INLINE {
        constexpr int GRP = decltype(gc)::value, S = decltype(sc)::value;
        const bool second = !WGT && (ACT ? S == 1 : v >= nk);
        const int t = second ? v - nk : v, k0 = WGT ? t * BK : min(t * BK, K - BK);
        const unsigned slot = lds0 + (GRP == 1 ? v % SA * A_BYTES : B_AT + v % SB * B_BYTES) + fw * 1024 + p * 4096;
        if constexpr (GRP == 1 && !WGT) {
            dma16<false>(slot, (second ? A1 : A0) + k0 * 2, off[p]);
        } else if constexpr (GRP == 0 && ACT && S == 0) {
            dma16<false>(slot, (p < PB0 / 2 ? B0 : B1) + k0 * 2, off[p % (PB0 / 2)]);
        } else if constexpr (GRP == 0 && ACT) {
            dma16<false>(slot, B2 + (size_t)(unsigned)(k0 + 16 * p) * pitch_b, col[0]);
        } else {
            const unsigned pitch = GRP == 1 ? pitch_a : pitch_b;
            const char* const src = GRP == 1 ? A0 : second ? B1 : B0;
            if constexpr (S == 2) {
                const int row = min(8 * p + t_row, K - 1 - k0);
                dma16<false>(slot, src + (size_t)(unsigned)k0 * pitch, col[p & 1] + (unsigned)(row - t_row) * pitch);
            } else {
                dma16<false>(slot, src + (size_t)(unsigned)(k0 + 8 * p) * pitch, col[p & 1]);
            }
        }
    };

    f32x4 acc[2 * MB][NI], acc2[ACT ? 2 * MB : 1][ACT ? NI / 2 : 1];
#pragma unroll
    for (int mi = 0; mi < 2 * MB; ++mi)
#pragma unroll
        for (int ni = 0; ni < NI; ++ni) acc[mi][ni] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (ACT) {
#pragma unroll
        for (int mi = 0; mi < 2 * MB; ++mi)
#pragma unroll
            for (int ni = 0; ni < NI / 2; ++ni) acc2[mi][ni] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int live = min(MB, max(0, ((min(rows_here, BM) + 31) / 32 + WAVES_M - 1 - wm) / WAVES_M));

    // ---- fragment reads.  Rows of 128 bytes: row l % 16 of a block, chunk 4 ks + l / 16.
    const unsigned c16 = ((lane >> 4) ^ ((lane & 15) >> 1)) << 4;
    const unsigned ra = lds0 + wm * 4096 + (lane & 15) * 128 + c16;
    const unsigned rb = lds0 + B_AT + wn * (BN / WAVES_N) * 128 + (lane & 15) * 128 + c16;  // (ACT, first pass)
    // rows read transposed: row 8 (l / 16) + (l % 16) / 4 (+ 4) of a 32-row half step, 8 bytes (l % 4) of unit u ^ f
    constexpr int T_ROW = ACT ? 256 : 512;
    const unsigned t_swz = (((lane & 15) >> 2) | ((lane >> 4) & 1) << 2) << 5;
    const unsigned t_lane = lds0 + (8 * (lane >> 4) + ((lane & 15) >> 2)) * T_ROW + (lane & 3) * 8;

    auto k_loop = [&](auto ma, auto gc) INLINE {
        constexpr int MA = decltype(ma)::value, GRP = decltype(gc)::value, MR = MA > 0 ? MA : 1;
        constexpr int NFA = WGT || MA == MB ? PA : std::min(PA, WAVES_M * (MA + 1) - 1);
        constexpr int AHEAD = GRP == 0 ? SB - 1 : SA;
        constexpr int HS = 2 / KS;  // half steps (32 k-values) of a phase
        bf16x8 fa[HS][2 * MR], fb[HS][NI];
        auto read = [&](auto sc, int v, int phase) INLINE {
            constexpr int S = decltype(sc)::value, N_I = ACT && S == 1 ? NI / 2 : NI;
            const unsigned pa = v % SA * A_BYTES, pb = v % SB * B_BYTES;
            // (an address for each unit is made here, of two instructions; kept over the loop, they did not fit the registers)
            unsigned swz = t_swz;
#if defined(__HIP_DEVICE_COMPILE__)
            if (!ACT || S == 1) asm volatile("" : "+v"(swz));
#endif
#pragma unroll
            for (int q = 0; q < HS; ++q) {
                const int ks = KS == 2 ? phase : q;
#pragma unroll
                for (int ni = 0; ni < N_I; ++ni) {
                    if constexpr (ACT && S == 0) {
                        fb[q][ni] = *reinterpret_cast<const __attribute__((address_space(3))) bf16x8*>(
                            (uintptr_t)((rb ^ (ks << 6)) + pb + (ni / (NI / 2)) * (BN * 128) + (ni % (NI / 2)) * 2048));
                    } else if constexpr (ACT) {
                        const unsigned unit = (unsigned)(wn * (NI / 2) + ni) << 5;
                        fb[q][ni] = read_transposed((unit ^ swz) + (t_lane + B_AT + pb) + ks * (32 * T_ROW), 4 * T_ROW);
                    } else {
                        const unsigned unit = (unsigned)(wn * NI + ni) << 5;
                        fb[q][ni] = read_transposed((unit ^ swz) + (t_lane + B_AT + pb) + ks * (32 * T_ROW), 4 * T_ROW);
                    }
                }
#pragma unroll
                for (int mi = 0; mi < 2 * MA; ++mi) {
                    if constexpr (WGT) {
                        const unsigned unit = (unsigned)((wm + (mi >> 1) * WAVES_M) * 2 + (mi & 1)) << 5;
                        fa[q][mi] = read_transposed((unit ^ swz) + (t_lane + pa) + ks * (32 * T_ROW), 4 * T_ROW);
                    } else {
                        fa[q][mi] = *reinterpret_cast<const __attribute__((address_space(3))) bf16x8*>(
                            (uintptr_t)((ra ^ (ks << 6)) + pa + (mi >> 1) * (WAVES_M * 4096) + (mi & 1) * 2048));
                    }
                }
            }
        };
        // the last step of a pass, `left` k-values of which are its own: the others are taken out of A (an infinite value of B there makes NaN of
        // an infinite result: non-finite inputs are unspecified)
        auto clear_others = [&](int left, int phase) INLINE {
#pragma unroll
            for (int q = 0; q < HS; ++q) {
                const int ks = KS == 2 ? phase : q;
                if constexpr (WGT) {  // they are the last ones
#pragma unroll
                    for (int mi = 0; mi < 2 * MA; ++mi) fa[q][mi] = first_of(fa[q][mi], ks * 32 + (lane >> 4) * 8, left);
                } else if (ks * 32 + (lane >> 4) * 8 < BK - left) {  // they are the first ones (a multiple of 8)
#pragma unroll
                    for (int mi = 0; mi < 2 * MA; ++mi) fa[q][mi] = bf16x8{};
                }
            }
        };
        // products of a phase of pass S, between them fills [p, p_end) of step vf of pass SF
        auto multiply = [&](auto sc, auto sf, auto pc, auto pn, int vf) INLINE {
            constexpr int S = decltype(sc)::value, N_I = ACT && S == 1 ? NI / 2 : NI;
            constexpr int P0 = decltype(pc)::value, P_END = decltype(pn)::value, NF = P_END - P0;
            constexpr int NM = MA * 2 * HS * N_I, GAP = std::max(1, NM / std::max(1, NF));
            int p = P0;
#pragma unroll
            for (int i = 0; i < NM; ++i) {
                const int ni = i % N_I, mi = i / N_I % (2 * MR), q = i / (N_I * 2 * MR);
                f32x4& c = ACT && S == 1 ? acc2[ACT ? mi : 0][ACT ? ni : 0] : acc[mi][ni];
                c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[q][ni], fa[q][mi], c, 0, 0, 0);
                if (i % GAP == GAP - 1 && p < P_END) {
                    __builtin_amdgcn_sched_barrier(0);
                    fill(gc, sf, vf, p);
                    ++p;
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
#pragma unroll
            for (; p < P_END; ++p) fill(gc, sf, vf, p);
        };
        // steps [from, to) of pass S while those AHEAD of them, of pass SF, are fetched
        auto steps = [&](int from, int to, auto sc, auto sf) INLINE {
            constexpr int S = decltype(sc)::value, SF = decltype(sf)::value;
            constexpr int NF = SF < 0 ? 0 : GRP == 1 ? NFA : SF == 1 ? PB1 : PB0;
            constexpr int FLY = SF < 0 ? 0 : GRP == 0 ? (AHEAD - 1) * NF : (SA - 2) * NFA;
            for (int v = from; v < to; ++v) {
                static_for<KS>([&](auto phase) INLINE {
                    constexpr bool LAST = phase == KS - 1;
                    if (MA > 0) {
                        read(sc, v, phase);
                        // (DX: the first pass may end among steps that still fetch)
                        if (SF < 0 || (ACT && SF != S) || OP == GRAD_DX) {
                            const int t = WGT || S == 0 ? (OP == GRAD_DX && v >= nk ? v - nk : v) : v - nk;
                            if (t == nk - 1 && K % BK) clear_others(K - t * BK, phase);
                        }
                    }
                    if (GRP == 1 && LAST) wait_vm<FLY>();  // A of step v + 1
                    phase_end();
                    // A's slot is free once its step's last phase has been read; B's is that of the step before
                    constexpr int P0 = GRP == 1 ? (LAST ? 0 : NF) : NF * phase / KS, P_END = GRP == 1 ? NF : NF * (phase + 1) / KS;
                    multiply(sc, sf, std::integral_constant<int, P0>{}, std::integral_constant<int, P_END>{}, v + AHEAD);
                    if (GRP == 0 && LAST) wait_vm<FLY>();  // B of step v + 1
                    phase_end();
                });
            }
        };
        typedef std::integral_constant<int, 0> s0;
        typedef std::integral_constant<int, 1> s1;
        typedef std::integral_constant<int, 2> s_last;
        typedef std::integral_constant<int, -1> none;
        const int nv = v_end - v0;
        const bool ragged = WGT && K % BK;
        constexpr int NF0 = GRP == 1 ? NFA : PB0;
#pragma unroll
        for (int q = 0; q < AHEAD; ++q)
            if (q < nv) {
                if (ragged && q == nk - 1) {
#pragma unroll
                    for (int p = 0; p < NF0; ++p) fill(gc, s_last{}, q, p);
                } else {
#pragma unroll
                    for (int p = 0; p < NF0; ++p) fill(gc, s0{}, v0 + q, p);
                }
            }
        if (nv >= AHEAD) wait_vm<(AHEAD - 1) * NF0>();  // the first step has landed
        else wait_vm<0>();
        phase_end();
        if (GRP == 1) phase_end();
        if constexpr (ACT) {  // (nk >= AHEAD: run_grad_mfma)
            steps(0, nk - AHEAD, s0{}, s0{});
            steps(nk - AHEAD, nk, s0{}, s1{});
            steps(nk, 2 * nk - AHEAD, s1{}, s1{});
            steps(2 * nk - AHEAD, 2 * nk, s1{}, none{});
        } else {
            const int mid = max(v0, v_end - AHEAD);
            const int whole = ragged ? max(v0, mid - 1) : mid;
            steps(v0, whole, s0{}, s0{});
            if constexpr (WGT) steps(whole, mid, s0{}, s_last{});
            steps(mid, v_end, s0{}, none{});
        }
    };
    auto loops = [&](auto ma) INLINE {
        if (grp == 0) k_loop(ma, std::integral_constant<int, 0>{});
        else k_loop(ma, std::integral_constant<int, 1>{});
    };
    if (v_end > v0) {  // (an expert without rows: zeros)
        if (live == MB) loops(std::integral_constant<int, MB>{});
        else if (live == 0) loops(std::integral_constant<int, 0>{});
        else if (live == 1) loops(std::integral_constant<int, 1>{});
        else if (live == 2) loops(std::integral_constant<int, (MB > 2 ? 2 : 1)>{});
        else loops(std::integral_constant<int, (MB > 3 ? 3 : 1)>{});
        if (grp == 0) phase_end();
    }

    // ---- epilogue: accumulator element i of a block is output column 4 (lane / 16) + i of row lane % 16.
    if constexpr (PARTS) {
        float* const out = g.parts + (size_t)part * g.P * N + (size_t)m0 * N + n0;
#pragma unroll
        for (int mi = 0; mi < 2 * MB; ++mi) {
            if (mi / 2 >= live) continue;
            const int row = (WAVES_M * (mi / 2) + wm) * 32 + mi % 2 * 16 + (lane & 15);
#pragma unroll
            for (int ni = 0; ni < NI; ++ni) {
                const int c = (wn * NI + ni) * 16 + (lane >> 4) * 4;
                if (row < rows_here && n0 + c < N) *reinterpret_cast<f32x4*>(out + (size_t)row * N + c) = acc[mi][ni];
            }
        }
        return;
    }
    // Staged through LDS, 32 rows at a time in a region per wave, so that the tile leaves in 16-byte stores.
    constexpr int OC = BN / WAVES_N, PITCH = OC * 2 + 16;
    constexpr int LPR = OC / 8, RPI = 64 / LPR;
    char* const region = smem + wave * (32 * PITCH);
    char* const wr = region + (lane & 15) * PITCH + (lane >> 4) * 8;
    const int rd_row = lane / LPR, rd_chunk = lane % LPR;
    const int c0 = wn * OC + rd_chunk * 8;
    auto leave = [&](int rbk, bf16_t* out) INLINE {  // the staged 32 rows
#pragma unroll
        for (int it = 0; it < (32 + RPI - 1) / RPI; ++it) {
            const int r = it * RPI + rd_row;
            if ((64 % LPR || 32 % RPI) && (rd_row >= RPI || r >= 32)) continue;
            const uint4 v = *reinterpret_cast<const uint4*>(region + r * PITCH + rd_chunk * 16);
            if (rbk + r >= rows_here || n0 + c0 >= N) continue;
            uint4* const to = reinterpret_cast<uint4*>(out + (size_t)(rbk + r) * N + c0);
            if (WGT) store_past(to, v);
            else *to = v;
        }
    };
    const size_t at0 = (size_t)m0 * N + n0;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        if (mb >= live) continue;
        const int rbk = (WAVES_M * mb + wm) * 32;
        if constexpr (ACT) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int nb = 0; nb < NI / 2; ++nb)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const ActGrad v = act_grad(acc[2 * mb + h][nb][j], acc[2 * mb + h][nb + NI / 2][j], acc2[2 * mb + h][nb][j]);
                        acc[2 * mb + h][nb][j] = v.h, acc[2 * mb + h][nb + NI / 2][j] = v.da, acc2[2 * mb + h][nb][j] = v.db;
                    }
            static_for<3>([&](auto what) INLINE {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int nb = 0; nb < NI / 2; ++nb) {
                        bf16x4 o;
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            o[j] = (bf16_t)(what == 0 ? acc[2 * mb + h][nb][j] : what == 1 ? acc[2 * mb + h][nb + NI / 2][j] : acc2[2 * mb + h][nb][j]);
                        *reinterpret_cast<bf16x4*>(wr + h * 16 * PITCH + nb * 32) = o;
                    }
                leave(rbk, static_cast<bf16_t*>(what == 0 ? g.h : what == 1 ? g.da : g.db) + at0);
            });
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int nb = 0; nb < NI; ++nb) {
                    bf16x4 o;
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[j] = (bf16_t)acc[2 * mb + h][nb][j];
                    *reinterpret_cast<bf16x4*>(wr + h * 16 * PITCH + nb * 32) = o;
                }
            bf16_t* const out = static_cast<bf16_t*>(!WGT ? g.gx : which == 0 ? g.gw_gate : which == 1 ? g.gw_up : g.gw_down);
            leave(rbk, out + (WGT ? (size_t)e * g.d * g.F : 0) + at0);
        }
    }
}

// ---- gradients of weights from few rows -----------------------------------------------------------------------
// A tile of few k-steps is mostly its beginning and its end: of 256 x 256 ones, alone on a CU, each took 10 us beside its steps.  Here two
// workgroups share a CU, one's stores beside the other's products: tiles of 128 x 256 on four waves, k-steps of 32 rows, three of them in
// LDS, one barrier a step.  A and B lie as in grad_kernel (A's rows of 256 bytes).
constexpr int kWgtM = 128, kWgtN = 256, kWgtK = 32, kWgtStages = 3;
constexpr int kWgtA = kWgtM * kWgtK * 2, kWgtStage = (kWgtM + kWgtN) * kWgtK * 2, kWgtLds = kWgtStages * kWgtStage;

__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void grad_weights_small_kernel(const GradArgs g) {
    extern __shared__ __align__(16) char smem[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    int lo, hi;
    group_bounds(g.offsets, g.E, g.P, lo, hi);
    lo = min(max(lo, 0), g.P), hi = min(max(hi, lo), g.P);
    // Strips of 256 hidden columns as in grad_kernel; for the gradients of W_gate and W_up a strip is two tiles high
    const int dt = 2 * ((g.d + 255) / 256), ft = (g.F + 255) / 256, slot = blockIdx.x >> 3;
    const int strip = uniform_div(slot, dt) * 8 + (blockIdx.x & 7), across = slot - uniform_div(slot, dt) * dt;
    const int rank = uniform_div(strip, 3 * ft), in = strip - rank * 3 * ft;
    if (rank >= g.E) return;
    const int e = MOE_READLANE(by_size(hi - lo, g.E), rank);
    const int which = uniform_div(in, ft), hidden = in - which * ft;
    bf16_t* const out = static_cast<bf16_t*>(which == 0 ? g.gw_gate : which == 1 ? g.gw_up : g.gw_down);
    const int M = which == 2 ? g.d : g.F, N = which == 2 ? g.F : g.d;
    const int m0 = which == 2 ? across * kWgtM : hidden * 256 + (across & 1) * kWgtM, n0 = which == 2 ? hidden * kWgtN : (across >> 1) * kWgtN;
    if (!out || m0 >= M || n0 >= N) return;
    const int first = MOE_READLANE(lo, e), K = MOE_READLANE(hi, e) - first, nk = (K + kWgtK - 1) / kWgtK;
    const unsigned pitch_a = (unsigned)M * 2, pitch_b = (unsigned)N * 2;
    const char* const A = static_cast<const char*>(which == 0 ? g.da : which == 1 ? g.db : g.gy) + (size_t)first * pitch_a;
    const char* const B = static_cast<const char*>(which == 2 ? g.h : g.x) + (size_t)first * pitch_b;

    // fills of a step: A by KB 4 p + wave, p < 2 (row 4 (4 p + wave) + l / 16), B by KB 4 p + wave, p < 4 (row 2 (4 p + wave) + l / 32)
    const unsigned lds0 = (unsigned)(uintptr_t)(lds_char*)smem;
    const int a_row = 4 * wave + (lane >> 4), b_row = 2 * wave + (lane >> 5);
    const int a_f = (lane >> 4) | (wave >> 1) << 2;
    const unsigned a_col = (unsigned)min(m0 + ((lane & 15) ^ (a_f << 1)) * 8, M - 8) * 2;
    const int b_chunk = (lane & 31) ^ ((b_row & 3) << 1);
    unsigned b_col[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) b_col[p] = (unsigned)min(n0 + (b_chunk ^ (p << 3)) * 8, N - 8) * 2;
    auto fill = [&](int v, auto last) INLINE {
        const int k0 = v * kWgtK, left = K - 1 - k0;  // (the last step: rows past the end are the last one again)
        const unsigned at = lds0 + v % kWgtStages * kWgtStage + wave * 1024;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int r = decltype(last)::value ? min(a_row + 16 * p, left) : a_row + 16 * p;
            dma16<false>(at + p * 4096, A + (size_t)(unsigned)k0 * pitch_a, (unsigned)r * pitch_a + a_col);
        }
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const int r = decltype(last)::value ? min(b_row + 8 * p, left) : b_row + 8 * p;
            dma16<false>(at + kWgtA + p * 4096, B + (size_t)(unsigned)k0 * pitch_b, (unsigned)r * pitch_b + b_col[p & 1]);
        }
    };
    auto fill_any = [&](int v) INLINE {
        if (v == nk - 1) fill(v, std::true_type{});
        else fill(v, std::false_type{});
    };
    f32x4 acc[4][8];
#pragma unroll
    for (int mi = 0; mi < 4; ++mi)
#pragma unroll
        for (int ni = 0; ni < 8; ++ni) acc[mi][ni] = f32x4{0.f, 0.f, 0.f, 0.f};
    const unsigned t_row = 8 * (lane >> 4) + ((lane & 15) >> 2), t_byte = (lane & 3) * 8;
    const unsigned swz = (((lane & 15) >> 2) | ((lane >> 4) & 1) << 2) << 5;
    if (nk > 0) fill_any(0);
    if (nk > 1) fill_any(1);
    for (int v = 0; v < nk; ++v) {
        if (v + 1 < nk) wait_vm<6>();  // step v has landed
        else wait_vm<0>();
        phase_end();                   // and that before it has been read
        if (v + 2 < nk) fill_any(v + 2);
        const unsigned pa = lds0 + v % kWgtStages * kWgtStage + t_row * 256 + t_byte, pb = lds0 + v % kWgtStages * kWgtStage + kWgtA + t_row * 512 + t_byte;
        bf16x8 fa[4], fb[8];
#pragma unroll
        for (int mi = 0; mi < 4; ++mi) fa[mi] = read_transposed(pa + (((unsigned)(wm * 4 + mi) << 5) ^ swz), 4 * 256);
#pragma unroll
        for (int ni = 0; ni < 8; ++ni) fb[ni] = read_transposed(pb + (((unsigned)(wn * 8 + ni) << 5) ^ swz), 4 * 512);
        if (v == nk - 1 && K % kWgtK) {
#pragma unroll
            for (int mi = 0; mi < 4; ++mi) fa[mi] = first_of(fa[mi], (lane >> 4) * 8, K - v * kWgtK);
        }
#pragma unroll
        for (int ni = 0; ni < 8; ++ni)
#pragma unroll
            for (int mi = 0; mi < 4; ++mi) acc[mi][ni] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[ni], fa[mi], acc[mi][ni], 0, 0, 0);
    }
    phase_end();
    // 16 rows at a time through LDS, a region per wave, so that the tile leaves in 16-byte stores: row l % 16, columns 4 (l / 16) .. + 4 of a block
    constexpr int PITCH = 128 * 2 + 16;
    char* const region = smem + wave * (16 * PITCH);
    bf16_t* const to = out + (size_t)e * g.d * g.F + (size_t)m0 * N + n0;
#pragma unroll
    for (int mi = 0; mi < 4; ++mi) {
#pragma unroll
        for (int ni = 0; ni < 8; ++ni) {
            bf16x4 o;
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = (bf16_t)acc[mi][ni][j];
            *reinterpret_cast<bf16x4*>(region + (lane & 15) * PITCH + ni * 32 + (lane >> 4) * 8) = o;
        }
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            const int r = it * 4 + (lane >> 4), row = wm * 64 + mi * 16 + r, c = wn * 128 + (lane & 15) * 8;
            const uint4 v = *reinterpret_cast<const uint4*>(region + r * PITCH + (lane & 15) * 16);
            if (m0 + row < M && n0 + c < N) store_past(to + (size_t)row * N + c, v);
        }
    }
}

template <int OP, int BM, int COLS, bool PARTS>
int launch(const GradArgs& g, int grid, hipStream_t st) {
    static std::atomic<uint64_t> lds_allowed;
    constexpr int lds = Form<OP, BM, COLS>::LDS;
    const auto kern = grad_kernel<OP, BM, COLS, PARTS>;
    if (allow_dynamic_lds(reinterpret_cast<const void*>(kern), lds, lds_allowed) != MOE_OK) return MOE_ERR_LAUNCH;
    hipLaunchKernelGGL(kern, dim3(grid), dim3(kThreads), lds, st, g);
    return launch_status();
}

}  // namespace

// A pass has as many k-steps as are fetched ahead of the first.  (Offsets within a tile, of 256 rows of at most 2^18 values, are 32 bits.)
bool grad_mfma_supported(const GradArgs& g) { return g.d > 2 * BK && g.F > 2 * BK; }

// gx = the sum of its parts, in order, rounded once; rows of no group stay as they are
__global__ __launch_bounds__(256) void sum_grad_parts_kernel(const float* __restrict__ parts, int q, const int32_t* __restrict__ offsets, int E, int P, int d,
                                                             bf16_t* __restrict__ gx) {
    const long long n = (long long)min(max(offsets[E], 0), P) * d, all = (long long)P * d;
    for (long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * 8; i < n; i += (long long)gridDim.x * (256 * 8)) {
        f32x4 lo{}, hi{};
        for (int p = 0; p < q; ++p) {
            lo += *reinterpret_cast<const f32x4*>(parts + p * all + i);
            hi += *reinterpret_cast<const f32x4*>(parts + p * all + i + 4);
        }
        bf16x8 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = (bf16_t)lo[j], o[4 + j] = (bf16_t)hi[j];
        *reinterpret_cast<bf16x8*>(gx + i) = o;
    }
}

int run_grad_mfma(const GradArgs& g, GradOp op, hipStream_t st) {
    const GradPlan plan = grad_plan(g.P, g.E, g.d, g.F);
    if (op == GRAD_WEIGHTS) {
        const int strips = (g.E * 3 * ((g.F + 255) / 256) + 7) / 8 * 8, across = (g.d + 255) / 256;
        if (!plan.small_weights) return launch<GRAD_WEIGHTS, 256, 256, false>(g, strips * across, st);
        static std::atomic<uint64_t> lds_allowed;
        if (allow_dynamic_lds(reinterpret_cast<const void*>(grad_weights_small_kernel), kWgtLds, lds_allowed) != MOE_OK) return MOE_ERR_LAUNCH;
        hipLaunchKernelGGL(grad_weights_small_kernel, dim3(strips * across * 2), dim3(256), kWgtLds, st, g);
        return launch_status();
    }
    if (op == GRAD_ACT) {
        const int grid = find_tile_grid(m_tiles_bound(g.P, g.E, plan.act_rows) * ((g.F + plan.act_cols - 1) / plan.act_cols), kSplitSlots);
        return plan.act_rows == 128   ? launch<GRAD_ACT, 128, 128, false>(g, grid, st)
               : plan.act_cols == 128 ? launch<GRAD_ACT, 256, 128, false>(g, grid, st)
                                      : launch<GRAD_ACT, 256, 96, false>(g, grid, st);
    }
    const int grid = find_tile_grid(m_tiles_bound(g.P, g.E, 256) * ((g.d + 255) / 256) * plan.dx_parts, kSplitSlots);
    if (plan.dx_parts == 1) return launch<GRAD_DX, 256, 256, false>(g, grid, st);
    GradArgs cut = g;
    cut.k_parts = plan.dx_parts;
    const int rc = launch<GRAD_DX, 256, 256, true>(cut, grid, st);
    if (rc != MOE_OK) return rc;
    const long long chunks = (long long)g.P * g.d / 8;
    hipLaunchKernelGGL(sum_grad_parts_kernel, dim3((unsigned)std::min<long long>((chunks + 255) / 256, 2048)), dim3(256), 0, st, g.parts, cut.k_parts,
                       g.offsets, g.E, g.P, g.d, static_cast<bf16_t*>(g.gx));
    return launch_status();
}

}  // namespace moe
