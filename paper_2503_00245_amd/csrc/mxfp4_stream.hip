// Grouped products in microscaled 4-bit floating point for some rows an expert: the weights are most of what there is to
// move.  A workgroup makes 32 output columns (with SWIGLU the same of gate and of up) of 32 rows of an expert; its waves
// cut K and meet in LDS once.  Operands come straight from memory into registers, in runs of 1 KB a request.
#include <algorithm>

#include "gemm.h"
#include "mxfp4.h"

namespace moe {

namespace {

constexpr int kWaves = 4;

// ONCE: most experts have one group of rows, and the weights need not stay in the caches (2048 / 5632, 32 tokens 45.1 -> 42.3 us a layer, 1024 / 2816, 24 tokens 28.6 -> 27.3)
template <bool SWIGLU, bool ONCE>
__global__ __launch_bounds__(kWaves* kWave) void mx_stream_kernel(ptr_arg a_starts, ptr_arg a_w0, ptr_arg a_w1, ptr_arg a_rows, int E, int N, int K, int all_blocks,
                                                                  ptr_arg a_out) {
    constexpr int M = SWIGLU ? 2 : 1, NT = 2;  // matrices, tiles of 16 rows
    __shared__ f32x4 s_part[kWaves][M * 2 * NT][kWave];
    const int32_t* const starts = from_arg<const int32_t>(a_starts);
    const char* const w_of[2] = {from_arg<const char>(a_w0), from_arg<const char>(a_w1)};
    const char* const rows = from_arg<const char>(a_rows);
    char* const out = from_arg<char>(a_out);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int fb = blockIdx.x, fbs = mx_blocks(N), units = mx_units(K), out_units = mx_units(N);
    const int sb = blockIdx.y;
    const int end = lane < E ? starts[lane + 1] : 0x7fffffff;
    const unsigned long long at_e = __ballot(lane < E && sb < end);
    if (!at_e) return;
    const int e = __ffsll((long long)at_e) - 1;

    f32x4 acc[M][2][NT];
#pragma unroll
    for (int i = 0; i < M * 2 * NT; ++i) acc[i / (2 * NT)][i / NT % 2][i % NT] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int u_begin = units * wave / kWaves, u_end = fb < fbs ? units * (wave + 1) / kWaves : u_begin;
    const size_t at = ((size_t)e * fbs + fb) * units, scales = (size_t)E * fbs * units * kMxCodes;
    const char* const row_scales = rows + (size_t)all_blocks * units * kMxCodes;
    for (int u = u_begin; u < u_end; ++u) {
        i32x4 fa[M][2][2], fx[2][2];
        int sa[M];
#pragma unroll
        for (int m = 0; m < M; ++m) {
#pragma unroll
            for (int ct = 0; ct < 4; ++ct) {
                const i32x4* p = reinterpret_cast<const i32x4*>(w_of[m] + (at + u) * kMxCodes + ct * 1024 + lane * 16);
                fa[m][ct / 2][ct % 2] = ONCE ? __builtin_nontemporal_load(p) : *p;
            }
            sa[m] = *reinterpret_cast<const int*>(w_of[m] + scales + (at + u) * kMxScales + lane * 4);
        }
        const size_t row_at = (size_t)sb * units + u;
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) fx[ct / 2][ct % 2] = *reinterpret_cast<const i32x4*>(rows + row_at * kMxCodes + ct * 1024 + lane * 16);
        const int sx = *reinterpret_cast<const int*>(row_scales + row_at * kMxScales + lane * 4);
#pragma unroll
        for (int m = 0; m < M; ++m) mx_unit(acc[m], fa[m], fx, sa[m], sx);
    }
#pragma unroll
    for (int i = 0; i < M * 2 * NT; ++i) s_part[wave][i][lane] = acc[i / (2 * NT)][i / NT % 2][i % NT];
    __syncthreads();
    // a tile of 16 rows a wave
    if (wave < NT) {
        const int n = wave;
        f32x4 sum[M][2];
#pragma unroll
        for (int i = 0; i < M * 2; ++i) {
            f32x4 v = s_part[0][i * NT + n][lane];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) {
                const f32x4 o = s_part[w][i * NT + n][lane];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] += o[j];
            }
            sum[i / 2][i % 2] = v;
        }
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = SWIGLU ? silu_f32(sum[0][j / 4][j % 4]) * sum[M - 1][j / 4][j % 4] : sum[0][j / 4][j % 4];
        if constexpr (SWIGLU) mx_store_hidden(f, out, out + (size_t)all_blocks * out_units * kMxCodes, out_units, sb, n, fb, lane);
        else mx_store_rows(f, out, N, sb, n, fb, lane);
    }
}

}  // namespace

int launch_mx_stream(bool swiglu, const void* w0, const void* w1, const char* a, char* out, const int32_t* starts, int P, int E,
                     int all_blocks, int N, int K, hipStream_t st) {
    const dim3 grid(swiglu ? mx_units(N) * (kMxUnit / 32) : mx_blocks(N), m_tiles_bound(P, E, 32));
    auto launch = [&](auto kern) {
        hipLaunchKernelGGL(kern, grid, dim3(kWaves * kWave), 0, st, as_arg(starts), as_arg(w0), as_arg(w1), as_arg(a), E, N, K, all_blocks, as_arg(out));
        return launch_status();
    };
    auto launch_of = [&](auto once) {
        constexpr bool O = decltype(once)::value;
        return swiglu ? launch(mx_stream_kernel<true, O>) : launch(mx_stream_kernel<false, O>);
    };
    return P <= 32 * E ? launch_of(std::true_type{}) : launch_of(std::false_type{});
}

}  // namespace moe
