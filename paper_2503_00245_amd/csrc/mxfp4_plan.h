// Which kernel a product of experts on MXFP4 weights takes, and how its launch is cut: host arithmetic (internal).
#pragma once

#include <algorithm>
#include <cmath>

#include "gemm.h"
#include "mxfp4.h"

namespace moe {

constexpr int kMxSplitSlots = 32;  // mxfp4_gemm.hip: one workgroup per CU
// Columns of a tile of that file, in blocks of 32 (with SWIGLU half of its 256 rows of weights are gate's, half up's), and tiles across N
constexpr int mx_tile_blocks(bool swiglu) { return swiglu ? 4 : 8; }
__host__ __device__ constexpr int mx_column_tiles(bool swiglu, int N) {
    // (SWIGLU: whole units of output columns, so that what pads the next product's K is written too)
    return ((swiglu ? mx_units(N) * (kMxUnit / 32) : mx_blocks(N)) + mx_tile_blocks(swiglu) - 1) / mx_tile_blocks(swiglu);
}
// Tiles of so many rows that such a product can need, and whether that many workgroups of 512 threads are a launch: fewer than 2^32 work items
inline long long mx_tiles(bool swiglu, int P, int E, int N, int rows) { return (long long)m_tiles_bound(P, E, rows) * mx_column_tiles(swiglu, N); }
inline bool mx_tiles_fit(bool swiglu, int P, int E, int N, int rows) { return mx_tiles(swiglu, P, E, N, rows) + 8 * kMxSplitSlots < 1 << 23; }

// Rows of a tile of a product of P rows in E groups: 32 (mxfp4_stream.hip), 64, 128 or 256 (mxfp4_gemm.hip), whichever is the shortest by what
// they measured, in us.  Tiles: rounds of 256 workgroups, a round so much a tile and so much a unit of K.  Streamed: so much of a CU for 32 rows of
// weights by 32.  In no case less than the weights at 4.6 TB/s.  How unevenly the rows are spread the host does not know: half a tile more
// an expert.  Whole layers, us, weights cold, this choice / the best of the sixteen pairs of choices: 2048 / 5632, 2 of 8 experts, 64 tokens 46.0 / 41.9,
// 200 tokens 52.9 / 52.5, 400 63.2 / 63.2, 800 76.7 / 73.1, 1200 95.7 / 95.7, 2048 136.3 / 135.9, 4096 225.3 / 223.7; 1024 / 2816, 256 tokens 24.5 / 24.2, 2048
// 58.9 / 58.9, 4 of 16 experts, 24 tokens 27.1 / 27.0, 4 of 32 experts, 2048 tokens 111.9 / 104.7; 1440 / 3840, 777 tokens 53.0 / 52.9; 432 / 1152, 300 tokens 15.1 / 15.1.
inline int mx_tile_rows(bool swiglu, int P, int E, int N, int K) {
    const double rows = (double)P / E, units = mx_units(K), weights_mb = 0.53e-6 * N * (double)K * (swiglu ? 2 : 1) * std::min(P, E);
    auto groups = [&](int of) { return std::min((double)P, E * std::max(1.0, rows / of + 0.5)); };
    double best = std::max(mx_blocks(N) * groups(32) / 256 * (0.35 + units * (swiglu ? 0.11 : 0.09)), weights_mb / 4.6) + 3.0;
    if (groups(32) + E > 65535) best = 1e30;  // (more than the grid's second dimension has)
    int choice = 32;
    struct {
        int rows;
        double tile, unit;
    } const tiles[] = {{64, swiglu ? 3.8 : 4.9, 0.55}, {128, 4.8, 0.85}, {256, swiglu ? 6.0 : 5.0, 1.52}};
    for (const auto& t : tiles) {
        if (!mx_tiles_fit(swiglu, P, E, N, t.rows)) continue;  // (those of 256 rows do: validate_mx)
        const double rounds = std::ceil(groups(t.rows) * ((N + (swiglu ? 127 : 255)) / (swiglu ? 128 : 256)) / 256);
        const double us = std::max(rounds * (t.tile + units * t.unit), weights_mb / 4.6) + 2.5;
        if (us < best) best = us, choice = t.rows;
    }
    return choice;
}

}  // namespace moe
