// Which tiles the bf16 products of the experts' gradient take, by sizes (internal; host only, so that a test can hold the tested sizes to
// every one of them).
#pragma once

#include <algorithm>
#include <cmath>
#include <cstddef>

namespace moe {

struct GradPlan {
    int act_rows, act_cols;  // tile of a, b and dh
    int dx_parts;            // runs that the k-steps of gx are cut into
    bool small_weights;      // gradients of weights by grad_weights_small_kernel
};

// Row tiles that a layer's groups are expected to need: beside whole ones about half a tile each, a little more as loads are uneven
inline double grad_row_tiles(int P, int E, int bm) {
    const double groups = std::min(P, E);
    return std::max(groups, (double)P / bm + 0.6 * groups);
}

// Room for gx in parts; does not fall as P grows
inline size_t grad_parts_bytes(long long P, int d) { return std::min<size_t>(16 * (size_t)P * d, 200u << 20); }

// The tiles of gx are few (rows by d, where the other products have F or F by d) and long (2 F deep).  Where they do not fill the CUs their k-steps are
// cut into up to four runs, summed by a launch of its own in fp32.  A model of the launch in us decides: rounds of 256 workgroups (the last
// one of halves where that does), 1.15 us a step of full tiles, 0.8 of near empty ones, 8 us beside the steps, and the sums at 4.5 TB/s.
// (gx in one part / in two / three / four, us with the sums, parts taken: 24 tokens of 1024 / 2816, 4 of 16 experts, 63 / 40 / 37 / 36, four; 64 of 2048 / 5632 135 / 84 / 68 /
// 66, four; 300 of 1024 / 2816 88 / 59 / 46 / 39, four; 777 of 1440 / 3840 138 / 90 / 70 / 84, three; 4096 of 432 / 1152 45 / 40 / 36 / 47, three; 2048 of 2048 / 5632
// 220 / 237 / 217 / 225, three; 2048 of 1024 / 2816, 4 of 64 experts, 141 / 179 / 199 / 217 and 8192, 2 of 32, 209 / 244 / 270 / 273, one.  Loads as trained
// routers' but for the 24 and the 4 of 64.  The model's constants are older than stores of the weights' gradients past the caches, which made the weights
// read here cheaper; no other number of parts than those taken is faster at these sizes.)
inline int grad_dx_parts(int P, int E, int d, int F) {
    const double groups = std::min(P, E), tiles = grad_row_tiles(P, E, 256) * ((d + 255) / 256);
    const double step = std::max(0.8, 1.15 * std::min(1.0, P / groups / 192));
    const int steps = 2 * ((F + 63) / 64), most = (int)std::min<size_t>(4, grad_parts_bytes(P, d) / (4 * (size_t)P * d));
    int best = 1;
    double best_cost = 0;
    for (int q = 1; q <= most && steps / q >= 8; ++q) {
        double rounds = tiles * q / 256;
        rounds = rounds <= 1 ? 1 : std::ceil(2 * rounds) / 2;
        const double cost = rounds * (steps / q * step + 8) + (q > 1 ? 6 + 4.0 * q * P * d / 4.5e6 : 0);
        if (q == 1 || cost < best_cost) best = q, best_cost = cost;
    }
    return best;
}

inline GradPlan grad_plan(int P, int E, int d, int F) {
    GradPlan p{256, 96, grad_dx_parts(P, E, d, F), false};
    // a, b, dh: 256 rows by 128 columns take 1.21 times as long as by 96, 128 rows by 128 0.72 times; whole rounds of 256 workgroups decide, and near
    // empty tiles are bound by the weights (us, 256 x 96 / 256 x 128 / 128 x 128: 24 tokens of 1024 / 2816, 4 of 16 experts, 57 / 71 / 58, 777 of
    // 1440 / 3840 130 / 136 / 107, 2048 of 2048 / 5632 336 / 329 / 348, 16384 2443 / 2128 / 2389; 300 of 1024 / 2816 42 / 48 / 31, 512, 6 of 64 experts, 294 / 307 / 244; 4096
    // of 432 / 1152 48 / 58 / 52.  It is wrong by 6 and 10 % where 128 rows are taken at 8192 of 1024 / 2816, 2 of 32 experts, 376 / 353 / 375, and 5000 of 1600 / 4264, 1 of 8,
    // 262 / 256 / 281.)  Of 128 rows four k-steps are fetched ahead.
    auto cost = [&](int bm, int cols, double tile) { return tile * std::ceil(grad_row_tiles(P, E, bm) * ((F + cols - 1) / cols) / 256); };
    const double wide = cost(256, 128, 1.21), narrow = cost(256, 96, 1.0), low = cost(128, 128, 0.72);
    if (low < wide && low < narrow && P > 32ll * E && d > 192) p.act_rows = p.act_cols = 128;
    else if (wide < narrow) p.act_cols = 128;
    // Gradients of weights: 256 x 256 / 128 x 256 tiles, us: 24 tokens of 1024 / 2816, 4 of 16 experts, 75 / 52, 300 40 / 35-38 (2 of 8), 777 of 1440 / 3840 105 / 90, 2048 of
    // 1024 / 2816, 4 of 64, 390-416 / 382-406, 1000 of 720 / 1920, 2 of 4, 36 / 36; 2048 of 2048 / 5632 331 / 365, 4096 of 432 / 1152 58 / 66, 8192 of 1024 / 2816, 2 of 32, 345 / 386, 16384 of
    // 2048 / 5632 1742 / 2174
    p.small_weights = P < 384ll * E;
    return p;
}

}  // namespace moe
