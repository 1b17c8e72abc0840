// Host only: which kernels the two products of a layer take.  Arguments: tokens x picks, experts, d_model, d_ff, then the pairs of every expert; prints the rows
// of a tile of gate/up and of down (32: streamed), and for each whether its last round of tiles is cut into halves.
#include <cstdio>
#include <cstdlib>

#include "gemm.h"
#include "mxfp4_plan.h"

using namespace moe;

static bool halves(bool swiglu, int rows, int E, char** loads, int N) {
    if (rows == 32) return false;
    int tiles = 0;
    for (int e = 0; e < E; ++e) tiles += (mx_blocks(atoi(loads[e])) * 32 + rows - 1) / rows;
    tiles *= mx_column_tiles(swiglu, N);
    bool any = false;
    for (int b = 0; b < find_tile_grid(tiles, kMxSplitSlots); ++b) {
        int tile, half;
        if (tile_of_block<kMxSplitSlots>(b, tiles, tile, half)) any |= half >= 0;
    }
    return any;
}

int main(int argc, char** argv) {
    if (argc < 5) return 1;
    const int P = atoi(argv[1]), E = atoi(argv[2]), d = atoi(argv[3]), F = atoi(argv[4]);
    if (argc != 5 + E) return 1;
    const int hidden = mx_tile_rows(true, P, E, F, d), down = mx_tile_rows(false, P, E, d, F);
    printf("%d %d %d %d\n", hidden, down, (int)halves(true, hidden, E, argv + 5, F), (int)halves(false, down, E, argv + 5, d));
    return 0;
}
