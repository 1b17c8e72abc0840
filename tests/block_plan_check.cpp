// Host only: how rows of the block are dealt out.  Arguments: rows, d_model; prints the waves that share a row, their chunks, the workgroups that have a row,
// the most of the forward pass and the most of a gradient with sums over rows.
#include <cstdio>
#include <cstdlib>

#include "block_plan.h"

int main(int argc, char** argv) {
    if (argc != 3) return 1;
    const int T = atoi(argv[1]), d = atoi(argv[2]);
    const moe::RowPlan p = moe::row_plan(d);
    printf("%d %d %d %d %d\n", p.waves, p.chunks, moe::row_groups(T, d), moe::kGroups, moe::most_grad_groups(d));
    return 0;
}
