// Host only: which forms the kernels between tokens and experts' rows take.  Arguments: tokens, d_model, experts, picks; prints the waves and pairs of rows_form, how
// pairs are counted (0 by ballots, 1 by additions, 2 in a launch of its own), the pairs of a chunk and the number of chunks.
#include <cstdio>
#include <cstdlib>

#include "rows_plan.h"

int main(int argc, char** argv) {
    if (argc != 5) return 1;
    const int T = atoi(argv[1]), d = atoi(argv[2]), E = atoi(argv[3]), k = atoi(argv[4]);
    const moe::RowsForm f = moe::rows_form(d, k);
    const moe::DispatchPlan p = moe::dispatch_plan(T, E);
    printf("%d %d %d %d %d\n", f.waves, f.pairs, (int)moe::dispatch_count((long long)T * k, E), p.tokens * k, p.chunks);
    return 0;
}
