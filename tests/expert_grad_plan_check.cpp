// Host only: which tiles the products of the experts' gradient take.  Arguments: pairs, experts, d_model, d_ff; prints rows and columns of a tile of the
// activation's gradient, the parts of the rows' gradient, and whether the weights' gradients take the smaller tiles.
#include <cstdio>
#include <cstdlib>

#include "expert_grad_plan.h"

int main(int argc, char** argv) {
    if (argc != 5) return 1;
    const moe::GradPlan p = moe::grad_plan(atoi(argv[1]), atoi(argv[2]), atoi(argv[3]), atoi(argv[4]));
    printf("%d %d %d %d\n", p.act_rows, p.act_cols, p.dx_parts, (int)p.small_weights);
    return 0;
}
