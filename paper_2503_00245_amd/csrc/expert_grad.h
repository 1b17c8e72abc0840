// What the kernels of the experts' gradient share (internal).
#pragma once

#include "gemm.h"
#include "moe_training.h"

namespace moe {

// The products of a call, all over the rows that offsets groups (x, gy, da, db, h: [P, .]):
//   ACT      a = x W_gate^T, b = x W_up^T, dh = gy W_down, and from them h, da, db       K = d, N = F
//   DX       gx = da W_gate + db W_up            K = F twice, N = d
//   WEIGHTS  da^T x, db^T x [F, d], gy^T h [d, F]: K = the group's rows
enum GradOp { GRAD_ACT, GRAD_DX, GRAD_WEIGHTS };

struct GradArgs {
    const void *x, *gy;
    const void *w_gate, *w_up, *w_down;
    void *da, *db, *h;  // [P, F]
    void *gx, *gw_gate, *gw_up, *gw_down;
    const int32_t* offsets;
    int P, E, d, F;
    int k_parts;      // DX in expert_grad_mfma.hip: fp32 outputs [P, d] that the k-steps are cut into, in parts
    float* parts;
};

// h and the gradients of a and b, from a, b and the gradient of h, in fp32
struct ActGrad {
    float h, da, db;
};
__device__ __forceinline__ ActGrad act_grad(float a, float b, float dh) {
#if defined(__HIP_DEVICE_COMPILE__)
    const float s = __builtin_amdgcn_rcpf(1.0f + __expf(-a));
#else
    const float s = 1.0f / (1.0f + __expf(-a));
#endif
    const float act = a * s;
    return ActGrad{act * b, dh * b * (s + act * (1.0f - s)), dh * act};
}

// any type and size (expert_grad.hip)
int run_grad_plain(const GradArgs& g, GradOp op, int act_dtype, hipStream_t st);

// bf16 (expert_grad_mfma.hip)
bool grad_mfma_supported(const GradArgs& g);
int run_grad_mfma(const GradArgs& g, GradOp op, hipStream_t st);

}  // namespace moe
