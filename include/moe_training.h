/*
 * moe_training.h - C ABI of a training step around and through the experts: tokens to the experts' rows and back
 * with their gradients, the gradient of the experts, and the block that stands around such a layer (norms before and
 * after it, gates, dropout, scaled residual) with its gradient.
 *
 * The conventions of moe.h hold here too: device pointers into the caller's memory, calls enqueued on
 * `stream` without synchronising, statuses found on the host before any launch, nothing allocated or kept,
 * the same bits for the same inputs.  Arrays of int32 and fp32 need 4-byte alignment only, but for post_w, gate and open_w below
 * (16 bytes).  No output may overlap an
 * input or another output unless it is said.  Calls may be captured into graphs.  Non-finite inputs give unspecified results (an
 * infinite one may be NaN), but what is said to play no part, or not to be read, may hold anything.
 */
#ifndef MOE_TRAINING_H_
#define MOE_TRAINING_H_

#include "moe.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * ---- Tokens to rows sorted by expert, and back ------------------------------------------------------
 *
 * Pair p = t k + j is token t's j-th pick.  As in moe_permute, rows are grouped by expert, and within a group pairs
 * stand in ascending order.  A pick outside [0, E) is switched off (the padding of a batch, a token that is not to be
 * trained on): its pair has no row.  Of the P = T k rows the last P - expert_offsets[E] then belong to no pair.
 * Of the shape d_model, n_tokens, n_experts, top_k and act_dtype are read (d_ff has to be valid).
 */

/* Bytes of workspace that moe_dispatch needs for this shape, whatever its experts (0 if invalid).  Does not fall as n_tokens grows. */
MOE_API size_t moe_dispatch_workspace_bytes(const moe_shape* shape);

/* Bytes of workspace that moe_expert_ffn_backward needs for this shape, and as many as moe_dispatch needs; 0 if moe_expert_ffn_backward
 * refuses the shape (see there).  As far as it takes them, does not fall as n_tokens grows. */
MOE_API size_t moe_training_workspace_bytes(const moe_shape* shape);

/*
 *   topk_idx       [T, k] int32 in
 *   weight         [T, k] fp32 in, or NULL (ones)
 *   x              [T, d] act_dtype in
 *   expert_offsets [E+1]  int32 out: group e is rows [offsets[e], offsets[e+1])
 *   perm           [P]    int32 out: the pair of each row, -1 from offsets[E] on
 *   inv_perm       [P]    int32 out: the row of each pair, -1 if it is switched off
 *   x_perm         [P, d] act_dtype out: x_perm[s] = weight[perm[s]] x[perm[s] / k]; zeros from offsets[E] on
 * workspace: moe_dispatch_workspace_bytes(shape), 4-byte aligned; up to 8192 pairs it is not needed (NULL will do).
 */
MOE_API int moe_dispatch(const moe_shape* shape, const int32_t* topk_idx, const float* weight, const void* x,
                         int32_t* expert_offsets, int32_t* perm, int32_t* inv_perm, void* x_perm,
                         void* workspace, size_t workspace_bytes, void* stream);

/*
 * Its gradient: grad_x[t] = sum_j weight[t,j] grad_x_perm[inv_perm[t,j]], summed in fp32 in ascending j and
 * rounded once, and grad_weight[t,j] = <x[t], grad_x_perm[inv_perm[t,j]]>, 0 for a pair without a row.  Values of
 * inv_perm outside [0, P) are pairs without a row.  grad_weight may be NULL; x is read only for it (else NULL will do).
 */
MOE_API int moe_dispatch_backward(const moe_shape* shape, const void* grad_x_perm, const int32_t* inv_perm,
                                  const void* x, const float* weight, void* grad_x, float* grad_weight,
                                  void* stream);

/*
 * y[t] = sum_j topk_gate[t,j] y_perm[inv_perm[t,j]] (+ residual[t]): moe_combine for pairs of which some have no row
 * (values of inv_perm outside [0, P)).  What stands in rows of no pair, and the gates of pairs without a row, play no part.
 */
MOE_API int moe_collect(const moe_shape* shape, const void* y_perm, const int32_t* inv_perm,
                        const float* topk_gate, const void* residual, void* y, void* stream);

/*
 * Its gradient (and moe_combine's): grad_y_perm[inv_perm[t,j]] = topk_gate[t,j] grad_y[t], rounded once, zeros from
 * expert_offsets[E] on; grad_gate[t,j] = <grad_y[t], y_perm[inv_perm[t,j]]>, 0 for a pair without a row.  The
 * residual's gradient is grad_y itself.  Either output may be NULL; y_perm is read only for grad_gate (else NULL will do),
 * topk_gate and expert_offsets only for grad_y_perm.  grad_y_perm may be y_perm itself: its rows are read first.
 */
MOE_API int moe_collect_backward(const moe_shape* shape, const void* grad_y, const void* y_perm,
                                 const int32_t* expert_offsets, const int32_t* inv_perm, const float* topk_gate,
                                 void* grad_y_perm, float* grad_gate, void* stream);

/*
 * ---- Gradient of the experts ------------------------------------------------------------------------
 *
 * Of moe_expert_ffn with rank 0: for every row v of expert e's group, with g its row of grad_y_perm,
 *   a = W_gate v, b = W_up v, h = silu(a) b                                 (formed again, not kept by the forward pass)
 *   dh = W_down^T g,  db = dh silu(a),  da = dh b s (1 + a (1 - s)),  s = 1 / (1 + exp(-a))
 *   grad_x_perm = W_gate^T da + W_up^T db
 *   grad_w_gate = sum of da v^T,  grad_w_up = sum of db v^T,  grad_w_down = sum of g h^T  over the group's rows
 * Sums are formed in fp32.  With bf16 storage h, da and db are rounded to bf16, as the matrix units take them.  Experts
 * without rows get gradients of zero.  Rows from expert_offsets[E] on are neither read nor written.
 *   x_perm, grad_y_perm [P, d] act_dtype in; expert_offsets [E+1] in, ascending from 0, at most P
 *   weights: w_gate, w_up [E, F, d], w_down [E, d, F] (the other fields are not read)
 *   grad_x_perm [P, d]; grad_w_gate, grad_w_up [E, F, d], grad_w_down [E, d, F] act_dtype out, each of them or NULL
 * Of no tokens the gradients of weights are zero.  workspace: moe_training_workspace_bytes(shape), 16-byte aligned.
 * Unsupported are rank > 0, d or F over 2^18, and layers of more tiles than a launch has: d' F', (ceil(P / 64) + E) max(d', F') and
 * (3 E ceil(F / 256) + 8) 2 ceil(d / 256) have to be below 2^23, with d' = ceil(d / 64), F' = ceil(F / 64).
 */
MOE_API int moe_expert_ffn_backward(const moe_shape* shape, const moe_weights* weights, const void* x_perm,
                                    const int32_t* expert_offsets, const void* grad_y_perm, void* grad_x_perm,
                                    void* grad_w_gate, void* grad_w_up, void* grad_w_down, void* workspace,
                                    size_t workspace_bytes, void* stream);

/*
 * ---- The block around the layer ---------------------------------------------------------------------
 *
 * With N(v; w) = v w / sqrt(mean(v^2) + eps) over a row of d values and D dropout, the end of one block and the start of
 * the next:
 *   y[t] = skip_scale x[t] + block_scale token_gate[t] gate D(N(b[t]; post_w))
 *   n[t] = N(y[t]; open_w), of y as it is stored
 * post_w, gate, open_w [d], token_gate [T] fp32.  A NULL post_w leaves b unnormalised; a NULL gate, or token_gate, is ones.
 * Statistics and sums are held in fp32 (the mean of squares of a row passes its range from values of about 1e17 on: unspecified).
 *
 * Dropout keeps value i = t d + c with probability 1 - r / 65536, r = dropout 65536 to the nearest, and multiplies what it
 * keeps by 65536 / (65536 - r).  Value i is dropped if half i % 8 of Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random
 * numbers: as easy as 1, 2, 3) is below r, halves counted from the lower one of word 0, with the counter (i / 8, rng[1]), each 64
 * bits, lower half first, and the key rng[0].  The mask is never stored: the backward pass makes it again.  rng [2] uint64 lies on the
 * device, 8-byte aligned, so that a captured graph takes new numbers at every replay; it is read only where r > 0.  Nothing else enters
 * the mask: calls of the same numbers drop the same places, so layers and steps whose masks shall not depend on one another need
 * numbers of their own (another seed, or another offset).
 */
typedef struct moe_block {
    float eps;                 /* > 0, finite */
    float skip_scale;          /* finite      */
    float block_scale;         /* finite      */
    float dropout;             /* 0 <= dropout, r < 65536 */
    const float* post_w;
    const float* gate;
    const float* token_gate;
    const uint64_t* rng;
} moe_block;

#define MOE_BLOCK_MAX_D 32768

/*
 *   x, b [T, d] act_dtype in; y [T, d] out, may be x itself
 *   open_w and n [T, d] (out): both or neither NULL
 * Without b (NULL, y NULL) it is the start of a block alone: n[t] = N(x[t]; open_w).  d: a multiple of 8, at most
 * MOE_BLOCK_MAX_D; n_tokens < 2^24.
 */
MOE_API int moe_block_norm(const moe_block* block, int32_t n_tokens, int32_t d_model, int32_t act_dtype,
                           const void* x, const void* b, const float* open_w, void* y, void* n, void* stream);

/*
 * Its gradient.  grad_y, grad_n [T, d]: gradients of the two outputs, either NULL if it has none (grad_n goes with open_w:
 * both or neither NULL); y [T, d] as moe_block_norm left it, read only with grad_n; b as it was given.  With
 * G = grad_y + (gradient of N(y; open_w) for grad_n):
 *   grad_x = skip_scale G, grad_b [T, d] act_dtype out; grad_x may be grad_y itself
 *   grad_open_w, grad_post_w, grad_gate [d], grad_token_gate [T] fp32 out, each of them or NULL (grad_post_w only with a
 *   post_w, grad_open_w only with open_w; the gates' also where the gate itself is NULL: at ones)
 * Without b (NULL; y then stands for x): grad_x = G, and grad_b, grad_post_w, grad_gate and grad_token_gate are NULL.
 * Sums over tokens are formed in fp32 in an order that the sizes alone decide.  workspace:
 * moe_block_workspace_bytes(n_tokens, d_model), 16-byte aligned; it is not read where the three [d] outputs are NULL.
 */
MOE_API size_t moe_block_workspace_bytes(int32_t n_tokens, int32_t d_model); /* 0 if invalid */
MOE_API int moe_block_norm_backward(const moe_block* block, int32_t n_tokens, int32_t d_model, int32_t act_dtype,
                                    const void* grad_y, const void* grad_n, const void* y, const void* b,
                                    const float* open_w, void* grad_x, void* grad_b, float* grad_open_w,
                                    float* grad_post_w, float* grad_gate, float* grad_token_gate,
                                    void* workspace, size_t workspace_bytes, void* stream);

/*
 * Stack of n_layers such blocks around moe_forward's layer, the residual stream held in act_dtype:
 *   n_0 = N(x; open_w[0]);  b_l = layer_l(n_l);  x_{l+1}, n_{l+1} by blocks[l] and open_w[l+1] as above;  y = x_{n_layers}
 * the end of a block and the start of the next in one launch.  layers, blocks [n_layers] and open_w [n_layers] (of device pointers)
 * are host arrays; every open_w[l] is needed, and its eps is that of blocks[l] for l = 0 and of blocks[l - 1] after.  A
 * token_gate and an rng are those of their block: with one rng for all blocks every layer drops the same places.  topk_trace [n_layers, T, k] int32 or NULL.  shape.flags' residual bit is
 * refused.  workspace: moe_block_stack_workspace_bytes(shape), 16-byte aligned.
 */
MOE_API size_t moe_block_stack_workspace_bytes(const moe_shape* shape); /* 0 if invalid */
MOE_API int moe_block_stack_forward(const moe_shape* shape, const moe_weights* layers, const moe_block* blocks,
                                    const float* const* open_w, int32_t n_layers, const void* x, void* y,
                                    int32_t* topk_trace, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MOE_TRAINING_H_ */
