/*
 * moe_quantised.h - C ABI of routing from logits and of experts in microscaled 4-bit floating point.
 *
 * The conventions of moe.h hold here too: device pointers into the caller's memory, calls enqueued on
 * `stream` without synchronising, statuses found on the host before any launch, nothing allocated or kept,
 * the same bits for the same inputs.
 */
#ifndef MOE_QUANTISED_H_
#define MOE_QUANTISED_H_

#include "moe.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * ---- Routing from logits, as routers of many experts have it ---------------------------------
 *
 * Scores s = softmax(l) (Sec. 2.3, Eq. 2) or, element by element, 1 / (1 + exp(-l)).  Experts are
 * picked by key c = s + select_bias (the bias balances loads; it does not enter the gates).  With
 * n_groups > 1 the E experts are n_groups runs of E / n_groups neighbours; a group's rank is the sum
 * of its group_top (1 or 2) largest keys, and only experts of the groups_kept highest groups are
 * eligible.  The k largest keys are picked in descending order.  Every tie, of experts and of
 * groups, goes to the lower index.  Gates: scale * s_S / sum_j s_S(j) if renormalize, else scale * s_S.
 * A logit of minus infinity (or NaN) switches its expert off: score 0, key minus infinity, no part in
 * its group's rank.  Where fewer than k eligible experts are left, switched-off ones of the kept
 * groups follow, in ascending order, with gate 0.  Other non-finite logits: unspecified values,
 * picks inside [0, E).
 * Without a bias, and unless groups are ranked by two keys, keys are compared through their logits, exactly.
 * Else near ties are decided by keys in 64 bits (in which sigmoid scores of logits above 37 are all 1, and tie).
 * Keys in 32 bits decide what they can; a token of nearer ones (2^-18 of 1 + |c| for a softmax, 2^-21 for a
 * sigmoid), or of fewer than k experts left, takes longer: a whole wave, one such token after the other.
 */
enum { MOE_SCORE_SOFTMAX = 0, MOE_SCORE_SIGMOID = 1 };

typedef struct moe_route_config {
    int32_t score;       /* MOE_SCORE_*                                               */
    int32_t n_groups;    /* 1 = no groups; at most 64, a divisor of n_experts          */
    int32_t groups_kept; /* 1 .. n_groups                                             */
    int32_t group_top;   /* 1 or 2 (at most the experts of a group)                    */
    int32_t renormalize; /* 0 or 1                                                    */
    float scale;         /* finite, of every gate                                     */
} moe_route_config;

#define MOE_ROUTE_MAX_EXPERTS 512

/*
 *   logits      [T, E] fp32 in
 *   select_bias [E]    fp32 or NULL (finite)
 *   topk_idx [T, k] int32, topk_gate [T, k] fp32 out; scores [T, E] fp32 out or NULL
 * 1 <= k <= groups_kept * E / n_groups, k <= 64, E <= MOE_ROUTE_MAX_EXPERTS; any number of tokens.
 * Pointers of 4-byte elements need 4-byte alignment only.
 */
MOE_API int moe_route_scored(const moe_route_config* config, int32_t n_tokens, int32_t n_experts, int32_t top_k,
                             const float* logits, const float* select_bias, int32_t* topk_idx,
                             float* topk_gate, float* scores, void* stream);

/*
 * Gradient of moe_route_scored's gates and scores with regard to the logits, for the picks it made (the
 * picks themselves, and through them the bias and the groups, have none).  grad_gate [T, k] fp32;
 * grad_scores [T, E] fp32 or NULL; grad_logits [T, E] fp32 out, every element written.  Of a row whose
 * picked scores are all 0 the gates have no gradient.  What the two hold for an expert that is switched
 * off (an infinity or a NaN, say) plays no part.  Entries of topk_idx outside [0, E) are ignored; an
 * expert that is named twice counts twice.
 */
MOE_API int moe_route_scored_backward(const moe_route_config* config, int32_t n_tokens, int32_t n_experts,
                                      int32_t top_k, const float* logits, const int32_t* topk_idx,
                                      const float* grad_gate, const float* grad_scores,
                                      float* grad_logits, void* stream);

/*
 * ---- Experts in microscaled 4-bit floating point (MXFP4) ------------------------------------------
 *
 * 32 neighbours of a row share a scale 2^(b - 127), b one byte (E8M0); each value is a code of 4 bits
 * (E2M1: 0, .5, 1, 1.5, 2, 3, 4, 6 and their negatives, the sign in the highest bit).  A row of C values
 * has C / 2 bytes of codes, the lower four bits first, and ceil(C / 32) bytes of scales; C is a multiple
 * of 8, and the last block may be short.  Quantisation: with 2^e <= max|x| < 2^(e+1) over the block,
 * b = max(0, e - 2 + 127) and code = the value of E2M1 nearest to x / 2^(b - 127), ties to the even code,
 * magnitudes above 6 to 6.  A block of zeros has b = 0; one that holds a NaN or an infinity has b = 255,
 * and all of its values read back as NaN.
 */

/* x [rows, cols] (act_dtype, 16-byte aligned) -> codes [rows, cols / 2], scales [rows, ceil(cols / 32)].  codes: 4-byte aligned; cols <= 2^24,
 * rows cols <= 2^40. */
MOE_API int moe_mxfp4_quantize(const void* x, int64_t rows, int32_t cols, int32_t act_dtype,
                               uint8_t* codes, uint8_t* scales, void* stream);
/* The values that codes and scales stand for, in act_dtype, exactly (subnormal ones too; above the type's range
 * infinity).  A block of b = 255 gives NaN. */
MOE_API int moe_mxfp4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int32_t cols,
                                 int32_t act_dtype, void* x, void* stream);

/* Layout of weights for moe_mxfp4_experts, made once: n_matrices row-major matrices [rows, cols] of codes and
 * scales as above, in the order in which the matrix units read them.  cols and rows: multiples of 8, at most 2^24; the
 * result (16-byte aligned) under 2^46 bytes. */
MOE_API size_t moe_mxfp4_packed_bytes(int32_t n_matrices, int32_t rows, int32_t cols); /* 0 if invalid */
MOE_API int moe_mxfp4_pack(const uint8_t* codes, const uint8_t* scales, int32_t n_matrices, int32_t rows,
                           int32_t cols, void* packed, void* stream);

/* Packed weights of one layer: gate, up from [E, F, d], down from [E, d, F].  The router's fields are
 * read by moe_mxfp4_forward alone: router_w [E, d] fp32, router_b [E] (of the logits) and select_bias [E]
 * fp32 or NULL.  All but the last two, which need 4-byte alignment only, are 16-byte aligned. */
typedef struct moe_mxfp4_weights {
    const float* router_w;
    const float* router_b;
    const float* select_bias;
    const void* gate;
    const void* up;
    const void* down;
} moe_mxfp4_weights;

/*
 * The expert layer on such weights, from the picks on: with Q the rounding of a row to MXFP4 and back,
 *   h_tj = silu(W_gate,e Q(x_t)) * (W_up,e Q(x_t)),  e = topk_idx[t,j],
 *   y_t  = sum_j topk_gate[t,j] W_down,e Q(h_tj)   (+ x_t with MOE_FLAG_RESIDUAL).
 * Products and the gated sum are formed in fp32, from rows as they were summed, and y is rounded once.  shape.rank must be 0, d_model and
 * d_ff at most 2^18, and tiles of 256 pairs by 128 hidden, or 256 output, columns fewer than 2^23 - 256 (T k F < 2^38 and T k d < 2^39, nearly: a
 * workspace of 137 GB); the other limits are the layer's (E <= 64, T k < 2^24).
 *   x, y [T, d] act_dtype, y not aliasing x; topk_idx [T, k] int32 (pairs outside [0, E) leave their token's row unspecified),
 *   topk_gate [T, k] fp32; workspace: moe_mxfp4_workspace_bytes(shape), 16-byte aligned.
 */
MOE_API size_t moe_mxfp4_workspace_bytes(const moe_shape* shape);
MOE_API int moe_mxfp4_experts(const moe_shape* shape, const moe_mxfp4_weights* weights, const void* x,
                              const int32_t* topk_idx, const float* topk_gate, void* y, void* workspace,
                              size_t workspace_bytes, void* stream);

/*
 * Whole layer: logits = router_w x (+ router_b), summed in fp32 as moe_route does, moe_route_scored with
 * weights.select_bias, moe_mxfp4_experts.  topk_idx, topk_gate [T, k] and logits [T, E] fp32 are outputs or
 * NULL (with the logits and the picks, moe_route_scored_backward has what it needs).
 */
MOE_API int moe_mxfp4_forward(const moe_shape* shape, const moe_route_config* config,
                              const moe_mxfp4_weights* weights, const void* x, void* y, int32_t* topk_idx,
                              float* topk_gate, float* logits, void* workspace, size_t workspace_bytes,
                              void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MOE_QUANTISED_H_ */
