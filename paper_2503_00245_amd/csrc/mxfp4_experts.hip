// Expert feed-forward on weights in microscaled 4-bit floating point: the entry points and the order of the
// stages, and the kernels between the picks and the combine.
//
// The pairs (token, slot) of an expert are brought together in blocks of 32 rows, every expert's from a block of
// its own, in the layout of mxfp4.h; the order inside an expert does not matter to any result.
#include <algorithm>

#include "mxfp4.h"

namespace moe {

namespace {

constexpr int kThreads = 256;

// ---- dispatch: the first block of every expert, and every pair's row -------------------------------------
constexpr int kDispatchThreads = 1024;
__global__ __launch_bounds__(kDispatchThreads) void mx_dispatch_kernel(const int32_t* __restrict__ idx, int P, int E, int32_t* __restrict__ starts,
                                                                       int32_t* __restrict__ slot) {
    __shared__ int s_count[kMaxExperts], s_next[kMaxExperts];
    if (threadIdx.x < kMaxExperts) s_count[threadIdx.x] = 0;
    __syncthreads();
    for (int p = threadIdx.x; p < P; p += kDispatchThreads) {
        const unsigned e = (unsigned)idx[p];
        if (e < (unsigned)E) atomicAdd(&s_count[e], 1);
    }
    __syncthreads();
    if (threadIdx.x < kWave) {
        const int e = threadIdx.x, n = e < E ? mx_blocks(s_count[e]) : 0;
        const int end = wave_scan(n);
        s_next[e] = (end - n) * 32;
        if (e < E) starts[e] = end - n;
        if (e == E - 1) starts[E] = end;
    }
    __syncthreads();
    for (int p = threadIdx.x; p < P; p += kDispatchThreads) {
        const unsigned e = (unsigned)idx[p];
        slot[p] = e < (unsigned)E ? atomicAdd(&s_next[e], 1) : -1;
    }
}

// ---- rows of the tokens, quantised, to the rows of their pairs ----------------------------------------------
// A wave takes 512 columns of a token: eight values a lane, four lanes a scale.
template <typename T>
__global__ __launch_bounds__(kThreads) void mx_rows_kernel(const T* __restrict__ x, const int32_t* __restrict__ slot, int T_, int k, int d, int units,
                                                           char* __restrict__ codes, char* __restrict__ scales) {
    typedef Store<T> S;
    const int lane = threadIdx.x & 63;
    const int t = blockIdx.x;
    for (int i = threadIdx.x * 8; i < units * kMxUnit; i += kThreads * 8) {
        float f[8];
#pragma unroll
        for (int q = 0; q < 8; q += S::VEC) {
            if (i < d) {
                const typename S::vec_t v = *reinterpret_cast<const typename S::vec_t*>(x + (size_t)t * d + i + q);
#pragma unroll
                for (int j = 0; j < S::VEC; ++j) f[q + j] = S::get(v, j);
            } else {
#pragma unroll
                for (int j = 0; j < S::VEC; ++j) f[q + j] = 0.f;
            }
        }
        int m = (int)mx_abs_max(f);
        m = max(m, dpp_i32<kDppSwap1>(m));
        m = max(m, dpp_i32<kDppSwap2>(m));
        const int b = mx_scale_byte(m);
        const unsigned c8 = mx_codes8(f, b);
        const int c = i >> 7, q = i >> 5 & 3;
        for (int j = 0; j < k; ++j) {
            const int r = slot[(size_t)t * k + j];
            if (r < 0) continue;
            const size_t unit = (size_t)(r >> 5) * units + (c >> 1);
            const int tile = r >> 4 & 1, ln = q * 16 + (r & 15);
            *reinterpret_cast<unsigned*>(codes + unit * kMxCodes + ((c & 1) * 2 + tile) * 1024 + ln * 16 + (lane & 3) * 4) = c8;
            if ((lane & 3) == 0) scales[unit * kMxScales + ln * 4 + (c & 1) * 2 + tile] = (char)b;
        }
    }
}

// ---- products ---------------------------------------------------------------------------------------------------
// The expert of a block of rows
__device__ __forceinline__ int expert_of(const int32_t* __restrict__ starts, int E, int block) {
    int e = 0;
    while (e < E - 1 && block >= starts[e + 1]) ++e;
    return e;
}

// One wave: 32 output columns (with SWIGLU the same of gate and of up) of 32 rows, operands straight from memory.
// SWIGLU: hidden rows, quantised again, in the layout of the next product; else rows of T.
template <bool SWIGLU, typename T>
__global__ __launch_bounds__(kThreads) void mx_product_kernel(const char* __restrict__ w0, const char* __restrict__ w1, const char* __restrict__ a,
                                                              const int32_t* __restrict__ starts, int E, int all_blocks, int N, int K,
                                                              char* __restrict__ out) {
    const int lane = threadIdx.x & 63;
    const int fb = blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6), sb = blockIdx.y;
    const int units = mx_units(K), fbs = mx_blocks(N), out_units = mx_units(N);
    if (sb >= starts[E]) return;
    const int e = expert_of(starts, E, sb);
    if (fb >= (SWIGLU ? out_units * (kMxUnit / 32) : fbs)) return;
    const char* ac = a + (size_t)sb * units * kMxCodes;
    const char* as = a + (size_t)all_blocks * units * kMxCodes + (size_t)sb * units * kMxScales;
    constexpr int M = SWIGLU ? 2 : 1;
    f32x4 acc[M][2][2];
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int n = 0; n < 2; ++n) acc[m][t][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (fb < fbs) {
        const size_t at = ((size_t)e * fbs + fb) * units, all = (size_t)E * fbs * units * kMxCodes;
        for (int u = 0; u < units; ++u) {
            i32x4 fa[M][2][2], fx[2][2];
            int sa[M];
            const int sx = *reinterpret_cast<const int*>(as + (size_t)u * kMxScales + lane * 4);
#pragma unroll
            for (int m = 0; m < M; ++m) {
                const char* w = m ? w1 : w0;
                sa[m] = *reinterpret_cast<const int*>(w + all + (at + u) * kMxScales + lane * 4);
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int t = 0; t < 2; ++t) fa[m][c][t] = *reinterpret_cast<const i32x4*>(w + (at + u) * kMxCodes + (c * 2 + t) * 1024 + lane * 16);
            }
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int t = 0; t < 2; ++t) fx[c][t] = *reinterpret_cast<const i32x4*>(ac + (size_t)u * kMxCodes + (c * 2 + t) * 1024 + lane * 16);
#pragma unroll
            for (int m = 0; m < M; ++m) {
                acc[m][0][0] = mx_mfma<0, 0>(fa[m][0][0], fx[0][0], acc[m][0][0], sa[m], sx);
                acc[m][0][1] = mx_mfma<0, 1>(fa[m][0][0], fx[0][1], acc[m][0][1], sa[m], sx);
                acc[m][1][0] = mx_mfma<1, 0>(fa[m][0][1], fx[0][0], acc[m][1][0], sa[m], sx);
                acc[m][1][1] = mx_mfma<1, 1>(fa[m][0][1], fx[0][1], acc[m][1][1], sa[m], sx);
                acc[m][0][0] = mx_mfma<2, 2>(fa[m][1][0], fx[1][0], acc[m][0][0], sa[m], sx);
                acc[m][0][1] = mx_mfma<2, 3>(fa[m][1][0], fx[1][1], acc[m][0][1], sa[m], sx);
                acc[m][1][0] = mx_mfma<3, 2>(fa[m][1][1], fx[1][0], acc[m][1][0], sa[m], sx);
                acc[m][1][1] = mx_mfma<3, 3>(fa[m][1][1], fx[1][1], acc[m][1][1], sa[m], sx);
            }
        }
    }
    // a lane holds columns 32 fb + 8 (lane / 16) .. + 8 of rows lane % 16 of both tiles
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = SWIGLU ? silu_f32(acc[0][i / 4][n][i % 4]) * acc[M - 1][i / 4][n][i % 4] : acc[0][i / 4][n][i % 4];
        if constexpr (SWIGLU) {
            int m = (int)mx_abs_max(f);
            m = max(m, __shfl_xor(m, 16, kWave));
            m = max(m, __shfl_xor(m, 32, kWave));
            const int b = mx_scale_byte(m);
            const int c = fb >> 2, q = fb & 3, ln = q * 16 + (lane & 15);
            const size_t unit = (size_t)sb * out_units + (c >> 1);
            *reinterpret_cast<unsigned*>(out + unit * kMxCodes + ((c & 1) * 2 + n) * 1024 + ln * 16 + (lane >> 4) * 4) = mx_codes8(f, b);
            if (lane < 16) out[(size_t)all_blocks * out_units * kMxCodes + unit * kMxScales + ln * 4 + (c & 1) * 2 + n] = (char)b;
        } else {
            const int col = fb * 32 + (lane >> 4) * 8;
            if (col < N) {
                T* y = reinterpret_cast<T*>(out) + ((size_t)sb * 32 + n * 16 + (lane & 15)) * N + col;
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = Store<T>::from_f32(f[i]);
            }
        }
    }
}

// ---- combine --------------------------------------------------------------------------------------------------------
// y_t = sum_j g_tj (row of pair (t, j)) (+ x_t), in fp32 and ascending j; a lane takes one 16-byte piece of a row.
template <typename T>
__global__ __launch_bounds__(kThreads) void mx_combine_kernel(const T* __restrict__ rows, const int32_t* __restrict__ slot, const float* __restrict__ gate,
                                                              const T* __restrict__ residual, T* __restrict__ y, int pieces, int k, long long all) {
    typedef Store<T> S;
    for (long long i = blockIdx.x * (long long)kThreads + threadIdx.x; i < all; i += gridDim.x * (long long)kThreads) {
        const long long t = i / pieces;
        const int at = (int)(i - t * pieces) * S::VEC;
        const size_t d = (size_t)pieces * S::VEC;
        float f[S::VEC];
#pragma unroll
        for (int q = 0; q < S::VEC; ++q) f[q] = 0.f;
        for (int j = 0; j < k; ++j) {
            const int r = max(slot[t * k + j], 0);
            const float g = gate[t * k + j];
            const typename S::vec_t v = *reinterpret_cast<const typename S::vec_t*>(rows + r * d + at);
#pragma unroll
            for (int q = 0; q < S::VEC; ++q) f[q] = fmaf(g, S::get(v, q), f[q]);
        }
        if (residual) {
            const typename S::vec_t v = *reinterpret_cast<const typename S::vec_t*>(residual + t * d + at);
#pragma unroll
            for (int q = 0; q < S::VEC; ++q) f[q] += S::get(v, q);
        }
        typename S::vec_t o;
#pragma unroll
        for (int q = 0; q < S::VEC; ++q) o[q] = S::from_f32(f[q]);
        *reinterpret_cast<typename S::vec_t*>(y + t * d + at) = o;
    }
}

}  // namespace

MxLayout mx_layout(const moe_shape& s) {
    MxLayout l{};
    const long long P = (long long)s.n_tokens * s.top_k;
    l.blocks = (int)std::min<long long>(P, (P + 31ll * std::min<long long>(s.n_experts, P)) / 32);
    size_t cur = 0;
    auto take = [&](size_t bytes) {
        const size_t at = cur;
        cur += round_up(bytes ? bytes : 1, 256);
        return at;
    };
    l.idx = take(P * sizeof(int32_t));
    l.gate = take(P * sizeof(float));
    l.logits = take((size_t)s.n_tokens * s.n_experts * sizeof(float));
    l.slot = take(P * sizeof(int32_t));
    l.starts = take((s.n_experts + 1) * sizeof(int32_t));
    l.xq = take((size_t)l.blocks * mx_units(s.d_model) * (kMxCodes + kMxScales));
    l.hq = take((size_t)l.blocks * mx_units(s.d_ff) * (kMxCodes + kMxScales));
    l.y = take((size_t)l.blocks * 32 * s.d_model * elt_size(s.act_dtype));
    l.total = cur;
    return l;
}

template <typename T>
static int experts(const moe_shape& s, const moe_mxfp4_weights& w, const T* x, const int32_t* idx, const float* gate, T* y, const MxLayout& l, char* ws,
                   hipStream_t st) {
    const int P = s.n_tokens * s.top_k, E = s.n_experts, d = s.d_model, F = s.d_ff;
    int32_t* slot = reinterpret_cast<int32_t*>(ws + l.slot);
    int32_t* starts = reinterpret_cast<int32_t*>(ws + l.starts);
    hipLaunchKernelGGL(mx_dispatch_kernel, dim3(1), dim3(kDispatchThreads), 0, st, idx, P, E, starts, slot);
    hipLaunchKernelGGL(mx_rows_kernel<T>, dim3(s.n_tokens), dim3(kThreads), 0, st, x, slot, s.n_tokens, s.top_k, d, mx_units(d), ws + l.xq,
                       ws + l.xq + (size_t)l.blocks * mx_units(d) * kMxCodes);
    constexpr int W = kThreads / 64;
    hipLaunchKernelGGL((mx_product_kernel<true, T>), dim3(mx_units(F) * (kMxUnit / 32) / W, l.blocks), dim3(kThreads), 0, st,
                       static_cast<const char*>(w.gate), static_cast<const char*>(w.up), ws + l.xq, starts, E, l.blocks, F, d, ws + l.hq);
    hipLaunchKernelGGL((mx_product_kernel<false, T>), dim3((mx_blocks(d) + W - 1) / W, l.blocks), dim3(kThreads), 0, st, static_cast<const char*>(w.down),
                       (const char*)nullptr, ws + l.hq, starts, E, l.blocks, d, F, ws + l.y);
    const int pieces = d / Store<T>::VEC;
    const long long all = (long long)s.n_tokens * pieces;
    hipLaunchKernelGGL(mx_combine_kernel<T>, dim3((unsigned)std::min<long long>((all + kThreads - 1) / kThreads, 1 << 20)), dim3(kThreads), 0, st,
                       reinterpret_cast<const T*>(ws + l.y), slot, gate, (s.flags & MOE_FLAG_RESIDUAL) ? x : nullptr, y, pieces, s.top_k, all);
    return launch_status();
}

int launch_mx_experts(const moe_shape& s, const moe_mxfp4_weights& w, const void* x, const int32_t* idx, const float* gate, void* y,
                      const MxLayout& l, char* ws, hipStream_t st) {
    if (s.act_dtype == MOE_F32) return experts<float>(s, w, static_cast<const float*>(x), idx, gate, static_cast<float*>(y), l, ws, st);
    return experts<bf16_t>(s, w, static_cast<const bf16_t*>(x), idx, gate, static_cast<bf16_t*>(y), l, ws, st);
}

static int validate_mx(const moe_shape* s) {
    const int rc = validate_shape(s);
    if (rc != MOE_OK) return rc;
    if (s->flags & MOE_FLAG_SHARED_BASE) return MOE_ERR_INVALID;
    return s->rank ? MOE_ERR_UNSUPPORTED : MOE_OK;
}
static int validate_call(const moe_shape* s, const moe_mxfp4_weights* w, const void* x, const void* y) {
    if (!w) return MOE_ERR_INVALID;
    for (const void* p : {w->gate, w->up, w->down, x, y})
        if (!p || !aligned16(p)) return MOE_ERR_INVALID;
    return x == y ? MOE_ERR_INVALID : MOE_OK;
}

}  // namespace moe

using namespace moe;

extern "C" size_t moe_mxfp4_workspace_bytes(const moe_shape* shape) {
    return validate_mx(shape) == MOE_OK ? mx_layout(*shape).total : 0;
}

extern "C" int moe_mxfp4_experts(const moe_shape* shape, const moe_mxfp4_weights* weights, const void* x, const int32_t* topk_idx,
                                 const float* topk_gate, void* y, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = validate_mx(shape);
    if (rc != MOE_OK || shape->n_tokens == 0) return rc;
    rc = validate_call(shape, weights, x, y);
    if (rc != MOE_OK) return rc;
    if (!topk_idx || !topk_gate || !workspace || !aligned16(topk_idx) || !aligned16(topk_gate) || !aligned16(workspace)) return MOE_ERR_INVALID;
    const MxLayout l = mx_layout(*shape);
    if (workspace_bytes < l.total) return MOE_ERR_WORKSPACE;
    return launch_mx_experts(*shape, *weights, x, topk_idx, topk_gate, y, l, static_cast<char*>(workspace), as_stream(stream));
}

extern "C" int moe_mxfp4_forward(const moe_shape* shape, const moe_route_config* config, const moe_mxfp4_weights* weights, const void* x, void* y,
                                 int32_t* topk_idx, float* topk_gate, float* logits, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = validate_mx(shape);
    if (rc != MOE_OK) return rc;
    rc = validate_route(config, shape->n_tokens, shape->n_experts, shape->top_k);
    if (rc != MOE_OK || shape->n_tokens == 0) return rc;
    rc = validate_call(shape, weights, x, y);
    if (rc != MOE_OK) return rc;
    if (!weights->router_w || !aligned16(weights->router_w) || !workspace || !aligned16(workspace)) return MOE_ERR_INVALID;
    for (const void* p : {(const void*)topk_idx, (const void*)topk_gate, (const void*)logits})
        if (!aligned16(p)) return MOE_ERR_INVALID;
    const MxLayout l = mx_layout(*shape);
    if (workspace_bytes < l.total) return MOE_ERR_WORKSPACE;
    char* ws = static_cast<char*>(workspace);
    if (!topk_idx) topk_idx = reinterpret_cast<int32_t*>(ws + l.idx);
    if (!topk_gate) topk_gate = reinterpret_cast<float*>(ws + l.gate);
    if (!logits) logits = reinterpret_cast<float*>(ws + l.logits);
    hipStream_t st = as_stream(stream);
    rc = launch_router_logits(*shape, x, weights->router_w, weights->router_b, logits, st);
    if (rc == MOE_OK)
        rc = launch_route_scored(*config, shape->n_tokens, shape->n_experts, shape->top_k, logits, weights->select_bias, topk_idx, topk_gate, nullptr, st);
    if (rc == MOE_OK) rc = launch_mx_experts(*shape, *weights, x, topk_idx, topk_gate, y, l, ws, st);
    return rc;
}
