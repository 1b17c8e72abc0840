// Expert feed-forward on weights in microscaled 4-bit floating point: the entry points and the order of the
// stages, and the kernels between the picks and the combine.
//
// The pairs (token, slot) of an expert are brought together in blocks of 32 rows, every expert's from a block of
// its own, in the layout of mxfp4.h; the order inside an expert does not matter to any result.
#include <algorithm>

#include "gemm.h"
#include "mxfp4.h"
#include "mxfp4_plan.h"

namespace moe {

namespace {

constexpr int kThreads = 256;

// ---- rows of the experts, quantised --------------------------------------------------------------------------
// A workgroup makes one block of 32 rows.  Up to kMxKeyPairs pairs it finds the expert of its block and the pairs of its rows
// from all picks itself (PairKeys); beyond, from the sorted pairs (perm, offsets).  A lane takes the 32 values of a
// row that share a scale, so that nothing is exchanged and the block leaves in runs of 1 KB.
constexpr int kRowThreads = 512, kRowWaves = kRowThreads / kWave;
constexpr int kMxKeyPairs = kKeyChunks * 4 * kRowThreads;
template <typename T>
__global__ __launch_bounds__(kRowThreads) void mx_rows_kernel(const T* __restrict__ x, const int32_t* __restrict__ idx, const int32_t* __restrict__ perm,
                                                              const int32_t* __restrict__ offsets, int P, int E, int k, int d, int32_t* __restrict__ starts,
                                                              int32_t* __restrict__ slot, char* __restrict__ codes, char* __restrict__ scales) {
    typedef Store<T> S;
    constexpr int VECS = 32 / S::VEC;
    __shared__ int s_count[kRowWaves][kMaxExperts], s_pair[32 + kWave];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), block = blockIdx.x;
    const int units = mx_units(d);
    int lo = 0, hi = 0;
    PairKeys<kRowThreads> keys;
    if (!perm) {
        keys.load(idx, P);
        keys.bounds(E, s_count, lo, hi);
    } else if (lane < E) {
        lo = offsets[lane];
        hi = offsets[lane + 1];
    }
    const int n_blocks = mx_blocks(hi - lo), end = wave_scan(n_blocks), start = end - n_blocks;
    if (block == 0 && blockIdx.y == 0 && wave == 0) {
        if (lane < E) starts[lane] = start;
        if (lane == E - 1) starts[E] = end;
    }
    const unsigned long long at = __ballot(start <= block && block < end);
    if (!at) return;
    const int e = __ffsll((long long)at) - 1, first = (block - MOE_READLANE(start, e)) * 32;
    const int e_lo = MOE_READLANE(lo, e), n = min(32, MOE_READLANE(hi, e) - e_lo - first);
    if (!perm) {
        keys.rows(e, first, n, 32, s_count, s_pair);
    } else {
        if (threadIdx.x < n) s_pair[threadIdx.x] = perm[e_lo + first + threadIdx.x];
        __syncthreads();
    }
    if (blockIdx.y == 0 && threadIdx.x < n) slot[s_pair[threadIdx.x]] = block * 32 + threadIdx.x;
    // a wave takes a k-step of 128 columns
    const int step = blockIdx.y * kRowWaves + wave, u = step >> 1, c = step & 1;
    if (u >= units) return;
    const int col = step * 128 + (lane >> 4) * 32;
    unsigned scale = 0;
    typename S::vec_t v[2][VECS];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int p = s_pair[min(16 * t + (lane & 15), n - 1)];  // (rows past the last are the last one again)
        const T* row = x + (size_t)quick_div(p, k) * d;
#pragma unroll
        for (int i = 0; i < VECS; ++i) v[t][i] = *reinterpret_cast<const typename S::vec_t*>(row + min(col + i * S::VEC, d - S::VEC));
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        if (col + 32 > d) {
#pragma unroll
            for (int i = 0; i < VECS; ++i)
                if (col + i * S::VEC >= d) v[t][i] = typename S::vec_t{};
        }
        i32x4 codes8;
        int b;
        mx_quantise_32<T>(v[t], codes8, b);
        *reinterpret_cast<i32x4*>(codes + ((size_t)block * units + u) * kMxCodes + (c * 2 + t) * 1024 + lane * 16) = codes8;
        scale |= (unsigned)b << (8 * t);
    }
    *reinterpret_cast<uint16_t*>(scales + ((size_t)block * units + u) * kMxScales + lane * 4 + c * 2) = (uint16_t)scale;
}

// ---- combine --------------------------------------------------------------------------------------------------------
// y_t = sum_j g_tj (row of pair (t, j)) (+ x_t), of rows in fp32, in fp32 and ascending j, rounded once; a lane takes one 16-byte piece
// of a row of y.  (Rows in bf16 are half the bytes here and for the product that writes them: 16384 tokens of 2048 / 5632, us, down 204 and this 34 with
// them, 236 and 54 now, a layer 7 % longer; 2048 tokens 130 and 136.)
template <typename T>
__global__ __launch_bounds__(kThreads) void mx_combine_kernel(const float* __restrict__ rows, const int32_t* __restrict__ slot, const float* __restrict__ gate,
                                                              const T* __restrict__ residual, T* __restrict__ y, int pieces, int k, long long all, int last_row) {
    typedef Store<T> S;
    for (long long i = blockIdx.x * (long long)kThreads + threadIdx.x; i < all; i += gridDim.x * (long long)kThreads) {
        const long long t = i / pieces;
        const int at = (int)(i - t * pieces) * S::VEC;
        const size_t d = (size_t)pieces * S::VEC;
        float f[S::VEC];
#pragma unroll
        for (int q = 0; q < S::VEC; ++q) f[q] = 0.f;
        // (four rows at a time: one after the other, each waits for its place and then for itself)
        for (int j0 = 0; j0 < k; j0 += 4) {
            int r[4];
            float w[4];
            f32x4 v[4][S::VEC / 4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                r[j] = slot[t * k + min(j0 + j, k - 1)];
                w[j] = gate[t * k + min(j0 + j, k - 1)];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                r[j] = min(max(r[j], 0), last_row);  // (in range for picks of no expert as well)
                if (j0 + j < k) {
#pragma unroll
                    for (int q = 0; q < S::VEC / 4; ++q) v[j][q] = *reinterpret_cast<const f32x4*>(rows + r[j] * d + at + 4 * q);
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (j0 + j >= k) break;
#pragma unroll
                for (int q = 0; q < S::VEC; ++q) f[q] = fmaf(w[j], v[j][q / 4][q % 4], f[q]);
            }
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
    l.offsets = take((s.n_experts + 1) * sizeof(int32_t));
    l.perm = take(P > kMxKeyPairs ? P * sizeof(int32_t) : 0);
    l.sort = take(P > kMxKeyPairs ? sizeof(int32_t) * 256 * s.n_experts : 0);  // (launch_permute: up to 256 counts an expert)
    l.xq = take((size_t)l.blocks * mx_units(s.d_model) * (kMxCodes + kMxScales));
    l.hq = take((size_t)l.blocks * mx_units(s.d_ff) * (kMxCodes + kMxScales));
    l.y = take((size_t)l.blocks * 32 * s.d_model * sizeof(float));
    l.total = cur;
    return l;
}

template <typename T>
static int experts(const moe_shape& s, const moe_mxfp4_weights& w, const T* x, const int32_t* idx, const float* gate, T* y, const MxLayout& l, char* ws,
                   hipStream_t st) {
    const int P = s.n_tokens * s.top_k, E = s.n_experts, d = s.d_model, F = s.d_ff;
    int32_t* slot = reinterpret_cast<int32_t*>(ws + l.slot);
    int32_t* starts = reinterpret_cast<int32_t*>(ws + l.starts);
    const int32_t *perm = nullptr, *offsets = nullptr;
    if (P > kMxKeyPairs) {
        int32_t* sorted = reinterpret_cast<int32_t*>(ws + l.perm);
        const int rc = launch_permute(P, E, idx, reinterpret_cast<int32_t*>(ws + l.offsets), sorted, slot, ws + l.sort, l.xq - l.sort, st);
        if (rc != MOE_OK) return rc;
        perm = sorted;
        offsets = reinterpret_cast<int32_t*>(ws + l.offsets);
    }
    const int units = mx_units(d);
    hipLaunchKernelGGL(mx_rows_kernel<T>, dim3(l.blocks, (2 * units + kRowWaves - 1) / kRowWaves), dim3(kRowThreads), 0, st, x, idx, perm, offsets, P, E, s.top_k, d,
                       starts, slot, ws + l.xq, ws + l.xq + (size_t)l.blocks * units * kMxCodes);
    auto product = [&](bool swiglu, const void* w0, const void* w1, char* a, char* out, int N, int K) {
        const int rows = mx_tile_rows(swiglu, P, E, N, K);
        return rows <= 32 ? launch_mx_stream(swiglu, w0, w1, a, out, starts, P, E, l.blocks, N, K, st)
                          : launch_mx_gemm(swiglu, w0, w1, a, out, starts, P, E, l.blocks, N, K, rows, st);
    };
    int rc = product(true, w.gate, w.up, ws + l.xq, ws + l.hq, F, d);
    if (rc == MOE_OK) rc = product(false, w.down, nullptr, ws + l.hq, ws + l.y, d, F);
    if (rc != MOE_OK) return rc;
    const int pieces = d / Store<T>::VEC;
    const long long all = (long long)s.n_tokens * pieces;
    hipLaunchKernelGGL(mx_combine_kernel<T>, dim3((unsigned)std::min<long long>((all + kThreads - 1) / kThreads, 1 << 20)), dim3(kThreads), 0, st,
                       reinterpret_cast<const float*>(ws + l.y), slot, gate, (s.flags & MOE_FLAG_RESIDUAL) ? x : nullptr, y, pieces, s.top_k, all, l.blocks * 32 - 1);
    return launch_status();
}

int launch_mx_experts(const moe_shape& s, const moe_mxfp4_weights& w, const void* x, const int32_t* idx, const float* gate, void* y,
                      const MxLayout& l, char* ws, hipStream_t st) {
    if (mx_few(s)) return launch_mx_few(s, w, x, idx, gate, y, l, ws, st);
    if (s.act_dtype == MOE_F32) return experts<float>(s, w, static_cast<const float*>(x), idx, gate, static_cast<float*>(y), l, ws, st);
    return experts<bf16_t>(s, w, static_cast<const bf16_t*>(x), idx, gate, static_cast<bf16_t*>(y), l, ws, st);
}

constexpr int kMxMaxWidth = 1 << 18;
static int validate_mx(const moe_shape* s) {
    const int rc = validate_shape(s);
    if (rc != MOE_OK) return rc;
    if (s->flags & MOE_FLAG_SHARED_BASE) return MOE_ERR_INVALID;
    // (tiles are counted, and scales of a matrix found, in 32 bits)
    if (s->d_model > kMxMaxWidth || s->d_ff > kMxMaxWidth) return MOE_ERR_UNSUPPORTED;
    const int P = s->n_tokens * s->top_k;
    if (!mx_tiles_fit(true, P, s->n_experts, s->d_ff, 256) || !mx_tiles_fit(false, P, s->n_experts, s->d_model, 256)) return MOE_ERR_UNSUPPORTED;
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
    for (const float* p : {weights->router_b, weights->select_bias})  // (read value by value)
        if (reinterpret_cast<uintptr_t>(p) & 3) return MOE_ERR_INVALID;
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
