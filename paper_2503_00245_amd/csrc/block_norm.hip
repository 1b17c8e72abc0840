// The block around a layer: its end (norm, gates, dropout, scaled residual) and the start of the next (norm), in one pass over the
// rows, and the gradient of both in one pass and a small sum over tokens (moe_training.h states them).
//
// A row is held in registers, so that every tensor is read once and written once: what bounds both is memory.
// WAVES of a workgroup share a row of up to WAVES * 512 * CHUNKS values; one wave a row where rows fill the chip (no barrier).
#include <algorithm>
#include <cmath>

#include "moe_training.h"
#include "rows8.h"

namespace moe {

namespace {

struct BlockArgs {
    const void *x, *b;                        // backward: x is grad_y, see there
    const float *post_w, *gate, *token_gate, *open_w;
    const uint64_t* rng;
    void *y, *n;
    int T, d;
    float eps, skip_scale, block_scale, keep_scale, inv_d;
    unsigned drop;                            // halves below this are dropped; 0: no dropout
    // backward
    const void *grad_y, *grad_n;
    void *grad_x, *grad_b;
    float *grad_token_gate, *parts;           // parts [workgroups][3][d]: open_w, post_w, gate
};

// Philox4x32-10: ten rounds of two 32 x 32 products of which the upper half is mixed with the other words and the key.
__device__ __forceinline__ void philox(uint64_t seed, uint64_t lo, uint64_t hi, unsigned (&w)[4]) {
    unsigned k0 = (unsigned)seed, k1 = (unsigned)(seed >> 32);
    w[0] = (unsigned)lo, w[1] = (unsigned)(lo >> 32), w[2] = (unsigned)hi, w[3] = (unsigned)(hi >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)w[0] * 0xD2511F53u, b = (uint64_t)w[2] * 0xCD9E8D57u;
        w[0] = (unsigned)(b >> 32) ^ w[1] ^ k0;
        w[1] = (unsigned)b;
        w[2] = (unsigned)(a >> 32) ^ w[3] ^ k1;
        w[3] = (unsigned)a;
        k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
    }
}
// Bit i: value i of the eight from element 8 q on is kept
__device__ __forceinline__ unsigned kept8(uint64_t seed, uint64_t offset, uint64_t q, unsigned drop) {
    unsigned w[4], m = 0;
    philox(seed, q, offset, w);
#pragma unroll
    for (int i = 0; i < 4; ++i) m |= ((w[i] & 0xFFFFu) >= drop ? 1u : 0u) << (2 * i) | ((w[i] >> 16) >= drop ? 1u : 0u) << (2 * i + 1);
    return m;
}

// Sums of N values over the waves of a row; s [2][N * WAVES], used in turn so that one barrier a sum is enough
template <int WAVES, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* s, int& turn) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (WAVES > 1) {
        const int wave = threadIdx.x / kWave;
        float* const at = s + turn * (4 * WAVES);
        turn ^= 1;
        if ((threadIdx.x & (kWave - 1)) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) at[i * WAVES + wave] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) v[i] += at[i * WAVES + w];
        }
    }
}

template <typename T, int WAVES, int CHUNKS>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * kWave) void block_norm_kernel(const BlockArgs g) {
    __shared__ float s_sum[2 * 4 * WAVES];
    int turn = 0;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int t = WAVES == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
    if (t >= g.T) return;
    const int c0 = ((WAVES == 1 ? 0 : wave * kWave) + lane) * 8;
    constexpr int STEP = WAVES * kWave * 8;
    const T *const x = static_cast<const T*>(g.x) + (size_t)t * g.d, *const b = static_cast<const T*>(g.b) + (size_t)t * g.d;
    Raw8<T> xv[CHUNKS], bv[CHUNKS];
#pragma unroll
    for (int q = 0; q < CHUNKS; ++q) {
        const int c = c0 + q * STEP;
        xv[q] = Raw8<T>{}, bv[q] = Raw8<T>{};
        if (c < g.d) {
            xv[q] = load8(x + c);
            if (g.b) bv[q] = load8(b + c);
        }
    }
    if (g.b) {
        float r = 1.f;
        if (g.post_w) {
            float sum[1] = {0.f};
#pragma unroll
            for (int q = 0; q < CHUNKS; ++q)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[0] = fmaf(at8(bv[q], i), at8(bv[q], i), sum[0]);
            row_sums<WAVES>(sum, s_sum, turn);
            r = rsqrtf(fmaf(sum[0], g.inv_d, g.eps));
        }
        const float scale = g.block_scale * (g.token_gate ? g.token_gate[t] : 1.f);
        uint64_t seed = 0, offset = 0;
        if (g.drop) seed = g.rng[0], offset = g.rng[1];
#pragma unroll
        for (int q = 0; q < CHUNKS; ++q) {
            const int c = c0 + q * STEP;
            if (c >= g.d) continue;
            const unsigned kept = g.drop ? kept8(seed, offset, ((uint64_t)t * g.d + c) >> 3, g.drop) : 0xFFu;
            Raw8<float> pw{}, gt{};
            if (g.post_w) pw = load8(g.post_w + c);
            if (g.gate) gt = load8(g.gate + c);
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float z = at8(bv[q], i);
                if (g.post_w) z = z * r * at8(pw, i);
                z = (kept >> i & 1u) ? z * g.keep_scale : 0.f;
                float m = scale;
                if (g.gate) m *= at8(gt, i);
                o[i] = fmaf(m, z, g.skip_scale * at8(xv[q], i));
            }
            xv[q] = round8<T>(o);
            store8(static_cast<T*>(g.y) + (size_t)t * g.d + c, xv[q]);
        }
    }
    if (!g.open_w) return;
    float sum[1] = {0.f};
#pragma unroll
    for (int q = 0; q < CHUNKS; ++q)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[0] = fmaf(at8(xv[q], i), at8(xv[q], i), sum[0]);
    row_sums<WAVES>(sum, s_sum, turn);
    const float r = rsqrtf(fmaf(sum[0], g.inv_d, g.eps));
#pragma unroll
    for (int q = 0; q < CHUNKS; ++q) {
        const int c = c0 + q * STEP;
        if (c >= g.d) continue;
        const Raw8<float> w = load8(g.open_w + c);
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = at8(xv[q], i) * r * at8(w, i);
        store8(static_cast<T*>(g.n) + (size_t)t * g.d + c, round8<T>(o));
    }
}

// G = grad_y + r2 (u - y r2^2 mean(u y)), u = grad_n open_w; z = G * (what the norm of b was multiplied by), and for a post_w the
// same once more: grad_b = r1 (v - b r1^2 mean(v b)), v = z post_w.  A workgroup takes rows in turn and keeps its sums over them for
// the [d] gradients in registers, a value per column (PARTS); they are added up over the workgroups by a second kernel.
// ROWS: rows that a workgroup has in hand (one wave each where WAVES is 1).
template <typename T, int WAVES, int CHUNKS, bool PARTS>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * kWave) void block_grad_kernel(const BlockArgs g) {
    constexpr int ROWS = WAVES == 1 ? 4 : 1;
    __shared__ float s_sum[2 * 4 * WAVES];
    __shared__ float s_parts[PARTS && ROWS > 1 ? ROWS * kWave * 8 : 1];
    int turn = 0;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int c0 = ((WAVES == 1 ? 0 : wave * kWave) + lane) * 8;
    constexpr int STEP = WAVES * kWave * 8;
    float acc[PARTS ? 3 : 1][PARTS ? CHUNKS : 1][8];
    if (PARTS) {
#pragma unroll
        for (int k = 0; k < 3; ++k)
#pragma unroll
            for (int q = 0; q < CHUNKS; ++q)
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[k][q][i] = 0.f;
    }
    uint64_t seed = 0, offset = 0;
    if (g.drop && g.b) seed = g.rng[0], offset = g.rng[1];
    for (int t = blockIdx.x * ROWS + (WAVES == 1 ? wave : 0); t < g.T; t += gridDim.x * ROWS) {
        const size_t row = (size_t)t * g.d;
        Raw8<T> gy[CHUNKS], gn[CHUNKS], y[CHUNKS], b[CHUNKS];
#pragma unroll
        for (int q = 0; q < CHUNKS; ++q) {
            const int c = c0 + q * STEP;
            gy[q] = gn[q] = y[q] = b[q] = Raw8<T>{};
            if (c < g.d) {
                if (g.grad_y) gy[q] = load8(static_cast<const T*>(g.grad_y) + row + c);
                if (g.grad_n) {
                    gn[q] = load8(static_cast<const T*>(g.grad_n) + row + c);
                    y[q] = load8(static_cast<const T*>(g.y) + row + c);
                }
                if (g.b) b[q] = load8(static_cast<const T*>(g.b) + row + c);
            }
        }
        float sum[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int q = 0; q < CHUNKS; ++q) {
            const int c = c0 + q * STEP;
            Raw8<float> w{};
            if (g.grad_n && c < g.d) w = load8(g.open_w + c);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float yi = at8(y[q], i), bi = at8(b[q], i);
                sum[0] = fmaf(yi, yi, sum[0]);
                sum[1] = fmaf(at8(gn[q], i) * at8(w, i), yi, sum[1]);
                sum[2] = fmaf(bi, bi, sum[2]);
            }
        }
        row_sums<WAVES>(sum, s_sum, turn);
        const float r2 = rsqrtf(fmaf(sum[0], g.inv_d, g.eps)), r1 = g.post_w ? rsqrtf(fmaf(sum[2], g.inv_d, g.eps)) : 1.f;
        const float m2 = sum[1] * g.inv_d * r2 * r2;
        const float tg = g.token_gate ? g.token_gate[t] : 1.f;
        float dots[2] = {0.f, 0.f};  // <v, b>; the token gate's gradient
        float v[CHUNKS][8];
#pragma unroll
        for (int q = 0; q < CHUNKS; ++q) {
            const int c = c0 + q * STEP;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[q][i] = 0.f;
            if (c >= g.d) continue;
            float G[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) G[i] = at8(gy[q], i);
            if (g.grad_n) {
                const Raw8<float> w = load8(g.open_w + c);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float yi = at8(y[q], i), ni = at8(gn[q], i);
                    G[i] += r2 * (ni * at8(w, i) - yi * m2);
                    if (PARTS) acc[0][q][i] = fmaf(ni, yi * r2, acc[0][q][i]);
                }
            }
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = g.b ? g.skip_scale * G[i] : G[i];
            store8(static_cast<T*>(g.grad_x) + row + c, round8<T>(o));
            if (!g.b) continue;
            const unsigned kept = g.drop ? kept8(seed, offset, (row + c) >> 3, g.drop) : 0xFFu;
            Raw8<float> pw{}, gt{};
            if (g.post_w) pw = load8(g.post_w + c);
            if (g.gate) gt = load8(g.gate + c);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float bi = at8(b[q], i), w = g.post_w ? at8(pw, i) : 1.f, gate = g.gate ? at8(gt, i) : 1.f;
                const float up = (kept >> i & 1u) ? G[i] * (g.block_scale * g.keep_scale) : 0.f;
                const float norm = bi * r1;
                const float bare = (kept >> i & 1u) ? up * (norm * w) : 0.f;  // (a dropped infinity has no part)
                dots[1] = fmaf(bare, gate, dots[1]);
                const float z = up * (tg * gate);
                if (PARTS) {
                    acc[1][q][i] += (kept >> i & 1u) ? z * norm : 0.f;
                    acc[2][q][i] = fmaf(bare, tg, acc[2][q][i]);
                }
                v[q][i] = z * w;
                dots[0] = fmaf(v[q][i], bi, dots[0]);
            }
        }
        if (!g.b) continue;
        if (g.post_w || g.grad_token_gate) row_sums<WAVES>(dots, s_sum, turn);
        const float m1 = g.post_w ? dots[0] * g.inv_d * r1 * r1 : 0.f;
#pragma unroll
        for (int q = 0; q < CHUNKS; ++q) {
            const int c = c0 + q * STEP;
            if (c >= g.d) continue;
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = g.post_w ? r1 * (v[q][i] - at8(b[q], i) * m1) : v[q][i];
            store8(static_cast<T*>(g.grad_b) + row + c, round8<T>(o));
        }
        if (g.grad_token_gate && lane == 0 && (WAVES == 1 || wave == 0)) g.grad_token_gate[t] = dots[1];
    }
    if constexpr (PARTS) {
        float* const out = g.parts + (size_t)blockIdx.x * 3 * g.d;
#pragma unroll
        for (int k = 0; k < 3; ++k)
#pragma unroll
            for (int q = 0; q < CHUNKS; ++q) {
                const int c = c0 + q * STEP;
                if constexpr (ROWS == 1) {
                    if (c < g.d) store8(out + (size_t)k * g.d + c, round8<float>(acc[k][q]));
                } else {  // over the four waves, 128 columns each
                    __syncthreads();
#pragma unroll
                    for (int i = 0; i < 8; ++i) s_parts[wave * 512 + i * kWave + lane] = acc[k][q][i];
                    __syncthreads();
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int at = h * 256 + (int)threadIdx.x, col = q * STEP + (at & 63) * 8 + (at >> 6);
                        const float f = (s_parts[at] + s_parts[512 + at]) + (s_parts[1024 + at] + s_parts[1536 + at]);
                        if (col < g.d) out[(size_t)k * g.d + col] = f;
                    }
                }
            }
    }
}

// Sums of the parts over workgroups: 64 columns by 16 runs of workgroups, joined in LDS
__global__ __launch_bounds__(1024) void block_parts_kernel(const float* __restrict__ parts, int n, int d, float* open_w, float* post_w, float* gate) {
    __shared__ float s_sum[16][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int k = blockIdx.y, c = blockIdx.x * kWave + lane;
    float* const out = k == 0 ? open_w : k == 1 ? post_w : gate;
    if (!out) return;
    float f = 0.f;
    if (c < d)
        for (int i = wave; i < n; i += 16) f += parts[((size_t)i * 3 + k) * d + c];
    s_sum[wave][lane] = f;
    __syncthreads();
    if (wave == 0 && c < d) {
        f = 0.f;
#pragma unroll
        for (int w = 0; w < 16; ++w) f += s_sum[w][lane];
        out[c] = f;
    }
}

// Waves that share a row, chunks of 512 values that one of them holds
struct RowPlan {
    int waves, chunks;
};
RowPlan row_plan(int T, int d) {
    const int chunks = (d + 511) / 512;
    if (chunks <= 4 && T >= 2048) return RowPlan{1, chunks};
    if (chunks <= 16) return RowPlan{4, (chunks + 3) / 4};
    return RowPlan{16, (chunks + 15) / 16};
}
int grad_groups(int T, int d) {  // workgroups of the backward pass where they keep sums over tokens
    const int most = row_plan(T, d).waves == 16 ? 256 : 512;
    return std::min(most, row_plan(T, d).waves == 1 ? (T + 3) / 4 : T);
}

template <typename F>
int by_plan(RowPlan p, F run) {
    typedef std::integral_constant<int, 1> c1;
    typedef std::integral_constant<int, 2> c2;
    typedef std::integral_constant<int, 3> c3;
    typedef std::integral_constant<int, 4> c4;
    typedef std::integral_constant<int, 16> c16;
    auto on = [&](auto waves) { return p.chunks == 1 ? run(waves, c1{}) : p.chunks == 2 ? run(waves, c2{}) : p.chunks == 3 ? run(waves, c3{}) : run(waves, c4{}); };
    return p.waves == 1 ? on(c1{}) : p.waves == 4 ? on(c4{}) : on(c16{});
}

template <typename T>
int run_forward(const BlockArgs& g, hipStream_t st) {
    return by_plan(row_plan(g.T, g.d), [&](auto waves, auto chunks) {
        constexpr int W = decltype(waves)::value;
        hipLaunchKernelGGL((block_norm_kernel<T, W, decltype(chunks)::value>), dim3(W == 1 ? (g.T + 3) / 4 : g.T), dim3(W == 1 ? 256 : W * kWave), 0, st, g);
        return launch_status();
    });
}
template <typename T>
int run_backward(const BlockArgs& g, float* open_w, float* post_w, float* gate, hipStream_t st) {
    const int groups = grad_groups(g.T, g.d);
    const int rc = by_plan(row_plan(g.T, g.d), [&](auto waves, auto chunks) {
        constexpr int W = decltype(waves)::value, C = decltype(chunks)::value;
        const int rows = W == 1 ? (g.T + 3) / 4 : g.T;
        if (g.parts) hipLaunchKernelGGL((block_grad_kernel<T, W, C, true>), dim3(groups), dim3(W == 1 ? 256 : W * kWave), 0, st, g);
        else hipLaunchKernelGGL((block_grad_kernel<T, W, C, false>), dim3(rows), dim3(W == 1 ? 256 : W * kWave), 0, st, g);
        return launch_status();
    });
    if (rc != MOE_OK || !g.parts) return rc;
    hipLaunchKernelGGL(block_parts_kernel, dim3((g.d + kWave - 1) / kWave, 3), dim3(1024), 0, st, g.parts, groups, g.d, open_w, post_w, gate);
    return launch_status();
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
// halves of 65536 that are dropped
unsigned drop_of(const moe_block& b) { return (unsigned)std::nearbyint((double)b.dropout * 65536.0); }

int validate_block(const moe_block* b, int T, int d, int act_dtype) {
    if (!b || T < 0 || d < 1) return MOE_ERR_INVALID;
    if (!(b->eps > 0) || !std::isfinite(b->eps) || !std::isfinite(b->skip_scale) || !std::isfinite(b->block_scale)) return MOE_ERR_INVALID;
    if (!(b->dropout >= 0 && b->dropout < 1) || drop_of(*b) > 65535) return MOE_ERR_INVALID;
    if (drop_of(*b) > 0 && (!b->rng || (reinterpret_cast<uintptr_t>(b->rng) & 7u))) return MOE_ERR_INVALID;
    for (const float* p : {b->post_w, b->gate})
        if (!aligned16(p)) return MOE_ERR_INVALID;
    if (!aligned4(b->token_gate)) return MOE_ERR_INVALID;
    if (act_dtype != MOE_F32 && act_dtype != MOE_BF16) return MOE_ERR_UNSUPPORTED;
    if (d % 8 || d > MOE_BLOCK_MAX_D || T >= (1 << 24)) return MOE_ERR_UNSUPPORTED;
    return MOE_OK;
}
BlockArgs block_args(const moe_block& b, int T, int d) {
    BlockArgs g{};
    g.post_w = b.post_w, g.gate = b.gate, g.token_gate = b.token_gate, g.rng = b.rng;
    g.T = T, g.d = d, g.inv_d = 1.0f / (float)d;
    g.eps = b.eps, g.skip_scale = b.skip_scale, g.block_scale = b.block_scale;
    g.drop = drop_of(b);
    g.keep_scale = (float)(65536.0 / (65536.0 - g.drop));
    return g;
}

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" int moe_block_norm(const moe_block* block, int32_t n_tokens, int32_t d_model, int32_t act_dtype, const void* x, const void* b,
                              const float* open_w, void* y, void* n, void* stream) {
    const int rc = validate_block(block, n_tokens, d_model, act_dtype);
    if (rc != MOE_OK) return rc;
    if (n_tokens == 0) return MOE_OK;
    if ((b == nullptr) != (y == nullptr) || (open_w == nullptr) != (n == nullptr) || (!b && !n)) return MOE_ERR_INVALID;
    for (const void* p : {x, b, (const void*)open_w, (const void*)y, (const void*)n})
        if (!aligned16(p)) return MOE_ERR_INVALID;
    if (!x || (n && (n == x || n == b || n == y)) || (y && y == b)) return MOE_ERR_INVALID;
    BlockArgs g = block_args(*block, n_tokens, d_model);
    g.x = x, g.b = b, g.open_w = open_w, g.y = y, g.n = n;
    return act_dtype == MOE_F32 ? run_forward<float>(g, as_stream(stream)) : run_forward<bf16_t>(g, as_stream(stream));
}

extern "C" size_t moe_block_workspace_bytes(int32_t n_tokens, int32_t d_model) {
    if (n_tokens < 0 || n_tokens >= (1 << 24) || d_model < 1 || d_model % 8 || d_model > MOE_BLOCK_MAX_D) return 0;
    // (a row more than the workgroups of any number of tokens up to this one)
    return round_up(sizeof(float) * 3 * (size_t)d_model * (size_t)std::min(512, n_tokens + 1), 256);
}

extern "C" int moe_block_norm_backward(const moe_block* block, int32_t n_tokens, int32_t d_model, int32_t act_dtype, const void* grad_y,
                                       const void* grad_n, const void* y, const void* b, const float* open_w, void* grad_x, void* grad_b,
                                       float* grad_open_w, float* grad_post_w, float* grad_gate, float* grad_token_gate, void* workspace,
                                       size_t workspace_bytes, void* stream) {
    const int rc = validate_block(block, n_tokens, d_model, act_dtype);
    if (rc != MOE_OK) return rc;
    for (const void* p : {grad_y, grad_n, y, b, (const void*)open_w, (const void*)grad_x, (const void*)grad_b})
        if (!aligned16(p)) return MOE_ERR_INVALID;
    for (const void* p : {grad_open_w, grad_post_w, grad_gate, grad_token_gate})
        if (!aligned4(p)) return MOE_ERR_INVALID;
    if (n_tokens > 0) {  // (of no tokens the rows may be NULL)
        if ((open_w == nullptr) != (grad_n == nullptr) || (!grad_y && !grad_n) || (grad_n && !y) || (b == nullptr) != (grad_b == nullptr)) return MOE_ERR_INVALID;
        if (!b && (grad_post_w || grad_gate || grad_token_gate || !grad_n)) return MOE_ERR_INVALID;
        if ((grad_post_w && !block->post_w) || (grad_open_w && !open_w)) return MOE_ERR_INVALID;
        if (!grad_x) return MOE_ERR_INVALID;
        for (const void* p : {grad_n, y, b})
            if (p && (p == grad_x || p == grad_b)) return MOE_ERR_INVALID;
        if (grad_b && (grad_b == grad_x || grad_b == grad_y)) return MOE_ERR_INVALID;
    }
    BlockArgs g = block_args(*block, n_tokens, d_model);
    g.grad_y = grad_y, g.grad_n = grad_n, g.y = const_cast<void*>(y), g.b = b, g.open_w = open_w;
    g.grad_x = grad_x, g.grad_b = grad_b, g.grad_token_gate = grad_token_gate;
    const bool sums = grad_open_w || grad_post_w || grad_gate;
    if (sums) {
        if (!workspace || workspace_bytes < moe_block_workspace_bytes(n_tokens, d_model)) return MOE_ERR_WORKSPACE;
        if (!aligned16(workspace)) return MOE_ERR_INVALID;
        g.parts = static_cast<float*>(workspace);
    }
    hipStream_t st = as_stream(stream);
    if (n_tokens == 0) {  // sums over no tokens: zeros
        if (!sums) return MOE_OK;
        hipLaunchKernelGGL(block_parts_kernel, dim3((d_model + kWave - 1) / kWave, 3), dim3(1024), 0, st, g.parts, 0, d_model, grad_open_w, grad_post_w, grad_gate);
        return launch_status();
    }
    return act_dtype == MOE_F32 ? run_backward<float>(g, grad_open_w, grad_post_w, grad_gate, st)
                                : run_backward<bf16_t>(g, grad_open_w, grad_post_w, grad_gate, st);
}

extern "C" size_t moe_block_stack_workspace_bytes(const moe_shape* shape) {
    if (validate_shape(shape) != MOE_OK || (shape->flags & MOE_FLAG_RESIDUAL) || shape->d_model > MOE_BLOCK_MAX_D) return 0;
    const size_t rows = round_up((size_t)shape->n_tokens * shape->d_model * elt_size(shape->act_dtype), 256);
    return moe_workspace_bytes(shape) + 2 * rows;
}

extern "C" int moe_block_stack_forward(const moe_shape* shape, const moe_weights* layers, const moe_block* blocks, const float* const* open_w,
                                       int32_t n_layers, const void* x, void* y, int32_t* topk_trace, void* workspace, size_t workspace_bytes,
                                       void* stream) {
    int rc = validate_shape(shape);
    if (rc != MOE_OK) return rc;
    const moe_shape& s = *shape;
    if (n_layers < 1 || !layers || !blocks || !open_w || (s.flags & MOE_FLAG_RESIDUAL)) return MOE_ERR_INVALID;
    moe_shape none = s;
    none.n_tokens = 0;
    for (int l = 0; l < n_layers; ++l) {  // everything is checked before the first launch
        if ((rc = validate_block(&blocks[l], s.n_tokens, s.d_model, s.act_dtype)) != MOE_OK) return rc;
        if (!open_w[l] || !aligned16(open_w[l])) return MOE_ERR_INVALID;
        if ((rc = moe_forward(&none, &layers[l], x, y, nullptr, nullptr, nullptr, 0, stream)) != MOE_OK) return rc;
    }
    if (s.n_tokens == 0) return MOE_OK;
    if (!x || !y || x == y || !aligned16(x) || !aligned16(y)) return MOE_ERR_INVALID;
    if (!workspace || !aligned16(workspace) || workspace_bytes < moe_block_stack_workspace_bytes(shape)) return MOE_ERR_WORKSPACE;
    const size_t layer_bytes = moe_workspace_bytes(shape);
    const size_t rows = round_up((size_t)s.n_tokens * s.d_model * elt_size(s.act_dtype), 256);
    char* const ws = static_cast<char*>(workspace);
    char *const n = ws + layer_bytes, *const b = n + rows;
    rc = moe_block_norm(&blocks[0], s.n_tokens, s.d_model, s.act_dtype, x, nullptr, open_w[0], nullptr, n, stream);
    for (int l = 0; rc == MOE_OK && l < n_layers; ++l) {
        int32_t* trace = topk_trace ? topk_trace + (size_t)l * s.n_tokens * s.top_k : nullptr;
        rc = moe_forward(shape, &layers[l], n, b, trace, nullptr, ws, layer_bytes, stream);
        const bool last = l + 1 == n_layers;
        if (rc == MOE_OK)
            rc = moe_block_norm(&blocks[l], s.n_tokens, s.d_model, s.act_dtype, l == 0 ? x : y, b, last ? nullptr : open_w[l + 1], y, last ? nullptr : n, stream);
    }
    return rc;
}
