// The block around a layer: its end (norm, gates, dropout, scaled residual) and the start of the next (norm), in one pass over the
// rows, and the gradient of both in one pass and a small sum over tokens (moe_training.h states them).
//
// A row of up to 8192 values is held in registers, so that every tensor is read once and written once: what bounds both is memory.
// WAVES of a workgroup share a row of up to WAVES * 512 * CHUNKS values: eight values a lane (CHUNKS 1), or sixteen, leave the registers for the weights and the next
// row.  (With a wave a row of 2048, 32 values a lane, weights read again for every row: 60 us forward, 131 back.)
// 16384 rows of 2048, bf16, dropout: forward 55 us (268 MB, 4.9 TB/s), back 85 + 5 (403 MB and 19 MB of sums); 2048 rows of 1440 back 15.3 + 4.5.
// Wider rows, of which sixteen waves leave a lane 128 registers, keep part of the gradient's values in scratch memory: with sums over rows 77 / 329 / 538 registers
// of two / three / four chunks in fp32, 45 / 196 / 335 in bf16; without sums 0 / 110 / 262 and 0 / 22 / 63.  1024 x 16384 bf16 forward 33 us, back 96 + 8; 512 x 32768
// back 260 + 17: 201 MB of rows either way, 39 us of a copy.
#include <algorithm>
#include <cmath>

#include "block_plan.h"
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

// Eight values of a [d] weight for each chunk of a lane.  HOLD: kept over the rows; else read for every row again (rows too wide for
// that).  Without the weight: ones.
template <int CHUNKS, bool HOLD>
struct Columns {
    const float* w;
    Raw8<float> v[HOLD ? CHUNKS : 1];
    __device__ __forceinline__ static Raw8<float> get(const float* w, int c, int d) {
        Raw8<float> r{};
        if (w && c < d) return load8(w + c);
        r.v[0] = r.v[1] = f32x4{1.f, 1.f, 1.f, 1.f};
        return r;
    }
    __device__ __forceinline__ void begin(const float* from, int c0, int step, int d) {
        w = from;
        if constexpr (HOLD) {
#pragma unroll
            for (int q = 0; q < CHUNKS; ++q) v[q] = get(w, c0 + q * step, d);
        }
    }
    __device__ __forceinline__ Raw8<float> at(int q, int c, int d) const {
        if constexpr (HOLD) return v[q];
        else return get(w, c, d);
    }
};

// Rows of one tensor that a lane has in hand (zeros where there is none)
template <typename T, int CHUNKS>
struct RowPart {
    Raw8<T> v[CHUNKS];
    __device__ __forceinline__ void load(const void* from, size_t row, int c0, int step, int d) {
#pragma unroll
        for (int q = 0; q < CHUNKS; ++q) {
            v[q] = Raw8<T>{};
            if (from && c0 + q * step < d) v[q] = load8(static_cast<const T*>(from) + row + c0 + q * step);
        }
    }
};

// Both kernels: workgroups take rows in turn.  What a lane needs of the [d] weights stays in its registers (up to 4096 values a row:
// eight a lane; bf16 up to 8192: sixteen), and the next row is on its way while one is summed.
template <typename T, int WAVES, int CHUNKS>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * kWave) void block_norm_kernel(const BlockArgs g) {
    constexpr int ROWS = WAVES == 1 ? 4 : 1, STEP = WAVES * kWave * 8;
    constexpr bool HOLD = CHUNKS == 1 || (WAVES == 8 && sizeof(T) == 2);
    __shared__ float s_sum[2 * 4 * WAVES];
    int turn = 0;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int c0 = ((WAVES == 1 ? 0 : wave * kWave) + lane) * 8, stride = gridDim.x * ROWS;
    int t = blockIdx.x * ROWS + (WAVES == 1 ? wave : 0);
    if (t >= g.T) return;
    RowPart<T, CHUNKS> x, b;
    x.load(g.x, (size_t)t * g.d, c0, STEP, g.d);
    b.load(g.b, (size_t)t * g.d, c0, STEP, g.d);
    Columns<CHUNKS, HOLD> post_w, gate, open_w;
    post_w.begin(g.post_w, c0, STEP, g.d);
    gate.begin(g.gate, c0, STEP, g.d);
    open_w.begin(g.open_w, c0, STEP, g.d);
    uint64_t seed = 0, offset = 0;
    if (g.drop && g.b) seed = g.rng[0], offset = g.rng[1];
    for (;;) {
        const size_t row = (size_t)t * g.d;
        const int next = t + stride;
        RowPart<T, CHUNKS> x1, b1;
        if (HOLD && next < g.T) {
            x1.load(g.x, (size_t)next * g.d, c0, STEP, g.d);
            b1.load(g.b, (size_t)next * g.d, c0, STEP, g.d);
        }
        if (g.b) {
            float r = 1.f;
            if (g.post_w) {
                float sum[1] = {0.f};
#pragma unroll
                for (int q = 0; q < CHUNKS; ++q)
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[0] = fmaf(at8(b.v[q], i), at8(b.v[q], i), sum[0]);
                row_sums<WAVES>(sum, s_sum, turn);
                r = rsqrtf(fmaf(sum[0], g.inv_d, g.eps));
            }
            const float scale = g.block_scale * g.keep_scale * (g.token_gate ? g.token_gate[t] : 1.f);
#pragma unroll
            for (int q = 0; q < CHUNKS; ++q) {
                const int c = c0 + q * STEP;
                if (c >= g.d) continue;
                const unsigned kept = g.drop ? kept8(seed, offset, (row + c) >> 3, g.drop) : 0xFFu;
                const Raw8<float> pw = post_w.at(q, c, g.d), gt = gate.at(q, c, g.d);
                float o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float z = at8(b.v[q], i) * r * at8(pw, i);
                    o[i] = fmaf(scale * at8(gt, i), (kept >> i & 1u) ? z : 0.f, g.skip_scale * at8(x.v[q], i));
                }
                x.v[q] = round8<T>(o);
                store8(static_cast<T*>(g.y) + row + c, x.v[q]);
            }
        }
        if (g.open_w) {
            float sum[1] = {0.f};
#pragma unroll
            for (int q = 0; q < CHUNKS; ++q)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[0] = fmaf(at8(x.v[q], i), at8(x.v[q], i), sum[0]);
            row_sums<WAVES>(sum, s_sum, turn);
            const float r = rsqrtf(fmaf(sum[0], g.inv_d, g.eps));
#pragma unroll
            for (int q = 0; q < CHUNKS; ++q) {
                const int c = c0 + q * STEP;
                if (c >= g.d) continue;
                const Raw8<float> w = open_w.at(q, c, g.d);
                float o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = at8(x.v[q], i) * r * at8(w, i);
                store8(static_cast<T*>(g.n) + row + c, round8<T>(o));
            }
        }
        t = next;
        if (t >= g.T) return;
        if (HOLD) {
            x = x1, b = b1;
        } else {
            x.load(g.x, (size_t)t * g.d, c0, STEP, g.d);
            b.load(g.b, (size_t)t * g.d, c0, STEP, g.d);
        }
    }
}

// G = grad_y + r2 (u - y r2^2 mean(u y)), u = grad_n open_w; z = G * (what the norm of b was multiplied by), and for a post_w the
// same once more: grad_b = r1 (v - b r1^2 mean(v b)), v = z post_w.  A workgroup keeps its sums over its rows for the [d] gradients in
// registers, a value per column (PARTS); they are added up over the workgroups by a second kernel.
template <typename T, int WAVES, int CHUNKS, bool PARTS>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * kWave) void block_grad_kernel(const BlockArgs g) {
    constexpr int ROWS = WAVES == 1 ? 4 : 1, STEP = WAVES * kWave * 8;
    constexpr bool HOLD = CHUNKS == 1 || (WAVES == 8 && sizeof(T) == 2);
    __shared__ float s_sum[2 * 4 * WAVES];
    __shared__ float s_parts[PARTS && ROWS > 1 ? ROWS * kWave * 8 : 1];
    int turn = 0;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int c0 = ((WAVES == 1 ? 0 : wave * kWave) + lane) * 8, stride = gridDim.x * ROWS;
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
    int t = blockIdx.x * ROWS + (WAVES == 1 ? wave : 0);
    RowPart<T, CHUNKS> gy, gn, y, b;
    auto fetch = [&](int at) {
        const size_t row = (size_t)at * g.d;
        gy.load(g.grad_y, row, c0, STEP, g.d);
        gn.load(g.grad_n, row, c0, STEP, g.d);
        y.load(g.grad_n ? g.y : nullptr, row, c0, STEP, g.d);
        b.load(g.b, row, c0, STEP, g.d);
    };
    if (t < g.T) fetch(t);
    Columns<CHUNKS, HOLD> post_w, gate, open_w;
    post_w.begin(g.post_w, c0, STEP, g.d);
    gate.begin(g.gate, c0, STEP, g.d);
    open_w.begin(g.open_w, c0, STEP, g.d);
    for (; t < g.T; t += stride) {
        const size_t row = (size_t)t * g.d;
        const RowPart<T, CHUNKS> gy0 = gy, gn0 = gn, y0 = y, b0 = b;
        if (HOLD && t + stride < g.T) fetch(t + stride);
        float sum[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int q = 0; q < CHUNKS; ++q) {
            const Raw8<float> w = open_w.at(q, c0 + q * STEP, g.d);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float yi = at8(y0.v[q], i), bi = at8(b0.v[q], i);
                sum[0] = fmaf(yi, yi, sum[0]);
                sum[1] = fmaf(at8(gn0.v[q], i) * at8(w, i), yi, sum[1]);
                sum[2] = fmaf(bi, bi, sum[2]);
            }
        }
        if (g.grad_n || g.post_w) row_sums<WAVES>(sum, s_sum, turn);
        const float r2 = rsqrtf(fmaf(sum[0], g.inv_d, g.eps)), r1 = g.post_w ? rsqrtf(fmaf(sum[2], g.inv_d, g.eps)) : 1.f;
        const float m2 = sum[1] * g.inv_d * r2 * r2;
        const float tg = g.token_gate ? g.token_gate[t] : 1.f, x_scale = g.b ? g.skip_scale : 1.f;
        float dots[2] = {0.f, 0.f};  // <v, b>; the token gate's gradient
        float v[CHUNKS][8];
#pragma unroll
        for (int q = 0; q < CHUNKS; ++q) {
            const int c = c0 + q * STEP;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[q][i] = 0.f;
            if (c >= g.d) continue;
            float G[8], o[8];
            const Raw8<float> w = open_w.at(q, c, g.d);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                G[i] = at8(gy0.v[q], i);
                if (g.grad_n) {
                    const float yi = at8(y0.v[q], i), ni = at8(gn0.v[q], i);
                    G[i] += r2 * (ni * at8(w, i) - yi * m2);
                    if (PARTS) acc[0][q][i] = fmaf(ni, yi * r2, acc[0][q][i]);
                }
                o[i] = x_scale * G[i];
            }
            store8(static_cast<T*>(g.grad_x) + row + c, round8<T>(o));
            if (!g.b) continue;
            const unsigned kept = g.drop ? kept8(seed, offset, (row + c) >> 3, g.drop) : 0xFFu;
            const Raw8<float> pw = post_w.at(q, c, g.d), gt = gate.at(q, c, g.d);
            const float scale = g.block_scale * g.keep_scale;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool on = kept >> i & 1u;  // (what is dropped has no part, not even where it is infinite)
                const float bi = at8(b0.v[q], i), up = on ? G[i] * scale : 0.f, norm = on ? bi * r1 : 0.f;
                const float bare = up * (norm * at8(pw, i)), z = up * (tg * at8(gt, i));
                dots[1] = fmaf(bare, at8(gt, i), dots[1]);
                if (PARTS) {
                    acc[1][q][i] = fmaf(z, norm, acc[1][q][i]);
                    acc[2][q][i] = fmaf(bare, tg, acc[2][q][i]);
                }
                v[q][i] = z * at8(pw, i);
                if (g.post_w) dots[0] = fmaf(v[q][i], bi, dots[0]);
            }
        }
        if (g.b) {
            if (g.post_w || g.grad_token_gate) row_sums<WAVES>(dots, s_sum, turn);
            const float m1 = g.post_w ? dots[0] * g.inv_d * r1 * r1 : 0.f;
#pragma unroll
            for (int q = 0; q < CHUNKS; ++q) {
                const int c = c0 + q * STEP;
                if (c >= g.d) continue;
                float o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = g.post_w ? r1 * (v[q][i] - at8(b0.v[q], i) * m1) : v[q][i];
                store8(static_cast<T*>(g.grad_b) + row + c, round8<T>(o));
            }
            if (g.grad_token_gate && lane == 0 && (WAVES == 1 || wave == 0)) g.grad_token_gate[t] = dots[1];
        }
        if (!HOLD && t + stride < g.T) fetch(t + stride);
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
    // (eight loads in flight: one after the other, 512 parts of 2048 took 10.8 us)
    float f = 0.f;
    if (c < d) {
        const float* const p = parts + (size_t)k * d + c;
        const size_t pitch = (size_t)3 * d;
        int i = wave;
        for (; i + 7 * 16 < n; i += 8 * 16) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = p[(size_t)(i + j * 16) * pitch];
#pragma unroll
            for (int j = 0; j < 8; ++j) f += v[j];
        }
        for (; i < n; i += 16) f += p[(size_t)i * pitch];
    }
    s_sum[wave][lane] = f;
    __syncthreads();
    if (wave == 0 && c < d) {
        f = 0.f;
#pragma unroll
        for (int w = 0; w < 16; ++w) f += s_sum[w][lane];
        out[c] = f;
    }
}

template <typename F>
int by_plan(RowPlan p, F run) {
    typedef std::integral_constant<int, 1> c1;
    typedef std::integral_constant<int, 2> c2;
    typedef std::integral_constant<int, 3> c3;
    typedef std::integral_constant<int, 4> c4;
    typedef std::integral_constant<int, 8> c8;
    typedef std::integral_constant<int, 16> c16;
    switch (p.waves) {
        case 1: return run(c1{}, c1{});
        case 2: return run(c2{}, c1{});
        case 3: return run(c3{}, c1{});
        case 4: return run(c4{}, c1{});
        case 8: return p.chunks == 1 ? run(c8{}, c1{}) : run(c8{}, c2{});
        default: return p.chunks == 2 ? run(c16{}, c2{}) : p.chunks == 3 ? run(c16{}, c3{}) : run(c16{}, c4{});
    }
}

template <typename T>
int run_forward(const BlockArgs& g, hipStream_t st) {
    return by_plan(row_plan(g.d), [&](auto waves, auto chunks) {
        constexpr int W = decltype(waves)::value;
        hipLaunchKernelGGL((block_norm_kernel<T, W, decltype(chunks)::value>), dim3(std::min(kGroups, row_groups(g.T, g.d))), dim3(W == 1 ? 256 : W * kWave), 0,
                           st, g);
        return launch_status();
    });
}
template <typename T>
int run_backward(const BlockArgs& g, float* open_w, float* post_w, float* gate, hipStream_t st) {
    const int groups = g.parts ? grad_groups(g.T, g.d) : std::min(kGroups, row_groups(g.T, g.d));
    const int rc = by_plan(row_plan(g.d), [&](auto waves, auto chunks) {
        constexpr int W = decltype(waves)::value, C = decltype(chunks)::value;
        const auto kern = g.parts ? block_grad_kernel<T, W, C, true> : block_grad_kernel<T, W, C, false>;
        hipLaunchKernelGGL(kern, dim3(groups), dim3(W == 1 ? 256 : W * kWave), 0, st, g);
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
    return round_up(sizeof(float) * 3 * (size_t)d_model * (size_t)std::min(most_grad_groups(d_model), n_tokens + 1), 256);
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
