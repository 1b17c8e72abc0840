// Tokens to rows sorted by expert and back, with weights, and the gradients of both (moe_training.h states them).
//
// All four move rows and little else: what bounds them is memory, or the launch.  A token's row is read once for all of its pairs, or
// written once from all of them, 16 bytes a lane; dot products for the weights are formed from the values that pass by.
// 16384 tokens of 2048, two of 8 experts, bf16, in a graph: dispatch 36.8 us (196 MB, 5.3 TB/s), collect 29.5 (201 MB, 6.8 TB/s, part of it from the
// memory-side cache), its gradient 63-66 (336 MB, 5.1-5.3 TB/s); a copy of 1 GiB moves 5.1 TB/s both ways together.
#include <algorithm>

#include "moe_training.h"
#include "rows8.h"
#include "rows_plan.h"

namespace moe {

namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / kWave;

__device__ __forceinline__ int live_key(const int32_t* keys, int p, int end, int E) {  // the pair's expert; E: it has none
    const int key = p < end ? keys[p] : E;
    return (unsigned)key < (unsigned)E ? key : E;
}

// counts [chunks][E]: live pairs of each expert in each chunk
__global__ __launch_bounds__(kThreads) void dispatch_count_kernel(const int32_t* __restrict__ keys, int P, int E, int chunk,
                                                                  int32_t* __restrict__ counts) {
    __shared__ int s_count[kWaves][kMaxExperts + 1];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
    s_count[wave][lane] = 0;
    const int p0 = blockIdx.x * chunk, p1 = min(P, p0 + chunk);
    for (int p = p0 + (int)threadIdx.x; p < p1; p += kThreads) atomicAdd(&s_count[wave][live_key(keys, p, p1, E)], 1);
    __syncthreads();
    if ((int)threadIdx.x < E) {
        int n = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) n += s_count[w][threadIdx.x];
        counts[blockIdx.x * E + threadIdx.x] = n;
    }
}

// One workgroup a chunk: where its pairs go, then their rows.  A pair's row is its group's start, the group's pairs of earlier
// chunks, and those before it in the chunk; the last by ballots, so that order by pair is kept.
template <typename T>
__global__ __launch_bounds__(kThreads) void dispatch_kernel(ptr_arg a_keys, ptr_arg a_counts, int n_tokens, int E, int k, int d, int chunk_tokens, ptr_arg a_x,
                                                            ptr_arg a_weight, ptr_arg a_offsets, ptr_arg a_perm, ptr_arg a_inv, ptr_arg a_rows) {
    const int32_t *const __restrict__ keys = from_arg<const int32_t>(a_keys), *const __restrict__ counts = from_arg<const int32_t>(a_counts);
    const float* const __restrict__ weight = from_arg<const float>(a_weight);
    const T* const __restrict__ x = from_arg<const T>(a_x);
    T* const __restrict__ x_perm = from_arg<T>(a_rows);
    int32_t *const __restrict__ offsets = from_arg<int32_t>(a_offsets), *const __restrict__ perm = from_arg<int32_t>(a_perm),
                               *const __restrict__ inv_perm = from_arg<int32_t>(a_inv);
    __shared__ int s_all[kMaxExperts + 1], s_run[kMaxExperts + 1];  // of each expert: pairs, the next row
    __shared__ int s_wave[kWaves][kMaxExperts + 1];
    __shared__ int s_row[kThreads];
    __shared__ int s_live;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
    const int P = n_tokens * k, chunk = chunk_tokens * k;
    const int p0 = min((long long)P, (long long)blockIdx.x * chunk), p1 = min((long long)P, (long long)p0 + chunk);
    for (int i = threadIdx.x; i <= E; i += kThreads) s_all[i] = s_run[i] = 0;
    __syncthreads();
    if (counts) {
        // (a thread sums chunks of one expert and adds once: an addition in LDS for every count was 10 us of 64 experts)
        const int per = kThreads / E, c0 = quick_div(threadIdx.x, E), e = (int)threadIdx.x - c0 * E;
        if (c0 < per) {
            int all = 0, before = 0;
            for (int c = c0; c < (int)gridDim.x; c += 8 * per) {  // eight loads in flight
                int v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = c + j * per < (int)gridDim.x ? counts[(c + j * per) * E + e] : 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    all += v[j];
                    before += c + j * per < (int)blockIdx.x ? v[j] : 0;
                }
            }
            atomicAdd(&s_all[e], all);
            atomicAdd(&s_run[e], before);
        }
    } else if (E <= kBallotExperts) {  // lane e counts expert e
        int all = 0, before = 0;
        for (int q = wave * kWave; q < P; q += kThreads) {
            const int key = live_key(keys, q + lane, P, E);
            const unsigned long long early = q + kWave <= p0 ? ~0ull : q >= p0 ? 0ull : (1ull << (p0 - q)) - 1ull;
            for (int e = 0; e < E; ++e) {
                const unsigned long long is = __ballot(key == e);
                all += lane == e ? __popcll(is) : 0;
                before += lane == e ? __popcll(is & early) : 0;
            }
        }
        if (lane < E) {
            atomicAdd(&s_all[lane], all);
            atomicAdd(&s_run[lane], before);
        }
    } else {
        for (int p = threadIdx.x; p < P; p += kThreads) {
            const int e = live_key(keys, p, P, E);
            atomicAdd(&s_all[e], 1);
            if (p < p0) atomicAdd(&s_run[e], 1);
        }
    }
    __syncthreads();
    if (wave == 0) {
        const int n = lane < E ? s_all[lane] : 0, upto = wave_scan(n);
        if (lane < E) {
            s_run[lane] += upto - n;
            if (blockIdx.x == 0) offsets[lane] = upto - n;
        }
        if (lane == E - 1) {
            s_live = upto;
            if (blockIdx.x == 0) offsets[E] = upto;
        }
    }
    __syncthreads();
    const int pass = kThreads / k * k;  // whole tokens (k <= 64)
    for (int q0 = p0; q0 < p1; q0 += pass) {
        for (int i = threadIdx.x; i < kWaves * (kMaxExperts + 1); i += kThreads) (&s_wave[0][0])[i] = 0;
        __syncthreads();
        const int q1 = min(p1, q0 + pass), p = q0 + (int)threadIdx.x;
        const int key = live_key(keys, p, q1, E);
        int rank = 0;
        unsigned long long pending = __ballot(key < E);
        while (pending) {
            const int one = __shfl(key, __ffsll((long long)pending) - 1, kWave);
            const unsigned long long same = __ballot(key == one);
            if (key == one) rank = __popcll(same & ((1ull << lane) - 1ull));
            if (lane == 0) s_wave[wave][one] = __popcll(same);
            pending &= ~same;
        }
        __syncthreads();
        int row = -1;
        if (key < E) {
            row = s_run[key] + rank;
            for (int w = 0; w < wave; ++w) row += s_wave[w][key];
            perm[row] = p;
        }
        if (p < q1) inv_perm[p] = row;
        s_row[threadIdx.x] = row;
        __syncthreads();
        if ((int)threadIdx.x < E) {
            int n = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) n += s_wave[w][threadIdx.x];
            s_run[threadIdx.x] += n;
        }
        const int tokens = (q1 - q0) / k;
        for (int t = wave; t < tokens; t += kWaves) {
            const T* src = x + ((size_t)(q0 / k) + t) * d;
            constexpr int AHEAD = 4;
            for (int c = lane * 8; c < d; c += kWave * 8 * AHEAD) {
                Raw8<T> v[AHEAD];
#pragma unroll
                for (int a = 0; a < AHEAD; ++a)
                    if (c + a * kWave * 8 < d) v[a] = load8(src + c + a * kWave * 8);
                for (int j = 0; j < k; ++j) {
                    const int s = s_row[t * k + j];
                    if (s < 0) continue;
                    T* dst = x_perm + (size_t)s * d;
                    const float w = weight ? weight[q0 + t * k + j] : 1.f;
#pragma unroll
                    for (int a = 0; a < AHEAD; ++a) {
                        const int at = c + a * kWave * 8;
                        if (at >= d) continue;
                        if (weight) {
                            float f[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) f[i] = w * at8(v[a], i);
                            store8(dst + at, round8<T>(f));
                        } else {
                            store8(dst + at, v[a]);
                        }
                    }
                }
            }
        }
        __syncthreads();
    }
    // rows of no pair
    const float zero[8] = {};
    for (int s = s_live + blockIdx.x * kWaves + wave; s < P; s += gridDim.x * kWaves) {
        if (lane == 0) perm[s] = -1;
        for (int c = lane * 8; c < d; c += kWave * 8) store8(x_perm + (size_t)s * d + c, round8<T>(zero));
    }
}

// ---- rows to tokens --------------------------------------------------------------------------------------
// WAVES of a workgroup of four share a token, by its width.  K: pairs of a token held in registers, 0: any number, their dot
// products in LDS.
template <int WAVES, int K>
struct Dots {
    float* lds;   // [k][64] of this wave (K == 0)
    float v[K ? K : 1];
    __device__ __forceinline__ void clear(int k, int lane) {
        if constexpr (K > 0) {
#pragma unroll
            for (int j = 0; j < K; ++j) v[j] = 0.f;
        } else {
            for (int j = 0; j < k; ++j) lds[j * kWave + lane] = 0.f;
        }
    }
    __device__ __forceinline__ void add(int j, int lane, float f) {
        if constexpr (K > 0) v[j] += f;
        else lds[j * kWave + lane] += f;
    }
    // out[j] for j < k from the sums of all of the token's waves; s_part [4][64]
    __device__ __forceinline__ void finish(int k, int lane, int wave, float (*s_part)[kWave], float* out, bool valid) {
        auto one = [&](int j, float f) {
            f = wave_sum(f);
            if (WAVES == 1) {
                if (lane == 0 && valid) out[j] = f;
            } else if (lane == 0) {
                s_part[wave][j] = f;
            }
        };
        if constexpr (K > 0) {
#pragma unroll
            for (int j = 0; j < K; ++j)
                if (j < k) one(j, v[j]);
        } else {
            for (int j = 0; j < k; ++j) one(j, lds[j * kWave + lane]);
        }
        if (WAVES > 1) {
            __syncthreads();
            if (wave % WAVES == 0 && lane < k && valid) {
                f32x4 sum{};
#pragma unroll
                for (int w = 0; w < WAVES; ++w) sum[w] = s_part[wave + w][lane];
                out[lane] = (sum[0] + sum[1]) + (sum[2] + sum[3]);
            }
        }
    }
};

// out[t] = sum_j w[t,j] rows[inv[t,j]] (+ residual[t]); dots[t,j] = <x[t], rows[inv[t,j]]>
template <typename T, int WAVES, int K, bool DOTS>
__global__ __launch_bounds__(256) void collect_kernel(ptr_arg a_inv, ptr_arg a_weight, ptr_arg a_rows, int n_tokens, int k, int d, int P, ptr_arg a_residual,
                                                      ptr_arg a_x, ptr_arg a_out, ptr_arg a_dots) {
    const T *const __restrict__ rows = from_arg<const T>(a_rows), *const __restrict__ residual = from_arg<const T>(a_residual),
                               *const __restrict__ x = from_arg<const T>(a_x);
    const int32_t* const __restrict__ inv_perm = from_arg<const int32_t>(a_inv);
    const float* const __restrict__ weight = from_arg<const float>(a_weight);
    T* const __restrict__ out = from_arg<T>(a_out);
    float* const __restrict__ dots = from_arg<float>(a_dots);
    extern __shared__ float s_dots[];
    __shared__ float s_part[4][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int t = blockIdx.x * (4 / WAVES) + wave / WAVES;
    const bool valid = t < n_tokens;
    if (WAVES == 1 && !valid) return;
    if (!valid) d = 0;  // (the waves of a token that is not there come to the barrier)
    Dots<WAVES, K> dot;
    dot.lds = s_dots + wave * k * kWave;
    if (DOTS) dot.clear(k, lane);
    const int32_t* const inv = inv_perm + (size_t)t * k;
    const float* const w = weight ? weight + (size_t)t * k : nullptr;
    int row[K ? K : 1];
    float g[K ? K : 1];
#pragma unroll
    for (int j = 0; j < K; ++j) {
        row[j] = j < k && valid ? inv[j] : -1;
        g[j] = j < k && valid && w ? w[j] : 1.f;
        if ((unsigned)row[j] >= (unsigned)P) row[j] = -1;
    }
    for (int c = (wave % WAVES * kWave + lane) * 8; c < d; c += WAVES * kWave * 8) {
        float acc[8];
        Raw8<T> xv{}, res{};
        if (DOTS) xv = load8(x + (size_t)t * d + c);
        if (residual) res = load8(residual + (size_t)t * d + c);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = 0.f;
        auto pair = [&](int j, float f, const Raw8<T>& v) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                acc[i] = fmaf(f, at8(v, i), acc[i]);
                if (DOTS) s = fmaf(at8(xv, i), at8(v, i), s);
            }
            if (DOTS) dot.add(j, lane, s);
        };
        if constexpr (K > 0) {
            Raw8<T> v[K];
#pragma unroll
            for (int j = 0; j < K; ++j)
                if (row[j] >= 0) v[j] = load8(rows + (size_t)row[j] * d + c);
#pragma unroll
            for (int j = 0; j < K; ++j)
                if (row[j] >= 0) pair(j, g[j], v[j]);
        } else {
            for (int j = 0; j < k; ++j) {
                const int s = inv[j];
                if ((unsigned)s < (unsigned)P) pair(j, w ? w[j] : 1.f, load8(rows + (size_t)s * d + c));
            }
        }
        if (residual) {
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] += at8(res, i);
        }
        store8(out + (size_t)t * d + c, round8<T>(acc));
    }
    if (DOTS) dot.finish(k, lane, wave, s_part, dots + (size_t)t * k, valid);
}

// grad_rows[inv[t,j]] = gate[t,j] gy[t]; dots[t,j] = <gy[t], rows[inv[t,j]]>.  Rows of no pair are cleared by all workgroups together.
template <typename T, int WAVES, int K, bool DOTS, bool ROWS>
__global__ __launch_bounds__(256) void spread_kernel(ptr_arg a_inv, ptr_arg a_gate, ptr_arg a_gy, int n_tokens, int E, int k, int d, int P, ptr_arg a_rows,
                                                     ptr_arg a_offsets, ptr_arg a_grad, ptr_arg a_dots) {
    const T* const __restrict__ gy = from_arg<const T>(a_gy);
    const T* const rows = from_arg<const T>(a_rows);  // (may be the output)
    T* const grad_rows = from_arg<T>(a_grad);
    const int32_t *const __restrict__ inv_perm = from_arg<const int32_t>(a_inv), *const __restrict__ offsets = from_arg<const int32_t>(a_offsets);
    const float* const __restrict__ gate = from_arg<const float>(a_gate);
    float* const __restrict__ dots = from_arg<float>(a_dots);
    extern __shared__ float s_dots[];
    __shared__ float s_part[4][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int t = blockIdx.x * (4 / WAVES) + wave / WAVES;
    const bool valid = t < n_tokens;
    if (ROWS) {
        const float zero[8] = {};
        for (int s = max(offsets[E], 0) + (int)blockIdx.x * 4 + wave; s < P; s += gridDim.x * 4)
            for (int c = lane * 8; c < d; c += kWave * 8) store8(grad_rows + (size_t)s * d + c, round8<T>(zero));
    }
    if (WAVES == 1 && !valid) return;
    if (!valid) d = 0;
    Dots<WAVES, K> dot;
    dot.lds = s_dots + wave * k * kWave;
    if (DOTS) dot.clear(k, lane);
    const int32_t* const inv = inv_perm + (size_t)t * k;
    const float* const w = ROWS ? gate + (size_t)t * k : nullptr;
    int row[K ? K : 1];
    float g[K ? K : 1];
#pragma unroll
    for (int j = 0; j < K; ++j) {
        row[j] = j < k && valid ? inv[j] : -1;
        g[j] = ROWS && valid && j < k ? w[j] : 0.f;
        if ((unsigned)row[j] >= (unsigned)P) row[j] = -1;
    }
    for (int c = (wave % WAVES * kWave + lane) * 8; c < d; c += WAVES * kWave * 8) {
        const Raw8<T> up = load8(gy + (size_t)t * d + c);
        auto pair = [&](int j, int s, float f, const Raw8<T>& v) {
            float sum = 0.f, o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (DOTS) sum = fmaf(at8(up, i), at8(v, i), sum);
                o[i] = f * at8(up, i);
            }
            if (DOTS) dot.add(j, lane, sum);
            if (ROWS) store8(grad_rows + (size_t)s * d + c, round8<T>(o));
        };
        if constexpr (K > 0) {
            Raw8<T> v[K];
#pragma unroll
            for (int j = 0; j < K; ++j)
                if (DOTS && row[j] >= 0) v[j] = load8(rows + (size_t)row[j] * d + c);
#pragma unroll
            for (int j = 0; j < K; ++j)
                if (row[j] >= 0) pair(j, row[j], g[j], v[j]);
        } else {
            for (int j = 0; j < k; ++j) {
                const int s = inv[j];
                if ((unsigned)s >= (unsigned)P) continue;
                Raw8<T> v{};
                if (DOTS) v = load8(rows + (size_t)s * d + c);
                pair(j, s, ROWS ? w[j] : 0.f, v);
            }
        }
    }
    if (DOTS) dot.finish(k, lane, wave, s_part, dots + (size_t)t * k, valid);
}

constexpr size_t kDotsLds = sizeof(float) * 4 * kWave * kMaxExperts;  // dot products of 64 pairs, a sum per lane

template <typename F>
int by_size(int d, int k, F run) {
    const RowsForm form = rows_form(d, k);
    auto on = [&](auto waves) {
        switch (form.pairs) {
            case 1: return run(waves, std::integral_constant<int, 1>{});
            case 2: return run(waves, std::integral_constant<int, 2>{});
            case 4: return run(waves, std::integral_constant<int, 4>{});
            case 8: return run(waves, std::integral_constant<int, 8>{});
            default: return run(waves, std::integral_constant<int, 0>{});
        }
    };
    switch (form.waves) {
        case 1: return on(std::integral_constant<int, 1>{});
        case 2: return on(std::integral_constant<int, 2>{});
        default: return on(std::integral_constant<int, 4>{});
    }
}

template <typename T>
int run_collect(const moe_shape& s, const void* rows, const int32_t* inv, const float* weight, const void* residual, const void* x, void* out,
                float* dots, hipStream_t st) {
    return by_size(s.d_model, s.top_k, [&](auto waves, auto kk) {
        constexpr int W = decltype(waves)::value, K = decltype(kk)::value;
        const int grid = (s.n_tokens + 4 / W - 1) / (4 / W);
        const size_t lds = K == 0 && dots ? sizeof(float) * 4 * kWave * s.top_k : 0;
        const auto kern = dots ? collect_kernel<T, W, K, true> : collect_kernel<T, W, K, false>;
        static std::atomic<uint64_t> lds_allowed;
        if (lds && allow_dynamic_lds(reinterpret_cast<const void*>(kern), kDotsLds, lds_allowed) != MOE_OK) return (int)MOE_ERR_LAUNCH;
        hipLaunchKernelGGL(kern, dim3(grid), dim3(256), lds, st, as_arg(inv), as_arg(weight), as_arg(rows), s.n_tokens, s.top_k, s.d_model,
                           s.n_tokens * s.top_k, as_arg(residual), as_arg(x), as_arg(out), as_arg(dots));
        return launch_status();
    });
}

template <typename T>
int run_spread(const moe_shape& s, const void* gy, const void* rows, const int32_t* offsets, const int32_t* inv, const float* gate, void* grad_rows,
               float* dots, hipStream_t st) {
    const int P = s.n_tokens * s.top_k;
    return by_size(s.d_model, s.top_k, [&](auto waves, auto kk) {
        constexpr int W = decltype(waves)::value, K = decltype(kk)::value;
        const int grid = (s.n_tokens + 4 / W - 1) / (4 / W);
        const size_t lds = K == 0 && dots ? sizeof(float) * 4 * kWave * s.top_k : 0;
        const auto kern = !grad_rows ? spread_kernel<T, W, K, true, false> : dots ? spread_kernel<T, W, K, true, true> : spread_kernel<T, W, K, false, true>;
        static std::atomic<uint64_t> lds_allowed[2];
        if (lds && allow_dynamic_lds(reinterpret_cast<const void*>(kern), kDotsLds, lds_allowed[grad_rows != nullptr]) != MOE_OK) return (int)MOE_ERR_LAUNCH;
        hipLaunchKernelGGL(kern, dim3(grid), dim3(256), lds, st, as_arg(inv), as_arg(gate), as_arg(gy), s.n_tokens, s.n_experts, s.top_k, s.d_model, P,
                           as_arg(rows), as_arg(offsets), as_arg(grad_rows), as_arg(dots));
        return launch_status();
    });
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace

size_t dispatch_scratch_bytes(long long T, int E) {
    // (the most chunks that any number of tokens up to this one has: a workspace for more tokens holds fewer)
    const long long most = std::min(512, kMaxCounts / E);
    return sizeof(int32_t) * (size_t)std::min<long long>(most, T / 4 + 1) * E;
}

}  // namespace moe

using namespace moe;

extern "C" size_t moe_dispatch_workspace_bytes(const moe_shape* shape) {
    return validate_shape(shape) == MOE_OK ? round_up(dispatch_scratch_bytes(shape->n_tokens, shape->n_experts), 256) : 0;
}

extern "C" int moe_dispatch(const moe_shape* shape, const int32_t* topk_idx, const float* weight, const void* x, int32_t* expert_offsets,
                            int32_t* perm, int32_t* inv_perm, void* x_perm, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = validate_shape(shape);
    if (rc != MOE_OK) return rc;
    const moe_shape& s = *shape;
    if (!expert_offsets || !aligned4(expert_offsets)) return MOE_ERR_INVALID;
    if (s.n_tokens > 0) {
        if (!topk_idx || !x || !perm || !inv_perm || !x_perm || x == x_perm || !aligned16(x) || !aligned16(x_perm)) return MOE_ERR_INVALID;
        for (const void* p : {(const void*)topk_idx, (const void*)weight, (const void*)perm, (const void*)inv_perm})
            if (!aligned4(p)) return MOE_ERR_INVALID;
    }
    const int P = s.n_tokens * s.top_k;
    const DispatchPlan plan = dispatch_plan(s.n_tokens, s.n_experts);
    int32_t* counts = nullptr;
    if (dispatch_count(P, s.n_experts) == COUNT_LAUNCH) {
        if (!workspace || workspace_bytes < dispatch_scratch_bytes(s.n_tokens, s.n_experts)) return MOE_ERR_WORKSPACE;
        if (!aligned4(workspace)) return MOE_ERR_INVALID;
        counts = static_cast<int32_t*>(workspace);
    }
    hipStream_t st = as_stream(stream);
    if (counts) {
        hipLaunchKernelGGL(dispatch_count_kernel, dim3(plan.chunks), dim3(kThreads), 0, st, topk_idx, P, s.n_experts, plan.tokens * s.top_k, counts);
        if ((rc = launch_status()) != MOE_OK) return rc;
    }
    const int grid = std::max(plan.chunks, 1);
    hipLaunchKernelGGL(s.act_dtype == MOE_F32 ? dispatch_kernel<float> : dispatch_kernel<bf16_t>, dim3(grid), dim3(kThreads), 0, st, as_arg(topk_idx),
                       as_arg(counts), s.n_tokens, s.n_experts, s.top_k, s.d_model, plan.tokens, as_arg(x), as_arg(weight), as_arg(expert_offsets),
                       as_arg(perm), as_arg(inv_perm), as_arg(x_perm));
    return launch_status();
}

extern "C" int moe_dispatch_backward(const moe_shape* shape, const void* grad_x_perm, const int32_t* inv_perm, const void* x, const float* weight,
                                     void* grad_x, float* grad_weight, void* stream) {
    const int rc = validate_shape(shape);
    if (rc != MOE_OK || shape->n_tokens == 0) return rc;
    if (!grad_x_perm || !inv_perm || !grad_x || grad_x == grad_x_perm || (grad_weight && !x) || (x && x == grad_x)) return MOE_ERR_INVALID;
    for (const void* p : {grad_x_perm, x, (const void*)grad_x})
        if (!aligned16(p)) return MOE_ERR_INVALID;
    for (const void* p : {(const void*)inv_perm, (const void*)weight, (const void*)grad_weight})
        if (!aligned4(p)) return MOE_ERR_INVALID;
    const auto run = shape->act_dtype == MOE_F32 ? run_collect<float> : run_collect<bf16_t>;
    return run(*shape, grad_x_perm, inv_perm, weight, nullptr, x, grad_x, grad_weight, as_stream(stream));
}

extern "C" int moe_collect(const moe_shape* shape, const void* y_perm, const int32_t* inv_perm, const float* topk_gate, const void* residual, void* y,
                           void* stream) {
    const int rc = validate_shape(shape);
    if (rc != MOE_OK || shape->n_tokens == 0) return rc;
    if (!y_perm || !inv_perm || !topk_gate || !y || y == y_perm || y == residual) return MOE_ERR_INVALID;
    for (const void* p : {y_perm, residual, (const void*)y})
        if (!aligned16(p)) return MOE_ERR_INVALID;
    if (!aligned4(inv_perm) || !aligned4(topk_gate)) return MOE_ERR_INVALID;
    const auto run = shape->act_dtype == MOE_F32 ? run_collect<float> : run_collect<bf16_t>;
    return run(*shape, y_perm, inv_perm, topk_gate, residual, nullptr, y, nullptr, as_stream(stream));
}

extern "C" int moe_collect_backward(const moe_shape* shape, const void* grad_y, const void* y_perm, const int32_t* expert_offsets,
                                    const int32_t* inv_perm, const float* topk_gate, void* grad_y_perm, float* grad_gate, void* stream) {
    const int rc = validate_shape(shape);
    if (rc != MOE_OK || shape->n_tokens == 0) return rc;
    if (!grad_y || !inv_perm || (grad_gate && !y_perm) || (grad_y_perm && (!topk_gate || !expert_offsets))) return MOE_ERR_INVALID;
    if (grad_y_perm == grad_y) return MOE_ERR_INVALID;
    for (const void* p : {grad_y, y_perm, (const void*)grad_y_perm})
        if (!aligned16(p)) return MOE_ERR_INVALID;
    for (const void* p : {(const void*)expert_offsets, (const void*)inv_perm, (const void*)topk_gate, (const void*)grad_gate})
        if (!aligned4(p)) return MOE_ERR_INVALID;
    if (!grad_y_perm && !grad_gate) return MOE_OK;
    const auto run = shape->act_dtype == MOE_F32 ? run_spread<float> : run_spread<bf16_t>;
    return run(*shape, grad_y, y_perm, expert_offsets, inv_perm, topk_gate, grad_y_perm, grad_gate, as_stream(stream));
}
