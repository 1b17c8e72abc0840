// Routing from logits: scores by softmax or sigmoid, picks by score and bias inside the best groups, gates; and
// the gradient of gates and scores with regard to the logits.  moe.h states the definition.
//
// A wave holds a token's row, expert 64 v + lane in value v of a lane.
#include <cmath>

#include "mxfp4.h"
#include "router.h"

namespace moe {

namespace {

constexpr int kWaves = 4;

// What the wave's lanes wrote to LDS is there for all of them
__device__ __forceinline__ void wave_lds() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ double shfl_xor_f64(double v, int m) { return __shfl_xor(v, m, kWave); }
__device__ __forceinline__ float shfl_xor_key(float v, int m) { return __shfl_xor(v, m, kWave); }
__device__ __forceinline__ double shfl_xor_key(double v, int m) { return __shfl_xor(v, m, kWave); }

template <typename F>
__device__ __forceinline__ F key_infinity() { return (F)INFINITY; }

// The best (value, lowest index) over a wave; v = -inf, i = INT_MAX: none
template <typename F>
__device__ __forceinline__ void wave_best(F& v, int& i) {
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) {
        const F ov = shfl_xor_key(v, m);
        const int oi = __shfl_xor(i, m, kWave);
        if (ov > v || (ov == v && oi < i)) v = ov, i = oi;
    }
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) v = fmaxf(v, __shfl_xor(v, m, kWave));
    return v;
}
__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) v += shfl_xor_f64(v, m);
    return v;
}

// F: the type of keys.  Without a bias the order of keys is that of the logits, which fp32 holds exactly, unless
// a group's rank is a sum; otherwise keys are formed and compared in 64 bits.
template <typename F, int V>
__global__ __launch_bounds__(kWaves* kWave) void route_scored_kernel(const float* __restrict__ logits, const float* __restrict__ bias,
                                                                     int32_t* __restrict__ topk_idx, float* __restrict__ topk_gate,
                                                                     float* __restrict__ scores, int T, int E, int k, int sigmoid, int G, int kept,
                                                                     int group_top, int renormalize, float scale) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t = blockIdx.x * kWaves + wave;
    __shared__ F s_key[kWaves][V * kWave];
    if (t >= T) return;  // (waves exchange nothing)
    const float* row = logits + (size_t)t * E;
    float l[V];
    float top = -INFINITY;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = v * kWave + lane;
        l[v] = e < E ? row[e] : -INFINITY;
        if (!(l[v] == l[v])) l[v] = -INFINITY;
        top = fmaxf(top, l[v]);
    }
    top = wave_max(top);
    const float base = top == -INFINITY ? 0.f : top;
    float s[V], den = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (sigmoid) {
            s[v] = 1.f / (1.f + expf(-l[v]));
        } else {
            s[v] = expf(l[v] - base);
            den += s[v];
        }
    }
    if (!sigmoid) {
        den = wave_sum(den);
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] = den > 0.f ? s[v] / den : 0.f;
    }
    if (scores) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (v * kWave + lane < E) scores[(size_t)t * E + v * kWave + lane] = s[v];
    }
    F key[V];
    if constexpr (sizeof(F) == 4) {
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = l[v];
    } else {
        double d64 = 0.0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const double z = l[v];
            key[v] = sigmoid ? 1.0 / (1.0 + exp(-z)) : exp(z - (double)base);
            d64 += l[v] == -INFINITY ? 0.0 : key[v];
        }
        if (!sigmoid) d64 = wave_sum64(d64);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = v * kWave + lane;
            const double b = bias && e < E ? (double)bias[e] : 0.0;
            key[v] = l[v] == -INFINITY ? -key_infinity<double>() : (sigmoid ? key[v] : key[v] / d64) + b;
            if (!(key[v] == key[v])) key[v] = -key_infinity<double>();  // (of a logit of infinity: every comparison has an answer)
        }
    }
    // groups: lane g ranks group g
    unsigned long long open = ~0ull;
    const int per = E / G;
    if (G > 1) {
#pragma unroll
        for (int v = 0; v < V; ++v) s_key[wave][v * kWave + lane] = key[v];
        wave_lds();
        F a = -key_infinity<F>(), b = -key_infinity<F>();
        if (lane < G) {
            for (int i = 0; i < per; ++i) {
                const F x = s_key[wave][lane * per + i];
                if (x > a) b = a, a = x;
                else if (x > b) b = x;
            }
        }
        F rank = group_top == 2 && b > -key_infinity<F>() ? a + b : a;
        open = 0;
        bool taken = lane >= G;
        for (int j = 0; j < kept; ++j) {
            F bv = taken ? -key_infinity<F>() : rank;
            int bi = taken ? 0x7fffffff : lane;
            wave_best(bv, bi);
            open |= 1ull << bi;
            if (lane == bi) taken = true;
        }
    }
    // state of a value: 0 open, 1 switched off (or taken: 2), 2 not to be picked
    int state[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = v * kWave + lane;
        const int g = G > 1 ? min(e / per, G - 1) : 0;
        state[v] = e >= E || !(open >> g & 1) ? 2 : key[v] == -key_infinity<F>() ? 1 : 0;
    }
    float my_l = 0.f;  // logit and expert of pick `lane`
    int my_e = 0;
    float my_s = 0.f;
    bool my_off = true;
    for (int j = 0; j < k; ++j) {
        F bv = -key_infinity<F>();
        int bi = 0x7fffffff;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = v * kWave + lane;
            if (state[v] == 0 && (key[v] > bv || bi == 0x7fffffff)) bv = key[v], bi = e;
        }
        wave_best(bv, bi);
        if (bi == 0x7fffffff) {  // none but switched-off ones: the lowest
#pragma unroll
            for (int v = V - 1; v >= 0; --v)
                if (state[v] == 1) bi = v * kWave + lane;
#pragma unroll
            for (int m = 1; m < kWave; m <<= 1) bi = min(bi, __shfl_xor(bi, m, kWave));
        }
        float pl = 0.f, ps = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (bi == v * kWave + lane) state[v] = 2, pl = l[v], ps = s[v];
        pl = __shfl(pl, bi & 63, kWave);
        ps = __shfl(ps, bi & 63, kWave);
        if (lane == j) my_e = bi, my_l = pl, my_s = ps, my_off = pl == -INFINITY;
    }
    if (renormalize) {
        // relative to the largest picked score, so that rows of tiny scores keep their shares
        const float big = wave_max(lane < k && !my_off ? my_l : -INFINITY);
        const float m = big == -INFINITY ? 0.f : sigmoid ? fminf(big, 0.f) : big;
        float w = 0.f;
        if (lane < k && !my_off) w = !sigmoid ? expf(my_l - m) : my_l >= 0.f ? 1.f / (1.f + expf(-my_l)) : expf(my_l - m) / (1.f + expf(my_l));
        const float total = wave_sum(w);
        my_s = total > 0.f ? w / total : 0.f;
    }
    if (lane < k) {
        topk_idx[(size_t)t * k + lane] = my_e;
        topk_gate[(size_t)t * k + lane] = my_s * scale;
    }
}

template <int V>
__global__ __launch_bounds__(kWaves* kWave) void route_scored_backward_kernel(const float* __restrict__ logits, const int32_t* __restrict__ topk_idx,
                                                                              const float* __restrict__ grad_gate, const float* __restrict__ grad_scores,
                                                                              float* __restrict__ grad_logits, int T, int E, int k, int sigmoid,
                                                                              int renormalize, float scale) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t = blockIdx.x * kWaves + wave;
    __shared__ float s_ds[kWaves][V * kWave];
    if (t >= T) return;
    const float* row = logits + (size_t)t * E;
    float l[V], ds[V];
    float top = -INFINITY;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = v * kWave + lane;
        l[v] = e < E ? row[e] : -INFINITY;
        ds[v] = e < E && grad_scores ? grad_scores[(size_t)t * E + e] : 0.f;
        if (!(l[v] == l[v])) l[v] = -INFINITY;
        top = fmaxf(top, l[v]);
        s_ds[wave][v * kWave + lane] = 0.f;
    }
    const int e_of = lane < k ? topk_idx[(size_t)t * k + lane] : -1;
    const bool named = lane < k && (unsigned)e_of < (unsigned)E;
    const float dg = named ? grad_gate[(size_t)t * k + lane] : 0.f;
    float pl = named ? row[e_of] : -INFINITY;
    if (!(pl == pl)) pl = -INFINITY;
    float s[V], den = 0.f;
    const float base = sigmoid ? 0.f : wave_max(top) == -INFINITY ? 0.f : wave_max(top);
#pragma unroll
    for (int v = 0; v < V; ++v) {
        s[v] = sigmoid ? 1.f / (1.f + expf(-l[v])) : expf(l[v] - base);
        den += s[v];
    }
    den = wave_sum(den);
    if (!sigmoid) {
#pragma unroll
        for (int v = 0; v < V; ++v) s[v] = den > 0.f ? s[v] / den : 0.f;
    }
    // d(loss)/d(logit) of the gates, but for the part that all logits of a softmax share
    float add;
    if (renormalize) {
        const float big = wave_max(pl);
        const float m = big == -INFINITY ? 0.f : sigmoid ? fminf(big, 0.f) : big;
        float w = 0.f;
        if (pl != -INFINITY) w = !sigmoid ? expf(pl - m) : pl >= 0.f ? 1.f / (1.f + expf(-pl)) : expf(pl - m) / (1.f + expf(pl));
        const float total = wave_sum(w);
        const float g = total > 0.f ? w / total : 0.f;
        const float mean = wave_sum(dg * g);
        add = scale * g * (dg - mean) * (sigmoid ? 1.f / (1.f + expf(pl)) : 1.f);
    } else {
        const float sp = sigmoid ? 1.f / (1.f + expf(-pl)) : den > 0.f ? expf(pl - base) / den : 0.f;
        add = scale * dg * sp * (sigmoid ? 1.f / (1.f + expf(pl)) : 1.f);
    }
    wave_lds();
    for (int j = 0; j < k; ++j) {  // (one after the other: an expert may be named twice)
        if (lane == j && named) s_ds[wave][e_of] += add;
        wave_lds();
    }
    float shared = 0.f;
    if (!sigmoid) {
        float part = renormalize || !named ? 0.f : add;
#pragma unroll
        for (int v = 0; v < V; ++v) part += ds[v] * s[v];
        shared = wave_sum(part);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = v * kWave + lane;
        if (e < E) {
            const float own = sigmoid ? ds[v] * s[v] * (l[v] == -INFINITY ? 0.f : 1.f / (1.f + expf(l[v]))) : s[v] * (ds[v] - shared);
            grad_logits[(size_t)t * E + e] = s_ds[wave][e] + own;
        }
    }
}

// Logits as moe_route sums them (router_logits: the same bits), of two tokens a workgroup
template <typename T>
__global__ __launch_bounds__(kRouteWaves* kWave) void router_logits_kernel(const T* __restrict__ x, const float* __restrict__ rw,
                                                                           const float* __restrict__ rb, int d, int E, int T_,
                                                                           float* __restrict__ logits) {
    typedef Store<T> S;
    constexpr int VEC = S::VEC;
    const int t0 = blockIdx.x * kRouteTok, ntok = min(kRouteTok, T_ - t0);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    auto load_x = [&](int t, int i, float* out) {
        const typename S::vec_t xv = *reinterpret_cast<const typename S::vec_t*>(x + (size_t)(t0 + t) * d + i);
#pragma unroll
        for (int q = 0; q < VEC; ++q) out[q] = S::get(xv, q);
    };
    for (int e = wave; e < E; e += kRouteWaves) {
        float acc[kRouteTok];
        const float b = rb ? rb[e] : 0.f;
        router_logits<VEC, kRouteTok, 4>(load_x, rw + (size_t)e * d, d, lane, ntok, acc);
#pragma unroll
        for (int t = 0; t < kRouteTok; ++t)
            if (lane == 0 && t < ntok) logits[(size_t)(t0 + t) * E + e] = acc[t] + b;
    }
}

// values a lane: a power of two
template <typename L>
int with_values(int E, L launch) {
    if (E <= 64) return launch(std::integral_constant<int, 1>{});
    if (E <= 128) return launch(std::integral_constant<int, 2>{});
    if (E <= 256) return launch(std::integral_constant<int, 4>{});
    return launch(std::integral_constant<int, 8>{});
}

}  // namespace

int validate_route(const moe_route_config* c, int T, int E, int k) {
    if (!c || T < 0 || E < 1 || k < 1 || k > E) return MOE_ERR_INVALID;
    if ((c->score != MOE_SCORE_SOFTMAX && c->score != MOE_SCORE_SIGMOID) || c->n_groups < 1 || c->groups_kept < 1 ||
        c->groups_kept > c->n_groups || c->renormalize < 0 || c->renormalize > 1 || !std::isfinite(c->scale))
        return MOE_ERR_INVALID;
    if (E % c->n_groups || c->group_top < 1 || c->group_top > 2 || c->group_top > E / c->n_groups) return MOE_ERR_INVALID;
    if ((long long)k > (long long)c->groups_kept * (E / c->n_groups)) return MOE_ERR_INVALID;
    if (E > MOE_ROUTE_MAX_EXPERTS || c->n_groups > kWave || k > kWave) return MOE_ERR_UNSUPPORTED;
    return MOE_OK;
}

int launch_route_scored(const moe_route_config& c, int T, int E, int k, const float* logits, const float* bias, int32_t* idx, float* gate,
                        float* scores, hipStream_t st) {
    if (T == 0) return MOE_OK;
    const bool by_logit = !bias && (c.n_groups == 1 || c.group_top == 1);
    return with_values(E, [&](auto V) {
        auto launch = [&](auto kern) {
            hipLaunchKernelGGL(kern, dim3((T + kWaves - 1) / kWaves), dim3(kWaves * kWave), 0, st, logits, bias, idx, gate, scores, T, E, k, c.score,
                               c.n_groups, c.groups_kept, c.group_top, c.renormalize, c.scale);
            return launch_status();
        };
        return by_logit ? launch(route_scored_kernel<float, V.value>) : launch(route_scored_kernel<double, V.value>);
    });
}

int launch_router_logits(const moe_shape& s, const void* x, const float* rw, const float* rb, float* logits, hipStream_t st) {
    const dim3 grid((s.n_tokens + kRouteTok - 1) / kRouteTok), block(kRouteWaves * kWave);
    if (s.act_dtype == MOE_F32)
        hipLaunchKernelGGL(router_logits_kernel<float>, grid, block, 0, st, (const float*)x, rw, rb, s.d_model, s.n_experts, s.n_tokens, logits);
    else
        hipLaunchKernelGGL(router_logits_kernel<bf16_t>, grid, block, 0, st, (const bf16_t*)x, rw, rb, s.d_model, s.n_experts, s.n_tokens, logits);
    return launch_status();
}

}  // namespace moe

using namespace moe;

static bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

extern "C" int moe_route_scored(const moe_route_config* config, int32_t n_tokens, int32_t n_experts, int32_t top_k, const float* logits,
                                const float* select_bias, int32_t* topk_idx, float* topk_gate, float* scores, void* stream) {
    const int rc = validate_route(config, n_tokens, n_experts, top_k);
    if (rc != MOE_OK || n_tokens == 0) return rc;
    if (!logits || !topk_idx || !topk_gate || !aligned4(logits) || !aligned4(select_bias) || !aligned4(topk_idx) || !aligned4(topk_gate) ||
        !aligned4(scores) || scores == logits)
        return MOE_ERR_INVALID;
    return launch_route_scored(*config, n_tokens, n_experts, top_k, logits, select_bias, topk_idx, topk_gate, scores, as_stream(stream));
}

extern "C" int moe_route_scored_backward(const moe_route_config* config, int32_t n_tokens, int32_t n_experts, int32_t top_k, const float* logits,
                                         const int32_t* topk_idx, const float* grad_gate, const float* grad_scores, float* grad_logits, void* stream) {
    const int rc = validate_route(config, n_tokens, n_experts, top_k);
    if (rc != MOE_OK || n_tokens == 0) return rc;
    if (!logits || !topk_idx || !grad_gate || !grad_logits || !aligned4(logits) || !aligned4(topk_idx) || !aligned4(grad_gate) ||
        !aligned4(grad_scores) || !aligned4(grad_logits) || grad_logits == logits || grad_logits == grad_scores)
        return MOE_ERR_INVALID;
    const moe_route_config& c = *config;
    return with_values(n_experts, [&](auto V) {
        hipLaunchKernelGGL(route_scored_backward_kernel<V.value>, dim3((n_tokens + kWaves - 1) / kWaves), dim3(kWaves * kWave), 0, as_stream(stream),
                           logits, topk_idx, grad_gate, grad_scores, grad_logits, n_tokens, n_experts, top_k, c.score, c.renormalize, c.scale);
        return launch_status();
    });
}
