// Routing from logits: scores by softmax or sigmoid, picks by score and bias inside the best groups, gates; and
// the gradient of gates and scores with regard to the logits.  moe_quantised.h states the definition.
#include <algorithm>
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
template <typename F>
__device__ __forceinline__ F key_infinity() { return (F)INFINITY; }

template <int CTRL>
__device__ __forceinline__ float dpp_any(float v) { return dpp_f32<CTRL>(v); }
template <int CTRL>
__device__ __forceinline__ int dpp_any(int v) { return dpp_i32<CTRL>(v); }
__device__ __forceinline__ bool aligned16_dev(const void* p) { return ((uintptr_t)p & 15u) == 0; }

template <int CTRL>
__device__ __forceinline__ long long dpp_any(long long v) {
    return (long long)dpp_i32<CTRL>((int)(v >> 32)) << 32 | (unsigned)dpp_i32<CTRL>((int)v);
}
__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, dpp_f32<kDppSwap1>(v));
    v = fmaxf(v, dpp_f32<kDppSwap2>(v));
    v = fmaxf(v, dpp_f32<kDppHalfMirror>(v));
    v = fmaxf(v, dpp_f32<kDppMirror>(v));
    v = fmaxf(v, __shfl_xor(v, 16, kWave));
    return fmaxf(v, __shfl_xor(v, 32, kWave));
}
__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) v += shfl_xor_f64(v, m);
    return v;
}

struct RouteArgs {
    const float *logits, *bias;
    int32_t* topk_idx;
    float *topk_gate, *scores;
    int T, E, k, sigmoid, G, kept, group_top, renormalize;
    float scale;
};

// A picked expert's score over the common factor of the row's: exp(m), m the largest picked logit (sigmoid: at most 0), so that rows
// of tiny scores keep their shares
__device__ __forceinline__ float pick_weight(float l, float m, int sigmoid) {
    return !sigmoid ? expf(l - m) : l >= 0.f ? 1.f / (1.f + expf(-l)) : expf(l - m) / (1.f + expf(l));
}

// Largest of a whole number of every lane, in all lanes: rows of 16 by register exchanges, the four rows through scalar registers
__device__ __forceinline__ long long wave_largest(long long v) {
    auto take = [&](long long o) { v = o > v ? o : v; };
    take(dpp_any<kDppSwap1>(v));
    take(dpp_any<kDppSwap2>(v));
    take(dpp_any<kDppHalfMirror>(v));
    take(dpp_any<kDppMirror>(v));
    auto row = [&](int r) {
        return (long long)MOE_READLANE((int)(v >> 32), r * 16) << 32 | (unsigned)MOE_READLANE((int)v, r * 16);
    };
    const long long a = row(0), b = row(1), c = row(2), d = row(3);
    const long long ab = a > b ? a : b, cd = c > d ? c : d;
    return ab > cd ? ab : cd;
}

// Doubles as whole numbers of the same order
constexpr long long kNoKey = (long long)0x800fffffffffffffull;  // of minus infinity
__device__ __forceinline__ long long key_order(double v) {
    const long long b = __double_as_longlong(v + 0.0);  // (-0 is 0)
    return b ^ (b >> 63 & 0x7fffffffffffffffll);
}

// The picks of one token by a whole wave, as the definition has them: every round looks for the largest key left, at its
// lowest index, and takes switched-off experts when there is no other.  Expert 64 v + lane is value v of a lane.  Keys:
// the logits themselves (KEYS: score and bias), in 64 bits.
// Few tokens come here (keys too near for 32 bits, too few experts left), but a launch lasts as long as its last wave: what a
// round takes is what counts.
template <int V, bool KEYS>
__device__ __forceinline__ void route_exactly(const RouteArgs& g, int t, double* s_key, float* s_logit, float* s_bias) {
    const int lane = threadIdx.x & 63, E = g.E, G = g.G, per = E / G;
    float l[V], bias[V], top = -INFINITY;
    // (read again: kept for this, they would cost every wave 2 V registers)
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = min(v * kWave + lane, E - 1);
        l[v] = g.logits[(size_t)t * E + e];
        bias[v] = KEYS && g.bias ? g.bias[e] : 0.f;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = v * kWave + lane;
        if (e >= E || !(l[v] == l[v])) l[v] = -INFINITY;
        top = fmaxf(top, l[v]);
        s_logit[e] = l[v];
        if (KEYS) s_bias[e] = bias[v];
    }
    wave_lds();
    top = wave_max(top);
    const float base = top == -INFINITY ? 0.f : top;
    double d64 = 0.0;
    float den = 0.f;
    if (!g.sigmoid) {
#pragma unroll
        for (int v = 0; v < V; ++v) den += expf(l[v] - base);
        den = wave_sum(den);
        if (KEYS) {
#pragma unroll 1
            for (int e = lane; e < E; e += kWave) d64 += exp((double)s_logit[e] - (double)base);
            d64 = wave_sum64(d64);
        }
    }
    // (one exponential after the other: this code runs a few times a launch, out of no cache)
#pragma unroll 1
    for (int e = lane; e < V * kWave; e += kWave) {
        double key = -key_infinity<double>();
        if (e < E) {
            const double z = s_logit[e];
            if (!KEYS) {
                key = z;
            } else if (z != -key_infinity<double>()) {
                const double x = exp(g.sigmoid ? -z : z - (double)base);
                key = (g.sigmoid ? 1.0 / (1.0 + x) : x / d64) + (double)s_bias[e];
                if (!(key == key)) key = -key_infinity<double>();  // (of a logit of infinity: every comparison has an answer)
            }
        }
        s_key[e] = key;
    }
    wave_lds();
    long long key[V];
    unsigned gone = 0;  // bit v: not to be picked
#pragma unroll
    for (int v = 0; v < V; ++v) {
        key[v] = key_order(s_key[v * kWave + lane]);
        if (v * kWave + lane >= E) gone |= 1u << v;
    }
    if (G > 1) {
        // a group to as many lanes as there are, a power of two; its rank in all of them
        const int lanes = 1 << (31 - __clz(kWave / G)), gr = lane / lanes;
        double a = -key_infinity<double>(), b = -key_infinity<double>();
        if (gr < G) {
            for (int i = lane & (lanes - 1); i < per; i += lanes) {
                const double x = s_key[gr * per + i];
                b = fmax(b, fmin(a, x));
                a = fmax(a, x);
            }
        }
#pragma unroll 1
        for (int m = 1; m < lanes; m <<= 1) {
            const double oa = __shfl_xor(a, m, kWave), ob = __shfl_xor(b, m, kWave);
            b = fmax(fmin(a, oa), fmax(b, ob));
            a = fmax(a, oa);
        }
        const long long none = -0x7fffffffffffffffll - 1;
        long long rank = gr < G ? key_order(g.group_top == 2 && b > -key_infinity<double>() ? a + b : a) : none;
        unsigned long long open = 0;
#pragma unroll 1
        for (int j = 0; j < g.kept; ++j) {
            const int first = __ffsll((long long)__ballot(rank == wave_largest(rank))) - 1, best = first / lanes;
            open |= 1ull << best;
            if (gr == best) rank = none;
        }
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (!(open >> min((v * kWave + lane) / per, 63) & 1)) gone |= 1u << v;
    }
    int my_e = 0;
#pragma unroll 1
    for (int j = 0; j < g.k; ++j) {
        long long best = kNoKey;
#pragma unroll
        for (int v = 0; v < V; ++v) best = !(gone >> v & 1) && key[v] > best ? key[v] : best;
        best = wave_largest(best);
        int e = -1;
#pragma unroll
        for (int v = V - 1; v >= 0; --v) {  // (switched-off experts have kNoKey: they come when that is the largest left)
            const unsigned long long here = __ballot(!(gone >> v & 1) && key[v] == best);
            if (here) e = v * kWave + __ffsll((long long)here) - 1;
        }
        e = max(e, 0);
        if (lane == (e & 63)) gone |= 1u << (e >> 6);
        if (lane == j) my_e = e;
    }
    const float my_l = lane < g.k ? s_logit[my_e] : -INFINITY;
    const float big = wave_max(my_l);
    float w = 0.f;
    if (g.renormalize) {
        if (my_l != -INFINITY) w = pick_weight(my_l, g.sigmoid ? fminf(big, 0.f) : big, g.sigmoid);
        const float total = wave_sum(w);
        w = total > 0.f ? w / total : 0.f;
    } else if (my_l != -INFINITY) {
        w = g.sigmoid ? 1.f / (1.f + expf(-my_l)) : expf(my_l - base) / den;
    }
    if (lane < g.k) {
        g.topk_idx[(size_t)t * g.k + lane] = my_e;
        g.topk_gate[(size_t)t * g.k + lane] = w * g.scale;
    }
    wave_lds();
}

// ---- a token to a row of 16 lanes --------------------------------------------------------------------------------
// Exchanges inside a row are register operations (DPP), and a wave has four tokens: the wave-wide form above, for every token, took
// 59 us at 16384 tokens of 256 experts where this takes 16, and 22 with some tokens on the long way.
constexpr int kTeam = 16;
constexpr int kNowhere = 1 << 20;  // above every index
template <typename F, typename Op>
__device__ __forceinline__ F team_all(F v, Op op) {
    v = op(v, dpp_any<kDppSwap1>(v));
    v = op(v, dpp_any<kDppSwap2>(v));
    v = op(v, dpp_any<kDppHalfMirror>(v));
    return op(v, dpp_any<kDppMirror>(v));
}
__device__ __forceinline__ float team_max(float v) { return team_all(v, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float team_sum(float v) { return team_all(v, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ int team_min(int v) { return team_all(v, [](int a, int b) { return min(a, b); }); }

// 1 / (1 + e^-z) with the hardware's exponential and reciprocal: off by 2^-22 and |z| 2^-24, relatively
__device__ __forceinline__ float quick_sigmoid(float z) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_rcpf(1.f + __expf(-z));
#else
    return 1.f / (1.f + __expf(-z));
#endif
}

// How many lanes of the row have a larger v than `above`, and how many one of at least `from`
template <int N = 1>
__device__ __forceinline__ void team_count(float v, float above, float from, int& n_above, int& n_from) {
    const float o = dpp_any<0x120 + N>(v);  // row_ror
    n_above += o > above ? 1 : 0;
    n_from += o >= from ? 1 : 0;
    if constexpr (N < kTeam - 1) team_count<N + 1>(v, above, from, n_above, n_from);
}

// What two keys in 32 bits may be wrong by together.  A sigmoid is off by s (1 - s) (|l| + 2) 2^-24 through its exponential and by
// 3 s 2^-24 through sum and quotient, under 2^-22; a share of a softmax by up to 36 s 2^-24 through the sum of a row; the
// sum with the bias by half a unit.
__device__ __forceinline__ float near_keys(float c, int sigmoid) { return (1.f + fabsf(c)) * (sigmoid ? 0x1p-21f : 0x1p-18f); }

// Values e0 .. e0 + V of a row of E; what lies past its end is some other value of it
template <int V>
__device__ __forceinline__ void load_values(const float* __restrict__ row, int e0, int E, bool aligned, float (&out)[V]) {
    if (V % 4 == 0 && E % 4 == 0 && aligned) {
#pragma unroll
        for (int v = 0; v < V; v += 4) {
            const f32x4 x = *reinterpret_cast<const f32x4*>(row + min(e0 + v, E - 4));
#pragma unroll
            for (int i = 0; i < 4; ++i) out[(v + i) % V] = x[i];
        }
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) out[v] = row[min(e0 + v, E - 1)];
    }
}

// V: experts of a lane, V lane + v; KQ: picks of a lane.  KEYS: keys are score and bias, else logits (exact)
template <int V, int KQ, bool KEYS>
__global__ __launch_bounds__(kWaves* kWave) void route_scored_kernel(const RouteArgs g) {
    constexpr int VW = (V * kTeam + kWave - 1) / kWave;  // values of a lane in route_exactly
    __shared__ double s_exact[kWaves][VW * kWave];
    __shared__ float s_logit[kWaves][VW * kWave], s_bias[kWaves][KEYS ? VW * kWave : 1];  // of one token at a time
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tl = lane & (kTeam - 1);
    const int t0 = (blockIdx.x * kWaves + wave) * (kWave / kTeam);
    if (t0 >= g.T) return;  // (waves exchange nothing)
    const int t = min(t0 + lane / kTeam, g.T - 1);
    const bool mine = t0 + lane / kTeam < g.T;
    const int E = g.E, k = g.k, e0 = tl * V;
    const float* row = g.logits + (size_t)t * E;
    float l[V], key[V], bias[V];
    // (requested together, and the bias with them: no load behind a branch of its own)
    load_values<V>(row, e0, E, aligned16_dev(g.logits), l);
#pragma unroll
    for (int v = 0; v < V; ++v) bias[v] = 0.f;
    if (KEYS && g.bias) load_values<V>(g.bias, e0, E, aligned16_dev(g.bias), bias);
#pragma unroll
    for (int v = 0; v < V; ++v) l[v] = v < E - e0 ? l[v] : -INFINITY;
    float top = -INFINITY;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (!(l[v] == l[v])) l[v] = -INFINITY;
        top = fmaxf(top, l[v]);
    }
    top = team_max(top);
    const float base = top == -INFINITY ? 0.f : top;
    // scores (in key, for a moment)
    float den = 1.f;
    if (KEYS || g.scores || (!g.renormalize && !g.sigmoid)) {
        if (g.sigmoid) {
#pragma unroll
            for (int v = 0; v < V; ++v) key[v] = quick_sigmoid(l[v]);
        } else {
            den = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                key[v] = __expf(l[v] - base);
                den += key[v];
            }
            den = team_sum(den);
            const float inv = den > 0.f ? 1.f / den : 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) key[v] *= inv;
        }
        if (g.scores && mine) {
            float* out = g.scores + (size_t)t * E + e0;
            if (V % 4 == 0 && E % 4 == 0 && aligned16_dev(g.scores)) {
#pragma unroll
                for (int v = 0; v < V; v += 4)
                    if (e0 + v < E) *reinterpret_cast<f32x4*>(out + v) = f32x4{key[v], key[(v + 1) % V], key[(v + 2) % V], key[(v + 3) % V]};
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (e0 + v < E) out[v] = key[v];
            }
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (KEYS) {
            key[v] = l[v] == -INFINITY ? -INFINITY : key[v] + bias[v];
            if (!(key[v] == key[v])) key[v] = -INFINITY;
        } else {
            key[v] = l[v];
        }
    }
    bool unsure = false;  // (of the token: all of its lanes agree)
    if (g.G > 1) {
        const int per = E / g.G, lanes = per / V;
        if (lanes * V == per && (lanes & (lanes - 1)) == 0 && lanes <= kTeam) {
            // a group is 2^n lanes: its two largest keys, in all of them
            float a = -INFINITY, b = -INFINITY;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                b = fmaxf(b, fminf(a, key[v]));
                a = fmaxf(a, key[v]);
            }
            auto join = [&](float oa, float ob) {
                b = fmaxf(fminf(a, oa), fmaxf(b, ob));
                a = fmaxf(a, oa);
            };
            if (lanes >= 2) join(dpp_any<kDppSwap1>(a), dpp_any<kDppSwap1>(b));
            if (lanes >= 4) join(dpp_any<kDppSwap2>(a), dpp_any<kDppSwap2>(b));
            if (lanes >= 8) join(dpp_any<kDppHalfMirror>(a), dpp_any<kDppHalfMirror>(b));
            if (lanes >= 16) join(dpp_any<kDppMirror>(a), dpp_any<kDppMirror>(b));
            float rank = g.group_top == 2 && b > -INFINITY ? a + b : a;
            if (e0 >= E) rank = __int_as_float(0x7fc00000);  // (no group: above and below none)
            const float gap = team_max(2.f * near_keys((a > -INFINITY ? fabsf(a) : 0.f) + (b > -INFINITY ? fabsf(b) : 0.f), g.sigmoid));
            int above = 0, from = 0;  // lanes of groups that are surely, or possibly, before this one
            team_count(rank, KEYS ? rank + gap : rank, KEYS ? rank - gap : rank, above, from);
            from -= lanes - 1;        // (its own)
            const bool in = from < g.kept * lanes, out = above >= g.kept * lanes;
            // (logits: equal ranks are decided by index, in route_exactly, where that matters)
            if (!in) {
#pragma unroll
                for (int v = 0; v < V; ++v) key[v] = -INFINITY;
            }
            unsure = team_min(e0 < E && !in && !out ? 0 : 1) == 0 || (KEYS && !(gap < INFINITY));  // (sums beyond fp32 compare as equal)
        } else {
            // other groups: the keys of one token at a time through LDS, a group a lane
            float* s_key = s_logit[wave];
            for (int q = 0; q < kWave / kTeam; ++q) {
                if (lane / kTeam == q) {
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        if (e0 + v < E) s_key[e0 + v] = key[v];
                }
                wave_lds();
                float a = -INFINITY, b = -INFINITY;
                if (lane < g.G) {
                    for (int i = 0; i < per; ++i) {
                        const float x = s_key[lane * per + i];
                        b = fmaxf(b, fminf(a, x));
                        a = fmaxf(a, x);
                    }
                }
                wave_lds();
                const float rank = g.group_top == 2 && b > -INFINITY ? a + b : a;
                const float gap = KEYS ? wave_max(2.f * near_keys((a > -INFINITY ? fabsf(a) : 0.f) + (b > -INFINITY ? fabsf(b) : 0.f), g.sigmoid)) : 0.f;
                int above = 0, from = 0;
                for (int i = 0; i < g.G; ++i) {
                    const float o = __shfl(rank, i, kWave);
                    above += o > rank + gap ? 1 : 0;
                    from += o >= rank - gap && i != lane ? 1 : 0;
                }
                const unsigned long long open = __ballot(lane < g.G && from < g.kept), maybe = __ballot(lane < g.G && from >= g.kept && above < g.kept);
                if (lane / kTeam == q) {
                    unsure = maybe != 0 || !(gap < INFINITY);
#pragma unroll
                    for (int v = 0; v < V; ++v)
                        if (!(open >> min((e0 + v) / per, 63) & 1)) key[v] = -INFINITY;
                }
            }
        }
    }
    // Keys as whole numbers of the same order (their maxima need no care for NaN, and join an exchange in one instruction)
    int rank[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int b = __float_as_int(key[v] + 0.f);  // (-0 is 0)
        rank[v] = b ^ (b >> 31 & 0x7fffffff);
    }
    const int none = (int)0x807fffff;  // of minus infinity
    auto as_key = [](int r) { return __int_as_float(r ^ (r >> 31 & 0x7fffffff)); };
    auto largest = [&]() {
        int best = rank[0];
#pragma unroll
        for (int v = 1; v < V; ++v) best = max(best, rank[v]);
        return team_all(best, [](int a, int b) { return max(a, b); });
    };
    int my_e[KQ];
    float last = INFINITY;
#pragma unroll
    for (int q = 0; q < KQ; ++q) my_e[q] = 0;
#pragma unroll
    for (int q = 0; q < KQ; ++q) {
        for (int j = 0; j < kTeam; ++j) {
            const int n = q * kTeam + j;
            if (n >= k) break;
            const int m = largest();
            int at = kNowhere, equal = 0;
            if (KEYS) {
                // (equal keys leave together: the token takes the long way)
#pragma unroll
                for (int v = V - 1; v >= 0; --v) {
                    const bool is = rank[v] == m;
                    at = is ? v : at;
                    equal += is ? 1 : 0;
                    rank[v] = is ? none : rank[v];
                }
            } else {
#pragma unroll
                for (int v = V - 1; v >= 0; --v) at = rank[v] == m ? v : at;
            }
            const int e = team_min(at + e0);
            if (KEYS) {
                unsure |= last - as_key(m) <= near_keys(as_key(m), g.sigmoid) || equal > 1 || (equal && at + e0 != e);
                last = as_key(m);
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v) rank[v] = v == e - e0 ? none : rank[v];
            }
            unsure |= m == none;  // (switched-off experts, or none: in their order)
            if (tl == j) my_e[q] = e;
        }
    }
    if (KEYS) {  // the best that was not picked
        const int m = largest();
        unsure |= m != none && last - as_key(m) <= near_keys(as_key(m), g.sigmoid);
        unsure = team_min(unsure ? 0 : 1) == 0;
    }
    // gates
    float pl[KQ], w[KQ], big = -INFINITY, total = 0.f;
#pragma unroll
    for (int q = 0; q < KQ; ++q) {
        const int n = q * kTeam + tl;
        pl[q] = -INFINITY;
        if (n < k) pl[q] = row[min(max(my_e[q], 0), E - 1)];
        if (!(pl[q] == pl[q])) pl[q] = -INFINITY;
        big = fmaxf(big, pl[q]);
    }
    big = team_max(big);
    const float m = g.sigmoid ? fminf(big, 0.f) : big;
#pragma unroll
    for (int q = 0; q < KQ; ++q) {
        w[q] = 0.f;
        if (pl[q] != -INFINITY)
            w[q] = g.renormalize ? pick_weight(pl[q], m, g.sigmoid) : g.sigmoid ? 1.f / (1.f + expf(-pl[q])) : expf(pl[q] - base) / den;
        total += w[q];
    }
    total = g.renormalize ? team_sum(total) : 1.f;
    const float f = total > 0.f ? g.scale / total : 0.f;
#pragma unroll
    for (int q = 0; q < KQ; ++q) {
        const int n = q * kTeam + tl;
        if (mine && !unsure && n < k) {
            g.topk_idx[(size_t)t * k + n] = my_e[q];  // (sure, so an expert's)
            g.topk_gate[(size_t)t * k + n] = w[q] * f;
        }
    }
    // tokens that take the long way
    unsigned long long again = __ballot(unsure && mine && tl == 0);
    while (again) {
        const int who = __ffsll((long long)again) - 1;
        again &= again - 1;
        route_exactly<VW, KEYS>(g, t0 + who / kTeam, s_exact[wave], s_logit[wave], s_bias[wave]);
    }
}

// ---- the gradient ------------------------------------------------------------------------------------------------------
// Of the gates g_j = scale w_j / sum w, w the picked scores, the derivative of a loss with gradient dg is, for the logit of pick j,
//   g_j (dg_j - sum_i dg_i g_i / scale), with a sigmoid times 1 - s_j:
// the softmax's own coupling adds nothing, since sum_j w_j d(loss)/d(w_j) = 0.  In this form no score is divided by, so
// that rows of tiny scores keep their gradient.  Without renormalisation, and for gradients of the scores themselves,
// d(loss)/d(l_e) = s_e (ds_e - sum ds s), or ds_e s_e (1 - s_e).
// A wave takes a token; four neighbouring experts to a lane where rows allow it (FOUR).  Bound by the chain of a wave: picks, their logits, sums over
// lanes, sums through LDS, and then the row.  (16384 tokens of 256 experts, without a gradient of the scores, us: 13.9 with all scores formed, 9.6 now, of which
// 0.8 are slopes of experts that were not picked; a fill of the 17 MB that it writes takes 4.6.)
template <int V, bool FOUR>
__global__ __launch_bounds__(kWaves* kWave) void route_scored_backward_kernel(const float* __restrict__ logits, const int32_t* __restrict__ topk_idx,
                                                                              const float* __restrict__ grad_gate, const float* __restrict__ grad_scores,
                                                                              float* __restrict__ grad_logits, int T, int E, int k, int sigmoid,
                                                                              int renormalize, float scale) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t = blockIdx.x * kWaves + wave;
    __shared__ __align__(16) float s_add[kWaves][V * kWave];
    if (t >= T) return;  // (waves exchange nothing)
    const float* row = logits + (size_t)t * E;
    constexpr int W = FOUR ? 4 : 1;  // neighbours of a lane
    static_assert(V % W == 0, "whole pieces");
    typedef float piece_t __attribute__((ext_vector_type(W)));
    auto expert = [&](int v) { return (v / W * kWave + lane) * W; };  // the first of piece v / W
    auto load = [&](const float* from, float (&out)[V], float beyond) {
#pragma unroll
        for (int v = 0; v < V; v += W) {
            const piece_t p = *reinterpret_cast<const piece_t*>(from + min(expert(v), E - W));
#pragma unroll
            for (int i = 0; i < W; ++i) out[v + i] = expert(v) < E ? p[i] : beyond;
        }
    };
    const int e_of = lane < k ? topk_idx[(size_t)t * k + lane] : -1;
    const bool named = (unsigned)e_of < (unsigned)E;
    float dg = named ? grad_gate[(size_t)t * k + lane] : 0.f;
    float pl = named ? row[e_of] : -INFINITY;
    if (!(pl > -INFINITY)) pl = -INFINITY, dg = 0.f;  // (of a constant, whatever the gradient: 0 times an infinity would be a NaN of the row)
    // Without a gradient of the scores the logits that were not picked have none, and are not read, unless a softmax's sum couples them
    const bool all = grad_scores || !(renormalize || sigmoid);
    float l[V], ds[V], s[V], base = 0.f, den = 1.f;
#pragma unroll
    for (int v = 0; v < V; ++v) l[v] = -INFINITY, ds[v] = s[v] = 0.f;
    if (all) {
        load(row, l, -INFINITY);
        if (grad_scores) load(grad_scores + (size_t)t * E, ds, 0.f);
        float top = -INFINITY;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!(l[v] > -INFINITY)) l[v] = -INFINITY, ds[v] = 0.f;
            top = fmaxf(top, l[v]);
        }
        if (sigmoid) {
#pragma unroll
            for (int v = 0; v < V; ++v) s[v] = quick_sigmoid(l[v]);
        } else {
            top = wave_max(top);
            base = top == -INFINITY ? 0.f : top;
            den = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                s[v] = __expf(l[v] - base);
                den += s[v];
            }
            den = wave_sum(den);
            const float inv = den > 0.f ? 1.f / den : 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) s[v] *= inv;
        }
    }
#pragma unroll
    for (int v = 0; v < V; v += W) *reinterpret_cast<piece_t*>(&s_add[wave][expert(v)]) = piece_t(0.f);
    // what a pick adds to the gradient of its logit
    float add;
    const float slope = sigmoid ? 1.f / (1.f + expf(pl)) : 1.f;  // 1 - s
    if (renormalize) {
        const float big = wave_max(pl);
        float w = 0.f;
        if (pl != -INFINITY) w = pick_weight(pl, sigmoid ? fminf(big, 0.f) : big, sigmoid);
        const float total = wave_sum(w);
        const float g = total > 0.f ? w / total : 0.f;
        add = scale * g * (dg - wave_sum(dg * g)) * slope;
    } else {
        add = scale * dg * (sigmoid ? 1.f / (1.f + expf(-pl)) : den > 0.f ? expf(pl - base) / den : 0.f) * slope;
    }
    // an expert may be named twice: then one pick after the other, so that sums have an order
    bool again = false;
    for (int j = 1; j < k; ++j) {
        const int o = MOE_READLANE(e_of, j);
        again |= named && lane < j && o == e_of;
    }
    wave_lds();
    if (!__ballot(again)) {
        if (named) s_add[wave][e_of] = add;
    } else {
        for (int j = 0; j < k; ++j) {
            if (lane == j && named) s_add[wave][e_of] += add;
            wave_lds();
        }
    }
    wave_lds();
    float shared = 0.f;
    if (!sigmoid && all) {
        float part = renormalize || !named ? 0.f : add;
#pragma unroll
        for (int v = 0; v < V; ++v) part += ds[v] * s[v];
        shared = wave_sum(part);
    }
#pragma unroll
    for (int v = 0; v < V; v += W) {
        const int e = expert(v);
        if (e >= E) continue;
        piece_t o = *reinterpret_cast<const piece_t*>(&s_add[wave][e]);
#pragma unroll
        for (int i = 0; i < W; ++i)
            o[i] += sigmoid ? ds[v + i] * s[v + i] * quick_sigmoid(-l[v + i]) : s[v + i] * (ds[v + i] - shared);
        *reinterpret_cast<piece_t*>(grad_logits + (size_t)t * E + e) = o;
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

// launch(t0, n) for runs of up to kTokenRun tokens, one after the other: the 2^32 work items that a dimension of a grid may not reach are 2^26 tokens of
// the gradient, 2^24 of the router's logits and 2^28 of the picks
constexpr int kTokenRun = 1 << 23;
template <typename L>
int in_runs(int T, L launch) {
    for (long long t0 = 0; t0 < T; t0 += kTokenRun) {
        const int rc = launch((size_t)t0, (int)std::min<long long>(kTokenRun, T - t0));
        if (rc != MOE_OK) return rc;
    }
    return MOE_OK;
}

// values a lane: a power of two
template <typename L>
int with_values(int E, L launch) {
    if (E <= 64) return launch(std::integral_constant<int, 1>{});
    if (E <= 128) return launch(std::integral_constant<int, 2>{});
    if (E <= 256) return launch(std::integral_constant<int, 4>{});
    return launch(std::integral_constant<int, 8>{});
}

template <typename L>
int with_team_values(int E, L launch) {
    if (E <= 16) return launch(std::integral_constant<int, 1>{});
    if (E <= 32) return launch(std::integral_constant<int, 2>{});
    if (E <= 64) return launch(std::integral_constant<int, 4>{});
    if (E <= 128) return launch(std::integral_constant<int, 8>{});
    if (E <= 256) return launch(std::integral_constant<int, 16>{});
    return launch(std::integral_constant<int, 32>{});
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
    // the order of keys is that of the logits, which fp32 holds exactly, unless there is a bias or a group's rank is a sum
    const bool by_logit = !bias && (c.n_groups == 1 || c.group_top == 1);
    constexpr int kTokens = kWaves * kWave / kTeam;
    return in_runs(T, [&](size_t t0, int n) {
        const RouteArgs g{logits + t0 * E, bias, idx + t0 * k, gate + t0 * k, scores ? scores + t0 * E : nullptr, n, E, k, c.score, c.n_groups, c.groups_kept,
                          c.group_top, c.renormalize, c.scale};
        return with_team_values(E, [&](auto V) {
            auto launch = [&](auto kern) {
                hipLaunchKernelGGL(kern, dim3((n + kTokens - 1) / kTokens), dim3(kWaves * kWave), 0, st, g);
                return launch_status();
            };
            constexpr int v = decltype(V)::value;
            if (by_logit) return k <= kTeam ? launch(route_scored_kernel<v, 1, false>) : launch(route_scored_kernel<v, 4, false>);
            return k <= kTeam ? launch(route_scored_kernel<v, 1, true>) : launch(route_scored_kernel<v, 4, true>);
        });
    });
}

int launch_router_logits(const moe_shape& s, const void* x, const float* rw, const float* rb, float* logits, hipStream_t st) {
    return in_runs(s.n_tokens, [&](size_t t0, int n) {
        const dim3 grid((n + kRouteTok - 1) / kRouteTok), block(kRouteWaves * kWave);
        auto launch = [&](auto kern, auto* rows) {
            hipLaunchKernelGGL(kern, grid, block, 0, st, rows + t0 * s.d_model, rw, rb, s.d_model, s.n_experts, n, logits + t0 * s.n_experts);
            return launch_status();
        };
        if (s.act_dtype == MOE_F32) return launch(router_logits_kernel<float>, static_cast<const float*>(x));
        return launch(router_logits_kernel<bf16_t>, static_cast<const bf16_t*>(x));
    });
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
    // four experts to a lane: rows of whole 16-byte pieces
    const bool four = n_experts >= 256 && n_experts % 4 == 0 && aligned16(logits) && aligned16(grad_scores) && aligned16(grad_logits);
    const size_t E = n_experts, k = top_k;
    return in_runs(n_tokens, [&](size_t t0, int n) {
        return with_values(n_experts, [&](auto V) {
            constexpr int v = decltype(V)::value;
            auto launch = [&](auto kern) {
                hipLaunchKernelGGL(kern, dim3((n + kWaves - 1) / kWaves), dim3(kWaves * kWave), 0, as_stream(stream), logits + t0 * E, topk_idx + t0 * k,
                                   grad_gate + t0 * k, grad_scores ? grad_scores + t0 * E : nullptr, grad_logits + t0 * E, n, n_experts, top_k, c.score,
                                   c.renormalize, c.scale);
                return launch_status();
            };
            if constexpr (v >= 4)
                if (four) return launch(route_scored_backward_kernel<v, true>);
            return launch(route_scored_backward_kernel<v, false>);
        });
    });
}
