// Experts on MXFP4 weights for a few tokens, in two launches: the weights are all there is to move.
//
// Both launches stream weights straight from memory into registers: the layout of mxfp4.h makes every request of a
// wave one run of 1 KB, in the order in which the matrix instruction takes it, and with up to 16 rows a result tile
// is one instruction for 1 KB of weights, so that nothing but the requests is in the way.
//   hidden: a workgroup makes 32 hidden columns of one expert's rows.  Its waves cut K; each quantises its own
//           columns of the tokens' rows (a lane holds the 32 values of one scale: no exchange), so that no launch
//           goes before it, and the sums meet in LDS once.
//   down:   a workgroup makes 16 columns of all tokens: its waves are cut over the experts in use and over K, and the
//           gated sum of the experts is formed where the parts meet, so that no launch comes after it.
// Hidden rows lie by pair, not by expert: which rows an expert has every wave finds from the picks.
#include <algorithm>

#include "mxfp4.h"

namespace moe {

namespace {

// The picks, a pair to a lane: its expert, or -1
struct Picks {
    int key;
    __device__ __forceinline__ void load(const int32_t* __restrict__ idx, int P, int E, int lane) {
        key = idx[min(lane, P - 1)];
        if (lane >= P || (unsigned)key >= (unsigned)E) key = -1;
    }
    // experts that have a pair
    __device__ __forceinline__ unsigned long long used() const {
        unsigned long long m = 0;
#pragma unroll
        for (int p = 0; p < kMxFewPairs; ++p) {
            const int e = MOE_READLANE(key, p);
            m |= e >= 0 ? 1ull << e : 0;
        }
        return m;
    }
    // Row `row` of expert e (rows in the order of pairs): its pair, or -1
    __device__ __forceinline__ int pair_of_row(int e, int row) const {
        const unsigned m = (unsigned)__ballot(key == e);
        int found = -1, n = 0;
#pragma unroll
        for (int p = 0; p < kMxFewPairs; ++p) {
            const bool is = m >> p & 1;
            found = is && n == row ? p : found;
            n += is ? 1 : 0;
        }
        return found;
    }
};
static_assert(kMxFewPairs <= 16, "the rows of an expert are one tile");

// The n-th set bit of m, or -1
__device__ __forceinline__ int nth_bit(unsigned long long m, int n) {
    for (; n > 0 && m; --n) m &= m - 1;
    return m ? __ffsll((long long)m) - 1 : -1;
}

// Where the codes of pair p, k-step c, columns 32 q .. lie in a matrix of hidden rows; and the byte of their scale
__device__ __forceinline__ size_t row_codes(int p, int c, int q, int units) {
    return ((size_t)(p >> 5) * units + (c >> 1)) * kMxCodes + ((c & 1) * 2 + (p >> 4 & 1)) * 1024 + (q * 16 + (p & 15)) * 16;
}
__device__ __forceinline__ size_t row_scale(int p, int c, int q, int units) {
    return ((size_t)(p >> 5) * units + (c >> 1)) * kMxScales + (q * 16 + (p & 15)) * 4 + (c & 1) * 2 + (p >> 4 & 1);
}

constexpr int kHiddenWaves = 4;  // (whole layer, us, with eight / with these: 2048 / 5632, one token 14.5 / 14.6, two 19.5 / 19.7, four 34.8 / 33.2; 1024 / 2816, two 17.5 / 15.9)

template <typename T>
__global__ __launch_bounds__(kHiddenWaves* kWave) void mx_few_hidden_kernel(ptr_arg a_idx, ptr_arg a_x, ptr_arg a_gate, ptr_arg a_up, int P, int E, int k, int d,
                                                                            int F, ptr_arg a_out, size_t out_scales) {
    typedef Store<T> S;
    constexpr int VECS = 32 / S::VEC;
    const char* const w_of[2] = {from_arg<const char>(a_gate), from_arg<const char>(a_up)};
    const T* const x = from_arg<const T>(a_x);
    char* const out = from_arg<char>(a_out);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int fb = blockIdx.x, fbs = mx_blocks(F), units = mx_units(d), out_units = mx_units(F);
    __shared__ f32x4 s_part[kHiddenWaves][4][kWave];
    Picks picks;
    picks.load(from_arg<const int32_t>(a_idx), P, E, lane);
    const int e = nth_bit(picks.used(), blockIdx.y);
    if (e < 0) return;
    const int ln = lane & 15, q = lane >> 4;
    // this wave's k-steps
    const int steps = units * 2, c_begin = steps * wave / kHiddenWaves, c_end = fb < fbs ? steps * (wave + 1) / kHiddenWaves : c_begin;
    const size_t at = ((size_t)e * fbs + fb) * units, scales = (size_t)E * fbs * units * kMxCodes;
    const int pair = picks.pair_of_row(e, ln);
    const T* const row = x + (size_t)(pair < 0 ? 0 : quick_div(pair, k)) * d;
    f32x4 acc[2][2];  // [gate, up][tile of columns]
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i / 2][i % 2] = f32x4{0.f, 0.f, 0.f, 0.f};
    constexpr int U = 2;  // k-steps requested together
    for (int c0 = c_begin; c0 < c_end; c0 += U) {
        i32x4 wv[U][2][2];
        int ws[U][2];
        typename S::vec_t xv[U][VECS];
#pragma unroll
        for (int s = 0; s < U; ++s) {
            const int c = min(c0 + s, c_end - 1);
#pragma unroll
            for (int m = 0; m < 2; ++m) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    wv[s][m][t] = *reinterpret_cast<const i32x4*>(w_of[m] + at * kMxCodes + (size_t)(c * 2 + t) * 1024 + lane * 16);
                ws[s][m] = *reinterpret_cast<const int*>(w_of[m] + scales + (at + (c >> 1)) * kMxScales + lane * 4) >> (c & 1) * 16;
            }
            // the lane's 32 values of its row: those past the row's end are zeros
            const int col = c * 128 + q * 32;
#pragma unroll
            for (int i = 0; i < VECS; ++i) xv[s][i] = *reinterpret_cast<const typename S::vec_t*>(row + min(col + i * S::VEC, d - S::VEC));
        }
#pragma unroll
        for (int s = 0; s < U; ++s) {
            if (c0 + s >= c_end) break;
            const int col = (c0 + s) * 128 + q * 32;
            if (col + 32 > d) {
#pragma unroll
                for (int i = 0; i < VECS; ++i)
                    if (col + i * S::VEC >= d) xv[s][i] = typename S::vec_t{};
            }
            i32x4 xc;
            int xs;
            mx_quantise_32<T>(xv[s], xc, xs);
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                acc[m][0] = mx_mfma<0, 0>(wv[s][m][0], xc, acc[m][0], ws[s][m], xs);
                acc[m][1] = mx_mfma<1, 0>(wv[s][m][1], xc, acc[m][1], ws[s][m], xs);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s_part[wave][i][lane] = acc[i / 2][i % 2];
    __syncthreads();
    // sums over the waves, a tile a wave
    if (wave < 4) {
        f32x4 sum = s_part[0][wave][lane];
#pragma unroll
        for (int w = 1; w < kHiddenWaves; ++w) {
            const f32x4 o = s_part[w][wave][lane];
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] += o[i];
        }
        s_part[0][wave][lane] = sum;
    }
    __syncthreads();
    if (wave == 0) {  // a lane has columns 32 fb + 8 (lane / 16) ... of row lane % 16
        float f[8];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const f32x4 g = s_part[0][t][lane], u = s_part[0][2 + t][lane];
#pragma unroll
            for (int i = 0; i < 4; ++i) f[t * 4 + i] = silu_f32(g[i]) * u[i];
        }
        const int b = mx_scale_byte(mx_max_of_rows((int)mx_abs_max(f)));
        if (pair >= 0) {
            *reinterpret_cast<unsigned*>(out + row_codes(pair, fb >> 2, fb & 3, out_units) + q * 4) = mx_codes8(f, b);
            if (q == 0) out[out_scales + row_scale(pair, fb >> 2, fb & 3, out_units)] = (char)b;
        }
    }
}

constexpr int kDownWaves = 16;

template <typename T>
struct Four;  // four neighbours of a row
template <>
struct Four<float> { typedef f32x4 vec_t; };
template <>
struct Four<bf16_t> { typedef bf16x4 vec_t; };

template <typename T>
__global__ __launch_bounds__(kDownWaves* kWave) void mx_few_down_kernel(ptr_arg a_idx, ptr_arg a_h, ptr_arg a_down, ptr_arg a_pick_gate, int P, int E, int k, int d,
                                                                        int F, size_t h_scales, ptr_arg a_residual, ptr_arg a_y) {
    __shared__ f32x4 s_part[kDownWaves][kWave];  // [expert in use x part of K]
    __shared__ int s_place[kMxFewPairs];         // of a pair: the first item of its expert * 16 + its row
    __shared__ float s_gate[kMxFewPairs];
    const char* const h = from_arg<const char>(a_h);
    const char* const w = from_arg<const char>(a_down);
    const float* const gate = from_arg<const float>(a_pick_gate);
    const T* const residual = from_arg<const T>(a_residual);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ln = lane & 15, q = lane >> 4;
    const int fb = blockIdx.x >> 1, tile = blockIdx.x & 1, fbs = mx_blocks(d), units = mx_units(F);
    // Four neighbouring columns a thread: token t, columns 32 fb + 8 a + 4 tile ...  (What the end needs is requested at the start.)
    typedef typename Four<T>::vec_t four_t;
    const int t = threadIdx.x >> 2, a = threadIdx.x & 3, col = fb * 32 + a * 8 + tile * 4;
    const bool mine = t * k < P && col < d;
    four_t base{};
    if (mine && residual) base = *reinterpret_cast<const four_t*>(residual + (size_t)t * d + col);
    const float my_gate = wave == 0 && lane < P ? gate[lane] : 0.f;
    Picks picks;
    picks.load(from_arg<const int32_t>(a_idx), P, E, lane);
    const unsigned long long used = picks.used();
    const int n_used = max(__popcll(used), 1), parts = kDownWaves / n_used;
    const int steps = units * 2;
    const int hit = uniform_div(wave, parts), part = wave - hit * parts;
    const int e = nth_bit(used, hit);
    if (e >= 0) {
        const int c_begin = uniform_div(steps * part, parts), c_end = uniform_div(steps * (part + 1), parts);
        const size_t at = ((size_t)e * fbs + fb) * units, scales = (size_t)E * fbs * units * kMxCodes;
        const int pair = max(picks.pair_of_row(e, ln), 0);
        f32x4 acc{0.f, 0.f, 0.f, 0.f};
        constexpr int U = 6;  // (5632 columns in eight parts: all of a wave's requests at once)
        for (int c0 = c_begin; c0 < c_end; c0 += U) {
            i32x4 wv[U], hv[U];
            int ws[U], hs[U];
#pragma unroll
            for (int s = 0; s < U; ++s) {
                const int c = min(c0 + s, c_end - 1);
                wv[s] = *reinterpret_cast<const i32x4*>(w + at * kMxCodes + (size_t)(c * 2 + tile) * 1024 + lane * 16);
                ws[s] = *reinterpret_cast<const int*>(w + scales + (at + (c >> 1)) * kMxScales + lane * 4) >> ((c & 1) * 16 + tile * 8);
                hv[s] = *reinterpret_cast<const i32x4*>(h + row_codes(pair, c, q, units));
                hs[s] = (uint8_t)h[h_scales + row_scale(pair, c, q, units)];
            }
#pragma unroll
            for (int s = 0; s < U; ++s) {
                if (c0 + s >= c_end) break;
                acc = mx_mfma<0, 0>(wv[s], hv[s], acc, ws[s], hs[s]);
            }
        }
        s_part[wave][lane] = acc;
    }
    if (wave == 0 && lane < kMxFewPairs) {
        // rows before this one among its expert's, and experts in use before its own
        int row = 0;
#pragma unroll
        for (int p = 0; p < kMxFewPairs; ++p) row += p < lane && MOE_READLANE(picks.key, p) == picks.key ? 1 : 0;
        s_gate[lane] = my_gate;
        s_place[lane] = picks.key < 0 ? -1 : __popcll(used & ((1ull << picks.key) - 1)) * parts * 16 + row;
    }
    __syncthreads();
    if (!mine) return;
    float f[4] = {0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < k; ++j) {
        const int place = s_place[t * k + j];
        if (place < 0) continue;
        const f32x4* from = &s_part[place >> 4][a * 16 + (place & 15)];
        f32x4 sum = *from;
        for (int p = 1; p < parts; ++p) {
            const f32x4 o = from[p * kWave];
#pragma unroll
            for (int c = 0; c < 4; ++c) sum[c] += o[c];
        }
        const float g = s_gate[t * k + j];
#pragma unroll
        for (int c = 0; c < 4; ++c) f[c] = fmaf(g, sum[c], f[c]);
    }
    four_t o;
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] = Store<T>::from_f32(f[c] + (float)base[c]);
    *reinterpret_cast<four_t*>(from_arg<T>(a_y) + (size_t)t * d + col) = o;
}

}  // namespace

template <typename T>
static int few(const moe_shape& s, const moe_mxfp4_weights& w, const void* x, const int32_t* idx, const float* gate, void* y, const MxLayout& l, char* ws,
               hipStream_t st) {
    const int P = s.n_tokens * s.top_k, E = s.n_experts, d = s.d_model, F = s.d_ff;
    const size_t h_scales = (size_t)l.blocks * mx_units(F) * kMxCodes;
    hipLaunchKernelGGL(mx_few_hidden_kernel<T>, dim3(mx_units(F) * (kMxUnit / 32), std::min(E, P)), dim3(kHiddenWaves * kWave), 0, st, as_arg(idx), as_arg(x),
                       as_arg(w.gate), as_arg(w.up), P, E, s.top_k, d, F, as_arg(ws + l.hq), h_scales);
    hipLaunchKernelGGL(mx_few_down_kernel<T>, dim3(mx_blocks(d) * 2), dim3(kDownWaves * kWave), 0, st, as_arg(idx), as_arg(ws + l.hq), as_arg(w.down),
                       as_arg(gate), P, E, s.top_k, d, F, h_scales, as_arg((s.flags & MOE_FLAG_RESIDUAL) ? x : nullptr), as_arg(y));
    return launch_status();
}

int launch_mx_few(const moe_shape& s, const moe_mxfp4_weights& w, const void* x, const int32_t* idx, const float* gate, void* y, const MxLayout& l, char* ws,
                  hipStream_t st) {
    return s.act_dtype == MOE_F32 ? few<float>(s, w, x, idx, gate, y, l, ws, st) : few<bf16_t>(s, w, x, idx, gate, y, l, ws, st);
}

}  // namespace moe
