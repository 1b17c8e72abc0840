// Gradient of the experts (moe_training.h states it): the order of its products, and kernels for any type and size.
//
// Three launches: a, b and dh with the activation's gradient behind them, then the gradients of the weights and of the rows.
// The forward pass keeps nothing for it: a and b are formed again (4 of 16 P d F operations), which is less than what reading
// them back would save in any program that holds more than a few layers' worth of rows.
//
// The kernels here: tiles of 64 x 64, or 32 x 32 where those are few, on four waves, operands widened to fp32 in LDS, v_mfma_f32_16x16x4_f32, a layout of
// operands that the k axis of either kind of product needs no transposition for.  97 to 108 TFLOP/s from 2048 tokens of 2048 / 5632 on (the fp32 matrix rate
// is 157); they serve fp32 layers, which are the small ones, and layers too narrow for expert_grad_mfma.hip.
#include "expert_grad.h"
#include "expert_grad_plan.h"

namespace moe {

namespace {

constexpr int kThreads = 256;
// Tiles of 64 by 64 up to which 32 by 32 ones are taken: a tile's k-steps follow one another, and smaller ones put more CUs to work on them.  (us, 64 / 32 by
// these: fp32, 10 tokens of 384 / 512, 4 of 4 experts, 73 / 38, 168 of 144 / 880 82 / 50, 300 of 256 / 512 79 / 49; bf16, 2048 of 128 / 1152 287 / 202.
// Beyond: the rows' gradient of 2048 of 432 / 1152, 504 tiles, 13 us longer in small ones)
constexpr int kFewRowTiles = 256, kFewWeightTiles = 1024;

// Tiles of SIDE by SIDE on four waves, k-steps of STEP, AHEAD of which are on their way while one is multiplied
template <int SIDE_>
struct Form {
    static constexpr int SIDE = SIDE_, STEP = 4 * kThreads / SIDE, PITCH = SIDE + 4, AHEAD = SIDE == 32 ? 4 : 2, NB = SIDE / 32;
    float a[2][STEP][PITCH], b[2][STEP][PITCH];
};

// A tile's share of one operand: STEP k by SIDE rows (or columns) in fp32, [k][row].  K_CONTIGUOUS: memory holds [row][k].
template <typename F, typename T, bool K_CONTIGUOUS>
struct Operand {
    static constexpr int PER_ROW = K_CONTIGUOUS ? F::STEP / 4 : F::SIDE / 4;  // threads that share a row of memory
    const T* base;       // of the expert's matrix or the group's first row
    long long pitch;     // elements from one row of memory to the next
    int rows, K;         // valid rows (columns) from `first` on, valid k
    int first;

    __device__ __forceinline__ f32x4 load(int k0) const {
        const int t = threadIdx.x, along = t % PER_ROW * 4, across = t / PER_ROW;
        const T* p;
        bool ok;
        if (K_CONTIGUOUS) {  // four k of a row
            const int r = across, k = k0 + along;
            ok = r < rows && k < K;
            p = base + (first + r) * pitch + k;
        } else {             // four rows of a k
            const int r = along, k = k0 + across;
            ok = r < rows && k < K;
            p = base + k * pitch + first + r;
        }
        f32x4 v{0.f, 0.f, 0.f, 0.f};
        if (ok) {
            if constexpr (sizeof(T) == 4) {
                v = *reinterpret_cast<const f32x4*>(p);
            } else {
                const bf16x4 b = *reinterpret_cast<const bf16x4*>(p);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = (float)b[i];
            }
        }
        return v;
    }
    __device__ __forceinline__ void store(float (*s)[F::PITCH], const f32x4& v) const {
        const int t = threadIdx.x, along = t % PER_ROW * 4, across = t / PER_ROW;
        if (K_CONTIGUOUS) {
#pragma unroll
            for (int i = 0; i < 4; ++i) s[along + i][across] = v[i];
        } else {
            *reinterpret_cast<f32x4*>(&s[across][along]) = v;
        }
    }
};

// acc[i][j] += the products of 16-row block i and 16-column block j of the wave's quarter; a lane's four values are neighbouring
// columns of one row
template <typename F, typename OA, typename OB>
__device__ __forceinline__ void multiply(F& s, const OA& a, const OB& b, int K, f32x4 (&acc)[F::NB][F::NB]) {
    constexpr int STEP = F::STEP, AHEAD = F::AHEAD, NB = F::NB;
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int m0 = (wave >> 1) * (F::SIDE / 2) + (lane & 15), n0 = (wave & 1) * (F::SIDE / 2) + (lane & 15);
    f32x4 va[AHEAD], vb[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) va[j] = a.load(j * STEP), vb[j] = b.load(j * STEP);
    __syncthreads();  // (what was multiplied before has been read)
    for (int k0 = 0; k0 < K; k0 += AHEAD * STEP) {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (k0 + j * STEP >= K) break;
            float(*const sa)[F::PITCH] = s.a[j & 1], (*const sb)[F::PITCH] = s.b[j & 1];
            a.store(sa, va[j]);
            b.store(sb, vb[j]);
            __syncthreads();
            va[j] = a.load(k0 + (j + AHEAD) * STEP), vb[j] = b.load(k0 + (j + AHEAD) * STEP);
#pragma unroll
            for (int k = 0; k < STEP; k += 4) {
                const int kk = k + (lane >> 4);
                float fa[NB], fb[NB];
#pragma unroll
                for (int i = 0; i < NB; ++i) fa[i] = sa[kk][m0 + 16 * i], fb[i] = sb[kk][n0 + 16 * i];
#pragma unroll
                for (int i = 0; i < NB; ++i)
#pragma unroll
                    for (int q = 0; q < NB; ++q) acc[i][q] = __builtin_amdgcn_mfma_f32_16x16x4f32(fb[q], fa[i], acc[i][q], 0, 0, 0);
            }
        }
    }
}

template <typename T>
__device__ __forceinline__ void put4(T* p, const f32x4& v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = Store<T>::from_f32(v[i]);
}

template <typename F, typename T, int OP>
__global__ __launch_bounds__(kThreads) void grad_rows_kernel(const GradArgs g) {
    constexpr int TILE = F::SIDE, NB = F::NB;
    __shared__ F s;
    const int K = OP == GRAD_DX ? g.F : g.d, N = OP == GRAD_DX ? g.d : g.F;
    int lo, hi, e, row0, row_end, nt;
    group_bounds(g.offsets, g.E, g.P, lo, hi);
    lo = min(max(lo, 0), g.P), hi = min(max(hi, lo), g.P);
    if (!find_tile(lo, hi, g.E, TILE, [&](int) { return (N + TILE - 1) / TILE; }, e, row0, row_end, nt)) return;
    const int n0 = nt * TILE;
    const size_t at_w = (size_t)e * g.d * g.F;
    const int rows = min(TILE, row_end - row0), cols = min(TILE, N - n0);
    f32x4 acc[NB][NB] = {}, up[NB][NB] = {}, dh[NB][NB] = {};
    if (OP == GRAD_ACT) {
        const Operand<F, T, true> a{static_cast<const T*>(g.x), g.d, rows, K, row0};
        const Operand<F, T, true> b{static_cast<const T*>(g.w_gate) + at_w, g.d, cols, K, n0}, b1{static_cast<const T*>(g.w_up) + at_w, g.d, cols, K, n0};
        multiply(s, a, b, K, acc);
        multiply(s, a, b1, K, up);
        const Operand<F, T, true> a2{static_cast<const T*>(g.gy), g.d, rows, K, row0};
        const Operand<F, T, false> b2{static_cast<const T*>(g.w_down) + at_w, g.F, cols, K, n0};
        multiply(s, a2, b2, K, dh);
    } else {
        const Operand<F, T, true> a{static_cast<const T*>(g.da), g.F, rows, K, row0}, a1{static_cast<const T*>(g.db), g.F, rows, K, row0};
        const Operand<F, T, false> b{static_cast<const T*>(g.w_gate) + at_w, g.d, cols, K, n0}, b1{static_cast<const T*>(g.w_up) + at_w, g.d, cols, K, n0};
        multiply(s, a, b, K, acc);
        multiply(s, a1, b1, K, acc);
    }
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int r = (wave >> 1) * (TILE / 2) + i * 16 + (lane & 15), c = (wave & 1) * (TILE / 2) + j * 16 + (lane >> 4) * 4;
            if (r >= rows || c >= cols) continue;
            const size_t at = (size_t)(row0 + r) * N + n0 + c;
            if (OP == GRAD_ACT) {
                f32x4 h, da, db;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const ActGrad v = act_grad(acc[i][j][q], up[i][j][q], dh[i][j][q]);
                    h[q] = v.h, da[q] = v.da, db[q] = v.db;
                }
                put4(static_cast<T*>(g.da) + at, da);
                put4(static_cast<T*>(g.db) + at, db);
                put4(static_cast<T*>(g.h) + at, h);
            } else {
                put4(static_cast<T*>(g.gx) + at, acc[i][j]);
            }
        }
}

// blockIdx.y: expert, z: which of the three gradients
template <typename F, typename T>
__global__ __launch_bounds__(kThreads) void grad_weights_kernel(const GradArgs g) {
    constexpr int TILE = F::SIDE, NB = F::NB;
    __shared__ F s;
    const int e = blockIdx.y, which = blockIdx.z;
    const int M = which == 2 ? g.d : g.F, N = which == 2 ? g.F : g.d;
    T* const out = static_cast<T*>(which == 0 ? g.gw_gate : which == 1 ? g.gw_up : g.gw_down);
    if (!out) return;
    const int mt_all = (M + TILE - 1) / TILE, nt = quick_div(blockIdx.x, mt_all), mt = blockIdx.x - nt * mt_all;
    const int m0 = mt * TILE, n0 = nt * TILE;
    if (n0 >= N) return;
    const int lo = g.P ? min(max(g.offsets[e], 0), g.P) : 0, hi = g.P ? min(max(g.offsets[e + 1], lo), g.P) : 0;
    const int rows = min(TILE, M - m0), cols = min(TILE, N - n0), K = hi - lo;
    f32x4 acc[NB][NB] = {};
    if (K > 0) {
        const T* const left = static_cast<const T*>(which == 0 ? g.da : which == 1 ? g.db : g.gy) + (size_t)lo * M;
        const T* const right = static_cast<const T*>(which == 2 ? g.h : g.x) + (size_t)lo * N;
        const Operand<F, T, false> a{left, M, rows, K, m0}, b{right, N, cols, K, n0};
        multiply(s, a, b, K, acc);
    }
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int r = (wave >> 1) * (TILE / 2) + i * 16 + (lane & 15), c = (wave & 1) * (TILE / 2) + j * 16 + (lane >> 4) * 4;
            if (r < rows && c < cols) put4(out + (size_t)e * M * N + (size_t)(m0 + r) * N + n0 + c, acc[i][j]);
        }
}

template <typename F, typename T>
int run_tiles(const GradArgs& g, GradOp op, hipStream_t st) {
    constexpr int TILE = F::SIDE;
    if (op == GRAD_WEIGHTS) {
        const unsigned tiles = (unsigned)((g.d + TILE - 1) / TILE) * ((g.F + TILE - 1) / TILE);
        hipLaunchKernelGGL((grad_weights_kernel<F, T>), dim3(tiles, g.E, 3), dim3(kThreads), 0, st, g);
        return launch_status();
    }
    const int N = op == GRAD_DX ? g.d : g.F;
    const int grid = find_tile_grid(m_tiles_bound(g.P, g.E, TILE) * ((N + TILE - 1) / TILE), 0);
    const auto kern = op == GRAD_ACT ? grad_rows_kernel<F, T, GRAD_ACT> : grad_rows_kernel<F, T, GRAD_DX>;
    hipLaunchKernelGGL(kern, dim3(grid), dim3(kThreads), 0, st, g);
    return launch_status();
}
template <typename T>
int run_plain(const GradArgs& g, GradOp op, hipStream_t st) {
    const int N = op == GRAD_DX ? g.d : g.F;
    const long long tiles = op == GRAD_WEIGHTS ? 3ll * g.E * ((g.d + 63) / 64) * ((g.F + 63) / 64) : (long long)m_tiles_bound(g.P, g.E, 64) * ((N + 63) / 64);
    return tiles <= (op == GRAD_WEIGHTS ? kFewWeightTiles : kFewRowTiles) ? run_tiles<Form<32>, T>(g, op, st) : run_tiles<Form<64>, T>(g, op, st);
}

struct GradLayout {
    size_t da, db, h, parts, total;
};
GradLayout grad_layout(const moe_shape& s) {
    const size_t hidden = round_up((size_t)s.n_tokens * s.top_k * s.d_ff * elt_size(s.act_dtype), 256);
    const size_t parts = s.act_dtype == MOE_BF16 ? round_up(grad_parts_bytes((long long)s.n_tokens * s.top_k, s.d_model), 256) : 0;
    return GradLayout{0, hidden, 2 * hidden, 3 * hidden, 3 * hidden + parts};
}

int validate_grad(const moe_shape* s) {
    const int rc = validate_shape(s);
    if (rc != MOE_OK) return rc;
    // a launch has fewer than 2^32 threads: tiles of 64 by 64 of the rows' products, strips of 256 hidden columns by tiles across d of the weights'
    const long long tiles_d = (s->d_model + 63) / 64, tiles_f = (s->d_ff + 63) / 64;
    const long long rows = ((long long)s->n_tokens * s->top_k + 63) / 64 + s->n_experts;
    if (s->rank != 0 || s->d_model > (1 << 18) || s->d_ff > (1 << 18) || tiles_d * tiles_f >= (1 << 23) || rows * (tiles_d > tiles_f ? tiles_d : tiles_f) >= (1 << 23) ||
        (s->n_experts * 3ll * ((s->d_ff + 255) / 256) + 8) * 2 * ((s->d_model + 255) / 256) >= (1 << 23))
        return MOE_ERR_UNSUPPORTED;
    return MOE_OK;
}

}  // namespace

size_t dispatch_scratch_bytes(long long T, int E);  // dispatch_rows.hip

int run_grad_plain(const GradArgs& g, GradOp op, int act_dtype, hipStream_t st) {
    return act_dtype == MOE_F32 ? run_plain<float>(g, op, st) : run_plain<bf16_t>(g, op, st);
}

}  // namespace moe

using namespace moe;

extern "C" size_t moe_training_workspace_bytes(const moe_shape* shape) {
    if (validate_grad(shape) != MOE_OK) return 0;
    const size_t sort = round_up(dispatch_scratch_bytes(shape->n_tokens, shape->n_experts), 256), grad = grad_layout(*shape).total;
    return sort > grad ? sort : grad;
}

extern "C" int moe_expert_ffn_backward(const moe_shape* shape, const moe_weights* weights, const void* x_perm, const int32_t* expert_offsets,
                                       const void* grad_y_perm, void* grad_x_perm, void* grad_w_gate, void* grad_w_up, void* grad_w_down,
                                       void* workspace, size_t workspace_bytes, void* stream) {
    int rc = validate_grad(shape);
    if (rc != MOE_OK) return rc;
    const moe_shape& s = *shape;
    const bool any_w = grad_w_gate || grad_w_up || grad_w_down;
    for (const void* p : {(const void*)grad_x_perm, (const void*)grad_w_gate, (const void*)grad_w_up, (const void*)grad_w_down})
        if (!aligned16(p) || (p && (p == x_perm || p == grad_y_perm))) return MOE_ERR_INVALID;
    GradArgs g{};
    g.P = s.n_tokens * s.top_k, g.E = s.n_experts, g.d = s.d_model, g.F = s.d_ff;
    g.gx = grad_x_perm, g.gw_gate = grad_w_gate, g.gw_up = grad_w_up, g.gw_down = grad_w_down;
    hipStream_t st = as_stream(stream);
    if (g.P == 0) return any_w ? run_grad_plain(g, GRAD_WEIGHTS, s.act_dtype, st) : MOE_OK;
    if (!weights || !x_perm || !grad_y_perm || !expert_offsets) return MOE_ERR_INVALID;
    for (const void* p : {weights->w_gate, weights->w_up, weights->w_down})
        if (!p || p == grad_w_gate || p == grad_w_up || p == grad_w_down) return MOE_ERR_INVALID;  // (gradients do not take the weights' place: those are read after them)
    for (const void* p : {weights->w_gate, weights->w_up, weights->w_down, x_perm, grad_y_perm})
        if (!aligned16(p)) return MOE_ERR_INVALID;
    if (reinterpret_cast<uintptr_t>(expert_offsets) & 3u) return MOE_ERR_INVALID;
    const GradLayout l = grad_layout(s);
    if (!workspace || workspace_bytes < l.total) return MOE_ERR_WORKSPACE;
    if (!aligned16(workspace)) return MOE_ERR_INVALID;
    if (!any_w && !grad_x_perm) return MOE_OK;
    char* const ws = static_cast<char*>(workspace);
    g.x = x_perm, g.gy = grad_y_perm, g.w_gate = weights->w_gate, g.w_up = weights->w_up, g.w_down = weights->w_down;
    g.da = ws + l.da, g.db = ws + l.db, g.h = ws + l.h, g.parts = reinterpret_cast<float*>(ws + l.parts), g.offsets = expert_offsets;
    const bool mfma = s.act_dtype == MOE_BF16 && grad_mfma_supported(g);
    auto run = [&](GradOp op) { return mfma ? run_grad_mfma(g, op, st) : run_grad_plain(g, op, s.act_dtype, st); };
    rc = run(GRAD_ACT);
    if (rc == MOE_OK && any_w) rc = run(GRAD_WEIGHTS);
    if (rc == MOE_OK && grad_x_perm) rc = run(GRAD_DX);
    return rc;
}
