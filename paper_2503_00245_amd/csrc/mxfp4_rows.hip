// Rows to microscaled 4-bit floating point and back, and the layout of weights for the expert products.
#include <algorithm>
#include <type_traits>

#include "mxfp4.h"

namespace moe {

namespace {

constexpr int kThreads = 256;
constexpr int kSteps = 4;  // requests of a lane in flight

template <typename T>
struct Eight;  // eight neighbours of a row
template <>
struct Eight<bf16_t> {
    bf16x8 v;
    template <bool PAST>
    __device__ __forceinline__ void load(const bf16_t* p) {
        const bf16x8* q = reinterpret_cast<const bf16x8*>(p);
        v = PAST ? __builtin_nontemporal_load(q) : *q;
    }
    __device__ __forceinline__ void get(float (&o)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = (float)v[i];
    }
    static __device__ __forceinline__ void store(bf16_t* p, const float (&o)[8]) {
        bf16x8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (bf16_t)o[i];
        *reinterpret_cast<bf16x8*>(p) = v;
    }
};
template <>
struct Eight<float> {
    f32x4 v[2];
    template <bool PAST>
    __device__ __forceinline__ void load(const float* p) {
        const f32x4* q = reinterpret_cast<const f32x4*>(p);
        v[0] = PAST ? __builtin_nontemporal_load(q) : q[0];
        v[1] = PAST ? __builtin_nontemporal_load(q + 1) : q[1];
    }
    __device__ __forceinline__ void get(float (&o)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = v[i / 4][i % 4];
    }
    static __device__ __forceinline__ void store(float* p, const float (&o)[8]) {
        reinterpret_cast<f32x4*>(p)[0] = f32x4{o[0], o[1], o[2], o[3]};
        reinterpret_cast<f32x4*>(p)[1] = f32x4{o[4], o[5], o[6], o[7]};
    }
};

// Where lane slot i of a run of rows lies: slots are eight values wide, four to a block, `slots` to a row.
// FLAT: rows are whole blocks, so that all of them are one long row.
struct Place {
    long long at, block;  // first value, block of scales
    bool live;            // there are eight values here (a short last block has fewer slots)
};
template <bool FLAT>
__device__ __forceinline__ Place place(long long row0, unsigned i, unsigned n, int cols, int slots) {
    if (FLAT) return Place{row0 * cols + (long long)i * 8, row0 * (cols / kMxBlock) + (i >> 2), i < n};
    const unsigned r = i / (unsigned)slots, s = i - r * (unsigned)slots;
    return Place{(row0 + r) * cols + (int)s * 8, (row0 + r) * (slots / 4) + (s >> 2), i < n && (int)s * 8 < cols};
}

// One pass: a lane holds eight values, four lanes a block; its largest magnitude takes two register exchanges
// between neighbours.  Bound by memory: 16 (fp32: 32) bytes in and 4.25 out for eight values.  PAST: the values are read past the
// caches, from 128 MB on, of which little can be there: 92 M of bf16 36.7 us, 41.9 without; 4 M 3.2 and 3.0, 17 M 8.3 and 8.1.
template <typename T, bool FLAT, bool PAST>
__global__ __launch_bounds__(kThreads) void mx_quantize_kernel(const T* __restrict__ x, unsigned* __restrict__ codes, uint8_t* __restrict__ scales,
                                                               long long rows, int rows_a_launch, int cols, int slots) {
    const long long row0 = (long long)blockIdx.y * rows_a_launch;
    const unsigned n = (unsigned)min((long long)rows_a_launch, rows - row0) * (unsigned)slots;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned i0 = (blockIdx.x * (kThreads / 64) + wave) * (64 * kSteps) + lane;
    Eight<T> v[kSteps];
    Place p[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        p[s] = place<FLAT>(row0, i0 + s * 64, n, cols, slots);
        if (p[s].live) v[s].template load<PAST>(x + p[s].at);
    }
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (p[s].live) v[s].get(f);
        int m = (int)mx_abs_max(f);
        m = max(m, dpp_i32<kDppSwap1>(m));
        m = max(m, dpp_i32<kDppSwap2>(m));
        const int b = mx_scale_byte(m);
        if (p[s].live) {
            codes[p[s].at >> 3] = mx_codes8(f, b);
            if ((lane & 3) == 0) scales[p[s].block] = (uint8_t)b;
        }
    }
}

template <typename T, bool FLAT>
__global__ __launch_bounds__(kThreads) void mx_dequantize_kernel(const unsigned* __restrict__ codes, const uint8_t* __restrict__ scales, T* __restrict__ x,
                                                                 long long rows, int rows_a_launch, int cols, int slots) {
    const long long row0 = (long long)blockIdx.y * rows_a_launch;
    const unsigned n = (unsigned)min((long long)rows_a_launch, rows - row0) * (unsigned)slots;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned i0 = (blockIdx.x * (kThreads / 64) + wave) * (64 * kSteps) + lane;
    unsigned c[kSteps];
    int b[kSteps];
    Place p[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        p[s] = place<FLAT>(row0, i0 + s * 64, n, cols, slots);
        if (p[s].live) {
            c[s] = codes[p[s].at >> 3];
            b[s] = scales[p[s].block];
        }
    }
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        if (!p[s].live) continue;
        float f[8];
        mx_values8(c[s], b[s], f);
        Eight<T>::store(x + p[s].at, f);
    }
}

// A lane's 16 bytes of codes, from a row-major matrix: four times eight neighbours, of which those past the row's
// end, and rows past the matrix's end, are zeros.
__global__ __launch_bounds__(kThreads) void mx_pack_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, char* __restrict__ packed,
                                                           int n_matrices, int rows, int cols) {
    const int blocks = mx_blocks(rows), units = mx_units(cols);
    const long long total = (long long)n_matrices * blocks * units;  // units of all matrices, a workgroup each
    const int lane = threadIdx.x & 63, ct = threadIdx.x >> 6, c = ct >> 1, t = ct & 1;
    static_assert(kThreads == 256, "a wave for each of the unit's four tiles");
    const int scale_cols = (cols + kMxBlock - 1) / kMxBlock;
    __shared__ uint8_t s_scale[4][64];
    for (long long at = blockIdx.x; at < total; at += gridDim.x) {
        const int u = (int)(at % units);
        const long long mb = at / units;
        const int rb = (int)(mb % blocks);
        const long long m = mb / blocks;
        const int r = rb * 32 + mx_weight_row(lane & 15, t), col = u * kMxUnit + c * 128 + (lane >> 4) * 32;
        i32x4 v{0, 0, 0, 0};
        uint8_t b = 0;
        if (r < rows) {
            const unsigned* src = reinterpret_cast<const unsigned*>(codes + ((size_t)m * rows + r) * (cols / 2));
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (col + 8 * i < cols) v[i] = (int)src[col / 8 + i];
            if (col < cols) b = scales[((size_t)m * rows + r) * scale_cols + col / 32];
        }
        *reinterpret_cast<i32x4*>(packed + (size_t)at * kMxCodes + ct * 1024 + lane * 16) = v;
        s_scale[ct][lane] = b;
        __syncthreads();
        if (threadIdx.x < 64) {
            const unsigned d = s_scale[0][lane] | s_scale[1][lane] << 8 | s_scale[2][lane] << 16 | (unsigned)s_scale[3][lane] << 24;
            *reinterpret_cast<unsigned*>(packed + (size_t)total * kMxCodes + (size_t)at * kMxScales + lane * 4) = d;
        }
        __syncthreads();
    }
}

// Grid of a pass over rows: x the lane slots of up to 2^28 of them, y runs of rows
struct RowsGrid {
    dim3 grid;
    int rows_a_launch, slots;
    bool flat;
};
RowsGrid rows_grid(long long rows, int cols) {
    RowsGrid g;
    g.flat = cols % kMxBlock == 0;
    g.slots = (cols + kMxBlock - 1) / kMxBlock * 4;
    g.rows_a_launch = (int)std::min<long long>(rows, (1 << 28) / g.slots);
    const unsigned n = (unsigned)g.rows_a_launch * g.slots, per = kThreads * kSteps;
    g.grid = dim3((n + per - 1) / per, (unsigned)((rows + g.rows_a_launch - 1) / g.rows_a_launch));
    return g;
}

int check_rows(const void* x, const void* codes, const void* scales, long long rows, int cols, int act_dtype) {
    if (rows < 0 || cols < 1) return MOE_ERR_INVALID;
    if (act_dtype != MOE_F32 && act_dtype != MOE_BF16) return MOE_ERR_UNSUPPORTED;
    if (cols % 8 || cols > (1 << 24) || rows > (1ll << 40) / cols) return MOE_ERR_UNSUPPORTED;
    if (rows == 0) return MOE_OK;
    if (!x || !codes || !scales || !aligned16(x) || (reinterpret_cast<uintptr_t>(codes) & 3)) return MOE_ERR_INVALID;
    return MOE_OK;
}

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" int moe_mxfp4_quantize(const void* x, int64_t rows, int32_t cols, int32_t act_dtype, uint8_t* codes, uint8_t* scales, void* stream) {
    const int rc = check_rows(x, codes, scales, rows, cols, act_dtype);
    if (rc != MOE_OK || rows == 0) return rc;
    const RowsGrid g = rows_grid(rows, cols);
    auto launch = [&](auto kern, auto* src) {
        hipLaunchKernelGGL(kern, g.grid, dim3(kThreads), 0, as_stream(stream), src, reinterpret_cast<unsigned*>(codes), scales, (long long)rows,
                           g.rows_a_launch, cols, g.slots);
    };
    auto launch_type = [&](auto* src) {
        typedef typename std::remove_const<typename std::remove_pointer<decltype(src)>::type>::type T;
        const bool past = (size_t)rows * cols * sizeof(T) >= (128u << 20);
        if (g.flat) past ? launch(mx_quantize_kernel<T, true, true>, src) : launch(mx_quantize_kernel<T, true, false>, src);
        else past ? launch(mx_quantize_kernel<T, false, true>, src) : launch(mx_quantize_kernel<T, false, false>, src);
    };
    if (act_dtype == MOE_F32) launch_type(static_cast<const float*>(x));
    else launch_type(static_cast<const bf16_t*>(x));
    return launch_status();
}

extern "C" int moe_mxfp4_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int32_t cols, int32_t act_dtype, void* x, void* stream) {
    const int rc = check_rows(x, codes, scales, rows, cols, act_dtype);
    if (rc != MOE_OK || rows == 0) return rc;
    const RowsGrid g = rows_grid(rows, cols);
    auto launch = [&](auto kern, auto* dst) {
        hipLaunchKernelGGL(kern, g.grid, dim3(kThreads), 0, as_stream(stream), reinterpret_cast<const unsigned*>(codes), scales, dst, (long long)rows,
                           g.rows_a_launch, cols, g.slots);
    };
    if (act_dtype == MOE_F32)
        g.flat ? launch(mx_dequantize_kernel<float, true>, (float*)x) : launch(mx_dequantize_kernel<float, false>, (float*)x);
    else
        g.flat ? launch(mx_dequantize_kernel<bf16_t, true>, (bf16_t*)x) : launch(mx_dequantize_kernel<bf16_t, false>, (bf16_t*)x);
    return launch_status();
}

extern "C" size_t moe_mxfp4_packed_bytes(int32_t n_matrices, int32_t rows, int32_t cols) {
    if (n_matrices < 1 || rows < 1 || cols < 1 || rows % 8 || cols % 8 || rows > (1 << 24) || cols > (1 << 24)) return 0;
    const unsigned __int128 n = (unsigned __int128)n_matrices * mx_blocks(rows) * mx_units(cols) * (kMxCodes + kMxScales);
    return n >> 46 ? 0 : (size_t)n;
}

extern "C" int moe_mxfp4_pack(const uint8_t* codes, const uint8_t* scales, int32_t n_matrices, int32_t rows, int32_t cols, void* packed, void* stream) {
    if (n_matrices < 1 || rows < 1 || cols < 1 || !codes || !scales || !packed || !aligned16(packed) || (reinterpret_cast<uintptr_t>(codes) & 3))
        return MOE_ERR_INVALID;
    if (!moe_mxfp4_packed_bytes(n_matrices, rows, cols)) return MOE_ERR_UNSUPPORTED;
    const long long units = (long long)n_matrices * mx_blocks(rows) * mx_units(cols);
    hipLaunchKernelGGL(mx_pack_kernel, dim3((unsigned)std::min<long long>(units, 1 << 20)), dim3(kThreads), 0, as_stream(stream), codes, scales,
                       static_cast<char*>(packed), n_matrices, rows, cols);
    return launch_status();
}
