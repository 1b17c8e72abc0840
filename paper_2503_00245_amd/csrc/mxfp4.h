// Microscaled 4-bit floating point: arithmetic of a block of 32 values, and the layout of operands in
// which a matrix instruction's lanes find their 16 bytes side by side (internal).
#pragma once

#include "common.h"
#include "moe_quantised.h"

namespace moe {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kMxBlock = 32;        // values that share a scale
constexpr int kMxUnit = 256;        // columns of a unit: two k-steps of 128 of v_mfma_scale_f32_16x16x128_f8f6f4
constexpr int kMxCodes = 32 * kMxUnit / 2, kMxScales = 32 * kMxUnit / kMxBlock;  // bytes of a unit of 32 rows

// An operand is cut into blocks of 32 rows by units of 256 columns.  Codes of a unit: [k-step c of 2][tile t of 2]
// [lane 64][16 bytes]; lane l holds 32 codes of row l % 16 of the tile, columns 128 c + 32 (l / 16) ...
// Scales of a unit: [lane][4 bytes], byte 2 c + t being that of the lane's 32 codes: one dword is what four matrix
// instructions take by byte select.  Rows and columns are padded with zeros to whole units.
// Activations (operand B, whose rows become the columns of the result): tile t holds rows 16 t ... of the block.
// Weights (operand A): row m of tile t is row 8 (m / 4) + 4 t + m % 4 of the block, so that a lane's four results
// of each of the two tiles are eight neighbours of an output row: one dword of codes or 32 bytes of fp32.
__host__ __device__ constexpr int mx_blocks(int rows) { return (rows + 31) / 32; }
__host__ __device__ constexpr int mx_units(int cols) { return (cols + kMxUnit - 1) / kMxUnit; }

__device__ __forceinline__ int mx_weight_row(int m, int t) { return 8 * (m >> 2) + 4 * t + (m & 3); }

// Scale byte of a block whose largest magnitude has these bits (of an fp32): 2^(b - 127) brings it to [4, 8)
__device__ __forceinline__ int mx_scale_byte(unsigned max_bits) {
    const int e = max_bits >> 23;
    return e == 255 ? 255 : max(e - 2, 0);
}
// 2^(b - 127): b = 0 is a subnormal number
__device__ __forceinline__ float mx_scale(int b) { return __int_as_float(b > 0 ? b << 23 : 1 << 22); }

// Eight values over a scale of the given byte as eight codes (round to nearest even, saturating: the
// instruction's own rounding)
__device__ __forceinline__ unsigned mx_codes8(const float (&v)[8], int b) {
#if defined(__HIP_DEVICE_COMPILE__)
    const float s = mx_scale(b);
    unsigned r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0], v[1], s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2], v[3], s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4], v[5], s, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6], v[7], s, 3);
    return r;
#else
    return 0;
#endif
}

// A lane's 32 values of a row, quantised: the operand of a k-step and its scale
template <typename T>
__device__ __forceinline__ void mx_quantise_32(const typename Store<T>::vec_t (&v)[32 / Store<T>::VEC], i32x4& codes, int& scale) {
    typedef Store<T> S;
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) m = max(m, (unsigned)__float_as_int(S::get(v[i / S::VEC], i % S::VEC)) & 0x7fffffffu);
    scale = mx_scale_byte(m);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = S::get(v[(w * 8 + i) / S::VEC], (w * 8 + i) % S::VEC);
        codes[w] = (int)mx_codes8(f, scale);
    }
}

// Eight codes as the values that they stand for; scale byte 255: NaN
__device__ __forceinline__ void mx_values8(unsigned codes, int b, float (&v)[8]) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const float s = mx_scale(b);
    f32x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 1),
                  __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 3)};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = b == 255 ? __int_as_float(0x7fc00000) : p[i / 2][i % 2];
#endif
}

__device__ __forceinline__ unsigned mx_abs_max(const float (&v)[8]) {
    // as whole numbers: a NaN is above every other magnitude and survives
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, (unsigned)__float_as_int(v[i]) & 0x7fffffffu);
    return m;
}

// Largest of the four lanes l, l ^ 16, l ^ 32, l ^ 48 (m >= 0), in all of them: rows of 16 lanes, then halves, change places between two
// registers, so that nothing goes through LDS
__device__ __forceinline__ int mx_max_of_rows(int m) {
#if defined(__HIP_DEVICE_COMPILE__)
    const auto rows = __builtin_amdgcn_permlane16_swap(m, m, false, false);
    m = max((int)rows[0], (int)rows[1]);
    const auto halves = __builtin_amdgcn_permlane32_swap(m, m, false, false);
    return max((int)halves[0], (int)halves[1]);
#else
    return m;
#endif
}

// Eight hidden columns (columns 32 fb + 8 (lane / 16) ..., row lane % 16 of tile n of block sb), quantised, into a matrix of `units`
// units a block: a dword of codes a lane, and a byte of scale for four lanes.
__device__ __forceinline__ void mx_store_hidden(const float (&f)[8], char* __restrict__ codes, char* __restrict__ scales, int units, int sb, int n, int fb, int lane) {
    const int b = mx_scale_byte(mx_max_of_rows((int)mx_abs_max(f))), c = fb >> 2, at = (fb & 3) * 16 + (lane & 15);
    const size_t unit = (size_t)sb * units + (c >> 1);
    *reinterpret_cast<unsigned*>(codes + unit * kMxCodes + ((c & 1) * 2 + n) * 1024 + at * 16 + (lane >> 4) * 4) = mx_codes8(f, b);
    if (lane < 16) scales[unit * kMxScales + at * 4 + (c & 1) * 2 + n] = (char)b;
}
// The same of a product that is not quantised: eight neighbours of row 32 sb + 16 n + lane % 16 of fp32 [.., N].  (fp32 whatever the
// activations' type: rounded to bf16 here, rows of experts that cancel would leave their roundings in the gated sum.)
__device__ __forceinline__ void mx_store_rows(const float (&f)[8], char* __restrict__ out, int N, int sb, int n, int fb, int lane) {
    const int col = fb * 32 + (lane >> 4) * 8;
    if (col >= N) return;
    f32x4* const y = reinterpret_cast<f32x4*>(reinterpret_cast<float*>(out) + ((size_t)sb * 32 + n * 16 + (lane & 15)) * N + col);
    y[0] = f32x4{f[0], f[1], f[2], f[3]};
    y[1] = f32x4{f[4], f[5], f[6], f[7]};
}

// D (16 x 16, fp32) += A (16 x 128) B^T; SA, SB: which byte of the dwords sa, sb scales the lane's 32 codes
template <int SA, int SB>
__device__ __forceinline__ f32x4 mx_mfma(const i32x4& a, const i32x4& b, const f32x4& c, int sa, int sb) {
#if defined(__HIP_DEVICE_COMPILE__)
    const i32x8 a8 = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);
    const i32x8 b8 = __builtin_shufflevector(b, b, 0, 1, 2, 3, -1, -1, -1, -1);
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, SA, sa, SB, sb);
#else
    return c;
#endif
}

// A unit: 32 rows of weights (tiles t of the first index) by 32 of activations.  w, x: [k-step][tile]
__device__ __forceinline__ void mx_unit(f32x4 (&acc)[2][2], const i32x4 (&w)[2][2], const i32x4 (&x)[2][2], int sw, int sx) {
    acc[0][0] = mx_mfma<0, 0>(w[0][0], x[0][0], acc[0][0], sw, sx);
    acc[0][1] = mx_mfma<0, 1>(w[0][0], x[0][1], acc[0][1], sw, sx);
    acc[1][0] = mx_mfma<1, 0>(w[0][1], x[0][0], acc[1][0], sw, sx);
    acc[1][1] = mx_mfma<1, 1>(w[0][1], x[0][1], acc[1][1], sw, sx);
    acc[0][0] = mx_mfma<2, 2>(w[1][0], x[1][0], acc[0][0], sw, sx);
    acc[0][1] = mx_mfma<2, 3>(w[1][0], x[1][1], acc[0][1], sw, sx);
    acc[1][0] = mx_mfma<3, 2>(w[1][1], x[1][0], acc[1][0], sw, sx);
    acc[1][1] = mx_mfma<3, 3>(w[1][1], x[1][1], acc[1][1], sw, sx);
}

// ---- launchers ---------------------------------------------------------------------------------------
struct MxLayout {  // byte offsets of a workspace; every region starts 256-byte aligned
    size_t idx, gate, logits, slot, starts, offsets, perm, sort, xq, hq, y, total;
    int blocks;    // blocks of 32 rows that hold the pairs of all experts, each expert's from a block of its own
};
MxLayout mx_layout(const moe_shape& s);
int launch_mx_experts(const moe_shape& s, const moe_mxfp4_weights& w, const void* x, const int32_t* idx, const float* gate, void* y,
                      const MxLayout& l, char* ws, hipStream_t st);
// Few pairs: two launches, without a dispatch (mxfp4_few.hip).  Whole layer, us, weights cold, in these / in four launches: 2048 / 5632, 2 of 8 experts:
// one token 14.6 / 23.8, two 19.7 / 26.7, four 33.2 / 39.3; 1024 / 2816, 4 of 16 experts, two tokens 15.9 / 19.5.  With up to 16 pairs, eight tokens of the
// former 42.2 / 42.7, four of the latter 24.7 / 22.0.
constexpr int kMxFewPairs = 8;
inline bool mx_few(const moe_shape& s) { return (long long)s.n_tokens * s.top_k <= kMxFewPairs; }
int launch_mx_few(const moe_shape& s, const moe_mxfp4_weights& w, const void* x, const int32_t* idx, const float* gate, void* y, const MxLayout& l, char* ws,
                  hipStream_t st);
// Products of some rows an expert (mxfp4_stream.hip), the same arguments
int launch_mx_stream(bool swiglu, const void* w0, const void* w1, const char* a, char* out, const int32_t* starts, int P, int E,
                     int all_blocks, int N, int K, hipStream_t st);
// Products of many rows (mxfp4_gemm.hip): swiglu: hidden rows (w0 gate, w1 up), else rows in fp32 (w0).  bs: rows of a tile, 256, 128 or 64
int launch_mx_gemm(bool swiglu, const void* w0, const void* w1, const char* a, char* out, const int32_t* starts, int P, int E,
                   int all_blocks, int N, int K, int bs, hipStream_t st);
int launch_router_logits(const moe_shape& s, const void* x, const float* rw, const float* rb, float* logits, hipStream_t st);
int launch_route_scored(const moe_route_config& c, int T, int E, int k, const float* logits, const float* bias, int32_t* idx, float* gate,
                        float* scores, hipStream_t st);
// MOE_OK, MOE_ERR_INVALID or MOE_ERR_UNSUPPORTED
int validate_route(const moe_route_config* c, int T, int E, int k);

}  // namespace moe
