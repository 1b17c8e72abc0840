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
// of each of the two tiles are eight neighbours of an output row: one dword of codes or 16 bytes of bf16.
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

// ---- launchers ---------------------------------------------------------------------------------------
struct MxLayout {  // byte offsets of a workspace; every region starts 256-byte aligned
    size_t idx, gate, logits, slot, starts, xq, hq, y, total;
    int blocks;    // blocks of 32 rows that hold the pairs of all experts, each expert's from a block of its own
};
MxLayout mx_layout(const moe_shape& s);
int launch_mx_experts(const moe_shape& s, const moe_mxfp4_weights& w, const void* x, const int32_t* idx, const float* gate, void* y,
                      const MxLayout& l, char* ws, hipStream_t st);
int launch_router_logits(const moe_shape& s, const void* x, const float* rw, const float* rb, float* logits, hipStream_t st);
int launch_route_scored(const moe_route_config& c, int T, int E, int k, const float* logits, const float* bias, int32_t* idx, float* gate,
                        float* scores, hipStream_t st);
// MOE_OK, MOE_ERR_INVALID or MOE_ERR_UNSUPPORTED
int validate_route(const moe_route_config* c, int T, int E, int k);

}  // namespace moe
