// Device code and host checks of microscaled 4-bit numbers: blocks of 32 elements along a contraction under one power of two.
#pragma once
#include "fxp_serve_device.h"

namespace fxp {

constexpr int kMxBlock = 32, kMxPanel = 256, kMxRowBytes = kMxPanel / 2, kMxRowScales = kMxPanel / kMxBlock;

__host__ __device__ inline int64_t mx_panels(int64_t cols) { return (cols + kMxPanel - 1) / kMxPanel; }

// Place of a block's scale among the eight of its panel: even blocks first.  A lane of the matrix instruction holds block l / 32 of each 64 elements
// (l / 16 of each 128), so that the scales it needs for a panel lie in four bytes of one word.
__host__ __device__ constexpr int mx_scale_place(int block) { return (block & 1) * 4 + (block >> 1); }

// The scale byte of a block whose largest magnitude has the bits m: the smallest power of two 2^(s - 127) under which it is at most 6 = 1.5 * 2^2; 255
// for one with Inf or NaN.
__device__ inline int mx_scale_of(uint32_t m) {
    const int e = static_cast<int>(m >> 23);
    return e == 255 ? 255 : max(e - 2 + ((m & 0x7fffffu) > 0x400000u ? 1 : 0), 0);
}
// 2^(127 - s); 0 for the scale that is none
__device__ inline float mx_inverse(int s) { return __uint_as_float(static_cast<uint32_t>(max(254 - s, 0)) << 23); }

// Four elements in units of their scale as four codes, the first in the lowest bits: a sign, then the magnitude's place in 0, 0.5, 1, 1.5, 2, 3, 4, 6.
// To nearest, ties to even: what the conversion instruction does.
__device__ inline uint32_t mx_nearest4(float a, float b, float c, float d) {
    uint32_t r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, a, b, 1.0f, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, c, d, 1.0f, 1);
    return r & 0xffffu;
}
// Stochastic: the magnitude as a fixed-point number whose upper part is the code, 22 bits behind the point.  From 1 on that is a float's bits less those of
// 2^-126 (the code counts binades and one mantissa bit); below it is |y| * 2^23.  A carry out of low + 2^22 - 1 - r is r < low.
__device__ inline uint32_t mx_stochastic(float y, uint32_t word) {
    const float m = fabsf(y);
    const uint32_t t = m < 1.0f ? static_cast<uint32_t>(m * 8388608.0f) : __float_as_uint(m) - (252u << 22);
    return min((t + ((word >> 10) ^ 0x3fffffu)) >> 22, 7u) | ((__float_as_uint(y) >> 28) & 8u);
}

// two values of a byte of codes
__device__ inline float2 mx_values(uint32_t codes, int byte) {
    typedef float v2f __attribute__((ext_vector_type(2)));
    v2f v;
    switch (byte) {
        case 0: v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 0); break;
        case 1: v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 1); break;
        case 2: v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 2); break;
        default: v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 3); break;
    }
    return make_float2(v[0], v[1]);
}

constexpr int64_t kMxMost = (int64_t{1} << 24) - (1 << 16);     // rows and columns: a panel stays below 2^31 bytes, panels below 65536

inline int check_mx4(const fxp_mx4* q) {
    if (!q) return FXP_ERR_NULL;
    if (q->rows < 0 || q->cols < 0 || q->rows > kMxMost || q->cols > kMxMost) return FXP_ERR_DIMS;
    if (q->rows == 0 || q->cols == 0) return FXP_OK;
    if (!q->data || !q->scales) return FXP_ERR_NULL;
    if (!aligned(q->data, 16) || !aligned(q->scales, 8)) return FXP_ERR_ALIGN;
    return FXP_OK;
}

// One matrix to map: q along its rows and / or t along its columns.
struct Mx4Map {
    const void* x;
    int64_t ld, rows, cols;
    uint8_t *q, *q_scales, *t, *t_scales;
    uint64_t stream_id;
};
// one or two matrices of a type in one launch
int mx4_map_launch(int type, const Mx4Map* jobs, int count, uint64_t seed, int rounding, hipStream_t s);
// C [A.rows, B.rows] = A B^T; ws: mx4_gemm_bytes
size_t mx4_gemm_bytes(int64_t M, int64_t N, int64_t K);
int mx4_gemm_launch(const fxp_mx4& A, const fxp_mx4& B, int type, void* C, int64_t ldc, void* ws, hipStream_t s);

}  // namespace fxp
