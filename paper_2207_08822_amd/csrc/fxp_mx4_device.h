// Device code and host checks of microscaled 4-bit numbers: blocks of 32 elements along a contraction under one power of two.
#pragma once
#include "fxp_serve_device.h"

namespace fxp {

constexpr int kMxBlock = 32, kMxPanel = 256, kMxRowBytes = kMxPanel / 2, kMxRowScales = kMxPanel / kMxBlock;

__host__ __device__ inline int64_t mx_panels(int64_t cols) { return (cols + kMxPanel - 1) / kMxPanel; }

// Place of a block's scale among the eight of its panel: even blocks first.  A lane of the matrix instruction holds block l / 32 of each 64 elements
// (l / 16 of each 128), so that the scales it needs for a panel lie in four bytes of one word.
__host__ __device__ constexpr int mx_scale_place(int block) { return (block & 1) * 4 + (block >> 1); }

// The scale byte of a block whose largest magnitude has the bits m: the smallest power of two 2^(s - 127) under which it is at most 6 = 1.5 * 2^2 (a mantissa above
// 1.5 carries into the exponent); 255 for one with Inf or NaN.
__device__ inline int mx_scale_of(uint32_t m) {
    const int s = max(static_cast<int>((m + 0x3fffffu) >> 23) - 2, 0);
    return m >= 0x7f800000u ? 255 : s;
}
// 2^(127 - s); 0 for the scale that is none
__device__ inline float mx_inverse(int s) { return __uint_as_float(static_cast<uint32_t>(max(254 - s, 0)) << 23); }

// Elements in units of their scale as codes, the first in the lowest bits: a sign, then the magnitude's place in 0, 0.5, 1, 1.5, 2, 3, 4, 6.
// To nearest, ties to even: what the conversion instruction does.
template <int N>
__device__ inline uint32_t mx_nearest(const float (&y)[N]) {
    static_assert(N == 4 || N == 8, "two or four bytes");
    uint32_t r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, y[0], y[1], 1.0f, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, y[2], y[3], 1.0f, 1);
    if constexpr (N == 8) {
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, y[4], y[5], 1.0f, 2);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, y[6], y[7], 1.0f, 3);
    }
    return r;
}
// Stochastic: a magnitude m as a fixed-point number whose upper part is the code, 22 bits behind the point.  From 1 on that is a float's bits less those of
// 2^-1 (the code counts binades and one mantissa bit), below it is m * 2^23: of the two and 2^23 the median, because from 1 on
// it is 2^23 <= the first <= the second, and below the first <= the second < 2^23.  A carry out of low + 2^22 - 1 - r (`add`) is r < low.  NaN, in a block that is none, gives
// some code.
__device__ inline uint32_t mx_stochastic(float m, uint32_t add) {
    const int line = static_cast<int>(m * 8388608.0f), bits = static_cast<int>(__float_as_uint(m)) - (252 << 22);
    int t;
    asm("v_med3_i32 %0, %1, %2, %3" : "=v"(t) : "v"(line), "v"(bits), "s"(1 << 23));
    return (static_cast<uint32_t>(t) + add) >> 22 & 7u;
}

// largest of four neighbouring lanes, in all of them
template <int CTRL>
__device__ inline uint32_t max_dpp(uint32_t m) {
    return max(m, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(m), CTRL, 0xf, 0xf, false)));
}
__device__ inline uint32_t max_of_4(uint32_t m) { return max_dpp<0x4e>(max_dpp<0xb1>(m)); }       // neighbours, then pairs
__device__ inline uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
// bits of the largest magnitude of a block of which each of eight neighbouring lanes has four elements
__device__ inline uint32_t mx_max_of_8(const float (&x)[4]) {
    return max_dpp<0x141>(max_of_4(max(max(magnitude(x[0]), magnitude(x[1])), max(magnitude(x[2]), magnitude(x[3])))));      // row_half_mirror
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
bool mx4_is_fused(int64_t M);
int mx4_fused_launch(int type, const void* x, int64_t ldx, int64_t M, const fxp_mx4& B, void* y, int64_t ldy, hipStream_t s);
int mx4_gemm_launch(const fxp_mx4& A, const fxp_mx4& B, int type, void* C, int64_t ldc, void* ws, hipStream_t s);
// two of them with outputs without gaps, in a workspace that is enough for each
int mx4_gemm_launch2(const fxp_mx4& A0, const fxp_mx4& B0, void* C0, const fxp_mx4& A1, const fxp_mx4& B1, void* C1, int type, void* ws, hipStream_t s);

}  // namespace fxp
