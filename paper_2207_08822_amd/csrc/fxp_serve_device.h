// Device code that the serving kernels share: element types, the mapping rounded to nearest, digits of a float row.
#pragma once
#include "fxp_internal.h"

namespace fxp {

typedef int v4i __attribute__((ext_vector_type(4)));

template <int TYPE>
struct Elem;
template <>
struct Elem<FXP_F32> {
    using T = float;
};
template <>
struct Elem<FXP_BF16> {
    using T = __bf16;
};
template <>
struct Elem<FXP_F16> {
    using T = _Float16;
};

inline int elem_size(int type) { return type == FXP_F32 ? 4 : 2; }
inline bool known_type(int type) { return type == FXP_F32 || type == FXP_BF16 || type == FXP_F16; }

// N consecutive elements as floats (exact); `vec`: the address is a multiple of N elements, so N of them are one load
// or, from 32 bytes on, several
template <int TYPE, int N>
__device__ inline void load_elems(const void* base, int64_t at, bool vec, float (&out)[N]) {
    using T = typename Elem<TYPE>::T;
    const T* p = static_cast<const T*>(base) + at;
    if (vec) {
        constexpr int kPiece = N * sizeof(T) < 16 ? N : 16 / static_cast<int>(sizeof(T));
        typedef T Vec __attribute__((ext_vector_type(kPiece)));
#pragma unroll
        for (int i = 0; i < N; i += kPiece) {
            const Vec v = *reinterpret_cast<const Vec*>(p + i);
#pragma unroll
            for (int j = 0; j < kPiece; ++j) out[i + j] = static_cast<float>(v[j]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) out[i] = static_cast<float>(p[i]);
    }
}

// four floats rounded to nearest, to an address that is a multiple of four elements
template <int TYPE>
__device__ inline void store4(void* base, int64_t at, bool vec, const float (&x)[4]) {
    using T = typename Elem<TYPE>::T;
    T* p = static_cast<T*>(base) + at;
    typedef T Vec __attribute__((ext_vector_type(4)));
    if (vec) {
        Vec v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = static_cast<T>(x[j]);
        *reinterpret_cast<Vec*>(p) = v;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) p[j] = static_cast<T>(x[j]);
    }
}

// The mapping of one value under scale e with `cut` = 25 - bits low bits dropped, half up on the magnitude (what
// fxp_map does with FXP_ROUND_NEAREST), as a signed byte.
__device__ inline int map_nearest(float x, int e, int cut) {
    const uint32_t b = __float_as_uint(x), field = (b >> 23) & 0xffu, f = b & 0x7fffffu, sat = (1u << (24 - cut)) - 1u;
    const int d = e - static_cast<int>(max(field, 1u));
    const uint32_t m = (f | (field ? 0x800000u : 0u)) >> min(max(d, 0), 31);
    uint32_t q = min((m + (1u << (cut - 1))) >> cut, sat);
    if (d < 0) q = sat;
    if (field == 255u) q = f == 0u ? sat : 0u;
    return (b >> 31) ? -static_cast<int>(q) : static_cast<int>(q);
}

// a mapped byte brought to a scale larger by d >= 1: half up on the magnitude
__device__ inline int remap_nearest(int q, int d) {
    const int s = min(d, 9);                             // 9: every magnitude becomes 0
    const int m = (abs(q) + (1 << (s - 1))) >> s;
    return q < 0 ? -m : m;
}
__device__ inline uint32_t remap_nearest4(uint32_t four, int d) {
    uint32_t r = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        r |= (static_cast<uint32_t>(remap_nearest(static_cast<int8_t>(four >> (8 * i)), d)) & 0xffu) << (8 * i);
    return r;
}

// bytes j of four words, one after the other
__device__ inline uint32_t bytes_of(uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3, int j) {
    const uint32_t s = static_cast<uint32_t>(j) | (static_cast<uint32_t>(j + 4) << 8);
    return perm(perm(w3, w2, s), perm(w1, w0, s), 0x05040100u);
}

// Digits of 16 integers, most significant first.  Adding 128 in every lower byte makes each lower digit its byte minus 128 (the byte
// with its top bit turned), and carries the rest into the one above it.
template <int ND>
__device__ inline void digits16(const int (&v)[16], v4i (&d)[ND]) {
    constexpr int kBias = ND == 2 ? 0x80 : 0x8080;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = static_cast<uint32_t>(v[4 * t + i] + kBias);
#pragma unroll
        for (int j = 0; j < ND; ++j) {
            const uint32_t by = bytes_of(w[0], w[1], w[2], w[3], ND - 1 - j);
            d[j][t] = static_cast<int>(j == 0 ? by : by ^ 0x80808080u);
        }
    }
}

template <int ND>
struct Digits {
    // largest magnitude: 127 in every digit
    static constexpr int kMost = ND == 2 ? 32639 : 8355711;
    static constexpr int kBits = ND == 2 ? 15 : 23;
};

// exponent of one unit of a row (or group) of floats whose largest magnitude has the bits m: the row stays below 127/128 of the binade
// (2^-7 and a little short of it: rounding must not reach 128 in a digit)
template <int ND>
__device__ inline int unit_of(uint32_t m) {
    return min(max(static_cast<int>((m + 0x10200u) >> 23), 1), 255) - 126 - Digits<ND>::kBits;
}
template <int ND>
__device__ inline int fixed_point(float x, int unit) {
    return min(max(static_cast<int>(rintf(ldexpf(x, -unit))), -Digits<ND>::kMost), Digits<ND>::kMost);
}
// Digits of 16 floats in units of 2^unit; `finite`: no Inf or NaN among the wave's.  Two digits: adding 1.5 * 2^23 rounds to a whole
// number (to even) and leaves it in the low bits of the sum, so that scaling, rounding, conversion and the bias of digits16 are one
// multiply-add (3 instructions an element in place of 9).
template <int ND>
__device__ inline void row_digits(const float (&x)[16], int unit, bool finite, v4i (&d)[ND]) {
    if (ND == 2 && finite) {
        // two factors: one alone passes the largest float for rows of sub-normal numbers
        const float f0 = ldexpf(1.0f, -unit >> 1), f1 = ldexpf(1.0f, -unit - (-unit >> 1));
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(fmaf(x[4 * t + i] * f0, f1, 12582912.0f + 128.0f));
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t by = bytes_of(w[0], w[1], w[2], w[3], 1 - j);
                d[j][t] = static_cast<int>(j == 0 ? by : by ^ 0x80808080u);
            }
        }
    } else {
        int v[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = fixed_point<ND>(x[j], unit);
        digits16<ND>(v, d);
    }
}

__device__ inline v4i mfma_i8(v4i a, v4i b, v4i c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }

// sum over the lanes up to this one, inside the vector ALU (rows of 16 first, then row to row); `add` adds two of them
template <typename F>
__device__ inline uint32_t wave_scan(uint32_t v, F add) {
    auto step = [&](uint32_t x, auto ctrl, auto rows) {
        return add(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), decltype(ctrl)::value, decltype(rows)::value, 0xf, false)));
    };
    using std::integral_constant;
    v = step(v, integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});     // row_shr:1
    v = step(v, integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});     // row_shr:2
    v = step(v, integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});     // row_shr:4
    v = step(v, integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});     // row_shr:8
    v = step(v, integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});     // row_bcast:15 into rows 1 and 3
    v = step(v, integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});     // row_bcast:31 into rows 2 and 3
    return v;
}
__device__ inline uint32_t wave_scan(uint32_t v) {
    return wave_scan(v, [](uint32_t a, uint32_t b) { return a + b; });
}
__device__ inline uint32_t wave_scan_up(uint32_t v) {               // stays at 2^32 - 1 where it would pass that
    return wave_scan(v, [](uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); });
}

// Loads through a buffer descriptor: `bytes` from a uniform address, at a uniform and a lane's offset; 0 bytes: zeros, and no memory access.
__device__ inline auto records(const void* base, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, bytes, 0x00027000);
}
constexpr int kNonTemporal = 2;

struct Run {
    int first, count, page, offset;
};
// whether the tokens, the page and the places of a run exist
__device__ inline bool run_ok(const Run& r, int64_t tokens, int64_t pages) {
    return r.count > 0 && r.count <= FXP_KV_PAGE && r.offset >= 0 && r.offset + r.count <= FXP_KV_PAGE && r.first >= 0 &&
           int64_t{r.first} + r.count <= tokens && r.page >= 0 && r.page < pages;
}

inline int check_cache(const fxp_kv_cache* c) {
    if (!c || !c->kq || !c->vq || !c->ek || !c->ev) return FXP_ERR_NULL;
    if (c->pages <= 0 || c->pages >= (int64_t{1} << 31) || c->heads <= 0 || c->heads > 65535 || c->dim <= 0 || c->dim > 256 ||
        c->dim % 16)
        return FXP_ERR_DIMS;
    if (c->bits < 2 || c->bits > 8) return FXP_ERR_BITS;
    if (!aligned(c->kq, 16) || !aligned(c->vq, 16) || !aligned(c->ek, 4) || !aligned(c->ev, 4)) return FXP_ERR_ALIGN;
    return FXP_OK;
}

// strides of a [tokens, heads, dim] operand; sizes stay far from 2^63
inline bool strides_ok(int64_t token, int64_t head) {
    return token >= 0 && head >= 0 && token < (int64_t{1} << 31) && head < (int64_t{1} << 40);
}

}  // namespace fxp
