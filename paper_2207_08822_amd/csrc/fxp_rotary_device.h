// Device code of rotary positions: the angle of a pair, its cosine and sine, in 32 and in 64 bits.
//
// The angle of pair i at position p is p * f_i, f_i a fixed-point fraction of a turn with 64 bits behind the point: the product modulo 2^64 is the angle
// modulo one turn, with an error of p * 2^-65 turns (2^-34 at the largest position), so that far positions cost no argument reduction and lose
// nothing.  In 32 bits the angle's lower half is cut off, up to 2^-32 turns: 1.5e-9 of the pair's length, where half a step of a cosine near one is 3e-8.  Its two top bits
// (after half a quarter is added) are the quarter, the rest an angle r in [-pi/4, pi/4), for which the Taylor series of
// sine and cosine are summed as far as their terms reach the last place: x^9 and x^10 in 32 bits (next terms 1.8e-9 and 1.2e-10 at pi/4, half a
// step is 3e-8), x^15 and x^16 in 64 (next terms 4.6e-17 and 2e-18, half a step 5.6e-17).
#pragma once
#include "fxp_serve_device.h"

namespace fxp {

__device__ inline uint64_t angle_of(uint64_t turns, int position) { return turns * static_cast<uint64_t>(static_cast<int64_t>(position)); }

// sine and cosine of r, moved on by a number of quarters
template <typename F>
__device__ inline void by_quarters(F sine, F cosine, uint32_t quarter, F& c, F& s) {
    const bool odd = quarter & 1u;
    const F a = odd ? sine : cosine, b = odd ? cosine : sine;
    c = (quarter + 1u) & 2u ? -a : a;
    s = quarter & 2u ? -b : b;
}

__device__ inline void cos_sin(uint64_t angle, float& c, float& s) {
    const uint32_t t = static_cast<uint32_t>(angle >> 32);
    const float x = static_cast<float>(static_cast<int>(t << 2) >> 2) * 1.46291807926715968e-9f;      // 2 pi / 2^32
    const float z = x * x;
    float p = fmaf(z, 2.7557319224e-6f, -1.9841269841e-4f), q = fmaf(z, -2.7557319224e-7f, 2.4801587302e-5f);
    p = fmaf(z, p, 8.3333333333e-3f);
    q = fmaf(z, q, -1.3888888889e-3f);
    p = fmaf(z, p, -1.6666666667e-1f);
    q = fmaf(z, q, 4.1666666667e-2f);
    q = fmaf(z, q, -0.5f);
    by_quarters(fmaf(x * z, p, x), fmaf(z, q, 1.0f), (t + 0x20000000u) >> 30, c, s);
}

__device__ inline void cos_sin(uint64_t angle, double& c, double& s) {
    const double x = static_cast<double>(static_cast<int64_t>(angle << 2) >> 2) * 3.4061215800865545e-19;        // 2 pi / 2^64
    const double z = x * x;
    double p = fma(z, -1.0 / 1307674368000.0, 1.0 / 6227020800.0), q = fma(z, 1.0 / 20922789888000.0, -1.0 / 87178291200.0);
    p = fma(z, p, -1.0 / 39916800.0);
    q = fma(z, q, 1.0 / 479001600.0);
    p = fma(z, p, 1.0 / 362880.0);
    q = fma(z, q, -1.0 / 3628800.0);
    p = fma(z, p, -1.0 / 5040.0);
    q = fma(z, q, 1.0 / 40320.0);
    p = fma(z, p, 1.0 / 120.0);
    q = fma(z, q, -1.0 / 720.0);
    p = fma(z, p, -1.0 / 6.0);
    q = fma(z, q, 1.0 / 24.0);
    q = fma(z, q, -0.5);
    by_quarters(fma(x * z, p, x), fma(z, q, 1.0), static_cast<uint32_t>((angle + (uint64_t{1} << 61)) >> 62), c, s);
}

// (u, w) turned by the angle whose cosine and sine are c and s
template <typename F>
__device__ inline void turn_pair(F& u, F& w, F c, F s) {
    const F a = u * c - w * s;
    w = u * s + w * c;
    u = a;
}

inline int check_rotation(const fxp_rotation* r, int64_t dim) {
    if (!r || !r->turns) return FXP_ERR_NULL;
    if (r->rot < 2 || r->rot > dim || r->rot % 2 || r->rot > FXP_ROTARY_MOST) return FXP_ERR_DIMS;
    if (!aligned(r->turns, 8)) return FXP_ERR_ALIGN;
    if (!(r->amplitude >= 0x1p-126 && r->amplitude < 1e30)) return FXP_ERR_VALUE;           // below, fp32 has fewer digits of it, or none
    return FXP_OK;
}

}  // namespace fxp
