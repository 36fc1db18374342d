// Products of a few rows with 4-bit weights: y[m,n] = sum over groups of 2^(e[group,n] - 129) * sum_k x[m,k] q[k,n].
//
// A 16 x 16 x 64 int8 matrix instruction has 16 outputs' weights as A (the lane's 16 mantissas of one output: 8 bytes) and the digits
// of up to 16 rows of x as B.  A mantissa is used in the upper half of its byte, 16 q, so that unpacking is a shift and two masks for
// eight of them; the factor 16 is taken out with the scales.  The int32 sums of a group are exact; group by group
// they are scaled into fp32 sums, by the exponents of x's unit and of the weights in one step (ldexp): scaled by one after the
// other, large x would pass the largest float before small weights bring it back, and tiny x be lost before large ones do.
#include "fxp_serve_device.h"

namespace fxp {

constexpr int kW4Waves = 8;
constexpr int kW4Threads = 64 * kW4Waves;

// x = digits * 2^unit and w = q 2^(e - 129), and q is used as 16 q: a sum counts 2^(unit + e - 133)
constexpr int kUnitBias = 133;

struct W4Args {
    const void* x;
    int64_t ldx;
    int M, K, N, k_tiles, n_tiles, m_tiles;
    int k_waves;         // waves that share a tile of outputs, 1 to 8 (k_w4_rows)
    const uint8_t* packed;
    const uint8_t* scales;
    void* y;
    int64_t ldy;
    uint8_t* digits;     // [k_tiles][m_tiles][ND][128 / S][64][S / 4] bytes
    int* units;          // [k_tiles * 128 / group][16 m_tiles]: exponent of one unit, less kUnitBias
    int vec_x;
};

// The digits of x in the order of the B operand.  A thread has 16 inputs of one row; group / 16 neighbours share a scale.
template <int TYPE, int GROUP>
__global__ __launch_bounds__(256) void k_w4_digits(W4Args a) {
    constexpr int ND = TYPE == FXP_F32 ? 3 : 2, S = GROUP < 64 ? GROUP : 64;
    const int i = blockIdx.x * 256 + threadIdx.x, pieces = a.k_tiles * 8, row = i / pieces, piece = i % pieces, k = piece * 16;
    if (row >= a.M) return;                                // whole groups of neighbours: pieces is a multiple of 8
    float x[16];
    if (k + 16 <= a.K) {
        load_elems<TYPE, 16>(a.x, row * a.ldx + k, a.vec_x, x);
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j)
            x[j] = k + j < a.K ? static_cast<float>(static_cast<const typename Elem<TYPE>::T*>(a.x)[row * a.ldx + k + j]) : 0.0f;
    }
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 16; ++j) m = max(m, __float_as_uint(x[j]) & 0x7fffffffu);
#pragma unroll
    for (int d = 1; d < GROUP / 16; d <<= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), d)));
    const int unit = unit_of<ND>(m);
    v4i d[ND];
    row_digits<ND>(x, unit, !__any(m >= 0x7f800000u), d);
    const int tile = k / 128, s = k % 128 / S, g = k % S / (S / 4), mt = row / 16, r = row % 16;
    uint8_t* base = a.digits + (static_cast<int64_t>(tile) * a.m_tiles + mt) * (ND * 2048);
#pragma unroll
    for (int j = 0; j < ND; ++j) {
        uint8_t* p = base + ((j * (128 / S) + s) * 64 + 16 * g + r) * (S / 4);
        if constexpr (S == 64) {
            *reinterpret_cast<v4i*>(p) = d[j];
        } else {
            *reinterpret_cast<int2*>(p) = make_int2(d[j][0], d[j][1]);
            *reinterpret_cast<int2*>(p + 16 * (S / 4)) = make_int2(d[j][2], d[j][3]);          // the next piece: 16 (g + 1) + r
        }
    }
    if (k % GROUP == 0) a.units[static_cast<int64_t>(k / GROUP) * (16 * a.m_tiles) + row] = unit - kUnitBias;
}

// Three rows or more: MT tiles of 16 rows, NT tiles of 16 outputs.  A wave has every eighth tile of 128 inputs.  U of its weight tiles and, up to
// two tiles of rows, the next digits are on their way while one is worked on; loads are always issued, those of tiles that are none without records
// (behind a branch the compiler would wait for all of them wherever it needs one).
template <int TYPE, int GROUP, int NT, int MT, int U>
__global__ __launch_bounds__(kW4Threads, 2) void k_w4_linear(W4Args a) {
    constexpr int ND = TYPE == FXP_F32 ? 3 : 2, S = GROUP < 64 ? GROUP : 64, STEPS = 128 / S, GT = 128 / GROUP, SG = STEPS / GT;
    constexpr int B = MT <= 2 ? 2 : 1;                      // buffers of digits
    // groups whose sums are in registers together: with three digits and two tiles of rows, some of four spilled (23 rows, 4096 x 14336: 42 us, 35 by
    // twos; with two digits, 64 rows, four 39.5, by twos 43.5)
    constexpr int GROUPS = ND * GT * MT == 24 && MT == 2 ? 2 : GT;
    static_assert(U % B == 0, "a turn begins with the same buffer");
    using Digit = std::conditional_t<S == 64, v4i, long>;
    __shared__ float red[kW4Waves][NT * 16][17];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
    const int nt0 = blockIdx.x * NT, mt0 = blockIdx.y * MT;
    float sum[MT][NT][4];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[i][n][j] = 0.0f;

    v4i w[U][NT];
    uint32_t e[U][NT][GT];
    Digit dig[B][MT][ND][STEPS];
    int unit[B][MT][GT];
    auto load_w = [&](int u, int kt) {
        const bool there = kt < a.k_tiles;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int64_t tile = static_cast<int64_t>(min(nt0 + n, a.n_tiles - 1)) * a.k_tiles + kt;
            w[u][n] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(records(a.packed + tile * 1024, there ? 1024 : 0), lane * 16, 0, kNonTemporal));
            const auto scales = records(a.scales + tile * (GT * 16), there ? GT * 16 : 0);
#pragma unroll
            for (int j = 0; j < GT; ++j) e[u][n][j] = __builtin_amdgcn_raw_buffer_load_b32(scales, 4 * g, 16 * j, 0);
        }
    };
    auto load_digits = [&](int c, int kt) {
        const bool there = kt < a.k_tiles;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int mt = min(mt0 + i, a.m_tiles - 1);
            const int piece = mt * 16 + col < a.M ? lane * static_cast<int>(sizeof(Digit)) : 1 << 30;      // no digits were made of rows that are none
            const auto digits = records(a.digits + (static_cast<int64_t>(kt) * a.m_tiles + mt) * (ND * 2048), there ? ND * 2048 : 0);
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    const int off = (d * STEPS + s) * static_cast<int>(64 * sizeof(Digit));
                    if constexpr (S == 64) dig[c][i][d][s] = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(digits, piece, off, 0));
                    else dig[c][i][d][s] = __builtin_bit_cast(long, __builtin_amdgcn_raw_buffer_load_b64(digits, piece, off, 0));
                }
            const auto units = records(a.units + static_cast<int64_t>(kt) * GT * (16 * a.m_tiles) + mt * 16, there ? (GT - 1) * 64 * a.m_tiles + 64 : 0);
#pragma unroll
            for (int j = 0; j < GT; ++j) unit[c][i][j] = __builtin_amdgcn_raw_buffer_load_b32(units, 4 * col, 64 * a.m_tiles * j, 0);
        }
    };
#pragma unroll
    for (int u = 0; u < U; ++u) load_w(u, wave + kW4Waves * u);
    if (B == 2) load_digits(0, wave);
    for (int kt0 = wave; kt0 < a.k_tiles; kt0 += kW4Waves * U) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int kt = kt0 + kW4Waves * u, c = u % B;
            load_digits(B == 2 ? 1 - c : 0, B == 2 ? kt + kW4Waves : kt);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
#pragma unroll
                for (int j0 = 0; j0 < GT; j0 += GROUPS) {
                    v4i acc[MT][GROUPS][ND];
#pragma unroll
                    for (int s = j0 * SG; s < (j0 + GROUPS) * SG; ++s) {
                        const uint32_t mask = 0xf0f0f0f0u;
                        Digit q;
                        if constexpr (S == 64) {
                            const uint32_t w0 = static_cast<uint32_t>(w[u][n][2 * s]), w1 = static_cast<uint32_t>(w[u][n][2 * s + 1]);
                            q = v4i{static_cast<int>((w0 << 4) & mask), static_cast<int>((w1 << 4) & mask), static_cast<int>(w0 & mask),
                                    static_cast<int>(w1 & mask)};
                        } else {
                            const uint32_t w0 = static_cast<uint32_t>(w[u][n][s]);
                            q = static_cast<long>(static_cast<uint64_t>(w0 & mask) << 32 | ((w0 << 4) & mask));
                        }
#pragma unroll
                        for (int i = 0; i < MT; ++i)
#pragma unroll
                            for (int d = 0; d < ND; ++d) {
                                const v4i before = s % SG ? acc[i][s / SG - j0][d] : v4i{0, 0, 0, 0};
                                if constexpr (S == 64) acc[i][s / SG - j0][d] = mfma_i8(q, dig[c][i][d][s], before);
                                else acc[i][s / SG - j0][d] = __builtin_amdgcn_mfma_i32_16x16x32_i8(q, dig[c][i][d][s], before, 0, 0, 0);
                            }
                    }
#pragma unroll
                    for (int j = 0; j < GROUPS; ++j)        // (of a tile that is none, all is zero)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int scale = static_cast<int>((e[u][n][j0 + j] >> (8 * r)) & 0xffu);
#pragma unroll
                            for (int i = 0; i < MT; ++i) {
                                float v = static_cast<float>((acc[i][j][0][r] << 8) + acc[i][j][1][r]);
                                if constexpr (ND == 3) v = fmaf(v, 256.0f, static_cast<float>(acc[i][j][2][r]));
                                sum[i][n][r] += ldexpf(v, unit[c][i][j0 + j] + scale);
                            }
                        }
                    if constexpr (GROUPS < GT) __builtin_amdgcn_sched_barrier(0);
                }
                __builtin_amdgcn_sched_barrier(0);          // one tile of outputs after the other: interleaved, some of these spilled
            }
            load_w(u, kt + kW4Waves * U);
        }
    }

    // the waves' shares of the contraction
    using T = typename Elem<TYPE>::T;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        if (i) __syncthreads();
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) red[wave][n * 16 + 4 * g + r][col] = sum[i][n][r];
        __syncthreads();
        for (int j = threadIdx.x; j < NT * 256; j += kW4Threads) {
            const int n = j % (NT * 16), m = j / (NT * 16);
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < kW4Waves; ++w) v += red[w][n][m];
            const int row = (mt0 + i) * 16 + m, out = nt0 * 16 + n;
            if (row < a.M && out < a.N) static_cast<T*>(a.y)[row * a.ldy + out] = static_cast<T>(v);
        }
    }
}

// One or two rows, one launch.  a.k_waves waves share a tile of outputs; a wave has every k_waves-th tile of 128 inputs, eight on their
// way at a time, and turns its own part of x into digits (a lane 16 inputs of a row, which is all of eight tiles at once).  With so few rows a matrix instruction
// would leave 15 of 16 columns empty and its scaling (22 vector instructions a group) would be for nothing: here a lane sums the 16
// mantissas it has loaded by byte dot products (one for four of them and a digit) and scales ONE sum a group.  Two workgroups a CU but for two
// rows in groups of 32: 128 registers are too few for their scales (4096 x 4096, bf16: 10.3 us with them, 7.8 with 256; fp32 12.4 / 8.9).
constexpr int kW4Ahead = 8;

template <int TYPE, int GROUP, int ROWS>
__global__ __launch_bounds__(kW4Threads, GROUP == 32 && ROWS == 2 ? 2 : 4) void k_w4_rows(W4Args a) {
    constexpr int ND = TYPE == FXP_F32 ? 3 : 2, S = GROUP < 64 ? GROUP : 64, STEPS = 128 / S, GT = 128 / GROUP, SG = STEPS / GT, U = kW4Ahead;
    __shared__ v4i s_digits[kW4Waves][U][ROWS][ND][8];          // pieces of 16 inputs
    __shared__ int s_unit[kW4Waves][U][ROWS][GT];
    __shared__ float red[kW4Waves][ROWS][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int k_waves = a.k_waves, wave_n = wave / k_waves, first = wave - wave_n * k_waves;
    const int nt = min(static_cast<int>(blockIdx.x) * (kW4Waves / k_waves) + wave_n, a.n_tiles - 1);      // a tile too many is done twice
    const uint8_t* const packed = a.packed + static_cast<int64_t>(nt) * a.k_tiles * 1024;
    const uint8_t* const scales = a.scales + static_cast<int64_t>(nt) * a.k_tiles * (GT * 16);
    v4i w[U];
    uint32_t e[U][GT];
    // tile i of a turn is kt + k_waves i; tiles behind the last are the last again, and their x is zero
    auto load_w = [&](int kt) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int t = min(kt + k_waves * i, a.k_tiles - 1);
            w[i] = __builtin_nontemporal_load(reinterpret_cast<const v4i*>(packed + t * 1024 + static_cast<uint32_t>(lane * 16)));
#pragma unroll
            for (int j = 0; j < GT; ++j) e[i][j] = scales[(t * GT + j) * 16 + static_cast<uint32_t>(r)];
        }
    };
    float x[ROWS][16];
    auto load_x = [&](int kt) {
        const int t = kt + k_waves * (lane >> 3), k = t * 128 + (lane & 7) * 16;
#pragma unroll
        for (int m = 0; m < ROWS; ++m) {
            const int row = min(m, a.M - 1);
            if (t < a.k_tiles && k + 16 <= a.K) {
                load_elems<TYPE, 16>(a.x, row * a.ldx + k, a.vec_x, x[m]);
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    x[m][j] = t < a.k_tiles && k + j < a.K ? static_cast<float>(static_cast<const typename Elem<TYPE>::T*>(a.x)[row * a.ldx + k + j]) : 0.0f;
            }
        }
    };
    float sum[ROWS];
#pragma unroll
    for (int m = 0; m < ROWS; ++m) sum[m] = 0.0f;
    // x before the weights: loads come back in order, and its digits are made while the weights are on their way
    if (first < a.k_tiles) {
        load_x(first);
        load_w(first);
    }
    for (int kt = first; kt < a.k_tiles; kt += k_waves * U) {
        // x's digits of this turn
#pragma unroll
        for (int m = 0; m < ROWS; ++m) {
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < 16; ++j) top = max(top, __float_as_uint(x[m][j]) & 0x7fffffffu);
#pragma unroll
            for (int d = 1; d < GROUP / 16; d <<= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), d)));
            const int unit = unit_of<ND>(top);
            v4i d[ND];
            row_digits<ND>(x[m], unit, !__any(top >= 0x7f800000u), d);
#pragma unroll
            for (int j = 0; j < ND; ++j) s_digits[wave][lane >> 3][m][j][lane & 7] = d[j];
            if ((lane & 7) % (GROUP / 16) == 0) s_unit[wave][lane >> 3][m][(lane & 7) / (GROUP / 16)] = unit - kUnitBias;
        }
        __builtin_amdgcn_wave_barrier();
        const bool more = kt + k_waves * U < a.k_tiles;
        if (more) load_x(kt + k_waves * U);
#pragma unroll
        for (int i = 0; i < U; ++i) {
            if (i && kt + k_waves * i >= a.k_tiles) break;
            const int mask = static_cast<int>(0xf0f0f0f0u);
            int q[8];                                       // 16 times the mantissas, four to a word, in the order of the inputs of a step
            if constexpr (S == 64) {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    q[4 * s] = (w[i][2 * s] << 4) & mask;
                    q[4 * s + 1] = (w[i][2 * s + 1] << 4) & mask;
                    q[4 * s + 2] = w[i][2 * s] & mask;
                    q[4 * s + 3] = w[i][2 * s + 1] & mask;
                }
            } else {
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    q[2 * s] = (w[i][s] << 4) & mask;
                    q[2 * s + 1] = w[i][s] & mask;
                }
            }
#pragma unroll
            for (int m = 0; m < ROWS; ++m)
#pragma unroll
                for (int j = 0; j < GT; ++j) {
                    int acc[ND];
#pragma unroll
                    for (int d = 0; d < ND; ++d) acc[d] = 0;
#pragma unroll
                    for (int t = 0; t < SG; ++t) {
                        const int s = j * SG + t;
#pragma unroll
                        for (int d = 0; d < ND; ++d) {
                            if constexpr (S == 64) {
                                const v4i b = s_digits[wave][i][m][d][4 * s + g];
#pragma unroll
                                for (int c = 0; c < 4; ++c) acc[d] = __builtin_amdgcn_sdot4(q[4 * s + c], b[c], acc[d], false);
                            } else {
                                const int2 b = reinterpret_cast<const int2*>(s_digits[wave][i][m][d])[4 * s + g];
                                acc[d] = __builtin_amdgcn_sdot4(q[2 * s], b.x, acc[d], false);
                                acc[d] = __builtin_amdgcn_sdot4(q[2 * s + 1], b.y, acc[d], false);
                            }
                        }
                    }
                    float v = static_cast<float>((acc[0] << 8) + acc[1]);
                    if constexpr (ND == 3) v = fmaf(v, 256.0f, static_cast<float>(acc[2]));
                    sum[m] += ldexpf(v, s_unit[wave][i][m][j] + static_cast<int>(e[i][j]));
                }
        }
        if (more) load_w(kt + k_waves * U);
        __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int m = 0; m < ROWS; ++m) {
        float v = sum[m];
        v += __shfl_xor(v, 16);
        v += __shfl_xor(v, 32);
        if (g == 0) red[wave][m][r] = v;
    }
    __syncthreads();
    const int tiles = kW4Waves / k_waves;
    for (int i = threadIdx.x; i < tiles * 16 * ROWS; i += kW4Threads) {
        const int m = i / 16 % ROWS, t = i / (16 * ROWS), tile = blockIdx.x * tiles + t, n = tile * 16 + (i & 15);
        float v = 0.0f;
        for (int w = 0; w < k_waves; ++w) v += red[t * k_waves + w][m][i & 15];
        using T = typename Elem<TYPE>::T;
        if (m < a.M && n < a.N) static_cast<T*>(a.y)[m * a.ldy + n] = static_cast<T>(v);
    }
}

// W -> mantissas and scales: a thread has one group of one output.
template <int TYPE, int GROUP>
__global__ __launch_bounds__(256) void k_w4_pack(const void* __restrict__ W, int64_t ldw, int64_t K, int64_t N, int k_tiles, int n_tiles,
                                                 uint8_t* __restrict__ packed, uint8_t* __restrict__ scales) {
    using T = typename Elem<TYPE>::T;
    constexpr int S = GROUP < 64 ? GROUP : 64, GT = 128 / GROUP;
    const int64_t n = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t kg = blockIdx.y, k0 = kg * GROUP;
    if (n >= static_cast<int64_t>(n_tiles) * 16) return;
    const T* w = static_cast<const T*>(W);
    auto value = [&](int64_t k) { return n < N && k < K ? static_cast<float>(w[k * ldw + n]) : 0.0f; };
    uint32_t m = 0;
    for (int k = 0; k < GROUP; ++k) m = max(m, __float_as_uint(value(k0 + k)) & 0x7fffffffu);
    // a scale byte is the exponent field of a power of two that multiplies in fp32: 254 at most
    const int e = min(max(static_cast<int>(m >> 23), 1), 254);
    const int64_t nt = n / 16, tile = nt * k_tiles + k0 / 128;
    const int r = static_cast<int>(n % 16);
    scales[(tile * GT + k0 % 128 / GROUP) * 16 + r] = static_cast<uint8_t>(e);
    for (int k = 0; k < GROUP; k += S / 4) {               // a lane's piece of a step: S / 4 inputs, S / 8 bytes
        const int kk = static_cast<int>((k0 + k) % 128), s = kk / S, g = kk % S / (S / 4);
        uint8_t* p = packed + tile * 1024 + (16 * g + r) * 16 + s * (S / 8);
#pragma unroll
        for (int j = 0; j < S / 8; j += 4) {
            uint32_t word = 0;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int lo = map_nearest(value(k0 + k + j + b), e, 21), hi = map_nearest(value(k0 + k + j + b + S / 8), e, 21);
                word |= static_cast<uint32_t>((lo & 15) | ((hi & 15) << 4)) << (8 * b);
            }
            *reinterpret_cast<uint32_t*>(p + j) = word;
        }
    }
}

static bool w4_group_ok(int group) { return group == 32 || group == 64 || group == 128; }
static bool w4_sizes_ok(int64_t K, int64_t N) { return K > 0 && N > 0 && K <= (int64_t{1} << 20) && N <= (int64_t{1} << 24); }

template <typename F>
static void w4_of_type(int type, F f) {
    if (type == FXP_F32) f(std::integral_constant<int, FXP_F32>{});
    else if (type == FXP_BF16) f(std::integral_constant<int, FXP_BF16>{});
    else f(std::integral_constant<int, FXP_F16>{});
}
template <typename F>
static void w4_of_group(int group, F f) {
    if (group == 32) f(std::integral_constant<int, 32>{});
    else if (group == 64) f(std::integral_constant<int, 64>{});
    else f(std::integral_constant<int, 128>{});
}

}  // namespace fxp

extern "C" size_t fxp_w4_packed_bytes(int64_t K, int64_t N) {
    return fxp::w4_sizes_ok(K, N) ? static_cast<size_t>((N + 15) / 16) * ((K + 127) / 128) * 1024 : 0;
}
extern "C" size_t fxp_w4_scale_bytes(int64_t K, int64_t N, int group) {
    return fxp::w4_sizes_ok(K, N) && fxp::w4_group_ok(group) ? static_cast<size_t>((N + 15) / 16) * ((K + 127) / 128) * (128 / group) * 16 : 0;
}
extern "C" size_t fxp_w4_workspace_bytes(int type, int64_t M, int64_t K, int group) {
    if (!fxp::known_type(type) || !fxp::w4_group_ok(group) || !fxp::w4_sizes_ok(K, 1) || M <= 0 || M >= (int64_t{1} << 20)) return 0;
    const size_t rows = (M + 15) / 16 * 16, tiles = (K + 127) / 128;
    return rows * tiles * 128 * (type == FXP_F32 ? 3 : 2) + rows * tiles * (128 / group) * sizeof(int);
}

extern "C" int fxp_w4_pack(int type, const void* W, int64_t ldw, int64_t K, int64_t N, int group, uint8_t* packed, uint8_t* scales,
                           void* stream) {
    using namespace fxp;
    if (!known_type(type)) return FXP_ERR_TYPE;
    if (!w4_group_ok(group)) return FXP_ERR_VALUE;
    if (!w4_sizes_ok(K, N) || ldw < N || ldw >= (int64_t{1} << 32)) return FXP_ERR_DIMS;
    if (!W || !packed || !scales) return FXP_ERR_NULL;
    if (!aligned(W, elem_size(type)) || !aligned(packed, 16) || !aligned(scales, 4)) return FXP_ERR_ALIGN;
    const int64_t k_tiles = (K + 127) / 128, n_tiles = (N + 15) / 16;
    const dim3 grid(static_cast<unsigned>((n_tiles * 16 + 255) / 256), static_cast<unsigned>(k_tiles * (128 / group)));
    w4_of_type(type, [&](auto t) {
        w4_of_group(group, [&](auto g) {
            hipLaunchKernelGGL((k_w4_pack<decltype(t)::value, decltype(g)::value>), grid, dim3(256), 0, static_cast<hipStream_t>(stream), W, ldw,
                               K, N, static_cast<int>(k_tiles), static_cast<int>(n_tiles), packed, scales);
        });
    });
    return launch_status();
}

extern "C" int fxp_w4_linear(int type, const void* X, int64_t ldx, int64_t M, int64_t K, int64_t N, const uint8_t* packed,
                             const uint8_t* scales, int group, void* Y, int64_t ldy, void* ws, size_t ws_bytes, void* stream) {
    using namespace fxp;
    if (!known_type(type)) return FXP_ERR_TYPE;
    if (!w4_group_ok(group)) return FXP_ERR_VALUE;
    if (!w4_sizes_ok(K, N) || M < 0 || M >= (int64_t{1} << 20) || ldx < K || ldy < N || ldx >= (int64_t{1} << 32) || ldy >= (int64_t{1} << 32))
        return FXP_ERR_DIMS;
    if (M == 0) return FXP_OK;
    if (!X || !packed || !scales || !Y) return FXP_ERR_NULL;
    const size_t size = elem_size(type);
    if (!aligned(X, size) || !aligned(Y, size) || !aligned(packed, 16) || !aligned(scales, 4)) return FXP_ERR_ALIGN;
    if (M > 2 && (!ws || ws_bytes < fxp_w4_workspace_bytes(type, M, K, group))) return FXP_ERR_WORKSPACE;
    if (M > 2 && !aligned(ws, 256)) return FXP_ERR_ALIGN;
    W4Args a;
    a.x = X;
    a.ldx = ldx;
    a.M = static_cast<int>(M);
    a.K = static_cast<int>(K);
    a.N = static_cast<int>(N);
    a.k_tiles = static_cast<int>((K + 127) / 128);
    a.n_tiles = static_cast<int>((N + 15) / 16);
    a.m_tiles = static_cast<int>((M + 15) / 16);
    a.packed = packed;
    a.scales = scales;
    a.y = Y;
    a.ldy = ldy;
    a.digits = static_cast<uint8_t*>(ws);
    a.units = reinterpret_cast<int*>(a.digits + static_cast<size_t>(a.m_tiles) * 16 * a.k_tiles * 128 * (type == FXP_F32 ? 3 : 2));
    a.vec_x = aligned(X, 16) && (M == 1 || ldx * size % 16 == 0);
    const int64_t pieces = M * a.k_tiles * 8;
    if (pieces > (int64_t{1} << 30)) return FXP_ERR_DIMS;
    hipStream_t s = static_cast<hipStream_t>(stream);
    w4_of_type(type, [&](auto t) {
        w4_of_group(group, [&](auto g) {
            constexpr int TYPE = decltype(t)::value, GROUP = decltype(g)::value;
            if (M <= 2) {
                // Waves to a tile of outputs: two a SIMD in all, and no more than eight tiles of inputs to each (8192 x 8192, one row: 9.4 us; half
                // as many waves 10.9, a quarter 15.7.  1024 x 16384: 6.0 us; with eight to each of the 1024 tiles 9.8).
                a.k_waves = 1;
                while (a.k_waves < kW4Waves && a.k_waves < a.k_tiles && (a.n_tiles * a.k_waves < 2048 || a.k_waves * kW4Ahead < a.k_tiles)) a.k_waves *= 2;
                const int tiles = kW4Waves / a.k_waves;
                const dim3 grid((a.n_tiles + tiles - 1) / tiles);
                if (M == 1) hipLaunchKernelGGL((k_w4_rows<TYPE, GROUP, 1>), grid, dim3(kW4Threads), 0, s, a);
                else hipLaunchKernelGGL((k_w4_rows<TYPE, GROUP, 2>), grid, dim3(kW4Threads), 0, s, a);
                return;
            }
            hipLaunchKernelGGL((k_w4_digits<TYPE, GROUP>), dim3(static_cast<unsigned>((pieces + 255) / 256)), dim3(256), 0, s, a);
            auto go = [&](auto nt_c, auto mt_c, auto u_c) {
                constexpr int NT = decltype(nt_c)::value, MT = decltype(mt_c)::value;
                hipLaunchKernelGGL((k_w4_linear<TYPE, GROUP, NT, MT, decltype(u_c)::value>), dim3((a.n_tiles + NT - 1) / NT, (a.m_tiles + MT - 1) / MT),
                                   dim3(kW4Threads), 0, s, a);
            };
            using std::integral_constant;
            constexpr integral_constant<int, 1> one{};
            constexpr integral_constant<int, 2> two{};
            constexpr integral_constant<int, 4> four{};
            constexpr integral_constant<int, 3> three{};
            // Three digits and four scales of two tiles of rows: registers for two tiles of outputs (23 rows, 4096 x 28672: two 65 us, three 88,
            // four 112), and none for four tiles of rows (64 rows: 107 us as two passes, 162 as one).
            constexpr bool kTight = TYPE == FXP_F32 && GROUP == 32;
            auto of_rows = [&](auto nt_c) {
                if (a.m_tiles == 1) go(nt_c, one, two);
                else if constexpr (kTight && decltype(nt_c)::value > 2) go(two, two, two);
                else go(nt_c, two, two);
            };
            // As many tiles of outputs to a workgroup as leave one for each CU: every wave reads its rows' digits (4 KB a tile of rows) for
            // 1 KB of weights a tile of outputs, and that is what bounds it (23 rows, 4090 x 11007: three tiles 10.5 us, two 13.8; 8192 x 8192,
            // two tiles 21.0 in all, one 25.8).  From 33 rows on, four tiles of rows read the weights half as often as two (64 rows, bf16, groups of
            // 64: 8192 x 8192 29 us against 32, 1024 x 16384 14 / 18, 4090 x 11007 30 / 27).
            constexpr int kCus = 256;
            if constexpr (!kTight)
                if (a.m_tiles > 2) return go(two, four, one);
            if (a.n_tiles <= kCus) of_rows(one);
            else if (a.n_tiles <= 2 * kCus) of_rows(two);
            else if (a.n_tiles <= 3 * kCus) of_rows(three);
            else of_rows(four);
        });
    });
    return launch_status();
}
