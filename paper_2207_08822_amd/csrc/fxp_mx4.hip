// Mapping to microscaled 4-bit numbers and back, and a linear layer's step in them.
//
// A mapped matrix serves products that contract over its columns; a training step contracts every operand along both of its axes and therefore maps it twice,
// with blocks of 32 along the rows and of 32 along the columns.  Both copies come out of one pass: 32 x 32 elements hold whole blocks of both.
#include <algorithm>
#include <initializer_list>

#include "fxp_mx4_device.h"

namespace fxp {

constexpr int kMxThreads = 256, kMxTileRows = 32;       // of a tile of both copies, which is a panel wide

struct Mx4Job {
    Mx4Map m;
    int tiles_c;            // tiles of a row of tiles
    unsigned first;         // workgroup of the job's first tile
    int vec;                // rows and the base are multiples of 16 bytes
};
struct Mx4Jobs {
    Mx4Job job[2];
    int count;
};

// largest of the lanes eight apart
__device__ inline uint32_t max_over_8(uint32_t m) {
    typedef unsigned v2u __attribute__((ext_vector_type(2)));
    m = max_dpp<0x128>(m);                                                                         // row_ror:8
    v2u p = __builtin_amdgcn_permlane16_swap(m, m, false, false);
    m = max(p[0], p[1]);
    p = __builtin_amdgcn_permlane32_swap(m, m, false, false);
    return max(p[0], p[1]);
}
// What stochastic rounding adds to eight elements from element `at` of the matrix on: 2^22 - 1 less the top 22 bits of their words.
__device__ inline void adds_of_8(uint64_t at, bool whole_quads, uint32_t sid0, uint32_t sid1, uint32_t key0, uint32_t key1, uint32_t (&add)[8]) {
    const uint64_t quad = at >> 2;
    auto words = [&](uint64_t q) { return philox4x32_10(static_cast<uint32_t>(q), static_cast<uint32_t>(q >> 32), sid0, sid1, key0, key1); };
    const uint4 a = words(quad), b = words(quad + 1);
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    if (!whole_quads) {                                    // they lie in three quads
        const uint4 c = words(quad + 2);
        const uint32_t all[11] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w, c.x, c.y, c.z};
        const int shift = static_cast<int>(at & 3);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = shift == 0 ? all[j] : shift == 1 ? all[j + 1] : shift == 2 ? all[j + 2] : all[j + 3];
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) add[j] = ~w[j] >> 10;
}

// Codes of N elements under the factor f; sign[j]: 8 for a negative element.
template <bool STOCH, int N>
__device__ inline uint32_t codes_of(const float (&x)[N], float f, const uint32_t (&add)[N], const uint32_t (&sign)[N]) {
    if constexpr (STOCH) {
        uint32_t r = 0;
#pragma unroll
        for (int j = N - 1; j >= 0; --j) r = r << 4 | mx_stochastic(fabsf(x[j]) * f, add[j]) | sign[j];
        return r;
    } else {
        float y[N];
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = x[j] * f;
        return mx_nearest(y);
    }
}

// A wave has 32 rows x 64 columns, whole blocks of both copies, a lane 4 x 8 elements of it; the four waves of a workgroup lie side by side along a panel, so that lines of
// q leave whole.  Codes are put together in LDS and leave in 16-byte pieces.
// Bound by memory for nearest: 8192 x 8192 in bf16 43.5 us (206 MB at 4.7 TB/s) over six sets of tensors in turn, back to back; 36 over one set, which stays in the
// Infinity Cache in part; 54 where each call is followed by the inverses of both copies, 268 MB of stores.  By the vector ALU for stochastic
// rounding (12608 x 768 in fp32: 15.7 us over two sets, 17.5 over sixteen; 44 instructions an element, 14 of them Philox's and the rest the scales and codes of two copies,
// are three quarters of the time).
// Other tiles, over six sets and sixteen: the waves below each other 61.5 us and 17.4, two by two 47.8 and 17.4; two steps a wave 47.7 and 23.4, eight 55.8 and 31.9.
template <int TYPE, bool STOCH>
__global__ __launch_bounds__(kMxThreads) void k_mx4_map(Mx4Jobs jobs, uint32_t key0, uint32_t key1) {
    constexpr int TR = kMxTileRows, TC = kMxPanel, BC = TC / kMxBlock, kPad = 16, SQ = TC / 2 + kPad, ST = TR / 2 + kPad;
    static_assert(TR == kMxBlock && TC == kMxThreads, "a block of rows, a panel");
    __shared__ __attribute__((aligned(16))) uint8_t lq[TR * SQ], lt[TC * ST];
    __shared__ uint8_t eq[TR * BC], et[TC];
    const Mx4Job& J = jobs.job[jobs.count > 1 && blockIdx.x >= jobs.job[1].first ? 1 : 0];
    const int tile = static_cast<int>(blockIdx.x - J.first);
    const int r0 = tile / J.tiles_c * TR, c0 = tile % J.tiles_c * TC;
    const int rows = static_cast<int>(J.m.rows), cols = static_cast<int>(J.m.cols);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, rb = lane >> 3, cb = lane & 7;
    const bool want_q = J.m.q != nullptr, want_t = J.m.t != nullptr, inside = J.vec && r0 + TR <= rows && c0 + TC <= cols;
    const uint32_t sid0 = static_cast<uint32_t>(J.m.stream_id), sid1 = static_cast<uint32_t>(J.m.stream_id >> 32);
    using T = typename Elem<TYPE>::T;
    const T* const corner = static_cast<const T*>(J.m.x) + r0 * J.m.ld + c0;

    const int r = 4 * rb, c = wave * 64 + 8 * cb;
    float x[4][8];
    auto load = [&] {           // a scope of its own: in line, loads and words are scheduled worse (12608 x 768 in fp32, stochastic, over sixteen sets 17.9 us, so 17.5)
        const T* const p = corner + r * J.m.ld + c;
        if (inside) {
#pragma unroll
            for (int i = 0; i < 4; ++i) load_elems<TYPE, 8>(p, i * J.m.ld, true, x[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (J.vec && r0 + r + i < rows && c0 + c + 8 <= cols) {
                    load_elems<TYPE, 8>(p, i * J.m.ld, true, x[i]);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[i][j] = r0 + r + i < rows && c0 + c + j < cols ? static_cast<float>(p[i * J.m.ld + j]) : 0.0f;
                }
            }
        }
    };
    load();
    uint32_t add[4][8], sign[4][8];
    if constexpr (STOCH) {
        const uint64_t at = static_cast<uint64_t>(r0 + r) * static_cast<uint32_t>(cols) + static_cast<uint32_t>(c0 + c);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            adds_of_8(at + static_cast<uint64_t>(i) * static_cast<uint32_t>(cols), (cols & 3) == 0, sid0, sid1, key0, key1, add[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) sign[i][j] = __float_as_uint(x[i][j]) >> 28 & 8u;
        }
    }
    if (want_q) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) m = max(m, magnitude(x[i][j]));
            const int s = mx_scale_of(max_of_4(m));
            *reinterpret_cast<uint32_t*>(&lq[(r + i) * SQ + wave * 32 + 4 * cb]) = codes_of<STOCH>(x[i], mx_inverse(s), add[i], sign[i]);
            if ((cb & 3) == 0) eq[(r + i) * BC + 2 * wave + (cb >> 2)] = static_cast<uint8_t>(s);
        }
    }
    if (want_t) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float y[4] = {x[0][j], x[1][j], x[2][j], x[3][j]};
            const uint32_t a[4] = {add[0][j], add[1][j], add[2][j], add[3][j]}, g[4] = {sign[0][j], sign[1][j], sign[2][j], sign[3][j]};
            const int s = mx_scale_of(max_over_8(max(max(magnitude(y[0]), magnitude(y[1])), max(magnitude(y[2]), magnitude(y[3])))));
            *reinterpret_cast<uint16_t*>(&lt[(c + j) * ST + 2 * rb]) = static_cast<uint16_t>(codes_of<STOCH>(y, mx_inverse(s), a, g));
            if (rb == 0) et[c + j] = static_cast<uint8_t>(s);
        }
    }
    __syncthreads();
    // `height` lines of `width` blocks: line l of the copy is row l0 + l of `lines`, its blocks begin at element b0 of the contraction
    auto leave = [&](const uint8_t* codes, const uint8_t* scales, int stride, auto height_c, auto width_c, int l0, int lines, int b0, uint8_t* data, uint8_t* out_scales) {
        constexpr int height = decltype(height_c)::value, width = decltype(width_c)::value;
        const int64_t line = static_cast<int64_t>(b0 / kMxPanel) * lines + l0;
        data += line * kMxRowBytes;
        out_scales += line * kMxRowScales;
        const int at = b0 % kMxPanel / kMxBlock, here = min(height, lines - l0) * width;
#pragma unroll
        for (int i0 = 0; i0 < height * width; i0 += kMxThreads) {
            const int i = i0 + static_cast<int>(threadIdx.x), l = i / width, p = i % width;
            if (i >= here) break;
            *reinterpret_cast<uint4*>(data + l * kMxRowBytes + (at + p) * 16) = *reinterpret_cast<const uint4*>(&codes[l * stride + p * 16]);
            out_scales[l * kMxRowScales + mx_scale_place(at + p)] = scales[i];
        }
    };
    using std::integral_constant;
    if (want_q) leave(lq, eq, SQ, integral_constant<int, TR>{}, integral_constant<int, BC>{}, r0, rows, c0, J.m.q, J.m.q_scales);
    if (want_t) leave(lt, et, ST, integral_constant<int, TC>{}, integral_constant<int, 1>{}, c0, cols, r0, J.m.t, J.m.t_scales);
}

// Rows alone: a lane has eight elements of a row, a block is four lanes, a panel of a row half a wave; nothing goes through LDS.  8192 x 8192 in bf16, nearest, over six sets of
// tensors in turn 33.7 us, 172 MB at 5.1 TB/s, through the tiles of both copies 33.8; 12608 x 768 in fp32, stochastic, over sixteen sets 11.0 and 12.8; 3001 x 1003 in bf16,
// stochastic 7.7 and 11.2.
template <int TYPE, bool STOCH>
__global__ __launch_bounds__(kMxThreads) void k_mx4_map_rows(Mx4Map m, int panels, int vec, uint32_t key0, uint32_t key1) {
    const int64_t piece = (int64_t{blockIdx.x} * kMxThreads + threadIdx.x) >> 5;        // a panel of a row, panel after panel of a row
    const int64_t row = piece / panels;
    if (row >= m.rows) return;                                                          // whole blocks leave together
    const int panel = static_cast<int>(piece - row * panels), lane = threadIdx.x & 31, c = panel * kMxPanel + 8 * lane, cols = static_cast<int>(m.cols);
    using T = typename Elem<TYPE>::T;
    const T* const p = static_cast<const T*>(m.x) + row * m.ld + c;
    float x[8];
    if (vec && c + 8 <= cols) {
        load_elems<TYPE, 8>(p, 0, true, x);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = c + j < cols ? static_cast<float>(p[j]) : 0.0f;
    }
    uint32_t add[8], sign[8], top = 0;
    if constexpr (STOCH) {
        adds_of_8(static_cast<uint64_t>(row) * static_cast<uint32_t>(cols) + static_cast<uint32_t>(c), (cols & 3) == 0, static_cast<uint32_t>(m.stream_id),
                  static_cast<uint32_t>(m.stream_id >> 32), key0, key1, add);
#pragma unroll
        for (int j = 0; j < 8; ++j) sign[j] = __float_as_uint(x[j]) >> 28 & 8u;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, magnitude(x[j]));
    const int s = mx_scale_of(max_of_4(top));
    const int64_t line = panel * m.rows + row;
    *reinterpret_cast<uint32_t*>(m.q + line * kMxRowBytes + 4 * lane) = codes_of<STOCH>(x, mx_inverse(s), add, sign);
    if ((lane & 3) == 0) m.q_scales[line * kMxRowScales + mx_scale_place(lane >> 2)] = static_cast<uint8_t>(s);
}

int mx4_map_launch(int type, const Mx4Map* maps, int count, uint64_t seed, int rounding, hipStream_t s) {
    const uint32_t key0 = static_cast<uint32_t>(seed), key1 = static_cast<uint32_t>(seed >> 32);
    auto vec_of = [&](const Mx4Map& m) { return aligned(m.x, 16) && m.ld * elem_size(type) % 16 == 0; };
    auto launch = [&](auto type_c, auto stoch_c) {
        constexpr int TR = kMxTileRows, TC = kMxPanel;
        Mx4Jobs jobs{};
        int64_t tiles = 0;
        for (int i = 0; i < count; ++i) {
            const Mx4Map& m = maps[i];
            if (m.rows == 0 || m.cols == 0) continue;
            Mx4Job& j = jobs.job[jobs.count++];
            j.m = m;
            // a copy is written up to the end of its last panel
            const int64_t R = m.t ? mx_panels(m.rows) * kMxPanel : m.rows, C = m.q ? mx_panels(m.cols) * kMxPanel : m.cols;
            j.tiles_c = static_cast<int>((C + TC - 1) / TC);
            j.first = static_cast<unsigned>(tiles);
            j.vec = vec_of(m);
            tiles += j.tiles_c * ((R + TR - 1) / TR);
        }
        if (tiles >= int64_t{1} << 24) return static_cast<int>(FXP_ERR_DIMS);          // 2^32 threads
        if (tiles == 0) return static_cast<int>(FXP_OK);
        hipLaunchKernelGGL((k_mx4_map<decltype(type_c)::value, decltype(stoch_c)::value>), dim3(static_cast<unsigned>(tiles)), dim3(kMxThreads), 0, s, jobs, key0, key1);
        return launch_status();
    };
    auto sized = [&](auto type_c, auto stoch_c) {
        const int64_t pieces = maps[0].rows * mx_panels(maps[0].cols), blocks = (pieces * 32 + kMxThreads - 1) / kMxThreads;
        if (count == 1 && !maps[0].t && blocks < int64_t{1} << 24) {                   // 2^32 threads
            if (blocks == 0) return static_cast<int>(FXP_OK);
            hipLaunchKernelGGL((k_mx4_map_rows<decltype(type_c)::value, decltype(stoch_c)::value>), dim3(static_cast<unsigned>(blocks)), dim3(kMxThreads), 0, s, maps[0],
                               static_cast<int>(mx_panels(maps[0].cols)), vec_of(maps[0]), key0, key1);
            return launch_status();
        }
        return launch(type_c, stoch_c);
    };
    auto typed = [&](auto type_c) {
        return rounding == FXP_ROUND_STOCHASTIC ? sized(type_c, std::true_type{}) : sized(type_c, std::false_type{});
    };
    if (type == FXP_F32) return typed(std::integral_constant<int, FXP_F32>{});
    if (type == FXP_BF16) return typed(std::integral_constant<int, FXP_BF16>{});
    return typed(std::integral_constant<int, FXP_F16>{});
}

// ---- inverse mapping ----
//
// A thread has 16 bytes of its output, neighbouring lanes beside each other, of one row or of two.  Bound by its stores (8192 x 8192 to bf16 30 us, 5.8 TB/s; 12608 x 768 to
// fp32 8.5, where eight elements a thread, in two stores that leave every other 16 bytes to each other, take 10.5; 8192 x 8192 to fp32 54 and 62.5).
constexpr int kUnmapRows = 8;           // of a workgroup

template <int TYPE>
__global__ __launch_bounds__(kMxThreads) void k_mx4_unmap(const uint8_t* __restrict__ data, const uint8_t* __restrict__ scales, int64_t rows, int64_t cols, void* y, int64_t ld,
                                                          int vec) {
    constexpr int N = 16 / static_cast<int>(sizeof(typename Elem<TYPE>::T)), kThreads = kMxPanel / N, kStep = kMxThreads / kThreads, kMine = kUnmapRows / kStep;
    const int piece = threadIdx.x % kThreads;
    const int64_t row = int64_t{blockIdx.x} * kUnmapRows + threadIdx.x / kThreads, c = int64_t{blockIdx.y} * kMxPanel + piece * N;
    if (c >= cols) return;
    uint32_t codes[kMine];
    int s[kMine];
#pragma unroll
    for (int n = 0; n < kMine; ++n) {
        if (row + n * kStep >= rows) break;
        const int64_t line = blockIdx.y * rows + row + n * kStep;
        const uint8_t* const p = data + line * kMxRowBytes + piece * (N / 2);
        codes[n] = N == 4 ? *reinterpret_cast<const uint16_t*>(p) : *reinterpret_cast<const uint32_t*>(p);
        s[n] = scales[line * kMxRowScales + mx_scale_place(piece * N / kMxBlock)];
    }
#pragma unroll
    for (int n = 0; n < kMine; ++n) {
        if (row + n * kStep >= rows) break;
        // 2^-127 is a sub-normal number, and there is no number for 255
        const float unit = s[n] == 255 ? __uint_as_float(0x7fc00000u) : s[n] == 0 ? __uint_as_float(0x400000u) : __uint_as_float(static_cast<uint32_t>(s[n]) << 23);
        float v[N];
#pragma unroll
        for (int b = 0; b < N / 2; ++b) {
            const float2 two = mx_values(codes[n], b);
            v[2 * b] = two.x * unit;
            v[2 * b + 1] = two.y * unit;
        }
        const int64_t at = (row + n * kStep) * ld + c;
        if (vec && c + N <= cols) {
            store_elems<TYPE, N>(y, at, v);
        } else {
            typename Elem<TYPE>::T* const p = static_cast<typename Elem<TYPE>::T*>(y) + at;
            for (int j = 0; j < N; ++j)
                if (c + j < cols) p[j] = static_cast<typename Elem<TYPE>::T>(v[j]);
        }
    }
}

static Mx4Map map_of(const void* x, int64_t ld, int64_t rows, int64_t cols, const fxp_mx4* q, const fxp_mx4* t, uint64_t stream_id) {
    Mx4Map m{x, ld, rows, cols, nullptr, nullptr, nullptr, nullptr, stream_id};
    if (q) m.q = q->data, m.q_scales = q->scales;
    if (t) m.t = t->data, m.t_scales = t->scales;
    return m;
}

// whether two buffers share bytes
static bool meet(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a_bytes > 0 && b_bytes > 0 && x < y + static_cast<uintptr_t>(b_bytes) && y < x + static_cast<uintptr_t>(a_bytes);
}
static bool meet(const fxp_mx4& a, const fxp_mx4& b) {
    const int64_t na = mx_panels(a.cols) * a.rows, nb = mx_panels(b.cols) * b.rows;
    return meet(a.data, na * kMxRowBytes, b.data, nb * kMxRowBytes) || meet(a.data, na * kMxRowBytes, b.scales, nb * kMxRowScales) ||
           meet(a.scales, na * kMxRowScales, b.data, nb * kMxRowBytes) || meet(a.scales, na * kMxRowScales, b.scales, nb * kMxRowScales);
}
// whether rows of a matrix, `stride` bytes from each other, share bytes with a mapped matrix
static bool meet(const void* m, int64_t rows, int64_t row_bytes, int64_t stride, const void* b, int64_t bytes) {
    if (rows <= 0 || row_bytes <= 0 || bytes <= 0) return false;
    // the first row that ends behind b's first byte: does it begin before b's end?
    const int64_t from = static_cast<int64_t>(reinterpret_cast<uintptr_t>(b) - reinterpret_cast<uintptr_t>(m));
    const int64_t row = from < row_bytes ? 0 : (from - row_bytes) / stride + 1;
    return row < rows && row * stride < from + bytes;
}
static bool meet(int type, const void* m, int64_t rows, int64_t cols, int64_t ld, const fxp_mx4& q) {
    const int64_t size = elem_size(type), n = mx_panels(q.cols) * q.rows;
    return meet(m, rows, cols * size, ld * size, q.data, n * kMxRowBytes) || meet(m, rows, cols * size, ld * size, q.scales, n * kMxRowScales);
}

static int check_map(int type, const void* x, int64_t ldx, int64_t rows, int64_t cols, const fxp_mx4* q, const fxp_mx4* qT) {
    if (!known_type(type)) return FXP_ERR_TYPE;
    if (rows < 0 || cols < 0 || rows > kMxMost || cols > kMxMost || ldx < cols || ldx >= int64_t{1} << 40) return FXP_ERR_DIMS;
    if (q) {
        const int rc = check_mx4(q);
        if (rc) return rc;
        if (q->rows != rows || q->cols != cols) return FXP_ERR_DIMS;
    }
    if (qT) {
        const int rc = check_mx4(qT);
        if (rc) return rc;
        if (qT->rows != cols || qT->cols != rows) return FXP_ERR_DIMS;
        if (q && meet(*q, *qT)) return FXP_ERR_VALUE;
    }
    if (rows && cols) {
        if (!x) return FXP_ERR_NULL;
        if (!aligned(x, static_cast<size_t>(elem_size(type)))) return FXP_ERR_ALIGN;
    }
    return FXP_OK;
}

static bool known_rounding(int r) { return r == FXP_ROUND_STOCHASTIC || r == FXP_ROUND_NEAREST; }

}  // namespace fxp

extern "C" size_t fxp_mx4_data_bytes(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 0 || rows > fxp::kMxMost || cols > fxp::kMxMost) return 0;
    return static_cast<size_t>(fxp::mx_panels(cols) * rows * fxp::kMxRowBytes);
}

extern "C" size_t fxp_mx4_scale_bytes(int64_t rows, int64_t cols) { return fxp_mx4_data_bytes(rows, cols) / 16; }

extern "C" int fxp_mx4_map(int type, const void* x, int64_t ldx, int64_t rows, int64_t cols, const fxp_mx4* q, const fxp_mx4* qT, uint64_t seed, uint64_t stream_id,
                           int rounding, void* stream) {
    if (!q && !qT) return FXP_ERR_NULL;
    const int rc = fxp::check_map(type, x, ldx, rows, cols, q, qT);
    if (rc) return rc;
    if (!fxp::known_rounding(rounding)) return FXP_ERR_ROUNDING;
    for (const fxp_mx4* t : {q, qT})
        if (t && fxp::meet(type, x, rows, cols, ldx, *t)) return FXP_ERR_VALUE;
    const fxp::Mx4Map m = fxp::map_of(x, ldx, rows, cols, q, qT, stream_id);
    return fxp::mx4_map_launch(type, &m, 1, seed, rounding, static_cast<hipStream_t>(stream));
}

extern "C" int fxp_mx4_unmap(const fxp_mx4* q, int type, void* y, int64_t ldy, void* stream) {
    using namespace fxp;
    const int rc = check_mx4(q);
    if (rc) return rc;
    if (!known_type(type)) return FXP_ERR_TYPE;
    if (ldy < q->cols || ldy >= int64_t{1} << 40) return FXP_ERR_DIMS;
    if (q->rows == 0 || q->cols == 0) return FXP_OK;
    if (!y) return FXP_ERR_NULL;
    if (!aligned(y, static_cast<size_t>(elem_size(type)))) return FXP_ERR_ALIGN;
    if (meet(type, y, q->rows, q->cols, ldy, *q)) return FXP_ERR_VALUE;
    const dim3 grid(static_cast<unsigned>((q->rows + kUnmapRows - 1) / kUnmapRows), static_cast<unsigned>(mx_panels(q->cols)));
    const int vec = aligned(y, 16) && ldy * elem_size(type) % 16 == 0;
    auto go = [&](auto type_c) {
        hipLaunchKernelGGL((k_mx4_unmap<decltype(type_c)::value>), grid, dim3(kMxThreads), 0, static_cast<hipStream_t>(stream), q->data, q->scales, q->rows, q->cols, y, ldy, vec);
    };
    if (type == FXP_F32) go(std::integral_constant<int, FXP_F32>{});
    else if (type == FXP_BF16) go(std::integral_constant<int, FXP_BF16>{});
    else go(std::integral_constant<int, FXP_F16>{});
    return launch_status();
}

// ---- products ----

extern "C" size_t fxp_mx4_gemm_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    for (int64_t n : {M, N, K})
        if (n < 0 || n > fxp::kMxMost) return 0;
    return fxp::mx4_gemm_bytes(M, N, K);
}

extern "C" int fxp_mx4_gemm(const fxp_mx4* A, const fxp_mx4* B, int type, void* C, int64_t ldc, void* ws, size_t ws_bytes, void* stream) {
    using namespace fxp;
    for (const fxp_mx4* q : {A, B}) {
        const int rc = check_mx4(q);
        if (rc) return rc;
    }
    if (!known_type(type)) return FXP_ERR_TYPE;
    if (A->cols != B->cols || ldc < B->rows || ldc >= int64_t{1} << 40) return FXP_ERR_DIMS;
    if (A->rows == 0 || B->rows == 0) return FXP_OK;
    if (!C) return FXP_ERR_NULL;
    if (!aligned(C, static_cast<size_t>(elem_size(type)))) return FXP_ERR_ALIGN;
    const size_t need = mx4_gemm_bytes(A->rows, B->rows, A->cols);
    if (need && (!ws || ws_bytes < need)) return FXP_ERR_WORKSPACE;
    if (need && !aligned(ws, 256)) return FXP_ERR_ALIGN;
    for (const fxp_mx4* q : {A, B})
        if (meet(type, C, A->rows, B->rows, ldc, *q)) return FXP_ERR_VALUE;
    return mx4_gemm_launch(*A, *B, type, C, ldc, ws, static_cast<hipStream_t>(stream));
}

// the mapped rows of x in a workspace: codes, scales, then the product's own
namespace fxp {
static size_t mapped_bytes(int64_t M, int64_t K) {
    return round_up(static_cast<size_t>(mx_panels(K) * M * kMxRowBytes), 256) + round_up(static_cast<size_t>(mx_panels(K) * M * kMxRowScales), 256);
}
}  // namespace fxp

extern "C" size_t fxp_mx4_linear_workspace_bytes(int64_t M, int64_t N, int64_t K) {
    for (int64_t n : {M, N, K})
        if (n < 0 || n > fxp::kMxMost) return 0;
    return fxp::mx4_is_fused(M) ? 0 : fxp::mapped_bytes(M, K) + fxp::mx4_gemm_bytes(M, N, K);
}

extern "C" int fxp_mx4_linear(int type, const void* X, int64_t ldx, int64_t M, const fxp_mx4* W, void* Y, int64_t ldy, void* ws, size_t ws_bytes, void* stream) {
    using namespace fxp;
    int rc = check_mx4(W);
    if (rc) return rc;
    const int64_t K = W->cols, N = W->rows;
    rc = check_map(type, X, ldx, M, K, nullptr, nullptr);
    if (rc) return rc;
    if (ldy < N || ldy >= int64_t{1} << 40) return FXP_ERR_DIMS;
    if (M == 0 || N == 0) return FXP_OK;
    if (!Y) return FXP_ERR_NULL;
    if (!aligned(Y, static_cast<size_t>(elem_size(type)))) return FXP_ERR_ALIGN;
    const bool shared = meet(type, Y, M, N, ldy, *W);
    if (mx4_is_fused(M)) return shared ? static_cast<int>(FXP_ERR_VALUE) : mx4_fused_launch(type, X, ldx, M, *W, Y, ldy, static_cast<hipStream_t>(stream));
    const size_t codes = round_up(static_cast<size_t>(mx_panels(K) * M * kMxRowBytes), 256), mapped = mapped_bytes(M, K);
    const size_t need = fxp_mx4_linear_workspace_bytes(M, N, K);               // 0: a few rows, or a contraction of nothing
    if (need && (!ws || ws_bytes < need)) return FXP_ERR_WORKSPACE;
    if (!aligned(ws, 256)) return FXP_ERR_ALIGN;
    if (shared) return FXP_ERR_VALUE;
    uint8_t* const at = static_cast<uint8_t*>(ws);
    const fxp_mx4 q{at, at + codes, M, K};
    const Mx4Map m = map_of(X, ldx, M, K, &q, nullptr, 0);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    rc = mx4_map_launch(type, &m, 1, 0, FXP_ROUND_NEAREST, s);
    return rc ? rc : mx4_gemm_launch(q, *W, type, Y, ldy, at + mapped, s);
}

// ---- a layer's training step ----

namespace fxp {
static int check_layer(const fxp_mx4_layer* l, int64_t M, int64_t K, int64_t N, bool backward, bool need_x, bool need_w) {
    if (!l) return FXP_ERR_NULL;
    for (int64_t n : {M, K, N})
        if (n < 0 || n > kMxMost) return FXP_ERR_DIMS;
    struct Want {
        const fxp_mx4* q;
        int64_t rows, cols;
        bool needed;
    };
    const Want forward[] = {{&l->X, M, K, true}, {&l->WT, N, K, true}, {&l->XT, K, M, false}, {&l->W, K, N, false}};
    const Want back[] = {{&l->dY, M, N, need_x}, {&l->W, K, N, need_x}, {&l->dYT, N, M, need_w}, {&l->XT, K, M, need_w}};
    for (const Want& w : backward ? back : forward) {
        if (!w.q->data && !w.needed) continue;
        if (w.q->rows != w.rows || w.q->cols != w.cols) return FXP_ERR_DIMS;
        const int rc = check_mx4(w.q);
        if (rc) return rc;
        // no two of the call's operands are one
        for (const Want& o : backward ? back : forward)
            if (o.q != w.q && o.q->data && meet(*w.q, *o.q)) return FXP_ERR_VALUE;
    }
    return FXP_OK;
}
// Whether a dense matrix shares bytes with one of the operands that are there.
static bool meets_one(int type, const void* m, int64_t rows, int64_t cols, std::initializer_list<const fxp_mx4*> operands) {
    for (const fxp_mx4* q : operands)
        if (m && q->data && meet(type, m, rows, cols, cols, *q)) return true;
    return false;
}
static const fxp_mx4* if_there(const fxp_mx4& q) { return q.data ? &q : nullptr; }
}  // namespace fxp

extern "C" size_t fxp_mx4_layer_workspace_bytes(int64_t M, int64_t K, int64_t N) {
    for (int64_t n : {M, N, K})
        if (n < 0 || n > fxp::kMxMost) return 0;
    return std::max({fxp::mx4_gemm_bytes(M, N, K), fxp::mx4_gemm_bytes(M, K, N), fxp::mx4_gemm_bytes(K, N, M), size_t{256}});
}

extern "C" int fxp_mx4_linear_fwd(int type, const void* X, const void* W, int64_t M, int64_t K, int64_t N, void* Y, const fxp_mx4_layer* layer, uint64_t seed,
                                  uint64_t step, int rounding, void* ws, size_t ws_bytes, void* stream) {
    using namespace fxp;
    int rc = check_layer(layer, M, K, N, false, true, true);
    if (rc) return rc;
    rc = check_map(type, X, K, M, K, nullptr, nullptr);
    if (!rc) rc = check_map(type, W, N, K, N, nullptr, nullptr);
    if (rc) return rc;
    if (!known_rounding(rounding)) return FXP_ERR_ROUNDING;
    if (M && N && !Y) return FXP_ERR_NULL;
    if (!aligned(Y, static_cast<size_t>(elem_size(type)))) return FXP_ERR_ALIGN;
    if (!ws || ws_bytes < fxp_mx4_layer_workspace_bytes(M, K, N)) return FXP_ERR_WORKSPACE;
    if (!aligned(ws, 256)) return FXP_ERR_ALIGN;
    const std::initializer_list<const fxp_mx4*> operands = {&layer->X, &layer->XT, &layer->W, &layer->WT};
    if (meets_one(type, X, M, K, operands) || meets_one(type, W, K, N, operands) || meets_one(type, Y, M, N, operands)) return FXP_ERR_VALUE;
    const Mx4Map maps[2] = {map_of(X, K, M, K, &layer->X, if_there(layer->XT), step << 8), map_of(W, N, K, N, if_there(layer->W), &layer->WT, (step << 8) | 1)};
    const hipStream_t s = static_cast<hipStream_t>(stream);
    rc = mx4_map_launch(type, maps, 2, seed, rounding, s);
    if (rc || M == 0 || N == 0) return rc;
    return mx4_gemm_launch(layer->X, layer->WT, type, Y, N, ws, s);
}

extern "C" int fxp_mx4_linear_bwd(int type, const void* dY, const fxp_mx4_layer* layer, int64_t M, int64_t K, int64_t N, void* dX, void* dW, uint64_t seed,
                                  uint64_t step, int rounding, void* ws, size_t ws_bytes, void* stream) {
    using namespace fxp;
    int rc = check_layer(layer, M, K, N, true, dX != nullptr, dW != nullptr);
    if (rc) return rc;
    rc = check_map(type, dY, N, M, N, nullptr, nullptr);
    if (rc) return rc;
    if (!known_rounding(rounding)) return FXP_ERR_ROUNDING;
    for (const void* p : {dX, dW})
        if (!aligned(p, static_cast<size_t>(elem_size(type)))) return FXP_ERR_ALIGN;
    if (!ws || ws_bytes < fxp_mx4_layer_workspace_bytes(M, K, N)) return FXP_ERR_WORKSPACE;
    if (!aligned(ws, 256)) return FXP_ERR_ALIGN;
    if (!dX && !dW) return FXP_OK;
    // what a call does not use may lie anywhere
    const fxp_mx4 none{};
    const std::initializer_list<const fxp_mx4*> operands = {dX ? &layer->dY : &none, dX ? &layer->W : &none, dW ? &layer->dYT : &none, dW ? &layer->XT : &none};
    if (meets_one(type, dY, M, N, {dX ? &layer->dY : &none, dW ? &layer->dYT : &none}) || meets_one(type, dX, M, K, operands) || meets_one(type, dW, K, N, operands) ||
        (dX && dW && meet(dX, M * K * elem_size(type), dW, K * N * elem_size(type))))
        return FXP_ERR_VALUE;
    const Mx4Map m = map_of(dY, N, M, N, dX ? &layer->dY : nullptr, dW ? &layer->dYT : nullptr, (step << 8) | 2);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    rc = mx4_map_launch(type, &m, 1, seed, rounding, s);
    if (!rc && dW && dX && M && K && N) return mx4_gemm_launch2(layer->XT, layer->dYT, dW, layer->dY, layer->W, dX, type, ws, s);
    if (!rc && dW && K && N) rc = mx4_gemm_launch(layer->XT, layer->dYT, type, dW, N, ws, s);
    if (!rc && dX && M && K) rc = mx4_gemm_launch(layer->dY, layer->W, type, dX, K, ws, s);
    return rc;
}
