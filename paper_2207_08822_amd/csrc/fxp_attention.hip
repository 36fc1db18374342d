// Attention over a paged cache of mapped keys and values, with int8 matrix products and the softmax in fp32 (Sec. 5).
//
// A tile is 16 rows (token, query head) of one request and one head of the cache.  All pages of all tiles stand in one line, request
// by request, tile by tile, head by head, and every workgroup takes an equal stretch of it: lengths differ by orders of magnitude
// and are known on the device alone.  A workgroup's waves take the pages of a stretch in turn.  Where a tile's pages fall into several
// stretches, each leaves (largest score, sum, output) of its part in the workspace, and the workgroup that is last to do so joins them.
//
// One page: S^T = K Q^T by v_mfma_i32_16x16x64_i8 with the key rows as they lie in memory as A operand (16 bytes a lane) and
// Q's digits as B; a lane then holds 16 scores of ONE row (column lane % 16), tokens 16 (lane / 16) .. + 15 - the
// rows of A are taken in the order that makes it so - which packed into bytes are exactly the B operand of O^T = V^T P^T, so the
// softmax's weights never leave their lane.
//
// Digits.  A row of Q is v * 2^u with |v| < 2^15 (2^23) and v = 256 d1 + d0 (65536 d2 + ...), d signed bytes; a page's weights
// likewise under their own largest one (below half a unit of it, 2^-16, they add nothing).  Rounding a row to 15 bits is off by up to
// 2^-15 of the lower end of its largest element's binade, or 2^-14 where that element is within 2^-7 of the next: no more than half a
// step of the type for bf16 elements down to 2^-7 (2^-6) of it and fp16 ones down to 2^-4 (2^-3).  Rows with single elements far above
// the rest lose bits of the rest; fp32 rows have 23.  Two digits, because a third of q alone costs 5 % over 70 shapes (4600 rows of
// prompts 250 us against 230, 64 requests of one row 63.6 against 62.3).  Outputs are divided by the sum of the weights as rounded, so
// that they stay weighted means of the values (constant values come out as they are, whatever the scores); the sum of the weights as they
// are serves lse alone.
#include <algorithm>
#include <limits>

#include "fxp_serve_device.h"

namespace fxp {

constexpr int kTile = 16;
constexpr int kFewRows = 2 * kTile;
constexpr int kShortTable = 32;      // pages
constexpr int kAttWaves = 4;
// Workgroups: as many as are resident, one round of them.  Up to 128 elements two a CU (768, which three a CU have room for, split more tiles: 57 -> 67 us
// for 64 requests); rows of more take the registers of one (64 requests of 200 to 4000 tokens, 4 heads of 192: 33 us, 39 with 512 workgroups, 35 with 512 and
// two a CU; of 256, 43, 50 and 61 - spilled).
constexpr int kAttGroups = 512;
template <int DB>
constexpr int kAttGroupsOf = DB <= 2 ? kAttGroups : kAttGroups / 2;

struct AttArgs {
    fxp_kv_cache c;
    const int32_t* first;
    const int32_t* lens;
    const int32_t* table;
    int64_t requests, blocks, tokens;
    const void* q;
    int64_t q_token, q_head;
    void* out;
    int64_t out_token, out_head;
    float* lse;
    float* part_o;          // [workgroup][2][16][dim]: parts of the tiles that the stretch ends in (0) and begins in (1)
    float4* part_ml;        // [workgroup][2][16]: reference score (log2), sum of the weights as rounded, sum of the weights
    uint32_t* tickets;      // [workgroup]: parts that are there of the tile that begins in this stretch and ends in another; zero between calls
    int group;              // query heads per head of the cache
    uint32_t group_inverse; // ceil(2^32 / group): (x * it) >> 32 is x / group for x * group < 2^32
    int vec_q, vec_out;
    float scale_log2;       // scale * log2(e)
    int window;             // 0: none
    float join_turns;       // of a workgroup over the elements of a tile, four a thread, as the requests are on average
    int rows_from;          // requests of more rows are k_kv_attend_rows's, unless they are too long for it
    int walk;               // window > 0: pages that 64 rows see, at most
    bool balance;           // both kernels are launched, and requests that are too long for k_kv_attend_rows left to the other
    int longest;            // walk from which on they are (longest_walk)
};

constexpr int kCus = 256, kShortWalk = 16, kRowWaves = 4, kBlock = kRowWaves * kTile;

// n, len: rows (tokens) and cached tokens of a request; tiles: of kTile rows, 0 where the request is k_kv_attend_rows's
struct Extent {
    int n, len, tiles, page0, pages, tok0;
};
// blocks of kBlock rows of a request of many rows
__device__ inline int blocks_of(const AttArgs& a, const Extent& e) {
    const int rows = e.n * a.group;
    return rows > a.rows_from ? (rows + kBlock - 1) / kBlock : 0;
}
// pages that a workgroup of k_kv_attend_rows goes through one after the other, at most
__device__ inline int walk_of(const AttArgs& a, const Extent& e) { return a.window > 0 ? min(e.pages, a.walk) : e.pages; }
__device__ inline Extent extent(const AttArgs& a, int64_t b) {
    Extent e;
    const int most = static_cast<int>(a.tokens);
    e.tok0 = min(max(a.first[b], 0), most);
    e.n = max(min(max(a.first[b + 1], 0), most) - e.tok0, 0);
    e.len = static_cast<int>(min(static_cast<int64_t>(max(a.lens[b], 0)), a.blocks * FXP_KV_PAGE));
    const int from = a.window > 0 ? max(e.len - e.n + 1 - a.window, 0) : 0;
    e.page0 = from / FXP_KV_PAGE;
    e.pages = max((e.len + FXP_KV_PAGE - 1) / FXP_KV_PAGE - e.page0, 1);       // an empty request still has its zeros to write
    e.tiles = blocks_of(a, e) && walk_of(a, e) <= a.longest ? 0 : (e.n * a.group + kTile - 1) / kTile;
    return e;
}

// The longest walk that k_kv_attend_rows takes on: a CU's share of the pages that all requests of many rows go through there.  It cannot split a
// context, and one that is longer than that would be walked by a few workgroups while the others have nothing left to do; k_kv_attend
// spreads it over all.  (22 requests of 40 rows, 8 heads of 64, one of them of 131000 tokens among 500s: 70 us, 1830 without this rule; all of 8000: 75
// / 127.)  Of one request it is whether it has 256 blocks.  Up to kShortWalk pages it is the better one all the same (22 requests of 500
// tokens: 16 us, 22 of the other).  In whole numbers: both kernels have to come to the same.
__device__ inline int longest_walk(const AttArgs& a) {
    static_assert(kAttWaves == kRowWaves, "workgroups of 256 threads, all of which come here");
    __shared__ unsigned long long s_sum[kAttWaves];
    unsigned long long sum = 0;
    for (int64_t b = threadIdx.x; b < a.requests; b += 64 * kAttWaves) {
        const Extent e = extent(a, b);
        sum += static_cast<unsigned long long>(blocks_of(a, e) * static_cast<int>(a.c.heads)) * static_cast<uint32_t>(walk_of(a, e));
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
    return __builtin_amdgcn_readfirstlane(static_cast<int>(min(max(sum / kCus, uint64_t{kShortWalk}), uint64_t{0x7fffffff})));
}

// Cost of a tile in pages besides its own: its rows of q, the join of its parts, the first loads' way.  (Without it a workgroup
// whose stretch is many short tiles takes as long as several others.)
constexpr int kTileCost = 2 * kAttWaves;

// Pages of a stretch: equal shares, but no fewer than one a wave, nor than this.  A stretch of p pages takes p / kAttWaves turns and the longest tile,
// of P pages, then has P / p parts, which one workgroup joins in `turns` turns over a tile's elements: the sum is least near p ~ sqrt(P turns).
// Measured best factors: 0.5 to 0.7 at one turn (1 head of 16, 4 of 128: 131000 tokens 59 us, 66 with 1.0), 0.7 to 1 at two and three (16 x 128, 14 x 160), 1
// at four (16 x 256, 2 x 32000 tokens: 52 us, 69 with 0.7, 62 with 2).
__device__ inline uint32_t stretch_of(const AttArgs& a, uint32_t units, int most_pages) {
    const uint32_t per = (units + gridDim.x - 1) / gridDim.x;
    const int least = static_cast<int>(0.55f * sqrtf(static_cast<float>(most_pages) * a.join_turns));
    return max(per, static_cast<uint32_t>(max(least, kAttWaves)));
}

__device__ inline int lane_of(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ inline Extent lane_of(const Extent& e, int lane) {
    return {lane_of(e.n, lane), lane_of(e.len, lane), lane_of(e.tiles, lane), lane_of(e.page0, lane), lane_of(e.pages, lane), lane_of(e.tok0, lane)};
}

// Units of all requests (`units_of` each; 32 bits, the host sees to it), and the request that unit at_of(all units, most pages of one) belongs
// to: its number (-1: behind the last), the units before it, its extent.  Every wave by itself: up to 64 requests are loaded once, a lane each;
// of more, a lane sums up a row of neighbours, and the row with the unit in it is gone through again.
struct Found {
    uint32_t units, at, before;
    int b;
    Extent e;
};
template <typename U, typename A>
__device__ inline Found find_request(const AttArgs& a, U units_of, A at_of) {
    const int lane = threadIdx.x & 63, requests = static_cast<int>(a.requests);
    Found found = {};
    found.b = -1;
    auto of_lane = [&](int b, int end, Extent& e) {
        e = Extent{};
        if (b < end) e = extent(a, b);
        return b < end ? units_of(e) : 0u;
    };
    auto take = [&](uint32_t v, uint32_t carry, int base, const Extent& e) {
        const uint32_t x = carry + wave_scan(v) - v;
        const uint64_t hit = __builtin_amdgcn_ballot_w64(found.at >= x && found.at < x + v);
        if (!hit) return false;
        const int w = __builtin_ctzll(hit);
        found.b = base + w;
        found.before = static_cast<uint32_t>(lane_of(static_cast<int>(x), w));
        found.e = lane_of(e, w);
        return true;
    };
    auto last = [](uint32_t v) { return static_cast<uint32_t>(lane_of(static_cast<int>(v), 63)); };
    if (requests <= 64) {
        Extent e;
        const uint32_t v = of_lane(lane, requests, e);
        found.units = last(wave_scan(v));
        found.at = at_of(found.units, static_cast<int>(wave_max(static_cast<uint32_t>(v ? e.pages : 0))));
        take(v, 0, 0, e);
        return found;
    }
    const int row = (requests + 63) / 64;
    uint32_t sum = 0;
    int most = 0;
#pragma unroll 4
    for (int i = 0; i < row; ++i) {
        Extent e;
        const uint32_t v = of_lane(lane * row + i, requests, e);
        sum += v;
        most = max(most, v ? e.pages : 0);
    }
    const uint32_t scan = wave_scan(sum), x = scan - sum;
    found.units = last(scan);
    found.at = at_of(found.units, static_cast<int>(wave_max(static_cast<uint32_t>(most))));
    const uint64_t hit = __builtin_amdgcn_ballot_w64(found.at >= x && found.at < x + sum);
    if (!hit) return found;
    const int w = __builtin_ctzll(hit), end = min((w + 1) * row, requests);
    uint32_t carry = static_cast<uint32_t>(lane_of(static_cast<int>(x), w));
    for (int base = w * row; base < end; base += 64) {
        Extent e;
        const uint32_t v = of_lane(base + lane, end, e);
        if (take(v, carry, base, e)) break;
        carry += last(wave_scan(v));
    }
    return found;
}
// the next request from b on that has tiles, or -1; 64 at a time: a padded batch has many that have none
__device__ inline int next_request(const AttArgs& a, int b, Extent& e) {
    const int lane = threadIdx.x & 63, requests = static_cast<int>(a.requests);
    for (; b < requests; b += 64) {
        Extent x = {};
        if (b + lane < requests) x = extent(a, b + lane);
        const uint64_t hit = __builtin_amdgcn_ballot_w64(x.tiles > 0);
        if (hit) {
            const int w = __builtin_ctzll(hit);
            e = lane_of(x, w);
            return b + w;
        }
    }
    return -1;
}

// T tiles of sums of products of digits, as floats: acc = d1 * 256 + d0 fits 32 bits over 256 terms, a third digit is added in fp32.
// The tiles go through each stage together: a matrix instruction's result can be used some 10 instructions later, and one tile after
// the other (what the compiler makes of a loop over tiles) waits for each.
template <int ND, int N, int T>
__device__ inline void dot_digits(const v4i (&a)[T][N], const v4i (&b)[N][ND], float (&out)[T][4]) {
    v4i acc[ND][T];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int t = 0; t < T; ++t) acc[d][t] = mfma_i8(a[t][0], b[0][d], v4i{0, 0, 0, 0});
#pragma unroll
    for (int i = 1; i < N; ++i)
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int t = 0; t < T; ++t) acc[d][t] = mfma_i8(a[t][i], b[i][d], acc[d][t]);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float top = static_cast<float>((acc[0][t][j] << 8) + acc[1][t][j]);
            if constexpr (ND == 3) out[t][j] = fmaf(top, 256.0f, static_cast<float>(acc[2][t][j]));
            else out[t][j] = top;
        }
}

// over the four lanes that hold a row, inside the vector ALU: exchanges of rows of 16 and of halves
template <typename F>
__device__ inline float over_row(float v, F f) {
    const uint32_t a = __float_as_uint(v);
    const auto x = __builtin_amdgcn_permlane16_swap(a, a, false, false);
    const uint32_t b = __float_as_uint(f(__uint_as_float(x[0]), __uint_as_float(x[1])));
    const auto y = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return f(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ inline float swap_max(float v) {
    return over_row(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ inline float swap_sum(float v) {
    return over_row(v, [](float a, float b) { return a + b; });
}

// This lane's row of Q (zeros where there is none); its digits, and the exponent of their unit
template <int TYPE, int DB>
__device__ inline void load_query(const AttArgs& a, const Extent& e, int tok, int qh, bool row_ok, int g, float (&x)[DB][16]) {
#pragma unroll
    for (int i = 0; i < DB; ++i) {
        const int d = 64 * i + 16 * g;
        if (row_ok && d < a.c.dim) {
            load_elems<TYPE, 16>(a.q, (int64_t{e.tok0} + tok) * a.q_token + qh * a.q_head + d, a.vec_q, x[i]);
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) x[i][j] = 0.0f;
        }
    }
}
template <int DB, int ND>
__device__ inline int query_digits(const float (&x)[DB][16], v4i (&qd)[DB][ND]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) m = max(m, __float_as_uint(x[i][j]) & 0x7fffffffu);
    m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 16)));
    m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 32)));
    const int unit = unit_of<ND>(m);
    const bool finite = !__any(m >= 0x7f800000u);
#pragma unroll
    for (int i = 0; i < DB; ++i) row_digits<ND>(x[i], unit, finite, qd[i]);
    return unit;
}

// Weights 2^(f s - top) of 16 scores as digits, and their sum before the rounding; `top` becomes the score that weighs 1 (32767 / 32639 for two digits: the
// packing conversion multiplies by 32767, and the largest weight has to stay at 127 in each digit).  rounded: of three digits, the sum
// of the weights in their units.
template <int ND>
__device__ inline float weigh(const float (&s)[16], float f, float& top, v4i (&pd)[1][ND], int& rounded) {
    float l = 0.0f;
    rounded = 0;
    if constexpr (ND == 2) {
        top += 0.00564698f;                    // log2(32767 / 32639), rounded up
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            float w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = __builtin_amdgcn_exp2f(fmaf(s[4 * t + i], f, -top));
                l += w[i];
            }
            typedef short v2s __attribute__((ext_vector_type(2)));
            const v2s a = __builtin_amdgcn_cvt_pknorm_i16(w[0], w[1]), b = __builtin_amdgcn_cvt_pknorm_i16(w[2], w[3]);
            const uint32_t x = __builtin_bit_cast(uint32_t, a) + 0x00800080u, y = __builtin_bit_cast(uint32_t, b) + 0x00800080u;
            pd[0][0][t] = static_cast<int>(perm(y, x, 0x07050301u));
            pd[0][1][t] = static_cast<int>(perm(y, x, 0x06040200u) ^ 0x80808080u);
        }
    } else {
        int v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float w = __builtin_amdgcn_exp2f(fmaf(s[i], f, -top));
            l += w;
            v[i] = static_cast<int>(rintf(w * Digits<ND>::kMost));
            rounded += v[i];
        }
        digits16<ND>(v, pd[0]);
    }
    return l;
}
template <int ND>
constexpr float kWeightUnit = ND == 2 ? 1.0f / 32767 : 1.0f / 8355711;

// The score that a row's sums are relative to: the first page's largest, and a new one where a page's is 8 (in log2) above it.  Sums
// grow by 2^8 at most in between, which fp32 has room for, and rescaling the outputs (a fifth of a page's vector work) is rare;
// a running maximum rises for some row of a tile on most pages.
struct Turn {
    float ref, keep, gain;
};
__device__ inline Turn next_reference(float ref, float page) {
    const float next = page > ref + 8.0f ? page : ref, r = next == -INFINITY ? 0.0f : next;     // -Inf + 8 = -Inf: the first page takes it
    return {next, __builtin_amdgcn_exp2f(ref - r), __builtin_amdgcn_exp2f(page - r)};
}

// What a sum of products of digits is multiplied with (2^`unit` is that of the sum).  Bounded so that no product of it and a sum (2^15 or 2^23,
// 7 bits, up to 256 terms) passes 2^127, and not zero: no Inf - Inf and no 0 * Inf in the softmax.
template <int ND>
__device__ inline float score_unit(const AttArgs& a, int unit) {
    return fminf(fmaxf(ldexpf(a.scale_log2, unit), 0x1p-126f), ND == 2 ? 0x1p97f : 0x1p89f);
}
// scores of places that this lane's row does not see: those behind `to` and before `from`, or all
__device__ inline void hide(float (&s)[16], bool all, int to, int from) {
    const int last = all ? -1 : to;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = ((i > last) | (i < from)) ? -INFINITY : s[i];
}
// One page of a row: the weights of this lane's 16 scores f * s as digits, the row's reference and sum (of this lane's tokens, for lse) moved on.
template <int ND>
__device__ inline Turn softmax_page(const float (&s)[16], float f, float& ref, float& l, v4i (&pd)[1][ND], int& rounded) {
    float m = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) m = fmaxf(m, s[i]);
    m = swap_max(m) * f;
    // a little above the largest score: f s - top rounds once, and must not come out above 0
    float top = m == -INFINITY ? 0.0f : fmaf(fabsf(m), 0x1p-22f, m);
    const float sum = weigh<ND>(s, f, top, pd, rounded);
    const Turn turn = next_reference(ref, m == -INFINITY ? m : top);
    l = l * turn.keep + sum * turn.gain;
    ref = turn.ref;
    return turn;
}

// One page's values, weighted by `pd`, added to a row's outputs in units of `fv`, and the sum of these weights to `r` in units of `fr`: two
// digits by one more tile of the products, whose values are ones, for all 64 tokens (the matrix cores have the time); three, which have no
// registers for its sums (12 spilled), by `rounded`, that of this lane's 16 tokens.
// value_of(i): this lane's bytes of the i-th 16 elements of the page's values.
template <int ND, int DB, typename F>
__device__ inline void add_values(F value_of, const v4i (&pd)[1][ND], int rounded, float fv, float fr, float (&o)[4 * DB][4], float& r) {
    auto add = [&](int i, const float(&y)[4]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) o[i][j] = fmaf(y[j], fv, o[i][j]);
    };
    if constexpr (ND == 3) r = fmaf(static_cast<float>(rounded), fr, r);
#pragma unroll
    for (int i = 0; i < 4 * DB; i += 4) {
        if (ND == 2 && i == 0) {
            constexpr int kOnes = 0x01010101;
            const v4i five[5][1] = {{value_of(0)}, {value_of(1)}, {value_of(2)}, {value_of(3)}, {v4i{kOnes, kOnes, kOnes, kOnes}}};
            float y[5][4];
            dot_digits<ND, 1, 5>(five, pd, y);
            r = fmaf(y[4][0], fr, r);
#pragma unroll
            for (int t = 0; t < 4; ++t) add(t, y[t]);
        } else {
            const v4i four[4][1] = {{value_of(i)}, {value_of(i + 1)}, {value_of(i + 2)}, {value_of(i + 3)}};
            float y[4][4];
            dot_digits<ND, 1, 4>(four, pd, y);
#pragma unroll
            for (int t = 0; t < 4; ++t) add(i + t, y[t]);
        }
    }
}
// the sum over a row's lanes, where add_values left each its own part
template <int ND>
__device__ inline float whole_sum(float r) {
    return ND == 3 ? swap_sum(r) : r;
}

// Rows of a tile: row i is token tok + (rest + i) / group of the request, head (rest + i) % group of its group.
struct TileRows {
    int tok, rest;
    __device__ void at(const AttArgs& a, int i, int& t, int& h) const {
        const int x = rest + i, q = static_cast<int>(__umulhi(static_cast<uint32_t>(x), a.group_inverse));
        t = tok + (a.group == 1 ? x : q);                               // the inverse of 1 does not fit
        h = x - (a.group == 1 ? x : q * a.group);
    }
};
__device__ inline TileRows tile_rows(const AttArgs& a, int tile) {
    const int r = tile * kTile, tok = static_cast<int>(static_cast<uint32_t>(r) / static_cast<uint32_t>(a.group));
    return {tok, r - tok * a.group};
}

// one row's share of four elements, and the join of two shares
struct Share {
    float m, r, x[4];           // reference, sum of the weights as rounded, elements
};
__device__ inline void join(Share& s, float m, float r, const float4 y) {
    const float top = fmaxf(s.m, m), ref = top == -INFINITY ? 0.0f : top;
    const float keep = __builtin_amdgcn_exp2f(s.m - ref), gain = __builtin_amdgcn_exp2f(m - ref);
    s.m = top;
    s.r = s.r * keep + r * gain;
    s.x[0] = s.x[0] * keep + y.x * gain;
    s.x[1] = s.x[1] * keep + y.y * gain;
    s.x[2] = s.x[2] * keep + y.z * gain;
    s.x[3] = s.x[3] * keep + y.w * gain;
}
// two floats to and from memory that other XCDs see: atomic accesses of device scope pass their L2 caches
__device__ inline void store_part(float* p, float x, float y) {
    const uint64_t v = static_cast<uint64_t>(__float_as_uint(y)) << 32 | __float_as_uint(x);
    __hip_atomic_store(reinterpret_cast<uint64_t*>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline float2 load_part(const float* p) {
    const uint64_t v = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float(static_cast<uint32_t>(v)), __uint_as_float(static_cast<uint32_t>(v >> 32)));
}
template <int TYPE>
__device__ inline void finish(const AttArgs& a, const Extent& e, const TileRows& rows_of, int head, int row, int d, Share s) {
    int tok, in_group;
    rows_of.at(a, row, tok, in_group);
    const float inv = s.r > 0.0f ? 1.0f / s.r : 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) s.x[j] *= inv;
    store4<TYPE>(a.out, (int64_t{e.tok0} + tok) * a.out_token + (head * a.group + in_group) * a.out_head + d, a.vec_out, s.x);
}
__device__ inline void finish_lse(const AttArgs& a, const Extent& e, const TileRows& rows_of, int head, int row, float m, float l) {
    int tok, in_group;
    rows_of.at(a, row, tok, in_group);
    a.lse[(int64_t{e.tok0} + tok) * (static_cast<int>(a.c.heads) * a.group) + head * a.group + in_group] =
        l > 0.0f ? (m + log2f(l)) * 0.693147180559945f : -INFINITY;
}

template <int TYPE, int DB>
__global__ __launch_bounds__(64 * kAttWaves, DB <= 2 ? 2 : 1) void k_kv_attend(AttArgs a) {
    constexpr int ND = TYPE == FXP_F32 ? 3 : 2, WAVES = kAttWaves, THREADS = 64 * WAVES, COST = kTileCost;
    constexpr int DMAX = 64 * DB, ROW = DMAX + 4;
    __shared__ float s_m[WAVES][kTile], s_r[WAVES][kTile], s_l[WAVES][kTile];
    __shared__ float4 s_o4[WAVES * kTile * ROW / 4];
    __shared__ int s_last;
    float* const s_o = reinterpret_cast<float*>(s_o4);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
    const int dim = static_cast<int>(a.c.dim), heads = static_cast<int>(a.c.heads), nd = dim / 4;
    uint32_t per = 0;
    if (a.balance) a.longest = longest_walk(a);
    const Found st = find_request(
        a, [&](const Extent& x) { return static_cast<uint32_t>(x.tiles * heads) * static_cast<uint32_t>(x.pages + COST); },
        [&](uint32_t units, int most_pages) {
            per = stretch_of(a, units, most_pages);
            return per * blockIdx.x;
        });
    const uint32_t u0 = st.at, u1 = min(u0 + per, st.units);
    if (st.b < 0) return;                                               // behind the end of the line
    int b = st.b;
    Extent e = st.e;
    // the tile of unit u0, and its first unit
    const uint32_t first_seg = (u0 - st.before) / static_cast<uint32_t>(e.pages + COST);
    int tile = static_cast<int>(first_seg / static_cast<uint32_t>(heads)), head = static_cast<int>(first_seg - static_cast<uint32_t>(tile * heads));
    uint32_t s0 = st.before + first_seg * static_cast<uint32_t>(e.pages + COST);

    while (s0 < u1) {
        // this workgroup's pages of the tile
        const int ahead = static_cast<int>(u0 - s0) - COST;             // of the stretch's begin, from the tile's first page
        const int p0 = max(ahead, 0), p1 = min(static_cast<int>(u1 - s0) - COST, e.pages);
        if (p0 < p1) {
            const TileRows rows_of = tile_rows(a, tile);
            int tok, in_group;
            rows_of.at(a, col, tok, in_group);
            const int qh = head * a.group + in_group;
            const bool row_ok = tok < e.n;
            const int place = e.len - e.n + tok;                       // negative: more rows than tokens; such a row sees nothing
            const int see_to = row_ok ? min(place, e.len - 1) : -1;
            const int see_from = a.window > 0 ? max(place - a.window + 1, 0) : 0;
            // places that every row of the tile sees
            const int rows = min(e.n * a.group - tile * kTile, kTile);
            int last_tok, unused;
            rows_of.at(a, rows - 1, last_tok, unused);
            const int all_to = e.len - e.n + rows_of.tok;
            const int all_from = a.window > 0 ? max(e.len - e.n + last_tok - a.window + 1, 0) : 0;

            // The pages' numbers: lane i has that of the wave's i-th page of 64.
            const int32_t* const table = a.table + int64_t{b} * a.blocks + e.page0;
            int from = p0 + wave, ids = -1;
            auto load_ids = [&] {
                const int p = from + WAVES * lane;
                ids = p < p1 ? table[p] : -1;
            };
            load_ids();
            float x[DB][16];
            load_query<TYPE, DB>(a, e, tok, qh, row_ok, g, x);

            // A page's loads are issued while the page before it is worked on, and always: a page that is none has no records, which costs
            // nothing.  (Behind a branch their number is unknown to the compiler, which then waits for all of them where it needs one, and
            // keeps 64-bit addresses: 235 registers in place of 179, 21.3 us in place of 19.7 for a few guessed tokens over windows of 1500.)  A
            // block's address is uniform; elements behind dim are loaded from the row's first ones - Q's digits are zero there.
            constexpr bool kAhead = DB * ND <= 4;                       // values too, where there are registers for them
            v4i kf[4][DB], vf[4 * DB];
            int ek_next = 0, ev_next = 0;
            bool dead_next = true;
            int64_t at_next = 0;
            const uint32_t k_row = static_cast<uint32_t>((16 * (col >> 2) + (col & 3)) * dim), k_off = k_row + 16u * g;
            const uint32_t k_last = 64 * (DB - 1) + 16 * g < dim ? k_row + 64u * (DB - 1) + 16u * g : k_row, v_off = static_cast<uint32_t>((g * dim + col) * 16);
            const int block_bytes = FXP_KV_PAGE * dim;
            auto piece = [&](const int8_t* base, int64_t at, bool dead, uint32_t lane_off, int off) {
                return __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(records(base + at * block_bytes, dead ? 0 : block_bytes), lane_off,
                                                                                     off, kNonTemporal));
            };
            auto load_k = [&](int64_t at, bool dead) {
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int i = 0; i < DB; ++i) kf[t][i] = piece(a.c.kq, at, dead, i < DB - 1 ? k_off : k_last, 4 * t * dim + (i < DB - 1 ? 64 * i : 0));
            };
            auto load_v = [&](int64_t at, bool dead) {
#pragma unroll
                for (int i = 0; i < 4 * DB; ++i) vf[i] = piece(a.c.vq, at, dead, v_off, i < 4 * (DB - 1) ? 256 * i : min(256 * i, 16 * (dim - 16)));
            };
            // scales and keys of the page that lane `index` has the number of
            auto begin = [&](int index) {
                const int id = __builtin_amdgcn_readlane(ids, index);
                dead_next = id < 0 || id >= a.c.pages;
                at_next = int64_t{dead_next ? 0 : id} * heads + head;
                ek_next = a.c.ek[at_next];
                ev_next = a.c.ev[at_next];
            };
            begin(0);
            load_k(at_next, dead_next);
            if (kAhead) load_v(at_next, dead_next);

            float o[4 * DB][4];
            float m_run = -INFINITY, r_run = 0.0f, l_run = 0.0f;       // l_run: of this lane's 16 tokens of each page
#pragma unroll
            for (int i = 0; i < 4 * DB; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[i][j] = 0.0f;
            v4i qd[DB][ND];
            const int qe = query_digits<DB, ND>(x, qd);

            while (from < p1) {
                const int count = min((p1 - from + WAVES - 1) / WAVES, 64);
                for (int n = 0; n < count; ++n) {
                    const int ek = min(max(ek_next, 1), 255) - 125 - a.c.bits, ev = min(max(ev_next, 1), 255) - 125 - a.c.bits;
                    const bool dead = dead_next;
                    if (!kAhead) load_v(at_next, dead);
                    begin(min(n + 1, count - 1));
                    const bool none = dead_next || n + 1 == count;
                    float s4[4][4];
                    dot_digits<ND, DB, 4>(kf, qd, s4);
                    load_k(at_next, none);                              // on their way while the softmax is worked out
                    float s[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = s4[i / 4][i % 4];
                    const int j0 = (e.page0 + from + WAVES * n) * FXP_KV_PAGE;
                    if (dead || j0 + FXP_KV_PAGE - 1 > all_to || j0 < all_from) hide(s, dead, see_to - j0 - 16 * g, see_from - j0 - 16 * g);
                    v4i pd[1][ND];
                    int rounded;
                    const Turn turn = softmax_page<ND>(s, score_unit<ND>(a, qe + ek), m_run, l_run, pd, rounded);
                    const float fr = turn.gain * kWeightUnit<ND>, fv = ldexpf(fr, ev);
                    if (__any(turn.keep != 1.0f)) {
                        r_run *= turn.keep;
#pragma unroll
                        for (int i = 0; i < 4 * DB; ++i)
#pragma unroll
                            for (int j = 0; j < 4; ++j) o[i][j] *= turn.keep;
                    }
                    add_values<ND, DB>([&](int i) { return vf[i]; }, pd, rounded, fv, fr, o, r_run);
                    if (kAhead) load_v(at_next, none);
                }
                from += 64 * WAVES;
                if (from < p1) {
                    load_ids();
                    begin(0);
                    load_k(at_next, dead_next);
                    if (kAhead) load_v(at_next, dead_next);
                }
            }

            // the waves' parts
            l_run = swap_sum(l_run);
            r_run = whole_sum<ND>(r_run);
            if (g == 0) {
                s_m[wave][col] = m_run;
                s_r[wave][col] = r_run;
                s_l[wave][col] = l_run;
            }
#pragma unroll
            for (int i = 0; i < 4 * DB; ++i)
                *reinterpret_cast<float4*>(s_o + (wave * kTile + col) * ROW + 16 * i + 4 * g) = make_float4(o[i][0], o[i][1], o[i][2], o[i][3]);
            __syncthreads();
            // the workgroups that have pages of this tile: w_first .. w_last; all but the first have it at the start of their stretch
            const int behind = static_cast<int>(s0 - u0) + COST + e.pages - 1;
            const int w_first = static_cast<int>(blockIdx.x) - (ahead > 0 ? static_cast<int>((static_cast<uint32_t>(ahead) + per - 1) / per) : 0);
            const int w_last = static_cast<int>(min(blockIdx.x + static_cast<uint32_t>(behind) / per, gridDim.x - 1));
            const bool whole = w_first == w_last;
            for (int i = threadIdx.x; i < rows * nd; i += THREADS) {
                const int row = i / nd, d = i % nd * 4;
                Share s = {s_m[0][row], 0.0f, {0.0f, 0.0f, 0.0f, 0.0f}};
                float l = 0.0f;
#pragma unroll
                for (int w = 1; w < WAVES; ++w) s.m = fmaxf(s.m, s_m[w][row]);
                const float ref = s.m == -INFINITY ? 0.0f : s.m;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    const float f = __builtin_amdgcn_exp2f(s_m[w][row] - ref);
                    const float4 y = *reinterpret_cast<const float4*>(s_o + (w * kTile + row) * ROW + d);
                    s.r = fmaf(s_r[w][row], f, s.r);
                    l = fmaf(s_l[w][row], f, l);
                    s.x[0] = fmaf(y.x, f, s.x[0]);
                    s.x[1] = fmaf(y.y, f, s.x[1]);
                    s.x[2] = fmaf(y.z, f, s.x[2]);
                    s.x[3] = fmaf(y.w, f, s.x[3]);
                }
                if (whole) {
                    finish<TYPE>(a, e, rows_of, head, row, d, s);
                    if (a.lse && d == 0) finish_lse(a, e, rows_of, head, row, s.m, l);
                } else {
                    const int64_t part = (int64_t{blockIdx.x} * 2 + (static_cast<int>(blockIdx.x) == w_first)) * kTile + row;
                    store_part(a.part_o + part * dim + d, s.x[0], s.x[1]);
                    store_part(a.part_o + part * dim + d + 2, s.x[2], s.x[3]);
                    if (d == 0) {
                        store_part(&a.part_ml[part].x, s.m, s.r);
                        store_part(&a.part_ml[part].z, l, 0.0f);
                    }
                }
            }
            if (!whole) {
                // The last to arrive joins the parts.  Parts are stored past the L2 of this XCD (store_part) and loaded past that of the
                // reader's, so it is enough that every wave's stores are there before the ticket is drawn.  That is no happens-before of the
                // memory model: it rests on what this chip does with relaxed atomics of device scope, whose stores write through to memory and
                // whose loads do not end in an L2, and on the wait, which lasts until the stores have arrived.  Release and acquire fences
                // instead write back and drop whole L2 caches, in every workgroup: 97 us in place of 65 for 64 requests of 200 to 8000 tokens.
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __syncthreads();
                if (threadIdx.x == 0) {
                    uint32_t* ticket = a.tickets + w_first;             // no other tile begins there and ends elsewhere
                    const uint32_t others = static_cast<uint32_t>(w_last - w_first);
                    s_last = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == others;
                    if (s_last) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                }
                __syncthreads();
                if (s_last) {
                    // `ways` threads share four elements of a row
                    constexpr int kBatch = 4;                           // (32000 tokens, 16 rows of one head of 128: 25 us; one by one 37, sixteen 28)
                    const int work = rows * nd, ways = max(THREADS / work, 1);
                    for (int i0 = 0; i0 < work; i0 += THREADS) {
                        const int i = i0 + static_cast<int>(threadIdx.x) % (work < THREADS ? work : THREADS);
                        const int way = work < THREADS ? static_cast<int>(threadIdx.x) / work : 0;
                        Share s = {-INFINITY, 0.0f, {0.0f, 0.0f, 0.0f, 0.0f}};
                        if (i < work && way < ways) {
                            const int row = i / nd, d = i % nd * 4;
                            // kBatch parts on their way at a time; one behind the last is the last again, left out of the sum
                            for (int w0 = w_first + way; w0 <= w_last; w0 += kBatch * ways) {
                                float2 mr[kBatch], x[kBatch], y[kBatch];
#pragma unroll
                                for (int n = 0; n < kBatch; ++n) {
                                    const int w = min(w0 + n * ways, w_last);
                                    const int64_t part = (int64_t{w} * 2 + (w == w_first)) * kTile + row;
                                    mr[n] = load_part(&a.part_ml[part].x);
                                    x[n] = load_part(a.part_o + part * dim + d);
                                    y[n] = load_part(a.part_o + part * dim + d + 2);
                                }
#pragma unroll
                                for (int n = 0; n < kBatch; ++n)
                                    if (w0 + n * ways <= w_last) join(s, mr[n].x, mr[n].y, make_float4(x[n].x, x[n].y, y[n].x, y[n].y));
                            }
                        }
                        if (ways > 1) {                                 // work < THREADS: one turn of the outer loop
                            s_o4[threadIdx.x] = make_float4(s.x[0], s.x[1], s.x[2], s.x[3]);
                            s_o4[THREADS + threadIdx.x] = make_float4(s.m, s.r, 0.0f, 0.0f);
                            __syncthreads();
                            if (way == 0)
                                for (int w = 1; w < ways; ++w) {
                                    const float4 mr = s_o4[THREADS + i + w * work];
                                    join(s, mr.x, mr.y, s_o4[i + w * work]);
                                }
                        }
                        if (i < work && way == 0) finish<TYPE>(a, e, rows_of, head, i / nd, i % nd * 4, s);
                    }
                    // apart from the rest: in the loop above these loads cost calls without lse as much (52000 tokens, 2 heads of 128: 31 us, 23 so)
                    if (a.lse && static_cast<int>(threadIdx.x) < rows) {
                        float m = -INFINITY, l = 0.0f;
                        for (int w = w_first; w <= w_last; ++w) {
                            const float* const part = &a.part_ml[(int64_t{w} * 2 + (w == w_first)) * kTile + threadIdx.x].x;
                            const float m_part = load_part(part).x, l_part = load_part(part + 2).x, top = fmaxf(m, m_part);
                            const float ref = top == -INFINITY ? 0.0f : top;
                            l = l * __builtin_amdgcn_exp2f(m - ref) + l_part * __builtin_amdgcn_exp2f(m_part - ref);
                            m = top;
                        }
                        finish_lse(a, e, rows_of, head, threadIdx.x, m, l);
                    }
                }
            }
            __syncthreads();
        }
        // on to the next tile
        s0 += e.pages + COST;
        if (++head == heads) {
            head = 0;
            if (++tile == e.tiles) {
                tile = 0;
                b = next_request(a, b + 1, e);
                if (b < 0) return;
            }
        }
    }
}

// ---- many rows of one request (prompts) ----
//
// A workgroup has 64 consecutive rows of one request and head, each of its four waves a tile of 16.  The waves share the pages:
// each page goes through LDS once (two buffers, the next page's loads in registers meanwhile).  Per page a wave issues 16 DB + 2
// matrix instructions of 16 cycles (two digits) and, at DB = 2, some 295 vector instructions, which is what bounds it: the vector ALU is busy 83 % of
// the time, the matrix cores 32 % (4600 rows behind up to 7000, 16 heads over 4 of 128: 221 us, 255 in the first calls of a process; in such
// calls 1, 2 and 3 workgroups a CU took 480, 305 and 250, and 32 rows a wave, which halves the LDS reads, 303: fewer, longer workgroups).
// In LDS the keys stand by pieces of 16 elements, [dim / 16][64 places][16], the places in the order that the A operand takes
// them, turned by twice the piece's number: 16 lanes then read 256 consecutive bytes, and the 16 pieces that 16
// lanes write (8 of a token, two tokens) fall on 16 different ones.
template <int TYPE, int DB>
__global__ __launch_bounds__(64 * kRowWaves, DB <= 2 ? 3 : 2) void k_kv_attend_rows(AttArgs a) {
    constexpr int ND = TYPE == FXP_F32 ? 3 : 2, PAGE_BYTES = 64 * 64 * DB, THREADS = 64 * kRowWaves;
    __shared__ v4i lds[2][2][PAGE_BYTES / 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
    const int dim = static_cast<int>(a.c.dim), heads = static_cast<int>(a.c.heads);

    // the request and the block of its rows, too long ones among them; the last blocks come first, because they see the most pages
    const int line = static_cast<int>(gridDim.x - 1 - blockIdx.x), want = line / heads, head = line - want * heads;
    const Found found = find_request(
        a, [&](const Extent& x) { return static_cast<uint32_t>(blocks_of(a, x)); }, [&](uint32_t, int) { return static_cast<uint32_t>(want); });
    if (found.b < 0) return;
    // (a request's own pages are its walk for each of its blocks: of 256 blocks and more it is within the share, whatever the others are)
    const int walk = walk_of(a, found.e);
    if (a.balance && walk > kShortWalk && blocks_of(a, found.e) * heads < kCus && walk > longest_walk(a)) return;
    const int b = found.b, block = want - static_cast<int>(found.before);
    const Extent e = found.e;

    // this lane's rows
    int tok, in_group;
    const TileRows wave_of = tile_rows(a, block * kRowWaves + wave);
    wave_of.at(a, col, tok, in_group);
    const bool row_ok = tok < e.n;
    const int shift = e.len - e.n, place = shift + tok;
    const int see_to = row_ok ? min(place, e.len - 1) : -1;
    const int see_from = a.window > 0 ? max(place - a.window + 1, 0) : 0;
    v4i qd[DB][ND];
    float x[DB][16];
    load_query<TYPE, DB>(a, e, tok, head * a.group + in_group, row_ok, g, x);
    const int qe = query_digits<DB, ND>(x, qd);
    // pages that any row of the workgroup sees, places that every and any row of the wave does
    const TileRows first_of = tile_rows(a, block * kRowWaves);
    int last_tok, wave_last, unused;
    first_of.at(a, kBlock - 1, last_tok, unused);
    wave_of.at(a, kTile - 1, wave_last, unused);
    last_tok = min(last_tok, e.n - 1);
    wave_last = min(wave_last, e.n - 1);
    const int p_end = min((max(shift + last_tok + 1, 0) + FXP_KV_PAGE - 1) / FXP_KV_PAGE, (e.len + FXP_KV_PAGE - 1) / FXP_KV_PAGE);
    const int p_begin = a.window > 0 ? max(shift + first_of.tok - a.window + 1, 0) / FXP_KV_PAGE : 0;
    const int all_to = shift + wave_of.tok, any_to = shift + wave_last;
    const int all_from = a.window > 0 ? max(shift + wave_last - a.window + 1, 0) : 0;

    // pieces of 16 bytes that this thread brings in, and where the keys among them go
    const int pieces = 4 * dim, per_row = dim / 16;
    int k_to[DB];
#pragma unroll
    for (int j = 0; j < DB; ++j) {
        const int piece = threadIdx.x + THREADS * j, token = piece / per_row, c = piece - token * per_row;
        k_to[j] = c * 64 + ((((token >> 2) & 3) * 16 + (token >> 4) * 4 + (token & 3)) ^ ((2 * c) & 15));
    }
    v4i kin[DB], vin[DB];
    const int32_t* const table = a.table + int64_t{b} * a.blocks;
    int ek_next = 0, ev_next = 0;
    bool dead_next = true;
    int id_next = p_begin < p_end ? table[p_begin] : -1;          // of the page that is fetched next
    auto fetch = [&](int p) {
        const int id = __builtin_amdgcn_readfirstlane(id_next);
        id_next = table[min(p + 1, p_end - 1)];
        dead_next = id < 0 || id >= a.c.pages;
        const int64_t at = int64_t{dead_next ? 0 : id} * heads + head;
        ek_next = a.c.ek[at];
        ev_next = a.c.ev[at];
        const v4i* const kp = reinterpret_cast<const v4i*>(a.c.kq + at * (FXP_KV_PAGE * dim));
        const v4i* const vp = reinterpret_cast<const v4i*>(a.c.vq + at * (FXP_KV_PAGE * dim));
#pragma unroll
        for (int j = 0; j < DB; ++j) {
            const int piece = min(static_cast<int>(threadIdx.x) + THREADS * j, pieces - 1);
            kin[j] = kp[piece];
            vin[j] = vp[piece];
        }
    };
    auto put = [&](int buffer) {
#pragma unroll
        for (int j = 0; j < DB; ++j) {
            const int piece = threadIdx.x + THREADS * j;
            if (piece < pieces) {
                lds[buffer][0][k_to[j]] = kin[j];
                lds[buffer][1][piece] = vin[j];
            }
        }
    };

    float o[4 * DB][4], m_run = -INFINITY, r_run = 0.0f, l_run = 0.0f;
#pragma unroll
    for (int i = 0; i < 4 * DB; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[i][j] = 0.0f;
    if (p_begin < p_end) {
        fetch(p_begin);
        put(0);
    }
    __syncthreads();
    int buffer = 0;
    for (int p = p_begin; p < p_end; ++p, buffer ^= 1) {
        const bool dead = dead_next;
        const int ek = min(max(ek_next, 1), 255) - 125 - a.c.bits, ev = min(max(ev_next, 1), 255) - 125 - a.c.bits;
        if (p + 1 < p_end) fetch(p + 1);
        const int j0 = p * FXP_KV_PAGE;
        if (j0 <= any_to && j0 + FXP_KV_PAGE - 1 >= (a.window > 0 ? shift + wave_of.tok - a.window + 1 : 0)) {
            const v4i* const kl = lds[buffer][0];
            const v4i* const vl = lds[buffer][1];
            float s[16];
            constexpr int QT = 2;                                       // tiles of tokens at a time: four take 32 registers more, and spill in fp32
#pragma unroll
            for (int h = 0; h < 4; h += QT) {
                v4i kf[QT][DB];
#pragma unroll
                for (int t = 0; t < QT; ++t)
#pragma unroll
                    for (int i = 0; i < DB; ++i) kf[t][i] = kl[(4 * i + g) * 64 + ((16 * (h + t) + col) ^ ((2 * (4 * i + g)) & 15))];
                float part[QT][4];
                dot_digits<ND, DB, QT>(kf, qd, part);
#pragma unroll
                for (int i = 0; i < 4 * QT; ++i) s[4 * h + i] = part[i / 4][i % 4];
            }
            if (dead || j0 + FXP_KV_PAGE - 1 > all_to || j0 < all_from) hide(s, dead, see_to - j0 - 16 * g, see_from - j0 - 16 * g);
            v4i pd[1][ND];
            int rounded;
            const Turn turn = softmax_page<ND>(s, score_unit<ND>(a, qe + ek), m_run, l_run, pd, rounded);
            const float fr = turn.gain * kWeightUnit<ND>, fv = ldexpf(fr, ev);
            if (__any(turn.keep != 1.0f)) {
                r_run *= turn.keep;
#pragma unroll
                for (int i = 0; i < 4 * DB; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[i][j] *= turn.keep;
            }
            add_values<ND, DB>([&](int i) { return vl[g * dim + 16 * i + col]; }, pd, rounded, fv, fr, o, r_run);
        }
        if (p + 1 < p_end) put(buffer ^ 1);
        __syncthreads();
    }
    const float l = swap_sum(l_run), r = whole_sum<ND>(r_run), inv = r > 0.0f ? 1.0f / r : 0.0f;
    if (!row_ok) return;
    const int64_t t = int64_t{e.tok0} + tok;
    const int h = head * a.group + in_group;
#pragma unroll
    for (int i = 0; i < 4 * DB; ++i) {
        if (16 * i >= dim) continue;
        float x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = o[i][j] * inv;
        store4<TYPE>(a.out, t * a.out_token + h * a.out_head + 16 * i + 4 * g, a.vec_out, x);
    }
    if (a.lse && g == 0) a.lse[t * (heads * a.group) + h] = l > 0.0f ? (m_run + log2f(l)) * 0.693147180559945f : -INFINITY;
}

static bool attention_sizes_ok(int64_t requests, int64_t tokens, int64_t q_heads, int64_t heads, int64_t dim) {
    constexpr int64_t kMost = int64_t{1} << 31;
    return requests > 0 && requests < kMost && tokens >= 0 && tokens < kMost && heads > 0 && heads <= 65535 && q_heads > 0 &&
           q_heads <= 16384 && q_heads % heads == 0 && dim > 0 && dim <= 256 && dim % 16 == 0 && tokens * q_heads < kMost;
}

}  // namespace fxp

extern "C" size_t fxp_kv_attention_workspace_bytes(int64_t requests, int64_t tokens, int64_t q_heads, int64_t heads, int64_t dim) {
    if (!fxp::attention_sizes_ok(requests, tokens, q_heads, heads, dim)) return 0;
    return FXP_KV_TICKET_BYTES + static_cast<size_t>(fxp::kAttGroups) * 2 * fxp::kTile * (dim * sizeof(float) + sizeof(float4));
}

extern "C" int fxp_kv_attention(const fxp_kv_cache* cache, const fxp_kv_step* st, int type, const void* q, int64_t q_token, int64_t q_head,
                                int64_t q_heads, float scale, int64_t window, void* out, int64_t out_token, int64_t out_head, float* lse,
                                void* ws, size_t ws_bytes, void* stream) {
    using namespace fxp;
    const int rc = check_cache(cache);
    if (rc) return rc;
    if (!st) return FXP_ERR_NULL;
    if (!known_type(type)) return FXP_ERR_TYPE;
    if (!attention_sizes_ok(st->requests, st->tokens, q_heads, cache->heads, cache->dim) || st->blocks <= 0 ||
        st->blocks >= (int64_t{1} << 31) / FXP_KV_PAGE || window < 0 || !strides_ok(q_token, q_head) || !strides_ok(out_token, out_head))
        return FXP_ERR_DIMS;
    if (!(scale > 0.0f) || !(scale < 0x1p64f)) return FXP_ERR_VALUE;
    if (st->tokens == 0) return FXP_OK;
    if (!q || !out || !st->first || !st->lens_after || !st->block_table) return FXP_ERR_NULL;
    const size_t size = elem_size(type);
    if (!aligned(q, size) || !aligned(out, size) || !aligned(st->first, 4) || !aligned(st->lens_after, 4) || !aligned(st->block_table, 4) ||
        !aligned(lse, 4))
        return FXP_ERR_ALIGN;
    if (!ws || ws_bytes < fxp_kv_attention_workspace_bytes(st->requests, st->tokens, q_heads, cache->heads, cache->dim)) return FXP_ERR_WORKSPACE;
    if (!aligned(ws, 256)) return FXP_ERR_ALIGN;
    AttArgs a;
    a.c = *cache;
    a.first = st->first;
    a.lens = st->lens_after;
    a.table = st->block_table;
    a.requests = st->requests;
    a.blocks = st->blocks;
    a.tokens = st->tokens;
    a.q = q;
    a.q_token = q_token;
    a.q_head = q_head;
    a.out = out;
    a.out_token = out_token;
    a.out_head = out_head;
    a.lse = lse;
    a.window = static_cast<int>(window < (int64_t{1} << 30) ? window : (int64_t{1} << 30));
    a.tickets = static_cast<uint32_t*>(ws);
    a.part_o = reinterpret_cast<float*>(static_cast<char*>(ws) + FXP_KV_TICKET_BYTES);
    static_assert(FXP_KV_TICKET_BYTES == kAttGroups * sizeof(uint32_t), "a ticket for each workgroup");
    a.part_ml = reinterpret_cast<float4*>(a.part_o + static_cast<size_t>(kAttGroups) * 2 * kTile * cache->dim);
    a.group = static_cast<int>(q_heads / cache->heads);
    a.group_inverse = static_cast<uint32_t>(((uint64_t{1} << 32) + a.group - 1) / a.group);
    a.vec_q = aligned(q, 16) && q_token * size % 16 == 0 && q_head * size % 16 == 0;
    a.vec_out = aligned(out, 4 * size) && out_token % 4 == 0 && out_head % 4 == 0;
    a.scale_log2 = scale * 1.44269504088896f;
    constexpr int64_t kTurn = 4 * 64 * kAttWaves;
    const int64_t rows = std::min<int64_t>(std::max<int64_t>((st->tokens * a.group + st->requests - 1) / st->requests, a.group), kTile);
    a.join_turns = static_cast<float>((rows * cache->dim + kTurn - 1) / kTurn);
    hipStream_t s = static_cast<hipStream_t>(stream);
    auto go = [&](auto type_c, auto db_c) -> int {
        constexpr int TYPE = decltype(type_c)::value, DB = decltype(db_c)::value;
        // Many rows a request, and enough blocks of 64 for every CU: the kernel that shares pages among rows (16 heads, 4 of the cache,
        // 128 elements, one request: 1024 rows of 0 earlier tokens 12 us against 13 of the other kernel, 2048 18 / 24, 8192 68 / 219).  It has no
        // way to split a context: with half as many blocks as CUs, 1024 rows behind 4000 tokens take 92 us against 53.  Requests of up to two
        // tiles stay with the other kernel (32 rows: 24 us against 30; 35 rows, three tiles: 36 / 28), and so do, found on the device, those
        // too long for their number of rows (longest_walk).  One request whose table holds few pages needs the one launch only: its walk is short
        // whatever its rows are.
        const int64_t blocks = (st->tokens * a.group + (kBlock - 1) * st->requests) / kBlock * cache->heads;
        const bool many = st->tokens * a.group > kFewRows * st->requests && blocks >= kCus && blocks < int64_t{1} << 24;
        // units of the line, which are counted in 32 bits
        auto fit = [&](int64_t tiles) { return tiles * (st->blocks + kTileCost) < int64_t{1} << 31; };
        const int64_t tiles = (st->tokens * a.group + (kTile - 1) * st->requests) / kTile * cache->heads;
        const int64_t short_tiles = std::min(tiles, 2 * st->requests * cache->heads);
        const bool both = many && (st->requests > 1 || (st->blocks > kShortTable && fit(short_tiles)));
        if ((!many && !fit(tiles)) || (both && !fit(short_tiles))) return FXP_ERR_DIMS;
        // walks that are longer than a CU's share have fewer blocks together than there are CUs
        a.balance = both && fit(short_tiles + std::min<int64_t>(tiles, kCus * kRowWaves));
        a.rows_from = !many ? std::numeric_limits<int>::max() : both ? kFewRows : 0;
        a.longest = std::numeric_limits<int>::max();
        a.walk = a.window / FXP_KV_PAGE + (kBlock / a.group + 1) / FXP_KV_PAGE + 3;
        if (many)
            hipLaunchKernelGGL((k_kv_attend_rows<TYPE, DB>), dim3(static_cast<unsigned>(blocks)), dim3(64 * kRowWaves), 0, s, a);
        if (!many || both) hipLaunchKernelGGL((k_kv_attend<TYPE, DB>), dim3(kAttGroupsOf<DB>), dim3(64 * kAttWaves), 0, s, a);
        return launch_status();
    };
    auto of_type = [&](auto type_c) {
        const int64_t db = (cache->dim + 63) / 64;
        if (db == 1) return go(type_c, std::integral_constant<int, 1>{});
        if (db == 2) return go(type_c, std::integral_constant<int, 2>{});
        if (db == 3) return go(type_c, std::integral_constant<int, 3>{});
        return go(type_c, std::integral_constant<int, 4>{});
    };
    if (type == FXP_F32) return of_type(std::integral_constant<int, FXP_F32>{});
    if (type == FXP_BF16) return of_type(std::integral_constant<int, FXP_BF16>{});
    return of_type(std::integral_constant<int, FXP_F16>{});
}
