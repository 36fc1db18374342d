// Attention over a paged cache of mapped keys and values, with int8 matrix products and the softmax in fp32 (Sec. 5).
//
// A tile is 16 rows (token, query head) of one request and one head of the cache; a unit of work is one page (64 tokens) of a tile.
// All units of a call stand in one line, request by request, tile by tile, head by head, page by page, and every workgroup takes an
// equal stretch of it: lengths differ by orders of magnitude and are known on the device alone.  The four waves of a
// workgroup take the pages of a stretch in turn.  Where a tile's pages fall into two stretches or more, each leaves
// (largest score, sum, output) of its part in the workspace and a second launch joins them.
//
// One page: S^T = K Q^T by v_mfma_i32_16x16x64_i8 with the key rows as they lie in memory as A operand (16 bytes a lane) and
// Q's digits as B; a lane then holds 16 scores of ONE row (column lane % 16), tokens 16 (lane / 16) .. + 15 - the
// rows of A are taken in the order that makes it so - which packed into bytes are exactly the B operand of O^T = V^T P^T, so the
// softmax's weights never leave their lane.
//
// Digits.  A row of Q is v * 2^u with |v| < 2^15 (2^23) and v = 256 d1 + d0 (65536 d2 + ...), d signed bytes; a page's weights
// likewise under their own largest one.  Rounding a row to 15 bits is off by at most 2^-16 of its largest element's binade
// - for bf16 and fp16 rows less than half a step of the type for elements within 2^-8 / 2^-5 of the largest - and weights
// relative to the page's own largest, so a long tail of small weights behind one large one keeps its sum.  fp32 has 23 bits.
#include "fxp_serve_device.h"

namespace fxp {

constexpr int kTile = 16;
constexpr int kAttWaves = 4;
constexpr int kAttThreads = 64 * kAttWaves;
constexpr int kAttGroups = 512;          // workgroups at most: two a CU

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
    float* part_o;          // [workgroup][2][16][dim]
    float2* part_ml;        // [workgroup][2][16]
    int group;              // query heads per head of the cache
    int vec_q, vec_out;
    float scale_log2;       // scale * log2(e)
    int64_t window;         // <= 0: none
};

// where a tile stands
struct Segment {
    int b, tile, head, rows, n, len, page0, pages, tok0;
    int64_t unit0;
};

struct Extent {
    int n, len, tiles, page0, pages, tok0;
};
__device__ inline Extent extent(const AttArgs& a, int64_t b) {
    Extent e;
    const int most = static_cast<int>(a.tokens);
    e.tok0 = min(max(a.first[b], 0), most);
    e.n = max(min(max(a.first[b + 1], 0), most) - e.tok0, 0);
    e.len = static_cast<int>(min(static_cast<int64_t>(max(a.lens[b], 0)), a.blocks * FXP_KV_PAGE));
    e.tiles = (e.n * a.group + kTile - 1) / kTile;
    const int64_t from = a.window > 0 ? max(int64_t{e.len} - e.n + 1 - a.window, int64_t{0}) : 0;
    e.page0 = static_cast<int>(from / FXP_KV_PAGE);
    e.pages = max((e.len + FXP_KV_PAGE - 1) / FXP_KV_PAGE - e.page0, 1);       // an empty request still has its zeros to write
    return e;
}

// sum over the workgroup, and the sum before the thread
template <int WAVES>
__device__ inline int64_t block_scan64(int64_t v, int64_t* lds, int64_t& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t s = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t t = __shfl_up(static_cast<long long>(s), d);
        if (lane >= d) s += t;
    }
    if (lane == 63) lds[wave] = s;
    __syncthreads();
    int64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w == wave) before = total;
        total += lds[w];
    }
    __syncthreads();
    return before + s - v;
}

// units of all requests; found[0..1] = (request, units before it) of the request that unit `at` belongs to
__device__ inline int64_t locate(const AttArgs& a, int64_t at, bool tiles_only, int64_t* lds, int64_t* found) {
    int64_t carry = 0, total;
    for (int64_t base = 0; base < a.requests; base += kAttThreads) {
        const int64_t b = base + threadIdx.x;
        int64_t v = 0;
        if (b < a.requests) {
            const Extent e = extent(a, b);
            v = tiles_only ? e.tiles : e.tiles * a.c.heads * e.pages;
        }
        const int64_t x = carry + block_scan64<kAttWaves>(v, lds, total);
        if (at >= x && at < x + v) {
            found[0] = b;
            found[1] = x;
        }
        carry += total;
    }
    __syncthreads();
    return carry;
}

__device__ inline int64_t units_per_group(int64_t units, unsigned groups) {
    const int64_t per = (units + groups - 1) / groups;
    return (max(per, int64_t{kAttWaves}) + kAttWaves - 1) / kAttWaves * kAttWaves;
}

__device__ inline float max_groups(float v) {              // over the four lanes that hold a row
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ inline float sum_groups(float v) {
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// sum of products of digits, as a float: acc = d1 * 256 + d0 fits 32 bits over 256 terms; a third digit is added in fp32
template <int ND, int N>
__device__ inline void dot_digits(const v4i (&a)[N], const v4i (&b)[N][ND], float (&out)[4]) {
    v4i acc = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < N; ++i) acc = mfma_i8(a[i], b[i][0], acc);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] <<= 8;
#pragma unroll
    for (int i = 0; i < N; ++i) acc = mfma_i8(a[i], b[i][1], acc);
    if constexpr (ND == 3) {
        v4i low = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < N; ++i) low = mfma_i8(a[i], b[i][2], low);
#pragma unroll
        for (int j = 0; j < 4; ++j) out[j] = fmaf(static_cast<float>(acc[j]), 256.0f, static_cast<float>(low[j]));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) out[j] = static_cast<float>(acc[j]);
    }
}

template <int TYPE, int DB>
__global__ __launch_bounds__(kAttThreads, DB <= 2 ? 2 : 1) void k_kv_attend(AttArgs a) {
    constexpr int ND = TYPE == FXP_F32 ? 3 : 2;
    constexpr int DMAX = 64 * DB, ROW = DMAX + 4;
    __shared__ int64_t scan[kAttWaves];
    __shared__ int64_t found[2];
    __shared__ float s_m[kAttWaves][kTile], s_l[kAttWaves][kTile];
    __shared__ float s_o[kAttWaves][kTile][ROW];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g = lane >> 4;
    const int dim = static_cast<int>(a.c.dim), heads = static_cast<int>(a.c.heads);
    if (threadIdx.x == 0) found[0] = -1;
    __syncthreads();
    // the stretch of this workgroup; the size of a stretch needs the sum first
    const int64_t units = locate(a, -1, false, scan, found);
    const int64_t per = units_per_group(units, gridDim.x);
    const int64_t u0 = per * blockIdx.x, u1 = min(u0 + per, units);
    if (u0 >= u1) return;
    locate(a, u0, false, scan, found);
    int64_t b = found[0], unit_b = found[1];
    Extent e = extent(a, b);
    int64_t u = u0;

    while (u < u1) {
        // the tile that unit u belongs to, and this workgroup's pages of it
        int64_t in_b = u - unit_b;
        while (in_b >= int64_t{e.tiles} * heads * e.pages) {
            unit_b += int64_t{e.tiles} * heads * e.pages;
            e = extent(a, ++b);
            in_b = u - unit_b;
        }
        const int seg = static_cast<int>(in_b / e.pages), p0 = static_cast<int>(in_b % e.pages);
        const int tile = seg / heads, head = seg % heads;
        const int p1 = static_cast<int>(min(int64_t{e.pages}, p0 + (u1 - u)));
        const bool whole = p0 == 0 && p1 == e.pages;
        const int slot = u == u0 ? 0 : 1;
        u += p1 - p0;

        // this lane's row
        const int r = tile * kTile + col, tok = r / a.group, qh = head * a.group + r % a.group;
        const bool row_ok = tok < e.n;
        const int place = e.len - e.n + tok;                           // negative: more rows than tokens; such a row sees nothing
        const int see_to = row_ok ? min(place, e.len - 1) : -1;
        const int64_t see_from = a.window > 0 ? int64_t{place} - a.window + 1 : 0;

        // Q's digits
        v4i qd[DB][ND];
        int qe;
        {
            float x[DB][16];
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < DB; ++i) {
                const int d = 64 * i + 16 * g;
                if (row_ok && d < dim) {
                    load_elems<TYPE, 16>(a.q, (int64_t{e.tok0} + tok) * a.q_token + qh * a.q_head + d, a.vec_q, x[i]);
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j) x[i][j] = 0.0f;
                }
#pragma unroll
                for (int j = 0; j < 16; ++j) m = max(m, __float_as_uint(x[i][j]) & 0x7fffffffu);
            }
            m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 16)));
            m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 32)));
            qe = unit_of<ND>(m);
#pragma unroll
            for (int i = 0; i < DB; ++i) {
                int v[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] = fixed_point<ND>(x[i][j], qe);
                digits16<ND>(v, qd[i]);
            }
        }

        float o[4 * DB][4];
        float m_run = -INFINITY, l_run = 0.0f;
#pragma unroll
        for (int i = 0; i < 4 * DB; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] = 0.0f;

        for (int p = p0 + wave; p < p1; p += kAttWaves) {
            const int block = e.page0 + p;
            const int page = block < a.blocks ? a.table[b * a.blocks + block] : -1;
            if (page < 0 || page >= a.c.pages) continue;
            const int64_t at = int64_t{page} * heads + head;
            const int8_t* kp = a.c.kq + at * (FXP_KV_PAGE * dim);
            const int8_t* vp = a.c.vq + at * (FXP_KV_PAGE * dim);
            const int ek = min(max(a.c.ek[at], 1), 255) - 125 - a.c.bits, ev = min(max(a.c.ev[at], 1), 255) - 125 - a.c.bits;
            v4i kf[4][DB], vf[4 * DB];
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < DB; ++i) {
                    const int token = 16 * (col >> 2) + 4 * t + (col & 3), d = 64 * i + 16 * g;
                    kf[t][i] = d < dim ? *reinterpret_cast<const v4i*>(kp + token * dim + d) : v4i{0, 0, 0, 0};
                }
#pragma unroll
            for (int i = 0; i < 4 * DB; ++i)
                if (16 * i < dim) vf[i] = *reinterpret_cast<const v4i*>(vp + (g * dim + 16 * i + col) * 16);
            // bounded so that no product of it and a sum of up to 2^15 terms (digits x 7 bits x dim) passes 2^127: no Inf - Inf below
            const float f = fminf(ldexpf(a.scale_log2, qe + ek), ND == 2 ? 0x1p97f : 0x1p89f);

            float s[16];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                float x[4];
                dot_digits<ND, DB>(kf[t], qd, x);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[4 * t + i] = x[i] * f;
            }
            const int j0 = block * FXP_KV_PAGE + 16 * g;
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (j0 + i > see_to || j0 + i < see_from) s[i] = -INFINITY;
            float m = s[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) m = fmaxf(m, s[i]);
            m = max_groups(m);
            const float top = m == -INFINITY ? 0.0f : m;
            float l = 0.0f;
            v4i pd[1][ND];
            int v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float w = exp2f(s[i] - top);
                l += w;
                v[i] = static_cast<int>(rintf(w * Digits<ND>::kMost));
            }
            digits16<ND>(v, pd[0]);
            l = sum_groups(l);
            const float m_new = fmaxf(m_run, m), ref = m_new == -INFINITY ? 0.0f : m_new;
            const float keep = exp2f(m_run - ref), gain = exp2f(m - ref);
            const float fv = ldexpf(gain * (1.0f / Digits<ND>::kMost), ev);
            l_run = l_run * keep + l * gain;
            m_run = m_new;
#pragma unroll
            for (int i = 0; i < 4 * DB; ++i) {
                if (16 * i >= dim) continue;
                float x[4];
                const v4i vfrag[1] = {vf[i]};
                dot_digits<ND, 1>(vfrag, pd, x);
#pragma unroll
                for (int j = 0; j < 4; ++j) o[i][j] = fmaf(x[j], fv, o[i][j] * keep);
            }
        }

        // the four waves' parts
        if (g == 0) {
            s_m[wave][col] = m_run;
            s_l[wave][col] = l_run;
        }
#pragma unroll
        for (int i = 0; i < 4 * DB; ++i)
            if (16 * i < dim) *reinterpret_cast<float4*>(&s_o[wave][col][16 * i + 4 * g]) = make_float4(o[i][0], o[i][1], o[i][2], o[i][3]);
        __syncthreads();
        const int rows = min(e.n * a.group - tile * kTile, kTile);
        for (int i = threadIdx.x; i < rows * (dim / 4); i += kAttThreads) {
            const int row = i / (dim / 4), d = i % (dim / 4) * 4;
            float m = s_m[0][row];
#pragma unroll
            for (int w = 1; w < kAttWaves; ++w) m = fmaxf(m, s_m[w][row]);
            const float ref = m == -INFINITY ? 0.0f : m;
            float l = 0.0f, x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < kAttWaves; ++w) {
                const float f = exp2f(s_m[w][row] - ref);
                const float4 y = *reinterpret_cast<const float4*>(&s_o[w][row][d]);
                l = fmaf(s_l[w][row], f, l);
                x[0] = fmaf(y.x, f, x[0]);
                x[1] = fmaf(y.y, f, x[1]);
                x[2] = fmaf(y.z, f, x[2]);
                x[3] = fmaf(y.w, f, x[3]);
            }
            const int rr = tile * kTile + row;
            const int64_t t = int64_t{e.tok0} + rr / a.group;
            const int h = head * a.group + rr % a.group;
            if (whole) {
                const float inv = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] *= inv;
                store4<TYPE>(a.out, t * a.out_token + h * a.out_head + d, a.vec_out, x);
                if (a.lse && d == 0) a.lse[t * (heads * a.group) + h] = l > 0.0f ? (m + log2f(l)) * 0.693147180559945f : -INFINITY;
            } else {
                const int64_t part = (int64_t{blockIdx.x} * 2 + slot) * kTile + row;
                *reinterpret_cast<float4*>(a.part_o + part * dim + d) = make_float4(x[0], x[1], x[2], x[3]);
                if (d == 0) a.part_ml[part] = make_float2(m, l);
            }
        }
        __syncthreads();
    }
}

// Joins the parts of a tile that fell into several stretches.  blockIdx.x = tile, blockIdx.y = head.
template <int TYPE>
__global__ __launch_bounds__(kAttThreads) void k_kv_attend_join(AttArgs a, unsigned groups) {
    __shared__ int64_t scan[kAttWaves];
    __shared__ int64_t found[2];
    const int dim = static_cast<int>(a.c.dim), heads = static_cast<int>(a.c.heads), head = blockIdx.y;
    if (threadIdx.x == 0) found[0] = -1;
    __syncthreads();
    locate(a, blockIdx.x, true, scan, found);
    const int64_t b = found[0], tile0 = found[1];
    if (b < 0) return;
    __syncthreads();
    // units before request b
    int64_t before = 0, units = 0, total;
    for (int64_t base = 0; base < a.requests; base += kAttThreads) {
        const int64_t i = base + threadIdx.x;
        int64_t v = 0;
        if (i < a.requests) {
            const Extent x = extent(a, i);
            v = x.tiles * a.c.heads * x.pages;
        }
        const int64_t x = units + block_scan64<kAttWaves>(v, scan, total);
        if (i == b) found[1] = x;
        units += total;
    }
    __syncthreads();
    before = found[1];
    const Extent e = extent(a, b);
    const int tile = static_cast<int>(blockIdx.x - tile0);
    const int64_t per = units_per_group(units, groups);
    const int64_t s0 = before + (int64_t{tile} * heads + head) * e.pages, s1 = s0 + e.pages;
    const int64_t w0 = s0 / per, w1 = (s1 - 1) / per;
    if (w0 == w1) return;
    const int rows = min(e.n * a.group - tile * kTile, kTile);
    for (int i = threadIdx.x; i < rows * (dim / 4); i += kAttThreads) {
        const int row = i / (dim / 4), d = i % (dim / 4) * 4;
        float m = -INFINITY;
        for (int64_t w = w0; w <= w1; ++w) m = fmaxf(m, a.part_ml[(w * 2 + (w * per < s0)) * kTile + row].x);
        const float ref = m == -INFINITY ? 0.0f : m;
        float l = 0.0f, x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int64_t w = w0; w <= w1; ++w) {
            const int64_t part = (w * 2 + (w * per < s0)) * kTile + row;
            const float2 ml = a.part_ml[part];
            const float f = exp2f(ml.x - ref);
            const float4 y = *reinterpret_cast<const float4*>(a.part_o + part * dim + d);
            l = fmaf(ml.y, f, l);
            x[0] = fmaf(y.x, f, x[0]);
            x[1] = fmaf(y.y, f, x[1]);
            x[2] = fmaf(y.z, f, x[2]);
            x[3] = fmaf(y.w, f, x[3]);
        }
        const int rr = tile * kTile + row;
        const int64_t t = int64_t{e.tok0} + rr / a.group;
        const int h = head * a.group + rr % a.group;
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] *= inv;
        store4<TYPE>(a.out, t * a.out_token + h * a.out_head + d, a.vec_out, x);
        if (a.lse && d == 0) a.lse[t * (heads * a.group) + h] = l > 0.0f ? (m + log2f(l)) * 0.693147180559945f : -INFINITY;
    }
}

static bool attention_sizes_ok(int64_t requests, int64_t tokens, int64_t q_heads, int64_t heads, int64_t dim) {
    constexpr int64_t kMost = int64_t{1} << 31;
    return requests > 0 && requests < kMost && tokens >= 0 && tokens < kMost && heads > 0 && heads <= 65535 && q_heads > 0 &&
           q_heads <= 65535 && q_heads % heads == 0 && dim > 0 && dim <= 256 && dim % 16 == 0 && tokens * q_heads < kMost;
}

// tiles of all requests, at most
static int64_t most_tiles(int64_t requests, int64_t tokens, int64_t group) { return (tokens * group + (kTile - 1) * requests) / kTile; }

}  // namespace fxp

extern "C" size_t fxp_kv_attention_workspace_bytes(int64_t requests, int64_t tokens, int64_t q_heads, int64_t heads, int64_t dim) {
    if (!fxp::attention_sizes_ok(requests, tokens, q_heads, heads, dim)) return 0;
    return static_cast<size_t>(fxp::kAttGroups) * 2 * fxp::kTile * (dim * sizeof(float) + sizeof(float2));
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
    a.part_o = static_cast<float*>(ws);
    a.part_ml = reinterpret_cast<float2*>(a.part_o + static_cast<size_t>(kAttGroups) * 2 * kTile * cache->dim);
    a.group = static_cast<int>(q_heads / cache->heads);
    a.vec_q = aligned(q, 16) && q_token * size % 16 == 0 && q_head * size % 16 == 0;
    a.vec_out = aligned(out, 4 * size) && out_token % 4 == 0 && out_head % 4 == 0;
    a.scale_log2 = scale * 1.44269504088896f;
    a.window = window;
    const int64_t tiles = most_tiles(st->requests, st->tokens, a.group);
    if (tiles >= int64_t{1} << 24) return FXP_ERR_DIMS;
    hipStream_t s = static_cast<hipStream_t>(stream);
    auto go = [&](auto type_c, auto db_c) {
        constexpr int TYPE = decltype(type_c)::value, DB = decltype(db_c)::value;
        hipLaunchKernelGGL((k_kv_attend<TYPE, DB>), dim3(kAttGroups), dim3(kAttThreads), 0, s, a);
        hipLaunchKernelGGL((k_kv_attend_join<TYPE>), dim3(static_cast<unsigned>(tiles), static_cast<unsigned>(cache->heads)), dim3(kAttThreads), 0,
                           s, a, static_cast<unsigned>(kAttGroups));
    };
    auto of_type = [&](auto type_c) {
        const int64_t db = (cache->dim + 63) / 64;
        if (db == 1) go(type_c, std::integral_constant<int, 1>{});
        else if (db == 2) go(type_c, std::integral_constant<int, 2>{});
        else if (db == 3) go(type_c, std::integral_constant<int, 3>{});
        else go(type_c, std::integral_constant<int, 4>{});
    };
    if (type == FXP_F32) of_type(std::integral_constant<int, FXP_F32>{});
    else if (type == FXP_BF16) of_type(std::integral_constant<int, FXP_BF16>{});
    else of_type(std::integral_constant<int, FXP_F16>{});
    return launch_status();
}
