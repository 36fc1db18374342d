// A paged cache of mapped keys and values: the tables of a step, the writer, the inverse mapping.
//
// Tables.  Request b with l tokens that receives n more needs ceil((l + n) / 64) - ceil(l / 64) pages; an exclusive sum
// over the requests gives each its first new token, its place in the stack of free pages and its first run (the new tokens
// that share a page).  One launch: every workgroup sums over all requests (4 KB per thousand of them, out of the L2) and
// fills 64 or 256 runs of its own, so nothing is exchanged between workgroups.
//
// Writer.  q = floor(|x| 2^(125 + bits - e) + 1/2) with e the largest exponent of the block.  A workgroup has one run of one
// head, keys or values; a thread has blocks of 4 tokens x 4 elements, which is one dword each way for keys (a token's four
// elements) and, transposed in registers, for values (an element's four tokens).
#include "fxp_serve_device.h"

namespace fxp {

constexpr int kTabThreads = 1024;
// Runs a workgroup fills: up to 256 runs one workgroup, which may then write lengths in place as it goes (256 requests: 4.1 us), and 64 beyond
// (999 requests, 100386 tokens in 2700 runs: 6.7 us; 128 a workgroup 7.4, 256 8.7).
constexpr int kTabOne = 256, kTabMany = 64;

// Sums over requests.  What requests ask for may pass 32 bits together (a thousand that ask for millions each): sums stay at 2^32 - 1 then, which
// no count of tokens, pages or runs reaches, so that nobody behind such a sum is taken to fit.
struct Three {
    uint32_t tokens, need, runs;
};
__device__ inline uint32_t add_up(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }
__device__ inline Three add3(const Three& a, const Three& b) {
    return {add_up(a.tokens, b.tokens), add_up(a.need, b.need), add_up(a.runs, b.runs)};
}
// a place that is written out: the largest int32 stands for all beyond
__device__ inline int as_int(uint32_t x) { return static_cast<int>(min(x, 0x7fffffffu)); }

// Exclusive sums over the workgroup's threads; `total` receives the sum of all.  (Where the inclusive sum is 2^32 - 1, at least that
// less a thread's own, which is below 2^31, is before the thread.)
__device__ inline Three block_scan3(const Three& v, Three* lds, Three& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Three s = {wave_scan_up(v.tokens), wave_scan_up(v.need), wave_scan_up(v.runs)};
    if (lane == 63) lds[wave] = s;
    __syncthreads();
    Three before = {0, 0, 0};
    total = {0, 0, 0};
#pragma unroll
    for (int w = 0; w < kTabThreads / 64; ++w) {
        if (w == wave) before = total;
        total = add3(total, lds[w]);
    }
    __syncthreads();
    return add3(before, {s.tokens - v.tokens, s.need - v.need, s.runs - v.runs});
}

struct Request {
    int len, had, after, served;
    uint32_t first, need0, run0;
    int row;
};

// what request b asks for; lengths that no device program should hold (negative, past the table) only have to stay harmless:
// every index that comes of them is compared with its array before it is used
__device__ inline Three asks(const fxp_kv_step& st, const int32_t* n_new, int64_t b, Request& r, bool& fits) {
    Three v = {0, 0, 0};
    fits = false;
    r.len = r.after = r.had = 0;
    if (b >= st.requests) return v;
    const int64_t len = max(st.lens[b], 0), asked = max(n_new[b], 0), n = min(asked, st.tokens), after = len + n;
    fits = asked == n && after <= st.blocks * FXP_KV_PAGE;
    r.len = static_cast<int>(len);
    r.after = static_cast<int>(min(after, (int64_t{1} << 31) - 1));
    r.had = static_cast<int>((len + FXP_KV_PAGE - 1) / FXP_KV_PAGE);
    v.tokens = static_cast<uint32_t>(n);
    v.need = fits ? static_cast<uint32_t>((after + FXP_KV_PAGE - 1) / FXP_KV_PAGE - r.had) : 0u;
    v.runs = n ? static_cast<uint32_t>((after - 1) / FXP_KV_PAGE - len / FXP_KV_PAGE + 1) : 0u;
    return v;
}

// Whether a request finds room: in its row, in the stack and among the step's tokens; `x` is the sum of those before it.  Both sums only
// grow, so the requests that are served and take pages come before those that find too few.
__device__ inline bool has_room(const fxp_kv_step& st, bool fits, const Three& v, const Three& x, int n_free) {
    const Three upto = add3(x, v);
    return fits && (v.need == 0 || upto.need <= static_cast<uint32_t>(n_free)) && (v.tokens == 0 || upto.tokens <= st.tokens);
}

// lengths of all requests and the stack's height, for the workgroup that is last to have read them
__device__ inline void commit_lengths(const fxp_kv_step& st, const int32_t* n_new, Three* lds) {
    const int n_free = min(static_cast<int64_t>(max(st.n_free[0], 0)), st.pages);
    __shared__ int taken;
    if (threadIdx.x == 0) taken = 0;
    __syncthreads();
    Three carry = {0, 0, 0}, total;
    for (int64_t base = 0; base < st.requests; base += kTabThreads) {
        Request r;
        bool fits;
        const Three v = asks(st, n_new, base + threadIdx.x, r, fits);
        const Three x = add3(carry, block_scan3(v, lds, total));
        const bool served = has_room(st, fits, v, x, n_free);
        if (base + threadIdx.x < st.requests) st.lens_after[base + threadIdx.x] = served ? r.after : st.lens[base + threadIdx.x];
        if (served && v.need) atomicMax(&taken, static_cast<int>(x.need + v.need));
        carry = add3(carry, total);
    }
    __syncthreads();
    if (threadIdx.x == 0) st.n_free_after[0] = n_free - taken;
}

template <int RUNS>
__global__ __launch_bounds__(kTabThreads) void k_kv_tables(fxp_kv_step st, const int32_t* __restrict__ n_new, int64_t run_rows,
                                                           uint32_t* ticket) {
    __shared__ Three lds[kTabThreads / 64];
    __shared__ Request req[RUNS];
    __shared__ int mark[RUNS];          // position of the request that a run belongs to, at the request's first run here
    __shared__ int64_t slot0[RUNS];
    __shared__ int4 span[RUNS];         // first token, count, position of the first token
    __shared__ int long_runs, last, taken;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t r0 = blockIdx.x * RUNS;
    const int n_free = min(static_cast<int64_t>(max(st.n_free[0], 0)), st.pages);
    if (tid < RUNS) mark[tid] = -1;
    if (tid == 0) long_runs = taken = 0;
    // A single workgroup has read what it replaces, and with outputs of their own nobody reads what is written: lengths and height are
    // written along the way.  Otherwise the last workgroup to arrive writes them in the end.
    const bool along = !ticket || gridDim.x == 1;
    __syncthreads();

    Three carry = {0, 0, 0}, total;
    for (int64_t base = 0; base < st.requests; base += kTabThreads) {
        const int64_t b = base + tid;
        Request r;
        bool fits;
        const Three v = asks(st, n_new, b, r, fits);
        const Three x = add3(carry, block_scan3(v, lds, total));
        r.served = has_room(st, fits, v, x, n_free);
        r.first = x.tokens;
        r.need0 = x.need;
        r.run0 = x.runs;
        r.row = static_cast<int>(b);
        // each thousand of requests has a workgroup that writes what belongs to a request
        if (b < st.requests && (base / kTabThreads) % gridDim.x == blockIdx.x) {
            st.first[b] = as_int(r.first);
            st.refused[b] = !r.served;
            if (along) st.lens_after[b] = r.served ? r.after : st.lens[b];
        }
        if (blockIdx.x == 0 && along && r.served && v.need) atomicMax(&taken, static_cast<int>(x.need + v.need));
        const uint32_t lo = max(x.runs, r0);
        if (v.runs > 0 && lo < add_up(x.runs, v.runs) && lo < r0 + RUNS) {
            req[lo - r0] = r;
            mark[lo - r0] = lo - r0;
        }
        carry = add3(carry, total);
    }
    if (blockIdx.x == 0 && tid == 0) st.first[st.requests] = as_int(carry.tokens);
    __syncthreads();
    if (blockIdx.x == 0 && tid == 0 && along) st.n_free_after[0] = n_free - taken;

    // the request of each run: the nearest mark at or before it
    int owner = -1;
    if (tid < RUNS) {
        owner = mark[tid];
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int t = __shfl_up(owner, d);
            if (lane >= d) owner = max(owner, t);
        }
        if (lane == 63) mark[tid] = owner;                  // the last of each wave: read below by the waves after it
    }
    __syncthreads();
    if (tid < RUNS) {
        for (int w = 0; w < wave; ++w) owner = max(owner, mark[64 * w + 63]);
        const uint32_t run = r0 + tid;
        int4 s = make_int4(0, 0, 0, 0);
        if (run < run_rows) {
            int4 out = make_int4(0, 0, -1, 0);
            if (run < carry.runs && owner >= 0) {
                const Request r = req[owner];
                const int j = static_cast<int>(run - r.run0), block = r.len / FXP_KV_PAGE + j, off = j ? 0 : r.len % FXP_KV_PAGE;
                const int t0 = as_int(add_up(r.first, j ? j * FXP_KV_PAGE - r.len % FXP_KV_PAGE : 0));
                const int count = min(FXP_KV_PAGE - off, r.after - (block * FXP_KV_PAGE + off));
                int page = -1;
                if (r.served && block < st.blocks) {
                    int32_t* entry = st.block_table + int64_t{r.row} * st.blocks + block;
                    if (block >= r.had) {
                        const int at = n_free - 1 - (static_cast<int>(r.need0) + block - r.had);
                        page = at >= 0 && at < n_free ? st.free_pages[at] : -1;
                        *entry = page;
                    } else {
                        page = *entry;
                    }
                }
                page = max(page, -1);
                const int64_t slot = page < 0 ? -1 : int64_t{page} * FXP_KV_PAGE + off;
                const int position = block * FXP_KV_PAGE + off;
                out = make_int4(t0, count, page, off);
                s = make_int4(t0, count, position, 0);
                slot0[tid] = slot;
                if (t0 >= 0 && t0 < st.tokens) {            // a run's first token here: in a decode step there is no other
                    st.slots[t0] = slot;
                    st.positions[t0] = position;
                }
                if (count > 1) long_runs = 1;
            }
            reinterpret_cast<int4*>(st.runs)[run] = out;
        }
        span[tid] = s;
    }
    __syncthreads();
    if (long_runs)
        for (int i = wave; i < RUNS; i += kTabThreads / 64) {
            const int4 s = span[i];
            const int64_t t = int64_t{s.x} + lane;
            if (lane >= 1 && lane < s.y && t >= 0 && t < st.tokens) {
                st.slots[t] = slot0[i] < 0 ? -1 : slot0[i] + lane;
                st.positions[t] = s.z + lane;
            }
        }
    for (int64_t t = int64_t{carry.tokens} + int64_t{blockIdx.x} * kTabThreads + tid; t < st.tokens; t += int64_t{gridDim.x} * kTabThreads)
        st.slots[t] = st.positions[t] = -1;

    // The lengths and the stack's height may be updated in place: by the workgroup that is last to have read them.
    if (!along) {
        __syncthreads();
        if (tid == 0) {
            last = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
            if (last) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (last) commit_lengths(st, n_new, lds);
    }
}

// ---- writer ----

// four tokens x four elements of a [tokens, heads, dim] operand, rows before `from` and from `to` on zero
template <int TYPE>
__device__ inline void load_block(const void* x, int64_t at, int64_t token, int from, int to, bool vec, float (&v)[4][4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i >= from && i < to) {
            load_elems<TYPE, 4>(x, at + i * token, vec, v[i]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i][j] = 0.0f;
        }
    }
}

// The mapping of finite values under a scale in [25, 250].  Two bytes have 11 significant bits at most, so |x| in units plus 1/2 is exact and is cut
// by the conversion; an fp32 value goes through its 24-bit mantissa as map_nearest has it (in units of its own, 0.5 - 2^-25 plus 1/2 rounds to 1).
struct MapNearest {
    float to;               // units (of the mantissa, for fp32) per 1
    int cut, sat;
};
template <int TYPE>
__device__ inline int map_finite(float x, const MapNearest& c) {
    if constexpr (TYPE == FXP_F32) {
        const uint32_t m = static_cast<uint32_t>(fabsf(x) * c.to);
        const int q = min(static_cast<int>((m + (1u << (c.cut - 1))) >> c.cut), c.sat), sign = static_cast<int>(__float_as_uint(x)) >> 31;
        return (q ^ sign) - sign;
    } else {
        const float y = x * c.to;
        return min(max(static_cast<int>(y + copysignf(0.5f, y)), -c.sat), c.sat);
    }
}

// Where a run's quads lie: the first, their number, the place behind the last token, quads of elements, ceil(2^32 / that).
struct Quads {
    int first, count, end, nd;
    uint32_t inverse;
    bool by_four;           // four quads of tokens beside each other in neighbouring threads: their values make 16 bytes
    __device__ void at(int i, int& tq, int& d) const {
        const int j = by_four ? i >> 2 : i, q = static_cast<int>(__umulhi(static_cast<uint32_t>(j), inverse));
        d = (j - q * nd) * 4;
        tq = first + (by_four ? 4 * q + (i & 3) : q);
    }
};
__device__ inline Quads quads_of(const Run& run, int dim, uint32_t inverse, bool values) {
    const int first = run.offset / 4, end = run.offset + run.count, count = (end + 3) / 4 - first;
    return {first, count, end, dim / 4, inverse, values && count % 4 == 0};
}
// dword of a page that holds element d + j of a quad of tokens (values), or elements d .. d + 3 of token j of it (keys)
__device__ inline int dword_of(bool values, int tq, int d, int j, int dim) {
    return values ? (tq >> 2) * (dim * 4) + (d + j) * 4 + (tq & 3) : ((4 * tq + j) * dim + d) / 4;
}

// What bounds it: a step of single tokens the way of one token (run, then values, scale and old bytes together, then stores), a prompt
// its reads and writes.
template <int TYPE, int THREADS>
__global__ __launch_bounds__(THREADS) void k_kv_append(fxp_kv_cache c, const void* __restrict__ k, int64_t k_token, int64_t k_head,
                                                       const void* __restrict__ v, int64_t v_token, int64_t v_head, int64_t tokens,
                                                       const int4* __restrict__ runs, int vec_k, int vec_v, uint32_t inverse) {
    __shared__ uint32_t lds[THREADS / 64];
    const int4 rr = runs[blockIdx.x];
    const Run run = {rr.x, rr.y, rr.z, rr.w};
    if (!run_ok(run, tokens, c.pages)) return;
    const bool values = blockIdx.z != 0;
    const int head = blockIdx.y, dim = static_cast<int>(c.dim);
    const Quads quads = quads_of(run, dim, inverse, values);
    const int work = quads.count * quads.nd, nd = quads.nd;
    const void* x = values ? v : k;
    const int64_t token = values ? v_token : k_token;
    const bool vec = values ? vec_v : vec_k;
    const int64_t row0 = int64_t{run.first} * token + head * (values ? v_head : k_head);
    const int64_t block = int64_t{run.page} * c.heads + head;
    int32_t* const scale = (values ? c.ev : c.ek) + block;
    uint32_t* const page = reinterpret_cast<uint32_t*>((values ? c.vq : c.kq) + block * (FXP_KV_PAGE * dim));

    const int e_old = run.offset ? min(max(*scale, 1), 255) : 1;
    constexpr int kKept = 2;             // blocks of 16 values that a thread keeps in registers; others are read again, out of the cache
    float kept[kKept][4][4];
    uint32_t old[kKept][4];              // of values: the dwords that the run's first tokens share with older ones
    uint32_t m = 0;
    auto fetch = [&](int i, float (&w)[4][4]) {
        int tq, d;
        quads.at(i, tq, d);
        const int place = 4 * tq;
        load_block<TYPE>(x, row0 + (int64_t{place} - run.offset) * token + d, token, max(run.offset - place, 0), min(quads.end - place, 4), vec, w);
    };
    auto fetch_old = [&](int i, uint32_t (&b)[4]) {
        int tq, d;
        quads.at(i, tq, d);
        if (values && 4 * tq < run.offset)
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = page[dword_of(true, tq, d, j, dim)];
    };
    auto largest = [&](const float (&w)[4][4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) m = max(m, __float_as_uint(w[i][j]) & 0x7fffffffu);
    };
#pragma unroll
    for (int n = 0; n < kKept; ++n)
        if (static_cast<int>(threadIdx.x) + n * THREADS < work) {
            fetch(threadIdx.x + n * THREADS, kept[n]);
            fetch_old(threadIdx.x + n * THREADS, old[n]);
        }
#pragma unroll
    for (int n = 0; n < kKept; ++n)
        if (static_cast<int>(threadIdx.x) + n * THREADS < work) largest(kept[n]);
    for (int i = threadIdx.x + kKept * THREADS; i < work; i += THREADS) {
        float w[4][4];
        fetch(i, w);
        largest(w);
    }
    m = THREADS == 64 ? wave_max(m) : block_max<THREADS / 64>(m, lds);
    const int e = max(e_old, min(max(static_cast<int>(m >> 23), 1), 255)), grown = e - e_old, cut = 25 - c.bits;
    if (threadIdx.x == 0) *scale = e;
    const bool plain = e >= 25 && e <= 250;
    const MapNearest how = {ldexpf(1.0f, TYPE == FXP_F32 ? 150 - e : 125 + c.bits - e), cut, (1 << (c.bits - 1)) - 1};

    auto write = [&](int i, const float (&w)[4][4], uint32_t (&was)[4]) {
        int tq, d;
        quads.at(i, tq, d);
        const int from = max(run.offset - 4 * tq, 0), to = min(quads.end - 4 * tq, 4);
        uint32_t o[4];
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            uint32_t b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = static_cast<uint32_t>(plain ? map_finite<TYPE>(w[a][j], how) : map_nearest(w[a][j], e, cut));
            o[a] = perm(perm(b[3], b[2], 0x0c0c0400u), perm(b[1], b[0], 0x0c0c0400u), 0x05040100u);
        }
        if (values) {
            uint32_t t[4];
            transpose4x4(o, t);
            const uint32_t keep = from ? (1u << (8 * from)) - 1u : 0u;       // bytes of the tokens before the run
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (from) t[j] = (t[j] & ~keep) | ((grown ? remap_nearest4(was[j], grown) : was[j]) & keep);
                page[dword_of(true, tq, d, j, dim)] = t[j];
            }
        } else {
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                uint32_t* const p = page + dword_of(false, tq, d, a, dim);
                if (a >= from && a < to) *p = o[a];
                else if (a < from && grown) *p = remap_nearest4(*p, grown);
            }
        }
    };
#pragma unroll
    for (int n = 0; n < kKept; ++n)
        if (static_cast<int>(threadIdx.x) + n * THREADS < work) write(threadIdx.x + n * THREADS, kept[n], old[n]);
    for (int i = threadIdx.x + kKept * THREADS; i < work; i += THREADS) {
        float w[4][4];
        uint32_t was[4];
        fetch(i, w);
        fetch_old(i, was);
        write(i, w, was);
    }
    // quads of old tokens alone
    if (run.offset && grown)
        for (int i = threadIdx.x; i < quads.first * nd; i += THREADS) {
            const int q = static_cast<int>(__umulhi(static_cast<uint32_t>(i), inverse));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t* const p = page + dword_of(values, q, (i - q * nd) * 4, j, dim);
                *p = remap_nearest4(*p, grown);
            }
        }
}

// ---- inverse mapping: a thread has blocks of 4 tokens x 4 elements ----
template <int TYPE>
__global__ __launch_bounds__(256) void k_kv_load(fxp_kv_cache c, void* __restrict__ k, void* __restrict__ v, int64_t tokens,
                                                 const int4* __restrict__ runs, uint32_t inverse) {
    const int4 rr = runs[blockIdx.x];
    const Run run = {rr.x, rr.y, rr.z, rr.w};
    if (!run_ok(run, tokens, c.pages)) return;
    const bool values = blockIdx.z != 0;
    const int head = blockIdx.y, dim = static_cast<int>(c.dim);
    const Quads quads = quads_of(run, dim, inverse, values);
    const int work = quads.count * quads.nd;
    const int64_t block = int64_t{run.page} * c.heads + head;
    const int unit = min(max((values ? c.ev : c.ek)[block], 1), 255) - 125 - c.bits;
    const bool plain = unit >= -126 && unit <= 120;                         // 2^unit and 127 of them are normal numbers
    const float one = ldexpf(1.0f, plain ? unit : 0);
    const uint32_t* const page = reinterpret_cast<const uint32_t*>((values ? c.vq : c.kq) + block * (FXP_KV_PAGE * dim));
    for (int i = threadIdx.x; i < work; i += 256) {
        int tq, d;
        quads.at(i, tq, d);
        uint32_t b[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = page[dword_of(values, tq, d, j, dim)];
        if (values) {
            uint32_t t[4];
            transpose4x4(b, t);
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = t[j];
        }
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            const int place = 4 * tq + a;
            if (place < run.offset || place >= quads.end) continue;
            float x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int q = static_cast<int8_t>(b[a] >> (8 * j));
                x[j] = plain ? static_cast<float>(q) * one : unmap_value(q, unit);
            }
            store4<TYPE>(values ? v : k, ((int64_t{run.first} + place - run.offset) * c.heads + head) * dim + d, true, x);
        }
    }
}

constexpr int64_t kMostRuns = (int64_t{1} << 24) - 1;      // 256 threads each, fewer than 2^32 in all

static uint32_t inverse_of(int64_t n) { return static_cast<uint32_t>(((uint64_t{1} << 32) + n - 1) / n); }        // n > 1

static bool multiple_of_4(const void* p, int64_t token, int64_t head, int type) {
    return aligned(p, 4 * elem_size(type)) && token % 4 == 0 && head % 4 == 0;
}

}  // namespace fxp

extern "C" int64_t fxp_kv_max_runs(int64_t requests, int64_t tokens) {
    if (requests < 0 || tokens < 0 || requests >= (int64_t{1} << 31) || tokens >= (int64_t{1} << 31)) return 0;
    // n tokens of one request touch at most (n + 126) / 64 pages, and at least one token each
    const int64_t most = (tokens + 2 * (FXP_KV_PAGE - 1) * requests) / FXP_KV_PAGE;
    return most < tokens ? most : tokens;
}

extern "C" int fxp_kv_tables(const fxp_kv_step* st, const int32_t* n_new, void* ws, size_t ws_bytes, void* stream) {
    if (!st) return FXP_ERR_NULL;
    constexpr int64_t kMost = int64_t{1} << 31;
    if (st->requests <= 0 || st->blocks <= 0 || st->tokens < 0 || st->pages <= 0 || st->requests >= kMost || st->tokens >= kMost ||
        st->pages >= kMost || st->blocks >= kMost / FXP_KV_PAGE)
        return FXP_ERR_DIMS;
    if (!n_new || !st->lens || !st->free_pages || !st->n_free || !st->block_table || !st->lens_after || !st->n_free_after || !st->first ||
        !st->refused || (st->tokens && (!st->slots || !st->positions || !st->runs)))
        return FXP_ERR_NULL;
    for (const void* p : {static_cast<const void*>(n_new), static_cast<const void*>(st->lens), static_cast<const void*>(st->free_pages),
                          static_cast<const void*>(st->n_free), static_cast<const void*>(st->block_table),
                          static_cast<const void*>(st->lens_after), static_cast<const void*>(st->n_free_after),
                          static_cast<const void*>(st->first), static_cast<const void*>(st->positions), static_cast<const void*>(st->refused)})
        if (!fxp::aligned(p, 4)) return FXP_ERR_ALIGN;
    if (!fxp::aligned(st->slots, 8) || !fxp::aligned(st->runs, 16)) return FXP_ERR_ALIGN;
    const bool in_place = st->lens_after == st->lens || st->n_free_after == st->n_free;
    if (in_place && (!ws || ws_bytes < 256)) return FXP_ERR_WORKSPACE;
    if (in_place && !fxp::aligned(ws, 4)) return FXP_ERR_ALIGN;
    const int64_t rows = fxp_kv_max_runs(st->requests, st->tokens);
    uint32_t* const ticket = in_place ? static_cast<uint32_t*>(ws) : nullptr;
    if (rows <= fxp::kTabOne)
        hipLaunchKernelGGL((fxp::k_kv_tables<fxp::kTabOne>), dim3(1), dim3(fxp::kTabThreads), 0, static_cast<hipStream_t>(stream), *st, n_new, rows,
                           ticket);
    else
        hipLaunchKernelGGL((fxp::k_kv_tables<fxp::kTabMany>), dim3(static_cast<unsigned>((rows + fxp::kTabMany - 1) / fxp::kTabMany)),
                           dim3(fxp::kTabThreads), 0, static_cast<hipStream_t>(stream), *st, n_new, rows, ticket);
    return fxp::launch_status();
}

extern "C" int fxp_kv_append(const fxp_kv_cache* cache, int type, const void* k, int64_t k_token, int64_t k_head, const void* v,
                             int64_t v_token, int64_t v_head, int64_t tokens, const int32_t* runs, int64_t n_runs, void* stream) {
    const int rc = fxp::check_cache(cache);
    if (rc) return rc;
    if (!fxp::known_type(type)) return FXP_ERR_TYPE;
    if (tokens < 0 || n_runs < 0 || tokens >= (int64_t{1} << 31) || n_runs > fxp::kMostRuns || !fxp::strides_ok(k_token, k_head) ||
        !fxp::strides_ok(v_token, v_head))
        return FXP_ERR_DIMS;
    if (tokens == 0 || n_runs == 0) return FXP_OK;
    if (!k || !v || !runs) return FXP_ERR_NULL;
    if (!fxp::aligned(k, fxp::elem_size(type)) || !fxp::aligned(v, fxp::elem_size(type)) || !fxp::aligned(runs, 16)) return FXP_ERR_ALIGN;
    const int vk = fxp::multiple_of_4(k, k_token, k_head, type), vv = fxp::multiple_of_4(v, v_token, v_head, type);
    const dim3 grid(static_cast<unsigned>(n_runs), static_cast<unsigned>(cache->heads), 2);
    const uint32_t inverse = fxp::inverse_of(cache->dim / 4);
    // One wave a run and head, or four: few tokens finish sooner without a barrier and with more runs on a CU, many want the threads (256 runs of
    // one token, 8 heads of 128: 7.5 us with one wave, 10.7 with four; of four tokens 8.5 / 11.5, 2 heads of 256 7.2 / 6.6; 80 runs of 64:
    // 29.8 / 11.6).
    const bool few = tokens <= 4 * n_runs;
    auto go = [&](auto type_c) {
        constexpr int TYPE = decltype(type_c)::value;
        if (few)
            hipLaunchKernelGGL((fxp::k_kv_append<TYPE, 64>), grid, dim3(64), 0, static_cast<hipStream_t>(stream), *cache, k, k_token, k_head, v,
                               v_token, v_head, tokens, reinterpret_cast<const int4*>(runs), vk, vv, inverse);
        else
            hipLaunchKernelGGL((fxp::k_kv_append<TYPE, 256>), grid, dim3(256), 0, static_cast<hipStream_t>(stream), *cache, k, k_token, k_head, v,
                               v_token, v_head, tokens, reinterpret_cast<const int4*>(runs), vk, vv, inverse);
    };
    if (type == FXP_F32) go(std::integral_constant<int, FXP_F32>{});
    else if (type == FXP_BF16) go(std::integral_constant<int, FXP_BF16>{});
    else go(std::integral_constant<int, FXP_F16>{});
    return fxp::launch_status();
}

extern "C" int fxp_kv_load(const fxp_kv_cache* cache, int type, void* k, void* v, int64_t tokens, const int32_t* runs, int64_t n_runs,
                           void* stream) {
    const int rc = fxp::check_cache(cache);
    if (rc) return rc;
    if (!fxp::known_type(type)) return FXP_ERR_TYPE;
    if (tokens < 0 || n_runs < 0 || tokens >= (int64_t{1} << 31) || n_runs > fxp::kMostRuns) return FXP_ERR_DIMS;
    if (tokens == 0 || n_runs == 0) return FXP_OK;
    if (!k || !v || !runs) return FXP_ERR_NULL;
    if (!fxp::aligned(k, 16) || !fxp::aligned(v, 16) || !fxp::aligned(runs, 16)) return FXP_ERR_ALIGN;
    const dim3 grid(static_cast<unsigned>(n_runs), static_cast<unsigned>(cache->heads), 2);
    auto go = [&](auto type_c) {
        hipLaunchKernelGGL((fxp::k_kv_load<decltype(type_c)::value>), grid, dim3(256), 0, static_cast<hipStream_t>(stream), *cache, k, v, tokens,
                           reinterpret_cast<const int4*>(runs), fxp::inverse_of(cache->dim / 4));
    };
    if (type == FXP_F32) go(std::integral_constant<int, FXP_F32>{});
    else if (type == FXP_BF16) go(std::integral_constant<int, FXP_BF16>{});
    else go(std::integral_constant<int, FXP_F16>{});
    return fxp::launch_status();
}
