// Rotary positions: pairs of elements of a head turned by the position of their token times a frequency of their own, and the gradient of that (the
// opposite angles).  Angles: fxp_rotary_device.h.
//
// Bound by memory: every element is read and written once (16384 tokens of 32 heads of 128 in bf16: 55 us, 4.9 TB/s read and written, the rate of a large copy; one token 2.3).
// A workgroup finds the cosines and sines of its tokens once, in LDS, for all of their heads (registers of the threads that use them would need one of each for every pair of
// every head), while its first loads are in flight.
#include <algorithm>

#include "fxp_rotary_device.h"

namespace fxp {

constexpr int kRotThreads = 256, kRotAhead = 4, kRotTable = 2048, kRotTokens = 64;

struct RotaryArgs {
    const void* x;
    void* y;
    const int32_t* positions;
    const uint64_t* turns;
    int64_t x_batch, x_token, x_head, y_batch, y_token, y_head, p_batch;
    int64_t tokens;
    int heads, pairs, rot, dim, pieces;         // pieces: items of a head
    int tb, hb, token_blocks;                   // tokens and heads of a workgroup
    uint32_t by_pieces, by_inner, by_pairs;     // ceil(2^32 / n) of the divisors
    int heads_inside;                           // heads of a token lie nearer to each other than tokens of a head
    float amplitude, side;                      // side: 1, or -1 for the gradient
    int zero;                                   // rows at negative positions become zeros
};

__device__ inline int divide(int n, int d, uint32_t inverse) { return d == 1 ? n : static_cast<int>(__umulhi(static_cast<uint32_t>(n), inverse)); }

// An item is P pairs: two runs of P elements, `half` apart or beside each other (NEAR); behind the rotated elements 2 P others.
template <int TYPE, int P, bool NEAR>
__global__ __launch_bounds__(kRotThreads) void k_rotary(RotaryArgs a) {
    __shared__ float2 table[kRotTable];
    const int block = static_cast<int>(blockIdx.x) % a.token_blocks, batch = static_cast<int>(blockIdx.x) / a.token_blocks;
    const int64_t t0 = int64_t{block} * a.tb;
    const int h0 = static_cast<int>(blockIdx.y) * a.hb;
    const int nt = static_cast<int>(min(int64_t{a.tb}, a.tokens - t0)), nh = min(a.hb, a.heads - h0);
    const int items = nt * nh * a.pieces, rotated = a.pairs / P, inner = a.heads_inside ? a.hb : a.tb;
    const int64_t x0 = batch * a.x_batch + t0 * a.x_token + h0 * a.x_head, y0 = batch * a.y_batch + t0 * a.y_token + h0 * a.y_head;

    struct Item {
        int token, first, second, pair;         // elements of the two runs in their head; second < 0: none; pair < 0: not rotated
        int64_t x, y;
    };
    // rows are counted in whole blocks of hb heads or tb tokens, so that the divisor is the launch's; rows past the tensor's are skipped
    auto item_of = [&](int i, Item& it) {
        const int row = divide(i, a.pieces, a.by_pieces), piece = i - row * a.pieces;
        const int outer = divide(row, inner, a.by_inner), in = row - outer * inner;
        const int head = a.heads_inside ? in : outer;
        it.token = a.heads_inside ? outer : in;
        it.x = x0 + it.token * a.x_token + head * a.x_head;
        it.y = y0 + it.token * a.y_token + head * a.y_head;
        if (piece < rotated) {
            it.pair = piece * P;
            it.first = NEAR ? 2 * it.pair : it.pair;
            it.second = NEAR ? it.first + P : it.first + a.pairs;
        } else {
            it.pair = -1;
            it.first = a.rot + (piece - rotated) * 2 * P;
            it.second = it.first + P < a.dim ? it.first + P : -1;
        }
        return it.token < nt && head < nh;
    };
    const int all = (a.heads_inside ? nt * a.hb : nh * a.tb) * a.pieces;
    if (items == 0) return;
    bool ready = false;
    uint64_t without = 0;                       // tokens at negative positions
    static_assert(kRotTokens <= 64, "a lane for each token");
    for (int base = 0; base < all; base += kRotThreads * kRotAhead) {
        float u[kRotAhead][P], w[kRotAhead][P];
        Item it[kRotAhead];
        bool there[kRotAhead];
#pragma unroll
        for (int n = 0; n < kRotAhead; ++n) {
            const int i = base + n * kRotThreads + static_cast<int>(threadIdx.x);
            there[n] = i < all && item_of(i, it[n]);
            if (there[n]) {
                load_elems<TYPE, P>(a.x, it[n].x + it[n].first, true, u[n]);
                if (it[n].second >= 0) load_elems<TYPE, P>(a.x, it[n].x + it[n].second, true, w[n]);
            }
        }
        if (!ready) {
            for (int e = threadIdx.x; e < nt * a.pairs; e += kRotThreads) {
                const int token = divide(e, a.pairs, a.by_pairs);
                float c, s;
                cos_sin(angle_of(a.turns[e - token * a.pairs], a.positions[batch * a.p_batch + t0 + token]), c, s);
                table[e] = make_float2(c * a.amplitude, s * a.amplitude * a.side);
            }
            const int lane = threadIdx.x & 63;
            without = __ballot(lane < nt && a.positions[batch * a.p_batch + t0 + lane] < 0);
            __syncthreads();
            ready = true;
        }
#pragma unroll
        for (int n = 0; n < kRotAhead; ++n) {
            if (!there[n] || (without >> it[n].token & 1)) continue;
            if (it[n].pair >= 0) {
                const float2* const t = table + it[n].token * a.pairs + it[n].pair;
                if constexpr (NEAR) {
#pragma unroll
                    for (int j = 0; j < P; ++j) {
                        // pair j is elements 2 j and 2 j + 1 of the two runs put together
                        float& p = 2 * j < P ? u[n][(2 * j) % P] : w[n][(2 * j) % P];
                        float& q = 2 * j + 1 < P ? u[n][(2 * j + 1) % P] : w[n][(2 * j + 1) % P];
                        turn_pair(p, q, t[j].x, t[j].y);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < P; ++j) turn_pair(u[n][j], w[n][j], t[j].x, t[j].y);
                }
            }
            store_elems<TYPE, P>(a.y, it[n].y + it[n].first, u[n]);
            if (it[n].second >= 0) store_elems<TYPE, P>(a.y, it[n].y + it[n].second, w[n]);
        }
    }
    if (!a.zero) return;
    // Rows without a token, on their own: in the loop above their stores would cost the registers of the others (16384 tokens of 32 x 128 in bf16, none of them
    // such a row: 54.6 us so and 54.4 without them; 55.3 where u and w are cleared there, 57.7 with stores of zeros there).
    for (; without; without &= without - 1) {
        const int t = __builtin_ctzll(without);
        for (int e = threadIdx.x; e < a.hb * a.pieces; e += kRotThreads) {
            const int head = divide(e, a.pieces, a.by_pieces);
            const float none[P] = {};
            Item it;
            if (!item_of((a.heads_inside ? t * a.hb + head : head * a.tb + t) * a.pieces + e - head * a.pieces, it)) continue;
            store_elems<TYPE, P>(a.y, it.y + it.first, none);
            if (it.second >= 0) store_elems<TYPE, P>(a.y, it.y + it.second, none);
        }
    }
}

static uint32_t inverse_of(int n) { return n <= 1 ? 0u : static_cast<uint32_t>(((uint64_t{1} << 32) + n - 1) / n); }

}  // namespace fxp

extern "C" int fxp_rotary(const fxp_rotation* rotation, int backward, int type, int64_t batch, int64_t tokens, int64_t heads, int64_t dim,
                          const void* x, int64_t x_batch, int64_t x_token, int64_t x_head, const int32_t* positions, int64_t p_batch, void* y,
                          int64_t y_batch, int64_t y_token, int64_t y_head, void* stream) {
    using namespace fxp;
    const int rc = check_rotation(rotation, dim);
    if (rc) return rc;
    if (!known_type(type)) return FXP_ERR_TYPE;
    const int zero = backward & FXP_ROTARY_ZERO;
    backward &= ~FXP_ROTARY_ZERO;
    constexpr int64_t kMost = int64_t{1} << 31;
    if (batch < 0 || tokens < 0 || heads < 0 || batch >= kMost || tokens >= kMost || heads > 65535 || dim > 65536 || !strides_ok(x_token, x_head) ||
        !strides_ok(y_token, y_head) || x_batch < 0 || y_batch < 0 || p_batch < 0 || x_batch >= (int64_t{1} << 40) || y_batch >= (int64_t{1} << 40) ||
        p_batch >= (int64_t{1} << 40))
        return FXP_ERR_DIMS;
    if (batch == 0 || tokens == 0 || heads == 0) return FXP_OK;
    if (!x || !y || !positions) return FXP_ERR_NULL;
    // single tokens of many sequences are the tokens of one
    if (tokens == 1 && (batch == 1 || p_batch == 1)) {
        tokens = batch;
        x_token = x_batch;
        y_token = y_batch;
        batch = 1;
    }
    // steps that are never taken
    if (batch == 1) x_batch = y_batch = p_batch = 0;
    if (tokens == 1) x_token = y_token = 0;
    if (heads == 1) x_head = y_head = 0;
    const int size = elem_size(type);
    if (!aligned(x, size) || !aligned(y, size) || !aligned(positions, 4)) return FXP_ERR_ALIGN;

    RotaryArgs a{};
    a.x = x;
    a.y = y;
    a.positions = positions;
    a.turns = rotation->turns;
    a.x_batch = x_batch; a.x_token = x_token; a.x_head = x_head;
    a.y_batch = y_batch; a.y_token = y_token; a.y_head = y_head;
    a.p_batch = p_batch;
    a.tokens = tokens;
    a.heads = static_cast<int>(heads);
    a.rot = static_cast<int>(rotation->rot);
    a.pairs = a.rot / 2;
    a.dim = static_cast<int>(dim);
    const bool in_place = x == y && x_batch == y_batch && x_token == y_token && x_head == y_head;
    const int rest = in_place && !zero ? 0 : a.dim - a.rot;
    // the widest accesses that every address allows
    int P = 16 / size;
    auto fits = [&](int p) {
        for (int64_t s : {x_batch, x_token, x_head, y_batch, y_token, y_head, int64_t{a.pairs}, int64_t{a.rot}, int64_t{rest}})
            if (s % p) return false;
        return aligned(x, static_cast<size_t>(p * size)) && aligned(y, static_cast<size_t>(p * size));
    };
    while (P > 1 && !fits(P)) P /= 2;
    a.pieces = a.pairs / P + (rest + 2 * P - 1) / (2 * P);
    a.heads_inside = x_head < x_token || tokens == 1;
    // About 1024 items a workgroup, four a thread, so that it finds its cosines once for many heads; fewer where that would leave CUs idle.
    const int64_t total = batch * tokens * heads * a.pieces;
    const int target = static_cast<int>(std::min<int64_t>(kRotThreads * kRotAhead, std::max<int64_t>(kRotThreads, total / 1024)));
    a.hb = static_cast<int>(std::min<int64_t>(heads, std::max(1, target / a.pieces)));
    a.tb = std::max(1, std::min({target / (a.hb * a.pieces), kRotTable / a.pairs, kRotTokens, static_cast<int>(std::min<int64_t>(tokens, kRotTokens))}));
    const int64_t blocks = (tokens + a.tb - 1) / a.tb;
    if (blocks * batch >= int64_t{1} << 24) return FXP_ERR_DIMS;           // 2^32 threads
    a.token_blocks = static_cast<int>(blocks);
    a.by_pieces = inverse_of(a.pieces);
    a.by_inner = inverse_of(a.heads_inside ? a.hb : a.tb);
    a.by_pairs = inverse_of(a.pairs);
    a.amplitude = static_cast<float>(rotation->amplitude);
    a.side = backward ? -1.0f : 1.0f;
    a.zero = zero;
    const dim3 grid(static_cast<unsigned>(blocks * batch), static_cast<unsigned>((heads + a.hb - 1) / a.hb));
    hipStream_t s = static_cast<hipStream_t>(stream);
    auto go = [&](auto type_c, auto p_c) {
        constexpr int TYPE = decltype(type_c)::value, PP = decltype(p_c)::value;
        if (rotation->interleaved) hipLaunchKernelGGL((k_rotary<TYPE, PP, true>), grid, dim3(kRotThreads), 0, s, a);
        else hipLaunchKernelGGL((k_rotary<TYPE, PP, false>), grid, dim3(kRotThreads), 0, s, a);
    };
    auto by_width = [&](auto type_c) {
        if constexpr (decltype(type_c)::value != FXP_F32)
            if (P == 8) return go(type_c, std::integral_constant<int, 8>{});
        if (P == 4) return go(type_c, std::integral_constant<int, 4>{});
        if (P == 2) return go(type_c, std::integral_constant<int, 2>{});
        go(type_c, std::integral_constant<int, 1>{});
    };
    if (type == FXP_F32) by_width(std::integral_constant<int, FXP_F32>{});
    else if (type == FXP_BF16) by_width(std::integral_constant<int, FXP_BF16>{});
    else by_width(std::integral_constant<int, FXP_F16>{});
    return launch_status();
}
