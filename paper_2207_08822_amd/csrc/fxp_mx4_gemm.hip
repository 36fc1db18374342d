// Products of matrices in microscaled 4-bit floats: C[M,N] = A[M,K] * B[N,K]^T on v_mfma_scale_f32_32x32x64_f8f6f4 (16x16x128 for a few rows).
//
// A lane of the instruction holds one block of one row - 32 codes in four registers - and its scale byte, so blocks need no work of their own: a panel of 256 columns is
// four instructions along the contraction, whose scales are the four bytes of one register.  Sums are fp32.
#include <algorithm>

#include "fxp_gemm_device.h"
#include "fxp_mx4_device.h"

namespace fxp {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));

constexpr int kFp4 = 4;                 // both operands' format in the instruction

// 4-bit operands are the low half of the operand registers
__device__ inline v8i wide(v4i x) { return __builtin_shufflevector(x, x, 0, 1, 2, 3, -1, -1, -1, -1); }

template <int BYTE_A, int BYTE_B>
__device__ inline v16f mfma32(v4i a, v4i b, v16f c, int sa, int sb) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(a), wide(b), c, kFp4, kFp4, BYTE_A, sa, BYTE_B, sb);
}
template <int BYTE_A, int BYTE_B>
__device__ inline v4f mfma16(v4i a, v4i b, v4f c, int sa, int sb) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(a), wide(b), c, kFp4, kFp4, BYTE_A, sa, BYTE_B, sb);
}

// BYTES a lane from `at` of the `bytes` at a uniform address to LDS, lane after lane; zeros past the end
template <int BYTES>
__device__ inline void load_to_lds(const uint8_t* from, int bytes, int at, uint8_t* to) {
    static_assert(BYTES == 16 || BYTES == 4, "sizes of the load");
    const auto lds = (__attribute__((address_space(3))) void*)to;
    if constexpr (BYTES == 16) __builtin_amdgcn_raw_ptr_buffer_load_lds(records(from, bytes), lds, 16, at, 0, 0, 0);
    else __builtin_amdgcn_raw_ptr_buffer_load_lds(records(from, bytes), lds, 4, at, 0, 0, 0);
}
// memory operations are not moved across it by the compiler
__device__ inline void barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// a wave's stores to LDS are done, and seen by its other lanes
__device__ inline void wave_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// 16 bytes at any address
struct __attribute__((packed, aligned(1))) Sixteen {
    v4i v;
};

struct Mx4Operand {
    const uint8_t *data, *scales;
    int rows;
};
struct Mx4Product {
    Mx4Operand a, b;
    int M, N, panels, per_split;        // panels of a workgroup's part of the contraction
    void* c;
    int64_t ldc, split_stride;          // of partial sums, in elements: 0 where there is one part
    int tiles_m, tiles_n, group_m;
};

template <int TYPE>
__device__ inline void store_one(void* c, int64_t at, float v) {
    static_cast<typename Elem<TYPE>::T*>(c)[at] = static_cast<typename Elem<TYPE>::T>(v);
}

// ---- partial sums ----
//
// Added in order: rows of `cols` elements, the parts' without gaps, four elements a thread where rows begin on a multiple of four.  A launch of its own, or the last workgroups
// of the product that follows (a layer's weight gradient before its input gradient: 4.8 us as a launch, 0.4 so).
struct Mx4Sum {
    const float* parts;
    int count, rows, cols, vec;         // vec: 0, 1 where parts are read by four, 2 where the result is written so too
    int64_t stride;
    void* c;
    int64_t ldc;
    int tiles;                          // riding: workgroups before the first of these
};
inline unsigned sum_blocks(const Mx4Sum& r, int threads) {
    return r.count == 0 ? 0u : static_cast<unsigned>(r.rows) * static_cast<unsigned>((r.cols + 4 * threads - 1) / (4 * threads));
}
template <int TYPE, int THREADS>
__device__ inline void sum_parts(const Mx4Sum& r, int block) {
    const int in_row = (r.cols + 4 * THREADS - 1) / (4 * THREADS), row = block / in_row, i = (block - row * in_row) * 4 * THREADS + static_cast<int>(threadIdx.x) * 4;
    if (i >= r.cols) return;
    const int64_t from = static_cast<int64_t>(row) * r.cols + i, to = static_cast<int64_t>(row) * r.ldc + i;
    if (r.vec && i + 4 <= r.cols) {
        v4f s = {};
#pragma unroll 4
        for (int n = 0; n < r.count; ++n) s += *reinterpret_cast<const v4f*>(r.parts + n * r.stride + from);
        store4<TYPE>(r.c, to, r.vec > 1, {s[0], s[1], s[2], s[3]});
    } else {
        for (int j = 0; j < 4 && i + j < r.cols; ++j) {
            float s = 0.0f;
            for (int n = 0; n < r.count; ++n) s += r.parts[n * r.stride + from + j];
            store_one<TYPE>(r.c, to + j, s);
        }
    }
}
template <int TYPE>
__global__ __launch_bounds__(256) void k_mx4_sum(Mx4Sum r) {
    sum_parts<TYPE, 256>(r, static_cast<int>(blockIdx.x));
}

// ---- tiles ----
//
// BM x BN outputs a workgroup in waves of WM x WN, STAGES panels in LDS, loaded straight from memory; rows past the operand's last read as zeros (the descriptor's
// bound).  16-byte pieces of a row of 128 bytes are exchanged by the row, so that a fragment's reads spread over all banks.
//
// Bound by the matrix cores and what they wait for: 8192^3 260 us, 4.2 PFLOP/s, the matrix cores busy 54 % of the time (of 197 us on zeros 109 are the instructions, 43 the
// starts and ends of four rounds of tiles, 30 loads); few panels by their outputs (12608 x 768 x 2304 in fp32 32 us, 3.6 TB/s written).
//
// A wave holds the fragments of two quarters of a panel: those of the next quarter are read while one is multiplied, across the barrier too, which stands before a
// panel's last quarter.  Behind it the slot of this panel is free: the next one's loads into it are spread over the multiplications of that quarter and of the first of the
// next panel.  (2048^3 to bf16 8.5 us; with every quarter read and then multiplied and outputs stored as they lie 12.1.)
//
// Outputs of two bytes: the operands change places, so that a lane has four neighbouring columns, and the wave's tile goes through LDS to leave in 16-byte pieces of whole
// rows, wherever these begin (1263 x 1016 x 7053 with its input's mapping: single elements 43 us, so 18).  fp32 leaves directly, 128 bytes in a row of C a store.
template <int BM, int BN, int WM, int WN, int STAGES, int TYPE>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64) void k_mx4_tiles(Mx4Product p, Mx4Sum rider) {
    if (rider.count != 0 && static_cast<int>(blockIdx.x) >= rider.tiles) {
        sum_parts<TYPE, (BM / WM) * (BN / WN) * 64>(rider, static_cast<int>(blockIdx.x) - rider.tiles);
        return;
    }
    constexpr int NW = (BM / WM) * (BN / WN), FM = WM / 32, FN = WN / 32;
    constexpr int kCodesA = BM * kMxRowBytes, kCodes = (BM + BN) * kMxRowBytes, kStage = kCodes + (BM + BN) * kMxRowScales;
    constexpr int LA = BM / 8 / NW, LB = BN / 8 / NW, LS = (BM + BN) / 32 / NW, kLoads = LA + LB + LS;       // loads of a wave a panel
    constexpr bool kTwoBytes = TYPE != FXP_F32;
    constexpr int kOutStride = WN * 2 + 16, kOut = WM * kOutStride;                                          // a wave's outputs of two bytes
    static_assert(LA * 8 * NW == BM && LB * 8 * NW == BN && LS * 32 * NW == BM + BN, "waves load as much");
    static_assert(kLoads * (STAGES - 1) < 64 && NW * kOut <= STAGES * kStage, "loads in flight, room for outputs");
    __shared__ __attribute__((aligned(1024))) uint8_t lds[STAGES * kStage];

    int tm, tn;
    tile_of_block(static_cast<int>(blockIdx.x), p.tiles_m, p.tiles_n, p.group_m, &tm, &tn);
    const int m0 = tm * BM, n0 = tn * BN;
    const int first = static_cast<int>(blockIdx.y) * p.per_split, panels = min(p.per_split, p.panels - first);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm0 = (wave / (BN / WN)) * WM, wn0 = (wave % (BN / WN)) * WN;

    // a wave's loads are NW x 8 rows apart (the exchange of pieces has a period of 16): one offset for all, the steps in the base
    const int row_l = wave * 8 + lane / 8, piece_l = ((lane % 8) ^ swizzle_of_row<kMxRowBytes>(row_l)) * 16;
    const int off_a = (m0 + row_l) * kMxRowBytes + piece_l, off_b = (n0 + row_l) * kMxRowBytes + piece_l;
    auto slot_of = [&](int t) { return lds + (t % STAGES) * kStage; };
    auto codes = [&](const Mx4Operand& o, int t, int j, int off, uint8_t* to) {
        const int size = o.rows * kMxRowBytes, step = j * NW * 1024;
        load_to_lds<16>(o.data + static_cast<int64_t>(first + t) * size + step, t < panels ? max(size - step, 0) : 0, off, to + wave * 1024 + step);
    };
    // past the last panel: no memory access, zeros
    auto issue_a = [&](int t) {
#pragma unroll
        for (int j = 0; j < LA; ++j) codes(p.a, t, j, off_a, slot_of(t));
    };
    auto issue_b = [&](int t) {
#pragma unroll
        for (int j = 0; j < LB; ++j) codes(p.b, t, j, off_b, slot_of(t) + kCodesA);
#pragma unroll
        for (int j = 0; j < LS; ++j) {
            const int i = wave + j * NW;                            // 256 bytes: 32 rows of scales
            const bool of_a = i < BM / 32;
            const Mx4Operand& o = of_a ? p.a : p.b;
            load_to_lds<4>(o.scales + static_cast<int64_t>(first + t) * o.rows * kMxRowScales, t < panels ? o.rows * kMxRowScales : 0,
                           (of_a ? m0 + 32 * i : n0 + 32 * (i - BM / 32)) * kMxRowScales + 4 * lane, slot_of(t) + kCodes + 256 * i);
        }
    };

    v16f acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = {};
    const int frow = lane & 31, fhalf = lane >> 5, fswz = swizzle_of_row<kMxRowBytes>(frow);
    v4i fa[2][FM], fb[2][FN];
    int ea[FM], eb[FN], next_a[FM], next_b[FN];
    auto read = [&](auto buf_c, int t, auto ks_c) {
        constexpr int BUF = decltype(buf_c)::value, KS = decltype(ks_c)::value;
        const uint8_t* const stage = slot_of(t);
        const int piece = ((2 * KS + fhalf) ^ fswz) * 16;
#pragma unroll
        for (int i = 0; i < FM; ++i) fa[BUF][i] = *reinterpret_cast<const v4i*>(stage + (wm0 + 32 * i + frow) * kMxRowBytes + piece);
#pragma unroll
        for (int j = 0; j < FN; ++j) fb[BUF][j] = *reinterpret_cast<const v4i*>(stage + (BM + wn0 + 32 * j + frow) * kMxRowBytes + piece);
    };
    auto read_scales = [&](int t) {
        const uint8_t* const at = slot_of(t) + kCodes + 4 * fhalf;
#pragma unroll
        for (int i = 0; i < FM; ++i) next_a[i] = *reinterpret_cast<const int*>(at + (wm0 + 32 * i + frow) * kMxRowScales);
#pragma unroll
        for (int j = 0; j < FN; ++j) next_b[j] = *reinterpret_cast<const int*>(at + (BM + wn0 + 32 * j + frow) * kMxRowScales);
    };
    auto take_scales = [&] {
#pragma unroll
        for (int i = 0; i < FM; ++i) ea[i] = next_a[i];
#pragma unroll
        for (int j = 0; j < FN; ++j) eb[j] = next_b[j];
    };
    auto multiply = [&](auto buf_c, auto ks_c, auto reads_c, auto loads_c) {
        constexpr int BUF = decltype(buf_c)::value, KS = decltype(ks_c)::value;
        constexpr int reads = decltype(reads_c)::value / 2, loads = decltype(loads_c)::value, rest = FM * FN - reads - loads;
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
                acc[i][j] = kTwoBytes ? mfma32<KS, KS>(fb[BUF][j], fa[BUF][i], acc[i][j], eb[j], ea[i]) : mfma32<KS, KS>(fa[BUF][i], fb[BUF][j], acc[i][j], ea[i], eb[j]);
        if constexpr (rest >= 0) {                                  // one multiplication, then two reads of LDS or a load, and so on
#pragma unroll
            for (int n = 0; n < reads; ++n) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            }
#pragma unroll
            for (int n = 0; n < loads; ++n) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
            }
            if constexpr (rest > 0) __builtin_amdgcn_sched_group_barrier(0x008, rest, 0);
        }
    };

#pragma unroll
    for (int t = 0; t + 1 < STAGES; ++t) {
        issue_a(t);
        issue_b(t);
    }
    issue_a(STAGES - 1);
    wait_loads_and_lds<(STAGES - 2) * kLoads + LA>();
    barrier();
    if (panels > 0) {
        read_scales(0);
        take_scales();
        read(IC<0>{}, 0, IC<0>{});
        int t = 0;
        for (; t + 1 < panels; ++t) {
            read(IC<1>{}, t, IC<1>{});
            issue_b(t + STAGES - 1);
            multiply(IC<0>{}, IC<0>{}, IC<FM + FN>{}, IC<LB + LS>{});
            read(IC<0>{}, t, IC<2>{});
            multiply(IC<1>{}, IC<1>{}, IC<FM + FN>{}, IC<0>{});
            read(IC<1>{}, t, IC<3>{});
            multiply(IC<0>{}, IC<2>{}, IC<FM + FN>{}, IC<0>{});
            wait_loads_and_lds<(STAGES - 2) * kLoads>();            // the next panel is there, and this one read
            barrier();
            read_scales(t + 1);
            read(IC<0>{}, t + 1, IC<0>{});
            issue_a(t + STAGES);
            multiply(IC<1>{}, IC<3>{}, IC<FM + FN>{}, IC<LA>{});
            take_scales();
        }
        read(IC<1>{}, t, IC<1>{});
        multiply(IC<0>{}, IC<0>{}, IC<FM + FN>{}, IC<0>{});
        read(IC<0>{}, t, IC<2>{});
        multiply(IC<1>{}, IC<1>{}, IC<FM + FN>{}, IC<0>{});
        read(IC<1>{}, t, IC<3>{});
        multiply(IC<0>{}, IC<2>{}, IC<FM + FN>{}, IC<0>{});
        multiply(IC<1>{}, IC<3>{}, IC<0>{}, IC<0>{});
    }
    wait_loads_and_lds<0>();                                        // none into LDS may outlive the workgroup

    const int row0 = m0 + wm0, col0 = n0 + wn0;
    if constexpr (!kTwoBytes) {
        // register r of a lane: row 8 (r / 4) + 4 (lane / 32) + r % 4, column lane % 32 of its fragment
        const int64_t base = static_cast<int64_t>(blockIdx.y) * p.split_stride + (row0 + 4 * fhalf) * p.ldc + col0 + frow;
        const bool inside = row0 + WM <= p.M && col0 + WN <= p.N;              // uniform
        float* const c = static_cast<float*>(p.c) + base;
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int dr = 32 * i + 8 * (r >> 2) + (r & 3);
                if (!inside && row0 + 4 * fhalf + dr >= p.M) continue;
#pragma unroll
                for (int j = 0; j < FN; ++j)
                    if (inside || col0 + 32 * j + frow < p.N) c[dr * p.ldc + 32 * j] = acc[i][j][r];
            }
    } else {
        // row lane % 32, column 8 (r / 4) + 4 (lane / 32) + r % 4
        using T = typename Elem<TYPE>::T;
        typedef T Four __attribute__((ext_vector_type(4)));
        barrier();                                                  // every wave is done with the panels
        uint8_t* const mine = lds + wave * kOut;
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    Four v;
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = static_cast<T>(acc[i][j][4 * q + k]);
                    *reinterpret_cast<Four*>(mine + (32 * i + frow) * kOutStride + (32 * j + 8 * q + 4 * fhalf) * 2) = v;
                }
        wave_barrier();
        constexpr int kPieces = WN / 8;                             // of 16 bytes in a row
#pragma unroll
        for (int n = 0; n < WM * kPieces / 64; ++n) {
            const int row = (n * 64 + lane) / kPieces, piece = lane % kPieces, col = col0 + 8 * piece;
            if (row0 + row >= p.M) continue;
            T* const c = static_cast<T*>(p.c) + (row0 + row) * p.ldc + col;
            const v4i v = *reinterpret_cast<const v4i*>(mine + row * kOutStride + piece * 16);
            if (col + 8 <= p.N) {
                reinterpret_cast<Sixteen*>(c)->v = v;
            } else {
                typedef T Eight __attribute__((ext_vector_type(8)));
                const Eight e = __builtin_bit_cast(Eight, v);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (col + k < p.N) c[k] = e[k];
            }
        }
    }
}

// ---- a few rows ----
//
// A workgroup has 16 rows of B (outputs) and all of A's; its waves take panels in turn and add up at the end.  A wave has U panels in flight, straight to LDS and out of it
// again: a load of its own registers would have neighbouring lanes in different rows, 64 accesses of a cache line where 1024 bytes in a row are eight (37 x 4096 x 8192
// 9.5 us, so 5.3).  Bound by B's bytes where all of its panels are in flight (one row by 8192 x 8192 8.6 us, 36 MB at 4.4 TB/s; 37 x 4100 x 9001 8.5).
// FUSED: A is not mapped yet; up to four rows of it.  A wave maps the panels that it takes, a row at a time, four elements a lane: less than a launch of its own.
constexpr int kTokens = 4;

struct Mx4Rows {
    Mx4Product p;
    const void* x;          // FUSED: A as it is
    int64_t ldx;
    int K, vec;
};

template <int MT, int U, int WAVES, int TYPE, int FUSED>         // FUSED: 0, or the rows of A
__global__ __launch_bounds__(WAVES * 64) void k_mx4_rows(Mx4Rows g) {
    const Mx4Product& p = g.p;
    constexpr int RA = FUSED ? FUSED : 16 * MT, RB = 16;
    constexpr int kScalesB = (RB * kMxRowScales + 255) / 256 * 256, kScalesA = FUSED ? (RA * kMxRowScales + 15) / 16 * 16 : (RA * kMxRowScales + 255) / 256 * 256;
    constexpr int kSlot = (RA + RB) * kMxRowBytes + kScalesA + kScalesB, kAtA = RB * kMxRowBytes, kAtSB = kAtA + RA * kMxRowBytes, kAtSA = kAtSB + kScalesB;
    constexpr int kBytes = WAVES * U * kSlot, kSums = WAVES * MT * 64 * 16;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kBytes > kSums ? kBytes : kSums];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = static_cast<int>(blockIdx.x) * RB, r = lane & 15, kb = lane >> 4;
    using T = typename Elem<TYPE>::T;
    v4f acc[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[m] = {};
    // lane l of a load has 16 bytes of row l / 8 of eight, exchanged by the row as in the tiles
    int from[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) from[i] = lane / 8 * kMxRowBytes + ((lane % 8) ^ swizzle_of_row<kMxRowBytes>(8 * i + lane / 8)) * 16;
    // block 4 h + kb of a panel: its scale is byte kb / 2 + 2 h of word kb % 2
    const int shift = 8 * (kb >> 1), swz = swizzle_of_row<kMxRowBytes>(r);
    uint8_t* const mine = lds + wave * U * kSlot;
    for (int t0 = wave; t0 < p.panels; t0 += WAVES * U) {
        float x[U][FUSED ? FUSED : 1][4];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int t = t0 + u * WAVES;
            const bool there = t < p.panels;                        // past the last: no memory access, zeros
            uint8_t* const slot = mine + u * kSlot;
            if constexpr (FUSED) {                                  // these first: they are waited for first
                const int c = t * kMxPanel + 4 * lane;
#pragma unroll
                for (int m = 0; m < FUSED; ++m) {
                    const T* const row = static_cast<const T*>(g.x) + m * g.ldx + c;
                    if (g.vec && c + 4 <= g.K && m < p.M) {
                        load_elems<TYPE, 4>(row, 0, true, x[u][m]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j) x[u][m][j] = c + j < g.K && m < p.M ? static_cast<float>(row[j]) : 0.0f;
                    }
                }
            }
            const uint8_t* const b = p.b.data + int64_t{t} * p.b.rows * kMxRowBytes;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                load_to_lds<16>(b, there ? p.b.rows * kMxRowBytes : 0, (n0 + 8 * i) * kMxRowBytes + from[i % 2], slot + i * 1024);
            const uint8_t* const sb = p.b.scales + int64_t{t} * p.b.rows * kMxRowScales;
            load_to_lds<4>(sb, there ? p.b.rows * kMxRowScales : 0, n0 * kMxRowScales + 4 * lane, slot + kAtSB);
            if constexpr (!FUSED) {
                const uint8_t* const a = p.a.data + int64_t{t} * p.a.rows * kMxRowBytes;
#pragma unroll
                for (int i = 0; i < 2 * MT; ++i)
                    load_to_lds<16>(a, there ? p.a.rows * kMxRowBytes : 0, 8 * i * kMxRowBytes + from[i % 2], slot + kAtA + i * 1024);
                const uint8_t* const sa = p.a.scales + int64_t{t} * p.a.rows * kMxRowScales;
#pragma unroll
                for (int i = 0; i < kScalesA / 256; ++i) load_to_lds<4>(sa, there ? p.a.rows * kMxRowScales : 0, 32 * i * kMxRowScales + 4 * lane, slot + kAtSA + 256 * i);
            }
        }
        if constexpr (FUSED) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int m = 0; m < FUSED; ++m) {
                    uint8_t* const slot = mine + u * kSlot;
                    const int s = mx_scale_of(mx_max_of_8(x[u][m]));
                    const float f = mx_inverse(s);
                    const float y[4] = {x[u][m][0] * f, x[u][m][1] * f, x[u][m][2] * f, x[u][m][3] * f};
                    *reinterpret_cast<uint16_t*>(slot + kAtA + m * kMxRowBytes + 2 * lane) = static_cast<uint16_t>(mx_nearest(y));
                    if ((lane & 7) == 0) slot[kAtSA + m * kMxRowScales + mx_scale_place(lane >> 3)] = static_cast<uint8_t>(s);
                }
        }
        wait_loads_and_lds<0>();
        wave_barrier();                                             // a wave's own slots
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint8_t* const slot = mine + u * kSlot;
            v4i b[2], a[MT][2];
            int ea[MT];
#pragma unroll
            for (int h = 0; h < 2; ++h) b[h] = *reinterpret_cast<const v4i*>(slot + r * kMxRowBytes + ((4 * h + kb) ^ swz) * 16);
            const int eb = *reinterpret_cast<const int*>(slot + kAtSB + r * kMxRowScales + 4 * (kb & 1)) >> shift;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                // rows of X that are not there: FUSED has zeros where it has a slot, and reads its last row again, as zeros, where it has none
                const int row = FUSED ? min(r, FUSED - 1) : 16 * m + r;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    a[m][h] = *reinterpret_cast<const v4i*>(slot + kAtA + row * kMxRowBytes + (FUSED ? 4 * h + kb : (4 * h + kb) ^ swz) * 16);
                    if (FUSED && r >= FUSED) a[m][h] = v4i{};
                }
                ea[m] = *reinterpret_cast<const int*>(slot + kAtSA + row * kMxRowScales + 4 * (kb & 1)) >> shift;
                if (FUSED && r >= FUSED) ea[m] = 0;
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                acc[m] = mfma16<0, 0>(b[0], a[m][0], acc[m], eb, ea[m]);
                acc[m] = mfma16<2, 2>(b[1], a[m][1], acc[m], eb, ea[m]);
            }
        }
        wait_loads_and_lds<0>();
        wave_barrier();                                             // before the slots are loaded again
    }
    v4f(*const sums)[MT][64] = reinterpret_cast<v4f(*)[MT][64]>(lds);
    if constexpr (WAVES > 1) {
        __syncthreads();                                            // the slots of other waves
#pragma unroll
        for (int m = 0; m < MT; ++m) sums[wave][m][lane] = acc[m];
        __syncthreads();
    }
    // outputs 4 kb .. 4 kb + 3 of B's rows, row r of a tile of A's
    for (int tile = wave; tile < MT; tile += WAVES) {
        v4f s;
        if constexpr (WAVES > 1) {
            s = sums[0][tile][lane];
            for (int w = 1; w < WAVES; ++w) s += sums[w][tile][lane];
        } else {
            s = acc[0];
#pragma unroll
            for (int i = 1; i < MT; ++i)
                if (i == tile) s = acc[i];
        }
        const int row = 16 * tile + r, col = n0 + 4 * kb;
        if (row >= p.M) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (col + j < p.N) store_one<TYPE>(p.c, row * p.ldc + col + j, s[j]);
    }
}

// Rows of A that go by workgroups of 16 rows of B: 64 x 4096 x 9008 9.1 us (by tiles 14.3), 37 x 4096 x 2048 3.8 (6.2); 65 rows are two such
// workgroups' work and 10.3 us by tiles.
constexpr int kRowsMost = 64;

// How a product is cut: tiles, and parts of the contraction where the tiles alone leave CUs idle.
//
// Tiles run in rounds of as many as are resident on 256 CUs: one a CU of 256 x 256, two of 128 x 128, three of 64 x 64.  A round of the smaller ones takes 0.57 and 0.38 of the
// time of one of the large (2048^3 14.7 / 8.5 / 11.0 us by 256, 128 and two rounds of 64; 768 x 12608 x 2304 62.8 / 38.6 / 26.6; 3000 x 1024 x 5000 15.6 / 16.4 in two rounds /
// 22.5 in five; 11000 x 300 x 500 11.9 / 9.1 / 9.6 in two): the tile with the shortest rounds in all is taken.
// Fewer than 256 tiles of 64 x 64 with eight panels or more: parts of at least four panels, about two workgroups a CU (768 x 12608 x 768 19.1 us in one part, 16.3 in four,
// 18.2 in eight; 192 x 9000 x 64 13.3 / 7.9 / 6.8; 300 x 4096 x 4096, 320 tiles, 10.2 in one, 15.2 in two).
struct Mx4Plan {
    bool rows;
    int tile, splits, per_split;
};
static Mx4Plan mx4_plan(int64_t M, int64_t N, int64_t K) {
    const int64_t panels = mx_panels(K);
    Mx4Plan p{M <= kRowsMost, 64, 1, static_cast<int>(panels)};
    if (p.rows) return p;
    auto tiles = [&](int64_t t) { return ((M + t - 1) / t) * ((N + t - 1) / t); };
    auto rounds = [&](int64_t t, int64_t resident) { return (tiles(t) + resident - 1) / resident; };
    const int64_t by_64 = 38 * rounds(64, 768), by_128 = 57 * rounds(128, 512), by_256 = 100 * rounds(256, 256);
    if (by_256 <= std::min(by_64, by_128)) p.tile = 256;
    else if (by_128 <= by_64) p.tile = 128;
    const int64_t count = tiles(p.tile);
    if (p.tile == 64 && count < 256 && panels >= 8) {
        const int64_t want = std::min<int64_t>(panels / 4, (512 + count - 1) / count);
        p.per_split = static_cast<int>((panels + want - 1) / want);
        p.splits = static_cast<int>((panels + p.per_split - 1) / p.per_split);
    }
    return p;
}
// of one part: parts begin on 16 bytes
static int64_t part_elements(int64_t M, int64_t N) { return (M * N + 3) / 4 * 4; }

size_t mx4_gemm_bytes(int64_t M, int64_t N, int64_t K) {
    const Mx4Plan p = mx4_plan(M, N, K);
    return p.splits > 1 ? round_up(static_cast<size_t>(p.splits) * part_elements(M, N) * sizeof(float), 256) : 0;
}

template <typename F>
static void by_type(int type, F go) {
    if (type == FXP_F32) go(IC<FXP_F32>{});
    else if (type == FXP_BF16) go(IC<FXP_BF16>{});
    else go(IC<FXP_F16>{});
}

static int sum_launch(const Mx4Sum& r, int type, hipStream_t s) {
    by_type(type, [&](auto type_c) { hipLaunchKernelGGL((k_mx4_sum<decltype(type_c)::value>), dim3(sum_blocks(r, 256)), dim3(256), 0, s, r); });
    return launch_status();
}

// U panels of a wave in flight, as many as leave room for two workgroups on a CU, where the contraction has more than 4 U (half of what a workgroup of eight waves holds then);
// else one, of eight waves, of four up to four panels (one row by 1024 x 16384 4.6 us, of eight 4.8), of one for a single panel.  us, launches back to back, weights out of memory
// (600 MB of them in turn), bf16, U in flight / one of eight waves; * what the rule takes:
//             N = 4096, K = 4096  8192          16384         N = 16384, K = 4096  8192  16384
//   1 row     5.5 / 5.2*   7.0* / 8.0    11.1* / 13.8  12.3 / 9.7*   18.5* / 17.7  33.3* / 31.6
//   2 rows    6.0* / 5.5   9.5* / 9.1    15.1* / 16.8  13.0* / 10.4  23.6* / 18.4  39.1* / 33.2
//   4 rows    7.6* / 6.3   12.6* / 10.7  21.2* / 21.3  16.7* / 11.7  31.2* / 21.2  50.2* / 38.7
//   9 rows    4.4* / 4.5   6.0* / 6.3    9.3* / 10.0   10.0* / 9.1   17.8* / 18.0  33.4* / 33.0
//   32 rows   5.5* / 5.0   8.3* / 7.2    14.1* / 11.7  13.0* / 12.3  22.5* / 22.2  40.9* / 41.4
// So U in flight is worth it for one row, and up to 16, where B has few rows; for 2 to 4 and for 17 to 32 rows, and where B's rows alone make four workgroups a CU, one panel of
// eight waves is as fast or faster.
static int rows_launch(const Mx4Rows& g, bool fused, int type, hipStream_t s) {
    const Mx4Product& p = g.p;
    by_type(type, [&](auto type_c) {
        constexpr int TYPE = decltype(type_c)::value;
        auto go = [&](auto mt_c, auto u_c, auto w_c, auto fused_c) {
            constexpr int W = decltype(w_c)::value;
            hipLaunchKernelGGL((k_mx4_rows<decltype(mt_c)::value, decltype(u_c)::value, W, TYPE, decltype(fused_c)::value>), dim3(static_cast<unsigned>((p.N + 15) / 16)),
                               dim3(64 * W), 0, s, g);
        };
        auto sized = [&](auto mt_c, auto u_c, auto w_c, auto fused_c) {
            constexpr int U = decltype(u_c)::value;
            if (p.panels > 4 * U) return go(mt_c, u_c, w_c, fused_c);
            if constexpr (U > 1)
                if (p.panels > 4) return go(mt_c, IC<1>{}, IC<8>{}, fused_c);
            if (p.panels > 1) go(mt_c, IC<1>{}, IC<4>{}, fused_c);
            else go(mt_c, IC<1>{}, IC<1>{}, fused_c);
        };
        if (fused && p.M == 1) sized(IC<1>{}, IC<4>{}, IC<8>{}, IC<1>{});
        else if (fused && p.M == 2) sized(IC<1>{}, IC<3>{}, IC<8>{}, IC<2>{});
        else if (fused) sized(IC<1>{}, IC<3>{}, IC<8>{}, IC<4>{});
        else if (p.M <= 16) sized(IC<1>{}, IC<2>{}, IC<8>{}, IC<0>{});
        else if (p.M <= 32) sized(IC<2>{}, IC<2>{}, IC<4>{}, IC<0>{});
        else if (p.M <= 48) sized(IC<3>{}, IC<1>{}, IC<4>{}, IC<0>{});          // 37 x 4100 x 9001 back to back 9.2 us, two panels a wave 10.4; 37 x 4096 x 4096 4.4 and 4.2
        else sized(IC<4>{}, IC<1>{}, IC<4>{}, IC<0>{});
    });
    return launch_status();
}

bool mx4_is_fused(int64_t M) { return M <= kTokens; }
// Y = X B^T for X as it is, up to kTokens rows of it: one launch, no workspace
int mx4_fused_launch(int type, const void* x, int64_t ldx, int64_t M, const fxp_mx4& B, void* y, int64_t ldy, hipStream_t s) {
    Mx4Rows g{};
    g.p.b = {B.data, B.scales, static_cast<int>(B.rows)};
    g.p.M = static_cast<int>(M);
    g.p.N = static_cast<int>(B.rows);
    g.p.panels = static_cast<int>(mx_panels(B.cols));
    g.p.c = y;
    g.p.ldc = ldy;
    g.x = x;
    g.ldx = ldx;
    g.K = static_cast<int>(B.cols);
    g.vec = aligned(x, 4 * static_cast<size_t>(elem_size(type))) && (M == 1 || ldx % 4 == 0);
    return rows_launch(g, true, type, s);
}

// rider: a sum to be done in this launch; rest: receives the product's own sum, if it has one, in place of a launch of it
static int gemm_launch(const fxp_mx4& A, const fxp_mx4& B, int type, void* C, int64_t ldc, void* ws, Mx4Sum rider, Mx4Sum* rest, hipStream_t s) {
    const int64_t M = A.rows, N = B.rows, K = A.cols;
    const Mx4Plan plan = mx4_plan(M, N, K);
    Mx4Product p{};
    p.a = {A.data, A.scales, static_cast<int>(M)};
    p.b = {B.data, B.scales, static_cast<int>(N)};
    p.M = static_cast<int>(M);
    p.N = static_cast<int>(N);
    p.panels = static_cast<int>(mx_panels(K));
    p.per_split = plan.per_split;
    p.c = C;
    p.ldc = ldc;
    const bool parts = plan.splits > 1;
    if (rider.count && (plan.rows || parts)) return FXP_ERR_DIMS;                        // cannot be: see mx4_gemm_launch2
    if (plan.rows) return rows_launch({p, nullptr, 0, 0, 0}, false, type, s);
    if (parts) {
        p.c = ws;
        p.ldc = N;
        p.split_stride = part_elements(M, N);
    }
    const int t = plan.tile;
    p.tiles_m = static_cast<int>((M + t - 1) / t);
    p.tiles_n = static_cast<int>((N + t - 1) / t);
    p.group_m = 8;
    const int64_t count = static_cast<int64_t>(p.tiles_m) * p.tiles_n;
    if (count >= int64_t{1} << 22) return FXP_ERR_DIMS;                                  // 2^32 threads, riders among them
    rider.tiles = static_cast<int>(count);
    by_type(parts ? FXP_F32 : type, [&](auto type_c) {
        constexpr int TYPE = decltype(type_c)::value;
        auto go = [&](auto kernel, int threads) {
            hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(count) + sum_blocks(rider, threads), static_cast<unsigned>(plan.splits)), dim3(threads), 0, s, p, rider);
        };
        if (t == 256) go(k_mx4_tiles<256, 256, 64, 128, 2, TYPE>, 512);
        else if (t == 128) go(k_mx4_tiles<128, 128, 64, 64, 2, TYPE>, 256);
        else go(k_mx4_tiles<64, 64, 32, 32, 3, TYPE>, 256);
    });
    const int rc = launch_status();
    if (rc || !parts) return rc;
    const bool flat = ldc == N;                                                          // one row (parts are of fewer than 2^24 outputs)
    Mx4Sum sum{static_cast<const float*>(ws), plan.splits, static_cast<int>(flat ? 1 : M), static_cast<int>(flat ? M * N : N), 0, p.split_stride, C, ldc, 0};
    if (flat || N % 4 == 0) sum.vec = aligned(C, 4 * static_cast<size_t>(elem_size(type))) && (flat || ldc % 4 == 0) ? 2 : 1;
    if (rest) {
        *rest = sum;
        return FXP_OK;
    }
    return sum_launch(sum, type, s);
}

int mx4_gemm_launch(const fxp_mx4& A, const fxp_mx4& B, int type, void* C, int64_t ldc, void* ws, hipStream_t s) {
    return gemm_launch(A, B, type, C, ldc, ws, Mx4Sum{}, nullptr, s);
}

// Two products, the first one's partial sums added up in the second's launch; both use ws only one after the other.  The second goes by whole tiles
// then: where it has parts the first one's sum is a launch of its own, and a first contraction that is split has 1793 rows or more, which are the second's.
int mx4_gemm_launch2(const fxp_mx4& A0, const fxp_mx4& B0, void* C0, const fxp_mx4& A1, const fxp_mx4& B1, void* C1, int type, void* ws, hipStream_t s) {
    Mx4Sum sum{};
    const bool alone = mx4_gemm_bytes(A1.rows, B1.rows, A1.cols) != 0;                   // the second wants the workspace too
    const int rc = gemm_launch(A0, B0, type, C0, B0.rows, ws, Mx4Sum{}, alone ? nullptr : &sum, s);
    return rc ? rc : gemm_launch(A1, B1, type, C1, B1.rows, ws, sum, nullptr, s);
}

}  // namespace fxp
