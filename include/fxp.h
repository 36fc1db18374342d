/*
 * fxp.h — C ABI of libfxp: the integer (dynamic fixed-point) layer step of "Is Integer
 * Arithmetic Enough for Deep Learning Training?" (arXiv 2207.08822) - linear, convolution
 * and batched-product layers, forward and backward, and the int16 weight update - as
 * hand-written HIP kernels for gfx950 (MI355X).
 *
 * Conventions that hold for every call
 *  - Every data pointer is a DEVICE pointer unless the argument says "host".
 *    The caller owns every buffer; the library never allocates, frees or keeps
 *    a pointer after the call's work has run.
 *  - All matrices are dense row-major.  X[M,K], W[K,N], Y[M,N], dY[M,N],
 *    dX[M,K], dW[K,N] (the paper's Y = XW, App. A.2).
 *  - `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *    Calls only enqueue work; they never synchronise and never read device
 *    memory from the host, so per-tensor scales stay on the device.
 *  - `ws` is device scratch of at least fxp_workspace_bytes(...) bytes, 256-byte
 *    aligned, private to the call until its work has finished on `stream`.
 *  - Return value: FXP_OK (0) or a negative fxp_status; nothing is enqueued when
 *    an argument error is returned.  Launch failures reported by the runtime map
 *    to FXP_ERR_LAUNCH.  No exception crosses this boundary.
 *  - A mapped tensor is int8 values q plus ONE int32 scale e_max (the biased
 *    fp32 exponent field of its largest magnitude, Sec. 3.1); q stands for the
 *    real number q * 2^(e_max - 127 - (bits - 2)), i.e. q * 2^(e_max - 133) for
 *    the paper's int8 (bits = 8: sign + 7 magnitude bits).
 *  - Inputs must be finite.  Non-finite input is not an error (it cannot be seen
 *    without a synchronisation): the scale then reads 255, +-Inf maps to the
 *    largest magnitude and NaN to 0.
 */
#ifndef FXP_H_
#define FXP_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum fxp_status {
    FXP_OK = 0,
    FXP_ERR_NULL = -1,      /* a required pointer is NULL */
    FXP_ERR_DIMS = -2,      /* negative size, leading dimension too small, or size beyond the supported range */
    FXP_ERR_ALIGN = -3,     /* a pointer misses the alignment stated for it */
    FXP_ERR_WORKSPACE = -4, /* ws is NULL or smaller than fxp_workspace_bytes says */
    FXP_ERR_ROUNDING = -5,  /* unknown rounding mode */
    FXP_ERR_BITS = -6,      /* bits outside [2, 8] */
    FXP_ERR_LAUNCH = -7,    /* the HIP runtime refused a launch */
    FXP_ERR_OVERFLOW = -8,  /* contraction longer than an int32 sum is sure to hold (> 133144 terms) where the call has no
                               64-bit path for it: int32 output, a batched product, or no room in ws for the slices */
    FXP_ERR_TYPE = -9,      /* unknown element type */
    FXP_ERR_VALUE = -10     /* a scalar argument outside its range, or operands that share memory where they must not */
} fxp_status;

/* Rounding of the 24-bit shifted mantissa to bits-1 magnitude bits. */
enum {
    FXP_ROUND_STOCHASTIC = 0, /* App. A.1: up with probability (dropped bits) / 2^(number dropped) */
    FXP_ROUND_NEAREST = 1     /* half up on the magnitude; for comparison runs only */
};

/* Operation selector of fxp_workspace_bytes. */
enum { FXP_OP_SCALE = 0, FXP_OP_GEMM = 1, FXP_OP_LINEAR_FWD = 2, FXP_OP_LINEAR_BWD = 3, FXP_OP_BMM_FWD = 4, FXP_OP_BMM_BWD = 5 };

/* Random-stream tags of the layer calls: stream_id = (step << 8) | tag. */
enum { FXP_TAG_X = 0, FXP_TAG_W = 1, FXP_TAG_DY = 2 };

/* Host string for a status code (static storage). */
const char* fxp_strerror(int status);

/* Library version, major * 100 + minor. */
int fxp_version(void);

/* Scratch bytes an operation needs.  FXP_OP_SCALE: M = number of elements.
 * FXP_OP_GEMM: worst case over the operand forms of fxp_gemm / fxp_gemm_unmap.
 * FXP_OP_GEMM includes the int32 slices a long, narrow product is split into along K.
 * FXP_OP_BMM_FWD / _BWD: scale scratch only, whatever the shapes.
 * FXP_OP_LINEAR_FWD / _BWD: layer shapes M, N, K as above.  Returns 0 on bad
 * arguments. */
size_t fxp_workspace_bytes(int op, int64_t M, int64_t N, int64_t K);

/* Scale of a tensor (Sec. 3.1: e_max = max(e_1 .. e_n)).
 * x: n fp32 values, 4-byte aligned, any n >= 0.  e_max: one int32, receives the
 * largest biased exponent field, counting zeros and sub-normals as 1, so the
 * result lies in [1, 255] (n = 0 gives 1). */
int fxp_scale(const float* x, size_t n, int32_t* e_max, void* ws, size_t ws_bytes, void* stream);

/* Linear fixed-point mapping (Sec. 3.1; stochastic rounding of App. A.1, Fig. 4).
 * x: [rows, cols] fp32.  e_max: the tensor's scale as fxp_scale wrote it (a
 * larger value is allowed, e.g. a scale shared between shards; elements whose
 * exponent exceeds it saturate).  q: [rows, cols] int8 or NULL.  qT: [cols,
 * rows] int8 or NULL, the same values transposed (one rounding decision per
 * element, shared by both copies).  At least one of q, qT is required.
 * Per element: 24-bit mantissa (hidden bit restored) shifted right by
 * e_max - e, cut after bits-1 magnitude bits, rounded up iff r < dropped bits,
 * saturated to 2^(bits-1) - 1, sign attached.  r is the top (25 - bits) bits
 * of word (i mod 4) of Philox-4x32-10 with key = seed and counter =
 * (i / 4, stream_id), i = row * cols + col: the result does not depend on the
 * launch geometry or on which copies are requested.
 * Fastest with x, q, qT 16-byte aligned and cols a multiple of 4 (or with q alone, whatever the shape);
 * other alignments and widths are tiled in the same way with unaligned accesses, results are identical. */
int fxp_map(const float* x, int64_t rows, int64_t cols, const int32_t* e_max, int8_t* q, int8_t* qT, uint64_t seed,
            uint64_t stream_id, int rounding, int bits, void* stream);

/* fxp_scale followed by fxp_map with the final reduction folded into the map
 * kernel: writes *e_max and q / qT exactly as the two calls would. */
int fxp_scale_map(const float* x, int64_t rows, int64_t cols, int32_t* e_max, int8_t* q, int8_t* qT, uint64_t seed,
                  uint64_t stream_id, int rounding, int bits, void* ws, size_t ws_bytes, void* stream);

/* Two tensors per launch: what fxp_map / fxp_scale_map do for one tensor, done for two with one map launch
 * (and one reduction launch) instead of two each - the layer calls use this for the activation and the
 * weight of a forward pass, where the second tensor is often too small to fill the chip by itself.  Results
 * are identical to two separate calls.  One launch needs both tensors tiled or flat (see fxp_map: rows of 16 columns or more,
 * or row-major only, whatever the width); otherwise two launches are made.  Two small tensors have their scales found in the
 * same launch.
 */
typedef struct fxp_map_desc {
    const float* x;      /* [rows, cols] fp32, device */
    int64_t rows, cols;
    int32_t* e_max;      /* device: read by fxp_map2, written by fxp_scale_map2 */
    int8_t* q;           /* [rows, cols] or NULL */
    int8_t* qT;          /* [cols, rows] or NULL */
    uint64_t stream_id;
} fxp_map_desc;
int fxp_map2(const fxp_map_desc* a, const fxp_map_desc* b, uint64_t seed, int rounding, int bits, void* stream);
/* ws: device, >= 2 * fxp_workspace_bytes(FXP_OP_SCALE, ...) bytes */
int fxp_scale_map2(const fxp_map_desc* a, const fxp_map_desc* b, uint64_t seed, int rounding, int bits, void* ws,
                   size_t ws_bytes, void* stream);

/* Number of uint32 words of an abs-max area (see fxp_gemm_unmap_absmax). */
#define FXP_ABSMAX_WORDS 256

/* fxp_map with the scale taken from the largest magnitude of the tensor, given as an abs-max area: device
 * array of FXP_ABSMAX_WORDS uint32 whose maximum is the IEEE bit pattern of max |x_i| (what
 * fxp_gemm_unmap_absmax leaves behind for its output).  The scale of Sec. 3.1 is the exponent field of that
 * maximum, at least 1.  It is written to *e_max (required) and used for the mapping in the same launch, so a
 * tensor produced by a product of this library is mapped without a reduction pass of its own.  An area below
 * the tensor's true maximum gives a scale below the tensor (elements above it saturate), as a too small e_max
 * does for fxp_map. */
int fxp_map_absmax(const float* x, int64_t rows, int64_t cols, const uint32_t* absmax, int32_t* e_max, int8_t* q, int8_t* qT,
                   uint64_t seed, uint64_t stream_id, int rounding, int bits, void* stream);

/* Integer GEMM (Sec. 3.3, Fig. 2: int8 x int8 products, int32 accumulation).
 * C[M,N] = op(A)[M,K] * op(B)[K,N], C overwritten.
 * transA = 0: A stored [M,K], lda >= K.  transA = 1: A stored [K,M], lda >= M.
 * transB = 0: B stored [K,N], ldb >= N.  transB = 1: B stored [N,K], ldb >= K.
 * Native form is (transA, transB) = (0, 1), both operands contiguous along the
 * contraction; other forms first transpose the operand into ws.  K <= 133144 (127^2 * K < 2^31: the int32
 * sums cannot wrap).
 * Fast loads need A, B 16-byte aligned and lda, ldb, K multiples of 16; other
 * shapes are loaded 16 bytes at a time at any address, results are identical.  C 4-byte aligned. */
int fxp_gemm(int transA, int transB, int64_t M, int64_t N, int64_t K, const int8_t* A, int64_t lda, const int8_t* B,
             int64_t ldb, int32_t* C, int64_t ldc, void* ws, size_t ws_bytes, void* stream);

/* Non-linear inverse mapping (Sec. 3.2, Fig. 1b) of an integer tensor with the
 * shared exponent of Sec. 3.3 (sum of the operand exponents):
 * out = fp32 nearest (ties to even, gradual underflow, overflow to Inf) to
 * acc * 2^E, E = (eA - 127 - (bitsA-2)) + (eB - 127 - (bitsB-2)); eB = NULL
 * drops the second term.  acc and out may be the same buffer. */
int fxp_unmap(const int32_t* acc, size_t n, const int32_t* eA, int bitsA, const int32_t* eB, int bitsB, float* out,
              void* stream);

/* Inverse mapping of a mapped int8 tensor itself: out = q * 2^(eA - 127 - (bitsA-2)). */
int fxp_unmap_i8(const int8_t* q, size_t n, const int32_t* eA, int bitsA, float* out, void* stream);

/* fxp_gemm with the inverse mapping fused into its epilogue: C is fp32 and
 * receives what fxp_unmap would make of the int32 result.
 * K may exceed 133144 here: the contraction then runs as slices of at most 133120 terms, each summed exactly
 * in int32 into ws, and the slices are added in 64 bits before the one rounding of the inverse mapping - C is
 * the exact integer sum times 2^E, rounded once, at any K < 2^31.  That needs the ws of
 * fxp_workspace_bytes(FXP_OP_GEMM, M, N, K); with less, FXP_ERR_OVERFLOW. */
int fxp_gemm_unmap(int transA, int transB, int64_t M, int64_t N, int64_t K, const int8_t* A, int64_t lda,
                   const int8_t* B, int64_t ldb, const int32_t* eA, int bitsA, const int32_t* eB, int bitsB, float* C,
                   int64_t ldc, void* ws, size_t ws_bytes, void* stream);

/* fxp_gemm_unmap that also leaves the largest output magnitude behind, so that the next layer can map C without
 * a reduction pass over it (Sec. 3.1's scale is the exponent field of that magnitude).  out_absmax (required):
 * device array of FXP_ABSMAX_WORDS uint32, 4-byte aligned; the call raises its words by atomic maxima so that
 * their maximum is at least the IEEE bit pattern of max |C_ij| (several words, so that the workgroups do not
 * all hit one address).  The caller zeroes the area before the first product that contributes to a tensor
 * (several products may fill parts of one tensor).  Consumed by fxp_map_absmax.  Everything else as
 * fxp_gemm_unmap. */
int fxp_gemm_unmap_absmax(int transA, int transB, int64_t M, int64_t N, int64_t K, const int8_t* A, int64_t lda,
                          const int8_t* B, int64_t ldb, const int32_t* eA, int bitsA, const int32_t* eB, int bitsB,
                          float* C, int64_t ldc, uint32_t* out_absmax, void* ws, size_t ws_bytes, void* stream);

/* Mapped operands a forward call leaves for the backward call (host struct of
 * device pointers, all caller-allocated, 16-byte aligned). */
typedef struct fxp_saved {
    int8_t* Xq;   /* [M,K] */
    int8_t* XqT;  /* [K,M] */
    int8_t* Wq;   /* [K,N] */
    int8_t* WqT;  /* [N,K] */
    int32_t* eX;  /* 1 */
    int32_t* eW;  /* 1 */
} fxp_saved;

/* Forward of one integer linear layer (App. A.2: Y_hat = X_hat W_hat):
 * scale + map X (stream tag FXP_TAG_X), scale + map W (FXP_TAG_W), int8 GEMM,
 * inverse mapping -> Y[M,N] fp32.  Fills every member of *saved. */
int fxp_linear_fwd(const float* X, const float* W, int64_t M, int64_t K, int64_t N, float* Y, const fxp_saved* saved,
                   uint64_t seed, uint64_t step, int rounding, int bits, void* ws, size_t ws_bytes, void* stream);

/* fxp_linear_fwd for callers that cannot allocate device memory or hand over a workspace: code under HIP graph
 * capture, tight serving loops, harnesses that forbid allocation.  Same arguments without ws, same results bit
 * for bit; the call allocates and frees nothing.  Its scratch (block maxima of the two scale reductions, int32
 * slices of a product that is split along its contraction) is a device array of FXP_STATIC_SCRATCH_BYTES bytes
 * inside the library, one copy per GPU, held until the process ends.  A layer that needs more -
 * fxp_workspace_bytes(FXP_OP_LINEAR_FWD, M, N, K) > FXP_STATIC_SCRATCH_BYTES, which only long contractions into
 * small outputs reach - returns FXP_ERR_WORKSPACE and enqueues nothing.  All calls on one GPU share that GPU's
 * array: two calls whose work overlaps in time on one GPU (different streams, or different threads) race;
 * calls on one stream are ordered and safe.  The array's previous contents never matter (every word read was
 * written by the same call).  The first call on a device looks the array's address up (no allocation), so make
 * one call per device before a capture begins. */
#define FXP_STATIC_SCRATCH_BYTES (32u << 20)
size_t fxp_static_scratch_bytes(void);
int fxp_linear_fwd_static(const float* X, const float* W, int64_t M, int64_t K, int64_t N, float* Y, const fxp_saved* saved,
                          uint64_t seed, uint64_t step, int rounding, int bits, void* stream);

/* Backward of the same layer (App. A.2: dL/dW = X_hat^T G_hat; chain rule for
 * dL/dX = G_hat W_hat^T): scale + map dY ONCE (FXP_TAG_DY; both GEMMs use the
 * same rounded gradient), then dX[M,K] and dW[K,N] as fp32.  dX or dW may be
 * NULL to skip it.  dYq [M,N], dYqT [N,M] and e_dY (1 int32) are caller-
 * allocated outputs/scratch.  Uses saved->XqT, saved->Wq, saved->eX, saved->eW.
 * M, K, N are not limited by the int32 accumulator: a contraction of more than 133144 terms (the weight
 * gradient of a layer applied to more rows than that) runs as slices, see fxp_gemm_unmap. */
int fxp_linear_bwd(const float* dY, const fxp_saved* saved, int64_t M, int64_t K, int64_t N, float* dX, float* dW,
                   int8_t* dYq, int8_t* dYqT, int32_t* e_dY, uint64_t seed, uint64_t step, int rounding, int bits,
                   void* ws, size_t ws_bytes, void* stream);

/* The same two calls for a training loop, where a tensor's scale seldom moves from one step to the next (Sec. 3.1:
 * the scale is the largest exponent of the tensor).  saved->eX, saved->eW and e_dY are read on entry as GUESSES of
 * the scales (what the previous step's call left there; any other content is harmless).  Each large tensor is then
 * read ONCE: a single pass maps it with the guess and finds its true largest magnitude, and a second, short launch
 * verifies - if the guess was the scale, the mapped tensor is already what fxp_linear_fwd / _bwd would have
 * written; if not (the maximum crossed a power of two, first call, garbage in the word), that launch maps the
 * tensor again with the true scale.  Results are bit for bit those of fxp_linear_fwd / fxp_linear_bwd in every
 * case; a hit saves the reduction's pass over the tensor (4 of 10 bytes per element), a miss costs one map pass
 * more.  Tensors below 2^22 elements and tensors off the fast path of fxp_map take the two-pass path as before. */
int fxp_linear_fwd_guess(const float* X, const float* W, int64_t M, int64_t K, int64_t N, float* Y, const fxp_saved* saved,
                         uint64_t seed, uint64_t step, int rounding, int bits, void* ws, size_t ws_bytes, void* stream);
int fxp_linear_bwd_guess(const float* dY, const fxp_saved* saved, int64_t M, int64_t K, int64_t N, float* dX, float* dW,
                         int8_t* dYq, int8_t* dYqT, int32_t* e_dY, uint64_t seed, uint64_t step, int rounding, int bits,
                         void* ws, size_t ws_bytes, void* stream);

/* Batched integer GEMM for the attention products (the paper runs Q K^T and A V as int8 matmuls with the
 * softmax in floating point, Sec. 5 / ViT): `batch` (<= 65535) independent products in the native form
 * C_b[M,N] = A_b[M,K] * B_b[N,K]^T, matrix b of an operand starting b * stride elements after matrix 0.
 * One scale per TENSOR (all matrices of A share eA, all of B share eB), as everywhere in the method.
 * Fast loads need 16-byte aligned bases, and lda, ldb, strideA, strideB, K multiples of 16. */
int fxp_gemm_batched(int64_t M, int64_t N, int64_t K, const int8_t* A, int64_t lda, int64_t strideA, const int8_t* B,
                     int64_t ldb, int64_t strideB, int32_t* C, int64_t ldc, int64_t strideC, int64_t batch, void* stream);

int fxp_gemm_unmap_batched(int64_t M, int64_t N, int64_t K, const int8_t* A, int64_t lda, int64_t strideA, const int8_t* B,
                           int64_t ldb, int64_t strideB, const int32_t* eA, int bitsA, const int32_t* eB, int bitsB, float* C,
                           int64_t ldc, int64_t strideC, int64_t batch, void* stream);

/* Mapped operands of a batched product layer (host struct of device pointers, caller-allocated, 16-byte
 * aligned).  Each tensor is mapped ONCE as a whole, as a matrix of (batch * rows) x cols, in both orientations:
 *   Aq [batch*M, K]      AqT [K, batch*M]
 *   Bq  as Bm is laid out: [batch*K, N], or [batch*N, K] with transB;   BqT its transpose
 * so that every one of the three products per matrix reads K-contiguous operands through a leading dimension
 * and a batch stride alone (matrix b of a transposed copy is a block of columns). */
typedef struct fxp_bmm_saved {
    int8_t* Aq;
    int8_t* AqT;
    int8_t* Bq;
    int8_t* BqT;
    int32_t* eA;  /* 1 */
    int32_t* eB;  /* 1 */
} fxp_bmm_saved;

/* Forward of a batched product layer, the attention matmuls of the vision transformer (Sec. 5: Q K^T and A V
 * run on the integer mantissas, the softmax stays in floating point): Y_b = unmap(map(A)_b * op(map(Bm)_b)),
 * b < batch <= 65535.  A[batch,M,K] fp32; Bm[batch,K,N], or [batch,N,K] with transB != 0 (keys: scores =
 * Q K^T); Y[batch,M,N] fp32.  One scale per tensor; random streams FXP_TAG_X for A, FXP_TAG_W for Bm, element
 * index = row-major index in the whole tensor.  Fills every member of *saved.  Full speed needs M, K, N
 * multiples of 16 (pad the sequence length); other sizes take 16-byte loads at any address, same results.
 * ws: fxp_workspace_bytes(FXP_OP_BMM_FWD, ...) bytes, 256-byte aligned. */
int fxp_bmm_fwd(const float* A, const float* Bm, int64_t batch, int64_t M, int64_t K, int64_t N, int transB, float* Y,
                const fxp_bmm_saved* saved, uint64_t seed, uint64_t step, int rounding, int bits, void* ws,
                size_t ws_bytes, void* stream);

/* Backward: dY[batch,M,N] is mapped once (FXP_TAG_DY; dYq [batch*M,N], dYqT [N,batch*M], e_dY returned);
 * dA_b = unmap(G_b * op(Bq_b)^T) [batch,M,K]; dBm_b = unmap(Aq_b^T * G_b), in the layout of Bm.  dA or dBm may
 * be NULL to skip it. */
int fxp_bmm_bwd(const float* dY, const fxp_bmm_saved* saved, int64_t batch, int64_t M, int64_t K, int64_t N,
                int transB, float* dA, float* dBm, int8_t* dYq, int8_t* dYqT, int32_t* e_dY, uint64_t seed,
                uint64_t step, int rounding, int bits, void* ws, size_t ws_bytes, void* stream);

/* fxp_bmm_fwd / fxp_bmm_bwd with the scales saved->eA, saved->eB and e_dY hold on entry taken as guesses: see
 * fxp_linear_fwd_guess.  Same results bit for bit. */
int fxp_bmm_fwd_guess(const float* A, const float* Bm, int64_t batch, int64_t M, int64_t K, int64_t N, int transB, float* Y,
                      const fxp_bmm_saved* saved, uint64_t seed, uint64_t step, int rounding, int bits, void* ws,
                      size_t ws_bytes, void* stream);
int fxp_bmm_bwd_guess(const float* dY, const fxp_bmm_saved* saved, int64_t batch, int64_t M, int64_t K, int64_t N,
                      int transB, float* dA, float* dBm, int8_t* dYq, int8_t* dYqT, int32_t* e_dY, uint64_t seed,
                      uint64_t step, int rounding, int bits, void* ws, size_t ws_bytes, void* stream);

/* ---- int16 weight update (Remark 5, App. A.4: w_hat_{k+1} = w_hat_k + alpha_hat_k * g_hat, every term in fixed
 * point with stochastic rounding; the paper's runs use "int16 SGD", Sec. 5) ----
 * fxp_axpy16: z = x_hat + SR(a_hat * y_hat) over n elements.  x_hat, y_hat, a_hat are the 16-bit instance of
 * the mapping (15 magnitude bits, scale = largest exponent of the tensor; the scalar's scale is its own
 * exponent); the int32 product is brought to the unit of x_hat by a shift, with stochastic rounding of the
 * dropped bits, saturating at 2^23 - 2^15 units; the integer sum goes through the inverse mapping.  The paper
 * does not spell this formula out: alignment and place of the rounding are this library's reading.
 * x, y, z: device, fp32; z may be x or y (in place).  e_out: device int32[3] receiving the scales of x, y, a,
 * or NULL.  Random streams (step << 8) | 3..6.  ws: device, >= 2 * fxp_workspace_bytes(FXP_OP_SCALE) bytes. */
int fxp_axpy16(const float* x, const float* y, float a, size_t n, float* z, int32_t* e_out, uint64_t seed,
               uint64_t step, int rounding, void* ws, size_t ws_bytes, void* stream);

/* One SGD step with weight decay and momentum (the optimiser of the paper's classification runs), every line
 * an fxp_axpy16 with stream steps 3*step, 3*step+1, 3*step+2:
 *   g1 = g + weight_decay * w      (skipped when weight_decay == 0; needs tmp[n])
 *   v  = g1 + momentum * v         (skipped when momentum == 0; v may then be NULL)
 *   w  = w + (-lr) * v             (g1 in place of v without momentum)
 * w, v are updated in place; g is read only.  The scales of the intermediates come out of the producing
 * kernel, so the step reads w, g, v once for their scales and once per line.
 * ws: device, fxp_sgd16_workspace_bytes() bytes. */
size_t fxp_sgd16_workspace_bytes(void);
int fxp_sgd16_step(float* w, const float* g, float* v, size_t n, float lr, float momentum, float weight_decay, float* tmp,
                   uint64_t seed, uint64_t step, int rounding, void* ws, size_t ws_bytes, void* stream);

/* The same step for a whole list of parameter tensors, each with its own scales (the method keeps one scale per
 * tensor), in four launches per 64 tensors instead of six per tensor: what a model with dozens of parameter
 * tensors needs, since a dependent launch costs several microseconds.  Tensor t is updated exactly as
 * fxp_sgd16_step would update it with the stream step (step << 16) | t (so no two tensors share random numbers);
 * count <= 65536, step < 2^32.  `tensors` is a HOST array of device pointers (v may be NULL without momentum,
 * tmp without weight decay; n = 0 entries are skipped); it is only read during the call.
 * ws: device, fxp_sgd16_multi_workspace_bytes(tensors, count) bytes. */
typedef struct fxp_sgd_tensor {
    float* w;
    const float* g;
    float* v;
    float* tmp;
    size_t n;
} fxp_sgd_tensor;
size_t fxp_sgd16_multi_workspace_bytes(const fxp_sgd_tensor* tensors, size_t count);
int fxp_sgd16_step_multi(const fxp_sgd_tensor* tensors, size_t count, float lr, float momentum, float weight_decay,
                         uint64_t seed, uint64_t step, int rounding, void* ws, size_t ws_bytes, void* stream);

/* ---- convolution layer (Sec. 3.4: "Linear and convolutional layers" share the integer inner product) ----
 * Channels-last tensors: X[N,H,W,C], W[Cout,KH,KW,C], Y and dY [N,Ho,Wo,Cout] with
 * Ho = (H + 2 pad - KH) / stride + 1 (same for Wo), zero padding.  Host struct. */
typedef struct fxp_conv2d_shape {
    int64_t N, H, W, C, Cout, KH, KW, stride, pad;
} fxp_conv2d_shape;

/* What a forward call leaves for the backward call (host struct of device pointers, caller-allocated,
 * 16-byte aligned): the int8 activation itself, the int8 weights in both orientations, the scales. */
typedef struct fxp_conv_saved {
    int8_t* Xq;   /* [N,H,W,C] */
    int8_t* Wq;   /* [Cout, KH*KW*C] */
    int8_t* WqT;  /* [KH*KW*C, Cout] */
    int8_t* WqF;  /* [C, KH*KW*Cout]: kernel flipped in both spatial axes; scratch of the backward call, which
                     fills it from WqT when it computes the input gradient of a stride-1 convolution */
    int32_t* eX;  /* 1 */
    int32_t* eW;  /* 1 */
} fxp_conv_saved;

/* Scratch bytes of fxp_conv2d_fwd (backward = 0) or fxp_conv2d_bwd (backward = 1); 0 on a bad shape. */
size_t fxp_conv2d_workspace_bytes(const fxp_conv2d_shape* shape, int backward);

/* Forward: the activation tensor is mapped once as a whole (element index = its channels-last flat index,
 * FXP_TAG_X), the weights likewise (FXP_TAG_W); the int8 patches are multiplied on the matrix cores - read
 * straight from the int8 activation when C is a multiple of 64 (by the GEMM loader, save for a few long contractions) or
 * at most 4 (filter rows of up to 32 bytes, up to 128 output channels), gathered into scratch first otherwise (a 1x1 layer's
 * patches are the activation itself) - and Y receives the inverse-mapped fp32 result.  Contractions KH*KW*C and KH*KW*Cout <= 133144. */
int fxp_conv2d_fwd(const float* X, const float* W, const fxp_conv2d_shape* shape, float* Y, const fxp_conv_saved* saved,
                   uint64_t seed, uint64_t step, int rounding, int bits, void* ws, size_t ws_bytes, void* stream);

/* Backward: dY is mapped once (FXP_TAG_DY); dW[Cout,KH,KW,C] sums over all N*Ho*Wo output pixels (any number: beyond
 * 133144 the sum runs as int32 slices added in 64 bits, like the long contractions of fxp_gemm_unmap),
 * dX[N,H,W,C] sums, per input pixel, the patch entries that read it (exact int32, then one inverse mapping).
 * dX or dW may be NULL.  dYq [N*Ho*Wo, Cout], dYqT [Cout, N*Ho*Wo] and e_dY are caller-allocated. */
int fxp_conv2d_bwd(const float* dY, const fxp_conv_saved* saved, const fxp_conv2d_shape* shape, float* dX, float* dW,
                   int8_t* dYq, int8_t* dYqT, int32_t* e_dY, uint64_t seed, uint64_t step, int rounding, int bits,
                   void* ws, size_t ws_bytes, void* stream);

/* ---- serving: a paged cache of mapped keys and values, attention over it, products with 4-bit weights ----
 * The mapping of Sec. 3.1 with one scale per BLOCK instead of one per tensor, rounded to nearest (FXP_ROUND_NEAREST: a
 * cache is written once and read many times, and a served answer does not depend on a seed). */

/* Element types of the tensors that these calls read and write. */
enum { FXP_F32 = 0, FXP_BF16 = 1, FXP_F16 = 2 };

/* Tokens of a page: the cache's block, and the contraction of one int8 matrix instruction. */
#define FXP_KV_PAGE 64

/* A cache of one layer (host struct of device pointers, caller-allocated, 16-byte aligned).  A block is the
 * FXP_KV_PAGE tokens of one page and one head; it has one scale for its keys and one for its values.
 *   kq [pages, heads, 64, dim]       keys, a token's row contiguous
 *   vq [pages, heads, 4, dim, 16]    values in four groups of 16 tokens, each group transposed: what a contraction over
 *                                    tokens reads without moving a byte, and a new token touches a quarter of the block
 *   ek, ev [pages, heads]            int32 scales
 * dim: a multiple of 16, at most 256.  pages < 2^31, heads <= 65535.  bits: width of the mantissas, 2..8 (stored as
 * int8 whatever the width).  A block's bytes behind its last token are never interpreted; a cache needs no clearing. */
typedef struct fxp_kv_cache {
    int8_t* kq;
    int8_t* vq;
    int32_t* ek;
    int32_t* ev;
    int64_t pages, heads, dim;
    int bits;
} fxp_kv_cache;

/* The tables of a step (host struct of device pointers, caller-allocated; slots 8-byte, runs 16-byte aligned, the others 4-byte).
 * Request b < requests holds lens[b] tokens, in ceil(lens[b] / 64) pages whose numbers are the first entries of
 * its row of block_table [requests, blocks].  free_pages [pages] is a stack of n_free[0] pages nobody holds.
 * requests, tokens, pages, blocks * 64 < 2^31.  All a step's calls read the same struct; every layer's cache shares it. */
typedef struct fxp_kv_step {
    int64_t requests, blocks, tokens, pages;
    const int32_t* lens;       /* [requests] */
    const int32_t* free_pages; /* [pages] */
    const int32_t* n_free;     /* [1] */
    int32_t* block_table;      /* [requests, blocks]: the pages taken are entered */
    int32_t* lens_after;       /* [requests]; may be lens */
    int32_t* n_free_after;     /* [1]; may be n_free */
    int32_t* first;            /* [requests + 1]: first new token of each request, and their number */
    int64_t* slots;            /* [tokens]: page * 64 + place in it of each new token, -1 where it has none */
    int32_t* positions;        /* [tokens]: place of each new token in its request, -1 behind the last one */
    int32_t* runs;             /* [fxp_kv_max_runs(requests, tokens), 4]: (first token, count, page, offset) of the new
                                  tokens that share a page; (0, 0, -1, 0) behind the last run */
    int32_t* refused;          /* [requests]: 1 = the request's new tokens found no room */
} fxp_kv_step;

/* Most runs that `tokens` new tokens of `requests` requests can fall into; 0 on bad arguments. */
int64_t fxp_kv_max_runs(int64_t requests, int64_t tokens);

/* Makes room for n_new[b] (device, >= 0) more tokens of each request and fills the tables of the step.  Pages are
 * taken from the top of the stack in the order of the requests.  A request that would outgrow its row of
 * block_table is refused; so is, from the first one that the stack cannot serve on, every request that needs a page, and from the first one
 * whose tokens pass `tokens` on, every request that has any.
 * A refused request keeps its length and its row, its tokens get slot -1 and runs on page -1 (fxp_kv_append skips them).
 * Pages are counted by lengths: a caller that lowers one pushes the pages behind the first ceil(length / 64) of the row on the stack itself.
 * Tokens and runs beyond `tokens` and the runs' capacity are not written, but counted in first (up to 2^31 - 1, which also stands for all
 * beyond).  Lengths that are negative count as 0.
 * ws: NULL, or at least 256 bytes, zero before the first call that uses them, which every call leaves zero; required where
 * lens_after or n_free_after is the input itself. */
int fxp_kv_tables(const fxp_kv_step* step, const int32_t* n_new, void* ws, size_t ws_bytes, void* stream);

/* Maps new tokens into the cache.  k, v: `tokens` rows of heads x dim elements of `type`, token t and head h at
 * t * k_token + h * k_head elements (any strides >= 0; fastest where base and strides are multiples of four elements).
 * runs [n_runs < 2^24, 4], 16-byte aligned: see fxp_kv_step; pages must differ, as those of fxp_kv_tables do.
 * A block's scale is the largest exponent of the values it holds: where a new token raises it, the tokens
 * before it are brought to the new scale (magnitude shifted right, rounded half up).  A run at offset 0 begins the block
 * anew.  A run whose tokens, page or places do not exist is skipped.  Non-finite values: see the top of this file. */
int fxp_kv_append(const fxp_kv_cache* cache, int type, const void* k, int64_t k_token, int64_t k_head, const void* v,
                  int64_t v_token, int64_t v_head, int64_t tokens, const int32_t* runs, int64_t n_runs, void* stream);

/* The inverse mapping of cached tokens: row t of k, v [tokens, heads, dim] of `type` receives the values that the
 * token stands for, rounded once (exact in fp32 and bf16 but for overflow and underflow).  runs as above: the tokens
 * at places offset .. offset + count - 1 of a page go to rows first ..; rows of no run are left as they are.  k and v share no elements. */
int fxp_kv_load(const fxp_kv_cache* cache, int type, void* k, void* v, int64_t tokens, const int32_t* runs, int64_t n_runs,
                void* stream);

/* Attention of new tokens over the cache (the paper's int8 attention products with the softmax in floating point,
 * Sec. 5).  Request b has step->first[b+1] - step->first[b] rows of q, which are its last ones (rows of a refused request, whose tokens
 * are not in the cache, are to be dropped): row i of n stands at place lens_after[b] - n + i and sees the tokens at and before it;
 * with window > 0 only the `window` last of them.
 * out = sum_j softmax_j(scale * q . k_j) v_j with k, v the values that the cache stands for.  Head h of q reads head
 * h / (q_heads / heads) of the cache; q_heads is a multiple of heads, at most 16384.  q and out: [tokens, q_heads, dim] of `type`, strides
 * as in fxp_kv_append; out may be q (with q's strides) and shares no elements with it otherwise, and its rows may not overlap; rows behind
 * the last request's are left as they are.  A row that sees nothing (no cached
 * token; all of its pages missing) gives zeros and lse -Inf.  Of *step only requests, blocks, tokens, first,
 * lens_after and block_table are used; firsts beyond `tokens` count as `tokens`, tokens on a page outside [0, pages) are not seen.
 * lse: NULL, or [tokens, q_heads] fp32 receiving log sum_j exp(scale * q . k_j).
 * Arithmetic: rows of q and the weights of 64 tokens are fixed-point numbers of two signed 8-bit digits (three for fp32: 23
 * bits) under a scale of their own, products are exact int32 sums over 64 terms, sums over more and the
 * softmax are fp32.  Outputs are divided by the sum of the weights as rounded, so that they are weighted means of the values; lse has that of
 * the weights as they are.  0 < scale < 2^64.  Scores are taken to lie below 2^89 in magnitude, and
 * values times the number of tokens that a row sees below 2^119 (beyond that outputs may be Inf or NaN).
 * step->first must not decrease.  Sizes whose tiles of 16 rows times their pages (all requests as long as blocks allows) pass 2^31 a call are refused.
 * ws: fxp_kv_attention_workspace_bytes bytes (0 on bad arguments), 256-byte aligned, of which the first FXP_KV_TICKET_BYTES are zero
 * before the first call that uses them; every call leaves them zero.  Calls of any sizes may take turns with one workspace; two at
 * once may not share it. */
#define FXP_KV_TICKET_BYTES 2048
size_t fxp_kv_attention_workspace_bytes(int64_t requests, int64_t tokens, int64_t q_heads, int64_t heads, int64_t dim);
int fxp_kv_attention(const fxp_kv_cache* cache, const fxp_kv_step* step, int type, const void* q, int64_t q_token, int64_t q_head,
                     int64_t q_heads, float scale, int64_t window, void* out, int64_t out_token, int64_t out_head, float* lse,
                     void* ws, size_t ws_bytes, void* stream);

/* ---- rotary positions ----
 * Pair i < rot / 2 of a head's elements stands for a point of the plane that is turned by position * f_i and stretched by `amplitude`:
 * (u, w) -> amplitude * (u cos - w sin, u sin + w cos).  Pairs are elements 2 i and 2 i + 1 (interleaved) or i and i + rot / 2; elements from rot
 * on stay as they are.  turns[i] is f_i as a fraction of a turn in units of 2^-64, modulo one turn: its product with a 31-bit position, modulo one turn, is
 * the angle to 2^-34 turns.  fxp_rotary and the writer's queries take the 32 top bits of it (to 2^-32 turns), the writer's keys all.  Host struct; rot
 * even, 2 .. min(dim, FXP_ROTARY_MOST), 2^-126 <= amplitude < 1e30; turns [rot / 2] on the device, 8-byte aligned. */
#define FXP_ROTARY_MOST 1024
#define FXP_ROTARY_ZERO 0x100       /* of fxp_rotary's `backward` */
typedef struct fxp_rotation {
    const uint64_t* turns;
    int64_t rot;
    int interleaved;
    double amplitude;
} fxp_rotation;

/* y = x turned by its positions, or with `backward` by the opposite angles (and stretched alike): the gradient of that.  x and y: [batch, tokens,
 * heads, dim] of `type` at any strides >= 0 of the first three (fastest where bases, strides, rot / 2 and dim - rot are multiples of 16 bytes);
 * positions: int32, sequence b's at p_batch * b (0: the same for all).  Rows at negative positions are left as they are in y; with FXP_ROTARY_ZERO
 * added to `backward` (0 or 1) they become zeros, every element of them.  y may be x (with x's strides) and shares no elements with it otherwise; y's
 * rows may not overlap.  Cosines and sums are fp32, rounded once to `type`.
 * heads <= 65535, dim <= 65536; fewer than 2^24 workgroups (of at least one token of one sequence, some 16 KiB of x where a sequence has them). */
int fxp_rotary(const fxp_rotation* rotation, int backward, int type, int64_t batch, int64_t tokens, int64_t heads, int64_t dim,
               const void* x, int64_t x_batch, int64_t x_token, int64_t x_head, const int32_t* positions, int64_t p_batch, void* y,
               int64_t y_batch, int64_t y_token, int64_t y_head, void* stream);

/* fxp_kv_append of keys that are turned on the way, and in the same launch the step's queries (q NULL: none): of *step only requests, tokens, runs
 * and positions are used (a run's token t stands at positions[t]).  A turned key is not rounded before it is mapped: rotation and rounding are
 * done in 64 bits.  Values are mapped as fxp_kv_append does.  q, out: [tokens, q_heads, dim] of `type`, q_heads a multiple of the cache's heads, at
 * most 16384; out receives the turned queries of every token of a run that is written (rows of others are left as they are), may be
 * q (with q's strides) and shares no elements with q otherwise, or with k or v; its rows may not overlap.  Inf and NaN spread to their pair. */
int fxp_kv_append_rotary(const fxp_kv_cache* cache, const fxp_kv_step* step, const fxp_rotation* rotation, int type, const void* k,
                         int64_t k_token, int64_t k_head, const void* v, int64_t v_token, int64_t v_head, const void* q, int64_t q_token,
                         int64_t q_head, int64_t q_heads, void* out, int64_t out_token, int64_t out_head, void* stream);

/* ---- products of a few rows with 4-bit weights ----
 * A weight matrix W [K, N] as mantissas -7..7 (the mapping with bits = 4, rounded to nearest) with one scale for
 * each group of `group` (32, 64 or 128) inputs of one output.  Packed layout, made once: tiles of 16 outputs x 128 inputs,
 * [ceil(N / 16), ceil(K / 128)] tiles of 1024 bytes.  With S = min(group, 64) and k counted in the tile, output r of
 * the tile and input k are in piece 16 * ((k % S) / (S / 4)) + r of 16 bytes, byte (k / S) * (S / 8) + k % (S / 8) of it, low
 * half if (k % (S / 4)) < S / 8, else the high half, in two's complement.  scales: uint8 biased exponents, 1 .. 254,
 * [ceil(N / 16), ceil(K / 128) * 128 / group, 16].  Inputs and outputs past K and N are zero.
 * K <= 2^20, N <= 2^24, M < 2^20; ceil128(K) * M <= 2^34. */
size_t fxp_w4_packed_bytes(int64_t K, int64_t N);
size_t fxp_w4_scale_bytes(int64_t K, int64_t N, int group);
/* W: K rows of N elements of `type`, row stride ldw >= N.  packed 16-byte, scales 4-byte aligned. */
int fxp_w4_pack(int type, const void* W, int64_t ldw, int64_t K, int64_t N, int group, uint8_t* packed, uint8_t* scales, void* stream);
/* Y[M,N] = X[M,K] * W.  X, Y of `type`, row strides ldx >= K, ldy >= N.  Made for few rows (one pass over the weights for each 32 to 64 of
 * them); any M is right.  A group of a row of X is a fixed-point number of two signed 8-bit digits (three for fp32)
 * under its own scale: products are exact int32 sums over a group, sums over groups fp32.  Y must not overlap X.
 * ws: fxp_w4_workspace_bytes bytes (0 on bad arguments), 256-byte aligned; not used, and may be NULL, for M <= 2. */
size_t fxp_w4_workspace_bytes(int type, int64_t M, int64_t K, int group);
int fxp_w4_linear(int type, const void* X, int64_t ldx, int64_t M, int64_t K, int64_t N, const uint8_t* packed, const uint8_t* scales,
                  int group, void* Y, int64_t ldy, void* ws, size_t ws_bytes, void* stream);

/* ---- products in microscaled 4-bit floating point ----
 * A mapped matrix [rows, cols] for products that contract over its columns: 32 elements of a row (a block) are 4-bit floats under one power of two,
 * the smallest under which the largest of them is at most 6 - the method's shared exponent, for 32 elements in place of a tensor.  A code is a sign (8)
 * and the place of a magnitude in 0, 0.5, 1, 1.5, 2, 3, 4, 6; a scale byte s stands for 2^(s - 127), 0 <= s <= 253.  A block with Inf or NaN has s = 255 and
 * is NaN, every element of it, in products too.  Panels of 256 columns, [ceil(cols / 256), rows, 128] bytes, even elements in the low halves; scales
 * [ceil(cols / 256), rows, 8], of the panel's blocks 0, 2, 4, 6, 1, 3, 5, 7.  Codes and scales behind the last column are zeros.
 * Host struct of device pointers; data 16-byte, scales 8-byte aligned; rows, cols <= 2^24 - 2^16. */
typedef struct fxp_mx4 {
    uint8_t* data;
    uint8_t* scales;
    int64_t rows, cols;
} fxp_mx4;
size_t fxp_mx4_data_bytes(int64_t rows, int64_t cols);  /* 0 on bad arguments */
size_t fxp_mx4_scale_bytes(int64_t rows, int64_t cols);

/* Maps x [rows, cols] of `type`, row stride ldx >= cols: q [rows, cols] with blocks along the rows and / or qT [cols, rows], x transposed, with blocks
 * along x's columns (either may be NULL), in one pass.  rounding: FXP_ROUND_NEAREST is to nearest, ties to even; FXP_ROUND_STOCHASTIC up with the
 * probability of what is cut off, in units of 2^-22: where the top 22 bits of the element's random word are less than the top 22 bits behind the code.
 * Words as in fxp_map: element i of x (row-major, without gaps) has word i % 4 of Philox block i / 4, in both copies.  Fewer than 2^24 tiles of 32 x 256
 * elements; q, qT and x share no memory (FXP_ERR_VALUE). */
int fxp_mx4_map(int type, const void* x, int64_t ldx, int64_t rows, int64_t cols, const fxp_mx4* q, const fxp_mx4* qT, uint64_t seed,
                uint64_t stream_id, int rounding, void* stream);
/* The values [rows, cols] that q stands for, rounded once to `type` (exact in fp32; in bf16 but for underflow).  y shares no memory with q (FXP_ERR_VALUE). */
int fxp_mx4_unmap(const fxp_mx4* q, int type, void* y, int64_t ldy, void* stream);

/* C[M,N] of `type` = A B^T for mapped A [M,K] and B [N,K], row stride ldc >= N: products are exact, sums fp32 in no stated order (the same order on every call
 * of a size), rounded once to `type`.  Fewer than 2^22 tiles of 64 x 64 to 256 x 256 outputs.  C shares no memory with A and B (FXP_ERR_VALUE).  ws: fxp_mx4_gemm_workspace_bytes bytes (may be 0), 256-byte aligned. */
size_t fxp_mx4_gemm_workspace_bytes(int64_t M, int64_t N, int64_t K);
int fxp_mx4_gemm(const fxp_mx4* A, const fxp_mx4* B, int type, void* C, int64_t ldc, void* ws, size_t ws_bytes, void* stream);

/* Y[M,N] = X[M,K] W of `type`, W = [N,K] mapped (W^T with blocks along the contraction: fxp_mx4_map's qT of W[K,N]); X is mapped to nearest on the way.  Row strides
 * ldx >= K, ldy >= N.  Any M, one row to many.  Y must not overlap X, and shares no memory with W (FXP_ERR_VALUE).  ws: fxp_mx4_linear_workspace_bytes bytes (0, and NULL allowed, for M <= 4), 256-byte aligned. */
size_t fxp_mx4_linear_workspace_bytes(int64_t M, int64_t N, int64_t K);
int fxp_mx4_linear(int type, const void* X, int64_t ldx, int64_t M, const fxp_mx4* W, void* Y, int64_t ldy, void* ws, size_t ws_bytes, void* stream);

/* A layer's training step, as fxp_linear_fwd / _bwd with blocks of 4-bit floats in place of int8 tensors: Y = X W, dX = dY W^T, dW = X^T dY, dense
 * row-major of one `type`, every operand mapped along the contraction that it is used in (the same random words in both copies).  The mapped operands belong to the
 * caller: fwd fills X [M,K], WT [N,K], XT [K,M] and W [K,N] (the last two may have data NULL where no backward call follows), bwd reads XT for dW and W for dX, and
 * fills dY [M,N] for dX and dYT [N,M] for dW.  dX or dW may be NULL.  The mapped operands of a call share no memory
 * with each other or with its dense matrices, nor does dX with dW (FXP_ERR_VALUE); Y may lie over X or W, dX and dW over dY, which are mapped before.  Streams: (step << 8) | 0, 1, 2 for X, W, dY; step < 2^56.
 * ws: fxp_mx4_layer_workspace_bytes bytes (at least 256), 256-byte aligned. */
typedef struct fxp_mx4_layer {
    fxp_mx4 X, XT, W, WT, dY, dYT;
} fxp_mx4_layer;
size_t fxp_mx4_layer_workspace_bytes(int64_t M, int64_t K, int64_t N);
int fxp_mx4_linear_fwd(int type, const void* X, const void* W, int64_t M, int64_t K, int64_t N, void* Y, const fxp_mx4_layer* layer, uint64_t seed, uint64_t step,
                       int rounding, void* ws, size_t ws_bytes, void* stream);
int fxp_mx4_linear_bwd(int type, const void* dY, const fxp_mx4_layer* layer, int64_t M, int64_t K, int64_t N, void* dX, void* dW, uint64_t seed, uint64_t step,
                       int rounding, void* ws, size_t ws_bytes, void* stream);

/* ---- measurement helper (not a step of the method) ----
 * Core clock while other work runs: enqueues one wave on `stream` (use a stream of its own, next to the kernels
 * under test) that stays alive for `microseconds` (1 .. 1000000) of the constant 100 MHz counter and then writes
 * out[0] = ticks of that counter, out[1] = core clock cycles in the same interval (device, 2 x uint64, 8-byte
 * aligned): core clock in MHz = 100 * out[1] / out[0].  The compute-bound products of Sec. 3.3 run the chip
 * into its power limit, so their rate is reported next to the clock they ran at. */
int fxp_clock_probe(uint64_t* out, uint32_t microseconds, void* stream);

/* Time stamps inside the linear-layer calls.  After fxp_timeline_begin(capacity) (host call; creates `capacity`
 * HIP events, 1 .. 2^20) every fxp_linear_fwd / fxp_linear_bwd records one event on its stream at its entry
 * (FXP_TL_ENTRY) and one after each of its launches, tagged with what the launch was, until the events are used
 * up.  fxp_timeline_end waits for the last recorded event and returns, for every pair of consecutive events, the
 * elapsed microseconds and the tag of the later one (so an interval is the in-stream duration of that launch
 * behind the launch that really precedes it in the step; an FXP_TL_ENTRY interval is the idle time between two
 * calls); *count receives the number of intervals written (at most `capacity`).  Then the events are destroyed.
 * The two gradients of a small or medium layer go out in one launch, FXP_TL_GEMM_GRADS in place of _DW and _DX; a small
 * layer's scales are found in its map launches, and their FXP_TL_SCALE intervals hold no launch, only the gap before it.
 * One timeline per process; not to be begun or ended while layer calls are running in other threads. */
enum { FXP_TL_ENTRY = 0, FXP_TL_SCALE = 1, FXP_TL_MAP = 2, FXP_TL_GEMM_FWD = 3, FXP_TL_GEMM_DW = 4, FXP_TL_GEMM_DX = 5,
       FXP_TL_REDUCE = 6, FXP_TL_GEMM_GRADS = 7 };
int fxp_timeline_begin(int capacity);
int fxp_timeline_end(float* microseconds, int* tags, int capacity, int* count);

#ifdef __cplusplus
}
#endif
#endif /* FXP_H_ */
