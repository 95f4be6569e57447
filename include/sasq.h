/*
 * sasq.h -- C ABI of the SASQ hot-path library for AMD MI355X (gfx950).
 *
 * SASQ (Static Activation Scaling for Quantization-aware training) trains nothing but the
 * activation quantization factors of an LLM's linear layers and then runs those layers with
 * the trained factors held fixed.  This library is the data-parallel hot path of that method:
 *
 *   training:   x' = fakequant(x; s)                     sasq_fakequant_fwd
 *               dx, ds = backward(x, dy; s)              sasq_fakequant_bwd
 *               s <- s - lr * ds                         sasq_scale_sgd
 *               the same with a byte in x's place    sasq_fakequant_fwd_ckpt, sasq_fakequant_bwd_ckpt
 *               loss, dx at the frozen output head       sasq_linear_ce
 *   inference:  Y = s * (q(X) . Wq^T) * s_w (+ bias)     sasq_static_linear
 *   set-up:     Wq, s_w from frozen fp32 weights         sasq_quantize_weight
 *               s0 = max|X| / (2^(bits-1) - 1)           sasq_absmax_scale
 *   serving:    between the linears q/k/v and o of an attention block, on a paged key/value cache:
 *               rotate by position, append           sasq_kv_append
 *               out = softmax(scale q k^T) v             sasq_paged_attention
 *
 * Conventions shared by every entry point
 *   - Every data pointer is DEVICE memory owned by the caller (the library never allocates,
 *     frees or keeps a pointer).  Scalars that are trained or produced on the device (s, ds)
 *     are device pointers too, so a training step needs no host synchronisation.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  Calls only
 *     enqueue work on that stream and return; outputs are valid once the stream has drained.
 *   - Matrices are dense row-major.  An activation matrix is [tokens, channels] (Sec. 2, Fig. 2).
 *   - 16-bit tensors are IEEE binary16 (SASQ_F16) or bfloat16 (SASQ_BF16).
 *   - Base pointers of 16-bit and weight tensors must be 16-byte aligned (SASQ_ERR_ALIGN).
 *   - Return value: a sasq_status.  Arguments are validated on the host before anything is
 *     launched; on error nothing has been enqueued.  The library never throws or aborts.
 *   - NOT validated (device-resident, checking would need a sync): *s finite and non-zero,
 *     inputs free of NaN.  Behaviour for such values is unspecified (but in-bounds).
 *   - Workspaces come from sasq_workspace_init(): a workspace is caller-owned device memory
 *     that must have been passed ONCE to sasq_workspace_init before its first use, may be reused
 *     by any number of later calls, and must not be used by two calls that can overlap in time.
 *     Its first 1024 bytes are control words that the reductions (sasq_absmax_scale, sasq_fakequant_bwd and its
 *     per-channel and batch forms) find zero and leave zero.  The linears and sasq_paged_attention may write over all
 *     of theirs: give them a workspace of their own, or initialise it again before a reduction uses it.
 *   - Graph capture: an entry point only launches kernels on the caller's stream (no allocation,
 *     no copy, no memset, no synchronisation), so calls may be recorded into a HIP graph and
 *     replayed; items arrays and other host arguments are read before the call returns.
 *
 * Numerical contract (the paper gives real-number formulas; these make them bit-level)
 *   - round(x/s) is round-half-to-even of the exact product x * inv_s, inv_s = fl32(1/s).
 *   - the straight-through clamp indicator is taken on the rounded value, bounds inclusive.
 *   - dequantisation is one fp32 multiply then one round-to-nearest-even to the 16-bit type.
 */
#ifndef SASQ_H
#define SASQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    SASQ_OK = 0,
    SASQ_ERR_NULL = 1,         /* a required pointer is NULL                               */
    SASQ_ERR_SHAPE = 2,        /* a size is <= 0, too large, or violates a stated multiple */
    SASQ_ERR_ALIGN = 3,        /* a base pointer is not 16-byte aligned                    */
    SASQ_ERR_UNSUPPORTED = 4,  /* unknown enum value or bits outside [2, 8]                */
    SASQ_ERR_WORKSPACE = 5,    /* workspace NULL or smaller than the matching query        */
    SASQ_ERR_LAUNCH = 6        /* the HIP runtime reported an error at launch              */
} sasq_status;

typedef enum { SASQ_F16 = 0, SASQ_BF16 = 1 } sasq_dtype;            /* activation / output type */
typedef enum {                       /* frozen weight storage                                    */
    SASQ_W_INT8 = 0,                 /* [N, K] int8, row-major                                   */
    SASQ_W_INT4_PACKED = 1,          /* [N, K/2] bytes, row-major, two codes per byte            */
    SASQ_W_INT8_BLOCKED = 2,         /* output of sasq_pack_weight from SASQ_W_INT8              */
    SASQ_W_INT4_BLOCKED = 3          /* output of sasq_pack_weight from SASQ_W_INT4_PACKED       */
} sasq_wfmt;

#define SASQ_MAX_BATCH 8                 /* tensors / projections per batched call                  */

/* Human-readable name of a status code (static storage, host pointer). */
const char* sasq_status_string(int status);

/* Library version as major*10000 + minor*100 + patch. */
int sasq_version(void);

/*
 * Test and tuning aid, not part of the method: force one of the library's kernel variants instead
 * of the choice the library makes from the shapes.  Every variant of a call computes the same
 * results bit for bit; the parity tests use this to cover each of them, the benchmark to compare
 * them.  The setting is process-wide and not thread-safe; value 0 restores the library's choice.
 * Unknown knob or value: SASQ_ERR_UNSUPPORTED.  The library reads no environment variables.
 */
typedef enum {
    SASQ_TUNE_LINEAR_PATH = 0,   /* 1: separate activation-quantize pass, 2: quantize on load          */
    SASQ_TUNE_LINEAR_TILE = 1,   /* 1: 256x256, 2: 128x256, 3: 128x128 workgroup tiles                  */
    SASQ_TUNE_LINEAR_MFMA = 2,   /* GEMMs: 1: the kernels on 32x32 MFMA tiles, 2: on 16x16 tiles (where they exist) */
    SASQ_TUNE_FQ_SHARE = 3,      /* 1..3: forward operators per group sharing one read of x, any size   */
    SASQ_TUNE_BWD_TILE = 4,      /* backward GEMM: 1: 256x256, 2: 128x128 tiles                         */
    SASQ_TUNE_COUNT = 5
} sasq_tune_knob;
int sasq_set_tuning(int knob, int value);

/*
 * Prepare a workspace for use by the calls below (zero-fills its control words, the first
 * 1024 bytes or the whole workspace if smaller, on `stream`).  Call once per workspace
 * allocation, before the first call that uses it.  Minimum size 256 bytes.
 */
int sasq_workspace_init(void* workspace, size_t workspace_bytes, void* stream);

/*
 * Fake quantization, forward (the operator Sec. 4.2 inserts before each linear; Sec. 3, Eq. 1;
 * dequantisation X' = S_x * X_int, Sec. 4.3, Eq. 5):
 *     q = clamp(round(x / s), -2^(bits-1), 2^(bits-1) - 1),   y = s * q.
 *   x      [rows, cols] device, 16-bit `dt`, read only
 *   s      device, one fp32: the per-tensor activation quantization factor
 *   y      [rows, cols] device, 16-bit `dt`, written (may alias x)
 *   codes  [rows, cols] device int8 or NULL: the integer codes q (for inspection and tests)
 *   bits   2..8
 */
int sasq_fakequant_fwd(const void* x, const float* s, void* y, int8_t* codes,
                       int64_t rows, int64_t cols, int bits, sasq_dtype dt, void* stream);

/* Bytes of workspace sasq_fakequant_bwd needs for this shape (pure function, host only). */
size_t sasq_fakequant_bwd_workspace(int64_t rows, int64_t cols);

/*
 * Fake quantization, backward with the straight-through estimator (Sec. 4.2, Eq. 4: the
 * gradient of round is 1, the gradient of clamp is 1 inside the range and 0 outside), and the
 * gradient of the scale, the only trained parameter (Sec. 4.2), by the chain rule:
 *     m  = 1 if -2^(bits-1) <= round(x/s) <= 2^(bits-1)-1 else 0
 *     dx = dy * m
 *     ds = sum over all elements of dy * (q - m * x/s)         (overwritten, not accumulated)
 *   x, dy  [rows, cols] device, 16-bit `dt`, read only
 *   s      device fp32 scalar
 *   dx     [rows, cols] device, 16-bit `dt`, written (may alias dy), or NULL to skip it
 *   ds     device fp32 scalar, written.  The reduction order is fixed: repeated calls with the
 *          same inputs give bit-identical results.
 *   workspace  >= sasq_fakequant_bwd_workspace(rows, cols) bytes, initialised once
 */
int sasq_fakequant_bwd(const void* x, const void* dy, const float* s, void* dx, float* ds,
                       int64_t rows, int64_t cols, int bits, sasq_dtype dt,
                       void* workspace, size_t workspace_bytes, void* stream);

/*
 * sasq_fakequant_bwd for callers that cannot allocate device memory or pass a workspace: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same inputs,
 * outputs, arithmetic and reduction order as sasq_fakequant_bwd (results are bit-identical); the
 * ticket word and the 256 fp64 block partials (3 KB) live in a device array that is part of the
 * library image instead of a caller workspace.  The call allocates nothing and frees nothing.
 *   - Each GPU holds one copy of that array for the life of the process; every call on a GPU uses
 *     it, so two calls that can overlap in time on one GPU (different streams) race: serialise them.
 *   - rows * cols above SASQ_FAKEQUANT_BWD_STATIC_MAX_ELEMENTS is rejected with SASQ_ERR_SHAPE.
 *   - The first call on a device looks the array's address up (no allocation); make that call
 *     outside graph capture.  A failed lookup returns SASQ_ERR_WORKSPACE.
 *   - Two kernels are enqueued: a one-thread clear of the ticket word, then the backward kernel (a small tensor's,
 *     up to 24583 elements, needs no ticket: one kernel, and the array is not touched).
 */
#define SASQ_FAKEQUANT_BWD_STATIC_MAX_ELEMENTS (INT64_C(1) << 40)
int sasq_fakequant_bwd_static(const void* x, const void* dy, const float* s, void* dx, float* ds,
                              int64_t rows, int64_t cols, int bits, sasq_dtype dt, void* stream);

/*
 * Per-channel variants of the fake-quant operator: one learned factor per activation channel
 * (column), the granularity of the paper's main experiments (Sec. 4; Sec. 5.1 "Implementation";
 * Sec. 2, Fig. 2(b)).  Same element arithmetic as above with s = s[k] for column k;
 *     ds[k] = sum over rows m of dy[m,k] * (q[m,k] - m[m,k] * x[m,k]/s[k])   (overwritten).
 *   s, ds   [cols] device fp32
 *   cols    at most 130560; the 128-bit path needs cols % 8 == 0, other widths take a slow
 *           one-thread-per-column kernel (and then need no workspace)
 * The per-channel backward uses one ticket per 512-column chunk of its workspace header; the
 * same workspace must not be shared with an overlapping call of any other entry point.
 */
int sasq_fakequant_fwd_pc(const void* x, const float* s, void* y, int8_t* codes,
                          int64_t rows, int64_t cols, int bits, sasq_dtype dt, void* stream);
size_t sasq_fakequant_bwd_pc_workspace(int64_t rows, int64_t cols);
int sasq_fakequant_bwd_pc(const void* x, const void* dy, const float* s, void* dx, float* ds,
                          int64_t rows, int64_t cols, int bits, sasq_dtype dt,
                          void* workspace, size_t workspace_bytes, void* stream);

/*
 * The fake-quant operators of several tensors in one launch (a decoder layer has seven, one in
 * front of each linear, Sec. 4.2; at LLaMA-2-7B sizes a separate launch per tensor spends a fifth
 * of its time ramping up and draining).  Element arithmetic, outputs and error rules are those of
 * sasq_fakequant_fwd / sasq_fakequant_bwd applied to each item; ds of an item is reduced in a
 * fixed order that depends on the batch's composition only (deterministic from run to run; it may
 * differ from the single-tensor call's ds in the last bits).
 *   items   HOST array of `count` descriptors (1 <= count <= SASQ_MAX_BATCH), read before the call
 *           returns; the pointers inside are device pointers with the meaning of the single calls:
 *           x, s always; out = y (forward, required) or dx (backward, may be NULL); dy and ds
 *           backward only.  Items must not overlap each other's outputs.
 *   workspace (backward)  >= sasq_fakequant_bwd_batch_workspace(count) bytes, initialised once
 *           with sasq_workspace_init; not shared with an overlapping call.
 * Forward items that name the same x (same pointer, same rows * cols; the operators in front of
 * q/k/v or of gate/up read one activation tensor, each with its own factor) may be run together, up
 * to three at a time, x being read from memory once for the group (large tensors only).  Outputs
 * are unchanged.
 */
typedef struct {
    const void* x;      /* [rows, cols] device, 16-bit `dt`                      */
    const void* dy;     /* backward: [rows, cols] device, 16-bit `dt`            */
    const float* s;     /* device fp32 scalar                                     */
    void* out;          /* forward: y; backward: dx or NULL                       */
    float* ds;          /* backward: device fp32 scalar, overwritten              */
    int64_t rows, cols;
} sasq_fq_item;
int sasq_fakequant_fwd_batch(const sasq_fq_item* items, int count, int bits, sasq_dtype dt, void* stream);
size_t sasq_fakequant_bwd_batch_workspace(int count);
int sasq_fakequant_bwd_batch(const sasq_fq_item* items, int count, int bits, sasq_dtype dt,
                             void* workspace, size_t workspace_bytes, void* stream);

/*
 * The same for per-channel factors (one factor per activation column, Sec. 4; Fig. 2(b)): each
 * item is a sasq_fakequant_fwd_pc / sasq_fakequant_bwd_pc call, `s` and `ds` pointing at `cols`
 * floats.  Outputs are bit-identical to the single-tensor calls (the column reduction of an item
 * does not depend on the batch).  Every item needs cols % 8 == 0 (SASQ_ERR_SHAPE otherwise: such
 * tensors take the single-tensor call), and the items of one backward call at most 256 column
 * blocks of 512 columns in all (SASQ_ERR_SHAPE; the workspace query then returns 0).
 *   workspace (backward)  >= sasq_fakequant_bwd_pc_batch_workspace(items, count) bytes, initialised
 *           once with sasq_workspace_init.
 */
int sasq_fakequant_fwd_pc_batch(const sasq_fq_item* items, int count, int bits, sasq_dtype dt, void* stream);
size_t sasq_fakequant_bwd_pc_batch_workspace(const sasq_fq_item* items, int count);
int sasq_fakequant_bwd_pc_batch(const sasq_fq_item* items, int count, int bits, sasq_dtype dt,
                                void* workspace, size_t workspace_bytes, void* stream);

/*
 * Fake quantization that keeps ONE BYTE an element for its backward: a scale-training step then holds [rows, cols] bytes per operator between
 * forward and backward, and x is free (y may overwrite it).  q, y, m and dx are those of sasq_fakequant_fwd / _bwd; with p = x / s as there,
 *     inside the range (m = 1):  e = fl32(q - p),  kept = round(252 e), in [-126, 126]           above it: kept = 127      below it: kept = -128
 *     dx = dy * m        ds = sum dy * v,   v = kept / 252 inside,  2^(bits-1) - 1 above,  -2^(bits-1) below
 * so that dx is that of the form which keeps x, and ds off from it by at most sum |dy| / 504 (the bytes' rounding, without bias).  The backward
 * reads neither x nor s.
 *   x, y, dy, dx   [rows, cols] device 16-bit `dt`;  y may alias x, dx may alias dy or be NULL (ds only)
 *   kept       [rows, cols] device int8, 16-byte aligned, written by the forward, read by the backward
 *   s, ds      device fp32: a scalar, or (pc) [cols];  ds is overwritten, its terms are summed in an order that follows from the sizes
 *   bits       2..8, the same in both directions;  cols (pc): any up to 2^24, multiples of 8 are fast
 *   workspace (backward)  >= the matching query's bytes, 16-byte aligned; needs no initialisation, and its control words stay as they are.  The
 *              query does not fall where tensors, rows or columns are added: a workspace for the largest batch serves smaller ones
 * The batch forms do up to SASQ_MAX_BATCH tensors in one launch, with the results of the single calls (pc: bit for bit; ds of a whole tensor may
 * differ in the last bits).  items: HOST array, read before the call returns; items must not overlap each other's outputs.
 */
typedef struct {
    const void* x;      /* forward                                                */
    const float* s;     /* forward                                                */
    void* out;          /* forward: y; backward: dx or NULL                       */
    int8_t* kept;       /* forward: written; backward: read                       */
    const void* dy;     /* backward                                               */
    float* ds;          /* backward, overwritten                                  */
    int64_t rows, cols;
} sasq_ckpt_item;
int sasq_fakequant_fwd_ckpt(const void* x, const float* s, void* y, int8_t* kept, int64_t rows, int64_t cols, int bits, sasq_dtype dt, void* stream);
size_t sasq_fakequant_bwd_ckpt_workspace(int64_t rows, int64_t cols);
int sasq_fakequant_bwd_ckpt(const int8_t* kept, const void* dy, void* dx, float* ds, int64_t rows, int64_t cols, int bits, sasq_dtype dt,
                            void* workspace, size_t workspace_bytes, void* stream);
int sasq_fakequant_fwd_pc_ckpt(const void* x, const float* s, void* y, int8_t* kept, int64_t rows, int64_t cols, int bits, sasq_dtype dt, void* stream);
size_t sasq_fakequant_bwd_pc_ckpt_workspace(int64_t rows, int64_t cols);
int sasq_fakequant_bwd_pc_ckpt(const int8_t* kept, const void* dy, void* dx, float* ds, int64_t rows, int64_t cols, int bits, sasq_dtype dt,
                               void* workspace, size_t workspace_bytes, void* stream);
int sasq_fakequant_fwd_ckpt_batch(const sasq_ckpt_item* items, int count, int bits, sasq_dtype dt, void* stream);
size_t sasq_fakequant_bwd_ckpt_batch_workspace(const sasq_ckpt_item* items, int count);
int sasq_fakequant_bwd_ckpt_batch(const sasq_ckpt_item* items, int count, int bits, sasq_dtype dt, void* workspace, size_t workspace_bytes, void* stream);
int sasq_fakequant_fwd_pc_ckpt_batch(const sasq_ckpt_item* items, int count, int bits, sasq_dtype dt, void* stream);
size_t sasq_fakequant_bwd_pc_ckpt_batch_workspace(const sasq_ckpt_item* items, int count);
int sasq_fakequant_bwd_pc_ckpt_batch(const sasq_ckpt_item* items, int count, int bits, sasq_dtype dt, void* workspace, size_t workspace_bytes, void* stream);

/* SGD step of sasq_scale_sgd on a vector of n scales (the scales of one layer in one launch). */
int sasq_scale_sgd_vec(float* s, const float* ds, int64_t n, float lr, void* stream);

/*
 * One plain SGD step on the scale (the optimiser state of SASQ is the scale alone, Sec. 4.2;
 * the paper's own runs use AdamW, Sec. 5.1):  *s = fl32(*s - fl32(lr * *ds)).
 */
int sasq_scale_sgd(float* s, const float* ds, float lr, void* stream);

/*
 * One AdamW step (decoupled weight decay) on a vector of n scales, the optimiser of the paper's
 * runs (Sec. 5.1: AdamW, learning rate 2e-4; the scales are the only parameters, Sec. 4.2):
 *     p <- p - lr*wd*p;  m <- b1*m + (1-b1)*g;  v <- b2*v + (1-b2)*g^2;
 *     p <- p - lr * (m/(1-b1^step)) / (sqrt(v/(1-b2^step)) + eps)
 *   s, ds, m, v  [n] device fp32 (m, v: first and second moment state, zero before step 1)
 *   step         1-based step count.  Hyper-parameters are doubles (1 - beta is formed in double);
 *                the update itself is fp32 arithmetic and agrees with an fp64 evaluation to ~1e-6 relative.
 */
int sasq_scale_adamw(float* s, const float* ds, float* m, float* v, int64_t n, int64_t step,
                     double lr, double beta1, double beta2, double eps, double weight_decay, void* stream);

/* Bytes of workspace sasq_static_linear needs (pure function, host only; may be 0). */
size_t sasq_static_linear_workspace(int64_t M, int64_t N, int64_t K, sasq_wfmt wf);

/*
 * Static-inference quantized linear (Sec. 3, Eq. 2: Y = S_x * (X_int . W_int) * S_w, integer
 * product first, inverse quantization after; bias not quantized).  The activation scale is a
 * fixed input: nothing is reduced over X at run time (static quantization, Sec. 3; Sec. 4.5).
 *     xq[m,k]  = clamp(round(X[m,k] / s), -2^(a_bits-1), 2^(a_bits-1) - 1)
 *     acc[m,n] = sum_k xq[m,k] * Wq[n,k]                      (exact, int32)
 *     Y[m,n]   = fl32(fl32(acc[m,n]) * fl32(s * s_w[n])) (+ bias[n])  -> 16-bit `dt`
 *   x        [M, K] device 16-bit `dt`
 *   s        device fp32 scalar
 *   wq       [N, K] device int8 (SASQ_W_INT8), or [N, K/2] bytes (SASQ_W_INT4_PACKED): element k
 *            even in the low nibble, k odd in the high nibble, two's complement, range [-8, 7];
 *            or the sasq_packed_weight_bytes(N, K, wf) bytes sasq_pack_weight made of either
 *            (SASQ_W_INT8_BLOCKED, SASQ_W_INT4_BLOCKED: same codes, same results bit for bit,
 *            arranged so that the GEMM reads them in whole cache lines; the fast path for
 *            frozen weights; K must be a multiple of 64, else SASQ_ERR_SHAPE)
 *   s_w      [N] device fp32, one factor per output channel
 *   bias     [N] device fp32 or NULL
 *   y        [M, N] device 16-bit `dt`, written
 *   acc_out  [M, N] device int32 or NULL; xq_out [M, K] device int8 or NULL (inspection/tests;
 *            requesting either selects a slower code path)
 *   K        multiple of 2 for int4.  Any M, N, K > 0 is accepted; K not a multiple of 64 takes
 *            a matrix-unit kernel that reads rows at any alignment.
 *   M*K, N*K, M*N must each be < 2^40; |acc| cannot overflow for K <= 131071.
 *   workspace  >= sasq_static_linear_workspace(M, N, K, wf) bytes (NULL allowed when that is 0);
 *              holds the int8 activation codes in a library-internal blocked order between the
 *              quantize pass and the GEMM; contents after the call are unspecified
 */
int sasq_static_linear(const void* x, const float* s, const void* wq, const float* s_w,
                       const float* bias, void* y, int32_t* acc_out, int8_t* xq_out,
                       int64_t M, int64_t N, int64_t K, int a_bits, sasq_wfmt wf, sasq_dtype dt,
                       void* workspace, size_t workspace_bytes, void* stream);

/*
 * The static linears of several projections (one decoder layer) in two launches: one activation
 * pre-pass and one GEMM over the tiles of all projections, longest K first, so that the layer pays
 * one launch ramp and one drain and the partly filled last round of a projection is filled by the
 * next one's tiles.  Arithmetic and results of each item are exactly those of sasq_static_linear.
 *   items   HOST array of `count` descriptors (1 <= count <= SASQ_MAX_BATCH), read before the call
 *           returns; pointers inside are device pointers as in sasq_static_linear (bias may be NULL).
 *           Every K must be a multiple of 64 (SASQ_ERR_SHAPE otherwise: use the single call).
 *   a_bits, wf, dt   shared by all items.  No inspection outputs.
 *   workspace >= sasq_static_linear_batch_workspace(items, count, wf) bytes.
 */
typedef struct {
    const void* x;        /* [M, K] device, 16-bit `dt`                 */
    const float* s;       /* device fp32 scalar                          */
    const void* wq;       /* weights in format `wf`                      */
    const float* s_w;     /* [N] device fp32                             */
    const float* bias;    /* [N] device fp32 or NULL                     */
    void* y;              /* [M, N] device, 16-bit `dt`, written         */
    int64_t M, N, K;
} sasq_linear_item;
size_t sasq_static_linear_batch_workspace(const sasq_linear_item* items, int count, sasq_wfmt wf);
int sasq_static_linear_batch(const sasq_linear_item* items, int count, int a_bits, sasq_wfmt wf,
                             sasq_dtype dt, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Static-inference quantized linear with one activation factor per group of `group` consecutive
 * input channels (Sec. 3, Eq. 3: Y = sum_i (S_x,i * S_w) * (X_int,i . W_int), the block-wise form
 * the paper gives for activations quantized per channel; Sec. 4 trains per-channel factors):
 *     xq[m,k]    = clamp(round(X[m,k] / s_g[k / group]), -2^(a_bits-1), 2^(a_bits-1) - 1)
 *     acc_i[m,n] = sum over the k of group i of xq[m,k] * Wq[n,k]          (exact, int32)
 *     f[m,n]     = fma(fl32(acc_i[m,n]), s_g[i], f[m,n]) for i = 0 .. K/group - 1, from f = 0
 *     Y[m,n]     = fl32(f[m,n] * s_w[n]) (+ bias[n])  -> 16-bit `dt`
 * (the paper fixes no rounding order for Eq. 3; this one is what the kernels and the test oracle
 * share.)  group = 1 is per-channel in the strict sense, group = K a per-tensor factor.
 *   s_g      [K / group] device fp32
 *   f_out    [M, N] device fp32 or NULL: f, for inspection and tests (slower path); xq_out as in
 *            sasq_static_linear
 *   group    divides K.  The MFMA path is taken when K and group are multiples of 64 (then all
 *            four weight formats are accepted), and for group = 32 with K a multiple of 64 and
 *            any format but row-major int4 (each 64-channel K tile is then multiplied twice, one
 *            half of the channels at a time); other shapes have kernels of their own (on the VALUs;
 *            groups of 2, 4, 8 and 16, and of 1 with more than a few rows, form their sums on the
 *            matrix units) and accept the row-major weight formats only (SASQ_ERR_SHAPE for the
 *            pre-arranged ones).
 *   every other argument, the workspace size and the limits are those of sasq_static_linear.
 */
int sasq_static_linear_grouped(const void* x, const float* s_g, const void* wq, const float* s_w,
                               const float* bias, void* y, float* f_out, int8_t* xq_out,
                               int64_t M, int64_t N, int64_t K, int64_t group, int a_bits,
                               sasq_wfmt wf, sasq_dtype dt, void* workspace, size_t workspace_bytes,
                               void* stream);

/*
 * Dynamic per-token quantized linear: the baseline whose online step the static factors remove
 * (Sec. 3: dynamic quantization computes the factors during inference, per-token = one factor per
 * row of X; Sec. 4.5 compares against it).  For every row m:
 *     s_m      = fl32(max_k |X[m,k]| / (2^(a_bits-1) - 1))      (1 if the row is all zero)
 *     xq[m,k]  = clamp(round(X[m,k] / s_m), -2^(a_bits-1), 2^(a_bits-1) - 1)
 *     acc[m,n] = sum_k xq[m,k] * Wq[n,k]                        (exact, int32)
 *     Y[m,n]   = fl32(fl32(acc[m,n]) * fl32(s_m * s_w[n])) (+ bias[n])  -> 16-bit `dt`
 *   x must be finite.  s_row_out [M] device fp32 or NULL: the factors (inspection, tests, or use as
 *   an absmax calibration pass).  acc_out, xq_out, wq, s_w, bias, y, shapes, weight formats
 *   and limits as in sasq_static_linear.
 *   workspace >= sasq_dynamic_linear_workspace(M, N, K, wf) bytes.
 */
size_t sasq_dynamic_linear_workspace(int64_t M, int64_t N, int64_t K, sasq_wfmt wf);
int sasq_dynamic_linear(const void* x, const void* wq, const float* s_w, const float* bias, void* y,
                        int32_t* acc_out, int8_t* xq_out, float* s_row_out,
                        int64_t M, int64_t N, int64_t K, int a_bits, sasq_wfmt wf, sasq_dtype dt,
                        void* workspace, size_t workspace_bytes, void* stream);

/*
 * Quantize frozen weights, symmetric, one factor per output channel (Sec. 3, Eq. 1 applied to
 * each row of W[N,K]; Sec. 5.1 fixes the weight granularity to per output channel):
 *     s_w[n]  = fl32(max_k |W[n,k]| / Qp)     (1 if the row is all zero),  Qp = 127 or 7
 *     Wq[n,k] = clamp(round(W[n,k] / s_w[n]), -Qp-1, Qp)     (same rounding rule as activations)
 *   w    [N, K] device fp32;  wq: [N, K] int8 or [N, K/2] packed int4 (K even);  s_w [N] fp32
 */
int sasq_quantize_weight(const float* w, void* wq, float* s_w, int64_t N, int64_t K,
                         sasq_wfmt wf, void* stream);

/*
 * Re-arrange quantized frozen weights for the GEMM (a set-up step, once per weight matrix; the
 * weights of static inference never change, Sec. 3).  A pure permutation of the codes:
 *   SASQ_W_INT8 -> SASQ_W_INT8_BLOCKED: 1 KB blocks of 16 rows x 64 K-bytes, block (n/16, k/64) at
 *     ((n/16) * K/64 + k/64) * 1024; inside, the 16-byte chunk c of row r at
 *     16 * (4r + (c ^ ((r >> 1) & 3) ^ ((r >> 3) & 1))).
 *   SASQ_W_INT4_PACKED -> SASQ_W_INT4_BLOCKED: 1 KB blocks of 32 rows x 64 k, block (n/32, k/64) at
 *     ((n/32) * K/64 + k/64) * 1024; the 16 codes k = 64*(k/64) + 32*kk + 16*g + (0..15) of row r
 *     are the 8 bytes at 512*kk + 256*g + 8*r: byte b of the first four holds code b (low nibble)
 *     and code 4+b (high nibble), byte b of the last four codes 8+b and 12+b.
 * Rows past N in the last block are zero.
 *   wq       device, row-major codes in format wf_src (SASQ_W_INT8 or SASQ_W_INT4_PACKED)
 *   packed   device, sasq_packed_weight_bytes(N, K, blocked format) bytes, written; not wq
 *   K        multiple of 64 (SASQ_ERR_SHAPE otherwise: use the row-major format for such shapes)
 * sasq_packed_weight_bytes is a pure host function; it returns 0 for shapes or formats that have
 * no blocked form.
 */
size_t sasq_packed_weight_bytes(int64_t N, int64_t K, sasq_wfmt wf);
int sasq_pack_weight(const void* wq, void* packed, int64_t N, int64_t K, sasq_wfmt wf_src, void* stream);

/*
 * Backward of the frozen quantized linear with respect to its input: the step that hands each
 * fake-quant operator its upstream gradient during scale training (Sec. 4.2; the weight is
 * Eq. 2's W_int * S_w, frozen):
 *     Wq[n,k] = round16(fl32(fl32(W_int[n,k]) * s_w[n]))        (prepared once)
 *     dX[m,k] = round16(sum_n dY[m,n] * Wq[n,k])                 (16-bit MFMA, fp32 accumulation)
 * The sum's rounding order is the matrix unit's: dX agrees with the exactly rounded result within
 * the fp32 accumulation bound N * 2^-24 * sum_n |dY[m,n] * Wq[n,k]| plus one 16-bit rounding.
 *
 * sasq_prepare_bwd_weight writes Wq transposed and cut into the GEMM's operand blocks:
 *   B[k][n] = Wq[n][k]; 1 KB blocks of 16 rows (k) x 32 columns (n), block (k/16, n/32) at
 *   ((k/16) * ceil(N/32) + n/32) * 1024; inside, the 16-byte chunk c (8 columns) of row r at
 *   16 * (4r + (c ^ ((r >> 1) & 3) ^ ((r >> 3) & 1))).  Rows past K and columns past N are zero.
 *   wq       device, row-major codes [N,K], SASQ_W_INT8 or SASQ_W_INT4_PACKED
 *   s_w      device, N floats
 *   wt       device, sasq_bwd_weight_bytes(N, K) bytes, 16-byte aligned, written
 *   N        any; the MFMA kernel runs when N is a multiple of 32, a scalar kernel otherwise
 * sasq_linear_bwd_input:
 *   dy       device, [M,N] row-major 16-bit, 16-byte aligned, read only
 *   wt       device, as prepared for the same N, K and dt
 *   dx       device, [M,K] row-major 16-bit, 16-byte aligned, written; must not alias dy
 *   acc_out  device, optional (NULL to skip): [M,K] floats, the fp32 sums before the 16-bit rounding
 * sasq_bwd_weight_bytes is a pure host function.
 */
size_t sasq_bwd_weight_bytes(int64_t N, int64_t K);
int sasq_prepare_bwd_weight(const void* wq, const float* s_w, void* wt, int64_t N, int64_t K,
                            sasq_wfmt wf, sasq_dtype dt, void* stream);
int sasq_linear_bwd_input(const void* dy, const void* wt, void* dx, float* acc_out,
                          int64_t M, int64_t N, int64_t K, sasq_dtype dt, void* stream);

/*
 * Cross entropy of a frozen output head, the loss of scale training and the measure of evaluation (Sec. 5: perplexity is exp of its mean), and
 * the gradient that the layers' backward starts from.  For row i of x with target t = targets[i] in [0, V):
 *     z[v] = sum_h x[i,h] W[v,h]      lse[i] = ln sum_v exp z[v]      loss[i] = lse[i] - z[t]      *mean = sum of loss / counted rows
 *     dx[i] = scale * g[i] * (sum_v p[v] W[v] - W[t])                  p[v] = exp(z[v] - lse[i])
 * with g[i] = row_weight[i], or 1 / counted rows (the gradient of the mean) where row_weight is NULL.  The logits are not stored: the vocabulary
 * goes by in pieces, and both products of a piece are done before the next.  The head is frozen and has no gradient.
 * A row whose target lies outside [0, V) is left out: loss = lse = 0, dx = 0, whatever its x holds; but for small calls no product is done for it.  No counted
 * row: *mean = 0.
 *   x          [T, H] device 16-bit `dt`, rows x_stride elements apart
 *   head       W as sasq_prepare_head laid it out with SASQ_HEAD_LOGITS;  head_grad: with SASQ_HEAD_GRAD, or NULL without dx
 *   targets    [T] device int32;  row_weight  [T] device fp32 or NULL;  scale: a factor on the gradient (loss scaling), 1 otherwise
 *   loss       [T] device fp32, written;  lse  [T] device fp32 or NULL, written;  mean  device fp32 scalar or NULL, written
 *   dx         [T, H] device 16-bit `dt`, rows dx_stride apart, written, or NULL: no gradient; may be x itself (with its stride)
 *   T at most 2^23, V 2^22, H 2^20;  any sizes, multiples of 64 of H cost nothing extra
 *   piece      columns of the vocabulary at a time, a multiple of 256, or 0: the library's choice
 *   workspace  >= sasq_linear_ce_workspace(T, V, H, dx != NULL, piece) bytes, 16-byte aligned; needs no initialisation, and its control words stay
 *              as they are
 *              It holds the counted rows of x, two numbers for every 64 columns of a piece and row (1.4 GB at most where the library chooses), and with
 *              the gradient a 16-bit exponential for every column of a piece (0.35 GB and 600 bytes a row at most where the library chooses) and the running
 *              sums, fp32 [rows, H] of T rows or of as many as fill the chip.  The query does not fall where T grows: a workspace for the longest
 *              batch serves shorter ones (of equal V, H, grad and piece).
 * Sums are fp32, those over a row's losses fp64; the exponentials that the gradient contracts with W are rounded to 16 bits, relative to the
 * largest of their row but for the target's, which is kept apart: rows whose target is all but certain lose nothing.  Results do not change from
 * run to run.  Logits must be finite and less than 2^24 in size, entries of a bf16 head less than 2^96.
 *
 * sasq_prepare_head lays W [V, H] (16-bit, rows w_stride elements apart) out for the two products, once for a head: 1 KB blocks of 16 rows x 32
 * columns as in sasq_prepare_bwd_weight, rows v and columns h (SASQ_HEAD_LOGITS), or rows h and columns v (SASQ_HEAD_GRAD), the columns padded to
 * 64 and the rows to 16 with zeros, an odd number of blocks for each 16 rows (the last may be unused).  sasq_head_bytes is a pure host function; 0 for sizes that are not supported.
 */
typedef enum { SASQ_HEAD_LOGITS = 0, SASQ_HEAD_GRAD = 1 } sasq_head_form;
size_t sasq_head_bytes(int64_t V, int64_t H, sasq_head_form form);
int sasq_prepare_head(const void* w, int64_t w_stride, void* head, int64_t V, int64_t H, sasq_head_form form, sasq_dtype dt, void* stream);
size_t sasq_linear_ce_workspace(int64_t T, int64_t V, int64_t H, int grad, int64_t piece);
int sasq_linear_ce(const void* x, int64_t x_stride, const void* head, const void* head_grad, const int32_t* targets,
                   const float* row_weight, float scale, float* loss, float* lse, float* mean, void* dx, int64_t dx_stride,
                   int64_t T, int64_t V, int64_t H, int64_t piece, sasq_dtype dt, void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of workspace sasq_absmax_scale needs (pure function, host only). */
size_t sasq_absmax_scale_workspace(int64_t rows, int64_t cols);

/*
 * Initial (post-training) scale of an activation tensor (Sec. 3, Eq. 1, right half; Sec. 4.1):
 *     *s = fl32(max|x| / (2^(bits-1) - 1)).
 * This is the dynamic-quantization reduction that static inference avoids; it is used once,
 * to initialise s before training.
 */
int sasq_absmax_scale(const void* x, float* s, int64_t rows, int64_t cols, int bits,
                      sasq_dtype dt, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Paged key/value cache of one attention block.  The cache is `pages` pages of `page_size` places; a place holds, for each of `heads`
 * kv heads, `dim` channels of a key in `k` and of a value in `v`.  Element (page, place, head, channel) lies at
 *     page * page_stride + place * token_stride + head * head_stride + channel                (elements; k and v alike),
 * so a cache may be stored [pages, heads, page_size, dim] or [pages, page_size, heads, dim], or be a part of a larger tensor.
 *   SASQ_KV_16    elements in the activations' 16-bit type
 *   SASQ_KV_INT8  int8 codes with a fixed factor for each kv head (static quantization, Sec. 3, applied to what is kept):
 *                 value = code * k_scale[head], code = clamp(round(x / k_scale[head]), -128, 127) of the 16-bit x (any finite
 *                 non-zero factor, negative allowed).
 *   page_size     a power of two, 16 to 65536;  dim: 64 or 128;  pages * page_size may pass 2^31 (all offsets are 64 bits)
 *   strides       at least dim, multiples of 16 bytes, token_stride at most 2^26 elements; k and v 16-byte aligned
 */
typedef enum { SASQ_KV_16 = 0, SASQ_KV_INT8 = 1 } sasq_kvfmt;
typedef struct {
    void* k;                /* device */
    void* v;                /* device */
    const float* k_scale;   /* [heads] device fp32; SASQ_KV_INT8 only */
    const float* v_scale;   /* [heads] device fp32; SASQ_KV_INT8 only */
    int64_t pages, page_size, heads, dim;
    int64_t page_stride, token_stride, head_stride;
    sasq_kvfmt fmt;
} sasq_kv_cache;

/*
 * The sequences of one step, shared by the calls of all layers.  Rows cu_q[b] .. cu_q[b+1]-1 of the `tokens` rows are the new tokens
 * of sequence b; kv_len[b] is the length of its cache with the new tokens in it, so new token i is at position
 * kv_len[b] - (cu_q[b+1] - cu_q[b]) + i.  Position j lies on page block_table[b][j / page_size], at place j % page_size.
 *   cu_q          [batch + 1] device int32, ascending from 0;  a sequence may have no new token
 *   kv_len        [batch] device int32;  block_table  [batch, max_pages] device int32
 *   tokens        rows of q, k, v and the outputs; rows from cu_q[batch] on belong to no sequence and are not touched
 *   max_q         at least the most new tokens that a sequence has (tokens will do); sasq_paged_attention leaves one with more out
 *   max_kv        at least the longest kv_len (max_pages * page_size will do): how far the work is split, not which keys count
 *   max_pages * page_size at most 2^30
 * What lies on the device is not validated but bounded: an entry of block_table outside [0, pages) is a page that is not there (its
 * keys do not count, tokens on it are not stored), as are positions past the table.
 */
typedef struct {
    const int32_t* cu_q;
    const int32_t* kv_len;
    const int32_t* block_table;
    int64_t batch, max_pages, tokens, max_q, max_kv;
} sasq_kv_batch;

/*
 * Append: rotate the new tokens' queries and keys by their positions and store keys and values in the cache.
 * With r = rot_dim, c = cos[row][j], s = sin[row][j], j < r/2, each head of q and k becomes (fp32, every product and sum rounded,
 * then one rounding to 16 bits; channels from r on unchanged)
 *     SASQ_ROPE_HALVES:  y[j]  = x[j] c - x[j + r/2] s      y[j + r/2] = x[j + r/2] c + x[j] s
 *     SASQ_ROPE_PAIRS:   y[2j] = x[2j] c - x[2j + 1] s      y[2j + 1]  = x[2j + 1] c + x[2j] s
 * and y of k, and v as it is, go to their place in the cache (SASQ_KV_INT8: their codes).
 *   q        [tokens, q_heads, dim] 16-bit `dt`, rows q_stride elements apart, or NULL with q_out: keys and values only
 *   k, v     [tokens, heads, dim] 16-bit `dt`, rows k_stride and v_stride apart (columns of one fused projection, for instance)
 *   q_out    [tokens, q_heads, dim] 16-bit `dt`, rows q_out_stride apart, written; may be q itself
 *   cos, sin [table_rows, rot_dim/2] device fp32, or both NULL: no rotation (rot_dim is then not read)
 *   positions  [tokens] device int32: the row of the table for each token, or NULL: the token's position in its cache.  A token
 *            whose row is not in the table is not stored, and its row of q_out is 0.
 *   rot_dim  a multiple of 16, at most dim;  q_heads a multiple of heads;  row strides: multiples of 8, at least a row's length
 *   k and v must not overlap the cache; the order in which tokens are stored does not matter (no two share a place).
 */
typedef enum { SASQ_ROPE_HALVES = 0, SASQ_ROPE_PAIRS = 1 } sasq_rope;
int sasq_kv_append(const void* q, const void* k, const void* v, void* q_out,
                   int64_t q_stride, int64_t k_stride, int64_t v_stride, int64_t q_out_stride, int64_t q_heads,
                   const float* cos, const float* sin, const int32_t* positions, int64_t table_rows, int64_t rot_dim, sasq_rope style,
                   const sasq_kv_cache* cache, const sasq_kv_batch* batch, sasq_dtype dt, void* stream);

/*
 * Causal attention of the new tokens over the paged cache, which holds their own keys and values already.  For the new token i of
 * sequence b at position p, head h, and the positions j <= p that are there:
 *     S[j] = scale * sum_d q[i,h,d] k[j,h',d]      P = softmax over j of S      out[i,h,d] = sum_j P[j] v[j,h',d]
 * with h' = h / (q_heads / heads).  Keys that are masked (later ones, places past kv_len, pages that are not there) do not count
 * whatever their places hold, infinities and NaN included.  A row without any key: out = 0, lse = -inf.
 *   q        [tokens, q_heads, dim] 16-bit `dt`, rows q_stride elements apart;  out: the same, rows out_stride apart, written;
 *            must not overlap q
 *   lse      [tokens, q_heads] device fp32 or NULL, written: ln sum_j exp S[j], with which results over parts of the keys are joined
 *   scale    above 0, at most 2^127;  tokens * q_heads under 2^31;  batch * heads at most 2^22 (up to 2^26 where max_kv makes few runs)
 * Sums, maxima and the softmax are fp32; probabilities are rounded to 16 bits before they multiply the values (with an int8 cache:
 * to fp16, which holds every code exactly; in fp16 one under 2^-32 of the row's largest is 0), and the output is rounded once.  The sums over d
 * and the scores may be any that fp32 holds.  Results do not change from run to run.
 *   workspace  >= sasq_paged_attention_workspace(...) bytes, 16-byte aligned (NULL allowed when that is 0), holds partial results of split sequences.
 *            The size is that of one combination of batch, tokens, max_q, max_kv, max_pages and heads, to be asked for each: keys are cut into
 *            as many runs as fill the chip, so a step of fewer sequences or tokens may need more than a larger one
 */
size_t sasq_paged_attention_workspace(const sasq_kv_cache* cache, const sasq_kv_batch* batch, int64_t q_heads);
int sasq_paged_attention(const void* q, void* out, float* lse, int64_t q_stride, int64_t out_stride, int64_t q_heads, float scale,
                         const sasq_kv_cache* cache, const sasq_kv_batch* batch, sasq_dtype dt,
                         void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SASQ_H */
