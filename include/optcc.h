/*
 * liboptcc -- low-rank power-iteration compressor with error feedback on one
 * AMD Instinct MI355X (gfx950).
 *
 * The compressor is the one Optimus-CC (arXiv 2301.09830) applies to
 * inter-stage activation gradients (Sec. 5, compressed backpropagation),
 * embedding gradients (Sec. 6) and data-parallel weight gradients (Sec. 7):
 * PowerSGD-style power iteration warm-started from the previous factor
 * (Sec. 2.3, Sec. 8), with the compression residual kept in memory and added
 * to the next input (Sec. 5.1, lazy error propagation, Eq. (star2)).
 *
 * One call of the fused entry point computes, for an m x n input M:
 *
 *     A     = M + err_prev                        (error-feedback add)
 *     repeat `iters` times:
 *         P     = A Q                             (left product, m x r)
 *         P_hat = orthonormal basis of P          (CholeskyQR, thin-QR factor)
 *         Q     = A^T P_hat                       (right product, n x r)
 *     M_hat = P_hat Q^T                           (decompression)
 *     err   = A - M_hat                           (residual for the next call)
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - Every array pointer is a DEVICE pointer owned by the caller.  No call
 *   allocates or frees device memory; the library keeps no per-call state
 *   outside the workspace the caller passes in.
 * - Matrices are row-major.  ld* is the leading dimension in elements
 *   (>= cols).  P is m x rank and Q is n x rank, both contiguous (ld = rank).
 *   err, P, Q and M_hat are fp32.  M is fp32 or bf16 (occ_dtype_t).
 * - Loads of M may pass the end of a row by up to 15 elements, always inside
 *   the array (never past the last row's last element), and what they read
 *   there is not used; occ_step_rows reads the listed rows only.  err is read
 *   inside its rows only.
 * - Any alignment is accepted, with vector accesses at any; rows that start on
 *   16 bytes (outputs: on 64 bytes, ld a multiple of 16) and hold a multiple of
 *   32 columns select the fastest forms.
 * - Argument errors are detected on the host before anything is enqueued and
 *   are returned as occ_status_t; nothing aborts.  A failed kernel launch
 *   returns OCC_E_HIP.
 * - Numeric conditions never fail a call.  They set sticky bits in the
 *   workspace header, read with occ_get_flags: a non-finite input propagates
 *   into the outputs and sets OCC_F_NONFINITE; a direction of P that is
 *   numerically dependent on the previous ones (Cholesky pivot below 1e-12 of
 *   the largest Gram diagonal) gives a zero column of P_hat and sets
 *   OCC_F_RANK_DEFICIENT.
 * - Work is enqueued on `stream` (a hipStream_t; NULL = the null stream) and
 *   runs asynchronously.  Only occ_get_flags and occ_profile_end synchronise.
 * - Calls that share one workspace must not overlap in time (same stream, or
 *   caller-side ordering); overlapping calls on one workspace race.
 */
#ifndef OPTCC_H
#define OPTCC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define OCC_ABI_VERSION 2
#define OCC_MAX_RANK 128
#define OCC_MAX_ITERS 64
#define OCC_MAX_EXPERTS 1024 /* of a layer of experts */
#define OCC_MAX_CHOICES 32   /* experts of a token */
#define OCC_MAX_TEACHER 1024 /* entries of a teacher's list */

typedef void* occ_stream_t; /* a hipStream_t */

typedef enum {
  OCC_OK = 0,
  OCC_E_NULL = 1,      /* a required pointer is NULL */
  OCC_E_SHAPE = 2,     /* rows/cols < 1, ld < cols, count < 1, or sizes overflow */
  OCC_E_RANK = 3,      /* rank < 1, rank > min(rows, cols) or rank > OCC_MAX_RANK */
  OCC_E_ITERS = 4,     /* iters < 1 or iters > OCC_MAX_ITERS */
  OCC_E_DTYPE = 5,     /* unknown dtype, or mixed dtypes in one batch */
  OCC_E_ALIGN = 6,     /* a pointer is not aligned to its element size */
  OCC_E_ALIAS = 7,     /* two buffers overlap (only err_new == err_prev may) */
  OCC_E_WORKSPACE = 8, /* workspace NULL, too small, or not 256-byte aligned */
  OCC_E_HIP = 9,       /* a HIP runtime call or kernel launch failed */
  OCC_E_FLAGS = 10,    /* unknown bit in the flags argument */
  OCC_E_VALUE = 11     /* an activation, hyperparameter or state form outside its range */
} occ_status_t;

typedef enum { OCC_F32 = 0, OCC_BF16 = 1 } occ_dtype_t;

/* sticky numeric flags, read with occ_get_flags; OCC_F_BAD_ROWS: the row list
 * of occ_step_rows was not strictly increasing inside [0, rows) (the results
 * of that call are then unspecified, but no memory outside the arguments is
 * touched).  The calls on experts' rows and on a teacher's list raise it in a
 * word of the caller's, where they say so. */
enum { OCC_F_NONFINITE = 1u, OCC_F_RANK_DEFICIENT = 2u, OCC_F_BAD_ROWS = 4u };

/* call flags for occ_step / occ_step_batched */
enum { OCC_NO_MHAT = 1u }; /* sender side: do not write M_hat (err is still updated) */

/* flags of occ_decompress_ex */
enum {
  /* run the products occ_step runs for a bf16 M: at padded ranks 32..128 on
   * bf16 matrix cores with each factor split into two bf16 parts (about 2^-16
   * of |M_hat| per element); at padded rank <= 16 the products are fp32 either
   * way and the flag changes nothing */
  OCC_DEC_SPLIT_BF16 = 1u,
  /* store M_hat as bf16 (round to nearest even from the fp32 result) */
  OCC_DEC_OUT_BF16 = 2u
};

/* One matrix and its compressor state.
 *   M      input gradient, rows x cols, leading dimension ldm, dtype m_dtype
 *   err    fp32 error buffer rows x cols (ld lde): read as err_prev, then
 *          overwritten with err_new by occ_step (in place)
 *   P      fp32 rows x rank: output P_hat (orthonormal columns)
 *   Q      fp32 cols x rank: input warm start, output A^T P_hat
 *   M_hat  fp32 rows x cols (ld ldh): output reconstruction P_hat Q^T;
 *          may be NULL when OCC_NO_MHAT is passed */
typedef struct {
  const void* M;
  int32_t m_dtype; /* occ_dtype_t */
  int32_t reserved;
  int64_t rows, cols, ldm;
  float* err;
  int64_t lde;
  float* P;
  float* Q;
  float* M_hat;
  int64_t ldh;
} occ_mat_t;

/* Library ABI version (OCC_ABI_VERSION). */
int occ_abi_version(void);

/* Static description of a status code; never NULL. */
const char* occ_status_str(int status);

/* Workspace bytes that occ_step_batched (count matrices) or occ_step
 * (count = 1) needs for these shapes, rank and iters.  The value does not
 * depend on the pointers.  Returns 0 for invalid arguments. */
size_t occ_workspace_bytes(const occ_mat_t* mats, int count, int rank, int iters);

/* Workspace bytes occ_compress needs for one m x n matrix whose M has dtype
 * m_dtype (the tiling of the large-rank passes depends on it).  Returns 0 for
 * invalid arguments. */
size_t occ_compress_workspace_bytes(int64_t m, int64_t n, int m_dtype, int rank, int iters);

/* Clear the workspace header (sticky flags) on `stream`.  Call once after
 * allocating a workspace; the rest of the workspace needs no initialisation. */
occ_status_t occ_workspace_init(void* ws, size_t ws_bytes, occ_stream_t stream);

/* Compression only (Sec. 2.3 power iteration with the Sec. 5.1 error add):
 * A = M + err_prev (err_prev is read, not modified; NULL means zero);
 * Q (n x rank) is the warm start on entry and A^T P_hat on return;
 * P (m x rank) receives P_hat. */
occ_status_t occ_compress(const void* M, int m_dtype, int64_t m, int64_t n, int64_t ldm,
                          const float* err_prev, int64_t lde, float* P, float* Q,
                          int rank, int iters, void* ws, size_t ws_bytes,
                          occ_stream_t stream);

/* Decompression (Sec. 9.6): M_hat = P Q^T with P m x rank and Q n x rank,
 * fp32 products with fp32 accumulation, M_hat fp32 (m x n, ld ldh). */
occ_status_t occ_decompress(const float* P, const float* Q, int64_t m, int64_t n, int rank,
                            float* M_hat, int64_t ldh, occ_stream_t stream);

/* Decompression on the receiving side of compressed backpropagation (Sec. 5:
 * the next pipeline stage rebuilds the activation gradient from the two
 * factors it received and continues its backward pass with it).  As
 * occ_decompress, with `flags` (OCC_DEC_*):
 *   OCC_DEC_SPLIT_BF16  the products occ_step runs for a bf16 M, so that
 *                       M_hat is bitwise the one the fused step writes;
 *   OCC_DEC_OUT_BF16    M_hat is stored as bf16 (M_hat points to uint16 bf16
 *                       bit patterns, ld ldh elements): each element is the
 *                       fp32 result rounded to nearest even, relative error
 *                       at most 2^-9 per element.
 * Unknown flag bits return OCC_E_FLAGS. */
occ_status_t occ_decompress_ex(const float* P, const float* Q, int64_t m, int64_t n, int rank,
                               unsigned flags, void* M_hat, int64_t ldh, occ_stream_t stream);

/* Error update (Sec. 5.1): err_new = (M + err_prev) - M_hat, elementwise.
 * err_prev and err_new share the leading dimension lde; err_new may equal
 * err_prev (in place); err_prev NULL means zero (lde is then err_new's). */
occ_status_t occ_err_update(const void* M, int m_dtype, int64_t m, int64_t n, int64_t ldm,
                            const float* err_prev, int64_t lde, const float* M_hat,
                            int64_t ldh, float* err_new, occ_stream_t stream);

/* Fused compress + decompress + error update of one matrix; err is updated
 * in place.  Bitwise equal to occ_compress, occ_decompress_ex (with
 * OCC_DEC_SPLIT_BF16 when M is bf16) and occ_err_update called in sequence on
 * the same inputs. */
occ_status_t occ_step(const occ_mat_t* mat, int rank, int iters, unsigned flags,
                      void* ws, size_t ws_bytes, occ_stream_t stream);

/* occ_step on `count` independent matrices (all of one pipeline stage,
 * Sec. 7), one kernel launch per pass for the whole batch.  All matrices
 * share rank, iters and M dtype.  At rank <= 16 each result is bitwise equal
 * to occ_step on that matrix alone.  Above it the grids are planned for the
 * whole batch: the fp32 sums of the two products may be split at other rows
 * and columns than alone, and the results then agree to fp32 rounding. */
occ_status_t occ_step_batched(const occ_mat_t* mats, int count, int rank, int iters,
                              unsigned flags, void* ws, size_t ws_bytes,
                              occ_stream_t stream);

/* Row-sparse step for embedding gradients.  The first pipeline stage's copy
 * of the embedding converts the batch's words into embedding values (Sec. 6),
 * so the gradient of that lookup is zero outside the rows of the words the
 * batch contains.  `rows` (DEVICE pointer, n_rows int32 entries, strictly
 * increasing, each in [0, mat->rows)) lists the rows to compress; the call
 * compresses the n_rows x cols matrix of those rows of M + err and reads and
 * writes nothing else of M, err and M_hat: every other row of err and M_hat
 * is left untouched.  When M and err are zero outside the listed rows (the
 * list is the union of the nonzero rows of both), the result equals
 * occ_step on the whole matrix with M_hat zero in the unlisted rows.
 *   mat->P   receives P_hat in compact form: n_rows x rank, row i belonging to
 *            matrix row rows[i];
 *   mat->Q   warm start in, A^T P_hat out (cols x rank), as in occ_step.
 * Requires n_rows >= rank, except n_rows == 0 (then A is zero: Q is set to
 * zero and OCC_F_RANK_DEFICIENT raised); a caller with fewer live rows than
 * `rank` can list additional zero rows.  The list is checked on the device:
 * a violation raises OCC_F_BAD_ROWS.  Workspace: occ_step_rows_workspace_bytes. */
occ_status_t occ_step_rows(const occ_mat_t* mat, const int32_t* rows, int64_t n_rows, int rank,
                           int iters, unsigned flags, void* ws, size_t ws_bytes,
                           occ_stream_t stream);

/* Workspace bytes occ_step_rows needs for n_rows listed rows of a matrix with
 * `cols` columns and M dtype m_dtype.  Returns 0 for invalid arguments. */
size_t occ_step_rows_workspace_bytes(int64_t n_rows, int64_t cols, int m_dtype, int rank,
                                     int iters);

/* occ_step_batched without a workspace argument and without any device
 * allocation, for callers that cannot allocate: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc.  The
 * workspace is a static device array of OCC_NOALLOC_MAX_BYTES inside the
 * library (one per GPU, held until the process ends); a call whose
 * occ_workspace_bytes exceeds it returns OCC_E_WORKSPACE before anything is
 * enqueued.  Every call on one GPU shares that GPU's array: calls that
 * overlap in time on one GPU (other streams, other threads) race, so callers
 * order them.  Numeric flags are OR-ed into *flags_out (a DEVICE word the
 * caller owns and clears), or dropped when flags_out is NULL.  Results are
 * bitwise those of occ_step_batched on the same arguments. */
#define OCC_NOALLOC_MAX_BYTES ((size_t)64 << 20)
occ_status_t occ_step_batched_noalloc(const occ_mat_t* mats, int count, int rank, int iters,
                                      unsigned flags, uint32_t* flags_out, occ_stream_t stream);

/* Selective stage compression (Sec. 7), host-side model.  With pipeline
 * parallelism the later stages finish their backward passes first and start
 * their data-parallel gradient exchange early; the exchange of the earliest
 * stage is left exposed.  Compressing the exchanges of chosen stages,
 * starting from the earliest, trades compression error for time; each choice
 * moves the bottleneck to another stage.  Times are in one unit of the
 * caller's choice; no device is touched. */

/* When each stage's last backward pass ends under the one-forward-one-
 * backward pipeline schedule (Sec. 2.2), by event simulation: n_stages
 * uniform stages, n_micro micro-batches, t_fwd / t_bwd per micro-batch and
 * stage, t_p2p per hop between adjacent stages.  bwd_done receives n_stages
 * values; *t_end (if not NULL) the end of the schedule.  Invalid counts or
 * negative / non-finite times return OCC_E_SHAPE. */
occ_status_t occ_pipeline_1f1b(int n_stages, int n_micro, double t_fwd, double t_bwd,
                               double t_p2p, double* bwd_done, double* t_end);

/* One stage for occ_sc_select. */
typedef struct {
  double bwd_done;        /* end of the stage's last backward pass */
  double comm;            /* its data-parallel gradient exchange, uncompressed */
  double comm_compressed; /* the exchange of the low-rank factors instead */
  double compress;        /* compressor time on the stage's gradients (e.g. a
                             measured occ_step_batched over the stage) */
} occ_stage_t;

/* Chooses the stages to compress: the exchange of stage s ends at
 * bwd_done + comm, or bwd_done + compress + comm_compressed when compressed.
 * Starting with none compressed, while fewer than max_compressed are, the
 * stage whose exchange ends last is compressed if that ends it earlier; the
 * selection stops at the first bottleneck that is compressed already or would
 * not gain.  selected[s] = 1 for a chosen stage, else 0; *n_selected (if not
 * NULL) the count; *t_end (if not NULL) the end of the last exchange, the
 * least that any choice of at most max_compressed stages reaches. */
occ_status_t occ_sc_select(const occ_stage_t* stages, int n_stages, int max_compressed,
                           uint8_t* selected, int* n_selected, double* t_end);

/* Read (and optionally clear) the sticky numeric flags of a workspace.
 * Synchronises `stream`. */
occ_status_t occ_get_flags(void* ws, uint32_t* flags_out, int clear, occ_stream_t stream);

/* ---------------------------------------------------------------------------
 * Stage operators: what a pipeline stage runs right before and right after
 * the compressor.  The backward pass of a layer takes the activation gradient
 * that occ_decompress_ex rebuilt and makes the weight gradients that
 * occ_step_batched compresses; AdamW takes the decompressed gradients, or the
 * factors themselves.  The conventions above hold: device pointers, row-major
 * matrices with leading dimensions, any alignment (rows that start on 16 bytes
 * and hold whole 16-byte pieces select the fastest forms), host-side checks,
 * work enqueued on `stream`.  Results are deterministic: no atomics, and sums
 * in an order that a call's sizes, types, alignment and the outputs that it asks
 * for decide.  (A backward call plans its products together: dX or dW asked for
 * alone may sum in another order, or on other units, than beside the other.)
 * ------------------------------------------------------------------------- */

/* Activation functions: z; max(z, 0); z Phi(z); the tanh form
 * z (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))) / 2; z / (1 + e^-z). */
typedef enum {
  OCC_ACT_NONE = 0,
  OCC_ACT_RELU = 1,
  OCC_ACT_GELU = 2,
  OCC_ACT_GELU_TANH = 3,
  OCC_ACT_SILU = 4
} occ_act_t;

/* Forward pass of a layer (all matrices of type `dtype`, products and sums in
 * fp32, one rounding at each store):
 *   occ_linear_fwd   Z = X W^T + bias, Y = act(Z) + R
 *                    W is out x in, bias holds `out` values, Z is tokens x out
 *   occ_gated_fwd    [G U] = X W^T + bias, Y = act(G) * U + R
 *                    W is 2 out x in (the gate's rows, then the other
 *                    projection's), bias holds 2 out values, Z = [G U] is
 *                    tokens x 2 out
 * X is tokens x in, Y and R tokens x out.  bias (fp32), R and Z may be NULL;
 * R may be Y (the residual is replaced in place).  Z is what the backward pass
 * needs: leave it out when serving.  tokens may be 0 (nothing is done).
 * in and out at most 2^24.
 * fp32 products of some size run on the bf16 matrix units, each operand as the
 * sum of three bf16 values: a product is then off by at most 2^-25 of itself
 * before it is added in fp32 (operands of 2^-99 and more; of smaller ones the
 * parts below 2^-126 are lost).  There every result that an infinite or NaN
 * operand enters is NaN, also where the fp32 units would give an infinity. */
typedef struct {
  int32_t dtype; /* occ_dtype_t */
  int32_t act;   /* occ_act_t */
  int64_t tokens, in, out;
  const void* X;
  int64_t ldx;
  const void* W;
  int64_t ldw;
  const float* bias;
  const void* R;
  int64_t ldr;
  void* Z;
  int64_t ldz;
  void* Y;
  int64_t ldy;
} occ_linear_t;

/* Backward pass.  With dZ the gradient at the pre-activation,
 *   linear: dZ = dY act'(Z)           gated: dZ = [dY U act'(G), dY act(G)]
 *   dX = dZ W      dW = dZ^T X      dbias = sum of dZ over the tokens
 * dX, dW and dbias may each be NULL (not wanted; at least one is given).  X is
 * needed for dW, W for dX, Z unless the layer is linear with OCC_ACT_NONE.
 * dW has type dw_dtype: `dtype`, or OCC_F32 for a bf16 layer.  With
 * OCC_GRAD_ACCUMULATE dW and dbias are added to (micro-batches), dX is not.
 * dZ is rounded to `dtype` before the products when it is not dY itself; dbias
 * is summed from it before that rounding.  With no tokens dW and dbias are set
 * to zero (or left, when accumulating). */
typedef struct {
  int32_t dtype;    /* occ_dtype_t */
  int32_t dw_dtype; /* occ_dtype_t */
  int32_t act;      /* occ_act_t */
  int32_t reserved;
  int64_t tokens, in, out;
  const void* dY;
  int64_t lddy;
  const void* X;
  int64_t ldx;
  const void* W;
  int64_t ldw;
  const void* Z;
  int64_t ldz;
  void* dX;
  int64_t lddx;
  void* dW;
  int64_t lddw;
  float* dbias;
} occ_linear_grad_t;

enum { OCC_GRAD_ACCUMULATE = 1u };

/* Workspace bytes of the calls below for these arguments (sizes, leading
 * dimensions, alignment and which outputs are asked for).  0: none is needed
 * and ws may be NULL, or the arguments are invalid.  The workspace needs no
 * initialisation; its first 256 bytes (the numeric flags of the compressor)
 * are left alone, so one workspace can serve every call of a stage. */
size_t occ_linear_fwd_workspace_bytes(const occ_linear_t* l);
size_t occ_gated_fwd_workspace_bytes(const occ_linear_t* l);
size_t occ_linear_bwd_workspace_bytes(const occ_linear_grad_t* l);
size_t occ_gated_bwd_workspace_bytes(const occ_linear_grad_t* l);

occ_status_t occ_linear_fwd(const occ_linear_t* l, void* ws, size_t ws_bytes, occ_stream_t stream);
occ_status_t occ_gated_fwd(const occ_linear_t* l, void* ws, size_t ws_bytes, occ_stream_t stream);
occ_status_t occ_linear_bwd(const occ_linear_grad_t* l, unsigned flags, void* ws, size_t ws_bytes,
                            occ_stream_t stream);
occ_status_t occ_gated_bwd(const occ_linear_grad_t* l, unsigned flags, void* ws, size_t ws_bytes,
                           occ_stream_t stream);

/* One tensor of occ_adamw_step.  W, W16, m and v are contiguous rows x cols
 * (a vector: rows = 1).
 *   W        fp32 weights, updated
 *   W16      bf16 copy of the new weights (nearest even), or NULL
 *   G        gradient of type g_dtype, leading dimension ldg, or NULL: then
 *   P, Q     the gradient is P Q^T (P rows x rank, Q cols x rank, contiguous,
 *            fp32: the compressor's factors); it is not written anywhere
 *   m, v     state_bits 32: the fp32 moments.
 *            state_bits 8: m and sqrt(v) as OCP e4m3 codes (one byte each),
 *            with m_scale and v_scale (fp32, rows x ceil(cols / 256)) holding
 *            a factor for each run of 256 columns of a row.  All zero bytes
 *            and scales are the state before the first step.
 *   decay    weight decay (decoupled) of this tensor */
typedef struct {
  int64_t rows, cols;
  float* W;
  void* W16;
  const void* G;
  int64_t ldg;
  int32_t g_dtype; /* occ_dtype_t */
  int32_t rank;
  const float* P;
  const float* Q;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  int32_t state_bits; /* 32 or 8 */
  float decay;
} occ_param_t;

/* Hyperparameters of a step.  step counts from 1.  seed selects the random
 * bits that the 8-bit codes are rounded with: another one each step, the same
 * one on every data-parallel rank; a code depends on seed, the tensor's place
 * in the list and the element's place in the tensor only.  These are values of
 * the call: a graph that holds it repeats its step and seed.
 *   grad_scale  device scalar that multiplies every gradient (a clipping
 *               coefficient, 1 / loss scale), or NULL
 *   flags       device word, e.g. flags_out of occ_step_batched_noalloc, or
 *               NULL: when it holds OCC_F_NONFINITE the call changes nothing */
typedef struct {
  double lr, beta1, beta2, eps;
  int64_t step;
  uint32_t seed;
  uint32_t reserved;
  const float* grad_scale;
  const uint32_t* flags;
} occ_adamw_t;

/* AdamW over `count` tensors (any mix of gradient and state forms):
 *   g = grad_scale G, m = beta1 m + (1 - beta1) g, v = beta2 v + (1 - beta2) g^2
 *   W = W (1 - lr decay) - lr / (1 - beta1^step) m / (sqrt(v / (1 - beta2^step)) + eps)
 * in fp32.  8-bit moments enter at their stored values, the step uses the new
 * moments before they are rounded again.  Codes are rounded up with the
 * probability of the part cut off; a positive v keeps a positive code.  A
 * non-finite gradient reaches W and the moments of its element (8-bit: of its
 * run of 256).  No workspace; nothing is copied to the device by itself. */
occ_status_t occ_adamw_step(const occ_param_t* params, int count, const occ_adamw_t* h,
                            occ_stream_t stream);

/* ---------------------------------------------------------------------------
 * Layers of experts: each token goes to k of the experts, each of which is a
 * linear or gated layer of its own.
 *   occ_route_fwd   the choice of the experts, and the plan of their rows
 *   occ_dispatch    the tokens' rows in the experts' order
 *   occ_experts_*   the layers on those rows
 *   occ_combine     the experts' rows back in the tokens' order, weighted
 * A plan: entry t k + j is the j-th choice of token t; `order` lists the entries
 * expert by expert, those of an expert by token; `offsets` (experts + 1 values)
 * says where each expert's begin, and its last value how many there are;
 * `slots` gives each entry's place in `order`, -1 for a choice that is none.
 * Offsets, order and slots are DEVICE arrays of int32.  The host does not read
 * them: values that fit no plan raise OCC_F_BAD_ROWS in *flags (a device word
 * that the caller owns and clears, or NULL), and no memory outside the
 * arguments is touched.
 * ------------------------------------------------------------------------- */

/* Router.  Of each token's logits the k largest, in falling order, the lower
 * index first among equals (0 and -0 are equal); -inf and NaN are never chosen,
 * and a token with fewer than k others has index -1 and weight 0 in the places
 * left.  Weights (fp32): renorm 1, the softmax over the chosen logits; renorm 0,
 * the softmax over all the experts at the chosen ones.  A NaN among a token's
 * logits makes its weights NaN.  Results of one call depend on its arguments
 * alone: no atomics on floating values, and a stable order.
 * index, weights and slots are tokens x k, order holds tokens k values (those
 * behind offsets[experts] are left alone). */
typedef struct {
  int32_t dtype; /* occ_dtype_t of the logits (and of their gradient) */
  int32_t k;     /* 1 .. OCC_MAX_CHOICES, at most experts */
  int32_t renorm;
  int32_t reserved;
  int64_t tokens, experts; /* tokens k < 2^30, experts <= OCC_MAX_EXPERTS */
  const void* logits;      /* tokens x experts */
  int64_t ldl;
  int32_t* index;
  float* weights;
  int32_t* offsets;
  int32_t* order;
  int32_t* slots;
} occ_route_t;

size_t occ_route_fwd_workspace_bytes(const occ_route_t* r);
occ_status_t occ_route_fwd(const occ_route_t* r, void* ws, size_t ws_bytes, occ_stream_t stream);

/* Gradient of the logits (tokens x experts, of their type, all of it written)
 * from dweights (fp32, tokens x k), with index and weights as occ_route_fwd left
 * them.  With s the sum of w dw over a token's choices:
 *   renorm 1   w (dw - s) at the chosen, 0 elsewhere (logits may be NULL)
 *   renorm 0   -p s at every expert, p their softmax, and w dw more at the chosen
 * dweights of a choice that is none are not looked at; choices of one expert (a
 * plan of the caller's) are added up in their order.  dlogits may be the logits. */
occ_status_t occ_route_bwd(const occ_route_t* r, const float* dweights, void* dlogits, int64_t ldd,
                           occ_stream_t stream);

/* The plan that rows are exchanged by: tokens x width on one side, rows x width
 * on the other (rows: what order holds, at least offsets[experts]). */
typedef struct {
  int32_t dtype; /* occ_dtype_t of all matrices */
  int32_t k;
  int64_t tokens, experts, rows, width;
  const int32_t* offsets; /* occ_dispatch */
  const int32_t* order;   /* occ_dispatch, occ_combine_bwd */
  const int32_t* slots;   /* occ_combine, occ_combine_bwd */
  uint32_t* flags;        /* may be NULL */
} occ_exchange_t;

/* Xs[s] = X[order[s] / k] for s < offsets[experts]; rows behind are left alone.
 * A last offset out of 0 .. rows is taken as the nearer end; it and an entry that
 * is none of the tokens' raise OCC_F_BAD_ROWS, and such an entry's row is left.
 * Its gradient is occ_combine of dXs without weights. */
occ_status_t occ_dispatch(const occ_exchange_t* x, const void* X, int64_t ldx, void* Xs, int64_t ldxs,
                          occ_stream_t stream);

/* Y[t] = sum over j of weights[t][j] Ys[slots[t][j]] + R[t], summed in fp32 in
 * the order of j, rounded once.  weights (fp32) NULL: ones; R may be NULL, or Y.
 * A slot of -1 adds nothing, whatever its weight; any other outside 0 .. rows - 1
 * adds nothing either and raises OCC_F_BAD_ROWS. */
occ_status_t occ_combine(const occ_exchange_t* x, const float* weights, const void* Ys, int64_t ldys, const void* R,
                         int64_t ldr, void* Y, int64_t ldy, occ_stream_t stream);

/* dYs[slots[t][j]] = weights[t][j] dY[t] and dweights[t][j] = <dY[t],
 * Ys[slots[t][j]]> (fp32); either may be NULL.  An entry without a row has
 * dweights 0; rows of dYs that no entry has are left alone.  A slot outside -1 ..
 * rows - 1 raises OCC_F_BAD_ROWS, as does an entry whose place in order does not
 * name it; both count as without. */
occ_status_t occ_combine_bwd(const occ_exchange_t* x, const float* weights, const void* dY, int64_t lddy,
                             const void* Ys, int64_t ldys, void* dYs, int64_t lddys, float* dweights,
                             occ_stream_t stream);

/* The layers.  l is the layer of the first expert: l.tokens counts all rows of
 * X, R, Z and Y (of dY, Z, X and dX), of which those from offsets[e] on up to
 * offsets[e + 1] belong to expert e; rows outside are neither read for a result
 * nor written.  Weights of expert e begin stride_w elements after those of
 * expert e - 1 (dW: stride_dw), biases follow each other: experts x out (gated:
 * experts x 2 out), contiguous.  An expert may have no rows: its dW and dbias
 * are zero (or left, when accumulating).  Offsets out of 0 .. l.tokens are taken as
 * the nearer end, and one that falls as the largest before it; either raises
 * OCC_F_BAD_ROWS (without any rows the offsets are not looked at).  All else is as
 * in occ_linear_fwd and its companions; the order of a sum depends on the number of
 * rows and experts, and of dbias on offsets. */
typedef struct {
  occ_linear_t l;
  int64_t experts; /* 1 .. OCC_MAX_EXPERTS */
  int64_t stride_w;
  const int32_t* offsets;
  uint32_t* flags; /* may be NULL */
} occ_experts_t;

typedef struct {
  occ_linear_grad_t l;
  int64_t experts;
  int64_t stride_w, stride_dw;
  const int32_t* offsets;
  uint32_t* flags;
} occ_experts_grad_t;

size_t occ_experts_linear_fwd_workspace_bytes(const occ_experts_t* l);
size_t occ_experts_gated_fwd_workspace_bytes(const occ_experts_t* l);
size_t occ_experts_linear_bwd_workspace_bytes(const occ_experts_grad_t* l);
size_t occ_experts_gated_bwd_workspace_bytes(const occ_experts_grad_t* l);

occ_status_t occ_experts_linear_fwd(const occ_experts_t* l, void* ws, size_t ws_bytes, occ_stream_t stream);
occ_status_t occ_experts_gated_fwd(const occ_experts_t* l, void* ws, size_t ws_bytes, occ_stream_t stream);
occ_status_t occ_experts_linear_bwd(const occ_experts_grad_t* l, unsigned flags, void* ws, size_t ws_bytes,
                                    occ_stream_t stream);
occ_status_t occ_experts_gated_bwd(const occ_experts_grad_t* l, unsigned flags, void* ws, size_t ws_bytes,
                                   occ_stream_t stream);

/* Loss of the last stage: a token's logits s over the vocabulary against the
 * teacher's k largest logits t, at columns i, and against a label:
 *   p = softmax(t / T) over the list, q = softmax(s / T), c = softmax(s)
 *   loss = scale [alpha T^2 sum p (log p - log q_i) + (1 - alpha) (-log c_label)]
 *   dS_j = scale [alpha T (q_j - p_j) + (1 - alpha) (c_j - [j = label])]
 * (a column listed twice has both its p).  A list entry with a negative index, or
 * a teacher's logit of -inf, is masked; a token whose entries all are has no
 * first part, one whose label is negative (or labels NULL) no second.  With
 * neither, or with scale 0, the loss is 0 and the gradient a row of zeros, and the
 * token's logits are not looked at.  An index or label of `vocab` or more counts
 * as masked and raises OCC_F_BAD_ROWS, also of a token whose scale is 0.  alpha 1
 * leaves labels, alpha 0 the list out of account.
 *   occ_distill_fwd   loss (fp32, a token each); lse, if given, receives the
 *                     logarithms of the two softmaxes' sums (tokens x 2: at T, at
 *                     1; 0 for a part that a token has not); dS, if given, the
 *                     gradient of the sum of the losses, in the same pass
 *   occ_distill_bwd   dS from lse (loss is not looked at); scale carries the
 *                     gradient of each loss: the forward's scale times it
 * dS has the type of S and may be S.  Sums are held in fp32, dS is rounded once.
 * From lse, itself rounded to fp32, a softmax is off by a few 2^-24 of |lse| + |s| / T
 * more; tokens whose lse is beyond +-1024 are summed anew from S. */
typedef struct {
  int32_t dtype;   /* occ_dtype_t of S and dS */
  int32_t t_dtype; /* occ_dtype_t of the teacher's logits */
  int64_t tokens, vocab; /* vocab <= 2^24 */
  const void* S;
  int64_t lds;
  int32_t k; /* 0 .. OCC_MAX_TEACHER */
  int32_t reserved;
  const int32_t* index; /* tokens x k */
  int64_t ldi;
  const void* teacher;  /* tokens x k */
  int64_t ldt;
  const int32_t* labels; /* a token each, or NULL */
  const float* scale;    /* a token each, or NULL: ones */
  float temperature, alpha; /* T > 0, its square a normal number; alpha 0 .. 1 */
  float* loss;
  float* lse;
  void* dS;
  int64_t ldds;
  uint32_t* flags; /* may be NULL */
} occ_distill_t;

occ_status_t occ_distill_fwd(const occ_distill_t* d, occ_stream_t stream);
occ_status_t occ_distill_bwd(const occ_distill_t* d, occ_stream_t stream);

/* Per-kernel timing with HIP events, for benchmarks.  Between
 * occ_profile_begin and occ_profile_end every kernel the library launches is
 * bracketed by events on its stream.  occ_profile_end synchronises those
 * events and fills up to `max` records (kernel name, launches, total
 * milliseconds), returning the number of distinct kernels in *n_out.  Not
 * thread-safe; intended for single-threaded measurement. */
typedef struct {
  char name[48];
  int32_t launches;
  int32_t reserved;
  double total_ms;
} occ_kernel_time_t;

occ_status_t occ_profile_begin(void);
occ_status_t occ_profile_end(occ_kernel_time_t* out, int max, int* n_out);

#ifdef __cplusplus
}
#endif

#endif /* OPTCC_H */
