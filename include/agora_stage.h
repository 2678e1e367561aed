/*
 * Model operators of a pipeline stage (libssn.so): what a Llama-style stage of the paper's model
 * (grouped-query attention, rotary positions, query/key norm: the model table of the appendix)
 * computes between its library matrix products, next to the boundary codec of ssn.h.
 *
 *   stage_qk_rope_*       the norm of every query and key head with the rotation by position, forward
 *                         and backward
 *   stage_distill_loss    the tail stage's loss against a teacher's top logits, with the logits' gradient
 *   stage_int8_*          products of a frozen stage in 8-bit integers, scaled per token and channel
 *
 * The common rules are those of ssn.h: raw DEVICE pointers owned by the caller, strides counted in
 * ELEMENTS, nothing allocated, freed or synchronised inside, work enqueued on `stream` (a cudaStream_t
 * passed as void*) of the current device, host-detectable mistakes refused before a launch, one
 * element type (ssn_dtype_t) per call unless stated, sums in fp32 or wider and ONE rounding at the end.
 * Buffers of one call must not overlap unless stated; each is aligned to its element (SSN_ERR_SHAPE if not).  A call's
 * result is the same bits every time.
 */
#ifndef AGORA_STAGE_H_
#define AGORA_STAGE_H_

#include "ssn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- query/key norm with rotary positions ---------------------------------------------------------- */

/* Which columns of a head turn together, i < rot_dim / 2: (i, i + rot_dim / 2), or (2 i, 2 i + 1). */
typedef enum { STAGE_PAIR_HALVES = 0, STAGE_PAIR_ADJACENT = 1 } stage_pairing_t;

#define STAGE_MAX_HEAD_DIM 256

/*
 * What every block of a stage shares.  Plain value struct, read on the host during the call.
 * The table holds one row per position: rot_dim / 2 cosines, then rot_dim / 2 sines.
 */
typedef struct stage_qk_rope {
  int32_t head_dim;     /* D: even, 2 .. STAGE_MAX_HEAD_DIM                                        */
  int32_t rot_dim;      /* rotated columns [0, rot_dim): even, 0 .. D; the others are only normed  */
  int32_t dtype;        /* ssn_dtype_t of heads, gradients and gains                               */
  int32_t pairing;      /* stage_pairing_t                                                         */
  float eps;            /* >= 0, finite                                                            */
  int32_t max_pos;      /* rows of the table (ignored when rot_dim is 0)                           */
  const void *wq;       /* device [D] gain of the query heads, or NULL: ones                       */
  const void *wk;       /* device [D] gain of the key heads, or NULL: ones                         */
  const float *table;   /* device [max_pos x rot_dim] fp32, required when rot_dim > 0              */
  int64_t ldt;          /* >= rot_dim                                                              */
  int32_t *dev_status;  /* device int32 or NULL                                                    */
} stage_qk_rope_t;

/*
 * A rotation table: row p has cos(p theta^(-2 i / rot_dim)) at column i and the sine at column
 * rot_dim / 2 + i, angles and functions in 64 bits, rounded once.  theta > 0, rot_dim >= 2 and even.
 */
ssn_status_t stage_rope_table(float *table, int64_t ldt, int32_t max_pos, int32_t rot_dim, double theta,
                              void *stream);

/*
 * For every token t and head h, with x the D values at x[t * token_stride + h * head_stride]:
 *     n = x / sqrt(mean(x^2) + eps) * w;     y = n with its column pairs (a, b) turned by the angle of pos(t):
 *     (a cos - b sin, b cos + a sin)
 *   q, k     [n_tokens x heads x D], D contiguous; any strides >= 0 (views of a fused projection's output,
 *            head-major buffers, broadcast rows), at most 65536 heads.  0 heads: that tensor is absent and may be NULL.
 *            The squares are summed in fp32: a row whose sum passes its range (values around 10^18) becomes zeros.
 *   q_out, k_out   the same with strides that keep its rows apart.  An output may be its own input
 *            (same address and strides).
 *   pos      device int32[n_tokens], or NULL: pos(t) = t mod seq_len (seq_len >= 1 required then).
 *            A position outside [0, max_pos) takes a ZERO table row (its rotated columns become 0) and ORs
 *            SSN_DEV_BAD_POS into *dev_status.
 */
ssn_status_t stage_qk_rope_forward(const stage_qk_rope_t *op, const void *q, int64_t q_token, int64_t q_head,
                                   int32_t q_heads, const void *k, int64_t k_token, int64_t k_head, int32_t k_heads,
                                   void *q_out, int64_t qo_token, int64_t qo_head, void *k_out, int64_t ko_token,
                                   int64_t ko_head, const int32_t *pos, int64_t n_tokens, int32_t seq_len, void *stream);

/*
 * The gradients: with g the incoming gradient turned back by the angle, r = 1 / sqrt(mean(x^2) + eps), u = x r,
 *     dx = r (g w - u mean(g w u)),     dw = sum over tokens and heads of g u
 *   dq, dk          gradients of the forward outputs (any strides >= 0)
 *   q, k            the forward INPUTS
 *   dq_in, dk_in    out, gradients of the inputs; may be dq / dk (same address and strides)
 *   dwq, dwk        out, fp32 [D] each, overwritten (zeros when there are no rows), or NULL: not wanted
 *   workspace       of stage_qk_rope_workspace_bytes(), 16-byte aligned; not needed when dwq and dwk are NULL.  The size is the
 *                   same for every n_tokens > 0; calls that may run at one time need one each
 */
size_t stage_qk_rope_workspace_bytes(const stage_qk_rope_t *op, int64_t n_tokens, int32_t q_heads, int32_t k_heads);
ssn_status_t stage_qk_rope_backward(const stage_qk_rope_t *op, const void *dq, int64_t dq_token, int64_t dq_head,
                                    const void *dk, int64_t dk_token, int64_t dk_head, const void *q, int64_t q_token,
                                    int64_t q_head, int32_t q_heads, const void *k, int64_t k_token, int64_t k_head,
                                    int32_t k_heads, void *dq_in, int64_t dqi_token, int64_t dqi_head, void *dk_in,
                                    int64_t dki_token, int64_t dki_head, float *dwq, float *dwk, const int32_t *pos,
                                    int64_t n_tokens, int32_t seq_len, void *workspace, size_t workspace_bytes,
                                    void *stream);

/* ---- loss against a teacher's top logits ----------------------------------------------------------- */

#define STAGE_DISTILL_MAX_TOP 1024
#define STAGE_DISTILL_MIN_TAU 1e-6f
#define STAGE_DISTILL_MAX_TAU 1e6f

/*
 * A teacher's K best logits of every token are what crosses a slow link instead of a row of the vocabulary.
 * With x = logits[t] / tau over the vocabulary and p the softmax of top[t] / tau over the row's entries,
 *     loss[t]       = weight[t] tau^2 sum_j p_j (log p_j - x[ids[t, j]] + log sum_v exp x_v)
 *     dlogits[t, v] = weight[t] tau (softmax(x)_v - sum over the j with ids[t, j] = v of p_j)
 *   logits   [n_tokens x vocab] of dtype, ldl >= vocab, vocab <= 2^31 - 16
 *   ids      int32 [n_tokens x top_k], ldi >= top_k, and top, fp32 [n_tokens x top_k], ldt >= top_k: the row's
 *            entries in any order, 1 <= top_k <= STAGE_DISTILL_MAX_TOP.  An id of -1 is padding; any other id outside
 *            [0, vocab) ORs SSN_DEV_BAD_ID into *dev_status and counts as padding.  An id may stand there twice.
 *   weight   fp32 [n_tokens] or NULL: ones
 *   tau      temperature, STAGE_DISTILL_MIN_TAU .. STAGE_DISTILL_MAX_TAU
 *   loss     fp32 [n_tokens], out
 *   dlogits  [n_tokens x vocab] of dtype, ldd >= vocab, out, or NULL: the loss alone.  It may be `logits` itself
 *            (same address and ldd == ldl).
 * A row of weight 0, one without entries and one whose entries are all -inf have loss 0 and a gradient of zeros,
 * whatever their logits hold.  Logits of -inf have probability 0 (a loss of +inf where the teacher gives them any).
 * With top_k = 1 and tau = 1 it is the cross entropy of the target ids[t, 0], whatever finite number its teacher logit is.
 * The loss has the same bits with the gradient and without.  The order of a row's sums goes by the number of rows (few rows are
 * shared by several CTAs) and by the row's place within 16 bytes.
 */
ssn_status_t stage_distill_loss(const void *logits, int64_t ldl, int32_t dtype, int64_t n_tokens, int64_t vocab,
                                const int32_t *ids, int64_t ldi, const float *top, int64_t ldt, int32_t top_k,
                                const float *weight, float tau, float *loss, void *dlogits, int64_t ldd,
                                int32_t *dev_status, void *stream);

/* ---- products in 8-bit integers -------------------------------------------------------------------- */

#define STAGE_INT8_MAX_INNER 131071   /* 128 * 128 * inner stays below 2^31 */

/*
 * Rows in 8 bits, one scale each (tokens of an activation, or output channels of a weight, stored [outer x inner]):
 *     scale[r] = max_i |x[r, i]| / 127 in fp32;    q[r, i] = x[r, i] / scale[r], the EXACT quotient rounded to the nearest
 * integer, halves to the even one, within [-127, 127].
 *   x      [rows x cols] of dtype, ldx >= cols;   q  int8 [rows x cols], ldq >= cols;   scale  fp32 [rows]
 * A row whose scale is 0 (zeros, or values below 127 times the smallest fp32 number) has q = 0.  A row with an infinity
 * or a NaN has q = 0 and scale NaN, so that its products are NaN.
 */
ssn_status_t stage_int8_quantize(const void *x, int64_t ldx, int32_t dtype, int64_t rows, int64_t cols, int8_t *q,
                                 int64_t ldq, float *scale, void *stream);

/*
 * A frozen projection:  y[t, o] = (sum_i xq[t, i] wq[o, i]) xs[t] ws[o], the sum in 32-bit integers (exact), then two
 * products in fp32 and one rounding to dtype.
 *   xq  int8 [n_tokens x inner], ldx >= inner;  xs  fp32 [n_tokens];  wq  int8 [outer x inner], ldw >= inner;
 *   ws  fp32 [outer];  y  [n_tokens x outer] of dtype, ldy >= outer;  1 <= inner <= STAGE_INT8_MAX_INNER
 *   dev_status  device int32 or NULL: SSN_DEV_TIMEOUT when an internal bounded wait ran out (y is invalid then)
 * Any int8 value may occur, -128 too.  Rows that start on 16-byte boundaries (address and leading dimension of xq and wq) are
 * fetched by TMA; with others the product takes twice as long (few tokens) to eight times (many).  Any y will do; rows on 16-byte boundaries are
 * stored 16 bytes at a time.
 */
ssn_status_t stage_int8_matmul(const int8_t *xq, int64_t ldx, const float *xs, const int8_t *wq, int64_t ldw,
                               const float *ws, int64_t n_tokens, int64_t inner, int64_t outer, void *y, int64_t ldy,
                               int32_t dtype, int32_t *dev_status, void *stream);

/*
 * A status word for callers that keep none of their own: its device address on the current device (NULL without one), the same
 * one for the life of the process, 0 at first.  Calls OR their bits into it where it is handed over as dev_status, and only
 * there; who clears it clears it for all of them.
 */
int32_t *stage_status_word(void);

/*
 * What ssn_last_kernel() says after a call of this header: family | (variant << 8).
 *   STAGE_KERNEL_ROPE       variant: columns per piece (1 .. 8) | the bits below.  The gains' sums are not told apart
 *   STAGE_KERNEL_DISTILL    CTAs per row (1 .. 8) | STAGE_KVAR_MANY (256 threads) | STAGE_KVAR_GRAD
 *   STAGE_KERNEL_QUANTIZE   pieces per thread | warps per row << 4; 0: rows of any length and place
 *   STAGE_KERNEL_INT8_DOT   tokens (1, 2) | STAGE_KVAR_ANYWHERE
 *   STAGE_KERNEL_INT8_UMMA  rows of the tile's B operand (16 .. 256) | STAGE_KVAR_PAIR, _SWAP, _SPLIT, _ANYWHERE
 */
enum {
  STAGE_KERNEL_ROPE = 16,
  STAGE_KERNEL_DISTILL = 17,
  STAGE_KERNEL_QUANTIZE = 18,
  STAGE_KERNEL_INT8_DOT = 19,
  STAGE_KERNEL_INT8_UMMA = 20
};
#define STAGE_KVAR_ADJACENT 16 /* ROPE: pairs of adjacent columns                                   */
#define STAGE_KVAR_CROSSED 32  /* ROPE: halves whose partners are read from shared memory           */
#define STAGE_KVAR_FULL 64     /* ROPE: every column turns                                          */
#define STAGE_KVAR_BACK 128    /* ROPE: the gradients                                               */
#define STAGE_KVAR_MANY 16     /* DISTILL                                                           */
#define STAGE_KVAR_GRAD 32     /* DISTILL                                                           */
#define STAGE_KVAR_PAIR 1      /* INT8_UMMA: two CTAs per tile                                      */
#define STAGE_KVAR_SWAP 2      /* INT8_UMMA: the weights on the M side                              */
#define STAGE_KVAR_SPLIT 4     /* INT8_UMMA: a cluster shares the inner dimension                   */
#define STAGE_KVAR_ANYWHERE 8  /* INT8: operand rows off 16-byte boundaries                         */

/* ---- the same calls with their arguments in one struct ---------------------------------------------- */

/*
 * For callers whose foreign-function layer takes long over each argument (calls of one token are shorter on the GPU than
 * that): the fields are the arguments of the call of that name, in its order.  `args` is read during the call.
 */
typedef struct stage_qk_rope_forward_args {
  const stage_qk_rope_t *op;
  const void *q; int64_t q_token, q_head; int32_t q_heads;
  const void *k; int64_t k_token, k_head; int32_t k_heads;
  void *q_out; int64_t qo_token, qo_head;
  void *k_out; int64_t ko_token, ko_head;
  const int32_t *pos; int64_t n_tokens; int32_t seq_len; void *stream;
} stage_qk_rope_forward_args_t;

typedef struct stage_qk_rope_backward_args {
  const stage_qk_rope_t *op;
  const void *dq; int64_t dq_token, dq_head;
  const void *dk; int64_t dk_token, dk_head;
  const void *q; int64_t q_token, q_head; int32_t q_heads;
  const void *k; int64_t k_token, k_head; int32_t k_heads;
  void *dq_in; int64_t dqi_token, dqi_head;
  void *dk_in; int64_t dki_token, dki_head;
  float *dwq, *dwk;
  const int32_t *pos; int64_t n_tokens; int32_t seq_len;
  void *workspace; size_t workspace_bytes; void *stream;
} stage_qk_rope_backward_args_t;

typedef struct stage_distill_loss_args {
  const void *logits; int64_t ldl; int32_t dtype; int64_t n_tokens, vocab;
  const int32_t *ids; int64_t ldi;
  const float *top; int64_t ldt; int32_t top_k;
  const float *weight; float tau; float *loss;
  void *dlogits; int64_t ldd;
  int32_t *dev_status; void *stream;
} stage_distill_loss_args_t;

typedef struct stage_int8_quantize_args {
  const void *x; int64_t ldx; int32_t dtype; int64_t rows, cols;
  int8_t *q; int64_t ldq;
  float *scale; void *stream;
} stage_int8_quantize_args_t;

typedef struct stage_int8_matmul_args {
  const int8_t *xq; int64_t ldx;
  const float *xs;
  const int8_t *wq; int64_t ldw;
  const float *ws;
  int64_t n_tokens, inner, outer;
  void *y; int64_t ldy; int32_t dtype;
  int32_t *dev_status; void *stream;
} stage_int8_matmul_args_t;

ssn_status_t stage_qk_rope_forward_packed(const stage_qk_rope_forward_args_t *args);
ssn_status_t stage_qk_rope_backward_packed(const stage_qk_rope_backward_args_t *args);
ssn_status_t stage_distill_loss_packed(const stage_distill_loss_args_t *args);
ssn_status_t stage_int8_quantize_packed(const stage_int8_quantize_args_t *args);
ssn_status_t stage_int8_matmul_packed(const stage_int8_matmul_args_t *args);

#ifdef __cplusplus
}
#endif

#endif /* AGORA_STAGE_H_ */
