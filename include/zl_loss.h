/* Losses over a vocabulary beside the chunk's own objective: against labels,
 * against a teacher's top logits, or both; of logits in memory, or of a readout
 * head's logits that are never kept, with the gradients of the head's input and
 * weight; and the top logits of a row that such a teacher is made of.
 *
 * Conventions are those of zl_layer.h: device pointers of the current device,
 * caller-owned buffers, calls asynchronous on `stream`, arguments checked before
 * any launch, structures read during the call only.  No call allocates memory or
 * uses atomics on device memory; all may be captured into a graph, and results do
 * not depend on timing.  T = 0 is an empty batch: nothing is read, a weight's
 * gradient is zero (or left alone with accumulate).  Buffers overlap only where a
 * call says so.  T <= 2^21 and V <= 2^30 (ZL_ERR_UNSUPPORTED above). */
#ifndef ZL_LOSS_H
#define ZL_LOSS_H

#include <stddef.h>
#include <stdint.h>

#include "zl.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------- the targets
 * Row t has logits z (V of them) and adds
 *   loss = a CE + b tau^2 KL,   tau = temperature, 2^-60 to 2^60,
 * a = alpha, b = 1 - alpha with labels and a teacher, else 1 for the one there is.  A term
 * of weight 0 adds nothing, also where it is infinite.
 *
 * Label y:  CE = log sum_v exp(z_v) - z_y.  A label outside [0, V) is none.
 *
 * Teacher:  ids[j], values[j] (j < k): its top logits.  Its distribution is over
 * those ids, p_j ~ exp(values[j] / tau), and, with rest, over one outcome more,
 * "any other column", r ~ exp(rest): rest = log of the sum of exp(logit / tau) over
 * the teacher's other columns (-inf: nothing).  The student's is softmax(z / tau),
 * summed over the other columns for that outcome.  KL = KL(teacher || student).
 * An id outside [0, V) is absent, and so is one that the row has named before; what
 * values holds there does not matter.  A row whose ids are all absent, or all of
 * whose outcomes weigh nothing (-inf), has no teacher.
 *
 * A row without label and teacher has loss 0 and gradient 0 whatever its logits
 * are, also infinite or NaN. */
enum { ZL_TARGETS_MAX_K = 256 };
typedef struct zl_targets {
  const int32_t* labels;  /* [T] or NULL                                       */
  const int32_t* ids;     /* [T, k] or NULL                                    */
  const float* values;    /* [T, k], with ids                                  */
  const float* rest;      /* [T] or NULL                                       */
  int k;                  /* 1 .. ZL_TARGETS_MAX_K with ids, else 0            */
  float alpha;            /* in [0, 1]                                         */
  float temperature;      /* in [2^-60, 2^60]                                  */
} zl_targets;

/* -------------------------------------------------------------- top logits
 * Of every row of x [T, V] (ZL_F32 or ZL_BF16, row stride ldx >= V, any
 * alignment) the k largest: ids and values [T, k], in descending order, equal
 * ones by ascending column (-0 equals 0).  A NaN counts as larger than any
 * number.  rest [T] (or NULL): log of the sum of exp(x / temperature) over the
 * other columns; -inf where there are none.  1 <= k <= V, k <= 256; temperature
 * in [2^-60, 2^60]. */
zl_status zl_top_logits(int64_t T, int V, const void* x, int64_t ldx, int dtype, int k, float temperature,
                        int32_t* ids, float* values, float* rest, void* stream);

/* ---------------------------------------------------------- loss of logits
 * loss [T] of z [T, V] (ZL_F32 or ZL_BF16, row stride ldz >= V, any alignment).
 * stats [T, 4], 16-byte aligned, is what the backward needs besides: the
 * log-sum of z (rows with a label, else 0), that of z / tau (rows with a teacher,
 * else 0), that of z / tau over the columns the teacher does not name (rows with a
 * teacher that has a rest, else 0), the label's logit (else 0). */
zl_status zl_logit_loss(int64_t T, int V, const void* z, int64_t ldz, int dtype, const zl_targets* targets,
                        float* loss, float* stats, void* stream);
/* dz [T, V] (z's type, row stride lddz; may be z with ldz) = scale * dloss[t] *
 * dloss_t / dz; dloss NULL = ones.  Rows of dz that start at another place in 16 bytes
 * than z's are written element by element, which takes longer. */
zl_status zl_logit_loss_backward(int64_t T, int V, const void* z, int64_t ldz, int dtype, const zl_targets* targets,
                                 const float* stats, const float* dloss, float scale, void* dz, int64_t lddz,
                                 void* stream);

/* --------------------------------------------------- loss of a readout head
 * The same loss of z = x w^T, x [T, d], w [V, d] (both ZL_BF16 or both ZL_F32; d a
 * multiple of 8, at most 65536; rows 16-byte aligned, strides multiples of 8 below
 * 2^21; the forward T V at most 2^36, the backward T d below 2^35).  z is held in fp32
 * accumulators and never stored: the forward keeps partial sums of 32 to 128 columns,
 * the backward forms z again, `columns` of the vocabulary at a time, and from it dL/dz
 * in x's type, which it multiplies on.  With ZL_BF16 log2(e) z and log2(e) z / tau have
 * to be numbers of fp32 (|z| up to 2^127).
 *
 * stats [T, 4 + k], contiguous: as above, then z at the teacher's ids (0 where
 * absent).
 *
 * dx [T, d] = scale * sum_t ..., dw [V, d] likewise (added to what is there with
 * accumulate: fp32 dw only); either may be NULL (both with T = 0).  A row of x without label and
 * teacher adds nothing to dw, also if it is infinite or NaN.  With ZL_BF16 dL/dz
 * is rounded to bf16 as an operand of both products, after division by the
 * largest |dloss| of rows with a target and by a (without labels b tau), so that rows of equal weight
 * round as with weight 1; sums are fp32.  A label's q - 1 is formed from the two
 * logarithms in stats (expm1): off by half a step of each, 4e-6 at 40, never above 0. */
typedef struct zl_head_args {
  int64_t T;
  int V, d;
  int dtype;
  const void* x;
  int64_t ldx;
  const void* w;
  int64_t ldw;
  zl_targets targets;
  float* stats;           /* forward: written; backward: read                  */
  float* loss;            /* forward: [T]                                      */
  /* backward */
  const float* dloss;     /* [T] or NULL = ones                                */
  float scale;
  int columns;            /* of a piece of the vocabulary; rounded up to a
                             multiple of 256; 0 = as many as 1 GiB of dL/dz
                             holds                                             */
  void* dx;
  int64_t lddx;
  int dx_dtype;
  void* dw;               /* with it T d < 2^30, V d < 2^35
                             (ZL_ERR_UNSUPPORTED above)                        */
  int64_t lddw;
  int dw_dtype;
  int accumulate;
  void* workspace;        /* zl_head_loss_workspace bytes, 256-byte aligned;
                             scratch of this call until it has run             */
  size_t workspace_bytes;
} zl_head_args;
zl_status zl_head_loss(const zl_head_args* args, void* stream);
zl_status zl_head_loss_backward(const zl_head_args* args, void* stream);
/* Bytes of workspace (host only).  k and has_rest: of the targets (the size does not
 * depend on has_rest as yet); need_dx, need_dw: whether the backward gives them (ignored
 * for the forward). */
zl_status zl_head_loss_workspace(int64_t T, int V, int d, int dtype, int k, int has_rest, int backward, int need_dx,
                                 int need_dw, int columns, size_t* bytes);

#ifdef __cplusplus
}
#endif
#endif /* ZL_LOSS_H */
