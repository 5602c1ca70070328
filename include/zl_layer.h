/* Operators of decoder layers beside those that a chunk runs: activations
 * saved in 8 bits and their use in the backward, norms before and after a block
 * with gate and residual scale, and rotary positions with several axes.
 * They stand next to zl_kernel_gemm and zl_kernel_attention (zl_inspect.h).
 *
 * Conventions are those of zl.h: device pointers, caller-owned buffers, calls
 * asynchronous on `stream`, arguments checked before any launch.  Argument
 * structures are read during the call only.  Pointers belong to the current
 * device.  Matrices are row-major with a row stride (ld, in elements); a
 * contiguous dimension is a multiple of 8 elements, a row stride too, and
 * pointers are 16-byte aligned (ZL_ERR_INVALID_ARG otherwise), unless a call
 * says less; a matrix has at most 2^30 columns (ZL_ERR_UNSUPPORTED above) and a
 * launch at most 2^32 threads (ZL_ERR_HIP above).  Buffers overlap only where a call says so.  T = 0 is an empty
 * batch: nothing is read, sums over rows are zero.  No call allocates memory;
 * all may be captured into a graph, and results do not depend on timing (no
 * atomics: every sum has a fixed order). */
#ifndef ZL_LAYER_H
#define ZL_LAYER_H

#include <stddef.h>
#include <stdint.h>

#include "zl.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------- 8-bit saved activations
 * A packed matrix [T, n]: per element a code of 8 bits (e4m3: sign, 4 bits of
 * exponent, 3 of fraction, largest value 448), per 32 columns of a row (the
 * last block may be shorter) one scale of 8 bits, byte b standing for
 * 2^(b - 127).  An element stands for code * scale.
 *
 * Packing takes the smallest scale 2^e, -117 <= e <= 119, that brings the
 * block's finite values within 448, and rounds value / scale to the nearest
 * code, ties to even.  So an element is off by at most 2^-4 of itself or, where
 * it is below 2^-6 scale, by 2^-10 scale; and it is exact in bf16 and fp32.
 * An infinite or NaN element becomes NaN and leaves its block's scale alone;
 * finite values beyond 448 * 2^119 = 1.75 * 2^127 become +-448 * 2^119.
 *
 * codes: T rows of ld_codes bytes, ld_codes >= n a multiple of 16, 16-byte
 * aligned.  scales: T rows of ld_scales >= ceil(n / 32) bytes.  Bytes of a row
 * past its n codes are not written and may hold anything, but are memory that
 * may be read. */
typedef struct zl_packed {
  void* codes;
  void* scales;
  int64_t ld_codes;
  int64_t ld_scales;
} zl_packed;

/* out = x [T, n] (ZL_F32 or ZL_BF16, row stride ldx) in 8 bits. */
zl_status zl_pack(int64_t T, int n, const void* x, int64_t ldx, int dtype, const zl_packed* out,
                  void* stream);
/* x = the values of `in`.  A scale byte of 255 is NaN. */
zl_status zl_unpack(int64_t T, int n, const zl_packed* in, void* x, int64_t ldx, int dtype,
                    void* stream);

/* ---------------------------------------------------------- MLP activation
 * ZL_MLP_SWIGLU: h = gate | up [T, 2 ff], a = silu(gate) * up;
 * ZL_MLP_GELU: h [T, ff], a = gelu(h) (tanh form).
 * Products give h and da (in_dtype: zl_kernel_gemm's fp32, or bf16), products
 * take a and dh (out_dtype). */
enum { ZL_MLP_SWIGLU = 0, ZL_MLP_GELU = 1 };
typedef struct zl_mlp_args {
  int64_t T;
  int ff;
  int kind;           /* ZL_MLP_*                                             */
  int in_dtype, out_dtype;
  const void* h;      /* [T, 2 ff or ff]; in the backward NULL with packed    */
  int64_t ldh;
  zl_packed packed;   /* h in 8 bits; codes NULL = none.  The forward writes
                         it, the backward reads it in place of h.  SwiGLU
                         needs ff % 32 == 0 with it (else
                         ZL_ERR_UNSUPPORTED: the halves share no block)       */
  void* a;            /* [T, ff] out; in the backward NULL = not wanted, else
                         the activation formed again (for the down
                         projection's weight gradient)                        */
  int64_t lda;
  const void* da;     /* backward: [T, ff]                                    */
  int64_t ldda;
  void* dh;           /* backward: out, the shape of h                        */
  int64_t lddh;
} zl_mlp_args;
zl_status zl_mlp_act(const zl_mlp_args* args, void* stream);
zl_status zl_mlp_act_backward(const zl_mlp_args* args, void* stream);

/* ------------------------------------------------------ norms around a block
 * The seam between two blocks of a layer, row by row (d columns):
 *   p  = Norm(y) w_post + b_post        norm after a block with output y
 *   xo = x + scale * gate * p           gated, scaled residual
 *   n  = Norm(xo) w_pre + b_pre         norm before the next block
 * Norm is RMSNorm, or LayerNorm (layernorm != 0); biases may be NULL.
 * Without the first norm (w_post NULL: the first block of a chunk) xo = x and
 * nothing but n is formed; without the second (w_pre NULL: the last block) n is
 * not formed.  gate [ceil(T / gate_rows), d] fp32, row r using gate row
 * r / gate_rows (1: per token, the sequence length: per sequence, T: shared);
 * NULL = 1.
 * The residual stream x, xo and its gradients are fp32 (row stride ldx); y and
 * dn come from products (in_dtype), n and dy go into products (out_dtype).
 * stats [T, 4] fp32, 16-byte aligned, contiguous: mean and 1 / deviation of y,
 * then those of xo (0 where there is no such norm; RMSNorm's mean is 0).
 * d <= 8192 (ZL_ERR_UNSUPPORTED above). */
typedef struct zl_norm_args {
  int64_t T;
  int d;
  int layernorm;
  int in_dtype, out_dtype;
  float eps, scale;
  const float* w_post;
  const float* b_post;
  const float* w_pre;
  const float* b_pre;
  const float* gate;
  int64_t gate_rows;  /* >= 1 with a gate                                     */
  float* stats;       /* forward: written; backward: read                     */
  /* forward */
  const float* x;     /* [T, d]                                               */
  float* xo;          /* [T, d], may be x; unused without w_post.  The
                         backward reads it with w_pre (x itself without
                         w_post)                                              */
  int64_t ldx;        /* of x, xo, dxo, dx                                    */
  const void* y;      /* [T, d]; in the backward NULL with y_packed           */
  int64_t ldy;        /* of y and dy                                          */
  void* n;            /* [T, d]                                               */
  int64_t ldn;        /* of n and dn                                          */
  zl_packed y_packed; /* y in 8 bits; codes NULL = none.  The forward writes
                         it, the backward reads it in place of y              */
  zl_packed n_packed; /* forward: n (as rounded to out_dtype) in 8 bits, for
                         the weight gradients of the projections that read n;
                         codes NULL = none                                    */
  /* backward */
  const float* dxo;   /* [T, d] gradient of xo besides that through n; NULL = 0 */
  const void* dn;     /* [T, d] with w_pre                                    */
  float* dx;          /* [T, d] out, may be dxo                               */
  void* dy;           /* [T, d] out, with w_post                              */
  /* gradients of the parameters, fp32: grad_scale * sum, added to what is
     there with accumulate; NULL = not wanted */
  float* dw_post;
  float* db_post;
  float* dw_pre;
  float* db_pre;
  float* dgate;       /* the shape of gate                                    */
  float grad_scale;
  int accumulate;
  float* workspace;   /* backward: zl_block_norm_workspace floats, 16-byte
                         aligned; scratch of this call until it has run       */
  size_t workspace_elems;
} zl_norm_args;
zl_status zl_block_norm(const zl_norm_args* args, void* stream);
zl_status zl_block_norm_backward(const zl_norm_args* args, void* stream);
/* Floats of workspace that zl_block_norm_backward needs (host only);
 * gate_rows as above, 0 without a gate. */
zl_status zl_block_norm_workspace(int64_t T, int d, int64_t gate_rows, size_t* elems);

/* ------------------------------------------- weight gradient, packed input
 * dw [n_out, n_in] (fp32, row stride lddw) = scale * dy^T x, or added to it
 * with accumulate: dy [T, n_out] (ZL_BF16 or ZL_F32), x [T, n_in] packed (read
 * as it is, its values exact).  Sums are fp32.
 * workspace (workspace_elems floats, 16-byte aligned, or NULL): lets a dw of
 * few tiles split T into fp32 partials there, summed in a fixed order. */
zl_status zl_wgrad_packed(int64_t T, int n_out, int n_in, const void* dy, int64_t lddy, int dtype,
                          const zl_packed* x, float scale, int accumulate, float* dw, int64_t lddw,
                          float* workspace, size_t workspace_elems, void* stream);

/* ------------------------------------------------------- rotary positions
 * out = x with every head's first `rot` columns rotated: columns j and
 * j + rot / 2 (j < rot / 2) by the angle
 *   pos[axis_of[j] * T + t] * theta^(-2 j / rot)   (inverse != 0: its negative,
 * which takes gradients of out to gradients of x); the others are copied.
 * x, out: T rows of n_heads heads of head_dim columns (row strides ldx, ldo;
 * the queries and keys of a packed row are n_heads = Hq + Hkv heads); out may
 * be x.  Any alignment; 16-byte aligned rows and rot % 16 == 0 are fastest.
 * pos: device [n_axes, T] int32, any values (for video and images: time,
 * height, width; n_axes = 1 is plain RoPE).  axis_of: HOST array of rot / 2
 * axis numbers in [0, n_axes), read during the call.  Angles are reduced in 64
 * bits.  head_dim even, at most 256; rot even, 2 .. head_dim; theta > 1;
 * n_axes 1 .. 16. */
zl_status zl_rotary(int64_t T, int n_heads, int head_dim, int rot, const void* x, int64_t ldx,
                    void* out, int64_t ldo, int dtype, const int32_t* pos, int n_axes,
                    const uint8_t* axis_of, double theta, int inverse, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* ZL_LAYER_H */
