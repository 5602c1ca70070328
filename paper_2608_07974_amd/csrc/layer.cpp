// Host side of the layer operators (include/zl_layer.h): argument checks, then
// one launch function each (layer.hip, block_norm.hip, wgrad_packed.hip).
#include <math.h>
#include <string.h>

#include <string>

#include "../../include/zl_layer.h"
#include "common.h"
#include "internal.h"
#include "layer.h"

using namespace zl;

namespace {

zl_status bad(const char* msg) { return set_error(ZL_ERR_INVALID_ARG, msg); }

zl_status done(hipError_t e, const char* what) {
  if (e == hipSuccess) return ZL_OK;
  return set_error(ZL_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

bool aligned(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
bool dtype_ok(int dt) { return dt == ZL_F32 || dt == ZL_BF16; }
int dt_of(int dt) { return dt == ZL_BF16 ? BF16 : F32; }

// A matrix of n columns: present, aligned, rows of whole 16-byte groups.  An
// empty batch (T = 0) has no memory to point at.
bool mat_ok(const void* p, int64_t ld, int64_t n, int64_t T) {
  return T == 0 || (p && aligned(p) && ld >= n && ld % 8 == 0);
}
bool packed_ok(const zl_packed& p, int64_t n, int64_t T) {
  return T == 0 || (p.codes && p.scales && aligned(p.codes) && p.ld_codes >= n && p.ld_codes % 16 == 0 &&
                    p.ld_scales >= (n + 31) / 32);
}
bool cols_ok(int n) { return n > 0 && n % 8 == 0; }
// column numbers, rounded up to a block's columns, stay within 32 bits
bool wide(int64_t n) { return n > (int64_t)1 << 30; }
zl_status too_wide() { return set_error(ZL_ERR_UNSUPPORTED, "more than 2^30 columns"); }

const char* kCols = "columns must be a positive multiple of 8";
const char* kMat = "matrix missing, not 16-byte aligned, or a bad row stride";
const char* kPacked =
    "packed matrix missing, codes not 16-byte aligned or their stride no multiple of 16, or a short row";

}  // namespace

extern "C" {

zl_status zl_pack(int64_t T, int n, const void* x, int64_t ldx, int dtype, const zl_packed* out, void* stream) {
  if (T < 0 || !out) return bad("bad pack args");
  if (!dtype_ok(dtype)) return bad("bad dtype");
  if (!cols_ok(n)) return bad(kCols);
  if (wide(n)) return too_wide();
  if (!mat_ok(x, ldx, n, T)) return bad(kMat);
  if (!packed_ok(*out, n, T)) return bad(kPacked);
  return done(launch_pack(T, n, x, ldx, dt_of(dtype), *out, (hipStream_t)stream), "pack");
}

zl_status zl_unpack(int64_t T, int n, const zl_packed* in, void* x, int64_t ldx, int dtype, void* stream) {
  if (T < 0 || !in) return bad("bad unpack args");
  if (!dtype_ok(dtype)) return bad("bad dtype");
  if (!cols_ok(n)) return bad(kCols);
  if (wide(n)) return too_wide();
  if (!mat_ok(x, ldx, n, T)) return bad(kMat);
  if (!packed_ok(*in, n, T)) return bad(kPacked);
  return done(launch_unpack(T, n, *in, x, ldx, dt_of(dtype), (hipStream_t)stream), "unpack");
}

static zl_status check_mlp(const zl_mlp_args* a, bool backward) {
  if (!a || a->T < 0) return bad("bad MLP activation args");
  if (a->kind != ZL_MLP_SWIGLU && a->kind != ZL_MLP_GELU) return bad("kind must be ZL_MLP_SWIGLU or ZL_MLP_GELU");
  if (!dtype_ok(a->in_dtype) || !dtype_ok(a->out_dtype)) return bad("bad dtype");
  if (!cols_ok(a->ff)) return bad(kCols);
  const int64_t nh = (a->kind == ZL_MLP_SWIGLU ? 2 : 1) * (int64_t)a->ff;
  if (wide(nh)) return too_wide();
  const bool pk = a->packed.codes != nullptr;
  if (pk && a->kind == ZL_MLP_SWIGLU && a->ff % 32)
    return set_error(ZL_ERR_UNSUPPORTED, "SwiGLU with a packed h needs ff to be a multiple of 32");
  if (pk && !packed_ok(a->packed, nh, a->T)) return bad(kPacked);
  if (backward) {
    if (pk && a->h) return bad("the backward takes h or its packed copy, not both");
    if (!pk && !mat_ok(a->h, a->ldh, nh, a->T)) return bad(kMat);
    if (!mat_ok(a->da, a->ldda, a->ff, a->T) || !mat_ok(a->dh, a->lddh, nh, a->T)) return bad(kMat);
    if (a->a && !mat_ok(a->a, a->lda, a->ff, a->T)) return bad(kMat);
  } else {
    if (!mat_ok(a->h, a->ldh, nh, a->T) || !mat_ok(a->a, a->lda, a->ff, a->T)) return bad(kMat);
  }
  return ZL_OK;
}

zl_status zl_mlp_act(const zl_mlp_args* args, void* stream) {
  if (zl_status st = check_mlp(args, false)) return st;
  return done(launch_mlp(*args, false, (hipStream_t)stream), "MLP activation");
}
zl_status zl_mlp_act_backward(const zl_mlp_args* args, void* stream) {
  if (zl_status st = check_mlp(args, true)) return st;
  return done(launch_mlp(*args, true, (hipStream_t)stream), "MLP activation backward");
}

static zl_status check_norm(const zl_norm_args* a, bool backward) {
  if (!a || a->T < 0) return bad("bad block norm args");
  if (!cols_ok(a->d)) return bad(kCols);
  if (a->d > 8192) return set_error(ZL_ERR_UNSUPPORTED, "block norm above 8192 columns");
  if (!dtype_ok(a->in_dtype) || !dtype_ok(a->out_dtype)) return bad("bad dtype");
  const bool post = a->w_post != nullptr, pre = a->w_pre != nullptr;
  if (!post && !pre) return bad("block norm needs w_post or w_pre");
  if (!(a->eps > 0.f) || !isfinite(a->eps)) return bad("eps must be > 0");
  if (!aligned(a->w_post) || !aligned(a->w_pre) || !aligned(a->b_post) || !aligned(a->b_pre))
    return bad("norm weights and biases must be 16-byte aligned");
  if ((a->b_post && (!post || !a->layernorm)) || (a->b_pre && (!pre || !a->layernorm)))
    return bad("a bias needs its weight and layernorm");
  if (a->gate && (!post || a->gate_rows < 1 || !aligned(a->gate)))
    return bad("a gate needs w_post, gate_rows >= 1 and 16-byte alignment");
  if ((a->T && !a->stats) || !aligned(a->stats)) return bad("stats missing or not 16-byte aligned");
  const int64_t T = a->T;
  const int d = a->d;
  if (!backward) {
    if (!mat_ok(a->x, a->ldx, d, T)) return bad(kMat);
    if (post && (!mat_ok(a->y, a->ldy, d, T) || !mat_ok(a->xo, a->ldx, d, T))) return bad(kMat);
    if (pre && !mat_ok(a->n, a->ldn, d, T)) return bad(kMat);
    if (a->y_packed.codes && (!post || !packed_ok(a->y_packed, d, T))) return bad(kPacked);
    if (a->n_packed.codes && (!pre || !packed_ok(a->n_packed, d, T))) return bad(kPacked);
    return ZL_OK;
  }
  if (a->dxo && !mat_ok(a->dxo, a->ldx, d, T)) return bad(kMat);
  if (!mat_ok(a->dx, a->ldx, d, T)) return bad(kMat);
  if (pre && (!mat_ok(a->xo, a->ldx, d, T) || !mat_ok(a->dn, a->ldn, d, T))) return bad(kMat);
  if (post) {
    if (a->y && a->y_packed.codes) return bad("the backward takes y or its packed copy, not both");
    if (a->y_packed.codes ? !packed_ok(a->y_packed, d, T) : !mat_ok(a->y, a->ldy, d, T))
      return bad(a->y_packed.codes ? kPacked : kMat);
    if (!mat_ok(a->dy, a->ldy, d, T)) return bad(kMat);
  }
  if (!aligned(a->dw_post) || !aligned(a->db_post) || !aligned(a->dw_pre) || !aligned(a->db_pre) ||
      !aligned(a->dgate))
    return bad("parameter gradients must be 16-byte aligned");
  if ((a->dw_post && !post) || (a->dw_pre && !pre) || (a->db_post && (!post || !a->layernorm)) ||
      (a->db_pre && (!pre || !a->layernorm)) || (a->dgate && !a->gate))
    return bad("a gradient of a parameter that is not there");
  size_t need = 0;
  if (zl_status st = zl_block_norm_workspace(T, d, a->gate ? a->gate_rows : 0, &need)) return st;
  if (need && (!a->workspace || a->workspace_elems < need))
    return set_error(ZL_ERR_WORKSPACE, "block norm workspace missing or too small");
  if (!aligned(a->workspace)) return set_error(ZL_ERR_WORKSPACE, "block norm workspace must be 16-byte aligned");
  return ZL_OK;
}

zl_status zl_block_norm_workspace(int64_t T, int d, int64_t gate_rows, size_t* elems) {
  if (T < 0 || !cols_ok(d) || gate_rows < 0 || !elems) return bad("bad block norm workspace args");
  const NormPlan p = norm_plan(T, d, gate_rows);
  *elems = (size_t)(4 * p.nblk + p.gate_part) * d;
  return ZL_OK;
}
zl_status zl_block_norm(const zl_norm_args* args, void* stream) {
  if (zl_status st = check_norm(args, false)) return st;
  return done(launch_block_norm(*args, (hipStream_t)stream), "block norm");
}
zl_status zl_block_norm_backward(const zl_norm_args* args, void* stream) {
  if (zl_status st = check_norm(args, true)) return st;
  return done(launch_block_norm_bwd(*args, (hipStream_t)stream), "block norm backward");
}

zl_status zl_wgrad_packed(int64_t T, int n_out, int n_in, const void* dy, int64_t lddy, int dtype, const zl_packed* x,
                          float scale, int accumulate, float* dw, int64_t lddw, float* workspace,
                          size_t workspace_elems, void* stream) {
  if (T < 0 || !x || !dw) return bad("bad weight gradient args");
  if (T > 0x7fffffff) return set_error(ZL_ERR_UNSUPPORTED, "more than 2^31 - 1 tokens");
  if (!dtype_ok(dtype)) return bad("bad dtype");
  if (!cols_ok(n_out) || !cols_ok(n_in)) return bad(kCols);
  if (wide(n_out) || wide(n_in)) return too_wide();
  if (!mat_ok(dy, lddy, n_out, T) || !mat_ok(dw, lddw, n_in, 1)) return bad(kMat);
  if (!packed_ok(*x, n_in, T)) return bad(kPacked);
  if (!aligned(workspace)) return bad("workspace must be 16-byte aligned");
  WgradArgs a = {T, n_out, n_in, dy, lddy, *x, scale, accumulate != 0, dw, lddw, workspace, workspace ? workspace_elems : 0};
  return done(launch_wgrad_packed(a, dt_of(dtype), (hipStream_t)stream), "weight gradient");
}

zl_status zl_rotary(int64_t T, int n_heads, int head_dim, int rot, const void* x, int64_t ldx, void* out, int64_t ldo,
                    int dtype, const int32_t* pos, int n_axes, const uint8_t* axis_of, double theta, int inverse,
                    void* stream) {
  if (T < 0 || n_heads < 1 || !axis_of) return bad("bad rotary args");
  if (!dtype_ok(dtype)) return bad("bad dtype");
  if (head_dim < 2 || head_dim % 2 || rot < 2 || rot % 2 || rot > head_dim)
    return bad("head_dim and rot must be even, 2 <= rot <= head_dim");
  if (head_dim > 256) return set_error(ZL_ERR_UNSUPPORTED, "head_dim above 256");
  if (n_axes < 1 || n_axes > 16) return bad("n_axes must be 1 .. 16");
  if (!(theta > 1.0) || !isfinite(theta)) return bad("theta must be > 1");
  const int64_t w = (int64_t)n_heads * head_dim;
  if (w > 0x7fffffff / 256) return set_error(ZL_ERR_UNSUPPORTED, "more than 2^23 columns of heads");
  if (T > 0) {
    if (!x || !out || !pos) return bad("bad rotary args");
    if (ldx < w || ldo < w) return bad("row stride below n_heads * head_dim");
    const uintptr_t es = dtype == ZL_BF16 ? 2 : 4;
    if ((uintptr_t)x % es || (uintptr_t)out % es || (uintptr_t)pos % 4) return bad("misaligned pointer");
    if (x == out && ldx != ldo) return bad("in place needs the same row stride");
  }
  RotaryArgs a;
  memset(&a, 0, sizeof(a));
  a.T = T;
  a.heads = n_heads;
  a.hd = head_dim;
  a.half = rot / 2;
  a.x = x;
  a.ldx = ldx;
  a.out = out;
  a.ldo = ldo;
  a.pos = pos;
  a.sign = inverse ? -1.f : 1.f;
  a.vec = rot % 16 == 0 && head_dim % 8 == 0 && ldx % 8 == 0 && ldo % 8 == 0 && aligned(x) && aligned(out);
  // powers by products of 64-bit fractions: 128 of them are off by less than the
  // rounding to double, and cost less than as many pow (0.2 us for 64, 1.5)
  const long double step = powl((long double)theta, -2.0L / rot);
  long double turn = 0.5L / 3.14159265358979323846264338327950288L;
  for (int j = 0; j < a.half; ++j, turn *= step) {
    if (axis_of[j] >= n_axes) return bad("axis_of must be below n_axes");
    a.axis[j] = axis_of[j];
    a.turns[j] = (double)turn;
  }
  return done(launch_rotary(a, dt_of(dtype), (hipStream_t)stream), "rotary");
}

}  // extern "C"
