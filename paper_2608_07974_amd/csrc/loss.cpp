// Host side of the losses (include/zl_loss.h): argument checks, then one launch
// function each (logit_loss.hip, head_loss.hip).
#include <math.h>

#include <string>

#include "loss.h"
#include "internal.h"

using namespace zl;

namespace {

constexpr int64_t MAX_T = (int64_t)1 << 21;
constexpr int MAX_V = 1 << 30;
constexpr int64_t MAX_ELEMS = (int64_t)1 << 35;  // of a matrix that a thread per eight goes over
constexpr int64_t MAX_LD = (int64_t)1 << 21;  // of x and w: a tile's 32-bit offsets

zl_status bad(const char* msg) { return set_error(ZL_ERR_INVALID_ARG, msg); }
zl_status unsupported(const char* msg) { return set_error(ZL_ERR_UNSUPPORTED, msg); }

zl_status done(hipError_t e, const char* what) {
  if (e == hipSuccess) return ZL_OK;
  return set_error(ZL_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

bool dtype_ok(int dt) { return dt == ZL_F32 || dt == ZL_BF16; }
int dt_of(int dt) { return dt == ZL_BF16 ? BF16 : F32; }
// log2(e) / tau and tau^2 have to be numbers of fp32: times a difference of 0 they are 0 then.
bool temperature_ok(float tau) { return tau >= 0x1p-60f && tau <= 0x1p60f; }
bool by(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

zl_status check_sizes(int64_t T, int V) {
  if (T < 0 || V < 1) return bad("T must be >= 0 and V >= 1");
  if (T > MAX_T) return unsupported("more than 2^21 rows");
  if (V > MAX_V) return unsupported("more than 2^30 columns");
  return ZL_OK;
}

// A matrix of logits: present, elements aligned, rows that do not overlap.
bool logits_ok(const void* p, int64_t ld, int V, int dtype, int64_t T) {
  return T == 0 || (p && ld >= V && by(p, dtype == ZL_BF16 ? 2 : 4));
}
// A matrix of rows in 16-byte groups.
bool mat_ok(const void* p, int64_t ld, int n, int64_t T) { return T == 0 || (p && by(p, 16) && ld >= n && ld % 8 == 0); }

zl_status check_targets(const zl_targets& t, int64_t T) {
  const bool hard = t.labels != nullptr, soft = t.ids != nullptr;
  if (T && !hard && !soft) return bad("labels, a teacher or both must be there");
  if (t.k < 0 || (soft && t.k < 1) || (T && !soft && t.k != 0)) return bad("k must be >= 1 with ids and 0 without");
  if (t.k > ZL_TARGETS_MAX_K) return unsupported("more than 256 ids per row");
  if (T && (soft != (t.values != nullptr) || (t.rest && !soft))) return bad("ids and values go together, rest with both");
  if (!(t.alpha >= 0.f && t.alpha <= 1.f)) return bad("alpha must be in [0, 1]");
  if (!temperature_ok(t.temperature)) return bad("temperature must be in [2^-60, 2^60]");
  if (!by(t.labels, 4) || !by(t.ids, 4) || !by(t.values, 4) || !by(t.rest, 4)) return bad("misaligned targets");
  return ZL_OK;
}

zl_status check_head(const zl_head_args* a, bool backward) {
  if (!a) return bad("bad head loss args");
  if (zl_status st = check_sizes(a->T, a->V)) return st;
  if (!dtype_ok(a->dtype)) return bad("bad dtype");
  if (a->d < 8 || a->d % 8) return bad("d must be a positive multiple of 8");
  if (a->d > 65536) return unsupported("d above 65536");
  if (zl_status st = check_targets(a->targets, a->T)) return st;
  if (!mat_ok(a->x, a->ldx, a->d, a->T) || !mat_ok(a->w, a->ldw, a->d, a->T))
    return bad("x or w missing, not 16-byte aligned, or a bad row stride");
  if (a->T && (a->ldx >= MAX_LD || a->ldw >= MAX_LD)) return unsupported("row strides of 2^21 and more");
  if (a->T && (!a->stats || !by(a->stats, 4))) return bad("stats missing or misaligned");
  if (!backward) {
    if (a->T * a->V > (int64_t)1 << 36) return unsupported("T V above 2^36: take the rows in parts");
    if (a->T && (!a->loss || !by(a->loss, 4))) return bad("loss missing or misaligned");
  } else {
    if (!by(a->dloss, 4)) return bad("misaligned dloss");
    if (a->T * a->d >= MAX_ELEMS) return unsupported("T d >= 2^35: take the rows in parts");
    if (a->columns < 0) return bad("columns must be >= 0");
    if (a->T && !a->dx && !a->dw) return bad("dx, dw or both must be there");
    if (a->dx && (!dtype_ok(a->dx_dtype) || !mat_ok(a->dx, a->lddx, a->d, 1))) return bad("dx: bad dtype, alignment or row stride");
    if (a->dw) {
      if (!dtype_ok(a->dw_dtype) || !mat_ok(a->dw, a->lddw, a->d, 1)) return bad("dw: bad dtype, alignment or row stride");
      if (a->accumulate && a->dw_dtype != ZL_F32) return unsupported("accumulation into a bf16 dw");
      if ((int64_t)a->V * a->d >= MAX_ELEMS) return unsupported("dw of V d >= 2^35");
      if ((a->T + 64) * a->d >= (int64_t)1 << 30) return unsupported("dw of T d >= 2^30: take the rows in parts, with accumulate");
    }
  }
  if (a->T == 0) return ZL_OK;
  const zl_targets& t = a->targets;
  const HeadPlan p = head_plan(a->T, a->V, a->d, dt_of(a->dtype), t.k, backward, a->dx != nullptr,
                               a->dw != nullptr, a->columns);
  if (!a->workspace || a->workspace_bytes < p.bytes)
    return set_error(ZL_ERR_WORKSPACE, "head loss workspace missing or too small");
  if (!by(a->workspace, 256)) return set_error(ZL_ERR_WORKSPACE, "head loss workspace must be 256-byte aligned");
  return ZL_OK;
}

}  // namespace

extern "C" {

zl_status zl_top_logits(int64_t T, int V, const void* x, int64_t ldx, int dtype, int k, float temperature, int32_t* ids,
                        float* values, float* rest, void* stream) {
  if (zl_status st = check_sizes(T, V)) return st;
  if (!dtype_ok(dtype)) return bad("bad dtype");
  if (k < 1 || k > V) return bad("k must be 1 .. V");
  if (k > TOP_MAX_K) return unsupported("k above 256");
  if (!temperature_ok(temperature)) return bad("temperature must be in [2^-60, 2^60]");
  if (!logits_ok(x, ldx, V, dtype, T)) return bad("logits missing, misaligned, or a row stride below V");
  if (T && (!ids || !values)) return bad("ids or values missing");
  if (!by(ids, 4) || !by(values, 4) || !by(rest, 4)) return bad("misaligned output");
  return done(launch_top_logits(T, V, x, ldx, dt_of(dtype), k, temperature, ids, values, rest, (hipStream_t)stream),
              "top logits");
}

zl_status zl_logit_loss(int64_t T, int V, const void* z, int64_t ldz, int dtype, const zl_targets* targets, float* loss,
                        float* stats, void* stream) {
  if (!targets) return bad("bad logit loss args");
  if (zl_status st = check_sizes(T, V)) return st;
  if (!dtype_ok(dtype)) return bad("bad dtype");
  if (zl_status st = check_targets(*targets, T)) return st;
  if (!logits_ok(z, ldz, V, dtype, T)) return bad("logits missing, misaligned, or a row stride below V");
  if (T && (!loss || !stats)) return bad("loss or stats missing");
  if (!by(loss, 4) || !by(stats, 16)) return bad("misaligned output");
  LogitLossArgs a = {T, V, z, ldz, *targets, 0.f, 0.f, loss, stats, nullptr, 0.f, nullptr, 0};
  loss_weights(*targets, a.a, a.b);
  return done(launch_logit_loss(a, dt_of(dtype), false, (hipStream_t)stream), "logit loss");
}

zl_status zl_logit_loss_backward(int64_t T, int V, const void* z, int64_t ldz, int dtype, const zl_targets* targets,
                                 const float* stats, const float* dloss, float scale, void* dz, int64_t lddz,
                                 void* stream) {
  if (!targets) return bad("bad logit loss args");
  if (zl_status st = check_sizes(T, V)) return st;
  if (!dtype_ok(dtype)) return bad("bad dtype");
  if (zl_status st = check_targets(*targets, T)) return st;
  if (!logits_ok(z, ldz, V, dtype, T) || !logits_ok(dz, lddz, V, dtype, T))
    return bad("logits missing, misaligned, or a row stride below V");
  if (T > 1 && z == dz && ldz != lddz) return bad("in place needs the same row stride");
  if (T && !stats) return bad("stats missing");
  if (!by(stats, 16) || !by(dloss, 4)) return bad("misaligned stats or dloss");
  LogitLossArgs a = {T, V, z, ldz, *targets, 0.f, 0.f, nullptr, const_cast<float*>(stats), dloss, scale, dz, lddz};
  loss_weights(*targets, a.a, a.b);
  return done(launch_logit_loss(a, dt_of(dtype), true, (hipStream_t)stream), "logit loss backward");
}

zl_status zl_head_loss_workspace(int64_t T, int V, int d, int dtype, int k, int has_rest, int backward, int need_dx,
                                 int need_dw, int columns, size_t* bytes) {
  if (!bytes || k < 0 || columns < 0) return bad("bad head loss workspace args");
  if (zl_status st = check_sizes(T, V)) return st;
  if (!dtype_ok(dtype)) return bad("bad dtype");
  if (d < 8 || d % 8) return bad("d must be a positive multiple of 8");
  if (d > 65536) return unsupported("d above 65536");
  if (k > ZL_TARGETS_MAX_K) return unsupported("more than 256 ids per row");
  *bytes = T ? head_plan(T, V, d, dt_of(dtype), k, backward != 0, need_dx != 0, need_dw != 0, columns).bytes : 0;
  return ZL_OK;
}

zl_status zl_head_loss(const zl_head_args* args, void* stream) {
  if (zl_status st = check_head(args, false)) return st;
  return done(launch_head_loss(*args, (hipStream_t)stream), "head loss");
}
zl_status zl_head_loss_backward(const zl_head_args* args, void* stream) {
  if (zl_status st = check_head(args, true)) return st;
  return done(launch_head_loss_bwd(*args, (hipStream_t)stream), "head loss backward");
}

}  // extern "C"
