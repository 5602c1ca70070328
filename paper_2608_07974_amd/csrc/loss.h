// Internal declarations of the losses (include/zl_loss.h): what the host code
// checks, the kernels take on trust.
#pragma once

#include "../../include/zl_loss.h"
#include "common.h"

namespace zl {

// 0, or which accesses of a call with so many bytes of output and input stream past the
// caches (layer.hip).
int streaming(int64_t out, int64_t in);

constexpr int TOP_MAX_K = 256;

hipError_t launch_top_logits(int64_t T, int V, const void* x, int64_t ldx, int dtype, int k, float temperature,
                             int32_t* ids, float* values, float* rest, hipStream_t s);

struct LogitLossArgs {
  int64_t T;
  int V;
  const void* z;
  int64_t ldz;
  zl_targets t;
  float a, b;           // weights of CE and tau^2 KL
  float* loss;          // forward
  float* stats;
  const float* dloss;   // backward
  float scale;
  void* dz;
  int64_t lddz;
};
hipError_t launch_logit_loss(const LogitLossArgs& a, int dtype, bool backward, hipStream_t s);

// Where a head loss keeps what in its workspace (byte offsets), and the pieces
// of the vocabulary that the backward goes through.
struct HeadPlan {
  bool large;           // 256 x 256 tiles of the logits' product, else 128 x 128
  int width, blocks;    // column blocks of the forward's partial sums
  int columns;          // per piece
  int64_t ldz;          // row stride of dL/dz
  int64_t ldb;          // blocks of a row as far as they have memory
  size_t tid, tval, part, span, order, named, gmax, coef, live, dz, dxa, xc, split, bytes;
  size_t split_elems;
};
HeadPlan head_plan(int64_t T, int V, int d, int dtype, int k, bool backward, bool need_dx, bool need_dw,
                   int columns);
hipError_t launch_head_loss(const zl_head_args& a, hipStream_t s);
hipError_t launch_head_loss_bwd(const zl_head_args& a, hipStream_t s);

// (a, b) of a CE + b tau^2 KL.
inline void loss_weights(const zl_targets& t, float& a, float& b) {
  const bool hard = t.labels != nullptr, soft = t.ids != nullptr;
  a = hard ? (soft ? t.alpha : 1.f) : 0.f;
  b = soft ? (hard ? 1.f - t.alpha : 1.f) : 0.f;
}

}  // namespace zl
