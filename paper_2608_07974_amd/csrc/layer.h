// Internal declarations of the layer operators (include/zl_layer.h): what the
// host code checks, the kernels take on trust.
#pragma once

#include "../../include/zl_layer.h"
#include "common.h"

namespace zl {

// 0, 1 (stores) or 2 (loads too): which accesses of a call with so many bytes of
// output and input stream past the caches.
int streaming(int64_t out, int64_t in);

// Blocks of 256 threads that one launch takes: fewer than 2^32 threads.
constexpr int64_t MAX_BLOCKS = (1 << 24) - 1;

hipError_t launch_pack(int64_t T, int n, const void* x, int64_t ldx, int dtype, const zl_packed& out,
                       hipStream_t s);
hipError_t launch_unpack(int64_t T, int n, const zl_packed& in, void* x, int64_t ldx, int dtype,
                         hipStream_t s);

hipError_t launch_mlp(const zl_mlp_args& a, bool backward, hipStream_t s);

hipError_t launch_block_norm(const zl_norm_args& a, hipStream_t s);
// How the backward's blocks take the rows: nblk blocks of `slots` slots; every
// slot has up to `rows` rows, each slot in turn one of them.  group > 0: every
// `group` rows (one gate row) have cpg blocks of their own.  gates > 0: all blocks
// go through that many gate rows.  Else, with a gate, a turn is the rows of one
// gate row, and `rows` a multiple of them.  gate_part: partial rows of dgate.
struct NormPlan {
  int64_t nblk, rows, group, cpg, gates, gate_part;
  int slots;
};
NormPlan norm_plan(int64_t T, int d, int64_t gate_rows);
hipError_t launch_block_norm_bwd(const zl_norm_args& a, hipStream_t s);

struct RotaryArgs {
  int64_t T;
  int heads, hd, half;
  const void* x;
  int64_t ldx;
  void* out;
  int64_t ldo;
  const int32_t* pos;
  int vec;               // 16-byte aligned rows of whole 8-column groups
  float sign;
  double turns[128];     // theta^(-2 j / rot) / (2 pi)
  uint8_t axis[128];
};
hipError_t launch_rotary(const RotaryArgs& a, int dtype, hipStream_t s);

struct WgradArgs {
  int64_t T;
  int M, N;              // n_out, n_in
  const void* dy;
  int64_t lddy;
  zl_packed x;
  float scale;
  int accumulate;
  float* dw;
  int64_t lddw;
  float* part;
  size_t part_elems;
};
hipError_t launch_wgrad_packed(const WgradArgs& a, int dtype, hipStream_t s);

}  // namespace zl
