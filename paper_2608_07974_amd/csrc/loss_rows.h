// Device parts that the losses share: sums over a block, online log-sums.
#pragma once

#include "common.h"

namespace zl {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o, 64));
  return x;
}
// Over the NT threads of a block, in a fixed order; every thread gets the result.
// red: NT / 64 floats; barriers on both sides.
template <int NT>
__device__ __forceinline__ float block_sum(float x, float* red) {
  x = wave_sum(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  float r = red[0];
#pragma unroll
  for (int i = 1; i < NT / 64; ++i) r += red[i];
  return r;
}
template <int NT>
__device__ __forceinline__ float block_max(float x, float* red) {
  x = wave_max(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  float r = red[0];
#pragma unroll
  for (int i = 1; i < NT / 64; ++i) r = fmaxf(r, red[i]);
  return r;
}

// sum of exp((v - m) c): m the largest value so far (-inf: none yet), c2 = c log2(e).
// Differences are taken before the scaling: a row of the type's lowest values would
// overflow in v c.  A NaN goes into the sum.
struct LogSum {
  float m = -INFINITY, s = 0.f;
  __device__ __forceinline__ float ref() const { return m == -INFINITY ? 0.f : m; }
  __device__ __forceinline__ void raise(float mx, float c2) {
    if (mx > m) {
      s *= __builtin_amdgcn_exp2f((m - mx) * c2);
      m = mx;
    }
  }
  __device__ __forceinline__ void merge(float om, float os, float c2) {
    raise(om, c2);
    if (om != -INFINITY) os *= __builtin_amdgcn_exp2f((om - m) * c2);
    s += os;
  }
  __device__ __forceinline__ float log(float c) const { return m * c + logf(s); }  // -inf where empty
};
template <int N>
__device__ __forceinline__ float max_of(const float (&v)[N]) {
  float m = v[0];
#pragma unroll
  for (int k = 1; k < N; ++k) m = fmaxf(m, v[k]);
  return m;
}
// Over a block; every thread gets the result.  red: 2 * NT / 64 floats.
template <int NT>
__device__ __forceinline__ LogSum block_logsum(LogSum a, float c2, float* red) {
  const float m = block_max<NT>(a.m, red);
  float s = a.s;
  if (a.m != -INFINITY) s *= __builtin_amdgcn_exp2f((a.m - m) * c2);
  LogSum r;
  r.m = m;
  r.s = block_sum<NT>(s, red);
  return r;
}

// Of a label's logit and the log-sum of the row's other columns (tau 1): CE, which is
// softplus(others - zy), and the log-sum of all.  From a log-sum of all columns CE would be a
// difference: of a sure label 0, or a step of the logits' magnitude (40 against 50000 columns at
// 16: 3.8e-6 where 1.9e-6 is right).
struct LabelTerm {
  float loss, logsum;
};
__device__ __forceinline__ LabelTerm label_term(const LogSum& others, float zy) {
  const float ls = __builtin_amdgcn_logf(others.s) * LN2;  // (1 step of 2^-23, as the reciprocal)
  const float x = (others.m - zy) + ls, lo = others.m + ls;
  const float y = __builtin_amdgcn_exp2f(-fabsf(x) * LOG2E), u = 1.f + y;
  // log(1 + y): the quotient mends u's rounding; a NaN stays
  float t = u == 1.f ? y : __builtin_amdgcn_logf(u) * LN2 * (y * __builtin_amdgcn_rcpf(u - 1.f));
  if (zy == INFINITY) t = NAN;
  return {fmaxf(x, 0.f) + t, zy == -INFINITY ? lo : (x > 0.f ? lo : zy) + t};
}

}  // namespace zl
