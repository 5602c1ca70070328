// Weight gradient from a packed activation (include/zl_layer.h):
//   dw[m, n] = sum_t dy[t, m] x[t, n],  x in 8 bits with a scale per 32 columns.
#include <string.h>

#include "gemm_epilogue.h"
#include "layer.h"
#include "packed.h"

namespace zl {

hipError_t launch_splitk_reduce(const float* part, int nz, int M, int N, const EpiArgs& e, hipStream_t s);

// ------------------------------------------------------------ vector ALUs
// 64 x 64 tiles, 16 tokens a step, 4 x 4 outputs per thread.  A block has
// tokens [z per, (z + 1) per); with splits it writes fp32 partials.
constexpr int VT = 64, VK = 16;

template <bool BF>
__global__ void __launch_bounds__(256) wgrad_valu_kernel(WgradArgs a, int64_t per, bool split) {
  __shared__ __align__(16) float As[VK][VT], Bs[VK][VT];
  const int m0 = blockIdx.y * VT, n0 = blockIdx.x * VT;
  const int64_t t0 = blockIdx.z * per, t1 = min(t0 + per, a.T);
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  float acc[4][4] = {};
  // this thread's 8 columns of one of the 16 tokens: threads 0 - 127 of dy, the others of x
  const int lt = (tid & 127) >> 3, lc = (tid & 7) * PW;
  for (int64_t t = t0; t < t1; t += VK) {
    float v[PW];
    const bool ok = t + lt < t1 && (tid < 128 ? m0 + lc < a.M : n0 + lc < a.N);
    if (tid < 128) {
      Raw8<BF> r;
      r.zero();
      if (ok) r.load(a.dy, (t + lt) * a.lddy + m0 + lc);
      r.get(v);
    } else {
      RawP r;
      r.zero();
      if (ok) r.load(a.x, t + lt, n0 + lc);
      r.get(v);
    }
    __syncthreads();
    float* d = tid < 128 ? &As[lt][lc] : &Bs[lt][lc];
#pragma unroll
    for (int i = 0; i < PW; ++i) d[i] = v[i];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < VK; ++k) {
      const float4 x = *reinterpret_cast<const float4*>(&As[k][ty * 4]);
      const float4 y = *reinterpret_cast<const float4*>(&Bs[k][tx * 4]);
      const float xa[4] = {x.x, x.y, x.z, x.w}, ya[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] += xa[i] * ya[j];
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = m0 + ty * 4 + i, n = n0 + tx * 4;
    if (m >= a.M || n >= a.N) continue;
    float* o = split ? a.part + ((int64_t)blockIdx.z * a.M + m) * a.N + n : a.dw + (int64_t)m * a.lddw + n;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (split) o[j] = acc[i][j];
      else o[j] = (a.accumulate ? o[j] : 0.f) + a.scale * acc[i][j];
    }
  }
}

static EpiArgs grad_epi(const WgradArgs& a) {
  EpiArgs e;
  memset(&e, 0, sizeof(e));
  e.kind = EPI_GRAD;
  e.out = a.dw;
  e.ldo = a.lddw;
  e.out_dtype = F32;
  e.scale = a.scale;
  e.accumulate = a.accumulate;
  return e;
}

template <bool BF>
static hipError_t wgrad_valu(const WgradArgs& a, hipStream_t s) {
  const int nx = (a.N + VT - 1) / VT, ny = (a.M + VT - 1) / VT;
  if (ny > 65535) return hipErrorInvalidValue;
  // splits of at least 256 tokens until there are four blocks per CU
  int64_t nz = 1024 / ((int64_t)nx * ny);
  if (nz > a.T / 256) nz = a.T / 256;
  const int64_t room = a.part ? (int64_t)(a.part_elems / ((size_t)a.M * a.N)) : 0;
  if (nz > room) nz = room;
  if (nz < 1) nz = 1;
  int64_t per = (a.T + nz - 1) / nz;
  per = (per + VK - 1) / VK * VK;
  nz = a.T > 0 ? (a.T + per - 1) / per : 1;
  hipLaunchKernelGGL((wgrad_valu_kernel<BF>), dim3(nx, ny, (unsigned)nz), dim3(256), 0, s, a, per, nz > 1);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || nz == 1) return e;
  return launch_splitk_reduce(a.part, (int)nz, a.M, a.N, grad_epi(a), s);
}

hipError_t launch_wgrad_packed(const WgradArgs& a, int dtype, hipStream_t s) {
  return dtype == BF16 ? wgrad_valu<true>(a, s) : wgrad_valu<false>(a, s);
}

}  // namespace zl
