// Norms around a block (include/zl_layer.h, zl_block_norm): the norm of a
// block's output, its gate and residual scale, the addition to the residual
// stream and the norm before the next block, in one pass over the rows, forward
// and backward.  Bound by memory: forward 12 to 18 bytes a column with bf16
// products, backward 17 to 19.
#include "layer.h"
#include "packed.h"

namespace zl {

// Sums over the NW waves of a row (nw at run time where NW is 0).  red: two
// buffers used in turn, so one barrier per sum.
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// ----------------------------------------------------------------- forward
// NW waves per row, lane columns 8 (64 NW k + lane), k < G: the row stays in
// registers between its sums (variance from centred values).
template <int NW, int G, bool BI, bool BO>
__global__ void __launch_bounds__(256) block_norm_fwd_kernel(zl_norm_args a) {
  __shared__ float red[2][4];
  const int lane = threadIdx.x % (64 * NW);
  const int64_t r = (int64_t)blockIdx.x * (4 / NW) + threadIdx.x / (64 * NW);
  if (NW == 1 && r >= a.T) return;
  int par = 0;
  auto row_sum = [&](float v) __attribute__((always_inline)) {
    v = lanes_sum(v);
    if (NW == 1) return v;
    if ((threadIdx.x & 63) == 0) red[par][threadIdx.x >> 6] = v;
    __syncthreads();
    v = (red[par][0] + red[par][1]) + (red[par][2] + red[par][3]);
    par ^= 1;
    return v;
  };
  // centred in place, 1 / deviation returned
  auto centre = [&](float (&v)[G][PW], float& mu) __attribute__((always_inline)) {
    mu = 0.f;
    if (a.layernorm) {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < G; ++k)
#pragma unroll
        for (int i = 0; i < PW; ++i) s += v[k][i];
      mu = row_sum(s) / a.d;
    }
    float q = 0.f;
#pragma unroll
    for (int k = 0; k < G; ++k) {
      const bool ok = (k * 64 * NW + lane) * PW < a.d;
#pragma unroll
      for (int i = 0; i < PW; ++i) {
        v[k][i] -= mu;
        q += ok ? v[k][i] * v[k][i] : 0.f;
      }
    }
    return 1.f / sqrtf(row_sum(q) / a.d + a.eps);
  };

  const bool post = a.w_post != nullptr;
  Raw8<false> rx[G];
  Raw8<BI> ry[G];
#pragma unroll
  for (int k = 0; k < G; ++k) {
    const int c = (k * 64 * NW + lane) * PW;
    rx[k].zero();
    ry[k].zero();
    if (c < a.d) {
      rx[k].load(a.x, r * a.ldx + c);
      if (post) ry[k].load(a.y, r * a.ldy + c);
    }
  }
  float x[G][PW];
#pragma unroll
  for (int k = 0; k < G; ++k) rx[k].get(x[k]);
  float m0 = 0.f, r0 = 0.f, m1 = 0.f, r1 = 0.f;
  if (post) {
    float y[G][PW];
#pragma unroll
    for (int k = 0; k < G; ++k) {
      ry[k].get(y[k]);
      if (a.y_packed.codes) {
        const int c = (k * 64 * NW + lane) * PW;
        uint32_t sb;
        const uint2 code = pack8(y[k], sb);
        if (c < a.d) store_packed(a.y_packed, r, c, code, sb);
      }
    }
    r0 = centre(y, m0);
    const float* gate = a.gate ? a.gate + r / a.gate_rows * a.d : nullptr;
#pragma unroll
    for (int k = 0; k < G; ++k) {
      const int c = (k * 64 * NW + lane) * PW;
      if (c >= a.d) continue;
      float w[PW], b[PW], g[PW];
      Raw8<false> t;
      t.load(a.w_post, c);
      t.get(w);
      t.zero();
      if (a.b_post) t.load(a.b_post, c);
      t.get(b);
#pragma unroll
      for (int i = 0; i < PW; ++i) g[i] = a.scale;
      if (gate) {
        t.load(gate, c);
        t.get(g);
#pragma unroll
        for (int i = 0; i < PW; ++i) g[i] *= a.scale;
      }
#pragma unroll
      for (int i = 0; i < PW; ++i) x[k][i] += g[i] * (y[k][i] * r0 * w[i] + b[i]);
      store8<false>(a.xo, r * a.ldx + c, x[k]);
    }
  }
  if (a.w_pre) {
    r1 = centre(x, m1);
#pragma unroll
    for (int k = 0; k < G; ++k) {
      const int c = (k * 64 * NW + lane) * PW;
      float o[PW];
#pragma unroll
      for (int i = 0; i < PW; ++i) o[i] = 0.f;
      if (c < a.d) {
        float w[PW], b[PW];
        Raw8<false> t;
        t.load(a.w_pre, c);
        t.get(w);
        t.zero();
        if (a.b_pre) t.load(a.b_pre, c);
        t.get(b);
#pragma unroll
        for (int i = 0; i < PW; ++i) o[i] = x[k][i] * r1 * w[i] + b[i];
        store8<BO>(a.n, r * a.ldn + c, o);
      }
      if (a.n_packed.codes) {
        if (BO)
#pragma unroll
          for (int i = 0; i < PW; i += 2) {  // the copy of n holds n as stored
            const uint32_t p = pack_bf16(o[i], o[i + 1]);
            o[i] = __uint_as_float(p << 16);
            o[i + 1] = __uint_as_float(p & 0xffff0000u);
          }
        uint32_t sb;
        const uint2 code = pack8(o, sb);
        if (c < a.d) store_packed(a.n_packed, r, c, code, sb);
      }
    }
  }
  if (lane == 0) *reinterpret_cast<float4*>(a.stats + r * 4) = make_float4(m0, r0, m1, r1);
}

template <int NW, int G>
static hipError_t norm_fwd_go(const zl_norm_args& a, hipStream_t s) {
  const int64_t nb = (a.T + 4 / NW - 1) / (4 / NW);
  if (nb > 0x7fffffff) return hipErrorInvalidValue;
  const dim3 g((unsigned)nb), b(256);
  const bool bi = a.in_dtype == ZL_BF16, bo = a.out_dtype == ZL_BF16;
  if (bi && bo) hipLaunchKernelGGL((block_norm_fwd_kernel<NW, G, true, true>), g, b, 0, s, a);
  else if (bi) hipLaunchKernelGGL((block_norm_fwd_kernel<NW, G, true, false>), g, b, 0, s, a);
  else if (bo) hipLaunchKernelGGL((block_norm_fwd_kernel<NW, G, false, true>), g, b, 0, s, a);
  else hipLaunchKernelGGL((block_norm_fwd_kernel<NW, G, false, false>), g, b, 0, s, a);
  return hipGetLastError();
}

hipError_t launch_block_norm(const zl_norm_args& a, hipStream_t s) {
  if (a.T <= 0) return hipSuccess;
  // a wave per row where there are rows for eight waves a CU and a row fits its
  // registers, else a block per row
  if (a.T >= 2048 && a.d <= 2048) {
    if (a.d <= 512) return norm_fwd_go<1, 1>(a, s);
    if (a.d <= 1024) return norm_fwd_go<1, 2>(a, s);
    return norm_fwd_go<1, 4>(a, s);
  }
  if (a.d <= 2048) return norm_fwd_go<4, 1>(a, s);
  if (a.d <= 4096) return norm_fwd_go<4, 2>(a, s);
  return norm_fwd_go<4, 4>(a, s);
}

// ---------------------------------------------------------------- backward
// A block per run of rows, 8 columns per thread; D = dL/dxo:
//   g = dn w_pre:  D = dxo + r1 (g - mean(g) - xh mean(g xh))   (mean(g): LayerNorm)
//   dp = scale gate D, q = dp w_post:  dy = r0 (q - mean(q) - yh mean(q yh))
// The parameters' sums over the block's rows stay in registers and go to
// one partial row per block (no atomics); a second kernel adds those.
// The next row is loaded while this one is reduced.  Rows of over 4096 columns
// take 1024 threads, which leaves 128 registers each: LEAN reads the row when
// it is due and the weights and the gate once per row (from the caches).
// What the norm after the block sums needs the gate row only once for a run of
// rows that share it: with S1 = sum D yh and S0 = sum D,
//   dgate = scale (w_post S1 + b_post S0),  dw_post = scale gate S1,  db_post = scale gate S0.
// MULTI: a block has several gate rows (whole ones) and adds up the latter two.
template <bool BI, bool PK> struct RawY : Raw8<BI> {
  __device__ __forceinline__ void fetch(const zl_norm_args& a, int64_t r, int c) { this->load(a.y, r * a.ldy + c); }
};
template <bool BI> struct RawY<BI, true> : RawP {
  __device__ __forceinline__ void fetch(const zl_norm_args& a, int64_t r, int c) { this->load(a.y_packed, r, c); }
};

template <int MAXT, bool LEAN, bool MULTI, bool LN, bool BI, bool PK>
__global__ void __launch_bounds__(MAXT) block_norm_bwd_kernel(zl_norm_args a, NormPlan pl) {
  __shared__ float red[2][2][MAXT / 64];
  const int tid = threadIdx.x, c = tid * PW, nw = blockDim.x >> 6;
  const bool ok = c < a.d, pre = a.w_pre != nullptr, post = a.w_post != nullptr;
  int64_t r0, r1;
  if (pl.group > 0) {
    const int64_t gi = blockIdx.x / pl.cpg, ci = blockIdx.x % pl.cpg;
    r0 = gi * pl.group + ci * pl.rpb;
    r1 = min(min(r0 + pl.rpb, (gi + 1) * pl.group), a.T);
  } else {
    r0 = blockIdx.x * pl.rpb;
    r1 = min(r0 + pl.rpb, a.T);
  }
  float wp[PW], wq[PW];  // w_pre, w_post
  auto vec = [&](const float* p, float (&v)[PW]) __attribute__((always_inline)) {
    Raw8<false> t;
    t.zero();
    if (ok && p) t.load(p, c);
    t.get(v);
  };
  if (!LEAN) {
    vec(a.w_pre, wp);
    vec(a.w_post, wq);
  }
  // gradient sums: the norm before the next block, S1 and S0, and MULTI's own
  float swp[PW], sbp[PW], s1[PW], s0[PW], swq[PW], sbq[PW], gt[PW];
#pragma unroll
  for (int i = 0; i < PW; ++i) {
    swp[i] = sbp[i] = s1[i] = s0[i] = swq[i] = sbq[i] = 0.f;
    gt[i] = a.scale;
  }
  // scale * the gate row of r
  auto load_gate = [&](int64_t r) __attribute__((always_inline)) {
    vec(a.gate + r / a.gate_rows * a.d, gt);
#pragma unroll
    for (int i = 0; i < PW; ++i) gt[i] *= a.scale;
  };
  if (!LEAN && !MULTI && a.gate && r0 < r1) load_gate(r0);
  Raw8<false> nd, nx;
  Raw8<BI> nn;
  RawY<BI, PK> ny;
  float4 nst;
  auto fetch = [&](int64_t r) __attribute__((always_inline)) {
    nd.zero();
    nx.zero();
    nn.zero();
    ny.zero();
    nst = *reinterpret_cast<const float4*>(a.stats + r * 4);
    if (!ok) return;
    if (a.dxo) nd.load(a.dxo, r * a.ldx + c);
    if (pre) {
      nx.load(a.xo, r * a.ldx + c);
      nn.load(a.dn, r * a.ldn + c);
    }
    if (post) ny.fetch(a, r, c);
  };
  int par = 0;
  auto sums = [&](float& u, float& v) __attribute__((always_inline)) {
    u = lanes_sum(u);
    if (LN) v = lanes_sum(v);
    if (nw == 1) return;
    if ((tid & 63) == 0) {
      red[par][0][tid >> 6] = u;
      red[par][1][tid >> 6] = v;
    }
    __syncthreads();
    u = v = 0.f;
    for (int w = 0; w < nw; ++w) {
      u += red[par][0][w];
      v += red[par][1][w];
    }
    par ^= 1;
  };
  if (!LEAN && r0 < r1) fetch(r0);
  int64_t left = 0;  // rows of the current gate row still to come in this block
  for (int64_t r = r0; r < r1; ++r) {
    if (LEAN) fetch(r);
    float dv[PW], xv[PW], nv[PW], yv[PW];
    nd.get(dv);
    nx.get(xv);
    nn.get(nv);
    ny.get(yv);
    const float4 st = nst;
    if (!LEAN && r + 1 < r1) fetch(r + 1);
    if (a.gate && (LEAN || (MULTI && left == 0))) load_gate(r);
    if (MULTI && left == 0) left = min(a.gate_rows, r1 - r);
    if (pre) {
      if (LEAN) vec(a.w_pre, wp);
      float u = 0.f, v = 0.f, g[PW];
#pragma unroll
      for (int i = 0; i < PW; ++i) {
        xv[i] = (xv[i] - st.z) * st.w;
        g[i] = nv[i] * wp[i];
        u += g[i] * xv[i];
        v += g[i];
        swp[i] += nv[i] * xv[i];
        if (LN) sbp[i] += nv[i];
      }
      sums(u, v);
      u /= a.d;
      v = LN ? v / a.d : 0.f;
#pragma unroll
      for (int i = 0; i < PW; ++i) dv[i] += st.w * (g[i] - v - xv[i] * u);
    }
    if (ok) store8<false>(a.dx, r * a.ldx + c, dv);
    if (post) {
      if (LEAN) vec(a.w_post, wq);
      float u = 0.f, v = 0.f, q[PW];
#pragma unroll
      for (int i = 0; i < PW; ++i) {
        yv[i] = (yv[i] - st.x) * st.y;
        const float dp = gt[i] * dv[i];
        q[i] = dp * wq[i];
        u += q[i] * yv[i];
        v += q[i];
        s1[i] += dv[i] * yv[i];
        if (LN) s0[i] += dv[i];
      }
      sums(u, v);
      u /= a.d;
      v = LN ? v / a.d : 0.f;
#pragma unroll
      for (int i = 0; i < PW; ++i) q[i] = st.y * (q[i] - v - yv[i] * u);
      if (ok) {
        if (a.out_dtype == ZL_BF16) store8<true>(a.dy, r * a.ldy + c, q);
        else store8<false>(a.dy, r * a.ldy + c, q);
      }
    }
    if (MULTI && post && --left == 0) {  // all rows of this gate row were this block's
      if (a.dgate && ok) {
        const int64_t o = r / a.gate_rows * a.d + c;
        float t[PW], w[PW], b[PW];
        vec(a.accumulate ? a.dgate + (o - c) : nullptr, t);
        vec(a.w_post, w);
        vec(LN ? a.b_post : nullptr, b);
#pragma unroll
        for (int i = 0; i < PW; ++i) t[i] += a.grad_scale * a.scale * (w[i] * s1[i] + b[i] * s0[i]);
        store8<false>(a.dgate, o, t);
      }
#pragma unroll
      for (int i = 0; i < PW; ++i) {
        swq[i] += gt[i] * s1[i];
        if (LN) sbq[i] += gt[i] * s0[i];
        s1[i] = s0[i] = 0.f;
      }
    }
  }
  if (!ok) return;
  float* part = a.workspace + blockIdx.x * (int64_t)a.d + c;
  const int64_t step = pl.nblk * a.d;
  if (a.dw_pre) store8<false>(part, 0, swp);
  if (LN && a.db_pre) store8<false>(part, step, sbp);
  if (!post) return;
  if (!MULTI) {
    if (LEAN && a.gate && r0 < r1) load_gate(r0);
    if (a.dgate) {
      float w[PW], b[PW], t[PW];
      vec(a.w_post, w);
      vec(LN ? a.b_post : nullptr, b);
#pragma unroll
      for (int i = 0; i < PW; ++i) t[i] = a.scale * (w[i] * s1[i] + b[i] * s0[i]);
      store8<false>(part, 4 * step, t);
    }
#pragma unroll
    for (int i = 0; i < PW; ++i) {
      swq[i] = gt[i] * s1[i];
      sbq[i] = gt[i] * s0[i];
    }
  }
  if (a.dw_post) store8<false>(part, 2 * step, swq);
  if (LN && a.db_post) store8<false>(part, 3 * step, sbq);
}

// out = (accumulate ? out : 0) + scale * sum of partial rows, in a fixed order:
// a block has 32 columns and 32 groups of rows with 8 loads in flight each.
// blockIdx.y: dw_pre, db_pre, dw_post, db_post, then the gate rows.
__global__ void __launch_bounds__(1024) block_norm_reduce_kernel(zl_norm_args a, NormPlan pl) {
  __shared__ float red[32][33];
  const int task = blockIdx.y;
  float* out = task == 0 ? a.dw_pre : task == 1 ? a.db_pre : task == 2 ? a.dw_post : task == 3 ? a.db_post : a.dgate;
  if (!out) return;
  const int64_t step = pl.nblk * a.d;
  const float* part = a.workspace + (task < 4 ? task : 4) * step;
  int64_t n = pl.nblk;
  if (task >= 4) {
    n = pl.cpg;
    part += (task - 4) * pl.cpg * a.d;
    out += (int64_t)(task - 4) * a.d;
  }
  const int cl = threadIdx.x & 31, grp = threadIdx.x >> 5;
  const int j = blockIdx.x * 32 + cl, jc = min(j, a.d - 1);
  float t = 0.f;
  for (int64_t b = grp; b < n; b += 256) {
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = part[min(b + 32 * k, n - 1) * a.d + jc];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = b + 32 * k < n ? v[k] : 0.f;
    t += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
  }
  red[grp][cl] = t;
  __syncthreads();
  if (grp == 0 && j < a.d) {
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 32; ++k) s[k & 3] += red[k][cl];
    const float v = a.grad_scale * ((s[0] + s[1]) + (s[2] + s[3]));
    out[j] = a.accumulate ? out[j] + v : v;
  }
}

NormPlan norm_plan(int64_t T, int d, int64_t gate_rows) {
  if (T <= 0) return {0, 0, 0, 0};
  // four waves per SIMD, but not below 8 rows a block (partial rows cost what
  // rows cost) until there are fewer blocks than CUs
  const int waves = (d + 64 * PW - 1) / (64 * PW);
  int64_t blocks = 256 * 16 / waves;
  if (blocks > 1024) blocks = 1024;
  if (blocks > T / 8) blocks = T / 8;
  if (blocks < 256) blocks = T < 256 ? T : 256;
  NormPlan p = {0, (T + blocks - 1) / blocks, 0, 0};
  if (gate_rows > T) gate_rows = T;
  if (gate_rows >= p.rpb) {
    p.group = gate_rows;
    p.cpg = (gate_rows + p.rpb - 1) / p.rpb;
    p.rpb = (gate_rows + p.cpg - 1) / p.cpg;
    p.nblk = (T + gate_rows - 1) / gate_rows * p.cpg;
  } else {
    if (gate_rows > 0) p.rpb = p.rpb / gate_rows * gate_rows;
    p.nblk = (T + p.rpb - 1) / p.rpb;
  }
  return p;
}

template <int MAXT, bool LEAN, bool MULTI, bool LN>
static void norm_bwd_types(const zl_norm_args& a, const NormPlan& pl, int threads, hipStream_t s) {
  const dim3 g((unsigned)pl.nblk), b(threads);
  const bool bi = a.in_dtype == ZL_BF16, pk = a.w_post && a.y_packed.codes;
  if (bi && pk) hipLaunchKernelGGL((block_norm_bwd_kernel<MAXT, LEAN, MULTI, LN, true, true>), g, b, 0, s, a, pl);
  else if (bi) hipLaunchKernelGGL((block_norm_bwd_kernel<MAXT, LEAN, MULTI, LN, true, false>), g, b, 0, s, a, pl);
  else if (pk) hipLaunchKernelGGL((block_norm_bwd_kernel<MAXT, LEAN, MULTI, LN, false, true>), g, b, 0, s, a, pl);
  else hipLaunchKernelGGL((block_norm_bwd_kernel<MAXT, LEAN, MULTI, LN, false, false>), g, b, 0, s, a, pl);
}

template <int MAXT, bool LEAN>
static void norm_bwd_go(const zl_norm_args& a, const NormPlan& pl, int threads, hipStream_t s) {
  const bool multi = a.gate && a.w_post && pl.group == 0;
  if (a.layernorm) {
    if (multi) norm_bwd_types<MAXT, LEAN, true, true>(a, pl, threads, s);
    else norm_bwd_types<MAXT, LEAN, false, true>(a, pl, threads, s);
  } else {
    if (multi) norm_bwd_types<MAXT, LEAN, true, false>(a, pl, threads, s);
    else norm_bwd_types<MAXT, LEAN, false, false>(a, pl, threads, s);
  }
}

hipError_t launch_block_norm_bwd(const zl_norm_args& a, hipStream_t s) {
  float* const out[4] = {a.dw_pre, a.db_pre, a.dw_post, a.db_post};
  if (a.T <= 0) {  // sums over no rows
    for (float* o : out)
      if (o && !a.accumulate)
        if (hipError_t e = launch_zero_block(o, a.d, 0, 1, 0, a.d, s)) return e;
    return hipSuccess;
  }
  const NormPlan pl = norm_plan(a.T, a.d, a.gate ? a.gate_rows : 0);
  if (pl.nblk > 0x7fffffff) return hipErrorInvalidValue;
  const int threads = (a.d + 64 * PW - 1) / (64 * PW) * 64;
  if (threads <= 256) norm_bwd_go<256, false>(a, pl, threads, s);
  else if (threads <= 512) norm_bwd_go<512, false>(a, pl, threads, s);
  else norm_bwd_go<1024, true>(a, pl, threads, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const bool gate = a.dgate && pl.group > 0;
  if (!gate && !out[0] && !out[1] && !out[2] && !out[3]) return hipSuccess;
  const int64_t tasks = 4 + (gate ? pl.nblk / pl.cpg : 0);
  if (tasks > 65535) return hipErrorInvalidValue;
  hipLaunchKernelGGL(block_norm_reduce_kernel, dim3((a.d + 31) / 32, (unsigned)tasks), dim3(1024), 0, s, a, pl);
  return hipGetLastError();
}

}  // namespace zl
