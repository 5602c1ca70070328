// Norms around a block (include/zl_layer.h, zl_block_norm): the norm of a
// block's output, its gate and residual scale, the addition to the residual
// stream and the norm before the next block, in one pass over the rows, forward
// and backward.  Bound by memory: with bf16 products 12 bytes a column forward
// (14 with both copies), 17 to 18 backward.
#include "layer.h"
#include "packed.h"

namespace zl {

// The sum of a wave's lanes, in every lane: within rows of 16 by DPP moves (lane
// bits 0 and 1, then the mirrored lane of 8 and of 16), two exchanges beyond.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float lanes_sum(float v) {
  v = dpp_add<0x140>(dpp_add<0x141>(dpp_add<0x4E>(dpp_add<0xB1>(v))));
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// ----------------------------------------------------------------- forward
// NW waves per row, lane columns 8 (64 NW k + lane), k < G: the row stays in
// registers between its sums (variance from centred values).
template <int NW, int G, bool BI, bool BO, bool NT>
__global__ void __launch_bounds__(256) block_norm_fwd_kernel(zl_norm_args a) {
  __shared__ float red[2][4];
  const int lane = threadIdx.x % (64 * NW);
  const int64_t r = (int64_t)blockIdx.x * (4 / NW) + __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * NW));
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
      rx[k].load(a.x, r * a.ldx, c);
      if (post) ry[k].load(a.y, r * a.ldy, c);
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
        if (c < a.d) store_packed<NT>(a.y_packed, r, c, code, sb);
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
      t.load(a.w_post, 0, c);
      t.get(w);
      t.zero();
      if (a.b_post) t.load(a.b_post, 0, c);
      t.get(b);
#pragma unroll
      for (int i = 0; i < PW; ++i) g[i] = a.scale;
      if (gate) {
        t.load(gate, 0, c);
        t.get(g);
#pragma unroll
        for (int i = 0; i < PW; ++i) g[i] *= a.scale;
      }
#pragma unroll
      for (int i = 0; i < PW; ++i) x[k][i] += g[i] * (y[k][i] * r0 * w[i] + b[i]);
      store8<false>(a.xo, r * a.ldx, c, x[k]);
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
        t.load(a.w_pre, 0, c);
        t.get(w);
        t.zero();
        if (a.b_pre) t.load(a.b_pre, 0, c);
        t.get(b);
#pragma unroll
        for (int i = 0; i < PW; ++i) o[i] = x[k][i] * r1 * w[i] + b[i];
        store8<BO, NT>(a.n, r * a.ldn, c, o);
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
        if (c < a.d) store_packed<NT>(a.n_packed, r, c, code, sb);
      }
    }
  }
  if (lane == 0) *reinterpret_cast<float4*>(a.stats + r * 4) = make_float4(m0, r0, m1, r1);
}

template <int NW, int G, bool NT>
static void norm_fwd_types(const zl_norm_args& a, dim3 g, hipStream_t s) {
  const dim3 b(256);
  const bool bi = a.in_dtype == ZL_BF16, bo = a.out_dtype == ZL_BF16;
  if (bi && bo) hipLaunchKernelGGL((block_norm_fwd_kernel<NW, G, true, true, NT>), g, b, 0, s, a);
  else if (bi) hipLaunchKernelGGL((block_norm_fwd_kernel<NW, G, true, false, NT>), g, b, 0, s, a);
  else if (bo) hipLaunchKernelGGL((block_norm_fwd_kernel<NW, G, false, true, NT>), g, b, 0, s, a);
  else hipLaunchKernelGGL((block_norm_fwd_kernel<NW, G, false, false, NT>), g, b, 0, s, a);
}
template <int NW, int G>
static hipError_t norm_fwd_go(const zl_norm_args& a, hipStream_t s) {
  const int64_t nb = (a.T + 4 / NW - 1) / (4 / NW);
  if (nb > MAX_BLOCKS) return hipErrorInvalidValue;
  // xo, n and the copies
  const int64_t out = a.T * a.d * ((a.w_post ? 4 : 0) + (a.w_pre ? (a.out_dtype == ZL_BF16 ? 2 : 4) : 0) +
                                   (a.y_packed.codes ? 1 : 0) + (a.n_packed.codes ? 1 : 0));
  if (streaming(out, 0)) norm_fwd_types<NW, G, true>(a, dim3((unsigned)nb), s);
  else norm_fwd_types<NW, G, false>(a, dim3((unsigned)nb), s);
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
// A block has slots of waves, each with rows of its own; a thread has G groups
// of 8 columns.  Rows go round the slots of all blocks, so that what is read at
// one time lies together (a run of rows per block, the runs a power of two apart:
// 251 us at 16384 x 4096 where this took 237; 8192 x 2048: 72 and 67).  With D = dL/dxo:
//   g = dn w_pre:  D = dxo + r1 (g - mean(g) - xh mean(g xh))   (mean(g): LayerNorm)
//   dp = scale gate D, q = dp w_post:  dy = r0 (q - mean(q) - yh mean(q yh))
// The parameters' sums over the block's rows stay in registers, meet across
// slots in LDS and go to one partial row per block (no atomics); a second kernel
// adds those.  What the norm after the block sums needs the gate row only once
// for a run of rows that share it: with S1 = sum D yh and S0 = sum D,
//   dgate = scale (w_post S1 + b_post S0),  dw_post = scale gate S1,  db_post = scale gate S0.
// MODE 0: a slot's rows share a gate row (or have none).  1: a slot has whole gate
// rows, short ones, and adds up the latter two; dgate is its own to write.  2: a
// slot's rows go through all of a few long gate rows, with a partial dgate of
// each (16384 x 4096, 4 gate rows: 215 us; in mode 0, which reads four places at a
// time, 232, and 223 with twice the blocks).
// The next row is loaded while this one is reduced; LEAN (registers short):
// the row is read when it is due, weights and gate once per row (from the caches).
template <bool BI, bool PK> struct RawY : Raw8<BI> {
  __device__ __forceinline__ void fetch(const zl_norm_args& a, int64_t r, uint32_t c) { this->load(a.y, r * a.ldy, c); }
};
template <bool BI> struct RawY<BI, true> : RawP {
  __device__ __forceinline__ void fetch(const zl_norm_args& a, int64_t r, uint32_t c) { this->load(a.y_packed, r, c); }
};

template <int NT, int G, bool LEAN, int MODE, bool LN, bool BI, bool PK>
__global__ void __launch_bounds__(NT) block_norm_bwd_kernel(zl_norm_args a, NormPlan pl) {
  constexpr int NW = NT / 64;
  __shared__ float red[2][2][NW];
  __shared__ float comb[G == 1 ? 3 * 64 * PW : 1];  // slots 1 ..: 3 of one wave or 1 of two
  // LEAN: the sums over gate rows, touched once per gate row, lie in LDS
  constexpr bool SL = LEAN && MODE == 1;
  __shared__ float sq[SL ? (LN ? 2 : 1) * G * PW * NT : 1];
  // waves of a slot, this wave's slot and its place there
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nw = NW / pl.slots, slot = wave / nw, lane = threadIdx.x & 63;
  const int tid = (wave - slot * nw) * 64 + lane, gs = nw * 64 * PW;  // columns of one group
  const bool pre = a.w_pre != nullptr, post = a.w_post != nullptr;
  uint32_t col[G];
  bool ok[G];
#pragma unroll
  for (int k = 0; k < G; ++k) {
    col[k] = k * gs + tid * PW;
    ok[k] = (int)col[k] < a.d;
  }
  // this slot's first row, the end of what it shares, and the rows from a unit
  // of `unit` rows (one gate row in mode 1) to this slot's next
  const int64_t unit = MODE == 1 ? a.gate_rows : 1;
  int64_t r0, end, step;
  if (pl.group > 0) {
    const int64_t gi = blockIdx.x / pl.cpg, ci = blockIdx.x % pl.cpg;
    r0 = gi * pl.group + ci * pl.slots + slot;
    end = min((gi + 1) * pl.group, a.T);
    step = pl.cpg * pl.slots;
  } else {
    r0 = ((int64_t)blockIdx.x * pl.slots + slot) * unit;
    end = a.T;
    step = pl.nblk * pl.slots * unit;
  }
  auto vec = [&](const float* p, int k, float (&v)[PW]) __attribute__((always_inline)) {
    Raw8<false> t;
    t.zero();
    if (ok[k] && p) t.load(p, 0, col[k]);
    t.get(v);
  };
  float wp[G][PW], wq[G][PW], gt[G][PW];  // w_pre, w_post, scale * gate
  // gradient sums: of the norm before the next block, S1 and S0, and over gate rows
  float swp[G][PW], sbp[G][PW], s1[G][PW], s0[G][PW], swq[G][PW], sbq[G][PW];
  auto load_gate = [&](int64_t r) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < G; ++k) {
      vec(a.gate + r / a.gate_rows * a.d, k, gt[k]);
#pragma unroll
      for (int i = 0; i < PW; ++i) gt[k][i] *= a.scale;
    }
  };
#pragma unroll
  for (int k = 0; k < G; ++k) {
    if (!LEAN) {
      vec(a.w_pre, k, wp[k]);
      vec(a.w_post, k, wq[k]);
    }
#pragma unroll
    for (int i = 0; i < PW; ++i) {
      swp[k][i] = sbp[k][i] = s1[k][i] = s0[k][i] = swq[k][i] = sbq[k][i] = 0.f;
      gt[k][i] = a.scale;
      if (SL) sq[(k * PW + i) * NT + threadIdx.x] = 0.f;
      if (SL && LN) sq[((G + k) * PW + i) * NT + threadIdx.x] = 0.f;
    }
  }
  if (!LEAN && MODE == 0 && a.gate && r0 < end) load_gate(r0);
  Raw8<false> nd[G], nx[G];
  Raw8<BI> nn[G];
  RawY<BI, PK> ny[G];
  float4 nst;
  constexpr bool LATE = LEAN && MODE == 1 && LN && !BI;  // registers shortest: y when it is due
  auto fetch = [&](int64_t r) __attribute__((always_inline)) {
    nst = *reinterpret_cast<const float4*>(a.stats + r * 4);
#pragma unroll
    for (int k = 0; k < G; ++k) {
      if (!ok[k]) continue;
      if (a.dxo) nd[k].load(a.dxo, r * a.ldx, col[k]);
      if (pre) {
        nx[k].load(a.xo, r * a.ldx, col[k]);
        nn[k].load(a.dn, r * a.ldn, col[k]);
      }
      if (post && !LATE) ny[k].fetch(a, r, col[k]);
    }
  };
  nst = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int k = 0; k < G; ++k) {
    nd[k].zero();
    nx[k].zero();
    nn[k].zero();
    ny[k].zero();
  }
  int par = 0;
  auto sums = [&](float& u, float& v) __attribute__((always_inline)) {
    u = lanes_sum(u);
    if (LN) v = lanes_sum(v);
    if (nw == 1) return;
    if (lane == 0) {
      red[par][0][wave] = u;
      red[par][1][wave] = v;
    }
    __syncthreads();
    // lane l takes the sum of wave l % nw (nw is a power of two)
    u = red[par][0][slot * nw + (lane & (nw - 1))];
    v = LN ? red[par][1][slot * nw + (lane & (nw - 1))] : 0.f;
    for (int o = 1; o < nw; o <<= 1) {
      u += __shfl_xor(u, o, 64);
      if (LN) v += __shfl_xor(v, o, 64);
    }
    par ^= 1;
  };
  if (!LEAN && r0 < end) fetch(r0);
  int64_t r = r0, at_unit = 0;  // this round's row and its place in its unit
  // mode 2: whether this is the slot's first row of a gate row, which, and the row behind it
  bool fresh = true;
  int64_t gate_row = -1, gate_end = 0;
  // t += f scale (w_post S1 + b_post S0)
  auto gate_grad = [&](int k, float f, float (&t)[PW]) __attribute__((always_inline)) {
    float w[PW], b[PW];
    vec(a.w_post, k, w);
    vec(LN ? a.b_post : nullptr, k, b);
#pragma unroll
    for (int i = 0; i < PW; ++i) t[i] += f * a.scale * (w[i] * s1[k][i] + b[i] * s0[k][i]);
  };
  const int64_t pstep = pl.nblk * a.d;  // floats of one array of partial rows
  // every slot takes the same number of rounds (barriers); rows past the end count nothing
  for (int64_t k0 = 0; k0 < pl.rows; ++k0) {
    const bool in = r < end;
    const int64_t next = MODE == 1 && at_unit + 1 < unit ? r + 1 : r + step - (unit - 1);
    if (MODE == 2 && in && fresh) {
      gate_row = r / a.gate_rows;
      gate_end = (gate_row + 1) * a.gate_rows;
    }
    // the slot's last row of its gate row
    const bool last = MODE == 1 ? at_unit + 1 == unit || r + 1 >= end : next >= gate_end || next >= end;
    if (LEAN && in) fetch(r);
    Raw8<false> rd[G], rx[G];
    Raw8<BI> rn[G];
    RawY<BI, PK> ry[G];
#pragma unroll
    for (int k = 0; k < G; ++k) {
      rd[k] = nd[k];
      rx[k] = nx[k];
      rn[k] = nn[k];
      ry[k] = ny[k];
    }
    const float4 st = nst;
    if (!LEAN && next < end) fetch(next);
    if (in && a.gate && (LEAN || (MODE == 1 && at_unit == 0) || (MODE == 2 && fresh))) load_gate(r);
    if (MODE == 2) fresh = false;
    float dv[G][PW];
#pragma unroll
    for (int k = 0; k < G; ++k) rd[k].get(dv[k]);
    if (pre) {
      float u = 0.f, v = 0.f, g[G][PW], xv[G][PW];
#pragma unroll
      for (int k = 0; k < G; ++k) {
        float nv[PW];
        if (LEAN) vec(a.w_pre, k, wp[k]);
        rx[k].get(xv[k]);
        rn[k].get(nv);
#pragma unroll
        for (int i = 0; i < PW; ++i) {
          xv[k][i] = (xv[k][i] - st.z) * st.w;
          g[k][i] = nv[i] * wp[k][i];
          u += g[k][i] * xv[k][i];
          v += g[k][i];
          if (in) {
            swp[k][i] += nv[i] * xv[k][i];
            if (LN) sbp[k][i] += nv[i];
          }
        }
      }
      sums(u, v);
      u /= a.d;
      v = LN ? v / a.d : 0.f;
#pragma unroll
      for (int k = 0; k < G; ++k)
#pragma unroll
        for (int i = 0; i < PW; ++i) dv[k][i] += st.w * (g[k][i] - v - xv[k][i] * u);
    }
#pragma unroll
    for (int k = 0; k < G; ++k)
      if (in && ok[k]) store8<false>(a.dx, r * a.ldx, col[k], dv[k]);
    if (post) {
      float u = 0.f, v = 0.f, q[G][PW], yv[G][PW];
#pragma unroll
      for (int k = 0; k < G; ++k) {
        if (LEAN) vec(a.w_post, k, wq[k]);
        if (LATE && in && ok[k]) ry[k].fetch(a, r, col[k]);
        ry[k].get(yv[k]);
#pragma unroll
        for (int i = 0; i < PW; ++i) {
          yv[k][i] = (yv[k][i] - st.x) * st.y;
          q[k][i] = gt[k][i] * dv[k][i] * wq[k][i];
          u += q[k][i] * yv[k][i];
          v += q[k][i];
          if (in) {
            s1[k][i] += dv[k][i] * yv[k][i];
            if (LN) s0[k][i] += dv[k][i];
          }
        }
      }
      sums(u, v);
      u /= a.d;
      v = LN ? v / a.d : 0.f;
#pragma unroll
      for (int k = 0; k < G; ++k) {
#pragma unroll
        for (int i = 0; i < PW; ++i) q[k][i] = st.y * (q[k][i] - v - yv[k][i] * u);
        if (in && ok[k]) {
          if (a.out_dtype == ZL_BF16) store8<true>(a.dy, r * a.ldy, col[k], q[k]);
          else store8<false>(a.dy, r * a.ldy, col[k], q[k]);
        }
      }
    }
    if (MODE != 0 && in && last) {
      if (MODE == 2) fresh = true;
#pragma unroll
      for (int k = 0; k < G; ++k) {
        if (a.dgate && ok[k]) {
          float t[PW] = {};
          if (MODE == 1) {
            const int64_t o = r / a.gate_rows * a.d;
            vec(a.accumulate ? a.dgate + o : nullptr, k, t);
            gate_grad(k, a.grad_scale, t);
            store8<false>(a.dgate, o, col[k], t);
          } else {
            gate_grad(k, 1.f, t);
            store8<false>(a.workspace, 4 * pstep + ((gate_row * pl.nblk + blockIdx.x) * pl.slots + slot) * a.d, col[k], t);
          }
        }
#pragma unroll
        for (int i = 0; i < PW; ++i) {
          if (SL) {
            sq[(k * PW + i) * NT + threadIdx.x] += gt[k][i] * s1[k][i];
            if (LN) sq[((G + k) * PW + i) * NT + threadIdx.x] += gt[k][i] * s0[k][i];
          } else {
            swq[k][i] += gt[k][i] * s1[k][i];
            if (LN) sbq[k][i] += gt[k][i] * s0[k][i];
          }
          s1[k][i] = s0[k][i] = 0.f;
        }
      }
    }
    if (MODE == 1) at_unit = at_unit + 1 < unit ? at_unit + 1 : 0;
    r = next;
  }
  // a last, shorter gate row that this slot had no row of
  if (MODE == 2 && a.dgate)
    for (int64_t g = gate_row + 1; g < pl.gates; ++g)
#pragma unroll
      for (int k = 0; k < G; ++k) {
        const float none[PW] = {};
        if (ok[k])
          store8<false>(a.workspace, 4 * pstep + ((g * pl.nblk + blockIdx.x) * pl.slots + slot) * a.d, col[k], none);
      }
  // the slots' sums, then this block's partial row `which`
  auto finish = [&](int which, int k, float (&v)[PW]) __attribute__((always_inline)) {
    if (G == 1 && pl.slots > 1) {
      __syncthreads();
      if (slot > 0)
#pragma unroll
        for (int i = 0; i < PW; ++i) comb[((slot - 1) * PW + i) * nw * 64 + tid] = v[i];
      __syncthreads();
      if (slot > 0) return;
      for (int t = 1; t < pl.slots; ++t)
#pragma unroll
        for (int i = 0; i < PW; ++i) v[i] += comb[((t - 1) * PW + i) * nw * 64 + tid];
    }
    if (ok[k]) store8<false>(a.workspace, which * pstep + blockIdx.x * (int64_t)a.d, col[k], v);
  };
  if (MODE == 0 && LEAN && a.gate && r0 < end) load_gate(r0);
#pragma unroll
  for (int k = 0; k < G; ++k) {
    if (a.dw_pre) finish(0, k, swp[k]);
    if (LN && a.db_pre) finish(1, k, sbp[k]);
    if (!post) continue;
#pragma unroll
    for (int i = 0; i < PW; ++i) {
      if (MODE == 0) {
        swq[k][i] = gt[k][i] * s1[k][i];
        sbq[k][i] = gt[k][i] * s0[k][i];
      } else if (SL) {
        swq[k][i] = sq[(k * PW + i) * NT + threadIdx.x];
        if (LN) sbq[k][i] = sq[((G + k) * PW + i) * NT + threadIdx.x];
      }
    }
    if (a.dw_post) finish(2, k, swq[k]);
    if (LN && a.db_post) finish(3, k, sbq[k]);
    if (MODE == 0 && a.dgate) {
      float t[PW] = {};
      gate_grad(k, 1.f, t);
      finish(4, k, t);
    }
  }
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
    n = pl.group > 0 ? pl.cpg : pl.nblk * pl.slots;
    part += (task - 4) * n * a.d;
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
  // rows of up to 512 columns: a wave each, four in a block, and so on
  const int slots = d <= 64 * PW ? 4 : d <= 128 * PW ? 2 : 1;
  NormPlan p = {0, 0, 0, 0, 0, 0, slots};
  if (T <= 0) return p;
  // as many blocks as are resident or half as many more rounds of them would gain
  // (2048 columns and fewer: three a CU measured 66.4 us at 8192 x 2048 where two
  // take 62.6, above one and two at 16384 x 4096 220 and 227), with 8 rows each at
  // least (partial rows cost what two rows cost) until there are fewer than CUs
  int64_t blocks = d <= 256 * PW ? 512 : 256;
  if (blocks > T / 8) blocks = T / 8;
  const int64_t most = (T + slots - 1) / slots;
  if (blocks < 256) blocks = most < 256 ? most : 256;
  p.rows = (T + blocks * slots - 1) / (blocks * slots);
  if (gate_rows > T) gate_rows = T;
  const int64_t gates = gate_rows > 0 ? (T + gate_rows - 1) / gate_rows : 0;
  // (above 4096 columns mode 2 lacks the registers for the next row: 4096 x 8192 157 us, 136 in mode 0)
  if (gates > 1 && gates <= 16 && gate_rows >= 4 * blocks * slots && d <= 512 * PW) {
    p.nblk = (T + p.rows * slots - 1) / (p.rows * slots);
    p.gates = gates;
    p.gate_part = gates * p.nblk * slots;
  } else if (gate_rows >= p.rows * slots) {
    // blocks of their own for every gate row, or (below) whole gate rows for a slot, which
    // leaves slots idle just below the border (128 and 127 rows at 65536 x 256: 61 and 152 us;
    // 64 and 63 at 16384 x 1024: 60 and 66; 32 and 31 at 16384 x 512: 42 and 44)
    p.group = gate_rows;
    p.cpg = (gate_rows + p.rows * slots - 1) / (p.rows * slots);
    p.rows = (gate_rows + p.cpg * slots - 1) / (p.cpg * slots);
    p.nblk = p.gate_part = gates * p.cpg;
  } else {
    if (gate_rows > 0) p.rows = p.rows > gate_rows ? p.rows / gate_rows * gate_rows : gate_rows;
    p.nblk = (T + p.rows * slots - 1) / (p.rows * slots);
  }
  return p;
}

template <int NT, int G, bool LEAN, int MODE, bool LN>
static void norm_bwd_types(const zl_norm_args& a, const NormPlan& pl, hipStream_t s) {
  const dim3 g((unsigned)pl.nblk), b(NT);
  const bool bi = a.in_dtype == ZL_BF16, pk = a.w_post && a.y_packed.codes;
  constexpr bool L32 = LEAN || G == 2;  // fp32 dn and y: twice the registers of a row in flight
  if (bi && pk) hipLaunchKernelGGL((block_norm_bwd_kernel<NT, G, LEAN, MODE, LN, true, true>), g, b, 0, s, a, pl);
  else if (bi) hipLaunchKernelGGL((block_norm_bwd_kernel<NT, G, LEAN, MODE, LN, true, false>), g, b, 0, s, a, pl);
  else if (pk) hipLaunchKernelGGL((block_norm_bwd_kernel<NT, G, LEAN, MODE, LN, false, true>), g, b, 0, s, a, pl);
  else hipLaunchKernelGGL((block_norm_bwd_kernel<NT, G, L32, MODE, LN, false, false>), g, b, 0, s, a, pl);
}

template <int NT, int G>
static void norm_bwd_go(const zl_norm_args& a, const NormPlan& pl, hipStream_t s) {
  const int mode = !a.gate || pl.group > 0 ? 0 : pl.gates > 0 ? 2 : 1;
  if (a.layernorm) {
    if (mode == 0) norm_bwd_types<NT, G, G == 2, 0, true>(a, pl, s);
    else if (mode == 1) norm_bwd_types<NT, G, G == 2, 1, true>(a, pl, s);
    else if constexpr (G == 1) norm_bwd_types<NT, G, false, 2, true>(a, pl, s);
  } else {
    if (mode == 0) norm_bwd_types<NT, G, false, 0, false>(a, pl, s);
    else if (mode == 1) norm_bwd_types<NT, G, G == 2, 1, false>(a, pl, s);
    else if constexpr (G == 1) norm_bwd_types<NT, G, false, 2, false>(a, pl, s);
  }
}

hipError_t launch_block_norm_bwd(const zl_norm_args& args, hipStream_t s) {
  zl_norm_args a = args;
  if (a.gate_rows > a.T) a.gate_rows = a.T;  // one gate row; products with it stay within 64 bits
  float* const out[4] = {a.dw_pre, a.db_pre, a.dw_post, a.db_post};
  if (a.T <= 0) {  // sums over no rows
    for (float* o : out)
      if (o && !a.accumulate)
        if (hipError_t e = launch_zero_block(o, a.d, 0, 1, 0, a.d, s)) return e;
    return hipSuccess;
  }
  const NormPlan pl = norm_plan(a.T, a.d, a.gate ? a.gate_rows : 0);
  // 8 columns a thread up to 4096 (16 on half the threads: 237 us at 16384 x 4096
  // where this takes 223), 16 above (8 on 1024 threads, registers short: 150 us at
  // 4096 x 8192 where this takes 134)
  if (a.d <= 256 * PW) norm_bwd_go<256, 1>(a, pl, s);
  else if (a.d <= 512 * PW) norm_bwd_go<512, 1>(a, pl, s);
  else norm_bwd_go<512, 2>(a, pl, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const bool gate = a.dgate && pl.gate_part > 0;
  if (!gate && !out[0] && !out[1] && !out[2] && !out[3]) return hipSuccess;
  // one task per gate row with partial rows: fewer than the blocks, a few thousand
  const int64_t tasks = 4 + (!gate ? 0 : pl.group > 0 ? pl.nblk / pl.cpg : pl.gates);
  hipLaunchKernelGGL(block_norm_reduce_kernel, dim3((a.d + 31) / 32, (unsigned)tasks), dim3(1024), 0, s, a, pl);
  return hipGetLastError();
}

}  // namespace zl
