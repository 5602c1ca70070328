// Elementwise layer operators: packing activations to 8 bits and back, the
// MLP activation with its packed pre-activations, rotary positions with several
// axes.  All bound by memory: each operand is read and written once, 16 bytes
// (8 for codes) per lane and access.
#include "gemm_epilogue.h"  // gelu
#include "layer.h"
#include "packed.h"

namespace zl {

constexpr int LT = 256;  // threads per block

// Columns to lanes, rows to blocks: a row takes 2^l2 lanes of 8 columns each
// (whole 32-column blocks), ncx column chunks of them where it is longer; a
// block has LT / 2^l2 rows at once, U times.  A row longer than a block's lanes
// goes in chunks of 128 or 64 lanes where that leaves an eighth fewer lanes past
// its end (pack and unpack of 8192 x 2056 bf16: 26.5 us in chunks of 256 lanes,
// 22.5 so).  Groups of columns dealt out without regard to rows leave none, but
// measured slower on long rows (SwiGLU backward 16384 x 14336: 401 us, 378 so).
struct RowGrid {
  int l2, ncx;
  int64_t T;
};
static RowGrid row_grid(int64_t T, int n) {
  const int lanes = (n + PBLK - 1) / PBLK * (PBLK / PW);
  int l2 = 2;
  while ((1 << l2) < lanes && (1 << l2) < LT) ++l2;
  auto padded = [&](int l) { return (lanes + (1 << l) - 1) >> l << l; };
  if (lanes > LT)
    for (int l = 7; l >= 6; --l)
      if (padded(l) * 8 <= padded(l2) * 7) l2 = l;
  return {l2, (lanes + (1 << l2) - 1) >> l2, T};
}
static int64_t row_blocks(const RowGrid& g, int U) {
  const int64_t rows = (int64_t)(LT >> g.l2) * U;
  return (g.T + rows - 1) / rows * g.ncx;
}
// This thread's first column and rows row(u), u < U.
struct RowPos {
  int col, step;
  int64_t r0;
  __device__ __forceinline__ RowPos(const RowGrid& g, int U) {
    const int cx = (int)(blockIdx.x % (unsigned)g.ncx), ry = (int)(blockIdx.x / (unsigned)g.ncx);
    step = LT >> g.l2;
    col = ((cx << g.l2) + ((int)threadIdx.x & ((1 << g.l2) - 1))) * PW;
    r0 = (int64_t)ry * step * U + (threadIdx.x >> g.l2);
  }
  __device__ __forceinline__ int64_t row(int u) const { return r0 + (int64_t)u * step; }
};

// How a call's accesses stream past the caches (NT of the kernels): 1, the stores,
// where the outputs are larger than the L2s (32 MB) and so leave them before
// the next kernel reads them; 2, the loads too, where the inputs are larger by far
// than the Infinity Cache (256 MB).  SwiGLU 16384 x 14336 forward 337, 325, 306 us for
// 0, 1, 2, backward 398, 380, 383; GELU 4096 x 3200 backward 22.5, 19.0, 20.7; pack
// and unpack 4096 x 4096 (16 MB of codes) 17.7, 19.1, 20.1.
int streaming(int64_t out, int64_t in) { return out <= (32 << 20) ? 0 : in <= (384 << 20) ? 1 : 2; }

// ------------------------------------------------------------ pack, unpack
// All loads of the U rows are in flight before the first is used.
template <bool BF, int U, int NT>
__global__ void __launch_bounds__(LT) pack_kernel(RowGrid g, int n, const void* __restrict__ x, int64_t ldx,
                                                  zl_packed out) {
  const RowPos p(g, U);
  Raw8<BF> raw[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    raw[u].zero();
    if (p.col < n && p.row(u) < g.T) raw[u].template load<(NT > 1)>(x, p.row(u) * ldx + p.col);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float v[PW];
    uint32_t sb;
    raw[u].get(v);
    const uint2 c = pack8(v, sb);  // every lane of a block, also past the row's end
    if (p.col < n && p.row(u) < g.T) store_packed<(NT > 0)>(out, p.row(u), p.col, c, sb);
  }
}

template <bool BF, int U, bool NT>
__global__ void __launch_bounds__(LT) unpack_kernel(RowGrid g, int n, zl_packed in, void* __restrict__ x,
                                                    int64_t ldx) {
  const RowPos p(g, U);
  if (p.col >= n) return;
  RawP raw[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    raw[u].zero();
    if (p.row(u) < g.T) raw[u].load(in, p.row(u), p.col);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (p.row(u) >= g.T) break;
    float v[PW];
    raw[u].get(v);
    store8<BF, NT>(x, p.row(u) * ldx + p.col, 0, v);
  }
}

// One row per thread where that gives no more than four blocks per CU (few
// rows: latency counts), else U rows in flight.
static bool few(const RowGrid& g) { return row_blocks(g, 1) <= 1024; }

// f(blocks, U, NT) with compile-time U and NT: U rows per thread where there are
// many, and streaming accesses only there.
template <int N> using Int = std::integral_constant<int, N>;
template <int U, typename F>
static hipError_t launch_rows(const RowGrid& g, int nt, F&& f) {
  if (g.T <= 0) return hipSuccess;
  const bool one = few(g);
  const int64_t b = row_blocks(g, one ? 1 : U);
  if (b > MAX_BLOCKS) return hipErrorInvalidValue;
  const dim3 grid((unsigned)b);
  if (one) f(grid, Int<1>{}, Int<0>{});
  else if (nt == 0) f(grid, Int<U>{}, Int<0>{});
  else if (nt == 1) f(grid, Int<U>{}, Int<1>{});
  else f(grid, Int<U>{}, Int<2>{});
  return hipGetLastError();
}

template <bool BF>
static hipError_t pack_go(int64_t T, int n, const void* x, int64_t ldx, const zl_packed& out, hipStream_t s) {
  const RowGrid g = row_grid(T, n);
  return launch_rows<4>(g, streaming(T * n, T * n * (BF ? 2 : 4)), [&](dim3 b, auto u, auto nt) {
    hipLaunchKernelGGL((pack_kernel<BF, u(), nt()>), b, dim3(LT), 0, s, g, n, x, ldx, out);
  });
}
hipError_t launch_pack(int64_t T, int n, const void* x, int64_t ldx, int dtype, const zl_packed& out, hipStream_t s) {
  return dtype == BF16 ? pack_go<true>(T, n, x, ldx, out, s) : pack_go<false>(T, n, x, ldx, out, s);
}

template <bool BF>
static hipError_t unpack_go(int64_t T, int n, const zl_packed& in, void* x, int64_t ldx, hipStream_t s) {
  const RowGrid g = row_grid(T, n);
  return launch_rows<4>(g, streaming(T * n * (BF ? 2 : 4), 0), [&](dim3 b, auto u, auto nt) {
    hipLaunchKernelGGL((unpack_kernel<BF, u(), (nt() > 0)>), b, dim3(LT), 0, s, g, n, in, x, ldx);
  });
}
hipError_t launch_unpack(int64_t T, int n, const zl_packed& in, void* x, int64_t ldx, int dtype, hipStream_t s) {
  return dtype == BF16 ? unpack_go<true>(T, n, in, x, ldx, s) : unpack_go<false>(T, n, in, x, ldx, s);
}

// -------------------------------------------------------------- activation
__device__ __forceinline__ float sigmoid_f(float x) { return __builtin_amdgcn_rcpf(1.f + __expf(-x)); }

// SW: gate | up, lane columns col and ff + col; else GELU.  PK: also packs h.
template <bool SW, bool PK, bool BI, bool BO, int U, int NT>
__global__ void __launch_bounds__(LT) mlp_fwd_kernel(RowGrid g, zl_mlp_args a) {
  const RowPos p(g, U);
  Raw8<BI> rg[U], ru[SW ? U : 1];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const bool ok = p.col < a.ff && p.row(u) < g.T;
    rg[u].zero();
    if (ok) rg[u].template load<(NT > 1)>(a.h, p.row(u) * a.ldh + p.col);
    if constexpr (SW) {
      ru[u].zero();
      if (ok) ru[u].template load<(NT > 1)>(a.h, p.row(u) * a.ldh + a.ff + p.col);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t r = p.row(u);
    const bool ok = p.col < a.ff && r < g.T;
    float x[PW], y[PW], o[PW];
    rg[u].get(x);
    if constexpr (SW) ru[u].get(y);
#pragma unroll
    for (int k = 0; k < PW; ++k) o[k] = SW ? x[k] * sigmoid_f(x[k]) * y[k] : gelu_f(x[k]);
    if (ok) store8<BO, (NT > 0)>(a.a, r * a.lda + p.col, 0, o);
    if constexpr (PK) {
      uint32_t sb;
      uint2 c = pack8(x, sb);
      if (ok) store_packed<(NT > 0)>(a.packed, r, p.col, c, sb);
      if constexpr (SW) {
        c = pack8(y, sb);
        if (ok) store_packed<(NT > 0)>(a.packed, r, a.ff + p.col, c, sb);
      }
    }
  }
}

// h from memory or from its packed copy.
template <bool BI, bool PK> struct RawH : Raw8<BI> {
  __device__ __forceinline__ void fetch(const zl_mlp_args& a, int64_t r, int col) { this->load(a.h, r * a.ldh + col); }
};
template <bool BI> struct RawH<BI, true> : RawP {
  __device__ __forceinline__ void fetch(const zl_mlp_args& a, int64_t r, int col) { this->load(a.packed, r, col); }
};

template <bool SW, bool PK, bool BI, bool BO, int U, int NT>
__global__ void __launch_bounds__(LT) mlp_bwd_kernel(RowGrid g, zl_mlp_args a) {
  const RowPos p(g, U);
  if (p.col >= a.ff) return;
  RawH<BI, PK> rg[U], ru[SW ? U : 1];
  Raw8<BI> rd[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t r = p.row(u);
    rg[u].zero();
    rd[u].zero();
    if constexpr (SW) ru[u].zero();
    if (r < g.T) {
      rg[u].fetch(a, r, p.col);
      if constexpr (SW) ru[u].fetch(a, r, a.ff + p.col);
      rd[u].load(a.da, r * a.ldda + p.col);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t r = p.row(u);
    if (r >= g.T) break;
    float x[PW], y[PW], d[PW], o[PW], dg[PW], du[PW];
    rg[u].get(x);
    rd[u].get(d);
    if constexpr (SW) {
      ru[u].get(y);
#pragma unroll
      for (int k = 0; k < PW; ++k) {
        const float s = sigmoid_f(x[k]), silu = x[k] * s;
        o[k] = silu * y[k];
        dg[k] = d[k] * y[k] * (s * (1.f + x[k] * (1.f - s)));
        du[k] = d[k] * silu;
      }
      store8<BO, (NT > 0)>(a.dh, r * a.lddh + a.ff + p.col, 0, du);
    } else {
#pragma unroll
      for (int k = 0; k < PW; ++k) {
        o[k] = gelu_f(x[k]);
        dg[k] = d[k] * gelu_grad_f(x[k]);
      }
    }
    store8<BO, (NT > 0)>(a.dh, r * a.lddh + p.col, 0, dg);
    if (a.a) store8<BO, (NT > 0)>(a.a, r * a.lda + p.col, 0, o);
  }
}

template <bool SW, bool PK, bool BI, bool BO>
static hipError_t mlp_go(const zl_mlp_args& a, bool backward, hipStream_t s) {
  const RowGrid g = row_grid(a.T, a.ff);
  const int64_t n = a.T * a.ff, nh = (SW ? 2 : 1) * n;
  const int64_t ei = BI ? 2 : 4, eo = BO ? 2 : 4;
  if (backward)  // loads that stream gained nothing here
    return launch_rows<2>(g, streaming(nh * eo + (a.a ? n * eo : 0), 0), [&](dim3 b, auto u, auto nt) {
      hipLaunchKernelGGL((mlp_bwd_kernel<SW, PK, BI, BO, u(), (nt() > 0)>), b, dim3(LT), 0, s, g, a);
    });
  return launch_rows<2>(g, streaming(n * eo + (PK ? nh : 0), nh * ei), [&](dim3 b, auto u, auto nt) {
    hipLaunchKernelGGL((mlp_fwd_kernel<SW, PK, BI, BO, u(), nt()>), b, dim3(LT), 0, s, g, a);
  });
}
template <bool SW, bool PK>
static hipError_t mlp_types(const zl_mlp_args& a, bool backward, hipStream_t s) {
  const bool bi = a.in_dtype == ZL_BF16, bo = a.out_dtype == ZL_BF16;
  if (bi && bo) return mlp_go<SW, PK, true, true>(a, backward, s);
  if (bi) return mlp_go<SW, PK, true, false>(a, backward, s);
  if (bo) return mlp_go<SW, PK, false, true>(a, backward, s);
  return mlp_go<SW, PK, false, false>(a, backward, s);
}
hipError_t launch_mlp(const zl_mlp_args& a, bool backward, hipStream_t s) {
  const bool sw = a.kind == ZL_MLP_SWIGLU, pk = a.packed.codes != nullptr;
  if (sw) return pk ? mlp_types<true, true>(a, backward, s) : mlp_types<true, false>(a, backward, s);
  return pk ? mlp_types<false, true>(a, backward, s) : mlp_types<false, false>(a, backward, s);
}

// ------------------------------------------------------------------ rotary
// A block has TB tokens: the angles' cosines and sines first (at most one
// per thread; 64-bit product, whole turns dropped, then fp32), kept in LDS for
// all heads of the token; then the pairs, V columns of either half per lane.
// grid.y splits the heads where there are few tokens.  V = 8 on aligned rows whose
// rotated half is whole groups of 8, else one column a lane, bound by its accesses of
// 2 or 4 bytes (16384 x 40 heads of 128, bf16 52 us and 110, fp32 132 and 140).
template <bool BF, int V>
__device__ __forceinline__ void load_cols(const void* p, int64_t i, float (&v)[V]) {
  if constexpr (V == PW) {
    Raw8<BF> r;
    r.load(p, i);
    r.get(v);
  } else {
    v[0] = BF ? bf16_to_f32(static_cast<const bf16_t*>(p)[i]) : static_cast<const float*>(p)[i];
  }
}
template <bool BF, int V, bool NT>
__device__ __forceinline__ void store_cols(void* p, int64_t i, const float (&v)[V]) {
  if constexpr (V == PW) store8<BF, NT>(p, i, 0, v);
  else if (BF) static_cast<bf16_t*>(p)[i] = f32_to_bf16(v[0]);
  else static_cast<float*>(p)[i] = v[0];
}

template <bool BF, int V, bool NT>
__global__ void __launch_bounds__(LT) rotary_kernel(RotaryArgs a, int tb, int hpb) {
  __shared__ __align__(16) float cs[LT], sn[LT];
  const int64_t t0 = (int64_t)blockIdx.x * tb;
  const int nt = (int)min((int64_t)tb, a.T - t0);
  if ((int)threadIdx.x < nt * a.half) {
    const int t = threadIdx.x / a.half, j = threadIdx.x % a.half;
    double w = (double)a.pos[(int64_t)a.axis[j] * a.T + t0 + t] * a.turns[j];
    w -= rint(w);
    float s, c;
    sincospif(2.f * (float)w, &s, &c);
    cs[threadIdx.x] = c;
    sn[threadIdx.x] = a.sign * s;
  }
  __syncthreads();
  const int h0 = blockIdx.y * hpb, nh = min(hpb, a.heads - h0);
  const int per = a.half / V;  // lanes per head
  const int row = nh * per;
  for (int i = threadIdx.x; i < nt * row; i += LT) {
    const int t = i / row, q = i - t * row, h = q / per, j = (q - h * per) * V;
    const int64_t col = (int64_t)(h0 + h) * a.hd + j;
    const int64_t xi = (t0 + t) * a.ldx + col, oi = (t0 + t) * a.ldo + col;
    float x[V], y[V], p[V], r[V];
    load_cols<BF, V>(a.x, xi, x);
    load_cols<BF, V>(a.x, xi + a.half, y);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const float c = cs[t * a.half + j + k], s = sn[t * a.half + j + k];
      p[k] = x[k] * c - y[k] * s;
      r[k] = y[k] * c + x[k] * s;
    }
    store_cols<BF, V, NT>(a.out, oi, p);
    store_cols<BF, V, NT>(a.out, oi + a.half, r);
  }
  const int rest = a.hd - 2 * a.half;
  if (rest == 0 || (a.out == a.x && a.ldo == a.ldx)) return;
  const int rper = rest / V, rrow = nh * rper;
  for (int i = threadIdx.x; i < nt * rrow; i += LT) {
    const int t = i / rrow, q = i - t * rrow, h = q / rper;
    const int64_t col = (int64_t)(h0 + h) * a.hd + 2 * a.half + (q - h * rper) * V;
    float x[V];
    load_cols<BF, V>(a.x, (t0 + t) * a.ldx + col, x);
    store_cols<BF, V, NT>(a.out, (t0 + t) * a.ldo + col, x);
  }
}

template <bool BF, int V>
static hipError_t rotary_go(const RotaryArgs& a, hipStream_t s) {
  const int tb = LT / a.half;
  const int64_t bx = (a.T + tb - 1) / tb;
  if (bx > MAX_BLOCKS) return hipErrorInvalidValue;
  // fewer than two blocks per CU: heads spread over blocks, whole lanes' worth
  // of pairs each
  int by = 1;
  while (bx * by < 512 && by < a.heads && (int64_t)tb * (a.heads / (2 * by)) * (a.half / V) >= LT) by *= 2;
  const int hpb = (a.heads + by - 1) / by;
  const dim3 grid((unsigned)bx, (a.heads + hpb - 1) / hpb);
  // whole lines: halves of 128 bytes and more, no columns left over
  const bool nt = BF && V == PW && a.half >= 64 && a.hd == 2 * a.half && streaming(a.T * a.heads * a.hd * 2, 0) > 0;
  if (nt) hipLaunchKernelGGL((rotary_kernel<BF, V, BF && V == PW>), grid, dim3(LT), 0, s, a, tb, hpb);
  else hipLaunchKernelGGL((rotary_kernel<BF, V, false>), grid, dim3(LT), 0, s, a, tb, hpb);
  return hipGetLastError();
}
hipError_t launch_rotary(const RotaryArgs& a, int dtype, hipStream_t s) {
  if (a.T <= 0) return hipSuccess;
  if (dtype == BF16) return a.vec ? rotary_go<true, PW>(a, s) : rotary_go<true, 1>(a, s);
  return a.vec ? rotary_go<false, PW>(a, s) : rotary_go<false, 1>(a, s);
}

}  // namespace zl
