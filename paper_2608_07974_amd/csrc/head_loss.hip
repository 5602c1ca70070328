// Loss of a readout head z = x w^T without its logits (include/zl_loss.h).
//
// Forward: the product's tiles leave, per row and column block, the largest logit
// and the sum of exponentials, and the logits of the teacher's ids (the matrix unit's
// accumulators are the only place where z exists); a kernel over the rows joins them.
// Backward, a piece of the vocabulary at a time: the product again, whose tiles
// write dL/dz (bf16 or fp32); the named columns' values over it; two products from
// there.
#include <string.h>

#include "gemm_tiles.h"
#include "loss.h"
#include "loss_rows.h"

namespace zl {

// ----------------------------------------------------------------- epilogues
// Tiles are taken transposed (EpiTransposed): a lane holds, for one row each of FM
// row blocks, four consecutive columns at a time, so a row's sums need two steps
// across lanes and its constants one load.

// The teacher's distinct ids of every row, found again in the tiles: ids in ascending
// order [T, k]; of every row and column block (a wave tile's columns) a span [T, ldb]: where
// its ids begin (8 bits), the first one's column in the block (8), where they end (16; 0:
// there are none); their logits [T, k], in that order.  Dot products of their own read k
// rows of w for each row of x (2117 x 1802 x 3824 bf16 with 60 ids: 220 us of forward, 84 so).
struct NamedCols {
  const int32_t* order;
  const uint32_t* span;  // null: no teacher
  int64_t ldb;
  float* z;
  int k;
};
// Partial sums.  PAIR false: (max z, sum exp((z - max) c)) over all columns but the label.
// PAIR true: those of z at c = 1 over all but the label, and of z at c over all, or (other)
// the columns that the teacher does not name.  The label's logit leaves from the tile that
// holds it, so that it is the one that the row's other logits were formed with (a dot product
// of its own differs in its last bits, and CE may be below 0 then).
template <bool PAIR>
struct StatEpi {
  float c2;               // log2(e) / tau
  float* part;            // [blocks, T, 2 or 4]
  int64_t T;
  NamedCols named;
  bool other;
  const int32_t* labels;  // or null
  float* stats;           // [T, 4 + named.k], the label's logit in column 3
};
// dL/dz of the columns [0, N) of a piece, zeros up to the row stride:
//   GRAD_ONE   ct exp(z / tau - lt)
//   GRAD_TWO   c1 exp(z - l1) + ct exp(z / tau - lt)
//   GRAD_SQUARE  the same at tau = 2, where with e = exp(z / 2 - lt) the first term is
//     c1 exp(2 lt - l1) e^2 (c1 holds the product): one exponential for two
enum { GRAD_ONE, GRAD_TWO, GRAD_SQUARE };
template <int MODE>
struct GradEpi {
  const float4* coef;     // [T]: c1, l1, ct, lt
  float inv;              // 1 / tau
  void* dz;
  int64_t ldz;
  int dtype;
};
// out = (accumulate ? out : 0) + scale * *gmax * C, or fp32 partials of split z.  Rows that
// are not live add 0 (dx: where w is infinite or NaN, C is NaN though dL/dz is 0).
struct OutEpi {
  void* out;
  int64_t ldo;
  int dtype;
  float scale;
  const float* gmax;      // or null
  int accumulate;
  int64_t zstride;
  const int32_t* live;    // [M] or null
};
// The epilogue of split z of K.
template <typename E> __device__ __forceinline__ E split_part(const E& e, int) { return e; }
__device__ __forceinline__ OutEpi split_part(OutEpi e, int z) {
  e.out = static_cast<float*>(e.out) + z * e.zstride;
  return e;
}
template <bool PAIR> struct EpiTransposed<StatEpi<PAIR>> { static constexpr bool value = true; };
template <int MODE> struct EpiTransposed<GradEpi<MODE>> { static constexpr bool value = true; };
template <> struct EpiTransposed<OutEpi> { static constexpr bool value = true; };

// The lanes that hold one row are MF apart.
template <int MF, typename F>
__device__ __forceinline__ float across(float x, F&& f) {
#pragma unroll
  for (int o = MF; o < 64; o <<= 1) x = f(x, __shfl_xor(x, o, 64));
  return x;
}

// A wave's own accesses to LDS stay in order; this keeps the compiler to it.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// bf16 results of MF rows of a wave's tile, four columns a lane, leave through LDS as
// rows of 16 bytes a lane: straight from the accumulators a store would touch 16 or
// 32 rows with 32 or 16 bytes each (dL/dz of 4096 x 50257 x 768: 437 us, 394 so).  The
// region is the wave's own; its accesses to LDS stay in order.
template <int TN, int MF>
struct RowsOut {
  static constexpr int LD = TN + 8;  // elements; 16 bytes of padding spread the rows over the banks
  static constexpr int BYTES = MF * LD * 2;
  bf16_t* lds;
  int lane;
  __device__ __forceinline__ RowsOut(unsigned char* smem, int wave, int lane_)
      : lds(reinterpret_cast<bf16_t*>(smem + wave * BYTES)), lane(lane_) {}
  // columns n .. n + 3 of this lane's row
  __device__ __forceinline__ void put(int n, uint2 v) { *reinterpret_cast<uint2*>(lds + (lane & (MF - 1)) * LD + n) = v; }
  // f(row, column, 8 values)
  template <typename F>
  __device__ __forceinline__ void flush(F&& f) {
    wave_sync();
    constexpr int LPR = TN / 8;
#pragma unroll
    for (int it = 0; it < MF * LPR / 64; ++it) {
      const int r = it * (64 / LPR) + lane / LPR, c = lane % LPR * 8;
      f(r, c, *reinterpret_cast<const uint4*>(lds + r * LD + c));
    }
    wave_sync();
  }
};

template <int BM, int BN, int WM, int WN, int MF = 32, bool PAIR>
__device__ __forceinline__ void store_tile(const typename Mma<MF>::acc_t (&acc)[BM / WM / MF][BN / WN / MF],
                                           unsigned char*, const GemmDesc& g, const StatEpi<PAIR>& e, int m0, int n0,
                                           int wave, int lane) {
  constexpr int TM = BM / WM, TN = BN / WN, FM = TM / MF, FN = TN / MF, NR = Mma<MF>::NR;
  const int wm = wave / WN, wn = wave % WN;
  const int nb = n0 + wn * TN;
  if (nb >= g.N) return;
  const bool cut = nb + TN > g.N;
  const int64_t block = nb / TN;
  auto fmax2 = [](float a, float b) { return fmaxf(a, b); };
  auto add2 = [](float a, float b) { return a + b; };
  // on their way before the first sums
  uint32_t span[FM];
  int label[FM];  // its column in the block; outside [0, TN): not here
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    const int m = m0 + wm * TM + i * MF + (lane & (MF - 1));
    span[i] = e.named.span && m < g.M ? e.named.span[m * e.named.ldb + block] : 0;
    const int y = e.labels && m < g.M ? e.labels[m] : -1;
    label[i] = y >= nb && y < g.N ? y - nb : -1;
  }
  static_for<0, FM>([&](auto ic) __attribute__((always_inline)) {
    constexpr int i = decltype(ic)::value;
    const int64_t m = m0 + wm * TM + i * MF + (lane & (MF - 1));
    float v[FN * NR];
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < NR; ++r) v[j * NR + r] = acc[i][j][r];
    if (cut)
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int r = 0; r < NR; ++r)
          if (nb + j * MF + Mma<MF>::row(lane, r) >= g.N) v[j * NR + r] = -INFINITY;
    auto sums = [&](float c2, float& mx, float& s) __attribute__((always_inline)) {
      mx = across<MF>(max_of(v), fmax2);
      const float ref = mx == -INFINITY ? 0.f : mx;
      s = 0.f;
#pragma unroll
      for (int k = 0; k < FN * NR; ++k) s += __builtin_amdgcn_exp2f((v[k] - ref) * c2);
      s = across<MF>(s, add2);
    };
    // a row's lanes look for the same column, one holds it
    float zy = 0.f;
    auto label_out = [&](bool out) __attribute__((always_inline)) {
      if ((unsigned)label[i] >= (unsigned)TN) return;
      bool here = false;
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int r = 0; r < NR; ++r)
          if (label[i] == j * MF + Mma<MF>::row(lane, r)) {
            if (out) zy = v[j * NR + r];
            v[j * NR + r] = out ? -INFINITY : zy;
            here = true;
          }
      if (out && here) e.stats[m * (4 + e.named.k) + 3] = zy;
    };
    auto name = [&](bool out) __attribute__((always_inline)) {
      const int end = span[i] >> 16, first = span[i] & 0xff;
      for (int at = first; at < end; ++at) {
        const int c = at == first ? (int)(span[i] >> 8 & 0xff) : e.named.order[m * e.named.k + at] - nb;
        float z = 0.f;
        bool here = false;
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int r = 0; r < NR; ++r)
            if (c == j * MF + Mma<MF>::row(lane, r)) {
              z = v[j * NR + r];
              here = true;
              if (out) v[j * NR + r] = -INFINITY;
            }
        if (here) e.named.z[m * e.named.k + at] = z;
      }
    };
    float mx, s;
    label_out(true);
    if constexpr (!PAIR) {
      sums(e.c2, mx, s);
      if (span[i] >> 16) label_out(false);
      name(false);
      if (lane < MF && m < g.M) *reinterpret_cast<float2*>(e.part + (block * e.T + m) * 2) = make_float2(mx, s);
    } else {
      float mt, st;
      sums(LOG2E, mx, s);
      label_out(false);
      name(e.other);
      sums(e.c2, mt, st);
      if (lane < MF && m < g.M)
        *reinterpret_cast<float4*>(e.part + (block * e.T + m) * 4) = make_float4(mx, s, mt, st);
    }
  });
}

// In fp32 the exponent's argument is a difference before it is scaled; where the
// result is rounded to bf16 one fused operation does (off by |lt| 2^-24 at most, 2^-8
// follow).  Rows without a target have coefficients 0; their logits may be NaN, so
// the finished words are masked.
template <int BM, int BN, int WM, int WN, int MF = 32, int MODE>
__device__ __forceinline__ void store_tile(const typename Mma<MF>::acc_t (&acc)[BM / WM / MF][BN / WN / MF],
                                           unsigned char* smem, const GemmDesc& g, const GradEpi<MODE>& e, int m0, int n0,
                                           int wave, int lane) {
  constexpr int TM = BM / WM, TN = BN / WN, FM = TM / MF, FN = TN / MF, NR = Mma<MF>::NR;
  const int wm = wave / WN, wn = wave % WN;
  const int nb = n0 + wn * TN;
  const bool cut = nb + TN > g.N, bf = e.dtype == BF16;
  RowsOut<TN, MF> rows(smem, wave, lane);
  const float ci = e.inv * LOG2E;
  static_for<0, FM>([&](auto ic) __attribute__((always_inline)) {
    constexpr int i = decltype(ic)::value;
    const int m = m0 + wm * TM + i * MF + (lane & (MF - 1));
    float4 c = make_float4(0.f, 0.f, 0.f, 0.f);
    if (m < g.M) c = e.coef[m];
    const uint32_t live = c.x != 0.f || c.z != 0.f ? 0xffffffffu : 0u;  // (NaN is not 0)
    const float wt = c.w * LOG2E, w1 = c.y * LOG2E;
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r0 = 0; r0 < NR; r0 += 4) {
        const int n = nb + j * MF + Mma<MF>::row(lane, r0);
        float o[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float v = acc[i][j][r0 + r];
          const float p = __builtin_amdgcn_exp2f(bf ? __builtin_fmaf(v, ci, -wt) : __builtin_fmaf(v, e.inv, -c.w) * LOG2E);
          if constexpr (MODE == GRAD_ONE) {
            o[r] = c.z * p;
          } else if constexpr (MODE == GRAD_SQUARE) {
            o[r] = p * __builtin_fmaf(p, c.x, c.z);
          } else {
            const float q = __builtin_amdgcn_exp2f(bf ? __builtin_fmaf(v, LOG2E, -w1) : (v - c.y) * LOG2E);
            o[r] = __builtin_fmaf(c.x, q, c.z * p);
          }
        }
        if (cut) {
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (n + r >= g.N) o[r] = 0.f;
        }
        if (bf)
          rows.put(n - nb, make_uint2(pack_bf16(o[0], o[1]) & live, pack_bf16(o[2], o[3]) & live));
        else if (m < g.M && n < e.ldz)
          *reinterpret_cast<uint4*>(static_cast<float*>(e.dz) + m * e.ldz + n) =
              make_uint4(__builtin_bit_cast(uint32_t, o[0]) & live, __builtin_bit_cast(uint32_t, o[1]) & live,
                         __builtin_bit_cast(uint32_t, o[2]) & live, __builtin_bit_cast(uint32_t, o[3]) & live);
      }
    if (bf)
      rows.flush([&](int r, int c, uint4 v) __attribute__((always_inline)) {
        const int mr = m0 + wm * TM + i * MF + r;
        if (mr < g.M && nb + c < e.ldz) *reinterpret_cast<uint4*>(static_cast<bf16_t*>(e.dz) + mr * e.ldz + nb + c) = v;
      });
  });
}

template <int BM, int BN, int WM, int WN, int MF = 32>
__device__ __forceinline__ void store_tile(const typename Mma<MF>::acc_t (&acc)[BM / WM / MF][BN / WN / MF],
                                           unsigned char* smem, const GemmDesc& g, const OutEpi& e, int m0, int n0,
                                           int wave, int lane) {
  constexpr int TM = BM / WM, TN = BN / WN, FM = TM / MF, FN = TN / MF, NR = Mma<MF>::NR;
  const int wm = wave / WN, wn = wave % WN;
  const int nb = n0 + wn * TN;
  const float scale = e.zstride ? 1.f : e.gmax ? e.scale * *e.gmax : e.scale;
  RowsOut<TN, MF> rows(smem, wave, lane);
  static_for<0, FM>([&](auto ic) __attribute__((always_inline)) {
    constexpr int i = decltype(ic)::value;
    const int64_t m = m0 + wm * TM + i * MF + (lane & (MF - 1));
    const bool on = !e.live || (m < g.M && e.live[m] != 0);
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r0 = 0; r0 < NR; r0 += 4) {
        const int n = nb + j * MF + Mma<MF>::row(lane, r0);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (on) v = make_float4(acc[i][j][r0], acc[i][j][r0 + 1], acc[i][j][r0 + 2], acc[i][j][r0 + 3]);
        v.x *= scale;
        v.y *= scale;
        v.z *= scale;
        v.w *= scale;
        if (e.dtype == BF16) {
          rows.put(n - nb, make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w)));
        } else if (m < g.M && n < g.N) {  // N is a multiple of 8: four columns are all there or none
          float4* o = reinterpret_cast<float4*>(static_cast<float*>(e.out) + m * e.ldo + n);
          if (e.accumulate) {
            const float4 f = *o;
            v.x += f.x;
            v.y += f.y;
            v.z += f.z;
            v.w += f.w;
          }
          *o = v;
        }
      }
    if (e.dtype == BF16)
      rows.flush([&](int r, int c, uint4 v) __attribute__((always_inline)) {
        const int64_t mr = m0 + wm * TM + i * MF + r;
        if (mr < g.M && nb + c < g.N) *reinterpret_cast<uint4*>(static_cast<bf16_t*>(e.out) + mr * e.ldo + nb + c) = v;
      });
  });
}

// ------------------------------------------------------------------ products
// Bound by the matrix units: 4096 x 65536 at K 768 takes 395 us with sums (1040 TFLOP/s),
// 500 with dL/dz, whose epilogue (6 us a tile of 256 x 256) hides behind nothing; at K 3200
// 1231 and 1373 (1400 and 1250).  Blocks that stay and copy the next tile during the epilogue
// gained 2 % at K 768 and lost 0.7 % at 4096.
template <int BM, int BN, int WM, int WN, int BK, int NST, bool AK, bool BKM, int MF, typename E>
__global__ void __launch_bounds__(WM * WN * 64) head_gemm_kernel(GemmDesc g, E e, int nz) {
  extern __shared__ __align__(16) unsigned char smem[];
  const int nbm = (g.M + BM - 1) / BM, nbn = (g.N + BN - 1) / BN;
  int tm, tn, z = 0, at = blockIdx.x;
  if (nz == 1) {
    tile_coords(at, nbm, nbn, tm, tn);
  } else {
    // tiles of one split of K side by side on an XCD, which reads their operands once
    // (dx of 4096 x 50257 x 768, 48 tiles in 5 splits: 289 us, 298 in the grid's order)
    at = xcd_order(at, nbm * nbn * nz);
    z = at / (nbm * nbn);
    grouped_coords(at - z * nbm * nbn, nbm, nbn, tm, tn);
  }
  gemm_dma_body<BM, BN, WM, WN, BK, NST, 1, AK, BKM, false, false, MF>(g, split_part(e, z), tm, tn, z, smem);
}

template <int BM, int BN, int WM, int WN, bool AK, bool BKM, typename E>
static hipError_t run_head_tiles(const GemmDesc& g, const E& e, int nz, hipStream_t s) {
  constexpr int BK = KTile<AK, BKM>::BK, NST = KTile<AK, BKM>::NST, MF = KTile<AK, BKM>::MF;
  auto kern = head_gemm_kernel<BM, BN, WM, WN, BK, NST, AK, BKM, MF, E>;
  constexpr size_t lds = (size_t)NST * (BM + BN) * BK * sizeof(bf16_t);
  static_assert(lds <= 160 * 1024, "pipeline exceeds LDS");
  static_assert(WM * WN * RowsOut<BN / WN, MF>::BYTES <= lds, "rows of the epilogue exceed LDS");
  if (lds > 64 * 1024) {
    const hipError_t err = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (err != hipSuccess) return err;
  }
  const int nb = ((g.M + BM - 1) / BM) * ((g.N + BN - 1) / BN);
  hipLaunchKernelGGL(kern, dim3(nb * nz), dim3(WM * WN * 64), lds, s, g, e, nz);
  return hipGetLastError();
}
template <bool AK, bool BKM, typename E>
static hipError_t run_head(const GemmDesc& g, const E& e, bool large, hipStream_t s, int nz = 1) {
  if (large) return run_head_tiles<256, 256, 4, 2, AK, BKM>(g, e, nz, s);
  return run_head_tiles<128, 128, 2, 2, AK, BKM>(g, e, nz, s);
}

// fp32: tiles of four waves, v_mfma_f32_32x32x2_f32, 32 of K a step, the next step's
// operands in registers while one is multiplied.  A matrix instruction takes k and k + 16
// of the step (the order of a sum is free), so that a lane's share of a K-major row is 16
// consecutive floats, read 16 bytes at a time from rows as they came.
constexpr int SK = 32;
template <int R, bool KMAJ>
struct F32Stage {
  static constexpr int LD = KMAJ ? SK + 4 : R + 4, ITEMS = R * SK / 4 / 256;
  static constexpr int FLOATS = KMAJ ? R * LD : SK * LD;
  static_assert(ITEMS >= 1, "a step fills the threads");
  float4 v[ITEMS];
  // rows r0 .., those below rmax valid; k0 .., those below kmax
  __device__ __forceinline__ void load(const float* base, int64_t ld, int r0, int rmax, int k0, int kmax) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int t = (int)threadIdx.x + 256 * i;
      v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (KMAJ) {
        const int r = r0 + (t >> 3), k = k0 + (t & 7) * 4;  // kmax is a multiple of 4
        if (r < rmax && k < kmax) v[i] = *reinterpret_cast<const float4*>(base + r * ld + k);
      } else {
        const int k = k0 + t / (R / 4), r = r0 + t % (R / 4) * 4;
        if (k < kmax && r < rmax) v[i] = *reinterpret_cast<const float4*>(base + k * ld + r);  // padded rows
      }
    }
  }
  __device__ __forceinline__ void store(float* s) const {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int t = (int)threadIdx.x + 256 * i;
      *reinterpret_cast<float4*>(s + (KMAJ ? (t >> 3) * LD + (t & 7) * 4 : t / (R / 4) * LD + t % (R / 4) * 4)) = v[i];
    }
  }
  // row r at k + 0 .. 3
  __device__ static __forceinline__ void read(const float* s, int r, int k, float (&o)[4]) {
    if constexpr (KMAJ) {
      const float4 f = *reinterpret_cast<const float4*>(s + r * LD + k);
      o[0] = f.x; o[1] = f.y; o[2] = f.z; o[3] = f.w;
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) o[q] = s[(k + q) * LD + r];
    }
  }
};
template <int BM, int BN, int WM, int WN, bool AK, bool BKM, typename E>
__global__ void __launch_bounds__(256) head_f32_kernel(GemmDesc g, E e) {
  constexpr int TM = BM / WM, TN = BN / WN, FM = TM / 32, FN = TN / 32;
  static_assert(WM * WN == 4, "four waves");
  using SA = F32Stage<BM, AK>;
  using SB = F32Stage<BN, BKM>;
  constexpr int OUT = 4 * RowsOut<TN, 32>::BYTES / 4;
  constexpr int LDS = SA::FLOATS + SB::FLOATS > OUT ? SA::FLOATS + SB::FLOATS : OUT;
  __shared__ __align__(16) float lds[LDS];
  float *As = lds, *Bs = lds + SA::FLOATS;
  const int nbm = (g.M + BM - 1) / BM, nbn = (g.N + BN - 1) / BN;
  int tm, tn;
  tile_coords(blockIdx.x, nbm, nbn, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int wm = wave / WN * TM, wn = wave % WN * TN, lr = lane & 31, lk = (lane >> 5) * (SK / 2);
  const int k_lo = blockIdx.z * g.ksplit, k_hi = min(g.K, k_lo + g.ksplit);
  const int ka = min(g.ka, k_hi), kb = min(g.kb, k_hi);
  const float* A = static_cast<const float*>(g.A);
  const float* B = static_cast<const float*>(g.B);
  Mma<32>::acc_t acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  SA sa;
  SB sb;
  sa.load(A, g.lda, m0, g.M, k_lo, ka);
  sb.load(B, g.ldb, n0, g.N, k_lo, kb);
  for (int k0 = k_lo; k0 < k_hi; k0 += SK) {
    __syncthreads();  // the step before is fully read
    sa.store(As);
    sb.store(Bs);
    __syncthreads();
    sa.load(A, g.lda, m0, g.M, k0 + SK, ka);
    sb.load(B, g.ldb, n0, g.N, k0 + SK, kb);
#pragma unroll
    for (int k = 0; k < SK / 2; k += 4) {
      float a[FM][4], b[FN][4];
#pragma unroll
      for (int i = 0; i < FM; ++i) SA::read(As, wm + 32 * i + lr, lk + k, a[i]);
#pragma unroll
      for (int j = 0; j < FN; ++j) SB::read(Bs, wn + 32 * j + lr, lk + k, b[j]);
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
          for (int j = 0; j < FN; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(b[j][q], a[i][q], acc[i][j], 0, 0, 0);
    }
  }
  __syncthreads();
  store_tile<BM, BN, WM, WN, 32>(acc, reinterpret_cast<unsigned char*>(lds), g, split_part(e, blockIdx.z), m0, n0, wave, lane);
}
template <int BM, int BN, int WM, int WN, bool AK, bool BKM, typename E>
static hipError_t run_f32_tiles(const GemmDesc& g, const E& e, hipStream_t s, int nz) {
  const int nb = ((g.M + BM - 1) / BM) * ((g.N + BN - 1) / BN);
  hipLaunchKernelGGL((head_f32_kernel<BM, BN, WM, WN, AK, BKM, E>), dim3(nb, 1, nz), dim3(256), 0, s, g, e);
  return hipGetLastError();
}
// Bound by the matrix units: 4096 x 32000 x 1024 2105 us (128 TFLOP/s, the library's product
// 139), one row 100 us (128256 x 1024, 5.2 TB/s).
// Tiles by size: 32 rows where there are no more (of a product with K-major A: dw has a
// row per column of the vocabulary); 64 x 64 where those of 128 x 128, with splits of 256 of
// K at least where they may be, leave CUs idle (a matrix instruction takes 64 cycles: 64 of
// K are 3.9 us in a tile of 128 x 128, 1 in one of 64 x 64; 4096 x 1000 x 512 60.7 and 53.8 us,
// 128 x 50257 x 768 108 and 116) or would be a tenth emptier (192 x 97946 x 200 103 and 95,
// dx of 264 x 10870 x 1552 from 265 for all to 249); else 128 x 128.
enum { F32_128, F32_64, F32_32 };
static int f32_tile(int64_t M, int64_t N, int64_t split, bool ak) {
  if (ak && M <= 32) return F32_32;
  const int64_t parts = split >= 512 ? split / 256 : 1;
  const int64_t wide = ((M + 127) / 128) * ((N + 127) / 128) * 4, narrow = ((M + 63) / 64) * ((N + 63) / 64);
  if (narrow * 10 <= wide * 9 && narrow < 1 << 23) return F32_64;  // (2^31 threads)
  return ((M + 127) / 128) * ((N + 127) / 128) * parts <= 256 ? F32_64 : F32_128;
}
template <bool AK, bool BKM, typename E>
static hipError_t run_head_f32(const GemmDesc& g, const E& e, int tile, hipStream_t s, int nz = 1) {
  if constexpr (AK) {
    if (tile == F32_32) return run_f32_tiles<32, 128, 1, 4, AK, BKM>(g, e, s, nz);
  }
  if (tile == F32_64) return run_f32_tiles<64, 64, 2, 2, AK, BKM>(g, e, s, nz);
  return run_f32_tiles<128, 128, 2, 2, AK, BKM>(g, e, s, nz);
}

// Few tiles: 32 x 32 each, whose K four waves take in turns of 64 (fp32: 32), operands
// straight into registers, the next turn's while one is multiplied; the first wave
// adds the others' sums.  Both operands K-major.  Bound by the latency of a wave's turns
// (2 x 462 x 3368 bf16: 13 of them, 9 us).
template <bool BF, typename E>
__global__ void __launch_bounds__(256) head_small_kernel(GemmDesc g, E e) {
  using el = typename std::conditional<BF, bf16_t, float>::type;
  constexpr int W = 16 / sizeof(el), U = 4, TURN = 2 * W * U;
  __shared__ __align__(16) float part[3][16][64];
  static_assert(RowsOut<32, 32>::BYTES <= sizeof(part), "rows of the epilogue exceed LDS");
  const int nbm = (g.M + 31) / 32, nbn = (g.N + 31) / 32;
  int tm, tn;
  tile_coords(blockIdx.x, nbm, nbn, tm, tn);
  const int m0 = tm * 32, n0 = tn * 32;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lk = (lane >> 5) * W;
  // rows past the end are others' once more; what they add is not stored
  const el* a = static_cast<const el*>(g.A) + min(m0 + (lane & 31), g.M - 1) * g.lda + lk;
  const el* b = static_cast<const el*>(g.B) + min(n0 + (lane & 31), g.N - 1) * g.ldb + lk;
  Mma<32>::acc_t acc[1][1];
#pragma unroll
  for (int r = 0; r < 16; ++r) acc[0][0][r] = 0.f;
  auto add = [&](uint4 x, uint4 w) __attribute__((always_inline)) {
    if constexpr (BF) {
      acc[0][0] = Mma<32>::run(__builtin_bit_cast(bf16x8_t, w), __builtin_bit_cast(bf16x8_t, x), acc[0][0]);
    } else {
      const float4 fx = __builtin_bit_cast(float4, x), fw = __builtin_bit_cast(float4, w);
      acc[0][0] = __builtin_amdgcn_mfma_f32_32x32x2f32(fw.x, fx.x, acc[0][0], 0, 0, 0);
      acc[0][0] = __builtin_amdgcn_mfma_f32_32x32x2f32(fw.y, fx.y, acc[0][0], 0, 0, 0);
      acc[0][0] = __builtin_amdgcn_mfma_f32_32x32x2f32(fw.z, fx.z, acc[0][0], 0, 0, 0);
      acc[0][0] = __builtin_amdgcn_mfma_f32_32x32x2f32(fw.w, fx.w, acc[0][0], 0, 0, 0);
    }
  };
  // whole turns, two at a time: loads without conditions between them and into registers of
  // their own, so that only the turn at hand is waited for
  const int turns = g.K / TURN;
  if (wave < turns) {
    const int mine = (turns - wave + 3) / 4;
    uint4 xa[U], wa[U], xb[U], wb[U];
    auto load = [&](int i, uint4 (&x)[U], uint4 (&w)[U]) __attribute__((always_inline)) {
      const int k = (wave + 4 * min(i, mine - 1)) * TURN;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        x[u] = *reinterpret_cast<const uint4*>(a + k + 2 * W * u);
        w[u] = *reinterpret_cast<const uint4*>(b + k + 2 * W * u);
      }
      asm volatile("" ::: "memory");  // the loads stay in front of the products
      __builtin_amdgcn_sched_barrier(0);
    };
    load(0, xa, wa);
    for (int i = 0; i + 1 < mine; i += 2) {
      load(i + 1, xb, wb);
#pragma unroll
      for (int u = 0; u < U; ++u) add(xa[u], wa[u]);
      load(i + 2, xa, wa);
#pragma unroll
      for (int u = 0; u < U; ++u) add(xb[u], wb[u]);
    }
    if (mine & 1)
#pragma unroll
      for (int u = 0; u < U; ++u) add(xa[u], wa[u]);
  }
  if (wave == turns % 4)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = turns * TURN + 2 * W * u;
      uint4 x = make_uint4(0, 0, 0, 0), w = x;
      if (k + lk < g.K) {  // K is a multiple of 8
        x = *reinterpret_cast<const uint4*>(a + k);
        w = *reinterpret_cast<const uint4*>(b + k);
      }
      add(x, w);
    }
  if (wave > 0)
#pragma unroll
    for (int r = 0; r < 16; ++r) part[wave - 1][r][lane] = acc[0][0][r];
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int w = 0; w < 3; ++w)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[0][0][r] += part[w][r][lane];
  wave_sync();
  store_tile<32, 32, 1, 1, 32>(acc, reinterpret_cast<unsigned char*>(part), g, e, m0, n0, 0, lane);
}
// Up to 1024 of them, 512 in fp32 (larger tiles against these, forward: bf16 2 x 462 x 3368
// 43.8 and 12.4 us, 345 x 2975 x 72 25.4 and 17.5, 112 x 12632 x 240 18.9 and 17.0 but
// 214 x 12343 x 704 39.7 and 59.7; fp32 6 x 5639 x 528 25.2 and 14.7, 159 x 132 x 1520 47.9
// and 20.5, 626 x 1585 x 440 27.9 and 29.9).
static bool small_head(int64_t M, int64_t N, bool bf) {
  return ((M + 31) / 32) * ((N + 31) / 32) <= (bf ? 1024 : 512);
}
template <typename E>
static hipError_t run_head_small(const GemmDesc& g, const E& e, bool bf, hipStream_t s) {
  const dim3 n(((g.M + 31) / 32) * ((g.N + 31) / 32));
  if (bf) hipLaunchKernelGGL((head_small_kernel<true, E>), n, dim3(256), 0, s, g, e);
  else hipLaunchKernelGGL((head_small_kernel<false, E>), n, dim3(256), 0, s, g, e);
  return hipGetLastError();
}
// The product of x and w: sums or dL/dz.
template <typename E>
static hipError_t run_logits(const GemmDesc& g, const E& e, bool bf, bool large, hipStream_t s) {
  if (small_head(g.M, g.N, bf)) return run_head_small(g, e, bf, s);
  if (bf) return run_head<true, true>(g, e, large, s);
  return run_head_f32<true, true>(g, e, f32_tile(g.M, g.N, 0, true), s);
}

// --------------------------------------------------------------- target rows
// The ids of a row, absent ones and repetitions as -1, into `ids` [256] (LDS of the wave's
// own): entries lane, lane + 64, ... of every lane.
__device__ __forceinline__ void row_ids(const zl_targets& t, int V, int64_t row, bool on, int lane, int32_t* ids,
                                        int32_t (&mine)[ZL_TARGETS_MAX_K / 64]) {
  constexpr int PER = ZL_TARGETS_MAX_K / 64;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = lane + 64 * i;
    mine[i] = -1;
    if (on && e < t.k) {
      const int32_t id = t.ids[row * t.k + e];
      if (id >= 0 && id < V) mine[i] = id;
    }
    ids[e] = mine[i];
  }
  wave_sync();
  bool twice[PER] = {};
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int e = lane + 64 * i;
#pragma unroll 4
    for (int f = 0; f < min(64 * (i + 1), t.k) && 64 * i < t.k; f += 4) {
      const int4 o = *reinterpret_cast<const int4*>(ids + f);
      twice[i] |= (o.x == mine[i] && f < e) || (o.y == mine[i] && f + 1 < e) || (o.z == mine[i] && f + 2 < e) ||
                  (o.w == mine[i] && f + 3 < e);
    }
  }
  wave_sync();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (twice[i]) mine[i] = -1;
    ids[lane + 64 * i] = mine[i];
  }
  wave_sync();
}
__device__ __forceinline__ int32_t row_label(const zl_targets& t, int V, int64_t row) {
  const int32_t y = t.labels ? t.labels[row] : -1;
  return y >= 0 && y < V ? y : -1;
}

// What the teacher names of every row, a wave each: NamedCols' order and spans, and the place
// of every entry in that order (slot [T, k], -1: absent or a repetition).
__global__ void __launch_bounds__(64) head_named_kernel(int V, zl_targets t, int width, int32_t* slot, int32_t* order,
                                                        uint32_t* span, int64_t ldb) {
  constexpr int PER = ZL_TARGETS_MAX_K / 64;
  __shared__ __align__(16) int32_t ids[ZL_TARGETS_MAX_K], sorted[ZL_TARGETS_MAX_K];
  const int lane = threadIdx.x, k = t.k;
  const int64_t row = blockIdx.x;
  span += row * ldb;
  for (int64_t i = (int64_t)lane * 4; i < ldb; i += 256) *reinterpret_cast<uint4*>(span + i) = make_uint4(0, 0, 0, 0);
  int n = 0;
  int32_t mine[PER], at[PER];
  row_ids(t, V, row, true, lane, ids, mine);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    // how many distinct ids are smaller (-1 is the largest unsigned number)
    at[i] = 0;
#pragma unroll 4
    for (int f = 0; f < k && 64 * i < k; f += 4) {
      const uint4 o = *reinterpret_cast<const uint4*>(ids + f);
      const uint32_t v = (uint32_t)mine[i];
      at[i] += (o.x < v) + (o.y < v) + (o.z < v) + (o.w < v);
    }
    const bool on = mine[i] >= 0;
    n += __popcll(__ballot(on));
    if (on) {
      sorted[at[i]] = mine[i];
      order[row * k + at[i]] = mine[i];
    }
    if (lane + 64 * i < k) slot[row * k + lane + 64 * i] = on ? at[i] : -1;
  }
  __syncthreads();  // the spans are cleared
  uint16_t* ends = reinterpret_cast<uint16_t*>(span);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int r = lane + 64 * i;
    if (r >= n) continue;
    const int b = sorted[r] / width;
    if (r == 0 || sorted[r - 1] / width != b) ends[2 * (int64_t)b] = (uint16_t)(r | sorted[r] % width << 8);
    if (r == n - 1 || sorted[r + 1] / width != b) ends[2 * (int64_t)b + 1] = (uint16_t)(r + 1);
  }
}

// The teacher's distribution over a row's entries, a wave per row.
struct WaveTeacher {
  static constexpr int PER = ZL_TARGETS_MAX_K / 64;
  int32_t id[PER];
  float t[PER], p[PER];
  bool on, rest;
  float L, r, u;
  // the row's entries on their way: ids (only those below 0 are told apart), values
  __device__ __forceinline__ void load(const zl_targets& q, int64_t row, const int32_t* ids, int lane) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = lane + 64 * i;
      id[i] = -1;
      t[i] = 0.f;
      if (e < q.k) {
        id[i] = ids[e];
        t[i] = q.values[row * q.k + e];
      }
    }
    u = q.rest ? q.rest[row] : -INFINITY;
  }
  __device__ __forceinline__ void form(const zl_targets& q) {
    const float inv = 1.f / q.temperature;
    bool any = false, bad = false;
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      t[i] = id[i] >= 0 ? t[i] * inv : -INFINITY;
      any |= id[i] >= 0;
      bad |= t[i] != t[i];
      m = fmaxf(m, t[i]);
    }
    m = fmaxf(wave_max(m), u);
    on = __ballot(any) != 0 && (m != -INFINITY || __ballot(bad) != 0 || u != u);
    const float ref = m == -INFINITY ? 0.f : m;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) s += expf(t[i] - ref);
    s = wave_sum(s) + expf(u - ref);
    L = ref + logf(s);
    rest = u != -INFINITY;
    r = on && rest ? expf(u - L) : 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) p[i] = on ? expf(t[i] - L) : 0.f;
  }
};

// Joins the partial sums of R rows, 256 / R strands of blocks each, then a wave per
// row forms its losses.  PAIR: both log-sums; masked: the second leaves the
// teacher's ids out; their logits go to the statistics in the ids' order.  The label joins
// the first of a pair, or the only one, here (label_term).
template <int R, bool PAIR>
__global__ void __launch_bounds__(256) head_rows_kernel(int64_t T, int V, int blocks, const float* part, zl_targets t,
                                                        float a, float b, bool masked, const int32_t* slot,
                                                        const float* named, float* loss, float* stats) {
  constexpr int S = 256 / R;
  __shared__ float4 red[S][R];
  const int r = threadIdx.x % R, st = threadIdx.x / R, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row0 = (int64_t)blockIdx.x * R;
  const float inv = t.ids ? 1.f / t.temperature : 1.f, c2 = inv * LOG2E;
  // what the first row of every wave takes is on its way before the sums are joined
  WaveTeacher w;
  int32_t yl = -1;
  float zl[WaveTeacher::PER] = {}, zy = 0.f;
  auto fetch = [&](int64_t row) __attribute__((always_inline)) {
    yl = row_label(t, V, row);
    zy = yl >= 0 ? stats[row * (4 + t.k) + 3] : 0.f;
    if (!t.ids) return;
    w.load(t, row, slot + row * t.k, lane);
#pragma unroll
    for (int j = 0; j < WaveTeacher::PER; ++j) zl[j] = w.id[j] >= 0 ? named[row * t.k + w.id[j]] : 0.f;
  };
  if (wave < R && row0 + wave < T) fetch(row0 + wave);
  LogSum x, y;
  if (row0 + r < T) {
#pragma unroll 4
    for (int j = st; j < blocks; j += S) {
      if constexpr (PAIR) {
        const float4 v = *reinterpret_cast<const float4*>(part + ((int64_t)j * T + row0 + r) * 4);
        x.merge(v.x, v.y, LOG2E);
        y.merge(v.z, v.w, c2);
      } else {
        const float2 v = *reinterpret_cast<const float2*>(part + ((int64_t)j * T + row0 + r) * 2);
        y.merge(v.x, v.y, c2);
      }
    }
  }
  red[st][r] = make_float4(x.m, x.s, y.m, y.s);
  __syncthreads();
  for (int i = wave; i < R; i += 4) {
    const int64_t row = row0 + i;
    if (row >= T) break;
    // the strands in a fixed tree over the lanes
    LogSum p, q;
    for (int j = lane; j < S; j += 64) {
      const float4 v = red[j][i];
      p.merge(v.x, v.y, LOG2E);
      q.merge(v.z, v.w, c2);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      // both lanes of a pair must see the sums before either changes
      const float pm = __shfl_xor(p.m, o, 64), ps = __shfl_xor(p.s, o, 64);
      const float qm = __shfl_xor(q.m, o, 64), qs = __shfl_xor(q.s, o, 64);
      p.merge(pm, ps, LOG2E);
      q.merge(qm, qs, c2);
    }
    if (i != wave) fetch(row);
    float* out = stats + row * (4 + t.k);
    const bool label = yl >= 0;
    const LabelTerm ce = label_term(PAIR ? p : q, zy);
    float total = 0.f, lt = 0.f, other = 0.f;
    bool on = false;
    if (t.ids) {
#pragma unroll
      for (int j = 0; j < WaveTeacher::PER; ++j)
        if (lane + 64 * j < t.k) out[4 + lane + 64 * j] = zl[j];
      w.form(t);
      on = w.on;
      if (!PAIR && label) q.merge(zy, zy == -INFINITY ? 0.f : 1.f, c2);
      float kl = 0.f;
      LogSum n;
#pragma unroll
      for (int j = 0; j < WaveTeacher::PER; ++j) {
        if (w.id[j] >= 0) {
          n.raise(zl[j], c2);
          n.s += n.m == -INFINITY ? 0.f : expf((zl[j] - n.m) * inv);
        }
        if (w.p[j] > 0.f || w.p[j] != w.p[j]) kl += w.p[j] * (w.t[j] - zl[j] * inv);
      }
      if (masked) {
        other = q.log(inv);
        const float nm = wave_max(n.m);
        const float ns = wave_sum(n.m == -INFINITY ? n.s : n.s * expf((n.m - nm) * inv));
        q.merge(nm, ns, c2);
      }
      lt = q.log(inv);
      kl = wave_sum(kl) + lt - w.L;
      if (masked && w.r != 0.f) kl += w.r * (w.u - other);
      if (on && b != 0.f) total = b * t.temperature * t.temperature * kl;  // (a term of weight 0 may be infinite)
    }
    if (lane == 0) {
      if (label && a != 0.f) total += a * ce.loss;
      if (!label && !on) total = 0.f;
      loss[row] = total;
      out[0] = label ? ce.logsum : 0.f;
      out[1] = on ? lt : 0.f;
      out[2] = on && masked ? other : 0.f;
      out[3] = zy;
    }
  }
}

// The largest |dloss| of rows with a target (0 and what is not finite count as 1): with a
// label, or a log-sum of z / tau, which rows without a teacher have not.  (One that is 0 by
// chance is passed over: the largest is a scale, no more.)
__device__ __forceinline__ float row_weight(const zl_targets& t, int V, const float* stats, const float* dloss,
                                            int64_t row) {
  const float w = fabsf(dloss[row]);
  bool on = row_label(t, V, row) >= 0;
  if (t.ids) on |= stats[row * (4 + t.k) + 1] != 0.f;
  return on ? w : 0.f;
}
// Its share of the rows each, GMAX_PARTS at most (one block of 1024 threads: 10 us for 16384
// rows, whose statistics are a cache line each).
constexpr int GMAX_PARTS = 64;
__global__ void __launch_bounds__(256) head_gmax_kernel(int64_t T, int V, zl_targets t, const float* stats,
                                                        const float* dloss, float* part) {
  __shared__ float red[4];
  float m = 0.f;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < T; i += (int64_t)gridDim.x * 256)
    m = fmaxf(m, row_weight(t, V, stats, dloss, i));
  m = block_max<256>(m, red);
  if (threadIdx.x == 0) part[blockIdx.x] = m;
}
// Up to so many rows every block of the next kernel looks for itself: a launch less.
__host__ __device__ inline bool gmax_by_block(int64_t T, const zl_targets& t) { return T <= (t.ids ? 1024 : 4096); }
__host__ __device__ inline int gmax_parts(int64_t T) { return (int)(T < 256 * GMAX_PARTS ? (T + 255) / 256 : GMAX_PARTS); }

// Per row what dL/dz takes (GradEpi), the named columns (tid as in the forward) and
// their values; a wave per row.
__global__ void __launch_bounds__(256) head_coef_kernel(int64_t T, int V, zl_targets t, float a, float b, int mode,
                                                        const float* stats, const float* dloss, float* gmax, int32_t* tid,
                                                        float* tval, float4* coef, int32_t* live) {
  __shared__ float red[4];
  __shared__ __align__(16) int32_t ids[4][ZL_TARGETS_MAX_K];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = (int64_t)blockIdx.x * 4 + wave;
  int32_t mine[ZL_TARGETS_MAX_K / 64];
  if (t.ids) row_ids(t, V, row, row < T, lane, ids[wave], mine);
  float most = 1.f;
  if (dloss) {
    float m = 0.f;
    if (gmax_by_block(T, t))
      for (int i = threadIdx.x; i < (int)T; i += 256) m = fmaxf(m, row_weight(t, V, stats, dloss, i));
    else if ((int)threadIdx.x < gmax_parts(T))
      m = gmax[1 + threadIdx.x];
    m = block_max<256>(m, red);
    most = m > 0.f && m < INFINITY ? m : 1.f;
    if (blockIdx.x == 0 && threadIdx.x == 0) *gmax = most;
  }
  if (row >= T) return;
  const int32_t* id = ids[wave];
  const float* s = stats + row * (4 + t.k);
  int32_t* to = tid + row * (t.k + 1);
  float* val = tval + row * (t.k + 1);
  const float l1 = s[0], ls = s[1], lo = s[2];
  const int32_t y = row_label(t, V, row);
  const float up = dloss ? dloss[row] / most : 1.f;
  const float c1 = y >= 0 ? a * up : 0.f;
  float ct = 0.f, lt = ls, inv = 1.f;
  bool named = false, on = false;
  if (t.ids) {
    WaveTeacher w;
    w.load(t, row, id, lane);
    w.form(t);
    inv = 1.f / t.temperature;
    on = w.on;
    const float f = on ? b * t.temperature * up : 0.f;
    ct = f;
    if (on && t.rest) {
      lt = lo;
      ct = lo == -INFINITY ? 0.f : f * (expf(lo - ls) - w.r);
    }
#pragma unroll
    for (int i = 0; i < WaveTeacher::PER; ++i) {
      const int e = lane + 64 * i;
      if (e < t.k) to[e] = mine[i];
      if (e < t.k && mine[i] >= 0) {
        const float z = s[4 + e];
        float g = on ? f * (expf(z * inv - ls) - w.p[i]) : 0.f;
        if (y >= 0) g += c1 * (mine[i] == y ? expm1f(z - l1) : expf(z - l1));
        val[e] = g;
        named |= mine[i] == y;
      }
    }
  }
  named = __ballot(named) != 0;
  if (lane == 0) {
    if (y >= 0 && !named) {
      float g = c1 * expm1f(s[3] - l1);
      if (ct != 0.f) g += ct * expf(s[3] * inv - lt);
      val[t.k] = g;
    }
    float4 c = make_float4(c1, l1, ct, lt);
    if (mode == GRAD_ONE) {
      // labels or a teacher alone, or both at tau = 1 without a rest
      c.x = 0.f;
      c.z = ct + c1;
      if (!on) c.w = l1;
    } else if (mode == GRAD_SQUARE) {
      if (!on || lt == -INFINITY) c.w = lt = 0.5f * l1;  // any shift does for the square alone
      c.x = c1 == 0.f ? 0.f : c1 * expf(2.f * lt - l1);
    }
    // a term that is not there vanishes also where its exponential would overflow
    if (c.z == 0.f && c.x == 0.f) c.w = INFINITY;
    if (mode == GRAD_TWO && c.z == 0.f) c.w = INFINITY;
    if (c.x == 0.f) c.y = INFINITY;
    coef[row] = c;
    live[row] = on || y >= 0;
  }
  // a label that an id names too is that id's entry
  if (lane == 0) to[t.k] = named ? -1 : y;
}

// The named columns of the piece [v0, v0 + n) over what the product wrote.
__global__ void __launch_bounds__(256) head_put_kernel(int64_t count, int k, int v0, int n, const int32_t* tid,
                                                       const float* tval, void* dz, int64_t ldz, int dtype) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= count) return;
  const int32_t id = tid[i];
  if (id < v0 || id >= v0 + n) return;
  const int64_t row = i < 0x80000000ll ? (int64_t)((uint32_t)i / (uint32_t)(k + 1)) : i / (k + 1);
  st_act(dz, dtype, row * ldz + (id - v0), tval[i]);
}

// Row and column of the i-th group of 8 among rows of `per` (a 64-bit division takes
// longer than the group's memory).
__device__ __forceinline__ int64_t split_groups(int64_t i, int per, int& c) {
  const int64_t row = i < 0x80000000ll ? (int64_t)((uint32_t)i / (uint32_t)per) : i / per;
  c = (int)(i - row * per) * 8;
  return row;
}

// x with zeros in the rows that have no target (0 times NaN would spoil dw).
__global__ void __launch_bounds__(256) head_clean_kernel(int64_t T, int d, const int32_t* live, const void* x,
                                                         int64_t ldx, void* xc, int dtype) {
  int c;
  const int64_t row = split_groups((int64_t)blockIdx.x * 256 + threadIdx.x, d / 8, c);
  if (row >= T) return;
  const bool on = live[row] != 0;
  if (dtype == BF16) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (on) v = *reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(x) + row * ldx + c);
    *reinterpret_cast<uint4*>(static_cast<bf16_t*>(xc) + row * d + c) = v;
  } else {
    float4 lo = make_float4(0.f, 0.f, 0.f, 0.f), hi = lo;
    if (on) {
      const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(x) + row * ldx + c);
      lo = p[0];
      hi = p[1];
    }
    float4* o = reinterpret_cast<float4*>(static_cast<float*>(xc) + row * d + c);
    o[0] = lo;
    o[1] = hi;
  }
}

// out = (accumulate ? out : 0) + scale * gmax * the sum of nz fp32 [rows, d], in order.
__global__ void __launch_bounds__(256) head_finish_kernel(int64_t rows, int d, const float* in, int nz, float scale,
                                                          const float* gmax, void* out, int64_t ldo, int dtype,
                                                          int accumulate) {
  int c;
  const int64_t row = split_groups((int64_t)blockIdx.x * 256 + threadIdx.x, d / 8, c);
  if (row >= rows) return;
  const float f = gmax ? scale * *gmax : scale;
  float v[8], u[8];
  ldv_f32(in + row * d + c, v);
#pragma unroll 4
  for (int z = 1; z < nz; ++z) {
    ldv_f32(in + z * rows * d + row * d + c, u);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] += u[k];
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] *= f;
  if (accumulate) {
    ldv_f32(static_cast<const float*>(out) + row * ldo + c, u);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] += u[k];
  }
  stv_act(out, dtype, row * ldo + c, v);
}

__global__ void __launch_bounds__(256) head_zero_kernel(int64_t rows, int d, void* out, int64_t ldo, int dtype) {
  int c;
  const int64_t row = split_groups((int64_t)blockIdx.x * 256 + threadIdx.x, d / 8, c);
  if (row >= rows) return;
  const float v[8] = {};
  stv_act(out, dtype, row * ldo + c, v);
}

// ------------------------------------------------------------------ launches
static unsigned grid(int64_t n, int per) { return (unsigned)((n + per - 1) / per); }

HeadPlan head_plan(int64_t T, int V, int d, int dtype, int k, bool backward, bool need_dx, bool need_dw,
                   int columns) {
  HeadPlan p;
  memset(&p, 0, sizeof(p));
  const int64_t es = dtype == BF16 ? 2 : 4;
  if (dtype == BF16) {
    GemmShape sh = {(int)T, V, d, true, true, false, 0, false, 0};
    p.large = plan_gemm(sh).large;
  }
  // columns of a wave tile
  p.width = small_head(T, V, dtype == BF16) ? 32 : p.large ? 128 : dtype == F32 && f32_tile(T, V, 0, true) != F32_128 ? 32 : 64;
  p.blocks = (V + p.width - 1) / p.width;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += (bytes + 255) / 256 * 256;
    return o;
  };
  p.tid = take(T * (k + 1) * 4);  // forward: slots
  if (!backward) {
    p.part = take((size_t)p.blocks * T * (k ? 16 : 8));  // a pair of sums only with a teacher
    p.ldb = ((int64_t)p.blocks + 3) / 4 * 4;
    if (k) {
      p.span = take(T * p.ldb * 4);
      p.order = take(T * k * 4);
      p.named = take(T * k * 4);
    }
  } else {
    // a piece of dL/dz has at most 1 GiB
    const int64_t all = ((int64_t)V + 255) / 256 * 256;
    int64_t most = ((int64_t)1 << 30) / (es * (T ? T : 1)) / 256 * 256;
    if (most < 256) most = 256;
    int64_t c = columns ? ((int64_t)columns + 255) / 256 * 256 : most;
    if (c > most) c = most;
    if (c > all) c = all;
    p.columns = (int)c;
    p.ldz = c;
    p.tval = take(T * (k + 1) * 4);
    p.gmax = take((1 + GMAX_PARTS) * 4);  // and of parts of the rows
    p.coef = take(T * 16);
    p.live = take(T * 4);
    p.dz = take(T * p.ldz * es);
    if (need_dx) p.dxa = take(T * (int64_t)d * 4);
    if (need_dw) p.xc = take(T * (int64_t)d * es);
    const int64_t rows = need_dw && c > T ? c : T;
    int64_t n = 64 * rows * d;
    if (n > (int64_t)1 << 24) n = (int64_t)1 << 24;
    p.split_elems = (size_t)n;
    p.split = take(n * 4);
  }
  p.bytes = at;
  return p;
}

static GemmDesc head_gemm(int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, bool ak, const void* B,
                          int64_t ldb, bool bk) {
  GemmDesc g;
  memset(&g, 0, sizeof(g));
  g.M = (int)M;
  g.N = (int)N;
  g.K = g.ka = g.kb = g.ksplit = (int)K;
  g.A = A;
  g.lda = lda;
  g.a_kmajor = ak;
  g.B = B;
  g.ldb = ldb;
  g.b_kmajor = bk;
  return g;
}

#define ZL_TRY(x)                        \
  do {                                   \
    const hipError_t err_ = (x);         \
    if (err_ != hipSuccess) return err_; \
  } while (0)

hipError_t launch_head_loss(const zl_head_args& a, hipStream_t s) {
  const int64_t T = a.T;
  if (T == 0) return hipSuccess;
  const zl_targets& t = a.targets;
  const bool bf = a.dtype == BF16, hard = t.labels != nullptr, soft = t.ids != nullptr, masked = soft && t.rest;
  const bool pair = hard && soft && (masked || t.temperature != 1.f);
  const HeadPlan p = head_plan(T, a.V, a.d, bf ? BF16 : F32, t.k, false, false, false, 0);
  char* ws = static_cast<char*>(a.workspace);
  int32_t* slot = reinterpret_cast<int32_t*>(ws + p.tid);
  float* part = reinterpret_cast<float*>(ws + p.part);
  uint32_t* span = soft ? reinterpret_cast<uint32_t*>(ws + p.span) : nullptr;
  int32_t* order = reinterpret_cast<int32_t*>(ws + p.order);
  float* named = reinterpret_cast<float*>(ws + p.named);
  float wa, wb;
  loss_weights(t, wa, wb);
  if (soft)
    hipLaunchKernelGGL(head_named_kernel, dim3((unsigned)T), dim3(64), 0, s, a.V, t, p.width, slot, order, span, p.ldb);
  // a masked sum is always the second of a pair
  const bool two = pair || masked;
  const GemmDesc g = head_gemm(T, a.V, a.d, a.x, a.ldx, true, a.w, a.ldw, true);
  auto sums = [&](auto pc) -> hipError_t {
    const StatEpi<decltype(pc)::value> e = {soft ? LOG2E / t.temperature : LOG2E, part, T, {order, span, p.ldb, named, t.k},
                                                 masked, t.labels, a.stats};
    return run_logits(g, e, bf, p.large, s);
  };
  if (two) ZL_TRY(sums(std::true_type{}));
  else ZL_TRY(sums(std::false_type{}));
  auto rows = [&](auto rc, auto pc) {
    constexpr int R = decltype(rc)::value;
    constexpr bool P = decltype(pc)::value;
    hipLaunchKernelGGL((head_rows_kernel<R, P>), dim3(grid(T, R)), dim3(256), 0, s, T, a.V, p.blocks, part, t, wa, wb, masked,
                       slot, named, a.loss, a.stats);
  };
  using std::integral_constant;
  auto by_rows = [&](auto pc) {
    // two rows a wave; a block each where rows are few
    if (T >= 512) rows(integral_constant<int, 8>{}, pc);
    else rows(integral_constant<int, 1>{}, pc);
  };
  if (two) by_rows(std::true_type{});
  else by_rows(std::false_type{});
  return hipGetLastError();
}

// Splits of a product's K; a part is a multiple of the k tile.
template <bool AK, bool BKM>
static int head_splits(int64_t M, int64_t N, int64_t K, bool bf, size_t elems, int& tile, int& ksplit) {
  if (bf) {
    const GemmShape sh = {(int)M, (int)N, (int)K, AK, BKM, true, elems, false, 0};
    const GemmPlan pl = plan_gemm(sh);
    tile = pl.large;
    return split_k((int)K, pl.nz, KTile<AK, BKM>::BK, ksplit);
  }
  // up to two blocks of 128 x 128 a CU, four of 64 x 64; 128 of K each at least
  tile = f32_tile(M, N, K, AK);
  const int64_t tiles = tile == F32_64 ? ((M + 63) / 64) * ((N + 63) / 64) : ((M + 127) / 128) * ((N + 127) / 128);
  int64_t nz = (tile == F32_64 ? 1024 : 512) / tiles;
  if (tile == F32_128 && tiles >= 256) nz = 1;
  if (nz > K / 128) nz = K / 128;
  if (nz > (int64_t)(elems / (size_t)(M * N))) nz = (int64_t)(elems / (size_t)(M * N));
  if (nz < 1) nz = 1;
  return split_k((int)K, (int)nz, SK, ksplit);
}

hipError_t launch_head_loss_bwd(const zl_head_args& a, hipStream_t s) {
  const int64_t T = a.T;
  const int d = a.d;
  const bool bf = a.dtype == BF16;
  const int dt = bf ? BF16 : F32, dxt = a.dx_dtype == ZL_BF16 ? BF16 : F32, dwt = a.dw_dtype == ZL_BF16 ? BF16 : F32;
  if (T == 0) {
    if (a.dw && !a.accumulate)
      hipLaunchKernelGGL(head_zero_kernel, dim3(grid((int64_t)a.V * (d / 8), 256)), dim3(256), 0, s, a.V, d, a.dw, a.lddw, dwt);
    return hipGetLastError();
  }
  const zl_targets& t = a.targets;
  const bool hard = t.labels != nullptr, soft = t.ids != nullptr, rest = soft && t.rest;
  const bool two = hard && soft && (rest || t.temperature != 1.f);
  const int mode = !two ? GRAD_ONE : t.temperature == 2.f ? GRAD_SQUARE : GRAD_TWO;
  const HeadPlan p = head_plan(T, a.V, d, dt, t.k, true, a.dx != nullptr, a.dw != nullptr, a.columns);
  char* ws = static_cast<char*>(a.workspace);
  int32_t* tid = reinterpret_cast<int32_t*>(ws + p.tid);
  float* tval = reinterpret_cast<float*>(ws + p.tval);
  float* gmax = reinterpret_cast<float*>(ws + p.gmax);
  float4* coef = reinterpret_cast<float4*>(ws + p.coef);
  int32_t* live = reinterpret_cast<int32_t*>(ws + p.live);
  float* dxa = reinterpret_cast<float*>(ws + p.dxa);
  float* split = reinterpret_cast<float*>(ws + p.split);
  void* dz = ws + p.dz;
  void* xc = ws + p.xc;
  float wa, wb;
  loss_weights(t, wa, wb);
  // The labels' weight (the teacher's, where that is all but alone) is taken out of dL/dz and
  // into the scale, as the largest |dloss| is: a sure label's entry is then -1, not a number
  // that is rounded alike in every row.
  const float weight = wa > 0x1p-20f * wb * t.temperature ? wa : wb * t.temperature, scale = a.scale * weight;
  wa /= weight;
  wb /= weight;
  if (a.dloss && !gmax_by_block(T, t))
    hipLaunchKernelGGL(head_gmax_kernel, dim3(gmax_parts(T)), dim3(256), 0, s, T, a.V, t, a.stats, a.dloss, gmax + 1);
  hipLaunchKernelGGL(head_coef_kernel, dim3(grid(T, 4)), dim3(256), 0, s, T, a.V, t, wa, wb, mode, a.stats, a.dloss, gmax,
                     tid, tval, coef, live);
  const float* most = a.dloss ? gmax : nullptr;
  if (a.dw)
    hipLaunchKernelGGL(head_clean_kernel, dim3(grid(T * (d / 8), 256)), dim3(256), 0, s, T, d, live, a.x, a.ldx, xc, dt);
  ZL_TRY(hipGetLastError());
  auto finish = [&](int64_t rows, const float* in, int nz, float scale, const float* by, void* out, int64_t ldo, int type,
                    int accumulate) {
    hipLaunchKernelGGL(head_finish_kernel, dim3(grid(rows * (d / 8), 256)), dim3(256), 0, s, rows, d, in, nz, scale, by, out,
                       ldo, type, accumulate);
  };
  const size_t es = bf ? 2 : 4;
  // a piece of w is read with 32-bit offsets
  const int64_t reach = (((int64_t)1 << 30) - 1) / a.ldw / 256 * 256;
  const int columns = p.columns < reach ? p.columns : (int)reach;
  for (int v0 = 0; v0 < a.V; v0 += columns) {
    const int n = a.V - v0 < columns ? a.V - v0 : columns;
    const int n8 = (n + 7) / 8 * 8;
    const char* w = static_cast<const char*>(a.w) + (size_t)v0 * a.ldw * es;
    {
      const GemmDesc g = head_gemm(T, n, d, a.x, a.ldx, true, w, a.ldw, true);
      GemmShape sh = {(int)T, n, d, true, true, false, 0, false, 0};
      auto grads = [&](auto mc) -> hipError_t {
        const GradEpi<decltype(mc)::value> e = {coef, soft ? 1.f / t.temperature : 1.f, dz, p.ldz, dt};
        return run_logits(g, e, bf, bf && plan_gemm(sh).large, s);
      };
      if (mode == GRAD_ONE) ZL_TRY(grads(std::integral_constant<int, GRAD_ONE>{}));
      else if (mode == GRAD_TWO) ZL_TRY(grads(std::integral_constant<int, GRAD_TWO>{}));
      else ZL_TRY(grads(std::integral_constant<int, GRAD_SQUARE>{}));
    }
    const int64_t named = T * (t.k + 1);
    hipLaunchKernelGGL(head_put_kernel, dim3(grid(named, 256)), dim3(256), 0, s, named, t.k, v0, n, tid, tval, dz, p.ldz, dt);
    ZL_TRY(hipGetLastError());
    // a product's tiles write where the result belongs; splits of K and, for dx, pieces
    // of the vocabulary meet in fp32 first
    const bool first = v0 == 0, last = v0 + n >= a.V;
    if (a.dx) {
      GemmDesc g = head_gemm(T, d, n8, dz, p.ldz, true, w, a.ldw, false);
      g.kb = n;
      int tile;
      const int nz = head_splits<true, false>(T, d, n8, bf, p.split_elems, tile, g.ksplit);
      const bool whole = first && last;
      OutEpi e = {dxa, d, F32, 1.f, nullptr, !first, 0, live};
      if (nz > 1) e = {split, d, F32, 1.f, nullptr, 0, T * d, live};
      else if (whole) e = {a.dx, a.lddx, dxt, scale, most, 0, 0, live};
      if (bf) ZL_TRY((run_head<true, false>(g, e, tile, s, nz)));
      else ZL_TRY((run_head_f32<true, false>(g, e, tile, s, nz)));
      if (nz > 1 && whole)
        finish(T, split, nz, scale, most, a.dx, a.lddx, dxt, 0);
      else if (nz > 1)
        finish(T, split, nz, 1.f, nullptr, dxa, d, F32, !first);
      if (last && !whole) finish(T, dxa, 1, scale, most, a.dx, a.lddx, dxt, 0);
    }
    if (a.dw) {
      GemmDesc g = head_gemm(n, d, T, dz, p.ldz, false, xc, d, false);
      char* out = static_cast<char*>(a.dw) + (size_t)v0 * a.lddw * (dwt == BF16 ? 2 : 4);
      int tile;
      const int nz = head_splits<false, false>(n, d, T, bf, p.split_elems, tile, g.ksplit);
      OutEpi e = {out, a.lddw, dwt, scale, most, a.accumulate, 0, nullptr};
      if (nz > 1) e = {split, d, F32, 1.f, nullptr, 0, (int64_t)n * d, nullptr};
      if (bf) ZL_TRY((run_head<false, false>(g, e, tile, s, nz)));
      else ZL_TRY((run_head_f32<false, false>(g, e, tile, s, nz)));
      if (nz > 1) finish(n, split, nz, scale, most, out, a.lddw, dwt, a.accumulate);
    }
  }
  return hipGetLastError();
}

}  // namespace zl
