// Weight gradient from a packed activation (include/zl_layer.h):
//   dw[m, n] = sum_t dy[t, m] x[t, n],  x in 8 bits with a scale per 32 columns.
//
// bf16: the weight-gradient GEMM's tiles (gemm_tiles.h, both operands
// MN-major): dy is copied to LDS by direct loads, x is loaded as codes into
// registers (half the bytes), turned into bf16 there (exact) and stored to the
// same LDS layout that the direct copies would leave.
#include <string.h>

#include "gemm_tiles.h"
#include "layer.h"
#include "packed.h"

namespace zl {

// --------------------------------------------------------------- fp32 MFMA
// BT x BT tiles of four waves (nx of them side by side), v_mfma_f32_32x32x2_f32 on
// fp32 tiles of 2048 / BT tokens in LDS; the next tile is loaded and the one after
// it widened while this one is multiplied (one barrier per tile).  64-bit
// addresses: also what bf16 dy takes whose rows lie too far apart for the buffer
// offsets of 512 tokens.  A block has tokens [z per, (z + 1) per); with splits it
// writes fp32 partials.  Registers for three blocks a CU: 256 x 4096 x 8192 154 us
// (two: 173; 64 x 64 tiles on the vector ALUs: 224).
template <bool BF, int BT>
__global__ void __launch_bounds__(256, 3) wgrad_f32_kernel(WgradArgs a, unsigned nx, int64_t per, bool split) {
  constexpr int VK = 2048 / BT, CH = BT / PW, F = BT / 64;  // 32 x 32 blocks per wave and side
  __shared__ __align__(16) float As[2][VK][BT], Bs[2][VK][BT];
  const int m0 = (int)(blockIdx.x / nx) * BT, n0 = (int)(blockIdx.x % nx) * BT;
  const int64_t t0 = blockIdx.z * per, t1 = min(t0 + per, a.T);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // this thread's 8 columns of one token of the tile, of dy and of x
  const int lt = tid / CH, lc = (tid % CH) * PW;
  const int lr = lane & 31, lk = lane >> 5, wm = (wave >> 1) * 32 * F, wn = (wave & 1) * 32 * F;
  f32x16_t acc[F][F];
#pragma unroll
  for (int i = 0; i < F; ++i)
#pragma unroll
    for (int j = 0; j < F; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  Raw8<BF> ra;
  RawP rb;
  auto load = [&](int64_t t) __attribute__((always_inline)) {
    ra.zero();
    rb.zero();
    if (t + lt < t1 && m0 + lc < a.M) ra.load(a.dy, (t + lt) * a.lddy + m0 + lc);
    if (t + lt < t1 && n0 + lc < a.N) rb.load(a.x, t + lt, n0 + lc);
  };
  auto put = [&](int buf) __attribute__((always_inline)) {
    float v[PW];
    ra.get(v);
    *reinterpret_cast<float4*>(&As[buf][lt][lc]) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(&As[buf][lt][lc + 4]) = make_float4(v[4], v[5], v[6], v[7]);
    rb.get(v);
    *reinterpret_cast<float4*>(&Bs[buf][lt][lc]) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(&Bs[buf][lt][lc + 4]) = make_float4(v[4], v[5], v[6], v[7]);
  };
  load(t0);
  put(0);
  load(t0 + VK);
  __syncthreads();
  int buf = 0;
  for (int64_t t = t0; t < t1; t += VK) {
    put(buf ^ 1);  // the tile after this one
    load(t + 2 * VK);
#pragma unroll
    for (int k = 0; k < VK; k += 2) {
      float x[F], y[F];
#pragma unroll
      for (int i = 0; i < F; ++i) {
        x[i] = As[buf][k + lk][wm + 32 * i + lr];
        y[i] = Bs[buf][k + lk][wn + 32 * i + lr];
      }
#pragma unroll
      for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[i], y[j], acc[i][j], 0, 0, 0);
    }
    __syncthreads();
    buf ^= 1;
  }
#pragma unroll
  for (int i = 0; i < F; ++i)
#pragma unroll
    for (int j = 0; j < F; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int m = m0 + wm + 32 * i + Mma<32>::row(lane, r), n = n0 + wn + 32 * j + lr;
        if (m >= a.M || n >= a.N) continue;
        if (split) {
          a.part[((int64_t)blockIdx.z * a.M + m) * a.N + n] = acc[i][j][r];
        } else {
          float* o = a.dw + (int64_t)m * a.lddw + n;
          *o = (a.accumulate ? *o : 0.f) + a.scale * acc[i][j][r];
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

template <bool BF, int BT>
static hipError_t wgrad_f32_go(const WgradArgs& a, hipStream_t s) {
  constexpr int VK = 2048 / BT;
  const int64_t nx = (a.N + BT - 1) / BT, ny = (a.M + BT - 1) / BT;
  if (nx * ny > MAX_BLOCKS) return hipErrorInvalidValue;
  // splits of at least 256 tokens until there are two blocks per CU, four of the
  // small ones (4096 x 1024 x 2048: 158 us, with two 166)
  int64_t nz = (BT == 128 ? 512 : 1024) / (nx * ny);
  if (nz > a.T / 256) nz = a.T / 256;
  const int64_t room = a.part ? (int64_t)(a.part_elems / ((size_t)a.M * a.N)) : 0;
  if (nz > room) nz = room;
  if (nz < 1) nz = 1;
  int64_t per = (a.T + nz - 1) / nz;
  per = (per + VK - 1) / VK * VK;
  nz = a.T > 0 ? (a.T + per - 1) / per : 1;
  hipLaunchKernelGGL((wgrad_f32_kernel<BF, BT>), dim3((unsigned)(nx * ny), 1, (unsigned)nz), dim3(256), 0, s, a, (unsigned)nx, per, nz > 1);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || nz == 1) return e;
  return launch_splitk_reduce(a.part, (int)nz, a.M, a.N, grad_epi(a), s);
}
template <bool BF>
static hipError_t wgrad_f32(const WgradArgs& a, hipStream_t s) {
  // large tiles where they fill the chip without splits (1024 x 2048 x 4096: 150 us;
  // 30 x 1000 x 2000, 128 of them, 13.0 where small ones take 6.7)
  const int64_t large = (int64_t)((a.M + 127) / 128) * ((a.N + 127) / 128);
  return large >= 256 ? wgrad_f32_go<BF, 128>(a, s) : wgrad_f32_go<BF, 64>(a, s);
}

// ------------------------------------------------------------------- MFMA
__device__ uint8_t llvm_amdgcn_raw_buffer_load_u8(i32x4_t rsrc, uint32_t voffset, uint32_t soffset, int aux)
    __asm("llvm.amdgcn.raw.buffer.load.i8");

// A buffer that ends with column `cols` of row `rows` - 1 (esz bytes each, row
// stride ld): offsets of later rows lie past it, and read as zero.
__device__ __forceinline__ i32x4_t rows_rsrc(const void* p, int64_t ld, int rows, int cols, int esz) {
  i32x4_t r = buffer_rsrc(p);
  r[2] = (int32_t)((uint32_t)((rows - 1) * ld + cols) * (uint32_t)esz);
  return r;
}

// One thread's share of a k tile of x: 16 codes of one token and their scale
// byte.  Columns outside the matrix have DMA_OOB, which no advance brings back.
template <int BN, int BK, int NT>
struct CodeTile {
  static constexpr int CPR = BN / 16;  // 16-code chunks per token
  static_assert(CPR * BK == NT, "one chunk per thread");
  uint32_t coff, soff;    // byte offsets at k0 = 0
  uint32_t cstep, sstep;  // bytes per token
  uint32_t lds;           // byte offset of the chunk's two 16-byte pieces in the bf16 tile

  __device__ __forceinline__ void init(const zl_packed& x, int nvalid) {
    const int k = threadIdx.x / CPR, q = threadIdx.x % CPR;
    const bool ok = q * 16 < nvalid;
    cstep = (uint32_t)x.ld_codes;
    sstep = (uint32_t)x.ld_scales;
    coff = ok ? k * cstep + q * 16 : DMA_OOB;
    soff = ok ? k * sstep + q / 2 : DMA_OOB;
    // pieces 2 q and 2 q + 1 of LDS row k; the swizzle is even, so they stay together
    lds = (uint32_t)(k * BN * 2 + ((2 * q) ^ xsk<32>(k)) * 16);
  }
  __device__ __forceinline__ void load(uint4& c, uint32_t& s, int k0, i32x4_t rc, i32x4_t rs) const {
    c = __builtin_bit_cast(uint4, buffer_load16(rc, coff + (uint32_t)k0 * cstep));
    s = llvm_amdgcn_raw_buffer_load_u8(rs, soff + (uint32_t)k0 * sstep, 0, 0);
  }
  // 4 codes to bf16; a scale byte of 255 makes NaN of any code
  __device__ static __forceinline__ uint2 widen(uint32_t w, uint32_t s) {
    w = s == 255 ? 0x7f7f7f7fu : w;
    const float f = __uint_as_float(s << 23);
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, f, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, f, true)));
  }
  // codes 8 h .. 8 h + 7 into the tile
  __device__ __forceinline__ void store_half(const uint4& c, uint32_t s, unsigned char* tile, int h) const {
    const uint2 a = widen(h ? c.z : c.x, s), b = widen(h ? c.w : c.y, s);
    *reinterpret_cast<uint4*>(tile + lds + 16 * h) = make_uint4(a.x, a.y, b.x, b.y);
  }
};

// NST LDS stages of BK tokens and as many register sets of codes.  In the last
// slice of tile kt, behind the barrier that releases its stage: x of tile kt + NST
// goes from its registers into the stage, the codes of tile kt + 2 NST are
// loaded in their place, and dy of tile kt + NST starts on its way.  Codes before
// dy: waiting for the oldest codes then leaves the newest copies of dy in flight.
// The loop runs whole rounds of NST tiles, so that stages and register sets are
// compile-time (16384 x 14336 x 4096, a run-time stage: 4 % more); tiles past the
// end are zeros by the buffers' ends, without a test per load (6 % more).  Of that
// size 1505 to 1585 us by card and clock, 1.21 to 1.28 PFLOP/s; the bf16 GEMM in turn
// with it on one card takes 1 to 3 % more.
template <int BM, int BN, int WM, int WN, int BK, int NST>
__global__ void __launch_bounds__(WM * WN * 64) wgrad_mfma_kernel(GemmDesc g, EpiArgs e, zl_packed x) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int MF = 32, NT = WM * WN * 64;
  constexpr int TM = BM / WM, TN = BN / WN, FM = TM / MF, FN = TN / MF, NS = BK / Mma<MF>::KS, NMF = FM * FN;
  constexpr uint32_t ABYTES = BM * BK * 2, STAGE = (BM + BN) * BK * 2;
  using TA = DmaTile<BM, BK, NT, false, MF>;
  constexpr int PER_TILE = TA::ITEMS + 2;
  static_assert(NS % 2 == 0 && NMF >= 2 && NST >= 3 && (NST - 2) * PER_TILE < 64, "schedule");

  int tm, tn;
  tile_coords(blockIdx.x, (g.M + BM - 1) / BM, (g.N + BN - 1) / BN, tm, tn);
  const int m0 = tm * BM, n0 = tn * BN;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int wm = wave / WN, wn = wave % WN;
  const int kbeg = blockIdx.z * g.ksplit, klen = min(g.K - kbeg, g.ksplit);
  const int mv = min(g.M - m0, BM), nv = min(g.N - n0, BN);
  const i32x4_t ra = rows_rsrc(static_cast<const bf16_t*>(g.A) + (int64_t)kbeg * g.lda + m0, g.lda, klen, mv, 2);
  const i32x4_t rc = rows_rsrc(static_cast<const uint8_t*>(x.codes) + kbeg * x.ld_codes + n0, x.ld_codes, klen,
                               (nv + 15) / 16 * 16, 1);
  const i32x4_t rs = rows_rsrc(static_cast<const uint8_t*>(x.scales) + kbeg * x.ld_scales + n0 / PBLK, x.ld_scales, klen,
                               (nv + PBLK - 1) / PBLK, 1);
  TA da;
  da.init(wave, lane, g.lda, mv);
  auto copy_dy = [&](uint32_t stage, int k0) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < TA::ITEMS; ++j)
      dma16(stage + (uint32_t)(wave * TA::ITEMS + j) * 1024u, da.off[j] + (uint32_t)k0 * da.kstride, ra);
  };
  CodeTile<BN, BK, NT> tb;
  tb.init(x, nv);
  FragTile<BM, BK, FM, false, MF> fa;
  FragTile<BN, BK, FN, false, MF> fb;
  fa.init(wm * TM, lane);
  fb.init(wn * TN, lane);

  f32x16_t acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;

  const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>(smem);
  const int nk = (klen + BK - 1) / BK;
  uint4 c[NST];
  uint32_t sc[NST];
  {
    uint4 pc[NST];
    uint32_t ps[NST];
#pragma unroll
    for (int t = 0; t < NST; ++t) tb.load(pc[t], ps[t], t * BK, rc, rs);
#pragma unroll
    for (int t = 0; t < NST; ++t) copy_dy(lds0 + t * STAGE, t * BK);
#pragma unroll
    for (int t = 0; t < NST; ++t) tb.load(c[t], sc[t], (NST + t) * BK, rc, rs);
#pragma unroll
    for (int t = 0; t < NST; ++t) {
      tb.store_half(pc[t], ps[t], smem + t * STAGE + ABYTES, 0);
      tb.store_half(pc[t], ps[t], smem + t * STAGE + ABYTES, 1);
    }
  }
  wait_vmcnt<2 * NST>();  // dy of the first NST tiles; the codes after it may be in flight
  __syncthreads();
  bf16x8_t af[2][FM], bfr[2][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i) af[0][i] = fa.read(reinterpret_cast<const bf16_t*>(smem), 0, i);
#pragma unroll
  for (int j = 0; j < FN; ++j) bfr[0][j] = fb.read(reinterpret_cast<const bf16_t*>(smem) + BM * BK, 0, j);
  for (int kt0 = 0; kt0 < nk; kt0 += NST) {
#pragma unroll
    for (int u = 0; u < NST; ++u) {
      const int kt = kt0 + u;
      const bf16_t* as = reinterpret_cast<const bf16_t*>(smem + u * STAGE);
      const bf16_t* an = reinterpret_cast<const bf16_t*>(smem + (u + 1 < NST ? u + 1 : 0) * STAGE);
#pragma unroll
      for (int q = 0; q < NS; ++q) {
        const int cb = q & 1, nb = cb ^ 1;
        const bf16_t* src = q + 1 < NS ? as : an;
        const int qs = q + 1 < NS ? q + 1 : 0;
        if (q + 1 == NS) {
          wait_vmcnt<(NST - 2) * PER_TILE>();  // this wave's share of dy of tile kt + 1
          __syncthreads();                      // everyone's share and x; tile kt fully read
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < NMF; ++t) {
          acc[t / FN][t % FN] = Mma<MF>::run(af[cb][t / FN], bfr[cb][t % FN], acc[t / FN][t % FN]);
#pragma unroll
          for (int r = 0; r < FM + FN; ++r) {
            if (r * NMF / (FM + FN) != t) continue;
            if (r < FM) af[nb][r] = fa.read(src, qs, r);
            else bfr[nb][r - FM] = fb.read(src + BM * BK, qs, r - FM);
          }
          if (q + 1 == NS) {
            if (t < 2) tb.store_half(c[u], sc[u], smem + u * STAGE + ABYTES, t);
            if (t == min(2, NMF - 1)) tb.load(c[u], sc[u], (kt + 2 * NST) * BK, rc, rs);
            if (t == min(3, NMF - 1)) copy_dy(lds0 + u * STAGE, (kt + NST) * BK);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  }
  dma_wait();  // zero-fill copies past the end must land before LDS is reused
  __syncthreads();
  store_tile<BM, BN, WM, WN, MF>(acc, smem, g, e, m0, n0, wave, lane);
}

template <int BM, int BN, int WM, int WN, int BK, int NST>
static hipError_t wgrad_mfma(const GemmDesc& g, const EpiArgs& e, const zl_packed& x, int nz, hipStream_t s) {
  auto kern = wgrad_mfma_kernel<BM, BN, WM, WN, BK, NST>;
  const size_t main = (size_t)NST * (BM + BN) * BK * sizeof(bf16_t);
  const size_t epi = (size_t)WM * WN * 32 * (BN / WN + 4) * sizeof(float);
  const size_t lds = main > epi ? main : epi;
  hipError_t err = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (err != hipSuccess) return err;
  const int nb = ((g.M + BM - 1) / BM) * ((g.N + BN - 1) / BN);
  hipLaunchKernelGGL(kern, dim3(nb, 1, nz), dim3(WM * WN * 64), lds, s, g, e, x);
  return hipGetLastError();
}

// One segment of tokens whose buffer offsets stay below 2^31.
static hipError_t wgrad_segment(const WgradArgs& a, int64_t t0, int T, bool accumulate, hipStream_t s) {
  GemmDesc g;
  memset(&g, 0, sizeof(g));
  g.M = a.M;
  g.N = a.N;
  g.K = T;
  g.A = static_cast<const bf16_t*>(a.dy) + t0 * a.lddy;
  g.lda = a.lddy;
  zl_packed x = a.x;
  x.codes = static_cast<uint8_t*>(x.codes) + t0 * x.ld_codes;
  x.scales = static_cast<uint8_t*>(x.scales) + t0 * x.ld_scales;
  EpiArgs e = grad_epi(a);
  e.accumulate = accumulate;
  const GemmPlan plan = plan_gemm({a.M, a.N, T, false, false, a.part != nullptr, a.part_elems, false, 0});
  // One block of eight waves a CU, 64 tokens a stage, where no CU would get a second
  // block and nothing is split, or the splits would be short.  Unsplit, against four
  // waves: 512 x 768 x 768 9.9 us and 11.4, 2048 x 2048 x 2048 25.2 and 26.7; without
  // room for partials at any T (4096 x 768 x 768 35.0 and 40.0, 8192 x 256 x 256 62.5 and
  // 66.4; at the least 64 x 2048 x 2048 10.5 and 10.2).  Instead of splits: 512 x 256 x
  // 256 9.5 and 11.1, 768 x 256 x 256 10.8 and 10.4, 800 x 256 x 256 12.1 and 10.5.  More
  // tiles: 512 x 4096 x 2048 23.8 and 20.3.
  const int64_t tiles = (int64_t)((a.M + 127) / 128) * ((a.N + 127) / 128);
  const bool deep = !plan.large && tiles <= 256 && (plan.nz == 1 || T <= 768);
  const int nz = split_k(T, deep ? 1 : plan.nz, 32, g.ksplit);
  EpiArgs ep = e;
  if (nz > 1) {
    memset(&ep, 0, sizeof(ep));
    ep.kind = EPI_STORE;
    ep.out = a.part;
    ep.ldo = a.N;
    ep.out_dtype = F32;
    ep.scale = 1.f;
    ep.zstride = (int64_t)a.M * a.N;
  }
  // 4 stages for large tiles (3 or 5: up to 1 % more at 16384 x 14336 x 4096), 3 for
  // small ones, which share a CU (4096 x 2304 x 768: 32.8; 4 stages 33.5, 8 42.2)
  hipError_t err = plan.large ? wgrad_mfma<256, 256, 4, 2, 32, 4>(g, ep, x, nz, s)
                   : deep     ? wgrad_mfma<128, 128, 4, 2, 64, 3>(g, ep, x, nz, s)
                              : wgrad_mfma<128, 128, 2, 2, 32, 3>(g, ep, x, nz, s);
  if (err != hipSuccess || nz == 1) return err;
  return launch_splitk_reduce(a.part, nz, a.M, a.N, e, s);
}

hipError_t launch_wgrad_packed(const WgradArgs& a, int dtype, hipStream_t s) {
  if (dtype != BF16) return wgrad_f32<false>(a, s);
  if (a.T == 0) return wgrad_f32<true>(a, s);  // zeros, or dw as it is; strides may be anything
  // tokens per launch: the largest offset from a tile's origin stays below 2^31.  As
  // many launches as it takes while each has 512 tokens and more (4096 x 262144 x 4096,
  // two of them: 8.8 ms, by 64-bit addresses and fp32 tiles 66; 4096 x 690000 x 1024,
  // nine: 12.7 and 44), which rows of up to 699050 gradients have.
  const int64_t dyb = a.lddy < (int64_t)1 << 31 ? 2 * a.lddy : a.lddy;  // (beyond, `most` is negative either way)
  const int64_t row = dyb > a.x.ld_codes ? dyb : a.x.ld_codes;
  const int64_t top = row > a.x.ld_scales ? row : a.x.ld_scales;
  const int64_t most = (((int64_t)1 << 31) - 1024) / top - 1024;
  if (a.T <= most) return wgrad_segment(a, 0, (int)a.T, a.accumulate != 0, s);
  if (most < 512) return wgrad_f32<true>(a, s);
  const int64_t step = most / 32 * 32;
  for (int64_t t = 0; t < a.T; t += step) {
    const int64_t n = a.T - t < step ? a.T - t : step;
    hipError_t err = wgrad_segment(a, t, (int)n, t > 0 || a.accumulate, s);
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

}  // namespace zl
