// Losses of logits in memory, and the top logits of a row (include/zl_loss.h).
// A block per row.  Bound by memory: the forward reads a row once, the backward
// reads and writes it once.
#include "loss.h"
#include "loss_rows.h"

namespace zl {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
template <bool STREAM>
__device__ __forceinline__ u32x4_t load16(const void* p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(static_cast<const u32x4_t*>(p));
  else return *static_cast<const u32x4_t*>(p);
}
template <bool STREAM>
__device__ __forceinline__ void store16(void* p, u32x4_t v) {
  if constexpr (STREAM) __builtin_nontemporal_store(v, static_cast<u32x4_t*>(p));
  else *static_cast<u32x4_t*>(p) = v;
}

// The largest of a group, two columns an instruction (fmaxf first quiets every operand,
// an instruction each).  With a NaN among them the result is any of them or NaN.
template <int N>
__device__ __forceinline__ float max_of_group(const float (&v)[N]) {
  float m = fmaxf(v[0], v[1]);
#pragma unroll
  for (int k = 2; k < N; k += 2) asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(m), "v"(v[k]), "v"(v[k + 1]));
  return m;
}

// ------------------------------------------------------------ rows of logits
// Columns in groups of W = 8 (fp32: 4), 16 bytes aligned from the first full group on,
// wherever the row starts: group g holds columns W g - pad .. W g - pad + W - 1 as far as
// they lie in [0, V); only the first and the last may be cut.
template <bool BF>
struct Row {
  using E = typename std::conditional<BF, bf16_t, float>::type;
  static constexpr int W = 16 / sizeof(E);
  const E* p;
  int V, pad, full0, full1;  // full groups [full0, full1)
  __device__ __forceinline__ Row(const void* base, int64_t off, int V_) : p(static_cast<const E*>(base) + off), V(V_) {
    const int skip = (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(E);
    pad = (W - skip) & (W - 1);
    full0 = pad ? 1 : 0;
    full1 = (V + pad) / W;
  }
  __device__ __forceinline__ int groups() const { return (V + pad + W - 1) / W; }
  // the cut groups: c = 0, 1; -1 where there is none
  __device__ __forceinline__ int cut(int c) const {
    if (c == 0) return pad ? 0 : -1;
    return ((V + pad) & (W - 1)) && full1 >= full0 ? full1 : -1;
  }
  __device__ __forceinline__ int group_of(int v) const { return (v + pad) / W; }
  __device__ __forceinline__ float at(int v) const { return Elem<E>::load(p, v); }
  template <bool STREAM = false>
  __device__ __forceinline__ u32x4_t load(int g) const {
    return load16<STREAM>(p + (W * (int64_t)g - pad));
  }
  __device__ static __forceinline__ void get(u32x4_t r, float (&v)[W]) {
#pragma unroll
    for (int k = 0; k < W; ++k) {
      if constexpr (BF) v[k] = __builtin_bit_cast(float, k & 1 ? r[k / 2] & 0xffff0000u : r[k / 2] << 16);
      else v[k] = __builtin_bit_cast(float, (uint32_t)r[k]);
    }
  }
  // a cut group, -inf outside the row and in column y
  __device__ __forceinline__ void get_cut(int g, float (&v)[W], int y = -1) const {
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const int c = W * g - pad + k;
      v[k] = c >= 0 && c < V && c != y ? at(c) : -INFINITY;
    }
  }
  // -inf in column y of its group
  __device__ __forceinline__ void drop(u32x4_t& r, int y) const {
    const int e = (y + pad) & (W - 1);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if constexpr (BF) {
        if (e >> 1 == w) r[w] = e & 1 ? (r[w] & 0xffffu) | 0xff800000u : (r[w] & 0xffff0000u) | 0xff80u;
      } else {
        if (e == w) r[w] = 0xff800000u;
      }
    }
  }
  // f(group, values) for this thread's groups, U loads in flight; DROP: column y (-1: none)
  // as -inf, found with a comparison per U groups
  template <int NT, int U, bool STREAM = false, bool DROP = false, typename F>
  __device__ __forceinline__ void each(F&& f, int y = -1) const {
    int g = full0 + (int)threadIdx.x, gy = -1;
    if constexpr (DROP) {
      if (y >= 0 && ((group_of(y) - g) & (NT - 1)) == 0) gy = group_of(y);
    }
    for (; g + (U - 1) * NT < full1; g += U * NT) {
      u32x4_t r[U];
#pragma unroll
      for (int u = 0; u < U; ++u) r[u] = load<STREAM>(g + u * NT);
      if constexpr (DROP) {
        if ((uint32_t)(gy - g) <= (U - 1) * NT) {
#pragma unroll
          for (int u = 0; u < U; ++u)
            if (g + u * NT == gy) drop(r[u], y);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float v[W];
        get(r[u], v);
        f(g + u * NT, v);
      }
    }
    for (; g < full1; g += NT) {
      u32x4_t r = load<STREAM>(g);
      if constexpr (DROP) {
        if (g == gy) drop(r, y);
      }
      float v[W];
      get(r, v);
      f(g, v);
    }
    if (threadIdx.x < 2) {
      const int c = cut((int)threadIdx.x);
      if (c >= 0) {
        float v[W];
        get_cut(c, v, y);
        f(c, v);
      }
    }
  }
};

// --------------------------------------------------- a row's named columns
// The label and the teacher's ids, found again while the row streams by: a bit for
// every group of columns (beyond BITS groups, several share one), and behind it chains
// of entries.  A test costs one broadcast LDS read per group; comparing every column
// with k ids would cost k.
template <int BITS, int HEADS, int K>
struct Names {
  static constexpr int MAX_K = K;
  uint32_t bits[BITS / 32];
  int head[HEADS];
  int id[K + 1];    // column, -1: absent
  int next[K + 1];
  float val[K + 1];

  template <int NT>
  __device__ __forceinline__ void clear() {
    for (int i = threadIdx.x; i < BITS / 32; i += NT) bits[i] = 0;
    for (int i = threadIdx.x; i < HEADS; i += NT) head[i] = -1;
  }
  __device__ __forceinline__ void add(int e, int column, int group) {
    id[e] = column;
    atomicOr(&bits[(group >> 5) & (BITS / 32 - 1)], 1u << (group & 31));
    next[e] = atomicExch(&head[group & (HEADS - 1)], e);
  }
  __device__ __forceinline__ int first(int group) const { return head[group & (HEADS - 1)]; }
  __device__ __forceinline__ bool maybe(int group) const {
    return bits[(group >> 5) & (BITS / 32 - 1)] >> (group & 31) & 1;
  }
};

// Those of a block of NT threads.  A wave of its own takes short rows of few ids.
template <int NT> struct NamesOf { using type = Names<32768, 512, ZL_TARGETS_MAX_K>; };
template <> struct NamesOf<64> { using type = Names<1024, 64, 64>; };

// What every thread of a block knows of its row's targets.
struct RowTargets {
  bool label, teacher, rest;
  int y;
  float zy;
  float L;   // log-sum of the teacher's outcomes
  float r;   // the rest's probability
  // this thread's id, where tid < k
  bool here;
  int id;
  float zi, t, p;  // the student's logit, the teacher's value / tau, its probability
};

// Reads the targets of row t, enters the ids (and, with `both`, the label as entry k)
// into `names`.  k <= NT.  Ends with a barrier.
template <int NT, bool BF>
__device__ __forceinline__ RowTargets row_targets(const LogitLossArgs& a, int64_t row, const Row<BF>& z,
                                                  typename NamesOf<NT>::type& names, bool both, float* red) {
  RowTargets q;
  const int tid = threadIdx.x, k = a.t.k, V = a.V;
  // every load is on its way before the first barrier
  q.y = a.t.labels ? a.t.labels[row] : -1;
  q.id = -1;
  float value = 0.f;
  if (tid < k) {
    q.id = a.t.ids[row * k + tid];
    value = a.t.values[row * k + tid];
  }
  const float u = a.t.ids && a.t.rest ? a.t.rest[row] : -INFINITY;
  q.label = q.y >= 0 && q.y < V;
  q.here = q.id >= 0 && q.id < V;
  q.zy = q.label ? z.at(q.y) : 0.f;
  q.zi = q.here ? z.at(q.id) : 0.f;
  q.teacher = q.rest = false;
  q.L = q.r = q.p = 0.f;
  q.t = -INFINITY;
  if (!a.t.ids && !(both && q.label)) return q;
  names.template clear<NT>();
  __syncthreads();
  if (tid < k) {
    names.id[tid] = q.here ? q.id : -1;
    if (q.here) names.add(tid, q.id, z.group_of(q.id));
  }
  if (both && tid == 0) {
    names.id[k] = -1;
    if (q.label) names.add(k, q.y, z.group_of(q.y));
  }
  __syncthreads();
  // the first entry of a column counts
  bool twice = false;
  if (q.here)
    for (int e = names.first(z.group_of(q.id)); e >= 0; e = names.next[e])
      twice |= e < tid && names.id[e] == q.id;
  bool named = false;
  if (both && tid == 0 && q.label)
    for (int e = names.first(z.group_of(q.y)); e >= 0; e = names.next[e])
      named |= e < k && names.id[e] == q.y;
  __syncthreads();
  if (twice) {
    names.id[tid] = -1;
    q.here = false;
    q.zi = 0.f;
  }
  if (named) names.id[k] = -1;
  if (a.t.ids) {
    if (q.here) q.t = value * (1.f / a.t.temperature);
    // -inf: no id; +inf: also a NaN, which a maximum would drop
    const float top = block_max<NT>(q.here ? (q.t != q.t ? INFINITY : fmaxf(q.t, -3.402823466e38f)) : -INFINITY, red);
    const float ref = fmaxf(top, u) == -INFINITY ? 0.f : fmaxf(top, u);
    const float s = block_sum<NT>(q.here ? expf(q.t - ref) : 0.f, red) + expf(u - ref);
    q.teacher = top != -INFINITY && s != 0.f;
    if (q.teacher) {
      q.L = ref + logf(s);
      q.rest = u != -INFINITY;
      q.r = q.rest ? expf(u - q.L) : 0.f;
      q.p = q.here ? expf(q.t - q.L) : 0.f;
    }
  }
  __syncthreads();
  return q;
}

// How many exponentials an element takes: one (labels or a teacher alone, or both at
// tau = 1 without a rest); two; or one for two at tau = 2, where exp(z) is the square
// of exp(z / 2).
enum { EXP_ONE, EXP_TWO, EXP_SQUARE };

// ---------------------------------------------------------------- forward
// Log-sums of z (unless EXP_ONE) and of z / tau; REST: the latter without the teacher's
// ids; all without the label, which joins them at the end (label_term).  The sums are taken
// relative to the largest of the row's first columns: no running maximum (8 instead of 10 cycles of the vector units per element, which come
// near the memory's time; 4096 x 128256 bf16, labels and 64 ids at tau 2: 175 us, 6.0 TB/s).
// Where that reference is so far off that either sum overflows or nearly vanishes (first
// columns at -inf: 0, which no column need be near; the columns beside the teacher's), the
// row goes by once more with running maxima.
template <bool BF, int NT, int MODE, bool REST, bool STREAM>
__global__ void __launch_bounds__(NT) logit_loss_kernel(LogitLossArgs a) {
  __shared__ typename NamesOf<NT>::type names;
  __shared__ float red[NT / 64];
  constexpr bool TWO = MODE != EXP_ONE;
  constexpr int W = Row<BF>::W;
  const int64_t row = blockIdx.x;
  const Row<BF> z(a.z, row * a.ldz, a.V);
  u32x4_t first = {};
  const int g0 = threadIdx.x;
  if (g0 >= z.full0 && g0 < z.full1) first = z.load(g0);
  const RowTargets q = row_targets<NT, BF>(a, row, z, names, false, red);
  if (!q.label && !q.teacher) {
    if (threadIdx.x == 0) {
      a.loss[row] = 0.f;
      *reinterpret_cast<float4*>(a.stats + 4 * row) = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    return;
  }
  const float inv = a.t.ids ? 1.f / a.t.temperature : 1.f;
  const float c2 = inv * LOG2E;  // of the teacher's log-sum
  // the named columns of group g out of v
  auto without = [&](int g, float (&v)[W]) __attribute__((always_inline)) {
    for (int e = names.first(g); e >= 0; e = names.next[e]) {
      const int c = names.id[e];
      if (c >= 0 && z.group_of(c) == g) {
#pragma unroll
        for (int k = 0; k < W; ++k) v[k] = W * g - z.pad + k == c ? -INFINITY : v[k];
      }
    }
  };
  // The label's column is left out of both sums, and out of their reference.
  const int y = q.label ? q.y : -1;
  LogSum s1, st;  // of z, of z / tau (EXP_ONE: st alone, at 1 / tau)
  float ref = -INFINITY;
  if (g0 < z.groups()) {
    float v[W];
    if (g0 >= z.full0 && g0 < z.full1) {
      if (y >= 0 && z.group_of(y) == g0) z.drop(first, y);
      z.get(first, v);
    } else {
      z.get_cut(g0, v, y);
    }
    ref = max_of(v);
  }
  ref = block_max<NT>(ref, red);
  if (!(fabsf(ref) < INFINITY)) ref = 0.f;
  s1.m = st.m = ref;
  z.template each<NT, 4, STREAM, true>([&](int g, float (&v)[W]) __attribute__((always_inline)) {
    if constexpr (MODE == EXP_TWO) {
#pragma unroll
      for (int k = 0; k < W; ++k) s1.s += __builtin_amdgcn_exp2f((v[k] - ref) * LOG2E);
    }
    if constexpr (REST) {
      if (q.teacher && names.maybe(g)) {
        if constexpr (MODE == EXP_SQUARE) {
#pragma unroll
          for (int k = 0; k < W; ++k) s1.s += __builtin_amdgcn_exp2f((v[k] - ref) * LOG2E);
        }
        without(g, v);
#pragma unroll
        for (int k = 0; k < W; ++k) st.s += __builtin_amdgcn_exp2f((v[k] - ref) * c2);
        return;
      }
    }
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const float p = __builtin_amdgcn_exp2f((v[k] - ref) * c2);
      st.s += p;
      if constexpr (MODE == EXP_SQUARE) s1.s = __builtin_fmaf(p, p, s1.s);
    }
  }, y);
  st.s = block_sum<NT>(st.s, red);
  if constexpr (TWO) s1.s = block_sum<NT>(s1.s, red);
  auto fits = [](float s) { return s > 1e-18f && s < INFINITY; };
  if (!fits(st.s) || (TWO && !fits(s1.s))) {
    s1 = st = LogSum();
    z.template each<NT, 1, false, true>([&](int g, float (&v)[W]) __attribute__((always_inline)) {
      if constexpr (TWO) {
        s1.raise(max_of(v), LOG2E);
        const float r = s1.ref();
#pragma unroll
        for (int k = 0; k < W; ++k) s1.s += __builtin_amdgcn_exp2f((v[k] - r) * LOG2E);
      }
      if constexpr (REST) {
        if (q.teacher && names.maybe(g)) without(g, v);
      }
      st.raise(max_of(v), c2);
      const float r = st.ref();
#pragma unroll
      for (int k = 0; k < W; ++k) st.s += __builtin_amdgcn_exp2f((v[k] - r) * c2);
    }, y);
    st = block_logsum<NT>(st, c2, red);
    if constexpr (TWO) s1 = block_logsum<NT>(s1, LOG2E, red);
  }
  const LabelTerm ce = label_term(TWO ? s1 : st, q.zy);
  if (q.label && q.teacher) {
    // the label's share of the teacher's log-sum, unless the teacher names it and has a rest
    bool named = false;
    if constexpr (REST)
      for (int e = names.first(z.group_of(q.y)); e >= 0; e = names.next[e]) named |= names.id[e] == q.y;
    if (!named) st.merge(q.zy, q.zy == -INFINITY ? 0.f : 1.f, c2);
  }
  float other = 0.f, lt = 0.f;
  if constexpr (REST) {
    // the named columns' share again, for the log-sum over all
    other = st.log(inv);
    LogSum n;
    if (q.here) {
      n.m = q.zi;
      n.s = 1.f;
    }
    if (n.m == -INFINITY) n.s = 0.f;
    n = block_logsum<NT>(n, c2, red);
    st.merge(n.m, n.s, c2);
  }
  float kl = 0.f;
  if (a.t.ids) {
    lt = st.log(inv);
    kl = block_sum<NT>(q.p > 0.f || q.p != q.p ? q.p * (q.t - q.zi * inv) : 0.f, red) + lt - q.L;
    if (REST && q.r != 0.f) kl += q.r * (a.t.rest[row] - other);
  }
  if (threadIdx.x == 0) {
    const float tau = a.t.temperature;
    // (a term of weight 0 may be infinite)
    float loss = q.label && a.a != 0.f ? a.a * ce.loss : 0.f;
    if (q.teacher && a.b != 0.f) loss += a.b * tau * tau * kl;
    a.loss[row] = loss;
    *reinterpret_cast<float4*>(a.stats + 4 * row) =
        make_float4(q.label ? ce.logsum : 0.f, q.teacher ? lt : 0.f, REST && q.teacher ? other : 0.f, q.zy);
  }
}

// --------------------------------------------------------------- backward
// Off the named columns c1 exp(z - l1) + ct exp(z / tau - lt): the softmax itself, or with
// a rest what is left of it once the teacher's share of the rest is taken off.  The
// named columns' values are formed first and put in as those come by, so that each
// element is written once (4096 x 128256 bf16, as above: 380 us, 5.5 TB/s).
// A sure label's q - 1 (q above 0.88) is the sum of the others' -q, taken on the way and
// stored by the wave that ends last: as expm1(z - l1) it would have the steps of z, not its
// own digits (all rows sure 385 us; bf16 16384 x 1000 17.4 against 13.9).  Others lose up to
// 3 bits of it, and no time.  Differences are taken before the scaling by log2(e), which
// would overflow in a row of the type's lowest values.
template <bool STREAM>
__device__ __forceinline__ void store_group(bf16_t* p, const float (&v)[8]) {
  store16<STREAM>(p, u32x4_t{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])});
}
template <bool STREAM>
__device__ __forceinline__ void store_group(float* p, const float (&v)[4]) {
  store16<STREAM>(p, __builtin_bit_cast(u32x4_t, v));
}

template <bool BF, int NT, int MODE, bool STREAM>
__global__ void __launch_bounds__(NT) logit_loss_bwd_kernel(LogitLossArgs a) {
  using E = typename Row<BF>::E;
  constexpr int W = Row<BF>::W;
  __shared__ typename NamesOf<NT>::type names;
  __shared__ float red[NT / 64];
  __shared__ int ended;
  const int64_t row = blockIdx.x;
  const Row<BF> z(a.z, row * a.ldz, a.V);
  E* out = static_cast<E*>(a.dz) + row * a.lddz;
  // whole groups where both rows start alike (4096 x 32000 bf16: 97 us, 196 column by column)
  const bool vec = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(z.p)) & 15) == 0;
  // but for column `last` of group `glast`
  auto put = [&](int g, const float (&v)[W], int glast = -1, int last = -1) __attribute__((always_inline)) {
    const int c0 = W * g - z.pad;
    if (vec && c0 >= 0 && c0 + W <= z.V && g != glast) {
      store_group<STREAM>(out + c0, v);
    } else {
#pragma unroll
      for (int k = 0; k < W; ++k)
        if (c0 + k >= 0 && c0 + k < z.V && c0 + k != last) Elem<E>::store(out, c0 + k, v[k]);
    }
  };
  const float4 s = *reinterpret_cast<const float4*>(a.stats + 4 * row);
  const float up = a.scale * (a.dloss ? a.dloss[row] : 1.f);
  const RowTargets q = row_targets<NT, BF>(a, row, z, names, true, red);
  if (!q.label && !q.teacher) {
    const float none[W] = {};
    for (int g = threadIdx.x; g < z.groups(); g += NT) put(g, none);
    return;
  }
  const float tau = a.t.ids ? a.t.temperature : 1.f, inv = 1.f / tau;
  float c1 = q.label ? a.a * up : 0.f, l1 = s.x;
  const float f = q.teacher ? a.b * tau * up : 0.f;
  float ct = f, lt = s.y;
  if (q.teacher && a.t.rest) {
    lt = s.z;
    ct = lt == -INFINITY ? 0.f : f * (expf(s.z - s.y) - q.r);
  }
  const float alpha = c1;
  const bool sure = q.label && alpha != 0.f && s.x - q.zy < 0.125f;
  float others = 0.f;  // exp(z - l1) of this thread's id
  if (q.here) {
    float g = q.teacher ? f * (expf(q.zi * inv - s.y) - q.p) : 0.f;  // (0 times what may overflow)
    if (q.label && q.id != q.y) {
      others = expf(q.zi - s.x);
      g += c1 * others;
    } else if (q.label && !sure) {
      g += c1 * expm1f(q.zi - s.x);
    }
    names.val[threadIdx.x] = g;
  }
  if (threadIdx.x == 0) {
    ended = 0;
    if (q.label) {
      float g = sure ? 0.f : c1 * expm1f(q.zy - s.x);
      if (ct != 0.f) g += ct * expf(q.zy * inv - lt);
      names.val[a.t.k] = g;
    }
  }
  __syncthreads();
  if constexpr (MODE == EXP_ONE) {
    if (!q.teacher) lt = s.x;
    ct += c1;
  } else if constexpr (MODE == EXP_SQUARE) {
    if (!q.teacher || lt == -INFINITY) lt = 0.5f * s.x;  // any shift does for the square alone
    c1 = c1 == 0.f ? 0.f : c1 * expf(2.f * lt - s.x);
  }
  // a term that is not there vanishes also where its exponential would overflow
  if (ct == 0.f && (MODE != EXP_SQUARE || c1 == 0.f)) lt = INFINITY;
  if (c1 == 0.f) l1 = INFINITY;
  float sum = 0.f;  // of unnamed columns' exp(z - l1), as the mode has them
  const int gy = sure ? z.group_of(q.y) : -1;
  auto pass = [&](auto of_sure) __attribute__((always_inline)) {
    constexpr bool SURE = decltype(of_sure)::value;
    z.template each<NT, 4, STREAM>([&](int g, float (&v)[W]) __attribute__((always_inline)) {
      const bool named = names.maybe(g);
      // f(column in the group, entry) of the named ones
      auto each_named = [&](auto&& f) __attribute__((always_inline)) {
        for (int e = names.first(g); e >= 0; e = names.next[e]) {
          const int c = names.id[e];
          if (c >= 0 && z.group_of(c) == g) f(c - (W * g - z.pad), e);
        }
      };
      if (SURE && named)
        each_named([&](int c, int) __attribute__((always_inline)) {
#pragma unroll
          for (int k = 0; k < W; ++k) v[k] = k == c ? -INFINITY : v[k];
        });
      float o[W];
#pragma unroll
      for (int k = 0; k < W; ++k) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(v[k], inv, -lt) * LOG2E);
        if constexpr (MODE == EXP_ONE) {
          o[k] = ct * p;
          if constexpr (SURE) sum += p;
        } else if constexpr (MODE == EXP_SQUARE) {
          o[k] = p * __builtin_fmaf(p, c1, ct);
          if constexpr (SURE) sum = __builtin_fmaf(p, p, sum);
        } else {
          const float p1 = __builtin_amdgcn_exp2f((v[k] - l1) * LOG2E);
          o[k] = __builtin_fmaf(c1, p1, ct * p);
          if constexpr (SURE) sum += p1;
        }
      }
      if (named)
        each_named([&](int c, int e) __attribute__((always_inline)) {
          const float w = names.val[e];
#pragma unroll
          for (int k = 0; k < W; ++k) o[k] = k == c ? w : o[k];
        });
      if constexpr (SURE) put(g, o, gy, q.y);
      else put(g, o);
    });
  };
  if (!sure) {
    pass(std::false_type{});
    return;
  }
  pass(std::true_type{});
  // EXP_SQUARE: c1 holds the factor between the terms and exp(z - l1)
  sum = wave_sum(MODE == EXP_SQUARE ? __builtin_fmaf(sum, c1, others * alpha) : (sum + others) * alpha);
  if ((threadIdx.x & 63) != 0) return;
  red[threadIdx.x >> 6] = sum;
  if (__hip_atomic_fetch_add(&ended, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_WORKGROUP) != NT / 64 - 1) return;
  sum = 0.f;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) sum += red[w];
  float base = 0.f;
  for (int e = names.first(gy); e >= 0; e = names.next[e])
    if (names.id[e] == q.y) base = names.val[e];
  Elem<E>::store(out, q.y, base - sum);
}

// --------------------------------------------------------------- top logits
// The row streams by once, TOP_U groups a thread and round.
//  1. Of the first round's columns the largest of 256 or 1024 strands go to LDS.  The
//     (k + 1)-th largest of them, cut to 16 bits, is a bound: at least k + 1 columns reach
//     it, and with columns in no special order few more do.
//  2. Columns that reach the bound are listed in LDS, the others go into the rest's sum
//     (relative to the bound, so that nothing overflows).  Between rounds a list of twice
//     the length wanted is cut at its own (k + 1)-th largest, the new bound.  What is cut
//     off adds to the rest in units of 2^-40 of the bound's term (the rest holds that
//     term): sums of integers, which do not depend on the order of the list.
//  3. The list is ordered by rank: keys are distinct (value, then lower column first).
// Where the list overflows (many equal values, ascending rows), or there is a NaN, a
// radix search by 8 bits finds the (k + 1)-th largest exactly and a last pass lists what
// is above it and, in order of the columns, what equals it.
// 2048 x 128256 bf16, k 64: 122 us, 4.3 TB/s; two passes over memory for bound and list 172.
constexpr int TOP_U = 8;

// Order of floats as unsigned numbers; -0 as 0, every NaN above all numbers.
__device__ __forceinline__ uint32_t order_of(float v) {
  if (v != v) return 0xffffffffu;
  const uint32_t u = __builtin_bit_cast(uint32_t, v + 0.f);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
  return __builtin_bit_cast(float, o == 0xffffffffu ? 0x7fc00000u : o >> 31 ? o & 0x7fffffffu : ~o);
}

// The largest number, down to bit `last`, that `want` of n keys reach (key lane + 64 i of a
// lane in s[i], 0 past the n-th); one wave.
template <int R>
__device__ __forceinline__ uint32_t reached_by(uint32_t want, int last, uint32_t n, const uint32_t (&s)[R]) {
  uint32_t b = 0;
#pragma unroll 1
  for (int bit = 31; bit >= last; --bit) {
    const uint32_t c = b | (1u << bit);
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (64u * i < n) m += __popcll(__ballot(s[i] >= c));
    if (m >= want) b = c;
    if (m == want) break;
  }
  return b;
}

// STRANDS: 256 up to k = 64, which shorten the search (four keys a lane), else 1024.
template <bool BF, int NT, int STRANDS>
__global__ void __launch_bounds__(NT) top_logits_kernel(int V, const void* x, int64_t ldx, int k, float inv,
                                                        int32_t* ids, float* values, float* rest) {
  constexpr int W = Row<BF>::W, PER = STRANDS > NT ? STRANDS / NT : 1, JOIN = NT > STRANDS ? NT / STRANDS : 1;
  constexpr int CAP = STRANDS == 256 ? 512 : 1024;
  constexpr int MINE = (CAP + NT - 1) / NT;
  static_assert(W % PER == 0, "whole strands a group");
  __shared__ uint32_t strands[CAP];
  __shared__ unsigned long long list[CAP];
  __shared__ float red[NT / 64];
  __shared__ uint32_t bound_s, count_s, hist[256];
  __shared__ unsigned long long cut_s[NT / 64];  // terms cut off the list, by wave
  __shared__ int scan[NT / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x;
  const Row<BF> z(x, row * ldx, V);
  const uint32_t want = (uint32_t)min(k + 1, V);
  const float c2 = inv * LOG2E;

  // groups z.full0 + tid + (at + u) NT; past the row: -inf
  u32x4_t raw[TOP_U];
  constexpr uint32_t NONE = BF ? 0xff80ff80u : 0xff800000u;
  auto load = [&](int at) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < TOP_U; ++u) {
      const int g = z.full0 + tid + (at + u) * NT;
      raw[u] = u32x4_t{NONE, NONE, NONE, NONE};
      if (g < z.full1) raw[u] = z.load(g);
    }
  };
  load(0);
  {
    float m[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) m[i] = -INFINITY;
#pragma unroll
    for (int u = 0; u < TOP_U; ++u) {
      float v[W];
      z.get(raw[u], v);
#pragma unroll
      for (int e = 0; e < W; ++e) m[e / (W / PER)] = fmaxf(m[e / (W / PER)], v[e]);
    }
    if constexpr (JOIN > 1) {
#pragma unroll
      for (int o = 1; o < JOIN; o <<= 1) m[0] = fmaxf(m[0], __shfl_xor(m[0], o, 64));
      if (lane % JOIN == 0) strands[tid / JOIN] = order_of(m[0]);
    } else {
#pragma unroll
      for (int i = 0; i < PER; ++i) strands[tid + NT * i] = order_of(m[i]);
    }
  }
  if (tid == 0) count_s = 0;
  if (tid < NT / 64) cut_s[tid] = 0;
  __syncthreads();
  if (wave == 0) {
    uint32_t s[STRANDS / 64];
#pragma unroll
    for (int i = 0; i < STRANDS / 64; ++i) s[i] = strands[i * 64 + lane];
    const uint32_t c = reached_by(want, 16, STRANDS, s);
    if (lane == 0) bound_s = c;
  }
  __syncthreads();
  uint32_t bound = bound_s;
  float sum = 0.f;  // of exp((x - ref) c) below the bound
  float ref = value_of(bound);
  const bool all = !(ref > -INFINITY && ref < INFINITY);  // no bound among numbers: list what there is
  float least = all ? -INFINITY : ref;
  if (all) ref = 0.f;
  // Entries beyond the list are counted only; the row is searched again then.
  auto append = [&](unsigned long long key) __attribute__((always_inline)) {
    const uint32_t at = atomicAdd(&count_s, 1u);
    if (at < CAP) list[at] = key;
  };
  auto enter = [&](int c, float v) __attribute__((always_inline)) {
    append((unsigned long long)order_of(v) << 32 | (0xffffffffu - (uint32_t)c));
  };
  // A group: the few columns that reach the bound leave it (a NaN too; one that the
  // maximum hides shows in the sum), the rest is summed.  Kept short: unrolled per
  // column, the listing made the kernel too long for the instruction cache (132 us).
  auto take = [&](int g, u32x4_t r) __attribute__((always_inline)) {
    float v[W];
    z.get(r, v);
    uint32_t hits = 0;
    if (!(max_of_group(v) < least)) {
#pragma unroll
      for (int e = 0; e < W; ++e)
        if (!(v[e] < least)) {
          hits |= 1u << e;
          v[e] = -INFINITY;
        }
    }
#pragma unroll
    for (int e = 0; e < W; ++e) sum += __builtin_amdgcn_exp2f((v[e] - ref) * c2);
    while (hits) {
      const int e = __builtin_ctz(hits);
      hits &= hits - 1;
      const int q = BF ? e >> 1 : e;
      const uint32_t lo = q & 1 ? r[1] : r[0], hi = q & 1 ? r[3] : r[2], d = q & 2 ? hi : lo;
      enter(W * g - z.pad + e, __builtin_bit_cast(float, BF ? (e & 1 ? d & 0xffff0000u : d << 16) : d));
    }
  };
  auto cut_off = [&]() -> float {
    unsigned long long c = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) c += cut_s[w];
    return (float)c * 0x1p-40f;
  };
  // cuts the list of n entries at its want-th largest; false where that is no number
  auto tighten = [&](uint32_t n) -> bool {
    if (wave == 0) {
      uint32_t s[CAP / 64];
#pragma unroll
      for (int i = 0; i < CAP / 64; ++i) {
        s[i] = 0;
        if (64u * i < n) s[i] = (uint32_t)(i * 64 + lane) < n ? (uint32_t)(list[i * 64 + lane] >> 32) : 0;
      }
      const uint32_t c = reached_by(want, 0, n, s);
      if (lane == 0) bound_s = c;
    }
    unsigned long long mine[MINE];
#pragma unroll
    for (int i = 0; i < MINE; ++i) mine[i] = (uint32_t)(tid + NT * i) < n ? list[tid + NT * i] : 0;
    __syncthreads();
    const float to = value_of(bound_s);
    if (all || !(to > -INFINITY && to < INFINITY)) return false;
    bound = bound_s;
    if (tid == 0) {
      sum += cut_off();
      count_s = 0;
    }
    __syncthreads();
    sum *= __builtin_amdgcn_exp2f((ref - to) * c2);
    ref = least = to;
    unsigned long long cut = 0;
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
      if (mine[i] == 0) continue;
      const uint32_t o = (uint32_t)(mine[i] >> 32);
      // (waves ahead of this one enter the next round's columns meanwhile)
      if (o >= bound) append(mine[i]);
      else cut += (unsigned long long)(__builtin_amdgcn_exp2f((value_of(o) - ref) * c2) * 0x1p40f);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) cut += __shfl_xor(cut, o, 64);
    if (lane == 0) cut_s[wave] = cut;
    return true;
  };
  const int rounds = (z.full1 - z.full0 + TOP_U * NT - 1) / (TOP_U * NT);
  bool fits = true;
  for (int r = 0; r < rounds && fits; ++r) {
#pragma unroll
    for (int u = 0; u < TOP_U; ++u) {
      const int g = z.full0 + tid + (r * TOP_U + u) * NT;
      if (g < z.full1) take(g, raw[u]);
    }
    if (r + 1 < rounds) load((r + 1) * TOP_U);
    __syncthreads();
    const uint32_t n = count_s;
    __syncthreads();
    if (n > CAP) fits = false;
    else if (n > 2 * want + 32 && r + 1 < rounds) fits = tighten(n);
  }
  if (tid < 2 && z.cut(tid) >= 0) {
    const int c0 = W * z.cut(tid) - z.pad;
#pragma unroll 1
    for (int c = max(c0, 0); c < min(c0 + W, V); ++c) {
      const float v = z.at(c);
      if (!(v < least)) enter(c, v);
      else sum += __builtin_amdgcn_exp2f((v - ref) * c2);
    }
  }
  const bool nan = block_max<NT>(sum == sum ? 0.f : 1.f, red) > 0.f;
  __syncthreads();
  uint32_t n = count_s;
  __syncthreads();
  if (n > CAP || nan) fits = false;
  else if (fits && n > want + 64 && tighten(n)) {
    __syncthreads();
    n = count_s;
  }
  float ties = 0.f;  // columns equal to the bound that are not listed
  if (!fits) {
    // the want-th largest, 8 bits at a time: `above` columns are larger
    uint32_t key = 0, above = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      __syncthreads();
      for (int i = tid; i < 256; i += NT) hist[i] = 0;
      __syncthreads();
      const uint32_t mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
      z.template each<NT, 1>([&](int g, float (&v)[W]) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < W; ++e) {
          const int c = W * g - z.pad + e;
          const uint32_t o = order_of(v[e]);
          if (c >= 0 && c < V && (o & mask) == key) atomicAdd(&hist[o >> shift & 255], 1u);
        }
      });
      __syncthreads();
      if (tid == 0) {
        uint32_t acc = above, d = 255;
        while (d > 0 && acc + hist[d] < want) acc += hist[d--];
        hist[0] = acc;
        hist[1] = d;
      }
      __syncthreads();
      above = hist[0];
      key |= hist[1] << shift;
    }
    // list what is above, then the first columns that equal it
    __syncthreads();
    if (tid == 0) count_s = 0;
    __syncthreads();
    bound = key;
    ref = value_of(bound);
    if (!(ref > -INFINITY && ref < INFINITY)) ref = 0.f;
    sum = 0.f;
    const uint32_t need = want - above;
    uint32_t seen = 0;  // equal columns before this step's
    const int groups = z.groups();
    for (int g0 = 0; g0 < groups; g0 += NT) {
      const int g = g0 + tid;
      float v[W];
#pragma unroll
      for (int e = 0; e < W; ++e) v[e] = 0.f;
      if (g < groups) z.get_cut(g, v);
      uint32_t eq = 0;
#pragma unroll
      for (int e = 0; e < W; ++e) {
        const int c = W * g - z.pad + e;
        if (g >= groups || c < 0 || c >= V) continue;
        const uint32_t o = order_of(v[e]);
        if (o > bound) {
          const uint32_t at = atomicAdd(&count_s, 1u);
          list[at] = (unsigned long long)o << 32 | (0xffffffffu - (uint32_t)c);
        } else if (o == bound) {
          eq |= 1u << e;
        } else {
          sum += __builtin_amdgcn_exp2f((v[e] - ref) * c2);
        }
      }
      // equal columns of the threads before this one
      const int mine = __popc(eq);
      int before = mine;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int t = __shfl_up(before, o, 64);
        if (lane >= o) before += t;
      }
      if (lane == 63) scan[wave] = before;
      __syncthreads();
      uint32_t rank = seen + (uint32_t)(before - mine), all = 0;
      for (int w = 0; w < NT / 64; ++w) {
        if (w < wave) rank += (uint32_t)scan[w];
        all += (uint32_t)scan[w];
      }
#pragma unroll
      for (int e = 0; e < W; ++e)
        if (eq >> e & 1) {
          if (rank < need)
            list[above + rank] = (unsigned long long)bound << 32 | (0xffffffffu - (uint32_t)(W * g - z.pad + e));
          ++rank;
        }
      seen += all;
      __syncthreads();
    }
    n = want;
    ties = (float)(seen - need);
  }
  // ranks; what is listed beyond k goes back to the rest, in order
  const uint32_t kk = (uint32_t)k;
  for (uint32_t i = tid; i < n; i += NT) {
    const unsigned long long me = list[i];
    uint32_t r = 0;
#pragma unroll 8
    for (uint32_t j = 0; j < n; ++j) r += list[j] > me;
    const float v = value_of((uint32_t)(me >> 32));
    if (r < kk) {
      ids[row * k + r] = (int32_t)(0xffffffffu - (uint32_t)me);
      values[row * k + r] = v;
    } else {
      strands[r - kk] = __builtin_bit_cast(uint32_t, v);
    }
  }
  if (!rest) return;
  if (fits && tid == 0) sum += cut_off();
  sum = block_sum<NT>(sum, red);
  if (tid < 64) {
    const float top = n > kk ? __builtin_bit_cast(float, strands[0]) : -INFINITY;  // the rest's largest
    float t = 0.f;
    for (uint32_t i = tid; i < n - kk; i += 64)
      t += __builtin_amdgcn_exp2f((__builtin_bit_cast(float, strands[i]) - top) * c2);
    t = wave_sum(t);
    if (tid == 0) {
      if (sum != 0.f) t += sum * __builtin_amdgcn_exp2f((ref - top) * c2);
      if (ties != 0.f) t += ties * __builtin_amdgcn_exp2f((value_of(bound) - top) * c2);
      rest[row] = top > -INFINITY && top < INFINITY ? top * inv + logf(t) : top;
    }
  }
}

// ----------------------------------------------------------------- launches
hipError_t launch_top_logits(int64_t T, int V, const void* x, int64_t ldx, int dtype, int k, float temperature,
                             int32_t* ids, float* values, float* rest, hipStream_t s) {
  if (T == 0) return hipSuccess;
  const dim3 g((unsigned)T);
  const float inv = 1.f / temperature;
  auto run = [&](auto bf) {
    constexpr bool BF = decltype(bf)::value;
    auto go = [&](auto nt, auto strands) {
      constexpr int NT = decltype(nt)::value, S = decltype(strands)::value;
      hipLaunchKernelGGL((top_logits_kernel<BF, NT, S>), g, dim3(NT), 0, s, V, x, ldx, k, inv, ids, values, rest);
    };
    using std::integral_constant;
    const integral_constant<int, 256> few{};
    const integral_constant<int, 1024> many{};
    // 16 waves a row where long rows are few (bf16, k 64, against four: 1 x 128256 19.6 and
    // 42.7 us, 256 x 128256 28.2 and 46.0, 512 x 128256 49.4 and 54.9, 1024 x 128256 93.5 and
    // 68.2; 256 x 8192 9.1 and 8.9, but 512 x 8192 16.2 and 9.7), a wave where rows are short
    if (T <= 512 && V >= 8192) {
      if (k <= 64) go(many, few);
      else go(many, many);
    } else if (k > 64) {
      go(few, many);
    } else if (V <= 256 * Row<BF>::W) {
      go(integral_constant<int, 64>{}, few);
    } else {
      go(few, few);
    }
  };
  if (dtype == BF16) run(std::true_type{});
  else run(std::false_type{});
  return hipGetLastError();
}

// Which blocks take the rows (times in us; forward / backward, labels alone):
//  - short rows a wave each: bf16 16384 x 1000 11.8 / 19.9, four waves 24.5 / 29.7.  Up to
//    128 groups; the forward up to 512 where there are rows enough (bf16 16384 x 4096
//    28.3 against 39.4; the backward 53.9 against 51.1);
//  - long rows 16 waves in the backward, whose reads and writes come in longer runs then
//    (bf16 4096 x 32000 95.5, four waves 106; 8192 x 16384 93.3 and 92.1), in the forward
//    only where rows are few (16 x 128256 10.3 and 11.9; 1024 x 128256 51.3 and 48.8);
//  - else four waves.
enum { ROW_WAVE, ROW_BLOCK, ROW_WIDE };
template <bool BF>
static int row_kind(const LogitLossArgs& a, bool backward) {
  constexpr int W = Row<BF>::W;
  if (a.t.k <= 64 && (a.V <= 128 * W || (!backward && a.V <= 512 * W && a.T >= 2048))) return ROW_WAVE;
  if (a.V >= 24576 && (backward || a.T <= 512)) return ROW_WIDE;
  return ROW_BLOCK;
}
// Whether loads and stores stream past the caches: where the logits outgrow the L2s
// (forward bf16 1024 x 128256 53.1 without, 48.8 with; 16 x 128256 11.9 and 16.0).
template <bool BF>
static bool row_streams(const LogitLossArgs& a) {
  return streaming(a.T * a.V * (BF ? 2 : 4), 0) > 0;
}

template <bool BF, int NT, int MODE, bool STREAM>
static void logit_forward(const LogitLossArgs& a, bool rest, hipStream_t s) {
  const dim3 g((unsigned)a.T), b(NT);
  if (rest) hipLaunchKernelGGL((logit_loss_kernel<BF, NT, MODE, true, STREAM>), g, b, 0, s, a);
  else hipLaunchKernelGGL((logit_loss_kernel<BF, NT, MODE, false, STREAM>), g, b, 0, s, a);
}
template <bool BF, int MODE>
static void logit_mode(const LogitLossArgs& a, bool rest, bool backward, hipStream_t s) {
  const dim3 g((unsigned)a.T);
  const int kind = row_kind<BF>(a, backward);
  const bool stream = row_streams<BF>(a);
  if (!backward) {
    if (kind == ROW_WAVE) logit_forward<BF, 64, MODE, false>(a, rest, s);
    else if (kind == ROW_WIDE) logit_forward<BF, 1024, MODE, false>(a, rest, s);
    else if (stream) logit_forward<BF, 256, MODE, true>(a, rest, s);
    else logit_forward<BF, 256, MODE, false>(a, rest, s);
  } else if (kind == ROW_WAVE) {
    hipLaunchKernelGGL((logit_loss_bwd_kernel<BF, 64, MODE, false>), g, dim3(64), 0, s, a);
  } else if (kind == ROW_WIDE) {
    if (stream) hipLaunchKernelGGL((logit_loss_bwd_kernel<BF, 1024, MODE, true>), g, dim3(1024), 0, s, a);
    else hipLaunchKernelGGL((logit_loss_bwd_kernel<BF, 1024, MODE, false>), g, dim3(1024), 0, s, a);
  } else {
    if (stream) hipLaunchKernelGGL((logit_loss_bwd_kernel<BF, 256, MODE, true>), g, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((logit_loss_bwd_kernel<BF, 256, MODE, false>), g, dim3(256), 0, s, a);
  }
}
template <bool BF>
static void logit_launch(const LogitLossArgs& a, bool backward, hipStream_t s) {
  const bool hard = a.t.labels != nullptr, soft = a.t.ids != nullptr, rest = soft && a.t.rest;
  const bool two = hard && soft && (rest || a.t.temperature != 1.f);
  if (!two) logit_mode<BF, EXP_ONE>(a, rest, backward, s);
  else if (a.t.temperature == 2.f) logit_mode<BF, EXP_SQUARE>(a, rest, backward, s);
  else logit_mode<BF, EXP_TWO>(a, rest, backward, s);
}

hipError_t launch_logit_loss(const LogitLossArgs& a, int dtype, bool backward, hipStream_t s) {
  if (a.T == 0) return hipSuccess;
  if (dtype == BF16) logit_launch<true>(a, backward, s);
  else logit_launch<false>(a, backward, s);
  return hipGetLastError();
}

}  // namespace zl
