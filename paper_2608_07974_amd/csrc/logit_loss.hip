// Losses of logits in memory, and the top logits of a row (include/zl_loss.h).
// A block per row.  Bound by memory: the forward reads a row once, the backward
// reads and writes it once.
#include "loss.h"
#include "loss_rows.h"

namespace zl {

// ------------------------------------------------------------ rows of logits
// Columns in groups of 8, whose memory is 16-byte aligned from the first full group
// on, wherever the row starts: group g holds columns 8 g - pad .. 8 g - pad + 7 as
// far as they lie in [0, V); only the first and the last may be cut.
template <bool BF>
struct Row {
  using E = typename std::conditional<BF, bf16_t, float>::type;
  const E* p;
  int V, pad, full0, full1;  // full groups [full0, full1)
  __device__ __forceinline__ Row(const void* base, int64_t off, int V_) : p(static_cast<const E*>(base) + off), V(V_) {
    const int skip = (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (int)sizeof(E);
    pad = (8 - skip) & 7;
    full0 = pad ? 1 : 0;
    full1 = (V + pad) >> 3;
  }
  __device__ __forceinline__ int groups() const { return (V + pad + 7) >> 3; }
  // the cut groups: c = 0, 1; -1 where there is none
  __device__ __forceinline__ int cut(int c) const {
    if (c == 0) return pad ? 0 : -1;
    return ((V + pad) & 7) && full1 >= full0 ? full1 : -1;
  }
  __device__ __forceinline__ int group_of(int v) const { return (v + pad) >> 3; }
  __device__ __forceinline__ float at(int v) const { return Elem<E>::load(p, v); }
  struct Raw { uint4 u[BF ? 1 : 2]; };
  __device__ __forceinline__ Raw load(int g) const {
    Raw r;
    const uint4* q = reinterpret_cast<const uint4*>(p + (8 * (int64_t)g - pad));
    r.u[0] = q[0];
    if constexpr (!BF) r.u[1] = q[1];
    return r;
  }
  __device__ static __forceinline__ void get(const Raw& r, float (&v)[8]) {
    if constexpr (BF) {
      const uint32_t w[4] = {r.u[0].x, r.u[0].y, r.u[0].z, r.u[0].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[2 * k] = __builtin_bit_cast(float, w[k] << 16);
        v[2 * k + 1] = __builtin_bit_cast(float, w[k] & 0xffff0000u);
      }
    } else {
      const uint32_t w[8] = {r.u[0].x, r.u[0].y, r.u[0].z, r.u[0].w, r.u[1].x, r.u[1].y, r.u[1].z, r.u[1].w};
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = __builtin_bit_cast(float, w[k]);
    }
  }
  // a cut group, -inf outside the row
  __device__ __forceinline__ void get_cut(int g, float (&v)[8]) const {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int c = 8 * g - pad + k;
      v[k] = c >= 0 && c < V ? at(c) : -INFINITY;
    }
  }
  // f(group, values) for this thread's groups, U loads in flight
  template <int NT, int U, typename F>
  __device__ __forceinline__ void each(F&& f) const {
    int g = full0 + (int)threadIdx.x;
    for (; g + (U - 1) * NT < full1; g += U * NT) {
      Raw r[U];
#pragma unroll
      for (int u = 0; u < U; ++u) r[u] = load(g + u * NT);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float v[8];
        get(r[u], v);
        f(g + u * NT, v);
      }
    }
    for (; g < full1; g += NT) {
      float v[8];
      get(load(g), v);
      f(g, v);
    }
    if (threadIdx.x < 2) {
      const int c = cut((int)threadIdx.x);
      if (c >= 0) {
        float v[8];
        get_cut(c, v);
        f(c, v);
      }
    }
  }
};

// --------------------------------------------------- a row's named columns
// The label and the teacher's ids, found again while the row streams by: a bit for
// every group of 8 columns (exact up to 262144 columns; beyond, groups share
// bits), and behind it chains of entries.  A test costs one broadcast LDS read per
// 8 columns; comparing every column with k ids would cost k.
constexpr int NAME_BITS = 32768, NAME_HEADS = 512, MAX_ENTRIES = ZL_TARGETS_MAX_K + 1;
struct Names {
  uint32_t bits[NAME_BITS / 32];
  int head[NAME_HEADS];
  int id[MAX_ENTRIES];    // column, -1: absent
  int next[MAX_ENTRIES];
  float val[MAX_ENTRIES];

  template <int NT>
  __device__ __forceinline__ void clear() {
    for (int i = threadIdx.x; i < NAME_BITS / 32; i += NT) bits[i] = 0;
    for (int i = threadIdx.x; i < NAME_HEADS; i += NT) head[i] = -1;
  }
  __device__ __forceinline__ void add(int e, int column, int group) {
    id[e] = column;
    atomicOr(&bits[(group >> 5) & (NAME_BITS / 32 - 1)], 1u << (group & 31));
    next[e] = atomicExch(&head[group & (NAME_HEADS - 1)], e);
  }
  __device__ __forceinline__ bool maybe(int group) const {
    return bits[(group >> 5) & (NAME_BITS / 32 - 1)] >> (group & 31) & 1;
  }
};

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
// into `names`.  NT >= ZL_TARGETS_MAX_K.  Ends with a barrier.
template <int NT, bool BF>
__device__ __forceinline__ RowTargets row_targets(const LogitLossArgs& a, int64_t row, const Row<BF>& z, Names& names,
                                                  bool both, float* red) {
  RowTargets q;
  const int tid = threadIdx.x, k = a.t.k, V = a.V;
  q.y = a.t.labels ? a.t.labels[row] : -1;
  q.label = q.y >= 0 && q.y < V;
  q.zy = q.label ? z.at(q.y) : 0.f;
  q.teacher = q.rest = q.here = false;
  q.L = q.r = q.zi = q.p = 0.f;
  q.t = -INFINITY;
  q.id = -1;
  if (!a.t.ids && !(both && q.label)) return q;
  names.template clear<NT>();
  __syncthreads();
  if (tid < k) {
    q.id = a.t.ids[row * k + tid];
    q.here = q.id >= 0 && q.id < V;
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
    for (int e = names.head[z.group_of(q.id) & (NAME_HEADS - 1)]; e >= 0; e = names.next[e])
      twice |= e < tid && names.id[e] == q.id;
  bool named = false;
  if (both && tid == 0 && q.label)
    for (int e = names.head[z.group_of(q.y) & (NAME_HEADS - 1)]; e >= 0; e = names.next[e])
      named |= e < k && names.id[e] == q.y;
  __syncthreads();
  if (twice) {
    names.id[tid] = -1;
    q.here = false;
  }
  if (named) names.id[k] = -1;
  if (a.t.ids) {
    const float inv = 1.f / a.t.temperature;
    if (q.here) {
      q.t = a.t.values[row * k + tid] * inv;
      q.zi = z.at(q.id);
    }
    const float u = a.t.rest ? a.t.rest[row] : -INFINITY;
    const bool any = block_max<NT>(q.here ? 1.f : 0.f, red) > 0.f;
    const float bad = block_sum<NT>(q.here && q.t != q.t ? 1.f : 0.f, red);  // max drops a NaN
    const float m = fmaxf(block_max<NT>(q.t, red), u);
    q.teacher = any && (m != -INFINITY || bad > 0.f || u != u);
    if (q.teacher) {
      const float ref = m == -INFINITY ? 0.f : m;
      const float s = block_sum<NT>(q.here ? expf(q.t - ref) : 0.f, red) + expf(u - ref);
      q.L = ref + logf(s);
      q.rest = u != -INFINITY;
      q.r = q.rest ? expf(u - q.L) : 0.f;
      q.p = q.here ? expf(q.t - q.L) : 0.f;
    }
  }
  __syncthreads();
  return q;
}

// ---------------------------------------------------------------- forward
// TWO: log-sums of z and of z / tau; REST: the latter without the teacher's ids.
template <bool BF, int NT, bool TWO, bool REST>
__global__ void __launch_bounds__(NT) logit_loss_kernel(LogitLossArgs a) {
  __shared__ Names names;
  __shared__ float red[NT / 64];
  const int64_t row = blockIdx.x;
  const Row<BF> z(a.z, row * a.ldz, a.V);
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
  LogSum s1, st;                 // of z, of z / tau (not TWO: st alone, at 1 / tau)
  z.template each<NT, 4>([&](int g, float (&v)[8]) __attribute__((always_inline)) {
    if constexpr (TWO) {
      s1.raise(max_of(v), LOG2E);
      const float ref = s1.ref();
      if constexpr (REST) {
#pragma unroll
        for (int k = 0; k < 8; ++k) s1.s += __builtin_amdgcn_exp2f((v[k] - ref) * LOG2E);
      } else {
        // one maximum serves both
        if (s1.m > st.m) {
          st.s *= __builtin_amdgcn_exp2f((st.m - s1.m) * c2);
          st.m = s1.m;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float x = v[k] - ref;
          s1.s += __builtin_amdgcn_exp2f(x * LOG2E);
          st.s += __builtin_amdgcn_exp2f(x * c2);
        }
      }
    }
    if constexpr (REST) {
      if (q.teacher && names.maybe(g)) {
        for (int e = names.head[g & (NAME_HEADS - 1)]; e >= 0; e = names.next[e]) {
          const int c = names.id[e];
          if (c >= 0 && z.group_of(c) == g) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = 8 * g - z.pad + k == c ? -INFINITY : v[k];
          }
        }
      }
    }
    if constexpr (!TWO || REST) {
      st.raise(max_of(v), c2);
      const float ref = st.ref();
#pragma unroll
      for (int k = 0; k < 8; ++k) st.s += __builtin_amdgcn_exp2f((v[k] - ref) * c2);
    }
  });
  st = block_logsum<NT>(st, c2, red);
  if constexpr (TWO) s1 = block_logsum<NT>(s1, LOG2E, red);
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
  lt = st.log(inv);
  const float l1 = TWO ? s1.log(1.f) : lt;  // (not TWO: tau = 1 where there are labels)
  float kl = 0.f;
  if (a.t.ids) {
    kl = block_sum<NT>(q.p > 0.f || q.p != q.p ? q.p * (q.t - q.zi * inv) : 0.f, red) + lt - q.L;
    if (REST && q.r != 0.f) kl += q.r * (a.t.rest[row] - other);
  }
  if (threadIdx.x == 0) {
    const float tau = a.t.temperature;
    float loss = q.label ? a.a * (l1 - q.zy) : 0.f;
    if (q.teacher) loss += a.b * tau * tau * kl;
    a.loss[row] = loss;
    *reinterpret_cast<float4*>(a.stats + 4 * row) =
        make_float4(q.label ? l1 : 0.f, q.teacher ? lt : 0.f, REST && q.teacher ? other : 0.f, q.zy);
  }
}

// --------------------------------------------------------------- backward
// The named columns' values are formed first and put in as those come by, so that
// each element is written once.
template <bool BF>
__device__ __forceinline__ void store8(typename Row<BF>::E* p, const float (&v)[8]) {
  if constexpr (BF) {
    uint4 u = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    *reinterpret_cast<uint4*>(p) = u;
  } else {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
  }
}

template <bool BF, int NT, bool TWO>
__global__ void __launch_bounds__(NT) logit_loss_bwd_kernel(LogitLossArgs a) {
  using E = typename Row<BF>::E;
  __shared__ Names names;
  __shared__ float red[NT / 64];
  const int64_t row = blockIdx.x;
  const Row<BF> z(a.z, row * a.ldz, a.V);
  E* out = static_cast<E*>(a.dz) + row * a.lddz;
  const bool vec = ((reinterpret_cast<uintptr_t>(out) ^ reinterpret_cast<uintptr_t>(z.p)) & 15) == 0;
  auto put = [&](int g, const float (&v)[8]) __attribute__((always_inline)) {
    const int c0 = 8 * g - z.pad;
    if (vec && c0 >= 0 && c0 + 8 <= z.V) {
      store8<BF>(out + c0, v);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (c0 + k >= 0 && c0 + k < z.V) Elem<E>::store(out, c0 + k, v[k]);
    }
  };
  const RowTargets q = row_targets<NT, BF>(a, row, z, names, true, red);
  if (!q.label && !q.teacher) {
    const float none[8] = {};
    for (int g = threadIdx.x; g < z.groups(); g += NT) put(g, none);
    return;
  }
  const float4 s = *reinterpret_cast<const float4*>(a.stats + 4 * row);
  const float up = a.scale * (a.dloss ? a.dloss[row] : 1.f);
  const float tau = a.t.ids ? a.t.temperature : 1.f, inv = 1.f / tau;
  const float c1 = q.label ? a.a * up : 0.f, f = q.teacher ? a.b * tau * up : 0.f;
  // off the named columns c1 exp(z - l1) + ct exp(z / tau - lt): the softmax itself, or
  // with a rest what is left of it once the teacher's share of the rest is taken off
  float ct = f, lt = s.y;
  if (q.teacher && a.t.rest) {
    lt = s.z;
    ct = lt == -INFINITY ? 0.f : f * (expf(s.z - s.y) - q.r);
  }
  // the named columns
  if (q.here) {
    float g = f * (expf(q.zi * inv - s.y) - q.p);
    if (q.label) g += c1 * (q.id == q.y ? expm1f(q.zi - s.x) : expf(q.zi - s.x));
    names.val[threadIdx.x] = g;
  }
  if (threadIdx.x == 0 && q.label) {
    float g = c1 * expm1f(q.zy - s.x);
    if (ct != 0.f) g += ct * expf(q.zy * inv - lt);
    names.val[a.t.k] = g;
  }
  __syncthreads();
  if constexpr (!TWO) {
    // one exponential: labels or a teacher alone, or both at tau = 1 without a rest
    if (!q.teacher) lt = s.x;
    ct += c1;
  }
  z.template each<NT, 4>([&](int g, float (&v)[8]) __attribute__((always_inline)) {
    float o[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(v[k], inv, -lt) * LOG2E);
      o[k] = ct != 0.f ? ct * p : 0.f;
      if constexpr (TWO) {
        const float p1 = __builtin_amdgcn_exp2f((v[k] - s.x) * LOG2E);
        o[k] += c1 != 0.f ? c1 * p1 : 0.f;
      }
    }
    if (names.maybe(g)) {
      for (int e = names.head[g & (NAME_HEADS - 1)]; e >= 0; e = names.next[e]) {
        const int c = names.id[e];
        if (c >= 0 && z.group_of(c) == g) {
          const float w = names.val[e];
#pragma unroll
          for (int k = 0; k < 8; ++k) o[k] = 8 * g - z.pad + k == c ? w : o[k];
        }
      }
    }
    put(g, o);
  });
}

// --------------------------------------------------------------- top logits
// 1. The row streams by once; the largest values of 1024 strands of it (a strand:
//    four of every 8 columns of one thread) go to LDS.  The (k + 1)-th largest of
//    them, cut to 16 bits, is a bound: at least k + 1 columns reach it, and with
//    columns in no special order few more do.
// 2. The row streams by again (mostly out of the caches): columns that reach the
//    bound are listed, the others go into the rest's sum.
// 3. The list is ordered by rank: keys are distinct (value, then lower column first).
// Where the list overflows (many equal values) a radix search by 8 bits finds the
// (k + 1)-th largest exactly and a last pass lists what is above it and, in order of
// the columns, what equals it.
constexpr int TT = 512, TOP_CAP = 1024;

// Order of floats as unsigned numbers; -0 as 0, every NaN above all numbers.
__device__ __forceinline__ uint32_t order_of(float v) {
  if (v != v) return 0xffffffffu;
  const uint32_t u = __builtin_bit_cast(uint32_t, v + 0.f);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
  return __builtin_bit_cast(float, o == 0xffffffffu ? 0x7fc00000u : o >> 31 ? o & 0x7fffffffu : ~o);
}

template <bool BF>
__global__ void __launch_bounds__(TT) top_logits_kernel(int V, const void* x, int64_t ldx, int k, float inv,
                                                        int32_t* ids, float* values, float* rest) {
  __shared__ uint32_t strands[2 * TT];
  __shared__ unsigned long long list[TOP_CAP];
  __shared__ float red[TT / 64];
  __shared__ uint32_t bound_s, count_s, hist[256];
  __shared__ int scan[TT / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x;
  const Row<BF> z(x, row * ldx, V);
  const uint32_t want = (uint32_t)min(k + 1, V);
  const float c2 = inv * LOG2E;

  float m0 = -INFINITY, m1 = -INFINITY;
  z.template each<TT, 4>([&](int, float (&v)[8]) __attribute__((always_inline)) {
    m0 = fmaxf(m0, fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])));
    m1 = fmaxf(m1, fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
  });
  strands[tid] = order_of(m0);
  strands[TT + tid] = order_of(m1);
  if (tid == 0) count_s = 0;
  __syncthreads();
  if (wave == 0) {
    // the largest bound of 16 bits that `want` strands reach
    uint32_t s[2 * TT / 64];
#pragma unroll
    for (int i = 0; i < 2 * TT / 64; ++i) s[i] = strands[i * 64 + lane];
    uint32_t b = 0;
    for (int bit = 31; bit >= 16; --bit) {
      const uint32_t c = b | (1u << bit);
      uint32_t n = 0;
#pragma unroll
      for (int i = 0; i < 2 * TT / 64; ++i) n += __popcll(__ballot(s[i] >= c));
      if (n >= want) b = c;
    }
    if (lane == 0) bound_s = b;
  }
  __syncthreads();
  uint32_t bound = bound_s;
  float sum = 0.f;  // of exp((x - ref) c) below the bound
  float ref = value_of(bound);
  if (!(ref > -INFINITY && ref < INFINITY)) ref = 0.f;
  z.template each<TT, 4>([&](int g, float (&v)[8]) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = 8 * g - z.pad + e;
      const uint32_t o = order_of(v[e]);
      if (o >= bound) {
        if (c >= 0 && c < V) {
          const uint32_t at = atomicAdd(&count_s, 1u);
          if (at < TOP_CAP) list[at] = (unsigned long long)o << 32 | (0xffffffffu - (uint32_t)c);
        }
      } else {
        sum += __builtin_amdgcn_exp2f((v[e] - ref) * c2);
      }
    }
  });
  __syncthreads();
  uint32_t n = count_s;
  float ties = 0.f;  // columns equal to the bound that are not listed
  if (n > TOP_CAP) {
    // the want-th largest, 8 bits at a time: `above` columns are larger
    uint32_t key = 0, above = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      __syncthreads();
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      const uint32_t mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
      z.template each<TT, 1>([&](int g, float (&v)[8]) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int c = 8 * g - z.pad + e;
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
    for (int g0 = 0; g0 < groups; g0 += TT) {
      const int g = g0 + tid;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.f;
      if (g < groups) z.get_cut(g, v);
      uint32_t eq = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = 8 * g - z.pad + e;
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
      for (int w = 0; w < TT / 64; ++w) {
        if (w < wave) rank += (uint32_t)scan[w];
        all += (uint32_t)scan[w];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (eq >> e & 1) {
          if (rank < need)
            list[above + rank] = (unsigned long long)bound << 32 | (0xffffffffu - (uint32_t)(8 * g - z.pad + e));
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
  for (uint32_t i = tid; i < n; i += TT) {
    const unsigned long long me = list[i];
    uint32_t r = 0;
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
  sum = block_sum<TT>(sum, red);
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
  const dim3 g((unsigned)T), b(TT);
  const float inv = 1.f / temperature;
  if (dtype == BF16)
    hipLaunchKernelGGL((top_logits_kernel<true>), g, b, 0, s, V, x, ldx, k, inv, ids, values, rest);
  else
    hipLaunchKernelGGL((top_logits_kernel<false>), g, b, 0, s, V, x, ldx, k, inv, ids, values, rest);
  return hipGetLastError();
}

template <bool BF, int NT>
static void logit_forward(const LogitLossArgs& a, bool two, bool rest, hipStream_t s) {
  const dim3 g((unsigned)a.T), b(NT);
  if (two && rest) hipLaunchKernelGGL((logit_loss_kernel<BF, NT, true, true>), g, b, 0, s, a);
  else if (two) hipLaunchKernelGGL((logit_loss_kernel<BF, NT, true, false>), g, b, 0, s, a);
  else if (rest) hipLaunchKernelGGL((logit_loss_kernel<BF, NT, false, true>), g, b, 0, s, a);
  else hipLaunchKernelGGL((logit_loss_kernel<BF, NT, false, false>), g, b, 0, s, a);
}
template <bool BF, int NT>
static void logit_backward(const LogitLossArgs& a, bool two, hipStream_t s) {
  const dim3 g((unsigned)a.T), b(NT);
  if (two) hipLaunchKernelGGL((logit_loss_bwd_kernel<BF, NT, true>), g, b, 0, s, a);
  else hipLaunchKernelGGL((logit_loss_bwd_kernel<BF, NT, false>), g, b, 0, s, a);
}

hipError_t launch_logit_loss(const LogitLossArgs& a, int dtype, bool backward, hipStream_t s) {
  if (a.T == 0) return hipSuccess;
  const bool hard = a.t.labels != nullptr, soft = a.t.ids != nullptr, rest = soft && a.t.rest;
  const bool two = hard && soft && (rest || a.t.temperature != 1.f);
  const bool bf = dtype == BF16;
  if (!backward) {
    if (bf) logit_forward<true, 256>(a, two, rest, s);
    else logit_forward<false, 256>(a, two, rest, s);
  } else {
    if (bf) logit_backward<true, 256>(a, two, s);
    else logit_backward<false, 256>(a, two, s);
  }
  return hipGetLastError();
}

}  // namespace zl
