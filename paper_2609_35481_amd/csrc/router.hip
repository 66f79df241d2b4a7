// The router on gfx950: top-k ids and weights of every token from its
// logits, and the gradient back to the logits.
//
//   route_list_kernel  up to eight experts a token: 4 to 16 lanes hold a row and
//                      merge sorted lists (below)
//   route_kernel       more than eight, or few tokens: 16 or 64 lanes take the
//                      largest key of the row k times
//   route_backward_chosen_kernel, route_backward_kernel  the gradient where the
//                      chosen logits alone count, and where all do
//
// Bound: the forward by its comparisons (846 vector instructions for 16 rows of
// 128; 200003 x 128: vector units busy 17.4 of 23.3 us, 4.9 TB/s; 200003 x 128 of 16 bits
// 23.1; 16384 x 512 with groups and a bias 1326 instructions, 9.1 of 13 us; beyond eight
// choices a maximum each: 200003 x 256, top-16, 143 us), few tokens by the chain of
// one row (3.0 us a launch); the gradient by memory: 200003 x 256 bf16 31 us for
// 102 MB written and 105 read, the lines that hold a chosen logit.
#include "router.h"

namespace {

using namespace topoep_dev;

typedef int v4i __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

struct Route {
  RouterArgs r;
  const void *logits;
  int64_t ld;
  int T;
  const float *bias;
  int32_t *ids;
  float *weights;
};

template <class T, int LPT, int V>
__global__ __launch_bounds__(kThreads) void route_kernel(Route a) {
  constexpr int kRows = kThreads / LPT;   // rows a workgroup holds at once
  __shared__ uint32_t scratch[kRows][kRouteScratch];
  const int slot = threadIdx.x / LPT, sub = threadIdx.x % LPT;
  float b[V];
#pragma unroll
  for (int v = 0; v < V; ++v) b[v] = a.bias && sub * V + v < a.r.E ? a.bias[sub * V + v] : 0.0f;
  for (int64_t t0 = (int64_t)blockIdx.x * kRows; t0 < a.T; t0 += (int64_t)gridDim.x * kRows) {
    const int64_t t = t0 + slot;
    const bool live = t < a.T;
    float x[V];
    load_logits<T, V>(static_cast<const T *>(a.logits) + (live ? t : t0) * a.ld, sub * V, a.r.E, x);
    route_row<LPT, V>(a.r, x, b, sub, scratch[slot], live, a.ids + t * a.r.k, a.weights + t * a.r.k);
  }
}

// ---------------------------------------------------------------- sorted lists

// Up to eight experts a token: a few lanes hold a row, V experts each, and
// keep the K largest as a sorted list; lists are merged over the lanes, after
// which every lane holds the row's.  An entry is the key as a 64-bit float,
// whose low bits, zero in every converted 32-bit float, hold the expert's id so
// that of equal keys the lower id is the larger number: a comparison and its
// exchange are one maximum and one minimum, with no tie to look after.
// -inf (masked) becomes -2^129, below every 32-bit float, an overflown key 2^129;
// what cannot be chosen lies below them all.
constexpr int kIdBits = 10;
constexpr uint32_t kIdMask = (1u << kIdBits) - 1;
static_assert(TOPOEP_ROUTER_MAX_EXPERTS <= (int)kIdMask + 1, "ids fit an entry");

// The larger and the smaller of two numbers, neither of them a signalling NaN
// (fmax and fmin would first quiet their operands, an instruction each: a
// third of all).
__device__ inline double larger(double a, double b) {
  double r;
  asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ inline double smaller(double a, double b) {
  double r;
  asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}

// anti: the id's complement in kIdBits, which goes into the low bits as it is
// where the key is not negative, and complemented again where it is.
template <bool Bias>
__device__ inline double entry(float key, uint32_t anti) {
  double d = key + 0.0f;   // -0 and +0 are one key
  if (Bias) {
    d = d != d ? -0x1p129 : d;
    d = smaller(d, 0x1p129);
  }
  d = larger(d, -0x1p129);
  const uint64_t u = (uint64_t)__double_as_longlong(d);
  const uint32_t code = ((uint32_t)((int32_t)(u >> 32) >> 31) ^ anti) & kIdMask;
  return __longlong_as_double((int64_t)(u | code));
}
__device__ inline int entry_id(double e) {
  const uint64_t u = (uint64_t)__double_as_longlong(e);
  return (int)(((uint32_t)u ^ ~(uint32_t)((int32_t)(u >> 32) >> 31)) & kIdMask);
}

__device__ inline void order(double &a, double &b) {   // a >= b
  const double hi = larger(a, b), lo = smaller(a, b);
  a = hi;
  b = lo;
}

// A list that rises and then falls, or the reverse, in descending order.
template <int K>
__device__ inline void settle(double (&l)[K]) {
#pragma unroll
  for (int d = K / 2; d > 0; d /= 2)
#pragma unroll
    for (int i = 0; i < K; ++i)
      if ((i & d) == 0) order(l[i], l[i + d]);
}

template <int K>
__device__ inline void sort(double (&l)[K]) {
  if constexpr (K == 4) {
    order(l[0], l[2]); order(l[1], l[3]);
    order(l[0], l[1]); order(l[2], l[3]);
    order(l[1], l[2]);
  } else {   // 19 exchanges: two halves of four, then their merge
    static_assert(K == 8, "");
    order(l[0], l[2]); order(l[1], l[3]); order(l[4], l[6]); order(l[5], l[7]);
    order(l[0], l[1]); order(l[2], l[3]); order(l[4], l[5]); order(l[6], l[7]);
    order(l[1], l[2]); order(l[5], l[6]);
    order(l[0], l[4]); order(l[1], l[5]); order(l[2], l[6]); order(l[3], l[7]);
    order(l[2], l[4]); order(l[3], l[5]);
    order(l[1], l[2]); order(l[3], l[4]); order(l[5], l[6]);
  }
}

// l: the K largest of two descending lists.
template <int K>
__device__ inline void merge(double (&l)[K], const double (&o)[K]) {
#pragma unroll
  for (int i = 0; i < K; ++i) l[i] = larger(l[i], o[K - 1 - i]);
  settle(l);
}

template <int C>
__device__ inline double dpp_movd(double v) { return __longlong_as_double((int64_t)dpp_mov64<C>((uint64_t)__double_as_longlong(v))); }

// Lanes exchange with a partner of the other half of 2, 4, 8 and 16 lanes
// (neighbour, next but one, mirror images), LPT lanes in all.
template <int K, int C>
__device__ inline void merge_over(double (&l)[K]) {
  // a lane move may read a register two wait states after its writing at the
  // earliest; the compiler counts them for its own instructions only
  if constexpr (K == 4)
    asm volatile("s_nop 1" : "+v"(l[0]), "+v"(l[1]), "+v"(l[2]), "+v"(l[3]));
  else
    asm volatile("s_nop 1" : "+v"(l[0]), "+v"(l[1]), "+v"(l[2]), "+v"(l[3]), "+v"(l[4]), "+v"(l[5]), "+v"(l[6]), "+v"(l[7]));
  double o[K];
#pragma unroll
  for (int i = 0; i < K; ++i) o[i] = dpp_movd<C>(l[i]);
  merge(l, o);
}
template <int LPT, int K>
__device__ inline void merge_row(double (&l)[K]) {
  if (LPT > 1) merge_over<K, 0xB1>(l);
  if (LPT > 2) merge_over<K, 0x4E>(l);
  if (LPT > 4) merge_over<K, 0x141>(l);
  if (LPT > 8) merge_over<K, 0x140>(l);
}
// The groups' largest keys in LDS (`best`, a word a group), where groups and
// lanes need not fit.
template <int LPT, int V, class Key>
__device__ inline void best_of_groups(const RouterArgs &r, int sub, uint32_t *best, const Key &key) {
  const int base = sub * V, m = r.per_group;
  for (int q = sub; q < r.groups; q += LPT) best[q] = 0;
  wave_sync();
  int g = base / m, pos = base - g * m;
  float run = -INFINITY;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    run = fmaxf(run, key(v));   // passes over a NaN key, which counts as -inf
    if (++pos == m || v == V - 1) {
      if (g < r.groups) atomicMax(&best[g], key_word(run));
      run = -INFINITY;
      pos = 0;
      ++g;
    }
  }
  wave_sync();
}

// Up to eight open groups, as a list of (key, group).
template <int LPT, bool Bias>
__device__ inline void list_groups(const RouterArgs &r, int sub, const uint32_t *best, double (&l)[8]) {
  double o[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) l[i] = -0x1p200;
  for (int q0 = 0; q0 < r.groups; q0 += 8 * LPT) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int q = q0 + i * LPT + sub;
      const uint32_t w = best[q < r.groups ? q : 0];
      const float k = __uint_as_float(w & 0x80000000u ? w ^ 0x80000000u : ~w);
      o[i] = entry<Bias>(k, (uint32_t)q ^ kIdMask);
      o[i] = q < r.groups ? o[i] : -0x1p200;
    }
    sort(o);
    merge(l, o);
  }
  merge_row<LPT>(l);
}

// Any number of open groups, a bit each: counted against each other.
template <int LPT>
__device__ inline uint64_t count_groups(const RouterArgs &r, int sub, const uint32_t *best) {
  uint64_t mask = 0;
  for (int q = sub; q < r.groups; q += LPT) {
    const uint32_t mine = best[q];
    int above = 0;
    for (int o = 0; o < r.groups; ++o) {
      const uint32_t w = best[o];
      above += w > mine || (w == mine && o < q) ? 1 : 0;
    }
    mask |= above < r.top_groups ? 1ull << q : 0ull;
  }
  if (LPT > 1) mask |= dpp_mov64<0xB1>(mask);
  if (LPT > 2) mask |= dpp_mov64<0x4E>(mask);
  if (LPT > 4) mask |= dpp_mov64<0x141>(mask);
  if (LPT > 8) mask |= dpp_mov64<0x140>(mask);
  return mask;
}

// The row's list from the experts of its open groups alone, which are read
// again: candidate c is expert c % m of open group c / m.  `chosen`: eight
// words of LDS of the row's own.
template <class T, int LPT, bool Bias>
__device__ inline void list_candidates(const Route &a, const T *row, int sub, const double (&groups)[8], uint32_t *chosen,
                                       double (&l)[8]) {
  if (sub == 0) {
#pragma unroll
    for (int i = 0; i < 8; ++i) chosen[i] = (uint32_t)(entry_id(groups[i]) * a.r.per_group);
  }
  wave_sync();
  const int m = a.r.per_group, n = a.r.top_groups * m;
  const uint32_t inverse = ((1u << 20) + (uint32_t)m - 1) / (uint32_t)m;   // exact: c m < 2^20
  for (int c0 = 0; c0 < n; c0 += 8 * LPT) {
    double o[8];
    T raw[8];
    float bias[8];
    uint32_t id[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t c = (uint32_t)imin(c0 + i * LPT + sub, n - 1), j = c * inverse >> 20;
      id[i] = chosen[j] + (c - j * (uint32_t)m);
      raw[i] = row[id[i]];
      bias[i] = Bias ? a.bias[id[i]] : 0.0f;
    }
    // entries formed among the loads (two scalings of an id, for 16-bit logits and
    // 32-bit biases) take 133 registers, of the 128 that four waves a SIMD have; behind them 120
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = clean_logit(to_float(raw[i]));
      o[i] = entry<Bias>(Bias ? x + bias[i] : x, id[i] ^ kIdMask);
      o[i] = c0 + i * LPT + sub < n ? o[i] : -0x1p200;
    }
    sort(o);
    if (c0 == 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) l[i] = o[i];
    } else {
      merge(l, o);
    }
  }
}

// GL: groups a lane holds (a group may also span 2, 4 or 8 lanes: GL = 1); 0: no
// groups; -1: groups of any size.  Places beyond E hold masked logits of ids that no expert has: any
// expert comes before them.
template <class T, int LPT, int V, int K, int GL, bool Bias>
__global__ __launch_bounds__(kThreads, V <= 32 ? 4 : 2) void route_list_kernel(Route a) {
  constexpr int kRows = kThreads / LPT;
  const int sub = threadIdx.x % LPT, E = a.r.E, base = sub * V;
  const int64_t t = (int64_t)blockIdx.x * kRows + threadIdx.x / LPT;
  const bool live = t < a.T;
  const T *row = static_cast<const T *>(a.logits) + (live ? t : (int64_t)a.T - 1) * a.ld;
  const uint32_t anti = (uint32_t)base ^ kIdMask;   // V is a power of two: ids base + v are base ^ v
  float x[V], b[Bias ? V : 1];
  load_logits<T, V>(row, base, E, x);
  if constexpr (Bias) {
    if (base + V <= E) {
      __builtin_memcpy(b, a.bias + base, sizeof(b));
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) b[v] = base + v < E ? a.bias[base + v] : 0.0f;
    }
  }
  // scores over every logit: their largest and the sum, before the logits become keys
  float all = 0.0f, most = 0.0f;
  if (!a.r.sigmoid && !a.r.renorm) {
    most = x[0];
#pragma unroll
    for (int v = 1; v < V; ++v) most = fmaxf(most, x[v]);
    most = row_maxf<LPT>(most);
    const float from = most == -INFINITY ? 0.0f : most;
    float e[V];
#pragma unroll
    for (int v = 0; v < V; ++v) e[v] = exp_term(x[v] - from);
    all = row_sum<LPT>(lane_sum(e));
  }
  if constexpr (Bias) {
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] += b[v];
  }
  const auto key = [&](int v) { return x[v]; };
  double l[K];
  uint64_t lane_open = ~0ull;   // bit v: expert base + v's group is open
  bool listed = false;          // l is made already
  if constexpr (GL != 0) {
    __shared__ uint32_t chosen[kRows][8];
    double groups[8];
    const int m = a.r.per_group;
    const bool few = a.r.top_groups <= 8;
    uint64_t mask = 0;
    if constexpr (GL < 0) {
      __shared__ uint32_t best[kRows][64];
      best_of_groups<LPT, V>(a.r, sub, best[threadIdx.x / LPT], key);
      if (few) list_groups<LPT, Bias>(a.r, sub, best[threadIdx.x / LPT], groups);
      else mask = count_groups<LPT>(a.r, sub, best[threadIdx.x / LPT]);
    } else {
      constexpr int M = V / GL;
      const int span = m / V;   // lanes a group spans, where it spans any
#pragma unroll
      for (int i = 0; i < 8; ++i) groups[i] = -0x1p200;
#pragma unroll
      for (int g = 0; g < GL; ++g) {
        float top = -INFINITY;
#pragma unroll
        for (int v = 0; v < M; ++v) top = fmaxf(top, key(g * M + v));   // passes over a NaN key, which counts as -inf
        if (GL == 1) {
          if (span > 1) top = fmaxf(top, dpp_movf<0xB1>(top));
          if (span > 2) top = fmaxf(top, dpp_movf<0x4E>(top));
          if (span > 4) top = fmaxf(top, dpp_movf<0x141>(top));
        }
        const int mine = GL == 1 && span > 1 ? sub / span : sub * GL + g;
        if (mine < a.r.groups && (GL > 1 || span <= 1 || sub % span == 0))
          groups[g] = entry<Bias>(top, (uint32_t)mine ^ kIdMask);
      }
      sort(groups);
      merge_row<LPT>(groups);
    }
    if (few && 2 * a.r.top_groups * m <= E) {   // half of the experts or fewer are left
      list_candidates<T, LPT, Bias>(a, row, sub, groups, chosen[threadIdx.x / LPT], l);
      listed = true;
    } else {
      if (few) {
#pragma unroll
        for (int i = 0; i < 8; ++i) mask |= i < a.r.top_groups ? 1ull << entry_id(groups[i]) : 0ull;
      }
      lane_open = 0;
      int g = base / m, pos = base - g * m;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        lane_open |= (g < a.r.groups ? (mask >> g) & 1 : 0ull) << v;
        if (++pos == m) {
          pos = 0;
          ++g;
        }
      }
    }
  }
  if (GL == 0 || !listed) {
#pragma unroll
    for (int c = 0; c < (V + K - 1) / K; ++c) {
      double o[K];
#pragma unroll
      for (int i = 0; i < K; ++i) {
        const int v = c * K + i;
        if (v >= V) {
          o[i] = -0x1p200;
          continue;
        }
        o[i] = entry<Bias>(key(v < V ? v : 0), anti ^ (uint32_t)v);
        if (GL != 0) o[i] = (lane_open >> (v < V ? v : 0)) & 1 ? o[i] : -0x1p200;
      }
      sort(o);
      if (c == 0) {
#pragma unroll
        for (int i = 0; i < K; ++i) l[i] = o[i];
      } else {
        merge(l, o);
      }
    }
  }
  merge_row<LPT>(l);
  float s[K];   // the chosen logits, then their weights
#pragma unroll
  for (int j = 0; j < K; ++j) s[j] = (float)l[j];   // the key: -2^129 becomes -inf again
  if (Bias) {
#pragma unroll
    for (int j = 0; j < K; ++j) s[j] = j < a.r.k ? clean_logit(to_float(row[entry_id(l[j])])) : -INFINITY;
  }
  float f = a.r.scale, m = s[0];   // m: the largest chosen logit, or of all
#pragma unroll
  for (int j = 1; j < K; ++j) m = j < a.r.k ? fmaxf(m, s[j]) : m;
  if (a.r.sigmoid) {
    const float top = a.r.renorm ? sigmoid_top(m) : 0.0f;
#pragma unroll
    for (int j = 0; j < K; ++j) s[j] = j < a.r.k ? sigmoid_score(s[j], top) : 0.0f;
    if (a.r.renorm) f = over(a.r.scale, lane_sum(s));
  } else {
    if (!a.r.renorm) m = most;
    const float from = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int j = 0; j < K; ++j) s[j] = j < a.r.k ? exp_from(s[j], from) : 0.0f;
    f = over(a.r.scale, a.r.renorm ? lane_sum(s) : all);
  }
#pragma unroll
  for (int j = 0; j < K; ++j) s[j] *= f;
  if (!live) return;
  int32_t *ids = a.ids + t * a.r.k;
  float *weights = a.weights + t * a.r.k;
  if (sub == 0) {
    if (a.r.k == K) {
      int32_t id[K];
#pragma unroll
      for (int j = 0; j < K; ++j) id[j] = entry_id(l[j]);
      __builtin_memcpy(ids, id, sizeof(id));
    } else {
#pragma unroll
      for (int j = 0; j < K; ++j)
        if (j < a.r.k) ids[j] = entry_id(l[j]);
    }
  }
  if (sub == 1) {
    if (a.r.k == K) {
      __builtin_memcpy(weights, s, sizeof(s));
    } else {
#pragma unroll
      for (int j = 0; j < K; ++j)
        if (j < a.r.k) weights[j] = s[j];
    }
  }
}

struct RouteBackward {
  RouterArgs r;
  const void *logits;
  int64_t ld;
  int T;
  const int32_t *ids;
  const float *grad;
  void *out;
  int64_t ldg;
};

// The chosen scores' gradients, back through the renormalisation (and the
// sigmoid): of the logits where only chosen ones count.  KP lanes hold a row's
// choices; `in`: this lane has one.  A score of zero gets no gradient, whatever
// the others', so that a row's NaN stays off its masked places.
template <int KP>
__device__ inline float chosen_gradient(const RouterArgs &r, bool in, float xj, float g) {
  const float m = r.renorm ? row_maxf<KP>(xj) : 0.0f;
  if (r.sigmoid) {
    float s = in ? sigmoid_score(xj, r.renorm ? sigmoid_top(m) : 0.0f) : 0.0f;
    if (r.renorm) {
      s *= over(1.0f, row_sum<KP>(s));
      g -= row_sum<KP>(g * s);
    }
    return s > 0.0f ? g * s * sigmoid_score(-xj, 0.0f) : 0.0f;
  }
  const float e = exp_from(xj, m == -INFINITY ? 0.0f : m);
  const float q = e * over(1.0f, row_sum<KP>(e));
  const float mean = row_sum<KP>(g * q);
  return q > 0.0f ? q * (g - mean) : 0.0f;
}

// Where only the chosen logits count, a wave takes `rows` rows at once: KP
// lanes a row form its choices' gradients, which go into a dense image of the
// rows in LDS, zero elsewhere; the image is written out in whole lines, and the
// choices' places are cleared for the next rows.  Bound: memory, the output's
// lines and those that hold a chosen logit.
constexpr int kImageBytes = 4096;   // of a wave

template <class T, int KP>
__global__ __launch_bounds__(kThreads) void route_backward_chosen_kernel(RouteBackward a, int rows) {
  constexpr int W = 16 / sizeof(T);
  __shared__ v4i images[kThreads / 64][kImageBytes / 16];
  const int lane = lane_id(), sub = lane % KP, slot = lane / KP, E = a.r.E;
  const int wave = uniform_i32(threadIdx.x >> 6);
  v4i *wide = images[wave];
  T *image = reinterpret_cast<T *>(wide);
  for (int i = lane; i < kImageBytes / 16; i += 64) wide[i] = v4i{0, 0, 0, 0};
  wave_sync();
  const int64_t every = (int64_t)gridDim.x * (kThreads / 64) * rows;
  for (int64_t t0 = ((int64_t)blockIdx.x * (kThreads / 64) + wave) * rows; t0 < a.T; t0 += every) {
    const int live = a.T - t0 < rows ? (int)(a.T - t0) : rows;
    const bool mine = slot < live && sub < a.r.k;
    const int64_t t = t0 + (mine ? slot : 0);
    const int id = mine ? a.ids[t * a.r.k + sub] : -1;
    const float dw = mine ? a.r.scale * a.grad[t * a.r.k + sub] : 0.0f;
    const bool in = (unsigned)id < (unsigned)E;
    const float xj = in ? clean_logit(to_float(static_cast<const T *>(a.logits)[t * a.ld + id])) : -INFINITY;
    const float g = xj > -INFINITY ? dw : 0.0f;   // a masked choice's weight is a constant zero
    const float d = chosen_gradient<KP>(a.r, in, xj, g);
    if (in) image[slot * E + id] = from_float<T>(d);
    wave_sync();
    T *to = static_cast<T *>(a.out) + t0 * a.ldg;
    if (a.ldg == E) {
      const int n = live * E;
      int i = lane * W;
      for (; i + W <= n; i += 64 * W) __builtin_memcpy(to + i, image + i, 16);
      if (i < n)
        for (; i < n; ++i) to[i] = image[i];
    } else {
      for (int r = 0; r < live; ++r)
        for (int i = lane; i < E; i += 64) to[r * a.ldg + i] = image[r * E + i];
    }
    wave_sync();
    if (in) image[slot * E + id] = from_float<T>(0.0f);
    wave_sync();
  }
}

// Softmax scores over every logit: d = gradient of the row's chosen scores lies
// in LDS by expert while the row's lanes write their elements, and is cleared
// again after them.
template <class T, int LPT, int V>
__global__ __launch_bounds__(kThreads) void route_backward_kernel(RouteBackward a) {
  constexpr int kRows = kThreads / LPT;
  __shared__ float dense[kRows][LPT * V];
  const int slot = threadIdx.x / LPT, sub = threadIdx.x % LPT;
  float *d = dense[slot];
#pragma unroll
  for (int v = 0; v < V; ++v) d[sub * V + v] = 0.0f;
  wave_sync();
  for (int64_t t0 = (int64_t)blockIdx.x * kRows; t0 < a.T; t0 += (int64_t)gridDim.x * kRows) {
    const int64_t t = t0 + slot;
    const bool live = t < a.T;
    const T *row = static_cast<const T *>(a.logits) + (live ? t : t0) * a.ld;
    const bool mine = live && sub < a.r.k;
    const int id = mine ? a.ids[t * a.r.k + sub] : -1;
    const float xj = (unsigned)id < (unsigned)a.r.E ? clean_logit(to_float(row[id])) : -INFINITY;
    const bool in = xj > -INFINITY;   // a masked choice's weight is a constant zero
    const float g = in ? a.r.scale * a.grad[t * a.r.k + sub] : 0.0f;
    float p[V];
    load_logits<T, V>(row, sub * V, a.r.E, p);
    float m = p[0];
#pragma unroll
    for (int v = 1; v < V; ++v) m = fmaxf(m, p[v]);
    m = row_maxf<LPT>(m);
    const float from = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int v = 0; v < V; ++v) p[v] = exp_term(p[v] - from);
    const float inv = over(1.0f, row_sum<LPT>(lane_sum(p)));
    const float back = row_sum<LPT>(in ? g * (exp_term(xj - from) * inv) : 0.0f);
    if (in) d[id] = g;
    wave_sync();
    T out[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      out[v] = from_float<T>(p[v] > 0.0f ? p[v] * inv * (d[sub * V + v] - back) : 0.0f);
    }
    wave_sync();
    if (in) d[id] = 0.0f;
    wave_sync();
    if (live) {
      T *to = static_cast<T *>(a.out) + t * a.ldg;
      if (sub * V + V <= a.r.E) {
        __builtin_memcpy(to + sub * V, out, sizeof(out));
      } else {
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (sub * V + v < a.r.E) to[sub * V + v] = out[v];
      }
    }
  }
}

// Launches K's kernel for these sizes: LPT lanes a row, V elements each.
template <class T, template <class, int, int> class K, class A>
int launch_rows(int E, int k, bool wide, const A &a, int T_rows, hipStream_t st) {
  if (!wide && k <= 16) {
    if (E <= 16) return K<T, 16, 1>::go(a, T_rows, st);
    if (E <= 32) return K<T, 16, 2>::go(a, T_rows, st);
    if (E <= 64) return K<T, 16, 4>::go(a, T_rows, st);
    if (E <= 128) return K<T, 16, 8>::go(a, T_rows, st);
    if (E <= 256) return K<T, 16, 16>::go(a, T_rows, st);
  }
  if (E <= 64) return K<T, 64, 1>::go(a, T_rows, st);
  if (E <= 128) return K<T, 64, 2>::go(a, T_rows, st);
  if (E <= 256) return K<T, 64, 4>::go(a, T_rows, st);
  if (E <= 512) return K<T, 64, 8>::go(a, T_rows, st);
  return K<T, 64, 16>::go(a, T_rows, st);
}

template <int LPT>
dim3 rows_grid(int T) {
  const int64_t blocks = ((int64_t)T + kThreads / LPT - 1) / (kThreads / LPT);
  return dim3((unsigned)(blocks < 4096 ? blocks : 4096));
}
template <class T, int LPT, int V>
struct Forward {
  static int go(const Route &a, int rows, hipStream_t st) {
    (void)hipGetLastError();
    hipLaunchKernelGGL((route_kernel<T, LPT, V>), rows_grid<LPT>(rows), dim3(kThreads), 0, st, a);
    return hipGetLastError() == hipSuccess ? TOPOEP_OK : TOPOEP_EHIP;
  }
};
template <class T, int LPT, int V>
struct Backward {
  static int go(const RouteBackward &a, int rows, hipStream_t st) {
    (void)hipGetLastError();
    hipLaunchKernelGGL((route_backward_kernel<T, LPT, V>), rows_grid<LPT>(rows), dim3(kThreads), 0, st, a);
    return hipGetLastError() == hipSuccess ? TOPOEP_OK : TOPOEP_EHIP;
  }
};

// Every row has lanes of its own, and a grid counts its lanes in 32 bits: more
// rows than that are several launches.
template <class T, int LPT, int V, int K, int GL>
int enqueue_list(const Route &a, hipStream_t st) {
  constexpr int kMostRows = (1 << 30) / LPT;
  (void)hipGetLastError();
  for (int64_t t0 = 0; t0 < a.T; t0 += kMostRows) {
    Route part = a;
    part.logits = static_cast<const T *>(a.logits) + t0 * a.ld;
    part.ids = a.ids + t0 * a.r.k;
    part.weights = a.weights + t0 * a.r.k;
    part.T = a.T - t0 < kMostRows ? (int)(a.T - t0) : kMostRows;
    const dim3 grid((unsigned)(((int64_t)part.T * LPT + kThreads - 1) / kThreads)), block(kThreads);
    if (a.bias) hipLaunchKernelGGL((route_list_kernel<T, LPT, V, K, GL, true>), grid, block, 0, st, part);
    else hipLaunchKernelGGL((route_list_kernel<T, LPT, V, K, GL, false>), grid, block, 0, st, part);
    if (hipGetLastError() != hipSuccess) return TOPOEP_EHIP;
  }
  return TOPOEP_OK;
}
template <class T, int LPT>
int enqueue_groups(const Route &a, int per_lane, hipStream_t st) {
  if (per_lane == 4) return enqueue_list<T, LPT, 32, 8, 4>(a, st);
  if (per_lane == 2) return enqueue_list<T, LPT, 32, 8, 2>(a, st);
  return enqueue_list<T, LPT, 32, 8, 1>(a, st);
}
template <class T, int K, int GL>
int enqueue_lists(const Route &a, hipStream_t st) {
  if (a.r.E <= 16) return enqueue_list<T, 4, 4, K, GL>(a, st);
  if (a.r.E <= 32) return enqueue_list<T, 4, 8, K, GL>(a, st);
  if (a.r.E <= 64) return enqueue_list<T, 4, 16, K, GL>(a, st);
  if (a.r.E <= 128) return enqueue_list<T, 4, 32, K, GL>(a, st);
  if (a.r.E <= 256) return enqueue_list<T, 8, 32, K, GL>(a, st);
  if (a.r.E <= 512) return enqueue_list<T, 16, 32, K, GL>(a, st);
  return enqueue_list<T, 16, 64, K, GL>(a, st);
}

// Groups a lane of 32 experts holds whole (1, 2, 4; 1 also where a group is 1, 2, 4
// or 8 lanes); 0 where groups and lanes do not fit.
int groups_of_lane(const RouterArgs &r) {
  const int m = r.per_group;
  if (m == 8 || m == 16) return 32 / m;
  return m == 32 || m == 64 || m == 128 || m == 256 ? 1 : 0;
}

template <class T>
int enqueue_route(const Route &a, hipStream_t st) {
  const RouterArgs &r = a.r;
  // Few tokens are a chain of dependent steps, shorter with a wave a token (one
  // token, 128 experts: 3.0 us a launch, lists 3.8; 512 tokens 3.2 and 4.2; 4096 tokens
  // 4.3 both); up to 64 experts without groups, or beyond 256, the lists' is no longer.
  if (a.T <= 1024 && r.E <= 256 && (r.groups > 1 || r.E > 64)) return launch_rows<T, Forward>(r.E, r.k, true, a, a.T, st);
  if (r.k <= 8 && r.groups == 1) return r.k <= 4 ? enqueue_lists<T, 4, 0>(a, st) : enqueue_lists<T, 8, 0>(a, st);
  const int per_lane = groups_of_lane(r);
  if (r.k <= 8 && r.top_groups <= 8 && r.E > 64 && r.E <= 512 && per_lane > 0) {
    if (r.E <= 128) return enqueue_groups<T, 4>(a, per_lane, st);
    if (r.E <= 256) return enqueue_groups<T, 8>(a, per_lane, st);
    return enqueue_groups<T, 16>(a, per_lane, st);
  }
  if (r.k <= 8) return enqueue_lists<T, 8, -1>(a, st);
  return launch_rows<T, Forward>(r.E, r.k, r.groups > 1 || a.T < 8192, a, a.T, st);
}

template <class T, int KP>
int enqueue_chosen(const RouteBackward &a, hipStream_t st) {
  const int rows = imin(64 / KP, kImageBytes / (a.r.E * (int)sizeof(T)));
  const int64_t blocks = ((int64_t)a.T + rows * (kThreads / 64) - 1) / (rows * (kThreads / 64));
  (void)hipGetLastError();
  hipLaunchKernelGGL((route_backward_chosen_kernel<T, KP>), dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(kThreads),
                     0, st, a, rows);
  return hipGetLastError() == hipSuccess ? TOPOEP_OK : TOPOEP_EHIP;
}
template <class T>
int enqueue_backward(const RouteBackward &a, hipStream_t st) {
  if (!a.r.sigmoid && !a.r.renorm) return launch_rows<T, Backward>(a.r.E, a.r.k, a.T < 8192, a, a.T, st);
  return a.r.k <= 8 ? enqueue_chosen<T, 8>(a, st) : enqueue_chosen<T, 64>(a, st);
}

// Bytes from the first row to the end of the last fit a pointer's range.
bool rows_fit(int T, int64_t ld, int E) { return ld >= E && (T < 2 || ld <= (INT64_MAX / 8 - E) / (T - 1)); }

}  // namespace

extern "C" {

int topoep_route(const topoep_router *r, const void *logits, int64_t ld, int32_t T, const float *bias, int32_t *ids,
                 float *weights, void *stream) {
  const int rc = check_router(r);
  if (rc != TOPOEP_OK) return rc;
  if (T < 0 || (int64_t)T * r->topk > INT32_MAX || !rows_fit(T, ld, r->num_experts)) return TOPOEP_EINVAL;
  if (T == 0) return TOPOEP_OK;
  if (!logits || !ids || !weights) return TOPOEP_EINVAL;
  Route a{router_args(r), logits, ld, T, bias, ids, weights};
  hipStream_t st = static_cast<hipStream_t>(stream);
  switch (r->dtype) {
    case TOPOEP_F32: return enqueue_route<float>(a, st);
    case TOPOEP_BF16: return enqueue_route<Bf16>(a, st);
    default: return enqueue_route<F16>(a, st);
  }
}

int topoep_route_backward(const topoep_router *r, const void *logits, int64_t ld, int32_t T, const int32_t *ids,
                          const float *grad_weights, void *grad_logits, int64_t ldg, void *stream) {
  const int rc = check_router(r);
  if (rc != TOPOEP_OK) return rc;
  if (T < 0 || (int64_t)T * r->topk > INT32_MAX || !rows_fit(T, ld, r->num_experts) ||
      !rows_fit(T, ldg, r->num_experts))
    return TOPOEP_EINVAL;
  if (T == 0) return TOPOEP_OK;
  if (!logits || !ids || !grad_weights || !grad_logits) return TOPOEP_EINVAL;
  RouteBackward a{router_args(r), logits, ld, T, ids, grad_weights, grad_logits, ldg};
  hipStream_t st = static_cast<hipStream_t>(stream);
  switch (r->dtype) {
    case TOPOEP_F32: return enqueue_backward<float>(a, st);
    case TOPOEP_BF16: return enqueue_backward<Bf16>(a, st);
    default: return enqueue_backward<F16>(a, st);
  }
}

}  // extern "C"
