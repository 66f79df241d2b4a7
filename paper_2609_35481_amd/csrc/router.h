// One token's routing, held by a group of lanes: shared by the router's
// kernels and the layer for a few tokens.
//
// LPT lanes hold a row, V consecutive experts each, so that among equal keys
// the lowest lane, and in it the lowest element, is the lowest expert id.
// Keys are compared as unsigned words in the order of the floats; 0 lies below
// every float's word (-inf's included) and marks what cannot be chosen: ids
// beyond E, experts of closed groups, experts already chosen.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "topoep_moe.h"
#include "wave.h"

namespace topoep_dev {

struct RouterArgs {
  int E, k;
  int groups, per_group, top_groups;
  int sigmoid, renorm;
  float scale;
};

__device__ inline float bf16_float(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
// Round to nearest even; NaN stays NaN.
__device__ inline uint16_t float_bf16(float f) {
  const uint32_t u = __float_as_uint(f);
  if (f != f) return (uint16_t)((u >> 16) | 0x40u);
  return (uint16_t)((u + 0x7FFFu + ((u >> 16) & 1u)) >> 16);
}

struct Bf16 { uint16_t v; };
struct F16 { _Float16 v; };
__device__ inline float to_float(float a) { return a; }
__device__ inline float to_float(Bf16 a) { return bf16_float(a.v); }
__device__ inline float to_float(F16 a) { return (float)a.v; }
template <class T> __device__ inline T from_float(float f);
template <> __device__ inline float from_float<float>(float f) { return f; }
template <> __device__ inline Bf16 from_float<Bf16>(float f) { return Bf16{float_bf16(f)}; }
template <> __device__ inline F16 from_float<F16>(float f) { return F16{(_Float16)f}; }

// A logit as the router takes it: NaN and -inf masked (-inf), +inf the
// largest finite number.  A median with a NaN among its operands is the least
// of the others; -inf goes by a register, or the compiler takes the median for
// the minimum of the other two, which gives a NaN the largest number.
__device__ inline float clean_logit(float x) {
  float low = -INFINITY;
  asm("" : "+v"(low));
  return __builtin_amdgcn_fmed3f(x, low, 3.402823466e38f);
}

// The float's place in ascending order.  k + 0 makes -0 and +0 one key.
__device__ inline uint32_t key_word(float k) {
  k += 0.0f;
  k = k != k ? -INFINITY : k;
  const int i = (int)__float_as_uint(k);
  return (uint32_t)i ^ ((uint32_t)(i >> 31) | 0x80000000u);
}

// Over a row's LPT lanes, the same value in each (every lane active).
template <int LPT>
__device__ inline uint32_t row_max(uint32_t v) {
  uint32_t o;
  o = dpp_mov<0x128>(v); v = o > v ? o : v;
  o = dpp_mov<0x124>(v); v = o > v ? o : v;
  o = dpp_mov<0x122>(v); v = o > v ? o : v;
  o = dpp_mov<0x121>(v); v = o > v ? o : v;
  if (LPT == 64) {
    const uint32_t a = (uint32_t)__builtin_amdgcn_readlane((int)v, 0);
    const uint32_t b = (uint32_t)__builtin_amdgcn_readlane((int)v, 16);
    const uint32_t c = (uint32_t)__builtin_amdgcn_readlane((int)v, 32);
    const uint32_t d = (uint32_t)__builtin_amdgcn_readlane((int)v, 48);
    const uint32_t e = a > b ? a : b, f = c > d ? c : d;
    v = e > f ? e : f;
  }
  return v;
}
template <int C>
__device__ inline float dpp_movf(float v) { return __uint_as_float(dpp_mov<C>(__float_as_uint(v))); }
// Sums go over a row's places as one binary tree of neighbours, first inside a
// lane, then over the lanes, whatever their number: a row's sum has the same
// bits in every form (places that hold nothing add zero).
template <int LPT>
__device__ inline float row_sum(float v) {
  if (LPT > 1) v += dpp_movf<0xB1>(v);
  if (LPT > 2) v += dpp_movf<0x4E>(v);
  if (LPT > 4) v += dpp_movf<0x141>(v);
  if (LPT > 8) v += dpp_movf<0x140>(v);
  if (LPT == 64) {
    const int u = (int)__float_as_uint(v);
    v = (__uint_as_float((uint32_t)__builtin_amdgcn_readlane(u, 0)) +
         __uint_as_float((uint32_t)__builtin_amdgcn_readlane(u, 16))) +
        (__uint_as_float((uint32_t)__builtin_amdgcn_readlane(u, 32)) +
         __uint_as_float((uint32_t)__builtin_amdgcn_readlane(u, 48)));
  }
  return v;
}
template <int V>
__device__ inline float lane_sum(const float (&v)[V]) {
  float s[V];
#pragma unroll
  for (int i = 0; i < V; ++i) s[i] = v[i];
#pragma unroll
  for (int d = 1; d < V; d *= 2)
#pragma unroll
    for (int i = 0; i < V; i += 2 * d) s[i] += s[i + d];
  return s[0];
}
template <int LPT>
__device__ inline float row_maxf(float v) {
  if (LPT > 1) v = fmaxf(v, dpp_movf<0xB1>(v));
  if (LPT > 2) v = fmaxf(v, dpp_movf<0x4E>(v));
  if (LPT > 4) v = fmaxf(v, dpp_movf<0x141>(v));
  if (LPT > 8) v = fmaxf(v, dpp_movf<0x140>(v));
  if (LPT == 64) {
    const int u = (int)__float_as_uint(v);
    v = fmaxf(fmaxf(__uint_as_float((uint32_t)__builtin_amdgcn_readlane(u, 0)),
                    __uint_as_float((uint32_t)__builtin_amdgcn_readlane(u, 16))),
              fmaxf(__uint_as_float((uint32_t)__builtin_amdgcn_readlane(u, 32)),
                    __uint_as_float((uint32_t)__builtin_amdgcn_readlane(u, 48))));
  }
  return v;
}

// V elements of a row from column `base`, cleaned; -inf beyond E.
template <class T, int V>
__device__ inline void load_logits(const T *row, int base, int E, float (&x)[V]) {
  if (base + V <= E) {
    T raw[V];
    __builtin_memcpy(raw, row + base, sizeof(raw));
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = clean_logit(to_float(raw[v]));
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = base + v < E ? clean_logit(to_float(row[base + v])) : -INFINITY;
  }
}

// LDS words a row's lanes need: a chosen (id, logit) pair per k, and the
// groups' largest keys.
constexpr int kRouteScratch = 2 * TOPOEP_ROUTER_MAX_TOPK + 64;

__device__ inline float sigmoid(float x) { return 1.0f / (1.0f + __expf(-x)); }

// exp(x - from), x <= from, to 1.5 x 2^-23 of it.  In 32 bits the difference and its
// product with log2 e are off by |x - from| 2^-24 each, which the exponential makes
// relative; both are formed in 64, and what 32 bits of them leave comes in as a factor.
__device__ inline float exp_from(float x, float from) {
  constexpr double kLog2e = 0x1.71547652b82fep+0;
  constexpr float kLn2 = 0x1.62e430p-1f;
  const double t = fmax(((double)x - (double)from) * kLog2e, -200.0);   // 0 from -150 on
  const float near = (float)t, rest = (float)(t - (double)near);
  const float e = __builtin_amdgcn_exp2f(near);
  return fmaf(e, rest * kLn2, e);
}
// A term of a sum of exp(d) next to one of 1: roundings of d and of its product move it
// by |d| exp(d) 2^-23 < 0.8 x 2^-24 of the sum.
__device__ inline float exp_term(float d) { return __expf(d); }

// A chosen logit's sigmoid score times exp(-top), where top (0, or the largest
// chosen logit below it, when only the scores' ratios count) keeps it from
// vanishing: exp(min(x, 0) - top) / (1 + exp(-|x|)).
__device__ inline float sigmoid_score(float x, float top) {
  const float e = exp_from(-fabsf(x), 0.0f), y = 1.0f + e;
  float r = __builtin_amdgcn_rcpf(y);
  r = fmaf(fmaf(-y, r, 1.0f), r, r);   // 1 <= y <= 2: a step takes the reciprocal's error out
  return (top < 0.0f ? exp_from(fminf(x, 0.0f), top) : x < 0.0f ? e : 1.0f) * r;
}
// `top` for renormalised scores with largest chosen logit m.  Scores below
// e^-709, where one in 64 bits ends, are zero.
__device__ inline float sigmoid_top(float m) { return m >= -709.0f ? fminf(m, 0.0f) : 0.0f; }

// The factor of a row's scores: the scale, over their sum where they have one.
__device__ inline float over(float scale, float sum) { return sum > 0.0f ? scale / sum : 0.0f; }

// Chooses a row's k experts and their weights.  x: the cleaned logits of
// experts sub * V .. + V - 1 (sub = this lane's place in the row), b: their
// biases; `scratch`: kRouteScratch words of LDS of the row's own.  Rows that
// are not live compute on, and write nothing.
template <int LPT, int V>
__device__ inline void route_row(const RouterArgs &r, const float (&x)[V], const float (&b)[V], int sub,
                                 uint32_t *scratch, bool live, int32_t *ids, float *weights) {
  uint32_t key[V];
#pragma unroll
  for (int v = 0; v < V; ++v) key[v] = sub * V + v < r.E ? key_word(x[v] + b[v]) : 0u;
  if (LPT == 64 && r.groups > 1) {
    // the groups' largest keys meet in LDS; lane g ranks group g
    uint32_t *best = scratch + 2 * TOPOEP_ROUTER_MAX_TOPK;
    if (sub < r.groups) best[sub] = 0;
    wave_sync();
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (sub * V + v < r.E) atomicMax(&best[(sub * V + v) / r.per_group], key[v]);
    wave_sync();
    const uint32_t mine = sub < r.groups ? best[sub] : 0u;
    int above = 0;
    for (int g = 0; g < r.groups; ++g) {
      const uint32_t o = (uint32_t)__builtin_amdgcn_readlane((int)mine, g);
      above += o > mine || (o == mine && g < sub) ? 1 : 0;
    }
    const uint64_t open = __ballot(sub < r.groups && above < r.top_groups);
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (sub * V + v < r.E && !((open >> ((sub * V + v) / r.per_group)) & 1)) key[v] = 0;
  }
  for (int j = 0; j < r.k; ++j) {
    uint32_t most = key[0];
#pragma unroll
    for (int v = 1; v < V; ++v) most = key[v] > most ? key[v] : most;
    const uint32_t top = row_max<LPT>(most);
    const uint64_t same = __ballot(most == top);
    const uint64_t row = LPT == 64 ? same : (same >> (lane_id() & ~(LPT - 1))) & ((1ull << (LPT & 63)) - 1);
    if (sub == __ffsll((unsigned long long)row) - 1) {
      int at = 0;
      float xv = x[0];
#pragma unroll
      for (int v = V - 1; v >= 0; --v) {
        at = key[v] == top ? v : at;
        xv = key[v] == top ? x[v] : xv;
      }
#pragma unroll
      for (int v = 0; v < V; ++v) key[v] = at == v ? 0u : key[v];
      scratch[2 * j] = (uint32_t)(sub * V + at);
      scratch[2 * j + 1] = __float_as_uint(xv);
    }
  }
  wave_sync();
  const bool mine = sub < r.k;
  const int id = mine ? (int)scratch[2 * sub] : 0;
  const float xj = mine ? __uint_as_float(scratch[2 * sub + 1]) : -INFINITY;
  wave_sync();
  float s, f = r.scale;
  if (r.sigmoid) {
    const float top = r.renorm ? sigmoid_top(row_maxf<LPT>(xj)) : 0.0f;
    s = mine ? sigmoid_score(xj, top) : 0.0f;
    if (r.renorm) f = over(r.scale, row_sum<LPT>(s));
  } else if (r.renorm) {
    const float m = row_maxf<LPT>(xj);
    s = exp_from(xj, m == -INFINITY ? 0.0f : m);
    f = over(r.scale, row_sum<LPT>(s));
  } else {
    float m = x[0];
#pragma unroll
    for (int v = 1; v < V; ++v) m = fmaxf(m, x[v]);
    m = row_maxf<LPT>(m);
    const float from = m == -INFINITY ? 0.0f : m;
    float e[V];
#pragma unroll
    for (int v = 0; v < V; ++v) e[v] = exp_term(x[v] - from);
    f = over(r.scale, row_sum<LPT>(lane_sum(e)));
    s = exp_from(xj, from);
  }
  if (live && mine) {
    ids[sub] = id;
    weights[sub] = s * f;
  }
}

// Host: the router's sizes.
inline int check_router(const topoep_router *r) {
  if (!r || r->num_experts < 1 || r->topk < 1 || r->topk > r->num_experts) return TOPOEP_EINVAL;
  if (r->groups < 1 || r->num_experts % r->groups != 0 || r->top_groups < 1 || r->top_groups > r->groups)
    return TOPOEP_EINVAL;
  if ((int64_t)r->top_groups * (r->num_experts / r->groups) < r->topk) return TOPOEP_EINVAL;
  if (r->scoring != TOPOEP_SOFTMAX && r->scoring != TOPOEP_SIGMOID) return TOPOEP_EINVAL;
  if (r->dtype < TOPOEP_F32 || r->dtype > TOPOEP_F16) return TOPOEP_EINVAL;
  if (!(r->scale - r->scale == 0.0f)) return TOPOEP_EINVAL;
  if (r->num_experts > TOPOEP_ROUTER_MAX_EXPERTS || r->topk > TOPOEP_ROUTER_MAX_TOPK || r->groups > 64)
    return TOPOEP_ELIMIT;
  return TOPOEP_OK;
}

inline RouterArgs router_args(const topoep_router *r) {
  RouterArgs a;
  a.E = r->num_experts;
  a.k = r->topk;
  a.groups = r->groups;
  a.per_group = r->num_experts / r->groups;
  a.top_groups = r->top_groups;
  a.sigmoid = r->scoring == TOPOEP_SIGMOID;
  a.renorm = r->renorm != 0;
  a.scale = r->scale;
  return a;
}

}  // namespace topoep_dev
