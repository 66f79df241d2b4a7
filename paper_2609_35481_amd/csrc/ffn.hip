// The gated feed-forward block and its gradients on gfx950, dense or for the rows of
// every expert of a routed layer.
//
//   up       h = w silu(g) u, (g, u) = up x: a tile's P holds gate and up rows of the same
//            units side by side, so that both of a unit end in one lane, and the
//            activation is the product's epilogue
//   down     y = down h, to out where dense, else by row in 32 bits
//   combine  out_t = the sum of a token's rows in the order of its choices
//
//   hidden   dh = down^T dout, whose epilogue makes da (and each row's part of
//            the weights' gradient)
//   input    dx = up^T da, by row, then combine
//   weights  dup = da^T x and ddown = dout^T h, an expert's rows being the inner axis
//
// A routed layer's tokens are never copied into the order of their experts: an
// operand's rows are read where they are, through the pairs (a row's address is a
// lane's own anyway).
//
// Which tiles there are depends on the experts' rows, which the host does not know:
// every workgroup counts them from the offsets and takes tiles by its number.
#include "fastdiv.h"
#include "few.h"
#include "spans.h"
#include "tile.h"
#include "topoep_ffn.h"

namespace {

using namespace topoep_dev;

struct Ffn {
  int T, H, I, L, rows;       // rows: at most
  int64_t expected;           // and about
  const void *x;
  int64_t ldx;
  const int32_t *offsets, *pairs, *places;   // NULL: dense
  const float *weights;
  int k;
  FastDiv per_token;
  const void *up, *down;
  void *out;
  float *gu;                  // [rows, 2, I]
  void *h;                    // [rows, I]
  float *y;                   // [parts, rows, H]
  const void *dout;           // [T, H]
  void *da;                   // [rows, 2I]
  float *part;                // [tiles of I, rows]
  void *dx;
  float *dw;
  void *dup, *ddown;
  float *sums;                // [parts, L, .., ..]: of a weights' gradient
};

__device__ inline int token_of_pair(const Ffn &a, int pair) {
  return a.k == 1 ? pair : (int)(__umulhi((uint32_t)pair, a.per_token.m) >> (a.per_token.sh - 32));   // (fdiv's upper half)
}
__device__ inline int token_of(const Ffn &a, int row) { return a.pairs ? token_of_pair(a, a.pairs[row]) : row; }
__device__ inline float weight_of(const Ffn &a, int row) { return a.pairs ? a.weights[a.pairs[row]] : 1.0f; }

// ---------------------------------------------------------------- forward

// BP rows of P are BP / 2 units: a wave's first half gate rows, its second half up rows.
template <class S, bool Save>
__global__ __launch_bounds__(S::kThreads, 2) void up_kernel(Ffn a) {
  typedef typename S::T T;
  TOPOEP_STAGES(S);
  constexpr int kUnits = S::BP / 2, kWaveUnits = S::TP * 8, kHalf = S::TP / 2;
  const int np = (a.I + kUnits - 1) / kUnits;
  Span s;
  const int nq = spans<S::BQ>(a.offsets, a.rows, a.L, -1, s);
  for (int t = blockIdx.x; t < nq * np; t += gridDim.x) {
    const Me me;
    const int tp = find_tile<S::BQ>(a.offsets, a.rows, a.L, t, np, nq * np, s);
    const int unit0 = tp * kUnits;
    ByRows<T, S::BP, S::kWaves> p;
    ByRows<T, S::BQ, S::kWaves> q;
    const char *w = static_cast<const char *>(a.up) + (int64_t)s.group * 4 * a.I * a.H;
    p.start(me, [&](int r) {
      const int in = r % (S::TP * 16), half = in / (kHalf * 16), unit = unit0 + r / (S::TP * 16) * kWaveUnits + in % (kHalf * 16);
      return w + (int64_t)(half * a.I + imin(unit, a.I - 1)) * a.H * 2;
    });
    q.start(me, [&](int r) {
      return static_cast<const char *>(a.x) + token_of(a, imin(s.first + r, s.end - 1)) * a.ldx * 2;
    });
    typename S::Sum d[S::TP][S::TQ] = {};
    __syncthreads();
    multiply<S>(p, q, me, a.H, start_of<S>(a.H, s.group), lds, d);
    float weights[S::TQ];   // (pairs, then weights: two readings deep, of all columns at once)
#pragma unroll
    for (int j = 0; j < S::TQ; ++j)
      weights[j] = weight_of(a, imin(s.first + (me.wave / S::NP * S::TQ + j) * 16 + (me.lane & 15), s.end - 1));
#pragma unroll
    for (int j = 0; j < S::TQ; ++j) {
      const int m = s.first + (me.wave / S::NP * S::TQ + j) * 16 + (me.lane & 15);
      if (m >= s.end) continue;
      const float weight = weights[j];
      const int first = unit0 + me.wave % S::NP * kWaveUnits;
      store_rows<T>(me, kHalf, static_cast<T *>(a.h) + (int64_t)m * a.I, first, a.I, [&](int i) {
        const v4f g = d[i][j], u = d[i + kHalf][j];
        if (Save) {
          const int unit = first + i * 16 + (me.lane >> 4) * 4;
          float *to = a.gu + (int64_t)m * 2 * a.I + unit;
          if (unit < a.I) {
            *reinterpret_cast<v4f *>(to) = g;
            *reinterpret_cast<v4f *>(to + a.I) = u;
          }
        }
        v4f h;
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = weight * (g[e] * sigmoid(g[e]) * u[e]);
        return h;
      });
    }
  }
}

// y = down h (Back false), dx = up^T da (Back true): to `to`, of T where dense and whole, else 32 bits.
// `parts` workgroups share a tile's inner axis where there are few tiles, each with sums of its own in `to`.
template <class S, bool Back>
__global__ __launch_bounds__(S::kThreads, 2) void out_kernel(Ffn a, void *to, int parts) {
  typedef typename S::T T;
  TOPOEP_STAGES(S);
  const int np = (a.H + S::BP - 1) / S::BP;
  const int n = Back ? 2 * a.I : a.I, each = ((n + parts - 1) / parts + S::kStage - 1) / S::kStage * S::kStage;
  Span s;
  const int nq = spans<S::BQ>(a.offsets, a.rows, a.L, -1, s);
  for (int u = blockIdx.x; u < nq * np * parts; u += gridDim.x) {
    const Me me;
    const int part = u / (nq * np), k0 = imin(part * each, n);
    const int tp = find_tile<S::BQ>(a.offsets, a.rows, a.L, u - part * nq * np, np, nq * np, s);
    typename std::conditional<Back, Across<T, S::BP, S::kWaves>, ByRows<T, S::BP, S::kWaves>>::type p;
    ByRows<T, S::BQ, S::kWaves> q;
    const T *w = static_cast<const T *>(Back ? a.up : a.down) + (int64_t)s.group * n * a.H;
    if constexpr (Back) p.start(me, w + (int64_t)k0 * a.H, a.H, tp * S::BP, a.H);
    else p.start(me, [&](int r) { return reinterpret_cast<const char *>(w + (int64_t)imin(tp * S::BP + r, a.H - 1) * n + k0); });
    const T *rows = static_cast<const T *>(Back ? a.da : a.h) + k0;
    q.start(me, [&](int r) { return reinterpret_cast<const char *>(rows + (int64_t)imin(s.first + r, s.end - 1) * n); });
    typename S::Sum d[S::TP][S::TQ] = {};
    __syncthreads();
    multiply<S>(p, q, me, imin(each, n - k0), start_of<S>(imin(each, n - k0), s.group), lds, d);
    const bool whole = !a.pairs && parts == 1;
    const int64_t at = (int64_t)part * a.rows * a.H;
#pragma unroll
    for (int j = 0; j < S::TQ; ++j) {
      const int m = s.first + (me.wave / S::NP * S::TQ + j) * 16 + (me.lane & 15);
      if (m >= s.end) continue;
      const int first = tp * S::BP + me.wave % S::NP * S::TP * 16;
      if (whole) {
        store_rows<T>(me, S::TP, static_cast<T *>(to) + (int64_t)m * a.H, first, a.H, [&](int i) { return d[i][j]; });
        continue;
      }
#pragma unroll
      for (int i = 0; i < S::TP; ++i) {
        const int c = first + i * 16 + (me.lane >> 4) * 4;
        if (c < a.H) *reinterpret_cast<v4f *>(static_cast<float *>(to) + at + (int64_t)m * a.H + c) = d[i][j];
      }
    }
  }
}

// A few rows an expert: up and down for 16 rows of weights and up to 4 C of a group at a time.
template <class T, bool Save, int C, int KS>
__global__ __launch_bounds__(64 * few_waves(KS), few_per_simd(C)) void few_up_kernel(Ffn a) {
  __shared__ FewSums<float, C, KS> lds;
  const int np = (a.I + 7) / 8;
  Span s;
  const int nq = spans<4 * C>(a.offsets, a.rows, a.L, -1, s);
  for (int t = few_first<KS>(); t < nq * np; t += few_next<KS>()) {
    const int tp = t / nq, unit0 = tp * 8;
    spans<4 * C>(a.offsets, a.rows, a.L, t - tp * nq, s);
    const char *w = static_cast<const char *>(a.up) + (int64_t)s.group * 4 * a.I * a.H;
    few_product<T, C, KS>(
        [&](int r) { return w + (int64_t)((r >> 3) * a.I + imin(unit0 + (r & 7), a.I - 1)) * a.H * 2; },
        [&](int c) { return static_cast<const char *>(a.x) + token_of(a, s.first + c) * a.ldx * 2; },
        imin(s.end - s.first, 4 * C), a.H * 2, lds, 8, [&](int u, int c, float g, float up) {
          if (unit0 + u >= a.I) return;
          const int m = s.first + c;
          static_cast<T *>(a.h)[(int64_t)m * a.I + unit0 + u] = from_float<T>(weight_of(a, m) * (g * sigmoid(g) * up));
          if (Save) {
            float *to = a.gu + (int64_t)m * 2 * a.I + unit0 + u;
            to[0] = g;
            to[a.I] = up;
          }
        });
  }
}

template <class T, int C, int KS>
__global__ __launch_bounds__(64 * few_waves(KS), few_per_simd(C)) void few_down_kernel(Ffn a, void *to) {
  __shared__ FewSums<float, C, KS> lds;
  const int np = (a.H + kFewRows - 1) / kFewRows;
  Span s;
  const int nq = spans<4 * C>(a.offsets, a.rows, a.L, -1, s);
  for (int t = few_first<KS>(); t < nq * np; t += few_next<KS>()) {
    const int tp = t / nq, h0 = tp * kFewRows;
    spans<4 * C>(a.offsets, a.rows, a.L, t - tp * nq, s);
    const char *w = static_cast<const char *>(a.down) + (int64_t)s.group * 2 * a.I * a.H;
    few_product<T, C, KS>([&](int r) { return w + (int64_t)imin(h0 + r, a.H - 1) * a.I * 2; },
                          [&](int c) { return static_cast<const char *>(a.h) + (int64_t)(s.first + c) * a.I * 2; },
                          imin(s.end - s.first, 4 * C), a.I * 2, lds, 16, [&](int r, int c, float v, float) {
                            if (h0 + r >= a.H) return;
                            const int64_t at = (int64_t)(s.first + c) * a.H + h0 + r;
                            if (a.pairs) static_cast<float *>(to)[at] = v;
                            else static_cast<T *>(to)[at] = from_float<T>(v);
                          });
  }
}

// A row's parts, in order, as its pair's gradient; 0 without a row.
__device__ inline float weight_grad(const Ffn &a, int row, int parts) {
  float s = 0.0f;
  if ((unsigned)row < (unsigned)a.rows)
    for (int p = 0; p < parts; ++p) s += a.part[(int64_t)p * a.rows + row];
  return s;
}

// out_t = the sum of its rows of `from`, in the order of its choices (dense: its row), each the sum
// of its parts.  A workgroup has a token and 1024 columns of it, the first also the token's weights' gradients
// of `of_weights` parts (0: none; a launch of their own took 4 us).
template <class T>
__global__ __launch_bounds__(256) void combine_kernel(Ffn a, const float *from, void *to, int parts, int of_weights) {
  const int c = (blockIdx.y * 256 + threadIdx.x) * 4;
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    int place = -1;
    if (lane_id() < a.k) place = a.pairs ? a.places[t * a.k + lane_id()] : (int)t;
    if (of_weights && blockIdx.y == 0 && (int)threadIdx.x < a.k) a.dw[t * a.k + threadIdx.x] = weight_grad(a, place, of_weights);
    uint64_t here = __ballot((unsigned)place < (unsigned)a.rows);
    v4f s = {0.0f, 0.0f, 0.0f, 0.0f};
    for (; here != 0; here &= here - 1) {
      const int64_t m = readlane_i32(place, __ffsll((unsigned long long)here) - 1);
      if (c >= a.H) continue;
      v4f row = *reinterpret_cast<const v4f *>(from + m * a.H + c);
      for (int p = 1; p < parts; ++p) row += *reinterpret_cast<const v4f *>(from + ((int64_t)p * a.rows + m) * a.H + c);
      s += row;
    }
    if (c < a.H) store4<T>(to, t * a.H + c, s);
  }
}

// ---------------------------------------------------------------- backward

template <class S>
__global__ __launch_bounds__(S::kThreads, 2) void hidden_kernel(Ffn a) {
  typedef typename S::T T;
  TOPOEP_STAGES(S);
  const int np = (a.I + S::BP - 1) / S::BP;
  Span s;
  const int nq = spans<S::BQ>(a.offsets, a.rows, a.L, -1, s);
  for (int t = blockIdx.x; t < nq * np; t += gridDim.x) {
    const Me me;
    const int tp = find_tile<S::BQ>(a.offsets, a.rows, a.L, t, np, nq * np, s);
    Across<T, S::BP, S::kWaves> p;
    ByRows<T, S::BQ, S::kWaves> q;
    p.start(me, static_cast<const char *>(a.down) + (int64_t)s.group * 2 * a.I * a.H, a.I, tp * S::BP, a.I);
    q.start(me, [&](int r) {
      return static_cast<const char *>(a.dout) + (int64_t)token_of(a, imin(s.first + r, s.end - 1)) * a.H * 2;
    });
    typename S::Sum d[S::TP][S::TQ] = {};
    __syncthreads();
    multiply<S>(p, q, me, a.H, start_of<S>(a.H, s.group), lds, d);
    __syncthreads();   // the stages are read: sums go where they were
    __attribute__((address_space(3))) float *sums = (__attribute__((address_space(3))) float *)lds.p[0];   // [NP, BQ]
    // g and u of a pair of tiles, read two pairs ahead where 64 registers hold d (301 tokens, two experts each of 16,
    // H = 520, I = 248: 16.3 us, and 20.0 where each pair waited for its own). 128 registers of d leave none for
    // another pair (8192 rows, H = 4096, I = 14336: 1.04 ms; one pair ahead, 17 registers in scratch: 1.07).
    constexpr int kPairs = S::TP / 2, kAll = kPairs * S::TQ, kHeld = S::TP * S::TQ > 16 ? 1 : 3;
    const int first = tp * S::BP + me.wave % S::NP * S::TP * 16, quad = (me.lane >> 4) * 4;
    const int col0 = me.wave / S::NP * S::TQ * 16 + (me.lane & 15);
    float weight[S::TQ], sum = 0.0f;
#pragma unroll
    for (int j = 0; j < S::TQ; ++j) weight[j] = weight_of(a, imin(s.first + col0 + j * 16, s.end - 1));
    v4f g[kHeld][2], u[kHeld][2];
    const auto fetch = [&](int n) {
      const int64_t row = imin(s.first + col0 + n / kPairs * 16, s.end - 1);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const float *from = a.gu + row * 2 * a.I + imin(first + (n % kPairs * 2 + t) * 16 + quad, a.I - 4);
        g[n % kHeld][t] = *reinterpret_cast<const v4f *>(from);
        u[n % kHeld][t] = *reinterpret_cast<const v4f *>(from + a.I);
      }
    };
#pragma unroll
    for (int n = 0; n < kHeld - 1 && n < kAll; ++n) fetch(n);
#pragma unroll
    for (int n = 0; n < kAll; ++n) {
      const int j = n / kPairs, i = n % kPairs * 2, m = s.first + col0 + j * 16;
      if (n + kHeld - 1 < kAll) fetch(n + kHeld - 1);
      __builtin_amdgcn_sched_barrier(0);
      v4f dg[2], du[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const bool in = first + (i + t) * 16 + quad < a.I;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float gate = g[n % kHeld][t][e], up = u[n % kHeld][t][e];
          const float sg = sigmoid(gate), act = gate * sg, dh = d[i + t][j][e];
          sum += in ? dh * (act * up) : 0.0f;
          dg[t][e] = weight[j] * (dh * up * (sg + act * (1.0f - sg)));
          du[t][e] = weight[j] * (dh * act);
        }
      }
      const v4i og = pair_of<T>(dg[0], dg[1]), ou = pair_of<T>(du[0], du[1]);
      const int unit = first + i * 16 + pair_column(me);
      if (m < s.end && unit < a.I) {
        T *const to = static_cast<T *>(a.da) + (int64_t)m * 2 * a.I + unit;
        *reinterpret_cast<v4i *>(to) = og;
        *reinterpret_cast<v4i *>(to + a.I) = ou;
      }
      if (i == S::TP - 2) {
        if (a.dw) {
          sum += __shfl_xor(sum, 16);
          sum += __shfl_xor(sum, 32);
          if (me.lane < 16) sums[me.wave % S::NP * S::BQ + col0 + j * 16] = sum;
        }
        sum = 0.0f;
      }
    }
    if (a.dw) {
      __syncthreads();
      for (int c = threadIdx.x; c < S::BQ && s.first + c < s.end; c += S::kThreads) {
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < S::NP; ++w) sum += sums[w * S::BQ + c];
        a.part[(int64_t)tp * a.rows + s.first + c] = sum;
      }
    }
  }
}

// The weights' gradients where the tokens' are not wanted.
__global__ __launch_bounds__(256) void weights_kernel(Ffn a, int parts) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < (int64_t)a.T * a.k) a.dw[i] = weight_grad(a, a.places[i], parts);
}

// An operand across whose rows of the inner axis are tokens', through the pairs.
template <class T, int B, int W>
struct Tokens : AcrossPlaces<B, W> {
  typedef AcrossPlaces<B, W> At;
  const Ffn *a;
  const char *from;
  int64_t ld;                       // bytes
  int first, pair[At::kLoads];      // of the next stage's rows
  __device__ void start(const Ffn &of, Me me, const void *base, int64_t stride, int row, int c0, int n, int len) {
    const int c = c0 + At::column_of(me);
    a = &of, from = static_cast<const char *>(base) + (c < n ? c : 0) * 2, ld = stride * 2, first = row;
    if (len > 0) next(me, 0, len);
  }
  // The pairs as they are: a token formed here would have to wait for them, and with them for
  // every load before them (128 experts of H = 2048, I = 768 with 32768 rows, both gradients: 861 us, and 726 so).
  __device__ void next(Me me, int k, int n) {
#pragma unroll
    for (int i = 0; i < At::kLoads; ++i) {
      const int at = k + At::row_of(i, me);
      pair[i] = a->pairs[first + (at < n ? at : 0)];
    }
  }
  __device__ void load(Lds *to, Me me, int k, int after, int n) {
#pragma unroll
    for (int i = 0; i < At::kLoads; ++i) {
      const char *p = from + token_of_pair(*a, pair[i]) * ld;
      to_lds(At::row_of(i, me) < n - k ? p : reinterpret_cast<const char *>(&kZeros), to + At::load_of(i, me.wave) * kApart);
    }
    next(me, after, n);
  }
};

// dup[g][r][c] = sum over the group's rows of da[m][r] x[token][c] (Down false), ddown[g][r][c] of
// dout[token][r] h[m][c] (Down true).  `parts` workgroups share a group's rows where there are few
// tiles, each with sums of its own in a.sums.
//
// A group's tiles (and parts) go to `xcds` XCDs, groups in turn: an L2 that has few tiles of every group reads
// most of their operands (10 experts of H = 7168, I = 2048, both gradients: 550 us with eight XCDs each, 520 so).
template <class S, bool Down, bool Routed>
__global__ __launch_bounds__(S::kThreads, 2) void grad_kernel(Ffn a, int parts, int xcds) {
  typedef typename S::T T;
  TOPOEP_STAGES(S);
  const Me me;
  const int cols = Down ? a.I : a.H, rows = Down ? a.H : 2 * a.I;
  const int np = (cols + S::BP - 1) / S::BP, nq = (rows + S::BQ - 1) / S::BQ;
  const int all = np * nq * parts, each_xcd = (all + xcds - 1) / xcds, xcd = blockIdx.x & 7, slot = blockIdx.x >> 3;
  const int turn = slot / each_xcd, g = turn * (8 / xcds) + xcd / xcds, tile = xcd % xcds * each_xcd + slot - turn * each_xcd;
  if (g >= a.L || tile >= all) return;
  const int part = tile / (np * nq);
  int tq, tp, first, end;
  place_of(tile - part * np * nq, nq, np, tq, tp);
  rows_of(a.offsets, a.rows, g, first, end);
  const int each = ((end - first + parts - 1) / parts + S::kStage - 1) / S::kStage * S::kStage;
  first = imin(first + part * each, end);
  const int n = imin(each, end - first);
  typename S::Sum d[S::TP][S::TQ] = {};
  constexpr int B = Down ? S::BQ : S::BP;
  typename std::conditional<Routed, Tokens<T, B, S::kWaves>, Across<T, B, S::kWaves>>::type tokens;
  const void *const from = Down ? a.dout : a.x;
  const int64_t ld = Down ? a.H : a.ldx;
  const int c0 = Down ? tq * S::BQ : tp * S::BP;
  if constexpr (Routed) tokens.start(a, me, from, ld, first, c0, a.H, n);
  else tokens.start(me, static_cast<const T *>(from) + first * ld, ld, c0, a.H);
  if constexpr (Down) {
    Across<T, S::BP, S::kWaves> p;
    p.start(me, static_cast<const T *>(a.h) + (int64_t)first * a.I, a.I, tp * S::BP, a.I);
    multiply<S>(p, tokens, me, n, 0, lds, d);
  } else {
    Across<T, S::BQ, S::kWaves> q;
    q.start(me, static_cast<const T *>(a.da) + (int64_t)first * 2 * a.I, 2 * a.I, tq * S::BQ, 2 * a.I);
    multiply<S>(tokens, q, me, n, 0, lds, d);
  }
  void *const to = Down ? a.ddown : a.dup;
  const int64_t at = ((int64_t)part * a.L + g) * rows;
#pragma unroll
  for (int j = 0; j < S::TQ; ++j) {
    const int r = tq * S::BQ + (me.wave / S::NP * S::TQ + j) * 16 + (me.lane & 15);
    if (r >= rows) continue;
    const int left = tp * S::BP + me.wave % S::NP * S::TP * 16;
    if (parts == 1) {
      store_rows<T>(me, S::TP, static_cast<T *>(to) + (at + r) * cols, left, cols, [&](int i) { return d[i][j]; });
      continue;
    }
#pragma unroll
    for (int i = 0; i < S::TP; ++i) {
      const int c = left + i * 16 + (me.lane >> 4) * 4;
      if (c < cols) *reinterpret_cast<v4f *>(a.sums + (at + r) * cols + c) = d[i][j];
    }
  }
}

// n values, each the sum of its parts in order.
template <class T>
__global__ __launch_bounds__(256) void parts_kernel(const float *from, void *to, int64_t n, int parts) {
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n; i += (int64_t)gridDim.x * 1024) {
    v4f s = *reinterpret_cast<const v4f *>(from + i);
    for (int p = 1; p < parts; ++p) s += *reinterpret_cast<const v4f *>(from + p * n + i);
    store4<T>(to, i, s);
  }
}

// ---------------------------------------------------------------- host

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool launched() { return hipGetLastError() == hipSuccess; }

constexpr int kPartUnits = 128;   // units of a part of the weights' gradient, at least: the hidden kernel's BP

// Rows of the experts that are here, at most and about.
struct Counts { int64_t rows, expected; };
Counts counts_of(const topoep_ffn *f, int32_t T, const topoep_ffn_rows *r) {
  if (!r) return Counts{T, T};
  const int64_t rows = (int64_t)T * r->topk;
  return Counts{rows, ceil_of(rows * imin(f->experts, r->num_experts), r->num_experts)};
}

// Of the products by rows with H columns (their sums are at most 256 MiB), n of the inner axis.
int out_parts(const topoep_ffn *f, const Counts &c, const topoep_ffn_rows *r, int n) {
  const int64_t tiles = likely_spans(r != nullptr, c.expected, f->experts, 128) * ceil_of(f->hidden, 128);
  const int p = parts_of(tiles, n / 64, 8);
  return c.rows * f->hidden * p > (int64_t)1 << 26 ? 1 : p;
}
// Of a weights' gradient of `rows` by `cols`.
int grad_parts(const topoep_ffn *f, const Counts &c, int rows, int cols) {
  return parts_of(f->experts * ceil_of(rows, 128) * ceil_of(cols, 128), c.expected / f->experts / 64, 16);
}

struct Sizes {
  size_t gu, h, y, back, da, part, sums, saved, forward, backward;
};

Sizes sizes_of(const topoep_ffn *f, int32_t T, const topoep_ffn_rows *r) {
  Sizes s;
  const Counts c = counts_of(f, T, r);
  const size_t n = (size_t)c.rows, H = (size_t)f->hidden, I = (size_t)f->inter;
  const int down = out_parts(f, c, r, f->inter), up = out_parts(f, c, r, 2 * f->inter);
  const int pu = grad_parts(f, c, 2 * f->inter, f->hidden), pd = grad_parts(f, c, f->hidden, f->inter);
  s.gu = align256(n * 2 * I * sizeof(float));
  s.h = align256(n * I * 2);
  s.y = r || down > 1 ? align256(down * n * H * sizeof(float)) : 0;
  s.back = r || up > 1 ? align256(up * n * H * sizeof(float)) : 0;
  s.da = align256(n * 2 * I * 2);
  s.part = r ? align256((I + kPartUnits - 1) / kPartUnits * n * sizeof(float)) : 0;
  const size_t su = pu > 1 ? (size_t)pu * f->experts * 2 * I * H : 0, sd = pd > 1 ? (size_t)pd * f->experts * I * H : 0;
  s.sums = align256((su > sd ? su : sd) * sizeof(float));
  s.saved = s.gu + s.h;
  s.forward = s.h + s.y;   // (h where nothing is saved)
  s.backward = s.da + s.back + s.part + s.sums;
  return s;
}

int check(const topoep_ffn *f, int32_t T, const topoep_ffn_rows *rows) {
  if (!f || T < 0 || T > 1 << 30) return TOPOEP_EINVAL;   // (a tile behind the last row is counted in 32 bits)
  if (f->hidden < 8 || (f->hidden & 7) || f->inter < 8 || (f->inter & 7) || f->experts < 1) return TOPOEP_EINVAL;
  if (f->hidden > 1 << 17 || f->inter > 1 << 17 || (int64_t)f->hidden * f->inter > 1 << 30) return TOPOEP_EINVAL;
  if (f->dtype != TOPOEP_BF16 && f->dtype != TOPOEP_F16) return TOPOEP_EINVAL;
  if (!rows && f->experts != 1) return TOPOEP_EINVAL;
  if (rows && (rows->topk < 1 || rows->num_experts < 1 || (int64_t)T * rows->topk > 1 << 30)) return TOPOEP_EINVAL;
  if (f->experts > TOPOEP_FFN_MAX_EXPERTS || (rows && rows->topk > TOPOEP_ROUTER_MAX_TOPK)) return TOPOEP_ELIMIT;
  return TOPOEP_OK;
}

Ffn args_of(const topoep_ffn *f, const void *x, int64_t ldx, int32_t T, const topoep_ffn_rows *rows, const void *up,
            const void *down) {
  Ffn a = {};
  a.T = T, a.H = f->hidden, a.I = f->inter, a.L = f->experts;
  a.x = x, a.ldx = ldx, a.up = up, a.down = down;
  a.k = rows ? rows->topk : 1;
  a.rows = T * a.k;
  a.expected = counts_of(f, T, rows).expected;
  a.per_token = make_fastdiv((uint32_t)a.k);
  if (rows) a.offsets = rows->offsets, a.pairs = rows->pairs, a.places = rows->places, a.weights = rows->weights;
  return a;
}

template <class T, bool PA> using Large = Shape<T, 256, 256, 2, 4, PA, false, 2>;
template <class T, bool PA> using Small = Shape<T, 128, 128, 2, 2, PA, false, 4>;
template <class T> using LargeGrad = Shape<T, 256, 256, 2, 4, true, true, 1>;
template <class T> using SmallGrad = Shape<T, 128, 128, 2, 2, true, true, 4>;

// Whether a product by rows with `cols` columns of out takes large tiles (`per`: columns of a tile of 256).
// Of groups those of 1024 rows and more: smaller ones leave large tiles half empty (16 experts of H =
// 2048, I = 768 with 512 rows, a training step: 565 against 550 us).
bool large_rows(const Ffn &a, int cols, int per) {
  const bool groups = a.offsets != nullptr;
  if (groups && a.expected < 1024 * (int64_t)a.L) return false;
  return large_tiles(likely_spans(groups, a.expected, a.L, 256) * ceil_of(cols, per),
                     likely_spans(groups, a.expected, a.L, 128) * ceil_of(cols, per / 2));
}

template <class S, bool Save>
int enqueue_up(const Ffn &a, hipStream_t st) {
  const int64_t tiles = most_spans<S::BQ>(a.offsets, a.rows, a.L) * ((a.I + S::BP / 2 - 1) / (S::BP / 2));
  hipLaunchKernelGGL((up_kernel<S, Save>), dim3(grid_of<S>(tiles)), dim3(S::kThreads), 0, st, a);
  return launched() ? TOPOEP_OK : TOPOEP_EHIP;
}
template <class T>
int enqueue_up(const Ffn &a, hipStream_t st) {
  if (large_rows(a, a.I, 128))
    return a.gu ? enqueue_up<Large<T, false>, true>(a, st) : enqueue_up<Large<T, false>, false>(a, st);
  return a.gu ? enqueue_up<Small<T, false>, true>(a, st) : enqueue_up<Small<T, false>, false>(a, st);
}

template <class S, bool Back>
int enqueue_out_of(const Ffn &a, void *to, int parts, hipStream_t st) {
  const int64_t tiles = most_spans<S::BQ>(a.offsets, a.rows, a.L) * ((a.H + S::BP - 1) / S::BP) * parts;
  hipLaunchKernelGGL((out_kernel<S, Back>), dim3(grid_of<S>(tiles)), dim3(S::kThreads), 0, st, a, to, parts);
  return launched() ? TOPOEP_OK : TOPOEP_EHIP;
}
template <class T>
int enqueue_combine(const Ffn &a, void *to, int parts, int of_weights, hipStream_t st) {
  hipLaunchKernelGGL((combine_kernel<T>), dim3(imin(a.T, 1 << 20), (a.H + 1023) / 1024), dim3(256), 0, st, a, a.y, to, parts, of_weights);
  return launched() ? TOPOEP_OK : TOPOEP_EHIP;
}
template <class T, bool Back>
int enqueue_out(const Ffn &a, void *to, int parts, int of_weights, hipStream_t st) {
  void *const product = a.pairs || parts > 1 ? static_cast<void *>(a.y) : to;
  const int rc = parts == 1 && large_rows(a, a.H, 256) ? enqueue_out_of<Large<T, Back>, Back>(a, product, 1, st)
                                                       : enqueue_out_of<Small<T, Back>, Back>(a, product, parts, st);
  return rc != TOPOEP_OK || product == to ? rc : enqueue_combine<T>(a, to, parts, of_weights, st);
}

template <class S>
int enqueue_hidden_of(const Ffn &a, int *of_weights, hipStream_t st) {
  const int parts = (a.I + S::BP - 1) / S::BP;
  *of_weights = a.dw ? parts : 0;
  const int64_t tiles = most_spans<S::BQ>(a.offsets, a.rows, a.L) * parts;
  hipLaunchKernelGGL((hidden_kernel<S>), dim3(grid_of<S>(tiles)), dim3(S::kThreads), 0, st, a);
  if (!launched()) return TOPOEP_EHIP;
  if (!a.dw || a.dx) return TOPOEP_OK;   // (combine_kernel sums them)
  hipLaunchKernelGGL(weights_kernel, dim3((unsigned)((a.rows + (int64_t)255) / 256)), dim3(256), 0, st, a, parts);
  return launched() ? TOPOEP_OK : TOPOEP_EHIP;
}
template <class T>
int enqueue_hidden(const Ffn &a, int *of_weights, hipStream_t st) {
  static_assert(Small<T, true>::BP >= kPartUnits, "parts of the weights' gradient");
  return large_rows(a, a.I, 256) ? enqueue_hidden_of<Large<T, true>>(a, of_weights, st)
                                 : enqueue_hidden_of<Small<T, true>>(a, of_weights, st);
}

template <class S, bool Down>
int enqueue_grad_of(const Ffn &a, int64_t tiles, int parts, hipStream_t st) {
  // XCDs of a group: 32 tiles for each, which its CUs take at once; all where there are few groups
  const int64_t all = tiles / a.L * parts;
  int xcds = 1;
  while (xcds < 8 && (all >= 24 * xcds || a.L * 2 < 8 / xcds * 4)) xcds *= 2;
  const int64_t blocks = 8 * ceil_of(all, xcds) * ceil_of(a.L, 8 / xcds);
  if (a.pairs) hipLaunchKernelGGL((grad_kernel<S, Down, true>), dim3((unsigned)blocks), dim3(S::kThreads), 0, st, a, parts, xcds);
  else hipLaunchKernelGGL((grad_kernel<S, Down, false>), dim3((unsigned)blocks), dim3(S::kThreads), 0, st, a, parts, xcds);
  return launched() ? TOPOEP_OK : TOPOEP_EHIP;
}
template <class T, bool Down>
int enqueue_grad(const Ffn &a, int parts, hipStream_t st) {
  const int cols = Down ? a.I : a.H, rows = Down ? a.H : 2 * a.I;
  const auto tiles = [&](int64_t n) { return a.L * ((cols + n - 1) / n) * ((rows + n - 1) / n); };
  if (parts == 1 && large_tiles(tiles(256), tiles(128))) return enqueue_grad_of<LargeGrad<T>, Down>(a, tiles(256), 1, st);
  const int rc = enqueue_grad_of<SmallGrad<T>, Down>(a, tiles(128), parts, st);
  if (rc != TOPOEP_OK || parts == 1) return rc;
  const int64_t n = (int64_t)a.L * rows * cols, blocks = (n + 1023) / 1024;
  hipLaunchKernelGGL((parts_kernel<T>), dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, st, a.sums,
                     Down ? a.ddown : a.dup, n, parts);
  return launched() ? TOPOEP_OK : TOPOEP_EHIP;
}

// A few rows a group, 16 and fewer: the weights' bytes count, not the tiles.  Up to 64 also where a product
// of `n` rows of weights is small (rows times weights of 512 MiB: 32 rows, H = I = 2048, both products:
// 17.8 against 30.2 us; I = 5632: 41.4 and 38.7).  The mean decides: a group far above it reads its weights once for
// every 4 C rows that it has.
bool few_rows(const Ffn &a, int64_t n, int64_t k) {
  const int64_t groups = imin(a.L, (int)a.expected);
  if ((double)a.rows * n >= 0x1p34) return false;   // (its tiles are numbered in 32 bits)
  return a.expected <= 16 * groups || (a.expected <= 64 * groups && (double)a.expected * groups * n * k <= 0x1p28);
}

// Columns for a group's rows at once: groups differ, and twice the mean is what most have at most (128
// experts, four rows on average: 190 against 225 us with the mean).
int64_t few_each(const Ffn &a) {
  const int64_t groups = imin(a.L, (int)a.expected), mean = (a.expected + groups - 1) / groups;
  return groups > 1 ? 2 * mean : mean;
}

// Grid of the tiles of a few rows, np of the weights' each.  Of T k rows that could be here about T k L / E are, and a
// workgroup without a tile starts, counts the groups and ends all the same: tiles are those of twice
// the expected rows, or as many as fill the chip, and more rows than that take turns (512 tokens, eight of 256 experts each, one
// of which is here, H = I = 4096: 660 us with all that could be, 354 so; eight here, H = 7168, I = 2048: 242 and 236).
template <int C, int KS>
dim3 few_blocks(const Ffn &a, int64_t np) {
  constexpr int64_t kFill = KS == 1 ? 4096 : 1024;
  const int64_t rows = a.expected * 2 < a.rows ? a.expected * 2 : a.rows;
  const int64_t most = most_spans<4 * C>(a.offsets, a.rows, a.L) * np, likely = most_spans<4 * C>(a.offsets, (int)rows, a.L) * np;
  const int64_t tiles = likely > kFill ? likely : kFill;
  return few_grid<KS>(tiles < most ? tiles : most);
}

template <class T>
int enqueue_few_up(const Ffn &a, hipStream_t st) {
  const int64_t groups = imin(a.L, (int)a.expected), nu = (a.I + 7) / 8;
  few_shape(few_each(a), groups * nu, [&](auto c, auto ks) {
    constexpr int C = decltype(c)::value, KS = decltype(ks)::value;
    const dim3 grid = few_blocks<C, KS>(a, nu), block(64 * few_waves(KS));
    if (a.gu) hipLaunchKernelGGL((few_up_kernel<T, true, C, KS>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((few_up_kernel<T, false, C, KS>), grid, block, 0, st, a);
  });
  return launched() ? TOPOEP_OK : TOPOEP_EHIP;
}
template <class T>
int enqueue_few_down(const Ffn &a, hipStream_t st) {
  const int64_t groups = imin(a.L, (int)a.expected), nh = (a.H + kFewRows - 1) / kFewRows;
  few_shape(few_each(a), groups * nh, [&](auto c, auto ks) {
    constexpr int C = decltype(c)::value, KS = decltype(ks)::value;
    const dim3 grid = few_blocks<C, KS>(a, nh), block(64 * few_waves(KS));
    hipLaunchKernelGGL((few_down_kernel<T, C, KS>), grid, block, 0, st, a, a.pairs ? static_cast<void *>(a.y) : a.out);
  });
  if (!launched()) return TOPOEP_EHIP;
  return a.pairs ? enqueue_combine<T>(a, a.out, 1, 0, st) : TOPOEP_OK;
}

template <class T>
int forward(const Ffn &a, int parts, hipStream_t st) {
  const int rc = few_rows(a, 2 * a.I, a.H) ? enqueue_few_up<T>(a, st) : enqueue_up<T>(a, st);
  if (rc != TOPOEP_OK) return rc;
  return few_rows(a, a.H, a.I) ? enqueue_few_down<T>(a, st) : enqueue_out<T, false>(a, a.out, parts, 0, st);
}

template <class T>
int backward(const Ffn &a, int parts, int up_parts, int down_parts, hipStream_t st) {
  int rc = TOPOEP_OK, of_weights = 0;
  if (a.rows > 0 && (a.dx || a.dw || a.dup)) rc = enqueue_hidden<T>(a, &of_weights, st);
  if (rc == TOPOEP_OK && a.rows > 0 && a.dx) rc = enqueue_out<T, true>(a, a.dx, parts, of_weights, st);
  if (rc == TOPOEP_OK && a.dup) rc = enqueue_grad<T, false>(a, up_parts, st);
  if (rc == TOPOEP_OK && a.ddown) rc = enqueue_grad<T, true>(a, down_parts, st);
  return rc;
}

}  // namespace

extern "C" {

int topoep_ffn_bytes(const topoep_ffn *f, int32_t T, const topoep_ffn_rows *rows, size_t *forward, size_t *saved,
                     size_t *backward) {
  const int rc = check(f, T, rows);
  if (rc != TOPOEP_OK) return rc;
  const Sizes s = sizes_of(f, T, rows);
  if (forward) *forward = s.forward;
  if (saved) *saved = s.saved;
  if (backward) *backward = s.backward;
  return TOPOEP_OK;
}

int topoep_ffn_forward(const topoep_ffn *f, const void *x, int64_t ldx, int32_t T, const topoep_ffn_rows *rows,
                       const void *up, const void *down, void *out, void *saved, void *workspace,
                       size_t workspace_bytes, void *stream) {
  const int rc = check(f, T, rows);
  if (rc != TOPOEP_OK) return rc;
  if (T == 0) return TOPOEP_OK;
  if (!x || !up || !down || !out || !workspace) return TOPOEP_EINVAL;
  if (rows && (!rows->offsets || !rows->pairs || !rows->places || !rows->weights)) return TOPOEP_EINVAL;
  if (ldx < f->hidden || (ldx & 7) || ldx > (int64_t)1 << 40) return TOPOEP_EINVAL;
  if (!aligned16(x) || !aligned16(up) || !aligned16(down) || !aligned16(out) || !aligned16(saved)) return TOPOEP_EINVAL;
  const Sizes s = sizes_of(f, T, rows);
  if ((reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < s.forward) return TOPOEP_EWORKSPACE;
  Ffn a = args_of(f, x, ldx, T, rows, up, down);
  a.out = out;
  a.h = saved ? static_cast<char *>(saved) + s.gu : workspace;
  a.gu = static_cast<float *>(saved);
  a.y = reinterpret_cast<float *>(static_cast<char *>(workspace) + s.h);
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const int parts = out_parts(f, counts_of(f, T, rows), rows, f->inter);
  return f->dtype == TOPOEP_BF16 ? forward<Bf16>(a, parts, st) : forward<F16>(a, parts, st);
}

int topoep_ffn_backward(const topoep_ffn *f, const void *x, int64_t ldx, int32_t T, const topoep_ffn_rows *rows,
                        const void *up, const void *down, const void *saved, const void *grad_out, void *grad_x,
                        float *grad_weights, void *grad_up, void *grad_down, void *workspace, size_t workspace_bytes,
                        void *stream) {
  const int rc = check(f, T, rows);
  if (rc != TOPOEP_OK) return rc;
  if (T > 0) {
    if (!x || !up || !down || !saved || !grad_out || !workspace) return TOPOEP_EINVAL;
    if (rows && (!rows->offsets || !rows->pairs || !rows->places || !rows->weights)) return TOPOEP_EINVAL;
    if (ldx < f->hidden || (ldx & 7) || ldx > (int64_t)1 << 40) return TOPOEP_EINVAL;
  }
  if (!aligned16(x) || !aligned16(up) || !aligned16(down) || !aligned16(saved) || !aligned16(grad_out) ||
      !aligned16(grad_x) || !aligned16(grad_up) || !aligned16(grad_down))
    return TOPOEP_EINVAL;
  const Sizes s = sizes_of(f, T, rows);
  if ((reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < s.backward) return TOPOEP_EWORKSPACE;
  Ffn a = args_of(f, x, ldx, T, rows, up, down);
  if (T == 0) a.offsets = nullptr;   // no rows, whatever they say
  char *const kept = static_cast<char *>(const_cast<void *>(saved)), *const ws = static_cast<char *>(workspace);
  a.gu = reinterpret_cast<float *>(kept);
  a.h = kept ? kept + s.gu : nullptr;
  a.da = ws;
  a.y = reinterpret_cast<float *>(ws + s.da);
  a.part = reinterpret_cast<float *>(ws + s.da + s.back);
  a.sums = reinterpret_cast<float *>(ws + s.da + s.back + s.part);
  a.dout = grad_out;
  a.dx = grad_x;
  a.dw = rows ? grad_weights : nullptr;
  a.dup = grad_up;
  a.ddown = grad_down;
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const Counts c = counts_of(f, T, rows);
  const int parts = out_parts(f, c, rows, 2 * f->inter);
  const int pu = grad_parts(f, c, 2 * f->inter, f->hidden), pd = grad_parts(f, c, f->hidden, f->inter);
  return f->dtype == TOPOEP_BF16 ? backward<Bf16>(a, parts, pu, pd, st) : backward<F16>(a, parts, pu, pd, st);
}

}  // extern "C"
