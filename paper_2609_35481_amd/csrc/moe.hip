// A whole mixture-of-experts layer for a few tokens on gfx950.
//
// What has to move is the weights of every expert that some token picked,
// once; the tokens, the logits and the hidden rows are small.  So every
// product keeps weight rows as the matrix instruction's A operand, read from
// memory straight into registers, and the tokens that need them as its
// columns, which come from the caches.
//
//   gate    16 experts' logits a workgroup, the hidden axis split over its
//           waves and over kSplits workgroups, partial sums to the workspace
//   route   one wave a token: joins the partial sums in order, ids, weights,
//           and appends the token to its experts' lists
//   up      16 rows (8 hidden units' gate and up rows) of one expert a wave,
//           or a workgroup where there are few: h = silu(gate) * up, kept in two
//           words of the weights' type
//   down    the same over h, 16 outputs; every pair's result to the workspace
//   combine the weighted sum of a token's pairs in the order of its choices
//
// One token of a small layer: gate, then up with the routing inside, then down
// and the sum in one.  Many pairs an expert: up and down share their columns
// in LDS.
//
// Bound: memory, and for one token the chain of three kernels.  128 experts of
// H = 2048, I = 768, top-8: one token 23.3 us (76 MB, 11 at the 7.0 TB/s of reads
// alone), 64 tokens 209 us (1.19 GB, 170).  In a traced run, whose passes take
// 32 and 217 us: one token gate 3.1, up 13.4, down 7.9; 64 tokens up 125 (6.4
// TB/s), down 74 (5.4), gate, route and combine 16.
#include "router.h"

namespace {

using namespace topoep_dev;

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

constexpr int kTile = 16;                       // rows and columns of a matrix tile

// D += A B on 16 rows, 16 columns and 32 of the inner axis: lane l holds 8
// inner elements from (l / 16) * 8 of row (column) l % 16, and of D the rows
// (l / 16) * 4 + 0..3 of column l % 16.
template <class T> __device__ inline v4f mfma(v4i a, v4i b, v4f d);
template <> __device__ inline v4f mfma<Bf16>(v4i a, v4i b, v4f d) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), d, 0, 0, 0);
}
template <> __device__ inline v4f mfma<F16>(v4i a, v4i b, v4f d) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), d, 0, 0, 0);
}

// A hidden value between the two products: two words of the weights' type, so
// that it keeps 16 bits (bf16) and 22 (f16), below what rounding an output costs,
// for no byte of weights, only a second matrix instruction an operand.  One word alone put
// outputs up to 2^-8 (bf16) of their terms away.  f16's first word counts 2^11-fold, so
// that values up to 2^27 are held, not 65504 alone; its products have sums of their own.
template <class T> struct Hidden;
template <> struct Hidden<Bf16> {
  static constexpr int kSums = 1;
  static constexpr float kFirst = 1.0f, kMost = INFINITY;
};
template <> struct Hidden<F16> {
  static constexpr int kSums = 2;
  static constexpr float kFirst = 2048.0f, kMost = 65504.0f;
};
// Column operands' words and sums of the first product (Up) and the second.
template <class T, bool Up> constexpr int kWords = Up ? 1 : 2;
template <class T, bool Up> constexpr int kSums = Up ? 1 : Hidden<T>::kSums;

__device__ inline float clamp(float f, float most) { return f > most ? most : f < -most ? -most : f; }   // NaN stays

template <class T>
__device__ inline void split(float h, T &first, T &second) {
  first = from_float<T>(clamp(h * (1.0f / Hidden<T>::kFirst), Hidden<T>::kMost));
  const float rest = h - to_float(first) * Hidden<T>::kFirst;
  // (an infinity's own difference is none)
  second = from_float<T>(clamp(rest == rest ? rest : 0.0f, Hidden<T>::kMost));
}

// The pairs (token, choice) by expert, in the workspace.  Waves append to
// them in any order: an expert's pairs are columns of a product, each
// computed by itself, and experts are taken in the order of their ids, so no
// result depends on that order.
struct Lists {
  uint32_t *active;     // [E / 32 rounded up] bit e % 32 of word e / 32: expert e has pairs
  int32_t *count;       // [E] its pairs
  int32_t *pairs;       // [E, T] t * k + j
};

struct Layer {
  RouterArgs r;
  int T, H, I, L;
  const void *x;
  int64_t ldx;
  const void *gate;
  const float *bias;
  const int32_t *slot;
  const void *up, *down;
  void *out;
  int32_t *ids;
  float *weights;
  float *logits;        // [kSplits, T, E]
  void *hidden;         // [T * k, 2, I] first and second words
  float *each;          // [T * k, H] what each pair's expert gives
  Lists lists;
};

// ---------------------------------------------------------------- products

// How a matrix instruction's operands are laid over the weights.  P = 1: A
// holds 16 rows, 32 elements of each (64 bytes a row and load).  P = 2 and 4:
// A holds 16 / P rows, 32 P consecutive elements of each, a row of A being one
// part of 32 (128 and 256 bytes a row and load), and B the same parts of 16 / P
// columns; of D only the products of equal parts are kept.  Memory gives 16
// rows of 64 bytes 5.0 to 6.2 TB/s, 4 rows of 256 bytes, read past the caches,
// 7.0 (768 MB, rows of 4 to 28 KB), which the dropped products are cheap for:
// a tile of 16 rows takes P A operands, so P times the instructions.  The P parts
// of a row or column are P lanes side by side, and a part is every P-th 16 bytes
// of it, so that neighbouring lanes read neighbouring bytes: a load then looks up as
// many lines as it has rows, not one a lane (64 tokens, 128 experts of H = 2048, I =
// 768, top-8: 211 us, 239 with a lane's neighbours in other rows).
template <int P>
struct Parts {
  static constexpr int kCols = kTile / P;    // rows of an A operand, columns of a B operand
  static constexpr int kStep = 32 * P;       // elements of the inner axis
  // This lane's row (column) of an operand, and its place in a step of it.
  static __device__ int index() { return lane_id() % kTile / P; }
  static __device__ int place() { return ((lane_id() >> 4) * P + lane_id() % P) * 8; }
  // Of an operand's products d the rows (lane / 16) * 4 / P + 0 .. 4 / P - 1 of column
  // index(), all parts joined, the same in each of the P lanes side by side.
  static __device__ void join(const v4f &d, float (&s)[4 / P]) {
    static_assert(P == 2 || P == 4, "");
    const int part = lane_id() % P;
#pragma unroll
    for (int j = 0; j < 4 / P; ++j) {
      float v = d[j * P];
#pragma unroll
      for (int i = 1; i < P; ++i) v = part == i ? d[j * P + i] : v;
      v += dpp_movf<0xB1>(v);
      if (P == 4) v += dpp_movf<0x4E>(v);
      s[j] = v;
    }
  }
};

// The inner axis is streamed in runs of S steps, all of whose loads are in flight
// before the first product; four and more waves a SIMD fill each other's gaps
// (two runs a wave in registers: fewer waves, and slower).  Rows and columns
// that do not exist read an existing one instead (their products are dropped),
// so that no load of a full run depends on a condition.
template <class T, int P, int NA, int C, int S, int W, int A>
struct Run {
  v4i a[S][NA], b[W][S][C];
  __device__ void load(const char *rows, const uint32_t (&row)[NA], const char *cols, const uint32_t (&col)[C],
                       uint32_t word) {
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
      for (int s = 0; s < S; ++s) {
        const v4i *p = reinterpret_cast<const v4i *>(rows + row[i] + Parts<P>::kStep * 2 * s);
        a[s][i] = P > 1 ? __builtin_nontemporal_load(p) : *p;
      }
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int s = 0; s < S; ++s)
          b[w][s][c] = *reinterpret_cast<const v4i *>(cols + w * word + col[c] + Parts<P>::kStep * 2 * s);
  }
  __device__ void multiply(v4f (&d)[A][NA][C]) const {
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int w = 0; w < W; ++w)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int i = 0; i < NA; ++i) d[w % A][i][c] = mfma<T>(a[s][i], b[w][s][c], d[w % A][i][c]);
  }
};

// d += rows * columns over k in [0, n): runs `first`, first + every, ... of
// this wave, from the `turn`-th of them on and round (tiles that run side by side
// then read different places of their rows), and its share of the steps behind
// the last run.  row, col: bytes from rows and cols to the lane's own place
// (Parts::place()) of k = 0; columns are W words of n elements, one behind the
// other, whose products go to A sums.
template <class T, int P, int S, int W, int NA, int C, int A>
__device__ inline void stream(const char *rows, const uint32_t (&row)[NA], const char *cols, const uint32_t (&col)[C],
                              int n, uint32_t word, int first, int every, uint32_t turn, v4f (&d)[A][NA][C]) {
  constexpr int kRun = Parts<P>::kStep * S;
  const int full = n / kRun;
  if (first < full) {
    const int mine = (full - first + every - 1) / every, step = every * kRun, end = (first + mine * every) * kRun;
    int k = (first + (int)(turn % (uint32_t)mine) * every) * kRun;
#pragma unroll 1
    for (int i = 0; i < mine; ++i) {
      Run<T, P, NA, C, S, W, A> x;
      x.load(rows + k * 2, row, cols + k * 2, col, word);
      k += step;
      if (k >= end) k = first * kRun;
      x.multiply(d);
    }
  }
  // the rest, a step at a time: what lies behind the axis reads the row's start and counts as zero
  const int place = Parts<P>::place();
#pragma unroll 1
  for (int k = full * kRun + first * Parts<P>::kStep; k < n; k += every * Parts<P>::kStep) {
    const bool in = k + place < n;
    const uint32_t at = in ? (uint32_t)k * 2u : 0u - (uint32_t)place * 2u;
    const v4i zero = {0, 0, 0, 0};
    v4i a[NA], b[W][C];
    __builtin_amdgcn_sched_barrier(0);   // (addresses formed before the loop: 16 bytes of scratch for f16)
#pragma unroll
    for (int i = 0; i < NA; ++i) a[i] = *reinterpret_cast<const v4i *>(rows + (row[i] + at));
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int c = 0; c < C; ++c) b[w][c] = *reinterpret_cast<const v4i *>(cols + (col[c] + w * word + at));
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < NA; ++i) d[w % A][i][c] = mfma<T>(in ? a[i] : zero, in ? b[w][c] : zero, d[w % A][i][c]);
  }
}

// The sums of a product's words, as one.
template <class T, int A>
__device__ inline v4f join_sums(const v4f &first, const v4f &second) {
  return A == 1 ? first : Hidden<T>::kFirst * first + second;
}

// ---------------------------------------------------------------- logits

constexpr int kGateWaves = 8;
constexpr int kSplits = 8;   // parts of the hidden axis, each a workgroup's

template <class T, int C>
__global__ __launch_bounds__(64 * kGateWaves) void gate_kernel(Layer a) {
  __shared__ v4f part[kGateWaves][64];
  if (blockIdx.x == 0 && blockIdx.y == 0)   // the routing kernel appends to these
    for (int e = threadIdx.x; e < a.r.E; e += 64 * kGateWaves) {
      a.lists.count[e] = 0;
      if ((e & 31) == 0) a.lists.active[e >> 5] = 0;
    }
  const int lane = lane_id(), wave = uniform_i32(threadIdx.x >> 6), col = lane & 15, inner = (lane >> 4) * 8;
  const uint32_t row[1] = {((uint32_t)imin(blockIdx.x * kTile + col, a.r.E - 1) * a.H + inner) * 2u};
  uint32_t src[C];
#pragma unroll
  for (int c = 0; c < C; ++c) src[c] = ((uint32_t)imin(c * kTile + col, a.T - 1) * (uint32_t)a.ldx + inner) * 2u;
  v4f d[1][1][C] = {};
  stream<T, 1, 2, 1>(static_cast<const char *>(a.gate), row, static_cast<const char *>(a.x), src, a.H, 0,
                     blockIdx.y * kGateWaves + wave, kSplits * kGateWaves, 0, d);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (c > 0) __syncthreads();
    part[wave][lane] = d[0][0][c];
    __syncthreads();
    const int l = threadIdx.x, t = c * kTile + (l & 15), e = blockIdx.x * kTile + (l >> 4) * 4;
    if (l < 64 && t < a.T) {
      v4f s = part[0][l];
#pragma unroll
      for (int w = 1; w < kGateWaves; ++w) s += part[w][l];
      float *to = a.logits + ((int64_t)blockIdx.y * a.T + t) * a.r.E + e;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (e + j < a.r.E) to[j] = s[j];
    }
  }
}

// ---------------------------------------------------------------- routing

// Token t's logits, the partial sums joined in order, and the biases of a
// lane's V experts.
template <int V>
__device__ inline void few_logits(const Layer &a, int t, float (&x)[V], float (&b)[V]) {
  const float *from = a.logits + (int64_t)t * a.r.E;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int e = imin(lane_id() * V + v, a.r.E - 1);
    float part[kSplits];
#pragma unroll
    for (int i = 0; i < kSplits; ++i) part[i] = from[(int64_t)i * a.T * a.r.E + e];
    b[v] = a.bias ? a.bias[e] : 0.0f;
    float s = part[0];
#pragma unroll
    for (int i = 1; i < kSplits; ++i) s += part[i];
    x[v] = lane_id() * V + v < a.r.E ? clean_logit(s) : -INFINITY;
  }
}

// An expert's place among the weights here, -1 where it is not here.
__device__ inline int slot_of(const Layer &a, int e) {
  const int s = a.slot ? a.slot[e] : e;
  return (unsigned)s < (unsigned)a.L ? s : -1;
}

template <int V>
__global__ __launch_bounds__(256) void few_route_kernel(Layer a) {
  __shared__ uint32_t scratch[4][kRouteScratch];
  const int wave = threadIdx.x >> 6, sub = lane_id();
  const int t = blockIdx.x * 4 + wave;
  const bool live = t < a.T;
  float x[V], b[V];
  few_logits<V>(a, live ? t : 0, x, b);
  route_row<64, V>(a.r, x, b, sub, scratch[wave], live, a.ids + (int64_t)t * a.r.k, a.weights + (int64_t)t * a.r.k);
  if (live && sub < a.r.k) {
    const int e = (int)scratch[wave][2 * sub];
    if (slot_of(a, e) >= 0) {
      const int at = atomicAdd(&a.lists.count[e], 1);
      a.lists.pairs[(int64_t)e * a.T + at] = t * a.r.k + sub;
      // (without waiting for the count, a bit for every pair: 7.0 us for 64 tokens, not 4.9)
      if (at == 0) atomicOr(&a.lists.active[e >> 5], 1u << (e & 31));
    }
  }
}

// The n-th expert with pairs, by id; -1 where there are fewer.
__device__ inline int nth_active(const Layer &a, int n) {
  const int words = (a.r.E + 31) / 32;
  const uint32_t w = lane_id() < words ? a.lists.active[lane_id()] : 0u;
  const int ones = __popc(w), before = wave_incl_scan(ones) - ones;
  const uint64_t has = __ballot(before <= n && n < before + ones);
  if (has == 0) return -1;
  const int l = __ffsll((unsigned long long)has) - 1;
  uint32_t bits = (uint32_t)__builtin_amdgcn_readlane((int)w, l);
  for (int skip = n - __builtin_amdgcn_readlane(before, l); skip > 0; --skip) bits &= bits - 1;
  return l * 32 + __ffs((int)bits) - 1;
}

// ---------------------------------------------------------------- experts

constexpr int kExpertWaves = 4;

// Steps of a run by P and C; with few tokens and shared tiles every load of a row
// of 2048 elements is in flight at once.
constexpr int run_steps(int P, int C, int KS, int W) {
  return P == 4 ? (C == 1 ? (KS > 1 ? (W > 1 ? 3 : 4) : 2) : 1) : 2;
}

// How many pairs an expert has, about; kFew serves any number.
enum Load { kOne, kFew };   // at most 4; mostly up to 16

// Columns' operands a wave's piece of LDS holds the sums of, and the quads of rows
// of one of them.
template <int Kind> constexpr int kPieces = Kind == kOne ? 1 : 2;
constexpr int kPiece = 32;

// A tile of 16 rows of one expert against 16 / P * C of its pairs.  Rows: 8
// hidden units' gate rows and their up rows (Up), or 16 outputs.  KS = 1: the
// tile is the wave's own; KS = kExpertWaves: the workgroup's waves share it, each
// with its part of the runs.
template <class T, bool Up, int P, int C, int KS, int Kind>
__device__ inline void expert_tile(const Layer &a, const char *weights, const int32_t *pairs, int count, int tile,
                                   v4f (*part)[kPiece]) {
  constexpr int R = Parts<P>::kCols, kRows = Up ? 8 : 16;
  const int lane = lane_id(), index = Parts<P>::index(), wave = uniform_i32(threadIdx.x >> 6), place = Parts<P>::place(), at0 = tile * kRows;
  const int n = Up ? a.H : a.I;
  uint32_t row[P], src[C];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int r = i * R + index;
    row[i] = ((uint32_t)(Up ? (r >> 3) * a.I + imin(at0 + (r & 7), a.I - 1) : imin(at0 + r, a.H - 1)) * n + place) * 2u;
  }
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = c * R + index;
    const int p = pairs[at < count ? at : 0];
    src[c] = ((Up ? (uint32_t)(p / a.r.k) * (uint32_t)a.ldx : (uint32_t)p * 2u * (uint32_t)a.I) + place) * 2u;
  }
  const char *cols = static_cast<const char *>(Up ? a.x : a.hidden);
  constexpr int W = kWords<T, Up>, A = kSums<T, Up>;
  v4f d[A][P][C] = {};
  // eight tiles side by side run on eight XCDs
  stream<T, P, run_steps(P, C, Kind == kOne ? KS : 1, W), W>(weights, row, cols, src, n, (uint32_t)n * 2u,
                                                             KS == 1 ? 0 : wave, KS, tile >> 3, d);
  constexpr int CE = C < 2 ? 1 : 2;   // columns' operands whose sums are joined at a time
  // a wave's piece does not depend on CE: waves with tiles of their own may be at
  // experts of other counts
  v4f (*own)[kPiece] = KS == 1 ? part + wave * kPieces<Kind> : part;
#pragma unroll
  for (int c0 = 0; c0 < C; c0 += CE) {
    if (KS == 1) wave_sync(); else __syncthreads();
#pragma unroll
    for (int c = 0; c < CE; ++c) {
      float s[P][4 / P];
#pragma unroll
      for (int i = 0; i < P; ++i)
        Parts<P>::join(join_sums<T, A>(d[0][i][c0 + c], d[A - 1][i][c0 + c]), s[i]);
      // of the lanes side by side the i-th leaves operand i's
      const int i = lane % P, row = i * R + (lane >> 4) * (4 / P);
      float *to = reinterpret_cast<float *>(&own[(KS == 1 ? 0 : wave * CE) + c][row / 4 * R + index]) + row % 4;
#pragma unroll
      for (int j = 0; j < 4 / P; ++j) {
        float v = s[0][j];
#pragma unroll
        for (int o = 1; o < P; ++o) v = i == o ? s[o][j] : v;
        to[j] = v;
      }
    }
    if (KS == 1) wave_sync(); else __syncthreads();
    const auto sum = [&](int c, int quad, int t) {   // rows quad * 4 + 0..3 of the tile
      v4f s = own[c][quad * R + t];
#pragma unroll
      for (int w = 1; w < KS; ++w) s += own[w * CE + c][quad * R + t];
      return s;
    };
    constexpr int kQuads = Up ? 2 : 4;
#pragma unroll 1
    for (int o = KS == 1 ? lane : (int)threadIdx.x; o < CE * R * kQuads; o += KS * 64) {
      const int quad = o % kQuads, t = o / kQuads % R, c = o / kQuads / R, at = at0 + quad * 4, n0 = (c0 + c) * R + t;
      if (n0 >= count || at >= (Up ? a.I : a.H)) continue;
      const int64_t pair = pairs[n0];
      const v4f g = sum(c, quad, t);
      if (Up) {
        const v4f u = sum(c, quad + 2, t);
        T h[2][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) split(g[j] * sigmoid(g[j]) * u[j], h[0][j], h[1][j]);
        T *to = static_cast<T *>(a.hidden) + pair * 2 * a.I + at;
        __builtin_memcpy(to, h[0], sizeof(h[0]));
        __builtin_memcpy(to + a.I, h[1], sizeof(h[1]));
      } else {
        *reinterpret_cast<v4f *>(a.each + pair * a.H + at) = g;
      }
    }
  }
}

// Workgroup b takes tile b % groups (KS = 1: its waves four tiles side by side) of
// the experts b / groups, b / groups + gridDim / groups, ... of those with pairs.
template <class T, bool Up, int KS, int Kind>
__global__ __launch_bounds__(64 * kExpertWaves, 4) void expert_kernel(Layer a, int groups) {
  __shared__ v4f part[kExpertWaves * kPieces<Kind>][kPiece];
  constexpr int kRows = Up ? 8 : 16;
  const int tiles = ((Up ? a.I : a.H) + kRows - 1) / kRows, group = (int)blockIdx.x % groups;
  const int tile = KS == 1 ? group * kExpertWaves + uniform_i32(threadIdx.x >> 6) : group;
  if (tile >= tiles) return;
  for (int i = blockIdx.x / groups;; i += gridDim.x / groups) {
    const int e = nth_active(a, i);
    if (e < 0) return;
    const int count = a.lists.count[e];
    const int32_t *pairs = a.lists.pairs + (int64_t)e * a.T;
    const int64_t slot = a.slot ? a.slot[e] : e;
    const char *w = Up ? static_cast<const char *>(a.up) + slot * 4 * a.I * a.H
                       : static_cast<const char *>(a.down) + slot * 2 * a.H * a.I;
    if (Kind == kOne || count <= 4) {
      expert_tile<T, Up, 4, 1, KS, Kind>(a, w, pairs, count, tile, part);
    } else if (count <= 8) {
      expert_tile<T, Up, 4, 2, KS, Kind>(a, w, pairs, count, tile, part);
    } else {
      for (int at = 0; at < count; at += 16) expert_tile<T, Up, 2, 2, KS, Kind>(a, w, pairs + at, count - at, tile, part);
    }
  }
}

// Many pairs an expert: the columns' operands would cost more of the caches than
// the rows' of memory, so a workgroup's waves share them.  A stage is 32 to 128 of
// the inner axis of all of the expert's columns in LDS (chunks of 16 bytes, their
// places turned by the column so that no bank is met twice), double-buffered;
// each wave has 32 rows of its own (16 hidden units' gate and up rows, or 32
// outputs) straight from memory, one stage ahead.
template <class T, bool Up, int kStage>
__global__ __launch_bounds__(64 * kExpertWaves, (kStage * (Up ? 1 : 2) > 128 ? 1 : 2)) void many_kernel(Layer a, int tiles) {
  constexpr int kChunks = kStage / 8, kSteps = kStage / 32, W = kWords<T, Up>, A = kSums<T, Up>;
  constexpr int kCols = TOPOEP_MOE_MAX_TOKENS / kTile, kEach = 64 * kExpertWaves / kChunks,
                kUnits = TOPOEP_MOE_MAX_TOKENS / kEach;   // columns a pass of the workgroup stages, and passes
  __shared__ v4i stage[2][W][TOPOEP_MOE_MAX_TOKENS][kChunks];
  const auto turned = [](int c) { return kChunks < 8 ? c >> 2 & 3 : c & 7; };
  const int lane = lane_id(), wave = uniform_i32(threadIdx.x >> 6), r = lane & 15, place = (lane >> 4) * 8;
  const int n = Up ? a.H : a.I, rows = Up ? a.I : a.H, stages = (n + kStage - 1) / kStage;
  const int first = ((int)blockIdx.x % tiles * kExpertWaves + wave) * (Up ? 16 : 32);   // of this wave's units or outputs
  for (int i = blockIdx.x / tiles;; i += gridDim.x / tiles) {
    const int e = nth_active(a, i);
    if (e < 0) return;
    const int count = a.lists.count[e], cols = (count + kTile - 1) / kTile;
    const int32_t *pairs = a.lists.pairs + (int64_t)e * a.T;
    const int64_t slot = a.slot ? a.slot[e] : e;
    const char *w = Up ? static_cast<const char *>(a.up) + slot * 4 * a.I * a.H
                       : static_cast<const char *>(a.down) + slot * 2 * a.H * a.I;
    const char *from = static_cast<const char *>(Up ? a.x : a.hidden);
    uint32_t row[2], src[kUnits];
    row[0] = ((uint32_t)imin(first + r, rows - 1) * n + place) * 2u;
    row[1] = ((uint32_t)(Up ? a.I + imin(first + r, rows - 1) : imin(first + 16 + r, rows - 1)) * n + place) * 2u;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {   // this thread's columns and chunk of a stage
      const int c = (int)threadIdx.x / kChunks + kEach * u, p = pairs[c < count ? c : 0];
      src[u] = ((Up ? (uint32_t)(p / a.r.k) * (uint32_t)a.ldx : (uint32_t)p * 2u * (uint32_t)a.I) + threadIdx.x % kChunks * 8) * 2u;
    }
    v4i x[2][kSteps], b[W][kUnits];
    v4f d[A][2][kCols] = {};
    const v4i zero = {0, 0, 0, 0};
    // what lies behind the axis reads its start and counts as zero
    const auto load = [&](int k) {
#pragma unroll
      for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          const bool in = k + 32 * s + place < n;
          const v4i v = *reinterpret_cast<const v4i *>(w + (row[q] + (in ? (uint32_t)(k + 32 * s) * 2u : 0u - place * 2u)));
          x[q][s] = in ? v : zero;
        }
      const uint32_t mine = threadIdx.x % kChunks * 8;
      const bool in = k + (int)mine < n;
#pragma unroll
      for (int u = 0; u < kUnits; ++u)
        if (kEach * u < count) {
#pragma unroll
          for (int m = 0; m < W; ++m) {
            const v4i v = *reinterpret_cast<const v4i *>(from + (src[u] + m * (uint32_t)n * 2u + (in ? (uint32_t)k * 2u : 0u - mine * 2u)));
            b[m][u] = in ? v : zero;
          }
        }
    };
    // tiles that run side by side start at different places of their rows
    int at_stage = (int)((uint32_t)((int)blockIdx.x % tiles >> 3) * 5u % (uint32_t)stages);
    load(at_stage * kStage);
    for (int g = 0; g < stages; ++g) {
#pragma unroll
      for (int u = 0; u < kUnits; ++u)
        if (kEach * u < count) {
          const int c = (int)threadIdx.x / kChunks + kEach * u;
#pragma unroll
          for (int m = 0; m < W; ++m) stage[g & 1][m][c][threadIdx.x % kChunks ^ turned(c)] = b[m][u];
        }
      v4i now[2][kSteps];
#pragma unroll
      for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int s = 0; s < kSteps; ++s) now[q][s] = x[q][s];
      __syncthreads();
      at_stage = at_stage + 1 < stages ? at_stage + 1 : 0;
      if (g + 1 < stages) load(at_stage * kStage);
#pragma unroll
      for (int c = 0; c < kCols; ++c)
        if (c < cols) {
#pragma unroll
          for (int s = 0; s < kSteps; ++s) {
            const int at = c * kTile + r;
#pragma unroll
            for (int m = 0; m < W; ++m) {
              const v4i col = stage[g & 1][m][at][(s * 4 + (lane >> 4)) ^ turned(at)];
#pragma unroll
              for (int q = 0; q < 2; ++q) d[m % A][q][c] = mfma<T>(now[q][s], col, d[m % A][q][c]);
            }
          }
        }
    }
    const int at = first + (lane >> 4) * 4;   // this lane's four units or outputs, of column r of each tile
#pragma unroll
    for (int c = 0; c < kCols; ++c) {
      if (c * kTile + r >= count) continue;
      const int64_t pair = pairs[c * kTile + r];
      if (Up) {
        const v4f g = d[0][0][c], up = d[0][1][c];
        T h[2][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) split(g[j] * sigmoid(g[j]) * up[j], h[0][j], h[1][j]);
        T *to = static_cast<T *>(a.hidden) + pair * 2 * a.I + at;
        if (at < rows) {
          __builtin_memcpy(to, h[0], sizeof(h[0]));
          __builtin_memcpy(to + a.I, h[1], sizeof(h[1]));
        }
      } else {
        float *to = a.each + pair * a.H + at;
        if (at < rows) *reinterpret_cast<v4f *>(to) = join_sums<T, A>(d[0][0][c], d[A - 1][0][c]);
        if (at + 16 < rows) *reinterpret_cast<v4f *>(to + 16) = join_sums<T, A>(d[0][1][c], d[A - 1][1][c]);
      }
    }
    __syncthreads();   // before the next expert's stages
  }
}

// One token: every wave routes it for itself, which takes the routing kernel and
// a launch off the path (one token, 128 experts of H = 2048, I = 768, from a graph:
// 29.5 us, 33.7 with five kernels); workgroup 0 leaves what the next kernel reads.  Workgroup b takes tile b % tiles of the token's choices b / tiles, b /
// tiles + gridDim / tiles, ... here: more than the places where some share one.
template <class T, int V>
__global__ __launch_bounds__(64 * kExpertWaves, 4) void one_up_kernel(Layer a, int tiles) {
  __shared__ uint32_t scratch[kExpertWaves][kRouteScratch];
  __shared__ v4f part[kExpertWaves][kPiece];
  const int wave = uniform_i32(threadIdx.x >> 6), lane = lane_id();
  const bool writes = blockIdx.x == 0 && wave == 0;
  float x[V], b[V];
  few_logits<V>(a, 0, x, b);
  route_row<64, V>(a.r, x, b, lane, scratch[wave], writes, a.ids, a.weights);
  const int mine = lane < a.r.k ? (int)scratch[wave][2 * lane] : 0;
  const int slot = lane < a.r.k ? slot_of(a, mine) : -1;
  if (writes && slot >= 0) {
    a.lists.count[mine] = 1;
    a.lists.pairs[mine] = lane;
    atomicOr(&a.lists.active[mine >> 5], 1u << (mine & 31));
  }
  const uint64_t here = __ballot(slot >= 0);
  int32_t *pair = reinterpret_cast<int32_t *>(scratch[wave]);
  for (int n = (int)blockIdx.x / tiles; n < __popcll((unsigned long long)here); n += (int)gridDim.x / tiles) {
    const uint64_t before = __ballot(slot >= 0 && count_below(here, 0) == n);
    const int j = __ffsll((unsigned long long)before) - 1;
    wave_sync();
    if (lane == 0) pair[0] = j;
    wave_sync();
    const char *w = static_cast<const char *>(a.up) + (int64_t)readlane_i32(slot, j) * 4 * a.I * a.H;
    expert_tile<T, true, 4, 1, kExpertWaves, kOne>(a, w, pair, 1, (int)blockIdx.x % tiles, part);
  }
}

// out_t = sum over t's choices in order, of those whose expert is here.
template <class T>
__global__ __launch_bounds__(256) void combine_kernel(Layer a) {
  const int t = blockIdx.y, h = (blockIdx.x * 256 + threadIdx.x) * 4, p0 = t * a.r.k;
  int here = 0;
  float weight = 0.0f;
  if (lane_id() < a.r.k) {
    here = slot_of(a, a.ids[p0 + lane_id()]) >= 0;
    weight = a.weights[p0 + lane_id()];
  }
  const float *from = a.each + (int64_t)p0 * a.H + imin(h, a.H - 4);
  v4f s = {0.0f, 0.0f, 0.0f, 0.0f};
  for (uint64_t left = __ballot(here); left != 0;) {
    v4f v[8];
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {   // up to eight choices in flight; the rest repeat the last with weight zero
      const int j = left != 0 ? __ffsll((unsigned long long)left) - 1 : -1;
      w[i] = j < 0 ? 0.0f : __uint_as_float((uint32_t)readlane_i32((int)__float_as_uint(weight), j < 0 ? 0 : j));
      if (j >= 0) v[i] = *reinterpret_cast<const v4f *>(from + (int64_t)j * a.H);
      else v[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
      left &= left - 1;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) s += w[i] * v[i];
  }
  if (h >= a.H) return;
  T out[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) out[j] = from_float<T>(s[j]);
  __builtin_memcpy(static_cast<T *>(a.out) + (int64_t)t * a.H + h, out, sizeof(out));
}

constexpr int kDownWaves = 8;

// One unit of a wave: `len` of the inner axis from `lo` of one expert's pairs,
// 4 NA outputs from row o0 on, 4 C columns.
template <class T, int NA, int C>
__device__ inline void down_unit(const Layer &a, const char *weights, int o0, const int32_t *pairs, int count, int lo,
                                 int len, v4f *mine) {
  const int lane = lane_id(), index = Parts<4>::index(), place = Parts<4>::place();
  uint32_t row[NA], src[C];
  int pair[C];
#pragma unroll
  for (int i = 0; i < NA; ++i) row[i] = ((uint32_t)imin(o0 + 4 * i + index, a.H - 1) * a.I + place) * 2u;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = c * 4 + index;
    pair[c] = pairs[at < count ? at : 0];
    src[c] = ((uint32_t)pair[c] * 2u * (uint32_t)a.I + place) * 2u;
    if (at >= count) pair[c] = -1;
  }
  const char *cols = static_cast<const char *>(a.hidden);
  constexpr int W = kWords<T, false>, A = kSums<T, false>;
  const uint32_t word = (uint32_t)a.I * 2u;
  v4f d[A][NA][C] = {};
  // four steps (512 elements) in flight, then two, then one
  constexpr int kLong = 4 * Parts<4>::kStep;
  const int most = len / kLong * kLong;
  if (C == 1) stream<T, 4, 4, W>(weights + lo * 2, row, cols + lo * 2, src, most, word, 0, 1, blockIdx.x / 8, d);
  const int done = C == 1 ? most : 0;
  stream<T, 4, 2, W>(weights + (lo + done) * 2, row, cols + (lo + done) * 2, src, len - done, word, 0, 1, 0, d);
  // output 4 i + lane / 16 of this lane's column, left by the i-th of the lanes side by side
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      float s[1];
      Parts<4>::join(join_sums<T, A>(d[0][i][c], d[A - 1][i][c]), s);
      if (lane % 4 == i && pair[c] >= 0) {
        float *to = reinterpret_cast<float *>(mine + pair[c] / a.r.k * NA + i) + (lane >> 4);
        *to = *to + a.weights[pair[c]] * s[0];
      }
    }
}

// The products with `down` and the weighted sum in one, for few pairs: a
// workgroup has 4 NA outputs of every token; its waves take the units (an
// expert, a part of the inner axis) in turn, each into LDS sums of its own.
template <class T, int NA>
__global__ __launch_bounds__(64 * kDownWaves, 3) void down_kernel(Layer a) {
  extern __shared__ v4f sums[];   // [kDownWaves][T][NA]
  const int wave = uniform_i32(threadIdx.x >> 6), lane = lane_id(), size = a.T * NA;
  const v4f zero = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int i = threadIdx.x; i < kDownWaves * size; i += 64 * kDownWaves) sums[i] = zero;
  __syncthreads();
  int active = lane < (a.r.E + 31) / 32 ? __popc(a.lists.active[lane]) : 0;
  active = readlane_i32(wave_incl_scan(active), 63);
  // parts of the axis so that every wave has a unit
  int parts = 1;
  while (parts < kDownWaves && active * parts < kDownWaves) parts *= 2;
  const int len = ((a.I + parts - 1) / parts + 127) & ~127;
  v4f *mine = sums + wave * size;
  for (int unit = wave; unit < active * parts; unit += kDownWaves) {
    const int e = nth_active(a, unit / parts), lo = unit % parts * len;
    if (lo >= a.I) continue;
    const int count = a.lists.count[e], m = imin(len, a.I - lo);
    const int32_t *pairs = a.lists.pairs + (int64_t)e * a.T;
    const char *w = static_cast<const char *>(a.down) + (int64_t)(a.slot ? a.slot[e] : e) * a.H * a.I * 2;
    const int o0 = blockIdx.x * 4 * NA;
    if (count <= 4) down_unit<T, NA, 1>(a, w, o0, pairs, count, lo, m, mine);
    else
      for (int at = 0; at < count; at += 8) down_unit<T, NA, 2>(a, w, o0, pairs + at, count - at, lo, m, mine);
    wave_sync();
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.T * NA; i += 64 * kDownWaves) {
    const int t = i / NA, at = i % NA, row = (blockIdx.x * NA + at) * 4;
    v4f s = zero;
#pragma unroll
    for (int w = 0; w < kDownWaves; ++w) s += sums[w * size + t * NA + at];
    if (row >= a.H) continue;
    T out[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) out[j] = from_float<T>(s[j]);
    __builtin_memcpy(static_cast<T *>(a.out) + (int64_t)t * a.H + row, out, sizeof(out));
  }
}

// ---------------------------------------------------------------- host

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

struct Places {
  size_t active, count, pairs, logits, hidden, each, total;
};

Places places_of(const topoep_moe *m, const topoep_router *r, int T) {
  Places p;
  const size_t E = (size_t)r->num_experts, pairs = (size_t)T * r->topk;
  size_t at = 0;
  p.active = at;
  at += align256((E + 31) / 32 * sizeof(uint32_t));
  p.count = at;
  at += align256(E * sizeof(int32_t));
  p.pairs = at;
  at += align256(E * T * sizeof(int32_t));
  p.logits = at;
  at += align256(kSplits * T * E * sizeof(float));
  p.hidden = at;
  at += align256(pairs * m->inter * 4);
  p.each = at;
  at += align256(pairs * m->hidden * sizeof(float));
  p.total = at;
  return p;
}

int check_layer(const topoep_moe *m, const topoep_router *r, int32_t T) {
  if (!m || !r) return TOPOEP_EINVAL;
  if (m->hidden < 8 || (m->hidden & 7) || m->inter < 8 || (m->inter & 7) || m->local_experts < 1) return TOPOEP_EINVAL;
  // an expert's matrices, the tokens and the hidden rows are addressed by 32-bit byte offsets
  if (m->hidden > 1 << 17 || m->inter > 1 << 17 || (int64_t)m->hidden * m->inter > 1 << 30) return TOPOEP_EINVAL;
  if (m->dtype != TOPOEP_BF16 && m->dtype != TOPOEP_F16) return TOPOEP_EINVAL;
  topoep_router own = *r;
  own.dtype = TOPOEP_F32;   // not read: the logits never leave 32 bits
  const int rc = check_router(&own);
  if (rc != TOPOEP_OK) return rc;
  if (T < 0) return TOPOEP_EINVAL;
  return T > TOPOEP_MOE_MAX_TOKENS ? TOPOEP_ELIMIT : TOPOEP_OK;
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

bool launched() { return hipGetLastError() == hipSuccess; }

template <class T, bool Up, int Kind>
int enqueue_experts(const Layer &a, int experts, hipStream_t st) {
  const int rows = Up ? 8 : 16, tiles = ((Up ? a.I : a.H) + rows - 1) / rows;
  const dim3 block(64 * kExpertWaves);
  // A wave to a tile where there are tiles for all of the chip's 4096 places, or
  // for half of them and rows are short (64 against 67 us for 32 experts, H = 2048,
  // I = 768); else the workgroup to a tile (two experts, H = 4096, I = 14336: 127
  // against 164 us)
  const int64_t all = (int64_t)experts * tiles;
  if (all < 2048 || (all < 4096 && (Up ? a.H : a.I) > 2048)) {
    hipLaunchKernelGGL((expert_kernel<T, Up, kExpertWaves, Kind>), dim3((unsigned)experts * tiles), block, 0, st, a, tiles);
  } else {
    const int groups = (tiles + kExpertWaves - 1) / kExpertWaves;
    hipLaunchKernelGGL((expert_kernel<T, Up, 1, Kind>), dim3((unsigned)experts * groups), block, 0, st, a, groups);
  }
  return launched() ? TOPOEP_OK : TOPOEP_EHIP;
}

template <class T, bool Up, int kStage>
int enqueue_many(const Layer &a, int blocks, int tiles, hipStream_t st) {
  hipLaunchKernelGGL((many_kernel<T, Up, kStage>), dim3((unsigned)blocks), dim3(64 * kExpertWaves), 0, st, a, tiles);
  return launched() ? TOPOEP_OK : TOPOEP_EHIP;
}

template <class T, bool Up>
int enqueue_experts(const Layer &a, hipStream_t st) {
  const int experts = imin(imin(a.T * a.r.k, a.r.E), a.L);   // with pairs, about
  if (a.T <= 4) return enqueue_experts<T, Up, kOne>(a, experts, st);
  const int rows = kExpertWaves * (Up ? 16 : 32), tiles = ((Up ? a.I : a.H) + rows - 1) / rows;
  // more than 12 pairs an expert (64 experts of H = 2048, I = 768, top-8: 128 tokens 178 us
  // shared, 219 not; 96 tokens, 12 pairs: 171 and 178; 64 tokens: 166 and 141)
  if (a.T * a.r.k <= 12 * a.r.E) return enqueue_experts<T, Up, kFew>(a, experts, st);
  // Longer stages read rows in longer pieces, but fewer workgroups fit a CU: of the
  // first product three with stages of 64 and two with 128, of the second (two words)
  // three with 32, two with 64, one with 128.  The longer one where the chip's rounds leave
  // it no more than a seventh emptier (second product, 8 experts of I = 14336, 256 workgroups:
  // layer 820, 799 and 751 us; 20 experts of I = 2048, 640 workgroups: 289, 314, 348).
  const int blocks = experts * tiles, rounds2 = (blocks + 511) / 512, rounds3 = (blocks + 767) / 768;
  const bool longer = rounds2 * 512 * 6 <= rounds3 * 768 * 7;
  if constexpr (Up) {
    return longer ? enqueue_many<T, true, 128>(a, blocks, tiles, st) : enqueue_many<T, true, 64>(a, blocks, tiles, st);
  } else {
    if (blocks <= 256) return enqueue_many<T, false, 128>(a, blocks, tiles, st);
    if constexpr (kSums<T, false> == 1)   // (f16: its sums' registers let two workgroups run at most)
      if (!longer) return enqueue_many<T, false, 32>(a, blocks, tiles, st);
    return enqueue_many<T, false, 64>(a, blocks, tiles, st);
  }
}

template <class T, int NA>
int enqueue_down_rows(const Layer &a, hipStream_t st) {
  hipLaunchKernelGGL((down_kernel<T, NA>), dim3((a.H + 4 * NA - 1) / (4 * NA)), dim3(64 * kDownWaves),
                     kDownWaves * a.T * NA * sizeof(v4f), st, a);
  return launched() ? TOPOEP_OK : TOPOEP_EHIP;
}

// Four outputs a workgroup where eight would leave too few of them (one token, I = 512, H = 1024:
// layer 20.5 against 20.9 us; two tokens, I = 1024: 37.9 and 41.6; H = 1536: 22.1 and 21.2, 48.4 and 46.9).
template <class T>
int enqueue_down(const Layer &a, hipStream_t st) {
  return a.H <= 1024 ? enqueue_down_rows<T, 1>(a, st) : enqueue_down_rows<T, 2>(a, st);
}

template <class T>
int enqueue(const Layer &a, hipStream_t st) {
  const int E = a.r.E, cols = (a.T + kTile - 1) / kTile;
  (void)hipGetLastError();
  const dim3 gg((E + kTile - 1) / kTile, kSplits), gb(64 * kGateWaves);
  if (cols <= 1) hipLaunchKernelGGL((gate_kernel<T, 1>), gg, gb, 0, st, a);
  else if (cols <= 2) hipLaunchKernelGGL((gate_kernel<T, 2>), gg, gb, 0, st, a);
  else if (cols <= 4) hipLaunchKernelGGL((gate_kernel<T, 4>), gg, gb, 0, st, a);
  else hipLaunchKernelGGL((gate_kernel<T, 8>), gg, gb, 0, st, a);
  if (!launched()) return TOPOEP_EHIP;
  const int experts = imin(imin(a.T * a.r.k, E), a.L), tiles = (a.I + 7) / 8;
  // One token, three kernels or five (H = 2048, I = 768, 8 of 128 experts: 29.5 against 33.7 us;
  // H = 4096, I = 14336, 1 of 8: 69 and 77): where a workgroup has a tile (the rule of
  // enqueue_experts), and for up to 16 choices, behind which neither is always the faster
  // (H = 2048, I = 256, 24 choices: 34.7 and 37.3; H = 1024, I = 512, 32: 45.1 and 42.8).
  if (a.T == 1 && E <= 256 && (int64_t)experts * tiles < 2048 && a.r.k <= 16) {
    const dim3 grid((unsigned)experts * tiles), block(64 * kExpertWaves);
    if (E <= 64) hipLaunchKernelGGL((one_up_kernel<T, 1>), grid, block, 0, st, a, tiles);
    else if (E <= 128) hipLaunchKernelGGL((one_up_kernel<T, 2>), grid, block, 0, st, a, tiles);
    else hipLaunchKernelGGL((one_up_kernel<T, 4>), grid, block, 0, st, a, tiles);
    if (!launched()) return TOPOEP_EHIP;
    return enqueue_down<T>(a, st);
  }
  const dim3 rg((a.T + 3) / 4), rb(256);
  if (E <= 64) hipLaunchKernelGGL((few_route_kernel<1>), rg, rb, 0, st, a);
  else if (E <= 128) hipLaunchKernelGGL((few_route_kernel<2>), rg, rb, 0, st, a);
  else if (E <= 256) hipLaunchKernelGGL((few_route_kernel<4>), rg, rb, 0, st, a);
  else if (E <= 512) hipLaunchKernelGGL((few_route_kernel<8>), rg, rb, 0, st, a);
  else hipLaunchKernelGGL((few_route_kernel<16>), rg, rb, 0, st, a);
  if (!launched()) return TOPOEP_EHIP;
  int rc = enqueue_experts<T, true>(a, st);
  if (rc != TOPOEP_OK) return rc;
  // The second product and the sum in one, or two kernels, few pairs of small experts (H = 512,
  // I = 256: 16 pairs 24.4 against 25.2 us, 32 pairs 27.7 and 27.0; two tokens, H = 4096, I = 2048,
  // 4 experts: 49.6 and 52.0; from 2^26 weights on the one is from 2 % faster to 2 % slower).
  if (a.T * a.r.k <= 16 && (int64_t)experts * a.H * a.I <= 1 << 25) return enqueue_down<T>(a, st);
  rc = enqueue_experts<T, false>(a, st);
  if (rc != TOPOEP_OK) return rc;
  hipLaunchKernelGGL((combine_kernel<T>), dim3((a.H + 1023) / 1024, a.T), dim3(256), 0, st, a);
  return launched() ? TOPOEP_OK : TOPOEP_EHIP;
}

}  // namespace

extern "C" {

int topoep_moe_workspace_bytes(const topoep_moe *m, const topoep_router *r, int32_t T, size_t *bytes_out) {
  const int rc = check_layer(m, r, T);
  if (rc != TOPOEP_OK) return rc;
  if (!bytes_out) return TOPOEP_EINVAL;
  *bytes_out = places_of(m, r, T).total;
  return TOPOEP_OK;
}

int topoep_moe_few(const topoep_moe *m, const topoep_router *r, const void *x, int64_t ldx, int32_t T,
                   const void *gate, const float *bias, const int32_t *expert_slot, const void *up, const void *down,
                   void *out, int32_t *ids, float *weights, void *workspace, size_t workspace_bytes, void *stream) {
  const int rc = check_layer(m, r, T);
  if (rc != TOPOEP_OK) return rc;
  if (T == 0) return TOPOEP_OK;
  if (!x || !gate || !up || !down || !out || !ids || !weights || !workspace) return TOPOEP_EINVAL;
  if (ldx < m->hidden || (ldx & 7) || ldx >= 1 << 24) return TOPOEP_EINVAL;
  if (!aligned16(x) || !aligned16(gate) || !aligned16(up) || !aligned16(down) || !aligned16(out)) return TOPOEP_EINVAL;
  const Places p = places_of(m, r, T);
  if ((reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < p.total) return TOPOEP_EWORKSPACE;
  char *ws = static_cast<char *>(workspace);
  Layer a;
  a.r = router_args(r);
  a.T = T;
  a.H = m->hidden;
  a.I = m->inter;
  a.L = m->local_experts;
  a.x = x;
  a.ldx = ldx;
  a.gate = gate;
  a.bias = bias;
  a.slot = expert_slot;
  a.up = up;
  a.down = down;
  a.out = out;
  a.ids = ids;
  a.weights = weights;
  a.logits = reinterpret_cast<float *>(ws + p.logits);
  a.hidden = ws + p.hidden;
  a.each = reinterpret_cast<float *>(ws + p.each);
  a.lists.active = reinterpret_cast<uint32_t *>(ws + p.active);
  a.lists.count = reinterpret_cast<int32_t *>(ws + p.count);
  a.lists.pairs = reinterpret_cast<int32_t *>(ws + p.pairs);
  hipStream_t st = static_cast<hipStream_t>(stream);
  return m->dtype == TOPOEP_BF16 ? enqueue<Bf16>(a, st) : enqueue<F16>(a, st);
}

}  // extern "C"
