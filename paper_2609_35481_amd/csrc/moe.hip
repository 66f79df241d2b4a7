// A whole mixture-of-experts layer for a few tokens on gfx950.
//
// What has to move is the weights of every expert that some token picked,
// once; the tokens, the logits and the hidden rows are small.  So every
// product keeps a tile of 16 weight rows as the matrix instruction's A operand
// and the tokens that need it as its columns (16 a tile, up to 8 tiles):
// weights are read from memory once, straight into registers, and the
// tokens' operands come from the caches.
//
//   gate   logits: 16 experts a workgroup, the hidden axis split over its
//          waves and over `splits` workgroups, partial sums to the workspace
//   route  one wave a token: sums the partials in order, ids and weights
//   lists  one workgroup: the pairs (token, choice) by expert
//   up     16 hidden units of one expert a workgroup, H split over its waves:
//          h = silu(gate) * up for the expert's pairs
//   down   16 outputs a workgroup: its waves take the (expert, part of I)
//          units in turn, each into LDS sums of its own, joined in order
#include "router.h"

namespace {

using namespace topoep_dev;

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

constexpr int kTile = 16;                       // rows and columns of a matrix tile
constexpr int kMaxCols = TOPOEP_MOE_MAX_TOKENS / kTile;

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

// Eight elements at p[k], zero where not ok.
template <class T>
__device__ inline v4i load8(const T *p, int k, bool ok) {
  v4i v = {0, 0, 0, 0};
  if (ok) v = *reinterpret_cast<const v4i *>(p + k);
  return v;
}

struct Lists {          // the pairs by expert, in the workspace
  int32_t *active;      // [1] experts with pairs
  int32_t *slot;        // [E] their weights' place
  int32_t *begin;       // [E + 1] their first pair
  int32_t *pairs;       // [T * k] pair t * k + j
};

struct Layer {
  RouterArgs r;
  int T, H, I, L, splits;
  const void *x;
  int64_t ldx;
  const void *gate;
  const float *bias;
  const int32_t *slot;
  const void *up, *down;
  void *out;
  int32_t *ids;
  float *weights;
  float *logits;        // [splits, T, E]
  void *hidden;         // [T * k, I]
  Lists lists;
};

// ---------------------------------------------------------------- logits

constexpr int kGateWaves = 4;

template <class T, int C>
__global__ __launch_bounds__(64 * kGateWaves) void gate_kernel(Layer a) {
  __shared__ v4f part[kGateWaves][C][64];
  const int lane = lane_id(), wave = threadIdx.x >> 6, col = lane & 15, inner = (lane >> 4) * 8;
  const int e = blockIdx.x * kTile + col;
  const T *row = static_cast<const T *>(a.gate) + (int64_t)e * a.H;
  v4f d[C] = {};
  const int step = 32 * kGateWaves * a.splits;
  for (int k = ((int)blockIdx.y * kGateWaves + wave) * 32 + inner; k - inner < a.H; k += step) {
    const v4i w = load8(row, k, e < a.r.E && k < a.H);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int t = c * kTile + col;
      d[c] = mfma<T>(w, load8(static_cast<const T *>(a.x) + t * a.ldx, k, t < a.T && k < a.H), d[c]);
    }
  }
#pragma unroll
  for (int c = 0; c < C; ++c) part[wave][c][lane] = d[c];
  __syncthreads();
  for (int i = threadIdx.x; i < C * 64; i += 64 * kGateWaves) {
    const int c = i >> 6, l = i & 63, t = c * kTile + (l & 15);
    v4f s = part[0][c][l];
#pragma unroll
    for (int w = 1; w < kGateWaves; ++w) s += part[w][c][l];
    if (t >= a.T) continue;
    float *to = a.logits + ((int64_t)blockIdx.y * a.T + t) * a.r.E;
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      const int o = blockIdx.x * kTile + (l >> 4) * 4 + i4;
      if (o < a.r.E) to[o] = s[i4];
    }
  }
}

// ---------------------------------------------------------------- routing

template <int V>
__global__ __launch_bounds__(256) void few_route_kernel(Layer a) {
  __shared__ uint32_t scratch[4][kRouteScratch];
  const int wave = threadIdx.x >> 6, sub = lane_id();
  const int t = blockIdx.x * 4 + wave;
  const bool live = t < a.T;
  float x[V], b[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int e = sub * V + v;
    x[v] = -INFINITY;
    b[v] = 0.0f;
    if (e < a.r.E) {
      float s = 0.0f;
      for (int i = 0; i < a.splits; ++i) s += a.logits[((int64_t)i * a.T + (live ? t : 0)) * a.r.E + e];
      x[v] = clean_logit(s);
      if (a.bias) b[v] = a.bias[e];
    }
  }
  route_row<64, V>(a.r, x, b, sub, scratch[wave], live, a.ids + (int64_t)t * a.r.k, a.weights + (int64_t)t * a.r.k);
}

constexpr int kListThreads = 1024;

__global__ __launch_bounds__(kListThreads) void few_lists_kernel(Layer a) {
  __shared__ int count[TOPOEP_ROUTER_MAX_EXPERTS], first[TOPOEP_ROUTER_MAX_EXPERTS],
      place[TOPOEP_ROUTER_MAX_EXPERTS], tmp[kListThreads / 64 + 1];
  const int e = threadIdx.x, pairs = a.T * a.r.k;
  count[e] = 0;
  __syncthreads();
  for (int p = threadIdx.x; p < pairs; p += kListThreads) {
    const int id = a.ids[p], s = a.slot ? a.slot[id] : id;
    if ((unsigned)s < (unsigned)a.L) atomicAdd(&count[id], 1);
  }
  __syncthreads();
  const int n = count[e];
  first[e] = n;
  place[e] = n > 0;
  __syncthreads();
  const int total = block_excl_scan(first, TOPOEP_ROUTER_MAX_EXPERTS, tmp);
  const int active = block_excl_scan(place, TOPOEP_ROUTER_MAX_EXPERTS, tmp);
  if (n > 0) {
    a.lists.slot[place[e]] = a.slot ? a.slot[e] : e;
    a.lists.begin[place[e]] = first[e];
  }
  if (e == 0) {
    a.lists.active[0] = active;
    a.lists.begin[active] = total;
  }
  __syncthreads();
  for (int p = threadIdx.x; p < pairs; p += kListThreads) {
    const int id = a.ids[p], s = a.slot ? a.slot[id] : id;
    if ((unsigned)s < (unsigned)a.L) a.lists.pairs[atomicAdd(&first[id], 1)] = p;
  }
}

// ---------------------------------------------------------------- experts

constexpr int kUpWaves = 4;

// One wave's share of a tile of 16 gate and 16 up rows against C tiles of
// columns, `src[c]` the lane's column (null: none).
template <class T, int C>
__device__ inline void up_tile(const T *gate, const T *up, bool row, const T *const (&src)[kMaxCols], int H, int wave,
                               v4f (&g)[kMaxCols], v4f (&u)[kMaxCols]) {
  const int inner = (lane_id() >> 4) * 8;
#pragma unroll 4
  for (int k = wave * 32 + inner; k - inner < H; k += 32 * kUpWaves) {
    const bool in = k < H;
    const v4i wg = load8(gate, k, row && in), wu = load8(up, k, row && in);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const v4i b = load8(src[c], k, src[c] && in);
      g[c] = mfma<T>(wg, b, g[c]);
      u[c] = mfma<T>(wu, b, u[c]);
    }
  }
}

template <class T> __device__ inline float saturate(float f) { return f; }
template <> __device__ inline float saturate<F16>(float f) { return f > 65504.0f ? 65504.0f : f < -65504.0f ? -65504.0f : f; }

template <class T>
__global__ __launch_bounds__(64 * kUpWaves) void up_kernel(Layer a) {
  __shared__ v4f part[kUpWaves][2][kMaxCols][64];
  const int tiles = (a.I + kTile - 1) / kTile;
  const int n = blockIdx.x / tiles, tile = blockIdx.x % tiles;
  if (n >= a.lists.active[0]) return;
  const int lane = lane_id(), wave = threadIdx.x >> 6, col = lane & 15;
  const int begin = a.lists.begin[n], count = a.lists.begin[n + 1] - begin;
  const int i = tile * kTile + col;
  const T *gate = static_cast<const T *>(a.up) + ((int64_t)a.lists.slot[n] * 2 * a.I + i) * a.H;
  const T *up = gate + (int64_t)a.I * a.H;
  const T *src[kMaxCols];
  v4f g[kMaxCols] = {}, u[kMaxCols] = {};
#pragma unroll
  for (int c = 0; c < kMaxCols; ++c) {
    const int at = c * kTile + col;
    src[c] = at < count ? static_cast<const T *>(a.x) + a.lists.pairs[begin + at] / a.r.k * a.ldx : nullptr;
  }
  const int cols = (count + kTile - 1) / kTile;
  if (cols <= 1) up_tile<T, 1>(gate, up, i < a.I, src, a.H, wave, g, u);
  else if (cols <= 2) up_tile<T, 2>(gate, up, i < a.I, src, a.H, wave, g, u);
  else if (cols <= 4) up_tile<T, 4>(gate, up, i < a.I, src, a.H, wave, g, u);
  else up_tile<T, 8>(gate, up, i < a.I, src, a.H, wave, g, u);
#pragma unroll
  for (int c = 0; c < kMaxCols; ++c)
    if (c < cols) {
      part[wave][0][c][lane] = g[c];
      part[wave][1][c][lane] = u[c];
    }
  __syncthreads();
  for (int o = threadIdx.x; o < cols * 64; o += 64 * kUpWaves) {
    const int c = o >> 6, l = o & 63, at = c * kTile + (l & 15), row = tile * kTile + (l >> 4) * 4;
    v4f sg = part[0][0][c][l], su = part[0][1][c][l];
#pragma unroll
    for (int w = 1; w < kUpWaves; ++w) {
      sg += part[w][0][c][l];
      su += part[w][1][c][l];
    }
    if (at >= count || row >= a.I) continue;
    T h[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) h[j] = from_float<T>(saturate<T>(sg[j] * sigmoid(sg[j]) * su[j]));
    __builtin_memcpy(static_cast<T *>(a.hidden) + (int64_t)a.lists.pairs[begin + at] * a.I + row, h, sizeof(h));
  }
}

constexpr int kDownWaves = 8;

template <class T, int C>
__device__ inline void down_tile(const T *down, bool row, const T *const (&src)[kMaxCols], int lo, int hi,
                                 v4f (&d)[kMaxCols]) {
  const int inner = (lane_id() >> 4) * 8;
#pragma unroll 4
  for (int k = lo + inner; k - inner < hi; k += 32) {
    const v4i w = load8(down, k, row && k < hi);
#pragma unroll
    for (int c = 0; c < C; ++c) d[c] = mfma<T>(w, load8(src[c], k, src[c] && k < hi), d[c]);
  }
}

template <class T>
__global__ __launch_bounds__(64 * kDownWaves) void down_kernel(Layer a) {
  extern __shared__ v4f sums[];   // [kDownWaves][T][4]: 16 outputs of every token, by wave
  const int lane = lane_id(), wave = threadIdx.x >> 6, col = lane & 15;
  const v4f zero = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int i = threadIdx.x; i < kDownWaves * a.T * 4; i += 64 * kDownWaves) sums[i] = zero;
  __syncthreads();
  const int active = a.lists.active[0];
  // parts of I so that every wave has a unit
  int parts = 1;
  while (parts < kDownWaves && active * parts < kDownWaves) parts *= 2;
  const int len = ((a.I + parts - 1) / parts + 31) & ~31;
  const int o = blockIdx.x * kTile + col;
  v4f *mine = sums + wave * a.T * 4;
  for (int unit = wave; unit < active * parts; unit += kDownWaves) {
    const int n = unit / parts, lo = unit % parts * len, hi = lo + len < a.I ? lo + len : a.I;
    const int begin = a.lists.begin[n], count = a.lists.begin[n + 1] - begin;
    const T *down = static_cast<const T *>(a.down) + ((int64_t)a.lists.slot[n] * a.H + o) * a.I;
    const T *src[kMaxCols];
    int pair[kMaxCols];
    v4f d[kMaxCols] = {};
#pragma unroll
    for (int c = 0; c < kMaxCols; ++c) {
      const int at = c * kTile + col;
      pair[c] = at < count ? a.lists.pairs[begin + at] : -1;
      src[c] = at < count ? static_cast<const T *>(a.hidden) + (int64_t)pair[c] * a.I : nullptr;
    }
    const int cols = (count + kTile - 1) / kTile;
    if (cols <= 1) down_tile<T, 1>(down, o < a.H, src, lo, hi, d);
    else if (cols <= 2) down_tile<T, 2>(down, o < a.H, src, lo, hi, d);
    else if (cols <= 4) down_tile<T, 4>(down, o < a.H, src, lo, hi, d);
    else down_tile<T, 8>(down, o < a.H, src, lo, hi, d);
#pragma unroll
    for (int c = 0; c < kMaxCols; ++c)
      if (c < cols && pair[c] >= 0) {
        v4f *to = mine + pair[c] / a.r.k * 4 + (lane >> 4);
        *to = *to + a.weights[pair[c]] * d[c];
      }
    wave_sync();
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.T * 4; i += 64 * kDownWaves) {
    v4f s = sums[i];
#pragma unroll
    for (int w = 1; w < kDownWaves; ++w) s += sums[w * a.T * 4 + i];
    const int row = blockIdx.x * kTile + (i & 3) * 4;
    if (row >= a.H) continue;
    T out[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) out[j] = from_float<T>(s[j]);
    __builtin_memcpy(static_cast<T *>(a.out) + (int64_t)(i >> 2) * a.H + row, out, sizeof(out));
  }
}

// ---------------------------------------------------------------- host

int gate_splits(int E, int H) {
  const int tiles = (E + kTile - 1) / kTile, most = (H + 32 * kGateWaves - 1) / (32 * kGateWaves);
  int s = 1;
  while (s < 8 && s * 2 <= most && tiles * s < 128) s *= 2;
  return s;
}

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

struct Parts {
  size_t lists, pairs, logits, hidden, total;
};

Parts parts_of(const topoep_moe *m, const topoep_router *r, int T) {
  Parts p;
  const size_t E = (size_t)r->num_experts, pairs = (size_t)T * r->topk;
  size_t at = 256;   // control words
  p.lists = at;
  at += align256((2 * E + 2) * sizeof(int32_t));
  p.pairs = at;
  at += align256(pairs * sizeof(int32_t));
  p.logits = at;
  at += align256((size_t)gate_splits(r->num_experts, m->hidden) * T * E * sizeof(float));
  p.hidden = at;
  at += align256(pairs * m->inter * 2);
  p.total = at;
  return p;
}

int check_layer(const topoep_moe *m, const topoep_router *r, int32_t T) {
  if (!m || !r) return TOPOEP_EINVAL;
  if (m->hidden < 8 || (m->hidden & 7) || m->inter < 8 || (m->inter & 7) || m->local_experts < 1) return TOPOEP_EINVAL;
  if (m->hidden > 1 << 20 || m->inter > 1 << 20) return TOPOEP_EINVAL;
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

template <class T>
int enqueue(const Layer &a, hipStream_t st) {
  const int E = a.r.E, cols = (a.T + kTile - 1) / kTile;
  (void)hipGetLastError();
  const dim3 gg((E + kTile - 1) / kTile, a.splits), gb(64 * kGateWaves);
  if (cols <= 1) hipLaunchKernelGGL((gate_kernel<T, 1>), gg, gb, 0, st, a);
  else if (cols <= 2) hipLaunchKernelGGL((gate_kernel<T, 2>), gg, gb, 0, st, a);
  else if (cols <= 4) hipLaunchKernelGGL((gate_kernel<T, 4>), gg, gb, 0, st, a);
  else hipLaunchKernelGGL((gate_kernel<T, 8>), gg, gb, 0, st, a);
  if (!launched()) return TOPOEP_EHIP;
  const dim3 rg((a.T + 3) / 4), rb(256);
  if (E <= 64) hipLaunchKernelGGL((few_route_kernel<1>), rg, rb, 0, st, a);
  else if (E <= 128) hipLaunchKernelGGL((few_route_kernel<2>), rg, rb, 0, st, a);
  else if (E <= 256) hipLaunchKernelGGL((few_route_kernel<4>), rg, rb, 0, st, a);
  else if (E <= 512) hipLaunchKernelGGL((few_route_kernel<8>), rg, rb, 0, st, a);
  else hipLaunchKernelGGL((few_route_kernel<16>), rg, rb, 0, st, a);
  if (!launched()) return TOPOEP_EHIP;
  hipLaunchKernelGGL(few_lists_kernel, dim3(1), dim3(kListThreads), 0, st, a);
  if (!launched()) return TOPOEP_EHIP;
  // experts with pairs: at most one a pair, one an expert (several experts may share a slot)
  const int most = imin(a.T * a.r.k, E);
  const int tiles = (a.I + kTile - 1) / kTile;
  hipLaunchKernelGGL((up_kernel<T>), dim3((unsigned)most * tiles), dim3(64 * kUpWaves), 0, st, a);
  if (!launched()) return TOPOEP_EHIP;
  hipLaunchKernelGGL((down_kernel<T>), dim3((a.H + kTile - 1) / kTile), dim3(64 * kDownWaves),
                     kDownWaves * a.T * 4 * sizeof(v4f), st, a);
  return launched() ? TOPOEP_OK : TOPOEP_EHIP;
}

}  // namespace

extern "C" {

int topoep_moe_workspace_bytes(const topoep_moe *m, const topoep_router *r, int32_t T, size_t *bytes_out) {
  const int rc = check_layer(m, r, T);
  if (rc != TOPOEP_OK) return rc;
  if (!bytes_out) return TOPOEP_EINVAL;
  *bytes_out = parts_of(m, r, T).total;
  return TOPOEP_OK;
}

int topoep_moe_few(const topoep_moe *m, const topoep_router *r, const void *x, int64_t ldx, int32_t T,
                   const void *gate, const float *bias, const int32_t *expert_slot, const void *up, const void *down,
                   void *out, int32_t *ids, float *weights, void *workspace, size_t workspace_bytes, void *stream) {
  const int rc = check_layer(m, r, T);
  if (rc != TOPOEP_OK) return rc;
  if (T == 0) return TOPOEP_OK;
  if (!x || !gate || !up || !down || !out || !ids || !weights || !workspace) return TOPOEP_EINVAL;
  if (ldx < m->hidden || (ldx & 7) || ldx > (int64_t)1 << 40) return TOPOEP_EINVAL;
  if (!aligned16(x) || !aligned16(gate) || !aligned16(up) || !aligned16(down) || !aligned16(out)) return TOPOEP_EINVAL;
  const Parts p = parts_of(m, r, T);
  if ((reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < p.total) return TOPOEP_EWORKSPACE;
  char *ws = static_cast<char *>(workspace);
  Layer a;
  a.r = router_args(r);
  a.T = T;
  a.H = m->hidden;
  a.I = m->inter;
  a.L = m->local_experts;
  a.splits = gate_splits(r->num_experts, m->hidden);
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
  int32_t *lists = reinterpret_cast<int32_t *>(ws + p.lists);
  a.lists.active = lists;
  a.lists.slot = lists + 1;
  a.lists.begin = lists + 1 + r->num_experts;
  a.lists.pairs = reinterpret_cast<int32_t *>(ws + p.pairs);
  hipStream_t st = static_cast<hipStream_t>(stream);
  return m->dtype == TOPOEP_BF16 ? enqueue<Bf16>(a, st) : enqueue<F16>(a, st);
}

}  // extern "C"
