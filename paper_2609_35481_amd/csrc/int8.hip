// Products in 8-bit integers on gfx950: rows quantised with a scale each, and their
// products with weights that have a scale for each channel, for all rows or the
// rows of every expert.
//
// The sums are whole numbers, exact in 32 bits; scales (and the activation of a gated
// block) are the epilogue, in 32 bits, rounded once.
#include "few.h"
#include "spans.h"
#include "topoep_ffn.h"

namespace {

using namespace topoep_dev;

// ---------------------------------------------------------------- quantisation

struct Quant {
  const void *x;
  int64_t ldx;
  int M, K;
  int8_t *q;
  float *scale;
};

// x / s to the nearest integer, ties to even, at most 127 in magnitude.  The quotient rounded to 32 bits
// can lie on the border of two integers where the quotient itself does not: then the sign of the
// remainder, which fma keeps, tells on which side it is.
__device__ inline int nearest(float x, float s) {
  const float t = x / s;
  float r = rintf(t);
  if (fabsf(t - r) == 0.5f) {
    const float rest = fmaf(-t, s, x);
    r = rest > 0.0f ? t + 0.5f : rest < 0.0f ? t - 0.5f : r;
  }
  return (int)fminf(fmaxf(r, -127.0f), 127.0f);
}

// What a row's elements are divided by.  A quotient is first taken as a product with the reciprocal, off by
// at most 127 (2^-24 + 2^-24) = 1.6 10^-5; only one that near to a border is divided (8192 rows of 14336 in
// 16 bits: 114 us with a division each, 64 so; 5.5 TB/s).
struct Divisor {
  float scale, inverse, lift;
  bool plain, quick;
  __device__ explicit Divisor(uint32_t top) {   // the largest magnitude's bits
    scale = __uint_as_float(top) / 127.0f;
    plain = scale > 0.0f && top < 0x7F800000u;
    quick = scale >= 0x1p-100f;
    // (both times 2^64 where a remainder could be too small for 32 bits)
    lift = quick ? 1.0f : 0x1p64f;
    inverse = 1.0f / scale;
  }
  template <int N>
  __device__ void divide(const float (&v)[N], int8_t (&q)[N]) const {
    bool near = !quick;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float t = v[e] * inverse, r = rintf(t);
      near |= fabsf(t - r) > 0.5f - 0x1p-14f;
      q[e] = plain ? (int8_t)(int)r : (int8_t)0;
    }
    if (near && plain)
#pragma unroll
      for (int e = 0; e < N; ++e) q[e] = (int8_t)nearest(v[e] * lift, scale * lift);
  }
};

// Of magnitudes as unsigned words the largest: NaN's lie above infinity's.
__device__ inline uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// Over a row's W waves.
template <int W>
__device__ inline uint32_t most_of(uint32_t top) {
  __shared__ uint32_t most[4];
  top = row_max<64>(top);
  if (W > 1) {
    __syncthreads();   // the row before
    most[threadIdx.x >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) top = max(top, most[w]);
  }
  return top;
}

// W waves a row, 4 / W rows a workgroup, 16 bytes a lane and load (x and its rows at multiples of that, K of
// the elements in it); V loads a lane stay in registers, what is behind them is read again.
template <class T, int W, int V>
__global__ __launch_bounds__(256) void quantize_kernel(Quant a) {
  constexpr int N = 16 / (int)sizeof(T), kAll = 64 * W * N;
  const int wave = uniform_i32(threadIdx.x >> 6), lane = threadIdx.x % (64 * W);
  const int K = a.K;
  for (int64_t m = (int64_t)blockIdx.x * (4 / W) + wave / W; m < a.M; m += (int64_t)gridDim.x * (4 / W)) {
    const T *row = static_cast<const T *>(a.x) + m * a.ldx;
    const auto load = [&](int k) { return *reinterpret_cast<const v4i *>(row + k); };
    const auto floats = [](v4i r, float (&v)[N]) {
      T e[N];
      __builtin_memcpy(e, &r, 16);
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = to_float(e[i]);
    };
    uint32_t top = 0;
    const auto look = [&](v4i r) {
      float v[N];
      floats(r, v);
#pragma unroll
      for (int i = 0; i < N; ++i) top = max(top, magnitude(v[i]));
    };
    v4i held[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int k = i * kAll + lane * N;
      held[i] = k < K ? load(k) : v4i{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < V; ++i) look(held[i]);
    for (int k = V * kAll + lane * N; k < K; k += kAll) look(load(k));
    const Divisor d(most_of<W>(top));
    if (lane == 0) a.scale[m] = d.scale;
    const auto store = [&](int k, v4i r) {
      float v[N];
      int8_t q[N];
      floats(r, v);
      d.divide(v, q);
      __builtin_memcpy(a.q + m * K + k, q, N);
    };
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i * kAll + lane * N < K) store(i * kAll + lane * N, held[i]);
    for (int k = V * kAll + lane * N; k < K; k += kAll) store(k, load(k));
  }
}

// Rows of any alignment: a workgroup a row, an element a lane.
template <class T>
__global__ __launch_bounds__(256) void quantize_any_kernel(Quant a) {
  for (int64_t m = blockIdx.x; m < a.M; m += gridDim.x) {
    const T *row = static_cast<const T *>(a.x) + m * a.ldx;
    uint32_t top = 0;
    for (int k = threadIdx.x; k < a.K; k += 256) top = max(top, magnitude(to_float(row[k])));
    const Divisor d(most_of<4>(top));
    if (threadIdx.x == 0) a.scale[m] = d.scale;
    for (int k = threadIdx.x; k < a.K; k += 256) {
      const float v[1] = {to_float(row[k])};
      int8_t q[1];
      d.divide(v, q);
      a.q[m * a.K + k] = q[0];
    }
  }
}

// ---------------------------------------------------------------- product

struct Int8 {
  int M, N, K, G, No;         // No: columns of out
  const int8_t *q, *w;
  int64_t ldq;
  const float *scale, *ws;
  const int32_t *offsets;
  void *out;
  int type;
  bool keep;
  int parts;
  int32_t *sums;              // [parts, M, N], parts > 1
};

__device__ inline void store1(void *out, int type, int64_t at, float v) {
  if (type == TOPOEP_F32) static_cast<float *>(out)[at] = v;
  else if (type == TOPOEP_BF16) static_cast<Bf16 *>(out)[at] = from_float<Bf16>(v);
  else static_cast<F16 *>(out)[at] = from_float<F16>(v);
}

// A sum as a float.  2^31, which 2^17 products of -128 and -128 reach and nothing else does, is in 32 bits -2^31, which
// no sum is: the least is -127 * 128 * 2^17.  (Top: of that many.)
constexpr int kTop = 1 << 17;
template <bool Top = true>
__device__ inline float of_sum(int s) { return Top && s == INT32_MIN ? 0x1p31f : (float)s; }

// Four neighbours of a row of `n`, from column c on.
__device__ inline void store_row(void *out, int type, int64_t row, int n, int c, v4f v) {
  const int64_t at = row * n + c;
  if ((n & 3) == 0) {
    if (type == TOPOEP_F32) store4<float>(out, at, v);
    else if (type == TOPOEP_BF16) store4<Bf16>(out, at, v);
    else store4<F16>(out, at, v);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < n) store1(out, type, at + e, v[e]);
  }
}

// Rows behind the groups' last are zeros.
__device__ inline void clear_rest(const Int8 &a) {
  if (!a.offsets || a.keep) return;
  const int64_t from = (int64_t)imin(imax(a.offsets[a.G], 0), a.M) * a.No;
  for (int64_t i = from + (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < (int64_t)a.M * a.No;
       i += (int64_t)gridDim.x * blockDim.x)
    store1(a.out, a.type, i, 0.0f);
}

template <class S, bool Gated>
__global__ __launch_bounds__(S::kThreads, 2) void int8_kernel(Int8 a) {
  TOPOEP_STAGES(S);
  constexpr int kCols = Gated ? S::BP / 2 : S::BP, kTiles = Gated ? S::TP / 2 : S::TP;   // columns of out, a wave's tiles of them
  const int np = (a.No + kCols - 1) / kCols;
  clear_rest(a);
  Span s;
  const int nq = spans<S::BQ>(a.offsets, a.M, a.G, -1, s);
  const int each = ((a.K + a.parts - 1) / a.parts + S::kStage - 1) / S::kStage * S::kStage;
  for (int t = blockIdx.x; t < nq * np * a.parts; t += gridDim.x) {
    const Me me;
    const int part = t / (nq * np), k0 = imin(part * each, a.K);
    const int tp = find_tile<S::BQ>(a.offsets, a.M, a.G, t - part * nq * np, np, nq * np, s);
    ByRows<I8, S::BP, S::kWaves> p;
    ByRows<I8, S::BQ, S::kWaves> q;
    const char *w = reinterpret_cast<const char *>(a.w) + (int64_t)s.group * a.N * a.K + k0;
    p.start(me, [&](int r) {
      const int in = r % (S::TP * 16), half = Gated ? in / (kTiles * 16) : 0;
      const int c = tp * kCols + r / (S::TP * 16) * (kTiles * 16) + in % (kTiles * 16);
      return w + (int64_t)(half * a.No + imin(c, a.No - 1)) * a.K;
    });
    q.start(me, [&](int r) { return reinterpret_cast<const char *>(a.q) + imin(s.first + r, s.end - 1) * a.ldq + k0; });
    typename S::Sum d[S::TP][S::TQ] = {};
    __syncthreads();
    multiply<S>(p, q, me, imin(each, a.K - k0), start_of<S>(imin(each, a.K - k0), s.group), lds, d);
    if (a.parts > 1) {
#pragma unroll
      for (int j = 0; j < S::TQ; ++j) {
        const int m = s.first + (me.wave / S::NP * S::TQ + j) * 16 + (me.lane & 15);
        if (m >= s.end) continue;
#pragma unroll
        for (int i = 0; i < S::TP; ++i) {
          const int c = tp * kCols + (me.wave % S::NP * kTiles + i % kTiles) * 16 + (me.lane >> 4) * 4;
          if (c < a.No) *reinterpret_cast<v4i *>(a.sums + ((int64_t)part * a.M + m) * a.N + i / kTiles * a.No + c) = d[i][j];
        }
      }
      continue;
    }
    const float *ws = a.ws + (int64_t)s.group * a.N;
    const auto finish = [&](auto top) {
#pragma unroll
      for (int i = 0; i < kTiles; ++i) {
        const int c = tp * kCols + (me.wave % S::NP * kTiles + i) * 16 + (me.lane >> 4) * 4;
        if (c >= a.No) continue;
        float w0[4], w1[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          w0[e] = ws[imin(c + e, a.No - 1)];
          if (Gated) w1[e] = ws[a.No + imin(c + e, a.No - 1)];
        }
#pragma unroll
        for (int j = 0; j < S::TQ; ++j) {
          const int m = s.first + (me.wave / S::NP * S::TQ + j) * 16 + (me.lane & 15);
          if (m >= s.end) continue;
          const float scale = a.scale[m];
          v4f v;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            v[e] = of_sum<decltype(top)::value>(d[i][j][e]) * scale * w0[e];
            if (Gated) {
              const float u = of_sum<decltype(top)::value>(d[i + kTiles * (Gated ? 1 : 0)][j][e]) * scale * w1[e];
              v[e] = v[e] * sigmoid(v[e]) * u;
            }
          }
          store_row(a.out, a.type, m, a.No, c, v);
        }
      }
    };
    // (asked of every sum, 8192 rows by 4096 x 14336 take 432 us instead of 428)
    if (a.K < kTop) finish(std::false_type());
    else finish(std::true_type());
  }
}

// The parts' sums, and what a product's epilogue makes of them; a workgroup has a row.
template <bool Gated>
__global__ __launch_bounds__(256) void parts_kernel(Int8 a) {
  const int m = blockIdx.x;
  int group = 0;
  if (a.offsets) {
    int first = 0, end = 0;
    bool found = false;
    for (int g0 = 0; g0 < a.G && !found; g0 += 64) {   // (the same in every lane)
      const int g = g0 + lane_id();
      if (g < a.G) rows_of(a.offsets, a.M, g, first, end);
      const uint64_t has = __ballot(g < a.G && first <= m && m < end);
      found = has != 0;
      if (found) group = g0 + __ffsll((unsigned long long)has) - 1;
    }
    if (!found) return;
  }
  const float scale = a.scale[m], *ws = a.ws + (int64_t)group * a.N;
  for (int c = (blockIdx.y * 256 + threadIdx.x) * 4; c < a.No; c += gridDim.y * 1024) {
    const auto sum = [&](int at) {
      typedef uint32_t v4u __attribute__((ext_vector_type(4)));
      v4u s = *reinterpret_cast<const v4u *>(a.sums + (int64_t)m * a.N + at);
      for (int p = 1; p < a.parts; ++p) s += *reinterpret_cast<const v4u *>(a.sums + ((int64_t)p * a.M + m) * a.N + at);
      v4f v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = of_sum((int)s[e]) * scale * ws[at + e];
      return v;
    };
    v4f v = sum(c);
    if (Gated) {
      const v4f u = sum(a.No + c);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = v[e] * sigmoid(v[e]) * u[e];
    }
    store_row(a.out, a.type, m, a.No, c, v);
  }
}

// A few rows a group: 16 rows of weights (8 columns' gate and up rows) against up to 4 C rows.
template <bool Gated, int C, int KS>
__global__ __launch_bounds__(64 * few_waves(KS), few_per_simd(C)) void few_int8_kernel(Int8 a) {
  __shared__ FewSums<int, C, KS> lds;
  constexpr int kCols = Gated ? 8 : 16;
  const int np = (a.No + kCols - 1) / kCols;
  clear_rest(a);
  Span s;
  const int nq = spans<4 * C>(a.offsets, a.M, a.G, -1, s);
  for (int t = few_first<KS>(); t < nq * np; t += few_next<KS>()) {
    const int tp = t / nq, c0 = tp * kCols;
    spans<4 * C>(a.offsets, a.M, a.G, t - tp * nq, s);
    const char *w = reinterpret_cast<const char *>(a.w) + (int64_t)s.group * a.N * a.K;
    few_product<I8, C, KS>(
        [&](int r) { return w + (int64_t)((Gated ? r >> 3 : 0) * a.No + imin(c0 + r % kCols, a.No - 1)) * a.K; },
        [&](int c) { return reinterpret_cast<const char *>(a.q) + (s.first + c) * a.ldq; },
        imin(s.end - s.first, 4 * C), a.K, lds, kCols, [&](int r, int c, int first, int second) {
          if (c0 + r >= a.No) return;
          const float *ws = a.ws + (int64_t)s.group * a.N + c0 + r;
          const float scale = a.scale[s.first + c];
          float v = of_sum(first) * scale * ws[0];
          if (Gated) v = v * sigmoid(v) * (of_sum(second) * scale * ws[a.No]);
          store1(a.out, a.type, (int64_t)(s.first + c) * a.No + c0 + r, v);
        });
  }
}

// ---------------------------------------------------------------- host

bool launched() { return hipGetLastError() == hipSuccess; }
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

int check(const topoep_int8 *p, int32_t M) {
  if (!p || M < 0 || M > 1 << 30) return TOPOEP_EINVAL;   // (a tile behind the last row is counted in 32 bits)
  if (p->n < 1 || p->n > 1 << 20 || p->k < 16 || (p->k & 15) || p->k > 1 << 17 || p->groups < 1) return TOPOEP_EINVAL;
  if (p->gated && (p->n & 1)) return TOPOEP_EINVAL;
  if (p->out_dtype < TOPOEP_F32 || p->out_dtype > TOPOEP_F16) return TOPOEP_EINVAL;
  return p->groups > TOPOEP_FFN_MAX_EXPERTS ? TOPOEP_ELIMIT : TOPOEP_OK;
}

typedef Shape<I8, 256, 256, 2, 4, false, false, 2> Large;
typedef Shape<I8, 128, 128, 2, 2, false, false, 4> Small;

int columns_of(const topoep_int8 *p) { return p->gated ? p->n / 2 : p->n; }
// Tiles of 128 x 128, about.
int64_t small_tiles(const topoep_int8 *p, int M) {
  return likely_spans(p->groups > 1, M, p->groups, 128) * ceil_of(columns_of(p), p->gated ? 64 : 128);
}
// A few rows a group, 16 and fewer: the weights' bytes count, not the tiles.  Up to 64 also where a
// product is small (rows times weights of 512 MiB: 32 rows, 4096 x 4096: 14.9 against 17.1 us, 64: 24.3 and 18.3).
bool few_rows(const topoep_int8 *p, int M) {
  const int64_t groups = imin(p->groups, M);
  return M <= 16 * groups || (M <= 64 * groups && (double)M * groups * p->n * p->k <= 0x1p29);
}
// Workgroups that share a tile's inner axis (their sums are at most 256 MiB).
int parts_of(const topoep_int8 *p, int M) {
  if (M == 0 || few_rows(p, M) || columns_of(p) % 4) return 1;
  const int parts = topoep_dev::parts_of(small_tiles(p, M), p->k / 128, 8);
  return (int64_t)parts * M * p->n > (int64_t)1 << 26 ? 1 : parts;
}
size_t need(const topoep_int8 *p, int M) {
  const int parts = parts_of(p, M);
  return parts > 1 ? ((size_t)parts * M * p->n * sizeof(int32_t) + 255) & ~(size_t)255 : 0;
}

template <class S, bool Gated>
int enqueue(const Int8 &a, hipStream_t st) {
  const int cols = Gated ? S::BP / 2 : S::BP;
  const int64_t tiles = most_spans<S::BQ>(a.offsets, a.M, a.G) * ((a.No + cols - 1) / cols) * a.parts;
  hipLaunchKernelGGL((int8_kernel<S, Gated>), dim3(grid_of<S>(tiles)), dim3(S::kThreads), 0, st, a);
  if (!launched()) return TOPOEP_EHIP;
  if (a.parts == 1) return TOPOEP_OK;
  hipLaunchKernelGGL((parts_kernel<Gated>), dim3(a.M, imin((a.No + 1023) / 1024, 64)), dim3(256), 0, st, a);
  return launched() ? TOPOEP_OK : TOPOEP_EHIP;
}

template <class T>
int enqueue_quantize(const Quant &a, hipStream_t st) {
  constexpr int N = 16 / (int)sizeof(T);
  const bool wide = aligned16(a.x) && a.ldx % N == 0 && a.K % N == 0 && reinterpret_cast<uintptr_t>(a.q) % N == 0;
  const dim3 rows(imin(a.M, 1 << 20)), fours(imin((a.M - 1) / 4 + 1, 1 << 20));
  // a wave a row where that keeps the row in registers
  if (!wide) hipLaunchKernelGGL((quantize_any_kernel<T>), rows, dim3(256), 0, st, a);
  else if (a.K <= 64 * N * 4 && a.M > 1) hipLaunchKernelGGL((quantize_kernel<T, 1, 4>), fours, dim3(256), 0, st, a);
  else if (a.K <= 256 * N * 4) hipLaunchKernelGGL((quantize_kernel<T, 4, 4>), rows, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((quantize_kernel<T, 4, 8>), rows, dim3(256), 0, st, a);
  return launched() ? TOPOEP_OK : TOPOEP_EHIP;
}

}  // namespace

extern "C" {

int topoep_quantize(const void *x, int32_t dtype, int64_t ldx, int32_t M, int32_t K, int8_t *q, float *scale,
                    void *stream) {
  if (M < 0 || K < 1 || K > 1 << 30 || ldx < K || ldx > (int64_t)1 << 40 || dtype < TOPOEP_F32 || dtype > TOPOEP_F16) return TOPOEP_EINVAL;
  if (M == 0) return TOPOEP_OK;
  const int size = dtype == TOPOEP_F32 ? 4 : 2;
  if (!x || !q || !scale || reinterpret_cast<uintptr_t>(x) % size || reinterpret_cast<uintptr_t>(scale) % 4) return TOPOEP_EINVAL;
  const Quant a{x, ldx, M, K, q, scale};
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (dtype == TOPOEP_F32) return enqueue_quantize<float>(a, st);
  return dtype == TOPOEP_BF16 ? enqueue_quantize<Bf16>(a, st) : enqueue_quantize<F16>(a, st);
}

int topoep_matmul_int8_workspace_bytes(const topoep_int8 *p, int32_t M, size_t *bytes_out) {
  const int rc = check(p, M);
  if (rc != TOPOEP_OK) return rc;
  if (!bytes_out) return TOPOEP_EINVAL;
  *bytes_out = need(p, M);
  return TOPOEP_OK;
}

int topoep_matmul_int8(const topoep_int8 *p, const int8_t *q, int64_t ldq, const float *scale, int32_t M,
                       const int32_t *offsets, int32_t keep_rest, const int8_t *w, const float *w_scale, void *out,
                       void *workspace, size_t workspace_bytes, void *stream) {
  const int rc = check(p, M);
  if (rc != TOPOEP_OK) return rc;
  if (M == 0) return TOPOEP_OK;
  if (!q || !scale || !w || !w_scale || !out || (!offsets && p->groups != 1)) return TOPOEP_EINVAL;
  if (ldq < p->k || (ldq & 15) || ldq > (int64_t)1 << 40 || !aligned16(q) || !aligned16(w) || !aligned16(out)) return TOPOEP_EINVAL;
  if ((reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < need(p, M)) return TOPOEP_EWORKSPACE;
  if (!workspace && need(p, M)) return TOPOEP_EINVAL;
  Int8 a = {};
  a.M = M, a.N = p->n, a.K = p->k, a.G = p->groups, a.No = p->gated ? p->n / 2 : p->n;
  a.q = q, a.w = w, a.ldq = ldq, a.scale = scale, a.ws = w_scale, a.offsets = offsets;
  a.out = out, a.type = p->out_dtype, a.keep = keep_rest != 0;
  a.parts = parts_of(p, M), a.sums = static_cast<int32_t *>(workspace);
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (few_rows(p, M)) {
    const int64_t groups = imin(a.G, M);
    const int64_t np = (a.No + (p->gated ? 7 : 15)) / (p->gated ? 8 : 16);
    // (groups differ: twice the mean is what most have at most)
    few_shape((M + groups - 1) / groups * (groups > 1 ? 2 : 1), groups * np, [&](auto c, auto ks) {
      constexpr int C = decltype(c)::value, KS = decltype(ks)::value;
      const dim3 grid = few_grid<KS>(most_spans<4 * C>(offsets, M, a.G) * np), block(64 * few_waves(KS));
      if (p->gated) hipLaunchKernelGGL((few_int8_kernel<true, C, KS>), grid, block, 0, st, a);
      else hipLaunchKernelGGL((few_int8_kernel<false, C, KS>), grid, block, 0, st, a);
    });
    return launched() ? TOPOEP_OK : TOPOEP_EHIP;
  }
  const int per = p->gated ? 128 : 256;
  if (a.parts == 1 && (!offsets || M >= 1024 * (int64_t)a.G) && large_tiles(likely_spans(offsets != nullptr, M, a.G, 256) * ((a.No + per - 1) / per),
                  likely_spans(offsets != nullptr, M, a.G, 128) * ((a.No + per / 2 - 1) / (per / 2))))
    return p->gated ? enqueue<Large, true>(a, st) : enqueue<Large, false>(a, st);
  return p->gated ? enqueue<Small, true>(a, st) : enqueue<Small, false>(a, st);
}

}  // extern "C"
