// The global gradient norm over many tensors and the clip on gfx950.
//
// The tensors' addresses and sizes travel as kernel arguments, kSet tensors a
// launch, so a call copies nothing to the device and may be captured.  A
// launch's elements are cut into chunks of kChunk elements that do not cross
// tensors, and workgroup b takes chunks b, b + grid, ...  The norm kernel
// leaves one 64-bit partial a workgroup; the reader sums them in a fixed
// order.  Squares are formed and summed in 64 bits: the square of any 32-bit
// number is exact there and neither overflows nor vanishes.
#include "router.h"

namespace {

using namespace topoep_dev;

constexpr int kThreads = 256;
constexpr int kSet = 112;          // tensors a launch takes (3.6 KB of arguments)
constexpr int64_t kChunk = 16384;  // elements of one step of a workgroup
constexpr int kBlocks = 1024;      // workgroups, and partials, a launch has at most
// elements a set may have (2^26 chunks: chunk numbers are 32-bit words)
constexpr int64_t kMostElements = (int64_t)1 << 40;

struct Set {
  int count, chunks;
  int first[kSet];     // chunks before tensor i
  int types[kSet];     // dtype | out_dtype << 4
  const void *grad[kSet];
  void *out[kSet];
  int64_t n[kSet];
};

// The tensor that holds a chunk (the last with first <= chunk).
__device__ inline int tensor_of(const Set &s, int chunk) {
  int lo = 0, hi = s.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (s.first[mid] <= chunk) lo = mid; else hi = mid - 1;
  }
  return lo;
}

struct Sum {      // the 2-norm's
  double v = 0.0;
  static __device__ double root(double v) { return sqrt(v); }
  __device__ void add(float g) { v = fma((double)g, (double)g, v); }
  __device__ void join(double o) { v += o; }
};
struct Largest {  // the largest magnitude; NaN wins
  double v = 0.0;
  static __device__ double root(double v) { return v; }
  __device__ void add(float g) { join(fabs((double)g)); }
  __device__ void join(double o) { v = o > v || o != o ? o : v; }
};

// Joins the workgroup's values; valid in thread 0.
template <class R>
__device__ inline double join_block(R r, double *lds) {
  for (int d = 32; d > 0; d >>= 1) r.join(__shfl_xor(r.v, d));
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = r.v;
  __syncthreads();
  for (int w = 1; w < (int)(blockDim.x >> 6); ++w) r.join(lds[w]);
  return r.v;
}

// Elements a thread loads at once (16 bytes).
template <class T> constexpr int kWide = 16 / sizeof(T);

template <class T, class R>
__device__ inline void reduce_chunk(const T *g, int64_t n, R &r) {
  constexpr int W = kWide<T>, U = 4;
  const int64_t step = (int64_t)kThreads * W;
  int64_t i = (int64_t)threadIdx.x * W;
  for (; i + (U - 1) * step + W <= n; i += U * step) {
    T raw[U][W];
#pragma unroll
    for (int u = 0; u < U; ++u) __builtin_memcpy(raw[u], g + i + u * step, 16);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int w = 0; w < W; ++w) r.add(to_float(raw[u][w]));
  }
  for (; i < n; i += step) {
#pragma unroll
    for (int w = 0; w < W; ++w)
      if (i + w < n) r.add(to_float(g[i + w]));
  }
}

template <class R>
__global__ __launch_bounds__(kThreads) void grad_norm_kernel(Set s, double *partials) {
  __shared__ double lds[kThreads / 64];
  R r;
  for (int c = blockIdx.x; c < s.chunks; c += gridDim.x) {
    const int i = tensor_of(s, c);
    const int64_t at = (int64_t)(c - s.first[i]) * kChunk;
    const int64_t n = s.n[i] - at < kChunk ? s.n[i] - at : kChunk;
    switch (s.types[i] & 15) {
      case TOPOEP_F32: reduce_chunk(static_cast<const float *>(s.grad[i]) + at, n, r); break;
      case TOPOEP_BF16: reduce_chunk(static_cast<const Bf16 *>(s.grad[i]) + at, n, r); break;
      default: reduce_chunk(static_cast<const F16 *>(s.grad[i]) + at, n, r); break;
    }
  }
  const double v = join_block(r, lds);
  if (threadIdx.x == 0) partials[blockIdx.x] = v;
}

// The norm of `count` partials; the same value in every thread.
template <class R>
__device__ inline float norm_of(const double *partials, int count, float scale, double *lds) {
  R r;
  for (int i = threadIdx.x; i < count; i += kThreads) r.join(partials[i]);
  const double v = join_block(r, lds);
  if (threadIdx.x == 0) lds[0] = (double)scale * R::root(v);
  __syncthreads();
  return (float)lds[0];
}

template <class R>
__global__ __launch_bounds__(kThreads) void grad_finish_kernel(const double *partials, int count, float scale,
                                                               float *norm) {
  __shared__ double lds[kThreads / 64];
  const float v = norm_of<R>(partials, count, scale, lds);
  if (threadIdx.x == 0) *norm = v;
}

template <class T, class O>
__device__ inline void scale_chunk(const T *g, O *out, int64_t n, float f) {
  constexpr int W = kWide<T>, U = 4;
  const int64_t step = (int64_t)kThreads * W;
  int64_t i = (int64_t)threadIdx.x * W;
  for (; i + (U - 1) * step + W <= n; i += U * step) {
    T raw[U][W];
#pragma unroll
    for (int u = 0; u < U; ++u) __builtin_memcpy(raw[u], g + i + u * step, 16);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      O to[W];
#pragma unroll
      for (int w = 0; w < W; ++w) to[w] = from_float<O>(to_float(raw[u][w]) * f);
      __builtin_memcpy(out + i + u * step, to, sizeof(to));
    }
  }
  for (; i < n; i += step) {
#pragma unroll
    for (int w = 0; w < W; ++w)
      if (i + w < n) out[i + w] = from_float<O>(to_float(g[i + w]) * f);
  }
}

template <class T>
__device__ inline void scale_chunk_to(const T *g, void *out, int type, int64_t at, int64_t n, float f) {
  switch (type) {
    case TOPOEP_F32: scale_chunk(g + at, static_cast<float *>(out) + at, n, f); break;
    case TOPOEP_BF16: scale_chunk(g + at, static_cast<Bf16 *>(out) + at, n, f); break;
    default: scale_chunk(g + at, static_cast<F16 *>(out) + at, n, f); break;
  }
}

struct Clip {
  const double *partials;
  int count;              // of partials; 0 = given
  float scale, max_norm;
  const float *given;
  float *norm;            // or null
};

template <class R>
__global__ __launch_bounds__(kThreads) void clip_kernel(Set s, Clip c) {
  __shared__ double lds[kThreads / 64];
  const float norm = c.given ? *c.given : norm_of<R>(c.partials, c.count, c.scale, lds);
  if (c.norm && blockIdx.x == 0 && threadIdx.x == 0) *c.norm = norm;
  if (!(norm - norm == 0.0f)) return;
  const float f = c.scale * fminf(1.0f, c.max_norm / (norm + 1e-6f));
  // the chunks that the norm read last come first: the caches may still hold them
  for (int i0 = s.chunks - 1 - (int)blockIdx.x; i0 >= 0; i0 -= gridDim.x) {
    const int i = tensor_of(s, i0);
    if (f == 1.0f && s.out[i] == s.grad[i]) continue;
    const int64_t at = (int64_t)(i0 - s.first[i]) * kChunk;
    const int64_t n = s.n[i] - at < kChunk ? s.n[i] - at : kChunk;
    const int to = s.types[i] >> 4;
    switch (s.types[i] & 15) {
      case TOPOEP_F32: scale_chunk_to(static_cast<const float *>(s.grad[i]), s.out[i], to, at, n, f); break;
      case TOPOEP_BF16: scale_chunk_to(static_cast<const Bf16 *>(s.grad[i]), s.out[i], to, at, n, f); break;
      default: scale_chunk_to(static_cast<const F16 *>(s.grad[i]), s.out[i], to, at, n, f); break;
    }
  }
}

// Walks the set in launches of kSet tensors: fills each one's arguments and
// calls go(set, index of the launch).
template <class F>
int each_set(const topoep_grad *grads, int count, const F &go) {
  Set s;
  int at = 0, launch = 0;
  do {
    s.count = 0;
    int64_t chunks = 0;
    for (; at < count && s.count < kSet; ++at) {
      const topoep_grad &g = grads[at];
      const int64_t more = (g.n + kChunk - 1) / kChunk;
      if (more == 0) continue;
      const int i = s.count++;
      s.first[i] = (int)chunks;
      s.types[i] = g.dtype | g.out_dtype << 4;
      s.grad[i] = g.grad;
      s.out[i] = g.out;
      s.n[i] = g.n;
      chunks += more;
    }
    s.chunks = (int)chunks;
    const int rc = go(s, launch++);
    if (rc != TOPOEP_OK) return rc;
  } while (at < count);
  return TOPOEP_OK;
}

int grid_of(const Set &s) { return s.chunks < kBlocks ? (s.chunks > 0 ? s.chunks : 1) : kBlocks; }

int check_set(const topoep_grad *grads, int32_t count, bool out) {
  if (count < 0 || (count > 0 && !grads)) return TOPOEP_EINVAL;
  int64_t left = kMostElements;
  for (int i = 0; i < count; ++i) {
    const topoep_grad &g = grads[i];
    if (g.n < 0 || g.n > left || g.dtype < TOPOEP_F32 || g.dtype > TOPOEP_F16) return TOPOEP_EINVAL;
    left -= g.n;
    if (g.n == 0) continue;
    if (!g.grad || (reinterpret_cast<uintptr_t>(g.grad) & (g.dtype == TOPOEP_F32 ? 3 : 1))) return TOPOEP_EINVAL;
    if (!out) continue;
    if (g.out_dtype < TOPOEP_F32 || g.out_dtype > TOPOEP_F16 || !g.out) return TOPOEP_EINVAL;
    if (reinterpret_cast<uintptr_t>(g.out) & (g.out_dtype == TOPOEP_F32 ? 3 : 1)) return TOPOEP_EINVAL;
    if (g.out == g.grad && g.out_dtype != g.dtype) return TOPOEP_EINVAL;
  }
  return TOPOEP_OK;
}

// kBlocks partials a launch, and a launch per kSet tensors.
size_t partials_bytes(int32_t count) { return ((size_t)count / kSet + 1) * kBlocks * sizeof(double); }

int check_workspace(const void *ws, size_t bytes, int32_t count) {
  if (!ws) return TOPOEP_EINVAL;
  size_t need = 0;
  const int rc = topoep_grads_workspace_bytes(count, &need);
  if (rc != TOPOEP_OK) return rc;
  return (reinterpret_cast<uintptr_t>(ws) & 255) || bytes < need ? TOPOEP_EWORKSPACE : TOPOEP_OK;
}

bool finite_scale(float s) { return s >= 0.0f && s - s == 0.0f; }

// Enqueues the partials; returns their number in *partials.
int enqueue_partials(const topoep_grad *grads, int count, int ord, double *ws, hipStream_t st, int *partials) {
  int total = 0;
  (void)hipGetLastError();
  const int rc = each_set(grads, count, [&](const Set &s, int) {
    const int grid = grid_of(s);
    if (ord == TOPOEP_NORM_2)
      hipLaunchKernelGGL((grad_norm_kernel<Sum>), dim3(grid), dim3(kThreads), 0, st, s, ws + total);
    else
      hipLaunchKernelGGL((grad_norm_kernel<Largest>), dim3(grid), dim3(kThreads), 0, st, s, ws + total);
    total += grid;
    return hipGetLastError() == hipSuccess ? TOPOEP_OK : TOPOEP_EHIP;
  });
  *partials = total;
  return rc;
}

}  // namespace

extern "C" {

int topoep_grads_workspace_bytes(int32_t count, size_t *bytes_out) {
  if (count < 0 || !bytes_out) return TOPOEP_EINVAL;
  *bytes_out = (partials_bytes(count) + 255) & ~(size_t)255;
  return TOPOEP_OK;
}

int topoep_grad_norm(const topoep_grad *grads, int32_t count, float scale, int32_t ord, float *norm, void *workspace,
                     size_t workspace_bytes, void *stream) {
  int rc = check_set(grads, count, false);
  if (rc != TOPOEP_OK) return rc;
  if (!finite_scale(scale) || (ord != TOPOEP_NORM_2 && ord != TOPOEP_NORM_INF) || !norm) return TOPOEP_EINVAL;
  rc = check_workspace(workspace, workspace_bytes, count);
  if (rc != TOPOEP_OK) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  double *ws = static_cast<double *>(workspace);
  int partials = 0;
  rc = enqueue_partials(grads, count, ord, ws, st, &partials);
  if (rc != TOPOEP_OK) return rc;
  if (ord == TOPOEP_NORM_2)
    hipLaunchKernelGGL((grad_finish_kernel<Sum>), dim3(1), dim3(kThreads), 0, st, ws, partials, scale, norm);
  else
    hipLaunchKernelGGL((grad_finish_kernel<Largest>), dim3(1), dim3(kThreads), 0, st, ws, partials, scale, norm);
  return hipGetLastError() == hipSuccess ? TOPOEP_OK : TOPOEP_EHIP;
}

int topoep_clip_grads(const topoep_grad *grads, int32_t count, float scale, int32_t ord, float max_norm,
                      const float *given_norm, float *norm, void *workspace, size_t workspace_bytes, void *stream) {
  int rc = check_set(grads, count, true);
  if (rc != TOPOEP_OK) return rc;
  if (!finite_scale(scale) || (ord != TOPOEP_NORM_2 && ord != TOPOEP_NORM_INF) || !(max_norm > 0.0f))
    return TOPOEP_EINVAL;
  rc = check_workspace(workspace, workspace_bytes, count);
  if (rc != TOPOEP_OK) return rc;
  hipStream_t st = static_cast<hipStream_t>(stream);
  double *ws = static_cast<double *>(workspace);
  int partials = 0;
  if (!given_norm) {
    rc = enqueue_partials(grads, count, ord, ws, st, &partials);
    if (rc != TOPOEP_OK) return rc;
  }
  (void)hipGetLastError();
  return each_set(grads, count, [&](const Set &s, int launch) {
    Clip c{ws, partials, scale, max_norm, given_norm, launch == 0 ? norm : nullptr};
    if (ord == TOPOEP_NORM_2)
      hipLaunchKernelGGL((clip_kernel<Sum>), dim3(grid_of(s)), dim3(kThreads), 0, st, s, c);
    else
      hipLaunchKernelGGL((clip_kernel<Largest>), dim3(grid_of(s)), dim3(kThreads), 0, st, s, c);
    return hipGetLastError() == hipSuccess ? TOPOEP_OK : TOPOEP_EHIP;
  });
}

}  // extern "C"
