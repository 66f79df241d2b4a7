// The router on gfx950: top-k ids and weights of every token from its
// logits, and the gradient back to the logits.
#include "router.h"

namespace {

using namespace topoep_dev;

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

// d = gradient of the row's chosen scores lies in LDS by expert while the
// row's lanes write their elements, and is cleared again after them.
template <class T, int LPT, int V>
__global__ __launch_bounds__(kThreads) void route_backward_kernel(RouteBackward a) {
  constexpr int kRows = kThreads / LPT;
  __shared__ float dense[kRows][LPT * V];
  const int slot = threadIdx.x / LPT, sub = threadIdx.x % LPT;
  float *d = dense[slot];
#pragma unroll
  for (int v = 0; v < V; ++v) d[sub * V + v] = 0.0f;
  wave_sync();
  const bool whole = !a.r.sigmoid && !a.r.renorm;
  for (int64_t t0 = (int64_t)blockIdx.x * kRows; t0 < a.T; t0 += (int64_t)gridDim.x * kRows) {
    const int64_t t = t0 + slot;
    const bool live = t < a.T;
    const T *row = static_cast<const T *>(a.logits) + (live ? t : t0) * a.ld;
    const bool mine = live && sub < a.r.k;
    const int id = mine ? a.ids[t * a.r.k + sub] : -1;
    const bool in = (unsigned)id < (unsigned)a.r.E;
    const float g = mine ? a.r.scale * a.grad[t * a.r.k + sub] : 0.0f;
    const float xj = in ? clean_logit(to_float(row[id])) : -INFINITY;   // masked: score 0
    float p[V], back = 0.0f, dj;
    if (whole) {
      load_logits<T, V>(row, sub * V, a.r.E, p);
      float m = p[0];
#pragma unroll
      for (int v = 1; v < V; ++v) m = fmaxf(m, p[v]);
      m = row_maxf<LPT>(m);
      float sum = 0.0f;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        p[v] = m == -INFINITY ? 0.0f : __expf(p[v] - m);
        sum += p[v];
      }
      sum = row_sum<LPT>(sum);
      const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
      for (int v = 0; v < V; ++v) p[v] *= inv;
      back = row_sum<LPT>(in && m != -INFINITY ? g * (__expf(xj - m) * inv) : 0.0f);
      dj = g;
    } else if (a.r.sigmoid) {
      const float s = in ? sigmoid(xj) : 0.0f;
      dj = g;
      if (a.r.renorm) {
        const float sum = row_sum<LPT>(s);
        const float mean = row_sum<LPT>(g * s);
        dj = sum > 0.0f ? (g - mean / sum) / sum : 0.0f;
      }
      dj *= s * sigmoid(-xj);
    } else {
      const float m = row_maxf<LPT>(xj);
      const float e = m == -INFINITY ? 0.0f : __expf(xj - m);
      const float sum = row_sum<LPT>(e);
      const float q = sum > 0.0f ? e / sum : 0.0f;
      dj = q * (g - row_sum<LPT>(g * q));
    }
    if (in) d[id] = dj;
    wave_sync();
    T out[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const float c = d[sub * V + v];
      out[v] = from_float<T>(whole ? p[v] * (c - back) : c);
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

// Calls f with the kernel for these sizes: LPT lanes a row, V elements each.
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
  const bool wide = r->groups > 1 || T < 8192;
  switch (r->dtype) {
    case TOPOEP_F32: return launch_rows<float, Forward>(a.r.E, a.r.k, wide, a, T, st);
    case TOPOEP_BF16: return launch_rows<Bf16, Forward>(a.r.E, a.r.k, wide, a, T, st);
    default: return launch_rows<F16, Forward>(a.r.E, a.r.k, wide, a, T, st);
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
  const bool wide = T < 8192;
  switch (r->dtype) {
    case TOPOEP_F32: return launch_rows<float, Backward>(a.r.E, a.r.k, wide, a, T, st);
    case TOPOEP_BF16: return launch_rows<Bf16, Backward>(a.r.E, a.r.k, wide, a, T, st);
    default: return launch_rows<F16, Backward>(a.r.E, a.r.k, wide, a, T, st);
  }
}

}  // extern "C"
