// The global gradient norm over many tensors and the clip on gfx950.
//
// The tensors' addresses and sizes travel as kernel arguments, so a call copies
// nothing to the device and may be captured; tensors that follow each other in
// memory (views of one flat buffer) count as one.  A launch's elements are cut
// into chunks of kChunk elements that do not cross tensors, and workgroup b takes
// pieces b, b + grid, ... of kPiece chunks.  The norm
// kernel leaves one 64-bit partial a workgroup; the reader sums them in a fixed
// order: every workgroup of the clip for itself, or, where there are more than one
// launch leaves, a kernel of its own once.  Squares are formed and summed in 64 bits: the square of any 32-bit
// number is exact there and neither overflows nor vanishes.
//
// Bound: memory.  The norm of 1.37 G 16-bit elements runs at 6.8 TB/s (7.0 for
// reads alone on this card), the clip of 441 M of them into a 32-bit buffer
// moves its 2.65 GB at 5.7 TB/s (6.0 for a plain copy), 440 M in place 1.76 GB at 5.6.  Loads and stores go past
// the caches (without: 4.6 and 4.5 TB/s).  The pieces lie in the order of the
// workgroups: one long range a workgroup took the clip 520 us, this order 458.
#include <algorithm>
#include <memory>
#include <new>

#include "router.h"

namespace {

using namespace topoep_dev;

constexpr int kThreads = 256;
constexpr int64_t kChunk = 2048;
constexpr int kBlocks = 2048;      // workgroups, and partials, a launch of the norm has at most
constexpr int kClipBlocks = 8192;  // workgroups a launch of the clip has at most

// elements a set may have (2^29 chunks: chunk numbers are 32-bit words)
constexpr int64_t kMostElements = (int64_t)1 << 40;
// elements of one entry at most; larger tensors are several
constexpr int64_t kMostEntry = (int64_t)1 << 31;

// The tensors of a launch, as many as 4 KB of arguments hold: 240 for the
// norm, 160 for the clip.  An address carries its elements' type in its top byte.
template <bool Out>
struct Set {
  static constexpr int kMost = Out ? 160 : 240;
  int count, chunks;
  uint64_t from[kMost], to[Out ? kMost : 1];
  uint32_t first[kMost];   // chunks before entry i
  uint32_t n[kMost];       // its elements
  static __host__ __device__ uint64_t tagged(const void *p, int type) { return reinterpret_cast<uint64_t>(p) | (uint64_t)type << 56; }
  static __host__ __device__ int type(uint64_t p) { return (int)(p >> 56); }
  static __host__ __device__ char *address(uint64_t p) { return reinterpret_cast<char *>(p & (((uint64_t)1 << 56) - 1)); }
};

// The tensor that holds a chunk (the last with first <= chunk).
template <bool Out>
__device__ inline int tensor_of(const Set<Out> &s, int chunk) {
  int lo = 0, hi = s.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if ((int)s.first[mid] <= chunk) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Calls f(tensor, first element, elements) for the parts of workgroup b's
// pieces, kPiece chunks each: b, b + grid, ... (Back: counted from the end), so
// that the workgroups' accesses move through memory together.
constexpr int kPiece = 4;
template <bool Back, bool Out, class F>
__device__ inline void each_part(const Set<Out> &s, int b, const F &f) {
  const int pieces = (s.chunks + kPiece - 1) / kPiece;
  for (int p = b; p < pieces; p += gridDim.x) {
    int c = (Back ? pieces - 1 - p : p) * kPiece;
    const int end = imin(c + kPiece, s.chunks);
    for (int i = tensor_of(s, c); c < end; ++i) {
      const int begin = (int)s.first[i], stop = i + 1 < s.count ? imin(end, (int)s.first[i + 1]) : end;
      const int64_t at = (int64_t)(c - begin) * kChunk, to = (int64_t)(stop - begin) * kChunk, n = s.n[i];
      f(i, at, (to < n ? to : n) - at);
      c = stop;
    }
  }
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

// W elements of T at once, 4 to 16 bytes, at any alignment of theirs.
template <int Bytes, int Align> struct Word;
template <> struct Word<16, 2> { typedef int type __attribute__((ext_vector_type(4), aligned(2))); };
template <> struct Word<16, 4> { typedef int type __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct Word<8, 2> { typedef int type __attribute__((ext_vector_type(2), aligned(2))); };

template <bool Stream, int W, class T>
__device__ inline void load_wide(const T *p, T (&raw)[W]) {
  typedef typename Word<W * sizeof(T), sizeof(T)>::type Q;
  const Q v = Stream ? __builtin_nontemporal_load(reinterpret_cast<const Q *>(p)) : *reinterpret_cast<const Q *>(p);
  __builtin_memcpy(raw, &v, sizeof(raw));
}
template <bool Stream, int W, class T>
__device__ inline void store_wide(T *p, const T (&raw)[W]) {
  typedef typename Word<W * sizeof(T), sizeof(T)>::type Q;
  Q v;
  __builtin_memcpy(&v, raw, sizeof(raw));
  if (Stream) __builtin_nontemporal_store(v, reinterpret_cast<Q *>(p));
  else *reinterpret_cast<Q *>(p) = v;
}

// Calls take(first element, raw) for W elements a thread at a time, U loads in
// flight, from element `head` on, and one(element) for those before it and
// those behind the last whole step of the workgroup.
template <bool Stream, int W, int U, class T, class F, class G>
__device__ inline void each_wide(const T *g, int64_t n, int head, const F &take, const G &one) {
  constexpr int64_t kStep = (int64_t)kThreads * W;
  if (head > n) head = (int)n;
  if ((int)threadIdx.x < head) one(threadIdx.x);
  int64_t i = head + (int64_t)threadIdx.x * W;
  int64_t steps = (n - head) / kStep;
  for (; steps >= U; steps -= U, i += U * kStep) {
    T raw[U][W];
#pragma unroll
    for (int u = 0; u < U; ++u) load_wide<Stream, W>(g + i + u * kStep, raw[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) take(i + u * kStep, raw[u]);
  }
  T raw[U][W];
#pragma unroll
  for (int u = 0; u < U - 1; ++u)
    if (u < steps) load_wide<Stream, W>(g + i + u * kStep, raw[u]);
#pragma unroll
  for (int u = 0; u < U - 1; ++u)
    if (u < steps) take(i + u * kStep, raw[u]);
  for (i = n - (n - head) % kStep + threadIdx.x; i < n; i += kThreads) one(i);
}

template <bool Stream, class T, class R>
__device__ inline void reduce_part(const T *g, int64_t n, R &r) {
  R other[3];   // four chains of sums
  constexpr int W = 16 / sizeof(T);
  each_wide<Stream, W, 8>(
      g, n, 0,
      [&](int64_t, const T(&raw)[W]) {
#pragma unroll
        for (int w = 0; w < W; w += 4) {
          r.add(to_float(raw[w]));
          other[0].add(to_float(raw[w + 1]));
          other[1].add(to_float(raw[w + 2]));
          other[2].add(to_float(raw[w + 3]));
        }
      },
      [&](int64_t i) { r.add(to_float(g[i])); });
  r.join(other[0].v);
  r.join(other[1].v);
  r.join(other[2].v);
}

template <class R, bool Stream>
__global__ __launch_bounds__(kThreads) void grad_norm_kernel(Set<false> s, double *partials) {
  __shared__ double lds[kThreads / 64];
  R r;
  each_part<false>(s, blockIdx.x, [&](int i, int64_t at, int64_t n) {
    const char *g = s.address(s.from[i]);
    switch (s.type(s.from[i])) {
      case TOPOEP_F32: reduce_part<Stream>(reinterpret_cast<const float *>(g) + at, n, r); break;
      case TOPOEP_BF16: reduce_part<Stream>(reinterpret_cast<const Bf16 *>(g) + at, n, r); break;
      default: reduce_part<Stream>(reinterpret_cast<const F16 *>(g) + at, n, r); break;
    }
  });
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

// Threads take as many elements as make 16 bytes of the wider type, from the
// first one on that starts a line of the outputs, so that whole lines are
// written at once.
template <bool Stream, class T, class O>
__device__ inline void scale_part(const T *g, O *out, int64_t n, float f) {
  constexpr int W = 16 / (sizeof(T) > sizeof(O) ? sizeof(T) : sizeof(O));
  const int head = (int)((0u - (uint32_t)reinterpret_cast<uintptr_t>(out)) & 127u) / (int)sizeof(O);
  each_wide<Stream, W, 4>(
      g, n, head,
      [&](int64_t i, const T(&raw)[W]) {
        O to[W];
#pragma unroll
        for (int w = 0; w < W; ++w) to[w] = from_float<O>(to_float(raw[w]) * f);
        store_wide<Stream, W>(out + i, to);
      },
      [&](int64_t i) { out[i] = from_float<O>(to_float(g[i]) * f); });
}

template <bool Stream, class T>
__device__ inline void scale_part_to(const T *g, char *out, int type, int64_t at, int64_t n, float f) {
  switch (type) {
    case TOPOEP_F32: scale_part<Stream>(g + at, reinterpret_cast<float *>(out) + at, n, f); break;
    case TOPOEP_BF16: scale_part<Stream>(g + at, reinterpret_cast<Bf16 *>(out) + at, n, f); break;
    default: scale_part<Stream>(g + at, reinterpret_cast<F16 *>(out) + at, n, f); break;
  }
}

struct Clip {
  const double *partials;
  int count;              // of partials; 0 = given
  float scale, max_norm;
  const float *given;
  float *norm;            // or null
};

template <class R, bool Stream>
__global__ __launch_bounds__(kThreads) void clip_kernel(Set<true> s, Clip c) {
  __shared__ double lds[kThreads / 64];
  const float norm = c.given ? *c.given : norm_of<R>(c.partials, c.count, c.scale, lds);
  if (c.norm && blockIdx.x == 0 && threadIdx.x == 0) *c.norm = norm;
  if (!(norm - norm == 0.0f)) return;
  const float f = c.scale * fminf(1.0f, c.max_norm / (norm + 1e-6f));
  each_part<true>(s, blockIdx.x, [&](int i, int64_t at, int64_t n) {
    if (f == 1.0f && s.to[i] == s.from[i]) return;
    const char *g = s.address(s.from[i]);
    char *out = s.address(s.to[i]);
    const int to = s.type(s.to[i]);
    switch (s.type(s.from[i])) {
      case TOPOEP_F32: scale_part_to<Stream>(reinterpret_cast<const float *>(g), out, to, at, n, f); break;
      case TOPOEP_BF16: scale_part_to<Stream>(reinterpret_cast<const Bf16 *>(g), out, to, at, n, f); break;
      default: scale_part_to<Stream>(reinterpret_cast<const F16 *>(g), out, to, at, n, f); break;
    }
  });
}

int bytes_of(int type) { return type == TOPOEP_F32 ? 4 : 2; }

// Walks the set in launches: fills each one's arguments and calls go(set,
// index of the launch).  Tensors that follow each other in memory (and their
// outputs too, where Out) are one entry.
template <bool Out, class F>
int each_set(const topoep_grad *grads, int count, const F &go) {
  Set<Out> s;
  int at = 0, launch = 0;
  int64_t done = 0;   // of tensor `at`
  do {
    s.count = 0;
    while (at < count) {
      const topoep_grad &g = grads[at];
      const int64_t left = g.n - done;
      if (left > 0) {
        const int width = bytes_of(g.dtype), wide = Out ? bytes_of(g.out_dtype) : 0;
        const uint64_t from = Set<Out>::tagged(static_cast<const char *>(g.grad) + done * width, g.dtype);
        const uint64_t to = Out ? Set<Out>::tagged(static_cast<char *>(g.out) + done * wide, g.out_dtype) : 0;
        const int last = s.count - 1;
        int64_t n = left < kMostEntry ? left : kMostEntry;
        if (last >= 0 && s.from[last] + (uint64_t)s.n[last] * width == from && s.n[last] + n <= kMostEntry &&
            (!Out || s.to[last] + (uint64_t)s.n[last] * wide == to)) {
          s.n[last] += (uint32_t)n;
        } else {
          if (s.count == Set<Out>::kMost) break;
          s.from[s.count] = from;
          if (Out) s.to[s.count] = to;
          s.n[s.count++] = (uint32_t)n;
        }
        done += n;
      }
      if (done == g.n) {
        ++at;
        done = 0;
      }
    }
    int64_t chunks = 0;
    for (int i = 0; i < s.count; ++i) {
      s.first[i] = (uint32_t)chunks;
      chunks += ((int64_t)s.n[i] + kChunk - 1) / kChunk;
    }
    s.chunks = (int)chunks;
    const int rc = go(s, launch++);
    if (rc != TOPOEP_OK) return rc;
  } while (at < count);
  return TOPOEP_OK;
}

// Bytes of the gradients from which on they are read (and results written) past
// the caches: what is larger than the 256 MB of the last one is not found
// there again anyway.
constexpr int64_t kStreamBytes = (int64_t)256 << 20;

bool streams(const topoep_grad *grads, int count) {
  int64_t bytes = 0;
  for (int i = 0; i < count; ++i) bytes += grads[i].n * bytes_of(grads[i].dtype);
  return bytes > kStreamBytes;
}

template <bool Out>
int grid_of(const Set<Out> &s, int most) { return imax(1, imin(most, (s.chunks + kPiece - 1) / kPiece)); }

struct Range {
  uintptr_t from, to;
};
Range range_of(const void *p, int64_t n, int type) {
  const uintptr_t from = reinterpret_cast<uintptr_t>(p);
  return Range{from, from + (uintptr_t)n * (uintptr_t)bytes_of(type)};
}

// Workgroups write the outputs in no order: no two may share memory, nor one with a
// gradient that is not its own.  Outputs in the order of their addresses, either way, apart
// from the gradients (or in place), are seen in one pass; others are sorted.
int check_overlaps(const topoep_grad *grads, int32_t count) {
  Range last{0, 0}, outs{UINTPTR_MAX, 0}, ins{UINTPTR_MAX, 0};
  bool up = true, down = true;
  for (int i = 0; i < count; ++i) {
    const topoep_grad &g = grads[i];
    if (g.n == 0) continue;
    const Range o = range_of(g.out, g.n, g.out_dtype);
    if (last.to) {
      up = up && o.from >= last.to;
      down = down && o.to <= last.from;
    }
    last = o;
    outs = Range{std::min(outs.from, o.from), std::max(outs.to, o.to)};
    if (g.out != g.grad) {
      const Range r = range_of(g.grad, g.n, g.dtype);
      ins = Range{std::min(ins.from, r.from), std::max(ins.to, r.to)};
    }
  }
  if ((up || down) && (ins.to <= outs.from || outs.to <= ins.from)) return TOPOEP_OK;
  std::unique_ptr<Range[]> sorted(new (std::nothrow) Range[count]);
  if (!sorted) return TOPOEP_ELIMIT;
  int n = 0;
  for (int i = 0; i < count; ++i)
    if (grads[i].n > 0) sorted[n++] = range_of(grads[i].out, grads[i].n, grads[i].out_dtype);
  const auto before = [](const Range &a, const Range &b) { return a.from < b.from; };
  std::sort(&sorted[0], &sorted[0] + n, before);
  for (int i = 1; i < n; ++i)
    if (sorted[i].from < sorted[i - 1].to) return TOPOEP_EINVAL;
  for (int i = 0; i < count; ++i) {
    const topoep_grad &g = grads[i];
    if (g.n == 0 || g.out == g.grad) continue;
    const Range r = range_of(g.grad, g.n, g.dtype);
    const Range *next = std::lower_bound(&sorted[0], &sorted[0] + n, r, before);   // the first output from r.from on
    if ((next < &sorted[0] + n && next->from < r.to) || (next > &sorted[0] && next[-1].to > r.from)) return TOPOEP_EINVAL;
  }
  return TOPOEP_OK;
}

int check_set(const topoep_grad *grads, int32_t count, bool out) {
  if (count < 0 || (count > 0 && !grads)) return TOPOEP_EINVAL;
  int64_t left = kMostElements;
  for (int i = 0; i < count; ++i) {
    const topoep_grad &g = grads[i];
    if (g.n < 0 || g.n > left || g.dtype < TOPOEP_F32 || g.dtype > TOPOEP_F16) return TOPOEP_EINVAL;
    left -= g.n;
    if (g.n == 0) continue;
    if (!g.grad || (reinterpret_cast<uintptr_t>(g.grad) & (g.dtype == TOPOEP_F32 ? 3 : 1)) ||
        reinterpret_cast<uintptr_t>(g.grad) >> 56)
      return TOPOEP_EINVAL;
    if (!out) continue;
    if (g.out_dtype < TOPOEP_F32 || g.out_dtype > TOPOEP_F16 || !g.out) return TOPOEP_EINVAL;
    if (reinterpret_cast<uintptr_t>(g.out) & (g.out_dtype == TOPOEP_F32 ? 3 : 1) || reinterpret_cast<uintptr_t>(g.out) >> 56)
      return TOPOEP_EINVAL;
    if (g.out == g.grad && g.out_dtype != g.dtype) return TOPOEP_EINVAL;
  }
  return out ? check_overlaps(grads, count) : TOPOEP_OK;
}

// kBlocks partials a launch; the entries are the tensors and the further parts
// of those beyond kMostEntry elements.
size_t partials_bytes(int32_t count) {
  return (((size_t)count + (size_t)(kMostElements / kMostEntry)) / Set<false>::kMost + 1) * kBlocks * sizeof(double);
}

// The partials and, behind them, the clip's norm.
size_t workspace_bytes_of(int32_t count) { return (partials_bytes(count) + sizeof(float) + 255) & ~(size_t)255; }

int check_workspace(const void *ws, size_t bytes, int32_t count) {
  if (!ws) return TOPOEP_EINVAL;
  size_t need = 0;
  const int rc = topoep_grads_workspace_bytes(count, &need);
  if (rc != TOPOEP_OK) return rc;
  return (reinterpret_cast<uintptr_t>(ws) & 255) || bytes < need ? TOPOEP_EWORKSPACE : TOPOEP_OK;
}

bool finite_scale(float s) { return s >= 0.0f && s - s == 0.0f; }

template <class R, bool Stream>
int enqueue_partials(const topoep_grad *grads, int count, double *ws, hipStream_t st, int *partials) {
  return each_set<false>(grads, count, [&](const Set<false> &s, int) {
    const int grid = grid_of(s, kBlocks);
    hipLaunchKernelGGL((grad_norm_kernel<R, Stream>), dim3(grid), dim3(kThreads), 0, st, s, ws + *partials);
    *partials += grid;
    return hipGetLastError() == hipSuccess ? TOPOEP_OK : TOPOEP_EHIP;
  });
}

template <class R>
int enqueue_norm(const topoep_grad *grads, int count, float scale, float *norm, double *ws, hipStream_t st) {
  int partials = 0;
  (void)hipGetLastError();
  const int rc = streams(grads, count) ? enqueue_partials<R, true>(grads, count, ws, st, &partials)
                                       : enqueue_partials<R, false>(grads, count, ws, st, &partials);
  if (rc != TOPOEP_OK) return rc;
  hipLaunchKernelGGL((grad_finish_kernel<R>), dim3(1), dim3(kThreads), 0, st, ws, partials, scale, norm);
  return hipGetLastError() == hipSuccess ? TOPOEP_OK : TOPOEP_EHIP;
}

template <class R, bool Stream>
int enqueue_clip(const topoep_grad *grads, int count, Clip c, double *ws, hipStream_t st) {
  (void)hipGetLastError();
  if (!c.given) {
    const int rc = enqueue_partials<R, Stream>(grads, count, ws, st, &c.count);
    if (rc != TOPOEP_OK) return rc;
    // Summed by every workgroup of every launch, the partials of many launches cost
    // more than the tensors (12 000 tensors of 65 536 elements: 8.6 ms, 2.4 so)
    if (c.count > kBlocks) {
      float *norm = c.norm ? c.norm : reinterpret_cast<float *>(reinterpret_cast<char *>(ws) + partials_bytes(count));
      hipLaunchKernelGGL((grad_finish_kernel<R>), dim3(1), dim3(kThreads), 0, st, ws, c.count, c.scale, norm);
      if (hipGetLastError() != hipSuccess) return TOPOEP_EHIP;
      c.given = norm;
      c.norm = nullptr;
    }
  }
  return each_set<true>(grads, count, [&](const Set<true> &s, int launch) {
    Clip own = c;
    if (launch > 0) own.norm = nullptr;
    hipLaunchKernelGGL((clip_kernel<R, Stream>), dim3(grid_of(s, kClipBlocks)), dim3(kThreads), 0, st, s, own);
    return hipGetLastError() == hipSuccess ? TOPOEP_OK : TOPOEP_EHIP;
  });
}

}  // namespace

extern "C" {

int topoep_grads_workspace_bytes(int32_t count, size_t *bytes_out) {
  if (count < 0 || !bytes_out) return TOPOEP_EINVAL;
  *bytes_out = workspace_bytes_of(count);
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
  return ord == TOPOEP_NORM_2 ? enqueue_norm<Sum>(grads, count, scale, norm, ws, st)
                              : enqueue_norm<Largest>(grads, count, scale, norm, ws, st);
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
  const Clip c{ws, 0, scale, max_norm, given_norm, norm};
  const bool stream_past = streams(grads, count);
  if (ord == TOPOEP_NORM_2)
    return stream_past ? enqueue_clip<Sum, true>(grads, count, c, ws, st) : enqueue_clip<Sum, false>(grads, count, c, ws, st);
  return stream_past ? enqueue_clip<Largest, true>(grads, count, c, ws, st)
                     : enqueue_clip<Largest, false>(grads, count, c, ws, st);
}

}  // extern "C"
