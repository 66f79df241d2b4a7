// The rows of a routed layer by expert: a stable counting sort of the router's
// choices on gfx950.
//
// A workgroup ranks a chunk of 1024 to 8192 pairs: its waves take equal shares of
// neighbours, 64 at a time, whose ranks among equals come from ballots and a row of counts a
// wave in LDS; the rows of counts are then summed in the order of the waves.  One chunk
// is one launch; more are three (ranks, sums over the chunks, places).  Nothing
// here is decided by the order in which anything runs.
//
// Bound: for a decoding batch the launch; for long ones memory would give 12
// bytes a pair in no time and the three launches and the sums over
// the chunks remain.
#include "topoep_ffn.h"
#include "wave.h"

namespace {

using namespace topoep_dev;

constexpr int kThreads = 1024, kWaves = kThreads / 64, kRounds = 8;

struct Rows {
  const int32_t *ids, *slot;
  int E, L, n, bits;
  int32_t *offsets, *pairs, *places;
  int32_t *counts;   // [chunks, L]
  int chunks, rounds;   // a chunk is kThreads * rounds pairs
};

// Where pair i's expert is among those here, -1 if nowhere.
__device__ inline int slot_at(const Rows &a, int i) {
  const int e = a.ids[i];
  if ((unsigned)e >= (unsigned)a.E) return -1;
  const int s = a.slot ? a.slot[e] : e;
  return (unsigned)s < (unsigned)a.L ? s : -1;
}

template <bool One>
__global__ __launch_bounds__(kThreads) void rank_kernel(Rows a) {
  extern __shared__ int lds[];   // counts [kWaves, L], totals [L], scan [kWaves + 1]
  int *totals = lds + kWaves * a.L, *tmp = totals + a.L;
  const int tid = threadIdx.x, wave = uniform_i32(tid >> 6);
  for (int i = tid; i < kWaves * a.L; i += kThreads) lds[i] = 0;
  __syncthreads();
  const int64_t first = ((int64_t)blockIdx.x * kWaves + wave) * (64 * a.rounds) + lane_id();
  int *mine = lds + wave * a.L;
  int slot[kRounds], rank[kRounds];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) slot[r] = r < a.rounds && first + r * 64 < a.n ? slot_at(a, (int)first + r * 64) : -1;
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    rank[r] = 0;
    if (__ballot(slot[r] >= 0)) rank[r] = wave_rank(slot[r], slot[r] >= 0, a.bits, mine);
  }
  __syncthreads();
  for (int e = tid; e < a.L; e += kThreads) {
    int run = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int t = lds[w * a.L + e];
      lds[w * a.L + e] = run;
      run += t;
    }
    if (One) totals[e] = run;
    else a.counts[(int64_t)blockIdx.x * a.L + e] = run;
  }
  __syncthreads();
  int here = 0;
  if (One) {
    here = block_excl_scan(totals, a.L, tmp);
    for (int e = tid; e < a.L; e += kThreads) a.offsets[e] = totals[e];
    if (tid == 0) a.offsets[a.L] = here;
  }
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int64_t i = first + r * 64;
    if (r >= a.rounds || i >= a.n) continue;
    const int at = slot[r] < 0 ? -1 : mine[slot[r]] + rank[r] + (One ? totals[slot[r]] : 0);
    a.places[i] = at;   // (more chunks than one: in the chunk)
    if (One) {
      if (at >= 0) a.pairs[at] = (int)i;
      if (i >= here) a.pairs[i] = -1;
    }
  }
}

// Over the chunks, then over the slots: counts become each chunk's first row of
// each slot.  `parts` threads share a slot, the chunks split over them.
__global__ __launch_bounds__(kThreads) void sum_kernel(Rows a, int parts) {
  __shared__ int part[kThreads], totals[TOPOEP_FFN_MAX_EXPERTS], tmp[kWaves + 1];
  const int tid = threadIdx.x, p = tid / a.L, e = tid % a.L;
  const int each = (a.chunks + parts - 1) / parts, lo = imin(p * each, a.chunks), hi = imin(lo + each, a.chunks);
  const bool live = p < parts;
  int run = 0;
  if (live)
    for (int c = lo; c < hi; ++c) run += a.counts[(int64_t)c * a.L + e];
  part[tid] = run;
  __syncthreads();
  if (tid < a.L) {
    int s = 0;
    for (int i = 0; i < parts; ++i) {
      const int t = part[i * a.L + tid];
      part[i * a.L + tid] = s;
      s += t;
    }
    totals[tid] = s;
  }
  __syncthreads();
  const int here = block_excl_scan(totals, a.L, tmp);
  if (tid < a.L) a.offsets[tid] = totals[tid];
  if (tid == 0) a.offsets[a.L] = here;
  if (!live) return;
  run = totals[e] + part[tid];
  for (int c = lo; c < hi; ++c) {
    const int t = a.counts[(int64_t)c * a.L + e];
    a.counts[(int64_t)c * a.L + e] = run;
    run += t;
  }
}

__global__ __launch_bounds__(256) void place_kernel(Rows a) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= a.n) return;
  const int s = slot_at(a, (int)i);
  if (s >= 0) {
    const int at = a.places[i] + a.counts[i / (kThreads * a.rounds) * a.L + s];
    a.places[i] = at;
    a.pairs[at] = (int)i;
  }
  if (i >= a.offsets[a.L]) a.pairs[i] = -1;
}

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

int check(int32_t T, int32_t k, int32_t L) {
  if (T < 0 || k < 1 || (int64_t)T * k > INT32_MAX || L < 1) return TOPOEP_EINVAL;
  return L > TOPOEP_FFN_MAX_EXPERTS ? TOPOEP_ELIMIT : TOPOEP_OK;
}

// Rounds of a chunk's waves: one chunk where eight do, else as few as leave the sums' one workgroup
// no more than 64 chunks.
constexpr int kChunks = 64;
int rounds_of(int64_t n) {
  const int64_t one = (n + kThreads - 1) / kThreads;
  if (one <= kRounds) return (int)one;
  const int64_t r = (one + kChunks - 1) / kChunks;
  return (int)(r < kRounds ? r : kRounds);
}

// (enough for fewer pairs too, which may have more chunks)
size_t need(int32_t T, int32_t k, int32_t L) {
  const int64_t one = ((int64_t)T * k + kThreads - 1) / kThreads, most = (one + kRounds - 1) / kRounds;
  return align256((size_t)(one < kChunks ? one : most < kChunks ? kChunks : most) * L * sizeof(int32_t));
}

bool launched() { return hipGetLastError() == hipSuccess; }

}  // namespace

extern "C" {

int topoep_expert_rows_workspace_bytes(int32_t T, int32_t k, int32_t L, size_t *bytes_out) {
  const int rc = check(T, k, L);
  if (rc != TOPOEP_OK) return rc;
  if (!bytes_out) return TOPOEP_EINVAL;
  *bytes_out = need(T, k, L);
  return TOPOEP_OK;
}

int topoep_expert_rows(const int32_t *ids, int32_t T, int32_t k, const int32_t *expert_slot, int32_t E, int32_t L,
                       int32_t *offsets, int32_t *pairs, int32_t *places, void *workspace, size_t workspace_bytes,
                       void *stream) {
  const int rc = check(T, k, L);
  if (rc != TOPOEP_OK) return rc;
  if (E < 1 || !offsets || (T > 0 && (!ids || !pairs || !places || !workspace))) return TOPOEP_EINVAL;
  if ((reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < need(T, k, L)) return TOPOEP_EWORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  Rows a;
  a.ids = ids;
  a.slot = expert_slot;
  a.E = E;
  a.L = L;
  a.n = T * k;
  a.bits = 0;
  while (1 << a.bits < L) ++a.bits;
  a.offsets = offsets;
  a.pairs = pairs;
  a.places = places;
  a.counts = static_cast<int32_t *>(workspace);
  a.rounds = rounds_of(a.n);
  a.chunks = a.n == 0 ? 0 : (int)(((int64_t)a.n + kThreads * a.rounds - 1) / (kThreads * a.rounds));
  const size_t lds = ((size_t)(kWaves + 1) * L + kWaves + 1) * sizeof(int);
  if (lds > 64 * 1024) {
    const int most = ((kWaves + 1) * TOPOEP_FFN_MAX_EXPERTS + kWaves + 1) * (int)sizeof(int);
    (void)hipFuncSetAttribute(reinterpret_cast<const void *>(rank_kernel<true>), hipFuncAttributeMaxDynamicSharedMemorySize, most);
    (void)hipFuncSetAttribute(reinterpret_cast<const void *>(rank_kernel<false>), hipFuncAttributeMaxDynamicSharedMemorySize, most);
  }
  (void)hipGetLastError();
  if (a.chunks <= 1) {
    hipLaunchKernelGGL((rank_kernel<true>), dim3(1), dim3(kThreads), lds, st, a);
    return launched() ? TOPOEP_OK : TOPOEP_EHIP;
  }
  hipLaunchKernelGGL((rank_kernel<false>), dim3(a.chunks), dim3(kThreads), lds, st, a);
  if (!launched()) return TOPOEP_EHIP;
  int parts = 1;
  while (parts * 2 * L <= kThreads && parts < a.chunks) parts *= 2;
  hipLaunchKernelGGL(sum_kernel, dim3(1), dim3(kThreads), 0, st, a, parts);
  if (!launched()) return TOPOEP_EHIP;
  hipLaunchKernelGGL(place_kernel, dim3((unsigned)(((int64_t)a.n + 255) / 256)), dim3(256), 0, st, a);
  return launched() ? TOPOEP_OK : TOPOEP_EHIP;
}

}  // extern "C"
