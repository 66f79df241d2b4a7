// Matrix products by tiles of a workgroup on gfx950: out[q][p] = sum_k P[p][k] Q[q][k].
//
// A tile is BP rows of P times BQ rows of Q.  Each stage brings 128 bytes of the
// inner axis of every row into LDS, past the registers (16 bytes a lane), while
// the stage before it is multiplied.  P is the matrix instruction's A operand, so
// a lane ends with four neighbouring p of one q: outputs are rows of p.
//
// An operand lies in memory either by rows (k runs along memory: 8 pieces of 16
// bytes a row and stage, the piece's place turned by the row so that the 16 rows
// a read takes meet every bank once), or across (p or q runs along memory, k over
// its rows: then LDS holds 64 rows of k, and reads transpose 16-bit elements on
// their way to the registers).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "router.h"

namespace topoep_dev {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v2i __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

struct I8 { int8_t v; };

// d += a b over 64 bytes of the inner axis, 16 by 16: lane l holds bytes (l / 16) * 16 .. + 15
// of row (column) l % 16, and of d the rows (l / 16) * 4 + 0..3 of column l % 16.
template <class T> struct Mul;
template <> struct Mul<Bf16> {
  typedef v4f Sum;
  static __device__ Sum add(v4i a, v4i b, Sum d) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), d, 0, 0, 0);
  }
};
template <> struct Mul<F16> {
  typedef v4f Sum;
  static __device__ Sum add(v4i a, v4i b, Sum d) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), d, 0, 0, 0);
  }
};
template <> struct Mul<I8> {
  typedef v4i Sum;
  static __device__ Sum add(v4i a, v4i b, Sum d) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, d, 0, 0, 0); }
};

constexpr int kLine = 128;            // bytes of the inner axis of a row and stage
constexpr int kAcross = kLine / 2;    // rows of the inner axis a stage holds where it runs across memory

typedef __attribute__((address_space(3))) char Lds;

// What lies behind the inner axis is read from here.
__device__ const v4i kZeros = {0, 0, 0, 0};

__device__ inline void to_lds(const char *from, Lds *to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                   (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}

// One operand of B rows, brought in by W waves.
template <class T, int B, int W, bool Across>
struct Operand {
  static constexpr int kBytes = B * kLine;
  static constexpr int kPieces = B / 8;                              // a wave's load is 1 KiB
  static constexpr int kLoads = (kPieces + W - 1) / W;               // (too few for all waves: some bring the same)
  static constexpr int kRowPieces = Across ? B / 8 : 8;              // 16 bytes each
  const char *from[kLoads];
  int64_t step;                                                      // bytes from a stage to the next

  // Which wave load is this thread's i-th, and of it the row and the piece in memory.
  static __device__ int load_of(int i, int wave) { return (i * W + wave) % kPieces; }
  static __device__ int turn(int row) {
    return Across ? ((row & 3) | (row >> 1 & 4)) * 2 & (kRowPieces - 1) & ~1 : row & 7;
  }
  static __device__ int row_of(int i, int wave) { return (load_of(i, wave) * 64 + lane_id()) / kRowPieces; }
  static __device__ int piece_of(int i, int wave) {
    return (load_of(i, wave) * 64 + lane_id()) % kRowPieces ^ turn(row_of(i, wave));
  }

  __device__ void load(Lds *to, int wave, int k, int n) {
    // k: elements done, n: of the inner axis
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = Across ? row_of(i, wave) : piece_of(i, wave) * (16 / (int)sizeof(T));
      const char *p = at < n - k ? from[i] : reinterpret_cast<const char *>(&kZeros);
      to_lds(p, to + load_of(i, wave) * 1024);
      from[i] += step;
    }
  }
};

// A wave's view of an operand in LDS: N tiles of 16 rows from row0 on.
template <class T, int B, int N, bool Across>
struct View {
  static constexpr int kBases = Across ? (N < 4 ? N : 4) : 2;
  int at[kBases];
  __device__ explicit View(int row0) {
    const int l = lane_id();
    if (!Across) {
#pragma unroll
      for (int s = 0; s < 2; ++s) at[s] = (row0 + l % 16) * kLine + ((s * 4 + l / 16) ^ (l & 7)) * 16;
    } else {
      // lanes 4 r .. 4 r + 3 of a block of 16 read row r's 32 bytes
      const int i = l & 15, k = (l >> 4) * 8 + (i >> 2), turn = Operand<T, B, 1, true>::turn(k);
#pragma unroll
      for (int t = 0; t < kBases; ++t)
        at[t] = k * B * 2 + ((((row0 / 16 + t) * 2) ^ turn) + (i >> 1 & 1)) * 16 + (i & 1) * 8;
    }
  }
  __device__ v4i get(const Lds *from, int tile, int s) const {
    if (!Across) return *reinterpret_cast<const __attribute__((address_space(3))) v4i *>(from + at[s] + tile * 16 * kLine);
    // (four tiles on, the place moves by 128 bytes: the turn, below 128, leaves that bit alone only if aligned)
    const Lds *p = from + (at[tile % kBases] ^ (tile / kBases * 128)) + s * 32 * B * 2;
    const v4s a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)p);
    const v4s b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)(p + 4 * B * 2));
    const v2i x = __builtin_bit_cast(v2i, a), y = __builtin_bit_cast(v2i, b);
    return v4i{x[0], x[1], y[0], y[1]};
  }
};

// Waits until at most N of this wave's loads are under way, then for the other waves.
template <int N>
__device__ inline void arrived() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x0F70);   // vmcnt alone
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The shape of a tile's work: BP x BQ, by NP x NQ waves.
template <class T_, int BP_, int BQ_, int NP_, int NQ_, bool PA_ = false, bool QA_ = false>
struct Shape {
  typedef T_ T;
  static constexpr int BP = BP_, BQ = BQ_, NP = NP_, NQ = NQ_, kWaves = NP * NQ, kThreads = 64 * kWaves;
  static constexpr bool PA = PA_, QA = QA_;
  static constexpr int TP = BP / NP / 16, TQ = BQ / NQ / 16;
  static constexpr int kStage = PA ? kAcross : kLine / (int)sizeof(T);
  static constexpr int kBytes = (BP + BQ) * kLine;
  typedef typename Mul<T>::Sum Sum;
  typedef View<T, BP, TP, PA> PView;
  typedef View<T, BQ, TQ, QA> QView;
};

template <class S>
__device__ inline void multiply_stage(const Lds *ps, const Lds *qs, const typename S::PView &pv, const typename S::QView &qv,
                                      typename S::Sum (&d)[S::TP][S::TQ]) {
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    v4i q[S::TQ];
#pragma unroll
    for (int j = 0; j < S::TQ; ++j) q[j] = qv.get(qs, j, s);
#pragma unroll
    for (int i = 0; i < S::TP; ++i) {
      const v4i p = pv.get(ps, i, s);
#pragma unroll
      for (int j = 0; j < S::TQ; ++j) d[i][j] = Mul<typename S::T>::add(p, q[j], d[i][j]);
    }
  }
}

template <class S, class P, class Q>
__device__ inline void multiply(P &p, Q &q, int wave, int n, Lds *p0, Lds *p1, Lds *q0, Lds *q1, typename S::Sum (&d)[S::TP][S::TQ]) {
  const typename S::PView pv(wave % S::NP * S::TP * 16);
  const typename S::QView qv(wave / S::NP * S::TQ * 16);
  const int stages = (n + S::kStage - 1) / S::kStage;
  if (stages > 0) p.load(p0, wave, 0, n), q.load(q0, wave, 0, n);
  int k = S::kStage;
  for (int g = stages >> 1; g > 0; --g) {
    arrived<0>();
    p.load(p1, wave, k, n), q.load(q1, wave, k, n);
    multiply_stage<S>(p0, q0, pv, qv, d);
    arrived<0>();
    // (behind the last stage: zeros)
    p.load(p0, wave, k + S::kStage, n), q.load(q0, wave, k + S::kStage, n);
    multiply_stage<S>(p1, q1, pv, qv, d);
    k += 2 * S::kStage;
  }
  arrived<0>();
  if (stages & 1) multiply_stage<S>(p0, q0, pv, qv, d);
}

}  // namespace topoep_dev
