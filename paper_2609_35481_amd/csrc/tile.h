// Matrix products by tiles of a workgroup on gfx950: out[q][p] = sum_k P[p][k] Q[q][k].
//
// A tile is BP rows of P times BQ rows of Q.  Each stage brings 128 bytes of the
// inner axis of every row into LDS, past the registers (16 bytes a lane), while
// the stage before it is multiplied.  P is the matrix instruction's A operand, so
// a lane ends with four neighbouring p of one q: outputs are rows of p.
//
// An operand lies in memory either by rows (k runs along memory), or across (p or
// q runs along memory, k over its rows: then reads from LDS transpose 16-bit
// elements on their way to the registers).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

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

// A thread's wave and lane.  Asked for anew for every tile, in a way that the compiler does not
// see through: what it forms from the lane would else stay in registers over all tiles, which
// the sums of 256 x 256 leave no room for.
struct Me {
  int wave, lane;
  __device__ Me() : wave(uniform_i32(threadIdx.x >> 6)), lane(lane_id()) { asm volatile("" : "+v"(lane)); }
};

// An operand by rows: B rows, brought in by W waves.  LDS holds 8 pieces of 16 bytes a row
// and stage, a piece's place turned by the row, so that the 16 rows that a read takes meet
// every bank once.
template <class T, int B, int W>
struct ByRows {
  static constexpr int kLoads = B / 8 / W;   // a wave's load is 8 rows
  static_assert(kLoads * W * 8 == B, "every wave as many");
  const char *from[kLoads];

  static __device__ int load_of(int i, int wave) { return i * W + wave; }
  static __device__ int row_of(int i, Me me) { return load_of(i, me.wave) * 8 + (me.lane >> 3); }
  static __device__ int piece_of(Me me) { return (me.lane & 7) ^ (me.lane >> 3); }

  // row(r) gives the address of row r of the tile.
  template <class F>
  __device__ void start(Me me, const F &row) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) from[i] = row(row_of(i, me)) + piece_of(me) * 16;
  }
  // The stage from element k of n on (`next`: the one after it).
  __device__ void load(Lds *to, Me me, int k, int next, int n) {
    const bool in = piece_of(me) * (16 / (int)sizeof(T)) < n - k;
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      to_lds(in ? from[i] + (int64_t)k * (int)sizeof(T) : reinterpret_cast<const char *>(&kZeros), to + load_of(i, me.wave) * 1024);
  }
};

// An operand across: 64 rows of k a stage, B elements of 16 bits each.  A transposing read takes, of
// 16 elements, the rows 8 b + 4 h + r (+ 32 s): b = 0..3 by the lane's block of 16, r = 0..3 inside it, h and
// s one read each.  A wave's load holds rows that no read takes together (h, for narrower rows s too),
// and loads lie 32 bytes more than their 1 KiB apart: a read's rows meet every bank once, and every
// place is one lane's base and a constant (turned places, as for rows, take a base a tile: spills).
constexpr int kApart = 1024 + 32;
template <int B, int W>
struct AcrossPlaces {
  static_assert(B == 128 || B == 256, "four or two rows a load");
  static constexpr int kRowPieces = B / 8, kPieces = B / 8;   // of 16 bytes in a row; loads of a stage
  static constexpr int kBytes = kPieces * kApart, kLoads = kPieces / W;
  static_assert(kLoads * W == kPieces, "every wave as many");
  static __device__ int load_of(int i, int wave) { return i * W + wave; }
  // The row of k of load j (the same for all lanes) and what the lane adds to it.
  static __device__ int row_of_load(int j) { return (j & 3) + (j >> 2 & 3) * 8 + (B == 256 ? j >> 4 : 0) * 32; }
  static __device__ int row_of_lane(Me me) {
    const int sub = me.lane / kRowPieces;
    return (sub & 1) * 4 + (B == 128 ? sub >> 1 : 0) * 32;
  }
  static __device__ int column_of(Me me) { return me.lane % kRowPieces * 8; }
  static __device__ int row_of(int i, Me me) { return row_of_load(load_of(i, me.wave)) + row_of_lane(me); }
};

template <class T, int B, int W>
struct Across : AcrossPlaces<B, W> {
  typedef AcrossPlaces<B, W> At;
  const char *from;
  int64_t ld;   // bytes

  // `base`: row 0 of the inner axis, rows `stride` elements apart; of its n columns those from c0 on (one
  // that does not exist is column 0).
  __device__ void start(Me me, const void *base, int64_t stride, int c0, int n) {
    const int c = c0 + At::column_of(me);
    ld = stride * 2;
    from = static_cast<const char *>(base) + At::row_of_lane(me) * ld + (c < n ? c : 0) * 2;
  }
  __device__ void load(Lds *to, Me me, int k, int next, int n) {
    const int left = n - k - At::row_of_lane(me);
#pragma unroll
    for (int i = 0; i < At::kLoads; ++i) {
      const int j = At::load_of(i, me.wave), row = At::row_of_load(j);
      to_lds(row < left ? from + (k + row) * ld : reinterpret_cast<const char *>(&kZeros), to + j * kApart);
    }
  }
};

// A wave's view of an operand in LDS: tiles of 16 rows from row0 on.
template <class T, int B, bool IsAcross>
struct View {
  int at[IsAcross ? 1 : 2];
  __device__ View(int row0, int l) {
    if constexpr (!IsAcross) {
#pragma unroll
      for (int s = 0; s < 2; ++s) at[s] = (row0 + l % 16) * kLine + ((s * 4 + l / 16) ^ (l & 7)) * 16;
    } else {
      // lanes 4 r .. 4 r + 3 of a block of 16 read row r's 32 bytes
      const int b = l >> 4, r = l >> 2 & 3;
      at[0] = (b * 4 + r) * kApart + row0 * 2 + (l & 3) * 8;
    }
  }
  __device__ v4i get(const Lds *from, int tile, int s) const {
    if constexpr (!IsAcross) {
      return *reinterpret_cast<const __attribute__((address_space(3))) v4i *>(from + at[s] + tile * 16 * kLine);
    } else {
      const Lds *p = from + at[0] + tile * 32 + (B == 256 ? s * 16 * kApart : s * 2 * B * 2);
      const v4s x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)p);
      const v4s y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)(p + B * 2));
      const v2i u = __builtin_bit_cast(v2i, x), v = __builtin_bit_cast(v2i, y);
      return v4i{u[0], u[1], v[0], v[1]};
    }
  }
};

// Waits until at most N of this wave's loads into LDS are under way, and for its reads from there, then
// for the other waves.
template <int N>
__device__ inline void arrived() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x0070);   // vmcnt N, lgkmcnt 0
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The shape of a tile's work: BP x BQ, by NP x NQ waves; Ahead: a stage's loads issued before
// each of its first groups of matrix instructions.
template <class T_, int BP_, int BQ_, int NP_, int NQ_, bool PA_, bool QA_, int Ahead_>
struct Shape {
  typedef T_ T;
  static constexpr int Ahead = Ahead_;
  static constexpr int BP = BP_, BQ = BQ_, NP = NP_, NQ = NQ_, kWaves = NP * NQ, kThreads = 64 * kWaves;
  static constexpr bool PA = PA_, QA = QA_;
  static constexpr int TP = BP / NP / 16, TQ = BQ / NQ / 16;
  static constexpr int kStage = PA ? kAcross : kLine / (int)sizeof(T);
  static constexpr bool kDeep = !PA;                     // three stages of P in LDS, not two
  static constexpr int kBytesP = PA ? AcrossPlaces<BP, kWaves>::kBytes : BP * kLine;
  static constexpr int kBytesQ = QA ? AcrossPlaces<BQ, kWaves>::kBytes : BQ * kLine;
  typedef typename Mul<T>::Sum Sum;
  typedef View<T, BP, PA> PView;
  typedef View<T, BQ, QA> QView;
};

// The order of a stage's instructions, which the compiler would leave to itself with
// the next stage's loads last: operands are read from LDS two groups of matrix
// instructions ahead, loads spread over the first groups (8192^3 in bf16, 256 x 256 tiles:
// 1093 TFLOP/s without, 1340 with).
template <class S, int Loads, int G = 0>
__device__ inline void stage_order() {
  constexpr int RP = S::PA ? 2 : 1, RQ = S::QA ? 2 : 1, kGroups = 2 * S::TP;
  if constexpr (G == 0) __builtin_amdgcn_sched_group_barrier(0x100, S::TQ * RQ + 2 * RP, 0);
  if constexpr (G < kGroups) {
    constexpr int loads = Loads - G * S::Ahead < S::Ahead ? Loads - G * S::Ahead : S::Ahead;
    if constexpr (loads > 0) __builtin_amdgcn_sched_group_barrier(0x20, loads, 0);
    __builtin_amdgcn_sched_group_barrier(0x8, S::TQ, 0);
    constexpr int kEarly = S::TP - 2;   // groups before which the second half's Q is read
    constexpr int reads = (G + 2 < kGroups ? RP : 0) + (G < kEarly ? (S::TQ * RQ + kEarly - 1) / kEarly : 0);
    if constexpr (reads > 0) __builtin_amdgcn_sched_group_barrier(0x100, reads, 0);
    stage_order<S, Loads, G + 1>();
  }
}

// LDS of the stages.
struct Stages { Lds *p[3], *q[2]; };

template <class S, int Loads>
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
  stage_order<S, Loads>();
}

// The first element of the next stage to load: from stage `start` on and round, behind the last one n
// (zeros).
template <int Stage>
struct Cursor {
  int k, left, n;
  __device__ Cursor(int n_, int start) : k(start * Stage), left((n_ + Stage - 1) / Stage), n(n_) {}
  __device__ int after() const { return left > 1 ? (k + Stage < n ? k + Stage : 0) : n; }
  template <class O>
  __device__ void load(O &o, Lds *to, Me me) {
    const int next = after();
    o.load(to, me, k, next, n);
    k = next;
    --left;
  }
};

// d += P Q over the n elements of the inner axis: one stage is multiplied while the next one is on its
// way, of P (weights, from memory) by rows the one after it too, which fills the 160 KB of LDS (64 rows, H = 4096, I
// = 11008: 91 against 64 us).  Every wave is done with a stage's LDS when the next barrier lets loads into it.
//
// 256 x 256 tiles, 8192^3 in bf16: 1340 TFLOP/s in each of the three layouts (a library's product 1397 by rows,
// 1231 and 1073 with one and two operands across), the matrix units busy for 57 % of the time; in 8 bits 2.4 POP/s.
// Tiles of 128 x 128, two workgroups a CU: 1100.  Measured and not kept: stages of 64 bytes, four of them (1150 by
// rows: their lines are fetched twice), 256 x 128 tiles (965), a wave's priority raised while it multiplies (4 % longer),
// the next tile's first stage loaded before a tile is stored (no different, and 6 % longer for the weights' gradients).
template <class S, class P, class Q>
__device__ inline void multiply(P &p, Q &q, Me me, int n, int start, const Stages &lds, typename S::Sum (&d)[S::TP][S::TQ]) {
  constexpr int kLoads = P::kLoads + Q::kLoads;
  const typename S::PView pv(me.wave % S::NP * S::TP * 16, me.lane);
  const typename S::QView qv(me.wave / S::NP * S::TQ * 16, me.lane);
  const int stages = (n + S::kStage - 1) / S::kStage;
  Cursor<S::kStage> kp(n, start);
  if constexpr (!S::kDeep) {
    // (P's loads first: the other order takes 5 to 10 % longer)
    const auto load = [&](int i) {
      const int next = kp.after();
      p.load(lds.p[i], me, kp.k, next, n), q.load(lds.q[i], me, kp.k, next, n);
      kp.k = next;
      --kp.left;
    };
    if (stages > 0) load(0);
#pragma unroll 1
    for (int g = stages >> 1; g > 0; --g) {
      arrived<0>();
      load(1);
      multiply_stage<S, kLoads>(lds.p[0], lds.q[0], pv, qv, d);
      arrived<0>();
      load(0);
      multiply_stage<S, kLoads>(lds.p[1], lds.q[1], pv, qv, d);
    }
    arrived<0>();
    if (stages & 1) multiply_stage<S, 0>(lds.p[0], lds.q[0], pv, qv, d);
  } else {
    Cursor<S::kStage> kq(n, start);
    if (stages > 0) {
      kp.load(p, lds.p[0], me);
      kq.load(q, lds.q[0], me);
      __builtin_amdgcn_sched_barrier(0);
      kp.load(p, lds.p[1], me);
    }
    const auto stage = [&](auto i) {
      constexpr int I = decltype(i)::value;
      arrived<P::kLoads>();
      kq.load(q, lds.q[(I + 1) % 2], me);
      // (the loads that a wait leaves under way are the last ones: nothing from memory passes here)
      __builtin_amdgcn_sched_barrier(0x78F);
      kp.load(p, lds.p[(I + 2) % 3], me);
      multiply_stage<S, kLoads>(lds.p[I % 3], lds.q[I % 2], pv, qv, d);
    };
    int g = stages;
#pragma unroll 1
    for (; g >= 6; g -= 6) {
      stage(std::integral_constant<int, 0>());
      stage(std::integral_constant<int, 1>());
      stage(std::integral_constant<int, 2>());
      stage(std::integral_constant<int, 3>());
      stage(std::integral_constant<int, 4>());
      stage(std::integral_constant<int, 5>());
    }
    if (g > 0) stage(std::integral_constant<int, 0>());
    if (g > 1) stage(std::integral_constant<int, 1>());
    if (g > 2) stage(std::integral_constant<int, 2>());
    if (g > 3) stage(std::integral_constant<int, 3>());
    if (g > 4) stage(std::integral_constant<int, 4>());
    arrived<0>();
  }
}

// The stage a workgroup starts with.  Rows lie multiples of some kilobytes apart: workgroups that read the
// same place of all their rows meet few of memory's channels.  Those of an XCD and a group share operands
// and stay together (a training step of 8192 rows, H = 4096, I = 14336: 7.49 ms from the same place, 7.35 so).
template <class S>
__device__ inline int start_of(int n, int group) {
  const int stages = (n + S::kStage - 1) / S::kStage;
  return stages > 0 ? (int)(((blockIdx.x & 7) * (unsigned)stages / 8 + (unsigned)group * 5u) % (unsigned)stages) : 0;
}

}  // namespace topoep_dev
