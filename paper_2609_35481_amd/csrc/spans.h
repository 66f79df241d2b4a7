// Which tiles a product has whose rows belong to groups (experts), and how its
// operands are reached.
#pragma once

#include <type_traits>

#include "tile.h"

namespace topoep_dev {

// The rows of a group: [first, end), those of `offsets` or all.
__device__ inline void rows_of(const int32_t *offsets, int rows, int g, int &first, int &end) {
  first = 0, end = rows;
  if (offsets) {
    first = imin(imax(offsets[g], 0), rows);
    end = imin(imax(offsets[g + 1], first), rows);
  }
}

// A tile of rows: `first` .. `end` - 1 are what is left of its group from its first on; the group's
// `tiles` start with number `before`.
struct Span { int group, first, end, before, tiles; };

// How many tiles of B rows the groups have, and the rows of tile n (n < 0: none).
template <int B>
__device__ inline int spans(const int32_t *offsets, int rows, int groups, int n, Span &s) {
  if (!offsets) {
    s = Span{0, n * B, rows, 0, (rows + B - 1) / B};
    return s.tiles;
  }
  int before = 0;
  for (int g0 = 0; g0 < groups; g0 += 64) {
    int first = 0, end = 0;
    const int g = g0 + lane_id();
    if (g < groups) rows_of(offsets, rows, g, first, end);
    const int mine = (end - first + B - 1) / B, upto = before + wave_incl_scan(mine);
    const uint64_t has = __ballot(upto - mine <= n && n < upto);
    if (has) {
      const int l = __ffsll((unsigned long long)has) - 1;
      s.group = g0 + l;
      s.tiles = readlane_i32(mine, l);
      s.before = readlane_i32(upto, l) - s.tiles;
      s.first = readlane_i32(first, l) + (n - s.before) * B;
      s.end = readlane_i32(end, l);
    }
    before = readlane_i32(upto, 63);
  }
  return before;
}

// The neighbour order of an XCD's workgroups (every eighth): tile t of `total`.
__device__ inline int by_xcd(int t, int total) {
  const int each = total / 8;
  return t < each * 8 ? t % 8 * each + t / 8 : t;
}
// Tile t of nq by np: bands of eight q, of a band q first, so that an L2 serves both operands.
__device__ inline void place_of(int t, int nq, int np, int &q, int &p) {
  constexpr int kBand = 8;
  const int band = t / (kBand * np), r = t - band * kBand * np, high = imin(kBand, nq - band * kBand);
  q = band * kBand + r % high;
  p = r / high;
}
// Tile t of all groups', np of P each: a group's tiles are neighbours, so that its weights come from
// memory once.  s: its rows; the result: its tile of P.
template <int B>
__device__ inline int find_tile(const int32_t *offsets, int rows, int groups, int t, int np, int total, Span &s) {
  t = by_xcd(t, total);
  spans<B>(offsets, rows, groups, t / np, s);
  int q, p;
  place_of(t - s.before * np, s.tiles, np, q, p);
  s.first += (s.before + q - t / np) * B;
  return p;
}

// Static LDS of a product: each stage of each operand is a variable of its own, so that the
// compiler sees that a stage's reads do not wait for the others' loads.
#define TOPOEP_STAGES(S)                                                                                  \
  __shared__ v4i stage_p0[S::kBytesP / 16], stage_p1[S::kBytesP / 16], stage_p2[S::kDeep ? S::kBytesP / 16 : 1]; \
  __shared__ v4i stage_q0[S::kBytesQ / 16], stage_q1[S::kBytesQ / 16];                                    \
  const Stages lds = {{(Lds *)stage_p0, (Lds *)stage_p1, S::kDeep ? (Lds *)stage_p2 : nullptr}, {(Lds *)stage_q0, (Lds *)stage_q1}}

// Four neighbours, rounded to nearest even.
template <class T>
__device__ inline void store4(void *to, int64_t at, v4f v) {
  typedef typename std::conditional<std::is_same<T, Bf16>::value, __bf16,
                                    typename std::conditional<std::is_same<T, F16>::value, _Float16, float>::type>::type E;
  typedef E v4e __attribute__((ext_vector_type(4)));
  const v4e o = __builtin_convertvector(v, v4e);
  __builtin_memcpy(static_cast<E *>(to) + at, &o, sizeof(o));
}

// A wave's 16-bit results, rows of neighbouring p (whole eights of them): two tiles of 16 at a time, whose
// halves lanes exchange, so that a lane stores 16 bytes and a row's 64 are together (with 8 bytes a lane a
// weights' gradient of 128 experts, 1536 x 2048, took 7 % longer).
template <class T>
__device__ inline v2i pack4(v4f v) {
  v2i o;
  store4<T>(&o, 0, v);
  return o;
}
// Of tiles i and i + 1: what a lane stores, and the columns (of those from tile i's first on) where.
template <class T>
__device__ inline v4i pair_of(v4f first, v4f second) {
  const v2i a = pack4<T>(first), b = pack4<T>(second);
  v4i o;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const auto x = __builtin_amdgcn_permlane16_swap((uint32_t)a[e], (uint32_t)b[e], false, false);
    o[e] = (int)x[0];
    o[e + 2] = (int)x[1];
  }
  return o;
}
__device__ inline int pair_column(Me me) { return (me.lane >> 4 & 1) * 16 + (me.lane >> 5) * 8; }

// `tiles` of them, value(i), to the columns from `c` on of the row at `to`, of which there are n.
template <class T, class FV>
__device__ inline void store_rows(Me me, int tiles, void *to, int c, int n, const FV &value) {
#pragma unroll
  for (int i = 0; i < tiles; i += 2) {
    const v4i o = pair_of<T>(value(i), value(i + 1));
    const int at = c + i * 16 + pair_column(me);
    if (at < n) *reinterpret_cast<v4i *>(static_cast<T *>(to) + at) = o;
  }
}

// Workgroups of S for at most `tiles` tiles: as many as a CU holds, which take them in turn.
template <class S>
inline unsigned grid_of(int64_t tiles) {
  const int64_t most = S::BP * S::BQ > 128 * 128 ? 256 : 512;
  return (unsigned)(tiles < most ? (tiles < 1 ? 1 : tiles) : most);
}

// Tiles of B rows at most.
template <int B>
inline int64_t most_spans(const int32_t *offsets, int rows, int groups) {
  return ((int64_t)rows + B - 1) / B + (offsets ? imin(groups, rows) : 0);
}
// And about, of `expected` rows (by groups or not; groups differ, and a quarter more leaves room for that).
inline int64_t likely_spans(bool by_groups, int64_t expected, int groups, int B) {
  if (!by_groups) return (expected + B - 1) / B;
  return (expected / B + ((expected < groups ? expected : groups) + 1) / 2) * 5 / 4;
}

// Whether tiles of 256 x 256 take less time than their number of 128 x 128: one of the former a CU,
// two of the latter, which reach 1340 and 1100 TFLOP/s (8192^3 in bf16: an inner axis of 128 stages, and the rule
// takes these rates for short ones too).
inline bool large_tiles(int64_t large, int64_t small) { return (large + 255) / 256 * 10 < (small + 511) / 512 * 6; }

inline int64_t ceil_of(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Workgroups that share a tile's inner axis, where `tiles` of 128 x 128 leave half of the chip's 512 places
// empty and every part has eight stages at least (256 rows, H = 4096, I = 11008: 210 us whole, 122 in
// parts; the weights' gradients of 16384 rows, H = 512, I = 256, a training step: 465 and 121).
inline int parts_of(int64_t tiles, int64_t stages, int most) {
  const int64_t n = tiles < 1 || tiles > 256 ? 1 : 512 / tiles, by_stages = stages / 8;
  const int64_t p = n < by_stages ? n : by_stages;
  return (int)(p < 1 ? 1 : p < most ? p : most);
}
}  // namespace topoep_dev
