// Which tiles a product has whose rows belong to groups (experts), and how its
// operands are reached.
#pragma once

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

// A tile of rows: `first` .. `end` - 1 are what is left of its group from its first on.
struct Span { int group, first, end; };

// How many tiles of B rows the groups have, and the rows of tile n (n < 0: none).
template <int B>
__device__ inline int spans(const int32_t *offsets, int rows, int groups, int n, Span &s) {
  if (!offsets) {
    s = Span{0, n * B, rows};
    return (rows + B - 1) / B;
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
      s.first = readlane_i32(first, l) + (n - (readlane_i32(upto, l) - readlane_i32(mine, l))) * B;
      s.end = readlane_i32(end, l);
    }
    before = readlane_i32(upto, 63);
  }
  return before;
}

// Tile t of nq by np: bands of eight q, of a band q first.  The tiles of an XCD (every eighth
// workgroup) are neighbours, so that its L2 serves both operands.
__device__ inline void place_of(int t, int nq, int np, int &q, int &p) {
  constexpr int kBand = 8;
  const int total = nq * np, each = total / 8;
  if (t < each * 8) t = t % 8 * each + t / 8;
  const int band = t / (kBand * np), r = t - band * kBand * np, high = imin(kBand, nq - band * kBand);
  q = band * kBand + r % high;
  p = r / high;
}

// Static LDS of a product: two stages of each operand, variables of their own, so
// that the compiler sees that a stage's reads do not wait for the other's loads.
#define TOPOEP_STAGES(S)                                                                 \
  __shared__ v4i stage_p0[S::BP * kLine / 16], stage_p1[S::BP * kLine / 16];             \
  __shared__ v4i stage_q0[S::BQ * kLine / 16], stage_q1[S::BQ * kLine / 16];             \
  Lds *const p0 = (Lds *)stage_p0, *const p1 = (Lds *)stage_p1, *const q0 = (Lds *)stage_q0, *const q1 = (Lds *)stage_q1

// An operand by rows: row(r) gives the address of tile row r.
template <class S, class O, class F>
__device__ inline void by_rows(O &o, int wave, const F &row) {
  o.step = kLine;
#pragma unroll
  for (int i = 0; i < O::kLoads; ++i) o.from[i] = row(o.row_of(i, wave)) + o.piece_of(i, wave) * 16;
}
// An operand across: `base` its first row of the inner axis, ld elements apart; of its `n` columns those
// from c0 on (a column that does not exist is column 0).
template <class S, class O>
__device__ inline void across(O &o, int wave, const void *base, int64_t ld, int c0, int n) {
  o.step = kAcross * ld * 2;
#pragma unroll
  for (int i = 0; i < O::kLoads; ++i) {
    const int c = c0 + o.piece_of(i, wave) * 8;
    o.from[i] = static_cast<const char *>(base) + (o.row_of(i, wave) * ld + (c < n ? c : 0)) * 2;
  }
}

template <class T>
__device__ inline void store4(void *to, int64_t at, v4f v) {
  T o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = from_float<T>(v[i]);
  __builtin_memcpy(static_cast<T *>(to) + at, o, sizeof(o));
}

// Workgroups for at most `tiles` tiles: two a CU, which take them in turn.
inline unsigned grid_of(int64_t tiles) { return (unsigned)(tiles < 512 ? (tiles < 1 ? 1 : tiles) : 512); }

// Tiles of B rows at most.
template <int B>
inline int64_t most_spans(const int32_t *offsets, int rows, int groups) {
  return ((int64_t)rows + B - 1) / B + (offsets ? imin(groups, rows) : 0);
}

}  // namespace topoep_dev
