// Products of a few rows on gfx950, where the weights' bytes are all that counts:
// 16 rows of P (weights) against up to 4 C of Q.
//
// Weights go from memory straight into registers, past the caches, as the matrix
// instruction's A operand.  An operand holds 4 rows, 256 neighbouring bytes of
// each (a row's four parts of 64 are rows of the instruction: memory gives 4 rows
// of 256 bytes 7.0 TB/s and 16 rows of 64 bytes 5 to 6), and Q's operand the same
// four parts of 4 columns; of the products only those of equal parts are kept,
// which costs matrix instructions that are idle anyway.
//
// KS = 1: a wave has a tile of its own; else a workgroup's KS waves share one, each with parts
// of the inner axis, which fills the chip where there are few tiles.
#pragma once

#include <type_traits>

#include "tile.h"

namespace topoep_dev {

constexpr int kFewRows = 16;          // of P
constexpr int kFewStep = 256;         // bytes of the inner axis an operand holds
constexpr int few_waves(int KS) { return KS == 1 ? 4 : KS; }
constexpr int few_per_simd(int C) { return C > 2 ? 2 : C > 1 ? 3 : 4; }   // waves, by their registers

// Of a lane: its row (column) of an operand, and its 16 bytes of a step.
struct FewPlace {
  int index, at;
  __device__ explicit FewPlace(int lane) : index(lane % 16 / 4), at(((lane >> 4) * 4 + lane % 4) * 16) {}
};

// d += P Q over the bytes [first, n) of the inner axis in steps `every` bytes apart: operand i is at row[i],
// column operand c at col[c] (both with the lane's place, at byte 0).
template <class T, int C>
__device__ inline void few_steps(const char *(&row)[4], const char *(&col)[C], int place, int first, int every, int n,
                                 typename Mul<T>::Sum (&d)[4][C]) {
  // steps whose loads are under way together, as many as leave few_per_simd its waves (128 experts, four rows on average, H =
  // 2048, I = 768: 203 us with three for C = 2, 190 so; for C = 4 no different)
  constexpr int U = C <= 2 ? 4 : 3;
  const v4i zero = {0, 0, 0, 0};
  v4i a[U][4], b[U][C];
  const auto load = [&](int k, bool whole) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // what lies behind the axis reads its start and counts as zero
      const bool in = whole || k + u * every + place < n;
      const int at = in ? k + u * every : -place;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[u][i] = __builtin_nontemporal_load(reinterpret_cast<const v4i *>(row[i] + at));
        if (!in) a[u][i] = zero;
      }
#pragma unroll
      for (int c = 0; c < C; ++c) {
        b[u][c] = *reinterpret_cast<const v4i *>(col[c] + at);
        if (!in) b[u][c] = zero;
      }
    }
  };
  const auto multiply = [&] {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i][c] = Mul<T>::add(a[u][i], b[u][c], d[i][c]);
  };
  int k = first;
#pragma unroll 1
  for (; k + (U - 1) * every + kFewStep <= n; k += U * every) {
    load(k, true);
    multiply();
  }
  if (k < n) {
    load(k, false);
    multiply();
  }
}

__device__ inline float quad_sum(float v) {
  v += dpp_movf<0xB1>(v);
  return v + dpp_movf<0x4E>(v);
}
// (whole numbers wrap round: of 2^31 its 32 bits are kept)
__device__ inline float plus(float a, float b) { return a + b; }
__device__ inline int plus(int a, int b) { return (int)((uint32_t)a + (uint32_t)b); }
__device__ inline int quad_sum(int v) {
  v = plus(v, (int)dpp_mov<0xB1>((uint32_t)v));
  return plus(v, (int)dpp_mov<0x4E>((uint32_t)v));
}

// LDS of a workgroup: each wave's sums, [row][column].
template <class E, int C, int KS>
struct FewSums { E at[few_waves(KS)][kFewRows][4 * C + 1]; };

// The products of 16 rows of P with `count` columns, n bytes of the inner axis: done(row, column,
// sum of it and of row + 8) for every column and the first `rows` rows, the waves' parts summed in their
// order.  row_at(r) and col_at(c) give addresses.
template <class T, int C, int KS, class E, class FR, class FC, class FD>
__device__ inline void few_product(const FR &row_at, const FC &col_at, int count, int n, FewSums<E, C, KS> &lds, int rows,
                                   const FD &done) {
  const int wave = uniform_i32(threadIdx.x >> 6), lane = lane_id();
  const FewPlace place(lane);
  const char *row[4], *col[C];
#pragma unroll
  for (int i = 0; i < 4; ++i) row[i] = row_at(i * 4 + place.index) + place.at;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int q = c * 4 + place.index;
    col[c] = col_at(q < count ? q : 0) + place.at;   // (columns that do not exist are column 0)
  }
  typename Mul<T>::Sum d[4][C] = {};
  few_steps<T, C>(row, col, place.at, (KS == 1 ? 0 : wave) * kFewStep, KS * kFewStep, n, d);
  const int mine = lane % 4;
  if (KS == 1) wave_sync(); else __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < C; ++c) {
      E v = d[i][c][0];
#pragma unroll
      for (int j = 1; j < 4; ++j) v = mine == j ? d[i][c][j] : v;
      v = quad_sum(v);
      if (mine == 0) lds.at[wave][i * 4 + (lane >> 4)][c * 4 + place.index] = v;
    }
  if (KS == 1) wave_sync(); else __syncthreads();
  const auto sum = [&](int r, int c) {
    E v = lds.at[KS == 1 ? wave : 0][r][c];
#pragma unroll
    for (int w = 1; w < KS; ++w) v = plus(v, lds.at[w][r][c]);
    return v;
  };
  for (int i = KS == 1 ? lane : (int)threadIdx.x; i < rows * count; i += KS == 1 ? 64 : 64 * KS) {
    const int r = i % rows, c = i / rows;
    done(r, c, sum(r, c), rows == 8 ? sum(r + 8, c) : E(0));
  }
}

// The tile of a workgroup (KS = 1: of a wave) that it starts with, and how many tiles on its next one is.
template <int KS> __device__ inline int few_first() {
  return KS == 1 ? (int)blockIdx.x * few_waves(1) + uniform_i32(threadIdx.x >> 6) : (int)blockIdx.x;
}
template <int KS> __device__ inline int few_next() { return (int)gridDim.x * (KS == 1 ? few_waves(1) : 1); }

// Calls f<C, KS> for about `rows` rows a group and `tiles` tiles in all (of 16 rows of weights): a wave has
// a tile of its own where there are enough of them, whatever the length of the inner axis.
template <class F>
inline void few_shape(int64_t rows, int64_t tiles, const F &f) {
  const auto by_ks = [&](auto c) {
    if (tiles >= 1024) f(c, std::integral_constant<int, 1>());
    else f(c, std::integral_constant<int, 8>());
  };
  if (rows <= 4) by_ks(std::integral_constant<int, 1>());
  else if (rows <= 8) by_ks(std::integral_constant<int, 2>());
  else by_ks(std::integral_constant<int, 4>());
}
// Its grid: every tile's wave at once, or enough of them to fill the chip.
template <int KS>
inline dim3 few_grid(int64_t tiles) {
  const int64_t blocks = KS == 1 ? (tiles + few_waves(1) - 1) / few_waves(1) : tiles;
  return dim3((unsigned)(blocks < 1 << 20 ? blocks : 1 << 20));
}

}  // namespace topoep_dev
