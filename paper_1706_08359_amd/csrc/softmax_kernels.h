// Softmax cross entropy over many classes, without the n_rows x n_classes scores ever being stored.
//
//   s_v = <h_d, c_v>      lse_d = log sum_v exp s_v      loss_d = lse_d - s_{y_d}
//   G_dv = w_d (exp(s_v - lse_d) - [v = y_d])      dh = scale G C      dC = scale G^T H
//
// softmax_scores_kernel multiplies a tile of rows by a tile of classes and keeps, per row, the tile's maximum and the sum of
// exponentials beneath it; softmax_join_kernel joins the tiles of a row, in order.  The gradient takes the classes in pieces:
// softmax_piece_kernel recomputes a piece's scores and stores G of that piece alone, in the operands' type, from which two
// products follow (piece_product_kernel): the piece's rows of dC, and the piece's share of dh, kept in f32 until the last.
// Recomputing costs a quarter of the operations; storing the scores instead would cost n_rows x n_classes x 4 bytes out and
// in, since a score rounded to 16 bits is off by up to 2^-8 of itself, and its exponential by as much as that times the score.
// G lies in [-w, w]: rounded to bf16 each element is off by 2^-8 of itself at most, independently.  Among many classes a row's
// label outweighs the rest of its G, and a class's own rows the rest of its column, so that the label's rounding alone would
// be as large as the result's.  What it loses is kept in f32, a number a row, and added to both products: to dh as that
// number times the label's row of C, to dC as further rows of G with that one element (label_rest).  (4,096 x 32,768 x 512:
// error of both results 0.0024 of their size without, 0.0017 with it, as much as rounding exact results.)
// Among few classes no element stands out like that.  Up to kPairClasses G goes into the products as the sum of two bf16 values,
// the rounded one and what rounding took, off by 2^-16 of an element at most; its row is padded for both, and the second
// product of so short an axis is cheap.  (4,000 rows x 2 to 128 classes x 64, labels drawn from the softmax: error 1.04 to 1.26 times that of
// rounding exact results without, 1.00 with it.)  With more classes it is 1.00 to 1.05 times as large where a row's
// probability is spread, up to 1.26 where a few classes share it; the second products would take half as long again as the whole.
// scale (1 / n_rows, as a rule) multiplies f32 sums, so it takes no part in that rounding.
//
// A row whose label is outside [0, n_classes) is ignored: loss, lse, G, gradient and hessian are zeros whatever h holds there
// (its row of H is zeros in the copy that meets G).
#pragma once

#include "leaf_product_kernels.h"

namespace gbdt_softmax {

using namespace gbdt_tile;
using gbdt_leaf::PlainRows;
using gbdt_leaf::plain_rows;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// The difference is taken first: it is exact where a score is close to its row's lse, however large both are, which
// s log2 e - lse log2 e is not.
__device__ __forceinline__ float exp_diff(float s, float base) { return __builtin_amdgcn_exp2f((s - base) * kLog2e); }
// The same without the rounding of the product: exp2(t + r) = exp2(t) (1 + r ln 2) up to r^2, where t + r is the product exactly.
// (Three more operations; for results in f32 whose kernel waits for memory.)
__device__ __forceinline__ float exp_diff_close(float s, float base) {
  const float x = s - base, t = x * kLog2e, r = __builtin_fmaf(x, kLog2e, -t), e = __builtin_amdgcn_exp2f(t);
  const float more = __builtin_fmaf(e, r * kLn2, e);
  return __builtin_isfinite(t) ? more : e;
}
// What a running maximum is subtracted as: exponentials beneath an infinite one are 0 or infinite, not inf - inf.
__device__ __forceinline__ float base_of(float m) { return __builtin_isinf(m) ? 0.0f : m; }

// Classes of a maximum and a sum, whatever the tile.
template <typename T>
constexpr int kPartClasses = sizeof(T) == 2 ? 128 : 64;

// Classes up to which bf16 G is kept as two values; the second ones lie this far behind the first.
constexpr int kPairClasses = 128;

struct MaxSum {
  float m, s;
};
__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b) {
  // a NaN in either sum or maximum stays in the sum
  const float m = fmaxf(a.m, b.m), base = base_of(m);
  return {m, a.s * exp_diff(a.m, base) + b.s * exp_diff(b.m, base)};
}

template <typename T>
struct ScoreArgs {
  const T* h;  // [n_rows][dim]
  const T* c;  // [n_classes][dim]
  const int32_t* labels;  // [n_rows] or null
  const float* lse;       // [n_rows]
  const float* weight;    // [n_rows] or null
  MaxSum* parts;          // [ceil(n_classes / kPartClasses<T>)][n_rows]
  float* picked;          // [n_rows]: the label's score
  float* rest;            // [n_rows]: what rounding took from the label's element of G, or null
  T* g;                   // [n_rows][ld_g]: G of the classes begin .. end, zeros behind; PAIR: kPairClasses, and as many rests
  float* grad;            // [end - begin][ld_out]
  float* hess;
  int64_t ld_h, ld_c, ld_g, ld_out;
  int32_t n_rows, n_classes, dim, begin, end;
  uint32_t row_tiles, col_tiles, group;
};

// A tile's place: `group` row tiles side by side go through all column tiles before the next ones do, so that what runs at
// the same time on an XCD shares both operands in its L2.
template <typename Args>
__device__ __forceinline__ void tile_place(const Args& g, uint32_t tile, uint32_t* row, uint32_t* col) {
  const uint32_t t = xcd_tile(tile, g.row_tiles * g.col_tiles);
  const uint32_t span = g.group * g.col_tiles;
  const uint32_t first = t / span * g.group;
  const uint32_t rows = g.row_tiles - first < g.group ? g.row_tiles - first : g.group;
  *row = first + t % span % rows;
  *col = t % span / rows;
}

// The scores of one tile after another (the grid is a multiple of 8, or one workgroup a tile: a workgroup's tiles are its
// XCD's), each handed to `use` with what `fetch` read for its rows and its first row and class.  The next tile's first steps
// are on their way while `use` works; `fetch` comes before them, since loads are waited for in order.
template <class S, bool N_INNER, typename T, class Fetch, class Use>
__device__ __forceinline__ void for_score_tiles(char* lds, const ScoreArgs<T>& g, const Fetch& fetch, const Use& use) {
  const PlainRows<T> rows_a = plain_rows(g.h, g.ld_h, g.n_rows, g.dim);
  const PlainRows<T> rows_b = plain_rows(g.c, g.ld_c, g.end, g.dim);
  typename S::RowsA a;
  typename S::RowsB b;
  const uint32_t tiles = g.row_tiles * g.col_tiles;
  int row0, col0;
  auto begin = [&](uint32_t tile) {
    uint32_t tr, tc;
    tile_place(g, tile, &tr, &tc);
    row0 = (int)tr * S::BM;
    col0 = g.begin + (int)tc * S::BN;
    a.init(rows_a, row0, 0, 0, g.dim);
    b.init(rows_b, col0, 0, 0, g.dim);
    tile_begin<S>(lds, a, b, rows_a, rows_b, 0, g.dim);
  };
  uint32_t tile = blockIdx.x;
  begin(tile);
  for (;;) {
    f32x4 acc[S::TM][S::TN];
    zeros<S>(acc);
    tile_run<S, N_INNER>(lds, a, b, rows_a, rows_b, 0, g.dim, acc, Nothing{});
    const int row = row0, col = col0;
    const auto of_rows = fetch(row);
    const uint32_t next = tile + gridDim.x;
    if (next < tiles) begin(next);
    use(acc, of_rows, row, col);
    if (next >= tiles) return;
    tile = next;
  }
}

// What an epilogue needs of the rows of its lane's blocks; all of it is asked for at once (one at a time, block by block, it
// cost more than everything else behind the products).  Rows past the last stand for an ignored one.
template <class S>
struct OfRows {
  int y[S::TM];
  float lse[S::TM], weight[S::TM];
};

// Bound by the matrix cores for many rows and by the read of c for few; a lane's values meet in its registers, lanes of a row
// through local memory, once a tile.  The exponentials are the next cost, one for every `dim` products, so that 512
// dimensions reach less of the rate than 1,024.  (8,192 x 65,536 x 1,024 bf16: 900 to 1,000 us, 1.1 to 1.2 PFLOP/s, the less the warmer
// the card, matrix cores busy for 57 % of the cycles; 4,096 x 32,768 x 512: 136 to 146, 0.94 to 1.0, 43 %; one row of 50,000 x 512: 14
// us, 3.7 TB/s; 1,537 x 10,007 x 137 f32, no whole chunks: 67 us, 63 TFLOP/s, 50 %.)
template <class S>
__global__ void __launch_bounds__(S::NT, 2) softmax_scores_kernel(const ScoreArgs<typename S::T> g) {
  __shared__ __align__(16) char lds[S::kLdsBytes];
  // [a part's classes: their wavefronts' lane groups][row]: the maximum and the sum of a lane's 4 TN values of a row
  __shared__ MaxSum lane_parts[S::WN * 4 * S::BM];
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int m0 = (w / S::WN) * (S::TM * 16) + (l & 15), wave_n = (w % S::WN) * (S::TN * 16) + 4 * (l >> 4);
  MaxSum* mine = lane_parts + (w % S::WN * 4 + (l >> 4)) * S::BM;
  auto fetch = [&](int row0) {
    OfRows<S> f;
#pragma unroll
    for (int i = 0; i < S::TM; ++i) {
      const int d = row0 + m0 + 16 * i;
      f.y[i] = g.labels ? g.labels[d < g.n_rows ? d : g.n_rows - 1] : -1;
    }
    return f;
  };
  for_score_tiles<S, true>(lds, g, fetch, [&](f32x4(&acc)[S::TM][S::TN], const OfRows<S>& f, int row0, int col0) {
    const int n0 = col0 + wave_n;
    if (col0 + S::BN > g.end) {  // classes past the last add nothing to either
#pragma unroll
      for (int i = 0; i < S::TM; ++i)
#pragma unroll
        for (int j = 0; j < S::TN; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[i][j][r] = n0 + 16 * j + r < g.end ? acc[i][j][r] : -__builtin_inff();
    }
#pragma unroll
    for (int i = 0; i < S::TM; ++i) {
      float top = acc[i][0][0];
#pragma unroll
      for (int j = 0; j < S::TN; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) top = fmaxf(top, acc[i][j][r]);
      const float base = base_of(top);
      float sum = 0.0f;
#pragma unroll
      for (int j = 0; j < S::TN; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) sum += exp_diff(acc[i][j][r], base);
      mine[m0 + 16 * i] = {top, sum};
    }
#pragma unroll
    for (int i = 0; i < S::TM; ++i) {
      const int rel = f.y[i] - n0, d = row0 + m0 + 16 * i;  // rarely here
      if (rel >= 0 && rel < 16 * S::TN && (rel & 15) < 4 && f.y[i] < g.end && d < g.n_rows) {
        float picked = 0.0f;
#pragma unroll
        for (int j = 0; j < S::TN; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) picked = rel == 16 * j + r ? acc[i][j][r] : picked;
        g.picked[d] = picked;
      }
    }
    __syncthreads();  // (the next tile's steps, with their barriers, come before these places are written again)
    constexpr int part = kPartClasses<typename S::T>;
    constexpr int lanes = 4 * part / (S::TN * 16);  // of a row in a part
    static_assert(S::BN % part == 0 && lanes >= 4, "tiles of whole parts");
    for (int e = threadIdx.x; e < S::BM * (S::BN / part); e += S::NT) {
      const int m = e % S::BM, q = e / S::BM;
      if (row0 + m >= g.n_rows || col0 + q * part >= g.end) continue;
      MaxSum p = lane_parts[q * lanes * S::BM + m];
#pragma unroll
      for (int k = 1; k < lanes; ++k) p = join(p, lane_parts[(q * lanes + k) * S::BM + m]);
      g.parts[((int64_t)(col0 / part) + q) * g.n_rows + row0 + m] = p;
    }
  });
}

// Joins a row's parts: 256 / ROWS lanes a row, each every so manieth part in order, then pairwise.  16 rows a workgroup read
// whole lines; one row a workgroup has 391 parts (50,000 classes) joined in 3 us where 16 lanes take 12.
template <int ROWS>
__global__ void __launch_bounds__(256) softmax_join_kernel(const MaxSum* parts, const float* picked, const int32_t* labels, int32_t n_rows,
                                                           int32_t n_classes, int32_t tiles, float* loss, float* lse) {
  constexpr int lanes = 256 / ROWS;
  const int i = threadIdx.x % ROWS, q = threadIdx.x / ROWS;  // row of the workgroup, turn
  __shared__ MaxSum all[lanes][ROWS + (ROWS > 1)];
  const int d = blockIdx.x * ROWS + i;
  MaxSum p = {-__builtin_inff(), 0.0f};
  if (d < n_rows)
    for (int t = q; t < tiles; t += lanes) p = join(p, parts[(int64_t)t * n_rows + d]);
  all[q][i] = p;
  __syncthreads();
  for (int k = lanes / 2; k > 0; k >>= 1) {
    if (q < k) all[q][i] = join(all[q][i], all[q + k][i]);
    __syncthreads();
  }
  if (q != 0 || d >= n_rows) return;
  p = all[0][i];
  const float z = base_of(p.m) + kLn2 * __builtin_amdgcn_logf(p.s);
  const bool use = labels == nullptr || (uint32_t)labels[d] < (uint32_t)n_classes;
  lse[d] = use ? z : 0.0f;
  if (loss) loss[d] = use ? z - picked[d] : 0.0f;
}

// The scores again, and G of a piece, stored in whole lines.  Bound by the same, and by the stores of G (for every `dim` products
// one exponential and one stored value): 8,192 x 65,536 x 1,024 bf16 in two pieces, 587 us each, 0.94 PFLOP/s and 0.9 TB/s of G,
// matrix cores busy for 44 % of the cycles.
// PAIR: one tile holds all classes, and what rounding takes from them is stored behind them.
template <class S, bool PAIR>
__global__ void __launch_bounds__(S::NT, 2) softmax_piece_kernel(const ScoreArgs<typename S::T> g) {
  typedef typename S::T T;
  __shared__ __align__(16) char lds[S::kLdsBytes];
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int m0 = (w / S::WN) * (S::TM * 16) + (l & 15), wave_n = (w % S::WN) * (S::TN * 16) + 4 * (l >> 4);
  auto fetch = [&](int row0) {
    OfRows<S> f;
#pragma unroll
    for (int i = 0; i < S::TM; ++i) {
      const int d = row0 + m0 + 16 * i, at = d < g.n_rows ? d : g.n_rows - 1;
      f.y[i] = g.labels[at];
      f.lse[i] = g.lse[at];
      f.weight[i] = g.weight ? g.weight[at] : 1.0f;
    }
    return f;
  };
  for_score_tiles<S, true>(lds, g, fetch, [&](f32x4(&acc)[S::TM][S::TN], const OfRows<S>& f, int row0, int col0) {
    const int n0 = col0 + wave_n;
#pragma unroll
    for (int i = 0; i < S::TM; ++i) {
      const int y = f.y[i];
      const bool use = (uint32_t)y < (uint32_t)g.n_classes;
#pragma unroll
      for (int j = 0; j < S::TN; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[i][j][r] = f.weight[i] * exp_diff(acc[i][j][r], f.lse[i]);
      const int rel = y - n0;  // rarely here
      if (rel >= 0 && rel < 16 * S::TN && (rel & 15) < 4) {
#pragma unroll
        for (int j = 0; j < S::TN; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[i][j][r] -= rel == 16 * j + r ? f.weight[i] : 0.0f;
        if (g.rest && use && row0 + m0 + 16 * i < g.n_rows) {
          float of_label = 0.0f;
#pragma unroll
          for (int j = 0; j < S::TN; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) of_label = rel == 16 * j + r ? acc[i][j][r] : of_label;
          g.rest[row0 + m0 + 16 * i] = of_label - (float)(T)of_label;
        }
      }
      if (!use || col0 + S::BN > g.end) {
#pragma unroll
        for (int j = 0; j < S::TN; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[i][j][r] = use && n0 + 16 * j + r < g.end ? acc[i][j][r] : 0.0f;
      }
    }
    const int wave_row = row0 + (w / S::WN) * (S::TM * 16);
    auto row = [&](int i, int r) {
      const int d = wave_row + 16 * i + r;
      return d < g.n_rows ? g.g + (int64_t)d * g.ld_g - g.begin : (T*)nullptr;
    };
    const int wave_col = n0 - 4 * (l >> 4), cols = PAIR ? kPairClasses : g.begin + (int)g.ld_g;
    store_tile<S, T, S::TM, S::TN>(lds + S::kLastStage, [&](int i, int j) { return acc[i][j]; }, row, wave_col, cols);
    if constexpr (PAIR) {
      static_assert(S::BN == kPairClasses, "one tile of all classes");
      store_tile<S, T, S::TM, S::TN>(
          lds + S::kLastStage,
          [&](int i, int j) {
            f32x4 v = acc[i][j];
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] -= (float)(T)v[r];
            return v;
          },
          [&](int i, int r) {
            T* to = row(i, r);
            return to != nullptr ? to + kPairClasses : to;
          },
          wave_col, cols);
    }
  });
}

// Two columns of f32 a score are stored, which bounds it up to some hundred dimensions: accumulators are transposed on their way
// out, so that a column's rows leave as whole lines.  (16 classes of 400,000 x 64 f32: 31 us, 5.0 TB/s of what it reads and
// writes, some of it from the last-level cache; 1,023 of 10,000 x 256 bf16: 28 us, 3.1 TB/s; matrix cores busy for 14 and 6 %.)
template <class S>
__global__ void __launch_bounds__(S::NT, 2) softmax_stats_kernel(const ScoreArgs<typename S::T> g) {
  __shared__ __align__(16) char lds[S::kLdsBytes];
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int m0 = (w / S::WN) * (S::TM * 16) + 4 * (l >> 4), wave_n = (w % S::WN) * (S::TN * 16) + (l & 15);
  struct OfFourRows {
    float lse[S::TM][4];
    int y[S::TM][4];
  };
  auto fetch = [&](int row0) {
    OfFourRows f;
#pragma unroll
    for (int i = 0; i < S::TM; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int d = row0 + m0 + 16 * i + r, at = d < g.n_rows ? d : g.n_rows - 1;
        f.lse[i][r] = g.lse[at];
        f.y[i][r] = g.labels ? g.labels[at] : -1;
      }
    return f;
  };
  for_score_tiles<S, false>(lds, g, fetch, [&](f32x4(&acc)[S::TM][S::TN], const OfFourRows& f, int row0, int col0) {
    const int n0 = col0 + wave_n;
    // p in place of the scores
#pragma unroll
    for (int i = 0; i < S::TM; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const bool use = g.labels == nullptr || (uint32_t)f.y[i][r] < (uint32_t)g.n_classes;
#pragma unroll
        for (int j = 0; j < S::TN; ++j) {
          const float e = exp_diff_close(acc[i][j][r], f.lse[i][r]);
          acc[i][j][r] = use ? e : 0.0f;
        }
      }
    const int wave_row = row0 + (w / S::WN) * (S::TM * 16);
    auto column = [&](float* out) {
      return [&g, out, n0, l](int j, int c) {
        const int n = n0 - (l & 15) + 16 * j + c;
        return n < g.end ? out + (int64_t)(n - g.begin) * g.ld_out : (float*)nullptr;
      };
    };
    store_tile<S, float, S::TN, S::TM>(
        lds + S::kLastStage, [&](int j, int i) { return acc[i][j] * (1.0f - acc[i][j]); }, column(g.hess), wave_row, g.n_rows);
    store_tile<S, float, S::TN, S::TM>(
        lds + S::kLastStage,
        [&](int j, int i) {
          f32x4 v = acc[i][j];
#pragma unroll
          for (int r = 0; r < 4; ++r) v[r] = n0 + 16 * j == f.y[i][r] ? v[r] - 1.0f : v[r];
          return v;
        },
        column(g.grad), wave_row, g.n_rows);
  });
}

// A copy whose rows are whole 16-byte chunks, filled up with zeros; rows whose label does not count (labels given) are all
// zeros.  What meets G must be so: G is zero in a row that does not count, but h there may be anything, and 0 x NaN is not 0.
// Bound by memory: 8,192 x 1,024 bf16 in 8 us, 4.2 TB/s.
template <typename T>
__global__ void __launch_bounds__(256) whole_rows_kernel(const T* from, int64_t ld, T* to, int32_t rows, int32_t cols, const int32_t* labels,
                                                         int32_t n_classes) {
  const uint32_t per = (uint32_t)(cols + kChunk<T> - 1) / kChunk<T>;
  const uint64_t n = (uint64_t)rows * per;
  for (uint64_t e = (uint64_t)blockIdx.x * 256 + threadIdx.x; e < n; e += (uint64_t)gridDim.x * 256) {
    const uint32_t r = (uint32_t)(e / per), c = (uint32_t)(e - (uint64_t)r * per) * kChunk<T>;
    u32x4 v = {0, 0, 0, 0};
    if (labels == nullptr || (uint32_t)labels[r] < (uint32_t)n_classes) {
      const T* p = from + (int64_t)r * ld + c;
      const int valid = cols - (int)c;
      if (valid >= kChunk<T>) {
        __builtin_memcpy(&v, p, 16);
      } else {
        v = last_chunk<T>(p, valid);
      }
    }
    *(u32x4*)(to + e * kChunk<T>) = v;
  }
}

// ---------------------------------------------------------------- the products with G

template <typename T>
struct PieceArgs {
  const T* a;  // G of the piece
  const T* b;  // C of the piece (dh) or H (dC)
  T* out;      // the result, if it is written here
  float* sums; // [splits][rows][cols] f32, otherwise
  const int32_t* labels;
  const float* rest;   // of the labels' elements of G, or null
  const T* c;          // all of C (dh)
  int64_t ld_a, ld_b, ld_out, ld_c;
  int32_t class0;      // the piece's first class
  float scale;
  int32_t rows, cols, k, n_classes;  // of the result; the summed axis
  int32_t k_split;                   // of the summed axis a workgroup takes, whole steps
  int32_t b_rows, b_cols;            // of b: k may pass its rows by the zeros behind G's classes; whole chunks of columns
  int32_t add;                       // sums hold earlier pieces' shares
  uint32_t row_tiles, col_tiles, splits, group;
};

template <typename T>
__device__ __forceinline__ bool counts(const PieceArgs<T>& g, int row) {
  return (uint32_t)g.labels[row] < (uint32_t)g.n_classes;
}

constexpr int kListed = 1536;  // rows of a list in local memory

// A list in local memory, as the rows of an operand.
struct Listed {
  static constexpr bool kEven = false;
  const __attribute__((address_space(3))) int* words;
  __device__ __forceinline__ int fetch(int k) const { return words[k]; }
};

// Adds rest[d] h_d to the tile's row of class labels[d], for the rows k0 <= d < k1 whose label is among the tile's classes: the
// rows are listed, in an order that hangs on their numbers alone, and multiplied like any others, by a G of one element a row.
template <class S>
__device__ __forceinline__ void label_rest(char* lds, const PieceArgs<typename S::T>& g, int row0, int col0, int k0, int k1,
                                           f32x4 (&acc)[S::TM][S::TN]) {
  typedef typename S::T T;
  constexpr int each = 1024 / S::NT, waves = S::NT / 64;  // labels a thread reads at a time
  static_assert(each >= 1 && kListed >= 1024, "one reading fits the list");
  __shared__ int ids[kListed + 64], values[kListed + 64], wave_n[waves];
  const int t = threadIdx.x, l = t & 63, w = t >> 6;
  const int first = g.class0 + row0, classes = g.rows - row0 < S::BM ? g.rows - row0 : S::BM;
  int count = 0;
  auto flush = [&]() {
    if (count == 0) return;
    for (int i = count + t; i < (count + 63) / 64 * 64; i += S::NT) ids[i] = values[i] = -1;
    __syncthreads();
    const Listed rows_a = {(const __attribute__((address_space(3))) int*)values};
    const gbdt_leaf::CopiedRows<T> rows_b = {g.b, nullptr, g.ld_b, (const __attribute__((address_space(3))) int*)ids, 0};
    OneHotOperand<S::BM, S::NT, S::KB> a;
    typename S::ColumnsB b;
    a.init(rows_a, 0, count);
    b.init(rows_b, col0, g.b_cols, 0, count);
    tile_begin<S>(lds, a, b, rows_a, rows_b, 0, count);
    tile_run<S, true>(lds, a, b, rows_a, rows_b, 0, count, acc, Nothing{});
    __syncthreads();
    count = 0;
  };
  for (int base = k0; base < k1; base += 1024) {
    int at[each], before = 0, mine[each];
#pragma unroll
    for (int i = 0; i < each; ++i) {
      const int d = base + i * S::NT + t;
      at[i] = d < k1 ? g.labels[d] - first : -1;
      if ((uint32_t)at[i] >= (uint32_t)classes) at[i] = -1;
      const uint64_t found = __ballot(at[i] >= 0);
      mine[i] = before + __popcll(found & ((1ull << l) - 1));
      before += __popcll(found);
    }
    if (l == 0) wave_n[w] = before;
    __syncthreads();
    int total = 0, mine_first = 0;
#pragma unroll
    for (int i = 0; i < waves; ++i) {
      mine_first += i < w ? wave_n[i] : 0;
      total += wave_n[i];
    }
    total = __builtin_amdgcn_readfirstlane(total);
    if (count + total > kListed) flush();
#pragma unroll
    for (int i = 0; i < each; ++i) {
      if (at[i] < 0) continue;
      const int d = base + i * S::NT + t, to = count + mine_first + mine[i];
      const T rest = (T)g.rest[d];
      uint16_t bits;
      __builtin_memcpy(&bits, &rest, 2);
      ids[to] = d;
      values[to] = at[i] << 16 | bits;
    }
    count += total;
    __syncthreads();
  }
  flush();
}

// TO_ROWS: dh (the result's rows are G's rows, k = classes); otherwise dC (its rows are classes, k = G's rows).
// Bound by the matrix cores and what feeds them: 8,192 x 65,536 x 1,024 bf16, a product in two pieces, dC 877 us, 1.25 PFLOP/s, matrix
// cores busy for 63 % of the cycles, dh 948, 1.16, 57 %; 1,537 x 10,007 x 137 f32: 71 and 76 us, 59 and 56 TFLOP/s, 53 and 51 % (137
// columns take three tiles of 64).
// PAIR: what rounding took from G, which lies behind it, is multiplied as well.
template <class S, bool TO_ROWS, bool PAIR>
__global__ void __launch_bounds__(S::NT, 2) piece_product_kernel(const PieceArgs<typename S::T> g) {
  typedef typename S::T T;
  __shared__ __align__(16) char lds[S::kLdsBytes];
  const uint32_t t = xcd_tile(blockIdx.x, gridDim.x);
  const uint32_t tiles = g.row_tiles * g.col_tiles;
  const uint32_t split = t / tiles, u = t % tiles;
  const uint32_t span = g.group * g.col_tiles, first = u / span * g.group;
  const uint32_t in = g.row_tiles - first < g.group ? g.row_tiles - first : g.group;
  const int row0 = (int)(first + u % span % in) * S::BM, col0 = (int)(u % span / in) * S::BN;
  const int k0 = (int)split * g.k_split;
  const int k1 = g.k - k0 < g.k_split ? g.k : k0 + g.k_split;
  f32x4 acc[S::TM][S::TN];
  typename S::ColumnsB b;
  if constexpr (TO_ROWS) {
    const PlainRows<T> rows_a = plain_rows(g.a, g.ld_a, g.rows, (int)g.ld_a);
    const PlainRows<T> rows_b = plain_rows(g.b, g.ld_b, g.b_rows, g.cols);
    typename S::RowsA a;
    a.init(rows_a, row0, 0, k0, k1);
    b.init(rows_b, col0, g.b_cols, k0, k1 < g.b_rows ? k1 : g.b_rows);
    tile_product<S, true>(lds, a, b, rows_a, rows_b, k0, k1, acc, Nothing{});
    if constexpr (PAIR) {
      const PlainRows<T> rests = plain_rows(g.a + kPairClasses, g.ld_a, g.rows, kPairClasses);
      a.init(rests, row0, 0, k0, k1);
      b.init(rows_b, col0, g.b_cols, k0, k1 < g.b_rows ? k1 : g.b_rows);
      tile_begin<S>(lds, a, b, rests, rows_b, k0, k1);
      tile_run<S, true>(lds, a, b, rests, rows_b, k0, k1, acc, Nothing{});
    }
  } else {
    const PlainRows<T> rows_a = plain_rows(g.a, g.ld_a, g.k, (int)g.ld_a);
    const PlainRows<T> rows_b = plain_rows(g.b, g.ld_b, g.b_rows, g.cols);
    typename S::ColumnsA a;
    a.init(rows_a, row0, (g.rows + kChunk<T> - 1) / kChunk<T> * kChunk<T>, k0, k1);  // G is zero up to ld_a
    b.init(rows_b, col0, g.b_cols, k0, k1);
    tile_product<S, true>(lds, a, b, rows_a, rows_b, k0, k1, acc, Nothing{});
    if constexpr (PAIR) {
      const PlainRows<T> rests = plain_rows(g.a + kPairClasses, g.ld_a, g.k, kPairClasses);
      a.init(rests, row0, (g.rows + kChunk<T> - 1) / kChunk<T> * kChunk<T>, k0, k1);
      b.init(rows_b, col0, g.b_cols, k0, k1);
      tile_begin<S>(lds, a, b, rests, rows_b, k0, k1);
      tile_run<S, true>(lds, a, b, rests, rows_b, k0, k1, acc, Nothing{});
    } else if constexpr (sizeof(T) == 2) label_rest<S>(lds, g, row0, col0, k0, k1, acc);
  }
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int m0 = row0 + (w / S::WN) * (S::TM * 16), wave_col = col0 + (w % S::WN) * (S::TN * 16);
  if (!g.sums) {
    if constexpr (TO_ROWS && sizeof(T) == 2 && !PAIR) {
#pragma unroll
      for (int i = 0; i < S::TM; ++i) {
        const int m = m0 + 16 * i + (l & 15);
        if (m >= g.rows || !counts(g, m)) continue;
        const float rest = g.rest[m];
        const T* c = g.c + (int64_t)g.labels[m] * g.ld_c;
#pragma unroll
        for (int j = 0; j < S::TN; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int n = wave_col + 16 * j + 4 * (l >> 4) + r;
            if (n < g.cols) acc[i][j][r] = __builtin_fmaf(rest, (float)c[n], acc[i][j][r]);
          }
      }
    }
    store_tile<S, T, S::TM, S::TN>(
        lds + S::kLastStage, [&](int i, int j) { return g.scale * acc[i][j]; },
        [&](int i, int r) {
          const int m = m0 + 16 * i + r;
          return m < g.rows && (!TO_ROWS || counts(g, m)) ? g.out + (int64_t)m * g.ld_out : (T*)nullptr;
        },
        wave_col, g.cols);
    if (TO_ROWS) {  // rows that do not count are zeros, whatever C holds
#pragma unroll
      for (int i = 0; i < S::TM; ++i) {
        const int m = m0 + 16 * i + (l & 15);
        if (m >= g.rows || counts(g, m)) continue;
#pragma unroll
        for (int j = 0; j < S::TN; ++j) {
          const int n = wave_col + 16 * j + 4 * (l >> 4);
          if (n < g.cols) store4(g.out + (int64_t)m * g.ld_out + n, f32x4{0.0f, 0.0f, 0.0f, 0.0f}, g.cols - n);
        }
      }
    }
    return;
  }
  float* sums = g.sums + (int64_t)split * g.rows * g.cols;
#pragma unroll
  for (int i = 0; i < S::TM; ++i) {
    const int m = m0 + 16 * i + (l & 15), n0 = wave_col + 4 * (l >> 4);
    if (m >= g.rows) continue;
    float* to = sums + (int64_t)m * g.cols + n0;
    if (g.add && n0 + 16 * (S::TN - 1) + 4 <= g.cols) {  // all of a row's loads, then its stores
      f32x4 v[S::TN];
#pragma unroll
      for (int j = 0; j < S::TN; ++j) __builtin_memcpy(&v[j], to + 16 * j, 16);
#pragma unroll
      for (int j = 0; j < S::TN; ++j) store4(to + 16 * j, v[j] + acc[i][j], 4);
      continue;
    }
#pragma unroll
    for (int j = 0; j < S::TN; ++j) {
      const int n = n0 + 16 * j;
      if (n >= g.cols) continue;
      f32x4 v = acc[i][j];
      if (g.add) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (n + r < g.cols) v[r] += to[16 * j + r];
      }
      store4(to + 16 * j, v, g.cols - n);
    }
  }
}

// out = scale * sums over the splits, in order.  labels given (dh): rows that do not count are zeros, and the labels' rests are
// added.  Bound by memory: 8,192 x 1,024, one sum of f32 and the labels' rows of C in 19 us, 3.5 TB/s.
template <typename T>
__global__ void __launch_bounds__(256) piece_join_kernel(const PieceArgs<T> g) {
  const uint32_t per = (uint32_t)(g.cols + 3) / 4;  // four columns a thread
  const uint64_t n = (uint64_t)g.rows * per, all = (uint64_t)g.rows * g.cols;
  for (uint64_t e = (uint64_t)blockIdx.x * 256 + threadIdx.x; e < n; e += (uint64_t)gridDim.x * 256) {
    const uint32_t m = (uint32_t)(e / per), c = (uint32_t)(e - (uint64_t)m * per) * 4;
    const int valid = g.cols - (int)c;
    const float* from = g.sums + (uint64_t)m * g.cols + c;
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    for (uint32_t k = 0; k < g.splits; ++k) {
      f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
      if (valid >= 4) {
        __builtin_memcpy(&v, from + k * all, 16);
      } else {
#pragma unroll
        for (int r = 0; r < 3; ++r)
          if (r < valid) v[r] = from[k * all + r];
      }
      s += v;
    }
    const int y = g.labels ? g.labels[m] : 0;
    const bool use = g.labels == nullptr || (uint32_t)y < (uint32_t)g.n_classes;
    if (use && g.labels && g.rest) {
      const float rest = g.rest[m];
      const T* of = g.c + (int64_t)y * g.ld_c + c;  // (rows of whole chunks: four values are there)
      T t[4];
      __builtin_memcpy(t, of, sizeof t);
#pragma unroll
      for (int r = 0; r < 4; ++r) s[r] = __builtin_fmaf(rest, (float)t[r], s[r]);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) s[r] = use ? g.scale * s[r] : 0.0f;
    store4(g.out + (int64_t)m * g.ld_out + c, s, valid);
  }
}

}  // namespace gbdt_softmax
