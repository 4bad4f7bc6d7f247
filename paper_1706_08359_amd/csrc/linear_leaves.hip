// Linear leaves and the softmax over many classes: host side of gbdt_leaf_product, gbdt_leaf_product_grad,
// gbdt_softmax_loss, gbdt_softmax_grad and gbdt_softmax_stats (checks, choice of tile, scratch, launches).  The kernels are
// in leaf_product_kernels.h and softmax_kernels.h, the tile that all of them share in tile_product.h.
#include <hip/hip_runtime.h>

#include <stdint.h>
#include <stdio.h>

#include <algorithm>
#include <type_traits>

#include "../../include/gbdt_hist.h"
#include "library_state.h"

#include "product_host.h"
#include "softmax_kernels.h"

namespace {

using namespace gbdt_host;

// ---------------------------------------------------------------- leaves

int leaf_check(int64_t n_positions, int32_t n_leaves, int64_t n_rows, int32_t d_in, int32_t d_out, const void* row_idx,
               const void* offsets, int32_t dtype) {
  if (n_positions < 0 || n_leaves <= 0 || n_rows < 0 || d_in <= 0 || d_out <= 0 || !offsets) return GBDT_EINVAL;
  if (((uintptr_t)offsets & 7) != 0 || ((uintptr_t)row_idx & 3) != 0) return GBDT_EINVAL;
  if (dtype != GBDT_F32 && dtype != GBDT_BF16) return GBDT_EINVAL;
  if (!row_idx && n_positions > n_rows) return GBDT_EINVAL;
  if (n_positions >= kMaxRows || n_rows >= kMaxRows || n_leaves >= kMaxWidth || d_in >= kMaxWidth || d_out >= kMaxWidth)
    return GBDT_EUNSUPPORTED;
  return GBDT_OK;
}

template <class S, typename T>
int launch_leaf_product(gbdt_leaf::LeafArgs<T>& g, hipStream_t s) {
  return leaf_rows_launches<S>(g, g.d_out, S::NT, true, [&](dim3 blocks) {
    gbdt_leaf::leaf_product_kernel<S><<<blocks, dim3(S::NT), 0, s>>>(g);
  });
}

// So few answers that a wavefront for every few of them takes less than tiles, whose rows are mostly empty then: four
// positions, or up to 2,048 with 16,384 outputs altogether (up to 64 of them twice that where rows are no whole chunks, which cost
// tiles more).  Where leaves have fewer than four positions on average, each has a tile of its own, and it is 64 positions whatever
// the outputs, or twice as many outputs (f32: four times).  (255 leaves, 2,000 -> 256: 64 positions in 12.5 us against 34 in
// tiles, f32 19.5 against 111; 128 in 18 against 36; 512 in 44 against 39; 700 -> 10,000: 64 in 190 against 282.  One leaf, 700 ->
// 256: 128 in 9.1 against 9.4, 256 in 14.5 against 9.3; 700 -> 10,000: 4 in 12 against 16, 16 in 34 against 16, 64 in 114 against
// 17; 137 -> 1,000: 32 in 6.5 against 8.8.  700 -> 1, 2,048 positions: 4.9 against 8.7; 28 -> 1, 4,096: 5.1 against 4.6.)
template <typename T>
bool few_answers(const gbdt_leaf::LeafArgs<T>& g, bool direct) {
  const int64_t n = g.n_positions;
  int64_t most = 16384;
  if (n < 4 * (int64_t)g.n_leaves) {
    if (n <= 64) return true;
    most *= sizeof(T) == 2 ? 2 : 4;
  } else if (n <= 64 && !direct) {
    most *= 2;
  }
  return n <= 4 || (n <= 2048 && n * g.d_out <= most);
}

template <typename T>
int leaf_product_few(gbdt_leaf::LeafArgs<T>& g, hipStream_t s) {
  // One output a wavefront where that leaves compute units without work, four otherwise.  (700 -> 256, one position: 4.1 us
  // against 4.9; 64 positions: 10.5 against 7.3.)
  if ((int64_t)g.n_positions * g.d_out <= 1024) {
    gbdt_leaf::leaf_product_few_kernel<T, 1><<<dim3(g.d_out, g.n_positions), dim3(64), 0, s>>>(g);
  } else {
    gbdt_leaf::leaf_product_few_kernel<T, 4><<<dim3((unsigned)ceil_div(g.d_out, 4), g.n_positions), dim3(64), 0, s>>>(g);
  }
  LAUNCHED("leaf_product_few_kernel");
  return GBDT_OK;
}

template <class S, int GROUPS, typename T>
int launch_leaf_product_split(gbdt_leaf::LeafArgs<T>& g, hipStream_t s) {
  return leaf_rows_launches<S>(g, g.d_out, S::NT * GROUPS, false, [&](dim3 blocks) {
    gbdt_leaf::leaf_product_split_kernel<S, GROUPS><<<blocks, dim3(S::NT * GROUPS), 0, s>>>(g);
  });
}

// No more tiles of 64 x 64 than compute units (f32: than half of them), and steps enough to split.  bf16: four groups of threads
// a tile of 64 x 64 (500 x 2,000 -> 64 in one leaf: 10.6 us against 16.9 in tiles of 128 x 128).  f32, where a unit's matrix
// instructions are the bound: eight a tile of 32 x 16, which spreads over eight times the units (the same: 10.8 us against 43
// in tiles of 64 x 64; 2,000 x 700 -> 256 in 31 leaves, 252 tiles: 34 against 19).
template <typename T>
bool few_tiles(const gbdt_leaf::LeafArgs<T>& g) {
  const int64_t tiles = (ceil_div(g.n_positions, 64) + std::min<int64_t>(g.n_leaves, g.n_positions)) * ceil_div(g.d_out, 64);
  return tiles <= gbdt_internal::cu_count() / (sizeof(T) == 2 ? 1 : 2) && (int64_t)g.d_in * (int64_t)sizeof(T) >= 8 * 128;
}

template <typename T>
int leaf_product(gbdt_leaf::LeafArgs<T>& g, hipStream_t s) {
  const bool direct = whole_chunks<T>(g.x, g.ld_x, g.d_in) && whole_chunks<T>(g.w, g.d_in, g.d_in);
  if (few_answers(g, direct)) return leaf_product_few(g, s);
  if (few_tiles(g)) {
    if constexpr (sizeof(T) == 2) {
      return direct ? launch_leaf_product_split<Shape<T, 64, 64, 2, 2, true>, 4>(g, s)
                    : launch_leaf_product_split<Shape<T, 64, 64, 2, 2, false>, 4>(g, s);
    } else {
      return direct ? launch_leaf_product_split<Shape<T, 32, 16, 1, 1, true>, 8>(g, s)
                    : launch_leaf_product_split<Shape<T, 32, 16, 1, 1, false>, 8>(g, s);
    }
  }
  // (100,000 x 700 -> 1: 36 us against 53 in the tiles below, f32 69 against 102; 10,000 x 28 -> 1: 5.4 against 8.6.)
  if (g.d_out <= 16)
    return direct ? launch_leaf_product<Shape<T, 128, 16, 4, 1, true>>(g, s) : launch_leaf_product<Shape<T, 128, 16, 4, 1, false>>(g, s);
  if (direct && sizeof(T) == 2) {
    // (1,024 positions in 255 leaves, 2,000 -> 64: 25 us against 29 in tiles of 128 x 128; 400,000: 425 against 428.)
    if (g.d_out <= 64) return launch_leaf_product<Shape<T, 128, 64, 4, 1, true>>(g, s);
    if (wide_leaves(g, g.d_out)) return launch_leaf_product<Wide<T>>(g, s);
    if (long_leaves(g, g.d_out, 128)) return launch_leaf_product<Shape<T, 256, 128, 4, 2, true, false, 3>>(g, s);
  }
  return direct ? launch_leaf_product<Square<T>>(g, s) : launch_leaf_product<SquareAny<T>>(g, s);
}

template <class S, typename T>
int launch_leaf_grad_input(gbdt_leaf::LeafArgs<T>& g, hipStream_t s) {
  return leaf_rows_launches<S>(g, g.d_in, S::NT, true, [&](dim3 blocks) {
    gbdt_leaf::leaf_grad_input_kernel<S><<<blocks, dim3(S::NT), 0, s>>>(g);
  });
}

template <typename T>
int leaf_grad_input(gbdt_leaf::LeafArgs<T> g, hipStream_t s) {
  const bool direct = whole_chunks<T>(g.dy, g.ld_dy, g.d_out) && whole_chunks<T>(g.w, g.d_in, g.d_in);
  return direct && wide_leaves(g, g.d_in) ? launch_leaf_grad_input<Wide<T>>(g, s)
         : direct                        ? launch_leaf_grad_input<Square<T>>(g, s)
                                         : launch_leaf_grad_input<SquareAny<T>>(g, s);
}

template <typename T>
int leaf_product_grad(gbdt_leaf::LeafArgs<T>& g, hipStream_t s) {
  const bool inputs = g.dx && g.n_positions > 0;
  if (!g.dw && !g.dbias) return inputs ? leaf_grad_input(g, s) : GBDT_OK;
  const gbdt_leaf::LeafArgs<T> of_inputs = g;
  // The outputs' sums alone do not read x, which may be null: the other operand is dy's first columns.
  const bool dy_whole = whole_chunks<T>(g.dy, g.ld_dy, g.d_out);
  if (!g.dw) g.x = g.dy, g.ld_x = g.ld_dy, g.d_in = dy_whole ? kChunk<T> : 1;
  const bool direct = dy_whole && whole_chunks<T>(g.x, g.ld_x, g.d_in);
  const LeafGradPlan plan = leaf_grad_plan(sizeof(T), g.n_positions, g.d_in, g.d_out, gbdt_internal::cu_count());
  if (plan.tiles > most_blocks(kGradThreads) / 8) return GBDT_EUNSUPPORTED;
  g.cut = (int32_t)plan.cut;
  int rc = GBDT_OK;
  if (plan.bytes) {
    void* ws = nullptr;
    if ((rc = gbdt_internal::workspace(plan.bytes, s, &ws)) != GBDT_OK) return rc;
    g.partial = (float*)ws;
  }
  if (inputs && (rc = leaf_grad_input(of_inputs, s)) != GBDT_OK) return rc;
  if constexpr (sizeof(T) == 2) {
    if (plan.bm == 64)
      rc = direct ? launch_leaf_grad_weight<Shape<T, 64, 128, 1, 4, true, true>, false>(g, s, g.d_out) : launch_leaf_grad_weight<Shape<T, 64, 128, 1, 4, false>, false>(g, s, g.d_out);
    else
      rc = direct ? launch_leaf_grad_weight<Square<T>, false>(g, s, g.d_out) : launch_leaf_grad_weight<SquareAny<T>, false>(g, s, g.d_out);
  } else {
    rc = direct ? launch_leaf_grad_weight<Square<T>, false>(g, s, g.d_out) : launch_leaf_grad_weight<SquareAny<T>, false>(g, s, g.d_out);
  }
  return rc != GBDT_OK ? rc : launch_leaf_grad_join<false>(g, s);
}

// ---------------------------------------------------------------- softmax

constexpr int64_t kPieceAlign = 256;                    // classes: whole tiles of every shape
// G of a piece, as long as it is kPieceAlign classes wide at least.  8,192 x 65,536 x 1,024 bf16, loss and gradients: 4.07 ms at
// 128 MiB, 3.95 at 256, 3.85 at 512, 3.95 in one piece of 1 GiB.
constexpr int64_t kPieceBytes = (int64_t)512 << 20;
constexpr int64_t kPartsBytes = (int64_t)256 << 20;     // maxima and sums of a launch's tiles, of 256 rows at least

int softmax_check(const void* h, int64_t ld_h, const void* c, int64_t ld_c, int64_t n_rows, int64_t n_classes, int32_t dim,
                  int32_t dtype) {
  if (n_rows < 0 || n_classes <= 0 || dim <= 0 || !c || (!h && n_rows > 0) || ld_h < dim || ld_c < dim) return GBDT_EINVAL;
  if (dtype != GBDT_F32 && dtype != GBDT_BF16) return GBDT_EINVAL;
  if (off_element(h, dtype) || off_element(c, dtype)) return GBDT_EINVAL;
  if (n_rows >= kMaxRows || n_classes >= kMaxRows || dim >= kMaxWidth || ld_h >= kMaxLd || ld_c >= kMaxLd) return GBDT_EUNSUPPORTED;
  return GBDT_OK;
}

// Row tiles that go through the classes together: 2 MiB of rows, half of an XCD's L2.  (Loss, 8,192 x 65,536 x 1,024: 888 us
// against 936 one at a time; 1,500 x 10,000 x 512: 25 against 32.)
uint32_t group_of(int64_t tile_rows, int64_t dim, int64_t bytes) {
  return (uint32_t)std::max<int64_t>(1, std::min<int64_t>(64, ((int64_t)2 << 20) / (tile_rows * dim * bytes)));
}

template <class S, typename T>
int score_grid(gbdt_softmax::ScoreArgs<T>& g, unsigned* blocks) {
  g.row_tiles = (uint32_t)ceil_div(g.n_rows, S::BM);
  g.col_tiles = (uint32_t)ceil_div(g.end - g.begin, S::BN);
  g.group = group_of(S::BM, g.dim, sizeof(T));
  const int64_t n = (int64_t)g.row_tiles * g.col_tiles;
  if (n > kMaxTiles || (int64_t)g.group * g.col_tiles > kMaxTiles) return GBDT_EUNSUPPORTED;
  // One workgroup a compute unit goes through the tiles where there is no room for two; else one a tile, as far as a launch goes.
  const int64_t units = std::max(8, gbdt_internal::cu_count() / 8 * 8);
  *blocks = (unsigned)std::min(n, S::BM >= 256 ? units : most_blocks(S::NT));
  return GBDT_OK;
}

struct LossPlan {
  int64_t rows;  // of a launch
  int64_t tiles;
  size_t parts_bytes, bytes;
};
template <typename T>
LossPlan loss_plan(int64_t n_rows, int64_t n_classes) {
  LossPlan p;
  p.tiles = ceil_div(n_classes, gbdt_softmax::kPartClasses<T>);
  const int64_t fit = kPartsBytes / (8 * p.tiles), whole = fit >= 4096 ? 4096 : 256;
  p.rows = std::min(n_rows, std::max<int64_t>(256, fit / whole * whole));
  p.parts_bytes = pad256((size_t)(p.rows * p.tiles) * 8);
  p.bytes = p.parts_bytes + pad256((size_t)p.rows * 4);
  return p;
}

template <class S, typename T>
int launch_scores(gbdt_softmax::ScoreArgs<T>& g, hipStream_t s) {
  unsigned blocks = 0;
  const int rc = score_grid<S>(g, &blocks);
  if (rc != GBDT_OK) return rc;
  gbdt_softmax::softmax_scores_kernel<S><<<dim3(blocks), dim3(S::NT), 0, s>>>(g);
  LAUNCHED("softmax_scores_kernel");
  return GBDT_OK;
}

template <typename T>
int softmax_loss(const T* h, int64_t ld_h, const T* c, int64_t ld_c, const int32_t* labels, int64_t n_rows, int64_t n_classes,
                 int32_t dim, float* loss, float* lse, hipStream_t s) {
  const LossPlan plan = loss_plan<T>(n_rows, n_classes);
  void* ws = nullptr;
  int rc = gbdt_internal::workspace(plan.bytes, s, &ws);
  if (rc != GBDT_OK) return rc;
  const bool direct = whole_chunks<T>(h, ld_h, dim) && whole_chunks<T>(c, ld_c, dim);
  for (int64_t r = 0; r < n_rows; r += plan.rows) {
    gbdt_softmax::ScoreArgs<T> g = {};
    g.h = h + r * ld_h;
    g.c = c;
    g.labels = labels ? labels + r : nullptr;
    g.parts = (gbdt_softmax::MaxSum*)ws;
    g.picked = (float*)((char*)ws + plan.parts_bytes);
    g.ld_h = ld_h;
    g.ld_c = ld_c;
    g.n_rows = (int32_t)std::min(plan.rows, n_rows - r);
    g.n_classes = g.end = (int32_t)n_classes;
    g.dim = dim;
    rc = direct && wide_tiles<T>(g.n_rows, n_classes) ? launch_scores<Wide<T>>(g, s)
         : direct                                     ? launch_scores<Square<T>>(g, s)
                                                      : launch_scores<SquareAny<T>>(g, s);
    if (rc != GBDT_OK) return rc;
    // (Whole call, 256 rows x 50,000 classes x 64: 13.5 us against 20 with 16 rows a workgroup; 4,096 x 1,000 x 64: 11.5
    // against 8.3.)
    if (g.n_rows <= 256) {
      gbdt_softmax::softmax_join_kernel<1><<<dim3((unsigned)g.n_rows), dim3(256), 0, s>>>(
          g.parts, g.picked, g.labels, g.n_rows, g.n_classes, (int32_t)plan.tiles, loss ? loss + r : nullptr, lse + r);
    } else {
      gbdt_softmax::softmax_join_kernel<16><<<dim3((unsigned)ceil_div(g.n_rows, 16)), dim3(256), 0, s>>>(
          g.parts, g.picked, g.labels, g.n_rows, g.n_classes, (int32_t)plan.tiles, loss ? loss + r : nullptr, lse + r);
    }
    LAUNCHED("softmax_join_kernel");
  }
  return GBDT_OK;
}

struct GradPlan {
  bool pair;       // G as two values: one piece, tiles of kPairClasses
  bool wide_dh;    // tiles of 256 x 256
  int64_t width;   // classes a piece
  int64_t pieces;
  int64_t dh_splits, dh_split, dc_splits, dc_split;
  size_t g_bytes, dh_bytes, dc_bytes, h_bytes, c_bytes, rest_bytes;
  size_t bytes() const { return g_bytes + dh_bytes + dc_bytes + h_bytes + c_bytes + rest_bytes; }
};
// Splits of a summed axis of `k`: as many as give `units` workgroups work, each 4 steps long at least.  (Loss and gradients, 64
// x 32,768 x 512: 91 us against 285 unsplit; 4,096 x 1,000 x 512: 79 against 107.)
void split_axis(int64_t tiles, int64_t k, int64_t step, int64_t units, int64_t* splits, int64_t* len) {
  const int64_t want = std::max<int64_t>(1, std::min(units / std::max<int64_t>(tiles, 1), ceil_div(k, 4 * step)));
  *len = std::max(step, round_up(ceil_div(k, want), step));
  *splits = std::max<int64_t>(1, ceil_div(k, *len));
}
GradPlan grad_plan(int64_t n_rows, int64_t n_classes, int64_t dim, int64_t e, bool c_whole, int64_t units) {
  GradPlan p;
  p.pair = e == 2 && n_classes <= gbdt_softmax::kPairClasses;
  const int64_t rows = std::max<int64_t>(n_rows, 1);
  const int64_t all = round_up(n_classes, kPieceAlign);
  p.width = std::min(all, std::max(kPieceAlign, kPieceBytes / (rows * e) / kPieceAlign * kPieceAlign));
  p.pieces = ceil_div(n_classes, p.width);
  p.width = round_up(ceil_div(n_classes, p.pieces), kPieceAlign);
  p.pieces = ceil_div(n_classes, p.width);
  const int64_t step = 128 / e;
  const int64_t tile = e == 2 ? 128 : 64;
  const int64_t cols = ceil_div(dim, tile);
  split_axis(ceil_div(rows, tile) * cols, p.width, step, 2 * units, &p.dh_splits, &p.dh_split);
  // Large tiles of dh for more than 128 columns, even if it takes splits to have as many as there are units, of 16 steps at
  // least.  (dh and its G, tiles of 128 x 128 against these: 3,000 x 50,000 x 1,024: 749 us against 602, 8,200 x 40,000 x 520: 1,143 against
  // 974, 500 x 33,000 x 512: 87 and 86; 1,400 x 65,536 x 40: 109 against 120.)
  const int64_t wide = ceil_div(rows, 256) * ceil_div(dim, 256);
  p.wide_dh = e == 2 && !p.pair && dim > 128 && wide * ceil_div(p.width, 16 * step) >= units;
  if (p.wide_dh && wide < units)
    split_axis(wide, p.width, step, units, &p.dh_splits, &p.dh_split);
  else if (p.wide_dh)
    p.dh_splits = 1, p.dh_split = round_up(p.width, step);
  split_axis(ceil_div(p.width, tile) * cols, n_rows, step, 2 * units, &p.dc_splits, &p.dc_split);
  p.g_bytes = pad256((size_t)(rows * p.width * e));
  p.dh_bytes = p.dh_splits > 1 || p.pieces > 1 ? pad256((size_t)(p.dh_splits * rows * dim) * 4) : 0;
  p.dc_bytes = p.dc_splits > 1 ? pad256((size_t)(p.dc_splits * p.width * dim) * 4) : 0;
  const int64_t row_bytes = round_up(dim * e, 16);
  p.h_bytes = pad256((size_t)(rows * row_bytes));
  p.rest_bytes = e == 2 && !p.pair ? pad256((size_t)rows * 4) : 0;
  p.c_bytes = c_whole ? 0 : pad256((size_t)(n_classes * row_bytes));
  return p;
}

template <typename T>
int whole_rows(const T* from, int64_t ld, T* to, int64_t rows, int32_t cols, const int32_t* labels, int64_t n_classes, hipStream_t s) {
  const int64_t blocks = ceil_div(rows * ceil_div(cols, kChunk<T>), 256);
  if (blocks == 0) return GBDT_OK;
  gbdt_softmax::whole_rows_kernel<T><<<dim3((unsigned)std::min<int64_t>(blocks, 16384)), dim3(256), 0, s>>>(
      from, ld, to, (int32_t)rows, cols, labels, (int32_t)n_classes);
  LAUNCHED("whole_rows_kernel");
  return GBDT_OK;
}

template <class S, bool PAIR, typename T>
int launch_piece(gbdt_softmax::ScoreArgs<T>& g, hipStream_t s) {
  static_assert(kPieceAlign % S::BN == 0 && kPieceAlign >= 2 * gbdt_softmax::kPairClasses, "G's rows hold whole tiles");
  unsigned blocks = 0;
  const int rc = score_grid<S>(g, &blocks);
  if (rc != GBDT_OK || blocks == 0) return rc;
  gbdt_softmax::softmax_piece_kernel<S, PAIR><<<dim3(blocks), dim3(S::NT), 0, s>>>(g);
  LAUNCHED("softmax_piece_kernel");
  return GBDT_OK;
}

template <class S, bool TO_ROWS, bool PAIR, typename T>
int launch_product(gbdt_softmax::PieceArgs<T>& g, hipStream_t s) {
  g.row_tiles = (uint32_t)ceil_div(g.rows, S::BM);
  g.col_tiles = (uint32_t)ceil_div(g.cols, S::BN);
  g.group = 8;
  const int64_t blocks = (int64_t)g.row_tiles * g.col_tiles * g.splits;
  if (blocks > most_blocks(S::NT)) return GBDT_EUNSUPPORTED;  // (operands and G of so many tiles fit no card)
  if (blocks == 0) return GBDT_OK;
  gbdt_softmax::piece_product_kernel<S, TO_ROWS, PAIR><<<dim3((unsigned)blocks), dim3(S::NT), 0, s>>>(g);
  LAUNCHED("piece_product_kernel");
  return GBDT_OK;
}

// The tile by the size of the result; PAIR is of bf16 alone and takes small ones, for its summed axis or its result is short.
template <bool TO_ROWS, typename T>
int product(gbdt_softmax::PieceArgs<T>& g, bool pair, bool wide, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (pair) return launch_product<Square<T>, TO_ROWS, true>(g, s);
  }
  return wide ? launch_product<Wide<T>, TO_ROWS, false>(g, s) : launch_product<Square<T>, TO_ROWS, false>(g, s);
}

template <typename T>
int piece_of_g(gbdt_softmax::ScoreArgs<T>& g, bool pair, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (pair) return launch_piece<Square<T>, true>(g, s);
  }
  return wide_tiles<T>(g.n_rows, g.end - g.begin) ? launch_piece<Wide<T>, false>(g, s) : launch_piece<Square<T>, false>(g, s);
}

template <typename T>
int join_product(const gbdt_softmax::PieceArgs<T>& g, hipStream_t s) {
  const int64_t n = ceil_div((int64_t)g.rows * ceil_div(g.cols, 4), 256);
  if (n == 0) return GBDT_OK;
  gbdt_softmax::piece_join_kernel<T><<<dim3((unsigned)std::min<int64_t>(n, 16384)), dim3(256), 0, s>>>(g);
  LAUNCHED("piece_join_kernel");
  return GBDT_OK;
}

template <typename T>
int softmax_grad(const T* h, int64_t ld_h, const T* c, int64_t ld_c, const int32_t* labels, const float* lse, const float* weight,
                 float scale, int64_t n_rows, int64_t n_classes, int32_t dim, T* dh, int64_t ld_dh, T* dc, int64_t ld_dc,
                 hipStream_t s) {
  const bool c_whole = whole_chunks<T>(c, ld_c, dim);
  const GradPlan plan = grad_plan(n_rows, n_classes, dim, sizeof(T), c_whole, gbdt_internal::cu_count());
  void* ws = nullptr;
  int rc = gbdt_internal::workspace(plan.bytes(), s, &ws);
  if (rc != GBDT_OK) return rc;
  char* at = (char*)ws;
  T* piece = (T*)at;
  at += plan.g_bytes;
  float* dh_sums = plan.dh_bytes ? (float*)at : nullptr;
  at += plan.dh_bytes;
  float* dc_sums = plan.dc_bytes ? (float*)at : nullptr;
  at += plan.dc_bytes;
  float* rest = plan.rest_bytes ? (float*)at : nullptr;
  at += plan.rest_bytes;
  // Both matrices are of whole chunks from here on; whole_dim is the length of their rows.
  const int32_t whole_dim = (int32_t)round_up(dim, kChunk<T>);
  if ((rc = whole_rows<T>(h, ld_h, (T*)at, n_rows, dim, labels, n_classes, s)) != GBDT_OK) return rc;
  h = (const T*)at;
  ld_h = whole_dim;
  at += plan.h_bytes;
  if (!c_whole) {
    if ((rc = whole_rows<T>(c, ld_c, (T*)at, n_classes, dim, nullptr, n_classes, s)) != GBDT_OK) return rc;
    c = (const T*)at;
    ld_c = whole_dim;
  }
  gbdt_softmax::PieceArgs<T> to_h = {}, to_c = {};
  for (int64_t begin = 0; begin < n_classes; begin += plan.width) {
    const int64_t end = std::min(n_classes, begin + plan.width);
    gbdt_softmax::ScoreArgs<T> g = {};
    g.h = h;
    g.c = c;
    g.labels = labels;
    g.lse = lse;
    g.weight = weight;
    g.g = piece;
    g.rest = rest;
    g.ld_h = ld_h;
    g.ld_c = ld_c;
    g.ld_g = plan.width;
    g.n_rows = (int32_t)n_rows;
    g.n_classes = (int32_t)n_classes;
    g.dim = whole_dim;
    g.begin = (int32_t)begin;
    g.end = (int32_t)end;
    if ((rc = piece_of_g(g, plan.pair, s)) != GBDT_OK) return rc;
    if (dc) {
      to_c.a = piece;
      to_c.b = h;
      to_c.out = dc + begin * ld_dc;
      to_c.sums = dc_sums;
      to_c.labels = labels;
      to_c.rest = rest;
      to_c.class0 = (int32_t)begin;
      to_c.ld_a = plan.width;
      to_c.ld_b = ld_h;
      to_c.ld_out = ld_dc;
      to_c.scale = scale;
      to_c.rows = (int32_t)(end - begin);
      to_c.cols = dim;
      to_c.k = to_c.b_rows = (int32_t)n_rows;
      to_c.b_cols = whole_dim;
      to_c.n_classes = (int32_t)n_classes;
      to_c.k_split = (int32_t)plan.dc_split;
      to_c.splits = (uint32_t)plan.dc_splits;
      if ((rc = product<false>(to_c, plan.pair, wide_tiles<T>(to_c.rows, dim), s)) != GBDT_OK) return rc;
      if (dc_sums) {
        gbdt_softmax::PieceArgs<T> sums = to_c;
        sums.labels = nullptr;
        if ((rc = join_product(sums, s)) != GBDT_OK) return rc;
      }
    }
    if (dh && n_rows > 0) {
      to_h.a = piece;
      to_h.b = c + begin * ld_c;
      to_h.out = dh;
      to_h.sums = dh_sums;
      to_h.labels = labels;
      to_h.rest = rest;
      to_h.c = c;
      to_h.ld_c = ld_c;
      to_h.ld_a = plan.width;
      to_h.ld_b = ld_c;
      to_h.ld_out = ld_dh;
      to_h.scale = scale;
      to_h.rows = (int32_t)n_rows;
      to_h.cols = dim;
      to_h.k = (int32_t)round_up(end - begin, kChunk<T>);
      to_h.b_rows = (int32_t)(end - begin);
      to_h.b_cols = whole_dim;
      to_h.n_classes = (int32_t)n_classes;
      to_h.k_split = (int32_t)plan.dh_split;
      to_h.splits = (uint32_t)plan.dh_splits;
      to_h.add = begin > 0;
      if ((rc = product<true>(to_h, plan.pair, plan.wide_dh, s)) != GBDT_OK) return rc;
    }
  }
  if (dh && n_rows > 0 && dh_sums) return join_product(to_h, s);
  return GBDT_OK;
}

template <class S, typename T>
int launch_stats(gbdt_softmax::ScoreArgs<T>& g, hipStream_t s) {
  unsigned blocks = 0;
  const int rc = score_grid<S>(g, &blocks);
  if (rc != GBDT_OK || blocks == 0) return rc;
  gbdt_softmax::softmax_stats_kernel<S><<<dim3(blocks), dim3(S::NT), 0, s>>>(g);
  LAUNCHED("softmax_stats_kernel");
  return GBDT_OK;
}

template <typename T>
int softmax_stats(gbdt_softmax::ScoreArgs<T>& g, hipStream_t s) {
  const bool direct = whole_chunks<T>(g.h, g.ld_h, g.dim) && whole_chunks<T>(g.c, g.ld_c, g.dim);
  // (16 of 1,000 classes, 400,000 x 64: 21 us against 55 in tiles of 128 x 128, f32 31 against 52 in 64 x 64.)
  if (g.end - g.begin <= 16)
    return direct ? launch_stats<Shape<T, 128, 16, 4, 1, true, false, 2, true>>(g, s) : launch_stats<Shape<T, 128, 16, 4, 1, false, false, 2, true>>(g, s);
  if constexpr (sizeof(T) == 2) {
    return direct ? launch_stats<Shape<T, 128, 128, 2, 2, true, true, 2, true>>(g, s) : launch_stats<Shape<T, 64, 64, 2, 2, false, false, 2, true>>(g, s);
  } else {
    return direct ? launch_stats<Square<T>>(g, s) : launch_stats<SquareAny<T>>(g, s);
  }
}

template <typename T>
int leaf_product_call(const void* x, int64_t ld_x, const void* weight, const void* bias, const int32_t* row_idx,
                      const int64_t* leaf_offsets, int64_t n_positions, int32_t n_leaves, int64_t n_rows, int32_t d_in, int32_t d_out,
                      void* y_out, int64_t ld_y, hipStream_t s) {
  gbdt_leaf::LeafArgs<T> g = {};
  g.x = (const T*)x;
  g.w = (const T*)weight;
  g.bias = (const T*)bias;
  g.y = (T*)y_out;
  g.row_idx = row_idx;
  g.offsets = leaf_offsets;
  g.ld_x = ld_x;
  g.ld_y = ld_y;
  g.n_positions = (int32_t)n_positions;
  g.n_leaves = n_leaves;
  g.n_rows = (int32_t)n_rows;
  g.d_in = d_in;
  g.d_out = d_out;
  return leaf_product(g, s);
}

template <typename T>
int leaf_product_grad_call(const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, const void* weight, const int32_t* row_idx,
                           const int64_t* leaf_offsets, int64_t n_positions, int32_t n_leaves, int64_t n_rows, int32_t d_in,
                           int32_t d_out, void* dx_out, int64_t ld_dx, void* dweight_out, void* dbias_out, hipStream_t s) {
  gbdt_leaf::LeafArgs<T> g = {};
  g.x = (const T*)x;
  g.dy = (const T*)dy;
  g.w = (const T*)weight;
  g.dx = (T*)dx_out;
  g.dw = (T*)dweight_out;
  g.dbias = (T*)dbias_out;
  g.row_idx = row_idx;
  g.offsets = leaf_offsets;
  g.ld_x = ld_x;
  g.ld_dy = ld_dy;
  g.ld_dx = ld_dx;
  g.n_positions = (int32_t)n_positions;
  g.n_leaves = n_leaves;
  g.n_rows = (int32_t)n_rows;
  g.d_in = d_in;
  g.d_out = d_out;
  return leaf_product_grad(g, s);
}

template <typename T>
int softmax_stats_call(const void* h, int64_t ld_h, const void* c, int64_t ld_c, const int32_t* labels, const float* lse,
                       int64_t n_rows, int64_t n_classes, int32_t dim, int64_t class_begin, int64_t class_end, float* grad_out,
                       float* hess_out, int64_t ld_out, hipStream_t s) {
  gbdt_softmax::ScoreArgs<T> g = {};
  g.h = (const T*)h;
  g.c = (const T*)c;
  g.labels = labels;
  g.lse = lse;
  g.grad = grad_out;
  g.hess = hess_out;
  g.ld_h = ld_h;
  g.ld_c = ld_c;
  g.ld_out = ld_out;
  g.n_rows = (int32_t)n_rows;
  g.n_classes = (int32_t)n_classes;
  g.dim = dim;
  g.begin = (int32_t)class_begin;
  g.end = (int32_t)class_end;
  return softmax_stats(g, s);
}

}  // namespace

using namespace gbdt_host;

extern "C" {

int gbdt_leaf_product(const void* x, int64_t ld_x, const void* weight, const void* bias, const int32_t* row_idx,
                      const int64_t* leaf_offsets, int64_t n_positions, int32_t n_leaves, int64_t n_rows, int32_t d_in,
                      int32_t d_out, int32_t dtype, void* y_out, int64_t ld_y, void* stream) {
  const int rc = leaf_check(n_positions, n_leaves, n_rows, d_in, d_out, row_idx, leaf_offsets, dtype);
  if (rc != GBDT_OK) return rc;
  if (ld_x < d_in || ld_y < d_out || !weight || off_element(x, dtype) || off_element(weight, dtype) || off_element(bias, dtype) ||
      off_element(y_out, dtype))
    return GBDT_EINVAL;
  if (ld_x >= kMaxLd || ld_y >= kMaxLd) return GBDT_EUNSUPPORTED;
  if (n_positions == 0 || n_rows == 0) return GBDT_OK;
  if (!x || !y_out) return GBDT_EINVAL;
  hipStream_t s = (hipStream_t)stream;
  return dtype == GBDT_F32 ? leaf_product_call<float>(x, ld_x, weight, bias, row_idx, leaf_offsets, n_positions, n_leaves, n_rows,
                                                      d_in, d_out, y_out, ld_y, s)
                           : leaf_product_call<bf16>(x, ld_x, weight, bias, row_idx, leaf_offsets, n_positions, n_leaves, n_rows,
                                                     d_in, d_out, y_out, ld_y, s);
}

size_t gbdt_leaf_product_grad_workspace_bytes(int64_t n_positions, int32_t d_in, int32_t d_out) {
  if (n_positions < 0 || n_positions >= kMaxRows || d_in <= 0 || d_out <= 0 || d_in >= kMaxWidth || d_out >= kMaxWidth) return 0;
  const int64_t units = gbdt_internal::cu_count();
  size_t most = 0;
  for (int64_t e : {2, 4})
    for (int64_t inputs : {(int64_t)d_in, 16 / e, (int64_t)1})  // with the weights' gradient and without
      most = std::max(most, leaf_grad_plan(e, n_positions, inputs, d_out, units).bytes);
  return gbdt_internal::workspace_head_bytes() + most;
}

int gbdt_leaf_product_grad(const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, const void* weight, const int32_t* row_idx,
                           const int64_t* leaf_offsets, int64_t n_positions, int32_t n_leaves, int64_t n_rows, int32_t d_in,
                           int32_t d_out, int32_t dtype, void* dx_out, int64_t ld_dx, void* dweight_out, void* dbias_out,
                           void* stream) {
  const int rc = leaf_check(n_positions, n_leaves, n_rows, d_in, d_out, row_idx, leaf_offsets, dtype);
  if (rc != GBDT_OK) return rc;
  if (ld_dy < d_out || (dweight_out && ld_x < d_in) || (dx_out && (ld_dx < d_in || !weight))) return GBDT_EINVAL;
  if (off_element(dy, dtype) || off_element(x, dtype) || off_element(weight, dtype) || off_element(dx_out, dtype) ||
      off_element(dweight_out, dtype) || off_element(dbias_out, dtype))
    return GBDT_EINVAL;
  if (ld_dy >= kMaxLd || ld_x >= kMaxLd || ld_dx >= kMaxLd) return GBDT_EUNSUPPORTED;
  if (n_rows == 0) n_positions = 0;
  if (n_positions > 0 && (!dy || (dweight_out && !x))) return GBDT_EINVAL;
  hipStream_t s = (hipStream_t)stream;
  return dtype == GBDT_F32 ? leaf_product_grad_call<float>(dy, ld_dy, x, ld_x, weight, row_idx, leaf_offsets, n_positions, n_leaves,
                                                           n_rows, d_in, d_out, dx_out, ld_dx, dweight_out, dbias_out, s)
                           : leaf_product_grad_call<bf16>(dy, ld_dy, x, ld_x, weight, row_idx, leaf_offsets, n_positions, n_leaves,
                                                          n_rows, d_in, d_out, dx_out, ld_dx, dweight_out, dbias_out, s);
}

size_t gbdt_softmax_workspace_bytes(int64_t n_rows, int64_t n_classes, int32_t dim, int32_t dtype) {
  if (n_rows < 0 || n_classes <= 0 || dim <= 0 || n_rows >= kMaxRows || n_classes >= kMaxRows || dim >= kMaxWidth ||
      (dtype != GBDT_F32 && dtype != GBDT_BF16))
    return 0;
  const GradPlan p = grad_plan(n_rows, n_classes, dim, dtype == GBDT_F32 ? 4 : 2, false, gbdt_internal::cu_count());
  const size_t grad = p.bytes(), loss = (dtype == GBDT_F32 ? loss_plan<float>(n_rows, n_classes) : loss_plan<bf16>(n_rows, n_classes)).bytes;
  return gbdt_internal::workspace_head_bytes() + std::max(grad, loss);
}

int gbdt_softmax_loss(const void* h, int64_t ld_h, const void* classes, int64_t ld_c, const int32_t* labels, int64_t n_rows,
                      int64_t n_classes, int32_t dim, int32_t dtype, float* loss_out, float* lse_out, void* stream) {
  const int rc = softmax_check(h, ld_h, classes, ld_c, n_rows, n_classes, dim, dtype);
  if (rc != GBDT_OK) return rc;
  if ((labels == nullptr) != (loss_out == nullptr)) return GBDT_EINVAL;
  if (n_rows == 0) return GBDT_OK;
  if (!lse_out) return GBDT_EINVAL;
  hipStream_t s = (hipStream_t)stream;
  return dtype == GBDT_F32 ? softmax_loss((const float*)h, ld_h, (const float*)classes, ld_c, labels, n_rows, n_classes, dim, loss_out,
                                          lse_out, s)
                           : softmax_loss((const bf16*)h, ld_h, (const bf16*)classes, ld_c, labels, n_rows, n_classes, dim, loss_out,
                                          lse_out, s);
}

int gbdt_softmax_grad(const void* h, int64_t ld_h, const void* classes, int64_t ld_c, const int32_t* labels, const float* lse,
                      const float* row_weight, float scale, int64_t n_rows, int64_t n_classes, int32_t dim, int32_t dtype, void* dh_out,
                      int64_t ld_dh, void* dclasses_out, int64_t ld_dc, void* stream) {
  const int rc = softmax_check(h, ld_h, classes, ld_c, n_rows, n_classes, dim, dtype);
  if (rc != GBDT_OK) return rc;
  if ((dh_out && ld_dh < dim) || (dclasses_out && ld_dc < dim) || off_element(dh_out, dtype) || off_element(dclasses_out, dtype))
    return GBDT_EINVAL;
  if (n_rows > 0 && (!labels || !lse)) return GBDT_EINVAL;
  if (!dh_out && !dclasses_out) return GBDT_OK;
  hipStream_t s = (hipStream_t)stream;
  return dtype == GBDT_F32 ? softmax_grad((const float*)h, ld_h, (const float*)classes, ld_c, labels, lse, row_weight, scale, n_rows,
                                          n_classes, dim, (float*)dh_out, ld_dh, (float*)dclasses_out, ld_dc, s)
                           : softmax_grad((const bf16*)h, ld_h, (const bf16*)classes, ld_c, labels, lse, row_weight, scale, n_rows,
                                          n_classes, dim, (bf16*)dh_out, ld_dh, (bf16*)dclasses_out, ld_dc, s);
}

int gbdt_softmax_stats(const void* h, int64_t ld_h, const void* classes, int64_t ld_c, const int32_t* labels, const float* lse,
                       int64_t n_rows, int64_t n_classes, int32_t dim, int32_t dtype, int64_t class_begin, int64_t class_end,
                       float* grad_out, float* hess_out, int64_t ld_out, void* stream) {
  const int rc = softmax_check(h, ld_h, classes, ld_c, n_rows, n_classes, dim, dtype);
  if (rc != GBDT_OK) return rc;
  if (class_begin < 0 || class_end < class_begin || class_end > n_classes || ld_out < n_rows) return GBDT_EINVAL;
  if (n_rows == 0 || class_begin == class_end) return GBDT_OK;
  if (!lse || !grad_out || !hess_out) return GBDT_EINVAL;
  hipStream_t s = (hipStream_t)stream;
  return dtype == GBDT_F32 ? softmax_stats_call<float>(h, ld_h, classes, ld_c, labels, lse, n_rows, n_classes, dim, class_begin,
                                                       class_end, grad_out, hess_out, ld_out, s)
                           : softmax_stats_call<bf16>(h, ld_h, classes, ld_c, labels, lse, n_rows, n_classes, dim, class_begin,
                                                      class_end, grad_out, hess_out, ld_out, s);
}

}  // extern "C"
