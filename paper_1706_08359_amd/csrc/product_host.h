// What the host sides of the products share: limits, tiles, launches of products over the rows of leaves, the plan of the
// weights' gradient.  (linear_leaves.hip: one leaf a row; routed_leaves.hip: several.)
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "../../include/gbdt_hist.h"
#include "library_state.h"

#include "leaf_product_kernels.h"

namespace gbdt_host {

using gbdt_internal::hip_failed;
using gbdt_tile::bf16;
using gbdt_tile::kChunk;
using gbdt_tile::Shape;

#define LAUNCHED(what)                                    \
  do {                                                    \
    hipError_t e_ = hipGetLastError();                    \
    if (e_ != hipSuccess) return hip_failed(e_, what);    \
  } while (0)

constexpr int64_t kMaxRows = (int64_t)1 << 30;     // rows, positions, classes
constexpr int64_t kMaxWidth = (int64_t)1 << 24;    // d_in, d_out, dim, leaves
constexpr int64_t kMaxLd = (int64_t)1 << 28;       // distances of rows
constexpr int64_t kMaxTiles = ((int64_t)1 << 31) - 1;   // of a call

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }
inline size_t pad256(size_t b) { return (b + 255) / 256 * 256; }

// Workgroups of `threads` that one launch takes, a multiple of 8: it counts its threads in 32 bits.
constexpr int64_t most_blocks(int threads) { return (((int64_t)1 << 32) - 1) / threads / 8 * 8; }

// Rows of whole 16-byte chunks: every row 16-byte aligned and `cols` whole chunks.
template <typename T>
bool whole_chunks(const void* p, int64_t ld, int64_t cols) {
  return ((uintptr_t)p & 15) == 0 && ld % kChunk<T> == 0 && cols % kChunk<T> == 0;
}

// A pointer that no element can lie at.
inline bool off_element(const void* p, int32_t dtype) { return ((uintptr_t)p & (dtype == GBDT_F32 ? 3 : 1)) != 0; }

// The tile of most calls, of whole chunks or not.  bf16: 128 x 128 by four wavefronts, two workgroups a compute unit.  f32: 64
// x 64, since its matrix instructions, 16 times slower, are the bound at any tile, and smaller tiles waste less of them.
template <typename T>
using Square = typename std::conditional<sizeof(T) == 2, Shape<T, 128, 128, 2, 2, true, true>, Shape<T, 64, 64, 2, 2, true>>::type;
template <typename T>
using SquareAny = typename std::conditional<sizeof(T) == 2, Shape<T, 128, 128, 2, 2, false>, Shape<T, 64, 64, 2, 2, false>>::type;

// Tiles of 256 x 256 by eight wavefronts, one workgroup a compute unit (f32: as any other; its products are 16 times slower
// and its loads never the bound).
template <typename T>
using Wide = typename std::conditional<sizeof(T) == 2, Shape<T, 256, 256, 2, 4, true, true>, Square<T>>::type;
// Taken where there is one for every unit.  (Softmax's loss, 4,096 x 32,768 x 512: 143 us against 159 in tiles of 128, 8,192 x
// 65,536 x 1,024: 917 against 1,100, 8,192 x 32,768 x 128: 141 against 153, 4,096 x 4,096 x 512, a tile a unit: 22 against 27; 2,048 x
// 4,096 x 1,024, a tile for every other unit: 30 against 25.)
template <typename T>
bool wide_tiles(int64_t rows, int64_t cols) {
  return sizeof(T) == 2 && ceil_div(rows, 256) * ceil_div(cols, 256) >= 256;
}

// Workgroups of the products over rows: the column tiles of a row tile are spread over as many as it takes to have eight a
// compute unit (four of the large ones), and no more, since a workgroup's first tile waits for its leaf and its rows.
// `launch(blocks)` is called with g.first set, more than once where there are millions of leaves.  many: the kernel takes more than one
// column tile.
template <class S, typename T, class Launch>
int leaf_rows_launches(gbdt_leaf::LeafArgs<T>& g, int64_t cols, int threads, bool many, const Launch& launch) {
  const int64_t row_tiles = (int64_t)g.n_positions / S::BM + g.n_leaves;
  const int64_t col_tiles = ceil_div(cols, S::BN);
  const int64_t most = (S::BM >= 256 ? 4 : 8) * gbdt_internal::cu_count();  // one or two at a time on a unit
  g.col_tiles = (uint32_t)col_tiles;
  g.cols_per = many ? (uint32_t)std::max<int64_t>(1, std::min(col_tiles, (int64_t)g.n_positions / S::BM * col_tiles / most)) : 1;
  const int64_t n = row_tiles * ceil_div(col_tiles, g.cols_per);
  if (n > kMaxTiles) return GBDT_EUNSUPPORTED;
  for (int64_t first = 0; first < n; first += most_blocks(threads)) {
    g.first = (uint32_t)first;
    launch(dim3((unsigned)std::min(n - first, most_blocks(threads))));
    LAUNCHED("a product of the leaves");
  }
  return GBDT_OK;
}

// The same by workgroups that stay (gbdt_leaf::rows_product): one a compute unit.
template <class S, typename T, class Launch>
int rows_launches(gbdt_leaf::LeafArgs<T>& g, int64_t cols, const Launch& launch) {
  if constexpr (!gbdt_leaf::kStays<S>) return leaf_rows_launches<S>(g, cols, S::NT, true, launch);
  const int64_t col_tiles = ceil_div(cols, S::BN), n = ((int64_t)g.n_positions / S::BM + g.n_leaves) * col_tiles;
  if (n > kMaxTiles || g.n_leaves > gbdt_leaf::kStayLeaves) return GBDT_EUNSUPPORTED;
  g.col_tiles = (uint32_t)col_tiles;
  launch(dim3((unsigned)std::min(round_up(n, 8), std::max<int64_t>(8, gbdt_internal::cu_count() / 8 * 8))));
  LAUNCHED("a product of the leaves");
  return GBDT_OK;
}

// Leaves long enough for tiles of 256 rows, columns for more than one of 128, and such tiles for all compute units.  (100,000 x
// 256 -> 2,000, gradient of the input, leaves of 392 rows on average: 277 us against 318 us in tiles of 128.  2,000 x 2,000 ->
// 256 in one leaf, 8 tiles: 42 us against 12 in small ones.)
template <typename T>
bool long_leaves(const gbdt_leaf::LeafArgs<T>& g, int64_t cols, int64_t bn) {
  return sizeof(T) <= 2 && g.n_positions >= 192 * (int64_t)g.n_leaves && g.n_positions / 256 * ceil_div(cols, bn) >= gbdt_internal::cu_count();
}
template <typename T>
bool wide_leaves(const gbdt_leaf::LeafArgs<T>& g, int64_t cols) {
  return cols > 128 && long_leaves(g, cols, 256);
}

// How the weights' gradient is taken: tiles of bm outputs x bn inputs, and the positions between cuts: two pieces of whole
// tiles a compute unit, from 256 positions on and up to as many as a workgroup lists at once, which evens out unequal leaves; more
// where the sums that pieces leave behind would pass kSlotBytes.  (Two pieces a unit whatever their length, 64 MiB of sums: dW and
// db of 400,000 x 2,000 x 256 in 255 leaves 946 us against 1,046, but f32 100,000 x 2,000 x 256 in 31 leaves 2,248 against 1,447.  Tiles of 256 x 256,
// one workgroup a unit, took as long: 100,000 x 2,000 x 256, leaves of 392 rows on average, 330 us against 350.  64 outputs a
// tile where there are no more: 100,000 x 700 -> 32, all gradients, 155 us against 173 with 128.)
constexpr int64_t kSlotBytes = (int64_t)512 << 20;
constexpr int kGradThreads = 256;  // of a workgroup
constexpr int64_t kMaxCuts = 65535;  // (of a launch's second dimension)
struct LeafGradPlan {
  int64_t bm, bn, tiles, cut;
  size_t bytes;
};
// few: tiles of 64 outputs whatever their number.
inline LeafGradPlan leaf_grad_plan(int64_t e, int64_t n_positions, int64_t d_in, int64_t d_out, int64_t units, bool few = false) {
  LeafGradPlan p;
  p.bm = e == 4 || d_out <= 64 || few ? 64 : 128;
  p.bn = e == 4 ? 64 : 128;
  p.tiles = ceil_div(d_out, p.bm) * ceil_div(d_in, p.bn);
  const int64_t fill = p.tiles >= 2 * units ? n_positions : ceil_div(n_positions * p.tiles, 2 * units);
  const int64_t slots = 2 * (d_in + 1) * d_out * (int64_t)sizeof(float);  // of a cut
  const int64_t most = std::max<int64_t>(1, std::min(kMaxCuts, kSlotBytes / slots));
  p.cut = std::min<int64_t>(gbdt_leaf::kCopiedIds, std::max<int64_t>(256, fill));
  p.cut = round_up(std::max(p.cut, ceil_div(n_positions, most)), 64);
  const int64_t blocks = ceil_div(n_positions, p.cut);
  p.bytes = blocks < 2 ? 0 : pad256((size_t)(blocks * slots));
  return p;
}

template <class S, bool LISTED, typename T>
int launch_leaf_grad_weight(gbdt_leaf::LeafArgs<T>& g, hipStream_t s, int64_t outputs) {
  g.col_tiles = (uint32_t)(g.dw ? ceil_div(g.d_in, S::BN) : 1);
  g.row_tiles = (uint32_t)ceil_div(outputs, S::BM);
  // (as leaf_rows_launches, counting a piece a cut)
  const int64_t pieces = (int64_t)g.n_positions / g.cut + g.n_leaves;
  const int64_t tiles = pieces * g.col_tiles * g.row_tiles, most = 8 * gbdt_internal::cu_count();
  g.cols_per = (uint32_t)std::max<int64_t>(1, std::min<int64_t>({(int64_t)g.col_tiles, tiles / most, 4}));
  const int64_t a_piece = (int64_t)g.col_tiles * g.row_tiles;
  static_assert(S::NT <= kGradThreads, "eight pieces at least are a launch");
  const int64_t at_once = most_blocks(S::NT) / a_piece / 8 * 8;
  for (int64_t first = 0; first < pieces; first += at_once) {
    g.first = (uint32_t)first;
    const int64_t blocks = round_up(std::min(pieces - first, at_once), 8) * a_piece;
    if (g.cut > gbdt_leaf::kCopiedIds) {
      gbdt_leaf::leaf_grad_weight_kernel<S, true, LISTED><<<dim3((unsigned)blocks), dim3(S::NT), 0, s>>>(g);
    } else {
      gbdt_leaf::leaf_grad_weight_kernel<S, false, LISTED><<<dim3((unsigned)blocks), dim3(S::NT), 0, s>>>(g);
    }
    LAUNCHED("leaf_grad_weight_kernel");
  }
  return GBDT_OK;
}

// Adds up the sums that pieces left behind.
template <bool LISTED, typename T>
int launch_leaf_grad_join(const gbdt_leaf::LeafArgs<T>& g, hipStream_t s) {
  const int64_t cuts = ceil_div(g.n_positions, g.cut) - 1;
  if (cuts > 0) {
    // (few workgroups a cut: most find that no leaf crosses theirs first)
    const int64_t per = ceil_div((int64_t)(g.d_in + 1) * g.d_out, 256);
    const int64_t most = std::max<int64_t>(16, 4096 / cuts);
    gbdt_leaf::leaf_grad_join_kernel<T, LISTED><<<dim3((unsigned)std::min<int64_t>(per, most), (unsigned)cuts), dim3(256), 0, s>>>(g);
    LAUNCHED("leaf_grad_join_kernel");
  }
  return GBDT_OK;
}

}  // namespace gbdt_host
