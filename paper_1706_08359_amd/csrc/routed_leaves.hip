// Rows routed to several linear leaves, and leaf products in 8-bit integers: host side of gbdt_route, gbdt_route_grad,
// gbdt_mixture_product, gbdt_mixture_product_grad, gbdt_rows_quantize, gbdt_leaf_product_codes and gbdt_mixture_product_codes (checks,
// choice of tile, scratch, launches).  The kernels are in route_kernels.h, routed_kernels.h and code_kernels.h.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "../../include/gbdt_hist.h"
#include "library_state.h"

#include "code_kernels.h"
#include "product_host.h"
#include "route_kernels.h"
#include "routed_kernels.h"

namespace {

using namespace gbdt_host;
using gbdt_code::CodeArgs;
using gbdt_router::RouteArgs;
using gbdt_routed::CombineArgs;
using gbdt_routed::RoutedArgs;

// ---------------------------------------------------------------- routing

int route_check(const void* logits, int64_t ld, int64_t n_rows, int32_t n_leaves, int32_t dtype, int32_t score, int32_t k, float scale) {
  if (n_rows < 0 || n_leaves <= 0 || k <= 0 || k > n_leaves || ld < n_leaves || !isfinite(scale)) return GBDT_EINVAL;
  if (dtype != GBDT_F32 && dtype != GBDT_BF16) return GBDT_EINVAL;
  if (score != GBDT_SOFTMAX && score != GBDT_SIGMOID) return GBDT_EINVAL;
  if (off_element(logits, dtype)) return GBDT_EINVAL;
  if (n_rows >= kMaxRows || ld >= kMaxLd || n_leaves > gbdt_router::kMaxLeaves || k > gbdt_router::kMaxChosen) return GBDT_EUNSUPPORTED;
  return GBDT_OK;
}

// launch(first, blocks) for `rows` rows, `per` of them a workgroup of 256 threads, as many at a time as a launch takes.
template <class Launch>
int row_launches(int64_t rows, int64_t per, const char* what, const Launch& launch) {
  for (int64_t first = 0; first < rows; first += most_blocks(256) * per) {
    launch(first, dim3((unsigned)std::min(ceil_div(rows - first, per), most_blocks(256))));
    LAUNCHED(what);
  }
  return GBDT_OK;
}

template <typename T, int LANES, int PER>
int launch_route(RouteArgs g, bool grad, hipStream_t s) {
  static_assert(gbdt_router::kThreads == 256, "");
  return row_launches(g.n_rows, 256 / LANES, "routing", [&](int64_t first, dim3 blocks) {
    g.first = first;
    if (grad) {
      gbdt_router::route_grad_kernel<T, LANES, PER><<<blocks, dim3(256), 0, s>>>(g);
    } else if (g.bias == nullptr && g.group_best == 1) {
      gbdt_router::route_kernel<T, LANES, PER, false><<<blocks, dim3(256), 0, s>>>(g);
    } else {
      gbdt_router::route_kernel<T, LANES, PER, true><<<blocks, dim3(256), 0, s>>>(g);
    }
  });
}

// (f32, calls among others.  By logits: 400,000 rows x 255, four leaves each: 107 us by sixteen lanes a row, 114 by eight, 139 by 32, 211 by 64;
// 100,000 x 285, 16 leaves each: 100 by sixteen, 114 by 32; x 700: 190 by 32, 216 by 64; x 1,024: 224 by 32, 251 by 64.  By values: 65,536 x
// 64 and the gradient: 22.6 by eight, 24.7 by sixteen; 100,000 x 285, 16 leaves each: 136 and 159; x 700: 269 and 320; x 1,024: 310 and 364; but
// 400,000 x 200, eight leaves each: 242 by sixteen, 223 by eight.)
template <typename T>
int route(const RouteArgs& g, bool grad, hipStream_t s) {
  if (g.n_leaves <= 64) return launch_route<T, 8, 8>(g, grad, s);
  if (g.n_leaves <= 128) return launch_route<T, 16, 8>(g, grad, s);
  if (g.n_leaves <= 256) return launch_route<T, 16, 16>(g, grad, s);
  if (g.n_leaves <= 384) return launch_route<T, 16, 24>(g, grad, s);
  if (g.n_leaves <= 512) return launch_route<T, 32, 16>(g, grad, s);
  if (g.n_leaves <= 768) return launch_route<T, 32, 24>(g, grad, s);
  return launch_route<T, 32, 32>(g, grad, s);
}

// ---------------------------------------------------------------- lists of pairs

struct ListPlan {
  int64_t pairs, run, runs;  // runs 0: one workgroup lists all
  size_t table_bytes;        // of the counts: no less for more pairs
  size_t offsets_bytes, row_bytes, count_bytes;
  size_t bytes() const { return offsets_bytes + 2 * row_bytes + count_bytes; }
};
// One workgroup lists few pairs by itself, which is one launch instead of three.
constexpr int64_t kFewPairs = 8192;
ListPlan list_plan(int64_t pairs, int64_t n_leaves) {
  ListPlan p;
  p.pairs = pairs;
  p.offsets_bytes = pad256((size_t)(n_leaves + 1) * 8);
  p.row_bytes = pad256((size_t)pairs * 4);
  p.table_bytes = p.count_bytes = 0;
  if (pairs <= kFewPairs && n_leaves <= gbdt_router::kFewListLeaves) {
    p.run = round_up(ceil_div(pairs, gbdt_router::kListWaves), 64);
    p.runs = 0;
  } else {
    const int64_t most = std::min<int64_t>(2048, std::max<int64_t>(64, ((int64_t)8 << 20) / n_leaves));
    p.run = std::max<int64_t>(256, round_up(ceil_div(pairs, most), 64));
    p.runs = std::max<int64_t>(1, ceil_div(pairs, p.run));
    p.table_bytes = pad256((size_t)(n_leaves * std::min(most, std::max<int64_t>(1, ceil_div(pairs, 256)))) * 4);
    p.count_bytes = p.table_bytes + pad256((size_t)n_leaves * 4);
  }
  return p;
}

template <int LEAVES>
int launch_lists(const gbdt_router::ListArgs& g, hipStream_t s) {
  gbdt_router::list_count_kernel<LEAVES><<<dim3(g.runs), dim3(64), 0, s>>>(g);
  LAUNCHED("list_count_kernel");
  gbdt_router::list_scan_kernel<<<dim3(g.n_leaves), dim3(64), 0, s>>>(g);
  LAUNCHED("list_scan_kernel");
  gbdt_router::list_place_kernel<LEAVES><<<dim3(g.runs), dim3(64), 0, s>>>(g);
  LAUNCHED("list_place_kernel");
  return GBDT_OK;
}

// Where a list lies in scratch of plan.bytes().
void list_places(const ListPlan& plan, char* scratch, const int64_t** offsets, const int32_t** row, const int32_t** pair) {
  *offsets = (int64_t*)scratch;
  *row = (int32_t*)(scratch + plan.offsets_bytes);
  *pair = (int32_t*)(scratch + plan.offsets_bytes + plan.row_bytes);
}

// Lists the pairs of the rows that `leaves` begins with, and says where.
int make_lists(const ListPlan& plan, const int32_t* leaves, int32_t n_leaves, int32_t k, char* scratch, const int64_t** offsets,
               const int32_t** row, const int32_t** pair, hipStream_t s) {
  list_places(plan, scratch, offsets, row, pair);
  gbdt_router::ListArgs g = {};
  g.leaves = leaves;
  g.offsets = const_cast<int64_t*>(*offsets);
  g.row = const_cast<int32_t*>(*row);
  g.pair = const_cast<int32_t*>(*pair);
  g.counts = (int32_t*)(scratch + plan.offsets_bytes + 2 * plan.row_bytes);
  g.totals = g.counts + plan.table_bytes / 4;
  g.n_pairs = (int32_t)plan.pairs;
  g.n_leaves = n_leaves;
  g.k = k;
  g.run = (int32_t)plan.run;
  g.runs = (int32_t)plan.runs;
  if (plan.runs == 0) {
    gbdt_router::list_few_kernel<<<dim3(1), dim3(gbdt_router::kListWaves * 64), 0, s>>>(g);
    LAUNCHED("list_few_kernel");
    return GBDT_OK;
  }
  if (n_leaves <= 1024) return launch_lists<1024>(g, s);
  if (n_leaves <= 4096) return launch_lists<4096>(g, s);
  return launch_lists<gbdt_router::kMaxListLeaves>(g, s);
}

// ---------------------------------------------------------------- mixtures

// Slots of so many rows at a time as take this, or of 1,024.
constexpr int64_t kSlotsBytes = (int64_t)256 << 20;
// Weighted gradients of so many outputs at a time as take this, or of a tile, which is one of 64 outputs where 128 would take more than the
// second number.
constexpr int64_t kGatedBytes = (int64_t)256 << 20, kTileBytes = (int64_t)1 << 30;
constexpr int32_t kMaxSlots = 64;  // leaves a row
constexpr int64_t kMaxGridRows = 65535;  // rows of a launch's second dimension

// block: columns of a part of a dot product.
struct SlotPlan {
  int64_t rows, ld, blocks;  // rows at a time
  ListPlan list;
  size_t slots_bytes, dots_bytes;
  size_t bytes() const { return list.bytes() + slots_bytes + dots_bytes; }
};
SlotPlan slot_plan(int64_t n_rows, int64_t k, int64_t n_leaves, int64_t cols, int64_t block, bool dots) {
  SlotPlan p = {};
  if (k == 1 && !dots) {  // answers go to their rows, all at once
    p.rows = n_rows;
    p.list = list_plan(n_rows, n_leaves);
    return p;
  }
  p.ld = round_up(cols, 4);
  p.blocks = ceil_div(cols, block);
  p.rows = std::min(n_rows, std::max<int64_t>(1024, kSlotsBytes / (k * p.ld * 4)));
  p.list = list_plan(p.rows * k, n_leaves);
  p.slots_bytes = pad256((size_t)(p.rows * k * p.ld * 4));
  p.dots_bytes = dots ? pad256((size_t)(p.rows * k * p.blocks) * 4) : 0;
  return p;
}

struct WeightPlan {
  ListPlan list;
  int64_t piece;  // outputs at a time
  int64_t ld;
  LeafGradPlan sums;
  size_t gated_bytes;
  size_t bytes() const { return list.bytes() + gated_bytes + sums.bytes; }
};
WeightPlan weight_plan(int64_t n_rows, int64_t k, int64_t n_leaves, int64_t d_in, int64_t d_out, int64_t e, int64_t units) {
  WeightPlan p;
  const int64_t pairs = n_rows * k;
  p.list = list_plan(pairs, n_leaves);
  const int64_t a_value = e == 2 ? 4 : e;  // (two of 16 bits, gbdt_leaf::kRowsEach)
  p.sums = leaf_grad_plan(e, pairs, d_in, d_out, units, pairs * 128 * a_value > kTileBytes);
  p.piece = std::max(p.sums.bm, kGatedBytes / std::max<int64_t>(1, pairs * a_value) / p.sums.bm * p.sums.bm);
  p.piece = std::min(p.piece, d_out);
  p.ld = round_up(p.piece, 16 / e);
  p.gated_bytes = pad256((size_t)(pairs * p.ld * a_value));
  return p;
}

int mixture_check(int64_t n_rows, int32_t k, int32_t n_leaves, int32_t d_in, int32_t d_out, const void* leaves, const void* gates,
                  int32_t dtype) {
  if (n_rows < 0 || k <= 0 || n_leaves <= 0 || d_in <= 0 || d_out <= 0) return GBDT_EINVAL;
  if (n_rows > 0 && (!leaves || !gates)) return GBDT_EINVAL;
  if (((uintptr_t)leaves & 3) != 0 || ((uintptr_t)gates & 3) != 0) return GBDT_EINVAL;
  if (dtype != GBDT_F32 && dtype != GBDT_BF16) return GBDT_EINVAL;
  if (n_rows >= kMaxRows || k > kMaxSlots || n_rows * k >= kMaxRows || n_leaves > gbdt_router::kMaxListLeaves || d_in >= kMaxWidth ||
      d_out >= kMaxWidth)
    return GBDT_EUNSUPPORTED;
  return GBDT_OK;
}

// Leaves of few positions: tiles of 32 rows, which waste less and leave room for more workgroups reading matrices.
template <typename T>
bool short_leaves(const gbdt_leaf::LeafArgs<T>& g) {
  return g.n_positions <= 32 * (int64_t)g.n_leaves;
}
template <typename T>
using Short = Shape<T, 32, 128, 1, 2, true>;

// Tiles of 256 rows need long leaves, and no more of them than a workgroup that stays has room for.
template <typename T>
bool long_leaves_of(const gbdt_leaf::LeafArgs<T>& g, int64_t cols, int64_t bn) {
  return g.n_leaves <= gbdt_leaf::kStayLeaves && (bn < 256 || cols > 128) && long_leaves(g, cols, bn);
}

template <class S, gbdt_routed::Leaves WHAT, typename T>
int launch_routed_product(RoutedArgs<T>& g, hipStream_t s) {
  return rows_launches<S>(g, g.d_out, [&](dim3 blocks) {
    gbdt_routed::routed_product_kernel<S, WHAT><<<blocks, dim3(S::NT), 0, s>>>(g);
  });
}

template <gbdt_routed::Leaves WHAT, typename T>
int routed_product(RoutedArgs<T>& g, hipStream_t s) {
  const bool direct = whole_chunks<T>(g.x, g.ld_x, g.d_in) && whole_chunks<T>(g.w, g.d_in, g.d_in);
  if constexpr (sizeof(T) == 2) {
    if (direct) {
      if (short_leaves(g)) return launch_routed_product<Short<T>, WHAT>(g, s);
      if (g.d_out <= 64) return launch_routed_product<Shape<T, 128, 64, 4, 1, true>, WHAT>(g, s);
      if (long_leaves_of(g, g.d_out, 256)) return launch_routed_product<Wide<T>, WHAT>(g, s);
      if (long_leaves_of(g, g.d_out, 128)) return launch_routed_product<Shape<T, 256, 128, 4, 2, true, false, 3>, WHAT>(g, s);
    }
  }
  return direct ? launch_routed_product<Square<T>, WHAT>(g, s) : launch_routed_product<SquareAny<T>, WHAT>(g, s);
}

template <class S, typename T>
int launch_routed_grad_input(RoutedArgs<T>& g, hipStream_t s) {
  return rows_launches<S>(g, g.d_in, [&](dim3 blocks) {
    if (g.dots) {
      gbdt_routed::routed_grad_input_kernel<S, true><<<blocks, dim3(S::NT), 0, s>>>(g);
    } else {
      gbdt_routed::routed_grad_input_kernel<S, false><<<blocks, dim3(S::NT), 0, s>>>(g);
    }
  });
}

template <typename T>
int routed_grad_input(RoutedArgs<T>& g, hipStream_t s) {
  const bool direct = whole_chunks<T>(g.dy, g.ld_dy, g.d_out) && whole_chunks<T>(g.w, g.d_in, g.d_in);
  if constexpr (sizeof(T) == 2) {
    if (direct && short_leaves(g)) return launch_routed_grad_input<Short<T>>(g, s);
    if (direct && long_leaves_of(g, g.d_in, 256)) return launch_routed_grad_input<Wide<T>>(g, s);
  }
  return direct ? launch_routed_grad_input<Square<T>>(g, s) : launch_routed_grad_input<SquareAny<T>>(g, s);
}

template <typename O, int LANES>
int launch_combine(const CombineArgs<O>& g, hipStream_t s) {
  const dim3 blocks((unsigned)ceil_div(g.n_rows, 256 / LANES));
  if (g.dgates) {
    gbdt_routed::combine_kernel<O, LANES, true><<<blocks, dim3(256), 0, s>>>(g);
  } else {
    gbdt_routed::combine_kernel<O, LANES, false><<<blocks, dim3(256), 0, s>>>(g);
  }
  LAUNCHED("combine_kernel");
  return GBDT_OK;
}
// (20,011 rows x 3 leaves, 137 -> 33, f32, a training step: 148 us with sixteen lanes a row of 137 values, 162 with 64.)
template <typename O>
int combine(const CombineArgs<O>& g, hipStream_t s) {
  return g.cols <= 256 ? launch_combine<O, 16>(g, s) : launch_combine<O, 64>(g, s);
}

// So few rows that a wavefront for every few outputs of a row takes less than lists, tiles and slots.  It reads a matrix again for
// every row that takes the leaf: pairs x outputs x inputs, of 64 chunks at least, at 3.8 million a us (f32 2.1, codes 9), after 4 us; the
// other way is 13 us and each matrix that is taken once, 0.3 us a million values more (f32, whose tiles are mostly empty, 1.2; codes
// 0.18).  (us, this way / the other, k = 4.  bf16, pairs of 64 matrices of 1,024 x 1,024: 64 19/26, 128 35/30, 256 58/32; of 255 of 700 x
// 256: 256 16/29, 512 25/29; of 8 of 256 x 64: 512 8.6/15, 2,000 16/16.  f32: 128 69/106, 256 138/107; 512 47/66, 2,000 170/80; 2,000 12/18.
// Codes: 128 18/25, 256 32/25; 512 15/23, 2,000 43/26; 512 9.6/16, 2,000 13/17.  The kernels take four leaves at a time, and a k that is no multiple
// of four costs this way more: k = 1 bf16 128 60/27, 512 56/26, 12/15; f32 83/102, 64/63; codes, the rule's worst, 30/22, 31/19,
// 10/16.)
template <typename T>
bool few_rows(int64_t n_rows, int64_t k, int64_t n_leaves, int64_t d_in, int64_t d_out) {
  const double products = (double)(n_rows * k) * (double)d_out * (double)std::max<int64_t>(d_in, 64 * kChunk<T>);
  const double taken = (double)std::min(n_leaves, n_rows * k) * (double)d_in * (double)d_out;
  const double room = sizeof(T) == 2 ? 34e6 + 1.2 * taken : sizeof(T) == 4 ? 23e6 + 2.5 * taken : 80e6 + 1.6 * taken;
  // (four rows: 2^24 outputs at most, two a wavefront)
  return n_rows <= 4 || (n_rows <= kMaxGridRows && products <= room && n_rows * ceil_div(d_out, 2) <= most_blocks(64));
}

// Products of all rows, kept in slots and added up, so many rows at a time as the plan says.  products(g, r): of the rows from r on,
// to the slots.  Where answers go to rows directly (`direct`), the plan's list is all that is used of the scratch.
template <class G, typename O, class Products>
int by_slots(const G& all, int64_t n_rows, int64_t cols, const CombineArgs<O>& to, const SlotPlan& plan, char* scratch, bool direct,
             const Products& products, hipStream_t s) {
  for (int64_t r = 0; r < n_rows; r += plan.rows) {
    const int64_t n = std::min(plan.rows, n_rows - r);
    G g = all;
    g.leaves += r * g.k;
    g.gates += r * g.k;
    const ListPlan list = n == plan.rows ? plan.list : list_plan(n * g.k, g.n_leaves);
    int rc = make_lists(list, g.leaves, g.n_leaves, g.k, scratch, &g.offsets, &g.row_idx, &g.pair_idx, s);
    if (rc != GBDT_OK) return rc;
    char* at = scratch + plan.list.bytes();
    g.slots = direct || !to.out ? nullptr : (float*)at;
    g.dots = to.dgates ? (float*)(at + plan.slots_bytes) : nullptr;
    g.ld_slots = plan.ld;
    g.blocks = (int32_t)plan.blocks;
    g.n_rows = (int32_t)n;
    g.n_positions = (int32_t)(n * g.k);
    if ((rc = products(g, r)) != GBDT_OK) return rc;
    if (direct) {
      gbdt_routed::clear_rows_kernel<O><<<dim3((unsigned)ceil_div(n, 256)), dim3(256), 0, s>>>(g.leaves, g.n_leaves, (int32_t)n, (int32_t)cols,
                                                                                              to.out + r * to.ld_out, to.ld_out);
      LAUNCHED("clear_rows_kernel");
      continue;
    }
    CombineArgs<O> c = to;
    c.slots = g.slots;
    c.dots = g.dots;
    c.leaves = g.leaves;
    c.gates = g.gates;
    if (c.out) c.out += r * c.ld_out;
    if (c.dgates) c.dgates += r * g.k, c.dy += r * c.ld_dy;
    c.ld = plan.ld;
    c.blocks = g.blocks;
    c.n_rows = (int32_t)n;
    c.n_leaves = g.n_leaves;
    c.k = g.k;
    c.cols = (int32_t)cols;
    if ((rc = combine(c, s)) != GBDT_OK) return rc;
  }
  return GBDT_OK;
}

template <typename T>
int mixture_product(RoutedArgs<T>& g, int64_t n_rows, hipStream_t s) {
  if (few_rows<T>(n_rows, g.k, g.n_leaves, g.d_in, g.d_out)) {
    if (n_rows * g.d_out <= 1024) {
      gbdt_routed::routed_few_kernel<T, 1><<<dim3(g.d_out, (unsigned)n_rows), dim3(64), 0, s>>>(g);
    } else {
      gbdt_routed::routed_few_kernel<T, 2><<<dim3((unsigned)ceil_div(g.d_out, 2), (unsigned)n_rows), dim3(64), 0, s>>>(g);
    }
    LAUNCHED("routed_few_kernel");
    return GBDT_OK;
  }
  const SlotPlan plan = slot_plan(n_rows, g.k, g.n_leaves, g.d_out, gbdt_routed::block_columns<T>, false);
  void* ws = nullptr;
  const int rc = gbdt_internal::workspace(plan.bytes(), s, &ws);
  if (rc != GBDT_OK) return rc;
  CombineArgs<T> to = {};
  to.out = g.y;
  to.ld_out = g.ld_y;
  const bool direct = g.k == 1;
  return by_slots(g, n_rows, g.d_out, to, plan, (char*)ws, direct,
                  [&](RoutedArgs<T>& piece, int64_t r) {
                    piece.x = g.x + r * g.ld_x;
                    piece.y = g.y + r * g.ld_y;
                    return direct ? routed_product<gbdt_routed::Leaves::kRows>(piece, s) : routed_product<gbdt_routed::Leaves::kSlots>(piece, s);
                  },
                  s);
}

// The outputs' sums, of all pieces.
template <typename T>
int gated_sums(const RoutedArgs<T>& g, hipStream_t s) {
  constexpr int columns = gbdt_routed::kSumLanes * kChunk<T>;
  const int64_t n = ((int64_t)g.n_positions / g.cut + g.n_leaves) * ceil_div(g.d_out, columns);
  for (int64_t first = 0; first < n; first += most_blocks(gbdt_routed::kSumThreads)) {
    const dim3 blocks((unsigned)std::min(n - first, most_blocks(gbdt_routed::kSumThreads)));
    gbdt_routed::gated_sums_kernel<T><<<blocks, dim3(gbdt_routed::kSumThreads), 0, s>>>(g, first);
    LAUNCHED("gated_sums_kernel");
  }
  return GBDT_OK;
}

template <typename T>
int mixture_weights(RoutedArgs<T> g, int64_t n_rows, const WeightPlan& plan, char* scratch, bool listed, hipStream_t s) {
  g.n_rows = (int32_t)n_rows;
  g.n_positions = (int32_t)(n_rows * g.k);
  list_places(plan.list, scratch, &g.offsets, &g.row_idx, &g.pair_idx);
  int rc = GBDT_OK;
  if (!listed && (rc = make_lists(plan.list, g.leaves, g.n_leaves, g.k, scratch, &g.offsets, &g.row_idx, &g.pair_idx, s)) != GBDT_OK) return rc;
  T* gated = (T*)(scratch + plan.list.bytes());
  if (!g.dw) g.d_in = kChunk<T>;  // (as the plan has it)
  g.cut = (int32_t)plan.sums.cut;
  g.partial = (float*)(scratch + plan.list.bytes() + plan.gated_bytes);
  const bool direct = whole_chunks<T>(g.x, g.ld_x, g.d_in);
  const RoutedArgs<T> whole = g;
  // (f32 operands of dW are as good as the products that the outputs' sums are of, and add them up on their way: 20,011 rows x 3 leaves,
  // 137 -> 33, a training step: 144 us, 153 with sums by themselves)
  if (sizeof(T) == 2 || !g.dw) {
    if (g.dbias && (rc = gated_sums(g, s)) != GBDT_OK) return rc;
    g.dbias = nullptr;
  }
  for (int64_t first = 0; g.dw && first < g.d_out; first += plan.piece) {
    const int64_t cols = std::min(plan.piece, whole.d_out - first);
    if (n_rows > 0) {
      const bool narrow = plan.ld * (int64_t)sizeof(T) <= 1024;
      rc = row_launches(g.n_positions, narrow ? 16 : 4, "gated_rows_kernel", [&](int64_t from, dim3 blocks) {
        if (narrow) {
          gbdt_routed::gated_rows_kernel<T, 16><<<blocks, dim3(256), 0, s>>>(whole, gated, plan.ld, (int)first, (int)cols, (int)from);
        } else {
          gbdt_routed::gated_rows_kernel<T, 64><<<blocks, dim3(256), 0, s>>>(whole, gated, plan.ld, (int)first, (int)cols, (int)from);
        }
      });
      if (rc != GBDT_OK) return rc;
    }
    g.dy = gated;
    g.ld_dy = plan.ld;
    g.row_first = (int32_t)first;
    if constexpr (sizeof(T) == 2) {
      if (plan.sums.bm == 64)
        rc = direct ? launch_leaf_grad_weight<Shape<T, 64, 128, 1, 4, true, true>, true>(g, s, cols)
                    : launch_leaf_grad_weight<Shape<T, 64, 128, 1, 4, false>, true>(g, s, cols);
      else
        rc = direct ? launch_leaf_grad_weight<Square<T>, true>(g, s, cols) : launch_leaf_grad_weight<SquareAny<T>, true>(g, s, cols);
    } else {
      rc = direct ? launch_leaf_grad_weight<Square<T>, true>(g, s, cols) : launch_leaf_grad_weight<SquareAny<T>, true>(g, s, cols);
    }
    if (rc != GBDT_OK) return rc;
  }
  return launch_leaf_grad_join<true>(whole, s);
}

template <typename T>
int mixture_product_grad(RoutedArgs<T>& g, int64_t n_rows, hipStream_t s) {
  const bool weights = g.dw || g.dbias, rows = (g.dx || g.dgates) && n_rows > 0;
  if (!weights && !rows) return GBDT_OK;
  const SlotPlan slots = slot_plan(n_rows, g.k, g.n_leaves, g.d_in, gbdt_routed::block_columns<T>, true);
  const WeightPlan sums = weight_plan(n_rows, g.k, g.n_leaves, g.dw ? g.d_in : kChunk<T>, g.d_out, sizeof(T), gbdt_internal::cu_count());
  if (weights && sums.sums.tiles > most_blocks(kGradThreads) / 8) return GBDT_EUNSUPPORTED;
  void* ws = nullptr;
  int rc = gbdt_internal::workspace(std::max(rows ? slots.bytes() : 0, weights ? sums.bytes() : 0), s, &ws);
  if (rc != GBDT_OK) return rc;
  if (rows) {
    CombineArgs<T> to = {};
    to.out = g.dx;
    to.ld_out = g.ld_dx;
    to.dy = g.dy;
    to.bias = g.bias;
    to.dgates = g.dgates;
    to.ld_dy = g.ld_dy;
    to.d_out = g.d_out;
    rc = by_slots(g, n_rows, g.d_in, to, slots, (char*)ws, false,
                  [&](RoutedArgs<T>& piece, int64_t r) {
                    piece.dy = g.dy + r * g.ld_dy;
                    if (g.dgates) piece.x = g.x + r * g.ld_x;
                    return routed_grad_input(piece, s);
                  },
                  s);
    if (rc != GBDT_OK) return rc;
  }
  // (rows that were all taken at once have left the whole list in its place)
  return weights ? mixture_weights(g, n_rows, sums, (char*)ws, rows && slots.rows == n_rows, s) : GBDT_OK;
}

template <typename T>
int mixture_call(const void* x, int64_t ld_x, const void* weight, const void* bias, const int32_t* leaves, const float* gates, int64_t n_rows,
                 int32_t k, int32_t n_leaves, int32_t d_in, int32_t d_out, void* y_out, int64_t ld_y, hipStream_t s) {
  RoutedArgs<T> g = {};
  g.x = (const T*)x;
  g.w = (const T*)weight;
  g.bias = (const T*)bias;
  g.y = (T*)y_out;
  g.leaves = leaves;
  g.gates = gates;
  g.ld_x = ld_x;
  g.ld_y = ld_y;
  g.n_leaves = n_leaves;
  g.d_in = d_in;
  g.d_out = d_out;
  g.k = k;
  return mixture_product(g, n_rows, s);
}

template <typename T>
int mixture_grad_call(const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, const void* weight, const void* bias, const int32_t* leaves,
                      const float* gates, int64_t n_rows, int32_t k, int32_t n_leaves, int32_t d_in, int32_t d_out, void* dx_out,
                      int64_t ld_dx, void* dweight_out, void* dbias_out, float* dgates_out, hipStream_t s) {
  RoutedArgs<T> g = {};
  g.x = (const T*)x;
  g.dy = (const T*)dy;
  g.w = (const T*)weight;
  g.bias = (const T*)bias;
  g.dx = (T*)dx_out;
  g.dw = (T*)dweight_out;
  g.dbias = (T*)dbias_out;
  g.dgates = dgates_out;
  g.leaves = leaves;
  g.gates = gates;
  g.ld_x = ld_x;
  g.ld_dy = ld_dy;
  g.ld_dx = ld_dx;
  g.n_leaves = n_leaves;
  g.d_in = d_in;
  g.d_out = d_out;
  g.k = k;
  return mixture_product_grad(g, n_rows, s);
}

// ---------------------------------------------------------------- 8-bit integers

int code_check(const void* codes, int64_t ld_codes, const float* scales, const void* weight, const float* weight_scales, const float* bias,
               int64_t n_rows, int32_t d_in, int32_t d_out, int32_t dtype, const void* y_out, int64_t ld_y) {
  const int64_t padded = round_up(d_in, 16);
  if (ld_codes < padded || ld_codes % 16 != 0 || ((uintptr_t)codes & 15) != 0 || ((uintptr_t)weight & 15) != 0) return GBDT_EINVAL;
  if (!weight || !weight_scales || ld_y < d_out || off_element(y_out, dtype)) return GBDT_EINVAL;
  if (((uintptr_t)scales & 3) != 0 || ((uintptr_t)weight_scales & 3) != 0 || ((uintptr_t)bias & 3) != 0) return GBDT_EINVAL;
  if (n_rows > 0 && (!codes || !scales || !y_out)) return GBDT_EINVAL;
  if (padded > gbdt_code::kMaxWidth || ld_codes >= kMaxLd || ld_y >= kMaxLd) return GBDT_EUNSUPPORTED;
  return GBDT_OK;
}

template <typename T, int CHUNKS>
int launch_quantize(const gbdt_code::QuantizeArgs& all, hipStream_t s) {
  return row_launches(all.n_rows, 4, "quantize_kernel", [&](int64_t first, dim3 blocks) {
    gbdt_code::QuantizeArgs g = all;
    g.x = (const T*)all.x + first * all.ld_x;
    g.codes += first * all.ld_codes;
    g.scales += first;
    g.n_rows -= first;
    gbdt_code::quantize_kernel<T, CHUNKS><<<blocks, dim3(256), 0, s>>>(g);
  });
}
template <typename T>
int quantize(const gbdt_code::QuantizeArgs& g, hipStream_t s) {
  if (g.padded <= 512) return launch_quantize<T, 1>(g, s);
  if (g.padded <= 1024) return launch_quantize<T, 2>(g, s);
  return launch_quantize<T, 4>(g, s);
}

using gbdt_code::Place;

template <class S, typename O, Place WHERE>
int launch_code_product(CodeArgs& g, hipStream_t s) {
  return rows_launches<S>(g, g.d_out, [&](dim3 blocks) {
    gbdt_code::code_product_kernel<S, O, WHERE><<<blocks, dim3(S::NT), 0, s>>>(g);
  });
}

template <typename O, Place WHERE>
int code_tiles(CodeArgs& g, hipStream_t s) {
  if (short_leaves(g)) return launch_code_product<Short<int8_t>, O, WHERE>(g, s);
  if (g.d_out <= 64) return launch_code_product<Shape<int8_t, 128, 64, 4, 1, true>, O, WHERE>(g, s);
  if (long_leaves_of(g, g.d_out, 256)) return launch_code_product<Shape<int8_t, 256, 256, 2, 4, true, true>, O, WHERE>(g, s);
  if (long_leaves_of(g, g.d_out, 128)) return launch_code_product<Shape<int8_t, 256, 128, 4, 2, true, false, 3>, O, WHERE>(g, s);
  return launch_code_product<Shape<int8_t, 128, 128, 2, 2, true, true>, O, WHERE>(g, s);
}

template <typename O, bool LISTED>
int code_few(const CodeArgs& g, int64_t rows, hipStream_t s) {
  if (rows * g.d_out <= 1024) {
    gbdt_code::code_few_kernel<O, 1, LISTED><<<dim3(g.d_out, (unsigned)rows), dim3(64), 0, s>>>(g);
  } else {
    gbdt_code::code_few_kernel<O, 2, LISTED><<<dim3((unsigned)ceil_div(g.d_out, 2), (unsigned)rows), dim3(64), 0, s>>>(g);
  }
  LAUNCHED("code_few_kernel");
  return GBDT_OK;
}

template <typename O>
int leaf_codes(CodeArgs& g, hipStream_t s) {
  // (as few positions as gbdt_leaf_product answers so)
  if (g.n_positions <= 4 || (g.n_positions <= 2048 && (int64_t)g.n_positions * g.d_out <= 16384)) return code_few<O, true>(g, g.n_positions, s);
  return code_tiles<O, Place::kRow>(g, s);
}

template <typename O>
int mixture_codes(CodeArgs& g, int64_t n_rows, hipStream_t s) {
  if (few_rows<int8_t>(n_rows, g.k, g.n_leaves, g.d_in, g.d_out)) return code_few<O, false>(g, n_rows, s);
  const SlotPlan plan = slot_plan(n_rows, g.k, g.n_leaves, g.d_out, gbdt_routed::block_columns<int8_t>, false);
  void* ws = nullptr;
  const int rc = gbdt_internal::workspace(plan.bytes(), s, &ws);
  if (rc != GBDT_OK) return rc;
  CombineArgs<O> to = {};
  to.out = (O*)g.out;
  to.ld_out = g.ld_out;
  const bool direct = g.k == 1;
  return by_slots(g, n_rows, g.d_out, to, plan, (char*)ws, direct,
                  [&](CodeArgs& piece, int64_t r) {
                    piece.x = g.x + r * g.ld_x;
                    piece.row_scales = g.row_scales + r;
                    piece.out = (O*)g.out + r * g.ld_out;
                    return direct ? code_tiles<O, Place::kGatedRow>(piece, s) : code_tiles<O, Place::kSlot>(piece, s);
                  },
                  s);
}

}  // namespace

using namespace gbdt_host;

extern "C" {

int gbdt_route(const void* logits, int64_t ld, const float* choice_bias, int64_t n_rows, int32_t n_leaves, int32_t dtype, int32_t score,
               int32_t n_groups, int32_t groups_kept, int32_t group_best, int32_t k, int32_t renormalise, float scale, int32_t* leaves_out,
               float* gates_out, void* stream) {
  const int rc = route_check(logits, ld, n_rows, n_leaves, dtype, score, k, scale);
  if (n_groups <= 0 || groups_kept <= 0 || groups_kept > n_groups || (group_best != 1 && group_best != 2)) return GBDT_EINVAL;
  if (rc != GBDT_OK) return rc;
  if (n_leaves % n_groups != 0 || (int64_t)k > (int64_t)n_leaves / n_groups * groups_kept) return GBDT_EINVAL;
  if (((uintptr_t)choice_bias & 3) != 0 || ((uintptr_t)leaves_out & 3) != 0 || ((uintptr_t)gates_out & 3) != 0) return GBDT_EINVAL;
  if (n_groups > gbdt_router::kMaxGroups) return GBDT_EUNSUPPORTED;
  if (n_rows == 0) return GBDT_OK;
  if (!logits || !leaves_out || !gates_out) return GBDT_EINVAL;
  RouteArgs g = {};
  g.logits = logits;
  g.bias = choice_bias;
  g.leaves = leaves_out;
  g.gates = gates_out;
  g.ld = ld;
  g.n_rows = (int32_t)n_rows;
  g.n_leaves = n_leaves;
  g.k = k;
  g.n_groups = n_groups;
  g.groups_kept = groups_kept;
  g.group_best = n_groups > 1 ? group_best : 1;
  g.group_size = n_leaves / n_groups;
  g.sigmoid = score == GBDT_SIGMOID;
  g.renormalise = renormalise != 0;
  g.scale = scale;
  hipStream_t s = (hipStream_t)stream;
  return dtype == GBDT_F32 ? route<float>(g, false, s) : route<bf16>(g, false, s);
}

int gbdt_route_grad(const void* logits, int64_t ld, const int32_t* leaves, const float* dgates, int64_t n_rows, int32_t n_leaves,
                    int32_t dtype, int32_t score, int32_t k, int32_t renormalise, float scale, void* dlogits_out, int64_t ld_out,
                    void* stream) {
  const int rc = route_check(logits, ld, n_rows, n_leaves, dtype, score, k, scale);
  if (rc != GBDT_OK) return rc;
  if (ld_out < n_leaves || off_element(dlogits_out, dtype) || ((uintptr_t)leaves & 3) != 0 || ((uintptr_t)dgates & 3) != 0) return GBDT_EINVAL;
  if (ld_out >= kMaxLd) return GBDT_EUNSUPPORTED;
  if (n_rows == 0) return GBDT_OK;
  if (!logits || !leaves || !dgates || !dlogits_out) return GBDT_EINVAL;
  RouteArgs g = {};
  g.logits = logits;
  g.leaves = const_cast<int32_t*>(leaves);
  g.dgates = dgates;
  g.dlogits = dlogits_out;
  g.ld = ld;
  g.ld_out = ld_out;
  g.n_rows = (int32_t)n_rows;
  g.n_leaves = n_leaves;
  g.k = k;
  g.sigmoid = score == GBDT_SIGMOID;
  g.renormalise = renormalise != 0;
  g.scale = scale;
  hipStream_t s = (hipStream_t)stream;
  return dtype == GBDT_F32 ? route<float>(g, true, s) : route<bf16>(g, true, s);
}

size_t gbdt_mixture_workspace_bytes(int64_t n_rows, int32_t k, int32_t n_leaves, int32_t d_in, int32_t d_out, int32_t dtype) {
  if (n_rows < 0 || k <= 0 || n_leaves <= 0 || d_in <= 0 || d_out <= 0 || (dtype != GBDT_F32 && dtype != GBDT_BF16)) return 0;
  if (mixture_check(n_rows, k, n_leaves, d_in, d_out, (const void*)4, (const void*)4, dtype) != GBDT_OK) return 0;
  const int64_t e = dtype == GBDT_F32 ? 4 : 2, units = gbdt_internal::cu_count();
  size_t most = 0;
  const int64_t block = dtype == GBDT_F32 ? 32 : 64;  // (a product of codes takes no more)
  for (int64_t cols : {d_in, d_out}) most = std::max(most, slot_plan(n_rows, k, n_leaves, cols, block, true).bytes());
  for (int64_t inputs : {(int64_t)d_in, 16 / e}) most = std::max(most, weight_plan(n_rows, k, n_leaves, inputs, d_out, e, units).bytes());
  return gbdt_internal::workspace_head_bytes() + most;
}

int gbdt_mixture_product(const void* x, int64_t ld_x, const void* weight, const void* bias, const int32_t* leaves, const float* gates,
                         int64_t n_rows, int32_t k, int32_t n_leaves, int32_t d_in, int32_t d_out, int32_t dtype, void* y_out, int64_t ld_y,
                         void* stream) {
  const int rc = mixture_check(n_rows, k, n_leaves, d_in, d_out, leaves, gates, dtype);
  if (rc != GBDT_OK) return rc;
  if (ld_x < d_in || ld_y < d_out || !weight || off_element(x, dtype) || off_element(weight, dtype) || off_element(bias, dtype) ||
      off_element(y_out, dtype))
    return GBDT_EINVAL;
  if (ld_x >= kMaxLd || ld_y >= kMaxLd) return GBDT_EUNSUPPORTED;
  if (n_rows == 0) return GBDT_OK;
  if (!x || !y_out) return GBDT_EINVAL;
  hipStream_t s = (hipStream_t)stream;
  return dtype == GBDT_F32
             ? mixture_call<float>(x, ld_x, weight, bias, leaves, gates, n_rows, k, n_leaves, d_in, d_out, y_out, ld_y, s)
             : mixture_call<bf16>(x, ld_x, weight, bias, leaves, gates, n_rows, k, n_leaves, d_in, d_out, y_out, ld_y, s);
}

int gbdt_mixture_product_grad(const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, const void* weight, const void* bias,
                              const int32_t* leaves, const float* gates, int64_t n_rows, int32_t k, int32_t n_leaves, int32_t d_in,
                              int32_t d_out, int32_t dtype, void* dx_out, int64_t ld_dx, void* dweight_out, void* dbias_out,
                              float* dgates_out, void* stream) {
  const int rc = mixture_check(n_rows, k, n_leaves, d_in, d_out, leaves, gates, dtype);
  if (rc != GBDT_OK) return rc;
  const bool reads_x = dweight_out || dgates_out, reads_w = dx_out || dgates_out;
  if (ld_dy < d_out || (reads_x && ld_x < d_in) || (dx_out && ld_dx < d_in) || (reads_w && !weight)) return GBDT_EINVAL;
  if (off_element(dy, dtype) || off_element(x, dtype) || off_element(weight, dtype) || off_element(bias, dtype) ||
      off_element(dx_out, dtype) || off_element(dweight_out, dtype) || off_element(dbias_out, dtype) || ((uintptr_t)dgates_out & 3) != 0)
    return GBDT_EINVAL;
  if (ld_dy >= kMaxLd || ld_x >= kMaxLd || ld_dx >= kMaxLd) return GBDT_EUNSUPPORTED;
  if (n_rows > 0 && (!dy || (reads_x && !x))) return GBDT_EINVAL;
  hipStream_t s = (hipStream_t)stream;
  return dtype == GBDT_F32 ? mixture_grad_call<float>(dy, ld_dy, x, ld_x, weight, bias, leaves, gates, n_rows, k, n_leaves, d_in, d_out,
                                                      dx_out, ld_dx, dweight_out, dbias_out, dgates_out, s)
                           : mixture_grad_call<bf16>(dy, ld_dy, x, ld_x, weight, bias, leaves, gates, n_rows, k, n_leaves, d_in, d_out,
                                                     dx_out, ld_dx, dweight_out, dbias_out, dgates_out, s);
}

int gbdt_rows_quantize(const void* x, int64_t ld_x, int64_t n_rows, int32_t n_cols, int32_t dtype, int8_t* codes_out, int64_t ld_codes,
                       float* scales_out, void* stream) {
  if (n_rows < 0 || n_cols <= 0 || ld_x < n_cols || (dtype != GBDT_F32 && dtype != GBDT_BF16)) return GBDT_EINVAL;
  const int64_t padded = round_up(n_cols, 16);
  if (ld_codes < padded || ld_codes % 16 != 0 || ((uintptr_t)codes_out & 15) != 0 || ((uintptr_t)scales_out & 3) != 0 || off_element(x, dtype))
    return GBDT_EINVAL;
  if (n_rows >= kMaxRows || n_cols >= kMaxWidth || ld_x >= kMaxLd || ld_codes >= kMaxLd) return GBDT_EUNSUPPORTED;
  if (n_rows == 0) return GBDT_OK;
  if (!x || !codes_out || !scales_out) return GBDT_EINVAL;
  const gbdt_code::QuantizeArgs g = {x, codes_out, scales_out, ld_x, ld_codes, n_rows, n_cols, (int32_t)padded};
  hipStream_t s = (hipStream_t)stream;
  return dtype == GBDT_F32 ? quantize<float>(g, s) : quantize<bf16>(g, s);
}

int gbdt_leaf_product_codes(const int8_t* codes, int64_t ld_codes, const float* scales, const int8_t* weight, const float* weight_scales,
                         const float* bias, const int32_t* row_idx, const int64_t* leaf_offsets, int64_t n_positions, int32_t n_leaves,
                         int64_t n_rows, int32_t d_in, int32_t d_out, int32_t dtype, void* y_out, int64_t ld_y, void* stream) {
  if (n_positions < 0 || n_leaves <= 0 || n_rows < 0 || d_in <= 0 || d_out <= 0 || !leaf_offsets) return GBDT_EINVAL;
  if (((uintptr_t)leaf_offsets & 7) != 0 || ((uintptr_t)row_idx & 3) != 0) return GBDT_EINVAL;
  if (dtype != GBDT_F32 && dtype != GBDT_BF16) return GBDT_EINVAL;
  if (!row_idx && n_positions > n_rows) return GBDT_EINVAL;
  if (n_positions >= kMaxRows || n_rows >= kMaxRows || n_leaves >= kMaxWidth || d_in >= kMaxWidth || d_out >= kMaxWidth)
    return GBDT_EUNSUPPORTED;
  if (n_rows == 0) n_positions = 0;
  const int rc = code_check(codes, ld_codes, scales, weight, weight_scales, bias, n_positions, d_in, d_out, dtype, y_out, ld_y);
  if (rc != GBDT_OK || n_positions == 0) return rc;
  CodeArgs g = {};
  g.x = codes;
  g.w = weight;
  g.row_idx = row_idx;
  g.offsets = leaf_offsets;
  g.row_scales = scales;
  g.col_scales = weight_scales;
  g.add = bias;
  g.out = y_out;
  g.ld_x = ld_codes;
  g.ld_out = ld_y;
  g.n_positions = (int32_t)n_positions;
  g.n_leaves = n_leaves;
  g.n_rows = (int32_t)n_rows;
  g.d_in = (int32_t)round_up(d_in, 16);
  g.d_out = d_out;
  hipStream_t s = (hipStream_t)stream;
  return dtype == GBDT_F32 ? leaf_codes<float>(g, s) : leaf_codes<bf16>(g, s);
}

int gbdt_mixture_product_codes(const int8_t* codes, int64_t ld_codes, const float* scales, const int8_t* weight, const float* weight_scales,
                            const float* bias, const int32_t* leaves, const float* gates, int64_t n_rows, int32_t k, int32_t n_leaves,
                            int32_t d_in, int32_t d_out, int32_t dtype, void* y_out, int64_t ld_y, void* stream) {
  int rc = mixture_check(n_rows, k, n_leaves, d_in, d_out, leaves, gates, dtype);
  if (rc != GBDT_OK) return rc;
  rc = code_check(codes, ld_codes, scales, weight, weight_scales, bias, n_rows, d_in, d_out, dtype, y_out, ld_y);
  if (rc != GBDT_OK || n_rows == 0) return rc;
  CodeArgs g = {};
  g.x = codes;
  g.w = weight;
  g.leaves = leaves;
  g.gates = gates;
  g.row_scales = scales;
  g.col_scales = weight_scales;
  g.add = bias;
  g.out = y_out;
  g.ld_x = ld_codes;
  g.ld_out = ld_y;
  g.n_leaves = n_leaves;
  g.d_in = (int32_t)round_up(d_in, 16);
  g.d_out = d_out;
  g.k = k;
  hipStream_t s = (hipStream_t)stream;
  return dtype == GBDT_F32 ? mixture_codes<float>(g, n_rows, s) : mixture_codes<bf16>(g, n_rows, s);
}

}  // extern "C"
