// Products grouped by leaf: y[d] = W_l x[d] + b_l for the rows d of leaf l, and its gradients.
//
// Positions p of the row list are grouped by leaf: leaf l holds offsets[l] <= p < offsets[l + 1], p's row is row_idx[p].
// offsets are read on the device, so nothing waits for the host between routing rows and using them; the host knows only
// the number of positions and of leaves.  Tiles of BM positions never cross a leaf: leaf l owns the tiles from
// T(l) = offsets[l] / BM + l on.  T rises by at least the number of tiles that the leaf needs, because
// ceil((b - a) / BM) <= floor(b / BM) - floor(a / BM) + 1, so positions / BM + leaves workgroups hold every tile whatever the
// lengths are, no sum over the leaves before a leaf is needed, and a tile finds its leaf by a search over T.
#pragma once

#include <type_traits>

#include "tile_product.h"

namespace gbdt_leaf {

using namespace gbdt_tile;

template <typename T>
struct LeafArgs {
  const T* x;         // [n_rows][d_in]
  const T* dy;        // [n_rows][d_out]
  const T* w;         // [n_leaves][d_out][d_in]
  const T* bias;      // [n_leaves][d_out] or null
  T* y;               // [n_rows][d_out]
  T* dx;              // [n_rows][d_in]
  T* dw;              // [n_leaves][d_out][d_in] or null
  T* dbias;           // [n_leaves][d_out] or null
  float* partial;     // 2 slots a cut of the position axis, of (d_in + 1) * d_out sums each
  const int32_t* row_idx;  // or null: row = position
  const int64_t* offsets;  // [n_leaves + 1]
  int64_t ld_x, ld_dy, ld_y, ld_dx;
  int32_t n_positions, n_leaves, n_rows, d_in, d_out;
  int32_t cut;        // gradient of the weights: positions between cuts
  uint32_t col_tiles, row_tiles, cols_per;  // cols_per: column tiles that a workgroup goes through
  int32_t row_first;  // gradient of the weights from listed rows: the output that dy's first column belongs to
  uint32_t first;     // of this launch's workgroups (gradient of the weights: of its pieces), among all of the call
};

// An offset as the kernels take it: inside the list, whatever the array holds.
__device__ __forceinline__ int offset_at(const int64_t* offsets, int l, int n_positions) {
  const int64_t o = offsets[l];
  return o < 0 ? 0 : o > n_positions ? n_positions : (int)o;
}

// The largest leaf l with T(l) = offset(l) / unit + l <= tile (unit 0: with offset(l) <= tile), by 64 probes at a time; -1 if
// there is none.
__device__ __forceinline__ int find_leaf(const int64_t* offsets, int n_leaves, int n_positions, int unit, int tile) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n_leaves;
  bool any = false;
  while (hi - lo > 1 || !any) {
    const int step = (hi - lo + 63) / 64;
    const int i = lo + lane * step;
    bool ok = i < hi;
    if (ok) {
      const int o = offset_at(offsets, i, n_positions);
      ok = (unit ? o / unit + i : o) <= tile;
    }
    const int n = __popcll(__ballot(ok));
    if (n == 0) return -1;
    any = true;
    lo += (n - 1) * step;
    hi = lo + step < hi ? lo + step : hi;
  }
  return lo;
}

// Row r >= 0: one 32 x 32 -> 64 bit product and sum (distances of rows are below 2^30 bytes).
template <typename T>
__device__ __forceinline__ const T* row_of(const T* base, int r, int64_t ld) {
  return (const T*)((const char*)base + (uint64_t)(uint32_t)r * (uint32_t)(ld * (int64_t)sizeof(T)));
}

// Rows of a matrix by position in the list; `end` is the matrix's, one past its last value.
template <typename T>
struct ListRows {
  static constexpr bool kEven = false;  // not a constant distance apart
  const T* base;
  const T* end;
  int64_t ld;
  const int32_t* row_idx;
  int32_t stop, n_rows;
  __device__ __forceinline__ int fetch(int p) const { return p < stop ? (row_idx ? row_idx[p] : p) : -1; }
  __device__ __forceinline__ const T* at(int, int d) const {
    return (uint32_t)d < (uint32_t)n_rows ? row_of(base, d, ld) : nullptr;
  }
};
template <typename T>
__device__ __forceinline__ ListRows<T> list_rows(const T* base, int64_t ld, int cols, const LeafArgs<T>& g, int stop) {
  return {base, base + (int64_t)(g.n_rows - 1) * ld + cols, ld, g.row_idx, stop, g.n_rows};
}

// The same from a copy of a part of the list in local memory, -1 where there is no row.  EACH: so many k stand for a position.
template <typename T, int EACH = 1>
struct CopiedRows {
  static constexpr bool kEven = false;
  const T* base;
  const T* end;
  int64_t ld;
  const __attribute__((address_space(3))) int* ids;  // (said outright: a flat load would be waited for with all others)
  int32_t first;  // the position of ids[0]
  __device__ __forceinline__ int fetch(int k) const { return ids[k / EACH - first]; }
  __device__ __forceinline__ const T* at(int, int d) const { return d >= 0 ? row_of(base, d, ld) : nullptr; }
};

// Rows of a matrix in order.
template <typename T>
struct PlainRows {
  static constexpr bool kEven = true;
  const T* base;
  const T* end;
  int64_t ld;
  int32_t n;
  __device__ __forceinline__ int fetch(int) const { return 0; }
  __device__ __forceinline__ const T* at(int r, int) const { return r < n ? row_of(base, r, ld) : nullptr; }
};
template <typename T>
__device__ __forceinline__ PlainRows<T> plain_rows(const T* base, int64_t ld, int n, int cols) {
  return {base, base + (int64_t)(n - 1) * ld + cols, ld, n};
}

// Where the results of a product over rows go: value + the leaf's bias, to the row of y that the position names.
template <typename T>
struct ToRows {
  typedef T Out;
  static constexpr bool kScaled = false, kFinished = false, kDots = false;
  const T* bias;  // [n_leaves][cols] or null
  T* out;
  int64_t ld;
  // The place of position p's results, -1 for none.
  __device__ __forceinline__ int place(const LeafArgs<T>& g, int p) const {
    const int d = g.row_idx ? g.row_idx[p] : p;
    return (uint32_t)d < (uint32_t)g.n_rows ? d : -1;
  }
  __device__ __forceinline__ float add(int64_t column) const { return bias ? (float)bias[column] : 0.0f; }
};

// Where a row of a tile goes, and what it is multiplied by (To::kScaled) or which row it is (To::kDots).
struct RowPlace {
  int id;  // -1 for none
  union {
    float factor;
    int row;
  };
};
template <class G, class To>
__device__ __forceinline__ RowPlace place_of(const G& g, const To& to, int p, int end) {
  static_assert(!(To::kScaled && To::kDots), "");
  RowPlace r;
  r.id = p < end ? to.place(g, p) : -1;
  r.row = 0;
  if constexpr (To::kScaled) r.factor = r.id >= 0 ? to.row_scale(g, p) : 0.0f;
  if constexpr (To::kDots) r.row = r.id >= 0 ? g.row_idx[p] : 0;
  return r;
}

// Those of a lane's rows of its blocks, kept in registers.
template <class S>
struct Places {
  RowPlace at[S::TM];
  template <class G, class To>
  __device__ __forceinline__ void fetch(const G& g, const To& to, int p0, int end) {
    const int m0 = p0 + (thread_of<S::NT>() >> 6) / S::WN * (S::TM * 16) + (threadIdx.x & 15);
#pragma unroll
    for (int i = 0; i < S::TM; ++i) at[i] = place_of(g, to, m0 + 16 * i, end);
  }
  __device__ __forceinline__ RowPlace operator()(int i) const { return at[i]; }
};

// Of a whole tile, kept in local memory.
template <class S>
struct TilePlaces {
  const RowPlace* of;  // [BM]
  __device__ __forceinline__ RowPlace operator()(int i) const {
    return of[(thread_of<S::NT>() >> 6) / S::WN * (S::TM * 16) + (threadIdx.x & 15) + 16 * i];
  }
};

// sum a b + add for scales a and b: times the smaller first, which neither overflows nor underflows (scales are 0 or normal numbers, a sum is
// 0 or at least 1) unless the product of all three does.
__device__ __forceinline__ float scaled(float sum, float a, float b, float add) {
  const bool first = fabsf(a) < fabsf(b);  // (a NaN is one of the two either way)
  return __builtin_fmaf(sum * (first ? a : b), first ? b : a, add);
}

// A tile's results to their rows, through the last stage.
template <class S, class G, class To, class Where>
__device__ __forceinline__ void store_rows(char* lds, const G& g, const To& to, typename S::Acc (&acc)[S::TM][S::TN], const Where& places,
                                           int leaf, int col, int cols) {
  typedef typename S::Acc Acc;
  const int w = thread_of<S::NT>() >> 6;
  const int l = threadIdx.x & 63, wave_col = col + w % S::WN * (S::TN * 16);
  f32x4 add[S::TN], scale[To::kScaled ? S::TN : 1];
#pragma unroll
  for (int j = 0; j < S::TN; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int n = wave_col + 16 * j + 4 * (l >> 4) + r;
      add[j][r] = n < cols ? to.add((int64_t)leaf * cols + n) : 0.0f;
      if constexpr (To::kScaled) scale[j][r] = n < cols ? to.column_scale((int64_t)leaf * cols + n) : 0.0f;
    }
  auto value = [&](int i, int j) {
    if constexpr (To::kScaled) {
      f32x4 v;
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = scaled((float)acc[i][j][r], places(i).factor, scale[j][r], add[j][r]);
      return v;
    } else {
      return acc[i][j] + add[j];
    }
  };
  if constexpr (To::kFinished) {
    constexpr int at_once = To::kDots ? 2 : 1;  // rows whose x is on its way together
#pragma unroll
    for (int i0 = 0; i0 < S::TM; i0 += at_once) {
      typename To::Beside x[at_once][S::TN];
      if constexpr (To::kDots) {
#pragma unroll
        for (int i = 0; i < at_once; ++i) to.template beside<S::TN>(g, places(i0 + i).row, wave_col, cols, x[i]);
      }
#pragma unroll
      for (int i = 0; i < at_once; ++i) {
        f32x4 v[S::TN];
#pragma unroll
        for (int j = 0; j < S::TN; ++j) v[j] = value(i0 + i, j);
        to.template finish<S::TN>(g, places(i0 + i).id, wave_col, cols, x[i], v);
#pragma unroll
        for (int j = 0; j < S::TN; ++j) acc[i0 + i][j] = __builtin_bit_cast(Acc, v[j]);
      }
    }
  }
  store_tile<S, typename To::Out, S::TM, S::TN>(
      lds + S::kLastStage,
      [&](int i, int j) {
        if constexpr (To::kFinished) {
          return __builtin_bit_cast(f32x4, acc[i][j]);
        } else {
          return value(i, j);
        }
      },
      [&](int i, int r) {
        const int d = __shfl(places(i).id, r);
        return d >= 0 && to.out != nullptr ? to.out + (int64_t)d * to.ld : (typename To::Out*)nullptr;
      },
      wave_col, cols);
}

// The rows of one tile of positions times a matrix of the leaf, g.cols_per column tiles one after another; the next one's
// first steps are on their way while one's values are stored.  B: the matrix' orientation, k its length along k.
// To::kScaled: values are multiplied by a factor of their position and one of the leaf's column.
// To::kFinished: a row's values of this wavefront's columns go through to.finish before they are stored; To::kDots: beside what
// to.beside reads of the position's row.
// GROUPS > 1: as many times the tile's threads take a part of k each, all of as many steps, and the first adds up; one column
// tile a workgroup then, since the other groups leave after it.
template <class S, class B, int GROUPS, typename T, class G, class To>
__device__ __forceinline__ void leaf_rows_product(char* lds, const G& g, const T* in, int64_t ld_in, int k, const To& to, int cols) {
  typedef typename S::Acc Acc;
  const uint32_t t = g.first + xcd_tile(blockIdx.x, gridDim.x);
  const uint32_t turns = (g.col_tiles + g.cols_per - 1) / g.cols_per;
  const int tile = (int)(t / turns), col_first = (int)(t % turns * g.cols_per) * S::BN;
  const int leaf = find_leaf(g.offsets, g.n_leaves, g.n_positions, S::BM, tile);
  if (leaf < 0) return;
  const int begin = offset_at(g.offsets, leaf, g.n_positions), end = offset_at(g.offsets, leaf + 1, g.n_positions);
  const int p0 = begin + (tile - (begin / S::BM + leaf)) * S::BM;
  if (p0 >= end || p0 < begin) return;
  const int col_last = cols < col_first + (int)g.cols_per * S::BN ? cols : col_first + (int)g.cols_per * S::BN;
  const ListRows<T> rows_a = list_rows(in, ld_in, k, g, end);
  const PlainRows<T> rows_b = plain_rows(g.w + (int64_t)leaf * g.d_out * g.d_in, g.d_in, g.d_out, g.d_in);
  Places<S> places;
  places.fetch(g, to, p0, end);
  const int group = GROUPS > 1 ? (int)threadIdx.x / S::NT : 0;
  lds += group * S::kLdsBytes;
  const int part = GROUPS > 1 ? ((k + GROUPS - 1) / GROUPS + S::kStep - 1) / S::kStep * S::kStep : k;
  const int k0 = group * part, k1 = k < k0 + part ? k : k0 + part;  // (steps past the end are zeros)
  typename S::RowsA a;
  B b;
  auto begin_columns = [&](int col) {
    a.init(rows_a, p0, 0, k0, k1);
    b.init(rows_b, col, cols, k0, k1);
    tile_begin<S>(lds, a, b, rows_a, rows_b, k0, k0 + part);
  };
  begin_columns(col_first);
  for (int col = col_first; col < col_last; col += S::BN) {
    Acc acc[S::TM][S::TN];
    zeros<S>(acc);
    tile_run<S, true>(lds, a, b, rows_a, rows_b, k0, k0 + part, acc, Nothing{});
    if constexpr (GROUPS > 1) {
      constexpr int values = S::TM * S::TN;
      static_assert(values * S::NT * 16 <= S::kLdsBytes, "a group's sums take its stages' place");
      Acc* sums = (Acc*)lds;
      __syncthreads();  // (the last reads of the stages)
#pragma unroll
      for (int v = 0; v < values; ++v) sums[v * S::NT + thread_of<S::NT>()] = acc[v / S::TN][v % S::TN];
      __syncthreads();
      if (group > 0) return;
#pragma unroll
      for (int other = 1; other < GROUPS; ++other)
#pragma unroll
        for (int v = 0; v < values; ++v)
          acc[v / S::TN][v % S::TN] += ((const Acc*)(lds + other * S::kLdsBytes))[v * S::NT + thread_of<S::NT>()];
    } else if (col + S::BN < col_last) {
      begin_columns(col + S::BN);
    }
    store_rows<S>(lds, g, to, acc, places, leaf, col, cols);
  }
}

// The same by workgroups that stay: as many as there are places for, each goes through tiles of rows and columns, and the next
// one's ids are on their way while one is multiplied, its first steps while one's values are stored.  (Where a compute unit holds one
// workgroup, nothing else hides a tile's beginning and end.)  The tiles of an XCD are neighbours.  first: room for the leaves' first tiles
// and positions, and for rows' places.
constexpr int kStayLeaves = 1024;
template <class S>
struct StayTable {
  int tile[kStayLeaves + 1], begin[kStayLeaves + 1];
  RowPlace rows[3][S::BM];  // of three tiles in turn: what is written while one is multiplied is read no more by a wavefront behind
};
template <class S, class B, typename T, class G, class To>
__device__ __forceinline__ void leaf_rows_stay(char* lds, StayTable<S>& first, const G& g, const T* in, int64_t ld_in, int k, const To& to, int cols) {
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x;
    int least = 0, base = 0;  // (offsets that decrease are taken as the largest before them)
    for (int l0 = 0; l0 <= g.n_leaves; l0 += 64) {
      const int l = l0 + lane;
      int begin = offset_at(g.offsets, l < g.n_leaves ? l : g.n_leaves, g.n_positions);
      begin = begin > least ? begin : least;
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) {
        const int other = __shfl_up(begin, m);
        if (lane >= m && other > begin) begin = other;
      }
      if (l <= g.n_leaves) first.begin[l] = begin;
      least = __shfl(begin, 63);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (int l0 = 0; l0 <= g.n_leaves; l0 += 64) {
      const int l = l0 + lane;
      const int n = l < g.n_leaves ? (first.begin[l + 1] - first.begin[l] + S::BM - 1) / S::BM : 0;
      int sum = n;
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) {
        const int other = __shfl_up(sum, m);
        if (lane >= m) sum += other;
      }
      if (l <= g.n_leaves) first.tile[l] = base + sum - n;
      base += __shfl(sum, 63);
    }
  }
  __syncthreads();
  const int64_t tiles = (int64_t)first.tile[g.n_leaves] * g.col_tiles;
  const int xcd = blockIdx.x % 8;
  const int64_t last = tiles * (xcd + 1) / 8, step = gridDim.x / 8;
  int64_t t = tiles * xcd / 8 + blockIdx.x / 8;
  struct At {
    int leaf, p0, end, col;
  };
  auto locate = [&](int64_t tile) {
    const int row_tile = (int)((uint32_t)tile / g.col_tiles);  // (fewer than 2^31)
    int lo = 0, hi = g.n_leaves;  // the last leaf whose first tile is no later (leaves without rows have the next one's)
    while (hi - lo > 1) {
      const int stride = (hi - lo + 63) / 64, i = lo + (int)(threadIdx.x & 63) * stride;
      const int n = __popcll(__ballot(i < hi && first.tile[i] <= row_tile));
      lo += (n - 1) * stride;
      hi = lo + stride < hi ? lo + stride : hi;
    }
    At at;
    at.leaf = __builtin_amdgcn_readfirstlane(lo);
    at.p0 = first.begin[at.leaf] + (row_tile - first.tile[at.leaf]) * S::BM;
    at.end = first.begin[at.leaf + 1];
    at.col = (int)((uint32_t)tile - (uint32_t)row_tile * g.col_tiles) * S::BN;
    return at;
  };
  typename S::RowsA a;
  B b;
  typename S::RowsA::Ids ids;
  auto fetch = [&](const At& at, int turn) {
    S::RowsA::fetch(list_rows(in, ld_in, k, g, at.end), at.p0, ids);
    if ((int)threadIdx.x < S::BM) first.rows[turn][threadIdx.x] = place_of(g, to, at.p0 + (int)threadIdx.x, at.end);
  };
  auto rows_a = [&](const At& at) { return list_rows(in, ld_in, k, g, at.end); };
  auto rows_b = [&](const At& at) { return plain_rows(g.w + (int64_t)at.leaf * g.d_out * g.d_in, g.d_in, g.d_out, g.d_in); };
  auto begin = [&](const At& at) {
    a.init(rows_a(at), at.p0, 0, 0, k, ids);
    b.init(rows_b(at), at.col, cols, 0, k);
    tile_begin<S>(lds, a, b, rows_a(at), rows_b(at), 0, k);
  };
  if (t >= last) return;
  static_assert(S::NT >= S::BM, "a thread a row");
  At at = locate(t);
  fetch(at, 0);
  begin(at);
  for (int turn = 0;;) {
    t += step;
    const bool more = t < last;
    At next = at;
    const int next_turn = turn == 2 ? 0 : turn + 1;
    if (more) {
      next = locate(t);
      fetch(next, next_turn);
    }
    typename S::Acc acc[S::TM][S::TN];
    zeros<S>(acc);
    tile_run<S, true>(lds, a, b, rows_a(at), rows_b(at), 0, k, acc, Nothing{});
    if (more) begin(next);
    store_rows<S>(lds, g, to, acc, TilePlaces<S>{first.rows[turn]}, at.leaf, at.col, cols);
    if (!more) return;
    at = next;
    turn = next_turn;
  }
}

// By workgroups that stay, in tiles so large that a compute unit holds one; by others in smaller ones.
template <class S>
constexpr bool kStays = S::BM >= 256;
template <class S, class B, typename T, class G, class To>
__device__ __forceinline__ void rows_product(char* lds, const G& g, const T* in, int64_t ld_in, int k, const To& to, int cols) {
  if constexpr (kStays<S>) {
    __shared__ StayTable<S> first;
    leaf_rows_stay<S, B>(lds, first, g, in, ld_in, k, to, cols);
  } else {
    leaf_rows_product<S, B, 1>(lds, g, in, ld_in, k, to, cols);
  }
}

// y: rows of x times the leaf's rows of w, both with k = input along memory.  Bound by reading x once: d_out products a value
// are fewer than the matrix cores do in the time of its read.  Hence tiles that hold all outputs where they can, and as many
// bytes on the way as local memory holds.  (400,000 x 2,000 -> 128 in 255 leaves, bf16: 466 us, 3.9 TB/s; 10,000 x 28 -> 1, f32:
// 5.4 us, a chain of the search for the leaf, a row's id, its values, the store.)
template <class S>
__global__ void __launch_bounds__(S::NT, 2) leaf_product_kernel(const LeafArgs<typename S::T> g) {
  __shared__ __align__(16) char lds[S::kLdsBytes];
  leaf_rows_product<S, typename S::RowsB, 1>(lds, g, g.x, g.ld_x, g.d_in, ToRows<typename S::T>{g.bias, g.y, g.ld_y}, g.d_out);
}

// The same where there are too few tiles for the compute units: a tile's k is split among GROUPS times the threads.
template <class S, int GROUPS>
__global__ void __launch_bounds__(S::NT* GROUPS) leaf_product_split_kernel(const LeafArgs<typename S::T> g) {
  __shared__ __align__(16) char lds[S::kLdsBytes * GROUPS];
  leaf_rows_product<S, typename S::RowsB, GROUPS>(lds, g, g.x, g.ld_x, g.d_in, ToRows<typename S::T>{g.bias, g.y, g.ld_y}, g.d_out);
}

// dx: rows of dy (k = output along memory) times w, whose rows are k.  Bound by its stores, d_in values a row, which a tile's
// short sum (d_out) leaves little time to hide: the next columns' first steps fly beneath them.  (100,000 x 256 -> 2,000 in 255
// leaves, bf16: 290 us, 2.5 TB/s with the matrices read once; 50,021 x 33 -> 137 in 63, f32, rows of no whole chunks: 26 us.)
template <class S>
__global__ void __launch_bounds__(S::NT, 2) leaf_grad_input_kernel(const LeafArgs<typename S::T> g) {
  __shared__ __align__(16) char lds[S::kLdsBytes];
  leaf_rows_product<S, typename S::ColumnsB, 1>(lds, g, g.dy, g.ld_dy, g.d_out, ToRows<typename S::T>{nullptr, g.dx, g.ld_dx}, g.d_in);
}

// A few positions (a row or a few answered at once): a wavefront takes OUTPUTS outputs of one position, each lane a chunk of k
// of every 64, and adds up across the lanes.  There is nothing to share between rows, so the leaf's matrix is read once a
// position, by as many compute units as there are outputs; a tile of 128 rows on the matrix cores reads it by two workgroups.
// The end of a row that is no whole chunk is read as the last whole chunk, whose values before it count for nothing.
// Bound by a chain of four round trips (offsets, row id, values, store) for a row, by re-reading matrices from L2 for many: 700
// -> 256 bf16, 255 leaves: 4.0 us for a row, 7.3 for 64.
template <typename T, int OUTPUTS>
__global__ void __launch_bounds__(64) leaf_product_few_kernel(const LeafArgs<T> g) {
  const int p = (int)blockIdx.y, o0 = (int)blockIdx.x * OUTPUTS, l = threadIdx.x;
  const int d = g.row_idx ? g.row_idx[p] : p;
  // the last leaf that begins at or before p
  const int leaf = find_leaf(g.offsets, g.n_leaves, g.n_positions, 0, p);
  if (leaf < 0 || (uint32_t)d >= (uint32_t)g.n_rows || p >= offset_at(g.offsets, leaf + 1, g.n_positions)) return;
  const T* x = row_of(g.x, d, g.ld_x);
  const T* w = g.w + ((int64_t)leaf * g.d_out + o0) * g.d_in;
  constexpr int n = kChunk<T>;
  float sum[OUTPUTS];
#pragma unroll
  for (int i = 0; i < OUTPUTS; ++i) sum[i] = 0.0f;
  if (g.d_in >= n) {
#pragma unroll 2
    for (int k = l * n; k < g.d_in; k += 64 * n) {
      const int at = k + n <= g.d_in ? k : g.d_in - n, skip = k - at;
      const u32x4 xc = load16(x + at);
      u32x4 wc[OUTPUTS];
#pragma unroll
      for (int i = 0; i < OUTPUTS; ++i) wc[i] = load16(w + (o0 + i < g.d_out ? (int64_t)i * g.d_in : 0) + at);
      T xv[n], wv[n];
      __builtin_memcpy(xv, &xc, 16);
#pragma unroll
      for (int i = 0; i < OUTPUTS; ++i) {
        __builtin_memcpy(wv, &wc[i], 16);
#pragma unroll
        for (int e = 0; e < n; ++e) sum[i] = e >= skip ? __builtin_fmaf((float)xv[e], (float)wv[e], sum[i]) : sum[i];
      }
    }
  } else if (l < g.d_in) {
#pragma unroll
    for (int i = 0; i < OUTPUTS; ++i)
      if (o0 + i < g.d_out) sum[i] = (float)x[l] * (float)w[(int64_t)i * g.d_in + l];
  }
#pragma unroll
  for (int i = 0; i < OUTPUTS; ++i) {
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) sum[i] += __shfl_xor(sum[i], s);
  }
  if (l != 0) return;
#pragma unroll
  for (int i = 0; i < OUTPUTS; ++i) {
    const int o = o0 + i;
    if (o < g.d_out) g.y[(int64_t)d * g.ld_y + o] = (T)(g.bias ? sum[i] + (float)g.bias[(int64_t)leaf * g.d_out + o] : sum[i]);
  }
}

// Sums over k of operand a's rows: every lane those of its values, of its row of each block.  (One register a block; a product
// with ones takes four.)
template <class S>
struct RowSums {
  float (&sum)[S::TM];
  bool on;
  template <class F>
  __device__ __forceinline__ void operator()(int i, const F& rows) const {
    if (!on) return;
    float s = (float)rows[0];
#pragma unroll
    for (int k = 1; k < kChunk<typename S::T>; ++k) s += (float)rows[k];
    sum[i] += s;
  }
};

// dW_l and db_l: both operands' rows are k = the leaf's positions.  The position axis is cut at multiples of g.cut, so that
// one long leaf is the work of many workgroups: a piece is what a leaf has between two cuts, and leaf l owns the pieces from
// offsets[l] / cut + l on (as above).  A leaf of one piece writes its result; the pieces of others leave f32 sums in slots: of
// the pieces between two cuts only the first can have begun before (slot 2 b) and only the last can end behind (2 b + 1).
// leaf_grad_join_kernel adds a leaf's slots in order, so the sums do not depend on which workgroup ran first.
// Bound by the rows' loads, which no tile shares with another leaf's, and by what short and unequal leaves leave unused:
// 100,000 x 2,000 x 256 in 255 leaves, bf16: 343 us, 2.1 TB/s, 300 TFLOP/s; 50,021 x 137 x 33 in 63, f32: 30 us.
// The list's ids are copied to local memory first, kCopiedIds at a time: loads are waited for in order, so a row's address that
// waits for an id on its way from memory waits for all chunks asked for before as well, and steps do not overlap.
// LONG: pieces may be longer than that.  (The loop over copies takes 38 registers more, and spills them without whole chunks.)
constexpr int kCopiedIds = 4096;
constexpr int kShortPiece = 1024;  // positions
static_assert(kShortPiece <= kCopiedIds, "a piece of several column tiles a workgroup is copied at once");

struct Piece {
  int leaf, p0, p1;  // leaf < 0: none
  bool whole;        // all of its leaf
  int64_t slot;      // of its sums, if not
};
// FROM_LEAF: pieces are cut from their leaf's first position on, so that a leaf no longer than a cut is whole: where leaves are many
// that is most of them, and no sums are left behind.  Slots then go by the block of positions that a piece begins in: of those that
// begin in one, at most one is its leaf's last (slot 2 b) and one is not (2 b + 1), since that one is a whole cut long.
template <bool FROM_LEAF, typename T>
__device__ __forceinline__ Piece find_piece(const LeafArgs<T>& g, int piece) {
  Piece r = {-1, 0, 0, false, 0};
  const int leaf = find_leaf(g.offsets, g.n_leaves, g.n_positions, g.cut, piece);
  if (leaf < 0) return r;
  const int begin = offset_at(g.offsets, leaf, g.n_positions), end = offset_at(g.offsets, leaf + 1, g.n_positions);
  if constexpr (FROM_LEAF) {
    const int first = begin / g.cut, nth = piece - (first + leaf);
    const int64_t p0 = (int64_t)begin + (int64_t)nth * g.cut;
    if (p0 >= end && nth > 0) return r;  // an empty leaf has one piece: zeros
    r.leaf = leaf;
    r.p0 = (int)(p0 < end ? p0 : end);
    r.p1 = p0 + g.cut < end ? (int)p0 + g.cut : end;
    r.whole = end - begin <= g.cut;
    r.slot = 2 * (p0 / g.cut) + (r.p1 == end ? 0 : 1);
    return r;
  }
  const int64_t block = piece - leaf;
  const int64_t b0 = block * g.cut, b1 = b0 + g.cut;
  r.p0 = begin > b0 ? begin : (int)(b0 < end ? b0 : end);
  r.p1 = end < b1 ? end : (int)b1;
  if (r.p0 >= r.p1 && (end > begin || block != begin / g.cut)) return r;  // only an empty leaf's one piece is empty: zeros
  r.leaf = leaf;
  r.whole = begin >= b0 && end <= b1;
  r.slot = 2 * block + (begin < b0 ? 0 : 1);
  return r;
}

// LISTED: dy holds a row for every position, in the list's order, of ld_dy values from output row_first on, zeros behind the outputs; of
// 16-bit values two one after the other, whose sum is meant, and dW alone.  (k then counts rows of dy, from the copied list's first on.)
template <typename T, bool LISTED>
constexpr int kRowsEach = LISTED && sizeof(T) == 2 ? 2 : 1;
template <class S, bool LONG, bool LISTED>
__global__ void __launch_bounds__(S::NT, 2) leaf_grad_weight_kernel(const LeafArgs<typename S::T> g) {
  typedef typename S::T T;
  __shared__ __align__(16) char lds[S::kLdsBytes];
  __shared__ int ids[kCopiedIds];
  // A piece's workgroups share its rows and so are one XCD's; pieces, which are of any length, go round.  LISTED: leaves that are whole
  // are of more unequal length than cuts make pieces, and each is all XCDs' work, a part of the columns each (with one row of dy a position, 8,192
  // rows x 4 leaves, 1,024 x 1,024 x 64: 148 us against 171), or of the outputs where dy has two (30,000 rows, one of 8 leaves, 1,024 ->
  // 512, lists and weighted rows included: 131 us against 147 by columns).
  const uint32_t tiles = g.col_tiles * g.row_tiles, at = blockIdx.x / 8;
  const int piece = (int)(g.first + (LISTED ? blockIdx.x / tiles : at / tiles * 8 + blockIdx.x % 8));
  const int r = (int)(LISTED ? blockIdx.x % tiles : at % tiles);
  const Piece at_piece = find_piece<LISTED>(g, piece);
  const int leaf = at_piece.leaf, p0 = at_piece.p0, p1 = at_piece.p1;
  if (leaf < 0) return;
  // A short piece's column tiles are gone through cols_per at a time, one after another, by the first of its workgroups; the
  // others leave.  (Not by every cols_per'th: workgroups go to an XCD's shader engines in turn as well.)
  const int cols_per = p1 - p0 <= kShortPiece ? (int)g.cols_per : 1;
  const int turns = ((int)g.col_tiles + cols_per - 1) / cols_per;
  if (r >= turns * (int)g.row_tiles) return;
  constexpr int each = kRowsEach<T, LISTED>;
  const int row_tile = each == 2 ? r % (int)g.row_tiles : r / turns, turn = each == 2 ? r / (int)g.row_tiles : r % turns;
  const int row0 = (LISTED ? g.row_first : 0) + row_tile * S::BM, col_first = turn * cols_per * S::BN;
  const bool whole = at_piece.whole;
  float* part = g.partial + at_piece.slot * ((int64_t)(g.d_in + 1) * g.d_out);
  const int all_cols = g.dw ? g.d_in : 1;  // (the outputs' sums alone come with the first tile)
  const int col_last = all_cols < col_first + cols_per * S::BN ? all_cols : col_first + cols_per * S::BN;
  const int w = threadIdx.x >> 6, l = threadIdx.x & 63;
  const int m0 = row0 + (w / S::WN) * (S::TM * 16);

  const auto listed = (const __attribute__((address_space(3))) int*)ids;
  typedef typename std::conditional<LISTED, PlainRows<T>, CopiedRows<T>>::type RowsOfDy;
  RowsOfDy rows_a;
  if constexpr (!LISTED) {
    rows_a = {g.dy, g.dy + (int64_t)(g.n_rows - 1) * g.ld_dy + g.d_out, g.ld_dy, listed, p0};
  }
  const int dy_cols = LISTED ? g.row_first + (int)g.ld_dy : g.d_out;
  CopiedRows<T, each> rows_b = {g.x, g.x + (int64_t)(g.n_rows - 1) * g.ld_x + g.d_in, g.ld_x, listed, p0};
  typename S::ColumnsA a;
  typename S::ColumnsB b;
  int c0 = p0, c1 = p0;  // the positions copied
  auto copy_ids = [&](int from) {
    c0 = from;
    c1 = !LONG || p1 - from < kCopiedIds ? p1 : from + kCopiedIds;
    rows_b.first = LISTED ? 0 : from;
    if constexpr (LISTED) {
      rows_a = plain_rows(g.dy + (int64_t)from * each * g.ld_dy - g.row_first, g.ld_dy, each * (c1 - from), dy_cols);
    } else {
      rows_a.first = from;
    }
    for (int p = c0 + (int)threadIdx.x; p < c1; p += S::NT) {
      const int d = g.row_idx ? g.row_idx[p] : p;
      ids[p - c0] = (uint32_t)d < (uint32_t)g.n_rows ? d : -1;
    }
    __syncthreads();
  };
  auto k0 = [&] { return LISTED ? 0 : c0; };
  auto k1 = [&] { return LISTED ? each * (c1 - c0) : c1; };
  auto begin_columns = [&](int col) {
    a.init(rows_a, row0, dy_cols, k0(), k1());
    b.init(rows_b, col, g.d_in, k0(), k1());
    tile_begin<S>(lds, a, b, rows_a, rows_b, k0(), k1());
  };
  copy_ids(p0);
  begin_columns(col_first);
  for (int col = col_first; col < col_last; col += S::BN) {
    f32x4 acc[S::TM][S::TN];
    zeros<S>(acc);
    float sum[S::TM];
#pragma unroll
    for (int i = 0; i < S::TM; ++i) sum[i] = 0.0f;
    const bool sums = (!LISTED || sizeof(T) == 4) && __builtin_amdgcn_readfirstlane(g.dbias != nullptr && col == 0 && w % S::WN == 0);
    for (;;) {
      tile_run<S, true>(lds, a, b, rows_a, rows_b, k0(), k1(), acc, RowSums<S>{sum, sums});
      if (!LONG || c1 >= p1) break;
      __syncthreads();  // everyone has read the last of these ids
      copy_ids(c1);
      begin_columns(col);
    }
    if (col + S::BN < col_last) begin_columns(col + S::BN);
    const int wave_col = col + (w % S::WN) * (S::TN * 16);
    if (g.dw && whole) {
      store_tile<S, T, S::TM, S::TN>(
          lds + S::kLastStage, [&](int i, int j) { return acc[i][j]; },
          [&](int i, int r) {
            const int o = m0 + 16 * i + r;
            return o < g.d_out ? g.dw + ((int64_t)leaf * g.d_out + o) * g.d_in : (T*)nullptr;
          },
          wave_col, g.d_in);
    } else if (g.dw) {
#pragma unroll
      for (int i = 0; i < S::TM; ++i) {
        const int o = m0 + 16 * i + (l & 15);
#pragma unroll
        for (int j = 0; j < S::TN; ++j) {
          const int n = wave_col + 16 * j + 4 * (l >> 4);
          if (o < g.d_out && n < g.d_in) store4(part + (int64_t)o * g.d_in + n, acc[i][j], g.d_in - n);
        }
      }
    }
    if (sums) {
#pragma unroll
      for (int i = 0; i < S::TM; ++i) {
        const int o = m0 + 16 * i + (l & 15);
        float all = sum[i] + __shfl_xor(sum[i], 16);
        all += __shfl_xor(all, 32);
        if (l >= 16 || o >= g.d_out) continue;
        if (whole) {
          g.dbias[(int64_t)leaf * g.d_out + o] = (T)all;
        } else {
          part[(int64_t)g.d_out * g.d_in + o] = all;
        }
      }
    }
  }
}

// One row of workgroups for each cut but the first position: the cut's leaf, if it crosses a cut here for the first time.
// Bound by the slots' bytes: 43 us after the 343 of the sums above, most of it the few longest leaves' slots in turn.
template <typename T, bool LISTED>
__global__ void __launch_bounds__(256) leaf_grad_join_kernel(const LeafArgs<T> g) {
  const int64_t block = (int64_t)blockIdx.y + 1;
  const int64_t at = block * g.cut;
  // the leaf that holds position at - 1 and position at: the last whose offset is < at
  int lo = 0, hi = g.n_leaves;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64, i = lo + (int)(threadIdx.x & 63) * step;
    const int n = __popcll(__ballot(i < hi && offset_at(g.offsets, i, g.n_positions) < at));
    if (n == 0) return;
    lo += (n - 1) * step;
    hi = lo + step < hi ? lo + step : hi;
  }
  const int begin = offset_at(g.offsets, lo, g.n_positions), end = offset_at(g.offsets, lo + 1, g.n_positions);
  if (begin >= at || end <= at || begin < at - g.cut) return;
  int64_t last = ((int64_t)end - 1) / g.cut;  // block of the last piece
  if constexpr (LISTED) {
    if (end - begin <= g.cut) return;
    last = begin / g.cut + (end - begin - 1) / g.cut;
  }
  const int64_t per = (int64_t)(g.d_in + 1) * g.d_out, n_w = (int64_t)g.d_in * g.d_out;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < per; e += (int64_t)gridDim.x * 256) {
    if (e < n_w ? g.dw == nullptr : g.dbias == nullptr) continue;
    float s = g.partial[(2 * (block - 1) + 1) * per + e];
    for (int64_t b = block; b <= last; b += 8) {  // (eight at a time on their way, added in order)
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        // (cut from the leaf: every piece but the last is one that is not the last of those that begin in its block)
        const int64_t slot = LISTED && b + k < last ? 2 * (b + k) + 1 : 2 * (b + k);
        v[k] = b + k <= last ? g.partial[slot * per + e] : 0.0f;
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) s = b + k <= last ? s + v[k] : s;
    }
    if (e < n_w) {
      g.dw[lo * n_w + e] = (T)s;
    } else {
      g.dbias[(int64_t)lo * g.d_out + (e - n_w)] = (T)s;
    }
  }
}

}  // namespace gbdt_leaf
