// Rows that several leaves answer with weights: y[d] = sum_j g[d][j] (W_l x[d] + b_l), l = leaves[d][j], and its gradients.
//
// A pair p = d * k + j is a row and one of its leaves.  Lists of pairs by leaf (route_kernels.h) make each product that of
// leaf_product_kernels.h, whose results go to a slot for every pair; a second kernel weighs and adds up a row's slots in order.  So
// nothing is added from several workgroups to one place, the same call gives the same bits, and sums are f32.
//
// Slots hold f32, of bf16 results as well: a row's answers may cancel in their sum, and outputs beside each other may be of any size.
// (Half the bytes, as fp16 values with a power of two that 64 columns share, lost outputs beside one 2^29 times as large or closed by the
// type's lowest value.)
#pragma once

#include "leaf_product_kernels.h"

namespace gbdt_routed {

using namespace gbdt_leaf;

template <typename T>
struct RoutedArgs : LeafArgs<T> {
  const int32_t* pair_idx;  // of the list's positions
  const int32_t* leaves;    // [n_rows][k]
  const float* gates;       // [n_rows][k]
  float* dgates;            // [n_rows][k] or null
  float* slots;             // [n_rows * k][ld_slots] or null
  float* dots;              // gradient: [n_rows * k][blocks], parts of <u, x>, or null
  int64_t ld_slots;         // a multiple of 16 bytes
  int32_t k, blocks;        // blocks of block_columns columns
};

// The columns of a wavefront in the tiles that make slots.
template <typename T> constexpr int block_columns = sizeof(T) == 4 ? 32 : 64;  // T: the operands'

// ---------------------------------------------------------------- products to slots

__device__ __forceinline__ float over_groups(float v) {  // over the four groups of 16 lanes
#pragma unroll
  for (int m = 16; m < 64; m <<= 1) v += __shfl_xor(v, m);
  return v;
}

// To the pairs' slots.  DOTS: each row's values also meet x's, and their sums over the wavefront's columns are left in
// dots: dg[d][j] = <dy, W x + b> = <W^T dy, x> + <dy, b>, so the gates' gradient needs the answers of neither pass, only f32 values
// that are in registers here.
template <typename T, bool DOTS>
struct ToSlots {
  typedef float Out;
  static constexpr bool kScaled = false, kFinished = DOTS, kDots = DOTS;
  const T* bias;
  float* out;
  int64_t ld;
  __device__ __forceinline__ int place(const RoutedArgs<T>& g, int p) const { return g.pair_idx[p]; }
  __device__ __forceinline__ float add(int64_t column) const { return bias ? (float)bias[column] : 0.0f; }
  struct Beside {
    T x[4];
  };
  // x's values at this lane's columns, zeros past the last.
  template <int TN>
  __device__ __forceinline__ void beside(const RoutedArgs<T>& g, int row, int col, int cols, Beside (&to)[TN]) const {
    const T* x = row_of(g.x, row, g.ld_x);
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int n = col + 16 * j + 4 * (int)((threadIdx.x & 63) >> 4);
      if (n + 4 <= cols) {
        __builtin_memcpy(to[j].x, x + n, sizeof to[j].x);
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) to[j].x[r] = n + r < cols ? x[n + r] : (T)0.0f;
      }
    }
  }
  template <int TN>
  __device__ __forceinline__ void finish(const RoutedArgs<T>& g, int pair, int col, int cols, const Beside (&x)[TN], f32x4 (&v)[TN]) const {
    static_assert(TN * 16 == block_columns<T>, "a wavefront's columns");
    const int l = threadIdx.x & 63;
    float dot = 0.0f;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int n = col + 16 * j + 4 * (l >> 4);
#pragma unroll
      for (int r = 0; r < 4; ++r) dot = n + r < cols ? __builtin_fmaf(v[j][r], (float)x[j].x[r], dot) : dot;
    }
    dot = over_groups(dot);
    if (l < 16 && pair >= 0 && col < cols) g.dots[(int64_t)pair * g.blocks + col / (TN * 16)] = dot;
  }
};

// k = 1: a row's only answer, weighed, is the result.
template <typename T>
struct ToGatedRows {
  typedef T Out;
  static constexpr bool kScaled = false, kFinished = true, kDots = false;
  const T* bias;
  T* out;
  int64_t ld;
  __device__ __forceinline__ int place(const RoutedArgs<T>& g, int p) const { return g.pair_idx[p]; }
  __device__ __forceinline__ float add(int64_t column) const { return bias ? (float)bias[column] : 0.0f; }
  struct Beside {};
  template <int TN>
  __device__ __forceinline__ void finish(const RoutedArgs<T>& g, int pair, int, int, const Beside (&)[TN], f32x4 (&v)[TN]) const {
    const float gate = pair >= 0 ? g.gates[pair] : 0.0f;
#pragma unroll
    for (int j = 0; j < TN; ++j) v[j] *= gate;
  }
};

// Where a product over pairs leaves its answers: in slots, or weighed in the rows of y (k = 1).
enum class Leaves { kSlots, kRows };

// Answers of all pairs.  Bound by the matrix cores and by what a tile's beginning and end leave them idle: 65,536 pairs, 1,024 -> 1,024 in
// 64 leaves, bf16: 205 us, 670 TFLOP/s, matrix cores busy for 33 % of the cycles, compute units for 77 (leaves end inside tiles of
// 256 rows, and 4.5 tiles a unit are five turns; 268 MB of answers are written beneath).  256 pairs of 64 leaves, tiles of 32 rows: 25 us, 5.1 TB/s of matrices, some of which
// the memory-side cache holds.
template <class S, Leaves WHAT>
__global__ void __launch_bounds__(S::NT, 2) routed_product_kernel(const RoutedArgs<typename S::T> g) {
  typedef typename S::T T;
  __shared__ __align__(16) char lds[S::kLdsBytes];
  if constexpr (WHAT == Leaves::kRows) {
    rows_product<S, typename S::RowsB>(lds, g, g.x, g.ld_x, g.d_in, ToGatedRows<T>{g.bias, g.y, g.ld_y}, g.d_out);
  } else {
    rows_product<S, typename S::RowsB>(lds, g, g.x, g.ld_x, g.d_in, ToSlots<T, false>{g.bias, g.slots, g.ld_slots}, g.d_out);
  }
}

// Gradients of the rows by every pair.  Bound as above, beside reading x once more for the gates' gradients: 32,768 pairs, 1,024 ->
// 1,024 in 64 leaves, bf16: 141 us (114 the answers); 60,033 pairs, 33 -> 137 in 63 leaves, f32: 39 us, tiles of 64 half full of k.
template <class S, bool DOTS>
__global__ void __launch_bounds__(S::NT, 2) routed_grad_input_kernel(const RoutedArgs<typename S::T> g) {
  typedef typename S::T T;
  __shared__ __align__(16) char lds[S::kLdsBytes];
  rows_product<S, typename S::ColumnsB>(lds, g, g.dy, g.ld_dy, g.d_out, ToSlots<T, DOTS>{nullptr, g.slots, g.ld_slots}, g.d_in);
}

// ---------------------------------------------------------------- sums of slots

template <typename O>
struct CombineArgs {
  const float* slots;     // [n_rows * k][ld]; a slot whose leaf is none holds anything
  const int32_t* leaves;  // [n_rows][k]
  const float* gates;     // [n_rows][k]
  O* out;                 // [n_rows][cols] or null
  int64_t ld, ld_out;
  int32_t n_rows, n_leaves, k, cols, blocks;
  // gradient of the gates
  const float* dots;      // [n_rows * k][blocks]
  const O* dy;            // [n_rows][d_out]
  const O* bias;          // [n_leaves][d_out] or null
  float* dgates;          // [n_rows][k] or null
  int64_t ld_dy;
  int32_t d_out;
};

template <int LANES>
__device__ __forceinline__ float over_row(float v) {
#pragma unroll
  for (int s = LANES / 2; s > 0; s >>= 1) v += __shfl_xor(v, s);
  return v;
}

// (said to be device memory, as load16 says)
__device__ __forceinline__ float load_float(const float* p) { return *(const __attribute__((address_space(1))) float*)p; }

// Eight of a row's slots: whether there is a leaf, and its weight.
constexpr int kSlotsAtOnce = 8;
struct SlotGates {
  int leaf[kSlotsAtOnce];  // -1 for none
  float gate[kSlotsAtOnce];
  template <typename O>
  __device__ __forceinline__ void load(const CombineArgs<O>& g, int64_t p0, int j0) {
#pragma unroll
    for (int i = 0; i < kSlotsAtOnce; ++i) {  // (loads without a branch, which would be waited for one by one)
      const int64_t p = p0 + (j0 + i < g.k ? j0 + i : g.k - 1);
      leaf[i] = g.leaves[p];
      gate[i] = g.gates[p];
    }
#pragma unroll
    for (int i = 0; i < kSlotsAtOnce; ++i)
      if (j0 + i >= g.k || (uint32_t)leaf[i] >= (uint32_t)g.n_leaves) leaf[i] = -1;
  }
};

// The gates' gradients of four slots of row d from slot j0 on.
template <typename O, int LANES>
__device__ __forceinline__ void gate_gradients(const CombineArgs<O>& g, int64_t d, int j0, const int* leaf) {
  constexpr int pairs = kSlotsAtOnce / 2, m = kChunk<O>;
  const int l = threadIdx.x & (LANES - 1);
  const int64_t p0 = d * g.k + j0;
  const O* dy = g.dy + d * g.ld_dy;
  float dot[pairs];
#pragma unroll
  for (int i = 0; i < pairs; ++i) dot[i] = 0.0f;
  for (int b = l; b < g.blocks; b += LANES) {
#pragma unroll
    for (int i = 0; i < pairs; ++i) dot[i] += load_float(leaf[i] >= 0 ? g.dots + (p0 + i) * g.blocks + b : (const float*)zero_chunk);
  }
  if (g.bias != nullptr) {
    for (int c = l * m; c < g.d_out; c += LANES * m) {
      O y[m], w[pairs][m];
      if (c + m <= g.d_out) {
        __builtin_memcpy(y, dy + c, sizeof y);
#pragma unroll
        for (int i = 0; i < pairs; ++i) __builtin_memcpy(w[i], g.bias + (int64_t)(leaf[i] < 0 ? 0 : leaf[i]) * g.d_out + c, sizeof y);
      } else {
#pragma unroll
        for (int e = 0; e < m; ++e) {
          y[e] = c + e < g.d_out ? dy[c + e] : (O)0.0f;
#pragma unroll
          for (int i = 0; i < pairs; ++i)
            w[i][e] = c + e < g.d_out ? g.bias[(int64_t)(leaf[i] < 0 ? 0 : leaf[i]) * g.d_out + c + e] : (O)0.0f;
        }
      }
#pragma unroll
      for (int i = 0; i < pairs; ++i)
#pragma unroll
        for (int e = 0; e < m; ++e) dot[i] = __builtin_fmaf((float)w[i][e], (float)y[e], dot[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < pairs; ++i) {
    const float all = over_row<LANES>(dot[i]);
    if (l == 0 && j0 + i < g.k) g.dgates[p0 + i] = leaf[i] >= 0 ? all : 0.0f;
  }
}

// out[d] = sum_j g[d][j] slot_j, LANES lanes a row, 16 bytes of a slot each at a time, eight slots on their way; dgates[d][j] =
// the sum of the pair's dots and <bias, dy>.  Bound by reading the slots: 8,192 rows x 8 slots of 1,024 values, 49 us, 5.5 TB/s (the
// memory-side cache has some); x 4, 28 us, with the gates' gradients 35.
template <typename O, int LANES, bool GATES>
__global__ void __launch_bounds__(256) combine_kernel(const CombineArgs<O> g) {
  constexpr int n = 4;
  const int64_t d = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (d >= g.n_rows) return;
  const int l = threadIdx.x & (LANES - 1);
  const int64_t p0 = d * g.k;
  const bool once = g.k <= kSlotsAtOnce;
  SlotGates slots;
  slots.load(g, p0, 0);
  if (g.out != nullptr) {
    for (int c = l * n; c < g.cols; c += LANES * n) {
      float sum[n];
#pragma unroll
      for (int e = 0; e < n; ++e) sum[e] = 0.0f;
      for (int j0 = 0; j0 < g.k; j0 += kSlotsAtOnce) {
        if (!once) slots.load(g, p0, j0);
        u32x4 raw[kSlotsAtOnce];
#pragma unroll
        for (int i = 0; i < kSlotsAtOnce; ++i)
          raw[i] = load16(slots.leaf[i] >= 0 ? (const void*)(g.slots + (p0 + j0 + i) * g.ld + c) : (const void*)zero_chunk);
#pragma unroll
        for (int i = 0; i < kSlotsAtOnce; ++i) {
          const float by = slots.leaf[i] < 0 ? 0.0f : slots.gate[i];
          float v[n];
          __builtin_memcpy(v, &raw[i], 16);
#pragma unroll
          for (int e = 0; e < n; ++e) sum[e] = __builtin_fmaf(by, v[e], sum[e]);
        }
      }
      O* to = g.out + d * g.ld_out + c;
      O t[n];
#pragma unroll
      for (int e = 0; e < n; ++e) t[e] = (O)sum[e];
      if (c + n <= g.cols) {
        __builtin_memcpy(to, t, sizeof t);
      } else {
#pragma unroll
        for (int e = 0; e < n; ++e)
          if (c + e < g.cols) to[e] = t[e];
      }
    }
  }
  if constexpr (!GATES) return;
  for (int j0 = 0; j0 < g.k; j0 += kSlotsAtOnce) {
    if (!once) slots.load(g, p0, j0);
    gate_gradients<O, LANES>(g, d, j0, &slots.leaf[0]);
    if (j0 + kSlotsAtOnce / 2 < g.k) gate_gradients<O, LANES>(g, d, j0 + kSlotsAtOnce / 2, &slots.leaf[kSlotsAtOnce / 2]);
  }
}

// Zeros for the rows that no leaf answers, where answers go to rows directly (k = 1).
template <typename O>
__global__ void __launch_bounds__(256) clear_rows_kernel(const int32_t* leaves, int32_t n_leaves, int32_t n_rows, int32_t cols, O* out, int64_t ld) {
  const int64_t d = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (d >= n_rows || (uint32_t)leaves[d] < (uint32_t)n_leaves) return;
  for (int c = 0; c < cols; ++c) out[d * ld + c] = (O)0.0f;
}

// ---------------------------------------------------------------- gradients of the weights

// g dy of every position, in the list's order: dW_l = sum (g dy) x^T then is the sum of leaf_grad_weight_kernel, 225 to 245 us for 32,768
// positions of 64 leaves, 1,024 x 1,024, bf16.  The matrix cores take bf16 only, so g dy is the sum of two such values: 2^-17 of a term at
// most is left out.  (One value, off by half a step of every term: 140 us, and 2.3e-3 of the results' size instead of the 1.7e-3 of their own rounding.)
// Bound by memory: the same case 32 us, 6.3 TB/s.
//  Columns [first, first + cols) of dy, zeros up to ld; positions from `from` on.
template <typename T, int LANES>
__global__ void __launch_bounds__(256) gated_rows_kernel(const RoutedArgs<T> g, T* out, int64_t ld, int first, int cols, int from) {
  const int p = from + (int)(blockIdx.x * (256 / LANES) + threadIdx.x / LANES);
  if (p >= offset_at(g.offsets, g.n_leaves, g.n_positions)) return;
  const float gate = g.gates[g.pair_idx[p]];
  const T* dy = row_of(g.dy, g.row_idx[p], g.ld_dy) + first;
  constexpr int n = kChunk<T>;
  for (int c = (int)(threadIdx.x & (LANES - 1)) * n; c < ld; c += LANES * n) {
    T t[n], rest[n];
    if (c + n <= cols) {
      __builtin_memcpy(t, dy + c, sizeof t);
    } else {
#pragma unroll
      for (int e = 0; e < n; ++e) t[e] = c + e < cols ? dy[c + e] : (T)0.0f;
    }
#pragma unroll
    for (int e = 0; e < n; ++e) {
      const float v = gate * (float)t[e];
      t[e] = c + e < cols ? (T)v : (T)0.0f;
      rest[e] = fabsf((float)t[e]) < INFINITY ? (T)(v - (float)t[e]) : (T)0.0f;
    }
    constexpr int each = kRowsEach<T, true>;
    T* to = out + (int64_t)p * each * ld + c;
    __builtin_memcpy(to, t, sizeof t);
    if constexpr (each == 2) __builtin_memcpy(to + ld, rest, sizeof rest);
  }
}

// db_l = sum of g dy over the leaf's positions, of products in f32: what rounds g dy for dW, that the matrix cores take it, has no part here, and
// a leaf's rows may cancel.  A workgroup takes a piece of the positions (leaf_product_kernels.h) and 16 chunks of columns, 16
// lanes a row, eight rows on their way; groups of lanes are added up in order.  Bound by the rows' lines, 256 bytes of each, and a chain of
// round trips: 32,768 positions of 64 leaves, 1,024 outputs, bf16, 30 us, 2.2 TB/s.
constexpr int kSumThreads = 1024, kSumLanes = 16, kSumsAtOnce = 8;
template <typename T>
__global__ void __launch_bounds__(kSumThreads) gated_sums_kernel(const RoutedArgs<T> g, int64_t first) {
  constexpr int n = kChunk<T>, groups = kSumThreads / kSumLanes, columns = kSumLanes * n;
  __shared__ float sums[groups][columns];
  const int64_t block = first + blockIdx.x;
  const int blocks = (g.d_out + columns - 1) / columns;
  const Piece piece = find_piece<true>(g, (int)(block / blocks));
  if (piece.leaf < 0) return;
  const int col0 = (int)(block % blocks) * columns, group = threadIdx.x / kSumLanes, c = col0 + (int)(threadIdx.x % kSumLanes) * n;
  float sum[n];
#pragma unroll
  for (int e = 0; e < n; ++e) sum[e] = 0.0f;
  for (int64_t p = (int64_t)piece.p0 + group; p < piece.p1; p += groups * kSumsAtOnce) {
    float gate[kSumsAtOnce];
    const T* dy[kSumsAtOnce];
#pragma unroll
    for (int i = 0; i < kSumsAtOnce; ++i) {
      const int64_t at = p + i * groups;
      const bool there = at < piece.p1;
      gate[i] = there ? g.gates[g.pair_idx[at]] : 0.0f;
      dy[i] = there ? row_of(g.dy, g.row_idx[at], g.ld_dy) : nullptr;
    }
    T t[kSumsAtOnce][n];
#pragma unroll
    for (int i = 0; i < kSumsAtOnce; ++i)
      if (dy[i] != nullptr && c + n <= g.d_out) {
        __builtin_memcpy(t[i], dy[i] + c, sizeof t[i]);
      } else {
#pragma unroll
        for (int e = 0; e < n; ++e) t[i][e] = dy[i] != nullptr && c + e < g.d_out ? dy[i][c + e] : (T)0.0f;
      }
#pragma unroll
    for (int i = 0; i < kSumsAtOnce; ++i)
#pragma unroll
      for (int e = 0; e < n; ++e) sum[e] = __builtin_fmaf(gate[i], (float)t[i][e], sum[e]);
  }
#pragma unroll
  for (int e = 0; e < n; ++e) sums[group][threadIdx.x % kSumLanes * n + e] = sum[e];
  __syncthreads();
  const int o = col0 + (int)threadIdx.x;
  if ((int)threadIdx.x >= columns || o >= g.d_out) return;
  float all = 0.0f;
  for (int q = 0; q < groups; ++q) all += sums[q][threadIdx.x];
  if (piece.whole) {
    g.dbias[(int64_t)piece.leaf * g.d_out + o] = (T)all;
  } else {
    g.partial[piece.slot * ((int64_t)(g.d_in + 1) * g.d_out) + (int64_t)g.d_out * g.d_in + o] = all;
  }
}

// ---------------------------------------------------------------- few rows

// A few rows: a wavefront takes OUTPUTS outputs of one row, all of its leaves one after another, four at a time; no lists, no slots,
// one launch.  (As leaf_product_few_kernel: the end of a row that is no whole chunk is read as its last whole chunk.)
template <typename T, int OUTPUTS>
__global__ void __launch_bounds__(64) routed_few_kernel(const RoutedArgs<T> g) {
  const int64_t d = blockIdx.y;
  const int o0 = (int)blockIdx.x * OUTPUTS, l = threadIdx.x;
  const T* x = g.x + d * g.ld_x;
  constexpr int n = kChunk<T>, at_once = 4;
  float y[OUTPUTS];
#pragma unroll
  for (int i = 0; i < OUTPUTS; ++i) y[i] = 0.0f;
  for (int j0 = 0; j0 < g.k; j0 += at_once) {
    int leaf[at_once];
    float gate[at_once], sum[at_once][OUTPUTS];
#pragma unroll
    for (int j = 0; j < at_once; ++j) {
      const int e = j0 + j < g.k ? g.leaves[d * g.k + j0 + j] : -1;
      leaf[j] = (uint32_t)e < (uint32_t)g.n_leaves ? e : -1;
      gate[j] = leaf[j] >= 0 ? g.gates[d * g.k + j0 + j] : 0.0f;
#pragma unroll
      for (int i = 0; i < OUTPUTS; ++i) sum[j][i] = 0.0f;
    }
    if (g.d_in >= n) {
      for (int k = l * n; k < g.d_in; k += 64 * n) {
        const int at = k + n <= g.d_in ? k : g.d_in - n, skip = k - at;
        const u32x4 xc = load16(x + at);
        u32x4 wc[at_once][OUTPUTS];
#pragma unroll
        for (int j = 0; j < at_once; ++j)
#pragma unroll
          for (int i = 0; i < OUTPUTS; ++i)
            wc[j][i] = load16(g.w + ((int64_t)(leaf[j] < 0 ? 0 : leaf[j]) * g.d_out + (o0 + i < g.d_out ? o0 + i : o0)) * g.d_in + at);
        T xv[n], wv[n];
        __builtin_memcpy(xv, &xc, 16);
#pragma unroll
        for (int j = 0; j < at_once; ++j)
#pragma unroll
          for (int i = 0; i < OUTPUTS; ++i) {
            __builtin_memcpy(wv, &wc[j][i], 16);
#pragma unroll
            for (int e = 0; e < n; ++e) sum[j][i] = e >= skip ? __builtin_fmaf((float)xv[e], (float)wv[e], sum[j][i]) : sum[j][i];
          }
      }
    } else if (l < g.d_in) {
#pragma unroll
      for (int j = 0; j < at_once; ++j)
#pragma unroll
        for (int i = 0; i < OUTPUTS; ++i)
          if (leaf[j] >= 0 && o0 + i < g.d_out) sum[j][i] = (float)x[l] * (float)g.w[((int64_t)leaf[j] * g.d_out + o0 + i) * g.d_in + l];
    }
#pragma unroll
    for (int j = 0; j < at_once; ++j) {
      if (leaf[j] < 0) continue;
#pragma unroll
      for (int i = 0; i < OUTPUTS; ++i) {
        const float all = over_row<64>(sum[j][i]);
        const float b = g.bias && o0 + i < g.d_out ? (float)g.bias[(int64_t)leaf[j] * g.d_out + o0 + i] : 0.0f;
        y[i] = __builtin_fmaf(gate[j], all + b, y[i]);
      }
    }
  }
  if (l != 0) return;
#pragma unroll
  for (int i = 0; i < OUTPUTS; ++i)
    if (o0 + i < g.d_out) g.y[d * g.ld_y + o0 + i] = (T)y[i];
}

}  // namespace gbdt_routed
