// Rows that several leaves answer with weights: y[d] = sum_j g[d][j] (W_l x[d] + b_l), l = leaves[d][j], and its gradients.
//
// A pair p = d * k + j is a row and one of its leaves.  Lists of pairs by leaf (route_kernels.h) make each product that of
// leaf_product_kernels.h, whose results go to a slot of f32 values for every pair; a second kernel weighs and adds up a row's slots
// in order.  So nothing is added from several workgroups to one place, the same call gives the same bits, and the result is rounded
// once.
#pragma once

#include "leaf_product_kernels.h"

namespace gbdt_routed {

using namespace gbdt_leaf;

template <typename T>
struct RoutedArgs : LeafArgs<T> {
  const int32_t* pair_idx;  // of the list's positions
  const int32_t* leaves;    // [n_rows][k]
  const float* gates;       // [n_rows][k]
  float* slots;             // [n_rows * k][ld_slots]
  float* dgates;            // [n_rows][k] or null
  int64_t ld_slots;         // a multiple of 4
  int32_t k;
};

// ---------------------------------------------------------------- products to slots

template <typename T>
struct ToSlots {
  typedef float Out;
  static constexpr bool kScaled = false;
  const T* bias;
  float* out;
  int64_t ld;
  __device__ __forceinline__ int place(const RoutedArgs<T>& g, int p) const { return g.pair_idx[p]; }
  __device__ __forceinline__ float add(int64_t column) const { return bias ? (float)bias[column] : 0.0f; }
};

template <class S>
__global__ void __launch_bounds__(S::NT, 2) routed_product_kernel(const RoutedArgs<typename S::T> g) {
  __shared__ __align__(16) char lds[S::kLdsBytes];
  leaf_rows_product<S, typename S::RowsB, 1>(lds, g, g.x, g.ld_x, g.d_in, ToSlots<typename S::T>{g.bias, g.slots, g.ld_slots}, g.d_out);
}

template <class S>
__global__ void __launch_bounds__(S::NT, 2) routed_grad_input_kernel(const RoutedArgs<typename S::T> g) {
  __shared__ __align__(16) char lds[S::kLdsBytes];
  leaf_rows_product<S, typename S::ColumnsB, 1>(lds, g, g.dy, g.ld_dy, g.d_out, ToSlots<typename S::T>{nullptr, g.slots, g.ld_slots}, g.d_in);
}

// ---------------------------------------------------------------- sums of slots

template <typename O>
struct CombineArgs {
  const float* slots;     // [n_rows * k][ld]
  const int32_t* leaves;  // [n_rows][k]; a slot whose leaf is none holds anything
  const float* gates;     // [n_rows][k]
  O* out;                 // [n_rows][cols] or null
  int64_t ld, ld_out;
  int32_t n_rows, n_leaves, k, cols;
  // gradient
  const O* x;             // [n_rows][cols]
  const O* dy;            // [n_rows][d_out]
  const O* bias;          // [n_leaves][d_out] or null
  float* dgates;          // [n_rows][k]
  int64_t ld_x, ld_dy;
  int32_t d_out;
};

__device__ __forceinline__ f32x4 load4(const float* p) { return *(const f32x4*)p; }

// Up to four values of any alignment, zeros behind.
template <typename T>
__device__ __forceinline__ f32x4 load4_any(const T* p, int valid) {
  f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
  if (valid >= 4) {
    T t[4];
    __builtin_memcpy(t, p, sizeof t);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)t[i];
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < valid) v[i] = (float)p[i];
  }
  return v;
}

__device__ __forceinline__ void add_scaled(f32x4& sum, float by, f32x4 v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) sum[i] = __builtin_fmaf(by, v[i], sum[i]);
}

// The weighted sum of a row's slots for four columns.
template <typename O>
__device__ __forceinline__ f32x4 weighted_sum(const CombineArgs<O>& g, int64_t d, int c) {
  f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
  const int64_t p0 = d * g.k;
#pragma unroll 4
  for (int j = 0; j < g.k; ++j)
    if ((uint32_t)g.leaves[p0 + j] < (uint32_t)g.n_leaves) add_scaled(sum, g.gates[p0 + j], load4(g.slots + (p0 + j) * g.ld + c));
  return sum;
}

// LANES lanes a row, four columns each at a time.
template <typename O, int LANES>
__global__ void __launch_bounds__(256) combine_kernel(const CombineArgs<O> g) {
  const int64_t d = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (d >= g.n_rows) return;
  for (int c = (int)(threadIdx.x & (LANES - 1)) * 4; c < g.cols; c += LANES * 4)
    store4(g.out + d * g.ld_out + c, weighted_sum(g, d, c), g.cols - c);
}

// dx[d] = sum_j g u_j and dg[d][j] = <u_j, x[d]> + <b_l, dy[d]>, u_j = W_l^T dy[d] in the row's slots: <W_l x, dy> is <x, W_l^T dy>, so
// the answers need not be kept.  A wavefront a row; up to kAtOnce slots are read once for both.
constexpr int kAtOnce = 8;
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) v += __shfl_xor(v, s);
  return v;
}
template <typename O>
__global__ void __launch_bounds__(256) combine_grad_kernel(const CombineArgs<O> g) {
  const int64_t d = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int l = threadIdx.x & 63;
  if (d >= g.n_rows) return;
  const int64_t p0 = d * g.k;
  if (g.dgates != nullptr) {
    const bool fused = g.k <= kAtOnce && g.out != nullptr;
    for (int j0 = 0; j0 < g.k; j0 += kAtOnce) {
      int leaf[kAtOnce];
      float gate[kAtOnce], dot[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int e = j0 + i < g.k ? g.leaves[p0 + j0 + i] : -1;
        leaf[i] = (uint32_t)e < (uint32_t)g.n_leaves ? e : -1;
        gate[i] = leaf[i] >= 0 ? g.gates[p0 + j0 + i] : 0.0f;
        dot[i] = 0.0f;
      }
      for (int c = l * 4; c < g.cols; c += 256) {
        const f32x4 x = load4_any(g.x + d * g.ld_x + c, g.cols - c);
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
        f32x4 u[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
          if (leaf[i] >= 0) u[i] = load4(g.slots + (p0 + j0 + i) * g.ld + c);
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          if (leaf[i] < 0) continue;
          const int valid = g.cols - c;
#pragma unroll
          for (int e = 0; e < 4; ++e) dot[i] = e < valid ? __builtin_fmaf(u[i][e], x[e], dot[i]) : dot[i];
          add_scaled(sum, gate[i], u[i]);
        }
        if (fused) store4(g.out + d * g.ld_out + c, sum, g.cols - c);
      }
      if (g.bias != nullptr) {
        for (int c = l * 4; c < g.d_out; c += 256) {
          const f32x4 dy = load4_any(g.dy + d * g.ld_dy + c, g.d_out - c);
#pragma unroll
          for (int i = 0; i < kAtOnce; ++i) {
            if (leaf[i] < 0) continue;
            const f32x4 b = load4_any(g.bias + (int64_t)leaf[i] * g.d_out + c, g.d_out - c);
#pragma unroll
            for (int e = 0; e < 4; ++e) dot[i] = __builtin_fmaf(b[e], dy[e], dot[i]);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        if (j0 + i >= g.k) break;
        const float all = wave_sum(dot[i]);
        if (l == 0) g.dgates[p0 + j0 + i] = leaf[i] >= 0 ? all : 0.0f;
      }
    }
    if (fused) return;
  }
  if (g.out != nullptr)
    for (int c = l * 4; c < g.cols; c += 256) store4(g.out + d * g.ld_out + c, weighted_sum(g, d, c), g.cols - c);
}

// ---------------------------------------------------------------- gradients of the weights

// g dy of every position, in the list's order, rounded to the products' type: dW_l = sum (g dy) x^T then is the sum of
// leaf_grad_weight_kernel.  (A value is off by half a step of its type; a sum of many such, of independent sign, by less than the
// rounding of the result.)  Columns [first, first + cols) of dy, zeros up to ld.
template <typename T>
__global__ void __launch_bounds__(256) gated_rows_kernel(const RoutedArgs<T> g, T* out, int64_t ld, int first, int cols) {
  const int p = (int)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (p >= offset_at(g.offsets, g.n_leaves, g.n_positions)) return;
  const float gate = g.gates[g.pair_idx[p]];
  const T* dy = row_of(g.dy, g.row_idx[p], g.ld_dy) + first;
  constexpr int n = kChunk<T>;
  for (int c = (int)(threadIdx.x & 63) * n; c < ld; c += 64 * n) {
    T t[n];
    if (c + n <= cols) {
      __builtin_memcpy(t, dy + c, sizeof t);
#pragma unroll
      for (int e = 0; e < n; ++e) t[e] = (T)(gate * (float)t[e]);
    } else {
#pragma unroll
      for (int e = 0; e < n; ++e) t[e] = c + e < cols ? (T)(gate * (float)dy[c + e]) : (T)0.0f;
    }
    __builtin_memcpy(out + (int64_t)p * ld + c, t, sizeof t);
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
        const float all = wave_sum(sum[j][i]);
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
