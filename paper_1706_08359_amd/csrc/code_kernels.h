// Leaf products in 8-bit integers: rows and matrices as codes with a scale each, x ~ q s.
//
//   s = max |x| * (1 / 127) (f32, both factors)      q = x / s to the nearest whole number, ties to even
//   y[d] = (sum q_x q_w) s_d s_lo + b_lo       sums of codes exact in 32 bits
//
// Rows of codes are a multiple of 16 long, zeros behind, so every operand is whole chunks.
#pragma once

#include "routed_kernels.h"

namespace gbdt_code {

using namespace gbdt_routed;

// A product's limit: 127 * 127 * kMaxWidth < 2^31.
constexpr int kMaxWidth = 131072;

struct CodeArgs : RoutedArgs<int8_t> {   // d_in: of the codes
  const float* row_scales;   // [n_rows]
  const float* col_scales;   // [n_leaves][d_out]
  const float* add;          // [n_leaves][d_out] or null
  void* out;
  int64_t ld_out;
};

// ---------------------------------------------------------------- rows to codes

struct QuantizeArgs {
  const void* x;
  int8_t* codes;
  float* scales;
  int64_t ld_x, ld_codes;
  int64_t n_rows;
  int32_t cols, padded;
};

__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ float value_of(float v) { return v; }
__device__ __forceinline__ float value_of(bf16 v) { return (float)v; }

// The code of v: the quotient's rounding in f32 may carry it over a half, so the remainder decides, which is exact where it
// is near half a scale (either both terms are multiples of the scale's last place, or v is below the scale and the difference of
// two numbers within a factor of two).
__device__ __forceinline__ int code_of(float v, float scale, float inverse) {
  float q = rintf(v * inverse);
  const float rest = __builtin_fmaf(-q, scale, v), twice = 2.0f * fabsf(rest);
  const bool odd = (int)q & 1;
  if (twice > scale || (twice == scale && odd)) q += copysignf(1.0f, rest);
  return (int)q;
}

// A wavefront a row, CHUNKS chunks of 8 values a lane held in registers; longer rows are read twice.  The largest magnitude as an
// integer: a NaN is larger than every number.  Bound by memory: 8,192 x 1,024 bf16 in 9.5 us, 2.7 TB/s, a third of it the launch.
template <typename T, int CHUNKS>
__global__ void __launch_bounds__(256) quantize_kernel(const QuantizeArgs g) {
  const int64_t d = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (d >= g.n_rows) return;
  const int l = threadIdx.x & 63;
  const T* x = (const T*)g.x + d * g.ld_x;
  float v[CHUNKS][8];
  uint32_t most = 0;
  auto load = [&](int c, float (&to)[8]) {
    if (c + 8 <= g.cols) {
      T t[8];
      __builtin_memcpy(t, x + c, sizeof t);
#pragma unroll
      for (int e = 0; e < 8; ++e) to[e] = value_of(t[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) to[e] = c + e < g.cols ? value_of(x[c + e]) : 0.0f;
    }
  };
  for (int c0 = 0; c0 < g.padded; c0 += CHUNKS * 512) {
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) load(c0 + (i * 64 + l) * 8, v[i]);
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t m = magnitude_bits(v[i][e]);
        most = m > most ? m : most;
      }
  }
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) {
    const uint32_t other = __shfl_xor(most, s);
    most = other > most ? other : most;
  }
  // a row with an infinity or a NaN has no scale; one whose scale would be below the normal numbers is zeros
  const bool finite = most < 0x7f800000u;
  float scale = finite ? __uint_as_float(most) * (1.0f / 127.0f) : __uint_as_float(0x7fc00000u);
  if (finite && scale < 0x1p-126f) scale = 0.0f;
  const bool zero = !(scale > 0.0f);
  const float inverse = zero ? 0.0f : 1.0f / scale;
  if (l == 0) g.scales[d] = scale;
  for (int c0 = 0; c0 < g.padded; c0 += CHUNKS * 512) {
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int c = c0 + (i * 64 + l) * 8;
      if (c >= g.padded) break;
      if (g.padded > CHUNKS * 512) load(c, v[i]);
      int8_t q[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) q[e] = zero ? (int8_t)0 : (int8_t)code_of(v[i][e], scale, inverse);
      __builtin_memcpy(g.codes + d * g.ld_codes + c, q, 8);
    }
  }
}

// ---------------------------------------------------------------- products

// Where the results go: to the row of y (kRow), weighed to the row of y (kGatedRow: k = 1), or to the pair's slot.
enum class Place { kRow, kGatedRow, kSlot };

template <typename O, Place WHERE>
struct ToScaled {
  typedef typename std::conditional<WHERE == Place::kSlot, float, O>::type Out;
  static constexpr bool kScaled = true, kFinished = WHERE == Place::kGatedRow, kDots = false;
  Out* out;
  int64_t ld;
  const float* row_scales;
  const float* col_scales;
  const float* bias;
  __device__ __forceinline__ int row(const CodeArgs& g, int p) const { return g.row_idx ? g.row_idx[p] : p; }
  __device__ __forceinline__ int place(const CodeArgs& g, int p) const {
    if (WHERE != Place::kRow) return g.pair_idx[p];
    const int d = row(g, p);
    return (uint32_t)d < (uint32_t)g.n_rows ? d : -1;
  }
  __device__ __forceinline__ float row_scale(const CodeArgs& g, int p) const { return row_scales[row(g, p)]; }
  __device__ __forceinline__ float column_scale(int64_t column) const { return col_scales[column]; }
  __device__ __forceinline__ float add(int64_t column) const { return bias ? bias[column] : 0.0f; }
  struct Beside {};
  template <int TN>
  __device__ __forceinline__ void finish(const CodeArgs& g, int pair, int, int, const Beside (&)[TN], f32x4 (&v)[TN]) const {
    const float gate = pair >= 0 ? g.gates[pair] : 0.0f;
#pragma unroll
    for (int j = 0; j < TN; ++j) v[j] *= gate;
  }
};

// Bound by the gathered rows of codes where outputs are few: 400,000 x 2,000 -> 128 in 255 leaves, 274 us, 3.6 TB/s of rows' lines and
// matrices, waiting for half of the cycles (tiles of 128 x 128, two a unit, 307; with two stages instead of three 293); by the ends
// of tiles where they are many: 32,768 pairs, 1,024 -> 1,024 in 64 leaves, 72 us, 950 TOP/s.
template <class S, typename O, Place WHERE>
__global__ void __launch_bounds__(S::NT, 2) code_product_kernel(const CodeArgs g) {
  __shared__ __align__(16) char lds[S::kLdsBytes];
  typedef ToScaled<O, WHERE> To;
  const bool slot = WHERE == Place::kSlot;
  const To to = {(typename To::Out*)(slot ? (void*)g.slots : g.out), slot ? g.ld_slots : g.ld_out, g.row_scales, g.col_scales, g.add};
  rows_product<S, typename S::RowsB>(lds, g, g.x, g.ld_x, g.d_in, to, g.d_out);
}

// A few rows: OUTPUTS outputs of one row a wavefront, sums of four products an instruction.  LISTED: one leaf a row, by position in
// the list; else the k leaves of row blockIdx.y with their weights.
template <typename O, int OUTPUTS, bool LISTED>
__global__ void __launch_bounds__(64) code_few_kernel(const CodeArgs g) {
  const int o0 = (int)blockIdx.x * OUTPUTS, l = threadIdx.x;
  int64_t d = blockIdx.y;
  int only = -1;
  if (LISTED) {
    const int p = (int)blockIdx.y;
    d = g.row_idx ? g.row_idx[p] : p;
    only = find_leaf(g.offsets, g.n_leaves, g.n_positions, 0, p);
    if (only < 0 || (uint64_t)d >= (uint64_t)g.n_rows || p >= offset_at(g.offsets, only + 1, g.n_positions)) return;
  }
  const int8_t* x = g.x + d * g.ld_x;
  const float row_scale = g.row_scales[d];
  constexpr int at_once = LISTED ? 1 : 4;
  const int k = LISTED ? 1 : g.k;
  float y[OUTPUTS];
#pragma unroll
  for (int i = 0; i < OUTPUTS; ++i) y[i] = 0.0f;
  for (int j0 = 0; j0 < k; j0 += at_once) {
    int leaf[at_once];
    float gate[at_once];
    int sum[at_once][OUTPUTS];
#pragma unroll
    for (int j = 0; j < at_once; ++j) {
      const int e = LISTED ? only : j0 + j < k ? g.leaves[d * k + j0 + j] : -1;
      leaf[j] = (uint32_t)e < (uint32_t)g.n_leaves ? e : -1;
      gate[j] = LISTED ? 1.0f : leaf[j] >= 0 ? g.gates[d * k + j0 + j] : 0.0f;
#pragma unroll
      for (int i = 0; i < OUTPUTS; ++i) sum[j][i] = 0;
    }
    for (int c = l * 16; c < g.d_in; c += 64 * 16) {
      const u32x4 xc = load16(x + c);
      u32x4 wc[at_once][OUTPUTS];
#pragma unroll
      for (int j = 0; j < at_once; ++j)
#pragma unroll
        for (int i = 0; i < OUTPUTS; ++i)
          wc[j][i] = load16(g.w + ((int64_t)(leaf[j] < 0 ? 0 : leaf[j]) * g.d_out + (o0 + i < g.d_out ? o0 + i : o0)) * g.d_in + c);
#pragma unroll
      for (int j = 0; j < at_once; ++j)
#pragma unroll
        for (int i = 0; i < OUTPUTS; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[j][i] = __builtin_amdgcn_sdot4((int)xc[e], (int)wc[j][i][e], sum[j][i], false);
    }
#pragma unroll
    for (int j = 0; j < at_once; ++j) {
      if (leaf[j] < 0) continue;
#pragma unroll
      for (int i = 0; i < OUTPUTS; ++i) {
        int all = sum[j][i];
#pragma unroll
        for (int s = 32; s > 0; s >>= 1) all += __shfl_xor(all, s);
        const int64_t o = (int64_t)leaf[j] * g.d_out + (o0 + i < g.d_out ? o0 + i : o0);
        y[i] = __builtin_fmaf(gate[j], scaled((float)all, row_scale, g.col_scales[o], g.add ? g.add[o] : 0.0f), y[i]);
      }
    }
  }
  if (l != 0) return;
#pragma unroll
  for (int i = 0; i < OUTPUTS; ++i)
    if (o0 + i < g.d_out) ((O*)g.out)[d * g.ld_out + o0 + i] = (O)y[i];
}

}  // namespace gbdt_code
