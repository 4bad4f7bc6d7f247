// A learned router: which k of the leaves answer a row, and with what weights; and the lists of rows by leaf that follow.
//
// Scores s are the softmax of a row's logits, or their sigmoids.  The k leaves of the largest choice values c = s + bias are
// taken, those of equal values from the lowest index; without a bias the order of s is that of the logits, which are compared
// themselves.  A row is LANES lanes' work, PER neighbouring columns each: a pick is a maximum over the lanes and the first lane
// that holds it.  Sixteen lanes where 16 columns each hold a row: the maximum then takes four moves of the vector unit for four rows.
//
// c decides between neighbours, so its roundings must not.  Values are taken in f32 with a bound of their error; a row that has two
// values closer than that among its first k + 1, or at the border of its groups, is taken again in 64 bits, by the whole wavefront.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

namespace gbdt_router {

constexpr int kMaxLeaves = 1024, kMaxChosen = 32, kMaxGroups = 64;
constexpr int kThreads = 256;

struct RouteArgs {
  const void* logits;   // [n_rows][n_leaves]
  const float* bias;    // [n_leaves] or null
  int32_t* leaves;      // [n_rows][k]
  float* gates;         // [n_rows][k]
  const float* dgates;  // gradient: [n_rows][k]
  void* dlogits;        // gradient: [n_rows][n_leaves]
  int64_t ld, ld_out;
  int64_t first;        // row of this launch's first
  int32_t n_rows, n_leaves, k;
  int32_t n_groups, groups_kept, group_best, group_size;
  int32_t sigmoid, renormalise;
  float scale;
};

// ---------------------------------------------------------------- lanes of a row

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

// op over the row's lanes, in all of them.  Within 16 lanes by moves of the vector unit: neighbours, pairs, the other half of
// eight and of sixteen (mirrored: each half is uniform by then); then by exchanges of rows of 16 and of halves.
template <int LANES, class Op>
__device__ __forceinline__ float over_lanes(float v, const Op& op) {
  v = op(v, dpp<0xB1>(v));                     // lanes 1 0 3 2
  if (LANES >= 4) v = op(v, dpp<0x4E>(v));     // lanes 2 3 0 1
  if (LANES >= 8) v = op(v, dpp<0x141>(v));    // mirrored within 8
  if (LANES >= 16) v = op(v, dpp<0x140>(v));   // mirrored within 16
  if (LANES >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  if (LANES >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  return v;
}
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
  const uint64_t bits = (uint64_t)__double_as_longlong(v);
  const uint32_t low = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)bits, CTRL, 0xf, 0xf, true);
  const uint32_t high = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(bits >> 32), CTRL, 0xf, 0xf, true);
  return __longlong_as_double((long long)((uint64_t)high << 32 | low));
}
template <int LANES, class Op>
__device__ __forceinline__ double over_lanes(double v, const Op& op) {
  v = op(v, dpp<0xB1>(v));
  if (LANES >= 4) v = op(v, dpp<0x4E>(v));
  if (LANES >= 8) v = op(v, dpp<0x141>(v));
  if (LANES >= 16) v = op(v, dpp<0x140>(v));
#pragma unroll
  for (int m = 16; m < LANES; m <<= 1) v = op(v, __shfl_xor(v, m));
  return v;
}
template <int CTRL>
__device__ __forceinline__ int dpp(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true);
}
template <int LANES, class Op>
__device__ __forceinline__ int over_lanes(int v, const Op& op) {
  v = op(v, dpp<0xB1>(v));
  if (LANES >= 4) v = op(v, dpp<0x4E>(v));
  if (LANES >= 8) v = op(v, dpp<0x141>(v));
  if (LANES >= 16) v = op(v, dpp<0x140>(v));
  if (LANES >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
    v = op((int)r[0], (int)r[1]);
  }
  if (LANES >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
    v = op((int)r[0], (int)r[1]);
  }
  return v;
}
struct Max {
  __device__ __forceinline__ int operator()(int a, int b) const { return a > b ? a : b; }
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
  __device__ __forceinline__ double operator()(double a, double b) const { return fmax(a, b); }
};
struct Sum {
  template <typename V>
  __device__ __forceinline__ V operator()(V a, V b) const { return a + b; }
};

// Which of the row's lanes say yes: bit i is its lane i.
template <int LANES>
__device__ __forceinline__ uint64_t row_ballot(bool yes) {
  const uint64_t all = __ballot(yes);
  return LANES == 64 ? all : (all >> ((threadIdx.x & 63) / LANES * LANES)) & ((1ull << (LANES & 63)) - 1);
}

template <typename V>
__device__ __forceinline__ V lowest() {
  return -(V)INFINITY;
}

// f32 values as whole numbers of the same order, equal where they are equal: a maximum of two is one instruction, where one of floats
// is two or three that see to NaN.  And back.
__device__ __forceinline__ int key_of(float v) {
  const int bits = __float_as_int(v + 0.0f);  // (-0 becomes 0)
  return bits ^ ((bits >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float value_of(int key) { return __int_as_float(key ^ ((key >> 31) & 0x7fffffff)); }
__device__ __forceinline__ double key_of(double v) { return v; }
__device__ __forceinline__ double value_of(double v) { return v; }
template <>
__device__ __forceinline__ int lowest<int>() {
  return (int)0x807fffff;  // of minus infinity
}

// The exponential of a value at or below 0; of a masked logit 0.  inf - inf counts as 0: the largest logit's is 1.
__device__ __forceinline__ float exp_below(float l, float top) { return l == top ? 1.0f : expf(l - top); }
__device__ __forceinline__ double exp_below(double l, double top) { return l == top ? 1.0 : exp(l - top); }

// The same for choice values in f32, whose errors are allowed for: by the exponential instruction, off by |x| 2^-24 of its result.
__device__ __forceinline__ float quick_below(float l, float top) { return l == top ? 1.0f : __expf(l - top); }
__device__ __forceinline__ double quick_below(double l, double top) { return exp_below(l, top); }

__device__ __forceinline__ float sigmoid(float l) { return 1.0f / (1.0f + expf(-l)); }
__device__ __forceinline__ double sigmoid(double l) { return 1.0 / (1.0 + exp(-l)); }
__device__ __forceinline__ float quick_sigmoid(float l) { return __builtin_amdgcn_rcpf(1.0f + __expf(-l)); }
__device__ __forceinline__ double quick_sigmoid(double l) { return sigmoid(l); }

// The largest of the row's values, and its first column, which is taken out; false if only masked ones are left.
template <typename V, int LANES, int PER>
__device__ __forceinline__ bool take_largest(V (&v)[PER], V* value, int* column) {
  V mine = v[0];
#pragma unroll
  for (int i = 1; i < PER; ++i) mine = Max{}(mine, v[i]);
  const V top = over_lanes<LANES>(mine, Max{});
  const bool any = top > lowest<V>();
  const uint64_t who = row_ballot<LANES>(mine == top);
  const int lane = threadIdx.x & (LANES - 1), first = __ffsll((unsigned long long)who) - 1;
  int at = 0;
#pragma unroll
  for (int i = PER - 1; i >= 0; --i) at = v[i] == top ? i : at;
  const int out = any && lane == first ? at : -1;
#pragma unroll
  for (int i = 0; i < PER; ++i) v[i] = i == out ? lowest<V>() : v[i];
  *value = top;
  *column = first * PER + __shfl(at, first, LANES);
  return any;
}

// What a group's value may be off by, for a value that is one or one + two (two: lowest() if there is none): each is off by tol and by
// 2^-23 of its own size, which may be any multiple of their sum's where they cancel.
template <typename V>
__device__ __forceinline__ V group_error(V one, V two, V tol) {
  return tol + (V)0x1p-22 * (fabs(one) + (two > lowest<V>() ? fabs(two) : (V)0));
}
// A group's value.  Two lowest values, as leaves are closed with, add up to minus infinity in f32, which is a group without a leaf: such a
// one has the lowest number, which its value is below, an error without end, and 64 bits tell it from its like.
template <typename V>
__device__ __forceinline__ V group_value(V one, V two) {
  if (!(two > lowest<V>())) return one;
  const V sum = one + two;
  return sum > lowest<V>() ? sum : -(V)__FLT_MAX__;
}
// The border between groups: `least` the least that the values of kept ones can be, `next` the most that the others' can.
template <typename V>
struct Border {
  V least = (V)INFINITY, next = lowest<V>();
  __device__ __forceinline__ void add(bool kept, V worth, V error) {
    const bool any = error < (V)INFINITY, closed = worth <= -(V)__FLT_MAX__;  // (values whose sum leaves the numbers otherwise are anywhere)
    const V low = any ? worth - error : lowest<V>(), high = any ? worth + error : closed ? worth : (V)INFINITY;
    if (kept) {
      least = low < least ? low : least;
    } else {
      next = high > next ? high : next;
    }
  }
  template <int LANES>
  __device__ __forceinline__ bool close() const {
    const V low = -over_lanes<LANES>(-least, Max{}), high = over_lanes<LANES>(next, Max{});
    return high > lowest<V>() && !(low > high);
  }
};

// Values of all but the best groups become masked.  True if the border is closer than the values' errors say.
template <typename V, int LANES, int PER>
__device__ __forceinline__ bool keep_groups(const RouteArgs& g, V (&v)[PER], V tol) {
  const int lane = threadIdx.x & (LANES - 1);
  const int lanes = g.group_size / PER;
  if (lanes >= 1 && lanes * PER == g.group_size && (lanes & (lanes - 1)) == 0) {
    // a group is `lanes` neighbouring lanes: the two largest of all groups at once
    V one = lowest<V>(), two = lowest<V>();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      two = Max{}(two, v[i] < one ? v[i] : one);
      one = Max{}(one, v[i]);
    }
    for (int m = 1; m < lanes; m <<= 1) {
      const V other = __shfl_xor(one, m), next = __shfl_xor(two, m);
      const V lower = other < one ? other : one;
      two = Max{}(Max{}(two, next), lower);
      one = Max{}(one, other);
    }
    if (g.group_best == 1) two = lowest<V>();
    const V worth = group_value(one, two);
    const int mine = lane / lanes;
    int before = 0;  // groups that come before this lane's
    for (int q = 0; q < g.n_groups; ++q) {
      const V other = __shfl(worth, q * lanes, LANES);
      before += other > worth || (other == worth && q < mine) ? 1 : 0;
    }
    const bool group = mine < g.n_groups, kept = group && before < g.groups_kept && worth > lowest<V>();
    Border<V> border;
    if (group && worth > lowest<V>()) border.add(kept, worth, group_error(one, two, tol));
#pragma unroll
    for (int i = 0; i < PER; ++i) v[i] = kept ? v[i] : lowest<V>();
    return border.template close<LANES>();
  }
  // groups of any size, one after another; lane q mod LANES keeps group q's value
  constexpr int most = (kMaxGroups + LANES - 1) / LANES;
  V mine[most], left[most], error[most];  // values, those not yet taken, errors
  int group[PER];
#pragma unroll
  for (int t = 0; t < most; ++t) mine[t] = error[t] = lowest<V>();
#pragma unroll
  for (int i = 0; i < PER; ++i) group[i] = (lane * PER + i) / g.group_size;
  for (int q = 0; q < g.n_groups; ++q) {
    V in[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) in[i] = group[i] == q ? v[i] : lowest<V>();
    V one = lowest<V>(), two = lowest<V>();
    int column;
    if (take_largest<V, LANES, PER>(in, &one, &column) && g.group_best == 2) take_largest<V, LANES, PER>(in, &two, &column);
    const V worth = group_value(one, two), off = group_error(one, two, tol);
#pragma unroll
    for (int t = 0; t < most; ++t)
      if (lane + t * LANES == q) mine[t] = worth, error[t] = off;
  }
  uint64_t kept = 0;
#pragma unroll
  for (int t = 0; t < most; ++t) left[t] = mine[t];
  for (int r = 0; r < g.groups_kept; ++r) {
    V top = left[0];
#pragma unroll
    for (int t = 1; t < most; ++t) top = Max{}(top, left[t]);
    top = over_lanes<LANES>(top, Max{});
    int who = kMaxGroups;
#pragma unroll
    for (int t = most - 1; t >= 0; --t) {
      const uint64_t w = row_ballot<LANES>(left[t] == top);
      if (w) who = t * LANES + __ffsll((unsigned long long)w) - 1;
    }
    if (top > lowest<V>()) {
      kept |= 1ull << who;
#pragma unroll
      for (int t = 0; t < most; ++t)
        if (lane + t * LANES == who) left[t] = lowest<V>();
    }
  }
  Border<V> border;
#pragma unroll
  for (int t = 0; t < most; ++t)
    if (mine[t] > lowest<V>()) border.add(kept >> (lane + t * LANES) & 1, mine[t], error[t]);
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (!(group[i] < g.n_groups && kept >> group[i] & 1)) v[i] = lowest<V>();
  return border.template close<LANES>();
}

// Slots of a row's k chosen leaves: lane i has the slots i, i + LANES, ..
template <int LANES>
constexpr int kSlotsOf = (kMaxChosen + LANES - 1) / LANES;

// The k columns of the largest values, -1 where fewer are left.  check: true if two of the first k + 1 are closer than their errors, tol of
// each and 2^-23 of its size.
template <typename V, int LANES, int PER>
__device__ __forceinline__ bool choose(const RouteArgs& g, V (&v)[PER], V tol, bool check, int (&picked)[kSlotsOf<LANES>]) {
  bool close = false;
  const int lane = threadIdx.x & (LANES - 1), more = check && g.k < g.n_leaves ? 1 : 0;
  typedef decltype(key_of(V())) Key;
  Key keys[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) keys[i] = key_of(v[i]);
  V before = lowest<V>();
#pragma unroll
  for (int t = 0; t < kSlotsOf<LANES>; ++t) picked[t] = -1;
  for (int j = 0; j < g.k + more; ++j) {
    Key key;
    int column;
    const bool any = take_largest<Key, LANES, PER>(keys, &key, &column);
    if (check) {
      const V top = value_of(key);
      if (any && j > 0) close |= !(before - top > tol + (V)0x1p-22 * fabs(before));
      before = top;
    }
#pragma unroll
    for (int t = 0; t < kSlotsOf<LANES>; ++t)
      if (lane + t * LANES == j) picked[t] = any ? column : -1;
  }
  return close;
}

// A lane's PER neighbouring logits; masked ones (NaN, minus infinity, past the end) are minus infinity.
template <typename T, int PER>
__device__ __forceinline__ void load_logits(const T* row, int column, int n, float (&l)[PER]) {
  T t[PER];
  if (row != nullptr && column + PER <= n) {
    __builtin_memcpy(t, row + column, sizeof t);
#pragma unroll
    for (int i = 0; i < PER; ++i) l[i] = (float)t[i];
  } else if (row != nullptr) {  // (loads without a branch each, which would be waited for one by one)
#pragma unroll
    for (int i = 0; i < PER; ++i) t[i] = row[column + i < n ? column + i : n - 1];
#pragma unroll
    for (int i = 0; i < PER; ++i) l[i] = column + i < n ? (float)t[i] : -INFINITY;
  } else {
#pragma unroll
    for (int i = 0; i < PER; ++i) l[i] = -INFINITY;
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) l[i] = l[i] == l[i] ? l[i] : -INFINITY;
}

// A row's choice values; *tol: the most that the difference of two may be off by in f32 beside 2^-23 of their sizes (the bias' sum).  In u = 2^-24,
// for x = |l| or top - l:
//   sigmoid   the exponential: its argument's roundings, 1.5 x u, and 2 u of the instruction, times s (1 - s): 0.9 u; 1 + it and the
//             reciprocal, 3 u.  Twice that: 8 u, of 16.
//   softmax   all divide by the same sum, so its error counts once, times a difference of scores, at most the largest score 1 / sum: 36
//             additions and the reciprocal 37 u, the exponentials (2.5 x + 2) u each, on average over their own sizes 14 u, since a
//             softmax of 1,024 has an average x below 4.5; the two scores' own, 2.5 x exp(-x) + 3, twice 4 u.  59 u of the largest score, of 64.
// (A group's value is two of them, and allowed for as much again.)
template <typename V, int LANES, int PER>
__device__ __forceinline__ void choice_values(const RouteArgs& g, const float (&l)[PER], float top, V (&v)[PER], V* tol) {
  const int lane = threadIdx.x & (LANES - 1);
  float bias[PER];  // (one that is NaN closes its leaf, as minus infinity does)
#pragma unroll
  for (int i = 0; i < PER; ++i) bias[i] = 0.0f;
  if (g.bias != nullptr) load_logits<float, PER>(g.bias, lane * PER, g.n_leaves, bias);
  V inverse = 1;
  if (!g.sigmoid) {
    V sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      v[i] = l[i] > -INFINITY ? quick_below((V)l[i], (V)top) : (V)0;
      sum += v[i];
    }
    inverse = 1 / over_lanes<LANES>(sum, Sum{});
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const V c = (g.sigmoid ? quick_sigmoid((V)l[i]) : v[i] * inverse) + (V)bias[i];
    v[i] = l[i] > -INFINITY && c == c ? c : lowest<V>();
  }
  *tol = g.sigmoid ? (V)0x1p-20 : (V)0x1p-18 * inverse;
}

// Without a bias, leaves of the groups that their values keep go by their logits, as they do without groups: scores may be equal where
// logits are not.  (Read again: few lanes have room for both.)
template <typename T, typename V, int PER>
__device__ __forceinline__ void logits_for_values(const T* row, int column, int n, V (&v)[PER]) {
  float l[PER];
  load_logits<T, PER>(row, column, n, l);
#pragma unroll
  for (int i = 0; i < PER; ++i) v[i] = v[i] > lowest<V>() ? (V)l[i] : lowest<V>();
}

// exp(l - c) / (1 + exp(l)) for l < 0, its limit for the others (whose c is 0): the sigmoid over exp(c), which renormalised
// weights leave out, so that they hold however small all scores are.
__device__ __forceinline__ float sigmoid_over(float l, float c) { return l >= 0.0f ? sigmoid(l) : expf(l - c) / (1.0f + expf(l)); }

// k slots of a row, lane i the slots i, i + LANES, ..; scores of the chosen, renormalised or not, without scale.
template <int LANES>
struct Slots {
  static constexpr int kMost = kSlotsOf<LANES>;
  int column[kMost];
  float logit[kMost], score[kMost];
  // f(column): the logit, minus infinity for a masked one
  template <class F>
  __device__ __forceinline__ void read(const RouteArgs& g, const int (&picked)[kMost], const F& f) {
    const int lane = threadIdx.x & (LANES - 1);
#pragma unroll
    for (int t = 0; t < kMost; ++t) {
      column[t] = lane + t * LANES < g.k ? picked[t] : -1;
      logit[t] = column[t] >= 0 ? f(column[t]) : -INFINITY;
    }
  }
  // top, inverse: of all logits, for a softmax that is not renormalised
  __device__ __forceinline__ void scores(const RouteArgs& g, float top, float inverse) {
    if (!g.renormalise) {
#pragma unroll
      for (int t = 0; t < kMost; ++t)
        score[t] = !(logit[t] > -INFINITY) ? 0.0f : g.sigmoid ? sigmoid(logit[t]) : exp_below(logit[t], top) * inverse;
      return;
    }
    float best = logit[0];
#pragma unroll
    for (int t = 1; t < kMost; ++t) best = fmaxf(best, logit[t]);
    best = over_lanes<LANES>(best, Max{});
    float sum = 0.0f;
#pragma unroll
    for (int t = 0; t < kMost; ++t) {
      score[t] = !(logit[t] > -INFINITY) ? 0.0f : g.sigmoid ? sigmoid_over(logit[t], fminf(best, 0.0f)) : exp_below(logit[t], best);
      sum += score[t];
    }
    sum = over_lanes<LANES>(sum, Sum{});
#pragma unroll
    for (int t = 0; t < kMost; ++t) score[t] = sum > 0.0f ? score[t] / sum : 0.0f;
  }
};

// Bound by reading the logits where rows are many and k is small: 400,000 x 255 f32, four leaves each, 107 us a call among others, 3.9 TB/s (115
// by itself under a profiler).  A pick is some 130 instructions for four rows of 256 columns: 16,384 x 256 bf16 in 8 groups, 8 leaves each by
// values, 17 to 19 us, 12 of it nine picks, 4 the few rows that 64 bits decide, which end last; 65,536 x 64 f32, four leaves each by values, 14 us.
// VALUES: leaves (without a bias: their groups) are chosen by their values, not by the logits themselves.
// (At most 128 registers.  From 24 columns a lane on by values, more would be taken, most of them on the 64-bit path, and some are kept
// in memory; even so, 100,000 rows f32, 16 leaves each by values: x 285 135 us against 149 with as many as it takes, x 512 187 against 258, x
// 700 274 against 375, x 1,024 316 against 767.)
template <typename T, int LANES, int PER, bool VALUES>
__global__ void __launch_bounds__(kThreads, 4) route_kernel(const RouteArgs g) {
  constexpr int rows = kThreads / LANES;
  const int r = threadIdx.x / LANES, lane = threadIdx.x & (LANES - 1);
  const int64_t d = g.first + (int64_t)blockIdx.x * rows + r;
  const T* row = d < g.n_rows ? (const T*)g.logits + d * g.ld : nullptr;
  int picked[kSlotsOf<LANES>];
  float top, inverse = 0.0f;
  {
    float l[PER];
    load_logits<T, PER>(row, lane * PER, g.n_leaves, l);
    top = l[0];
#pragma unroll
    for (int i = 1; i < PER; ++i) top = fmaxf(top, l[i]);
    top = over_lanes<LANES>(top, Max{});
    if (!g.sigmoid && !g.renormalise) {
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < PER; ++i) sum += l[i] > -INFINITY ? exp_below(l[i], top) : 0.0f;
      inverse = 1.0f / over_lanes<LANES>(sum, Sum{});
    }
    if constexpr (!VALUES) {
      if (g.n_groups > 1) keep_groups<float, LANES, PER>(g, l, 0.0f);
      choose<float, LANES, PER>(g, l, 0.0f, false, picked);
    } else {
      float v[PER], tol;
      choice_values<float, LANES, PER>(g, l, top, v, &tol);
      bool close = g.n_groups > 1 && keep_groups<float, LANES, PER>(g, v, tol);
      const bool by_values = g.bias != nullptr;
      if (!by_values) logits_for_values<T, float, PER>(row, lane * PER, g.n_leaves, v);
      close |= choose<float, LANES, PER>(g, v, tol, by_values, picked);
      // rows to be taken again, all 64 lanes a row
      constexpr int wide = (LANES * PER + 63) / 64;
      uint64_t again = __ballot(close && lane == 0);
      while (again) {
        const int from = __ffsll((unsigned long long)again) - 1;
        again &= again - 1;
        const int64_t other = g.first + (int64_t)blockIdx.x * rows + ((threadIdx.x & ~63) + from) / LANES;
        float logits[wide], most;
        load_logits<T, wide>((const T*)g.logits + other * g.ld, (threadIdx.x & 63) * wide, g.n_leaves, logits);
        most = logits[0];
#pragma unroll
        for (int i = 1; i < wide; ++i) most = fmaxf(most, logits[i]);
        most = over_lanes<64>(most, Max{});
        double exact[wide], none;
        choice_values<double, 64, wide>(g, logits, most, exact, &none);
        int chosen[kSlotsOf<64>];
        if (g.n_groups > 1) keep_groups<double, 64, wide>(g, exact, none);
        if (!by_values) logits_for_values<T, double, wide>((const T*)g.logits + other * g.ld, (threadIdx.x & 63) * wide, g.n_leaves, exact);
        choose<double, 64, wide>(g, exact, none, false, chosen);
#pragma unroll
        for (int t = 0; t < kSlotsOf<LANES>; ++t) {
          const int e = __shfl(chosen[0], lane + t * LANES);
          if ((int)(threadIdx.x & 63) / LANES == from / LANES) picked[t] = e;
        }
      }
    }
  }
  Slots<LANES> s;
  s.read(g, picked, [&](int e) { return (float)row[e]; });
  s.scores(g, top, inverse);
  if (row == nullptr) return;
#pragma unroll
  for (int t = 0; t < Slots<LANES>::kMost; ++t) {
    const int j = lane + t * LANES;
    if (j >= g.k) break;
    g.leaves[d * g.k + j] = s.column[t];
    g.gates[d * g.k + j] = g.scale * s.score[t];
  }
}

// With s the score and r the share of a slot:
//   softmax, renormalised   scale r (dg - sum r dg) at the slot's leaf
//   softmax                 scale s ([chosen] dg - sum s dg) at every leaf
//   sigmoid, renormalised   scale r (1 - s) (dg - sum r dg) at the slot's leaf
//   sigmoid                 scale s (1 - s) dg at the slot's leaf
// and zeros elsewhere.  Bound by writing the gradients and, for the second, reading the logits: 65,536 x 64 f32, 11 us, 3.0 TB/s.
template <typename T, int LANES, int PER>
__global__ void __launch_bounds__(kThreads) route_grad_kernel(const RouteArgs g) {
  constexpr int rows = kThreads / LANES;
  const int r = threadIdx.x / LANES, lane = threadIdx.x & (LANES - 1);
  const int64_t d = g.first + (int64_t)blockIdx.x * rows + r;
  const T* row = d < g.n_rows ? (const T*)g.logits + d * g.ld : nullptr;
  int picked[kSlotsOf<LANES>];
#pragma unroll
  for (int t = 0; t < kSlotsOf<LANES>; ++t) {
    const int j = lane + t * LANES, e = row != nullptr && j < g.k ? g.leaves[d * g.k + j] : -1;
    picked[t] = (uint32_t)e < (uint32_t)g.n_leaves ? e : -1;
  }
  const bool all = !g.sigmoid && !g.renormalise;
  float p[PER], top = 0.0f, inverse = 0.0f;
#pragma unroll
  for (int i = 0; i < PER; ++i) p[i] = 0.0f;
  if (all) {
    float l[PER];
    load_logits<T, PER>(row, lane * PER, g.n_leaves, l);
    top = l[0];
#pragma unroll
    for (int i = 1; i < PER; ++i) top = fmaxf(top, l[i]);
    top = over_lanes<LANES>(top, Max{});
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      p[i] = l[i] > -INFINITY ? exp_below(l[i], top) : 0.0f;
      sum += p[i];
    }
    sum = over_lanes<LANES>(sum, Sum{});
    inverse = sum > 0.0f ? 1.0f / sum : 0.0f;
  }
  Slots<LANES> s;
  s.read(g, picked, [&](int e) {
    const float l = (float)row[e];
    return l == l ? l : -INFINITY;
  });
  s.scores(g, top, inverse);
  float dg[Slots<LANES>::kMost], inner = 0.0f;
#pragma unroll
  for (int t = 0; t < Slots<LANES>::kMost; ++t) {
    dg[t] = s.logit[t] > -INFINITY ? g.dgates[d * g.k + lane + t * LANES] : 0.0f;
    inner += s.score[t] * dg[t];
  }
  inner = over_lanes<LANES>(inner, Sum{});
  float each[Slots<LANES>::kMost];
#pragma unroll
  for (int t = 0; t < Slots<LANES>::kMost; ++t) {
    float v = g.scale * s.score[t] * (g.renormalise ? dg[t] - inner : dg[t]);
    if (g.sigmoid) v *= sigmoid(-s.logit[t]);
    each[t] = s.logit[t] > -INFINITY ? v : 0.0f;
  }
  float out[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) out[i] = all ? -g.scale * (p[i] * inverse) * inner : 0.0f;
#pragma unroll
  for (int t = 0; t < Slots<LANES>::kMost; ++t)
    for (int j = 0; j < LANES && j + t * LANES < g.k; ++j) {
      const int at = __shfl(s.column[t], j, LANES) - lane * PER;
      const float v = __shfl(each[t], j, LANES);
#pragma unroll
      for (int i = 0; i < PER; ++i) out[i] += at == i ? v : 0.0f;
    }
  if (row == nullptr) return;
  T* to = (T*)g.dlogits + d * g.ld_out + lane * PER;
  T t[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) t[i] = (T)out[i];
  const int left = g.n_leaves - lane * PER;
  if (left >= PER) {
    __builtin_memcpy(to, t, sizeof t);
  } else {
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (i < left) to[i] = t[i];
  }
}

// ---------------------------------------------------------------- lists of rows by leaf

// Pairs p = row * k + slot, grouped by leaf, ascending within one: what the products take.  Pairs whose leaf is none are in no
// list.  A wavefront counts a run of neighbouring pairs in local memory, a table of its own for all leaves; sums over the runs give
// each its places, and it goes through its pairs again.  No order hangs on which ran first.  Three launches of 5 us each, whose lengths
// are those of a launch and a chain of two or three round trips (65,536 pairs, 64 leaves); one of 3.5 us for 256 pairs.
struct ListArgs {
  const int32_t* leaves;   // [n_pairs]
  int64_t* offsets;        // [n_leaves + 1]
  int32_t* row;            // [n_pairs] of each position
  int32_t* pair;           // [n_pairs]
  int32_t* counts;         // [n_leaves][runs], then the first places within the leaf
  int32_t* totals;         // [n_leaves]
  int32_t n_pairs, n_leaves, k, run, runs;  // run: pairs, a multiple of 64
};

constexpr int kListWaves = 16;             // of the one workgroup that lists few pairs
constexpr int kFewListLeaves = 1024;       // it takes that many leaves
constexpr int kMaxListLeaves = 16384;

// The leaves of kAhead x 64 pairs at once (-1: none), since each load would be waited for otherwise.
constexpr int kAhead = 8;
__device__ __forceinline__ void load_leaves(const ListArgs& g, int first, int end, int (&e)[kAhead]) {
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    const int p = first + i * 64 + (int)(threadIdx.x & 63);
    e[i] = p < end ? g.leaves[p] : -1;
  }
#pragma unroll
  for (int i = 0; i < kAhead; ++i) e[i] = (uint32_t)e[i] < (uint32_t)g.n_leaves ? e[i] : -1;
}

// Adds the run's pairs to a table.
__device__ __forceinline__ void count_run(const ListArgs& g, int first, int end, int* table) {
  for (int p = first; p < end; p += 64 * kAhead) {
    int e[kAhead];
    load_leaves(g, p, end, e);
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (e[i] >= 0) __hip_atomic_fetch_add(&table[e[i]], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  }
}

// Puts the run's pairs to the places that the table has for them, in order.
__device__ __forceinline__ void place_run(const ListArgs& g, int first, int end, int* table) {
  const int lane = threadIdx.x & 63, bits = 32 - __clz(g.n_leaves);
  const uint64_t below = (1ull << lane) - 1;
  int next[kAhead];
  load_leaves(g, first, end, next);
  for (int p0 = first; p0 < end; p0 += 64 * kAhead) {
    int leaves[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) leaves[i] = next[i];
    if (p0 + 64 * kAhead < end) load_leaves(g, p0 + 64 * kAhead, end, next);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (p0 + i * 64 >= end) break;
      const int p = p0 + i * 64 + lane, e = leaves[i];
      uint64_t same = __ballot(e >= 0);
      for (int b = 0; b < bits; ++b) {
        const uint64_t ones = __ballot(e >> b & 1);
        same &= e >> b & 1 ? ones : ~ones;
      }
      if (e >= 0) {
        const int at = table[e];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if ((same >> lane) == 1) table[e] = at + __popcll(same);  // the last of them
        const int to = at + __popcll(same & below);
        g.row[to] = p / g.k;
        g.pair[to] = p;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  }
}

// Sum over the lanes before this one; *all: over all lanes.
__device__ __forceinline__ int before_lane(int v, int* all) {
  const int lane = threadIdx.x & 63;
  int sum = v;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int other = __shfl_up(sum, m);
    if (lane >= m) sum += other;
  }
  *all = __shfl(sum, 63);
  return sum - v;
}

__global__ void __launch_bounds__(kListWaves * 64) list_few_kernel(const ListArgs g) {
  __shared__ int table[kListWaves][kFewListLeaves];
  __shared__ int sums[kListWaves];
  const int t = threadIdx.x, w = t >> 6;
  for (int i = t & 63; i < g.n_leaves; i += 64) table[w][i] = 0;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  const int first = w * g.run < g.n_pairs ? w * g.run : g.n_pairs;
  const int end = first + g.run < g.n_pairs ? first + g.run : g.n_pairs;
  count_run(g, first, end, table[w]);
  __syncthreads();
  static_assert(kListWaves * 64 >= kFewListLeaves, "a thread a leaf");
  int total = 0;
  if (t < g.n_leaves)
    for (int i = 0; i < kListWaves; ++i) {
      const int n = table[i][t];
      table[i][t] = total;
      total += n;
    }
  int wave_total;
  int at = before_lane(total, &wave_total);
  if ((t & 63) == 0) sums[w] = wave_total;
  __syncthreads();
  for (int i = 0; i < w; ++i) at += sums[i];
  if (t < g.n_leaves) {
    g.offsets[t] = at;
    if (t == g.n_leaves - 1) g.offsets[g.n_leaves] = at + total;
    for (int i = 0; i < kListWaves; ++i) table[i][t] += at;
  }
  __syncthreads();
  place_run(g, first, end, table[w]);
}

// Many pairs: a wavefront a workgroup and run.
template <int LEAVES>
__global__ void __launch_bounds__(64) list_count_kernel(const ListArgs g) {
  __shared__ int table[LEAVES];
  for (int i = threadIdx.x; i < g.n_leaves; i += 64) table[i] = 0;
  __syncthreads();
  const int first = (int)blockIdx.x * g.run, end = g.n_pairs - first < g.run ? g.n_pairs : first + g.run;
  count_run(g, first, end, table);
  __syncthreads();
  for (int i = threadIdx.x; i < g.n_leaves; i += 64) g.counts[(int64_t)i * g.runs + blockIdx.x] = table[i];
}

// A leaf a workgroup: its counts become sums of those before.
__global__ void __launch_bounds__(64) list_scan_kernel(const ListArgs g) {
  int32_t* counts = g.counts + (int64_t)blockIdx.x * g.runs;
  int base = 0;
  for (int i0 = 0; i0 < g.runs; i0 += 64) {
    const int i = i0 + threadIdx.x, n = i < g.runs ? counts[i] : 0;
    int all;
    const int at = before_lane(n, &all);
    if (i < g.runs) counts[i] = base + at;
    base += all;
  }
  if (threadIdx.x == 0) g.totals[blockIdx.x] = base;
}

template <int LEAVES>
__global__ void __launch_bounds__(64) list_place_kernel(const ListArgs g) {
  __shared__ int table[LEAVES];
  int base = 0;
  for (int i0 = 0; i0 < g.n_leaves; i0 += 64) {
    const int i = i0 + threadIdx.x, n = i < g.n_leaves ? g.totals[i] : 0;
    int all;
    const int at = base + before_lane(n, &all);
    if (i < g.n_leaves) {
      table[i] = at + g.counts[(int64_t)i * g.runs + blockIdx.x];
      if (blockIdx.x == 0) g.offsets[i] = at;
    }
    base += all;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) g.offsets[g.n_leaves] = base;
  __syncthreads();
  const int first = (int)blockIdx.x * g.run, end = g.n_pairs - first < g.run ? g.n_pairs : first + g.run;
  place_run(g, first, end, table);
}

}  // namespace gbdt_router
