// One workgroup's tile of a matrix product on the matrix cores, for operands of either orientation.
//
//   acc[m][n] = sum_k A(m, k) * B(n, k)
//
// An operand whose k runs along memory ("row operand": its rows are m or n) is staged as rows of 128 bytes of k; one whose
// m or n runs along memory ("column operand": its rows are k) is staged as it lies, and turned while it is read: 16-bit
// values by ds_read_b64_tr_b16 (the 16 lanes of a group address four k rows of 16 values and each lane receives one
// column's four), 32-bit values by single-word reads.  So none of the products of a linear layer (values, gradient of the
// input, gradient of the weights) needs a transposed copy of anything.
//
// A step takes 128 bytes of k (64 bf16, 32 f32): R x 128 bytes of an operand of R rows, in chunks of 16 bytes.  Chunk s of
// the stage (thread s mod NT) lies at byte 16 s.  Within a row operand's row the chunks are permuted by the row's low
// three bits, within a column operand's row by bits of k, so that the lanes of one fragment read spread over the banks.
// Rows are found through functors that return a row's address or null; null rows and values past a limit are zeros.
// There are two stages: the next step's chunks travel while the present one is multiplied.
//   DIRECT: chunks go from memory to the stage without registers (every row 16-byte aligned, limits whole chunks).
//   otherwise: through registers, by unaligned 16-byte loads, and value by value where a limit cuts a chunk.
// Products of bf16 values are exact in f32 and sums are f32 throughout; f32 operands use the f32 matrix instruction.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace gbdt_tile {

typedef __bf16 bf16;
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kStepBytes = 128;  // of k, per staged row

template <typename T> struct Traits;
template <> struct Traits<bf16> {
  typedef bf16x8 Frag;
};
template <> struct Traits<float> {
  typedef f32x4 Frag;
};
template <typename T> constexpr int kChunk = 16 / (int)sizeof(T);       // values a chunk
template <typename T> constexpr int kStep = kStepBytes / (int)sizeof(T);  // k a step

// 16 zero bytes in device memory: what a masked lane of a DIRECT load reads.
static __device__ __align__(16) const uint32_t zero_chunk[4] = {0, 0, 0, 0};

template <typename T>
__device__ __forceinline__ u32x4 load_chunk(const T* p, int valid) {
  u32x4 v = {0, 0, 0, 0};
  if (p == nullptr || valid <= 0) return v;
  if (valid >= kChunk<T>) {
    __builtin_memcpy(&v, p, 16);  // any alignment
    return v;
  }
  T part[kChunk<T>];
#pragma unroll
  for (int i = 0; i < kChunk<T>; ++i) part[i] = i < valid ? p[i] : (T)0.0f;
  __builtin_memcpy(&v, part, 16);
  return v;
}

__device__ __forceinline__ void direct_chunk(const void* src, char* lds_wave_base) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                   (__attribute__((address_space(3))) void*)lds_wave_base, 16, 0, 0);
}

// How the 16-byte chunks of a column operand's row k are permuted (R columns a row).
template <typename T, int R>
__device__ __forceinline__ int column_swizzle(int k) {
  constexpr int chunks = R / kChunk<T>;
  if (sizeof(T) == 2) return (((k & 3) | ((k >> 1) & 4)) << 1) & (chunks - 1);
  return (((k >> 2) & 3) << 2) & (chunks - 1);
}

// ---------------------------------------------------------------- operands

// Rows are m or n, k along memory.  rows(r): address of row r (k = 0), or null.
template <typename T, int R, int NT, bool DIRECT>
struct RowOperand {
  static constexpr int kSlots = R * 8;
  static constexpr int kPer = (kSlots + NT - 1) / NT;
  static constexpr int kBytes = R * kStepBytes;
  static constexpr bool kColumns = false;
  static constexpr int kRows = R;
  const T* row[kPer];
  u32x4 reg[DIRECT ? 1 : kPer];
  int k_of, k_end;

  template <class Rows>
  __device__ __forceinline__ void init(const Rows& rows, int r0, int /*limit*/, int k0, int k1) {
    const int t = threadIdx.x;
    k_of = k0 + ((t & 7) ^ ((t >> 3) & 7)) * kChunk<T>;
    k_end = k1;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int s = i * NT + t;
      row[i] = s < kSlots ? rows(r0 + (s >> 3)) : nullptr;
    }
  }
  template <class Rows>
  __device__ __forceinline__ void load(const Rows&, char* stage) {
    const int t = threadIdx.x;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (kSlots % NT != 0 && i * NT + t >= kSlots) break;
      if constexpr (DIRECT) {
        const void* p = row[i] != nullptr && k_of < k_end ? (const void*)(row[i] + k_of) : (const void*)zero_chunk;
        direct_chunk(p, stage + (i * NT + (t & ~63)) * 16);
      } else {
        reg[i] = load_chunk<T>(row[i] == nullptr ? nullptr : row[i] + k_of, k_end - k_of);
      }
    }
    k_of += kStep<T>;
  }
  __device__ __forceinline__ void store(char* stage) {
    if constexpr (!DIRECT) {
      const int t = threadIdx.x;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (kSlots % NT != 0 && i * NT + t >= kSlots) break;
        *(u32x4*)(stage + (i * NT + t) * 16) = reg[i];
      }
    }
  }
  // Values of rows r0 .. r0 + 15 for the part'th half of the step: lane l holds row l mod 16; k as both operands order it.
  __device__ __forceinline__ static typename Traits<T>::Frag frag(const char* stage, int r0, int part) {
    const int l = threadIdx.x & 63;
    const int r = r0 + (l & 15);
    const int c = ((l >> 4) + 4 * part) ^ (r & 7);
    return *(const typename Traits<T>::Frag*)(stage + r * kStepBytes + c * 16);
  }
};

// Rows are k, m or n along memory.  rows(k): address of row k (column 0), or null.
template <typename T, int R, int NT, bool DIRECT>
struct ColumnOperand {
  static constexpr int kSlots = R * 8;
  static constexpr int kPer = (kSlots + NT - 1) / NT;
  static constexpr int kBytes = R * kStepBytes;
  static constexpr int kChunks = R / kChunk<T>;  // a row
  static constexpr bool kColumns = true;
  static constexpr int kRows = R;
  const T* row[kPer];  // of the step that is loaded next
  u32x4 reg[DIRECT ? 1 : kPer];
  int k_at, k_end, c0, lim;

  template <class Rows>
  __device__ __forceinline__ void find(const Rows& rows) {
    const int t = threadIdx.x;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int s = i * NT + t;
      const int k = k_at + s / kChunks;
      row[i] = s < kSlots && k < k_end ? rows(k) : nullptr;
    }
  }
  template <class Rows>
  __device__ __forceinline__ void init(const Rows& rows, int col0, int limit, int k0, int k1) {
    k_at = k0;
    k_end = k1;
    c0 = col0;
    lim = limit;
    find(rows);
  }
  template <class Rows>
  __device__ __forceinline__ void load(const Rows& rows, char* stage) {
    const int t = threadIdx.x;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int s = i * NT + t;
      if (kSlots % NT != 0 && s >= kSlots) break;
      const int c = c0 + ((s % kChunks) ^ column_swizzle<T, R>(s / kChunks)) * kChunk<T>;
      if constexpr (DIRECT) {
        const void* p = row[i] != nullptr && c < lim ? (const void*)(row[i] + c) : (const void*)zero_chunk;
        direct_chunk(p, stage + (i * NT + (t & ~63)) * 16);
      } else {
        reg[i] = load_chunk<T>(row[i] == nullptr ? nullptr : row[i] + c, lim - c);
      }
    }
    k_at += kStep<T>;
    find(rows);
  }
  __device__ __forceinline__ void store(char* stage) {
    if constexpr (!DIRECT) {
      const int t = threadIdx.x;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (kSlots % NT != 0 && i * NT + t >= kSlots) break;
        *(u32x4*)(stage + (i * NT + t) * 16) = reg[i];
      }
    }
  }
  __device__ __forceinline__ static typename Traits<T>::Frag frag(const char* stage, int r0, int part) {
    const int l = threadIdx.x & 63;
    constexpr int row_bytes = R * (int)sizeof(T);
    typename Traits<T>::Frag f;
    if constexpr (sizeof(T) == 2) {
      // lane j of a group of 16 addresses row j / 4, values 4 (j mod 4) .. + 3, and receives column j of the four rows
      const int j = l & 15;
      const int c = r0 / 8 + ((j & 3) >> 1);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = part * 32 + (l >> 4) * 8 + h * 4 + (j >> 2);
        const char* a = stage + k * row_bytes + (c ^ column_swizzle<T, R>(k)) * 16 + (j & 1) * 8;
        const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)a);
        __builtin_memcpy((char*)&f + h * 8, &v, 8);
      }
    } else {
      const int c = (r0 + (l & 15)) / 4, w = l & 3;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int k = part * 16 + (l >> 4) * 4 + i;
        f[i] = *(const float*)(stage + k * row_bytes + (c ^ column_swizzle<T, R>(k)) * 16 + w * 4);
      }
    }
    return f;
  }
};

__device__ __forceinline__ f32x4 mma(bf16x8 rows, bf16x8 cols, f32x4 acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(rows, cols, acc, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma(f32x4 rows, f32x4 cols, f32x4 acc) {
#pragma unroll
  for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(rows[i], cols[i], acc, 0, 0, 0);
  return acc;
}

// ---------------------------------------------------------------- the tile

// BM x BN values by WM x WN wavefronts.  A lane's four values of the 16 x 16 block (i, j) of its wavefront:
//   N_INNER: m = 16 i + lane mod 16, n = 16 j + 4 (lane / 16) + 0..3   (rows of an output along n)
//   else:    n = 16 j + lane mod 16, m = 16 i + 4 (lane / 16) + 0..3   (columns of an output along m)
template <typename T_, int BM_, int BN_, int WM_, int WN_, bool DIRECT_>
struct Shape {
  typedef T_ T;
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NT = WM_ * WN_ * 64;
  static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;
  static constexpr bool DIRECT = DIRECT_;
  static constexpr int kStageBytes = (BM + BN) * kStepBytes;
  static constexpr int kLdsBytes = 2 * kStageBytes;
  static_assert(TM >= 1 && TN >= 1 && BM % (WM * 16) == 0 && BN % (WN * 16) == 0, "whole 16 x 16 blocks");
};

template <class S, bool N_INNER, class A, class B, class RowsA, class RowsB, class Also>
__device__ __forceinline__ void tile_product(char* lds, A& a, B& b, const RowsA& rows_a, const RowsB& rows_b, int k0, int k1,
                                             f32x4 (&acc)[S::TM][S::TN], const Also& also) {
  typedef typename Traits<typename S::T>::Frag Frag;
  const int w = threadIdx.x >> 6;
  const int m0 = (w / S::WN) * (S::TM * 16), n0 = (w % S::WN) * (S::TN * 16);
#pragma unroll
  for (int i = 0; i < S::TM; ++i)
#pragma unroll
    for (int j = 0; j < S::TN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const int steps = (k1 - k0 + kStep<typename S::T> - 1) / kStep<typename S::T>;
  if (steps <= 0) return;

  auto multiply = [&](const char* stage) {
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      Frag fa[S::TM], fb[S::TN];
#pragma unroll
      for (int i = 0; i < S::TM; ++i) fa[i] = A::frag(stage, m0 + 16 * i, part);
#pragma unroll
      for (int j = 0; j < S::TN; ++j) fb[j] = B::frag(stage + A::kBytes, n0 + 16 * j, part);
#pragma unroll
      for (int i = 0; i < S::TM; ++i)
#pragma unroll
        for (int j = 0; j < S::TN; ++j)
          acc[i][j] = N_INNER ? mma(fb[j], fa[i], acc[i][j]) : mma(fa[i], fb[j], acc[i][j]);
      also(fa, fb);
    }
  };

  a.load(rows_a, lds);
  b.load(rows_b, lds + A::kBytes);
  if constexpr (!S::DIRECT) {
    a.store(lds);
    b.store(lds + A::kBytes);
  }
  for (int s = 0; s < steps; ++s) {
    char* here = lds + (s & 1) * S::kStageBytes;
    char* next = lds + ((s + 1) & 1) * S::kStageBytes;
    if constexpr (S::DIRECT) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wavefront's chunks have arrived
    __syncthreads();  // everyone's have, and everyone has read the other stage
    if (s + 1 < steps) {
      a.load(rows_a, next);
      b.load(rows_b, next + A::kBytes);
    }
    multiply(here);
    if constexpr (!S::DIRECT) {
      if (s + 1 < steps) {
        a.store(next);
        b.store(next + A::kBytes);
      }
    }
  }
}

struct Nothing {
  template <class FA, class FB>
  __device__ __forceinline__ void operator()(const FA&, const FB&) const {}
};

// ---------------------------------------------------------------- results

// Rounded once, to nearest even, where it leaves f32.
template <typename T>
__device__ __forceinline__ void store4(T* p, f32x4 v, int valid) {
  T t[4] = {(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
  if (valid >= 4) {
    __builtin_memcpy(p, t, sizeof t);
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < valid) p[i] = t[i];
  }
}

// Workgroups go to the eight XCDs in turn; this gives each XCD a run of neighbouring tiles, which share operands in its L2.
__device__ __forceinline__ uint32_t xcd_tile(uint32_t block, uint32_t blocks) {
  const uint32_t per = blocks / 8, extra = blocks % 8;
  const uint32_t x = block % 8, i = block / 8;
  return x * per + (x < extra ? x : extra) + i;
}

}  // namespace gbdt_tile
