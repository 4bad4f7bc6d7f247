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
// A step takes KB = 128 or 64 bytes of k: R x KB bytes of an operand of R rows, in chunks of 16 bytes.  Chunk s of the stage
// (thread s mod NT) lies at byte 16 s.  Within a row operand's row the chunks are permuted by bits of the row, within a
// column operand's row by bits of k, so that the lanes of one fragment read spread over the banks.
// Rows are found through functors: fetch(r) reads what the row's place hangs on (its id in a list, its label), at(r, that)
// is its address or null.  Null rows and values past a limit are zeros.  A column operand fetches a step ahead, so that the
// address of a gathered row does not wait for its id.
// There are several stages: the next steps' chunks travel while the present one is multiplied.
//   DIRECT: chunks go from memory to the stage without registers (every row 16-byte aligned, limits whole chunks).  A lane
//   whose chunk is all zeros writes them itself; a row or column past its limit is any other, because what it yields is
//   past the result's limit as well and is not stored.
//   otherwise: through registers, by 16-byte loads of any alignment.  A chunk that a limit cuts is read whole, into the next
//   row, and masked on its way to the stage; only where that would pass the matrix's end is it read value by value, behind
//   the other loads (a branch among them made every load wait for the one before: 63 leaves of 50,021 x 137 f32, gradient of
//   weights of 33 outputs, 159 us so).
// Products of bf16 values are exact in f32 and sums are f32 throughout; f32 operands use the f32 matrix instruction; products of
// 8-bit integers and their sums are exact in 32 bits (row operands and DIRECT only: rows of codes are whole chunks).
// Measured in the kernels that use it: 256 x 256 tiles of bf16 1.2 PFLOP/s with a long k (dC of 65,536 classes x 1,024 over 8,192
// rows), where a large library product reached 1.2 to 1.6 on the same card; f32, whose matrix instructions are the bound, 58 to
// 63 TFLOP/s where rows of 137 values end inside tiles of 64, of 153.  Reads of the stages meet no bank
// conflicts, of rows (the scores) or turned (dh); stores by way of local memory spend up to 16 % of its cycles on them.
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
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

// A fragment is 16 bytes of k; Acc holds four sums.
template <typename T> struct Traits;
template <> struct Traits<bf16> {
  typedef bf16x8 Frag;
  typedef f32x4 Acc;
};
template <> struct Traits<float> {
  typedef f32x4 Frag;
  typedef f32x4 Acc;
};
template <> struct Traits<int8_t> {
  typedef i32x4 Frag;
  typedef i32x4 Acc;
};
template <typename T> constexpr int kChunk = 16 / (int)sizeof(T);       // values a chunk

// 16 zero bytes in device memory: what a lane without a chunk loads.
static __device__ __align__(16) const uint32_t zero_chunk[4] = {0, 0, 0, 0};

// The first `valid` values of a chunk, zeros behind.
template <typename T>
__device__ __forceinline__ u32x4 first_values(u32x4 v, int valid) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (sizeof(T) == 4) {
      v[i] = i < valid ? v[i] : 0;
    } else {
      v[i] = 2 * i + 1 < valid ? v[i] : 2 * i < valid ? v[i] & 0xffffu : 0;
    }
  }
  return v;
}

// 16 bytes of device memory, of any alignment.  (Said to be device memory: a choice between a matrix and the zeros above is
// not seen to be, and a flat load is waited for with every other kind.)
__device__ __forceinline__ u32x4 load16(const void* p) {
  typedef u32x4 __attribute__((aligned(1))) any_u32x4;
  return *(const __attribute__((address_space(1))) any_u32x4*)p;
}

// A chunk that begins less than 16 bytes before the matrix ends.
template <typename T>
__device__ __forceinline__ u32x4 last_chunk(const T* p, int valid) {
  T part[kChunk<T>];
#pragma unroll
  for (int i = 0; i < kChunk<T>; ++i) part[i] = i < valid ? p[i] : (T)0.0f;
  u32x4 v;
  __builtin_memcpy(&v, part, 16);
  return v;
}

// The thread's number among the NT of its tile; a workgroup may hold several tiles' threads.
template <int NT>
__device__ __forceinline__ int thread_of() {
  return (int)threadIdx.x % NT;
}

// The byte of local memory where a wavefront's first chunk of a stage goes, for scalar registers.
template <int NT>
__device__ __forceinline__ uint32_t wave_place(const char* stage) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)stage +
         __builtin_amdgcn_readfirstlane(thread_of<NT>() >> 6) * 1024u;
}

// 16 bytes from each lane's `src` to lane-consecutive places from byte `place` of local memory on (the same in all lanes).  Written as a
// statement of its own, without results: the compiler, which would wait for every such load before the next turned read of
// local memory, counts none of them, and arrived() below does.
__device__ __forceinline__ void direct_chunk(const void* src, uint32_t place) {
  const uint32_t to = __builtin_amdgcn_readfirstlane(place);  // (nothing, where the compiler knows that it is one value)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // m0 is a reserved register: nothing is kept in it
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(src) : "memory", "m0");
#pragma clang diagnostic pop
}

// How the 16-byte chunks of a column operand's row k are permuted (R columns a row).
template <typename T, int R>
__device__ __forceinline__ int column_swizzle(int k) {
  constexpr int chunks = R / kChunk<T>;
  if (sizeof(T) == 2) return (((k & 3) | ((k >> 1) & 4)) << 1) & (chunks - 1);
  return (((k >> 2) & 3) << 2) & (chunks - 1);
}

// ---------------------------------------------------------------- operands

// Rows are m or n, k along memory.
template <typename T, int R, int NT, bool DIRECT, int KB>
struct RowOperand {
  static constexpr int kStep = KB / (int)sizeof(T);
  static constexpr int kRowChunks = KB / 16;
  static constexpr int kSlots = R * kRowChunks;
  static constexpr int kPer = (kSlots + NT - 1) / NT;
  static constexpr int kLoads = kPer;  // of device memory, a step
  static constexpr int kBytes = R * KB;
  const T* row[kPer];  // DIRECT: of the chunk that is loaded next
  const T* end;
  u32x4 reg[DIRECT ? 1 : kPer];
  int k_of, k_end;

  // How the chunks of row r are permuted: rows of 128 bytes by three of its bits, two rows of 64 bytes alike.
  __device__ __forceinline__ static int swizzle(int r) { return KB == 128 ? r & 7 : (r >> 1) & 3; }
  static_assert(KB == 128 || KB == 64, "");
  static_assert(NT / kRowChunks % 8 == 0, "a thread's chunks lie in the same place of their rows");

  // What init needs of the rows' ids: it may be asked for long before.
  struct Ids {
    int id[kPer];
  };
  template <class Rows>
  __device__ __forceinline__ static void fetch(const Rows& rows, int r0, Ids& ids) {
    const int t = thread_of<NT>();
#pragma unroll
    for (int i = 0; i < kPer; ++i) ids.id[i] = i * NT + t < kSlots ? rows.fetch(r0 + (i * NT + t) / kRowChunks) : -1;
  }
  template <class Rows>
  __device__ __forceinline__ void init(const Rows& rows, int r0, int limit, int k0, int k1) {
    Ids ids;
    fetch(rows, r0, ids);
    init(rows, r0, limit, k0, k1, ids);
  }
  template <class Rows>
  __device__ __forceinline__ void init(const Rows& rows, int r0, int /*limit*/, int k0, int k1, const Ids& ids) {
    const int t = thread_of<NT>();
    k_of = k0 + (t % kRowChunks ^ swizzle(t / kRowChunks)) * kChunk<T>;
    k_end = k1;
    end = rows.end;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      row[i] = i * NT + t < kSlots ? rows.at(r0 + (i * NT + t) / kRowChunks, ids.id[i]) : nullptr;
      if (DIRECT) row[i] = (row[i] != nullptr ? row[i] : rows.base) + k_of;
    }
  }
  // DIRECT: the i'th of a step's chunks (WHOLE: of a step that no limit cuts); after the last, `advance`.
  template <bool WHOLE, class Rows>
  __device__ __forceinline__ void load_one(const Rows&, char* stage, int i) {
    const int t = thread_of<NT>();
    if (kSlots % NT != 0 && i * NT + t >= kSlots) return;
    if (WHOLE || k_of < k_end) {
      direct_chunk(row[i], wave_place<NT>(stage) + i * NT * 16);
    } else {
      *(u32x4*)(stage + (i * NT + t) * 16) = u32x4{0, 0, 0, 0};
    }
    row[i] += kStep;
  }
  template <class Rows>
  __device__ __forceinline__ void advance(const Rows&) {
    k_of += kStep;
  }
  template <class Rows>
  __device__ __forceinline__ void load(const Rows&, char* stage) {
    const int t = thread_of<NT>();
    if constexpr (DIRECT) {
      if (k_of < k_end) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          if (kSlots % NT != 0 && i * NT + t >= kSlots) break;
          direct_chunk(row[i], wave_place<NT>(stage) + i * NT * 16);
          row[i] += kStep;
        }
      } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          if (kSlots % NT != 0 && i * NT + t >= kSlots) break;
          *(u32x4*)(stage + (i * NT + t) * 16) = u32x4{0, 0, 0, 0};
        }
      }
    } else {
      bool cut = false;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const bool any = row[i] != nullptr && k_of < k_end;
        const bool fits = any && row[i] + k_of + kChunk<T> <= end;
        const void* p = fits ? (const void*)(row[i] + k_of) : (const void*)zero_chunk;
        reg[i] = load16(p);
        cut |= any && !fits;
      }
      if (cut) {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          if (row[i] != nullptr && k_of < k_end && row[i] + k_of + kChunk<T> > end) reg[i] = last_chunk<T>(row[i] + k_of, k_end - k_of);
      }
    }
    k_of += kStep;
  }
  __device__ __forceinline__ void store(char* stage) {
    if constexpr (!DIRECT) {
      const int t = thread_of<NT>();
      const int valid = k_end - (k_of - kStep);
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (kSlots % NT != 0 && i * NT + t >= kSlots) break;
        *(u32x4*)(stage + (i * NT + t) * 16) = valid < kChunk<T> ? first_values<T>(reg[i], valid) : reg[i];
      }
    }
  }
  // Where a wavefront whose rows begin at r0 (a multiple of 16) reads: lane l holds row l mod 16 of a block of 16 and 16 bytes
  // of k.  Blocks lie a constant distance apart, since the permutation hangs on a row's low three bits alone.
  template <int BLOCKS>
  struct Lanes {
    int at[KB / 64];
    __device__ __forceinline__ explicit Lanes(int r0) {
      const int l = threadIdx.x & 63;
#pragma unroll
      for (int part = 0; part < KB / 64; ++part) at[part] = (r0 + (l & 15)) * KB + (((l >> 4) + 4 * part) ^ swizzle(l & 15)) * 16;
    }
  };
  // The block'th 16 rows for the part'th half of the step; k as both operands order it.
  template <int BLOCKS>
  __device__ __forceinline__ static typename Traits<T>::Frag frag(const char* stage, const Lanes<BLOCKS>& lanes, int block, int part) {
    return *(const typename Traits<T>::Frag*)(stage + lanes.at[part] + block * 16 * KB);
  }
};

// Rows are k, m or n along memory.
template <typename T, int R, int NT, bool DIRECT, int KB>
struct ColumnOperand {
  static constexpr int kStep = KB / (int)sizeof(T);
  static constexpr int kSlots = R * (KB / 16);
  static constexpr int kPer = (kSlots + NT - 1) / NT;
  static constexpr int kLoads = kPer;  // of device memory, a step
  static constexpr int kBytes = R * KB;
  static constexpr int kChunks = R / kChunk<T>;  // a row
  static_assert(kSlots % NT == 0, "every thread has as many chunks");
  int id[kPer];  // of the step that is loaded next
  const T* here[DIRECT ? kPer : 1];  // DIRECT and rows a constant distance apart: the chunk that is loaded next
  u32x4 reg[DIRECT ? 1 : kPer];
  int k_at, k_end, c0, lim;

  __device__ __forceinline__ static int slot_k(int i) { return (i * NT + thread_of<NT>()) / kChunks; }
  // (the same for all of a thread's chunks where as many rows lie between them as the permutation repeats after)
  __device__ __forceinline__ int slot_column(int i) const {
    const int s = (NT / kChunks % 16 == 0 ? 0 : i) * NT + thread_of<NT>();
    return c0 + ((s % kChunks) ^ column_swizzle<T, R>(s / kChunks)) * kChunk<T>;
  }
  template <class Rows>
  __device__ __forceinline__ void fetch(const Rows& rows) {
    if (DIRECT && Rows::kEven) return;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int k = k_at + slot_k(i);
      id[i] = k < k_end ? rows.fetch(k) : -1;
    }
  }
  template <class Rows>
  __device__ __forceinline__ void init(const Rows& rows, int col0, int limit, int k0, int k1) {
    k_at = k0;
    k_end = k1;
    c0 = col0;
    lim = limit;
    fetch(rows);
    if constexpr (DIRECT && Rows::kEven) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) here[i] = rows.base + (int64_t)(k_at + slot_k(i)) * rows.ld + direct_column(i);
    }
  }
  // Any column that exists stands in for one past the limit.  (Rows that are none are zeros, loaded as such if rows come from
  // a list: then every step has as many loads as any other.)
  __device__ __forceinline__ int direct_column(int i) const {
    const int c = slot_column(i);
    return c < lim ? c : lim - kChunk<T>;
  }
  // DIRECT: the i'th of a step's chunks (WHOLE: of a step that no limit cuts); after the last, `advance`.
  template <bool WHOLE, class Rows>
  __device__ __forceinline__ void load_one(const Rows& rows, char* stage, int i) {
    static_assert(DIRECT, "");
    const int t = thread_of<NT>();
    if constexpr (!Rows::kEven) {
      const T* row = rows.at(k_at + slot_k(i), id[i]);
      direct_chunk(row != nullptr ? (const void*)(row + direct_column(i)) : (const void*)zero_chunk, wave_place<NT>(stage) + i * NT * 16);
    } else {
      if (WHOLE || k_at + slot_k(i) < k_end) {
        direct_chunk(here[i], wave_place<NT>(stage) + i * NT * 16);
      } else {
        *(u32x4*)(stage + (i * NT + t) * 16) = u32x4{0, 0, 0, 0};
      }
      here[i] += (int64_t)kStep * rows.ld;
    }
  }
  template <class Rows>
  __device__ __forceinline__ void advance(const Rows& rows) {
    k_at += kStep;
    fetch(rows);
  }
  template <class Rows>
  __device__ __forceinline__ void load(const Rows& rows, char* stage) {
    const int t = thread_of<NT>();
    if constexpr (DIRECT) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (Rows::kEven && k_at + kStep <= k_end) {
          load_one<true>(rows, stage, i);
        } else {
          load_one<false>(rows, stage, i);
        }
      }
    } else {
      const T* p[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int k = k_at + slot_k(i), c = slot_column(i);
        const T* row = k < k_end && c < lim ? rows.at(k, id[i]) : nullptr;
        p[i] = row != nullptr ? row + c : nullptr;
      }
      bool cut = false;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const bool fits = p[i] != nullptr && p[i] + kChunk<T> <= rows.end;
        const void* q = fits ? (const void*)p[i] : (const void*)zero_chunk;
        reg[i] = load16(q);
        cut |= p[i] != nullptr && !fits;
      }
      if (cut) {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          if (p[i] != nullptr && p[i] + kChunk<T> > rows.end) reg[i] = last_chunk<T>(p[i], lim - slot_column(i));
      }
    }
    k_at += kStep;
    fetch(rows);
  }
  __device__ __forceinline__ void store(char* stage) {
    if constexpr (!DIRECT) {
      const int t = thread_of<NT>();
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int valid = lim - slot_column(i);
        *(u32x4*)(stage + (i * NT + t) * 16) = valid < kChunk<T> ? first_values<T>(reg[i], valid) : reg[i];
      }
    }
  }
  // Here the permutation reaches the bits that tell blocks apart, and an offset a block is kept; it hangs on neither the
  // half nor the reads of a fragment.
  static constexpr int kRowBytes = R * (int)sizeof(T);
  template <int BLOCKS>
  struct Lanes {
    int at[BLOCKS];
    __device__ __forceinline__ explicit Lanes(int r0) {
      const int l = threadIdx.x & 63, j = l & 15;
#pragma unroll
      for (int i = 0; i < BLOCKS; ++i) {
        if (sizeof(T) == 2) {
          // lane j of a group of 16 addresses row j / 4, values 4 (j mod 4) .. + 3, and receives column j of the four rows
          const int k = (l >> 4) * 8 + (j >> 2), c = (r0 + 16 * i) / 8 + ((j & 3) >> 1);
          at[i] = k * kRowBytes + (c ^ column_swizzle<T, R>(k)) * 16 + (j & 1) * 8;
        } else {
          const int k = (l >> 4) * 4, c = (r0 + 16 * i + j) / 4;
          at[i] = k * kRowBytes + (c ^ column_swizzle<T, R>(k)) * 16 + (j & 3) * 4;
        }
      }
    }
  };
  template <int BLOCKS>
  __device__ __forceinline__ static typename Traits<T>::Frag frag(const char* stage, const Lanes<BLOCKS>& lanes, int block, int part) {
    typename Traits<T>::Frag f;
    const char* a = stage + lanes.at[block];
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)(a + (part * 32 + h * 4) * kRowBytes));
        __builtin_memcpy((char*)&f + h * 8, &v, 8);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = *(const float*)(a + (part * 16 + i) * kRowBytes);
    }
    return f;
  }
};

// A column operand (bf16) whose row k has one value that is not zero, as rows.fetch(k) tells: its column in the upper half of
// the word and its bits in the lower, -1 for none.  Made in the stage, not loaded.
template <int R, int NT, int KB>
struct OneHotOperand : ColumnOperand<bf16, R, NT, true, KB> {
  typedef ColumnOperand<bf16, R, NT, true, KB> Base;
  static constexpr int kLoads = 0;
  template <class Rows>
  __device__ __forceinline__ void init(const Rows&, int k0, int k1) {
    this->k_at = k0;
    this->k_end = k1;
    this->c0 = 0;
    this->lim = R;
  }
  template <bool WHOLE, class Rows>
  __device__ __forceinline__ void load_one(const Rows& rows, char* stage, int i) {
    const int k = this->k_at + Base::slot_k(i), c = this->slot_column(i);
    const int entry = k < this->k_end ? rows.fetch(k) : -1;
    const int at = (entry >> 16) - c;
    u32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (at == e) v[e / 2] = ((uint32_t)entry & 0xffffu) << (e % 2 * 16);
    *(u32x4*)(stage + (i * NT + thread_of<NT>()) * 16) = v;
  }
  template <class Rows>
  __device__ __forceinline__ void advance(const Rows&) {
    this->k_at += Base::kStep;
  }
  template <class Rows>
  __device__ __forceinline__ void load(const Rows& rows, char* stage) {
#pragma unroll
    for (int i = 0; i < Base::kPer; ++i) load_one<false>(rows, stage, i);
    advance(rows);
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

// 16 codes each: exact sums in 32 bits.
__device__ __forceinline__ i32x4 mma(i32x4 rows, i32x4 cols, i32x4 acc) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(rows, cols, acc, 0, 0, 0);
}

// ---------------------------------------------------------------- the tile

// BM x BN values by WM x WN wavefronts.  A lane's four values of the 16 x 16 block (i, j) of its wavefront:
//   N_INNER: m = 16 i + lane mod 16, n = 16 j + 4 (lane / 16) + 0..3   (rows of an output along n)
//   else:    n = 16 j + lane mod 16, m = 16 i + 4 (lane / 16) + 0..3   (columns of an output along m)
// DEEP (DIRECT only): steps of 64 bytes of k and four stages instead of 128 bytes and STAGES (more than two: DIRECT only).
// PARTS: sums are taken in parts of 128 k (see tile_run); f32 operands' always are.
template <typename T_, int BM_, int BN_, int WM_, int WN_, bool DIRECT_, bool DEEP_ = false, int STAGES_ = 2, bool PARTS_ = false>
struct Shape {
  typedef T_ T;
  typedef typename Traits<T_>::Acc Acc;
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NT = WM_ * WN_ * 64;
  static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;
  static constexpr bool DIRECT = DIRECT_, DEEP = DEEP_, PARTS = PARTS_ || sizeof(T_) == 4;
  static constexpr int KB = DEEP ? 64 : 128, kStep = KB / (int)sizeof(T), kStages = DEEP ? 4 : STAGES_;
  static constexpr int kStageBytes = (BM + BN) * KB;
  static constexpr int kLdsBytes = kStages * kStageBytes;
  static constexpr int kLastStage = (kStages - 1) * kStageBytes;
  static_assert(TM >= 1 && TN >= 1 && BM % (WM * 16) == 0 && BN % (WN * 16) == 0, "whole 16 x 16 blocks");
  static_assert(DIRECT || (!DEEP && kStages == 2), "");
  static_assert(!DEEP || TM >= 4, "a turn's chunks are asked for between its row blocks, but for the last two");
  typedef RowOperand<T, BM, NT, DIRECT, KB> RowsA;
  typedef RowOperand<T, BN, NT, DIRECT, KB> RowsB;
  typedef ColumnOperand<T, BM, NT, DIRECT, KB> ColumnsA;
  typedef ColumnOperand<T, BN, NT, DIRECT, KB> ColumnsB;
};

// All chunks that this wavefront has asked for, but for the LATER last ones, have arrived and its reads are done; then
// everyone's.
template <int LATER>
__device__ __forceinline__ void arrived() {
  static_assert(LATER < 64, "the counter's six bits");
  // (the builtin, not an asm statement: the compiler then knows that nothing is outstanding, scalar loads among it, and
  // waits for single reads afterwards, where it would wait for all)
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((LATER & 15) | 7 << 4 | (LATER >> 4) << 14);  // vmcnt(LATER) lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Nothing is moved across: reads and products stay in the order they are written in.  (Left to itself the compiler reads
// just before it multiplies, and waits.)
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

template <int I>
struct Int {
  static constexpr int value = I;
};
template <int I, int END, class F>
__device__ __forceinline__ void for_blocks(const F& f) {
  if constexpr (I < END) {
    f(Int<I>{});
    for_blocks<I + 1, END>(f);
  }
}

// The second half's column fragments that are read before a row block: all of them in the first half, evenly.
template <class S>
constexpr int columns_before(int block) {
  return block >= S::TM ? S::TN : (block * S::TN + S::TM - 1) / S::TM;
}

// Asks for a tile's first steps.  tile_run must follow; a kernel may do something else with the tile before, if it leaves
// the stages alone: load the next tile's first steps and then store this one's results.
template <class S, class A, class B, class RowsA, class RowsB>
__device__ __forceinline__ void tile_begin(char* lds, A& a, B& b, const RowsA& rows_a, const RowsB& rows_b, int k0, int k1) {
  const int steps = (k1 - k0 + S::kStep - 1) / S::kStep;
  if (steps <= 0) return;
  // (DEEP: an even number of steps, the last of them zeros if need be)
  for_blocks<0, S::kStages - 1>([&](auto at) {
    constexpr int i = decltype(at)::value;
    if (i < steps || (S::DEEP && i == 1)) {
      a.load(rows_a, lds + i * S::kStageBytes);
      b.load(rows_b, lds + i * S::kStageBytes + A::kBytes);
    }
  });
}

template <class S>
__device__ __forceinline__ void zeros(typename S::Acc (&acc)[S::TM][S::TN]) {
#pragma unroll
  for (int i = 0; i < S::TM; ++i)
#pragma unroll
    for (int j = 0; j < S::TN; ++j) acc[i][j] = typename S::Acc{0, 0, 0, 0};
}

// Adds the products of k0 <= k < k1 to acc.
template <class S, bool N_INNER, class A, class B, class RowsA, class RowsB, class Also>
__device__ __forceinline__ void tile_run(char* lds, A& a, B& b, const RowsA& rows_a, const RowsB& rows_b, int k0, int k1,
                                         typename S::Acc (&acc)[S::TM][S::TN], const Also& also) {
  typedef typename Traits<typename S::T>::Frag Frag;
  // (with more stages than two a wait counts loads, and every wavefront must have asked for as many)
  static_assert(S::kStages == 2 || (A::kSlots % S::NT == 0 && B::kSlots % S::NT == 0), "every thread has as many chunks");
  const int w = thread_of<S::NT>() >> 6;
  const int m0 = (w / S::WN) * (S::TM * 16), n0 = (w % S::WN) * (S::TN * 16);
  const int steps = (k1 - k0 + S::kStep - 1) / S::kStep;
  if (steps <= 0) return;

  const typename A::template Lanes<S::TM> lanes_a(m0);
  const typename B::template Lanes<S::TN> lanes_b(n0);
  // A step is TM row blocks of 16 x (16 TN) for each 64 bytes of k.  The fragment of a block's rows is read two blocks ahead,
  // those of its columns a turn of TM blocks ahead: 2 TN + 4 fragments are held, where two whole turns would be 2 (TN + TM)
  // and take more registers than 256 x 256 tiles leave.
  static_assert(S::TM == 2 || S::TM % 4 == 0, "four fragments in turn, two blocks ahead");
  Frag fa[4], fb[2][S::TN];
  auto read_rows = [&](const char* stage, int part, int i, int slot) { fa[slot & 3] = A::frag(stage, lanes_a, i, part); };
  auto read_columns = [&](const char* stage, int part, int j, int turn) {
    fb[turn][j] = B::frag(stage + A::kBytes, lanes_b, j, part);
  };
  // f32 operands: products are added four k at a time, so a sum over 1,024 is a chain of 256 roundings; every 128 k
  // what has come together is added to the rest instead, which leaves two chains of 32 and 8.  (Scores of 1,024 dimensions:
  // three times the error of a product summed in parts without it.)  bf16 ones are added 32 k at a time, and only what ends in
  // f32, the columns of statistics, is worth the registers.
  constexpr bool kParts = S::PARTS;
  typename S::Acc part_sum[kParts ? S::TM : 1][kParts ? S::TN : 1];
  auto multiply = [&](int i, int slot, int turn) {
#pragma unroll
    for (int j = 0; j < S::TN; ++j) {
      typename S::Acc& to = kParts ? part_sum[kParts ? i : 0][kParts ? j : 0] : acc[i][j];
      to = N_INNER ? mma(fb[turn][j], fa[slot & 3], to) : mma(fa[slot & 3], fb[turn][j], to);
    }
    also(i, fa[slot & 3]);
  };
  auto add_part = [&](bool now) {
    if constexpr (kParts) {
      if (!now) return;
#pragma unroll
      for (int i = 0; i < S::TM; ++i)
#pragma unroll
        for (int j = 0; j < S::TN; ++j) {
          acc[i][j] += part_sum[i][j];
          part_sum[i][j] = typename S::Acc{0, 0, 0, 0};
        }
    }
  };
  if constexpr (kParts) zeros<S>(part_sum);
  constexpr int part_steps = 128 / S::kStep;  // (f32: 4; bf16: 2, or 4 of half the length)

  if constexpr (S::DEEP) {
    // A turn is a step.  Its stage is given up two blocks before the turn ends, when all of it has been read; the step four
    // turns ahead goes there, a chunk at a time between the next turn's blocks: eight wavefronts that ask for all their chunks
    // at once wait for the address units before they can go on to multiply.  (With two stages of twice the length a chunk
    // would have to be on its way before the next turn.)  Turns go in pairs, so that the fragments' places are known to the
    // compiler; an odd number is filled up with zeros.
    constexpr int per = A::kPer + B::kPer, loads = A::kLoads + B::kLoads;
    const int full = ((a.k_end < b.k_end ? a.k_end : b.k_end) - k0) / S::kStep;  // steps whose every chunk is loaded
    const int turns = (steps + 1) / 2 * 2;
    auto load_one = [&](auto whole, int step, int i) {
      char* to = lds + (step & 3) * S::kStageBytes;
      if (i < A::kPer) {
        a.template load_one<decltype(whole)::value>(rows_a, to, i);
      } else {
        b.template load_one<decltype(whole)::value>(rows_b, to + A::kBytes, i - A::kPer);
      }
    };
    auto first_reads = [&](const char* stage, int turn) {
#pragma unroll
      for (int j = 0; j < S::TN; ++j) read_columns(stage, 0, j, turn);
      read_rows(stage, 0, 0, 0);
      in_order();
      read_rows(stage, 0, 1, 1);
    };
    // WHOLE: the step that is loaded in this turn has no limit in it.
    auto one_turn = [&](auto whole, auto which, int at_turn) {
      constexpr int turn = decltype(which)::value;
      const char* here = lds + (at_turn & 3) * S::kStageBytes;
      const char* next = lds + ((at_turn + 1) & 3) * S::kStageBytes;
      const bool more = decltype(whole)::value || at_turn + 3 < turns;
      for_blocks<0, S::TM - 2>([&](auto at) {
        constexpr int i = decltype(at)::value;
        read_rows(here, 0, i + 2, i + 2);
        in_order();
        multiply(i, i, turn);
        in_order();
        if (more) {
#pragma unroll
          for (int k = i * per / (S::TM - 2); k < (i + 1) * per / (S::TM - 2); ++k) load_one(whole, at_turn + 3, k);
        }
        in_order();
      });
      if (more) {
        a.advance(rows_a);
        b.advance(rows_b);
      }
      // The next step is there; the two behind it may be on their way.
      if (decltype(whole)::value) {
        arrived<2 * loads>();
      } else {
        arrived<0>();
      }
      first_reads(next, 1 - turn);  // (of whatever is there after the last step)
      in_order();
      multiply(S::TM - 2, S::TM - 2, turn);
      multiply(S::TM - 1, S::TM - 1, turn);
      add_part(at_turn % part_steps == part_steps - 1 || at_turn + 1 == turns);
      in_order();
    };
    if (full > 2) {
      arrived<2 * loads>();
    } else {
      arrived<0>();
    }
    first_reads(lds, 0);
    int s = 0;
    for (; s + 4 < full; s += 2) {
      one_turn(Int<1>{}, Int<0>{}, s);
      one_turn(Int<1>{}, Int<1>{}, s + 1);
    }
    for (; s < turns; s += 2) {
      one_turn(Int<0>{}, Int<0>{}, s);
      one_turn(Int<0>{}, Int<1>{}, s + 1);
    }
  } else {
    // Two turns a step.
    auto first_reads = [&](const char* stage) {
#pragma unroll
      for (int j = 0; j < S::TN; ++j) read_columns(stage, 0, j, 0);
      read_rows(stage, 0, 0, 0);
      in_order();
      read_rows(stage, 0, 1, 1);
    };
    // All blocks but the last two, whose fragments have been read by then.
    constexpr int blocks = 2 * S::TM;
    auto most_blocks = [&](const char* stage) {
      for_blocks<0, blocks - 2>([&](auto at) {
        constexpr int block = decltype(at)::value;
        constexpr int columns = columns_before<S>(block + 1) - columns_before<S>(block);
        read_rows(stage, (block + 2) / S::TM, (block + 2) % S::TM, block + 2);
#pragma unroll
        for (int j = 0; j < columns; ++j) read_columns(stage, 1, columns_before<S>(block) + j, 1);
        in_order();
        multiply(block % S::TM, block, block / S::TM);
        in_order();
      });
    };
    if constexpr (S::DIRECT) {
      // A stage is given up two blocks before its step ends, when all of it has been read, and the step kStages later goes
      // there: one barrier a step is enough, and the last two blocks cover the first reads of the next stage.
      constexpr int ns = S::kStages, loads = A::kLoads + B::kLoads;
      const int full = ((a.k_end < b.k_end ? a.k_end : b.k_end) - k0) / S::kStep;  // steps whose every chunk is loaded
      // Step `next` is there; the kStages - 2 behind it may be on their way.
      auto wait = [&](int next) {
        if (ns > 2 && next + ns - 2 < full) {
          arrived<(ns - 2) * loads>();
        } else {
          arrived<0>();
        }
      };
      wait(0);
      char* here = lds;
      char* free = lds + (ns - 1) * S::kStageBytes;
      if (ns - 1 < steps) {
        a.load(rows_a, free);
        b.load(rows_b, free + A::kBytes);
      }
      first_reads(lds);
      for (int s = 0; s < steps; ++s) {
        char* next = here + S::kStageBytes == lds + ns * S::kStageBytes ? lds : here + S::kStageBytes;
        most_blocks(here);
        wait(s + 1);
        first_reads(next);  // (of whatever is there after the last step)
        in_order();
        multiply(S::TM - 2, blocks - 2, 1);
        in_order();
        if (s + ns < steps) {
          a.load(rows_a, here);
          b.load(rows_b, here + A::kBytes);
        }
        in_order();
        multiply(S::TM - 1, blocks - 1, 1);
        add_part(s % part_steps == part_steps - 1 || s + 1 == steps);
        in_order();
        here = next;
      }
    } else {
      a.store(lds);
      b.store(lds + A::kBytes);
      for (int s = 0; s < steps; ++s) {
        char* here = lds + (s & 1) * S::kStageBytes;
        char* next = lds + ((s + 1) & 1) * S::kStageBytes;
        __syncthreads();  // everyone has written this stage and read the other
        if (s + 1 < steps) {
          a.load(rows_a, next);
          b.load(rows_b, next + A::kBytes);
        }
        first_reads(here);
        most_blocks(here);
        multiply(S::TM - 2, blocks - 2, 1);
        multiply(S::TM - 1, blocks - 1, 1);
        add_part(s % part_steps == part_steps - 1 || s + 1 == steps);
        if (s + 1 < steps) {
          a.store(next);
          b.store(next + A::kBytes);
        }
      }
      __syncthreads();  // everyone has read the last stage: what comes next may write any
    }
  }
}

template <class S, bool N_INNER, class A, class B, class RowsA, class RowsB, class Also>
__device__ __forceinline__ void tile_product(char* lds, A& a, B& b, const RowsA& rows_a, const RowsB& rows_b, int k0, int k1,
                                             typename S::Acc (&acc)[S::TM][S::TN], const Also& also) {
  zeros<S>(acc);
  tile_begin<S>(lds, a, b, rows_a, rows_b, k0, k1);
  tile_run<S, N_INNER>(lds, a, b, rows_a, rows_b, k0, k1, acc, also);
}

struct Nothing {
  template <class F>
  __device__ __forceinline__ void operator()(int, const F&) const {}
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

// Stores a wavefront's tile, ROWS blocks of 16 rows of INNER x 16 values (N_INNER: TM and TN; the other way round: TN and TM),
// by whole 16-byte chunks of its rows: each block of 16 rows goes through a piece of local
// memory of the wavefront's own, so that a store writes lines of 128 bytes at once.  (Straight from the registers a store
// writes 32 bytes of each of 16 rows, and the next 96 of them come with the stores after it: 100,000 x 256 -> 2,000 bf16,
// gradient of the input, 341 us so against 210 us without any stores.)
//   value(i, j): the four values of the block; row(i, r): where row r of block i begins, or null; col0, cols: the wavefront's
//   first column and the end of the rows.  scratch: of the workgroup, the last stage, which tile_begin does not touch.
template <class S, typename O, int ROWS, int INNER, class Value, class Row>
__device__ __forceinline__ void store_tile(char* scratch, const Value& value, const Row& row, int col0, int cols) {
  const int l = threadIdx.x & 63, w = thread_of<S::NT>() >> 6;
  constexpr int row_bytes = INNER * 16 * (int)sizeof(O);
  if constexpr (row_bytes >= 128) {
    constexpr int chunks = row_bytes / 16, at_once = 64 / chunks, n = 16 / (int)sizeof(O);
    static_assert(S::WM * S::WN * 16 * row_bytes <= S::kStageBytes, "a piece a wavefront");
    char* mine = scratch + w * (16 * row_bytes);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
#pragma unroll
      for (int j = 0; j < INNER; ++j) {
        const f32x4 v = value(i, j);
        const O t[4] = {(O)v[0], (O)v[1], (O)v[2], (O)v[3]};
        const int byte = (16 * j + 4 * (l >> 4)) * (int)sizeof(O), r = l & 15;
        __builtin_memcpy(mine + r * row_bytes + ((byte / 16) ^ (r & 7)) * 16 + byte % 16, t, sizeof t);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int k = 0; k < 16 / at_once; ++k) {
        const int r = l / chunks + k * at_once, c = l % chunks;
        const u32x4 v = *(const u32x4*)(mine + r * row_bytes + (c ^ (r & 7)) * 16);
        O* to = row(i, r);
        const int at = col0 + c * n;
        if (to == nullptr || at >= cols) continue;
        if (at + n <= cols) {
          __builtin_memcpy(to + at, &v, 16);
        } else {
          O t[n];
          __builtin_memcpy(t, &v, 16);
#pragma unroll
          for (int e = 0; e < n; ++e)
            if (at + e < cols) to[at + e] = t[e];
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  } else {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      O* to = row(i, l & 15);
      if (to == nullptr) continue;
#pragma unroll
      for (int j = 0; j < INNER; ++j) {
        const int at = col0 + 16 * j + 4 * (l >> 4);
        if (at < cols) store4(to + at, value(i, j), cols - at);
      }
    }
  }
}

// Workgroups go to the eight XCDs in turn; this gives each XCD a run of neighbouring tiles, which share operands in its L2.
__device__ __forceinline__ uint32_t xcd_tile(uint32_t block, uint32_t blocks) {
  const uint32_t per = blocks / 8, extra = blocks % 8;
  const uint32_t x = block % 8, i = block / 8;
  return x * per + (x < extra ? x : extra) + i;
}

}  // namespace gbdt_tile
