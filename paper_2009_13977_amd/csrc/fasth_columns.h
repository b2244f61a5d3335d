// Device-side helpers of the operators around the layers (fasth_embed.h, fasth_norm.h, fasth_log_prob.h,
// fasth_grad.h): element types, VEC neighbouring columns of a [rows][m] matrix in one access, token numbers.
#pragma once
#include <hip/hip_runtime.h>

#include "fasth.h"
#include "fasth_device.h"

namespace fasth {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// VEC neighbouring elements in registers, as they are in memory. A row of an odd number of columns starts at any
// multiple of the element's size, which global memory accesses of any width allow on this hardware.
template <typename T, int VEC>
struct Cols {
  typedef T vec __attribute__((ext_vector_type(VEC)));
  vec v;
  __device__ __forceinline__ float get(int i) const { return (float)v[i]; }
  __device__ __forceinline__ void set(int i, float x) { v[i] = (T)x; }  // rounds to nearest, ties to even
};
template <typename T>
struct Cols<T, 1> {
  typedef T vec;
  T v;
  __device__ __forceinline__ float get(int) const { return (float)v; }
  __device__ __forceinline__ void set(int, float x) { v = (T)x; }
};

// `left`: columns that exist from p on; the others read as `fill` and are not written.
template <typename T, int VEC>
__device__ __forceinline__ Cols<T, VEC> load_cols(const T* p, int left, float fill = 0.f) {
  Cols<T, VEC> c;
  if (VEC == 1 ? left > 0 : left >= VEC) {
    __builtin_memcpy(&c.v, p, VEC * sizeof(T));
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      c.set(i, fill);
      if (i < left) c.set(i, (float)p[i]);
    }
  }
  return c;
}
template <typename T, int VEC>
__device__ __forceinline__ void store_cols(T* p, int left, const Cols<T, VEC>& c) {
  if (VEC == 1 ? left > 0 : left >= VEC) {
    __builtin_memcpy(p, &c.v, VEC * sizeof(T));
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i)
      if (i < left) p[i] = (T)c.get(i);
  }
}

// Buffer accesses: the descriptor (scalar registers) holds the matrix and its size, a lane has 32 bits of offset: enough for the
// largest mini-batch, 16384 x 65535 fp32. A lane beyond the end reads zeros and writes nothing, so that rows need no
// bounds check, and many loads in flight need no registers for 64-bit addresses.
constexpr unsigned kBeyond = 0xfffffff0u;  // beyond the end of every matrix that fits
__device__ __forceinline__ BufferDesc whole(const void* matrix, size_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(matrix), 0, (int)(unsigned)bytes, 0x00020000);
}
// The same number in a way that the compiler cannot see: what is computed from it (an offset per row) is computed again
// for the next loop over a thread's rows instead of being kept until then.
__device__ __forceinline__ unsigned again(unsigned x) {
  asm volatile("" : "+v"(x));
  return x;
}
constexpr int kPastCaches = 2;  // HOW: what is read or written is not needed again soon
template <typename T, int VEC, int HOW = 0>
__device__ __forceinline__ Cols<T, VEC> load_from(BufferDesc desc, unsigned offset) {
  constexpr int BYTES = VEC * (int)sizeof(T);
  static_assert(BYTES == 2 || BYTES == 4 || BYTES == 8 || BYTES == 16, "one access");
  Cols<T, VEC> c;
  if constexpr (BYTES == 16) c.v = __builtin_bit_cast(decltype(c.v), __builtin_amdgcn_raw_buffer_load_b128(desc, offset, 0, HOW));
  else if constexpr (BYTES == 8) c.v = __builtin_bit_cast(decltype(c.v), __builtin_amdgcn_raw_buffer_load_b64(desc, offset, 0, HOW));
  else if constexpr (BYTES == 4) c.v = __builtin_bit_cast(decltype(c.v), __builtin_amdgcn_raw_buffer_load_b32(desc, offset, 0, HOW));
  else c.v = __builtin_bit_cast(decltype(c.v), __builtin_amdgcn_raw_buffer_load_b16(desc, offset, 0, HOW));
  return c;
}
template <typename T, int VEC, int HOW = 0>
__device__ __forceinline__ void store_to(BufferDesc desc, unsigned offset, const Cols<T, VEC>& c) {
  constexpr int BYTES = VEC * (int)sizeof(T);
  if constexpr (BYTES == 16) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, c.v), desc, offset, 0, HOW);
  else if constexpr (BYTES == 8) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, c.v), desc, offset, 0, HOW);
  else if constexpr (BYTES == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, c.v), desc, offset, 0, HOW);
  else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, c.v), desc, offset, 0, HOW);
}

// The same for matrices of any size: a base that is the same for the wave, to which a lane adds 32 bits. No bounds checks.
template <typename T, int VEC>
__device__ __forceinline__ Cols<T, VEC> load_at(const T* base, unsigned lane_bytes) {
  Cols<T, VEC> c;
  __builtin_memcpy(&c.v, reinterpret_cast<const char*>(base) + lane_bytes, VEC * sizeof(T));
  return c;
}
template <typename T, int VEC>
__device__ __forceinline__ void store_at(T* base, unsigned lane_bytes, const Cols<T, VEC>& c) {
  __builtin_memcpy(reinterpret_cast<char*>(base) + lane_bytes, &c.v, VEC * sizeof(T));
}
// The same past the caches.
template <typename T, int VEC>
__device__ __forceinline__ Cols<T, VEC> load_once(const T* base, unsigned lane_bytes) {
  typedef typename Cols<T, VEC>::vec vec;
  typedef vec loose __attribute__((aligned(sizeof(T))));
  Cols<T, VEC> c;
  c.v = __builtin_nontemporal_load(reinterpret_cast<const loose*>(reinterpret_cast<const char*>(base) + lane_bytes));
  return c;
}
template <typename T, int VEC>
__device__ __forceinline__ void store_once(T* base, unsigned lane_bytes, const Cols<T, VEC>& c) {
  typedef typename Cols<T, VEC>::vec vec;
  typedef vec loose __attribute__((aligned(sizeof(T))));
  __builtin_nontemporal_store(c.v, reinterpret_cast<loose*>(reinterpret_cast<char*>(base) + lane_bytes));
}

// The VEC columns of a thread, of a matrix with m >= VEC columns. A thread whose columns reach beyond the last one looks
// at the last VEC instead, so that its loads are as wide as everyone's; the first `skip` of them belong to another
// thread: they are computed as well (columns do not meet) and not written. `ragged` is the same for the workgroup.
template <int VEC>
struct ColumnRange {
  int first, skip;
  bool ragged;
  __device__ __forceinline__ ColumnRange(int j, int m, bool last_tile)
      : first(j + VEC <= m ? j : m - VEC), skip(j - first < VEC ? j - first : VEC), ragged(last_tile && VEC > 1) {}
  __device__ __forceinline__ bool own(int e) const { return e >= skip; }
  // FULL: not ragged
  template <bool FULL, int HOW = 0, typename T>
  __device__ __forceinline__ void store(BufferDesc desc, unsigned offset, const Cols<T, VEC>& c) const {
    if constexpr (FULL) {
      store_to<T, VEC, HOW>(desc, offset, c);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        Cols<T, 1> one;
        one.v = (T)c.get(e);
        store_to<T, 1>(desc, own(e) ? offset + e * (unsigned)sizeof(T) : kBeyond, one);
      }
    }
  }
};

// The token of column j, or -1 where its number is no row of the vocabulary.
__device__ __forceinline__ int token_at(const void* ids, int id_bits, int j, int vocab) {
  if (!ids) return -1;  // (the same for all threads, as the numbers' width is)
  if (id_bits == 64) {
    const unsigned long long id = static_cast<const unsigned long long*>(ids)[j];
    return id < (unsigned)vocab ? (int)id : -1;
  }
  const unsigned id = static_cast<const unsigned*>(ids)[j];
  return id < (unsigned)vocab ? (int)id : -1;
}

// Workgroups start on the eight XCDs in turn. This order gives each XCD a run of consecutive blocks. Blocks are numbered
// along the rows of a matrix first, so that an XCD reads and writes whole rows: with the columns dealt out to the XCDs (a
// row of 32 blocks, say), each would reach for the same few memory channels in every row (log_prob_grad_kernel on
// 128000 x 4096 logits: 500 us in the order of starting, 371 us in this one).
__device__ __forceinline__ int xcd_run(int block, int blocks) {
  const int x = block & 7, each = blocks >> 3, more = blocks & 7;
  return x * each + (x < more ? x : more) + (block >> 3);
}
// The column tile and the row block of a workgroup of a one-dimensional grid.
struct TileAt {
  int col, row;
  __device__ __forceinline__ explicit TileAt(int tiles) {
    const int at = xcd_run(blockIdx.x, gridDim.x);
    row = at / tiles;
    col = at - row * tiles;
  }
};

// A value combined over the lanes of a wave that differ in the bits from FROM (a power of two) up to 32: in all of them,
// with the same bits if op(a, b) has those of op(b, a). V is made of 32-bit words. Halves and rows of 16 lanes are exchanged by permlane
// swaps; within a row a rotation by 8, then 4, 2, 1 reaches the partner, because what is left repeats with that period.
template <typename V>
struct Words {
  unsigned w[sizeof(V) / 4];
};
template <int BIT, typename V, typename Op>
__device__ __forceinline__ V combine_bit(V x, Op op) {
  constexpr int N = sizeof(V) / 4, kRowRor = 0x120;
  Words<V> a = __builtin_bit_cast(Words<V>, x), b = a;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if constexpr (BIT >= 16) {
      const u32x2 r = BIT == 32 ? __builtin_amdgcn_permlane32_swap(a.w[i], a.w[i], false, false)
                                : __builtin_amdgcn_permlane16_swap(a.w[i], a.w[i], false, false);
      a.w[i] = r[0];
      b.w[i] = r[1];
    } else {
      b.w[i] = __builtin_amdgcn_mov_dpp(a.w[i], kRowRor + BIT, 0xF, 0xF, false);
    }
  }
  return op(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b));
}
template <int FROM, typename V, typename Op>
__device__ __forceinline__ V combine_lanes_from(V x, Op op) {
  if constexpr (FROM <= 32) x = combine_bit<32>(x, op);
  if constexpr (FROM <= 16) x = combine_bit<16>(x, op);
  if constexpr (FROM <= 8) x = combine_bit<8>(x, op);
  if constexpr (FROM <= 4) x = combine_bit<4>(x, op);
  if constexpr (FROM <= 2) x = combine_bit<2>(x, op);
  if constexpr (FROM <= 1) x = combine_bit<1>(x, op);
  return x;
}
template <int FROM>
__device__ __forceinline__ float sum_lanes_from(float x) {
  return combine_lanes_from<FROM>(x, [](float a, float b) { return a + b; });
}

}  // namespace fasth
