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

// The token of column j, or -1 where its number is no row of the vocabulary.
__device__ __forceinline__ int token_at(const void* ids, int id_bits, int j, int vocab) {
  if (!ids) return -1;
  const long long id = id_bits == 64 ? static_cast<const long long*>(ids)[j] : (long long)static_cast<const int*>(ids)[j];
  return id >= 0 && id < vocab ? (int)id : -1;
}

// Workgroups start on the eight XCDs in turn. This order gives each XCD a run of consecutive tiles, so that tiles
// which share cache lines at their edges share an L2.
__device__ __forceinline__ int xcd_run(int block, int blocks) {
  const int x = block & 7, each = blocks >> 3, more = blocks & 7;
  return x * each + (x < more ? x : more) + (block >> 3);
}

// Sum over the lanes of a wave that differ in the bits from FROM (a power of two) up to 32.
template <int FROM>
__device__ __forceinline__ float sum_lanes_from(float x) {
#pragma unroll
  for (int mask = FROM; mask < kWave; mask <<= 1) x += __shfl_xor(x, mask, kWave);
  return x;
}

}  // namespace fasth
