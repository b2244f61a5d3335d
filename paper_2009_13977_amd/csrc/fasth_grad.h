// The global norm over a list of gradients, and the gradients scaled so that it stays below a limit.
//
//   N = (sum over all entries of all tensors g^2)^(1/2),   out = g * (N > limit ? limit / N : 1)
//
// Bound by memory: all gradients are read for the norm and once more for the scaling (608 MB fp32 and bf16: 106 us, 5.7 TB/s,
// and 179 us, 6.8 TB/s, some of it from the last level cache; 100 MB: 18 and 31 us; in place the same). Squares are summed in fp64: the
// vector units have time to spare at this rate, no square of an fp32 number overflows, and the result does not depend on
// how many entries there are.
#pragma once
#include "fasth_columns.h"
#include "fasth_common.h"

namespace fasth {

constexpr int kGradItems = 96;      // tensors per launch: their descriptions are the kernel's arguments (at most 4 KiB)
constexpr int kGradChunk = 8192;    // entries of a tensor that a workgroup takes at a time
constexpr int kGradThreads = 256;
constexpr int kGradGroups = 8 * kComputeUnits;  // workgroups of a launch at most, each with one partial sum
// Chunks from which the clip kernel's workgroups take one each, because a wave waits for its stores before it can use what
// it loads next; the norm is then finished by a launch of its own (4.7 us), else by every workgroup for itself (608 MB: 223
// and 213 us; with reads past the caches 176 us; 100 MB, 3096 chunks: 34 us and a launch more). Also lists of several
// launches, so that no workgroup adds more than one launch's partial sums.
constexpr int kGradLarge = 4 * kGradGroups;
constexpr int kGradMaxGroups = 1 << 23;         // (workgroups x 256 threads fit 32 bits)
constexpr unsigned long long kGradMaxCount = 1ull << 36;  // entries of one tensor: the chunks of a launch fit an int

struct GradItem {
  const void* src;
  void* dst;
  unsigned long long n;
  int first;  // chunks of the launch's tensors before this one
  int dtype;
};
struct GradArgs {
  GradItem item[kGradItems];
  int items, chunks;
  double* part;  // this launch's partial sums (norm), all partial sums (clip)
  int parts;
  float limit;
  float* norm;
};

__device__ __forceinline__ const GradItem& item_of(const GradArgs& a, int chunk) {
  int lo = 0, hi = a.items;  // the last item whose first chunk is not beyond
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.item[mid].first <= chunk) lo = mid;
    else hi = mid;
  }
  return a.item[lo];
}

template <typename T>
__device__ __forceinline__ double square_sum(const void* src, unsigned long long n) {
  constexpr int VEC = 16 / sizeof(T), STEP = kGradThreads * VEC;
  const T* p = static_cast<const T*>(src);
  double s[4] = {0., 0., 0., 0.};  // (one sum would wait for itself)
  if (n == kGradChunk) {
    Cols<T, VEC> x[kGradChunk / STEP];
#pragma unroll
    for (int k = 0; k < kGradChunk / STEP; ++k) x[k] = load_cols<T, VEC>(p + k * STEP + threadIdx.x * VEC, VEC);
#pragma unroll
    for (int k = 0; k < kGradChunk / STEP; ++k) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) s[e & 3] += (double)x[k].get(e) * (double)x[k].get(e);
    }
  } else {
    for (unsigned k = threadIdx.x; k < n; k += kGradThreads) s[0] += (double)(float)p[k] * (double)(float)p[k];
  }
  return (s[0] + s[1]) + (s[2] + s[3]);
}
// F: the type of the factor and the product
template <typename T, typename F>
__device__ __forceinline__ void scale_chunk(const void* src, void* dst, unsigned long long n, F c) {
  constexpr int VEC = 16 / sizeof(T), STEP = kGradThreads * VEC;
  const T* p = static_cast<const T*>(src);
  T* o = static_cast<T*>(dst);
  if (n == kGradChunk) {
    Cols<T, VEC> x[kGradChunk / STEP];
#pragma unroll
    for (int k = 0; k < kGradChunk / STEP; ++k) {
      const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + k * STEP + threadIdx.x * VEC));
      __builtin_memcpy(&x[k].v, &w, 16);
    }
#pragma unroll
    for (int k = 0; k < kGradChunk / STEP; ++k) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[k].set(e, (float)((F)x[k].get(e) * c));
      __builtin_nontemporal_store(__builtin_bit_cast(u32x4, x[k].v), reinterpret_cast<u32x4*>(o + k * STEP + threadIdx.x * VEC));
    }
  } else {
    for (unsigned k = threadIdx.x; k < n; k += kGradThreads) o[k] = (T)(float)((F)(float)p[k] * c);
  }
}

// Sum over the workgroup, the same bits in every thread.
__device__ __forceinline__ double sum_threads(double s, double* red) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
#pragma unroll
  for (int mask = 1; mask < kWave; mask <<= 1) s += __shfl_xor(s, mask, kWave);
  if (lane == 0) red[wave] = s;
  __syncthreads();
  s = 0.;
#pragma unroll
  for (int w = 0; w < kGradThreads / kWave; ++w) s += red[w];
  return s;
}

__global__ void __launch_bounds__(kGradThreads) grad_norm_kernel(GradArgs a) {
  __shared__ double red[kGradThreads / kWave];
  double s = 0.;
  for (int c = blockIdx.x; c < a.chunks; c += gridDim.x) {
    const GradItem& it = item_of(a, c);
    const unsigned long long at = (unsigned long long)(c - it.first) * kGradChunk, n = min(it.n - at, (unsigned long long)kGradChunk);
    if (it.dtype == FASTH_F32) s += square_sum<float>(static_cast<const float*>(it.src) + at, n);
    else if (it.dtype == FASTH_BF16) s += square_sum<bf16_t>(static_cast<const bf16_t*>(it.src) + at, n);
    else s += square_sum<f16_t>(static_cast<const f16_t*>(it.src) + at, n);
  }
  s = sum_threads(s, red);
  if (threadIdx.x == 0) a.part[blockIdx.x] = s;
}

// All workgroups add the partial sums in the same order, so all have the same bits.
__device__ __forceinline__ double sum_parts(const GradArgs& a, double* red) {
  double s = 0.;
  for (int p = threadIdx.x; p < a.parts; p += kGradThreads) s += a.part[p];
  return sum_threads(s, red);
}

// The norm, and the partial sums' sum in the place of the first (sum_threads' barrier stands between its reading and that).
__global__ void __launch_bounds__(kGradThreads) grad_finish_kernel(GradArgs a) {
  __shared__ double red[kGradThreads / kWave];
  const double s = sum_parts(a, red);
  if (threadIdx.x == 0) {
    a.norm[0] = (float)sqrt(s);
    a.part[0] = s;
  }
}

__global__ void __launch_bounds__(kGradThreads) grad_clip_kernel(GradArgs a) {
  __shared__ double red[kGradThreads / kWave];
  const double n = sqrt(sum_parts(a, red));
  if (a.norm && blockIdx.x == 0 && threadIdx.x == 0) a.norm[0] = (float)n;
  // a norm that reads infinite (also a finite one beyond fp32's range) or NaN leaves the gradients as they are
  const double f = n > (double)a.limit && (float)n < INFINITY ? (double)a.limit / n : 1.;
  auto scale = [&](auto c) {
    for (int k = blockIdx.x; k < a.chunks; k += gridDim.x) {
      const GradItem& it = item_of(a, k);
      if (c == 1 && it.src == it.dst) continue;
      const unsigned long long at = (unsigned long long)(k - it.first) * kGradChunk, n = min(it.n - at, (unsigned long long)kGradChunk);
      if (it.dtype == FASTH_F32) scale_chunk<float>(static_cast<const float*>(it.src) + at, static_cast<float*>(it.dst) + at, n, c);
      else if (it.dtype == FASTH_BF16) scale_chunk<bf16_t>(static_cast<const bf16_t*>(it.src) + at, static_cast<bf16_t*>(it.dst) + at, n, c);
      else scale_chunk<f16_t>(static_cast<const f16_t*>(it.src) + at, static_cast<f16_t*>(it.dst) + at, n, c);
    }
  };
  if (f < 0x1p-126) scale(f);  // in fp32 a subnormal factor would be a few bits, or zero
  else scale((float)f);
}

// Launches that a list needs: kGradItems tensors each.
static int grad_launches(int n) { return std::max(1, (n + kGradItems - 1) / kGradItems); }
static size_t grad_workspace(int n) { return align_up((size_t)grad_launches(n) * kGradGroups * sizeof(double), 256); }

// The norm, and (clip) the scaled gradients into `out`, or in place where it is null.
static int launch_grads(const fasth_tensor* tensors, void* const* out, int n, bool clip, float limit, float* norm, void* workspace,
                        hipStream_t stream) {
  const int launches = grad_launches(n);
  GradArgs a;
  auto describe = [&](int launch) {
    a.items = std::min(kGradItems, n - launch * kGradItems);
    a.chunks = 0;
    for (int i = 0; i < a.items; ++i) {
      const fasth_tensor& t = tensors[launch * kGradItems + i];
      a.item[i] = {t.data, out ? out[launch * kGradItems + i] : t.data, (unsigned long long)t.count, a.chunks, t.dtype};
      a.chunks += (int)((t.count + kGradChunk - 1) / kGradChunk);
    }
  };
  int parts = 0;
  bool large = launches > 1;
  a.limit = limit;
  a.parts = 0;
  a.norm = nullptr;
  for (int l = 0; l < launches; ++l) {
    describe(l);
    const int groups = std::max(1, std::min(a.chunks, kGradGroups));
    large |= a.chunks > kGradLarge;
    a.part = static_cast<double*>(workspace) + parts;
    hipLaunchKernelGGL(grad_norm_kernel, dim3(groups), dim3(kGradThreads), 0, stream, a);
    FASTH_HIP(hipGetLastError());
    parts += groups;
  }
  a.part = static_cast<double*>(workspace);
  a.parts = parts;
  a.norm = norm;
  if (!clip || large) {
    hipLaunchKernelGGL(grad_finish_kernel, dim3(1), dim3(kGradThreads), 0, stream, a);
    FASTH_HIP(hipGetLastError());
    a.parts = 1;
    a.norm = nullptr;
  }
  for (int l = 0; clip && l < launches; ++l) {
    describe(l);
    const int groups = std::max(1, std::min(a.chunks, large ? kGradMaxGroups : kGradGroups));
    hipLaunchKernelGGL(grad_clip_kernel, dim3(groups), dim3(kGradThreads), 0, stream, a);
    FASTH_HIP(hipGetLastError());
    a.norm = nullptr;
  }
  return FASTH_OK;
}

}  // namespace fasth
