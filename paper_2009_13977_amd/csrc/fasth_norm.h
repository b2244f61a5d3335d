// The residual's addition and the root-mean-square norm of every column, and their gradients.
//
//   S = X + R,   r_j = (mean_i S_ij^2 + eps)^(-1/2),   Y_ij = w_i r_j S_ij
//   with p_ij = w_i dL/dY_ij:   dX_ij = dS_ij + r_j p_ij - S_ij (r_j^3 / d) sum_i p_ij S_ij,   dw_i = sum_j dL/dY_ij r_j S_ij
//   (dS: what reaches S past the norm; dL/dR = dL/dX)
//
// Bound by memory: a workgroup holds all d rows of a few neighbouring columns in registers, so that every operand is
// read once although the column's sum is needed before its first output.
#pragma once
#include "fasth_columns.h"
#include "fasth_common.h"

namespace fasth {

struct NormArgs {
  const float *X, *R, *w;
  float* S;
  void* Y;
  float* rstd;
  int d, m, tiles;
  float eps;
};

// Sums of VEC columns per thread over all rows: over the wave's row lanes in registers, over the waves in LDS.
// red: [waves][LC * VEC] floats; callers alternate between two so that one barrier per sum is enough.
template <int LC, int VEC>
__device__ __forceinline__ void sum_rows(float (&s)[VEC], float* red) {
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int cl = threadIdx.x % LC;
#pragma unroll
  for (int e = 0; e < VEC; ++e) s[e] = sum_lanes_from<LC>(s[e]);
  if (waves == 1) return;
  if (lane < LC) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) red[wave * (LC * VEC) + cl * VEC + e] = s[e];
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < VEC; ++e) s[e] = 0.f;
  for (int w = 0; w < waves; ++w) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) s[e] += red[w * (LC * VEC) + cl * VEC + e];
  }
}

// LC lanes x VEC columns wide, U rows per thread (blockDim.x / LC rows apart).
template <typename T, int LC, int VEC, int U>
__global__ void __launch_bounds__(1024) norm_kernel(NormArgs a) {
  __shared__ float red[16 * LC * VEC];
  const int rl = threadIdx.x / LC, cl = threadIdx.x % LC, step = blockDim.x / LC;
  const int j = (xcd_run(blockIdx.x, a.tiles) * LC + cl) * VEC, left = a.m - j;
  Cols<float, VEC> s[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = rl + u * step;
    s[u] = load_cols<float, VEC>(a.X + (size_t)i * a.m + j, i < a.d ? left : 0);
  }
  if (a.R) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = rl + u * step;
      const Cols<float, VEC> r = load_cols<float, VEC>(a.R + (size_t)i * a.m + j, i < a.d ? left : 0);
#pragma unroll
      for (int e = 0; e < VEC; ++e) s[u].set(e, s[u].get(e) + r.get(e));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = rl + u * step;
      store_cols<float, VEC>(a.S + (size_t)i * a.m + j, i < a.d ? left : 0, s[u]);
    }
  }
  float q[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) q[e] = 0.f;
#pragma unroll
  for (int u = 0; u < U; ++u) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) q[e] += s[u].get(e) * s[u].get(e);
  }
  sum_rows<LC, VEC>(q, red);
#pragma unroll
  for (int e = 0; e < VEC; ++e) q[e] = 1.f / sqrtf(q[e] / (float)a.d + a.eps);
  if (rl == 0) {
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (e < left) a.rstd[j + e] = q[e];
  }
  T* Y = static_cast<T*>(a.Y);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = rl + u * step;
    const float w = i < a.d ? a.w[i] : 0.f;
    Cols<T, VEC> y;
#pragma unroll
    for (int e = 0; e < VEC; ++e) y.set(e, s[u].get(e) * q[e] * w);
    store_cols<T, VEC>(Y + (size_t)i * a.m + j, i < a.d ? left : 0, y);
  }
}

struct NormGradArgs {
  const void* G;
  const float *S, *w, *rstd, *dS;
  float *dX, *part;  // part: [workgroups][d], a workgroup's share of dw; dw itself for one workgroup; null: not wanted
  int d, m, tiles;
};

// A workgroup takes every gridDim.x-th tile of columns and keeps its share of dw in registers until the last one.
template <typename T, int LC, int VEC, int U>
__global__ void __launch_bounds__(1024) norm_grad_kernel(NormGradArgs a) {
  __shared__ float red[2][16 * LC * VEC];
  const int rl = threadIdx.x / LC, cl = threadIdx.x % LC, step = blockDim.x / LC;
  const T* G = static_cast<const T*>(a.G);
  float dw[U];
#pragma unroll
  for (int u = 0; u < U; ++u) dw[u] = 0.f;
  int odd = 0;
  for (int tile = xcd_run(blockIdx.x, gridDim.x); tile < a.tiles; tile += gridDim.x, odd ^= 1) {
    const int j = (tile * LC + cl) * VEC, left = a.m - j;
    Cols<float, VEC> s[U];
    Cols<T, VEC> g[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = rl + u * step;
      s[u] = load_cols<float, VEC>(a.S + (size_t)i * a.m + j, i < a.d ? left : 0);
      g[u] = load_cols<T, VEC>(G + (size_t)i * a.m + j, i < a.d ? left : 0);
    }
    float q[VEC], r[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      q[e] = 0.f;
      r[e] = e < left ? a.rstd[j + e] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = rl + u * step;
      const float w = i < a.d ? a.w[i] : 0.f;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float gs = g[u].get(e) * s[u].get(e);
        q[e] += w * gs;
        dw[u] += gs * r[e];
      }
    }
    sum_rows<LC, VEC>(q, red[odd]);
#pragma unroll
    for (int e = 0; e < VEC; ++e) q[e] *= r[e] * r[e] * r[e] / (float)a.d;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = rl + u * step, here = i < a.d ? left : 0;
      const float w = i < a.d ? a.w[i] : 0.f;
      Cols<float, VEC> x;
      if (a.dS) x = load_cols<float, VEC>(a.dS + (size_t)i * a.m + j, here);
      else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) x.set(e, 0.f);
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) x.set(e, x.get(e) + r[e] * w * g[u].get(e) - s[u].get(e) * q[e]);
      store_cols<float, VEC>(a.dX + (size_t)i * a.m + j, here, x);
    }
  }
  if (!a.part) return;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = rl + u * step;
#pragma unroll
    for (int mask = 1; mask < LC; mask <<= 1) dw[u] += __shfl_xor(dw[u], mask, kWave);
    if (cl == 0 && i < a.d) a.part[(size_t)blockIdx.x * a.d + i] = dw[u];
  }
}

// dw from the workgroups' shares, in a fixed order: 64 rows per workgroup, every 16th share per wave.
__global__ void __launch_bounds__(1024) norm_weight_kernel(const float* __restrict__ part, int parts, int d, float* __restrict__ dw) {
  __shared__ float red[16][kWave];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6, i = blockIdx.x * kWave + lane;
  float s = 0.f;
  if (i < d) {
#pragma unroll 8
    for (int p = wave; p < parts; p += 16) s += part[(size_t)p * d + i];
  }
  red[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && i < d) {
    s = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) s += red[w][lane];
    dw[i] = s;
  }
}

constexpr int kNormMaxParts = 2 * kComputeUnits;

static size_t norm_workspace(const fasth_norm_shape& s) {
  return align_up((size_t)kNormMaxParts * s.d * sizeof(float), 256);
}

// How a launch covers d rows: LC lanes of VEC columns, `threads` threads of up to U rows each.
struct NormPlan { int lc, vec, u, threads, tiles; };
static NormPlan plan_norm(int d, int m, int u_wide, int lc_wide) {
  NormPlan p;
  p.vec = m >= 4 ? 4 : 1;
  p.u = u_wide;
  p.lc = p.vec == 4 ? lc_wide : 1;
  while (p.lc > 1 && (d + p.u - 1) / p.u * p.lc > 1024) p.lc /= 2;
  while (p.lc > 1 && (m + p.lc * p.vec - 1) / (p.lc * p.vec) < kComputeUnits) p.lc /= 2;
  if ((d + p.u - 1) / p.u * p.lc > 1024) p.u = 16;
  p.threads = std::max(kWave, (int)align_up((size_t)((d + p.u - 1) / p.u) * p.lc, kWave));
  p.tiles = (m + p.lc * p.vec - 1) / (p.lc * p.vec);
  return p;
}

#define FASTH_NORM_CASE(KERNEL, LC_, VEC_, U_)                                                     \
  if (p.lc == LC_ && p.vec == VEC_ && p.u == U_) {                                                 \
    hipLaunchKernelGGL((KERNEL<T, LC_, VEC_, U_>), dim3(grid), dim3(p.threads), 0, stream, a);     \
    FASTH_HIP(hipGetLastError());                                                                  \
    return FASTH_OK;                                                                               \
  }

template <typename T>
static int launch_norm(const NormArgs& args, hipStream_t stream) {
  const NormPlan p = plan_norm(args.d, args.m, 16, 4);
  NormArgs a = args;
  a.tiles = p.tiles;
  const int grid = p.tiles;
  FASTH_NORM_CASE(norm_kernel, 4, 4, 16)
  FASTH_NORM_CASE(norm_kernel, 2, 4, 16)
  FASTH_NORM_CASE(norm_kernel, 1, 4, 16)
  FASTH_NORM_CASE(norm_kernel, 1, 1, 16)
  return FASTH_EUNSUPPORTED;
}

template <typename T>
static int launch_norm_grad(const NormGradArgs& args, float* dweight, void* workspace, hipStream_t stream) {
  const NormPlan p = plan_norm(args.d, args.m, 8, 4);
  NormGradArgs a = args;
  a.tiles = p.tiles;
  const int grid = std::min(p.tiles, kNormMaxParts);
  a.part = !dweight ? nullptr : grid == 1 ? dweight : static_cast<float*>(workspace);
  auto main_pass = [&]() -> int {
    FASTH_NORM_CASE(norm_grad_kernel, 4, 4, 8)
    FASTH_NORM_CASE(norm_grad_kernel, 2, 4, 8)
    FASTH_NORM_CASE(norm_grad_kernel, 1, 4, 8)
    FASTH_NORM_CASE(norm_grad_kernel, 1, 1, 8)
    FASTH_NORM_CASE(norm_grad_kernel, 1, 4, 16)
    FASTH_NORM_CASE(norm_grad_kernel, 1, 1, 16)
    return FASTH_EUNSUPPORTED;
  };
  const int rc = main_pass();
  if (rc != FASTH_OK || !dweight || grid == 1) return rc;
  hipLaunchKernelGGL(norm_weight_kernel, dim3((a.d + kWave - 1) / kWave), dim3(1024), 0, stream, static_cast<const float*>(workspace),
                     grid, a.d, dweight);
  FASTH_HIP(hipGetLastError());
  return FASTH_OK;
}

}  // namespace fasth
