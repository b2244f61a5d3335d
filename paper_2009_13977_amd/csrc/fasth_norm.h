// The residual's addition and the root-mean-square norm of every column, and their gradients.
//
//   S = X + R,   r_j = (mean_i S_ij^2 + eps)^(-1/2),   Y_ij = w_i r_j S_ij
//   with p_ij = w_i dL/dY_ij and u_ij = r_j S_ij:   dX_ij = dS_ij + r_j (p_ij - u_ij (sum_i p_ij u_ij) / d),   dw_i = sum_j dL/dY_ij u_ij
//   (dS: what reaches S past the norm; dL/dR = dL/dX)
//
// u is of order one in columns of any size, while r^3 leaves the range of fp32 for columns above some 1e12 and below 1e-12.
//
// Bound by memory: a column's sum is needed before its first output. Either a workgroup holds all rows of some columns in
// registers and reads every operand once, or the rows are split over workgroups and some operands are read twice.
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
  int splits, rows;  // rows split over workgroups: how often, rows each
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

// One pass: a thread keeps U rows of LC lanes x VEC columns in registers, rl, rl + step, rl + 2 step ... Rows beyond the last
// one lie beyond the end of their buffer (no row number exceeds 16384, and so no offset 32 bits).
template <typename T, int LC, int VEC, int U>
__global__ void __launch_bounds__(1024) norm_kernel(NormArgs a) {
  __shared__ float red[16 * LC * VEC];
  constexpr int N = 4;  // rows of R in flight beside all of X: more would not fit the registers
  const int rl = threadIdx.x / LC, cl = threadIdx.x % LC, step = blockDim.x / LC;
  const int tile = xcd_run(blockIdx.x, a.tiles);
  const ColumnRange<VEC> cols((tile * LC + cl) * VEC, a.m, tile == a.tiles - 1);
  const size_t all = (size_t)a.d * a.m;
  const unsigned own = (unsigned)rl * a.m + cols.first, jump = (unsigned)step * a.m;  // in elements
  const BufferDesc X = whole(a.X, 4 * all), W = whole(a.w, 4 * (size_t)a.d);
  Cols<float, VEC> s[U];
  float w[U];
  const unsigned x_own = again(own);
#pragma unroll
  for (int u = 0; u < U; ++u) s[u] = load_from<float, VEC>(X, (x_own + u * jump) * 4);
#pragma unroll
  for (int u = 0; u < U; ++u) w[u] = load_from<float, 1>(W, (unsigned)(rl + u * step) * 4).v;
  if (a.R) {
    const BufferDesc R = whole(a.R, 4 * all), S = whole(a.S, 4 * all);
    const unsigned r_own = again(own);
#pragma unroll
    for (int u0 = 0; u0 < U; u0 += N) {
      Cols<float, VEC> r[N];
#pragma unroll
      for (int n = 0; n < N; ++n) r[n] = load_from<float, VEC>(R, (r_own + (u0 + n) * jump) * 4);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < N; ++n) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) s[u0 + n].set(e, s[u0 + n].get(e) + r[n].get(e));
      }
    }
    const unsigned s_own = again(own);
    auto write = [&](auto full) {
#pragma unroll
      for (int u = 0; u < U; ++u) cols.template store<decltype(full)::value>(S, (s_own + u * jump) * 4, s[u]);
    };
    if (cols.ragged) write(std::false_type());
    else write(std::true_type());
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
      if (cols.own(e)) a.rstd[cols.first + e] = q[e];
  }
  const BufferDesc Y = whole(a.Y, sizeof(T) * all);
  const unsigned y_own = again(own);
  auto write = [&](auto full) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      Cols<T, VEC> y;
#pragma unroll
      for (int e = 0; e < VEC; ++e) y.set(e, s[u].get(e) * q[e] * w[u]);
      cols.template store<decltype(full)::value>(Y, (y_own + u * jump) * (unsigned)sizeof(T), y);
    }
  };
  if (cols.ragged) write(std::false_type());
  else write(std::true_type());
}

// The same over tiles of LC x 4 columns with the rows split over workgroups: the columns' sums of squares of every split
// (and S), their sum, then the outputs (4096 x 8192 fp32: 69 us for 403 MB, 5 us, 43 us for 268 MB). S is read
// twice, the second time from the last level cache where it fits, but whole cache lines are read and written by one
// workgroup, and any number of columns fills the GPU. The sums wait in Y,
// which the last pass overwrites: [splits][m] fp32 from its start, two rows of Y in 16 bits each. split_norm makes no
// more than d / 2 splits (a split has 64 rows and more, so that is far off), and fewer than two rows never come here.
constexpr int kNormThreads = 256;
constexpr int kNormSplits = 32;
template <int LC, int HOW = 0>
__global__ void __launch_bounds__(kNormThreads) norm_sum_kernel(NormArgs a) {
  constexpr int VEC = 4, U = 8, RL = kNormThreads / LC;
  __shared__ float red[kNormThreads / kWave * LC * VEC];
  const int rl = threadIdx.x / LC, cl = threadIdx.x % LC;
  const TileAt tile(a.tiles);
  const ColumnRange<VEC> cols((tile.col * LC + cl) * VEC, a.m, tile.col == a.tiles - 1);
  const size_t all = (size_t)a.d * a.m;
  const int row0 = tile.row * a.rows, row1 = min(a.d, row0 + a.rows);
  const BufferDesc X = whole(a.X, 4 * all), R = whole(a.R, a.R ? 4 * all : 0), S = whole(a.S, a.S ? 4 * all : 0);
  const unsigned jump = (unsigned)RL * a.m;
  float q[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) q[e] = 0.f;
  for (int row = row0; row < row1; row += RL * U) {
    const unsigned own = again((unsigned)(row + rl) * a.m + cols.first);
    Cols<float, VEC> s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) s[u] = load_from<float, VEC, HOW>(X, (own + u * jump) * 4);
    if (a.R) {
      Cols<float, VEC> r[U];
#pragma unroll
      for (int u = 0; u < U; ++u) r[u] = load_from<float, VEC, HOW>(R, (own + u * jump) * 4);
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) s[u].set(e, s[u].get(e) + r[u].get(e));
      }
      if (cols.ragged) {
#pragma unroll
        for (int u = 0; u < U; ++u) cols.template store<false>(S, (own + u * jump) * 4, s[u]);
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u) cols.template store<true>(S, (own + u * jump) * 4, s[u]);
      }
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      float t = 0.f;  // a sum of U terms at a time: fewer roundings in a row
#pragma unroll
      for (int u = 0; u < U; ++u) t += s[u].get(e) * s[u].get(e);
      q[e] += t;
    }
  }
  sum_rows<LC, VEC>(q, red);
  if (rl == 0) {
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (cols.own(e)) static_cast<float*>(a.Y)[(size_t)tile.row * a.m + cols.first + e] = q[e];
  }
}

__global__ void __launch_bounds__(kNormThreads) norm_root_kernel(NormArgs a) {
  const int j = blockIdx.x * kNormThreads + threadIdx.x;
  if (j >= a.m) return;
  const float* part = static_cast<const float*>(a.Y) + j;
  float q = 0.f;
#pragma unroll 8
  for (int k = 0; k < a.splits; ++k) q += part[(size_t)k * a.m];
  a.rstd[j] = 1.f / sqrtf(q / (float)a.d + a.eps);
}

// A column's sum over the splits, for the VEC columns of a thread.
template <int VEC>
__device__ __forceinline__ void sum_splits(float (&q)[VEC], const float* part, int splits, int m, int first) {
  const BufferDesc P = whole(part, 4 * (size_t)splits * m);
#pragma unroll
  for (int e = 0; e < VEC; ++e) q[e] = 0.f;
#pragma unroll 8
  for (int s = 0; s < splits; ++s) {
    const Cols<float, VEC> c = load_from<float, VEC>(P, ((unsigned)s * m + first) * 4);
#pragma unroll
    for (int e = 0; e < VEC; ++e) q[e] += c.get(e);
  }
}

template <typename T, int LC>
__global__ void __launch_bounds__(kNormThreads) norm_scale_kernel(NormArgs a) {
  constexpr int VEC = 4, U = 8, RL = kNormThreads / LC;
  const int rl = threadIdx.x / LC, cl = threadIdx.x % LC;
  const TileAt tile(a.tiles);
  const ColumnRange<VEC> cols((tile.col * LC + cl) * VEC, a.m, tile.col == a.tiles - 1);
  const int row0 = tile.row * a.rows, row1 = min(a.d, row0 + a.rows);
  const size_t all = (size_t)a.d * a.m;
  const BufferDesc S = whole(a.R ? a.S : a.X, 4 * all), Y = whole(a.Y, sizeof(T) * all), W = whole(a.w, 4 * (size_t)a.d);
  const unsigned jump = (unsigned)RL * a.m;
  const Cols<float, VEC> rstd = load_from<float, VEC>(whole(a.rstd, 4 * (size_t)a.m), (unsigned)cols.first * 4);
  for (int row = row0; row < row1; row += RL * U) {
    const unsigned own = again((unsigned)(row + rl) * a.m + cols.first);
    Cols<float, VEC> s[U];
    float w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      s[u] = load_from<float, VEC>(S, (own + u * jump) * 4);
      w[u] = load_from<float, 1>(W, (unsigned)(row + rl + u * RL) * 4).v;
    }
    auto write = [&](auto full) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        Cols<T, VEC> y;
#pragma unroll
        for (int e = 0; e < VEC; ++e) y.set(e, s[u].get(e) * rstd.get(e) * w[u]);
        cols.template store<decltype(full)::value>(Y, (own + u * jump) * (unsigned)sizeof(T), y);
      }
    };
    if (cols.ragged) write(std::false_type());
    else write(std::true_type());
  }
}

struct NormGradArgs {
  const void* G;
  const float *S, *w, *rstd, *dS;
  float *dX, *part;  // part: [workgroups (two passes: tiles)][d], shares of dw; dw itself for one of them; null: not wanted
  float* sums;       // two passes: [splits][m]
  int d, m, tiles;
  int rows;          // two passes: rows per split
};

// A workgroup takes every gridDim.x-th tile of columns and keeps its share of dw in registers until the last one.
template <typename T, int LC, int VEC, int U>
__global__ void __launch_bounds__(1024) norm_grad_kernel(NormGradArgs a) {
  __shared__ float red[2][16 * LC * VEC];
  constexpr int N = U < 4 ? U : 4;  // rows of dS in flight beside S and G (a store may be to where the next load is from)
  const int rl = threadIdx.x / LC, cl = threadIdx.x % LC, step = blockDim.x / LC;
  const size_t all = (size_t)a.d * a.m;
  const unsigned jump = (unsigned)step * a.m;  // in elements
  const BufferDesc W = whole(a.w, 4 * (size_t)a.d), RSTD = whole(a.rstd, 4 * (size_t)a.m), S = whole(a.S, 4 * all), G = whole(a.G, sizeof(T) * all),
                   DS = whole(a.dS, 4 * all), DX = whole(a.dX, 4 * all);
  float dw[U];
#pragma unroll
  for (int u = 0; u < U; ++u) dw[u] = 0.f;
  int odd = 0;
  for (int tile = xcd_run(blockIdx.x, gridDim.x); tile < a.tiles; tile += gridDim.x, odd ^= 1) {
    const ColumnRange<VEC> cols((tile * LC + cl) * VEC, a.m, tile == a.tiles - 1);
    const unsigned own = (unsigned)rl * a.m + cols.first;
    float q[VEC], r[VEC];
    Cols<float, VEC> s[U], p[U];  // p = w dL/dY
    const unsigned in_own = again(own), w_row = again(rl);
    {
      Cols<T, VEC> g[U];
      float w[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        g[u] = load_from<T, VEC>(G, (in_own + u * jump) * (unsigned)sizeof(T));
        s[u] = load_from<float, VEC>(S, (in_own + u * jump) * 4);
        w[u] = load_from<float, 1>(W, (w_row + u * step) * 4).v;
      }
      const Cols<float, VEC> rstd = load_from<float, VEC>(RSTD, (unsigned)cols.first * 4);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        q[e] = 0.f;
        r[e] = rstd.get(e);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          s[u].set(e, s[u].get(e) * r[e]);  // u from here on
          const float gu = g[u].get(e) * s[u].get(e);
          q[e] += w[u] * gu;
          dw[u] += cols.own(e) ? gu : 0.f;
          p[u].set(e, w[u] * g[u].get(e));
        }
      }
    }
    sum_rows<LC, VEC>(q, red[odd]);
#pragma unroll
    for (int e = 0; e < VEC; ++e) q[e] /= (float)a.d;
    const unsigned out_own = again(own);
    auto write = [&](auto full, auto more) {
#pragma unroll
      for (int u0 = 0; u0 < U; u0 += N) {
        Cols<float, VEC> ds[N];
        if constexpr (decltype(more)::value) {
#pragma unroll
          for (int n = 0; n < N; ++n) ds[n] = load_from<float, VEC>(DS, (out_own + (u0 + n) * jump) * 4);
          __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int n = 0; n < N; ++n) {
          const int u = u0 + n;
          Cols<float, VEC> x;
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const float t = r[e] * (p[u].get(e) - s[u].get(e) * q[e]);
            x.set(e, decltype(more)::value ? ds[n].get(e) + t : t);
          }
          cols.template store<decltype(full)::value>(DX, (out_own + u * jump) * 4, x);
        }
      }
    };
    if (cols.ragged) {
      if (a.dS) write(std::false_type(), std::true_type());
      else write(std::false_type(), std::false_type());
    } else {
      if (a.dS) write(std::true_type(), std::true_type());
      else write(std::true_type(), std::false_type());
    }
  }
  if (!a.part) return;
  const BufferDesc part = whole(a.part + (size_t)blockIdx.x * a.d, 4 * (size_t)a.d);
  const unsigned dw_row = cl == 0 ? again(rl) * 4 : kBeyond;
#pragma unroll
  for (int u = 0; u < U; ++u) {
#pragma unroll
    for (int mask = 1; mask < LC; mask <<= 1) dw[u] += __shfl_xor(dw[u], mask, kWave);
    store_to<float, 1>(part, cl == 0 ? dw_row + u * step * 4 : kBeyond, Cols<float, 1>{dw[u]});
  }
}

// The two passes of the gradient: column sums of p u per split and row sums for dw per tile of columns, then dX. Bound by
// memory: 4096 x 8192 fp32 45 us for 268 MB, 6.0 TB/s, and 82 us for 537 MB, 6.5 TB/s, where part of S and G is still in
// the last level cache.
template <typename T, int LC>
__global__ void __launch_bounds__(kNormThreads) norm_grad_sum_kernel(NormGradArgs a) {
  constexpr int VEC = 4, U = 4, RL = kNormThreads / LC;
  __shared__ float red[kNormThreads / kWave * LC * VEC];
  const int rl = threadIdx.x / LC, cl = threadIdx.x % LC;
  const TileAt tile(a.tiles);
  const ColumnRange<VEC> cols((tile.col * LC + cl) * VEC, a.m, tile.col == a.tiles - 1);
  const int row0 = tile.row * a.rows, row1 = min(a.d, row0 + a.rows);
  const size_t all = (size_t)a.d * a.m;
  const BufferDesc S = whole(a.S, 4 * all), G = whole(a.G, sizeof(T) * all), W = whole(a.w, 4 * (size_t)a.d),
                   RSTD = whole(a.rstd, 4 * (size_t)a.m), DW = whole(a.part + (size_t)tile.col * a.d, a.part ? 4 * (size_t)a.d : 0);
  const unsigned jump = (unsigned)RL * a.m;
  const Cols<float, VEC> rstd = load_from<float, VEC>(RSTD, (unsigned)cols.first * 4);
  float q[VEC], r[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    q[e] = 0.f;
    r[e] = rstd.get(e);
  }
  for (int row = row0; row < row1; row += RL * U) {
    const unsigned own = again((unsigned)(row + rl) * a.m + cols.first);
    Cols<float, VEC> s[U];
    Cols<T, VEC> g[U];
    float w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      s[u] = load_from<float, VEC>(S, (own + u * jump) * 4);
      g[u] = load_from<T, VEC>(G, (own + u * jump) * (unsigned)sizeof(T));
      w[u] = load_from<float, 1>(W, (unsigned)(row + rl + u * RL) * 4).v;
    }
    float t[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) t[e] = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float dw = 0.f;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float gu = g[u].get(e) * (s[u].get(e) * r[e]);
        t[e] += w[u] * gu;
        dw += cols.own(e) ? gu : 0.f;
      }
      constexpr int kRowRor = 0x120;  // (rotations in a row of 16 lanes: what is left repeats with that period)
      if constexpr (LC == 32) dw = swap16_sum(dw, dw);
      if constexpr (LC >= 16) dw += dpp_move<kRowRor + 8>(dw);
      if constexpr (LC >= 16) dw += dpp_move<kRowRor + 4>(dw);
      dw += dpp_move<kDppQuadXor2>(dw);
      dw += dpp_move<kDppQuadXor1>(dw);
      store_to<float, 1>(DW, cl == 0 ? (unsigned)(row + rl + u * RL) * 4 : kBeyond, Cols<float, 1>{dw});
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) q[e] += t[e];  // a sum of U terms at a time: fewer roundings in a row
  }
  sum_rows<LC, VEC>(q, red);
  if (rl == 0) {
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (cols.own(e)) a.sums[(size_t)tile.row * a.m + cols.first + e] = q[e];
  }
}

template <typename T, int LC, int HOW = 0>
__global__ void __launch_bounds__(kNormThreads) norm_grad_apply_kernel(NormGradArgs a) {
  constexpr int VEC = 4, U = 4, RL = kNormThreads / LC;
  const int rl = threadIdx.x / LC, cl = threadIdx.x % LC;
  const TileAt tile(a.tiles);
  const ColumnRange<VEC> cols((tile.col * LC + cl) * VEC, a.m, tile.col == a.tiles - 1);
  const int row0 = tile.row * a.rows, row1 = min(a.d, row0 + a.rows);
  const size_t all = (size_t)a.d * a.m;
  const BufferDesc S = whole(a.S, 4 * all), G = whole(a.G, sizeof(T) * all), W = whole(a.w, 4 * (size_t)a.d),
                   RSTD = whole(a.rstd, 4 * (size_t)a.m), DS = whole(a.dS, a.dS ? 4 * all : 0), DX = whole(a.dX, 4 * all);
  const unsigned jump = (unsigned)RL * a.m;
  const Cols<float, VEC> rstd = load_from<float, VEC>(RSTD, (unsigned)cols.first * 4);
  float q[VEC], r[VEC];
  sum_splits<VEC>(q, a.sums, gridDim.x / a.tiles, a.m, cols.first);
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    r[e] = rstd.get(e);
    q[e] /= (float)a.d;
  }
  for (int row = row0; row < row1; row += RL * U) {
    const unsigned own = again((unsigned)(row + rl) * a.m + cols.first);
    Cols<float, VEC> s[U], ds[U];
    Cols<T, VEC> g[U];
    float w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      s[u] = load_from<float, VEC, HOW>(S, (own + u * jump) * 4);
      g[u] = load_from<T, VEC, HOW>(G, (own + u * jump) * (unsigned)sizeof(T));
      ds[u] = load_from<float, VEC, HOW>(DS, (own + u * jump) * 4);  // zeros where there is none
      w[u] = load_from<float, 1>(W, (unsigned)(row + rl + u * RL) * 4).v;
    }
    auto write = [&](auto full) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        Cols<float, VEC> x;
#pragma unroll
        for (int e = 0; e < VEC; ++e) x.set(e, ds[u].get(e) + r[e] * (w[u] * g[u].get(e) - (s[u].get(e) * r[e]) * q[e]));
        cols.template store<decltype(full)::value, HOW>(DX, (own + u * jump) * 4, x);
      }
    };
    if (cols.ragged) write(std::false_type());
    else write(std::true_type());
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

// How a launch covers the mini-batch: in one pass, `threads` threads hold u rows of lc x vec columns each; or split.
//
// Measured (us, forward with a residual / backward, fp32, launched from a graph):
//                        2048 x 5   1024 x 16   784 x 1001  1024 x 2048  512 x 16384  2048 x 4096  2048 x 65535  16384 x 30
//   a lane per column    4.6 / -    4.7 / -     -           -            -            -            -             -
//   one pass, 4 columns  4.7 / -    6.8 / -     8.1 / -     17.0 / -     42.5 / -     45.3 / -     -             70.3 / -
//   one pass, 32 columns 20.5 / -   11.6 / 11.3 12.1 / 13.3 20.2 / 19.6  22.1 / 28.6  40.4 / -     587 / -       -
//   split                8.5 / 6.1  10.0 / 6.7  12.2 / 9.9  13.8 / 13.4  30.1 / 37.4  38.0 / 38.9  657 / 684     11.4 / 11.6
// One pass of 32 columns reads whole cache lines, but needs m / 32 workgroups to fill the GPU and 16 rows per thread at most
// (8 backward, where two matrices are held); one of 4 columns pays only while three launches cost more than its part lines.
struct NormPlan {
  bool split;
  int lc, vec, u, threads, tiles;
  int splits, rows;
};
static NormPlan split_norm(int d, int m, int u) {
  NormPlan p = {};
  p.split = true;
  p.threads = kNormThreads;
  p.lc = m >= 512 ? 32 : m >= 64 ? 16 : 4;
  p.tiles = (m + 4 * p.lc - 1) / (4 * p.lc);
  // (a power of two that divides 16384: no row number beyond that is formed)
  const int step = kNormThreads / p.lc * u, steps = (d + step - 1) / step;
  p.splits = std::max(1, std::min({steps, kNormSplits, 8 * kComputeUnits / p.tiles, d / 2}));  // d / 2: see norm_sum_kernel
  p.rows = (steps + p.splits - 1) / p.splits * step;
  p.splits = (d + p.rows - 1) / p.rows;
  return p;
}
static NormPlan one_pass_norm(int d, int m, int lc, int vec, int u) {
  NormPlan p = {};
  p.lc = lc;
  p.vec = vec;
  p.u = u;
  p.tiles = (m + lc * vec - 1) / (lc * vec);
  p.threads = (int)align_up((size_t)((d + u - 1) / u) * lc, kWave);
  return p;
}
// From 96 MiB per matrix on, what the split kernels need once only goes past the caches, so that S stays there for the
// second pass (us, three mini-batches in turn, with all through the caches and as it is: 4096 x 8192 forward with a residual
// 135 and 122, backward 160 and 132; 4096 x 16384 286 and 277, 334 and 286). Forward only where no cache line lies in two
// workgroups' columns (4099 x 16383: 329, but 348; backward 349 and 334). Up to 192 MiB that also beats one pass
// (2048 x 16384: 147 and 132).
static bool past_caches_backward(int d, int m) { return (int64_t)d * m >= 24 << 20; }
static bool past_caches_forward(int d, int m) { return past_caches_backward(d, m) && m % 32 == 0; }
static NormPlan plan_norm(int d, int m, bool residual) {
  // few columns: a lane per column, so that a wave's rows lie side by side in memory
  const int lanes = m <= 1 ? 1 : m <= 2 ? 2 : m <= 4 ? 4 : m <= 8 ? 8 : 16;
  if (m <= 16 && (int64_t)d * lanes <= 16384) return one_pass_norm(d, m, lanes, 1, 16);
  if (m < 4) return one_pass_norm(d, m, 1, 1, 16);
  const bool kept = residual && past_caches_forward(d, m) && (int64_t)d * m <= 48 << 20;
  if (d <= 2048 && m >= 1024 && m >= 4 * d && !kept) return one_pass_norm(d, m, 8, 4, 16);
  if (d <= 1024 && (int64_t)d * m <= 3 << 19) return one_pass_norm(d, m, 1, 4, 16);
  return split_norm(d, m, 8);
}
static NormPlan plan_norm_grad(int d, int m) {
  if (m < 4) return one_pass_norm(d, m, 1, 1, d <= 8192 ? 8 : 16);
  if (d <= 1024 && m >= 1024 && m >= 8 * d) return one_pass_norm(d, m, 8, 4, 8);
  return split_norm(d, m, 4);
}
constexpr int kNormMaxParts = 2 * kComputeUnits;

struct NormLayout {  // shares of dw, then the splits' column sums
  size_t off_sums, total;
};
static NormLayout norm_layout(int d, int m) {
  NormLayout L;
  L.off_sums = align_up((size_t)std::max(kNormMaxParts, (m + 63) / 64) * d * sizeof(float), 256);
  L.total = L.off_sums + align_up((size_t)kNormSplits * m * sizeof(float), 256);
  return L;
}
static size_t norm_workspace(const fasth_norm_shape& s) { return norm_layout(s.d, s.m).total; }

#define FASTH_NORM_LAUNCH(GRID, ...)                                        \
  do {                                                                       \
    hipLaunchKernelGGL((__VA_ARGS__), GRID, dim3(p.threads), 0, stream, a);  \
    FASTH_HIP(hipGetLastError());                                            \
  } while (0)

template <typename T>
static int launch_norm(const NormArgs& args, hipStream_t stream) {
  const NormPlan p = plan_norm(args.d, args.m, args.R != nullptr);
  NormArgs a = args;
  a.tiles = p.tiles; a.splits = p.splits; a.rows = p.rows;
  if (p.split) {
    const dim3 grid(p.tiles * p.splits);
    if (p.lc == 32 && a.R && past_caches_forward(a.d, a.m)) FASTH_NORM_LAUNCH(grid, norm_sum_kernel<32, kPastCaches>);
    else if (p.lc == 32) FASTH_NORM_LAUNCH(grid, norm_sum_kernel<32>);
    else if (p.lc == 16) FASTH_NORM_LAUNCH(grid, norm_sum_kernel<16>);
    else FASTH_NORM_LAUNCH(grid, norm_sum_kernel<4>);
    FASTH_NORM_LAUNCH(dim3((a.m + kNormThreads - 1) / kNormThreads), norm_root_kernel);
    if (p.lc == 32) FASTH_NORM_LAUNCH(grid, norm_scale_kernel<T, 32>);
    else if (p.lc == 16) FASTH_NORM_LAUNCH(grid, norm_scale_kernel<T, 16>);
    else FASTH_NORM_LAUNCH(grid, norm_scale_kernel<T, 4>);
  } else {
    const dim3 grid(p.tiles);
    if (p.vec == 1 && p.lc == 1) FASTH_NORM_LAUNCH(grid, norm_kernel<T, 1, 1, 16>);
    else if (p.vec == 1 && p.lc == 2) FASTH_NORM_LAUNCH(grid, norm_kernel<T, 2, 1, 16>);
    else if (p.vec == 1 && p.lc == 4) FASTH_NORM_LAUNCH(grid, norm_kernel<T, 4, 1, 16>);
    else if (p.vec == 1 && p.lc == 8) FASTH_NORM_LAUNCH(grid, norm_kernel<T, 8, 1, 16>);
    else if (p.vec == 1) FASTH_NORM_LAUNCH(grid, norm_kernel<T, 16, 1, 16>);
    else if (p.lc == 1) FASTH_NORM_LAUNCH(grid, norm_kernel<T, 1, 4, 16>);
    else FASTH_NORM_LAUNCH(grid, norm_kernel<T, 8, 4, 16>);
  }
  return FASTH_OK;
}

template <typename T>
static int launch_norm_grad(const NormGradArgs& args, float* dweight, void* workspace, hipStream_t stream) {
  const NormPlan p = plan_norm_grad(args.d, args.m);
  NormGradArgs a = args;
  a.tiles = p.tiles; a.rows = p.rows;
  const int parts = p.split ? p.tiles : std::min(p.tiles, kNormMaxParts);
  a.part = !dweight ? nullptr : parts == 1 ? dweight : static_cast<float*>(workspace);
  a.sums = reinterpret_cast<float*>(static_cast<char*>(workspace) + norm_layout(a.d, a.m).off_sums);
  if (p.split) {
    const dim3 grid(p.tiles * p.splits);
    if (p.lc == 32) {
      FASTH_NORM_LAUNCH(grid, norm_grad_sum_kernel<T, 32>);
      if (past_caches_backward(a.d, a.m)) FASTH_NORM_LAUNCH(grid, norm_grad_apply_kernel<T, 32, kPastCaches>);
      else FASTH_NORM_LAUNCH(grid, norm_grad_apply_kernel<T, 32>);
    } else if (p.lc == 16) {
      FASTH_NORM_LAUNCH(grid, norm_grad_sum_kernel<T, 16>);
      FASTH_NORM_LAUNCH(grid, norm_grad_apply_kernel<T, 16>);
    } else {
      FASTH_NORM_LAUNCH(grid, norm_grad_sum_kernel<T, 4>);
      FASTH_NORM_LAUNCH(grid, norm_grad_apply_kernel<T, 4>);
    }
  } else {
    const dim3 grid(parts);
    if (p.vec == 1 && p.u == 8) FASTH_NORM_LAUNCH(grid, norm_grad_kernel<T, 1, 1, 8>);
    else if (p.vec == 1) FASTH_NORM_LAUNCH(grid, norm_grad_kernel<T, 1, 1, 16>);
    else FASTH_NORM_LAUNCH(grid, norm_grad_kernel<T, 8, 4, 8>);
  }
  if (!dweight || parts == 1) return FASTH_OK;
  hipLaunchKernelGGL(norm_weight_kernel, dim3((a.d + kWave - 1) / kWave), dim3(1024), 0, stream, static_cast<const float*>(workspace),
                     parts, a.d, dweight);
  FASTH_HIP(hipGetLastError());
  return FASTH_OK;
}

}  // namespace fasth
