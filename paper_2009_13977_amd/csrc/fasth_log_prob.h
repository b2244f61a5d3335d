// Log probabilities of the given tokens, entropy and the most probable alternatives of every column of logits
// [vocab][m], and the gradient with respect to the logits.
//
//   M_j = max_v x_vj,  L_j = log sum_v e^(x_vj - M_j),  log p_vj = (x_vj - M_j) - L_j
//   entropy H_j = -sum_v p_vj log p_vj = L_j - sum_v p_vj (x_vj - M_j)
//   dx_vj = gl_j (delta(v = id_j) - p_vj) - ge_j p_vj (log p_vj + H_j)
//
// M and L stay apart: their sum would lose bits of L where the logits are large. A logit of -infinity is masked: its
// probability, its term of the entropy and its gradient are zero. Both directions are bound by reading the logits
// (and writing their gradient): one pass each, with a running maximum per thread and column.
#pragma once
#include "fasth_columns.h"
#include "fasth_common.h"

namespace fasth {

constexpr int kLogitRows = 16;        // rows of a column in a thread's registers: one rescaling of the sums per 16 terms
constexpr int kLogitThreads = 256;
constexpr int kLogitMaxSplits = 64;   // workgroups that share a column
constexpr int kLogitMaxVocab = 1 << 21;
constexpr int kLogitMaxChunks = 8192; // parts of a column whose largest logits are kept for the alternatives: 16 waves x 64 lanes x 8
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Running sums of a column: s = sum of 2^t, q = sum of t 2^t with t = (x - max) log2(e).
struct ColumnSum {
  float max, s, q;
};
__device__ __forceinline__ ColumnSum empty_sum() { return {-INFINITY, 0.f, 0.f}; }
// A part without any finite logit has max = -infinity and zero sums; against another such part the difference would be
// NaN, so differences are taken from a finite maximum. (2^-150 is zero in fp32, so nothing is lost by the bound on t.)
__device__ __forceinline__ ColumnSum rescale(const ColumnSum& a, float to) {
  const float t = fmaxf((a.max - to) * kLog2e, -150.f), f = __builtin_amdgcn_exp2f(t);
  return {to, a.s * f, (a.q + a.s * t) * f};
}
__device__ __forceinline__ ColumnSum join(const ColumnSum& a, const ColumnSum& b) {
  const float to = fmaxf(fmaxf(a.max, b.max), -3.402823466e38f);
  const ColumnSum x = rescale(a, to), y = rescale(b, to);
  return {fmaxf(a.max, b.max), x.s + y.s, x.q + y.q};
}
template <int FROM>
__device__ __forceinline__ ColumnSum join_lanes_from(ColumnSum a) {
#pragma unroll
  for (int mask = FROM; mask < kWave; mask <<= 1) {
    const ColumnSum b = {__shfl_xor(a.max, mask, kWave), __shfl_xor(a.s, mask, kWave), __shfl_xor(a.q, mask, kWave)};
    // both partners join in the same order, so that all lanes end with the same bits
    a = (threadIdx.x & mask) ? join(b, a) : join(a, b);
  }
  return a;
}

struct LogProbArgs {
  const void *logits, *ids;
  float *logp, *entropy, *stats;  // stats: [2][m], M and L
  float *part;                    // [splits][3][m]: the splits' sums; null: one split, which writes the outputs itself
  float *largest;                 // [m][chunks]: the largest logit of every chunk of rows; null: no alternatives
  float *top_logp;                // [top][m]
  int *top_ids;                   // [top][m]
  int id_bits, vocab, m, top;
  int splits, rows_per_split, chunk, chunks;
};

template <typename T>
__device__ __forceinline__ void write_column(const LogProbArgs& a, int j, ColumnSum c) {
  float M = c.max, L = 0.f, H = 0.f;
  if (c.s == 0.f) M = 0.f;  // nothing but masked logits (NaN fails the test and stays)
  else {
    L = logf(c.s);
    H = L - kLn2 * c.q / c.s;
  }
  a.stats[j] = M;
  a.stats[a.m + j] = L;
  a.entropy[j] = H;
  const int id = token_at(a.ids, a.id_bits, j, a.vocab);
  float lp = 0.f;
  if (id >= 0) lp = ((float)static_cast<const T*>(a.logits)[(size_t)id * a.m + j] - M) - L;
  a.logp[j] = lp;
}

// LC lanes x VEC columns wide; a thread takes chunks of consecutive rows, 16 rows in registers at a time.
template <typename T, int LC, int VEC>
__global__ void __launch_bounds__(kLogitThreads) log_prob_kernel(LogProbArgs a) {
  constexpr int RL = kLogitThreads / LC, WAVES = kLogitThreads / kWave;
  __shared__ ColumnSum red[WAVES][LC * VEC];
  const int rl = threadIdx.x / LC, cl = threadIdx.x % LC;
  const int j = (blockIdx.x * LC + cl) * VEC, left = a.m - j;
  const T* x0 = static_cast<const T*>(a.logits) + j;
  const int row0 = blockIdx.y * a.rows_per_split, row1 = min(a.vocab, row0 + a.rows_per_split);
  ColumnSum sum[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) sum[e] = empty_sum();
  for (int r0 = row0 + rl * a.chunk; r0 < row1; r0 += RL * a.chunk) {
    float most[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) most[e] = -INFINITY;
    const int r2 = min(row1, r0 + a.chunk);
    for (int r = r0; r < r2; r += kLogitRows) {
      Cols<T, VEC> x[kLogitRows];
#pragma unroll
      for (int u = 0; u < kLogitRows; ++u) x[u] = load_cols<T, VEC>(x0 + (size_t)(r + u) * a.m, r + u < r2 ? left : 0, -INFINITY);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        float here = -INFINITY;
#pragma unroll
        for (int u = 0; u < kLogitRows; ++u) here = fmaxf(here, x[u].get(e));
        most[e] = fmaxf(most[e], here);
        const float to = fmaxf(fmaxf(sum[e].max, here), -3.402823466e38f);
        ColumnSum c = rescale(sum[e], to);
        c.max = fmaxf(sum[e].max, here);
#pragma unroll
        for (int u = 0; u < kLogitRows; ++u) {
          const float t = (x[u].get(e) - to) * kLog2e, p = __builtin_amdgcn_exp2f(t);
          c.s += p;
          c.q += p * fmaxf(t, -150.f);
        }
        sum[e] = c;
      }
    }
    if (a.largest) {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (e < left) a.largest[(size_t)(j + e) * a.chunks + r0 / a.chunk] = most[e];
    }
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) sum[e] = join_lanes_from<LC>(sum[e]);
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  if (lane < LC) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) red[wave][cl * VEC + e] = sum[e];
  }
  __syncthreads();
  const int col = blockIdx.x * (LC * VEC) + threadIdx.x;
  if (threadIdx.x >= LC * VEC || col >= a.m) return;
  ColumnSum c = red[0][threadIdx.x];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) c = join(c, red[w][threadIdx.x]);
  if (a.part) {
    float* p = a.part + (size_t)blockIdx.y * 3 * a.m + col;
    p[0] = c.max;
    p[a.m] = c.s;
    p[2 * (size_t)a.m] = c.q;
  } else {
    write_column<T>(a, col, c);
  }
}

__device__ __forceinline__ ColumnSum split_sum(const LogProbArgs& a, int split, int j) {
  const float* p = a.part + (size_t)split * 3 * a.m + j;
  return {p[0], p[a.m], p[2 * (size_t)a.m]};
}

// The splits' sums of 16 columns per workgroup, 16 splits at a time.
template <typename T>
__global__ void __launch_bounds__(256) log_prob_join_kernel(LogProbArgs a) {
  __shared__ ColumnSum red[4][16];
  const int col = threadIdx.x & 15, j = blockIdx.x * 16 + col, lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  ColumnSum c = empty_sum();
  if (j < a.m) {
    for (int s = threadIdx.x >> 4; s < a.splits; s += 16) c = join(c, split_sum(a, s, j));
  }
  c = join_lanes_from<16>(c);
  if (lane < 16) red[wave][col] = c;
  __syncthreads();
  if (threadIdx.x < 16 && j < a.m) {
    c = red[0][col];
#pragma unroll
    for (int w = 1; w < 4; ++w) c = join(c, red[w][col]);
    write_column<T>(a, j, c);
  }
}

// The k largest of 64 x 8 numbers, lane l holding numbers 8 l .. 8 l + 7: out_v[r], out_at[r] = the r-th largest and its
// number, ties to the lower number. -infinity is never taken: at[r] = -1 from where nothing else is left. NaN is never
// the larger of two. Every round removes one number.
__device__ __forceinline__ void wave_top(float (&v)[8], int k, float* out_v, int* out_at) {
  const int lane = threadIdx.x & (kWave - 1);
  for (int r = 0; r < k; ++r) {
    float best = -INFINITY;
    int at = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (v[i] > best) { best = v[i]; at = i; }
    const float most = combine_lanes_from<1>(best, [](float a, float b) { return fmaxf(a, b); });
    const unsigned long long who = __ballot(best == most);
    const int first = __builtin_ctzll(who);
    if (lane == first) {
      out_v[r] = most;
      out_at[r] = most == -INFINITY ? -1 : 8 * lane + at;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i == at) v[i] = -INFINITY;
    }
  }
}

// The alternatives of one column per workgroup. An entry among the k largest lies in one of the k chunks with the
// largest maxima (ties to the lower chunk: every better chunk holds an entry that comes first), so only those are read
// again. Two rounds of the same selection: the chunks, then the entries of the chosen ones in the order of their rows.
template <typename T>
__global__ void __launch_bounds__(1024) log_prob_top_kernel(LogProbArgs a) {
  __shared__ float wave_v[16][FASTH_MAX_TOP], all_v[FASTH_MAX_TOP];
  __shared__ int wave_at[16][FASTH_MAX_TOP], all_at[FASTH_MAX_TOP], chosen[FASTH_MAX_TOP];
  const int j = blockIdx.x, k = a.top, waves = blockDim.x >> 6;
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  const T* x = static_cast<const T*>(a.logits) + j;
  float v[8];
  // the waves' lists into one: number w * k + r of the merged order is the r-th of wave w
  auto merge = [&]() {
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int c = 8 * lane + i;
        v[i] = c < waves * k && wave_at[c / k][c % k] >= 0 ? wave_v[c / k][c % k] : -INFINITY;
      }
      wave_top(v, k, all_v, all_at);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if (lane < k) {
        const int c = all_at[lane];
        all_at[lane] = c < 0 ? -1 : (c / k) * 512 + wave_at[c / k][c % k];
      }
    }
    __syncthreads();
  };
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int c = 512 * wave + 8 * lane + i;
    v[i] = c < a.chunks ? a.largest[(size_t)j * a.chunks + c] : -INFINITY;
  }
  wave_top(v, k, wave_v[wave], wave_at[wave]);
  merge();
  // the chosen chunks in the order of their rows
  if (threadIdx.x < k) {
    const int c = all_at[threadIdx.x];
    int before = 0;
    for (int r = 0; r < k; ++r) before += all_at[r] >= 0 && all_at[r] < c;
    if (c >= 0) chosen[before] = c;
  }
  int found = 0;
  for (int r = 0; r < k; ++r) found += all_at[r] >= 0;
  __syncthreads();
  auto row_of = [&](int number) { return chosen[number / a.chunk] * a.chunk + number % a.chunk; };
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int number = 512 * wave + 8 * lane + i;
    v[i] = -INFINITY;
    if (number < found * a.chunk) {
      const int row = row_of(number);
      if (row < a.vocab) v[i] = (float)x[(size_t)row * a.m];
    }
  }
  wave_top(v, k, wave_v[wave], wave_at[wave]);
  merge();
  if (wave == 0) {
    ColumnSum c = empty_sum();
    for (int s = lane; s < a.splits; s += kWave) c = join(c, split_sum(a, s, j));
    c = join_lanes_from<1>(c);
    if (lane == 0) write_column<T>(a, j, c);
    const float L = c.s == 0.f ? 0.f : logf(c.s);
    if (lane < k) {
      const int number = all_at[lane];
      a.top_ids[(size_t)lane * a.m + j] = number < 0 ? -1 : row_of(number);
      a.top_logp[(size_t)lane * a.m + j] = number < 0 ? -INFINITY : (all_v[lane] - c.max) - L;
    }
  }
}

struct LogProbGradArgs {
  const void *logits, *ids;
  const float *stats, *entropy, *g_logp, *g_entropy;
  void* dlogits;
  int id_bits, vocab, m, rows_per_split;
};

template <typename T, int LC, int VEC>
__global__ void __launch_bounds__(kLogitThreads) log_prob_grad_kernel(LogProbGradArgs a) {
  constexpr int RL = kLogitThreads / LC, U = 8;
  const int rl = threadIdx.x / LC, cl = threadIdx.x % LC;
  const int j = (blockIdx.x * LC + cl) * VEC, left = a.m - j;
  const T* x0 = static_cast<const T*>(a.logits) + j;
  T* y0 = static_cast<T*>(a.dlogits) + j;
  const int row0 = blockIdx.y * a.rows_per_split, row1 = min(a.vocab, row0 + a.rows_per_split);
  float M[VEC], L[VEC], H[VEC], gl[VEC], ge[VEC];
  int id[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const bool in = e < left;
    M[e] = in ? a.stats[j + e] : 0.f;
    L[e] = in ? a.stats[a.m + j + e] : 0.f;
    id[e] = in ? token_at(a.ids, a.id_bits, j + e, a.vocab) : -1;
    gl[e] = in && id[e] >= 0 && a.g_logp ? a.g_logp[j + e] : 0.f;
    ge[e] = in && a.g_entropy ? a.g_entropy[j + e] : 0.f;
    H[e] = in && a.g_entropy ? a.entropy[j + e] : 0.f;
  }
  for (int r = row0 + rl; r < row1; r += RL * U) {
    Cols<T, VEC> x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = load_cols<T, VEC>(x0 + (size_t)(r + u * RL) * a.m, r + u * RL < row1 ? left : 0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int row = r + u * RL;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float v = x[u].get(e), t = (v - M[e]) - L[e];
        const float p = __builtin_amdgcn_exp2f(t * kLog2e);  // zero below the smallest normal number
        // (p is zero long before the bound on t counts; it keeps 0 * infinity out)
        float dx = -p * (gl[e] + ge[e] * (fmaxf(t, -1e4f) + H[e]));
        if (row == id[e] && v != -INFINITY) dx += gl[e];
        x[u].set(e, dx);
      }
      store_cols<T, VEC>(y0 + (size_t)row * a.m, row < row1 ? left : 0, x[u]);
    }
  }
}

struct LogProbPlan {
  bool wide;  // 4 columns per thread, 16 threads per row; else one column, 4 threads (or 1) per row
  int lc, tiles, splits, rows_per_split, chunk, chunks;
  size_t off_largest, total;
};
static LogProbPlan plan_log_prob(int vocab, int m, int top) {
  LogProbPlan p;
  p.wide = m >= 16;
  p.lc = p.wide ? 16 : m >= 4 ? 4 : 1;
  const int cols = p.wide ? 64 : p.lc;
  p.tiles = (m + cols - 1) / cols;
  p.chunk = kLogitRows;
  while ((vocab + p.chunk - 1) / p.chunk > kLogitMaxChunks) p.chunk *= 2;
  p.chunks = (vocab + p.chunk - 1) / p.chunk;
  const int step = kLogitThreads / p.lc * p.chunk;  // rows of one step of a workgroup
  const int steps = (vocab + step - 1) / step;
  p.splits = std::max(1, std::min({steps, kLogitMaxSplits, 8 * kComputeUnits / p.tiles}));
  p.rows_per_split = (steps + p.splits - 1) / p.splits * step;
  p.splits = (vocab + p.rows_per_split - 1) / p.rows_per_split;
  p.off_largest = align_up((size_t)p.splits * 3 * m * sizeof(float), 256);
  p.total = p.off_largest + (top ? align_up((size_t)m * p.chunks * sizeof(float), 256) : 0);
  return p;
}

template <typename T>
static int launch_log_prob(const LogProbArgs& args, void* workspace, hipStream_t stream) {
  LogProbArgs a = args;
  const LogProbPlan p = plan_log_prob(a.vocab, a.m, a.top);
  a.splits = p.splits; a.rows_per_split = p.rows_per_split; a.chunk = p.chunk; a.chunks = p.chunks;
  const bool own = p.splits == 1 && !a.top;
  a.part = own ? nullptr : static_cast<float*>(workspace);
  a.largest = a.top ? reinterpret_cast<float*>(static_cast<char*>(workspace) + p.off_largest) : nullptr;
  const dim3 grid(p.tiles, p.splits);
  if (p.wide) hipLaunchKernelGGL((log_prob_kernel<T, 16, 4>), grid, dim3(kLogitThreads), 0, stream, a);
  else if (p.lc == 4) hipLaunchKernelGGL((log_prob_kernel<T, 4, 1>), grid, dim3(kLogitThreads), 0, stream, a);
  else hipLaunchKernelGGL((log_prob_kernel<T, 1, 1>), grid, dim3(kLogitThreads), 0, stream, a);
  FASTH_HIP(hipGetLastError());
  if (own) return FASTH_OK;
  if (a.top) {
    // waves for the chunks' maxima (512 each) and for the entries of the chosen chunks
    const int numbers = std::max(p.chunks, std::min(a.top, p.chunks) * p.chunk), waves = (numbers + 511) / 512;
    hipLaunchKernelGGL((log_prob_top_kernel<T>), dim3(a.m), dim3(waves * kWave), 0, stream, a);
  } else {
    hipLaunchKernelGGL((log_prob_join_kernel<T>), dim3((a.m + 15) / 16), dim3(256), 0, stream, a);
  }
  FASTH_HIP(hipGetLastError());
  return FASTH_OK;
}

template <typename T>
static int launch_log_prob_grad(const LogProbGradArgs& args, hipStream_t stream) {
  LogProbGradArgs a = args;
  const bool wide = a.m >= 16;
  const int lc = wide ? 16 : a.m >= 4 ? 4 : 1, cols = wide ? 64 : lc, tiles = (a.m + cols - 1) / cols;
  const int step = kLogitThreads / lc * 8, steps = (a.vocab + step - 1) / step;
  const int splits = std::max(1, std::min(steps, std::max(1, 16 * kComputeUnits / tiles)));
  a.rows_per_split = (steps + splits - 1) / splits * step;
  const dim3 grid(tiles, (a.vocab + a.rows_per_split - 1) / a.rows_per_split);
  if (wide) hipLaunchKernelGGL((log_prob_grad_kernel<T, 16, 4>), grid, dim3(kLogitThreads), 0, stream, a);
  else if (lc == 4) hipLaunchKernelGGL((log_prob_grad_kernel<T, 4, 1>), grid, dim3(kLogitThreads), 0, stream, a);
  else hipLaunchKernelGGL((log_prob_grad_kernel<T, 1, 1>), grid, dim3(kLogitThreads), 0, stream, a);
  FASTH_HIP(hipGetLastError());
  return FASTH_OK;
}

}  // namespace fasth
