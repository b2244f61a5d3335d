// Log probabilities of the given tokens, entropy and the most probable alternatives of every column of logits
// [vocab][m], and the gradient with respect to the logits.
//
//   M_j = max_v x_vj,  L_j = log sum_v e^(x_vj - M_j),  log p_vj = (x_vj - M_j) - L_j
//   entropy H_j = -sum_v p_vj log p_vj = L_j - sum_v p_vj (x_vj - M_j)
//   dx_vj = gl_j (delta(v = id_j) - p_vj) - ge_j p_vj (log p_vj + H_j)
//
// M and L stay apart: their sum would lose bits of L where the logits are large. So does the largest logit's own term, 1,
// stay apart from the others' sum R, with L = log(1 + R): where a column is sure of a token, R is all that 1 - p and the
// entropy are made of. A logit of -infinity is masked: its probability, its term of the entropy and its gradient are
// zero. Both directions are bound by reading the logits (and writing their gradient): one pass each.
#pragma once
#include "fasth_columns.h"
#include "fasth_common.h"

namespace fasth {

constexpr int kLogitRows = 16;        // consecutive rows of a column that a thread takes at a time, in two groups
constexpr int kLogitThreads = 256;
constexpr int kLogitMaxSplits = 128;  // workgroups that share a column
constexpr int kLogitMaxVocab = 1 << 21;
constexpr int kLogitMaxChunks = 8192; // parts of a column whose largest logits are kept for the alternatives: 16 waves x 64 lanes x 8
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Running sums of a column: ref = the largest logit so far, s = the sum of 2^t less 1, q = the sum of t 2^t, with
// t = (x - ref) log2(e). The 1 that s leaves out is ref's own term.
struct ColumnSum {
  float ref, s, q;
};
constexpr float kLowest = -3.402823466e38f;  // the reference of nothing: differences from -infinity would be NaN
__device__ __forceinline__ ColumnSum empty_sum() { return {kLowest, -1.f, 0.f}; }
// What terms that count from `from` are multiplied by to count from `to`, and its logarithm. (2^-150 is zero in fp32, so
// nothing is lost by the bound; zero sums stay zero.)
struct Rebase {
  float t, f;
};
__device__ __forceinline__ Rebase rebase(float from, float to) {
  const float t = fmaxf((from - to) * kLog2e, -150.f);
  return {t, __builtin_amdgcn_exp2f(t)};
}
__device__ __forceinline__ ColumnSum join(const ColumnSum& a, const ColumnSum& b) {
  const bool second = b.ref > a.ref;
  const ColumnSum hi = second ? b : a, lo = second ? a : b;
  const Rebase r = rebase(lo.ref, hi.ref);
  return {hi.ref, (hi.s + lo.s * r.f) + r.f, hi.q + (lo.q + (lo.s + 1.f) * r.t) * r.f};
}
template <int FROM>
__device__ __forceinline__ ColumnSum join_lanes_from(ColumnSum a) {
  return combine_lanes_from<FROM>(a, [](ColumnSum x, ColumnSum y) { return join(x, y); });
}

__host__ __device__ __forceinline__ constexpr int chunk_stride(int chunks) { return (chunks + 7) & ~7; }

struct LogProbArgs {
  const void *logits, *ids;
  float *logp, *entropy, *stats;  // stats: [2][m], M and L
  float *part;                    // [splits][3][m]: the splits' sums; null: one split, which writes the outputs itself
  float *largest;                 // [m][chunk_stride(chunks)]: the largest logit of every chunk of rows; null: no alternatives
  float *top_logp;                // [top][m]
  int *top_ids;                   // [top][m]
  int id_bits, vocab, m, top, tiles;
  int splits, rows_per_split, chunk, chunks;
};

// The given token's logit, fetched while the sums are still under way.
struct Given {
  bool is;
  float x;
};
template <typename T>
__device__ __forceinline__ Given given_logit(const LogProbArgs& a, int j) {
  const int id = token_at(a.ids, a.id_bits, j, a.vocab);
  return {id >= 0, id >= 0 ? (float)static_cast<const T*>(a.logits)[(size_t)id * a.m + j] : 0.f};
}
__device__ __forceinline__ void write_column(const LogProbArgs& a, int j, ColumnSum c, Given g) {
  float M = c.ref, L = 0.f, H = 0.f;
  if (c.s == -1.f) M = 0.f;  // nothing but masked logits (NaN fails the test and stays)
  else {
    L = log1pf(c.s);
    H = L - kLn2 * c.q / (1.f + c.s);
  }
  a.stats[j] = M;
  a.stats[a.m + j] = L;
  a.entropy[j] = H;
  a.logp[j] = g.is ? (g.x - M) - L : 0.f;
}

// A group of G rows of VEC columns into the running sums; top: the group's largest logits. The reference has to be the
// largest logit itself: with one below it, L = log s and x - M are large numbers whose difference is the answer, and
// with one that merely is near, s is not 1 + R. A group without a new largest logit adds all its terms to s; one that has
// it loses at most three roundings of 1 (or its own other terms, if they are less).
template <bool LATER, typename T, int VEC, int G>
__device__ __forceinline__ void take_group(ColumnSum (&sum)[VEC], const Cols<T, VEC> (&x)[G], float (&top)[VEC]) {
  static_assert(G == 8, "three levels of sums");
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    top[e] = x[0].get(e);
#pragma unroll
    for (int u = 1; u < G; ++u) top[e] = fmaxf(top[e], x[u].get(e));
    const float from = sum[e].ref, ref = fmaxf(from, top[e]);
    float p[G], q = 0.f;
#pragma unroll
    for (int u = 0; u < G; ++u) {
      const float t = (x[u].get(e) - ref) * kLog2e;
      p[u] = __builtin_amdgcn_exp2f(t);
      q += p[u] * fmaxf(t, -150.f);
    }
    const float s = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    const Rebase r = rebase(from, ref);
    sum[e].q = (sum[e].q + (sum[e].s + 1.f) * r.t) * r.f + q;
    sum[e].s = sum[e].s * r.f + (ref > from ? r.f + (s - 1.f) : s);
    sum[e].ref = ref;
    // Now: put off, the sums would keep x in registers of its own beside what is loaded next (128000 x 4096 bf16: 208 us,
    // 187 in this order; with the largest logits of all chunks to be kept it is the other way round: the call 464 us, 500 in this order)
    if constexpr (!LATER) asm volatile("" : "+v"(sum[e].ref), "+v"(sum[e].s), "+v"(sum[e].q));
  }
}

// LC lanes x VEC columns wide; a thread takes chunks of consecutive rows, 16 rows at a time in two groups: while one is
// worked on, the other's 8 loads are in flight. Bound by memory and the vector units at once: 128000 x 4096 bf16 184 us,
// 5.7 TB/s, while nine instructions per logit, one of which is an exponential and counts four, are some 165 us. (A reference
// that stayed what the first rows made it took nine in all and 180 us, and lost the small probabilities.) ONCE: past the caches.
template <typename T, int LC, int VEC, bool TOP, bool ONCE>
__global__ void __launch_bounds__(kLogitThreads) log_prob_kernel(LogProbArgs a) {
  constexpr int RL = kLogitThreads / LC, WAVES = kLogitThreads / kWave, G = kLogitRows / 2;
  __shared__ ColumnSum red[WAVES][LC * VEC];
  const int rl = threadIdx.x / LC, cl = threadIdx.x % LC;
  const TileAt tile(a.tiles);
  const ColumnRange<VEC> cols((tile.col * LC + cl) * VEC, a.m, tile.col == a.tiles - 1);
  const T* logits = static_cast<const T*>(a.logits);
  const int row0 = tile.row * a.rows_per_split, row1 = min(a.vocab, row0 + a.rows_per_split);
  const unsigned own = ((unsigned)rl * a.chunk * a.m + cols.first) * (unsigned)sizeof(T);  // at most 4096 x 65535 elements
  const int col = tile.col * (LC * VEC) + threadIdx.x;  // the column that this thread writes in the end, if any
  Given given = {false, 0.f};
  if (!a.part && threadIdx.x < LC * VEC && col < a.m) given = given_logit<T>(a, col);
  ColumnSum sum[VEC];
  float most[VEC];
  auto fetch = [&](const T* row) {
    if constexpr (ONCE) return load_once<T, VEC>(row, own);
    else return load_at<T, VEC>(row, own);
  };
  // the rows from `row` (of the first of the workgroup's threads) on; -infinity beyond the split's last row
  auto load = [&](Cols<T, VEC> (&x)[G], int row, int last) {
    if (last < row1) {  // `last`: the last thread's last row, so this is the same for the workgroup
#pragma unroll
      for (int u = 0; u < G; ++u) x[u] = fetch(logits + (size_t)(row + u) * a.m);
    } else {
#pragma unroll
      for (int u = 0; u < G; ++u) {
        const int r = row + u + rl * a.chunk;
        x[u] = load_cols<T, VEC>(logits + (size_t)min(r, a.vocab - 1) * a.m + cols.first, r < row1 ? VEC : 0, -INFINITY);
      }
    }
  };
  auto take = [&](const Cols<T, VEC> (&x)[G]) {
    float top[VEC];
    take_group<TOP, T, VEC, G>(sum, x, top);
    if constexpr (TOP) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) most[e] = fmaxf(most[e], top[e]);
    }
  };
  const int span = (RL - 1) * a.chunk + G - 1;  // from a group's first row to its last
  Cols<T, VEC> x0[G], x1[G];
  load(x0, row0, row0 + span);
  load(x1, row0 + G, row0 + G + span);
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    sum[e] = empty_sum();
    most[e] = -INFINITY;
  }
  for (int r0 = row0, part = 0; r0 < row1;) {
    int next = r0, next_part = part + kLogitRows;
    if (next_part >= a.chunk) {
      next += RL * a.chunk;
      next_part = 0;
    }
    const int at = next + next_part;
    take(x0);
    if (next < row1) load(x0, at, at + span);
    take(x1);
    if (next < row1) load(x1, at + G, at + G + span);
    if constexpr (TOP) {
      const int mine = r0 + rl * a.chunk;
      if (next_part == 0 && mine < row1) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          if (cols.own(e)) a.largest[(size_t)(cols.first + e) * chunk_stride(a.chunks) + mine / a.chunk] = most[e];
          most[e] = -INFINITY;
        }
      }
    }
    r0 = next;
    part = next_part;
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) sum[e] = join_lanes_from<LC>(sum[e]);
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  if (lane < LC) {
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (cols.own(e)) red[wave][cols.first + e - tile.col * (LC * VEC)] = sum[e];
  }
  __syncthreads();
  if (threadIdx.x >= LC * VEC || col >= a.m) return;
  static_assert(WAVES == 4, "two levels of joins");
  const ColumnSum c = join(join(red[0][threadIdx.x], red[1][threadIdx.x]), join(red[2][threadIdx.x], red[3][threadIdx.x]));
  if (a.part) {
    float* p = a.part + (size_t)tile.row * 3 * a.m + col;
    p[0] = c.ref;
    p[a.m] = c.s;
    p[2 * (size_t)a.m] = c.q;
  } else {
    write_column(a, col, c, given);
  }
}

__device__ __forceinline__ ColumnSum split_sum(const LogProbArgs& a, int split, int j) {
  const float* p = a.part + (size_t)split * 3 * a.m + j;
  return {p[0], p[a.m], p[2 * (size_t)a.m]};
}

// The splits' sums of 16 columns per workgroup, 16 splits at a time: one round of loads (4096 columns of 125 splits: 5 us).
template <typename T>
__global__ void __launch_bounds__(256) log_prob_join_kernel(LogProbArgs a) {
  __shared__ ColumnSum red[4][16];
  const int col = threadIdx.x & 15, j = blockIdx.x * 16 + col, lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  ColumnSum c = empty_sum();
  Given given = {false, 0.f};
  if (j < a.m) {
    if (threadIdx.x < 16) given = given_logit<T>(a, j);
    constexpr int N = kLogitMaxSplits / 16;  // all of a thread's splits in flight
    ColumnSum part[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int s = (threadIdx.x >> 4) + 16 * n;
      part[n] = s < a.splits ? split_sum(a, s, j) : empty_sum();
    }
#pragma unroll
    for (int half = N / 2; half; half /= 2) {
#pragma unroll
      for (int n = 0; n < half; ++n) part[n] = join(part[n], part[n + half]);
    }
    c = part[0];
  }
  c = join_lanes_from<16>(c);
  if (lane < 16) red[wave][col] = c;
  __syncthreads();
  if (threadIdx.x < 16 && j < a.m) {
    c = join(join(red[0][col], red[1][col]), join(red[2][col], red[3][col]));
    write_column(a, j, c, given);
  }
}

// Floating-point numbers as integers in the same order, NaN apart (v_max_i32 needs no quieting of its operands). The sum
// makes the two zeros one.
__device__ __forceinline__ int order_key(float x) {
  const int b = __float_as_int(x + 0.f);
  return b ^ ((b >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float order_value(int key) { return __int_as_float(key ^ ((key >> 31) & 0x7fffffff)); }
constexpr int kNothing = (int)0x807fffff;  // order_key(-infinity)

// The k largest of 64 x 8 keys, lane l holding numbers 8 l .. 8 l + 7: out_v[r], out_at[r] = the r-th largest and its number
// plus `base`, ties to the lower number. kNothing is never taken: out_at[r] = -1 from where nothing else is left. Every
// round removes one number.
__device__ __forceinline__ void wave_top(int (&v)[8], int k, int base, int* out_v, int* out_at) {
  const int lane = threadIdx.x & (kWave - 1);
  for (int r = 0; r < k; ++r) {
    const int best = max(max(max(v[0], v[1]), max(v[2], v[3])), max(max(v[4], v[5]), max(v[6], v[7])));
    const int most = combine_lanes_from<1>(best, [](int a, int b) { return max(a, b); });
    const int first = __builtin_ctzll(__ballot(best == most));
    if (lane == first) {
      int at = 7;
#pragma unroll
      for (int i = 6; i >= 0; --i) at = v[i] == most ? i : at;
      out_v[r] = most;
      out_at[r] = most == kNothing ? -1 : base + 8 * lane + at;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i == at ? kNothing : v[i];
    }
  }
}

// The alternatives of one column per workgroup. An entry among the k largest lies in one of the k chunks with the
// largest maxima (ties to the lower chunk: every better chunk holds an entry that comes first), so only those are read
// again. Two rounds of the same selection: the chunks, then the entries of the chosen ones in the order of their rows. Bound
// by the latency of k rounds of a reduction over a wave, four times (by one wave for few rows): 128000 x 1, 8 alternatives
// 13 us; 32003 x 48, 5 alternatives 12 us; 128000 x 4096, 8 alternatives 153 us, behind 307 us of log_prob_kernel, which
// stores the chunks' largest logits, four bytes with a column's stride (181 us without).
template <typename T>
__global__ void __launch_bounds__(1024) log_prob_top_kernel(LogProbArgs a) {
  __shared__ float column[2];
  __shared__ int list_v[16 * FASTH_MAX_TOP], list_at[16 * FASTH_MAX_TOP], all_v[FASTH_MAX_TOP], all_at[FASTH_MAX_TOP], chosen[FASTH_MAX_TOP];
  const int j = blockIdx.x, k = a.top, waves = blockDim.x >> 6;
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  const T* x = static_cast<const T*>(a.logits) + j;
  int v[8];
  {
    const int c = 512 * wave + 8 * lane;
    float4 lo = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY), hi = lo;
    if (c < a.chunks) {  // (the columns are padded to whole eights, whose rest is not used)
      const float4* p = reinterpret_cast<const float4*>(a.largest + (size_t)j * chunk_stride(a.chunks) + c);
      lo = p[0];
      hi = p[1];
    }
    const float f[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < a.chunks ? order_key(f[i]) : kNothing;
  }
  // the waves' lists into one, in the order of the waves where entries are equal; `beside` is for the last wave meanwhile
  auto merge = [&](auto beside) {
    __syncthreads();
    if (wave == waves - 1) beside();
    if (waves == 1) {
      if (lane < k) {
        all_v[lane] = list_v[lane];
        all_at[lane] = list_at[lane];
      }
    } else if (wave == 0) {
      int at[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int c = 8 * lane + i;
        at[i] = c < waves * k ? list_at[c] : -1;
        v[i] = at[i] >= 0 ? list_v[c] : kNothing;
      }
      wave_top(v, k, 0, all_v, all_at);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if (lane < k && all_at[lane] >= 0) all_at[lane] = list_at[all_at[lane]];
    }
    __syncthreads();
  };
  ColumnSum c = empty_sum();
  Given given = {false, 0.f};
  if (wave == waves - 1) {  // the column's sums, for later
    for (int s = lane; s < a.splits; s += kWave) c = join(c, split_sum(a, s, j));
    if (lane == 0) given = given_logit<T>(a, j);
  }
  wave_top(v, k, 512 * wave, list_v + wave * k, list_at + wave * k);
  merge([&]() {
    c = join_lanes_from<1>(c);
    if (lane == 0) {
      write_column(a, j, c, given);
      column[0] = c.ref;
      column[1] = c.s == -1.f ? 0.f : log1pf(c.s);
    }
  });
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
  const int shift = __builtin_ctz(a.chunk);  // (a power of two)
  auto row_of = [&](int number) { return (chosen[number >> shift] << shift) + (number & (a.chunk - 1)); };
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int number = 512 * wave + 8 * lane + i;
    v[i] = kNothing;
    if (number < found << shift) {
      const int row = row_of(number);
      if (row < a.vocab) v[i] = order_key(fmaxf((float)x[(size_t)row * a.m], -INFINITY));  // NaN is no alternative
    }
  }
  wave_top(v, k, 512 * wave, list_v + wave * k, list_at + wave * k);
  merge([]() {});
  if (threadIdx.x < k) {
    const int number = all_at[threadIdx.x];
    a.top_ids[(size_t)threadIdx.x * a.m + j] = number < 0 ? -1 : row_of(number);
    a.top_logp[(size_t)threadIdx.x * a.m + j] = number < 0 ? -INFINITY : (order_value(all_v[threadIdx.x]) - column[0]) - column[1];
  }
}

struct LogProbGradArgs {
  const void *logits, *ids;
  const float *stats, *entropy, *g_logp, *g_entropy;
  void* dlogits;
  int id_bits, vocab, m, tiles;
};

// With A = ge ln 2, B = gl + ge H and L in units of log 2: t = log2 p, and -p (A t + B) of a logit that is not the given token's.
__device__ __forceinline__ float log_prob_slope(float x, float M, float L, float A, float B) {
  const float t = (x - M) * kLog2e - L;
  const float p = __builtin_amdgcn_exp2f(t);  // zero below the smallest normal number
  // (p is zero long before the bound on t counts; it keeps 0 * infinity out)
  return -p * (A * fmaxf(t, -1e4f) + B);
}

// 1 - p of t = log2 p <= 0. From p = 1/2 on the difference would lose what a sure column leaves of it: there by the series
// of 1 - e^y, nine terms (the tenth is 2^-26 of the first at most).
__device__ __forceinline__ float one_less(float t) {
  const float y = t * kLn2;
  float c = 1.f / 362880.f;
  c = c * y + 1.f / 40320.f;
  c = c * y + 1.f / 5040.f;
  c = c * y + 1.f / 720.f;
  c = c * y + 1.f / 120.f;
  c = c * y + 1.f / 24.f;
  c = c * y + 1.f / 6.f;
  c = c * y + 0.5f;
  c = c * y + 1.f;
  return t > -1.f ? -y * c : 1.f - __builtin_amdgcn_exp2f(t);
}

// Rows rl, rl + RL, ... of the workgroup's RL x U rows per thread, all at once and no loop: a wave waits for its stores
// before it can use what it loads next, a new workgroup does not (a copy of 1 GiB in this pattern: 354 us, looping 420 to 450).
// Bound by memory: 128000 x 4096 bf16 376 us for 2.1 GB, 5.6 TB/s; 256 x 16384 fp32 9 us.
template <typename T, int LC, int VEC, int U, bool ONCE>
__global__ void __launch_bounds__(kLogitThreads) log_prob_grad_kernel(LogProbGradArgs a) {
  constexpr int RL = kLogitThreads / LC;
  const int rl = threadIdx.x / LC, cl = threadIdx.x % LC;
  const TileAt tile(a.tiles);
  const ColumnRange<VEC> cols((tile.col * LC + cl) * VEC, a.m, tile.col == a.tiles - 1);
  const int row0 = (blockIdx.y * (int)(gridDim.x / a.tiles) + tile.row) * (RL * U);
  if (row0 >= a.vocab) return;
  const bool all = row0 + RL * U <= a.vocab;  // the same for the workgroup
  const T* logits = static_cast<const T*>(a.logits) + (size_t)row0 * a.m;
  T* out = static_cast<T*>(a.dlogits) + (size_t)row0 * a.m;
  const unsigned own = ((unsigned)rl * a.m + cols.first) * (unsigned)sizeof(T);
  Cols<T, VEC> x[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int row = all ? u * RL : min(u * RL, a.vocab - 1 - row0 - rl);  // (a row that exists)
    if constexpr (ONCE) x[u] = load_once<T, VEC>(logits + (ptrdiff_t)row * a.m, own);
    else x[u] = load_at<T, VEC>(logits + (ptrdiff_t)row * a.m, own);
  }
  // the columns' numbers, in flight together with the rows
  const unsigned at = (unsigned)cols.first * 4;
  const Cols<float, VEC> m = load_at<float, VEC>(a.stats, at), l = load_at<float, VEC>(a.stats + a.m, at);
  const Cols<float, VEC> gl = load_at<float, VEC>(a.g_logp ? a.g_logp : a.stats, at);  // (any readable numbers: see below)
  const Cols<float, VEC> ge = load_at<float, VEC>(a.g_entropy ? a.g_entropy : a.stats, at);
  const Cols<float, VEC> h = load_at<float, VEC>(a.g_entropy ? a.entropy : a.stats, at);
  int id[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) id[e] = token_at(a.ids, a.id_bits, cols.first + e, a.vocab);
  float M[VEC], L[VEC], A[VEC], B[VEC], g[VEC];
  bool given = false;  // whether the thread has a given token's row
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    g[e] = id[e] >= 0 && a.g_logp ? gl.get(e) : 0.f;
    M[e] = m.get(e);
    L[e] = l.get(e) * kLog2e;
    A[e] = a.g_entropy ? ge.get(e) * kLn2 : 0.f;
    B[e] = a.g_entropy ? g[e] + ge.get(e) * h.get(e) : g[e];
    id[e] -= row0 + rl;  // in rows of the thread, times RL
    given |= (unsigned)id[e] < (unsigned)(RL * U) && (id[e] & (RL - 1)) == 0;
  }
  // the given tokens' entries
  float own_row[VEC];
  if (given) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      float v = -INFINITY;
#pragma unroll
      for (int u = 0; u < U; ++u) v = id[e] == u * RL ? x[u].get(e) : v;
      const float C = a.g_entropy ? ge.get(e) * h.get(e) : 0.f;
      own_row[e] = v == -INFINITY ? 0.f : log_prob_slope(v, M[e], L[e], A[e], C) + g[e] * one_less((v - M[e]) * kLog2e - L[e]);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    Cols<T, VEC> y;
#pragma unroll
    for (int e = 0; e < VEC; ++e) y.set(e, log_prob_slope(x[u].get(e), M[e], L[e], A[e], B[e]));
    if (given) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        if (id[e] == u * RL) y.set(e, own_row[e]);
      }
    }
    if (all && !cols.ragged) {
      if constexpr (ONCE) store_once<T, VEC>(out + (size_t)(u * RL) * a.m, own, y);
      else store_at<T, VEC>(out + (size_t)(u * RL) * a.m, own, y);
    } else if (row0 + u * RL + rl < a.vocab) {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (cols.own(e)) out[(size_t)(u * RL + rl) * a.m + cols.first + e] = (T)y.get(e);
    }
  }
}

// Lanes per row, of 16 bytes each for 16 columns and more: half a KiB of a row per workgroup where the logits do not fit the
// caches, 64 columns else (us, forward, through the caches: 128000 x 4096 bf16 198 and 219 with 64 columns, 50001 x 3001 bf16
// 74 and 83, but 256 x 16384 fp32 10.5 and 7.0); one column per lane, 4 or 1, below.
static int logit_lanes(int vocab, int m, int size) {
  if (m < 16) return m >= 4 ? 4 : 1;
  return m >= 256 && (int64_t)vocab * m * size > 64 << 20 ? 32 : 4 * size;
}

// Logits that no cache holds until they are used again are read past the caches (us, forward, with caches and past them:
// 128000 x 4096 bf16 197 and 185, 32000 x 4096 fp32 103 and 88, 128000 x 4097 bf16 222 and 221; smaller ones may be there still
// from the call before: 128000 x 512 bf16 used again at once 33 and 34, the gradient 51 and 69).
static bool past_caches(int vocab, int m, int size) { return (int64_t)vocab * m * size >= 400 << 20; }
// Their gradient is written past the caches too, but only where no cache line lies in two rows: a line that two workgroups
// write a part of each is else written twice (us, with caches and past them: 128000 x 4096 bf16 398 and 381, x 4160 415 and
// 389, 32000 x 4128 fp32 193 and 182, but 128000 x 4097 bf16 432 and 583, x 4112 417 and 502, 3300 x 65535 bf16 207 and 294).
static bool gradient_past_caches(int vocab, int m, int size) { return past_caches(vocab, m, size) && (int64_t)m * size % 128 == 0; }

struct LogProbPlan {
  int lc, tiles, splits, rows_per_split, chunk, chunks;
  size_t off_largest, total;
};
static LogProbPlan plan_log_prob(int vocab, int m, int top, int size) {
  LogProbPlan p;
  p.lc = logit_lanes(vocab, m, size);
  const int cols = p.lc * (m >= 16 ? 16 / size : 1);
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
  p.total = p.off_largest + (top ? align_up((size_t)m * chunk_stride(p.chunks) * sizeof(float), 256) : 0);
  return p;
}

static size_t log_prob_workspace(const fasth_log_prob_shape& s) {
  // (enough for any type, so that a workspace serves logits in whichever they come)
  return std::max(plan_log_prob(s.vocab, s.m, s.top, 2).total, plan_log_prob(s.vocab, s.m, s.top, 4).total);
}

template <typename T>
static int launch_log_prob(const LogProbArgs& args, void* workspace, hipStream_t stream) {
  LogProbArgs a = args;
  const LogProbPlan p = plan_log_prob(a.vocab, a.m, a.top, sizeof(T));
  a.splits = p.splits; a.rows_per_split = p.rows_per_split; a.chunk = p.chunk; a.chunks = p.chunks;
  const bool own = p.splits == 1 && !a.top;
  a.part = own ? nullptr : static_cast<float*>(workspace);
  a.largest = a.top ? reinterpret_cast<float*>(static_cast<char*>(workspace) + p.off_largest) : nullptr;
  a.tiles = p.tiles;
  const dim3 grid(p.tiles * p.splits);
  constexpr int VEC = 16 / sizeof(T);
#define FASTH_LOGIT_LAUNCH(LC, VEC, ONCE)                                                                                    \
  if (a.top) hipLaunchKernelGGL((log_prob_kernel<T, LC, VEC, true, ONCE>), grid, dim3(kLogitThreads), 0, stream, a);         \
  else hipLaunchKernelGGL((log_prob_kernel<T, LC, VEC, false, ONCE>), grid, dim3(kLogitThreads), 0, stream, a)
  if (p.lc == 32 && past_caches(a.vocab, a.m, sizeof(T))) { FASTH_LOGIT_LAUNCH(32, VEC, true); }
  else if (p.lc == 32) { FASTH_LOGIT_LAUNCH(32, VEC, false); }
  else if (a.m >= 16) { FASTH_LOGIT_LAUNCH(64 / VEC, VEC, false); }
  else if (a.m >= 4) { FASTH_LOGIT_LAUNCH(4, 1, false); }
  else { FASTH_LOGIT_LAUNCH(1, 1, false); }
#undef FASTH_LOGIT_LAUNCH
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
#define FASTH_LOGIT_LAUNCH(LC, VEC, ONCE)                                                                                           \
  do {                                                                                                                            \
    a.tiles = (a.m + LC * VEC - 1) / (LC * VEC);                                                                                  \
    const int step = kLogitThreads / LC * 8, steps = (a.vocab + step - 1) / step;                                                 \
    const int deep = (steps + 4095) / 4096;  /* at most 1024 x 4096 x 256 threads in a grid dimension */                          \
    hipLaunchKernelGGL((log_prob_grad_kernel<T, LC, VEC, 8, ONCE>), dim3(a.tiles * ((steps + deep - 1) / deep), deep), dim3(kLogitThreads), 0, stream, a); \
  } while (0)
  if (a.m >= 256 && gradient_past_caches(a.vocab, a.m, sizeof(T))) FASTH_LOGIT_LAUNCH(32, 4, true);
  else if (a.m >= 128) FASTH_LOGIT_LAUNCH(32, 4, false);
  else if (a.m >= 16) FASTH_LOGIT_LAUNCH(16, 4, false);
  else if (a.m >= 4) FASTH_LOGIT_LAUNCH(4, 1, false);
  else FASTH_LOGIT_LAUNCH(1, 1, false);
#undef FASTH_LOGIT_LAUNCH
  FASTH_HIP(hipGetLastError());
  return FASTH_OK;
}

}  // namespace fasth
