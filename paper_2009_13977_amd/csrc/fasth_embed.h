// Embedding of token numbers into the columns of a mini-batch, and its gradient.
//
//   X[i][j] = scale * table[id_j][i],       dTable[t][i] = scale * sum over the columns j with id_j = t of G[i][j]
//
// A number that is no row of the table marks a padded column: zeros forward, no part in the gradient.
#pragma once
#include "fasth_columns.h"
#include "fasth_common.h"

namespace fasth {

constexpr int kEmbedTile = 64;            // columns and features of a tile that is turned over in LDS
constexpr int kEmbedPad = kEmbedTile + 1;  // row stride in LDS: rows and columns both meet all banks
constexpr int kEmbedMaxVocab = 1 << 24;

// One tile of 64 columns x 64 features per workgroup: rows of the table come in as 64 consecutive features, the tile is
// turned over in LDS, rows of X leave as 64 consecutive columns. Bound by memory (a table row's and X's bytes once):
// 32000 x 1024 fp32, 4096 columns 11.0 us for 34 MB, one column 3.2 us, which is a launch and two dependent loads.
template <typename T>
__global__ void __launch_bounds__(256) embed_kernel(const T* __restrict__ table, const void* __restrict__ ids, int id_bits,
                                                    float scale, float* __restrict__ X, int vocab, int d, int m) {
  __shared__ float tile[kEmbedTile * kEmbedPad];
  const TileAt at((m + kEmbedTile - 1) / kEmbedTile);
  const int j0 = at.col * kEmbedTile, i0 = at.row * kEmbedTile;
  const int q = threadIdx.x & 15, p = threadIdx.x >> 4;  // four features or columns each; 16 rows at a time
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const int j = j0 + p + 16 * s, i = i0 + 4 * q;
    const int t = j < m ? token_at(ids, id_bits, j, vocab) : -1;
    float* dst = tile + (p + 16 * s) * kEmbedPad + 4 * q;
    Cols<T, 4> c;
    const bool some = t >= 0 && i < d;
    if (some) c = load_cols<T, 4>(table + (size_t)t * d + i, d - i);
#pragma unroll
    for (int e = 0; e < 4; ++e) dst[e] = some ? scale * c.get(e) : 0.f;
  }
  __syncthreads();
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const int i = i0 + p + 16 * s, j = j0 + 4 * q;
    if (i >= d || j >= m) continue;
    Cols<float, 4> c;
#pragma unroll
    for (int e = 0; e < 4; ++e) c.set(e, tile[(4 * q + e) * kEmbedPad + p + 16 * s]);
    store_cols<float, 4>(X + (size_t)i * m + j, m - j, c);
  }
}

// The order of the columns by token, columns of the same token in their own order: rank[j] is column j's place
// (-1 for a padded column), start[t] the first place of token t, start[vocab] the number of columns that are not padded.
//
// Every workgroup owns `per` consecutive tokens and looks at all columns (512 KiB of numbers at most, from the L2),
// so nothing is exchanged between workgroups and no atomic's order reaches the result. A wave takes a contiguous run of
// the columns: it counts its own tokens in LDS, the counts become places (by token, then by wave), and the second walk
// hands them out group by group of 64 columns, the lanes of one token in lane order. Bound by latencies: 9 us for 4096
// columns, 12 us for 9001, 16 us for 16384 (vocabulary 32000, 50021 and 256). From 131072 tokens on there are vocab / 512
// workgroups, and with a vocabulary much larger than that, looking at all columns is what the call costs: 2^24 tokens and
// 65535 columns 2.6 ms.
constexpr int kIndexWaves = 16;
constexpr int kIndexMaxPer = 512;  // tokens of a workgroup: 32 KiB of counts, at most a thread each while they become places
__global__ void __launch_bounds__(kIndexWaves * kWave)
embed_index_kernel(const void* __restrict__ ids, int id_bits, int vocab, int m, int per, int* __restrict__ rank, int* __restrict__ start) {
  extern __shared__ int count[];  // [kIndexWaves][per]
  __shared__ int below_of[kIndexWaves], total_of[kIndexWaves];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid >> 6;
  const int lo = blockIdx.x * per, own = vocab - lo < per ? vocab - lo : per;
  for (int x = tid; x < kIndexWaves * per; x += kIndexWaves * kWave) count[x] = 0;
  __syncthreads();
  volatile int* mine = count + wave * per;  // from the second walk on, one lane writes what the whole wave reads next
  const int groups = (m + kWave - 1) / kWave;
  const int g0 = (int)((long long)groups * wave / kIndexWaves), g1 = (int)((long long)groups * (wave + 1) / kIndexWaves);
  constexpr int N = 16;  // groups of 64 columns in flight
  int t[N], below = 0;
  auto fetch = [&](int g) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int j = (g + n) * kWave + lane;
      t[n] = g + n < g1 && j < m ? token_at(ids, id_bits, j, vocab) : -1;
    }
  };
  for (int g = g0; g < g1; g += N) {
    fetch(g);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      below += t[n] >= 0 && t[n] < lo;
      if (t[n] >= lo && t[n] < lo + own) atomicAdd(count + wave * per + (t[n] - lo), 1);
    }
  }
#pragma unroll
  for (int mask = 1; mask < kWave; mask <<= 1) below += __shfl_xor(below, mask, kWave);
  if (lane == 0) below_of[wave] = below;
  __syncthreads();
  int base = 0;
#pragma unroll
  for (int w = 0; w < kIndexWaves; ++w) base += below_of[w];
  // exclusive sum over this workgroup's tokens, one thread per token
  int n = 0;
  if (tid < own)
    for (int w = 0; w < kIndexWaves; ++w) n += count[w * per + tid];
  int upto = n;
#pragma unroll
  for (int step = 1; step < kWave; step <<= 1) {
    const int left = __shfl_up(upto, step, kWave);
    if (lane >= step) upto += left;
  }
  if (lane == kWave - 1) total_of[wave] = upto;
  __syncthreads();
  int at = base + upto - n;
#pragma unroll
  for (int w = 0; w < kIndexWaves; ++w) at += w < wave ? total_of[w] : 0;
  if (tid < own) {
    start[lo + tid] = at;
    if (lo + tid == vocab - 1) start[vocab] = at + n;
    for (int w = 0; w < kIndexWaves; ++w) {
      const int c = count[w * per + tid];
      count[w * per + tid] = at;
      at += c;
    }
  }
  __syncthreads();
  for (int g = g0; g < g1; g += N) {
    if (g1 - g0 > N) fetch(g);  // (else they are still there)
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int j = (g + n) * kWave + lane;
      if (blockIdx.x == 0 && g + n < g1 && j < m && t[n] < 0) rank[j] = -1;
      unsigned long long left = __ballot(t[n] >= lo && t[n] < lo + own);
      while (left) {  // one token of the group at a time; every round clears at least one bit
        const int u = __builtin_amdgcn_readlane(t[n], __builtin_ctzll(left));
        const unsigned long long same = __ballot(t[n] == u) & left;
        const int place = mine[u - lo];
        if (t[n] == u) rank[j] = place + __builtin_popcountll(same & ((1ull << lane) - 1));
        if (lane == 0) mine[u - lo] = place + __builtin_popcountll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        left &= ~same;
      }
    }
  }
}

// G [d][m] turned over into rows [place][dp], a tile of 64 columns x 64 features per workgroup. The only column of its
// token needs no sum: its row goes straight into the table's gradient. Bound by memory: 13 us for 1024 x 4096, 20 us for
// 784 x 9001 (its rows' starts lie off the cache lines).
template <typename T>
__global__ void __launch_bounds__(256) embed_turn_kernel(const float* __restrict__ G, const void* __restrict__ ids, int id_bits,
                                                         const int* __restrict__ rank, const int* __restrict__ start,
                                                         float scale, T* __restrict__ dTable, float* __restrict__ rows,
                                                         int vocab, int d, int dp, int m) {
  __shared__ float tile[kEmbedTile * kEmbedPad];
  const TileAt at((m + kEmbedTile - 1) / kEmbedTile);
  const int j0 = at.col * kEmbedTile, i0 = at.row * kEmbedTile;
  const int q = threadIdx.x & 15, p = threadIdx.x >> 4;
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const int i = i0 + p + 16 * s, j = j0 + 4 * q;
    if (i < d && j < m) {
      const Cols<float, 4> c = load_cols<float, 4>(G + (size_t)i * m + j, m - j);
#pragma unroll
      for (int e = 0; e < 4; ++e) tile[(4 * q + e) * kEmbedPad + p + 16 * s] = c.get(e);
    }
  }
  __syncthreads();
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const int j = j0 + p + 16 * s, i = i0 + 4 * q;
    if (j >= m || i >= d) continue;
    const int t = token_at(ids, id_bits, j, vocab);
    if (t < 0) continue;
    const float* src = tile + (p + 16 * s) * kEmbedPad + 4 * q;
    if (start[t + 1] - start[t] == 1) {
      Cols<T, 4> c;
#pragma unroll
      for (int e = 0; e < 4; ++e) c.set(e, scale * src[e]);
      store_cols<T, 4>(dTable + (size_t)t * d + i, d - i, c);
    } else {
      // (columns of the tile beyond d are never read: the row's end is padding up to dp)
      *reinterpret_cast<float4*>(rows + (size_t)rank[j] * dp + i) = make_float4(src[0], src[1], src[2], src[3]);
    }
  }
}

// Rows of the table's gradient, 64 tokens x 64 features per workgroup, 16 lanes x 4 features per token, four tokens per
// lane one after the other. A token with up to kEmbedFew columns is summed by its own lanes; for each one with more, all 16
// groups of lanes take every 16th column and their sums are added in a fixed order. Sums in fp32, rounded once to the
// table's type. Bound by writing the table's gradient, most of whose rows are zero for a mini-batch much smaller than
// the vocabulary: 32000 x 1024 fp32 (131 MB) 21 us, 6.2 TB/s. A small vocabulary leaves most of the GPU idle, as a tile's
// workgroup sums all columns of its tokens: 16384 columns of 64 features, 64 tokens 145 us, 256 tokens 68 us (of 1024
// features 159 and 78 us).
constexpr int kEmbedFew = 16;
template <typename T>
__global__ void __launch_bounds__(256) embed_sum_kernel(const float* __restrict__ rows, const int* __restrict__ start, float scale,
                                                        T* __restrict__ dTable, int vocab, int d, int dp) {
  __shared__ float part[4][kEmbedTile];
  const int features = (d + kEmbedTile - 1) / kEmbedTile;
  const TileAt at(features);
  const int t0 = (blockIdx.y * (int)(gridDim.x / features) + at.row) * kEmbedTile, i0 = at.col * kEmbedTile;
  if (t0 >= vocab) return;
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x >> 6;
  const int q = threadIdx.x & 15, p = threadIdx.x >> 4, i = i0 + 4 * q;
  // every wave holds the 64 tokens' places, one per lane
  const int first = start[min(t0 + lane, vocab)], count = start[min(t0 + lane + 1, vocab)] - first;
#pragma unroll
  for (int k = 0; k < kEmbedTile / 16; ++k) {
    const int u = p + 16 * k, t = t0 + u;
    const int a = __shfl(first, u, kWave), n = __shfl(count, u, kWave);
    if (t >= vocab || i >= d || n == 1 || n > kEmbedFew) continue;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    const float* src = rows + (size_t)a * dp + i;
#pragma unroll 4
    for (int c = 0; c < n; ++c) {
      const float4 g = *reinterpret_cast<const float4*>(src + (size_t)c * dp);
      sum.x += g.x; sum.y += g.y; sum.z += g.z; sum.w += g.w;
    }
    const float f = n ? scale : 0.f;  // a row of zeros, not of -0
    Cols<T, 4> c;
    c.set(0, f * sum.x); c.set(1, f * sum.y); c.set(2, f * sum.z); c.set(3, f * sum.w);
    store_cols<T, 4>(dTable + (size_t)t * d + i, d - i, c);
  }
  for (unsigned long long many = __ballot(count > kEmbedFew); many; many &= many - 1) {  // the same in all waves
    const int u = __builtin_ctzll(many);
    const int a = __builtin_amdgcn_readlane(first, u), n = __builtin_amdgcn_readlane(count, u);
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i < d) {
#pragma unroll 8
      for (int c = p; c < n; c += 16) {
        const float4 g = *reinterpret_cast<const float4*>(rows + (size_t)(a + c) * dp + i);
        sum.x += g.x; sum.y += g.y; sum.z += g.z; sum.w += g.w;
      }
    }
    sum.x = sum_lanes_from<16>(sum.x); sum.y = sum_lanes_from<16>(sum.y);
    sum.z = sum_lanes_from<16>(sum.z); sum.w = sum_lanes_from<16>(sum.w);
    if (lane < 16) *reinterpret_cast<float4*>(&part[wave][4 * q]) = sum;
    __syncthreads();
    if (wave == 0 && i0 + lane < d)
      dTable[(size_t)(t0 + u) * d + i0 + lane] = (T)(scale * ((part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane])));
    __syncthreads();
  }
}

struct EmbedLayout {
  int per, owners, dp;  // tokens per workgroup of embed_index_kernel, its workgroups; row length of the turned gradient
  size_t off_rank, off_start, off_rows, total;
};
static EmbedLayout make_embed_layout(const fasth_embed_shape& s) {
  EmbedLayout L;
  L.owners = std::max(kComputeUnits, (s.vocab + kIndexMaxPer - 1) / kIndexMaxPer);
  L.per = (s.vocab + L.owners - 1) / L.owners;
  L.owners = (s.vocab + L.per - 1) / L.per;
  L.dp = (s.d + 3) / 4 * 4;
  L.off_rank = 0;
  L.off_start = align_up((size_t)s.m * sizeof(int), 256);
  L.off_rows = L.off_start + align_up(((size_t)s.vocab + 1) * sizeof(int), 256);
  L.total = L.off_rows + align_up((size_t)s.m * L.dp * sizeof(float), 256);
  return L;
}

template <typename T>
static int launch_embed(const fasth_embed_shape& s, const void* table, const void* ids, float scale, float* X, hipStream_t stream) {
  const dim3 grid((s.m + kEmbedTile - 1) / kEmbedTile * ((s.d + kEmbedTile - 1) / kEmbedTile));
  hipLaunchKernelGGL((embed_kernel<T>), grid, dim3(256), 0, stream, static_cast<const T*>(table), ids, s.id_bits, scale, X,
                     s.vocab, s.d, s.m);
  FASTH_HIP(hipGetLastError());
  return FASTH_OK;
}

template <typename T>
static int launch_embed_grad(const fasth_embed_shape& s, const void* ids, const float* G, float scale, void* dTable, void* workspace,
                             hipStream_t stream) {
  const EmbedLayout L = make_embed_layout(s);
  char* ws = static_cast<char*>(workspace);
  int* rank = reinterpret_cast<int*>(ws + L.off_rank);
  int* start = reinterpret_cast<int*>(ws + L.off_start);
  float* rows = reinterpret_cast<float*>(ws + L.off_rows);
  T* out = static_cast<T*>(dTable);
  const int features = (s.d + kEmbedTile - 1) / kEmbedTile;
  hipLaunchKernelGGL(embed_index_kernel, dim3(L.owners), dim3(kIndexWaves * kWave), sizeof(int) * kIndexWaves * L.per, stream, ids,
                     s.id_bits, s.vocab, s.m, L.per, rank, start);
  FASTH_HIP(hipGetLastError());
  hipLaunchKernelGGL((embed_turn_kernel<T>), dim3((s.m + kEmbedTile - 1) / kEmbedTile * features), dim3(256), 0, stream, G, ids,
                     s.id_bits, rank, start, scale, out, rows, s.vocab, s.d, L.dp, s.m);
  FASTH_HIP(hipGetLastError());
  const int tokens = (s.vocab + kEmbedTile - 1) / kEmbedTile, deep = (tokens + 16383) / 16384;  // 256 x 16384 x 256 threads at most in a dimension
  hipLaunchKernelGGL((embed_sum_kernel<T>), dim3(features * ((tokens + deep - 1) / deep), deep), dim3(256), 0, stream, rows, start,
                     scale, out, s.vocab, s.d, L.dp);
  FASTH_HIP(hipGetLastError());
  return FASTH_OK;
}

}  // namespace fasth
