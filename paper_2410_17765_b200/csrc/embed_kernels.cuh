// Embedding lookup with scaling, and its gradient by sorted tokens.
#pragma once
#include "vec_io.cuh"

namespace cpmtp {
namespace embed {

using io::bf16_t;

constexpr int kSlab = 256;        // columns that a warp works on: eight to a lane

// The row of the table that token `x` names; V for padding.  Any other token out of range is clamped and reported.
__device__ __forceinline__ int row_of(int x, int V, int* dev_status) {
  if (x == CPMTP_EMBED_PAD) return V;
  if (x >= 0 && x < V) return x;
  if (dev_status != nullptr) atomicMax(dev_status, 1);
  return x < 0 ? 0 : V - 1;
}

// A warp copies kRowsPerWarp slabs of consecutive tokens, all read before the first is written.
constexpr int kFwdRows = 4;
template <class T, bool VEC>
__global__ void __launch_bounds__(256) embed_fwd_kernel(const bf16_t* __restrict__ E, long long ld_table, const int* __restrict__ x,
                                                        T* __restrict__ out, long long ld, int tokens, int V, int d, int slabs, float scale,
                                                        int* dev_status) {
  const int lane = threadIdx.x & 31;
  const long long item = static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5);
  const long long i0 = item / slabs * kFwdRows;
  const int c0 = static_cast<int>(item % slabs) * kSlab;
  ptx::grid_dep_wait();
  if (i0 >= tokens) return;
  int row = V;
  if (lane < kFwdRows && i0 + lane < tokens) row = row_of(x[i0 + lane], V, dev_status);
  float v[kFwdRows][8];
#pragma unroll
  for (int r = 0; r < kFwdRows; ++r) {
    const int id = __shfl_sync(0xffffffffu, row, r);
    if (id < V) {
      io::load_cols<VEC>(E + id * ld_table + c0, lane, 32, d - c0, v[r]);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[r][k] = 0.f;
    }
  }
#pragma unroll
  for (int r = 0; r < kFwdRows; ++r) {
    if (i0 + r >= tokens) break;
#pragma unroll
    for (int k = 0; k < 8; ++k) v[r][k] *= scale;
    // the zeros of padding stay zeros whatever the scale
    if (__shfl_sync(0xffffffffu, row, r) >= V) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[r][k] = 0.f;
    }
    io::store_cols<VEC>(out + (i0 + r) * ld + c0, lane, 32, d - c0, v[r]);
  }
}

// ---- sorting (token, position) by token, stable: least significant digit first ----
constexpr int kSortThreads = 512;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortRounds = 4;                              // keys per thread
constexpr int kSortKeys = kSortThreads * kSortRounds;       // keys per block
constexpr int kMaxBits = 9;                                 // bits per pass
constexpr int kMaxDigits = 1 << kMaxBits;

// Digit counts of the first pass per block, and zeros for those of the second.
__global__ void __launch_bounds__(kSortThreads) embed_hist_kernel(const int* __restrict__ x, int tokens, int V, int bits, int* __restrict__ hist,
                                                                  int* __restrict__ hist_next, int* dev_status) {
  __shared__ int h[kMaxDigits];
  const int digits = 1 << bits;
  for (int t = threadIdx.x; t < digits; t += kSortThreads) h[t] = 0;
  ptx::grid_dep_wait();
  __syncthreads();
  for (int r = 0; r < kSortRounds; ++r) {
    const long long i = static_cast<long long>(blockIdx.x) * kSortKeys + r * kSortThreads + threadIdx.x;
    if (i < tokens) atomicAdd(&h[row_of(x[i], V, dev_status) & (digits - 1)], 1);
  }
  __syncthreads();
  for (int t = threadIdx.x; t < digits; t += kSortThreads) {
    hist[static_cast<size_t>(blockIdx.x) * digits + t] = h[t];
    if (hist_next != nullptr) hist_next[static_cast<size_t>(blockIdx.x) * digits + t] = 0;
  }
}

// One pass: every key goes to its place among the keys of its digit.  FIRST: keys come from the tokens.  The digit
// counts that the next pass needs per block are taken as the keys are placed (integer atomics: order does not matter).
template <bool FIRST>
__global__ void __launch_bounds__(kSortThreads) embed_sort_kernel(const int* __restrict__ x, const uint2* __restrict__ in, uint2* __restrict__ out,
                                                                  int tokens, int V, int bits, int shift, const int* __restrict__ hist,
                                                                  int* __restrict__ hist_next, int* __restrict__ hist_zero) {
  __shared__ int counts[kSortWarps][kMaxDigits];
  __shared__ int warp_sums[kSortWarps];
  const int digits = 1 << bits, mask = digits - 1;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int j = threadIdx.x; j < kSortWarps * digits; j += kSortThreads) counts[j / digits][j % digits] = 0;
  ptx::grid_dep_wait();
  __syncthreads();
  uint2 key[kSortRounds];
  int rank[kSortRounds];
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const long long i = static_cast<long long>(blockIdx.x) * kSortKeys + warp * (32 * kSortRounds) + r * 32 + lane;
    const bool valid = i < tokens;
    key[r] = make_uint2(0xffffffffu, 0u);
    if (valid) key[r] = FIRST ? make_uint2(row_of(x[i], V, nullptr), static_cast<unsigned>(i)) : in[i];
    const int digit = valid ? static_cast<int>(key[r].x >> shift) & mask : -1;
    const unsigned peers = __match_any_sync(0xffffffffu, digit);
    const int leader = __ffs(peers) - 1;
    int base = 0;
    if (valid && lane == leader) {
      base = counts[warp][digit];
      counts[warp][digit] = base + __popc(peers);
    }
    rank[r] = __shfl_sync(0xffffffffu, base, leader) + __popc(peers & ((1u << lane) - 1u));
    __syncwarp();
  }
  __syncthreads();
  // thread = digit: keys of it in earlier warps of this block, in earlier blocks, and of smaller digits anywhere
  int total = 0, before = 0;
  if (static_cast<int>(threadIdx.x) < digits) {
    int run = 0;
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
      const int c = counts[w][threadIdx.x];
      counts[w][threadIdx.x] = run;
      run += c;
    }
    for (unsigned b = 0; b < gridDim.x; ++b) {
      const int c = hist[static_cast<size_t>(b) * digits + threadIdx.x];
      total += c;
      if (b < blockIdx.x) before += c;
    }
    if (hist_zero != nullptr) hist_zero[static_cast<size_t>(blockIdx.x) * digits + threadIdx.x] = 0;
  }
  int incl = total;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  int smaller = incl - total + before;
  for (int w = 0; w < warp; ++w) smaller += warp_sums[w];
  if (static_cast<int>(threadIdx.x) < digits) {
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) counts[w][threadIdx.x] += smaller;
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kSortRounds; ++r) {
    const long long i = static_cast<long long>(blockIdx.x) * kSortKeys + warp * (32 * kSortRounds) + r * 32 + lane;
    if (i < tokens) {
      const int to = counts[warp][(key[r].x >> shift) & mask] + rank[r];
      out[to] = key[r];
      if (hist_next != nullptr) atomicAdd(&hist_next[static_cast<size_t>(to / kSortKeys) * digits + ((key[r].x >> (shift + bits)) & mask)], 1);
    }
  }
}

// ---- sums over equal tokens ----
// A warp takes kChunk sorted positions and one slab of columns, and adds up each run of equal tokens in it.  A run that lies
// inside the chunk is written to the table; one that began before goes to head[chunk], one that began here and goes on to
// tail[chunk], and embed_join_kernel adds those up.  Work per warp is the same however unequal the tokens' counts are.
constexpr int kChunk = 32;
constexpr int kZeroRows = 32;     // rows of the table that a block looks at for rows without a token

struct SumParams {
  const uint2* sorted;
  long long ld, ld_table;
  bf16_t* dE;
  float *head, *tail;             // [chunks][slabs * kSlab]
  int tokens, V, d, slabs, chunks, accum, sum_blocks;
  float scale;
};

template <bool VEC>
__device__ __forceinline__ void write_row(const SumParams& p, int row, int c0, int lane, const float (&acc)[8]) {
  bf16_t* dst = p.dE + row * p.ld_table + c0;
  float v[8];
  if (p.accum) {
    io::load_cols<VEC>(dst, lane, 32, p.d - c0, v);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = fmaf(acc[k], p.scale, v[k]);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = acc[k] * p.scale;
  }
  io::store_cols<VEC>(dst, lane, 32, p.d - c0, v);
}

template <class T, bool VEC>
__global__ void __launch_bounds__(256) embed_sum_kernel(const T* __restrict__ dy, const SumParams p) {
  const int lane = threadIdx.x & 31;
  ptx::grid_dep_wait();
  if (static_cast<int>(blockIdx.x) >= p.sum_blocks) {
    // rows without a token: zeros
    __shared__ int present[kZeroRows];
    const int r0 = (blockIdx.x - p.sum_blocks) * kZeroRows;
    if (threadIdx.x < kZeroRows) present[threadIdx.x] = 0;
    int lo = 0, hi = p.tokens;                   // first sorted position whose token is at least r0
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (static_cast<int>(p.sorted[mid].x) < r0) lo = mid + 1; else hi = mid;
    }
    __syncthreads();
    for (int j = lo + threadIdx.x; j < p.tokens; j += 256) {
      const int at = static_cast<int>(p.sorted[j].x) - r0;
      if (at >= kZeroRows) break;
      present[at] = 1;
    }
    __syncthreads();
    const float zeros[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int r = 0; r < kZeroRows && r0 + r < p.V; ++r) {
      if (present[r]) continue;
      bf16_t* dst = p.dE + (r0 + r) * p.ld_table;
      for (int c0 = (threadIdx.x >> 5) * kSlab; c0 < p.d; c0 += 8 * kSlab) io::store_cols<VEC>(dst + c0, lane, 32, p.d - c0, zeros);
    }
    return;
  }
  const long long item = static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5);
  const long long chunk = item / p.slabs;
  if (chunk >= p.chunks) return;
  const int slab = static_cast<int>(item % p.slabs), c0 = slab * kSlab;
  const long long j0 = chunk * kChunk;
  uint2 kp = make_uint2(p.V, 0u);
  if (j0 + lane < p.tokens) kp = p.sorted[j0 + lane];
  const int before = j0 > 0 ? static_cast<int>(p.sorted[j0 - 1].x) : -1;
  const int after = j0 + kChunk < p.tokens ? static_cast<int>(p.sorted[j0 + kChunk].x) : -1;
  float acc[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) acc[k] = 0.f;
  int cur = __shfl_sync(0xffffffffu, static_cast<int>(kp.x), 0);
  bool began_before = cur == before;
  auto flush = [&](bool goes_on) {
    if (cur >= p.V) return;
    if (!began_before && !goes_on) {
      write_row<VEC>(p, cur, c0, lane, acc);
    } else {
      float* to = (began_before ? p.head : p.tail) + (chunk * p.slabs + slab) * kSlab;
#pragma unroll
      for (int k = 0; k < 8; ++k) to[lane * 8 + k] = acc[k];
    }
  };
  constexpr int kAhead = 8;
#pragma unroll 1
  for (int k0 = 0; k0 < kChunk; k0 += kAhead) {
    float v[kAhead][8];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int row = __shfl_sync(0xffffffffu, static_cast<int>(kp.x), k0 + u);
      const long long pos = __shfl_sync(0xffffffffu, kp.y, k0 + u);
      if (row < p.V) {
        io::load_cols<VEC>(dy + pos * p.ld + c0, lane, 32, p.d - c0, v[u]);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) v[u][k] = 0.f;
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int row = __shfl_sync(0xffffffffu, static_cast<int>(kp.x), k0 + u);
      if (row != cur) {
        flush(false);
        cur = row;
        began_before = false;
#pragma unroll
        for (int k = 0; k < 8; ++k) acc[k] = 0.f;
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) acc[k] += v[u][k];
    }
  }
  flush(cur == after);
}

// Runs that cross a chunk's end: the warp of the chunk in which one begins adds its parts up in order.
template <bool VEC>
__global__ void __launch_bounds__(256) embed_join_kernel(const SumParams p) {
  const int lane = threadIdx.x & 31;
  const long long item = static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5);
  ptx::grid_dep_wait();
  const long long chunk = item / p.slabs;
  if (chunk + 1 >= p.chunks) return;
  const int slab = static_cast<int>(item % p.slabs), c0 = slab * kSlab;
  const long long j0 = chunk * kChunk;
  const int row = static_cast<int>(p.sorted[j0 + kChunk - 1].x);
  if (row >= p.V || static_cast<int>(p.sorted[j0 + kChunk].x) != row) return;
  if (j0 > 0 && static_cast<int>(p.sorted[j0].x) == row && static_cast<int>(p.sorted[j0 - 1].x) == row) return;
  const size_t width = static_cast<size_t>(p.slabs) * kSlab;
  float acc[8], v[8];
  io::load8(p.tail + chunk * width + c0 + 8 * lane, acc);
  for (long long c = chunk + 1; c < p.chunks && static_cast<int>(p.sorted[c * kChunk].x) == row; ++c) {
    io::load8(p.head + c * width + c0 + 8 * lane, v);
#pragma unroll
    for (int k = 0; k < 8; ++k) acc[k] += v[k];
  }
  write_row<VEC>(p, row, c0, lane, acc);
}

}  // namespace embed
}  // namespace cpmtp
