// Embedding lookup with scaling, and its gradient by sorted tokens.  Bound by bandwidth where there is much to move (lookup of
// 8192 x 2048 into fp32: 13.7 us, 5.6 TB/s; gradient of 16384 x 4096 over 128256 rows: 196 us, 6.0 TB/s); a gradient that touches
// few rows also pays for the sort and the joining of runs (8192 x 4096 into a tied table: 8 + 21 + 5 us).
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

// A lane's eight columns of a slab as they lie in memory: 8 lane .. 8 lane + 7 (VEC), else every 32nd.  They become numbers
// only when they are used, so that a warp has the loads of several rows under way.  `left`: columns from the slab's start on.
template <class T, bool VEC>
struct Slab {
  T v[8];
  __device__ __forceinline__ void read(const T* row, int lane, int left) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = row[min(lane + 32 * k, left - 1)];       // (past the end: the last one, not written)
  }
  __device__ __forceinline__ void get(float (&out)[8]) const {
#pragma unroll
    for (int k = 0; k < 8; ++k) out[k] = io::to_f(v[k]);
  }
};
template <class T>
struct Slab<T, true> {
  uint32_t v[2 * sizeof(T)];
  __device__ __forceinline__ void read(const T* row, int lane, int left) { io::load8_raw(row + min(8 * lane, left - 8), v); }
  __device__ __forceinline__ void get(float (&out)[8]) const { io::numbers8<T>(v, out); }
};

// A warp copies the slabs of kFwdRows consecutive tokens, all read before the first is written.
constexpr int kFwdRows = 4;
template <class T, bool VEC>
__global__ void __launch_bounds__(256) embed_fwd_kernel(const bf16_t* __restrict__ E, long long ld_table, const int* __restrict__ x,
                                                        T* __restrict__ out, long long ld, int tokens, int V, int d, int slabs, float scale,
                                                        int* dev_status) {
  const int lane = threadIdx.x & 31;
  const long long item = static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5);
  const long long i0 = item / slabs * kFwdRows;
  const int c0 = static_cast<int>(item % slabs) * kSlab, left = d - c0;
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  if (i0 >= tokens) return;
  int row = V;
  if (lane < kFwdRows && i0 + lane < tokens) row = row_of(x[i0 + lane], V, dev_status);
  Slab<bf16_t, VEC> in[kFwdRows];
#pragma unroll
  for (int r = 0; r < kFwdRows; ++r) {
    const int id = __shfl_sync(0xffffffffu, row, r);
    in[r].read(E + (id < V ? id : 0) * ld_table + c0, lane, left);
  }
#pragma unroll
  for (int r = 0; r < kFwdRows; ++r) {
    if (i0 + r >= tokens) break;
    float v[8];
    in[r].get(v);
    const bool pad = __shfl_sync(0xffffffffu, row, r) >= V;
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = pad ? 0.f : v[k] * scale;      // (padding is zero whatever the scale)
    io::store_cols<VEC>(out + (i0 + r) * ld + c0, lane, 32, left, v);
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
  ptx::grid_dep_launch();
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
  for (int j = threadIdx.x; j < kSortWarps * digits; j += kSortThreads) counts[j >> bits][j & mask] = 0;
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
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
    int next = -1;                               // where this key is counted for the next pass
    if (i < tokens) {
      const int to = counts[warp][(key[r].x >> shift) & mask] + rank[r];
      out[to] = key[r];
      next = (to / kSortKeys << bits) + static_cast<int>(key[r].x >> (shift + bits) & mask);
    }
    if (hist_next != nullptr) {
      // one atomic for the keys of a warp that count at the same place: frequent tokens have small ids, and so one digit here
      const unsigned peers = __match_any_sync(0xffffffffu, next);
      if (next >= 0 && lane == __ffs(peers) - 1) atomicAdd(&hist_next[next], __popc(peers));
    }
  }
}

// ---- the same in one launch, for as many tokens as the shared memory of a cluster holds ----
// CTAs blocks of 1024 threads keep KPT keys a thread between passes in their shared memory, tell one another their digit
// counts and hand the keys over through it.  Three launches and their gaps become one: 13 -> 8 us at 8192 tokens.
constexpr int kClusterThreads = 1024, kClusterWarps = kClusterThreads / 32, kClusterSize = 8;

__host__ __device__ constexpr int cluster_sort_bytes(int ctas, int kpt) {
  return kClusterThreads * kpt * 8 + kClusterWarps * kMaxDigits * 2 + (ctas + 1) * kMaxDigits * 4;
}

template <int CTAS>
__device__ __forceinline__ void sync_ctas() {
  if (CTAS == 1) {
    __syncthreads();
  } else {
    __syncwarp();                                             // (a warp arrives as a whole)
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
}
// The address in block `cta` of the cluster of what `p` is here.
__device__ __forceinline__ uint32_t remote(const void* p, int cta) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(ptx::smem_u32(p)), "r"(cta));
  return r;
}

template <int CTAS, int KPT>
__global__ void __launch_bounds__(kClusterThreads) embed_sort_cluster_kernel(const int* __restrict__ x, uint2* __restrict__ out, int tokens, int V,
                                                                             int bits, int passes, int* dev_status) {
  extern __shared__ __align__(16) uint8_t smem[];
  constexpr int kKeys = kClusterThreads * KPT;                // of one block
  uint2* keys = reinterpret_cast<uint2*>(smem);
  auto counts = reinterpret_cast<uint16_t (*)[kMaxDigits]>(smem + kKeys * 8);      // [kClusterWarps][kMaxDigits]
  int* base = reinterpret_cast<int*>(smem + kKeys * 8 + kClusterWarps * kMaxDigits * 2);
  int* all = base + kMaxDigits;                               // [CTAS][kMaxDigits]: every block's digit counts
  __shared__ int warp_sums[kClusterWarps];
  const int digits = 1 << bits, mask = digits - 1, cta = CTAS == 1 ? 0 : blockIdx.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = threadIdx.x;
  if (CTAS > 1) sync_ctas<CTAS>();                // every block is there before its memory is written to
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
#pragma unroll 1
  for (int pass = 0; pass < passes; ++pass) {
    const int shift = pass * bits;
    for (int j = t; j < kClusterWarps * kMaxDigits / 8; j += kClusterThreads) reinterpret_cast<uint4*>(counts)[j] = make_uint4(0u, 0u, 0u, 0u);
    uint2 key[KPT];
    int rank[KPT];
#pragma unroll
    for (int r = 0; r < KPT; ++r) {
      const int local = warp * (32 * KPT) + r * 32 + lane, i = cta * kKeys + local;
      key[r] = make_uint2(0xffffffffu, 0u);
      if (i < tokens) key[r] = pass == 0 ? make_uint2(row_of(x[i], V, dev_status), static_cast<unsigned>(i)) : keys[local];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < KPT; ++r) {
      const bool valid = cta * kKeys + warp * (32 * KPT) + r * 32 + lane < tokens;
      const int digit = valid ? static_cast<int>(key[r].x >> shift) & mask : -1;
      const unsigned peers = __match_any_sync(0xffffffffu, digit);
      const int leader = __ffs(peers) - 1;
      int first = 0;
      if (valid && lane == leader) {
        first = counts[warp][digit];
        counts[warp][digit] = static_cast<uint16_t>(first + __popc(peers));
      }
      rank[r] = __shfl_sync(0xffffffffu, first, leader) + __popc(peers & ((1u << lane) - 1u));
      __syncwarp();
    }
    __syncthreads();
    // thread = digit: its keys in earlier warps; its count to every block of the cluster
    if (t < digits) {
      int run = 0;
#pragma unroll
      for (int w = 0; w < kClusterWarps; ++w) {
        const int c = counts[w][t];
        counts[w][t] = static_cast<uint16_t>(run);
        run += c;
      }
      if (CTAS == 1) {
        all[t] = run;
      } else {
#pragma unroll
        for (int c = 0; c < CTAS; ++c)
          asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(remote(all + cta * kMaxDigits + t, c)), "r"(run) : "memory");
      }
    }
    sync_ctas<CTAS>();
    int total = 0, before = 0;
    if (t < digits) {
#pragma unroll
      for (int c = 0; c < CTAS; ++c) {
        const int n = all[c * kMaxDigits + t];
        total += n;
        if (c < cta) before += n;
      }
    }
    int incl = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += v;
    }
    if (lane == 31) warp_sums[warp] = incl;
    __syncthreads();
    if (t < digits) {
      int smaller = incl - total + before;
      for (int w = 0; w < warp; ++w) smaller += warp_sums[w];
      base[t] = smaller;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < KPT; ++r) {
      if (cta * kKeys + warp * (32 * KPT) + r * 32 + lane >= tokens) continue;
      const int digit = static_cast<int>(key[r].x >> shift) & mask;
      const int to = base[digit] + counts[warp][digit] + rank[r];
      if (pass + 1 == passes) {
        out[to] = key[r];
      } else if (CTAS == 1) {
        keys[to] = key[r];
      } else {
        asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(remote(keys + to % kKeys, to / kKeys)), "r"(key[r].x), "r"(key[r].y) : "memory");
      }
    }
    if (pass + 1 < passes) sync_ctas<CTAS>();
  }
}

// ---- sums over equal tokens ----
// A warp takes a chunk of sorted positions and one slab of columns, and adds up each run of equal tokens in it.  A run that lies
// inside the chunk is written to the table; one that began before goes to head[chunk], one that began here and goes on to
// tail[chunk], and embed_join_kernel adds those up.  Work per warp is the same however unequal the tokens' counts are.
// Rows are read kAhead at a time, and with them the rows of the table that the runs ending among them are added to: a
// warp that waited for one of those at every run's end spent three quarters of its time there.
// Chunks are kChunk long, or kShortChunk where few tokens would leave most of the GPU without a warp (736 tokens of 564
// columns: 44 -> 16 us; at 9300 tokens of 256 the parts of a frequent token get too many, 25 -> 31 us).
constexpr int kChunk = 32, kShortChunk = 8;
constexpr int kAhead = 4;
constexpr int kZeroRows = 32;     // rows of the table that a block looks at for rows without a token

struct SumParams {
  const uint2* sorted;
  long long ld, ld_table;
  bf16_t* dE;
  float *head, *tail;             // [chunks][slabs * kSlab]
  int tokens, V, d, slabs, chunk, chunks, sum_blocks;
  float scale;
};

using io::f32x2;

template <bool VEC, bool ACCUM>
__device__ __forceinline__ void write_slab(bf16_t* row, int lane, int left, float scale, const f32x2 (&acc)[4], const Slab<bf16_t, VEC>& before) {
  float v[8], old[8];
  io::singles(acc, v);
  if (ACCUM) before.get(old);
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = ACCUM ? fmaf(v[k], scale, old[k]) : v[k] * scale;
  io::store_cols<VEC>(row, lane, 32, left, v);
}

// Zeros for the rows of the table that no token names.
template <bool VEC>
__device__ __forceinline__ void zero_rows(const SumParams& p, int r0) {
  __shared__ int present[kZeroRows];
  const int lane = threadIdx.x & 31;
  if (threadIdx.x < kZeroRows) present[threadIdx.x] = 0;
  int lo = 0, hi = p.tokens;                     // first sorted position whose token is at least r0
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
}

template <class T, bool VEC, bool ACCUM>
__global__ void __launch_bounds__(256, sizeof(T) == 4 || !VEC ? 2 : 4) embed_sum_kernel(const T* __restrict__ dy, const SumParams p) {
  const int lane = threadIdx.x & 31;
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  if (static_cast<int>(blockIdx.x) >= p.sum_blocks) {
    zero_rows<VEC>(p, (blockIdx.x - p.sum_blocks) * kZeroRows);
    return;
  }
  const long long item = static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5);
  const long long chunk = item / p.slabs;
  if (chunk >= p.chunks) return;
  const int slab = static_cast<int>(item % p.slabs), c0 = slab * kSlab, left = p.d - c0;
  const long long j0 = chunk * p.chunk;
  uint2 kp = make_uint2(p.V, 0u);
  if (lane < p.chunk && j0 + lane < p.tokens) kp = p.sorted[j0 + lane];
  const int before = j0 > 0 ? static_cast<int>(p.sorted[j0 - 1].x) : -1;
  const int after = j0 + p.chunk < p.tokens ? static_cast<int>(p.sorted[j0 + p.chunk].x) : -1;
  const int mine = static_cast<int>(kp.x), last = p.chunk - 1;
  int next = __shfl_down_sync(0xffffffffu, mine, 1);
  if (lane == last) next = after;
  // by position: whether its run ends there; whether that run is all in this chunk and goes to the table
  const unsigned ends = __ballot_sync(0xffffffffu, mine != next);
  const bool first_run = mine == before;         // (only the run that the chunk begins with can have begun before)
  const unsigned writes = __ballot_sync(0xffffffffu, mine != next && mine < p.V && !first_run);
  const unsigned head = __ballot_sync(0xffffffffu, first_run);
  const unsigned none = __ballot_sync(0xffffffffu, mine >= p.V);
  const size_t part = (chunk * p.slabs + slab) * kSlab + 8 * lane;
  f32x2 acc[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) acc[k] = 0ull;
#pragma unroll 1
  for (int k0 = 0; k0 < p.chunk; k0 += kAhead) {
    Slab<T, VEC> rows[kAhead];
    Slab<bf16_t, VEC> old[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const long long pos = __shfl_sync(0xffffffffu, kp.y, k0 + u);      // (0 where there is none)
      rows[u].read(dy + pos * p.ld + c0, lane, left);
    }
    if (ACCUM) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const long long row = __shfl_sync(0xffffffffu, mine, k0 + u);
        if ((writes >> (k0 + u)) & 1u) old[u].read(p.dE + row * p.ld_table + c0, lane, left);
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const unsigned bit = 1u << (k0 + u);
      if (none & bit) return;                    // padding sorts last
      float v[8];
      rows[u].get(v);
      f32x2 add[4];
      io::pairs(v, add);
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[k] = io::add2(acc[k], add[k]);
      const long long row = __shfl_sync(0xffffffffu, mine, k0 + u);
      if (ends & bit) {
        if (writes & bit) {
          write_slab<VEC, ACCUM>(p.dE + row * p.ld_table + c0, lane, left, p.scale, acc, old[u]);
        } else {
          io::singles(acc, v);
          io::store8(p.head + part, v);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[k] = 0ull;
      }
    }
  }
  if (!((ends >> last) & 1u)) {                  // the last run goes on
    float v[8];
    io::singles(acc, v);
    io::store8((((head >> last) & 1u) ? p.head : p.tail) + part, v);
  }
}

// Runs that cross a chunk's end: the warp of the chunk in which one begins adds its parts up in order.
template <bool VEC, bool ACCUM>
__global__ void __launch_bounds__(256) embed_join_kernel(const SumParams p) {
  const int lane = threadIdx.x & 31;
  const long long item = static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5);
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const long long chunk = item / p.slabs;
  if (chunk + 1 >= p.chunks) return;
  const int slab = static_cast<int>(item % p.slabs), c0 = slab * kSlab, left = p.d - c0;
  const long long j0 = chunk * p.chunk;
  const int row = static_cast<int>(p.sorted[j0 + p.chunk - 1].x), first = static_cast<int>(p.sorted[j0].x);
  const int before = j0 > 0 ? static_cast<int>(p.sorted[j0 - 1].x) : -1, after = static_cast<int>(p.sorted[j0 + p.chunk].x);
  if (row >= p.V || after != row || (first == row && before == row)) return;
  const size_t width = static_cast<size_t>(p.slabs) * kSlab;
  const float* tail = p.tail + chunk * width + c0 + 8 * lane;
  const float* head = p.head + (chunk + 1) * width + c0 + 8 * lane;
  bf16_t* dst = p.dE + row * p.ld_table + c0;
  float t[8];
  Slab<bf16_t, VEC> old;
  io::load8(tail, t);
  if (ACCUM) old.read(dst, lane, left);
  f32x2 acc[4];
  io::pairs(t, acc);
  // chunks that the run reaches into: 32 are looked at together, and their parts read kParts at a time
  constexpr int kParts = 8;
  for (long long c = chunk + 1;; c += 32) {
    const bool goes = c + lane < p.chunks && static_cast<int>(p.sorted[(c + lane) * p.chunk].x) == row;
    const unsigned mask = __ballot_sync(0xffffffffu, goes);
    const int n = mask == 0xffffffffu ? 32 : __ffs(~mask) - 1;
    for (int j = 0; j < n; j += kParts) {
      float v[kParts][8];
#pragma unroll
      for (int u = 0; u < kParts; ++u)
        if (j + u < n) io::load8(head + (j + u) * width, v[u]);
#pragma unroll
      for (int u = 0; u < kParts; ++u) {
        if (j + u >= n) break;
        f32x2 add[4];
        io::pairs(v[u], add);
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[k] = io::add2(acc[k], add[k]);
      }
    }
    if (n < 32) break;
    head += 32 * width;
  }
  write_slab<VEC, ACCUM>(dst, lane, left, p.scale, acc, old);
}

}  // namespace embed
}  // namespace cpmtp
