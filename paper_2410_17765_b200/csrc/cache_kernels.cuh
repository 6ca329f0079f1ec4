// Paged cache of keys and values: appending, and eviction by accumulated attention weight.
#pragma once
#include <cstdint>

#include "../../include/cpmtp.h"
#include "cluster.cuh"
#include "ptx.cuh"
#include "vec_io.cuh"

namespace cpmtp {
namespace cache {

using io::bf16_t;

constexpr int kBadIndex = 1, kWaitTimeout = 2;      // values of the device status word

__device__ __forceinline__ void raise_status(int* dev_status, int value) {
  if (dev_status != nullptr) atomicMax(dev_status, value);
}

// Slots in use, and new tokens, of sequence b; numbers out of range are clamped.
__device__ __forceinline__ int seq_len(const cpmtp_cache& c, const cpmtp_cache_seqs& s, int b, int* dev_status) {
  const int n = s.lens[b], most = s.width * c.page_slots;
  if (n < 0 || n > most) raise_status(dev_status, kBadIndex);
  return min(max(n, 0), most);
}
__device__ __forceinline__ int seq_new(const cpmtp_cache_seqs& s, int b, int* dev_status) {
  if (s.q_lens == nullptr) return s.Q;
  const int n = s.q_lens[b];
  if (n < 0 || n > s.Q) raise_status(dev_status, kBadIndex);
  return min(max(n, 0), s.Q);
}
// Page number, or -1 where the table has none.
__device__ __forceinline__ int page_of(int page, int pages, int* dev_status) {
  if (page >= 0 && page < pages) return page;
  raise_status(dev_status, kBadIndex);
  return -1;
}

constexpr int kThreads = 256;
// One thread for a piece of eight elements of the keys and values of four tokens in one head: eight loads under way.  Four prompts of up to 2048 tokens,
// 8 heads of 128 (50 MB in all): 7.8 us, 6.4 TB/s, mostly within L2; with a token to a thread 12.4.  A draft's tokens take 3.1, the latency of lengths, table and copy.
constexpr int kTokens = 4;
template <bool VEC>
__global__ void __launch_bounds__(kThreads) append_kernel(const __grid_constant__ cpmtp_cache c, const __grid_constant__ cpmtp_cache_seqs s,
                                                          const __grid_constant__ cpmtp_tokens k, const __grid_constant__ cpmtp_tokens v,
                                                          int* dev_status) {
  ptx::grid_dep_wait();
  const unsigned pieces = c.D / 8, runs = (s.Q + kTokens - 1) / kTokens, row = pieces * c.H;      // a row of threads has one run of tokens
  const long long items = static_cast<long long>(s.B) * runs * row;
  for (long long i = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x; i < items; i += static_cast<long long>(gridDim.x) * kThreads) {
    const long long r = i / row;
    const unsigned in = static_cast<unsigned>(i - r * row);
    const int h = in / pieces, col = 8 * (in % pieces), b = static_cast<int>(r / runs), j0 = static_cast<int>(r - static_cast<long long>(b) * runs) * kTokens;
    const int fresh = seq_new(s, b, dev_status);
    if (j0 >= fresh) continue;
    // (a length that is too large is not clamped: the tokens that have slots keep them, and the others are left out)
    const int len = s.lens[b], most = s.width * c.page_slots, slot0 = min(max(len, 0), most + fresh) - fresh + j0;
    if (len < 0 || len > most) raise_status(dev_status, kBadIndex);
    const bf16_t* kp = static_cast<const bf16_t*>(k.data) + b * k.seq + h * k.head + col;
    const bf16_t* vp = static_cast<const bf16_t*>(v.data) + b * v.seq + h * v.head + col;
    uint4 x[kTokens], y[kTokens];
    int page[kTokens];
#pragma unroll
    for (int q = 0; q < kTokens; ++q) {
      const int j = j0 + q, slot = slot0 + q;
      page[q] = -1;
      if (j >= fresh) continue;
      if (slot < 0 || slot >= most) {
        raise_status(dev_status, kBadIndex);
        continue;
      }
      page[q] = s.table[b * s.ld_table + slot / c.page_slots];
      if (VEC) {
        x[q] = *reinterpret_cast<const uint4*>(kp + j * k.token);
        y[q] = *reinterpret_cast<const uint4*>(vp + j * v.token);
      } else {
        bf16_t e[16];
#pragma unroll
        for (int w = 0; w < 8; ++w) {
          e[w] = kp[j * k.token + w];
          e[8 + w] = vp[j * v.token + w];
        }
        x[q] = make_uint4(e[0] | static_cast<uint32_t>(e[1]) << 16, e[2] | static_cast<uint32_t>(e[3]) << 16, e[4] | static_cast<uint32_t>(e[5]) << 16,
                          e[6] | static_cast<uint32_t>(e[7]) << 16);
        y[q] = make_uint4(e[8] | static_cast<uint32_t>(e[9]) << 16, e[10] | static_cast<uint32_t>(e[11]) << 16, e[12] | static_cast<uint32_t>(e[13]) << 16,
                          e[14] | static_cast<uint32_t>(e[15]) << 16);
      }
      page[q] = page_of(page[q], c.pages, dev_status);
    }
#pragma unroll
    for (int q = 0; q < kTokens; ++q) {
      if (page[q] < 0) continue;
      const int at = (slot0 + q) % c.page_slots;
      *reinterpret_cast<uint4*>(static_cast<bf16_t*>(c.k) + page[q] * c.k_page + at * c.k_slot + h * c.k_head + col) = x[q];
      *reinterpret_cast<uint4*>(static_cast<bf16_t*>(c.v) + page[q] * c.v_page + at * c.v_slot + h * c.v_head + col) = y[q];
      if (col == 0 && c.acc != nullptr) c.acc[page[q] * c.acc_page + h * c.acc_head + at] = 0.f;
    }
  }
}

// ---------------------------------------------------------------------------------------------- eviction

constexpr int kSelectThreads = 512, kSelectWarps = kSelectThreads / 32;
constexpr int kDigits = 2048;                    // eleven bits at a time

struct Select {
  uint32_t hist[kDigits];
  uint32_t scan[kSelectWarps], scan2[kSelectWarps];
  cluster::u64 box[4][cluster::kMostCtas];
  uint32_t digit, left, unused[2];
};
static_assert(sizeof(Select) % 16 == 0, "the keys follow");

// The order in which slots are kept: the last `recent` ones before all others, then by accumulated weight; NaN is the least.
__device__ __forceinline__ uint32_t keep_key(float acc) { return acc != acc ? 0u : cluster::order_key(acc); }

// A cluster for each head of each sequence, a block for `span` of its slots.  The last key to be kept is found by its digits, eleven bits at
// a time from histograms; then every warp numbers the kept slots of its range.  Keys stay in shared memory (HELD).  `vec`: acc can be read
// 16 bytes at a time.  Latency bounds it, of barriers of the cluster above all: three to a digit (under the profiler, cold: 128 heads of 4352 slots 16 us, 16 of 65536 24).
// Slots are shared out by the width of the table: 16 sequences of 4352 slots, eviction in all, take 105 us in a table of their own, 145 in one for 131072 and 188 in one for 2^20.
template <bool HELD>
__global__ void __launch_bounds__(kSelectThreads) select_kernel(const __grid_constant__ cpmtp_cache c, const __grid_constant__ cpmtp_cache_seqs s,
                                                                int ctas, int span, int vec, int budget, int recent, int* lens_out, int* kept, int* dev_status) {
  extern __shared__ __align__(16) uint8_t smem[];
  Select& sh = *reinterpret_cast<Select*>(smem);
  uint32_t* keys = reinterpret_cast<uint32_t*>(smem + sizeof(Select));
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int rank = static_cast<int>(blockIdx.x) % ctas, h = static_cast<int>(blockIdx.x) / ctas, b = blockIdx.y;
  ptx::grid_dep_wait();
  const int len = seq_len(c, s, b, dev_status);
  const int* row = s.table + b * s.ld_table;
  int* out = kept + (static_cast<long long>(b) * c.H + h) * budget;
  if (h == 0 && rank == 0 && t == 0) lens_out[b] = min(len, budget);
  if (len <= budget) {
    for (int i = rank * kSelectThreads + t; i < budget; i += ctas * kSelectThreads) out[i] = i < len ? i : -1;
    ptx::grid_dep_launch();
    return;                                      // (all blocks of the cluster do)
  }
  const int from = len - recent, base = min(rank * span, len), n = min(span, len - base);
  auto read = [&](int i) {                       // of the i-th slot of this block
    const int slot = base + i;
    if (slot >= from) return 0xffffffffu;
    const int page = page_of(row[slot / c.page_slots], c.pages, dev_status);
    return page < 0 ? 0u : keep_key(c.acc[page * c.acc_page + h * c.acc_head + slot % c.page_slots]);
  };
  auto key = [&](int i) { return HELD ? keys[i] : read(i); };
  auto sync = [&] { cluster::sync_row(ctas); };
  int boxes = 0;
  auto exchange = [&](cluster::u64 v) {          // v of thread 0 to every block, and theirs
    cluster::u64* box = sh.box[boxes++ & 3];
    v = __shfl_sync(0xffffffffu, v, 0);
    if (t < ctas) {
      if (ctas == 1) box[0] = v;
      else cluster::store_remote(box + rank, t, v);
    }
    sync();
    return box;
  };
  for (int i = t; i < kDigits; i += kSelectThreads) sh.hist[i] = 0;
  __syncthreads();
  uint32_t prefix = 0, mask = 0, need = budget;  // how many of the keys with this prefix are kept, the largest first
#pragma unroll 1
  for (int d = 0; d < 3; ++d) {
    const int shift = d == 0 ? 21 : d == 1 ? 10 : 0;
    const uint32_t digits = d < 2 ? kDigits - 1 : 1023;
    if (d == 0) {
      // eight slots at a time, which lie in one page: one lookup, and the next one's under way
      int page = -1;
      auto look = [&](int i) { return i < n ? row[(base + i) / c.page_slots] : 0; };
      int next = look(8 * t);
      for (int i = 8 * t; i < n; i += 8 * kSelectThreads) {
        page = page_of(next, c.pages, dev_status);
        next = look(i + 8 * kSelectThreads);
        const float* acc = c.acc + (page < 0 ? 0 : page * c.acc_page + h * c.acc_head + (base + i) % c.page_slots);
        float v[8];
        if (vec) {
          const float4 x = *reinterpret_cast<const float4*>(acc), y = *reinterpret_cast<const float4*>(acc + 4);
          v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
          v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
        } else {
#pragma unroll
          for (int q = 0; q < 8; ++q) v[q] = acc[q];
        }
        uint32_t k[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          k[q] = base + i + q >= from ? 0xffffffffu : page < 0 ? 0u : keep_key(v[q]);
          if (i + q < n) atomicAdd(&sh.hist[k[q] >> 21], 1u);
        }
        if (HELD) {
          *reinterpret_cast<uint4*>(keys + i) = make_uint4(k[0], k[1], k[2], k[3]);
          *reinterpret_cast<uint4*>(keys + i + 4) = make_uint4(k[4], k[5], k[6], k[7]);
        }
      }
    } else {
#pragma unroll 4
      for (int i = t; i < n; i += kSelectThreads) {
        const uint32_t k = key(i);
        if ((k & mask) == prefix) atomicAdd(&sh.hist[k >> shift & digits], 1u);
      }
    }
    sync();
    // this block's share of the digits, the largest first; four to a thread at most
    const int per = kDigits / ctas, each = (per + kSelectThreads - 1) / kSelectThreads;
    uint32_t mine[kDigits / kSelectThreads], sum = 0;
#pragma unroll
    for (int j = 0; j < kDigits / kSelectThreads; ++j) {
      mine[j] = 0;
      const int at = t * each + j;
      if (j < each && at < per) {
        const int digit = kDigits - 1 - (rank * per + at);
        uint32_t v[cluster::kMostCtas];
#pragma unroll
        for (int r = 0; r < cluster::kMostCtas; ++r) v[r] = r < ctas ? (ctas == 1 ? sh.hist[digit] : cluster::load_remote32(&sh.hist[digit], r)) : 0;
#pragma unroll
        for (int r = 0; r < cluster::kMostCtas; ++r) mine[j] += v[r];
        sum += mine[j];
      }
    }
    uint32_t upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += v;
    }
    __syncthreads();
    if (lane == 31) sh.scan[warp] = upto;
    __syncthreads();
    uint32_t all = 0;
    for (int w = 0; w < kSelectWarps; ++w) {
      if (w < warp) upto += sh.scan[w];
      all += sh.scan[w];
    }
    const cluster::u64* box = exchange(all);     // (and the histograms have been read)
    uint32_t run = upto - sum;
    for (int r = 0; r < rank; ++r) run += static_cast<uint32_t>(box[r]);
#pragma unroll
    for (int j = 0; j < kDigits / kSelectThreads; ++j) {
      if (run < need && run + mine[j] >= need) {
        const uint32_t digit = kDigits - 1 - (rank * per + t * each + j);
        for (int r = 0; r < ctas; ++r) {
          asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster::remote(&sh.digit, r)), "r"(digit) : "memory");
          asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster::remote(&sh.left, r)), "r"(need - run) : "memory");
        }
      }
      run += mine[j];
    }
    for (int i = t; i < kDigits; i += kSelectThreads) sh.hist[i] = 0;
    sync();
    prefix |= sh.digit << shift;
    need = sh.left;
    mask |= digits << shift;
  }
  // keys above `prefix`, and the first `need` equal to it
  const int range = ((n + kSelectWarps - 1) / kSelectWarps + 31) / 32 * 32, w0 = min(warp * range, n), w1 = min(w0 + range, n);
  uint32_t above = 0, ties = 0;
  for (int i = w0 + lane; i < w1; i += 32) {
    const uint32_t k = key(i);
    above += k > prefix;
    ties += k == prefix;
  }
  above = __reduce_add_sync(0xffffffffu, above);
  ties = __reduce_add_sync(0xffffffffu, ties);
  __syncthreads();
  if (lane == 0) {
    sh.scan[warp] = above;
    sh.scan2[warp] = ties;
  }
  __syncthreads();
  uint32_t all = 0, all_ties = 0;
  above = ties = 0;
  for (int w = 0; w < kSelectWarps; ++w) {
    if (w < warp) {
      above += sh.scan[w];
      ties += sh.scan2[w];
    }
    all += sh.scan[w];
    all_ties += sh.scan2[w];
  }
  const cluster::u64* box = exchange(static_cast<cluster::u64>(all) << 32 | all_ties);
  for (int r = 0; r < rank; ++r) {
    above += static_cast<uint32_t>(box[r] >> 32);
    ties += static_cast<uint32_t>(box[r]);
  }
#pragma unroll 4
  for (int i0 = w0; i0 < w1; i0 += 32) {
    const int i = i0 + lane;
    const uint32_t k = i < w1 ? key(i) : 0;
    const uint32_t tie = __ballot_sync(0xffffffffu, i < w1 && k == prefix), over = __ballot_sync(0xffffffffu, i < w1 && k > prefix), below = (1u << lane) - 1;
    const uint32_t nth = ties + __popc(tie & below);
    if (i < w1 && (k > prefix || (k == prefix && nth < need))) out[above + __popc(over & below) + min(nth, need)] = base + i;
    above += __popc(over);
    ties += __popc(tie);
  }
  ptx::grid_dep_launch();
}

// A warp for `rows` kept slots of a head: a lane looks one of them up, then has a 16-byte piece of a row, kAhead rows at a time; the lanes of a
// row have its key's pieces and then its value's.  Many rows to a warp save lookups (16 x 4096 slots: 32 take 75 us, 16 take 85); few rows in all
// want more warps instead (2 x 2048 slots: 8 take 11 us, 32 take 15).  Bandwidth bounds many rows: 16 x 4096 slots of 8 heads of 128 (537 MB read
// and written) take 63 us (under the profiler 67); few rows the latency of three loads, each of which needs the one before.
constexpr int kAhead = 8;
__host__ __device__ constexpr int rows_at_once(int D) { return 32 / (D / 4); }
inline int least_rows(int D) { return kAhead * rows_at_once(D) < 32 ? kAhead * rows_at_once(D) : 32; }

__global__ void __launch_bounds__(kThreads) move_kernel(const __grid_constant__ cpmtp_cache c, const __grid_constant__ cpmtp_cache_seqs s,
                                                        const int* table_out, long long ld_table_out, int budget, int rows, const int* kept, int* dev_status) {
  const int lane = threadIdx.x & 31, h = blockIdx.y, b = blockIdx.z;
  const int j = (blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5)) * rows + lane;
  ptx::grid_dep_wait();
  const int slot = lane < rows && j < budget ? kept[(static_cast<long long>(b) * c.H + h) * budget + j] : -1;
  int src_page = -1, src_slot = 0, dst_page = -1, dst_slot = 0;
  if (slot >= 0) {
    src_page = page_of(s.table[b * s.ld_table + slot / c.page_slots], c.pages, dev_status);
    src_slot = slot % c.page_slots;
    dst_page = page_of(table_out[b * ld_table_out + j / c.page_slots], c.pages, dev_status);
    dst_slot = j % c.page_slots;
  }
  const bool both = src_page >= 0 && dst_page >= 0;
  float acc = 0.f;
  if (both) acc = c.acc[src_page * c.acc_page + h * c.acc_head + src_slot];
  const uint32_t some = __ballot_sync(0xffffffffu, both);
  const int pieces = c.D / 8, width = 2 * pieces, at_once = rows_at_once(c.D), sub = lane / width, piece = lane % width;
  const bool value = piece >= pieces;
  const int64_t page = value ? c.v_page : c.k_page, step = value ? c.v_slot : c.k_slot;
  bf16_t* data = value ? static_cast<bf16_t*>(c.v) + h * c.v_head + 8 * (piece - pieces) : static_cast<bf16_t*>(c.k) + h * c.k_head + 8 * piece;
  for (int r0 = 0; r0 < rows && (some >> r0) != 0; r0 += kAhead * at_once) {
    uint4 v[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int r = r0 + i * at_once + sub;
      const int64_t from = __shfl_sync(0xffffffffu, src_page, r & 31) * page + __shfl_sync(0xffffffffu, src_slot, r & 31) * step;
      if (sub < at_once && r < rows && (some >> r & 1)) v[i] = *reinterpret_cast<const uint4*>(data + from);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int r = r0 + i * at_once + sub;
      const int64_t to = __shfl_sync(0xffffffffu, dst_page, r & 31) * page + __shfl_sync(0xffffffffu, dst_slot, r & 31) * step;
      if (sub < at_once && r < rows && (some >> r & 1)) *reinterpret_cast<uint4*>(data + to) = v[i];
    }
  }
  if (both) c.acc[dst_page * c.acc_page + h * c.acc_head + dst_slot] = acc;
}

}  // namespace cache
}  // namespace cpmtp
