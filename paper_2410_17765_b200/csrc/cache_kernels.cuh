// Paged cache of keys and values: appending, and eviction by accumulated attention weight.
#pragma once
#include <cstdint>

#include "../../include/cpmtp.h"
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

// One thread for each piece of eight elements of a new token's key and value in one head.
template <bool VEC>
__global__ void __launch_bounds__(kThreads) append_kernel(const __grid_constant__ cpmtp_cache c, const __grid_constant__ cpmtp_cache_seqs s,
                                                          const __grid_constant__ cpmtp_tokens k, const __grid_constant__ cpmtp_tokens v,
                                                          int* dev_status) {
  ptx::grid_dep_wait();
  const int pieces = c.D / 8;
  const long long items = static_cast<long long>(s.B) * s.Q * c.H * pieces;
  for (long long i = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x; i < items; i += static_cast<long long>(gridDim.x) * kThreads) {
    const int piece = static_cast<int>(i % pieces);
    long long r = i / pieces;
    const int h = static_cast<int>(r % c.H);
    r /= c.H;
    const int j = static_cast<int>(r % s.Q), b = static_cast<int>(r / s.Q);
    const int fresh = seq_new(s, b, dev_status);
    if (j >= fresh) continue;
    const int len = seq_len(c, s, b, dev_status), slot = len - fresh + j;
    if (slot < 0) {
      raise_status(dev_status, kBadIndex);
      continue;
    }
    const int page = page_of(s.table[b * s.ld_table + slot / c.page_slots], c.pages, dev_status);
    if (page < 0) continue;
    const int at = slot % c.page_slots, col = 8 * piece;
    const bf16_t* kp = static_cast<const bf16_t*>(k.data) + b * k.seq + j * k.token + h * k.head + col;
    const bf16_t* vp = static_cast<const bf16_t*>(v.data) + b * v.seq + j * v.token + h * v.head + col;
    bf16_t* ko = static_cast<bf16_t*>(c.k) + page * c.k_page + at * c.k_slot + h * c.k_head + col;
    bf16_t* vo = static_cast<bf16_t*>(c.v) + page * c.v_page + at * c.v_slot + h * c.v_head + col;
    if (VEC) {
      const uint4 a = *reinterpret_cast<const uint4*>(kp), d = *reinterpret_cast<const uint4*>(vp);
      *reinterpret_cast<uint4*>(ko) = a;
      *reinterpret_cast<uint4*>(vo) = d;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        ko[e] = kp[e];
        vo[e] = vp[e];
      }
    }
    if (piece == 0 && c.acc != nullptr) c.acc[page * c.acc_page + h * c.acc_head + at] = 0.f;
  }
}

// ---------------------------------------------------------------------------------------------- eviction

constexpr int kSelectThreads = 1024;

// The order in which slots are kept: the last `recent` ones before all others, then by accumulated weight.
__device__ __forceinline__ uint32_t keep_key(float acc) {
  if (acc != acc) return 0;                                    // NaN: the least
  const uint32_t u = __float_as_uint(acc + 0.f);               // (-0 as +0)
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ uint32_t slot_key(const cpmtp_cache& c, const int* row, int h, int slot, int recent_from, int* dev_status) {
  if (slot >= recent_from) return 0xffffffffu;
  const int page = page_of(row[slot / c.page_slots], c.pages, dev_status);
  return page < 0 ? 0 : keep_key(c.acc[page * c.acc_page + h * c.acc_head + slot % c.page_slots]);
}

// One block for each head of each sequence: the key of the last slot to be kept by four passes over eight bits each, then the kept slots in their
// order.  kept [B, H, budget].
__global__ void __launch_bounds__(kSelectThreads) select_kernel(const __grid_constant__ cpmtp_cache c, const __grid_constant__ cpmtp_cache_seqs s,
                                                                int budget, int recent, int* lens_out, int* kept, int* dev_status) {
  __shared__ int hist[256];
  __shared__ uint32_t sh_prefix;
  __shared__ int sh_need, warp_sums[32], warp_ties[32];
  ptx::grid_dep_wait();
  const int h = blockIdx.x, b = blockIdx.y, t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int len = seq_len(c, s, b, dev_status);
  const int* row = s.table + b * s.ld_table;
  int* out = kept + (static_cast<long long>(b) * c.H + h) * budget;
  if (h == 0 && t == 0) lens_out[b] = min(len, budget);
  if (len <= budget) {
    for (int i = t; i < budget; i += kSelectThreads) out[i] = i < len ? i : -1;
    return;
  }
  const int from = len - recent;
  uint32_t prefix = 0, mask = 0;
  int need = budget;                             // how many of the keys with this prefix are kept, the largest first
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (t < 256) hist[t] = 0;
    __syncthreads();
    for (int i = t; i < len; i += kSelectThreads) {
      const uint32_t key = slot_key(c, row, h, i, from, dev_status);
      if ((key & mask) == prefix) atomicAdd(&hist[(key >> shift) & 255], 1);
    }
    __syncthreads();
    if (t == 0) {
      int left = need, d = 255;
      while (d > 0 && hist[d] < left) left -= hist[d--];
      sh_prefix = prefix | (static_cast<uint32_t>(d) << shift);
      sh_need = left;
    }
    __syncthreads();
    prefix = sh_prefix;
    need = sh_need;
    mask |= 255u << shift;
  }
  // keys above `prefix`, and the first `need` equal to it
  int done = 0, ties = 0;
  for (int base = 0; base < len; base += kSelectThreads) {
    const int i = base + t;
    const uint32_t key = i < len ? slot_key(c, row, h, i, from, dev_status) : 0;
    const bool tie = i < len && key == prefix;
    const uint32_t tie_lanes = __ballot_sync(0xffffffffu, tie);
    if (lane == 0) warp_ties[warp] = __popc(tie_lanes);
    __syncthreads();
    int rank = ties + __popc(tie_lanes & ((1u << lane) - 1));
    for (int w = 0; w < 32; ++w) {
      if (w < warp) rank += warp_ties[w];
      ties += warp_ties[w];
    }
    const bool keep = i < len && (key > prefix || (tie && rank < need));
    const uint32_t lanes = __ballot_sync(0xffffffffu, keep);
    if (lane == 0) warp_sums[warp] = __popc(lanes);
    __syncthreads();
    int at = done + __popc(lanes & ((1u << lane) - 1));
    for (int w = 0; w < 32; ++w) {
      if (w < warp) at += warp_sums[w];
      done += warp_sums[w];
    }
    if (keep) out[at] = i;
    __syncthreads();
  }
}

// One thread for each piece of eight elements of a kept key and value.
__global__ void __launch_bounds__(kThreads) move_kernel(const __grid_constant__ cpmtp_cache c, const __grid_constant__ cpmtp_cache_seqs s,
                                                        const int* table_out, long long ld_table_out, int budget, const int* kept, int* dev_status) {
  ptx::grid_dep_wait();
  const int pieces = c.D / 8;
  const long long items = static_cast<long long>(s.B) * c.H * budget * pieces;
  for (long long i = static_cast<long long>(blockIdx.x) * kThreads + threadIdx.x; i < items; i += static_cast<long long>(gridDim.x) * kThreads) {
    const int piece = static_cast<int>(i % pieces);
    const long long r = i / pieces;
    const int j = static_cast<int>(r % budget), h = static_cast<int>(r / budget % c.H), b = static_cast<int>(r / budget / c.H);
    const int slot = kept[r];
    if (slot < 0) continue;
    const int from = page_of(s.table[b * s.ld_table + slot / c.page_slots], c.pages, dev_status);
    const int to = page_of(table_out[b * ld_table_out + j / c.page_slots], c.pages, dev_status);
    if (from < 0 || to < 0) continue;
    const int at = slot % c.page_slots, in = j % c.page_slots;
    bf16_t *k = static_cast<bf16_t*>(c.k) + h * c.k_head + 8 * piece, *v = static_cast<bf16_t*>(c.v) + h * c.v_head + 8 * piece;
    const uint4 a = *reinterpret_cast<const uint4*>(k + from * c.k_page + at * c.k_slot);
    const uint4 d = *reinterpret_cast<const uint4*>(v + from * c.v_page + at * c.v_slot);
    *reinterpret_cast<uint4*>(k + to * c.k_page + in * c.k_slot) = a;
    *reinterpret_cast<uint4*>(v + to * c.v_page + in * c.v_slot) = d;
    if (piece == 0) c.acc[to * c.acc_page + h * c.acc_head + in] = c.acc[from * c.acc_page + h * c.acc_head + at];
  }
}

}  // namespace cache
}  // namespace cpmtp
