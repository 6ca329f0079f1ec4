// Sampling from logits with temperature, top-k, top-p and min-p by given uniform numbers.
#pragma once
#include <cstdint>

#include "../../include/cpmtp.h"
#include "ptx.cuh"
#include "vec_io.cuh"

namespace cpmtp {
namespace sample {

using io::bf16_t;
typedef unsigned long long u64;
constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;

struct Row {
  double inv_t, top_p, min_p;
  int top_k;
  bool greedy;
};
__device__ __forceinline__ Row row_settings(const cpmtp_sample_args& a, int i) {
  Row r;
  const float t = a.temperatures != nullptr ? a.temperatures[i] : a.temperature;
  r.greedy = !(t > 0.f);
  r.inv_t = r.greedy ? 1.0 : 1.0 / static_cast<double>(t);
  const float p = a.top_ps != nullptr ? a.top_ps[i] : a.top_p, mp = a.min_ps != nullptr ? a.min_ps[i] : a.min_p;
  r.top_p = p < 1.f ? static_cast<double>(p) : 1.0;
  r.min_p = mp > 0.f ? static_cast<double>(mp) : 0.0;
  const int k = a.top_ks != nullptr ? a.top_ks[i] : a.top_k;
  r.top_k = k > 0 && k < a.V ? k : a.V;
  if (r.greedy || r.min_p > 1.0) r.top_k = 1;
  return r;
}

// Unsigned keys in the order of the logits; 0: an entry that is never kept (-infinity, NaN).
__device__ __forceinline__ uint32_t logit_key(float x) {
  if (!(x > -INFINITY)) return 0;
  const uint32_t u = __float_as_uint(x + 0.f);     // (-0 as +0)
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_logit(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k); }

// exp((x - m) / T), and as an integer
__device__ __forceinline__ double z_of(float x, float m, double inv_t) { return x == m ? 0.0 : (static_cast<double>(x) - static_cast<double>(m)) * inv_t; }
__device__ __forceinline__ u64 fixed(double w, double unit) { return static_cast<u64>(w * unit); }

template <class Op>
__device__ __forceinline__ u64 block_all(u64 v, u64* sh, Op op) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  u64 r = sh[0];
  for (int w = 1; w < kWarps; ++w) r = op(r, sh[w]);
  return r;
}
__device__ __forceinline__ u64 block_sum(u64 v, u64* sh) { return block_all(v, sh, [](u64 a, u64 b) { return a + b; }); }

// One block to a row, several passes over it.
template <class T>
__global__ void __launch_bounds__(kThreads) sample_kernel(const __grid_constant__ cpmtp_sample_args a, double unit, int* dev_status) {
  __shared__ u64 sh[kWarps];
  __shared__ u64 mass[256];
  __shared__ int count[256];
  __shared__ uint32_t sh_key;
  __shared__ int sh_need, sh_token, sh_ties[kWarps];
  __shared__ u64 sh_above;
  ptx::grid_dep_wait();
  const int i = blockIdx.x, t = threadIdx.x, lane = t & 31, warp = t >> 5, V = a.V;
  const T* x = static_cast<const T*>(a.logits) + i * a.ld;
  const Row r = row_settings(a, i);
  auto key = [&](int v) { return logit_key(io::to_f(x[v])); };

  uint32_t top = 0;
  for (int v = t; v < V; v += kThreads) top = max(top, key(v));
  top = static_cast<uint32_t>(block_all(top, sh, [](u64 p, u64 q) { return p > q ? p : q; }));
  const int given = a.given != nullptr ? a.given[i] : CPMTP_EMBED_PAD;
  if (t == 0 && given != CPMTP_EMBED_PAD && (given < 0 || given >= V) && dev_status != nullptr) atomicMax(dev_status, 1);
  if (top == 0) {
    if (t == 0) {
      a.tokens[i] = -1;
      if (a.logp != nullptr) a.logp[i] = -INFINITY;
      if (a.kept != nullptr) a.kept[i] = 0;
      if (a.given != nullptr) a.logp_given[i] = -INFINITY;
    }
    return;
  }
  const float m = key_logit(top);
  auto weight = [&](uint32_t k) { return exp(z_of(key_logit(k), m, r.inv_t)); };

  // The key of the last entry that a filter keeps, and how many of the entries with that key: by their number (what = 0) or their mass (1).
  uint32_t floor_key = 0;
  int floor_need = 0;                      // entries with key floor_key that are kept
  u64 total = 0;                           // mass of the entries kept so far
  auto find = [&](bool by_mass, u64 want, uint32_t low, int low_need) {
    uint32_t prefix = 0, mask = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (t < 256) {
        mass[t] = 0;
        count[t] = 0;
      }
      __syncthreads();
      for (int v = t; v < V; v += kThreads) {
        const uint32_t k = key(v);
        if (k == 0 || k < low || (k & mask) != prefix) continue;
        atomicAdd(&count[(k >> shift) & 255], 1);
        if (by_mass && k > low) atomicAdd(&mass[(k >> shift) & 255], fixed(weight(k), unit));
      }
      __syncthreads();
      if (by_mass && t == 0 && low > 0 && (low & mask) == prefix) mass[(low >> shift) & 255] += low_need * fixed(weight(low), unit);
      __syncthreads();
      if (t == 0) {
        int d = 255;
        u64 left = want;
        while (d > 0 && (by_mass ? mass[d] : static_cast<u64>(count[d])) < left) left -= by_mass ? mass[d--] : static_cast<u64>(count[d--]);
        sh_key = prefix | (static_cast<uint32_t>(d) << shift);
        sh_above = left;
        sh_need = count[d];
      }
      __syncthreads();
      prefix = sh_key;
      want = sh_above;
      mask |= 255u << shift;
    }
    floor_key = prefix;
    // `want` of the entries' number or mass is still missing, and they are all equal
    if (!by_mass) {
      floor_need = static_cast<int>(want);
    } else {
      const u64 w = fixed(weight(prefix), unit);
      const int most = prefix == low ? low_need : sh_need;     // (a prefix is never 0)
      const u64 n = w > 0 ? (want + w - 1) / w : 1;
      floor_need = n < 1 ? 1 : n > static_cast<u64>(most) ? most : static_cast<int>(n);
    }
    __syncthreads();
  };
  u64 n = 0;
  for (int v = t; v < V; v += kThreads) n += key(v) > 0;
  n = block_sum(n, sh);
  if (static_cast<u64>(r.top_k) < n) find(false, r.top_k, 0, 0);
  if (r.top_p < 1.0 && !r.greedy) {
    u64 sum = 0;
    for (int v = t; v < V; v += kThreads) {
      const uint32_t k = key(v);
      if (k > floor_key) sum += fixed(weight(k), unit);
    }
    sum = block_sum(sum, sh);
    if (floor_key > 0) sum += floor_need * fixed(weight(floor_key), unit);
    const double w = r.top_p * static_cast<double>(sum);
    u64 want = w > 0.0 ? static_cast<u64>(ceil(w)) : 1;
    if (want < 1) want = 1;
    find(true, want, floor_key, floor_need);
  }
  // min_p: a border between weights, so between keys
  auto passes = [&](uint32_t k) { return k == top || weight(k) >= r.min_p; };

  // Kept entries by index: each warp has a range of its own.
  const int span = (V + kWarps - 1) / kWarps, begin = min(warp * span, V), end = min(begin + span, V);
  int ties = 0;
  for (int v = begin + lane; v < end; v += 32) ties += key(v) == floor_key;
  ties = __reduce_add_sync(0xffffffffu, ties);
  if (lane == 0) sh_ties[warp] = ties;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < warp; ++w) before += sh_ties[w];
  u64 sum = 0;
  int kept = 0, last = -1, seen = before;
  bool given_kept = false;
  for (int base = begin; base < end; base += 32) {
    const int v = base + lane;
    const uint32_t k = v < end ? key(v) : 0;
    const uint32_t same = __ballot_sync(0xffffffffu, k == floor_key);
    const int rank = seen + __popc(same & ((1u << lane) - 1));
    seen += __popc(same);
    if (k != 0 && (k > floor_key || (k == floor_key && rank < floor_need)) && passes(k)) {
      const u64 w = fixed(weight(k), unit);
      sum += w;
      ++kept;
      if (w > 0) last = v;
      given_kept |= v == given;
    }
  }
  const u64 mine = [&] {
    u64 q = sum;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) q += __shfl_xor_sync(0xffffffffu, q, o);
    return q;
  }();
  total = block_sum(sum, sh);             // leaves the warps' sums in sh
  const int all_kept = static_cast<int>(block_sum(kept, mass));
  const int last_token = static_cast<int>(block_all(static_cast<u64>(last + 1), mass, [](u64 p, u64 q) { return p > q ? p : q; })) - 1;
  const bool any_given = __syncthreads_or(given_kept);
  const float u = a.uniform[i];
  const u64 target = u > 0.f ? (u < 1.f ? static_cast<u64>(static_cast<double>(u) * static_cast<double>(total)) : total) : 0;
  u64 low = 0;
  for (int w = 0; w < warp; ++w) low += sh[w];
  if (t == 0) sh_token = last_token;
  __syncthreads();
  if (low <= target && target < low + mine) {
    // this warp's range holds the token
    int at = before;
    for (int base = begin; base < end; base += 32) {
      const int v = base + lane;
      const uint32_t k = v < end ? key(v) : 0;
      const uint32_t same = __ballot_sync(0xffffffffu, k == floor_key);
      const int rank = at + __popc(same & ((1u << lane) - 1));
      at += __popc(same);
      u64 w = 0;
      if (k != 0 && (k > floor_key || (k == floor_key && rank < floor_need)) && passes(k)) w = fixed(weight(k), unit);
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const u64 q = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += q;
      }
      const uint32_t over = __ballot_sync(0xffffffffu, low + w > target);
      if (over != 0) {
        if (lane == 0) sh_token = base + __ffs(over) - 1;
        break;
      }
      low += __shfl_sync(0xffffffffu, w, 31);
    }
  }
  __syncthreads();
  if (t == 0) {
    const double log_total = log(static_cast<double>(total) / unit);
    a.tokens[i] = sh_token;
    if (a.logp != nullptr) a.logp[i] = static_cast<float>(z_of(key_logit(key(sh_token)), m, r.inv_t) - log_total);
    if (a.kept != nullptr) a.kept[i] = all_kept;
    if (a.given != nullptr) a.logp_given[i] = any_given ? static_cast<float>(z_of(key_logit(key(given)), m, r.inv_t) - log_total) : -INFINITY;
  }
}

}  // namespace sample
}  // namespace cpmtp
