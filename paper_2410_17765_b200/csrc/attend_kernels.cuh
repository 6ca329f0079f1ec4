// Attention of a few new tokens over the paged cache.
#pragma once
#include "cache_kernels.cuh"

namespace cpmtp {
namespace attend {

using io::bf16_t;
constexpr int kThreads = 128;
constexpr float kLog2e = 1.4426950408889634f;

// One block for each new token and query head; a warp takes every fourth slot, a lane up to four columns.
__global__ void __launch_bounds__(kThreads) attend_kernel(const __grid_constant__ cpmtp_cache c, const __grid_constant__ cpmtp_cache_seqs s,
                                                          const __grid_constant__ cpmtp_attend_args a, float* lse_all, int* dev_status) {
  __shared__ float sh_m[4], sh_l[4], sh_o[4][128];
  ptx::grid_dep_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int hq = blockIdx.x % a.Hq, j = blockIdx.x / a.Hq, b = blockIdx.y;
  const int h = hq / (a.Hq / c.H);
  const int fresh = cache::seq_new(s, b, dev_status);
  if (j >= fresh) return;
  const int last = cache::seq_len(c, s, b, dev_status) - (fresh - 1 - j);
  const int* row = s.table + b * s.ld_table;
  const bf16_t* qp = static_cast<const bf16_t*>(a.q.data) + b * a.q.seq + j * a.q.token + hq * a.q.head;
  float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
  for (int e = 0; e < 4; ++e) q[e] = lane + 32 * e < c.D ? io::to_f(qp[lane + 32 * e]) * a.scale : 0.f;
  for (int i = warp; i < last; i += 4) {
    const int page = cache::page_of(row[i / c.page_slots], c.pages, dev_status);
    const int at = i % c.page_slots;
    float x = 0.f, vals[4] = {0.f, 0.f, 0.f, 0.f};
    if (page >= 0) {
      const bf16_t* kp = static_cast<const bf16_t*>(c.k) + page * c.k_page + at * c.k_slot + h * c.k_head;
      const bf16_t* vp = static_cast<const bf16_t*>(c.v) + page * c.v_page + at * c.v_slot + h * c.v_head;
      for (int e = 0; e < 4; ++e)
        if (lane + 32 * e < c.D) {
          x += q[e] * io::to_f(kp[lane + 32 * e]);
          vals[e] = io::to_f(vp[lane + 32 * e]);
        }
    }
    x = io::sum_lanes(x);
    const float top = fmaxf(m, x), keep = exp2f((m - top) * kLog2e), p = exp2f((x - top) * kLog2e);
    m = top;
    l = l * keep + p;
    for (int e = 0; e < 4; ++e) o[e] = o[e] * keep + p * vals[e];
  }
  if (lane == 0) {
    sh_m[warp] = m;
    sh_l[warp] = l;
  }
  for (int e = 0; e < 4; ++e) sh_o[warp][lane + 32 * e] = o[e];
  __syncthreads();
  float top = -INFINITY, sum = 0.f, out = 0.f;
  for (int w = 0; w < 4; ++w) top = fmaxf(top, sh_m[w]);
  if (top > -INFINITY)
    for (int w = 0; w < 4; ++w) {
      const float f = exp2f((sh_m[w] - top) * kLog2e);
      sum += sh_l[w] * f;
      out += sh_o[w][threadIdx.x] * f;
    }
  const float lse = sum > 0.f ? top + logf(sum) : -INFINITY;
  const long long r = (static_cast<long long>(b) * s.Q + j) * a.Hq + hq;
  if (threadIdx.x < c.D)
    (static_cast<bf16_t*>(a.out.data) + b * a.out.seq + j * a.out.token + hq * a.out.head)[threadIdx.x] = io::from_f<bf16_t>(sum > 0.f ? out / sum : 0.f);
  if (threadIdx.x == 0) {
    if (a.lse != nullptr) a.lse[r] = lse;
    if (lse_all != nullptr) lse_all[r] = lse;
  }
}

// One thread for each slot of a head: the weights of all rows that see it.
__global__ void __launch_bounds__(kThreads) weight_kernel(const __grid_constant__ cpmtp_cache c, const __grid_constant__ cpmtp_cache_seqs s,
                                                          const __grid_constant__ cpmtp_attend_args a, const float* lse_all, int* dev_status) {
  ptx::grid_dep_wait();
  const int slot = blockIdx.x * kThreads + threadIdx.x, h = blockIdx.y, b = blockIdx.z, G = a.Hq / c.H;
  const int fresh = cache::seq_new(s, b, dev_status), len = cache::seq_len(c, s, b, dev_status);
  if (slot >= len) return;
  const int page = cache::page_of(s.table[b * s.ld_table + slot / c.page_slots], c.pages, dev_status);
  if (page < 0) return;
  const int at = slot % c.page_slots;
  const bf16_t* kp = static_cast<const bf16_t*>(c.k) + page * c.k_page + at * c.k_slot + h * c.k_head;
  float w = 0.f;
  for (int j = 0; j < fresh; ++j) {
    if (slot >= len - (fresh - 1 - j)) continue;
    for (int g = 0; g < G; ++g) {
      const bf16_t* qp = static_cast<const bf16_t*>(a.q.data) + b * a.q.seq + j * a.q.token + (h * G + g) * a.q.head;
      float x = 0.f;
      for (int e = 0; e < c.D; ++e) x += io::to_f(qp[e]) * io::to_f(kp[e]);
      w += exp2f((x * a.scale - lse_all[(static_cast<long long>(b) * s.Q + j) * a.Hq + h * G + g]) * kLog2e);
    }
  }
  float* acc = c.acc + page * c.acc_page + h * c.acc_head + at;
  *acc += w;
}

}  // namespace attend
}  // namespace cpmtp
