// Norms before and after a block, fused with its gate and the residual addition: forward and backward.
//
// A row is owned by W warps, eight columns to a thread, and stays in registers from its only read to its only write;
// a block holds G rows at a time (G = 1 from 2049 columns on).
#pragma once
#include "vec_io.cuh"

namespace cpmtp {
namespace norm {

using io::bf16_t;

constexpr int kMaxWarps = 32;

template <class T>
struct Rows {
  T* data;
  long long ld;
  __device__ __forceinline__ T* at(long long i) const { return data + i * ld; }
};

template <class S>
struct Params {
  int N, d;
  int W, G;          // warps per row, rows per block
  int gate_kind;
  float eps, res_scale, inv_d;
  Rows<const S> x;
  Rows<const bf16_t> block, gate;
  const bf16_t *w_post, *w_pre;
  Rows<S> x_out;
  Rows<bf16_t> y;
  float *rstd_post, *rstd_pre;
  Rows<const bf16_t> dy;
  Rows<const S> dx_out;
  Rows<S> dx;
  Rows<bf16_t> dblock, dgate;
  float* part;       // [blocks][2][d] sums of dw_post, dw_pre over the rows of a block; nullptr: not wanted
};

__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.f, 1.f + __expf(-z)); }

// Sums of NV values over the W warps of a row, in every thread of them.  `red` [NV][kMaxWarps] belongs to this row
// and to this reduction alone until the one after the next.
template <int NV>
__device__ __forceinline__ void row_sum(float (&v)[NV], float (*red)[kMaxWarps], int W, int group, int wg, int lane) {
#pragma unroll
  for (int n = 0; n < NV; ++n) v[n] = io::sum_lanes(v[n]);
  if (W == 1) return;
  if (lane == 0) {
#pragma unroll
    for (int n = 0; n < NV; ++n) red[n][wg] = v[n];
  }
  asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(W * 32) : "memory");
#pragma unroll
  for (int n = 0; n < NV; ++n) v[n] = io::sum_lanes(lane < W ? red[n][lane] : 0.f);
}

template <class S, bool VEC, int MAXT>
__global__ void __launch_bounds__(MAXT) norm_fwd_kernel(const __grid_constant__ Params<S> p) {
  __shared__ float red[2][MAXT > 512 ? 1 : 8][1][kMaxWarps];     // rows of more than one warp: at most 8 to a block
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int group = warp / p.W, wg = warp - group * p.W;
  const int t = wg * 32 + lane, tg = p.W * 32;
  const long long i = static_cast<long long>(blockIdx.x) * p.G + group;
  ptx::grid_dep_wait();
  if (i >= p.N) return;                          // a whole row's warps: no other row waits for them
  const int rg = p.W == 1 ? 0 : group;
  float x[8];
  io::load_cols<VEC>(p.x.at(i), t, tg, p.d, x);
  if (p.block.data != nullptr) {
    float b[8], g[8];
    io::load_cols<VEC>(p.block.at(i), t, tg, p.d, b);
    if (p.gate_kind == CPMTP_GATE_CHANNEL) {
      io::load_cols<VEC>(p.gate.at(i), t, tg, p.d, g);
#pragma unroll
      for (int k = 0; k < 8; ++k) g[k] = sigmoid(g[k]);
    } else {
      const float one = p.gate_kind == CPMTP_GATE_ROW ? sigmoid(io::to_f(*p.gate.at(i))) : 1.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) g[k] = one;
    }
    if (p.w_post != nullptr) {
      float w[8];
      io::load_cols<VEC>(p.w_post, t, tg, p.d, w);
      float ss[1] = {0.f};
#pragma unroll
      for (int k = 0; k < 8; ++k) ss[0] = fmaf(b[k], b[k], ss[0]);
      row_sum(ss, red[0][rg], p.W, group, wg, lane);
      const float rb = rsqrtf(fmaf(ss[0], p.inv_d, p.eps));
      if (t == 0 && p.rstd_post != nullptr) p.rstd_post[i] = rb;
#pragma unroll
      for (int k = 0; k < 8; ++k) b[k] *= rb * w[k];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = fmaf(p.res_scale, x[k], g[k] * b[k]);
    io::store_cols<VEC>(p.x_out.at(i), t, tg, p.d, x);
  }
  if (p.w_pre != nullptr) {
    float w[8];
    io::load_cols<VEC>(p.w_pre, t, tg, p.d, w);
    float ss[1] = {0.f};
#pragma unroll
    for (int k = 0; k < 8; ++k) ss[0] = fmaf(x[k], x[k], ss[0]);
    row_sum(ss, red[1][rg], p.W, group, wg, lane);
    const float rx = rsqrtf(fmaf(ss[0], p.inv_d, p.eps));
    if (t == 0 && p.rstd_pre != nullptr) p.rstd_pre[i] = rx;
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] *= rx * w[k];
    io::store_cols<VEC>(p.y.at(i), t, tg, p.d, x);
  }
}

// Backward.  Persistent blocks: a thread keeps its eight columns' sums of dw_post and dw_pre over all rows of its
// block.  The gradient t of x_out needs the row mean c1 = mean(w_pre dy xh); the norm after the block then needs the mean
// of w_post du bh, which holds t.  Both come out of one reduction over the row, since t = a - rstd_pre c1 xh with
// a = dx_out + rstd_pre w_pre dy is linear in c1:
//   sum q t = sum q a - rstd_pre c1 sum q xh,      q = g w_post bh.
// Rows ahead are fetched with cp.async, every thread the elements that it will itself use, so no barrier is spent on them.
constexpr int kStages = 2;

template <class S>
struct Slots {                                   // 16-byte slots per thread and stage: dy, block, gate, x_out, dx_out
  static constexpr int kS = sizeof(S) / 2;
  static constexpr int kDy = 0, kBlock = 1, kGate = 2, kX = 3, kDxOut = 3 + kS, kCount = 3 + 2 * kS;
};

__device__ __forceinline__ void cp16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void slot8(const uint8_t* s, int, float (&v)[8], bf16_t) {
  io::unpack8(*reinterpret_cast<const uint4*>(s), v);
}
__device__ __forceinline__ void slot8(const uint8_t* s, int stride, float (&v)[8], float) {
  const float4 a = *reinterpret_cast<const float4*>(s), b = *reinterpret_cast<const float4*>(s + stride);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

template <class S, bool VEC, int MAXT>
__global__ void __launch_bounds__(MAXT) norm_bwd_kernel(const __grid_constant__ Params<S> p) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float red[2][MAXT > 512 ? 1 : 8][3][kMaxWarps];
  using L = Slots<S>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int group = warp / p.W, wg = warp - group * p.W;
  const int t = wg * 32 + lane, tg = p.W * 32;
  const int rg = p.W == 1 ? 0 : group;
  const int stride = blockDim.x * 16;            // from one slot of a thread to its next
  const bool mine = 8 * t < p.d;
  const long long step = static_cast<long long>(gridDim.x) * p.G;
  const bool has_block = p.block.data != nullptr, has_post = has_block && p.w_post != nullptr;
  const bool channel = p.gate_kind == CPMTP_GATE_CHANNEL, row_gate = p.gate_kind == CPMTP_GATE_ROW;
  const bool has_y = p.dy.data != nullptr, has_dx_out = p.dx_out.data != nullptr;
  ptx::grid_dep_wait();

  auto fetch = [&](long long i, int stage) {
    if (VEC && i < p.N && mine) {
      const uint32_t s = ptx::smem_u32(smem) + stage * L::kCount * stride + threadIdx.x * 16;
      if (has_y) cp16(s + L::kDy * stride, p.dy.at(i) + 8 * t);
      if (has_block) cp16(s + L::kBlock * stride, p.block.at(i) + 8 * t);
      if (channel) cp16(s + L::kGate * stride, p.gate.at(i) + 8 * t);
#pragma unroll
      for (int k = 0; k < L::kS; ++k) {
        cp16(s + (L::kX + k) * stride, p.x_out.at(i) + 8 * t + 4 * k);
        if (has_dx_out) cp16(s + (L::kDxOut + k) * stride, p.dx_out.at(i) + 8 * t + 4 * k);
      }
    }
    if (VEC) asm volatile("cp.async.commit_group;" ::: "memory");
  };
  auto get = [&](auto rows, bool present, int slot, long long i, int stage, float (&v)[8]) {
    using T = std::remove_cv_t<std::remove_pointer_t<decltype(rows.data)>>;
    if (VEC ? (present && mine) : present) {
      if (VEC) {
        slot8(smem + (stage * L::kCount + slot) * stride + threadIdx.x * 16, stride, v, T());
      } else {
        io::load_cols<false>(rows.at(i), t, tg, p.d, v);
      }
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = 0.f;
    }
  };

  float w_pre[8], w_post[8], acc_pre[8], acc_post[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) w_pre[k] = w_post[k] = acc_pre[k] = acc_post[k] = 0.f;
  if (has_y) io::load_cols<VEC>(p.w_pre, t, tg, p.d, w_pre);
  if (has_post) io::load_cols<VEC>(p.w_post, t, tg, p.d, w_post);

  long long i = static_cast<long long>(blockIdx.x) * p.G + group;
  for (int s = 0; s < kStages - 1; ++s) fetch(i + s * step, s);
  float rx_next = 0.f, rb_next = 1.f, gl_next = 0.f;
  auto scalars = [&](long long row) {
    if (row >= p.N) return;
    if (has_y) rx_next = p.rstd_pre[row];
    if (has_post) rb_next = p.rstd_post[row];
    if (row_gate) gl_next = io::to_f(*p.gate.at(row));
  };
  scalars(i);
  for (int it = 0; i < p.N; i += step, ++it) {
    const float rx = rx_next, rb = rb_next;
    const float grow = row_gate ? sigmoid(gl_next) : 1.f;
    scalars(i + step);
    const int stage = it % kStages;
    fetch(i + (kStages - 1) * step, (it + kStages - 1) % kStages);
    if (VEC) asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
    float dy[8], xh[8], a[8], bh[8], g[8];
    get(p.dy, has_y, L::kDy, i, stage, dy);
    get(p.x_out, true, L::kX, i, stage, xh);
    get(p.dx_out, has_dx_out, L::kDxOut, i, stage, a);
    get(p.block, has_block, L::kBlock, i, stage, bh);
    get(p.gate, channel, L::kGate, i, stage, g);
    float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      xh[k] *= rx;
      bh[k] *= rb;
      g[k] = channel ? sigmoid(g[k]) : 1.f;
      const float wdy = w_pre[k] * dy[k];
      a[k] = fmaf(rx, wdy, a[k]);
      const float q = (has_post ? w_post[k] * bh[k] : bh[k]) * g[k];
      s[0] = fmaf(wdy, xh[k], s[0]);
      s[1] = fmaf(q, a[k], s[1]);
      s[2] = fmaf(q, xh[k], s[2]);
      acc_pre[k] = fmaf(dy[k], xh[k], acc_pre[k]);
    }
    row_sum(s, red[it & 1][rg], p.W, group, wg, lane);
    const float c1 = rx * s[0] * p.inv_d;
    const float dot = s[1] - c1 * s[2];
    const float c2 = grow * dot * p.inv_d;
    float dgate[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float tk = fmaf(-c1, xh[k], a[k]);
      const float du = grow * g[k] * tk;
      const float u = has_post ? w_post[k] * bh[k] : bh[k];
      dgate[k] = tk * u * g[k] * (1.f - g[k]);
      acc_post[k] = fmaf(du, bh[k], acc_post[k]);
      xh[k] = p.res_scale * tk;                                               // dx
      a[k] = has_post ? rb * fmaf(w_post[k], du, -bh[k] * c2) : du;           // dblock
    }
    if (p.dx.data != nullptr) io::store_cols<VEC>(p.dx.at(i), t, tg, p.d, xh);
    if (p.dblock.data != nullptr) io::store_cols<VEC>(p.dblock.at(i), t, tg, p.d, a);
    if (p.dgate.data != nullptr) {
      if (channel) io::store_cols<VEC>(p.dgate.at(i), t, tg, p.d, dgate);
      else if (t == 0) *p.dgate.at(i) = io::from_f<bf16_t>(grow * (1.f - grow) * dot);
    }
  }
  if (p.part == nullptr) return;
  float* out = p.part + static_cast<size_t>(blockIdx.x) * 2 * p.d;
  if (p.G == 1) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int c = io::col_of<VEC>(t, tg, k);
      if (c < p.d) {
        out[c] = acc_post[k];
        out[p.d + c] = acc_pre[k];
      }
    }
    return;
  }
  // the rows that the block held at a time, one after the other
  if (VEC) asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();
  float* sums = reinterpret_cast<float*>(smem);                 // [2][G][8 tg]
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int c = io::col_of<VEC>(t, tg, k);
    sums[group * 8 * tg + c] = acc_post[k];
    sums[(p.G + group) * 8 * tg + c] = acc_pre[k];
  }
  __syncthreads();
  for (int c = threadIdx.x; c < 2 * p.d; c += blockDim.x) {
    const int which = c >= p.d, col = c - which * p.d;
    float v = 0.f;
    for (int gr = 0; gr < p.G; ++gr) v += sums[(which * p.G + gr) * 8 * tg + col];
    out[c] = v;
  }
}

// dw[c] = sum over blocks of part[block][which][c]; a block of this kernel has 32 columns of one of the two sums.
__global__ void __launch_bounds__(1024) norm_dw_kernel(const float* __restrict__ part, int blocks, int d, bf16_t* dw_post, bf16_t* dw_pre,
                                                       int accum) {
  __shared__ float s[32][33];
  ptx::grid_dep_wait();
  const int which = blockIdx.y, lane = threadIdx.x & 31, r = threadIdx.x >> 5;
  bf16_t* out = which ? dw_pre : dw_post;
  if (out == nullptr) return;
  const int c = blockIdx.x * 32 + lane;
  float v = 0.f;
  if (c < d)
    for (int b = r; b < blocks; b += 32) v += part[(static_cast<size_t>(b) * 2 + which) * d + c];
  s[r][lane] = v;
  __syncthreads();
  v = io::sum_lanes(s[lane][r]);                 // warp r: column r
  const int col = blockIdx.x * 32 + r;
  if (lane == 0 && col < d) out[col] = io::from_f<bf16_t>(accum ? io::to_f(out[col]) + v : v);
}

}  // namespace norm
}  // namespace cpmtp
