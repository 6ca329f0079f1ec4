// Norms before and after a block, fused with its gate and the residual addition: forward and backward.
//
// A row is owned by W warps, eight columns to a thread, and stays in registers from its only read to its only write; a
// block holds G rows at a time (W G <= 16, or G = 1).  Blocks are persistent.  Both directions move
// 10 to 20 bytes per element and compute some tens of operations on them, so what counts is that every SM always has tens of
// kilobytes of reads under way: rows ahead are fetched with cp.async into a ring of rows in shared memory while the
// current row goes through its reductions.  8192 x 4096, bf16, a gate per channel: forward 59 us (5.7 TB/s), backward 99 us
// with the sums of the weights' gradients (5.4 TB/s); a plain copy on this card reaches 6.5 TB/s.
#pragma once
#include <type_traits>

#include "vec_io.cuh"

namespace cpmtp {
namespace norm {

using io::add2;
using io::bf16_t;
using io::both;
using io::f32x2;
using io::fma2;
using io::mul2;

constexpr int kMaxWarps = 32;

template <class T>
struct Rows {
  T* data;
  long long ld;
  __device__ __forceinline__ T* at(unsigned i) const { return data + i * static_cast<unsigned long long>(ld); }
  // where in its 16-byte piece row i starts: the low bits of the address alone
  __device__ __forceinline__ int offset(unsigned i) const {
    return (static_cast<unsigned>(reinterpret_cast<uintptr_t>(data)) + i * static_cast<unsigned>(ld) * static_cast<unsigned>(sizeof(T))) & 15;
  }
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

// 1 / (1 + 2^(-z log2 e)); the flush of results below 2^-126 keeps both steps single instructions
__device__ __forceinline__ float rcp(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float exp_minus(float z) { return ptx::ex2_approx(z * -1.4426950408889634f); }
__device__ __forceinline__ f32x2 exp_minus2(f32x2 z) {
  const f32x2 e = mul2(z, both(-1.4426950408889634f));
  return io::pair(ptx::ex2_approx(io::lo(e)), ptx::ex2_approx(io::hi(e)));
}
// the gate from e = exp(-z)
__device__ __forceinline__ float gate_of(float e) { return rcp(1.f + e); }
__device__ __forceinline__ f32x2 gate_of2(f32x2 e) {
  const f32x2 s = add2(e, both(1.f));
  return io::pair(rcp(io::lo(s)), rcp(io::hi(s)));
}
// What an open gate leaves, 1 - g, as e g: the difference has no digit left at a logit of 17.  Where e is infinite and g zero, or
// both are NaN, saturation makes the product zero; g, which everything it is multiplied with holds, says the rest.
__device__ __forceinline__ float rest_of(float e, float g) { return __saturatef(e * g); }
__device__ __forceinline__ f32x2 rest_of2(f32x2 e, f32x2 g) {
  return io::pair(rest_of(io::lo(e), io::lo(g)), rest_of(io::hi(e), io::hi(g)));
}

// Barrier of the W warps of a row.  It counts warps, so a warp's lanes come together first.
// MANY: known to be more than one.
template <bool MANY>
__device__ __forceinline__ void row_barrier(int W, int group) {
  __syncwarp();
  if (MANY || W > 1) asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(W * 32) : "memory");
}
// What crosses that barrier is written and read in assembly, so that the order of the three is the written one.
__device__ __forceinline__ void put_shared(float* p, float v) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(ptx::smem_u32(p)), "f"(v) : "memory"); }
__device__ __forceinline__ float get_shared(const float* p) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(ptx::smem_u32(p)) : "memory");
  return v;
}

// Sums over the W warps of a row, in every thread of them, in two steps: what comes between them does not wait for the other
// warps.  `red` is this row's and this reduction's alone until the row after the next.  Two values at once take 11 shuffles
// where two single sums take 20: half of the lanes finish the one, half the other.  No lane branches: all lanes of a half write
// the sum that they share, and all read.  (Written under (lane & 15) == 0, red[lane >> 4] also cost correctness: the compiler
// took that lane >> 4 for exact and used it for the reads, where it is not.)
__device__ __forceinline__ float half_sum(float c) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
  return c;
}
template <bool MANY>
__device__ __forceinline__ float begin_sum2(const float (&v)[2], float (*red)[kMaxWarps], int W, int wg, int lane) {
  const bool hi = lane & 16;
  float c = hi ? v[1] : v[0];
  c += __shfl_xor_sync(0xffffffffu, hi ? v[0] : v[1], 16);
  c = half_sum(c);
  if (MANY || W > 1) put_shared(&red[lane >> 4][wg], c);   // (the lanes of a half have the same sum, and no branch is taken)
  return c;
}
template <bool MANY>
__device__ __forceinline__ void end_sum2(float (&v)[2], float c, float (*red)[kMaxWarps], int W, int group, int lane) {
  if (MANY || W > 1) {
    row_barrier<MANY>(W, group);
    const int j = lane & 15;
    const float* mine = red[lane >> 4];
    c = 0.f;
#pragma unroll
    for (int k = 0; k < kMaxWarps; k += 16) {
      if (k >= W) break;                     // (every lane reads; what lies past W does not count)
      const float x = get_shared(mine + j + k);
      c += j + k < W ? x : 0.f;
    }
    c = half_sum(c);
  }
#pragma unroll
  for (int n = 0; n < 2; ++n) v[n] = __shfl_sync(0xffffffffu, c, 16 * n);
}

// Three values in 12 shuffles: lanes hand over the values that the other half will finish, so that each octet of lanes ends up
// with the sum of one of them (the last one with that of zeros).
__device__ __forceinline__ float octet_sum(float c) {
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
  return c;
}
template <bool MANY>
__device__ __forceinline__ float begin_sum3(const float (&v)[3], float (*red)[kMaxWarps], int W, int wg, int lane) {
  const bool hi = lane & 16, odd = lane & 8;
  float a = hi ? v[2] : v[0], b = hi ? 0.f : v[1];
  a += __shfl_xor_sync(0xffffffffu, hi ? v[0] : v[2], 16);
  b += __shfl_xor_sync(0xffffffffu, hi ? v[1] : 0.f, 16);
  float c = odd ? b : a;
  c += __shfl_xor_sync(0xffffffffu, odd ? a : b, 8);
  c = octet_sum(c);
  if (MANY || W > 1) put_shared(&red[lane >> 3][wg], c);
  return c;
}
template <bool MANY>
__device__ __forceinline__ void end_sum3(float (&v)[3], float c, float (*red)[kMaxWarps], int W, int group, int lane) {
  if (MANY || W > 1) {
    row_barrier<MANY>(W, group);
    const int j = lane & 7;
    const float* mine = red[lane >> 3];
    c = 0.f;
#pragma unroll
    for (int k = 0; k < kMaxWarps; k += 8) {
      if (k >= W) break;                      // (every lane reads; what lies past W does not count)
      const float x = get_shared(mine + j + k);
      c += j + k < W ? x : 0.f;
    }
    c = octet_sum(c);
  }
#pragma unroll
  for (int n = 0; n < 3; ++n) v[n] = __shfl_sync(0xffffffffu, c, 8 * n);
}

// ---- rows in shared memory ----
// A row of d elements of T, wherever it starts, lies in at most d sizeof(T) / 16 + 1 aligned pieces of 16 bytes, and it is
// these that are copied (the last one only as far as the row goes), so that rows of any width and stride move in whole
// 16-byte accesses; zeros follow up to column 256 W, so that what is read needs no bounds.  VEC (rows start on a piece and
// d % 8 == 0): a thread copies exactly what it will use itself, and no barrier is spent on the copy; what is read and written in
// shared and global memory then are eight columns at a time (8192 x 4096: forward 59 us against 83, backward 95 against 145).
// ALL: besides, d = 256 W and every input and output is there, which takes the questions out of the loop (4096 x 8192:
// forward 59 us against 62, backward 127 against 147; 8192 x 2048: 31 against 32, 52 against 55; 8192 x 4096: 59 against 58, 95 against 99).
template <class T>
__host__ __device__ constexpr int region_bytes(int threads) { return (threads * static_cast<int>(sizeof(T)) / 2 + 1) * 16; }

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

template <bool VEC, bool FULL, class T>
__device__ __forceinline__ void fetch_row(uint32_t region, const T* row, int t, int tg, int d) {
  constexpr int kPer = sizeof(T) / 2;                     // pieces to a thread
  if (VEC) {
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      cp16(region + (t * kPer + k) * 16, reinterpret_cast<const char*>(row + (FULL || 8 * t < d ? 8 * t : 0)) + 16 * k, FULL || 8 * t < d ? 16 : 0);
  } else {
    const int off = static_cast<int>(reinterpret_cast<uintptr_t>(row) & 15);
    const char* base = reinterpret_cast<const char*>(row) - off;
    const int end = off + d * static_cast<int>(sizeof(T));
    const int left = end - 16 * t;
    const char* from = base + 16 * t;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int bytes = max(0, min(16, left - 16 * k * tg));   // zeros from the row's end to the region's
      cp16(region + (t + k * tg) * 16, bytes > 0 ? from + 16 * k * tg : base, bytes);
    }
    if (t == 0) {
      const int bytes = max(0, min(16, end - 16 * kPer * tg));
      cp16(region + kPer * tg * 16, bytes > 0 ? base + 16 * kPer * tg : base, bytes);
    }
  }
}

// A thread's eight columns: 8t .. 8t+7 (VEC), else every 32nd of its warp's 256.
template <bool VEC>
__device__ __forceinline__ int col_of(int t, int k) { return VEC ? 8 * t + k : (t >> 5) * 256 + (t & 31) + 32 * k; }

// This thread's columns of a fetched row; zeros past the row's end.
template <bool VEC, class T>
__device__ __forceinline__ void take8(const uint8_t* region, const Rows<T>& rows, unsigned i, int t, f32x2 (&p)[4]) {
  float v[8];
  if (VEC) {
    io::load8_shared(region + t * static_cast<int>(8 * sizeof(T)), v, std::remove_const_t<T>());
  } else {
    const T* s = reinterpret_cast<const T*>(region + rows.offset(i)) + col_of<false>(t, 0);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = io::to_f(s[32 * k]);
  }
  io::pairs(v, p);
}
template <bool VEC, bool FULL, class T>
__device__ __forceinline__ void put8(T* row, int t, int d, const f32x2 (&p)[4]) {
  float v[8];
  io::singles(p, v);
  if (VEC && FULL) io::store8(row + 8 * t, v);
  else if (VEC) io::store_cols<true>(row, t, 0, d, v);
  else io::store_cols<false>(row + (t >> 5) * 256, t & 31, 32, d - (t >> 5) * 256, v);
}
__device__ __forceinline__ void fill8(f32x2 (&p)[4], float v) {
#pragma unroll
  for (int k = 0; k < 4; ++k) p[k] = both(v);
}

__device__ __forceinline__ void commit_row() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void wait_row() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// Where a thread stands: its row's group of W warps, and its place among them.  ONE (a block holds one row at a time):
// known to be the same for all threads, so that addresses of rows are computed once per warp.
template <bool ONE>
struct Place {
  int lane, group, wg, t, tg, rg;
  __device__ __forceinline__ explicit Place(int W) {
    const int warp = threadIdx.x >> 5;
    lane = threadIdx.x & 31;
    group = ONE ? 0 : warp / W;
    wg = warp - group * W;
    t = wg * 32 + lane;
    tg = W * 32;
    rg = W == 1 ? 0 : group;                              // rows of one warp do not use the reductions' memory
  }
};

// A norm's weights, or `otherwise` where there is none.
template <bool VEC>
__device__ __forceinline__ void load_weights(const bf16_t* w, int t, int d, float otherwise, f32x2 (&p)[4]) {
  if (w == nullptr) {
    fill8(p, otherwise);
  } else {
    float v[8];
    if (VEC) io::load_cols<true>(w, t, 0, d, v);
    else io::load_cols<false>(w + (t >> 5) * 256, t & 31, 32, d - (t >> 5) * 256, v);
    io::pairs(v, p);
  }
}

__device__ __forceinline__ float square_sum(const f32x2 (&v)[4]) {
  f32x2 s = mul2(v[0], v[0]);
#pragma unroll
  for (int k = 1; k < 4; ++k) s = fma2(v[k], v[k], s);
  return io::lo(s) + io::hi(s);
}

// One value per row, for the rows that a group of warps goes through: lane l holds that of the l-th row from here, so that a
// row costs a shuffle and every 32nd one a load.
template <class T>
__device__ __forceinline__ float row_values(const T* at, long long ld, unsigned i, unsigned step, unsigned N, int lane) {
  const long long row = i + static_cast<long long>(lane) * step;
  return row < N ? io::to_f(at[row * ld]) : 0.f;
}

// ---- forward ----
template <class S>
__host__ __device__ constexpr int fwd_stage_bytes(int threads) { return region_bytes<S>(threads) + 2 * region_bytes<bf16_t>(threads); }

// A row takes two sums, one after the other: of block^2, then of x_out^2.  The second one of a row and the first one of the
// next are formed together, so that a row costs one barrier.
template <class S, bool VEC, int MAXT, int STAGES, bool ONE, bool ALL>
__global__ void __launch_bounds__(MAXT, 1024 / MAXT) norm_fwd_kernel(const __grid_constant__ Params<S> p) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float red[2][ONE ? 1 : 8][2][kMaxWarps];
  const Place<ONE> at(p.W);
  const int t = at.t, tg = at.tg, d = p.d;
  const int rs = region_bytes<S>(tg), rb16 = region_bytes<bf16_t>(tg), stage_bytes = fwd_stage_bytes<S>(tg);
  uint8_t* ring = smem + at.group * STAGES * stage_bytes;
  const bool has_block = ALL || p.block.data != nullptr, has_post = ALL || p.w_post != nullptr, has_y = ALL || p.w_pre != nullptr;
  const bool channel = ALL || p.gate_kind == CPMTP_GATE_CHANNEL, row_gate = !ALL && p.gate_kind == CPMTP_GATE_ROW;
  const unsigned step = gridDim.x * (ONE ? 1 : p.G);      // rows; N < 2^31, so that a few steps past N do not wrap
  unsigned i = blockIdx.x * (ONE ? 1 : p.G) + at.group;
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const uint32_t ring_at = ptx::smem_u32(ring);
  const unsigned N = p.N;
  auto fetch = [&](unsigned row, int stage) {
    if (row < N) {
      uint32_t s = ring_at + stage * stage_bytes;
      fetch_row<VEC, ALL>(s, p.x.at(row), t, tg, d);
      if (has_block) fetch_row<VEC, ALL>(s + rs, p.block.at(row), t, tg, d);
      if (channel) fetch_row<VEC, ALL>(s + rs + rb16, p.gate.at(row), t, tg, d);
    }
    commit_row();
  };
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) fetch(i + s * step, s);
  f32x2 w_post[4], w_pre[4];
  load_weights<VEC>(p.w_post, t, d, 0.f, w_post);
  load_weights<VEC>(p.w_pre, t, d, 0.f, w_pre);
  float logits = 0.f, sum[2] = {0.f, 0.f};
  // sum of block^2 over this thread's columns of the row in `stage`
  auto block_square = [&](unsigned row, int stage) -> float {
    if (!has_post || row >= N) return 0.f;
    f32x2 b[4];
    take8<VEC>(ring + stage * stage_bytes + rs, p.block, row, t, b);
    return square_sum(b);
  };
  wait_row<STAGES - 2>();
  if (!VEC) row_barrier<ONE>(p.W, at.group);
  if (i < N) {
    const float first[2] = {0.f, block_square(i, 0)};
    const float c = begin_sum2<ONE>(first, red[1][at.rg], p.W, at.wg, at.lane);
    end_sum2<ONE>(sum, c, red[1][at.rg], p.W, at.group, at.lane);
  }
  int stage = 0;
  for (int it = 0; i < N; i += step, ++it) {
    const float rb = rsqrtf(fmaf(sum[1], p.inv_d, p.eps));
    float gl = 0.f;
    if (row_gate) {
      if ((it & 31) == 0) logits = row_values(p.gate.data, p.gate.ld, i, step, N, at.lane);
      gl = __shfl_sync(0xffffffffu, logits, it & 31);
    }
    const uint8_t* s = ring + stage * stage_bytes;
    f32x2 x[4];
    take8<VEC>(s, p.x, i, t, x);
    if (has_block) {
      f32x2 b[4], g[4];
      take8<VEC>(s + rs, p.block, i, t, b);
      if (channel) {
        take8<VEC>(s + rs + rb16, p.gate, i, t, g);
#pragma unroll
        for (int k = 0; k < 4; ++k) g[k] = gate_of2(exp_minus2(g[k]));
      } else {
        fill8(g, row_gate ? gate_of(exp_minus(gl)) : 1.f);
      }
      if (has_post) {
        if (t == 0 && (ALL || p.rstd_post != nullptr)) p.rstd_post[i] = rb;
        const f32x2 rb2 = both(rb);
#pragma unroll
        for (int k = 0; k < 4; ++k) b[k] = mul2(b[k], mul2(rb2, w_post[k]));
      }
      const f32x2 scale = both(p.res_scale);
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = fma2(scale, x[k], mul2(g[k], b[k]));
    }
    // the next row is here; the one that comes STAGES - 1 after this goes into the stage before this one's, which every
    // thread has read since the last barrier of the row before (one warp: before this one)
    if (!VEC && p.W == 1) __syncwarp();
    fetch(i + (STAGES - 1) * step, stage == 0 ? STAGES - 1 : stage - 1);
    wait_row<STAGES - 2>();
    if (!VEC) row_barrier<ONE>(p.W, at.group);
    stage = stage + 1 == STAGES ? 0 : stage + 1;
    const float mine[2] = {has_y ? square_sum(x) : 0.f, block_square(i + step, stage)};
    const float c = begin_sum2<ONE>(mine, red[it & 1][at.rg], p.W, at.wg, at.lane);
    if (has_block) put8<VEC, ALL>(p.x_out.at(i), t, d, x);
    end_sum2<ONE>(sum, c, red[it & 1][at.rg], p.W, at.group, at.lane);
    if (has_y) {
      const float rx = rsqrtf(fmaf(sum[0], p.inv_d, p.eps));
      if (t == 0 && (ALL || p.rstd_pre != nullptr)) p.rstd_pre[i] = rx;
      const f32x2 rx2 = both(rx);
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = mul2(x[k], mul2(rx2, w_pre[k]));
      put8<VEC, ALL>(p.y.at(i), t, d, x);
    }
  }
}

// ---- backward ----
// A thread keeps its eight columns' sums of dw_post and dw_pre over all rows of its block.  The gradient t of x_out needs the
// row mean c1 = mean(w_pre dy xh); the norm after the block then needs the mean of w_post du bh, which holds t.  Both come
// out of one reduction over the row, since t = a - c1 rstd_pre xh with a = dx_out + rstd_pre w_pre dy is linear in c1:
//   sum q t = sum q a - c1 rstd_pre sum q xh,      q = g w_post bh.
// The row's two rstd are taken out of the sums and put into per-row factors, which leaves about 30 operations per element.
template <class S>
__host__ __device__ constexpr int bwd_stage_bytes(int threads) { return 2 * region_bytes<S>(threads) + 3 * region_bytes<bf16_t>(threads); }

// Forms of the kernel: a gate per row or none, which leaves out all arithmetic on gates of channels (8192 x 4096, a gate per row: 89 us
// against 113 in one form with the next); a gate per channel; and the latter with everything there (see above).
enum { kRowGate, kChannelGate, kAll };

template <class S, bool VEC, int MAXT, int STAGES, bool ONE, int FORM>
__global__ void __launch_bounds__(MAXT) norm_bwd_kernel(const __grid_constant__ Params<S> p) {
  constexpr bool ALL = FORM == kAll, CHANNEL = FORM != kRowGate;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float red[2][ONE ? 1 : 8][4][kMaxWarps];
  const Place<ONE> at(p.W);
  const int t = at.t, tg = at.tg, d = p.d;
  const int rs = region_bytes<S>(tg), rb16 = region_bytes<bf16_t>(tg), stage_bytes = bwd_stage_bytes<S>(tg);
  uint8_t* ring = smem + at.group * STAGES * stage_bytes;
  const unsigned step = gridDim.x * (ONE ? 1 : p.G);      // rows; N < 2^31, so that a few steps past N do not wrap
  const bool has_block = ALL || p.block.data != nullptr, has_post = ALL || (has_block && p.w_post != nullptr);
  const bool row_gate = !CHANNEL && p.gate_kind == CPMTP_GATE_ROW;
  const bool has_y = ALL || p.dy.data != nullptr, has_dx_out = ALL || p.dx_out.data != nullptr;
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  unsigned i = blockIdx.x * (ONE ? 1 : p.G) + at.group;
  const uint32_t ring_at = ptx::smem_u32(ring);
  const unsigned N = p.N;
  auto fetch = [&](unsigned row, int stage) {
    if (row < N) {
      uint32_t s = ring_at + stage * stage_bytes;
      fetch_row<VEC, ALL>(s, p.x_out.at(row), t, tg, d);
      if (has_dx_out) fetch_row<VEC, ALL>(s + rs, p.dx_out.at(row), t, tg, d);
      s += 2 * rs;
      if (has_y) fetch_row<VEC, ALL>(s, p.dy.at(row), t, tg, d);
      if (has_block) fetch_row<VEC, ALL>(s + rb16, p.block.at(row), t, tg, d);
      if (CHANNEL) fetch_row<VEC, ALL>(s + 2 * rb16, p.gate.at(row), t, tg, d);
    }
    commit_row();
  };
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) fetch(i + s * step, s);
  f32x2 w_pre[4], w_post[4], acc_pre[4], acc_post[4];
  fill8(acc_pre, 0.f);
  fill8(acc_post, 0.f);
  load_weights<VEC>(has_y ? p.w_pre : nullptr, t, d, 0.f, w_pre);
  load_weights<VEC>(has_post ? p.w_post : nullptr, t, d, 1.f, w_post);
  float rstds_pre = 0.f, rstds_post = 1.f, logits = 0.f;
  int stage = 0;

  // Row r, the it-th of this group: what comes before its sums, into `row`, and the sums as far as this warp goes.
  // Gates are held as e = exp(-logit), from which g and 1 - g are made where they are used (holding both: 123 us against 96 at
  // 8192 x 4096).  Where registers are short not even that, the logits are read from the ring again: two ragged rows at a time
  // (16384 x 2047: 145 us against 156), 64 registers (4096 x 8192: 127 against 146); elsewhere e is better kept (8192 x 4096: 99 against 106).
  constexpr bool KEEP_E = MAXT <= 512 && (VEC || !ONE);
  // A row is finished while the warps' sums of the next one are on their way: two rows are held at a time, which 128 registers
  // allow where rows' addresses are common to the block.  It pays where a row is short of other work to wait with, bf16 with
  // everything there (8192 x 4096: 94 us against 96) and ragged rows (16384 x 2047, 1023: 144 and 60 us against 147 and 63); it does not
  // with fewer arrays or an fp32 stream (8192 x 4096: row gates 89 us against 82, fp32 129 against 125).
  constexpr bool PIPE = ONE && MAXT <= 512 && (!VEC || (ALL && sizeof(S) == 2));
  struct Row {
    f32x2 x[4], a[4], b[4], e[CHANNEL && KEEP_E ? 4 : 1];
    float rx, rb, erow;
  };
  auto gates = [&](unsigned r, int stage, f32x2 (&e)[4]) {
    take8<VEC>(ring + stage * stage_bytes + 2 * rs + 2 * rb16, p.gate, r, t, e);
#pragma unroll
    for (int k = 0; k < 4; ++k) e[k] = exp_minus2(e[k]);
  };
  auto before_sums = [&](unsigned r, int it, Row& row) -> float {
    if ((it & 31) == 0) {
      if (has_y) rstds_pre = row_values(p.rstd_pre, 1, r, step, N, at.lane);
      if (has_post) rstds_post = row_values(p.rstd_post, 1, r, step, N, at.lane);
      if (row_gate) logits = row_values(p.gate.data, p.gate.ld, r, step, N, at.lane);
    }
    row.rx = __shfl_sync(0xffffffffu, rstds_pre, it & 31);
    row.rb = __shfl_sync(0xffffffffu, rstds_post, it & 31);
    row.erow = row_gate ? exp_minus(__shfl_sync(0xffffffffu, logits, it & 31)) : 0.f;
    wait_row<STAGES - 2>();
    if (!VEC) row_barrier<ONE>(p.W, at.group);
    const uint8_t* s = ring + stage * stage_bytes;
    f32x2 dy[4], e[4];
    if (CHANNEL) gates(r, stage, e);
    stage = stage + 1 == STAGES ? 0 : stage + 1;
    take8<VEC>(s, p.x_out, r, t, row.x);
    if (has_dx_out) take8<VEC>(s + rs, p.dx_out, r, t, row.a);
    else fill8(row.a, 0.f);
    s += 2 * rs;
    if (has_y) take8<VEC>(s, p.dy, r, t, dy);
    else fill8(dy, 0.f);
    if (has_block) take8<VEC>(s + rb16, p.block, r, t, row.b);
    else fill8(row.b, 0.f);
    f32x2 s0 = both(0.f), s1 = s0, s2 = s0;
    const f32x2 rx2 = both(row.rx);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const f32x2 dyr = mul2(dy[k], rx2), wdyr = mul2(w_pre[k], dyr);
      acc_pre[k] = fma2(dyr, row.x[k], acc_pre[k]);
      row.a[k] = add2(row.a[k], wdyr);
      f32x2 q = mul2(w_post[k], row.b[k]);
      if (CHANNEL) q = mul2(q, gate_of2(e[k]));
      if (CHANNEL && KEEP_E) row.e[k] = e[k];
      s0 = fma2(wdyr, row.x[k], s0);
      s1 = fma2(q, row.a[k], s1);
      s2 = fma2(q, row.x[k], s2);
    }
    const float sum[3] = {io::lo(s0) + io::hi(s0), io::lo(s1) + io::hi(s1), io::lo(s2) + io::hi(s2)};
    return begin_sum3<ONE>(sum, red[it & 1][at.rg], p.W, at.wg, at.lane);
  };
  // And what comes after them, when `ago` rows from this one on have been read: it is still in the ring.
  auto after_sums = [&](unsigned r, const Row& row, const float (&sum)[3], int ago) {
    const float c1 = row.rx * row.rx * sum[0] * p.inv_d;              // t = a - c1 x
    const float dot = row.rb * fmaf(-c1, sum[2], sum[1]);             // sum of t u (the row gate left out)
    const float grow = row_gate ? gate_of(row.erow) : 1.f;
    const f32x2 minus_c1 = both(-c1), grb = both(grow * row.rb), scale = both(p.res_scale);
    const f32x2 minus_c2 = both(has_post ? -row.rb * row.rb * grow * dot * p.inv_d : 0.f);
    f32x2 dx[4], dblock[4], dgate[4], e[4];
    if (CHANNEL && !KEEP_E) gates(r, stage >= ago ? stage - ago : stage + STAGES - ago, e);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const f32x2 tk = fma2(minus_c1, row.x[k], row.a[k]);
      f32x2 dur = mul2(grb, tk), rest = 0ull;                         // rstd_post du
      if (CHANNEL) {
        if (KEEP_E) {
          e[k] = row.e[k];
          asm("" : "+l"(e[k]));                                       // (a new value: else g is held since before the sums)
        }
        const f32x2 g = gate_of2(e[k]);
        dur = mul2(dur, g);
        rest = rest_of2(e[k], g);
      }
      acc_post[k] = fma2(dur, row.b[k], acc_post[k]);
      dblock[k] = fma2(w_post[k], dur, mul2(minus_c2, row.b[k]));
      if (CHANNEL) dgate[k] = mul2(mul2(mul2(w_post[k], row.b[k]), dur), rest);
      dx[k] = mul2(scale, tk);
    }
    if (ALL || p.dx.data != nullptr) put8<VEC, ALL>(p.dx.at(r), t, d, dx);
    if (ALL || p.dblock.data != nullptr) put8<VEC, ALL>(p.dblock.at(r), t, d, dblock);
    if (ALL || p.dgate.data != nullptr) {
      if (CHANNEL) put8<VEC, ALL>(p.dgate.at(r), t, d, dgate);
      else if (t == 0) *p.dgate.at(r) = io::from_f<bf16_t>(grow * rest_of(row.erow, grow) * dot);
    }
  };

  // the row that comes STAGES - 1 after row r goes into the stage before the one read last
  auto fetch_after = [&](unsigned r) {
    if (!VEC && p.W == 1) __syncwarp();
    fetch(r + (STAGES - 1) * step, stage >= 2 ? stage - 2 : stage + STAGES - 2);
  };
  float sum[3];
  if (PIPE) {
    if (i < N) {
      Row row;
      end_sum3<ONE>(sum, before_sums(i, 0, row), red[0][at.rg], p.W, at.group, at.lane);
#pragma unroll 2
      for (int it = 1; i + step < N; i += step, ++it) {
        fetch_after(i);
        Row next;
        const float c = before_sums(i + step, it, next);
        after_sums(i, row, sum, 2);
        end_sum3<ONE>(sum, c, red[it & 1][at.rg], p.W, at.group, at.lane);
        row = next;
      }
      after_sums(i, row, sum, 1);
    }
  } else {
    for (int it = 0; i < N; i += step, ++it) {
      Row row;
      const float c = before_sums(i, it, row);
      fetch_after(i);
      end_sum3<ONE>(sum, c, red[it & 1][at.rg], p.W, at.group, at.lane);
      after_sums(i, row, sum, 1);
    }
  }
  if (p.part == nullptr) return;
  float sum_pre[8], sum_post[8];
  io::singles(acc_pre, sum_pre);
  io::singles(acc_post, sum_post);
  float* out = p.part + static_cast<size_t>(blockIdx.x) * 2 * d;
  if (ONE) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int c = col_of<VEC>(t, k);
      if (c < d) {
        out[c] = sum_post[k];
        out[d + c] = sum_pre[k];
      }
    }
    return;
  }
  // the rows that the block held at a time, one after the other
  wait_row<0>();
  __syncthreads();
  float* sums = reinterpret_cast<float*>(smem);               // [2][G][8 tg]
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int c = col_of<VEC>(t, k);
    sums[at.group * 8 * tg + c] = sum_post[k];
    sums[(p.G + at.group) * 8 * tg + c] = sum_pre[k];
  }
  __syncthreads();
  for (int c = threadIdx.x; c < 2 * d; c += blockDim.x) {
    const int which = c >= d, col = c - which * d;
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
  ptx::grid_dep_launch();
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
