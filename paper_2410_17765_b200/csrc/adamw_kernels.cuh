// AdamW over many tensors in one launch, states in fp32 or 8 bits, and the norm of all gradients.
//
// The tensors' descriptors travel in the kernel's parameters (up to 32 KB), so a step is one launch with no copy to
// the device, and can be captured.  Every block takes one run of kRun elements of one tensor; a warp takes 256 elements at a time, which
// are also what shares an exponent in an 8-bit state.
#pragma once
#include "vec_io.cuh"

namespace cpmtp {
namespace adamw {

using io::bf16_t;

constexpr int kThreads = 256;
constexpr int kBlock = CPMTP_ADAMW_BLOCK;
constexpr int kRun = 8192;                       // elements per thread block
static_assert(kBlock == 32 * 8, "a warp holds one block of an 8-bit state");

struct Tensor {
  void* param;
  const void* grad;
  float* master;
  void *m, *v;
  uint8_t *m_exp, *v_exp;
  long long numel;
  long long place;                               // of its first element among all tensors' elements
  float step_size, keep;                         // lr / (1 - beta1^t) and 1 - lr wd, with the tensor's factors
  int16_t param_f32, grad_f32;
  int32_t vec;                                   // every pointer allows accesses of eight elements
};

struct Hyper {
  float b1, omb1, b2, omb2, rsqrt_bc2, eps;
  uint32_t key;                                  // of the rounding noise: seed and step
  const float* coef;
};

template <int CAP>
struct Table {
  Hyper h;
  int count;
  int first[CAP];                                // first run (thread block) of each tensor
  Tensor t[CAP];
};
constexpr int kSmallTable = 24, kLargeTable = 300;

// lowbias32 of Chris Wellons' hash-prospector: a bijection of 32 bits whose output bits each depend on every input bit
__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0x7feb352du;
  x ^= x >> 15;
  x *= 0x846ca68bu;
  return x ^ (x >> 16);
}

// 2^(e - 127) for e in [0, 254]
__device__ __forceinline__ float pow2(int e) { return __uint_as_float(e > 0 ? static_cast<uint32_t>(e) << 23 : 1u << 22); }

// 8-bit codes.  A magnitude relative to its block's exponent e, moved so that e becomes exponent field 15 of an
// fp32 number, has its code in the top bits of that number: 4 exponent bits and 23 - DROP mantissa bits, and fp32's own
// subnormals are the code's.  Rounding up or down at random is adding noise below the last kept bit.
constexpr int kDropM = 20, kDropV = 19;
constexpr float kTiny = 1.f / 5192296858534827628530496329220096.f;    // 2^-112: exponent field 127 -> 15
constexpr float kHuge = 5192296858534827628530496329220096.f;          // 2^112

template <int DROP>
__device__ __forceinline__ int block_exp(uint32_t top_bits) { return static_cast<int>((top_bits + (1u << DROP)) >> 23); }
template <int DROP>
__device__ __forceinline__ uint32_t encode(float a, float to_one, uint32_t noise) {
  return (__float_as_uint(__fmul_rn(__fmul_rn(a, to_one), kTiny)) + noise) >> DROP;
}
template <int DROP>
__device__ __forceinline__ float decode(uint32_t code, float unit) {
  return __fmul_rn(__fmul_rn(__uint_as_float(code << DROP), kHuge), unit);
}
__device__ __forceinline__ float block_unit(int e) { return e == 255 ? __uint_as_float(0x7fc00000u) : pow2(e); }

template <int CAP>
__device__ __forceinline__ int tensor_of(const Table<CAP>& tab, int run) {
  int lo = 0, hi = tab.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (tab.first[mid] <= run) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Element k of eight of lane's share of a warp's 256: consecutive ones (VEC) or every 32nd.
template <bool VEC>
__device__ __forceinline__ int elem(int lane, int k) { return VEC ? 8 * lane + k : lane + 32 * k; }

template <bool VEC, class T>
__device__ __forceinline__ void read(const T* base, int lane, int left, float (&v)[8]) {
  if (VEC && left >= kBlock) {
    io::load8(base + 8 * lane, v);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = elem<VEC>(lane, k) < left ? io::to_f(base[elem<VEC>(lane, k)]) : 0.f;
  }
}
template <bool VEC, class T>
__device__ __forceinline__ void write(T* base, int lane, int left, const float (&v)[8]) {
  if (VEC && left >= kBlock) {
    io::store8(base + 8 * lane, v);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (elem<VEC>(lane, k) < left) base[elem<VEC>(lane, k)] = io::from_f<T>(v[k]);
  }
}
template <bool VEC>
__device__ __forceinline__ void read_any(const void* p, bool f32, long long at, int lane, int left, float (&v)[8]) {
  if (f32) read<VEC>(static_cast<const float*>(p) + at, lane, left, v);
  else read<VEC>(static_cast<const bf16_t*>(p) + at, lane, left, v);
}
template <bool VEC>
__device__ __forceinline__ void read_codes(const uint8_t* base, int lane, int left, uint32_t (&c)[8]) {
  if (VEC && left >= kBlock) {
    const uint2 r = *reinterpret_cast<const uint2*>(base + 8 * lane);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      c[k] = (r.x >> (8 * k)) & 255u;
      c[k + 4] = (r.y >> (8 * k)) & 255u;
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) c[k] = elem<VEC>(lane, k) < left ? base[elem<VEC>(lane, k)] : 0u;
  }
}
template <bool VEC>
__device__ __forceinline__ void write_codes(uint8_t* base, int lane, int left, const uint32_t (&c)[8]) {
  if (VEC && left >= kBlock) {
    uint2 r;
    r.x = c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24;
    r.y = c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24;
    *reinterpret_cast<uint2*>(base + 8 * lane) = r;
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (elem<VEC>(lane, k) < left) base[elem<VEC>(lane, k)] = static_cast<uint8_t>(c[k]);
  }
}

// One warp's 256 elements, `left` of them inside the tensor.
template <int BITS, bool VEC>
__device__ __forceinline__ void update(const Tensor& t, const Hyper& h, float coef, long long at, int left, int lane) {
  float g[8], m[8], v[8], p[8];
  read_any<VEC>(t.grad, t.grad_f32, at, lane, left, g);
  if (t.master != nullptr) read<VEC>(t.master + at, lane, left, p);
  else read_any<VEC>(t.param, t.param_f32, at, lane, left, p);
  uint8_t* m8 = static_cast<uint8_t*>(t.m) + at;
  uint8_t* v8 = static_cast<uint8_t*>(t.v) + at;
  float* m32 = static_cast<float*>(t.m) + at;
  float* v32 = static_cast<float*>(t.v) + at;
  if (BITS == 8) {
    uint32_t cm[8], cv[8];
    read_codes<VEC>(m8, lane, left, cm);
    read_codes<VEC>(v8, lane, left, cv);
    const float um = block_unit(t.m_exp[at / kBlock]), uv = block_unit(t.v_exp[at / kBlock]);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float a = decode<kDropM>(cm[k] & 127u, um);
      m[k] = cm[k] > 127u ? -a : a;
      v[k] = decode<kDropV>(cv[k], uv);
    }
  } else {
    read<VEC>(m32, lane, left, m);
    read<VEC>(v32, lane, left, v);
  }
  // products and sums are rounded one by one: the 8-bit codes depend on the last bit
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float gk = __fmul_rn(g[k], coef);
    m[k] = __fadd_rn(__fmul_rn(m[k], h.b1), __fmul_rn(gk, h.omb1));
    v[k] = __fadd_rn(__fmul_rn(v[k], h.b2), __fmul_rn(__fmul_rn(gk, h.omb2), gk));
    p[k] = p[k] * t.keep - __fdividef(m[k] * t.step_size, fmaf(sqrtf(v[k]), h.rsqrt_bc2, h.eps));
  }
  const bool rounds_p = t.master == nullptr && !t.param_f32;
  uint32_t noise[8];
  if (BITS == 8 || rounds_p) {
    const unsigned long long place = static_cast<unsigned long long>(t.place + at);
    const uint32_t key = h.key ^ (static_cast<uint32_t>(place >> 32) * 0x9E3779B9u);
#pragma unroll
    for (int k = 0; k < 8; ++k) noise[k] = mix((static_cast<uint32_t>(place) + elem<VEC>(lane, k)) ^ key);
  }
  if (BITS == 8) {
    uint32_t top_m = 0, top_v = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      top_m = max(top_m, __float_as_uint(fabsf(m[k])));
      top_v = max(top_v, __float_as_uint(fabsf(v[k])));
    }
    top_m = __reduce_max_sync(0xffffffffu, top_m);
    top_v = __reduce_max_sync(0xffffffffu, top_v);
    const int em = min(block_exp<kDropM>(top_m), 255), ev = min(block_exp<kDropV>(top_v), 255);
    const float to_m = pow2(254 - min(em, 254)), to_v = pow2(254 - min(ev, 254));
    uint32_t cm[8], cv[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      cv[k] = ev > 0 && ev < 255 ? encode<kDropV>(fabsf(v[k]), to_v, noise[k] >> 13) : 0u;
      cm[k] = em > 0 && em < 255 ? encode<kDropM>(fabsf(m[k]), to_m, (noise[k] & 0xFFFFu) << 4) : 0u;
      if (m[k] < 0.f) cm[k] |= 128u;
      if (cv[k] == 0u) cm[k] = 0u;
    }
    write_codes<VEC>(m8, lane, left, cm);
    write_codes<VEC>(v8, lane, left, cv);
    if (lane == 0) {
      t.m_exp[at / kBlock] = static_cast<uint8_t>(em);
      t.v_exp[at / kBlock] = static_cast<uint8_t>(ev);
    }
  } else {
    write<VEC>(m32, lane, left, m);
    write<VEC>(v32, lane, left, v);
  }
  if (t.master != nullptr) write<VEC>(t.master + at, lane, left, p);
  if (t.param_f32) {
    write<VEC>(static_cast<float*>(t.param) + at, lane, left, p);
  } else {
    if (rounds_p) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        // infinities and NaN are left to the conversion; the sum may carry a finite number to infinity
        const uint32_t bits = __float_as_uint(p[k]);
        if ((bits & 0x7f800000u) != 0x7f800000u) p[k] = __uint_as_float((bits + ((noise[k] >> 8) & 0xFFFFu)) & 0xFFFF0000u);
      }
    }
    write<VEC>(static_cast<bf16_t*>(t.param) + at, lane, left, p);
  }
}

template <int BITS, int CAP>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ Table<CAP> tab) {
  const int which = tensor_of(tab, blockIdx.x);
  const Tensor& t = tab.t[which];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  ptx::grid_dep_wait();
  const float coef = tab.h.coef != nullptr ? *tab.h.coef : 1.f;
  if (coef != coef) return;                      // the gradients were not finite
  const long long start = static_cast<long long>(static_cast<int>(blockIdx.x) - tab.first[which]) * kRun;
#pragma unroll 1
  for (int b = warp * kBlock; b < kRun; b += kThreads / 32 * kBlock) {
    const long long at = start + b;
    if (at >= t.numel) break;
    const int left = static_cast<int>(min(t.numel - at, static_cast<long long>(kBlock)));
    if (t.vec) update<BITS, true>(t, tab.h, coef, at, left, lane);
    else update<BITS, false>(t, tab.h, coef, at, left, lane);
  }
}

template <bool SECOND>
__global__ void __launch_bounds__(kThreads) state_values_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ exps, long long n,
                                                                bf16_t* __restrict__ out, int vec) {
  const int lane = threadIdx.x & 31;
  const long long at = (static_cast<long long>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5)) * kBlock;
  ptx::grid_dep_wait();
  if (at >= n) return;
  const int left = static_cast<int>(min(n - at, static_cast<long long>(kBlock)));
  const float unit = block_unit(exps[at / kBlock]);
  uint32_t c[8];
  float v[8];
  if (vec) read_codes<true>(codes + at, lane, left, c); else read_codes<false>(codes + at, lane, left, c);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (SECOND) {
      v[k] = decode<kDropV>(c[k], unit);
    } else {
      const float a = decode<kDropM>(c[k] & 127u, unit);
      v[k] = c[k] > 127u ? -a : a;
    }
  }
  if (vec) write<true>(out + at, lane, left, v); else write<false>(out + at, lane, left, v);
}

// Sum of squares of every gradient: a block takes runs of kRun elements, in turn with the others.
template <int CAP>
__global__ void __launch_bounds__(kThreads) grad_square_kernel(const __grid_constant__ Table<CAP> tab, int runs, double* __restrict__ part) {
  __shared__ double sums[kThreads / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float acc[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) acc[k] = 0.f;
  ptx::grid_dep_wait();
  for (int run = blockIdx.x; run < runs; run += gridDim.x) {
    const int which = tensor_of(tab, run);
    const Tensor& t = tab.t[which];
    const long long start = static_cast<long long>(run - tab.first[which]) * kRun;
#pragma unroll 1
    for (int b = warp * kBlock; b < kRun; b += kThreads / 32 * kBlock) {
      const long long at = start + b;
      if (at >= t.numel) break;
      const int left = static_cast<int>(min(t.numel - at, static_cast<long long>(kBlock)));
      float g[8];
      if (t.vec) read_any<true>(t.grad, t.grad_f32, at, lane, left, g);
      else read_any<false>(t.grad, t.grad_f32, at, lane, left, g);
#pragma unroll
      for (int k = 0; k < 8; ++k) acc[k] = fmaf(g[k], g[k], acc[k]);
    }
  }
  double s = 0.0;
#pragma unroll
  for (int k = 0; k < 8; ++k) s += acc[k];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane == 0) sums[warp] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kThreads / 32; ++w) s += sums[w];
    part[blockIdx.x] = s;
  }
}

__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const double* __restrict__ part, int parts, float max_norm, float* norm, float* coef) {
  __shared__ double sums[kThreads / 32];
  double s = 0.0;
  ptx::grid_dep_wait();
  for (int j = threadIdx.x; j < parts; j += kThreads) s += part[j];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int w = 1; w < kThreads / 32; ++w) s += sums[w];
  const float n = static_cast<float>(sqrt(s));
  if (norm != nullptr) *norm = n;
  if (coef != nullptr) *coef = isfinite(n) ? fminf(1.f, max_norm / (n + 1e-6f)) : __uint_as_float(0x7fc00000u);
}

}  // namespace adamw
}  // namespace cpmtp
