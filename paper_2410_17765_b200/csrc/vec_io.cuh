// Eight consecutive elements of a row at a time: bf16 as one 16-byte access, fp32 as one 32-byte access.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

#include "ptx.cuh"

namespace cpmtp {
namespace io {

using bf16_t = uint16_t;

__device__ __forceinline__ float to_f(bf16_t v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); }
__device__ __forceinline__ float to_f(float v) { return v; }

template <class T>
__device__ __forceinline__ T from_f(float v);
template <>
__device__ __forceinline__ float from_f<float>(float v) { return v; }
template <>
__device__ __forceinline__ bf16_t from_f<bf16_t>(float v) {
  return static_cast<bf16_t>(ptx::pack_bf16x2(v, 0.f) & 0xFFFFu);
}

__device__ __forceinline__ void unpack8(const uint4& r, float (&v)[8]) {
  v[0] = ptx::bf16_lo(r.x); v[1] = ptx::bf16_hi(r.x);
  v[2] = ptx::bf16_lo(r.y); v[3] = ptx::bf16_hi(r.y);
  v[4] = ptx::bf16_lo(r.z); v[5] = ptx::bf16_hi(r.z);
  v[6] = ptx::bf16_lo(r.w); v[7] = ptx::bf16_hi(r.w);
}
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
  return make_uint4(ptx::pack_bf16x2(v[0], v[1]), ptx::pack_bf16x2(v[2], v[3]), ptx::pack_bf16x2(v[4], v[5]),
                    ptx::pack_bf16x2(v[6], v[7]));
}

__device__ __forceinline__ void load8(const bf16_t* p, float (&v)[8]) {
  unpack8(*reinterpret_cast<const uint4*>(p), v);
}
// 32-byte accesses are one instruction on sm_100 (a 16-byte pair would touch every sector twice)
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
               : "l"(p)
               : "memory");
}
// The same as words, for loads whose values are wanted later.
__device__ __forceinline__ void load8_raw(const bf16_t* p, uint32_t (&w)[4]) {
  const uint4 r = *reinterpret_cast<const uint4*>(p);
  w[0] = r.x; w[1] = r.y; w[2] = r.z; w[3] = r.w;
}
__device__ __forceinline__ void load8_raw(const float* p, uint32_t (&w)[8]) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
               : "l"(p)
               : "memory");
}
template <class T, int N>
__device__ __forceinline__ void numbers8(const uint32_t (&w)[N], float (&v)[8]) {
  if (sizeof(T) == 4) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(w[k % N]);
  } else {
    unpack8(make_uint4(w[0], w[1], w[2], w[3]), v);
  }
}
// (the last argument names the type of the elements)
__device__ __forceinline__ void load8_shared(const uint8_t* s, float (&v)[8], bf16_t) { unpack8(*reinterpret_cast<const uint4*>(s), v); }
__device__ __forceinline__ void load8_shared(const uint8_t* s, float (&v)[8], float) {
  const float4 a = *reinterpret_cast<const float4*>(s), b = *reinterpret_cast<const float4*>(s + 16);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void store8(bf16_t* p, const float (&v)[8]) { *reinterpret_cast<uint4*>(p) = pack8(v); }
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]),
               "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
               : "memory");
}

// Two fp32 values in one register pair: sm_100 multiplies and adds pairs in one instruction, which is what counts where
// the issue slots are what a kernel runs out of.  Each half is rounded as the single operation would be.
using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 pair(float lo, float hi) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ f32x2 both(float v) { return pair(v, v); }
__device__ __forceinline__ float lo(f32x2 v) { return __uint_as_float(static_cast<uint32_t>(v)); }
__device__ __forceinline__ float hi(f32x2 v) { return __uint_as_float(static_cast<uint32_t>(v >> 32)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// Eight values, as pairs and one by one.
__device__ __forceinline__ void pairs(const float (&v)[8], f32x2 (&p)[4]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) p[k] = pair(v[2 * k], v[2 * k + 1]);
}
__device__ __forceinline__ void singles(const f32x2 (&p)[4], float (&v)[8]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[2 * k] = lo(p[k]);
    v[2 * k + 1] = hi(p[k]);
  }
}

// Whether rows of T at `p`, `ld` elements apart and `d` wide, can be read eight elements at a time.
template <class T>
inline bool vec_ok(const void* p, long long ld, long long d) {
  return reinterpret_cast<uintptr_t>(p) % (8 * sizeof(T)) == 0 && ld % 8 == 0 && d % 8 == 0;
}

// The elements of a row of `d` that thread `t` of `threads` owns: columns 8t .. 8t+7 (VEC), else t, t + threads, ...
// Columns past the end read as zero and are not written.
template <bool VEC, class T>
__device__ __forceinline__ void load_cols(const T* row, int t, int threads, int d, float (&v)[8]) {
  if (VEC) {
    if (8 * t < d) {
      load8(row + 8 * t, v);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = 0.f;
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int c = t + k * threads;
      v[k] = c < d ? to_f(row[c]) : 0.f;
    }
  }
}

template <bool VEC, class T>
__device__ __forceinline__ void store_cols(T* row, int t, int threads, int d, const float (&v)[8]) {
  if (VEC) {
    if (8 * t < d) store8(row + 8 * t, v);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int c = t + k * threads;
      if (c < d) row[c] = from_f<T>(v[k]);
    }
  }
}

__device__ __forceinline__ float sum_lanes(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

}  // namespace io
}  // namespace cpmtp
