// AdamW over many tensors in one launch, states in fp32 or 8 bits, and the norm of all gradients.
//
// The tensors' descriptors travel in the kernel's parameters (up to 32 KB), so a step is one launch with no copy to
// the device, and can be captured; to be replayed as the steps that follow it takes what changes from step to step from a
// clock in device memory, which a second, tiny launch advances.  Bound by bandwidth with fp32 states (133 M parameters with an
// fp32 copy, 28 bytes each: 561 us, 6.6 TB/s), by instruction issue with 8-bit ones (10 bytes each: 290 us).  Every block takes one run
// of elements of one tensor; a warp takes 256 elements at a time, which are also what shares an exponent in an 8-bit state.
#pragma once
#include "vec_io.cuh"

namespace cpmtp {
namespace adamw {

using io::bf16_t;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kBlock = CPMTP_ADAMW_BLOCK;
// Elements per thread block: short runs where there are few blocks, long ones for the kernel that has a ring to fill (a warp
// of it goes through at most 32 blocks, whose exponents its lanes hold).
constexpr int kShortRun = 2048, kRun = 8192, kLongRun = 32768;
static_assert(kLongRun <= 32 * kWarps * kBlock, "one exponent to a lane");
static_assert(kBlock == 32 * 8, "a warp holds one block of an 8-bit state");

struct Tensor {
  void* param;
  const void* grad;
  float* master;
  void *m, *v;
  uint8_t *m_exp, *v_exp;
  long long numel;
  long long place;                               // of its first element among all tensors' elements
  float step_size, keep;                         // see Rates; with a clock the tensor's factors of lr and wd alone
  int16_t param_f32, grad_f32;
  int32_t vec;                                   // every pointer allows accesses of eight elements
};

// What changes from step to step: of all tensors, and (the first two) of one.
struct Rates {
  float step_size, keep, rsqrt_bc2;              // lr / (1 - beta1^t) and 1 - lr wd, with the tensor's factors; (1 - beta2^t)^(-1/2)
  uint32_t key;                                  // of the rounding noise: seed and step
  int small_eps;                                 // roots of subnormal second moments count beside eps
};

struct Hyper {
  float b1, omb1, b2, omb2, eps;
  Rates r;                                       // (no clock) but for what depends on the tensor
  const float* coef;
  float one;                                     // 1, see update_block8()
  const cpmtp_adamw_clock* clock;                // the step's number and rate are there, nullptr: in r
  double wd;
};
// A root below 2^-63 (of a moment below 2^-126) adds less than half a unit of fp32 to eps from here on, per unit of rsqrt_bc2.
constexpr float kSmallEps = 1.f / 549755813888.f;                      // 2^-39

template <int CAP>
struct Table {
  Hyper h;
  int count;
  int run;                                       // elements to a thread block
  int first[CAP];                                // first run (thread block) of each tensor
  Tensor t[CAP];
};
constexpr int kSmallTable = 24, kMiddleTable = 96, kLargeTable = 300;   // a launch takes 3, 5 and up to 9 us with them

// Products and differences of doubles rounded one by one, so that host and device get the same bits.
__host__ __device__ __forceinline__ double product(double a, double b) {
#ifdef __CUDA_ARCH__
  return __dmul_rn(a, b);
#else
  return a * b;
#endif
}
__host__ __device__ __forceinline__ double one_minus(double a) {
#ifdef __CUDA_ARCH__
  return __dsub_rn(1.0, a);
#else
  return 1.0 - a;
#endif
}
__host__ __device__ __forceinline__ double power(double base, unsigned long long n) {
  double r = 1.0;
  for (; n > 0; n >>= 1, base = product(base, base))
    if (n & 1) r = product(r, base);
  return r;
}
__host__ __device__ __forceinline__ float step_size_of(double lr, float factor, double bc1) { return static_cast<float>(product(lr, factor) / bc1); }
__host__ __device__ __forceinline__ float keep_of(double lr, float factor, double wd, float decay_factor) {
  return static_cast<float>(one_minus(product(product(product(lr, factor), wd), decay_factor)));
}
__host__ __device__ __forceinline__ float rsqrt_bc2_of(double beta2, unsigned long long t) {
  return static_cast<float>(1.0 / sqrt(one_minus(power(beta2, t))));
}

// lowbias32 of Chris Wellons' hash-prospector: a bijection of 32 bits whose output bits each depend on every input bit
__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0x7feb352du;
  x ^= x >> 15;
  x *= 0x846ca68bu;
  return x ^ (x >> 16);
}

__host__ __device__ __forceinline__ uint32_t noise_key(uint32_t seed, unsigned long long t) { return mix(mix(seed) ^ static_cast<uint32_t>(t)); }

// The clock's next step.
__global__ void adamw_clock_kernel(cpmtp_adamw_clock* clock, double beta1, double beta2) {
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const unsigned long long t = (clock->step > 0 ? clock->step : 0) + 1;
  clock->step = static_cast<long long>(t);
  clock->bc1 = one_minus(power(beta1, t));
  clock->rsqrt_bc2 = rsqrt_bc2_of(beta2, t);
  clock->key = noise_key(clock->seed, t);
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
__device__ __forceinline__ void read_codes(const uint8_t* base, int lane, int left, uint32_t (&c)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) c[k] = elem<false>(lane, k) < left ? base[elem<false>(lane, k)] : 0u;
}
__device__ __forceinline__ void write_codes(uint8_t* base, int lane, int left, const uint32_t (&c)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k)
    if (elem<false>(lane, k) < left) base[elem<false>(lane, k)] = static_cast<uint8_t>(c[k]);
}

// To a neighbouring bf16 value, the upper one with the probability that keeps the mean.  Infinities and NaN are left to
// the conversion; the sum may carry a finite number to infinity.
__device__ __forceinline__ float round_up_or_down(float p, uint32_t noise) {
  const uint32_t bits = __float_as_uint(p);
  return (bits & 0x7f800000u) == 0x7f800000u ? p : __uint_as_float((bits + ((noise >> 8) & 0xFFFFu)) & 0xFFFF0000u);
}

// One warp's 256 elements, `left` of them inside the tensor.  8-bit states that allow wide accesses go through update_block8().
template <int BITS, bool VEC>
__device__ __forceinline__ void update(const Tensor& t, const Hyper& h, const Rates& r, float coef, long long at, int left, int lane) {
  static_assert(BITS == 32 || !VEC, "see above");
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
    read_codes(m8, lane, left, cm);
    read_codes(v8, lane, left, cv);
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
    p[k] = p[k] * r.keep - __fdividef(m[k] * r.step_size, fmaf(sqrtf(v[k]), r.rsqrt_bc2, h.eps));
  }
  const bool rounds_p = t.master == nullptr && !t.param_f32;
  uint32_t noise[8];
  if (BITS == 8 || rounds_p) {
    const unsigned long long place = static_cast<unsigned long long>(t.place + at);
    const uint32_t key = r.key ^ (static_cast<uint32_t>(place >> 32) * 0x9E3779B9u);
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
      cm[k] |= (__float_as_uint(m[k]) >> 31) << 7;
      if (cv[k] == 0u) cm[k] = 0u;
    }
    write_codes(m8, lane, left, cm);
    write_codes(v8, lane, left, cv);
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
      for (int k = 0; k < 8; ++k) p[k] = round_up_or_down(p[k], noise[k]);
    }
    write<VEC>(static_cast<bf16_t*>(t.param) + at, lane, left, p);
  }
}

// ---- 8-bit states, a whole block of a tensor that allows wide accesses ----
// 10 bytes move per element and some 60 operations are due, which is what an SM issues in the time those bytes take: so
// everything is counted.  Pairs are multiplied and added together (rounded as the single operations are); codes are
// unpacked and packed in place, four to a word; and where the exponents leave room, the two powers of two of encode() and
// decode() are one, and the decoder's goes into beta's product.  Both forms give the same bits.
using io::add2;
using io::both;
using io::f32x2;
using io::fma2;
using io::mul2;

// decode() is exact from here on up (the smallest code stays a normal number); its factors merge up to there
constexpr int kMergeLow = 20, kMergeHigh = 141;
__device__ __forceinline__ bool merges(int e) { return e == 0 || (e >= kMergeLow && e <= kMergeHigh); }
// 2^(e - 15): from the code's units to values
__device__ __forceinline__ float unit_of(int e) { return __uint_as_float(static_cast<uint32_t>(e + 112) << 23); }
// 2^(15 - e): back
__device__ __forceinline__ float inverse_unit_of(int e) { return __uint_as_float(static_cast<uint32_t>(142 - e) << 23); }

// Root and reciprocal; FLUSH: single instructions, which take subnormal numbers for zeros (668 M bf16 parameters: the
// question which of the two a block takes costs 0.7 %; without the flush the root of a subnormal moment stays beside a small eps).
template <bool FLUSH>
__device__ __forceinline__ float sqrt_approx(float x) {
  float r;
  if (FLUSH) asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  else asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
template <bool FLUSH>
__device__ __forceinline__ float rcp_approx(float x) {
  float r;
  if (FLUSH) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  else asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
template <bool FLUSH>
__device__ __forceinline__ void update_params(f32x2 (&p)[4], const f32x2 (&m)[4], const f32x2 (&v)[4], const Hyper& h, const Rates& r) {
  const f32x2 step = both(-r.step_size), keep = both(r.keep), bias = both(r.rsqrt_bc2), eps = both(h.eps);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const f32x2 below = fma2(io::pair(sqrt_approx<FLUSH>(io::lo(v[k])), sqrt_approx<FLUSH>(io::hi(v[k]))), bias, eps);
    p[k] = fma2(p[k], keep, mul2(mul2(m[k], step), io::pair(rcp_approx<FLUSH>(io::lo(below)), rcp_approx<FLUSH>(io::hi(below)))));
  }
}
__device__ __forceinline__ float max_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// bytes 3 of four words, as one word
__device__ __forceinline__ uint32_t tops(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}

// Blocks ahead are fetched with cp.async into a ring of kAhead blocks per warp, each lane its own share: 1.5 to 2.5 KB a
// block is too little for a warp to have under way at a time (2.1 us of waiting per block, half of the bandwidth).
constexpr int kAhead = 4;

// Eight elements of either type as they lie in memory.
struct Raw8 {
  uint4 a, b;                     // b: of fp32 elements the upper four
};
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, int bytes) {
  if (bytes == 8) asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void fetch_raw(uint32_t dst, const void* p, bool f32, long long at) {
  if (f32) {
    copy_async(dst, static_cast<const float*>(p) + at, 16);
    copy_async(dst + 512, static_cast<const float*>(p) + at + 4, 16);
  } else {
    copy_async(dst, static_cast<const bf16_t*>(p) + at, 16);
  }
}
__device__ __forceinline__ Raw8 take_raw(const uint8_t* s, bool f32) {
  Raw8 r;
  r.a = *reinterpret_cast<const uint4*>(s);
  if (f32) r.b = *reinterpret_cast<const uint4*>(s + 512);
  return r;
}
__device__ __forceinline__ void numbers(const Raw8& r, bool f32, f32x2 (&v)[4]) {
  if (f32) {
    const uint32_t w[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = io::pair(__uint_as_float(w[2 * k]), __uint_as_float(w[2 * k + 1]));
  } else {
    float f[8];
    io::unpack8(r.a, f);
    io::pairs(f, v);
  }
}

struct Loaded8 {                  // a lane's share of a block as it is read
  uint2 m, v;
  Raw8 g, p;
  int em, ev;
};

// A block in shared memory: m and v, 8 bytes a lane; then the gradient and what the update works on, 16 bytes a lane and
// once more 16 for fp32.
__host__ __device__ constexpr int stage_bytes(bool g32, bool p32) { return 512 + 512 * (2 + (g32 ? 1 : 0) + (p32 ? 1 : 0)); }

__device__ __forceinline__ void fetch_block8(const Tensor& t, long long at, int lane, uint32_t stage) {
  copy_async(stage + 8 * lane, static_cast<const uint8_t*>(t.m) + at + 8 * lane, 8);
  copy_async(stage + 256 + 8 * lane, static_cast<const uint8_t*>(t.v) + at + 8 * lane, 8);
  const uint32_t g = stage + 512 + 16 * lane, p = g + (t.grad_f32 ? 1024 : 512);
  fetch_raw(g, t.grad, t.grad_f32, at + 8 * lane);
  if (t.master != nullptr) fetch_raw(p, t.master, true, at + 8 * lane);
  else fetch_raw(p, t.param, t.param_f32, at + 8 * lane);
}
__device__ __forceinline__ void take_block8(const Tensor& t, const uint8_t* stage, int lane, Loaded8& in) {
  in.m = *reinterpret_cast<const uint2*>(stage + 8 * lane);
  in.v = *reinterpret_cast<const uint2*>(stage + 256 + 8 * lane);
  const uint8_t *g = stage + 512 + 16 * lane, *p = g + (t.grad_f32 ? 1024 : 512);
  in.g = take_raw(g, t.grad_f32);
  in.p = take_raw(p, t.param_f32 || t.master != nullptr);
}

__device__ __forceinline__ void update_block8(const Tensor& t, const Hyper& h, const Rates& r, float coef, long long at, int lane, const Loaded8& in) {
  f32x2 g[4], m[4], v[4], p[4];
  numbers(in.g, t.grad_f32, g);
  numbers(in.p, t.param_f32 || t.master != nullptr, p);
  const int em0 = in.em, ev0 = in.ev;         // the block's exponents
  // codes to the places that encode() gives them in a number, with the sign on top for m
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t wm = k < 2 ? in.m.x : in.m.y, wv = k < 2 ? in.v.x : in.v.y;
    const int j = 2 * (k & 1);
    const auto place_m = [](uint32_t w, int j) {
      return __uint_as_float(static_cast<uint32_t>(static_cast<int32_t>(w << (24 - 8 * j)) >> 4) & 0x87F00000u);
    };
    const auto place_v = [](uint32_t w, int j) { return __uint_as_float((j < 3 ? w << (19 - 8 * j) : w >> 5) & 0x07F80000u); };
    m[k] = io::pair(place_m(wm, j), place_m(wm, j + 1));
    v[k] = io::pair(place_v(wv, j), place_v(wv, j + 1));
  }
  if (merges(em0) && merges(ev0)) {
    const f32x2 b1 = both(h.b1 * unit_of(em0)), b2 = both(h.b2 * unit_of(ev0));
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      m[k] = mul2(m[k], b1);
      v[k] = mul2(v[k], b2);
    }
  } else {
    const f32x2 huge = both(kHuge), um = both(block_unit(em0)), uv = both(block_unit(ev0)), b1 = both(h.b1), b2 = both(h.b2);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      m[k] = mul2(mul2(mul2(m[k], huge), um), b1);
      v[k] = mul2(mul2(mul2(v[k], huge), uv), b2);
    }
  }
  const f32x2 coef2 = both(coef), omb1 = both(h.omb1), omb2 = both(h.omb2);
  // sums as products with a 1 that the compiler does not know: a packed sum of a packed product was found to come out as one
  // operation with one rounding, for all the explicit roundings of the two
  const f32x2 one = both(h.one);
  float top_m = 0.f, top_v = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const f32x2 gk = mul2(g[k], coef2);
    m[k] = fma2(m[k], one, mul2(gk, omb1));
    v[k] = fma2(v[k], one, mul2(mul2(gk, omb2), gk));
    top_m = max_nan(top_m, fabsf(io::lo(m[k])), fabsf(io::hi(m[k])));
    top_v = max_nan(top_v, io::lo(v[k]), io::hi(v[k]));
  }
  if (r.small_eps) update_params<false>(p, m, v, h, r);
  else update_params<true>(p, m, v, h, r);
  const uint32_t top_mb = __reduce_max_sync(0xffffffffu, __float_as_uint(top_m)), top_vb = __reduce_max_sync(0xffffffffu, __float_as_uint(top_v));
  const int em = min(block_exp<kDropM>(top_mb), 255), ev = min(block_exp<kDropV>(top_vb), 255);
  // the first step of mix() for eight places that differ in their lowest three bits alone
  const unsigned long long place = static_cast<unsigned long long>(t.place + at);
  uint32_t base = (static_cast<uint32_t>(place) + 8 * lane) ^ r.key ^ (static_cast<uint32_t>(place >> 32) * 0x9E3779B9u);
  base ^= base >> 16;
  uint32_t noise[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    uint32_t x = (base ^ k) * 0x7feb352du;
    x ^= x >> 15;
    x *= 0x846ca68bu;
    noise[k] = x ^ (x >> 16);
  }
  uint32_t cm[8], cv[8];          // codes in the words' top bytes
  if (em >= 1 && em <= kMergeHigh && ev >= 1 && ev <= kMergeHigh) {
    const f32x2 to_m = both(inverse_unit_of(em)), to_v = both(inverse_unit_of(ev));
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const f32x2 a = mul2(m[k], to_m), b = mul2(v[k], to_v);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        // encode()'s sums, moved up until the code is the top byte (what is below the noise then does not carry)
        const uint32_t u = noise[2 * k + i];
        const uint32_t am = __float_as_uint(i == 0 ? io::lo(a) : io::hi(a)), av = __float_as_uint(i == 0 ? io::lo(b) : io::hi(b));
        const uint32_t sm = (am << 4) + __byte_perm(u, 0u, 0x4104);
        cm[2 * k + i] = (sm & 0x7FFFFFFFu) | (am & 0x80000000u);
        cv[2 * k + i] = (av << 5) + (u >> 8);
      }
    }
  } else {
    const float to_m = pow2(254 - min(em, 254)), to_v = pow2(254 - min(ev, 254));
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float mk = (k & 1) ? io::hi(m[k / 2]) : io::lo(m[k / 2]), vk = (k & 1) ? io::hi(v[k / 2]) : io::lo(v[k / 2]);
      cv[k] = (ev > 0 && ev < 255 ? encode<kDropV>(fabsf(vk), to_v, noise[k] >> 13) : 0u) << 24;
      cm[k] = ((em > 0 && em < 255 ? encode<kDropM>(fabsf(mk), to_m, (noise[k] & 0xFFFFu) << 4) : 0u) | (__float_as_uint(mk) >> 31) << 7) << 24;
    }
  }
  uint2 mw, vw;
  mw.x = tops(cm[0], cm[1], cm[2], cm[3]);
  mw.y = tops(cm[4], cm[5], cm[6], cm[7]);
  vw.x = tops(cv[0], cv[1], cv[2], cv[3]);
  vw.y = tops(cv[4], cv[5], cv[6], cv[7]);
  // where v is zero m is too
  const auto nonzero = [](uint32_t w) { return ((((w & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | w) >> 7 & 0x01010101u) * 255u; };
  mw.x &= nonzero(vw.x);
  mw.y &= nonzero(vw.y);
  *reinterpret_cast<uint2*>(static_cast<uint8_t*>(t.m) + at + 8 * lane) = mw;
  *reinterpret_cast<uint2*>(static_cast<uint8_t*>(t.v) + at + 8 * lane) = vw;
  if (lane == 0) {
    t.m_exp[at / kBlock] = static_cast<uint8_t>(em);
    t.v_exp[at / kBlock] = static_cast<uint8_t>(ev);
  }
  float q[8];
  io::singles(p, q);
  if (t.master != nullptr) write<true>(t.master + at, lane, kBlock, q);
  if (t.param_f32) {
    write<true>(static_cast<float*>(t.param) + at, lane, kBlock, q);
  } else if (t.master != nullptr) {
    write<true>(static_cast<bf16_t*>(t.param) + at, lane, kBlock, q);
  } else {
    const f32x2 sum = add2(add2(p[0], p[1]), add2(p[2], p[3]));
    if (io::lo(sum) + io::hi(sum) == io::lo(sum) + io::hi(sum)) {
      // no NaN among them (infinities take the noise unharmed): the rounded values are the words' upper halves
      uint32_t w[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) w[k] = __float_as_uint(q[k]) + __byte_perm(noise[k], 0u, 0x4421);
      *reinterpret_cast<uint4*>(static_cast<bf16_t*>(t.param) + at + 8 * lane) =
          make_uint4(__byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x7632), __byte_perm(w[4], w[5], 0x7632), __byte_perm(w[6], w[7], 0x7632));
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) q[k] = round_up_or_down(q[k], noise[k]);
      write<true>(static_cast<bf16_t*>(t.param) + at, lane, kBlock, q);
    }
  }
}

// The rates of tensor t.  CLOCK: from the clock, with the operations that the host would have made.
template <bool CLOCK>
__device__ __forceinline__ Rates rates_of(const Tensor& t, const Hyper& h) {
  Rates r = h.r;
  r.step_size = t.step_size;
  r.keep = t.keep;
  if (CLOCK) {
    const double lr = h.clock->lr;
    r.step_size = step_size_of(lr, t.step_size, h.clock->bc1);
    r.keep = keep_of(lr, t.step_size, h.wd, t.keep);
    r.rsqrt_bc2 = h.clock->rsqrt_bc2;
    r.key = h.clock->key;
    r.small_eps = h.eps < kSmallEps * r.rsqrt_bc2;
  }
  return r;
}

template <int CAP, bool CLOCK>
__global__ void __launch_bounds__(kThreads) adamw32_kernel(const __grid_constant__ Table<CAP> tab) {
  const int which = tensor_of(tab, blockIdx.x);
  const Tensor& t = tab.t[which];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const float coef = tab.h.coef != nullptr ? *tab.h.coef : 1.f;
  if (coef != coef) return;                      // the gradients were not finite
  const Rates r = rates_of<CLOCK>(t, tab.h);
  const long long start = static_cast<long long>(static_cast<int>(blockIdx.x) - tab.first[which]) * tab.run;
#pragma unroll 1
  for (int b = warp * kBlock; b < tab.run; b += kWarps * kBlock) {
    const long long at = start + b;
    if (at >= t.numel) break;
    const int left = static_cast<int>(min(t.numel - at, static_cast<long long>(kBlock)));
    if (t.vec) update<32, true>(t, tab.h, r, coef, at, left, lane);
    else update<32, false>(t, tab.h, r, coef, at, left, lane);
  }
}

template <int CAP, bool CLOCK>
__global__ void __launch_bounds__(kThreads, 4) adamw8_kernel(const __grid_constant__ Table<CAP> tab, const int bytes) {
  extern __shared__ __align__(16) uint8_t smem[];
  const int which = tensor_of(tab, blockIdx.x);
  const Tensor& t = tab.t[which];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long start = static_cast<long long>(static_cast<int>(blockIdx.x) - tab.first[which]) * tab.run;
  const long long here = min(t.numel - start, static_cast<long long>(tab.run));
  // blocks of this run: all, and those that are whole and go through shared memory; the warp's are warp, warp + kWarps, ...
  const int blocks = static_cast<int>((here + kBlock - 1) / kBlock), whole = t.vec ? static_cast<int>(here / kBlock) : 0;
  const uint8_t* ring = smem + warp * kAhead * bytes;
  const uint32_t ring_at = ptx::smem_u32(ring);
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const float coef = tab.h.coef != nullptr ? *tab.h.coef : 1.f;
  // lane l: the exponents of the warp's l-th block
  const int mine = warp + kWarps * lane;
  int em = 0, ev = 0;
  if (mine < whole) {
    em = t.m_exp[start / kBlock + mine];
    ev = t.v_exp[start / kBlock + mine];
  }
  const auto fetch = [&](int b, int stage) {
    if (b < whole) fetch_block8(t, start + static_cast<long long>(b) * kBlock, lane, ring_at + stage * bytes);
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int s = 0; s < kAhead - 1; ++s) fetch(warp + s * kWarps, s);
  if (coef != coef) {                            // the gradients were not finite: nothing changes
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    return;
  }
  const Rates r = rates_of<CLOCK>(t, tab.h);
  int n = 0;
#pragma unroll 1
  for (int b = warp; b < whole; b += kWarps, ++n) {
    fetch(b + (kAhead - 1) * kWarps, (n + kAhead - 1) % kAhead);
    asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
    Loaded8 in;
    take_block8(t, ring + (n % kAhead) * bytes, lane, in);
    in.em = __shfl_sync(0xffffffffu, em, n);
    in.ev = __shfl_sync(0xffffffffu, ev, n);
    update_block8(t, tab.h, r, coef, start + static_cast<long long>(b) * kBlock, lane, in);
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  // what is left: the tensor's last block, or all of one whose pointers do not allow wide accesses
  for (int b = whole + (warp - whole % kWarps + kWarps) % kWarps; b < blocks; b += kWarps) {
    const long long at = start + static_cast<long long>(b) * kBlock;
    update<8, false>(t, tab.h, r, coef, at, static_cast<int>(min(t.numel - at, static_cast<long long>(kBlock))), lane);
  }
}

// A warp decodes kValueBlocks blocks, all read before the first is written.
constexpr int kValueBlocks = 4;
template <bool SECOND>
__global__ void __launch_bounds__(kThreads) state_values_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ exps, long long n,
                                                                bf16_t* __restrict__ out, int vec) {
  const int lane = threadIdx.x & 31;
  const long long first = (static_cast<long long>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5)) * (kValueBlocks * kBlock);
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const auto value = [](uint32_t c, float unit) {
    if (SECOND) return decode<kDropV>(c, unit);
    const float a = decode<kDropM>(c & 127u, unit);
    return c > 127u ? -a : a;
  };
  if (vec && first + kValueBlocks * kBlock <= n) {
    uint2 r[kValueBlocks];
    float unit[kValueBlocks];
#pragma unroll
    for (int j = 0; j < kValueBlocks; ++j) {
      r[j] = *reinterpret_cast<const uint2*>(codes + first + j * kBlock + 8 * lane);
      unit[j] = block_unit(exps[first / kBlock + j]);
    }
#pragma unroll
    for (int j = 0; j < kValueBlocks; ++j) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = value(((k < 4 ? r[j].x : r[j].y) >> (8 * (k & 3))) & 255u, unit[j]);
      io::store8(out + first + j * kBlock + 8 * lane, v);
    }
    return;
  }
  for (int j = 0; j < kValueBlocks; ++j) {
    const long long at = first + j * kBlock;
    if (at >= n) return;
    const int left = static_cast<int>(min(n - at, static_cast<long long>(kBlock)));
    const float unit = block_unit(exps[at / kBlock]);
    uint32_t c[8];
    float v[8];
    read_codes(codes + at, lane, left, c);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = value(c[k], unit);
    write<false>(out + at, lane, left, v);
  }
}

// Sum of squares of every gradient: a block takes runs of elements, in turn with the others.  A warp reads the kSquareBlocks
// blocks of a whole run that are its own before it uses the first (one at a time it reached half of the bandwidth).
constexpr int kSquareBlocks = kRun / (kWarps * kBlock);

template <class T>
__device__ __forceinline__ void add_squares(const T* g, int lane, float (&acc)[8]) {
  uint32_t w[kSquareBlocks][2 * sizeof(T)];
#pragma unroll
  for (int j = 0; j < kSquareBlocks; ++j) io::load8_raw(g + j * kWarps * kBlock + 8 * lane, w[j]);
#pragma unroll
  for (int j = 0; j < kSquareBlocks; ++j) {
    float v[8];
    io::numbers8<T>(w[j], v);
#pragma unroll
    for (int k = 0; k < 8; ++k) acc[k] = fmaf(v[k], v[k], acc[k]);
  }
}

template <int CAP>
__global__ void __launch_bounds__(kThreads) grad_square_kernel(const __grid_constant__ Table<CAP> tab, int runs, double* __restrict__ part) {
  __shared__ double sums[kWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float acc[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) acc[k] = 0.f;
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  for (int run = blockIdx.x; run < runs; run += gridDim.x) {
    const int which = tensor_of(tab, run);
    const Tensor& t = tab.t[which];
    const long long start = static_cast<long long>(run - tab.first[which]) * tab.run;
    if (t.vec && tab.run == kRun && start + kRun <= t.numel) {
      const long long at = start + warp * kBlock;
      if (t.grad_f32) add_squares(static_cast<const float*>(t.grad) + at, lane, acc);
      else add_squares(static_cast<const bf16_t*>(t.grad) + at, lane, acc);
      continue;
    }
#pragma unroll 1
    for (int b = warp * kBlock; b < tab.run; b += kWarps * kBlock) {
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
    for (int w = 1; w < kWarps; ++w) s += sums[w];
    part[blockIdx.x] = s;
  }
}

__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const double* __restrict__ part, int parts, float max_norm, float* norm, float* coef) {
  __shared__ double sums[kThreads / 32];
  double s = 0.0;
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
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
