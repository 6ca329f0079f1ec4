// Sampling from logits with temperature, top-k, top-p and min-p by given uniform numbers.
//
// A row is shared out over the blocks of a cluster, which pass over it one to three times (after the first time it comes from L2).  Its weights
// w = 2^z, z = (x - m) log2(e) / T, are integers (62 - log2 V bits below the point) whose sums are exact in any order, so borders between
// kept and dropped entries, and the token that a number draws, do not depend on how the row is shared out.  Where a filter ends is found in two
// steps: a histogram over z in steps of 1/64 names the few bins in which it lies, and their entries, a few hundred of 128256, are sorted in one
// block.  Should they be too many (long runs of equal logits, flat rows), the key of the last kept entry is found by digits instead.
//
// What bounds it: at many rows the instructions, about 35 for a weight and 8 for its bin; at few rows the latency of a dozen barriers of a
// cluster.  512 x 128256 in fp32 (263 MB): greedy 62 us, top-k of 50 113, no filter 160, top-p 313; 8 rows in bf16: 5, 16, 13 and 31 (in captured graphs).  Holding the
// row in shared memory was slower at many rows (512 x 128256 in bf16 with top-p: 473 us against 357 then), since it leaves room for fewer
// blocks, and 1 us faster at few.
#pragma once
#include <cfloat>
#include <climits>
#include <cstdint>

#include "../../include/cpmtp.h"
#include "cluster.cuh"
#include "ptx.cuh"
#include "vec_io.cuh"

namespace cpmtp {
namespace sample {

using io::bf16_t;
using cluster::load_remote32;
using cluster::load_remote64;
using cluster::remote;
using cluster::store_remote;
using cluster::sync_row;
using cluster::u64;

using cluster::kMostCtas;
constexpr int kBins = 2048;            // of the histogram, 64 to a factor of two
constexpr int kList = 2048;            // entries that one block sorts ...
constexpr int kCounted = 192;          // ... by counting the larger ones for each (more: by a bitonic network)
constexpr int kTable = 1024;           // powers of two between one and two
constexpr int kQueue = 9 * 32;         // logits that a warp collects before it weighs them

template <int THREADS>
struct Shared {
  static constexpr int kWarps = THREADS / 32;
  u64 table[kTable];
  u64 list[kList];
  union {
    uint32_t hist[kBins];
    struct {
      u64 mass[256];
      uint32_t count[256];
    } digit;
  };
  float queue[kWarps][kQueue];
  double scan[kWarps];
  u64 sums[kWarps];                    // kept mass of the warps' ranges
  u64 box[8][kMostCtas];               // numbers from the blocks of the cluster; two places in turn
  u64 word[4];
  int listed, number[3];
};

// -------------------------------------------------------------------------------------------- keys and weights
// Unsigned keys in the order of the logits.
__device__ __forceinline__ uint32_t logit_key(float x) { return cluster::order_key(x); }
__device__ __forceinline__ float key_logit(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k); }

// z <= 0 with 32 bits below the point, in two words.
struct Fixed {
  int whole;             // floor(z)
  uint32_t part;         // z - floor(z)
};
// Conditions of the inner loops are put together without branches, which would cost more than what they skip.
__device__ __forceinline__ bool at_least(Fixed z, Fixed least) {
  return (static_cast<long long>(z.whole) << 32 | z.part) >= (static_cast<long long>(least.whole) << 32 | least.part);
}
__device__ __forceinline__ u64 only_if(bool c, u64 v) { return v & -static_cast<u64>(c); }

struct Weigh {
  double m, c;           // largest logit; log2(e) / T
  float x_min, x_max;    // what logits are limited to: below the one is no weight, above the other is nothing
  int down;              // 62 minus the bits below the point
  uint32_t table;        // address in shared memory

  // A weight below 2^-160 is none (the least min_p is 2^-149).  Where the next number below the largest logit is further away
  // than that, it is put at 2^-1000, so that z has always few enough digits before the point; so is everything below an infinite one, for
  // which the largest finite number stands.
  __device__ __forceinline__ void set(float top, double inv_t, int bits) {
    x_max = fminf(top, FLT_MAX);
    m = static_cast<double>(x_max);
    c = inv_t * 1.4426950408889634074;
    const double low = m - 160.0 / c;                  // (c may be 0: minus infinity)
    x_min = low > -FLT_MAX ? __double2float_rd(low) : -FLT_MAX;
    if (top > x_max || !(x_min < top) || !((m - static_cast<double>(x_min)) * c < 1000.0)) {
      x_min = nextafterf(x_max, -INFINITY);
      if (x_min >= -FLT_MAX) c = 1000.0 / (m - static_cast<double>(x_min));
    }
    down = 62 - bits;
  }
  // (x - m) c: the product is added to a number whose last bit is 2^-32.
  __device__ __forceinline__ Fixed z(float x) const {
    constexpr double kMagic = 1572864.0;               // 1.5 x 2^20
    const double v = fma(static_cast<double>(fminf(fmaxf(x, x_min), x_max)) - m, c, kMagic);
    return Fixed{__double2hiint(v) - 0x41380000, static_cast<uint32_t>(__double2loint(v))};
  }
  // 2^(z - floor(z)) with 62 bits below the point.  The leading ten bits by table, the others by three terms of the series of
  // 2^r - 1, r < 2^-10, in fp32: an error of 2^-24 of a number below 2^-10.5.  With the 2^-33 of z and the 2^-34 of its own
  // rounding below 2^-32 in all.
  __device__ __forceinline__ u64 mantissa(Fixed z) const {
    u64 e;
    asm("ld.shared.u64 %0, [%1];" : "=l"(e) : "r"(table + ((z.part >> 22) << 3)));
    const float r = __uint_as_float(0x3f800000u | (z.part & 0x3fffffu) << 1) - 1.f;           // in units of 2^-10
    constexpr double kA = 0.69314718055994530942 / 1024.0, kS = 8589934592.0;                 // ln 2 2^-10; 2^33
    const float q = fmaf(r, fmaf(r, static_cast<float>(kA * kA * kA / 6.0 * kS), static_cast<float>(kA * kA / 2.0 * kS)), static_cast<float>(kA * kS));
    const uint32_t n = __float_as_uint(fmaf(r, q, 8388608.f)) & 0x7fffffu;
    return e + static_cast<u64>(static_cast<uint32_t>(e >> 33)) * n;
  }
  __device__ __forceinline__ u64 fixed(u64 mantissa, Fixed z) const { return mantissa >> min(down - z.whole, 63); }
  __device__ __forceinline__ u64 weight(Fixed z) const { return fixed(mantissa(z), z); }
  __device__ __forceinline__ u64 weight(float x) const { return weight(z(x)); }
};

struct Settings {
  double inv_t, top_p, min_p;
  int top_k;             // V: none
  bool one;              // the first entry alone is kept
};
__device__ __forceinline__ Settings settings_of(const cpmtp_sample_args& a, int i) {
  Settings r;
  const float t = a.temperatures != nullptr ? a.temperatures[i] : a.temperature;
  const float p = a.top_ps != nullptr ? a.top_ps[i] : a.top_p, mp = a.min_ps != nullptr ? a.min_ps[i] : a.min_p;
  const int k = a.top_ks != nullptr ? a.top_ks[i] : a.top_k;
  r.inv_t = t > 0.f ? 1.0 / static_cast<double>(t) : 1.0;
  r.top_p = p < 1.f ? static_cast<double>(p) : 1.0;
  r.min_p = mp > 0.f ? static_cast<double>(mp) : 0.0;
  r.top_k = k > 0 && k < a.V ? k : a.V;
  r.one = !(t > 0.f) || r.top_p <= 0.0 || r.min_p > 1.0 || r.top_k == 1;
  return r;
}

// -------------------------------------------------------------------------------------------- the kernel
// A cluster of `ctas` blocks to a row.  A block's entries are read in whole 16-byte pieces, the first and last of which may reach beyond
// them; its warps have equal ranges of pieces.
template <class T, int THREADS>
struct Row {
  static constexpr int kThreads = THREADS, kWarps = THREADS / 32;
  static constexpr int kEach = kList / THREADS;        // entries of a full list to a thread
  static constexpr int kPer = 16 / sizeof(T);
  Shared<THREADS>& sh;
  const int ctas, rank, t, lane, warp;
  int base, n;           // this block's entries
  int off;               // entries of the first piece that lie before them
  int pieces, each;      // pieces of the block, of a warp
  const uint4* data;
  int boxes;

  __device__ __forceinline__ void sync() const { sync_row(ctas); }

  static __device__ __forceinline__ void unpack(const uint4& raw, float (&v)[kPer]) {
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (sizeof(T) == 4) {
        v[q % kPer] = __uint_as_float(w[q]);
      } else {
        v[(2 * q) % kPer] = ptx::bf16_lo(w[q]);
        v[(2 * q + 1) % kPer] = ptx::bf16_hi(w[q]);
      }
    }
  }
  __device__ __forceinline__ void load(int piece, float (&v)[kPer]) const { unpack(__ldg(data + piece), v); }
  // What a piece has beyond the block's entries counts as never kept; only the first and the last can.
  __device__ __forceinline__ void limit(int piece, float (&v)[kPer]) const {
#pragma unroll
    for (int q = 0; q < kPer; ++q) {
      const int i = piece * kPer + q - off;
      if (i < 0 || i >= n) v[q] = -INFINITY;
    }
  }
  // f(piece, its entries) for this warp's pieces, all lanes in step (a lane without a piece gets entries that are never kept): first those that lie
  // inside, then the block's first and last one.
  template <class F>
  __device__ __forceinline__ void for_pieces(F f) const {
    const int begin = warp * each, end = min(begin + each, pieces), inner = min(end, pieces - 1);
    uint4 raw = make_uint4(0, 0, 0, 0);
    if (max(begin, 1) + lane < inner) raw = __ldg(data + max(begin, 1) + lane);
#pragma unroll 1
    for (int p = max(begin, 1) + lane; p - lane < inner; p += 32) {
      float v[kPer];
      unpack(raw, v);
      if (p >= inner) {
#pragma unroll
        for (int q = 0; q < kPer; ++q) v[q] = -INFINITY;
      }
      if (p + 32 < inner) raw = __ldg(data + p + 32);          // under way meanwhile
      f(p, v);
    }
    const int last = pieces - 1;
    const bool has_first = begin == 0 && end > 0, has_last = last > 0 && last >= begin && last < end;
    if (has_first || has_last) {
      const int p = has_first && lane == 0 ? 0 : has_last && lane == 1 ? last : -1;
      float v[kPer];
      if (p >= 0) load(p, v);
      limit(p < 0 ? -8 : p, v);
      f(p, v);
    }
  }
  // f(logit, index in the row) for the entries of this warp's pieces.
  template <class F>
  __device__ __forceinline__ void for_each(F f) const {
    for_pieces([&](int p, const float (&v)[kPer]) {
#pragma unroll
      for (int q = 0; q < kPer; ++q) f(v[q], base + p * kPer + q - off);
    });
  }
  __device__ __forceinline__ int warp_of(int index) const { return (index - base + off) / kPer / each; }

  __device__ __forceinline__ u64 warp_sum(u64 v) const {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
  }
  // Sum over the block's threads, in every thread.
  __device__ __forceinline__ u64 block_sum(u64 v) {
    v = warp_sum(v);
    __syncthreads();
    u64* part = reinterpret_cast<u64*>(sh.scan);
    if (lane == 0) part[warp] = v;
    __syncthreads();
    v = lane < kWarps ? part[lane] : 0;
#pragma unroll
    for (int o = kWarps / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return __shfl_sync(0xffffffffu, v, 0);
  }
  // Sums up to and with each thread's v over the block.
  __device__ __forceinline__ u64 block_scan(u64 v) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u64 u = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += u;
    }
    u64* part = reinterpret_cast<u64*>(sh.scan);
    __syncthreads();
    if (lane == 31) part[warp] = v;
    __syncthreads();
    u64 before = lane < warp ? part[lane & (kWarps - 1)] : 0;
    return v + warp_sum(before);
  }
  // Gives numbers (of the first warp's threads) to every block and brings theirs: box[r] of block r.  A barrier of the cluster.
  __device__ __forceinline__ const u64* exchange(u64 v) { return exchange(v, 0, 1); }
  __device__ __forceinline__ const u64* exchange(u64 v, u64 second, int boxes_used = 2) {
    u64* box = sh.box[boxes];
    boxes = (boxes + 2) & 7;
    if (t < ctas) {
      if (ctas == 1) {
        box[0] = v;
        box[kMostCtas] = second;
      } else {
        store_remote(box + rank, t, v);
        if (boxes_used > 1) store_remote(box + kMostCtas + rank, t, second);
      }
    }
    sync();
    return box;
  }
  __device__ __forceinline__ u64 sum_of(const u64* box) const {
    u64 s = 0;
    for (int r = 0; r < ctas; ++r) s += box[r];
    return s;
  }
  __device__ __forceinline__ u64 row_sum(u64 v) { return sum_of(exchange(block_sum(v))); }

  // The first bin at which the running sum of the histogram, bin b weighing scale(b), reaches `low` and leaves no more than low_left behind it, what lies
  // before that bin, and the first bin at which the sum reaches `high` or leaves no more than high_left; the last bin where there is none.  Returns
  // the whole sum.
  template <class Scale>
  __device__ __forceinline__ double find_bins(Scale scale, double low, double high, double low_left, double high_left, int& b1, int& b2, double& before) {
    constexpr int kOwn = kBins / kThreads > 0 ? kBins / kThreads : 1;
    sync();                                            // the blocks' histograms are complete
    const int per = kBins / ctas, mine_of = (per + kThreads - 1) / kThreads;       // bins of this block, of a thread
    double mine[kOwn], sum = 0.0;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      mine[j] = 0.0;
      const int b = t * mine_of + j;
      if (j < mine_of && b < per) {
        u64 c = 0;
        if (ctas == 1) {
          c = sh.hist[b];
        } else {
          uint32_t h[kMostCtas];
#pragma unroll
          for (int r = 0; r < kMostCtas; ++r) h[r] = r < ctas ? load_remote32(&sh.hist[rank * per + b], r) : 0;
#pragma unroll
          for (int r = 0; r < kMostCtas; ++r) c += h[r];
        }
        mine[j] = static_cast<double>(c) * scale(rank * per + b);
        sum += mine[j];
      }
    }
    double upto = sum;                                 // of this thread's bins and those before them in the warp
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double v = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += v;
    }
    __syncthreads();
    if (lane == 31) sh.scan[warp] = upto;
    if (t == 0) {
      sh.number[0] = sh.number[1] = kBins - 1;
      sh.word[0] = 0;
    }
    __syncthreads();
    double all = 0.0;
    for (int w = 0; w < kWarps; ++w) all += sh.scan[w];
    const u64* box = exchange(__double_as_longlong(all));
    double run = 0.0, total = 0.0;
    for (int r = 0; r < ctas; ++r) {
      if (r == rank) run = total;
      total += __longlong_as_double(box[r]);
    }
    for (int w = 0; w < warp; ++w) run += sh.scan[w];
    low = fmax(low, total - low_left);
    high = fmin(high, total - high_left);
    // a thread begins with the very number that the one before it ends with, so that no border falls between them
    upto += run;
    const double left = __shfl_up_sync(0xffffffffu, upto, 1);
    if (lane > 0) run = left;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const double next = j + 1 == mine_of ? upto : run + mine[j];
      const int b = rank * per + t * mine_of + j;
      if (j < mine_of && t * mine_of + j < per) {
        if (run < low && next >= low)
          for (int r = 0; r < ctas; ++r) {
            store_remote(&sh.word[0], r, __double_as_longlong(run));
            asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(remote(&sh.number[0], r)), "r"(b) : "memory");
          }
        if (run < high && next >= high)
          for (int r = 0; r < ctas; ++r) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(remote(&sh.number[1], r)), "r"(b) : "memory");
      }
      run = next;
    }
    sync();
    b1 = sh.number[0];
    b2 = sh.number[1];
    before = __longlong_as_double(sh.word[0]);
    return total;
  }

  __device__ __forceinline__ void clear_hist() {
    for (int b = t; b < kBins; b += kThreads) sh.hist[b] = 0;
    if (t == 0) sh.listed = 0;
    __syncthreads();
  }

  // Entries (logit, index) as keys that sort in falling order of the logit and rising order of the index.
  static __device__ __forceinline__ u64 entry(float x, int index) { return static_cast<u64>(logit_key(x)) << 32 | static_cast<uint32_t>(~index); }
  static __device__ __forceinline__ float entry_logit(u64 e) { return key_logit(static_cast<uint32_t>(e >> 32)); }
  static __device__ __forceinline__ int entry_index(u64 e) { return static_cast<int>(~static_cast<uint32_t>(e)); }

  // Into the block's list, in any order: it is sorted later.
  __device__ __forceinline__ void list_add(float v, int index) {
    const int place = atomicAdd(&sh.listed, 1);
    if (place < kList) sh.list[place] = entry(v, index);
  }
  // All blocks' lists in block 0's, and their length in every block; more than kList: not gathered.  box: the lists' lengths.
  __device__ __forceinline__ int gather_list(const u64* box) {
    const int total = static_cast<int>(sum_of(box));
    if (ctas > 1 && total <= kList && rank == 0 && warp > 0 && warp < ctas) {
      int to = 0;
      for (int r = 0; r < warp; ++r) to += static_cast<int>(box[r]);
      const int c = static_cast<int>(box[warp]);
      for (int i = lane; i < c; i += 32) sh.list[to + i] = load_remote64(&sh.list[i], warp);
    }
    return total;
  }
  // Sorts the first `count` keys of this block's list, falling; they are all different.
  __device__ __forceinline__ void sort_list(int count) {
    __syncthreads();
    if (count <= kThreads && count <= kCounted) {
      // a key's place is the number of larger ones
      const u64 mine = t < count ? sh.list[t] : 0;
      int place = 0;
      if (warp * 32 < count) {
#pragma unroll 4
        for (int j = 0; j < count; ++j) place += sh.list[j] > mine;
      }
      __syncthreads();
      if (t < count) sh.list[place] = mine;
      __syncthreads();
      return;
    }
    int size = 2;
    while (size < count) size *= 2;
    for (int i = count + t; i < size; i += kThreads) sh.list[i] = 0;
    __syncthreads();
    for (int k = 2; k <= size; k *= 2)
      for (int j = k / 2; j > 0; j /= 2) {
        for (int p = t; p < size / 2; p += kThreads) {
          const int i = 2 * p - (p & (j - 1)), o = i + j;
          const u64 u = sh.list[i], v = sh.list[o];
          if ((u < v) == ((i & k) == 0)) {
            sh.list[i] = v;
            sh.list[o] = u;
          }
        }
        __syncthreads();
      }
  }
  // Running sums over the block of kEach numbers to a thread, those of entries kEach t and on: v becomes the sum up to and with itself.
  __device__ __forceinline__ void scan_list(u64 (&v)[kEach]) {
#pragma unroll
    for (int j = 1; j < kEach; ++j) v[j] += v[j - 1];
    const u64 before = block_scan(v[kEach - 1]) - v[kEach - 1];
#pragma unroll
    for (int j = 0; j < kEach; ++j) v[j] += before;
  }

  // The first entry at which the running sum of f over the row exceeds `target`, as (index + 1) << 32 | logit; sh.sums has the warps'
  // sums of f, box those of the blocks.
  template <class F>
  __device__ __forceinline__ u64 locate(F f, u64 target, const u64* box) {
    u64 here = 0;
    for (int r = 0; r < rank; ++r) here += box[r];
    if (t == 0) sh.word[1] = 0;
    __syncthreads();
    if (here <= target && target < here + box[rank]) {       // (the same for the whole block)
      int w = 0;
      while (target >= here + sh.sums[w]) here += sh.sums[w++];
      // this warp's pieces, by all threads of the block
      const int end = min((w + 1) * each, pieces);
      for (int p0 = w * each; p0 < end; p0 += kThreads) {
        const int p = p0 + t;
        float v[kPer];
        u64 g[kPer], sum = 0;
        if (p < end) {
          load(p, v);
          limit(p, v);
        }
#pragma unroll
        for (int q = 0; q < kPer; ++q) {
          g[q] = p < end ? f(v[q], base + p * kPer + q - off) : 0;
          sum += g[q];
        }
        const u64 upto = here + block_scan(sum);
        u64 run = upto - sum;
        if (run <= target && target < upto) {
#pragma unroll
          for (int q = 0; q < kPer; ++q) {
            if (run <= target && target < run + g[q])
              sh.word[1] = static_cast<u64>(base + p * kPer + q - off + 1) << 32 | __float_as_uint(v[q]);
            run += g[q];
          }
        }
        __syncthreads();
        here += block_total();
        if (sh.word[1] != 0) break;
      }
    }
    __syncthreads();
    const u64* found = exchange(sh.word[1]);
    u64 r = 0;
    for (int i = 0; i < ctas; ++i) r |= found[i];
    return r;
  }
  // What the last block_scan has summed in all.
  __device__ __forceinline__ u64 block_total() const {
    const u64* part = reinterpret_cast<const u64*>(sh.scan);
    u64 s = 0;
    for (int w = 0; w < kWarps; ++w) s += part[w];
    return s;
  }

  // The last entry that a filter keeps, by the digits of its key: of the entries with `in`, by their number (`want` of them) or by their
  // mass (the first at which it reaches `want`).
  template <class In>
  __device__ __noinline__ void find_by_digits(const Weigh& w, In in, bool by_mass, u64 want, float& tx, int& ti) {
    uint32_t prefix = 0, mask = 0;
    u64 ties = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      sync();
      if (t < 256) {
        sh.digit.mass[t] = 0;
        sh.digit.count[t] = 0;
      }
      __syncthreads();
      for_each([&](float v, int i) {
        const uint32_t k = logit_key(v);
        if (!in(v, i) || (k & mask) != prefix) return;
        const int d = (k >> shift) & 255;
        atomicAdd(&sh.digit.count[d], 1u);
        if (by_mass) atomicAdd(&sh.digit.mass[d], w.weight(v));
      });
      sync();
      u64 mass = 0, count = 0;
      if (t < 256)
        for (int r = 0; r < ctas; ++r) {
          mass += load_remote64(&sh.digit.mass[t], r);
          count += load_remote32(&sh.digit.count[t], r);
        }
      sync();
      if (t < 256) {
        sh.digit.mass[t] = by_mass ? mass : count;
        sh.digit.count[t] = static_cast<uint32_t>(count);
      }
      __syncthreads();
      if (t == 0) {
        int d = 255;
        u64 left = want;
        while (d > 0 && sh.digit.mass[d] < left) left -= sh.digit.mass[d--];
        sh.number[0] = d;
        sh.word[1] = left;
        sh.word[2] = sh.digit.count[d];
      }
      __syncthreads();
      prefix |= static_cast<uint32_t>(sh.number[0]) << shift;
      want = sh.word[1];
      ties = sh.word[2];
      mask |= 255u << shift;
    }
    tx = key_logit(prefix);
    if (by_mass) {
      const u64 one = w.weight(tx);
      want = one > 0 ? (want + one - 1) / one : 1;
    }
    want = want < 1 ? 1 : want > ties ? ties : want;
    // the want-th of the equal ones
    const float x0 = tx;
    auto tie = [&](float v, int i) -> u64 { return v == x0 && in(v, i); };
    u64 s = 0;
    for_each([&](float v, int i) { s += tie(v, i); });
    s = warp_sum(s);
    __syncthreads();
    if (lane == 0) sh.sums[warp] = s;
    __syncthreads();
    const u64* box = exchange(block_sum(t < kWarps ? sh.sums[t] : 0));
    ti = static_cast<int>(locate(tie, want - 1, box) >> 32) - 1;
  }
};

template <class T, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) sample_kernel(const __grid_constant__ cpmtp_sample_args a, int ctas, int span, int bits, int* dev_status) {
  extern __shared__ __align__(16) uint8_t smem[];
  constexpr int kThreads = THREADS, kWarps = THREADS / 32;
  Shared<THREADS>& sh = *reinterpret_cast<Shared<THREADS>*>(smem);
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int rank = static_cast<int>(blockIdx.x) % ctas, row = static_cast<int>(blockIdx.x) / ctas;
  cluster::tell_begun(ctas);
  // between one and two, while nothing else can be done
  for (int i = t; i < kTable; i += kThreads) sh.table[i] = static_cast<u64>(exp2(static_cast<double>(i) / kTable) * 4611686018427387904.0);
  ptx::grid_dep_wait();
  using R_t = Row<T, THREADS>;
  constexpr int kPer = R_t::kPer, kEach = R_t::kEach;
  const T* src = static_cast<const T*>(a.logits) + row * a.ld;
  R_t R{sh, ctas, rank, t, lane, warp, 0, 0, 0, 0, 1, nullptr, 0};
  R.base = min(rank * span, a.V);
  R.n = min(span, a.V - R.base);
  const uintptr_t first = reinterpret_cast<uintptr_t>(src + R.base);
  R.off = static_cast<int>(first & 15) / static_cast<int>(sizeof(T));
  R.pieces = R.n > 0 ? (R.off + R.n + kPer - 1) / kPer : 0;
  R.each = max(1, (R.pieces + kWarps - 1) / kWarps);
  const Settings set = settings_of(a, row);
  const int given = a.given != nullptr ? a.given[row] : CPMTP_EMBED_PAD;
  const float u = a.uniform[row];
  const bool writer = rank == 0 && t == 0;
  float x_given = -INFINITY;
  if (writer && given >= 0 && given < a.V) x_given = io::to_f(src[given]);

  // ---- the entries, and the largest
  float mine_top = -INFINITY;                // of this thread's pieces ...
  int top_at = 0;                            // ... and the first that has it
  {
    const uint4* from = reinterpret_cast<const uint4*>(first & ~static_cast<uintptr_t>(15));
    R.data = from;
    constexpr int kAhead = 8;
    for (int p0 = t; p0 < R.pieces; p0 += kAhead * kThreads) {
      uint4 raw[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (p0 + j * kThreads < R.pieces) raw[j] = __ldg(from + p0 + j * kThreads);
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int p = p0 + j * kThreads;
        if (p >= R.pieces) break;
        float v[kPer];
        R.unpack(raw[j], v);
        if (p == 0 || p + 1 == R.pieces) R.limit(p, v);
        float most = v[0];
#pragma unroll
        for (int q = 1; q < kPer; ++q) most = fmaxf(most, v[q]);     // (which passes over NaN)
        if (most > mine_top) {
          mine_top = most;
          top_at = p;
        }
      }
    }
  }
  float top = mine_top;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  float* tops = reinterpret_cast<float*>(sh.sums);
  if (lane == 0) tops[warp] = top;
  __syncthreads();
  top = tops[lane & (kWarps - 1)];
#pragma unroll
  for (int o = kWarps / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  cluster::await_begun(ctas);                // (told before the table, so the pass has covered the wait)
  {
    const u64* box = R.exchange(__float_as_uint(top));
    for (int r = 0; r < ctas; ++r) top = fmaxf(top, __uint_as_float(static_cast<uint32_t>(box[r])));
  }
  if (writer && given != CPMTP_EMBED_PAD && (given < 0 || given >= a.V) && dev_status != nullptr) atomicMax(dev_status, 1);
  auto answer = [&](int token, float logp, int kept, float logp_given) {
    if (!writer) return;
    a.tokens[row] = token;
    if (a.logp != nullptr) a.logp[row] = logp;
    if (a.kept != nullptr) a.kept[row] = kept;
    if (a.given != nullptr) a.logp_given[row] = logp_given;
  };
  if (!(top > -INFINITY)) {
    answer(-1, -INFINITY, 0, -INFINITY);
    return;                                  // (the same in every block of the cluster, after its barrier)
  }
  if (set.one) {
    // the first of the largest
    int at = __reduce_min_sync(0xffffffffu, mine_top == top ? top_at : INT_MAX);
    int* places = reinterpret_cast<int*>(sh.scan);
    if (lane == 0) places[warp] = at;
    __syncthreads();
    at = __reduce_min_sync(0xffffffffu, places[lane & (kWarps - 1)]);
    u64 index = ~0ull;
    if (at != INT_MAX) {
      float v[kPer];
      R.load(at, v);
      R.limit(at, v);
#pragma unroll
      for (int q = kPer - 1; q >= 0; --q)
        if (v[q] == top) index = R.base + at * kPer + q - R.off;
    }
    const u64* box = R.exchange(index);
    for (int r = 0; r < ctas; ++r) index = min(index, box[r]);
    const int token = static_cast<int>(index);
    answer(token, 0.f, 1, given == token ? 0.f : -INFINITY);
    return;
  }
  Weigh w;
  w.set(top, set.inv_t, bits);
  w.table = ptx::smem_u32(sh.table);
  const double unit = static_cast<double>(1ull << bits);
  const long long z_least = set.min_p > 0.0 ? static_cast<long long>(ceil(log2(set.min_p) * 4294967296.0)) : -(1ll << 62);
  const Fixed z_min{static_cast<int>(z_least >> 32), static_cast<uint32_t>(z_least)};
  auto target_of = [&](u64 total) {
    return u > 0.f ? (u < 1.f ? min(static_cast<u64>(static_cast<double>(u) * static_cast<double>(total)), total - 1) : total - 1) : 0;
  };
  auto finish = [&](int token, float x_token, u64 total, int kept, float tx, int ti) {
    if (!writer || token < 0) return;
    const double all = log(static_cast<double>(total) / unit);
    // (a temperature of a row's own may be infinite: its inverse is 0)
    auto logp = [&](float v) {
      return static_cast<float>((v >= w.x_max ? 0.0 : top > w.x_max ? -INFINITY : (static_cast<double>(v) - static_cast<double>(top)) * set.inv_t) - all);
    };
    const bool in = x_given > -INFINITY && (x_given > tx || (x_given == tx && given <= ti)) && at_least(w.z(x_given), z_min);
    answer(token, logp(x_token), kept, in ? logp(x_given) : -INFINITY);
  };

  // ---- entries x > tx, and x == tx up to index ti, are kept
  float tx = -INFINITY;
  int ti = INT_MIN;                          // (nothing: places before a piece's first entry have negative numbers)
  auto kept_by = [&](float v, int i) { return (v > tx) | ((v == tx) & (i <= ti)); };

  // (of copies: what a function that is not inlined has the address of lives in memory)
  auto by_digits = [&](auto in, bool by_mass, u64 want) {
    R_t row_copy = R;
    const Weigh w_copy = w;
    float x;
    int i;
    row_copy.find_by_digits(w_copy, in, by_mass, want, x, i);
    R.boxes = row_copy.boxes;
    tx = x;
    ti = i;
  };

  // ---- top-k
  if (set.top_k < a.V) {
    bool found = false;
    u64 valid = 0;
    if (top < INFINITY) {
      // bins of 1/64 in units of ln 2 of the logits themselves; the magic number rounds to integers
      const float step = 64.f * 1.4426950408889634f;
      auto bin_of = [&](float v) { return __float_as_uint(fminf(fmaf(top - v, step, 8388608.f), 8388608.f + (kBins - 1))) & 0x7fffffu; };
      // At first the threads' largest entries stand for all: down to the bin of the top_k-th of them there are as many entries or more, but not many more
      // unless nearly all threads are needed.  Their list is enough, or too long; then all entries are counted.  (512 x 128256 with k = 50: 113 us, and
      // 160 with all entries counted at once.)
#pragma unroll 1
      for (int counted = 8ll * set.top_k > 7ll * kThreads * ctas; counted < 2 && !found; ++counted) {
        R.clear_hist();
        if (counted) {
          R.for_each([&](float v, int) {
            if (v > -INFINITY) atomicAdd(&sh.hist[bin_of(v)], 1u);
          });
        } else if (mine_top > -INFINITY) {
          atomicAdd(&sh.hist[bin_of(mine_top)], 1u);
        }
        int b, b2;
        double before;
        valid = static_cast<u64>(R.find_bins([](int) { return 1.0; }, set.top_k, set.top_k, INFINITY, -INFINITY, b, b2, before));
        if (counted ? static_cast<u64>(set.top_k) >= valid : static_cast<u64>(set.top_k) > valid || b == kBins - 1) continue;
        // all entries down to that bin, if they are few; else those of the bin
        const bool all = !counted || (before + kList / 2 <= kList && b < kBins - 1);
        if (all) {
          // (by a border that is half a bin lower); from the pieces of the threads that have any, where these are few: 512 x 128256 with k = 50
          // 113 us, and 134 from all pieces, but 2000 x 32000 with k = 450 241 and 232
          const float least = fmaxf(nextafterf(__double2float_rd(static_cast<double>(top) - (b + 1) / static_cast<double>(step)), -INFINITY), -FLT_MAX);
          int* who = reinterpret_cast<int*>(sh.hist);
          if (t == 0) sh.number[2] = 0;
          __syncthreads();
          if (mine_top >= least) who[atomicAdd(&sh.number[2], 1)] = t;
          __syncthreads();
          const bool few = sh.number[2] <= kThreads / 4;
          const int of_thread = (R.pieces + kThreads - 1) / kThreads, items = few ? sh.number[2] * of_thread : R.pieces;
          constexpr int kAhead = 4;
          for (int i0 = t; i0 < items; i0 += kAhead * kThreads) {
            int p[kAhead];
            uint4 raw[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
              const int i = i0 + j * kThreads;
              p[j] = i >= items ? INT_MAX : few ? who[i / of_thread] + i % of_thread * kThreads : i;
              if (p[j] < R.pieces) raw[j] = __ldg(R.data + p[j]);
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
              if (p[j] >= R.pieces) continue;
              float v[kPer];
              R.unpack(raw[j], v);
              if (p[j] == 0 || p[j] + 1 == R.pieces) R.limit(p[j], v);
              bool some = false;
#pragma unroll
              for (int q = 0; q < kPer; ++q) some |= v[q] >= least;
              if (!some) continue;
#pragma unroll
              for (int q = 0; q < kPer; ++q)
                if (v[q] >= least) R.list_add(v[q], R.base + p[j] * kPer + q - R.off);
            }
          }
        } else {
          R.for_each([&](float v, int i) {
            if (bin_of(v) == static_cast<uint32_t>(b) && v > -INFINITY) R.list_add(v, i);
          });
        }
        __syncthreads();
        const int count = R.gather_list(R.exchange(sh.listed));
        if (count <= kList && all) {
          // the rest is block 0's alone
          R.sync();
          if (rank != 0) return;
          R.sort_list(count);
          u64 v[kEach], own[kEach];
          Fixed z[kEach];
#pragma unroll
          for (int j = 0; j < kEach; ++j) {
            const int i = kEach * t + j;
            z[j] = w.z(i < set.top_k ? R.entry_logit(sh.list[i]) : top);
            own[j] = v[j] = i < set.top_k ? w.weight(z[j]) : 0;
          }
          R.scan_list(v);
          const double border = set.top_p * static_cast<double>(R.block_total());
          u64 left = 0;
#pragma unroll
          for (int j = 0; j < kEach; ++j) {
            const int i = kEach * t + j;
            left += i < set.top_k && (set.top_p >= 1.0 || i == 0 || static_cast<double>(v[j] - own[j]) < border) && at_least(z[j], z_min);
          }
          const int kept = static_cast<int>(R.block_sum(left));
          if (kept - 1 >= kEach * t && kept - 1 < kEach * (t + 1)) {
#pragma unroll
            for (int j = 0; j < kEach; ++j)
              if (kept - 1 == kEach * t + j) sh.word[2] = v[j];
          }
          __syncthreads();
          const u64 total = sh.word[2], last = sh.list[kept - 1];
          // by index: the keys' halves change places (and fall, so the index is inverted as it stands)
          __syncthreads();
          for (int i = t; i < kept; i += kThreads) sh.list[i] = sh.list[i] << 32 | sh.list[i] >> 32;
          R.sort_list(kept);
#pragma unroll
          for (int j = 0; j < kEach; ++j) {
            const int i = kEach * t + j;
            own[j] = v[j] = i < kept ? w.weight(key_logit(static_cast<uint32_t>(sh.list[i]))) : 0;
          }
          R.scan_list(v);
          const u64 target = target_of(total);
#pragma unroll
          for (int j = 0; j < kEach; ++j)
            if (v[j] > target && v[j] - own[j] <= target) sh.word[3] = sh.list[kEach * t + j];
          __syncthreads();
          finish(static_cast<int>(~static_cast<uint32_t>(sh.word[3] >> 32)), key_logit(static_cast<uint32_t>(sh.word[3])), total, kept,
                 R.entry_logit(last), R.entry_index(last));
          return;
        }
        if (count <= kList) {
          const int nth = set.top_k - static_cast<int>(before) - 1;          // of the bin's entries, the last that is kept
          if (rank == 0) {
            R.sort_list(count);
            if (t < ctas) store_remote(&sh.word[2], t, sh.list[nth]);
          }
          R.sync();
          tx = R.entry_logit(sh.word[2]);
          ti = R.entry_index(sh.word[2]);
          found = true;
        }
      }
    } else {
      R.for_each([&](float v, int) { valid += v > -INFINITY; });
      valid = R.row_sum(valid);
    }
    if (!found && static_cast<u64>(set.top_k) < valid) by_digits([](float v, int) { return v > -INFINITY; }, false, set.top_k);
  }

  const bool floor = tx > -INFINITY;         // (without one the passes ask for less)

  // ---- top-p, and the kept mass of every warp's range
  u64 sum = 0;
  uint32_t number = 0;
  bool counted = false;
  if (set.top_p < 1.0) {
    const int less = max(0, 32 - __clz(span - 1) - 14);                    // bits that the histogram's sums have to do without
    u64 mass = 0;
    R.clear_hist();
    auto measure = [&](float v, bool in) {
      const Fixed z = w.z(v);
      const u64 q = w.mantissa(z);
      mass += only_if(in, w.fixed(q, z));
      // (an entry of bin b has -b <= 64 z < 1 - b; one that is not kept adds nothing to its bin)
      const int bin = min(-(z.whole * 64 + static_cast<int>(z.part >> 26)), kBins - 1);
      atomicAdd(&sh.hist[bin & (kBins - 1)], in ? static_cast<uint32_t>(q >> 32) >> (13 + less) : 0u);
    };
    if (floor) R.for_each([&](float v, int i) { measure(v, kept_by(v, i)); });
    else R.for_each([&](float v, int) { measure(v, v > -INFINITY); });
    mass = R.row_sum(mass);
    const double border = set.top_p * static_cast<double>(mass);
    bool found = false;
    {
      // An entry of bin b has floor(z) = -ceil(b / 64).  A sum is short by 2^(less - 17) of itself at most, which bounds what lies before a border and
      // what lies behind it: with top_p near one that is little, and so is then the doubt.  (A border by what lies before it alone: a row with
      // top_p = 0.9996 took 140 us, a list too long.)  The last bin, where smaller weights are too, has no sum.
      const double one = unit * ldexp(1.0, less - 17), slack = ldexp(1.0, less - 15), behind = static_cast<double>(mass) - border;
      const double tiny = ldexp(static_cast<double>(mass), -45), least = static_cast<double>(a.V) * unit * ldexp(1.0, -31);
      int b1, b2;
      double before;
      R.find_bins([&](int b) { return b == kBins - 1 ? 0.0 : one * exp2f(static_cast<float>(-((b + 63) >> 6))); }, border * (1.0 - slack), border * (1.0 + slack),
                  behind + tiny, (behind - least) * (1.0 - slack) - tiny, b1, b2, before);
      // Entries above xa lie in bins before b1, those below xb in bins behind b2; the bins' edges, rounded outwards.
      const float xa = nextafterf(__double2float_ru(w.m - (b1 - 1) / (64.0 * w.c)), INFINITY);
      // (-infinity, which stands for what is not kept, must not reach xb)
      const float xb = b2 == kBins - 1 ? -FLT_MAX : fmaxf(nextafterf(__double2float_rd(w.m - b2 / (64.0 * w.c)), -INFINITY), -FLT_MAX);
      u64 above = 0;
      // few entries are that large: a warp collects them, and weighs 32 at a time
      float* queue = sh.queue[warp];
      const uint32_t below = (1u << lane) - 1, queue_at = ptx::smem_u32(queue);
      int queued = 0;
      auto weigh = [&](float v, bool on) {
        const Fixed z = w.z(v);
        const u64 q = only_if(on, w.weight(z));
        const bool in = on & at_least(z, z_min);
        above += q;
        sum += only_if(in, q);
        number += in;
      };
      R.for_pieces([&](int p, const float (&v)[kPer]) {
        uint32_t to_list = 0;
#pragma unroll
        for (int q = 0; q < kPer; ++q) {
          bool in = v[q] >= xb;
          if (floor) in &= kept_by(v[q], R.base + p * kPer + q - R.off);
          const bool over = in & (v[q] > xa);
          const uint32_t lanes = __ballot_sync(0xffffffffu, over);
          // (a store under a predicate: the compiler would branch)
          asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %0, 0;\n\t@p st.shared.f32 [%1], %2;\n\t}" ::"r"(static_cast<int>(over)),
                       "r"(queue_at + 4 * (queued + __popc(lanes & below))), "f"(v[q]) : "memory");
          queued += __popc(lanes);
          to_list |= static_cast<uint32_t>(in & !over) << q;
        }
        if (to_list != 0) {
#pragma unroll
          for (int q = 0; q < kPer; ++q)
            if (to_list >> q & 1) R.list_add(v[q], R.base + p * kPer + q - R.off);
        }
        __syncwarp();
        int done = 0;
        for (; queued - done >= 32; done += 32) weigh(queue[done + lane], true);
        if (done > 0) {
          const float rest = lane < queued - done ? queue[done + lane] : 0.f;
          __syncwarp();
          queue[lane] = rest;
          queued -= done;
        }
        __syncwarp();
      });
      weigh(lane < queued ? queue[lane] : top, lane < queued);
      above = R.block_sum(above);
      const int mine = sh.listed;
      const u64* box = R.exchange(above, mine);
      above = R.sum_of(box);
      const int count = R.gather_list(box + kMostCtas);
      if (count <= kList) {
        if (rank == 0) {
          // (its own entries stay in the list: their shares are found by index)
          R.sort_list(count);
          u64 v[kEach], own[kEach];
#pragma unroll
          for (int j = 0; j < kEach; ++j) own[j] = v[j] = kEach * t + j < count ? w.weight(R.entry_logit(sh.list[kEach * t + j])) : 0;
          R.scan_list(v);
          u64 left = 0;
          bool reached = false;
#pragma unroll
          for (int j = 0; j < kEach; ++j) {
            left += kEach * t + j < count && static_cast<double>(above + v[j] - own[j]) < border;
            reached |= kEach * t + j < count && static_cast<double>(above + v[j]) >= border;
          }
          const int kept = static_cast<int>(R.block_sum(left));
          reached = __syncthreads_or(reached);
          // the border has to lie among these entries, as the histogram said; 0: it does not
          const u64 last = kept > 0 && (reached || b2 == kBins - 1) ? sh.list[kept - 1] : 0;
          if (t < ctas) store_remote(&sh.word[2], t, last);
        }
        R.sync();
        const u64 last = sh.word[2];
        if (last != 0) {
          found = counted = true;
          tx = R.entry_logit(last);
          ti = R.entry_index(last);
          // the listed entries that are kept, to the sums of the ranges they lie in
          sum = R.warp_sum(sum);
          if (lane == 0) sh.sums[warp] = sum;
          __syncthreads();
          for (int i = t; i < (rank == 0 ? count : mine); i += kThreads) {
            const u64 e = sh.list[i];
            const int index = R.entry_index(e);
            if (e < last || index < R.base || index >= R.base + R.n) continue;
            const Fixed z = w.z(R.entry_logit(e));
            if (!at_least(z, z_min)) continue;
            ++number;
            atomicAdd(&sh.sums[R.warp_of(index)], w.weight(z));
          }
        }
      }
    }
    if (!found) {
      const float x1 = tx;
      const int i1 = ti;
      sum = number = 0;
      by_digits([=](float v, int i) { return v > x1 || (v == x1 && i <= i1); }, true, max(1ull, static_cast<u64>(ceil(border))));
    }
  }
  auto drawn = [&](float v, int i) -> u64 {
    const Fixed z = w.z(v);
    return only_if(kept_by(v, i) & at_least(z, z_min), w.weight(z));
  };
  if (!counted) {
    if ((tx > -INFINITY) | (set.min_p > 0.0)) {
      R.for_each([&](float v, int i) {
        const Fixed z = w.z(v);
        const bool in = kept_by(v, i) & at_least(z, z_min);
        sum += only_if(in, w.weight(z));
        number += in;
      });
    } else {
      R.for_each([&](float v, int) {
        const bool in = v > -INFINITY;
        sum += only_if(in, w.weight(v));
        number += in;
      });
    }
    sum = R.warp_sum(sum);
    __syncthreads();
    if (lane == 0) sh.sums[warp] = sum;
  }
  const u64 numbers = R.block_sum(number);             // (a barrier: the warps' sums are complete)
  const u64 here = R.block_sum(t < kWarps ? sh.sums[t] : 0);
  const u64* box = R.exchange(here, numbers);
  const u64 total = R.sum_of(box);
  const int kept = static_cast<int>(R.sum_of(box + kMostCtas));
  const u64 token = R.locate(drawn, target_of(total), box);
  finish(static_cast<int>(token >> 32) - 1, __uint_as_float(static_cast<uint32_t>(token)), total, kept, tx, ti);
}

}  // namespace sample
}  // namespace cpmtp
