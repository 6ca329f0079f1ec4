// Attention of a few new tokens over the paged cache.
//
//   s_i = scale <q, k_i>,  p = softmax(s),  out = sum_i p_i v_i
//
// Every key and value is read once and used for a few rows only (the new tokens times the query heads that share a head of the
// cache), so the time is that of reading the cache.  The products run on the tensor cores with the cache's tile as the operand of
// 128 rows and the queries as the narrow one:
//   S^T [128 slots, NT rows] = K_tile [128, D] Q^T,   O^T [D, 2 NT] = V_tile^T [D, 128] [P_high; P_low]^T
// in TMEM: a lane is a slot in the first and a column of the head in the second, and nothing is padded to 128 but D.  A product this
// narrow takes the time of reading its wide operand from shared memory, so the low parts of the weights ride along.
//
// The tiles of 128 slots of all (sequence, head, chunk of NT rows) form one list, which is cut into equal shares, one for each
// SM, whatever the lengths.  A share that ends inside a unit leaves (max, sum, unnormalised out) behind; join_kernel joins them.
//
//   warps 0, 1   TMA: pages into a ring of K tiles and one of V tiles, a warp to each
//   warp 2       tcgen05.mma: S of tile g, then O of tile g - 1
//   warp 3       queries of the next unit into shared memory
//   warps 4-11   two groups of 128 threads, half of the rows to each: a thread is a slot and makes its weights, then a column and
//                sums O in registers
//
// What bounds it (times in captured graphs): bandwidth where there is enough to read (32 sequences of 8192 slots, 8 heads of 128 for 32 queries, 1.07 GB: 161 to 171 us in pages of 32
// slots and more, 6.3 to 6.7 TB/s); the start, the last tiles and the joining, 11 us in all, where there are few tiles for each SM.  Pages of 16 and 8
// slots take 180 to 192 and 235 us: a TMA box costs its warp the same whatever it holds.  (A second warp to each ring: pages of 8 201 us, but 240 against
// 238 for 64 ragged sequences and 63 against 62 with acc.)  Heads of 64 take 114 us (131 where heads lie within slots) for half the bytes: a tile costs its products, barriers and weights.
// Heads of 80 take 122 us, but 210 where heads lie within slots: rows of 160 bytes, 1280 apart, are fetched in pieces of 256.  Rows above 32 read the cache again, and every chunk of rows
// all tiles of its sequence: 8 tokens 177 us, 16 355, 64 1456; four prompts of 2048 tokens over their own slots 2147, 84 of which are operations.
#pragma once
#include <cuda.h>

#include <cfloat>
#include <climits>

#include "cache_kernels.cuh"

namespace cpmtp {
namespace attend {

using io::bf16_t;

constexpr int kTile = 128;                  // slots of a tile
constexpr int kThreads = 12 * 32;
constexpr int kHalfBytes = kTile * 128;     // 128 slots of 64 columns
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNone = -FLT_MAX;           // the reference of a row that has seen nothing yet; no finite score lies below it
// The reference that weights are taken relative to follows the running maximum only when that has risen by so much (a factor of
// 256 in the weights, which costs neither fp32 nor bf16 a digit): nearly every tile then leaves the sums as they are.
constexpr float kSlack = 8.f;

struct Params {
  cpmtp_cache c;
  cpmtp_cache_seqs s;
  cpmtp_attend_args a;
  int G;                       // query heads that share a head of the cache
  int chunks;                  // chunks of NT rows that Q new tokens make
  int piece;                   // slots that one TMA box covers: they lie in one page, and pieces tile a tile
  int halves, ksteps;          // 64-column halves and 16-column steps of a head
  int k_slots, v_slots;        // tiles of the two rings
  int tiles;                   // most tiles of a sequence
  int ctas;                    // of the launch
  int q_vec;                   // queries can be read 16 bytes at a time
  float scale2;                // scale * log2(e)
  float* part_o;               // [CTA][2][NT][128]
  float2* part_ml;             // [CTA][2][NT] reference and sum
  int2* unit_ctas;             // [B][H][chunks] first and last CTA
  float2* whole_ml;            // [B][H][chunks][NT]; with acc
  float* scores;               // [B][H][chunks][tiles][NT][128] scores in log2 units; with acc
  unsigned wait_limit_us;
  int test_skip_load;
};

// ------------------------------------------------------------------------------------------ shares of the work
struct Seq {
  int len, fresh, tiles, units;
};
__device__ __forceinline__ Seq make_seq(const Params& p, int len, int fresh, int nt) {
  Seq q;
  q.len = min(max(len, 0), p.s.width * p.c.page_slots);
  q.fresh = min(max(fresh, 0), p.s.Q);
  q.tiles = max(1, (q.len + kTile - 1) / kTile);
  q.units = p.c.H * ((q.fresh * p.G + nt - 1) / nt);
  return q;
}
__device__ __forceinline__ int raw_new(const Params& p, int b) { return p.s.q_lens != nullptr ? p.s.q_lens[b] : p.s.Q; }

struct Start {
  int b, u, t, first, left, total, ctas;
};

// A place in the list: tile t of unit u of sequence b.  The next sequence's numbers are read ahead.
struct Walk {
  Seq q;
  int b, u, t, left, nt;
  int next_len, next_new;
  __device__ __forceinline__ void fetch(const Params& p) {
    const int n = min(b + 1, p.s.B - 1);
    next_len = p.s.lens[n];
    next_new = raw_new(p, n);
  }
  __device__ __forceinline__ Walk(const Params& p, const Start& s, int nt_) : b(s.b), u(s.u), t(s.t), left(s.left), nt(nt_) {
    if (left == 0) return;
    q = make_seq(p, p.s.lens[b], raw_new(p, b), nt);
    fetch(p);
  }
  __device__ __forceinline__ int piece_end() const { return min(q.tiles, t + left); }
  // To the first tile of the next unit, `done` tiles further.
  __device__ __forceinline__ void next_unit(const Params& p, int done) {
    left -= done;
    if (left == 0) return;
    t = 0;
    if (++u < q.units) return;
    u = 0;
    do {
      if (++b >= p.s.B) {            // (only if the lengths change under the kernel)
        left = 0;
        return;
      }
      q = make_seq(p, next_len, next_new, nt);
      fetch(p);
    } while (q.units == 0);
  }
  __device__ __forceinline__ void next_tile(const Params& p) {
    if (t + 1 < q.tiles) {
      ++t;
      --left;
    } else {
      next_unit(p, 1);
    }
  }
};

// Where this CTA's share begins: every thread adds up a run of sequences.
__device__ __forceinline__ void find_start(const Params& p, int nt, int* sh_warp, Start* sh, int* dev_status) {
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int per = (p.s.B + kThreads - 1) / kThreads;
  const int b0 = min(t * per, p.s.B), b1 = min(b0 + per, p.s.B);
  int mine = 0;
  for (int b = b0; b < b1; ++b) {
    const int len = p.s.lens[b], fresh = raw_new(p, b);
    const Seq q = make_seq(p, len, fresh, nt);
    if (blockIdx.x == 0 && (q.len != len || q.fresh != fresh)) cache::raise_status(dev_status, cache::kBadIndex);
    mine += q.units * q.tiles;
  }
  int upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 31) sh_warp[warp] = upto;
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) upto += sh_warp[w];
    total += sh_warp[w];
  }
  const int ctas = min(static_cast<int>(gridDim.x), total), c = blockIdx.x;
  const int begin = c < ctas ? static_cast<int>(static_cast<long long>(c) * total / ctas) : 0;
  const int end = c < ctas ? static_cast<int>(static_cast<long long>(c + 1) * total / ctas) : 0;
  if (t == 0 && end == begin) *sh = Start{0, 0, 0, 0, 0, total, ctas};
  int at = upto - mine;
  if (end > begin && at <= begin && begin < upto) {
    for (int b = b0; b < b1; ++b) {
      const Seq q = make_seq(p, p.s.lens[b], raw_new(p, b), nt);
      const int n = q.units * q.tiles;
      if (begin < at + n) {
        *sh = Start{b, (begin - at) / q.tiles, (begin - at) % q.tiles, begin, end - begin, total, ctas};
        break;
      }
      at += n;
    }
  }
  __syncthreads();
}
// The CTA that has the i-th tile of the list.
__device__ __forceinline__ int cta_of(const Start& s, int i) {
  return static_cast<int>((static_cast<long long>(i + 1) * s.ctas - 1) / s.total);
}

// ------------------------------------------------------------------------------------------ shared memory
template <int NT>
struct Layout {
  static constexpr int kQ = NT * 256;                // queries of a unit: two halves of NT rows of 128 bytes
  static constexpr int kP = 2 * NT * 256;            // weights of a tile: 128 slots of NT rows, bf16, high and low parts
  static constexpr int kBars = 512;
  static constexpr int kRows = NT / 2;               // of a group
  static constexpr int kGroup = 11 * kRows;          // words of a group's small arrays
  static constexpr int kOdd = 2 * 2 * 128;           // words: of two units, the first slots with infinities of either sign in each column
  static constexpr int kSmall = (2 * kGroup + kOdd) * 4 + 128;
  static constexpr int kFixed = 1024 + 2 * kQ + 2 * kP + kBars + kSmall;
  static constexpr int kTmem = 8 * NT;               // two S accumulators and two O, of the high and the low parts of the weights (6 NT)
};
// Half tiles of both rings.  With 16 columns there is room for twelve (with 32 for ten), but with that much under way memory answers more slowly: 1.07 GB of heads of 128 columns take 168 us
// with six tiles, 161 with five, 160 with four and 180 with three; ragged 1.4 GB in small pages 226 with four and more.
constexpr int kMaxSlots = 10;

// Barriers of a group's 128 threads.
__device__ __forceinline__ bool any_of_group(int group, bool v) {
  int r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.or.aligned.pred q, %2, 128, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
               : "=r"(r) : "r"(static_cast<int>(v)), "r"(group + 1) : "memory");
  return r != 0;
}
__device__ __forceinline__ void group_sync(int group) { asm volatile("barrier.cta.sync.aligned %0, 128;" ::"r"(group + 1) : "memory"); }
// The same number in every lane, and known to be.
__device__ __forceinline__ int uniform(int v) { return __reduce_max_sync(0xffffffffu, v); }
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __reduce_max_sync(0xffffffffu, v); }
__device__ __forceinline__ float warp_max(float v) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const void* tmap, uint32_t bar, int c0, int c1, int c2, int c3, uint64_t policy) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%3, %4, %5, %6}], [%2], %7;"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tmap)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "l"(policy) : "memory");
}
// What is read once is the first to leave L2, so that the scores and parts, which are read again, stay.
__device__ __forceinline__ uint64_t l2_policy(bool once) {
  uint64_t p;
  if (once) asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
  else asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(p));
  return p;
}
__device__ __forceinline__ void tmem_load(uint32_t addr, float (&v)[16]) {
  ptx::tmem_ld_32x16(addr, v);
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]),
                 "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])::"memory");
}
__device__ __forceinline__ void tmem_load(uint32_t addr, float (&v)[8]) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(addr) : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7])::"memory");
}

template <int NT>
__global__ void __launch_bounds__(kThreads, 1) attend_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                                                             const __grid_constant__ Params p, int* dev_status) {
  using L = Layout<NT>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = ptx::smem_u32(smem_raw), pad = (1024u - (raw & 1023u)) & 1023u;
  const uint32_t slot_bytes = p.halves * kHalfBytes;
  // [ring of K][ring of V][queries x 2][weights: two tiles of (high, low)][barriers][small arrays]
  const uint32_t ring = raw + pad, qbuf = ring + (p.k_slots + p.v_slots) * slot_bytes, pbuf = qbuf + 2 * L::kQ, bars = pbuf + 2 * L::kP;
  float* small = reinterpret_cast<float*>(smem_raw + (bars + L::kBars - raw));
  int* odd_sh = reinterpret_cast<int*>(small + 2 * L::kGroup);
  int* misc = odd_sh + L::kOdd;  // [0..11] scan, [12..18] start, [20] TMEM address, [21] abort flag, [22], [23] the groups'
  Start* start_sh = reinterpret_cast<Start*>(misc + 12);
  volatile int* abort_flag = misc + 21;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (kMaxSlots + s); };
  auto bar = [&](int i) { return bars + 8u * (2 * kMaxSlots + i); };
  auto qfull = [&](int s) { return bar(s); };
  auto qfree = [&](int s) { return bar(2 + s); };
  auto pfull = [&](int s) { return bar(4 + s); };
  auto ofull = [&](int s) { return bar(6 + s); };
  auto sfull = [&](int s) { return bar(8 + s); };
  const uint32_t drain = bar(10);
  static_assert(8 * (2 * kMaxSlots + 11) <= L::kBars, "barriers");

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint64_t wait_ns = static_cast<uint64_t>(p.wait_limit_us) * 1000ull;
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.k_slots + p.v_slots; ++s) {
      ptx::mbar_init(full(s), 1);
      ptx::mbar_init(empty(s), 1);
    }
    for (int s = 0; s < 2; ++s) {
      ptx::mbar_init(qfull(s), 32);
      ptx::mbar_init(qfree(s), 1);
      ptx::mbar_init(pfull(s), 8);       // a lane of each of the groups' warps
      ptx::mbar_init(ofull(s), 1);
      ptx::mbar_init(sfull(s), 1);
    }
    ptx::mbar_init(drain, 1);
    misc[21] = misc[22] = misc[23] = 0;
    ptx::fence_mbar_init();
    ptx::prefetch_tmap(&tm_k);
    ptx::prefetch_tmap(&tm_v);
  }
  if (warp == 2) {
    ptx::tmem_alloc(ptx::smem_u32(misc + 20), L::kTmem);
    ptx::tmem_relinquish();
  }
  ptx::grid_dep_wait();
  ptx::tc_fence_before_sync();
  find_start(p, NT, misc, start_sh, dev_status);
  ptx::tc_fence_after_sync();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(misc + 20);
  const Start start = *start_sh;
  Walk w(p, start, NT);

  if (warp < 2) {
    // ------------------------------------------------------------------------------------------ pages into the ring
    const int pieces = kTile / p.piece;
    auto page_at = [&](const Walk& x) {          // the page of this lane's piece of the tile; -1: nothing to load
      const int slot = x.t * kTile + lane * p.piece;
      if (lane >= pieces || slot >= x.q.len) return -1;
      const int page = p.s.table[x.b * p.s.ld_table + slot / p.c.page_slots];
      return page >= 0 && page < p.c.pages ? page : p.c.pages;      // out of range: the box reads as zeros
    };
    // (a ring has one warp that fills it: a second one could be a whole lap ahead, which the parity of a barrier does not tell)
    const int base = warp == 0 ? 0 : p.k_slots, n = warp == 0 ? p.k_slots : p.v_slots;
    const uint64_t policy = l2_policy(p.chunks == 1);      // (another chunk of rows reads the same tiles, at about the same time)
    int it = 0, page = w.left > 0 ? page_at(w) : -1;
    bool alive = true;
    while (w.left > 0 && alive) {
      const int u_chunks = (w.q.fresh * p.G + NT - 1) / NT;
      const int h = w.u / u_chunks, slot = w.t * kTile + lane * p.piece, in_page = slot % p.c.page_slots;
      const int here = page;
      w.next_tile(p);
      if (w.left > 0) page = page_at(w);         // read while this tile's loads are under way
      if (here == p.c.pages) cache::raise_status(dev_status, cache::kBadIndex);
      const uint32_t lanes = __ballot_sync(0xffffffffu, here >= 0);
      const uint32_t bytes = __popc(lanes) * p.piece * 128u * p.halves;
      const int s = base + it % n;
      const bool skip = 2 * it + warp + 1 == p.test_skip_load;
      if (lane == 0) {
        alive = ptx::mbar_wait(empty(s), ((it / n) & 1) ^ 1u, abort_flag, wait_ns);
        if (alive && !skip) {
          if (bytes > 0) ptx::mbar_arrive_expect_tx(full(s), bytes);
          else ptx::mbar_arrive(full(s));
        }
      }
      alive = __shfl_sync(0xffffffffu, alive, 0);
      if (!alive) break;
      if (here >= 0 && !skip) {
        const uint32_t dst = ring + s * slot_bytes + lane * p.piece * 128u;
        for (int half = 0; half < p.halves; ++half) tma_load_4d(dst + half * kHalfBytes, warp == 0 ? &tm_k : &tm_v, full(s), half * 64, in_page, h, here, policy);
      }
      ++it;
    }
    ptx::grid_dep_launch();
    if (lane == 0)               // what was issued has to land before the shared memory is given back
      for (int j = it - 1; j >= 0 && j >= it - n; --j) ptx::mbar_wait(full(base + j % n), (j / n) & 1, abort_flag, wait_ns, false);
  } else if (warp == 2) {
    // ------------------------------------------------------------------------------------------ products
    // The whole warp runs this, in step, with one lane that issues: what the products need is then the same in every lane for the
    // compiler too and stays in uniform registers.  (With one lane alone in a branch a product took 80 clocks to issue.)
    constexpr uint32_t idesc_s = ptx::make_idesc_bf16(128, NT, 0, 0), idesc_o = ptx::make_idesc_bf16(128, 2 * NT, 1, 0);
    const uint32_t one = ptx::elect_one(), d_base = uniform(tmem);
    const uint64_t k_desc = ptx::make_smem_desc_sw128(ring, 16, 1024), q_desc = ptx::make_smem_desc_sw128(qbuf, 16, 1024);
    const uint64_t v_desc = ptx::make_smem_desc_sw128(ring + p.k_slots * slot_bytes, kHalfBytes, 1024), p_desc = ptx::make_smem_desc_sw128(pbuf, 16, 1024);
    int g = 0, unit = 0, ks = 0, vs = 0;
    uint32_t k_phase = 0, v_phase = 0;
    bool alive = true;
    auto ready = [&](uint32_t b, uint32_t phase) {
      if (!ptx::mbar_wait(b, phase & 1u, abort_flag, wait_ns)) alive = false;
      alive = __all_sync(0xffffffffu, alive);
      ptx::tc_fence_after_sync();
    };
    auto second = [&](int k) {                 // O of tile k
      ready(full(p.k_slots + vs), v_phase);
      ready(pfull(k & 1), k >> 1);
      if (!alive) return;
      const uint64_t a = v_desc + vs * (slot_bytes >> 4), w_at = p_desc + (k & 1) * (L::kP >> 4);
      const uint32_t d = d_base + 2 * NT + (k & 1) * 2 * NT;
#pragma unroll
      for (int s = 0; s < 8; ++s) ptx::umma_bf16_if(one, d, a + s * (2048 >> 4), w_at + (((s >> 2) * (2 * NT * 128) + (s & 3) * 32) >> 4), idesc_o, s != 0);
      ptx::umma_commit_if(one, empty(p.k_slots + vs));
      ptx::umma_commit_if(one, ofull(k & 1));
      if (++vs == p.v_slots) {
        vs = 0;
        v_phase ^= 1u;
      }
    };
    int left = uniform(w.left);
    while (left > 0 && alive) {
      const int tiles = uniform(w.piece_end() - w.t), qs = unit & 1;
      ready(qfull(qs), unit >> 1);
      for (int i = 0; i < tiles && alive; ++i, ++g) {
        ready(full(ks), k_phase);
        if (!alive) break;
        const uint64_t a = k_desc + ks * (slot_bytes >> 4), q_at = q_desc + qs * (L::kQ >> 4);
        const uint32_t d = d_base + (g & 1) * NT;
#pragma unroll
        for (int s = 0; s < 8; ++s)
          if (s < p.ksteps)
            ptx::umma_bf16_if(one, d, a + (((s >> 2) * kHalfBytes + (s & 3) * 32) >> 4), q_at + (((s >> 2) * (NT * 128) + (s & 3) * 32) >> 4), idesc_s, s != 0);
        ptx::umma_commit_if(one, empty(ks));
        ptx::umma_commit_if(one, sfull(g & 1));
        if (i + 1 == tiles) ptx::umma_commit_if(one, qfree(qs));
        if (++ks == p.k_slots) {
          ks = 0;
          k_phase ^= 1u;
        }
        if (g > 0) second(g - 1);
      }
      w.next_unit(p, tiles);
      left = uniform(w.left);
      ++unit;
    }
    if (alive && g > 0) second(g - 1);
    ptx::umma_commit_if(one, drain);
    ptx::mbar_wait(drain, 0, abort_flag, wait_ns, false);
  } else if (warp == 3) {
    // ------------------------------------------------------------------------------------------ queries
    bool alive = true;
    for (int unit = 0; w.left > 0; ++unit) {
      const int end = w.piece_end();
      const int u_chunks = (w.q.fresh * p.G + NT - 1) / NT, h = w.u / u_chunks, row0 = (w.u % u_chunks) * NT, rows = w.q.fresh * p.G;
      const int qs = unit & 1;
      alive = ptx::mbar_wait(qfree(qs), ((unit >> 1) & 1) ^ 1u, abort_flag, wait_ns);
      if (!__all_sync(0xffffffffu, alive)) break;
      const uint32_t qb = qbuf + qs * L::kQ;
      const bf16_t* q = static_cast<const bf16_t*>(p.a.q.data) + w.b * p.a.q.seq;
      const int per = 8 * p.halves;              // 16-byte pieces of a row in shared memory
#pragma unroll 8
      for (int i = lane; i < NT * per; i += 32) {
        const int r = i / per, piece = i % per, row = row0 + r;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (row < rows && 8 * piece < p.c.D) {
          const bf16_t* at = q + (row / p.G) * p.a.q.token + (h * p.G + row % p.G) * p.a.q.head + 8 * piece;
          if (p.q_vec) {
            v = *reinterpret_cast<const uint4*>(at);
          } else {
            v.x = at[0] | static_cast<uint32_t>(at[1]) << 16;
            v.y = at[2] | static_cast<uint32_t>(at[3]) << 16;
            v.z = at[4] | static_cast<uint32_t>(at[5]) << 16;
            v.w = at[6] | static_cast<uint32_t>(at[7]) << 16;
          }
        }
        const uint32_t dst = qb + (piece >> 3) * (NT * 128) + r * 128 + (((piece & 7) ^ (r & 7)) << 4);
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
      }
      ptx::fence_proxy_async_smem();
      ptx::mbar_arrive(qfull(qs));
      w.next_unit(p, end - w.t);
    }
  } else {
    // ------------------------------------------------------------------------------------------ weights and sums
    constexpr int R = L::kRows;
    const int group = (warp - 4) >> 2, quarter = warp & 3, x = quarter * 32 + lane;      // slot of the tile, and column of the head
    const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
    // of this group's first row, without its swizzle; rows NT .. 2 NT - 1 are the low parts
    const uint32_t p_at = pbuf + (x >> 6) * (2 * NT * 128) + group * R * 128 + (x & 7) * 2, chunk = (x & 63) >> 3;
    float* wmax = small + group * L::kGroup;                                 // [4][R] the warps' maxima
    float* lsum = wmax + 4 * R;                                              // [4][R]
    float* ref = lsum + 4 * R;                                               // [R]
    float* alpha = ref + R;                                                  // [R]
    int* bound = reinterpret_cast<int*>(alpha + R);                          // [R] slots that a row sees
    volatile int* group_abort = misc + 22 + group;
    float o[R], l[R];
    int g = 0, flat = start.first, unit = 0;
    auto fail = [&] { *abort_flag = 1; *group_abort = 1; };
    auto wait = [&](uint32_t b, int phase) {
      if (!ptx::mbar_wait(b, phase & 1, abort_flag, wait_ns, false)) fail();
      __syncwarp();
    };
    auto read_row = [&](const float* from, float (&to)[R]) {
#pragma unroll
      for (int r = 0; r < R; r += 4) {
        const float4 q = *reinterpret_cast<const float4*>(from + r);
        to[r] = q.x; to[r + 1] = q.y; to[r + 2] = q.z; to[r + 3] = q.w;
      }
    };
    auto add_o = [&](int k) {                    // O of tile k
      wait(ofull(k & 1), k >> 1);
      ptx::tc_fence_after_sync();
#pragma unroll
      for (int low = 0; low < 2; ++low) {
        float v[R];
        tmem_load(tmem + lanes + 2 * NT + (2 * (k & 1) + low) * NT + group * R, v);
#pragma unroll
        for (int r = 0; r < R; ++r) o[r] += v[r];
      }
    };
    // A slot that some of the new tokens see must not reach the others by way of a weight of zero: infinities and NaN are taken out of its
    // value, and `odd` keeps the first slot with each (NaN counts as both signs), for the sums of the rows that see it.
    auto set_apart = [&](uint32_t row, int slot, int* odd) {
      for (int i = 0; i < 8; ++i) {
        const uint32_t at = row + ((i ^ (x & 7)) << 4);
        uint32_t e[4];
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(e[0]), "=r"(e[1]), "=r"(e[2]), "=r"(e[3]) : "r"(at) : "memory");
        bool some = false;
#pragma unroll
        for (int q = 0; q < 4; ++q) some |= (~e[q] & 0x7f80u) == 0 || (~e[q] & 0x7f800000u) == 0;
        if (!some) continue;
        for (int q = 0; q < 8; ++q) {
          uint16_t bits;
          asm volatile("ld.shared.u16 %0, [%1];" : "=h"(bits) : "r"(at + 2 * q) : "memory");
          if ((~bits & 0x7f80) != 0) continue;
          const bool nan = (bits & 0x7f) != 0, negative = (bits & 0x8000) != 0;
          int* first = odd + group * 64 + i * 8 + q;
          if (nan || !negative) atomicMin(first, slot);
          if (nan || negative) atomicMin(first + 128, slot);
          asm volatile("st.shared.u16 [%0], %1;" ::"r"(at + 2 * q), "h"(static_cast<uint16_t>(0)) : "memory");
        }
      }
    };
    // Whether this thread's column has +infinity (1), -infinity (2) or NaN (3) among the values of slots [s0, s1).
    auto column_kinds = [&](int b, int h, int s0, int s1) {
      const uint16_t* col = static_cast<const uint16_t*>(p.c.v) + h * p.c.v_head + x;
      const int* pages = p.s.table + b * p.s.ld_table;
      int kinds = 0;
      for (int s = s0; s < s1 && kinds != 3; s += 8) {          // (pages are multiples of eight slots)
        const int page = pages[s / p.c.page_slots];
        if (page < 0 || page >= p.c.pages) continue;
        const uint16_t* at = col + page * p.c.v_page + s % p.c.page_slots * p.c.v_slot;
        uint16_t bits[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) bits[i] = s + i < s1 ? at[i * p.c.v_slot] : 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if ((~bits[i] & 0x7f80) == 0) kinds |= (bits[i] & 0x7f) != 0 ? 3 : (bits[i] & 0x8000) != 0 ? 2 : 1;
      }
      return kinds;
    };
    bool alive = true;
    for (; w.left > 0; ++unit) {
      const int end = w.piece_end(), begin = w.t, tiles = end - begin;
      const int u_chunks = (w.q.fresh * p.G + NT - 1) / NT, h = w.u / u_chunks, row0 = (w.u % u_chunks) * NT + group * R;
      const int rows = min(R, w.q.fresh * p.G - row0);          // of this group; none: it keeps in step, and its weights are not looked at
      const long long unit_at = (static_cast<long long>(w.b) * p.c.H + h) * p.chunks + w.u % u_chunks;
      const int len = w.q.len, sure = len - (w.q.fresh - 1);    // every row sees the slots below `sure`
      if (group == 0 && begin == 0 && x == 0) p.unit_ctas[unit_at] = make_int2(blockIdx.x, cta_of(start, flat + w.q.tiles - 1));
      const bool ragged = end * kTile > sure;
      int* odd = odd_sh + (unit & 1) * 256;                     // [sign][column] (the other group may still read the last unit's)
      if (ragged) {
        if (group < p.halves) odd[(x >> 6) * 128 + group * 64 + (x & 63)] = INT_MAX;
        if (x < R) bound[x] = x < rows ? len - (w.q.fresh - 1 - (row0 + x) / p.G) : len;
        group_sync(group);
      }
#pragma unroll
      for (int r = 0; r < R; ++r) o[r] = l[r] = 0.f;
      for (int t = begin; t < end; ++t, ++g) {
        const int slot = t * kTile + x;
        const bool masked = (t + 1) * kTile > sure, first = t == begin;
        wait(sfull(g & 1), g >> 1);
        ptx::tc_fence_after_sync();
        bool rise = false;
        float v[R], rf[R];
        if (rows > 0) {
          tmem_load(tmem + lanes + (g & 1) * NT + group * R, v);
#pragma unroll
          for (int r = 0; r < R; ++r) v[r] *= p.scale2;
          if (masked) {
#pragma unroll
            for (int r = 0; r < R; ++r) v[r] = slot < bound[r] ? v[r] : -INFINITY;
          }
          if (p.scores != nullptr) {
            float* to = p.scores + ((unit_at * p.tiles + t) * NT + group * R) * kTile + x;
#pragma unroll
            for (int r = 0; r < R; ++r)
              if (r < rows) to[r * kTile] = v[r];
          }
          read_row(ref, rf);
          rise = first;
          if (!first) {
#pragma unroll
            for (int r = 0; r < R; ++r) rise |= v[r] > rf[r] + kSlack;
          }
        }
        rise = any_of_group(group, rise);
        if (*group_abort) { alive = false; break; }
        if (rows > 0) {
          if (rise) {
            float top = 0.f;
#pragma unroll
            for (int r = 0; r < R; ++r) {
              const float m = warp_max(v[r]);
              if (lane == r) top = m;
            }
            if (lane < R) wmax[quarter * R + lane] = top;
            group_sync(group);
            if (x < R) {
              const float old = first ? kNone : ref[x];
              const float m = fmaxf(fmaxf(fmaxf(wmax[x], wmax[R + x]), fmaxf(wmax[2 * R + x], wmax[3 * R + x])), old);
              ref[x] = m;
              alpha[x] = ptx::ex2_approx(old - m);
            }
            group_sync(group);
            read_row(ref, rf);
            float f[R];
            read_row(alpha, f);
#pragma unroll
            for (int r = 0; r < R; ++r) l[r] *= f[r];
          }
          const uint32_t to = p_at + (g & 1) * L::kP;
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const float e = ptx::ex2_approx(v[r] - rf[r]);
            l[r] += e;
            // as the sum of two bf16: one would add its own rounding, 2^-9 of a weight, to that of the output
            const uint32_t hi = ptx::pack_bf16x2(e, 0.f);
            const uint32_t lo = ptx::pack_bf16x2(e - ptx::bf16_lo(hi), 0.f);
            const uint32_t at = to + r * 128 + ((chunk ^ (r & 7)) << 4);
            asm volatile("st.shared.b16 [%0], %1;" ::"r"(at), "h"(static_cast<uint16_t>(hi)));
            asm volatile("st.shared.b16 [%0], %1;" ::"r"(at + NT * 128), "h"(static_cast<uint16_t>(lo)));
          }
        }
        if (masked && group < p.halves) {
          // rows of V that no slot of the sequence fills: whatever lies there must not meet a weight of zero
          const int s = p.k_slots + g % p.v_slots;
          wait(full(s), g / p.v_slots);
          const uint32_t row = ring + s * slot_bytes + group * kHalfBytes + x * 128;
          if (slot >= len) {
            for (int i = 0; i < 8; ++i) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(row + i * 16), "r"(0) : "memory");
          } else if (slot >= sure) {
            set_apart(row, slot, odd);
          }
        }
        ptx::tc_fence_before_sync();
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(pfull(g & 1));
        if (rows > 0) {
          if (!first) add_o(g - 1);
          if (rise) {
            float f[R];
            read_row(alpha, f);
#pragma unroll
            for (int r = 0; r < R; ++r) o[r] *= f[r];
          }
        } else if (!first) {
          wait(ofull((g - 1) & 1), (g - 1) >> 1);
        }
      }
      if (!alive) break;
      if (rows > 0) {
        add_o(g - 1);
        // A value that is infinite or NaN in a slot that every row sees has made all of this column so, but rarely of the right kind: the low part of its weight may be
        // zero or negative.  Then the column's values say what it is (which takes nothing elsewhere: sums that have overflowed, or weights of NaN, stay).
        if (x < p.c.D && !(fabsf(o[0]) <= FLT_MAX)) {
          const int kinds = column_kinds(w.b, h, begin * kTile, min(end * kTile, sure));
          if (kinds != 0) {
#pragma unroll
            for (int r = 0; r < R; ++r) o[r] = (kinds & 1 ? INFINITY : 0.f) + (kinds & 2 ? -INFINITY : 0.f);
          }
        }
        if (ragged && w.q.fresh > 1 && x < 64 * p.halves) {
          const int above = odd[x], below = odd[128 + x];
          if (min(above, below) != INT_MAX) {
#pragma unroll
            for (int r = 0; r < R; ++r) o[r] += (above < bound[r] ? INFINITY : 0.f) + (below < bound[r] ? -INFINITY : 0.f);
          }
        }
        // sums over the slots' threads
        float mine = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float sum = io::sum_lanes(l[r]);
          if (lane == r) mine = sum;
        }
        if (lane < R) lsum[quarter * R + lane] = mine;
        group_sync(group);
        mine = x < R ? (lsum[x] + lsum[R + x]) + (lsum[2 * R + x] + lsum[3 * R + x]) : 0.f;
        if (begin == 0 && end == w.q.tiles) {
          bf16_t* out = static_cast<bf16_t*>(p.a.out.data) + w.b * p.a.out.seq + x;
          if (x < p.c.D) {
#pragma unroll
            for (int r = 0; r < R; ++r)
              if (r < rows) {
                const float sum = (lsum[r] + lsum[R + r]) + (lsum[2 * R + r] + lsum[3 * R + r]);
                const int row = row0 + r;
                out[(row / p.G) * p.a.out.token + (h * p.G + row % p.G) * p.a.out.head] = io::from_f<bf16_t>(sum == 0.f ? 0.f : __fdividef(o[r], sum));
              }
          }
          if (x < rows) {
            const int row = row0 + x;
            if (p.a.lse != nullptr)
              p.a.lse[(static_cast<long long>(w.b) * p.s.Q + row / p.G) * p.a.Hq + h * p.G + row % p.G] = mine == 0.f ? -INFINITY : (ref[x] + log2f(mine)) * kLn2;
            if (p.scores != nullptr) p.whole_ml[unit_at * NT + group * R + x] = make_float2(ref[x], mine);
          }
        } else {
          const long long at = (blockIdx.x * 2 + (begin == 0 ? 1 : 0)) * NT + group * R;
#pragma unroll
          for (int r = 0; r < R; ++r)
            if (r < rows) p.part_o[(at + r) * 128 + x] = o[r];
          if (x < rows) p.part_ml[at + x] = make_float2(ref[x], mine);
        }
      } else {
        wait(ofull((g - 1) & 1), (g - 1) >> 1);
      }
      flat += tiles;
      w.next_unit(p, tiles);
    }
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  if (warp == 2) ptx::tmem_dealloc(tmem, L::kTmem);
  if (threadIdx.x == 0 && *abort_flag != 0) cache::raise_status(dev_status, cache::kWaitTimeout);
}

// ------------------------------------------------------------------------------------------ joining the shares
constexpr int kJoinThreads = 256;
constexpr int kJoinTiles = 8;            // tiles whose weights one block adds to acc: four slots to a thread
constexpr int kFewParts = 6;

// (A CTA that has given up on a wait leaves its units' numbers unwritten.)
__device__ __forceinline__ bool parts_known(const Params& p, int2 ctas) { return ctas.x >= 0 && ctas.x <= ctas.y && ctas.y < p.ctas; }

// Reference and sum of row r over the CTAs c0 .. c1 that had parts of a unit, in every lane of the warp.
template <int NT>
__device__ __forceinline__ float2 joined(const Params& p, int2 ctas, long long unit_at, int r) {
  if (ctas.x == ctas.y) return p.whole_ml[unit_at * NT + r];
  const int lane = threadIdx.x & 31;
  float m = kNone, l = 0.f;
  for (int c = ctas.x + lane; c <= ctas.y; c += 32) {
    const float2 ml = p.part_ml[(c * 2 + (c == ctas.x ? 1 : 0)) * NT + r];
    const float top = fmaxf(m, ml.x);
    l = l * ptx::ex2_approx(m - top) + ml.y * ptx::ex2_approx(ml.x - top);
    m = top;
  }
  const float top = warp_max(m);
  return make_float2(top, io::sum_lanes(l * ptx::ex2_approx(m - top)));
}

// Blocks [0, H * chunks) of a sequence join a unit's parts, a warp to a row; the others, with acc, add the weights of kJoinTiles
// tiles of a head to acc.
template <int NT>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ Params p) {
  __shared__ float sh[NT];
  const int b = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  ptx::grid_dep_wait();
  const Seq q = make_seq(p, p.s.lens[b], raw_new(p, b), NT);
  const int all_rows = q.fresh * p.G, chunks = (all_rows + NT - 1) / NT;
  if (blockIdx.x < p.c.H * p.chunks) {
    const int h = blockIdx.x / p.chunks, chunk = blockIdx.x % p.chunks;
    if (chunk >= chunks) return;
    const long long unit_at = (static_cast<long long>(b) * p.c.H + h) * p.chunks + chunk;
    const int2 ctas = p.unit_ctas[unit_at];
    if (ctas.x == ctas.y || !parts_known(p, ctas)) return;
    for (int r = warp; r < NT && chunk * NT + r < all_rows; r += kJoinThreads / 32) {
      const float2 ml = joined<NT>(p, ctas, unit_at, r);
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
      for (int c = ctas.x; c <= ctas.y; ++c) {
        const long long at = (c * 2 + (c == ctas.x ? 1 : 0)) * NT + r;
        const float f = ptx::ex2_approx(p.part_ml[at].x - ml.x);
        const float4 v = reinterpret_cast<const float4*>(p.part_o + at * 128)[lane];
        // (what is infinite is so with any factor, also one that has underflown)
        sum.x += fabsf(v.x) <= FLT_MAX ? f * v.x : v.x;
        sum.y += fabsf(v.y) <= FLT_MAX ? f * v.y : v.y;
        sum.z += fabsf(v.z) <= FLT_MAX ? f * v.z : v.z;
        sum.w += fabsf(v.w) <= FLT_MAX ? f * v.w : v.w;
      }
      const float inv = ml.y == 0.f ? 0.f : __fdividef(1.f, ml.y);
      const int row = chunk * NT + r, j = row / p.G, hq = h * p.G + row % p.G;
      bf16_t* out = static_cast<bf16_t*>(p.a.out.data) + b * p.a.out.seq + j * p.a.out.token + hq * p.a.out.head + 4 * lane;
      if (4 * lane < p.c.D) {
        out[0] = io::from_f<bf16_t>(sum.x * inv);
        out[1] = io::from_f<bf16_t>(sum.y * inv);
        out[2] = io::from_f<bf16_t>(sum.z * inv);
        out[3] = io::from_f<bf16_t>(sum.w * inv);
      }
      if (lane == 0 && p.a.lse != nullptr)
        p.a.lse[(static_cast<long long>(b) * p.s.Q + j) * p.a.Hq + hq] = ml.y == 0.f ? -INFINITY : (ml.x + log2f(ml.y)) * kLn2;
    }
    return;
  }
  // a thread has four slots next to one another: scores are read 16 bytes at a time, and eight rows at once
  const int rest = blockIdx.x - p.c.H * p.chunks, h = rest % p.c.H, tile0 = rest / p.c.H * kJoinTiles;
  if (chunks == 0 || tile0 * kTile >= q.len) return;
  const int first = tile0 * kTile + 4 * threadIdx.x;
  // (pages are multiples of eight slots: the four lie in one; what acc holds is read while the rows' sums are)
  const int page = first < q.len ? p.s.table[b * p.s.ld_table + first / p.c.page_slots] : -1;
  const bool known = page >= 0 && page < p.c.pages;
  float* acc = p.c.acc + (known ? page * p.c.acc_page + h * p.c.acc_head + first % p.c.page_slots : 0);
  float old[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) old[i] = known && first + i < q.len ? acc[i] : 0.f;
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int chunk = 0; chunk < chunks; ++chunk) {
    const long long unit_at = (static_cast<long long>(b) * p.c.H + h) * p.chunks + chunk;
    const int2 ctas = p.unit_ctas[unit_at];
    if (!parts_known(p, ctas)) return;
    const int rows = min(NT, all_rows - chunk * NT);
    bool nan = false;
    __syncthreads();
    if (ctas.y - ctas.x < kFewParts) {
      // few parts: a thread to a row
      if (threadIdx.x < NT) {
        float m = kNone, l = 0.f;
        if (threadIdx.x < rows) {
          float2 ml[kFewParts];
#pragma unroll
          for (int i = 0; i < kFewParts; ++i) {
            ml[i] = make_float2(kNone, 0.f);
            if (ctas.x == ctas.y && i == 0) ml[i] = p.whole_ml[unit_at * NT + threadIdx.x];
            else if (ctas.x + i <= ctas.y) ml[i] = p.part_ml[((ctas.x + i) * 2 + (i == 0 ? 1 : 0)) * NT + threadIdx.x];
            m = fmaxf(m, ml[i].x);
          }
#pragma unroll
          for (int i = 0; i < kFewParts; ++i) l += ml[i].y * ptx::ex2_approx(ml[i].x - m);
        }
        sh[threadIdx.x] = l == 0.f ? INFINITY : m + log2f(l);
        nan = l != l;
      }
    } else {
      for (int r = warp; r < rows; r += kJoinThreads / 32) {
        const float2 ml = joined<NT>(p, ctas, unit_at, r);
        if (lane == 0) sh[r] = ml.y == 0.f ? INFINITY : ml.x + log2f(ml.y);
        nan |= ml.y != ml.y;
      }
    }
    const bool broken = __syncthreads_or(nan);
    if (first >= q.len) continue;
    const float4* s = reinterpret_cast<const float4*>(p.scores + (unit_at * p.tiles + first / kTile) * NT * kTile + first % kTile);
    if (!broken) {
#pragma unroll 8
      for (int r = 0; r < rows; ++r) {
        const float4 v = s[r * (kTile / 4)];
        const float f = sh[r];
        sum.x += ptx::ex2_approx(v.x - f);
        sum.y += ptx::ex2_approx(v.y - f);
        sum.z += ptx::ex2_approx(v.z - f);
        sum.w += ptx::ex2_approx(v.w - f);
      }
    } else {
      // a row whose sum is NaN has no weight, not even that, for the slots that it does not see
#pragma unroll 1
      for (int r = 0; r < rows; ++r) {
        const float4 v = s[r * (kTile / 4)];
        const float f = sh[r];
        const int seen = q.len - (q.fresh - 1 - (chunk * NT + r) / p.G) - first;
        sum.x += seen > 0 ? ptx::ex2_approx(v.x - f) : 0.f;
        sum.y += seen > 1 ? ptx::ex2_approx(v.y - f) : 0.f;
        sum.z += seen > 2 ? ptx::ex2_approx(v.z - f) : 0.f;
        sum.w += seen > 3 ? ptx::ex2_approx(v.w - f) : 0.f;
      }
    }
  }
  const float add[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (known && first + i < q.len) acc[i] = old[i] + add[i];
}

}  // namespace attend
}  // namespace cpmtp
