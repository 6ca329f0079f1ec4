// Attention of a few new tokens over the paged cache.
//
//   s_i = scale <q, k_i>,  p = softmax(s),  out = sum_i p_i v_i
//
// Every key and value is read once and used for a few rows only (the new tokens times the query heads that share a head of the
// cache), so the time is that of reading the cache.  The products run on the tensor cores with the cache's tile as the operand of
// 128 rows and the queries as the narrow one:
//   S^T [128 slots, NT rows] = K_tile [128, D] Q^T,   O^T [D, NT] = V_tile^T [D, 128] P^T
// in TMEM: a lane is a slot in the first and a column of the head in the second, and nothing is padded to 128 but D.
//
// The tiles of 128 slots of all (sequence, head, chunk of NT rows) form one list, which is cut into equal shares, one for each
// SM, whatever the lengths.  A share that ends inside a unit leaves (max, sum, unnormalised out) behind; join_kernel joins them.
//
//   warp 0      TMA: pages into a ring of K and V tiles in turn
//   warp 1      tcgen05.mma: S of tile g, then O of tile g - 1
//   warps 2-5   a thread is a slot: weights; then a column: sums O in registers
//   warp 6      queries of the next unit into shared memory
#pragma once
#include <cuda.h>

#include "cache_kernels.cuh"

namespace cpmtp {
namespace attend {

using io::bf16_t;

constexpr int kTile = 128;                  // slots of a tile
constexpr int kThreads = 7 * 32;
constexpr int kHalfBytes = kTile * 128;     // 128 slots of 64 columns
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNone = -1.7e38f;           // the reference of a row that has seen nothing yet
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
  int slots;                   // of the ring; a slot holds one K or V tile
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
  static constexpr int kP = NT * 256;                // weights of a tile: 128 slots of NT rows, bf16
  static constexpr int kQueries = NT < 64 ? 2 : 1;   // units whose queries are held: one where two would cost the ring a slot
  static constexpr int kBars = 512;
  static constexpr int kSmall = 11 * NT * 4 + 128;
  static constexpr int kFixed = 1024 + kQueries * kQ + 4 * kP + kBars + kSmall;
  static constexpr int kTmem = 4 * NT;               // two S and two O accumulators
};
constexpr int kMaxSlots = 12;

__device__ __forceinline__ bool any_of_group(bool v) {      // of the 128 softmax threads; a barrier
  int r;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.or.aligned.pred q, 1, 128, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
               : "=r"(r) : "r"(static_cast<int>(v)) : "memory");
  return r != 0;
}
__device__ __forceinline__ void group_sync() { asm volatile("barrier.cta.sync.aligned 1, 128;" ::: "memory"); }
__device__ __forceinline__ float warp_max(float v) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const void* tmap, uint32_t bar, int c0, int c1, int c2, int c3) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tmap)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
__device__ __forceinline__ void tmem_load(uint32_t addr, float (&v)[16]) {
  ptx::tmem_ld_32x16(addr, v);
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]),
                 "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])::"memory");
}
__device__ __forceinline__ void tmem_load(uint32_t addr, float (&v)[32]) {
  ptx::tmem_ld_32x32(addr, v);
  ptx::tmem_ld_wait_for(v);
}

template <int NT>
__global__ void __launch_bounds__(kThreads, 1) attend_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                                                             const __grid_constant__ Params p, int* dev_status) {
  using L = Layout<NT>;
  constexpr int CH = NT < 32 ? NT : 32, NCH = NT / CH;        // columns of an accumulator handled at a time
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = ptx::smem_u32(smem_raw), pad = (1024u - (raw & 1023u)) & 1023u;
  const uint32_t slot_bytes = p.halves * kHalfBytes;
  // [ring][queries x 2][weights: two tiles of (high, low)][barriers][small arrays]
  const uint32_t ring = raw + pad, qbuf = ring + p.slots * slot_bytes, pbuf = qbuf + L::kQueries * L::kQ, bars = pbuf + 4 * L::kP;
  uint8_t* small = smem_raw + (bars + L::kBars - raw);
  int* bound = reinterpret_cast<int*>(small);                 // [NT] slots that a row sees
  float* wmax = reinterpret_cast<float*>(bound + NT);     // [4][NT] the warps' maxima
  float* ref = wmax + 4 * NT;                                 // [NT]
  float* alpha = ref + NT;                                    // [NT]
  float* lsum = alpha + NT;                                   // [4][NT]
  int* misc = reinterpret_cast<int*>(lsum + 4 * NT);          // [0..6] scan, [8..14] start, [16] TMEM address, [17], [18] abort flags
  Start* start_sh = reinterpret_cast<Start*>(misc + 8);
  volatile int* abort_flag = misc + 17;
  volatile int* group_abort = misc + 18;
  auto full = [&](int s) { return bars + 8u * s; };
  auto empty = [&](int s) { return bars + 8u * (kMaxSlots + s); };
  auto qfull = [&](int s) { return bars + 8u * (2 * kMaxSlots + s); };
  auto qfree = [&](int s) { return bars + 8u * (2 * kMaxSlots + 2 + s); };
  auto sfull = [&](int s) { return bars + 8u * (2 * kMaxSlots + 4 + s); };
  auto pfull = [&](int s) { return bars + 8u * (2 * kMaxSlots + 6 + s); };
  auto ofull = [&](int s) { return bars + 8u * (2 * kMaxSlots + 8 + s); };
  const uint32_t drain = bars + 8u * (2 * kMaxSlots + 10);
  static_assert(8 * (2 * kMaxSlots + 11) <= L::kBars, "barriers");

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint64_t wait_ns = static_cast<uint64_t>(p.wait_limit_us) * 1000ull;
  if (threadIdx.x == 0) {
    for (int s = 0; s < p.slots; ++s) {
      ptx::mbar_init(full(s), 1);
      ptx::mbar_init(empty(s), 1);
    }
    for (int s = 0; s < 2; ++s) {
      ptx::mbar_init(qfull(s), 32);
      ptx::mbar_init(qfree(s), 1);
      ptx::mbar_init(sfull(s), 1);
      ptx::mbar_init(pfull(s), 128);
      ptx::mbar_init(ofull(s), 1);
    }
    ptx::mbar_init(drain, 1);
    *abort_flag = 0;
    *group_abort = 0;
    ptx::fence_mbar_init();
    ptx::prefetch_tmap(&tm_k);
    ptx::prefetch_tmap(&tm_v);
  }
  if (warp == 1) {
    ptx::tmem_alloc(ptx::smem_u32(misc + 16), L::kTmem);
    ptx::tmem_relinquish();
  }
  ptx::grid_dep_wait();
  ptx::tc_fence_before_sync();
  find_start(p, NT, misc, start_sh, dev_status);
  ptx::tc_fence_after_sync();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(misc + 16);
  const Start start = *start_sh;
  Walk w(p, start, NT);

  if (warp == 0) {
    // ------------------------------------------------------------------------------------------ pages into the ring
    const int pieces = kTile / p.piece;
    auto page_at = [&](const Walk& x) {          // the page of this lane's piece of the tile; -1: nothing to load
      const int slot = x.t * kTile + lane * p.piece;
      if (lane >= pieces || slot >= x.q.len) return -1;
      const int page = p.s.table[x.b * p.s.ld_table + slot / p.c.page_slots];
      return page >= 0 && page < p.c.pages ? page : p.c.pages;      // out of range: the box reads as zeros
    };
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
      for (int kv = 0; kv < 2; ++kv, ++it) {
        const int s = it % p.slots;
        if (lane == 0) {
          alive = ptx::mbar_wait(empty(s), ((it / p.slots) & 1) ^ 1u, abort_flag, wait_ns);
          if (alive && it + 1 != p.test_skip_load) {
            if (bytes > 0) ptx::mbar_arrive_expect_tx(full(s), bytes);
            else ptx::mbar_arrive(full(s));
          }
        }
        alive = __shfl_sync(0xffffffffu, alive, 0);
        if (!alive) break;
        if (here >= 0 && it + 1 != p.test_skip_load) {
          const uint32_t dst = ring + s * slot_bytes + lane * p.piece * 128u;
          const void* tm = kv == 0 ? &tm_k : &tm_v;
          for (int half = 0; half < p.halves; ++half) tma_load_4d(dst + half * kHalfBytes, tm, full(s), half * 64, in_page, h, here);
        }
      }
    }
    ptx::grid_dep_launch();
    if (lane == 0)               // what was issued has to land before the shared memory is given back
      for (int back = 1; back <= p.slots && back <= it; ++back) ptx::mbar_wait(full((it - back) % p.slots), ((it - back) / p.slots) & 1, abort_flag, wait_ns, false);
  } else if (warp == 1) {
    // ------------------------------------------------------------------------------------------ products
    if (lane == 0) {
      constexpr uint32_t idesc_s = ptx::make_idesc_bf16(128, NT, 0, 0), idesc_o = ptx::make_idesc_bf16(128, NT, 1, 0);
      bool alive = true;
      int g = 0, unit = 0;
      auto second = [&](int k) {                 // O of tile k
        const int s = (2 * k + 1) % p.slots;
        if (!ptx::mbar_wait(full(s), ((2 * k + 1) / p.slots) & 1, abort_flag, wait_ns) || !ptx::mbar_wait(pfull(k & 1), (k >> 1) & 1, abort_flag, wait_ns)) return false;
        ptx::tc_fence_after_sync();
        const uint32_t v = ring + s * slot_bytes, pw = pbuf + (k & 1) * 2 * L::kP, d = tmem + 2 * NT + (k & 1) * NT;
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
          const uint64_t a = ptx::make_smem_desc_sw128(v + ks * 2048, kHalfBytes, 1024);
#pragma unroll
          for (int low = 0; low < 2; ++low)
            ptx::umma_bf16(d, a, ptx::make_smem_desc_sw128(pw + low * L::kP + (ks >> 2) * (NT * 128) + (ks & 3) * 32, 16, 1024), idesc_o, (ks | low) != 0);
        }
        ptx::umma_commit(empty(s));
        ptx::umma_commit(ofull(k & 1));
        return true;
      };
      while (w.left > 0 && alive) {
        const int end = w.piece_end();
        const int qs = unit % L::kQueries;
        const uint32_t qb = qbuf + qs * L::kQ;
        if (!ptx::mbar_wait(qfull(qs), (unit / L::kQueries) & 1, abort_flag, wait_ns)) { alive = false; break; }
        for (int t = w.t; t < end; ++t, ++g) {
          const int s = (2 * g) % p.slots;
          if (!ptx::mbar_wait(full(s), ((2 * g) / p.slots) & 1, abort_flag, wait_ns)) { alive = false; break; }
          ptx::tc_fence_after_sync();
          const uint32_t k = ring + s * slot_bytes;
          for (int ks = 0; ks < p.ksteps; ++ks)
            ptx::umma_bf16(tmem + (g & 1) * NT, ptx::make_smem_desc_sw128(k + (ks >> 2) * kHalfBytes + (ks & 3) * 32, 16, 1024),
                           ptx::make_smem_desc_sw128(qb + (ks >> 2) * (NT * 128) + (ks & 3) * 32, 16, 1024), idesc_s, ks != 0);
          ptx::umma_commit(empty(s));
          ptx::umma_commit(sfull(g & 1));
          if (t + 1 == end) ptx::umma_commit(qfree(qs));
          if (g > 0 && !second(g - 1)) { alive = false; break; }
        }
        w.next_unit(p, end - w.t);
        ++unit;
      }
      if (alive && g > 0) second(g - 1);
      ptx::umma_commit(drain);
      ptx::mbar_wait(drain, 0, abort_flag, wait_ns, false);
    }
  } else if (warp == 6) {
    // ------------------------------------------------------------------------------------------ queries
    bool alive = true;
    for (int unit = 0; w.left > 0; ++unit) {
      const int end = w.piece_end();
      const int u_chunks = (w.q.fresh * p.G + NT - 1) / NT, h = w.u / u_chunks, row0 = (w.u % u_chunks) * NT, rows = w.q.fresh * p.G;
      const int qs = unit % L::kQueries;
      alive = ptx::mbar_wait(qfree(qs), ((unit / L::kQueries) & 1) ^ 1u, abort_flag, wait_ns);
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
    const int quarter = warp & 3, x = quarter * 32 + lane;      // slot of the tile, and column of the head
    const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
    const uint32_t p_at = pbuf + (x >> 6) * (NT * 128) + (x & 7) * 2;      // of row 0, without its swizzle
    const uint32_t chunk = (x & 63) >> 3;
    float o[NT], l[NT];
    int g = 0, flat = start.first;
    auto fail = [&] { *abort_flag = 1; *group_abort = 1; };
    auto add_o = [&](int k) {                    // O of tile k
      if (!ptx::mbar_wait(ofull(k & 1), (k >> 1) & 1, abort_flag, wait_ns, false)) fail();
      __syncwarp();
      ptx::tc_fence_after_sync();
#pragma unroll
      for (int ch = 0; ch < NCH; ++ch) {
        float v[CH];
        tmem_load(tmem + lanes + 2 * NT + (k & 1) * NT + ch * CH, v);
#pragma unroll
        for (int r = 0; r < CH; ++r) o[ch * CH + r] += v[r];
      }
    };
    bool alive = true;
    while (w.left > 0) {
      const int end = w.piece_end(), begin = w.t;
      const int u_chunks = (w.q.fresh * p.G + NT - 1) / NT, h = w.u / u_chunks, chunk_no = w.u % u_chunks;
      const int rows = min(NT, w.q.fresh * p.G - chunk_no * NT);
      const long long unit_at = (static_cast<long long>(w.b) * p.c.H + h) * p.chunks + chunk_no;
      const int len = w.q.len, sure = len - (w.q.fresh - 1);    // every row sees the slots below `sure`
      if (begin == 0 && x == 0) p.unit_ctas[unit_at] = make_int2(blockIdx.x, cta_of(start, flat + w.q.tiles - 1));
      if (end * kTile > sure) {
        if (x < NT) bound[x] = x < rows ? len - (w.q.fresh - 1 - (chunk_no * NT + x) / p.G) : len;
        group_sync();
      }
#pragma unroll
      for (int r = 0; r < NT; ++r) o[r] = l[r] = 0.f;
      for (int t = begin; t < end; ++t, ++g) {
        const int slot = t * kTile + x;
        const bool masked = (t + 1) * kTile > sure, first = t == begin;
        if (!ptx::mbar_wait(sfull(g & 1), (g >> 1) & 1, abort_flag, wait_ns, false)) fail();
        __syncwarp();
        ptx::tc_fence_after_sync();
        const uint32_t s_at = tmem + lanes + (g & 1) * NT;
        float v[CH];
        auto scores = [&](int ch) {
          tmem_load(s_at + ch * CH, v);
#pragma unroll
          for (int r = 0; r < CH; ++r) v[r] *= p.scale2;
          if (masked) {
#pragma unroll
            for (int r = 0; r < CH; ++r) v[r] = slot < bound[ch * CH + r] ? v[r] : -INFINITY;
          }
        };
        bool rise = first;
#pragma unroll
        for (int ch = 0; ch < NCH; ++ch) {
          scores(ch);
          if (p.scores != nullptr) {
            float* to = p.scores + ((unit_at * p.tiles + t) * NT + ch * CH) * kTile + x;
#pragma unroll
            for (int r = 0; r < CH; ++r)
              if (ch * CH + r < rows) to[r * kTile] = v[r];
          }
          if (!first) {
#pragma unroll
            for (int r = 0; r < CH; ++r) rise |= v[r] > ref[ch * CH + r] + kSlack;
          }
        }
        rise = any_of_group(rise);
        if (*group_abort) { alive = false; break; }
        if (rise) {
#pragma unroll
          for (int ch = 0; ch < NCH; ++ch) {
            if (NCH > 1) scores(ch);
            float top = 0.f;
#pragma unroll
            for (int r = 0; r < CH; ++r) {
              const float m = warp_max(v[r]);
              if (lane == r) top = m;
            }
            if (lane < CH) wmax[quarter * NT + ch * CH + lane] = top;
          }
          group_sync();
          if (x < NT) {
            const float old = first ? kNone : ref[x];
            const float m = fmaxf(fmaxf(fmaxf(wmax[x], wmax[NT + x]), fmaxf(wmax[2 * NT + x], wmax[3 * NT + x])), old);
            ref[x] = m;
            alpha[x] = ptx::ex2_approx(old - m);
          }
          group_sync();
#pragma unroll
          for (int r = 0; r < NT; ++r) l[r] *= alpha[r];
        }
#pragma unroll
        for (int ch = 0; ch < NCH; ++ch) {
          if (NCH > 1) scores(ch);
          const uint32_t to = p_at + (g & 1) * 2 * L::kP + ch * CH * 128;
#pragma unroll
          for (int r = 0; r < CH; ++r) {
            const float e = ptx::ex2_approx(v[r] - ref[ch * CH + r]);
            l[ch * CH + r] += e;
            // as the sum of two bf16: one would add its own rounding, 2^-9 of a weight, to that of the output
            const uint32_t hi = ptx::pack_bf16x2(e, 0.f);
            const uint32_t lo = ptx::pack_bf16x2(e - ptx::bf16_lo(hi), 0.f);
            const uint32_t at = to + r * 128 + ((chunk ^ (r & 7)) << 4);
            asm volatile("st.shared.b16 [%0], %1;" ::"r"(at), "h"(static_cast<uint16_t>(hi)) : "memory");
            asm volatile("st.shared.b16 [%0], %1;" ::"r"(at + L::kP), "h"(static_cast<uint16_t>(lo)) : "memory");
          }
        }
        if ((t + 1) * kTile > len) {
          // rows of V that no slot of the sequence fills: whatever lies there must not meet a weight of zero
          const int s = (2 * g + 1) % p.slots;
          if (!ptx::mbar_wait(full(s), ((2 * g + 1) / p.slots) & 1, abort_flag, wait_ns, false)) fail();
          if (slot >= len)
            for (int i = 0; i < 8 * p.halves; ++i)
              asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(ring + s * slot_bytes + (i >> 3) * kHalfBytes + x * 128 + (i & 7) * 16), "r"(0) : "memory");
        }
        ptx::tc_fence_before_sync();
        ptx::fence_proxy_async_smem();
        ptx::mbar_arrive(pfull(g & 1));
        if (!first) add_o(g - 1);
        if (rise) {
#pragma unroll
          for (int r = 0; r < NT; ++r) o[r] *= alpha[r];
        }
      }
      if (!alive) break;
      add_o(g - 1);
      // sums over the slots' threads
#pragma unroll
      for (int ch = 0; ch < NCH; ++ch) {
        float mine = 0.f;
#pragma unroll
        for (int r = 0; r < CH; ++r) {
          const float sum = io::sum_lanes(l[ch * CH + r]);
          if (lane == r) mine = sum;
        }
        if (lane < CH) lsum[quarter * NT + ch * CH + lane] = mine;
      }
      group_sync();
      const bool whole = begin == 0 && end == w.q.tiles;
      float mine = 0.f;
      if (x < NT) mine = (lsum[x] + lsum[NT + x]) + (lsum[2 * NT + x] + lsum[3 * NT + x]);
      if (whole) {
        bf16_t* out = static_cast<bf16_t*>(p.a.out.data) + w.b * p.a.out.seq + x;
#pragma unroll
        for (int r = 0; r < NT; ++r)
          if (r < rows) {
            const float sum = (lsum[r] + lsum[NT + r]) + (lsum[2 * NT + r] + lsum[3 * NT + r]);
            const int row = chunk_no * NT + r;
            if (x < p.c.D) out[(row / p.G) * p.a.out.token + (h * p.G + row % p.G) * p.a.out.head] = io::from_f<bf16_t>(sum == 0.f ? 0.f : __fdividef(o[r], sum));
          }
        if (x < rows) {
          const int row = chunk_no * NT + x;
          if (p.a.lse != nullptr)
            p.a.lse[(static_cast<long long>(w.b) * p.s.Q + row / p.G) * p.a.Hq + h * p.G + row % p.G] = mine == 0.f ? -INFINITY : (ref[x] + log2f(mine)) * kLn2;
          if (p.scores != nullptr) p.whole_ml[unit_at * NT + x] = make_float2(ref[x], mine);
        }
      } else {
        const long long at = (blockIdx.x * 2 + (begin == 0 ? 1 : 0)) * NT;
#pragma unroll
        for (int r = 0; r < NT; ++r)
          if (r < rows) p.part_o[(at + r) * 128 + x] = o[r];
        if (x < NT) p.part_ml[at + x] = make_float2(ref[x], mine);
      }
      flat += end - begin;
      w.next_unit(p, end - begin);
    }
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  if (warp == 1) ptx::tmem_dealloc(tmem, L::kTmem);
  if (threadIdx.x == 0 && *abort_flag != 0) cache::raise_status(dev_status, cache::kWaitTimeout);
}

// ------------------------------------------------------------------------------------------ joining the shares
constexpr int kJoinThreads = 256;
constexpr int kJoinTiles = 8;            // tiles whose weights one block adds to acc

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
// tiles of a head to acc, a thread to a slot.
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
        sum.x += f * v.x; sum.y += f * v.y; sum.z += f * v.z; sum.w += f * v.w;
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
  const int rest = blockIdx.x - p.c.H * p.chunks, h = rest % p.c.H, tile0 = rest / p.c.H * kJoinTiles;
  if (chunks == 0 || tile0 * kTile >= q.len) return;
  constexpr int kPer = kJoinTiles * kTile / kJoinThreads;
  float sum[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) sum[i] = 0.f;
  for (int chunk = 0; chunk < chunks; ++chunk) {
    const long long unit_at = (static_cast<long long>(b) * p.c.H + h) * p.chunks + chunk;
    const int2 ctas = p.unit_ctas[unit_at];
    if (!parts_known(p, ctas)) return;
    const int rows = min(NT, all_rows - chunk * NT);
    __syncthreads();
    for (int r = warp; r < rows; r += kJoinThreads / 32) {
      const float2 ml = joined<NT>(p, ctas, unit_at, r);
      if (lane == 0) sh[r] = ml.y == 0.f ? INFINITY : ml.x + log2f(ml.y);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int slot = tile0 * kTile + i * kJoinThreads + threadIdx.x;
      if (slot >= q.len) continue;
      const float* s = p.scores + (unit_at * p.tiles + slot / kTile) * NT * kTile + slot % kTile;
#pragma unroll 4
      for (int r = 0; r < rows; ++r) sum[i] += ptx::ex2_approx(s[r * kTile] - sh[r]);
    }
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int slot = tile0 * kTile + i * kJoinThreads + threadIdx.x;
    if (slot >= q.len) continue;
    const int page = p.s.table[b * p.s.ld_table + slot / p.c.page_slots];
    if (page >= 0 && page < p.c.pages) p.c.acc[page * p.c.acc_page + h * p.c.acc_head + slot % p.c.page_slots] += sum[i];
  }
}

}  // namespace attend
}  // namespace cpmtp
