// C-ABI of the operators of the base model's pass over a draft: paged cache of keys and values, attention over it, eviction from
// it, sampling from logits.  See include/cpmtp.h for the contract.
#include "../../include/cpmtp.h"

#include <cuda_runtime.h>
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "attend_kernels.cuh"
#include "cache_kernels.cuh"
#include "host_util.cuh"
#include "sample_kernels.cuh"
#include "tmap.cuh"

namespace cpmtp {
namespace {

using io::bf16_t;

constexpr int64_t kMaxStride = int64_t{1} << 38;       // elements: what a tensor map's strides hold

// Whether rows of `extent` elements at all places of some dimensions lie apart from one another, within what an offset can count.
// (Sorts the dimensions.)
struct Dim { int64_t stride, size; };
template <int N>
int check_apart(Dim (&d)[N], int64_t extent) {
  constexpr int64_t kMost = int64_t{1} << 60;
  std::sort(d, d + N, [](const Dim& a, const Dim& b) { return a.stride < b.stride; });
  for (const Dim& x : d) {
    if (x.size <= 1) continue;
    if (x.stride < extent) return CPMTP_ERR_SHAPE;
    if (x.stride > (kMost - extent) / (x.size - 1)) return CPMTP_ERR_LIMIT;
    extent += x.stride * (x.size - 1);
  }
  return CPMTP_OK;
}

// Distances of a cache's pages, slots and heads: rows of D elements must not overlap.
int check_strides(const cpmtp_cache& c, int64_t page, int64_t slot, int64_t head) {
  Dim d[3] = {{page, c.pages}, {slot, c.page_slots}, {head, c.H}};
  for (const Dim& x : d) {
    if (x.stride < 0) return CPMTP_ERR_SHAPE;
    if (x.stride >= kMaxStride) return CPMTP_ERR_LIMIT;
    if (x.stride % 8 != 0) return CPMTP_ERR_ALIGN;
  }
  return check_apart(d, c.D);
}
// Those of the pages and heads of acc, whose slots lie next to one another.
int check_acc(const cpmtp_cache& c) {
  Dim d[2] = {{c.acc_page, c.pages}, {c.acc_head, c.H}};
  for (const Dim& x : d) {
    if (x.stride < c.page_slots) return CPMTP_ERR_SHAPE;
    if (x.stride >= kMaxStride) return CPMTP_ERR_LIMIT;
  }
  return check_apart(d, c.page_slots);
}

int check_cache(const cpmtp_cache* c) {
  if (c == nullptr) return CPMTP_ERR_NULL;
  if (c->pages < 1 || c->page_slots < 8 || c->page_slots % 8 != 0 || c->page_slots > 65536) return CPMTP_ERR_SHAPE;
  if (c->H < 1 || c->H > 65535 || c->D < 8 || c->D % 8 != 0) return CPMTP_ERR_SHAPE;
  if (c->D > CPMTP_CACHE_MAX_D) return CPMTP_ERR_LIMIT;
  int rc;
  if ((rc = check_strides(*c, c->k_page, c->k_slot, c->k_head)) != CPMTP_OK || (rc = check_strides(*c, c->v_page, c->v_slot, c->v_head)) != CPMTP_OK)
    return rc;
  return c->acc != nullptr ? check_acc(*c) : CPMTP_OK;
}
int check_cache_data(const cpmtp_cache& c) {
  if (c.k == nullptr || c.v == nullptr) return CPMTP_ERR_NULL;
  return aligned(c.k, 16) && aligned(c.v, 16) && aligned(c.acc, 4) ? CPMTP_OK : CPMTP_ERR_ALIGN;
}

int check_seqs(const cpmtp_cache& c, const cpmtp_cache_seqs* s) {
  if (s == nullptr) return CPMTP_ERR_NULL;
  if (s->B < 0 || s->width < 0 || s->Q < 0 || s->ld_table < s->width) return CPMTP_ERR_SHAPE;
  if (s->B > 65535 || s->Q > (1 << 20) || static_cast<int64_t>(s->width) * c.page_slots >= (1 << 30)) return CPMTP_ERR_LIMIT;
  return CPMTP_OK;
}
int check_seqs_data(const cpmtp_cache_seqs& s) {
  if (s.lens == nullptr || (s.table == nullptr && s.width > 0)) return CPMTP_ERR_NULL;
  return aligned(s.table, 4) && aligned(s.lens, 4) && aligned(s.q_lens, 4) ? CPMTP_OK : CPMTP_ERR_ALIGN;
}

int check_tokens(const cpmtp_tokens* t, int64_t Q, int64_t H, int D) {
  if (t == nullptr || t->data == nullptr) return CPMTP_ERR_NULL;
  if (t->seq < 0 || (Q > 1 && t->token < D) || (H > 1 && t->head < D)) return CPMTP_ERR_SHAPE;
  return aligned(t->data, 2) ? CPMTP_OK : CPMTP_ERR_ALIGN;
}
// Those that are written: no two of them in one place.
int check_written(const cpmtp_tokens* t, int64_t B, int64_t Q, int64_t H, int D) {
  const int rc = check_tokens(t, Q, H, D);
  if (rc != CPMTP_OK) return rc;
  Dim d[3] = {{t->seq, B}, {t->token, Q}, {t->head, H}};
  return check_apart(d, D);
}
bool tokens_vec(const cpmtp_tokens& t) { return aligned(t.data, 16) && t.seq % 8 == 0 && t.token % 8 == 0 && t.head % 8 == 0; }

int blocks_for(long long items, int threads, int sms) {
  const long long blocks = (items + threads - 1) / threads, most = 64ll * sms;
  return static_cast<int>(blocks < most ? blocks : most);
}

// Columns of the narrow operand: the new tokens times the query heads that share a head, rounded up to a size there is a kernel for.  16 rows with 16 and 32
// columns: one sequence of 1024 slots 10.7 and 11.7 us, 64 ragged ones 226 and 232; 20 rows: 16 sequences of 4096 with acc 66 and 53, 32 of 8192 327 and 168 (in captured graphs).
int attend_columns(const cpmtp_cache& c, const cpmtp_cache_seqs& s, int Hq) {
  const long long rows = static_cast<long long>(s.Q) * (Hq / c.H);
  return rows <= 16 ? 16 : 32;
}

struct AttendLayout {
  int nt, chunks, tiles;
  size_t part_o, part_ml, unit_ctas, whole_ml, scores, total;
};
AttendLayout attend_layout(const cpmtp_cache& c, const cpmtp_cache_seqs& s, int Hq) {
  AttendLayout L;
  L.nt = attend_columns(c, s, Hq);
  L.chunks = static_cast<int>((static_cast<long long>(s.Q) * (Hq / c.H) + L.nt - 1) / L.nt);
  const long long slots = static_cast<long long>(s.width) * c.page_slots;
  L.tiles = static_cast<int>(slots > 0 ? (slots + attend::kTile - 1) / attend::kTile : 1);
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t o = off; off = align_up(off + bytes); return o; };
  const size_t parts = 2 * static_cast<size_t>(sm_count()) * L.nt, units = static_cast<size_t>(s.B) * c.H * L.chunks;
  L.part_o = take(parts * 128 * sizeof(float));
  L.part_ml = take(parts * sizeof(float2));
  L.unit_ctas = take(units * sizeof(int2));
  L.whole_ml = take(c.acc != nullptr ? units * L.nt * sizeof(float2) : 0);
  L.scores = take(c.acc != nullptr ? units * L.tiles * L.nt * attend::kTile * sizeof(float) : 0);
  L.total = off;
  return L;
}
// Whether the list of all tiles can be counted in 31 bits.
bool attend_fits(const cpmtp_cache& c, const cpmtp_cache_seqs& s, int Hq) {
  if (static_cast<long long>(s.Q) * (Hq / c.H) > (1 << 24)) return false;
  const AttendLayout L = attend_layout(c, s, Hq);
  return static_cast<double>(s.B) * c.H * L.chunks * L.tiles < 2147483648.0;
}

// Slots of a TMA box: they have to lie in one page, and a tile has to be made of whole boxes.
int piece_slots(int page_slots) {
  int piece = attend::kTile;
  while (page_slots % piece != 0) piece /= 2;
  return piece;
}

template <int NT>
cudaError_t launch_attend(const CUtensorMap& tk, const CUtensorMap& tv, attend::Params& p, int sms, int* dev_status, cudaStream_t st) {
  constexpr int kMost = 232448;
  const int slots = std::min(kMost - attend::Layout<NT>::kFixed, attend::kMaxSlots * attend::kHalfBytes) / (p.halves * attend::kHalfBytes);
  p.k_slots = slots / 2;          // (a K tile is done with sooner than a V tile, which waits for the weights)
  p.v_slots = slots - p.k_slots;
  p.ctas = sms;
  static bool done[64] = {};
  cudaError_t e = allow_smem(attend::attend_kernel<NT>, done, kMost);
  if (e != cudaSuccess) return e;
  const int bytes = attend::Layout<NT>::kFixed + slots * p.halves * attend::kHalfBytes;
  e = launch_pdl(attend::attend_kernel<NT>, dim3(sms), dim3(attend::kThreads), bytes, st, tk, tv, p, dev_status);
  if (e != cudaSuccess) return e;
  const int adders = p.scores != nullptr ? p.c.H * ((p.tiles + attend::kJoinTiles - 1) / attend::kJoinTiles) : 0;
  return launch_pdl(attend::join_kernel<NT>, dim3(p.c.H * p.chunks + adders, p.s.B), dim3(attend::kJoinThreads), 0, st, p);
}

size_t evict_bytes(const cpmtp_cache& c, const cpmtp_cache_seqs& s, int budget) {
  return align_up(sizeof(int) * static_cast<size_t>(s.B) * c.H * budget + kAlign);
}

// Blocks of a cluster that share the slots of a head: enough to use all SMs and to hold the keys in half of an SM's shared memory, as long as
// each has some slots for its threads (128 heads of 4352 slots with 1, 2, 4 and 8 blocks: 83, 82, 84 and 84 us; 16 of 65536 with 2, 4 and 8: 40, 29 and 28).
cudaError_t launch_select(const cpmtp_cache& c, const cpmtp_cache_seqs& s, const cpmtp_evict_args& e, int* kept, int sms, int* dev_status, cudaStream_t st) {
  constexpr size_t kMost = 232448, kShare = 110000;
  const int slots = s.width * c.page_slots;
  int ctas = 1;
  while (ctas < cluster::kMostCtas && slots / ctas >= 4 * cache::kSelectThreads &&
         (static_cast<size_t>(slots) * 4 / ctas > kShare || static_cast<long long>(s.B) * c.H * ctas < sms))
    ctas *= 2;
  const int span = ((slots + ctas - 1) / ctas + 31) / 32 * 32;
  const int vec = aligned(c.acc, 16) && c.acc_page % 4 == 0 && c.acc_head % 4 == 0;
  const size_t held = sizeof(cache::Select) + static_cast<size_t>(span) * 4;
  const dim3 grid(c.H * ctas, s.B), threads(cache::kSelectThreads);
  static bool done[64] = {}, done_far[64] = {};
  if (held <= kMost) {
    const cudaError_t rc = allow_smem(cache::select_kernel<true>, done, kMost);
    return rc != cudaSuccess ? rc : launch_clusters(ctas, cache::select_kernel<true>, grid, threads, held, st, c, s, ctas, span, vec, e.budget, e.recent, e.lens_out, kept, dev_status);
  }
  const cudaError_t rc = allow_smem(cache::select_kernel<false>, done_far, static_cast<int>(sizeof(cache::Select)));
  return rc != cudaSuccess ? rc : launch_clusters(ctas, cache::select_kernel<false>, grid, threads, sizeof(cache::Select), st, c, s, ctas, span, vec, e.budget, e.recent, e.lens_out, kept, dev_status);
}

template <class T, int THREADS>
cudaError_t launch_sample(const cpmtp_sample_args& a, int ctas, int* dev_status, cudaStream_t st) {
  const int span = ((a.V + ctas - 1) / ctas + 7) / 8 * 8;
  int width = 0;
  while ((1ll << width) < a.V) ++width;
  constexpr int kBytes = static_cast<int>(sizeof(sample::Shared<THREADS>));
  static bool done[64] = {};
  const cudaError_t e = allow_smem(sample::sample_kernel<T, THREADS>, done, kBytes);
  if (e != cudaSuccess) return e;
  return launch_clusters(ctas, sample::sample_kernel<T, THREADS>, dim3(static_cast<unsigned>(a.N) * ctas), dim3(THREADS), kBytes, st, a, ctas, span, 62 - width, dev_status);
}
// Blocks of a cluster that share a row: what takes the least time if two blocks fit on an SM, a block takes 17 us, 3 more for every doubling of the
// cluster, and half a nanosecond an entry if it has an SM to itself, one if not, one and a half if the rows under way do not fit in L2.
// (Measured with top-p and 1, 2, 4 and 8 blocks: 512 rows of 128256 311, 306, 381 and 572 us; 64 rows 89, 60, 62 and 79; 8 rows 88, 56, 42 and 32; 64 rows
// of 1024 18, 22, 24 and 47.)  Many rows of few entries get blocks of half the size, four to an SM: 1000 x 1024 45 us against 67, 2000 x 32000 295 against
// 319, but 512 x 128256 327 against 311.
template <class T>
cudaError_t launch_sample(const cpmtp_sample_args& a, int sms, int* dev_status, cudaStream_t st) {
  if (a.N > 2 * sms && a.V <= 32768) return launch_sample<T, 256>(a, 1, dev_status, st);
  int ctas = 1;
  long long best = 0;
  for (int n = 1, k = 0; n <= cluster::kMostCtas; n *= 2, ++k) {
    const long long blocks = static_cast<long long>(a.N) * n, waves = (blocks + 2 * sms - 1) / (2 * sms), rows = std::min<long long>(a.N, 2 * sms / n);
    const int entry = rows * a.V * static_cast<long long>(sizeof(T)) > (100ll << 20) ? 3 : blocks > sms ? 2 : 1;
    const long long time = waves * (34000 + 6000 * k + static_cast<long long>(entry) * (a.V / n));
    if (n > 1 && time >= best) continue;
    best = time;
    ctas = n;
  }
  return launch_sample<T, 512>(a, ctas, dev_status, st);
}

}  // namespace
}  // namespace cpmtp

using namespace cpmtp;

extern "C" {

int cpmtp_cache_append(const cpmtp_cache* cache, const cpmtp_cache_seqs* seqs, const cpmtp_tokens* k, const cpmtp_tokens* v,
                       int32_t* dev_status, cpmtp_stream stream) {
  int rc;
  if ((rc = check_cache(cache)) != CPMTP_OK || (rc = check_seqs(*cache, seqs)) != CPMTP_OK) return rc;
  const cpmtp_cache& c = *cache;
  const cpmtp_cache_seqs& s = *seqs;
  if (s.B == 0 || s.Q == 0) return CPMTP_OK;
  if ((rc = check_cache_data(c)) != CPMTP_OK || (rc = check_seqs_data(s)) != CPMTP_OK) return rc;
  if ((rc = check_tokens(k, s.Q, c.H, c.D)) != CPMTP_OK || (rc = check_tokens(v, s.Q, c.H, c.D)) != CPMTP_OK) return rc;
  if (!aligned(dev_status, 4)) return CPMTP_ERR_ALIGN;
  DeviceInfo* di = nullptr;
  if ((rc = check_device(&di)) != CPMTP_OK) return rc;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  ProfScope prof(CPMTP_STAGE_CACHE_APPEND, st);
  const dim3 grid(blocks_for(static_cast<long long>(s.B) * ((s.Q + cache::kTokens - 1) / cache::kTokens) * c.H * (c.D / 8), cache::kThreads, di->sms));
  if (tokens_vec(*k) && tokens_vec(*v)) CPMTP_TRY(launch_pdl(cache::append_kernel<true>, grid, dim3(cache::kThreads), 0, st, c, s, *k, *v, dev_status));
  else CPMTP_TRY(launch_pdl(cache::append_kernel<false>, grid, dim3(cache::kThreads), 0, st, c, s, *k, *v, dev_status));
  return CPMTP_OK;
}

size_t cpmtp_cache_attend_workspace_bytes(const cpmtp_cache* cache, const cpmtp_cache_seqs* seqs, int32_t Hq) {
  if (check_cache(cache) != CPMTP_OK || check_seqs(*cache, seqs) != CPMTP_OK || Hq < 1 || Hq % cache->H != 0) return 0;
  return attend_fits(*cache, *seqs, Hq) ? attend_layout(*cache, *seqs, Hq).total : 0;
}

int cpmtp_cache_attend(const cpmtp_cache* cache, const cpmtp_cache_seqs* seqs, const cpmtp_attend_args* args, void* workspace,
                       size_t workspace_bytes, int32_t* dev_status, cpmtp_stream stream) {
  int rc;
  if ((rc = check_cache(cache)) != CPMTP_OK || (rc = check_seqs(*cache, seqs)) != CPMTP_OK) return rc;
  if (args == nullptr) return CPMTP_ERR_NULL;
  const cpmtp_cache& c = *cache;
  const cpmtp_cache_seqs& s = *seqs;
  const cpmtp_attend_args& a = *args;
  if (a.Hq < 1 || a.Hq % c.H != 0 || !std::isfinite(a.scale)) return CPMTP_ERR_SHAPE;
  if (!attend_fits(c, s, a.Hq)) return CPMTP_ERR_LIMIT;
  if (s.B == 0 || s.Q == 0) return CPMTP_OK;
  if ((rc = check_cache_data(c)) != CPMTP_OK || (rc = check_seqs_data(s)) != CPMTP_OK) return rc;
  if ((rc = check_tokens(&a.q, s.Q, a.Hq, c.D)) != CPMTP_OK || (rc = check_written(&a.out, s.B, s.Q, a.Hq, c.D)) != CPMTP_OK) return rc;
  if (workspace == nullptr) return CPMTP_ERR_NULL;
  if (!aligned(a.lse, 4) || !aligned(dev_status, 4) || !aligned(workspace, kAlign)) return CPMTP_ERR_ALIGN;
  const AttendLayout L = attend_layout(c, s, a.Hq);
  if (workspace_bytes < L.total) return CPMTP_ERR_WORKSPACE;
  DeviceInfo* di = nullptr;
  if ((rc = check_device(&di)) != CPMTP_OK) return rc;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  ProfScope prof(CPMTP_STAGE_CACHE_ATTEND, st);
  attend::Params p = {};
  p.c = c; p.s = s; p.a = a;
  p.G = a.Hq / c.H; p.chunks = L.chunks; p.tiles = L.tiles;
  p.piece = piece_slots(c.page_slots);
  p.halves = c.D > 64 ? 2 : 1;
  p.ksteps = (c.D + 15) / 16;
  p.q_vec = tokens_vec(a.q);
  p.scale2 = a.scale * attend::kLog2e;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  p.part_o = reinterpret_cast<float*>(ws + L.part_o);
  p.part_ml = reinterpret_cast<float2*>(ws + L.part_ml);
  p.unit_ctas = reinterpret_cast<int2*>(ws + L.unit_ctas);
  if (c.acc != nullptr) {
    p.whole_ml = reinterpret_cast<float2*>(ws + L.whole_ml);
    p.scores = reinterpret_cast<float*>(ws + L.scores);
  }
  const WaitKnobs wait = wait_knobs();
  p.wait_limit_us = wait.limit_us;
  p.test_skip_load = wait.skip_load;
  CUtensorMap tk, tv;
  if (!make_paged_tmap_bf16(&tk, c.k, c.D, c.page_slots, c.H, c.pages, c.k_slot, c.k_head, c.k_page, p.piece) ||
      !make_paged_tmap_bf16(&tv, c.v, c.D, c.page_slots, c.H, c.pages, c.v_slot, c.v_head, c.v_page, p.piece))
    return CPMTP_ERR_LAUNCH;
  if (L.nt == 16) CPMTP_TRY(launch_attend<16>(tk, tv, p, di->sms, dev_status, st));
  else CPMTP_TRY(launch_attend<32>(tk, tv, p, di->sms, dev_status, st));
  return CPMTP_OK;
}

size_t cpmtp_cache_evict_workspace_bytes(const cpmtp_cache* cache, const cpmtp_cache_seqs* seqs, int32_t budget) {
  if (check_cache(cache) != CPMTP_OK || check_seqs(*cache, seqs) != CPMTP_OK || budget < 1) return 0;
  return evict_bytes(*cache, *seqs, budget);
}

int cpmtp_cache_evict(const cpmtp_cache* cache, const cpmtp_cache_seqs* seqs, const cpmtp_evict_args* args, void* workspace,
                      size_t workspace_bytes, int32_t* dev_status, cpmtp_stream stream) {
  int rc;
  if ((rc = check_cache(cache)) != CPMTP_OK || (rc = check_seqs(*cache, seqs)) != CPMTP_OK) return rc;
  if (args == nullptr) return CPMTP_ERR_NULL;
  const cpmtp_cache& c = *cache;
  const cpmtp_cache_seqs& s = *seqs;
  const cpmtp_evict_args& e = *args;
  if (e.budget < 1 || e.budget >= (1 << 30) || e.recent < 0 || e.recent > e.budget) return CPMTP_ERR_SHAPE;
  if (e.ld_table_out < (e.budget + c.page_slots - 1) / c.page_slots) return CPMTP_ERR_SHAPE;
  if (s.B == 0) return CPMTP_OK;
  if ((rc = check_cache_data(c)) != CPMTP_OK || (rc = check_seqs_data(s)) != CPMTP_OK) return rc;
  if (c.acc == nullptr || e.table_out == nullptr || e.lens_out == nullptr || (workspace == nullptr && e.kept == nullptr)) return CPMTP_ERR_NULL;
  if (!aligned(e.table_out, 4) || !aligned(e.lens_out, 4) || !aligned(e.kept, 4) || !aligned(dev_status, 4) || !aligned(workspace, kAlign))
    return CPMTP_ERR_ALIGN;
  if (e.lens_out < s.lens + s.B && s.lens < e.lens_out + s.B) return CPMTP_ERR_SHAPE;      // (read by other blocks than the one that writes)
  if (e.kept == nullptr && workspace_bytes < evict_bytes(c, s, e.budget)) return CPMTP_ERR_WORKSPACE;
  DeviceInfo* di = nullptr;
  if ((rc = check_device(&di)) != CPMTP_OK) return rc;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  ProfScope prof(CPMTP_STAGE_CACHE_EVICT, st);
  int* kept = e.kept != nullptr ? e.kept : static_cast<int*>(workspace);
  CPMTP_TRY(launch_select(c, s, e, kept, di->sms, dev_status, st));
  const int rows = static_cast<long long>(s.B) * c.H * e.budget >= 32ll * 64 * di->sms ? 32 : cache::least_rows(c.D), per = cache::kThreads / 32 * rows;
  const dim3 grid((e.budget + per - 1) / per, c.H, s.B);
  CPMTP_TRY(launch_pdl(cache::move_kernel, grid, dim3(cache::kThreads), 0, st, c, s, e.table_out, e.ld_table_out, e.budget, rows, kept, dev_status));
  return CPMTP_OK;
}

int cpmtp_sample_logits(const cpmtp_sample_args* args, int32_t* dev_status, cpmtp_stream stream) {
  if (args == nullptr) return CPMTP_ERR_NULL;
  const cpmtp_sample_args& a = *args;
  if (a.N < 0 || a.V < 1 || (a.N > 1 && a.ld < a.V) || (a.type != CPMTP_BF16 && a.type != CPMTP_F32)) return CPMTP_ERR_SHAPE;
  if (a.V > CPMTP_SAMPLE_MAX_V || a.N > (1 << 27)) return CPMTP_ERR_LIMIT;
  if (!(a.temperature >= 0.f) || !std::isfinite(a.temperature) || !(a.top_p >= 0.f) || !(a.min_p >= 0.f) || a.top_k < 0) return CPMTP_ERR_SHAPE;
  if (a.N == 0) return CPMTP_OK;
  if (!a.logits || !a.uniform || !a.tokens || (a.given && !a.logp_given)) return CPMTP_ERR_NULL;
  if (!aligned(a.logits, a.type == CPMTP_F32 ? 4 : 2)) return CPMTP_ERR_ALIGN;
  for (const void* p : {static_cast<const void*>(a.temperatures), static_cast<const void*>(a.top_ks), static_cast<const void*>(a.top_ps),
                        static_cast<const void*>(a.min_ps), static_cast<const void*>(a.uniform), static_cast<const void*>(a.given),
                        static_cast<const void*>(a.tokens), static_cast<const void*>(a.logp), static_cast<const void*>(a.logp_given),
                        static_cast<const void*>(a.kept), static_cast<const void*>(dev_status)})
    if (!aligned(p, 4)) return CPMTP_ERR_ALIGN;
  DeviceInfo* di = nullptr;
  const int rc = check_device(&di);
  if (rc != CPMTP_OK) return rc;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  ProfScope prof(CPMTP_STAGE_SAMPLE, st);
  if (a.type == CPMTP_F32) CPMTP_TRY(launch_sample<float>(a, di->sms, dev_status, st));
  else CPMTP_TRY(launch_sample<bf16_t>(a, di->sms, dev_status, st));
  return CPMTP_OK;
}

}  // extern "C"
