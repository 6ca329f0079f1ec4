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

namespace cpmtp {
namespace {

using io::bf16_t;

int check_device(DeviceInfo** out) {
  DeviceInfo* di = device_info();
  if (di == nullptr) return CPMTP_ERR_LAUNCH;
  if (di->cc_major != 10) return CPMTP_ERR_ARCH;
  *out = di;
  return CPMTP_OK;
}

constexpr int64_t kMaxStride = int64_t{1} << 38;       // elements: what a tensor map's strides hold

// Distances of a cache's pages, slots and heads: rows of D elements must not overlap.
int check_strides(const cpmtp_cache& c, int64_t page, int64_t slot, int64_t head) {
  struct Dim { int64_t stride, size; } d[3] = {{page, c.pages}, {slot, c.page_slots}, {head, c.H}};
  std::sort(d, d + 3, [](const Dim& a, const Dim& b) { return a.stride < b.stride; });
  int64_t extent = c.D;
  for (const Dim& x : d) {
    if (x.stride < 0) return CPMTP_ERR_SHAPE;
    if (x.stride >= kMaxStride) return CPMTP_ERR_LIMIT;
    if (x.stride % 8 != 0) return CPMTP_ERR_ALIGN;
    if (x.size == 1) continue;
    if (x.stride < extent) return CPMTP_ERR_SHAPE;
    extent += x.stride * (x.size - 1);
  }
  return CPMTP_OK;
}

int check_cache(const cpmtp_cache* c) {
  if (c == nullptr) return CPMTP_ERR_NULL;
  if (c->pages < 1 || c->page_slots < 8 || c->page_slots % 8 != 0 || c->page_slots > 65536) return CPMTP_ERR_SHAPE;
  if (c->H < 1 || c->H > 65535 || c->D < 8 || c->D % 8 != 0) return CPMTP_ERR_SHAPE;
  if (c->D > CPMTP_CACHE_MAX_D) return CPMTP_ERR_LIMIT;
  int rc;
  if ((rc = check_strides(*c, c->k_page, c->k_slot, c->k_head)) != CPMTP_OK || (rc = check_strides(*c, c->v_page, c->v_slot, c->v_head)) != CPMTP_OK)
    return rc;
  if (c->acc != nullptr && (c->acc_head < c->page_slots || c->acc_page < c->page_slots)) return CPMTP_ERR_SHAPE;
  return CPMTP_OK;
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
bool tokens_vec(const cpmtp_tokens& t) { return aligned(t.data, 16) && t.seq % 8 == 0 && t.token % 8 == 0 && t.head % 8 == 0; }

int blocks_for(long long items, int threads, int sms) {
  const long long blocks = (items + threads - 1) / threads, most = 64ll * sms;
  return static_cast<int>(blocks < most ? blocks : most);
}

size_t attend_bytes(const cpmtp_cache& c, const cpmtp_cache_seqs& s, int Hq) {
  return align_up(sizeof(float) * static_cast<size_t>(s.B) * s.Q * Hq + kAlign);
}
size_t evict_bytes(const cpmtp_cache& c, const cpmtp_cache_seqs& s, int budget) {
  return align_up(sizeof(int) * static_cast<size_t>(s.B) * c.H * budget + kAlign);
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
  const dim3 grid(blocks_for(static_cast<long long>(s.B) * s.Q * c.H * (c.D / 8), cache::kThreads, di->sms));
  if (tokens_vec(*k) && tokens_vec(*v)) CPMTP_TRY(launch_pdl(cache::append_kernel<true>, grid, dim3(cache::kThreads), 0, st, c, s, *k, *v, dev_status));
  else CPMTP_TRY(launch_pdl(cache::append_kernel<false>, grid, dim3(cache::kThreads), 0, st, c, s, *k, *v, dev_status));
  return CPMTP_OK;
}

size_t cpmtp_cache_attend_workspace_bytes(const cpmtp_cache* cache, const cpmtp_cache_seqs* seqs, int32_t Hq) {
  if (check_cache(cache) != CPMTP_OK || check_seqs(*cache, seqs) != CPMTP_OK || Hq < 1 || Hq % cache->H != 0) return 0;
  return attend_bytes(*cache, *seqs, Hq);
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
  if (static_cast<long long>(s.Q) * a.Hq > (1 << 24)) return CPMTP_ERR_LIMIT;
  if (s.B == 0 || s.Q == 0) return CPMTP_OK;
  if ((rc = check_cache_data(c)) != CPMTP_OK || (rc = check_seqs_data(s)) != CPMTP_OK) return rc;
  if ((rc = check_tokens(&a.q, s.Q, a.Hq, c.D)) != CPMTP_OK || (rc = check_tokens(&a.out, s.Q, a.Hq, c.D)) != CPMTP_OK) return rc;
  if (workspace == nullptr) return CPMTP_ERR_NULL;
  if (!aligned(a.lse, 4) || !aligned(dev_status, 4) || !aligned(workspace, kAlign)) return CPMTP_ERR_ALIGN;
  if (workspace_bytes < attend_bytes(c, s, a.Hq)) return CPMTP_ERR_WORKSPACE;
  DeviceInfo* di = nullptr;
  if ((rc = check_device(&di)) != CPMTP_OK) return rc;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  ProfScope prof(CPMTP_STAGE_CACHE_ATTEND, st);
  float* lse = static_cast<float*>(workspace);
  CPMTP_TRY(launch_pdl(attend::attend_kernel, dim3(s.Q * a.Hq, s.B), dim3(attend::kThreads), 0, st, c, s, a, lse, dev_status));
  if (c.acc != nullptr) {
    const int blocks = (s.width * c.page_slots + attend::kThreads - 1) / attend::kThreads;
    CPMTP_TRY(launch_pdl(attend::weight_kernel, dim3(blocks, c.H, s.B), dim3(attend::kThreads), 0, st, c, s, a, lse, dev_status));
  }
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
  if (c.acc == nullptr || e.table_out == nullptr || e.lens_out == nullptr || workspace == nullptr) return CPMTP_ERR_NULL;
  if (e.lens_out == s.lens) return CPMTP_ERR_SHAPE;
  if (!aligned(e.table_out, 4) || !aligned(e.lens_out, 4) || !aligned(e.kept, 4) || !aligned(dev_status, 4) || !aligned(workspace, kAlign))
    return CPMTP_ERR_ALIGN;
  if (workspace_bytes < evict_bytes(c, s, e.budget)) return CPMTP_ERR_WORKSPACE;
  DeviceInfo* di = nullptr;
  if ((rc = check_device(&di)) != CPMTP_OK) return rc;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  ProfScope prof(CPMTP_STAGE_CACHE_EVICT, st);
  int* kept = e.kept != nullptr ? e.kept : static_cast<int*>(workspace);
  CPMTP_TRY(launch_pdl(cache::select_kernel, dim3(c.H, s.B), dim3(cache::kSelectThreads), 0, st, c, s, e.budget, e.recent, e.lens_out, kept, dev_status));
  const dim3 grid(blocks_for(static_cast<long long>(s.B) * c.H * e.budget * (c.D / 8), cache::kThreads, di->sms));
  CPMTP_TRY(launch_pdl(cache::move_kernel, grid, dim3(cache::kThreads), 0, st, c, s, e.table_out, e.ld_table_out, e.budget, kept, dev_status));
  return CPMTP_OK;
}

int cpmtp_sample_logits(const cpmtp_sample_args* args, int32_t* dev_status, cpmtp_stream stream) {
  if (args == nullptr) return CPMTP_ERR_NULL;
  const cpmtp_sample_args& a = *args;
  if (a.N < 0 || a.V < 1 || (a.N > 1 && a.ld < a.V) || (a.type != CPMTP_BF16 && a.type != CPMTP_F32)) return CPMTP_ERR_SHAPE;
  if (a.V > CPMTP_SAMPLE_MAX_V) return CPMTP_ERR_LIMIT;
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
  int bits = 0;
  while ((1ll << bits) < a.V) ++bits;
  const double unit = std::ldexp(1.0, 62 - bits);      // V weights of at most one sum to less than 2^63
  if (a.type == CPMTP_F32) CPMTP_TRY(launch_pdl(sample::sample_kernel<float>, dim3(a.N), dim3(sample::kThreads), 0, st, a, unit, dev_status));
  else CPMTP_TRY(launch_pdl(sample::sample_kernel<bf16_t>, dim3(a.N), dim3(sample::kThreads), 0, st, a, unit, dev_status));
  return CPMTP_OK;
}

}  // extern "C"
