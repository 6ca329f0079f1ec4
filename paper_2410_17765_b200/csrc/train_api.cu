// C-ABI of the operators around the head in a training step: embedding lookup and its gradient, norms with gate
// and residual addition, AdamW and gradient clipping.  See include/cpmtp.h for the contract.
#include "../../include/cpmtp.h"

#include <cuda_runtime.h>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <type_traits>

#include "adamw_kernels.cuh"
#include "embed_kernels.cuh"
#include "host_util.cuh"
#include "norm_kernels.cuh"

namespace cpmtp {
namespace {

using io::bf16_t;

bool known_type(int t) { return t == CPMTP_BF16 || t == CPMTP_F32; }
size_t type_bytes(int t) { return t == CPMTP_F32 ? 4 : 2; }

// ------------------------------------------------------------------------------------------- embedding
int check_embed(const cpmtp_embed_shape* s) {
  if (s == nullptr) return CPMTP_ERR_NULL;
  if (s->T < 0 || s->T >= (1 << 30) || s->V < 1 || s->V >= (1 << 30) || s->d < 1 || s->d >= (1 << 24)) return CPMTP_ERR_SHAPE;
  if (s->ld_table < s->d || s->ld_rows < s->d || !known_type(s->type)) return CPMTP_ERR_SHAPE;
  return CPMTP_OK;
}

struct EmbedLayout {
  int bits, passes, blocks;      // digits of the sort; thread blocks of a pass
  int slabs, chunk, chunks;      // columns and sorted positions that the summing warps take
  size_t hist, keys, head, tail, total;
};

// Short chunks of the sums: up to this many tokens, if long ones make fewer warps than this on each SM.
constexpr long long kShortTokens = 2048, kWarpsWanted = 8;

EmbedLayout embed_layout(const cpmtp_embed_shape& s) {
  EmbedLayout L;
  int width = 1;
  while ((1ll << width) <= s.V) ++width;         // keys are 0 .. V
  L.passes = (width + embed::kMaxBits - 1) / embed::kMaxBits;
  L.bits = (width + L.passes - 1) / L.passes;
  L.blocks = (s.T + embed::kSortKeys - 1) / embed::kSortKeys;
  L.slabs = (s.d + embed::kSlab - 1) / embed::kSlab;
  L.chunk = s.T <= kShortTokens && static_cast<long long>(s.T) * L.slabs < kWarpsWanted * sm_count() * embed::kChunk ? embed::kShortChunk : embed::kChunk;
  L.chunks = (s.T + L.chunk - 1) / L.chunk;
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off = align_up(off + bytes); return o; };
  L.hist = take(3 * sizeof(int) * (static_cast<size_t>(L.blocks) << L.bits));
  L.keys = take(2 * sizeof(uint2) * static_cast<size_t>(s.T));
  const size_t part = L.chunks > 1 ? sizeof(float) * static_cast<size_t>(L.chunks) * L.slabs * embed::kSlab : 0;
  L.head = take(part);
  L.tail = take(part);
  L.total = off;
  return L;
}

template <int CTAS, int KPT>
cudaError_t sort_in_cluster_as(const int* x, uint2* out, int T, int V, const EmbedLayout& L, int* dev_status, cudaStream_t st) {
  constexpr int kBytes = embed::cluster_sort_bytes(CTAS, KPT);
  static bool done[64] = {};
  auto* kernel = embed::embed_sort_cluster_kernel<CTAS, KPT>;
  const cudaError_t e = allow_smem(kernel, done, kBytes);
  return e != cudaSuccess ? e : launch_clusters(CTAS, kernel, dim3(CTAS), dim3(embed::kClusterThreads), kBytes, st, x, out, T, V, L.bits, L.passes, dev_status);
}
cudaError_t sort_in_cluster(const int* x, uint2* out, int T, int V, const EmbedLayout& L, int* dev_status, cudaStream_t st) {
  constexpr int kOne = embed::kClusterThreads, kAll = kOne * embed::kClusterSize;
  if (T <= kOne) return sort_in_cluster_as<1, 1>(x, out, T, V, L, dev_status, st);
  if (T <= kAll) return sort_in_cluster_as<embed::kClusterSize, 1>(x, out, T, V, L, dev_status, st);
  if (T <= 2 * kAll) return sort_in_cluster_as<embed::kClusterSize, 2>(x, out, T, V, L, dev_status, st);
  if (T <= 4 * kAll) return sort_in_cluster_as<embed::kClusterSize, 4>(x, out, T, V, L, dev_status, st);
  return sort_in_cluster_as<embed::kClusterSize, 8>(x, out, T, V, L, dev_status, st);
}

// The result is in keys[(L.passes + 1) % 2].
cudaError_t sort_in_memory(const int* x, uint2* const (&keys)[2], int* hists, int T, int V, const EmbedLayout& L, int* dev_status, cudaStream_t st) {
  int* hist[3];
  for (int j = 0; j < 3; ++j) hist[j] = hists + j * (static_cast<size_t>(L.blocks) << L.bits);
  const dim3 grid(L.blocks), threads(embed::kSortThreads);
  cudaError_t e = launch_pdl(embed::embed_hist_kernel, grid, threads, 0, st, x, T, V, L.bits, hist[0], L.passes > 1 ? hist[1] : nullptr, dev_status);
  for (int pass = 0; pass < L.passes && e == cudaSuccess; ++pass) {
    int* next = pass + 1 < L.passes ? hist[(pass + 1) % 3] : nullptr;
    int* zero = pass + 2 < L.passes ? hist[(pass + 2) % 3] : nullptr;
    if (pass == 0) e = launch_pdl(embed::embed_sort_kernel<true>, grid, threads, 0, st, x, nullptr, keys[0], T, V, L.bits, 0, hist[0], next, zero);
    else e = launch_pdl(embed::embed_sort_kernel<false>, grid, threads, 0, st, nullptr, keys[(pass + 1) % 2], keys[pass % 2], T, V, L.bits,
                        pass * L.bits, hist[pass % 3], next, zero);
  }
  return e;
}

template <class T, bool VEC, bool ACCUM>
cudaError_t launch_embed_sum_as(const T* dy, const embed::SumParams& p, int zero_blocks, cudaStream_t st) {
  const cudaError_t e = launch_pdl(embed::embed_sum_kernel<T, VEC, ACCUM>, dim3(p.sum_blocks + zero_blocks), dim3(256), 0, st, dy, p);
  if (e != cudaSuccess || p.chunks < 2) return e;
  return launch_pdl(embed::embed_join_kernel<VEC, ACCUM>, dim3(p.sum_blocks), dim3(256), 0, st, p);
}
template <class T>
cudaError_t launch_embed_sum(const T* dy, const embed::SumParams& p, bool accum, int zero_blocks, cudaStream_t st) {
  const bool vec = io::vec_ok<T>(dy, p.ld, p.d) && io::vec_ok<bf16_t>(p.dE, p.ld_table, p.d);
  if (accum) return vec ? launch_embed_sum_as<T, true, true>(dy, p, 0, st) : launch_embed_sum_as<T, false, true>(dy, p, 0, st);
  return vec ? launch_embed_sum_as<T, true, false>(dy, p, zero_blocks, st) : launch_embed_sum_as<T, false, false>(dy, p, zero_blocks, st);
}

// ------------------------------------------------------------------------------------------------ norms
struct NormLayout {
  int W, G, threads;             // warps per row, rows per block, threads per block
  int per_sm;                    // blocks that make sixteen warps on an SM
};

// `vec`: the rows allow accesses of eight columns.  Blocks of several rows are better for those (8192 x 2048: backward 52 us
// against 57 for blocks of one row), blocks of one row for others, whose addresses take more operations and are then common to
// a block (8192 x 2047: 77 us against 80; 16384 x 1023 in fp32 with row gates: 60 against 66) -- where one row is wide enough to leave few blocks: their sums are added up afterwards.
NormLayout norm_layout(int d, bool vec) {
  NormLayout L;
  L.W = (d + 255) / 256;
  const int rows = L.W >= 16 ? 1 : 16 / L.W;
  L.G = !vec && L.W >= 4 ? 1 : rows;
  L.per_sm = rows / L.G;
  L.threads = L.W * L.G * 32;
  return L;
}

// Rows kept in shared memory per row group, the current one included: as many as 227 KB hold for one block of the
// backward kernel per SM, or half of that for two of the forward kernel.
template <class S>
constexpr int fwd_stages() { return sizeof(S) == 4 ? 3 : 4; }
template <class S, int MAXT>
constexpr int bwd_stages() { return MAXT > 512 ? 2 : (sizeof(S) == 4 ? 3 : 5); }

template <bool ONE>
constexpr int kMaxGroups = ONE ? 1 : 16;

int row_blocks(const cpmtp_norm_args& a, const NormLayout& L, int most) {
  const long long rows = (static_cast<long long>(a.N) + L.G - 1) / L.G;
  return static_cast<int>(rows < most ? rows : most);
}
int norm_bwd_blocks(const cpmtp_norm_args& a, const NormLayout& L, int sms) { return row_blocks(a, L, sms * L.per_sm); }

int check_rows(const cpmtp_rows& r, int d, size_t bytes) {
  if (r.data == nullptr) return CPMTP_ERR_NULL;
  if (r.ld < d) return CPMTP_ERR_SHAPE;
  return aligned(r.data, bytes) ? CPMTP_OK : CPMTP_ERR_ALIGN;
}

int check_norm(const cpmtp_norm_args* a) {
  if (a == nullptr) return CPMTP_ERR_NULL;
  if (a->N < 0 || a->d < 1 || !known_type(a->stream_type)) return CPMTP_ERR_SHAPE;
  if (a->d > CPMTP_NORM_MAX_D) return CPMTP_ERR_LIMIT;
  if (a->gate_kind < CPMTP_GATE_NONE || a->gate_kind > CPMTP_GATE_CHANNEL) return CPMTP_ERR_SHAPE;
  // (of a subnormal eps the rstd of a row of zeros would have an infinite square, which the gradient multiplies by zero)
  if (!(a->eps >= FLT_MIN) || !std::isfinite(a->eps) || !std::isfinite(a->res_scale)) return CPMTP_ERR_SHAPE;
  if (a->N > 0 && a->block.data == nullptr) {      // (without rows a block may have no address)
    // a norm alone: nothing to gate, to scale or to norm before the addition
    if (a->gate_kind != CPMTP_GATE_NONE || a->w_post != nullptr || a->res_scale != 1.f) return CPMTP_ERR_SHAPE;
    if (a->w_pre == nullptr) return CPMTP_ERR_NULL;
  }
  return CPMTP_OK;
}

int check_gate(const cpmtp_norm_args& a, const cpmtp_rows& g) {
  if (a.gate_kind == CPMTP_GATE_CHANNEL) return check_rows(g, a.d, 2);
  return a.gate_kind == CPMTP_GATE_ROW ? check_rows(g, 1, 2) : CPMTP_OK;
}

template <class S>
norm::Params<S> norm_params(const cpmtp_norm_args& a, const NormLayout& L) {
  norm::Params<S> p;
  std::memset(&p, 0, sizeof(p));
  p.N = a.N; p.d = a.d; p.W = L.W; p.G = L.G; p.gate_kind = a.gate_kind;
  p.eps = a.eps; p.res_scale = a.res_scale; p.inv_d = 1.f / static_cast<float>(a.d);
  p.x = {static_cast<const S*>(a.x.data), a.x.ld};
  p.block = {static_cast<const bf16_t*>(a.block.data), a.block.ld};
  p.gate = {static_cast<const bf16_t*>(a.gate.data), a.gate.ld};
  p.w_post = static_cast<const bf16_t*>(a.w_post);
  p.w_pre = static_cast<const bf16_t*>(a.w_pre);
  p.x_out = {static_cast<S*>(a.x_out.data), a.x_out.ld};
  p.y = {static_cast<bf16_t*>(a.y.data), a.y.ld};
  p.rstd_post = a.rstd_post; p.rstd_pre = a.rstd_pre;
  p.dy = {static_cast<const bf16_t*>(a.dy.data), a.dy.ld};
  p.dx_out = {static_cast<const S*>(a.dx_out.data), a.dx_out.ld};
  p.dx = {static_cast<S*>(a.dx.data), a.dx.ld};
  p.dblock = {static_cast<bf16_t*>(a.dblock.data), a.dblock.ld};
  p.dgate = {static_cast<bf16_t*>(a.dgate.data), a.dgate.ld};
  return p;
}

template <class T>
bool rows_vec(const cpmtp_rows& r, int d) { return d % 8 == 0 && (r.data == nullptr || io::vec_ok<T>(r.data, r.ld, d)); }

template <class S, bool VEC, int MAXT, bool ONE, bool ALL>
cudaError_t launch_norm_fwd_as(const norm::Params<S>& p, const NormLayout& L, int blocks, cudaStream_t st) {
  constexpr int kStages = fwd_stages<S>();
  static bool done[64] = {};
  auto* kernel = norm::norm_fwd_kernel<S, VEC, MAXT, kStages, ONE, ALL>;
  const cudaError_t e = allow_smem(kernel, done, kStages * kMaxGroups<ONE> * norm::fwd_stage_bytes<S>(MAXT / kMaxGroups<ONE>));
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3(blocks), dim3(L.threads), kStages * L.G * norm::fwd_stage_bytes<S>(L.W * 32), st, p);
}

template <class S, int MAXT, bool ONE>
cudaError_t launch_norm_fwd(const cpmtp_norm_args& a, const NormLayout& L, bool vec, int sms, cudaStream_t st) {
  const norm::Params<S> p = norm_params<S>(a, L);
  const int blocks = row_blocks(a, L, sms * (1024 / MAXT) * L.per_sm);
  const bool all = a.d % 256 == 0 && a.gate_kind == CPMTP_GATE_CHANNEL && a.w_post != nullptr && a.w_pre != nullptr && a.rstd_post != nullptr &&
                   a.rstd_pre != nullptr;
  if (!vec) return launch_norm_fwd_as<S, false, MAXT, ONE, false>(p, L, blocks, st);
  return all ? launch_norm_fwd_as<S, true, MAXT, ONE, true>(p, L, blocks, st) : launch_norm_fwd_as<S, true, MAXT, ONE, false>(p, L, blocks, st);
}
template <class S>
cudaError_t launch_norm_fwd(const cpmtp_norm_args& a, int sms, cudaStream_t st) {
  const bool vec = rows_vec<S>(a.x, a.d) && rows_vec<bf16_t>(a.block, a.d) && rows_vec<S>(a.x_out, a.d) && rows_vec<bf16_t>(a.y, a.d) &&
                   (a.gate_kind != CPMTP_GATE_CHANNEL || rows_vec<bf16_t>(a.gate, a.d)) && aligned(a.w_post, 16) && aligned(a.w_pre, 16);
  const NormLayout L = norm_layout(a.d, vec);
  if (L.threads > 512) return launch_norm_fwd<S, 1024, true>(a, L, vec, sms, st);
  return L.G == 1 ? launch_norm_fwd<S, 512, true>(a, L, vec, sms, st) : launch_norm_fwd<S, 512, false>(a, L, vec, sms, st);
}

template <class S, bool VEC, int MAXT, bool ONE, int FORM>
cudaError_t launch_norm_bwd_as(const norm::Params<S>& p, const NormLayout& L, int blocks, cudaStream_t st) {
  constexpr int kStages = bwd_stages<S, MAXT>();
  static bool done[64] = {};
  auto* kernel = norm::norm_bwd_kernel<S, VEC, MAXT, kStages, ONE, FORM>;
  const cudaError_t e = allow_smem(kernel, done, kStages * kMaxGroups<ONE> * norm::bwd_stage_bytes<S>(MAXT / kMaxGroups<ONE>));
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3(blocks), dim3(L.threads), kStages * L.G * norm::bwd_stage_bytes<S>(L.W * 32), st, p);
}

template <class S, int MAXT, bool ONE>
cudaError_t launch_norm_bwd(const cpmtp_norm_args& a, const NormLayout& L, bool vec, int blocks, float* part, cudaStream_t st) {
  norm::Params<S> p = norm_params<S>(a, L);
  p.part = part;
  const bool all = a.d % 256 == 0 && a.gate_kind == CPMTP_GATE_CHANNEL && a.w_post != nullptr && a.dy.data != nullptr && a.dx_out.data != nullptr &&
                   a.dx.data != nullptr && a.dblock.data != nullptr && a.dgate.data != nullptr;
  if (vec && all) return launch_norm_bwd_as<S, true, MAXT, ONE, norm::kAll>(p, L, blocks, st);
  if (a.gate_kind == CPMTP_GATE_CHANNEL)
    return vec ? launch_norm_bwd_as<S, true, MAXT, ONE, norm::kChannelGate>(p, L, blocks, st)
               : launch_norm_bwd_as<S, false, MAXT, ONE, norm::kChannelGate>(p, L, blocks, st);
  return vec ? launch_norm_bwd_as<S, true, MAXT, ONE, norm::kRowGate>(p, L, blocks, st)
             : launch_norm_bwd_as<S, false, MAXT, ONE, norm::kRowGate>(p, L, blocks, st);
}
// Leaves the number of blocks, and so of partial sums of the weights' gradients, in `blocks`.
template <class S>
cudaError_t launch_norm_bwd(const cpmtp_norm_args& a, int sms, int& blocks, float* part, cudaStream_t st) {
  const bool vec = rows_vec<S>(a.x_out, a.d) && rows_vec<bf16_t>(a.block, a.d) && rows_vec<bf16_t>(a.dy, a.d) && rows_vec<S>(a.dx_out, a.d) &&
                   rows_vec<S>(a.dx, a.d) && rows_vec<bf16_t>(a.dblock, a.d) &&
                   (a.gate_kind != CPMTP_GATE_CHANNEL || (rows_vec<bf16_t>(a.gate, a.d) && rows_vec<bf16_t>(a.dgate, a.d))) &&
                   aligned(a.w_post, 16) && aligned(a.w_pre, 16);
  const NormLayout L = norm_layout(a.d, vec);
  blocks = norm_bwd_blocks(a, L, sms);
  if (L.threads > 512) return launch_norm_bwd<S, 1024, true>(a, L, vec, blocks, part, st);
  return L.G == 1 ? launch_norm_bwd<S, 512, true>(a, L, vec, blocks, part, st) : launch_norm_bwd<S, 512, false>(a, L, vec, blocks, part, st);
}

// ---------------------------------------------------------------------------------------------- optimiser
int check_grads(const cpmtp_adamw_tensor* tensors, int32_t count) {
  if (count < 0) return CPMTP_ERR_SHAPE;
  if (count > 0 && tensors == nullptr) return CPMTP_ERR_NULL;
  for (int i = 0; i < count; ++i) {
    const cpmtp_adamw_tensor& t = tensors[i];
    if (t.numel < 0 || t.numel >= (1ll << 40) || !known_type(t.grad_type)) return CPMTP_ERR_SHAPE;
    if (!aligned(t.grad, type_bytes(t.grad_type))) return CPMTP_ERR_ALIGN;
  }
  return CPMTP_OK;
}

int check_adamw(const cpmtp_adamw_tensor* tensors, int32_t count, const cpmtp_adamw_hyper* h) {
  if (h == nullptr) return CPMTP_ERR_NULL;
  const bool betas = h->beta1 >= 0.0 && h->beta1 < 1.0 && h->beta2 >= 0.0 && h->beta2 < 1.0;
  if (!betas || !(h->lr >= 0.0) || !(h->eps >= 0.0) || !(h->weight_decay >= 0.0)) return CPMTP_ERR_SHAPE;
  if (!std::isfinite(h->lr) || !std::isfinite(h->eps) || !std::isfinite(h->weight_decay)) return CPMTP_ERR_SHAPE;
  if (h->step < 1 || (h->state_bits != 32 && h->state_bits != 8)) return CPMTP_ERR_SHAPE;
  if (!aligned(h->coef, 4)) return CPMTP_ERR_ALIGN;
  const int rc = check_grads(tensors, count);
  if (rc != CPMTP_OK) return rc;
  for (int i = 0; i < count; ++i) {
    const cpmtp_adamw_tensor& t = tensors[i];
    if (!known_type(t.param_type) || (t.master != nullptr && t.param_type != CPMTP_BF16)) return CPMTP_ERR_SHAPE;
    if (!std::isfinite(t.lr_scale) || !std::isfinite(t.decay_scale)) return CPMTP_ERR_SHAPE;
    if (t.grad == nullptr || t.numel == 0) continue;
    if (!t.param || !t.m || !t.v) return CPMTP_ERR_NULL;
    if (h->state_bits == 8 && (!t.m_exp || !t.v_exp)) return CPMTP_ERR_NULL;
    const size_t state = h->state_bits == 8 ? 1 : 4;
    if (!aligned(t.param, type_bytes(t.param_type)) || !aligned(t.master, 4) || !aligned(t.m, state) || !aligned(t.v, state))
      return CPMTP_ERR_ALIGN;
  }
  return CPMTP_OK;
}

// Elements per thread block: `most`, unless that leaves the SMs with few blocks each.
int run_length(const cpmtp_adamw_tensor* tensors, int32_t count, int most, int sms) {
  long long total = 0;
  for (int i = 0; i < count; ++i) total += tensors[i].numel;
  if (total >= 16ll * sms * most) return most;
  return total >= 4ll * sms * adamw::kRun ? adamw::kRun : adamw::kShortRun;
}

// Launches over tables of at most CAP tensors; `fn(table, runs)` enqueues one of them.
template <int CAP, class Fill, class Fn>
int for_tables(const cpmtp_adamw_tensor* tensors, int32_t count, const adamw::Hyper& h, int run, Fill fill, Fn fn) {
  adamw::Table<CAP> tab;
  tab.h = h;
  tab.count = 0;
  tab.run = run;
  long long place = 0, runs = 0;
  constexpr long long kMaxRuns = 1ll << 30;
  for (int i = 0; i < count; ++i) {
    const cpmtp_adamw_tensor& t = tensors[i];
    const long long here = place;
    place += (t.numel + adamw::kBlock - 1) / adamw::kBlock * adamw::kBlock;
    if (t.grad == nullptr || t.numel == 0) continue;
    const long long more = (t.numel + run - 1) / run;
    if (tab.count == CAP || runs + more > kMaxRuns) {
      const int rc = fn(tab, static_cast<int>(runs));
      if (rc != CPMTP_OK) return rc;
      tab.count = 0;
      runs = 0;
    }
    tab.first[tab.count] = static_cast<int>(runs);
    fill(t, here, tab.t[tab.count]);
    ++tab.count;
    runs += more;
  }
  return tab.count > 0 ? fn(tab, static_cast<int>(runs)) : CPMTP_OK;
}

template <int CAP, bool CLOCK>
int adamw_step(const cpmtp_adamw_tensor* tensors, int32_t count, const cpmtp_adamw_hyper& hyper, const cpmtp_adamw_clock* clock, int sms,
               cudaStream_t st) {
  adamw::Hyper h = {};
  h.b1 = static_cast<float>(hyper.beta1);
  h.omb1 = static_cast<float>(1.0 - hyper.beta1);
  h.b2 = static_cast<float>(hyper.beta2);
  h.omb2 = static_cast<float>(1.0 - hyper.beta2);
  h.eps = static_cast<float>(hyper.eps);
  const unsigned long long t = CLOCK ? 1 : hyper.step;
  const double bc1 = adamw::one_minus(adamw::power(hyper.beta1, t));
  h.r.rsqrt_bc2 = adamw::rsqrt_bc2_of(hyper.beta2, t);
  h.r.key = adamw::noise_key(hyper.seed, t);
  h.r.small_eps = h.eps < adamw::kSmallEps * h.r.rsqrt_bc2;
  h.clock = clock;
  h.wd = hyper.weight_decay;
  h.coef = hyper.coef;
  h.one = 1.f;
  const size_t state = hyper.state_bits == 8 ? 8 : 32;
  return for_tables<CAP>(
      tensors, count, h, run_length(tensors, count, hyper.state_bits == 8 ? adamw::kLongRun : adamw::kRun, sms),
      [&](const cpmtp_adamw_tensor& in, long long place, adamw::Tensor& out) {
        out.param = in.param; out.grad = in.grad; out.master = in.master;
        out.m = in.m; out.v = in.v; out.m_exp = in.m_exp; out.v_exp = in.v_exp;
        out.numel = in.numel; out.place = place;
        out.step_size = CLOCK ? in.lr_scale : adamw::step_size_of(hyper.lr, in.lr_scale, bc1);
        out.keep = CLOCK ? in.decay_scale : adamw::keep_of(hyper.lr, in.lr_scale, hyper.weight_decay, in.decay_scale);
        out.param_f32 = in.param_type == CPMTP_F32; out.grad_f32 = in.grad_type == CPMTP_F32;
        out.vec = aligned(in.param, 8 * type_bytes(in.param_type)) && aligned(in.grad, 8 * type_bytes(in.grad_type)) &&
                  aligned(in.master, 32) && aligned(in.m, state) && aligned(in.v, state);
      },
      [&](const adamw::Table<CAP>& tab, int runs) -> int {
        ProfScope prof(CPMTP_STAGE_ADAMW, st);
        if (hyper.state_bits != 8) {
          CPMTP_TRY(launch_pdl(adamw::adamw32_kernel<CAP, CLOCK>, dim3(runs), dim3(adamw::kThreads), 0, st, tab));
          return CPMTP_OK;
        }
        bool g32 = false, p32 = false;
        for (int i = 0; i < tab.count; ++i) {
          g32 |= tab.t[i].grad_f32 != 0;
          p32 |= tab.t[i].param_f32 != 0 || tab.t[i].master != nullptr;
        }
        constexpr int kPer = adamw::kWarps * adamw::kAhead;
        static bool done[64] = {};
        CPMTP_TRY(allow_smem(adamw::adamw8_kernel<CAP, CLOCK>, done, kPer * adamw::stage_bytes(true, true)));
        const int bytes = adamw::stage_bytes(g32, p32);
        CPMTP_TRY(launch_pdl(adamw::adamw8_kernel<CAP, CLOCK>, dim3(runs), dim3(adamw::kThreads), kPer * bytes, st, tab, bytes));
        return CPMTP_OK;
      });
}

template <bool CLOCK>
int adamw_step(const cpmtp_adamw_tensor* tensors, int32_t count, const cpmtp_adamw_hyper& hyper, cpmtp_adamw_clock* clock, cpmtp_stream stream) {
  DeviceInfo* di = nullptr;
  const int rd = check_device(&di);
  if (rd != CPMTP_OK) return rd;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (CLOCK) {
    ProfScope prof(CPMTP_STAGE_ADAMW, st);
    CPMTP_TRY(launch_pdl(adamw::adamw_clock_kernel, dim3(1), dim3(1), 0, st, clock, hyper.beta1, hyper.beta2));
  }
  if (count <= adamw::kSmallTable) return adamw_step<adamw::kSmallTable, CLOCK>(tensors, count, hyper, clock, di->sms, st);
  if (count <= adamw::kMiddleTable) return adamw_step<adamw::kMiddleTable, CLOCK>(tensors, count, hyper, clock, di->sms, st);
  return adamw_step<adamw::kLargeTable, CLOCK>(tensors, count, hyper, clock, di->sms, st);
}

int grad_blocks(int sms) { return 4 * sms; }

template <int CAP>
int grad_squares(const cpmtp_adamw_tensor* tensors, int32_t count, int sms, double* part, int most, int* parts, cudaStream_t st) {
  adamw::Hyper h = {};
  return for_tables<CAP>(
      tensors, count, h, run_length(tensors, count, adamw::kRun, sms),
      [&](const cpmtp_adamw_tensor& in, long long, adamw::Tensor& out) {
        std::memset(&out, 0, sizeof(out));
        out.grad = in.grad; out.numel = in.numel; out.grad_f32 = in.grad_type == CPMTP_F32;
        out.vec = aligned(in.grad, 8 * type_bytes(in.grad_type));
      },
      [&](const adamw::Table<CAP>& tab, int runs) -> int {
        const int blocks = runs < grad_blocks(sms) ? runs : grad_blocks(sms);
        if (*parts + blocks > most) return CPMTP_ERR_LIMIT;
        CPMTP_TRY(launch_pdl(adamw::grad_square_kernel<CAP>, dim3(blocks), dim3(adamw::kThreads), 0, st, tab, runs, part + *parts));
        *parts += blocks;
        return CPMTP_OK;
      });
}

}  // namespace
}  // namespace cpmtp

using namespace cpmtp;

extern "C" {

int cpmtp_embed_forward(const cpmtp_embed_shape* shape, const void* E, const int32_t* x, void* out,
                        int32_t* dev_status, cpmtp_stream stream) {
  const int rc = check_embed(shape);
  if (rc != CPMTP_OK) return rc;
  const cpmtp_embed_shape& s = *shape;
  if (s.T == 0) return CPMTP_OK;
  if (!E || !x || !out) return CPMTP_ERR_NULL;
  if (!aligned(E, 2) || !aligned(x, 4) || !aligned(out, type_bytes(s.type)) || !aligned(dev_status, 4)) return CPMTP_ERR_ALIGN;
  DeviceInfo* di = nullptr;
  const int rd = check_device(&di);
  if (rd != CPMTP_OK) return rd;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const bf16_t* table = static_cast<const bf16_t*>(E);
  const int slabs = (s.d + embed::kSlab - 1) / embed::kSlab;
  const long long items = (static_cast<long long>(s.T) + embed::kFwdRows - 1) / embed::kFwdRows * slabs;
  const long long blocks = (items + 7) / 8;
  if (blocks > 2147483647ll) return CPMTP_ERR_LIMIT;
  const dim3 grid(static_cast<unsigned>(blocks));
  ProfScope prof(CPMTP_STAGE_EMBED, st);
  auto launch = [&](auto kernel, auto* to) {
    return launch_pdl(kernel, grid, dim3(256), 0, st, table, s.ld_table, x, to, s.ld_rows, s.T, s.V, s.d, slabs, s.scale, dev_status);
  };
  const bool table_vec = io::vec_ok<bf16_t>(E, s.ld_table, s.d);
  if (s.type == CPMTP_F32) {
    float* to = static_cast<float*>(out);
    if (table_vec && io::vec_ok<float>(out, s.ld_rows, s.d)) CPMTP_TRY(launch(embed::embed_fwd_kernel<float, true>, to));
    else CPMTP_TRY(launch(embed::embed_fwd_kernel<float, false>, to));
  } else {
    bf16_t* to = static_cast<bf16_t*>(out);
    if (table_vec && io::vec_ok<bf16_t>(out, s.ld_rows, s.d)) CPMTP_TRY(launch(embed::embed_fwd_kernel<bf16_t, true>, to));
    else CPMTP_TRY(launch(embed::embed_fwd_kernel<bf16_t, false>, to));
  }
  return CPMTP_OK;
}

size_t cpmtp_embed_workspace_bytes(const cpmtp_embed_shape* shape) {
  return check_embed(shape) == CPMTP_OK && shape->T <= CPMTP_EMBED_MAX_GRAD_T ? embed_layout(*shape).total : 0;
}

int cpmtp_embed_backward(const cpmtp_embed_shape* shape, const void* dy, const int32_t* x, void* dE,
                         void* workspace, size_t workspace_bytes, int32_t* dev_status, cpmtp_stream stream) {
  const int rc = check_embed(shape);
  if (rc != CPMTP_OK) return rc;
  const cpmtp_embed_shape& s = *shape;
  const bool accum = (s.flags & CPMTP_FLAG_ACCUM_GRADS) != 0;
  if (s.T == 0 && accum) return CPMTP_OK;
  if (s.T > CPMTP_EMBED_MAX_GRAD_T) return CPMTP_ERR_LIMIT;
  const EmbedLayout L = embed_layout(s);
  if (!dE || (s.T > 0 && (!dy || !x || !workspace))) return CPMTP_ERR_NULL;
  if (!aligned(dE, 2) || !aligned(x, 4) || !aligned(dy, type_bytes(s.type)) || !aligned(workspace, kAlign) || !aligned(dev_status, 4))
    return CPMTP_ERR_ALIGN;
  if (s.T > 0 && workspace_bytes < L.total) return CPMTP_ERR_WORKSPACE;
  const long long sum_blocks = (static_cast<long long>(L.chunks) * L.slabs + 7) / 8;
  const int zero_blocks = accum ? 0 : (s.V + embed::kZeroRows - 1) / embed::kZeroRows;
  if (sum_blocks + zero_blocks > 2147483647ll) return CPMTP_ERR_LIMIT;
  DeviceInfo* di = nullptr;
  const int rd = check_device(&di);
  if (rd != CPMTP_OK) return rd;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  ProfScope prof(CPMTP_STAGE_EMBED_GRAD, st);
  const uint2* sorted = nullptr;
  if (s.T > 0) {
    uint2* keys[2] = {reinterpret_cast<uint2*>(ws + L.keys), reinterpret_cast<uint2*>(ws + L.keys) + s.T};
    if (s.T <= embed::kClusterThreads * embed::kClusterSize * 8) {
      sorted = keys[0];
      CPMTP_TRY(sort_in_cluster(x, keys[0], s.T, s.V, L, dev_status, st));
    } else {
      sorted = keys[(L.passes + 1) % 2];
      CPMTP_TRY(sort_in_memory(x, keys, reinterpret_cast<int*>(ws + L.hist), s.T, s.V, L, dev_status, st));
    }
  }
  embed::SumParams p;
  p.sorted = sorted; p.ld = s.ld_rows; p.ld_table = s.ld_table; p.dE = static_cast<bf16_t*>(dE);
  p.head = reinterpret_cast<float*>(ws + L.head); p.tail = reinterpret_cast<float*>(ws + L.tail);
  p.tokens = s.T; p.V = s.V; p.d = s.d; p.slabs = L.slabs; p.chunk = L.chunk; p.chunks = L.chunks;
  p.sum_blocks = static_cast<int>(sum_blocks); p.scale = s.scale;
  if (s.type == CPMTP_F32) CPMTP_TRY(launch_embed_sum(static_cast<const float*>(dy), p, accum, zero_blocks, st));
  else CPMTP_TRY(launch_embed_sum(static_cast<const bf16_t*>(dy), p, accum, zero_blocks, st));
  return CPMTP_OK;
}

int cpmtp_norm_forward(const cpmtp_norm_args* args, cpmtp_stream stream) {
  int rc = check_norm(args);
  if (rc != CPMTP_OK) return rc;
  const cpmtp_norm_args& a = *args;
  if (a.N == 0) return CPMTP_OK;
  const size_t sb = type_bytes(a.stream_type);
  if ((rc = check_rows(a.x, a.d, sb)) != CPMTP_OK) return rc;
  if (a.block.data != nullptr) {
    if ((rc = check_rows(a.block, a.d, 2)) != CPMTP_OK || (rc = check_rows(a.x_out, a.d, sb)) != CPMTP_OK || (rc = check_gate(a, a.gate)) != CPMTP_OK)
      return rc;
  }
  if (a.w_pre != nullptr && (rc = check_rows(a.y, a.d, 2)) != CPMTP_OK) return rc;
  if (!aligned(a.w_post, 2) || !aligned(a.w_pre, 2) || !aligned(a.rstd_post, 4) || !aligned(a.rstd_pre, 4)) return CPMTP_ERR_ALIGN;
  DeviceInfo* di = nullptr;
  if ((rc = check_device(&di)) != CPMTP_OK) return rc;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  ProfScope prof(CPMTP_STAGE_NORM, st);
  if (a.stream_type == CPMTP_F32) CPMTP_TRY(launch_norm_fwd<float>(a, di->sms, st));
  else CPMTP_TRY(launch_norm_fwd<bf16_t>(a, di->sms, st));
  return CPMTP_OK;
}

size_t cpmtp_norm_workspace_bytes(const cpmtp_norm_args* args) {
  if (check_norm(args) != CPMTP_OK) return 0;
  const int sms = sm_count();
  const int blocks[2] = {norm_bwd_blocks(*args, norm_layout(args->d, true), sms), norm_bwd_blocks(*args, norm_layout(args->d, false), sms)};
  return align_up(2 * sizeof(float) * static_cast<size_t>(blocks[0] > blocks[1] ? blocks[0] : blocks[1]) * args->d + kAlign);
}

int cpmtp_norm_backward(const cpmtp_norm_args* args, void* workspace, size_t workspace_bytes, cpmtp_stream stream) {
  int rc = check_norm(args);
  if (rc != CPMTP_OK) return rc;
  const cpmtp_norm_args& a = *args;
  const bool has_block = a.block.data != nullptr, has_y = a.dy.data != nullptr, has_post = has_block && a.w_post != nullptr;
  const bool accum = (a.flags & CPMTP_FLAG_ACCUM_GRADS) != 0;
  if (!aligned(a.w_post, 2) || !aligned(a.w_pre, 2) || !aligned(a.rstd_post, 4) || !aligned(a.rstd_pre, 4) || !aligned(a.dw_post, 2) ||
      !aligned(a.dw_pre, 2) || !aligned(workspace, kAlign))
    return CPMTP_ERR_ALIGN;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  DeviceInfo* di = nullptr;
  if (a.N == 0) {
    if (accum || (!a.dw_post && !a.dw_pre)) return CPMTP_OK;
    if ((rc = check_device(&di)) != CPMTP_OK) return rc;
    if (a.dw_post) CPMTP_TRY(cudaMemsetAsync(a.dw_post, 0, 2ull * a.d, st));
    if (a.dw_pre) CPMTP_TRY(cudaMemsetAsync(a.dw_pre, 0, 2ull * a.d, st));
    return CPMTP_OK;
  }
  if (!a.dx.data && !a.dblock.data && !a.dgate.data && !a.dw_post && !a.dw_pre) return CPMTP_ERR_NULL;   // nothing asked for
  if (a.dw_post && !has_post) return CPMTP_ERR_NULL;
  if (a.dw_pre && !has_y) return CPMTP_ERR_NULL;
  const size_t sb = type_bytes(a.stream_type);
  if ((rc = check_rows(a.x_out, a.d, sb)) != CPMTP_OK) return rc;
  if (has_y && (!a.w_pre || !a.rstd_pre)) return CPMTP_ERR_NULL;
  if (has_post && !a.rstd_post) return CPMTP_ERR_NULL;
  if (!has_y && !a.dx_out.data) return CPMTP_ERR_NULL;          // no gradient comes in
  if (has_y && (rc = check_rows(a.dy, a.d, 2)) != CPMTP_OK) return rc;
  if (a.dx_out.data && (rc = check_rows(a.dx_out, a.d, sb)) != CPMTP_OK) return rc;
  if (a.dx.data && (rc = check_rows(a.dx, a.d, sb)) != CPMTP_OK) return rc;
  if (has_block && ((rc = check_rows(a.block, a.d, 2)) != CPMTP_OK || (rc = check_gate(a, a.gate)) != CPMTP_OK)) return rc;
  if (a.dblock.data) {
    if (!has_block) return CPMTP_ERR_NULL;
    if ((rc = check_rows(a.dblock, a.d, 2)) != CPMTP_OK) return rc;
  }
  if (a.dgate.data) {
    if (a.gate_kind == CPMTP_GATE_NONE) return CPMTP_ERR_NULL;
    if ((rc = check_gate(a, a.dgate)) != CPMTP_OK) return rc;
  }
  if ((rc = check_device(&di)) != CPMTP_OK) return rc;
  int blocks = 0;
  float* part = nullptr;
  if (a.dw_post || a.dw_pre) {
    if (!workspace) return CPMTP_ERR_NULL;
    if (workspace_bytes < cpmtp_norm_workspace_bytes(args)) return CPMTP_ERR_WORKSPACE;
    part = static_cast<float*>(workspace);
  }
  ProfScope prof(CPMTP_STAGE_NORM_GRAD, st);
  if (a.stream_type == CPMTP_F32) CPMTP_TRY(launch_norm_bwd<float>(a, di->sms, blocks, part, st));
  else CPMTP_TRY(launch_norm_bwd<bf16_t>(a, di->sms, blocks, part, st));
  if (part != nullptr)
    CPMTP_TRY(launch_pdl(norm::norm_dw_kernel, dim3((a.d + 31) / 32, 2), dim3(1024), 0, st, part, blocks, a.d, static_cast<bf16_t*>(a.dw_post),
                         static_cast<bf16_t*>(a.dw_pre), accum ? 1 : 0));
  return CPMTP_OK;
}

int cpmtp_adamw_step(const cpmtp_adamw_tensor* tensors, int32_t count, const cpmtp_adamw_hyper* hyper,
                     cpmtp_stream stream) {
  const int rc = check_adamw(tensors, count, hyper);
  return rc != CPMTP_OK ? rc : adamw_step<false>(tensors, count, *hyper, nullptr, stream);
}

int cpmtp_adamw_step_clocked(const cpmtp_adamw_tensor* tensors, int32_t count, const cpmtp_adamw_hyper* hyper,
                             cpmtp_adamw_clock* clock, cpmtp_stream stream) {
  if (hyper == nullptr || clock == nullptr) return CPMTP_ERR_NULL;
  if (!aligned(clock, 8)) return CPMTP_ERR_ALIGN;
  cpmtp_adamw_hyper h = *hyper;
  h.lr = 0.0; h.step = 1; h.seed = 0;              // (the clock's)
  const int rc = check_adamw(tensors, count, &h);
  return rc != CPMTP_OK ? rc : adamw_step<true>(tensors, count, h, clock, stream);
}

int cpmtp_adamw_state_values(const void* codes, const uint8_t* exps, int64_t n, int32_t second, void* out_bf16,
                             cpmtp_stream stream) {
  if (n < 0 || n >= (1ll << 40)) return CPMTP_ERR_SHAPE;
  if (n == 0) return CPMTP_OK;
  if (!codes || !exps || !out_bf16) return CPMTP_ERR_NULL;
  if (!aligned(out_bf16, 2)) return CPMTP_ERR_ALIGN;
  DeviceInfo* di = nullptr;
  const int rd = check_device(&di);
  if (rd != CPMTP_OK) return rd;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  constexpr long long kPer = 8ll * adamw::kValueBlocks * adamw::kBlock;
  const dim3 grid(static_cast<unsigned>((n + kPer - 1) / kPer));
  const int vec = aligned(codes, 8) && aligned(out_bf16, 16);
  const uint8_t* c = static_cast<const uint8_t*>(codes);
  bf16_t* out = static_cast<bf16_t*>(out_bf16);
  ProfScope prof(CPMTP_STAGE_ADAMW, st);
  if (second) CPMTP_TRY(launch_pdl(adamw::state_values_kernel<true>, grid, dim3(adamw::kThreads), 0, st, c, exps, n, out, vec));
  else CPMTP_TRY(launch_pdl(adamw::state_values_kernel<false>, grid, dim3(adamw::kThreads), 0, st, c, exps, n, out, vec));
  return CPMTP_OK;
}

size_t cpmtp_grad_norm_workspace_bytes(const cpmtp_adamw_tensor* tensors, int32_t count) {
  if (check_grads(tensors, count) != CPMTP_OK) return 0;
  const int sms = sm_count();
  const size_t launches = (count + adamw::kLargeTable - 1) / adamw::kLargeTable + 1;
  return align_up(launches * grad_blocks(sms) * sizeof(double));
}

int cpmtp_grad_norm(const cpmtp_adamw_tensor* tensors, int32_t count, float max_norm, float* norm, float* coef,
                    void* workspace, size_t workspace_bytes, cpmtp_stream stream) {
  const int rc = check_grads(tensors, count);
  if (rc != CPMTP_OK) return rc;
  if (!(max_norm > 0.f)) return CPMTP_ERR_SHAPE;
  if (!workspace || (!norm && !coef)) return CPMTP_ERR_NULL;
  if (!aligned(workspace, kAlign) || !aligned(norm, 4) || !aligned(coef, 4)) return CPMTP_ERR_ALIGN;
  if (workspace_bytes < cpmtp_grad_norm_workspace_bytes(tensors, count)) return CPMTP_ERR_WORKSPACE;
  DeviceInfo* di = nullptr;
  const int rd = check_device(&di);
  if (rd != CPMTP_OK) return rd;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  double* part = static_cast<double*>(workspace);
  const int most = static_cast<int>(workspace_bytes / sizeof(double) < (1u << 30) ? workspace_bytes / sizeof(double) : 1u << 30);
  int parts = 0;
  ProfScope prof(CPMTP_STAGE_GRAD_NORM, st);
  const int rs = count <= adamw::kSmallTable    ? grad_squares<adamw::kSmallTable>(tensors, count, di->sms, part, most, &parts, st)
                 : count <= adamw::kMiddleTable ? grad_squares<adamw::kMiddleTable>(tensors, count, di->sms, part, most, &parts, st)
                                                : grad_squares<adamw::kLargeTable>(tensors, count, di->sms, part, most, &parts, st);
  if (rs != CPMTP_OK) return rs;
  CPMTP_TRY(launch_pdl(adamw::grad_norm_kernel, dim3(1), dim3(adamw::kThreads), 0, st, part, parts, max_norm, norm, coef));
  return CPMTP_OK;
}

}  // extern "C"
