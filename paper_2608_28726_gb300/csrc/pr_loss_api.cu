// Host side of the training losses (pr_policy_loss, pr_preference_loss): argument
// checks, the context's workspace and the launches of the kernels in pr_loss.cuh.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "pr_ctx.h"
#include "pr_loss.cuh"

using namespace prh;

static_assert(sizeof(prk::OwnPlan) <= prk::RG_BYTES, "a place of the ring holds the list");
static_assert(PR_NPOL == prk::LS_NSTAT && PR_NPREF < prk::LS_NSTAT, "statistics");

namespace {

size_t esize(pr_dtype dt) { return dt == PR_DTYPE_BF16 ? 2 : 4; }

size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

pr_status check_loss(pr_dtype dt, const void* logits, int64_t n_rows, int64_t vocab,
                     int64_t row_stride, const int32_t* chosen, const int64_t* offsets,
                     int32_t n_req, float temperature, float grad_scale, const float* stats,
                     const float* logp, const void* grad, int64_t grad_stride) {
  if (dt != PR_DTYPE_F32 && dt != PR_DTYPE_BF16) return PR_ERR_INVALID_ARG;
  if (n_rows < 0 || n_rows > 0x7fffffffLL || vocab <= 0 || vocab > 0x7fffffffLL ||
      row_stride < vocab || n_req < 0)
    return PR_ERR_INVALID_ARG;
  if (!stats || (n_rows > 0 && (!logits || !chosen || !logp))) return PR_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(logits) % esize(dt) != 0) return PR_ERR_INVALID_ARG;
  if (grad && (grad_stride < vocab || reinterpret_cast<uintptr_t>(grad) % esize(dt) != 0 ||
               (grad == logits && grad_stride != row_stride)))
    return PR_ERR_INVALID_ARG;
  if (offsets ? n_req < 1 : n_req != 0) return PR_ERR_INVALID_ARG;
  // log2(e) / T and 1 / T have to be finite, and not zero
  if (!(temperature >= 1e-30f) || !(temperature <= 1e30f) || !std::isfinite(grad_scale))
    return PR_ERR_INVALID_ARG;
  return PR_OK;
}

int64_t forward_grid(const pr_ctx* c) { return (int64_t)c->num_sms * prk::FW_CTAS; }

// The workspace: what is zero between calls, [tickets, totals][arrivals per row], and the
// rest, [per CTA][per request][per pair][per row][per group].  Neither is freed before the
// context is: a captured graph may hold them.
pr_status workspace(pr_ctx* c, prk::LossArgs& a, int64_t groups, bool pref, bool state) {
  const size_t n_req = (size_t)a.n_req, n_rows = (size_t)a.n_rows;
  const size_t at_count = (size_t)forward_grid(c) * 16, at_coef = at_count + up16(n_req * 4),
               at_term = at_coef + up16(pref ? n_req * 4 : 0),
               at_req = at_term + up16(pref ? n_req / 2 * prk::LS_NSTAT * 4 : 0),
               at_block = at_req + up16(n_rows * 4),
               at_list = at_block + up16((n_rows / prk::PL_BLOCK + 1) * 4),
               at_skipped = at_list + n_rows * 16,
               at_state = at_skipped + up16(n_rows * 4),
               at_z = at_state + (state ? n_rows * 16 : 0),
               at_part = at_z + up16(state ? n_rows * 4 : 0),
               bytes = at_part + (pref ? 0 : (size_t)groups * prk::LS_NSTAT * 8);
  pr_status st = grow(c->loss_zero, 64 + n_rows * 4, true);
  if (st != PR_OK || (st = grow(c->loss_ws, bytes, false)) != PR_OK) return st;
  char* const z = static_cast<char*>(c->loss_zero.p);
  a.ticket = reinterpret_cast<int32_t*>(z);
  a.totals = reinterpret_cast<int64_t*>(z + 16);
  a.arrived = reinterpret_cast<int32_t*>(z + 64);
  char* const w = static_cast<char*>(c->loss_ws.p);
  a.piece = reinterpret_cast<float2*>(w);
  a.count = reinterpret_cast<int32_t*>(w + at_count);
  a.coef = reinterpret_cast<float*>(w + at_coef);
  a.term = reinterpret_cast<float*>(w + at_term);
  a.row_req = reinterpret_cast<int32_t*>(w + at_req);
  a.block = reinterpret_cast<int32_t*>(w + at_block);
  a.list = reinterpret_cast<int4*>(w + at_list);
  a.skipped = reinterpret_cast<int32_t*>(w + at_skipped);
  a.state = state ? reinterpret_cast<float4*>(w + at_state) : nullptr;
  a.z = state ? reinterpret_cast<float*>(w + at_z) : nullptr;
  a.part = reinterpret_cast<double*>(w + at_part);
  return PR_OK;
}

// early: set up while the kernel before it still runs
pr_status launch(const void* kern, unsigned grid, unsigned threads, size_t smem, unsigned cluster,
                 void** args, cudaStream_t s, bool early = true) {
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (early) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (cluster > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = cluster;
    attr[n].val.clusterDim.y = 1;
    attr[n++].val.clusterDim.z = 1;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  PR_CUDA(cudaLaunchKernelExC(&cfg, kern, args));
  g_launches.fetch_add(1, std::memory_order_relaxed);
  return PR_OK;
}

size_t ring_bytes(int places, int cluster, bool own) {
  return prk::ring_start(cluster) + (size_t)places * prk::RG_BYTES +
         (own ? sizeof(prk::OwnPlan) : 0);
}

bool own_list(const prk::LossArgs& a) {
  return a.n_rows > 0 && a.n_rows <= prk::OWN_MOST && a.n_req <= prk::OWN_MOST;
}

template <typename T, bool HOLD>
const void* ring_kernel(bool own) {
  return own ? reinterpret_cast<const void*>(&prk::loss_ring<T, HOLD, true>)
             : reinterpret_cast<const void*>(&prk::loss_ring<T, HOLD, false>);
}

const void* ring_kernel(pr_dtype dt, bool hold, bool own) {
  if (dt == PR_DTYPE_BF16)
    return hold ? ring_kernel<__nv_bfloat16, true>(own) : ring_kernel<__nv_bfloat16, false>(own);
  return hold ? ring_kernel<float, true>(own) : ring_kernel<float, false>(own);
}

template <typename T>
const void* forward_kernel(bool pref) {
  return pref ? reinterpret_cast<const void*>(&prk::loss_forward<T, true>)
              : reinterpret_cast<const void*>(&prk::loss_forward<T, false>);
}

template <typename T>
const void* rows_kernel(bool pref, bool hold) {
  return pref   ? reinterpret_cast<const void*>(&prk::loss_rows<T, true, false>)
         : hold ? reinterpret_cast<const void*>(&prk::loss_rows<T, false, true>)
                : reinterpret_cast<const void*>(&prk::loss_rows<T, false, false>);
}

const void* rows_kernel(pr_dtype dt, bool pref, bool hold) {
  return dt == PR_DTYPE_BF16 ? rows_kernel<__nv_bfloat16>(pref, hold)
                             : rows_kernel<float>(pref, hold);
}

// half of an SM's shared memory
constexpr size_t HALF = prk::ring_start(4) + (size_t)prk::RG_FEW * prk::RG_BYTES;

// shared memory opt-ins, and the clusters of 2, 4 and 8 CTAs that the GPU has room for
// with half and with all of an SM's shared memory each; once per context
pr_status ring_setup(pr_ctx* c) {
  if (c->loss_ready) return PR_OK;
  for (pr_dtype dt : {PR_DTYPE_F32, PR_DTYPE_BF16})
    for (bool hold : {false, true})
      for (bool own : {false, true})
        PR_CUDA(cudaFuncSetAttribute(ring_kernel(dt, hold, own),
                                     cudaFuncAttributeMaxDynamicSharedMemorySize,
                                     (int)ring_bytes(prk::RG_MOST, 8, false)));
  for (pr_dtype dt : {PR_DTYPE_F32, PR_DTYPE_BF16})
    for (int kind = 0; kind < 3; ++kind)
      PR_CUDA(cudaFuncSetAttribute(rows_kernel(dt, kind == 2, kind == 1),
                                   cudaFuncAttributeMaxDynamicSharedMemorySize, (int)HALF));
  for (int i = 0; i < 4; ++i)
    for (int whole = 0; whole < 2; ++whole) {
      if (i == 0) {
        c->loss_places[whole][0] = c->num_sms * (whole ? 1 : 2);
        continue;
      }
      cudaLaunchConfig_t cfg;
      memset(&cfg, 0, sizeof cfg);
      cfg.gridDim = dim3(1u << i);
      cfg.blockDim = dim3(prk::RG_NT);
      cfg.dynamicSmemBytes = ring_bytes(whole ? prk::RG_MOST : prk::RG_FEW, 1 << i, false);
      cudaLaunchAttribute attr[1];
      attr[0].id = cudaLaunchAttributeClusterDimension;
      attr[0].val.clusterDim.x = 1u << i;
      attr[0].val.clusterDim.y = 1;
      attr[0].val.clusterDim.z = 1;
      cfg.attrs = attr;
      cfg.numAttrs = 1;
      int n = 0;
      PR_CUDA(cudaOccupancyMaxActiveClusters(&n, ring_kernel(PR_DTYPE_BF16, true, false), &cfg));
      c->loss_places[whole][i] = std::max(n, 1);
    }
  c->loss_ready = true;
  return PR_OK;
}

// The one-pass kernel's launch: 2^split CTAs per row, `places` chunks in a CTA's ring.
struct RingShape {
  int split, places;
  int here;         // chunks of a row's part
  bool hold;        // a row's chunks fit the cluster's rings
  bool spare;       // and leave a place free
  bool full;        // every place is taken
  int64_t groups;   // rows in work at a time
};

// Of the launches whose CTAs hold a row, with two places left for the next row's chunks,
// the one that takes the least time by this count, in the time that an SM takes for a
// chunk: each cluster's rows come one after the other, a row takes its CTA's chunks and about
// three for its end, which two CTAs on an SM hide from one another.  The same with and
// without a gradient, so that the losses' bits are.
RingShape choose_ring(const pr_ctx* c, pr_dtype dt, int64_t n_rows, int64_t vocab) {
  const int64_t words = vocab * (int64_t)esize(dt) / 16;
  const int64_t chunks = (words + prk::RG_CHUNK - 1) / prk::RG_CHUNK;
  RingShape s;
  s.split = 3;
  s.places = prk::RG_MOST;
  int64_t best = -1;
  for (int whole = 0; whole < 2; ++whole)
    for (int split = 0; split < (whole ? 4 : 3); ++split) {
      const int64_t here = (chunks + (1 << split) - 1) >> split, at_once = c->loss_places[whole][split];
      const int places = whole ? prk::RG_MOST : prk::RG_FEW;
      if (here > places - 2) continue;
      const int64_t time = (n_rows + at_once - 1) / at_once *
                           (whole ? here + 3 : std::max(2 * here, here + 3));
      if (best < 0 || time < best) {
        best = time;
        s.split = split;
        s.places = places;
      }
    }
  const int64_t at_once = c->loss_places[s.places == prk::RG_MOST][s.split];
  s.here = (int)std::min<int64_t>((chunks + (1 << s.split) - 1) >> s.split, prk::RG_MOST + 1);
  s.hold = s.here <= s.places;
  s.spare = s.here < s.places;
  s.groups = std::min<int64_t>(n_rows, at_once);
  s.full = n_rows >= at_once;
  return s;
}

// One CTA where it takes no longer than the second launch (about 3 us) that many need.
pr_status launch_plan(pr_ctx* c, prk::LossArgs& a, int pairs, cudaStream_t s) {
  if (a.own) return PR_OK;
  void* args[] = {&a, &pairs};
  if (a.n_rows <= 4 * prk::PL_BLOCK && a.n_req <= prk::PL_FEW) {
    const pr_status st = launch(reinterpret_cast<const void*>(&prk::loss_plan), 1, prk::PL_BLOCK, 0,
                                1, args, s);
    return st == PR_OK ? timing_mark(c, s) : st;
  }
  const int64_t blocks = (a.n_rows + prk::PL_BLOCK - 1) / prk::PL_BLOCK, grid = a.n_req + blocks;
  if (grid > 0x7fffffffLL) return PR_ERR_INVALID_ARG;
  pr_status st = launch(reinterpret_cast<const void*>(&prk::loss_count), (unsigned)grid,
                        prk::PL_BLOCK, 0, 1, args, s);
  if (st != PR_OK || (st = timing_mark(c, s)) != PR_OK || blocks == 0) return st;
  st = launch(reinterpret_cast<const void*>(&prk::loss_list), (unsigned)blocks, prk::PL_BLOCK, 0, 1,
              args, s);
  return st == PR_OK ? timing_mark(c, s) : st;
}

pr_status launch_ring(pr_ctx* c, prk::LossArgs& a, pr_dtype dt, const RingShape& shape, bool hold,
                      cudaStream_t s) {
  int places = shape.places - (a.own ? 1 : 0);  // (the rows' list takes one)
  int lag = shape.split == 0 && 2 * shape.here + 1 <= places ? 1 : 0;
  void* args[] = {&a, &places, &lag};
  // A grid that takes every place is not set up early: clusters placed around the CTAs
  // of the launch before do not all find one, and the last run alone (8,657 rows of V =
  // 151,936 bf16 back to back: 1,538 us, 890 set up after it).
  const pr_status st = launch(ring_kernel(dt, hold, a.own), (unsigned)(shape.groups << shape.split),
                              prk::RG_NT, ring_bytes(places, 1 << shape.split, a.own), 1u << shape.split, args, s,
                              !shape.full);
  return st == PR_OK ? timing_mark(c, s) : st;
}

// Warps of a CTA of loss_rows, or 0 where the other kernels take less time: with fewer than
// ten rows of an SM in work (rows of over 22 KB), or no more than two rows for each of the
// CTAs that have a row each (620 rows of V = 8,192 bf16: 27 us for 25, 1,500: 29 for 33).
int rows_warps(const pr_ctx* c, const prk::LossArgs& a, pr_dtype dt) {
  if (a.own || a.n_rows <= 4 * c->num_sms) return 0;
  const int64_t part = std::max<int64_t>(16, a.vocab * (int64_t)esize(dt) / 16 * 16);
  const int64_t w = std::min<int64_t>(prk::RW_MOST, ((int64_t)HALF - (int64_t)prk::RW_CTL) / part);
  return w >= 5 ? (int)w : 0;
}

pr_status launch_rows(pr_ctx* c, prk::LossArgs& a, pr_dtype dt, int warps, bool pref, bool hold,
                      cudaStream_t s) {
  int part = (int)std::max<int64_t>(16, a.vocab * (int64_t)esize(dt) / 16 * 16);
  void* args[] = {&a, &part};
  const pr_status st = launch(rows_kernel(dt, pref, hold),
                              (unsigned)std::min<int64_t>(2 * c->num_sms, a.n_rows), 32u * warps,
                              prk::RW_CTL + (size_t)warps * part, 1, args, s);
  return st == PR_OK ? timing_mark(c, s) : st;
}

pr_status launch_forward(pr_ctx* c, prk::LossArgs& a, pr_dtype dt, bool pref, cudaStream_t s) {
  void* args[] = {&a};
  const pr_status st = launch(dt == PR_DTYPE_BF16 ? forward_kernel<__nv_bfloat16>(pref)
                                                  : forward_kernel<float>(pref),
                              (unsigned)forward_grid(c), prk::FW_NT, a.own ? sizeof(prk::OwnPlan) : 0, 1,
                              args, s);
  return st == PR_OK ? timing_mark(c, s) : st;
}

pr_status launch_backward(pr_ctx* c, prk::LossArgs& a, pr_dtype dt, bool pref, cudaStream_t s) {
  const int64_t words = (a.vocab * (int64_t)esize(dt)) / 16;
  int32_t segs = (int32_t)std::max<int64_t>(1, (words + prk::BW_SEG - 1) / prk::BW_SEG);
  if (a.n_rows * segs > 0x7fffffffLL) return PR_ERR_INVALID_ARG;
  void* args[] = {&a, &segs};
  const void* kern =
      dt == PR_DTYPE_BF16
          ? (pref ? reinterpret_cast<const void*>(&prk::loss_backward<__nv_bfloat16, true>)
                  : reinterpret_cast<const void*>(&prk::loss_backward<__nv_bfloat16, false>))
          : (pref ? reinterpret_cast<const void*>(&prk::loss_backward<float, true>)
                  : reinterpret_cast<const void*>(&prk::loss_backward<float, false>));
  const pr_status st = launch(kern, (unsigned)(a.n_rows * segs), prk::BW_NT, 0, 1, args, s);
  return st == PR_OK ? timing_mark(c, s) : st;
}

void fill(prk::LossArgs& a, pr_ctx* c, const void* logits, int64_t n_rows, int64_t vocab,
          int64_t row_stride, const int32_t* chosen, const uint8_t* mask, const int64_t* offsets,
          int32_t n_req, const float* ref_logp, float temperature, float grad_scale, float* stats,
          float* logp, void* grad, int64_t grad_stride) {
  memset(&a, 0, sizeof a);
  a.logits = logits;
  a.n_rows = n_rows;
  a.vocab = vocab;
  a.row_stride = row_stride;
  a.chosen = chosen;
  a.mask = mask;
  a.offsets = offsets;
  a.n_req = offsets ? n_req : 1;
  a.ref_logp = ref_logp;
  a.inv_t = (float)(1.0 / (double)temperature);
  a.c2 = (float)(1.4426950408889634 / (double)temperature);
  a.grad_scale = grad_scale;
  a.stats = stats;
  a.logp = logp;
  a.grad = grad;
  a.grad_stride = grad_stride;
  a.ctx_flags = c->flags;
}

}  // namespace

extern "C" {

pr_status pr_policy_loss(pr_ctx* c, const void* logits, pr_dtype dt, int64_t n_rows,
                         int64_t vocab, int64_t row_stride, const int32_t* chosen,
                         const uint8_t* mask, const int64_t* offsets, int32_t n_req,
                         const float* old_logp, const float* ref_logp, const float* advantage,
                         const pr_policy* p, float* stats, float* logp, void* grad,
                         int64_t grad_stride, void* stream) {
  if (!c || !p) return PR_ERR_INVALID_ARG;
  pr_status st = check_loss(dt, logits, n_rows, vocab, row_stride, chosen, offsets, n_req,
                            p->temperature, p->grad_scale, stats, logp, grad, grad_stride);
  if (st != PR_OK) return st;
  if (n_rows > 0 && !advantage) return PR_ERR_INVALID_ARG;
  if (!(p->clip_low >= 0.f) || !(p->clip_low <= 1.f) || !(p->clip_high >= 0.f) ||
      !(p->kl_coef >= 0.f) || !std::isfinite(p->kl_coef))
    return PR_ERR_INVALID_ARG;
  if (p->norm != PR_NORM_TOKENS && p->norm != PR_NORM_REQUESTS) return PR_ERR_INVALID_ARG;
  if (p->adv_per_request && !offsets) return PR_ERR_INVALID_ARG;
  if ((st = set_device(c)) != PR_OK) return st;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  prk::LossArgs a;
  fill(a, c, logits, n_rows, vocab, row_stride, chosen, mask, offsets, n_req, ref_logp,
       p->temperature, p->grad_scale, stats, logp, grad, grad_stride);
  a.old_logp = old_logp;
  a.adv = advantage;
  a.per_request = p->adv_per_request ? 1 : 0;
  a.norm = p->norm;
  a.clip_lo = 1.f - p->clip_low;
  a.clip_hi = 1.f + p->clip_high;
  a.kl_coef = p->kl_coef;
  if (n_rows == 0) {  // the requests' bounds are looked at all the same
    if ((st = timing_begin(c, s)) != PR_OK) return st;
    if (offsets && ((st = workspace(c, a, 0, false, false)) != PR_OK ||
                    (st = launch_plan(c, a, 0, s)) != PR_OK))
      return st;
    PR_CUDA(cudaMemsetAsync(stats, 0, PR_NPOL * sizeof(float), s));
    return PR_OK;
  }
  if ((st = ring_setup(c)) != PR_OK) return st;
  const RingShape ring = choose_ring(c, dt, n_rows, vocab);
  if ((st = workspace(c, a, std::max(ring.groups, forward_grid(c)), false, !ring.hold)) != PR_OK)
    return st;
  a.own = own_list(a) && (!ring.hold || ring.spare);
  if ((st = timing_begin(c, s)) != PR_OK) return st;
  if ((st = launch_plan(c, a, 0, s)) != PR_OK) return st;
  if (const int warps = rows_warps(c, a, dt))
    return launch_rows(c, a, dt, warps, false, grad != nullptr, s);
  if (ring.hold) return launch_ring(c, a, dt, ring, grad != nullptr, s);
  // rows of more than eight SMs' shared memory
  if ((st = launch_forward(c, a, dt, false, s)) != PR_OK) return st;
  return grad ? launch_backward(c, a, dt, false, s) : PR_OK;
}

pr_status pr_preference_loss(pr_ctx* c, const void* logits, pr_dtype dt, int64_t n_rows,
                             int64_t vocab, int64_t row_stride, const int32_t* chosen,
                             const uint8_t* mask, const int64_t* offsets, int32_t n_req,
                             const float* ref_logp, const pr_preference* p, float* stats,
                             float* ratio, float* logp, void* grad, int64_t grad_stride,
                             void* stream) {
  if (!c || !p) return PR_ERR_INVALID_ARG;
  pr_status st = check_loss(dt, logits, n_rows, vocab, row_stride, chosen, offsets, n_req,
                            p->temperature, p->grad_scale, stats, logp, grad, grad_stride);
  if (st != PR_OK) return st;
  if (!offsets || n_req % 2 != 0 || !ratio) return PR_ERR_INVALID_ARG;
  if (p->loss != PR_PREF_SIGMOID && p->loss != PR_PREF_SQUARED && p->loss != PR_PREF_HINGE)
    return PR_ERR_INVALID_ARG;
  if (!(p->beta > 0.f) || !std::isfinite(p->beta) || !std::isfinite(p->margin) ||
      !(p->label_smoothing >= 0.f) || !(p->label_smoothing <= 1.f) ||
      (p->loss != PR_PREF_SIGMOID && p->label_smoothing != 0.f) ||
      (p->loss == PR_PREF_SQUARED && p->margin != 0.f))
    return PR_ERR_INVALID_ARG;
  if ((st = set_device(c)) != PR_OK) return st;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  prk::LossArgs a;
  fill(a, c, logits, n_rows, vocab, row_stride, chosen, mask, offsets, n_req, ref_logp,
       p->temperature, p->grad_scale, stats, logp, grad, grad_stride);
  a.ratio = ratio;
  a.beta = p->beta;
  a.smooth = p->label_smoothing;
  a.margin = p->margin;
  a.loss = p->loss;
  a.length_norm = p->length_norm ? 1 : 0;
  if ((st = ring_setup(c)) != PR_OK) return st;
  if ((st = workspace(c, a, 0, true, true)) != PR_OK) return st;
  a.own = own_list(a);
  if ((st = timing_begin(c, s)) != PR_OK) return st;
  if ((st = launch_plan(c, a, 1, s)) != PR_OK) return st;
  const int warps = rows_warps(c, a, dt);
  if (n_rows > 0 && (st = warps ? launch_rows(c, a, dt, warps, true, false, s)
                                : launch_forward(c, a, dt, true, s)) != PR_OK)
    return st;
  void* args[] = {&a};
  if ((st = launch(reinterpret_cast<const void*>(&prk::loss_pairs), 
                   (unsigned)((n_req / 2 + prk::PR_PAIRS - 1) / prk::PR_PAIRS), 64 * prk::PR_PAIRS, 0, 1,
                   args, s)) != PR_OK ||
      (st = timing_mark(c, s)) != PR_OK)
    return st;
  return grad && n_rows > 0 ? launch_backward(c, a, dt, true, s) : PR_OK;
}

}  // extern "C"
