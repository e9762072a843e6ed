// Host side of the training losses (pr_policy_loss, pr_preference_loss): argument
// checks, the context's workspace and the launches of the kernels in pr_loss.cuh.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "pr_loss_host.h"

using namespace prh;

static_assert(sizeof(prk::OwnPlan) <= prk::RG_BYTES, "a place of the ring holds the list");
static_assert(PR_NPOL == prk::LS_NSTAT && PR_NPREF < prk::LS_NSTAT, "statistics");

namespace {

size_t ring_bytes(int places, int cluster, bool own) {
  return prk::ring_start(cluster) + (size_t)places * prk::RG_BYTES +
         (own ? sizeof(prk::OwnPlan) : 0);
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

}  // namespace

extern "C" {

pr_status pr_policy_loss(pr_ctx* c, const void* logits, pr_dtype dt, int64_t n_rows,
                         int64_t vocab, int64_t row_stride, const int32_t* chosen,
                         const uint8_t* mask, const int64_t* offsets, int32_t n_req,
                         const float* old_logp, const float* ref_logp, const float* advantage,
                         const pr_policy* p, float* stats, float* logp, void* grad,
                         int64_t grad_stride, void* stream) {
  if (!c || !p) return PR_ERR_INVALID_ARG;
  pr_status st = check_loss(dt, logits, n_rows, vocab, row_stride, offsets, n_req,
                            p->temperature, p->grad_scale, stats, logp, grad, grad_stride);
  if (st != PR_OK) return st;
  if (n_rows > 0 && (!chosen || !advantage)) return PR_ERR_INVALID_ARG;
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
  const RingShape ring = choose_ring(c->loss_places, dt, n_rows, vocab);
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
  pr_status st = check_loss(dt, logits, n_rows, vocab, row_stride, offsets, n_req,
                            p->temperature, p->grad_scale, stats, logp, grad, grad_stride);
  if (st != PR_OK) return st;
  if (!offsets || n_req % 2 != 0 || !ratio || (n_rows > 0 && !chosen)) return PR_ERR_INVALID_ARG;
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
