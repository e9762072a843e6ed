// Host side of pr_distill_loss: argument checks, the context's workspace and the launches of
// the kernels in pr_distill.cuh.
#include "pr_loss_host.h"
#include "pr_distill.cuh"

using namespace prh;

static_assert(PR_MAX_LISTED == prk::DS_MAX && PR_NDIS == prk::DS_TERMS + 1, "lists, statistics");
static_assert(prk::DS_TERMS <= prk::LS_NSTAT, "the workspace's places for sums");

extern "C" {

pr_status pr_distill_loss(pr_ctx* c, const void* logits, pr_dtype dt, int64_t n_rows,
                          int64_t vocab, int64_t row_stride, const int32_t* ids,
                          const float* t_logp, int32_t k, const int32_t* chosen,
                          const uint8_t* mask, const int64_t* offsets, int32_t n_req,
                          const pr_distill* p, float* stats, float* kl, void* grad,
                          int64_t grad_stride, void* stream) {
  if (!c || !p) return PR_ERR_INVALID_ARG;
  pr_status st = check_loss(dt, logits, n_rows, vocab, row_stride, chosen, offsets, n_req,
                            p->temperature, p->grad_scale, stats, kl, grad, grad_stride);
  if (st != PR_OK) return st;
  if (vocab > PR_DISTILL_MAX_VOCAB || k < 1 || k > PR_MAX_LISTED) return PR_ERR_INVALID_ARG;
  if (n_rows > 0 && (!ids || !t_logp)) return PR_ERR_INVALID_ARG;
  if (!(p->kl_coef >= 0.f) || !std::isfinite(p->kl_coef) || !(p->ce_coef >= 0.f) ||
      !std::isfinite(p->ce_coef) || (p->ce_coef > 0.f && n_rows > 0 && !chosen))
    return PR_ERR_INVALID_ARG;
  if (!(p->temperature >= 1e-3f) || !(p->temperature <= 1e3f)) return PR_ERR_INVALID_ARG;
  if ((p->loss != PR_DISTILL_FORWARD && p->loss != PR_DISTILL_REVERSE) ||
      (p->rest != PR_REST_CLASS && p->rest != PR_REST_NONE) ||
      (p->norm != PR_NORM_TOKENS && p->norm != PR_NORM_REQUESTS))
    return PR_ERR_INVALID_ARG;
  if ((st = set_device(c)) != PR_OK) return st;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  prk::DistillArgs d;
  memset(&d, 0, sizeof d);
  fill(d.a, c, logits, n_rows, vocab, row_stride, chosen, mask, offsets, n_req, nullptr,
       p->temperature, p->grad_scale, stats, kl, grad, grad_stride);
  d.a.norm = p->norm;
  d.ids = ids;
  d.t_logp = t_logp;
  d.k = k;
  d.reverse = p->loss == PR_DISTILL_REVERSE;
  d.none = p->rest == PR_REST_NONE;
  d.kl_coef = p->kl_coef;
  d.ce_coef = p->ce_coef;
  d.big = (float)(1e9 * (double)p->temperature);
  if (n_rows == 0) {  // the requests' bounds are looked at all the same
    if ((st = timing_begin(c, s)) != PR_OK) return st;
    if (offsets && ((st = workspace(c, d.a, 0, false, false)) != PR_OK ||
                    (st = launch_plan(c, d.a, 0, s)) != PR_OK))
      return st;
    PR_CUDA(cudaMemsetAsync(stats, 0, PR_NDIS * sizeof(float), s));
    return PR_OK;
  }
  const unsigned grid = (unsigned)std::min<int64_t>(n_rows, 4 * c->num_sms);
  if ((st = workspace(c, d.a, std::max<int64_t>(grid, forward_grid(c)), false, false)) != PR_OK) return st;
  if ((st = timing_begin(c, s)) != PR_OK) return st;
  if ((st = launch_plan(c, d.a, 0, s)) != PR_OK) return st;
  void* args[] = {&d};
  const size_t smem = (size_t)(vocab + 31) / 32 * 4;
  const void* kern = dt == PR_DTYPE_BF16 ? reinterpret_cast<const void*>(&prk::distill_plain<__nv_bfloat16>)
                                         : reinterpret_cast<const void*>(&prk::distill_plain<float>);
  if (!c->distill_ready) {
    for (const void* q : {reinterpret_cast<const void*>(&prk::distill_plain<__nv_bfloat16>),
                          reinterpret_cast<const void*>(&prk::distill_plain<float>)})
      PR_CUDA(cudaFuncSetAttribute(q, cudaFuncAttributeMaxDynamicSharedMemorySize, PR_DISTILL_MAX_VOCAB / 8));
    c->distill_ready = true;
  }
  st = launch(kern, grid, prk::DL_NT, smem, 1, args, s);
  return st == PR_OK ? timing_mark(c, s) : st;
}

}  // extern "C"
