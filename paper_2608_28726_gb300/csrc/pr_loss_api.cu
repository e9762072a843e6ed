// Host side of the training losses (pr_policy_loss, pr_preference_loss): argument
// checks, the context's workspace and the launches of the kernels in pr_loss.cuh.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "pr_ctx.h"
#include "pr_loss.cuh"

using namespace prh;

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

// the workspace: [tickets, totals][per request][per pair][per row][per group]
pr_status workspace(pr_ctx* c, prk::LossArgs& a, int64_t n_req, int64_t groups, bool pref) {
  const size_t at_count = 64, at_coef = at_count + up16((size_t)n_req * 4),
               at_term = at_coef + up16(pref ? (size_t)n_req * 4 : 0),
               at_state = at_term + up16(pref ? (size_t)(n_req / 2) * prk::LS_NSTAT * 4 : 0),
               at_part = at_state + (pref ? (size_t)a.n_rows * 16 : 0),
               bytes = at_part + (pref ? 0 : (size_t)groups * prk::LS_NSTAT * 8);
  if (bytes > c->loss_ws_bytes) {
    PR_CUDA(cudaDeviceSynchronize());  // kernels may still use the old one
    cudaFree(c->loss_ws);
    c->loss_ws = nullptr;
    c->loss_ws_bytes = 0;
    const size_t room = bytes + bytes / 4;
    if (cudaMalloc(&c->loss_ws, room) != cudaSuccess) {
      cudaGetLastError();
      c->loss_ws = nullptr;
      return PR_ERR_NO_MEMORY;
    }
    PR_CUDA(cudaMemset(c->loss_ws, 0, room));
    PR_CUDA(cudaDeviceSynchronize());
    c->loss_ws_bytes = room;
  }
  char* w = static_cast<char*>(c->loss_ws);
  a.ticket = reinterpret_cast<int32_t*>(w);
  a.totals = reinterpret_cast<int64_t*>(w + 16);
  a.count = reinterpret_cast<int32_t*>(w + at_count);
  a.coef = reinterpret_cast<float*>(w + at_coef);
  a.term = reinterpret_cast<float*>(w + at_term);
  a.state = reinterpret_cast<float4*>(w + at_state);
  a.part = reinterpret_cast<double*>(w + at_part);
  return PR_OK;
}

pr_status launch(const void* kern, dim3 grid, unsigned threads, void** args, cudaStream_t s) {
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  PR_CUDA(cudaLaunchKernelExC(&cfg, kern, args));
  g_launches.fetch_add(1, std::memory_order_relaxed);
  return PR_OK;
}

template <int KIND>
const void* row_kernel(pr_dtype dt) {
  return dt == PR_DTYPE_BF16 ? reinterpret_cast<const void*>(&prk::loss_rows<__nv_bfloat16, KIND>)
                             : reinterpret_cast<const void*>(&prk::loss_rows<float, KIND>);
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
  a.skew = (float)((double)a.c2 * 0.6931471805599453 - (double)a.inv_t);
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
  if (n_rows == 0) {
    PR_CUDA(cudaMemsetAsync(stats, 0, PR_NPOL * sizeof(float), s));
    return PR_OK;
  }
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
  const int64_t grid = std::min<int64_t>(n_rows, (int64_t)c->num_sms * 4);
  if ((st = workspace(c, a, a.n_req, grid, false)) != PR_OK) return st;
  if ((st = timing_begin(c, s)) != PR_OK) return st;
  int pairs = 0;
  void* pargs[] = {&a, &pairs};
  if ((st = launch(reinterpret_cast<const void*>(&prk::loss_plan), dim3((unsigned)a.n_req), 256,
                   pargs, s)) != PR_OK)
    return st;
  if ((st = timing_mark(c, s)) != PR_OK) return st;
  void* args[] = {&a};
  if ((st = launch(row_kernel<prk::LOSS_POLICY>(dt), dim3((unsigned)grid), prk::LS_NT, args, s)) !=
      PR_OK)
    return st;
  return timing_mark(c, s);
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
  const int64_t grid = std::min<int64_t>(std::max<int64_t>(n_rows, 1), (int64_t)c->num_sms * 4);
  if ((st = workspace(c, a, n_req, 0, true)) != PR_OK) return st;
  if ((st = timing_begin(c, s)) != PR_OK) return st;
  int pairs = 1;
  void* pargs[] = {&a, &pairs};
  if ((st = launch(reinterpret_cast<const void*>(&prk::loss_plan), dim3((unsigned)n_req), 256,
                   pargs, s)) != PR_OK)
    return st;
  if ((st = timing_mark(c, s)) != PR_OK) return st;
  void* args[] = {&a};
  if ((st = launch(row_kernel<prk::LOSS_PREF_FWD>(dt), dim3((unsigned)grid), prk::LS_NT, args,
                   s)) != PR_OK)
    return st;
  if ((st = timing_mark(c, s)) != PR_OK) return st;
  if ((st = launch(reinterpret_cast<const void*>(&prk::loss_pairs),
                   dim3((unsigned)((n_req / 2 + 7) / 8)), 256, args, s)) != PR_OK)
    return st;
  if ((st = timing_mark(c, s)) != PR_OK) return st;
  if (grad && n_rows > 0) {
    if ((st = launch(row_kernel<prk::LOSS_PREF_BWD>(dt), dim3((unsigned)grid), prk::LS_NT, args,
                     s)) != PR_OK)
      return st;
    return timing_mark(c, s);
  }
  return PR_OK;
}

}  // extern "C"
