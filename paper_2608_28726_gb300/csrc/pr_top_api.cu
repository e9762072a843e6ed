// Host side of pr_top_logits: argument checks and the launches of the kernels in pr_top.cuh.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "pr_ctx.h"
#include "pr_top.cuh"

using namespace prh;

static_assert(PR_MAX_LISTED == prk::TP_MAX, "list length");

extern "C" {

pr_status pr_top_logits(pr_ctx* c, const void* logits, pr_dtype dt, int64_t n_rows, int64_t vocab,
                        int64_t row_stride, int32_t k, float temperature, int32_t* ids,
                        float* logp, void* stream) {
  if (!c || (dt != PR_DTYPE_F32 && dt != PR_DTYPE_BF16)) return PR_ERR_INVALID_ARG;
  if (n_rows < 0 || n_rows > 0x7fffffffLL || vocab <= 0 || vocab > 0x7fffffffLL ||
      row_stride < vocab || k < 1 || k > PR_MAX_LISTED)
    return PR_ERR_INVALID_ARG;
  if (n_rows > 0 && (!logits || !ids || !logp)) return PR_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(logits) % (dt == PR_DTYPE_BF16 ? 2 : 4) != 0)
    return PR_ERR_INVALID_ARG;
  if (!(temperature >= 1e-3f) || !(temperature <= 1e3f)) return PR_ERR_INVALID_ARG;
  pr_status st = set_device(c);
  if (st != PR_OK) return st;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if ((st = timing_begin(c, s)) != PR_OK || n_rows == 0) return st;
  prk::TopArgs a;
  a.logits = logits;
  a.n_rows = n_rows;
  a.vocab = vocab;
  a.row_stride = row_stride;
  a.k = k;
  a.c2 = (float)(1.4426950408889634 / (double)temperature);
  a.big = (float)(1e9 * (double)temperature);
  a.ids = ids;
  a.logp = logp;
  a.ctx_flags = c->flags;
  const int64_t group = std::max<int64_t>(32, (vocab + prk::TP_GROUPS - 1) / prk::TP_GROUPS);
  if (dt == PR_DTYPE_BF16)
    prk::top_rows<__nv_bfloat16><<<(unsigned)n_rows, prk::TP_NT, 0, s>>>(a, group);
  else
    prk::top_rows<float><<<(unsigned)n_rows, prk::TP_NT, 0, s>>>(a, group);
  PR_CUDA(cudaGetLastError());
  g_launches.fetch_add(1, std::memory_order_relaxed);
  return timing_mark(c, s);
}

}  // extern "C"
