// Host side of pr_layernorm and pr_layernorm_backward: argument checks and the launches of
// the kernels in pr_norm.cuh.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "pr_ctx.h"
#include "pr_norm.cuh"
#include "pr_norm_host.h"

using namespace prh;

namespace {

bool type_ok(pr_dtype dt) { return dt == PR_DTYPE_F32 || dt == PR_DTYPE_BF16; }
size_t esize(pr_dtype dt) { return dt == PR_DTYPE_BF16 ? 2 : 4; }
bool on_grid(const void* p, pr_dtype dt) { return reinterpret_cast<uintptr_t>(p) % esize(dt) == 0; }

// rows [n][stride] of a call that has any
bool rows_ok(const void* p, int64_t d, int64_t stride, pr_dtype dt) {
  return p && stride >= d && on_grid(p, dt);
}
// an output that is an input's buffer has its rows where the input has them
bool same_rows(const void* out, int64_t out_stride, const void* in, int64_t in_stride) {
  return out != in || out_stride == in_stride;
}

bool on_words(const void* p, int64_t stride, pr_dtype dt) {
  return !p || (aligned16(p) && stride * (int64_t)esize(dt) % 16 == 0);
}
// The kernel for rows of so many words, [of whole ones on the grid], and whether it stages them;
// threads of a row, words of each.
struct NormShape {
  const void* kernel[2];
  bool staged;
  int threads, words;
};
template <typename T, int L, int N>
NormShape forward_shape() {
  return {{reinterpret_cast<const void*>(&prk::norm_rows<T, L, N, (L > 8), false>),
           reinterpret_cast<const void*>(&prk::norm_rows<T, L, N, (L > 8), true>)}, L > 8, L, N};
}
template <typename T>
NormShape forward_of(int64_t words) {
  if (words <= 16) return forward_shape<T, 8, 2>();
  if (words <= 64) return forward_shape<T, 32, 2>();
  if (words <= 128) return forward_shape<T, 32, 4>();
  if (words <= 256) return forward_shape<T, 128, 2>();
  if (words <= 512) return forward_shape<T, 128, 4>();
  if (words <= 1024) return forward_shape<T, 256, 4>();
  if (words <= 2048) return forward_shape<T, 512, 4>();
  if constexpr (sizeof(T) == 4) {  // (wider bf16 rows: norm_wide)
    if (words <= 4096) return forward_shape<T, 512, 8>();
  }
  return {{nullptr, nullptr}, false, 0, 0};
}
template <typename T, int L, int N>
NormShape backward_shape() {
  return {{reinterpret_cast<const void*>(&prk::dnorm_rows<T, L, N, (L > 8), false>),
           reinterpret_cast<const void*>(&prk::dnorm_rows<T, L, N, (L > 8), true>)}, L > 8, L, N};
}
template <typename T>
NormShape backward_of(int64_t words, bool two_rows) {
  if (words <= 16) return backward_shape<T, 8, 2>();
  if (words <= 64) return backward_shape<T, 32, 2>();
  if (words <= 128) return backward_shape<T, 64, 2>();
  if (words <= 256) return backward_shape<T, 128, 2>();
  if (words <= 512) return backward_shape<T, 256, 2>();
  if (words <= 768 && two_rows) return backward_shape<T, 256, 3>();
  if (words <= 1024) return backward_shape<T, 512, 2>();
  if (words <= 2048) return backward_shape<T, 512, 4>();
  if constexpr (sizeof(T) == 4) {
    if (words <= 4096) return backward_shape<T, 512, 8>();
  }
  return {{nullptr, nullptr}, false, 0, 0};
}

// `ctas` CTAs on an SM (see norm_stages): whether it fits
bool stage(prk::NormArgs& a, const NormShape& shape, pr_dtype dt, int ctas, int k, int weights,
           int least, size_t& smem) {
  const int groups = shape.staged ? std::max(shape.threads, prk::NR_NT) / shape.threads : 0;
  const NormStages s = norm_stages(a.d, esize(dt), a.wide_w ? 4 : 2, groups, ctas, k, weights, least);
  a.row_bytes = s.row_bytes;
  a.stages = s.stages;
  smem = s.smem;
  return s.fits;
}

// shared memory opt-ins, once per context
pr_status setup(pr_ctx* c) {
  if (c->norm_ready) return PR_OK;
  for (int64_t words : {16, 64, 128, 256, 512, 768, 1024, 2048, 4096})
    for (const NormShape& s : {forward_of<float>(words), forward_of<__nv_bfloat16>(words),
                               backward_of<float>(words, true), backward_of<__nv_bfloat16>(words, true)})
      for (const void* kernel : s.kernel)
        if (kernel)
          PR_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       (int)norm_room(1)));
  c->norm_ready = true;
  return PR_OK;
}

pr_status launch(pr_ctx* c, const void* kernel, dim3 grid, unsigned threads, size_t smem,
                 void** args, cudaStream_t s) {
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  PR_CUDA(cudaLaunchKernelExC(&cfg, kernel, args));
  g_launches.fetch_add(1, std::memory_order_relaxed);
  return timing_mark(c, s);
}

pr_status finish(pr_ctx* c, cudaStream_t s) {
  PR_CUDA(cudaGetLastError());
  g_launches.fetch_add(1, std::memory_order_relaxed);
  return timing_mark(c, s);
}

}  // namespace

extern "C" {

pr_status pr_layernorm(pr_ctx* c, const void* x, pr_dtype dt, int64_t n_rows, int64_t d,
                       int64_t x_stride, const void* residual, int64_t residual_stride,
                       const void* weight, const void* bias, pr_dtype wdt, float eps, int32_t rms,
                       void* total, int64_t total_stride, void* y, int64_t y_stride, float* mean,
                       float* rstd, void* stream) {
  if (!c || !type_ok(dt) || !type_ok(wdt)) return PR_ERR_INVALID_ARG;
  if (n_rows < 0 || n_rows > 0x7fffffffLL || d < 1 || d > PR_NORM_MAX_D) return PR_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || !std::isfinite(eps)) return PR_ERR_INVALID_ARG;
  if (!weight || !on_grid(weight, wdt) || !on_grid(bias, wdt)) return PR_ERR_INVALID_ARG;
  if (n_rows > 0) {
    if (!rows_ok(x, d, x_stride, dt) || !rows_ok(y, d, y_stride, dt) ||
        (residual && !rows_ok(residual, d, residual_stride, dt)) ||
        (total && !rows_ok(total, d, total_stride, dt)) || y == total)
      return PR_ERR_INVALID_ARG;
    if (!same_rows(y, y_stride, x, x_stride) ||
        !same_rows(y, y_stride, residual, residual_stride) ||
        (total && (!same_rows(total, total_stride, x, x_stride) ||
                   !same_rows(total, total_stride, residual, residual_stride))))
      return PR_ERR_INVALID_ARG;
  }
  pr_status st = set_device(c);
  if (st != PR_OK) return st;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if ((st = timing_begin(c, s)) != PR_OK || n_rows == 0) return st;
  prk::NormArgs a;
  memset(&a, 0, sizeof a);
  a.x = x;
  a.res = residual;
  a.w = weight;
  a.b = bias;
  a.total = total;
  a.y = y;
  a.mean = mean;
  a.rstd = rstd;
  a.n_rows = n_rows;
  a.d = d;
  a.x_stride = x_stride;
  a.res_stride = residual_stride;
  a.total_stride = total_stride;
  a.y_stride = y_stride;
  a.eps = eps;
  a.inv_d = (float)(1.0 / (double)d);
  a.rms = rms ? 1 : 0;
  a.wide_w = wdt == PR_DTYPE_F32;
  a.vec_w = aligned16(weight) && aligned16(bias);
  a.ctx_flags = c->flags;
  const bool whole = d * (int64_t)esize(dt) % 16 == 0 && on_words(x, x_stride, dt) &&
                     on_words(residual, residual_stride, dt) && on_words(total, total_stride, dt) &&
                     on_words(y, y_stride, dt);
  const int64_t words = (d * (int64_t)esize(dt) + 15) / 16;
  const NormShape shape =
      dt == PR_DTYPE_BF16 ? forward_of<__nv_bfloat16>(words) : forward_of<float>(words);
  if (shape.threads) {
    if ((st = setup(c)) != PR_OK) return st;
    const int threads = std::max(shape.threads, prk::NR_NT), rows = threads / shape.threads;
    const int k = residual ? 2 : 1, weights = bias ? 2 : 1;
    int ctas = threads > prk::NR_NT ? 1 : 3;
    size_t smem = 0;
    a.stage_res = residual != nullptr;
    while (ctas > 1 && !stage(a, shape, dt, ctas, k, weights, 2, smem)) --ctas;
    bool fits = ctas > 1 || stage(a, shape, dt, 1, k, weights, 1, smem);
    if (!fits && residual) {
      a.stage_res = 0;
      fits = stage(a, shape, dt, 1, 1, weights, 1, smem);
    }
    if (fits) {
      if (!shape.staged) ctas = 2048 / threads;
      const int64_t grid =
          std::min<int64_t>((n_rows + rows - 1) / rows, (int64_t)c->num_sms * ctas);
      void* args[] = {&a};
      return launch(c, shape.kernel[whole], dim3((unsigned)grid), (unsigned)threads, smem, args, s);
    }
  }
  if (dt == PR_DTYPE_BF16)
    prk::norm_wide<__nv_bfloat16><<<(unsigned)n_rows, prk::NW_NT, 0, s>>>(a);
  else
    prk::norm_wide<float><<<(unsigned)n_rows, prk::NW_NT, 0, s>>>(a);
  return finish(c, s);
}

pr_status pr_layernorm_backward(pr_ctx* c, const void* dy, int64_t dy_stride, const void* x,
                                int64_t x_stride, pr_dtype dt, int64_t n_rows, int64_t d,
                                const void* weight, pr_dtype wdt, const float* mean,
                                const float* rstd, int32_t rms, const void* dtotal,
                                int64_t dtotal_stride, void* dx, int64_t dx_stride, float* dweight,
                                float* dbias, int32_t accumulate, void* stream) {
  if (!c || !type_ok(dt) || !type_ok(wdt)) return PR_ERR_INVALID_ARG;
  if (n_rows < 0 || n_rows > 0x7fffffffLL || d < 1 || d > PR_NORM_MAX_D) return PR_ERR_INVALID_ARG;
  if (!weight || !on_grid(weight, wdt) || (!dx && !dweight && !dbias)) return PR_ERR_INVALID_ARG;
  if (n_rows > 0) {
    if (!rows_ok(dy, d, dy_stride, dt) || !rows_ok(x, d, x_stride, dt) || !rstd ||
        (!mean && !rms) || (dtotal && !rows_ok(dtotal, d, dtotal_stride, dt)) ||
        (dx && !rows_ok(dx, d, dx_stride, dt)))
      return PR_ERR_INVALID_ARG;
    if (dx && (!same_rows(dx, dx_stride, dy, dy_stride) || !same_rows(dx, dx_stride, x, x_stride) ||
               !same_rows(dx, dx_stride, dtotal, dtotal_stride)))
      return PR_ERR_INVALID_ARG;
  }
  pr_status st = set_device(c);
  if (st != PR_OK) return st;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if ((st = timing_begin(c, s)) != PR_OK) return st;
  if (n_rows == 0) {
    for (float* p : {dweight, dbias})
      if (p && !accumulate) PR_CUDA(cudaMemsetAsync(p, 0, (size_t)d * sizeof(float), s));
    return PR_OK;
  }
  prk::NormArgs a;
  memset(&a, 0, sizeof a);
  a.x = x;
  a.dy = dy;
  a.res = dtotal;
  a.w = weight;
  a.y = dx;
  a.mean = const_cast<float*>(mean);
  a.rstd = const_cast<float*>(rstd);
  a.dw = dweight;
  a.db = dbias;
  a.n_rows = n_rows;
  a.d = d;
  a.x_stride = x_stride;
  a.dy_stride = dy_stride;
  a.res_stride = dtotal_stride;
  a.y_stride = dx_stride;
  a.inv_d = (float)(1.0 / (double)d);
  a.rms = rms ? 1 : 0;
  a.wide_w = wdt == PR_DTYPE_F32;
  a.accumulate = accumulate ? 1 : 0;
  a.vec_w = aligned16(weight);
  a.ctx_flags = c->flags;
  const bool whole = d * (int64_t)esize(dt) % 16 == 0 && on_words(x, x_stride, dt) &&
                     on_words(dy, dy_stride, dt) && on_words(dtotal, dtotal_stride, dt) &&
                     on_words(dx, dx_stride, dt);
  const int64_t words = (d * (int64_t)esize(dt) + 15) / 16;
  const bool two_rows = norm_two_rows(n_rows, c->num_sms, d, esize(dt), esize(wdt));
  const NormShape shape = dt == PR_DTYPE_BF16 ? backward_of<__nv_bfloat16>(words, two_rows)
                                              : backward_of<float>(words, two_rows);
  if (shape.threads) {
    if ((st = setup(c)) != PR_OK) return st;
    const int threads = std::max(shape.threads, prk::NR_NT), rows = threads / shape.threads;
    int ctas = threads > prk::NR_NT ? 1 : 2;
    size_t smem = 0;
    // Places for three rows each decide how many CTAs an SM has, whether dtotal is there or not:
    // the order of the columns' sums is to depend on the sizes alone.  Two places at least, as one
    // is filled again a row later; where those do not fit dtotal is read by its threads, and the
    // widest rows (eight words a thread) have one place.
    while (ctas > 1 && !stage(a, shape, dt, ctas, 3, 1, 2, smem)) --ctas;
    a.stage_res = dtotal && dx && stage(a, shape, dt, ctas, 3, 1, 2, smem);
    const bool fits = stage(a, shape, dt, ctas, a.stage_res ? 3 : 2, 1, shape.words == 8 ? 1 : 2,
                            smem);
    if (fits) {
      const int64_t grid =
          std::min<int64_t>((n_rows + rows - 1) / rows, (int64_t)c->num_sms * ctas);
      if (dweight || dbias) {
        if ((st = grow(c->norm_ws, (size_t)grid * 2 * d * sizeof(float), false)) != PR_OK)
          return st;
        a.part = static_cast<float*>(c->norm_ws.p);
        if (rows > 1)  // the rows' columns, added up at the end
          smem = std::max(smem, (size_t)threads * shape.words * (16 / esize(dt)) * sizeof(float));
      }
      void* args[] = {&a};
      st = launch(c, shape.kernel[whole], dim3((unsigned)grid), (unsigned)threads, smem, args, s);
      if (st != PR_OK) return st;
      if (!a.part) return PR_OK;
      int parts = (int)grid;
      void* sum_args[] = {&a, &parts};
      return launch(c, reinterpret_cast<const void*>(&prk::dnorm_sum),
                    dim3((unsigned)((d + 31) / 32), 2), prk::NS_NT, 0, sum_args, s);
    }
  }
  if (dweight || dbias) {  // first: dx may be written over dy and x
    const unsigned grid = (unsigned)((d + 31) / 32);
    if (dt == PR_DTYPE_BF16)
      prk::dnorm_columns<__nv_bfloat16><<<grid, prk::NC_NT, 0, s>>>(a);
    else
      prk::dnorm_columns<float><<<grid, prk::NC_NT, 0, s>>>(a);
    if ((st = finish(c, s)) != PR_OK) return st;
  }
  if (!dx) return PR_OK;
  if (dt == PR_DTYPE_BF16)
    prk::dnorm_wide<__nv_bfloat16><<<(unsigned)n_rows, prk::NW_NT, 0, s>>>(a);
  else
    prk::dnorm_wide<float><<<(unsigned)n_rows, prk::NW_NT, 0, s>>>(a);
  return finish(c, s);
}

}  // extern "C"
