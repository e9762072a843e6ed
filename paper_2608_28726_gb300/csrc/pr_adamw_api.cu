// Host side of the optimiser step (pr_adamw_step, pr_adamw_unpack): argument checks,
// the tensors of each launch and the launches of the kernels in pr_adamw.cuh.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <type_traits>

#include "pr_adamw.cuh"
#include "pr_ctx.h"

using namespace prh;

static_assert(prk::AW_BLOCK == PR_ADAMW_BLOCK, "block of an 8-bit state");
static_assert(sizeof(prk::AdamwArgs<prk::AW_MANY>) <= 32764, "kernel parameters");

namespace {

bool fits(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

size_t esize(int32_t dt) { return dt == PR_DTYPE_BF16 ? 2 : 4; }

pr_status check(const pr_adamw_tensor& t) {
  if (t.n < 0 || t.n > (int64_t)1 << 42) return PR_ERR_INVALID_ARG;
  if ((t.param_dtype != PR_DTYPE_F32 && t.param_dtype != PR_DTYPE_BF16) ||
      (t.grad_dtype != PR_DTYPE_F32 && t.grad_dtype != PR_DTYPE_BF16) ||
      (t.state_bits != 8 && t.state_bits != 32) || !std::isfinite(t.weight_decay))
    return PR_ERR_INVALID_ARG;
  if (t.master && t.param_dtype != PR_DTYPE_BF16) return PR_ERR_INVALID_ARG;
  if (t.n == 0) return PR_OK;
  if (!t.param || !t.grad || !t.m || !t.v || !fits(t.param, esize(t.param_dtype)) ||
      !fits(t.grad, esize(t.grad_dtype)) || !fits(t.master, 4))
    return PR_ERR_INVALID_ARG;
  if (t.state_bits == 8) {
    if (!t.m_scale || !t.v_scale || !fits(t.m_scale, 4) || !fits(t.v_scale, 4))
      return PR_ERR_INVALID_ARG;
  } else if (t.m_scale || t.v_scale || !fits(t.m, 4) || !fits(t.v, 4)) {
    return PR_ERR_INVALID_ARG;
  }
  return PR_OK;
}

// the kernel's instantiation: parameters, master copy, gradients, bits
int kind_of(const pr_adamw_tensor& t) {
  return (t.param_dtype == PR_DTYPE_BF16 ? (t.master ? 2 : 1) : 0) +
         3 * (t.grad_dtype == PR_DTYPE_BF16 ? 1 : 0) + 6 * (t.state_bits == 8 ? 1 : 0);
}
constexpr int KINDS = 12;

struct Kernel {
  void* f;
  size_t smem;
};

template <int N, int KIND>
Kernel step_kernel() {
  using B = __nv_bfloat16;
  constexpr int BITS = KIND >= 6 ? 8 : 32;
  constexpr bool GB = (KIND / 3) % 2 == 1, MASTER = KIND % 3 == 2;
  using G = typename std::conditional<GB, B, float>::type;
  using P = typename std::conditional<KIND % 3 != 0, B, float>::type;
  return {reinterpret_cast<void*>(&prk::adamw_step<P, G, MASTER, BITS, N>),
          BITS == 8 ? prk::Staged<P, G, MASTER>::BYTES : 0};
}

template <int N>
Kernel kernel_of(int kind, bool unpack) {
  if (unpack) return {reinterpret_cast<void*>(&prk::adamw_unpack<N>), 0};
  const Kernel k[KINDS] = {step_kernel<N, 0>(), step_kernel<N, 1>(),  step_kernel<N, 2>(),
                          step_kernel<N, 3>(), step_kernel<N, 4>(),  step_kernel<N, 5>(),
                          step_kernel<N, 6>(), step_kernel<N, 7>(),  step_kernel<N, 8>(),
                          step_kernel<N, 9>(), step_kernel<N, 10>(), step_kernel<N, 11>()};
  return k[kind];
}

template <int N>
pr_status launch(pr_ctx* c, prk::AdamwArgs<N>& a, const Kernel& kern, cudaStream_t s) {
  cudaLaunchConfig_t cfg;
  memset(&cfg, 0, sizeof cfg);
  cfg.gridDim = dim3((unsigned)a.chunk0[a.count]);
  cfg.blockDim = dim3(prk::AW_NT);
  cfg.dynamicSmemBytes = kern.smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  void* args[] = {&a};
  PR_CUDA(cudaLaunchKernelExC(&cfg, kern.f, args));
  g_launches.fetch_add(1, std::memory_order_relaxed);
  a.count = 0;
  return timing_mark(c, s);
}

struct Step {
  float lr = 0.f, eps = 0.f, b1 = 0.f, c1 = 0.f, b2 = 0.f, c2 = 0.f, ibc1 = 0.f, ibc2 = 0.f, root_ibc2 = 0.f;
  const float* grad_scale = nullptr;
  float *m_out = nullptr, *v_out = nullptr;
};

// the launches over the tensors of one kind, N at a time
template <int N>
pr_status run_kind(pr_ctx* c, const pr_adamw_tensor* t, int32_t n_tensors, int kind,
                   const Step& step, bool unpack, int per_warp, cudaStream_t s) {
  prk::AdamwArgs<N> a;
  a.count = 0;
  a.per_warp = per_warp;
  a.lr = step.lr;
  a.eps = step.eps;
  a.b1 = step.b1;
  a.c1 = step.c1;
  a.b2 = step.b2;
  a.c2 = step.c2;
  a.ibc1 = step.ibc1;
  a.ibc2 = step.ibc2;
  a.root_ibc2 = step.root_ibc2;
  a.one = 1.f;
  a.grad_scale = step.grad_scale;
  a.m_out = step.m_out;
  a.v_out = step.v_out;
  a.ctx_flags = c->flags;
  a.chunk0[0] = 0;
  const Kernel kern = kernel_of<N>(kind, unpack);
  bool& ready = c->adamw_ready[N == prk::AW_MANY][kind];
  if (!unpack && !ready) {
    PR_CUDA(cudaFuncSetAttribute(kern.f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kern.smem));
    ready = true;
  }
  const int64_t chunk = (int64_t)prk::AW_NW * per_warp, most = (int64_t)1 << 30;
  int64_t block0 = 0;
  for (int32_t i = 0; i < n_tensors; ++i) {
    const int64_t blocks = (t[i].n + prk::AW_BLOCK - 1) / prk::AW_BLOCK;
    const int64_t mine = block0;
    block0 += blocks;
    if (blocks == 0 || (!unpack && kind_of(t[i]) != kind)) continue;
    const int64_t chunks = (blocks + chunk - 1) / chunk;
    if (chunks > most) return PR_ERR_INVALID_ARG;
    if (a.count == N || (a.count > 0 && a.chunk0[a.count] + chunks > most)) {
      const pr_status st = launch(c, a, kern, s);
      if (st != PR_OK) return st;
    }
    prk::AdamwEntry& e = a.t[a.count];
    e.p = t[i].param;
    e.g = t[i].grad;
    e.master = t[i].master;
    e.m = t[i].m;
    e.v = t[i].v;
    e.ms = t[i].m_scale;
    e.vs = t[i].v_scale;
    e.n = t[i].n;
    e.wd = t[i].weight_decay;
    e.block0 = mine;
    // (the step copies codes 16 bytes at a time, the expansion loads 8)
    const size_t sb = t[i].state_bits == 32 ? 32 : unpack ? 8 : 16;
    e.wide = fits(t[i].m, sb) && fits(t[i].v, sb) && (unpack ||
             (fits(t[i].param, 8 * esize(t[i].param_dtype)) && fits(t[i].master, 32) &&
              fits(t[i].grad, 8 * esize(t[i].grad_dtype))));
    if (unpack) e.wide = e.wide && fits(step.m_out, 32) && fits(step.v_out, 32);
    a.chunk0[a.count + 1] = a.chunk0[a.count] + (int32_t)chunks;
    ++a.count;
  }
  return a.count > 0 ? launch(c, a, kern, s) : PR_OK;
}

// Blocks per warp: enough for the GPU's CTAs to be filled several times over; with
// 8-bit states 16, for a warp's pipeline of blocks to begin seldom (134 M fp32 parameters:
// 524 us with their expansion, 617 with four), else four (LM head with states in 32 bits:
// 2.21 ms, 2.22 with 16); one where the step is short and a warp's blocks would follow one
// another.
int blocks_per_warp(const pr_ctx* c, int64_t blocks, bool eight) {
  const int64_t wave = (int64_t)prk::AW_NW * 3 * c->num_sms;
  if (eight && blocks >= 2 * 16 * wave) return 16;
  return blocks >= 2 * 4 * wave ? 4 : 1;
}

pr_status run(pr_ctx* c, const pr_adamw_tensor* t, int32_t n_tensors, const Step& step,
              bool unpack, cudaStream_t s) {
  int32_t of[KINDS] = {};
  int64_t blocks[KINDS] = {};
  for (int32_t i = 0; i < n_tensors; ++i) {
    const int k = unpack ? 0 : kind_of(t[i]);
    if (t[i].n > 0) ++of[k];
    blocks[k] += (t[i].n + prk::AW_BLOCK - 1) / prk::AW_BLOCK;
  }
  for (int k = 0; k < KINDS; ++k) {
    if (of[k] == 0) continue;
    const int per_warp = blocks_per_warp(c, blocks[k], !unpack && k >= 6);
    const pr_status st =
        of[k] <= prk::AW_FEW
            ? run_kind<prk::AW_FEW>(c, t, n_tensors, k, step, unpack, per_warp, s)
            : run_kind<prk::AW_MANY>(c, t, n_tensors, k, step, unpack, per_warp, s);
    if (st != PR_OK) return st;
  }
  return PR_OK;
}

}  // namespace

extern "C" {

pr_status pr_adamw_step(pr_ctx* c, const pr_adamw_tensor* tensors, int32_t n_tensors, double lr,
                        double beta1, double beta2, double eps, int64_t step,
                        const float* grad_scale, void* stream) {
  if (!c || n_tensors < 0 || (n_tensors > 0 && !tensors)) return PR_ERR_INVALID_ARG;
  if (!std::isfinite(lr) || !(beta1 >= 0.0) || !(beta1 < 1.0) || !(beta2 >= 0.0) ||
      !(beta2 < 1.0) || !(eps >= 0.0) || !std::isfinite(eps) || step < 1)
    return PR_ERR_INVALID_ARG;
  for (int32_t i = 0; i < n_tensors; ++i) {
    const pr_status st = check(tensors[i]);
    if (st != PR_OK) return st;
  }
  pr_status st = set_device(c);
  if (st != PR_OK) return st;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if ((st = timing_begin(c, s)) != PR_OK) return st;
  Step a;
  a.lr = (float)lr;
  a.eps = (float)eps;
  a.b1 = (float)beta1;
  a.c1 = (float)(1.0 - beta1);
  a.b2 = (float)beta2;
  a.c2 = (float)(1.0 - beta2);
  a.ibc1 = (float)(1.0 / (1.0 - std::pow(beta1, (double)step)));
  a.ibc2 = (float)(1.0 / (1.0 - std::pow(beta2, (double)step)));
  a.root_ibc2 = (float)std::sqrt(1.0 / (1.0 - std::pow(beta2, (double)step)));
  a.grad_scale = grad_scale;
  return run(c, tensors, n_tensors, a, false, s);
}

pr_status pr_adamw_unpack(pr_ctx* c, const pr_adamw_tensor* tensors, int32_t n_tensors, float* m,
                          float* v, void* stream) {
  if (!c || n_tensors < 0 || (n_tensors > 0 && !tensors)) return PR_ERR_INVALID_ARG;
  if (!fits(m, 4) || !fits(v, 4)) return PR_ERR_INVALID_ARG;
  for (int32_t i = 0; i < n_tensors; ++i) {
    const pr_status st = check(tensors[i]);
    if (st != PR_OK) return st;
    if (tensors[i].state_bits != 8 || (tensors[i].n > 0 && (!m || !v))) return PR_ERR_INVALID_ARG;
  }
  pr_status st = set_device(c);
  if (st != PR_OK) return st;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if ((st = timing_begin(c, s)) != PR_OK) return st;
  Step a;
  a.m_out = m;
  a.v_out = v;
  return run(c, tensors, n_tensors, a, true, s);
}

}  // extern "C"
