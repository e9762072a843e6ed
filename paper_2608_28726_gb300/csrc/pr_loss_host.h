// Host side that the calls over logit rows with a mask and offsets share: their argument
// checks, the context's workspace, launches and the listing of the rows that count.
#pragma once

#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "pr_ctx.h"
#include "pr_loss.cuh"

namespace prh {

inline size_t esize(pr_dtype dt) { return dt == PR_DTYPE_BF16 ? 2 : 4; }

inline size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

inline pr_status check_loss(pr_dtype dt, const void* logits, int64_t n_rows, int64_t vocab,
                            int64_t row_stride, const int64_t* offsets, int32_t n_req,
                            float temperature, float grad_scale, const float* stats,
                            const float* logp, const void* grad, int64_t grad_stride) {
  if (dt != PR_DTYPE_F32 && dt != PR_DTYPE_BF16) return PR_ERR_INVALID_ARG;
  if (n_rows < 0 || n_rows > 0x7fffffffLL || vocab <= 0 || vocab > 0x7fffffffLL ||
      row_stride < vocab || n_req < 0)
    return PR_ERR_INVALID_ARG;
  if (!stats || (n_rows > 0 && (!logits || !logp))) return PR_ERR_INVALID_ARG;
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

inline int64_t forward_grid(const pr_ctx* c) { return (int64_t)c->num_sms * prk::FW_CTAS; }

// The workspace: what is zero between calls, [tickets, totals][arrivals per row], and the
// rest, [per CTA][per request][per pair][per row][per group].  Neither is freed before the
// context is: a captured graph may hold them.
inline pr_status workspace(pr_ctx* c, prk::LossArgs& a, int64_t groups, bool pref, bool state) {
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
inline pr_status launch(const void* kern, unsigned grid, unsigned threads, size_t smem,
                        unsigned cluster, void** args, cudaStream_t s, bool early = true) {
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

inline bool own_list(const prk::LossArgs& a) {
  return a.n_rows > 0 && a.n_rows <= prk::OWN_MOST && a.n_req <= prk::OWN_MOST;
}

// One CTA where it takes no longer than the second launch (about 3 us) that many need.
inline pr_status launch_plan(pr_ctx* c, prk::LossArgs& a, int pairs, cudaStream_t s) {
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

// The one-pass kernel's launch: 2^split CTAs per row, `places` chunks in a CTA's ring.
struct RingShape {
  int split, places;
  int here;         // chunks of a row's part
  bool hold;        // a row's chunks fit the cluster's rings
  bool spare;       // and leave a place free
  bool full;        // every place is taken
  int64_t groups;   // rows in work at a time
};

// Of the launches whose CTAs hold a row, with two places left for the next row's chunks, the one
// that takes the least time by this count (room: clusters resident, as ring_setup finds), in the
// time that an SM takes for a chunk: each cluster's rows come one after the other, a row takes its
// CTA's chunks and about three for its end, which two CTAs on an SM hide from one another.  The
// same with and without a gradient, so that the losses' bits are.
inline RingShape choose_ring(const int (&room)[2][4], pr_dtype dt, int64_t n_rows, int64_t vocab) {
  const int64_t words = vocab * (int64_t)esize(dt) / 16;
  const int64_t chunks = (words + prk::RG_CHUNK - 1) / prk::RG_CHUNK;
  RingShape s;
  s.split = 3;
  s.places = prk::RG_MOST;
  int64_t best = -1;
  for (int whole = 0; whole < 2; ++whole)
    for (int split = 0; split < (whole ? 4 : 3); ++split) {
      const int64_t here = (chunks + (1 << split) - 1) >> split, at_once = room[whole][split];
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
  const int64_t at_once = room[s.places == prk::RG_MOST][s.split];
  s.here = (int)std::min<int64_t>((chunks + (1 << s.split) - 1) >> s.split, prk::RG_MOST + 1);
  s.hold = s.here <= s.places;
  s.spare = s.here < s.places;
  s.groups = std::min<int64_t>(n_rows, at_once);
  s.full = n_rows >= at_once;
  return s;
}

inline void fill(prk::LossArgs& a, pr_ctx* c, const void* logits, int64_t n_rows, int64_t vocab,
                 int64_t row_stride, const int32_t* chosen, const uint8_t* mask,
                 const int64_t* offsets, int32_t n_req, const float* ref_logp, float temperature,
                 float grad_scale, float* stats, float* logp, void* grad, int64_t grad_stride) {
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

}  // namespace prh
