// Host side of pr_distill_loss: argument checks, the context's workspace and the launches of
// the kernels in pr_distill.cuh.
#include "pr_loss_host.h"
#include "pr_distill.cuh"

using namespace prh;

static_assert(PR_MAX_LISTED == prk::DS_MAX && PR_NDIS == prk::DS_TERMS + 1, "lists, statistics");
static_assert(prk::DS_TERMS <= prk::LS_NSTAT, "the workspace's places for sums");

namespace {

size_t ring_bytes(int places, int cluster, int lag, bool own) {
  return prk::distill_start(cluster, places, lag) + (size_t)places * prk::RG_BYTES +
         (own ? sizeof(prk::OwnPlan) : 0);
}

template <typename T>
const void* ring_kernel(bool hold, bool own) {
  return hold ? (own ? reinterpret_cast<const void*>(&prk::distill_ring<T, true, true>)
                     : reinterpret_cast<const void*>(&prk::distill_ring<T, true, false>))
              : (own ? reinterpret_cast<const void*>(&prk::distill_ring<T, false, true>)
                     : reinterpret_cast<const void*>(&prk::distill_ring<T, false, false>));
}
const void* ring_kernel(pr_dtype dt, bool hold, bool own) {
  return dt == PR_DTYPE_BF16 ? ring_kernel<__nv_bfloat16>(hold, own)
                             : ring_kernel<float>(hold, own);
}

const void* rows_kernel(pr_dtype dt, bool hold) {
  if (dt == PR_DTYPE_BF16)
    return hold ? reinterpret_cast<const void*>(&prk::distill_rows<__nv_bfloat16, true>)
                : reinterpret_cast<const void*>(&prk::distill_rows<__nv_bfloat16, false>);
  return hold ? reinterpret_cast<const void*>(&prk::distill_rows<float, true>)
              : reinterpret_cast<const void*>(&prk::distill_rows<float, false>);
}

// half of an SM's shared memory
constexpr size_t HALF = prk::distill_start(4, prk::RG_FEW, 0) + (size_t)prk::RG_FEW * prk::RG_BYTES;

// shared memory opt-ins, and the clusters that the GPU has room for, as ring_setup of the other
// losses
pr_status setup(pr_ctx* c) {
  if (c->distill_ready) return PR_OK;
  for (pr_dtype dt : {PR_DTYPE_F32, PR_DTYPE_BF16})
    for (bool hold : {false, true}) {
      for (bool own : {false, true})
        PR_CUDA(cudaFuncSetAttribute(ring_kernel(dt, hold, own),
                                     cudaFuncAttributeMaxDynamicSharedMemorySize,
                                     (int)ring_bytes(prk::RG_MOST, 8, 0, false)));
      PR_CUDA(cudaFuncSetAttribute(rows_kernel(dt, hold),
                                   cudaFuncAttributeMaxDynamicSharedMemorySize, (int)HALF));
    }
  for (int i = 0; i < 4; ++i)
    for (int whole = 0; whole < 2; ++whole) {
      if (i == 0) {
        c->distill_places[whole][0] = c->num_sms * (whole ? 1 : 2);
        continue;
      }
      cudaLaunchConfig_t cfg;
      memset(&cfg, 0, sizeof cfg);
      cfg.gridDim = dim3(1u << i);
      cfg.blockDim = dim3(prk::RG_NT);
      cfg.dynamicSmemBytes = ring_bytes(whole ? prk::RG_MOST : prk::RG_FEW, 1 << i, 0, false);
      cudaLaunchAttribute attr[1];
      attr[0].id = cudaLaunchAttributeClusterDimension;
      attr[0].val.clusterDim.x = 1u << i;
      attr[0].val.clusterDim.y = 1;
      attr[0].val.clusterDim.z = 1;
      cfg.attrs = attr;
      cfg.numAttrs = 1;
      int n = 0;
      PR_CUDA(cudaOccupancyMaxActiveClusters(&n, ring_kernel(PR_DTYPE_BF16, true, false), &cfg));
      c->distill_places[whole][i] = std::max(n, 1);
    }
  c->distill_ready = true;
  return PR_OK;
}

pr_status launch_lists(pr_ctx* c, prk::DistillArgs& d, pr_dtype dt, cudaStream_t s) {
  void* args[] = {&d};
  const pr_status st = launch(dt == PR_DTYPE_BF16
                                  ? reinterpret_cast<const void*>(&prk::distill_lists<__nv_bfloat16>)
                                  : reinterpret_cast<const void*>(&prk::distill_lists<float>),
                              (unsigned)((d.a.n_rows + prk::DP_NT / 32 - 1) / (prk::DP_NT / 32)),
                              prk::DP_NT, 0, 1, args, s);
  return st == PR_OK ? timing_mark(c, s) : st;
}

pr_status launch_ring(pr_ctx* c, prk::DistillArgs& d, pr_dtype dt, const RingShape& shape,
                      bool hold, cudaStream_t s) {
  int places = shape.places, parts = 1, cluster = 1 << shape.split;
  int64_t groups = shape.groups;
  bool full = shape.full;
  // rows one to a CTA, all their parts, once there are some for each: see distill_ring
  if (!hold && cluster > 1 && d.a.n_rows >= 4 * c->num_sms) {
    parts = cluster;
    cluster = 1;
    places = prk::RG_FEW - 1;
    groups = std::min<int64_t>(d.a.n_rows, 2 * c->num_sms);
    full = true;
  }
  if (d.a.own) --places;  // (the rows' list takes one)
  int lag = hold && shape.split == 0 && 2 * shape.here + 1 <= places ? 1 : 0;
  void* args[] = {&d, &places, &lag, &parts};
  // (a grid that takes every place is not set up early: see launch_ring of the other losses)
  const pr_status st = launch(ring_kernel(dt, hold, d.a.own), (unsigned)(groups * cluster),
                              prk::RG_NT, ring_bytes(places, cluster * parts, lag, d.a.own),
                              (unsigned)cluster, args, s, !full);
  return st == PR_OK ? timing_mark(c, s) : st;
}

// Warps of a CTA of distill_rows, or 0 where the ring takes no more time: the other losses' rule.
// us with a gradient, rows for the ring, k = 32 bf16:
//   V 2,000   700 rows 17 for 24   8,000 37 for 108     V 8,192    700 21 for 25   8,000 84 for 120
//   V 11,000  700 rows 23 for 26   8,000 106 for 137    V 17,000   700 27 for 28   8,000 174 for 170
// (The border could lie higher without a gradient: V 14,000, 8,000 rows 79 for 99.)
int rows_warps(const pr_ctx* c, const prk::LossArgs& a, pr_dtype dt) {
  if (a.own || a.n_rows <= 4 * c->num_sms) return 0;
  const int64_t part = std::max<int64_t>(16, a.vocab * (int64_t)esize(dt) / 16 * 16);
  const int64_t w = std::min<int64_t>(prk::RW_MOST, ((int64_t)HALF - (int64_t)prk::DR_CTL) / part);
  return w >= 5 ? (int)w : 0;
}

pr_status launch_rows(pr_ctx* c, prk::DistillArgs& d, pr_dtype dt, int warps, bool hold,
                      cudaStream_t s) {
  int part = (int)std::max<int64_t>(16, d.a.vocab * (int64_t)esize(dt) / 16 * 16);
  void* args[] = {&d, &part};
  const pr_status st = launch(rows_kernel(dt, hold),
                              (unsigned)std::min<int64_t>(2 * c->num_sms, d.a.n_rows), 32u * warps,
                              prk::DR_CTL + (size_t)warps * part, 1, args, s);
  return st == PR_OK ? timing_mark(c, s) : st;
}

}  // namespace

extern "C" {

pr_status pr_distill_loss(pr_ctx* c, const void* logits, pr_dtype dt, int64_t n_rows,
                          int64_t vocab, int64_t row_stride, const int32_t* ids,
                          const float* t_logp, int32_t k, const int32_t* chosen,
                          const uint8_t* mask, const int64_t* offsets, int32_t n_req,
                          const pr_distill* p, float* stats, float* kl, void* grad,
                          int64_t grad_stride, void* stream) {
  if (!c || !p) return PR_ERR_INVALID_ARG;
  pr_status st = check_loss(dt, logits, n_rows, vocab, row_stride, offsets, n_req,
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
  if ((st = setup(c)) != PR_OK) return st;
  // (up to PR_DISTILL_MAX_VOCAB a cluster holds the row)
  const RingShape ring = choose_ring(c->distill_places, dt, n_rows, vocab);
  if ((st = workspace(c, d.a, std::max(ring.groups, forward_grid(c)), false, false)) != PR_OK)
    return st;
  d.a.own = own_list(d.a);
  const bool prepared = grad && !d.a.own && rows_warps(c, d.a, dt) == 0;
  if (prepared) {
    const size_t scalars = (size_t)n_rows * 32;
    if ((st = grow(c->distill_ws, scalars + (size_t)n_rows * k * 16, false)) != PR_OK) return st;
    d.scalars = static_cast<float4*>(c->distill_ws.p);
    d.entries = reinterpret_cast<int4*>(static_cast<char*>(c->distill_ws.p) + scalars);
  }
  if ((st = timing_begin(c, s)) != PR_OK) return st;
  if ((st = launch_plan(c, d.a, 0, s)) != PR_OK) return st;
  if (const int warps = rows_warps(c, d.a, dt))
    return launch_rows(c, d, dt, warps, grad != nullptr, s);
  if (prepared && (st = launch_lists(c, d, dt, s)) != PR_OK) return st;
  return launch_ring(c, d, dt, ring, grad != nullptr, s);
}

}  // extern "C"
