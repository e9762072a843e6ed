// Training losses over logit rows: the clipped policy loss with a KL term and the
// loss of paired log ratios, with the gradient of the logits.
//
// Row t with logits x, emitted token y and temperature T has z = x / T,
// l = z_y - log sum_v exp(z_v), and for any loss L that depends on the row through
// l alone dL/dx_v = (dL/dl) (onehot_y(v) - p_v) / T, p = softmax(z).  So a row needs
// two sweeps over its logits, with the scalar dL/dl between them.  With c = log2(e) / T:
//   forward   R = sum over v != y of 2^(c x_v - k), k a reference that each thread takes
//             from its first logits and raises only where the sum would overflow
//   backward  g_v = dL/dl / T (onehot - 2^(c x_v - K)), K = k + log2(R + e_y)
// one FMA and one ex2 per logit and sweep.  The emitted token's own term e_y stays out
// of the forward sum: 1 - p_y = R / (R + e_y) and l = -log(1 + R / e_y) keep their
// relative accuracy where p_y is close to 1 and 1 - p_y or log(R + e_y) would cancel.
// Rows whose sum is 0 or not finite that way (NaN, infinities, logits beyond 1e38) are
// summed again with c (x_v - M) in place of c x_v - k, M the row's maximum: exact for
// equal logits of any magnitude, and what is NaN then is NaN by the formula.
// The policy loss' dL/dl needs the row alone; the preference loss' needs the log
// ratios of the row's whole answer pair.
#pragma once

#include "pr_kernels.cuh"

namespace prk {

constexpr int LS_NSTAT = 6;   // statistics of a loss (the preference loss has 5)
constexpr float LS_MIN = -3.402823466e38f;  // "no maximum yet": the lowest finite value

struct LossArgs {
  const void* logits;
  int64_t n_rows, vocab, row_stride;  // strides in elements
  const int32_t* chosen;
  const uint8_t* mask;
  const int64_t* offsets;  // NULL: one request of all rows
  int32_t n_req;
  const float* old_logp;
  const float* ref_logp;
  const float* adv;
  int32_t per_request, norm;
  float clip_lo, clip_hi, kl_coef;
  float beta, smooth, margin;
  int32_t loss, length_norm;
  float inv_t, c2;  // 1 / T, log2(e) / T
  float grad_scale;
  float* stats;
  float* ratio;
  float* logp;
  void* grad;
  int64_t grad_stride;
  // workspace
  int32_t* ticket;     // [3] zero between calls: arrivals (the plan's, the statistics'); offsets decrease
  int64_t* totals;     // counted tokens; requests with some (policy) or pairs of such
  int32_t* count;      // [n_req] counted tokens
  int32_t* row_req;    // [n_rows] request of a row that counts, else -1
  int32_t* block;      // [blocks of PL_BLOCK rows] counted rows, then those before the block
  int4* list;          // [n_rows] {row, request, token} of the rows that count
  int32_t* skipped;    // [n_rows] the others
  int32_t* arrived;    // [n_rows] pieces of a row that are summed; zero between calls
  float2* piece;       // [CTAs][2] their sums
  float* coef;         // [n_req] dL / d log ratio (preference)
  float* term;         // [n_req / 2][LS_NSTAT] the pairs' statistics
  float4* state;       // [n_rows] K, adj, rest, M: RowState
  float* z;            // [n_rows] l - ref (preference) or dL/dl / T
  double* part;        // [groups][LS_NSTAT] statistics of each group's rows
  uint32_t* ctx_flags;
  int32_t own;  // every CTA lists the rows by itself (loss_forward)
};

// ---- which rows count -----------------------------------------------------------------
//
// The rows that count are listed in order, so that every CTA gets its even share of
// them whatever the mask.  (Dealt out as they lie, a tenth of 8,847 rows masked at random
// leaves 15 for some CTAs where the mean is 13.1.)
constexpr int PL_BLOCK = 1024;  // rows of a block
constexpr int PL_FEW = 1024;    // requests that one CTA counts in shared memory

// The request that counts row t, else -1.  Where offsets decrease, the request that this
// search finds is the row's, on every way of listing.
__device__ __forceinline__ int32_t counted_by(const LossArgs& a, int64_t t) {
  if (a.mask && a.mask[t] == 0) return -1;
  if (!a.offsets) return 0;
  int32_t r = 0, hi = a.n_req - 1;  // the largest r with offsets[r] <= t
  while (r < hi) {
    const int32_t mid = (int32_t)(((int64_t)r + hi + 1) >> 1);
    if (a.offsets[mid] <= t) r = mid;
    else hi = mid - 1;
  }
  const int64_t lo = a.offsets[r], up = a.offsets[r + 1];
  return lo < 0 || up > a.n_rows || t < lo || t >= up ? -1 : r;
}
// whether request r's bounds are wrong; its flags
__device__ __forceinline__ bool bad_bounds(const LossArgs& a, int64_t r, int64_t& lo, int64_t& hi) {
  lo = a.offsets ? a.offsets[r] : 0;
  hi = a.offsets ? a.offsets[r + 1] : a.n_rows;
  const bool bad = lo < 0 || hi < lo || hi > a.n_rows;
  if (bad) atomicOr(a.ctx_flags, FLAG_BAD_OFFSETS);
  else if (lo == hi) atomicOr(a.ctx_flags, FLAG_EMPTY_REQ);
  return bad;
}
// row t, counted by r, among the others: `before` counted ones precede it
__device__ __forceinline__ void put_row(const LossArgs& a, int64_t t, int32_t r, int32_t before) {
  a.row_req[t] = r;
  if (r >= 0) {
    a.list[before] = make_int4((int32_t)t, r, a.chosen[t], 0);
  } else {
    a.skipped[t - before] = (int32_t)t;
    a.logp[t] = 0.f;
  }
}
// exclusive sum over a CTA of 1,024 threads of a flag; the total in `all`
__device__ __forceinline__ int32_t block_rank(bool on, int32_t* warps, int32_t& all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const unsigned b = __ballot_sync(FULL, on);
  __syncthreads();
  if (lane == 0) warps[warp] = __popc(b);
  __syncthreads();
  const int32_t c = warps[lane];
  const int32_t below = __reduce_add_sync(FULL, lane < warp ? c : 0);
  all = __reduce_add_sync(FULL, c);
  return below + __popc(b & ((1u << lane) - 1u));
}
__device__ __forceinline__ int64_t block_total(int64_t v, int64_t* part) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
  __syncthreads();
  if (lane == 0) part[warp] = v;
  __syncthreads();
  v = part[lane];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
  return v;
}

// Small batches: everything by one CTA.
static __global__ void __launch_bounds__(PL_BLOCK) loss_plan(const LossArgs a, int pairs) {
  __shared__ int32_t count[PL_FEW], warps[32];
  __shared__ int64_t part[32];
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x;
  if (tid < a.n_req) count[tid] = 0;
  int32_t before = 0;
  for (int64_t t0 = 0; t0 < a.n_rows; t0 += PL_BLOCK) {
    const int64_t t = t0 + tid;
    const int32_t r = t < a.n_rows ? counted_by(a, t) : -1;
    int32_t all;
    const int32_t rank = block_rank(r >= 0, warps, all);
    if (t < a.n_rows) put_row(a, t, r, before + rank);
    if (r >= 0) atomicAdd(&count[r], 1);  // (whole numbers: in any order)
    before += all;
  }
  __syncthreads();
  int64_t used = 0;
  if (tid < a.n_req) {
    int64_t lo, hi;
    bad_bounds(a, tid, lo, hi);
    a.count[tid] = count[tid];
    if (!pairs) used = count[tid] > 0;
    else if ((tid & 1) == 0) used = count[tid] > 0 && count[tid + 1] > 0;
  }
  used = block_total(used, part);
  if (tid == 0) {
    a.totals[0] = before;
    a.totals[1] = used;
  }
}

// Large ones: the first n_req CTAs count a request's rows each, the others those of a
// block of rows; the last to finish sums up.  Then loss_list.
static __global__ void __launch_bounds__(PL_BLOCK) loss_count(const LossArgs a, int pairs) {
  __shared__ int32_t warps[32];
  __shared__ int64_t part[32];
  __shared__ int last;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x;
  const int32_t blocks = (int32_t)((a.n_rows + PL_BLOCK - 1) / PL_BLOCK);
  if ((int64_t)blockIdx.x >= a.n_req) {
    const int64_t b = (int64_t)blockIdx.x - a.n_req, t = b * PL_BLOCK + tid;
    const int32_t r = t < a.n_rows ? counted_by(a, t) : -1;
    if (t < a.n_rows) a.row_req[t] = r;
    int32_t all;
    block_rank(r >= 0, warps, all);
    if (tid == 0) a.block[b] = all;
  } else {
    int64_t lo = 0, hi = 0, n = 0;
    const int64_t r = blockIdx.x;
    __shared__ int bad;
    if (tid == 0) {
      bad = bad_bounds(a, r, lo, hi);
      if (hi < lo) a.ticket[2] = 1;  // (seen by the last CTA with this one's arrival)
    }
    __syncthreads();
    lo = a.offsets ? a.offsets[r] : 0;
    hi = a.offsets ? a.offsets[r + 1] : a.n_rows;
    if (!bad) {
      if (!a.mask) n = tid == 0 ? hi - lo : 0;
      else
        for (int64_t t = lo + tid; t < hi; t += PL_BLOCK) n += a.mask[t] != 0;
    }
    n = block_total(n, part);
    if (tid == 0) a.count[r] = (int32_t)n;
  }
  __syncthreads();
  if (tid == 0) {
    __threadfence();
    last = atom_add_acq_rel(a.ticket, 1) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  if (__ldcg(a.ticket + 2)) {
    // Offsets that decrease: requests' bounds overlap, and which rows are whose is for the
    // rows to say.
    for (int64_t q = tid; q < a.n_req; q += PL_BLOCK) a.count[q] = 0;
    __syncthreads();
    for (int64_t t = tid; t < a.n_rows; t += PL_BLOCK) {
      const int32_t r = __ldcg(a.row_req + t);
      if (r >= 0) atomicAdd(a.count + r, 1);
    }
    __syncthreads();
  }
  int64_t used = 0;
  for (int64_t q = tid; q < a.n_req; q += PL_BLOCK) {
    const int32_t k = __ldcg(a.count + q);
    if (!pairs) used += k > 0;
    else if ((q & 1) == 0) used += k > 0 && __ldcg(a.count + q + 1) > 0;
  }
  used = block_total(used, part);
  int32_t before = 0;  // (blocks: a thousand at a time)
  for (int32_t b0 = 0; b0 < blocks; b0 += PL_BLOCK) {
    const int32_t c = b0 + tid < blocks ? __ldcg(a.block + b0 + tid) : 0;
    int32_t x = c;
    const int lane = tid & 31, warp = tid >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int32_t y = __shfl_up_sync(FULL, x, o);
      if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 31) warps[warp] = x;
    __syncthreads();
    const int32_t w = warps[lane];
    x += __reduce_add_sync(FULL, lane < warp ? w : 0);
    if (b0 + tid < blocks) a.block[b0 + tid] = before + x - c;
    before += __reduce_add_sync(FULL, w);
  }
  if (tid == 0) {
    a.totals[0] = before;
    a.totals[1] = used;
    a.ticket[0] = a.ticket[2] = 0;
  }
}
static __global__ void __launch_bounds__(PL_BLOCK) loss_list(const LossArgs a) {
  __shared__ int32_t warps[32];
  pdl_wait();
  pdl_trigger();
  const int64_t t = (int64_t)blockIdx.x * PL_BLOCK + threadIdx.x;
  const int32_t r = t < a.n_rows ? __ldcg(a.row_req + t) : -1;
  int32_t all;
  const int32_t rank = block_rank(r >= 0, warps, all);
  if (t < a.n_rows) put_row(a, t, r, __ldcg(a.block + blockIdx.x) + rank);
}

// The smallest batches: by every CTA of the kernel that reads the logits, in its shared
// memory, without a launch before it; the first CTA leaves what later kernels need.  (24 rows
// of V = 32,000 fp32: 24 us a call for 27 with a launch; 285 rows of V = 151,936 bf16 28 for
// 30.)
constexpr int OWN_MOST = 512;  // rows, requests
struct OwnPlan {
  int4 list[OWN_MOST];
  int32_t skipped[OWN_MOST], count[OWN_MOST];
  uint32_t on[OWN_MOST / 32];  // which rows count
  int32_t live, used;
};
template <int NT>
__device__ __forceinline__ void own_plan(const LossArgs& a, OwnPlan& p, bool pairs) {
  constexpr int NW = NT / 32, W = (OWN_MOST / 32 + NW - 1) / NW;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool leaves = blockIdx.x == 0;
  for (int q = tid; q < a.n_req; q += NT) p.count[q] = 0;
  if (tid == 0) p.used = 0;
  int32_t r[W], y[W];
#pragma unroll
  for (int k = 0; k < W; ++k) {
    const int64_t t = 32 * (warp + k * NW) + lane;
    y[k] = t < a.n_rows ? __ldcg(a.chosen + t) : 0;
    r[k] = t < a.n_rows ? counted_by(a, t) : -1;
    const unsigned b = __ballot_sync(FULL, r[k] >= 0);
    if (lane == 0 && warp + k * NW < OWN_MOST / 32) p.on[warp + k * NW] = b;
  }
  __syncthreads();
  const int32_t c = lane < OWN_MOST / 32 ? __popc(p.on[lane]) : 0;
#pragma unroll
  for (int k = 0; k < W; ++k) {
    const int g = warp + k * NW;
    const int32_t t = 32 * g + lane;
    const int32_t below = __reduce_add_sync(FULL, lane < g ? c : 0);
    if (t < a.n_rows) {
      const int32_t before = below + __popc(p.on[g] & ((1u << lane) - 1u));
      if (r[k] >= 0) {
        p.list[before] = make_int4(t, r[k], y[k], 0);
        atomicAdd(&p.count[r[k]], 1);
      } else {
        p.skipped[t - before] = t;
        if (leaves) a.logp[t] = 0.f;
      }
      if (leaves) a.row_req[t] = r[k];
    }
  }
  __syncthreads();
  for (int q = tid; q < a.n_req; q += NT) {
    if (pairs ? (q & 1) == 0 && p.count[q] > 0 && p.count[q + 1] > 0 : p.count[q] > 0)
      atomicAdd(&p.used, 1);
    if (leaves) {
      int64_t lo, hi;
      bad_bounds(a, q, lo, hi);
      a.count[q] = p.count[q];
    }
  }
  const int32_t live = __reduce_add_sync(FULL, c);
  if (tid == 0) p.live = live;
  __syncthreads();
  if (leaves && tid == 0) {
    a.totals[0] = live;
    a.totals[1] = p.used;
  }
}
// the counted rows of a batch and their i-th, and the rest, wherever they are listed
struct Rows {
  const OwnPlan* own;
  int32_t live;
  __device__ __forceinline__ int4 at(const LossArgs& a, int64_t i) const {
    if (i >= live) return make_int4(0, -1, 0, 0);
    return own ? own->list[i] : __ldcg(a.list + i);
  }
  __device__ __forceinline__ int32_t skipped(const LossArgs& a, int64_t i) const {
    return own ? own->skipped[i] : __ldcg(a.skipped + i);
  }
  __device__ __forceinline__ int32_t count(const LossArgs& a, int32_t r) const {
    return own ? own->count[r] : __ldcg(a.count + r);
  }
  // 1 / what the losses are divided by: rows, or requests with some
  __device__ __forceinline__ double share(const LossArgs& a) const {
    return 1.0 / (double)(a.norm ? (own ? own->used : __ldcg(a.totals + 1)) : live);
  }
};
template <int NT>
__device__ __forceinline__ Rows rows_of(const LossArgs& a, bool own, OwnPlan* p, bool pairs) {
  if (!own) return Rows{nullptr, (int32_t)__ldcg(a.totals)};
  own_plan<NT>(a, *p, pairs);
  return Rows{p, p->live};
}

// ---- the losses of one row / pair -------------------------------------------------------

struct PolicyTerms {
  float d, q, e;  // l - old, ref - l, e^q - 1
  float surrogate, ratio, clipped;
  float slope;    // dloss / dl
};

__device__ __forceinline__ PolicyTerms policy_terms(const LossArgs& a, float l, float l_lo,
                                                    float old, float ref, float adv) {
  PolicyTerms p;
  p.d = a.old_logp ? (l - old) + l_lo : l - l;  // (NaN for a row without l)
  p.ratio = expf(p.d);
  // (a ratio beyond single precision under an advantage of 0: its surrogate is 0)
  const float free = p.ratio == INFINITY && adv == 0.f ? 0.f : p.ratio * adv;
  const float bound = fminf(fmaxf(p.ratio, a.clip_lo), a.clip_hi) * adv;
  p.clipped = bound < free ? 1.f : 0.f;
  p.surrogate = bound < free ? bound : free;
  p.slope = bound < free ? 0.f : -free;
  p.q = p.e = 0.f;
  if (a.ref_logp) {
    p.q = (ref - l) - l_lo;
    p.e = expm1f(p.q);
    if (a.kl_coef != 0.f) p.slope = fmaf(-a.kl_coef, p.e, p.slope);
  }
  return p;
}

// ---- a row's words ------------------------------------------------------------------------

// 2^d for the factors between references: expf, whose mean error is a tenth of ex2's
// (-5e-8): a row's sum would take that on at each step of its merges
__device__ __forceinline__ float rescale2(float d) { return expf(d * LN2); }

// the word without its element j
template <typename T>
__device__ __forceinline__ uint4 without(uint4 w, int j) {
  uint32_t* u = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if (sizeof(T) == 4) {
      if (q == j) u[q] = 0xff800000u;
    } else {
      if (2 * q == j) u[q] = (u[q] & 0xffff0000u) | 0xff80u;
      if (2 * q + 1 == j) u[q] = (u[q] & 0xffffu) | 0xff800000u;
    }
  }
  return w;
}

// S += sum of 2^(c x - k) over the word
template <typename T>
__device__ __forceinline__ void add_word(float2& S, const uint4& w, float c2, float nk) {
  using Tr = Traits<T>;
#pragma unroll
  for (int j = 0; j < Tr::VEC; j += 2) {
    const float2 d = __ffma2_rn(make_float2(Tr::at(w, j), Tr::at(w, j + 1)),
                                make_float2(c2, c2), make_float2(nk, nk));
    S = __fadd2_rn(S, make_float2(ex2(d.x), ex2(d.y)));
  }
}

// A row's l = l_hi + l_lo, 1 - p_y and log2 S = e + f, from R and u + u_lo, the emitted
// token's exponent against the same reference; shift: what the reference was raised by.
// A log ratio sums hundreds of differences l - ref, whose errors must neither be
// l's rounding (2^-24 |l|) nor lean to one side.  So sums and products keep their
// roundings, the scale is the one that the row's sum was taken with (an error of c common
// to both has no mean over sampled tokens), and factors between references come from
// rescale2.  Mean error of l over sampled rows: below 2e-8 (1e-7 without all this).
constexpr float LN2_LOW = -1.90465421e-9f;  // ln 2 - LN2
struct RowEnd {
  float l, l_lo, rest, shift, e, f;
  __device__ __forceinline__ RowEnd(float R, float u, float u_lo) {
    shift = fmaxf(u, 0.f);
    if (u > 0.f) R *= rescale2(-u);
    const float ey = u > 0.f ? 1.f : ex2(u);
    const float S = R + ey;
    int ei = (int)(__float_as_uint(S) >> 23) - 127;
    float m = __uint_as_float((__float_as_uint(S) & 0x7fffffu) | 0x3f800000u);
    if (m > 1.41f) {
      m *= 0.5f;
      ++ei;
    }
    e = (float)ei;
    f = log2f(m);
    rest = R / S;
    if (ey > 0.25f * S) {
      l = -log1pf(R / ey);
      l_lo = 0.f;
    } else {
      const float v = u - shift, w = v - e, t = w - v;  // w's rounding: (v - (w - t)) + (-e - t)
      const float w_lo = ((v - (w - t)) + (-e - t)) + u_lo - f;
      const float hi = w * LN2;
      const float lo = fmaf(w, LN2, -hi) + w * LN2_LOW + w_lo * LN2;
      l = hi + lo;
      l_lo = (hi - l) + lo;
      if (u == -INFINITY) {  // a masked token
        l = u;
        l_lo = 0.f;
      }
    }
    if (!(S > 0.f) || !(S < INFINITY)) l = l_lo = NAN;
  }
};

// What a row's backward sweep needs: entries nk 2^(c x - K) (FAST), nk 2^(c (x - M) - K)
// (ROBUST) or 0; gy at the emitted token.
enum RowMode { ROW_ZERO = 0, ROW_FAST = 1, ROW_ROBUST = 2 };
struct RowOut {
  float K, nk, gy, M;
  int mode;
};
struct RowState {   // the same before dL/dl is known
  float K, adj, rest, M;  // adj: 2^-(what K lost to rounding)
};
__device__ __forceinline__ RowOut row_out(const RowState& s, float k) {
  RowOut o;
  o.K = s.K;
  o.nk = -k * s.adj;
  o.gy = k == 0.f ? 0.f : k * s.rest;  // (0, too, where rest is NaN)
  o.M = s.M;
  o.mode = k == 0.f ? ROW_ZERO : s.M == INFINITY ? ROW_FAST : ROW_ROBUST;
  return o;
}

template <bool ROBUST>
__device__ __forceinline__ float2 grad2(const RowOut& o, float c2, float x, float y) {
  float2 d = make_float2(x, y);
  if (ROBUST) d = __fadd2_rn(d, make_float2(-o.M, -o.M));
  d = __ffma2_rn(d, make_float2(c2, c2), make_float2(-o.K, -o.K));
  return __fmul2_rn(make_float2(ex2(d.x), ex2(d.y)), make_float2(o.nk, o.nk));
}
__device__ __forceinline__ float grad1(const RowOut& o, float c2, float x) {
  if (o.mode == ROW_ZERO) return 0.f;
  return o.mode == ROW_FAST ? grad2<false>(o, c2, x, x).x : grad2<true>(o, c2, x, x).x;
}
__device__ __forceinline__ uint32_t bf16_pair(float2 v) {
  const __nv_bfloat162 h = __float22bfloat162_rn(v);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <typename T, bool ROBUST>
__device__ __forceinline__ uint4 grad_word(const RowOut& o, float c2, const uint4& w) {
  using Tr = Traits<T>;
  if constexpr (sizeof(T) == 2) {
    return make_uint4(bf16_pair(grad2<ROBUST>(o, c2, Tr::at(w, 0), Tr::at(w, 1))),
                      bf16_pair(grad2<ROBUST>(o, c2, Tr::at(w, 2), Tr::at(w, 3))),
                      bf16_pair(grad2<ROBUST>(o, c2, Tr::at(w, 4), Tr::at(w, 5))),
                      bf16_pair(grad2<ROBUST>(o, c2, Tr::at(w, 6), Tr::at(w, 7))));
  } else {
    const float2 u = grad2<ROBUST>(o, c2, Tr::at(w, 0), Tr::at(w, 1));
    const float2 v = grad2<ROBUST>(o, c2, Tr::at(w, 2), Tr::at(w, 3));
    return make_uint4(__float_as_uint(u.x), __float_as_uint(u.y), __float_as_uint(v.x),
                      __float_as_uint(v.y));
  }
}
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
template <typename T>
__device__ __forceinline__ void put_word(T* p, const uint4& w, bool vec) {
  if (vec) {
    *reinterpret_cast<uint4*>(p) = w;
  } else {
#pragma unroll
    for (int j = 0; j < Traits<T>::VEC; ++j) put(p + j, Traits<T>::at(w, j));
  }
}

// A row as the 16-byte words of the address grid that lie in it, and the elements
// before and after them.
struct RowWords {
  int64_t head, words, tail;  // elements, words, elements
  template <typename T>
  __device__ __forceinline__ static RowWords of(const T* row, int64_t V) {
    RowWords w;
    const int64_t off = (int64_t)(reinterpret_cast<uintptr_t>(row) & 15u) / (int64_t)sizeof(T);
    w.head = off ? Traits<T>::VEC - off : 0;
    if (w.head > V) w.head = V;
    w.words = (V - w.head) / Traits<T>::VEC;
    w.tail = V - w.head - w.words * Traits<T>::VEC;
    return w;
  }
};

// ---- barriers in shared memory --------------------------------------------------------------

__device__ __forceinline__ bool ring_wait(uint32_t bar, uint32_t parity, uint32_t* flags) {
  // (the clock of ring_wait_slow is read only after some thousand tests)
  for (int i = 0; i < 4096; ++i)
    if (ring_test(bar, parity)) return true;
  return ring_wait_slow(bar, parity, flags);
}
__device__ __forceinline__ uint32_t sm_addr(const void* p) {
  return (uint32_t)__cvta_generic_to_shared(p);
}
__device__ __forceinline__ void bar_init(uint64_t* b, int n) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(sm_addr(b)), "r"(n) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t* b) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(sm_addr(b)) : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t* b, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(sm_addr(b)), "r"(bytes)
               : "memory");
}

// ---- a row among CTAs -------------------------------------------------------------------

// a CTA's part of a row
struct Share {
  const char* x;              // the row
  int32_t head, tail, words;  // elements before its 16-byte words and after them
  int32_t w0, w1;             // this CTA's words [w0, w1)
};
constexpr int SH_CHUNK = 1024;  // a CTA's part is a multiple of so many words
template <typename T>
__device__ __forceinline__ Share share_of(const LossArgs& a, int64_t row, uint32_t C,
                                          uint32_t rank) {
  constexpr uint32_t VEC = Traits<T>::VEC;
  Share s;
  const T* x = reinterpret_cast<const T*>(a.logits) + row * a.row_stride;
  s.x = reinterpret_cast<const char*>(x);
  const uint32_t off = ((uint32_t)reinterpret_cast<uintptr_t>(x) & 15u) / (uint32_t)sizeof(T);
  const uint32_t V = (uint32_t)a.vocab, head = min(off ? VEC - off : 0u, V);
  const uint32_t words = (V - head) / VEC;
  s.head = (int32_t)head;
  s.words = (int32_t)words;
  s.tail = (int32_t)(V - head - words * VEC);
  s.w0 = 0;
  s.w1 = s.words;
  if (C > 1) {
    const uint32_t all = (words + SH_CHUNK - 1) / SH_CHUNK, per = (all + C - 1) / C * SH_CHUNK;
    s.w0 = (int32_t)min(words, rank * per);
    s.w1 = (int32_t)min(words, (uint32_t)s.w0 + per);
  }
  return s;
}
// the emitted token's word, or -1
template <typename T>
__device__ __forceinline__ int32_t word_of(const LossArgs& a, const Share& s, int32_t y) {
  return y >= s.head && y < (int32_t)a.vocab - s.tail ? (y - s.head) / Traits<T>::VEC : -1;
}
// the element of this lane before or after the row's words, or -1
__device__ __forceinline__ int32_t end_of(const LossArgs& a, const Share& s, int lane) {
  return lane < 8 ? (lane < s.head ? lane : -1)
                  : (lane - 8 < s.tail ? (int32_t)a.vocab - s.tail + lane - 8 : -1);
}

// what a row's end needs, fetched while the rows before it are in work
struct RowIn {
  int32_t y, count;
  float xy, old, ref, adv, edge;
};

// The sum of a row (in a cluster: of this CTA's part of it) once more in M's terms, by one
// warp from global memory.  Rows with NaN or infinities, or of nothing but masked or
// lowest values.
template <typename T>
__device__ __noinline__ void robust_sum(const LossArgs& a, const Share s, bool ends, int32_t y,
                                        float& M, float& R, int lane) {
  using Tr = Traits<T>;
  const T* x = reinterpret_cast<const T*>(s.x);
  M = LS_MIN;
  float sum = 0.f;
  const int64_t lo = ends && s.w0 == 0 ? 0 : s.head + (int64_t)s.w0 * Tr::VEC;
  const int64_t hi = ends && s.w0 == 0 && s.w1 == s.words ? a.vocab
                                                         : s.head + (int64_t)s.w1 * Tr::VEC;
  auto add = [&](int64_t v) {
    const float e = Tr::elem(x, v);
    if (v == y) return;
    if (e != e) sum = e;
    if (e > M) {
      sum *= rescale2((M - e) * a.c2);
      M = e;
    }
    sum += ex2((e - M) * a.c2);
  };
  for (int64_t v = lo + lane; v < hi; v += 32) add(v);
  if (ends && hi < a.vocab && lane < s.tail) add(a.vocab - s.tail + lane);
  const float m = unord(__reduce_max_sync(FULL, ord(M)));
  R = sum * rescale2((M - m) * a.c2);
  M = m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) R += __shfl_xor_sync(FULL, R, o);
}

constexpr int RG_TERMS = 5;  // statistics that are summed row by row

// A row's end from its sums: R against 2^k, or against its maximum M where that is not
// infinite.  Writes logp, the statistics' terms (weight wt), and the result: to `out`,
// whose barrier (where there is one) learns of it first, else the row's state.  Whole warp; apart from the
// kernel's registers.
template <bool PREF>
__device__ __noinline__ void end_math(const LossArgs& a, int64_t row, const RowIn in, float k,
                                      float R, float M, float wt, bool writes, RowOut* out,
                                      uint64_t* out_bar, float2* stat, int lane) {
  float u, u_lo = 0.f;
  bool far = false;
  if (M == INFINITY) {
    const float h = in.xy * a.c2, hl = fmaf(in.xy, a.c2, -h);
    u = h - k;
    if (isfinite(h)) {  // h's and the difference's roundings: 2^-9 where logits are about 3e4
      const float t = u - h, left = ((h - (u - t)) + (-k - t)) + hl, all = u + left;
      u_lo = (u - all) + left;
      u = all;
    }
  } else {
    const float d = in.xy - M;
    u = d * a.c2;
    if (isfinite(u)) u_lo = fmaf(d, a.c2, -u);
    else far = d > -INFINITY;  // a finite logit that many below the maximum
    k = 0.f;
  }
  const RowEnd e(R, u, u_lo);
  const float l = far && e.l == -INFINITY ? (in.xy - M) * a.inv_t : e.l;
  // K = k + shift + e + f, and what its rounding left
  RowState st;
  const float b = k + e.shift, bt = b - k, b_lo = (k - (b - bt)) + (e.shift - bt);
  const float c = b + e.e, ct = c - b, c_lo = (b - (c - ct)) + (e.e - ct);
  st.K = c + e.f;
  st.adj = exp2f(-(((c - st.K) + e.f) + (b_lo + c_lo)));
  st.rest = e.rest;
  st.M = M;
  float kk = 0.f;
  PolicyTerms p;
  if (!PREF) {
    p = policy_terms(a, l, e.l_lo, in.old, in.ref, in.adv);
    kk = wt * p.slope * (a.grad_scale * a.inv_t);
  }
  if (out && lane == 0) {
    *out = row_out(st, kk);
    if (out_bar) bar_arrive(out_bar);
  }
  if (!PREF && lane < RG_TERMS) {
    const float x = wt * (lane == 0 ? p.surrogate : lane == 1 ? p.e - p.q : lane == 2 ? p.ratio
                                                : lane == 3 ? p.clipped : expm1f(p.d) - p.d);
    const float2 q = stat[lane];
    const float y = q.x + x, z = y - q.x;
    stat[lane] = make_float2(y, q.y + ((q.x - (y - z)) + (x - z)));
  }
  if (lane == 0 && writes) {
    a.logp[row] = l;
    if (in.y < 0 || (int64_t)in.y >= a.vocab) atomicOr(a.ctx_flags, FLAG_BAD_CHOSEN);
    else if (isnan(l)) atomicOr(a.ctx_flags, FLAG_NONFINITE);
    if (a.state) {
      a.state[row] = make_float4(st.K, st.adj, st.rest, st.M);
      a.z[row] = PREF ? (l - in.ref) + e.l_lo : kk;
    }
  }
}

// The scalars of a listed row {row, request, token}.  Whole warp.
template <typename T, bool PREF>
__device__ __forceinline__ RowIn fetch_row(const LossArgs& a, const Rows& rows, const Share& s,
                                           const int4& ref, int lane) {
  const int64_t row = ref.x;
  const int32_t r = ref.y, y = ref.z;
  RowIn in;
  in.y = y;
  in.count = 1;
  in.xy = NAN;
  in.old = in.ref = in.adv = in.edge = 0.f;
  if (r < 0) return in;
  const T* x = reinterpret_cast<const T*>(s.x);
  if (y >= 0 && (int64_t)y < a.vocab) in.xy = Traits<T>::elem(x, y);
  if (a.ref_logp) in.ref = __ldcg(a.ref_logp + row);
  if (!PREF) {
    if (a.old_logp) in.old = __ldcg(a.old_logp + row);
    in.adv = __ldcg(a.adv + (a.per_request ? (int64_t)r : row));
    if (a.norm) in.count = rows.count(a, r);
  }
  const int32_t v = end_of(a, s, lane);
  if (v >= 0) in.edge = Traits<T>::elem(x, v);
  return in;
}
// the elements at the row's ends into its sums
__device__ __forceinline__ void add_ends(const LossArgs& a, const Share& s, const RowIn& in,
                                         float& k, float& R, int lane) {
  if (s.head + s.tail == 0) return;
  const int32_t v = end_of(a, s, lane);
  const bool add = v >= 0 && v != in.y;
  const float top =
      unord(__reduce_max_sync(FULL, ord(add ? fmaxf(in.edge * a.c2, -3e38f) : -3e38f)));
  if (top > k) {
    R *= rescale2(k - top);
    k = top;
  }
  float e = add ? ex2(fmaf(in.edge, a.c2, -k)) : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) e += __shfl_xor_sync(FULL, e, o);
  R += e;
}
// (k, R) of the lanes together, against the largest k.  `unit`: what a k counts in 2's exponent
__device__ __forceinline__ void join(float2 q, float unit, float& k, float& R) {
  k = unord(__reduce_max_sync(FULL, ord(q.x)));
  R = q.y * rescale2((q.x - k) * unit);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) R += __shfl_xor_sync(FULL, R, o);
}
// whether a row has to be summed once more: sums that are 0 or not finite (0 is right where
// all others are masked and the emitted token is not)
__device__ __forceinline__ bool sum_again(float k, float R, float xy, float c2) {
  const float h = xy * c2;
  return !isfinite(R) || !isfinite(k) || !(h < INFINITY) || (h == -INFINITY && xy > -INFINITY) ||
         (R == 0.f && (k > -3e38f || h == -INFINITY));
}
// the robust sum's M raised to the emitted token's logit
__device__ __forceinline__ void raise_to(const LossArgs& a, float xy, float& M, float& R) {
  const float top = isnan(xy) ? M : fmaxf(M, xy);
  R *= rescale2((M - top) * a.c2);
  // (an infinite row is NaN by its factor; infinity here means an ordinary sum)
  if (top == INFINITY) R = NAN;
  M = fminf(top, -LS_MIN);
}

// A thread's words into its sum (k, S); the row's first ones give k.  They are summed by
// themselves first: one by one, the many terms below 2^-25 of S would all be lost (rows of
// V = 262,144 whose logits spread by 4: l 1e-7 too high on average, now 1e-8).
template <typename T, int N>
__device__ __forceinline__ void add_words(float& k, float2& S, const uint4 (&v)[N], float c2,
                                          bool begin) {
  using Tr = Traits<T>;
  auto top = [&]() {
    float m = Tr::gmax(v[0]);
#pragma unroll
    for (int q = 1; q < N; ++q) m = fmaxf(m, Tr::gmax(v[q]));
    return fmaxf(m * c2, -3e38f);
  };
  if (begin) k = top();
  float2 here = make_float2(0.f, 0.f);
#pragma unroll
  for (int q = 0; q < N; ++q) add_word<T>(here, v[q], c2, -k);
  const float2 sum = __fadd2_rn(S, here);
  if (__any_sync(FULL, !(sum.x + sum.y < 1e30f))) {
    const float up = fmaxf(top(), k), f = rescale2(k - up);
    k = up;
    here = make_float2(0.f, 0.f);
#pragma unroll
    for (int q = 0; q < N; ++q) add_word<T>(here, v[q], c2, -k);
    S = make_float2(fmaf(S.x, f, here.x), fmaf(S.y, f, here.y));
  } else {
    S = sum;
  }
}

// The statistics: a CTA's sums (of `warps` warps' rows) to a.part[at], the last of `count`
// CTAs joins all in order.  Whole warp.
__device__ __forceinline__ void write_stats(const LossArgs& a, const float2* stat, int warps,
                                            int64_t at, int64_t count, int lane) {
  int last = 0;
  if (lane < RG_TERMS) {
    double v = 0.;
    for (int w = 0; w < warps; ++w) {  // (an infinite sum's compensation is NaN)
      const float2 q = stat[w * RG_TERMS + lane];
      v += isinf(q.x) ? (double)q.x : (double)q.x + (double)q.y;
    }
    a.part[at * RG_TERMS + lane] = v;
  }
  __syncwarp();
  if (lane == 0) {
    __threadfence();
    last = atom_add_acq_rel(a.ticket + 1, 1) == (int)count - 1;
  }
  if (!__shfl_sync(FULL, last, 0)) return;
  double total[RG_TERMS];
#pragma unroll
  for (int j = 0; j < RG_TERMS; ++j) {
    double v = 0.;
    for (int64_t i = lane; i < count; i += 32) v += __ldcg(a.part + i * RG_TERMS + j);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
    total[j] = v;
  }
  if (lane == 0) {
    // (a KL term that is only watched, coefficient 0, may be infinite)
    const double kl = a.kl_coef != 0.f ? (double)a.kl_coef * total[1] : 0.;
    a.stats[0] = (float)(kl - total[0]);
    for (int j = 0; j < RG_TERMS; ++j) a.stats[1 + j] = (float)total[j];
    a.ticket[1] = 0;
  }
}

// ---- forward alone ----------------------------------------------------------------------
//
// The rows' tiles of 16 KB, one row after the other, are dealt out in equal runs: a CTA
// has the end of a row, some whole ones and the beginning of another, or, where there are few
// rows, a piece of one.  (A row each instead, dealt out as they lie: the preference loss of
// 64 answers at V = 151,936 bf16 takes 1.25 ms for 1.20, log-probabilities of 24
// responses at V = 70,001 bf16 93 us for 73.)  Eight warps sum, with wide loads
// into registers, four per thread in flight; a ninth joins their sums and takes the end
// of the rows that lie in this CTA whole.  The sums of the other rows' pieces go through
// global memory, and the warp that brings a row's last piece joins them in the row's
// order and takes its end.
constexpr int FW_NW = 8;
constexpr int FW_NT = 32 * (FW_NW + 1);
constexpr int FW_U = 4;
constexpr int FW_TILE = 32 * FW_NW * FW_U;  // words
constexpr int FW_CTAS = 4;                  // on an SM
struct ForwardSmem {
  float2 part[2][FW_NW];
  float2 stat[RG_TERMS];
};
// the run of CTA b: tiles [run_begin(b), run_begin(b + 1)); the CTA of tile t
__device__ __forceinline__ int64_t run_begin(int64_t b, int64_t tiles, int64_t G) {
  return b * tiles / G;
}
__device__ __forceinline__ int64_t run_of(int64_t t, int64_t tiles, int64_t G) {
  return ((t + 1) * G - 1) / tiles;
}

template <typename T, bool PREF>
__global__ void __launch_bounds__(FW_NT, FW_CTAS) loss_forward(const __grid_constant__ LossArgs a) {
  using Tr = Traits<T>;
  __shared__ ForwardSmem sm;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid < RG_TERMS) sm.stat[tid] = make_float2(0.f, 0.f);
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(16) unsigned char fw_raw[];
  const Rows rows = rows_of<FW_NT>(a, a.own, reinterpret_cast<OwnPlan*>(fw_raw), PREF);
  const int64_t live = rows.live;
  const int64_t most = (a.vocab + Tr::VEC - 1) / Tr::VEC;              // words of a row
  const int64_t per_row = (most + FW_TILE - 1) / FW_TILE, tiles = live * per_row;
  const int64_t G = min((int64_t)gridDim.x, max(tiles, (int64_t)1)), b = blockIdx.x;
  if (b >= G) return;
  const int64_t t0 = run_begin(b, tiles, G), t1 = run_begin(b + 1, tiles, G);
  auto ref_of = [&](int64_t i) { return rows.at(a, i); };
  int64_t i = t0 / per_row;
  int32_t j0 = (int32_t)(t0 - i * per_row);  // the first tile of row i here
  int64_t left = t1 - t0;
  uint32_t n = 0;  // pieces summed
  if (warp == FW_NW) {
    // ---- the rows' ends
    const double share = PREF ? 0.0 : rows.share(a);
    int4 ref = ref_of(i), ref1 = ref_of(i + 1);
    RowIn in = fetch_row<T, PREF>(a, rows, share_of<T>(a, ref.x, 1, 0), ref, lane);
    for (; left > 0; ++i, j0 = 0) {
      const RowIn next = fetch_row<T, PREF>(a, rows, share_of<T>(a, ref1.x, 1, 0), ref1, lane);
      const int64_t row = ref.x;
      ref = ref1;
      ref1 = ref_of(i + 2);
      const int64_t here = min(left, per_row - j0);
      left -= here;
      const int buf = n & 1;
      ++n;
      named_bar_sync(BAR_FULL + buf, FW_NT);
      float k, R, M = INFINITY;
      join(lane < FW_NW ? sm.part[buf][lane] : make_float2(-3e38f, 0.f), 1.f, k, R);
      __syncwarp();
      named_bar_arrive(BAR_EMPTY + buf, FW_NT);
      if (here < per_row) {
        const int64_t bs = run_of(i * per_row, tiles, G), be = run_of((i + 1) * per_row - 1, tiles, G);
        int last = 0;
        if (lane == 0) {
          a.piece[2 * b + (j0 == 0 ? 1 : 0)] = make_float2(k, R);
          last = atom_add_acq_rel(a.arrived + i, 1) == (int)(be - bs);
          if (last) a.arrived[i] = 0;
        }
        last = __shfl_sync(FULL, last, 0);
        if (!last) {
          in = next;
          continue;
        }
        k = -3e38f;
        R = 0.f;
        for (int64_t q = bs; q <= be; q += 32) {  // 32 pieces at a time
          const float2 p = q + lane <= be ? __ldcg(a.piece + 2 * (q + lane) + (q + lane == bs ? 1 : 0))
                                          : make_float2(-3e38f, 0.f);
          float k1, R1;
          join(p, 1.f, k1, R1);
          const float top = fmaxf(k, k1);
          R = R * rescale2(k - top) + R1 * rescale2(k1 - top);
          k = top;
        }
      }
      const Share sh = share_of<T>(a, row, 1, 0);
      add_ends(a, sh, in, k, R, lane);
      if (sum_again(k, R, in.xy, a.c2)) {
        robust_sum<T>(a, sh, true, in.y, M, R, lane);
        raise_to(a, in.xy, M, R);
      }
      const float wt = PREF ? 0.f : (float)(a.norm ? share / (double)in.count : share);
      end_math<PREF>(a, row, in, k, R, M, wt, true, nullptr, nullptr, sm.stat, lane);
      in = next;
    }
  } else {
    const uint4 NEG = make_uint4(Tr::NEG_WORD, Tr::NEG_WORD, Tr::NEG_WORD, Tr::NEG_WORD);
    int4 ref = ref_of(i);
    for (; left > 0; ++i, j0 = 0) {
      const int4 ref1 = ref_of(i + 1);
      const int32_t here = (int32_t)min(left, per_row - j0);
      left -= here;
      const Share sh = share_of<T>(a, ref.x, 1, 0);
      const int32_t yw = word_of<T>(a, sh, ref.z);
      const int yj = ref.z - sh.head - yw * Tr::VEC;
      const uint4* xw = reinterpret_cast<const uint4*>(sh.x + sizeof(T) * sh.head) + tid;
      float k = -3e38f;
      float2 S = make_float2(0.f, 0.f);
      uint4 v[FW_U];
      int32_t w = j0 * FW_TILE;
      const int32_t w0 = w, w1 = min(sh.words, w + here * FW_TILE);
      for (; w + FW_TILE <= w1; w += FW_TILE) {
#pragma unroll
        for (int q = 0; q < FW_U; ++q) v[q] = ld_stream(xw + w + q * 32 * FW_NW);
        if ((uint32_t)(yw - w) < (uint32_t)FW_TILE) {
#pragma unroll
          for (int q = 0; q < FW_U; ++q)
            if (w + q * 32 * FW_NW + tid == yw) v[q] = without<T>(v[q], yj);
        }
        add_words<T>(k, S, v, a.c2, w == w0);
      }
      if (w < w1) {
#pragma unroll
        for (int q = 0; q < FW_U; ++q) {
          const int32_t at = w + q * 32 * FW_NW + tid;
          v[q] = at < w1 ? ld_stream(xw + w + q * 32 * FW_NW) : NEG;
          if (at == yw) v[q] = without<T>(v[q], yj);
        }
        add_words<T>(k, S, v, a.c2, w == w0);
      }
      float R;
      join(make_float2(k, S.x + S.y), 1.f, k, R);
      const int buf = n & 1;
      if (n >= 2) named_bar_sync(BAR_EMPTY + buf, FW_NT);
      ++n;
      if (lane == 0) sm.part[buf][warp] = make_float2(k, R);
      __syncwarp();
      __threadfence_block();
      named_bar_arrive(BAR_FULL + buf, FW_NT);
      ref = ref1;
    }
    // the last pieces' places: the other warp has arrived for each
    for (uint32_t q = n >= 2 ? n - 2 : 0; q < n; ++q) named_bar_sync(BAR_EMPTY + (q & 1), FW_NT);
  }
  __syncthreads();
  if (!PREF && warp == 0) write_stats(a, sm.stat, 1, b, G, lane);
}

// ---- forward and backward in one pass -----------------------------------------------------
//
// A row belongs to a CTA, or its parts to the CTAs of a cluster.  Eight warps sum it and
// write its gradient, one brings it in, one takes its end.  Chunks of 16 KB come
// into a ring of shared memory by bulk copies; with HOLD a row's chunks stay there
// between the two sweeps, so that the logits are read from memory once, and the ring's
// other places take the next row's chunks meanwhile.  The row's end (the warps' sums
// joined, those of a cluster's CTAs through distributed shared memory, the elements
// before and after the row's 16-byte words, l and dL/dl) is a chain of 3,000 to 5,000 cycles:
// two CTAs share an SM where half its shared memory holds a part, and one streams
// while the other waits.
constexpr int RG_NW = 8;                       // warps that sum and write
constexpr int RG_NT = 32 * (RG_NW + 2);
constexpr int RG_W = 4;                        // words per lane and chunk
constexpr int RG_CHUNK = 32 * RG_NW * RG_W;    // words of a chunk
constexpr int RG_BYTES = 16 * RG_CHUNK;
constexpr int RG_MOST = 14, RG_FEW = 7;        // places of the ring: one or two CTAs on an SM
// A warp sends row n + 2's sum after it has waited for row n + 1's result.  That took row
// n + 1's sums of all CTAs, whose senders had waited for row n's result in their own CTA, and
// that one's sums have been read by then: two slots.
constexpr int RG_SLOTS = 2;
struct RingCtl {
  uint64_t full[RG_MOST], empty[RG_MOST];      // a chunk has landed; has been read
  uint64_t sum_bar[RG_SLOTS];                  // the warps' sums are there
  uint64_t out_bar[RG_SLOTS];                  // a row's result is there
  float2 again[MAXC];                          // the CTAs' sums of a row summed once more
  uint64_t again_bar;
  float2 stat[RG_TERMS];                       // sums over the rows
  RowOut out[RG_SLOTS];                        // a row's result
};
// then the (k, R) of all warps of the cluster, [RG_SLOTS][C][RG_NW]; then the ring
constexpr size_t RING_SUMS = (sizeof(RingCtl) + 15) / 16 * 16;
__host__ __device__ constexpr size_t ring_start(int C) {
  return RING_SUMS + (size_t)RG_SLOTS * C * RG_NW * sizeof(float2);
}
static_assert(ring_start(4) <= 1024 && SH_CHUNK == RG_CHUNK, "two CTAs of a cluster of 4 on an SM");
constexpr int BAR_IN = 5;  // the first row's scalars are there

// (k, R) to the same place of each of a cluster's CTAs; its barrier there counts the bytes
__device__ __forceinline__ void send(float2* to, uint64_t* bar, float k, float R, uint32_t C,
                                     int lane) {
  if (lane < (int)C)
    asm volatile(
        "st.async.shared::cluster.mbarrier::complete_tx::bytes.b64 [%0], %1, [%2];" ::"r"(
            dsmem_addr(to, (uint32_t)lane)),
        "l"((uint64_t)__float_as_uint(k) | (uint64_t)__float_as_uint(R) << 32),
        "r"(dsmem_addr(bar, (uint32_t)lane))
        : "memory");
}
// every CTA's (k, R) of a cluster, by lane: written into the peers' `to`, whose barrier
// counts the bytes.  Whole warp; ok turns false when the wait runs out.
__device__ __forceinline__ float2 exchange(float2* to, uint64_t* bar, uint32_t phase, float k,
                                           float R, uint32_t C, uint32_t rank, bool& ok,
                                           uint32_t* flags, int lane) {
  send(to + rank, bar, k, R, C, lane);
  __syncwarp();
  if (ok) ok = ring_wait(sm_addr(bar), phase, flags);
  __syncwarp();
  const float2 p = lane < (int)C ? to[lane] : make_float2(LS_MIN, 0.f);
  __syncwarp();
  if (lane == 0) bar_expect(bar, 8 * C);
  return p;
}


// (OWN as an argument: 2.5% of the time of 8,657 rows of V = 151,936 bf16.)
//
// lag 1: a row's gradient is written when the next row has been summed, so that its end is
// worked out meanwhile; the ring has to hold both (30,400 rows of V = 24,576 bf16: 465 us for
// 510, V = 12,480: 352 for 410).  For one CTA to a row: a cluster's would need more slots.
template <typename T, bool HOLD, bool OWN>
__global__ void __launch_bounds__(RG_NT, 2)
    loss_ring(const __grid_constant__ LossArgs a, const int places, const int lag) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  RingCtl& sm = *reinterpret_cast<RingCtl*>(smem_raw);
  using Tr = Traits<T>;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t C, rank;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(C));
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const int64_t G = gridDim.x / C, first = blockIdx.x / C;
  float2* const sums = reinterpret_cast<float2*>(smem_raw + RING_SUMS);
  unsigned char* const ring = smem_raw + ring_start((int)C);
  if (threadIdx.x == 0) {
    for (int i = 0; i < places; ++i) {
      bar_init(&sm.full[i], 1);
      bar_init(&sm.empty[i], RG_NW);
    }
    for (int s = 0; s < RG_SLOTS; ++s) {
      bar_init(&sm.sum_bar[s], C > 1 ? 1 : RG_NW);
      bar_init(&sm.out_bar[s], 1);
      if (C > 1) bar_expect(&sm.sum_bar[s], 8 * RG_NW * C);
    }
    bar_init(&sm.again_bar, 1);
    if (C > 1) bar_expect(&sm.again_bar, 8 * C);
    for (int j = 0; j < RG_TERMS; ++j) sm.stat[j] = make_float2(0.f, 0.f);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
  if (C > 1) cluster_sync_all();  // every CTA's barriers are there
  pdl_wait();
  pdl_trigger();

  bool ok = true;  // no wait has run out
  auto wait = [&](uint64_t* b, uint32_t phase) {
    if (ok) ok = ring_wait(sm_addr(b), phase, a.ctx_flags);
    __syncwarp();
  };
  const Rows rows = rows_of<RG_NT>(
      a, OWN, reinterpret_cast<OwnPlan*>(ring + (size_t)places * RG_BYTES), false);
  const int32_t live = rows.live;
  auto ref_of = [&](int64_t i) { return rows.at(a, i); };
  int place = 0;         // of the ring
  uint32_t turn = 0u;    // how often it has been gone around, its last bit
  auto step = [&]() {
    if (++place == places) {
      place = 0;
      turn ^= 1u;
    }
  };

  if (warp == RG_NW) {
    // ---- bringing chunks in
    int64_t n = 0;
    int4 ref = ref_of(first);
    for (int64_t i = first; i < live; i += G) {
      const int4 ref1 = ref_of(i + G);
      const Share sh = share_of<T>(a, ref.x, C, rank);
      const char* src = sh.x + sizeof(T) * sh.head + 16 * (int64_t)sh.w0;
      for (int32_t left = sh.w1 - sh.w0; left > 0; left -= RG_CHUNK) {
        if (n >= places) wait(&sm.empty[place], turn ^ 1u);
        if (ok && lane == 0) {
          const uint32_t bytes = 16u * (uint32_t)min(RG_CHUNK, left);
          bar_expect(&sm.full[place], bytes);
          asm volatile(
              "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::
                  "r"(sm_addr(ring + (size_t)place * RG_BYTES)),
              "l"(src), "r"(bytes), "r"(sm_addr(&sm.full[place]))
              : "memory");
        }
        src += RG_BYTES;
        if (ok) ++n;
        step();
      }
      ref = ref1;
    }
    // no copy may be in flight when the CTA ends (as none is unless a wait ran out)
    ok = true;
    for (int64_t i = n < places ? 0 : n - places; i < n; ++i)
      wait(&sm.full[(int)(i % places)], (uint32_t)(i / places) & 1u);
  } else if (warp == RG_NW + 1) {
    // ---- the rows' ends
    const double share = rows.share(a);
    uint32_t n = 0, agains = 0;
    int4 ref = ref_of(first), ref1 = ref_of(first + G);
    RowIn in = fetch_row<T, false>(a, rows, share_of<T>(a, ref.x, C, rank), ref, lane);
    // What a peer's gradient may be written over (the logits' own buffer) has been read when
    // this CTA's sums are sent: the next row's scalars are there before a result is given.
    auto landed = [&](RowIn& q) {
      q.xy = __shfl_sync(FULL, q.xy, lane);
      q.edge = __shfl_sync(FULL, q.edge, lane);
    };
    landed(in);
    if (C > 1) named_bar_arrive(BAR_IN, 32 * (RG_NW + 1));
    for (int64_t i = first; i < live; i += G) {
      RowIn next = fetch_row<T, false>(a, rows, share_of<T>(a, ref1.x, C, rank), ref1, lane);
      const int64_t row = ref.x;
      const Share sh = share_of<T>(a, row, C, rank);
      ref = ref1;
      ref1 = ref_of(i + 2 * G);
      const int32_t v = end_of(a, sh, lane);
      T* const g = reinterpret_cast<T*>(a.grad) + row * a.grad_stride;
      const int s = n % RG_SLOTS;
      const uint32_t phase = (n / RG_SLOTS) & 1u;
      ++n;
      wait(&sm.sum_bar[s], phase);
      float k, R, M = INFINITY;
      {
        const float2* q = sums + s * RG_NW * C;
        const float2 none = make_float2(-3e38f, 0.f);
        float2 p = lane < (int)(RG_NW * C) ? q[lane] : none;
        if (C > 4) {
          const float2 p2 = q[32 + lane];
          const float top = fmaxf(p.x, p2.x);
          p = make_float2(top, p.y * rescale2(p.x - top) + p2.y * rescale2(p2.x - top));
        }
        __syncwarp();
        if (C > 1 && lane == 0) bar_expect(&sm.sum_bar[s], 8 * RG_NW * C);
        join(p, 1.f, k, R);
      }
      add_ends(a, sh, in, k, R, lane);
      if (sum_again(k, R, in.xy, a.c2)) {
        robust_sum<T>(a, sh, rank == 0, in.y, M, R, lane);
        if (C > 1) {
          join(exchange(sm.again, &sm.again_bar, agains & 1u, M, R, C, rank, ok,
                        a.ctx_flags, lane), a.c2, M, R);
          ++agains;
        }
        raise_to(a, in.xy, M, R);
      }
      const float wt = (float)(a.norm ? share / (double)in.count : share);
      landed(next);
      end_math<false>(a, row, in, k, R, M, wt, rank == 0, &sm.out[s], &sm.out_bar[s], sm.stat, lane);
      __syncwarp();
      if (HOLD && rank == 0 && v >= 0) put(g + v, v == in.y ? sm.out[s].gy : grad1(sm.out[s], a.c2, in.edge));
      in = next;
    }
  } else {
    // ---- the rows' words
    uint32_t n = 0, m = 0;  // rows summed; written
    const uint32_t mine = first < live ? (uint32_t)((live - 1 - first) / G) + 1u : 0u;
    if (C > 1) named_bar_sync(BAR_IN, 32 * (RG_NW + 1));
    const int at = warp * 32 + lane;  // this lane's first word of a chunk
    int4 ref = ref_of(first), next = ref_of(first + G);  // the row to be summed; the one after it
    int4 held = ref, last = ref;  // the row to be written; the one summed last
    int place0 = 0;               // its place
    while ((HOLD ? m : n) < mine) {
      if (n < mine) {
        // forward
        const Share sh = share_of<T>(a, ref.x, C, rank);
        const int32_t yw = word_of<T>(a, sh, ref.z);
        const int yj = ref.z - sh.head - yw * Tr::VEC;
        float k = -3e38f;
        float2 S = make_float2(0.f, 0.f);
        for (int32_t w = sh.w0; w < sh.w1; w += RG_CHUNK) {
          wait(&sm.full[place], turn);
          const uint4* st = reinterpret_cast<const uint4*>(ring + (size_t)place * RG_BYTES) + at;
          uint4 v[RG_W];
#pragma unroll
          for (int q = 0; q < RG_W; ++q) v[q] = st[32 * RG_NW * q];
          if (w + RG_CHUNK > sh.w1) {
#pragma unroll
            for (int q = 0; q < RG_W; ++q)
              if (w + 32 * RG_NW * q + at >= sh.w1)
                v[q] = make_uint4(Tr::NEG_WORD, Tr::NEG_WORD, Tr::NEG_WORD, Tr::NEG_WORD);
          }
          if ((uint32_t)(yw - w) < (uint32_t)RG_CHUNK) {
#pragma unroll
            for (int q = 0; q < RG_W; ++q)
              if (w + 32 * RG_NW * q + at == yw) v[q] = without<T>(v[q], yj);
          }
          if (!HOLD) {
            __syncwarp();  // every lane has its words
            if (lane == 0) bar_arrive(&sm.empty[place]);
          }
          step();
          add_words<T>(k, S, v, a.c2, w == sh.w0);
        }
        float R;
        join(make_float2(k, S.x + S.y), 1.f, k, R);
        const int s = n % RG_SLOTS;
        if (!HOLD && n >= 1) wait(&sm.out_bar[s ^ 1], ((n - 1) / RG_SLOTS) & 1u);
        if (C > 1) {
          send(sums + (s * C + rank) * RG_NW + warp, &sm.sum_bar[s], k, R, C, lane);
        } else if (lane == 0) {
          sums[s * RG_NW + warp] = make_float2(k, R);
          bar_arrive(&sm.sum_bar[s]);
        }
        last = ref;
        ++n;
        ref = next;
        next = ref_of(first + (int64_t)(n + 1) * G);
      }
      if (HOLD && (n > (uint32_t)lag || n == mine)) {
        // backward
        const Share sh = share_of<T>(a, held.x, C, rank);
        T* const g = reinterpret_cast<T*>(a.grad) + held.x * a.grad_stride + sh.head;
        const bool vec = ((reinterpret_cast<uintptr_t>(sh.x + sizeof(T) * sh.head) ^
                           reinterpret_cast<uintptr_t>(g)) & 15u) == 0;
        const int32_t yw = word_of<T>(a, sh, held.z);
        const int yj = held.z - sh.head - yw * Tr::VEC;
        const int s = m % RG_SLOTS;
        wait(&sm.out_bar[s], (m / RG_SLOTS) & 1u);
        const RowOut o = sm.out[s];
        for (int32_t w = sh.w0; w < sh.w1; w += RG_CHUNK) {
          const uint4* st = reinterpret_cast<const uint4*>(ring + (size_t)place0 * RG_BYTES) + at;
          T* const to = g + (int64_t)(w + at) * Tr::VEC;
          uint4 v[RG_W];
#pragma unroll
          for (int q = 0; q < RG_W; ++q) v[q] = st[32 * RG_NW * q];
          if (o.mode == ROW_FAST) {
#pragma unroll
            for (int q = 0; q < RG_W; ++q) v[q] = grad_word<T, false>(o, a.c2, v[q]);
          } else if (o.mode == ROW_ROBUST) {
#pragma unroll
            for (int q = 0; q < RG_W; ++q) v[q] = grad_word<T, true>(o, a.c2, v[q]);
          } else {
#pragma unroll
            for (int q = 0; q < RG_W; ++q) v[q] = make_uint4(0u, 0u, 0u, 0u);
          }
          __syncwarp();
          if (lane == 0) bar_arrive(&sm.empty[place0]);
          if (++place0 == places) place0 = 0;
          if (vec && w + RG_CHUNK <= sh.w1) {
#pragma unroll
            for (int q = 0; q < RG_W; ++q)
              *reinterpret_cast<uint4*>(to + 32 * RG_NW * q * Tr::VEC) = v[q];
          } else {
#pragma unroll
            for (int q = 0; q < RG_W; ++q)
              if (w + 32 * RG_NW * q + at < sh.w1) put_word(to + 32 * RG_NW * q * Tr::VEC, v[q], vec);
          }
          if ((uint32_t)(yw - w) < (uint32_t)RG_CHUNK && ((yw - w) % (32 * RG_NW)) == at)
            put(g + (int64_t)yw * Tr::VEC + yj, o.gy);
        }
        ++m;
        held = m == n ? ref : last;
      }
    }
    if (HOLD)  // the rows that do not count
      for (int64_t i = first; i < a.n_rows - live; i += G) {
        const int64_t row = rows.skipped(a, i);
        const Share sh = share_of<T>(a, row, C, rank);
        T* const g = reinterpret_cast<T*>(a.grad) + row * a.grad_stride;
        const bool vec = ((reinterpret_cast<uintptr_t>(sh.x) ^ reinterpret_cast<uintptr_t>(g)) & 15u) == 0;
        for (int32_t w = sh.w0 + at; w < sh.w1; w += 32 * RG_NW)
          put_word(g + sh.head + (int64_t)w * Tr::VEC, make_uint4(0u, 0u, 0u, 0u), vec);
        const int32_t v = end_of(a, sh, lane);
        if (warp == 0 && rank == 0 && v >= 0) put(g + v, 0.f);
      }
  }
  __syncthreads();
  if (C > 1) cluster_sync_all();  // no peer writes here any more
  const int64_t groups = max((int64_t)1, min(G, (int64_t)live));
  if (warp == 0 && rank == 0 && first < groups) write_stats(a, sm.stat, 1, first, groups, lane);
}

// ---- short rows: one to a warp ---------------------------------------------------------------
//
// A row's end is some 500 instructions one after the other, 2,600 to 4,400 cycles of a warp.
// Where a row is short that is longer than its data take, so each warp has a row of its
// own, brought into its part of shared memory by one bulk copy: up to 20 rows of an SM are
// in work at a time, some of them on their way while others are summed, ended or written.
// (30,400 rows of V = 5,504 bf16 with their gradient: 133 us for 317 with a CTA to a row,
// 1,500 of them 27 for 33; V = 512: 51 for 301.  Rows of 25 KB, eight on an SM: 356 for 352 as
// the ring does them now, 61 for 55 with 2,500.  More warps leave a warp fewer registers:
// sixteen 143, unrolling the gradient's loop with them 188, twelve 145.)
constexpr int RW_MOST = 10;  // warps of a CTA; two CTAs on an SM
struct RowsCtl {
  uint64_t full[RW_MOST];    // a row has landed
  RowOut out[RW_MOST];
  float2 stat[RW_MOST * RG_TERMS];
};
constexpr size_t RW_CTL = (sizeof(RowsCtl) + 15) / 16 * 16;

template <typename T, bool PREF, bool HOLD>
__global__ void __launch_bounds__(32 * RW_MOST, 2)
    loss_rows(const __grid_constant__ LossArgs a, const int bytes) {  // of a warp's part
  extern __shared__ __align__(16) unsigned char smem_raw[];
  RowsCtl& sm = *reinterpret_cast<RowsCtl*>(smem_raw);
  using Tr = Traits<T>;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  unsigned char* const part = smem_raw + RW_CTL + (size_t)warp * bytes;
  uint64_t* const full = &sm.full[warp];
  float2* const stat = sm.stat + warp * RG_TERMS;
  if (lane == 0) {
    bar_init(full, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (lane < RG_TERMS) stat[lane] = make_float2(0.f, 0.f);
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  const Rows rows{nullptr, (int32_t)__ldcg(a.totals)};
  const double share = PREF ? 0.0 : rows.share(a);
  const int64_t G = (int64_t)gridDim.x * warps, first = (int64_t)warp * gridDim.x + blockIdx.x;
  uint32_t phase = 0;
  int4 ref = rows.at(a, first);
  for (int64_t i = first; i < rows.live; i += G) {
    const Share sh = share_of<T>(a, ref.x, 1, 0);
    if (lane == 0) {
      const uint32_t n = 16u * (uint32_t)sh.words;
      bar_expect(full, n);
      if (n > 0)
        asm volatile(
            "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::
                "r"(sm_addr(part)),
            "l"(sh.x + sizeof(T) * sh.head), "r"(n), "r"(sm_addr(full))
            : "memory");
    }
    const RowIn in = fetch_row<T, PREF>(a, rows, sh, ref, lane);
    const int4 ref1 = rows.at(a, i + G);
    const int32_t yw = word_of<T>(a, sh, in.y);
    const int yj = in.y - sh.head - yw * Tr::VEC;
    if (!ring_wait(sm_addr(full), phase, a.ctx_flags)) {
      ring_wait(sm_addr(full), phase, a.ctx_flags);  // no copy may be in flight at the end
      break;
    }
    phase ^= 1u;
    __syncwarp();
    const uint4* const st = reinterpret_cast<const uint4*>(part) + lane;
    float k = -3e38f, R, M = INFINITY;
    float2 S = make_float2(0.f, 0.f);
    for (int32_t w = 0; w < sh.words; w += 32 * RG_W) {
      uint4 v[RG_W];
#pragma unroll
      for (int q = 0; q < RG_W; ++q)
        v[q] = w + 32 * q + lane < sh.words
                   ? st[w + 32 * q]
                   : make_uint4(Tr::NEG_WORD, Tr::NEG_WORD, Tr::NEG_WORD, Tr::NEG_WORD);
      if ((uint32_t)(yw - w) < 32u * RG_W) {
#pragma unroll
        for (int q = 0; q < RG_W; ++q)
          if (w + 32 * q + lane == yw) v[q] = without<T>(v[q], yj);
      }
      add_words<T>(k, S, v, a.c2, w == 0);
    }
    join(make_float2(k, S.x + S.y), 1.f, k, R);
    add_ends(a, sh, in, k, R, lane);
    if (sum_again(k, R, in.xy, a.c2)) {
      robust_sum<T>(a, sh, true, in.y, M, R, lane);
      raise_to(a, in.xy, M, R);
    }
    const float wt = PREF ? 0.f : (float)(a.norm ? share / (double)in.count : share);
    end_math<PREF>(a, ref.x, in, k, R, M, wt, true, HOLD ? &sm.out[warp] : nullptr, nullptr, stat,
                   lane);
    __syncwarp();
    if (HOLD) {
      const RowOut o = sm.out[warp];
      T* const g = reinterpret_cast<T*>(a.grad) + (int64_t)ref.x * a.grad_stride;
      T* const gw = g + sh.head;
      const bool vec = ((reinterpret_cast<uintptr_t>(sh.x) ^ reinterpret_cast<uintptr_t>(g)) & 15u) == 0;
      for (int32_t w = lane; w < sh.words; w += 32) {
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (o.mode == ROW_FAST) v = grad_word<T, false>(o, a.c2, st[w - lane]);
        else if (o.mode == ROW_ROBUST) v = grad_word<T, true>(o, a.c2, st[w - lane]);
        put_word(gw + (int64_t)w * Tr::VEC, v, vec);
        if (w == yw) put(gw + (int64_t)w * Tr::VEC + yj, o.gy);
      }
      const int32_t v = end_of(a, sh, lane);
      if (v >= 0) put(g + v, v == in.y ? o.gy : grad1(o, a.c2, in.edge));
      __syncwarp();  // every lane has read what the next row is written over
    }
    ref = ref1;
  }
  if (HOLD)  // the rows that do not count
    for (int64_t i = first; i < a.n_rows - rows.live; i += G) {
      const int64_t row = rows.skipped(a, i);
      const Share sh = share_of<T>(a, row, 1, 0);
      T* const g = reinterpret_cast<T*>(a.grad) + row * a.grad_stride;
      const bool vec = ((reinterpret_cast<uintptr_t>(sh.x) ^ reinterpret_cast<uintptr_t>(g)) & 15u) == 0;
      for (int32_t w = lane; w < sh.words; w += 32)
        put_word(g + sh.head + (int64_t)w * Tr::VEC, make_uint4(0u, 0u, 0u, 0u), vec);
      const int32_t v = end_of(a, sh, lane);
      if (v >= 0) put(g + v, 0.f);
    }
  if (PREF) return;
  __syncthreads();
  const int64_t groups = max((int64_t)1, min((int64_t)gridDim.x, (int64_t)rows.live));
  if (warp == 0 && blockIdx.x < groups) write_stats(a, sm.stat, warps, blockIdx.x, groups, lane);
}

// ---- backward from the rows' states ---------------------------------------------------------
//
// One CTA per segment of a row, the last rows first: those are still in L2 after the
// forward sweep.
constexpr int BW_NT = 256;
constexpr int BW_W = 4;                      // words per thread
constexpr int BW_SEG = BW_NT * BW_W;         // words of a segment

template <typename T, bool PREF>
__global__ void __launch_bounds__(BW_NT) loss_backward(const LossArgs a, int32_t segs) {
  using Tr = Traits<T>;
  const int tid = threadIdx.x;
  pdl_wait();
  pdl_trigger();
  const int64_t row = a.n_rows - 1 - blockIdx.x / segs;
  const int32_t seg = (int32_t)(blockIdx.x % segs);
  const T* x = reinterpret_cast<const T*>(a.logits) + row * a.row_stride;
  T* g = reinterpret_cast<T*>(a.grad) + row * a.grad_stride;
  const RowWords rw = RowWords::of(x, a.vocab);
  const uint4* xw = reinterpret_cast<const uint4*>(x + rw.head);
  const int32_t w0 = seg * BW_SEG + tid, words = (int32_t)rw.words;
  const bool vec = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(g)) & 15u) == 0;
  const int32_t r = __ldcg(a.row_req + row);
  uint4 v[BW_W];
#pragma unroll
  for (int k = 0; k < BW_W; ++k)
    if (r >= 0 && w0 + k * BW_NT < words) v[k] = ld_stream(xw + w0 + k * BW_NT);
  RowOut o;
  o.mode = ROW_ZERO;
  o.K = o.nk = o.gy = o.M = 0.f;
  int32_t y = -1;
  if (r >= 0) {
    const float4 q = __ldcg(a.state + row);
    const float k = PREF ? __ldcg(a.coef + r) * (a.grad_scale * a.inv_t) : __ldcg(a.z + row);
    RowState st;
    st.K = q.x;
    st.adj = q.y;
    st.rest = q.z;
    st.M = q.w;
    o = row_out(st, k);
    y = __ldcg(a.chosen + row);
  }
  const int64_t yo = (int64_t)y - rw.head;
  const int32_t yw = y >= 0 && (int64_t)y < a.vocab && yo >= 0 ? (int32_t)(yo / Tr::VEC) : -1;
#pragma unroll
  for (int q = 0; q < BW_W; ++q) {
    const int32_t i = w0 + q * BW_NT;
    if (i < words) {
      T* to = g + rw.head + (int64_t)i * Tr::VEC;
      uint4 w = make_uint4(0u, 0u, 0u, 0u);
      if (o.mode == ROW_FAST) w = grad_word<T, false>(o, a.c2, v[q]);
      else if (o.mode == ROW_ROBUST) w = grad_word<T, true>(o, a.c2, v[q]);
      put_word(to, w, vec);
      if (i == yw) put(to + (yo - (int64_t)yw * Tr::VEC), o.gy);
    }
  }
  if (seg > 0) return;
  const int64_t ve = tid < 8 ? (tid < rw.head ? tid : -1)
                             : (tid - 8 < rw.tail ? rw.head + rw.words * Tr::VEC + tid - 8 : -1);
  if (ve >= 0) put(g + ve, ve == y ? o.gy : grad1(o, a.c2, Tr::elem(x, ve)));
}

// ---- answer pairs -------------------------------------------------------------------------

// log ratio of request r: sum over its counted tokens of l - ref.  Whole warp.
__device__ __forceinline__ double pair_ratio(const LossArgs& a, int64_t r, int lane) {
  const int64_t lo = a.offsets[r], hi = a.offsets[r + 1];
  double s = 0.;
  if (__ldcg(a.count + r) > 0)
    for (int64_t t = lo + lane; t < hi; t += 4 * 32) {
      float z[4];
      bool on[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        on[q] = t + 32 * q < hi && __ldcg(a.row_req + t + 32 * q) == (int32_t)r;
        z[q] = t + 32 * q < hi ? __ldcg(a.z + t + 32 * q) : 0.f;
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) s += on[q] ? (double)z[q] : 0.;
    }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(FULL, s, o);
  return s;
}

// Two warps per pair, one for each answer; the last CTA sums the statistics.
constexpr int PR_PAIRS = 4;  // pairs of a CTA
static __global__ void __launch_bounds__(64 * PR_PAIRS) loss_pairs(const LossArgs a) {
  __shared__ double ratio[2 * PR_PAIRS];
  __shared__ int last;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t n_pairs = a.n_req / 2, i0 = (int64_t)blockIdx.x * PR_PAIRS;
  {
    const int64_t r = 2 * i0 + warp;
    double s = 0.;
    if (r < a.n_req) s = pair_ratio(a, r, lane);
    if (lane == 0) ratio[warp] = s;
  }
  __syncthreads();
  const int64_t i = i0 + tid;
  if (tid < PR_PAIRS && i < n_pairs) {
    double sw = ratio[2 * tid], sl = ratio[2 * tid + 1];
    const int32_t nw = __ldcg(a.count + 2 * i), nl = __ldcg(a.count + 2 * i + 1);
    if (a.length_norm) {
      sw /= (double)max(nw, 1);
      sl /= (double)max(nl, 1);
    }
    a.ratio[2 * i] = (float)sw;
    a.ratio[2 * i + 1] = (float)sl;
    float t[LS_NSTAT] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    float cw = 0.f, cl = 0.f;
    if (nw > 0 && nl > 0) {
      const double d = sw - sl;
      const float h = (float)((double)a.beta * d - (double)a.margin);
      float f, slope;  // loss and d loss / d d
      if (a.loss == 0) {
        const float e = log1pf(expf(-fabsf(h)));
        const float up = e + fmaxf(-h, 0.f), down = e + fmaxf(h, 0.f);
        // (either may be infinite: a masked emitted token; without weight it is no part)
        f = (a.smooth < 1.f ? (1.f - a.smooth) * up : 0.f) + (a.smooth > 0.f ? a.smooth * down : 0.f);
        slope = a.beta * (a.smooth / (1.f + expf(-h)) - (1.f - a.smooth) / (1.f + expf(h)));
      } else if (a.loss == 1) {
        const double q = d - 0.5 / (double)a.beta;
        f = (float)(q * q);
        slope = (float)(2. * q);
      } else {
        f = fmaxf(1.f - h, 0.f);
        slope = h < 1.f ? -a.beta : 0.f;
        if (h != h) f = slope = h;
      }
      t[0] = f;
      t[1] = d > 0. ? 1.f : 0.f;
      t[2] = h;
      t[3] = (float)((double)a.beta * sw);
      t[4] = (float)((double)a.beta * sl);
      const float share = slope / (float)__ldcg(a.totals + 1);
      cw = a.length_norm ? share / (float)nw : share;
      cl = a.length_norm ? -share / (float)nl : -share;
    }
    a.coef[2 * i] = cw;
    a.coef[2 * i + 1] = cl;
    for (int j = 0; j < LS_NSTAT; ++j) a.term[i * LS_NSTAT + j] = t[j];
    __threadfence();
  }
  __syncthreads();
  if (tid == 0) last = atom_add_acq_rel(a.ticket + 1, 1) == (int)gridDim.x - 1;
  __syncthreads();
  if (!last || warp >= LS_NSTAT - 1) return;
  double v = 0.;
  for (int64_t q = lane; q < n_pairs; q += 32) v += (double)__ldcg(a.term + q * LS_NSTAT + warp);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
  const int64_t used = __ldcg(a.totals + 1);
  if (lane == 0) a.stats[warp] = used > 0 ? (float)(v / (double)used) : 0.f;
  if (tid == 0) a.ticket[1] = 0;
}

}  // namespace prk
