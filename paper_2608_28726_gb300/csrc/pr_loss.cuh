// Training losses over logit rows: the clipped policy loss with a KL term and the
// loss of paired log ratios, with the gradient of the logits.
//
// Row t with logits x, emitted token y and temperature T has z = x / T,
// l = z_y - log sum_v exp(z_v), and for any loss L that depends on the row through
// l alone dL/dx_v = (dL/dl) (onehot_y(v) - p_v) / T, p = softmax(z).  So a row needs
// two sweeps over its logits, with the scalar dL/dl between them:
//   forward   M = max x and S = sum 2^(c (x - M)), c = log2(e) / T; both are kept
//             against a reference m of each thread's own: x - m is exact where it
//             matters (equal logits of any magnitude give 2^0), -inf gives 2^-inf = 0,
//             and the lowest finite value is a maximum like any other
//   backward  g_v = dL/dl / T (onehot - 2^(c (x_v - M) - log2 S))
// The emitted token's own term e_y stays out of the forward sum: with R the sum of the
// others, 1 - p_y = R / (R + e_y) and l = -log(1 + R / e_y) keep their relative
// accuracy where p_y is close to 1 and 1 - p_y or log(R + e_y) would cancel.
// The policy loss' dL/dl needs the row alone; the preference loss' needs the log
// ratios of the row's whole answer pair.
#pragma once

#include "pr_kernels.cuh"

namespace prk {

constexpr int LS_NT = 512;
constexpr int LS_NW = LS_NT / 32;
constexpr int LS_NSTAT = 6;   // statistics of a loss (the preference loss has 5)
constexpr float LS_MIN = -3.402823466e38f;  // "no maximum yet": the lowest finite value

enum LossKind { LOSS_POLICY = 0, LOSS_PREF_FWD = 1, LOSS_PREF_BWD = 2 };

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
  float inv_t, c2, skew;  // 1 / T, log2(e) / T, c2 ln 2 - inv_t
  float grad_scale;
  float* stats;
  float* ratio;
  float* logp;
  void* grad;
  int64_t grad_stride;
  // workspace
  int32_t* ticket;     // [2] arrivals, zero between calls
  int64_t* totals;     // counted tokens; requests with some (policy) or pairs of such
  int32_t* count;      // [n_req] counted tokens
  float* coef;         // [n_req] dL / d log ratio (preference)
  float* term;         // [n_req / 2][LS_NSTAT] the pairs' statistics
  float4* state;       // [n_rows] M, log2 S, l - ref, 1 - p_y (preference)
  double* part;        // [groups][LS_NSTAT] statistics of each group's rows
  uint32_t* ctx_flags;
};

// the request that owns row t and its counted tokens; -1 when there is none or its
// bounds are not inside the batch.  Whole warp.
__device__ __forceinline__ int32_t loss_request(const LossArgs& a, int64_t t, int lane) {
  if (!a.offsets) return 0;
  const int32_t r = find_request(a.offsets, a.n_req, t, lane);
  if (r < 0) return -1;
  return a.offsets[r] >= 0 && a.offsets[r + 1] <= a.n_rows ? r : -1;
}

// ---- counted tokens -------------------------------------------------------------------

// One CTA per request; the last one to finish sums up.
static __global__ void __launch_bounds__(256) loss_plan(const LossArgs a, int pairs) {
  __shared__ int64_t part[8];
  __shared__ int last;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t r = blockIdx.x;
  const int64_t lo = a.offsets ? a.offsets[r] : 0, hi = a.offsets ? a.offsets[r + 1] : a.n_rows;
  const bool bad = lo < 0 || hi < lo || hi > a.n_rows;
  int64_t n = 0;
  if (!bad) {
    if (!a.mask) n = tid == 0 ? hi - lo : 0;
    else
      for (int64_t t = lo + tid; t < hi; t += 256) n += a.mask[t] != 0;
  }
  auto block_sum = [&](int64_t v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
    __syncthreads();
    if (lane == 0) part[warp] = v;
    __syncthreads();
    v = 0;
    for (int w = 0; w < 8; ++w) v += part[w];
    return v;
  };
  n = block_sum(n);
  if (tid == 0) {
    a.count[r] = (int32_t)n;
    if (bad) atomicOr(a.ctx_flags, FLAG_BAD_OFFSETS);
    else if (lo == hi) atomicOr(a.ctx_flags, FLAG_EMPTY_REQ);
    last = atom_add_acq_rel(a.ticket, 1) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  int64_t total = 0, used = 0;
  for (int64_t q = tid; q < a.n_req; q += 256) {
    const int32_t k = __ldcg(a.count + q);
    total += k;
    if (!pairs) used += k > 0;
    else if ((q & 1) == 0) used += k > 0 && __ldcg(a.count + q + 1) > 0;
  }
  total = block_sum(total);
  used = block_sum(used);
  if (tid == 0) {
    a.totals[0] = total;
    a.totals[1] = used;
    *a.ticket = 0;
  }
}

// ---- the losses of one row / pair -------------------------------------------------------

struct PolicyTerms {
  float loss, surrogate, kl, ratio, clipped, old_kl;
  float slope;  // dloss / dl
};

__device__ __forceinline__ PolicyTerms policy_terms(const LossArgs& a, float l, float l_lo,
                                                    float old, float ref, float adv) {
  PolicyTerms p;
  const float d = a.old_logp ? (l - old) + l_lo : l - l;  // (NaN for a row without l)
  p.ratio = expf(d);
  p.old_kl = expm1f(d) - d;
  const float free = p.ratio * adv;
  const float bound = fminf(fmaxf(p.ratio, a.clip_lo), a.clip_hi) * adv;
  p.clipped = bound < free ? 1.f : 0.f;
  p.surrogate = bound < free ? bound : free;
  p.slope = bound < free ? 0.f : -free;
  p.loss = -p.surrogate;
  p.kl = 0.f;
  if (a.ref_logp) {
    const float q = (ref - l) - l_lo, e = expm1f(q);
    p.kl = e - q;
    p.loss = fmaf(a.kl_coef, p.kl, p.loss);
    if (a.kl_coef != 0.f) p.slope = fmaf(-a.kl_coef, e, p.slope);
  }
  return p;
}

// ---- a row's words ------------------------------------------------------------------------

// the factor from the reference m to M: expf, whose mean error is a tenth of ex2's
// (below): a row's sum would take that on at each step of its merges
__device__ __forceinline__ float rescale(float m, float M, float inv_t) {
  return expf((m - M) * inv_t);
}

// running (m, S): S = sum 2^(c (x - m)).  m is raised when a word goes past it by
// enough that S could grow out of proportion, not at every new maximum.
struct RowSum {
  float m;
  float2 S;
  __device__ __forceinline__ void reset() {
    m = LS_MIN;
    S = make_float2(0.f, 0.f);
  }
  __device__ __forceinline__ void raise(float top, float c2, float inv_t) {
    if ((top - m) * c2 > 8.f) {
      const float f = rescale(m, top, inv_t);
      S = __fmul2_rn(S, make_float2(f, f));
      m = top;
    }
  }
  __device__ __forceinline__ void add2(float x, float y, float c2) {
    float2 d = __fadd2_rn(make_float2(x, y), make_float2(-m, -m));
    d = __fmul2_rn(d, make_float2(c2, c2));
    S = __fadd2_rn(S, make_float2(ex2(d.x), ex2(d.y)));
  }
  __device__ __forceinline__ void add1(float x, float c2, float inv_t) {
    if (x != x) S.x = x;
    raise(x, c2, inv_t);
    S.x += ex2((x - m) * c2);
  }
};

template <typename T>
__device__ __forceinline__ void add_word(RowSum& s, const uint4& w, float c2) {
  using Tr = Traits<T>;
#pragma unroll
  for (int j = 0; j < Tr::VEC; j += 2) s.add2(Tr::at(w, j), Tr::at(w, j + 1), c2);
}

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

// A row's state from R = sum over the other tokens of 2^(c (x_v - m)) and the emitted
// token's logit: M, log2 S, 1 - p_y, and l = l_hi + l_lo: a log ratio sums hundreds of
// differences l - ref, whose errors must neither be l's rounding (2^-24 |l|) nor
// lean to one side.  So ln S = e ln 2 + ln f is taken with e ln 2 in two parts (Cody
// and Waite's reduction; the first product is exact), c (x_y - M) keeps its rounding, the
// scale is the one that the sums were taken with (c2, not 1 / T: an error common to both
// cancels in the mean), and ex2's mean error, -5.1e-8 relative over 2^24 arguments in
// [-30, 0], is added back.  Mean error of l over sampled rows: 1e-7 without all this.
constexpr float LN2_A = 0.693145751953125f;       // ln 2 to 16 bits
constexpr float LN2_B = 1.42860682e-06f;  // ln 2 - LN2_A
constexpr float EX2_LOW = 5.1e-8f;
struct RowEnd {
  float M, lS, l, l_lo, rest;
  __device__ __forceinline__ RowEnd(const LossArgs& a, float m, float R, float xy, bool ok) {
    M = ok ? fmaxf(m, xy) : m;  // (an xy of NaN leaves m, and its term is NaN)
    R *= rescale(m, M, a.inv_t);
    const float ey = ok ? ex2((xy - M) * a.c2) : NAN;
    const float S = R + ey;
    lS = log2f(S);
    rest = R / S;
    if (ey > 0.25f * S) {
      const float q = R / ey;
      l = -log1pf(fmaf(q, EX2_LOW, q));
      l_lo = 0.f;
    } else {
      const float d = xy - M, u = d * a.inv_t;
      int e = (int)(__float_as_uint(S) >> 23) - 127;
      float f = __uint_as_float((__float_as_uint(S) & 0x7fffffu) | 0x3f800000u);
      if (f > 1.41f) {
        f *= 0.5f;
        ++e;
      }
      const float big = (float)e * LN2_A, hi = u - big, t = hi - u;
      float lo = (u - (hi - t)) + (-big - t);  // hi's rounding
      lo += fmaf(d, a.inv_t, -u) + d * a.skew;
      lo -= log1pf(f - 1.f) + fmaf((float)e, LN2_B, EX2_LOW);
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

// backward of two logits: nk (p_x, p_y), nk = -dL/dl / T
struct RowGrad {
  float M, lS, nk, c2;
  __device__ __forceinline__ float2 two(float x, float y) const {
    float2 d = __fadd2_rn(make_float2(x, y), make_float2(-M, -M));
    d = __ffma2_rn(d, make_float2(c2, c2), make_float2(-lS, -lS));
    return __fmul2_rn(make_float2(ex2(d.x), ex2(d.y)), make_float2(nk, nk));
  }
  __device__ __forceinline__ float one(float x) const { return nk * ex2(fmaf(x - M, c2, -lS)); }
};

__device__ __forceinline__ uint32_t bf16_pair(float2 v) {
  const __nv_bfloat162 h = __float22bfloat162_rn(v);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <typename T>
__device__ __forceinline__ uint4 grad_word(const RowGrad& g, const uint4& w) {
  using Tr = Traits<T>;
  if constexpr (sizeof(T) == 2) {
    return make_uint4(bf16_pair(g.two(Tr::at(w, 0), Tr::at(w, 1))),
                      bf16_pair(g.two(Tr::at(w, 2), Tr::at(w, 3))),
                      bf16_pair(g.two(Tr::at(w, 4), Tr::at(w, 5))),
                      bf16_pair(g.two(Tr::at(w, 6), Tr::at(w, 7))));
  } else {
    const float2 u = g.two(Tr::at(w, 0), Tr::at(w, 1)), v = g.two(Tr::at(w, 2), Tr::at(w, 3));
    return make_uint4(__float_as_uint(u.x), __float_as_uint(u.y), __float_as_uint(v.x),
                      __float_as_uint(v.y));
  }
}
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }

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

// ---- rows, one CTA each, two sweeps over global memory --------------------------------------

template <typename T, int KIND>
__global__ void __launch_bounds__(LS_NT) loss_rows(const LossArgs a) {
  using Tr = Traits<T>;
  __shared__ float pm[LS_NW], pS[LS_NW];
  __shared__ float sh[4];
  __shared__ int32_t sreq;
  __shared__ int last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  double stat[LS_NSTAT] = {0., 0., 0., 0., 0., 0.};
  pdl_wait();
  pdl_trigger();
  for (int64_t row = blockIdx.x; row < a.n_rows; row += gridDim.x) {
    const T* x = reinterpret_cast<const T*>(a.logits) + row * a.row_stride;
    T* g = reinterpret_cast<T*>(a.grad) + row * a.grad_stride;
    const RowWords rw = RowWords::of(x, a.vocab);
    const uint4* xw = reinterpret_cast<const uint4*>(x + rw.head);
    const int32_t y = a.chosen[row];
    __syncthreads();
    if (warp == 0) {
      const bool on = !a.mask || a.mask[row] != 0;
      const int32_t r = on ? loss_request(a, row, lane) : -1;
      if (lane == 0) {
        sreq = r;
        sh[3] = y >= 0 && (int64_t)y < a.vocab ? Tr::elem(x, y) : NAN;
      }
    }
    __syncthreads();
    const int32_t r = sreq;
    const bool yok = y >= 0 && (int64_t)y < a.vocab;
    const int64_t ye = (int64_t)y - rw.head, yw = yok && ye >= 0 ? ye / Tr::VEC : -1;
    const int yj = (int)(ye - yw * Tr::VEC);
    float M, lS, k = 0.f, rest = 0.f;
    if (KIND != LOSS_PREF_BWD) {
      if (r < 0) {
        if (tid == 0) a.logp[row] = 0.f;
      } else {
        RowSum s;
        s.reset();
        for (int64_t i = tid; i < rw.words; i += LS_NT) {
          uint4 w = xw[i];
          if (i == yw) w = without<T>(w, yj);
          s.raise(Tr::gmax(w), a.c2, a.inv_t);
          add_word<T>(s, w, a.c2);
        }
        if (tid < rw.head && tid != y) s.add1(Tr::elem(x, tid), a.c2, a.inv_t);
        const int64_t vt = rw.head + rw.words * Tr::VEC + tid;
        if (tid < rw.tail && vt != y) s.add1(Tr::elem(x, vt), a.c2, a.inv_t);
        float S = s.S.x + s.S.y;
        const float m = unord(__reduce_max_sync(FULL, ord(s.m)));
        S *= rescale(s.m, m, a.inv_t);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) S += __shfl_xor_sync(FULL, S, o);
        if (lane == 0) {
          pm[warp] = m;
          pS[warp] = S;
        }
        __syncthreads();
        M = LS_MIN;
        for (int w = 0; w < LS_NW; ++w) M = fmaxf(M, pm[w]);
        S = 0.f;
        for (int w = 0; w < LS_NW; ++w) S = fmaf(pS[w], rescale(pm[w], M, a.inv_t), S);
        const RowEnd e(a, M, S, sh[3], yok);
        const float l = e.l;
        M = e.M;
        lS = e.lS;
        rest = e.rest;
        if (tid == 0) {
          a.logp[row] = l;
          if (!yok) atomicOr(a.ctx_flags, FLAG_BAD_CHOSEN);
          else if (isnan(l)) atomicOr(a.ctx_flags, FLAG_NONFINITE);
        }
        if (KIND == LOSS_POLICY) {
          const float old = a.old_logp ? a.old_logp[row] : 0.f;
          const float ref = a.ref_logp ? a.ref_logp[row] : 0.f;
          const PolicyTerms p = policy_terms(a, l, e.l_lo, old, ref, a.adv[a.per_request ? r : row]);
          const double wt = a.norm ? 1.0 / ((double)a.totals[1] * (double)a.count[r])
                                   : 1.0 / (double)a.totals[0];
          k = (float)wt * p.slope * (a.grad_scale * a.inv_t);
          stat[0] += wt * (double)p.loss;
          stat[1] += wt * (double)p.surrogate;
          stat[2] += wt * (double)p.kl;
          stat[3] += wt * (double)p.ratio;
          stat[4] += wt * (double)p.clipped;
          stat[5] += wt * (double)p.old_kl;
        } else if (tid == 0) {
          a.state[row] = make_float4(M, lS, (l - (a.ref_logp ? a.ref_logp[row] : 0.f)) + e.l_lo, rest);
        }
      }
    } else if (r >= 0) {
      const float4 st = a.state[row];
      M = st.x;
      lS = st.y;
      rest = st.w;
      k = a.coef[r] * (a.grad_scale * a.inv_t);
    }
    if (KIND == LOSS_PREF_FWD || !a.grad) continue;
    const bool zero = r < 0 || k == 0.f;
    const RowGrad rg{M, lS, -k, a.c2};
    // the emitted token's entry k (1 - p_y) is written by the thread whose word holds it
    const bool vec = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(g)) & 15u) == 0;
    const float gy = zero ? 0.f : k * rest;
    __syncthreads();  // every thread has read what the row's gradient may overwrite
    for (int64_t i = tid; i < rw.words; i += LS_NT) {
      uint4 o = make_uint4(0u, 0u, 0u, 0u);
      if (!zero) o = grad_word<T>(rg, xw[i]);
      const int64_t v0 = rw.head + i * Tr::VEC;
      if (vec) *reinterpret_cast<uint4*>(g + v0) = o;
      else
        for (int j = 0; j < Tr::VEC; ++j) put(g + v0 + j, Tr::at(o, j));
      if (!zero && i == yw) put(g + y, gy);
    }
    auto edge = [&](int64_t v) {
      put(g + v, zero ? 0.f : (v == y ? gy : rg.one(Tr::elem(x, v))));
    };
    if (tid < rw.head) edge(tid);
    if (tid < rw.tail) edge(rw.head + rw.words * Tr::VEC + tid);
  }
  if (KIND != LOSS_POLICY) return;
  // the statistics: each CTA's sum over its rows, then the CTAs' in order
  if (tid == 0) {
    for (int j = 0; j < LS_NSTAT; ++j) a.part[(int64_t)blockIdx.x * LS_NSTAT + j] = stat[j];
    last = atom_add_acq_rel(a.ticket + 1, 1) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!last || warp >= LS_NSTAT) return;
  double v = 0.;
  for (int64_t i = lane; i < gridDim.x; i += 32) v += __ldcg(a.part + i * LS_NSTAT + warp);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
  if (lane == 0) a.stats[warp] = (float)v;
  if (tid == 0) a.ticket[1] = 0;
}

// ---- answer pairs -------------------------------------------------------------------------

// log ratio of request r: sum over its counted tokens of l - ref.  Whole warp.
__device__ __forceinline__ double pair_ratio(const LossArgs& a, int64_t r, int lane) {
  const int64_t lo = a.offsets[r], hi = a.offsets[r + 1];
  double s = 0.;
  if (__ldcg(a.count + r) > 0)
    for (int64_t t = lo + lane; t < hi; t += 32)
      if (!a.mask || a.mask[t] != 0) s += (double)__ldcg(&a.state[t].z);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(FULL, s, o);
  return s;
}

// One warp per pair; the last CTA sums the statistics.
static __global__ void __launch_bounds__(256) loss_pairs(const LossArgs a) {
  __shared__ int last;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t i = (int64_t)blockIdx.x * 8 + warp, n_pairs = a.n_req / 2;
  if (i < n_pairs) {
    double sw = pair_ratio(a, 2 * i, lane), sl = pair_ratio(a, 2 * i + 1, lane);
    const int32_t nw = __ldcg(a.count + 2 * i), nl = __ldcg(a.count + 2 * i + 1);
    if (a.length_norm) {
      sw /= (double)max(nw, 1);
      sl /= (double)max(nl, 1);
    }
    if (lane == 0) {
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
          f = (1.f - a.smooth) * (e + fmaxf(-h, 0.f)) + a.smooth * (e + fmaxf(h, 0.f));
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
        const double share = (double)slope / (double)__ldcg(a.totals + 1);
        cw = (float)(a.length_norm ? share / (double)nw : share);
        cl = (float)(a.length_norm ? -share / (double)nl : -share);
      }
      a.coef[2 * i] = cw;
      a.coef[2 * i + 1] = cl;
      for (int j = 0; j < LS_NSTAT; ++j) a.term[i * LS_NSTAT + j] = t[j];
    }
  }
  __syncthreads();
  if (tid == 0) {
    __threadfence();
    last = atom_add_acq_rel(a.ticket + 1, 1) == (int)gridDim.x - 1;
  }
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
