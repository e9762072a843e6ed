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
  int32_t* row_req;    // [n_rows] request of a row that counts, else -1
  float* coef;         // [n_req] dL / d log ratio (preference)
  float* term;         // [n_req / 2][LS_NSTAT] the pairs' statistics
  float4* state;       // [n_rows] M, log2 S, l - ref (preference) or dL/dx's factor, 1 - p_y
  double* part;        // [groups][LS_NSTAT] statistics of each group's rows
  uint32_t* ctx_flags;
};

// ---- counted tokens -------------------------------------------------------------------

// The first n_req CTAs count a request's tokens each, the last of them to finish sums
// up; the others find the requests of 256 rows each.
static __global__ void __launch_bounds__(256) loss_plan(const LossArgs a, int pairs) {
  __shared__ int64_t part[8];
  __shared__ int last;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if ((int64_t)blockIdx.x >= a.n_req) {
    const int64_t t = ((int64_t)blockIdx.x - a.n_req) * 256 + tid;
    if (t >= a.n_rows) return;
    int32_t r = -1;
    if (!a.mask || a.mask[t] != 0) {
      r = 0;
      if (a.offsets) {
        int32_t hi = a.n_req - 1;  // the largest r with offsets[r] <= t
        while (r < hi) {
          const int32_t mid = (int32_t)(((int64_t)r + hi + 1) >> 1);
          if (a.offsets[mid] <= t) r = mid;
          else hi = mid - 1;
        }
        const int64_t lo = a.offsets[r], up = a.offsets[r + 1];
        if (lo < 0 || up > a.n_rows || t < lo || t >= up) r = -1;
      }
    }
    a.row_req[t] = r;
    return;
  }
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
    last = atom_add_acq_rel(a.ticket, 1) == a.n_req - 1;
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

// ---- forward: rows through rings of shared memory ---------------------------------------
//
// A group of warps takes a row: 1, 4 or the 16 warps of a CTA, or 16 of each CTA of a
// cluster.  Warp w of the group takes every w-th chunk of 2 KB of (its CTA's share of)
// the row, brings it into a ring of its own with one bulk copy, and runs ahead over its
// next rows as far as the ring has room: nothing but the row's two sums is ever
// waited for together.  With HOLD a row's chunks stay in the ring for the backward
// sweep, so that its logits are read from memory once; a stage is free, and the next
// row's chunk on its way into it, as soon as its part of the gradient is written.
// What does not fit (or has to wait for other rows: answer pairs) leaves the row's
// state to loss_backward.
constexpr int RG_NW = 16;
constexpr int RG_W = 4;                        // words per lane and chunk
constexpr int RG_CHUNK = 32 * RG_W;            // words of a chunk
constexpr int RG_BYTES = 16 * RG_CHUNK;
constexpr int RG_NS = 7;                       // stages per warp
struct RingSmem {
  unsigned char stage[RG_NW][RG_NS][RG_BYTES];
  uint64_t bar[RG_NW][RG_NS];
  float2 part[2][RG_NW * MAXC];                // the warps' (m, R), two rows deep
};
static_assert(sizeof(RingSmem) <= 232448, "227 KB");

// a group's share of a row: its words, those of this CTA, and this warp's chunks of those
struct Share {
  const char* x;       // the row
  RowWords rw;
  int32_t w0, w1;      // this CTA's words [w0, w1)
  int32_t chunks;      // this warp's chunks
};
template <typename T, int GW>
__device__ __forceinline__ Share share_of(const LossArgs& a, int64_t row, uint32_t C, uint32_t rank,
                                          int wg) {
  Share s;
  const T* x = reinterpret_cast<const T*>(a.logits) + row * a.row_stride;
  s.x = reinterpret_cast<const char*>(x);
  s.rw = RowWords::of(x, a.vocab);
  const int32_t words = (int32_t)s.rw.words;
  const int32_t all = (words + RG_CHUNK - 1) / RG_CHUNK;
  const int32_t per = GW < RG_NW ? all : (all + (int32_t)C - 1) / (int32_t)C;  // chunks of a CTA
  s.w0 = min(words, (int32_t)rank * per * RG_CHUNK);
  s.w1 = min(words, s.w0 + per * RG_CHUNK);
  const int32_t mine = (s.w1 - s.w0 + RG_CHUNK - 1) / RG_CHUNK;
  s.chunks = mine > wg ? (mine - wg + GW - 1) / GW : 0;
  return s;
}

// what a row's epilogue needs, fetched while the rows before it are in work
struct RowIn {
  int32_t r, y, count;
  float xy, old, ref, adv;
};

template <typename T, int GW, bool HOLD, bool PREF>
__global__ void __launch_bounds__(RG_NW * 32, 1) loss_ring(const LossArgs a) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  RingSmem& sm = *reinterpret_cast<RingSmem*>(smem_raw);
  using Tr = Traits<T>;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int wg = warp % GW;
  uint32_t C = 1, rank = 0;
  if (GW == RG_NW) {
    asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(C));
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  }
  const int64_t G = GW == RG_NW ? gridDim.x / C : (int64_t)gridDim.x * (RG_NW / GW);
  const int64_t first = GW == RG_NW ? blockIdx.x / C : (int64_t)blockIdx.x * (RG_NW / GW) + warp / GW;
  const bool leader = wg == 0 && rank == 0;
  auto bar_of = [&](int s) { return (uint32_t)__cvta_generic_to_shared(&sm.bar[warp][s]); };
  if (lane == 0) {
    for (int s = 0; s < RG_NS; ++s)
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar_of(s)) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncwarp();
  if (GW == RG_NW && C > 1) cluster_sync_all();  // every CTA's memory is there
  pdl_wait();
  pdl_trigger();

  // ---- bringing chunks in
  int64_t lrow = first;            // the next chunk's row, its request and the next row's
  int32_t lreq = lrow < a.n_rows ? __ldcg(a.row_req + lrow) : -1;
  int32_t lreq2 = lrow + G < a.n_rows ? __ldcg(a.row_req + lrow + G) : -1;
  int32_t lchunk = 0;
  int lstage = 0, room = RG_NS, flying = 0;
  bool landed = true;
  uint32_t parity = 0u;            // bit s: stage s' next phase
  Share ls;
  ls.chunks = 0;
  if (lrow < a.n_rows) ls = share_of<T, GW>(a, lrow, C, rank, wg);
  auto bring = [&]() {
    // rows that do not count, or of which this warp has nothing
    while (lrow < a.n_rows && (lreq < 0 || lchunk >= ls.chunks)) {
      lrow += G;
      lreq = lreq2;
      lreq2 = lrow + G < a.n_rows ? __ldcg(a.row_req + lrow + G) : -1;
      lchunk = 0;
      if (lrow < a.n_rows) ls = share_of<T, GW>(a, lrow, C, rank, wg);
    }
    if (lrow >= a.n_rows || room == 0 || !landed) return;
    if (lane == 0) {
      const int32_t w = ls.w0 + (wg + lchunk * GW) * RG_CHUNK;
      const uint32_t bytes = 16u * (uint32_t)min(RG_CHUNK, ls.w1 - w);
      const uint32_t bar = bar_of(lstage);
      asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes)
                   : "memory");
      asm volatile(
          "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::
              "r"((uint32_t)__cvta_generic_to_shared(sm.stage[warp][lstage])),
          "l"(ls.x + (int64_t)sizeof(T) * ls.rw.head + 16 * (int64_t)w), "r"(bytes), "r"(bar)
          : "memory");
    }
    lstage = lstage + 1 == RG_NS ? 0 : lstage + 1;
    --room;
    ++flying;
    ++lchunk;
  };
  for (int s = 0; s < RG_NS; ++s) bring();

  // ---- the rows' scalars, two rows ahead and one
  auto fetch_id = [&](int64_t row, int32_t& r, int32_t& y) {
    r = -1;
    y = 0;
    if (row < a.n_rows) {
      r = __ldcg(a.row_req + row);
      y = __ldcg(a.chosen + row);
    }
  };
  auto fetch = [&](int64_t row, int32_t r, int32_t y) {
    RowIn in;
    in.r = r;
    in.y = y;
    in.count = 1;
    in.xy = NAN;
    in.old = in.ref = in.adv = 0.f;
    if (r >= 0) {
      const T* x = reinterpret_cast<const T*>(a.logits) + row * a.row_stride;
      if (y >= 0 && (int64_t)y < a.vocab) in.xy = Tr::elem(x, y);
      if (a.ref_logp) in.ref = __ldcg(a.ref_logp + row);
      if (!PREF) {
        if (a.old_logp) in.old = __ldcg(a.old_logp + row);
        in.adv = __ldcg(a.adv + (a.per_request ? (int64_t)r : row));
        if (a.norm) in.count = __ldcg(a.count + r);
      }
    }
    return in;
  };
  int32_t r1, y1;
  fetch_id(first, r1, y1);
  RowIn in = fetch(first, r1, y1);
  fetch_id(first + G, r1, y1);
  const double share = PREF ? 0.0 : 1.0 / (double)__ldcg(a.totals + (a.norm ? 1 : 0));
  double stat[LS_NSTAT] = {0., 0., 0., 0., 0., 0.};

  int stage = 0, buf = 0;
  for (int64_t row = first; row < a.n_rows; row += G) {
    const RowIn next = row + G < a.n_rows ? fetch(row + G, r1, y1) : in;
    fetch_id(row + 2 * G, r1, y1);
    const Share sh = share_of<T, GW>(a, row, C, rank, wg);
    const T* x = reinterpret_cast<const T*>(sh.x);
    T* g = reinterpret_cast<T*>(a.grad) + row * a.grad_stride;
    const int64_t tail0 = sh.rw.head + sh.rw.words * Tr::VEC;
    // element of this lane before or after the words
    const int64_t ve = lane < 8 ? (lane < sh.rw.head ? lane : -1)
                                : (lane - 8 < sh.rw.tail ? tail0 + lane - 8 : -1);
    const bool edge = leader && ve >= 0;
    if (in.r < 0) {
      if (leader && lane == 0) a.logp[row] = 0.f;
      if (HOLD) {
        const bool vec = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(g)) & 15u) == 0;
        for (int32_t c = 0; c < sh.chunks; ++c) {
          const int32_t w = sh.w0 + (wg + c * GW) * RG_CHUNK;
#pragma unroll
          for (int k = 0; k < RG_W; ++k) {
            const int32_t i = w + 32 * k + lane;
            if (i < sh.w1) put_word(g + sh.rw.head + (int64_t)i * Tr::VEC, make_uint4(0u, 0u, 0u, 0u), vec);
          }
        }
        if (edge) put(g + ve, 0.f);
      }
      in = next;
      continue;
    }
    const int32_t y = in.y;
    const bool yok = y >= 0 && (int64_t)y < a.vocab;
    const int64_t yo = (int64_t)y - sh.rw.head;
    const int32_t yw = yok && yo >= 0 ? (int32_t)(yo / Tr::VEC) : -1;
    const int yj = (int)(yo - (int64_t)yw * Tr::VEC);

    // ---- forward
    RowSum s;
    s.reset();
    const int held = stage;
    for (int32_t c = 0; c < sh.chunks; ++c) {
      if (landed) {
        if (!ring_test(bar_of(stage), (parity >> stage) & 1u))
          landed = ring_wait_slow(bar_of(stage), (parity >> stage) & 1u, a.ctx_flags);
        if (landed) {
          parity ^= 1u << stage;
          --flying;
        }
      }
      __syncwarp();
      const uint4* st = reinterpret_cast<const uint4*>(sm.stage[warp][stage]) + lane;
      const int32_t w = sh.w0 + (wg + c * GW) * RG_CHUNK;
      uint4 v[RG_W];
#pragma unroll
      for (int k = 0; k < RG_W; ++k) v[k] = st[32 * k];
      if (w + RG_CHUNK > sh.w1) {
#pragma unroll
        for (int k = 0; k < RG_W; ++k)
          if (w + 32 * k + lane >= sh.w1)
            v[k] = make_uint4(Tr::NEG_WORD, Tr::NEG_WORD, Tr::NEG_WORD, Tr::NEG_WORD);
      }
      if (yw >= w && yw < w + RG_CHUNK) {
#pragma unroll
        for (int k = 0; k < RG_W; ++k)
          if (w + 32 * k + lane == yw) v[k] = without<T>(v[k], yj);
      }
      const float top = Tr::tile_max(v);
      if (__any_sync(FULL, (top - s.m) * a.c2 > 8.f)) s.raise(top, a.c2, a.inv_t);
#pragma unroll
      for (int k = 0; k < RG_W; ++k) add_word<T>(s, v[k], a.c2);
      stage = stage + 1 == RG_NS ? 0 : stage + 1;
      if (!HOLD) {
        __syncwarp();
        ++room;
        bring();
      }
    }
    const float xe = edge ? Tr::elem(x, ve) : 0.f;
    if (edge && ve != y) s.add1(xe, a.c2, a.inv_t);
    // the warp's, then the group's sums
    float R = s.S.x + s.S.y;
    float m = unord(__reduce_max_sync(FULL, ord(s.m)));
    R *= rescale(s.m, m, a.inv_t);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) R += __shfl_xor_sync(FULL, R, o);
    if (GW > 1) {
      const float2 mine = make_float2(m, R);
      int n = GW;
      if (GW == RG_NW && C > 1) {
        n = RG_NW * (int)C;
        if (lane < (int)C)
          dsmem_st_u64(dsmem_addr(&sm.part[buf][rank * RG_NW + warp], (uint32_t)lane),
                       (uint64_t)__float_as_uint(m) | (uint64_t)__float_as_uint(R) << 32);
        __syncwarp();
        cluster_sync_all();
      } else {
        if (lane == 0) sm.part[buf][warp] = mine;
        if (GW == RG_NW) __syncthreads();
        else named_bar_sync(1 + warp / GW, 32 * GW);
      }
      const float2* pt = sm.part[buf] + (GW == RG_NW ? 0 : warp - wg);
      float2 q[MAXC * RG_NW / 32];
      m = LS_MIN;
#pragma unroll
      for (int k = 0; k < MAXC * RG_NW / 32; ++k) {
        q[k] = lane + 32 * k < n ? pt[lane + 32 * k] : make_float2(LS_MIN, 0.f);
        m = fmaxf(m, q[k].x);
      }
      m = unord(__reduce_max_sync(FULL, ord(m)));
      R = 0.f;
#pragma unroll
      for (int k = 0; k < MAXC * RG_NW / 32; ++k)
        if (32 * k < n) R = fmaf(q[k].y, rescale(q[k].x, m, a.inv_t), R);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) R += __shfl_xor_sync(FULL, R, o);
      buf ^= 1;
    }
    const RowEnd e(a, m, R, in.xy, yok);
    float k = 0.f;
    if (!PREF) {
      const double wt = a.norm ? share / (double)in.count : share;
      const PolicyTerms p = policy_terms(a, e.l, e.l_lo, in.old, in.ref, in.adv);
      k = (float)wt * p.slope * (a.grad_scale * a.inv_t);
      if (leader && lane == 0) {
        stat[0] += wt * (double)p.loss;
        stat[1] += wt * (double)p.surrogate;
        stat[2] += wt * (double)p.kl;
        stat[3] += wt * (double)p.ratio;
        stat[4] += wt * (double)p.clipped;
        stat[5] += wt * (double)p.old_kl;
      }
    }
    if (leader && lane == 0) {
      a.logp[row] = e.l;
      if (!yok) atomicOr(a.ctx_flags, FLAG_BAD_CHOSEN);
      else if (isnan(e.l)) atomicOr(a.ctx_flags, FLAG_NONFINITE);
      if (!HOLD && a.state) {
        a.state[row] = make_float4(e.M, e.lS, PREF ? (e.l - in.ref) + e.l_lo : k, e.rest);
      }
    }

    // ---- backward
    if (HOLD) {
      const bool vec = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(g)) & 15u) == 0;
      const RowGrad rg{e.M, e.lS, -k, a.c2};
      const float gy = k * e.rest;
      int bs = held;
      for (int32_t c = 0; c < sh.chunks; ++c) {
        const uint4* st = reinterpret_cast<const uint4*>(sm.stage[warp][bs]) + lane;
        const int32_t w = sh.w0 + (wg + c * GW) * RG_CHUNK;
#pragma unroll
        for (int q = 0; q < RG_W; ++q) {
          const int32_t i = w + 32 * q + lane;
          if (i < sh.w1) {
            T* to = g + sh.rw.head + (int64_t)i * Tr::VEC;
            put_word(to, grad_word<T>(rg, st[32 * q]), vec);
            if (i == yw) put(to + yj, gy);
          }
        }
        __syncwarp();
        bs = bs + 1 == RG_NS ? 0 : bs + 1;
        ++room;
        bring();
      }
      if (edge) put(g + ve, ve == y ? gy : rg.one(xe));
    }
    in = next;
  }
  if (!landed) {  // a wait ran out: no copy may be in flight when the CTA ends
    for (int i = 0; i < flying; ++i) {
      lstage = lstage == 0 ? RG_NS - 1 : lstage - 1;
      ring_wait_slow(bar_of(lstage), (parity >> lstage) & 1u, a.ctx_flags);
    }
  }
  if (PREF || !leader || first >= a.n_rows) return;
  // the statistics: each group's sum over its rows, then the groups' in order
  int last = 0;
  if (lane == 0) {
    for (int j = 0; j < LS_NSTAT; ++j) a.part[first * LS_NSTAT + j] = stat[j];
    last = atom_add_acq_rel(a.ticket + 1, 1) == (int)min(G, a.n_rows) - 1;
  }
  if (!__shfl_sync(FULL, last, 0)) return;
  const int64_t groups = min(G, a.n_rows);
  for (int j = 0; j < LS_NSTAT; ++j) {
    double v = 0.;
    for (int64_t i = lane; i < groups; i += 32) v += __ldcg(a.part + i * LS_NSTAT + j);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
    if (lane == 0) a.stats[j] = (float)v;
  }
  if (lane == 0) a.ticket[1] = 0;
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
  float k = 0.f;
  float4 st = make_float4(0.f, 0.f, 0.f, 0.f);
  int32_t y = -1;
  if (r >= 0) {
    st = __ldcg(a.state + row);
    k = PREF ? __ldcg(a.coef + r) * (a.grad_scale * a.inv_t) : st.z;
    y = __ldcg(a.chosen + row);
  }
  const bool zero = r < 0 || k == 0.f;
  const RowGrad rg{st.x, st.y, -k, a.c2};
  const float gy = k * st.w;
  const int64_t yo = (int64_t)y - rw.head;
  const int32_t yw = y >= 0 && (int64_t)y < a.vocab && yo >= 0 ? (int32_t)(yo / Tr::VEC) : -1;
#pragma unroll
  for (int q = 0; q < BW_W; ++q) {
    const int32_t i = w0 + q * BW_NT;
    if (i < words) {
      T* to = g + rw.head + (int64_t)i * Tr::VEC;
      put_word(to, zero ? make_uint4(0u, 0u, 0u, 0u) : grad_word<T>(rg, v[q]), vec);
      if (!zero && i == yw) put(to + (yo - (int64_t)yw * Tr::VEC), gy);
    }
  }
  if (seg > 0) return;
  const int64_t ve = tid < 8 ? (tid < rw.head ? tid : -1)
                             : (tid - 8 < rw.tail ? rw.head + rw.words * Tr::VEC + tid - 8 : -1);
  if (ve >= 0) put(g + ve, zero ? 0.f : (ve == y ? gy : rg.one(Tr::elem(x, ve))));
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
