// Distillation from a large model's first logits: a row's loss against its list of tokens
// S and their log-probabilities, with the gradient of the logits.
//
// With z = x / T, l = z - log sum exp(z), q = exp(l) and sigma the mass of q outside S, a
// row's loss depends on its logits through l over S, log sigma and the label's l_y alone.
// With a_v = d loss / d l_v, b = d loss / d log sigma and A = sum a + b
//   g_v = a_v - A q_v              v in S (a_y less the label's coefficient)
//   g_v = q_v / sigma (b - A sigma)   elsewhere (less that coefficient at y)
// so a row needs one sum R = sum over v outside S and not y of 2^(c x_v - k), c = log2(e) / T
// (k a reference that the sum itself raises), some sixty values more, and one sweep
// g_v = n 2^(c x_v - k) with n = (b - A sigma) / (T R), which neither a small sigma
// nor a small q makes lose anything.  The list's own entries and the label's are then written over
// that.  S stays out of the sum, as a rest of 1e-6 has no digits in 1 - sum_S q; for
// the same reason rho = 1 - sum_S p is summed in fp64 (a list is short).
#pragma once

#include "pr_loss.cuh"

namespace prk {

constexpr int DS_MAX = 64;          // longest list: two entries per lane
constexpr int DS_TERMS = 4;         // statistics that are summed row by row
constexpr float DS_RHO = 5.9604645e-8f;  // 2^-24

struct DistillArgs {
  LossArgs a;                       // a.chosen: the labels or NULL; a.logp: the rows' KL
  const int32_t* ids;
  const float* t_logp;
  int32_t k;
  int32_t reverse, none;            // direction; no class of the rest
  float kl_coef, ce_coef;
  float big;                        // logits from here on are infinite: 1e9 T
};

// a row's list and scalars: entries lane and 32 + lane, absent ones with id -1
struct ListIn {
  int32_t id[2];
  float t[2], x[2];
  int32_t y, count;
  float xy, edge;
};
// What a row's gradient needs.
struct ListOut {
  RowOut o;                         // o.gy: the label's entry, where it is not listed
  float g[DS_MAX];
};

template <typename T>
__device__ __forceinline__ ListIn fetch_list(const DistillArgs& d, const Rows& rows, const Share& s,
                                             const int4& ref, int lane) {
  const LossArgs& a = d.a;
  const int64_t row = ref.x;
  const T* x = reinterpret_cast<const T*>(s.x);
  ListIn in;
  in.y = ref.z;
  in.count = 1;
  in.xy = -INFINITY;
  in.edge = 0.f;
  in.id[0] = in.id[1] = -1;
  in.t[0] = in.t[1] = in.x[0] = in.x[1] = -INFINITY;
  if (ref.y < 0) return in;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int j = 32 * h + lane;
    if (j < d.k) {
      in.id[h] = __ldcg(d.ids + row * d.k + j);
      in.t[h] = __ldcg(d.t_logp + row * d.k + j);
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (in.t[h] == -INFINITY) in.id[h] = -1;
    if (in.id[h] >= 0 && (int64_t)in.id[h] < a.vocab) in.x[h] = Traits<T>::elem(x, in.id[h]);
  }
  if (a.chosen && in.y >= 0 && (int64_t)in.y < a.vocab) in.xy = Traits<T>::elem(x, in.y);
  if (a.norm) in.count = rows.count(a, ref.y);
  const int32_t v = end_of(a, s, lane);
  if (v >= 0) in.edge = Traits<T>::elem(x, v);
  return in;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
  return v;
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
  return v;
}
__device__ __forceinline__ float warp_max(float v) { return unord(__reduce_max_sync(FULL, ord(v))); }

// whether an id is listed twice.  Whole warp.
__device__ __forceinline__ bool listed_twice(const ListIn& in, int lane) {
  bool twice = false;
  const unsigned at = 1u << lane;
  const unsigned m0 = __match_any_sync(FULL, in.id[0]), m1 = __match_any_sync(FULL, in.id[1]);
  twice = (in.id[0] >= 0 && m0 != at) || (in.id[1] >= 0 && m1 != at);
  if (__any_sync(FULL, in.id[1] >= 0))
    for (int o = 0; o < 32; ++o) {
      const int32_t other = __shfl_xor_sync(FULL, in.id[1], o);  // (by every lane)
      twice |= in.id[0] >= 0 && in.id[0] == other;
    }
  return __any_sync(FULL, twice);
}

// A row's end: its sum R against 2^k, the list's and label's logits left out.  Writes the row's
// KL, the statistics' terms (weight wt) and the result.  Whole warp.
__device__ __noinline__ void list_math(const DistillArgs& d, int64_t row, const ListIn in, float k,
                                       float R, float wt, bool writes, ListOut* out, float2* stat,
                                       int lane) {
  const LossArgs& a = d.a;
  const float big = d.big * a.c2;
  bool on[2];
  float x[2];
  bool bad_id = a.chosen && !(in.y >= 0 && (int64_t)in.y < a.vocab), bad = false;
  bool labelled = false;  // the label is listed
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    on[h] = in.id[h] != -1;
    x[h] = in.x[h] <= -d.big ? -INFINITY : in.x[h];
    bad_id |= on[h] && (in.id[h] < 0 || (int64_t)in.id[h] >= a.vocab);
    bad |= on[h] && (!(in.t[h] < INFINITY) || !(x[h] < d.big));
    labelled |= on[h] && in.id[h] == in.y;
  }
  bad_id = __any_sync(FULL, bad_id) || listed_twice(in, lane);
  labelled = __any_sync(FULL, labelled);
  const bool apart = a.chosen && !labelled;
  const float xy = in.xy <= -d.big ? -INFINITY : in.xy;
  bad |= !(k < big) || !(R >= 0.f) || !(R < INFINITY) || (a.chosen && !(xy < d.big));
  bad = __any_sync(FULL, bad);
  if (!(k > -big)) R = 0.f;
  // the rest with the label's term, against 2^k: R; without it R0
  float R0 = R, ey = 0.f;
  if (apart && xy > -INFINITY) {
    const float top = R > 0.f ? fmaxf(k, xy * a.c2) : xy * a.c2;
    R0 = R > 0.f ? R * exp2f(k - top) : 0.f;
    ey = exp2f(fmaf(xy, a.c2, -top));
    R = R0 + ey;
    k = top;
  }
  const bool rest = R > 0.f;
  // everything against K, the largest exponent
  const float K = fmaxf(warp_max(fmaxf(on[0] ? x[0] * a.c2 : -INFINITY,
                                       on[1] ? x[1] * a.c2 : -INFINITY)),
                        rest ? k : -INFINITY);
  if (!(K > -INFINITY)) bad = true;
  float u[2], e[2], l[2], q[2], p[2], lt[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    u[h] = on[h] ? fmaf(x[h], a.c2, -K) : -INFINITY;
    e[h] = exp2f(u[h]);
  }
  const float f = rest ? exp2f(k - K) : 0.f, Rk = R * f, eyk = ey * f;
  // the largest listed term stays out of the sum of the others: 1 - q of it is others / S
  const float m = warp_max(fmaxf(e[0], e[1]));
  const unsigned w0 = __ballot_sync(FULL, on[0] && e[0] == m), w1 = __ballot_sync(FULL, on[1] && e[1] == m);
  const int first = w0 ? __ffs(w0) - 1 : w1 ? 32 + __ffs(w1) - 1 : -1;  // its place
  const bool is[2] = {first == lane, first == 32 + lane};
  const float listed = warp_sum((is[0] ? 0.f : e[0]) + (is[1] ? 0.f : e[1]));  // but the largest
  const float others = Rk + listed, S = first >= 0 ? others + m : Rk;
  const float L = log2f(S), inv = 1.f / S;
  const bool most = first >= 0 && m > 0.5f * S;
  const float compl1 = most ? others * inv : 0.f;  // 1 - q of the largest
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    l[h] = (u[h] - L) * LN2;
    if (most && is[h]) l[h] = -log1pf(others / m);
    q[h] = on[h] ? e[h] * inv : 0.f;
  }
  const float E = listed + (first >= 0 ? m : 0.f), sigma = Rk * inv;
  const float l_sigma = Rk > 0.5f * S ? -log1pf(E / Rk) : (k - K + log2f(R) - L) * LN2;
  // the large model's side
  const bool any = first >= 0 || __any_sync(FULL, on[0] || on[1]);
  const bool klass = !d.none && rest;
  float l_rho = 0.f, rho = 0.f, mass;
  if (d.none) {
    const float tm = warp_max(fmaxf(in.id[0] != -1 ? in.t[0] : -INFINITY, in.id[1] != -1 ? in.t[1] : -INFINITY));
#pragma unroll
    for (int h = 0; h < 2; ++h) p[h] = on[h] ? expf(in.t[h] - tm) : 0.f;
    const float P = warp_sum(p[0] + p[1]), lP = logf(P);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      lt[h] = (in.t[h] - tm) - lP;
      p[h] /= P;
    }
    mass = any ? expf(tm) * P : 0.f;
  } else {
    double s = 0.;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const double v = on[h] ? exp((double)in.t[h]) : 0.;
      p[h] = (float)v;
      lt[h] = in.t[h];
      s += v;
    }
    s = warp_sum(s);
    mass = (float)s;
    rho = fmaxf((float)(1. - s), DS_RHO);
    l_rho = logf(rho);
  }
  // KL, a and b
  float kl = 0.f, av[2] = {0.f, 0.f}, b = 0.f;
  if (any) {
    if (!d.reverse) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (on[h] && p[h] > 0.f) kl += p[h] * (lt[h] - l[h]);
        av[h] = -p[h];
      }
      kl = warp_sum(kl);
      if (klass) {
        kl += rho * (l_rho - l_sigma);
        b = -rho;
      }
    } else {
      if (d.none) {  // q over the list
        const float um = warp_max(fmaxf(u[0], u[1]));
        if (um == -INFINITY) bad = true;
        float qe[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) qe[h] = on[h] ? exp2f(u[h] - um) : 0.f;
        const float Q = warp_sum(qe[0] + qe[1]), lQ = logf(Q);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          l[h] = (u[h] - um) * LN2 - lQ;
          qe[h] /= Q;
          av[h] = qe[h];
        }
      } else {
        av[0] = q[0];
        av[1] = q[1];
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (av[h] > 0.f) kl += av[h] * (l[h] - lt[h]);
      kl = warp_sum(kl);
      const float far = l_sigma - l_rho;
      if (klass && sigma > 0.f) kl += sigma * far;
#pragma unroll
      for (int h = 0; h < 2; ++h) av[h] = av[h] > 0.f ? av[h] * (l[h] - lt[h] - kl) : 0.f;
      if (klass && sigma > 0.f) b = sigma * (far - kl);
    }
  }
  // the label
  float ce = 0.f;
  if (a.chosen) {
    if (apart) {
      const float not_y = R0 * f + E;
      ce = eyk > 0.25f * S ? log1pf(not_y / eyk) : -(fmaf(xy, a.c2, -K) - L) * LN2;
    } else {
      const float v = on[0] && in.id[0] == in.y ? l[0] : on[1] && in.id[1] == in.y ? l[1] : 0.f;
      // (reverse over the list alone has put other logarithms in l)
      const float w = d.reverse && d.none
                          ? (on[0] && in.id[0] == in.y ? (most && is[0] ? -log1pf(others / m) : (u[0] - L) * LN2)
                             : on[1] && in.id[1] == in.y ? (most && is[1] ? -log1pf(others / m) : (u[1] - L) * LN2)
                                                         : 0.f)
                          : v;
      const unsigned who = __ballot_sync(FULL, (on[0] && in.id[0] == in.y) || (on[1] && in.id[1] == in.y));
      ce = -__shfl_sync(FULL, w, (who ? __ffs(who) - 1 : 0));
    }
  }
  bad |= bad_id;
  // the gradient
  const float kc = d.kl_coef, cc = a.chosen ? d.ce_coef : 0.f;
  const float w = wt * (a.grad_scale * a.inv_t);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    av[h] = kc != 0.f ? kc * av[h] : 0.f;
    if (on[h] && !apart && in.id[h] == in.y) av[h] -= cc;
  }
  b = kc != 0.f ? kc * b : 0.f;
  const float lesser = warp_sum((is[0] ? 0.f : av[0]) + (is[1] ? 0.f : av[1]));
  const float a1 = warp_sum((is[0] ? av[0] : 0.f) + (is[1] ? av[1] : 0.f));
  // A without the rounding of sums that are 0 by their form: reverse has sum a + b = 0
  const float kA = d.reverse || !any ? 0.f : kc * (klass ? -(warp_sum(p[0] + p[1]) + rho) : -warp_sum(p[0] + p[1]));
  const float A = kA - cc;
  (void)a1;
  if (out) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float g = av[h] - A * q[h];
      // a - A q = (a - A) + A (1 - q), with a - A = -(the other a and b)
      if (most && is[h]) g = fmaf(A, compl1, -(lesser + b - (apart ? cc : 0.f)));
      out->g[32 * h + lane] = bad ? NAN : w * g;
    }
    if (lane == 0) {
      RowOut o;
      const float D = b - A * sigma;
      o.K = k;
      o.M = 0.f;
      o.nk = bad ? NAN : rest ? w * D / R : 0.f;
      o.mode = o.nk == 0.f ? ROW_ZERO : ROW_FAST;
      // q_y (b / sigma - kA) - ce (1 - q_y)
      const float share = rest ? ey / R : 0.f;
      o.gy = bad ? NAN : w * (share * (b - kA * sigma) - cc * ((R0 * f + E) * inv));
      out->o = o;
    }
  }
  if (bad) kl = ce = mass = NAN;
  if (lane < DS_TERMS) {
    const float covered = bad ? NAN : E * inv;
    const float t = wt * (lane == 0 ? kl : lane == 1 ? ce : lane == 2 ? mass : covered);
    const float2 s = stat[lane];
    const float y = s.x + t, z = y - s.x;
    stat[lane] = make_float2(y, s.y + ((s.x - (y - z)) + (t - z)));
  }
  if (lane == 0 && writes) {
    a.logp[row] = kl;
    if (bad) atomicOr(a.ctx_flags, bad_id ? FLAG_BAD_CHOSEN : FLAG_NONFINITE);
  }
}

// The statistics, as write_stats' of the other losses.  Whole warp.
__device__ __forceinline__ void list_stats(const DistillArgs& d, const float2* stat, int warps,
                                           int64_t at, int64_t count, int lane) {
  const LossArgs& a = d.a;
  int last = 0;
  if (lane < DS_TERMS) {
    double v = 0.;
    for (int w = 0; w < warps; ++w) {  // (an infinite sum's compensation is NaN)
      const float2 q = stat[w * DS_TERMS + lane];
      v += isinf(q.x) ? (double)q.x : (double)q.x + (double)q.y;
    }
    a.part[at * DS_TERMS + lane] = v;
  }
  __syncwarp();
  if (lane == 0) {
    __threadfence();
    last = atom_add_acq_rel(a.ticket + 1, 1) == (int)count - 1;
  }
  if (!__shfl_sync(FULL, last, 0)) return;
  double total[DS_TERMS];
#pragma unroll
  for (int j = 0; j < DS_TERMS; ++j) {
    double v = 0.;
    for (int64_t i = lane; i < count; i += 32) v += __ldcg(a.part + i * DS_TERMS + j);
    total[j] = warp_sum(v);
  }
  if (lane == 0) {
    // (a term of coefficient 0 may be infinite)
    const double kl = d.kl_coef != 0.f ? (double)d.kl_coef * total[0] : 0.;
    const double ce = d.ce_coef != 0.f && a.chosen ? (double)d.ce_coef * total[1] : 0.;
    a.stats[0] = (float)(kl + ce);
    for (int j = 0; j < DS_TERMS; ++j) a.stats[1 + j] = (float)total[j];
    a.ticket[1] = 0;
  }
}

// ---- a CTA per row, which it reads twice -------------------------------------------------

constexpr int DL_NT = 256;
struct PlainSmem {
  float2 part[DL_NT / 32];
  float2 stat[DS_TERMS];
  ListOut out;
  int4 unused;
};

template <typename T>
__global__ void __launch_bounds__(DL_NT) distill_plain(const DistillArgs d) {
  extern __shared__ __align__(16) unsigned char ds_raw[];
  uint32_t* const listed = reinterpret_cast<uint32_t*>(ds_raw);  // a bit per token
  __shared__ PlainSmem sm;
  const LossArgs& a = d.a;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid < DS_TERMS) sm.stat[tid] = make_float2(0.f, 0.f);
  pdl_wait();
  pdl_trigger();
  const Rows rows{nullptr, (int32_t)__ldcg(a.totals)};
  const double share = rows.share(a);
  for (int64_t i = blockIdx.x; i < rows.live; i += gridDim.x) {
    const int4 ref = rows.at(a, i);
    const Share s = share_of<T>(a, ref.x, 1, 0);
    const T* x = reinterpret_cast<const T*>(s.x);
    __syncthreads();
    for (int q = tid; q < (int)((a.vocab + 31) / 32); q += DL_NT) listed[q] = 0u;
    __syncthreads();
    if (tid <= d.k) {
      const int32_t v = tid < d.k ? d.ids[(int64_t)ref.x * d.k + tid] : ref.z;
      const bool on = tid < d.k ? d.t_logp[(int64_t)ref.x * d.k + tid] != -INFINITY : true;
      if (on && v >= 0 && (int64_t)v < a.vocab) atomicOr(&listed[v >> 5], 1u << (v & 31));
    }
    __syncthreads();
    float k = -3e38f, S = 0.f;
    for (int64_t v = tid; v < a.vocab; v += DL_NT) {
      if (listed[v >> 5] >> (v & 31) & 1u) continue;
      const float f = Traits<T>::elem(x, v), t = f * a.c2;
      if (t > k) {
        S *= exp2f(k - t);
        k = t;
      }
      S += exp2f(fmaf(f, a.c2, -k));
    }
    float R;
    join(make_float2(k, S), 1.f, k, R);
    if (lane == 0) sm.part[warp] = make_float2(k, R);
    __syncthreads();
    if (warp == 0) {
      join(lane < DL_NT / 32 ? sm.part[lane] : make_float2(-3e38f, 0.f), 1.f, k, R);
      const ListIn in = fetch_list<T>(d, rows, s, ref, lane);
      const float wt = (float)(a.norm ? share / (double)in.count : share);
      list_math(d, ref.x, in, k, R, wt, true, &sm.out, sm.stat, lane);
    }
    __syncthreads();
    if (!a.grad) continue;
    const RowOut o = sm.out.o;
    T* const g = reinterpret_cast<T*>(a.grad) + (int64_t)ref.x * a.grad_stride;
    for (int64_t v = tid; v < a.vocab; v += DL_NT) {
      const bool l = listed[v >> 5] >> (v & 31) & 1u;
      const float f = Traits<T>::elem(x, v);
      if (!l) put(g + v, f <= -d.big && o.nk == o.nk ? 0.f : grad1(o, a.c2, f));
    }
    __syncthreads();
    if (tid < d.k) {
      const int32_t v = d.ids[(int64_t)ref.x * d.k + tid];
      const bool on = d.t_logp[(int64_t)ref.x * d.k + tid] != -INFINITY;
      if (on && v >= 0 && (int64_t)v < a.vocab) put(g + v, sm.out.g[tid]);
      else if (false) put(g, 0.f);
    }
    if (tid == 0 && ref.z >= 0 && (int64_t)ref.z < a.vocab) {
      bool in = false;
      for (int j = 0; j < d.k; ++j)
        in |= d.ids[(int64_t)ref.x * d.k + j] == ref.z && d.t_logp[(int64_t)ref.x * d.k + j] != -INFINITY;
      if (!in) put(g + ref.z, o.gy);
    }
  }
  if (a.grad)
    for (int64_t i = blockIdx.x; i < a.n_rows - rows.live; i += gridDim.x) {
      T* const g = reinterpret_cast<T*>(a.grad) + (int64_t)rows.skipped(a, i) * a.grad_stride;
      for (int64_t v = tid; v < a.vocab; v += DL_NT) put(g + v, 0.f);
    }
  __syncthreads();
  const int64_t groups = max((int64_t)1, min((int64_t)gridDim.x, (int64_t)rows.live));
  if (warp == 0 && blockIdx.x < groups) list_stats(d, sm.stat, 1, blockIdx.x, groups, lane);
}

}  // namespace prk
