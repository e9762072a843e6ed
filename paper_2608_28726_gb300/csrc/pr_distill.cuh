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
// the same reason rho = 1 - sum_S p is summed in two fp32 parts.
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
  // workspace: the listed rows' entries and what their ends need beside them (distill_lists)
  int4* entries;                    // [n_rows][k] {id, logit, p, log p}
  float4* scalars;                  // [n_rows][2]
};

// a row's list and scalars: entries lane and 32 + lane, absent ones with id -1
struct ListIn {
  int32_t id[2];
  float t[2];
  int32_t y, count;
  uint32_t x[2], xy, edge;  // logits as they came from memory: what widens them would wait for them
};
template <typename T>
__device__ __forceinline__ uint32_t raw_at(const void* row, int64_t v) {
  if constexpr (sizeof(T) == 2) return reinterpret_cast<const uint16_t*>(row)[v];
  else return reinterpret_cast<const uint32_t*>(row)[v];
}
template <typename T>
__device__ __forceinline__ float wide(uint32_t raw) {
  return __uint_as_float(sizeof(T) == 2 ? raw << 16 : raw);
}
template <typename T>
constexpr uint32_t DS_MASKED = sizeof(T) == 2 ? 0xff80u : 0xff800000u;  // -inf
// A listed row's entries and scalars; then, once those are there, its logits at them.  Two steps,
// as each waits for memory: a row's entries are fetched two rows ahead, its logits one.
__device__ __forceinline__ ListIn fetch_list(const DistillArgs& d, const Rows& rows,
                                             const int4& ref, int lane) {
  ListIn in;
  in.y = ref.z;
  in.count = 1;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int j = 32 * h + lane;
    const int64_t at = (int64_t)ref.x * d.k + j;
    const bool on = ref.y >= 0 && j < d.k;
    in.id[h] = on ? __ldcg(d.ids + at) : -1;
    in.t[h] = on ? __ldcg(d.t_logp + at) : -INFINITY;
  }
  if (d.a.norm && ref.y >= 0) in.count = rows.count(d.a, ref.y);
  return in;
}
template <typename T>
__device__ __forceinline__ void fetch_logits(const DistillArgs& d, const Share& s, const int4& ref,
                                             ListIn& in, int lane) {
  const LossArgs& a = d.a;
  in.xy = DS_MASKED<T>;
  in.edge = 0u;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (in.t[h] == -INFINITY) in.id[h] = -1;
    in.x[h] = DS_MASKED<T>;
    if (in.id[h] >= 0 && (int64_t)in.id[h] < a.vocab) in.x[h] = raw_at<T>(s.x, in.id[h]);
  }
  if (ref.y < 0) return;
  if (a.chosen && in.y >= 0 && (int64_t)in.y < a.vocab) in.xy = raw_at<T>(s.x, in.y);
  const int32_t v = end_of(a, s, lane);
  if (v >= 0) in.edge = raw_at<T>(s.x, v);
}

// A value as the sum of two fp32 numbers, for 1 - sum p.  (In fp64 the exponentials of a list and
// their sum are 3,400 cycles of the warp that takes the rows' ends: 1,500 rows of V = 262,144 fp32
// without a gradient and lists of 64 784 us for 588.)
struct Pair {
  float hi, lo;
};
__device__ __forceinline__ Pair operator+(const Pair& a, const Pair& b) {
  Pair r;
  r.hi = a.hi + b.hi;
  const float v = r.hi - a.hi;
  r.lo = (a.lo + b.lo) + ((a.hi - (r.hi - v)) + (b.hi - v));
  return r;
}
__device__ __forceinline__ Pair warp_sum(Pair v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Pair w;
    w.hi = __shfl_xor_sync(FULL, v.hi, o);
    w.lo = __shfl_xor_sync(FULL, v.lo, o);
    v = v + w;
  }
  return v;
}
// 2^(j / 16) in two parts
__constant__ float2 DS_ROOTS[16] = {
    {1.0f, 0.0f}, {1.0442737340927124f, 4.8334701574503924e-08f},
    {1.0905077457427979f, -1.3077539939843064e-08f}, {1.1387885808944702f, 5.386222312608879e-08f},
    {1.1892070770263672f, 3.797635272917432e-08f}, {1.2418577671051025f, 4.496838101886169e-08f},
    {1.2968395948410034f, -4.018999533172973e-08f}, {1.3542555570602417f, -1.0123349269974824e-08f},
    {1.4142135381698608f, 2.4203234971764687e-08f}, {1.4768261909484863f, -4.500898853621038e-08f},
    {1.5422108173370361f, 8.070904833346049e-09f}, {1.610490322113037f, 9.836217174097328e-09f},
    {1.6817928552627563f, -2.4755326677450284e-08f}, {1.7562521696090698f, -9.235770370707996e-09f},
    {1.8340080976486206f, -1.1239277952768134e-08f}, {1.9152065515518188f, 9.845328108326612e-09f}};
// exp(t) within 1e-12 of itself for t >= -62 (below that rounded once, which is under 1e-34):
// t log2(e) = n / 16 + z log2(e) with z in two parts and below ln 2 / 32, 2^(n / 16) from its table,
// exp(z) - 1 = z + z^2 / 2 + z^3 / 6 + ... whose first two terms are in two parts.  (rho down to
// 2^-24 is to keep five digits.)
__device__ __forceinline__ Pair exp_pair(float t) {
  constexpr float L2E_LOW = 1.925963033500011e-08f;  // log2(e) - L2E
  const float y = t * L2E, n = rintf(y * 16.f), r = fmaf(n, -0.0625f, y);
  const float y_lo = fmaf(t, L2E, -y) + t * L2E_LOW;
  const float z0 = r * LN2, z0_lo = fmaf(r, LN2, -z0) + (r * LN2_LOW + y_lo * LN2);
  const float z = z0 + z0_lo, z_lo = z0_lo - (z - z0);
  const float c = z * z * z * fmaf(z, fmaf(z, 1.f / 120.f, 1.f / 24.f), 1.f / 6.f);
  const float h = 0.5f * z, q = h * z, q_lo = fmaf(h, z, -q) + z * z_lo;
  const float w = z + q, w_lo = ((q - (w - z)) + q_lo) + (z_lo + c);
  const int whole = (int)fminf(fmaxf(n, -3200.f), 3200.f);
  const float2 root = DS_ROOTS[whole & 15];
  const float p = root.x * w, p_lo = fmaf(root.x, w, -p) + fmaf(root.x, w_lo, root.y * w);
  const float s = root.x + p, s_lo = (p - (s - root.x)) + (p_lo + root.y);
  const int e = whole >> 4;
  const float scale = e < -126 ? 0.f : exp2f((float)e);  // (a power of two: exact)
  const float all = s + s_lo;  // (its first part alone is a probability: rounded once)
  Pair v;
  v.hi = scale * all;
  v.lo = e < -90 ? 0.f : scale * (s_lo - (all - s));
  if (!(t < 1000.f)) v.hi = t;  // (what is no log-probability: NaN, infinity)
  return v;
}

// log2 of a sum in two parts, e + f
struct LogSum {
  float e, f;
  __device__ __forceinline__ explicit LogSum(float S) {
    int ei = (int)(__float_as_uint(S) >> 23) - 127;
    float m = __uint_as_float((__float_as_uint(S) & 0x7fffffu) | 0x3f800000u);
    if (m > 1.41f) {
      m *= 0.5f;
      ++ei;
    }
    e = (float)ei;
    f = log2f(m);
  }
};
// whether an id is listed twice.  Whole warp.
__device__ __forceinline__ bool listed_twice(const ListIn& in, int lane) {
  bool twice = false;
  const unsigned at = 1u << lane;
  const unsigned m0 = __match_any_sync(FULL, in.id[0]), m1 = __match_any_sync(FULL, in.id[1]);
  twice = (in.id[0] >= 0 && m0 != at) || (in.id[1] >= 0 && m1 != at);
  if (__any_sync(FULL, in.id[1] >= 0))
#pragma unroll 8
    for (int o = 0; o < 32; ++o) {
      const int32_t other = __shfl_xor_sync(FULL, in.id[1], o);  // (by every lane)
      twice |= in.id[0] >= 0 && in.id[0] == other;
    }
  return __any_sync(FULL, twice);
}

// The large model's side of a row, which does not wait for the row's sum.
struct ListPre {
  float p[2], lt[2];     // probabilities and their logarithms
  float sum;             // of p
  float rho, l_rho;      // without a class of the rest: two parts of what lt has too much
  float mass;
  bool bad, bad_id, labelled;
};
// Whole warp.
__device__ __forceinline__ void list_pre(const DistillArgs& d, const ListIn& in, ListPre& o,
                                         int lane) {
  const LossArgs& a = d.a;
  bool bad_id = a.chosen && !(in.y >= 0 && (int64_t)in.y < a.vocab), bad = false, labelled = false;
  bool on[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    on[h] = in.id[h] != -1;
    bad_id |= on[h] && (in.id[h] < 0 || (int64_t)in.id[h] >= a.vocab);
    bad |= on[h] && !(in.t[h] < INFINITY);
    labelled |= on[h] && in.id[h] == in.y;
  }
  const bool twice = listed_twice(in, lane);
  o.bad_id = __any_sync(FULL, bad_id) || twice;
  o.bad = __any_sync(FULL, bad);
  o.labelled = __any_sync(FULL, labelled);
  o.sum = o.rho = o.l_rho = o.mass = 0.f;
  if (d.none) {
    const float tm = warp_max(fmaxf(on[0] ? in.t[0] : -INFINITY, on[1] ? in.t[1] : -INFINITY));
#pragma unroll
    for (int h = 0; h < 2; ++h) o.p[h] = on[h] ? expf(in.t[h] - tm) : 0.f;
    const float P = warp_sum(o.p[0] + o.p[1]), inv = __fdividef(1.f, P);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      o.lt[h] = in.t[h] - tm;
      o.p[h] *= inv;
    }
    if (tm > -INFINITY) {
      const LogSum l(P);
      o.rho = l.e * LN2;
      o.l_rho = fmaf(l.e, LN2, -o.rho) + (l.e * LN2_LOW + l.f * LN2);
      o.sum = 1.f;
      o.mass = expf(tm) * P;
    }
  } else {
    Pair v[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      v[h] = on[h] ? exp_pair(in.t[h]) : Pair{0.f, 0.f};
      o.p[h] = v[h].hi;
      o.lt[h] = in.t[h];
    }
    const Pair s = warp_sum(v[0] + v[1]);
    o.sum = o.mass = s.hi;
    o.rho = fmaxf((1.f - s.hi) - s.lo, DS_RHO);
    o.l_rho = o.rho > 0.5f ? log1pf(-s.hi) : logf(o.rho);
  }
}

// The same for the i-th listed row, and its weight wt, as distill_lists left them.
__device__ __forceinline__ void fetch_prepared(const DistillArgs& d, int64_t i, const int4& ref,
                                               ListIn& in, ListPre& o, float& wt, int lane) {
  in.y = ref.z;
  in.edge = 0u;
  wt = 0.f;
  in.xy = 0u;
  o.sum = o.rho = o.l_rho = o.mass = 0.f;
  o.bad = o.bad_id = o.labelled = false;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int j = 32 * h + lane;
    int4 e = make_int4(-1, 0, 0, 0);
    if (ref.y >= 0 && j < d.k) e = __ldcg(d.entries + i * d.k + j);
    in.id[h] = e.x;
    in.x[h] = (uint32_t)e.y;
    o.p[h] = __int_as_float(e.z);
    o.lt[h] = __int_as_float(e.w);
  }
  if (ref.y < 0) return;
  const float4 q = __ldcg(d.scalars + 2 * i), r = __ldcg(d.scalars + 2 * i + 1);
  o.sum = q.x;
  o.rho = q.y;
  o.l_rho = q.z;
  o.mass = q.w;
  wt = r.x;
  in.xy = __float_as_uint(r.y);
  const uint32_t f = __float_as_uint(r.z);
  o.bad = f & 1u;
  o.bad_id = f & 2u;
  o.labelled = f & 4u;
}

// ln 2 (c x - K - log2 S) in two parts.  A divergence sums differences of logarithms that nearly
// cancel: what the roundings of c x - K (2^-24 of it) and of the logarithm would leave, 1e-6 of
// a KL of 0.1, has to stay.  (c is the one that the row's sum was taken with: an error of it
// is a temperature's, which hardly shows where both models agree.)
struct LogProb {
  float hi, lo;
  __device__ __forceinline__ LogProb(float x, float c2, float K, const LogSum& S) {
    const float h = x * c2;
    float u = h - K, u_lo = 0.f;
    if (h > -INFINITY) {
      const float t = u - h, left = ((h - (u - t)) + (-K - t)) + fmaf(x, c2, -h), all = u + left;
      u_lo = (u - all) + left;
      u = all;
    }
    const float w = u - S.e, t = w - u;
    const float w_lo = ((u - (w - t)) + (-S.e - t)) + u_lo - S.f;
    const float p = w * LN2, rest = fmaf(w, LN2, -p) + w * LN2_LOW + w_lo * LN2;
    hi = p + rest;
    lo = (p - hi) + rest;
    if (!(u > -INFINITY)) {  // a masked token
      hi = -INFINITY;
      lo = 0.f;
    }
  }
};

// (K, n) with n 2^(c x - K) = nR / R 2^(c x - k), for a sum of up to 1e33: nR / R by itself would
// be denormal, or 0, for small weights.  R = r 2^up, and K is k + up less what its rounding lost.
// (Apart, for sums above 1e9: with every row's here the batch takes 0.8 to 2% longer.)
__device__ __noinline__ float2 far_factor(float nR, float R, float k) {
  const float r = __uint_as_float((__float_as_uint(R) & 0x7fffffu) | 0x3f800000u);
  const float up = (float)((int)(__float_as_uint(R) >> 23) - 127), K = k + up;
  const float t = K - k, lost = (k - (K - t)) + (up - t);
  return make_float2(K, nR * __fdividef(exp2f(-lost), r));
}

// A row's end: its sum R against 2^k, the list's and label's logits left out.  Writes the result
// (out, and the list's entries of the gradient to g), whose barrier learns of it first, then the
// row's KL and the statistics' terms (weight wt).  Whole warp; apart from the kernel's registers.
template <typename T>
__device__ __forceinline__ void list_math(const DistillArgs& d, int64_t row, const ListIn& in,
                                          const ListPre& pre, float k, float R, float wt,
                                          bool writes, RowOut* out, float* g, uint64_t* out_bar,
                                          float2* stat, int lane) {
  const LossArgs& a = d.a;
  const float big = d.big * a.c2;
  bool on[2], bad = false;
  float x[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    on[h] = in.id[h] != -1;
    x[h] = wide<T>(in.x[h]);
    if (x[h] <= -d.big) x[h] = -INFINITY;
    bad |= on[h] && !(x[h] < d.big);
  }
  const bool apart = a.chosen && !pre.labelled;
  const float yx = wide<T>(in.xy), xy = yx <= -d.big ? -INFINITY : yx;
  bad |= pre.bad || !(k < big) || !(R >= 0.f) || !(R < INFINITY) || (a.chosen && !(xy < d.big));
  bad = __any_sync(FULL, bad);
  if (!(k > -big)) R = 0.f;
  // the rest with the label's term, against 2^k: R; without it R0
  float R0 = R, ey = 0.f;
  if (apart && xy > -INFINITY) {
    const float top = R > 0.f ? fmaxf(k, xy * a.c2) : xy * a.c2;
    R0 = R > 0.f ? R * ex2(k - top) : 0.f;
    ey = ex2(fmaf(xy, a.c2, -top));
    R = R0 + ey;
    k = top;
  }
  const bool rest = R > 0.f;
  // everything against K, the largest exponent
  const float K = fmaxf(warp_max(fmaxf(on[0] ? x[0] * a.c2 : -INFINITY,
                                       on[1] ? x[1] * a.c2 : -INFINITY)),
                        rest ? k : -INFINITY);
  if (!(K > -INFINITY)) bad = true;
  float u[2], e[2], q[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    u[h] = on[h] ? fmaf(x[h], a.c2, -K) : -INFINITY;
    e[h] = rescale2(u[h]);  // (as exact as a sum of few terms needs)
  }
  const float f = rest ? rescale2(k - K) : 0.f, Rk = R * f, eyk = ey * f;
  // the largest listed term stays out of the sum of the others: 1 - q of it is others / S
  const float m = warp_max(fmaxf(e[0], e[1]));
  const unsigned w0 = __ballot_sync(FULL, on[0] && e[0] == m);
  const unsigned w1 = __ballot_sync(FULL, on[1] && e[1] == m);
  const int first = w0 ? __ffs(w0) - 1 : w1 ? 32 + __ffs(w1) - 1 : -1;  // its place
  const bool any = first >= 0;
  const bool is[2] = {first == lane, first == 32 + lane};
  const float listed = warp_sum((is[0] ? 0.f : e[0]) + (is[1] ? 0.f : e[1]));
  const float others = Rk + listed, S = any ? others + m : Rk;
  const float inv = __fdividef(1.f, S);  // (S is at least about 1)
  const bool most = any && m > 0.5f * S;
  q[0] = on[0] ? e[0] * inv : 0.f;
  q[1] = on[1] ? e[1] * inv : 0.f;
  const float E = listed + (any ? m : 0.f), sigma = Rk * inv, not_y = R0 * f + E;
  const bool klass = !d.none && rest;
  float av[2] = {0.f, 0.f}, b = 0.f, a_all = 0.f, kA = 0.f;
  // the gradient, from a (av), its sum a_all, b, and A = a_all + b (kA).  b - A sigma is taken as
  // b (1 - sigma) - sigma sum a: sigma and rho near 1 differ by what the lists' masses do.
  auto result = [&]() {
    const float kc = d.kl_coef, cc = a.chosen ? d.ce_coef : 0.f;
    const float w = wt * (a.grad_scale * a.inv_t), A = (kc != 0.f ? kc * kA : 0.f) - cc;
    const float bc = kc != 0.f ? kc * b : 0.f;
    float ac[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      ac[h] = kc != 0.f ? kc * av[h] : 0.f;
      if (on[h] && in.id[h] == in.y && a.chosen) ac[h] -= cc;
    }
    const float lesser = warp_sum((is[0] ? 0.f : ac[0]) + (is[1] ? 0.f : ac[1]));
    const bool nan = bad || pre.bad_id;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      // a - A q = (a - A) + A (1 - q), with a - A = -(the other a and b)
      const float v = most && is[h] ? fmaf(A, others * inv, -(lesser + bc - (apart ? cc : 0.f)))
                                    : ac[h] - A * q[h];
      g[32 * h + lane] = nan ? NAN : w * v;
    }
    if (lane == 0) {
      RowOut o;
      o.M = 0.f;
      const float per_R = rest ? __fdividef(1.f, R) : 0.f;
      const float sum_a = kc != 0.f ? kc * a_all : 0.f, ba = bc * (E * inv);
      const float nR = nan ? NAN : w * (ba - (sum_a - cc) * sigma);
      o.K = k;
      o.nk = nR * per_R;
      if (R > 1e9f) {
        const float2 f = far_factor(nR, R, k);
        o.K = f.x;
        o.nk = f.y;
      }
      o.mode = o.nk == 0.f ? ROW_ZERO : ROW_FAST;
      // q_y (b / sigma - kA) - ce (1 - q_y)
      o.gy = nan ? NAN : w * (ey * per_R * (ba - sum_a * sigma) - cc * (not_y * inv));
      *out = o;
    }
    __syncwarp();
  };
  if (!d.reverse) {  // its gradient needs no logarithm: given first
    if (any) {
      av[0] = -pre.p[0];
      av[1] = -pre.p[1];
      b = klass ? -pre.rho : 0.f;
      a_all = -pre.sum;
      kA = b + a_all;
    }
    if (out) result();
    if (out_bar && lane == 0) bar_arrive(out_bar);
  }
  const LogSum log_S(S);
  LogProb l[2] = {LogProb(x[0], a.c2, K, log_S), LogProb(x[1], a.c2, K, log_S)};
  const LogSum log_R(R);
  const float l_sigma = sigma > 0.5f
                            ? log1pf(-E * inv)
                            : ((k - K) + (log_R.e - log_S.e) + (log_R.f - log_S.f)) * LN2;
  // the divergence
  const float to = d.none ? pre.rho : 0.f, to_lo = d.none ? pre.l_rho : 0.f;
  auto more = [&](const LogProb& v, float t) {  // log q - log p
    return ((v.hi - t) + to) + (v.lo + to_lo);
  };
  float kl = 0.f;
  if (!d.reverse) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (pre.p[h] > 0.f) kl -= pre.p[h] * more(l[h], pre.lt[h]);
    kl = warp_sum(kl);
    if (klass && any) kl += pre.rho * (pre.l_rho - l_sigma);
  } else {
    if (any) {  // (a and b add up to 0)
      float off[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        av[h] = q[h];
        off[h] = more(l[h], pre.lt[h]);
      }
      if (d.none) {  // q over the list
        const float xm = warp_max(fmaxf(on[0] ? x[0] : -INFINITY, on[1] ? x[1] : -INFINITY));
        if (xm == -INFINITY) bad = true;
#pragma unroll
        for (int h = 0; h < 2; ++h) av[h] = on[h] ? rescale2((x[h] - xm) * a.c2) : 0.f;
        const float Q = warp_sum(av[0] + av[1]), per_Q = __fdividef(1.f, Q);
        const LogSum log_Q(Q);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          off[h] = more(LogProb(x[h] - xm, a.c2, 0.f, log_Q), pre.lt[h]);
          av[h] *= per_Q;
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (av[h] > 0.f) kl += av[h] * off[h];
      kl = warp_sum(kl);
      const float far = l_sigma - pre.l_rho;
      const bool out_there = klass && sigma > 0.f;
      if (out_there) kl += sigma * far;
#pragma unroll
      for (int h = 0; h < 2; ++h) av[h] = av[h] > 0.f ? av[h] * (off[h] - kl) : 0.f;
      if (out_there) b = sigma * (far - kl);
      a_all = -b;
    }
    if (out) result();
    if (out_bar && lane == 0) bar_arrive(out_bar);
  }
  // the label, from 1 - q where that is small
  float ce = 0.f;
  if (a.chosen) {
    float v, less, log_v;
    if (apart) {
      v = eyk * inv;
      less = not_y * inv;
      log_v = LogProb(xy, a.c2, K, log_S).hi;
    } else {
      const bool y0 = on[0] && in.id[0] == in.y, y1 = on[1] && in.id[1] == in.y;
      const unsigned who = __ballot_sync(FULL, y0 || y1);
      const int from = who ? __ffs(who) - 1 : 0;
      const bool sure = most && (y0 ? is[0] : is[1]);
      v = __shfl_sync(FULL, y0 ? q[0] : q[1], from);
      less = __shfl_sync(FULL, sure ? others * inv : 1.f - (y0 ? q[0] : q[1]), from);
      log_v = __shfl_sync(FULL, y0 ? l[0].hi : l[1].hi, from);
    }
    ce = v > 0.5f ? -log1pf(-less) : -log_v;
  }
  bad |= pre.bad_id;
  if (bad) kl = ce = NAN;
  if (lane < DS_TERMS) {
    const float t =
        wt * (lane == 0 ? kl : lane == 1 ? ce : bad ? NAN : lane == 2 ? pre.mass : E * inv);
    const float2 s = stat[lane];
    const float y = s.x + t, z = y - s.x;
    stat[lane] = make_float2(y, s.y + ((s.x - (y - z)) + (t - z)));
  }
  if (lane == 0 && writes) {
    a.logp[row] = kl;
    if (bad) atomicOr(a.ctx_flags, pre.bad_id ? FLAG_BAD_CHOSEN : FLAG_NONFINITE);
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

// ---- the lists of larger batches, ahead of the rows ---------------------------------------------
//
// What of a row's end does not wait for its sum, a row to a warp: the warp that takes the ends
// would wait for the entries, then for the logits at them, and work out their probabilities, longer
// than its row takes (7,800 rows of V = 151,936 bf16 with lists of 64 and their gradient: 796 us
// for 837).
constexpr int DP_NT = 256;
template <typename T>
__global__ void __launch_bounds__(DP_NT) distill_lists(const __grid_constant__ DistillArgs d) {
  const LossArgs& a = d.a;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_wait();
  pdl_trigger();
  const Rows rows{nullptr, (int32_t)__ldcg(a.totals)};
  const int64_t i = (int64_t)blockIdx.x * (DP_NT / 32) + warp;
  if (i >= rows.live) return;
  const int4 ref = rows.at(a, i);
  ListIn in = fetch_list(d, rows, ref, lane);
  fetch_logits<T>(d, share_of<T>(a, ref.x, 1, 0), ref, in, lane);
  ListPre o;
  list_pre(d, in, o, lane);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int j = 32 * h + lane;
    if (j < d.k)
      d.entries[i * d.k + j] = make_int4(in.id[h], (int32_t)in.x[h], __float_as_int(o.p[h]),
                                         __float_as_int(o.lt[h]));
  }
  if (lane == 0) {
    const double share = rows.share(a);
    const float wt = (float)(a.norm ? share / (double)in.count : share);
    d.scalars[2 * i] = make_float4(o.sum, o.rho, o.l_rho, o.mass);
    d.scalars[2 * i + 1] = make_float4(
        wt, __uint_as_float(in.xy),
        __uint_as_float((o.bad ? 1u : 0u) | (o.bad_id ? 2u : 0u) | (o.labelled ? 4u : 0u)), 0.f);
  }
}

// The elements at a row's ends (this lane's at v, its value in.edge) into the sum, but the
// listed ones and the label.  `at`: what v is, an entry's place, DS_LABEL, or DS_REST.
constexpr int DS_REST = -1, DS_LABEL = -2;
__device__ __forceinline__ int end_kind(const DistillArgs& d, const Share& s, const ListIn& in,
                                        int32_t v, int lane) {
  int kind = d.a.chosen && v == in.y ? DS_LABEL : DS_REST;
  const int32_t lo = s.head, hi = (int32_t)d.a.vocab - s.tail;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    unsigned b = __ballot_sync(FULL, in.id[h] >= 0 && (in.id[h] < lo || in.id[h] >= hi));
    while (b) {
      const int q = __ffs(b) - 1;
      b &= b - 1;
      const int32_t id = __shfl_sync(FULL, in.id[h], q);
      if (id == v) kind = 32 * h + q;
    }
  }
  return kind;
}
__device__ __forceinline__ void add_rest_ends(const DistillArgs& d, const Share& s, float edge,
                                              int32_t v, int kind, float& k, float& R) {
  if (s.head + s.tail == 0) return;
  const float c2 = d.a.c2;
  const bool add = v >= 0 && kind == DS_REST;
  const float top = warp_max(add ? fmaxf(edge * c2, LOWEST_REF) : LOWEST_REF);
  if (top > k) {
    R *= rescale2(k - top);
    k = top;
  }
  R += warp_sum(add ? ex2(fmaf(edge, c2, -k)) : 0.f);
}
template <typename T>
__device__ __forceinline__ void put_end(T* g, int32_t v, int kind, const RowOut& o,
                                        const float* list, float c2, float edge) {
  if (v >= 0) put(g + v, kind >= 0 ? list[kind] : kind == DS_LABEL ? o.gy : grad1(o, c2, edge));
}

// Element `e` of a row in shared memory is no part of its sum.  The next copy into the place is the
// async proxy's: a fence lies between, of the thread that issues the copy, which has no stores on
// their way.  (Fences of the threads that write gradients waited for those: 1 to 2%.  In registers,
// a loaded word's elements left out one by one: 9,000 rows of 151,936 bf16 with k = 64 1,045 us for
// 930.)
template <typename T>
__device__ __forceinline__ void leave_out(unsigned char* row, int32_t e) {
  if constexpr (sizeof(T) == 2) reinterpret_cast<uint16_t*>(row)[e] = 0xff80u;
  else reinterpret_cast<uint32_t*>(row)[e] = 0xff800000u;
}
__device__ __forceinline__ void fence_async() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// ---- rows in a ring of shared memory ---------------------------------------------------------
//
// As the policy loss': a row to a CTA, or its parts to the CTAs of a cluster; one warp
// brings chunks of 16 KB in by bulk copies, eight sum them and write the gradient from
// them, one takes the row's end.  Before a warp sums its words of a chunk, the lanes that
// hold one of the row's listed tokens there write -inf over it; when it has written the words'
// gradient, the same lanes write the list's entries over that.
//
// Without a gradient nothing has to be held, and `parts` of a row may go through one CTA, one after
// the other: a row of a cluster's eight parts fills 120 of 152 SMs, as clusters of eight find no
// more room.  Sums are kept apart as a cluster's CTAs keep them, so that the loss has the same bits.

// a lane's tokens among its warp's words of this CTA's part of a row: their elements from the
// row's first word on, or -1
struct Mine {
  int32_t e[3];     // entries lane and 32 + lane; the label (lane 0)
  uint32_t chunks;  // of the CTA's part in which the warp has any, a bit each
};
struct Ids {
  int32_t id[2];
  float t[2];
};
__device__ __forceinline__ Ids fetch_ids(const DistillArgs& d, const int4& ref, int lane) {
  Ids r;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int j = 32 * h + lane;
    const int64_t at = (int64_t)ref.x * d.k + j;
    const bool on = ref.y >= 0 && j < d.k;
    r.id[h] = on ? __ldcg(d.ids + at) : -1;  // (both loads at once: the row is the next one)
    r.t[h] = on ? __ldcg(d.t_logp + at) : -INFINITY;
  }
  return r;
}
template <int VEC>
__device__ __forceinline__ Mine mine_of(const DistillArgs& d, const Share& s, const Ids& ids,
                                        int32_t y, int warp, int lane) {
  Mine m;
  m.chunks = 0u;
  const int32_t l[2] = {ids.t[0] == -INFINITY ? -1 : ids.id[0],
                        ids.t[1] == -INFINITY ? -1 : ids.id[1]};
  const bool listed = l[0] == y || l[1] == y;
  const bool apart = d.a.chosen && !__any_sync(FULL, listed);
#pragma unroll
  for (int h = 0; h < 3; ++h) {
    const int32_t id = h < 2 ? l[h] : apart && lane == 0 ? y : -1;
    const int32_t e = id - s.head, w = e / VEC - s.w0;  // (`in` looks at a negative e)
    const bool in = id >= s.head && w >= 0 && e / VEC < s.w1;
    const bool here = in && ((w % (32 * RG_NW)) >> 5) == warp;
    m.e[h] = here ? e : -1;
    m.chunks |= here ? 1u << (w / RG_CHUNK) : 0u;
  }
  m.chunks = __reduce_or_sync(FULL, m.chunks);
  return m;
}

struct DistillCtl {
  uint64_t sum_bar[RG_SLOTS];  // the warps' sums are there
  uint64_t out_bar[RG_SLOTS];  // a row's result is there
  float2 stat[DS_TERMS];       // sums over the rows
  RowOut out[RG_SLOTS];        // a row's result
};
// then the bars of the ring's places (landed, read), the warps' (k, R) [RG_SLOTS][C][RG_NW], the
// lists' entries of the gradient [1 + lag][DS_MAX], and the ring
constexpr size_t DS_BARS = (sizeof(DistillCtl) + 15) / 16 * 16;
__host__ __device__ constexpr size_t distill_sums(int places) {
  return DS_BARS + 16 * (size_t)places;
}
__host__ __device__ constexpr size_t distill_list(int C, int places) {
  return distill_sums(places) + (size_t)RG_SLOTS * C * RG_NW * sizeof(float2);
}
__host__ __device__ constexpr size_t distill_start(int C, int places, int lag) {
  return distill_list(C, places) + (size_t)(1 + lag) * DS_MAX * sizeof(float);
}
static_assert(distill_start(4, RG_FEW, 0) <= 1024 && distill_start(1, RG_FEW, 1) <= 1024,
              "two CTAs on an SM");

// PREPARED: distill_lists ran ahead (with a gradient, which has the ends on the way of the rows).
template <typename T, bool HOLD, bool OWN>
__global__ void __launch_bounds__(RG_NT, 2)
    distill_ring(const __grid_constant__ DistillArgs d, const int places, const int lag,
                 const int parts) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  DistillCtl& sm = *reinterpret_cast<DistillCtl*>(smem_raw);
  const LossArgs& a = d.a;
  using Tr = Traits<T>;
  constexpr bool PREPARED = HOLD && !OWN;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t C, rank;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(C));
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const int64_t G = gridDim.x / C, first = blockIdx.x / C;
  const uint32_t P = HOLD ? C : C * parts;  // parts of a row; this CTA has rank, or all of them
  const uint32_t p_first = HOLD || parts == 1 ? rank : 0,
      p_last = HOLD ? p_first + 1 : parts == 1 ? rank + 1 : P;
  uint64_t* const full = reinterpret_cast<uint64_t*>(smem_raw + DS_BARS);
  uint64_t* const empty = full + places;
  float2* const sums = reinterpret_cast<float2*>(smem_raw + distill_sums(places));
  float* const list = reinterpret_cast<float*>(smem_raw + distill_list((int)P, places));
  unsigned char* const ring = smem_raw + distill_start((int)P, places, lag);
  if (threadIdx.x == 0) {
    for (int i = 0; i < places; ++i) {
      bar_init(&full[i], 1);
      bar_init(&empty[i], RG_NW);
    }
    for (int s = 0; s < RG_SLOTS; ++s) {
      bar_init(&sm.sum_bar[s], C > 1 ? 1 : RG_NW);
      bar_init(&sm.out_bar[s], 1);
      if (C > 1) bar_expect(&sm.sum_bar[s], 8 * RG_NW * C);
    }
    for (int j = 0; j < DS_TERMS; ++j) sm.stat[j] = make_float2(0.f, 0.f);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async();
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
      for (uint32_t p = p_first; p < p_last; ++p) {
        const Share sh = share_of<T>(a, ref.x, P, p);
        const char* src = sh.x + sizeof(T) * sh.head + 16 * (int64_t)sh.w0;
        for (int32_t left = sh.w1 - sh.w0; left > 0; left -= RG_CHUNK) {
          if (n >= places) {
            wait(&empty[place], turn ^ 1u);
            fence_async();
          }
          if (ok && lane == 0) {
            const uint32_t bytes = 16u * (uint32_t)min(RG_CHUNK, left);
            bar_expect(&full[place], bytes);
            asm volatile(
                "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::
                    "r"(sm_addr(ring + (size_t)place * RG_BYTES)),
                "l"(src), "r"(bytes), "r"(sm_addr(&full[place]))
                : "memory");
          }
          src += RG_BYTES;
          if (ok) ++n;
          step();
        }
      }
      ref = ref1;
    }
    // no copy may be in flight when the CTA ends (as none is unless a wait ran out)
    ok = true;
    for (int64_t i = n < places ? 0 : n - places; i < n; ++i)
      wait(&full[(int)(i % places)], (uint32_t)(i / places) & 1u);
  } else if (warp == RG_NW + 1) {
    // ---- the rows' ends
    const double share = !PREPARED ? rows.share(a) : 0.0;
    uint32_t n = 0;
    int4 ref = ref_of(first), ref1 = ref_of(first + G), ref2 = ref_of(first + 2 * G);
    ListIn in, next;
    ListPre pre, pre1;
    float wt, wt1;
    auto edge = [&](const int4& r, ListIn& q) {  // the element at the row's ends of this lane
      const Share sh = share_of<T>(a, r.x, C, rank);
      const int32_t v = r.y >= 0 ? end_of(a, sh, lane) : -1;
      if (v >= 0) q.edge = raw_at<T>(sh.x, v);
    };
    if constexpr (!PREPARED) {
      in = fetch_list(d, rows, ref, lane);
      next = fetch_list(d, rows, ref1, lane);
      fetch_logits<T>(d, share_of<T>(a, ref.x, C, rank), ref, in, lane);
    } else {
      fetch_prepared(d, first, ref, in, pre, wt, lane);
      edge(ref, in);
    }
    // What a peer's gradient may be written over (the logits' own buffer) has been read when
    // this CTA's sums are sent: the next row's logits are there before a result is given.
    auto landed = [&](ListIn& q) {
      if (!PREPARED) {
        q.x[0] = __shfl_sync(FULL, q.x[0], lane);
        q.x[1] = __shfl_sync(FULL, q.x[1], lane);
        q.xy = __shfl_sync(FULL, q.xy, lane);
      }
      q.edge = __shfl_sync(FULL, q.edge, lane);
    };
    landed(in);
    if (C > 1) named_bar_arrive(BAR_IN, 32 * (RG_NW + 1));
    for (int64_t i = first; i < live; i += G) {
      const int64_t row = ref.x;
      const Share sh = share_of<T>(a, row, C, rank);
      ListIn after;
      if constexpr (!PREPARED) {
        fetch_logits<T>(d, share_of<T>(a, ref1.x, C, rank), ref1, next, lane);
        after = fetch_list(d, rows, ref2, lane);
      } else {
        fetch_prepared(d, i + G, ref1, next, pre1, wt1, lane);
        edge(ref1, next);
      }
      ref = ref1;
      ref1 = ref2;
      ref2 = ref_of(i + 3 * G);
      const int32_t v = end_of(a, sh, lane);
      const int kind = sh.head + sh.tail ? end_kind(d, sh, in, v, lane) : DS_REST;
      if constexpr (!PREPARED) {
        list_pre(d, in, pre, lane);
        wt = (float)(a.norm ? share / (double)in.count : share);
      }
      T* const g = reinterpret_cast<T*>(a.grad) + row * a.grad_stride;
      const int s = n % RG_SLOTS;
      const uint32_t phase = (n / RG_SLOTS) & 1u;
      float* const entries = list + (lag ? s : 0) * DS_MAX;
      ++n;
      wait(&sm.sum_bar[s], phase);
      float k, R;
      {
        const float2* q = sums + s * RG_NW * P;
        const float2 none = make_float2(-3e38f, 0.f);
        float2 p = lane < (int)(RG_NW * P) ? q[lane] : none;
        if (P > 4) {
          const float2 p2 = q[32 + lane];
          const float top = fmaxf(p.x, p2.x);
          p = make_float2(top, p.y * rescale2(p.x - top) + p2.y * rescale2(p2.x - top));
        }
        __syncwarp();
        if (C > 1 && lane == 0) bar_expect(&sm.sum_bar[s], 8 * RG_NW * C);
        join(p, 1.f, k, R);
      }
      add_rest_ends(d, sh, wide<T>(in.edge), v, kind, k, R);
      if (C > 1) landed(next);
      list_math<T>(d, row, in, pre, k, R, wt, rank == 0, HOLD ? &sm.out[s] : nullptr, entries,
                   &sm.out_bar[s], sm.stat, lane);
      __syncwarp();
      if (HOLD && rank == 0) put_end(g, v, kind, sm.out[s], entries, a.c2, wide<T>(in.edge));
      in = next;
      if constexpr (!PREPARED) {
        next = after;
      } else {
        pre = pre1;
        wt = wt1;
      }
    }
  } else {
    // ---- the rows' words
    uint32_t n = 0, m = 0;  // rows summed; written
    const uint32_t mine = first < live ? (uint32_t)((live - 1 - first) / G) + 1u : 0u;
    if (C > 1) named_bar_sync(BAR_IN, 32 * (RG_NW + 1));
    const int at = warp * 32 + lane;  // this lane's first word of a chunk
    int4 ref = ref_of(first), next = ref_of(first + G);  // the row to be summed; the one after it
    int4 held = ref;              // the row to be written
    Ids ids = fetch_ids(d, ref, lane);
    int4 last = ref;              // the one summed last
    Mine own, kept;               // the tokens of that one; of the one to be written
    int place0 = 0;               // its place
    auto within = [&](int32_t e, int32_t w) {  // whether element e is in the chunk at word w
      return e >= 0 && (uint32_t)(e / Tr::VEC - w) < (uint32_t)RG_CHUNK;
    };
    while ((HOLD ? m : n) < mine) {
      if (n < mine) {
        // forward
        const int s = n % RG_SLOTS;
        const Ids here_ids = ids;
        ids = fetch_ids(d, next, lane);
        for (uint32_t p = p_first; p < p_last; ++p) {
          const Share sh = share_of<T>(a, ref.x, P, p);
          own = mine_of<Tr::VEC>(d, sh, here_ids, ref.z, warp, lane);
          if (m == n) kept = own;
          float k = -3e38f;
          float2 S = make_float2(0.f, 0.f);
          uint32_t chunks = own.chunks;
          for (int32_t w = sh.w0; w < sh.w1; w += RG_CHUNK, chunks >>= 1) {
            wait(&full[place], turn);
            unsigned char* const here = ring + (size_t)place * RG_BYTES;
            const uint4* st = reinterpret_cast<const uint4*>(here) + at;
            uint4 v[RG_W];
#pragma unroll
            for (int q = 0; q < RG_W; ++q) v[q] = st[32 * RG_NW * q];
            // (The loads come first: most chunks hold none of a warp's tokens.  9,000 rows of
            // 151,936 bf16, k = 32: 907 us, with the branch ahead of them 933.)
            if (chunks & 1u) {
              __syncwarp();
#pragma unroll
              for (int h = 0; h < 3; ++h)
                if (within(own.e[h], w)) leave_out<T>(here, own.e[h] - w * Tr::VEC);
              __syncwarp();
#pragma unroll
              for (int q = 0; q < RG_W; ++q) v[q] = st[32 * RG_NW * q];
            }
            if (w + RG_CHUNK > sh.w1) {
#pragma unroll
              for (int q = 0; q < RG_W; ++q)
                if (w + 32 * RG_NW * q + at >= sh.w1)
                  v[q] = make_uint4(Tr::NEG_WORD, Tr::NEG_WORD, Tr::NEG_WORD, Tr::NEG_WORD);
            }
            add_words<T>(k, S, v, a.c2, w == sh.w0, LOWEST_REF);
            if (!HOLD) {
              // The place is given back once every lane's words are in its sum: given back right
              // after their loads, with a chunk's listed tokens just left out, one row in 2,000
              // of V = 262,144 fp32 k = 64 summed some of the next chunk.  (No time between them.)
              __syncwarp();
              if (lane == 0) bar_arrive(&empty[place]);
            }
            step();
          }
          float R;
          join(make_float2(k, S.x + S.y), 1.f, k, R);
          if (!HOLD && p == p_first && n >= 1) wait(&sm.out_bar[s ^ 1], ((n - 1) / RG_SLOTS) & 1u);
          if (C > 1) send(sums + (s * C + rank) * RG_NW + warp, &sm.sum_bar[s], k, R, C, lane);
          else if (lane == 0) sums[(s * P + p) * RG_NW + warp] = make_float2(k, R);
        }
        if (C == 1 && lane == 0) bar_arrive(&sm.sum_bar[s]);
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
        const int s = m % RG_SLOTS;
        wait(&sm.out_bar[s], (m / RG_SLOTS) & 1u);
        const RowOut o = sm.out[s];
        const float* const entries = list + (lag ? s : 0) * DS_MAX;
        const float mine0 = entries[lane], mine1 = entries[32 + lane];
        uint32_t chunks = kept.chunks;
        for (int32_t w = sh.w0; w < sh.w1; w += RG_CHUNK, chunks >>= 1) {
          const uint4* st = reinterpret_cast<const uint4*>(ring + (size_t)place0 * RG_BYTES) + at;
          T* const to = g + (int64_t)(w + at) * Tr::VEC;
          uint4 v[RG_W];
#pragma unroll
          for (int q = 0; q < RG_W; ++q) v[q] = st[32 * RG_NW * q];
          if (o.mode == ROW_FAST) {
#pragma unroll
            for (int q = 0; q < RG_W; ++q) v[q] = grad_word<T, false>(o, a.c2, v[q]);
          } else {
#pragma unroll
            for (int q = 0; q < RG_W; ++q) v[q] = make_uint4(0u, 0u, 0u, 0u);
          }
          __syncwarp();
          if (lane == 0) bar_arrive(&empty[place0]);
          if (++place0 == places) place0 = 0;
          if (vec && w + RG_CHUNK <= sh.w1) {
#pragma unroll
            for (int q = 0; q < RG_W; ++q)
              *reinterpret_cast<uint4*>(to + 32 * RG_NW * q * Tr::VEC) = v[q];
          } else {
#pragma unroll
            for (int q = 0; q < RG_W; ++q)
              if (w + 32 * RG_NW * q + at < sh.w1)
                put_word(to + 32 * RG_NW * q * Tr::VEC, v[q], vec);
          }
          if (chunks & 1u) {
            __syncwarp();  // the warp's words are written: the list's entries over them
#pragma unroll
            for (int h = 0; h < 3; ++h)
              if (within(kept.e[h], w)) put(g + kept.e[h], h == 0 ? mine0 : h == 1 ? mine1 : o.gy);
          }
        }
        ++m;
        held = m == n ? ref : last;
        kept = own;
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
  if (warp == 0 && rank == 0 && first < groups) list_stats(d, sm.stat, 1, first, groups, lane);
}

// ---- short rows: one to a warp ----------------------------------------------------------------
//
// As the other losses': a row's end is longer than a short row's data take, so that up to
// 20 rows of an SM are in work at a time.

struct DistillRowsCtl {
  uint64_t full[RW_MOST];    // a row has landed
  RowOut out[RW_MOST];
  float2 stat[RW_MOST * DS_TERMS];
  float list[RW_MOST * DS_MAX];
};
constexpr size_t DR_CTL = (sizeof(DistillRowsCtl) + 15) / 16 * 16;

template <typename T, bool HOLD>
__global__ void __launch_bounds__(32 * RW_MOST, 2)
    distill_rows(const __grid_constant__ DistillArgs d, const int bytes) {  // of a warp's part
  extern __shared__ __align__(16) unsigned char smem_raw[];
  DistillRowsCtl& sm = *reinterpret_cast<DistillRowsCtl*>(smem_raw);
  const LossArgs& a = d.a;
  using Tr = Traits<T>;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  unsigned char* const part = smem_raw + DR_CTL + (size_t)warp * bytes;
  uint64_t* const full = &sm.full[warp];
  float2* const stat = sm.stat + warp * DS_TERMS;
  float* const list = sm.list + warp * DS_MAX;
  if (lane == 0) {
    bar_init(full, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async();
  }
  if (lane < DS_TERMS) stat[lane] = make_float2(0.f, 0.f);
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  const Rows rows{nullptr, (int32_t)__ldcg(a.totals)};
  const double share = rows.share(a);
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
    ListIn in = fetch_list(d, rows, ref, lane);
    const int4 ref1 = rows.at(a, i + G);
    fetch_logits<T>(d, sh, ref, in, lane);
    const int32_t v = end_of(a, sh, lane);
    const int kind = sh.head + sh.tail ? end_kind(d, sh, in, v, lane) : DS_REST;
    ListPre pre;
    list_pre(d, in, pre, lane);
    if (!ring_wait(sm_addr(full), phase, a.ctx_flags)) {
      ring_wait(sm_addr(full), phase, a.ctx_flags);  // no copy may be in flight at the end
      break;
    }
    phase ^= 1u;
    __syncwarp();
    const int32_t end = sh.words * Tr::VEC;
    auto inside = [&](int32_t id) { return id >= sh.head && id - sh.head < end; };
    const bool label = a.chosen && inside(in.y);
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (inside(in.id[h])) leave_out<T>(part, in.id[h] - sh.head);
    if (lane == 0 && label) leave_out<T>(part, in.y - sh.head);
    fence_async();
    __syncwarp();
    const uint4* const st = reinterpret_cast<const uint4*>(part) + lane;
    float k = -3e38f, R;
    float2 S = make_float2(0.f, 0.f);
    for (int32_t w = 0; w < sh.words; w += 32 * RG_W) {
      uint4 x[RG_W];
#pragma unroll
      for (int q = 0; q < RG_W; ++q)
        x[q] = w + 32 * q + lane < sh.words
                   ? st[w + 32 * q]
                   : make_uint4(Tr::NEG_WORD, Tr::NEG_WORD, Tr::NEG_WORD, Tr::NEG_WORD);
      add_words<T>(k, S, x, a.c2, w == 0, LOWEST_REF);
    }
    join(make_float2(k, S.x + S.y), 1.f, k, R);
    add_rest_ends(d, sh, wide<T>(in.edge), v, kind, k, R);
    const float wt = (float)(a.norm ? share / (double)in.count : share);
    list_math<T>(d, ref.x, in, pre, k, R, wt, true, HOLD ? &sm.out[warp] : nullptr, list, nullptr,
                 stat, lane);
    __syncwarp();
    if (HOLD) {
      const RowOut o = sm.out[warp];
      T* const g = reinterpret_cast<T*>(a.grad) + (int64_t)ref.x * a.grad_stride;
      T* const gw = g + sh.head;
      const bool vec = ((reinterpret_cast<uintptr_t>(sh.x) ^ reinterpret_cast<uintptr_t>(g)) & 15u) == 0;
      for (int32_t w = lane; w < sh.words; w += 32) {
        uint4 x = make_uint4(0u, 0u, 0u, 0u);
        if (o.mode == ROW_FAST) x = grad_word<T, false>(o, a.c2, st[w - lane]);
        put_word(gw + (int64_t)w * Tr::VEC, x, vec);
      }
      put_end(g, v, kind, o, list, a.c2, wide<T>(in.edge));
      __syncwarp();  // the row is written: the list's entries over it
      if (lane == 0 && label && !pre.labelled) put(g + in.y, o.gy);
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (inside(in.id[h])) put(g + in.id[h], list[32 * h + lane]);
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
  __syncthreads();
  const int64_t groups = max((int64_t)1, min((int64_t)gridDim.x, (int64_t)rows.live));
  if (warp == 0 && blockIdx.x < groups) list_stats(d, sm.stat, warps, blockIdx.x, groups, lane);
}

}  // namespace prk
