// The k largest logits of a row: their tokens in the order (value descending, index
// ascending) and their log-probabilities.
//
// Cut the row into groups of neighbouring elements and order the groups by (largest
// element descending, position ascending): the first k elements lie in the first k
// groups.  (An element of another group has k elements before it, one at least in each of
// those.)  So the stream keeps one maximum per group beside the sum of exponentials, the
// k groups are chosen among the maxima, and the elements among theirs, whatever the row
// holds: ties and rows in order cost what others do.
// l_v = (c x_v - K) ln 2 - ln sum_u 2^(c x_u - K) with c = log2(e) / T and K the largest
// c x, rounded; the difference is one FMA, exact but for its last place as far as |c x| 2^-24 stays
// within the exponent's range: hence the bound of 1e9 T on what counts as finite.
#pragma once

#include "pr_kernels.cuh"

namespace prk {

constexpr int TP_MAX = 64;             // longest list
constexpr int TP_NT = 256;
constexpr int TP_GROUPS = 8192;        // of a row, at most

struct TopArgs {
  const void* logits;
  int64_t n_rows, vocab, row_stride;
  int32_t k;
  float c2;                            // log2(e) / T
  float big;                           // logits from here on are infinite: 1e9 T
  int32_t* ids;
  float* logp;
  uint32_t* ctx_flags;
};

// ---- a warp's list of the largest keys -----------------------------------------------

// a, b sorted descending across lanes: a gets the 32 largest of both, b the others, sorted
__device__ __forceinline__ uint64_t top_clean(uint64_t t, int lane) {
#pragma unroll
  for (int stride = 16; stride > 0; stride >>= 1) {
    const uint64_t o = shfl_xor64(t, stride);
    t = ((lane & stride) == 0) == (t > o) ? t : o;
  }
  return t;
}
__device__ __forceinline__ void top_split(uint64_t& a, uint64_t& b, int lane) {
  const uint64_t r = shfl64(b, 31 - lane), hi = a > r ? a : r, lo = a > r ? r : a;
  a = top_clean(hi, lane);
  b = top_clean(lo, lane);
}

// The k largest of the keys that are pushed; all are different and not 0.  Whole warp.
struct TopList {
  uint64_t* buf;            // 64 entries of shared memory
  int k, cnt = 0;           // entries in buf
  uint64_t hi = 0, lo = 0;  // ranks lane and 32 + lane
  uint64_t least = 0;       // the k-th largest so far
  __device__ __forceinline__ TopList(uint64_t* b, int k_) : buf(b), k(k_) {}
  __device__ __forceinline__ void take(uint64_t key, int lane) {  // 32 keys, 0 for none
    key = warp_sort_desc(key, lane);
    top_split(hi, key, lane);
    if (k > 32) lo = warp_merge_desc(lo, key, lane);
    least = shfl64(k > 32 ? lo : hi, (k - 1) & 31);
  }
  __device__ __forceinline__ void push(bool on, uint64_t key, int lane) {
    on = on && key > least;
    const unsigned b = __ballot_sync(FULL, on);
    if (b == 0) return;
    if (on) buf[cnt + __popc(b & ((1u << lane) - 1u))] = key;
    cnt += __popc(b);
    __syncwarp();
    if (cnt >= 32) {
      cnt -= 32;
      const uint64_t q = buf[cnt + lane];
      __syncwarp();
      take(q, lane);
    }
  }
  __device__ __forceinline__ void finish(int lane) {
    if (cnt == 0) return;
    __syncwarp();
    const uint64_t q = lane < cnt ? buf[lane] : 0ull;
    __syncwarp();
    cnt = 0;
    take(q, lane);
  }
};

// a value as a key has it: -0 is 0
__device__ __forceinline__ uint64_t top_key(float v, uint32_t index) { return make_key(v + 0.f, index); }

// The first k of n groups by their maxima at gm (shared memory): ranks lane and 32 + lane in hi and lo.
__device__ __forceinline__ void top_groups(TopList& l, const float* gm, int n, float big, int lane) {
  // a bound that k groups reach: of 64 sets of groups the k-th largest maximum
  float m0 = -INFINITY, m1 = -INFINITY;
  for (int g = lane; g < n; g += 64) {
    m0 = fmaxf(m0, gm[g]);
    if (g + 32 < n) m1 = fmaxf(m1, gm[g + 32]);
  }
  TopList s(l.buf, l.k);
  s.take(top_key(m0, lane), lane);
  s.take(top_key(m1, 32 + lane), lane);
  const float bound = fmaxf(key_val(s.least), -big);
  for (int g0 = 0; g0 < n; g0 += 32) {
    const int g = g0 + lane;
    const float m = g < n ? gm[g] : -INFINITY;
    l.push(m >= bound && m > -big, top_key(m, (uint32_t)g), lane);
  }
  l.finish(lane);
}

// ---- one row to a CTA -----------------------------------------------------------------

struct TopSmem {
  float gm[TP_GROUPS];
  float2 part[TP_NT / 32];
  uint64_t buf[64];
};

template <typename T>
__global__ void __launch_bounds__(TP_NT) top_rows(const TopArgs a, const int64_t group) {
  __shared__ TopSmem sm;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_wait();
  pdl_trigger();
  const int64_t row = blockIdx.x;
  const T* x = reinterpret_cast<const T*>(a.logits) + row * a.row_stride;
  const int groups = (int)((a.vocab + group - 1) / group);
  float k = -3e38f, S = 0.f;
  for (int g = tid; g < groups; g += TP_NT) {
    const int64_t v0 = g * group, v1 = min(a.vocab, v0 + group);
    float m = -INFINITY;
    for (int64_t v = v0; v < v1; ++v) m = fmaxf(m, Traits<T>::elem(x, v));
    sm.gm[g] = m;
    const float top = fmaxf(k, m * a.c2);
    float e = 0.f;
    for (int64_t v = v0; v < v1; ++v) e += ex2(fmaf(Traits<T>::elem(x, v), a.c2, -top));
    S = S * exp2f(k - top) + e;
    k = top;
  }
  const float kw = unord(__reduce_max_sync(FULL, ord(k)));
  S *= exp2f(k - kw);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) S += __shfl_xor_sync(FULL, S, o);
  if (lane == 0) sm.part[warp] = make_float2(kw, S);
  __syncthreads();
  if (warp > 0) return;
  const float2 p = lane < TP_NT / 32 ? sm.part[lane] : make_float2(-3e38f, 0.f);
  const float K = unord(__reduce_max_sync(FULL, ord(p.x)));
  float R = p.y * exp2f(p.x - K);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) R += __shfl_xor_sync(FULL, R, o);
  int32_t* const ids = a.ids + row * a.k;
  float* const logp = a.logp + row * a.k;
  if (!(K < a.big * a.c2) || !(K > -a.big * a.c2) || !(R > 0.f) || !(R < INFINITY)) {
    for (int j = lane; j < a.k; j += 32) {
      ids[j] = -1;
      logp[j] = NAN;
    }
    if (lane == 0) atomicOr(a.ctx_flags, FLAG_NONFINITE);
    return;
  }
  TopList l(sm.buf, a.k);
  top_groups(l, sm.gm, groups, a.big, lane);
  TopList e(sm.buf, a.k);
  for (int j = 0; j < a.k; ++j) {
    const uint64_t q = shfl64(j < 32 ? l.hi : l.lo, j & 31);
    if (q == 0) break;
    const int64_t v0 = (int64_t)key_idx(q) * group, v1 = min(a.vocab, v0 + group);
    for (int64_t w = v0; w < v1; w += 32) {
      const int64_t v = w + lane;
      const float f = v < v1 ? Traits<T>::elem(x, v) : -INFINITY;
      e.push(f > -a.big, top_key(f, (uint32_t)v), lane);
    }
  }
  e.finish(lane);
  const float lS = logf(R);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int j = 32 * h + lane;
    const uint64_t q = h == 0 ? e.hi : e.lo;
    if (j < a.k) {
      ids[j] = q ? (int32_t)key_idx(q) : -1;
      logp[j] = q ? fmaf(key_val(q), a.c2, -K) * LN2 - lS : -INFINITY;
    }
  }
}

}  // namespace prk
