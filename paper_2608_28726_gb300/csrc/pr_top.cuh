// The k largest logits of a row: their tokens in the order (value descending, index
// ascending) and their log-probabilities.
//
// Cut the row into groups of neighbouring elements and order the groups by (largest
// element descending, position ascending): the first k elements lie in the first k
// groups.  (An element of another group has k elements before it, one at least in each of
// those.)  So the stream keeps one maximum per group beside the sum of exponentials, the
// k groups are chosen among the maxima, and the elements among theirs, whatever the row
// holds: no threshold that rises along the row, which rows in order would raise at every step.
// l_v = (c x_v - K) ln 2 - ln sum_u 2^(c x_u - K) with c = log2(e) / T and K the largest
// c x, rounded; the difference is one FMA, exact but for its last place as far as |c x| 2^-24 stays
// within the exponent's range: hence the bound of 1e9 T on what counts as finite.
#pragma once

#include "pr_loss.cuh"

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
__device__ __forceinline__ uint64_t top_key(float v, uint32_t index) {
  return make_key(v + 0.f, index);
}

__device__ __forceinline__ float top_max(float m) { return m; }
__device__ __forceinline__ float top_max(uint16_t m) { return __uint_as_float((uint32_t)m << 16); }

// The first k of n groups by their maxima at gm (shared memory): ranks lane and 32 + lane in hi
// and lo.
template <typename M>
__device__ __forceinline__ void top_groups(TopList& l, const M* gm, int n, float big, int lane) {
  // a bound that k groups reach: of 64 sets of groups the k-th largest maximum
  float m0 = -INFINITY, m1 = -INFINITY;
  for (int g = lane; g < n; g += 64) {
    m0 = fmaxf(m0, top_max(gm[g]));
    if (g + 32 < n) m1 = fmaxf(m1, top_max(gm[g + 32]));
  }
  TopList s(l.buf, l.k);
  s.take(top_key(m0, lane), lane);
  s.take(top_key(m1, 32 + lane), lane);
  const float bound = fmaxf(key_val(s.least), -big);
  for (int g0 = 0; g0 < n; g0 += 32) {
    const int g = g0 + lane;
    const float m = g < n ? top_max(gm[g]) : -INFINITY;
    l.push(m >= bound && m > -big, top_key(m, (uint32_t)g), lane);
  }
  l.finish(lane);
}

// ---- a row's sum ------------------------------------------------------------------------------
//
// The losses leave the emitted token or the listed ones out of a row's sum, where here the largest
// element is nearly all of it.  So references are whole numbers, which the parts of a sum are
// brought to one another by exactly, and a term is below 2^15: its exponent is rounded by 2^-21 at
// most.  (With a reference that only an overflow raised, exponents of 30 and factors between
// references had a token of p = 1 - 1e-6 come out at -1e-6 +- 3e-6, now +- 4e-7; 4,096 rows of
// V = 151,936 bf16 k = 32 take 208 us for 207, with terms below 2^6 214.)

// 2^d of a whole d <= 0
__device__ __forceinline__ float top_scale(float d) {
  return d < -126.f ? 0.f : __uint_as_float((uint32_t)(127 + (int)d) << 23);
}

// A thread's words into its sum (k, S), as add_words' of the losses.
template <typename T, int N>
__device__ __forceinline__ void top_words(float& k, float2& S, const uint4 (&v)[N], float c2,
                                          bool begin) {
  using Tr = Traits<T>;
  auto top = [&]() {
    float m = Tr::gmax(v[0]);
#pragma unroll
    for (int q = 1; q < N; ++q) m = fmaxf(m, Tr::gmax(v[q]));
    return rintf(fmaxf(m * c2, LOWEST_REF));
  };
  if (begin) k = top();
  float2 here = make_float2(0.f, 0.f);
#pragma unroll
  for (int q = 0; q < N; ++q) add_word<T>(here, v[q], c2, -k);
  if (__any_sync(FULL, !(here.x + here.y < 32768.f))) {
    const float up = fmaxf(top(), k), f = top_scale(k - up);
    k = up;
    S.x *= f;
    S.y *= f;
    here = make_float2(0.f, 0.f);
#pragma unroll
    for (int q = 0; q < N; ++q) add_word<T>(here, v[q], c2, -k);
  }
  S = __fadd2_rn(S, here);
}

// (k, R) of the lanes together
__device__ __forceinline__ void top_join(float2 q, float& k, float& R) {
  k = warp_max(q.x);
  R = warp_sum(q.y * top_scale(q.x - k));
}

// The elements of the lanes that have one (x, else -inf), at a row's ends, into its sum
__device__ __forceinline__ void top_ends(float x, float c2, float& k, float& R) {
  const float t = fmaxf(warp_max(rintf(x * c2)), LOWEST_REF);
  if (t > k) {
    R *= top_scale(k - t);
    k = t;
  }
  R += warp_sum(x > -INFINITY || x != x ? ex2(fmaf(x, c2, -k)) : 0.f);
}

// ln of the sum, R against 2^k, in units of 2^K; an element's log-probability from it.  (In fp32
// the sum of a row that is one token may come out below its term.)
__device__ __forceinline__ float top_log(float k, float R, float K) { return logf(R * exp2f(k - K)); }
__device__ __forceinline__ float top_logp(float x, float c2, float K, float log_sum) {
  return fminf(fmaf(x, c2, -K) * LN2 - log_sum, 0.f);
}

// ---- any row: one to a CTA, in up to 8,192 groups, whatever their length --------------------

struct TopSmem {
  float gm[TP_GROUPS];
  float2 part[TP_NT / 32];
  float best[TP_NT / 32];
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
  float k = LOWEST_REF, S = 0.f, best = -INFINITY;
  for (int g = tid; g < groups; g += TP_NT) {
    const int64_t v0 = g * group, v1 = min(a.vocab, v0 + group);
    float m = -INFINITY;
    for (int64_t v = v0; v < v1; ++v) m = fmaxf(m, Traits<T>::elem(x, v));
    sm.gm[g] = m;
    best = fmaxf(best, m);
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
  best = warp_max(best);
  if (lane == 0) {
    sm.part[warp] = make_float2(kw, S);
    sm.best[warp] = best;
  }
  __syncthreads();
  if (warp > 0) return;
  best = warp_max(lane < TP_NT / 32 ? sm.best[lane] : -INFINITY);
  const float2 p = lane < TP_NT / 32 ? sm.part[lane] : make_float2(-3e38f, 0.f);
  const float K = unord(__reduce_max_sync(FULL, ord(p.x)));
  float R = p.y * exp2f(p.x - K);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) R += __shfl_xor_sync(FULL, R, o);
  int32_t* const ids = a.ids + row * a.k;
  float* const logp = a.logp + row * a.k;
  if (!(best < a.big) || !(best > -a.big) || !(R > 0.f) || !(R < INFINITY)) {
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
      logp[j] = q ? top_logp(key_val(q), a.c2, K, lS) : -INFINITY;
    }
  }
}

// ---- rows through a ring of shared memory ------------------------------------------------------
//
// A row to a CTA, or its parts to the CTAs of a cluster; a warp brings 16 KB chunks in by bulk
// copies, eight sum them and keep the groups' maxima: a group is what a thread takes of a chunk, GW
// 16-byte words side by side.  Then the eight choose together, by counting instead of sorting: of
// the threads' own maxima the k-th largest is a bound that k groups reach; the groups that reach it
// (some 75 for k = 64 in a row of random values) are read again, which the chunks of the next row
// do not wait for, and each of their elements that reaches it finds its place by counting the ones
// before it.  Where more groups or elements reach the bound than there is room for (rows of few
// values), a warp finds the first k groups and elements in TopLists.
constexpr int TR_NW = 8;
constexpr int TR_NT = 32 * (TR_NW + 1);
constexpr int TR_W = 4;                       // words of a thread and chunk
constexpr int TR_CHUNK = 32 * TR_NW * TR_W;   // words
constexpr int TR_BYTES = 16 * TR_CHUNK;
constexpr int TR_MOST = 12;                   // places of the ring
constexpr int TR_GROUPS = 64, TR_KEYS = 512;  // that reach the bound: groups of a warp, elements
constexpr int BAR_TOP = 1;                    // the eight warps
static_assert(TR_CHUNK == SH_CHUNK, "parts of a row are multiples of chunks");

struct TopRing {
  uint64_t full[TR_MOST], empty[TR_MOST];
  float2 part[TR_NW];            // the warps' sums
  uint32_t max[32 * TR_NW];      // the threads' largest elements as ord() has them, each warp's in order
  float bound;
  int keys[2];                   // how many elements reach it; of rows of either parity
  int crowded[2];                // there is no room for what reaches it
  uint16_t group[TR_NW][TR_GROUPS];
  uint64_t key[TR_KEYS];
  uint64_t top[TP_MAX];          // the first ones of this CTA's part, in order; 0: none
  // cluster rank 0: the CTAs' sums and lists
  float2 sums[MAXC];
  uint64_t lists[MAXC][TP_MAX];
};
static_assert(32 * TR_NW == 256 && TP_MAX == 64, "bisections and places below");
constexpr size_t TR_START = (sizeof(TopRing) + 127) / 128 * 128;  // then the groups' maxima, then the ring

template <typename T>
struct TopMax;
template <>
struct TopMax<float> {
  using type = float;
  static __device__ __forceinline__ float of(float m) { return m; }
};
template <>
struct TopMax<__nv_bfloat16> {
  using type = uint16_t;
  static __device__ __forceinline__ uint16_t of(float m) { return (uint16_t)(__float_as_uint(m) >> 16); }
};

// GW 4: rows of many words; GW 1: where a bound needs more groups than those have
template <typename T, int GW>
__global__ void __launch_bounds__(TR_NT, 3)
    top_ring(const __grid_constant__ LossArgs a, const int k, const float big,
             int32_t* const out_ids, const int places, const int gm_bytes) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  TopRing& sm = *reinterpret_cast<TopRing*>(smem_raw);
  using Tr = Traits<T>;
  using M = typename TopMax<T>::type;
  M* const gm = reinterpret_cast<M*>(smem_raw + TR_START);
  unsigned char* const ring = smem_raw + TR_START + gm_bytes;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  uint32_t C, rank;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(C));
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const int64_t G = gridDim.x / C, first = blockIdx.x / C;
  if (tid == 0) {
    for (int i = 0; i < places; ++i) {
      bar_init(&sm.full[i], 1);
      bar_init(&sm.empty[i], TR_NW);
    }
    sm.keys[0] = sm.keys[1] = sm.crowded[0] = sm.crowded[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
  if (C > 1) cluster_sync_all();
  pdl_wait();
  pdl_trigger();

  bool ok = true;  // no wait has run out
  auto wait = [&](uint64_t* b, uint32_t phase) {
    if (ok) ok = ring_wait(sm_addr(b), phase, a.ctx_flags);
    __syncwarp();
  };
  int place = 0;
  uint32_t turn = 0u;
  auto step = [&]() {
    if (++place == places) {
      place = 0;
      turn ^= 1u;
    }
  };
  uint32_t parity = 0u;
  int64_t n = 0;  // chunks brought in
  for (int64_t row = first; row < a.n_rows; row += G, parity ^= 1u) {
    const Share sh = share_of<T>(a, row, C, rank);
    if (warp == TR_NW) {
      const char* src = sh.x + sizeof(T) * sh.head + 16 * (int64_t)sh.w0;
      for (int32_t left = sh.w1 - sh.w0; left > 0; left -= TR_CHUNK) {
        if (n >= places) wait(&sm.empty[place], turn ^ 1u);
        if (ok && lane == 0) {
          const uint32_t bytes = 16u * (uint32_t)min(TR_CHUNK, left);
          bar_expect(&sm.full[place], bytes);
          asm volatile(
              "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::
                  "r"(sm_addr(ring + (size_t)place * TR_BYTES)),
              "l"(src), "r"(bytes), "r"(sm_addr(&sm.full[place]))
              : "memory");
        }
        src += TR_BYTES;
        if (ok) ++n;
        step();
      }
      if (C > 1) {
        cluster_sync_all();
        cluster_sync_all();
      }
      continue;
    }
    // ---- the row's sum and its groups' maxima
    float ref = -3e38f, top = -INFINITY;
    // (GW 4) this thread's first groups by their maxima, top being the first's, and where they are
    float top2 = -INFINITY, top3 = -INFINITY, top4 = -INFINITY;
    int32_t at1 = 0, at2 = 0, at3 = 0;
    float2 S = make_float2(0.f, 0.f);
    const int32_t groups = (sh.w1 - sh.w0 + GW - 1) / GW;
    for (int32_t w = sh.w0; w < sh.w1; w += TR_CHUNK) {
      wait(&sm.full[place], turn);
      const uint4* st = reinterpret_cast<const uint4*>(ring + (size_t)place * TR_BYTES);
      uint4 v[TR_W];
      int32_t at[TR_W];
#pragma unroll
      for (int q = 0; q < TR_W; ++q) {
        // (GW 4: neighbouring lanes begin with different words, so that no two meet in a bank)
        at[q] = GW == 4 ? 4 * tid + ((q + (lane >> 1)) & 3) : 32 * TR_NW * q + tid;
        v[q] = st[at[q]];
      }
      if (w + TR_CHUNK > sh.w1) {
#pragma unroll
        for (int q = 0; q < TR_W; ++q)
          if (w + at[q] >= sh.w1)
            v[q] = make_uint4(Tr::NEG_WORD, Tr::NEG_WORD, Tr::NEG_WORD, Tr::NEG_WORD);
      }
      const int32_t g = (w - sh.w0) / GW + tid;
      if constexpr (GW == 4) {
        const float m = Tr::tile_max(v);
        if (g < groups) gm[g] = TopMax<T>::of(m);
        if (m > top4) {
          const bool b1 = m > top, b2 = m > top2, b3 = m > top3;
          top4 = b3 ? top3 : m;
          top3 = b2 ? top2 : b3 ? m : top3;
          at3 = b2 ? at2 : b3 ? g : at3;
          top2 = b1 ? top : b2 ? m : top2;
          at2 = b1 ? at1 : b2 ? g : at2;
          top = b1 ? m : top;
          at1 = b1 ? g : at1;
        }
      } else {
#pragma unroll
        for (int q = 0; q < TR_W; ++q) {
          const float m = Tr::gmax(v[q]);
          if (g + 32 * TR_NW * q < groups) gm[g + 32 * TR_NW * q] = TopMax<T>::of(m);
          top = fmaxf(top, m);
        }
      }
      top_words<T>(ref, S, v, a.c2, w == sh.w0);
      __syncwarp();  // every lane's words are summed
      if (lane == 0) bar_arrive(&sm.empty[place]);
      step();
    }
    float R;
    top_join(make_float2(ref, S.x + S.y), ref, R);
    // the elements before and after the words: the first CTA's
    const float first_max = top;
    int32_t v_end = -1;
    float x_end = -INFINITY;
    if (warp == 0) {
      v_end = rank == 0 ? end_of(a, sh, lane) : -1;
      if (v_end >= 0) x_end = Tr::elem(sh.x, v_end);
      top_ends(x_end, a.c2, ref, R);
      top = fmaxf(top, x_end);
      if (lane == 0) sm.crowded[parity ^ 1u] = sm.keys[parity ^ 1u] = 0;
    }
    if (lane == 0) sm.part[warp] = make_float2(ref, R);
    const uint32_t sorted = warp_sort_desc(ord(top), lane);
    sm.max[tid] = sorted;
    named_bar_sync(BAR_TOP, 32 * TR_NW);
    // ---- the bound: the k-th largest of the threads' maxima
    top_join(lane < TR_NW ? sm.part[lane] : make_float2(-3e38f, 0.f), ref, R);
    {
      // the values before this lane's in each warp's list, of equal ones those of earlier warps
      int before = 0;
#pragma unroll
      for (int w = 0; w < TR_NW; ++w) {
        const uint32_t* l = sm.max + 32 * w;
        const uint32_t least = w < warp ? sorted : sorted + 1u;
        int n_before = 0;
#pragma unroll
        for (int s = 16; s > 0; s >>= 1)
          if (l[n_before + s - 1] >= least) n_before += s;
        if (l[n_before] >= least) ++n_before;
        before += w == warp ? lane : n_before;
      }
      if (before == k - 1) sm.bound = unord(sorted);
    }
    named_bar_sync(BAR_TOP, 32 * TR_NW);
    const float bound = sm.bound;
    auto reaches = [&](float x) { return x >= bound && x > -big; };
    // ---- the groups that reach it: each warp those of its threads
    int found = 0;
    auto list_groups = [&](bool on, int32_t g) {
      const unsigned b = __ballot_sync(FULL, on);
      const int i = found + __popc(b & ((1u << lane) - 1u));
      if (on && i < TR_GROUPS) sm.group[warp][i] = (uint16_t)g;
      found += __popc(b);
    };
    if (GW == 4 && !__any_sync(FULL, reaches(top4))) {
      list_groups(reaches(first_max), at1);
      list_groups(reaches(top2), at2);
      list_groups(reaches(top3), at3);
    } else if (__any_sync(FULL, reaches(top))) {
      for (int32_t g0 = 32 * warp; g0 < groups; g0 += 4 * 32 * TR_NW) {
        bool on[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int32_t g = g0 + 32 * TR_NW * q + lane;
          on[q] = g < groups && reaches(top_max(gm[g]));
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) list_groups(on[q], g0 + 32 * TR_NW * q + lane);
      }
    }
    __syncwarp();
    // ---- their elements that do
    const char* const words = sh.x + sizeof(T) * sh.head;
    auto take = [&](int mine) {  // the place of this lane's elements, `mine` of them
      int at = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int u = __shfl_up_sync(FULL, at, o);
        if (lane >= o) at += u;
      }
      const int all = __shfl_sync(FULL, at, 31);
      int base = 0;
      if (lane == 0 && all > 0) base = atomicAdd(&sm.keys[parity], all);
      return __shfl_sync(FULL, base, 0) + at - mine;
    };
    if (found <= TR_GROUPS) {
      constexpr int U = 2;  // words of a lane on their way
      for (int i0 = 0; i0 < found * GW; i0 += 32 * U) {
        uint4 q[U];
        int32_t w[U];
        int mine = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = i0 + 32 * u + lane;
          q[u] = make_uint4(Tr::NEG_WORD, Tr::NEG_WORD, Tr::NEG_WORD, Tr::NEG_WORD);
          w[u] = i < found * GW ? sh.w0 + (int32_t)sm.group[warp][i / GW] * GW + i % GW : sh.w1;
          if (w[u] < sh.w1) q[u] = ld_reread(words + 16 * (int64_t)w[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (reaches(Tr::gmax(q[u]))) {
#pragma unroll
            for (int j = 0; j < Tr::VEC; ++j) mine += reaches(Tr::at(q[u], j));
          }
        int to = take(mine);
        if (mine > 0) {
#pragma unroll
          for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int j = 0; j < Tr::VEC; ++j) {
              const float x = Tr::at(q[u], j);
              if (reaches(x)) {
                if (to < TR_KEYS) sm.key[to] = top_key(x, (uint32_t)(sh.head + w[u] * Tr::VEC + j));
                ++to;
              }
            }
          }
        }
      }
    } else if (lane == 0) {
      sm.crowded[parity] = 1;
    }
    if (warp == 0 && sh.head + sh.tail > 0) {
      const int mine = v_end >= 0 && reaches(x_end);
      const int to = take(mine);
      if (mine && to < TR_KEYS) sm.key[to] = top_key(x_end, (uint32_t)v_end);
    }
    named_bar_sync(BAR_TOP, 32 * TR_NW);
    // ---- their order
    const int count = sm.keys[parity];
    if (count <= TR_KEYS && !sm.crowded[parity]) {
      for (int i0 = 0; i0 < count; i0 += 8 * TR_NW) {  // four lanes a key
        const int i = i0 + (tid >> 2);
        const uint64_t mine = i < count ? sm.key[i] : 0ull;
        int before = 0;
#pragma unroll 4
        for (int j = lane & 3; j < count; j += 4) before += sm.key[j] > mine;
        before += __shfl_xor_sync(FULL, before, 1);
        before += __shfl_xor_sync(FULL, before, 2);
        if ((lane & 3) == 0 && i < count && before < k) sm.top[before] = mine;
      }
      if (tid >= count && tid < k) sm.top[tid] = 0ull;
    } else if (warp == 0) {
      TopList l(sm.key, k);
      top_groups(l, gm, groups, big, lane);
      TopList e(sm.key, k);
      for (int j = 0; j < k; ++j) {
        const uint64_t q = shfl64(j < 32 ? l.hi : l.lo, j & 31);
        if (q == 0) break;
        const int32_t w = sh.w0 + (int32_t)key_idx(q) * GW, el = (w - sh.w0) * Tr::VEC + lane;
        const bool in = lane < GW * Tr::VEC && el < (sh.w1 - sh.w0) * Tr::VEC;
        const int32_t v = sh.head + sh.w0 * Tr::VEC + el;
        const float x = in ? Tr::elem(sh.x, v) : -INFINITY;
        e.push(x > -big, top_key(x, (uint32_t)v), lane);
      }
      e.push(v_end >= 0 && x_end > -big, top_key(x_end, (uint32_t)v_end), lane);
      e.finish(lane);
      if (lane < k) sm.top[lane] = e.hi;
      if (32 + lane < k) sm.top[32 + lane] = e.lo;
    }
    named_bar_sync(BAR_TOP, 32 * TR_NW);
    // ---- the list
    const uint64_t mine = tid < k ? sm.top[tid] : 0ull;
    float2 all = make_float2(ref, R);
    if (C > 1) {
      if (tid < TP_MAX) dsmem_st_u64(dsmem_addr(&sm.lists[rank][tid], 0), mine);
      if (tid == 0)
        dsmem_st_u64(dsmem_addr(&sm.sums[rank], 0),
                     (uint64_t)__float_as_uint(ref) | (uint64_t)__float_as_uint(R) << 32);
      __syncwarp();
      cluster_sync_all();
    }
    if (rank == 0) {
      if (C > 1) top_join(lane < (int)C ? sm.sums[lane] : make_float2(-3e38f, 0.f), all.x, all.y);
      // against the row's largest element
      uint64_t best = 0ull;
      for (uint32_t c = 0; c < C; ++c) best = max(best, C > 1 ? sm.lists[c][0] : sm.top[0]);
      const float K = best ? key_val(best) * a.c2 : -INFINITY;
      // (the border by the element itself: times c it is one with its neighbours)
      const bool bad = !best || !(key_val(best) < big) || !(all.y < INFINITY) || !(all.y >= 0.f);
      const float log_sum = top_log(all.x, all.y, K);
      auto give = [&](int j, uint64_t q) {
        out_ids[row * k + j] = bad || q == 0 ? -1 : (int32_t)key_idx(q);
        a.logp[row * k + j] =
            bad ? NAN : q ? top_logp(key_val(q), a.c2, K, log_sum) : -INFINITY;
      };
      if (C == 1) {
        if (tid < k) give(tid, mine);
      } else {
        // an element's place is the number of those before it in each list, found by bisection
        // (lists end with zeros, which come after everything)
        for (int i = tid; i < (int)C * TP_MAX; i += 32 * TR_NW) {
          const int c = i / TP_MAX, j = i % TP_MAX;
          const uint64_t q = sm.lists[c][j];
          int before = j;
#pragma unroll
          for (int o = 0; o < MAXC; ++o) {
            const uint64_t* l = sm.lists[o];
            if (o < (int)C && o != c) {
              // of zeros, too, one comes after the other
              const uint64_t least = q == 0ull ? (o < c ? 0ull : 1ull) : q;
              int n_before = 0;
#pragma unroll
              for (int s = TP_MAX / 2; s > 0; s >>= 1)
                if (l[n_before + s - 1] >= least) n_before += s;
              if (l[n_before] >= least) ++n_before;
              before += n_before;
            }
          }
          if (before < k) give(before, q);
        }
      }
      if (bad && tid == 0) atomicOr(a.ctx_flags, FLAG_NONFINITE);
    }
    __syncwarp();
    if (C > 1) cluster_sync_all();
  }
  if (warp == TR_NW) {
    // no copy may be in flight when the CTA ends (as none is unless a wait ran out)
    ok = true;
    for (int64_t i = n < places ? 0 : n - places; i < n; ++i)
      wait(&sm.full[(int)(i % places)], (uint32_t)(i / places) & 1u);
  }
  __syncthreads();
  if (C > 1) cluster_sync_all();
}

// ---- short rows: one to a warp ---------------------------------------------------------------
//
// A CTA's choice is a chain of some 10,000 cycles, many times what a short row's data take.  So
// each warp has a row of its own, brought into its part of shared memory by one bulk copy: a group
// is a word, the bound is found bit by bit among the lanes' four largest groups each, and the
// elements that reach it go through a TopList.
constexpr int TS_MOST = 10;  // warps of a CTA; two CTAs on an SM
struct TopShort {
  uint64_t full[TS_MOST];    // a row has landed
  uint64_t buf[TS_MOST][64];
};
constexpr size_t TS_START = (sizeof(TopShort) + 15) / 16 * 16;

template <typename T>
__global__ void __launch_bounds__(32 * TS_MOST, 2)
    top_short(const __grid_constant__ LossArgs a, const int k, const float big,
              int32_t* const out_ids, const int bytes) {  // of a warp's part
  extern __shared__ __align__(16) unsigned char smem_raw[];
  TopShort& sm = *reinterpret_cast<TopShort*>(smem_raw);
  using Tr = Traits<T>;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  unsigned char* const part = smem_raw + TS_START + (size_t)warp * bytes;
  uint64_t* const full = &sm.full[warp];
  if (lane == 0) {
    bar_init(full, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncwarp();
  pdl_wait();
  pdl_trigger();
  const int64_t G = (int64_t)gridDim.x * warps;
  uint32_t phase = 0;
  for (int64_t row = (int64_t)warp * gridDim.x + blockIdx.x; row < a.n_rows; row += G) {
    const Share sh = share_of<T>(a, row, 1, 0);
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
    const int32_t v_end = end_of(a, sh, lane);
    const float x_end = v_end >= 0 ? Tr::elem(sh.x, v_end) : -INFINITY;
    if (!ring_wait(sm_addr(full), phase, a.ctx_flags)) {
      ring_wait(sm_addr(full), phase, a.ctx_flags);  // no copy may be in flight at the end
      break;
    }
    phase ^= 1u;
    __syncwarp();
    const uint4* const st = reinterpret_cast<const uint4*>(part) + lane;
    // ---- the sum, and the lane's four largest groups
    float ref = -3e38f, R, t1 = x_end, t2 = -INFINITY, t3 = -INFINITY, t4 = -INFINITY;
    float2 S = make_float2(0.f, 0.f);
    for (int32_t w = 0; w < sh.words; w += 32 * TR_W) {
      uint4 v[TR_W];
#pragma unroll
      for (int q = 0; q < TR_W; ++q)
        v[q] = w + 32 * q + lane < sh.words
                   ? st[w + 32 * q]
                   : make_uint4(Tr::NEG_WORD, Tr::NEG_WORD, Tr::NEG_WORD, Tr::NEG_WORD);
#pragma unroll
      for (int q = 0; q < TR_W; ++q) {
        float m = Tr::gmax(v[q]), u = fminf(t1, m);
        t1 = fmaxf(t1, m);
        m = u;
        u = fminf(t2, m);
        t2 = fmaxf(t2, m);
        m = u;
        u = fminf(t3, m);
        t3 = fmaxf(t3, m);
        t4 = fmaxf(t4, u);
      }
      top_words<T>(ref, S, v, a.c2, w == 0);
    }
    top_join(make_float2(ref, S.x + S.y), ref, R);
    if (sh.head + sh.tail > 0) top_ends(x_end, a.c2, ref, R);
    int32_t* const ids = out_ids + row * k;
    float* const logp = a.logp + row * k;
    const float best = warp_max(t1), K = best * a.c2;
    if (!(best < big) || !(best > -big) || !(R >= 0.f) || !(R < INFINITY)) {
      for (int j = lane; j < k; j += 32) {
        ids[j] = -1;
        logp[j] = NAN;
      }
      if (lane == 0) atomicOr(a.ctx_flags, FLAG_NONFINITE);
      __syncwarp();
      continue;
    }
    // ---- the bound: the k-th largest of those, from the first bit on
    const uint32_t o1 = ord(t1), o2 = ord(t2), o3 = ord(t3), o4 = ord(t4);
    uint32_t reach = 0u;
#pragma unroll
    for (int b = 31; b >= (sizeof(T) == 2 ? 16 : 0); --b) {
      const uint32_t c = reach | 1u << b;
      const int n = __popc(__ballot_sync(FULL, o1 >= c)) + __popc(__ballot_sync(FULL, o2 >= c)) +
                    __popc(__ballot_sync(FULL, o3 >= c)) + __popc(__ballot_sync(FULL, o4 >= c));
      if (n >= k) reach = c;
    }
    // (fewer than k finite ones: the bound is below all)
    const float bound = reach > ord(-big) ? unord(reach) : -big;
    auto reaches = [&](float x) { return x >= bound && x > -big; };
    // ---- the elements that reach it
    TopList l(sm.buf[warp], k);
    for (int32_t w = 0; w < sh.words; w += 32) {
      const bool in = w + lane < sh.words;
      const uint4 q =
          in ? st[w] : make_uint4(Tr::NEG_WORD, Tr::NEG_WORD, Tr::NEG_WORD, Tr::NEG_WORD);
      if (!__any_sync(FULL, reaches(Tr::gmax(q)))) continue;
      uint32_t on = 0u;  // a bit per element
#pragma unroll
      for (int j = 0; j < Tr::VEC; ++j) on |= reaches(Tr::at(q, j)) ? 1u << j : 0u;
      while (__any_sync(FULL, on != 0u)) {
        const int j = __ffs(on) - 1;
        float x = -INFINITY;
#pragma unroll
        for (int i = 0; i < Tr::VEC; ++i)
          if (i == j) x = Tr::at(q, i);
        l.push(on != 0u, top_key(x, (uint32_t)(sh.head + (w + lane) * Tr::VEC + j)), lane);
        on &= on - 1u;
      }
    }
    if (sh.head + sh.tail > 0)
      l.push(v_end >= 0 && reaches(x_end), top_key(x_end, (uint32_t)v_end), lane);
    l.finish(lane);
    const float log_sum = top_log(ref, R, K);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int j = 32 * h + lane;
      const uint64_t q = h == 0 ? l.hi : l.lo;
      if (j < k) {
        ids[j] = q ? (int32_t)key_idx(q) : -1;
        logp[j] = q ? top_logp(key_val(q), a.c2, K, log_sum) : -INFINITY;
      }
    }
    __syncwarp();  // every lane has read what the next row is written over
  }
}

}  // namespace prk
