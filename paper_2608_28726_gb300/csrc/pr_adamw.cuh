// AdamW over many tensors in one launch.
//
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
//   p = p - lr ((m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps) + wd p)
//
// A tensor is cut into blocks of 256 elements, one per warp, eight neighbouring
// elements to a lane (32-byte loads and stores).  With 8-bit states a block is also
// what shares a scale: the warp expands the codes, steps, takes the block's
// largest |m| and v, and writes codes and scales again; the parameters step with the
// new states before their rounding.
//   m: q = round(127 sqrt(|m| / max)) with m's sign, held value q |q| max / 127^2
//   v: q = round(255 (v / max)^(1/4)),               held value q^4 max / 255^4
// Equal steps of the root put the codes where the values are: a v of 4e-9 of the
// block's largest still has a code of its own (its square root divides the
// update), an m of 6e-5.  All products, sums and roundings of the states are IEEE single
// operations in the order written, so that the states do not depend on how a compiler
// contracts them, and the codes are those of IEEE roots (codes_of).  The parameters'
// update takes approximate roots and reciprocals (EPS_FAST).
#pragma once

#include <type_traits>

#include "pr_device.cuh"

namespace prk {

constexpr int AW_BLOCK = 256;  // elements of a block
constexpr int AW_NT = 256;     // a CTA's threads
constexpr int AW_NW = AW_NT / 32;
constexpr int AW_FEW = 32, AW_MANY = 384;  // tensors of a launch (kernel parameters: 32,764 bytes)

struct AdamwEntry {
  void* p;
  const void* g;
  float* master;
  void* m;
  void* v;
  float* ms;
  float* vs;
  int64_t n;
  float wd;
  int32_t wide;     // every pointer fits the 8-element accesses (the step's codes: 16)
  int64_t block0;   // blocks of the tensors before it in the caller's list
};

template <int N>
struct AdamwArgs {
  AdamwEntry t[N];
  int32_t chunk0[N + 1];  // first chunk of each tensor; a chunk is AW_NW * per_warp blocks
  int32_t count, per_warp;
  float lr, eps, b1, c1, b2, c2, ibc1, ibc2, root_ibc2;  // c = 1 - b, ibc = 1 / (1 - b^t)
  float one;              // 1: see sum2
  const float* grad_scale;
  float *m_out, *v_out;  // expansion: [blocks][256]
  uint32_t* ctx_flags;
};

// a + b, two at a time, where a or b is a product that has to be rounded by itself: a
// packed product and sum become one operation in the compiler, whatever rounding they ask
// for.  `one` is 1, unknown to it.
__device__ __forceinline__ float2 sum2(float2 a, float2 b, float one) {
  return __ffma2_rn(a, make_float2(one, one), b);
}

// ---- eight elements of a lane ---------------------------------------------------------
//
// In a block that lies in the tensor whole, of pointers on a grid of eight elements: eight
// neighbours from element `at` on (wide).  Else those at + 32 j, of which the first
// `left` after `at` exist.

template <typename T>
struct Raw {
  static constexpr int WORDS = 2 * sizeof(T);
  uint32_t w[WORDS];
  __device__ __forceinline__ void load(const void* from, int64_t at, bool wide, int left) {
    const T* p = reinterpret_cast<const T*>(from) + at;
    if (wide) {
      if constexpr (WORDS == 8)
        asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]),
                       "=r"(w[6]), "=r"(w[7])
                     : "l"(p));
      else if constexpr (WORDS == 4)
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                     : "l"(p));
      else
        asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];"
                     : "=r"(w[0]), "=r"(w[1])
                     : "l"(p));
    } else {
#pragma unroll
      for (int j = 0; j < WORDS; ++j) w[j] = 0u;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (32 * j < left) {
          if constexpr (sizeof(T) == 4)
            w[j] = reinterpret_cast<const uint32_t*>(p)[32 * j];
          else if constexpr (sizeof(T) == 2)
            w[j >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[32 * j] << (16 * (j & 1));
          else
            w[j >> 2] |= (uint32_t)p[32 * j] << (8 * (j & 3));
        }
    }
  }
  __device__ __forceinline__ void expand(float (&x)[8]) const {  // (of numbers, not codes)
    if constexpr (WORDS == 8) {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(w[j]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[2 * j] = __uint_as_float(w[j] << 16);
        x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
      }
    }
  }
};

__device__ __forceinline__ void set8(float* p, const float (&x)[8]) {
  asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(x[0]), "f"(x[1]),
               "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7])
               : "memory");
}
__device__ __forceinline__ void set8(__nv_bfloat16* p, const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const __nv_bfloat162 h = __float22bfloat162_rn(make_float2(x[2 * j], x[2 * j + 1]));
    w[j] = *reinterpret_cast<const uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void set1(float* p, float x) { *p = x; }
__device__ __forceinline__ void set1(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
template <typename T>
__device__ __forceinline__ void set(T* p, int64_t at, bool wide, int left, const float (&x)[8]) {
  if (wide) {
    set8(p + at, x);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (32 * j < left) set1(p + at + 32 * j, x[j]);
  }
}
__device__ __forceinline__ void set_codes(uint8_t* p, int64_t at, bool wide, int left,
                                          const uint2& q) {
  if (wide) {
    *reinterpret_cast<uint2*>(p + at) = q;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (32 * j < left) p[at + 32 * j] = (uint8_t)((j < 4 ? q.x : q.y) >> (8 * (j & 3)));
  }
}

// ---- 8-bit states ---------------------------------------------------------------------

// Byte j of w over 2^K as a float: into the last byte of a significand whose last place counts
// 2^-K, and the rest of that number away again.  `bias` more goes with it: signed codes come
// with their top bit turned, 128 too much.
template <int K>
__device__ __forceinline__ float byte_of(uint32_t w, int j, float bias) {
  constexpr uint32_t BASE = (uint32_t)(127 + 23 - K) << 23;
  constexpr float SIZE = (float)(1 << (23 - K)), LAST = 1.f / (float)(1 << K);
  return __uint_as_float(__byte_perm(w, BASE, 0x7640 + j)) - (SIZE + bias * LAST);
}
// What the codes of a word's half (bytes j, j + 1) stand for; unit: the scale's share.  The
// codes are taken over 2^6 and 2^7, exactly, so that the unit is a quarter and a sixteenth
// of the scale, not 1 / 127^2 and 1 / 255^4 of it, which small scales have no normal number
// for.
constexpr int M_K = 6, V_K = 7;
__device__ __forceinline__ float2 held_m(uint32_t w, int j, float unit) {
  w ^= 0x80808080u;
  const float a = byte_of<M_K>(w, j, 128.f), b = byte_of<M_K>(w, j + 1, 128.f);
  return __fmul2_rn(make_float2(__fmul_rn(a, fabsf(a)), __fmul_rn(b, fabsf(b))),
                    make_float2(unit, unit));
}
__device__ __forceinline__ float2 held_v(uint32_t w, int j, float unit) {
  float2 q = make_float2(byte_of<V_K>(w, j, 0.f), byte_of<V_K>(w, j + 1, 0.f));
  q = __fmul2_rn(q, q);
  return __fmul2_rn(__fmul2_rn(q, q), make_float2(unit, unit));
}
constexpr float UNIT_M = (float)(4096.0 / (127.0 * 127.0));                      // 2^(2 M_K)
constexpr float UNIT_V = (float)(268435456.0 / (255.0 * 255.0 * 255.0 * 255.0));  // 2^(4 V_K)

// the block's largest magnitude as its scale (bit patterns of non-negative floats are
// ordered, NaN above all): NaN where it is not finite, 0 below the normal numbers
__device__ __forceinline__ float block_top(const float2 (&x)[4]) {
  float t = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(t) : "f"(fabsf(x[j].x)));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(t) : "f"(fabsf(x[j].y)));
  }
  const float top = __uint_as_float(__reduce_max_sync(FULL, __float_as_uint(t)));
  if (!(top < INFINITY)) return NAN;
  return top >= 1.175494351e-38f ? top : 0.f;
}
__device__ __forceinline__ float sqrt_fast(float x) {
  float y;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_fast(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// From this eps on m / (sqrt(v) + eps) takes approximate roots and reciprocals (within
// 2^-21): subnormal numbers taken for 0 then have roots far below eps.
constexpr float EPS_FAST = 1e-12f;
// The codes round(STEPS r) of ratios' roots r = sqrt(x) (ROOTS = 1) or x^(1/4) (2), x
// already divided by the scale, in the last bytes of q.  The definition takes IEEE roots;
// approximate ones (within 2^-22) give the same code unless STEPS r lies within 255 x 2^-21
// of the middle between two, which the whole warp then looks up exactly (one block in
// ten).  45% fewer instructions than with IEEE roots throughout.
// With ROOTS = 1 they take the signs of `m`.  `rooted`: x, or with ROOTS = 2 its root.
template <int ROOTS, typename Rooted>
__device__ __forceinline__ void codes_of(const float2 (&x)[4], const float2 (&m)[4], Rooted rooted,
                                         uint32_t (&q)[8]) {
  constexpr float STEPS = ROOTS == 1 ? 127.f : 255.f;
  constexpr float MAGIC = 12582912.f;  // 1.5 x 2^23: a sum's last bits are the rounded addend
  float off = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float2 r = rooted(j);
    r = make_float2(sqrt_fast(r.x), sqrt_fast(r.y));
    if (ROOTS == 1) r = make_float2(copysignf(r.x, m[j].x), copysignf(r.y, m[j].y));
    const float2 steps = make_float2(STEPS, STEPS);
    const float2 t = __ffma2_rn(r, steps, make_float2(MAGIC, MAGIC));
    const float2 w = __fadd2_rn(make_float2(MAGIC, MAGIC), make_float2(-t.x, -t.y));
    q[2 * j] = __float_as_uint(t.x);
    q[2 * j + 1] = __float_as_uint(t.y);
    const float2 d = __ffma2_rn(r, steps, w);
    off = fmaxf(off, fmaxf(fabsf(d.x), fabsf(d.y)));
  }
  if (__any_sync(FULL, off > 0.49987f)) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float r = __fsqrt_rn(j & 1 ? x[j >> 1].y : x[j >> 1].x);
      if (ROOTS == 2) r = __fsqrt_rn(r);
      if (ROOTS == 1) r = copysignf(r, j & 1 ? m[j >> 1].y : m[j >> 1].x);
      q[j] = (uint32_t)__float2int_rn(__fmul_rn(r, STEPS));
    }
  }
}
__device__ __forceinline__ uint2 pack_codes(const uint32_t (&q)[8]) {
  auto four = [](uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
  };
  return make_uint2(four(q[0], q[1], q[2], q[3]), four(q[4], q[5], q[6], q[7]));
}

// ---- the step -----------------------------------------------------------------------------

template <int N>
__device__ __forceinline__ int find_tensor(const AdamwArgs<N>& a, int32_t chunk) {
  int lo = 0, hi = a.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.chunk0[mid] <= chunk) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// What a warp reads of a block
template <typename P, typename G, bool MASTER, int BITS>
struct BlockIn {
  Raw<typename std::conditional<MASTER, float, P>::type> p;
  Raw<G> g;
  Raw<typename std::conditional<BITS == 32, float, uint8_t>::type> m, v;
  float um, uv;  // units of the codes
};

// A lane's part of block `block` of tensor t
struct BlockAt {
  int64_t at;
  int left;
  __device__ __forceinline__ BlockAt(const AdamwEntry& t, int64_t block, bool wide, int lane) {
    at = block * AW_BLOCK + (wide ? 8 * lane : lane);
    left = wide ? AW_BLOCK : (int)min((int64_t)AW_BLOCK, t.n - block * AW_BLOCK) - lane;
  }
};
template <typename P, typename G, bool MASTER, int BITS>
__device__ __forceinline__ void load_block(BlockIn<P, G, MASTER, BITS>& x, const AdamwEntry& t,
                                           int64_t block, bool wide, int lane) {
  const BlockAt b(t, block, wide, lane);
  if (MASTER) x.p.load(t.master, b.at, wide, b.left);
  else x.p.load(t.p, b.at, wide, b.left);
  x.g.load(t.g, b.at, wide, b.left);
  x.m.load(t.m, b.at, wide, b.left);
  x.v.load(t.v, b.at, wide, b.left);
  if (BITS == 8) {
    x.um = t.ms[block];
    x.uv = t.vs[block];
  }
}
template <typename P, typename G, bool MASTER, int BITS, int N>
__device__ __forceinline__ void step_block(const BlockIn<P, G, MASTER, BITS>& in,
                                           const AdamwArgs<N>& a, const AdamwEntry& t, float gs,
                                           int64_t block, bool wide, int lane) {
  const BlockAt b(t, block, wide, lane);
  float p[8], g[8];
  float2 m[4], v[4];
  in.p.expand(p);
  in.g.expand(g);
  if constexpr (BITS == 32) {
    in.m.expand(reinterpret_cast<float(&)[8]>(m));
    in.v.expand(reinterpret_cast<float(&)[8]>(v));
  } else {
    const float um = __fmul_rn(in.um, UNIT_M), uv = __fmul_rn(in.uv, UNIT_V);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m[j] = held_m(in.m.w[j >> 1], 2 * (j & 1), um);
      v[j] = held_v(in.v.w[j >> 1], 2 * (j & 1), uv);
    }
    if (!wide)  // what lies past the tensor's end is 0 even under a scale of NaN
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (64 * j >= b.left) m[j].x = v[j].x = 0.f;
        if (64 * j + 32 >= b.left) m[j].y = v[j].y = 0.f;
      }
  }
  auto both = [](float x) { return make_float2(x, x); };
  float2 roots[4];  // of v
  auto update = [&](auto quotient) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 x = __fmul2_rn(make_float2(g[2 * j], g[2 * j + 1]), both(gs));
      m[j] = sum2(__fmul2_rn(m[j], both(a.b1)), __fmul2_rn(x, both(a.c1)), a.one);
      v[j] = sum2(__fmul2_rn(v[j], both(a.b2)), __fmul2_rn(__fmul2_rn(x, x), both(a.c2)), a.one);
      const float2 mh = __fmul2_rn(m[j], both(a.ibc1));
      float2 q = make_float2(p[2 * j], p[2 * j + 1]);
      const float2 by = __ffma2_rn(both(t.wd), q, quotient(mh, j));
      q = __ffma2_rn(both(-a.lr), by, q);
      p[2 * j] = q.x;
      p[2 * j + 1] = q.y;
    }
  };
  const bool fast = a.eps >= EPS_FAST;
  if (fast)
    update([&](const float2& mh, int j) {
      roots[j] = make_float2(sqrt_fast(v[j].x), sqrt_fast(v[j].y));
      const float2 d = __ffma2_rn(roots[j], both(a.root_ibc2), both(a.eps));
      return __fmul2_rn(mh, make_float2(rcp_fast(d.x), rcp_fast(d.y)));
    });
  else
    update([&](const float2& mh, int j) {
      const float2 vh = __fmul2_rn(v[j], both(a.ibc2));
      return make_float2(mh.x / (sqrtf(vh.x) + a.eps), mh.y / (sqrtf(vh.y) + a.eps));
    });
  if (MASTER) set(t.master, b.at, wide, b.left, p);
  set(reinterpret_cast<P*>(t.p), b.at, wide, b.left, p);
  if constexpr (BITS == 32) {
    set(reinterpret_cast<float*>(t.m), b.at, wide, b.left, reinterpret_cast<float(&)[8]>(m));
    set(reinterpret_cast<float*>(t.v), b.at, wide, b.left, reinterpret_cast<float(&)[8]>(v));
  } else {
    const float tm = block_top(m), tv = block_top(v);
    // both reciprocals by one division: m's in the even lanes
    const float top = lane & 1 ? tv : tm, inv = top > 0.f ? __fdiv_rn(1.f, top) : 0.f;
    const float im = __shfl_sync(FULL, inv, 0), iv = __shfl_sync(FULL, inv, 1);
    uint32_t q[8];
    float2 x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      x[j] = __fmul2_rn(make_float2(fabsf(m[j].x), fabsf(m[j].y)), both(im));
    codes_of<1>(x, m, [&](int j) { return x[j]; }, q);
    uint2 c = pack_codes(q);
    if (isnan(tm)) c = make_uint2(0u, 0u);
    set_codes(reinterpret_cast<uint8_t*>(t.m), b.at, wide, b.left, c);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = __fmul2_rn(v[j], both(iv));
    // v's roots are there; those of subnormal numbers, taken for 0, have code 0 next to 1e-26,
    // and above 2^126 the scale's reciprocal would be taken for 0
    if (fast && tv > 1e-26f && tv < 8.5e37f) {
      const float by = sqrt_fast(iv);
      codes_of<2>(x, m, [&](int j) { return __fmul2_rn(roots[j], both(by)); }, q);
    } else {
      codes_of<2>(x, m, [&](int j) { return make_float2(sqrt_fast(x[j].x), sqrt_fast(x[j].y)); }, q);
    }
    c = pack_codes(q);
    if (isnan(tv)) c = make_uint2(0u, 0u);
    set_codes(reinterpret_cast<uint8_t*>(t.v), b.at, wide, b.left, c);
    if (lane < 2) (lane ? t.vs : t.ms)[block] = top;
    if (isnan(top) && lane < 2) atomicOr(a.ctx_flags, FLAG_NONFINITE);
  }
}

// With 8-bit states a block's arithmetic takes as long as its data: each warp has those of
// the next AW_STAGES - 1 blocks on their way into shared memory meanwhile.  (155 M bf16
// parameters: 295 us, 380 with the next block's data in registers, 433 with none; 287 since
// the update and the codes share v's roots.  The arithmetic, some 55 instructions per
// element, bounds it there: issue slots 72% busy, DRAM 61%; four CTAs on an SM, with spills,
// gain 1% there and lose 2% in fp32.  Memory bounds 134 M fp32 ones: 310 us, 2.1 GB.)
constexpr int AW_STAGES = 3;
template <typename P, typename G, bool MASTER>
struct Staged {
  using In = BlockIn<P, G, MASTER, 8>;
  static constexpr int PW = sizeof(In::p) / 16, GW = sizeof(In::g) / 16;  // 16-byte words
  static constexpr int WORDS = PW + GW + 1;                               // and the codes
  static constexpr size_t BYTES = (size_t)AW_STAGES * AW_NT * WORDS * 16;
};
__device__ __forceinline__ void copy_async(uint4* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(
                   (uint32_t)__cvta_generic_to_shared(to)),
               "l"(from)
               : "memory");
}
template <typename P, typename G, bool MASTER, int BITS, int N>
__global__ void __launch_bounds__(AW_NT, 3)
    adamw_step(const __grid_constant__ AdamwArgs<N> a) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int k = find_tensor(a, (int32_t)blockIdx.x);
  const AdamwEntry t = a.t[k];
  const float gs = a.grad_scale ? __ldcg(a.grad_scale) : 1.f;
  int64_t block = ((int64_t)blockIdx.x - a.chunk0[k]) * (AW_NW * a.per_warp) + warp;
  const int64_t blocks = min((t.n + AW_BLOCK - 1) / AW_BLOCK, block - warp + AW_NW * a.per_warp);
  const int64_t whole = t.wide ? min(t.n / AW_BLOCK, blocks) : 0;
  if constexpr (BITS == 8) {
    using St = Staged<P, G, MASTER>;
    using PT = typename std::conditional<MASTER, float, P>::type;
    // a warp's words of a stage: parameters, gradients, m's codes, v's codes
    uint4* const mine = reinterpret_cast<uint4*>(smem_raw) + warp * (AW_STAGES * St::WORDS * 32);
    const int64_t e0 = block * AW_BLOCK;
    const uint4* gp = reinterpret_cast<const uint4*>(
        (MASTER ? reinterpret_cast<const PT*>(t.master) : reinterpret_cast<const PT*>(t.p)) + e0) + lane;
    const uint4* gg = reinterpret_cast<const uint4*>(reinterpret_cast<const G*>(t.g) + e0) + lane;
    const uint4* gc = reinterpret_cast<const uint4*>(
        reinterpret_cast<const uint8_t*>(lane < 16 ? t.m : t.v) + e0) + (lane & 15);
    constexpr int STEP = AW_NW * AW_BLOCK;  // elements from one block to this warp's next
    int64_t ahead = block;
    int into = 0, from = 0;
    auto bring = [&]() {
      if (ahead < whole) {
        uint4* to = mine + into * (St::WORDS * 32) + lane;
#pragma unroll
        for (int j = 0; j < St::PW; ++j) copy_async(to + 32 * j, gp + 32 * j);
#pragma unroll
        for (int j = 0; j < St::GW; ++j) copy_async(to + 32 * (St::PW + j), gg + 32 * j);
        copy_async(to + 32 * (St::PW + St::GW), gc);
        gp += STEP * sizeof(PT) / 16;
        gg += STEP * sizeof(G) / 16;
        gc += STEP / 16;
        ahead += AW_NW;
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
      into = into + 1 == AW_STAGES ? 0 : into + 1;
    };
#pragma unroll
    for (int j = 0; j < AW_STAGES - 1; ++j) bring();
    // the scales of 16 blocks at a time: m's in the lower lanes, v's in the upper ones
    float scales = 0.f;
    int of = 16;
    for (; block < whole; block += AW_NW) {
      if (of == 16) {
        of = 0;
        const int64_t q = block + (int64_t)(lane & 15) * AW_NW;
        if (q < whole) scales = lane < 16 ? t.ms[q] : t.vs[q];
      }
      __syncwarp();  // every lane has read what is written next
      bring();
      asm volatile("cp.async.wait_group %0;" ::"n"(AW_STAGES - 1) : "memory");
      __syncwarp();  // every lane's copies are there
      typename St::In in;
      const uint4* st = mine + from * (St::WORDS * 32);
      auto words = [&](auto& raw, const uint4* q) {
#pragma unroll
        for (int j = 0; j < (int)sizeof(raw) / 16; ++j) {
          const uint4 w = q[j];
          raw.w[4 * j] = w.x, raw.w[4 * j + 1] = w.y, raw.w[4 * j + 2] = w.z, raw.w[4 * j + 3] = w.w;
        }
      };
      words(in.p, st + St::PW * lane);
      words(in.g, st + 32 * St::PW + St::GW * lane);
      const uint2* codes = reinterpret_cast<const uint2*>(st + 32 * (St::PW + St::GW)) + lane;
      in.m.w[0] = codes[0].x, in.m.w[1] = codes[0].y;
      in.v.w[0] = codes[32].x, in.v.w[1] = codes[32].y;
      in.um = __shfl_sync(FULL, scales, of);
      in.uv = __shfl_sync(FULL, scales, 16 + of);
      ++of;
      from = from + 1 == AW_STAGES ? 0 : from + 1;
      step_block(in, a, t, gs, block, true, lane);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (block < whole) {
    BlockIn<P, G, MASTER, BITS> in;
    for (; block < whole; block += AW_NW) {
      load_block(in, t, block, true, lane);
      step_block(in, a, t, gs, block, true, lane);
    }
  }
  for (; block < blocks; block += AW_NW) {
    BlockIn<P, G, MASTER, BITS> in;
    load_block(in, t, block, false, lane);
    step_block(in, a, t, gs, block, false, lane);
  }
}

// The values that 8-bit states stand for.
template <int N>
__global__ void __launch_bounds__(AW_NT) adamw_unpack(const __grid_constant__ AdamwArgs<N> a) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int k = find_tensor(a, (int32_t)blockIdx.x);
  const AdamwEntry& t = a.t[k];
  const int64_t first = ((int64_t)blockIdx.x - a.chunk0[k]) * (AW_NW * a.per_warp) + warp;
  for (int i = 0; i < a.per_warp; ++i) {
    const int64_t block = first + (int64_t)i * AW_NW, e0 = block * AW_BLOCK;
    if (e0 >= t.n) return;
    const bool wide = t.wide && e0 + AW_BLOCK <= t.n;
    const int64_t at = e0 + (wide ? 8 * lane : lane);
    const int left = wide ? AW_BLOCK : (int)min((int64_t)AW_BLOCK, t.n - e0) - lane;
    Raw<uint8_t> qm, qv;
    qm.load(t.m, at, wide, left);
    qv.load(t.v, at, wide, left);
    const float um = __fmul_rn(t.ms[block], UNIT_M), uv = __fmul_rn(t.vs[block], UNIT_V);
    float m[8], v[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 x = held_m(qm.w[j >> 1], 2 * (j & 1), um);
      const float2 y = held_v(qv.w[j >> 1], 2 * (j & 1), uv);
      const bool in0 = wide || 64 * j < left, in1 = wide || 64 * j + 32 < left;
      m[2 * j] = in0 ? x.x : 0.f;
      m[2 * j + 1] = in1 ? x.y : 0.f;
      v[2 * j] = in0 ? y.x : 0.f;
      v[2 * j + 1] = in1 ? y.y : 0.f;
    }
    // the output's blocks are whole
    const int64_t to = (t.block0 + block) * AW_BLOCK + (wide ? 8 * lane : lane);
    set(a.m_out, to, wide, AW_BLOCK, m);
    set(a.v_out, to, wide, AW_BLOCK, v);
  }
}

}  // namespace prk
