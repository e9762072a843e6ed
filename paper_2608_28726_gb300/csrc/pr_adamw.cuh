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
// update), an m of 6e-5.  All products, roots and roundings of the states are IEEE single
// operations in the order written, so that the codes do not depend on how a compiler
// contracts them.
#pragma once

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
  int32_t wide;     // every pointer fits the 8-element accesses
  int64_t block0;   // blocks of the tensors before it in the caller's list
};

template <int N>
struct AdamwArgs {
  AdamwEntry t[N];
  int32_t chunk0[N + 1];  // first chunk of each tensor; a chunk is AW_NW * per_warp blocks
  int32_t count, per_warp;
  float lr, eps, b1, c1, b2, c2, ibc1, ibc2;  // c = 1 - b, ibc = 1 / (1 - b^t)
  const float* grad_scale;
  float *m_out, *v_out;  // expansion: [blocks][256]
  uint32_t* ctx_flags;
};

// ---- eight elements of a lane ---------------------------------------------------------

__device__ __forceinline__ void get8(const float* p, float (&x)[8]) {
  asm volatile("ld.global.L1::no_allocate.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]),
                 "=f"(x[6]), "=f"(x[7])
               : "l"(p));
}
__device__ __forceinline__ void get8(const __nv_bfloat16* p, float (&x)[8]) {
  uint32_t w[4];
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
               : "l"(p));
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[2 * j] = __uint_as_float(w[j] << 16);
    x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
  }
}
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
__device__ __forceinline__ float get1(const float* p) { return *p; }
__device__ __forceinline__ float get1(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void set1(float* p, float x) { *p = x; }
__device__ __forceinline__ void set1(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// A block's lane: the elements at + j (wide) or at + 32 j, of which those before n exist.
template <typename T>
__device__ __forceinline__ void get(const T* p, int64_t at, bool wide, int left, float (&x)[8]) {
  if (wide) {
    get8(p + at, x);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = 32 * j < left ? get1(p + at + 32 * j) : 0.f;
  }
}
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
__device__ __forceinline__ void get_codes(const uint8_t* p, int64_t at, bool wide, int left,
                                          uint8_t (&q)[8]) {
  if (wide) {
    const uint2 w = *reinterpret_cast<const uint2*>(p + at);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      q[j] = (uint8_t)(w.x >> (8 * j));
      q[4 + j] = (uint8_t)(w.y >> (8 * j));
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = 32 * j < left ? p[at + 32 * j] : (uint8_t)0;
  }
}
__device__ __forceinline__ void set_codes(uint8_t* p, int64_t at, bool wide, int left,
                                          const int (&q)[8]) {
  if (wide) {
    uint2 w = make_uint2(0u, 0u);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w.x |= (uint32_t)(q[j] & 255) << (8 * j);
      w.y |= (uint32_t)(q[4 + j] & 255) << (8 * j);
    }
    *reinterpret_cast<uint2*>(p + at) = w;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (32 * j < left) p[at + 32 * j] = (uint8_t)(q[j] & 255);
  }
}

// ---- 8-bit states ---------------------------------------------------------------------

__device__ __forceinline__ float held_m(uint8_t code, float unit) {
  const float q = (float)(int8_t)code;
  return __fmul_rn(__fmul_rn(q, fabsf(q)), unit);
}
__device__ __forceinline__ float held_v(uint8_t code, float unit) {
  float q = (float)code;
  q = __fmul_rn(q, q);
  return __fmul_rn(__fmul_rn(q, q), unit);
}
constexpr float UNIT_M = (float)(1.0 / (127.0 * 127.0));
constexpr float UNIT_V = (float)(1.0 / (255.0 * 255.0 * 255.0 * 255.0));

// the block's largest magnitude (bit patterns of non-negative floats are ordered, NaN
// above all), as its scale: NaN where it is not finite, 0 below the normal numbers
__device__ __forceinline__ float block_top(const float (&x)[8]) {
  uint32_t t = 0u;
#pragma unroll
  for (int j = 0; j < 8; ++j) t = max(t, __float_as_uint(x[j]) & 0x7fffffffu);
  const float top = __uint_as_float(__reduce_max_sync(FULL, t));
  if (!(top < INFINITY)) return NAN;
  return top >= 1.175494351e-38f ? top : 0.f;
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

template <typename P, typename G, bool MASTER, int BITS, int N>
__global__ void __launch_bounds__(AW_NT) adamw_step(const __grid_constant__ AdamwArgs<N> a) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int k = find_tensor(a, (int32_t)blockIdx.x);
  const AdamwEntry& t = a.t[k];
  const float gs = a.grad_scale ? __ldcg(a.grad_scale) : 1.f;
  const int64_t first = ((int64_t)blockIdx.x - a.chunk0[k]) * (AW_NW * a.per_warp) + warp;
  for (int i = 0; i < a.per_warp; ++i) {
    const int64_t block = first + (int64_t)i * AW_NW, e0 = block * AW_BLOCK;
    if (e0 >= t.n) return;
    const bool wide = t.wide && e0 + AW_BLOCK <= t.n;
    const int64_t at = e0 + (wide ? 8 * lane : lane);
    const int left = wide ? AW_BLOCK : (int)min((int64_t)AW_BLOCK, t.n - e0) - lane;
    P* pp = reinterpret_cast<P*>(t.p);
    float p[8], g[8], m[8], v[8];
    if (MASTER) get(t.master, at, wide, left, p);
    else get(pp, at, wide, left, p);
    get(reinterpret_cast<const G*>(t.g), at, wide, left, g);
    if (BITS == 32) {
      get(reinterpret_cast<const float*>(t.m), at, wide, left, m);
      get(reinterpret_cast<const float*>(t.v), at, wide, left, v);
    } else {
      uint8_t qm[8], qv[8];
      get_codes(reinterpret_cast<const uint8_t*>(t.m), at, wide, left, qm);
      get_codes(reinterpret_cast<const uint8_t*>(t.v), at, wide, left, qv);
      const float um = __fmul_rn(t.ms[block], UNIT_M), uv = __fmul_rn(t.vs[block], UNIT_V);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        m[j] = held_m(qm[j], um);
        v[j] = held_v(qv[j], uv);
      }
      if (!wide)  // what lies past the tensor's end is 0 even under a scale of NaN
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (32 * j >= left) m[j] = v[j] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float x = __fmul_rn(g[j], gs);
      m[j] = __fadd_rn(__fmul_rn(m[j], a.b1), __fmul_rn(x, a.c1));
      v[j] = __fadd_rn(__fmul_rn(v[j], a.b2), __fmul_rn(__fmul_rn(x, x), a.c2));
      const float by = (m[j] * a.ibc1) / (sqrtf(v[j] * a.ibc2) + a.eps) + t.wd * p[j];
      p[j] = fmaf(-a.lr, by, p[j]);
    }
    if (MASTER) set(t.master, at, wide, left, p);
    set(pp, at, wide, left, p);
    if (BITS == 32) {
      set(reinterpret_cast<float*>(t.m), at, wide, left, m);
      set(reinterpret_cast<float*>(t.v), at, wide, left, v);
    } else {
      const float tm = block_top(m), tv = block_top(v);
      const float im = tm > 0.f ? __fdiv_rn(1.f, tm) : 0.f, iv = tv > 0.f ? __fdiv_rn(1.f, tv) : 0.f;
      int qm[8], qv[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int c = __float2int_rn(__fmul_rn(__fsqrt_rn(__fmul_rn(fabsf(m[j]), im)), 127.f));
        qm[j] = m[j] < 0.f ? -c : c;
        qv[j] = __float2int_rn(
            __fmul_rn(__fsqrt_rn(__fsqrt_rn(__fmul_rn(v[j], iv))), 255.f));
      }
      set_codes(reinterpret_cast<uint8_t*>(t.m), at, wide, left, qm);
      set_codes(reinterpret_cast<uint8_t*>(t.v), at, wide, left, qv);
      if (lane == 0) {
        t.ms[block] = tm;
        t.vs[block] = tv;
        if (isnan(tm) || isnan(tv)) atomicOr(a.ctx_flags, FLAG_NONFINITE);
      }
    }
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
    uint8_t qm[8], qv[8];
    get_codes(reinterpret_cast<const uint8_t*>(t.m), at, wide, left, qm);
    get_codes(reinterpret_cast<const uint8_t*>(t.v), at, wide, left, qv);
    const float um = __fmul_rn(t.ms[block], UNIT_M), uv = __fmul_rn(t.vs[block], UNIT_V);
    float m[8], v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool in = wide || 32 * j < left;
      m[j] = in ? held_m(qm[j], um) : 0.f;
      v[j] = in ? held_v(qv[j], uv) : 0.f;
    }
    // the output's blocks are whole
    const int64_t to = (t.block0 + block) * AW_BLOCK + (wide ? 8 * lane : lane);
    set(a.m_out, to, wide, AW_BLOCK, m);
    set(a.v_out, to, wide, AW_BLOCK, v);
  }
}

}  // namespace prk
