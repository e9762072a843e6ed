// Layer norm and RMS norm of rows, a residual added first, and the backward pass.
//
//   forward   h = x + r;  m = mean h;  s = 1 / sqrt(mean (h - m)^2 + eps);
//             y = (h - m) s w + b
//   backward  xhat = (h - m) s, g = dy w;  dx = s (g - mean g - xhat mean(g xhat)) + dtotal;
//             dw = sum over rows of dy xhat, db = sum of dy
// RMS norm is the same with m = 0 and without mean g.  A first mean m is off by its sum's
// roundings, which a constant row would have for its deviation; the sum of h - m that comes with
// the variance's corrects both.
#pragma once

#include "pr_device.cuh"

namespace prk {

struct NormArgs {
  const void* x;
  const void* res;      // residual (forward), dtotal (backward), or NULL
  const void* dy;       // backward
  const void* w;
  const void* b;
  void* total;
  void* y;              // y, or dx; NULL: dx is not asked for
  float* mean;
  float* rstd;
  float* dw;
  float* db;
  int64_t n_rows, d;
  int64_t x_stride, res_stride, dy_stride, total_stride, y_stride;
  float eps, inv_d;
  int32_t rms, wide_w;  // wide_w: weights are fp32 (else bf16)
  int32_t accumulate;
  int32_t vec, vec_w;   // rows (weights) begin at multiples of 16 bytes
  float* part;          // workspace: [CTAs][2][d] sums of dy xhat and of dy
};

__device__ __forceinline__ float nm_get(const float* p) { return *p; }
__device__ __forceinline__ float nm_get(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void nm_put(float* p, float v) { *p = v; }
__device__ __forceinline__ void nm_put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
// v as the rows' type holds it
template <typename T>
__device__ __forceinline__ float nm_held(float v) {
  if constexpr (sizeof(T) == 4) return v;
  else return __bfloat162float(__float2bfloat16_rn(v));
}
__device__ __forceinline__ float nm_weight(const void* w, int32_t wide, int64_t i) {
  return wide ? reinterpret_cast<const float*>(w)[i]
              : __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(w)[i]);
}

// 1 / deviation, from the sum of (h - m)^2 where m is `off` short of the mean
__device__ __forceinline__ float nm_rstd(float s, float off, const NormArgs& a) {
  return 1.f / sqrtf(fmaxf(fmaf(s, a.inv_d, -off * off), 0.f) + a.eps);
}

// the sum over a CTA, in every thread
__device__ __forceinline__ float nm_block_sum(float v, float* part) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
  __syncthreads();
  if (lane == 0) part[warp] = v;
  __syncthreads();
  v = lane < warps ? part[lane] : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
  return v;
}

// ---- rows in registers -----------------------------------------------------------------
//
// L threads have a row, N 16-byte words each, and read it once: what the moments and the output
// need stays in registers.  Rows of up to 32 threads are summed by shuffles, wider ones
// through shared memory with a barrier of the row's threads alone, so that the CTA's other rows
// go on meanwhile; enough CTAs are on an SM to keep memory busy.

constexpr int NR_NT = 256;  // threads of a CTA of rows of up to so many

template <typename T>
struct RowWord {
  static constexpr int VEC = 16 / (int)sizeof(T);
  static __device__ __forceinline__ float at(const uint4& w, int j) {
    if constexpr (sizeof(T) == 4) {
      return __uint_as_float(j == 0 ? w.x : j == 1 ? w.y : j == 2 ? w.z : w.w);
    } else {
      const int q = j >> 1;
      const uint32_t u = q == 0 ? w.x : q == 1 ? w.y : q == 2 ? w.z : w.w;
      return __uint_as_float((j & 1) ? (u & 0xffff0000u) : (u << 16));
    }
  }
  static __device__ __forceinline__ uint4 of(const float (&f)[VEC]) {
    uint4 r;
    uint32_t* u = reinterpret_cast<uint32_t*>(&r);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (sizeof(T) == 4) {
        u[q] = __float_as_uint(f[q]);
      } else {
        const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * q], f[2 * q + 1]);
        u[q] = *reinterpret_cast<const uint32_t*>(&h);
      }
    }
    return r;
  }
  // word i of a row of d elements, 0 past its end
  static __device__ __forceinline__ uint4 load(const T* row, int64_t i, int64_t d, bool vec) {
    if (vec && (i + 1) * VEC <= d) return ld_stream(row + i * VEC);
    uint4 r = make_uint4(0u, 0u, 0u, 0u);
    float f[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) f[j] = i * VEC + j < d ? nm_get(row + i * VEC + j) : 0.f;
    if (i * VEC < d) r = of(f);
    return r;
  }
  static __device__ __forceinline__ void store(T* row, int64_t i, int64_t d, bool vec, const float (&f)[VEC]) {
    if (vec && (i + 1) * VEC <= d) {
      *reinterpret_cast<uint4*>(row + i * VEC) = of(f);
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        if (i * VEC + j < d) nm_put(row + i * VEC + j, f[j]);
    }
  }
  // the weights of word i's elements (they stay in L1)
  static __device__ __forceinline__ void weights(const void* w, bool wide, bool vec, int64_t i, int64_t d,
                                                 float (&f)[VEC]) {
    if (vec && (i + 1) * VEC <= d) {
      if (wide) {
#pragma unroll
        for (int q = 0; q < VEC / 4; ++q) {
          const float4 v = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(w) + i * VEC + 4 * q);
          f[4 * q] = v.x;
          f[4 * q + 1] = v.y;
          f[4 * q + 2] = v.z;
          f[4 * q + 3] = v.w;
        }
      } else {
#pragma unroll
        for (int q = 0; q < VEC / 4; ++q) {
          const uint2 v = *reinterpret_cast<const uint2*>(reinterpret_cast<const __nv_bfloat16*>(w) + i * VEC + 4 * q);
          f[4 * q] = __uint_as_float(v.x << 16);
          f[4 * q + 1] = __uint_as_float(v.x & 0xffff0000u);
          f[4 * q + 2] = __uint_as_float(v.y << 16);
          f[4 * q + 3] = __uint_as_float(v.y & 0xffff0000u);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) f[j] = i * VEC + j < d ? nm_weight(w, wide, i * VEC + j) : 0.f;
    }
  }
};

// (a, b) summed over a row's L threads.  `part`: two buffers of a float2 per warp of the CTA, used in turn.
template <int L>
__device__ __forceinline__ float2 nm_row_sum(float2 v, float2 (*part)[32], int turn) {
#pragma unroll
  for (int o = (L < 32 ? L : 32) / 2; o > 0; o >>= 1) {
    v.x += __shfl_xor_sync(FULL, v.x, o);
    v.y += __shfl_xor_sync(FULL, v.y, o);
  }
  if constexpr (L > 32) {
    constexpr int W = L / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = warp / W;
    if (lane == 0) part[turn][warp] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(1 + row), "r"(L) : "memory");
    v = lane < W ? part[turn][row * W + lane] : make_float2(0.f, 0.f);
#pragma unroll
    for (int o = (W > 16 ? 32 : W > 8 ? 16 : W > 4 ? 8 : W > 2 ? 4 : 2) / 2; o > 0; o >>= 1) {
      v.x += __shfl_xor_sync(FULL, v.x, o);
      v.y += __shfl_xor_sync(FULL, v.y, o);
    }
    v.x = __shfl_sync(FULL, v.x, 0);
    v.y = __shfl_sync(FULL, v.y, 0);
  }
  return v;
}

template <typename T, int L, int N>
__global__ void __launch_bounds__(L > NR_NT ? L : NR_NT) norm_rows(const __grid_constant__ NormArgs a) {
  using W = RowWord<T>;
  __shared__ float2 part[2][32];
  pdl_wait();
  pdl_trigger();
  const int rows = blockDim.x / L, in_row = threadIdx.x % L;
  const int64_t d = a.d;
  const bool vec = a.vec, vec_w = a.vec_w, wide = a.wide_w;
  int turn = 0;  // of the sums' buffers
  // (every thread of a warp goes through the sums: the last rows of a CTA may be none)
  for (int64_t r0 = (int64_t)blockIdx.x * rows; r0 < a.n_rows; r0 += (int64_t)gridDim.x * rows) {
    const int64_t row = r0 + threadIdx.x / L;
    const bool on = row < a.n_rows;
    uint4 h[N];
    const T* x = reinterpret_cast<const T*>(a.x) + row * a.x_stride;
#pragma unroll
    for (int i = 0; i < N; ++i)
      h[i] = on ? W::load(x, in_row + (int64_t)i * L, d, vec) : make_uint4(0u, 0u, 0u, 0u);
    if (a.res) {
      const T* res = reinterpret_cast<const T*>(a.res) + row * a.res_stride;
      uint4 r[N];
#pragma unroll
      for (int i = 0; i < N; ++i)
        r[i] = on ? W::load(res, in_row + (int64_t)i * L, d, vec) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float f[W::VEC];
#pragma unroll
        for (int j = 0; j < W::VEC; ++j) f[j] = W::at(h[i], j) + W::at(r[i], j);
        h[i] = W::of(f);
      }
    }
    float m = 0.f;
    if (!a.rms) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < W::VEC; ++j) s += W::at(h[i], j);
      m = nm_row_sum<L>(make_float2(s, 0.f), part, turn).x * a.inv_d;
      turn ^= 1;
    }
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < W::VEC; ++j) {
        const bool in = (in_row + (int64_t)i * L) * W::VEC + j < d;
        const float v = in ? W::at(h[i], j) - m : 0.f;
        s.x = fmaf(v, v, s.x);
        s.y += v;
      }
    s = nm_row_sum<L>(s, part, turn);
    turn ^= 1;
    const float off = a.rms ? 0.f : s.y * a.inv_d, rstd = nm_rstd(s.x, off, a);
    if (on) {
      T* y = reinterpret_cast<T*>(a.y) + row * a.y_stride;
      T* total = reinterpret_cast<T*>(a.total) + row * a.total_stride;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int64_t at = in_row + (int64_t)i * L;
        if (at * W::VEC >= d) continue;
        float w[W::VEC], b[W::VEC], f[W::VEC];
        W::weights(a.w, wide, vec_w, at, d, w);
#pragma unroll
        for (int j = 0; j < W::VEC; ++j) b[j] = 0.f;
        if (a.b) W::weights(a.b, wide, vec_w, at, d, b);
        if (a.total) {
#pragma unroll
          for (int j = 0; j < W::VEC; ++j) f[j] = W::at(h[i], j);
          W::store(total, at, d, vec, f);
        }
#pragma unroll
        for (int j = 0; j < W::VEC; ++j) f[j] = fmaf(((W::at(h[i], j) - m) - off) * rstd, w[j], b[j]);
        W::store(y, at, d, vec, f);
      }
      if (in_row == 0) {
        if (a.mean && !a.rms) a.mean[row] = m + off;
        if (a.rstd) a.rstd[row] = rstd;
      }
    }
  }
}

// The backward pass.  A thread keeps the sums of its columns over all rows of its CTA; the CTA's
// rows are added up in order at the end and go to the workspace, and dnorm_sum adds up the CTAs.
// The next row's words are on their way while one is summed.
template <typename T, int L, int N>
__global__ void __launch_bounds__(L > NR_NT ? L : NR_NT)
    dnorm_rows(const __grid_constant__ NormArgs a) {
  using W = RowWord<T>;
  constexpr int VEC = W::VEC, NT = L > NR_NT ? L : NR_NT, ROWS = NT / L;
  __shared__ float2 part[2][32];
  __shared__ float columns[ROWS > 1 ? NT * N * VEC : 1];
  pdl_wait();
  pdl_trigger();
  const int in_row = threadIdx.x % L, group = threadIdx.x / L;
  const int64_t d = a.d;
  const bool vec = a.vec, vec_w = a.vec_w, wide = a.wide_w, sums = a.part != nullptr;
  float cw[N][VEC], cb[N][VEC];
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < VEC; ++j) cw[i][j] = cb[i][j] = 0.f;
  struct Row {
    uint4 x[N], dy[N];
    float m, rstd;
  };
  auto fetch = [&](int64_t row) {
    Row r;
    const bool on = row < a.n_rows;
    const T* x = reinterpret_cast<const T*>(a.x) + row * a.x_stride;
    const T* dy = reinterpret_cast<const T*>(a.dy) + row * a.dy_stride;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t at = in_row + (int64_t)i * L;
      r.x[i] = on ? W::load(x, at, d, vec) : make_uint4(0u, 0u, 0u, 0u);
      r.dy[i] = on ? W::load(dy, at, d, vec) : make_uint4(0u, 0u, 0u, 0u);
    }
    r.m = on && !a.rms ? __ldcg(a.mean + row) : 0.f;
    r.rstd = on ? __ldcg(a.rstd + row) : 0.f;
    return r;
  };
  const int64_t step = (int64_t)gridDim.x * ROWS;
  int64_t r0 = (int64_t)blockIdx.x * ROWS;
  int turn = 0;
  Row r = fetch(r0 + group);
  for (; r0 < a.n_rows; r0 += step, turn ^= 1) {
    const int64_t row = r0 + group;
    const bool on = row < a.n_rows;
    const Row next = fetch(row + step);
    uint4 t[N];
    if (a.res && a.y) {
      const T* res = reinterpret_cast<const T*>(a.res) + row * a.res_stride;
#pragma unroll
      for (int i = 0; i < N; ++i)
        t[i] = on ? W::load(res, in_row + (int64_t)i * L, d, vec) : make_uint4(0u, 0u, 0u, 0u);
    }
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t at = in_row + (int64_t)i * L;
      float w[VEC];
      W::weights(a.w, wide, vec_w, at, d, w);
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float dy = W::at(r.dy[i], j), hat = (W::at(r.x[i], j) - r.m) * r.rstd, g = dy * w[j];
        // (past the row's end dy and w are 0)
        s.x += g;
        s.y = fmaf(g, hat, s.y);
        cw[i][j] = fmaf(dy, hat, cw[i][j]);
        cb[i][j] += dy;
      }
    }
    if (a.y) {
      s = nm_row_sum<L>(s, part, turn);
      const float s1 = a.rms ? 0.f : s.x * a.inv_d, s2 = s.y * a.inv_d;
      if (on) {
        T* dx = reinterpret_cast<T*>(a.y) + row * a.y_stride;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int64_t at = in_row + (int64_t)i * L;
          if (at * VEC >= d) continue;
          float w[VEC], f[VEC];
          W::weights(a.w, wide, vec_w, at, d, w);
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            const float hat = (W::at(r.x[i], j) - r.m) * r.rstd;
            f[j] = r.rstd * (W::at(r.dy[i], j) * w[j] - s1 - hat * s2);
            if (a.res) f[j] += W::at(t[i], j);
          }
          W::store(dx, at, d, vec, f);
        }
      }
    }
    r = next;
  }
  if (!sums) return;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float* to = a.part + ((int64_t)blockIdx.x * 2 + which) * d;
    if constexpr (ROWS > 1) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j)
          columns[(group * N * L + i * L + in_row) * VEC + j] = which ? cb[i][j] : cw[i][j];
      __syncthreads();
      for (int c = threadIdx.x; c < L * N * VEC && c < d; c += NT) {
        float v = 0.f;
        for (int g = 0; g < ROWS; ++g) v += columns[g * N * L * VEC + c];
        to[c] = v;
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const int64_t c = (in_row + (int64_t)i * L) * VEC + j;
          if (c < d) to[c] = which ? cb[i][j] : cw[i][j];
        }
    }
  }
}

// The gradients of the weights from the CTAs' sums: 32 columns a CTA, each warp every eighth of them
constexpr int NS_NT = 256;
static __global__ void __launch_bounds__(NS_NT) dnorm_sum(const __grid_constant__ NormArgs a, const int ctas) {
  __shared__ float part[NS_NT / 32][32];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, which = blockIdx.y;
  const int64_t c = (int64_t)blockIdx.x * 32 + lane;
  float* to = which ? a.db : a.dw;
  if (!to) return;
  float v = 0.f;
  if (c < a.d) {
    const float* p = a.part + which * a.d + c;
#pragma unroll 4
    for (int i = warp; i < ctas; i += NS_NT / 32) v += __ldcg(p + (int64_t)i * 2 * a.d);
  }
  part[warp][lane] = v;
  __syncthreads();
  if (warp > 0 || c >= a.d) return;
  v = 0.f;
#pragma unroll
  for (int w = 0; w < NS_NT / 32; ++w) v += part[w][lane];
  to[c] = a.accumulate ? to[c] + v : v;
}

// ---- any width: a CTA per row, which it reads again for each sweep ---------------------

constexpr int NW_NT = 256;

template <typename T>
__global__ void __launch_bounds__(NW_NT) norm_wide(const NormArgs a) {
  __shared__ float part[32];
  pdl_wait();
  pdl_trigger();
  const int64_t row = blockIdx.x, d = a.d;
  const T* x = reinterpret_cast<const T*>(a.x) + row * a.x_stride;
  const T* r = a.res ? reinterpret_cast<const T*>(a.res) + row * a.res_stride : nullptr;
  T* total = a.total ? reinterpret_cast<T*>(a.total) + row * a.total_stride : nullptr;
  T* y = reinterpret_cast<T*>(a.y) + row * a.y_stride;
  auto h = [&](int64_t i) {
    const float v = nm_get(x + i);
    return r ? nm_held<T>(v + nm_get(r + i)) : v;
  };
  float m = 0.f, s = 0.f;
  if (!a.rms) {
    for (int64_t i = threadIdx.x; i < d; i += NW_NT) s += h(i);
    m = nm_block_sum(s, part) * a.inv_d;
  }
  s = 0.f;
  float s1 = 0.f;
  for (int64_t i = threadIdx.x; i < d; i += NW_NT) {
    const float v = h(i) - m;
    s = fmaf(v, v, s);
    s1 += v;
  }
  const float off = a.rms ? 0.f : nm_block_sum(s1, part) * a.inv_d;  // what m is short of the mean
  const float rstd = nm_rstd(nm_block_sum(s, part), off, a);
  for (int64_t i = threadIdx.x; i < d; i += NW_NT) {
    const float v = h(i);  // (before either output, which may be its buffer)
    const float b = a.b ? nm_weight(a.b, a.wide_w, i) : 0.f;
    if (total) nm_put(total + i, v);
    nm_put(y + i, fmaf(((v - m) - off) * rstd, nm_weight(a.w, a.wide_w, i), b));
  }
  if (threadIdx.x == 0) {
    if (a.mean && !a.rms) a.mean[row] = m + off;
    if (a.rstd) a.rstd[row] = rstd;
  }
}

template <typename T>
__global__ void __launch_bounds__(NW_NT) dnorm_wide(const NormArgs a) {
  __shared__ float part[32];
  pdl_wait();
  pdl_trigger();
  const int64_t row = blockIdx.x, d = a.d;
  const T* x = reinterpret_cast<const T*>(a.x) + row * a.x_stride;
  const T* dy = reinterpret_cast<const T*>(a.dy) + row * a.dy_stride;
  const T* r = a.res ? reinterpret_cast<const T*>(a.res) + row * a.res_stride : nullptr;
  T* dx = reinterpret_cast<T*>(a.y) + row * a.y_stride;
  const float m = a.rms ? 0.f : a.mean[row], rstd = a.rstd[row];
  float s1 = 0.f, s2 = 0.f;
  for (int64_t i = threadIdx.x; i < d; i += NW_NT) {
    const float g = nm_get(dy + i) * nm_weight(a.w, a.wide_w, i);
    s1 += g;
    s2 = fmaf(g, (nm_get(x + i) - m) * rstd, s2);
  }
  s1 = a.rms ? 0.f : nm_block_sum(s1, part) * a.inv_d;
  s2 = nm_block_sum(s2, part) * a.inv_d;
  for (int64_t i = threadIdx.x; i < d; i += NW_NT) {
    const float g = nm_get(dy + i) * nm_weight(a.w, a.wide_w, i);
    const float v = rstd * (g - s1 - (nm_get(x + i) - m) * rstd * s2);
    nm_put(dx + i, r ? v + nm_get(r + i) : v);
  }
}

// the gradients of the weights: a CTA of 32 warps per 32 columns, each warp every 32nd row
constexpr int NC_NT = 1024;
template <typename T>
__global__ void __launch_bounds__(NC_NT) dnorm_columns(const NormArgs a) {
  __shared__ float part[2][32][33];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t i = (int64_t)blockIdx.x * 32 + lane;
  float w = 0.f, b = 0.f;
  if (i < a.d)
    for (int64_t row = warp; row < a.n_rows; row += 32) {
      const float g = nm_get(reinterpret_cast<const T*>(a.dy) + row * a.dy_stride + i);
      const float x = nm_get(reinterpret_cast<const T*>(a.x) + row * a.x_stride + i);
      w = fmaf(g, (x - (a.rms ? 0.f : a.mean[row])) * a.rstd[row], w);
      b += g;
    }
  part[0][warp][lane] = w;
  part[1][warp][lane] = b;
  __syncthreads();
  if (warp >= 2 || i >= a.d) return;
  float v = 0.f;
  for (int q = 0; q < 32; ++q) v += part[warp][q][lane];
  float* to = warp == 0 ? a.dw : a.db;
  if (to) to[i] = a.accumulate ? to[i] + v : v;
}

}  // namespace prk
