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
