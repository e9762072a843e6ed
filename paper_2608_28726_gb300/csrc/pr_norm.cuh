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

#include "pr_loss.cuh"

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
  int32_t vec_w;        // the weights begin at multiples of 16 bytes
  int32_t stages;       // rows of a group on their way into shared memory
  int32_t row_bytes;    // room of one there
  int32_t stage_res;    // the residual's (dtotal's), too; else its threads read it
  float* part;          // workspace: [CTAs][2][d] sums of dy xhat and of dy
  uint32_t* ctx_flags;
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
  const float v = fmaf(s, a.inv_d, -off * off);
  return 1.f / sqrtf((v < 0.f ? 0.f : v) + a.eps);  // (NaN stays NaN)
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

// ---- rows in shared memory -------------------------------------------------------------
//
// L threads have a row, N words of 16 bytes each, and memory is read once: rows come into shared
// memory by bulk copies, a few ahead, so that what is on its way takes no registers and memory
// stays busy while rows are summed.  Rows of up to 16 words are read by their threads.  Rows of up
// to 32 threads are summed by shuffles, wider ones through shared memory with a barrier of the
// row's threads alone, so that the CTA's other rows go on meanwhile.  The weights are in shared
// memory, too.  8,847 x 3,584 bf16: forward with a residual 49 us, 5.2 TB/s of its four passes over
// the rows, backward 54; what bounds both is the rows' chain of two sums (one) and some 2,000
// instructions a row, not memory.
//
// Columns of thread t's word i: VEC neighbours from (t + i L) VEC on; in rows off the 16-byte grid,
// L apart from t + i VEC L on, so that a warp's accesses stay side by side.  Of such a row the copy
// takes every 16-byte word that it touches (a word with a byte of an allocation lies in it whole).

constexpr int NR_NT = 256;  // threads of a CTA of rows of up to so many

// WHOLE: rows on the grid, of whole words.  (A template: what chooses at run time issues both ways'
// instructions: 8,847 x 3,584 bf16 forward 58 us for 48.)
template <typename T, int L, bool WHOLE>
struct RowWord {
  static constexpr int VEC = 16 / (int)sizeof(T);
  float2 f[VEC / 2];
  static __device__ __forceinline__ int column(int t, int i, int j) {
    return WHOLE ? (t + i * L) * VEC + j : t + (i * VEC + j) * L;
  }
  // whether word i has all of its columns, or any
  static __device__ __forceinline__ bool full(int t, int i, int d) {
    return column(t, i, VEC - 1) < d;
  }
  static __device__ __forceinline__ bool some(int t, int i, int d) { return column(t, i, 0) < d; }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int j = 0; j < VEC / 2; ++j) f[j] = make_float2(0.f, 0.f);
  }
  __device__ __forceinline__ void set(int j, float v) {
    if (j & 1) f[j / 2].y = v;
    else f[j / 2].x = v;
  }
  __device__ __forceinline__ float get(int j) const { return j & 1 ? f[j / 2].y : f[j / 2].x; }
  __device__ __forceinline__ void from(const uint4& w) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    if constexpr (sizeof(T) == 4) {
      f[0] = make_float2(__uint_as_float(u[0]), __uint_as_float(u[1]));
      f[1] = make_float2(__uint_as_float(u[2]), __uint_as_float(u[3]));
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        f[q] = make_float2(__uint_as_float(u[q] << 16), __uint_as_float(u[q] & 0xffff0000u));
    }
  }
  __device__ __forceinline__ uint4 packed() const {
    if constexpr (sizeof(T) == 4) {
      return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x),
                        __float_as_uint(f[1].y));
    } else {
      uint32_t u[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const __nv_bfloat162 h = __float22bfloat162_rn(f[q]);
        u[q] = *reinterpret_cast<const uint32_t*>(&h);
      }
      return make_uint4(u[0], u[1], u[2], u[3]);
    }
  }
  // word i of thread t of a row of d elements (in shared or global memory), 0 past its end
  __device__ __forceinline__ void load(const T* row, int t, int i, int d) {
    if constexpr (WHOLE) {
      if (full(t, i, d)) from(*reinterpret_cast<const uint4*>(row + (t + i * L) * VEC));
      else zero();
    } else if (full(t, i, d)) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) set(j, nm_get(row + column(t, i, j)));
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        set(j, column(t, i, j) < d ? nm_get(row + column(t, i, j)) : 0.f);
    }
  }
  __device__ __forceinline__ void store(T* row, int t, int i, int d) const {  // (of a word with some)
    if constexpr (WHOLE) {
      *reinterpret_cast<uint4*>(row + (t + i * L) * VEC) = packed();
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        if (column(t, i, j) < d) nm_put(row + column(t, i, j), get(j));
    }
  }
  // its weights, which shared memory holds
  __device__ __forceinline__ void weights(const unsigned char* w, bool wide, int t, int i, int d) {
    if constexpr (WHOLE) {
      const int c0 = (t + i * L) * VEC;
      if (!some(t, i, d)) {
        zero();
      } else if (wide) {
#pragma unroll
        for (int q = 0; q < VEC / 4; ++q) {
          const float4 v = reinterpret_cast<const float4*>(w)[c0 / 4 + q];
          f[2 * q] = make_float2(v.x, v.y);
          f[2 * q + 1] = make_float2(v.z, v.w);
        }
      } else {
#pragma unroll
        for (int q = 0; q < VEC / 4; ++q) {
          const uint2 v = reinterpret_cast<const uint2*>(w)[c0 / 4 + q];
          f[2 * q] = make_float2(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u));
          f[2 * q + 1] =
              make_float2(__uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u));
        }
      }
    } else if (wide) {
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        set(j, column(t, i, j) < d ? reinterpret_cast<const float*>(w)[column(t, i, j)] : 0.f);
    } else {
      const __nv_bfloat16* const narrow = reinterpret_cast<const __nv_bfloat16*>(w);
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        set(j, column(t, i, j) < d ? nm_get(narrow + column(t, i, j)) : 0.f);
    }
  }
};
__device__ __forceinline__ float2 nm_both(float v) { return make_float2(v, v); }

// the weights of d columns into shared memory, 0 up to a multiple of eight; by a CTA, then a
// barrier
__device__ __forceinline__ int nm_weight_bytes(int d, bool wide) {
  return (d + 7) / 8 * 8 * (wide ? 4 : 2);
}
__device__ __forceinline__ void nm_keep(unsigned char* to, const void* w, bool wide, bool vec,
                                        int d) {
  const int words = vec ? d / (wide ? 4 : 8) : 0;
#pragma unroll 4
  for (int i = threadIdx.x; i < words; i += blockDim.x)
    reinterpret_cast<uint4*>(to)[i] = reinterpret_cast<const uint4*>(w)[i];
#pragma unroll 4
  for (int i = words * (wide ? 4 : 8) + threadIdx.x; i < (d + 7) / 8 * 8; i += blockDim.x) {
    if (wide)
      reinterpret_cast<float*>(to)[i] = i < d ? reinterpret_cast<const float*>(w)[i] : 0.f;
    else
      reinterpret_cast<uint16_t*>(to)[i] =
          i < d ? reinterpret_cast<const uint16_t*>(w)[i] : (uint16_t)0;
  }
}

// (a, b) summed over a row's L threads.  `part`: two buffers of a float2 per warp of the CTA, used
// in turn.
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
    v = part[turn][row * W + (lane & (W - 1))];
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) {
      v.x += __shfl_xor_sync(FULL, v.x, o);
      v.y += __shfl_xor_sync(FULL, v.y, o);
    }
  }
  return v;
}

// The rows of a group of L threads in shared memory: `stages` places for the words of K rows each
// (x and the residual; x, dy and dtotal).  One thread fills them; a place is filled again once
// every thread is past a later sum.
template <typename T, int L>
struct RowStages {
  uint64_t* full;        // a barrier per place
  unsigned char* at;     // this group's places
  int stages, bytes, row_bytes, d;  // bytes of a place, and of a row in it
  int place = 0;
  uint32_t turn = 0u;
  uint32_t* flags;
  bool ok = true;
  __device__ __forceinline__ RowStages(unsigned char* smem, const NormArgs& a, int k)
      : stages(a.stages), row_bytes(a.row_bytes), d((int)a.d), flags(a.ctx_flags) {
    const int groups = blockDim.x / L, group = threadIdx.x / L;
    bytes = k * row_bytes;
    full = reinterpret_cast<uint64_t*>(smem) + group * stages;
    at = smem + (groups * stages * 8 + 127) / 128 * 128 + (size_t)group * stages * bytes;
  }
  __device__ __forceinline__ void init() {  // then a barrier of the CTA
    if (threadIdx.x % L == 0) {
      for (int i = 0; i < stages; ++i) bar_init(&full[i], 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
  }
  // the words that a row touches
  __device__ __forceinline__ uint32_t size(const T* row) const {
    const uint32_t head = (uint32_t)(reinterpret_cast<uintptr_t>(row) & 15u);
    return (head + (uint32_t)d * (uint32_t)sizeof(T) + 15u) & ~15u;
  }
  __device__ __forceinline__ void expect(int i, uint32_t all) { bar_expect(&full[i], all); }
  __device__ __forceinline__ void copy(int i, int j, const T* row) {
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
            sm_addr(at + (size_t)i * bytes + (size_t)j * row_bytes)),
        "l"(reinterpret_cast<uintptr_t>(row) & ~(uintptr_t)15), "r"(size(row)), "r"(sm_addr(&full[i]))
        : "memory");
  }
  __device__ __forceinline__ void wait() {
    if (ok) ok = ring_wait(sm_addr(&full[place]), turn, flags);
    __syncwarp();
  }
  // the j-th row of the place, whose memory is at `row`
  __device__ __forceinline__ const T* here(int j, const T* row) const {
    return reinterpret_cast<const T*>(at + (size_t)place * bytes + (size_t)j * row_bytes +
                                      (reinterpret_cast<uintptr_t>(row) & 15u));
  }
  __device__ __forceinline__ void step() {
    if (++place == stages) {
      place = 0;
      turn ^= 1u;
    }
  }
};

template <typename T, int L, int N, bool STAGED, bool WHOLE>
__global__ void __launch_bounds__(L > NR_NT ? L : NR_NT, L > NR_NT ? 1 : 3)
    norm_rows(const __grid_constant__ NormArgs a) {
  using W = RowWord<T, L, WHOLE>;
  constexpr int H = W::VEC / 2;
  extern __shared__ __align__(16) unsigned char nm_raw[];
  __shared__ float2 part[2][32];
  const int rows = blockDim.x / L, in_row = threadIdx.x % L, group = threadIdx.x / L;
  const int d = (int)a.d;
  const bool wide = a.wide_w, res = a.res != nullptr;
  const int w_bytes = nm_weight_bytes(d, wide);
  const int64_t step = (int64_t)gridDim.x * rows, first = (int64_t)blockIdx.x * rows;
  auto x_of = [&](int64_t row) { return reinterpret_cast<const T*>(a.x) + row * a.x_stride; };
  auto res_of = [&](int64_t row) { return reinterpret_cast<const T*>(a.res) + row * a.res_stride; };
  const bool res_staged = res && a.stage_res;
  RowStages<T, L> st(nm_raw + (a.b ? 2 : 1) * w_bytes, a, res_staged ? 2 : 1);
  auto fill = [&](int i, int64_t row) {
    st.expect(i, st.size(x_of(row)) + (res_staged ? st.size(res_of(row)) : 0u));
    st.copy(i, 0, x_of(row));
    if (res_staged) st.copy(i, 1, res_of(row));
  };
  if (STAGED) {
    st.init();
    __syncthreads();
  }
  pdl_wait();
  pdl_trigger();
  if (STAGED && in_row == 0)
    for (int i = 0; i < a.stages; ++i)
      if (first + group + i * step < a.n_rows) fill(i, first + group + i * step);
  nm_keep(nm_raw, a.w, wide, a.vec_w, d);
  if (a.b) nm_keep(nm_raw + w_bytes, a.b, wide, a.vec_w, d);
  __syncthreads();
  int turn = 0;  // of the sums' buffers
  // (every thread of a warp goes through the sums: the last rows of a CTA may be none)
  for (int64_t r0 = first; r0 < a.n_rows; r0 += step) {
    const int64_t row = r0 + group;
    const bool on = row < a.n_rows;
    W h[N];
    float2 sum = make_float2(0.f, 0.f);
    if (on) {
      const T *x = x_of(row), *r = res_of(row);
      if (STAGED) {
        st.wait();
        x = st.here(0, x);
        if (res_staged) r = st.here(1, r);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) h[i].load(x, in_row, i, d);
      if (res) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          W q;
          q.load(r, in_row, i, d);
#pragma unroll
          for (int j = 0; j < H; ++j) h[i].f[j] = __fadd2_rn(h[i].f[j], q.f[j]);
          h[i].from(h[i].packed());  // rounded
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < H; ++j) h[i].f[j] = make_float2(0.f, 0.f);
    }
    float m = 0.f;
    if (!a.rms) {
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < H; ++j) sum = __fadd2_rn(sum, h[i].f[j]);
      m = nm_row_sum<L>(make_float2(sum.x + sum.y, 0.f), part, turn).x * a.inv_d;
      turn ^= 1;
    }
    float2 sq = make_float2(0.f, 0.f);
    sum = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (W::full(in_row, i, d)) {
#pragma unroll
        for (int j = 0; j < H; ++j) {
          const float2 v = __fadd2_rn(h[i].f[j], nm_both(-m));
          sq = __ffma2_rn(v, v, sq);
          sum = __fadd2_rn(sum, v);
        }
      } else if (!WHOLE) {
#pragma unroll
        for (int j = 0; j < W::VEC; ++j) {
          const float v = W::column(in_row, i, j) < d ? h[i].get(j) - m : 0.f;
          sq.x = fmaf(v, v, sq.x);
          sum.x += v;
        }
      }
    }
    const float2 s = nm_row_sum<L>(make_float2(sq.x + sq.y, sum.x + sum.y), part, turn);
    turn ^= 1;
    if (STAGED) {  // every thread has its words
      if (in_row == 0 && row + a.stages * step < a.n_rows) fill(st.place, row + a.stages * step);
      st.step();
    }
    const float off = a.rms ? 0.f : s.y * a.inv_d, rstd = nm_rstd(s.x, off, a);
    if (on) {
      T* y = reinterpret_cast<T*>(a.y) + row * a.y_stride;
      T* total = reinterpret_cast<T*>(a.total) + row * a.total_stride;
      const float mean = m + off;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (!W::some(in_row, i, d)) continue;
        if (a.total) h[i].store(total, in_row, i, d);
        W w, b;
        w.weights(nm_raw, wide, in_row, i, d);
#pragma unroll
        for (int j = 0; j < H; ++j) b.f[j] = make_float2(0.f, 0.f);
        if (a.b) b.weights(nm_raw + w_bytes, wide, in_row, i, d);
#pragma unroll
        for (int j = 0; j < H; ++j) {
          const float2 v = __fmul2_rn(__fadd2_rn(h[i].f[j], nm_both(-mean)), nm_both(rstd));
          h[i].f[j] = __ffma2_rn(v, w.f[j], b.f[j]);
        }
        h[i].store(y, in_row, i, d);
      }
      if (in_row == 0) {
        if (a.mean && !a.rms) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
      }
    }
  }
}

// The backward pass.  A thread keeps the sums of its columns over all rows of its CTA; the CTA's
// rows are added up in order at the end and go to the workspace, and dnorm_sum adds up the CTAs.
template <typename T, int L, int N, bool STAGED, bool WHOLE>
__global__ void __launch_bounds__(L > NR_NT ? L : NR_NT, L > NR_NT ? 1 : 2)
    dnorm_rows(const __grid_constant__ NormArgs a) {
  using W = RowWord<T, L, WHOLE>;
  constexpr int VEC = W::VEC, H = VEC / 2, NT = L > NR_NT ? L : NR_NT, ROWS = NT / L;
  constexpr bool KEEP = N <= 3;  // xhat and g of a row's words stay in registers
  extern __shared__ __align__(16) unsigned char nm_raw[];
  __shared__ float2 part[2][32];
  const int in_row = threadIdx.x % L, group = threadIdx.x / L;
  const int d = (int)a.d;
  const bool wide = a.wide_w, res = a.res && a.y, res_staged = res && a.stage_res;
  const int w_bytes = nm_weight_bytes(d, wide);
  const int64_t step = (int64_t)gridDim.x * ROWS, first = (int64_t)blockIdx.x * ROWS;
  auto x_of = [&](int64_t row) { return reinterpret_cast<const T*>(a.x) + row * a.x_stride; };
  auto dy_of = [&](int64_t row) { return reinterpret_cast<const T*>(a.dy) + row * a.dy_stride; };
  auto res_of = [&](int64_t row) { return reinterpret_cast<const T*>(a.res) + row * a.res_stride; };
  RowStages<T, L> st(nm_raw + w_bytes, a, res_staged ? 3 : 2);
  auto fill = [&](int i, int64_t row) {
    st.expect(i, st.size(x_of(row)) + st.size(dy_of(row)) +
                     (res_staged ? st.size(res_of(row)) : 0u));
    st.copy(i, 0, x_of(row));
    st.copy(i, 1, dy_of(row));
    if (res_staged) st.copy(i, 2, res_of(row));
  };
  if (STAGED) {
    st.init();
    __syncthreads();
  }
  pdl_wait();
  pdl_trigger();
  if (STAGED && in_row == 0)
    for (int i = 0; i < a.stages; ++i)
      if (first + group + i * step < a.n_rows) fill(i, first + group + i * step);
  nm_keep(nm_raw, a.w, wide, a.vec_w, d);
  __syncthreads();
  W cw[N], cb[N];
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < H; ++j) cw[i].f[j] = cb[i].f[j] = make_float2(0.f, 0.f);
  auto moments = [&](int64_t row) {
    return row < a.n_rows ? make_float2(a.rms ? 0.f : __ldcg(a.mean + row), __ldcg(a.rstd + row))
                          : make_float2(0.f, 0.f);
  };
  int turn = 0, free_place = -1;  // the place of the row before this one
  float2 mo = moments(first + group);
  for (int64_t r0 = first; r0 < a.n_rows; r0 += step, turn ^= 1) {
    const int64_t row = r0 + group;
    const bool on = row < a.n_rows;
    const float2 next = moments(row + step);
    const T *x = x_of(row), *dy = dy_of(row), *t = res_of(row);
    float2 s1 = make_float2(0.f, 0.f), s2 = make_float2(0.f, 0.f);
    W hats[KEEP ? N : 1], gs[KEEP ? N : 1];
    if (on) {
      if (STAGED) {
        st.wait();
        x = st.here(0, x);
        dy = st.here(1, dy);
        if (res_staged) t = st.here(2, t);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        W xv, dv, w;
        xv.load(x, in_row, i, d);
        dv.load(dy, in_row, i, d);
        w.weights(nm_raw, wide, in_row, i, d);
#pragma unroll
        for (int j = 0; j < H; ++j) {  // (past the row's end dy and w are 0)
          const float2 hat = __fmul2_rn(__fadd2_rn(xv.f[j], nm_both(-mo.x)), nm_both(mo.y));
          const float2 g = __fmul2_rn(dv.f[j], w.f[j]);
          s1 = __fadd2_rn(s1, g);
          s2 = __ffma2_rn(g, hat, s2);
          cw[i].f[j] = __ffma2_rn(dv.f[j], hat, cw[i].f[j]);
          cb[i].f[j] = __fadd2_rn(cb[i].f[j], dv.f[j]);
          if (KEEP) {
            hats[i].f[j] = hat;
            gs[i].f[j] = g;
          }
        }
      }
    }
    const float2 s = nm_row_sum<L>(make_float2(s1.x + s1.y, s2.x + s2.y), part, turn);
    const bool alone = N == 8 && a.stages == 1;  // (rows of up to 64 KB: one place)
    if (STAGED && !alone) {  // every thread is past the row before
      if (in_row == 0 && free_place >= 0 && row + (a.stages - 1) * step < a.n_rows)
        fill(free_place, row + (a.stages - 1) * step);
      free_place = st.place;
      st.step();
    }
    if (a.y && on) {
      const float m1 = a.rms ? 0.f : s.x * a.inv_d, m2 = s.y * a.inv_d;
      T* dx = reinterpret_cast<T*>(a.y) + row * a.y_stride;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (!W::some(in_row, i, d)) continue;
        W xv, tv;
        if (!KEEP) {
          W dv, w;
          xv.load(x, in_row, i, d);
          dv.load(dy, in_row, i, d);
          w.weights(nm_raw, wide, in_row, i, d);
#pragma unroll
          for (int j = 0; j < H; ++j) {
            hats[0].f[j] = __fmul2_rn(__fadd2_rn(xv.f[j], nm_both(-mo.x)), nm_both(mo.y));
            gs[0].f[j] = __fmul2_rn(dv.f[j], w.f[j]);
          }
        }
        const W &hat = hats[KEEP ? i : 0], &gw = gs[KEEP ? i : 0];
        tv.zero();
        if (res) tv.load(t, in_row, i, d);
#pragma unroll
        for (int j = 0; j < H; ++j) {
          const float2 g = __fadd2_rn(gw.f[j], nm_both(-m1));
          xv.f[j] = __ffma2_rn(__ffma2_rn(hat.f[j], nm_both(-m2), g), nm_both(mo.y), tv.f[j]);
        }
        xv.store(dx, in_row, i, d);
      }
    }
    if (STAGED && alone) {  // filled when every thread is past this row
      nm_row_sum<L>(make_float2(0.f, 0.f), part, turn ^ 1);
      if (in_row == 0 && row + step < a.n_rows) fill(0, row + step);
      st.step();
    }
    mo = next;
  }
  if (!a.part) return;
  float* const columns = reinterpret_cast<float*>(nm_raw);  // (ROWS > 1: [ROWS][L N VEC])
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float* to = a.part + ((int64_t)blockIdx.x * 2 + which) * a.d;
    float* const at = ROWS > 1 ? columns + group * N * L * VEC : to;
    if (ROWS > 1) __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const W& v = which ? cb[i] : cw[i];
      if constexpr (WHOLE) {
        // (four columns at once: one by one a warp's stores would lie 32 bytes apart)
        if (ROWS > 1 || W::some(in_row, i, d)) {
#pragma unroll
          for (int j = 0; j < VEC; j += 4)
            *reinterpret_cast<float4*>(at + W::column(in_row, i, j)) =
                make_float4(v.f[j / 2].x, v.f[j / 2].y, v.f[j / 2 + 1].x, v.f[j / 2 + 1].y);
        }
      } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j)
          if (ROWS > 1 || W::column(in_row, i, j) < d) at[W::column(in_row, i, j)] = v.get(j);
      }
    }
    if constexpr (ROWS > 1) {
      __syncthreads();
      for (int c = threadIdx.x; c < L * N * VEC && c < d; c += NT) {
        float v = 0.f;
        for (int g = 0; g < ROWS; ++g) v += columns[g * N * L * VEC + c];
        to[c] = v;
      }
    }
  }
}

// The gradients of the weights from the CTAs' sums: 32 columns a CTA, each warp every 32nd of them
constexpr int NS_NT = 1024;
static __global__ void __launch_bounds__(NS_NT)
    dnorm_sum(const __grid_constant__ NormArgs a, const int ctas) {
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
#pragma unroll 10
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
