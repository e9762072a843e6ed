// Host side of pr_top_logits: argument checks and the launches of the kernels in pr_top.cuh.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "pr_loss_host.h"
#include "pr_top.cuh"

using namespace prh;

static_assert(PR_MAX_LISTED == prk::TP_MAX, "list length");

namespace {

template <typename T>
const void* ring_kernel(bool words) {
  return words ? reinterpret_cast<const void*>(&prk::top_ring<T, 1>)
               : reinterpret_cast<const void*>(&prk::top_ring<T, 4>);
}
const void* ring_kernel(pr_dtype dt, bool words) {
  return dt == PR_DTYPE_BF16 ? ring_kernel<__nv_bfloat16>(words) : ring_kernel<float>(words);
}

const void* short_kernel(pr_dtype dt) {
  return dt == PR_DTYPE_BF16 ? reinterpret_cast<const void*>(&prk::top_short<__nv_bfloat16>)
                             : reinterpret_cast<const void*>(&prk::top_short<float>);
}

// shared memory of one, two or three CTAs on an SM
constexpr size_t SM_BYTES = 227 * 1024, HALF_BYTES = 113 * 1024, THIRD_BYTES = 75 * 1024;

// The ring's launch: CTAs per row, words of a group, bytes of the groups' maxima, places.
struct TopShape {
  int cluster, places, on_sm;
  bool words, fits;
  size_t gm, smem;
};

// Warps of a CTA of top_short, or 0 where the ring takes less time: with fewer than five rows of a
// CTA, or no more than one for each of the ring's CTAs (k = 20, V = 4,000 bf16: 300 rows 7.9 us for
// the ring's 6.4, 456 7.8 for 8.1, 608 7.8 for 12.3; V = 10,000: 13.2 for 9.3, 13.4 for 14.1).
int short_warps(const pr_ctx* c, int64_t n_rows, int64_t vocab, pr_dtype dt) {
  if (n_rows <= 3 * c->num_sms) return 0;
  const int64_t part = std::max<int64_t>(16, vocab * (int64_t)esize(dt) / 16 * 16);
  const int64_t w = std::min<int64_t>(
      prk::TS_MOST, ((int64_t)HALF_BYTES - (int64_t)prk::TS_START) / part);
  return w >= 5 ? (int)w : 0;
}

TopShape choose(const pr_ctx* c, pr_dtype dt, int64_t n_rows, int64_t vocab) {
  const int64_t words = vocab * (int64_t)esize(dt) / 16 + 1;
  TopShape s;
  s.cluster = 1;
  s.fits = false;
  // as many CTAs per row as the SMs have room for, while each has a chunk
  while (s.cluster < 8 && n_rows * s.cluster * 2 <= 2 * c->num_sms &&
         words > (int64_t)s.cluster * prk::TR_CHUNK)
    s.cluster *= 2;
  for (; s.cluster <= 8; s.cluster *= 2) {
    const int64_t chunks = (words + prk::TR_CHUNK - 1) / prk::TR_CHUNK;
    const int64_t part = std::min(words, (chunks + s.cluster - 1) / s.cluster * prk::TR_CHUNK);
    s.words = part <= 4096;  // (a bound from fewer than 1,024 groups lets too much through)
    const int64_t groups = s.words ? part : (part + 3) / 4;
    s.gm = ((size_t)groups * (dt == PR_DTYPE_BF16 ? 2 : 4) + 127) / 128 * 128;
    const size_t fixed = prk::TR_START + s.gm;
    if (fixed + 2 * prk::TR_BYTES > SM_BYTES || groups > 65536) continue;
    // Three CTAs on an SM where their rings keep three places, two with four: while one chooses,
    // the others stream (4,096 rows of V = 151,936 bf16, k = 20: 206 us for 234 with two).  Where
    // that leaves one CTA, two with a row's parts are better (1,000 rows of V = 262,144 fp32: 190
    // for 202).  Fewer CTAs than would fit get the room of the others.
    const int64_t ctas = n_rows * s.cluster;
    s.on_sm = fixed + 3 * prk::TR_BYTES <= THIRD_BYTES  ? 3
              : fixed + 4 * prk::TR_BYTES <= HALF_BYTES ? 2
                                                        : 1;
    if (s.on_sm == 1 && s.cluster < 4 && words > 2 * s.cluster * prk::TR_CHUNK) continue;
    s.on_sm = (int)std::min<int64_t>(s.on_sm, (ctas + c->num_sms - 1) / c->num_sms);
    const size_t room = s.on_sm == 3 ? THIRD_BYTES : s.on_sm == 2 ? HALF_BYTES : SM_BYTES;
    s.places = (int)((room - fixed) / prk::TR_BYTES);
    s.places = std::min(s.places, (int)prk::TR_MOST);
    s.smem = fixed + (size_t)s.places * prk::TR_BYTES;
    s.fits = true;
    return s;
  }
  return s;
}

}  // namespace

extern "C" {

pr_status pr_top_logits(pr_ctx* c, const void* logits, pr_dtype dt, int64_t n_rows, int64_t vocab,
                        int64_t row_stride, int32_t k, float temperature, int32_t* ids,
                        float* logp, void* stream) {
  if (!c || (dt != PR_DTYPE_F32 && dt != PR_DTYPE_BF16)) return PR_ERR_INVALID_ARG;
  if (n_rows < 0 || n_rows > 0x7fffffffLL || vocab <= 0 || vocab > 0x7fffffffLL ||
      row_stride < vocab || k < 1 || k > PR_MAX_LISTED)
    return PR_ERR_INVALID_ARG;
  if (n_rows > 0 && (!logits || !ids || !logp)) return PR_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(logits) % (dt == PR_DTYPE_BF16 ? 2 : 4) != 0)
    return PR_ERR_INVALID_ARG;
  if (!(temperature >= 1e-3f) || !(temperature <= 1e3f)) return PR_ERR_INVALID_ARG;
  pr_status st = set_device(c);
  if (st != PR_OK) return st;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if ((st = timing_begin(c, s)) != PR_OK || n_rows == 0) return st;
  const float big = (float)(1e9 * (double)temperature);
  if (!c->top_ready) {
    for (pr_dtype t : {PR_DTYPE_F32, PR_DTYPE_BF16}) {
      for (bool words : {false, true})
        PR_CUDA(cudaFuncSetAttribute(ring_kernel(t, words),
                                     cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SM_BYTES));
      PR_CUDA(cudaFuncSetAttribute(short_kernel(t), cudaFuncAttributeMaxDynamicSharedMemorySize,
                                   (int)HALF_BYTES));
    }
    c->top_ready = true;
  }
  prk::LossArgs l;
  fill(l, c, logits, n_rows, vocab, row_stride, nullptr, nullptr, nullptr, 0, nullptr, temperature,
       1.f, nullptr, logp, nullptr, 0);
  int kk = k;
  float limit = big;
  int32_t* out = ids;
  if (const int warps = short_warps(c, n_rows, vocab, dt)) {
    int part = (int)std::max<int64_t>(16, vocab * (int64_t)esize(dt) / 16 * 16);
    void* args[] = {&l, &kk, &limit, &out, &part};
    st = launch(short_kernel(dt), 2 * c->num_sms, 32u * warps,
                prk::TS_START + (size_t)warps * part, 1, args, s);
    return st == PR_OK ? timing_mark(c, s) : st;
  }
  const TopShape shape = choose(c, dt, n_rows, vocab);
  if (shape.fits) {
    int places = shape.places, gm = (int)shape.gm;
    const int64_t at_once = (int64_t)shape.on_sm * c->num_sms;
    const int64_t groups = std::min<int64_t>(n_rows, std::max<int64_t>(1, at_once / shape.cluster));
    void* args[] = {&l, &kk, &limit, &out, &places, &gm};
    st = launch(ring_kernel(dt, shape.words), (unsigned)(groups * shape.cluster), prk::TR_NT,
                shape.smem, (unsigned)shape.cluster, args, s,
                n_rows < groups + 1 && groups * shape.cluster < at_once);
    return st == PR_OK ? timing_mark(c, s) : st;
  }
  prk::TopArgs a;
  a.logits = logits;
  a.n_rows = n_rows;
  a.vocab = vocab;
  a.row_stride = row_stride;
  a.k = k;
  a.c2 = (float)(1.4426950408889634 / (double)temperature);
  a.big = big;
  a.ids = ids;
  a.logp = logp;
  a.ctx_flags = c->flags;
  int64_t group = std::max<int64_t>(32, (vocab + prk::TP_GROUPS - 1) / prk::TP_GROUPS);
  void* args[] = {&a, &group};
  st = launch(dt == PR_DTYPE_BF16 ? reinterpret_cast<const void*>(&prk::top_rows<__nv_bfloat16>)
                                  : reinterpret_cast<const void*>(&prk::top_rows<float>),
              (unsigned)n_rows, prk::TP_NT, 0, 1, args, s);
  return st == PR_OK ? timing_mark(c, s) : st;
}

}  // extern "C"
