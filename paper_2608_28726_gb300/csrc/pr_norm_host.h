// The norms' shared memory: the weights, then places of a few rows that are on their way, with a
// barrier each (RowStages).  Arithmetic alone, without a CUDA header.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace prh {

constexpr int NORM_STAGES = 4;             // places of a group of rows, at most
constexpr size_t NORM_FIXED = 1024 + 512;  // what a CTA has besides: the system's, the sums

// dynamic shared memory of a CTA, `ctas` of which are to be on an SM of 228 KB
constexpr size_t norm_room(int ctas) { return 228 * 1024 / ctas - NORM_FIXED; }
// bytes of the barriers of `groups` groups
constexpr size_t norm_bars(int groups, int stages) {
  return ((size_t)groups * stages * 8 + 127) / 128 * 128;
}

struct NormStages {
  bool fits;
  int32_t stages, row_bytes;
  size_t smem;
};
// Rows of d elements of `esize` bytes, `weights` arrays of such of `wsize`; places for k rows each,
// at least `least`, for each of `groups` groups of threads (0: rows are not staged).
inline NormStages norm_stages(int64_t d, size_t esize, size_t wsize, int groups, int ctas, int k,
                              int weights, int least) {
  NormStages s;
  s.row_bytes = (int32_t)((d * (int64_t)esize + 30) / 16 * 16);  // wherever a row begins
  s.stages = 0;
  s.smem = (size_t)weights * ((d + 7) / 8 * 8) * wsize;
  s.fits = true;
  if (groups == 0) return s;
  const size_t room = norm_room(ctas) - norm_bars(groups, NORM_STAGES);
  const size_t place = (size_t)groups * k * s.row_bytes;
  s.fits = room >= s.smem + least * place;
  if (!s.fits) return s;
  s.stages = (int32_t)std::min<size_t>(NORM_STAGES, (room - s.smem) / place);
  s.smem += norm_bars(groups, s.stages) + s.stages * place;
  return s;
}

}  // namespace prh
