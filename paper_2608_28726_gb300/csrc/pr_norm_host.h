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

// The backward pass of rows of 513 to 768 words: two rows of three words a thread on an SM, or one of
// two on all of its threads.  Two rows pay from eight of an SM on and with three places each, as fit
// up to some 715 words with weights of the rows' type.  us, two rows for one:
//   5,120 bf16       304 rows 14.2 for 11.9   1,400 22.4 for 22.6   8,000 72.1 for 83.7
//   4,288 bf16       608      13.1 for 12.7   1,216 17.1 for 18.3   8,000 68.3 for 82.5
//   6,144, 2 places  304      16.1 for 12.4   1,700 29.7 for 27.0   8,000 87.4 for 86.4
//   2,960 fp32, 2    608      10.8 for 10.6   2,000 24.5 for 22.0   8,000 73.7 for 67.5
inline bool norm_two_rows(int64_t n_rows, int num_sms, int64_t d, size_t esize, size_t wsize) {
  return n_rows > 8 * (int64_t)num_sms && norm_stages(d, esize, wsize, 1, 2, 3, 1, 3).fits;
}

}  // namespace prh
