// How the attention calls deal out their work: arithmetic on lengths and sizes alone, which host and device share and which can be compiled
// and looked at without CUDA.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define FPT_RULE __host__ __device__ __forceinline__
#else
#define FPT_RULE inline
#endif

namespace fpt {

// Rows lo .. hi-1 of a buffer of M.
FPT_RULE bool rows_fit(int lo, int hi, int M) { return lo >= 0 && hi >= lo && hi <= M; }

// A launch over the pages (or blocks of `block` rows) that packed sequences touch, without their lengths on the host:
// sequence s, rows lo .. hi-1, is given floor(hi / block) - floor(lo / block) + 2 tasks, which is at least the number of
// blocks that its rows can touch.  block 0: a task for each row.  The place of task `id` among those of sequence s, or -1.
FPT_RULE int place_of_task(int lo, int hi, int s, int block, int id) {
  if (block == 0) return lo <= id && id < hi ? 0 : -1;
  const int first = lo / block + 2 * s;
  return first <= id && id < hi / block + 2 * s + 2 ? id - first : -1;
}
// Tasks of a launch.
FPT_RULE int64_t block_tasks(int M, int n_seqs, int block) { return block == 0 ? M : (int64_t)M / block + 2 * (int64_t)n_seqs; }

}  // namespace fpt
