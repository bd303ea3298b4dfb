// How the attention calls deal out their work: arithmetic on lengths and sizes alone, which host and device share and which can be compiled
// and looked at without CUDA.
#pragma once

#include <math.h>
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

// ---- single tokens: the tiles of all sequences and key heads in one line, cut into equal ranges
constexpr int kDecTile = 64;               // tokens of a tile

// `total` tiles in `ctas` ranges: the first `longer` of them have each + 1 tiles, the others `each` (at least 1).
struct Ranges {
  int each, longer;
  FPT_RULE int first_of(int i) const { return i * each + (i < longer ? i : longer); }
  FPT_RULE int cta_of(int x) const {
    const int edge = longer * (each + 1);
    return x < edge ? x / (each + 1) : longer + (x - edge) / each;
  }
};

FPT_RULE int tiles_of(int len) { return len > 0 ? (len + kDecTile - 1) / kDecTile : 1; }

// ---- prompts: keys split where few query rows would leave SMs idle
constexpr int kPrTile = 128;               // query rows of a tile, keys of a tile
constexpr int kPrPartTiles = 4, kPrParts = 32;       // a part's tiles at the least, a task's parts at the most
constexpr int kPrSplitGain = 6;                        // tiles less to walk through for which keys are split

// The tasks of one sequence with more tiles of keys than L, which are its last ones, in equal parts of at most L tiles.  L is a quarter more
// than an SM's share of all tiles, at least kPrPartTiles, and as much more as it takes for the workspace to hold the parts' sums.
// (32 heads of 128 and 8 of keys: 64 queries behind 4 000 keys 62 -> 30 us, 256 behind 30 000 409 -> 164; 16 behind
// 100 000, 8 heads and one of keys: 1 197 -> 70; one prompt of 5 400, 5 heads and one of keys, 83 -> 60; of 4 000, 4 heads and one, 60 -> 42.)
struct Splitting {
  int len_k, len_q, places, per_log2, causal;                // places: tasks a unit
  FPT_RULE int most() const { return (int)(((uint32_t)len_k + kPrTile - 1) / kPrTile); }
  // all its tasks' tiles
  FPT_RULE uint32_t tiles() const {
    const int64_t first = (int64_t)len_k - len_q + (1 << per_log2);           // keys that the first task sees
    const int least = !causal ? most() : first <= 0 ? 0 : first >= len_k ? most() : (int)((first + kPrTile - 1) / kPrTile);
    return (uint32_t)(((int64_t)places * (most() + least) + 1) / 2);
  }
  FPT_RULE int split(int L) const {
    if (most() <= L || places <= 0) return 0;
    const int64_t seen = (int64_t)L * kPrTile - ((int64_t)len_k - len_q);     // rows from the first on whose keys are L tiles or fewer
    const int64_t from = !causal || seen <= 0 ? 0 : seen >> per_log2;
    return from < places ? places - (int)from : 1;
  }
  FPT_RULE int parts(int L) const {
    const int p = (most() + L - 1) / L;
    return p < 1 ? 1 : p > kPrParts ? kPrParts : p;
  }
  FPT_RULE static int first_length(uint32_t all, int sms) {
    const int share = (int)fminf((float)all * (1.25f / (float)sms), 1e9f) + 1;       // (a division of 64 bits would take longer than the search)
    return share > kPrPartTiles ? share : kPrPartTiles;
  }
};

}  // namespace fpt
