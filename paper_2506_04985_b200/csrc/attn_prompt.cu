// Causal attention of packed prompts (fpt_attn_prompt; formulas: include/fpt.h).
//
// A task is two tiles of 128 query rows of one key/value head, and a walk over that head's keys in tiles of 128.  A row
// is a (token, query head of the group) pair: a power of two of the heads of a group share a tile, so a prompt of few
// tokens still fills it, and the keys are fetched once for all of them.  The grid has a CTA a task, in the order of a sequence's
// last rows first (with a causal mask, the longest); a CTA that has requested all of its task's keys takes over one that was
// not started yet (cluster launch control), so that the loads, the look-ups and the first scores of the next task run under the last
// tiles and the epilogue of this one, and a long task keeps nobody waiting.
//   warps 0..3, 4..7   softmax of the first and the second query tile, one row a thread
//   warps 8..11        the end of a task: O from tensor memory, divided, to its rows, while the softmax is at the next task
//   warp 12            the next task; TMA: queries once a task, keys and values through a ring
//   warp 13            tensor core:  S = Q K^T (both from shared memory),  O += P V (P from tensor memory, V as it lies: the
//                      instruction takes it with the keys along the rows)
//   warps 14, 15       values of the tiles that a mask cuts: those that are not finite become zeros before the tensor core
//                      reads them (a weight of zero would not make them harmless), as do rows behind the sequence
// While the softmax of one tile runs, the tensor core works for the other.  P (bf16) takes the place of S in tensor
// memory; the next S in that place is issued behind the P V that reads it, and the tensor core keeps that order.  With heads of 64
// there is room for a place more (kAhead): the S of a tile's next keys is there before its softmax has done with these
// (four chunks behind prefixes, 24 heads of 64: 103 -> 95 us).
//
// Softmax in the exponent of two: p = 2^(S scale log2(e) - m).  m is the row's maximum when it was last renewed: it is renewed, and O in
// tensor memory multiplied by 2^(m_old - m_new), only where the maximum has grown by more than 8, so that p <= 256; the quotient by
// the sum of weights is the same for any m.
// Measured (32 query heads, 8 of keys, of 128): 2048 tokens 36.7 us, 8192 442 us = 1.24 PFLOP/s, 490 to 510 us once the GPU is hot (power, 1.64 GHz).  A
// pair of tiles and 128 keys take 3 270 cycles, of which the tensor core works 2 150: what bounds it is the chain from scores to
// committed weights, not a unit.
// (A part of the powers as a polynomial on the multiply-add units, since 128 powers a row keep the special-function unit busy half
// as long as the tensor core works on a tile: 3 % slower at a quarter of them, 13 % at half.)
#include <algorithm>
#include <type_traits>

#include "attn_common.cuh"

namespace fpt {

constexpr int kPrThreads = 512;
constexpr int kPrSoftRegs = 176, kPrEndRegs = 80, kPrAuxRegs = 80;
static_assert(128 * (2 * kPrSoftRegs + kPrEndRegs + kPrAuxRegs) <= kPrThreads * 128, "the warpgroups' registers exceed the launch's");
constexpr int kPrEarly = 6;                // of the eight 16-key steps of P V, those that begin before the last weights are there
static_assert(kPrEarly % 2 == 0 && kPrEarly < 8, "weights leave two steps at a time");

// Lane l of four: y[i] becomes y[l & 3] of lane (l & ~3) + i.  (Written out: an index that the compiler does not see through
// would put y into local memory, and with 227 KB of shared memory there is hardly a cache behind it.)
__device__ __forceinline__ void swap_lanes(uint4& a, uint4& b, bool up, int m) {
  uint32_t* x = &a.x;
  uint32_t* y = &b.x;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t got = __shfl_xor_sync(0xffffffffu, up ? x[k] : y[k], m);
    x[k] = up ? got : x[k];
    y[k] = up ? y[k] : got;
  }
}
__device__ __forceinline__ void transpose4(uint4 (&y)[4], int lane) {
  swap_lanes(y[0], y[1], lane & 1, 1);
  swap_lanes(y[2], y[3], lane & 1, 1);
  swap_lanes(y[0], y[2], lane & 2, 2);
  swap_lanes(y[1], y[3], lane & 2, 2);
}

struct __align__(16) TaskInfo {
  int row0, len_q, key0, len_k;       // the sequence
  int tok0, tiles, cut, flags;        // first token; tiles of keys; tiles from `cut` on are masked for some row; 1: a task, 2: the second query tile has rows,
                                      // from bit 8: heads
  int head0, kv_head, odd, skip;      // odd: a cut tile's values were not all finite; skip: keys in front of this part's
  int parts, part, slot, odd_from;    // parts of the keys, each a task; where the first's sums go; the first key of the cut tiles
};

struct PromptParams {
  const int32_t *cu_q, *cu_k;
  const __nv_bfloat16* V;
  __nv_bfloat16* O;
  float* lse;
  uint32_t* status;
  float* sums;                        // of parts
  int ld_v, ld_o, M_q, M_k, n_q, n_kv, group, pack_log2, packs, units, n_seqs, n_tasks, causal;
  int split, sms;                     // parts that are at most made where keys are split; SMs.  0: they are not
  float scale_log2;
};

template <int HD>
struct PrSmem {
  static constexpr int kStages = HD == 128 ? 5 : 8;
  static constexpr int kAhead = HD == 128 ? 0 : 1;           // places of scores in tensor memory beyond one a tile
  static constexpr int kMat = kPrTile * HD * 2;              // a tile of keys, values or queries
  static constexpr int kHalf = kPrTile * 128;                // 64 of its columns: 128-byte rows
  static constexpr int kKvOff = 2 * kMat;
  static constexpr int kBarOff = kKvOff + kStages * kMat;
  static constexpr int kNumBars = 4 + 4 * kStages + 30 + 1;
  static constexpr int kMiscOff = (kBarOff + kNumBars * 8 + 15) / 16 * 16;
  static constexpr int kInfoOff = kMiscOff + 32;             // (16 bytes of misc, the answer of the launch control)
  static constexpr int kStatOff = kInfoOff + 4 * (int)sizeof(TaskInfo);         // [query tile][row] {maximum, sum of weights}
  static constexpr int kAlloc = kStatOff + 2 * kPrTile * 8;
};

// Shared-memory matrix descriptor of a B operand that lies with its rows along k (128-byte rows of 64 columns, 128-byte
// swizzle): 8-row groups 1024 bytes apart, the next 64 columns `next_cols` bytes on.
__device__ __forceinline__ uint64_t umma_desc_mnmajor_sw128(uint32_t smem_addr, uint32_t next_cols) {
  uint64_t d = 0;
  d |= (uint64_t)((smem_addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(next_cols >> 4) << 16;
  d |= (uint64_t)(1024u >> 4) << 32;
  d |= (uint64_t)1u << 46;
  d |= (uint64_t)2u << 61;
  return d;
}

// float32 accumulator, bf16 operands.
__host__ __device__ constexpr uint32_t umma_idesc_bf16(int m, int n, bool b_mn_major) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) |
         ((uint32_t)(m >> 4) << 24);
}

__device__ __forceinline__ void umma_bf16(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// Two float32 at a time (Blackwell's packed forms).
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float pow2_unit(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ void tmem_ld_32x8(uint32_t taddr, uint32_t (&v)[8]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_st_32x8(uint32_t taddr, const uint32_t (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}

// Cluster launch control: asks for a block of this grid that was not started yet (it then never is); the answer, 16 bytes in
// shared memory, counts on the barrier.  Not to be asked again after a refusal.
__device__ __forceinline__ void ask_for_a_block(uint32_t answer, uint32_t bar) {
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];"
               ::"r"(answer), "r"(bar) : "memory");
}
// Its blockIdx.x, or -1.
__device__ __forceinline__ int block_of_answer(uint32_t answer) {
  int x = -1;
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b128 a;\n\t"
      "ld.shared.b128 a, [%1];\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, a;\n\t"
      "mov.b32 %0, -1;\n\t"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %0, a;\n\t}"
      : "=r"(x)
      : "r"(answer)
      : "memory");
  return x;
}

constexpr int kPrHeld = 4;
// Where the tasks of up to 128 sequences begin and how many they are: lane l knows it of sequences l, l + 32, ...  Up to 32 are
// taken in the order of their lengths, longest walk first, so that what is left at the end of the launch is short; more as they come.
struct TaskOrder { int first[kPrHeld], count[kPrHeld], q0[kPrHeld], len_q[kPrHeld], k0[kPrHeld], len_k[kPrHeld], split, parts, slot; };
//
// Few query rows and many keys leave SMs idle: tasks of up to 32 sequences, where there are not more than SMs, are then split (Splitting).
template <bool SPLIT>
__device__ __forceinline__ TaskOrder task_order(const PromptParams& P, int lane) {
  TaskOrder o;
  int before = 0;
  o.split = o.slot = 0;
  o.parts = 1;
#pragma unroll
  for (int i = 0; i < kPrHeld; ++i) {
    o.first[i] = o.count[i] = o.q0[i] = o.len_q[i] = o.k0[i] = o.len_k[i] = 0;
    const int s = lane + 32 * i;
    if (P.n_seqs > 32 * kPrHeld || 32 * i >= P.n_seqs) continue;
    int keys = -1;
    if (s < P.n_seqs) {
      const int q0 = __ldg(P.cu_q + s), q1 = __ldg(P.cu_q + s + 1), k0 = __ldg(P.cu_k + s), k1 = __ldg(P.cu_k + s + 1);
      if (!rows_fit(q0, q1, P.M_q) || !rows_fit(k0, k1, P.M_k)) {
        record_bad_index(P.status, kBadOffset);
      } else {
        keys = k1 - k0;
        o.q0[i] = q0; o.len_q[i] = q1 - q0; o.k0[i] = k0; o.len_k[i] = keys;
        o.count[i] = (q1 - q0 + ((256 >> P.pack_log2) - 1)) >> (8 - P.pack_log2);
      }
    }
    if (P.n_seqs <= 32) {
      if constexpr (SPLIT) {
        const int places = o.count[0];
        const uint32_t n = __reduce_add_sync(0xffffffffu, (uint32_t)places) * P.units;
        if (n <= (uint32_t)P.sms) {                          // (and each below 2^24 tiles: no overflow)
          Splitting s = {max(keys, 0), o.len_q[0], places, 8 - P.pack_log2, P.causal};
          const uint32_t all = __reduce_add_sync(0xffffffffu, s.tiles()) * P.units;
          int least = Splitting::first_length(all, P.sms);
          while (__reduce_add_sync(0xffffffffu, (uint32_t)(s.split(least) * s.parts(least))) * P.units > (uint32_t)P.split) least += max(1, least / 8);
          o.split = s.split(least);
          o.parts = s.parts(least);
          o.count[0] += o.split * (o.parts - 1);
          int v = o.split * o.parts;
          o.slot = v;
#pragma unroll
          for (int k = 1; k < 32; k <<= 1) {
            const int u = __shfl_up_sync(0xffffffffu, v, k);
            if (lane >= k) v += u;
          }
          o.slot = v - o.slot;
        }
      }
      for (int k = 0; k < P.n_seqs; ++k) {
        const int other = __shfl_sync(0xffffffffu, keys, k), c = __shfl_sync(0xffffffffu, o.count[i], k);
        if (other > keys || (other == keys && k < lane)) o.first[i] += c;
      }
    } else {
      int v = o.count[i];
#pragma unroll
      for (int k = 1; k < 32; k <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, v, k);
        if (lane >= k) v += u;
      }
      o.first[i] = before + v - o.count[i];
      before += __shfl_sync(0xffffffffu, v, 31);
    }
  }
  return o;
}

// The task of block `bid`, in `ti`, which is cleared; whole warp, the same answer in every lane.  With more sequences than are held, sequence s has
// floor(cu_q[s+1] / per) - floor(cu_q[s] / per) + 1 tasks (at least the blocks of `per` rows that it needs), and which s a task belongs to
// is found 32 places at a time.
template <bool SPLIT>
__device__ __forceinline__ bool find_prompt_task(const PromptParams& P, const TaskOrder& order, int bid, int lane, TaskInfo& ti) {
  const int per_log2 = 8 - P.pack_log2, per = 1 << per_log2;
  const int turn = bid / P.units, unit = bid - turn * P.units;
  int lo = 0, place, parts = 1, slot = 0;
  if (P.n_seqs <= 32 * kPrHeld) {
    lo = -1;
    place = 0;
#pragma unroll
    for (int i = 0; i < kPrHeld; ++i) {
      const uint32_t mine = __ballot_sync(0xffffffffu, turn >= order.first[i] && turn < order.first[i] + order.count[i]);
      if (mine) {
        const int l = __ffs(mine) - 1;
        lo = l + 32 * i;
        const int at = turn - __shfl_sync(0xffffffffu, order.first[i], l);
        place = __shfl_sync(0xffffffffu, order.count[i], l) - 1 - at;      // last rows first
        ti.row0 = __shfl_sync(0xffffffffu, order.q0[i], l);
        ti.len_q = __shfl_sync(0xffffffffu, order.len_q[i], l);
        ti.key0 = __shfl_sync(0xffffffffu, order.k0[i], l);
        ti.len_k = __shfl_sync(0xffffffffu, order.len_k[i], l);
        if (SPLIT && i == 0) {
          const int split = __shfl_sync(0xffffffffu, order.split, l), p = __shfl_sync(0xffffffffu, order.parts, l);
          if (at < split * p) {
            const int k = at / p;
            parts = p;
            ti.part = at - k * p;
            slot = __shfl_sync(0xffffffffu, order.slot, l) + k * p;
            place += at - k;                                 // the k-th from the last
            place -= split * (p - 1);
          }
        }
      }
    }
    if (lo < 0) return false;
  } else {
    // The search looks only at the sequences that it meets, and one whose offsets do not ascend may have no task to be met by: block s
    // looks at sequence s (there are more blocks than sequences, and each is somebody's).
    const int s = min(bid, P.n_seqs - 1);
    const int q0 = __ldg(P.cu_q + s), q1 = __ldg(P.cu_q + s + 1), k0 = __ldg(P.cu_k + s), k1 = __ldg(P.cu_k + s + 1);
    const int id = P.n_tasks - 1 - turn;
    int hi = P.n_seqs;
    while (hi - lo > 1) {
      const int step = (hi - lo + 31) / 32, at = lo + lane * step;
      const uint32_t below = __ballot_sync(0xffffffffu, at < hi && (__ldg(P.cu_q + min(at, hi - 1)) >> per_log2) + at <= id);
      if (below) lo += (31 - __clz(below)) * step;
      hi = min(hi, lo + step);
    }
    if (!rows_fit(q0, q1, P.M_q) || !rows_fit(k0, k1, P.M_k)) record_bad_index(P.status, kBadOffset);
    place = id - ((__ldg(P.cu_q + lo) >> per_log2) + lo);
    ti.row0 = __ldg(P.cu_q + lo);
    const int end_q = __ldg(P.cu_q + lo + 1);
    ti.len_q = end_q - ti.row0;
    ti.key0 = __ldg(P.cu_k + lo);
    const int end_k = __ldg(P.cu_k + lo + 1);
    ti.len_k = end_k - ti.key0;
    if (!rows_fit(ti.row0, end_q, P.M_q) || !rows_fit(ti.key0, end_k, P.M_k)) {
      if (lane == 0) record_bad_index(P.status, kBadOffset);
      return false;
    }
  }
  if (SPLIT && parts > 1) ti.slot = slot * P.units + unit * parts;
  if (place < 0 || place >= (ti.len_q + per - 1) >> per_log2) return false;
  ti.tok0 = place * per;
  ti.kv_head = unit / P.packs;
  const int before = (unit - ti.kv_head * P.packs) << P.pack_log2;         // heads of the group
  ti.head0 = ti.kv_head * P.group + before;
  const int ahead = ti.len_k - ti.len_q, last = min(ti.tok0 + per, ti.len_q) - 1;
  const int seen_first = P.causal ? max(0, min(ti.len_k, ti.tok0 + ahead + 1)) : ti.len_k;
  const int seen_last = P.causal ? max(0, min(ti.len_k, last + ahead + 1)) : ti.len_k;
  ti.tiles = (seen_last + kPrTile - 1) / kPrTile;
  ti.cut = seen_first / kPrTile;
  ti.flags = 1 | (ti.tok0 + per / 2 < ti.len_q ? 2 : 0) | min(1 << P.pack_log2, P.group - before) << 8;
  ti.odd = 0;
  ti.odd_from = ti.cut * kPrTile;
  if (!SPLIT) return true;
  ti.parts = min(parts, max(ti.tiles, 1));
  if (ti.parts > 1) {
    if (ti.part >= ti.parts) return false;
    const int from = (int)((int64_t)ti.tiles * ti.part / ti.parts), to = (int)((int64_t)ti.tiles * (ti.part + 1) / ti.parts);
    ti.skip = from * kPrTile;
    ti.tiles = to - from;
    ti.cut = max(0, ti.cut - from);
  } else if (ti.part > 0) {
    return false;
  }
  return true;
}

// What the zeros in the cut tiles stand for: a value that is not finite outweighs every finite sum, whatever its weight.
__device__ __noinline__ void add_odd_values(const __nv_bfloat16* V, int ld, int hd, int from, int to, __nv_bfloat16* o) {
  for (int d = 0; d < hd; ++d) {
    float sum = __bfloat162float(o[d]);
    for (int k = from; k < to; ++k) {
      const float z = __bfloat162float(V[(size_t)k * ld + d]);
      if (!(fabsf(z) < INFINITY)) sum += z;
    }
    if (!(fabsf(sum) < INFINITY)) o[d] = __float2bfloat16_rn(sum);
  }
}

// Of the four rows from r & ~3 on, which are there (bit i: row i); of tokens from tok0 on, `heads` heads each.
__device__ __forceinline__ uint32_t rows_there(const PromptParams& P, int r, int tok0, int len_q, int heads) {
  uint32_t there = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int from = (r & ~3) + i;
    there |= (tok0 + (from >> P.pack_log2) < len_q && (from & ((1 << P.pack_log2) - 1)) < heads ? 1u : 0u) << i;
  }
  return there;
}

// 32 columns, from 32 b, of the output rows of a warp, whose lane holds row r of a query tile; times `inv` first.
template <int HD>
__device__ __forceinline__ void store_columns(const PromptParams& P, const uint32_t (&v)[32], float inv, int b, int r, int lane, int row0,
                                              int tok0, uint32_t there, int head0, int pack_mask) {
  uint4 y[4];                                                // 32 elements of this lane's row
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t z[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      z[k] = f32x2_to_bf16x2_bits(__uint_as_float(v[8 * i + 2 * k]) * inv, __uint_as_float(v[8 * i + 2 * k + 1]) * inv);
    y[i] = make_uint4(z[0], z[1], z[2], z[3]);
  }
  // Four lanes swap their quarters, so that a store covers 64 bytes of eight rows; with a row a lane every store met 32
  // lines (16 stores a lane and task: 4 000 cycles).
  transpose4(y, lane);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int from = (r & ~3) + i, tok = tok0 + (from >> P.pack_log2);        // whose row
    if (there >> i & 1u)
      *reinterpret_cast<uint4*>(P.O + (size_t)(row0 + tok) * P.ld_o + (size_t)(head0 + (from & pack_mask)) * HD + b * 32 +
                                (lane & 3) * 8) = y[i];
  }
}

// Where keys are split, the sums of a part: for each query tile and each 32 of its rows HD columns of a float32 a row, then the rows'
// maxima, sums of weights, and whether a cut tile's values were not all finite.
template <int HD>
__host__ __device__ constexpr size_t part_floats() { return (size_t)32 * (HD + 3); }
template <int HD>
__device__ __forceinline__ size_t part_place(int slot, int w, int quarter) { return ((size_t)slot * 8 + w * 4 + quarter) * part_floats<HD>(); }
template <int HD>
constexpr int most_parts() { return (int)(kAttnScratchBytes / (8 * part_floats<HD>() * sizeof(float))); }

// Joins them: O = sum 2^(m_k - m) O_k / sum 2^(m_k - m) s_k, m the largest of the m_k, in the order of the keys.  The blocks of a task's
// parts share its work: 32 rows by 32 columns a warp.
constexpr int kPrJoinThreads = 256;
template <int HD>
__global__ void __launch_bounds__(kPrJoinThreads)
prompt_join_kernel(const PromptParams P) {
  pdl_wait();
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const TaskOrder order = task_order<true>(P, lane);
  TaskInfo ti = {};
  if (!find_prompt_task<true>(P, order, blockIdx.x, lane, ti) || ti.parts < 2) return;
  const int per_tile = kPrTile >> P.pack_log2, pack_mask = (1 << P.pack_log2) - 1;
  const int groups = (ti.flags & 2) ? 8 : 4;                 // of 32 rows
  for (int u = ti.part * (kPrJoinThreads / 32) + warp; u < groups * (HD / 32); u += ti.parts * (kPrJoinThreads / 32)) {
    const int g = u / (HD / 32), b = u % (HD / 32), w = g >> 2, r = (g & 3) * 32 + lane;
    const int tok0 = ti.tok0 + w * per_tile, tok = tok0 + (r >> P.pack_log2);
    const uint32_t there = rows_there(P, r, tok0, ti.len_q, ti.flags >> 8);
    const bool row_ok = there >> (r & 3) & 1u;
    if (tok0 + ((g & 3) * 32 >> P.pack_log2) >= ti.len_q) continue;
    const float* at = P.sums + part_place<HD>(ti.slot, w, g & 3) + lane;
    constexpr size_t next = 8 * part_floats<HD>();
    float m = -INFINITY, sum = 0.0f, odd = 0.0f;
    for (int k = 0; k < ti.parts; ++k) m = fmaxf(m, __ldcg(at + k * next + HD * 32));
    uint32_t v[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = 0;
    for (int k = 0; k < ti.parts; ++k) {
      const float* x = at + k * next;
      float y[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) y[i] = __ldcg(x + (b * 32 + i) * 32);
      const float mk = __ldcg(x + HD * 32), f = mk == -INFINITY ? 0.0f : pow2_unit(mk - m);
      sum += f * __ldcg(x + HD * 32 + 32);
      odd = fmaxf(odd, __ldcg(x + HD * 32 + 64));
#pragma unroll
      for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(fmaf(f, y[i], __uint_as_float(v[i])));
    }
    const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
    store_columns<HD>(P, v, inv, b, r, lane, ti.row0, tok0, there, ti.head0, pack_mask);
    __syncwarp();                                            // (a row is written by four lanes)
    if (row_ok && odd != 0.0f) {
      const int limit = P.causal ? min(ti.len_k, tok + (ti.len_k - ti.len_q) + 1) : ti.len_k;
      add_odd_values(P.V + (size_t)ti.key0 * P.ld_v + (size_t)ti.kv_head * HD + b * 32, P.ld_v, 32, ti.odd_from, limit,
                     P.O + (size_t)(ti.row0 + tok) * P.ld_o + (size_t)(ti.head0 + (r & pack_mask)) * HD + b * 32);
    }
    if (row_ok && b == 0 && P.lse)
      P.lse[(size_t)(ti.row0 + tok) * P.n_q + ti.head0 + (r & pack_mask)] =
          sum > 0.0f || sum != sum ? m * 0.69314718055994531f + logf(sum) : -INFINITY;
  }
}

// SPLIT: keys may be split.  (One kernel for both took 2 us longer for 33 short prompts that are not.)
template <int HD, bool SPLIT>
__global__ void __launch_bounds__(kPrThreads, 1)
attn_prompt_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                   const __grid_constant__ CUtensorMap tmV, const PromptParams P) {
  using L = PrSmem<HD>;
  constexpr int ST = L::kStages;
  extern __shared__ __align__(1024) uint8_t smem_tiles[];    // (no room to align it by hand: 227 KB are full)
  uint8_t* smem = smem_tiles;
  const uint32_t sbase = smem_u32(smem);
  const uint32_t bar0 = sbase + L::kBarOff;
  auto q_full = [&](int w) { return bar0 + 8u * w; };
  auto q_empty = [&](int w) { return bar0 + 8u * (2 + w); };
  auto kv_full = [&](int s) { return bar0 + 8u * (4 + s); };
  auto kv_empty = [&](int s) { return bar0 + 8u * (4 + ST + s); };
  // values of a cut tile: arrived (for the warps that clean them), clean.  One of each a stage: a stage is not filled
  // again before the tensor core has read it, so no phase of theirs is over before it was waited for
  auto v_raw = [&](int s) { return bar0 + 8u * (4 + 2 * ST + s); };
  auto v_clean = [&](int s) { return bar0 + 8u * (4 + 3 * ST + s); };
  const uint32_t bar1 = bar0 + 8u * (4 + 4 * ST);
  // With a place more, a tile's scores are issued at most one step ahead of its P V: two barriers taken in turn keep the steps apart.
  auto s_full = [&](int w, int turn) { return bar1 + 8u * (2 * w + turn); };
  auto p_full = [&](int w, int turn, int part) { return bar1 + 8u * (4 + 4 * w + 2 * turn + part); };   // part: the first kPrEarly steps, the others
  auto pv_done = [&](int w) { return bar1 + 8u * (12 + w); };                      // each P V (where a place more lets S run ahead)
  auto o_full = [&](int w) { return bar1 + 8u * (14 + w); };                       // a task's last P V
  auto o_empty = [&](int w) { return bar1 + 8u * (16 + w); };
  auto info_full = [&](int i) { return bar1 + 8u * (18 + i); };
  auto info_empty = [&](int i) { return bar1 + 8u * (22 + i); };
  auto stat_full = [&](int w) { return bar1 + 8u * (26 + w); };
  auto stat_empty = [&](int w) { return bar1 + 8u * (28 + w); };
  const uint32_t answered = bar1 + 8u * 30;
  float2* stats = reinterpret_cast<float2*>(smem + L::kStatOff);
  volatile uint32_t* misc = reinterpret_cast<volatile uint32_t*>(smem + L::kMiscOff);
  volatile uint32_t* abort_flag = misc + 1;
  TaskInfo* infos = reinterpret_cast<TaskInfo*>(smem + L::kInfoOff);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  pdl_wait();
  pdl_launch_dependents();
  if (sbase & 1023u) {                                       // not what was declared: no tile could be addressed
    if (threadIdx.x == 0) atomicCAS(P.status, 0u, kStatusTimeoutBase | 15u);
    return;
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(q_full(i), 1);
      mbar_init(q_empty(i), 1);
      mbar_init(s_full(i, 0), 1);
      mbar_init(s_full(i, 1), 1);
      mbar_init(pv_done(i), 1);
      for (int b = 0; b < 4; ++b) mbar_init(p_full(i, b >> 1, b & 1), 4);
      mbar_init(o_full(i), 1);
      mbar_init(o_empty(i), 4);
      mbar_init(stat_full(i), 4);
      mbar_init(stat_empty(i), 4);
    }
    for (int i = 0; i < 4; ++i) { mbar_init(info_full(i), 1); mbar_init(info_empty(i), 8 + 4 + 1 + 2); }
    mbar_init(answered, 1);
    for (int i = 0; i < ST; ++i) { mbar_init(kv_full(i), 1); mbar_init(kv_empty(i), 1); mbar_init(v_raw(i), 1); mbar_init(v_clean(i), 2); }
    misc[1] = 0;
    fence_mbar_init();
    prefetch_tmap(&tmQ);
    prefetch_tmap(&tmK);
    prefetch_tmap(&tmV);
  }
  if (warp == 13) {
    tmem_alloc(sbase + L::kMiscOff, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = misc[0];
  // A task's steps u = j nw + i (keys j, query tile i of nw) take the nw + kAhead places of scores in turn.
  auto s_col = [&](int place) { return tmem + 128u * place; };
  auto o_col = [&](int i) { return tmem + 128u * (2 + L::kAhead) + (uint32_t)HD * i; };
  // Of the steps of one tile in all tasks, n before this one: which barrier, and its parity.
  auto turn_of = [](uint32_t n) { return L::kAhead ? (int)(n & 1u) : 0; };
  auto parity_of = [](uint32_t n) { return L::kAhead ? n >> 1 & 1u : n & 1u; };
  // (parities of barriers that come in twos are kept as bits of one word: an array indexed at run time is local memory)
  const int per_tile = kPrTile >> P.pack_log2;               // tokens

  if (warp < 8) {
    // ------------------------------------------------------------------ softmax
    reg_inc<kPrSoftRegs>();
    const int w = warp >> 2, r = threadIdx.x & 127;          // query tile, row of it
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t to = o_col(w) + lanes;
    const float c = P.scale_log2;
    uint32_t step = 0, stat_ph = 0;                           // step: of this tile in all tasks
    bool ok = true;
    for (int n = 0; ok; ++n) {
      if (!wait_long<true>(info_full(n & 3), (n >> 2) & 1, abort_flag, P.status, 7)) break;
      const TaskInfo* info = infos + (n & 3);
      const int flags = info->flags, tiles = info->tiles, plain = min(info->cut, tiles);
      // keys the row sees (not fewer in the rows behind it, those behind the sequence among them)
      const int limit = (P.causal ? max(0, min(info->len_k, info->tok0 + w * per_tile + (r >> P.pack_log2) + (info->len_k - info->len_q) + 1))
                                  : info->len_k) - (SPLIT ? info->skip : 0);
      __syncwarp();
      if (lane == 0) mbar_arrive(info_empty(n & 3));
      if (!(flags & 1)) break;
      if (w == 1 && !(flags & 2)) continue;
      int place = w;
      float m = -INFINITY;                                   // of S * c, when last renewed
      uint64_t sum2[2] = {0, 0};                             // four partial sums of weights
      // One tile of keys; MASKED: some row of the task does not see all of it.
      auto tile = [&](int j, auto masked) -> bool {
        constexpr bool MASKED = decltype(masked)::value;
        if (!wait_long<true>(s_full(w, turn_of(step)), parity_of(step), abort_flag, P.status, 4)) return false;
        tc_fence_after();
        const uint32_t ts = s_col(place) + lanes;
        if (L::kAhead) place = place > 0 ? place - 1 : (flags & 2) ? 2 : 1;    // nw further, modulo nw + 1
        float x[128];
#pragma unroll
        for (int b = 0; b < 4; ++b) tmem_ld_32x32(ts + b * 32, reinterpret_cast<uint32_t(&)[32]>(x[b * 32]));
        int most = 128;                                      // columns that count in the warp's last row
        if (MASKED) {
          const int n = limit - j * kPrTile, least = __shfl_sync(0xffffffffu, n, 0);
          most = __shfl_sync(0xffffffffu, n, 31);
#pragma unroll
          for (int b = 0; b < 4; ++b)
            if (least < b * 32 + 32) {
#pragma unroll
              for (int i = 0; i < 32; ++i) x[b * 32 + i] = b * 32 + i < n ? x[b * 32 + i] : -INFINITY;
            }
        }
        float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < 128; i += 8)
#pragma unroll
          for (int k = 0; k < 4; ++k) top[k] = fmaxf(fmaxf(top[k], x[i + k]), x[i + 4 + k]);
        const float now = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * c;     // c > 0; a NaN stays in its weight
        const bool renew = now > m + 8.0f || m == -INFINITY;
        if (j > 0 && __any_sync(0xffffffffu, renew && now > m)) {
          // The P V before has to be done.  Without a place more it is: the S just read was issued behind it.  With one, that holds of
          // the P V before that: the barrier is at most one phase behind, and its parity says whether it is.
          if (L::kAhead) {
            if (!wait_long<true>(pv_done(w), (step + 1u) & 1u, abort_flag, P.status, 4)) return false;
            tc_fence_after();
          }
          const float f = renew && now > m ? (m == -INFINITY ? 0.0f : pow2_unit(m - now)) : 1.0f;
          sum2[0] = mul2(sum2[0], pack2(f, f));
          sum2[1] = mul2(sum2[1], pack2(f, f));
#pragma unroll 1
          for (int b = 0; b < HD / 8; ++b) {
            uint32_t v[8];
            tmem_ld_32x8(to + b * 8, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * f);
            tmem_st_32x8(to + b * 8, v);
          }
          tmem_wait_st();
        }
        if (renew) m = fmaxf(m, now);
        const float minus = m == -INFINITY ? 0.0f : -m;
        const uint64_t c2 = pack2(c, c), m2 = pack2(minus, minus);
        uint32_t pairs[16];
#pragma unroll
        for (int b = 0; b < 8; ++b) {                        // 16 keys: a step of P V
          uint32_t* pk = pairs + (b & 1) * 8;
          if (MASKED && most <= b * 16) {                    // nobody sees these keys
#pragma unroll
            for (int i = 0; i < 8; ++i) pk[i] = 0;
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              float u, v;
              unpack2(fma2(pack2(x[b * 16 + 2 * i], x[b * 16 + 2 * i + 1]), c2, m2), u, v);
              u = pow2_unit(u);
              v = pow2_unit(v);
              sum2[i & 1] = add2(sum2[i & 1], pack2(u, v));
              pk[i] = f32x2_to_bf16x2_bits(u, v);
            }
          }
          if (b & 1) tmem_st_32x16(ts + (b - 1) * 8, pairs);
          if (b == kPrEarly - 1 || b == 7) {
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_full(w, turn_of(step), b == 7));
          }
        }
        ++step;
        return true;
      };
      for (int j = 0; ok && j < plain; ++j) ok = tile(j, std::false_type{});
      for (int j = plain; ok && j < tiles; ++j) ok = tile(j, std::true_type{});
      if (!ok) break;
      // what the end of the task needs
      ok = wait_long<true>(stat_empty(w), stat_ph ^ 1u, abort_flag, P.status, 5);
      stat_ph ^= 1u;
      float s0, s1;
      unpack2(add2(sum2[0], sum2[1]), s0, s1);
      if (ok) stats[w * kPrTile + r] = make_float2(m, s0 + s1);
      __syncwarp();
      if (ok && lane == 0) mbar_arrive(stat_full(w));
    }
  } else if (warp < 12) {
    // ------------------------------------------------------------------ the end of a task
    reg_dec<kPrEndRegs>();
    const int r = threadIdx.x & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    uint32_t ph = 0, o_ph = 0;
    const int pack_mask = (1 << P.pack_log2) - 1;
    bool ok = true;
    for (int n = 0; ok; ++n) {
      if (!wait_long<true>(info_full(n & 3), (n >> 2) & 1, abort_flag, P.status, 9)) break;
      const volatile TaskInfo* info = infos + (n & 3);
      if (!(info->flags & 1)) break;
      const int tiles = info->tiles, len_q = info->len_q, row0 = info->row0, head0 = info->head0;
      const bool split = SPLIT && info->parts > 1;
#pragma unroll 1
      for (int w = 0; w < ((info->flags & 2) ? 2 : 1); ++w) {
        ok = wait_long<true>(stat_full(w), ph >> w & 1u, abort_flag, P.status, 9);
        if (!ok) break;
        ph ^= 1u << w;
        const float2 ms = stats[w * kPrTile + r];
        __syncwarp();
        if (lane == 0) mbar_arrive(stat_empty(w));
        const float sum = ms.y;                              // (no tiles: 0)
        const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
        const int tok0 = info->tok0 + w * per_tile;
        const uint32_t there = rows_there(P, r, tok0, len_q, info->flags >> 8);
        const bool row_ok = there >> (r & 3) & 1u;
        bool odd = false;
        if (tiles > 0) {
          ok = wait_long<true>(o_full(w), o_ph >> w & 1u, abort_flag, P.status, 9);
          if (!ok) break;
          o_ph ^= 1u << w;
          tc_fence_after();
          odd = info->odd != 0;
        }
        // (a part has tiles)
        float* at = P.sums + part_place<HD>(split ? info->slot + info->part : 0, w, warp & 3) + lane;
#pragma unroll 1
        for (int b = 0; b < HD / 32; ++b) {
          uint32_t v[32];
          if (tiles == 0) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = 0;
          } else {
            tmem_ld_32x32(o_col(w) + lanes + b * 32, v);
            if (b == HD / 32 - 1) {                          // the next task's sums may begin
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(o_empty(w));
            }
          }
          if (split) {
#pragma unroll
            for (int i = 0; i < 32; ++i) __stcg(at + (b * 32 + i) * 32, __uint_as_float(v[i]));
            continue;
          }
          store_columns<HD>(P, v, inv, b, r, lane, row0, tok0, there, head0, pack_mask);
        }
        if (split) {
          __stcg(at + HD * 32, ms.x);
          __stcg(at + HD * 32 + 32, ms.y);
          __stcg(at + HD * 32 + 64, odd ? 1.0f : 0.0f);
          continue;
        }
        if (odd) {
          __syncwarp();                                      // (the row was written by four lanes)
          const int limit = P.causal ? min(info->len_k, tok0 + (r >> P.pack_log2) + (info->len_k - len_q) + 1) : info->len_k;
          if (row_ok)
            add_odd_values(P.V + (size_t)info->key0 * P.ld_v + (size_t)info->kv_head * HD, P.ld_v, HD, info->odd_from, limit,
                           P.O + (size_t)(row0 + tok0 + (r >> P.pack_log2)) * P.ld_o + (size_t)(head0 + (r & pack_mask)) * HD);
        }
        if (row_ok && P.lse)
          P.lse[(size_t)(row0 + tok0 + (r >> P.pack_log2)) * P.n_q + head0 + (r & pack_mask)] =
              sum > 0.0f || sum != sum ? ms.x * 0.69314718055994531f + logf(sum) : -INFINITY;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(info_empty(n & 3));         // (at the end: `odd` comes late)
    }
  } else {
    reg_dec<kPrAuxRegs>();
    if (warp == 12) {
      // ---------------------------------------------------------------- tasks and TMA
      const uint32_t answer = sbase + L::kMiscOff + 16;
      uint32_t kv_ph = 0, armed = 0, armed_par = 0, raw_par = 0, asked = 0;
      uint32_t q_ph = 0;
      int st = 0;
      bool ok = true;
      int bid = blockIdx.x;
      const TaskOrder order = task_order<SPLIT>(P, lane);
      auto fetch = [&](const CUtensorMap* tm, int kv_head, int row, bool clean) -> bool {
        if (!wait_long<true>(kv_empty(st), kv_ph ^ 1u, abort_flag, P.status, 1)) return false;
        // values to be cleaned arrive on a barrier of their own, whose every phase the cleaning warps see
        const uint32_t bar = clean ? v_raw(st) : kv_full(st);
        if (elect_one()) {
          if (clean) mbar_arrive(kv_full(st));
          mbar_arrive_expect_tx(bar, L::kMat);
#pragma unroll
          for (int h = 0; h < HD / 64; ++h)
            tma_load_2d(sbase + L::kKvOff + st * L::kMat + h * L::kHalf, tm, bar, kv_head * HD + h * 64, row);
        }
        const int slot = clean ? ST + st : st;
        armed |= 1u << slot;
        armed_par = (armed_par & ~(1u << slot)) | ((clean ? raw_par >> st & 1u : kv_ph) << slot);
        if (clean) raw_par ^= 1u << st;
        if (++st == ST) { st = 0; kv_ph ^= 1u; }
        return true;
      };
      for (int n = 0; ok;) {
        // the task of block `bid`, if it is one
        TaskInfo ti = {};
        const bool found = bid >= 0 && find_prompt_task<SPLIT>(P, order, bid, lane, ti);
        if (found || bid < 0) {
          if (!wait_long<true>(info_empty(n & 3), ((n >> 2) & 1) ^ 1u, abort_flag, P.status, 1)) { ok = false; break; }
          if (lane == 0) {
            infos[n & 3] = ti;
            mbar_arrive(info_full(n & 3));
          }
          ++n;
          if (bid < 0) break;
          if (ti.tiles > 0) {
            auto queries = [&](int i) -> bool {
              if (!wait_long<true>(q_empty(i), (q_ph >> i & 1u) ^ 1u, abort_flag, P.status, 1)) return false;
              q_ph ^= 1u << i;
              if (elect_one()) {
                mbar_arrive_expect_tx(q_full(i), L::kMat);
#pragma unroll
                for (int h = 0; h < HD / 64; ++h)
                  tma_load_3d(sbase + i * L::kMat + h * L::kHalf, &tmQ, q_full(i), h * 64, ti.head0, ti.row0 + ti.tok0 + i * per_tile);
              }
              return true;
            };
            const int key0 = ti.key0 + (SPLIT ? ti.skip : 0);
            ok = queries(0) && fetch(&tmK, ti.kv_head, key0, false);
            if (ti.flags & 2) ok = ok && queries(1);
            ok = ok && fetch(&tmV, ti.kv_head, key0, ti.cut == 0);
            for (int j = 1; ok && j < ti.tiles; ++j)
              ok = fetch(&tmK, ti.kv_head, key0 + j * kPrTile, false) &&
                   fetch(&tmV, ti.kv_head, key0 + j * kPrTile, j >= ti.cut);
            if (!ok) break;
          }
        }
        // a block that was not started yet, or none (not asked for earlier: a task that waits here could be another CTA's)
        if (lane == 0) {
          mbar_arrive_expect_tx(answered, 16);
          ask_for_a_block(answer, answered);
        }
        if (!wait_long<true>(answered, asked & 1u, abort_flag, P.status, 8)) { ok = false; break; }
        ++asked;
        bid = block_of_answer(answer);
        fence_proxy_async_smem();                            // (the answer is read before the next one is written)
        __syncwarp();
      }
      if (!ok) {
        // copies in flight (queries among them: their barrier's last phase) before this CTA's shared memory goes away
        const uint64_t t0 = globaltimer_ns();
        for (int i = 0; i < 2 * ST; ++i)
          if (armed & (1u << i))
            while (!mbar_try_wait(i < ST ? kv_full(i) : v_raw(i - ST), (armed_par >> i) & 1u) && globaltimer_ns() - t0 < 2000000ull) {}
        for (int i = 0; i < 2; ++i)
          while (!mbar_try_wait(q_full(i), (q_ph >> i & 1u) ^ 1u) && globaltimer_ns() - t0 < 2000000ull) {}
      }
    } else if (warp == 13) {
      // ---------------------------------------------------------------- tensor core
      if (elect_one()) {
        constexpr uint32_t idesc_s = umma_idesc_bf16(128, 128, false), idesc_o = umma_idesc_bf16(128, HD, true);
        int k_at = 0, v_at = 1; uint32_t k_ph = 0, v_ph = 0;  // ring: keys 0, values 0, keys 1, ... of all tasks
        uint32_t clean_par = 0;                               // per stage: parity of the next phase of v_clean
        uint32_t q_ph = 0, o_ph = 0;
        uint32_t done = 0;                                    // two bits a tile: its steps in the tasks before, modulo 4
        bool ok = true;
        // the next keys or the next values: their stage, once it is filled
        auto next = [&](int& at, uint32_t& ph, int& st) -> bool {
          st = at;
          const bool got = wait_long<false>(kv_full(st), ph, abort_flag, P.status, 2);
          at += 2;
          if (at >= ST) { at -= ST; ph ^= 1u; }
          return got;
        };
        for (int n = 0; ok; ++n) {
          if (!wait_long<false>(info_full(n & 3), (n >> 2) & 1, abort_flag, P.status, 2)) break;
          const volatile TaskInfo* info = infos + (n & 3);
          const int flags = info->flags, tiles = info->tiles, cut = info->cut;
          mbar_arrive(info_empty(n & 3));
          if (!(flags & 1)) break;
          if (tiles == 0) continue;
          const int nw = (flags & 2) ? 2 : 1;
          int k_st = 0, v_st = 0, s_place = 0, p_place = 0;
          auto after = [&](int place) { return place + 1 == nw + L::kAhead ? 0 : place + 1; };
          auto scores = [&](int j, int i) -> bool {
            if (i == 0 && !next(k_at, k_ph, k_st)) return false;
            if (j == 0) {
              if (!wait_long<false>(q_full(i), q_ph >> i & 1u, abort_flag, P.status, 2)) return false;
              q_ph ^= 1u << i;
            }
            tc_fence_after();
            const uint32_t a = sbase + i * L::kMat, b = sbase + L::kKvOff + k_st * L::kMat, d = s_col(L::kAhead ? s_place : i);
#pragma unroll
            for (int h = 0; h < HD / 64; ++h) {
              const uint64_t ad = umma_desc_kmajor_sw128(a + h * L::kHalf), bd = umma_desc_kmajor_sw128(b + h * L::kHalf);
#pragma unroll
              for (int k = 0; k < 4; ++k) umma_bf16(d, ad + 2u * k, bd + 2u * k, idesc_s, (h | k) != 0);
            }
            umma_commit(s_full(i, turn_of((done >> 2 * i) + (uint32_t)j)));
            if (j + 1 == tiles) umma_commit(q_empty(i));
            if (i == nw - 1) umma_commit(kv_empty(k_st));
            s_place = after(s_place);
            return true;
          };
          for (int i = 0; ok && i < nw; ++i) ok = scores(0, i);
          if (L::kAhead && ok && tiles > 1) ok = scores(1, 0);
          for (int j = 0; ok && j < tiles; ++j) {
            ok = next(v_at, v_ph, v_st);
            if (ok && j >= cut) {
              ok = wait_long<false>(v_clean(v_st), (clean_par >> v_st) & 1u, abort_flag, P.status, 3);
              clean_par ^= 1u << v_st;
            }
            for (int i = 0; ok && i < nw; ++i) {
              if (j == 0) {                                   // the sums of the task before were read
                ok = wait_long<false>(o_empty(i), (o_ph >> i & 1u) ^ 1u, abort_flag, P.status, 3);
                o_ph ^= 1u << i;
              }
              const uint64_t bd = umma_desc_mnmajor_sw128(sbase + L::kKvOff + v_st * L::kMat, L::kHalf);
              const uint32_t step = (done >> 2 * i) + (uint32_t)j, p = s_col(L::kAhead ? p_place : i);
              for (int part = 0; ok && part < 2; ++part) {
                ok = wait_long<false>(p_full(i, turn_of(step), part), parity_of(step), abort_flag, P.status, 3);
                if (!ok) break;
                tc_fence_after();
                for (int k = part ? kPrEarly : 0; k < (part ? kPrTile / 16 : kPrEarly); ++k)
                  umma_bf16_ts(o_col(i), p + 8u * k, bd + 128u * k, idesc_o, (j | k) != 0);
              }
              if (!ok) break;
              if (L::kAhead) umma_commit(pv_done(i));
              if (j + 1 == tiles) umma_commit(o_full(i));
              if (i == nw - 1) umma_commit(kv_empty(v_st));
              p_place = after(p_place);
              // the scores that take this place: nw + kAhead steps on
              const int to_i = L::kAhead ? (nw == 2 ? 1 - i : 0) : i, to_j = L::kAhead ? (nw == 2 ? j + 1 + i : j + 2) : j + 1;
              if (to_j < tiles) ok = scores(to_j, to_i);
            }
          }
          done = ((done & 3u) + (uint32_t)tiles & 3u) | (nw == 2 ? ((done >> 2) + (uint32_t)tiles & 3u) << 2 : done & 12u);
        }
      }
    } else {
      // ---------------------------------------------------------------- values of the cut tiles
      uint32_t raw_par = 0;
      int first = 1;                                          // place in the ring of the task's first values
      for (int n = 0;; ++n) {
        if (!wait_long<true>(info_full(n & 3), (n >> 2) & 1, abort_flag, P.status, 6)) break;
        TaskInfo* info = infos + (n & 3);
        const int flags = info->flags, tiles = info->tiles, cut = info->cut, len_k = info->len_k - (SPLIT ? info->skip : 0);
        bool ok = true;
        for (int j = cut; ok && j < tiles; ++j) {
          const int st = (first + 2 * j) % ST;
          ok = wait_long<true>(v_raw(st), (raw_par >> st) & 1u, abort_flag, P.status, 6);
          if (!ok) break;
          raw_par ^= 1u << st;
          // this thread's 16-byte pieces: every 64th; 128-byte rows, 128 of them for each 64 columns
          uint4* v = reinterpret_cast<uint4*>(smem + L::kKvOff + st * L::kMat) + (warp - 14) * 32 + lane;
          constexpr int N = L::kMat / 16 / 64;
          const int rows = len_k - j * kPrTile, row = ((warp - 14) * 32 + lane) >> 3;     // piece i: row + 8 i of its half
          if (rows < kPrTile) {
#pragma unroll 4
            for (int i = 0; i < N; ++i)
              if (((row + 8 * i) & 127) >= rows) v[64 * i] = make_uint4(0, 0, 0, 0);
          }
          // zero times a value is NaN where the value is not finite
          __nv_bfloat162 sum = __floats2bfloat162_rn(0.0f, 0.0f);
          const __nv_bfloat162 zero = sum;
#pragma unroll 1
          for (int i = 0; i < N; i += 8) {
            uint4 x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = v[64 * (i + k)];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const uint32_t y[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
              for (int e = 0; e < 4; ++e) sum = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&y[e]), zero, sum);
            }
          }
          if (__hisnan(sum.x) || __hisnan(sum.y)) {
            for (int i = 0; i < N; ++i) {
              uint32_t* x = reinterpret_cast<uint32_t*>(v + 64 * i);
              for (int e = 0; e < 4; ++e) {
                if ((x[e] & 0x7F80u) == 0x7F80u) x[e] &= 0xFFFF0000u;
                if ((x[e] & 0x7F800000u) == 0x7F800000u) x[e] &= 0x0000FFFFu;
              }
            }
            *reinterpret_cast<volatile int*>(&info->odd) = 1;
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(v_clean(st));
        }
        first = (first + 2 * tiles) % ST;
        __syncwarp();
        if (lane == 0) mbar_arrive(info_empty(n & 3));
        if (!ok || !(flags & 1)) break;
      }
    }
  }

  // ---- teardown
  tc_fence_before();
  __syncthreads();
  if (warp == 13) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// ------------------------------------------------------------------------------------ host side
static bool make_rows_map(CUtensorMap* m, const void* base, int cols, int64_t rows, int ld) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)kPrTile};
  const cuuint32_t estr[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static bool make_query_map(CUtensorMap* m, const void* base, int hd, int n_q, int64_t rows, int ld, int pack) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)hd, (cuuint64_t)n_q, (cuuint64_t)rows};
  const cuuint64_t strides[2] = {(cuuint64_t)hd * 2, (cuuint64_t)ld * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)pack, (cuuint32_t)(kPrTile / pack)};
  const cuuint32_t estr[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int HD, bool SPLIT>
static int launch_tasks(cudaStream_t st, unsigned blocks, const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV,
                        const PromptParams& P) {
  using L = PrSmem<HD>;
  static_assert(L::kAlloc <= 227 * 1024, "the ring does not fit");
  auto kern = attn_prompt_kernel<HD, SPLIT>;
  static PerDeviceInt attr_set;
  if (!ensure_smem_attr(attr_set, kern, L::kAlloc)) return FPT_ERR_CUDA;
  return launch_kernel(kern, dim3(blocks), dim3(kPrThreads), L::kAlloc, st, true, tmQ, tmK, tmV, P) == cudaSuccess ? FPT_OK : FPT_ERR_CUDA;
}

template <int HD>
static int launch_prompt(cudaStream_t st, const void* Q, int ld_q, const void* K, int ld_k, const void* V, PromptParams P) {
  CUtensorMap tmQ, tmK, tmV;
  // Without keys nothing is fetched; a map has to have a row all the same.
  const bool keys = P.M_k > 0;
  if (!make_query_map(&tmQ, Q, HD, P.n_q, P.M_q, ld_q, 1 << P.pack_log2) ||
      !make_rows_map(&tmK, keys ? K : Q, P.n_kv * HD, keys ? P.M_k : 1, keys ? ld_k : ld_q) ||
      !make_rows_map(&tmV, keys ? V : Q, P.n_kv * HD, keys ? P.M_k : 1, keys ? P.ld_v : ld_q))
    return FPT_ERR_CUDA;
  const int64_t tasks = (int64_t)P.M_q / (2 * kPrTile >> P.pack_log2) + P.n_seqs;
  if (tasks * P.units > INT32_MAX) return FPT_ERR_UNSUPPORTED;
  P.n_tasks = (int)tasks;
  // Keys are split on the device, which knows the lengths; whether they are, and the join with it, follows from the sizes, as if all sequences were
  // equally long.  The join takes 4 to 7 us, as long as a task with four tiles: 100 queries behind 500 keys, 16 us, took 23 with it.
  P.split = 0;
  P.sms = device_sm_count();
  if (P.n_seqs <= 32) {
    const int per_log2 = 8 - P.pack_log2, len_q = (P.M_q + P.n_seqs - 1) / P.n_seqs, len_k = P.M_k / P.n_seqs;
    const Splitting s = {len_k, len_q, (len_q + (1 << per_log2) - 1) >> per_log2, per_log2, P.causal};
    const int64_t n = (int64_t)s.places * P.n_seqs * P.units;
    if (n <= P.sms) {
      int L = Splitting::first_length((uint32_t)std::min<int64_t>((int64_t)s.tiles() * P.n_seqs * P.units, UINT32_MAX), P.sms);
      while ((int64_t)s.split(L) * s.parts(L) * P.n_seqs * P.units > most_parts<HD>()) L += std::max(1, L / 8);
      if (s.most() >= std::max(L, (s.most() + kPrParts - 1) / kPrParts) + kPrSplitGain) P.split = most_parts<HD>();
    }
  }
  if (!P.split) return launch_tasks<HD, false>(st, (unsigned)(tasks * P.units), tmQ, tmK, tmV, P);
  const unsigned blocks = (unsigned)(tasks * P.units + P.split);
  const int got = launch_tasks<HD, true>(st, blocks, tmQ, tmK, tmV, P);
  if (got != FPT_OK) return got;
  if (launch_kernel(prompt_join_kernel<HD>, dim3(blocks), dim3(kPrJoinThreads), 0, st, true, P) != cudaSuccess) return FPT_ERR_CUDA;
  return FPT_OK;
}

}  // namespace fpt

using namespace fpt;

extern "C" int fpt_attn_prompt(void* stream, const void* Q, int ld_q, int M_q, const void* K, int ld_k, const void* V, int ld_v,
                               int M_k, int n_q, int n_kv, int head_dim, const int32_t* cu_q, const int32_t* cu_k, int n_seqs,
                               int causal, float scale, void* O, int ld_o, float* lse, void* workspace,
                               size_t workspace_bytes) {
  if (!Q || !O || !cu_q || M_q <= 0 || M_k < 0 || !K != (M_k == 0) || !V != (M_k == 0) || n_q <= 0 || n_kv <= 0 || n_seqs <= 0)
    return FPT_ERR_BAD_ARG;
  if (head_dim != 64 && head_dim != 128) return FPT_ERR_UNSUPPORTED;
  if (n_q % n_kv || n_q > 65535) return FPT_ERR_UNSUPPORTED;
  if (!(scale > 0.0f) || !(scale < 1e30f)) return FPT_ERR_BAD_ARG;
  const int64_t wq = (int64_t)n_q * head_dim, wk = (int64_t)n_kv * head_dim;
  if (ld_q < wq || ld_o < wq || ld_k < wk || ld_v < wk) return FPT_ERR_BAD_ARG;
  if (M_q > INT32_MAX - 1024 || M_k > INT32_MAX - 1024) return FPT_ERR_UNSUPPORTED;
  if (ld_q % 8 || ld_k % 8 || ld_v % 8 || ld_o % 8) return FPT_ERR_ALIGNMENT;
  if (((uintptr_t)Q | (uintptr_t)K | (uintptr_t)V | (uintptr_t)O | (uintptr_t)workspace) & 15) return FPT_ERR_ALIGNMENT;
  if (((uintptr_t)cu_q | (uintptr_t)cu_k | (uintptr_t)lse) & 3) return FPT_ERR_ALIGNMENT;
  if (!workspace || workspace_bytes < attn_workspace_bytes()) return FPT_ERR_WORKSPACE;
  PromptParams P{};
  P.cu_q = cu_q; P.cu_k = cu_k ? cu_k : cu_q;
  P.V = reinterpret_cast<const __nv_bfloat16*>(V);
  P.O = reinterpret_cast<__nv_bfloat16*>(O);
  P.lse = lse;
  P.status = reinterpret_cast<uint32_t*>(workspace);
  P.sums = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(workspace) + kStatusBytes);
  P.ld_v = ld_v; P.ld_o = ld_o; P.M_q = M_q; P.M_k = M_k; P.n_q = n_q; P.n_kv = n_kv; P.group = n_q / n_kv;
  P.n_seqs = n_seqs;
  // The heads of a group in one tile: the largest power of two that divides the group, so that every row of a tile is one; or more, rows of
  // no head among them, where sequences as long as the average then take an eighth less, a task counted as long as two of its tiles.
  // (42 prompts of 3..15 tokens, 8 groups of 5 heads: 54 -> 15 us; 63 of 19..78, 4 groups of 5: 41 -> 22.)
  while (P.pack_log2 < 4 && (P.group >> P.pack_log2) % 2 == 0) ++P.pack_log2;
  const int64_t len = ((int64_t)M_q + n_seqs - 1) / n_seqs;
  auto packs = [&](int log2) { return (P.group + (1 << log2) - 1) >> log2; };
  auto cost = [&](int log2) {
    const int per = kPrTile >> log2;
    return ((len + 2 * per - 1) / (2 * per) * 2 + (len + per - 1) / per) * packs(log2);
  };
  for (int log2 = P.pack_log2 + 1; log2 <= 4 && 1 << (log2 - 1) < P.group; ++log2)
    if (cost(log2) * 8 < cost(P.pack_log2) * 7) P.pack_log2 = log2;
  P.packs = packs(P.pack_log2);
  P.units = n_kv * P.packs;
  P.causal = causal != 0;
  P.scale_log2 = scale * 1.4426950408889634f;
  return head_dim == 128 ? launch_prompt<128>((cudaStream_t)stream, Q, ld_q, K, ld_k, V, P)
                         : launch_prompt<64>((cudaStream_t)stream, Q, ld_q, K, ld_k, V, P);
}
