// What the attention kernels share: 8-bit codes into floating point, the packed-sequence task search, the argument
// checks of a paged cache.
#pragma once

#include "attn_rules.h"
#include "fpt_internal.cuh"

namespace fpt {

// A page, position, length or offset was out of range: a word of its own behind the status word, so that a wait that gave up, in
// whatever call on the workspace, is never covered up.
constexpr int kIndexWord = 1;
constexpr uint32_t kStatusIndexBase = 0x7200u;
enum : uint32_t { kBadPage = 1, kBadPosition = 2, kBadLength = 3, kBadOffset = 4 };
static_assert(kIndexWord < kCounterWord0, "a counter's place");

__device__ __forceinline__ void record_bad_index(uint32_t* status, uint32_t what) {      // the first one stays
  atomicCAS(status + kIndexWord, 0u, kStatusIndexBase | what);
}

// The i-th of four two's complement bytes whose sign bits the caller has flipped, as a float32: 2^23 + (code + 128) is
// one byte permutation, and the subtraction is exact.
__device__ __forceinline__ float flipped_byte_to_f32(uint32_t flipped, int i) {
  return __fsub_rn(__uint_as_float(__byte_perm(flipped, 0x4B000000u, 0x7440u | (uint32_t)i)), 8388736.0f);
}

// clamp(rne(x), -127, 127) in the low byte, a NaN -> -127 (fmaxf takes the other operand): after the clamp the sum with
// 1.5 * 2^23 rounds to an integer, ties to even, whose two's complement low byte it carries.
__device__ __forceinline__ uint32_t code_of(float x) {
  return __float_as_uint(__fadd_rn(fminf(fmaxf(x, -127.0f), 127.0f), 12582912.0f));
}
__device__ __forceinline__ uint32_t pack_codes(float a, float b, float c, float d) {
  return __byte_perm(__byte_perm(code_of(a), code_of(b), 0x0040u), __byte_perm(code_of(c), code_of(d), 0x0040u), 0x5410u);
}

// The bounded waits of fpt_common.cuh with a suspend hint: these kernels have up to sixteen warps that wait most of the time, and
// without the hint the instruction comes back at once, so that the polling takes issue slots from the warps that work.
__device__ __forceinline__ uint32_t mbar_try_wait_long(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(bar), "r"(parity), "r"(20000u)
      : "memory");
  return done;
}
template <bool WARP>
__device__ __forceinline__ bool wait_long(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, uint32_t* status, uint32_t role) {
  auto done = [&]() -> bool {
    const uint32_t d = mbar_try_wait_long(bar, parity);
    return WARP ? __all_sync(0xffffffffu, d) : d != 0;
  };
  if (done()) return true;
  const uint64_t t0 = globaltimer_ns();
  for (;;) {
    if (done()) return true;
    const bool late = globaltimer_ns() - t0 > kWaitLimitNs;
    const bool give_up = late || *abort_flag;
    if (WARP ? __any_sync(0xffffffffu, give_up) : give_up) {
      if (late) {
        *abort_flag = 1u;
        atomicCAS(status, 0u, kStatusTimeoutBase | role);
      }
      return false;
    }
  }
}

// What a page's codes are multiplied with before rounding.
__device__ __forceinline__ float inverse_scale(float s) { return s >= 1.17549435e-38f ? __fdiv_rn(1.0f, s) : 0.0f; }

// The task of this CTA in a launch over the pages (or blocks of rows) that packed sequences touch (attn_rules.h); false: none.  All
// sequences are looked at side by side, and what is asked of the found one (its first row, its rows, its entry of `extra`) comes with the
// look: one round of loads, where a binary search would wait for one load after the other.  Offsets that do not ascend can give one task to
// several sequences, each with rows below M: claims are counted, the first alone is stored, so that no first row of one meets the rows of
// another, and a task with more than one is nobody's.  (Counted by the barrier instead, or stored once the lowest is known: the kernels
// around it came out 10 % slower, 8190 tokens 45 us against 41.)
struct FoundTask { int seq, place, row0, rows, extra; };
__device__ __forceinline__ bool find_task(const int32_t* __restrict__ cu, const int32_t* __restrict__ extra, int n_seqs, int M, int block,
                                          int id, FoundTask* found /* shared */, uint32_t* status) {
  __shared__ int claims;
  if (threadIdx.x == 0) claims = 0;
  __syncthreads();
  for (int s = threadIdx.x; s < n_seqs; s += blockDim.x) {
    const int lo = __ldg(cu + s), hi = __ldg(cu + s + 1), e = extra ? __ldg(extra + s) : 0;
    if (!rows_fit(lo, hi, M)) {
      if (blockIdx.x == 0) record_bad_index(status, kBadOffset);
    } else {
      const int place = place_of_task(lo, hi, s, block, id);
      if (place >= 0 && atomicAdd(&claims, 1) == 0) *found = FoundTask{s, place, lo, hi - lo, e};
    }
  }
  __syncthreads();
  return claims == 1;
}

int check_cache(const fpt_kv_cache* c, bool with_storage);

constexpr int kAttnMaxCtas = 640;         // launches of the single-token attention are never larger
// A part of a row's result in the workspace: for at most 16 query heads the sums [head_dim], the reference exponent and the
// sum of weights, float32.
constexpr int kAttnPartFloats = 16 * (128 + 2);
// The attention of prompts keeps the sums of at most this many parts of 256 rows of 128 (of 64: twice as many), maxima, sums of weights and
// a flag beside them.
constexpr int kAttnPromptParts = 125;
constexpr size_t kAttnScratchBytes = (size_t)kAttnPromptParts * 256 * (128 + 3) * 4;
static_assert(kAttnScratchBytes >= (size_t)kAttnMaxCtas * 2 * kAttnPartFloats * 4, "the single-token attention's parts");
inline size_t attn_workspace_bytes() { return kStatusBytes + kAttnScratchBytes; }

}  // namespace fpt
