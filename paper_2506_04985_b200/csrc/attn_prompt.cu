// Causal attention of packed prompts (fpt_attn_prompt; formulas: include/fpt.h).
//
// One CTA has two tiles of 128 query rows of one key/value head and walks over that head's keys in tiles of 128.  A row
// is a (token, query head of the group) pair: as many heads of the group as divide 128 share a tile, so a prompt of few
// tokens still fills it, and the keys are fetched once for all of them.
//   warps 0..3, 4..7   softmax of the first and the second query tile, one row a thread
//   warp 8             TMA: queries once, keys and values through a ring
//   warp 9             tensor core:  S = Q K^T (both from shared memory),  O += P V (P from tensor memory, V as it lies: the
//                      instruction takes it with the keys along the rows)
//   warps 10, 11       values of the tiles that a mask cuts: those that are not finite become zeros before the tensor core
//                      reads them (a weight of zero would not make them harmless), as do rows behind the sequence
// While the softmax of one tile runs, the tensor core works for the other.  P (bf16) takes the place of S in tensor
// memory; the next S of a tile is issued behind the P V that reads it, and the tensor core keeps that order.
//
// Softmax in the exponent of two: p = 2^(S scale log2(e) - m).  m is the row's maximum when it was last renewed: it is renewed, and O in
// tensor memory multiplied by 2^(m_old - m_new), only where the maximum has grown by more than 8, so that p <= 256; the quotient by
// the sum of weights is the same for any m.  In tiles without a mask a part of the powers is computed by a polynomial
// on the multiply-add units, since the special-function unit would be the slower side.
#include "attn_common.cuh"

namespace fpt {

constexpr int kPrTile = 128;               // query rows of a tile, keys of a tile
constexpr int kPrThreads = 384;
constexpr int kPrSoftRegs = 208, kPrAuxRegs = 88;
static_assert(2 * 128 * kPrSoftRegs + 128 * kPrAuxRegs <= kPrThreads * 168, "the warpgroups' registers exceed the launch's");

struct PromptParams {
  const int32_t *cu_q, *cu_k;
  const __nv_bfloat16* V;
  __nv_bfloat16* O;
  float* lse;
  uint32_t* status;
  int ld_v, ld_o, M_q, M_k, n_q, n_kv, group, pack, units, n_seqs, n_tasks, causal;
  float scale_log2;
};

template <int HD>
struct PrSmem {
  static constexpr int kStages = HD == 128 ? 5 : 8;
  static constexpr int kMat = kPrTile * HD * 2;              // a tile of keys, values or queries
  static constexpr int kHalf = kPrTile * 128;                // 64 of its columns: 128-byte rows
  static constexpr int kKvOff = 2 * kMat;
  static constexpr int kBarOff = kKvOff + kStages * kMat;
  static constexpr int kNumBars = 2 + 4 * kStages + 2 + 2 + 2;
  static constexpr int kMiscOff = (kBarOff + kNumBars * 8 + 15) / 16 * 16;
  static constexpr int kAlloc = kMiscOff + 32 + 1024;
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
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float y;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
// 2^a, 2^b for a, b in [-126, 127): x = n + f with n the nearest integer (left in the low bits by the sum with 1.5 * 2^23),
// 2^f by the polynomial of degree 4 with the least largest relative error on [-1/2, 1/2] (2.7e-6, 4e-8 in the
// mean; found by reweighted least squares), n added to the exponent.
__device__ __forceinline__ void pow2_poly(float& a, float& b) {
  const uint64_t magic = pack2(12582912.0f, 12582912.0f), back = pack2(-12582912.0f, -12582912.0f);
  const uint64_t x = pack2(fmaxf(a, -126.0f), fmaxf(b, -126.0f));
  const uint64_t t = add2(x, magic);
  const uint64_t n = add2(t, back);
  const uint64_t f = fma2(n, pack2(-1.0f, -1.0f), x);
  uint64_t p = fma2(f, pack2(0.009570102207362652f, 0.009570102207362652f), pack2(0.05591786280274391f, 0.05591786280274391f));
  p = fma2(f, p, pack2(0.240247443318367f, 0.240247443318367f));
  p = fma2(f, p, pack2(0.6931217908859253f, 0.6931217908859253f));
  p = fma2(f, p, pack2(0.9999992847442627f, 0.9999992847442627f));
  float t0, t1, p0, p1;
  unpack2(t, t0, t1);
  unpack2(p, p0, p1);
  a = __uint_as_float(__float_as_uint(p0) + (__float_as_uint(t0) << 23));
  b = __uint_as_float(__float_as_uint(p1) + (__float_as_uint(t1) << 23));
}

template <int HD>
__global__ void __launch_bounds__(kPrThreads, 1)
attn_prompt_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                   const __grid_constant__ CUtensorMap tmV, const PromptParams P) {
  using L = PrSmem<HD>;
  constexpr int ST = L::kStages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t sbase = smem_u32(smem);
  const uint32_t bar0 = sbase + L::kBarOff;
  auto q_full = [&](int w) { return bar0 + 8u * w; };
  auto kv_full = [&](int s) { return bar0 + 8u * (2 + s); };
  auto kv_empty = [&](int s) { return bar0 + 8u * (2 + ST + s); };
  auto s_full = [&](int w) { return bar0 + 8u * (2 + 2 * ST + w); };
  auto p_full = [&](int w) { return bar0 + 8u * (4 + 2 * ST + w); };
  auto o_full = [&](int w) { return bar0 + 8u * (6 + 2 * ST + w); };
  // values of a cut tile: arrived (for the warps that clean them), clean.  One of each a stage: a stage is not filled
  // again before the tensor core has read it, so no phase of theirs is over before it was waited for
  auto v_raw = [&](int s) { return bar0 + 8u * (8 + 2 * ST + s); };
  auto v_clean = [&](int s) { return bar0 + 8u * (8 + 3 * ST + s); };
  volatile uint32_t* misc = reinterpret_cast<volatile uint32_t*>(smem + L::kMiscOff);
  volatile uint32_t* abort_flag = misc + 1;
  volatile uint32_t* odd_values = misc + 2;                  // a cut tile's values were not all finite
  int* found = reinterpret_cast<int*>(smem + L::kMiscOff + 16);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  pdl_wait();
  pdl_launch_dependents();

  // ---- which rows
  const int per_tile = kPrTile / P.pack, per_cta = 2 * per_tile;          // tokens
  int place;
  const int s = find_task(P.cu_q, P.n_seqs, per_cta, 1, P.n_tasks - 1 - (int)(blockIdx.x / P.units), found, P.status, place);
  if (s < 0) return;
  const int row0 = __ldg(P.cu_q + s), len_q = __ldg(P.cu_q + s + 1) - row0;
  const int key0 = __ldg(P.cu_k + s), key1 = __ldg(P.cu_k + s + 1);
  const int len_k = key1 - key0;
  if (row0 > P.M_q - len_q || key0 < 0 || len_k < 0 || key0 > P.M_k - len_k) {
    if (threadIdx.x == 0) record_bad_index(P.status, kBadOffset);
    return;
  }
  const int tok0 = place * per_cta;
  if (place < 0 || tok0 >= len_q) return;
  const int unit = blockIdx.x % P.units, packs = P.group / P.pack;
  const int kv_head = unit / packs;
  const int head0 = kv_head * P.group + (unit - kv_head * packs) * P.pack;
  // keys that a token sees: the first `seen(tok)` of its sequence
  auto seen = [&](int tok) { return P.causal ? max(0, min(len_k, tok + (len_k - len_q) + 1)) : len_k; };
  const int tiles = (seen(min(tok0 + per_cta, len_q) - 1) + kPrTile - 1) / kPrTile;
  const int cut = seen(tok0) / kPrTile;                      // tiles from here on are masked for some row
  const bool two = tok0 + per_tile < len_q;                  // the second query tile has rows

  // this thread's row
  const int w = warp >> 2;                                   // softmax warps: query tile
  const int r = threadIdx.x & 127;
  const int tok = tok0 + w * per_tile + r / P.pack;
  const bool row_ok = warp < 8 && tok < len_q;
  const size_t out_row = (size_t)row0 + (size_t)tok;
  const int head = head0 + r % P.pack;

  if (tiles == 0) {                                          // no row of this CTA sees a key
    if (row_ok) {
      uint4* o = reinterpret_cast<uint4*>(P.O + out_row * P.ld_o + (size_t)head * HD);
#pragma unroll
      for (int i = 0; i < HD / 8; ++i) o[i] = make_uint4(0, 0, 0, 0);
      if (P.lse) P.lse[out_row * P.n_q + head] = -INFINITY;
    }
    return;
  }

  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(q_full(i), 1);
      mbar_init(s_full(i), 1);
      mbar_init(p_full(i), 4);
      mbar_init(o_full(i), 1);
    }
    for (int i = 0; i < ST; ++i) { mbar_init(kv_full(i), 1); mbar_init(kv_empty(i), 1); mbar_init(v_raw(i), 1); mbar_init(v_clean(i), 2); }
    misc[1] = 0;
    misc[2] = 0;
    fence_mbar_init();
    prefetch_tmap(&tmQ);
    prefetch_tmap(&tmK);
    prefetch_tmap(&tmV);
  }
  if (warp == 9) {
    tmem_alloc(sbase + L::kMiscOff, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = misc[0];
  const uint32_t s_col[2] = {tmem, tmem + 128}, o_col[2] = {tmem + 256, tmem + 384};

  if (warp < 8) {
    // ------------------------------------------------------------------ softmax
    reg_inc<kPrSoftRegs>();
    if (w == 0 || two) {
      const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
      const uint32_t ts = s_col[w] + lanes, to = o_col[w] + lanes;
      const int limit = tok < len_q ? seen(tok) : 0;
      const float c = P.scale_log2;
      float m = -INFINITY;                                   // of S * c, when last renewed
      uint64_t sum2 = 0;                                     // two partial sums of weights
      bool ok = true;
      for (int j = 0; j < tiles; ++j) {
        if (!mbar_wait_warp(s_full(w), j & 1, abort_flag, P.status, 4)) { ok = false; break; }
        tc_fence_after();
        float x[128];
#pragma unroll
        for (int b = 0; b < 4; ++b) tmem_ld_32x32(ts + b * 32, reinterpret_cast<uint32_t(&)[32]>(x[b * 32]));
        const bool masked = j >= cut;
        if (masked) {
          const int n = limit - j * kPrTile;                 // columns that count
#pragma unroll
          for (int i = 0; i < 128; ++i) x[i] = i < n ? x[i] : -INFINITY;
        }
        float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < 128; i += 8)
#pragma unroll
          for (int k = 0; k < 4; ++k) top[k] = max3_nan(top[k], x[i + k], x[i + 4 + k]);
        const float now = max3_nan(max3_nan(top[0], top[1], top[2]), top[3], top[3]) * c;     // c > 0
        const bool renew = now > m + 8.0f || m == -INFINITY || now != now;      // (a NaN takes the whole row)
        if (j > 0 && __any_sync(0xffffffffu, renew && now > m)) {
          // (the P V before is done: the S just read was issued behind it)
          const float f = renew && now > m ? (m == -INFINITY ? 0.0f : pow2_unit(m - now)) : 1.0f;
          float s0, s1;
          unpack2(sum2, s0, s1);
          sum2 = pack2(s0 * f, s1 * f);
#pragma unroll 1
          for (int b = 0; b < HD / 32; ++b) {
            uint32_t v[32];
            tmem_ld_32x32(to + b * 32, v);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * f);
            tmem_st_32x32(to + b * 32, v);
          }
          tmem_wait_st();
        }
        if (renew && !(now < m)) m = now;
        const float minus = m == -INFINITY ? 0.0f : -m;
        const uint64_t c2 = pack2(c, c), m2 = pack2(minus, minus);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          uint32_t pk[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float u, v;
            unpack2(fma2(pack2(x[b * 32 + 2 * i], x[b * 32 + 2 * i + 1]), c2, m2), u, v);
            if ((i & 3) == 3 && !masked) {
              pow2_poly(u, v);
            } else {
              u = pow2_unit(u);
              v = pow2_unit(v);
            }
            sum2 = add2(sum2, pack2(u, v));
            pk[i] = f32x2_to_bf16x2_bits(u, v);
          }
          tmem_st_32x16(ts + b * 16, pk);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full(w));
      }
      if (ok && mbar_wait_warp(o_full(w), (tiles - 1) & 1, abort_flag, P.status, 5)) {
        tc_fence_after();
        float s0, s1;
        unpack2(sum2, s0, s1);
        const float sum = s0 + s1;
        const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
        const bool odd = *odd_values != 0;
        __nv_bfloat16* o = P.O + out_row * P.ld_o + (size_t)head * HD;
#pragma unroll 1
        for (int b = 0; b < HD / 32; ++b) {
          uint32_t v[32];
          tmem_ld_32x32(to + b * 32, v);
          if (row_ok) {
            if (odd) {
              // what the cut tiles' zeros stand for: a value that is not finite outweighs every finite sum
              for (int k = cut * kPrTile; k < limit; ++k) {
                const __nv_bfloat16* val = P.V + (size_t)(key0 + k) * P.ld_v + (size_t)kv_head * HD + b * 32;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                  const float z = __bfloat162float(val[i]);
                  if (!(fabsf(z) < INFINITY)) v[i] = __float_as_uint(__uint_as_float(v[i]) + z);
                }
              }
            }
            uint32_t y[16];
#pragma unroll
            for (int i = 0; i < 16; ++i)
              y[i] = f32x2_to_bf16x2_bits(__uint_as_float(v[2 * i]) * inv, __uint_as_float(v[2 * i + 1]) * inv);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *reinterpret_cast<uint4*>(o + b * 32 + i * 8) = make_uint4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
          }
        }
        if (row_ok && P.lse)
          P.lse[out_row * P.n_q + head] =
              sum > 0.0f || sum != sum ? m * 0.69314718055994531f + logf(sum) : -INFINITY;
      }
    }
  } else {
    reg_dec<kPrAuxRegs>();
    if (warp == 8) {
      // ---------------------------------------------------------------- TMA
      if (elect_one()) {
        int st = 0; uint32_t ph = 0, armed = 0, armed_par = 0;
        bool ok = true;
        auto queries = [&](int i) {
          mbar_arrive_expect_tx(q_full(i), L::kMat);
#pragma unroll
          for (int h = 0; h < HD / 64; ++h)
            tma_load_3d(sbase + i * L::kMat + h * L::kHalf, &tmQ, q_full(i), h * 64, head0, row0 + tok0 + i * per_tile);
        };
        uint32_t raw_par = 0;                                 // per stage: parity of the next phase of v_raw
        auto fetch = [&](const CUtensorMap* tm, int j, bool clean) {
          if (!mbar_wait(kv_empty(st), ph ^ 1u, abort_flag, P.status, 1)) return false;
          // values to be cleaned arrive on a barrier of their own, whose every phase the cleaning warps see
          const uint32_t bar = clean ? v_raw(st) : kv_full(st);
          if (clean) mbar_arrive(kv_full(st));
          mbar_arrive_expect_tx(bar, L::kMat);
#pragma unroll
          for (int h = 0; h < HD / 64; ++h)
            tma_load_2d(sbase + L::kKvOff + st * L::kMat + h * L::kHalf, tm, bar, kv_head * HD + h * 64, key0 + j * kPrTile);
          const int slot = clean ? ST + st : st;
          armed |= 1u << slot;
          armed_par = (armed_par & ~(1u << slot)) | ((clean ? raw_par >> st & 1u : ph) << slot);
          if (clean) raw_par ^= 1u << st;
          if (++st == ST) { st = 0; ph ^= 1u; }
          return true;
        };
        queries(0);
        ok = fetch(&tmK, 0, false);
        if (two) queries(1);
        ok = ok && fetch(&tmV, 0, cut == 0);
        for (int j = 1; ok && j < tiles; ++j) ok = fetch(&tmK, j, false) && fetch(&tmV, j, j >= cut);
        if (!ok) {
          const uint64_t t0 = globaltimer_ns();
          for (int i = 0; i < 2 * ST; ++i)
            if (armed & (1u << i))
              while (!mbar_try_wait(i < ST ? kv_full(i) : v_raw(i - ST), (armed_par >> i) & 1u) &&
                     globaltimer_ns() - t0 < 2000000ull) {}
        }
      }
    } else if (warp == 9) {
      // ---------------------------------------------------------------- tensor core
      if (elect_one()) {
        constexpr uint32_t idesc_s = umma_idesc_bf16(128, 128, false), idesc_o = umma_idesc_bf16(128, HD, true);
        const int nw = two ? 2 : 1;
        int st = 0; uint32_t ph = 0;                          // ring: keys 0, values 0, keys 1, ...
        int k_st = 0, v_st = 0;
        uint32_t clean_par = 0;                               // per stage: parity of the next phase of v_clean
        bool ok = true;
        auto next = [&](int& mine) {
          mine = st;
          const bool got = mbar_wait(kv_full(st), ph, abort_flag, P.status, 2);
          if (++st == ST) { st = 0; ph ^= 1u; }
          return got;
        };
        auto scores = [&](int i) {
          const uint32_t a = sbase + i * L::kMat, b = sbase + L::kKvOff + k_st * L::kMat;
#pragma unroll
          for (int h = 0; h < HD / 64; ++h) {
            const uint64_t ad = umma_desc_kmajor_sw128(a + h * L::kHalf), bd = umma_desc_kmajor_sw128(b + h * L::kHalf);
#pragma unroll
            for (int k = 0; k < 4; ++k) umma_bf16(s_col[i], ad + 2u * k, bd + 2u * k, idesc_s, (h | k) != 0);
          }
          umma_commit(s_full(i));
        };
        ok = next(k_st);
        for (int i = 0; ok && i < nw; ++i) {
          ok = mbar_wait(q_full(i), 0, abort_flag, P.status, 2);
          if (ok) { tc_fence_after(); scores(i); }
        }
        if (ok) umma_commit(kv_empty(k_st));
        for (int j = 0; ok && j < tiles; ++j) {
          ok = next(v_st);
          if (ok && j >= cut) {
            ok = mbar_wait(v_clean(v_st), (clean_par >> v_st) & 1u, abort_flag, P.status, 3);
            clean_par ^= 1u << v_st;
          }
          if (ok && j + 1 < tiles) ok = next(k_st);
          for (int i = 0; ok && i < nw; ++i) {
            ok = mbar_wait(p_full(i), j & 1, abort_flag, P.status, 3);
            if (!ok) break;
            tc_fence_after();
            const uint64_t bd = umma_desc_mnmajor_sw128(sbase + L::kKvOff + v_st * L::kMat, L::kHalf);
#pragma unroll
            for (int k = 0; k < kPrTile / 16; ++k)
              umma_bf16_ts(o_col[i], s_col[i] + 8u * k, bd + 128u * k, idesc_o, (j | k) != 0);
            umma_commit(o_full(i));
            if (i == nw - 1) umma_commit(kv_empty(v_st));
            if (j + 1 < tiles) {
              scores(i);
              if (i == nw - 1) umma_commit(kv_empty(k_st));
            }
          }
        }
      }
    } else {
      // ---------------------------------------------------------------- values of the cut tiles
      uint32_t raw_par = 0;
      for (int j = cut; j < tiles; ++j) {
        const int st = (2 * j + 1) % ST;                      // place in the ring
        if (!mbar_wait_warp(v_raw(st), (raw_par >> st) & 1u, abort_flag, P.status, 6)) break;
        raw_par ^= 1u << st;
        uint8_t* v = smem + L::kKvOff + st * L::kMat;
        bool odd = false;
        for (int i = (warp - 10) * 32 + lane; i < L::kMat / 16; i += 64) {
          const int row = (i >> 3) & 127;                     // 128-byte rows, 128 of them for each 64 columns
          uint4* p = reinterpret_cast<uint4*>(v + (size_t)i * 16);
          uint4 x = *p;
          if (j * kPrTile + row >= len_k) {
            *p = make_uint4(0, 0, 0, 0);
          } else {
            uint32_t y[4] = {x.x, x.y, x.z, x.w};
            uint32_t hit = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              // the exponent's bits carry into the sign's when they are all ones
              const uint32_t e = ((y[k] & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
              if (e & 0x8000u) y[k] &= 0xFFFF0000u;
              if (e & 0x80000000u) y[k] &= 0x0000FFFFu;
              hit |= e;
            }
            if (hit) { *p = make_uint4(y[0], y[1], y[2], y[3]); odd = true; }
          }
        }
        if (odd) *odd_values = 1;
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(v_clean(st));
      }
    }
  }

  // ---- teardown
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
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

template <int HD>
static int launch_prompt(cudaStream_t st, const void* Q, int ld_q, const void* K, int ld_k, const void* V, PromptParams P) {
  using L = PrSmem<HD>;
  static_assert(L::kAlloc <= 227 * 1024, "the ring does not fit");
  auto kern = attn_prompt_kernel<HD>;
  static PerDeviceInt attr_set;
  if (!ensure_smem_attr(attr_set, kern, L::kAlloc)) return FPT_ERR_CUDA;
  CUtensorMap tmQ, tmK, tmV;
  if (!make_query_map(&tmQ, Q, HD, P.n_q, P.M_q, ld_q, P.pack) || !make_rows_map(&tmK, K, P.n_kv * HD, P.M_k, ld_k) ||
      !make_rows_map(&tmV, V, P.n_kv * HD, P.M_k, P.ld_v))
    return FPT_ERR_CUDA;
  const int64_t tasks = (int64_t)P.M_q / (2 * kPrTile / P.pack) + P.n_seqs;
  if (tasks * P.units > INT32_MAX) return FPT_ERR_UNSUPPORTED;
  P.n_tasks = (int)tasks;
  return launch_kernel(kern, dim3((unsigned)(tasks * P.units)), dim3(kPrThreads), L::kAlloc, st, true, tmQ, tmK, tmV, P) ==
                 cudaSuccess
             ? FPT_OK
             : FPT_ERR_CUDA;
}

}  // namespace fpt

using namespace fpt;

extern "C" int fpt_attn_prompt(void* stream, const void* Q, int ld_q, int M_q, const void* K, int ld_k, const void* V, int ld_v,
                               int M_k, int n_q, int n_kv, int head_dim, const int32_t* cu_q, const int32_t* cu_k, int n_seqs,
                               int causal, float scale, void* O, int ld_o, float* lse, void* workspace,
                               size_t workspace_bytes) {
  if (!Q || !K || !V || !O || !cu_q || M_q <= 0 || M_k <= 0 || n_q <= 0 || n_kv <= 0 || n_seqs <= 0) return FPT_ERR_BAD_ARG;
  if (head_dim != 64 && head_dim != 128) return FPT_ERR_UNSUPPORTED;
  if (n_q % n_kv || n_q > 65535) return FPT_ERR_UNSUPPORTED;
  if (!(scale > 0.0f) || !(scale < 1e30f)) return FPT_ERR_BAD_ARG;
  const int64_t wq = (int64_t)n_q * head_dim, wk = (int64_t)n_kv * head_dim;
  if (ld_q < wq || ld_o < wq || ld_k < wk || ld_v < wk) return FPT_ERR_BAD_ARG;
  if (M_q > INT32_MAX - 1024 || M_k > INT32_MAX - 1024) return FPT_ERR_UNSUPPORTED;
  if (ld_q % 8 || ld_k % 8 || ld_v % 8 || ld_o % 8) return FPT_ERR_ALIGNMENT;
  if (((uintptr_t)Q | (uintptr_t)K | (uintptr_t)V | (uintptr_t)O | (uintptr_t)workspace) & 15) return FPT_ERR_ALIGNMENT;
  if (((uintptr_t)cu_q | (uintptr_t)cu_k | (uintptr_t)lse) & 3) return FPT_ERR_ALIGNMENT;
  if (!workspace || workspace_bytes < kStatusBytes) return FPT_ERR_WORKSPACE;
  PromptParams P{};
  P.cu_q = cu_q; P.cu_k = cu_k ? cu_k : cu_q;
  P.V = reinterpret_cast<const __nv_bfloat16*>(V);
  P.O = reinterpret_cast<__nv_bfloat16*>(O);
  P.lse = lse;
  P.status = reinterpret_cast<uint32_t*>(workspace);
  P.ld_v = ld_v; P.ld_o = ld_o; P.M_q = M_q; P.M_k = M_k; P.n_q = n_q; P.n_kv = n_kv; P.group = n_q / n_kv;
  P.pack = 1;
  while (P.pack < 16 && P.group % (2 * P.pack) == 0) P.pack *= 2;
  P.units = n_q / P.pack;
  P.n_seqs = n_seqs; P.causal = causal != 0;
  P.scale_log2 = scale * 1.4426950408889634f;
  return head_dim == 128 ? launch_prompt<128>((cudaStream_t)stream, Q, ld_q, K, ld_k, V, P)
                         : launch_prompt<64>((cudaStream_t)stream, Q, ld_q, K, ld_k, V, P);
}
