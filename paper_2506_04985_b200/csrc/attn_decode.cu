// Attention of one token a sequence over the paged 8-bit cache (fpt_attn_decode; formulas: include/fpt.h).
//
// Every cached code is read once and takes 2 * (query heads of the group) multiply-adds: the bound is the memory's rate.
// So the kernel is a stream: a warp of each CTA requests tiles of 64 tokens (codes of keys and values) by TMA into a ring,
// four warps take 16 tokens of a tile each.  The tiles of all sequences and key heads form one line that is cut into
// equal ranges, one a CTA, whatever the lengths; a row (sequence, head) that is cut leaves partial results in the
// workspace, and the CTA that finishes the row's last part joins them, in the order of the parts.
// Measured (graph replay, 32 query heads, 8 of keys, of 128): one sequence of 131 072 tokens 56 us = 4.8 TB/s, 64 of 4096 98 us = 5.5 TB/s
// of codes, one of 1000 8.6 us (launch, length, page number, copy and join, one after the other).
//
// A warp's arithmetic, per 16 tokens (T) and up to 8 NT query heads of the group (H):
//   S^T[T x H] = K Q^T      m16n8k16, fp16 x fp16 -> fp32: codes are exact in fp16 (one byte permutation and one packed subtract make two), and
//                           the elements' order along the sum is free: a thread's 16 contiguous codes are its operand registers
//                           of four instructions, so keys need no transposition
//   w = 2^(S' - M + 9)      S' = S scale_k scale log2(e) + log2(scale_v): the scale of the page's values rides in the exponent.
//                           M is a maximum of S' that is renewed once S' grows 6 beyond it: w stays below 2^15, with as much
//                           room below for small ones as fp16 has
//   O^T[D x H] += V^T w     w through one 8x8 transposition between lanes; two tokens' bytes are interleaved by the
//                           permutations that widen them, so values need no transposition either
//   l += w / scale_v        float32, unrounded
// Rows of the swizzled tile are taken in an order (token_row) in which eight lanes' 16-byte loads meet 32 different banks.
#include "attn_common.cuh"

namespace fpt {

constexpr int kDecWarps = 4;                       // consumer warps, 16 tokens of a tile each
constexpr int kDecThreads = (kDecWarps + 1) * 32;
constexpr float kDecLift = 9.0f;                   // log2 of the weight of a score at the reference ...
constexpr float kDecFar = 6.0f;                    // ... and what a score may lie above it: weights stay below 2^15
constexpr float kDecTinyV = 8.271806125530277e-25f;    // 2^-80

struct DecodeParams {
  const __nv_bfloat16* Q;
  const int32_t* kv_len;
  const int32_t* pages;
  const float *k_scale, *v_scale;
  __nv_bfloat16* O;
  float* lse;
  uint32_t* ws;                 // control block: status word, counters
  float* parts;                 // two a CTA, kAttnPartFloats each
  int ld_q, ld_o, n_q, n_kv, group, blocks, n_seqs, n_pages, max_pages;   // blocks: of 8 NT query heads in a group
  int page, page_log2;
  float scale_log2;             // scale * log2(e)
};

// One tile, as the producer leaves it for the consumers.
struct __align__(16) TileInfo {
  float ks[4];                  // per 16 tokens: scale of the keys * scale * log2(e)
  float vl[4];                  // log2 of the scale of the values
  int flags;                    // bit 0: first of this CTA's part of the row, 1: last of it, 2: the part is the whole row;
                                // from bit 4: groups with values; from bit 8: tokens of the tile that count
  int seq, head;                // head: kv head * blocks + block
  uint32_t parts;               // of a part: CTA of the row's first part, and from bit 16 the number of parts
};

template <int HD, int NT, int ST>
struct DecSmem {
  static constexpr int kMat = kDecTile * HD;                     // bytes of a tile's keys (or values)
  static constexpr int kQ = 8 * NT * HD * 2;
  static constexpr int kRing = 0;
  static constexpr int kQOff = ST * 2 * kMat;
  static constexpr int kMergeOff = kQOff + ST * kQ;              // [warps][8 NT][HD] float
  static constexpr int kMergeStats = kMergeOff + kDecWarps * 8 * NT * HD * 4;   // [warps][8 NT] {M, l}
  static constexpr int kInfoOff = kMergeStats + kDecWarps * 8 * NT * 8;
  static constexpr int kBarOff = kInfoOff + 64 * (int)sizeof(TileInfo);
  static constexpr int kMiscOff = kBarOff + (2 * ST + 2) * 8;
  static constexpr int kAlloc = kMiscOff + 16 + 1024;            // slack to align the base to 1024
};

constexpr int kDecWhole = 5;                       // see the producer warp's search

// Row of the tile that stands at place l (0..15) of a 16-token group.
__device__ __forceinline__ int token_row(int l) { return l ^ ((l & 1) << 2); }

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ uint32_t half2_bits(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }

// Two of the four sign-flipped bytes (code + 128) as fp16: 0x6400 + byte is 1024 + code + 128; the difference is exact.
template <int SEL>
__device__ __forceinline__ uint32_t bytes_to_half2(uint32_t flipped) {
  const uint32_t w = __byte_perm(flipped, 0x64646464u, SEL);
  const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&w), __floats2half2_rn(1152.0f, 1152.0f));
  return half2_bits(h);
}

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}

__device__ __forceinline__ uint32_t add_acq_rel(uint32_t* counter) {
  uint32_t old;
  asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(old) : "l"(counter) : "memory");
  return old;
}

// Four elements, from d on, of the finished head h of a row.
__device__ __forceinline__ void finish(__nv_bfloat16* O, float* lse, int hd, int h, int d, float4 o, float m, float sum) {
  const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
  *reinterpret_cast<uint2*>(O + h * hd + d) = make_uint2(f32x2_to_bf16x2_bits(o.x * inv, o.y * inv), f32x2_to_bf16x2_bits(o.z * inv, o.w * inv));
  if (d == 0 && lse) lse[h] = sum > 0.0f || sum != sum ? (m - kDecLift) * 0.69314718055994531f + logf(sum) : -INFINITY;
}

// The join of a row's parts where they are few: each thread looks at all of them for four elements of a head, in one round of loads and
// without a meeting.  (Not inlined: the main loop keeps its registers.)
constexpr int kFew = 16;
template <int HD, int NT>
__device__ __noinline__ void join_few(const float* parts, int nparts, int gh, __nv_bfloat16* O, float* lse) {
  constexpr int NH = 8 * NT, D4 = HD / 4;
  auto part_at = [&](int p) { return parts + (size_t)(2 * p + (p == 0 ? 1 : 0)) * kAttnPartFloats; };
#pragma unroll 1
  for (int e = threadIdx.x; e < gh * D4; e += kDecWarps * 32) {
    const int h = e / D4, d = (e % D4) * 4;
    float m[kFew], l[kFew];
#pragma unroll
    for (int p = 0; p < kFew; ++p) {
      const float* w = part_at(p < nparts ? p : 0) + NH * HD;
      m[p] = p < nparts ? __ldcg(w + h) : -INFINITY;
      l[p] = p < nparts ? __ldcg(w + NH + h) : 0.0f;
    }
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    float top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int from = 0; from < kFew; from += 8) {
      float4 x[8];
#pragma unroll
      for (int b = 0; b < 8; ++b)
        x[b] = from + b < nparts ? __ldcg(reinterpret_cast<const float4*>(part_at(from + b) + (size_t)h * HD + d))
                                 : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (from == 0) {
#pragma unroll
        for (int p = 0; p < kFew; ++p) top = fmaxf(top, m[p]);
      }
#pragma unroll
      for (int b = 0; b < 8; ++b) {
        const float r = m[from + b] == -INFINITY ? 0.0f : ex2(m[from + b] - top);
        sum = fmaf(l[from + b], r, sum);
        o.x = fmaf(x[b].x, r, o.x); o.y = fmaf(x[b].y, r, o.y);
        o.z = fmaf(x[b].z, r, o.z); o.w = fmaf(x[b].w, r, o.w);
      }
    }
    finish(O, lse, HD, h, d, o, top, sum);
  }
}

template <int HD, int NT, int ST, int MINB>
__global__ void __launch_bounds__(kDecThreads, MINB)
attn_decode_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const DecodeParams P) {
  using L = DecSmem<HD, NT, ST>;
  constexpr int NH = 8 * NT;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t sbase = smem_u32(smem);
  auto full = [&](int s) { return sbase + L::kBarOff + 8u * s; };
  auto empty = [&](int s) { return sbase + L::kBarOff + 8u * (ST + s); };
  const uint32_t met = sbase + L::kBarOff + 8u * (2 * ST);
  volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(smem + L::kMiscOff);
  int* last_flag = reinterpret_cast<int*>(smem + L::kMiscOff + 4);
  int* n_tiles_s = reinterpret_cast<int*>(smem + L::kMiscOff + 8);
  TileInfo* infos = reinterpret_cast<TileInfo*>(smem + L::kInfoOff);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < ST; ++s) { mbar_init(full(s), 2); mbar_init(empty(s), kDecWarps); }
    mbar_init(met, kDecWarps);
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_tmap(&tmK);
    prefetch_tmap(&tmV);
  }
  pdl_wait();
  pdl_launch_dependents();

  // The producer warp finds the number of tiles, this CTA's range of them and the sequence of the first: 32 sequences at a time; up to 32
  // are looked at once.
  const int heads = P.n_kv * P.blocks;
  const int cap = P.max_pages * P.page;
  int first = 0, end = 0, off = 0, seq = 0;           // off: first tile of sequence `seq`
  Ranges ranges = {1, 0};
  if (warp == kDecWarps) {
    int mine = 0, longest = 0;                        // of the sequences lane, lane + 32, ...
    bool bad = false;
    for (int s = lane; s < P.n_seqs; s += 32) {
      const int len = __ldg(P.kv_len + s);
      bad |= len < 0 || len > cap;
      const int nt = tiles_of(min(len, cap));
      longest = max(longest, nt);
      mine += nt * heads;
    }
    auto scan = [&](int v) -> int {
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int w = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += w;
      }
      return v;
    };
    int incl = scan(mine);
    const int total = __shfl_sync(0xffffffffu, incl, 31), ctas = min((int)gridDim.x, total);
    if (bad && blockIdx.x == 0) record_bad_index(P.ws, kBadLength);
    ranges.each = total / ctas;
    ranges.longer = total - ranges.each * ctas;
    // Where there is a CTA for each row of tiles, and the longest has not many more tiles than a range, rows stay whole: the join of parts
    // takes longer than those tiles.  (32 heads, 8 of keys, of 128: 30 sequences of 400 tokens, seven tiles against three, 16.2 -> 13.9 us,
    // 50 of 600 22.7 -> 18.2; one of 200, four against one, 7.7 -> 8.3, 30 of 1000, 16 against eight, 21.6 -> 24.4: those are split.)
    const int n_rows = P.n_seqs * heads, wanted = (int)blockIdx.x / heads;
    const bool whole_rows = n_rows <= (int)gridDim.x && (int)__reduce_max_sync(0xffffffffu, (unsigned)longest) <= ranges.each + min(ranges.each + 1, kDecWhole);
    if ((int)blockIdx.x < (whole_rows ? n_rows : ctas)) {
      first = ranges.first_of(blockIdx.x);
      end = ranges.first_of(blockIdx.x + 1);
      for (int s0 = 0;; s0 += 32) {                   // (ends: the tiles add up to `total`)
        if (P.n_seqs > 32) {
          const int s = s0 + lane;
          mine = s < P.n_seqs ? tiles_of(min(__ldg(P.kv_len + s), cap)) * heads : 0;
          incl = scan(mine);
        }
        const uint32_t hit = __ballot_sync(0xffffffffu, whole_rows ? s0 + lane == wanted : off + incl > first);
        if (hit) {
          const int src = __ffs(hit) - 1;
          off += __shfl_sync(0xffffffffu, incl - mine, src);
          seq = s0 + src;
          if (whole_rows) {
            const int nt = __shfl_sync(0xffffffffu, mine, src) / heads;
            first = off + ((int)blockIdx.x - seq * heads) * nt;
            end = first + nt;
          }
          break;
        }
        off += __shfl_sync(0xffffffffu, incl, 31);
        if (s0 + 32 >= P.n_seqs) { end = first; break; }
      }
    }
    if (lane == 0) *n_tiles_s = end - first;
  }
  __syncthreads();

  if (warp == kDecWarps) {
    // ------------------------------------------------------------------ producer
    const int pieces_max = P.page >= kDecTile ? 1 : kDecTile / P.page;    // pages of a tile
    const int piece = min(P.page, kDecTile);                              // their tokens
    // What a lane knows about its tile of a batch of 32, in three steps that each wait for what the one before asked of memory: its place and
    // pages, the pages' scales, the entry for the consumers.
    TileInfo ti;
    int ids[4], cells[4], rows[4], tok_n = 0, tok0 = 0, kv_head = 0, q_heads = 0, q_at = 0;
    auto look_pages = [&](int base) {
      const int x = base + lane;
      tok_n = 0;
      ti.flags = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) ids[i] = -1;
      if (x >= end) return;
      int s = seq, o = off;
      int len = min(__ldg(P.kv_len + s), cap);
      int nt = tiles_of(len);
      while (x >= o + nt * heads) {                   // (x is below the sum of all: there is a next sequence)
        o += nt * heads;
        ++s;
        len = min(__ldg(P.kv_len + s), cap);
        nt = tiles_of(len);
      }
      const int in = x - o, h = in / nt, t = in - h * nt;
      tok0 = t * kDecTile;
      tok_n = max(0, min(kDecTile, len - tok0));
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < pieces_max && i * piece < tok_n)
          ids[i] = __ldg(P.pages + (size_t)s * P.max_pages + ((tok0 + i * piece) >> P.page_log2));
      kv_head = h / P.blocks;
      const int blk = h - kv_head * P.blocks;
      q_heads = min(NH, P.group - blk * NH);
      q_at = kv_head * P.group + blk * NH;
      ti.seq = s; ti.head = h;
      const bool whole = x - t >= first && x - t + nt <= end;
      const bool a = t == 0 || x == first, z = t == nt - 1 || x == end - 1;
      ti.flags = (a ? 1 : 0) | (z ? 2 : 0) | (whole ? 4 : 0) | (tok_n << 8);
      ti.parts = 0;
      if (z && !whole) {
        const int c0 = ranges.cta_of(x - t), c1 = ranges.cta_of(x - t + nt - 1);
        ti.parts = (uint32_t)c0 | (uint32_t)(c1 - c0 + 1) << 16;
      }
    };
    auto find_rows = [&]() {
      bool bad = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool used = i < pieces_max && i * piece < tok_n, fine = ids[i] >= 0 && ids[i] < P.n_pages;
        bad |= used && !fine;
        cells[i] = (fine ? ids[i] : 0) * P.n_kv + kv_head;
        rows[i] = used ? (cells[i] << P.page_log2) + ((tok0 + i * piece) & (P.page - 1)) : -1;
      }
      if (bad) record_bad_index(P.ws, kBadPage);
    };
    auto look_scales = [&]() {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (rows[i] >= 0) {
          ti.ks[i] = __ldg(P.k_scale + cells[i]);
          ti.vl[i] = __ldg(P.v_scale + cells[i]);
        }
    };
    auto publish = [&](int base) {                    // laid out per 16 tokens
      const int x = base + lane;
      if (x >= end) return;
      TileInfo out = ti;
      const int per = piece / 16;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        // (index of the piece of group i, kept out of local memory: per is 1, 2 or 4)
        const float k = per == 4 ? ti.ks[0] : per == 2 ? (i < 2 ? ti.ks[0] : ti.ks[1]) : ti.ks[i];
        const float v = per == 4 ? ti.vl[0] : per == 2 ? (i < 2 ? ti.vl[0] : ti.vl[1]) : ti.vl[i];
        const bool used = i * 16 < tok_n;
        const bool live = v >= kDecTinyV;
        out.ks[i] = used ? k * P.scale_log2 : 0.0f;
        out.vl[i] = !used ? 0.0f : v != v ? v : live ? __log2f(v) : -80.0f;
        if (used && (live || v != v)) out.flags |= 16 << i;
      }
      infos[(x - first) & 63] = out;
    };
    int st = 0; uint32_t ph = 0, armed = 0, armed_par = 0;
    bool ok = true;
    if (first < end) { look_pages(first); find_rows(); look_scales(); }
    for (int base = first; ok && base < end; base += 32) {
      // a lane requests its own tile
      const int my_rows[4] = {rows[0], rows[1], rows[2], rows[3]};
      const uint32_t q_bytes = (ti.flags & 1) ? (uint32_t)q_heads * HD * 2 : 0u;
      const __nv_bfloat16* q_from = P.Q + (size_t)ti.seq * P.ld_q + (size_t)q_at * HD;
      const int my_seq = ti.seq;
      const int count = min(32, end - base);
      const bool more = base + 32 < end;
      // The first tiles of all are requested before their scales are there: the consumers' barrier counts the copies and, apart
      // from them, the entry.
      const int ahead = base == first ? min(count, ST) : 0;
      for (int i = 0; i < count; ++i) {
        if (!wait_long<true>(empty(st), ph ^ 1u, abort_flag, P.ws, 1)) { ok = false; break; }
        if (lane == i) {
          int boxes = 0;
#pragma unroll
          for (int j = 0; j < 4; ++j) boxes += my_rows[j] >= 0;
          mbar_arrive_expect_tx(full(st), (uint32_t)(boxes * piece * HD * 2) + q_bytes);
          const uint32_t dst = sbase + L::kRing + st * 2 * L::kMat;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (my_rows[j] >= 0) {
              tma_load_2d(dst + j * piece * HD, &tmK, full(st), 0, my_rows[j]);
              tma_load_2d(dst + L::kMat + j * piece * HD, &tmV, full(st), 0, my_rows[j]);
            }
          if (q_bytes) bulk_load_1d(sbase + L::kQOff + st * L::kQ, q_from, q_bytes, full(st));
          if (i >= ahead) mbar_arrive(full(st));
        }
        armed |= 1u << st;
        armed_par = (armed_par & ~(1u << st)) | (ph << st);
        if (++st == ST) { st = 0; ph ^= 1u; }
        if (i == ahead - 1) {
          publish(base);
          __syncwarp();
          if (lane == 0)
            for (int k = 0; k < ahead; ++k) mbar_arrive(full(k));
        }
        // the next batch, a step at a time between the tiles of this one
        if (more && i == 8) {
          const int s_last = __shfl_sync(0xffffffffu, my_seq, 31);          // where it starts to look
          while (seq < s_last) { off += tiles_of(min(__ldg(P.kv_len + seq), cap)) * heads; ++seq; }
          look_pages(base + 32);
        }
        if (more && i == 16) { find_rows(); look_scales(); }
      }
      // The half of the ring of entries that the next batch takes was read when the tile 32 back was let go, long before the last of
      // these 32 could be requested (the ring of tiles is shorter).
      if (ok && more) { publish(base + 32); __syncwarp(); }
    }
    if (!ok && lane == 0) {
      const uint64_t t0 = globaltimer_ns();
      for (int q = 0; q < ST; ++q)
        if (armed & (1u << q))
          while (!mbar_try_wait(full(q), (armed_par >> q) & 1u) && globaltimer_ns() - t0 < 2000000ull) {}
    }
  } else {
    // ------------------------------------------------------------------ consumers
    constexpr int KS = HD / 16;                       // k-steps of S, and 16-row tiles of O
    const int g = lane >> 2, q = lane & 3;
    const int n_tiles = *n_tiles_s;
    const int row_a = warp * 16 + token_row(g), row_b = row_a + 8;            // keys: this lane's two rows
    const int tok0 = warp * 16 + token_row(2 * q), tok1 = warp * 16 + token_row(2 * q + 1);
    auto chunk = [&](int row, int c) -> int {                                   // byte of a row's 16-byte chunk
      return HD == 128 ? row * 128 + ((c ^ (row & 7)) << 4) : row * 64 + ((c ^ ((row >> 1) & 3)) << 4);
    };
    float* merge = reinterpret_cast<float*>(smem + L::kMergeOff);
    float2* stats = reinterpret_cast<float2*>(smem + L::kMergeStats);
    uint32_t qf[NT][KS][2];
    float qscale[NT][2];                              // of heads 2 q and 2 q + 1
    float O[NT][KS][4];
    float M[NT][2], l[NT][2];
    int st = 0; uint32_t ph = 0, met_ph = 0;
    // The consumer warps meet (a bounded wait: a named barrier would hold them for good where one of them has given up).
    auto meet = [&]() -> bool {
      __syncwarp();
      if (lane == 0) mbar_arrive(met);
      const bool ok = wait_long<true>(met, met_ph, abort_flag, P.ws, 3);
      met_ph ^= 1u;
      return ok;
    };
    for (int i = 0; i < n_tiles; ++i) {
      if (!wait_long<true>(full(st), ph, abort_flag, P.ws, 2)) break;
      const TileInfo& ti = infos[i & 63];
      const int flags = ti.flags, n = flags >> 8, head = ti.head;
      if (flags & 1) {
        const int blk = head % P.blocks;
        const int gh = min(NH, P.group - blk * NH);
        const uint8_t* qs = smem + L::kQOff + st * L::kQ;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          // this lane's 8 KS/2 ... elements of head 8 t + g: of chunk c (16 elements), those of its quad place
          uint32_t raw[KS][2];
          uint32_t mag = 0;
#pragma unroll
          for (int c = 0; c < HD / 64; ++c) {
            uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
            if (8 * t + g < gh) {
              const uint4* src = reinterpret_cast<const uint4*>(qs + ((8 * t + g) * HD + (c * 4 + q) * 16) * 2);
              lo = src[0]; hi = src[1];
            }
            raw[c * 4 + 0][0] = lo.x; raw[c * 4 + 0][1] = lo.y;
            raw[c * 4 + 1][0] = lo.z; raw[c * 4 + 1][1] = lo.w;
            raw[c * 4 + 2][0] = hi.x; raw[c * 4 + 2][1] = hi.y;
            raw[c * 4 + 3][0] = hi.z; raw[c * 4 + 3][1] = hi.w;
          }
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            mag = __vmaxu2(mag, raw[k][0] & 0x7FFF7FFFu);
            mag = __vmaxu2(mag, raw[k][1] & 0x7FFF7FFFu);
          }
          mag = max(mag & 0xFFFFu, mag >> 16);
          mag = max(mag, __shfl_xor_sync(0xffffffffu, mag, 1));
          mag = max(mag, __shfl_xor_sync(0xffffffffu, mag, 2));
          // 2^(14 - e) for a largest magnitude in [2^e, 2^(e+1)); two factors, since one may leave the range
          int e = (int)(mag >> 7) - 127;
          e = min(max(e, -126), 128);                 // (subnormal or zero: -126; not finite: 128, and the values stay so)
          const float f1 = __uint_as_float((uint32_t)(127 + (14 - e) / 2) << 23);
          const float f2 = __uint_as_float((uint32_t)(127 + (14 - e) - (14 - e) / 2) << 23);
#pragma unroll
          for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int j = 0; j < 2; ++j)
              qf[t][k][j] = half2_bits(__floats2half2_rn(bf16lo_to_f32(raw[k][j]) * f1 * f2, bf16hi_to_f32(raw[k][j]) * f1 * f2));
          const float back = __uint_as_float((uint32_t)max(1, 127 + e - 14) << 23);      // 2^(e - 14)
          qscale[t][0] = __shfl_sync(0xffffffffu, back, 8 * q);
          qscale[t][1] = __shfl_sync(0xffffffffu, back, 8 * q + 4);
          M[t][0] = M[t][1] = -INFINITY;
          l[t][0] = l[t][1] = 0.0f;
#pragma unroll
          for (int k = 0; k < KS; ++k) O[t][k][0] = O[t][k][1] = O[t][k][2] = O[t][k][3] = 0.0f;
        }
      }
      if (warp * 16 < n) {
        const uint8_t* ks = smem + L::kRing + st * 2 * L::kMat;
        const uint8_t* vs = ks + L::kMat;
        const float kf = ti.ks[warp], vl = ti.vl[warp];
        const bool v_live = (flags >> (4 + warp)) & 1;
        // values: tokens 2q, 2q+1, 2q+8, 2q+9 of the group, elements g * HD/8 ...  (asked for first: they arrive under the scores)
        constexpr int W = HD / 32;
        uint32_t v[4][W];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int row = (j & 1 ? tok1 : tok0) + (j >> 1) * 8;
          if (HD == 128) {
            const uint4 x = *reinterpret_cast<const uint4*>(vs + chunk(row, g));
            v[j][0] = x.x; v[j][1] = x.y; v[j][W - 2] = x.z; v[j][W - 1] = x.w;
          } else {
            const uint2 x = *reinterpret_cast<const uint2*>(vs + chunk(row, g >> 1) + (g & 1) * 8);
            v[j][0] = x.x; v[j][1] = x.y;
          }
        }
        // scores, in two chains of accumulators
        float S[NT][2][4];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int k = 0; k < 8; ++k) S[t][k >> 2][k & 3] = 0.0f;
#pragma unroll
        for (int c = 0; c < HD / 64; ++c) {
          const uint4 ra = *reinterpret_cast<const uint4*>(ks + chunk(row_a, c * 4 + q));
          const uint4 rb = *reinterpret_cast<const uint4*>(ks + chunk(row_b, c * 4 + q));
          const uint32_t wa[4] = {ra.x, ra.y, ra.z, ra.w}, wb[4] = {rb.x, rb.y, rb.z, rb.w};
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t fa = wa[w] ^ 0x80808080u, fb = wb[w] ^ 0x80808080u;
            const uint32_t a0 = bytes_to_half2<0x4140>(fa), a2 = bytes_to_half2<0x4342>(fa);
            const uint32_t a1 = bytes_to_half2<0x4140>(fb), a3 = bytes_to_half2<0x4342>(fb);
#pragma unroll
            for (int t = 0; t < NT; ++t) mma_f16(S[t][w & 1], a0, a1, a2, a3, qf[t][c * 4 + w][0], qf[t][c * 4 + w][1]);
          }
        }
        uint32_t p0[NT], p1[NT];
        const bool in_a = row_a < n, in_b = row_b < n;
        const float inv_v = ex2(-vl);
        float s[NT][4];
        bool far = false;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const float f0 = qscale[t][0] * kf, f1 = qscale[t][1] * kf;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            s[t][k] = fmaf(S[t][0][k] + S[t][1][k], k & 1 ? f1 : f0, vl);
            if (!(k < 2 ? in_a : in_b)) s[t][k] = -INFINITY;
            far |= s[t][k] > M[t][k & 1] + kDecFar;
          }
        }
        // The reference of a head is renewed only where a score lies far above it (the first one does): the maximum over the
        // lanes is six shuffles that nothing waits for otherwise.
        if (__any_sync(0xffffffffu, far)) {
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              float m = fmaxf(s[t][j], s[t][2 + j]);
#pragma unroll
              for (int o = 4; o <= 16; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
              m = fmaxf(M[t][j], m);
              const float r = M[t][j] == -INFINITY ? 0.0f : ex2(M[t][j] - m);
              M[t][j] = m;
              l[t][j] *= r;
#pragma unroll
              for (int k = 0; k < KS; ++k) { O[t][k][j] *= r; O[t][k][2 + j] *= r; }
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          // a reference of -inf: nothing counts yet, and no difference of infinities is formed
          const float b0 = M[t][0] == -INFINITY ? 0.0f : M[t][0] - kDecLift, b1 = M[t][1] == -INFINITY ? 0.0f : M[t][1] - kDecLift;
          float w[4] = {ex2(s[t][0] - b0), ex2(s[t][1] - b1), ex2(s[t][2] - b0), ex2(s[t][3] - b1)};
          l[t][0] = fmaf(w[0] + w[2], inv_v, l[t][0]);
          l[t][1] = fmaf(w[1] + w[3], inv_v, l[t][1]);
          if (!v_live) w[0] = w[1] = w[2] = w[3] = 0.0f;
          p0[t] = transpose8x8(half2_bits(__floats2half2_rn(w[0], w[1])));
          p1[t] = transpose8x8(half2_bits(__floats2half2_rn(w[2], w[3])));
        }
#pragma unroll
        for (int w = 0; w < W; ++w) {
          const uint32_t x0 = v[0][w] ^ 0x80808080u, x1 = v[1][w] ^ 0x80808080u;
          const uint32_t x2 = v[2][w] ^ 0x80808080u, x3 = v[3][w] ^ 0x80808080u;
          const uint32_t lo01 = __byte_perm(x0, x1, 0x5140), hi01 = __byte_perm(x0, x1, 0x7362);
          const uint32_t lo23 = __byte_perm(x2, x3, 0x5140), hi23 = __byte_perm(x2, x3, 0x7362);
          const uint32_t a0 = bytes_to_half2<0x4140>(lo01), a1 = bytes_to_half2<0x4342>(lo01);
          const uint32_t a2 = bytes_to_half2<0x4140>(lo23), a3 = bytes_to_half2<0x4342>(lo23);
          const uint32_t c0 = bytes_to_half2<0x4140>(hi01), c1 = bytes_to_half2<0x4342>(hi01);
          const uint32_t c2 = bytes_to_half2<0x4140>(hi23), c3 = bytes_to_half2<0x4342>(hi23);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            mma_f16(O[t][2 * w], a0, a1, a2, a3, p0[t], p1[t]);
            mma_f16(O[t][2 * w + 1], c0, c1, c2, c3, p0[t], p1[t]);
          }
        }
      }
      const int row_seq = ti.seq;                     // (before the tile is let go)
      const int part0 = (int)(ti.parts & 0xFFFFu), nparts = (int)(ti.parts >> 16);
      __syncwarp();
      if (lane == 0) mbar_arrive(empty(st));
      if (++st == ST) { st = 0; ph ^= 1u; }

      if (flags & 2) {
        // ---------------------------------------------------------------- end of this CTA's part of a row
        const int kvh = head / P.blocks, blk = head - kvh * P.blocks;
        const int gh = min(NH, P.group - blk * NH);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
          for (int o = 4; o <= 16; o <<= 1) {
            l[t][0] += __shfl_xor_sync(0xffffffffu, l[t][0], o);
            l[t][1] += __shfl_xor_sync(0xffffffffu, l[t][1], o);
          }
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int h = 8 * t + 2 * q + j;
            if (h < gh) {
              if (g == 0) stats[warp * NH + h] = make_float2(M[t][j], l[t][j]);
              float* dst = merge + (size_t)(warp * NH + h) * HD + g * (HD / 8);
#pragma unroll
              for (int k = 0; k < KS; ++k) { dst[2 * k] = O[t][k][j]; dst[2 * k + 1] = O[t][k][2 + j]; }
            }
          }
        }
        if (!meet()) break;
        const int tid = threadIdx.x;
        const size_t q0 = (size_t)kvh * P.group + (size_t)blk * NH;        // first query head of the row
        auto emit = [&](int h, int d, float4 o, float m, float sum) {      // four elements of a finished head
          finish(P.O + (size_t)row_seq * P.ld_o + q0 * HD, P.lse ? P.lse + (size_t)row_seq * P.n_q + q0 : nullptr, HD, h, d, o, m, sum);
        };
        constexpr int D4 = HD / 4, kPerThread = NH * D4 / (kDecWarps * 32);
        float* part = P.parts + (size_t)(2 * (int)blockIdx.x + ((int)blockIdx.x == part0 ? 1 : 0)) * kAttnPartFloats;
        for (int e = tid; e < gh * D4; e += kDecWarps * 32) {
          const int h = e / D4, d = (e % D4) * 4;
          float top = -INFINITY;
#pragma unroll
          for (int w = 0; w < kDecWarps; ++w) top = fmaxf(top, stats[w * NH + h].x);
          float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          float sum = 0.0f;
#pragma unroll
          for (int w = 0; w < kDecWarps; ++w) {
            const float2 ml = stats[w * NH + h];
            const float r = ml.x == -INFINITY ? 0.0f : ex2(ml.x - top);
            const float4 x = *reinterpret_cast<const float4*>(merge + (size_t)(w * NH + h) * HD + d);
            o.x = fmaf(x.x, r, o.x); o.y = fmaf(x.y, r, o.y); o.z = fmaf(x.z, r, o.z); o.w = fmaf(x.w, r, o.w);
            sum = fmaf(ml.y, r, sum);
          }
          if (flags & 4) {
            emit(h, d, o, top, sum);
          } else {
            __stcg(reinterpret_cast<float4*>(part + (size_t)h * HD + d), o);
            if (d == 0) { __stcg(part + NH * HD + h, top); __stcg(part + NH * HD + NH + h, sum); }
          }
        }
        if (!(flags & 4)) {
          if (!meet()) break;
          if (tid == 0) {
            // (releases the whole CTA's part, which the warps' meeting put before this, and acquires the others')
            uint32_t* counter = P.ws + kCounterWord0 + part0;
            const bool last = add_acq_rel(counter) == (uint32_t)nparts - 1u;
            if (last) *counter = 0;                   // as the next call finds it
            *last_flag = last;
          }
          if (!meet()) break;
          if (*last_flag) {
            // The row's parts, in their order: the first is the tail part of its CTA, the others head parts of theirs.  First the
            // exponents (a head and every 128 / NH-th part a thread), then weights into shared memory, as many parts at a time as it
            // has room for, then the sums: loads of one step do not wait for one another.
            auto part_at = [&](int p) { return P.parts + (size_t)(2 * (part0 + p) + (p == 0 ? 1 : 0)) * kAttnPartFloats; };
            constexpr int kStep = kDecWarps * 32 / NH, kBatch = 12;
            if (nparts <= kFew) {
              join_few<HD, NT>(P.parts + (size_t)(2 * part0) * kAttnPartFloats, nparts, gh, P.O + (size_t)row_seq * P.ld_o + q0 * HD,
                               P.lse ? P.lse + (size_t)row_seq * P.n_q + q0 : nullptr);
            } else {
            constexpr int kRoom = kDecWarps * HD;       // parts whose weights fit
            float* weights = merge;                     // [part][NH]
            const int h0 = tid % NH, p0 = tid / NH;
            float top = -INFINITY;
            // (a batch of loads has a fixed length, what lies behind the last part left out: the tail of an unrolled loop would
            // wait for one load after the other, 6 us of 11 with 55 parts)
            float m0[4], l0[4];                         // the first batch stays
            auto load = [&](int from, int until, float (&m)[4], float (&l)[4]) {
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const bool there = from + k * kStep < until && h0 < gh;
                const float* w = part_at(there ? from + k * kStep : 0) + NH * HD;
                m[k] = there ? __ldcg(w + h0) : -INFINITY;
                l[k] = there ? __ldcg(w + NH + h0) : 0.0f;
              }
            };
            load(p0, nparts, m0, l0);
            top = fmaxf(fmaxf(m0[0], m0[1]), fmaxf(m0[2], m0[3]));
            for (int p = p0 + 4 * kStep; p < nparts; p += 4 * kStep) {
              float m[4], l[4];
              load(p, nparts, m, l);
              top = fmaxf(top, fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])));
            }
            merge[tid] = top;
            if (!meet()) break;
            top = -INFINITY;
#pragma unroll
            for (int k = 0; k < kStep; ++k) top = fmaxf(top, merge[k * NH + h0]);
            if (!meet()) break;
            float4 o[kPerThread];
#pragma unroll
            for (int k = 0; k < kPerThread; ++k) o[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            float sum = 0.0f;                           // of head h0, this thread's parts
            bool fine = true;
            for (int from = 0; from < nparts; from += kRoom) {
              const int n_here = min(kRoom, nparts - from);
              for (int p = p0; p < n_here; p += 4 * kStep) {
                float m[4] = {m0[0], m0[1], m0[2], m0[3]}, l[4] = {l0[0], l0[1], l0[2], l0[3]};
                if (from + p != p0) load(from + p, from + n_here, m, l);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  const float r = m[k] == -INFINITY ? 0.0f : ex2(m[k] - top);
                  sum = fmaf(l[k], r, sum);
                  if (p + k * kStep < n_here) weights[(p + k * kStep) * NH + h0] = r;
                }
              }
              if (!(fine = meet())) break;
#pragma unroll
              for (int k = 0; k < kPerThread; ++k) {
                const int e = tid + k * kDecWarps * 32, h = e / D4, d = (e % D4) * 4;
                if (e < gh * D4) {
                  for (int p = 0; p < n_here; p += kBatch) {
                    float4 x[kBatch];
#pragma unroll
                    for (int b = 0; b < kBatch; ++b)
                      x[b] = p + b < n_here ? __ldcg(reinterpret_cast<const float4*>(part_at(from + p + b) + (size_t)h * HD + d))
                                            : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                    for (int b = 0; b < kBatch; ++b) {
                      const float r = p + b < n_here ? weights[(p + b) * NH + h] : 0.0f;
                      o[k].x = fmaf(x[b].x, r, o[k].x); o[k].y = fmaf(x[b].y, r, o[k].y);
                      o[k].z = fmaf(x[b].z, r, o[k].z); o[k].w = fmaf(x[b].w, r, o[k].w);
                    }
                  }
                }
              }
              if (!(fine = meet())) break;
            }
            if (!fine) break;
            merge[tid] = sum;
            if (p0 == 0) merge[kDecWarps * 32 + h0] = top;
            if (!meet()) break;
#pragma unroll
            for (int k = 0; k < kPerThread; ++k) {
              const int e = tid + k * kDecWarps * 32, h = e / D4, d = (e % D4) * 4;
              if (e < gh * D4) {
                float all = 0.0f;
#pragma unroll
                for (int i = 0; i < kStep; ++i) all += merge[i * NH + h];
                emit(h, d, o[k], merge[kDecWarps * 32 + h], all);
              }
            }
            }
          }
        }
        if (!meet()) break;                           // the buffers are free for the next row
        // (the next tile begins a row; said here, so that nothing of this one is kept in registers through the join)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          M[t][0] = M[t][1] = l[t][0] = l[t][1] = qscale[t][0] = qscale[t][1] = 0.0f;
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            qf[t][k][0] = qf[t][k][1] = 0;
            O[t][k][0] = O[t][k][1] = O[t][k][2] = O[t][k][3] = 0.0f;
          }
        }
      }
    }
  }
}

// ------------------------------------------------------------------------------------ host side
static bool make_code_map(CUtensorMap* m, const void* base, int64_t rows, int hd, int box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)hd, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)hd};
  const cuuint32_t box[2] = {(cuuint32_t)hd, (cuuint32_t)box_rows};
  const cuuint32_t estr[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, hd == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int HD, int NT, int ST, int MINB>
static int launch_decode(cudaStream_t st, const fpt_kv_cache* c, DecodeParams P) {
  using L = DecSmem<HD, NT, ST>;
  static_assert((L::kAlloc + 1024) * MINB <= 228 * 1024, "the ring does not fit");
  static_assert(ST <= 8, "a batch of tiles has to be longer than the ring");
  P.blocks = (P.group + 8 * NT - 1) / (8 * NT);
  // a CTA for each tile at most; tiles are counted in 32 bits
  const int64_t rows_of_heads = (int64_t)P.n_seqs * P.n_kv * P.blocks, longest = ((int64_t)c->max_pages * c->page + kDecTile - 1) / kDecTile;
  if (rows_of_heads > INT32_MAX / longest) return FPT_ERR_UNSUPPORTED;
  const int64_t most = rows_of_heads * longest;
  auto kern = attn_decode_kernel<HD, NT, ST, MINB>;
  static PerDeviceInt attr_set;
  if (!ensure_smem_attr(attr_set, kern, L::kAlloc)) return FPT_ERR_CUDA;
  CUtensorMap tmK, tmV;
  const int64_t rows = (int64_t)c->n_pages * c->n_kv * c->page;
  const int box = c->page < kDecTile ? c->page : kDecTile;
  if (!make_code_map(&tmK, c->k, rows, HD, box) || !make_code_map(&tmV, c->v, rows, HD, box)) return FPT_ERR_CUDA;
  int64_t grid = (int64_t)device_sm_count() * MINB;
  if (grid > kAttnMaxCtas) grid = kAttnMaxCtas;
  if (grid > most) grid = most;
  return launch_kernel(kern, dim3((unsigned)grid), dim3(kDecThreads), L::kAlloc, st, true, tmK, tmV, P) == cudaSuccess
             ? FPT_OK
             : FPT_ERR_CUDA;
}

}  // namespace fpt

using namespace fpt;

extern "C" int fpt_attn_decode(void* stream, const void* Q, int ld_q, int n_q, const fpt_kv_cache* cache,
                               const int32_t* kv_len, int n_seqs, float scale, void* O, int ld_o, float* lse,
                               void* workspace, size_t workspace_bytes) {
  if (!Q || !kv_len || !O || n_q <= 0 || n_seqs <= 0) return FPT_ERR_BAD_ARG;
  const int rc = check_cache(cache, true);
  if (rc) return rc;
  if (n_q % cache->n_kv) return FPT_ERR_UNSUPPORTED;
  if (ld_q < (int64_t)n_q * cache->head_dim || ld_o < (int64_t)n_q * cache->head_dim) return FPT_ERR_BAD_ARG;
  if (!(scale > 0.0f) || !(scale < 1e30f)) return FPT_ERR_BAD_ARG;
  if (ld_q % 8 || ld_o % 8 || (((uintptr_t)Q | (uintptr_t)O | (uintptr_t)workspace) & 15)) return FPT_ERR_ALIGNMENT;
  if (((uintptr_t)kv_len | (uintptr_t)lse) & 3) return FPT_ERR_ALIGNMENT;
  if (!workspace || workspace_bytes < attn_workspace_bytes()) return FPT_ERR_WORKSPACE;
  DecodeParams P{};
  P.Q = reinterpret_cast<const __nv_bfloat16*>(Q);
  P.kv_len = kv_len; P.pages = cache->pages; P.k_scale = cache->k_scale; P.v_scale = cache->v_scale;
  P.O = reinterpret_cast<__nv_bfloat16*>(O);
  P.lse = lse;
  P.ws = reinterpret_cast<uint32_t*>(workspace);
  P.parts = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(workspace) + kStatusBytes);
  P.ld_q = ld_q; P.ld_o = ld_o; P.n_q = n_q; P.n_kv = cache->n_kv; P.group = n_q / cache->n_kv; P.n_seqs = n_seqs;
  P.n_pages = cache->n_pages; P.max_pages = cache->max_pages; P.page = cache->page;
  while ((1 << P.page_log2) < P.page) ++P.page_log2;
  P.scale_log2 = scale * 1.4426950408889634f;
  cudaStream_t st = (cudaStream_t)stream;
  // Three CTAs an SM where registers and shared memory allow it: with two, and as much in flight, a tile in each takes its time
  // (131071 tokens of 8 heads: 57 and 64 us, 64 ragged sequences: 136 and 161, replayed from a graph; one call after the other the latter take
  // 139 to 153 with three).
  if (cache->head_dim == 128)
    return P.group <= 8 ? launch_decode<128, 1, 3, 3>(st, cache, P) : launch_decode<128, 2, 3, 2>(st, cache, P);
  return P.group <= 8 ? launch_decode<64, 1, 6, 3>(st, cache, P) : launch_decode<64, 2, 4, 3>(st, cache, P);
}
