// The paged key/value cache in 8 bits: rotary positions with the append (fpt_rope_append), and cached tokens in 16 bits
// again (fpt_kv_gather).  Formulas: include/fpt.h.
//
// Both move bytes and little else: a prompt's append reads a row of n_q + 2 n_kv heads, writes n_q (+ n_kv) rotated heads
// and 2 n_kv heads of codes; per pair of elements the rotation is six float operations.
//
// One CTA has one page of one key/value head, so that the largest magnitude of the page's new tokens, its scale and its
// codes need no second pass over memory and no exchange between CTAs: the 16-bit values stay in registers while
// their maximum goes around the CTA.  The query heads of the group ride along, with the rotations of their tokens already in
// registers.  Page and head are contiguous ([page][head][slot][element]), so a full page of codes leaves as one
// 8 KB run.
#include "attn_common.cuh"

namespace fpt {

struct RopeParams {
  const __nv_bfloat16* X;
  const float* rope;
  const int32_t* cu;        // or nullptr: one row a sequence
  const int32_t* ctx;
  const int32_t* pages;
  int8_t *k, *v;
  float *k_scale, *v_scale;
  __nv_bfloat16 *Qo, *Ko;
  uint32_t* status;
  int M, ld, ld_q, ld_k, n_q, n_kv, n_pos, rot, interleaved, n_seqs, n_pages, page, max_pages;
};

// Sixteen elements of a head that belong together: two runs of eight, at `a` and at `b`.  Below rot: with the half layout the second
// run holds the partners of the first, with the interleaved one both hold pairs of neighbours; `pair` is the first
// pair of the sixteen elements' eight.
struct Item { int a, b, pair; };
__device__ __forceinline__ Item item_of(int sub, int rot, int interleaved) {
  Item i;
  const bool turned = sub * 16 < rot;
  i.a = turned && !interleaved ? sub * 8 : sub * 16;
  i.b = turned && !interleaved ? i.a + rot / 2 : i.a + 8;
  i.pair = turned ? sub * 8 : -1;
  return i;
}

__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
  const float x = __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s));
  b = __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
  a = x;
}

// cs: eight (cos, sin) pairs.
__device__ __forceinline__ void rotate16(uint4& lo, uint4& hi, const float4 (&cs)[4], int interleaved) {
  uint32_t l[4] = {lo.x, lo.y, lo.z, lo.w}, h[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float l0 = bf16lo_to_f32(l[i]), l1 = bf16hi_to_f32(l[i]), h0 = bf16lo_to_f32(h[i]), h1 = bf16hi_to_f32(h[i]);
    if (interleaved) {                       // l[i] is pair i, h[i] pair 4 + i
      const float4 p = cs[i >> 1], q = cs[2 + (i >> 1)];
      turn(l0, l1, (i & 1) ? p.z : p.x, (i & 1) ? p.w : p.y);
      turn(h0, h1, (i & 1) ? q.z : q.x, (i & 1) ? q.w : q.y);
    } else {                                 // pairs 2 i and 2 i + 1 across the two runs
      const float4 p = cs[i];
      turn(l0, h0, p.x, p.y);
      turn(l1, h1, p.z, p.w);
    }
    l[i] = f32x2_to_bf16x2_bits(l0, l1);
    h[i] = f32x2_to_bf16x2_bits(h0, h1);
  }
  lo = make_uint4(l[0], l[1], l[2], l[3]);
  hi = make_uint4(h[0], h[1], h[2], h[3]);
}

// Largest magnitude pattern of the finite values among two words of bf16, joined to `acc` (patterns order like magnitudes).
__device__ __forceinline__ uint32_t max_finite(uint32_t w, uint32_t acc) {
  const uint32_t m = w & 0x7FFF7FFFu;
  const uint32_t inf = __vcmpgeu2(m, 0x7F807F80u);           // 0xFFFF per half that is not finite
  return __vmaxu2(acc, m & ~inf);
}
__device__ __forceinline__ uint32_t max_finite(const uint4& v, uint32_t acc) {
  return max_finite(v.x, max_finite(v.y, max_finite(v.z, max_finite(v.w, acc))));
}

__device__ __forceinline__ uint2 codes8(const uint4& v, float inv) {
  uint2 o;
  o.x = pack_codes(__fmul_rn(bf16lo_to_f32(v.x), inv), __fmul_rn(bf16hi_to_f32(v.x), inv),
                   __fmul_rn(bf16lo_to_f32(v.y), inv), __fmul_rn(bf16hi_to_f32(v.y), inv));
  o.y = pack_codes(__fmul_rn(bf16lo_to_f32(v.z), inv), __fmul_rn(bf16hi_to_f32(v.z), inv),
                   __fmul_rn(bf16lo_to_f32(v.w), inv), __fmul_rn(bf16hi_to_f32(v.w), inv));
  return o;
}

// T threads; every thread holds up to N items of keys and as many of values.
template <int HD, int T, int N>
__global__ void __launch_bounds__(T) rope_append_kernel(const RopeParams P) {
  constexpr int I = HD / 16;                    // items of a head
  __shared__ int found[2];
  __shared__ uint32_t peak[2][T / 32];
  pdl_wait();
  pdl_launch_dependents();

  const int head = blockIdx.y, tid = threadIdx.x;
  int s, place, row0 = 0, n_new = 1;
  if (P.cu) {
    s = find_task(P.cu, P.n_seqs, P.page, 2, blockIdx.x, found, P.status, place);
    if (s < 0) return;
    row0 = __ldg(P.cu + s);
    n_new = __ldg(P.cu + s + 1) - row0;
    if (row0 > P.M - n_new) {                   // (both are at least 0)
      if (tid == 0) record_bad_index(P.status, kBadOffset);
      return;
    }
  } else {
    s = blockIdx.x; place = 0; row0 = s;
  }
  const int ctx = __ldg(P.ctx + s);
  if (ctx < 0 || ctx > P.n_pos - n_new) {       // a position without a rotation
    if (tid == 0 && n_new > 0) record_bad_index(P.status, kBadPosition);
    return;
  }
  // without a cache the pages are blocks of rows, counted from the sequence's first
  const int base = P.k ? ctx : 0;
  const int page_no = base / P.page + place;
  const int lo = max(base, page_no * P.page), hi = min(base + n_new, (page_no + 1) * P.page);
  if (lo >= hi) return;
  const int n = hi - lo;                        // new tokens of this page
  const int slot0 = lo - page_no * P.page;
  const int row = row0 + (lo - base), pos = ctx + (lo - base);
  int page = -1;
  if (P.k) {
    page = page_no < P.max_pages ? __ldg(P.pages + (size_t)s * P.max_pages + page_no) : -1;
    if (page < 0 || page >= P.n_pages) {
      if (tid == 0 && head == 0) record_bad_index(P.status, kBadPage);
      page = -1;                                // the rotated rows leave all the same
    }
  }
  const size_t cell = (size_t)(page < 0 ? 0 : page) * P.n_kv + head;     // scale index; codes start at cell * page * HD

  const int group = P.n_q / P.n_kv;
  uint4 kv[N][4];                               // keys: two runs of eight; values: two more
  uint32_t mk = 0, mv = 0;
  float old_k = 0.0f, old_v = 0.0f;
  if (page >= 0 && slot0 > 0) { old_k = P.k_scale[cell]; old_v = P.v_scale[cell]; }
#pragma unroll
  for (int it = 0; it < N; ++it) {
    const int id = it * T + tid, j = id / I;
    if (j < n) {
      const Item e = item_of(id % I, P.rot, P.interleaved);
      const __nv_bfloat16* x = P.X + (size_t)(row + j) * P.ld;
      const __nv_bfloat16* xk = x + (size_t)(P.n_q + head) * HD;
      const __nv_bfloat16* xv = xk + (size_t)P.n_kv * HD;
      kv[it][0] = *reinterpret_cast<const uint4*>(xk + e.a);
      kv[it][1] = *reinterpret_cast<const uint4*>(xk + e.b);
      if (page >= 0) {
        kv[it][2] = *reinterpret_cast<const uint4*>(xv + e.a);
        kv[it][3] = *reinterpret_cast<const uint4*>(xv + e.b);
      }
    }
  }
#pragma unroll
  for (int it = 0; it < N; ++it) {
    const int id = it * T + tid, j = id / I;
    if (j < n) {
      const Item e = item_of(id % I, P.rot, P.interleaved);
      float4 cs[4];
      if (e.pair >= 0) {
        const float4* t = reinterpret_cast<const float4*>(P.rope + ((size_t)(pos + j) * (P.rot / 2) + e.pair) * 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) cs[i] = __ldg(t + i);
        rotate16(kv[it][0], kv[it][1], cs, P.interleaved);
      }
      if (P.Ko) {
        __nv_bfloat16* o = P.Ko + (size_t)(row + j) * P.ld_k + (size_t)head * HD;
        *reinterpret_cast<uint4*>(o + e.a) = kv[it][0];
        *reinterpret_cast<uint4*>(o + e.b) = kv[it][1];
      }
      if (page >= 0) {
        mk = max_finite(kv[it][0], max_finite(kv[it][1], mk));
        mv = max_finite(kv[it][2], max_finite(kv[it][3], mv));
      }
      // the group's queries of the same token, four heads in flight
      const __nv_bfloat16* xq = P.X + (size_t)(row + j) * P.ld + (size_t)head * group * HD;
      __nv_bfloat16* oq = P.Qo + (size_t)(row + j) * P.ld_q + (size_t)head * group * HD;
      for (int h = 0; h < group; h += 4) {
        uint4 q[4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (h + i < group) {
            q[i][0] = *reinterpret_cast<const uint4*>(xq + (h + i) * HD + e.a);
            q[i][1] = *reinterpret_cast<const uint4*>(xq + (h + i) * HD + e.b);
          }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (h + i < group) {
            if (e.pair >= 0) rotate16(q[i][0], q[i][1], cs, P.interleaved);
            *reinterpret_cast<uint4*>(oq + (h + i) * HD + e.a) = q[i][0];
            *reinterpret_cast<uint4*>(oq + (h + i) * HD + e.b) = q[i][1];
          }
      }
    }
  }
  if (page < 0) return;                         // (the same in the whole CTA)

  mk = max(mk & 0xFFFFu, mk >> 16);
  mv = max(mv & 0xFFFFu, mv >> 16);
  mk = __reduce_max_sync(0xffffffffu, mk);
  mv = __reduce_max_sync(0xffffffffu, mv);
  if ((tid & 31) == 0) { peak[0][tid >> 5] = mk; peak[1][tid >> 5] = mv; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < T / 32; ++w) { mk = max(mk, peak[0][w]); mv = max(mv, peak[1][w]); }
  const float s_k = fmaxf(old_k, __fdiv_rn(__uint_as_float(mk << 16), 127.0f));
  const float s_v = fmaxf(old_v, __fdiv_rn(__uint_as_float(mv << 16), 127.0f));
  const float inv_k = inverse_scale(s_k), inv_v = inverse_scale(s_v);
  int8_t* ck = P.k + cell * P.page * HD;
  int8_t* cv = P.v + cell * P.page * HD;
#pragma unroll
  for (int it = 0; it < N; ++it) {
    const int id = it * T + tid, j = id / I;
    if (j < n) {
      const Item e = item_of(id % I, P.rot, P.interleaved);
      const int o = (slot0 + j) * HD;
      *reinterpret_cast<uint2*>(ck + o + e.a) = codes8(kv[it][0], inv_k);
      *reinterpret_cast<uint2*>(ck + o + e.b) = codes8(kv[it][1], inv_k);
      *reinterpret_cast<uint2*>(cv + o + e.a) = codes8(kv[it][2], inv_v);
      *reinterpret_cast<uint2*>(cv + o + e.b) = codes8(kv[it][3], inv_v);
    }
  }
  // tokens that the page held before, on the grown scale
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const float before = which ? old_v : old_k, now = which ? s_v : s_k;
    if (slot0 > 0 && now > before) {
      const float r = __fmul_rn(before, which ? inv_v : inv_k);
      uint4* c = reinterpret_cast<uint4*>(which ? cv : ck);
      for (int i = tid; i < slot0 * HD / 16; i += T) {
        const uint4 w = c[i];
        uint32_t u[4] = {w.x ^ 0x80808080u, w.y ^ 0x80808080u, w.z ^ 0x80808080u, w.w ^ 0x80808080u};
#pragma unroll
        for (int b = 0; b < 4; ++b)
          u[b] = pack_codes(__fmul_rn(flipped_byte_to_f32(u[b], 0), r), __fmul_rn(flipped_byte_to_f32(u[b], 1), r),
                            __fmul_rn(flipped_byte_to_f32(u[b], 2), r), __fmul_rn(flipped_byte_to_f32(u[b], 3), r));
        c[i] = make_uint4(u[0], u[1], u[2], u[3]);
      }
    }
  }
  if (tid == 0) { P.k_scale[cell] = s_k; P.v_scale[cell] = s_v; }
}

struct GatherParams {
  const int8_t *k, *v;
  const float *k_scale, *v_scale;
  const int32_t *pages, *first, *cu;
  __nv_bfloat16 *Ko, *Vo;
  uint32_t* status;
  int M, ld, n_kv, n_seqs, n_pages, page, max_pages;
};

__device__ __forceinline__ uint4 values8(uint2 codes, float scale) {
  const uint32_t a = codes.x ^ 0x80808080u, b = codes.y ^ 0x80808080u;
  auto val = [&](uint32_t w, int i) { return __fmul_rn(flipped_byte_to_f32(w, i), scale); };
  return make_uint4(f32x2_to_bf16x2_bits(val(a, 0), val(a, 1)), f32x2_to_bf16x2_bits(val(a, 2), val(a, 3)),
                    f32x2_to_bf16x2_bits(val(b, 0), val(b, 1)), f32x2_to_bf16x2_bits(val(b, 2), val(b, 3)));
}

// One CTA: the rows of one page and head.  A thread turns 8 codes into 16 bytes, neighbours' neighbours: a warp writes
// whole rows of the head.
template <int HD, int T>
__global__ void __launch_bounds__(T) kv_gather_kernel(const GatherParams P) {
  __shared__ int found[2];
  pdl_wait();
  pdl_launch_dependents();
  int place;
  const int s = find_task(P.cu, P.n_seqs, P.page, 2, blockIdx.x, found, P.status, place);
  if (s < 0) return;
  const int head = blockIdx.y, tid = threadIdx.x;
  const int row0 = __ldg(P.cu + s), n_rows = __ldg(P.cu + s + 1) - row0;
  const int first = P.first ? __ldg(P.first + s) : 0;
  if (row0 > P.M - n_rows || first < 0 || first > INT32_MAX - 1024 - n_rows) {
    if (tid == 0) record_bad_index(P.status, kBadOffset);
    return;
  }
  const int page_no = first / P.page + place;
  const int lo = max(first, page_no * P.page), hi = min(first + n_rows, (page_no + 1) * P.page);
  if (lo >= hi) return;
  const int page = page_no < P.max_pages ? __ldg(P.pages + (size_t)s * P.max_pages + page_no) : -1;
  if (page < 0 || page >= P.n_pages) {
    if (tid == 0) record_bad_index(P.status, kBadPage);
    return;
  }
  const size_t cell = (size_t)page * P.n_kv + head;
  const float sk = __ldg(P.k_scale + cell), sv = __ldg(P.v_scale + cell);
  const size_t from = (cell * P.page + (lo - page_no * P.page)) * HD;
  const uint2* ck = reinterpret_cast<const uint2*>(P.k + from);
  const uint2* cv = reinterpret_cast<const uint2*>(P.v + from);
  const size_t to = (size_t)(row0 + (lo - first)) * P.ld + (size_t)head * HD;
  constexpr int C = HD / 8;                      // 8-element chunks of a row
#pragma unroll 2
  for (int i = tid; i < (hi - lo) * C; i += T) {
    const uint2 a = __ldg(ck + i), b = __ldg(cv + i);
    const size_t o = to + (size_t)(i / C) * P.ld + (i % C) * 8;
    *reinterpret_cast<uint4*>(P.Ko + o) = values8(a, sk);
    *reinterpret_cast<uint4*>(P.Vo + o) = values8(b, sv);
  }
}

// ------------------------------------------------------------------------------------ host side
int check_cache(const fpt_kv_cache* c, bool with_storage) {
  if (!c) return FPT_ERR_BAD_ARG;
  if (c->n_kv <= 0) return FPT_ERR_BAD_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return FPT_ERR_UNSUPPORTED;
  if (!with_storage) return FPT_OK;
  if (!c->k || !c->v || !c->k_scale || !c->v_scale || !c->pages || c->n_pages <= 0 || c->max_pages <= 0) return FPT_ERR_BAD_ARG;
  if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return FPT_ERR_UNSUPPORTED;
  // tokens of a sequence and rows of the cache are counted in 32 bits
  if ((int64_t)c->max_pages * c->page > INT32_MAX - 256) return FPT_ERR_UNSUPPORTED;
  if ((int64_t)c->n_pages * c->n_kv * c->page > INT32_MAX) return FPT_ERR_UNSUPPORTED;
  if (((uintptr_t)c->k | (uintptr_t)c->v) & 15) return FPT_ERR_ALIGNMENT;
  if (((uintptr_t)c->k_scale | (uintptr_t)c->v_scale | (uintptr_t)c->pages) & 3) return FPT_ERR_ALIGNMENT;
  return FPT_OK;
}

template <int HD, int T, int N>
static int launch_rope(cudaStream_t st, const RopeParams& P, unsigned tasks) {
  return launch_kernel(rope_append_kernel<HD, T, N>, dim3(tasks, P.n_kv), dim3(T), 0, st, true, P) == cudaSuccess ? FPT_OK
                                                                                                           : FPT_ERR_CUDA;
}

}  // namespace fpt

using namespace fpt;

extern "C" int fpt_rope_append(void* stream, const void* QKV, int M, int ld, int n_q, const float* rope, int n_pos,
                               int rot_dim, int layout, const int32_t* cu_new, const int32_t* ctx, int n_seqs,
                               const fpt_kv_cache* cache, void* Q_out, int ld_q, void* K_out, int ld_k, void* workspace,
                               size_t workspace_bytes) {
  if (!QKV || !rope || !ctx || !Q_out || M <= 0 || n_seqs <= 0 || n_q <= 0 || n_pos <= 0) return FPT_ERR_BAD_ARG;
  const bool store = cache && cache->k;
  const int rc = check_cache(cache, store);
  if (rc) return rc;
  if (layout != FPT_ROPE_HALF && layout != FPT_ROPE_INTERLEAVED) return FPT_ERR_BAD_ARG;
  const int hd = cache->head_dim, n_kv = cache->n_kv;
  if (rot_dim <= 0 || rot_dim % 16 || rot_dim > hd || n_q % n_kv) return FPT_ERR_UNSUPPORTED;
  if (ld < (n_q + 2 * (int64_t)n_kv) * hd || ld_q < (int64_t)n_q * hd || (K_out && ld_k < (int64_t)n_kv * hd)) return FPT_ERR_BAD_ARG;
  if (!cu_new && n_seqs > M) return FPT_ERR_BAD_ARG;
  if (n_kv > 65535 || n_pos > INT32_MAX - 1024 || M > INT32_MAX - 1024) return FPT_ERR_UNSUPPORTED;
  if (ld % 8 || ld_q % 8 || (K_out && ld_k % 8)) return FPT_ERR_ALIGNMENT;
  if (((uintptr_t)QKV | (uintptr_t)Q_out | (uintptr_t)K_out | (uintptr_t)rope | (uintptr_t)workspace) & 15) return FPT_ERR_ALIGNMENT;
  if (((uintptr_t)cu_new | (uintptr_t)ctx) & 3) return FPT_ERR_ALIGNMENT;
  if (!workspace || workspace_bytes < kStatusBytes) return FPT_ERR_WORKSPACE;
  RopeParams P{};
  P.X = reinterpret_cast<const __nv_bfloat16*>(QKV);
  P.rope = rope; P.cu = cu_new; P.ctx = ctx;
  P.Qo = reinterpret_cast<__nv_bfloat16*>(Q_out);
  P.Ko = reinterpret_cast<__nv_bfloat16*>(K_out);
  P.status = reinterpret_cast<uint32_t*>(workspace);
  P.M = M; P.ld = ld; P.ld_q = ld_q; P.ld_k = ld_k; P.n_q = n_q; P.n_kv = n_kv;
  P.n_pos = n_pos; P.rot = rot_dim; P.interleaved = layout == FPT_ROPE_INTERLEAVED; P.n_seqs = n_seqs;
  P.page = 64;
  if (store) {
    P.k = cache->k; P.v = cache->v; P.k_scale = cache->k_scale; P.v_scale = cache->v_scale; P.pages = cache->pages;
    P.n_pages = cache->n_pages; P.page = cache->page; P.max_pages = cache->max_pages;
  }
  cudaStream_t st = (cudaStream_t)stream;
  const int64_t tasks = cu_new ? (int64_t)M / P.page + 2 * (int64_t)n_seqs : n_seqs;
  if (tasks > INT32_MAX) return FPT_ERR_UNSUPPORTED;
  // one token a sequence: its heads' items are few, and small CTAs start faster; otherwise a page a CTA
  if (!cu_new) return hd == 128 ? launch_rope<128, 32, 1>(st, P, (unsigned)tasks) : launch_rope<64, 32, 1>(st, P, (unsigned)tasks);
  const int items = P.page * (hd / 16);
  if (hd == 128) {
    if (items <= 128) return launch_rope<128, 128, 1>(st, P, (unsigned)tasks);
    if (items <= 256) return launch_rope<128, 256, 1>(st, P, (unsigned)tasks);
    return items <= 512 ? launch_rope<128, 256, 2>(st, P, (unsigned)tasks) : launch_rope<128, 256, 4>(st, P, (unsigned)tasks);
  }
  if (items <= 128) return launch_rope<64, 128, 1>(st, P, (unsigned)tasks);
  return items <= 256 ? launch_rope<64, 256, 1>(st, P, (unsigned)tasks) : launch_rope<64, 256, 2>(st, P, (unsigned)tasks);
}

extern "C" int fpt_kv_gather(void* stream, const fpt_kv_cache* cache, const int32_t* first, const int32_t* cu_out, int n_seqs,
                             int M, void* K_out, void* V_out, int ld, void* workspace, size_t workspace_bytes) {
  if (!cu_out || !K_out || !V_out || n_seqs <= 0 || M <= 0) return FPT_ERR_BAD_ARG;
  const int rc = check_cache(cache, true);
  if (rc) return rc;
  if (ld < (int64_t)cache->n_kv * cache->head_dim) return FPT_ERR_BAD_ARG;
  if (cache->n_kv > 65535 || M > INT32_MAX - 1024) return FPT_ERR_UNSUPPORTED;
  if (ld % 8 || (((uintptr_t)K_out | (uintptr_t)V_out | (uintptr_t)workspace) & 15)) return FPT_ERR_ALIGNMENT;
  if (((uintptr_t)first | (uintptr_t)cu_out) & 3) return FPT_ERR_ALIGNMENT;
  if (!workspace || workspace_bytes < kStatusBytes) return FPT_ERR_WORKSPACE;
  GatherParams P{};
  P.k = cache->k; P.v = cache->v; P.k_scale = cache->k_scale; P.v_scale = cache->v_scale; P.pages = cache->pages;
  P.first = first; P.cu = cu_out;
  P.Ko = reinterpret_cast<__nv_bfloat16*>(K_out);
  P.Vo = reinterpret_cast<__nv_bfloat16*>(V_out);
  P.status = reinterpret_cast<uint32_t*>(workspace);
  P.M = M; P.ld = ld; P.n_kv = cache->n_kv; P.n_seqs = n_seqs; P.n_pages = cache->n_pages; P.page = cache->page;
  P.max_pages = cache->max_pages;
  const int64_t tasks = (int64_t)M / P.page + 2 * (int64_t)n_seqs;
  if (tasks > INT32_MAX) return FPT_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)tasks, cache->n_kv);
  cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t e = cache->head_dim == 128
                            ? launch_kernel(kv_gather_kernel<128, 256>, grid, dim3(256), 0, st, true, P)
                            : launch_kernel(kv_gather_kernel<64, 128>, grid, dim3(128), 0, st, true, P);
  return e == cudaSuccess ? FPT_OK : FPT_ERR_CUDA;
}
