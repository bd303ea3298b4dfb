// The paged key/value cache in 8 bits: rotary positions with the append (fpt_rope_append), and cached tokens in 16 bits
// again (fpt_kv_gather).  Formulas: include/fpt.h.
//
// Both move bytes and little else: a prompt's append reads a row of n_q + 2 n_kv heads, writes n_q (+ n_kv) rotated heads
// and 2 n_kv heads of codes; per pair of elements the rotation is six float operations.
//
// One CTA has one page of one key/value head, so that the largest magnitude of the page's new tokens, its scale and its
// codes need no second pass over memory and no exchange between CTAs: the 16-bit values stay in registers while
// their maximum goes around the CTA.  Page and head are contiguous ([page][head][slot][element]), so a full page of codes leaves as one
// 8 KB run.  The queries of the page's tokens have CTAs of their own, a group of heads each: with them in the same CTA its
// registers held two CTAs an SM (8190 tokens of 32 + 8 heads: 43.6 us, now 41.0 at 203 MB).
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
  int M, ld, ld_q, ld_k, n_q, n_kv, n_pos, rot, interleaved, n_seqs, n_pages, page, max_pages, by_row;
};

// Sixteen elements of a head: two runs of eight, at `a` and at `b`.  Neighbours' runs follow each other (16 bytes a lane at a
// stride of 32 would write half sectors).  With the half layout a turned item's second run holds the partners of its first, and `pa` is
// the first of their eight pairs; with the interleaved one each run holds four pairs of neighbours, from pa and from pb on.  -1: not turned.
struct Item { int a, b, pa, pb; };
template <int HD>
__device__ __forceinline__ Item item_of(int sub, int rot, int interleaved) {
  Item i;
  if (interleaved) {
    i.a = sub * 8;
    i.b = HD / 2 + sub * 8;
    i.pa = i.a < rot ? i.a / 2 : -1;
    i.pb = i.b < rot ? i.b / 2 : -1;
  } else {
    const bool turned = sub * 16 < rot;
    const int from = turned ? 0 : rot, len = turned ? rot : HD - rot, k = turned ? sub : sub - rot / 16;
    i.a = from + k * 8;
    i.b = i.a + len / 2;
    i.pa = turned ? sub * 8 : -1;
    i.pb = -1;
  }
  return i;
}

// The rotations of an item at one position: eight (cos, sin) pairs, those that it has.
__device__ __forceinline__ void load_rotations(const RopeParams& P, const Item& e, int pos, float4 (&cs)[4]) {
  const float* r = P.rope + (size_t)pos * P.rot;
  if (e.pa >= 0) {
    const float4* f = reinterpret_cast<const float4*>(r + e.pa * 2);
    cs[0] = __ldg(f);
    cs[1] = __ldg(f + 1);
    if (!P.interleaved) { cs[2] = __ldg(f + 2); cs[3] = __ldg(f + 3); }
  }
  if (e.pb >= 0) {
    const float4* f = reinterpret_cast<const float4*>(r + e.pb * 2);
    cs[2] = __ldg(f);
    cs[3] = __ldg(f + 1);
  }
}

__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
  const float x = __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s));
  b = __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
  a = x;
}

__device__ __forceinline__ void rotate_item(const Item& e, uint4& lo, uint4& hi, const float4 (&cs)[4], int interleaved) {
  uint32_t l[4] = {lo.x, lo.y, lo.z, lo.w}, h[4] = {hi.x, hi.y, hi.z, hi.w};
  if (interleaved) {                           // word i of a run is one pair
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 p = cs[i >> 1], q = cs[2 + (i >> 1)];
      if (e.pa >= 0) {
        float x = bf16lo_to_f32(l[i]), y = bf16hi_to_f32(l[i]);
        turn(x, y, (i & 1) ? p.z : p.x, (i & 1) ? p.w : p.y);
        l[i] = f32x2_to_bf16x2_bits(x, y);
      }
      if (e.pb >= 0) {
        float x = bf16lo_to_f32(h[i]), y = bf16hi_to_f32(h[i]);
        turn(x, y, (i & 1) ? q.z : q.x, (i & 1) ? q.w : q.y);
        h[i] = f32x2_to_bf16x2_bits(x, y);
      }
    }
  } else if (e.pa >= 0) {                      // words i of the two runs are pairs 2 i and 2 i + 1
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float l0 = bf16lo_to_f32(l[i]), l1 = bf16hi_to_f32(l[i]), h0 = bf16lo_to_f32(h[i]), h1 = bf16hi_to_f32(h[i]);
      turn(l0, h0, cs[i].x, cs[i].y);
      turn(l1, h1, cs[i].z, cs[i].w);
      l[i] = f32x2_to_bf16x2_bits(l0, l1);
      h[i] = f32x2_to_bf16x2_bits(h0, h1);
    }
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
__global__ void __launch_bounds__(T, (N <= 2 ? 1024 : 512) / T) rope_append_kernel(const RopeParams P) {
  constexpr int I = HD / 16;                    // items of a head
  __shared__ FoundTask found;
  __shared__ uint32_t peak[2][T / 32];
  pdl_wait();
  pdl_launch_dependents();

  const int head = blockIdx.y % P.n_kv, tid = threadIdx.x;
  if (P.cu && !find_task(P.cu, P.ctx, P.n_seqs, P.M, P.by_row ? 0 : P.page, blockIdx.x, &found, P.status)) return;
  const FoundTask task = P.cu ? found : FoundTask{(int)blockIdx.x, 0, (int)blockIdx.x, 1, __ldg(P.ctx + blockIdx.x)};
  const int s = task.seq, row0 = task.row0, n_new = task.rows, ctx = task.extra;
  if (ctx < 0 || ctx > P.n_pos - n_new) {       // a position without a rotation
    if (tid == 0 && n_new > 0) record_bad_index(P.status, kBadPosition);
    return;
  }
  // without a cache the pages are blocks of rows, counted from the sequence's first
  const int base = P.k ? ctx : 0;
  int page_no = base / P.page + task.place;
  if (P.by_row) {                               // the first of the sequence's rows in a page has the page
    const int at = base + ((int)blockIdx.x - row0);
    if (at != base && at % P.page) return;
    page_no = at / P.page;
  }
  const int lo = max(base, page_no * P.page), hi = min(base + n_new, (page_no + 1) * P.page);
  if (lo >= hi) return;
  const int n = hi - lo;                        // new tokens of this page
  const int slot0 = lo - page_no * P.page;
  const int row = row0 + (lo - base), pos = ctx + (lo - base);
  if (blockIdx.y >= (unsigned)P.n_kv) {
    // ---- queries: pieces of 16 elements, neighbours in a token's heads; two in flight a thread
    const int group = P.n_q / P.n_kv, row_items = group * I, items = n * row_items;
    const __nv_bfloat16* xq = P.X + (size_t)row * P.ld + (size_t)head * group * HD;
    __nv_bfloat16* oq = P.Qo + (size_t)row * P.ld_q + (size_t)head * group * HD;
    constexpr int U = 2;
    for (int id0 = tid; id0 < items; id0 += U * T) {
      uint4 x[U][2];
      float4 cs[U][4];
      int at[U][3];                                // token, head of the group, piece
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int id = id0 + u * T, j = id / row_items, in = id - j * row_items;
        at[u][0] = j; at[u][1] = in / I; at[u][2] = in % I;
        if (id < items) {
          const Item e = item_of<HD>(at[u][2], P.rot, P.interleaved);
          const __nv_bfloat16* src = xq + (size_t)j * P.ld + at[u][1] * HD;
          x[u][0] = *reinterpret_cast<const uint4*>(src + e.a);
          x[u][1] = *reinterpret_cast<const uint4*>(src + e.b);
          load_rotations(P, e, pos + j, cs[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (id0 + u * T < items) {
          const Item e = item_of<HD>(at[u][2], P.rot, P.interleaved);
          rotate_item(e, x[u][0], x[u][1], cs[u], P.interleaved);
          __nv_bfloat16* o = oq + (size_t)at[u][0] * P.ld_q + at[u][1] * HD;
          *reinterpret_cast<uint4*>(o + e.a) = x[u][0];
          *reinterpret_cast<uint4*>(o + e.b) = x[u][1];
        }
    }
    return;
  }

  // ---- keys and values
  int page = -1;
  if (P.k) {
    page = page_no < P.max_pages ? __ldg(P.pages + (size_t)s * P.max_pages + page_no) : -1;
    if (page < 0 || page >= P.n_pages) {
      if (tid == 0 && head == 0) record_bad_index(P.status, kBadPage);
      page = -1;                                // the rotated keys leave all the same
    }
  }
  const size_t cell = (size_t)(page < 0 ? 0 : page) * P.n_kv + head;     // scale index; codes start at cell * page * HD
  uint4 kv[N][4];                               // keys: two runs of eight; values: two more
  uint32_t mk = 0, mv = 0;
#pragma unroll
  for (int it = 0; it < N; ++it) {
    const int id = it * T + tid, j = id / I;
    if (j < n) {
      const Item e = item_of<HD>(id % I, P.rot, P.interleaved);
      const __nv_bfloat16* x = P.X + (size_t)(row + j) * P.ld;
      const __nv_bfloat16* xk = x + (size_t)(P.n_q + head) * HD;
      const __nv_bfloat16* xv = xk + (size_t)P.n_kv * HD;
      kv[it][0] = *reinterpret_cast<const uint4*>(xk + e.a);
      kv[it][1] = *reinterpret_cast<const uint4*>(xk + e.b);
      kv[it][2] = *reinterpret_cast<const uint4*>(xv + e.a);
      kv[it][3] = *reinterpret_cast<const uint4*>(xv + e.b);
    }
  }
  float old_k = 0.0f, old_v = 0.0f;
  if (page >= 0 && slot0 > 0) { old_k = P.k_scale[cell]; old_v = P.v_scale[cell]; }
#pragma unroll
  for (int it = 0; it < N; ++it) {
    const int id = it * T + tid, j = id / I;
    if (j < n) {
      const Item e = item_of<HD>(id % I, P.rot, P.interleaved);
      float4 cs[4];
      load_rotations(P, e, pos + j, cs);
      rotate_item(e, kv[it][0], kv[it][1], cs, P.interleaved);
      if (P.Ko) {
        __nv_bfloat16* o = P.Ko + (size_t)(row + j) * P.ld_k + (size_t)head * HD;
        *reinterpret_cast<uint4*>(o + e.a) = kv[it][0];
        *reinterpret_cast<uint4*>(o + e.b) = kv[it][1];
      }
      mk = max_finite(kv[it][0], max_finite(kv[it][1], mk));
      mv = max_finite(kv[it][2], max_finite(kv[it][3], mv));
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
      const Item e = item_of<HD>(id % I, P.rot, P.interleaved);
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
      const int n_old = slot0 * HD / 16;
      for (int i0 = tid; i0 < n_old; i0 += 4 * T) {      // four loads in flight
        uint4 w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (i0 + k * T < n_old) w[k] = c[i0 + k * T];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (i0 + k * T < n_old) {
            uint32_t u[4] = {w[k].x ^ 0x80808080u, w[k].y ^ 0x80808080u, w[k].z ^ 0x80808080u, w[k].w ^ 0x80808080u};
#pragma unroll
            for (int b = 0; b < 4; ++b)
              u[b] = pack_codes(__fmul_rn(flipped_byte_to_f32(u[b], 0), r), __fmul_rn(flipped_byte_to_f32(u[b], 1), r),
                                __fmul_rn(flipped_byte_to_f32(u[b], 2), r), __fmul_rn(flipped_byte_to_f32(u[b], 3), r));
            c[i0 + k * T] = make_uint4(u[0], u[1], u[2], u[3]);
          }
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
  int M, ld, n_kv, n_seqs, n_pages, page, max_pages, heads;
};

__device__ __forceinline__ uint4 values8(uint2 codes, float scale) {
  const uint32_t a = codes.x ^ 0x80808080u, b = codes.y ^ 0x80808080u;
  auto val = [&](uint32_t w, int i) { return __fmul_rn(flipped_byte_to_f32(w, i), scale); };
  return make_uint4(f32x2_to_bf16x2_bits(val(a, 0), val(a, 1)), f32x2_to_bf16x2_bits(val(a, 2), val(a, 3)),
                    f32x2_to_bf16x2_bits(val(b, 0), val(b, 1)), f32x2_to_bf16x2_bits(val(b, 2), val(b, 3)));
}

// One CTA: the rows of one page and `heads` heads (P.heads; about 8 KB of codes each of keys and values: with a head a
// CTA, pages of 16 tokens of 64 values left it 2 KB, and the launch took 25 us for 37 ragged prefixes of 16 heads instead of
// 18).  A thread turns 8 codes into 16 bytes; neighbours' pieces follow each other along the heads of a token, as they
// lie in the output.
template <int HD>
__global__ void __launch_bounds__(256) kv_gather_kernel(const GatherParams P) {
  __shared__ FoundTask found;
  pdl_wait();
  pdl_launch_dependents();
  if (!find_task(P.cu, P.first, P.n_seqs, P.M, P.page, blockIdx.x, &found, P.status)) return;
  const FoundTask task = found;
  const int s = task.seq, place = task.place, row0 = task.row0, n_rows = task.rows, first = task.extra, tid = threadIdx.x;
  if (first < 0 || first > INT32_MAX - 1024 - n_rows) {
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
  constexpr int C = HD / 8;                      // pieces of a row of one head
  const int head0 = blockIdx.y * P.heads, heads = min(P.heads, P.n_kv - head0);
  const size_t cell0 = (size_t)page * P.n_kv + head0;
  const int slot0 = lo - page_no * P.page, row_items = heads * C, items = (hi - lo) * row_items;
  __nv_bfloat16* const ko = P.Ko + (size_t)(row0 + (lo - first)) * P.ld + (size_t)head0 * HD;
  __nv_bfloat16* const vo = P.Vo + (size_t)(row0 + (lo - first)) * P.ld + (size_t)head0 * HD;
  constexpr int U = 4;
  for (int id0 = tid; id0 < items; id0 += U * 256) {
    uint2 a[U], b[U];
    float sk[U], sv[U];
    int to[U];                                   // element of the output, from the CTA's first
    int64_t row[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int id = id0 + u * 256, j = id / row_items, in = id - j * row_items, h = in / C;
      row[u] = (int64_t)j * P.ld;
      to[u] = in * 8;
      if (id < items) {
        const size_t from = ((cell0 + h) * P.page + slot0 + j) * HD + (in % C) * 8;
        a[u] = __ldg(reinterpret_cast<const uint2*>(P.k + from));
        b[u] = __ldg(reinterpret_cast<const uint2*>(P.v + from));
        sk[u] = __ldg(P.k_scale + cell0 + h);
        sv[u] = __ldg(P.v_scale + cell0 + h);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (id0 + u * 256 < items) {
        *reinterpret_cast<uint4*>(ko + row[u] + to[u]) = values8(a[u], sk[u]);
        *reinterpret_cast<uint4*>(vo + row[u] + to[u]) = values8(b[u], sv[u]);
      }
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
  return launch_kernel(rope_append_kernel<HD, T, N>, dim3(tasks, 2 * P.n_kv), dim3(T), 0, st, true, P) == cudaSuccess ? FPT_OK
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
  if (n_kv > 32767 || n_pos > INT32_MAX - 1024 || M > INT32_MAX - 1024) return FPT_ERR_UNSUPPORTED;
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
  // The pages that the rows may touch, numbered without their lengths; few rows a sequence: a task for each row, of which the first in a page
  // works (64 sequences of one token, 16 CTAs a task: 7.6 -> 5.9 us).
  const int64_t by_page = block_tasks(M, n_seqs, P.page);
  P.by_row = cu_new && M < by_page;
  const int64_t tasks = !cu_new ? n_seqs : P.by_row ? M : by_page;
  if (tasks > INT32_MAX) return FPT_ERR_UNSUPPORTED;
  // one token a sequence: its heads' pieces are few, and what a CTA has to do beside them is to round the page's held tokens
  // again where its scale grows; otherwise a page a CTA
  if (!cu_new) return hd == 128 ? launch_rope<128, 64, 1>(st, P, (unsigned)tasks) : launch_rope<64, 64, 1>(st, P, (unsigned)tasks);
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
  if (!cu_out || n_seqs <= 0 || M < 0 || !K_out != (M == 0) || !V_out != (M == 0)) return FPT_ERR_BAD_ARG;
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
  const int64_t tasks = block_tasks(M, n_seqs, P.page);
  if (tasks > INT32_MAX) return FPT_ERR_UNSUPPORTED;
  P.heads = 8192 / (cache->page * cache->head_dim);
  if (P.heads < 1) P.heads = 1;
  if (P.heads > cache->n_kv) P.heads = cache->n_kv;
  const dim3 grid((unsigned)tasks, (unsigned)((cache->n_kv + P.heads - 1) / P.heads));
  cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t e = cache->head_dim == 128 ? launch_kernel(kv_gather_kernel<128>, grid, dim3(256), 0, st, true, P)
                                               : launch_kernel(kv_gather_kernel<64>, grid, dim3(256), 0, st, true, P);
  return e == cudaSuccess ? FPT_OK : FPT_ERR_CUDA;
}
