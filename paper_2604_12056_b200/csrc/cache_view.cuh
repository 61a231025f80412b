// The paged cache in its formats, new tokens over it, and which keys each of them sees: what the kernels of windowed attention and of
// the keys' weights share.
#pragma once
#include "common.cuh"
#include "page_formats.cuh"

namespace losa {

enum : int { kRowsF32 = 0, kRowsBf16 = 1, kRowsFp8 = 2, kRowsInt4 = 3 };      // how a token's row lies in the cache
template <int FMT> struct RowFormat;
template <> struct RowFormat<kRowsF32> { using Query = float; static constexpr int bits = 32; };
template <> struct RowFormat<kRowsBf16> { using Query = __nv_bfloat16; static constexpr int bits = 16; };
template <> struct RowFormat<kRowsFp8> { using Query = __nv_bfloat16; static constexpr int bits = 8; };
template <> struct RowFormat<kRowsInt4> { using Query = __nv_bfloat16; static constexpr int bits = 4; };

struct CacheParams {
  const uint8_t *k_pages, *v_pages;
  int64_t stride_page, stride_head, stride_tok;      // bytes
  const void *k_scale, *v_scale;
  const int32_t *page_table, *kv_len;
  int N, Hkv, G, g, Pmax, n_phys;
};
struct QueryParams {
  const void* q;
  int64_t stride;                                    // elements
  const int32_t *cu, *start;
  int T, max_tokens, window, sinks, span;
};
// A sequence as it is worked on: its tokens are cu .. cu + count - 1 at places start .., over len keys.  One that is left out has start -1 and no tokens.
struct alignas(16) Sequence { int cu, count, start, len; };

// What of a sequence can be used (called by one lane per sequence where a report shall come once).
__device__ __forceinline__ Sequence sequence_of(const CacheParams& c, const QueryParams& q, int s, int32_t* status) {
  Sequence x;
  const int next = q.cu[s + 1];
  x.cu = q.cu[s];
  x.start = q.start[s];
  x.len = c.kv_len[s];
  x.count = next - x.cu;
  const long long held = static_cast<long long>(c.Pmax) * c.g;
  bool bad = false;
  if (x.len < 0 || x.len > held) { x.len = x.len < 0 ? 0 : static_cast<int>(held); bad = true; }
  if (x.cu < 0 || next > q.T || x.count < 0 || x.start < 0 || x.start > (1 << 30)) {
    x.count = 0;
    x.start = -1;
    bad = true;
  } else if (x.count > q.max_tokens) {
    x.count = q.max_tokens;
    bad = true;
  }
  if (bad && status) set_status(status, LOSA_ERR_BOUNDS);
  return x;
}
// Keys of the token at `place`: 0 <= j < x, and j >= y or j < sinks.
__device__ __forceinline__ int2 keys_of(const QueryParams& q, const Sequence& x, int place) {
  const int end = q.span == 1 ? place + 1 : (place / q.span + 1) * q.span;
  return make_int2(min(end, x.len), q.window > 0 ? max(0, place + 1 - q.window) : 0);
}

// Physical page of a place, -1 (reported) where the table names none of the pool.
__device__ __forceinline__ int page_of(const CacheParams& c, int s, int page, int32_t* status) {
  const int at = c.page_table[static_cast<size_t>(s) * c.Pmax + page];
  if (at >= 0 && at < c.n_phys) return at;
  set_status(status, LOSA_ERR_BOUNDS);
  return -1;
}
// Eight elements of the row at (page, head, slot), element 8 c on.
template <int FMT, int D>
__device__ __forceinline__ void cache_load8(const CacheParams& c, const uint8_t* pool, const void* scales, int page, int kh, int slot, int chunk, float (&v)[8]) {
  const uint8_t* row = pool + page * c.stride_page + kh * c.stride_head + slot * c.stride_tok;
  if constexpr (FMT == kRowsF32) {
    load8(reinterpret_cast<const float*>(row) + chunk * 8, v);
  } else if constexpr (FMT == kRowsBf16) {
    load8(reinterpret_cast<const __nv_bfloat16*>(row) + chunk * 8, v);
  } else if constexpr (FMT == kRowsFp8) {
    const uint2 w = *reinterpret_cast<const uint2*>(row + chunk * 8);
    const float scale = static_cast<const float*>(scales)[static_cast<size_t>(page) * c.Hkv + kh];
    fp8_decode8(w, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= scale;
  } else {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(row + chunk * 4);
    const size_t at = ((static_cast<size_t>(page) * c.Hkv + kh) * c.g + slot) * (D / kInt4Run) + chunk / 4;
    int4_decode8(w, int4_scale_value(static_cast<const uint8_t*>(scales)[at]), v);
  }
}

inline CacheParams cache_params(const losa_ctx* c, const losa_kv_t* kv) {
  const losa_shape_t& sh = c->shape;
  const int64_t es = kv->kv_format != LOSA_KV_NATIVE ? 1 : sh.dtype == LOSA_BF16 ? 2 : 4;
  CacheParams p;
  p.k_pages = static_cast<const uint8_t*>(kv->k_pages);
  p.v_pages = static_cast<const uint8_t*>(kv->v_pages);
  p.stride_page = kv->stride_page * es;
  p.stride_head = kv->stride_head * es;
  p.stride_tok = kv->stride_tok * es;
  p.k_scale = kv->k_scale;
  p.v_scale = kv->v_scale;
  p.page_table = kv->page_table;
  p.kv_len = kv->kv_len;
  p.N = sh.batch;
  p.Hkv = sh.n_kv_heads;
  p.G = sh.n_q_heads / sh.n_kv_heads;
  p.g = sh.page_size;
  p.Pmax = sh.max_pages_per_seq;
  p.n_phys = kv->n_phys_pages;
  return p;
}
inline QueryParams query_params(const losa_queries_t* q) {
  return {q->q, q->q_stride, q->cu, q->start, q->n_tokens, q->max_tokens, q->window, q->sinks, q->span};
}
inline int row_format(const losa_ctx* c, const losa_kv_t* kv) {
  return kv->kv_format == LOSA_KV_FP8_E4M3 ? kRowsFp8 : kv->kv_format == LOSA_KV_INT4 ? kRowsInt4 : c->shape.dtype == LOSA_BF16 ? kRowsBf16 : kRowsF32;
}

}  // namespace losa
