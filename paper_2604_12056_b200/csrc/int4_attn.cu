// Attention over a cache held in 4 bits: losa_int4_attn (every block token over the whole cache) and stage 4 of the
// method on such a cache (active tokens over the listed pages; Section 2.2, Section 4.2).
//
// The pages to read form one flat list over (sequence, KV head, group of query rows), cut into equal shares, so
// ragged batches leave no SM idle; partial results of a segment that several CTAs share meet by log-sum-exp.
#include <algorithm>
#include <type_traits>

#include "kernels.h"
#include "page_formats.cuh"

namespace losa {
namespace {

struct I4Params {
  const __nv_bfloat16* q;
  const uint8_t *k_pages, *v_pages, *k_scale, *v_scale;
  int64_t stride_page, stride_head, stride_tok;
  const int32_t *page_table, *kv_len;
  const int32_t *active_idx, *n_active;            // null: all block tokens
  const int32_t *union_pages, *union_count;        // null: every page of the prefix
  void* out;                                       // [N, B, H_q, d] fp32 or bf16
  float* lse;                                      // or null
  int out_bf16;
  float* partials;
  int2* seg_records;                                // per segment: first CTA and number of its records (0: none to merge)
  int32_t* status;
  int N, B, Hq, Hkv, G, g, Pmax, n_phys, n_sk, n_rg, min_units, pad;
  float sm_scale;
};

__device__ __forceinline__ int clamp_rows(int na, int B) { return na < 0 ? 0 : (na > B ? B : na); }
// row of q / out (in units of d elements) of query row r of (s, kh); -1: no such token
__device__ __forceinline__ long long i4_row(const I4Params& p, int s, int kh, int r) {
  const int a = r / p.G, gi = r - a * p.G;
  int tok = a;
  if (p.active_idx) {
    tok = p.active_idx[s * p.B + a];
    if (tok < 0 || tok >= p.B) { set_status(p.status, LOSA_ERR_BOUNDS); return -1; }
  }
  return (static_cast<long long>(s) * p.B + tok) * p.Hq + kh * p.G + gi;
}
__device__ __forceinline__ void i4_store4(const I4Params& p, long long at, float a, float b, float c, float d) {
  if (p.out_bf16) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(a, b), y = __floats2bfloat162_rn(c, d);
    *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.out) + at) = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
  } else {
    *reinterpret_cast<float4*>(static_cast<float*>(p.out) + at) = make_float4(a, b, c, d);
  }
}
// columns c .. c + 3 of a row from its un-normalised sums (relative to 2^M, a quarter of the values)
__device__ __forceinline__ void i4_finish(const I4Params& p, int s, int kh, int r, int c, int d, const float4& acc, float M, float L) {
  const long long row = i4_row(p, s, kh, r);
  if (row < 0) return;
  const bool empty = L == 0.f;                      // (a sum that is no number stays visible)
  const float inv = empty ? 0.f : 4.f / L;
  i4_store4(p, row * d + c, acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
  if (c == 0 && p.lse) p.lse[row] = empty ? -INFINITY : (M + log2f(L)) * kLn2;
}
__device__ __forceinline__ float i4_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
#include "int4_attn_mma.cuh"

// ===================================================================== host side
constexpr int kI4SmemLimit = 232448;

int unit_tokens(const losa_shape_t& sh) { return std::min(32, sh.page_size); }

template <int D, int NT>
int mma_smem(int warps, int stages, int ut, int n_sk) {
  return 1024 + warps * (stages * (i4_unit_codes<D>(ut) + i4_unit_scales<D>(ut) + 4) + 8 * NT * D * 2) + i4_merge_bytes<D, NT>(warps) + (32 + n_sk + 1) * 4;
}

template <int D, int NT, int UT>
int32_t launch_mma(losa_ctx* c, I4Params p, int max_rows, cudaStream_t st) {
  constexpr int R = 8 * NT;
  constexpr int S = 2;
  auto kernel = int4_mma_kernel<D, NT, UT, S>;
  const int bit = NT;        // a context has one head dimension and one page size
  if (!(c->int4_attr_set & bit)) {
    LOSA_CUDA_TRY(c, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kI4SmemLimit));
    c->int4_attr_set |= bit;
  }
  p.n_rg = (max_rows + R - 1) / R;
  // Few segments: one CTA of all warps per SM.  More segments than SMs: CTAs of four warps, whose ends and starts overlap.
  const bool many = p.n_sk * p.n_rg > c->n_sms;
  const int W = many ? 4 : i4_warps(NT), per_sm = many ? i4_warps(NT) / 4 : 1;
  p.min_units = 1;
  p.pad = many ? 10 : 24;
  int grid = c->n_sms * per_sm;
  grid = std::min<long long>(grid, static_cast<long long>(c->lay.n_slots) * kRowsPerGroup / (2 * R));      // room for the records
  if (c->profile) LOSA_CUDA_TRY(c, cudaEventRecord(c->ev_begin, st));
  launch_k(kernel, grid, W * 32, mma_smem<D, NT>(W, S, UT, p.n_sk), st, p);
  if (c->profile) LOSA_CUDA_TRY(c, cudaEventRecord(c->ev_end, st));
  const int32_t rc = after_launch(c);
  if (rc != LOSA_OK) return rc;
  launch_k(int4_combine_kernel<D, R>, (p.n_sk * p.n_rg * R + kI4CombineWarps - 1) / kI4CombineWarps, kI4CombineWarps * 32, 0, st, p);
  return after_launch(c);
}

template <int D, int UT>
int32_t launch_rows(losa_ctx* c, const I4Params& p, cudaStream_t st) {
  const int max_rows = p.B * p.G;
  if (max_rows <= 8) return launch_mma<D, 1, UT>(c, p, max_rows, st);
  return launch_mma<D, 2, UT>(c, p, max_rows, st);
}

int32_t launch(losa_ctx* c, I4Params& p, const void* q, const losa_kv_t* kv, cudaStream_t st) {
  const losa_shape_t& sh = c->shape;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.k_pages = static_cast<const uint8_t*>(kv->k_pages);
  p.v_pages = static_cast<const uint8_t*>(kv->v_pages);
  p.stride_page = kv->stride_page;
  p.stride_head = kv->stride_head;
  p.stride_tok = kv->stride_tok;
  p.k_scale = reinterpret_cast<const uint8_t*>(kv->k_scale);
  p.v_scale = reinterpret_cast<const uint8_t*>(kv->v_scale);
  p.page_table = kv->page_table;
  p.kv_len = kv->kv_len;
  p.partials = reinterpret_cast<float*>(c->ws + c->lay.partials);
  p.seg_records = reinterpret_cast<int2*>(c->ws + c->lay.int4_records);
  p.status = status_ptr(c);
  p.N = sh.batch;
  p.B = sh.block_size;
  p.Hq = sh.n_q_heads;
  p.Hkv = sh.n_kv_heads;
  p.G = sh.n_q_heads / sh.n_kv_heads;
  p.g = sh.page_size;
  p.Pmax = sh.max_pages_per_seq;
  p.n_phys = kv->n_phys_pages;
  p.n_sk = sh.batch * sh.n_kv_heads;
  p.sm_scale = sh.sm_scale;
  const bool ut16 = unit_tokens(sh) == 16;
  if (sh.head_dim == 128) return ut16 ? launch_rows<128, 16>(c, p, st) : launch_rows<128, 32>(c, p, st);
  return ut16 ? launch_rows<64, 16>(c, p, st) : launch_rows<64, 32>(c, p, st);
}

}  // namespace

int32_t launch_int4_attn(losa_ctx* c, const void* q, const losa_kv_t* kv, void* out, float* lse_opt, cudaStream_t st) {
  I4Params p = {};
  p.out = out;
  p.out_bf16 = 1;
  p.lse = lse_opt;
  return launch(c, p, q, kv, st);
}

int32_t launch_int4_prefix_attn(losa_ctx* c, const void* q, const losa_kv_t* kv, const int32_t* active_idx, const int32_t* n_active,
                                const int32_t* union_pages, const int32_t* union_count, losa_state_t* state, cudaStream_t st) {
  I4Params p = {};
  p.active_idx = active_idx;
  p.n_active = n_active;
  p.union_pages = union_pages;
  p.union_count = union_count;
  p.out = state->o_p;
  p.out_bf16 = state->o_p_format == LOSA_STATE_BF16 ? 1 : 0;
  p.lse = state->lse_p;
  return launch(c, p, q, kv, st);
}

}  // namespace losa
