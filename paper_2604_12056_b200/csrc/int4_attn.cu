// Attention over a cache held in 4 bits: losa_int4_attn (every block token over the whole cache) and stage 4 of the
// method on such a cache (active tokens over the listed pages; Section 2.2, Section 4.2).
//
// The pages to read form one flat list over (sequence, KV head, group of query rows), cut into equal shares, so
// ragged batches leave no SM idle; partial results of a segment that several CTAs share meet by log-sum-exp.
#include <cuda.h>

#include <algorithm>
#include <cstring>
#include <type_traits>

#include "kernels.h"
#include "page_formats.cuh"

namespace losa {
namespace {

struct I4Params {
  const __nv_bfloat16* q;
  const uint8_t *k_scale, *v_scale;
  const int32_t *page_table, *kv_len;
  const int32_t *active_idx, *n_active;            // null: all block tokens
  const int32_t *union_pages, *union_count;        // null: every page of the prefix
  void* out;                                       // [N, B, H_q, d] fp32 or bf16
  float* lse;                                      // or null
  int out_bf16;
  float* partials;
  uint32_t* tickets;
  int32_t* status;
  int N, B, Hq, Hkv, G, g, Pmax, n_phys, n_sk, n_rg, stages, min_units, bar_off;
  float sm_scale;
  long long wait_cycles;
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
__device__ __forceinline__ void i4_tma(uint32_t dst, const CUtensorMap* map, uint32_t bar, int t0, int kh, int phys, unsigned long long policy) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%3, %4, %5, %6}], [%2], %7;"
      ::"r"(dst), "l"(map), "r"(bar), "r"(0), "r"(t0), "r"(kh), "r"(phys), "l"(policy) : "memory");
}
__device__ __forceinline__ void i4_bulk(uint32_t dst, const uint8_t* src, uint32_t bar, uint32_t bytes) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

#include "int4_attn_mma.cuh"

// ===================================================================== host side
constexpr int kI4SmemLimit = 232448;

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

int unit_tokens(const losa_shape_t& sh) { return std::min(32, sh.page_size); }

int32_t encode_codes(losa_ctx* c, unsigned char* blob, const void* pool, const losa_kv_t* kv) {
  const losa_shape_t& sh = c->shape;
  if (!c->encode_fn) {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult qres;
    LOSA_CUDA_TRY(c, cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres));
    if (!fn || qres != cudaDriverEntryPointSuccess) return cuda_fail(c, cudaErrorSymbolNotFound);
    c->encode_fn = fn;
  }
  const cuuint32_t row = static_cast<cuuint32_t>(sh.head_dim / 2);
  const cuuint64_t dims[4] = {row, static_cast<cuuint64_t>(sh.page_size), static_cast<cuuint64_t>(sh.n_kv_heads), static_cast<cuuint64_t>(kv->n_phys_pages)};
  const cuuint64_t strides[3] = {static_cast<cuuint64_t>(kv->stride_tok), static_cast<cuuint64_t>(kv->stride_head), static_cast<cuuint64_t>(kv->stride_page)};
  const cuuint32_t box[4] = {row, static_cast<cuuint32_t>(unit_tokens(sh)), 1, 1}, estr[4] = {1, 1, 1, 1};
  const CUresult r = reinterpret_cast<EncodeTiledFn>(c->encode_fn)(
      reinterpret_cast<CUtensorMap*>(blob), CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void*>(pool), dims, strides, box, estr,
      CU_TENSOR_MAP_INTERLEAVE_NONE, sh.head_dim == 128 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_NONE,
      CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) {
    c->last_cuda_error = static_cast<int32_t>(r);
    return LOSA_ERR_CUDA;
  }
  return LOSA_OK;
}

int32_t ensure_code_maps(losa_ctx* c, const losa_kv_t* kv) {
  losa::Int4Maps& m = c->int4_maps;
  if (m.key_k == kv->k_pages && m.key_v == kv->v_pages && m.strides[0] == kv->stride_page && m.strides[1] == kv->stride_head &&
      m.strides[2] == kv->stride_tok && m.n_phys == kv->n_phys_pages)
    return LOSA_OK;
  alignas(64) unsigned char k[128], v[128];
  int32_t rc = encode_codes(c, k, kv->k_pages, kv);
  if (rc == LOSA_OK) rc = encode_codes(c, v, kv->v_pages, kv);
  if (rc != LOSA_OK) return rc;
  memcpy(m.k, k, sizeof(k));
  memcpy(m.v, v, sizeof(v));
  m.key_k = kv->k_pages;
  m.key_v = kv->v_pages;
  m.strides[0] = kv->stride_page;
  m.strides[1] = kv->stride_head;
  m.strides[2] = kv->stride_tok;
  m.n_phys = kv->n_phys_pages;
  return LOSA_OK;
}

// where the barriers lie: behind the rings, whose place the merge tile takes
template <int D, int NT>
int mma_bar_off(int warps, int stages, int ut) {
  return (std::max(warps * stages * (i4_unit_codes<D>(ut) + i4_unit_scales<D>(ut)), i4_merge_bytes<D, NT>(warps)) + 15) / 16 * 16;
}
template <int D, int NT>
int mma_smem(int warps, int stages, int ut, int n_sk) {
  return 1024 + mma_bar_off<D, NT>(warps, stages, ut) + warps * stages * (8 + 4) + 16 + kI4Head + (NT == 4 ? (D / 16) * NT * 32 * 8 : 0) + (n_sk + 1) * 4;
}

template <int D, int NT, int UT>
int32_t launch_mma(losa_ctx* c, I4Params p, int max_rows, cudaStream_t st) {
  constexpr int R = 8 * NT;
  auto kernel = int4_mma_kernel<D, NT, UT>;
  const int bit = 1 << (NT == 1 ? 0 : NT == 2 ? 1 : 2);        // a context has one head dimension and one page size
  if (!(c->int4_attr_set & bit)) {
    LOSA_CUDA_TRY(c, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kI4SmemLimit));
    c->int4_attr_set |= bit;
  }
  p.n_rg = (max_rows + R - 1) / R;
  const int W = i4_warps(NT);
  int stages = kI4Stages;
  while (stages < 8 && mma_smem<D, NT>(W, stages + 1, UT, p.n_sk) <= kI4SmemLimit) ++stages;
  p.stages = stages;
  p.bar_off = mma_bar_off<D, NT>(W, stages, UT);
  p.min_units = 2;
  int grid = c->n_sms;
  grid = std::min<long long>(grid, static_cast<long long>(c->lay.n_slots) * kRowsPerGroup / (2 * R));      // room for the records
  if (c->profile) LOSA_CUDA_TRY(c, cudaEventRecord(c->ev_begin, st));
  launch_k(kernel, grid, W * 32, mma_smem<D, NT>(W, stages, UT, p.n_sk), st, *reinterpret_cast<const CUtensorMap*>(c->int4_maps.k),
           *reinterpret_cast<const CUtensorMap*>(c->int4_maps.v), p);
  if (c->profile) LOSA_CUDA_TRY(c, cudaEventRecord(c->ev_end, st));
  return after_launch(c);
}

template <int D, int UT>
int32_t launch_rows(losa_ctx* c, const I4Params& p, cudaStream_t st) {
  const int max_rows = p.B * p.G;
  if (max_rows <= 8) return launch_mma<D, 1, UT>(c, p, max_rows, st);
  if (max_rows <= 16) return launch_mma<D, 2, UT>(c, p, max_rows, st);
  return launch_mma<D, 4, UT>(c, p, max_rows, st);
}

int32_t launch(losa_ctx* c, I4Params& p, const void* q, const losa_kv_t* kv, cudaStream_t st) {
  const losa_shape_t& sh = c->shape;
  const int32_t rc = ensure_code_maps(c, kv);
  if (rc != LOSA_OK) return rc;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.k_scale = reinterpret_cast<const uint8_t*>(kv->k_scale);
  p.v_scale = reinterpret_cast<const uint8_t*>(kv->v_scale);
  p.page_table = kv->page_table;
  p.kv_len = kv->kv_len;
  p.partials = reinterpret_cast<float*>(c->ws + c->lay.partials);
  p.tickets = reinterpret_cast<uint32_t*>(c->ws + c->lay.int4_tickets);
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
  p.wait_cycles = c->wait_cycles > 0 ? c->wait_cycles : kWaitCycles;
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
