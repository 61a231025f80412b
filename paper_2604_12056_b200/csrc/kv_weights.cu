// The softmax weight that every cached token receives from new tokens: losa_kv_weights.
//
// The log-normalisers are known, so a key's weight is a sum over the rows (token, head of its KV head) that see it and needs nothing of
// the other keys.  No sum depends on the order in which CTAs run.
#include <algorithm>
#include <cstring>
#include <type_traits>

#include "kernels.h"
#include "tc_cache_ops.cuh"
#include "work_list.cuh"

namespace losa {
namespace {

struct WeightParams : ListParams {
  const float* lse;
  float* weights;                                    // [n_phys, H_kv, g]
  float* partials;                                   // [n_ctas][2][keys of a tile]
  float scale_log2;
};

// Tokens of a sequence that see any of the keys key0 .. key0 + n - 1: x .. y - 1.
__device__ __forceinline__ int2 tokens_over(const ListParams& p, const Sequence& x, int key0, int n) {
  const int first = p.q.span == 1 ? key0 : key0 / p.q.span * p.q.span;              // the first place that sees key0
  const long long last = p.q.window == 0 || key0 < p.q.sinks ? 1ll << 40 : static_cast<long long>(key0) + n - 1 + p.q.window;
  const int t0 = min(max(0, first - x.start), x.count), t1 = static_cast<int>(max(0ll, min(static_cast<long long>(x.count), last - x.start)));
  return make_int2(t0, max(t0, t1));
}

// Where a key's weight stands (null: there is no such key), and what is left of it.
struct Held {
  float* at;
  float old;
  bool kept;
};
__device__ __forceinline__ Held held_weight(const WeightParams& p, const Sequence& x, int s, int kh, int key) {
  Held h = {nullptr, 0.f, false};
  if (key >= x.len) return h;
  const int page = page_of(p.c, s, key / p.c.g, p.status);
  if (page < 0) return h;
  h.at = p.weights + (static_cast<size_t>(page) * p.c.Hkv + kh) * p.c.g + key % p.c.g;
  h.kept = key < x.start && p.keep != 0.f;           // (what stood for tokens that are new is not looked at; with keep 0 neither is the rest)
  if (h.kept) h.old = *h.at;
  return h;
}
// ... and the weight from the rows' sum.
__device__ __forceinline__ void put_weight(const WeightParams& p, const Held& h, float sum) {
  if (h.at) *h.at = h.kept ? fmaf(p.keep, h.old, sum) : sum;
}

#include "kv_weights_f32.cuh"
#include "kv_weights_tc.cuh"

template <int D>
int32_t launch_f32(losa_ctx* c, const WeightParams& p, cudaStream_t st) {
  auto kernel = weights_f32_kernel<D>;
  constexpr int bit = 16 << kRowsF32;
  if (!(c->window_attr_set & bit)) {
    LOSA_CUDA_TRY(c, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, weights_smem<D>()));
    c->window_attr_set |= bit;
  }
  const int tiles = (p.c.Pmax * p.c.g + kWgtKeys - 1) / kWgtKeys;
  if (tiles == 0) return LOSA_OK;
  launch_k(kernel, dim3(tiles, p.c.Hkv, p.c.N), kWgtThreads, weights_smem<D>(), st, p);
  return after_launch(c);
}

template <int FMT, int D, int GP>
int32_t launch_tc(losa_ctx* c, WeightParams& p, const losa_kv_t* kv, cudaStream_t st) {
  using Tc = WeightsTc<FMT, D, GP>;
  const int32_t rc = Tc::quant ? raw_tensor_maps(c, kv) : pool_tensor_maps(c, kv);
  if (rc != LOSA_OK) return rc;
  CUtensorMap mk, mq;
  memcpy(&mk, Tc::quant ? c->tmap_raw[0] : c->tmap_k, sizeof(mk));
  if (p.q.T > 0) {
    const int32_t rq = query_tensor_map(c, p.q.q, p.q.stride, p.q.T, 128 / p.c.G, &mq);
    if (rq != LOSA_OK) return rq;
  } else {
    mq = mk;                                         // (not used)
  }
  p.n_ctas = c->n_sms;
  p.pad = 1;
  p.least = 2;
  place_plan(c, p);
  p.partials = reinterpret_cast<float*>(c->ws + c->lay.scores);
  auto kernel = weights_tc_kernel<FMT, D, GP>;
  constexpr int bit = 16 << FMT;
  if (!(c->window_attr_set & bit)) {
    LOSA_CUDA_TRY(c, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Tc::smem));
    c->window_attr_set |= bit;
  }
  launch_k(list_plan_kernel<KeyTiles>, 1, kPlanThreads, 0, st, static_cast<const ListParams&>(p));
  launch_k(kernel, p.n_ctas, Tc::warps * 32, Tc::smem, st, mk, mq, p);
  launch_k(weights_join_kernel, p.n_ctas, kKwKeys, 0, st, p);
  return after_launch(c, 3);
}

}  // namespace

int32_t launch_kv_weights(losa_ctx* c, const losa_queries_t* q, const losa_kv_t* kv, const float* lse, float keep, float* weights, cudaStream_t st) {
  WeightParams p = {};
  p.c = cache_params(c, kv);
  p.q = query_params(q);
  p.lse = lse;
  p.weights = weights;
  p.keep = keep;
  p.status = status_ptr(c);
  set_bounds(c, p);
  p.scale_log2 = c->shape.sm_scale * kLog2e;
  auto run = [&](auto f, auto d) -> int32_t {
    constexpr int FMT = decltype(f)::value, D = decltype(d)::value;
    if constexpr (FMT == kRowsF32) {
      return launch_f32<D>(c, p, st);
    } else {
      return c->shape.page_size == 16 ? launch_tc<FMT, D, 16>(c, p, kv, st) : c->shape.page_size == 32 ? launch_tc<FMT, D, 32>(c, p, kv, st) : launch_tc<FMT, D, 64>(c, p, kv, st);
    }
  };
  auto with_dim = [&](auto f) { return c->shape.head_dim == 128 ? run(f, std::integral_constant<int, 128>{}) : run(f, std::integral_constant<int, 64>{}); };
  switch (row_format(c, kv)) {
    case kRowsF32: return with_dim(std::integral_constant<int, kRowsF32>{});
    case kRowsBf16: return with_dim(std::integral_constant<int, kRowsBf16>{});
    case kRowsFp8: return with_dim(std::integral_constant<int, kRowsFp8>{});
    default: return with_dim(std::integral_constant<int, kRowsInt4>{});
  }
}

}  // namespace losa
