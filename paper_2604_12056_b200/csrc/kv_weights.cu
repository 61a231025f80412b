// The softmax weight that every cached token receives from new tokens: losa_kv_weights.
//
// The log-normalisers are known, so a key's weight is a sum over the rows (token, head of its KV head) that see it and needs nothing of
// the other keys: a CTA has a run of keys to itself and goes over the rows, in order, and no sum depends on another CTA.
#include <algorithm>
#include <type_traits>

#include "cache_view.cuh"
#include "kernels.h"

namespace losa {
namespace {

struct WeightParams {
  CacheParams c;
  QueryParams q;
  const float* lse;
  float* weights;                                    // [n_phys, H_kv, g]
  float keep;
  int32_t* status;
  float scale_log2;
};

// Rows of a sequence that see any of the keys key0 .. key0 + n - 1.
__device__ __forceinline__ int2 rows_over(const WeightParams& p, const Sequence& x, int key0, int n) {
  const int first = p.q.span == 1 ? key0 : key0 / p.q.span * p.q.span;              // the first place that sees key0
  const long long last = p.q.window == 0 || key0 < p.q.sinks ? 1ll << 40 : static_cast<long long>(key0) + n - 1 + p.q.window;
  const int t0 = min(max(0, first - x.start), x.count), t1 = static_cast<int>(max(0ll, min(static_cast<long long>(x.count), last - x.start)));
  return make_int2(t0 * p.c.G, max(t0, t1) * p.c.G);
}

constexpr int kWgtKeys = 64, kWgtRows = 64, kWgtThreads = 128;
template <int D> constexpr int weights_smem() { return (kWgtRows * D + kWgtKeys * (D + 4) + 3 * kWgtRows + 8 * kWgtKeys) * 4; }

// fp32 on the CUDA cores: 64 keys of a CTA, 64 rows at a time, a thread has 8 rows by 4 keys.
template <int FMT, int D>
__global__ void __launch_bounds__(kWgtThreads, 3) weights_f32_kernel(const __grid_constant__ WeightParams p) {
  using T = typename RowFormat<FMT>::Query;
  constexpr int R = kWgtRows, GT = kWgtKeys, KS = D + 4, C8 = D / 8;
  extern __shared__ __align__(16) float smem[];
  float *sq = smem, *sk = sq + R * D, *sl = sk + GT * KS, *part = sl + R;
  int2* ends = reinterpret_cast<int2*>(part + 8 * GT);
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  grid_dep_wait();
  const int s = blockIdx.z, kh = blockIdx.y, key0 = blockIdx.x * GT;
  const Sequence x = sequence_of(p.c, p.q, s, blockIdx.x == 0 && kh == 0 && tid == 0 ? p.status : nullptr);
  if (key0 >= x.len) return;
  const int2 rows = rows_over(p, x, key0, min(GT, x.len - key0));
  if (rows.x >= rows.y && p.keep == 1.f && key0 + GT <= x.start) return;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  if (rows.x < rows.y) {
    for (int i = tid; i < GT * C8; i += kWgtThreads) {
      const int t = i / C8, ch = i - t * C8, key = key0 + t;
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = 0.f;
      const int page = key < x.len ? page_of(p.c, s, key / p.c.g, p.status) : -1;
      if (page >= 0) cache_load8<FMT, D>(p.c, p.c.k_pages, p.c.k_scale, page, kh, key % p.c.g, ch, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) sk[t * KS + ch * 8 + k] = v[k];
    }
  }
  for (int row0 = rows.x; row0 < rows.y; row0 += R) {
    __syncthreads();
    for (int i = tid; i < R * C8; i += kWgtThreads) {
      const int r = i / C8, ch = i - r * C8, row = row0 + r;
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = 0.f;
      if (row < rows.y) {
        const int t = row / p.c.G;
        load8(static_cast<const T*>(p.q.q) + (static_cast<long long>(x.cu) + t) * p.q.stride + (kh * p.c.G + row - t * p.c.G) * D + ch * 8, v);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) sq[r * D + ch * 8 + k] = v[k];
    }
    for (int r = tid; r < R; r += kWgtThreads) {
      const int row = row0 + r, t = row / p.c.G;
      const bool on = row < rows.y;
      const float l = on ? p.lse[(static_cast<long long>(x.cu) + t) * (p.c.Hkv * p.c.G) + kh * p.c.G + (row - t * p.c.G)] : -INFINITY;
      sl[r] = l * kLog2e;
      ends[r] = on && l != -INFINITY ? keys_of(p.q, x, x.start + t) : make_int2(0, 0);       // (a row that saw nothing gives nothing)
    }
    __syncthreads();
    float a[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) a[i][k] = 0.f;
#pragma unroll 2
    for (int c = 0; c < D; c += 4) {
      float4 u[8], b[4];
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = *reinterpret_cast<const float4*>(sq + (ty * 8 + i) * D + c);
#pragma unroll
      for (int k = 0; k < 4; ++k) b[k] = *reinterpret_cast<const float4*>(sk + (tx + 16 * k) * KS + c);
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) a[i][k] = fmaf(u[i].x, b[k].x, fmaf(u[i].y, b[k].y, fmaf(u[i].z, b[k].z, fmaf(u[i].w, b[k].w, a[i][k]))));
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int2 e = ends[ty * 8 + i];
      const float l = sl[ty * 8 + i];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int key = key0 + tx + 16 * k;
        if (key < e.x && (key >= e.y || key < p.q.sinks)) sum[k] += exp2f(fmaf(a[i][k], p.scale_log2, -l));
      }
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) part[ty * GT + tx + 16 * k] = sum[k];
  __syncthreads();
  if (tid < GT && key0 + tid < x.len) {
    const int key = key0 + tid, page = page_of(p.c, s, key / p.c.g, p.status);
    if (page < 0) return;
    float* at = p.weights + (static_cast<size_t>(page) * p.c.Hkv + kh) * p.c.g + key % p.c.g;
    float total = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) total += part[i * GT + tid];
    // (what stood for tokens that are new is not looked at; with keep 0 neither is the rest)
    *at = key < x.start && p.keep != 0.f ? fmaf(p.keep, *at, total) : total;
  }
}

template <int FMT, int D>
int32_t launch(losa_ctx* c, const WeightParams& p, cudaStream_t st) {
  auto kernel = weights_f32_kernel<FMT, D>;
  LOSA_CUDA_TRY(c, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, weights_smem<D>()));
  const int tiles = (p.c.Pmax * p.c.g + kWgtKeys - 1) / kWgtKeys;
  if (tiles == 0) return LOSA_OK;
  launch_k(kernel, dim3(tiles, p.c.Hkv, p.c.N), kWgtThreads, weights_smem<D>(), st, p);
  return after_launch(c);
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
  p.scale_log2 = c->shape.sm_scale * kLog2e;
  auto run = [&](auto f) {
    constexpr int FMT = decltype(f)::value;
    return c->shape.head_dim == 128 ? launch<FMT, 128>(c, p, st) : launch<FMT, 64>(c, p, st);
  };
  switch (row_format(c, kv)) {
    case kRowsF32: return run(std::integral_constant<int, kRowsF32>{});
    case kRowsBf16: return run(std::integral_constant<int, kRowsBf16>{});
    case kRowsFp8: return run(std::integral_constant<int, kRowsFp8>{});
    default: return run(std::integral_constant<int, kRowsInt4>{});
  }
}

}  // namespace losa
