// Attention of new tokens over the paged cache with a sliding window and first tokens that stay visible: losa_window_attn.
//
// Rows (token, head of a KV head) are taken in tiles; a tile reads the groups of keys that any of its rows sees.  All
// (tile, KV head, group) form one list, cut into equal shares, so prompts, blocks and single tokens of any lengths fill
// the GPU alike.  A tile that several CTAs share leaves records (reference, sum, un-normalised output per row), joined by log-sum-exp.
#include <algorithm>
#include <cstring>
#include <type_traits>

#include "kernels.h"
#include "tc_cache_ops.cuh"
#include "work_list.cuh"

namespace losa {
namespace {

struct WindowParams : ListParams {
  void* out;                                         // [T, H_q, d] dtype
  float* lse;                                        // or null
  float* partials;                                   // [n_ctas][2][R * (d + 2)]
  float scale_log2;                                  // sm_scale * log2(e)
};

// The groups (of GT keys) that tokens t0 .. t0 + n - 1 of a sequence see: the first `first`, then those from `from` on, up to `end` keys.
struct Reach { int first, from, groups, end, lo; };
template <int GT>
__device__ __forceinline__ Reach reach_of(const ListParams& p, const Sequence& x, int t0, int n) {
  Reach r;
  r.end = keys_of(p.q, x, x.start + t0 + n - 1).x;
  r.lo = keys_of(p.q, x, x.start + t0).y;
  const int sinks = r.lo > 0 ? min(p.q.sinks, r.end) : 0;
  r.first = (sinks + GT - 1) / GT;
  r.from = max(r.first, r.lo / GT);
  r.groups = r.first + max(0, (r.end + GT - 1) / GT - r.from);
  return r;
}
template <int GT> __device__ __forceinline__ int group_key(const Reach& r, int i) { return (i < r.first ? i : r.from + i - r.first) * GT; }

// A tile's rows: SETS sets of SR, each of as many whole tokens as fit.
template <int SR, int SETS, int GT>
struct RowTiles {
  static constexpr int rows = SR * SETS, set_rows = SR;
  static __device__ __forceinline__ int per_set(const ListParams& p) { return SR / p.c.G; }
  static __device__ __forceinline__ int tiles(const ListParams& p, const Sequence& x) {
    const int n = SETS * per_set(p);
    return (x.count + n - 1) / n;
  }
  static __device__ __forceinline__ int groups(const ListParams& p, const Sequence& x, int j) {
    const int n = SETS * per_set(p);
    return reach_of<GT>(p, x, j * n, min(n, x.count - j * n)).groups;
  }
};
struct Piece : Part {
  int token0, tokens;                                // of the sequence's tokens
  Reach r;
};
template <class Tiles, int GT>
__device__ __forceinline__ Piece next_piece(Walk& walk) {
  Piece w;
  static_cast<Part&>(w) = walk.next();
  if (w.any) {
    const int n = Tiles::rows / Tiles::set_rows * Tiles::per_set(walk.p);
    w.token0 = w.j * n;
    w.tokens = min(n, w.x.count - w.token0);
    w.r = reach_of<GT>(walk.p, w.x, w.token0, w.tokens);
  }
  return w;
}
// Row rr of a set: its token in the tile (-1: there is none), and its row of q / out in units of d elements.
template <int SR>
__device__ __forceinline__ int row_token(const ListParams& p, int tokens, int set, int rr) {
  const int per = SR / p.c.G, t = rr / p.c.G;
  return t < per && set * per + t < tokens ? set * per + t : -1;
}
__device__ __forceinline__ long long token_head(const ListParams& p, const Sequence& x, int token, int kh, int rr) {
  return (static_cast<long long>(x.cu) + token) * (p.c.Hkv * p.c.G) + kh * p.c.G + rr % p.c.G;
}
template <int R, int D>
__device__ __forceinline__ float* record_of(const WindowParams& p, int b, bool first) { return p.partials + record_at(b, first) * (R * (D + 2)); }

// Tiles that several CTAs share: a warp per row joins their records.  Blocks (b, .): the tile that share b begins in.
constexpr int kMergeWarps = 8;
template <class Tiles, int D, typename T>
__global__ void __launch_bounds__(kMergeWarps * 32) window_merge_kernel(const __grid_constant__ WindowParams p) {
  grid_dep_wait();
  const int b = blockIdx.x + 1, lane = threadIdx.x & 31, r = blockIdx.y * kMergeWarps + (threadIdx.x >> 5);
  Share x;
  const int last = records_from(p, b, x);
  if (last < b) return;
  constexpr int R = Tiles::rows, SR = Tiles::set_rows;
  const int per = R / SR * Tiles::per_set(p), token = row_token<SR>(p, x.t.x.count - x.t.j * per, r / SR, r % SR);
  if (token < 0) return;
  constexpr int C = D / 32, kBatch = 4;
  float acc[C], M = -INFINITY, L = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c) acc[c] = 0.f;
  for (int i0 = b - 1; i0 <= last; i0 += kBatch) {
    float m[kBatch], l[kBatch], o[kBatch][C];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c) o[i][c] = 0.f;
      if (i0 + i <= last) {
        const float* at = record_of<R, D>(p, i0 + i, i0 + i == b - 1);
        m[i] = at[r];
        l[i] = at[R + r];
#pragma unroll
        for (int c = 0; c < C; ++c) o[i][c] = at[2 * R + r * D + c * 32 + lane];
      }
    }
    float top = M;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) top = fmaxf(top, m[i]);
    if (top == -INFINITY) {                          // nothing seen so far: sums are zero, or no number, which stays visible
#pragma unroll
      for (int i = 0; i < kBatch; ++i) L += l[i];
      continue;
    }
    const float keep = exp2f(M - top);
    L *= keep;
#pragma unroll
    for (int c = 0; c < C; ++c) acc[c] *= keep;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const float f = exp2f(m[i] - top);
      L = fmaf(l[i], f, L);
#pragma unroll
      for (int c = 0; c < C; ++c) acc[c] = fmaf(o[i][c], f, acc[c]);
    }
    M = top;
  }
  const long long row = token_head(p, x.t.x, x.t.j * per + token, x.kh, r % SR);
  const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
  for (int c = 0; c < C; ++c) static_cast<T*>(p.out)[row * D + c * 32 + lane] = from_f32<T>(acc[c] * inv);
  if (lane == 0 && p.lse) p.lse[row] = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
}

#include "window_attn_f32.cuh"
#include "window_attn_tc.cuh"

// ===================================================================== host side
template <class Tiles, int D, typename Launch, typename T>
int32_t with_plan(losa_ctx* c, WindowParams& p, cudaStream_t st, T, Launch&& main_kernel) {
  place_plan(c, p);
  p.partials = reinterpret_cast<float*>(c->ws + c->lay.scores);
  launch_k(list_plan_kernel<Tiles>, 1, kPlanThreads, 0, st, static_cast<const ListParams&>(p));
  int32_t rc = after_launch(c);
  if (rc == LOSA_OK) rc = main_kernel();
  if (rc != LOSA_OK) return rc;
  launch_k(window_merge_kernel<Tiles, D, T>, dim3(p.n_ctas, Tiles::rows / kMergeWarps), kMergeWarps * 32, 0, st, p);
  return after_launch(c);
}

template <int D>
int32_t launch_f32(losa_ctx* c, WindowParams& p, cudaStream_t st) {
  p.n_ctas = 2 * c->n_sms;
  p.pad = 1;
  p.least = 2;
  auto kernel = window_f32_kernel<D>;
  constexpr int bit = 1 << kRowsF32;
  if (!(c->window_attr_set & bit)) {
    LOSA_CUDA_TRY(c, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, win_smem<D>()));
    c->window_attr_set |= bit;
  }
  return with_plan<WinTiles, D>(c, p, st, float{}, [&]() -> int32_t {
    launch_k(kernel, p.n_ctas, kWinThreads, win_smem<D>(), st, p);
    return after_launch(c);
  });
}

template <int FMT, int D, int GP>
int32_t launch_tc(losa_ctx* c, WindowParams& p, const losa_kv_t* kv, cudaStream_t st) {
  using Tc = WindowTc<FMT, D, GP>;
  const int32_t rc = Tc::quant ? raw_tensor_maps(c, kv) : pool_tensor_maps(c, kv);
  if (rc != LOSA_OK) return rc;
  CUtensorMap mk, mv, mq;
  memcpy(&mk, Tc::quant ? c->tmap_raw[0] : c->tmap_k, sizeof(mk));
  memcpy(&mv, Tc::quant ? c->tmap_raw[1] : c->tmap_v, sizeof(mv));
  if constexpr (!Tc::quant) {
    const int32_t rq = query_tensor_map(c, p.q.q, p.q.stride, p.q.T, 128 / p.c.G, &mq);
    if (rq != LOSA_OK) return rq;
  } else {
    mq = mk;                                         // (not used)
  }
  p.n_ctas = c->n_sms;
  // Entering a tile costs a CTA as much as this many groups, or a little less where tiles are many.  2, 4, 5, 6 groups, us: blocks of 32 tokens over windows of 4,096
  // 57.3, 56.4, 54.3, 53.5, decoded tokens over FP8 caches 123, 118, 116, 118, over windows of 512 62.8, 63.7, 62.8, 63.5; ragged prompts with a window of 1,024 with 2 and 4 473, 480.
  p.pad = p.q.max_tokens <= 128 / p.c.G ? 5 : 2;
  p.least = p.pad + 1;
  auto kernel = window_tc_kernel<FMT, D, GP>;
  constexpr int bit = 1 << FMT;
  if (!(c->window_attr_set & bit)) {
    LOSA_CUDA_TRY(c, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Tc::smem));
    c->window_attr_set |= bit;
  }
  return with_plan<typename Tc::Tiles, D>(c, p, st, __nv_bfloat16{}, [&]() -> int32_t {
    launch_k(kernel, p.n_ctas, Tc::warps * 32, Tc::smem, st, mk, mv, mq, p);
    return after_launch(c);
  });
}

}  // namespace

int32_t launch_window_attn(losa_ctx* c, const losa_queries_t* q, const losa_kv_t* kv, void* out, float* lse_opt, cudaStream_t st) {
  WindowParams p = {};
  p.c = cache_params(c, kv);
  p.q = query_params(q);
  p.out = out;
  p.lse = lse_opt;
  p.status = status_ptr(c);
  p.scale_log2 = c->shape.sm_scale * kLog2e;
  set_bounds(c, p);
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
