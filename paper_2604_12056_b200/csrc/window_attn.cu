// Attention of new tokens over the paged cache with a sliding window and first tokens that stay visible: losa_window_attn.
//
// Rows (token, head of a KV head) are taken in tiles; a tile reads the groups of keys that any of its rows sees.  All
// (tile, KV head, group) form one list, cut into equal shares, one per CTA, so prompts, blocks and single tokens of any lengths fill
// the GPU alike.  A tile that several CTAs share leaves records (reference, sum, un-normalised output per row) that a kernel of
// its own merges by log-sum-exp.  A first small kernel writes the list's tiles and where each share begins.
#include <cuda.h>

#include <algorithm>
#include <cstring>
#include <type_traits>

#include "cache_view.cuh"
#include "kernels.h"
#include "tcgen05_ops.cuh"

namespace losa {
namespace {

// Where a share begins: tile, KV head, position in the (tile, KV head): `pad` positions that stand for no group (entering a tile
// costs a CTA as much time), then its groups.
struct Share { int tile, kh, at, unused; };
struct Tile { int s, j, groups, unused; };           // rows j * R .. of sequence s
struct Plan {
  int* head;                                         // [4]: shares, tiles
  Sequence* seqs;                                    // [N]
  Share* shares;                                     // [n_ctas + 1]
  Tile* tiles;
};

struct WindowParams {
  CacheParams c;
  QueryParams q;
  Plan plan;
  void* out;                                         // [T, H_q, d] dtype
  float* lse;                                        // or null
  float* partials;                                   // [n_ctas][2][R * (d + 2)]
  int32_t* status;
  long long max_tiles;                               // room of the plan
  int n_ctas, pad, least;
  float scale_log2;                                  // sm_scale * log2(e)
  float sm_scale;
  long long wait_cycles;
};

// The groups (of GT keys) that a tile's rows see: the first `first`, then those from `from` on, up to `end` keys.
struct Reach { int first, from, groups, end, lo; };
template <int GT>
__device__ __forceinline__ Reach reach_of(const WindowParams& p, const Sequence& x, int row0, int rows) {
  const int t0 = row0 / p.c.G, t1 = min(x.count - 1, (row0 + rows - 1) / p.c.G);
  Reach r;
  r.end = keys_of(p.q, x, x.start + t1).x;
  r.lo = keys_of(p.q, x, x.start + t0).y;
  const int sinks = r.lo > 0 ? min(p.q.sinks, r.end) : 0;
  r.first = (sinks + GT - 1) / GT;
  r.from = max(r.first, r.lo / GT);
  r.groups = r.first + max(0, (r.end + GT - 1) / GT - r.from);
  return r;
}
template <int GT> __device__ __forceinline__ int group_key(const Reach& r, int i) { return (i < r.first ? i : r.from + i - r.first) * GT; }

// ===================================================================== the list of work
constexpr int kPlanThreads = 1024;
template <int R, int GT>
__global__ void __launch_bounds__(kPlanThreads) window_plan_kernel(const __grid_constant__ WindowParams p) {
  __shared__ int before[kPlanThreads + 1];           // tiles before a sequence
  __shared__ long long sums[kPlanThreads / 32 + 1];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  auto scan = [&](long long v) {                     // exclusive; the total is left in sums[32]
    long long inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long t = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += t;
    }
    if (lane == 31) sums[warp] = inc;
    __syncthreads();
    if (warp == 0) {
      const long long w = sums[lane];
      long long winc = w;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long t = __shfl_up_sync(0xffffffffu, winc, o);
        if (lane >= o) winc += t;
      }
      sums[lane] = winc - w;
      if (lane == 31) sums[32] = winc;
    }
    __syncthreads();
    const long long out = sums[warp] + inc - v;
    return out;
  };
  grid_dep_trigger();
  grid_dep_wait();
  Sequence x = {0, 0, 0, 0};
  if (tid < p.c.N) {
    x = sequence_of(p.c, p.q, tid, p.status);
    p.plan.seqs[tid] = x;
  }
  const int mine = static_cast<int>((static_cast<long long>(x.count) * p.c.G + R - 1) / R);
  const long long tiles_before = scan(mine);
  const bool fits = sums[32] <= p.max_tiles;         // (sequences that overlap in `cu` can make more tiles than the tokens have)
  if (!fits && tid == 0) set_status(p.status, LOSA_ERR_BOUNDS);
  before[tid] = fits ? static_cast<int>(tiles_before) : 0;
  const int X = fits ? static_cast<int>(sums[32]) : 0;
  if (tid == 0) before[kPlanThreads] = X;
  __syncthreads();
  // every thread: a run of tiles
  const int per = (X + kPlanThreads - 1) / kPlanThreads, a = min(X, tid * per), z = min(X, a + per);
  int s = 0;
  if (a < z) {
    int b = kPlanThreads;                            // before[s] <= a < before[b]
    while (b - s > 1) {
      const int m = (s + b) >> 1;
      if (before[m] <= a) s = m; else b = m;
    }
  }
  long long sum = 0;
  Sequence y = {0, 0, 0, 0};
  int have = -1, at = s;
  for (int t = a; t < z; ++t) {
    while (before[at + 1] <= t) ++at;
    if (at != have) { y = p.plan.seqs[at]; have = at; }
    const int j = t - before[at];
    const int n = reach_of<GT>(p, y, j * R, R).groups;
    p.plan.tiles[t] = {at, j, n, 0};
    sum += p.pad + n;
  }
  __syncthreads();
  long long pos = scan(sum) * p.c.Hkv;
  const long long total = sums[32] * p.c.Hkv;
  const int n = static_cast<int>(max(1ll, min(static_cast<long long>(p.n_ctas), total / p.least)));
  auto lo = [&](long long b) { return cta_lo(total, static_cast<int>(b), n); };
  for (int t = a; t < z; ++t) {
    const int length = p.pad + p.plan.tiles[t].groups;
    const long long end = pos + static_cast<long long>(length) * p.c.Hkv;
    long long b = pos * n / total;                   // shares that begin in this tile
    while (b > 0 && lo(b - 1) >= pos) --b;
    while (b < n && lo(b) < pos) ++b;
    for (; b < n && lo(b) < end; ++b) {
      const int off = static_cast<int>(lo(b) - pos);
      p.plan.shares[b] = {t, off / length, off % length, 0};
    }
    pos = end;
  }
  if (tid == 0) {
    p.plan.head[0] = X > 0 ? n : 0;
    p.plan.head[1] = X;
    p.plan.shares[X > 0 ? n : 0] = {X, 0, 0, 0};
  }
}

// A CTA's part of one (tile, KV head).
struct Piece {
  int tile, kh, s, row0, rows;                       // rows: that exist
  int first, last, groups;                           // groups first .. last - 1 of `groups`
  Sequence x;
  Reach r;
  bool any;                                          // false: the share is at its end
  __device__ __forceinline__ bool whole() const { return first == 0 && last == groups; }
};
template <int R, int GT>
struct Walk {
  const WindowParams& p;
  Share at, end;                                     // next position, the share's end
  __device__ __forceinline__ Walk(const WindowParams& params, int b) : p(params) {
    const int n = p.plan.head[0];
    if (b >= n) {
      at = end = {0, 0, 0, 0};
      return;
    }
    at = p.plan.shares[b];
    end = p.plan.shares[b + 1];
  }
  __device__ __forceinline__ bool done() const { return at.tile == end.tile && at.kh == end.kh && at.at == end.at; }
  // the next piece that has groups, or that stands for a tile without any (whose results are those of no key)
  __device__ __forceinline__ Piece next() {
    Piece w;
    w.any = false;
    while (!done()) {
      const Tile t = p.plan.tiles[at.tile];
      const int length = p.pad + t.groups;
      const bool cut = at.tile == end.tile && at.kh == end.kh;
      const int from = at.at, to = cut ? end.at : length;
      w.tile = at.tile;
      w.kh = at.kh;
      w.s = t.s;
      w.groups = t.groups;
      w.first = max(0, from - p.pad);
      w.last = max(0, to - p.pad);
      const bool begins = from == 0;
      if (cut) at = end;
      else if (at.kh + 1 < p.c.Hkv) at = {at.tile, at.kh + 1, 0, 0};
      else at = {at.tile + 1, 0, 0, 0};
      if (w.last > w.first || (t.groups == 0 && begins)) {
        w.x = p.plan.seqs[t.s];
        w.row0 = t.j * R;
        w.rows = min(R, w.x.count * p.c.G - w.row0);
        w.r = reach_of<GT>(p, w.x, w.row0, R);
        w.any = true;
        break;
      }
    }
    return w;
  }
};
// row of q / out (in units of d elements) of row r of a piece
__device__ __forceinline__ long long token_head(const WindowParams& p, const Piece& w, int r) {
  const int row = w.row0 + r, t = row / p.c.G;
  return (static_cast<long long>(w.x.cu) + t) * (p.c.Hkv * p.c.G) + w.kh * p.c.G + (row - t * p.c.G);
}
// the record of a piece: the first piece of a tile in its CTA's second place, the others (their CTA's first piece) in the first
template <int R, int D>
__device__ __forceinline__ float* record_of(const WindowParams& p, int b, bool first) {
  return p.partials + (static_cast<size_t>(b) * 2 + (first ? 1 : 0)) * (R * (D + 2));
}

// Tiles that several CTAs share: a warp per row merges their records, in CTA order.  Block (b, .) looks after the tile that share b
// begins in, if it is the first share to begin among that tile's groups.
constexpr int kMergeWarps = 8;
template <int R, int D, typename T>
__global__ void __launch_bounds__(kMergeWarps * 32) window_merge_kernel(const __grid_constant__ WindowParams p) {
  grid_dep_wait();
  const int b = blockIdx.x + 1, lane = threadIdx.x & 31, r = blockIdx.y * kMergeWarps + (threadIdx.x >> 5);
  const int n = p.plan.head[0];
  if (b >= n) return;
  const Share x = p.plan.shares[b], prev = p.plan.shares[b - 1];
  if (x.at <= p.pad) return;                         // cut before its first group: it is whole in this CTA, or the next one's
  if (prev.tile == x.tile && prev.kh == x.kh && prev.at > p.pad) return;
  const Tile t = p.plan.tiles[x.tile];
  Piece w;
  w.x = p.plan.seqs[t.s];
  w.kh = x.kh;
  w.row0 = t.j * R;
  if (r >= w.x.count * p.c.G - w.row0) return;
  int last = b;
  while (last + 1 < n) {
    const Share y = p.plan.shares[last + 1];
    if (y.tile != x.tile || y.kh != x.kh) break;
    ++last;
  }
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
  const long long row = token_head(p, w, r);
  const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
  for (int c = 0; c < C; ++c) static_cast<T*>(p.out)[row * D + c * 32 + lane] = from_f32<T>(acc[c] * inv);
  if (lane == 0 && p.lse) p.lse[row] = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
}

#include "window_attn_f32.cuh"
#include "window_attn_tc.cuh"

// ===================================================================== host side
template <int R, int GT, int D, typename Launch, typename T>
int32_t with_plan(losa_ctx* c, WindowParams& p, cudaStream_t st, T, Launch&& main_kernel) {
  char* at = c->ws + c->lay.plan;
  p.plan.head = reinterpret_cast<int*>(at);
  p.plan.seqs = reinterpret_cast<Sequence*>(at + 256);
  p.plan.shares = reinterpret_cast<Share*>(at + 256 + sizeof(Sequence) * c->shape.batch);
  p.plan.tiles = reinterpret_cast<Tile*>(p.plan.shares + p.n_ctas + 1);
  p.max_tiles = c->lay.plan_tiles;
  p.partials = reinterpret_cast<float*>(c->ws + c->lay.scores);
  launch_k(window_plan_kernel<R, GT>, 1, kPlanThreads, 0, st, p);
  int32_t rc = after_launch(c);
  if (rc == LOSA_OK) rc = main_kernel();
  if (rc != LOSA_OK) return rc;
  launch_k(window_merge_kernel<R, D, T>, dim3(p.n_ctas, R / kMergeWarps), kMergeWarps * 32, 0, st, p);
  return after_launch(c);
}

template <int FMT, int D>
int32_t launch_rows(losa_ctx* c, WindowParams& p, cudaStream_t st) {
  p.n_ctas = 2 * c->n_sms;
  p.pad = 1;
  p.least = 2;
  using T = typename RowFormat<FMT>::Query;
  return with_plan<kWinRows, kWinKeys, D>(c, p, st, T{}, [&]() -> int32_t {
    auto kernel = window_f32_kernel<FMT, D>;
    LOSA_CUDA_TRY(c, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, win_smem<D>()));
    launch_k(kernel, p.n_ctas, kWinThreads, win_smem<D>(), st, p);
    return after_launch(c);
  });
}

template <int D, int GP>
int32_t launch_tc(losa_ctx* c, WindowParams& p, const losa_kv_t* kv, cudaStream_t st) {
  const int32_t rc = pool_tensor_maps(c, kv);
  if (rc != LOSA_OK) return rc;
  CUtensorMap mk, mv;
  memcpy(&mk, c->tmap_k, sizeof(mk));
  memcpy(&mv, c->tmap_v, sizeof(mv));
  p.n_ctas = c->n_sms;
  p.pad = 2;
  p.least = 3;
  auto kernel = window_tc_kernel<D, GP>;
  if (!(c->window_attr_set & 1)) {
    static_assert(wt_smem<D>() <= 232448, "shared memory");
    LOSA_CUDA_TRY(c, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, wt_smem<D>()));
    // the kernel moves registers between its warps: a build that is launched with fewer than it deals out would wait for ever
    cudaFuncAttributes fa;
    LOSA_CUDA_TRY(c, cudaFuncGetAttributes(&fa, kernel));
    if (fa.numRegs < kWtLaunchRegs) return LOSA_ERR_UNSUPPORTED;
    c->window_attr_set |= 1;
  }
  return with_plan<kWtRows, kWtKeys, D>(c, p, st, __nv_bfloat16{}, [&]() -> int32_t {
    launch_k(kernel, p.n_ctas, kWtWarps * 32, wt_smem<D>(), st, mk, mv, p);
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
  p.sm_scale = c->shape.sm_scale;
  p.scale_log2 = c->shape.sm_scale * kLog2e;
  p.wait_cycles = c->wait_cycles > 0 ? c->wait_cycles : kWaitCycles;
  auto run = [&](auto f) {
    constexpr int FMT = decltype(f)::value;
    return c->shape.head_dim == 128 ? launch_rows<FMT, 128>(c, p, st) : launch_rows<FMT, 64>(c, p, st);
  };
  switch (row_format(c, kv)) {
    case kRowsF32: return run(std::integral_constant<int, kRowsF32>{});
    case kRowsBf16: {
      auto with_page = [&](auto d) {
        constexpr int D = decltype(d)::value;
        return c->shape.page_size == 16 ? launch_tc<D, 16>(c, p, kv, st) : c->shape.page_size == 32 ? launch_tc<D, 32>(c, p, kv, st) : launch_tc<D, 64>(c, p, kv, st);
      };
      return c->shape.head_dim == 128 ? with_page(std::integral_constant<int, 128>{}) : with_page(std::integral_constant<int, 64>{});
    }
    case kRowsFp8: return run(std::integral_constant<int, kRowsFp8>{});
    default: return run(std::integral_constant<int, kRowsInt4>{});
  }
}

}  // namespace losa
