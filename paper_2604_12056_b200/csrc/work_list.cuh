// Work over the paged cache as one list that is cut into equal shares, one per CTA: the windowed attention's (tiles of query rows, the groups
// of keys that they see) and the keys' weights' (tiles of keys, the groups of query rows that see them).
//
// A tile of a sequence stands for all its KV heads, one after the other in the list; each (tile, KV head) has `pad` positions that stand for no
// group (entering it costs a CTA as much time), then its groups.  A kernel of one CTA writes the tiles and where each share begins.  A
// (tile, KV head) that several CTAs share leaves a record per CTA, which a last kernel joins in CTA order.
#pragma once
#include "cache_view.cuh"

namespace losa {

struct alignas(16) Tile { int s, j, groups, unused; Sequence x; };      // tile j of sequence s
struct alignas(16) Share { int tile, kh, at, unused; Tile t; };         // where a share begins: position `at` of (tile, KV head)
struct Plan {
  int* head;                                         // shares
  Share* shares;                                     // [n_ctas + 1]
  Tile* tiles;
};
struct ListParams {
  CacheParams c;
  QueryParams q;
  Plan plan;
  long long max_tiles;                               // room of the plan
  int n_ctas, pad, least;                            // least: positions below which a share is not cut
  float keep;                                        // weights only
  int32_t* status;
  long long wait_cycles;
  int copies;                                        // groups of keys or values after which the warps that copy them give up
};

// Ops: static int tiles(p, sequence); static int groups(p, sequence, j).
constexpr int kPlanThreads = 1024;
template <class Ops>
__global__ void __launch_bounds__(kPlanThreads) list_plan_kernel(const __grid_constant__ ListParams p) {
  __shared__ int before[kPlanThreads + 1];           // tiles before a sequence
  __shared__ Sequence seqs[kPlanThreads];
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
    return sums[warp] + inc - v;
  };
  grid_dep_trigger();
  grid_dep_wait();
  Sequence x = {0, 0, 0, 0};
  int mine = 0;
  if (tid < p.c.N) {
    x = sequence_of(p.c, p.q, tid, p.status);
    mine = Ops::tiles(p, x);
  }
  seqs[tid] = x;
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
  int at = s;
  for (int t = a; t < z; ++t) {
    while (before[at + 1] <= t) ++at;
    const Sequence y = seqs[at];
    const int j = t - before[at], n = Ops::groups(p, y, j);
    p.plan.tiles[t] = {at, j, n, 0, y};
    sum += p.pad + n;
  }
  __syncthreads();
  long long pos = scan(sum) * p.c.Hkv;
  const long long total = sums[32] * p.c.Hkv;
  const int n = static_cast<int>(max(1ll, min(static_cast<long long>(p.n_ctas), total / p.least)));
  auto lo = [&](long long b) { return cta_lo(total, static_cast<int>(b), n); };
  for (int t = a; t < z; ++t) {
    const Tile tile = p.plan.tiles[t];
    const int length = p.pad + tile.groups;
    const long long end = pos + static_cast<long long>(length) * p.c.Hkv;
    long long b = pos * n / total;                   // shares that begin in this tile
    while (b > 0 && lo(b - 1) >= pos) --b;
    while (b < n && lo(b) < pos) ++b;
    for (; b < n && lo(b) < end; ++b) {
      const int off = static_cast<int>(lo(b) - pos);
      p.plan.shares[b] = {t, off / length, off % length, 0, tile};
    }
    pos = end;
  }
  if (tid == 0) {
    p.plan.head[0] = X > 0 ? n : 0;
    p.plan.shares[X > 0 ? n : 0] = {X, 0, 0, 0, {0, 0, 0, 0, {0, 0, 0, 0}}};
  }
}

// A CTA's part of one (tile, KV head).
struct Part {
  int tile, kh, s, j;
  int first, last, groups;                           // groups first .. last - 1 of `groups`
  Sequence x;
  bool any;                                          // false: the share is at its end
  __device__ __forceinline__ bool whole() const { return first == 0 && last == groups; }
};
struct Walk {
  const ListParams& p;
  int tile, kh, at, end_tile, end_kh, end_at;        // next position, the share's end
  Tile t;                                            // the tile that `tile` names
  __device__ __forceinline__ Walk(const ListParams& params, int b) : p(params) {
    if (b >= p.plan.head[0]) {
      tile = kh = at = end_tile = end_kh = end_at = 0;
      return;
    }
    const Share x = p.plan.shares[b];
    tile = x.tile;
    kh = x.kh;
    at = x.at;
    t = x.t;
    const Share y = p.plan.shares[b + 1];
    end_tile = y.tile;
    end_kh = y.kh;
    end_at = y.at;
  }
  // the next part that has groups, or that stands for a tile without any
  __device__ __forceinline__ Part next() {
    Part w;
    w.any = false;
    while (!(tile == end_tile && kh == end_kh && at == end_at)) {
      const int length = p.pad + t.groups, from = at;
      const bool cut = tile == end_tile && kh == end_kh;
      const int to = cut ? end_at : length;
      w.tile = tile;
      w.kh = kh;
      w.s = t.s;
      w.j = t.j;
      w.x = t.x;
      w.groups = t.groups;
      w.first = max(0, from - p.pad);
      w.last = max(0, to - p.pad);
      if (cut) {
        at = end_at;
      } else {
        at = 0;
        if (++kh == p.c.Hkv) {
          kh = 0;
          ++tile;
          if (!(tile == end_tile && end_kh == 0 && end_at == 0)) t = p.plan.tiles[tile];
        }
      }
      if (w.last > w.first || (w.groups == 0 && from == 0)) {
        w.any = true;
        break;
      }
    }
    return w;
  }
};

// Shares b - 1 .. `last` leave records of the (tile, KV head) that share b begins in, if share b is the first to begin among its groups; else last < b.
__device__ __forceinline__ int records_from(const ListParams& p, int b, Share& x) {
  const int n = p.plan.head[0];
  if (b >= n) return 0;
  x = p.plan.shares[b];
  if (x.at <= p.pad) return 0;                       // cut before its first group: it is whole in this CTA, or the next one's
  const int tile = p.plan.shares[b - 1].tile, kh = p.plan.shares[b - 1].kh, at = p.plan.shares[b - 1].at;
  if (tile == x.tile && kh == x.kh && at > p.pad) return 0;
  int last = b;
  while (last + 1 < n && p.plan.shares[last + 1].tile == x.tile && p.plan.shares[last + 1].kh == x.kh) ++last;
  return last;
}
// Where a record lies, in records: the first part of a tile in its CTA's second place, the others (their CTA's first part) in the first.
__device__ __forceinline__ size_t record_at(int b, bool first) { return static_cast<size_t>(b) * 2 + (first ? 1 : 0); }

// The bound of the waits.  One of n cycles that is shorter than a look at a barrier takes holds for none; the warps that copy pages give up before their n-th group
// instead, and the others with them: the way out is taken with copies and products in flight, whatever the hardware's speed (a look may put its warp to sleep for
// longer than a short bound).
inline void set_bounds(const losa_ctx* c, ListParams& p) {
  const bool few = c->wait_cycles > 0 && c->wait_cycles < kLookCycles;
  p.wait_cycles = c->wait_cycles > 0 && !few ? c->wait_cycles : kWaitCycles;
  p.copies = few ? static_cast<int>(c->wait_cycles) - 1 : 0x7fffffff;
}

inline void place_plan(const losa_ctx* c, ListParams& p) {
  char* at = c->ws + c->lay.plan;
  p.plan.head = reinterpret_cast<int*>(at);
  p.plan.shares = reinterpret_cast<Share*>(at + 256);
  p.plan.tiles = reinterpret_cast<Tile*>(p.plan.shares + p.n_ctas + 1);
  p.max_tiles = c->lay.plan_tiles;
}

}  // namespace losa
