// Eviction from the paged cache by accumulated weight: losa_kv_evict.
//
// Two kernels.  The first chooses, a CTA per (sequence, KV head): the budget's smallest weight by digits of the weights' bits, then
// the places that stay, in order.  The second moves rows towards the front, in place, a CTA per (page that stays, KV head): a row
// never moves backwards, so what a page is overwritten with is read from that page or later ones, and the rows that stood in
// it are wanted by that page or earlier ones.  A CTA reads its page's rows into registers, says so, waits until all earlier
// pages of its head have said so, and writes.  CTAs take pages in the order in which they start, so those that are waited for run.
// In place, read once and written once: a copy through a second buffer would double the traffic and need the room.  Eight sequences of up to 16,384 tokens
// cut to 4,096: 81 us, 22 for choosing (64 CTAs, four passes over 16K weights in shared memory each) and 57 for moving 201 MB (3.5 TB/s: a chain
// of ticket, list, page table, rows and flags per 16 KB).  With a fence per thread instead of one release after the barrier moving took 63 us; twelve CTAs per SM spill
// and take 89.  One sequence of 8,201 FP8 tokens cut to 2,048: 19 us, latency.  A page looks at the flags of all pages before it, though at most two want its rows, so that
// looks grow with the square of the pages: 60,001 tokens of 8 heads cut to 59,000 take 335 us in pages of 16 tokens, 280 in pages of 32 or 64.
#include <algorithm>
#include <type_traits>

#include "cache_view.cuh"
#include "kernels.h"

namespace losa {
namespace {

struct EvictParams {
  CacheParams c;
  uint8_t *k_pages, *v_pages;
  void *k_scale, *v_scale, *kmin, *kmax;
  float* weights;
  const int32_t *length, *budget;
  int32_t *kept, *kv_len;
  int kept_stride, sinks, recent, pages;             // pages: of the largest budget
  int32_t* goes;                                     // [N * H_kv] tokens that stay, -1: the sequence is left as it is
  uint32_t* read;                                    // [N * H_kv][pages] a page's rows have been read
  uint32_t* ticket;
  int32_t* status;
  long long wait_cycles;
};

// ===================================================================== choosing
constexpr int kChooseThreads = 1024, kDigits = 2048, kChooseHeld = 49152;      // weights held in shared memory
// Weights in order as unsigned numbers: NaN above everything, -0 as +0.
__device__ __forceinline__ uint32_t weight_order(float w) {
  if (w != w) return 0xffffffffu;
  const uint32_t b = __float_as_uint(w + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__global__ void __launch_bounds__(kChooseThreads, 1) evict_choose_kernel(const __grid_constant__ EvictParams p) {
  extern __shared__ uint32_t held[];
  __shared__ uint32_t hist[kDigits];
  __shared__ uint32_t sums[33];
  __shared__ uint32_t found[2];                      // digit, what is still wanted among its equals
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  grid_dep_trigger();
  grid_dep_wait();
  const int sk = blockIdx.x, s = sk / p.c.Hkv, kh = sk - s * p.c.Hkv;
  const int L = p.length[s], b = p.budget[s];
  bool bad = L < 0 || L > static_cast<long long>(p.c.Pmax) * p.c.g || (b >= 0 && b < L && b > p.kept_stride);
  const bool stays = !bad && (b < 0 || b >= L);
  if (!bad && !stays) {                              // every page of the sequence has to be one of the pool
    int miss = 0;
    for (int i = tid; i < (L + p.c.g - 1) / p.c.g; i += kChooseThreads) {
      const int at = p.c.page_table[static_cast<size_t>(s) * p.c.Pmax + i];
      miss |= at < 0 || at >= p.c.n_phys;
    }
    bad = __syncthreads_or(miss) != 0;
  }
  if (bad && tid == 0) set_status(p.status, LOSA_ERR_BOUNDS);
  if (bad || stays) {
    if (tid == 0) p.goes[sk] = -1;
    return;
  }
  for (int i = tid; i < p.pages; i += kChooseThreads) p.read[static_cast<size_t>(sk) * p.pages + i] = 0u;
  if (tid == 0) {
    p.goes[sk] = b;
    if (kh == 0) p.kv_len[s] = b;
  }
  const int first = min(p.sinks, b), tail = L - min(p.recent, b - first);      // candidates: first .. tail - 1
  uint32_t want = b - first - (L - tail);
  const bool in_smem = L <= kChooseHeld;
  const int g_log = __ffs(p.c.g) - 1;
  auto from_cache = [&](int j) {
    const int page = p.c.page_table[static_cast<size_t>(s) * p.c.Pmax + (j >> g_log)];
    return weight_order(p.weights[((static_cast<size_t>(page) * p.c.Hkv + kh) << g_log) + (j & (p.c.g - 1))]);
  };
  if (in_smem) {
#pragma unroll 8
    for (int j = tid; j < L; j += kChooseThreads) held[j] = from_cache(j);
    __syncthreads();
  }
  auto order = [&](int j) { return in_smem ? held[j] : from_cache(j); };
  // the want-th largest of the candidates, digit by digit
  uint32_t prefix = 0, mask = 0;
  if (want > 0) {
    constexpr int shifts[3] = {21, 10, 0}, bits[3] = {11, 11, 10};
#pragma unroll
    for (int d = 0; d < 3; ++d) {
      for (int i = tid; i < kDigits; i += kChooseThreads) hist[i] = 0u;
      __syncthreads();
      for (int j = first + tid; j < tail; j += kChooseThreads) {
        const uint32_t u = order(j);
        if ((u & mask) == prefix) atomicAdd(&hist[(u >> shifts[d]) & ((1u << bits[d]) - 1u)], 1u);
      }
      __syncthreads();
      // thread i: the digits 2047 - 2 i and the one below; how many candidates have larger ones
      const uint32_t hi = hist[kDigits - 1 - 2 * tid], lo = hist[kDigits - 2 - 2 * tid];
      uint32_t inc = hi + lo;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
      }
      if (lane == 31) sums[warp] = inc;
      __syncthreads();
      if (warp == 0) {
        const uint32_t w = sums[lane];
        uint32_t winc = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t t = __shfl_up_sync(0xffffffffu, winc, o);
          if (lane >= o) winc += t;
        }
        sums[lane] = winc - w;
      }
      __syncthreads();
      const uint32_t above = sums[warp] + inc - hi - lo;
      if (above < want && above + hi >= want) { found[0] = kDigits - 1 - 2 * tid; found[1] = want - above; }
      if (above + hi < want && above + hi + lo >= want) { found[0] = kDigits - 2 - 2 * tid; found[1] = want - above - hi; }
      __syncthreads();
      prefix |= found[0] << shifts[d];
      mask |= ((1u << bits[d]) - 1u) << shifts[d];
      want = found[1];
      __syncthreads();
    }
  }
  // (want: how many of the candidates equal to the threshold stay, the first ones)
  const bool any = mask != 0;
  auto kind = [&](int j) {                           // 2: stays, 1: equal to the threshold, 0: goes
    if (j >= L) return 0;
    if (j < first || j >= tail) return 2;
    if (!any) return 0;
    const uint32_t u = order(j);
    return u > prefix ? 2 : u == prefix ? 1 : 0;
  };
  const int seg = ((L + kChooseThreads - 1) / kChooseThreads) * 32, j0 = warp * seg, j1 = min(L, j0 + seg);
  uint32_t more = 0, equal = 0;                      // of this warp's places
  for (int j = j0; j < j1; j += 32) {
    const int k = kind(j + lane);                    // (j1 is a segment's end or L)
    more += __popc(__ballot_sync(0xffffffffu, k == 2));
    equal += __popc(__ballot_sync(0xffffffffu, k == 1));
  }
  __syncthreads();
  if (lane == 0) { hist[warp] = more; hist[32 + warp] = equal; }
  __syncthreads();
  uint32_t more_before = 0, equal_before = 0;
  for (int w = 0; w < warp; ++w) { more_before += hist[w]; equal_before += hist[32 + w]; }
  int32_t* kept = p.kept + static_cast<size_t>(sk) * p.kept_stride;
  const uint32_t below = (1u << lane) - 1u;
  for (int j = j0; j < j1; j += 32) {
    const int k = kind(j + lane);
    const uint32_t is2 = __ballot_sync(0xffffffffu, k == 2), is1 = __ballot_sync(0xffffffffu, k == 1);
    const uint32_t e = equal_before + __popc(is1 & below), at = more_before + __popc(is2 & below) + min(e, want);
    if (k == 2 || (k == 1 && e < want)) kept[at] = j + lane;
    more_before += __popc(is2);
    equal_before += __popc(is1);
  }
}

// ===================================================================== moving
constexpr int kMoveThreads = 128;
__device__ __forceinline__ uint32_t load_acquire(const uint32_t* p) {
  uint32_t v;
  asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
template <int FMT> constexpr int piece_elems() { return 128 / RowFormat<FMT>::bits; }       // elements of 16 bytes
template <int FMT>
__device__ __forceinline__ void piece_values(const uint4& u, float scale, float (&v)[piece_elems<FMT>()]) {
  if constexpr (FMT == kRowsF32) {
    v[0] = __uint_as_float(u.x); v[1] = __uint_as_float(u.y); v[2] = __uint_as_float(u.z); v[3] = __uint_as_float(u.w);
  } else if constexpr (FMT == kRowsBf16) {
    load8(reinterpret_cast<const __nv_bfloat16*>(&u), v);
  } else if constexpr (FMT == kRowsFp8) {
    float a[8], b[8];
    fp8_decode8(make_uint2(u.x, u.y), a);
    fp8_decode8(make_uint2(u.z, u.w), b);
#pragma unroll
    for (int i = 0; i < 8; ++i) { v[i] = a[i] * scale; v[8 + i] = b[i] * scale; }
  } else {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a[8];
      int4_decode8(w[i], scale, a);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[i * 8 + k] = a[k];
    }
  }
}

template <int FMT, int D, int GP>
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const __grid_constant__ EvictParams p) {
  using T = typename RowFormat<FMT>::Query;
  constexpr int E = piece_elems<FMT>(), TPR = D / E, RPP = kMoveThreads / TPR, NP = (GP + RPP - 1) / RPP;
  __shared__ float lows[4][D], highs[4][D];
  __shared__ float amax[2][4];
  __shared__ uint32_t order;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, col = tid % TPR, row0 = tid / TPR;
  grid_dep_wait();
  if (tid == 0) order = atomicInc(p.ticket, gridDim.x - 1);
  __syncthreads();
  const int n_sk = p.c.N * p.c.Hkv, c = order / n_sk, sk = order - c * n_sk, s = sk / p.c.Hkv, kh = sk - s * p.c.Hkv;
  const int b = p.goes[sk];
  if (b < 0 || c * GP >= b) return;
  const int32_t* kept = p.kept + static_cast<size_t>(sk) * p.kept_stride;
  const int32_t* table = p.c.page_table + static_cast<size_t>(s) * p.c.Pmax;
  const int n = min(GP, b - c * GP);                 // rows of the page
  uint32_t* read = p.read + static_cast<size_t>(sk) * p.pages;
  uint4 k[NP], v[NP];
  float ks[NP], vs[NP];                              // scales of the quantised formats
  uint32_t kb[NP], vb[NP];                           // the 4-bit format's scale bytes
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int r = row0 + i * RPP;
    k[i] = v[i] = make_uint4(0u, 0u, 0u, 0u);
    ks[i] = vs[i] = 1.f;
    kb[i] = vb[i] = 0u;
    if (r < n) {
      const int src = kept[c * GP + r], page = table[src / GP], slot = src % GP;
      const int64_t at = page * p.c.stride_page + kh * p.c.stride_head + slot * p.c.stride_tok + col * 16;
      k[i] = *reinterpret_cast<const uint4*>(p.k_pages + at);
      v[i] = *reinterpret_cast<const uint4*>(p.v_pages + at);
      const size_t ph = static_cast<size_t>(page) * p.c.Hkv + kh;
      if constexpr (FMT == kRowsFp8) {
        ks[i] = static_cast<const float*>(p.k_scale)[ph];
        vs[i] = static_cast<const float*>(p.v_scale)[ph];
      }
      if constexpr (FMT == kRowsInt4) {
        kb[i] = static_cast<const uint8_t*>(p.k_scale)[(ph * GP + slot) * TPR + col];
        vb[i] = static_cast<const uint8_t*>(p.v_scale)[(ph * GP + slot) * TPR + col];
        ks[i] = int4_scale_value(kb[i]);
      }
    }
  }
  float w = 0.f;
  if (tid < n) {
    const int src = kept[c * GP + tid];
    w = p.weights[(static_cast<size_t>(table[src / GP]) * p.c.Hkv + kh) * GP + src % GP];
  }
  // The page's new scales come from all of its rows.
  float inv[2] = {1.f, 1.f}, now[2] = {1.f, 1.f};
  if constexpr (FMT == kRowsFp8) {
    float top[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      float x[E];
      piece_values<FMT>(k[i], ks[i], x);
#pragma unroll
      for (int e = 0; e < E; ++e) top[0] = fmaxf(top[0], fabsf(x[e]));
      piece_values<FMT>(v[i], vs[i], x);
#pragma unroll
      for (int e = 0; e < E; ++e) top[1] = fmaxf(top[1], fabsf(x[e]));
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      top[t] = warp_max(top[t]);
      if (lane == 0) amax[t][warp] = top[t];
    }
  }
  __syncthreads();                                   // (with it the release below is every thread's: their loads come before it)
  if (tid == 0) asm volatile("st.release.gpu.global.u32 [%0], %1;" ::"l"(read + c), "r"(1u) : "memory");
  if constexpr (FMT == kRowsFp8) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int e = fp8_scale_exp(fmaxf(fmaxf(amax[t][0], amax[t][1]), fmaxf(amax[t][2], amax[t][3])));
      now[t] = pow2f(e);
      inv[t] = pow2f(-e);
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      auto code = [&](uint4 u, float scale, float to) {
        float x[E], a[8], z[8];
        piece_values<FMT>(u, scale, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) { a[e] = x[e]; z[e] = x[8 + e]; }
        const uint2 lo = fp8_encode8(a, to), hi = fp8_encode8(z, to);
        return make_uint4(lo.x, lo.y, hi.x, hi.y);
      };
      k[i] = code(k[i], ks[i], inv[0]);
      v[i] = code(v[i], vs[i], inv[1]);
      ks[i] = now[0];
    }
  }
  if (p.kmin) {
    float lo[E], hi[E];
#pragma unroll
    for (int e = 0; e < E; ++e) { lo[e] = INFINITY; hi[e] = -INFINITY; }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if (row0 + i * RPP < n) {
        float x[E];
        piece_values<FMT>(k[i], ks[i], x);
#pragma unroll
        for (int e = 0; e < E; ++e) { lo[e] = fminf(lo[e], x[e]); hi[e] = fmaxf(hi[e], x[e]); }
      }
    }
#pragma unroll
    for (int o = TPR; o < 32; o <<= 1)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        lo[e] = fminf(lo[e], __shfl_xor_sync(0xffffffffu, lo[e], o));
        hi[e] = fmaxf(hi[e], __shfl_xor_sync(0xffffffffu, hi[e], o));
      }
    if (lane < TPR)
#pragma unroll
      for (int e = 0; e < E; ++e) { lows[warp][col * E + e] = lo[e]; highs[warp][col * E + e] = hi[e]; }
  }
  // the earlier pages of this head have been read
  bool ok = c == 0 || p.wait_cycles >= kLookCycles;  // (a bound shorter than a look has run out)
  for (int i = tid; i < c && ok; i += kMoveThreads) {
    if (load_acquire(read + i)) continue;
    const long long t0 = clock64();
    while (!load_acquire(read + i))
      if (clock64() - t0 > p.wait_cycles) { ok = false; break; }
  }
  if (!__syncthreads_and(ok)) {
    if (tid == 0) set_status(p.status, LOSA_ERR_TIMEOUT);
    return;
  }
  const int page = table[c];
  const size_t ph = static_cast<size_t>(page) * p.c.Hkv + kh;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int r = row0 + i * RPP;
    if (r < n || (FMT == kRowsFp8 && r < GP)) {      // (FP8: slots behind the end hold zeros, which k and v are there)
      const int64_t at = page * p.c.stride_page + kh * p.c.stride_head + r * p.c.stride_tok + col * 16;
      *reinterpret_cast<uint4*>(p.k_pages + at) = k[i];
      *reinterpret_cast<uint4*>(p.v_pages + at) = v[i];
      if constexpr (FMT == kRowsInt4) {
        static_cast<uint8_t*>(p.k_scale)[(ph * GP + r) * TPR + col] = static_cast<uint8_t>(kb[i]);
        static_cast<uint8_t*>(p.v_scale)[(ph * GP + r) * TPR + col] = static_cast<uint8_t>(vb[i]);
      }
    }
  }
  if (tid < n) p.weights[ph * GP + tid] = w;
  if (FMT == kRowsFp8 && tid < 2) static_cast<float*>(tid ? p.v_scale : p.k_scale)[ph] = now[tid];
  if (p.kmin)
    for (int e = tid; e < D; e += kMoveThreads) {
      static_cast<T*>(p.kmin)[ph * D + e] = from_f32<T>(fminf(fminf(lows[0][e], lows[1][e]), fminf(lows[2][e], lows[3][e])));
      static_cast<T*>(p.kmax)[ph * D + e] = from_f32<T>(fmaxf(fmaxf(highs[0][e], highs[1][e]), fmaxf(highs[2][e], highs[3][e])));
    }
}

}  // namespace

int32_t launch_kv_evict(losa_ctx* c, losa_kv_t* kv, float* weights, const losa_eviction_t* ev, cudaStream_t st) {
  const losa_shape_t& sh = c->shape;
  EvictParams p = {};
  p.c = cache_params(c, kv);
  p.k_pages = static_cast<uint8_t*>(kv->k_pages);
  p.v_pages = static_cast<uint8_t*>(kv->v_pages);
  p.k_scale = kv->k_scale;
  p.v_scale = kv->v_scale;
  p.kmin = kv->kmin;
  p.kmax = kv->kmax;
  p.weights = weights;
  p.length = ev->length;
  p.budget = ev->budget;
  p.kept = ev->kept;
  p.kv_len = kv->kv_len;
  p.kept_stride = ev->kept_stride;
  p.sinks = ev->sinks;
  p.recent = ev->recent;
  const int n_sk = sh.batch * sh.n_kv_heads;
  p.pages = std::min(sh.max_pages_per_seq, (ev->kept_stride - 1) / sh.page_size + 1);      // (a stride may be any positive number)
  p.goes = reinterpret_cast<int32_t*>(c->ws + c->lay.scores);
  p.read = reinterpret_cast<uint32_t*>(p.goes + n_sk);
  p.ticket = reinterpret_cast<uint32_t*>(c->ws + c->lay.evict_ticket);
  p.status = status_ptr(c);
  p.wait_cycles = c->wait_cycles > 0 ? c->wait_cycles : kWaitCycles;
  const int smem = std::min(kChooseHeld, std::max(1, sh.max_pages_per_seq * sh.page_size)) * 4;
  LOSA_CUDA_TRY(c, cudaFuncSetAttribute(evict_choose_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kChooseHeld * 4));
  launch_k(evict_choose_kernel, n_sk, kChooseThreads, smem, st, p);
  const int32_t rc = after_launch(c);
  if (rc != LOSA_OK || p.pages == 0) return rc;
  auto run = [&](auto f, auto d, auto gp) {
    launch_k(evict_move_kernel<decltype(f)::value, decltype(d)::value, decltype(gp)::value>, n_sk * p.pages, kMoveThreads, 0, st, p);
    return after_launch(c);
  };
  auto with_page = [&](auto f, auto d) {
    return sh.page_size == 16 ? run(f, d, std::integral_constant<int, 16>{})
         : sh.page_size == 32 ? run(f, d, std::integral_constant<int, 32>{}) : run(f, d, std::integral_constant<int, 64>{});
  };
  auto with_dim = [&](auto f) { return sh.head_dim == 128 ? with_page(f, std::integral_constant<int, 128>{}) : with_page(f, std::integral_constant<int, 64>{}); };
  switch (row_format(c, kv)) {
    case kRowsF32: return with_dim(std::integral_constant<int, kRowsF32>{});
    case kRowsBf16: return with_dim(std::integral_constant<int, kRowsBf16>{});
    case kRowsFp8: return with_dim(std::integral_constant<int, kRowsFp8>{});
    default: return with_dim(std::integral_constant<int, kRowsInt4>{});
  }
}

}  // namespace losa
