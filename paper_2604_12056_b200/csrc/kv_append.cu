// New tokens into the paged cache: rotation of queries and keys by position, storage in the cache's format, page
// summaries (losa_rope_append); the same pass without rotation appends a finished block to 4-bit pages, turns a bf16
// cache into 4-bit pages and summarises 4-bit pages.
//
// A copy with a little arithmetic on the way, so HBM bounds it (32,768 tokens of 32 / 8 heads x 128, bf16: 184 us, 70 % of the copy rate; the
// queries' launch 83 %, the pages' 52 %: two pieces a lane are too few in flight), and a chain of dependent reads (lengths, page table,
// rows) when there are few tokens.  Work is cut into units of one warp each, handed out over a flat list, so ragged
// batches leave no warp idle and empty sequences cost nothing:
//   (touched page, tensor, KV head)   the new rows of a page: 16 bytes of a row per lane, four loads in flight,
//                                     rotated in registers, written in the cache's format; for keys also the page's
//                                     element-wise extremes, old rows included, which one warp can therefore
//                                     write without any exchange with others
//   (token, run of query heads)       a token's queries: the table's row is loaded once for all its heads
// The page is the unit because summaries and FP8 scales belong to it.  A rotated pair lies in two lanes (or in one,
// for neighbouring pairs); the partner's 16 bytes come by shuffle, not by a second load.
#include <algorithm>

#include "kernels.h"
#include "page_formats.cuh"

namespace losa {
namespace {

constexpr int kApWarps = 8, kApThreads = kApWarps * 32;
constexpr int kFmtNative = 0, kFmtFp8 = 1, kFmtInt4 = 2;
// what a launch does: all of it, the pages, the queries (two launches, with the registers that each needs, where there is much to do)
constexpr int kAll = 0, kPagesOnly = 1, kQueriesOnly = 2;
// ... and the 16-byte pieces that a lane has in flight: of a page's rows (at three blocks per SM, 80 registers a thread, four with the table's
// parts beside them spill 630 to 760 bytes: 32,768 tokens 226 us; two still spill 56 to 80: 186), of a token's heads (eight, 120 bytes).
constexpr int kApRows = 2;
// 16-byte pieces per lane of an FP8 page that a warp holds in shared memory
constexpr int kApHeld = 16;
constexpr int kApHeldBytes = kApWarps * kApHeld * 32 * 16;
// FP8 pages: two rows' parts of the table in flight and one block per SM in the one launch (few pages: latency), one and two blocks in a launch of
// its own (many).  64 / 1,024 tokens in one launch: 12.1 / 16.9 us the first way, 16.0 / 17.2 the second; 8,192 in two 79.8 and 69.5, with three
// blocks 86.4.
constexpr int fp8_rows(int role) { return role == kAll ? 2 : 1; }
constexpr int blocks_per_sm(int fmt, int role) { return (role == kAll ? 2 : 3) - (fmt == kFmtFp8 ? 1 : 0); }
constexpr int heads_in_flight(int role) { return role == kAll ? 4 : 8; }
// where the new rows come from: the call's tokens, the pages of a bf16 cache, nowhere (summaries of what is there)
constexpr int kSrcTokens = 0, kSrcPages = 1, kSrcNone = 2;

struct AppendParams {
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;            // elements; kSrcPages: k, v are pools with the strides below
  int64_t src_stride_page, src_stride_head, src_stride_tok;
  const int32_t *cu, *start, *pos;
  int uniform;                                     // cu null: this many tokens in every sequence
  const float *cos_t, *sin_t;
  int n_pos, half, interleaved;                    // half = rot_dim / 2; 0: no rotation
  void *q_out, *k_out, *v_out;
  uint8_t *k_pages, *v_pages;                      // null: rotation only
  int64_t stride_page, stride_head, stride_tok;    // bytes
  void *k_scale, *v_scale, *kmin, *kmax;
  const int32_t* page_table;
  int32_t* kv_len_out;
  int N, T, Hq, Hkv, g, Pmax, n_phys;
  int32_t* status;
};

template <typename T> constexpr int vec_of() { return 16 / static_cast<int>(sizeof(T)); }   // elements of 16 bytes
__device__ __forceinline__ void unpack(const uint4& r, float (&x)[8]) { load8(reinterpret_cast<const __nv_bfloat16*>(&r), x); }
__device__ __forceinline__ void unpack(const uint4& r, float (&x)[4]) {
  x[0] = __uint_as_float(r.x); x[1] = __uint_as_float(r.y); x[2] = __uint_as_float(r.z); x[3] = __uint_as_float(r.w);
}
__device__ __forceinline__ uint4 pack(const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&t);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 pack(const float (&x)[4]) {
  return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}

// The part of a table row that a lane with elements j .. j + V - 1 of a head needs.  Always a load (of some row, where there is nothing to
// rotate): one under a condition would be waited for on the spot, and the rows in flight came one after the other.
template <int V> struct Turn { float c[V], s[V]; };
template <int V>
__device__ __forceinline__ Turn<V> load_turn(const AppendParams& p, int pos, int j) {
  Turn<V> t;
  const size_t row = static_cast<size_t>(min(max(pos, 0), p.n_pos - 1)) * p.half;
  if (j >= 2 * p.half) j = 0;
  if (p.interleaved) {
    const float* c = p.cos_t + row + j / 2;
    const float* s = p.sin_t + row + j / 2;
#pragma unroll
    for (int i = 0; i < V / 2; i += 2) {
      const float2 a = __ldg(reinterpret_cast<const float2*>(c + i)), b = __ldg(reinterpret_cast<const float2*>(s + i));
      t.c[i] = a.x; t.c[i + 1] = a.y; t.s[i] = b.x; t.s[i + 1] = b.y;
    }
  } else {
    const int at = j < p.half ? j : j - p.half;
    const float* c = p.cos_t + row + at;
    const float* s = p.sin_t + row + at;
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const float4 a = __ldg(reinterpret_cast<const float4*>(c + i)), b = __ldg(reinterpret_cast<const float4*>(s + i));
      t.c[i] = a.x; t.c[i + 1] = a.y; t.c[i + 2] = a.z; t.c[i + 3] = a.w;
      t.s[i] = b.x; t.s[i + 1] = b.y; t.s[i + 2] = b.z; t.s[i + 3] = b.w;
    }
    if (j < p.half) {                                // the lower half takes its partner with a minus: x cos + (-sin) y
#pragma unroll
      for (int i = 0; i < V; ++i) t.s[i] = -t.s[i];
    }
  }
  return t;
}
// two at a time
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 c;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(c.x), "=f"(c.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return c;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\tfma.rn.f32x2 z, x, y, z;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
// A lane's 16 bytes, rotated.  The partner's product is rounded, the element's own is added to it unrounded, said outright so that the result does
// not hang on what the compiler would contract.  All lanes of the warp take part; `on`: this lane's elements are rotated.
template <typename T, int V>
__device__ __forceinline__ uint4 rotate(const AppendParams& p, const uint4& raw, const Turn<V>& t, int j, bool on, int lane) {
  float x[V], y[V];
  unpack(raw, x);
  if (p.interleaved) {
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
      y[2 * i] = __fmaf_rn(x[2 * i], t.c[i], -__fmul_rn(x[2 * i + 1], t.s[i]));
      y[2 * i + 1] = __fmaf_rn(x[2 * i + 1], t.c[i], __fmul_rn(x[2 * i], t.s[i]));
    }
  } else {
    const int d = p.half / V, from = on ? (j < p.half ? lane + d : lane - d) : lane;
    uint4 o;
    o.x = __shfl_sync(0xffffffffu, raw.x, from);
    o.y = __shfl_sync(0xffffffffu, raw.y, from);
    o.z = __shfl_sync(0xffffffffu, raw.z, from);
    o.w = __shfl_sync(0xffffffffu, raw.w, from);
    float z[V];
    unpack(o, z);
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      const float2 r = fma2(make_float2(x[i], x[i + 1]), make_float2(t.c[i], t.c[i + 1]), mul2(make_float2(z[i], z[i + 1]), make_float2(t.s[i], t.s[i + 1])));
      y[i] = r.x;
      y[i + 1] = r.y;
    }
  }
  return on ? pack(y) : raw;
}

// Tokens and place of sequence s; n = -1: it does not fit and is left out.
struct Span { int a, n, first; };
template <int SRC>
__device__ __forceinline__ Span span_of(const AppendParams& p, int s) {
  Span r;
  if (SRC != kSrcTokens) {                         // the whole sequence; what is longer than its page-table row is not there
    r.first = 0;
    r.a = 0;
    r.n = p.start[s];
    const long long cap = static_cast<long long>(p.Pmax) * p.g;
    if (r.n < 0) r.n = -1;
    if (r.n > cap) r.n = static_cast<int>(cap);
    return r;
  }
  r.first = p.cu ? p.cu[s] : s * p.uniform;
  const int end = p.cu ? p.cu[s + 1] : r.first + p.uniform;
  r.a = p.start ? p.start[s] : 0;
  r.n = end - r.first;
  const long long last = static_cast<long long>(r.a) + r.n;
  const bool stored = p.k_pages != nullptr;
  bool ok = r.first >= 0 && r.n >= 0 && end <= p.T && r.a >= 0;
  if (ok && r.n > 0) {
    if (stored && last > static_cast<long long>(p.Pmax) * p.g) ok = false;
    if (p.half > 0 && !p.pos && last > p.n_pos) ok = false;
  }
  if (!ok) r.n = -1;
  return r;
}

// Touched pages of all sequences as a prefix over them, in shared memory (one warp).
template <int SRC>
__device__ __forceinline__ void page_prefix(const AppendParams& p, int* pre, int lane) {
  int run = 0;
  for (int base = 0; base < p.N; base += 32) {
    const int s = base + lane;
    int c = 0;
    if (s < p.N) {
      const Span sp = span_of<SRC>(p, s);
      if (sp.n < 0 && blockIdx.x == 0) set_status(p.status, LOSA_ERR_BOUNDS);
      if (sp.n > 0) c = (sp.a + sp.n - 1) / p.g - sp.a / p.g + 1;
    }
    int inc = c;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += t;
    }
    if (s < p.N) pre[s] = run + inc - c;
    run += __shfl_sync(0xffffffffu, inc, 31);
  }
  if (lane == 0) pre[p.N] = run;
}
// the last s of n with first[s] <= i (ascending, first[0] <= i)
__device__ __forceinline__ int find_seq(const int* first, int n, int i) {
  int a = 0, b = n;
  while (b - a > 1) {
    const int m = (a + b) >> 1;
    if (first[m] <= i) a = m; else b = m;
  }
  return a;
}

__device__ __forceinline__ void copy_async16(uint4* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(static_cast<uint32_t>(__cvta_generic_to_shared(dst))), "l"(src) : "memory");
}
// One page's new rows of one KV head and tensor; hold: this lane's first piece of kApHeld, 32 apart (FP8 pages).
template <typename T, int FMT, int D, int SRC, int ROLE>
__device__ __forceinline__ void append_page(const AppendParams& p, int s, int page, int kh, bool is_v, uint4* hold, int lane) {
  constexpr int U = kApRows, V = vec_of<T>(), LPR = D / V, RPI = 32 / LPR;
  constexpr int RUNS = D / kInt4Run, LRUN = kInt4Run / V;        // 4-bit: runs per row, lanes per run
  const Span sp = span_of<SRC>(p, s);
  const int base = page * p.g;
  const int t_hi = min(p.g, sp.a + sp.n - base), t_lo = SRC == kSrcNone ? t_hi : max(0, sp.a - base);
  const int phys = p.page_table[static_cast<size_t>(s) * p.Pmax + page];
  if (phys < 0 || phys >= p.n_phys) { if (lane == 0) set_status(p.status, LOSA_ERR_BOUNDS); return; }
  const int sub = lane / LPR, j = (lane % LPR) * V;
  uint8_t* row0 = (is_v ? p.v_pages : p.k_pages) + static_cast<int64_t>(phys) * p.stride_page + static_cast<int64_t>(kh) * p.stride_head;
  const size_t slice = static_cast<size_t>(phys) * p.Hkv + kh;
  uint8_t* run_scale = static_cast<uint8_t*>(is_v ? p.v_scale : p.k_scale) + slice * p.g * RUNS;           // 4-bit
  float* page_scale = static_cast<float*>(is_v ? p.v_scale : p.k_scale) + slice;                         // FP8
  const bool rot = !is_v && p.half > 0 && SRC == kSrcTokens;
  const bool summaries = !is_v && p.kmin != nullptr;
  T* keep = SRC == kSrcTokens ? static_cast<T*>(is_v ? p.v_out : p.k_out) : nullptr;

  float lo[V], hi[V];
#pragma unroll
  for (int x = 0; x < V; ++x) { lo[x] = INFINITY; hi[x] = -INFINITY; }
  auto extremes = [&](const float (&v)[V]) {
#pragma unroll
    for (int x = 0; x < V; ++x) { lo[x] = fminf(lo[x], v[x]); hi[x] = fmaxf(hi[x], v[x]); }
  };
  auto token_of = [&](int t) { return sp.first + base + t - sp.a; };
  // a lane's 16 bytes of new row t (rotated); all lanes take part, `here` says whether the row exists
  auto source = [&](int t) {
    if (SRC == kSrcPages)
      return static_cast<const T*>(is_v ? p.v : p.k) + static_cast<int64_t>(phys) * p.src_stride_page + static_cast<int64_t>(kh) * p.src_stride_head + static_cast<int64_t>(t) * p.src_stride_tok + j;
    return static_cast<const T*>(is_v ? p.v : p.k) + static_cast<int64_t>(token_of(t)) * (is_v ? p.v_stride : p.k_stride) + static_cast<int64_t>(kh) * D + j;
  };
  auto fetch = [&](int t, bool here) { return here ? __ldcs(reinterpret_cast<const uint4*>(source(t))) : make_uint4(0u, 0u, 0u, 0u); };
  // the table's part for new row t; on: this lane's elements of it are to be rotated
  auto turn = [&](int t, bool here, bool& on) {
    on = here && j < 2 * p.half;
    int pos = base + t;
    if (p.pos) {
      pos = here ? p.pos[token_of(t)] : 0;
      if (pos < 0 || pos >= p.n_pos) { on = false; set_status(p.status, LOSA_ERR_BOUNDS); }
    }
    return load_turn<V>(p, pos, j);
  };
  auto out_row = [&](int t) { return reinterpret_cast<uint4*>(keep + (static_cast<size_t>(token_of(t)) * p.Hkv + kh) * D + j); };

  if constexpr (FMT == kFmtFp8) {
    // one scale for the page, from its old rows and the new ones together.  A page that a warp can hold (16 pieces per lane) is requested as
    // a whole, by asynchronous copies, and stays in shared memory until its codes are written; a larger one is gone over twice.
    constexpr int M = kApHeld;
    const float old_scale = *page_scale;
    const bool held = p.g <= M * RPI;
    auto encode = [&](int t, const uint4& raw, float scale, float inv) {
      float v[8];
      unpack(raw, v);
      const uint2 code = t < t_hi ? fp8_encode8(v, inv) : make_uint2(0u, 0u);
      *reinterpret_cast<uint2*>(row0 + static_cast<int64_t>(t) * p.stride_tok + j) = code;
      if (keep && t >= t_lo && t < t_hi) {
        float w[8];
        fp8_decode8(code, w);
#pragma unroll
        for (int x = 0; x < 8; ++x) w[x] *= scale;
        *out_row(t) = pack(w);
      }
    };
    auto old_row = [&](uint2 codes) {
      float v[8];
      fp8_decode8(codes, v);
#pragma unroll
      for (int x = 0; x < 8; ++x) v[x] *= old_scale;
      return pack(v);                                // exact: four significant bits
    };
    constexpr int F = fp8_rows(ROLE);                // rows whose part of the table is in flight
    auto values = [&](int tb, uint4 (&raw)[F]) {     // all lanes
#pragma unroll
      for (int u = 0; u < F; ++u) {
        const int t = tb + u * RPI + sub;
        raw[u] = fetch(t, t >= t_lo && t < t_hi);
      }
      uint2 old[F];
      Turn<V> tn[F];
      bool on[F];
      if (rot) {
#pragma unroll
        for (int u = 0; u < F; ++u) tn[u] = turn(tb + u * RPI + sub, tb + u * RPI + sub >= t_lo && tb + u * RPI + sub < t_hi, on[u]);
      }
#pragma unroll
      for (int u = 0; u < F; ++u) {
        const int t = tb + u * RPI + sub;
        old[u] = t < t_lo ? *reinterpret_cast<const uint2*>(row0 + static_cast<int64_t>(t) * p.stride_tok + j) : make_uint2(0u, 0u);
      }
#pragma unroll
      for (int u = 0; u < F; ++u) {
        const int t = tb + u * RPI + sub;
        if (rot) raw[u] = rotate<T, V>(p, raw[u], tn[u], j, on[u], lane);
        if (t < t_lo) raw[u] = old_row(old[u]);
      }
    };
    if (held) {
#pragma unroll 4
      for (int i = 0; i < M; ++i) {
        const int t = i * RPI + sub;
        if (t >= t_lo && t < t_hi) copy_async16(hold + 32 * i, source(t));
        else hold[32 * i] = make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll 1
      for (int t = sub; t < t_lo; t += RPI)          // (few pages have old rows)
        hold[32 * (t / RPI)] = old_row(*reinterpret_cast<const uint2*>(row0 + static_cast<int64_t>(t) * p.stride_tok + j));
      asm volatile("cp.async.wait_all;" ::: "memory");      // a lane reads what it has copied itself
#pragma unroll 1
      for (int tb = 0; tb < t_hi; tb += RPI * F) {
        uint4 raw[F];
#pragma unroll
        for (int u = 0; u < F; ++u) raw[u] = hold[32 * (tb / RPI + u)];
        if (rot && tb + RPI * F > t_lo) {
          Turn<V> tn[F];
          bool on[F];
#pragma unroll
          for (int u = 0; u < F; ++u) tn[u] = turn(tb + u * RPI + sub, tb + u * RPI + sub >= t_lo && tb + u * RPI + sub < t_hi, on[u]);
#pragma unroll
          for (int u = 0; u < F; ++u) {
            raw[u] = rotate<T, V>(p, raw[u], tn[u], j, on[u], lane);
            hold[32 * (tb / RPI + u)] = raw[u];
          }
        }
#pragma unroll
        for (int u = 0; u < F; ++u)
          if (tb + u * RPI + sub < t_hi) {
            float v[8];
            unpack(raw[u], v);
            extremes(v);
          }
      }
    } else {
#pragma unroll 1
      for (int tb = 0; tb < t_hi; tb += RPI * F) {
        uint4 raw[F];
        values(tb, raw);
#pragma unroll
        for (int u = 0; u < F; ++u)
          if (tb + u * RPI + sub < t_hi) {
            float v[8];
            unpack(raw[u], v);
            extremes(v);
          }
      }
    }
    float amax = 0.f;
#pragma unroll
    for (int x = 0; x < V; ++x)
      if (lo[x] <= hi[x]) amax = fmaxf(amax, fmaxf(fabsf(lo[x]), fabsf(hi[x])));
    const int e = fp8_scale_exp(warp_max(amax));
    const float scale = pow2f(e), inv = pow2f(-e);
    if (held) {
#pragma unroll 2
      for (int i = 0; i < M; ++i)
        if (i * RPI + sub < p.g) encode(i * RPI + sub, hold[32 * i], scale, inv);
    } else {
#pragma unroll 1
      for (int tb = 0; tb < p.g; tb += RPI * F) {
        uint4 raw[F];
        values(tb, raw);
#pragma unroll
        for (int u = 0; u < F; ++u) encode(tb + u * RPI + sub, raw[u], scale, inv);
      }
    }
    __syncwarp();                                    // every lane has read the old scale
    if (lane == 0) *page_scale = scale;
    if (!summaries) return;
    float a[8], b[8];                                // encoding is monotone: the extremes of the codes are the codes of the extremes
    fp8_decode8(fp8_encode8(lo, inv), a);
    fp8_decode8(fp8_encode8(hi, inv), b);
#pragma unroll
    for (int x = 0; x < 8; ++x)                      // (a column without rows in this lane, or with NaN alone, has none)
      if (lo[x] <= hi[x]) { lo[x] = a[x] * scale; hi[x] = b[x] * scale; }
  } else {
    uint4 raw[U];                                    // the first rows are requested before those of the page that were there
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = fetch(t_lo + u * RPI + sub, t_lo + u * RPI + sub < t_hi);
    if (summaries)                                   // rows that were there before
      for (int t = sub; t < t_lo; t += RPI) {
        float v[V];
        if constexpr (FMT == kFmtInt4) {
          const uint32_t w = *reinterpret_cast<const uint32_t*>(row0 + static_cast<int64_t>(t) * p.stride_tok + j / 2);
          int4_decode8(w, int4_scale_value(run_scale[t * RUNS + j / kInt4Run]), v);
        } else {
          unpack(*reinterpret_cast<const uint4*>(row0 + static_cast<int64_t>(t) * p.stride_tok + j * sizeof(T)), v);
        }
        extremes(v);
      }
    for (int tb = t_lo; tb < t_hi; tb += RPI * U) {
      if (tb > t_lo) {
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = fetch(tb + u * RPI + sub, tb + u * RPI + sub < t_hi);
      }
      if (rot) {
        Turn<V> tn[U];
        bool on[U];
#pragma unroll
        for (int u = 0; u < U; ++u) tn[u] = turn(tb + u * RPI + sub, tb + u * RPI + sub < t_hi, on[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = rotate<T, V>(p, raw[u], tn[u], j, on[u], lane);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int t = tb + u * RPI + sub;
        const bool here = t < t_hi;
        float v[V];
        unpack(raw[u], v);
        if constexpr (FMT == kFmtInt4) {
          float amax = fabsf(v[0]);                  // the run's largest value; a NaN is kept
#pragma unroll
          for (int x = 1; x + 1 < V; x += 2) amax = max_nan(amax, fabsf(v[x]), fabsf(v[x + 1]));
          amax = max_nan(amax, fabsf(v[V - 1]), 0.f);
#pragma unroll
          for (int o = 1; o < LRUN; o <<= 1) amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, o), 0.f);
          const float scale = int4_scale(amax), mul = int4_multiplier(scale), held = int4_held_scale(scale, amax);
          if (amax > 7.f * kInt4MaxScale) {          // saturate
#pragma unroll
            for (int x = 0; x < V; ++x) v[x] = fminf(fmaxf(v[x], -7.f * kInt4MaxScale), 7.f * kInt4MaxScale);
          }
          uint32_t w = 0;
#pragma unroll
          for (int x = 0; x < V; ++x) {
            const float m = int4_round(v[x], mul);
            w |= int4_bits(m) << (4 * x);
            v[x] = (m - kInt4Magic) * held;          // exact; what the pages hold, a NaN too
          }
          if (here) {
            *reinterpret_cast<uint32_t*>(row0 + static_cast<int64_t>(t) * p.stride_tok + j / 2) = w;
            if ((lane & (LRUN - 1)) == 0) run_scale[t * RUNS + j / kInt4Run] = static_cast<uint8_t>(int4_scale_byte(held));
            if (keep) *out_row(t) = pack(v);
          }
        } else if (here) {
          *reinterpret_cast<uint4*>(row0 + static_cast<int64_t>(t) * p.stride_tok + j * sizeof(T)) = raw[u];
          if (keep) *out_row(t) = raw[u];
        }
        if (summaries && here) extremes(v);
      }
    }
    if (!summaries) return;
  }
#pragma unroll
  for (int o = LPR; o < 32; o <<= 1)
#pragma unroll
    for (int x = 0; x < V; ++x) {
      lo[x] = fminf(lo[x], __shfl_xor_sync(0xffffffffu, lo[x], o));
      hi[x] = fmaxf(hi[x], __shfl_xor_sync(0xffffffffu, hi[x], o));
    }
  if (sub == 0) {
    const size_t at = slice * D + j;
    *reinterpret_cast<uint4*>(static_cast<T*>(p.kmin) + at) = pack(lo);
    *reinterpret_cast<uint4*>(static_cast<T*>(p.kmax) + at) = pack(hi);
  }
}

// Rotated heads h0 .. of one token, out of place or in place.
template <typename T, int D, int U>
__device__ __forceinline__ void rotate_token(const AppendParams& p, int t, int h0, const void* x, int64_t stride, void* out, int H, int lane) {
  constexpr int V = vec_of<T>(), LPR = D / V, RPI = 32 / LPR;
  const int sub = lane / LPR, j = (lane % LPR) * V;
  const T* src = static_cast<const T*>(x) + static_cast<int64_t>(t) * stride + j;
  T* dst = static_cast<T*>(out) + static_cast<size_t>(t) * H * D + j;
  uint4 raw[U];                                      // requested before it is known where the token belongs
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int h = h0 + u * RPI + sub;
    raw[u] = h < H ? *reinterpret_cast<const uint4*>(src + h * D) : make_uint4(0u, 0u, 0u, 0u);
  }
  int pos = 0;
  if (p.pos) {
    pos = p.pos[t];
  }
  if (!p.pos || p.k_pages) {                         // (with positions and no cache the sequences do not matter)
    const int s = find_seq(p.cu, p.N, t);
    const Span sp = span_of<kSrcTokens>(p, s);
    if (sp.n < 0 || t < sp.first || t >= sp.first + sp.n) return;
    if (!p.pos) pos = sp.a + t - sp.first;
  }
  bool on = j < 2 * p.half;
  if (p.half > 0 && (pos < 0 || pos >= p.n_pos)) { on = false; set_status(p.status, LOSA_ERR_BOUNDS); }
  Turn<V> tn;
  if (p.half > 0) tn = load_turn<V>(p, pos, j);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int h = h0 + u * RPI + sub;
    if (p.half > 0) raw[u] = rotate<T, V>(p, raw[u], tn, j, on, lane);
    if (h < H) __stcs(reinterpret_cast<uint4*>(dst + h * D), raw[u]);
  }
}

template <typename T, int FMT, int D, int SRC, int ROLE>
__global__ void __launch_bounds__(kApThreads, blocks_per_sm(FMT, ROLE)) append_kernel(const __grid_constant__ AppendParams p) {
  extern __shared__ uint4 shared[];                  // FP8: pages; then [N + 1]
  int* pre = reinterpret_cast<int*>(reinterpret_cast<char*>(shared) + (FMT == kFmtFp8 ? kApHeldBytes : 0));
  grid_dep_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const bool stored = p.k_pages != nullptr;
  if (stored && ROLE != kQueriesOnly) {
    if (warp == 0) page_prefix<SRC>(p, pre, lane);
    __syncthreads();
  }
  if (SRC == kSrcTokens && ROLE != kQueriesOnly && blockIdx.x == 0) {
    for (int s = threadIdx.x; s < p.N && (p.kv_len_out || !stored); s += kApThreads) {
      if (!stored && p.pos) break;
      const Span sp = span_of<SRC>(p, s);
      if (sp.n < 0) set_status(p.status, LOSA_ERR_BOUNDS);
      else if (sp.n > 0 && stored) p.kv_len_out[s] = sp.a + sp.n;
    }
  }
  constexpr int RPI = 32 / (D / vec_of<T>()), QU = heads_in_flight(ROLE), HEADS = RPI * QU;      // heads of a token that a unit takes
  const int tensors = SRC == kSrcNone ? 1 : 2;
  const long long page_units = stored && ROLE != kQueriesOnly ? static_cast<long long>(pre[p.N]) * tensors * p.Hkv : 0;
  const int q_runs = SRC == kSrcTokens && ROLE != kPagesOnly && p.q_out ? (p.Hq + HEADS - 1) / HEADS : 0;
  const int k_runs = SRC == kSrcTokens && ROLE != kPagesOnly && !stored && p.k_out ? (p.Hkv + HEADS - 1) / HEADS : 0;
  const long long units = page_units + static_cast<long long>(p.T) * (q_runs + k_runs);
  for (long long u = static_cast<long long>(blockIdx.x) * kApWarps + warp; u < units; u += static_cast<long long>(gridDim.x) * kApWarps) {
    if (ROLE != kQueriesOnly && u < page_units) {
      const int item = static_cast<int>(u / (tensors * p.Hkv)), rest = static_cast<int>(u % (tensors * p.Hkv));
      const int s = find_seq(pre, p.N, item);
      const int first_page = SRC == kSrcTokens ? p.start[s] / p.g : 0;
      append_page<T, FMT, D, SRC, ROLE>(p, s, first_page + item - pre[s], rest % p.Hkv, rest >= p.Hkv, shared + warp * kApHeld * 32 + lane, lane);
    } else if constexpr (SRC == kSrcTokens && ROLE != kPagesOnly) {
      const long long v = u - page_units;
      const int t = static_cast<int>(v / (q_runs + k_runs)), r = static_cast<int>(v % (q_runs + k_runs));
      if (r < q_runs) rotate_token<T, D, QU>(p, t, r * HEADS, p.q, p.q_stride, p.q_out, p.Hq, lane);
      else rotate_token<T, D, QU>(p, t, (r - q_runs) * HEADS, p.k, p.k_stride, p.k_out, p.Hkv, lane);
    }
  }
}

// `units`: at most so many
template <typename T, int FMT, int D, int SRC, int ROLE>
int32_t launch_units(losa_ctx* c, const AppendParams& p, long long units, cudaStream_t st) {
  if (units <= 0) return LOSA_OK;
  const long long blocks = std::min<long long>((units + kApWarps - 1) / kApWarps, static_cast<long long>(c->n_sms) * 8);
  auto kernel = append_kernel<T, FMT, D, SRC, ROLE>;
  if constexpr (FMT == kFmtFp8) {
    const size_t bytes = kApHeldBytes + (p.N + 1) * sizeof(int);
    // the most that any context asks for: the limit is the kernel's, whose other contexts have batches of their own
    constexpr int most = kApHeldBytes + (kMaxSegments + 1) * static_cast<int>(sizeof(int));
    if (!(c->append_attr_set & (1 << ROLE))) {       // (a context has one head dimension)
      LOSA_CUDA_TRY(c, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most));
      c->append_attr_set |= 1 << ROLE;
    }
    launch_k(kernel, static_cast<unsigned>(blocks), kApThreads, bytes, st, p);
  } else {
    launch_streaming(kernel, static_cast<unsigned>(blocks), kApThreads, (p.N + 1) * sizeof(int), st, p);
  }
  return after_launch(c);
}
template <typename T, int FMT, int SRC, int ROLE = kAll>
int32_t launch_dim(losa_ctx* c, const AppendParams& p, long long units, cudaStream_t st) {
  return c->shape.head_dim == 128 ? launch_units<T, FMT, 128, SRC, ROLE>(c, p, units, st) : launch_units<T, FMT, 64, SRC, ROLE>(c, p, units, st);
}
// From so many bytes of queries on, queries and pages are two launches, each with the registers that it needs.  One launch and two, tokens of
// 32 / 8 heads x 128 (8 KB of queries each): 64 11.2 and 15.2 us, 2,048 16.3 and 24.2, 4,096 31.7 and 37.3, 8,192 58.1 and 57.7, 32,768
// 240 and 199; into 4 bits 64 15.1 and 19.5, 4,096 36.1 and 42.8, 8,192 66.6 and 68.6, 15,164 119 and 113.
// FP8, whose pages take most of the time, from a quarter of that on: 1,024 16.9 and 19.3, 2,048 27.1 and 26.4, 4,096 53.7 and 41.5, 8,192 100.6 and 69.4.
template <int FMT> constexpr long long split_bytes() { return (FMT == kFmtFp8 ? 16ll : 64ll) << 20; }
template <typename T, int FMT>
int32_t launch_tokens(losa_ctx* c, const AppendParams& p, long long pages, long long tokens, cudaStream_t st) {
  if (p.k_pages && p.q_out && tokens * p.Hq * c->shape.head_dim * static_cast<long long>(sizeof(T)) >= split_bytes<FMT>()) {
    const int32_t rc = launch_dim<T, FMT, kSrcTokens, kPagesOnly>(c, p, pages * 2 * p.Hkv, st);
    return rc != LOSA_OK ? rc : launch_dim<T, kFmtNative, kSrcTokens, kQueriesOnly>(c, p, tokens * p.Hq, st);
  }
  return launch_dim<T, FMT, kSrcTokens>(c, p, pages * 2 * p.Hkv + tokens * (p.Hq + p.Hkv), st);
}

AppendParams base_params(const losa_ctx* c, const losa_kv_t* kv) {
  const losa_shape_t& sh = c->shape;
  AppendParams p = {};
  p.N = sh.batch;
  p.Hq = sh.n_q_heads;
  p.Hkv = sh.n_kv_heads;
  p.g = sh.page_size;
  p.Pmax = sh.max_pages_per_seq;
  p.status = status_ptr(c);
  if (kv) {
    const int64_t es = kv->kv_format == LOSA_KV_NATIVE ? (sh.dtype == LOSA_BF16 ? 2 : 4) : 1;
    p.k_pages = static_cast<uint8_t*>(kv->k_pages);
    p.v_pages = static_cast<uint8_t*>(kv->v_pages);
    p.stride_page = kv->stride_page * es;
    p.stride_head = kv->stride_head * es;
    p.stride_tok = kv->stride_tok * es;
    p.k_scale = kv->k_scale;
    p.v_scale = kv->v_scale;
    p.kmin = kv->kmin;
    p.kmax = kv->kmax;
    p.page_table = kv->page_table;
    p.n_phys = kv->n_phys_pages;
  }
  return p;
}
long long all_pages(const losa_ctx* c) { return static_cast<long long>(c->shape.batch) * c->shape.max_pages_per_seq; }

}  // namespace

int32_t launch_rope_append(losa_ctx* c, losa_kv_t* kv, const losa_rope_t* rope, const losa_new_tokens_t* tk, cudaStream_t st) {
  const losa_shape_t& sh = c->shape;
  AppendParams p = base_params(c, kv);
  p.q = tk->q; p.k = tk->k; p.v = tk->v;
  p.q_stride = tk->q_stride; p.k_stride = tk->k_stride; p.v_stride = tk->v_stride;
  p.cu = tk->cu; p.start = tk->start; p.pos = rope ? tk->pos_opt : nullptr;
  if (rope) {
    p.cos_t = rope->cos_table;
    p.sin_t = rope->sin_table;
    p.n_pos = rope->n_pos;
    p.half = rope->rot_dim / 2;
    p.interleaved = rope->interleaved ? 1 : 0;
  }
  p.q_out = tk->q_out; p.k_out = tk->k_out; p.v_out = tk->v_out;
  p.kv_len_out = kv ? kv->kv_len : nullptr;
  p.T = tk->n_tokens;
  // a sequence's tokens touch one page more than they fill at most, and no more pages than there are tokens
  const long long pages = std::min<long long>(p.T, p.T / sh.page_size + 2ll * sh.batch);
  const long long stored = kv ? pages : 0;
  if (sh.dtype == LOSA_F32) return launch_tokens<float, kFmtNative>(c, p, stored, p.T, st);
  const int fmt = kv ? kv->kv_format : LOSA_KV_NATIVE;
  if (fmt == LOSA_KV_FP8_E4M3) return launch_tokens<__nv_bfloat16, kFmtFp8>(c, p, stored, p.T, st);
  if (fmt == LOSA_KV_INT4) return launch_tokens<__nv_bfloat16, kFmtInt4>(c, p, stored, p.T, st);
  return launch_tokens<__nv_bfloat16, kFmtNative>(c, p, stored, p.T, st);
}

// the kv_len / step counters are bumped by the caller's counter kernel afterwards
int32_t launch_int4_append(losa_ctx* c, losa_kv_t* kv, const void* k_blk, const void* v_blk, cudaStream_t st) {
  const losa_shape_t& sh = c->shape;
  AppendParams p = base_params(c, kv);
  p.k = k_blk;
  p.v = v_blk;
  p.k_stride = p.v_stride = static_cast<int64_t>(sh.n_kv_heads) * sh.head_dim;
  p.start = kv->kv_len;
  p.uniform = sh.block_size;
  p.T = sh.batch * sh.block_size;
  const long long pages = static_cast<long long>(sh.batch) * ((sh.block_size + sh.page_size - 1) / sh.page_size + 1);
  return launch_dim<__nv_bfloat16, kFmtInt4, kSrcTokens>(c, p, pages * 2 * p.Hkv, st);
}

int32_t launch_int4_quantize(losa_ctx* c, const losa_kv_t* src, losa_kv_t* dst, cudaStream_t st) {
  AppendParams p = base_params(c, dst);
  p.k = src->k_pages;
  p.v = src->v_pages;
  p.src_stride_page = src->stride_page;
  p.src_stride_head = src->stride_head;
  p.src_stride_tok = src->stride_tok;
  p.start = dst->kv_len;
  return launch_dim<__nv_bfloat16, kFmtInt4, kSrcPages>(c, p, all_pages(c) * 2 * p.Hkv, st);
}

int32_t launch_int4_summaries(losa_ctx* c, losa_kv_t* kv, cudaStream_t st) {
  AppendParams p = base_params(c, kv);
  p.start = kv->kv_len;
  return launch_dim<__nv_bfloat16, kFmtInt4, kSrcNone>(c, p, all_pages(c) * p.Hkv, st);
}

}  // namespace losa
