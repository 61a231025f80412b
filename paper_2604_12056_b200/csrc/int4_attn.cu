// Attention over a cache held in 4 bits: losa_int4_attn (every block token over the whole cache) and stage 4 of the
// method on such a cache (active tokens over the listed pages; Section 2.2, Section 4.2).
//
// The pages to read form one flat list over (sequence, KV head, group of query rows), cut into equal shares, so
// ragged batches leave no SM idle; partial results of a segment that several CTAs share meet by log-sum-exp.
#include <algorithm>
#include <type_traits>

#include "kernels.h"
#include "page_formats.cuh"
#include "tcgen05_ops.cuh"

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
  int N, B, Hq, Hkv, G, g, Pmax, n_phys, n_sk, n_rg, pad;
  int rows_above, rows_upto;                       // segments with as many query rows are this kernel's
  float sm_scale;
  long long wait_cycles;                           // bound of every mbarrier wait, in SM clock cycles
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
// ===================================================================== codes into operands
// A word of eight codes becomes four half2 operands with their scale in ten instructions: two shifts, and
// for each half2 one LOP3 ((x & mask) | 0x6400: 1024 + 4u or 1024 + 64u as fp16) and one HFMA2 whose result,
// scale * (u - 8) / 4, is exact: scales have four significant bits, so the addends 66 scale and 6 scale have ten and six.
// (The quarter keeps 66 scale below fp16's end for scales up to 960; the softmax scale and the end result take it back.)  Integers put into the
// mantissa of 1024 as fp16 are a published way (Kim, Henry, Fahim, Awadalla: Who Says Elephants Can't Run, 2022); two places and one fused step are this format's.
//
// (x & MASK) | 0x6400 of both halves, as one instruction
template <uint32_t MASK>
__device__ __forceinline__ uint32_t i4_take(uint32_t x) {
  uint32_t d;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(d) : "r"(x), "n"(MASK), "r"(0x64006400u));
  return d;
}
__device__ __forceinline__ uint32_t fma_h2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ uint32_t mul_h2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// multipliers and addends of the two places a code is taken from
struct I4Scale { uint32_t m4, a4, m64, a64; };
__device__ __forceinline__ I4Scale i4_scale(uint32_t s2) {     // s2: the scales of the two halves as fp16
  I4Scale r;
  r.m4 = mul_h2(s2, 0x2c002c00u);                    // 1 / 16
  r.a4 = mul_h2(s2, 0xd420d420u);                    // -66
  r.m64 = mul_h2(s2, 0x1c001c00u);                   // 1 / 256
  r.a64 = mul_h2(s2, 0xc600c600u);                   // -6
  return r;
}
// the four codes of each half of x -> h[0..3], each half2 one code of either half
__device__ __forceinline__ void i4_operands(uint32_t x, const I4Scale& s, uint32_t (&h)[4]) {
  const uint32_t y = x << 2, z = x >> 6;              // codes 0, 1 and 2, 3 of each half at bits 2 .. 5 and 6 .. 9
  h[0] = fma_h2(i4_take<0x003c003cu>(y), s.m4, s.a4);
  h[1] = fma_h2(i4_take<0x03c003c0u>(y), s.m64, s.a64);
  h[2] = fma_h2(i4_take<0x003c003cu>(z), s.m4, s.a4);
  h[3] = fma_h2(i4_take<0x03c003c0u>(z), s.m64, s.a64);
}

// ===================================================================== the list of work
// A piece of a CTA's share: pages first_page .. of one (sequence, KV head, group of R query rows).
struct I4Piece { int s, kh, rg, sk, seg_lo, pages, hi, first_page, n_units; };

// The pages to read, over all segments (sequence, KV head, row group), as one list that is cut into equal shares.  Every segment
// begins with `pad` positions that stand for no page: entering one costs a CTA about as much as that many pages.
template <int D, int R>
struct I4Work {
  const I4Params& p;
  int* pre;                                          // [n_sk + 1] charged positions before a (sequence, KV head)
  int* runs;                                         // [32]
  int upp_log, upp_mask, T, n_share, lo, hi, sk0;

  // unit: tokens by which work is handed out inside a CTA (a page or a part of one)
  __device__ __forceinline__ I4Work(const I4Params& params, int* prefix, int* run_sums, int unit) : p(params), pre(prefix), runs(run_sums) {
    upp_log = p.g > unit ? (p.g == 2 * unit ? 1 : 2) : 0;
    upp_mask = (1 << upp_log) - 1;
  }
  // query rows of a sequence that are this kernel's business
  __device__ __forceinline__ int rows_of(int s) const {
    const int rows = (p.n_active ? clamp_rows(p.n_active[s], p.B) : p.B) * p.G;
    return rows > p.rows_above && rows <= p.rows_upto ? rows : 0;
  }
  __device__ __forceinline__ int pages_in(int sk) const {
    if (p.union_count) return min(max(p.union_count[sk], 0), p.Pmax);
    return min(max((p.kv_len[sk / p.Hkv] + p.g - 1) / p.g, 0), p.Pmax);
  }
  // All threads of the CTA: the prefix, this CTA's share; results of rows without any page; false: nothing (more) to do.
  // least: units below which a share is not cut.
  __device__ __forceinline__ bool begin(int least) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, W = blockDim.x >> 5;
    const int n_runs = (p.n_sk + 31) >> 5;
    for (int b = warp; b < n_runs; b += W) {         // runs of 32 by the warps, then the runs' sums
      const int sk = b * 32 + lane;
      int c = 0;
      if (sk < p.n_sk) {
        const int pages = pages_in(sk);
        if (pages > 0) c = (pages + p.pad) * ((rows_of(sk / p.Hkv) + R - 1) / R);
      }
      int inc = c;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
      }
      if (sk < p.n_sk) pre[sk] = inc - c;
      if (lane == 31) runs[b] = inc;
    }
    __syncthreads();
    if (warp == 0) {
      const int c = lane < n_runs ? runs[lane] : 0;
      int inc = c;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
      }
      runs[lane] = inc - c;
      if (lane == 31) pre[p.n_sk] = inc;
    }
    __syncthreads();
    for (int i = 32 + tid; i < p.n_sk; i += blockDim.x) pre[i] += runs[i >> 5];
    __syncthreads();
    T = pre[p.n_sk];
    n_share = max(1, min(static_cast<int>(gridDim.x), ((T << upp_log) + least - 1) / least));
    for (int sk = blockIdx.x; sk < p.n_sk; sk += gridDim.x) {
      const int s = sk / p.Hkv, kh = sk - s * p.Hkv, rows = rows_of(s), pages = pages_in(sk);
      if (!p.union_count && kh == 0 && tid == 0 && (p.kv_len[s] + p.g - 1) / p.g > p.Pmax) set_status(p.status, LOSA_ERR_BOUNDS);
      // no records to merge but those of the segments that have pages, which the CTAs that begin them write
      for (int r = (pages > 0 ? (rows + R - 1) / R : 0) + tid; r < p.n_rg; r += blockDim.x) p.seg_records[sk * p.n_rg + r] = make_int2(0, 0);
      if (pages > 0) continue;
      for (int i = tid; i < rows * (D / 4); i += blockDim.x) {       // empty sums
        const int r = i / (D / 4);
        const long long row = i4_row(p, s, kh, r);
        if (row >= 0) i4_store4(p, row * D + (i % (D / 4)) * 4, 0.f, 0.f, 0.f, 0.f);
        if (row >= 0 && p.lse && i % (D / 4) == 0) p.lse[row] = -INFINITY;
      }
    }
    if (static_cast<int>(blockIdx.x) >= n_share) return false;
    lo = cta_lo(T, blockIdx.x, n_share);
    hi = cta_lo(T, blockIdx.x + 1, n_share);
    if (lo >= hi) return false;
    int a = 0, b = p.n_sk;                           // pre[a] <= lo < pre[b]
    while (b - a > 1) {
      const int m = (a + b) >> 1;
      if (pre[m] <= lo) a = m; else b = m;
    }
    sk0 = a;
    return true;
  }
  // the piece at position item, whose (sequence, KV head) is `from` or one after it
  __device__ __forceinline__ I4Piece piece_at(int item, int from) const {
    I4Piece x;
    x.sk = from;
    while (pre[x.sk + 1] <= item) ++x.sk;
    x.s = x.sk / p.Hkv;
    x.kh = x.sk - x.s * p.Hkv;
    const int groups = p.n_rg == 1 ? 1 : (rows_of(x.s) + R - 1) / R, all = pre[x.sk + 1] - pre[x.sk], length = groups == 1 ? all : all / groups;
    x.rg = groups == 1 ? 0 : (item - pre[x.sk]) / length;
    x.seg_lo = pre[x.sk] + x.rg * length;
    x.pages = length - p.pad;
    x.hi = min(hi, x.seg_lo + length);
    x.first_page = max(0, item - x.seg_lo - p.pad);
    x.n_units = (max(0, x.hi - x.seg_lo - p.pad) - x.first_page) << upp_log;
    return x;
  }
  // the next one that has pages, or an empty one at the end
  __device__ __forceinline__ I4Piece next_piece(int item, int from) const {
    I4Piece x{};
    x.hi = hi;
    while (item < hi) {
      x = piece_at(item, from);
      if (x.n_units > 0) break;
      item = x.hi;
      from = x.sk;
    }
    return x;
  }
  // first CTA and number of the records of a segment that several CTAs share
  __device__ __forceinline__ int2 records(const I4Piece& x) const {
    return segment_records(T, n_share, x.seg_lo + p.pad, x.seg_lo + p.pad + x.pages);
  }
};

// Physical page of entry `page` of a piece's list and its valid tokens from token t0 on, at most `most` of them (0: none).
__device__ __forceinline__ int2 i4_resolve(const I4Params& p, const I4Piece& x, int entry, int t0, int most) {
  const int page = p.union_pages ? p.union_pages[static_cast<size_t>(x.sk) * p.Pmax + entry] : entry;
  int at = -1, left = 0;
  if (page >= 0 && page < p.Pmax) {
    at = p.page_table[static_cast<size_t>(x.s) * p.Pmax + page];
    left = p.kv_len[x.s] - page * p.g;
  }
  if (at < 0 || at >= p.n_phys || left <= 0) {
    set_status(p.status, LOSA_ERR_BOUNDS);
    return make_int2(0, 0);
  }
  return make_int2(at, min(most, max(0, left - t0)));
}

// Segments that several CTAs share: a warp per row merges their records by log-sum-exp, in CTA order.
constexpr int kI4CombineWarps = 4;
template <int D, int R, bool BY_SEGMENT>
__global__ void __launch_bounds__(kI4CombineWarps * 32) int4_combine_kernel(const __grid_constant__ I4Params p) {
  grid_dep_wait();
  const int lane = threadIdx.x & 31, w = blockIdx.x * kI4CombineWarps + (threadIdx.x >> 5);
  const int seg = w / R, r = w % R;
  if (seg >= p.n_sk * p.n_rg) return;
  const int2 rec = p.seg_records[seg];
  if (rec.y == 0) return;
  const int sk = seg / p.n_rg, rg = seg - sk * p.n_rg, s = sk / p.Hkv, kh = sk - s * p.Hkv;
  if (rg * R + r >= (p.n_active ? clamp_rows(p.n_active[s], p.B) : p.B) * p.G) return;
  constexpr size_t kRecord = static_cast<size_t>(R) * (D + 2);
  constexpr int C = D / 32, kBatch = 8;
  // records of the CTAs one after the other, at CTA + segment; or two places per CTA, the first CTA's record in its second one, the
  // others' in their first
  const float* first = p.partials + (BY_SEGMENT ? static_cast<size_t>(rec.x + seg) : static_cast<size_t>(rec.x) * 2) * kRecord;
  float acc[C], M = -INFINITY, L = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c) acc[c] = 0.f;
  for (int b = 0; b < rec.y; b += kBatch) {
    float m[kBatch], l[kBatch], x[kBatch][C];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int j = b + i;
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c) x[i][c] = 0.f;
      if (j < rec.y) {
        const float* at = first + (BY_SEGMENT ? j : 2 * j + (j == 0 ? 1 : 0)) * kRecord;
        m[i] = at[r];
        l[i] = at[R + r];
        if constexpr (C == 4) {
          const float4 t = *reinterpret_cast<const float4*>(at + 2 * R + r * D + lane * 4);
          x[i][0] = t.x; x[i][1] = t.y; x[i][2] = t.z; x[i][3] = t.w;
        } else {
          const float2 t = *reinterpret_cast<const float2*>(at + 2 * R + r * D + lane * 2);
          x[i][0] = t.x; x[i][1] = t.y;
        }
      }
    }
    float top = M;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) top = fmaxf(top, m[i]);
    if (top == -INFINITY) {                          // no record with a reference so far: their sums are zero, or no number, which stays visible
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
      for (int c = 0; c < C; ++c) acc[c] = fmaf(x[i][c], f, acc[c]);
    }
    M = top;
  }
  const long long row = i4_row(p, s, kh, rg * R + r);
  if (row < 0) return;
  const bool empty = L == 0.f;
  const float inv = empty ? 0.f : 4.f / L;
  if constexpr (C == 4) {
    i4_store4(p, row * D + lane * 4, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
  } else {
    // two columns a lane: pairs of lanes store four
    const float o0 = __shfl_down_sync(0xffffffffu, acc[0], 1), o1 = __shfl_down_sync(0xffffffffu, acc[1], 1);
    if ((lane & 1) == 0) i4_store4(p, row * D + lane * 2, acc[0] * inv, acc[1] * inv, o0 * inv, o1 * inv);
  }
  if (lane == 0 && p.lse) p.lse[row] = empty ? -INFINITY : (M + log2f(L)) * kLn2;
}

#include "int4_attn_mma.cuh"
#include "int4_attn_tc.cuh"

// ===================================================================== host side
constexpr int kI4SmemLimit = 232448;
// Stage 4 is timed from its first main kernel's start to its last one's end (two where the number of rows is known on the device only).
bool i4_times(const losa_ctx* c, const I4Params& p) { return c->profile && p.n_active; }

template <int D, int NT>
int mma_smem(int warps, int stages, int ut, int n_sk) {
  return 1024 + warps * (stages * (i4_unit_codes<D>(ut) + i4_unit_scales<D>(ut) + 4) + 8 * NT * D * 2) + i4_merge_bytes<D, NT>(warps) + (32 + n_sk + 1) * 4;
}

template <int D, int NT, int UT>
int32_t launch_mma(losa_ctx* c, I4Params p, int max_rows, cudaStream_t st) {
  constexpr int R = 8 * NT;
  auto kernel = int4_mma_kernel<D, NT, UT>;
  const int bit = NT;        // a context has one head dimension and one page size
  if (!(c->int4_attr_set & bit)) {
    LOSA_CUDA_TRY(c, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kI4SmemLimit));
    c->int4_attr_set |= bit;
  }
  p.n_rg = (max_rows + R - 1) / R;
  // Few segments: one CTA of all warps per SM.  More segments than SMs: CTAs of four warps, whose ends and starts overlap.  One token each,
  // large and small CTAs: 8 segments of 8,192 tokens 14.2 and 15.6 us, 64 of 32,768 76.6 and 76.7, 496 of up to 4,095 67.8 and 62.8.
  // The pads are pages that a CTA reads in the time that entering a segment takes; 12 instead of 24 for the large CTAs: 94.9 instead of 67.8.
  const bool many = p.n_sk * p.n_rg > c->n_sms;
  const int W = many ? 4 : i4_warps(NT), per_sm = many ? i4_warps(NT) / 4 : 1;
  p.pad = many ? 10 : 24;
  int grid = c->n_sms * per_sm;
  grid = std::min<long long>(grid, static_cast<long long>(c->lay.n_slots) * kRowsPerGroup / (2 * R));      // room for the records
  if (i4_times(c, p) && p.rows_above == 0) LOSA_CUDA_TRY(c, cudaEventRecord(c->ev_begin, st));
  launch_k(kernel, grid, W * 32, mma_smem<D, NT>(W, kI4Ring, UT, p.n_sk), st, p);
  if (i4_times(c, p) && p.rows_upto >= p.B * p.G) LOSA_CUDA_TRY(c, cudaEventRecord(c->ev_end, st));
  const int32_t rc = after_launch(c);
  if (rc != LOSA_OK) return rc;
  launch_k(int4_combine_kernel<D, R, false>, (p.n_sk * p.n_rg * R + kI4CombineWarps - 1) / kI4CombineWarps, kI4CombineWarps * 32, 0, st, p);
  return after_launch(c);
}

template <int D, int GP>
int32_t launch_tc(losa_ctx* c, I4Params p, cudaStream_t st) {
  auto kernel = int4_tc_kernel<D, GP>;
  if (!(c->int4_attr_set & 4)) {
    LOSA_CUDA_TRY(c, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kI4SmemLimit));
    // the kernel moves registers between its warps: a build that is launched with fewer than it deals out would wait for ever
    cudaFuncAttributes fa;
    LOSA_CUDA_TRY(c, cudaFuncGetAttributes(&fa, kernel));
    if (fa.numRegs < kTcLaunchRegs) return LOSA_ERR_UNSUPPORTED;
    c->int4_attr_set |= 4;
  }
  static_assert(tc_smem<D>(kMaxSegments) <= kI4SmemLimit, "shared memory");
  p.n_rg = c->lay.n_row_groups;
  p.pad = 4 * (kTcTok / GP);                         // four groups' time
  if (i4_times(c, p) && p.rows_above == 0) LOSA_CUDA_TRY(c, cudaEventRecord(c->ev_begin, st));
  launch_k(kernel, c->lay.n_ctas, kTcWarps * 32, tc_smem<D>(p.n_sk), st, p);
  if (i4_times(c, p) && p.rows_upto >= p.B * p.G) LOSA_CUDA_TRY(c, cudaEventRecord(c->ev_end, st));
  const int32_t rc = after_launch(c);
  if (rc != LOSA_OK) return rc;
  launch_k(int4_combine_kernel<D, kTcRows, true>, (p.n_sk * p.n_rg * kTcRows + kI4CombineWarps - 1) / kI4CombineWarps, kI4CombineWarps * 32, 0, st, p);
  return after_launch(c);
}

// Up to 16 rows the kernel on registers is the faster one, whose time grows with every pass of 16 rows; the other's does not depend on the
// rows.  Registers and tensor memory, 16 rows: eight prompts of 32,768 tokens 104 and 175 us, four of 16K to 32K 52 and 78, 64 of
// about 1,400 81 and 93, one of 8,201 18.1 and 18.6.  32 rows: 194 and 175, 90 and 78, 164 and 94, 21.0 and 20.3.
constexpr int kI4MmaRows = 16;
template <int D, int GP>
int32_t launch_rows(losa_ctx* c, I4Params p, cudaStream_t st) {
  constexpr int UT = GP < 32 ? GP : 32;
  const int most = p.B * p.G;
  p.rows_above = 0;
  p.rows_upto = most;
  if (most <= 8) return launch_mma<D, 1, UT>(c, p, most, st);
  if (most <= kI4MmaRows) return launch_mma<D, 2, UT>(c, p, most, st);
  if (p.n_active) {                                  // how many rows there are is known on the device only: each kernel takes its segments
    p.rows_upto = kI4MmaRows;
    const int32_t rc = launch_mma<D, 2, UT>(c, p, kI4MmaRows, st);
    if (rc != LOSA_OK) return rc;
    p.rows_above = kI4MmaRows;
    p.rows_upto = most;
  }
  return launch_tc<D, GP>(c, p, st);
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
  p.wait_cycles = c->wait_cycles > 0 ? c->wait_cycles : kWaitCycles;
  auto with_page = [&](auto d) {
    constexpr int D = decltype(d)::value;
    return sh.page_size == 16 ? launch_rows<D, 16>(c, p, st) : sh.page_size == 32 ? launch_rows<D, 32>(c, p, st) : launch_rows<D, 64>(c, p, st);
  };
  return sh.head_dim == 128 ? with_page(std::integral_constant<int, 128>{}) : with_page(std::integral_constant<int, 64>{});
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
