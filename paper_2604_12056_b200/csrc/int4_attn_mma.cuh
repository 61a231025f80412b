// Attention over 4-bit pages, up to 16 query rows per pass: included by int4_attn.cu (same namespace).
//
// The cache's bytes bound this kernel (68 per row of 128), and right behind them the instructions that turn codes into
// operands.  So tokens, not query rows, are the M side of every product, codes become operands in registers, and
// nothing but codes passes through shared memory:
//   S^T[16 tokens x 8 rows] += K[16 x 16 d] Q^T[16 d x 8]     mma.sync.m16n8k16, A = keys: a lane takes the quarter
//                                (d/4 elements, 16 bytes at d = 128) of two rows that lies in one piece; which elements the
//                                instruction thinks they are does not matter, Q's fragments are laid out the same way
//   O^T[16 d x 8 rows]      += V^T[16 d x 16 tokens] P^T      A = values: a half2 is one element of two tokens, which two
//                                byte permutes put together from the words of the two rows; P^T is S^T, transposed 8 x 8 by movmatrix
// A word of eight codes becomes four half2 operands with their scale in ten instructions: two shifts, and
// for each half2 one LOP3 ((x & mask) | 0x6400: 1024 + 4u or 1024 + 64u as fp16) and one HFMA2 whose result,
// scale * (u - 8) / 4, is exact: scales have four significant bits, so the addends 66 scale and 6 scale have ten and six.
// (The quarter keeps 66 scale below fp16's end for scales up to 960; the softmax scale and the end result take it back.)
//
// Warps take units of up to 32 tokens in turn, each through a ring of its own that it fills by asynchronous copies, 16 bytes per lane: no
// barrier, and no instruction that one lane executes for the others (tensor copies, issued by one lane of each warp or by a warp
// for all rings, cost 90 instructions a unit or kept the rings in step).  The rings run on over the pieces of a
// share.  A warp keeps its own maximum, sum and output; the reference maximum only moves when it
// would grow by more than 2^8, which one vote per unit finds out.  At the end of a piece the warps of the CTA
// merge through shared memory; what CTAs leave of a segment that several of them share is merged by a kernel of its own, whose
// start overlaps this one's end (merging by the last CTA to arrive, behind a ticket, took 5 us of its own at the end of the longest share).
#pragma once

constexpr float kI4Tau = 8.f;                       // log2 units
constexpr float kI4None = -3e38f;                   // a reference before the first score
constexpr int i4_warps(int nt) { return nt == 1 ? 12 : 8; }     // most warps of an SM: 168, 255 registers a thread

template <int D> constexpr int i4_unit_codes(int ut) { return ut * D; }          // bytes of a unit's codes, K and V
template <int D> constexpr int i4_unit_scales(int ut) { return ut * D / 16; }    // ... and scales
template <int D, int NT> constexpr int i4_merge_bytes(int warps) { return ((warps * 8 * NT * (D + 4) * 4 + warps * 8 * NT * 8) + 15) / 16 * 16; }
constexpr int kI4Stride = 4;                        // floats between the rows of the merge tile: a row is D + 4

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
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t movmatrix(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) { uint32_t v; asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a)); return v; }
__device__ __forceinline__ uint32_t lds8(uint32_t a) { uint32_t v; asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a)); return v; }
__device__ __forceinline__ uint2 lds64(uint32_t a) { uint2 v; asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a)); return v; }
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}

// Which token of a run of 16 is row r (0..7) of the MMA's M side; row r + 8 is eight tokens on.  With these orders a quarter warp's 16-byte
// (d = 64: half warp's 8-byte) reads of K rows and a half warp's reads of V rows meet all banks: rows of 64 bytes lie under the copy's
// 64-byte swizzle, rows of 32 bytes as they are.
template <int D> __device__ __forceinline__ int i4_token(int r) {
  return static_cast<int>(((D == 128 ? 0x65742130u : 0x53427160u) >> (4 * r)) & 15u);
}

__device__ __forceinline__ void i4_copy16(uint32_t dst, const uint8_t* src, unsigned long long policy) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(policy) : "memory");
}
__device__ __forceinline__ void i4_copy4(uint32_t dst, const uint8_t* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

// UT: tokens of a unit, S: units of a ring
template <int D, int NT, int UT, int S>
__global__ void __launch_bounds__(i4_warps(NT) * 32, 1)
int4_mma_kernel(const __grid_constant__ I4Params p) {
  constexpr int R = 8 * NT, KS = D / 16, MT = D / 16, E = D / 8, WL = D / 32, RUNS = D / kInt4Run;
  constexpr int UC = i4_unit_codes<D>(UT), US = i4_unit_scales<D>(UT), SUBS = UT / 16;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, W = blockDim.x >> 5;
  const int gid = lane >> 2, tig = lane & 3;
  // layout: rings of codes, rings of scales, queries of a piece per warp, merge tile [W][R][D + 4] and [W][R] maxima and sums, valid
  // counts, sums of the prefix's runs, charged prefix
  const uint32_t codes0 = base + warp * S * UC, scales0 = base + W * S * UC + warp * S * US;
  const uint32_t q0 = base + W * S * (UC + US) + warp * (R * D * 2);
  float* merge_o = reinterpret_cast<float*>(gen + W * (S * (UC + US) + R * D * 2));
  float* merge_ml = merge_o + W * R * (D + kI4Stride);
  uint8_t* tail = gen + W * (S * (UC + US) + R * D * 2) + i4_merge_bytes<D, NT>(W);
  int* valid_s = reinterpret_cast<int*>(tail) + warp * S;
  int* chunk_s = reinterpret_cast<int*>(tail + W * S * 4);       // [32]
  int* pre = chunk_s + 32;

  grid_dep_trigger();                                // (the merging kernel comes up beside this one)
  grid_dep_wait();
  auto rows_of = [&](int s) { return (p.n_active ? clamp_rows(p.n_active[s], p.B) : p.B) * p.G; };
  auto pages_in = [&](int sk) {                      // pages of a segment
    const int s = sk / p.Hkv;
    if (p.union_count) return min(max(p.union_count[sk], 0), p.Pmax);
    return min(max((p.kv_len[s] + p.g - 1) / p.g, 0), p.Pmax);
  };
  // prefix of the segments' lengths, `pad` pages added to each: runs of 32 by the warps, then the runs' sums
  const int n_runs = (p.n_sk + 31) >> 5;
  for (int b = warp; b < n_runs; b += W) {
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
    if (lane == 31) chunk_s[b] = inc;
  }
  __syncthreads();
  if (warp == 0) {
    const int c = lane < n_runs ? chunk_s[lane] : 0;
    int inc = c;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += t;
    }
    chunk_s[lane] = inc - c;
    if (lane == 31) pre[p.n_sk] = inc;
  }
  __syncthreads();
  for (int i = 32 + tid; i < p.n_sk; i += blockDim.x) pre[i] += chunk_s[i >> 5];
  __syncthreads();
  const int T = pre[p.n_sk], upp = p.g / UT, upp_log = upp == 2 ? 1 : 0;    // units per page: one or two
  // no more shares than give every warp min_units units
  const int n_share = max(1, min(static_cast<int>(gridDim.x), (T * upp + W * p.min_units - 1) / (W * p.min_units)));
  // rows without any page: empty sums
  for (int sk = blockIdx.x; sk < p.n_sk; sk += gridDim.x) {
    const int s = sk / p.Hkv, kh = sk - s * p.Hkv;
    if (!p.union_count && kh == 0 && tid == 0 && (p.kv_len[s] + p.g - 1) / p.g > p.Pmax) set_status(p.status, LOSA_ERR_BOUNDS);
    const int rows = rows_of(s);
    if (pages_in(sk) > 0 && rows > 0) {
      for (int r = (rows + R - 1) / R + tid; r < p.n_rg; r += blockDim.x) p.seg_records[sk * p.n_rg + r] = make_int2(0, 0);
      continue;
    }
    for (int r = tid; r < p.n_rg; r += blockDim.x) p.seg_records[sk * p.n_rg + r] = make_int2(0, 0);
    for (int i = tid; i < rows * (D / 4); i += blockDim.x) {
      const int r = i / (D / 4);
      const long long row = i4_row(p, s, kh, r);
      if (row >= 0) i4_store4(p, row * D + (i % (D / 4)) * 4, 0.f, 0.f, 0.f, 0.f);
      if (row >= 0 && p.lse && i % (D / 4) == 0) p.lse[row] = -INFINITY;
    }
  }
  if (static_cast<int>(blockIdx.x) >= n_share) return;
  const int lo = cta_lo(T, blockIdx.x, n_share), hi = cta_lo(T, blockIdx.x + 1, n_share);
  if (lo >= hi) return;
  int sk0 = 0;
  {
    int a = 0, b = p.n_sk;                           // pre[a] <= lo < pre[b]
    while (b - a > 1) {
      const int m = (a + b) >> 1;
      if (pre[m] <= lo) a = m; else b = m;
    }
    sk0 = a;
  }
  // the pieces of the share: runs of pages of one (sequence, KV head, row group).  Every such segment begins with `pad` positions
  // that stand for no page: entering one costs a CTA about as much as that many pages
  struct Piece { int s, kh, rg, sk, seg_lo, pages, hi, first_page, n_units; };
  auto piece_at = [&](int item, int from) {          // the piece at position item, whose segment is `from` or one after it
    Piece x;
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
  };
  auto next_piece = [&](int item, int from) {        // the next one that has pages, or an empty one at the end
    Piece x{};
    x.hi = hi;
    while (item < hi) {
      x = piece_at(item, from);
      if (x.n_units > 0) break;
      item = x.hi;
      from = x.sk;
    }
    return x;
  };

  // ---- the ring: units warp, warp + W, ... of every piece, one piece after the other; the copies run S - 1 units ahead
  unsigned long long policy;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
  constexpr int RB = D / 2, LPR = RB / 16, RPI = 32 / LPR, SL = US / 8;  // bytes of a row, lanes per row, rows per copy, lanes per copy of scales
  auto swz = [](int t, int chunk) { return D == 128 ? (chunk ^ ((t >> 1) & 3)) << 4 : chunk << 4; };   // (the same eight rows further on)
  const int64_t copy_src = static_cast<int64_t>(lane / LPR) * p.stride_tok + (lane % LPR) * 16;
  const uint32_t copy_dst = codes0 + (lane / LPR) * RB + swz(lane / LPR, lane % LPR), scale_dst = scales0 + lane * 4;
  Piece ahead = next_piece(lo, sk0), piece = ahead;
  int ahead_k = 0;                                   // the next unit to be copied: number ahead_k of this warp in its piece
  // queries of a piece, as they lie, into this warp's tile: with the next unit's copies
  auto copy_queries = [&](const Piece& x) {
    const int rows = rows_of(x.s) - x.rg * R;
#pragma unroll
    for (int i = 0; i < R * (D / 8) / 32; ++i) {
      const int r = (i * 32 + lane) / (D / 8), c = (i * 32 + lane) % (D / 8);
      const long long row = r < rows ? i4_row(p, x.s, x.kh, x.rg * R + r) : -1;
      const uint32_t at = q0 + r * (D * 2) + ((c ^ (r & 7)) << 4);
      if (row >= 0) i4_copy16(at, reinterpret_cast<const uint8_t*>(p.q + row * D + c * 8), policy);
      else asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0) : "memory");
    }
  };
  if (piece.n_units > 0) copy_queries(piece);
  int b_phys = 0, b_valid = 0;                       // physical pages and valid tokens of 32 of them, one per lane
  auto issue = [&](int ahead_slot) {                 // into this slot
    while (warp + W * ahead_k >= ahead.n_units && ahead.hi < hi) {
      ahead = next_piece(ahead.hi, ahead.sk);
      ahead_k = 0;
    }
    if (warp + W * ahead_k < ahead.n_units) {
      if ((ahead_k & 31) == 0) {
        const int u = warp + W * (ahead_k + lane);
        b_phys = 0;
        b_valid = 0;
        if (u < ahead.n_units) {
          const int pg = ahead.first_page + (u >> upp_log);
          const int page = p.union_pages ? p.union_pages[static_cast<size_t>(ahead.sk) * p.Pmax + pg] : pg;
          int at = -1, left = 0;
          if (page >= 0 && page < p.Pmax) {
            at = p.page_table[static_cast<size_t>(ahead.s) * p.Pmax + page];
            left = p.kv_len[ahead.s] - page * p.g;
          }
          if (at < 0 || at >= p.n_phys || left <= 0) {
            set_status(p.status, LOSA_ERR_BOUNDS);
          } else {
            b_phys = at;
            b_valid = min(UT, max(0, left - (u & (upp - 1)) * UT));
          }
        }
      }
      const int phys = __shfl_sync(0xffffffffu, b_phys, ahead_k & 31), valid = __shfl_sync(0xffffffffu, b_valid, ahead_k & 31);
      const int t0 = ((warp + W * ahead_k) & (upp - 1)) * UT;
      if (lane == 0) valid_s[ahead_slot] = valid;
      const int64_t src = phys * p.stride_page + ahead.kh * p.stride_head + t0 * p.stride_tok + copy_src;
      const uint8_t *ksrc = p.k_pages + src, *vsrc = p.v_pages + src;
      const uint32_t dst = copy_dst + ahead_slot * UC, dsc = scale_dst + ahead_slot * US;
      if (p.stride_tok == RB) {                        // rows one after the other: offsets known at compile time
#pragma unroll
        for (int j = 0; j < UT / RPI; ++j) {
          i4_copy16(dst + j * RPI * RB, ksrc + j * RPI * RB, policy);
          i4_copy16(dst + UC / 2 + j * RPI * RB, vsrc + j * RPI * RB, policy);
        }
      } else {
#pragma unroll
        for (int j = 0; j < UT / RPI; ++j) {
          i4_copy16(dst + j * RPI * RB, ksrc, policy);
          i4_copy16(dst + UC / 2 + j * RPI * RB, vsrc, policy);
          ksrc += RPI * p.stride_tok;
          vsrc += RPI * p.stride_tok;
        }
      }
      const int64_t at = ((static_cast<int64_t>(phys) * p.Hkv + ahead.kh) * p.g + t0) * RUNS + lane * 4;
      if (SL == 32 || lane < SL) {
        i4_copy4(dsc, p.k_scale + at);
        i4_copy4(dsc + US / 2, p.v_scale + at);
      }
      ++ahead_k;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");           // (empty where there is nothing left: the groups count units)
  };
#pragma unroll
  for (int i = 0; i < S - 1; ++i) issue(i);

  int next_slot = 0;                                 // of the next unit to be taken
  const int row_a = i4_token<D>(gid);                // tokens of this lane's K rows: row_a, row_a + 8
  const int row_v0 = i4_token<D>(2 * tig), row_v1 = i4_token<D>(2 * tig + 1);
  // where they lie in a unit
  const uint32_t at_k = codes0 + row_a * RB + (D == 128 ? swz(row_a, tig) : tig * 8);
  const uint32_t at_v0 = codes0 + UC / 2 + row_v0 * RB + (D == 128 ? swz(row_v0, gid >> 1) + (gid & 1) * 8 : gid * 4);
  const uint32_t at_v1 = codes0 + UC / 2 + row_v1 * RB + (D == 128 ? swz(row_v1, gid >> 1) + (gid & 1) * 8 : gid * 4);
  const uint32_t at_ks = scales0 + row_a * RUNS + (D == 128 ? tig : tig >> 1);
  const uint32_t at_vs0 = scales0 + US / 2 + row_v0 * RUNS + (D == 128 ? gid >> 1 : gid >> 2), at_vs1 = scales0 + US / 2 + row_v1 * RUNS + (D == 128 ? gid >> 1 : gid >> 2);

  while (piece.n_units > 0) {
    const int s = piece.s, kh = piece.kh, rg = piece.rg, rows = rows_of(s), n_units = piece.n_units;
    const int mine = n_units > warp ? (n_units - warp + W - 1) / W : 0;      // units warp, warp + W, ...

    // ---- queries: fp16 under a power of two of the row
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncwarp();
    uint32_t qf[NT][KS][2];
    float sc[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float x[D / 4];
      float amax = 0.f;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        float t[8];
        const int c = tig * (D / 32) + i, r = nt * 8 + gid;
        const uint4 raw4 = lds128(q0 + r * (D * 2) + ((c ^ (r & 7)) << 4));
        load8(reinterpret_cast<const __nv_bfloat16*>(&raw4), t);
#pragma unroll
        for (int e = 0; e < 8; ++e) { x[i * 8 + e] = t[e]; amax = fmaxf(amax, fabsf(t[e])); }
      }
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
      // the row's largest element comes to 2^14 .. 2^15
      const int e = max(-100, min(127, static_cast<int>(__float_as_uint(amax) >> 23) - 127));
      const float up = __int_as_float((127 + 14 - e) << 23), down = __int_as_float((127 - 14 + e) << 23) * (4.f * p.sm_scale * kLog2e);
#pragma unroll
      for (int w = 0; w < WL; ++w) {
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const __half2 t = __floats2half2_rn(x[w * 8 + i] * up, x[w * 8 + i + 4] * up);
          h[i] = *reinterpret_cast<const uint32_t*>(&t);
        }
        qf[nt][2 * w][0] = h[0]; qf[nt][2 * w][1] = h[1];
        qf[nt][2 * w + 1][0] = h[2]; qf[nt][2 * w + 1][1] = h[3];
      }
      sc[nt][0] = __shfl_sync(0xffffffffu, down, 8 * tig);
      sc[nt][1] = __shfl_sync(0xffffffffu, down, 8 * tig + 4);
    }

    __syncwarp();
    const Piece following = next_piece(piece.hi, piece.sk);
    if (following.n_units > 0) copy_queries(following);
    asm volatile("cp.async.commit_group;" ::: "memory");           // (older than the next unit's group: waited for with the unit before that)

    float o[NT][MT][4], m[NT][2], l[NT][2], tau[NT][2];      // m: in units of the scores as they are; a difference times sc is in log2 units
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      m[nt][0] = m[nt][1] = kI4None;
      l[nt][0] = l[nt][1] = 0.f;
      tau[nt][0] = kI4Tau / sc[nt][0];
      tau[nt][1] = kI4Tau / sc[nt][1];
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[nt][i][c] = 0.f;
    }

    const int next_slot_was = next_slot;
    auto take = [&](auto slot_c) {
      constexpr int slot = decltype(slot_c)::value;
      issue((slot + S - 1) % S);                     // into the slot that was read last
      asm volatile("cp.async.wait_group %0;" ::"n"(S - 1) : "memory");
      __syncwarp();
      const int valid = valid_s[slot];
      const uint32_t ck = at_k + slot * UC, cv0 = at_v0 + slot * UC, cv1 = at_v1 + slot * UC;
      const uint32_t ks = at_ks + slot * US, vs0 = at_vs0 + slot * US, vs1 = at_vs1 + slot * US;
      if (valid > 0) {
        float sT[SUBS][NT][4];
#pragma unroll
        for (int b = 0; b < SUBS; ++b) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 4; ++c) sT[b][nt][c] = 0.f;
          uint32_t x0[WL], x1[WL];
          if constexpr (D == 128) {
            const uint4 a0 = lds128(ck + b * 16 * RB), a1 = lds128(ck + (b * 16 + 8) * RB);
            x0[0] = a0.x; x0[1] = a0.y; x0[2] = a0.z; x0[3] = a0.w;
            x1[0] = a1.x; x1[1] = a1.y; x1[2] = a1.z; x1[3] = a1.w;
          } else {
            const uint2 a0 = lds64(ck + b * 16 * RB), a1 = lds64(ck + (b * 16 + 8) * RB);
            x0[0] = a0.x; x0[1] = a0.y;
            x1[0] = a1.x; x1[1] = a1.y;
          }
          const I4Scale s0 = i4_scale(lds8(ks + b * 16 * RUNS) * 0x00800080u), s1 = i4_scale(lds8(ks + (b * 16 + 8) * RUNS) * 0x00800080u);
#pragma unroll
          for (int w = 0; w < WL; ++w) {
            uint32_t h0[4], h1[4];
            i4_operands(x0[w], s0, h0);
            i4_operands(x1[w], s1, h1);
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                mma_f16(sT[b][nt], h0[2 * half], h1[2 * half], h0[2 * half + 1], h1[2 * half + 1], qf[nt][2 * w + half][0], qf[nt][2 * w + half][1]);
              }
          }
        }
        // tokens past the end drop out; scores times sc are in log2 units
        bool grow = false;
        if (valid < UT) {
#pragma unroll
          for (int b = 0; b < SUBS; ++b)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int c = 0; c < 4; ++c)
                if (b * 16 + row_a + (c >> 1) * 8 >= valid) sT[b][nt][c] = -INFINITY;
        }
        float top[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float t = fmaxf(sT[0][nt][c], sT[0][nt][c + 2]);
#pragma unroll
            for (int b = 1; b < SUBS; ++b) t = fmaxf(t, fmaxf(sT[b][nt][c], sT[b][nt][c + 2]));
            top[nt][c] = t;
            grow |= t - m[nt][c] > tau[nt][c];
          }
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              float t = top[nt][c];
#pragma unroll
              for (int x = 4; x < 32; x <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, x));
              const float mn = fmaxf(m[nt][c], t), f = exp2f((m[nt][c] - mn) * sc[nt][c]);
              m[nt][c] = mn;
              l[nt][c] *= f;
#pragma unroll
              for (int i = 0; i < MT; ++i) { o[nt][i][c] *= f; o[nt][i][c + 2] *= f; }
            }
        }
        uint32_t pf[SUBS][NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int b = 0; b < SUBS; ++b) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const float e = i4_ex2((sT[b][nt][c] - m[nt][c & 1]) * sc[nt][c & 1]);
              sT[b][nt][c] = e;
              l[nt][c & 1] += e;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const __half2 t = __floats2half2_rn(sT[b][nt][2 * h], sT[b][nt][2 * h + 1]);
              pf[b][nt][h] = movmatrix(*reinterpret_cast<const uint32_t*>(&t));
            }
          }
        }
#pragma unroll
        for (int b = 0; b < SUBS; ++b) {
          // values of four tokens (two pairs), E elements each
          uint32_t v[4][E / 8], byte[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int t = b * 16 + (i >> 1) * 8;
            if constexpr (D == 128) {
              const uint2 x = lds64((i & 1 ? cv1 : cv0) + t * RB);
              v[i][0] = x.x; v[i][1] = x.y;
            } else {
              v[i][0] = lds32((i & 1 ? cv1 : cv0) + t * RB);
            }
            byte[i] = lds8((i & 1 ? vs1 : vs0) + t * RUNS);
          }
          if (valid < UT) {                          // whatever lies past the end: codes are finite, scales may be anything
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (b * 16 + (i >> 1) * 8 + (i & 1 ? row_v1 : row_v0) >= valid) byte[i] = 0;
          }
          const I4Scale s0 = i4_scale(byte[0] * 0x80u + byte[1] * 0x800000u), s1 = i4_scale(byte[2] * 0x80u + byte[3] * 0x800000u);
#pragma unroll
          for (int w = 0; w < E / 8; ++w)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const uint32_t sel = half ? 0x7632u : 0x5410u;
              uint32_t h0[4], h1[4];
              i4_operands(__byte_perm(v[0][w], v[1][w], sel), s0, h0);
              i4_operands(__byte_perm(v[2][w], v[3][w], sel), s1, h1);
#pragma unroll
              for (int pr = 0; pr < 2; ++pr)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
                  mma_f16(o[nt][w * 4 + half * 2 + pr], h0[2 * pr], h0[2 * pr + 1], h1[2 * pr], h1[2 * pr + 1], pf[b][nt][0], pf[b][nt][1]);
            }
        }
      }
      __syncwarp();                                  // the slot has been read
    };
    // slots in turn, known at compile time: addresses are then one register and an offset
    int k = 0;
    if constexpr (S == 2) {
      if (mine > 0 && next_slot == 1) { take(std::integral_constant<int, 1>{}); ++k; }
#pragma unroll 1
      for (; k + 2 <= mine; k += 2) {
        take(std::integral_constant<int, 0>{});
        take(std::integral_constant<int, 1>{});
      }
      next_slot = 0;
      if (k < mine) { take(std::integral_constant<int, 0>{}); next_slot = 1; }
      if (mine == 0) next_slot = next_slot_was;
    }

    // ---- merge of the CTA's warps
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], x);
        const int r = nt * 8 + 2 * tig + c;
        float* dst = merge_o + (warp * R + r) * (D + kI4Stride) + gid * E;
#pragma unroll
        for (int i = 0; i < MT; i += 2)
          *reinterpret_cast<float4*>(dst + 2 * i) = make_float4(o[nt][i][c], o[nt][i][c + 2], o[nt][i + 1][c], o[nt][i + 1][c + 2]);
        if (gid == 0) {
          merge_ml[(warp * R + r) * 2] = m[nt][c] == kI4None ? -INFINITY : m[nt][c] * sc[nt][c];
          merge_ml[(warp * R + r) * 2 + 1] = l[nt][c];
        }
      }
    }
    __syncthreads();
    const bool first = piece.first_page == 0, whole = first && (n_units >> upp_log) == piece.pages;
    float* record = p.partials + static_cast<size_t>(blockIdx.x * 2 + (first ? 1 : 0)) * R * (D + 2);
    for (int i = tid; i < R * (D / 4); i += blockDim.x) {
      const int r = i / (D / 4), c = (i % (D / 4)) * 4;
      if (rg * R + r >= rows) continue;
      float M = -INFINITY;
      for (int w = 0; w < W; ++w) M = fmaxf(M, merge_ml[(w * R + r) * 2]);
      float L = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int w = 0; w < W; ++w) {
        const float mw = merge_ml[(w * R + r) * 2], f = mw == -INFINITY ? 0.f : exp2f(mw - M);
        const float4 x = *reinterpret_cast<const float4*>(merge_o + (w * R + r) * (D + kI4Stride) + c);
        L += merge_ml[(w * R + r) * 2 + 1] * f;
        acc.x += x.x * f; acc.y += x.y * f; acc.z += x.z * f; acc.w += x.w * f;
      }
      if (whole) {
        i4_finish(p, s, kh, rg * R + r, c, D, acc, M, L);
      } else {
        *reinterpret_cast<float4*>(record + 2 * R + r * D + c) = acc;
        if (c == 0) { record[r] = M; record[R + r] = L; }
      }
    }
    // the CTAs whose shares meet this segment are consecutive; the first of them leaves word for the kernel that merges their records
    if (first && tid == 0)
      p.seg_records[piece.sk * p.n_rg + rg] = whole ? make_int2(0, 0) : segment_records(T, n_share, piece.seg_lo + p.pad, piece.seg_lo + p.pad + piece.pages);
    piece = following;
    if (piece.n_units > 0) __syncthreads();          // the merge tile has been read
  }
}

// Segments that several CTAs share: a warp per row merges their records by log-sum-exp, in CTA order.
constexpr int kI4CombineWarps = 4;
template <int D, int R>
__global__ void __launch_bounds__(kI4CombineWarps * 32) int4_combine_kernel(const __grid_constant__ I4Params p) {
  grid_dep_wait();
  const int lane = threadIdx.x & 31, w = blockIdx.x * kI4CombineWarps + (threadIdx.x >> 5);
  const int seg = w / R, r = w % R;
  if (seg >= p.n_sk * p.n_rg) return;
  const int2 rec = p.seg_records[seg];
  if (rec.y == 0) return;
  const int sk = seg / p.n_rg, rg = seg - sk * p.n_rg, s = sk / p.Hkv, kh = sk - s * p.Hkv;
  if (rg * R + r >= (p.n_active ? clamp_rows(p.n_active[s], p.B) : p.B) * p.G) return;
  constexpr size_t kStep = static_cast<size_t>(2) * R * (D + 2);           // from a CTA's record to the next one's
  constexpr int C = D / 32, kBatch = 8;
  // the first CTA's record lies in its second place, the others' in their first
  const float* first = p.partials + static_cast<size_t>(rec.x) * kStep;
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
        const float* at = first + j * kStep + (j == 0 ? R * (D + 2) : 0);
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
    if (top == -INFINITY) continue;
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
