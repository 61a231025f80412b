// Attention over 4-bit pages, up to 32 query rows per pass: included by int4_attn.cu (same namespace).
//
// The cache's bytes bound this kernel (68 per row of 128), and right behind them the instructions that turn codes into
// operands.  So tokens, not query rows, are the M side of every product, codes become operands in registers, and
// nothing but codes passes through shared memory:
//   S^T[16 tokens x 8 rows] += K[16 x 16 d] Q^T[16 d x 8]     mma.sync.m16n8k16, A = keys: a lane takes the quarter
//                                (d/4 elements, 16 bytes at d = 128) of two rows that lies in one piece; which elements the
//                                instruction thinks they are does not matter, Q's fragments are laid out the same way
//   O^T[16 d x 8 rows]      += V^T[16 d x 16 tokens] P^T      A = values: a half2 is one element of two tokens, which two
//                                byte permutes put together from the words of the two rows; P^T is S^T, transposed 8 x 8 by movmatrix
// A word of eight codes becomes four half2 operands with their scale in ten instructions: two rotations, and
// for each half2 one LOP3 ((x & mask) | 0x6400: 1024 + 4u or 1024 + 64u as fp16) and one HFMA2 whose result,
// scale * (u - 8) / 4, is exact: scales have four significant bits, so the addends 66 scale and 6 scale have ten and six.
// (The quarter keeps 66 scale below fp16's end for scales up to 960; the softmax scale and the end result take it back.)
//
// Warps stream units of up to 32 tokens, each through a ring of its own: one lane issues two tensor copies (codes of K and V) and
// two bulk copies (scales) per unit.  A warp keeps its own maximum, sum and output; the reference maximum only moves when it
// would grow by more than 2^8, which one vote per unit finds out.  At the end of a piece the warps of the CTA
// merge through shared memory, and a segment that several CTAs share is merged by the last of them to arrive (in CTA order, so the
// result does not depend on which one that is).
#pragma once

constexpr float kI4Tau = 8.f;                       // log2 units
constexpr int i4_warps(int nt) { return nt == 1 ? 16 : nt == 2 ? 12 : 8; }     // most warps per CTA: 128, 168, 255 registers a thread
constexpr int kI4Stages = 3;                        // units in flight per warp, at least

template <int D> constexpr int i4_unit_codes(int ut) { return ut * D; }          // bytes of a unit's codes, K and V
template <int D> constexpr int i4_unit_scales(int ut) { return ut * D / 16; }    // ... and scales
template <int D, int NT> constexpr int i4_merge_bytes(int warps) { return warps * 8 * NT * (D + 4) * 4 + warps * 8 * NT * 8; }
constexpr int kI4Stride = 4;                        // floats between the rows of the merge tile: a row is D + 4
constexpr int kI4Head = 128;                        // abort flag, whether this CTA is a segment's last one

__device__ __forceinline__ uint32_t rotl(uint32_t x, int n) { return __funnelshift_l(x, x, n); }
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
  const uint32_t y = rotl(x, 2), z = rotl(y, 24);
  h[0] = fma_h2((y & 0x003c003cu) | 0x64006400u, s.m4, s.a4);
  h[1] = fma_h2((y & 0x03c003c0u) | 0x64006400u, s.m64, s.a64);
  h[2] = fma_h2((z & 0x003c003cu) | 0x64006400u, s.m4, s.a4);
  h[3] = fma_h2((z & 0x03c003c0u) | 0x64006400u, s.m64, s.a64);
}
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t movmatrix(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) { uint32_t v; asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a)); return v; }
__device__ __forceinline__ uint32_t lds8(uint32_t a) { uint32_t v; asm volatile("{\n\t.reg .u8 t;\n\tld.shared.u8 t, [%1];\n\tcvt.u32.u8 %0, t;\n\t}" : "=r"(v) : "r"(a)); return v; }
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

// 16 x 16 x 8 products of one run of 16 tokens; UT: tokens of a unit
template <int D, int NT, int UT>
__global__ void __launch_bounds__(i4_warps(NT) * 32, 1)
int4_mma_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, I4Params p) {
  constexpr int R = 8 * NT, KS = D / 16, MT = D / 16, E = D / 8, WL = D / 32, RUNS = D / kInt4Run;
  constexpr int UC = i4_unit_codes<D>(UT), US = i4_unit_scales<D>(UT), SUBS = UT / 16;
  constexpr bool QS = NT == 4;                       // the queries' fragments in shared memory (else in registers)
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, W = blockDim.x >> 5, S = p.stages;
  const int gid = lane >> 2, tig = lane & 3;
  // layout: rings of codes, rings of scales, barriers, valid counts, head, Q fragments, page prefix
  const uint32_t codes0 = base + warp * S * UC, scales0 = base + W * S * UC + warp * S * US;
  const uint32_t bars0 = base + p.bar_off + warp * S * 8;                 // (bar_off: behind the rings and the merge tile)
  int* valid_s = reinterpret_cast<int*>(gen + p.bar_off + W * S * 8) + warp * S;
  uint8_t* tail = gen + p.bar_off + W * S * (8 + 4);
  tail += (16 - (reinterpret_cast<uintptr_t>(tail) & 15)) & 15;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tail);
  int* last_s = reinterpret_cast<int*>(tail) + 1;
  uint32_t* q_s = reinterpret_cast<uint32_t*>(tail + kI4Head);             // [KS][NT][32 lanes][2]
  int* pre = reinterpret_cast<int*>(tail + kI4Head + (QS ? KS * NT * 32 * 8 : 0));
  float* merge_o = reinterpret_cast<float*>(gen);    // after the rings have been read: [W][R][D + 4], then [W][R] maxima and sums
  float* merge_ml = merge_o + W * R * (D + kI4Stride);

  if (lane == 0) {
    for (int i = 0; i < S; ++i) mbar_init(bars0 + 8 * i, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (tid == 0) *abort_flag = 0;
  grid_dep_wait();
  auto rows_of = [&](int s) { return (p.n_active ? clamp_rows(p.n_active[s], p.B) : p.B) * p.G; };
  auto pages_in = [&](int sk) {                      // pages of a segment
    const int s = sk / p.Hkv;
    if (p.union_count) return min(max(p.union_count[sk], 0), p.Pmax);
    return min(max((p.kv_len[s] + p.g - 1) / p.g, 0), p.Pmax);
  };
  if (warp == 0) {
    int run = 0;
    for (int b = 0; b < p.n_sk; b += 32) {
      const int sk = b + lane;
      int c = 0;
      if (sk < p.n_sk) c = pages_in(sk) * ((rows_of(sk / p.Hkv) + R - 1) / R);
      int inc = c;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
      }
      if (sk < p.n_sk) pre[sk] = run + inc - c;
      run += __shfl_sync(0xffffffffu, inc, 31);
    }
    if (lane == 0) pre[p.n_sk] = run;
  }
  __syncthreads();
  const int T = pre[p.n_sk], upp = p.g / UT;
  // no more shares than give every warp min_units units
  const int n_share = max(1, min(static_cast<int>(gridDim.x), (T * upp + W * p.min_units - 1) / (W * p.min_units)));
  // rows without any page: empty sums
  for (int sk = blockIdx.x; sk < p.n_sk; sk += gridDim.x) {
    const int s = sk / p.Hkv, kh = sk - s * p.Hkv, rows = rows_of(s);
    if (!p.union_count && kh == 0 && tid == 0 && (p.kv_len[s] + p.g - 1) / p.g > p.Pmax) set_status(p.status, LOSA_ERR_BOUNDS);
    if (pages_in(sk) > 0) continue;
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
  int sk = 0;
  {
    int a = 0, b = p.n_sk;                           // pre[a] <= lo < pre[b]
    while (b - a > 1) {
      const int m = (a + b) >> 1;
      if (pre[m] <= lo) a = m; else b = m;
    }
    sk = a;
  }
  unsigned long long policy;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
  uint32_t stage_use = 0;                            // units of this warp so far: stage and parity go on over the pieces
  const int row_a = i4_token<D>(gid);                // tokens of this lane's K rows: row_a, row_a + 8
  const int row_v0 = i4_token<D>(2 * tig), row_v1 = i4_token<D>(2 * tig + 1);

  for (int item = lo; item < hi;) {
    while (pre[sk + 1] <= item) ++sk;
    const int s = sk / p.Hkv, kh = sk - s * p.Hkv, rows = rows_of(s), pages = pages_in(sk);
    const int rg = (item - pre[sk]) / pages, seg_lo = pre[sk] + rg * pages, seg_hi = seg_lo + pages;
    const int piece_hi = min(hi, seg_hi), n_units = (piece_hi - item) * upp, first_page = item - seg_lo;
    const int len = p.kv_len[s];
    const int mine = n_units > warp ? (n_units - warp + W - 1) / W : 0;      // units warp, warp + W, ...

    // ---- physical pages of 32 units at a time, one per lane
    int b_phys = 0, b_valid = 0;
    auto resolve = [&](int k0) {
      const int u = warp + W * (k0 + lane);
      b_phys = 0;
      b_valid = 0;
      if (k0 + lane < mine) {
        const int pg = first_page + u / upp;
        const int page = p.union_pages ? p.union_pages[static_cast<size_t>(sk) * p.Pmax + pg] : pg;
        int phys = -1, left = 0;
        if (page >= 0 && page < p.Pmax) {
          phys = p.page_table[static_cast<size_t>(s) * p.Pmax + page];
          left = len - page * p.g;
        }
        if (phys < 0 || phys >= p.n_phys || left <= 0) {
          set_status(p.status, LOSA_ERR_BOUNDS);
        } else {
          b_phys = phys;
          b_valid = min(UT, max(0, left - (u % upp) * UT));
        }
      }
    };
    auto issue = [&](int k) {                        // unit k of this warp into its ring; all lanes
      if ((k & 31) == 0) resolve(k);
      const int phys = __shfl_sync(0xffffffffu, b_phys, k & 31), valid = __shfl_sync(0xffffffffu, b_valid, k & 31);
      if (lane == 0) {
        const uint32_t st = (stage_use + k) % S, bar = bars0 + 8 * st;
        const int t0 = ((warp + W * k) % upp) * UT;
        valid_s[st] = valid;
        mbar_expect_tx(bar, UC + US);
        const uint32_t ck = codes0 + st * UC, cs = scales0 + st * US;
        i4_tma(ck, &map_k, bar, t0, kh, phys, policy);
        i4_tma(ck + UC / 2, &map_v, bar, t0, kh, phys, policy);
        const size_t at = ((static_cast<size_t>(phys) * p.Hkv + kh) * p.g + t0) * RUNS;
        i4_bulk(cs, p.k_scale + at, bar, US / 2);
        i4_bulk(cs + US / 2, p.v_scale + at, bar, US / 2);
      }
      __syncwarp();
    };
    const int ahead = min(S, mine);
    for (int k = 0; k < ahead; ++k) issue(k);

    // ---- queries: fp16 under a power of two of the row
    uint32_t qf[QS ? 1 : NT][QS ? 1 : KS][2];
    float sc[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = rg * R + nt * 8 + gid;
      const long long row = r < rows ? i4_row(p, s, kh, r) : -1;
      uint4 raw4[D / 32];
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
        raw4[i] = row >= 0 ? *reinterpret_cast<const uint4*>(p.q + row * D + tig * (D / 4) + i * 8) : make_uint4(0u, 0u, 0u, 0u);
      float x[D / 4];
      float amax = 0.f;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        float t[8];
        load8(reinterpret_cast<const __nv_bfloat16*>(&raw4[i]), t);
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
        if constexpr (QS) {
          if (warp == 0) {
            uint2* at = reinterpret_cast<uint2*>(q_s) + (2 * w * NT + nt) * 32 + lane;
            at[0] = make_uint2(h[0], h[1]);
            at[NT * 32] = make_uint2(h[2], h[3]);
          }
        } else {
          qf[nt][2 * w][0] = h[0]; qf[nt][2 * w][1] = h[1];
          qf[nt][2 * w + 1][0] = h[2]; qf[nt][2 * w + 1][1] = h[3];
        }
      }
      sc[nt][0] = __shfl_sync(0xffffffffu, down, 8 * tig);
      sc[nt][1] = __shfl_sync(0xffffffffu, down, 8 * tig + 4);
    }
    if constexpr (QS) __syncthreads();

    float o[NT][MT][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      m[nt][0] = m[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[nt][i][c] = 0.f;
    }

    bool ok = true;
    int k = 0;
    for (; k < mine; ++k) {
      const uint32_t use = stage_use + k, st = use % S;
      ok = __all_sync(0xffffffffu, mbar_wait_or_expire(bars0 + 8 * st, (use / S) & 1, abort_flag, p.status, p.wait_cycles));
      if (!ok) break;
      const int valid = valid_s[st];
      const uint32_t ck = codes0 + st * UC, cv = ck + UC / 2, ks = scales0 + st * US, vs = ks + US / 2;
      if (valid > 0) {
        float sT[SUBS][NT][4];
#pragma unroll
        for (int b = 0; b < SUBS; ++b) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 4; ++c) sT[b][nt][c] = 0.f;
          const int t0 = b * 16 + row_a, t1 = t0 + 8;
          uint32_t x0[WL], x1[WL];
          if constexpr (D == 128) {
            const uint4 a0 = lds128(ck + t0 * 64 + ((tig ^ ((t0 >> 1) & 3)) << 4)), a1 = lds128(ck + t1 * 64 + ((tig ^ ((t1 >> 1) & 3)) << 4));
            x0[0] = a0.x; x0[1] = a0.y; x0[2] = a0.z; x0[3] = a0.w;
            x1[0] = a1.x; x1[1] = a1.y; x1[2] = a1.z; x1[3] = a1.w;
          } else {
            const uint2 a0 = lds64(ck + t0 * 32 + tig * 8), a1 = lds64(ck + t1 * 32 + tig * 8);
            x0[0] = a0.x; x0[1] = a0.y;
            x1[0] = a1.x; x1[1] = a1.y;
          }
          const int run = D == 128 ? tig : tig >> 1;
          const I4Scale s0 = i4_scale(lds8(ks + t0 * RUNS + run) * 0x00800080u), s1 = i4_scale(lds8(ks + t1 * RUNS + run) * 0x00800080u);
#pragma unroll
          for (int w = 0; w < WL; ++w) {
            uint32_t h0[4], h1[4];
            i4_operands(x0[w], s0, h0);
            i4_operands(x1[w], s1, h1);
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                uint32_t q0, q1;
                if constexpr (QS) {
                  const uint2 f = reinterpret_cast<const uint2*>(q_s)[((2 * w + half) * NT + nt) * 32 + lane];
                  q0 = f.x; q1 = f.y;
                } else {
                  q0 = qf[nt][2 * w + half][0]; q1 = qf[nt][2 * w + half][1];
                }
                mma_f16(sT[b][nt], h0[2 * half], h1[2 * half], h0[2 * half + 1], h1[2 * half + 1], q0, q1);
              }
          }
        }
        // scores in log2 units; tokens past the end drop out
        bool grow = false;
#pragma unroll
        for (int b = 0; b < SUBS; ++b)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 4; ++c) sT[b][nt][c] *= sc[nt][c & 1];
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
            grow |= t > m[nt][c] + kI4Tau;
          }
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              float t = top[nt][c];
#pragma unroll
              for (int x = 4; x < 32; x <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, x));
              const float mn = fmaxf(m[nt][c], t), f = mn == -INFINITY ? 1.f : exp2f(m[nt][c] - mn);
              m[nt][c] = mn;
              l[nt][c] *= f;
#pragma unroll
              for (int i = 0; i < MT; ++i) { o[nt][i][c] *= f; o[nt][i][c + 2] *= f; }
            }
        }
        uint32_t pf[SUBS][NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float r0 = m[nt][0] == -INFINITY ? 0.f : m[nt][0], r1 = m[nt][1] == -INFINITY ? 0.f : m[nt][1];
#pragma unroll
          for (int b = 0; b < SUBS; ++b) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const float e = i4_ex2(sT[b][nt][c] - ((c & 1) ? r1 : r0));
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
          const int tt[4] = {b * 16 + row_v0, b * 16 + row_v1, b * 16 + row_v0 + 8, b * 16 + row_v1 + 8};
          uint32_t v[4][E / 8], byte[4];
          const int run = D == 128 ? gid >> 1 : gid >> 2;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if constexpr (D == 128) {
              const uint2 t = lds64(cv + tt[i] * 64 + (((gid >> 1) ^ ((tt[i] >> 1) & 3)) << 4) + (gid & 1) * 8);
              v[i][0] = t.x; v[i][1] = t.y;
            } else {
              v[i][0] = lds32(cv + tt[i] * 32 + gid * 4);
            }
            byte[i] = lds8(vs + tt[i] * RUNS + run);
          }
          if (valid < UT) {                          // whatever lies past the end: codes are finite, scales may be anything
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (tt[i] >= valid) byte[i] = 0;
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
      if (k + S < mine) issue(k + S);
    }
    if (!ok) {                                       // given up: the copies in flight must have landed before the ring is reused or left
      const int upto = min(mine, k + S);
      for (int x = k; x < upto; ++x) mbar_drain(bars0 + 8 * ((stage_use + x) % S), ((stage_use + x) / S) & 1);
      stage_use += upto;                             // (nothing is waited for after this: the abort flag ends every wait)
    } else {
      stage_use += mine;
    }

    // ---- merge of the CTA's warps
    __syncthreads();                                 // the rings have been read
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
          merge_ml[(warp * R + r) * 2] = m[nt][c];
          merge_ml[(warp * R + r) * 2 + 1] = l[nt][c];
        }
      }
    }
    __syncthreads();
    const bool whole = item == seg_lo && piece_hi == seg_hi;
    float* record = p.partials + static_cast<size_t>(blockIdx.x * 2 + (item == seg_lo ? 1 : 0)) * R * (D + 2);
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
        *reinterpret_cast<float2*>(record + 2 * R + r * D + c) = make_float2(acc.x, acc.y);
        *reinterpret_cast<float2*>(record + 2 * R + r * D + c + 2) = make_float2(acc.z, acc.w);
        if (c == 0) { record[r] = M; record[R + r] = L; }
      }
    }
    if (!whole) {
      // the CTAs whose shares meet this segment are consecutive; the last of them to get here merges their records
      const int2 rec = segment_records(T, n_share, seg_lo, seg_hi);
      __syncthreads();
      if (tid == 0) *last_s = atomic_inc_acq_rel(p.tickets + sk * p.n_rg + rg, rec.y - 1) == static_cast<unsigned>(rec.y - 1);
      __syncthreads();
      if (*last_s) {
        // weights of the records of every row, then their sum
        float* wts = merge_o;                        // [R][n]; the tile has been read
        const int n = rec.y;
        auto at = [&](int j) { return p.partials + static_cast<size_t>((rec.x + j) * 2 + (j == 0 ? 1 : 0)) * R * (D + 2); };
        for (int r = warp; r < R; r += W) {
          if (rg * R + r >= rows) continue;
          float M = -INFINITY, L = 0.f;
          for (int j = lane; j < n; j += 32) M = fmaxf(M, __ldcg(at(j) + r));
          M = warp_max(M);
          for (int j = lane; j < n; j += 32) {
            const float mj = __ldcg(at(j) + r), f = mj == -INFINITY ? 0.f : exp2f(mj - M);
            wts[r * (n + 2) + j] = f;
            L += f * __ldcg(at(j) + R + r);
          }
          L = warp_sum(L);
          if (lane == 0) { wts[r * (n + 2) + n] = M; wts[r * (n + 2) + n + 1] = L; }
        }
        __syncthreads();
        for (int i = tid; i < R * (D / 4); i += blockDim.x) {
          const int r = i / (D / 4), c = (i % (D / 4)) * 4;
          if (rg * R + r >= rows) continue;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
          for (int j = 0; j < n; ++j) {
            const float f = wts[r * (n + 2) + j];
            const float2 a = __ldcg(reinterpret_cast<const float2*>(at(j) + 2 * R + r * D + c)), b = __ldcg(reinterpret_cast<const float2*>(at(j) + 2 * R + r * D + c + 2));
            acc.x = fmaf(a.x, f, acc.x); acc.y = fmaf(a.y, f, acc.y); acc.z = fmaf(b.x, f, acc.z); acc.w = fmaf(b.y, f, acc.w);
          }
          i4_finish(p, s, kh, rg * R + r, c, D, acc, wts[r * (n + 2) + n], wts[r * (n + 2) + n + 1]);
        }
      }
    }
    item = piece_hi;
    if (item < hi) {
      __syncthreads();                               // the merge tile has been read
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // ... and is written by copies next
    }
  }
}
