// Attention over 4-bit pages, up to 16 query rows per pass: included by int4_attn.cu (same namespace).
//
// What it cannot do without are the cache's bytes (68 per row of 128); what bounds it are instructions and their latencies: about 680 per
// unit of 32 tokens, half of them conversion and products, issued at 2.1 a cycle and SM of four possible, which is what three warps per scheduler
// (two at 16 rows, with 255 registers) cover.  Eight prompts of 32,768 tokens, one token each (8 rows per KV
// head): 75 us, 59 % of the copy rate; 16 rows 104; one prompt of 8,192 14.5, most of it latency.  So tokens, not query rows, are the M side of every product, codes become operands in registers, and
// nothing but codes passes through shared memory:
//   S^T[16 tokens x 8 rows] += K[16 x 16 d] Q^T[16 d x 8]     mma.sync.m16n8k16, A = keys: a lane takes the quarter
//                                (d/4 elements, 16 bytes at d = 128) of two rows that lies in one piece; which elements the
//                                instruction thinks they are does not matter, Q's fragments are laid out the same way
//   O^T[16 d x 8 rows]      += V^T[16 d x 16 tokens] P^T      A = values: a half2 is one element of two tokens, which two
//                                byte permutes put together from the words of the two rows; P^T is S^T, transposed 8 x 8 by movmatrix
// Warps take units of up to 32 tokens in turn, each through a ring of its own that it fills by asynchronous copies, 16 bytes per lane: no
// barrier, and no instruction that one lane executes for the others (tensor copies, issued by one lane of each warp or by a warp
// for all rings, cost 90 instructions a unit or kept the rings in step).  The rings run on over the pieces of a
// share.  A warp keeps its own maximum, sum and output; the reference maximum only moves when it
// would grow by more than 2^8, which one vote per unit finds out.  At the end of a piece the warps of the CTA
// merge through shared memory; what CTAs leave of a segment that several of them share is merged by a kernel of its own, whose
// start overlaps this one's end (merging by the last CTA to arrive, behind a ticket, took 5 us of its own at the end of the longest share).
#pragma once

constexpr float kI4Tau = 8.f;                       // log2 units
// Weights are taken times 2^7, in log2 units: the largest, 2^8 of the reference's, comes to 2^15 and fits fp16, and those below 2^-14 of a row's
// largest keep their bits: eleven down to 2^-21 of it, and below that to within 2^-32 of it.  A reference that leaves a warp is in the same units.
constexpr float kI4Lift = 7.f;
constexpr float kI4None = -3e38f;                   // a reference before the first score
constexpr float kI4MostTau = 1e38f;                 // no threshold is larger: the first score outgrows the reference before it whatever the scale
// (Scores are fp16 products under 2^36, so none of them meets either of the two.)  A row's factor from scores to log2 units, which is not zero:
// with rows of zeros and the smallest softmax scales it would be, and -inf times it no number.
__device__ __forceinline__ float i4_score_scale(int e, float sm_scale) { return fmaxf(__int_as_float((127 - 14 + e) << 23) * (4.f * sm_scale * kLog2e), 1.17549435e-38f); }
constexpr int i4_warps(int nt) { return nt == 1 ? 12 : 8; }     // most warps of an SM: 168, 255 registers a thread

template <int D> constexpr int i4_unit_codes(int ut) { return ut * D; }          // bytes of a unit's codes, K and V
template <int D> constexpr int i4_unit_scales(int ut) { return ut * D / 16; }    // ... and scales
template <int D, int NT> constexpr int i4_merge_bytes(int warps) { return ((warps * 8 * NT * (D + 4) * 4 + warps * 8 * NT * 8) + 15) / 16 * 16; }
constexpr int kI4Ring = 2;                          // units of a ring
constexpr int kI4Stride = 4;                        // floats between the rows of the merge tile: a row is D + 4

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

// UT: tokens of a unit
template <int D, int NT, int UT>
__global__ void __launch_bounds__(i4_warps(NT) * 32, 1)
int4_mma_kernel(const __grid_constant__ I4Params p) {
  constexpr int S = kI4Ring, R = 8 * NT, KS = D / 16, MT = D / 16, E = D / 8, WL = D / 32, RUNS = D / kInt4Run;
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
  // no more shares than give every warp a unit
  I4Work<D, R> work(p, pre, chunk_s, UT);
  if (!work.begin(W)) return;
  // ---- the ring: units warp, warp + W, ... of every piece, one piece after the other; the copies run S - 1 units ahead
  unsigned long long policy;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
  constexpr int RB = D / 2, LPR = RB / 16, RPI = 32 / LPR, SL = US / 8;  // bytes of a row, lanes per row, rows per copy, lanes per copy of scales
  auto swz = [](int t, int chunk) { return D == 128 ? (chunk ^ ((t >> 1) & 3)) << 4 : chunk << 4; };   // (the same eight rows further on)
  const int64_t copy_src = static_cast<int64_t>(lane / LPR) * p.stride_tok + (lane % LPR) * 16;
  const uint32_t copy_dst = codes0 + (lane / LPR) * RB + swz(lane / LPR, lane % LPR), scale_dst = scales0 + lane * 4;
  I4Piece ahead = work.next_piece(work.lo, work.sk0), piece = ahead;
  int ahead_k = 0;                                   // the next unit to be copied: number ahead_k of this warp in its piece
  // queries of a piece, as they lie, into this warp's tile: with the next unit's copies
  auto copy_queries = [&](const I4Piece& x) {
    const int rows = work.rows_of(x.s) - x.rg * R;
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
    while (warp + W * ahead_k >= ahead.n_units && ahead.hi < work.hi) {
      ahead = work.next_piece(ahead.hi, ahead.sk);
      ahead_k = 0;
    }
    if (warp + W * ahead_k < ahead.n_units) {
      if ((ahead_k & 31) == 0) {
        const int u = warp + W * (ahead_k + lane);
        const int2 at = u < ahead.n_units ? i4_resolve(p, ahead, ahead.first_page + (u >> work.upp_log), (u & work.upp_mask) * UT, UT) : make_int2(0, 0);
        b_phys = at.x;
        b_valid = at.y;
      }
      const int phys = __shfl_sync(0xffffffffu, b_phys, ahead_k & 31), valid = __shfl_sync(0xffffffffu, b_valid, ahead_k & 31);
      const int t0 = ((warp + W * ahead_k) & work.upp_mask) * UT;
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
    const int s = piece.s, kh = piece.kh, rg = piece.rg, rows = work.rows_of(s), n_units = piece.n_units;
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
      const float up = __int_as_float((127 + 14 - e) << 23), down = i4_score_scale(e, p.sm_scale);
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
    const I4Piece following = work.next_piece(piece.hi, piece.sk);
    if (following.n_units > 0) copy_queries(following);
    asm volatile("cp.async.commit_group;" ::: "memory");           // (older than the next unit's group: waited for with the unit before that)

    float o[NT][MT][4], m[NT][2], l[NT][2], tau[NT][2];      // m: in units of the scores as they are; a difference times sc is in log2 units
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      m[nt][0] = m[nt][1] = kI4None;
      l[nt][0] = l[nt][1] = 0.f;
      tau[nt][0] = fminf(kI4Tau / sc[nt][0], kI4MostTau);
      tau[nt][1] = fminf(kI4Tau / sc[nt][1], kI4MostTau);
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
              const float e = ex2(fmaf(sT[b][nt][c] - m[nt][c & 1], sc[nt][c & 1], kI4Lift));
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
    static_assert(S == 2, "two slots");
    int k = 0;
    if (mine > 0 && next_slot == 1) { take(std::integral_constant<int, 1>{}); ++k; }
#pragma unroll 1
    for (; k + 2 <= mine; k += 2) {
      take(std::integral_constant<int, 0>{});
      take(std::integral_constant<int, 1>{});
    }
    next_slot = 0;
    if (k < mine) { take(std::integral_constant<int, 0>{}); next_slot = 1; }
    if (mine == 0) next_slot = next_slot_was;

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
          merge_ml[(warp * R + r) * 2] = m[nt][c] == kI4None ? -INFINITY : fmaf(m[nt][c], sc[nt][c], -kI4Lift);
          merge_ml[(warp * R + r) * 2 + 1] = l[nt][c];
        }
      }
    }
    __syncthreads();
    const bool first = piece.first_page == 0, whole = first && (n_units >> work.upp_log) == piece.pages;
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
      p.seg_records[piece.sk * p.n_rg + rg] = whole ? make_int2(0, 0) : work.records(piece);
    piece = following;
    if (piece.n_units > 0) __syncthreads();          // the merge tile has been read
  }
}
