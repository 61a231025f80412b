// Attention over 4-bit pages, many query rows: included by int4_attn.cu (same namespace).
//
// From 17 rows of a KV head on the products bound the pass, not the bytes, so this kernel gives them to the 5th-generation tensor
// cores, 128 query rows at a time (one per tensor-memory lane), and the cache is turned into fp16 operands once for
// all of them.  Pages are taken in groups of 128 tokens:
//   eight warps   turn codes into fp16 tiles in shared memory (sixteen tokens each, keys and values): 16 bytes of codes, one scale, per
//                 lane from global memory into registers a group ahead, four 16-byte stores of swizzled chunks each; the
//                 eight elements of a chunk lie in the order 0 4 1 5 2 6 3 7 in which the conversion yields them, and so do
//                 the queries' and the output's columns
//   S[128 x 128] = Q K^T           an issuing warp; A = Q, B = keys, both from shared memory; D / 16 instructions
//   two sets of four softmax warps, thread = query row, take alternate groups.  Each set has its own scores, its own output and its own
//                 running maximum and sum, so that nothing passes between them before a piece ends; weights go back over the
//                 scores as fp16.  The reference maximum only moves when it would grow by more than 2^8.
//   O[128 x D] += P V              another issuing warp; A = P from tensor memory, B = values as they lie (tokens x d); 8 instructions
// Tensor memory is full: two outputs of D columns, two score tiles of 128.  Everything is handed on by mbarriers with bounded waits.
#pragma once

constexpr int kTcTok = 128, kTcRows = 128;         // tokens of a group, query rows
constexpr int kTcNK = 2, kTcNV = 3;                // tiles of keys, of values: values wait for the products of three groups back
constexpr int kTcSoftWarps = 8, kTcCvtWarps = 8, kTcQkWarp = 16, kTcPvWarp = 17, kTcWarps = 18;
constexpr int kTcMeta = 8;                         // groups whose valid tokens are kept: a group's are written once the keys' tile before the last is free
template <int D> constexpr int tc_tile() { return kTcTok * D * 2; }
template <int D> constexpr int tc_smem(int n_sk) {
  return 1024 + kTcRows * D * 2 + (kTcNK + kTcNV) * tc_tile<D>() + 512 + kTcMeta * 8 * 4 + 2 * 2 * kTcRows * 4 + (32 + n_sk + 1) * 4;
}

template <int D, int GP>
__global__ void __launch_bounds__(kTcWarps * 32, 1) int4_tc_kernel(const __grid_constant__ I4Params p) {
  constexpr int R = kTcRows, PG = kTcTok / GP, TILE = tc_tile<D>(), HS = kTcTok * 128, RUNS = D / kInt4Run;
  constexpr int NJ = D == 128 ? 2 : 1;             // 16-byte pieces of codes per lane, tensor and group
  constexpr uint32_t COL_O = 0, COL_S = 256;       // tensor-memory columns: two outputs of 128, two score tiles of 128
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const uint32_t qtile = base, kring = base + R * D * 2, vring = kring + kTcNK * TILE;
  constexpr int TAIL = R * D * 2 + (kTcNK + kTcNV) * TILE;
  const uint32_t bars = base + TAIL;
  const uint32_t k_full = bars, k_free = k_full + 8 * kTcNK, v_full = k_free + 8 * kTcNK, v_free = v_full + 8 * kTcNV;
  const uint32_t s_full = v_free + 8 * kTcNV, s_free = s_full + 16, p_full = s_free + 16, q_full = p_full + 16, o_free = q_full + 8, drain = o_free + 8;
  static_assert(8 * (2 * kTcNK + 2 * kTcNV + 6 + 2 + 2) + 16 <= 512, "barriers");
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + TAIL + 480);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(gen + TAIL + 484);
  int* meta = reinterpret_cast<int*>(gen + TAIL + 512);                  // [kTcMeta][8] valid tokens of every sixteen
  float* xm = reinterpret_cast<float*>(meta + kTcMeta * 8);              // [set][row] maximum (log2 units), then sum
  float* xl = xm + 2 * R;
  int* runs = reinterpret_cast<int*>(xl + 2 * R);
  int* pre = runs + 32;
  const int tid = threadIdx.x, lane = tid & 31, warp = warp_uniform(tid >> 5);

  if (tid == 0) {
    for (int i = 0; i < kTcNK; ++i) { mbar_init(k_full + 8 * i, kTcCvtWarps); mbar_init(k_free + 8 * i, 1); }
    for (int i = 0; i < kTcNV; ++i) { mbar_init(v_full + 8 * i, kTcCvtWarps); mbar_init(v_free + 8 * i, 1); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full + 8 * i, 1);                  // tcgen05.commit after Q K^T
      mbar_init(s_free + 8 * i, 1);                  // tcgen05.commit after P V: the set's scores may be replaced, its output holds the group
      mbar_init(p_full + 8 * i, 4);
      mbar_init(drain + 8 * i, 1);
    }
    mbar_init(q_full, kTcSoftWarps);
    mbar_init(o_free, kTcSoftWarps);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 0) {                                   // tensor memory: taken while the previous kernel drains
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "n"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  grid_dep_trigger();                                // (the merging kernel comes up beside this one)
  grid_dep_wait();
  I4Work<D, R> work(p, pre, runs, GP);
  const bool any = work.begin(2 * PG);               // (meets all threads; shares of two groups at least)
  tc5_fence_before();
  __syncthreads();
  tc5_fence_after();
  const uint32_t tmem = warp_uniform(*tmem_slot);
  bool ok = true;
  auto wait = [&](uint32_t bar, uint32_t parity) {
    if (ok) ok = warp_mbar_wait(bar, parity, abort_flag, p.status, p.wait_cycles);
    return ok;
  };

  if (!any) {
  } else if (warp < kTcSoftWarps) {
    // ================================================================== softmax: thread = (set, query row)
    const int set = warp >> 2, row = tid & 127;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_at = tmem + COL_S + set * 128 + lanes, o_at = tmem + COL_O + set * 128 + lanes;
    I4Piece piece = work.next_piece(work.lo, work.sk0);
    int g = 0;                                       // groups before the piece
    float sc = 1.f;
    // this thread's half of its row of Q: fp16 under a power of two of the row
    auto write_q = [&](const I4Piece& x) {
      const int r = x.rg * R + row;
      const long long at = r < work.rows_of(x.s) ? i4_row(p, x.s, x.kh, r) : -1;
      float amax = 0.f;
#pragma unroll 4
      for (int c = 0; c < D / 8; ++c) {
        float v[8];
        if (at >= 0) load8(p.q + at * D + c * 8, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = at >= 0 ? fmaxf(amax, fabsf(v[i])) : 0.f;
      }
      const int e = max(-100, min(127, static_cast<int>(__float_as_uint(amax) >> 23) - 127));       // the largest element comes to 2^14 .. 2^15
      const float up = __int_as_float((127 + 14 - e) << 23);
      sc = __int_as_float((127 - 14 + e) << 23) * (4.f * p.sm_scale * kLog2e);
#pragma unroll 4
      for (int c = set * (D / 16); c < (set + 1) * (D / 16); ++c) {
        uint32_t h[4] = {0u, 0u, 0u, 0u};
        if (at >= 0) {
          float v[8];
          load8(p.q + at * D + c * 8, v);
#pragma unroll
          for (int i = 0; i < 4; ++i) h[i] = pack_f16(v[i] * up, v[i + 4] * up);
        }
        *reinterpret_cast<uint4*>(gen + (c >> 3) * HS + tc5_sw(row, c & 7)) = make_uint4(h[0], h[1], h[2], h[3]);
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(q_full, 1);
    };
    write_q(piece);
    while (piece.n_units > 0) {
      const int groups = (piece.n_units + PG - 1) / PG;
      const bool idle = piece.rg * R + (warp & 3) * 32 >= work.rows_of(piece.s);       // none of the warp's rows exists
      float m = kI4None, l = 0.f;
      bool used = false;
      for (int i = 0; i < groups; ++i) {
        const int gg = g + i;
        if ((gg & 1) != set) continue;
        if (!wait(s_full + 8 * set, (gg >> 1) & 1)) break;
        tc5_fence_after();
        if (!idle) {
          // valid tokens: all of them, or a count for every sixteen
          const int* val = meta + (gg % kTcMeta) * 8;
          const int4 va = *reinterpret_cast<const int4*>(val), vb = *reinterpret_cast<const int4*>(val + 4);
          const bool full = va.x + va.y + va.z + va.w + vb.x + vb.y + vb.z + vb.w == kTcTok;
          uint32_t live[4] = {~0u, ~0u, ~0u, ~0u};
          if (!full) {
            const int n[8] = {va.x, va.y, va.z, va.w, vb.x, vb.y, vb.z, vb.w};
#pragma unroll
            for (int c = 0; c < 4; ++c) live[c] = ((1u << n[2 * c]) - 1u) | (((1u << n[2 * c + 1]) - 1u) << 16);
          }
          float top = kI4None;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            float x[32];
            tc5_ld32(s_at + c * 32, x);
            if (!full) {
#pragma unroll
              for (int k = 0; k < 32; ++k) x[k] = (live[c] >> k) & 1u ? x[k] : kI4None;
            }
#pragma unroll
            for (int k = 0; k < 32; k += 2) top = fmaxf(top, fmaxf(x[k], x[k + 1]));
          }
          const bool grow = (top - m) * sc > kI4Tau;
          if (__any_sync(0xffffffffu, grow)) {
            const float to = grow ? top : m, f = exp2f((m - to) * sc);
            if (used) {                              // the output of the set's earlier groups is complete: its product released these scores
#pragma unroll
              for (int c = 0; c < D / 16; ++c) {
                uint32_t x[16];
                tc5_ld16(o_at + c * 16, x);
#pragma unroll
                for (int k = 0; k < 16; ++k) x[k] = __float_as_uint(__uint_as_float(x[k]) * f);
                tc5_st16(o_at + c * 16, x);
              }
            }
            l *= f;
            m = to;
          }
          float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            float x[32];
            tc5_ld32(s_at + c * 32, x);
            uint32_t h[16];
#pragma unroll
            for (int k = 0; k < 32; ++k) {
              float e = ex2((x[k] - m) * sc);
              if (!full) e = (live[c] >> k) & 1u ? e : 0.f;
              x[k] = e;
              part[k & 3] += e;
            }
#pragma unroll
            for (int k = 0; k < 16; ++k) h[k] = pack_f16(x[2 * k], x[2 * k + 1]);
            tc5_st16(s_at + c * 16, h);
          }
          l += (part[0] + part[1]) + (part[2] + part[3]);
          tc5_wait_st();
        }
        used = true;
        tc5_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full + 8 * set, 1);
      }
      // ---- end of the piece: the set's last product, then both sets' outputs, half of the columns each
      const int last = g + groups - 1, mine = ((last & 1) == set ? last : last - 1);
      if (mine >= g) wait(s_free + 8 * set, (mine >> 1) & 1);
      xm[set * R + row] = l > 0.f || l != l ? m * sc : -INFINITY;
      xl[set * R + row] = l;
      tc5_fence_before();
      asm volatile("bar.sync 1, %0;" ::"n"(kTcSoftWarps * 32) : "memory");
      tc5_fence_after();
      const I4Piece following = work.next_piece(piece.hi, piece.sk);
      const float m0 = xm[row], m1 = xm[R + row], l0 = xl[row], l1 = xl[R + row], M = fmaxf(m0, m1);
      const float f0 = m0 == -INFINITY ? 0.f : exp2f(m0 - M), f1 = m1 == -INFINITY ? 0.f : exp2f(m1 - M), L = l0 * f0 + l1 * f1;
      if (following.n_units > 0) write_q(following);       // every product with the old queries has run
      const bool first = piece.first_page == 0, whole = first && (piece.n_units >> work.upp_log) == piece.pages;
      const int seg = piece.sk * p.n_rg + piece.rg, r = piece.rg * R + row;
      if (first && tid == 0) p.seg_records[seg] = whole ? make_int2(0, 0) : work.records(piece);
      float* record = p.partials + static_cast<size_t>(blockIdx.x + seg) * (R * (D + 2));
      const long long out_row = !idle && r < work.rows_of(piece.s) ? i4_row(p, piece.s, piece.kh, r) : -1;
      const float inv = L == 0.f ? 0.f : 4.f / L;
      if (!idle) {
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {               // 16 columns at a time of this set's half
          const int col = set * (D / 2) + c * 16;
          uint32_t a[16], b[16];
          tc5_ld16(tmem + COL_O + lanes + col, a);
          tc5_ld16(tmem + COL_O + 128 + lanes + col, b);
          float x[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) {               // (an output that was never written holds anything)
            const float y0 = f0 > 0.f || f0 != f0 ? __uint_as_float(a[k]) * f0 : 0.f, y1 = f1 > 0.f || f1 != f1 ? __uint_as_float(b[k]) * f1 : 0.f;
            // column 8 j + (0 4 1 5 2 6 3 7)[i] of the result lies at 8 j + i
            x[(k & 8) + ((k & 7) >> 1) + (k & 1) * 4] = y0 + y1;
          }
          if (out_row >= 0) {
#pragma unroll
            for (int k = 0; k < 16; k += 4) {
              if (whole) i4_store4(p, out_row * D + col + k, x[k] * inv, x[k + 1] * inv, x[k + 2] * inv, x[k + 3] * inv);
              else *reinterpret_cast<float4*>(record + 2 * R + row * D + col + k) = make_float4(x[k], x[k + 1], x[k + 2], x[k + 3]);
            }
          }
        }
        if (out_row >= 0 && set == 0) {
          if (whole) {
            if (p.lse) p.lse[out_row] = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
          } else {
            record[row] = M;
            record[R + row] = L;
          }
        }
      }
      tc5_fence_before();
      asm volatile("bar.sync 1, %0;" ::"n"(kTcSoftWarps * 32) : "memory");      // (the exchange has been read)
      if (lane == 0) mbar_arrive(o_free, 1);
      g += groups;
      piece = following;
    }
  } else if (warp < kTcSoftWarps + kTcCvtWarps) {
    // ================================================================== codes into tiles: tokens 16 w .. 16 w + 15 of every group
    const int w = warp - kTcSoftWarps;
    const int tok = D == 128 ? lane & 7 : lane & 15, piece16 = D == 128 ? lane >> 3 : lane >> 4;     // token (of eight or sixteen), run of 32 elements
    I4Piece ahead = work.next_piece(work.lo, work.sk0);
    int ahead_i = 0, b_phys = 0, b_valid = 0;        // the group that is fetched next: number ahead_i of its piece
    struct Fetched { uint4 k[NJ], v[NJ]; uint32_t ks[NJ], vs[NJ]; int valid; bool any; };
    auto fetch = [&](Fetched& f) {
      f.any = false;
      f.valid = 0;
      if (ahead.n_units > 0 && ahead_i * PG >= ahead.n_units) {
        ahead = work.next_piece(ahead.hi, ahead.sk);
        ahead_i = 0;
      }
      if (ahead.n_units == 0) return;
      f.any = true;
      constexpr int SPP = GP / 16;                   // sixteens per page
      if ((ahead_i & 31) == 0) {
        const int e = (ahead_i + lane) * PG + w / SPP;
        const int2 at = e < ahead.n_units ? i4_resolve(p, ahead, ahead.first_page + e, (w % SPP) * 16, 16) : make_int2(0, 0);
        b_phys = at.x;
        b_valid = at.y;
      }
      const int phys = __shfl_sync(0xffffffffu, b_phys, ahead_i & 31);
      f.valid = __shfl_sync(0xffffffffu, b_valid, ahead_i & 31);
      const int t0 = (w % SPP) * 16;
      const int64_t src = phys * p.stride_page + ahead.kh * p.stride_head + (t0 + tok) * p.stride_tok + piece16 * 16;
      const int64_t sat = ((static_cast<int64_t>(phys) * p.Hkv + ahead.kh) * p.g + t0 + tok) * RUNS + piece16;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        f.k[j] = make_uint4(0u, 0u, 0u, 0u);
        f.v[j] = f.k[j];
        f.ks[j] = f.vs[j] = 0u;
        if (tok + 8 * j < f.valid) {
          f.k[j] = __ldcs(reinterpret_cast<const uint4*>(p.k_pages + src + 8 * j * p.stride_tok));
          f.v[j] = __ldcs(reinterpret_cast<const uint4*>(p.v_pages + src + 8 * j * p.stride_tok));
          f.ks[j] = p.k_scale[sat + 8 * j * RUNS];
          f.vs[j] = p.v_scale[sat + 8 * j * RUNS];
        }
      }
      ++ahead_i;
    };
    auto convert = [&](uint8_t* tile, const uint4 (&x)[NJ], const uint32_t (&byte)[NJ]) {
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const I4Scale s = i4_scale(byte[j] * 0x00800080u);
        const uint32_t words[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t h[4];
          i4_operands(words[i], s, h);
          const int c = piece16 * 4 + i;
          *reinterpret_cast<uint4*>(tile + (c >> 3) * HS + tc5_sw(w * 16 + 8 * j + tok, c & 7)) = make_uint4(h[0], h[1], h[2], h[3]);
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");       // the products read the tile through the async proxy
      __syncwarp();
    };
    Fetched cur, next;
    fetch(cur);
    for (int g = 0; cur.any; ++g) {
      fetch(next);
      const int ks = g % kTcNK, vs = g % kTcNV;
      if (g >= kTcNK && !wait(k_free + 8 * ks, (g / kTcNK - 1) & 1)) break;
      if (lane == 0) meta[(g % kTcMeta) * 8 + w] = cur.valid;
      convert(gen + R * D * 2 + ks * TILE, cur.k, cur.ks);
      if (lane == 0) mbar_arrive(k_full + 8 * ks, 1);
      if (g >= kTcNV && !wait(v_free + 8 * vs, (g / kTcNV - 1) & 1)) break;
      convert(gen + R * D * 2 + (kTcNK + vs) * TILE, cur.v, cur.vs);
      if (lane == 0) mbar_arrive(v_full + 8 * vs, 1);
      cur = next;
    }
  } else if (warp == kTcQkWarp) {
    // ================================================================== Q K^T
    const uint32_t qt = warp_uniform(qtile), kr = warp_uniform(kring), idesc = tc5_idesc(R, kTcTok, 0, 0u, 0u);
    I4Piece piece = work.next_piece(work.lo, work.sk0);
    int g = 0;
    for (int n = 0; piece.n_units > 0 && ok; ++n) {
      const int groups = warp_uniform((piece.n_units + PG - 1) / PG);
      if (!wait(q_full, n & 1)) break;
      for (int i = 0; i < groups; ++i, ++g) {
        const int set = g & 1, use = g >> 1, slot = g % kTcNK;
        if (!wait(k_full + 8 * slot, (g / kTcNK) & 1) || (use > 0 && !wait(s_free + 8 * set, (use - 1) & 1))) break;
        tc5_fence_after();
        if (elect_one()) {
          const uint64_t qd = tc5_desc(qt, 16), kd = tc5_desc(kr + slot * TILE, 16);
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            const uint32_t at = ((ks >> 2) * HS + (ks & 3) * 32) / 16;
            tc5_mma_ss(tmem + COL_S + set * 128, qd + at, kd + at, idesc, ks > 0 ? 1u : 0u);
          }
          tc5_commit(s_full + 8 * set);
          tc5_commit(k_free + 8 * slot);
        }
        __syncwarp();
      }
      piece = work.next_piece(piece.hi, piece.sk);
    }
  } else if (warp == kTcPvWarp) {
    // ================================================================== P V
    const uint32_t vr = warp_uniform(vring), idesc = tc5_idesc(R, D, 1, 0u, 0u);
    I4Piece piece = work.next_piece(work.lo, work.sk0);
    int g = 0;
    for (int n = 0; piece.n_units > 0 && ok; ++n) {
      const int groups = warp_uniform((piece.n_units + PG - 1) / PG);
      if (n > 0 && !wait(o_free, (n - 1) & 1)) break;
      for (int i = 0; i < groups; ++i, ++g) {
        const int set = g & 1, slot = g % kTcNV;
        if (!wait(v_full + 8 * slot, (g / kTcNV) & 1) || !wait(p_full + 8 * set, (g >> 1) & 1)) break;
        tc5_fence_after();
        if (elect_one()) {
          const uint64_t vd = tc5_desc(vr + slot * TILE, HS);
          const uint32_t p_col = tmem + COL_S + set * 128, o_col = tmem + COL_O + set * 128, fresh = i < 2 ? 0u : 1u;      // the set's first group of the piece
#pragma unroll
          for (int ks = 0; ks < kTcTok / 16; ++ks) tc5_mma_ts(o_col, p_col + ks * 8, vd + ks * 128, idesc, ks == 0 ? fresh : 1u);
          tc5_commit(v_free + 8 * slot);
          tc5_commit(s_free + 8 * set);
        }
        __syncwarp();
      }
      piece = work.next_piece(piece.hi, piece.sk);
    }
  }
  // ---- the products in flight have run before tensor memory is given back
  if (warp == kTcQkWarp || warp == kTcPvWarp) {
    const uint32_t bar = drain + 8 * (warp - kTcQkWarp);
    if (elect_one()) {
      tc5_commit(bar);
      mbar_drain(bar, 0);
    }
    __syncwarp();
  }
  tc5_fence_before();
  __syncthreads();
  if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
}
