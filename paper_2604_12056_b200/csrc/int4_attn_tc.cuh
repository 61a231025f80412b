// Attention over 4-bit pages, many query rows: included by int4_attn.cu (same namespace).
//
// From 17 rows of a KV head on the products bound the pass, not the bytes, so this kernel gives them to the 5th-generation tensor
// cores, 128 query rows at a time (one per tensor-memory lane), and the cache is turned into fp16 operands once for
// all of them.  Pages are taken in groups of 128 tokens:
//   eight warps   turn codes into fp16 tiles in shared memory (32 tokens each, four warps for keys and four for values): 16 bytes of
//                 codes and their scale from global memory into registers a group ahead (L2: sixteen), four 16-byte stores of swizzled chunks; the
//                 eight elements of a chunk lie in the order 0 4 1 5 2 6 3 7 in which the conversion yields them, and so do
//                 the queries' and the output's columns
//   S[128 x 64] = Q K^T            an issuing warp; A = Q, B = half a group's keys, both from shared memory; D / 16 instructions
//   two sets of four softmax warps, thread = query row, take alternate groups.  Each set has its own scores (two halves, so that the
//                 products of one run while the other is worked on), its own output and its own running maximum and sum: nothing
//                 passes between the sets before a piece ends.  A row's 64 scores are read once and stay in registers; weights go
//                 back over them as fp16.  The reference maximum only moves when it would grow by more than 2^8.
//   O[128 x D] += P V              another issuing warp; A = P from tensor memory, B = values as they lie (tokens x d); 4 instructions per half
// A block of 32 tokens (128 rows) over eight prompts of 32,768: 201 us over several input sets (183 with two in turn, as the steps below were
// timed), where the products need 84 at the dense bf16 rate; they and their barriers alone take 132, since an operand in shared memory is read
// again by every instruction.
// Tensor memory is full: two outputs of D columns, two score tiles of 128.  Everything is handed on by mbarriers with bounded waits.
#pragma once

constexpr int kTcTok = 128, kTcRows = 128;         // tokens of a group, query rows
constexpr int kTcNK = 2, kTcNV = 3;                // tiles of keys, of values: values wait for the products of three groups back
constexpr int kTcSoftWarps = 8, kTcCvtWarps = 8, kTcQkWarp = 16, kTcPvWarp = 17, kTcWarps = 20;     // (whole groups of four: registers are dealt out by them)
// Registers per thread at the launch, and as they are dealt out: 8 x 32 x 120 + 12 x 32 x 80 = 640 x 96
constexpr int kTcLaunchRegs = 96, kTcSoftRegs = 120, kTcOtherRegs = 80;
static_assert(kTcSoftWarps * kTcSoftRegs + (kTcWarps - kTcSoftWarps) * kTcOtherRegs <= kTcWarps * kTcLaunchRegs, "registers");
constexpr float kTcFused = 1048576.f;              // a reference up to this: its product with the scale may be subtracted in one operation
constexpr int kTcMeta = 8;                         // groups whose valid tokens are kept: a group's are written once the keys' tile before the last is free
template <int D> constexpr int tc_tile() { return kTcTok * D * 2; }
template <int D> constexpr int tc_smem(int n_sk) {
  return 1024 + kTcRows * D * 2 + (kTcNK + kTcNV) * tc_tile<D>() + 512 + kTcMeta * 8 * 4 + (2 + 2 + 2) * kTcRows * 4 + (32 + n_sk + 1) * 4;
}

__device__ __forceinline__ void tc_store16(void* at, bool on, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %1, 0;\n\t@p st.global.v4.b32 [%0], {%2, %3, %4, %5};\n\t}"
               ::"l"(at), "r"(static_cast<int>(on)), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ void i4_prefetch(const uint8_t* at) { asm volatile("prefetch.global.L2 [%0];" ::"l"(at)); }
// loads that are issued where they are written
__device__ __forceinline__ uint4 i4_load16(const uint8_t* src) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(src));
  return v;
}
__device__ __forceinline__ uint32_t i4_load1(const uint8_t* src) {
  uint32_t v;
  asm volatile("ld.global.nc.u8 %0, [%1];" : "=r"(v) : "l"(src));
  return v;
}
// two at a time
__device__ __forceinline__ float2 add_f32x2(float2 a, float2 b) {
  float2 c;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(c.x), "=f"(c.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return c;
}
__device__ __forceinline__ float2 fma_f32x2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\tfma.rn.f32x2 z, x, y, z;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}

template <int D, int GP>
__global__ void __launch_bounds__(kTcWarps * 32, 1) int4_tc_kernel(const __grid_constant__ I4Params p) {
  constexpr int R = kTcRows, PG = kTcTok / GP, TILE = tc_tile<D>(), HS = kTcTok * 128, RUNS = D / kInt4Run;
  constexpr int NJ = D == 128 ? 4 : 2;             // 16-byte pieces of codes per converting lane and group
  constexpr uint32_t COL_O = 0, COL_S = 256;       // tensor-memory columns: two outputs of 128, two score tiles of 128
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const uint32_t qtile = base, kring = base + R * D * 2, vring = kring + kTcNK * TILE;
  constexpr int TAIL = R * D * 2 + (kTcNK + kTcNV) * TILE;
  const uint32_t bars = base + TAIL;
  const uint32_t k_full = bars, k_free = k_full + 8 * kTcNK, v_full = k_free + 8 * kTcNK, v_free = v_full + 8 * kTcNV;
  const uint32_t s_full = v_free + 8 * kTcNV, s_free = s_full + 32, p_full = s_free + 32, q_full = p_full + 32, o_free = q_full + 8, drain = o_free + 8;
  static_assert(8 * (2 * kTcNK + 2 * kTcNV + 12 + 2 + 2) <= 480, "barriers");
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + TAIL + 480);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(gen + TAIL + 484);
  int* meta = reinterpret_cast<int*>(gen + TAIL + 512);                  // [kTcMeta][8] valid tokens of every sixteen
  float* xm = reinterpret_cast<float*>(meta + kTcMeta * 8);              // [set][row] reference maximum (log2 units, less the weights' lift)
  float* xl = xm + 2 * R;                                                // [set][row] sum of weights
  float* xt = xl + 2 * R;                                                // [half][row] largest element of a query
  int* runs = reinterpret_cast<int*>(xt + 2 * R);
  int* pre = runs + 32;
  const int tid = threadIdx.x, lane = tid & 31, warp = warp_uniform(tid >> 5);

  if (tid == 0) {
    for (int i = 0; i < kTcNK; ++i) { mbar_init(k_full + 8 * i, kTcCvtWarps / 2); mbar_init(k_free + 8 * i, 1); }
    for (int i = 0; i < kTcNV; ++i) { mbar_init(v_full + 8 * i, kTcCvtWarps / 2); mbar_init(v_free + 8 * i, 1); }
    for (int i = 0; i < 4; ++i) {                    // [set][half]
      mbar_init(s_full + 8 * i, 1);                  // tcgen05.commit after Q K^T
      mbar_init(s_free + 8 * i, 1);                  // tcgen05.commit after P V: the scores may be replaced, the set's output holds them
      mbar_init(p_full + 8 * i, kTcSoftWarps / 2);
    }
    mbar_init(drain, 1);
    mbar_init(drain + 8, 1);
    mbar_init(q_full, kTcSoftWarps);
    mbar_init(o_free, kTcSoftWarps);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  grid_dep_trigger();                                // (the merging kernel comes up beside this one)
  grid_dep_wait();
  I4Work<D, R> work(p, pre, runs, GP);
  if (!work.begin(2 * PG)) return;                   // (one answer for the CTA; shares of two groups at least)
  __syncwarp();
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "n"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc5_fence_before();
  __syncthreads();
  tc5_fence_after();
  const uint32_t tmem = warp_uniform(*tmem_slot);
  // a bound shorter than a look at a barrier takes has run out by then (which is how the way out is exercised)
  bool ok = p.wait_cycles >= kLookCycles;
  if (!ok && tid == 0) set_status(p.status, LOSA_ERR_TIMEOUT);
  auto wait = [&](uint32_t bar, uint32_t parity) {
    if (ok) ok = warp_mbar_wait(bar, parity, abort_flag, p.status, p.wait_cycles);
    __syncwarp();                                    // (what follows is for whole warps)
    return ok;
  };

  __syncwarp();
  if (warp < kTcSoftWarps) {
    // ================================================================== softmax: thread = (set, query row)
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kTcSoftRegs));
    const int set = warp >> 2, row = tid & 127;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_at = tmem + COL_S + set * 128 + lanes, o_at = tmem + COL_O + set * 128 + lanes;
    auto all_meet = [&]() {
      __syncwarp();
      asm volatile("bar.sync 1, %0;" ::"n"(kTcSoftWarps * 32) : "memory");
    };
    I4Piece piece = work.next_piece(work.lo, work.sk0);
    int g = 0;                                       // groups before the piece
    float sc = 1.f;
    // this thread's half of its row of Q: fp16 under a power of two of the row
    auto write_q = [&](const I4Piece& x) {
      const int r = x.rg * R + row;
      const long long at = r < work.rows_of(x.s) ? i4_row(p, x.s, x.kh, r) : -1;
      uint4 q[D / 16];
      float amax = 0.f;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) q[c] = at >= 0 ? *reinterpret_cast<const uint4*>(p.q + at * D + set * (D / 2) + c * 8) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        float v[8];
        load8(reinterpret_cast<const __nv_bfloat16*>(&q[c]), v);
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(v[i]));
      }
      xt[set * R + row] = amax;
      all_meet();
      amax = fmaxf(xt[row], xt[R + row]);
      const int e = max(-100, min(127, static_cast<int>(__float_as_uint(amax) >> 23) - 127));       // the largest element comes to 2^14 .. 2^15
      const float up = __int_as_float((127 + 14 - e) << 23);
      sc = i4_score_scale(e, p.sm_scale);
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        float v[8];
        load8(reinterpret_cast<const __nv_bfloat16*>(&q[c]), v);
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = pack_f16(v[i] * up, v[i + 4] * up);
        const int chunk = set * (D / 16) + c;
        *reinterpret_cast<uint4*>(gen + (chunk >> 3) * HS + tc5_sw(row, chunk & 7)) = make_uint4(h[0], h[1], h[2], h[3]);
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
        const uint32_t turn = (gg >> 1) & 1;
#pragma unroll 1
        for (int hf = 0; hf < 2; ++hf) {
          const int mine = set * 2 + hf;
          if (!wait(s_full + 8 * mine, turn)) break;
          tc5_fence_after();
          if (!idle) {
            const uint32_t at = s_at + hf * 64;
            uint32_t x[64];
            tc5_ld32_nowait(at, x);
            tc5_ld32_nowait(at + 32, x + 32);
            // valid tokens of every sixteen
            const int4 n = *reinterpret_cast<const int4*>(meta + (gg % kTcMeta) * 8 + hf * 4);
            const bool full = n.x + n.y + n.z + n.w == kTcTok / 2;
            tc5_wait_ld();
            tc5_pin32(x);
            tc5_pin32(x + 32);
            auto score = [&](int k) { return __uint_as_float(x[k]); };
            if (!full) {
              const uint32_t live[2] = {((1u << n.x) - 1u) | (((1u << n.y) - 1u) << 16), ((1u << n.z) - 1u) | (((1u << n.w) - 1u) << 16)};
#pragma unroll
              for (int k = 0; k < 64; ++k) x[k] = (live[k >> 5] >> (k & 31)) & 1u ? x[k] : 0xff800000u;       // -inf: no weight
            }
            float top = kI4None, top2 = kI4None;
#pragma unroll
            for (int k = 0; k < 64; k += 4) {
              top = max3(top, score(k), score(k + 1));
              top2 = max3(top2, score(k + 2), score(k + 3));
            }
            top = fmaxf(top, top2);
            const bool grow = (top - m) * sc > kI4Tau || m == kI4None;       // (none yet: whatever the scale)
            if (__any_sync(0xffffffffu, grow)) {
              const float to = grow ? top : m, f = exp2f((m - to) * sc);
              if (used) {                            // the output of all that came before: the half before this one was the last
                if (hf == 1) wait(s_free + 8 * (set * 2), turn);
                else wait(s_free + 8 * (set * 2 + 1), turn ^ 1);
                tc5_fence_after();
#pragma unroll 1
                for (int c = 0; c < D / 16; ++c) {
                  uint32_t y[16];
                  tc5_ld16(o_at + c * 16, y);
#pragma unroll
                  for (int k = 0; k < 16; ++k) y[k] = __float_as_uint(__uint_as_float(y[k]) * f);
                  tc5_st16(o_at + c * 16, y);
                }
              }
              l *= f;
              m = to;
            }
            const float shift = m == kI4None ? 0.f : fmaf(-m, sc, kI4Lift);
            float2 part[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
            const float2 scale = make_float2(sc, sc);
            // a reference so large that only differences can be scaled: subtracted from the scores first (not an infinite one, whose row is
            // lost: the warp's other rows are computed as they are beside any other)
            const bool apart = __any_sync(0xffffffffu, fabsf(shift) > kTcFused && fabsf(shift) < INFINITY);
            if (apart) {
#pragma unroll
              for (int k = 0; k < 64; ++k) x[k] = __float_as_uint(score(k) - m);
            }
            const float2 sh = apart ? make_float2(kI4Lift, kI4Lift) : make_float2(shift, shift);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              uint32_t h[16];
#pragma unroll
              for (int k = 0; k < 16; ++k) {
                float2 e = fma_f32x2(make_float2(score(c * 32 + 2 * k), score(c * 32 + 2 * k + 1)), scale, sh);
                e.x = ex2(e.x);
                e.y = ex2(e.y);
                part[k & 1] = add_f32x2(part[k & 1], e);
                h[k] = pack_f16(e.x, e.y);
              }
              tc5_st16(at + c * 16, h);
            }
            part[0] = add_f32x2(part[0], part[1]);
            l += part[0].x + part[0].y;
            tc5_wait_st();
          }
          used = true;
          tc5_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(p_full + 8 * mine, 1);
        }
      }
      // ---- end of the piece: the set's last product, then both sets' outputs, half of the columns each
      const int last = g + groups - 1, mine = ((last & 1) == set ? last : last - 1);
      if (mine >= g) wait(s_free + 8 * (set * 2 + 1), (mine >> 1) & 1);
      xm[set * R + row] = m == kI4None ? -INFINITY : fmaf(m, sc, -kI4Lift);
      xl[set * R + row] = l;
      tc5_fence_before();
      all_meet();
      tc5_fence_after();
      const I4Piece following = work.next_piece(piece.hi, piece.sk);
      const float m0 = xm[row], m1 = xm[R + row], l0 = xl[row], l1 = xl[R + row], M = fmaxf(m0, m1);
      const float f0 = m0 == -INFINITY ? 0.f : exp2f(m0 - M), f1 = m1 == -INFINITY ? 0.f : exp2f(m1 - M), L = l0 * f0 + l1 * f1;
      if (following.n_units > 0) write_q(following);       // every product with the old queries has run
      const bool first = piece.first_page == 0, whole = first && (piece.n_units >> work.upp_log) == piece.pages;
      const int seg = piece.sk * p.n_rg + piece.rg, r = piece.rg * R + row;
      if (first && tid == 0) p.seg_records[seg] = whole ? make_int2(0, 0) : work.records(piece);
      __syncwarp();
      if (!idle) {
        float* record = p.partials + static_cast<size_t>(blockIdx.x + seg) * (R * (D + 2));
        const long long out_row = r < work.rows_of(piece.s) ? i4_row(p, piece.s, piece.kh, r) : -1;
        const float inv = L == 0.f ? 0.f : 4.f / L;
        __syncwarp();                                    // (the lanes have found their rows each for itself; the loads below need the whole warp)
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {               // 16 columns at a time
          const int col = set * (D / 2) + c * 16;
          uint32_t a[16], b[16];
          tc5_ld16(tmem + COL_O + lanes + col, a);
          tc5_ld16(tmem + COL_O + 128 + lanes + col, b);
          float x[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) {               // (an output that was never written holds anything)
            const float y0 = m0 != -INFINITY ? __uint_as_float(a[k]) * f0 : 0.f, y1 = m1 != -INFINITY ? __uint_as_float(b[k]) * f1 : 0.f;
            // column 8 j + (0 4 1 5 2 6 3 7)[i] of the result lies at 8 j + i
            x[(k & 8) + ((k & 7) >> 1) + (k & 1) * 4] = y0 + y1;
          }
          // (stores under a predicate, not a branch: the loads of tensor memory around them need the whole warp)
          if (!whole) {
#pragma unroll
            for (int k = 0; k < 16; k += 4) tc_store16(record + 2 * R + row * D + col + k, out_row >= 0, __float_as_uint(x[k]), __float_as_uint(x[k + 1]), __float_as_uint(x[k + 2]), __float_as_uint(x[k + 3]));
          } else if (p.out_bf16) {
            auto pack = [&](int k) {
              const __nv_bfloat162 t = __floats2bfloat162_rn(x[k] * inv, x[k + 1] * inv);
              return *reinterpret_cast<const uint32_t*>(&t);
            };
#pragma unroll
            for (int k = 0; k < 16; k += 8) tc_store16(static_cast<__nv_bfloat16*>(p.out) + out_row * D + col + k, out_row >= 0, pack(k), pack(k + 2), pack(k + 4), pack(k + 6));
          } else {
#pragma unroll
            for (int k = 0; k < 16; k += 4)
              tc_store16(static_cast<float*>(p.out) + out_row * D + col + k, out_row >= 0, __float_as_uint(x[k] * inv), __float_as_uint(x[k + 1] * inv), __float_as_uint(x[k + 2] * inv), __float_as_uint(x[k + 3] * inv));
          }
          __syncwarp();
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
      __syncwarp();
      tc5_fence_before();
      all_meet();                                      // (the exchange has been read)
      if (lane == 0) mbar_arrive(o_free, 1);
      g += groups;
      piece = following;
    }
  } else {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kTcOtherRegs));
  if (warp < kTcSoftWarps + kTcCvtWarps) {
    // ================================================================== codes into tiles: tokens 32 w .. 32 w + 31 of every group, of one tensor
    const int w = (warp - kTcSoftWarps) & 3;
    const bool is_v = warp >= kTcSoftWarps + 4;
    constexpr int TPJ = D == 128 ? 8 : 16, SPP = GP / 16;                // tokens per access of the warp; sixteens per page
    const int tok = lane % TPJ, run = lane / TPJ;    // the lane's token, and which 32 of its elements
    const uint8_t *pages = is_v ? p.v_pages : p.k_pages, *scales = is_v ? p.v_scale : p.k_scale;
    I4Piece ahead = work.next_piece(work.lo, work.sk0);
    int ahead_i = 0, b_valid = 0;                    // the group that is fetched next: number ahead_i of its piece
    const uint8_t *b_src = nullptr, *b_scale = nullptr;      // 16 groups at a time, two sixteens each, one per lane: where codes and scales lie
    const int64_t my_src = tok * p.stride_tok + run * 16;
    const int my_scale = tok * RUNS + run;
    uint4 x[NJ];
    uint32_t scale[NJ];
    int2 valid = make_int2(0, 0);                    // of the two sixteens
    auto fetch = [&]() {                             // false: there is no further group
      if (ahead.n_units > 0 && ahead_i * PG >= ahead.n_units) {
        ahead = work.next_piece(ahead.hi, ahead.sk);
        ahead_i = 0;
      }
      if (ahead.n_units == 0) return false;
      if ((ahead_i & 15) == 0) {
        const int sixteen = w * 2 + (lane & 1), e = (ahead_i + (lane >> 1)) * PG + sixteen / SPP;
        const int2 at = e < ahead.n_units ? i4_resolve(p, ahead, ahead.first_page + e, (sixteen % SPP) * 16, 16) : make_int2(0, 0);
        b_src = pages + at.x * p.stride_page + ahead.kh * p.stride_head + (sixteen % SPP) * 16 * p.stride_tok;
        b_scale = scales + ((static_cast<int64_t>(at.x) * p.Hkv + ahead.kh) * GP + (sixteen % SPP) * 16) * RUNS;
        b_valid = at.y;
        // The sixteen groups after these into L2, a row per prefetch: the one group that registers hold in flight covers a hit there, not
        // memory (eight prompts of 32,768 tokens, a block of 32: 198 -> 183 us, over several input sets 207 -> 200).  148 CTAs x 2 tensors x 144 KB lie in the 126 MB.
        const int f = e + 16 * PG;
        if (f < ahead.n_units) {
          const int2 to = i4_resolve(p, ahead, ahead.first_page + f, (sixteen % SPP) * 16, 16);
          const uint8_t* row = pages + to.x * p.stride_page + ahead.kh * p.stride_head + (sixteen % SPP) * 16 * p.stride_tok;
          const uint8_t* byte = scales + ((static_cast<int64_t>(to.x) * p.Hkv + ahead.kh) * GP + (sixteen % SPP) * 16) * RUNS;
#pragma unroll 4
          for (int t = 0; t < 16; ++t) i4_prefetch(row + t * p.stride_tok);
          i4_prefetch(byte);
        }
        __syncwarp();
      }
      const int from = (ahead_i & 15) * 2;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int n = __shfl_sync(0xffffffffu, b_valid, from + h);
        const uint8_t* src = reinterpret_cast<const uint8_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(b_src), from + h)) + my_src;
        const uint8_t* sat = reinterpret_cast<const uint8_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(b_scale), from + h)) + my_scale;
        (h ? valid.y : valid.x) = n;
#pragma unroll
        for (int j = 0; j < NJ / 2; ++j) {
          // (also past the end, where a page's codes are finite whatever they are and the scale is left out below: a load under a
          // condition would be waited for here)
          x[h * (NJ / 2) + j] = i4_load16(src);
          scale[h * (NJ / 2) + j] = i4_load1(sat + TPJ * j * RUNS);
          src += TPJ * p.stride_tok;
        }
      }
      ++ahead_i;
      return true;
    };
    const int tiles = is_v ? kTcNV : kTcNK;
    const uint32_t full = is_v ? v_full : k_full, free = is_v ? v_free : k_free;
    uint8_t* ring = gen + R * D * 2 + (is_v ? kTcNK * TILE : 0);
    int slot = 0;
    uint32_t parity = 1;
    bool more = fetch();
    for (int g = 0; more; ++g) {
      if (g >= tiles && !wait(free + 8 * slot, parity)) break;
      if (!is_v && lane < 2) meta[(g % kTcMeta) * 8 + w * 2 + lane] = lane ? valid.y : valid.x;
      uint8_t* tile = ring + slot * TILE;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const I4Scale s = i4_scale(tok + TPJ * (j % (NJ / 2)) < (j < NJ / 2 ? valid.x : valid.y) ? scale[j] * 0x00800080u : 0u);
        const uint32_t words[4] = {x[j].x, x[j].y, x[j].z, x[j].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t h[4];
          i4_operands(words[i], s, h);
          const int c = run * 4 + i;
          *reinterpret_cast<uint4*>(tile + (c >> 3) * HS + tc5_sw(w * 32 + TPJ * j + tok, c & 7)) = make_uint4(h[0], h[1], h[2], h[3]);
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");       // the products read the tile through the async proxy
      __syncwarp();
      if (lane == 0) mbar_arrive(full + 8 * slot, 1);
      more = fetch();                                // the next group's, requested as soon as these have been converted
      if (++slot == tiles) { slot = 0; parity ^= 1; }
    }
  } else if (warp == kTcQkWarp) {
    // ================================================================== Q K^T
    const uint32_t qt = warp_uniform(qtile), kr = warp_uniform(kring), idesc = tc5_idesc(R, kTcTok / 2, 0, 0u, 0u);
    I4Piece piece = work.next_piece(work.lo, work.sk0);
    int g = 0;
    for (int n = 0; piece.n_units > 0 && ok; ++n) {
      const int groups = warp_uniform((piece.n_units + PG - 1) / PG);
      if (!wait(q_full, n & 1)) break;
      for (int i = 0; i < groups; ++i, ++g) {
        const int set = g & 1, use = g >> 1, slot = g % kTcNK;
        if (!wait(k_full + 8 * slot, (g / kTcNK) & 1)) break;
#pragma unroll 1
        for (int hf = 0; hf < 2; ++hf) {
          const int mine = set * 2 + hf;
          if (use > 0 && !wait(s_free + 8 * mine, (use - 1) & 1)) break;
          tc5_fence_after();
          if (elect_one()) {
            const uint64_t qd = tc5_desc(qt, 16), kd = tc5_desc(kr + slot * TILE, 16) + hf * 512;      // 64 rows of 128 bytes
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
              const uint32_t at = ((ks >> 2) * HS + (ks & 3) * 32) / 16;
              tc5_mma_ss(tmem + COL_S + mine * 64, qd + at, kd + at, idesc, ks > 0 ? 1u : 0u);
            }
            tc5_commit(s_full + 8 * mine);
            if (hf == 1) tc5_commit(k_free + 8 * slot);
          }
          __syncwarp();
        }
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
        if (!wait(v_full + 8 * slot, (g / kTcNV) & 1)) break;
#pragma unroll 1
        for (int hf = 0; hf < 2; ++hf) {
          const int mine = set * 2 + hf;
          if (!wait(p_full + 8 * mine, (g >> 1) & 1)) break;
          tc5_fence_after();
          if (elect_one()) {
            const uint64_t vd = tc5_desc(vr + slot * TILE, HS) + hf * 512;           // 64 tokens of 128 bytes
            const uint32_t p_col = tmem + COL_S + mine * 64, o_col = tmem + COL_O + set * 128, fresh = i < 2 && hf == 0 ? 0u : 1u;      // the set's first of the piece
#pragma unroll
            for (int ks = 0; ks < kTcTok / 32; ++ks) tc5_mma_ts(o_col, p_col + ks * 8, vd + ks * 128, idesc, ks == 0 ? fresh : 1u);
            if (hf == 1) tc5_commit(v_free + 8 * slot);
            tc5_commit(s_free + 8 * mine);
          }
          __syncwarp();
        }
      }
      piece = work.next_piece(piece.hi, piece.sk);
    }
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
