// Windowed attention on the 5th-generation tensor cores: included by window_attn.cu (same namespace).
//
// A tile has two sets of as many tokens as fit into 128 rows (32 of four heads per KV head), one softmax set of four warps for either (one row per
// tensor-memory lane); a tile whose tokens fit into one is worked on by both sets, which take alternate groups and are joined at its end.  Keys
// come in groups of 128.  A job is a set's work on a group, and jobs go to the sets by turns, across the tiles' ends too:
//   a warp            walks the list and tells the others the pieces; queries and keys by TMA into swizzled tiles, of the pages only those that any row of the tile sees
//   a warp            values likewise (a copy takes its warp 130 cycles to issue, and a group of pages of 32 has eight of either)
//   S[128 x 128] = Q K^T, O[128 x D] += P V   one issuing warp, in the order PV(j), QK(j + 2): the tensor cores run them in order, so that the scores may replace
//                     the weights that were read before without a word from anybody; both operands of Q K^T and V come from shared memory, P from tensor memory
//   softmax set       a row's scores are read twice, for their maximum and for the weights, 32 at a time (whole rows in registers, without a split of the registers between the
//                     warps, were slower: 134 of 170 are in use as it is), masked where the
//                     group is not seen whole; weights go back over the scores as 16-bit operands, in two halves, so that the products of one run while
//                     the other is worked on.  The reference maximum only moves when it would grow by more than 2^8.  Short loops and the special function unit alone: unrolled
//                     whole, with the next 32 scores on their way and a third of the exponentials as polynomials on the FMA units, a prompt of 16,384 tokens took 5 to 8 % longer.
//                     Weights have the values' type, as both operands of a product must: beside bf16 pages each is off by up to 2^-8 of itself (the sum takes them unrounded), outputs are
//                     off by 2.2e-3 where a last rounding alone is 1.7e-3; beside fp16 tiles of quantised pages by 2^-11, and 1.7e-3 remain.
//   a warp            clears the rows of V that no row of the tile sees (they may hold anything), and where rows see different keys, what is
//                     no finite number among them (a weight of zero would not keep it out); the rows that do see it get it at the tile's end
// Measured: a prompt of 16,384 tokens, 32 heads, window 4,096: 1,210 to 1,250 us, by card (777 TFLOP/s, 46 % of the rate of a large library product); ragged prompts of 15,164 tokens, window
// 1,024: 472, from FP8 or 4-bit pages 1,320; eight decoded tokens over 8,192 keys each 65 us (4.1 TB/s), over FP8 caches of up to 16,383 tokens 115.  With the softmax left out a pass over the 16,384 tokens still takes three quarters: what
// bounds it is the chain products -> scores -> weights -> products of either set (each hand-over 100 to 300 cycles) more than any unit: the tensor pipe is busy for 40 %.
// 256 rows a tile because a group's K and V (64 KB) then serve two jobs: with 128 the fill of shared memory alone would be 64 bytes a cycle.
// Tensor memory is full: scores and output of either set, 128 columns each.  Everything is handed on by mbarriers with bounded waits.
// Quantised pages come as they lie, four more warps turn them into fp16 operands, and queries become fp16 under a power of two of their row; there is room for one set's tokens.
#pragma once

constexpr int kWtKeys = 128, kWtSoftWarps = 8;
constexpr int kWtLoadWarp = 8, kWtMmaWarp = 9, kWtFixWarp = 10, kWtValueWarp = 11, kWtConvertWarp = 12;
constexpr float kWtNone = -3.0e38f;                 // reference of a row that has seen no key
constexpr float kWtTau = 8.f, kWtFused = 1048576.f;  // a reference up to this: its product with the scale may be subtracted in one operation
constexpr int kWtAhead = 4, kWtNote = 20;           // pieces told ahead, words of one
template <int FMT, int D, int GP> struct WindowTc {
  static constexpr bool quant = FMT != kRowsBf16;
  using Tiles = RowTiles<128, quant ? 1 : 2, kWtKeys>;
  static constexpr int rows = Tiles::rows, warps = quant ? 16 : 12;
  static constexpr int nk = 2, nv = quant ? 2 : 3, nr = 2;       // tiles of keys, of values; of either as they lie
  static constexpr int tile = kWtKeys * D * 2, qtile = 128 * D * 2;
  static constexpr int raw = quant ? RawTile<FMT, D, GP>::bytes : 0;
  // shared memory: tiles, barriers, [quantised pages: the rows' scales,] notes, exchange between the sets
  static constexpr int bars = rows / 128 * qtile + (nk + nv) * tile + 2 * nr * raw;
  static constexpr int scales = bars + 512, notes = scales + (quant ? 512 : 0), sets = quant ? 0 : notes + kWtAhead * kWtNote * 4;
  static constexpr int smem = notes + kWtAhead * kWtNote * 4 + (quant ? 0 : 2048);       // (quantised pages: the sets meet in the tile of Q, once the products have run)
  static_assert(smem <= 232448, "shared memory");
};

__device__ __forceinline__ void wt_store32(void* at, bool on, const uint32_t (&v)[8]) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %1, 0;\n\t@p st.global.v8.b32 [%0], {%2, %3, %4, %5, %6, %7, %8, %9};\n\t}"
               ::"l"(at), "r"(static_cast<int>(on)), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
__device__ __forceinline__ void wt_store16(void* at, bool on, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %1, 0;\n\t@p st.global.v4.b32 [%0], {%2, %3, %4, %5};\n\t}"
               ::"l"(at), "r"(static_cast<int>(on)), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// A piece as the others are told of it (one that has groups).  Every row sees the keys below all_end, from all_lo on or below the sinks; some row those below end, from lo on.
struct Note {
  int any, kh, s, cu, start, len, token0, tokens, first, last, groups, r_first, r_from, end, lo, all_end, all_lo, joint, flip;      // flip: the set that has the first job, or the first half of the tile
  // a group that some row does not see whole
  __device__ __forceinline__ bool in_part(int key0, int sinks) const { return key0 + kWtKeys > all_end || (key0 < all_lo && key0 + kWtKeys > sinks); }
  __device__ __forceinline__ int key(int i) const { return (i < r_first ? i : r_from + i - r_first) * kWtKeys; }
};
static_assert(sizeof(Note) <= kWtNote * 4, "notes");

template <int FMT, int D, int GP>
__global__ void __launch_bounds__(WindowTc<FMT, D, GP>::warps * 32, 1) window_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                                                                    const __grid_constant__ CUtensorMap map_q, const __grid_constant__ WindowParams p) {
  using Tc = WindowTc<FMT, D, GP>;
  constexpr bool QUANT = Tc::quant;
  constexpr int R = Tc::rows, GT = kWtKeys, TILE = Tc::tile, HS = GT * 128, PG = GT / GP, QTILE = Tc::qtile, QALL = R / 128 * QTILE;
  constexpr int NK = Tc::nk, NV = Tc::nv, NR = Tc::nr, RAW = QALL + (NK + NV) * TILE;
  constexpr uint32_t kType = QUANT ? 0u : 1u;        // operands: fp16, bf16
  constexpr uint32_t COL_S = 0, COL_O = 256;         // tensor-memory columns: scores and outputs of the two sets, 128 each
  extern __shared__ __align__(1024) uint8_t gen[];
  const uint32_t base = smem_u32(gen);
  const uint32_t qtile = base, kring = base + QALL, vring = kring + NK * TILE;
  const uint32_t k_full = base + Tc::bars, k_free = k_full + 8 * NK, v_full = k_free + 8 * NK, v_free = v_full + 8 * NV, v_fixed = v_free + 8 * NV;
  const uint32_t s_full = v_fixed + 8 * NV, p_full = s_full + 16, q_full = p_full + 32, q_free = q_full + 16, o_full = q_free + 16, o_free = o_full + 16, drain = o_free + 16;
  const uint32_t n_full = drain + 8, n_free = n_full + 8 * kWtAhead;
  [[maybe_unused]] const uint32_t r_full = n_free + 8 * kWtAhead, r_free = r_full + 16 * NR;       // [tensor][slot]
  static_assert(8 * (2 * NK + 3 * NV + 15 + 2 * kWtAhead + 4 * NR) <= 400, "barriers");
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + Tc::bars + 400);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(gen + Tc::bars + 404);
  // [kOdd] the last piece (counting from one) that has met what is no finite number.  The warp that looks is at most the V ring
  // ahead of the end of a piece, so a number is read before it is replaced.
  constexpr int kOdd = 8;
  static_assert(kOdd > NV + 1, "pieces ahead");
  volatile int* odd_piece = reinterpret_cast<volatile int*>(gen + Tc::bars + 408);
  float2* exchange = reinterpret_cast<float2*>(gen + Tc::sets);          // [set][128] reference and sum of the sets' rows, at the end of a piece that both sets have
  [[maybe_unused]] float* xs = reinterpret_cast<float*>(gen + Tc::scales);       // [128] quantised pages: what a row's scores are multiplied by
  const int tid = threadIdx.x, lane = tid & 31, warp = warp_uniform(tid >> 5);

  grid_dep_trigger();                                // (the merging kernel comes up beside this one)
  if (tid == 0) {
    for (int i = 0; i < NK; ++i) { mbar_init(k_full + 8 * i, QUANT ? 4 : 1); mbar_init(k_free + 8 * i, 1); }
    if constexpr (QUANT)
      for (int i = 0; i < 2 * NR; ++i) { mbar_init(r_full + 8 * i, 1); mbar_init(r_free + 8 * i, 4); }
    for (int i = 0; i < NV; ++i) { mbar_init(v_full + 8 * i, QUANT ? 4 : 1); mbar_init(v_free + 8 * i, 1); mbar_init(v_fixed + 8 * i, 1); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full + 8 * i, 1);                  // tcgen05.commit after Q K^T (and after the set's P V before it)
      mbar_init(p_full + 16 * i, 4);                 // [set][half]
      mbar_init(p_full + 16 * i + 8, 4);
      mbar_init(q_full + 8 * i, QUANT ? 4 : 1);
      mbar_init(q_free + 8 * i, 1);                  // tcgen05.commit after the tile's last Q K^T
      mbar_init(o_full + 8 * i, 1);                  // tcgen05.commit after a set's last P V of a piece
      mbar_init(o_free + 8 * i, 4);
    }
    mbar_init(drain, 1);
    for (int i = 0; i < kWtAhead; ++i) { mbar_init(n_full + 8 * i, 1); mbar_init(n_free + 8 * i, kWtSoftWarps + 3 + (QUANT ? 4 : 0)); }
    *abort_flag = 0;
    for (int i = 0; i < kOdd; ++i) odd_piece[i] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  grid_dep_wait();
  if (static_cast<int>(blockIdx.x) >= p.plan.head[0]) return;            // (one answer for the CTA)
  __syncwarp();
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "n"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc5_fence_before();
  __syncthreads();
  tc5_fence_after();
  const uint32_t tmem = warp_uniform(*tmem_slot);
  bool ok = true;
  // (written out small: there are dozens of waits, and the loops have to stay in the instruction cache)
  auto wait = [&](uint32_t bar, uint32_t parity) {
    if (ok) {
      const long long t0 = clock64();
      while (!__all_sync(0xffffffffu, mbar_try_wait(bar, parity)))
        if (__any_sync(0xffffffffu, *abort_flag != 0 || clock64() - t0 > p.wait_cycles)) {
          *abort_flag = 1;                           // (reported at the end)
          ok = false;
          break;
        }
    }
    __syncwarp();                                    // (what follows is for whole warps)
    return ok;
  };
  // the next piece, of all warps but the one that walks the list
  int heard = 0;
  auto next = [&]() {
    Note w;
    const int slot = heard % kWtAhead;
    if (!wait(n_full + 8 * slot, (heard / kWtAhead) & 1)) {
      w.any = 0;
      return w;
    }
    ++heard;
    w = *reinterpret_cast<const Note*>(gen + Tc::notes + slot * kWtNote * 4);
    __syncwarp();
    if (lane == 0) mbar_arrive(n_free + 8 * slot, 1);
    __syncwarp();
    return w;
  };

  __syncwarp();
  if (warp < kWtSoftWarps) {
    // ================================================================== softmax: thread = (set, row)
    const int set = warp >> 2, at128 = tid & 127;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_at = tmem + COL_S + set * 128 + lanes, o_at = tmem + COL_O + set * 128 + lanes;
    // The sets meet in pieces that both of them have, and a meeting has no bound.  So all eight warps agree before such a piece, and before they leave the list: one
    // that has given up does not hear of the piece that the others go on to, and takes them with it here.  Within the piece nobody leaves.
    auto all_meet = [&]() {
      __syncwarp();
      asm volatile("bar.sync 1, %0;" ::"n"(kWtSoftWarps * 32) : "memory");
    };
    auto all_go_on = [&](bool mine) {
      uint32_t all;
      __syncwarp();
      asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbar.red.and.pred q, 2, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                   : "=r"(all) : "r"(static_cast<int>(mine)), "n"(kWtSoftWarps * 32) : "memory");
      return all != 0;
    };
    // fp16 weights are taken times 2^7, so that they keep eleven bits down to 2^-21 of a row's largest and are within 2^-32 of it below
    constexpr float kLift = QUANT ? 7.f : 0.f;
    // Quantised pages: queries as fp16 under a power of two of their row, whose largest element comes to 2^14 .. 2^15 (one below 2^-28 of that loses low bits).  Four
    // warps, D / 8 lanes to a row.
    auto write_q = [&](const Note& w) {
      if constexpr (QUANT) {
        if (!w.any || set == 1) return;
        constexpr int LPR = D / 8, RPL = 32 / LPR;
        const int col = lane % LPR;
#pragma unroll 4
        for (int i = 0; i < 32 / RPL; ++i) {
          const int rr = warp * 32 + i * RPL + lane / LPR, t = row_token<128>(p, w.tokens, 0, rr);
          uint4 v = make_uint4(0u, 0u, 0u, 0u);
          if (t >= 0) v = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.q.q) + (static_cast<long long>(w.cu) + w.token0 + t) * p.q.stride + (w.kh * p.c.G + rr % p.c.G) * D + col * 8);
          float x[8], amax = 0.f;
          load8(reinterpret_cast<const __nv_bfloat16*>(&v), x);
#pragma unroll
          for (int k = 0; k < 8; ++k) amax = fmaxf(amax, fabsf(x[k]));
#pragma unroll
          for (int o = 1; o < LPR; o <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
          const int e = max(-100, min(127, static_cast<int>(__float_as_uint(amax) >> 23) - 127));
          const float up = pow2f(14 - e);
          if (col == 0) xs[rr] = p.scale_log2 * pow2f(e - 14);
          *reinterpret_cast<uint4*>(gen + (col >> 3) * HS + tc5_sw(rr, col & 7)) =
              make_uint4(pack_f16(x[0] * up, x[1] * up), pack_f16(x[2] * up, x[3] * up), pack_f16(x[4] * up, x[5] * up), pack_f16(x[6] * up, x[7] * up));
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(q_full, 1);
      }
    };
    Note w = next();
    write_q(w);
    int n = 0, pieces = 0, ends = 0;                 // jobs of this set before; pieces so far, and those in which the set had a job
    while (true) {
      if ((!w.any || w.joint) && !all_go_on(w.any)) break;
      float sc = p.scale_log2;
      const bool both = w.joint;
      const int turn = set ^ w.flip;                 // which half of the tile, or which of every two groups, is this set's
      const int token = row_token<128>(p, w.tokens, both ? 0 : turn, at128);     // this thread's row: -1, there is none
      const bool idle = !__any_sync(0xffffffffu, token >= 0);
      int2 sees = make_int2(0, 0);
      if (token >= 0) sees = keys_of(p.q, Sequence{w.cu, 0, w.start, w.len}, w.start + w.token0 + token);
      float m = kWtNone, l = 0.f;
      const int n0 = n;
      for (int gi = w.first + (both ? turn : 0); gi < w.last; gi += both ? 2 : 1) {
        if (!wait(s_full + 8 * set, n & 1)) break;
        tc5_fence_after();
        if (!idle) {
          if (QUANT && n == n0) sc = xs[at128];
          const int key0 = w.key(gi);
          const bool part = token >= 0 && (key0 + GT > sees.x || (key0 < sees.y && key0 + GT > p.q.sinks));
          const bool any_part = __any_sync(0xffffffffu, part);
          // the scores of 32 keys, -inf where this row does not see one
          auto masked = [&](uint32_t (&x)[32], int c) {
            const int k0 = key0 + c * 32;
            const uint32_t on = low_bits(sees.x - k0) & (~low_bits(sees.y - k0) | low_bits(p.q.sinks - k0));
#pragma unroll
            for (int k = 0; k < 32; ++k) x[k] = (on >> k) & 1u ? x[k] : 0xff800000u;
          };
          float tops[4] = {kWtNone, kWtNone, kWtNone, kWtNone};          // (NaN where there is one)
#pragma unroll 2
          for (int c = 0; c < 4; ++c) {
            uint32_t x[32];
            tc5_ld32_nowait(s_at + c * 32, x);
            tc5_wait_ld();
            tc5_pin32(x);
            if (any_part) masked(x, c);
#pragma unroll
            for (int k = 0; k < 32; k += 8)
#pragma unroll
              for (int i = 0; i < 4; ++i) tops[i] = max_nan(tops[i], __uint_as_float(x[k + 2 * i]), __uint_as_float(x[k + 2 * i + 1]));
          }
          float top = max_nan(max_nan(tops[0], tops[1], tops[2]), tops[3], tops[3]);
          const bool lost = top != top;              // (the exponentials below make the row NaN)
          if (lost) top = m;
          const bool grow = (top - m) * sc > kWtTau || m == kWtNone;     // (none yet: whatever the scale)
          if (__any_sync(0xffffffffu, grow)) {
            const float to = grow ? top : m, f = exp2f((m - to) * sc);
            if (n > n0) {                            // (the products of the job before have run: this job's scores came after them)
              __syncwarp();
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
          // a reference so large that only differences can be scaled: subtracted from the scores first (not an infinite one, whose row is lost)
          float shift = m == kWtNone ? 0.f : kLift - m * sc, less = 0.f;
          const bool apart = __any_sync(0xffffffffu, fabsf(shift) > kWtFused && fabsf(shift) < INFINITY);
          if (apart) {
            less = m == kWtNone ? 0.f : m;
            shift = kLift;
          }
          const float2 scale = make_float2(sc, sc), sh = make_float2(shift, shift);
          float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
          __syncwarp();
          // weights of 32 keys at a time: into the sum, and over the scores that have been read
#pragma unroll 2
          for (int c = 0; c < 4; ++c) {
            uint32_t x[32], h[16];
            tc5_ld32_nowait(s_at + c * 32, x);
            tc5_wait_ld();
            tc5_pin32(x);
            if (any_part) masked(x, c);
            if (apart) {
#pragma unroll
              for (int k = 0; k < 32; ++k) x[k] = __float_as_uint(__uint_as_float(x[k]) - less);
            }
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              float2 e = fma2_f32(make_float2(__uint_as_float(x[2 * k]), __uint_as_float(x[2 * k + 1])), scale, sh);
              e.x = ex2(e.x);
              e.y = ex2(e.y);
              sum[k & 1] = add2_f32(sum[k & 1], e);
              h[k] = QUANT ? pack_f16(e.x, e.y) : pack_b16(e.x, e.y);
            }
            tc5_st16(s_at + c * 16, h);
            if (c & 1) {
              tc5_wait_st();
              tc5_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(p_full + 16 * set + 8 * (c >> 1), 1);
              __syncwarp();
            }
          }
          sum[0] = add2_f32(sum[0], sum[1]);
          l += sum[0].x + sum[0].y;
        } else {
          tc5_fence_before();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(p_full + 16 * set, 1);
            mbar_arrive(p_full + 16 * set + 8, 1);
          }
          __syncwarp();
        }
        ++n;
      }
      // ---- end of the piece
      const bool had = n > n0;
      if (had) wait(o_full + 8 * set, ends++ & 1);
      const float M = m == kWtNone ? -INFINITY : m * sc - kLift;
      float f0 = 1.f, f1 = 0.f, top = M, L = l;      // both sets: what either's output counts
      bool use0 = had && m != kWtNone, use1 = false;
      if (both) {
        if constexpr (QUANT) all_meet();
        const float2 mine = make_float2(M, l);
        exchange[tid] = mine;
        tc5_fence_before();
        all_meet();
        const float2 theirs = exchange[tid ^ 128];
        tc5_fence_after();
        const float2 e0 = set ? theirs : mine, e1 = set ? mine : theirs;
        top = fmaxf(e0.x, e1.x);
        f0 = e0.x == -INFINITY ? 0.f : exp2f(e0.x - top);
        f1 = e1.x == -INFINITY ? 0.f : exp2f(e1.x - top);
        use0 = e0.x != -INFINITY;
        use1 = e1.x != -INFINITY;
        L = top == -INFINITY ? e0.y + e1.y : e0.y * f0 + e1.y * f1;      // (nothing seen: zero, or no number, which stays visible)
      }
      tc5_fence_after();
      ++pieces;
      const bool whole = w.first == 0 && w.last == w.groups, odd = odd_piece[pieces % kOdd] == pieces, on = token >= 0;
      if (!idle) {
        float* record = record_of<R, D>(p, blockIdx.x, w.first == 0);
        const int r = (both ? 0 : turn * 128) + at128;
        const long long out_row = on ? (static_cast<long long>(w.cu) + w.token0 + token) * (p.c.Hkv * p.c.G) + w.kh * p.c.G + at128 % p.c.G : 0;
        const float inv = L == 0.f ? 0.f : 1.f / L;
        const bool wide = (reinterpret_cast<uintptr_t>(p.out) & 31u) == 0;       // (outputs are aligned to 16 bytes)
        // this thread's columns, 16 at a time: all of its set's output, or half of both sets'
        const uint32_t a_at = tmem + COL_O + (both ? 0 : set * 128) + lanes;
        const int nc = both ? D / 32 : D / 16, c0 = both ? set * nc : 0;
        __syncwarp();                                // (the lanes have found their rows each for itself; the loads below need the whole warp)
#pragma unroll 1
        for (int c = c0; c < c0 + nc; ++c) {
          uint32_t a[16], b[16];
          tc5_ld16(a_at + c * 16, a);
          if (both) tc5_ld16(a_at + 128 + c * 16, b);
          float x[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) {             // (an output that was never written holds anything)
            x[k] = use0 ? __uint_as_float(a[k]) * f0 : 0.f;
            if (both && use1) x[k] = fmaf(__uint_as_float(b[k]), f1, x[k]);
          }
          // (stores under a predicate, not a branch: the loads of tensor memory around them need the whole warp)
          if (!whole) {
#pragma unroll
            for (int k = 0; k < 16; k += 8) {
              const uint32_t v[8] = {__float_as_uint(x[k]), __float_as_uint(x[k + 1]), __float_as_uint(x[k + 2]), __float_as_uint(x[k + 3]),
                                     __float_as_uint(x[k + 4]), __float_as_uint(x[k + 5]), __float_as_uint(x[k + 6]), __float_as_uint(x[k + 7])};
              wt_store32(record + 2 * R + r * D + c * 16 + k, on, v);
            }
          } else {
            uint32_t v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = pack_b16(x[2 * i] * inv, x[2 * i + 1] * inv);
            __nv_bfloat16* at = static_cast<__nv_bfloat16*>(p.out) + out_row * D + c * 16;
            if (wide) {
              wt_store32(at, on, v);
            } else {
              wt_store16(at, on, v[0], v[1], v[2], v[3]);
              wt_store16(at + 8, on, v[4], v[5], v[6], v[7]);
            }
          }
          __syncwarp();
        }
        if (on && (!both || set == 0)) {
          if (!whole) {
            record[r] = top;
            record[R + r] = L;
          } else if (p.lse) {
            p.lse[out_row] = L == 0.f ? -INFINITY : (top + log2f(L)) * kLn2;
          }
        }
        if (odd && on) {                             // values that are no finite number, and that this row sees: they were left out of the products
#pragma unroll 1
          for (int gi = w.first; gi < w.last; ++gi) {
            const int key0 = w.key(gi);
            if (!w.in_part(key0, p.q.sinks)) continue;
#pragma unroll 1
            for (int key = key0; key < key0 + GT; ++key) {
              if (!(key < sees.x && (key >= sees.y || key < p.q.sinks))) continue;
              const int page = page_of(p.c, w.s, key / GP, p.status);
              if (page < 0) continue;
#pragma unroll 1
              for (int ch = c0 * 2; ch < (c0 + nc) * 2; ++ch) {
                float v[8];
                cache_load8<FMT, D>(p.c, p.c.v_pages, p.c.v_scale, page, w.kh, key % GP, ch, v);
#pragma unroll 1
                for (int k = 0; k < 8; ++k) {
                  if (fabsf(v[k]) < INFINITY) continue;
                  if (whole) {
                    __nv_bfloat16* at = static_cast<__nv_bfloat16*>(p.out) + out_row * D + ch * 8 + k;
                    *at = __float2bfloat16_rn(__bfloat162float(*at) + v[k]);
                  } else {
                    record[2 * R + r * D + ch * 8 + k] += v[k];
                  }
                }
              }
            }
          }
        }
      }
      __syncwarp();
      tc5_fence_before();
      if (both) all_meet();                          // (the exchange and both outputs have been read)
      __syncwarp();
      if (lane == 0 && had) mbar_arrive(o_free + 8 * set, 1);
      __syncwarp();
      w = next();
      write_q(w);
    }
  } else {
    // The copies of a tensor's pages (v: values), one warp each; behind a piece's first keys its queries, a box per set (a box reaches past the sequence's last token: rows
    // that nobody uses).
    const int per = 128 / p.c.G;
    int g = 0, nq0 = 0, nq1 = 0;                     // groups; boxes of queries begun
    auto load = [&](const Note& w, int first, int last, int v) {
      const int slots = QUANT ? NR : v ? NV : NK;
      const uint32_t full = QUANT ? r_full + 8 * NR * v : v ? v_full : k_full, free = QUANT ? r_free + 8 * NR * v : v ? v_free : k_free;
      int pages = 0;                                 // of the next 32 / PG groups, one per lane; -1: nobody sees it
      [[maybe_unused]] float scale = 0.f;            // FP8: theirs
      for (int gi = first; gi < last; ++gi, ++g) {
        if (g >= p.copies) {
          *abort_flag = 1;
          ok = false;
          return false;
        }
        const int i = (gi - first) % (32 / PG), slot = g % slots, turns = g / slots;
        if (i == 0) {
          const int mine = gi + lane / PG, key = mine < last ? w.key(mine) + (lane % PG) * GP : w.end;
          pages = -1;
          if (key < w.end && (key + GP > w.lo || key < p.q.sinks)) pages = max(0, page_of(p.c, w.s, key / GP, p.status));
          if (FMT == kRowsFp8 && pages >= 0) scale = static_cast<const float*>(v ? p.c.v_scale : p.c.k_scale)[static_cast<size_t>(pages) * p.c.Hkv + w.kh];
          __syncwarp();
        }
        if (turns > 0 && !wait(free + 8 * slot, (turns - 1) & 1)) return false;
        if constexpr (QUANT) {
          raw_load<FMT, D, GP>(p.c, v ? &map_v : &map_k, v ? p.c.v_scale : p.c.k_scale, w.kh, pages, scale, i * PG, base + RAW + (v * NR + slot) * Tc::raw, full + 8 * slot);
        } else {
          const uint32_t have = __ballot_sync(0xffffffffu, pages >= 0) >> (i * PG) & ((1u << PG) - 1u);
          if (elect_one()) mbar_expect_tx(full + 8 * slot, __popc(have) * (GP * D * 2));
          __syncwarp();
          if (lane / PG == i && pages >= 0) {
            const uint32_t dst = (v ? vring : kring) + slot * TILE + (lane % PG) * (GP * 128);
#pragma unroll
            for (int h = 0; h < D / 64; ++h) tma_load_page(dst + h * HS, v ? &map_v : &map_k, full + 8 * slot, h * 64, w.kh, pages);
          }
          __syncwarp();
          if (v == 0 && gi == first) {
#pragma unroll 1
            for (int t = 0; t < (w.joint ? 1 : 2); ++t) {
              const int before = t ? nq1 : nq0;
              if (before > 0 && !wait(q_free + 8 * t, (before - 1) & 1)) { ++g; return false; }
              t ? ++nq1 : ++nq0;
              if (elect_one()) {
                mbar_expect_tx(q_full + 8 * t, per * p.c.G * D * 2);
#pragma unroll
                for (int h = 0; h < D / 64; ++h) tma_load_queries(qtile + t * QTILE + h * HS, &map_q, q_full + 8 * t, h * 64, w.kh * p.c.G, w.cu + w.token0 + t * per);
              }
              __syncwarp();
            }
          }
        }
      }
      return ok;
    };
    // What is in flight has landed before the CTA's shared memory is given up.  Whoever gave up: another warp's wait may have run out when this one has begun its last
    // copies and has nothing left to wait for.
    auto settle = [&]() {
      const int v = warp == kWtValueWarp, slots = QUANT ? NR : v ? NV : NK;
      const uint32_t full = QUANT ? r_full + 8 * NR * v : v ? v_full : k_full;
      for (int i = 0; i < min(slots, g); ++i) mbar_drain(full + 8 * i, ((g - 1 - i) / slots) & 1);
      if (!QUANT && nq0 > 0) mbar_drain(q_full, (nq0 - 1) & 1);
      if (!QUANT && nq1 > 0) mbar_drain(q_full + 8, (nq1 - 1) & 1);
      __syncwarp();
    };
    if (warp == kWtLoadWarp) {
      // ================================================================== the list; queries, pages
      Walk walk(p, blockIdx.x);
      int told = 0, jobs = 0;                        // pieces told; jobs before
      while (ok) {
        const Piece piece = next_piece<typename Tc::Tiles, GT>(walk);
        if (piece.any && piece.groups == 0) {        // tokens that see nothing: nobody else has to know
          for (int t = 0; t < piece.tokens; ++t) {
            const long long row = token_head(p, piece.x, piece.token0 + t, piece.kh, 0);
            for (int i = lane; i < p.c.G * (D / 8); i += 32) reinterpret_cast<uint4*>(p.out)[row * (D / 8) + i] = make_uint4(0u, 0u, 0u, 0u);
            if (lane < p.c.G && p.lse) p.lse[row + lane] = -INFINITY;
          }
          __syncwarp();
          continue;
        }
        Note w;
        w.any = piece.any;
        if (piece.any) {
          w.kh = piece.kh;
          w.s = piece.s;
          w.cu = piece.x.cu;
          w.start = piece.x.start;
          w.len = piece.x.len;
          w.token0 = piece.token0;
          w.tokens = piece.tokens;
          w.first = piece.first;
          w.last = piece.last;
          w.groups = piece.groups;
          w.r_first = piece.r.first;
          w.r_from = piece.r.from;
          w.end = piece.r.end;
          w.lo = piece.r.lo;
          w.all_end = keys_of(p.q, piece.x, piece.x.start + piece.token0).x;
          w.all_lo = keys_of(p.q, piece.x, piece.x.start + piece.token0 + piece.tokens - 1).y;
          w.joint = piece.tokens <= per;             // its tokens fit into a set: both sets'
          w.flip = jobs & 1;
          jobs += (w.last - w.first) * (w.joint ? 1 : 2);
        }
        const int note = told % kWtAhead;
        if (told >= kWtAhead && !wait(n_free + 8 * note, (told / kWtAhead - 1) & 1)) break;
        if (lane == 0) {
          *reinterpret_cast<Note*>(gen + Tc::notes + note * kWtNote * 4) = w;
          mbar_arrive(n_full + 8 * note, 1);
        }
        __syncwarp();
        ++told;
        if (!w.any) break;
        if (!load(w, w.first, w.last, 0)) break;
      }
      settle();
    } else if (warp == kWtValueWarp) {
      // ================================================================== values
      for (Note w = next(); w.any && ok; w = next())
        if (!load(w, w.first, w.last, 1)) break;
      settle();
    } else if (warp == kWtMmaWarp) {
      // ================================================================== products: PV(j), QK(j + 2)
      const uint32_t qt = warp_uniform(qtile), kr = warp_uniform(kring), vr = warp_uniform(vring);
      const uint32_t id_qk = tc5_idesc(128, GT, 0, kType, kType), id_pv = tc5_idesc(128, D, 1, kType, kType);
      // the next Q K^T: group gq of all, job jq of `jobs` of the piece
      int gq = 0, jq = 0, jobs = 0, q0 = 0, q1 = 0;
      bool both = false, more = true;
      // what P V of either set's job in flight needs: 1 the set's first of the piece, 2 its last, 4 the group's last, 8 the group's first; -1 none
      int todo0 = -1, todo1 = -1, ends0 = 0, ends1 = 0, gp = 0;
      auto issue_qk = [&](int set, int& todo, bool cross) {
        todo = -1;
        if (jq == jobs && !cross) return;
        if (more && jq == jobs) {                    // the next piece
          const Note w = next();
          more = warp_uniform(w.any) != 0 && ok;
          both = warp_uniform(w.joint) != 0;
          jobs = more ? warp_uniform(w.last - w.first) * (both ? 1 : 2) : 0;
          jq = 0;
        }
        if (!more) return;
        const int t = both ? 0 : jq & 1, slot = gq % NK;
        const bool tile_first = jq < (both ? 1 : 2), tile_last = jq >= jobs - (both ? 1 : 2), group_first = both || t == 0, group_last = both || t == 1;
        if (tile_first && !(t ? wait(q_full + 8, q1++ & 1) : wait(q_full, q0++ & 1))) return;
        if (group_first && !wait(k_full + 8 * slot, (gq / NK) & 1)) return;
        tc5_fence_after();
        const uint32_t q_at = qt + t * QTILE, k_at = kr + slot * TILE, s_col = tmem + COL_S + set * 128;
        if (elect_one()) {
          const uint64_t qd = tc5_desc(q_at, 16), kd = tc5_desc(k_at, 16);
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            const uint32_t at = ((ks >> 2) * HS + (ks & 3) * 32) / 16;
            tc5_mma_ss(s_col, qd + at, kd + at, id_qk, ks > 0 ? 1u : 0u);
          }
          tc5_commit(s_full + 8 * set);
          if (group_last) tc5_commit(k_free + 8 * slot);
          if (!QUANT && tile_last) tc5_commit(q_free + 8 * t);
        }
        __syncwarp();
        // (a set's first and last jobs of a piece are among the piece's first two and last two)
        todo = (jq < 2 ? 1 : 0) | (jq >= jobs - 2 ? 2 : 0) | (group_last ? 4 : 0) | (group_first ? 8 : 0);
        ++jq;
        if (group_last) ++gq;
      };
      // Quantised pages: the queries of the next piece are written when this one has ended, so its products are not begun before.
      for (int j = 0; ok; ++j) {
        const int set = j & 1;
        if (j == 0 || (QUANT && (set ? todo1 : todo0) < 0)) {            // (jobs take turns: the other set has none either)
          if (set) issue_qk(1, todo1, true); else issue_qk(0, todo0, true);
          if (set) issue_qk(0, todo0, !QUANT); else issue_qk(1, todo1, !QUANT);
        }
        const int todo = set ? todo1 : todo0, slot = gp % NV;
        if (todo < 0) break;
        if ((todo & 8) && (!wait(v_full + 8 * slot, (gp / NV) & 1) || !wait(v_fixed + 8 * slot, (gp / NV) & 1))) break;
        if (todo & 1) {                              // the set's last output has been read
          const int e = set ? ends1 : ends0;
          if (e > 0 && !wait(o_free + 8 * set, (e - 1) & 1)) break;
          set ? ++ends1 : ++ends0;
        }
        const uint32_t v_at = vr + slot * TILE, s_col = tmem + COL_S + set * 128, go_on = todo & 1 ? 0u : 1u;
#pragma unroll 1
        for (int hf = 0; hf < 2; ++hf) {
          if (!wait(p_full + 16 * set + 8 * hf, (j >> 1) & 1)) break;
          tc5_fence_after();
          if (elect_one()) {
            const uint64_t vd = tc5_desc(v_at, HS) + hf * 512;                   // 64 tokens of 128 bytes
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) tc5_mma_ts(s_col + (COL_O - COL_S), s_col + hf * 32 + ks * 8, vd + ks * 128, id_pv, ks > 0 || hf > 0 ? 1u : go_on);
            if (hf == 1) {
              if (todo & 4) tc5_commit(v_free + 8 * slot);
              if (todo & 2) tc5_commit(o_full + 8 * set);
            }
          }
          __syncwarp();
        }
        if (todo & 4) ++gp;
        if (set) issue_qk(1, todo1, !QUANT); else issue_qk(0, todo0, !QUANT);
      }
      // the products in flight have run before tensor memory is given back
      if (elect_one()) {
        tc5_commit(drain);
        mbar_drain(drain, 0);
      }
      __syncwarp();
    } else if (warp == kWtFixWarp) {
      // ================================================================== values that must not count
      int g = 0, pieces = 0;
      for (Note w = next(); w.any && ok; w = next()) {
        ++pieces;
        const bool same = w.all_end == w.end && w.all_lo == w.lo;        // every row sees the same keys
        for (int gi = w.first; gi < w.last; ++gi, ++g) {
          const int key0 = w.key(gi), slot = g % NV;
          if (!wait(v_full + 8 * slot, (g / NV) & 1)) break;
          if (w.in_part(key0, p.q.sinks)) {
            uint8_t* tile = gen + QALL + (NK + slot) * TILE;
            bool odd = false;
            // 16 bytes per lane, four 128-byte rows of the tile at a time
#pragma unroll 2
            for (int t = 0; t < GT; t += 4) {
              const int row = t + (lane >> 3), key = key0 + row;
              const bool live = key < w.end && (key >= w.lo || key < p.q.sinks);
#pragma unroll
              for (int h = 0; h < D / 64; ++h) {
                uint4* at = reinterpret_cast<uint4*>(tile + h * HS + row * 128 + (lane & 7) * 16);
                if (!live) {
                  *at = make_uint4(0u, 0u, 0u, 0u);
                } else if (!same) {
                  uint4 v = *at;
                  const uint32_t old[4] = {v.x, v.y, v.z, v.w};
                  uint32_t u[4];
#pragma unroll
                  for (int k = 0; k < 4; ++k) {
                    constexpr uint32_t kExp = QUANT ? 0x7c00u : 0x7f80u;
                    u[k] = (old[k] & kExp) == kExp ? old[k] & 0xffff0000u : old[k];
                    u[k] = (u[k] & (kExp << 16)) == kExp << 16 ? u[k] & 0x0000ffffu : u[k];
                  }
                  if (u[0] != old[0] || u[1] != old[1] || u[2] != old[2] || u[3] != old[3]) {
                    *at = make_uint4(u[0], u[1], u[2], u[3]);
                    odd = true;
                  }
                }
              }
            }
            if (__any_sync(0xffffffffu, odd) && lane == 0) odd_piece[pieces % kOdd] = pieces;
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // the products read the tile through the async proxy
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(v_fixed + 8 * slot, 1);
          __syncwarp();
        }
      }
    } else if (warp >= kWtConvertWarp) {
      // ================================================================== quantised pages into operands
      if constexpr (QUANT) {
        int g = 0;
        for (Note w = next(); w.any && ok; w = next()) {
          for (int gi = w.first; gi < w.last && ok; ++gi, ++g) {
#pragma unroll 1
            for (int v = 0; v < 2; ++v) {
              const int slot = g % NR, to = v ? g % NV : g % NK;
              const uint32_t full = (v ? v_full : k_full) + 8 * to, free = (v ? v_free : k_free) + 8 * to;
              const int turns = v ? g / NV : g / NK;
              if (!wait(r_full + 8 * (v * NR + slot), (g / NR) & 1)) break;
              if (turns > 0 && !wait(free, (turns - 1) & 1)) break;
              raw_convert<FMT, D, GP, true>(gen + RAW + (v * NR + slot) * Tc::raw, gen + QALL + ((v ? NK : 0) + to) * TILE, tid - kWtConvertWarp * 32);
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // the products read the tile through the async proxy
              __syncwarp();
              if (lane == 0) {
                mbar_arrive(full, 1);
                mbar_arrive(r_free + 8 * (v * NR + slot), 1);
              }
              __syncwarp();
            }
          }
        }
      }
    }
  }
  tc5_fence_before();
  __syncthreads();
  if (tid == 0 && *abort_flag) set_status(p.status, LOSA_ERR_TIMEOUT);
  __syncwarp();
  if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
}
