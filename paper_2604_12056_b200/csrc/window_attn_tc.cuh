// Windowed attention on the 5th-generation tensor cores: included by window_attn.cu (same namespace).
//
// A tile has 256 rows (64 tokens of four heads per KV head), one softmax set of four warps for 128 of them each (one row per
// tensor-memory lane); a tile of at most 128 rows is worked on by both sets, which take alternate groups and are joined at its end.  Keys
// come in groups of 128:
//   a warp            pages by TMA into rings of swizzled K and V tiles, only those that any row of the tile sees
//   S[128 x 128] = Q K^T   an issuing warp; both operands from shared memory
//   softmax set       a row's 128 scores in registers, masked where the group is not seen whole; weights go back over the scores as 16-bit operands, in two halves, so
//                     that the products of one run while the other is worked on.  The reference maximum only moves when it would grow by more than 2^8.
//   O[128 x D] += P V      another issuing warp; A = P from tensor memory, B = values as they lie
//   a warp            clears the rows of V that no row of the tile sees (they may hold anything), and where rows see different keys, what is
//                     no finite number among them (a weight of zero would not keep it out); the rows that do see it get it at the tile's end
// Tensor memory is full: scores and output of either set, 128 columns each.  Everything is handed on by mbarriers with bounded waits.
#pragma once

constexpr int kWtKeys = 128, kWtSoftWarps = 8;
constexpr int kWtLoadWarp = 8, kWtQkWarp = 9, kWtPvWarp = 10, kWtFixWarp = 11, kWtConvertWarp = 12;
constexpr float kWtNone = -3.0e38f;                 // reference of a row that has seen no key
constexpr float kWtTau = 8.f, kWtFused = 1048576.f;  // a reference up to this: its product with the scale may be subtracted in one operation
// Quantised pages leave room for half the rows, and four more warps.
template <int FMT, int D, int GP> struct WindowTc {
  static constexpr bool quant = FMT != kRowsBf16;
  static constexpr int rows = quant ? 128 : 256, warps = quant ? 16 : 12;
  static constexpr int nk = 2, nv = quant ? 2 : 3, nr = 2;       // tiles of keys, of values; of either as they lie
  // registers per thread at the launch, and as they are dealt out
  static constexpr int launch_regs = quant ? 128 : 168, soft_regs = quant ? 184 : 208, other_regs = quant ? 72 : 80;
  static_assert(kWtSoftWarps * soft_regs + (warps - kWtSoftWarps) * other_regs <= warps * launch_regs, "registers");
  static constexpr int tile = kWtKeys * D * 2, qtile = 128 * D * 2;
  static constexpr int raw = quant ? RawTile<FMT, D, GP>::bytes : 0;
  static constexpr int tail = rows / 128 * qtile + (nk + nv) * tile + 2 * nr * raw;       // where the barriers lie
  static constexpr int smem = 1024 + tail + 512 + (quant ? 512 : 0);
  static_assert(smem <= 232448, "shared memory");
};

__device__ __forceinline__ void wt_store16(void* at, bool on, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %1, 0;\n\t@p st.global.v4.b32 [%0], {%2, %3, %4, %5};\n\t}"
               ::"l"(at), "r"(static_cast<int>(on)), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
// What the rows of a piece have in common: every row sees the keys below `end`, from `lo` on or below the sinks.
struct Common { int end, lo; bool same; };
__device__ __forceinline__ Common common_of(const WindowParams& p, const Piece& w) {
  const int first = keys_of(p.q, w.x, w.x.start + w.row0 / p.c.G).x, last = keys_of(p.q, w.x, w.x.start + (w.row0 + w.rows - 1) / p.c.G).y;
  return {first, last, first == w.r.end && last == w.r.lo};
}
// A piece without any group is the softmax warps' alone: nothing is handed on for it (they could run ahead of the others' barriers by any number of them).
// One of at most 128 rows is both sets'.
__device__ __forceinline__ bool filled(const Piece& w) { return w.last > w.first; }
__device__ __forceinline__ bool joint(const Piece& w) { return w.rows <= 128 && filled(w); }
// a group that some row of the piece does not see whole
__device__ __forceinline__ bool in_part(const WindowParams& p, const Common& c, int key0) {
  return key0 + kWtKeys > c.end || (key0 < c.lo && key0 + kWtKeys > p.q.sinks);
}

template <int FMT, int D, int GP>
__global__ void __launch_bounds__(WindowTc<FMT, D, GP>::warps * 32, 1) window_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                                                                    const __grid_constant__ WindowParams p) {
  using Tc = WindowTc<FMT, D, GP>;
  constexpr bool QUANT = Tc::quant;
  constexpr int R = Tc::rows, GT = kWtKeys, TILE = Tc::tile, HS = GT * 128, PG = GT / GP, QTILE = Tc::qtile, TAIL = Tc::tail, QALL = R / 128 * QTILE;
  constexpr int kWtNK = Tc::nk, kWtNV = Tc::nv, NR = Tc::nr;
  constexpr uint32_t kType = QUANT ? 0u : 1u;        // operands: fp16, bf16
  constexpr uint32_t COL_S = 0, COL_O = 256;         // tensor-memory columns: scores and outputs of the two sets, 128 each
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const uint32_t qtile = base, kring = base + QALL, vring = kring + kWtNK * TILE;
  [[maybe_unused]] constexpr int RAW = QALL + (kWtNK + kWtNV) * TILE;       // quantised pages as they lie: [tensor][slot]
  const uint32_t bars = base + TAIL;
  const uint32_t k_full = bars, k_free = k_full + 8 * kWtNK, v_full = k_free + 8 * kWtNK, v_free = v_full + 8 * kWtNV, v_fixed = v_free + 8 * kWtNV;
  const uint32_t s_full = v_fixed + 8 * kWtNV, s_free = s_full + 16, p_full = s_free + 16, q_full = p_full + 32, o_free = q_full + 16, drain = o_free + 16;
  [[maybe_unused]] const uint32_t r_full = drain + 16, r_free = r_full + 16 * NR;       // [tensor][slot]
  static_assert(8 * (2 * kWtNK + 3 * kWtNV + 2 + 2 + 4 + 2 + 2 + 2 + 4 * NR) <= 320, "barriers");
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + TAIL + 320);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(gen + TAIL + 324);
  // [kOdd] the last piece (counting from one those that have groups) that has met what is no finite number.  The warp that looks is at most the V ring
  // ahead of the end of a piece, so a number is read before it is replaced.
  constexpr int kOdd = 8;
  static_assert(kOdd > kWtNV + 1, "pieces ahead");
  volatile int* odd_piece = reinterpret_cast<volatile int*>(gen + TAIL + 328);
  // [set][128] reference, sum: at the end of a piece that both sets have.  It lies in the second tile of Q, which is not in use then, or in the only one, once
  // both sets' products have run.
  float* xm = reinterpret_cast<float*>(gen + (QUANT ? 0 : QTILE));
  float* xl = xm + 256;
  [[maybe_unused]] float* xs = reinterpret_cast<float*>(gen + TAIL + 512);       // [128] quantised pages: what a row's scores are multiplied by
  const int tid = threadIdx.x, lane = tid & 31, warp = warp_uniform(tid >> 5);

  grid_dep_trigger();                                // (the merging kernel comes up beside this one)
  if (tid == 0) {
    for (int i = 0; i < kWtNK; ++i) { mbar_init(k_full + 8 * i, QUANT ? 4 : 1); mbar_init(k_free + 8 * i, 1); }
    if constexpr (QUANT)
      for (int i = 0; i < 2 * NR; ++i) { mbar_init(r_full + 8 * i, 1); mbar_init(r_free + 8 * i, 4); }
    for (int i = 0; i < kWtNV; ++i) { mbar_init(v_full + 8 * i, QUANT ? 4 : 1); mbar_init(v_free + 8 * i, 1); mbar_init(v_fixed + 8 * i, 1); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full + 8 * i, 1);                  // tcgen05.commit after Q K^T
      mbar_init(s_free + 8 * i, 1);                  // tcgen05.commit after P V: the scores may be replaced, the set's output holds them
      mbar_init(q_full + 8 * i, 4);
      mbar_init(o_free + 8 * i, 4);
      mbar_init(drain + 8 * i, 1);
    }
    for (int i = 0; i < 4; ++i) mbar_init(p_full + 8 * i, 4);            // [set][half]
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
  // a bound shorter than a look at a barrier takes has run out by then (which is how the way out is exercised)
  bool ok = p.wait_cycles >= kLookCycles;
  if (!ok && tid == 0) set_status(p.status, LOSA_ERR_TIMEOUT);
  auto wait = [&](uint32_t bar, uint32_t parity) {
    if (ok) ok = warp_mbar_wait(bar, parity, abort_flag, p.status, p.wait_cycles);
    __syncwarp();                                    // (what follows is for whole warps)
    return ok;
  };
  Walk walk(p, blockIdx.x);
  auto next = [&]() { return next_piece<R, GT>(walk); };

  __syncwarp();
  if (warp < kWtSoftWarps) {
    // ================================================================== softmax: thread = (set, row)
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Tc::soft_regs));
    const int set = warp >> 2, at128 = tid & 127;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_at = tmem + COL_S + set * 128 + lanes, o_at = tmem + COL_O + set * 128 + lanes;
    auto all_meet = [&]() {
      __syncwarp();
      asm volatile("bar.sync 1, %0;" ::"n"(kWtSoftWarps * 32) : "memory");
    };
    // fp16 weights are taken times 2^7, so that they keep eleven bits down to 2^-21 of a row's largest and are within 2^-32 of it below
    constexpr float kLift = QUANT ? 7.f : 0.f;
    // ... and queries times a power of two of their row, whose largest element comes to 2^14 .. 2^15 (one below 2^-28 of that loses low bits)
    // this thread's row of Q into the set's tile
    auto write_q = [&](const Piece& w) {
      if (!w.any || !filled(w)) return;
      const bool both = joint(w);
      if (both && set == 1) return;
      const int r = set * 128 + at128;
      if (set * 128 + (warp & 3) * 32 < w.rows) {
        const int row = w.row0 + r, t = row / p.c.G;
        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(p.q.q) + (static_cast<long long>(w.x.cu) + t) * p.q.stride + (w.kh * p.c.G + row - t * p.c.G) * D;
        if constexpr (QUANT) {
          uint4 v[D / 8];
          float amax = 0.f;
#pragma unroll
          for (int c = 0; c < D / 8; ++c) v[c] = r < w.rows ? *reinterpret_cast<const uint4*>(src + c * 8) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
          for (int c = 0; c < D / 8; ++c) {
            float x[8];
            load8(reinterpret_cast<const __nv_bfloat16*>(&v[c]), x);
#pragma unroll
            for (int k = 0; k < 8; ++k) amax = fmaxf(amax, fabsf(x[k]));
          }
          const int e = max(-100, min(127, static_cast<int>(__float_as_uint(amax) >> 23) - 127));
          const float up = pow2f(14 - e);
          xs[at128] = p.scale_log2 * pow2f(e - 14);
#pragma unroll
          for (int c = 0; c < D / 8; ++c) {
            float x[8];
            load8(reinterpret_cast<const __nv_bfloat16*>(&v[c]), x);
            *reinterpret_cast<uint4*>(gen + (c >> 3) * HS + tc5_sw(at128, c & 7)) =
                make_uint4(pack_f16(x[0] * up, x[1] * up), pack_f16(x[2] * up, x[3] * up), pack_f16(x[4] * up, x[5] * up), pack_f16(x[6] * up, x[7] * up));
          }
        } else {
#pragma unroll
          for (int c = 0; c < D / 8; ++c) {
            const uint4 v = r < w.rows ? *reinterpret_cast<const uint4*>(src + c * 8) : make_uint4(0u, 0u, 0u, 0u);
            *reinterpret_cast<uint4*>(gen + set * QTILE + (c >> 3) * HS + tc5_sw(at128, c & 7)) = v;
          }
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(q_full + 8 * set, 1);
    };
    Piece w = next();
    write_q(w);
    int n = 0, pieces = 0;                           // jobs of this set before; pieces with groups so far
    while (w.any) {
      float sc = p.scale_log2;
      const bool both = joint(w);
      const int r = (both ? 0 : set * 128) + at128;
      const bool idle = r - lane >= w.rows;          // none of the warp's rows exists
      const int2 sees = r < w.rows ? keys_of(p.q, w.x, w.x.start + (w.row0 + r) / p.c.G) : make_int2(0, 0);
      float m = kWtNone, l = 0.f;
      const int n0 = n;
      for (int gi = w.first + (both ? set : 0); gi < w.last; gi += both ? 2 : 1) {
        if (!wait(s_full + 8 * set, n & 1)) break;
        tc5_fence_after();
        if (!idle) {
          if (QUANT && n == n0) sc = xs[at128];
          uint32_t x[128];
#pragma unroll
          for (int c = 0; c < 4; ++c) tc5_ld32_nowait(s_at + c * 32, x + c * 32);
          const int key0 = group_key<GT>(w.r, gi);
          const bool part = r < w.rows && (key0 + GT > sees.x || (key0 < sees.y && key0 + GT > p.q.sinks));
          const bool any_part = __any_sync(0xffffffffu, part);
          tc5_wait_ld();
#pragma unroll
          for (int c = 0; c < 4; ++c) tc5_pin32(x + c * 32);
          auto score = [&](int k) { return __uint_as_float(x[k]); };
          if (any_part) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const int k0 = key0 + c * 32;
              const uint32_t on = low_bits(sees.x - k0) & (~low_bits(sees.y - k0) | low_bits(p.q.sinks - k0));
#pragma unroll
              for (int k = 0; k < 32; ++k) x[c * 32 + k] = (on >> k) & 1u ? x[c * 32 + k] : 0xff800000u;       // -inf: no weight
            }
          }
          float top = kWtNone, top2 = kWtNone;
#pragma unroll
          for (int k = 0; k < 128; k += 4) {
            top = max3_f32(top, score(k), score(k + 1));
            top2 = max3_f32(top2, score(k + 2), score(k + 3));
          }
          top = fmaxf(top, top2);
          const bool grow = (top - m) * sc > kWtTau || m == kWtNone;       // (none yet: whatever the scale)
          if (__any_sync(0xffffffffu, grow)) {
            const float to = grow ? top : m, f = exp2f((m - to) * sc);
            if (n > n0) {                            // (the products of the job before have run: this job's scores came after them)
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
          const float shift = m == kWtNone ? 0.f : kLift - m * sc;
          // a reference so large that only differences can be scaled: subtracted from the scores first (not an infinite one, whose row is lost)
          const bool apart = __any_sync(0xffffffffu, fabsf(shift) > kWtFused && fabsf(shift) < INFINITY);
          if (apart) {
#pragma unroll
            for (int k = 0; k < 128; ++k) x[k] = __float_as_uint(score(k) - (m == kWtNone ? 0.f : m));
          }
          const float2 scale = make_float2(sc, sc), sh = apart ? make_float2(kLift, kLift) : make_float2(shift, shift);
          float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            uint32_t h[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              float2 e = fma2_f32(make_float2(score(c * 32 + 2 * k), score(c * 32 + 2 * k + 1)), scale, sh);
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
              if (lane == 0) mbar_arrive(p_full + 8 * (set * 2 + (c >> 1)), 1);
              __syncwarp();
            }
          }
          sum[0] = add2_f32(sum[0], sum[1]);
          l += sum[0].x + sum[0].y;
        } else {
          tc5_fence_before();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(p_full + 8 * (set * 2), 1);
            mbar_arrive(p_full + 8 * (set * 2 + 1), 1);
          }
        }
        ++n;
      }
      // ---- end of the piece
      if (n > n0) wait(s_free + 8 * set, (n - 1) & 1);
      const float M = m == kWtNone ? -INFINITY : m * sc - kLift;
      float f0 = 1.f, f1 = 0.f, top = M, L = l;      // both sets: what either's output counts
      bool use0 = n > n0 && m != kWtNone, use1 = false;
      if (both) {
        if constexpr (QUANT) {
          tc5_fence_before();
          all_meet();
          tc5_fence_after();
        }
        xm[set * 128 + at128] = M;
        xl[set * 128 + at128] = l;
        tc5_fence_before();
        all_meet();
        const float m0 = xm[at128], m1 = xm[128 + at128];
        top = fmaxf(m0, m1);
        f0 = m0 == -INFINITY ? 0.f : exp2f(m0 - top);
        f1 = m1 == -INFINITY ? 0.f : exp2f(m1 - top);
        use0 = m0 != -INFINITY;
        use1 = m1 != -INFINITY;
        L = xl[at128] * f0 + xl[128 + at128] * f1;
        if (top == -INFINITY) L = xl[at128] + xl[128 + at128];       // (zero, or no number, which stays visible)
      }
      tc5_fence_after();
      const Piece following = next();
      const bool q_now = !both || (!QUANT && joint(following));      // (else the exchange lies where the tile goes)
      if (q_now) write_q(following);
      if (filled(w)) ++pieces;
      const bool whole = w.whole(), odd = filled(w) && odd_piece[pieces % kOdd] == pieces;
      __syncwarp();
      if (!idle) {
        const bool on = r < w.rows;
        float* record = record_of<R, D>(p, blockIdx.x, w.first == 0);
        const long long out_row = on ? token_head(p, w, r) : 0;
        const float inv = L == 0.f ? 0.f : 1.f / L;
        const uint32_t a_at = tmem + COL_O + (both ? 0 : set * 128) + lanes;
        const int c0 = both ? set * (D / 32) : 0, c1 = both ? c0 + D / 32 : D / 16;      // columns, sixteen at a time
        __syncwarp();                                // (the lanes have found their rows each for itself; the loads below need the whole warp)
#pragma unroll 1
        for (int c = c0; c < c1; ++c) {
          uint32_t a[16], b[16];
          tc5_ld16(a_at + c * 16, a);
          if (both) tc5_ld16(a_at + 128 + c * 16, b);
          float x[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) {             // (an output that was never written holds anything)
            x[k] = use0 ? __uint_as_float(a[k]) * f0 : 0.f;
            if (both && use1) x[k] = fmaf(__uint_as_float(b[k]), f1, x[k]);
          }
          if (odd && on) {                           // values that are no finite number, and that this row sees: they were left out of the products
            const Common com = common_of(p, w);
            for (int gi = w.first; gi < w.last; ++gi) {
              const int key0 = group_key<GT>(w.r, gi);
              if (!in_part(p, com, key0)) continue;
              for (int key = key0; key < key0 + GT; ++key) {
                if (!(key < sees.x && (key >= sees.y || key < p.q.sinks))) continue;
                const int page = page_of(p.c, w.s, key / GP, p.status);
                if (page < 0) continue;
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
                  float v[8];
                  cache_load8<FMT, D>(p.c, p.c.v_pages, p.c.v_scale, page, w.kh, key % GP, c * 2 + h, v);
#pragma unroll
                  for (int k = 0; k < 8; ++k)
                    if (!(fabsf(v[k]) < INFINITY)) {
                      if (h == 0) x[k] += v[k]; else x[8 + k] += v[k];
                    }
                }
              }
            }
          }
          __syncwarp();
          // (stores under a predicate, not a branch: the loads of tensor memory around them need the whole warp)
          if (!whole) {
#pragma unroll
            for (int k = 0; k < 16; k += 4)
              wt_store16(record + 2 * R + r * D + c * 16 + k, on, __float_as_uint(x[k]), __float_as_uint(x[k + 1]), __float_as_uint(x[k + 2]), __float_as_uint(x[k + 3]));
          } else {
            __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out) + out_row * D + c * 16;
#pragma unroll
            for (int k = 0; k < 16; k += 8)
              wt_store16(out + k, on, pack_b16(x[k] * inv, x[k + 1] * inv), pack_b16(x[k + 2] * inv, x[k + 3] * inv), pack_b16(x[k + 4] * inv, x[k + 5] * inv), pack_b16(x[k + 6] * inv, x[k + 7] * inv));
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
      }
      __syncwarp();
      tc5_fence_before();
      if (both) all_meet();                          // (the exchange and both outputs have been read)
      __syncwarp();
      if (lane == 0 && filled(w)) mbar_arrive(o_free + 8 * set, 1);
      if (!q_now) write_q(following);
      w = following;
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Tc::other_regs));
    if (warp == kWtLoadWarp) {
      // ================================================================== pages
      int g = 0, nk = 0, nv = 0;                     // groups; copies begun
      for (Piece w = next(); w.any && ok; w = next()) {
        int pages = 0;                               // of the next 32 / PG groups, one per lane; -1: nobody sees it
        [[maybe_unused]] float k_scale = 0.f, v_scale = 0.f;                   // FP8: theirs
        for (int gi = w.first; gi < w.last; ++gi, ++g) {
          const int i = (gi - w.first) % (32 / PG);
          if (i == 0) {
            const int mine = gi + lane / PG, key = mine < w.last ? group_key<GT>(w.r, mine) + (lane % PG) * GP : w.r.end;
            pages = -1;
            if (key < w.r.end && (key + GP > w.r.lo || key < p.q.sinks)) pages = max(0, page_of(p.c, w.s, key / GP, p.status));
            if (FMT == kRowsFp8 && pages >= 0) {
              k_scale = static_cast<const float*>(p.c.k_scale)[static_cast<size_t>(pages) * p.c.Hkv + w.kh];
              v_scale = static_cast<const float*>(p.c.v_scale)[static_cast<size_t>(pages) * p.c.Hkv + w.kh];
            }
            __syncwarp();
          }
          [[maybe_unused]] const uint32_t have = __ballot_sync(0xffffffffu, pages >= 0) >> (i * PG) & ((1u << PG) - 1u);
          if constexpr (QUANT) {
            const int slot = g % NR;
            if (g >= NR && !wait(r_free + 8 * slot, (g / NR - 1) & 1)) break;
            raw_load<FMT, D, GP>(p.c, &map_k, p.c.k_scale, w.kh, pages, k_scale, i * PG, base + RAW + slot * Tc::raw, r_full + 8 * slot);
            ++nk;
            if (g >= NR && !wait(r_free + 8 * (NR + slot), (g / NR - 1) & 1)) break;
            raw_load<FMT, D, GP>(p.c, &map_v, p.c.v_scale, w.kh, pages, v_scale, i * PG, base + RAW + (NR + slot) * Tc::raw, r_full + 8 * (NR + slot));
            ++nv;
          } else {
            const uint32_t bytes = __popc(have) * (GP * D * 2);
            const int ks = g % kWtNK, vs = g % kWtNV;
            if (g >= kWtNK && !wait(k_free + 8 * ks, (g / kWtNK - 1) & 1)) break;
            if (elect_one()) mbar_expect_tx(k_full + 8 * ks, bytes);
            ++nk;
            __syncwarp();
#pragma unroll 1
            for (int j = 0; j < PG; ++j) {
              const int page = __shfl_sync(0xffffffffu, pages, i * PG + j);
              if (page >= 0 && elect_one())
#pragma unroll
                for (int h = 0; h < D / 64; ++h) tma_load_page(kring + ks * TILE + h * HS + j * GP * 128, &map_k, k_full + 8 * ks, h * 64, w.kh, page);
              __syncwarp();
            }
            if (g >= kWtNV && !wait(v_free + 8 * vs, (g / kWtNV - 1) & 1)) break;
            if (elect_one()) mbar_expect_tx(v_full + 8 * vs, bytes);
            ++nv;
            __syncwarp();
#pragma unroll 1
            for (int j = 0; j < PG; ++j) {
              const int page = __shfl_sync(0xffffffffu, pages, i * PG + j);
              if (page >= 0 && elect_one())
#pragma unroll
                for (int h = 0; h < D / 64; ++h) tma_load_page(vring + vs * TILE + h * HS + j * GP * 128, &map_v, v_full + 8 * vs, h * 64, w.kh, page);
              __syncwarp();
            }
          }
        }
      }
      // (what is in flight has landed before the CTA's shared memory is given up)
      if (!ok) {
        constexpr int sk = QUANT ? NR : kWtNK, sv = QUANT ? NR : kWtNV;
        for (int i = 0; i < min(sk, nk); ++i) mbar_drain((QUANT ? r_full : k_full) + 8 * i, ((nk - 1 - i) / sk) & 1);
        for (int i = 0; i < min(sv, nv); ++i) mbar_drain((QUANT ? r_full + 8 * NR : v_full) + 8 * i, ((nv - 1 - i) / sv) & 1);
      }
      __syncwarp();
    } else if (warp == kWtQkWarp) {
      // ================================================================== Q K^T
      const uint32_t qt = warp_uniform(qtile), kr = warp_uniform(kring), idesc = tc5_idesc(128, GT, 0, kType, kType);
      int g = 0, n[2] = {0, 0}, q0 = 0, q1 = 0;
      for (Piece w = next(); w.any && ok; w = next()) {
        const bool both = joint(w);
        if (!filled(w)) continue;
        wait(q_full, q0++ & 1);
        if (!both) wait(q_full + 8, q1++ & 1);
        for (int gi = w.first; gi < w.last && ok; ++gi, ++g) {
          const int slot = g % kWtNK;
          if (!wait(k_full + 8 * slot, (g / kWtNK) & 1)) break;
          const int from = both ? (gi - w.first) & 1 : 0, to = both ? from + 1 : 2;
#pragma unroll 1
          for (int set = from; set < to; ++set) {
            const int c = set ? n[1]++ : n[0]++;
            if (c > 0 && !wait(s_free + 8 * set, (c - 1) & 1)) break;
            tc5_fence_after();
            if (elect_one()) {
              const uint64_t qd = tc5_desc(qt + (both ? 0 : set * QTILE), 16), kd = tc5_desc(kr + slot * TILE, 16);
#pragma unroll
              for (int ks = 0; ks < D / 16; ++ks) {
                const uint32_t at = ((ks >> 2) * HS + (ks & 3) * 32) / 16;
                tc5_mma_ss(tmem + COL_S + set * 128, qd + at, kd + at, idesc, ks > 0 ? 1u : 0u);
              }
              tc5_commit(s_full + 8 * set);
              if (set + 1 == to) tc5_commit(k_free + 8 * slot);
            }
            __syncwarp();
          }
        }
      }
    } else if (warp == kWtPvWarp) {
      // ================================================================== P V
      const uint32_t vr = warp_uniform(vring), idesc = tc5_idesc(128, D, 1, kType, kType);
      int g = 0, n[2] = {0, 0}, piece = 0;
      for (Piece w = next(); w.any && ok; w = next()) {
        const bool both = joint(w);
        if (!filled(w)) continue;
        if (piece++ > 0) {
          wait(o_free, piece & 1);
          wait(o_free + 8, piece & 1);
        }
        for (int gi = w.first; gi < w.last && ok; ++gi, ++g) {
          const int slot = g % kWtNV;
          if (!wait(v_full + 8 * slot, (g / kWtNV) & 1) || !wait(v_fixed + 8 * slot, (g / kWtNV) & 1)) break;
          const int from = both ? (gi - w.first) & 1 : 0, to = both ? from + 1 : 2;
          const bool first = gi - w.first < (both ? 2 : 1);
#pragma unroll 1
          for (int set = from; set < to; ++set) {
            const int c = set ? n[1]++ : n[0]++;
#pragma unroll 1
            for (int hf = 0; hf < 2; ++hf) {
              if (!wait(p_full + 8 * (set * 2 + hf), c & 1)) break;
              tc5_fence_after();
              if (elect_one()) {
                const uint64_t vd = tc5_desc(vr + slot * TILE, HS) + hf * 512;       // 64 tokens of 128 bytes
                const uint32_t p_col = tmem + COL_S + set * 128 + hf * 32, o_col = tmem + COL_O + set * 128;
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) tc5_mma_ts(o_col, p_col + ks * 8, vd + ks * 128, idesc, ks > 0 || hf > 0 || !first ? 1u : 0u);
                if (hf == 1) {
                  if (set + 1 == to) tc5_commit(v_free + 8 * slot);
                  tc5_commit(s_free + 8 * set);
                }
              }
              __syncwarp();
            }
          }
        }
      }
    } else if (warp == kWtFixWarp) {
      // ================================================================== values that must not count
      int g = 0, pieces = 0;
      for (Piece w = next(); w.any && ok; w = next()) {
        const Common com = common_of(p, w);
        if (filled(w)) ++pieces;
        for (int gi = w.first; gi < w.last; ++gi, ++g) {
          const int key0 = group_key<GT>(w.r, gi), slot = g % kWtNV;
          if (!wait(v_full + 8 * slot, (g / kWtNV) & 1)) break;
          if (in_part(p, com, key0)) {
            uint8_t* tile = gen + QALL + (kWtNK + slot) * TILE;
            bool odd = false;
            // 16 bytes per lane, four 128-byte rows of the tile at a time
#pragma unroll 2
            for (int t = 0; t < GT; t += 4) {
              const int row = t + (lane >> 3), key = key0 + row;
              const bool live = key < w.r.end && (key >= w.r.lo || key < p.q.sinks);
#pragma unroll
              for (int h = 0; h < D / 64; ++h) {
                uint4* at = reinterpret_cast<uint4*>(tile + h * HS + row * 128 + (lane & 7) * 16);
                if (!live) {
                  *at = make_uint4(0u, 0u, 0u, 0u);
                } else if (!com.same) {
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
        }
      }
    } else {
      // ================================================================== quantised pages into operands
      if constexpr (QUANT) {
        int g = 0;
        for (Piece w = next(); w.any && ok; w = next()) {
          for (int gi = w.first; gi < w.last && ok; ++gi, ++g) {
#pragma unroll 1
            for (int v = 0; v < 2; ++v) {
              const int slot = g % NR, to = v ? g % kWtNV : g % kWtNK;
              const uint32_t full = (v ? v_full : k_full) + 8 * to, free = (v ? v_free : k_free) + 8 * to;
              const int turns = v ? g / kWtNV : g / kWtNK;
              if (!wait(r_full + 8 * (v * NR + slot), (g / NR) & 1)) break;
              if (turns > 0 && !wait(free, (turns - 1) & 1)) break;
              raw_convert<FMT, D, GP, true>(gen + RAW + (v * NR + slot) * Tc::raw, gen + QALL + ((v ? kWtNK : 0) + to) * TILE, tid - kWtConvertWarp * 32);
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
  // ---- the products in flight have run before tensor memory is given back
  if (warp == kWtQkWarp || warp == kWtPvWarp) {
    const uint32_t bar = drain + 8 * (warp - kWtQkWarp);
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
