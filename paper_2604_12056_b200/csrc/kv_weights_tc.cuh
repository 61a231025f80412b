// The keys' weights on the 5th-generation tensor cores: included by kv_weights.cu (same namespace).
//
// Keys take the 128 lanes, query rows the columns, so that a thread has a key to itself and its sum never leaves the register: a job is
// 128 keys by up to 128 rows.
//   a warp            pages of keys by TMA into a ring of swizzled tiles
//   some warps        jobs by turns: queries by TMA, as many whole tokens as 128 rows hold, and their log-normalisers, into another
//   S[128 x rows] = K Q^T   an issuing warp; four score tiles in tensor memory
//   two sets of four warps  take alternate jobs: exponentials, added up by key; at a tile's end the sets' sums meet in shared memory
// Keys and not rows on the lanes because the sum over rows then needs no other thread.  Measured: a prompt of 8,192 tokens, 32 heads 418 us (657 TFLOP/s; the exponentials of the special
// function unit alone need 246), the last 64 tokens of two prompts of 32,768 and 20,065 72 us, eight decoded tokens over caches of up to 16,384 65 us (3.3 TB/s; entering
// a tile, with its pages' places and the old weights to be looked up, costs more than its 32 KB of keys).
// A key is seen by a run of tokens, so a job that is not seen whole is masked by two numbers per thread.
// Operands of 16 bits hold keys and queries exactly; sums are fp32, one per job and one over the jobs (a prompt of 8,192 tokens: off by 3.3e-7, 2.2e-7 of it in one direction).
#pragma once

constexpr int kKwKeys = 128, kKwRows = 128, kKwBufs = 4;
constexpr int kKwSumWarps = 8, kKwLoadWarp = 8, kKwMmaWarp = 9, kKwQWarp = 10;
template <int FMT, int D, int GP> struct WeightsTc {
  static constexpr bool quant = FMT != kRowsBf16;
  static constexpr int q_warps = quant ? 2 : 3, convert_warp = kKwQWarp + 2;              // quantised pages: the last four warps turn them into operands
  static constexpr int warps = quant ? 16 : 13;
  static constexpr int nk = quant ? 2 : 3, nq = q_warps, nr = 3; // tiles of keys, of rows (one per warp that fills them: it waits for every one of its phases in turn); of keys as they lie
  static constexpr int tile = 128 * D * 2, raw = quant ? RawTile<FMT, D, GP>::bytes : 0;
  static constexpr int norms = (nk + nq) * tile + (quant ? nr * raw : 0), other = norms + nq * kKwRows * 4, gives = other + 2 * kKwKeys * 4, tail = gives + nq * kKwRows / 8;
  static constexpr int smem = 1024 + tail + 256;
  static_assert(smem <= 232448, "shared memory");
};

// Tiles of keys that have anything to do (none of a sequence that is left out): those under the first tokens, and from the window of the first token on; all where weights are forgotten.
struct KeyReach { int first, from, tiles; };
__device__ __forceinline__ KeyReach key_reach(const ListParams& p, const Sequence& x) {
  KeyReach r = {0, 0, 0};
  const int all = (x.len + kKwKeys - 1) / kKwKeys;
  if (x.start < 0) return r;
  if (p.keep != 1.f) {
    r.tiles = all;
    return r;
  }
  const int lo = min(x.start, x.count > 0 ? keys_of(p.q, x, x.start).y : x.start), sinks = lo > 0 && x.count > 0 ? min(p.q.sinks, x.len) : 0;
  r.first = (sinks + kKwKeys - 1) / kKwKeys;
  r.from = max(r.first, lo / kKwKeys);
  r.tiles = r.first + max(0, all - r.from);
  return r;
}
__device__ __forceinline__ int tile_key(const KeyReach& r, int j) { return (j < r.first ? j : r.from + j - r.first) * kKwKeys; }
struct KeyTiles {
  static __device__ __forceinline__ int tiles(const ListParams& p, const Sequence& x) { return key_reach(p, x).tiles; }
  static __device__ __forceinline__ int groups(const ListParams& p, const Sequence& x, int j) {
    const int key0 = tile_key(key_reach(p, x), j);
    const int2 seen = tokens_over(p, x, key0, min(kKwKeys, x.len - key0));
    const int per = kKwRows / p.c.G;
    return (seen.y - seen.x + per - 1) / per;
  }
};
struct KeyPiece : Part { int key0, token0, tokens; };      // tokens token0 .. token0 + tokens - 1 see any of the tile's keys
__device__ __forceinline__ KeyPiece next_keys(Walk& walk) {
  KeyPiece w;
  static_cast<Part&>(w) = walk.next();
  if (w.any) {
    w.key0 = tile_key(key_reach(walk.p, w.x), w.j);
    const int2 seen = tokens_over(walk.p, w.x, w.key0, min(kKwKeys, w.x.len - w.key0));
    w.token0 = seen.x;
    w.tokens = seen.y - seen.x;
  }
  return w;
}

template <int FMT, int D, int GP>
__global__ void __launch_bounds__(WeightsTc<FMT, D, GP>::warps * 32, 1) weights_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_q,
                                                                     const __grid_constant__ WeightParams p) {
  using Tc = WeightsTc<FMT, D, GP>;
  constexpr bool QUANT = Tc::quant;
  constexpr int TILE = Tc::tile, HS = 128 * 128, PG = kKwKeys / GP, NK = Tc::nk, NQ = Tc::nq, NR = Tc::nr;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const uint32_t kring = base, qring = kring + NK * TILE;
  [[maybe_unused]] constexpr int RAW = (NK + NQ) * TILE;                 // quantised pages as they lie
  float* norms = reinterpret_cast<float*>(gen + Tc::norms);              // [slot][row] log-normaliser in log2 units
  uint32_t* gives = reinterpret_cast<uint32_t*>(gen + Tc::gives);        // [slot][row / 32] rows that give anything
  float* other = reinterpret_cast<float*>(gen + Tc::other);              // [2][key] the second set's sums, by turns
  const uint32_t bars = base + Tc::tail;
  const uint32_t k_full = bars, k_free = k_full + 8 * NK, q_full = k_free + 8 * NK, q_free = q_full + 8 * NQ;
  const uint32_t s_full = q_free + 8 * NQ, s_free = s_full + 8 * kKwBufs, drain = s_free + 8 * kKwBufs;
  [[maybe_unused]] const uint32_t r_full = drain + 8, r_free = r_full + 8 * NR;
  constexpr int MISC = 8 * (2 * NK + 2 * NQ + 2 * kKwBufs + 1 + 2 * NR);
  static_assert(MISC + 8 <= 256, "barriers");
  volatile int* abort_flag = reinterpret_cast<volatile int*>(gen + Tc::tail + MISC);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(gen + Tc::tail + MISC + 4);
  const int tid = threadIdx.x, lane = tid & 31, warp = warp_uniform(tid >> 5);

  grid_dep_trigger();
  if (tid == 0) {
    for (int i = 0; i < NK; ++i) { mbar_init(k_full + 8 * i, QUANT ? 4 : 1); mbar_init(k_free + 8 * i, 1); }
    if constexpr (QUANT)
      for (int i = 0; i < NR; ++i) { mbar_init(r_full + 8 * i, 1); mbar_init(r_free + 8 * i, 4); }
    for (int i = 0; i < NQ; ++i) { mbar_init(q_full + 8 * i, 1); mbar_init(q_free + 8 * i, 1 + 4); }      // the products, and the set that reads the log-normalisers
    for (int i = 0; i < kKwBufs; ++i) { mbar_init(s_full + 8 * i, 1); mbar_init(s_free + 8 * i, 4); }
    mbar_init(drain, 1);
    *abort_flag = 0;
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
  auto wait = [&](uint32_t bar, uint32_t parity) {
    if (ok) ok = warp_mbar_wait(bar, parity, abort_flag, p.status, p.wait_cycles);
    __syncwarp();                                    // (what follows is for whole warps)
    return ok;
  };
  Walk walk(p, blockIdx.x);
  const int per = kKwRows / p.c.G;                   // tokens of a job
  __syncwarp();
  if (warp < kKwSumWarps) {
    // ================================================================== sums: thread = (set, key)
    const int set = warp >> 2, at128 = tid & 127;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const float2 scale = make_float2(p.scale_log2, p.scale_log2);
    int job = 0, turn = 0;
    for (KeyPiece w = next_keys(walk); w.any; w = next_keys(walk)) {
      const int key = w.key0 + at128, jobs = w.last - w.first;
      // the tokens, counted from the tile's first, that see this key
      const int2 seen = tokens_over(p, w.x, key, 1);
      const int ta = seen.x - w.token0, tb = min(seen.y - w.token0, w.tokens);
      const Held held = held_weight(p, w.x, w.s, w.kh, key);             // (asked for before the sum)
      // a sum for each job and one over the jobs: a chain of all the terms would lose three bits of the weights of a long prompt
      float total = 0.f;
      for (int gi = w.first; gi < w.last; ++gi, ++job) {
        if ((job & 1) != set) continue;
        const int buf = job % kKwBufs, slot = job % NQ, n = min(per, w.tokens - gi * per) * p.c.G;
        const int a = (ta - gi * per) * p.c.G, b = min((tb - gi * per) * p.c.G, n);      // of the job's columns this key counts a .. b - 1
        const bool part = __any_sync(0xffffffffu, a > 0 || b < n || (n & 31));      // (columns behind n may hold anything)
        if (!wait(s_full + 8 * buf, (job / kKwBufs) & 1)) break;
        tc5_fence_after();
        const float* norm = norms + slot * kKwRows;
        const uint32_t* give = gives + slot * (kKwRows / 32);
        float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll 1
        for (int c = 0; c < n; c += 32) {
          uint32_t x[32];
          tc5_ld32_nowait(tmem + buf * 128 + c + lanes, x);
          tc5_wait_ld();
          tc5_pin32(x);
          const uint32_t rows = give[c >> 5], on = part ? low_bits(b - c) & ~low_bits(a - c) & rows : rows;
          const bool mask = part || rows != 0xffffffffu;       // (a row that gives nothing may have any scores)
#pragma unroll
          for (int k = 0; k < 32; k += 4) {
            const float4 l = *reinterpret_cast<const float4*>(norm + c + k);
            float2 e = fma2_f32(make_float2(__uint_as_float(x[k]), __uint_as_float(x[k + 1])), scale, make_float2(-l.x, -l.y));
            float2 f = fma2_f32(make_float2(__uint_as_float(x[k + 2]), __uint_as_float(x[k + 3])), scale, make_float2(-l.z, -l.w));
            e.x = ex2(e.x);
            e.y = ex2(e.y);
            f.x = ex2(f.x);
            f.y = ex2(f.y);
            if (mask) {
              e.x = (on >> k) & 1u ? e.x : 0.f;
              e.y = (on >> (k + 1)) & 1u ? e.y : 0.f;
              f.x = (on >> (k + 2)) & 1u ? f.x : 0.f;
              f.y = (on >> (k + 3)) & 1u ? f.y : 0.f;
            }
            sum[0] = add2_f32(sum[0], e);
            sum[1] = add2_f32(sum[1], f);
          }
        }
        const float2 both = add2_f32(sum[0], sum[1]);
        total += both.x + both.y;
        tc5_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(s_free + 8 * buf, 1);
          mbar_arrive(q_free + 8 * slot, 1);
        }
        __syncwarp();
      }
      int writer = jobs == 1 ? (job + 1) & 1 : 0;    // (the set that had the only job; a tile without any is the first one's)
      if (jobs > 1) {
        if (set == 1) other[(turn & 1) * kKwKeys + at128] = total;
        __syncwarp();
        asm volatile("bar.sync 1, %0;" ::"n"(kKwSumWarps * 32) : "memory");
        if (set == 0) total += other[(turn & 1) * kKwKeys + at128];
        ++turn;                                      // (a place is written again after the next meeting, which comes after this reading)
      }
      if (set == writer && ok) {
        if (w.whole()) {
          put_weight(p, held, total);
        } else {
          p.partials[record_at(blockIdx.x, w.first == 0) * kKwKeys + at128] = total;
        }
      }
      __syncwarp();
    }
  } else if (warp == kKwLoadWarp) {
    // ================================================================== keys
    int n = 0;
    for (KeyPiece w = next_keys(walk); w.any && ok; w = next_keys(walk)) {
      if (w.last == w.first) continue;
      if (n >= p.copies) {
        *abort_flag = 1;
        if (lane == 0) set_status(p.status, LOSA_ERR_TIMEOUT);
        break;
      }
      const int slot = n % (QUANT ? NR : NK), key = w.key0 + lane * GP;
      int page = -1;
      if (lane < PG && key < w.x.len) page = max(0, page_of(p.c, w.s, key / GP, p.status));
      __syncwarp();
      if constexpr (QUANT) {
        if (n >= NR && !wait(r_free + 8 * slot, (n / NR - 1) & 1)) break;
        float scale = 0.f;
        if (FMT == kRowsFp8 && page >= 0) scale = static_cast<const float*>(p.c.k_scale)[static_cast<size_t>(page) * p.c.Hkv + w.kh];
        __syncwarp();
        raw_load<FMT, D, GP>(p.c, &map_k, p.c.k_scale, w.kh, page, scale, 0, base + RAW + slot * Tc::raw, r_full + 8 * slot);
        ++n;
        continue;
      }
      const uint32_t have = __ballot_sync(0xffffffffu, page >= 0);
      if (n >= NK && !wait(k_free + 8 * slot, (n / NK - 1) & 1)) break;
      if (elect_one()) mbar_expect_tx(k_full + 8 * slot, __popc(have) * (GP * D * 2));
      __syncwarp();
      if (page >= 0)                                 // (each lane its page: a copy in a loop of the warp takes 185 cycles)
#pragma unroll
        for (int h = 0; h < D / 64; ++h) tma_load_page(kring + slot * TILE + h * HS + lane * GP * 128, &map_k, k_full + 8 * slot, h * 64, w.kh, page);
      __syncwarp();
      ++n;
    }
    // (what is in flight has landed before the CTA's shared memory is given up, whichever warp's wait has run out)
    constexpr int slots = QUANT ? NR : NK;
    for (int i = 0; i < min(slots, n); ++i) mbar_drain((QUANT ? r_full : k_full) + 8 * i, ((n - 1 - i) / slots) & 1);
    __syncwarp();
  } else if (warp == kKwMmaWarp) {
    // ================================================================== K Q^T
    const uint32_t kr = warp_uniform(kring), qr = warp_uniform(qring);
    int job = 0, n = 0;
    for (KeyPiece w = next_keys(walk); w.any && ok; w = next_keys(walk)) {
      if (w.last == w.first) continue;
      const int kslot = n % NK;
      if (!wait(k_full + 8 * kslot, (n / NK) & 1)) break;
      // (numbers that the compiler knows to be the warp's: a product whose operands come from ordinary registers takes 120 cycles to issue)
      const int first = warp_uniform(w.first), last = warp_uniform(w.last), tokens = warp_uniform(w.tokens);
      for (int gi = first; gi < last; ++gi, ++job) {
        const int buf = job % kKwBufs, slot = job % NQ, cols = min(per, tokens - gi * per) * p.c.G;
        if (!wait(q_full + 8 * slot, (job / NQ) & 1)) break;
        if (job >= kKwBufs && !wait(s_free + 8 * buf, (job / kKwBufs - 1) & 1)) break;
        tc5_fence_after();
        if (elect_one()) {
          const uint32_t idesc = tc5_idesc(128, (cols + 31) & ~31, 0, 1u, 1u);
          const uint64_t kd = tc5_desc(kr + kslot * TILE, 16), qd = tc5_desc(qr + slot * TILE, 16);
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            const uint32_t at = ((ks >> 2) * HS + (ks & 3) * 32) / 16;
            tc5_mma_ss(tmem + buf * 128, kd + at, qd + at, idesc, ks > 0 ? 1u : 0u);
          }
          tc5_commit(s_full + 8 * buf);
          tc5_commit(q_free + 8 * slot);
          if (gi + 1 == last) tc5_commit(k_free + 8 * kslot);
        }
        __syncwarp();
      }
      ++n;
    }
    // the products in flight have run before tensor memory is given back
    if (elect_one()) {
      tc5_commit(drain);
      mbar_drain(drain, 0);
    }
    __syncwarp();
  } else if (QUANT && warp >= Tc::convert_warp) {
    // ================================================================== quantised pages into operands
    if constexpr (QUANT) {
      int n = 0;
      for (KeyPiece w = next_keys(walk); w.any && ok; w = next_keys(walk)) {
        if (w.last == w.first) continue;
        const int slot = n % NR, to = n % NK;
        if (!wait(r_full + 8 * slot, (n / NR) & 1)) break;
        if (n >= NK && !wait(k_free + 8 * to, (n / NK - 1) & 1)) break;
        raw_convert<FMT, D, GP, false>(gen + RAW + slot * Tc::raw, gen + to * TILE, tid - Tc::convert_warp * 32);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");     // the products read the tile through the async proxy
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(k_full + 8 * to, 1);
          mbar_arrive(r_free + 8 * slot, 1);
        }
        __syncwarp();
        ++n;
      }
    }
  } else {
    // ================================================================== queries and log-normalisers, jobs by turns
    const int mine = warp - kKwQWarp;
    int tok[4], head[4];                             // of rows lane, lane + 32, ..
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      tok[i] = (lane + 32 * i) / p.c.G;
      head[i] = lane + 32 * i - tok[i] * p.c.G;
    }
    int job = 0, begun = -1;                         // the last of this warp's jobs
    for (KeyPiece w = next_keys(walk); w.any && ok; w = next_keys(walk)) {
      for (int gi = w.first; gi < w.last; ++gi, ++job) {
        if (job % Tc::q_warps != mine) continue;
        const int slot = job % NQ, n = min(per, w.tokens - gi * per);
        const long long t0 = static_cast<long long>(w.x.cu) + w.token0 + gi * per;
        float l[4];                                  // a row that does not exist, or saw nothing, gives nothing
#pragma unroll
        for (int i = 0; i < 4; ++i) l[i] = tok[i] < n ? p.lse[(t0 + tok[i]) * (p.c.Hkv * p.c.G) + w.kh * p.c.G + head[i]] : -INFINITY;
        if (job >= NQ && !wait(q_free + 8 * slot, (job / NQ - 1) & 1)) break;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          norms[slot * kKwRows + lane + 32 * i] = l[i] * kLog2e;
          const uint32_t rows = __ballot_sync(0xffffffffu, l[i] != -INFINITY);
          if (lane == 0) gives[slot * (kKwRows / 32) + i] = rows;
        }
        __syncwarp();
        if (elect_one()) {
          mbar_expect_tx(q_full + 8 * slot, per * p.c.G * D * 2);
#pragma unroll
          for (int h = 0; h < D / 64; ++h) tma_load_queries(qring + slot * TILE + h * HS, &map_q, q_full + 8 * slot, h * 64, w.kh * p.c.G, static_cast<int>(t0));
        }
        __syncwarp();
        begun = job;
      }
    }
    // (likewise)
    if (begun >= 0) mbar_drain(q_full + 8 * (begun % NQ), (begun / NQ) & 1);
    __syncwarp();
  }
  tc5_fence_before();
  __syncthreads();
  if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
}

// Tiles that several CTAs share: a thread per key adds their sums, in CTA order.
__global__ void __launch_bounds__(kKwKeys) weights_join_kernel(const __grid_constant__ WeightParams p) {
  grid_dep_wait();
  const int b = blockIdx.x + 1;
  Share x;
  const int last = records_from(p, b, x);
  if (last < b) return;
  const int key = tile_key(key_reach(p, x.t.x), x.t.j) + threadIdx.x;
  const Held held = held_weight(p, x.t.x, x.t.s, x.kh, key);
  float total = 0.f;
  for (int i = b - 1; i <= last; ++i) total += p.partials[record_at(i, i == b - 1) * kKwKeys + threadIdx.x];
  put_weight(p, held, total);
}
