// Windowed attention in fp32 on the CUDA cores: included by window_attn.cu (same namespace).
//
// 64 rows against 64 keys at a time, 128 threads: a thread has 8 rows by 4 keys of the scores and 8 rows by D / 16 columns of the
// output, so that a float4 from shared memory feeds 10 to 32 products.  One pass: running maximum and sum per row.
// Prompts of 1,024 and 777 tokens, four heads of 64, window 333: 52 us a pass; each by itself, from cold caches, the list takes 6, this kernel 45, the merge 8.  Its shares are even, two or three groups
// for each of the 296 CTAs: what it waits for is a group's chain of page table, rows, shared memory and products, with nothing beside it.
#pragma once

constexpr int kWinRows = 64, kWinKeys = 64, kWinThreads = 128;
using WinTiles = RowTiles<kWinRows, 1, kWinKeys>;
template <int D> constexpr int win_smem() { return (kWinRows * D + kWinKeys * (D + 4) + kWinKeys * D + kWinRows * (kWinKeys + 4)) * 4; }

template <int D>
__global__ void __launch_bounds__(kWinThreads, 2) window_f32_kernel(const __grid_constant__ WindowParams p) {
  using T = float;
  constexpr int R = kWinRows, GT = kWinKeys, KS = D + 4, PS = GT + 4, C8 = D / 8, NC = D / 64;
  extern __shared__ __align__(16) float smem[];
  float *sq = smem, *sk = sq + R * D, *sv = sk + GT * KS, *sp = sv + GT * D;
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  grid_dep_trigger();
  grid_dep_wait();
  Walk walk(p, blockIdx.x);
  for (Piece w = next_piece<WinTiles, GT>(walk); w.any; w = next_piece<WinTiles, GT>(walk)) {
    __syncthreads();
    for (int i = tid; i < R * C8; i += kWinThreads) {
      const int r = i / C8, ch = i - r * C8;
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = 0.f;
      const int t = row_token<R>(p, w.tokens, 0, r);
      if (t >= 0) load8(static_cast<const T*>(p.q.q) + (static_cast<long long>(w.x.cu) + w.token0 + t) * p.q.stride + (w.kh * p.c.G + r % p.c.G) * D + ch * 8, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) sq[r * D + ch * 8 + k] = v[k];
    }
    int2 sees[8];                                    // keys of this thread's rows: below x, from y on or below the sinks
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int t = row_token<R>(p, w.tokens, 0, ty * 8 + i);
      sees[i] = t >= 0 ? keys_of(p.q, w.x, w.x.start + w.token0 + t) : make_int2(0, 0);
    }
    float m[8], l[8], o[8][NC * 4];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int k = 0; k < NC * 4; ++k) o[i][k] = 0.f;
    }
    for (int gi = w.first; gi < w.last; ++gi) {
      const int key0 = group_key<GT>(w.r, gi);
      __syncthreads();
      int odd = 0;                                   // a value that is no finite number
      for (int i = tid; i < GT * C8; i += kWinThreads) {
        const int t = i / C8, ch = i - t * C8, key = key0 + t;
        float kx[8], vx[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) kx[k] = vx[k] = 0.f;
        if (key < w.r.end && (key >= w.r.lo || key < p.q.sinks)) {
          const int page = page_of(p.c, w.s, key / p.c.g, p.status), slot = key % p.c.g;
          if (page >= 0) {
            cache_load8<kRowsF32, D>(p.c, p.c.k_pages, p.c.k_scale, page, w.kh, slot, ch, kx);
            cache_load8<kRowsF32, D>(p.c, p.c.v_pages, p.c.v_scale, page, w.kh, slot, ch, vx);
          }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          sk[t * KS + ch * 8 + k] = kx[k];
          sv[t * D + ch * 8 + k] = vx[k];
          odd |= !(fabsf(vx[k]) < INFINITY);
        }
      }
      odd = __syncthreads_or(odd);
      float s[8][4];
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) s[i][k] = 0.f;
#pragma unroll 2
      for (int c = 0; c < D; c += 4) {
        float4 a[8], b[4];
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = *reinterpret_cast<const float4*>(sq + (ty * 8 + i) * D + c);
#pragma unroll
        for (int k = 0; k < 4; ++k) b[k] = *reinterpret_cast<const float4*>(sk + (tx + 16 * k) * KS + c);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int k = 0; k < 4; ++k) s[i][k] = fmaf(a[i].x, b[k].x, fmaf(a[i].y, b[k].y, fmaf(a[i].z, b[k].z, fmaf(a[i].w, b[k].w, s[i][k]))));
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float top = -INFINITY;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int key = key0 + tx + 16 * k;
          const bool on = key < sees[i].x && (key >= sees[i].y || key < p.q.sinks);
          s[i][k] = on ? s[i][k] * p.scale_log2 : -INFINITY;
          top = fmaxf(top, s[i][k]);
        }
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
        const float to = fmaxf(m[i], top), f = to == -INFINITY ? 1.f : exp2f(m[i] - to);
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float e = to == -INFINITY ? (s[i][k] == s[i][k] ? 0.f : s[i][k]) : exp2f(s[i][k] - to);      // (a score that is no number stays visible)
          sum += e;
          sp[(ty * 8 + i) * PS + tx + 16 * k] = e;
        }
        l[i] = fmaf(l[i], f, sum);                   // (this thread's keys; the sixteen threads of a row meet at the end)
        m[i] = to;
#pragma unroll
        for (int k = 0; k < NC * 4; ++k) o[i][k] *= f;
      }
      __syncwarp();                                  // (a row's sixteen threads are in one warp)
      if (!odd) {
#pragma unroll 2
        for (int t = 0; t < GT; t += 4) {
          float4 a[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) a[i] = *reinterpret_cast<const float4*>(sp + (ty * 8 + i) * PS + t);
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int h = 0; h < NC; ++h) {
              const float4 v = *reinterpret_cast<const float4*>(sv + (t + k) * D + h * 64 + tx * 4);
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                const float e = k == 0 ? a[i].x : k == 1 ? a[i].y : k == 2 ? a[i].z : a[i].w;
                o[i][h * 4 + 0] = fmaf(e, v.x, o[i][h * 4 + 0]);
                o[i][h * 4 + 1] = fmaf(e, v.y, o[i][h * 4 + 1]);
                o[i][h * 4 + 2] = fmaf(e, v.z, o[i][h * 4 + 2]);
                o[i][h * 4 + 3] = fmaf(e, v.w, o[i][h * 4 + 3]);
              }
            }
        }
      } else {                                       // infinities or NaN among the values: rows that do not see them stay clean
        for (int t = 0; t < GT; ++t) {
          const int key = key0 + t;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if (!(key < sees[i].x && (key >= sees[i].y || key < p.q.sinks))) continue;
            const float e = sp[(ty * 8 + i) * PS + t];
#pragma unroll
            for (int k = 0; k < NC * 4; ++k) o[i][k] = fmaf(e, sv[t * D + (k >> 2) * 64 + tx * 4 + (k & 3)], o[i][k]);
          }
        }
      }
    }
    float* record = record_of<R, D>(p, blockIdx.x, w.first == 0);
    const bool whole = w.whole();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float sum = l[i];
#pragma unroll
      for (int off = 8; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
      const int r = ty * 8 + i;
      const int t = row_token<R>(p, w.tokens, 0, r);
      if (t < 0) continue;
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      const long long row = token_head(p, w.x, w.token0 + t, w.kh, r);
#pragma unroll
      for (int h = 0; h < NC; ++h)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int col = h * 64 + tx * 4 + k;
          if (whole) static_cast<T*>(p.out)[row * D + col] = from_f32<T>(o[i][h * 4 + k] * inv);
          else record[2 * R + r * D + col] = o[i][h * 4 + k];
        }
      if (tx == 0) {
        if (!whole) {
          record[r] = m[i];
          record[R + r] = sum;
        } else if (p.lse) {
          p.lse[row] = sum == 0.f ? -INFINITY : (m[i] + log2f(sum)) * kLn2;
        }
      }
    }
  }
}
