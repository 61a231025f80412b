// The keys' weights in fp32 on the CUDA cores: included by kv_weights.cu (same namespace).
//
// fp32 products stay on the CUDA cores, as stage 4's do; shared memory bounds them (twelve 16-byte reads for 128 products).
// A CTA has 64 keys and takes 64 rows at a time, 8 rows by 4 keys a thread.
#pragma once

constexpr int kWgtKeys = 64, kWgtRows = 64, kWgtThreads = 128;
template <int D> constexpr int weights_smem() { return (kWgtRows * D + kWgtKeys * (D + 4) + 3 * kWgtRows + 8 * kWgtKeys) * 4; }

template <int D>
__global__ void __launch_bounds__(kWgtThreads, 3) weights_f32_kernel(const __grid_constant__ WeightParams p) {
  using T = float;
  constexpr int R = kWgtRows, GT = kWgtKeys, KS = D + 4, C8 = D / 8;
  extern __shared__ __align__(16) float smem[];
  float *sq = smem, *sk = sq + R * D, *sl = sk + GT * KS, *part = sl + R;
  int2* ends = reinterpret_cast<int2*>(part + 8 * GT);
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  grid_dep_wait();
  const int s = blockIdx.z, kh = blockIdx.y, key0 = blockIdx.x * GT;
  const Sequence x = sequence_of(p.c, p.q, s, blockIdx.x == 0 && kh == 0 && tid == 0 ? p.status : nullptr);
  if (key0 >= x.len || x.start < 0) return;
  const int2 seen = tokens_over(p, x, key0, min(GT, x.len - key0)), rows = make_int2(seen.x * p.c.G, seen.y * p.c.G);
  if (rows.x >= rows.y && p.keep == 1.f && key0 + GT <= x.start) return;
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  if (rows.x < rows.y) {
    for (int i = tid; i < GT * C8; i += kWgtThreads) {
      const int t = i / C8, ch = i - t * C8, key = key0 + t;
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = 0.f;
      const int page = key < x.len ? page_of(p.c, s, key / p.c.g, p.status) : -1;
      if (page >= 0) cache_load8<kRowsF32, D>(p.c, p.c.k_pages, p.c.k_scale, page, kh, key % p.c.g, ch, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) sk[t * KS + ch * 8 + k] = v[k];
    }
  }
  for (int row0 = rows.x; row0 < rows.y; row0 += R) {
    __syncthreads();
    for (int i = tid; i < R * C8; i += kWgtThreads) {
      const int r = i / C8, ch = i - r * C8, row = row0 + r;
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = 0.f;
      if (row < rows.y) {
        const int t = row / p.c.G;
        load8(static_cast<const T*>(p.q.q) + (static_cast<long long>(x.cu) + t) * p.q.stride + (kh * p.c.G + row - t * p.c.G) * D + ch * 8, v);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) sq[r * D + ch * 8 + k] = v[k];
    }
    for (int r = tid; r < R; r += kWgtThreads) {
      const int row = row0 + r, t = row / p.c.G;
      const bool on = row < rows.y;
      const float l = on ? p.lse[(static_cast<long long>(x.cu) + t) * (p.c.Hkv * p.c.G) + kh * p.c.G + (row - t * p.c.G)] : -INFINITY;
      sl[r] = l * kLog2e;
      ends[r] = on && l != -INFINITY ? keys_of(p.q, x, x.start + t) : make_int2(0, 0);       // (a row that saw nothing gives nothing)
    }
    __syncthreads();
    float a[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) a[i][k] = 0.f;
#pragma unroll 2
    for (int c = 0; c < D; c += 4) {
      float4 u[8], b[4];
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = *reinterpret_cast<const float4*>(sq + (ty * 8 + i) * D + c);
#pragma unroll
      for (int k = 0; k < 4; ++k) b[k] = *reinterpret_cast<const float4*>(sk + (tx + 16 * k) * KS + c);
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) a[i][k] = fmaf(u[i].x, b[k].x, fmaf(u[i].y, b[k].y, fmaf(u[i].z, b[k].z, fmaf(u[i].w, b[k].w, a[i][k]))));
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int2 e = ends[ty * 8 + i];
      const float l = sl[ty * 8 + i];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int key = key0 + tx + 16 * k;
        if (key < e.x && (key >= e.y || key < p.q.sinks)) sum[k] += exp2f(fmaf(a[i][k], p.scale_log2, -l));
      }
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) part[ty * GT + tx + 16 * k] = sum[k];
  __syncthreads();
  if (tid < GT && key0 + tid < x.len) {
    float total = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) total += part[i * GT + tid];
    put_weight(p, held_weight(p, x, s, kh, key0 + tid), total);
  }
}
