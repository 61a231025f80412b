// What the tensor-core kernels of windowed attention and of the keys' weights share: pages by TMA, arithmetic on two numbers at a time.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>

#include "cache_view.cuh"
#include "tcgen05_ops.cuh"

namespace losa {

// a page's tokens by 64 elements, swizzled
__device__ __forceinline__ void tma_load_page(uint32_t dst, const CUtensorMap* map, uint32_t bar, int col, int head, int page) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
               ::"r"(dst), "l"(map), "r"(bar), "r"(col), "r"(0), "r"(head), "r"(page) : "memory");
}
// a box of queries: the heads of a KV head of consecutive tokens, 64 elements of each
__device__ __forceinline__ void tma_load_queries(uint32_t dst, const CUtensorMap* map, uint32_t bar, int col, int head, int token) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
               ::"r"(dst), "l"(map), "r"(bar), "r"(col), "r"(head), "r"(token) : "memory");
}
// two at a time
__device__ __forceinline__ float2 fma2_f32(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\tfma.rn.f32x2 z, x, y, z;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2_f32(float2 a, float2 b) {
  float2 c;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(c.x), "=f"(c.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return c;
}
__device__ __forceinline__ uint32_t pack_b16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }


// ---- quantised pages: a tile of 128 tokens as it lies in the cache, and as 16-bit operands (which hold its values exactly)
template <int FMT, int D, int GP> struct RawTile {
  static constexpr int row = D * RowFormat<FMT>::bits / 8, pieces = row / 16, codes = 128 * row, pages = 128 / GP;
  static constexpr int scales = FMT == kRowsFp8 ? pages * 4 : 128 * (D / kInt4Run);          // a float per page, or a byte per run
  static constexpr int bytes = (codes + scales + 127) / 128 * 128;
};
// One warp begins the copies of a tile's pages to shared memory (lane `first` + j of `pages` names page j of the tile; -1: nobody sees it).  FP8: that lane of `scale` holds the
// page's scale.  `bar` (one arrival) completes when they have landed.
template <int FMT, int D, int GP>
__device__ __forceinline__ void raw_load(const CacheParams& c, const CUtensorMap* map, const void* scales, int kh, int pages, float scale, int first, uint32_t dst, uint32_t bar) {
  using Raw = RawTile<FMT, D, GP>;
  constexpr int kScaleBytes = GP * (D / kInt4Run);   // of a 4-bit page
  const int lane = threadIdx.x & 31;
  const uint32_t have = __ballot_sync(0xffffffffu, pages >= 0) >> first & ((1u << Raw::pages) - 1u);
  if constexpr (FMT == kRowsFp8) {
    if (lane >= first && lane < first + Raw::pages) asm volatile("st.shared.f32 [%0], %1;" ::"r"(dst + Raw::codes + (lane - first) * 4), "f"(scale) : "memory");
    __syncwarp();
  }
  if (elect_one()) mbar_expect_tx(bar, __popc(have) * (GP * Raw::row + (FMT == kRowsInt4 ? kScaleBytes : 0)));
  __syncwarp();
  const int j = lane - first;
  if (j >= 0 && j < Raw::pages && pages >= 0) {
    tma_load_page(dst + j * GP * Raw::row, map, bar, 0, kh, pages);
    if constexpr (FMT == kRowsInt4)
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst + Raw::codes + j * kScaleBytes),
                   "l"(static_cast<const uint8_t*>(scales) + (static_cast<size_t>(pages) * c.Hkv + kh) * kScaleBytes), "r"(kScaleBytes), "r"(bar) : "memory");
  }
  __syncwarp();
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t add_f16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("add.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// Eight elements as fp16, every step exact.  FP8: codes times a power of two from 2^-6 to 2^7.
__device__ __forceinline__ uint4 fp8_half8(uint2 w, uint32_t scale2) {
  const uint32_t x[2] = {w.x, w.y};
  uint32_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(x[i >> 1] >> (16 * (i & 1))), __NV_E4M3);
    h[i] = mul_f16x2(static_cast<uint32_t>(r.x) | (static_cast<uint32_t>(r.y) << 16), scale2);
  }
  return make_uint4(h[0], h[1], h[2], h[3]);
}
// 4 bits: of two codes u in a byte, as integers in the mantissa of 1024, the lower one counts 1, the upper one 16: less 1024 + 8 and 1024 + 128, times the scale and a sixteenth of it.
__device__ __forceinline__ uint4 int4_half8(uint32_t w, uint32_t scale, uint32_t scale16) {
  const uint32_t mul = scale | (scale16 << 16);
  uint32_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t twice = __byte_perm(w, 0u, 0x4040 | (i << 8) | i);                       // the byte in both halves
    h[i] = mul_f16x2(add_f16x2((twice & 0x00f0000fu) | 0x64006400u, 0xe480e408u), mul);     // -1152, -1032
  }
  return make_uint4(h[0], h[1], h[2], h[3]);
}
// Four warps (id 0 .. 127) turn it into a swizzled operand tile of fp16 (HALF) or bf16.
template <int FMT, int D, int GP, bool HALF>
__device__ __forceinline__ void raw_convert(const uint8_t* raw, uint8_t* tile, int id) {
  using Raw = RawTile<FMT, D, GP>;
  constexpr int E = 128 / RowFormat<FMT>::bits;      // elements of a piece
#pragma unroll 1
  for (int i = id; i < 128 * Raw::pieces; i += 128) {
    const int t = i / Raw::pieces, piece = i % Raw::pieces;
    const uint4 u = *reinterpret_cast<const uint4*>(raw + i * 16);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    float scale;
    if constexpr (FMT == kRowsFp8) scale = *reinterpret_cast<const float*>(raw + Raw::codes + t / GP * 4);
    else scale = int4_scale_value(raw[Raw::codes + i]);
    [[maybe_unused]] const uint32_t half = __half_as_ushort(__float2half_rn(scale)), half16 = __half_as_ushort(__float2half_rn(scale * 0.0625f));
#pragma unroll
    for (int k = 0; k < E / 8; ++k) {
      uint4 out;
      if constexpr (HALF && FMT == kRowsFp8) {
        out = fp8_half8(make_uint2(w[2 * k], w[2 * k + 1]), half | (half << 16));
      } else if constexpr (HALF) {
        out = int4_half8(w[k], half, half16);
      } else {
        float v[8];
        if constexpr (FMT == kRowsFp8) {
          fp8_decode8(make_uint2(w[2 * k], w[2 * k + 1]), v);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] *= scale;
        } else {
          int4_decode8(w[k], scale, v);
        }
        out = make_uint4(pack_b16(v[0], v[1]), pack_b16(v[2], v[3]), pack_b16(v[4], v[5]), pack_b16(v[6], v[7]));
      }
      const int c = piece * (E / 8) + k;
      *reinterpret_cast<uint4*>(tile + (c >> 3) * (128 * 128) + tc5_sw(t, c & 7)) = out;
    }
  }
}

}  // namespace losa
