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
// two at a time
__device__ __forceinline__ float max3_f32(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
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


// ---- quantised pages: a tile of 128 tokens as it lies in the cache, and as bf16 operands (which hold its values exactly)
template <int FMT, int D, int GP> struct RawTile {
  static constexpr int row = D * RowFormat<FMT>::bits / 8, pieces = row / 16, codes = 128 * row;
  static constexpr int scales = FMT == kRowsFp8 ? 128 / GP * 4 : 128 * (D / kInt4Run);       // a float per page, or a byte per run
  static constexpr int bytes = (codes + scales + 127) / 128 * 128;
};
__device__ __forceinline__ void copy_async16(uint32_t dst, const void* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
// One warp begins the copies of a tile's pages (lane `first` + j of `pages` names page j of the tile; -1: nobody sees it) to shared memory; `bar` (32 arrivals) completes
// when they have landed.
template <int FMT, int D, int GP>
__device__ __forceinline__ void raw_load(const CacheParams& c, const uint8_t* pool, const void* scales, int kh, int pages, int first, uint32_t dst, uint32_t bar) {
  using Raw = RawTile<FMT, D, GP>;
  const int lane = threadIdx.x & 31;
#pragma unroll 4
  for (int i = lane; i < 128 * Raw::pieces; i += 32) {
    const int t = i / Raw::pieces, page = __shfl_sync(0xffffffffu, pages, first + t / GP);
    if (page >= 0) copy_async16(dst + i * 16, pool + page * c.stride_page + kh * c.stride_head + (t % GP) * c.stride_tok + (i % Raw::pieces) * 16);
  }
  if constexpr (FMT == kRowsFp8) {
    const int page = __shfl_sync(0xffffffffu, pages, first + (lane & (128 / GP - 1)));
    if (lane < 128 / GP && page >= 0)
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst + Raw::codes + lane * 4), "l"(static_cast<const float*>(scales) + static_cast<size_t>(page) * c.Hkv + kh) : "memory");
  } else {
    constexpr int per = GP * (D / kInt4Run) / 16;    // 16-byte pieces of a page's scale bytes
    const int page = __shfl_sync(0xffffffffu, pages, first + (lane / per & (128 / GP - 1)));
    if (lane < Raw::scales / 16 && page >= 0)
      copy_async16(dst + Raw::codes + lane * 16, static_cast<const uint8_t*>(scales) + ((static_cast<size_t>(page) * c.Hkv + kh) * GP) * (D / kInt4Run) + lane % per * 16);
  }
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
// Four warps (id 0 .. 127) turn it into a swizzled operand tile.
template <int FMT, int D, int GP>
__device__ __forceinline__ void raw_convert(const uint8_t* raw, uint8_t* tile, int id) {
  using Raw = RawTile<FMT, D, GP>;
  constexpr int E = 128 / RowFormat<FMT>::bits;      // elements of a piece
#pragma unroll 2
  for (int i = id; i < 128 * Raw::pieces; i += 128) {
    const int t = i / Raw::pieces, piece = i % Raw::pieces;
    const uint4 u = *reinterpret_cast<const uint4*>(raw + i * 16);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    float scale;
    if constexpr (FMT == kRowsFp8) scale = *reinterpret_cast<const float*>(raw + Raw::codes + t / GP * 4);
    else scale = int4_scale_value(raw[Raw::codes + i]);
#pragma unroll
    for (int k = 0; k < E / 8; ++k) {
      float v[8];
      if constexpr (FMT == kRowsFp8) {
        fp8_decode8(make_uint2(w[2 * k], w[2 * k + 1]), v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= scale;
      } else {
        int4_decode8(w[k], scale, v);
      }
      const int c = piece * (E / 8) + k;
      *reinterpret_cast<uint4*>(tile + (c >> 3) * (128 * 128) + tc5_sw(t, c & 7)) =
          make_uint4(pack_b16(v[0], v[1]), pack_b16(v[2], v[3]), pack_b16(v[4], v[5]), pack_b16(v[6], v[7]));
    }
  }
}

}  // namespace losa
