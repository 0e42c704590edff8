// The 8-bit cache's format on the device: e4m3 codes, and for each head and block of 32 rows a scale s = 2^k with k the
// smallest integer, -100 <= k <= 119, for which the block's largest magnitude is at most 448 s.
//
// Powers of two: e4m3's relative steps do not depend on the scale then, so a block whose scale grows keeps its codes' values
// (but for e4m3's subnormals), and code * s has 4 significant bits, which bf16 holds.  k >= -100 keeps every code * s a normal
// bf16 number; k <= 119 keeps 448 s below infinity.
#pragma once

#include <cuda_fp16.h>
#include <stdint.h>

namespace stepkv {

constexpr int kQ8Block = STEPKV_Q8_BLOCK;
constexpr int kQ8MinExp = -100, kQ8MaxExp = 119;

// The scale 2^k of a largest magnitude (finite, not negative).  448 = 1.75 2^8: with m = 1.f 2^(e - 127), k = e - 127 - 8, and
// one more where 1.f > 1.75.
__device__ __forceinline__ float q8_scale(float most) {
  const uint32_t b = __float_as_uint(most);
  const int k = (int)(b >> 23) - 135 + ((b & 0x7FFFFFu) > 0x600000u);
  return __uint_as_float((uint32_t)(min(max(k, kQ8MinExp), kQ8MaxExp) + 127) << 23);
}
// 1 / s for s = 2^k, exactly.
__device__ __forceinline__ float q8_inverse(float s) { return __uint_as_float((254u << 23) - __float_as_uint(s)); }

// Two codes (the first in the low byte) as fp16, exactly; and two values as codes, ties to even, saturating, NaN for NaN.
__device__ __forceinline__ uint32_t q8_half2(uint32_t codes) {
  uint32_t r;
  asm("{\n .reg .b16 c;\n cvt.u16.u32 c, %1;\n cvt.rn.f16x2.e4m3x2 %0, c;\n}\n" : "=r"(r) : "r"(codes));
  return r;
}
__device__ __forceinline__ float2 q8_float2(uint32_t codes) {
  const uint32_t h = q8_half2(codes);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
__device__ __forceinline__ uint32_t q8_codes2(float lo, float hi) {
  uint32_t r;
  asm("{\n .reg .b16 c;\n cvt.rn.satfinite.e4m3x2.f32 c, %2, %1;\n cvt.u32.u16 %0, c;\n}\n" : "=r"(r) : "f"(lo), "f"(hi));
  return r;
}

// Four codes (a word) under a scale `ratio` times as fine: e4m3(code * ratio).
__device__ __forceinline__ uint32_t q8_rescale(uint32_t w, float ratio) {
  const float2 a = q8_float2(w & 0xFFFFu), b = q8_float2(w >> 16);
  return q8_codes2(a.x * ratio, a.y * ratio) | q8_codes2(b.x * ratio, b.y * ratio) << 16;
}
__device__ __forceinline__ uint4 q8_rescale(const uint4& v, float ratio) {
  return make_uint4(q8_rescale(v.x, ratio), q8_rescale(v.y, ratio), q8_rescale(v.z, ratio), q8_rescale(v.w, ratio));
}

// A warp brings the rows of `rows` (a bit each) of a block to a scale `ratio` times as fine, 16 bytes a lane, AT loads ahead.
template <int D, int AT>
__device__ __forceinline__ void q8_rescale_rows(uint8_t* block, uint32_t rows, float ratio) {
  constexpr int LPR = D / 16, RPI = 32 / LPR, NI = kQ8Block / RPI;
  const int lane = threadIdx.x & 31, sub = lane / LPR;
  uint4* p = reinterpret_cast<uint4*>(block) + lane;
#pragma unroll 1
  for (int u0 = 0; u0 < NI; u0 += AT) {
    uint4 v[AT];
#pragma unroll
    for (int u = 0; u < AT; ++u)
      if (rows >> ((u0 + u) * RPI + sub) & 1u) v[u] = __ldcg(p + (u0 + u) * 32);
#pragma unroll
    for (int u = 0; u < AT; ++u)
      if (rows >> ((u0 + u) * RPI + sub) & 1u) p[(u0 + u) * 32] = q8_rescale(v[u], ratio);
  }
}

constexpr int kQ8Threads = 256;  // of a CTA of the kernels that move rows

__device__ __forceinline__ uint4 q8_ld_stream(const void* p) {
  uint4 v;
  asm volatile("ld.global.cs.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ void q8_st_stream(void* p, const uint4& v) {
  asm volatile("st.global.cs.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// (n_chunks >= 1.)
// The chunks of a warp: chunk `pos` of row set `set` (layer, tensor, head), every `step`-th of the list of all sets' chunks.
struct Q8Chunks {
  int chunks, sets;
  int set, pos;
  int d_set, d_pos;
  __device__ __forceinline__ Q8Chunks(int n_chunks, int n_sets) : chunks(n_chunks), sets(n_sets) {
    const int step = gridDim.x * (kQ8Threads / 32), first = blockIdx.x * (kQ8Threads / 32) + (threadIdx.x >> 5);
    set = first / chunks;
    pos = first - set * chunks;
    d_set = step / chunks;
    d_pos = step - d_set * chunks;
  }
  __device__ __forceinline__ bool any() const { return set < sets; }
  __device__ __forceinline__ void next() {
    set += d_set;
    pos += d_pos;
    if (pos >= chunks) {
      pos -= chunks;
      ++set;
    }
  }
};

}  // namespace stepkv
