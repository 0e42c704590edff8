// A cache held in 8 bits (format in q8.cuh): quantising rows as they are appended, and reading them back.
//
// (Launched dependently: what a kernel before may have written is read after the wait, and not by the read-only path.)
#include <algorithm>

#include "common.cuh"
#include "fastdiv.h"
#include "internal.h"
#include "q8.cuh"

namespace stepkv {

struct Q8Args {
  const void* src[2 * kQ8Layers];  // per (layer, tensor): bf16 rows, or the codes where they are read
  void* dst[2 * kQ8Layers];        // the codes where they are written, or bf16 rows
  float* scale[2 * kQ8Layers];
  int64_t head_stride, row_stride; // of the bf16 rows, elements
  int64_t code_head_stride;        // bytes
  int64_t scale_head_stride;       // floats
  FastDiv by_heads, by_tensors;
  int sets;                        // layers * tensors * Hkv
  int layer0;                      // of row0_dev
  int T;                           // rows of the source
  int rows;                        // rows of the cache
  Q4Rows r;
  int32_t* status;
};
static_assert(sizeof(Q8Args) <= 32000, "kernel parameter space");

// The rows of a call, as every warp of it sees them: count -1 where nothing may be done.
__device__ __forceinline__ int q8_count(const Q4Rows& r, int32_t* status) {
  if (!r.n_dev) return r.n;
  const int n = *r.n_dev;
  if (n >= 0 && n <= r.n) return n;
  if (blockIdx.x == 0 && threadIdx.x == 0) record_status(status, n < 0 ? STEPKV_EDATA : STEPKV_ENOSPACE);
  return -1;
}

// A warp takes a block of 32 rows: all of it in registers (64 a lane at d = 128), its largest magnitude by a reduction over
// the warp, then the codes.  A lane has 8 consecutive channels of every 2nd (4th) row.  (With three CTAs an SM, d = 128, 15 words
// of a lane's 80 go through local memory, which is L1's: still the faster of the two.)
// CTAs an SM holds: two have the registers for all of a block's loads at once, which is faster where a warp has few blocks to take
// (1 layer x 8 heads x 8272 rows 8.0 us, with three 10.1); with many, three (d = 64: four) keep more in flight (32 layers x
// 8272 rows 271 -> 253 us = 6.4 TB/s, 639 rows 23.6 -> 21.1; 64 channels x 4000 rows 79 -> 65).  By index, 8272 of 32768 rows: 259
// us of 32 layers; of one layer, out of DRAM, 19.6, and 16.6 in order.
constexpr int q8_write_ctas(int D, bool many) { return !many ? 2 : D == 128 ? 3 : 4; }
constexpr int kQ8WriteFew = 3;  // blocks a warp
template <int D, bool IDX, bool MANY>
__global__ void __launch_bounds__(kQ8Threads, q8_write_ctas(D, MANY)) q8_write_kernel(const __grid_constant__ Q8Args a) {
  constexpr int LPR = D / 8, RPI = 32 / LPR, NI = kQ8Block / RPI;  // lanes a row, rows an instruction, instructions a block
  pdl_wait();
  pdl_launch_dependents();
  const int n = q8_count(a.r, a.status);
  if (n <= 0) return;
  const int lane = threadIdx.x & 31, sub = lane / LPR, col = lane & (LPR - 1);
  for (Q8Chunks c((int)(((int64_t)n + 2 * kQ8Block - 2) / kQ8Block), a.sets); c.any(); c.next()) {  // (blocks that n rows touch at most)
    int h;
    const int lt = fdivmod(c.set, a.by_heads, h), layer = fdiv(lt, a.by_tensors);
    const int row0 = a.r.row0_dev ? a.r.row0_dev[(a.layer0 + layer) * a.r.row0_stride] : a.r.row0;
    if (row0 < 0 || (int64_t)row0 + n > a.rows) {
      if (lane == 0) record_status(a.status, STEPKV_ENOSPACE);
      continue;
    }
    const int lead = c.pos == 0 ? row0 & (kQ8Block - 1) : 0;                          // rows of the block that stay
    const int t0 = c.pos * kQ8Block - (row0 & (kQ8Block - 1));                        // the row of the call that is the block's row 0
    const int end = min(kQ8Block, n - t0);                                            // rows of the block up to the last written
    if (end <= 0) continue;
    const int64_t block = row0 / kQ8Block + c.pos;
    const uint16_t* src = static_cast<const uint16_t*>(a.src[lt]) + (int64_t)h * a.head_stride + col * 8;
    int at = t0 + lane;  // lane i: the source's row of the block's row i, -1 for none
    if (lane < lead || lane >= end) {
      at = -1;
    } else if (IDX) {
      at = __ldcg(a.r.idx + at);
      if (at < 0 || at >= a.T) {
        record_status(a.status, STEPKV_EDATA);
        at = -1;
      }
    }
    uint4 v[NI];
#pragma unroll
    for (int u = 0; u < NI; ++u) {
      const int t = __shfl_sync(0xffffffffu, at, u * RPI + sub);
      v[u] = make_uint4(0, 0, 0, 0);
      if (t >= 0) v[u] = q8_ld_stream(src + t * a.row_stride);
    }
    uint32_t most2 = 0;  // of the channels of even, and of odd number: bf16 magnitudes, which order as integers
#pragma unroll
    for (int u = 0; u < NI; ++u) {
      const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) most2 = __vmaxu2(most2, w[i] & 0x7FFF7FFFu);
    }
    uint32_t most = __reduce_max_sync(0xffffffffu, max(most2 & 0xFFFFu, most2 >> 16));
    if (most >= 0x7F80u) {  // infinities or NaN: they become NaN and do not count
      most = 0;
#pragma unroll 1
      for (int u = 0; u < NI; ++u) {
        // (indexing a register array by u would put it into local memory: the row is read again)
        const int t = __shfl_sync(0xffffffffu, at, u * RPI + sub);
        if (t < 0) continue;
        const uint4 x = q8_ld_stream(src + t * a.row_stride);
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t b = w[i >> 1] >> (16 * (i & 1)) & 0x7FFFu;
          if (b < 0x7F80u) most = max(most, b);
        }
      }
      most = __reduce_max_sync(0xffffffffu, most);
#pragma unroll
      for (int u = 0; u < NI; ++u) {
        uint32_t* w = reinterpret_cast<uint32_t*>(&v[u]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if ((w[i] & 0x7F80u) == 0x7F80u) w[i] |= 0x7FFFu;
          if ((w[i] & 0x7F800000u) == 0x7F800000u) w[i] |= 0x7FFF0000u;
        }
      }
    }
    float s = q8_scale(__uint_as_float(most << 16));
    uint8_t* codes = static_cast<uint8_t*>(a.dst[lt]) + (int64_t)h * a.code_head_stride + block * (kQ8Block * D);
    float* scale = a.scale[lt] + (int64_t)h * a.scale_head_stride + block;
    if (lead > 0) {
      const float old = __ldcg(scale);
      if (old > s) {
        s = old;
      } else if (old < s) {  // (some words of a lane at a time: the new rows are in registers)
        constexpr int kAt = MANY ? 2 : 8;
        const float ratio = old * q8_inverse(s);
        uint32_t* w = reinterpret_cast<uint32_t*>(codes) + lane;
        const int words = lead * (D / 4);
#pragma unroll 1
        for (int i = 0; i < words; i += kAt * 32) {
          uint32_t x[kAt];
#pragma unroll
          for (int k = 0; k < kAt; ++k) x[k] = i + k * 32 + lane < words ? __ldcg(w + i + k * 32) : 0u;
#pragma unroll
          for (int k = 0; k < kAt; ++k)
            if (i + k * 32 + lane < words) w[i + k * 32] = q8_rescale(x[k], ratio);
        }
      }
      __syncwarp();  // every lane has read the old scale
    }
    const float inv = q8_inverse(s);
#pragma unroll
    for (int u = 0; u < NI; ++u) {
      const int i = u * RPI + sub;
      const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
      uint32_t p[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        p[k] = q8_codes2(__uint_as_float(w[k] << 16) * inv, __uint_as_float(w[k] & 0xFFFF0000u) * inv);
      if (i >= lead && i < end)
        *reinterpret_cast<uint2*>(codes + i * D + col * 8) = make_uint2(p[0] | p[1] << 16, p[2] | p[3] << 16);
    }
    if (lane == 0) *scale = s;
  }
}

// A lane takes 8 codes of a row.  32 layers x 8 heads x 8272 rows: 265 us = 6.1 TB/s, 64 layers x 4240 rows 6.2; two and eight rows of
// a lane in flight, 3 to 16 CTAs an SM and plain stores 266-279.
// Right behind a call of this library it takes longer: its CTAs are launched while that one's still fill the SMs, gather on those that
// are free first, up to eight on one, and each keeps its share of the rows.  After an eviction of 256 heads (38 us) the two take 373
// us, launched in ordinary order 303; 639 rows written and read back 47 us, 37.
constexpr int kQ8ReadUnroll = 4;
constexpr int kQ8ReadCtas = 4;

template <int D, bool IDX>
__global__ void __launch_bounds__(kQ8Threads) q8_read_kernel(const __grid_constant__ Q8Args a) {
  constexpr int LPR = D / 8, RPI = 32 / LPR, kChunk = RPI * kQ8ReadUnroll;
  pdl_wait();
  pdl_launch_dependents();
  const int n = q8_count(a.r, a.status);
  if (n <= 0) return;
  const int lane = threadIdx.x & 31, sub = lane / LPR, col = lane & (LPR - 1);
  for (Q8Chunks c((n + kChunk - 1) / kChunk, a.sets); c.any(); c.next()) {
    int h;
    const int lt = fdivmod(c.set, a.by_heads, h), layer = fdiv(lt, a.by_tensors);
    int row0 = 0;
    if (!IDX) {
      row0 = a.r.row0_dev ? a.r.row0_dev[(a.layer0 + layer) * a.r.row0_stride] : a.r.row0;
      if (row0 < 0 || (int64_t)row0 + n > a.rows) {
        if (lane == 0) record_status(a.status, STEPKV_EDATA);
        continue;
      }
    }
    const int r0 = c.pos * kChunk + sub;
    const uint8_t* codes = static_cast<const uint8_t*>(a.src[lt]) + (int64_t)h * a.code_head_stride + col * 8;
    const float* scales = a.scale[lt] + (int64_t)h * a.scale_head_stride;
    uint16_t* dst = static_cast<uint16_t*>(a.dst[lt]) + (int64_t)h * a.head_stride + r0 * a.row_stride + col * 8;
    int t[kQ8ReadUnroll];
    uint2 w[kQ8ReadUnroll];
    float s[kQ8ReadUnroll];
#pragma unroll
    for (int u = 0; u < kQ8ReadUnroll; ++u) {
      const int r = r0 + u * RPI;
      t[u] = -1;
      if (r < n) {
        t[u] = IDX ? __ldcg(a.r.idx + r) : row0 + r;
        if (IDX && (t[u] < 0 || t[u] >= a.rows)) {
          record_status(a.status, STEPKV_EDATA);
          t[u] = -1;
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kQ8ReadUnroll; ++u) {
      w[u] = make_uint2(0, 0);
      s[u] = 0.f;
      if (t[u] >= 0) {
        w[u] = __ldcg(reinterpret_cast<const uint2*>(codes + (int64_t)t[u] * D));
        s[u] = __ldcg(scales + t[u] / kQ8Block);
      }
    }
    const int64_t step = RPI * a.row_stride;
#pragma unroll
    for (int u = 0; u < kQ8ReadUnroll; ++u) {
      uint32_t p[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 f = q8_float2(((k < 2 ? w[u].x : w[u].y) >> (16 * (k & 1))) & 0xFFFFu);
        p[k] = __byte_perm(__float_as_uint(f.x * s[u]), __float_as_uint(f.y * s[u]), 0x7632);  // exact in bf16
      }
      if (t[u] >= 0) q8_st_stream(dst + u * step, make_uint4(p[0], p[1], p[2], p[3]));
    }
  }
}

// Write and read differ in which side the bf16 rows are on.
template <int D>
static stepkv_status_t q8_rows_run(bool write, const stepkv_q8_cache_t& c, const void* const* K, const void* const* V,
                                   int64_t head_stride, int64_t row_stride, int T, const Q4Rows& rows, int32_t* status,
                                   cudaStream_t stream) {
  int n_sm = 0;
  cudaError_t e = device_sm_count(&n_sm);
  for (int l0 = 0; e == cudaSuccess && l0 < c.n_layers; l0 += kQ8Layers) {
    const int nl = std::min(kQ8Layers, c.n_layers - l0);
    Q8Args a;
    memset(&a, 0, sizeof(a));
    int lt = 0;
    for (int l = l0; l < l0 + nl; ++l) {
      for (int t = 0; t < 2; ++t) {
        const void* const* x = t ? V : K;
        if (!x) continue;
        void* codes = t ? c.V[l] : c.K[l];
        a.src[lt] = write ? x[l] : codes;
        a.dst[lt] = write ? codes : const_cast<void*>(x[l]);
        a.scale[lt] = t ? c.V_scale[l] : c.K_scale[l];
        ++lt;
      }
    }
    a.head_stride = head_stride;
    a.row_stride = row_stride;
    a.code_head_stride = c.code_head_stride;
    a.scale_head_stride = c.scale_head_stride;
    a.by_heads = make_fastdiv(c.Hkv);
    a.by_tensors = make_fastdiv((K != nullptr) + (V != nullptr));
    a.sets = lt * c.Hkv;
    a.layer0 = l0;
    a.T = T;
    a.rows = c.rows;
    a.r = rows;
    a.status = status;
    const int per_chunk = write ? kQ8Block : 256 / D * kQ8ReadUnroll;
    const int64_t chunks = (int64_t)a.sets * ((rows.n + (write ? 2 * kQ8Block - 2 : per_chunk - 1)) / per_chunk);
    const int64_t ctas = (chunks + kQ8Threads / 32 - 1) / (kQ8Threads / 32);
    const bool many = write && ctas > kQ8WriteFew * n_sm * q8_write_ctas(D, false);
    const int grid = (int)std::max<int64_t>(1, std::min<int64_t>(n_sm * (write ? q8_write_ctas(D, many) : kQ8ReadCtas), ctas));
    auto kern = !write ? (rows.idx ? q8_read_kernel<D, true> : q8_read_kernel<D, false>)
                : many ? (rows.idx ? q8_write_kernel<D, true, true> : q8_write_kernel<D, false, true>)
                       : (rows.idx ? q8_write_kernel<D, true, false> : q8_write_kernel<D, false, false>);
    e = launch_kernel(kern, dim3(grid), dim3(kQ8Threads), 0, stream, a, true);
  }
  if (e == cudaSuccess) return STEPKV_OK;
  set_last_cuda_error(e);
  return STEPKV_ECUDA;
}

stepkv_status_t q8_write_run(const stepkv_q8_cache_t& c, const void* const* K, const void* const* V, int64_t head_stride,
                             int64_t row_stride, int T, const Q4Rows& rows, int32_t* status, cudaStream_t stream) {
  return (c.d == 128 ? q8_rows_run<128> : q8_rows_run<64>)(true, c, K, V, head_stride, row_stride, T, rows, status, stream);
}

stepkv_status_t q8_read_run(const stepkv_q8_cache_t& c, const Q4Rows& rows, void* const* K, void* const* V,
                            int64_t head_stride, int64_t row_stride, int32_t* status, cudaStream_t stream) {
  return (c.d == 128 ? q8_rows_run<128> : q8_rows_run<64>)(false, c, K, V, head_stride, row_stride, c.rows, rows, status, stream);
}

}  // namespace stepkv
