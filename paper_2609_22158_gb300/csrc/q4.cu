// A cache held in 4 bits: quantising rows as they are written, reading them back, and moving retained rows
// (Eq. 1's C_hat with 4.5 bits a channel).
//
// A row is cut into groups of 32 channels; a group has one fp16 scale s of 5 significant bits and 32 codes n in 0..15, a
// code stands for s (n - 8):
//   x* = M if M >= -m else m,   s = fp16(r5(-x* / 8)),   n = 8 + clamp(rint(x / s), -8, 7)
// Five bits of scale times three of code fit bf16's eight, so reading back is exact, and so is quantising what was read
// back.  Everything is row-local, so a compaction moves codes and scales as they are.
//
// All three kernels stream: a warp takes chunks of a few rows of one row set (layer, tensor, head), a lane 8 channels
// (16 bytes of bf16, one 32-bit word of codes), a quad of lanes a group.
#include <cuda_fp16.h>

#include <algorithm>

#include "common.cuh"
#include "fastdiv.h"
#include "internal.h"

namespace stepkv {

constexpr int kQ4Threads = 256;
constexpr int kQ4Unroll = 4;       // row groups of a warp's chunk

struct Q4Args {
  const void* src[2 * kQ4Layers];  // per (layer, tensor): bf16 rows, or the codes where they are read
  void* dst[2 * kQ4Layers];        // the codes where they are written, or bf16 rows
  void* scale[2 * kQ4Layers];
  int64_t head_stride, row_stride; // of the bf16 rows, elements
  int64_t code_head_stride;        // bytes
  int64_t scale_head_stride;       // elements
  FastDiv by_heads, by_tensors;
  int sets;                        // layers * tensors * Hkv
  int layer0;                      // of row0_dev
  int d;
  int T;                           // rows of the source
  int rows;                        // rows of the cache
  Q4Rows r;
  int32_t* status;
};
static_assert(sizeof(Q4Args) <= 32000, "kernel parameter space");

// The rows of a call, as every warp of it sees them: count -1 where nothing may be done.
__device__ __forceinline__ int q4_count(const Q4Rows& r, int32_t* status) {
  if (!r.n_dev) return r.n;
  const int n = *r.n_dev;
  if (n >= 0 && n <= r.n) return n;
  if (blockIdx.x == 0 && threadIdx.x == 0) record_status(status, n < 0 ? STEPKV_EDATA : STEPKV_ENOSPACE);
  return -1;
}

__device__ __forceinline__ uint4 q4_ld_stream(const void* p) {
  uint4 v;
  asm volatile("ld.global.cs.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ void q4_st_stream(void* p, const uint4& v) {
  asm volatile("st.global.cs.v4.u32 [%0], {%1,%2,%3,%4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// max / min that give NaN where either is one
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// The scale of a group from its maximum and minimum.
__device__ __forceinline__ __half q4_scale(float hi, float lo) {
  const float x = hi >= -lo ? hi : lo;
  if (!(fabsf(x) < INFINITY)) return __ushort_as_half(0x7FFF);
  uint32_t b = __float_as_uint(x * -0.125f);
  b = (b + 0x3FFFFu + ((b >> 19) & 1u)) & ~0x7FFFFu;  // 4 of the 23 explicit bits, ties to even
  return __float2half_rn(fminf(fmaxf(__uint_as_float(b), -896.f), 896.f));
}

// The codes of 8 channels as one word, channel i in bits 4i .. 4i + 3.
__device__ __forceinline__ uint32_t q4_codes(const float (&x)[8], __half s) {
  const float step = __half2float(s);
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float q = step == 0.f || step != step ? 0.f : fminf(fmaxf(rintf(x[i] / step), -8.f), 7.f);
    w |= (uint32_t)((int)q + 8) << (4 * i);
  }
  return w;
}

__device__ __forceinline__ void bf16x8_to_float(const uint4& v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}

// Where a warp's chunk lies: row set -> (layer, tensor) entry, layer and head.
struct Q4Set {
  int lt, layer, h;
};
__device__ __forceinline__ Q4Set q4_set(const Q4Args& a, int set) {
  Q4Set s;
  s.lt = fdivmod(set, a.by_heads, s.h);
  s.layer = fdiv(s.lt, a.by_tensors);
  return s;
}

__global__ void __launch_bounds__(kQ4Threads) q4_write_kernel(const __grid_constant__ Q4Args a) {
  pdl_wait();
  pdl_launch_dependents();
  const int n = q4_count(a.r, a.status);
  if (n <= 0) return;
  const int lpr = a.d >> 3, rpi = 32 / lpr;  // lanes a row, rows an instruction
  const int lane = threadIdx.x & 31, sub = lane / lpr, col = lane - sub * lpr;
  const int per_chunk = rpi * kQ4Unroll, chunks = (n + per_chunk - 1) / per_chunk;
  const int total = a.sets * chunks;
  const int warps = gridDim.x * (kQ4Threads / 32);
  for (int c = blockIdx.x * (kQ4Threads / 32) + (threadIdx.x >> 5); c < total; c += warps) {
    const int set = c / chunks, r0 = (c - set * chunks) * per_chunk;
    const Q4Set s = q4_set(a, set);
    const int row0 = a.r.row0_dev ? a.r.row0_dev[(a.layer0 + s.layer) * a.r.row0_stride] : a.r.row0;
    if (row0 < 0 || (int64_t)row0 + n > a.rows) {
      if (lane == 0) record_status(a.status, STEPKV_ENOSPACE);
      continue;
    }
    const uint16_t* src = static_cast<const uint16_t*>(a.src[s.lt]) + (int64_t)s.h * a.head_stride + col * 8;
    uint8_t* codes = static_cast<uint8_t*>(a.dst[s.lt]) + (int64_t)s.h * a.code_head_stride;
    __half* scales = static_cast<__half*>(a.scale[s.lt]) + (int64_t)s.h * a.scale_head_stride;
    uint4 v[kQ4Unroll];
    bool ok[kQ4Unroll];
#pragma unroll
    for (int u = 0; u < kQ4Unroll; ++u) {
      const int r = r0 + u * rpi + sub;
      ok[u] = sub < rpi && r < n;
      v[u] = make_uint4(0, 0, 0, 0);
      if (ok[u]) {
        const int t = a.r.idx ? a.r.idx[r] : r;
        if (t < 0 || t >= a.T) {
          record_status(a.status, STEPKV_EDATA);
          ok[u] = false;
        } else {
          v[u] = q4_ld_stream(src + (int64_t)t * a.row_stride);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kQ4Unroll; ++u) {
      float x[8];
      bf16x8_to_float(v[u], x);
      float hi = x[0], lo = x[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) {
        hi = max_nan(hi, x[i]);
        lo = min_nan(lo, x[i]);
      }
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) {
        hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
      }
      const __half sc = q4_scale(hi, lo);
      const uint32_t w = q4_codes(x, sc);
      if (ok[u]) {
        const int64_t row = (int64_t)row0 + r0 + u * rpi + sub;
        *reinterpret_cast<uint32_t*>(codes + row * (a.d >> 1) + col * 4) = w;
        if ((col & 3) == 0) scales[row * (a.d >> 5) + (col >> 2)] = sc;
      }
    }
  }
}

__global__ void __launch_bounds__(kQ4Threads) q4_read_kernel(const __grid_constant__ Q4Args a) {
  pdl_wait();
  pdl_launch_dependents();
  const int n = q4_count(a.r, a.status);
  if (n <= 0) return;
  const int lpr = a.d >> 3, rpi = 32 / lpr;
  const int lane = threadIdx.x & 31, sub = lane / lpr, col = lane - sub * lpr;
  const int per_chunk = rpi * kQ4Unroll, chunks = (n + per_chunk - 1) / per_chunk;
  const int total = a.sets * chunks;
  const int warps = gridDim.x * (kQ4Threads / 32);
  for (int c = blockIdx.x * (kQ4Threads / 32) + (threadIdx.x >> 5); c < total; c += warps) {
    const int set = c / chunks, r0 = (c - set * chunks) * per_chunk;
    const Q4Set s = q4_set(a, set);
    int row0 = 0;
    if (!a.r.idx) {
      row0 = a.r.row0_dev ? a.r.row0_dev[(a.layer0 + s.layer) * a.r.row0_stride] : a.r.row0;
      if (row0 < 0 || (int64_t)row0 + n > a.rows) {
        if (lane == 0) record_status(a.status, STEPKV_EDATA);
        continue;
      }
    }
    const uint8_t* codes = static_cast<const uint8_t*>(a.src[s.lt]) + (int64_t)s.h * a.code_head_stride;
    const __half* scales = static_cast<const __half*>(a.scale[s.lt]) + (int64_t)s.h * a.scale_head_stride;
    uint16_t* dst = static_cast<uint16_t*>(a.dst[s.lt]) + (int64_t)s.h * a.head_stride + col * 8;
#pragma unroll
    for (int u = 0; u < kQ4Unroll; ++u) {
      const int r = r0 + u * rpi + sub;
      if (sub >= rpi || r >= n) continue;
      const int64_t row = a.r.idx ? a.r.idx[r] : (int64_t)row0 + r;
      if (row < 0 || row >= a.rows) {
        record_status(a.status, STEPKV_EDATA);
        continue;
      }
      const uint32_t w = *reinterpret_cast<const uint32_t*>(codes + row * (a.d >> 1) + col * 4);
      const float step = __half2float(scales[row * (a.d >> 5) + (col >> 2)]);
      uint32_t o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {  // exact in bf16: the upper halves of the fp32 values
        const float x = (float)((int)((w >> (8 * i)) & 15u) - 8) * step, y = (float)((int)((w >> (8 * i + 4)) & 15u) - 8) * step;
        o[i] = __byte_perm(__float_as_uint(x), __float_as_uint(y), 0x7632);
      }
      q4_st_stream(dst + (int64_t)r * a.row_stride, make_uint4(o[0], o[1], o[2], o[3]));
    }
  }
}

struct Q4CompactArgs {
  const uint8_t* src[2 * kQ4Layers];
  const __half* src_scale[2 * kQ4Layers];
  uint8_t* dst[2 * kQ4Layers];
  __half* dst_scale[2 * kQ4Layers];
  int64_t in_code_stride, in_scale_stride, out_code_stride, out_scale_stride;
  FastDiv by_heads;
  int sets;
  int d;
  int T;
  int kept_cap;
  int gather_meta;  // this launch gathers the step ids and positions
  const int32_t* kept_idx;
  const int32_t* n_kept;
  const int32_t* step_id_in;
  const int32_t* pos_in;
  int32_t* step_id_out;
  int32_t* pos_out;
  int32_t* status;
};
static_assert(sizeof(Q4CompactArgs) <= 32000, "kernel parameter space");

__global__ void __launch_bounds__(kQ4Threads) q4_compact_kernel(const __grid_constant__ Q4CompactArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  const int n = *a.n_kept;
  if (n < 0 || n > a.kept_cap) {
    if (blockIdx.x == 0 && threadIdx.x == 0) record_status(a.status, STEPKV_ENOSPACE);
    return;
  }
  if (a.gather_meta) {
    for (int r = blockIdx.x * kQ4Threads + threadIdx.x; r < n; r += gridDim.x * kQ4Threads) {
      const int t = a.kept_idx[r];
      const bool ok = t >= 0 && t < a.T;
      if (!ok) record_status(a.status, STEPKV_EDATA);
      if (a.step_id_out) a.step_id_out[r] = ok && a.step_id_in ? a.step_id_in[t] : -1;
      if (a.pos_out) a.pos_out[r] = ok ? (a.pos_in ? a.pos_in[t] : t) : -1;
    }
  }
  if (n == 0) return;
  const int row_bytes = a.d >> 1, groups = a.d >> 5;
  const int lpr = row_bytes >> 4, rpi = 32 / lpr;
  const int lane = threadIdx.x & 31, sub = lane / lpr, col = lane - sub * lpr;
  const int per_chunk = rpi * kQ4Unroll, chunks = (n + per_chunk - 1) / per_chunk;
  const int total = a.sets * chunks;
  const int warps = gridDim.x * (kQ4Threads / 32);
  for (int c = blockIdx.x * (kQ4Threads / 32) + (threadIdx.x >> 5); c < total; c += warps) {
    const int set = c / chunks, r0 = (c - set * chunks) * per_chunk;
    int h;
    const int lt = fdivmod(set, a.by_heads, h);
    const uint8_t* src = a.src[lt] + (int64_t)h * a.in_code_stride + col * 16;
    const __half* ss = a.src_scale[lt] + (int64_t)h * a.in_scale_stride;
    uint8_t* dst = a.dst[lt] + (int64_t)h * a.out_code_stride + col * 16;
    __half* ds = a.dst_scale[lt] + (int64_t)h * a.out_scale_stride;
#pragma unroll
    for (int u = 0; u < kQ4Unroll; ++u) {
      const int r = r0 + u * rpi + sub;
      if (sub >= rpi || r >= n) continue;
      const int t = a.kept_idx[r];
      if (t < 0 || t >= a.T) {
        record_status(a.status, STEPKV_EDATA);
        continue;
      }
      q4_st_stream(dst + (int64_t)r * row_bytes, q4_ld_stream(src + (int64_t)t * row_bytes));
      for (int g = col; g < groups; g += lpr) ds[(int64_t)r * groups + g] = ss[(int64_t)t * groups + g];
    }
  }
}

// Enough CTAs for the chunks, at most 8 a SM.
static int q4_grid(int n_sm, int64_t sets, int64_t n, int rows_per_chunk) {
  const int64_t chunks = sets * ((std::max<int64_t>(n, 1) + rows_per_chunk - 1) / rows_per_chunk);
  return (int)std::max<int64_t>(1, std::min<int64_t>((int64_t)n_sm * 8, (chunks + kQ4Threads / 32 - 1) / (kQ4Threads / 32)));
}

static stepkv_status_t q4_done(cudaError_t e) {
  if (e == cudaSuccess) return STEPKV_OK;
  set_last_cuda_error(e);
  return STEPKV_ECUDA;
}

// Write and read differ in which side the bf16 rows are on.
static stepkv_status_t q4_rows_run(bool write, const stepkv_q4_cache_t& c, const void* const* K, const void* const* V,
                                   int64_t head_stride, int64_t row_stride, int T, const Q4Rows& rows, int32_t* status,
                                   cudaStream_t stream) {
  int n_sm = 0;
  cudaError_t e = device_sm_count(&n_sm);
  const int tensors = (K != nullptr) + (V != nullptr);
  for (int l0 = 0; e == cudaSuccess && l0 < c.n_layers; l0 += kQ4Layers) {
    const int nl = std::min(kQ4Layers, c.n_layers - l0);
    Q4Args a;
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
    a.by_tensors = make_fastdiv(tensors);
    a.sets = lt * c.Hkv;
    a.layer0 = l0;
    a.d = c.d;
    a.T = T;
    a.rows = c.rows;
    a.r = rows;
    a.status = status;
    const int grid = q4_grid(n_sm, a.sets, rows.n, 32 / (c.d >> 3) * kQ4Unroll);
    e = launch_kernel(write ? q4_write_kernel : q4_read_kernel, dim3(grid), dim3(kQ4Threads), 0, stream, a, true);
  }
  return q4_done(e);
}

stepkv_status_t q4_write_run(const stepkv_q4_cache_t& c, const void* const* K, const void* const* V, int64_t head_stride,
                             int64_t row_stride, int T, const Q4Rows& rows, int32_t* status, cudaStream_t stream) {
  return q4_rows_run(true, c, K, V, head_stride, row_stride, T, rows, status, stream);
}

stepkv_status_t q4_read_run(const stepkv_q4_cache_t& c, const Q4Rows& rows, void* const* K, void* const* V,
                            int64_t head_stride, int64_t row_stride, int32_t* status, cudaStream_t stream) {
  return q4_rows_run(false, c, K, V, head_stride, row_stride, c.rows, rows, status, stream);
}

stepkv_status_t q4_compact_run(const stepkv_q4_cache_t& in, int T, const int32_t* kept_idx, const int32_t* n_kept,
                               int kept_cap, const stepkv_q4_cache_t& out, const int32_t* step_id_in, const int32_t* pos_in,
                               int32_t* step_id_out, int32_t* pos_out, int32_t* status, cudaStream_t stream) {
  int n_sm = 0;
  cudaError_t e = device_sm_count(&n_sm);
  for (int l0 = 0; e == cudaSuccess && l0 < in.n_layers; l0 += kQ4Layers) {
    const int nl = std::min(kQ4Layers, in.n_layers - l0);
    Q4CompactArgs a;
    memset(&a, 0, sizeof(a));
    int lt = 0;
    for (int l = l0; l < l0 + nl; ++l) {
      for (int t = 0; t < (in.V ? 2 : 1); ++t) {
        a.src[lt] = static_cast<const uint8_t*>(t ? in.V[l] : in.K[l]);
        a.src_scale[lt] = static_cast<const __half*>(t ? in.V_scale[l] : in.K_scale[l]);
        a.dst[lt] = static_cast<uint8_t*>(t ? out.V[l] : out.K[l]);
        a.dst_scale[lt] = static_cast<__half*>(t ? out.V_scale[l] : out.K_scale[l]);
        ++lt;
      }
    }
    a.in_code_stride = in.code_head_stride;
    a.in_scale_stride = in.scale_head_stride;
    a.out_code_stride = out.code_head_stride;
    a.out_scale_stride = out.scale_head_stride;
    a.by_heads = make_fastdiv(in.Hkv);
    a.sets = lt * in.Hkv;
    a.d = in.d;
    a.T = T;
    a.kept_cap = kept_cap;
    a.gather_meta = l0 == 0;
    a.kept_idx = kept_idx;
    a.n_kept = n_kept;
    a.step_id_in = step_id_in;
    a.pos_in = pos_in;
    a.step_id_out = step_id_out;
    a.pos_out = pos_out;
    a.status = status;
    const int grid = q4_grid(n_sm, a.sets, kept_cap, 32 / (in.d >> 5) * kQ4Unroll);
    e = launch_kernel(q4_compact_kernel, dim3(grid), dim3(kQ4Threads), 0, stream, a, true);
  }
  return q4_done(e);
}

}  // namespace stepkv
