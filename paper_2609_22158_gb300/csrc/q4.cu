// A cache held in 4 bits: quantising rows as they are written, reading them back, and moving retained rows
// (Eq. 1's C_hat with 4.5 bits a channel).
//
// A row is cut into groups of 32 channels; a group has one fp16 scale s of 5 significant bits and 32 codes n in 0..15, a
// code stands for s (n - 8):
//   x* = M if M >= -m else m,   s = fp16(r5(-x* / 8)),   n = 8 + clamp(rint(x / s), -8, 7)
// Five bits of scale times three of code fit bf16's eight, so reading back is exact, and so is quantising what was read
// back.  Everything is row-local, so a compaction moves codes and scales as they are.
//
// (Launched dependently: what a kernel before may have written is read after the wait, and not by the read-only path.)
// All three kernels stream: a warp takes chunks of a few rows of one row set (layer, tensor, head), loads everything a
// chunk needs before it uses any of it, and steps to its next chunk without a division.
#include <cuda_fp16.h>

#include <algorithm>

#include "common.cuh"
#include "fastdiv.h"
#include "internal.h"

namespace stepkv {

constexpr int kQ4Threads = 256;
// CTAs an SM holds of the write and read kernels, all of them at once: more waves, or more of them resident with less in
// flight each, were slower (write 216 us with four of three row groups; five of two 223, eight of one 234, two waves 256).
constexpr int kQ4CtasPerSm = 4;

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

// The larger, and the smaller, halves of two bf16 pairs, NaN where either is one.
__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t min2_nan(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// The scale of a group from its element of the largest magnitude.
__device__ __forceinline__ __half q4_scale(float x) {
  if (!(fabsf(x) < INFINITY)) return __ushort_as_half(0x7FFF);
  uint32_t b = __float_as_uint(x * -0.125f);
  b = (b + 0x3FFFFu + ((b >> 19) & 1u)) & ~0x7FFFFu;  // 4 of the 23 explicit bits, ties to even
  return __float2half_rn(fminf(fmaxf(__uint_as_float(b), -896.f), 896.f));
}

// The codes of 8 channels (four bf16 pairs) as one word, channel i in bits 4i .. 4i + 3; inv: 1 / s (0 where s is 0).
// rint(x / s) with the exact quotient's ties: x has 8 bits and s 5, so a quotient near a tie k + 1/2 (k < 8) is the tie or
// at least 2^-9 from it (1/2 - 255 2^-5 / 16), and x inv is off by 2^-19 at most.  Added to 6144 it is rounded to multiples
// of 2^-11, a tie to itself and nothing else to a tie; the next sum rounds that to an integer, ties to even, which lies in
// the low bits.
// LOW: quotients below -8 can occur (a saturated scale, or one on fp16's last steps).
template <bool LOW>
__device__ __forceinline__ uint32_t q4_codes(const uint32_t (&v)[4], float inv) {
  constexpr float kMagic = 12582912.f;  // 1.5 2^23: the last place is 1
  const uint64_t inv2 = f2_pack(inv, inv), c0 = f2_pack(6144.f, 6144.f), c1 = f2_pack(kMagic + 8.f - 6144.f, kMagic + 8.f - 6144.f);
  float u[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint64_t x = f2_pack(__uint_as_float(v[i] << 16), __uint_as_float(v[i] & 0xFFFF0000u));
    f2_unpack(f2_add(f2_fma(x, inv2, c0), c1), u[2 * i], u[2 * i + 1]);
  }
  uint32_t w = 0;
#pragma unroll
  for (int i = 7; i >= 0; --i)  // 16 w + bits of u: what the constant's bits add up to is taken off at the end
    w = w * 16u + __float_as_uint(fminf(LOW ? fmaxf(u[i], kMagic) : u[i], kMagic + 15.f));
  return w - (0x4B400000u * 0x11111111u);
}

// The chunks of a warp: chunk `pos` of row set `set`, every `step`-th of the list of all sets' chunks.
struct Q4Chunks {
  int chunks, sets;         // of a set; sets in all
  int set, pos;
  int d_set, d_pos;
  __device__ __forceinline__ Q4Chunks(int n, int per_chunk, int n_sets) : chunks((n + per_chunk - 1) / per_chunk), sets(n_sets) {
    const int step = gridDim.x * (kQ4Threads / 32), first = blockIdx.x * (kQ4Threads / 32) + (threadIdx.x >> 5);
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

// Where a row set lies: (layer, tensor) entry, layer and head.
struct Q4Set {
  int lt, layer, h;
};
__device__ __forceinline__ Q4Set q4_set(const Q4Args& a, int set) {
  Q4Set s;
  s.lt = fdivmod(set, a.by_heads, s.h);
  s.layer = fdiv(s.lt, a.by_tensors);
  return s;
}

// A lane takes 16 channels of a row, vectors (8 channels) v and v + 2 of a group with v = lane & 1, so that a pair of lanes has
// a group and reads 32 consecutive bytes at a time.  32 layers x 8 heads x 8272 rows: 216 us = 6.4 TB/s (by an index list of
// 8272 in 8911 rows 236), bound by the copies; a division per channel took 655, lanes of 8 channels 272.
constexpr int kQ4WriteUnroll = 3;

template <bool IDX>
__global__ void __launch_bounds__(kQ4Threads, kQ4CtasPerSm) q4_write_kernel(const __grid_constant__ Q4Args a) {
  pdl_wait();
  pdl_launch_dependents();
  const int n = q4_count(a.r, a.status);
  if (n <= 0) return;
  const int lpr = a.d >> 4, rpi = 32 / lpr;  // lanes a row, rows an instruction
  const int lane = threadIdx.x & 31, sub = lane / lpr, col = lane - sub * lpr;
  const int vec = (col >> 1) * 4 + (col & 1);
  const int per_chunk = rpi * kQ4WriteUnroll;
  for (Q4Chunks c(n, per_chunk, a.sets); c.any(); c.next()) {
    const Q4Set s = q4_set(a, c.set);
    const int row0 = a.r.row0_dev ? a.r.row0_dev[(a.layer0 + s.layer) * a.r.row0_stride] : a.r.row0;
    if (row0 < 0 || (int64_t)row0 + n > a.rows) {
      if (lane == 0) record_status(a.status, STEPKV_ENOSPACE);
      continue;
    }
    const uint16_t* src = static_cast<const uint16_t*>(a.src[s.lt]) + (int64_t)s.h * a.head_stride + vec * 8;
    const int r0 = c.pos * per_chunk + sub;
    uint4 v[kQ4WriteUnroll][2];
    bool ok[kQ4WriteUnroll];
    int t[kQ4WriteUnroll];
#pragma unroll
    for (int u = 0; u < kQ4WriteUnroll; ++u) {
      ok[u] = sub < rpi && r0 + u * rpi < n;
      t[u] = r0 + u * rpi;
      if (IDX && ok[u]) {
        t[u] = __ldcg(a.r.idx + t[u]);
        if (t[u] < 0 || t[u] >= a.T) {
          record_status(a.status, STEPKV_EDATA);
          ok[u] = false;
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kQ4WriteUnroll; ++u) {
      v[u][0] = v[u][1] = make_uint4(0, 0, 0, 0);
      if (ok[u]) {
        const uint16_t* p = src + t[u] * a.row_stride;
        v[u][0] = q4_ld_stream(p);
        v[u][1] = q4_ld_stream(p + 16);
      }
    }
    const int64_t row = (int64_t)row0 + r0;
    uint8_t* codes = static_cast<uint8_t*>(a.dst[s.lt]) + (int64_t)s.h * a.code_head_stride + row * (a.d >> 1) + vec * 4;
    __half* scales = static_cast<__half*>(a.scale[s.lt]) + (int64_t)s.h * a.scale_head_stride + row * (a.d >> 5) + (col >> 1);
#pragma unroll
    for (int u = 0; u < kQ4WriteUnroll; ++u) {
      const uint32_t x[2][4] = {{v[u][0].x, v[u][0].y, v[u][0].z, v[u][0].w}, {v[u][1].x, v[u][1].y, v[u][1].z, v[u][1].w}};
      // (maximum, -minimum) of the group as a bf16 pair
      uint32_t hi = x[0][0], lo = x[0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) {
        hi = max2_nan(hi, x[i >> 2][i & 3]);
        lo = min2_nan(lo, x[i >> 2][i & 3]);
      }
      lo ^= 0x80008000u;
      uint32_t both = max2_nan(__byte_perm(hi, lo, 0x5410), __byte_perm(hi, lo, 0x7632));
      both = max2_nan(both, __shfl_xor_sync(0xffffffffu, both, 1));
      const float top = __uint_as_float(both << 16), bottom = __uint_as_float(both & 0xFFFF0000u);
      const float most = top >= bottom ? top : -bottom;
      const __half sc = q4_scale(most);
      const float step = __half2float(sc);
      const float inv = step == 0.f ? 0.f : rcp_approx(step);
      uint32_t w[2];
      if (__all_sync(0xffffffffu, !ok[u] || (fabsf(most) >= 7.62939453125e-6f && fabsf(most) <= 7168.f))) {  // 8 2^-20, 8 896
        w[0] = q4_codes<false>(x[0], inv);
        w[1] = q4_codes<false>(x[1], inv);
      } else {
#pragma unroll
        for (int k = 0; k < 2; ++k) w[k] = step == step ? q4_codes<true>(x[k], inv) : 0x88888888u;
      }
      if (ok[u]) {
        uint32_t* dst = reinterpret_cast<uint32_t*>(codes + u * rpi * (a.d >> 1));
        dst[0] = w[0];
        dst[2] = w[1];
        if ((col & 1) == 0) scales[u * rpi * (a.d >> 5)] = sc;
      }
    }
  }
}

// A lane takes a word of codes (8 channels).  The codes of a pair of channels become bf16 by a mask, s (n - 8) by one sum and
// one product, both exact.  32 layers x 8 heads x 8272 rows: 219 us = 6.3 TB/s; eight row groups in flight 223-265, two 292.
constexpr int kQ4ReadUnroll = 4;

__device__ __forceinline__ uint32_t q4_bf16_pair(uint32_t x, uint32_t s) {
  uint32_t y, z;
  asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(y) : "r"((x & 0x000F000Fu) | 0x43004300u), "r"(0xC308C308u));  // (128 + n) - 136
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(z) : "r"(y), "r"(s));
  return z;
}

template <bool IDX>
__global__ void __launch_bounds__(kQ4Threads, kQ4CtasPerSm) q4_read_kernel(const __grid_constant__ Q4Args a) {
  pdl_wait();
  pdl_launch_dependents();
  const int n = q4_count(a.r, a.status);
  if (n <= 0) return;
  const int lpr = a.d >> 3, rpi = 32 / lpr;
  const int lane = threadIdx.x & 31, sub = lane / lpr, col = lane - sub * lpr;
  const int per_chunk = rpi * kQ4ReadUnroll;
  for (Q4Chunks c(n, per_chunk, a.sets); c.any(); c.next()) {
    const Q4Set s = q4_set(a, c.set);
    int row0 = 0;
    if (!IDX) {
      row0 = a.r.row0_dev ? a.r.row0_dev[(a.layer0 + s.layer) * a.r.row0_stride] : a.r.row0;
      if (row0 < 0 || (int64_t)row0 + n > a.rows) {
        if (lane == 0) record_status(a.status, STEPKV_EDATA);
        continue;
      }
    }
    const int r0 = c.pos * per_chunk + sub;
    const int64_t row = IDX ? 0 : (int64_t)row0 + r0;
    const uint8_t* codes = static_cast<const uint8_t*>(a.src[s.lt]) + (int64_t)s.h * a.code_head_stride + row * (a.d >> 1) + col * 4;
    const __half* scales = static_cast<const __half*>(a.scale[s.lt]) + (int64_t)s.h * a.scale_head_stride + row * (a.d >> 5) + (col >> 2);
    uint16_t* dst = static_cast<uint16_t*>(a.dst[s.lt]) + (int64_t)s.h * a.head_stride + r0 * a.row_stride + col * 8;
    uint32_t w[kQ4ReadUnroll];
    __half sc[kQ4ReadUnroll];
    bool ok[kQ4ReadUnroll];
    int t[kQ4ReadUnroll];
#pragma unroll
    for (int u = 0; u < kQ4ReadUnroll; ++u) {
      ok[u] = sub < rpi && r0 + u * rpi < n;
      t[u] = u * rpi;
      if (IDX && ok[u]) {
        t[u] = __ldcg(a.r.idx + r0 + u * rpi);
        if (t[u] < 0 || t[u] >= a.rows) {
          record_status(a.status, STEPKV_EDATA);
          ok[u] = false;
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kQ4ReadUnroll; ++u) {
      w[u] = 0;
      sc[u] = __ushort_as_half(0);
      if (ok[u]) {
        w[u] = __ldcg(reinterpret_cast<const uint32_t*>(codes + (int64_t)t[u] * (a.d >> 1)));
        sc[u] = __ldcg(scales + (int64_t)t[u] * (a.d >> 5));
      }
    }
    const int64_t step = rpi * a.row_stride;
#pragma unroll
    for (int u = 0; u < kQ4ReadUnroll; ++u) {
      const uint32_t f = __float_as_uint(__half2float(sc[u])), s2 = __byte_perm(f, f, 0x3232);  // exact in bf16
      uint32_t x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = q4_bf16_pair(w[u] >> (4 * i), s2);  // channels i and i + 4
      if (ok[u])
        q4_st_stream(dst, make_uint4(__byte_perm(x[0], x[1], 0x5410), __byte_perm(x[2], x[3], 0x5410),
                                     __byte_perm(x[0], x[1], 0x7632), __byte_perm(x[2], x[3], 0x7632)));
      dst += step;
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

// A lane takes 16 bytes of a row's codes; its first lanes also the scales, in words as wide as a row of them allows (T).
// 8272 of 8911 rows of 32 layers x 8 heads: 104 us = 5.9 TB/s (two row groups in flight 112, eight 116).
constexpr int kQ4CompactUnroll = 4;
constexpr int kQ4CompactCtasPerSm = 8;

template <typename T>
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
  const int row_bytes = a.d >> 1, words = (a.d >> 5) * 2 / (int)sizeof(T);  // words: of a row's scales
  const int lpr = row_bytes >> 4, rpi = 32 / lpr;
  const int lane = threadIdx.x & 31, sub = lane / lpr, col = lane - sub * lpr;
  const int per_chunk = rpi * kQ4CompactUnroll;
  for (Q4Chunks c(n, per_chunk, a.sets); c.any(); c.next()) {
    int h;
    const int lt = fdivmod(c.set, a.by_heads, h);
    const uint8_t* src = a.src[lt] + (int64_t)h * a.in_code_stride + col * 16;
    const T* ss = reinterpret_cast<const T*>(a.src_scale[lt] + (int64_t)h * a.in_scale_stride) + col;
    uint8_t* dst = a.dst[lt] + (int64_t)h * a.out_code_stride + col * 16;
    T* ds = reinterpret_cast<T*>(a.dst_scale[lt] + (int64_t)h * a.out_scale_stride) + col;
    const int r0 = c.pos * per_chunk + sub;
    int t[kQ4CompactUnroll];
    uint4 v[kQ4CompactUnroll];
    T sc[kQ4CompactUnroll];
#pragma unroll
    for (int u = 0; u < kQ4CompactUnroll; ++u) {
      const int r = r0 + u * rpi;
      t[u] = -1;
      if (sub < rpi && r < n) {
        t[u] = __ldcg(a.kept_idx + r);
        if (t[u] < 0 || t[u] >= a.T) {
          record_status(a.status, STEPKV_EDATA);
          t[u] = -1;
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kQ4CompactUnroll; ++u) {
      sc[u] = T();
      if (t[u] >= 0) {
        v[u] = q4_ld_stream(src + (int64_t)t[u] * row_bytes);
        if (col < words) sc[u] = __ldcg(ss + (int64_t)t[u] * words);
      }
    }
#pragma unroll
    for (int u = 0; u < kQ4CompactUnroll; ++u) {
      if (t[u] < 0) continue;
      const int64_t r = r0 + u * rpi;
      q4_st_stream(dst + r * row_bytes, v[u]);
      if (col < words) ds[r * words] = sc[u];
    }
  }
}

// Enough CTAs for the chunks, at most as many as `ctas`.
static int q4_grid(int64_t ctas, int64_t sets, int64_t n, int rows_per_chunk) {
  const int64_t chunks = sets * ((std::max<int64_t>(n, 1) + rows_per_chunk - 1) / rows_per_chunk);
  return (int)std::max<int64_t>(1, std::min<int64_t>(ctas, (chunks + kQ4Threads / 32 - 1) / (kQ4Threads / 32)));
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
    const int grid = q4_grid(n_sm * kQ4CtasPerSm, a.sets, rows.n, write ? 32 / (c.d >> 4) * kQ4WriteUnroll : 32 / (c.d >> 3) * kQ4ReadUnroll);
    auto kern = write ? (rows.idx ? q4_write_kernel<true> : q4_write_kernel<false>)
                      : (rows.idx ? q4_read_kernel<true> : q4_read_kernel<false>);
    e = launch_kernel(kern, dim3(grid), dim3(kQ4Threads), 0, stream, a, true);
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
    const int grid = q4_grid(n_sm * kQ4CompactCtasPerSm, a.sets, kept_cap, 32 / (in.d >> 5) * kQ4CompactUnroll);
    const int groups = in.d >> 5;
    auto kern = groups % 4 == 0 ? q4_compact_kernel<unsigned long long>
                                : groups % 2 == 0 ? q4_compact_kernel<unsigned int> : q4_compact_kernel<unsigned short>;
    e = launch_kernel(kern, dim3(grid), dim3(kQ4Threads), 0, stream, a, true);
  }
  return q4_done(e);
}

}  // namespace stepkv
