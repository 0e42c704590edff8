// Decode attention over a cache held in 4 bits (format in q4.cu):
//   out[g][:] = sum_{j < n} softmax_j( q[g] . K[g/G][j] / sqrt(d) ) V[g/G][j][:]
// with K and V the values the codes stand for, one count n per cache or one for all.
//
// The rows of a (cache, KV head) pair are split over CTAs; a warp takes every eighth row of its CTA's share, a lane d / 32
// channels.  Partial states (maximum, sum, weighted values) meet in the CTA, and a second kernel joins the CTAs' in order.
#include <cuda_fp16.h>
#include <math.h>

#include <algorithm>

#include "common.cuh"
#include "internal.h"

namespace stepkv {

constexpr int kQ4DecWarps = 8;
constexpr int kQ4DecThreads = kQ4DecWarps * 32;
constexpr int kQ4SplitRows = 512;   // a pair has at most one CTA per 512 rows of capacity
constexpr int kQ4MaxG = 8;

struct Q4DecodeArgs {
  const uint16_t* q[kQ4Layers];
  const uint8_t* K[kQ4Layers];
  const uint8_t* V[kQ4Layers];
  const __half* K_scale[kQ4Layers];
  const __half* V_scale[kQ4Layers];
  float* out[kQ4Layers];
  int64_t code_head_stride, scale_head_stride;
  int layer0;
  int Hkv, G;
  int splits;
  const int32_t* n_dev;
  int n_stride;
  int n_host;
  int n_cap;
  float c;       // log2(e) / sqrt(d)
  float* part;   // [pair][split][G][d + 4]: m, l, -, -, values
  int32_t* status;
};
static_assert(sizeof(Q4DecodeArgs) <= 32000, "kernel parameter space");

__device__ __forceinline__ int q4_keys(const Q4DecodeArgs& a, int layer, bool tell) {
  if (!a.n_dev) return a.n_host;
  const int n = a.n_dev[(a.layer0 + layer) * a.n_stride];
  if (tell && n > a.n_cap) record_status(a.status, STEPKV_ENOSPACE);
  if (tell && n < 0) record_status(a.status, STEPKV_EDATA);
  return max(0, min(n, a.n_cap));
}

// Channels 4 lane .. (d = 128) or 2 lane .. (d = 64) of a row.
template <int PER>
__device__ __forceinline__ void q4_row(const uint8_t* codes, const __half* scales, int64_t row, int lane, float (&x)[PER]) {
  constexpr int D = PER * 32;
  const uint32_t w = PER == 4 ? *reinterpret_cast<const uint16_t*>(codes + row * (D / 2) + lane * 2) : codes[row * (D / 2) + lane];
  const float s = __half2float(scales[row * (D / 32) + lane * PER / 32]);
#pragma unroll
  for (int e = 0; e < PER; ++e) x[e] = (float)((int)((w >> (4 * e)) & 15u) - 8) * s;
}

template <int D>
__global__ void __launch_bounds__(kQ4DecThreads) q4_decode_kernel(const __grid_constant__ Q4DecodeArgs a) {
  constexpr int PER = D / 32;
  __shared__ float s_m[kQ4DecWarps][kQ4MaxG], s_l[kQ4DecWarps][kQ4MaxG];
  __shared__ float s_v[kQ4DecWarps][D];
  pdl_wait();
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int pair = blockIdx.x / a.splits, split = blockIdx.x - pair * a.splits;
  const int layer = pair / a.Hkv, h = pair - layer * a.Hkv;
  const int n = q4_keys(a, layer, h == 0 && split == 0 && threadIdx.x == 0);
  const int share = (n + a.splits - 1) / a.splits;
  const int lo = min(n, split * share), hi = min(n, lo + share);
  const uint8_t* K = a.K[layer] + h * a.code_head_stride;
  const uint8_t* V = a.V[layer] + h * a.code_head_stride;
  const __half* Ks = a.K_scale[layer] + h * a.scale_head_stride;
  const __half* Vs = a.V_scale[layer] + h * a.scale_head_stride;
  float q[kQ4MaxG][PER], m[kQ4MaxG], l[kQ4MaxG], acc[kQ4MaxG][PER];
#pragma unroll
  for (int g = 0; g < kQ4MaxG; ++g) {
    m[g] = -INFINITY;
    l[g] = 0.f;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      acc[g][e] = 0.f;
      q[g][e] = g < a.G ? __uint_as_float((uint32_t)a.q[layer][(size_t)(h * a.G + g) * D + lane * PER + e] << 16) * a.c : 0.f;
    }
  }
  for (int j = lo + warp; j < hi; j += kQ4DecWarps) {
    float k[PER], v[PER];
    q4_row<PER>(K, Ks, j, lane, k);
    q4_row<PER>(V, Vs, j, lane, v);
#pragma unroll
    for (int g = 0; g < kQ4MaxG; ++g) {
      if (g >= a.G) break;
      float x = 0.f;
#pragma unroll
      for (int e = 0; e < PER; ++e) x += q[g][e] * k[e];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
      const float mn = fmaxf(m[g], x);  // a NaN logit leaves the maximum, and makes the sum NaN
      const float sc = exp2f(m[g] - mn), p = exp2f(x - mn);
      l[g] = l[g] * sc + p;
#pragma unroll
      for (int e = 0; e < PER; ++e) acc[g][e] = acc[g][e] * sc + p * v[e];
      m[g] = mn;
    }
  }
  if (lane == 0)
#pragma unroll
    for (int g = 0; g < kQ4MaxG; ++g) {
      s_m[warp][g] = m[g];
      s_l[warp][g] = l[g];
    }
  float* part = a.part + (size_t)blockIdx.x * a.G * (D + 4);
#pragma unroll
  for (int g = 0; g < kQ4MaxG; ++g) {
    if (g >= a.G) break;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < PER; ++e) s_v[warp][lane * PER + e] = acc[g][e];
    __syncthreads();
    float top = -INFINITY;
    for (int w = 0; w < kQ4DecWarps; ++w) top = fmaxf(top, s_m[w][g]);
    if ((int)threadIdx.x < D) {
      float ll = 0.f, v = 0.f;
      for (int w = 0; w < kQ4DecWarps; ++w) {
        const float b = s_l[w][g] == 0.f ? 0.f : exp2f(s_m[w][g] - top);
        if (s_l[w][g] == 0.f) continue;
        ll += s_l[w][g] * b;
        v += s_v[w][threadIdx.x] * b;
      }
      part[g * (D + 4) + 4 + threadIdx.x] = v;
      if (threadIdx.x == 0) {
        part[g * (D + 4)] = top;
        part[g * (D + 4) + 1] = ll;
      }
    }
  }
}

// One (pair, head) a block, one channel a thread.
template <int D>
__global__ void __launch_bounds__(D) q4_merge_kernel(const __grid_constant__ Q4DecodeArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  const int pair = blockIdx.x / a.G, g = blockIdx.x - pair * a.G;
  const int layer = pair / a.Hkv, h = pair - layer * a.Hkv;
  const float* part = a.part + (size_t)pair * a.splits * a.G * (D + 4) + g * (D + 4);
  const size_t step = (size_t)a.G * (D + 4);
  float top = -INFINITY, l = 0.f, v = 0.f;
  for (int s = 0; s < a.splits; ++s) top = fmaxf(top, part[s * step]);
  for (int s = 0; s < a.splits; ++s) {
    if (part[s * step + 1] == 0.f) continue;
    const float b = exp2f(part[s * step] - top);
    l += part[s * step + 1] * b;
    v += part[s * step + 4 + threadIdx.x] * b;
  }
  a.out[layer][(size_t)(h * a.G + g) * D + threadIdx.x] = l == 0.f ? 0.f : v / l;
}

static int q4_splits(int n_cap) { return std::max(1, std::min(64, (n_cap + kQ4SplitRows - 1) / kQ4SplitRows)); }

size_t q4_decode_ws_bytes(int n_layers, int Hkv, int Hq, int d, int n_cap) {
  (void)Hkv;
  return (size_t)n_layers * Hq * q4_splits(n_cap) * (d + 4) * sizeof(float);
}

template <int D>
static cudaError_t q4_decode_launch(const Q4DecodeArgs& a, int pairs, cudaStream_t stream) {
  cudaError_t e = launch_kernel(q4_decode_kernel<D>, dim3(pairs * a.splits), dim3(kQ4DecThreads), 0, stream, a, true);
  if (e == cudaSuccess) e = launch_kernel(q4_merge_kernel<D>, dim3(pairs * a.G), dim3(D), 0, stream, a, true);
  return e;
}

stepkv_status_t q4_decode_run(const stepkv_q4_cache_t& c, const void* const* q, int Hq, const int32_t* n_dev, int n_stride,
                              int n_host, int n_cap, float* const* out, void* ws, int32_t* status, cudaStream_t stream) {
  cudaError_t e = cudaSuccess;
  for (int l0 = 0; e == cudaSuccess && l0 < c.n_layers; l0 += kQ4Layers) {
    const int nl = std::min(kQ4Layers, c.n_layers - l0);
    Q4DecodeArgs a;
    memset(&a, 0, sizeof(a));
    for (int l = 0; l < nl; ++l) {
      a.q[l] = static_cast<const uint16_t*>(q[l0 + l]);
      a.K[l] = static_cast<const uint8_t*>(c.K[l0 + l]);
      a.V[l] = static_cast<const uint8_t*>(c.V[l0 + l]);
      a.K_scale[l] = static_cast<const __half*>(c.K_scale[l0 + l]);
      a.V_scale[l] = static_cast<const __half*>(c.V_scale[l0 + l]);
      a.out[l] = out[l0 + l];
    }
    a.code_head_stride = c.code_head_stride;
    a.scale_head_stride = c.scale_head_stride;
    a.layer0 = l0;
    a.Hkv = c.Hkv;
    a.G = Hq / c.Hkv;
    a.splits = q4_splits(n_cap);
    a.n_dev = n_dev;
    a.n_stride = n_stride;
    a.n_host = n_host;
    a.n_cap = n_cap;
    a.c = (float)(1.4426950408889634 / sqrt((double)c.d));
    a.part = static_cast<float*>(ws);
    a.status = status;
    e = c.d == 128 ? q4_decode_launch<128>(a, nl * c.Hkv, stream) : q4_decode_launch<64>(a, nl * c.Hkv, stream);
  }
  if (e == cudaSuccess) return STEPKV_OK;
  set_last_cuda_error(e);
  return STEPKV_ECUDA;
}

}  // namespace stepkv
