// Decode attention over a cache held in 8 bits (format in q8.cuh):
//   out[g][:] = sum_{j < n} softmax_j( q[g] . K[g/G][j] / sqrt(d) ) V[g/G][j][:]
// with K and V the values the codes stand for, one count n per cache or one for all, and, where masses are given,
//   mass[h][j] += (1/G) sum_g softmax_j( q[g] . K[h][j] / sqrt(d) ).
//
// One CTA per (cache, KV head); its warps take the keys in turn, a lane D / 32 channels of each, with a running maximum and
// sum per query head; the warps' states are joined in shared memory.  Logits are kept for the masses.
#include <math.h>

#include <algorithm>

#include "common.cuh"
#include "internal.h"
#include "q8.cuh"

namespace stepkv {

constexpr int kQ8DecWarps = 8;
constexpr int kQ8MaxG = 8;

struct Q8DecodeArgs {
  const uint16_t* q[kQ8Layers];
  const uint8_t* K[kQ8Layers];
  const uint8_t* V[kQ8Layers];
  const float* K_scale[kQ8Layers];
  const float* V_scale[kQ8Layers];
  float* out[kQ8Layers];
  float* mass[kQ8Layers];
  int64_t code_head_stride, scale_head_stride, mass_stride;
  int layer0, Hkv, G;
  const int32_t* n_dev;
  int n_stride, n_host, n_cap;
  float c;        // log2(e) / sqrt(d)
  float* logits;  // [pair][n_cap][G], or NULL
  int32_t* status;
};
static_assert(sizeof(Q8DecodeArgs) <= 32000, "kernel parameter space");

template <int D>
__global__ void __launch_bounds__(kQ8DecWarps * 32) q8_decode_kernel(const __grid_constant__ Q8DecodeArgs a) {
  constexpr int E = D / 32;
  __shared__ float s_ml[kQ8DecWarps][kQ8MaxG][2];
  __shared__ float s_v[kQ8DecWarps][kQ8MaxG][D];
  __shared__ float s_joined[kQ8MaxG][2];
  pdl_wait();
  pdl_launch_dependents();
  const int pair = blockIdx.x, layer = pair / a.Hkv, h = pair - layer * a.Hkv, G = a.G;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int n = a.n_host;
  if (a.n_dev) {
    n = a.n_dev[(a.layer0 + layer) * a.n_stride];
    if (threadIdx.x == 0 && (n < 0 || n > a.n_cap)) record_status(a.status, n < 0 ? STEPKV_EDATA : STEPKV_ENOSPACE);
    n = max(0, min(n, a.n_cap));
  }
  float q[kQ8MaxG][E], m[kQ8MaxG], l[kQ8MaxG], acc[kQ8MaxG][E];
#pragma unroll
  for (int g = 0; g < kQ8MaxG; ++g) {
    m[g] = -INFINITY;
    l[g] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      acc[g][e] = 0.f;
      q[g][e] = g < G ? __uint_as_float((uint32_t)a.q[layer][(h * G + g) * D + lane * E + e] << 16) : 0.f;
    }
  }
  const uint8_t* K = a.K[layer] + (int64_t)h * a.code_head_stride + lane * E;
  const uint8_t* V = a.V[layer] + (int64_t)h * a.code_head_stride + lane * E;
  const float* ks = a.K_scale[layer] + (int64_t)h * a.scale_head_stride;
  const float* vs = a.V_scale[layer] + (int64_t)h * a.scale_head_stride;
  float* logits = a.logits ? a.logits + (int64_t)pair * a.n_cap * G : nullptr;
  for (int j = warp; j < n; j += kQ8DecWarps) {
    float k[E], v[E];
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      const float2 x = q8_float2(__ldcg(reinterpret_cast<const uint16_t*>(K + (int64_t)j * D + e)));
      const float2 y = q8_float2(__ldcg(reinterpret_cast<const uint16_t*>(V + (int64_t)j * D + e)));
      k[e] = x.x * ks[j / kQ8Block];
      k[e + 1] = x.y * ks[j / kQ8Block];
      v[e] = y.x * vs[j / kQ8Block];
      v[e + 1] = y.y * vs[j / kQ8Block];
    }
#pragma unroll
    for (int g = 0; g < kQ8MaxG; ++g) {
      if (g >= G) break;
      float x = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) x = fmaf(q[g][e], k[e], x);
#pragma unroll
      for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
      x *= a.c;
      if (logits && lane == 0) logits[(int64_t)j * G + g] = x;
      const float mn = fmaxf(m[g], x);
      const float was = m[g] == mn ? 1.f : exp2f(m[g] - mn), p = mn == -INFINITY && x == x ? 0.f : exp2f(x - mn);
      l[g] = l[g] * was + p;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[g][e] = fmaf(acc[g][e], was, p * v[e]);
      m[g] = mn;
    }
  }
#pragma unroll
  for (int g = 0; g < kQ8MaxG; ++g) {
    if (lane == 0) {
      s_ml[warp][g][0] = m[g];
      s_ml[warp][g][1] = l[g];
    }
#pragma unroll
    for (int e = 0; e < E; ++e) s_v[warp][g][lane * E + e] = acc[g][e];
  }
  __syncthreads();
  for (int t = threadIdx.x; t < G * D; t += blockDim.x) {
    const int g = t / D, e = t - g * D;
    float mm = -INFINITY, ll = 0.f, o = 0.f;
    for (int w = 0; w < kQ8DecWarps; ++w) mm = fmaxf(mm, s_ml[w][g][0]);
    for (int w = 0; w < kQ8DecWarps; ++w) {
      const float f = s_ml[w][g][0] == -INFINITY && s_ml[w][g][1] == 0.f ? 0.f : exp2f(s_ml[w][g][0] - mm);
      ll += s_ml[w][g][1] * f;
      o += s_v[w][g][e] * f;
    }
    a.out[layer][(size_t)(h * G + g) * D + e] = n > 0 ? o / ll : 0.f;
    if (e == 0) {
      s_joined[g][0] = mm;
      s_joined[g][1] = 1.f / ll;
    }
  }
  if (!logits) return;
  __syncthreads();
  float* mass = a.mass[layer] + (int64_t)h * a.mass_stride;
  for (int j = threadIdx.x; j < n; j += blockDim.x) {
    float sum = 0.f;
    for (int g = 0; g < G; ++g) sum += exp2f(logits[(int64_t)j * G + g] - s_joined[g][0]) * s_joined[g][1];
    mass[j] += sum / (float)G;
  }
}

size_t q8_decode_ws_bytes(int n_layers, int Hkv, int Hq, int d, int n_cap, bool mass) {
  return std::max<size_t>(256, mass ? (size_t)n_layers * Hq * n_cap * sizeof(float) : 0);
}

stepkv_status_t q8_decode_run(const stepkv_q8_cache_t& c, const void* const* q, int Hq, const int32_t* n_dev, int n_stride,
                              int n_host, int n_cap, float* const* out, float* const* mass, int64_t mass_stride, void* ws,
                              int32_t* status, cudaStream_t stream) {
  cudaError_t e = cudaSuccess;
  for (int l0 = 0; e == cudaSuccess && l0 < c.n_layers; l0 += kQ8Layers) {
    const int nl = std::min(kQ8Layers, c.n_layers - l0);
    Q8DecodeArgs a;
    memset(&a, 0, sizeof(a));
    for (int l = 0; l < nl; ++l) {
      a.q[l] = static_cast<const uint16_t*>(q[l0 + l]);
      a.K[l] = static_cast<const uint8_t*>(c.K[l0 + l]);
      a.V[l] = static_cast<const uint8_t*>(c.V[l0 + l]);
      a.K_scale[l] = c.K_scale[l0 + l];
      a.V_scale[l] = c.V_scale[l0 + l];
      a.out[l] = out[l0 + l];
      a.mass[l] = mass ? mass[l0 + l] : nullptr;
    }
    a.code_head_stride = c.code_head_stride;
    a.scale_head_stride = c.scale_head_stride;
    a.mass_stride = mass_stride;
    a.layer0 = l0;
    a.Hkv = c.Hkv;
    a.G = Hq / c.Hkv;
    a.n_dev = n_dev;
    a.n_stride = n_stride;
    a.n_host = n_host;
    a.n_cap = n_cap;
    a.c = (float)(1.4426950408889634 / sqrt((double)c.d));
    a.logits = mass ? static_cast<float*>(ws) : nullptr;
    a.status = status;
    e = launch_kernel(c.d == 128 ? q8_decode_kernel<128> : q8_decode_kernel<64>, dim3(nl * c.Hkv), dim3(kQ8DecWarps * 32), 0,
                      stream, a, true);
  }
  if (e == cudaSuccess) return STEPKV_OK;
  set_last_cuda_error(e);
  return STEPKV_ECUDA;
}

}  // namespace stepkv
