// Decode attention over a cache held in 8 bits (format in q8.cuh):
//   out[g][:] = sum_{j < n} softmax_j( q[g] . K[g/G][j] / sqrt(d) ) V[g/G][j][:]
// with K and V the values the codes stand for, one count n per cache or one for all, and, where masses are given,
//   mass[h][j] += (1/G) sum_g softmax_j( q[g] . K[h][j] / sqrt(d) ).
//
// A row pair is 2 d bytes, read once.  Both contractions run on the tensor cores (mma.sync, whose operands may come from
// registers: a KV head's G <= 8 query heads are the 8 columns of a tile, rows of the cache or channels its 16 rows), a warp on
// 32 keys at a time, which share one scale for their keys and one for their values:
//   S^T = K Q^T.  A word of four codes is two fp16 pairs by two conversions, exactly: the A operand of a k-step of 16 channels
//     (lane: channels 4c .. 4c + 3 of a key), Q laid out to match.  Q is scaled by a power of two and exact in fp16.  Two k-steps
//     are summed from zero in the tensor core, whose accumulation truncates, the rest in fp32; the block's scale is part of
//     the one factor that a logit is multiplied by.
//   O^T = V^T P^T.  ldmatrix with transposition puts two channels of two keys into a word; a byte permute and two
//     conversions make them the A operand's pairs of keys, for rows of even and of odd channels.  The weights are two fp16
//     terms, 22 bits, and come from the layout of S^T by movmatrix.  A block's sum starts from zero and is added, times the
//     block's scale, in fp32.
// For G <= 4 columns 4-7 repeat the heads of columns 0-3, and P has its first terms in 0-3 and its second in 4-7.
//
// The blocks go to warps as in the 4-bit decode (decode_list.cuh): each warp copies its blocks of 32 rows into a ring of its
// own with cp.async; a group of warps takes a pair (q8_whole) or a range of the list of all pairs' blocks (list_split), joins
// its warps' states in shared memory, and writes the output where it had the whole pair, or else leaves a partial state, which a second
// kernel joins with the others in key order.
//
// 445 instructions a block of 32 keys (G <= 4, d = 128), issued at a third of the rate that the schedulers have: the reads bound it.
// 64 layers x 8 heads x 16417 rows, G = 5: 300 us = 7.2 TB/s; 32 layers x 8272 rows 86 us = 6.3 (the first rows and the join are 6 of
// them); one layer 9.1 us (17 MB; launch, first rows, two rounds of blocks, join). On CUDA cores, a lane's share of the channels
// per key, 5393, 1190 and 796 us.  Eight warps of up to 255 registers on an SM with three stages of 8 KB each (d = 128, G <= 4).
// Clusters of 2 to 16 CTAs a pair, joined through distributed shared memory in one launch: 1 layer x 8 heads x 1024 rows 6.4 -> 6.2
// us, 4096 8.2 -> 8.3, 8272 9.1 -> 10.7, with masses 7.2 -> 8.2: not kept, nor a dry run of the second kernel before its wait (9.2).
//
// Masses need the sums over all keys: the logits go to the workspace (keys and values leave L2 first, so that they stay there: 32
// layers x 8272 rows 115 -> 107 us), and blocks of the second kernel join the (maximum, sum) of a pair's states and add
// exp2(x - m) / l to its keys' masses; short pairs taken whole do that themselves (kQ8FewRounds).
#include <cuda_fp16.h>
#include <math.h>

#include <algorithm>

#include "common.cuh"
#include "decode_list.cuh"
#include "fastdiv.h"
#include "internal.h"
#include "q8.cuh"

namespace stepkv {

constexpr int kQ8DecWarps = kListWarps;
constexpr int kQ8DecThreads = kQ8DecWarps * 32;
constexpr int kQ8DecCtasPerSm = 2;
constexpr int kQ8DecMinSmem = 228 * 1024 / (kQ8DecCtasPerSm + 1);
// Rounds of blocks up to which a pair taken whole has its masses added by its own warps, in the same launch (1 layer x 8 heads x
// 512 rows 8.7 -> 7.2 us, 32 layers 12.0 -> 9.5; at 8 rounds 10.9, by the second kernel's blocks 7.2).
constexpr int kQ8FewRounds = 4;
constexpr float kQ8WeightLog2 = 14.f;  // the largest weight is held as 2^14 (fp16 reaches 65504)
// Blocks that a pair of a ragged batch counts besides its own (list_counts): what its query, its state and the join with the CTA's
// other warps cost.  64 caches x 16 heads of 0 to 4096 rows, d = 64: 85 us without, 60 with 8, 51 with 16, 49 with 32; 32 x 8 heads,
// lengths spread over their logarithm up to 8192 46, 22, 21, 23; one of 8192 among 64 rows 17, 12.6, 12.3, 12.7.
constexpr int kQ8Pad = 16;
static_assert(kListBlock == kQ8Block && kListLayers == kQ8Layers, "a warp step is a block of the cache");

struct Q8DecodeArgs : DecodeList {
  const uint16_t* q[kQ8Layers];
  const uint8_t* K[kQ8Layers];
  const uint8_t* V[kQ8Layers];
  const float* K_scale[kQ8Layers];
  const float* V_scale[kQ8Layers];
  float* out[kQ8Layers];
  float* mass[kQ8Layers];
  int64_t code_head_stride, scale_head_stride, mass_stride;
  int G;
  FastDiv by_G;
  float c;          // log2(e) / sqrt(d)
  float* part;      // [slot][G][d + 4]: m, l, -, -, values
  float* logits;    // [pair][G][n_cap], log2 units, or NULL
  int whole;        // warps of a CTA that take a pair, all of it: one launch (0: the pairs are cut, list_split)
  int mass_here;    // whole pairs: the first kernel adds to the masses
  int join_blocks;  // blocks of the second kernel that join states; those after them add to masses
  FastDiv by_chunks;  // chunks of keys of a pair, a block of the mass pass each
};
static_assert(sizeof(Q8DecodeArgs) <= 32000, "kernel parameter space");

// A ring stage: codes of 32 keys, codes of 32 values, as they lie in memory but for the 16-byte vectors of a row, which are
// permuted (vector ^ mask of the row) so that the eight rows an ldmatrix takes lie in different banks; then the two scales.
template <int D, int GP>
struct Q8Stage {
  static constexpr int kV = kQ8Block * D;
  static constexpr int kScales = 2 * kV;
  static constexpr int kBytes = kScales + 128;  // (stages begin on 128 bytes: the permutation is of address bits)
  static constexpr int kStages = D == 128 ? (GP == 4 ? 3 : 2) : (GP == 4 ? 5 : 4);
  static __device__ __forceinline__ int swizzle(int row) { return D == 128 ? row & 7 : (row >> 1) & 3; }
};

// A copy of 16 bytes that leaves L2 first (masses: so that the logits stay there until they are read again).
__device__ __forceinline__ void q8_cp_hint(uint32_t dst, const void* src, uint64_t policy) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(policy) : "memory");
}
__device__ __forceinline__ uint64_t q8_evict_first() {
  uint64_t policy;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
  return policy;
}

// The two pairs of codes of a word as fp16.
__device__ __forceinline__ void q8_unpack(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.rn.f16x2.e4m3x2 %0, a;\n cvt.rn.f16x2.e4m3x2 %1, b;\n}\n"
      : "=r"(lo), "=r"(hi) : "r"(w));
}

// One warp's state over the keys of a pair.  A lane has columns 2 c4 and 2 c4 + 1 (heads; GP = 4: heads (2 c4) & 3 and the
// next: of P the first terms where c4 < 2, the second terms else) and keys r8, r8 + 8, ...; acc[v] holds channel 16 v + 2 r8 (of
// both columns) and, in its second pair, the next one.
template <int D, int GP>
struct Q8State {
  static constexpr int NV = D / 16;     // 16-channel tiles of a row
  static constexpr int NB = GP == 4 ? 2 : 4;
  float m[2];                           // largest logit so far (log2 units)
  uint64_t nm;                          // -m, 0 before the first key
  uint64_t l;
  uint64_t acc[NV][2];
  uint32_t q[NV][2];                    // B operand of the k-steps
  float unit[2];                        // what Q was divided by (a power of two), NaN for a head that is not all numbers

  __device__ __forceinline__ void clear() {
    m[0] = m[1] = -INFINITY;
    nm = l = 0ull;
#pragma unroll
    for (int t = 0; t < NV; ++t) acc[t][0] = acc[t][1] = 0ull;
  }

  // Q of a pair's heads, [G][D] at src, in fp16: a head's elements are scaled by a power of two (at most 2^126) that brings the
  // largest to [2^10, 2^11), which is exact down to 2^-24 of it.
  __device__ __forceinline__ void load_q(const uint16_t* src, int G, int lane) {
    const int r8 = lane >> 2, c4 = lane & 3, head = GP == 4 ? r8 & 3 : r8;
    uint2 v[NV];
    uint32_t top = 0;
#pragma unroll
    for (int t = 0; t < NV; ++t) {
      v[t] = make_uint2(0, 0);
      if (head < G) v[t] = __ldcg(reinterpret_cast<const uint2*>(src + head * D + t * 16) + c4);
      top = max(top, max(max(v[t].x & 0x7FFFu, (v[t].x >> 16) & 0x7FFFu), max(v[t].y & 0x7FFFu, (v[t].y >> 16) & 0x7FFFu)));
    }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const uint32_t e = top >> 7, up = min(264u - e, 253u);  // exponent fields: of the largest, of the factor 2^(137 - e)
    const float mul = __uint_as_float(up << 23);
    const float back = __uint_as_float(e == 255u ? 0x7FC00000u : (254u - up) << 23);
#pragma unroll
    for (int t = 0; t < NV; ++t) {
      const uint32_t w[2] = {v[t].x, v[t].y};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const __half2 h = __floats2half2_rn(__uint_as_float(w[i] << 16) * mul, __uint_as_float(w[i] & 0xFFFF0000u) * mul);
        q[t][i] = *reinterpret_cast<const uint32_t*>(&h);
      }
    }
    unit[0] = __shfl_sync(0xffffffffu, back, 8 * c4);
    unit[1] = __shfl_sync(0xffffffffu, back, 8 * c4 + 4);
  }

  // The logits (log2 units) of keys r8 + 8 i of the 32 whose codes this lane's ldmatrix address is `codes` in; scale: the keys'
  // times c.
  __device__ __forceinline__ void logits(uint64_t (&s)[4], uint32_t codes, float scale) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int p = 0; p < NV / 2; ++p) {
        uint32_t w[4], a[4];
        ldmatrix_x4(w, (codes + h * 16 * D) ^ (p << 5));
        float d[4];
        q8_unpack(w[0], a[0], a[2]);
        q8_unpack(w[1], a[1], a[3]);
        mma_f16_zero(d, a, q[2 * p][0], q[2 * p][1]);
        q8_unpack(w[2], a[0], a[2]);
        q8_unpack(w[3], a[1], a[3]);
        mma_f16(d, a, q[2 * p + 1][0], q[2 * p + 1][1]);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint64_t d2 = f2_pack(d[2 * k], d[2 * k + 1]);
          s[2 * h + k] = p == 0 ? d2 : f2_add(s[2 * h + k], d2);
        }
      }
    }
    // (a factor past the largest number meets logits past 2^90 only)
    const uint64_t f = f2_pack(min_nan(unit[0] * scale, 3.4e38f), min_nan(unit[1] * scale, 3.4e38f));
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = f2_mul(s[i], f);
  }

  // Keys kb .. kb + 31 (those at or past n do not count) in the ring stage; off: this lane's ldmatrix offset for keys, toff for
  // values; MASS: x: the pair's logits of this lane's first column, G of them.
  template <bool MASS>
  __device__ __forceinline__ void block(uint32_t stage, uint32_t off, uint32_t toff, int kb, int n, float c, int lane, float* x, int n_cap, int G) {
    using St = Q8Stage<D, GP>;
    const int r8 = lane >> 2, c4 = lane & 3;
    uint32_t sc[2];  // scales of the keys, of the values
    lds<8>(sc, stage + St::kScales);
    uint64_t s[4];   // key r8 + 8 i, both columns
    logits(s, stage + off, __uint_as_float(sc[0]) * c);
    if constexpr (MASS) {  // (GP = 4: columns 4-7 are columns 0-3 again: their lanes keep the second half of the keys)
      constexpr int kMine = GP == 4 ? 2 : 4;
      const int col = GP == 4 ? 2 * (c4 & 1) : 2 * c4;
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const bool second = GP == 4 && c4 >= 2;
        const int j = kb + 8 * i + r8 + (second ? 16 : 0);
        float v[2];
        f2_unpack(second ? s[(i + 2) & 3] : s[i], v[0], v[1]);
        if (j < n && col < G) x[j] = v[0];
        if (j < n && col + 1 < G) x[n_cap + j] = v[1];
      }
    }
    if (kb + kQ8Block > n) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (kb + 8 * i + r8 >= n) s[i] = f2_pack(-INFINITY, -INFINITY);
    }
    float t[2];
    {
      float y[4][2];
#pragma unroll
      for (int i = 0; i < 4; ++i) f2_unpack(s[i], y[i][0], y[i][1]);
#pragma unroll
      for (int e = 0; e < 2; ++e) t[e] = fmaxf(fmax3(y[0][e], y[1][e], y[2][e]), y[3][e]);
    }
    if (__any_sync(0xffffffffu, t[0] > m[0] || t[1] > m[1])) {
      float was[2], k[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) t[e] = fmaxf(t[e], __shfl_xor_sync(0xffffffffu, t[e], o));
        const float mn = fmaxf(m[e], t[e]);
        was[e] = m[e] == mn ? 1.f : ex2_approx(m[e] - mn);
        m[e] = mn;
        k[e] = mn == -INFINITY ? 0.f : -mn;
      }
      nm = f2_pack(k[0], k[1]);
      const uint64_t was2 = f2_pack(was[0], was[1]);
      l = f2_mul(l, was2);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        acc[v][0] = f2_mul(acc[v][0], was2);
        acc[v][1] = f2_mul(acc[v][1], was2);
      }
    }
    // (14 is added to the difference: 14 - m would round to a multiple of 4 or more once a logit reaches 2^25, with weights of 2^16
    // and masses off by powers of two.  Four instructions a block: 32 layers x 8272 rows 89.9 us either way)
    const uint64_t top = f2_pack(kQ8WeightLog2, kQ8WeightLog2);
    const float take = GP == 4 && c4 < 2 ? 0.f : -1.f;
    const uint64_t minus_hi = f2_pack(take, take);
    uint32_t b[2][NB];  // B operand of P: [16 keys][b0, b1 (GP = 8: of both terms)]
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float p[2];
      f2_unpack(f2_add(f2_add(s[i], nm), top), p[0], p[1]);
      p[0] = ex2_approx(p[0]);
      p[1] = ex2_approx(p[1]);
      const uint64_t p2 = f2_pack(p[0], p[1]);
      l = f2_add(l, p2);
      const __half2 hi = __floats2half2_rn(p[0], p[1]);
      const float2 back = __half22float2(hi);
      float r[2];  // less the first term: GP = 4, in the lanes of the second terms only
      f2_unpack(f2_fma(f2_pack(back.x, back.y), minus_hi, p2), r[0], r[1]);
      const __half2 lo = __floats2half2_rn(r[0], r[1]);
      const uint32_t h = *reinterpret_cast<const uint32_t*>(&hi), e = *reinterpret_cast<const uint32_t*>(&lo);
      if (GP == 4) {
        b[i >> 1][i & 1] = movmatrix_trans(e);
      } else {
        b[i >> 1][i & 1] = movmatrix_trans(h);
        b[i >> 1][NB - 2 + (i & 1)] = movmatrix_trans(e);
      }
    }
    // (weights count as 2^14: with the values' scale 2^14 smaller the sums are in units of 1)
    const float vs = __uint_as_float(sc[1]) * (1.f / 16384.f);
    const uint64_t vs2 = f2_pack(vs, vs);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      uint32_t w[4];
      ldmatrix_x4_trans(w, (stage + St::kV + toff) ^ (v << 4));
      float d[4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t a[4];
        q8_unpack(__byte_perm(w[2 * h], 0, 0x3120), a[0], a[1]);
        q8_unpack(__byte_perm(w[2 * h + 1], 0, 0x3120), a[2], a[3]);
        if (h == 0) mma_f16_zero(d, a, b[h][NB - 2], b[h][NB - 1]);
        else mma_f16(d, a, b[h][NB - 2], b[h][NB - 1]);
        if (GP == 8) mma_f16(d, a, b[h][0], b[h][1]);
      }
      acc[v][0] = f2_fma(f2_pack(d[0], d[1]), vs2, acc[v][0]);
      acc[v][1] = f2_fma(f2_pack(d[2], d[3]), vs2, acc[v][1]);
    }
  }

  // Written out: m and l of head g at ml[2 g], the values at vals + g * D.
  __device__ __forceinline__ void store(float* ml, float* vals, int G, int lane) {
    const int r8 = lane >> 2, c4 = lane & 3;
    float ls[2];
    f2_unpack(l, ls[0], ls[1]);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) ls[e] += __shfl_xor_sync(0xffffffffu, ls[e], o);
      ls[e] *= 1.f / 16384.f;
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      float x[2][2];
      f2_unpack(acc[v][0], x[0][0], x[0][1]);
      f2_unpack(acc[v][1], x[1][0], x[1][1]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (GP == 4) {
          x[0][e] += __shfl_xor_sync(0xffffffffu, x[0][e], 2);
          x[1][e] += __shfl_xor_sync(0xffffffffu, x[1][e], 2);
        }
        const int head = 2 * c4 + e;
        if (head < G && (GP == 8 || c4 < 2)) *reinterpret_cast<float2*>(vals + head * D + 16 * v + 2 * r8) = make_float2(x[0][e], x[1][e]);
      }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int head = 2 * c4 + e;
      if (head < G && (GP == 8 || c4 < 2) && r8 == 0) {
        ml[2 * head] = ls[e] == ls[e] ? m[e] : INFINITY;  // a NaN sum is not to be merged as an empty state
        ml[2 * head + 1] = ls[e];
      }
    }
  }
};

// RAGGED: a count for each cache.  MASS: logits are kept, and the state of every pair, unless its masses are added here.
template <int D, int GP, bool RAGGED, bool MASS>
__global__ void __launch_bounds__(kQ8DecThreads, kQ8DecCtasPerSm) q8_decode_kernel(const __grid_constant__ Q8DecodeArgs a) {
  using State = Q8State<D, GP>;
  using St = Q8Stage<D, GP>;
  constexpr int kNoMore = -0x40000000;
  extern __shared__ __align__(128) uint8_t q8_smem[];  // per-warp rings, then per-warp states
  __shared__ ListCounts s_list;  // RAGGED
  __shared__ float s_ml[kQ8DecWarps][2 * GP];
  __shared__ float s_joined[kQ8DecWarps][2 * GP];     // MASS, whole pairs: of each head m and 1 / (G l)
  __shared__ ListCursor s_cursor[kQ8DecWarps], s_here[kQ8DecWarps];  // where each warp's copies and its arithmetic are, out of its registers
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();
  pdl_launch_dependents();
  int n_all = 0, total;
  if constexpr (!RAGGED) {
    n_all = list_keys(a, 0, blockIdx.x == 0 && threadIdx.x == 0);
    total = list_blocks(n_all) * a.n_layers * a.Hkv;
  } else {
    if (warp == 0) list_counts<kQ8Pad>(a, s_list, blockIdx.x == 0);
    __syncthreads();
    total = s_list.first[a.n_layers];
  }
  auto keys_of = [&](int layer) { return RAGGED ? s_list.n[layer] : n_all; };
  auto blocks_of = [&](int layer) { return list_blocks(keys_of(layer)); };
  constexpr int kPad = RAGGED ? kQ8Pad : 0;
  const ListSplit sp = list_split(a, !RAGGED, list_blocks(n_all), total);
  const int W = a.whole ? a.whole : sp.W, rank = warp & (W - 1);
  const int group = W == 1 ? blockIdx.x * kQ8DecWarps + warp : blockIdx.x;
  float* s_vals = reinterpret_cast<float*>(q8_smem + kQ8DecWarps * St::kStages * St::kBytes);
  const uint32_t ring = smem_u32(q8_smem + warp * St::kStages * St::kBytes);

  // the range and its first pair
  ListCursor ci;
  ci.layer = a.n_layers;
  if (a.whole) {
    if (group < a.n_layers * a.Hkv) {
      ci.pair = group;
      const int layer = fdivmod(group, a.by_heads, ci.h), nb = blocks_of(layer);
      ci.blk = 0;
      ci.end = ci.left = nb;
      if (nb > 0) {
        ci.layer = layer;
      } else {
        float4* out = reinterpret_cast<float4*>(a.out[layer] + (size_t)ci.h * a.G * D);
        for (int t = rank * 32 + lane; t < a.G * D / 4; t += W * 32) out[t] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
    }
  } else if (!RAGGED && sp.k > 0) {
    const int nb = list_blocks(n_all);
    ci.pair = (unsigned)group / (unsigned)sp.k;
    ci.blk = (group - ci.pair * sp.k) * sp.per;
    if (ci.pair < a.n_layers * a.Hkv && ci.blk < nb) {
      ci.layer = fdivmod(ci.pair, a.by_heads, ci.h);
      ci.end = min(nb, ci.blk + sp.per);
      ci.left = ci.end;
    }
  } else {
    const int lo = min(total, group * sp.per), hi = min(total, lo + sp.per);
    if (lo < hi) {
      int at, nb;
      if constexpr (!RAGGED) {
        nb = list_blocks(n_all);
        ci.pair = (unsigned)lo / (unsigned)nb;
        ci.layer = fdivmod(ci.pair, a.by_heads, ci.h);
        at = lo - ci.pair * nb;
      } else {
        ci.layer = 0;
        while (s_list.first[ci.layer + 1] <= lo) ++ci.layer;
        nb = blocks_of(ci.layer);
        at = lo - s_list.first[ci.layer];
        ci.h = (unsigned)at / (unsigned)(nb + kPad);
        ci.pair = ci.layer * a.Hkv + ci.h;
        at -= ci.h * (nb + kPad);
      }
      ci.blk = at;
      ci.left = hi - lo + at;
      ci.end = min(nb, ci.left);
    }
  }
  auto next_pair = [&](ListCursor& c) {
    c.left -= blocks_of(c.layer) + kPad;
    if (c.left <= 0) {
      c.layer = a.n_layers;
      return;
    }
    ++c.pair;
    if (++c.h == a.Hkv) {
      c.h = 0;
      ++c.layer;
      while (keys_of(c.layer) == 0) {
        ++c.layer;
        c.pair += a.Hkv;
      }
    }
    c.blk = 0;
    c.end = min(blocks_of(c.layer), c.left);
  };

  if (RAGGED && ci.layer < a.n_layers && ci.blk >= ci.end) next_pair(ci);  // (the range begins behind a pair's own blocks)
  if (ci.layer == a.n_layers) return;  // whole groups
  if (lane == 0) s_here[warp] = ci;

  // copies: kStages blocks ahead of the arithmetic, across pairs
  constexpr int kVecRow = D / 16, kRows = 32 / kVecRow, kCopies = kQ8Block / kRows;  // vectors a row, rows an instruction, instructions
  const int cp_row = lane / kVecRow, cp_vec = lane & (kVecRow - 1);
  const uint32_t cp_dst = cp_row * D + ((cp_vec ^ St::swizzle(cp_row)) << 4);  // (D = 128: of odd instructions, rows 4 further, ^ 64)
  const uint8_t *Kc = nullptr, *Vc = nullptr;  // this lane's part of the next block
  const float* Sc = nullptr;                   // lane 0: the block's scale of keys; lane 1: of values
  auto bases = [&](const ListCursor& c) {
    const int64_t code = c.h * a.code_head_stride + (int64_t)c.blk * (kQ8Block * D) + lane * 16;
    Kc = a.K[c.layer] + code;
    Vc = a.V[c.layer] + code;
    Sc = (lane == 0 ? a.K_scale[c.layer] : a.V_scale[c.layer]) + c.h * a.scale_head_stride + c.blk;
  };
  // RAGGED: a pair of which the range holds a block or two is one warp's, the warps taking turns, and the others go on: the
  // short lists run side by side.
  auto alone = [&](const ListCursor& c) { return RAGGED && c.end - c.blk <= kListAlone; };
  auto mine = [&](const ListCursor& c) { return !alone(c) || (c.pair & (W - 1)) == rank; };
  ListCursor& is = s_cursor[warp];
  // from the next block on: blocks of this warp left in the pair (<= 0: none), rows of the pair; blocks from one to the next
  int ahead, rows, step;
  auto enter = [&](ListCursor& c) {  // c: a pair's, its first block
    step = alone(c) ? 1 : W;
    ahead = mine(c) ? c.end - c.blk : 0;
    if (!alone(c)) {
      c.blk += rank;
      ahead = (c.end - c.blk + W - 1) / W;
    }
    rows = keys_of(c.layer) - c.blk * kQ8Block;
    bases(c);
  };
  {
    ListCursor c = ci;
    enter(c);
    if (lane == 0) is = c;
    __syncwarp();
  }
  const uint64_t policy = MASS ? q8_evict_first() : 0ull;
  auto issue_next = [&](uint32_t dst) {
    if (ahead <= 0 && ahead > kNoMore / 2) {
      ListCursor c = is;
      do {
        next_pair(c);
        if (c.layer < a.n_layers) enter(c);
        else ahead = kNoMore;
      } while (ahead <= 0 && ahead > kNoMore / 2);
      __syncwarp();
      if (lane == 0) is = c;
      __syncwarp();
    }
    if (ahead > 0) {
      const uint32_t d16 = dst + cp_dst;
      if (rows >= kQ8Block) {
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
          const uint32_t to = (D == 128 && (i & 1) ? d16 ^ 64 : d16) + i * 512;
          if constexpr (MASS) {
            q8_cp_hint(to, Kc + i * 512, policy);
            q8_cp_hint(to + St::kV, Vc + i * 512, policy);
          } else {
            cp_async<16>(to, Kc + i * 512);
            cp_async<16>(to + St::kV, Vc + i * 512);
          }
        }
      } else {  // rows past the count: zeros, nothing is read
#pragma unroll 1
        for (int i = 0; i < kCopies; ++i) {
          const int bytes = i * kRows + cp_row < rows ? 16 : 0;
          const uint32_t to = (D == 128 && (i & 1) ? d16 ^ 64 : d16) + i * 512;
          cp_async_part<16>(to, Kc + i * 512, bytes);
          cp_async_part<16>(to + St::kV, Vc + i * 512, bytes);
        }
      }
      if (lane < 2) cp_async<4>(dst + St::kScales + 4 * lane, Sc);
    }
    cp_async_commit();
    --ahead;
    rows -= step * kQ8Block;
    Kc += step * (kQ8Block * D);
    Vc += step * (kQ8Block * D);
    Sc += step;
  };
#pragma unroll
  for (int i = 0; i < St::kStages - 1; ++i) issue_next(ring + i * St::kBytes);

  const int lm_row = (lane & 7) + (lane & 8), lm_vec = lane >> 4;  // ldmatrix: keys 0-7 and 8-15 of a vector, then of the next
  const uint32_t off = lm_row * D + ((lm_vec ^ St::swizzle(lm_row)) << 4);
  const uint32_t toff = lane * D + (St::swizzle(lane) << 4);       // 32 values of a vector
  State st;
  int stage = 0, fill = St::kStages - 1;
  for (;;) {
    __syncwarp();
    ListCursor ci = s_here[warp];
    const bool solo = alone(ci) || W == 1, my = mine(ci);
    if (my) {
      const int n = keys_of(ci.layer), kstep = (solo ? 1 : W) * kQ8Block, k_end = ci.end * kQ8Block;
      int kb = (ci.blk + (solo ? 0 : rank)) * kQ8Block;
      float* x = MASS ? a.logits + ((size_t)ci.pair * a.G + 2 * (lane & (GP == 4 ? 1 : 3))) * a.n_cap : nullptr;
      st.clear();
      if (kb < k_end) st.load_q(a.q[ci.layer] + (size_t)ci.h * a.G * D, a.G, lane);
#pragma unroll 1
      for (; kb < k_end; kb += kstep) {
        issue_next(ring + fill * St::kBytes);
        fill = fill + 1 == St::kStages ? 0 : fill + 1;
        cp_async_wait<St::kStages - 1>();
        __syncwarp();
        st.template block<MASS>(ring + stage * St::kBytes, off, toff, kb, n, a.c, lane, x, a.n_cap, a.G);
        __syncwarp();
        stage = stage + 1 == St::kStages ? 0 : stage + 1;
      }
      ci = s_here[warp];
      const int first = ci.blk, G = a.G;
      st.store(s_ml[warp], s_vals + warp * GP * D, G, lane);
      auto sync_group = [&]() {
        if (solo) __syncwarp();
        else named_bar_sync(1, kQ8DecThreads);
      };
      sync_group();
      const int w0 = solo ? warp : 0, w1 = solo ? warp + 1 : kQ8DecWarps;
      const int t0 = solo ? lane : (int)threadIdx.x, t_step = solo ? 32 : kQ8DecThreads;
      const bool all = first == 0 && ci.end == blocks_of(ci.layer);
      for (int t = t0; t < G * (D / 4); t += t_step) {
        const int g = t / (D / 4), e0 = (t - g * (D / 4)) * 4;
        float mm = -INFINITY, ll = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
        for (int w = w0; w < w1; ++w) {
          const float4 y = *reinterpret_cast<const float4*>(s_vals + (w * GP + g) * D + e0);
          const float v2[4] = {y.x, y.y, y.z, y.w};
          merge_state<4>(mm, ll, v, s_ml[w][2 * g], s_ml[w][2 * g + 1], v2);
        }
        if (all)
          *reinterpret_cast<float4*>(a.out[ci.layer] + (size_t)(ci.h * G + g) * D + e0) =
              make_float4(v[0] / ll, v[1] / ll, v[2] / ll, v[3] / ll);
        if (MASS && a.mass_here) {
          if (e0 == 0) {
            s_joined[w0][2 * g] = mm;
            s_joined[w0][2 * g + 1] = 1.f / (ll * (float)G);
          }
        } else if (!all || MASS) {
          const int slot = a.whole ? ci.pair : !RAGGED && sp.k > 0 ? group : group + ci.pair;
          float* dst = a.part + ((size_t)slot * G + g) * (D + 4);
          if (e0 == 0) {
            dst[0] = mm;
            dst[1] = ll;
          }
          if (!all) *reinterpret_cast<float4*>(dst + 4 + e0) = make_float4(v[0], v[1], v[2], v[3]);
        }
      }
      sync_group();
      if (MASS && a.mass_here) {  // this warp's blocks, whose logits it wrote
        const float* lg = a.logits + (size_t)ci.pair * G * a.n_cap;
        float* mass = a.mass[ci.layer] + (int64_t)ci.h * a.mass_stride;
        const float* joined = s_joined[w0];
        constexpr int U = 4;  // blocks in flight
        for (int b = solo ? 0 : rank; b < ci.end; b += U * (solo ? 1 : W)) {
          float was[U], sum[U];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int j = (b + u * (solo ? 1 : W)) * kQ8Block + lane;
            was[u] = j < n ? __ldcg(mass + j) : 0.f;
            sum[u] = 0.f;
          }
#pragma unroll
          for (int g = 0; g < GP; ++g) {
            if (g >= G) break;
#pragma unroll
            for (int u = 0; u < U; ++u) {
              const int j = (b + u * (solo ? 1 : W)) * kQ8Block + lane;
              const float y = j < n ? __ldcg(lg + (size_t)g * a.n_cap + j) : 0.f;
              sum[u] = fmaf(ex2_approx(y - joined[2 * g]), joined[2 * g + 1], sum[u]);
            }
          }
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int j = (b + u * (solo ? 1 : W)) * kQ8Block + lane;
            if (j < n) mass[j] = was[u] + sum[u];
          }
        }
      }
      sync_group();
    }
    __syncwarp();  // (another warp's pair: all lanes have read s_here)
    next_pair(ci);
    if (ci.layer == a.n_layers) break;
    if (lane == 0) s_here[warp] = ci;
  }
}

// Where the states of a pair are: `count` slots from `slot` on.
struct Q8Slots {
  int n, slot, count;  // keys
};
__device__ __forceinline__ Q8Slots q8_slots(const Q8DecodeArgs& a, const ListCounts& s, bool uniform, int pair, int layer, int h) {
  Q8Slots r;
  int first, total;  // the pair's first block in the list, all blocks
  if (uniform) {
    r.n = list_keys(a, 0);
    first = layer * a.Hkv * list_blocks(r.n);
    total = a.n_layers * a.Hkv * list_blocks(r.n);
  } else {
    r.n = s.n[layer];
    first = s.first[layer];
    total = s.first[a.n_layers];
  }
  const int nb = list_blocks(r.n), pad = uniform ? 0 : kQ8Pad;
  r.slot = r.count = 0;
  if (nb == 0) return r;
  if (a.whole) {
    r.slot = pair;
    r.count = 1;
    return r;
  }
  const ListSplit sp = list_split(a, uniform, nb, total);
  if (sp.k > 0) {
    r.slot = pair * sp.k;
    r.count = sp.k;
  } else {
    const int b0 = first + h * (nb + pad), g0 = (unsigned)b0 / (unsigned)sp.per;
    r.slot = g0 + pair;
    r.count = (unsigned)(b0 + nb - 1) / (unsigned)sp.per - g0 + 1;
  }
  return r;
}

// The masses of a chunk of a pair's keys, from the logits and the joined (maximum, sum) of the pair's states.  All loads of a
// thread's keys are on their way before the states are joined.
constexpr int q8_mass_keys(int GP) { return GP == 4 ? 8 : 4; }  // of a thread
template <int D, int GP>
__device__ __forceinline__ void q8_add_mass(const Q8DecodeArgs& a, const ListCounts& s, bool uniform, int chunk, float (*s_joined)[2]) {
  constexpr int U = q8_mass_keys(GP);
  int h, part;
  const int pair = fdivmod(chunk, a.by_chunks, part), layer = fdivmod(pair, a.by_heads, h), G = a.G;
  const Q8Slots sl = q8_slots(a, s, uniform, pair, layer, h);
  const int j0 = part * U * (int)blockDim.x + (int)threadIdx.x;
  if (part * U * (int)blockDim.x >= sl.n) return;  // (the whole block)
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float* x = a.logits + (size_t)pair * G * a.n_cap;
  float* mass = a.mass[layer] + (int64_t)h * a.mass_stride;
  float y[GP][U], was[U];
#pragma unroll
  for (int g = 0; g < GP; ++g)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = j0 + u * (int)blockDim.x;
      y[g][u] = g < G && k < sl.n ? __ldcg(x + (size_t)g * a.n_cap + k) : 0.f;
    }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int k = j0 + u * (int)blockDim.x;
    was[u] = k < sl.n ? __ldcg(mass + k) : 0.f;
  }
  for (int g = warp; g < G; g += blockDim.x >> 5) {
    float m = -INFINITY, l = 0.f;
    const float none[1] = {0.f};
    float dummy[1] = {0.f};
    for (int i = lane; i < sl.count; i += 32) {
      const float2 ml = __ldcg(reinterpret_cast<const float2*>(a.part + ((size_t)(sl.slot + i) * G + g) * (D + 4)));
      merge_state<1>(m, l, dummy, ml.x, ml.y, none);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      const float m2 = __shfl_xor_sync(0xffffffffu, m, o), l2 = __shfl_xor_sync(0xffffffffu, l, o);
      merge_state<1>(m, l, dummy, m2, l2, none);
    }
    if (lane == 0) {
      s_joined[g][0] = m;
      s_joined[g][1] = 1.f / (l * (float)G);
    }
  }
  __syncthreads();
  float sum[U];
#pragma unroll
  for (int u = 0; u < U; ++u) sum[u] = 0.f;
#pragma unroll
  for (int g = 0; g < GP; ++g) {
    if (g >= G) break;
    const float m = s_joined[g][0], f = s_joined[g][1];
#pragma unroll
    for (int u = 0; u < U; ++u) sum[u] = fmaf(ex2_approx(y[g][u] - m), f, sum[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int k = j0 + u * (int)blockDim.x;
    if (k < sl.n) mass[k] = was[u] + sum[u];
  }
}

// The partial states of a pair joined in key order, by NW warps a (pair, head); pairs that one range held whole are
// written already; those without keys are set to zero.  Blocks from join_blocks on add to masses.
// Which slots a pair has follows from the counts, which are final once the kernel before has passed its own wait: they are
// read before this one's.
template <int D, int GP, int NW>
__global__ void __launch_bounds__(NW == 1 ? 128 : NW * 32) q8_merge_kernel(const __grid_constant__ Q8DecodeArgs a) {
  constexpr int PER = D / 32, kInFlight = NW == 1 ? 4 : NW, kItems = NW == 1 ? 4 : 1;
  __shared__ ListCounts s_list;
  __shared__ float s_ml[NW][2];
  __shared__ float s_v[NW][D];
  __shared__ float s_joined[8][2];
  const int warp = NW == 1 ? 0 : threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool uniform = list_uniform(a);
  if (!uniform) {
    if (threadIdx.x < 32) list_counts<kQ8Pad>(a, s_list, false);
    __syncthreads();
  }
  if ((int)blockIdx.x >= a.join_blocks) {
    pdl_wait();
    pdl_launch_dependents();
    q8_add_mass<D, GP>(a, s_list, uniform, blockIdx.x - a.join_blocks, s_joined);
    return;
  }
  const int item = blockIdx.x * kItems + (NW == 1 ? threadIdx.x >> 5 : 0);
  int g, h;
  const int pair = fdivmod(item, a.by_G, g), layer = fdivmod(pair, a.by_heads, h);
  if (layer >= a.n_layers) return;  // NW == 1: past the last pair
  const Q8Slots sl = q8_slots(a, s_list, uniform, pair, layer, h);
  float* out = a.out[layer] + (size_t)(h * a.G + g) * D;
  pdl_wait();
  pdl_launch_dependents();
  const int t = NW == 1 ? lane : threadIdx.x;
  if (sl.n == 0 && t < D / 4) reinterpret_cast<float4*>(out)[t] = make_float4(0.f, 0.f, 0.f, 0.f);
  if (sl.count <= 1) return;
  float mm = -INFINITY, ll = 0.f, aa[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) aa[e] = 0.f;
#pragma unroll 1
  for (int i0 = warp; i0 < sl.count; i0 += kInFlight * NW) {
    float2 ml[kInFlight];
    float a2[kInFlight][PER];
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) {
      const float* src = a.part + ((size_t)(sl.slot + i0 + u * NW) * a.G + g) * (D + 4);
      const bool ok = i0 + u * NW < sl.count;
      ml[u] = ok ? __ldcg(reinterpret_cast<const float2*>(src)) : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int e = 0; e < PER; ++e) a2[u][e] = ok ? __ldcg(src + 4 + e * 32 + lane) : 0.f;
    }
#pragma unroll
    for (int u = 0; u < kInFlight; ++u) merge_state<PER>(mm, ll, aa, ml[u].x, ml[u].y, a2[u]);
  }
  if constexpr (NW == 1) {
#pragma unroll
    for (int e = 0; e < PER; ++e) out[e * 32 + lane] = aa[e] / ll;
  } else {
    if (lane == 0) {
      s_ml[warp][0] = mm;
      s_ml[warp][1] = ll;
    }
#pragma unroll
    for (int e = 0; e < PER; ++e) s_v[warp][e * 32 + lane] = aa[e];
    __syncthreads();
    if ((int)threadIdx.x < D) {
      float m1 = -INFINITY, l1 = 0.f, v1[1] = {0.f};
#pragma unroll 1
      for (int w = 0; w < NW; ++w) {
        const float v2[1] = {s_v[w][threadIdx.x]};
        merge_state<1>(m1, l1, v1, s_ml[w][0], s_ml[w][1], v2);
      }
      out[threadIdx.x] = v1[0] / l1;
    }
  }
}

// Partial states: a pair of n rows leaves at most one slot per block of the list, and all pairs together at most one per group
// and pair.
// Behind them, for masses, the logits.
static size_t q8_part_bytes(int n_layers, int Hkv, int Hq, int d, int n_cap) {
  const int64_t pairs = (int64_t)n_layers * Hkv, blocks = pairs * (((int64_t)n_cap + kQ8Block - 1) / kQ8Block + kQ8Pad);
  const size_t b = (size_t)(std::min<int64_t>(kListMaxGroups, blocks) + pairs) * (Hq / Hkv) * (d + 4) * sizeof(float);
  return (b + 255) & ~(size_t)255;
}
size_t q8_decode_ws_bytes(int n_layers, int Hkv, int Hq, int d, int n_cap, bool mass) {
  return q8_part_bytes(n_layers, Hkv, Hq, d, n_cap) + (mass ? (size_t)n_layers * Hq * n_cap * sizeof(float) : 0);
}

// Warps that take a pair whole, which needs no partial states and no second kernel, or 0; by the most blocks a pair can have (where
// the counts are on the device: by n_cap).  A warp each where pairs are many and short (64 layers x 8 heads, G = 1, 32 rows 3.9 us, a CTA
// each 6.8, cut 5.4), else a CTA, while what its last wave leaves idle costs less than that kernel (1 layer x 8 heads x 512 rows 5.9
// us, cut 7.0; 32 x 8 heads x 2048 rows 24.7, cut 27.5).
static int q8_whole(int pairs, int slots, int nb, bool ragged) {
  if (pairs > slots && nb <= 12) return 1;
  const int64_t rounds = (nb + kQ8DecWarps - 1) / kQ8DecWarps, idle = pairs % slots ? slots - pairs % slots : 0;
  return rounds * idle <= 6 * slots && !(ragged && rounds > 12) ? kQ8DecWarps : 0;
}

template <int D, int GP>
static cudaError_t q8_decode_launch(Q8DecodeArgs& a, cudaStream_t stream) {
  const bool ragged = a.n_dev && a.n_stride && a.n_layers > 1, mass = a.logits != nullptr;
  void (*kern)(Q8DecodeArgs) = ragged ? (mass ? q8_decode_kernel<D, GP, true, true> : q8_decode_kernel<D, GP, true, false>)
                                      : (mass ? q8_decode_kernel<D, GP, false, true> : q8_decode_kernel<D, GP, false, false>);
  using St = Q8Stage<D, GP>;
  const int smem = std::max(kQ8DecMinSmem, kQ8DecWarps * (St::kStages * St::kBytes + GP * D * (int)sizeof(float)));
  cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(kern), smem);
  const int pairs = a.n_layers * a.Hkv;
  if (e == cudaSuccess) e = launch_kernel(kern, dim3(a.n_groups), dim3(kQ8DecThreads), smem, stream, a, true);
  if (e != cudaSuccess || (a.whole && (!mass || a.mass_here))) return e;
  const int nw = a.whole ? 1 : a.n_groups >= 16 * pairs ? 8 : a.n_groups > 5 * pairs ? 4 : 1;
  a.join_blocks = a.whole ? 0 : nw == 1 ? (pairs * a.G + 3) / 4 : pairs * a.G;
  int64_t blocks = a.join_blocks;
  if (mass) {
    const int keys = q8_mass_keys(GP) * (nw == 8 ? 256 : 128), chunks = std::max(1, ((a.n_dev ? a.n_cap : a.n_host) + keys - 1) / keys);
    a.by_chunks = make_fastdiv(chunks);
    blocks += (int64_t)pairs * chunks;
  }
  void (*merge)(Q8DecodeArgs) = nw == 8 ? q8_merge_kernel<D, GP, 8> : nw == 4 ? q8_merge_kernel<D, GP, 4> : q8_merge_kernel<D, GP, 1>;
  return launch_kernel(merge, dim3((unsigned)blocks), dim3(nw == 8 ? 256 : 128), 0, stream, a, true);
}

stepkv_status_t q8_decode_run(const stepkv_q8_cache_t& c, const void* const* q, int Hq, const int32_t* n_dev, int n_stride,
                              int n_host, int n_cap, float* const* out, float* const* mass, int64_t mass_stride, void* ws,
                              int32_t* status, cudaStream_t stream) {
  int n_sm = 0;
  cudaError_t e = device_sm_count(&n_sm);
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
    a.n_layers = nl;
    a.layer0 = l0;
    a.Hkv = c.Hkv;
    a.G = Hq / c.Hkv;
    // as many groups as run at once, none without a block
    const int64_t blocks = (int64_t)nl * c.Hkv * ((n_cap + kQ8Block - 1) / kQ8Block);
    const int slots = std::min(kListMaxGroups / kQ8DecWarps, n_sm * kQ8DecCtasPerSm);
    a.n_groups = (int)std::min<int64_t>(slots, blocks);
    const bool ragged = n_dev && n_stride && nl > 1;
    const int nb = ((n_dev ? n_cap : n_host) + kQ8Block - 1) / kQ8Block;
    a.whole = q8_whole(nl * c.Hkv, slots, nb, ragged);
    a.mass_here = mass && a.whole && nb <= kQ8FewRounds * a.whole;
    if (a.whole) a.n_groups = (nl * c.Hkv * a.whole + kQ8DecWarps - 1) / kQ8DecWarps;
    for (int i = 0; i < 2; ++i) {
      const int groups = a.n_groups * (i ? kQ8DecWarps : 1);
      a.by_groups[i] = make_fastdiv(groups);
      a.by_k[i] = make_fastdiv(std::max(1, groups / (nl * c.Hkv)));
    }
    a.by_heads = make_fastdiv(c.Hkv);
    a.by_G = make_fastdiv(a.G);
    a.n_dev = n_dev;
    a.n_stride = n_stride;
    a.n_host = n_host;
    a.n_cap = n_cap;
    a.c = (float)(1.4426950408889634 / sqrt((double)c.d));
    a.part = static_cast<float*>(ws);
    a.logits = mass ? reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + q8_part_bytes(nl, c.Hkv, Hq, c.d, n_cap)) : nullptr;
    a.status = status;
    if (c.d == 128)
      e = a.G <= 4 ? q8_decode_launch<128, 4>(a, stream) : q8_decode_launch<128, 8>(a, stream);
    else
      e = a.G <= 4 ? q8_decode_launch<64, 4>(a, stream) : q8_decode_launch<64, 8>(a, stream);
  }
  if (e == cudaSuccess) return STEPKV_OK;
  set_last_cuda_error(e);
  return STEPKV_ECUDA;
}

}  // namespace stepkv
