// Decode attention over a cache held in 4 bits (format in q4.cu):
//   out[g][:] = sum_{j < n} softmax_j( q[g] . K[g/G][j] / sqrt(d) ) V[g/G][j][:]
// with K and V the values the codes stand for, one count n per cache or one for all.
//
// A row pair is 144 bytes at d = 128 where bf16 takes 512, so at the copy rate a scheduler has 24 cycles per row pair and
// turning codes into operands has to cost next to nothing.  Both contractions run on the tensor cores (mma.sync: a KV
// head's G <= 8 query heads are the 8 columns of a tile, the rows of the cache its 16 rows; tcgen05 takes none
// from registers: the unpacked codes would go through shared or tensor memory first, 16 bits a code, for tiles of which the few
// heads fill an eighth or less), a warp on 32 keys at a time:
//   S^T = K Q^T.  A half whose bits 7-10 hold a code n, and nothing else, is the fp16 number n 2^-17 (its subnormals and
//     first binade run on linearly), with the code in bits 3-6 n 2^-21: two shifts and four masks turn a word of eight codes
//     into operands.  (Lower still the tensor core loses bits: it does not normalise subnormals.  e4m3 operands, 0000nnnn =
//     n 2^-9, take a shift and two masks, but their mma.sync runs as conversions and two fp16 MMAs: 81 us where this
//     took 77.)  Q is scaled by a power of two and exact in fp16.  A group's 32 channels are two k-steps from
//     -8 sum(q) of the group, which the sum of n q nearly cancels where the codes are near 8; the scale is applied to what is
//     left, so that groups do not round against each other.  (The -8 of all groups first, as one MMA of the scales and -8
//     sum(q), took 12 instructions a block fewer, 60.5 us, but logits rounded by the sum of all |s| 8 sum(q): outputs off by
//     1.5e-6 instead of 1.9e-7 for queries of one sign over keys with one channel a group.)
//   O^T = V^T P^T.  ldmatrix with transposition puts the codes of two keys and one chunk of 4 channels into a word; each
//     pair of codes becomes (64 + n) s - 72 s = (n - 8) s by a mask and one packed FMA, exactly (s has 5 bits, 72 has 4).
//     The weights are two fp16 terms, 22 bits, and come from the layout of S^T by movmatrix.
// For G <= 4 columns 4-7 repeat the heads of columns 0-3, and P has its first terms in 0-3 and its second in 4-7.
// Every sum over keys starts from zero in the tensor core for 32 keys and is added in fp32, as its accumulation truncates.
//
// 556 instructions a block of 32 keys (G <= 4), of which unpacking V takes 176, K 96.  Mixed, they issue at 0.64 a cycle at
// most (a probe of LOP3, HFMA2, FFMA and MMA together), which bounds the kernel: 32 layers x 8 heads x 8272 rows 60.8 us, G =
// 5: 67.7, where the reads take 45 and the scalar kernel took 995.  12 warps of 168 registers on an SM; 16 warps of 128 took
// 66.0 (more moves), 8 of 255 72.4; three ring stages 66.0; a barrier that keeps the SM's warps in step 64-70 (they finish
// between 45 and 60 us without, at the same rate in all); scales laid out in shared memory for their users 67.0.
// (Times here and below: a call of a captured graph of ten equal ones.  Caches under some 100 MB, as those of one layer, short
// lists or ragged batches are, then come out of L2; a chain of 32 layers, one call each from DRAM, takes 10.5 us a layer where
// the captured loop of one layer takes 10.1.)
//
// Each warp copies its blocks of 32 rows into a ring of its own with cp.async.  A group of warps takes a pair (q4_whole) or a
// range of the list of all pairs' blocks (q4_split); its warps interleave the blocks of a pair, join their states in shared
// memory, and write the output where they had the whole pair, or else leave a partial state, which a second kernel joins with
// the others in key order.
#include <cuda_fp16.h>
#include <math.h>

#include <algorithm>

#include "common.cuh"
#include "fastdiv.h"
#include "internal.h"

namespace stepkv {

constexpr int kQ4DecWarps = 4;      // of a CTA: a group, unless the pairs are many and short
constexpr int kQ4DecThreads = kQ4DecWarps * 32;
constexpr int kQ4DecCtasPerSm = 3;
constexpr int kQ4DecMinSmem = 228 * 1024 / (kQ4DecCtasPerSm + 1);
constexpr int kQ4Block = 32;        // keys per warp step
constexpr int kQ4Stages = 2;
constexpr int kQ4Few = 16;          // blocks of a pair that one CTA takes at once, though the pair might be cut
constexpr int kQ4Alone = 2;         // blocks of a pair that a warp takes by itself
constexpr int kQ4MaxGroups = 4096;  // workspace sizing: groups (single warps) of a launch at most
constexpr float kQ4WeightLog2 = 14.f;  // the largest weight is held as 2^14 (fp16 reaches 65504)

struct Q4DecodeArgs {
  const uint16_t* q[kQ4Layers];
  const uint8_t* K[kQ4Layers];
  const uint8_t* V[kQ4Layers];
  const __half* K_scale[kQ4Layers];
  const __half* V_scale[kQ4Layers];
  float* out[kQ4Layers];
  int64_t code_head_stride, scale_head_stride;
  int n_layers, layer0;
  int Hkv, G;
  int n_groups;     // CTAs
  // with groups of kQ4DecWarps warps, and of one: divisors groups and k = groups / pairs (1 where there are more pairs)
  FastDiv by_groups[2], by_k[2];
  FastDiv by_heads, by_G;
  const int32_t* n_dev;
  int n_stride;
  int n_host;
  int n_cap;
  float c;          // log2(e) / sqrt(d)
  float* part;      // [slot][G][d + 4]: m, l, -, -, values
  int32_t* status;
  int whole;        // warps that take a pair, all of it: no states to join (0: the pairs are cut, q4_split)
  uint32_t magic;   // kQ4Magic: as a literal it is brought into a register 16 times a block (63.6 -> 61.8 us)
};
constexpr uint32_t kQ4Magic = 0x54005400u;  // two fp16 64
static_assert(sizeof(Q4DecodeArgs) <= 32000, "kernel parameter space");

// The keys of a cache of this launch.
__device__ __forceinline__ int q4_keys(const Q4DecodeArgs& a, int layer, bool tell = false) {
  if (!a.n_dev) return a.n_host;
  const int n = __ldcg(a.n_dev + (a.layer0 + layer) * a.n_stride);  // (the merge reads it early: not from L1)
  if (tell && n > a.n_cap) record_status(a.status, STEPKV_ENOSPACE);
  if (tell && n < 0) record_status(a.status, STEPKV_EDATA);
  return max(0, min(n, a.n_cap));
}

// Keys of every cache and the first block of each in the list of all pairs' blocks; first[n_layers]: all blocks.  By the
// first warp of a CTA; the caller synchronises.  Not used where all caches have one count.
struct Q4Lists {
  int n[kQ4Layers];
  int first[kQ4Layers + 1];
};
__device__ __forceinline__ int q4_blocks(int n) { return (n + kQ4Block - 1) / kQ4Block; }
__device__ __forceinline__ bool q4_uniform(const Q4DecodeArgs& a) { return !a.n_dev || a.n_stride == 0 || a.n_layers == 1; }
__device__ __forceinline__ void q4_lists(const Q4DecodeArgs& a, Q4Lists& s, bool tell) {
  const int lane = threadIdx.x & 31;
  int sum[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int l = 2 * lane + i;
    const int n = l < a.n_layers ? q4_keys(a, l, tell) : 0;
    s.n[l] = n;
    sum[i] = q4_blocks(n) * a.Hkv;
  }
  int total = sum[0] + sum[1];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, total, o);
    if (lane >= o) total += x;
  }
  s.first[2 * lane + 2] = total;
  s.first[2 * lane + 1] = total - sum[1];
  if (lane == 0) s.first[0] = 0;
}

// How the list of blocks is cut, where pairs are.  Ranges of `per` blocks of the list, one after another; or (k > 0: one count
// for all, and ranges that each lie in one pair, k in each, are nearly as even) these, which spares a second start and end to
// those that would reach over.  Groups are single warps where there are more pairs than CTAs and the pairs are short: a warp
// then takes a range by itself instead of waiting for three others at its end.
struct Q4Split {
  int W, per, k;
};
__device__ __forceinline__ Q4Split q4_split(const Q4DecodeArgs& a, bool uniform, int nb, int total) {
  Q4Split p;
  const int pairs = a.n_layers * a.Hkv;
  const int single = pairs > a.n_groups && total <= 16 * pairs;
  p.W = single ? 1 : kQ4DecWarps;
  const FastDiv groups = a.by_groups[single], ks = a.by_k[single];
  p.per = fdiv(total + groups.d - 1, groups);
  p.k = 0;
  if (uniform && nb > 0 && pairs <= groups.d) {
    // rounded up to whole rounds: a part of one takes as long, and fewer ranges are joined faster
    const int per = fdiv(nb + ks.d - 1, ks), whole = (per + p.W - 1) & -p.W;
    if (!single && nb <= kQ4Few) {  // (14 layers x 8 heads x 379 rows 8.0 -> 7.0 us; at 24 blocks 9.6 and 9.1, or slower)
      p.k = 1;
      p.per = nb;
    } else if (per <= p.per + 2 * p.W) {
      p.per = whole;
      p.k = (unsigned)(nb + whole - 1) / (unsigned)whole;
    }
  }
  return p;
}

// Copies of N bytes, and with fewer to read (then zeros).
template <int N>
__device__ __forceinline__ void q4_cp(uint32_t dst, const void* src) {
  if constexpr (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(N) : "memory");
}
template <int N>
__device__ __forceinline__ void q4_cp_part(uint32_t dst, const void* src, int bytes) {
  if constexpr (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(N), "r"(bytes) : "memory");
}
__device__ __forceinline__ void q4_cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void q4_cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) );
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) );
}
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
template <int BYTES>
__device__ __forceinline__ void q4_lds(uint32_t (&w)[BYTES / 4], uint32_t addr) {
  if constexpr (BYTES == 16)
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(addr));
  else if constexpr (BYTES == 8)
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(addr));
  else
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(addr));
}

// D = A B, D = A B + (c0, c1 in both rows), and D += A B, for one m16n8k16 tile of fp16.
__device__ __forceinline__ void mma_f16_zero(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void mma_f16_from(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, uint32_t c0, uint32_t c1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%10,%11};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(__uint_as_float(c0)), "f"(__uint_as_float(c1)));
}
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Codes I of the two 4-code chunks in w (one per half) times their scales: (64 + n) s - 72 s.
template <int I>
__device__ __forceinline__ uint32_t q4_pair(uint32_t w, uint32_t s, uint32_t b, uint32_t magic) {
  const uint32_t sh = I == 0 ? w << 4 : I == 1 ? w : I == 2 ? w >> 4 : w >> 8;
  uint32_t x, y;
  asm("lop3.b32 %0, %1, 0x00F000F0, %2, 0xEA;" : "=r"(x) : "r"(sh), "r"(magic));
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(y) : "r"(x), "r"(s), "r"(b));
  return y;
}
__device__ __forceinline__ uint32_t q4_times_m72(uint32_t s) {
  uint32_t y;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(y) : "r"(s), "r"(0xD480D480u));
  return y;
}

// Merge the state (m2, l2, acc2) into (m, l, acc), m in log2 units; -inf marks an empty state.
template <int E>
__device__ __forceinline__ void q4_merge_state(float& m, float& l, float (&acc)[E], float m2, float l2, const float (&acc2)[E]) {
  const float mn = fmaxf(m, m2);
  if (mn == -INFINITY) return;
  const float a = ex2_approx(m - mn), b = ex2_approx(m2 - mn);
  l = l * a + l2 * b;
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = acc[e] * a + acc2[e] * b;
  m = mn;
}

// A ring stage: codes of 32 keys, codes of 32 values, their scales, as they lie in memory but for the 16-byte vectors of a
// row of codes, which are permuted (vector ^ mask of the row) so that the eight rows an ldmatrix takes lie in different banks.
template <int D>
struct Q4Stage {
  static constexpr int kRow = D / 2, kScaleRow = D / 16;
  static constexpr int kV = kQ4Block * kRow;
  static constexpr int kKs = 2 * kV, kVs = kKs + kQ4Block * kScaleRow;
  static constexpr int kBytes = kVs + kQ4Block * kScaleRow;
  static __device__ __forceinline__ int swizzle(int row) { return D == 128 ? (row >> 1) & 3 : (row >> 2) & 1; }
};

// One warp's state over the keys of a pair.  A lane has columns 2 c4 and 2 c4 + 1 (heads; GP = 4: heads (2 c4) & 3 and the
// next: of P the first terms where c4 < 2, the second terms else) and keys r8, r8 + 8, ...; acc[4 p + i] holds channels 64 p + 4 r8 + i (of
// both columns) and, in its second pair, the channels 32 further.
template <int D, int GP>
struct Q4State {
  static constexpr int NG = D / 32;     // groups of a row
  static constexpr int NT = D / 16;     // 16-channel tiles of a value row
  static constexpr int NB = GP == 4 ? 2 : 4;
  // (Q itself lies in shared memory, a lane's B operand [group][b0, b1 of both k-steps] at q + 512 group + 16 lane.)
  // (behind it, for each c4: at 64 p the offsets -8 sum(q) of its columns in groups 2p and 2p + 1, at 64 NG / 2 their logits per sum)
  static constexpr int kOffsets = 512 * NG, kPerSum = 64 * (NG / 2), kQBytes = kOffsets + kPerSum + 64;
  float m[2];                           // largest logit so far (log2 units)
  uint64_t nm;                          // 14 - m, 0 before the first key
  uint64_t l;
  uint64_t acc[NT][2];

  __device__ __forceinline__ void clear() {
    m[0] = m[1] = -INFINITY;
    nm = l = 0ull;
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t][0] = acc[t][1] = 0ull;
  }

  // Q of a pair's heads, [G][D] at q, in fp16: a head's elements are scaled by a power of two that brings the largest to
  // [2^10, 2^11), which is exact down to 2^-24 of it, and 16 times that where the codes lie four bits lower.  A head that
  // holds an infinity or a NaN gets the factor NaN.
  __device__ __forceinline__ void load_q(const uint16_t* q, int G, float c, uint8_t* q_smem, int lane) {
    const int r8 = lane >> 2, c4 = lane & 3, head = GP == 4 ? r8 & 3 : r8;
    uint4 v[NG];
    uint32_t top = 0;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      v[g] = make_uint4(0, 0, 0, 0);
      if (head < G) v[g] = __ldcg(reinterpret_cast<const uint4*>(q + head * D + g * 32) + c4);
      const uint32_t w[4] = {v[g].x, v[g].y, v[g].z, v[g].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) top = max(top, max(w[i] & 0x7FFFu, (w[i] >> 16) & 0x7FFFu));
    }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const uint32_t e = top >> 7, up = min(264u - e, 254u);  // exponent fields: of the largest, of the factor 2^(137 - e)
    const float mul = __uint_as_float(up << 23);
    // 2^17: codes count as n 2^-17
    const float per_sum = e == 255u ? __uint_as_float(0x7FC00000u) : fminf(c * 131072.f * __uint_as_float((254u - up) << 23), 3.4e38f);
    float off[2][2];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const uint32_t w[4] = {v[g].x, v[g].y, v[g].z, v[g].w};
      float x[8], sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16) * mul;
        sum += x[i];
      }
      uint32_t b[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {  // channels i and i + 4, as the codes of a word pair up
        const float k = i & 1 ? 1.f : 16.f;
        const __half2 h = __floats2half2_rn(x[i] * k, x[i + 4] * k);
        b[i] = *reinterpret_cast<const uint32_t*>(&h);
      }
      *reinterpret_cast<uint4*>(q_smem + 512 * g + 16 * lane) = make_uint4(b[0], b[1], b[2], b[3]);
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);  // column r8's sum over the group
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      sum *= -8.f / 131072.f;
      off[g & 1][0] = __shfl_sync(0xffffffffu, sum, 8 * c4);
      off[g & 1][1] = __shfl_sync(0xffffffffu, sum, 8 * c4 + 4);
      if ((g & 1) && r8 == 0)
        *reinterpret_cast<float4*>(q_smem + kOffsets + 64 * (g / 2) + 16 * c4) = make_float4(off[0][0], off[0][1], off[1][0], off[1][1]);
    }
    const float2 ps = make_float2(__shfl_sync(0xffffffffu, per_sum, 8 * c4), __shfl_sync(0xffffffffu, per_sum, 8 * c4 + 4));
    if (r8 == 0) *reinterpret_cast<float2*>(q_smem + kOffsets + kPerSum + 16 * c4) = ps;
  }

  // The logits (log2 units) of keys r8 + 8 i of the 32 whose codes this lane's ldmatrix address is `codes` in, their scales at
  // `scales` (key r8).
  __device__ __forceinline__ void logits(uint64_t (&s)[4], uint32_t codes, uint32_t scales, uint32_t q, uint32_t offsets) {
    uint32_t sk[4][D / 64], per_sum[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) q4_lds<D / 16>(sk[i], scales + 8 * i * (D / 16));
#pragma unroll
    for (int p = 0; p < NG / 2; ++p) {
      uint32_t qb[2][4], of[4];
      q4_lds<16>(of, offsets + 64 * p);
      q4_lds<16>(qb[0], q + 1024 * p);
      q4_lds<16>(qb[1], q + 1024 * p + 512);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t w[4];
        ldmatrix_x4(w, (codes + h * 16 * Q4Stage<D>::kRow) ^ (p << 5));
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          const uint32_t l0 = w[2 * v] * 8u, l1 = w[2 * v + 1] * 8u, r0 = w[2 * v] >> 5, r1 = w[2 * v + 1] >> 5;
          const uint32_t a[4] = {l0 & 0x00780078u, l1 & 0x00780078u, l0 & 0x07800780u, l1 & 0x07800780u};
          const uint32_t b[4] = {r0 & 0x00780078u, r1 & 0x00780078u, r0 & 0x07800780u, r1 & 0x07800780u};
          float d[4];
          mma_f16_from(d, a, qb[v][0], qb[v][1], of[2 * v], of[2 * v + 1]);
          mma_f16(d, b, qb[v][2], qb[v][3]);
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const __half2 sc = *reinterpret_cast<const __half2*>(&sk[2 * h + k][p]);
            const float sf = v ? __high2float(sc) : __low2float(sc);
            const uint64_t d2 = f2_pack(d[2 * k], d[2 * k + 1]), sf2 = f2_pack(sf, sf);
            s[2 * h + k] = p == 0 && v == 0 ? f2_mul(d2, sf2) : f2_fma(d2, sf2, s[2 * h + k]);
          }
        }
      }
    }
    q4_lds<8>(per_sum, offsets + kPerSum);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = f2_mul(s[i], f2_pack(__uint_as_float(per_sum[0]), __uint_as_float(per_sum[1])));
  }

  uint32_t magic;                       // kQ4Magic

  // Keys kb .. kb + 31 (those at or past n do not count) in the ring stage; off: this lane's ldmatrix offset.
  __device__ __forceinline__ void block(uint32_t stage, uint32_t off, uint32_t q, int kb, int n, int lane) {
    using St = Q4Stage<D>;
    const int r8 = lane >> 2, c4 = lane & 3;
    uint64_t s[4];  // key r8 + 8 i, both columns
    logits(s, stage + off, stage + St::kKs + r8 * St::kScaleRow, q, q + kOffsets - 64 * r8);
    if (kb + kQ4Block > n) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (kb + 8 * i + r8 >= n) s[i] = f2_pack(-INFINITY, -INFINITY);
    }
    float t[2];
    {
      float x[4][2];
#pragma unroll
      for (int i = 0; i < 4; ++i) f2_unpack(s[i], x[i][0], x[i][1]);
#pragma unroll
      for (int e = 0; e < 2; ++e) t[e] = fmaxf(fmax3(x[0][e], x[1][e], x[2][e]), x[3][e]);
    }
    if (__any_sync(0xffffffffu, t[0] > m[0] || t[1] > m[1])) {
      float sc[2], k[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) t[e] = fmaxf(t[e], __shfl_xor_sync(0xffffffffu, t[e], o));
        const float mn = fmaxf(m[e], t[e]);
        sc[e] = m[e] == mn ? 1.f : ex2_approx(m[e] - mn);
        m[e] = mn;
        k[e] = mn == -INFINITY ? 0.f : kQ4WeightLog2 - mn;
      }
      nm = f2_pack(k[0], k[1]);
      const uint64_t sc2 = f2_pack(sc[0], sc[1]);
      l = f2_mul(l, sc2);
#pragma unroll
      for (int k = 0; k < NT; ++k) {
        acc[k][0] = f2_mul(acc[k][0], sc2);
        acc[k][1] = f2_mul(acc[k][1], sc2);
      }
    }
    const float take = GP == 4 && c4 < 2 ? 0.f : -1.f;
    const uint64_t minus_hi = f2_pack(take, take);
    uint32_t b[2][NB];  // B operand of P: [16 keys][b0, b1 (GP = 8: of both terms)]
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float p[2];
      f2_unpack(f2_add(s[i], nm), p[0], p[1]);
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
    // scales of keys 2 c4, 2 c4 + 1 (and 8 further) side by side
    uint32_t ss[2][2][NG];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint32_t w[D / 32];
        q4_lds<D / 8>(w, stage + St::kVs + (h * 16 + 8 * k + 2 * c4) * St::kScaleRow);
#pragma unroll
        for (int g = 0; g < NG; ++g) ss[h][k][g] = __byte_perm(w[g >> 1], w[NG / 2 + (g >> 1)], g & 1 ? 0x7632 : 0x5410);
      }
#pragma unroll
    for (int p = 0; p < NG / 2; ++p) {
      uint32_t w[2][4], sc[2][4], bi[2][4];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        ldmatrix_x4_trans(w[h], (stage + off + St::kV + h * 16 * St::kRow) ^ (p << 5));
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          sc[h][k] = ss[h][k & 1][2 * p + (k >> 1)];
          bi[h][k] = q4_times_m72(sc[h][k]);
        }
      }
      auto tile = [&](auto I) {
        constexpr int i = decltype(I)::value;
        float d[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t a[4] = {q4_pair<i>(w[h][0], sc[h][0], bi[h][0], magic), q4_pair<i>(w[h][2], sc[h][2], bi[h][2], magic),
                                 q4_pair<i>(w[h][1], sc[h][1], bi[h][1], magic), q4_pair<i>(w[h][3], sc[h][3], bi[h][3], magic)};
          if (h == 0) mma_f16_zero(d, a, b[h][NB - 2], b[h][NB - 1]);
          else mma_f16(d, a, b[h][NB - 2], b[h][NB - 1]);
          if (GP == 8) mma_f16(d, a, b[h][0], b[h][1]);
        }
        acc[4 * p + i][0] = f2_add(acc[4 * p + i][0], f2_pack(d[0], d[1]));
        acc[4 * p + i][1] = f2_add(acc[4 * p + i][1], f2_pack(d[2], d[3]));
      };
      tile(std::integral_constant<int, 0>{});
      tile(std::integral_constant<int, 1>{});
      tile(std::integral_constant<int, 2>{});
      tile(std::integral_constant<int, 3>{});
    }
  }

  // Written out: m and l of head g at ml[2 g], the values at vals + g * D.
  __device__ __forceinline__ void store(float* ml, float* vals, int G, int lane) {
    const int r8 = lane >> 2, c4 = lane & 3;
    float ls[2], x[NT][2][2];
    f2_unpack(l, ls[0], ls[1]);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int z = 0; z < 2; ++z) f2_unpack(acc[t][z], x[t][z][0], x[t][z][1]);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) ls[e] += __shfl_xor_sync(0xffffffffu, ls[e], o);
      const int head = 2 * c4 + e;
      const bool writes = head < G && (GP == 8 || c4 < 2);
#pragma unroll
      for (int p = 0; p < NG / 2; ++p)
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          float v[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[i] = x[4 * p + i][z][e];
            if (GP == 4) v[i] += __shfl_xor_sync(0xffffffffu, v[i], 2);
          }
          if (writes) *reinterpret_cast<float4*>(vals + head * D + 64 * p + 32 * z + 4 * r8) = make_float4(v[0], v[1], v[2], v[3]);
        }
      if (writes && r8 == 0) {
        ml[2 * head] = ls[e] == ls[e] ? m[e] : INFINITY;  // a NaN sum is not to be merged as an empty state
        ml[2 * head + 1] = ls[e];
      }
    }
  }
};

// A warp's blocks in the order it takes them: of each pair that the group's range touches, every W-th block.
struct Q4Cursor {
  int pair, layer, h;   // the pair at hand; layer == n_layers: none
  int blk, end;         // its next block for this warp, and where the range ends in it
  int left;             // blocks of the range from this pair's first one on
};

// RAGGED: a count for each cache.
template <int D, int GP, bool RAGGED>
__global__ void __launch_bounds__(kQ4DecThreads, kQ4DecCtasPerSm) q4_decode_kernel(const __grid_constant__ Q4DecodeArgs a) {
  using State = Q4State<D, GP>;
  using St = Q4Stage<D>;
  constexpr int kNoMore = -0x40000000;
  extern __shared__ __align__(128) uint8_t q4_smem[];  // per-warp rings, then per-warp states, then per-warp queries
  __shared__ Q4Lists s_list;  // RAGGED
  __shared__ float s_ml[kQ4DecWarps][2 * GP];
  __shared__ Q4Cursor s_cursor[kQ4DecWarps], s_here[kQ4DecWarps];  // where each warp's copies and its arithmetic are, out of its registers
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();
  pdl_launch_dependents();
  int n_all = 0, total;
  if constexpr (!RAGGED) {
    n_all = q4_keys(a, 0, blockIdx.x == 0 && threadIdx.x == 0);
    total = q4_blocks(n_all) * a.n_layers * a.Hkv;
  } else {
    if (warp == 0) q4_lists(a, s_list, blockIdx.x == 0);
    __syncthreads();
    total = s_list.first[a.n_layers];
  }
  auto keys_of = [&](int layer) { return RAGGED ? s_list.n[layer] : n_all; };
  auto blocks_of = [&](int layer) { return q4_blocks(keys_of(layer)); };
  const Q4Split sp = q4_split(a, !RAGGED, q4_blocks(n_all), total);
  const int W = a.whole ? a.whole : sp.W, rank = warp & (W - 1);
  const int group = W == 1 ? blockIdx.x * kQ4DecWarps + warp : blockIdx.x;
  float* s_vals = reinterpret_cast<float*>(q4_smem + kQ4DecWarps * kQ4Stages * St::kBytes);
  uint8_t* s_q = reinterpret_cast<uint8_t*>(s_vals + kQ4DecWarps * GP * D) + warp * State::kQBytes;
  const uint32_t ring = smem_u32(q4_smem + warp * kQ4Stages * St::kBytes), q_at = smem_u32(s_q) + 16 * lane;

  // the range and its first pair
  Q4Cursor ci;
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
    const int nb = q4_blocks(n_all);
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
        nb = q4_blocks(n_all);
        ci.pair = (unsigned)lo / (unsigned)nb;
        ci.layer = fdivmod(ci.pair, a.by_heads, ci.h);
        at = lo - ci.pair * nb;
      } else {
        ci.layer = 0;
        while (s_list.first[ci.layer + 1] <= lo) ++ci.layer;
        nb = blocks_of(ci.layer);
        at = lo - s_list.first[ci.layer];
        ci.h = (unsigned)at / (unsigned)nb;
        ci.pair = ci.layer * a.Hkv + ci.h;
        at -= ci.h * nb;
      }
      ci.blk = at;
      ci.left = hi - lo + at;
      ci.end = min(nb, ci.left);
    }
  }
  if (ci.layer == a.n_layers) return;  // whole groups
  if (lane == 0) s_here[warp] = ci;
  auto next_pair = [&](Q4Cursor& c) {
    c.left -= c.end;
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

  // copies: kQ4Stages blocks ahead of the arithmetic, across pairs
  constexpr int kVecRow = D / 32;  // 16-byte vectors of a row of codes
  const int cp_row = lane / kVecRow, cp_vec = lane & (kVecRow - 1);
  const uint32_t cp_dst = cp_row * St::kRow + ((cp_vec ^ St::swizzle(cp_row)) << 4);
  const uint8_t *Kc = nullptr, *Vc = nullptr, *Ks = nullptr, *Vs = nullptr;  // this lane's part of the next block
  auto bases = [&](const Q4Cursor& c) {
    const int64_t row = (int64_t)c.blk * kQ4Block;
    const int64_t code = c.h * a.code_head_stride + row * St::kRow + lane * 16;
    const int64_t scale = 2 * c.h * a.scale_head_stride + (row + lane) * St::kScaleRow;
    Kc = a.K[c.layer] + code;
    Vc = a.V[c.layer] + code;
    Ks = reinterpret_cast<const uint8_t*>(a.K_scale[c.layer]) + scale;
    Vs = reinterpret_cast<const uint8_t*>(a.V_scale[c.layer]) + scale;
  };
  // RAGGED: a pair of which the range holds a block or two is one warp's, the warps taking turns, and the others go on: the
  // short lists run side by side (24 caches of 1 to 8191 rows 15.7 -> 11.2 us).
  auto alone = [&](const Q4Cursor& c) { return RAGGED && c.end - c.blk <= kQ4Alone; };
  auto mine = [&](const Q4Cursor& c) { return !alone(c) || (c.pair & (W - 1)) == rank; };
  Q4Cursor& is = s_cursor[warp];
  // from the next block on: blocks of this warp left in the pair (<= 0: none), rows of the pair; from one block to the next:
  // rows, bytes of codes and of scales
  int ahead, rows, row_step, code_step, scale_step;
  auto enter = [&](Q4Cursor& c) {  // c: a pair's, its first block
    row_step = (alone(c) ? 1 : W) * kQ4Block;
    code_step = row_step * St::kRow;
    scale_step = row_step * St::kScaleRow;
    ahead = mine(c) ? c.end - c.blk : 0;
    if (!alone(c)) {
      c.blk += rank;
      ahead = (c.end - c.blk + W - 1) / W;
    }
    rows = keys_of(c.layer) - c.blk * kQ4Block;
    bases(c);
  };
  {
    Q4Cursor c = ci;
    enter(c);
    if (lane == 0) is = c;
    __syncwarp();
  }
  auto issue_next = [&](uint32_t dst) {
    if (ahead <= 0 && ahead > kNoMore / 2) {
      Q4Cursor c = is;
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
      const uint32_t d16 = dst + cp_dst, ds = dst + lane * St::kScaleRow;
      if (rows >= kQ4Block) {
#pragma unroll
        for (int i = 0; i < kVecRow; ++i) {
          q4_cp<16>(d16 + i * 512, Kc + i * 512);
          q4_cp<16>(d16 + St::kV + i * 512, Vc + i * 512);
        }
        q4_cp<St::kScaleRow>(ds + St::kKs, Ks);
        q4_cp<St::kScaleRow>(ds + St::kVs, Vs);
      } else {  // rows past the count: zeros, nothing is read
#pragma unroll 1
        for (int i = 0; i < kVecRow; ++i) {
          const int bytes = i * (32 / kVecRow) + cp_row < rows ? 16 : 0;
          q4_cp_part<16>(d16 + i * 512, Kc + i * 512, bytes);
          q4_cp_part<16>(d16 + St::kV + i * 512, Vc + i * 512, bytes);
        }
        const int bytes = lane < rows ? St::kScaleRow : 0;
        q4_cp_part<St::kScaleRow>(ds + St::kKs, Ks, bytes);
        q4_cp_part<St::kScaleRow>(ds + St::kVs, Vs, bytes);
      }
    }
    q4_cp_commit();
    --ahead;
    rows -= row_step;
    Kc += code_step;
    Vc += code_step;
    Ks += scale_step;
    Vs += scale_step;
  };
  issue_next(ring);

  const int lm_row = (lane & 7) + (lane & 8), lm_vec = lane >> 4;  // ldmatrix: keys 0-7 and 8-15 of a vector, then of the next
  const uint32_t off = lm_row * St::kRow + ((lm_vec ^ St::swizzle(lm_row)) << 4);
  State st;
  st.magic = a.magic;
  int stage = 0;
  bool fresh = true;
  for (;;) {
    __syncwarp();
    Q4Cursor ci = s_here[warp];
    const bool solo = alone(ci) || W == 1, my = mine(ci);
    if (my) {
      const int n = keys_of(ci.layer), step = (solo ? 1 : W) * kQ4Block, k_end = ci.end * kQ4Block;
      int kb = (ci.blk + (solo ? 0 : rank)) * kQ4Block;
      st.clear();
      if (kb < k_end) st.load_q(a.q[ci.layer] + (size_t)ci.h * a.G * D, a.G, a.c, s_q, lane);
      if (fresh) issue_next(ring + St::kBytes);  // (the first blocks of all warps go ahead of the second)
      fresh = false;
#pragma unroll 1
      for (; kb < k_end; kb += step) {
        q4_cp_wait<kQ4Stages - 1>();
        __syncwarp();
        st.block(ring + stage * St::kBytes, off, q_at, kb, n, lane);
        __syncwarp();
        issue_next(ring + stage * St::kBytes);
        stage = stage + 1 == kQ4Stages ? 0 : stage + 1;
      }
      ci = s_here[warp];
      const int first = ci.blk, G = a.G;
      st.store(s_ml[warp], s_vals + warp * GP * D, G, lane);
      auto sync_group = [&]() {
        if (solo) __syncwarp();
        else named_bar_sync(1, kQ4DecThreads);
      };
      sync_group();
      const int w0 = solo ? warp : 0, w1 = solo ? warp + 1 : kQ4DecWarps;
      const int t0 = solo ? lane : (int)threadIdx.x, t_step = solo ? 32 : kQ4DecThreads;
      const bool whole = first == 0 && ci.end == blocks_of(ci.layer);
      for (int t = t0; t < G * (D / 4); t += t_step) {
        const int g = t / (D / 4), e0 = (t - g * (D / 4)) * 4;
        float mm = -INFINITY, ll = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
        for (int w = w0; w < w1; ++w) {
          const float4 x = *reinterpret_cast<const float4*>(s_vals + (w * GP + g) * D + e0);
          const float v2[4] = {x.x, x.y, x.z, x.w};
          q4_merge_state<4>(mm, ll, v, s_ml[w][2 * g], s_ml[w][2 * g + 1], v2);
        }
        if (whole) {
          *reinterpret_cast<float4*>(a.out[ci.layer] + (size_t)(ci.h * G + g) * D + e0) =
              make_float4(v[0] / ll, v[1] / ll, v[2] / ll, v[3] / ll);
        } else {
          float* dst = a.part + ((size_t)(!RAGGED && sp.k > 0 ? group : group + ci.pair) * G + g) * (D + 4);
          if (e0 == 0) {
            dst[0] = mm;
            dst[1] = ll;
          }
          *reinterpret_cast<float4*>(dst + 4 + e0) = make_float4(v[0], v[1], v[2], v[3]);
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

// The partial states of a pair joined in key order, by NW warps a (pair, head).  Pairs that one range held whole are
// written already; those without keys are set to zero.
// Which slots a pair has follows from the counts, which are final once the kernel before has passed its own wait: they are
// read before this one's, as is the code that comes after it, run once with nothing to join (its blocks lie idle then).
// Many slots a pair: eight warps with eight slots each in flight (57 slots of 8 pairs: 10.6 -> 10.2 us a call, 228 of 2: 9.1 ->
// 8.3); some: four of four (8 layers 11.7 us, by one warp 12.5); few: a warp by itself, four in a block (64 layers x 8 heads x
// 1019 rows 25.4 -> 21.9 us, x 16000, G = 5, 224 -> 220: it is the number of blocks that costs).
template <int D, int NW>
__global__ void __launch_bounds__(NW == 1 ? 128 : NW * 32) q4_merge_kernel(const __grid_constant__ Q4DecodeArgs a) {
  constexpr int PER = D / 32, kInFlight = NW == 1 ? 4 : NW, kItems = NW == 1 ? 4 : 1;
  __shared__ Q4Lists s_list;
  __shared__ float s_ml[NW][2];
  __shared__ float s_v[NW][D];
  const int warp = NW == 1 ? 0 : threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int item = blockIdx.x * kItems + (NW == 1 ? threadIdx.x >> 5 : 0);
  const bool uniform = q4_uniform(a);
  if (!uniform) {
    if (threadIdx.x < 32) q4_lists(a, s_list, false);
    __syncthreads();
  }
  int g, h;
  const int pair = fdivmod(item, a.by_G, g), layer = fdivmod(pair, a.by_heads, h);
  if (layer >= a.n_layers) return;  // NW == 1: past the last pair
  int n, first, total;  // keys of the pair's cache, its first block in the list, all blocks
  if (uniform) {
    n = q4_keys(a, 0);
    first = layer * a.Hkv * q4_blocks(n);
    total = a.n_layers * a.Hkv * q4_blocks(n);
  } else {
    n = s_list.n[layer];
    first = s_list.first[layer];
    total = s_list.first[a.n_layers];
  }
  const int nb = q4_blocks(n);
  const Q4Split sp = q4_split(a, uniform, nb, total);
  int slot = 0, count = 0;
  if (nb > 0 && sp.k > 0) {
    slot = pair * sp.k;
    count = sp.k;
  } else if (nb > 0) {
    const int b0 = first + h * nb, g0 = (unsigned)b0 / (unsigned)sp.per;
    slot = g0 + pair;
    count = (unsigned)(b0 + nb - 1) / (unsigned)sp.per - g0 + 1;
  }
  float* out = a.out[layer] + (size_t)(h * a.G + g) * D;
#pragma unroll 1
  for (int live = count <= 1; live < 2; ++live) {
    if (live) {
      pdl_wait();
      pdl_launch_dependents();
      const int t = NW == 1 ? lane : threadIdx.x;
      if (nb == 0 && t < D / 4) reinterpret_cast<float4*>(out)[t] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (count <= 1) return;
    }
    float mm = -INFINITY, ll = 0.f, aa[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) aa[e] = 0.f;
#pragma unroll 1
    for (int i0 = warp; i0 < max(count, NW); i0 += kInFlight * NW) {
      float2 ml[kInFlight];
      float a2[kInFlight][PER];
#pragma unroll
      for (int u = 0; u < kInFlight; ++u) {
        const float* src = a.part + ((size_t)(slot + i0 + u * NW) * a.G + g) * (D + 4);
        const bool ok = live && i0 + u * NW < count;
        ml[u] = ok ? __ldcg(reinterpret_cast<const float2*>(src)) : make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int e = 0; e < PER; ++e) a2[u][e] = ok ? __ldcg(src + 4 + e * 32 + lane) : 0.f;
      }
#pragma unroll
      for (int u = 0; u < kInFlight; ++u) q4_merge_state<PER>(mm, ll, aa, ml[u].x, ml[u].y, a2[u]);
    }
    if constexpr (NW == 1) {
      if (live)
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
          q4_merge_state<1>(m1, l1, v1, s_ml[w][0], s_ml[w][1], v2);
        }
        if (live) out[threadIdx.x] = v1[0] / l1;
      }
      __syncthreads();
    }
  }
}

// A pair of n rows leaves at most one slot per block, and all pairs together at most one per group and pair.
size_t q4_decode_ws_bytes(int n_layers, int Hkv, int Hq, int d, int n_cap) {
  const int64_t pairs = (int64_t)n_layers * Hkv, blocks = pairs * (((int64_t)n_cap + kQ4Block - 1) / kQ4Block);
  return (size_t)(std::min<int64_t>(kQ4MaxGroups, blocks) + pairs) * (Hq / Hkv) * (d + 4) * sizeof(float);
}

// Warps that take a pair whole, which needs no partial states and no second kernel (1.5 to 4 us of a call), or 0; by the most
// blocks a pair can have (where the counts are on the device: by n_cap).  More pairs than CTAs, and short: a warp each (64 layers x 8 heads
// x 91 rows 8.8 -> 6.6 us, by a CTA each 8.6; at 16 blocks that was faster).  Else a CTA, while what its last wave leaves idle
// costs less than that kernel: a round (32 keys a warp) of an idle SM counts 0.4 of a busy one's time, and both sides met at
// 4 to 8 rounds (1 layer x 8 heads x 507 rows 6.6 -> 6.2 us, 763 rows 6.8 -> 7.4; 57 layers 94.5 -> 92.1 at 8272 rows).
// Counts that differ leave CTAs idle too, at worst all but one: 12 rounds (64 layers x 8 heads x up to 1531 rows 32 -> 22 us).
static int q4_whole(int pairs, int slots, int nb, bool ragged) {
  if (pairs > slots && nb <= 12) return 1;
  const int64_t rounds = (nb + kQ4DecWarps - 1) / kQ4DecWarps, idle = pairs % slots ? slots - pairs % slots : 0;
  return rounds * idle <= 6 * slots && !(ragged && rounds > 12) ? kQ4DecWarps : 0;
}

template <int D, int GP>
static cudaError_t q4_decode_launch(const Q4DecodeArgs& a, cudaStream_t stream) {
  void (*kern)(Q4DecodeArgs) =
      a.n_dev && a.n_stride && a.n_layers > 1 ? q4_decode_kernel<D, GP, true> : q4_decode_kernel<D, GP, false>;
  // (at least what lets no more than kQ4DecCtasPerSm on an SM: a fourth where registers allow one leaves other SMs without,
  // d = 64: 41 -> 51 us)
  const int smem = std::max(kQ4DecMinSmem, kQ4DecWarps * (kQ4Stages * Q4Stage<D>::kBytes + GP * D * (int)sizeof(float) + Q4State<D, GP>::kQBytes));
  cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(kern), smem);
  const int pairs = a.n_layers * a.Hkv;
  if (e == cudaSuccess) e = launch_kernel(kern, dim3(a.n_groups), dim3(kQ4DecThreads), smem, stream, a, true);
  if (e == cudaSuccess && !a.whole) {
    if (a.n_groups >= 16 * pairs) e = launch_kernel(q4_merge_kernel<D, 8>, dim3(pairs * a.G), dim3(256), 0, stream, a, true);
    else if (a.n_groups > 5 * pairs) e = launch_kernel(q4_merge_kernel<D, 4>, dim3(pairs * a.G), dim3(128), 0, stream, a, true);
    else e = launch_kernel(q4_merge_kernel<D, 1>, dim3((pairs * a.G + 3) / 4), dim3(128), 0, stream, a, true);
  }
  return e;
}

stepkv_status_t q4_decode_run(const stepkv_q4_cache_t& c, const void* const* q, int Hq, const int32_t* n_dev, int n_stride,
                              int n_host, int n_cap, float* const* out, void* ws, int32_t* status, cudaStream_t stream) {
  int n_sm = 0;
  cudaError_t e = device_sm_count(&n_sm);
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
    a.n_layers = nl;
    a.layer0 = l0;
    a.Hkv = c.Hkv;
    a.G = Hq / c.Hkv;
    // as many groups as run at once, none without a block
    const int64_t blocks = (int64_t)nl * c.Hkv * ((n_cap + kQ4Block - 1) / kQ4Block);
    const int slots = std::min(kQ4MaxGroups / kQ4DecWarps, n_sm * kQ4DecCtasPerSm);
    a.n_groups = (int)std::min<int64_t>(slots, blocks);
    a.whole = q4_whole(nl * c.Hkv, slots, ((n_dev ? n_cap : n_host) + kQ4Block - 1) / kQ4Block, n_dev && n_stride && nl > 1);
    if (a.whole) a.n_groups = (nl * c.Hkv * a.whole + kQ4DecWarps - 1) / kQ4DecWarps;
    for (int i = 0; i < 2; ++i) {
      const int groups = a.n_groups * (i ? kQ4DecWarps : 1);
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
    a.status = status;
    a.magic = kQ4Magic;
    if (c.d == 128)
      e = a.G <= 4 ? q4_decode_launch<128, 4>(a, stream) : q4_decode_launch<128, 8>(a, stream);
    else
      e = a.G <= 4 ? q4_decode_launch<64, 4>(a, stream) : q4_decode_launch<64, 8>(a, stream);
  }
  if (e == cudaSuccess) return STEPKV_OK;
  set_last_cuda_error(e);
  return STEPKV_ECUDA;
}

}  // namespace stepkv
