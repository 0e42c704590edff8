// What the decodes over narrow caches (4 bits, 8 bits) share: the list of all (cache, KV head) pairs' blocks of 32 keys and how
// it is cut into ranges for groups of warps, and the copies and tensor-core operations of a warp.
#pragma once

#include <stdint.h>

#include <algorithm>

#include "common.cuh"
#include "fastdiv.h"
#include "internal.h"

namespace stepkv {

constexpr int kListLayers = 64;     // caches of a launch (pointer arrays travel in the kernel parameters)
constexpr int kListWarps = 4;       // of a CTA: a group, unless the pairs are many and short
constexpr int kListBlock = 32;      // keys per warp step
constexpr int kListFew = 16;        // blocks of a pair that one CTA takes at once, though the pair might be cut
constexpr int kListAlone = 2;       // blocks of a pair that a warp takes by itself
constexpr int kListMaxGroups = 4096;  // workspace sizing: groups (single warps) of a launch at most

// The caches of a launch and the groups that take them.
struct DecodeList {
  int n_layers, layer0;
  int Hkv;
  int n_groups;     // CTAs
  // with groups of kListWarps warps, and of one: divisors groups and k = groups / pairs (1 where there are more pairs)
  FastDiv by_groups[2], by_k[2];
  FastDiv by_heads;
  const int32_t* n_dev;
  int n_stride;
  int n_host;
  int n_cap;
  int32_t* status;
};

// The keys of a cache of this launch.
__device__ __forceinline__ int list_keys(const DecodeList& a, int layer, bool tell = false) {
  if (!a.n_dev) return a.n_host;
  const int n = __ldcg(a.n_dev + (a.layer0 + layer) * a.n_stride);  // (the merge reads it early: not from L1)
  if (tell && n > a.n_cap) record_status(a.status, STEPKV_ENOSPACE);
  if (tell && n < 0) record_status(a.status, STEPKV_EDATA);
  return max(0, min(n, a.n_cap));
}

// Keys of every cache and the first block of each in the list of all pairs' blocks; first[n_layers]: all blocks.  By the
// first warp of a CTA; the caller synchronises.  Not used where all caches have one count.
// PAD: blocks without keys that each pair has behind its own in the list, for what a pair costs whatever its length: ranges of
// the same length then take the same time, whether they hold a few long pairs or many short ones.
struct ListCounts {
  int n[kListLayers];
  int first[kListLayers + 1];
};
__device__ __forceinline__ int list_blocks(int n) { return (n + kListBlock - 1) / kListBlock; }
__device__ __forceinline__ bool list_uniform(const DecodeList& a) { return !a.n_dev || a.n_stride == 0 || a.n_layers == 1; }
template <int PAD = 0>
__device__ __forceinline__ void list_counts(const DecodeList& a, ListCounts& s, bool tell) {
  const int lane = threadIdx.x & 31;
  int sum[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int l = 2 * lane + i;
    const int n = l < a.n_layers ? list_keys(a, l, tell) : 0;
    s.n[l] = n;
    sum[i] = n > 0 ? (list_blocks(n) + PAD) * a.Hkv : 0;
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
// then takes a range by itself instead of waiting for three others at its end.  (`total` is the list's, blocks without keys
// included: where every pair has 16 of these, as in the 8-bit decode of a ragged batch, it passes 16 * pairs unless a part of the
// caches is empty, so that only batches of mostly empty caches go to single warps there.)
struct ListSplit {
  int W, per, k;
};
__device__ __forceinline__ ListSplit list_split(const DecodeList& a, bool uniform, int nb, int total) {
  ListSplit p;
  const int pairs = a.n_layers * a.Hkv;
  const int single = pairs > a.n_groups && total <= 16 * pairs;
  p.W = single ? 1 : kListWarps;
  const FastDiv groups = a.by_groups[single], ks = a.by_k[single];
  p.per = fdiv(total + groups.d - 1, groups);
  p.k = 0;
  if (uniform && nb > 0 && pairs <= groups.d) {
    // rounded up to whole rounds: a part of one takes as long, and fewer ranges are joined faster
    const int per = fdiv(nb + ks.d - 1, ks), whole = (per + p.W - 1) & -p.W;
    if (!single && nb <= kListFew) {  // (14 layers x 8 heads x 379 rows 8.0 -> 7.0 us; at 24 blocks 9.6 and 9.1, or slower)
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
__device__ __forceinline__ void cp_async(uint32_t dst, const void* src) {
  if constexpr (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(N) : "memory");
}
template <int N>
__device__ __forceinline__ void cp_async_part(uint32_t dst, const void* src, int bytes) {
  if constexpr (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(N), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
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
__device__ __forceinline__ void lds(uint32_t (&w)[BYTES / 4], uint32_t addr) {
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

// Merge the state (m2, l2, acc2) into (m, l, acc), m in log2 units; -inf marks an empty state.
template <int E>
__device__ __forceinline__ void merge_state(float& m, float& l, float (&acc)[E], float m2, float l2, const float (&acc2)[E]) {
  const float mn = fmaxf(m, m2);
  if (mn == -INFINITY) return;
  const float a = ex2_approx(m - mn), b = ex2_approx(m2 - mn);
  l = l * a + l2 * b;
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = acc[e] * a + acc2[e] * b;
  m = mn;
}

// A warp's blocks in the order it takes them: of each pair that the group's range touches, every W-th block.
struct ListCursor {
  int pair, layer, h;   // the pair at hand; layer == n_layers: none
  int blk, end;         // its next block for this warp, and where the range ends in it
  int left;             // blocks of the range from this pair's first one on
};

}  // namespace stepkv
