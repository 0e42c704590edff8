// Eviction by accumulated attention: every (layer, KV head) keeps `keep` of its n rows, in place.
//   protected(j) = pos[j] < n_sink or pos[j] > max(pos) - n_recent
//   retained     = the first `keep` by (protected, mass descending, slot ascending)
//   the i-th slot below keep that goes receives the i-th slot at or above keep that stays
//
// A CTA takes a (layer, head): it finds the retained rows from n masses and positions, makes the list of moves, and moves masses
// and positions.  Where there are enough heads to fill the machine it moves the rows of keys and values too, in one launch;
// else a second kernel moves them over the whole machine.  In 8 bits a block that receives rows may have to take a larger scale.
//
// A row's rank is a 32-bit key: all ones where it is protected, else the mass as an integer that orders like the number (0 for
// a NaN).  Keys stay in registers, a warp's being consecutive slots (of 64 a thread: the 8-bit kernels of 20 and 32 keys a thread
// spill 2 to 5 words, the cluster kernels of 32 keys 17, in bf16 1).  The key T of the last retained row comes from histograms
// of 11, 11 and 10 bits, as many as it takes; with R(j) = min(rows below j that equal T, those of them that stay) + rows below
// j above T, the retained rows below slot j,
//   a slot j < keep that goes is number j - R(j) of those, a slot j >= keep that stays number R(j) - R(keep).
//
// 32 layers x 8 heads: 8273 to 8272 rows 13 us (positions 1.6, masses and the first histogram 3.1, its bin 0.7, counts 0.8, moves
// listed 1.6, done 1.2, of a CTA's 9), where the 16 MB that are read take 2.5; 32768 to 8272 in bf16 313 us, of which the moves of 1.7 GB
// are 254 at the copy rate: one CTA an SM, so that 104 heads wait for the first 152, and their search leaves DRAM idle.  Keys in shared
// memory instead of registers, with every pass over all of them: 24 and 393 us.
#include <cooperative_groups.h>
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "common.cuh"
#include "fastdiv.h"
#include "internal.h"
#include "q8.cuh"

namespace stepkv {

constexpr int kEvictLongThreads = 1024;    // of a head of more than kEvictShort rows
constexpr int kEvictShortThreads = 512;
constexpr int kEvictShort = 32 * kEvictShortThreads;  // (a thread holds 32 keys at most)
constexpr int kEvictLong = 32 * kEvictLongThreads;
constexpr int kEvictCluster = 8;           // CTAs of a head at most: as many as a cluster has without asking the device for more
static_assert(kEvictCluster * kEvictLong >= kEvictMaxRows, "every key has a place");
// Moves of a head held in shared memory at most (16 KB).  48 heads 2200 to 2048 rows: 7.6 us, 8.6 listed in the workspace; 256 heads
// 8911 to 8272 38.6 and 39.5, codes 45.7 and 47.8.  Two CTAs of an SM have room for some 10000; of longer lists the moves themselves are
// most of the time: 256 heads 11172 to 8272 109 us, 109 with 4096 and with 6144, codes 98, 94, 95; 14272 to 8272 169, 170, 168 and 140, 139,
// 130.
constexpr int kEvictSmemPlan = 2048;
constexpr uint32_t kEvictProtected = 0xFFFFFFFFu;

struct EvictArgs {
  float* mass[kQ8Layers];
  int32_t* pos[kQ8Layers];
  uint8_t* K[kQ8Layers];            // bf16 rows, or codes
  uint8_t* V[kQ8Layers];
  float* K_scale[kQ8Layers];        // 8 bits
  float* V_scale[kQ8Layers];
  int64_t mass_stride, pos_stride, head_bytes, scale_stride;
  int layer0, n_layers, Hkv;
  int row_bytes;
  const int32_t* n_dev;
  int n_stride, n_host, n_cap, keep, n_sink, n_recent;
  int cluster;      // CTAs of a head
  int moves_rows;   // this launch moves keys and values
  int32_t* n_out;   // NULL: not this launch
  // workspace, per (layer, head):
  int2* plan;       // [plan_cap]: (slot filled, slot it is filled from), both ascending
  int2* blocks;     // [block_cap], 8 bits: (block, number of its first move * 64 + moves) of blocks that receive rows, in any order
  int2* counts;     // (moves, blocks that receive rows)
  float2* cut;      // 8 bits: the scales (K, V) of the block that `keep` cuts
  int plan_cap, block_cap;
  int smem_plan;    // moves held in shared memory (plan_cap), 0: in the workspace
  int32_t* status;
};
static_assert(sizeof(EvictArgs) <= 32000, "kernel parameter space");

__device__ __forceinline__ uint32_t evict_key(float mass, int pos, int n_sink, int64_t recent) {
  if (pos < n_sink || pos > recent) return kEvictProtected;
  return mass == mass ? float_to_ordered(mass + 0.f) : 0u;  // (-0 + 0 is 0)
}

// The bin of the histogram (2048 bins, counted from the top) in which the `ties`-th key lies, and its number there; `count`: the
// keys of that bin.  All threads get them; one barrier, after the counting's.
template <int NT>
__device__ __forceinline__ uint32_t evict_bin(const uint32_t* hist, uint32_t* s_total, uint32_t& ties, uint32_t& count) {
  constexpr int NW = NT / 32, BPL = 2048 / NT, SEG = 32 * BPL;  // bins a lane, a warp
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t sum = 0;
#pragma unroll
  for (int i = 0; i < BPL; ++i) sum += hist[warp * SEG + i * 32 + lane];
  sum = __reduce_add_sync(0xffffffffu, sum);
  if (lane == 0) s_total[warp] = sum;
  __syncthreads();
  // (every warp by itself from here on) the warp's part, from the top
  uint32_t t = lane < NW ? s_total[NW - 1 - lane] : 0u, upto = t;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += y;
  }
  const int at = __ffs(__ballot_sync(0xffffffffu, upto >= ties)) - 1;
  ties -= __shfl_sync(0xffffffffu, upto - t, at);
  const int seg = NW - 1 - at;
  // its bins, 32 at a time from the top
  uint32_t bin = 0;
  count = 0;
#pragma unroll
  for (int i = BPL - 1; i >= 0; --i) {
    if (count) continue;
    t = hist[seg * SEG + i * 32 + 31 - lane];
    upto = t;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += y;
    }
    const uint32_t hit = __ballot_sync(0xffffffffu, upto >= ties);
    if (hit) {
      const int l = __ffs(hit) - 1;
      ties -= __shfl_sync(0xffffffffu, upto - t, l);
      count = __shfl_sync(0xffffffffu, t, l);
      bin = seg * SEG + i * 32 + 31 - l;
    } else {
      ties -= __shfl_sync(0xffffffffu, upto, 31);
    }
  }
  return bin;
}

// Rows of bf16 by one CTA, 16 bytes a lane.
template <int NT>
__device__ __forceinline__ void evict_move_rows(const EvictArgs& a, const int2* plan, int moves, int layer, int h) {
  constexpr int U = 4;
  const int lpr = a.row_bytes >> 4, rpi = 32 / lpr;  // lanes a row, rows an instruction
  const int lane = threadIdx.x & 31, sub = lane / lpr, col = lane - sub * lpr;
  const int per_chunk = rpi * U, chunks = (moves + per_chunk - 1) / per_chunk;
  for (int c = threadIdx.x >> 5; c < 2 * chunks; c += NT / 32) {
    const bool v_rows = c >= chunks;
    const int i0 = (v_rows ? c - chunks : c) * per_chunk + sub;
    uint8_t* rows = (v_rows ? a.V : a.K)[layer] + h * a.head_bytes + col * 16;
    int2 p[U];
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      p[u] = make_int2(-1, -1);
      if (sub < rpi && i0 + u * rpi < moves) p[u] = plan[i0 + u * rpi];
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (p[u].y >= 0) v[u] = q8_ld_stream(rows + (int64_t)p[u].y * a.row_bytes);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (p[u].x >= 0) q8_st_stream(rows + (int64_t)p[u].x * a.row_bytes, v[u]);
  }
}

// The largest magnitude of 16 codes (NaN does not count), as a code.
__device__ __forceinline__ uint32_t evict_top_code(const uint4& v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t top = 0;  // magnitudes order as integers
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t m = w[i] & 0x7F7F7F7Fu;
    top = __vmaxu4(top, m & ~__vcmpeq4(m, 0x7F7F7F7Fu));
  }
  return max(max(top & 0xFFu, top >> 8 & 0xFFu), max(top >> 16 & 0xFFu, top >> 24));
}
// The rows of a block that lie below keep (those at or past it are only read), a bit each.
__device__ __forceinline__ uint32_t evict_rows_below(int keep, int block) {
  const int rows = keep - block * kQ8Block;
  return rows >= kQ8Block ? 0xFFFFFFFFu : (1u << rows) - 1u;
}

// Rows of an 8-bit cache by one CTA: what the blocks need of the rows they receive, then their scales, then the rows.  A block
// can only have to grow for a row of a larger scale than its own, so that few rows are looked at twice.
// s_scale: [2][blocks], zeroed; s_holes: the slots of each block that are filled; cut: the scales of the block that `keep` cuts.
template <int D, int NT>
__device__ __forceinline__ void evict_move_codes(const EvictArgs& a, const int2* plan, int moves, int layer, int h, float* s_scale,
                                                 const uint32_t* s_holes, const float (&cut)[2]) {
  constexpr int LPR = D / 16, RPI = 32 / LPR, U = 4, kChunk = RPI * U;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane / LPR, col = lane & (LPR - 1);
  const int nblk = (a.keep + kQ8Block - 1) / kQ8Block;
  const int cut_block = a.keep % kQ8Block ? a.keep / kQ8Block : -1;
  const int tests = (moves + 31) / 32;
  for (int c = warp; c < 2 * tests; c += NT / 32) {
    const int z = c >= tests, i = (z ? c - tests : c) * 32 + lane;
    uint8_t* rows = (z ? a.V : a.K)[layer] + h * a.head_bytes + col * 16;
    const float* scale = (z ? a.V_scale : a.K_scale)[layer] + h * a.scale_stride;
    int2 p = make_int2(0, 0);
    float from = 0.f, old = 0.f;
    if (i < moves) {
      p = plan[i];
      from = __ldcg(scale + p.y / kQ8Block);  // (no scale changes before the barrier)
      old = __ldcg(scale + p.x / kQ8Block);
    }
    const uint32_t larger = __ballot_sync(0xffffffffu, from > old);
    if (!larger) continue;
#pragma unroll 1
    for (int k0 = 0; k0 < LPR; k0 += U) {  // (LPR instructions cover the 32 rows)
      uint4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int row = (k0 + u) * RPI + sub, y = __shfl_sync(0xffffffffu, p.y, row);
        v[u] = make_uint4(0, 0, 0, 0);
        if (larger >> row & 1u) v[u] = __ldcg(reinterpret_cast<const uint4*>(rows + (int64_t)y * D));
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int row = (k0 + u) * RPI + sub, x = __shfl_sync(0xffffffffu, p.x, row);
        float most = q8_float2(evict_top_code(v[u])).x * __shfl_sync(0xffffffffu, from, row);
#pragma unroll
        for (int o = 1; o < LPR; o <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        if (col == 0 && (larger >> row & 1u))  // (positive numbers order as integers)
          atomicMax(reinterpret_cast<unsigned*>(s_scale) + z * nblk + x / kQ8Block, __float_as_uint(most));
      }
    }
  }
  __syncthreads();
  // the blocks' scales; where one grows, the rows that stay
  for (int i0 = warp * 32; i0 < 2 * nblk; i0 += NT) {
    const int i = i0 + lane, z = i >= nblk, b = z ? i - nblk : i;
    float old = 0.f, s = 0.f;
    if (i < 2 * nblk && s_holes[b]) {
      float* scale = (z ? a.V_scale : a.K_scale)[layer] + h * a.scale_stride + b;
      old = __ldcg(scale);
      s = fmaxf(old, q8_scale(s_scale[i]));
      s_scale[i] = s;
      if (old < s) *scale = s;
    }
    uint32_t grows = __ballot_sync(0xffffffffu, old < s);
    while (grows) {
      const int l = __ffs(grows) - 1, k = i0 + l, y = k >= nblk, block = y ? k - nblk : k;
      grows &= grows - 1;
      const float ratio = __shfl_sync(0xffffffffu, old, l) * q8_inverse(__shfl_sync(0xffffffffu, s, l));
      q8_rescale_rows<D, 4>((y ? a.V : a.K)[layer] + h * a.head_bytes + (int64_t)block * (kQ8Block * D),
                         evict_rows_below(a.keep, block) & ~s_holes[block], ratio);
    }
  }
  __syncthreads();
  const int chunks = (moves + kChunk - 1) / kChunk;
  for (int c = warp; c < 2 * chunks; c += NT / 32) {
    const int z = c >= chunks;
    const int i0 = (z ? c - chunks : c) * kChunk + sub;
    uint8_t* rows = (z ? a.V : a.K)[layer] + h * a.head_bytes + col * 16;
    const float* scale = (z ? a.V_scale : a.K_scale)[layer] + h * a.scale_stride;
    int2 p[U];
    uint4 v[U];
    float from[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      p[u] = make_int2(-1, -1);
      if (i0 + u * RPI < moves) p[u] = plan[i0 + u * RPI];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (p[u].y < 0) continue;
      const int b = p[u].y / kQ8Block;
      v[u] = q8_ld_stream(rows + (int64_t)p[u].y * D);
      from[u] = b == cut_block ? cut[z] : __ldcg(scale + b);  // (that block's scale may have grown)
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (p[u].x < 0) continue;
      const float s = s_scale[z * nblk + p[u].x / kQ8Block];
      if (from[u] != s) v[u] = q8_rescale(v[u], from[u] * q8_inverse(s));
      *reinterpret_cast<uint4*>(rows + (int64_t)p[u].x * D) = v[u];
    }
  }
}

// min(n, keep) of this launch's layers, where n_out is not what the launch's CTAs read n from.
__device__ __forceinline__ void evict_counts(const EvictArgs& a, int threads) {
  if (!a.n_out || blockIdx.x != 0) return;
  const bool each = a.n_dev && a.n_stride;
  for (int l = threadIdx.x; l < (each ? a.n_layers : 1); l += threads) {
    const int at = each ? a.layer0 + l : 0;
    const int n = a.n_dev ? __ldcg(a.n_dev + at) : a.n_host;
    if (n >= 0 && n <= a.n_cap) a.n_out[at] = min(n, a.keep);
  }
}
__global__ void evict_counts_kernel(const __grid_constant__ EvictArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  evict_counts(a, blockDim.x);
}

namespace cg = cooperative_groups;

// DQ: 0: bf16, else the channels of a row of codes.  R: groups of 32 slots that a warp has at most.  CL: a cluster of CTAs takes the
// head, each a part of its slots; maxima, histograms and counts meet through distributed shared memory.
template <int DQ, int NT, int R, bool CL>
__global__ void __launch_bounds__(NT, NT == kEvictShortThreads ? 2 : 1) evict_select_kernel(const __grid_constant__ EvictArgs a) {
  constexpr int NW = NT / 32;
  constexpr bool Q8 = DQ != 0;
  extern __shared__ __align__(8) uint32_t s_dyn[];  // moves; 8 bits: [2][blocks] scales, [blocks] holes
  __shared__ uint32_t s_hist[3][2048];
  __shared__ uint32_t s_sum[CL ? 2048 : 1];         // a histogram of all the cluster's CTAs
  __shared__ uint32_t s_total[2][NW];
  __shared__ uint2 s_count[NW];
  __shared__ uint32_t s_blocks;
  __shared__ uint32_t s_top, s_safe;                // CL: what this CTA tells the others, each written once
  __shared__ uint4 s_part;
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int C = CL ? a.cluster : 1, pair = CL ? blockIdx.x / C : blockIdx.x, rank = blockIdx.x - pair * C;
  const int layer = pair / a.Hkv, h = pair - layer * a.Hkv;
  const int keep = a.keep, nblk = Q8 && a.moves_rows ? (keep + kQ8Block - 1) / kQ8Block : 0;
  for (int i = t; i < 3 * 2048; i += NT) s_hist[0][i] = 0;
  uint32_t* s_scale = s_dyn + 2 * a.smem_plan;
  for (int i = t; i < 2 * nblk; i += NT) s_scale[i] = 0;
  uint32_t* s_holes = s_scale + 2 * nblk;
  if (t == 0) s_blocks = 0;
  pdl_wait();
  pdl_launch_dependents();
  evict_counts(a, NT);
  int n = a.n_host;
  if (a.n_dev) {
    n = __ldcg(a.n_dev + (a.layer0 + layer) * a.n_stride);
    if (n < 0 || n > a.n_cap) {
      if (t == 0) record_status(a.status, n < 0 ? STEPKV_EDATA : STEPKV_ENOSPACE);
      n = 0;
    }
  }
  if (n <= keep) {  // (the whole cluster)
    if (t == 0 && rank == 0) a.counts[pair] = make_int2(0, 0);
    return;
  }
  auto meet = [&] {
    if constexpr (CL) cg::this_cluster().sync();
    else __syncthreads();
  };
  auto peer = [&](auto* p, int r) { return cg::this_cluster().map_shared_rank(p, r); };
  float* mass = a.mass[layer] + (int64_t)h * a.mass_stride;
  int32_t* pos = a.pos[layer] + (int64_t)h * a.pos_stride;
  // groups of 32 slots: this CTA's, of which warp w has `per` from g0 on
  const int all = (n + 31) / 32, part = (all + C - 1) / C, c0 = rank * part, c1 = min(all, c0 + part);
  const int per = (part + NW - 1) / NW, g0 = c0 + warp * per, rounds = max(0, min(c1 - g0, per));
  const int first = g0 * 32 + lane;
  uint32_t keys[R];

  int top = INT_MIN;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    keys[r] = (uint32_t)INT_MIN;
    if (r < rounds && first + r * 32 < n) keys[r] = (uint32_t)__ldcg(pos + first + r * 32);
  }
#pragma unroll
  for (int r = 0; r < R; ++r) top = max(top, (int)keys[r]);
  top = __reduce_max_sync(0xffffffffu, top);
  if (lane == 0) s_total[0][warp] = (uint32_t)top;
  __syncthreads();
  top = __reduce_max_sync(0xffffffffu, (int)s_total[0][lane & (NW - 1)]);
  if constexpr (CL) {
    if (t == 0) s_top = (uint32_t)top;
    meet();
    top = __reduce_max_sync(0xffffffffu, lane < C ? (int)*peer(&s_top, lane) : INT_MIN);
  }
  const int64_t recent = (int64_t)top - a.n_recent;
  uint32_t safe = 0;
  constexpr int kBatch = R < 8 ? R : 8;
#pragma unroll
  for (int r0 = 0; r0 < R; r0 += kBatch) {
    asm volatile("" ::: "memory");  // (a batch's loads at a time: all at once take another register a group)
    float m[kBatch];
#pragma unroll
    for (int r = 0; r < kBatch; ++r) {
      m[r] = 0.f;
      if (r0 + r < R && r0 + r < rounds && first + (r0 + r) * 32 < n) m[r] = __ldcg(mass + first + (r0 + r) * 32);
    }
#pragma unroll
    for (int r = 0; r < kBatch; ++r)
      if (r0 + r < R) keys[r0 + r] = first + (r0 + r) * 32 < n ? evict_key(m[r], (int)keys[r0 + r], a.n_sink, recent) : 0u;
  }
  // f(key, slot, slot < n) for this lane's slots, the whole warp at once; keys of slots behind the last are 0
  auto each = [&](auto f) {
    int at = first;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r < rounds) {
        if (R > 20 && r) {  // (slots known ahead push keys out of the registers: 32768 to 8272 rows 332 us)
          at += 32;
          asm volatile("" : "+r"(at));
        }
        const int j = R > 20 ? at : first + r * 32;
        f(keys[r], j, j < n);
      }
    }
  };
  // a histogram of all the head's keys, complete and counted in
  auto counted = [&](uint32_t* hist) -> const uint32_t* {
    meet();
    if constexpr (CL) {
      for (int i = t; i < 2048; i += NT) {
        uint32_t x = 0;
        for (int r = 0; r < C; ++r) x += peer(hist, r)[i];
        s_sum[i] = x;
      }
      __syncthreads();
      return s_sum;
    }
    return hist;
  };
  // the first histogram, and the protected rows
  each([&](uint32_t k, int, bool in) {
    const bool p = in && k == kEvictProtected;
    safe += p;
    if (in && !p) atomicAdd(&s_hist[0][k >> 21], 1u);
  });
  safe = __reduce_add_sync(0xffffffffu, safe);
  if (lane == 0) s_total[1][warp] = safe;
  if constexpr (CL) {
    __syncthreads();
    safe = __reduce_add_sync(0xffffffffu, lane < NW ? s_total[1][lane] : 0u);
    if (t == 0) s_safe = safe;
  }
  const uint32_t* hist = counted(s_hist[0]);
  if constexpr (CL) safe = __reduce_add_sync(0xffffffffu, lane < C ? *peer(&s_safe, lane) : 0u);
  else safe = __reduce_add_sync(0xffffffffu, lane < NW ? s_total[1][lane] : 0u);

  // the last retained row's key T under a mask, and how many of those that equal it stay
  uint32_t T = kEvictProtected, mask = 0xFFFFFFFFu, ties = keep, count = safe;
  if ((int)safe < keep) {
    ties = keep - safe;
    T = evict_bin<NT>(hist, s_total[0], ties, count) << 21;
    mask = 0xFFE00000u;
    if (ties < count) {
      each([&](uint32_t k, int, bool in) {
        if (in && (k & mask) == T) atomicAdd(&s_hist[1][k >> 10 & 2047u], 1u);
      });
      hist = counted(s_hist[1]);
      T |= evict_bin<NT>(hist, s_total[1], ties, count) << 10;
      mask = 0xFFFFFC00u;
    }
    if (ties < count) {
      each([&](uint32_t k, int, bool in) {
        if (in && (k & mask) == T) atomicAdd(&s_hist[2][k & 1023u], 1u);
      });
      hist = counted(s_hist[2]);
      T |= evict_bin<NT>(hist, s_total[0], ties, count);
      mask = 0xFFFFFFFFu;
    }
  }
  // Rows above T, and equal to it under the mask: of each warp's slots, and of those below keep.  (No key but a protected row's
  // reaches 0xFFE00000, so that one stays above a T under any mask.)  Where all that equal T stay, a row stays if its key is
  // not below T, and the slots behind the last, whose keys are 0, do not count.
  const bool all_equal = ties >= count && T != 0;
  uint32_t here = 0, low = 0;  // above + 2^16 equal
  each([&](uint32_t k, int j, bool in) {
    uint32_t x;
    if (all_equal) x = k >= T;
    else x = in && (k & mask) > T ? 1u : in && (k & mask) == T ? 65536u : 0u;
    here += x;
    if (j < keep) low += x;
  });
  const uint32_t below = (1u << lane) - 1u;
  here = __reduce_add_sync(0xffffffffu, here);
  low = __reduce_add_sync(0xffffffffu, low);
  if (lane == 0) s_count[warp] = make_uint2(here, low);
  __syncthreads();
  const uint2 mine = lane < NW ? s_count[lane] : make_uint2(0, 0);
  uint32_t gt0 = __reduce_add_sync(0xffffffffu, lane < warp ? mine.x & 0xFFFFu : 0u);
  uint32_t eq0 = __reduce_add_sync(0xffffffffu, lane < warp ? mine.x >> 16 : 0u);
  uint32_t gt_low = __reduce_add_sync(0xffffffffu, mine.y & 0xFFFFu), eq_low = __reduce_add_sync(0xffffffffu, mine.y >> 16);
  if constexpr (CL) {
    const uint32_t gt = __reduce_add_sync(0xffffffffu, mine.x & 0xFFFFu), eq = __reduce_add_sync(0xffffffffu, mine.x >> 16);
    if (t == 0) s_part = make_uint4(gt, eq, gt_low, eq_low);
    meet();
    const uint4 other = lane < C ? *peer(&s_part, lane) : make_uint4(0, 0, 0, 0);
    gt0 += __reduce_add_sync(0xffffffffu, lane < rank ? other.x : 0u);
    eq0 += __reduce_add_sync(0xffffffffu, lane < rank ? other.y : 0u);
    gt_low = __reduce_add_sync(0xffffffffu, other.z);
    eq_low = __reduce_add_sync(0xffffffffu, other.w);
  }
  const int kept_low = gt_low + min(eq_low, ties), moves = keep - kept_low;
  int2* plan = a.smem_plan ? reinterpret_cast<int2*>(s_dyn) : a.plan + (int64_t)pair * a.plan_cap;
  int2* blocks = a.blocks + (int64_t)pair * a.block_cap;
  each([&](uint32_t k, int j, bool in) {
    bool stays;
    int kept;  // R(j)
    if (all_equal) {
      stays = k >= T;
      const uint32_t ge = __ballot_sync(0xffffffffu, stays);
      kept = gt0 + __popc(ge & below);
      gt0 += __popc(ge);
    } else {
      const uint32_t gt = __ballot_sync(0xffffffffu, in && (k & mask) > T), eq = __ballot_sync(0xffffffffu, in && (k & mask) == T);
      const uint32_t eqb = eq0 + __popc(eq & below);
      stays = (gt >> lane & 1u) || ((eq >> lane & 1u) && eqb < ties);
      kept = gt0 + __popc(gt & below) + min(eqb, ties);
      gt0 += __popc(gt);
      eq0 += __popc(eq);
    }
    const bool hole = j < keep && !stays;
    if (hole) plan[j - kept].x = j;
    if (j >= keep && stays) plan[kept - kept_low].y = j;
    if (Q8) {
      const uint32_t holes = __ballot_sync(0xffffffffu, hole);
      if (lane == 0 && j < keep) {
        if (a.moves_rows) s_holes[j / kQ8Block] = holes;
        else if (holes)
          blocks[atomicAdd(CL ? peer(&s_blocks, 0) : &s_blocks, 1u)] = make_int2(j / kQ8Block, (j - kept) * 64 + __popc(holes));
      }
    }
  });
  float cut[2] = {0.f, 0.f};
  if (Q8 && keep % kQ8Block) {
    cut[0] = __ldcg(a.K_scale[layer] + (int64_t)h * a.scale_stride + keep / kQ8Block);
    cut[1] = __ldcg(a.V_scale[layer] + (int64_t)h * a.scale_stride + keep / kQ8Block);
  }
  meet();
  if (t == 0 && rank == 0 && !a.moves_rows) {
    a.counts[pair] = make_int2(moves, s_blocks);
    if (Q8) a.cut[pair] = make_float2(cut[0], cut[1]);
  }
  for (int i = rank * NT + t; i < moves; i += C * NT) {
    const int2 p = CL ? __ldcg(plan + i) : plan[i];
    mass[p.x] = __ldcg(mass + p.y);
    pos[p.x] = __ldcg(pos + p.y);
  }
  meet();
  for (int j = keep + rank * NT + t; j < n; j += C * NT) mass[j] = 0.f;
  if (!CL && a.moves_rows) {
    if constexpr (Q8) evict_move_codes<DQ, NT>(a, plan, moves, layer, h, reinterpret_cast<float*>(s_scale), s_holes, cut);
    else evict_move_rows<NT>(a, plan, moves, layer, h);
  }
}

struct EvictMoveArgs {
  uint8_t* rows[2 * kQ8Layers];  // per (layer, tensor): bf16 rows, or codes
  float* scale[2 * kQ8Layers];   // 8 bits
  int64_t head_bytes, scale_stride;
  FastDiv by_heads;
  int sets;                      // layers * 2 * Hkv
  int Hkv, n_layers, layer0;
  int row_bytes;
  int keep, plan_cap, block_cap;
  const int2* plan;
  const int2* blocks;
  const int2* counts;
  const float2* cut;
  const int32_t* n_dev;          // the counts, for n_out
  int n_stride, n_host, n_cap;
  int32_t* n_out;                // NULL: not this launch
};
static_assert(sizeof(EvictMoveArgs) <= 32000, "kernel parameter space");

// min(n, keep) of this launch's layers.  (n_out may be n_dev: nothing else reads it here.)
__device__ __forceinline__ void evict_move_counts(const EvictMoveArgs& a) {
  if (!a.n_out || blockIdx.x != 0) return;
  const bool each = a.n_dev && a.n_stride;
  for (int l = threadIdx.x; l < (each ? a.n_layers : 1); l += blockDim.x) {
    const int at = each ? a.layer0 + l : 0;
    const int n = a.n_dev ? __ldcg(a.n_dev + at) : a.n_host;
    if (n >= 0 && n <= a.n_cap) a.n_out[at] = min(n, a.keep);
  }
}

constexpr int kEvictMoveUnroll = 4;

// bf16: a warp takes chunks of a head's moves, 16 bytes a lane.
__global__ void __launch_bounds__(kQ8Threads) evict_move_kernel(const __grid_constant__ EvictMoveArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  evict_move_counts(a);
  if (a.plan_cap == 0) return;  // no head can have more than `keep`
  const int lpr = a.row_bytes >> 4, rpi = 32 / lpr;  // lanes a row, rows an instruction
  const int lane = threadIdx.x & 31, sub = lane / lpr, col = lane - sub * lpr;
  const int per_chunk = rpi * kEvictMoveUnroll;
  for (Q8Chunks c((a.plan_cap + per_chunk - 1) / per_chunk, a.sets); c.any(); c.next()) {
    int h;
    const int lt = fdivmod(c.set, a.by_heads, h), pair = (lt >> 1) * a.Hkv + h;
    const int moves = __ldcg(&a.counts[pair].x);
    if (c.pos * per_chunk >= moves) continue;
    const int2* plan = a.plan + (int64_t)pair * a.plan_cap;
    uint8_t* rows = a.rows[lt] + h * a.head_bytes + col * 16;
    int2 p[kEvictMoveUnroll];
    uint4 v[kEvictMoveUnroll];
#pragma unroll
    for (int u = 0; u < kEvictMoveUnroll; ++u) {
      const int i = c.pos * per_chunk + u * rpi + sub;
      p[u] = make_int2(-1, -1);
      if (sub < rpi && i < moves) p[u] = __ldcg(plan + i);
    }
#pragma unroll
    for (int u = 0; u < kEvictMoveUnroll; ++u)
      if (p[u].y >= 0) v[u] = q8_ld_stream(rows + (int64_t)p[u].y * a.row_bytes);
#pragma unroll
    for (int u = 0; u < kEvictMoveUnroll; ++u)
      if (p[u].x >= 0) q8_st_stream(rows + (int64_t)p[u].x * a.row_bytes, v[u]);
  }
}

// 8 bits: a warp takes a block that receives rows: all of them in registers (16 bytes a lane, 32 at d = 128), the scale they
// need, the codes of the rows that stay if the scale grows, and theirs.
template <int D>
__global__ void __launch_bounds__(kQ8Threads) evict_q8_move_kernel(const __grid_constant__ EvictMoveArgs a) {
  constexpr int LPR = D / 16, RPI = 32 / LPR, NI = kQ8Block / RPI;
  pdl_wait();
  pdl_launch_dependents();
  evict_move_counts(a);
  if (a.block_cap == 0) return;  // no head can have more than `keep`
  const int lane = threadIdx.x & 31, sub = lane / LPR, col = lane & (LPR - 1);
  for (Q8Chunks c(a.block_cap, a.sets); c.any(); c.next()) {
    int h;
    const int lt = fdivmod(c.set, a.by_heads, h), pair = (lt >> 1) * a.Hkv + h;
    if (c.pos >= __ldcg(&a.counts[pair].y)) continue;
    const int2 entry = __ldcg(a.blocks + (int64_t)pair * a.block_cap + c.pos);
    const int block = entry.x, moves = entry.y & 63;
    const int2* plan = a.plan + (int64_t)pair * a.plan_cap + (entry.y >> 6);
    uint8_t* codes = a.rows[lt] + h * a.head_bytes;
    float* scale = a.scale[lt] + h * a.scale_stride;
    // lane i: move i
    int2 p = make_int2(-1, -1);
    float from = 0.f;
    if (lane < moves) {
      p = __ldcg(plan + lane);
      const int b = p.y / kQ8Block;
      if (a.keep % kQ8Block && b == a.keep / kQ8Block) {  // (that block's scale may be growing: as it was before the moves)
        const float2 cut = __ldcg(a.cut + pair);
        from = lt & 1 ? cut.y : cut.x;
      } else {
        from = __ldcg(scale + b);
      }
    }
    const uint32_t filled = __reduce_or_sync(0xffffffffu, lane < moves ? 1u << (p.x & 31) : 0u);
    uint4 v[NI];
    float most = 0.f;
#pragma unroll
    for (int u = 0; u < NI; ++u) {
      const int y = __shfl_sync(0xffffffffu, p.y, u * RPI + sub);
      v[u] = make_uint4(0, 0, 0, 0);
      if (y >= 0) v[u] = q8_ld_stream(codes + (int64_t)y * D + col * 16);
    }
#pragma unroll
    for (int u = 0; u < NI; ++u) {
      const float f = __shfl_sync(0xffffffffu, from, u * RPI + sub);
      most = fmaxf(most, q8_float2(evict_top_code(v[u])).x * f);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    const float old = __ldcg(scale + block);
    float s = q8_scale(most);
    if (old >= s) s = old;
    if (old < s) {  // the rows that stay (those at or past keep are only read now)
      q8_rescale_rows<D, 4>(codes + (int64_t)block * (kQ8Block * D), evict_rows_below(a.keep, block) & ~filled, old * q8_inverse(s));
    }
    __syncwarp();  // every lane has read the old scale
#pragma unroll
    for (int u = 0; u < NI; ++u) {
      const int x = __shfl_sync(0xffffffffu, p.x, u * RPI + sub);
      const float f = __shfl_sync(0xffffffffu, from, u * RPI + sub);
      if (x >= 0) {
        if (f != s) {
          v[u] = q8_rescale(v[u], f * q8_inverse(s));
        }
        *reinterpret_cast<uint4*>(codes + (int64_t)x * D + col * 16) = v[u];
      }
    }
    if (lane == 0 && old < s) scale[block] = s;
  }
}

// Workspace of n_layers <= kQ8Layers: moves (at most n_cap / 2 of a head), blocks, counts, scales.
static size_t evict_align(size_t x) { return (x + 255) & ~(size_t)255; }
size_t evict_ws_bytes(int n_layers, int Hkv, int n_cap) {
  const size_t pairs = (size_t)n_layers * Hkv;
  return evict_align(pairs * (n_cap / 2) * sizeof(int2)) + evict_align(pairs * (n_cap / kQ8Block + 1) * sizeof(int2)) +
         evict_align(pairs * sizeof(int2)) + evict_align(pairs * sizeof(float2));
}

// Whether a head's CTA moves its rows by itself, by what either way is to take at most (in ns; 152 SMs).  By itself: 12 a row of
// 256 bytes (4 that do not go by its bytes), 20 a row of codes, heads beyond those that run at once in a second turn.  By a second kernel:
// its launch, and the bytes at the rate of scattered rows, or a turn of 8 us for the blocks that its warps take at once.
// Measured, by itself against a second kernel, us: 8 heads 8911 to 8272 rows bf16 18.5, 15.4, codes 26, 20.5; 32 heads 19.0, 18.1
// and 27, 34; 64 heads 19.4, 22.0 and 29, 54; 8 heads 2100 to 2048 6.7, 8.2; 64 heads 16384 to 8272 105, 77 and 127, 75; 256 heads 176, 270
// (codes), 32768 to 8272 313, 355.
// Where the count is on the device this, the kernel's number of keys and the place of the list go by the rows there may be.  8273 to 8272
// rows in caches of 8273, 8337 and 12369 rows: 8 heads 10.5, 10.5, 14.4 us (codes 10.8, 12.7, 14.4), 256 heads 12.4, 12.4, 16.5 (16.6, 16.4, 22.7).
static bool evict_moves_rows(int pairs, int plan_cap, int block_cap, int row_bytes, bool q8, int at_once, int n_sm) {
  const double turns = (pairs + at_once - 1) / at_once, rows = (double)pairs * plan_cap;
  const double itself = turns * plan_cap * (q8 ? 20.0 : 4.0 + row_bytes / 32.0);
  const double second = 4000.0 + (q8 ? 8000.0 * ceil(2.0 * pairs * block_cap / (n_sm * 32)) : rows * 4 * row_bytes / 6500.0);
  return itself <= second;
}

// By the most rows a CTA can have: a loop over slots is unrolled to its limit.  48 heads 1025 rows 5.4 us, 10.7 with the kernel of 32
// groups; 2200 rows 7.0, 12.2; 256 heads 8273 rows 12.3, 16.4; a cluster's 8 heads 16384 rows 21, 32.  A kernel of 24 groups in place of
// that of 20: 256 heads 8273 rows 12.6 -> 14.5 (codes 16.5 -> 18.5), 10240 to 8272 81 -> 82 (74 -> 76), 12288 to 8272 133 -> 131 (114 -> 111).
template <int DQ, bool CL>
static void (*evict_kernel(int rows, int* threads))(EvictArgs) {
  *threads = rows <= kEvictShort && !CL ? kEvictShortThreads : kEvictLongThreads;
  const int groups = (rows + *threads - 1) / *threads;  // of 32 slots, a warp
  if constexpr (CL) {
    return groups <= 8 ? evict_select_kernel<DQ, kEvictLongThreads, 8, true> : evict_select_kernel<DQ, kEvictLongThreads, 32, true>;
  } else {
    if (rows > kEvictShort) return evict_select_kernel<DQ, kEvictLongThreads, 32, false>;
    if (groups <= 4) return evict_select_kernel<DQ, kEvictShortThreads, 4, false>;
    if (groups <= 8) return evict_select_kernel<DQ, kEvictShortThreads, 8, false>;
    if (groups <= 16) return evict_select_kernel<DQ, kEvictShortThreads, 16, false>;
    if (groups <= 20) return evict_select_kernel<DQ, kEvictShortThreads, 20, false>;
    return evict_select_kernel<DQ, kEvictShortThreads, 32, false>;
  }
}

// CTAs of a head: as many as its keys need, and, where heads leave SMs idle, more while each has kEvictPart rows.  Against as many as
// its keys need: 2 heads 8911 to 2048 rows 15.2 us, 14.8 (codes 17.8, 20.3); 8 heads 16384 to 8272 21, 26 (26, 33), 32768 28, 31
// (29, 48), 65536 32, 43 (32, 58).
constexpr int kEvictPart = 4096;
static int evict_cluster(int pairs, int n_most, int n_sm) {
  int c = 1;
  while (c * kEvictLong < n_most) c *= 2;
  while (c < kEvictCluster && 2 * c * pairs <= n_sm && n_most >= 2 * c * kEvictPart) c *= 2;
  return c;
}

// dq: 0: bf16 rows of row_bytes, else the channels of a row of codes.
static stepkv_status_t evict_all(int n_layers, void* const* K, void* const* V, float* const* K_scale, float* const* V_scale,
                                 int64_t head_bytes, int64_t scale_stride, int row_bytes, int Hkv, int dq, const EvictSpec& s,
                                 cudaStream_t stream) {
  int n_sm = 0;
  cudaError_t e = device_sm_count(&n_sm);
  for (int l0 = 0; e == cudaSuccess && l0 < n_layers; l0 += kQ8Layers) {
    const int nl = std::min(kQ8Layers, n_layers - l0), pairs = nl * Hkv;
    const bool last = l0 + nl == n_layers;
    EvictArgs a;
    memset(&a, 0, sizeof(a));
    for (int l = 0; l < nl; ++l) {
      a.mass[l] = s.mass[l0 + l];
      a.pos[l] = s.pos[l0 + l];
      a.K[l] = static_cast<uint8_t*>(K[l0 + l]);
      a.V[l] = static_cast<uint8_t*>(V[l0 + l]);
      a.K_scale[l] = dq ? K_scale[l0 + l] : nullptr;
      a.V_scale[l] = dq ? V_scale[l0 + l] : nullptr;
    }
    a.mass_stride = s.mass_stride;
    a.pos_stride = s.pos_stride;
    a.head_bytes = head_bytes;
    a.scale_stride = scale_stride;
    a.layer0 = l0;
    a.n_layers = nl;
    a.Hkv = Hkv;
    a.row_bytes = row_bytes;
    a.n_dev = s.n_dev;
    a.n_stride = s.n_stride;
    a.n_host = s.n_host;
    a.n_cap = s.n_cap;
    a.keep = s.keep;
    a.n_sink = s.n_sink;
    a.n_recent = s.n_recent;
    const int n_most = s.n_dev ? s.n_cap : s.n_host;
    a.plan_cap = std::max(0, std::min(s.keep, n_most - s.keep));
    a.block_cap = std::min(a.plan_cap, (s.keep + kQ8Block - 1) / kQ8Block);
    uint8_t* w = static_cast<uint8_t*>(s.ws);
    a.plan = reinterpret_cast<int2*>(w);
    w += evict_align((size_t)pairs * a.plan_cap * sizeof(int2));
    a.blocks = reinterpret_cast<int2*>(w);
    w += evict_align((size_t)pairs * a.block_cap * sizeof(int2));
    a.counts = reinterpret_cast<int2*>(w);
    w += evict_align((size_t)pairs * sizeof(int2));
    a.cut = reinterpret_cast<float2*>(w);
    a.status = s.status;
    a.cluster = 1;
    a.moves_rows = n_most <= kEvictLong && evict_moves_rows(pairs, a.plan_cap, a.block_cap, row_bytes, dq != 0, n_most <= kEvictShort ? 2 * n_sm : n_sm, n_sm);
    if (!a.moves_rows) a.cluster = evict_cluster(pairs, n_most, n_sm);
    // one count for all is read by every launch: replaced by the last; n itself only after all CTAs have read it
    int32_t* const n_out = s.n_dev && s.n_stride ? s.n_out : last ? s.n_out : nullptr;
    const bool late = n_out && n_out == s.n_dev;
    a.n_out = late || !a.moves_rows ? nullptr : n_out;
    int threads = 0;
    const int rows = (n_most + a.cluster - 1) / a.cluster;
    auto select = a.cluster > 1 ? (dq == 0 ? evict_kernel<0, true>(rows, &threads) : evict_kernel<64, true>(rows, &threads))
                  : dq == 0     ? evict_kernel<0, false>(rows, &threads)
                  : dq == 64    ? evict_kernel<64, false>(rows, &threads)
                                : evict_kernel<128, false>(rows, &threads);
    a.smem_plan = a.moves_rows && a.plan_cap <= kEvictSmemPlan ? a.plan_cap : 0;
    const int smem = (2 * a.smem_plan + (dq && a.moves_rows ? 3 * ((s.keep + kQ8Block - 1) / kQ8Block) : 0)) * (int)sizeof(uint32_t);
    e = ensure_smem_attr(reinterpret_cast<const void*>(select), smem);
    if (e == cudaSuccess)
      e = a.cluster > 1 ? launch_cluster(select, dim3(pairs * a.cluster), dim3(threads), a.cluster, smem, stream, a, true)
                        : launch_kernel(select, dim3(pairs), dim3(threads), smem, stream, a, true);
    if (e != cudaSuccess) break;
    if (a.moves_rows) {
      if (late) {
        a.n_out = n_out;
        e = launch_kernel(evict_counts_kernel, dim3(1), dim3(64), 0, stream, a, true);
      }
      continue;
    }
    EvictMoveArgs m;
    memset(&m, 0, sizeof(m));
    for (int l = 0; l < nl; ++l) {
      m.rows[2 * l] = a.K[l];
      m.rows[2 * l + 1] = a.V[l];
      m.scale[2 * l] = a.K_scale[l];
      m.scale[2 * l + 1] = a.V_scale[l];
    }
    m.head_bytes = head_bytes;
    m.scale_stride = scale_stride;
    m.by_heads = make_fastdiv(Hkv);
    m.sets = 2 * pairs;
    m.Hkv = Hkv;
    m.n_layers = nl;
    m.layer0 = l0;
    m.row_bytes = row_bytes;
    m.keep = s.keep;
    m.plan_cap = a.plan_cap;
    m.block_cap = a.block_cap;
    m.plan = a.plan;
    m.blocks = a.blocks;
    m.counts = a.counts;
    m.cut = a.cut;
    m.n_dev = s.n_dev;
    m.n_stride = s.n_stride;
    m.n_host = s.n_host;
    m.n_cap = s.n_cap;
    m.n_out = n_out;
    const int per_chunk = dq ? 1 : 32 / (row_bytes >> 4) * kEvictMoveUnroll;
    const int64_t chunks = (int64_t)m.sets * (((dq ? m.block_cap : m.plan_cap) + per_chunk - 1) / per_chunk);
    const int64_t ctas = (chunks + kQ8Threads / 32 - 1) / (kQ8Threads / 32);
    const int grid = (int)std::max<int64_t>(1, std::min<int64_t>(n_sm * 4, ctas));
    auto move = !dq ? evict_move_kernel : dq == 128 ? evict_q8_move_kernel<128> : evict_q8_move_kernel<64>;
    e = launch_kernel(move, dim3(grid), dim3(kQ8Threads), 0, stream, m, true);
  }
  if (e == cudaSuccess) return STEPKV_OK;
  set_last_cuda_error(e);
  return STEPKV_ECUDA;
}

stepkv_status_t evict_run(int n_layers, void* const* K, void* const* V, int64_t kv_head_stride, int Hkv, int d,
                          const EvictSpec& s, cudaStream_t stream) {
  return evict_all(n_layers, K, V, nullptr, nullptr, 2 * kv_head_stride, 0, 2 * d, Hkv, 0, s, stream);
}

stepkv_status_t q8_evict_run(const stepkv_q8_cache_t& c, const EvictSpec& s, cudaStream_t stream) {
  return evict_all(c.n_layers, c.K, c.V, c.K_scale, c.V_scale, c.code_head_stride, c.scale_head_stride, c.d, c.Hkv, c.d, s, stream);
}

}  // namespace stepkv
