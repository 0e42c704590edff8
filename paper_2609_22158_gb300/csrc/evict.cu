// Eviction by accumulated attention: every (layer, KV head) keeps `keep` of its n rows, in place.
//   protected(j) = pos[j] < n_sink or pos[j] > max(pos) - n_recent
//   retained     = the first `keep` by (protected, mass descending, slot ascending)
//   the i-th slot below keep that goes receives the i-th slot at or above keep that stays
//
// Two kernels.  The first, a CTA per (layer, head), finds the retained rows from n masses and positions, writes the list of
// moves, and moves masses and positions; the second moves rows of keys and values over the whole machine.  In 8 bits it moves
// them block by block, as the block's scale may have to grow.
//
// A row's rank is a 32-bit key: all ones where it is protected, else the mass as an integer that orders like the number (0 for
// a NaN).  The key T of the last retained row comes from three histograms of 11, 11 and 10 bits; with R(j) = min(rows below j
// that equal T, those of them that stay) + rows below j above T, the retained rows below slot j,
//   a slot j < keep that goes is number j - R(j) of those, a slot j >= keep that stays number R(j) - R(keep).
#include <limits.h>

#include <algorithm>

#include "common.cuh"
#include "fastdiv.h"
#include "internal.h"
#include "q8.cuh"

namespace stepkv {

constexpr int kEvictThreads = 1024;
constexpr int kEvictWarps = kEvictThreads / 32;
constexpr int kEvictSmemKeys = 49152;  // keys held in shared memory (192 KB); the rest are made anew in every pass
constexpr uint32_t kEvictProtected = 0xFFFFFFFFu;

struct EvictArgs {
  float* mass[kQ8Layers];
  int32_t* pos[kQ8Layers];
  const float* K_scale[kQ8Layers];  // 8 bits: read before the moves where a block is cut by `keep`
  const float* V_scale[kQ8Layers];
  int64_t mass_stride, pos_stride, scale_stride;
  int layer0, Hkv;
  const int32_t* n_dev;
  int n_stride, n_host, n_cap, keep, n_sink, n_recent;
  int smem_keys;
  // workspace, per (layer, head):
  int2* plan;       // [plan_cap]: (slot filled, slot it is filled from), both ascending
  int2* blocks;     // [block_cap], 8 bits: (block, number of its first move * 64 + moves) of blocks that receive rows, in any order
  int2* counts;     // (moves, blocks that receive rows)
  float2* cut;      // 8 bits: the scales (K, V) of the block that `keep` cuts
  int plan_cap, block_cap;
  int32_t* status;
};
static_assert(sizeof(EvictArgs) <= 32000, "kernel parameter space");

__device__ __forceinline__ uint32_t evict_key(float mass, int pos, int n_sink, int64_t recent) {
  if (pos < n_sink || pos > recent) return kEvictProtected;
  return mass == mass ? float_to_ordered(mass + 0.f) : 0u;  // (-0 + 0 is 0)
}

// Inclusive sums over the CTA's threads; s_warp: 32 words.  Two barriers.
__device__ __forceinline__ uint32_t evict_scan(uint32_t x, uint32_t* s_warp) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) s_warp[warp] = x;
  __syncthreads();
  uint32_t w = s_warp[lane];
  const uint32_t before = __reduce_add_sync(0xffffffffu, lane < warp ? w : 0u);
  __syncthreads();
  return x + before;
}

template <bool Q8>
__global__ void __launch_bounds__(kEvictThreads) evict_select_kernel(const __grid_constant__ EvictArgs a) {
  extern __shared__ uint32_t s_key[];
  __shared__ uint32_t s_hist[2048];
  __shared__ uint32_t s_warp[kEvictWarps];
  __shared__ uint4 s_count[kEvictWarps];
  __shared__ int s_top[kEvictWarps];
  __shared__ uint32_t s_bin, s_rem, s_safe, s_blocks;
  pdl_wait();
  pdl_launch_dependents();
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int pair = blockIdx.x, layer = pair / a.Hkv, h = pair - layer * a.Hkv;
  int n = a.n_host;
  if (a.n_dev) {
    n = __ldcg(a.n_dev + (a.layer0 + layer) * a.n_stride);
    if (n < 0 || n > a.n_cap) {
      if (t == 0) record_status(a.status, n < 0 ? STEPKV_EDATA : STEPKV_ENOSPACE);
      n = 0;
    }
  }
  const int keep = a.keep;
  if (n <= keep) {
    if (t == 0) a.counts[pair] = make_int2(0, 0);
    return;
  }
  float* mass = a.mass[layer] + (int64_t)h * a.mass_stride;
  int32_t* pos = a.pos[layer] + (int64_t)h * a.pos_stride;

  int top = INT_MIN;
  for (int j = t; j < n; j += kEvictThreads) top = max(top, __ldcg(pos + j));
  top = __reduce_max_sync(0xffffffffu, top);
  if (lane == 0) s_top[warp] = top;
  if (t == 0) s_safe = s_blocks = 0;
  __syncthreads();
  top = __reduce_max_sync(0xffffffffu, s_top[lane]);
  const int64_t recent = (int64_t)top - a.n_recent;
  auto make_key = [&](int j) { return evict_key(__ldcg(mass + j), __ldcg(pos + j), a.n_sink, recent); };
  uint32_t safe = 0;
  for (int j = t; j < n; j += kEvictThreads) {
    const uint32_t k = make_key(j);
    if (j < a.smem_keys) s_key[j] = k;
    safe += k == kEvictProtected;
  }
  safe = __reduce_add_sync(0xffffffffu, safe);
  if (lane == 0 && safe) atomicAdd(&s_safe, safe);
  __syncthreads();
  auto key = [&](int j) { return j < a.smem_keys ? s_key[j] : make_key(j); };

  // the key of the last retained row, and how many of those that equal it stay
  uint32_t T = kEvictProtected, ties = keep;
  if ((int)s_safe < keep) {
    uint32_t mask = 0;
    T = 0;
    ties = keep - s_safe;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
      const uint32_t digits = pass == 2 ? 1023u : 2047u;
      s_hist[t] = s_hist[t + kEvictThreads] = 0;
      __syncthreads();
      for (int j = t; j < n; j += kEvictThreads) {
        const uint32_t k = key(j);
        if ((k & mask) == T && k != kEvictProtected) atomicAdd(&s_hist[k >> shift & digits], 1u);
      }
      __syncthreads();
      const uint32_t first = s_hist[2047 - 2 * t], second = s_hist[2046 - 2 * t];  // bins from the top
      const uint32_t upto = evict_scan(first + second, s_warp), above = upto - first - second;
      if (above < ties && ties <= upto) {
        const bool in_first = ties <= above + first;
        s_bin = in_first ? 2047 - 2 * t : 2046 - 2 * t;
        s_rem = ties - above - (in_first ? 0 : first);
      }
      __syncthreads();
      T |= s_bin << shift;
      mask |= digits << shift;
      ties = s_rem;
    }
  }

  // rows above T and equal to it: of each warp's part of the slots, and of those below keep
  const int groups = (n + 31) / 32, per_warp = (groups + kEvictWarps - 1) / kEvictWarps;
  const int g0 = min(groups, warp * per_warp), g1 = min(groups, g0 + per_warp);
  uint4 c = make_uint4(0, 0, 0, 0);
  for (int g = g0; g < g1; ++g) {
    const int j = g * 32 + lane;
    const uint32_t k = j < n ? key(j) : 0u;
    const uint32_t gt = __ballot_sync(0xffffffffu, j < n && k > T), eq = __ballot_sync(0xffffffffu, j < n && k == T);
    const uint32_t low = __ballot_sync(0xffffffffu, j < keep);
    c.x += __popc(gt);
    c.y += __popc(eq);
    c.z += __popc(gt & low);
    c.w += __popc(eq & low);
  }
  if (lane == 0) s_count[warp] = c;
  __syncthreads();
  const uint4 mine = s_count[lane];
  uint32_t gt0 = __reduce_add_sync(0xffffffffu, lane < warp ? mine.x : 0u);
  uint32_t eq0 = __reduce_add_sync(0xffffffffu, lane < warp ? mine.y : 0u);
  const uint32_t gt_low = __reduce_add_sync(0xffffffffu, mine.z), eq_low = __reduce_add_sync(0xffffffffu, mine.w);
  const int kept_low = gt_low + min(eq_low, ties), moves = keep - kept_low;
  int2* plan = a.plan + (int64_t)pair * a.plan_cap;
  int2* blocks = a.blocks + (int64_t)pair * a.block_cap;
  for (int g = g0; g < g1; ++g) {
    const int j = g * 32 + lane;
    const uint32_t k = j < n ? key(j) : 0u;
    const uint32_t gt = __ballot_sync(0xffffffffu, j < n && k > T), eq = __ballot_sync(0xffffffffu, j < n && k == T);
    const uint32_t below = (1u << lane) - 1u;
    const uint32_t eqb = eq0 + __popc(eq & below);
    const bool stays = (gt >> lane & 1u) || ((eq >> lane & 1u) && eqb < ties);
    const int R = gt0 + __popc(gt & below) + min(eqb, ties);
    const bool hole = j < keep && !stays;
    if (hole) plan[j - R].x = j;
    if (j >= keep && stays) plan[R - kept_low].y = j;
    if (Q8) {
      const uint32_t holes = __ballot_sync(0xffffffffu, hole);
      if (lane == 0 && holes) blocks[atomicAdd(&s_blocks, 1u)] = make_int2(g, (g * 32 - R) * 64 + __popc(holes));
    }
    gt0 += __popc(gt);
    eq0 += __popc(eq);
  }
  __syncthreads();
  if (t == 0) {
    a.counts[pair] = make_int2(moves, s_blocks);
    if (Q8 && keep % kQ8Block)
      a.cut[pair] = make_float2(__ldcg(a.K_scale[layer] + (int64_t)h * a.scale_stride + keep / kQ8Block),
                                __ldcg(a.V_scale[layer] + (int64_t)h * a.scale_stride + keep / kQ8Block));
  }
  for (int i = t; i < moves; i += kEvictThreads) {
    const int2 p = plan[i];
    mass[p.x] = __ldcg(mass + p.y);
    pos[p.x] = __ldcg(pos + p.y);
  }
  __syncthreads();
  for (int j = keep + t; j < n; j += kEvictThreads) mass[j] = 0.f;
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
__device__ __forceinline__ void evict_counts(const EvictMoveArgs& a) {
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
  evict_counts(a);
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
  evict_counts(a);
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
      const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
      uint32_t top = 0;  // magnitudes order as integers; NaN does not count
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t m = w[i] & 0x7F7F7F7Fu;
        top = __vmaxu4(top, m & ~__vcmpeq4(m, 0x7F7F7F7Fu));
      }
      top = max(max(top & 0xFFu, top >> 8 & 0xFFu), max(top >> 16 & 0xFFu, top >> 24));
      most = fmaxf(most, q8_float2(top).x * f);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    const float old = __ldcg(scale + block);
    float s = q8_scale(most);
    if (old >= s) s = old;
    if (old < s) {  // the rows that stay (those at or past keep are only read now)
      const float ratio = old * q8_inverse(s);
      const int end = min(kQ8Block, a.keep - block * kQ8Block);
      uint32_t* w = reinterpret_cast<uint32_t*>(codes + (int64_t)block * (kQ8Block * D));
      for (int i = lane; i < end * (D / 4); i += 32)
        if (!(filled >> (i / (D / 4)) & 1u)) w[i] = q8_rescale(__ldcg(w + i), ratio);
    }
    __syncwarp();  // every lane has read the old scale
#pragma unroll
    for (int u = 0; u < NI; ++u) {
      const int x = __shfl_sync(0xffffffffu, p.x, u * RPI + sub);
      const float f = __shfl_sync(0xffffffffu, from, u * RPI + sub);
      if (x >= 0) {
        if (f != s) {
          const float ratio = f * q8_inverse(s);
          v[u] = make_uint4(q8_rescale(v[u].x, ratio), q8_rescale(v[u].y, ratio), q8_rescale(v[u].z, ratio), q8_rescale(v[u].w, ratio));
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

static cudaError_t evict_launch(int nl, int l0, bool last, int Hkv, const EvictSpec& s, EvictMoveArgs& m, const float* const* K_scale,
                                const float* const* V_scale, int64_t scale_stride, int d, bool q8, cudaStream_t stream) {
  int n_sm = 0;
  cudaError_t e = device_sm_count(&n_sm);
  if (e != cudaSuccess) return e;
  EvictArgs a;
  memset(&a, 0, sizeof(a));
  for (int l = 0; l < nl; ++l) {
    a.mass[l] = s.mass[l0 + l];
    a.pos[l] = s.pos[l0 + l];
    a.K_scale[l] = q8 ? K_scale[l0 + l] : nullptr;
    a.V_scale[l] = q8 ? V_scale[l0 + l] : nullptr;
  }
  a.mass_stride = s.mass_stride;
  a.pos_stride = s.pos_stride;
  a.scale_stride = scale_stride;
  a.layer0 = l0;
  a.Hkv = Hkv;
  a.n_dev = s.n_dev;
  a.n_stride = s.n_stride;
  a.n_host = s.n_host;
  a.n_cap = s.n_cap;
  a.keep = s.keep;
  a.n_sink = s.n_sink;
  a.n_recent = s.n_recent;
  const int n_most = s.n_dev ? s.n_cap : s.n_host;
  a.smem_keys = std::min(kEvictSmemKeys, n_most);
  const int pairs = nl * Hkv;
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
  auto select = q8 ? evict_select_kernel<true> : evict_select_kernel<false>;
  const int smem = a.smem_keys * (int)sizeof(uint32_t);
  e = ensure_smem_attr(reinterpret_cast<const void*>(select), smem);
  if (e == cudaSuccess) e = launch_kernel(select, dim3(pairs), dim3(kEvictThreads), smem, stream, a, true);
  if (e != cudaSuccess) return e;
  m.by_heads = make_fastdiv(Hkv);
  m.sets = 2 * pairs;
  m.Hkv = Hkv;
  m.n_layers = nl;
  m.layer0 = l0;
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
  m.n_out = s.n_dev && s.n_stride ? s.n_out : last ? s.n_out : nullptr;  // (one count for all: read by every launch)
  const int per_chunk = q8 ? 1 : 32 / (d >> 3) * kEvictMoveUnroll;
  const int64_t chunks = (int64_t)m.sets * (((q8 ? m.block_cap : m.plan_cap) + per_chunk - 1) / per_chunk);
  const int64_t ctas = (chunks + kQ8Threads / 32 - 1) / (kQ8Threads / 32);
  const int grid = (int)std::max<int64_t>(1, std::min<int64_t>(n_sm * 4, ctas));
  auto move = !q8 ? evict_move_kernel : d == 128 ? evict_q8_move_kernel<128> : evict_q8_move_kernel<64>;
  return launch_kernel(move, dim3(grid), dim3(kQ8Threads), 0, stream, m, true);
}

stepkv_status_t evict_run(int n_layers, void* const* K, void* const* V, int64_t kv_head_stride, int Hkv, int d,
                          const EvictSpec& s, cudaStream_t stream) {
  cudaError_t e = cudaSuccess;
  for (int l0 = 0; e == cudaSuccess && l0 < n_layers; l0 += kQ8Layers) {
    const int nl = std::min(kQ8Layers, n_layers - l0);
    EvictMoveArgs m;
    memset(&m, 0, sizeof(m));
    for (int l = 0; l < nl; ++l) {
      m.rows[2 * l] = static_cast<uint8_t*>(K[l0 + l]);
      m.rows[2 * l + 1] = static_cast<uint8_t*>(V[l0 + l]);
    }
    m.head_bytes = 2 * kv_head_stride;
    m.row_bytes = 2 * d;
    e = evict_launch(nl, l0, l0 + nl == n_layers, Hkv, s, m, nullptr, nullptr, 0, d, false, stream);
  }
  if (e == cudaSuccess) return STEPKV_OK;
  set_last_cuda_error(e);
  return STEPKV_ECUDA;
}

stepkv_status_t q8_evict_run(const stepkv_q8_cache_t& c, const EvictSpec& s, cudaStream_t stream) {
  cudaError_t e = cudaSuccess;
  for (int l0 = 0; e == cudaSuccess && l0 < c.n_layers; l0 += kQ8Layers) {
    const int nl = std::min(kQ8Layers, c.n_layers - l0);
    EvictMoveArgs m;
    memset(&m, 0, sizeof(m));
    for (int l = 0; l < nl; ++l) {
      m.rows[2 * l] = static_cast<uint8_t*>(c.K[l0 + l]);
      m.rows[2 * l + 1] = static_cast<uint8_t*>(c.V[l0 + l]);
      m.scale[2 * l] = c.K_scale[l0 + l];
      m.scale[2 * l + 1] = c.V_scale[l0 + l];
    }
    m.head_bytes = c.code_head_stride;
    m.scale_stride = c.scale_head_stride;
    m.row_bytes = c.d;
    e = evict_launch(nl, l0, l0 + nl == c.n_layers, c.Hkv, s, m, c.K_scale, c.V_scale, c.scale_head_stride, c.d, true, stream);
  }
  if (e == cudaSuccess) return STEPKV_OK;
  set_last_cuda_error(e);
  return STEPKV_ECUDA;
}

}  // namespace stepkv
