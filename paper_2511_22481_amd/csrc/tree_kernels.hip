// Trees of drafted tokens over the paged 8-bit cache: who follows whom, and the rows that stay.
//
// A request with L tokens brings n <= 64 of them as nodes of a tree, parents before children, in the cache positions L - n .. L - 1.
// mask(t) = 2^t + mask(parent of t): the nodes that node t follows, and itself; its position in the text is L - n + |mask(t)| - 1.
//
// Of the tree a path p_0 < p_1 < ... stays: row L - n + p_i of every layer's cache goes to row L - n + i.  A row that comes to another
// block meets another scale: the block's new one is the largest of the scales that its rows come with (and of its own, where
// tokens of the text lie in it), and a row's codes are multiplied by old / new <= 1 and rounded, which is exact for powers of two but for
// numbers that become subnormal.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "gqa.h"
#include "wave.h"

namespace omniattn {
namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kNodes = OMNIATTN_TREE_NODES;

// First token of a request among the call's, and how many it has.
struct Nodes {
  int begin, n;
};
__device__ __forceinline__ Nodes nodes_of(const int32_t* q_start, int b, int num_tokens) {
  const int lo = q_start ? q_start[b] : b, hi = q_start ? q_start[b + 1] : b + 1;
  Nodes r;
  r.begin = min(max(lo, 0), num_tokens);
  r.n = min(max(hi, r.begin), num_tokens) - r.begin;
  return r;
}

// A wave to a request, a lane to a node.  Every pass doubles the way that a set reaches up: six at the most, and no loop over a node's ancestors, of which a
// chain has 63.  A launch, two loads one after the other, and the passes bound it: 1.6 us (1 request of 8 nodes), 3.7 us (1500 of up to 64).
__global__ __launch_bounds__(kThreads) void tree_masks_kernel(TreeMasksParams p) {
  const int lane = threadIdx.x & 63, b = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (b >= p.batch) return;
  const Nodes r = nodes_of(p.q_start, b, p.num_tokens);
  const int text = p.seq_lens[b] - r.n;
  if (r.n > kNodes) {
    for (int t = lane; t < r.n; t += 64) {
      p.masks[r.begin + t] = 0;
      if (p.positions) p.positions[r.begin + t] = -1;
    }
    return;
  }
  int up = lane < r.n ? p.parents[r.begin + lane] : lane;
  up = up >= 0 && up < lane ? up : lane;
  uint64_t mask = (uint64_t)1 << lane;
  while (true) {
    const uint32_t lo = (uint32_t)__shfl((int)mask, up), hi = (uint32_t)__shfl((int)(mask >> 32), up);
    mask |= (uint64_t)hi << 32 | lo;
    const int next = __shfl(up, up);
    if (!__any(next != up)) break;  // (every way has reached its root, whose set is its own)
    up = next;
  }
  if (lane < r.n) {
    p.masks[r.begin + lane] = mask;
    if (p.positions) p.positions[r.begin + lane] = text + __popcll(mask) - 1;
  }
}

__device__ __forceinline__ uint32_t recode(uint32_t codes, float ratio) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
  return __builtin_amdgcn_cvt_pk_fp8_f32(b[0] * ratio, b[1] * ratio, __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * ratio, a[1] * ratio, 0, false), true);
}
__device__ __forceinline__ u32x4 recode(const u32x4& x, float ratio) {
  return u32x4{recode(x[0], ratio), recode(x[1], ratio), recode(x[2], ratio), recode(x[3], ratio)};
}
__device__ __forceinline__ float scale_ratio(float old, float now) { return now > 0.f ? old / now : 1.f; }
// The largest of a wave's scales, which are not negative.
__device__ __forceinline__ float wave_max(float x) {
  return __builtin_bit_cast(float, wave_join(__builtin_bit_cast(uint32_t, x), [](uint32_t a, uint32_t b) { return max(a, b); }));
}

// A wave to a request, kUnits of its (KV head, K or V), and up to kMostLayers layers, one after the other.  Rows go up in order, kRows at a time: a row's source
// lies at or behind its place, so what a pass writes is no later pass's source, and within a pass all loads are done before the first store.
//
// Chains of loads bound it (the request's nodes, its length and path, the pages, scales and rows, the store) and rows of 128 bytes here and there.  So a
// wave asks for the next layer's scales and first rows before it works on a layer's, and where there are more waves than the compute units hold (32 each),
// they take more layers instead.  us a call (replayed), requests of up to 32 nodes, 8 KV heads of 128, layers to a wave up to 1 / 2 / 4 / 8:
//   16 x 32 layers   6.5 / 6.6 / 6.5 / 6.5       64 x 64 layers   25.6 / 19.7 / 18.7 / 18.9
//   64 x 32         15.2 / 12.6 / 12.6 / 12.6   256 x 32          37.1 / 27.2 / 24.0 / 28.5
// (More layers from 16 waves on: 64 x 32 14.9.)  Of (KV head, K or V) to a wave, with a layer each, 64 x 32 and 1 x 4 layers: 1 18.4 and 4.8 us, 2
// 14.0 and 5.2, 4 15.0 and 6.0, 8 13.3 and 8.7.
constexpr int kUnits = 2, kMostLayers = 4;
static_assert(2 % kUnits == 0);  // (a wave's units are all there, however many KV heads)
template <int D>
__global__ __launch_bounds__(kThreads) void gqa_keep_kernel(GqaKeepParams p) {
  constexpr int kLanes = D / 16, kRows = 64 / kLanes;  // lanes of a row, 16 codes each; rows of a pass
  const int lane = threadIdx.x & 63, each = p.scale_tokens, blocks = kPage / each, sharers = 2 * p.kv_heads / kUnits;
  const uint32_t id = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t group = id / (uint32_t)sharers, run = group / (uint32_t)p.batch;
  const int b = (int)(group - run * p.batch), unit0 = (int)(id - group * sharers) * kUnits;
  if (run * (uint32_t)p.run >= (uint32_t)p.layers) return;
  const int layer0 = (int)run * p.run, layers = min(p.run, p.layers - layer0);
  const Nodes r = nodes_of(p.q_start, b, p.num_tokens);
  const int text = min(p.seq_lens[b], p.max_pages * kPage) - r.n;
  if (r.n > kNodes || text < 0) return;
  // the nodes that stay: an ascending path, which ends where an entry is none
  const int from = lane < r.n ? p.path[r.begin + lane] : -1, before = __shfl_up(from, 1);
  const uint64_t off = ~__ballot(from >= lane && from < r.n && (lane == 0 || from > before));
  const int kept = off ? __builtin_ctzll(off) : 64;
  const uint64_t moved = __ballot(lane < kept && from != lane);
  if (!moved) return;
  // rows of the blocks that rows move to, from the first of them on
  const int first = max(0, (text + __builtin_ctzll(moved)) / each * each - text);
  const bool mine = lane >= first && lane < kept;
  const int32_t* const table = p.page_table + b * p.table_stride;
  const int src = text + (mine ? from : first), dst = text + (mine ? lane : first);
  const int64_t src_page = ((int64_t)layer0 * p.num_pages + table[src / kPage]) * p.kv_heads, dst_page = ((int64_t)layer0 * p.num_pages + table[dst / kPage]) * p.kv_heads;
  const int64_t next_layer = p.num_pages * p.kv_heads;
  // up to three blocks (64 tokens, 32 to a block)
  const int block0 = (text + first) / each, block = dst / each - block0, last_block = (text + kept - 1) / each - block0;
  const int held = text - block0 * each;  // tokens of the text in the first of them, if any
  const int64_t page0 = __shfl(dst_page, first);
  const int64_t src_at = (src_page * kPage + src % kPage) * D, dst_at = (dst_page * kPage + dst % kPage) * D;
  const int col = lane % kLanes * 16, in_pass = lane / kLanes;
  auto cache = [&](int j, int64_t pages) { return p.cache[(unit0 + j) & 1] + (size_t)(pages + ((unit0 + j) >> 1)) * kPage * D; };
  auto scale_at = [&](int j, int64_t page, int at) { return p.scales[(unit0 + j) & 1] + (page + ((unit0 + j) >> 1)) * blocks + at % kPage / each; };
  u32x4 x[kUnits];
  auto load = [&](int64_t pages, int row0) {
    const int64_t s = __shfl(src_at, min(row0 + in_pass, 63));
    if (row0 + in_pass < kept) {
#pragma unroll
      for (int j = 0; j < kUnits; ++j) x[j] = *(const u32x4*)(cache(j, pages) + s + col);
    }
  };
  float old[kUnits], own[kUnits], next_old[kUnits], next_own[kUnits];
  auto load_scales = [&](int64_t pages) {
#pragma unroll
    for (int j = 0; j < kUnits; ++j) {
      next_old[j] = *scale_at(j, pages + src_page, src);
      next_own[j] = held > 0 ? *scale_at(j, pages + page0, block0 * each) : 0.f;
    }
  };
  load(0, first);
  load_scales(0);
  int64_t pages = 0;  // those of the layers before
  for (int i = 0; i < layers; ++i, pages += next_layer) {
    float ratio[kUnits], now[kUnits], now0[kUnits];
#pragma unroll
    for (int j = 0; j < kUnits; ++j) {
      old[j] = next_old[j];
      own[j] = next_own[j];
      now[j] = now0[j] = 0.f;
      for (int k = 0; k <= last_block; ++k) {
        float top = wave_max(mine && block == k ? old[j] : 0.f);
        if (k == 0) now0[j] = top = fmaxf(top, own[j]);
        if (block == k) now[j] = top;
      }
      ratio[j] = scale_ratio(old[j], now[j]);
    }
    if (i + 1 < layers) load_scales(pages + next_layer);
    for (int row0 = first; row0 < kept; row0 += kRows) {
      const int row = row0 + in_pass, at = min(row, 63);
      const int64_t d = __shfl(dst_at, at);
      u32x4 y[kUnits];
#pragma unroll
      for (int j = 0; j < kUnits; ++j) {
        const float f = __shfl(ratio[j], at);
        y[j] = x[j];
        if (f != 1.f) y[j] = recode(y[j], f);
      }
      if (row0 + kRows < kept) load(pages, row0 + kRows);
      else if (i + 1 < layers) load(pages + next_layer, first);
      if (row < kept) {
#pragma unroll
        for (int j = 0; j < kUnits; ++j) *(u32x4*)(cache(j, pages) + d + col) = y[j];
      }
    }
#pragma unroll
    for (int j = 0; j < kUnits; ++j) {
      // tokens of the text in the first block, if its scale has grown
      if (held > 0 && now0[j] > own[j]) {
        const float f = scale_ratio(own[j], now0[j]);
        uint8_t* const rows = cache(j, pages) + (page0 * kPage + block0 * each % kPage) * D;
        for (int row = in_pass; row < held; row += kRows) {
          u32x4* const at = (u32x4*)(rows + row * D + col);
          *at = recode(*at, f);
        }
      }
      // (the first row of each block writes its scale)
      if (mine && (lane == first || dst % each == 0)) *scale_at(j, pages + dst_page, dst) = now[j];
    }
  }
}

}  // namespace

hipError_t launch_tree_masks(const TreeMasksParams& p, hipStream_t stream) {
  hipLaunchKernelGGL(tree_masks_kernel, dim3((p.batch + kWaves - 1) / kWaves), dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

hipError_t launch_gqa_keep(GqaKeepParams p, int cus, hipStream_t stream) {
  const int64_t of_layer = (int64_t)p.batch * (2 * p.kv_heads / kUnits);
  p.run = (int)std::min<int64_t>(kMostLayers, std::max<int64_t>(1, of_layer * p.layers / (32 * cus)));
  const int64_t waves = (p.layers + p.run - 1) / p.run * of_layer;
  const dim3 grid((uint32_t)((waves + kWaves - 1) / kWaves));
  if (p.head_dim == 64) hipLaunchKernelGGL(gqa_keep_kernel<64>, grid, dim3(kThreads), 0, stream, p);
  else if (p.head_dim == 128) hipLaunchKernelGGL(gqa_keep_kernel<128>, grid, dim3(kThreads), 0, stream, p);
  else hipLaunchKernelGGL(gqa_keep_kernel<256>, grid, dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace omniattn
