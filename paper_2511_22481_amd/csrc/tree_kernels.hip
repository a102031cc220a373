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

// A wave to a request, a lane to a node.  Every pass doubles the way that a set reaches up.
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
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x = fmaxf(x, __shfl_xor(x, d));
  return x;
}
__device__ __forceinline__ float scale_ratio(float old, float now) { return now > 0.f ? old / now : 1.f; }

// A wave to a (layer, request, KV head, K or V).  Rows go up in order, kRows at a time: a row's source lies at or behind its place, so what a pass
// writes is no later pass's source, and within a pass all loads are done before the first store.
template <int D>
__global__ __launch_bounds__(kThreads) void gqa_keep_kernel(GqaKeepParams p) {
  constexpr int kLanes = D / 16, kRows = 64 / kLanes;  // lanes of a row, 16 codes each; rows of a pass
  const int lane = threadIdx.x & 63, each = p.scale_tokens, blocks = kPage / each;
  int64_t id = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kv = id % 2;
  id /= 2;
  const int head = id % p.kv_heads;
  id /= p.kv_heads;
  const int b = id % p.batch, layer = (int)(id / p.batch);
  if (layer >= p.layers) return;
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
  const int64_t src_ph = ((int64_t)layer * p.num_pages + table[src / kPage]) * p.kv_heads + head;
  const int64_t dst_ph = ((int64_t)layer * p.num_pages + table[dst / kPage]) * p.kv_heads + head;
  float* const scales = p.scales[kv];
  const float old = scales[src_ph * blocks + src % kPage / each];
  // up to three blocks (64 tokens, 32 to a block)
  const int block0 = (text + first) / each, block = dst / each - block0;
  const int held = text - block0 * each;  // tokens of the text in the first of them, if any
  const int64_t ph0 = __shfl(dst_ph, first);
  const float own = held > 0 ? scales[ph0 * blocks + block0 * each % kPage / each] : 0.f;
  float now = 0.f, now0 = 0.f;
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    float top = wave_max(mine && block == k ? old : 0.f);
    if (k == 0) now0 = top = fmaxf(top, own);
    if (block == k) now = top;
  }
  const float ratio = scale_ratio(old, now);
  uint8_t* const cache = p.cache[kv];
  const int64_t src_at = (src_ph * kPage + src % kPage) * D, dst_at = (dst_ph * kPage + dst % kPage) * D;
  const int col = lane % kLanes * 16;
  for (int row0 = first; row0 < kept; row0 += kRows) {
    const int row = row0 + lane / kLanes, at = min(row, 63);
    const int64_t s = __shfl(src_at, at), d = __shfl(dst_at, at);
    const float f = __shfl(ratio, at);
    if (row < kept) {
      u32x4 x = *(const u32x4*)(cache + s + col);
      if (f != 1.f) x = recode(x, f);
      *(u32x4*)(cache + d + col) = x;
    }
  }
  // tokens of the text in the first block, if its scale has grown
  if (held > 0 && now0 > own) {
    const float f = scale_ratio(own, now0);
    uint8_t* const rows = cache + (ph0 * kPage + block0 * each % kPage) * D;
    for (int row = lane / kLanes; row < held; row += kRows) {
      u32x4* const at = (u32x4*)(rows + row * D + col);
      *at = recode(*at, f);
    }
  }
  // (the first row of each block writes its scale)
  if (mine && (lane == first || dst % each == 0)) scales[dst_ph * blocks + dst % kPage / each] = now;
}

}  // namespace

hipError_t launch_tree_masks(const TreeMasksParams& p, hipStream_t stream) {
  hipLaunchKernelGGL(tree_masks_kernel, dim3((p.batch + kWaves - 1) / kWaves), dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

hipError_t launch_gqa_keep(const GqaKeepParams& p, hipStream_t stream) {
  const dim3 grid((uint32_t)(((int64_t)p.layers * p.batch * p.kv_heads * 2 + kWaves - 1) / kWaves));
  if (p.head_dim == 64) hipLaunchKernelGGL(gqa_keep_kernel<64>, grid, dim3(kThreads), 0, stream, p);
  else if (p.head_dim == 128) hipLaunchKernelGGL(gqa_keep_kernel<128>, grid, dim3(kThreads), 0, stream, p);
  else hipLaunchKernelGGL(gqa_keep_kernel<256>, grid, dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace omniattn
