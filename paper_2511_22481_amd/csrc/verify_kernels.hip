// Which drafted tokens stay.
//
// Node i of a request's tree has the target's logits l for the token behind it; p = softmax(l / T).  A token y is chosen for every node by
// itself, so that all rows of the call are looked at in parallel; the walk from node 0 to the child that holds y, and so on, comes last.
//   T = 0:           y = argmax l, the first of equals.
//   no draft's q:    y = the first v with p_0 + .. + p_v > u1 (p_0 + .. + p_V-1).
//   q given:         the node's first child x was drawn from q.  It is taken if u0 q(x) < p(x); otherwise y is found as above with max(p - q, 0)
//                    in p's place, so that y is distributed as p either way (where that is 0 everywhere, p itself).
// A child that holds y (the first such) is next; without one, y is the text's new last token.
//
// Sums and exponentials are in 64 bits: a border between two tokens that is off by 2^-24 of the whole gives another token once in some
// thousand draws from a large vocabulary, and then the same inputs would give other tokens with another order of summation.  (2^x is a
// Taylor polynomial of degree 10 on [-1/2, 1/2], off by at most 3e-13.)
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "verify.h"

namespace omniattn {
namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef u32x4 __attribute__((aligned(2))) u32x4_any;  // (rows begin where they will)

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kPickThreads = 1024;
constexpr int kNodes = OMNIATTN_TREE_NODES;
constexpr int kTile = 512, kTiles = kVerifyColumns / kTile;  // columns of a wave's tile, 8 neighbours to a lane
constexpr double kLog2e = 1.4426950408889634074, kLn2 = 0.69314718055994530942;

// 2^x for x <= 0; 0 for NaN and below 2^-1100.
__device__ __forceinline__ double exp2_64(double x) {
  x = fmax(x, -1100.0);
  const double n = rint(x), f = x - n;
  // ln(2)^k / k!
  double y = 7.0549116208011233e-9;
  y = fma(y, f, 1.0178086009239699e-7);
  y = fma(y, f, 1.3215486790144309e-6);
  y = fma(y, f, 1.5252733804059841e-5);
  y = fma(y, f, 1.5403530393381609e-4);
  y = fma(y, f, 1.3333558146428443e-3);
  y = fma(y, f, 9.6181291076284772e-3);
  y = fma(y, f, 5.5504108664821580e-2);
  y = fma(y, f, 2.4022650695910071e-1);
  y = fma(y, f, 6.9314718055994531e-1);
  y = fma(y, f, 1.0);
  return ldexp(y, (int)n);
}

__device__ __forceinline__ double shfl64(double x, int lane) {
  const int64_t v = __builtin_bit_cast(int64_t, x);
  const uint32_t lo = (uint32_t)__shfl((int)v, lane), hi = (uint32_t)__shfl((int)(v >> 32), lane);
  return __builtin_bit_cast(double, (int64_t)((uint64_t)hi << 32 | lo));
}
__device__ __forceinline__ double shfl_up64(double x, int d) {
  const int64_t v = __builtin_bit_cast(int64_t, x);
  const uint32_t lo = (uint32_t)__shfl_up((int)v, d), hi = (uint32_t)__shfl_up((int)(v >> 32), d);
  return __builtin_bit_cast(double, (int64_t)((uint64_t)hi << 32 | lo));
}
__device__ __forceinline__ double wave_sum(double x) {  // (every lane has the same one)
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x += shfl64(x, (threadIdx.x & 63) ^ d);
  return x;
}
__device__ __forceinline__ double wave_sum_up_to(double x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const double y = shfl_up64(x, d);
    if (lane >= d) x += y;
  }
  return x;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x = fmaxf(x, __shfl_xor(x, d));
  return x;
}
__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x = min(x, __shfl_xor(x, d));
  return x;
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

struct Nodes {
  int begin, n;
};
__device__ __forceinline__ Nodes nodes_of(const VerifyParams& p, int b) {
  const int lo = p.q_start ? p.q_start[b] : b, hi = p.q_start ? p.q_start[b + 1] : b + 1;
  Nodes r;
  r.begin = min(max(lo, 0), p.num_tokens);
  r.n = min(max(hi, r.begin), p.num_tokens) - r.begin;
  return r;
}
// The request that row `row` of the call belongs to, or -1.
__device__ __forceinline__ int request_of(const VerifyParams& p, int row) {
  if (!p.q_start) return row < p.batch ? row : -1;
  const int lane = threadIdx.x & 63;
  int ended = 0;
  for (int b0 = 0; b0 < p.batch; b0 += 64) ended += __popcll(__ballot(b0 + lane < p.batch && p.q_start[b0 + lane + 1] <= row));
  return ended < p.batch && row >= p.q_start[0] ? ended : -1;
}
// Factor of a logit's distance to the largest, in base 2.  (A request without a temperature takes the likeliest token; its probabilities are those at 1.)
__device__ __forceinline__ double factor_of(float T) { return T > 0.f ? kLog2e / (double)T : kLog2e; }

// Eight neighbouring logits; those from column `stop` on are -inf.
template <typename T>
__device__ __forceinline__ void load8(float (&x)[8], const void* row, int col, int stop) {
  const T* at = (const T*)row + col;
  if (col + 8 <= stop) {
    if constexpr (sizeof(T) == 2) {
      const u32x4 w = *(const u32x4_any*)at;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __builtin_bit_cast(float, i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    } else {
      const u32x4 lo = *(const u32x4_any*)at, hi = *(const u32x4_any*)(at + 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __builtin_bit_cast(float, i < 4 ? lo[i] : hi[i - 4]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(T) == 2) x[i] = col + i < stop ? __builtin_bit_cast(float, (uint32_t)*(const uint16_t*)(at + i) << 16) : -INFINITY;
      else x[i] = col + i < stop ? at[i] : -INFINITY;
    }
  }
}
__device__ __forceinline__ double weight(float l, double top, double c) { return exp2_64(((double)l - top) * c); }

// A wave to kVerifyColumns columns of a row.
template <typename T>
__global__ __launch_bounds__(kThreads) void verify_sums_kernel(VerifyParams p) {
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * kWaves + uniform(threadIdx.x >> 6);
  const int row = (int)(id / p.num_parts), part = (int)(id % p.num_parts);
  if (row >= p.num_tokens) return;
  const void* const logits = (const T*)p.logits + row * p.stride;
  float x[kTiles][8];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) load8<T>(x[t], logits, part * kVerifyColumns + t * kTile + lane * 8, p.vocab);
  const int b = request_of(p, row);
  if (b < 0) return;
  const float T0 = p.temperature[b];
  float top = -INFINITY;
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, x[t][i]);
  top = wave_max(top);
  const double c = factor_of(T0), m = top;
  double sum = 0.0;
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += weight(x[t][i], m, c);
  sum = wave_sum(sum);
  int best = 0x7fffffff;
  if (!(T0 > 0.f) || top == INFINITY) {
#pragma unroll
    for (int t = kTiles - 1; t >= 0; --t)
#pragma unroll
      for (int i = 7; i >= 0; --i)
        if (x[t][i] == top) best = part * kVerifyColumns + t * kTile + lane * 8 + i;
    best = wave_min(best);
  }
  if (lane == 0) p.parts[(int64_t)row * p.num_parts + part] = VerifyPart{sum, top, best};
}

// A row's maximum, the first column that has it, and the sum of its weights.
struct Row {
  double top, sum;
  float ftop;
  int best;
};
__device__ __forceinline__ Row row_of(const VerifyParams& p, int row, double c) {
  const int lane = threadIdx.x & 63;
  const VerifyPart* const parts = p.parts + (int64_t)row * p.num_parts;
  Row r;
  r.ftop = -INFINITY;
  for (int k = lane; k < p.num_parts; k += 64) r.ftop = fmaxf(r.ftop, parts[k].top);
  r.ftop = wave_max(r.ftop);
  r.top = r.ftop;
  r.sum = 0.0;
  r.best = 0x7fffffff;
  for (int k = lane; k < p.num_parts; k += 64) {
    const VerifyPart e = parts[k];
    r.sum += e.sum * weight(e.top, r.top, c);
    if (e.top == r.ftop) r.best = min(r.best, e.best);
  }
  r.sum = wave_sum(r.sum);
  r.best = wave_min(r.best);
  return r;
}
template <typename T>
__device__ __forceinline__ float logit_at(const VerifyParams& p, int row, int col) {
  const T x = ((const T*)p.logits)[row * p.stride + col];
  if constexpr (sizeof(T) == 2) return __builtin_bit_cast(float, (uint32_t)x << 16);
  else return x;
}

// What becomes of a node whose first child (of token `child`) was drawn from q.  Rows with infinite logits: the first such token has p = 1.
template <typename T>
__device__ __forceinline__ bool takes_child(const VerifyParams& p, const Row& r, int row, int child, double c) {
  if ((uint32_t)child >= (uint32_t)p.vocab) return false;
  double chance;
  if (r.ftop == INFINITY) chance = child == r.best ? 1.0 : 0.0;
  else chance = r.sum > 0.0 ? weight(logit_at<T>(p, row, child), r.top, c) / r.sum : 0.0;
  return (double)p.uniforms[2 * (int64_t)row] * (double)p.draft_probs[row * p.draft_stride + child] < chance;
}
// max(p - q, 0) of eight neighbours.
template <typename T>
__device__ __forceinline__ void rest8(double (&w)[8], const VerifyParams& p, const Row& r, int row, int col, double c) {
  float x[8], q[8];
  load8<T>(x, (const T*)p.logits + row * p.stride, col, p.vocab);
  load8<float>(q, p.draft_probs + row * p.draft_stride, col, p.vocab);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    double chance;
    if (r.ftop == INFINITY) chance = col + i == r.best ? 1.0 : 0.0;
    else chance = r.sum > 0.0 ? weight(x[i], r.top, c) / r.sum : 0.0;
    w[i] = col + i < p.vocab ? fmax(chance - (double)q[i], 0.0) : 0.0;
  }
}

// Sums of max(p - q, 0), of the rows whose first child is refused.  A wave to kVerifyColumns columns.
template <typename T>
__global__ __launch_bounds__(kThreads) void verify_rest_kernel(VerifyParams p) {
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * kWaves + uniform(threadIdx.x >> 6);
  const int row = (int)(id / p.num_parts), part = (int)(id % p.num_parts);
  if (row >= p.num_tokens) return;
  const int b = request_of(p, row);
  if (b < 0) return;
  const float T0 = p.temperature[b];
  const Nodes r = nodes_of(p, b);
  if (!(T0 > 0.f) || r.n > kNodes) return;
  const uint64_t children = __ballot(lane < r.n && lane > row - r.begin && p.parents[r.begin + min(lane, r.n - 1)] == row - r.begin);
  if (!children) return;
  const double c = factor_of(T0);
  const Row all = row_of(p, row, c);
  if (takes_child<T>(p, all, row, p.tokens[r.begin + __builtin_ctzll(children)], c)) return;
  double sum = 0.0;
#pragma unroll 1
  for (int t = 0; t < kTiles; ++t) {
    double w[8];
    rest8<T>(w, p, all, row, part * kVerifyColumns + t * kTile + lane * 8, c);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += w[i];
  }
  sum = wave_sum(sum);
  if (lane == 0) p.rest[(int64_t)row * p.num_parts + part] = sum;
}

// First column at which the running sum of a row's weights is above `border`.  part_sum(k): the sum of part k; weights8(w, col): of eight
// neighbours.  (The last column with a weight if rounding leaves none above the border.)
template <typename F, typename G>
__device__ __forceinline__ int find(const VerifyParams& p, double border, F part_sum, G weights8) {
  const int lane = threadIdx.x & 63;
  double before = 0.0;
  int part = -1;
  double at_part = 0.0;
  for (int k0 = 0; k0 < p.num_parts; k0 += 64) {
    const int k = k0 + lane;
    const double s = k < p.num_parts ? part_sum(k) : 0.0, upto = wave_sum_up_to(s);
    const uint64_t above = __ballot(before + upto > border), some = __ballot(s > 0.0);
    if (above & some) {
      const int i = __builtin_ctzll(above & some);
      part = k0 + i;
      at_part = before + shfl64(upto, i) - shfl64(s, i);
      break;
    }
    if (some) {
      const int i = 63 - __builtin_clzll(some);
      part = k0 + i;
      at_part = before + shfl64(upto, i) - shfl64(s, i);
    }
    before += shfl64(upto, 63);
  }
  if (part < 0) return -1;
  int last = -1;
#pragma unroll 1
  for (int t = 0; t < kTiles; ++t) {
    const int col = part * kVerifyColumns + t * kTile + lane * 8;
    double w[8], s = 0.0;
    weights8(w, col);
#pragma unroll
    for (int i = 0; i < 8; ++i) s += w[i];
    const double upto = wave_sum_up_to(s);
    double run = at_part + upto - s;
    int hit = 0x7fffffff, mine = -1;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      run += w[i];
      if (w[i] > 0.0) {
        mine = col + i;
        if (run > border) hit = min(hit, col + i);
      }
    }
    hit = wave_min(hit);
    if (hit != 0x7fffffff) return hit;
    last = max(last, -wave_min(-mine));
    at_part += shfl64(upto, 63);
  }
  return last;
}

// A work group to a request: its waves choose the tokens, a node each at a time, then one walks down the tree.
template <typename T>
__global__ __launch_bounds__(kPickThreads) void verify_pick_kernel(VerifyParams p) {
  __shared__ int next[kNodes], chosen[kNodes];
  __shared__ float chance[kNodes];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), b = blockIdx.x;
  const Nodes r = nodes_of(p, b);
  if (r.n > kNodes) {
    for (int t = threadIdx.x; t < r.n; t += kPickThreads) {
      p.path[r.begin + t] = -1;
      p.out_tokens[r.begin + t] = -1;
      if (p.logprobs) p.logprobs[r.begin + t] = 0.f;
    }
    if (threadIdx.x == 0) p.dropped[b] = r.n;
    return;
  }
  const float T0 = p.temperature[b];
  const double c = factor_of(T0);
  const int parent = lane < r.n ? p.parents[r.begin + lane] : -1, token = lane < r.n ? p.tokens[r.begin + lane] : -1;
  for (int i = wave; i < r.n; i += kPickThreads / 64) {
    const int row = r.begin + i;
    const Row all = row_of(p, row, c);
    const uint64_t children = __ballot(lane > i && lane < r.n && parent == i);
    int y, go = -1;
    if (!(T0 > 0.f)) {
      y = all.ftop == -INFINITY ? -1 : all.best;
    } else if (p.draft_probs && children && takes_child<T>(p, all, row, __shfl(token, __builtin_ctzll(children)), c)) {
      go = __builtin_ctzll(children);
      y = __shfl(token, go);
    } else {
      y = -1;
      const double u = p.uniforms[2 * (int64_t)row + 1];
      if (p.draft_probs && children) {
        const double* const rest = p.rest + (int64_t)row * p.num_parts;
        double sum = 0.0;
        for (int k = lane; k < p.num_parts; k += 64) sum += rest[k];
        sum = wave_sum(sum);
        if (sum > 0.0) y = find(p, u * sum, [&](int k) { return rest[k]; }, [&](double (&w)[8], int col) { rest8<T>(w, p, all, row, col, c); });
      }
      if (y < 0) {
        if (all.ftop == INFINITY) y = all.best;
        else if (all.sum > 0.0) {
          const VerifyPart* const parts = p.parts + (int64_t)row * p.num_parts;
          y = find(p, u * all.sum, [&](int k) { return parts[k].sum * weight(parts[k].top, all.top, c); },
                   [&](double (&w)[8], int col) {
                     float x[8];
                     load8<T>(x, (const T*)p.logits + row * p.stride, col, p.vocab);
#pragma unroll
                     for (int i = 0; i < 8; ++i) w[i] = weight(x[i], all.top, c);
                   });
        }
      }
    }
    if (go < 0 && y >= 0) {
      const uint64_t same = children & __ballot(token == y);
      if (same) go = __builtin_ctzll(same);
    }
    if (lane == 0) {
      next[i] = go;
      chosen[i] = y;
      if (y < 0) chance[i] = 0.f;
      else if (all.ftop == INFINITY) chance[i] = y == all.best ? 0.f : -INFINITY;
      else chance[i] = (float)((((double)logit_at<T>(p, row, y) - all.top) * c - log2(all.sum)) * kLn2);
    }
  }
  __syncthreads();
  if (wave) return;
  // lane k takes the k-th node of the path
  const int my_next = lane < r.n ? next[lane] : -1;
  int kept = 0, node = -1;
  for (int at = r.n > 0 ? 0 : -1; at >= 0; at = __builtin_amdgcn_readlane(my_next, at)) {
    if (lane == kept) node = at;
    ++kept;
  }
  if (lane < r.n) {
    p.path[r.begin + lane] = node;
    p.out_tokens[r.begin + lane] = node >= 0 ? chosen[node] : -1;
    if (p.logprobs) p.logprobs[r.begin + lane] = node >= 0 ? chance[node] : 0.f;
  }
  if (lane == 0) p.dropped[b] = r.n - kept;
}

template <typename T>
hipError_t start(const VerifyParams& p, hipStream_t stream) {
  const dim3 grid((uint32_t)(((int64_t)p.num_tokens * p.num_parts + kWaves - 1) / kWaves));
  if (p.num_tokens > 0) {
    hipLaunchKernelGGL(verify_sums_kernel<T>, grid, dim3(kThreads), 0, stream, p);
    if (p.draft_probs) hipLaunchKernelGGL(verify_rest_kernel<T>, grid, dim3(kThreads), 0, stream, p);
  }
  hipLaunchKernelGGL(verify_pick_kernel<T>, dim3(p.batch), dim3(kPickThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_tree_verify(const VerifyParams& p, hipStream_t stream) {
  return p.logits_fp32 ? start<float>(p, stream) : start<uint16_t>(p, stream);
}

}  // namespace omniattn
