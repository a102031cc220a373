// New K and V rows of a grouped-query layer into its 8-bit cache.
//
// A block of s tokens of one KV head shares one scale, a power of two: 2^ceil(log2(a / 448)) for the largest finite
// magnitude a of its rows, so that the largest lands in (224, 448].  (A power of two costs e4m3, a floating-point
// format, none of its relative precision, and lets a block's scale grow later: the codes held before are multiplied by
// an exact power of two, and only those that become subnormal are rounded again.)  code = e4m3(x / scale), to nearest
// even; a number that is not finite becomes the NaN code and does not count towards a.
//
// A work group looks through C consecutive tokens of the call for runs (tokens that follow one another in one block) that begin
// there, for one head and K or V.  A long run is the work of all its waves: the rows stay in registers between the maximum
// and the rounding, so they are read once.  Runs that fit one pass of a wave are dealt out to the waves, and single tokens (a
// decode step's) to the groups of lanes that hold a row, so that the 32 of a mixed step's C are two passes and not eight.
//
// What bounds it: 65536 tokens of 8 heads of 128 (302 MB) 67 us, 4.5 TB/s of the 4.78 that a copy reaches.  A decode step's 64 tokens 4.2 us: a
// launch, and slots, rows and scales one behind the other.  133 requests with chunks of prompts (5.7 MB) 7.6 us: the same, once for
// the single tokens and once or twice for long runs.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "gqa.h"

namespace omniattn {
namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;

constexpr int kThreads = 256;

__device__ __forceinline__ float low(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }

// Bits of a bf16 magnitude that counts: 0 for infinities and NaN.
__device__ __forceinline__ uint32_t finite_bits(uint32_t h) {
  h &= 0x7fffu;
  return h < 0x7f80u ? h : 0u;
}

// Scale of a block whose largest magnitude has these bf16 bits: a = 1.m 2^e fits 448 = 1.75 * 2^8 times 2^(e - 8), or
// 2^(e - 7) where 1.m > 1.75.  Not below 2^-126, so that its reciprocal is finite and normal.
__device__ __forceinline__ float block_scale(uint32_t bits) {
  if (bits == 0) return 0.f;
  const int e = (int)(bits >> 7) + ((bits & 0x7f) > 0x60 ? -7 : -8);  // (biased; subnormal a: below the floor)
  return __builtin_bit_cast(float, (uint32_t)max(e, 1) << 23);
}

__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}
__device__ __forceinline__ uint32_t encode_words(uint32_t w0, uint32_t w1, float inv) {
  return encode4(low(w0) * inv, high(w0) * inv, low(w1) * inv, high(w1) * inv);
}
__device__ __forceinline__ uint32_t recode(uint32_t codes, float ratio) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(codes, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
  return encode4(a[0] * ratio, a[1] * ratio, b[0] * ratio, b[1] * ratio);
}

// What a run's block and cache are, for one thread's eight columns.
struct Run {
  uint8_t* codes;   // of the run's first token
  float* scale;
  int off;          // tokens that the block has before the run
};

template <int D>
__device__ __forceinline__ Run run_at(const GqaAppendParams& p, int kv, int head, int slot, int col) {
  const int page = slot / kPage, in_page = slot % kPage, each = p.scale_tokens;
  const size_t ph = (size_t)page * p.kv_heads + head;
  return Run{p.cache[kv] + (ph * kPage + in_page) * D + col, p.scales[kv] + ph * (kPage / each) + in_page / each, slot % each};
}

// The earlier tokens of a block whose scale has grown; `row` of `rows` threads that share the work by rows.
template <int D>
__device__ __forceinline__ void regrow(const Run& run, float old, float scale, int row, int rows) {
  if (run.off > 0 && scale > old) {
    const float ratio = old / scale;
    constexpr int kBatch = 8;  // rows under way: one at a time, a single token late in its block would wait for each of them in turn
    for (int k0 = row - run.off; k0 < 0; k0 += kBatch * rows) {
      u32x2 c[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) c[i] = *(const u32x2*)(run.codes + (ptrdiff_t)min(k0 + i * rows, -1) * D);
#pragma unroll
      for (int i = 0; i < kBatch; ++i)
        if (k0 + i * rows < 0) *(u32x2*)(run.codes + (ptrdiff_t)(k0 + i * rows) * D) = u32x2{recode(c[i][0], ratio), recode(c[i][1], ratio)};
    }
  }
}

__device__ __forceinline__ uint32_t largest(const u32x4& x) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) top = max(top, max(finite_bits(x[j]), finite_bits(x[j] >> 16)));
  return top;
}
// Largest of each LANES neighbouring lanes (8, 16, 32 or 64), in all of them.
template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
#define OMNIATTN_MAX(ctrl) x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, 0xf, 0xf, true))
  OMNIATTN_MAX(0xb1);   // the other of two
  OMNIATTN_MAX(0x4e);   // the other two of four
  OMNIATTN_MAX(0x141);  // eight, mirrored
  if constexpr (LANES >= 16) OMNIATTN_MAX(0x140);  // sixteen, mirrored
#undef OMNIATTN_MAX
  if constexpr (LANES >= 32) {
    const auto y = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max(y[0], y[1]);
  }
  if constexpr (LANES >= 64) {
    const auto y = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    x = max(y[0], y[1]);
  }
  return x;
}

template <int D>
__global__ __launch_bounds__(kThreads) void gqa_append_kernel(GqaAppendParams p, int C) {
  constexpr int kPer = D / 8;                // threads that share a row, 8 numbers each
  constexpr int kWaveRows = 64 / kPer;       // rows of a wave's pass: runs up to this long are one wave's
  constexpr int kRows = kThreads / kPer;     // rows of the work group's pass
  constexpr int kPasses = kPage / kRows;     // a run has up to 128 rows
  __shared__ uint32_t tot[2][4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = tid / kPer, col = (tid % kPer) * 8;
  const int head = blockIdx.x % p.kv_heads, kv = blockIdx.x / p.kv_heads % 2;
  const int i0 = (int)(blockIdx.x / (2 * p.kv_heads)) * C, many = min(C, p.num_tokens - i0);
  const uint16_t* rows = p.rows[kv] + (size_t)head * D + col;
  const int64_t stride = p.stride[kv];
  const int each = p.scale_tokens;

  // Slots of the tokens looked through and of the 128 behind them, four to a lane; bit i of `next`: token i0 + i continues the
  // run of the one before it.  (Every wave does this for itself.)
  int slot[4];
  uint64_t next[4], valid[2];
  {
    const int left = p.num_tokens - i0, want = min(left, C + kPage);
    int prev = i0 > 0 ? p.slot_map[i0 - 1] : -1;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int i = w * 64 + lane;
      slot[w] = i < want ? p.slot_map[i0 + i] : -1;
    }
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      int before = __shfl_up(slot[w], 1);
      if (lane == 0) before = prev;
      prev = __builtin_amdgcn_readlane(slot[w], 63);
      const bool in_cache = (uint32_t)slot[w] < p.num_slots;
      next[w] = __ballot(in_cache && before >= 0 && slot[w] == before + 1 && slot[w] % each != 0);
      if (w < 2) valid[w] = __ballot(in_cache && w * 64 + lane < many);
    }
  }
  // length of the run that begins at token i (of those looked through)
  auto length = [&](int i, int off) {
    int r = 1;
    for (int j = i + 1; j < 256; j = (j | 63) + 1) {
      const uint64_t rest = ~(next[j >> 6] >> (j & 63));
      const int ones = rest ? __builtin_ctzll(rest) : 64;
      r += min(ones, 64 - (j & 63));
      if (ones < 64 - (j & 63)) break;
    }
    return min(r, each - off);
  };
  auto slot_of = [&](int i) { return __builtin_amdgcn_readlane(i < 64 ? slot[0] : slot[1], i & 63); };
  uint64_t begins[2], single[2];
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    begins[w] = valid[w] & ~next[w];
    single[w] = begins[w] & ~(next[w] >> 1 | next[w + 1] << 63);
    begins[w] &= ~single[w];
  }

  // single tokens, kRows at a time
  int count = 0, my_token = -1, my_slot = 0;
  auto append_singles = [&] {
    if (my_token >= 0) {
      const u32x4 x = *(const u32x4*)(rows + (int64_t)my_token * stride);
      const Run run = run_at<D>(p, kv, head, my_slot, col);
      const float old = run.off > 0 ? *run.scale : 0.f;
      const float scale = fmaxf(old, block_scale(lanes_max<kPer>(largest(x)))), inv = scale > 0.f ? 1.f / scale : 0.f;
      *(u32x2*)run.codes = u32x2{encode_words(x[0], x[1], inv), encode_words(x[2], x[3], inv)};
      regrow<D>(run, old, scale, 0, 1);
      if (col == 0) *run.scale = scale;
    }
    my_token = -1;
  };
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    for (uint64_t rest = single[w]; rest; rest &= rest - 1) {
      const int i = w * 64 + __builtin_ctzll(rest), s0 = slot_of(i);
      if (count % kRows == row) {
        my_token = i0 + i;
        my_slot = s0;
      }
      if (++count % kRows == 0) append_singles();
    }
  }
  if (count % kRows) append_singles();

  // long runs
  int parity = 0, turn = 0;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    for (uint64_t begin = begins[w]; begin; begin &= begin - 1) {
      const int i = w * 64 + __builtin_ctzll(begin), s0 = slot_of(i);
      const int r = length(i, s0 % each);
      if (r <= kWaveRows) continue;
      u32x4 x[kPasses];
#pragma unroll
      for (int s = 0; s < kPasses; ++s) {
        const int k = s * kRows + row;
        if (s * kRows < r) x[s] = k < r ? *(const u32x4*)(rows + (int64_t)(i0 + i + k) * stride) : u32x4{0, 0, 0, 0};
      }
      const Run run = run_at<D>(p, kv, head, s0, col);
      const float old = run.off > 0 ? *run.scale : 0.f;
      uint32_t top = 0;
#pragma unroll
      for (int s = 0; s < kPasses; ++s)
        if (s * kRows < r) top = max(top, largest(x[s]));
      top = lanes_max<64>(top);
      if (lane == 0) tot[parity][wave] = top;
      __syncthreads();  // (also: every thread has read the old scale)
      top = max(max(tot[parity][0], tot[parity][1]), max(tot[parity][2], tot[parity][3]));
      parity ^= 1;
      const float scale = fmaxf(old, block_scale(top)), inv = scale > 0.f ? 1.f / scale : 0.f;
#pragma unroll
      for (int s = 0; s < kPasses; ++s) {
        const int k = s * kRows + row;
        if (k < r) *(u32x2*)(run.codes + (size_t)k * D) = u32x2{encode_words(x[s][0], x[s][1], inv), encode_words(x[s][2], x[s][3], inv)};
      }
      regrow<D>(run, old, scale, row, kRows);
      if (tid == 0) *run.scale = scale;
    }
  }
  // short ones
  const int wrow = lane / kPer;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    for (uint64_t begin = begins[w]; begin; begin &= begin - 1) {
      const int i = w * 64 + __builtin_ctzll(begin), s0 = slot_of(i);
      const int r = length(i, s0 % each);
      if (r > kWaveRows || (turn++ & 3) != wave) continue;
      const u32x4 x = wrow < r ? *(const u32x4*)(rows + (int64_t)(i0 + i + wrow) * stride) : u32x4{0, 0, 0, 0};
      const Run run = run_at<D>(p, kv, head, s0, col);
      const float old = run.off > 0 ? *run.scale : 0.f;
      const float scale = fmaxf(old, block_scale(lanes_max<64>(largest(x)))), inv = scale > 0.f ? 1.f / scale : 0.f;
      if (wrow < r) *(u32x2*)(run.codes + (size_t)wrow * D) = u32x2{encode_words(x[0], x[1], inv), encode_words(x[2], x[3], inv)};
      regrow<D>(run, old, scale, wrow, kWaveRows);
      if (lane == 0) *run.scale = scale;
    }
  }
}

}  // namespace

hipError_t launch_gqa_append(const GqaAppendParams& p, hipStream_t stream) {
  if (p.num_tokens <= 0) return hipSuccess;
  // 1024 to 2048 work groups (looking through the slots costs each of them more than its rows do), of no more tokens than their scale's block
  // has.  us, 133 requests with chunks, 7 heads / 65536 tokens, 8 heads: at least 1024 groups 8.0 / 66.3, 2048 9.4 / 66.3, 4096 12.3 / 66.4.
  int C = 1;
  while (C < p.scale_tokens && (int64_t)p.num_tokens * p.kv_heads * 2 > (int64_t)1024 * C) C *= 2;
  const dim3 grid((uint32_t)(((int64_t)p.num_tokens + C - 1) / C * p.kv_heads * 2));
  if (p.head_dim == 64) hipLaunchKernelGGL(gqa_append_kernel<64>, grid, dim3(kThreads), 0, stream, p, C);
  else if (p.head_dim == 128) hipLaunchKernelGGL(gqa_append_kernel<128>, grid, dim3(kThreads), 0, stream, p, C);
  else hipLaunchKernelGGL(gqa_append_kernel<256>, grid, dim3(kThreads), 0, stream, p, C);
  return hipGetLastError();
}

}  // namespace omniattn
