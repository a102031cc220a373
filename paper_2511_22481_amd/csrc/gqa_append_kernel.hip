// New K and V rows of a grouped-query layer into its 8-bit cache.
//
// A block of s tokens of one KV head shares one scale, a power of two: 2^ceil(log2(a / 448)) for the largest finite
// magnitude a of its rows, so that the largest lands in (224, 448].  (A power of two costs e4m3, a floating-point
// format, none of its relative precision, and lets a block's scale grow later: the codes held before are multiplied by
// an exact power of two, and only those that become subnormal are rounded again.)  code = e4m3(x / scale), to nearest
// even; a number that is not finite becomes the NaN code and does not count towards a.
//
// One work group takes one (run of tokens in one block, head, K or V): the run's rows stay in registers between the
// maximum and the rounding, so they are read once.
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

// C: consecutive tokens of the call that a work group looks through for runs that begin there.
template <int D>
__global__ __launch_bounds__(kThreads) void gqa_append_kernel(GqaAppendParams p, int C) {
  constexpr int kPer = D / 8;                // threads that share a row, 8 numbers each
  constexpr int kRows = kThreads / kPer;     // rows of a pass
  constexpr int kPasses = kPage / kRows;     // a run has up to 128 rows
  __shared__ uint32_t tot[2][4];
  const int tid = threadIdx.x, row = tid / kPer, col = (tid % kPer) * 8;
  const int head = blockIdx.x % p.kv_heads, kv = blockIdx.x / p.kv_heads % 2;
  const int i0 = (int)(blockIdx.x / (2 * p.kv_heads)) * C, i1 = min(i0 + C, p.num_tokens);
  const uint16_t* rows = p.rows[kv] + (size_t)head * D + col;
  const int64_t stride = p.stride[kv];
  const int each = p.scale_tokens;
  int parity = 0;
  int before = i0 > 0 ? p.slot_map[i0 - 1] : -1;
  for (int i = i0; i < i1; ++i) {
    const int slot = p.slot_map[i], off = slot % each;
    const bool begins = (uint32_t)slot < p.num_slots && !(off != 0 && before == slot - 1);
    before = slot;
    if (!begins) continue;
    // the run's length: tokens that follow in the call and in the block
    const int most = min(each - off, p.num_tokens - i);
    int r = 1;
    for (; r < most; r += 64) {
      const int k = r + (tid & 63);
      const uint64_t other = __ballot(k >= most || p.slot_map[i + k] != slot + k);
      if (other) {
        r += __builtin_ctzll(other);
        break;
      }
    }
    r = min(r, most);
    u32x4 x[kPasses];
    uint32_t top = 0;
#pragma unroll
    for (int s = 0; s < kPasses; ++s) {
      const int k = s * kRows + row;
      if (s * kRows < r) {  // (uniform)
        x[s] = k < r ? *(const u32x4*)(rows + (int64_t)(i + k) * stride) : u32x4{0, 0, 0, 0};
      }
    }
    const int page = slot / kPage, in_page = slot % kPage;
    float* scale_at = p.scales[kv] + ((size_t)page * p.kv_heads + head) * (kPage / each) + in_page / each;
    const float old = off > 0 ? *scale_at : 0.f;
#pragma unroll
    for (int s = 0; s < kPasses; ++s) {
      if (s * kRows < r) {
#pragma unroll
        for (int j = 0; j < 4; ++j) top = max(top, max(finite_bits(x[s][j]), finite_bits(x[s][j] >> 16)));
      }
    }
    for (int d = 1; d < 64; d *= 2) top = max(top, (uint32_t)__shfl_xor(top, d));
    if ((tid & 63) == 0) tot[parity][tid >> 6] = top;
    __syncthreads();  // (also: every thread has read the old scale)
    top = max(max(tot[parity][0], tot[parity][1]), max(tot[parity][2], tot[parity][3]));
    parity ^= 1;
    const float scale = fmaxf(old, block_scale(top)), inv = scale > 0.f ? 1.f / scale : 0.f;
    uint8_t* codes = p.cache[kv] + (((size_t)page * p.kv_heads + head) * kPage + in_page) * D + col;
#pragma unroll
    for (int s = 0; s < kPasses; ++s) {
      const int k = s * kRows + row;
      if (k < r) *(u32x2*)(codes + (size_t)k * D) = u32x2{encode_words(x[s][0], x[s][1], inv), encode_words(x[s][2], x[s][3], inv)};
    }
    if (off > 0 && scale > old) {  // tokens that the block held before take the grown scale
      const float ratio = old / scale;
      for (int k = row - off; k < 0; k += kRows) {
        u32x2* at = (u32x2*)(codes + (ptrdiff_t)k * D);
        const u32x2 c = *at;
        *at = u32x2{recode(c[0], ratio), recode(c[1], ratio)};
      }
    }
    if (tid == 0) *scale_at = scale;
  }
}

}  // namespace

hipError_t launch_gqa_append(const GqaAppendParams& p, hipStream_t stream) {
  if (p.num_tokens <= 0) return hipSuccess;
  // About 8192 work groups, or fewer; no more tokens to one than its scale's block has.
  int C = 1;
  while (C < p.scale_tokens && (int64_t)p.num_tokens * p.kv_heads * 2 > (int64_t)8192 * C) C *= 2;
  const dim3 grid((uint32_t)(((int64_t)p.num_tokens + C - 1) / C * p.kv_heads * 2));
  if (p.head_dim == 64) hipLaunchKernelGGL(gqa_append_kernel<64>, grid, dim3(kThreads), 0, stream, p, C);
  else if (p.head_dim == 128) hipLaunchKernelGGL(gqa_append_kernel<128>, grid, dim3(kThreads), 0, stream, p, C);
  else hipLaunchKernelGGL(gqa_append_kernel<256>, grid, dim3(kThreads), 0, stream, p, C);
  return hipGetLastError();
}

}  // namespace omniattn
