// Attention of grouped-query layers over the paged 8-bit cache.
//
// Query token t of a request with L tokens, n of them new, sees the keys j < L - n + t + 1 that the compression rule
// keeps (j < S, or among the last W of them): out = sum_j p_j v_j / sum_j p_j, p_j = exp(scale q.k_j), lse = ln sum p_j.
//
// Work.  The query rows (t, head of the group) of one (request, KV head) are cut into blocks of 16, 32 or 64; a block
// reads the pages that hold kept tokens.  A block counts as many units as it has pages, and kStart.  All units of the call, in
// order of request, KV head and block, are dealt out evenly: work group u of U takes units [u T / U, (u + 1) T / U).  Every work group finds its share by
// itself from the lengths on the device, so the host needs to know nothing but the sizes of the arrays.  A block whose
// pages went to several groups leaves one partial row each, which gqa_combine_kernel joins.
//
// A page.  The four waves take 32 of its 128 tokens each and keep a running maximum, sum and output of their own; they meet
// only at the end of a block's share.  K rows come from memory in the operand order of S^T = K Q^T (16x16x32 bf16 matrix
// instructions; an e4m3 code is exact in bf16), V rows as 8 tokens x D/16 columns per lane, which a byte permutation turns
// into the operand of O^T += V^T P^T (f16: exact for the codes, and 2^-11 relative for the weights, which the reference
// scales into [0, 2^15]).  The contraction's order of tokens is free, so P^T is what S^T's layout already gives each lane.
// No LDS and no barrier in the loop.  A block's scale is one number per wave and page: K's goes into the softmax factor,
// V's multiplies the page's product when it is added.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "decode_common.h"
#include "gqa.h"

namespace omniattn {
namespace {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;

constexpr int kThreads = 256;
constexpr int kWaveTokens = 32;
// Work groups of a compute unit, as far as their registers allow.
constexpr int groups_per_cu(int head_dim, int row_tiles) { return head_dim * row_tiles <= 64 ? 4 : head_dim * row_tiles <= 128 ? 2 : head_dim * row_tiles <= 256 ? 2 : 1; }
// Weights are 2^(s - m + kLift) for the reference m, which a logit (log2) may exceed by kSlack before it is raised: the largest
// weight is at most 2^15 (f16 holds 65504), and weights keep full precision down to 2^-25 of the largest.
constexpr float kLift = 11.f, kSlack = 4.f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// What a block costs beside its pages, in pages: its query, the meeting of the waves, its results.
constexpr int kStart = 2;

// What a request brings: its tokens, its first query token and how many it has.
struct Request {
  int L, begin, n;
};
__device__ __forceinline__ Request request_of(const GqaDecodeParams& p, int b) {
  Request r;
  r.L = min(max(p.seq_lens[b], 0), p.max_pages * kPage);
  const int lo = p.q_start ? p.q_start[b] : b, hi = p.q_start ? p.q_start[b + 1] : b + 1;
  r.begin = min(max(lo, 0), p.num_queries);
  r.n = min(max(hi, r.begin), p.num_queries) - r.begin;
  return r;
}
// Pages of a block of query rows: the union of its queries' kept sets.
struct Block {
  int t0, t1;  // its query tokens, both included
  TileLayout pages;
  __device__ __forceinline__ int units() const { return kStart + pages.count(); }
};
template <int ROWS>
__device__ __forceinline__ Block block_of(const GqaDecodeParams& p, const Request& r, int rb) {
  Block k;
  k.t0 = rb * ROWS / p.group;
  k.t1 = min(r.n - 1, ((rb + 1) * ROWS - 1) / p.group);
  k.pages = tile_layout(r.L - r.n + k.t1 + 1, p.S, p.W > 0 ? p.W + (k.t1 - k.t0) : 0, kPage);
  return k;
}
template <int ROWS>
__device__ __forceinline__ int blocks_of(const GqaDecodeParams& p, const Request& r) {
  return (int)(((int64_t)r.n * p.group + ROWS - 1) / ROWS);
}
// Units of work (pages, and kStart for each block) of one KV head of a request
template <int ROWS>
__device__ __forceinline__ int64_t cost_of(const GqaDecodeParams& p, const Request& r) {
  const int blocks = blocks_of<ROWS>(p, r);
  int64_t sum = 0;
  for (int rb = 0; rb < blocks; ++rb) sum += block_of<ROWS>(p, r, rb).units();
  return sum;
}

__device__ __forceinline__ float row_max(float x) {  // over the four lanes that hold tokens of the same row
  float y = x;
  swap16(x, y);
  x = fmaxf(x, y);
  y = x;
  swap32(x, y);
  return fmaxf(x, y);
}
__device__ __forceinline__ float row_sum(float x) {
  float y = x;
  swap16(x, y);
  x += y;
  y = x;
  swap32(x, y);
  return x + y;
}

// 2^(ref - top); 1 where both are -inf (no tokens)
__device__ __forceinline__ float factor(float ref, float top) { return ref == top ? 1.f : exp2_fast(ref - top); }

// Two tokens' codes of four columns (a word each) as f16 pairs, one column's two tokens to a word.
__device__ __forceinline__ uint32_t f16_pair(uint32_t w, bool upper) {
  return upper ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, true))
               : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, false));
}
// The lower or upper two columns' codes of two tokens (four columns each), a column's two tokens side by side.
__device__ __forceinline__ uint32_t token_pair(uint32_t a, uint32_t b, bool upper) { return __builtin_amdgcn_perm(b, a, upper ? 0x07030602 : 0x05010400); }
__device__ __forceinline__ uint32_t bf16_pair(uint32_t w, bool upper) {
  return upper ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, true))
               : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, false));
}

// Codes of one (page, KV head): `bytes` of them may be read, behind that the loads return zeros and touch no memory.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t codes_at(const uint8_t* base, uint32_t bytes) {
  const uint64_t a = uniform64((uint64_t)(uintptr_t)base);
  return __builtin_amdgcn_make_buffer_rsrc((void*)(uintptr_t)a, 0, (int)__builtin_amdgcn_readfirstlane(bytes), 0x00027000);
}

// What a variant of the kernel keeps where.
template <int D, int RT>
struct Gqa {
  static constexpr int kRows = 16 * RT;
  static constexpr int kCols = D / 16;    // columns of V per lane
  static constexpr int kWords = D / 64;   // 64-byte pieces of a K row; also words of V per lane and token
  static constexpr int kGroups = groups_per_cu(D, RT);
  // The query block: registers, or LDS (two buffers, one for the next block) where they are needed for the output
  static constexpr bool kQLds = D == 256 || D * RT > 256;
  static constexpr size_t kQBytes = kQLds ? (size_t)kRows * D * 2 : 0;
  static constexpr size_t kMlBytes = (size_t)4 * kRows * 16;
  // Columns of the output that meet at a time, 1 / kParts of them, as far as LDS holds them for all four waves
  static constexpr size_t o_bytes(int parts) { return (size_t)4 * kRows * (D / parts + 4) * 4; }
  static constexpr size_t kRoom = 160 * 1024 / kGroups - 8 * 1024 - 2 * kQBytes - 2 * kMlBytes;
  static constexpr int kParts = o_bytes(1) <= kRoom ? 1 : o_bytes(2) <= kRoom ? 2 : 4;
  static_assert(o_bytes(kParts) <= kRoom, "the waves' outputs have to fit LDS");
  static constexpr int kOStride = D / kParts + 4;  // floats of a row in LDS
  static constexpr size_t kLds = o_bytes(kParts) + 2 * kMlBytes + 2 * kQBytes;
};

template <int WORDS>
struct VWord { typedef u32x4 type; };
template <>
struct VWord<1> { typedef uint32_t type; };
template <>
struct VWord<2> { typedef u32x2 type; };

template <int D>
struct Tile {
  static constexpr int kWords = D / 64;
  u32x4 k[2][kWords];                     // [16-token half][64-byte piece]
  typename VWord<kWords>::type v[8];      // [token of the lane]
};

template <int WORDS>
__device__ __forceinline__ uint32_t word(const typename VWord<WORDS>::type& v, int i) {
  if constexpr (WORDS == 1) return v;
  else return v[i];
}

template <int D>
__device__ __forceinline__ void load_k(Tile<D>& t, __amdgpu_buffer_rsrc_t rsrc, int at) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
      t.k[h][c] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at + h * 16 * D + c * 64, 0, 0));
}
template <int D>
__device__ __forceinline__ void load_v(Tile<D>& t, __amdgpu_buffer_rsrc_t rsrc, int at) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int off = at + (j < 4 ? j : 12 + j) * D;
    if constexpr (D == 64) t.v[j] = __builtin_amdgcn_raw_buffer_load_b32(rsrc, off, 0, 0);
    else if constexpr (D == 128) t.v[j] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rsrc, off, 0, 0));
    else t.v[j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, off, 0, 0));
  }
}

// Whether one of four codes is NaN (0x7f or 0xff).
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// NaN codes as 0.
__device__ __forceinline__ uint32_t without_nan(uint32_t w) {
  const uint32_t high = nan_codes(w);  // 0x80 in the bytes that are NaN
  return w & ~(high | (high - (high >> 7)));
}
template <int WORDS>
__device__ __forceinline__ typename VWord<WORDS>::type without_nan(typename VWord<WORDS>::type v) {
  if constexpr (WORDS == 1) return without_nan((uint32_t)v);
  else {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) v[i] = without_nan((uint32_t)v[i]);
    return v;
  }
}

// Orders LDS between the waves of a work group without waiting for the loads of the next block, which are under way.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// The kernel's arguments, to be read again where they are used: kept in scalar registers through the loop they push others out.
__device__ __forceinline__ const GqaDecodeParams* late_arguments() {
  uint64_t at = (uint64_t)(uintptr_t)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(at));
  return (const GqaDecodeParams*)(const __attribute__((address_space(4))) GqaDecodeParams*)(uintptr_t)at;
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// The share of work group u of U: units [bound(u), bound(u + 1)), bound(u) = floor(u T / U).
struct Shares {
  int64_t T, each;  // each = T / U
  int U, rest;      // rest = T % U
  __device__ __forceinline__ int64_t bound(int u) const { return u * each + u * rest / U; }  // (U is at most 2^12)
  // the work group that has unit x
  __device__ __forceinline__ int owner(int64_t x) const {
    int u = min((int)((double)x * U / (double)T), U - 1);
    while (bound(u) > x) --u;
    while (bound(u + 1) <= x) ++u;
    return u;
  }
};

template <int D, int RT, bool OUT32>
__global__ __launch_bounds__(kThreads, groups_per_cu(D, RT)) void gqa_decode_kernel(GqaDecodeParams p) {
  using C = Gqa<D, RT>;
  constexpr int R = C::kRows, kCols = C::kCols, kWords = C::kWords;
  extern __shared__ __align__(16) float lds[];
  float* const o_lds = lds;                                    // [4 waves][R][kOStride]
  float4* const ml_lds = (float4*)(lds + 4 * R * C::kOStride); // [2][4 waves][R]
  bf16x8* const q_lds = (bf16x8*)(ml_lds + 2 * 4 * R);         // [2][operands of the products][64 lanes]
  __shared__ int64_t wave_tot[4];
  __shared__ int4 requests[kThreads];  // (batches of up to 256: L, begin, n, units of one KV head)
  __shared__ int64_t found_off;
  __shared__ int found_at;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int n16 = lane & 15, g = lane >> 4;

  // Share of this work group: running sum of the units over the batch, a run of requests per thread.  The thread whose requests
  // hold the share's first unit says so.
  const int per = (p.batch + kThreads - 1) / kThreads;
  Shares shares;
  int64_t begin, off;
  int at_request;
  {
    int64_t mine = 0;
    for (int i = 0; i < per; ++i) {
      const int b = tid * per + i;
      if (b < p.batch) {
        const Request r = request_of(p, b);
        const int64_t cost = cost_of<R>(p, r);
        mine += cost * p.kv_heads;
        if (per == 1) requests[tid] = make_int4(r.L, r.begin, r.n, (int)cost);
      }
    }
    int64_t sum = mine;
    for (int d = 1; d < 64; d *= 2) {
      const int64_t y = __shfl_up(sum, d);
      if (lane >= d) sum += y;
    }
    if (lane == 63) wave_tot[wave] = sum;
    __syncthreads();
    shares.T = 0;
    for (int w = 0; w < 4; ++w) {
      if (w == wave) sum += shares.T;
      shares.T += (int64_t)uniform64(wave_tot[w]);
    }
    shares.U = (int)min((int64_t)gridDim.x, shares.T);
    if ((int)blockIdx.x >= shares.U) return;
    if (shares.T >> 31) shares.each = shares.T / shares.U;
    else shares.each = (uint32_t)shares.T / (uint32_t)shares.U;
    shares.rest = (int)(shares.T - shares.each * shares.U);
    begin = shares.bound(blockIdx.x);
    if (sum - mine <= begin && begin < sum) {
      found_at = tid;
      found_off = begin - (sum - mine);
    }
    __syncthreads();
    at_request = uniform(found_at) * per;
    off = (int64_t)uniform64(found_off);
  }
  auto request = [&](int b) {
    if (per == 1) {
      const int4 r = requests[b];
      return Request{uniform(r.x), uniform(r.y), uniform(r.z)};
    }
    const Request r = request_of(p, b);
    return Request{uniform(r.L), uniform(r.begin), uniform(r.n)};
  };
  const int64_t stop = shares.bound(blockIdx.x + 1);

  // The part of a block that this work group computes.
  struct Piece {
    int b, h, rb;
    Request rq;
    Block bk;
    int off;               // the block's units before it
    int tile_lo, tile_hi;  // its pages, by their number among the block's
    int64_t left;          // units of the share from its first one on
  };
  auto cut = [&](Piece& w) {
    w.bk = block_of<R>(p, w.rq, w.rb);
    w.tile_lo = max(w.off - kStart, 0);
    w.tile_hi = (int)min(max(w.left + w.off - kStart, (int64_t)0), (int64_t)w.bk.pages.count());
  };
  // Whether there is something to do: pages, or the empty result of a block that keeps nothing, which is whose share has its first unit.
  auto counts = [&](const Piece& w) { return w.tile_lo < w.tile_hi || (w.bk.pages.count() == 0 && w.off == 0); };
  // The next block with something to do for this work group; false if there is none.
  auto follow = [&](Piece& w) {
    do {
      w.left -= w.bk.units() - w.off;
      w.off = 0;
      if (w.left <= 0) return false;
      if (++w.rb >= blocks_of<R>(p, w.rq)) {
        w.rb = 0;
        if (++w.h == p.kv_heads) {
          w.h = 0;
          do w.rq = request(++w.b);
          while (w.rq.n == 0);
        }
      }
      cut(w);
    } while (!counts(w));
    return true;
  };
  Piece now;
  now.left = stop - begin;
  if (per == 1) {
    now.b = at_request;
    const int4 r = requests[now.b];
    now.rq = Request{uniform(r.x), uniform(r.y), uniform(r.z)};
    const uint32_t cost = uniform(r.w);
    now.h = (int)((uint32_t)off / cost);  // (one request's units are below 2^31)
    off -= (int64_t)now.h * cost;
  } else {
    int64_t cost;
    for (now.b = at_request;; ++now.b) {
      now.rq = request(now.b);
      cost = cost_of<R>(p, now.rq);
      if (off < cost * p.kv_heads) break;
      off -= cost * p.kv_heads;
    }
    now.h = (int)((uint32_t)off / (uint32_t)cost);
    off -= now.h * cost;
  }
  for (now.rb = 0;; ++now.rb) {
    const int units = block_of<R>(p, now.rq, now.rb).units();
    if (off < units) break;
    off -= units;
  }
  now.off = (int)off;
  cut(now);
  if (!counts(now) && !follow(now)) return;

  const size_t head_bytes = (size_t)kPage * D;
  const int k_at = (wave * kWaveTokens + n16) * D + g * 16;
  const int v_at = (wave * kWaveTokens + 4 * g) * D + n16 * kCols;
  const int blocks_per_page = kPage >> p.scale_shift, my_block = (wave * kWaveTokens) >> p.scale_shift;
  int parity = 0, first_partial = 0;  // first_partial: 1 once this work group has left its first block behind

  // Page-table entries of up to 64 of a block's pages from number `held` on, one per lane.
  auto entries = [&](int b, const TileLayout& pages, int from) {
    const int last = pages.count() - 1;
    return last >= 0 ? p.page_table[b * p.table_stride + pages.logical(min(from + lane, last))] : 0;
  };
  // Query rows of a block: lane n16 of every group of 16 holds one row of each row tile, the columns that its K loads
  // bring.  Rows past the last hold zeros.  reach: tokens that the row's query sees.
  constexpr int kQs = C::kQLds ? RT * kWords / 2 : RT * 2 * kWords;  // operands that the wave reads: its share, or all
  bf16x8 q[kQs];
  int reach[RT];
  auto rows_of = [&](const Piece& w) { return (int)min((int64_t)w.rq.n * p.group - (int64_t)w.rb * R, (int64_t)R); };
  auto load_q = [&](const Piece& w) {
    const int rows = rows_of(w);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int row = rt * 16 + n16;
      const uint32_t t = (uint32_t)(w.rb * R + row) / (uint32_t)p.group, gi = (uint32_t)(w.rb * R + row) - t * p.group;
      const bool valid = row < rows;
      reach[rt] = valid ? w.rq.L - w.rq.n + (int)t + 1 : 0;
      const uint16_t* src = p.q + (int64_t)(w.rq.begin + (int)t) * p.q_stride + (size_t)(w.h * p.group + (int)gi) * D + g * 16;
      if constexpr (C::kQLds) {
        // (operand 2 c + u holds columns 64 c + 16 g + 8 u on; the wave reads those with the remainder `wave` by 4)
#pragma unroll
        for (int i = 0; i < kWords / 2; ++i) q[rt * kWords / 2 + i] = valid ? *(const bf16x8*)(src + (2 * i + wave / 2) * 64 + wave % 2 * 8) : bf16x8{};
      } else {
#pragma unroll
        for (int i = 0; i < 2 * kWords; ++i) q[rt * 2 * kWords + i] = valid ? *(const bf16x8*)(src + i / 2 * 64 + i % 2 * 8) : bf16x8{};
      }
    }
  };
  // The operands that the wave has read go to LDS, where all waves find them behind the next barrier.
  int q_side = 0;
  auto store_q = [&](int side) {
    if constexpr (C::kQLds) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int i = 0; i < kWords / 2; ++i) q_lds[((side * RT + rt) * 2 * kWords + 4 * i + wave) * 64 + lane] = q[rt * kWords / 2 + i];
    }
  };
  auto query = [&](int rt, int i) {
    if constexpr (C::kQLds) return q_lds[((q_side * RT + rt) * 2 * kWords + i) * 64 + lane];
    else return q[rt * 2 * kWords + i];
  };
  // What a page's loads need: where its codes are, and the wave's two scales.
  __amdgpu_buffer_rsrc_t rk, rv;
  float ks = 0.f, vs = 0.f;
  auto aim = [&](const Piece& w, int tile, int ids, int held) {
    const int page = __builtin_amdgcn_readlane(ids, tile - held);
    const size_t ph = (size_t)page * p.kv_heads + w.h;
    const int seen = w.rq.L - w.rq.n + w.bk.t1 + 1;
    const int live = min(seen - w.bk.pages.logical(tile) * kPage, kPage);
    rk = codes_at(p.k_cache + ph * head_bytes, live * D);
    rv = codes_at(p.v_cache + ph * head_bytes, live * D);
    ks = p.k_scales[ph * blocks_per_page + my_block];
    vs = p.v_scales[ph * blocks_per_page + my_block];
  };

  Tile<D> t;
  int held = now.tile_lo, ids = entries(now.b, now.bk.pages, held);
  load_q(now);
  if (now.tile_lo < now.tile_hi) {
    aim(now, now.tile_lo, ids, held);
    load_k<D>(t, rk, k_at);
    load_v<D>(t, rv, v_at);
  }
  if constexpr (C::kQLds) {
    store_q(0);
    lds_barrier();
  }
  // Entries of the next request's first block, asked for as soon as the one before it begins: short requests come and go faster
  // than a chain of loads from the table to the codes.
  int ahead_b = -1, ahead_ids = 0;

  while (true) {
    Piece next = now;
    bool more_blocks = false, next_loads = false;
    if (ahead_b <= now.b) {
      ahead_b = now.b + 1;
      if (ahead_b < p.batch) {
        const Request r = request(ahead_b);
        if (r.n > 0) ahead_ids = entries(ahead_b, block_of<R>(p, r, 0).pages, 0);
      }
    }
    const int reach_lo = now.rq.L - now.rq.n + now.bk.t0 + 1, reach_hi = now.rq.L - now.rq.n + now.bk.t1 + 1;

    // What the next block is (asked late, so that its description need not be kept through the loop), and where its first page is: its
    // entries are the same as this block's for another KV head, or were asked for before, or are asked for now.
    auto turn_to_next = [&] {
      more_blocks = follow(next);
      next_loads = more_blocks && next.tile_lo < next.tile_hi;
      if (!next_loads) return;
      if (!(next.b == now.b && next.rb == now.rb && held == 0)) {
        held = 0;
        ids = next.b == ahead_b && next.rb == 0 ? ahead_ids : entries(next.b, next.bk.pages, 0);
      }
      aim(next, next.tile_lo, ids, held);
    };

    // O holds sum 2^(x - n + kLift) v_scale v_code and l sum 2^(x - m + kLift) for the row's logits x (log2): two references,
    // so that neither a small nor a large scale of a block of values costs the weights their range.
    f32x4 o[RT][kCols];
    float m[RT], n[RT], l[RT], ratio[RT];  // ratio = 2^(m - n)
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      m[rt] = n[rt] = -INFINITY;
      l[rt] = ratio[rt] = 0.f;
#pragma unroll
      for (int c = 0; c < kCols; ++c) o[rt][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    float saw_nan = 0.f;
    for (int tile = now.tile_lo; tile < now.tile_hi; ++tile) {
      const int pos0 = now.bk.pages.logical(tile) * kPage + wave * kWaveTokens;
      // every query sees and keeps all 32 tokens
      const bool full = pos0 + kWaveTokens <= reach_lo && (pos0 + kWaveTokens <= p.S || pos0 >= reach_hi - p.W);
      // S^T of the wave's tokens: lane (n16, g) has tokens 16 h2 + 4 g + i of row n16
      f32x4 s[RT][2];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[rt][0] = s[rt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 2 * kWords; ++i) {
        bf16x8 k[2];
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2) {
          u32x4 w;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            w[2 * j] = bf16_pair(t.k[h2][i / 2][i % 2 * 2 + j], false);
            w[2 * j + 1] = bf16_pair(t.k[h2][i / 2][i % 2 * 2 + j], true);
          }
          k[h2] = __builtin_bit_cast(bf16x8, w);
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          const bf16x8 x = query(rt, i);
#pragma unroll
          for (int h2 = 0; h2 < 2; ++h2) s[rt][h2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[h2], x, s[rt][h2], 0, 0, 0);
        }
      }
      // (the scale of a block without kept tokens may be anything)
      const bool some = pos0 < reach_hi && (pos0 < p.S || (p.W > 0 && pos0 + kWaveTokens > reach_lo - p.W));
      const float factor = p.scale_log2 * ks, v_scale = some ? vs : 0.f;
      // (at least 2^-100: ratio stays finite)
      const float v_log = fmaxf(__log2f(v_scale), -100.f);
      int seen[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) seen[rt] = reach[rt];
      // the next page's loads, of this block or the next one, as soon as their registers are free
      bool more = true;
      if (tile + 1 < now.tile_hi) {
        if (tile + 1 - held >= 64) {
          held = tile + 1;
          ids = entries(now.b, now.bk.pages, held);
        }
        aim(now, tile + 1, ids, held);
      } else {
        turn_to_next();
        more = next_loads;
        if (more_blocks) load_q(next);
      }
      if (more) load_k<D>(t, rk, k_at);

      f16x8 w_hi[RT], w_lo[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = s[rt][i / 4][i % 4] * factor;
        if (!full) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int pos = pos0 + 16 * (i / 4) + 4 * g + i % 4;
            x[i] = retained(pos, seen[rt], p.S, p.W) ? x[i] : -INFINITY;
          }
        }
        float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        if (__any(top > fminf(m[rt], n[rt] - v_log) + kSlack)) {
          top = row_max(top);
          const float next_m = top > m[rt] + kSlack ? top : m[rt];
          const float next_n = top + v_log > n[rt] + kSlack ? top + v_log : n[rt];
          l[rt] *= next_m == m[rt] ? 1.f : exp2_fast(m[rt] - next_m);
          const float shrink = next_n == n[rt] ? 1.f : exp2_fast(n[rt] - next_n);
          m[rt] = next_m;
          n[rt] = next_n;
          ratio[rt] = next_n == -INFINITY ? 0.f : exp2_fast(next_m - next_n);
#pragma unroll
          for (int c = 0; c < kCols; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[rt][c][i] *= shrink;
        }
        // (a row that has kept nothing so far has reference -inf, and only masked logits)
        const float ref = m[rt] == -INFINITY ? 0.f : m[rt] - kLift, value = ratio[rt] * v_scale;
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          w[i] = exp2_fast(x[i] - ref);
          float y = w[i] * value;
          // (fixed here: the compiler may fuse the product with one of its two uses and round the other in two steps, which
          // near a tie of f16 leaves the second term for another first term)
          if constexpr (OUT32) asm("" : "+v"(y));
          w_hi[rt][i] = (_Float16)y;
          if constexpr (OUT32) w_lo[rt][i] = (_Float16)(y - (float)w_hi[rt][i]);
        }
        l[rt] += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
      }
      if (!full) {
        // tokens that no row of the block keeps may hold anything
        uint32_t any_nan = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int pos = pos0 + (j < 4 ? 0 : 16) + 4 * g + j % 4;
          const bool keep = pos < reach_hi && (pos < p.S || (p.W > 0 && pos >= reach_lo - p.W));
          if (!keep) t.v[j] = typename VWord<kWords>::type{};
#pragma unroll
          for (int i = 0; i < kWords; ++i) any_nan |= nan_codes(word<kWords>(t.v[j], i));
        }
        // NaN in a value row is for the rows that keep the token, and only for those, but a weight of 0 would not stop it in the
        // product: it goes on as 0, and the block's end sees to it.
        if (now.bk.t1 > now.bk.t0 && __ballot(any_nan != 0) != 0) {
          saw_nan = 1.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) t.v[j] = without_nan<kWords>(t.v[j]);
        }
      }
#pragma unroll
      for (int wd = 0; wd < kWords; ++wd) {
#pragma unroll
        for (int col = 0; col < 4; ++col) {
          u32x4 f;
#pragma unroll
          for (int j = 0; j < 4; ++j) f[j] = f16_pair(token_pair(word<kWords>(t.v[2 * j], wd), word<kWords>(t.v[2 * j + 1], wd), col / 2), col % 2);
          const f16x8 vt = __builtin_bit_cast(f16x8, f);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            f32x4& acc = o[rt][4 * wd + col];
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(vt, w_hi[rt], acc, 0, 0, 0);
            if constexpr (OUT32) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(vt, w_lo[rt], acc, 0, 0, 0);
          }
        }
      }
      if (more) load_v<D>(t, rv, v_at);
    }
    if (now.tile_lo >= now.tile_hi) {  // (nothing kept: the next block has not been asked for yet)
      turn_to_next();
      if (more_blocks) load_q(next);
      if (next_loads) {
        load_k<D>(t, rk, k_at);
        load_v<D>(t, rv, v_at);
      }
    }

    if (more_blocks) store_q(q_side ^ 1);
    q_side ^= 1;

    // The waves' shares meet: references and sum first, then the outputs at the common reference.
    float4* const ml = ml_lds + parity * 4 * R;
    parity ^= 1;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      l[rt] = row_sum(l[rt]);
      if (g == 0) ml[wave * R + rt * 16 + n16] = make_float4(m[rt], l[rt], n[rt], saw_nan);
    }
    lds_barrier();
    float shrink[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < 4; ++w) top = fmaxf(top, ml[w * R + rt * 16 + n16].z);
      // (a wave that kept nothing has zeros, or NaN that has to stay: nothing is skipped)
      shrink[rt] = factor(n[rt], top);
    }
    const int slot = 2 * blockIdx.x + first_partial;
    const GqaDecodeParams& end = *late_arguments();
    constexpr int kChunks = D / 8 / C::kParts;
    const int rows = rows_of(now);
    const bool whole = now.tile_lo == 0 && now.tile_hi == now.bk.pages.count();
#pragma unroll
    for (int part = 0; part < C::kParts; ++part) {
    if (part) lds_barrier();  // (the part before has been read)
    if (C::kParts == 1 || g / (4 / C::kParts) == part) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float* const dst = o_lds + (wave * R + rt * 16 + n16) * C::kOStride + (4 * g % (16 / C::kParts)) * kCols;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int c = 0; c < kCols; c += 4)
            *(f32x4*)(dst + i * kCols + c) = f32x4{o[rt][c][i] * shrink[rt], o[rt][c + 1][i] * shrink[rt], o[rt][c + 2][i] * shrink[rt], o[rt][c + 3][i] * shrink[rt]};
      }
    }
    lds_barrier();
    for (int k = tid; k < rows * kChunks; k += kThreads) {
      const int row = k / kChunks, in_part = k % kChunks * 8, col = part * (D / C::kParts) + in_part;
      f32x4 a = {0.f, 0.f, 0.f, 0.f}, c = a;
      float top = -INFINITY, vtop = -INFINITY, sum = 0.f, nans = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        top = fmaxf(top, ml[w * R + row].x);
        vtop = fmaxf(vtop, ml[w * R + row].z);
        nans += ml[w * R + row].w;
      }
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float4 e = ml[w * R + row];
        sum += e.y * (e.x == top ? 1.f : exp2_fast(e.x - top));
        const f32x4* src = (const f32x4*)(o_lds + (w * R + row) * C::kOStride + in_part);
        a += src[0];
        c += src[1];
      }
      const uint32_t qt = (uint32_t)(now.rb * R + row) / (uint32_t)end.group, gi = (uint32_t)(now.rb * R + row) - qt * end.group;
      if (__builtin_expect(nans != 0.f, 0)) {
        // NaN that the loop has taken for 0: the columns of the tokens that this row keeps are looked through again
        const int sees = now.rq.L - now.rq.n + (int)qt + 1;
#pragma unroll 1
        for (int tile = now.tile_lo; tile < now.tile_hi; ++tile) {
          const int lp = now.bk.pages.logical(tile);
          const size_t ph = (size_t)p.page_table[now.b * p.table_stride + lp] * p.kv_heads + now.h;
#pragma unroll 1
          for (int j = 0; j < kPage; ++j) {
            if (!retained(lp * kPage + j, sees, p.S, p.W)) continue;
            const u32x2 codes = *(const u32x2*)(p.v_cache + ph * head_bytes + (size_t)j * D + col);
            const uint32_t lo = nan_codes(codes[0]), hi = nan_codes(codes[1]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if ((lo >> (8 * i)) & 0x80u) a[i] = NAN;
              if ((hi >> (8 * i)) & 0x80u) c[i] = NAN;
            }
          }
        }
      }
      const int64_t out_row = (int64_t)(now.rq.begin + (int)qt) * end.q_heads + now.h * end.group + (int)gi;
      if (whole) {
        const float inv = sum == 0.f ? 0.f : exp2_fast(vtop - top) / sum;  // (nothing kept: 0 and -inf)
        if constexpr (OUT32) {
          f32x4* dst = (f32x4*)((float*)end.out + out_row * D + col);
          dst[0] = a * inv;
          dst[1] = c * inv;
        } else {
          bf16x8 y;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            y[i] = (__bf16)(a[i] * inv);
            y[4 + i] = (__bf16)(c[i] * inv);
          }
          *(bf16x8*)((uint16_t*)end.out + out_row * D + col) = y;
        }
        if (col == 0) {
          end.lse[out_row] = sum == 0.f ? -INFINITY : (top + __log2f(sum) - kLift) * 0.69314718055994531f;
          end.rows[out_row] = make_int2(0, 0);
        }
      } else {
        float* dst = end.part_o + ((size_t)slot * R + row) * D + col;
        ((f32x4*)dst)[0] = a;
        ((f32x4*)dst)[1] = c;
        if (col == 0) {
          end.part_ml[(size_t)slot * R + row] = make_float4(top, sum, vtop, 0.f);
          // the work group that takes a block's first page knows which ones take the others
          if (now.tile_lo == 0) end.rows[out_row] = make_int2(slot, (shares.owner(stop - now.left - now.off + now.bk.units() - 1) - (int)blockIdx.x + 1) * 64 + row);
        }
      }
    }
    }
    first_partial = 1;
    if (!more_blocks) break;
    now = next;
  }
}

// Joins the partial rows of blocks whose pages went to several work groups: o = sum_i 2^(n_i - n) o_i, l = sum_i 2^(m_i - m) l_i.  Partial i of a
// row lies in the slot of the i-th work group: the first one may have had another block before (slot 2 u + 1), the others
// begin with this one (2 u).  WAVES waves share a row, each every WAVES-th partial.
template <int D, bool OUT32, int WAVES>
__global__ __launch_bounds__(256) void gqa_combine_kernel(GqaDecodeParams p, int block_rows, int units) {
  constexpr int kPer = D / 64;  // columns per lane
  typedef __attribute__((ext_vector_type(kPer))) float vec;
  __shared__ float sh_o[WAVES > 1 ? 4 : 1][WAVES > 1 ? D : 1];
  __shared__ float4 sh_ml[4];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * (4 / WAVES) + wave / WAVES;
  if (row >= (int64_t)p.num_queries * p.q_heads) return;
  // (rows of no request: nothing was written for them)
  if (p.q_start && (row / p.q_heads < p.q_start[0] || row / p.q_heads >= p.q_start[p.batch])) return;
  const int2 d = p.rows[row];
  const int count = __builtin_amdgcn_readfirstlane(d.y / 64), in_block = d.y % 64;
  if (count <= 0 || d.x < 0 || d.x / 2 + count > units) return;
  const int u0 = d.x / 2;
  float m = -INFINITY, n = -INFINITY, l = 0.f;
  vec o = {};
  constexpr int kBatch = 8;
  for (int i0 = wave % WAVES; i0 < count; i0 += kBatch * WAVES) {
    float4 e[kBatch];
    vec x[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int i = min(i0 + k * WAVES, count - 1);
      const size_t slot = i == 0 ? d.x : 2 * (u0 + i);
      e[k] = p.part_ml[slot * block_rows + in_block];
      x[k] = *(const vec*)(p.part_o + (slot * block_rows + in_block) * D + lane * kPer);
    }
    float top = m, vtop = n;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      top = fmaxf(top, e[k].x);
      vtop = fmaxf(vtop, e[k].z);
    }
    l *= factor(m, top);
    o *= factor(n, vtop);
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (i0 + k * WAVES < count) {
        l += factor(e[k].x, top) * e[k].y;
        o += factor(e[k].z, vtop) * x[k];
      }
    m = top;
    n = vtop;
  }
  if constexpr (WAVES > 1) {
    if (lane == 0) sh_ml[wave] = make_float4(m, l, n, 0.f);
    *(vec*)(&sh_o[wave][lane * kPer]) = o;
    __syncthreads();
    if (wave) return;
    float top = m, vtop = n;
    for (int w = 1; w < WAVES; ++w) {
      top = fmaxf(top, sh_ml[w].x);
      vtop = fmaxf(vtop, sh_ml[w].z);
    }
    l *= factor(m, top);
    o *= factor(n, vtop);
    for (int w = 1; w < WAVES; ++w) {
      l += factor(sh_ml[w].x, top) * sh_ml[w].y;
      o += factor(sh_ml[w].z, vtop) * *(const vec*)(&sh_o[w][lane * kPer]);
    }
    m = top;
    n = vtop;
  }
  const float inv = l == 0.f ? 0.f : exp2_fast(n - m) / l;
  if constexpr (OUT32) {
    *(vec*)((float*)p.out + row * D + lane * kPer) = o * inv;
  } else if constexpr (kPer == 1) {
    ((__bf16*)p.out)[row * D + lane] = (__bf16)(o[0] * inv);
  } else {
    typedef __attribute__((ext_vector_type(kPer))) __bf16 bvec;
    bvec y;
#pragma unroll
    for (int i = 0; i < kPer; ++i) y[i] = (__bf16)(o[i] * inv);
    *(bvec*)((uint16_t*)p.out + row * D + lane * kPer) = y;
  }
  if (lane == 0) p.lse[row] = l == 0.f ? -INFINITY : (m + __log2f(l) - kLift) * 0.69314718055994531f;
}

template <int D, int RT, bool OUT32>
hipError_t start(const GqaDecodeParams& p, int units, hipStream_t stream) {
  constexpr size_t lds = Gqa<D, RT>::kLds;
  hipLaunchKernelGGL((gqa_decode_kernel<D, RT, OUT32>), dim3(units), dim3(kThreads), lds, stream, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t rows = (int64_t)p.num_queries * p.q_heads;
  // Few rows: four waves to a row.
  if (rows <= 2048) hipLaunchKernelGGL((gqa_combine_kernel<D, OUT32, 4>), dim3((uint32_t)rows), dim3(256), 0, stream, p, 16 * RT, units);
  else hipLaunchKernelGGL((gqa_combine_kernel<D, OUT32, 1>), dim3((uint32_t)((rows + 3) / 4)), dim3(256), 0, stream, p, 16 * RT, units);
  return hipGetLastError();
}

template <int D, int RT>
hipError_t allow_lds() {
  hipError_t e = hipFuncSetAttribute((const void*)gqa_decode_kernel<D, RT, false>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)Gqa<D, RT>::kLds);
  if (e == hipSuccess) e = hipFuncSetAttribute((const void*)gqa_decode_kernel<D, RT, true>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)Gqa<D, RT>::kLds);
  return e;
}

}  // namespace

GqaShape gqa_shape(int batch, int num_queries, int group, int head_dim) {
  const int64_t rows = (int64_t)((num_queries + batch - 1) / batch) * group;
  const int rt = (int)std::min<int64_t>((rows + 15) / 16, head_dim == 256 ? 2 : 4);
  return GqaShape{std::max(rt, 1), groups_per_cu(head_dim, std::max(rt, 1))};
}

hipError_t init_gqa_kernels() {
  hipError_t e = allow_lds<64, 1>();
  if (e == hipSuccess) e = allow_lds<64, 2>();
  if (e == hipSuccess) e = allow_lds<64, 3>();
  if (e == hipSuccess) e = allow_lds<64, 4>();
  if (e == hipSuccess) e = allow_lds<128, 1>();
  if (e == hipSuccess) e = allow_lds<128, 2>();
  if (e == hipSuccess) e = allow_lds<128, 3>();
  if (e == hipSuccess) e = allow_lds<128, 4>();
  if (e == hipSuccess) e = allow_lds<256, 1>();
  if (e == hipSuccess) e = allow_lds<256, 2>();
  return e;
}

hipError_t launch_gqa_decode(const GqaDecodeParams& p, const GqaShape& shape, int units, hipStream_t stream) {
  auto with = [&](auto d, auto rt) {
    return p.out_fp32 ? start<decltype(d)::value, decltype(rt)::value, true>(p, units, stream)
                      : start<decltype(d)::value, decltype(rt)::value, false>(p, units, stream);
  };
  using std::integral_constant;  // (the kernel variants)
  auto dims = [&](auto rt) {
    if (p.head_dim == 64) return with(integral_constant<int, 64>{}, rt);
    if (p.head_dim == 128) return with(integral_constant<int, 128>{}, rt);
    if constexpr (decltype(rt)::value <= 2) return with(integral_constant<int, 256>{}, rt);
    else return hipErrorInvalidValue;
  };
  switch (shape.row_tiles) {
    case 1: return dims(integral_constant<int, 1>{});
    case 2: return dims(integral_constant<int, 2>{});
    case 3: return dims(integral_constant<int, 3>{});
    default: return dims(integral_constant<int, 4>{});
  }
}

}  // namespace omniattn
