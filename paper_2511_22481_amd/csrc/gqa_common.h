// What the two attention kernels of the grouped-query part share: how the work is dealt out, the arithmetic of a tile's
// softmax, and the end of a block, where the waves' shares meet.  See gqa_decode_kernel.hip for the whole.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "decode_common.h"
#include "gqa.h"
#include "gqa_deal.h"

namespace omniattn {
namespace {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;

constexpr int kWaveTokens = 32;
// Weights are 2^(s - m + kLift) for the reference m, which a logit (log2) may exceed by kSlack before it is raised: the largest
// weight is at most 2^15 (f16 holds 65504), and its two f16 terms keep 2^-22 of weights down to 2^-14 of the largest, below that 2^-36 of the largest.
constexpr float kLift = 11.f, kSlack = 4.f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }


__device__ __forceinline__ Request request_of(const GqaDecodeParams& p, int b) {
  Request r;
  r.L = min(max(p.seq_lens[b], 0), p.max_pages * kPage);
  const int lo = p.q_start ? p.q_start[b] : b, hi = p.q_start ? p.q_start[b + 1] : b + 1;
  r.begin = min(max(lo, 0), p.num_queries);
  r.n = min(max(hi, r.begin), p.num_queries) - r.begin;
  return r;
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

template <int WORDS>
struct VWord { typedef u32x4 type; };
template <>
struct VWord<1> { typedef uint32_t type; };
template <>
struct VWord<2> { typedef u32x2 type; };

template <int WORDS>
__device__ __forceinline__ uint32_t word(const typename VWord<WORDS>::type& v, int i) {
  if constexpr (WORDS == 1) return v;
  else return v[i];
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

// Running sum over a wave.
__device__ __forceinline__ int wave_sum_up_to(int x) {
#define OMNIATTN_ADD(ctrl, rows) x += __builtin_amdgcn_update_dpp(0, x, ctrl, rows, 0xf, true)
  OMNIATTN_ADD(0x111, 0xf);  // from the lane one, two, four, eight before, in rows of 16
  OMNIATTN_ADD(0x112, 0xf);
  OMNIATTN_ADD(0x114, 0xf);
  OMNIATTN_ADD(0x118, 0xf);
  OMNIATTN_ADD(0x142, 0xa);  // a row's last lane to the row behind it
  OMNIATTN_ADD(0x143, 0xc);  // lane 31 to the upper half
#undef OMNIATTN_ADD
  return x;
}

// Tokens that a query sees: those before `reach`; TREE: of the text, and the nodes of a set (without those that the rule does not keep).
template <bool TREE>
struct Sight {
  int reach;
};
template <>
struct Sight<true> {
  int reach;
  uint64_t nodes;
};
template <bool TREE>
__device__ __forceinline__ Sight<TREE> sight_of(const GqaDecodeParams& p, const Piece& w, int t, bool valid) {
  if constexpr (TREE) {
    const int n = w.rq.n, text = w.rq.L - n;
    uint64_t nodes = valid ? p.masks[w.rq.begin + t] : 0;
    if (n < 64) nodes &= ((uint64_t)1 << n) - 1;
    const int count = __popcll(nodes);
    const int reach = count ? max(text + count, 0) : 0;
    if (count > p.W) {  // nodes in front of the window, but for sinks
      const int from = max(p.S - text, 0);
      uint64_t rest = nodes;
      for (int k = 0; k < count - p.W; ++k, rest &= rest - 1)
        if (k >= from) nodes &= ~(rest & -rest);
    }
    return Sight<true>{reach, nodes};
  } else {
    return Sight<false>{valid ? w.reach(t) : 0};
  }
}
// The 32 nodes whose slots begin `off` behind the first one's.
__device__ __forceinline__ uint32_t nodes_at(uint64_t nodes, int off) {
  if (off >= 0) return off < 64 ? (uint32_t)(nodes >> off) : 0;
  return off > -32 ? (uint32_t)nodes << -off : 0;
}
template <bool TREE>
__device__ __forceinline__ bool sees(const GqaDecodeParams& p, const Sight<TREE>& s, int text, int pos) {
  if constexpr (TREE) {
    if (pos >= text) return nodes_at(s.nodes, pos - text) & 1;
  }
  return retained(pos, s.reach, p.S, p.W);
}

// What a loop over a block's pages needs of it.
struct Span {
  TileLayout pages;
  int lo, hi;            // tokens that the block's first and last query see (of a tree: a first and a last node's)
  int tile_hi;
  bool several;          // several queries
  int text;              // tokens before the request's queries
  __device__ __forceinline__ explicit Span(const Piece& w)
      : pages{uniform(w.bk.pages.ns), uniform(w.bk.pages.w0), uniform(w.bk.pages.w1)}, lo(uniform(w.reach(w.bk.t0))), hi(uniform(w.reach(w.bk.t1))),
        tile_hi(uniform(w.tile_hi)), several(uniform(w.bk.t1 - w.bk.t0) > 0), text(uniform(w.rq.L - w.rq.n)) {}
};

// Finds shares and walks through their blocks (see Walk in gqa_deal.h).  SHARES: of a work group, 1 or one for each wave, which counts quarters of
// pages.  All threads call begin.
template <int R, int THREADS, int START, int SHARES = 1, bool TREE = false>
struct Dealer {
  static constexpr int kGrain = SHARES > 1 ? kWaveTokens : kPage;
  using Walker = Walk<R, START, kGrain, GqaDecodeParams, TREE>;

  // What is needed only from block to block stays here: in scalar registers it would push the loop's own out.
  struct Lds {
    int64_t wave_tot[THREADS / 64], off[SHARES], stop[SHARES];  // the share's first unit among the units of request `at`; its end
    int64_t cost[SHARES];    // (batches of up to THREADS: units of one KV head of that request)
    int4 requests[THREADS];  // (the same: L, begin, n)
    int at[SHARES];
    Shares shares;
    int pieces[THREADS / 64][3][16];
  };
  const GqaDecodeParams& p;
  const Walker walk;
  Lds& lds;
  int per;  // requests per thread

  __device__ __forceinline__ Dealer(const GqaDecodeParams& params, Lds& memory) : p(params), walk(params), lds(memory) {}

  __device__ __forceinline__ static int which() { return SHARES > 1 ? uniform(threadIdx.x >> 6) : 0; }
  __device__ __forceinline__ static int share() { return (int)blockIdx.x * SHARES + which(); }
  __device__ __forceinline__ Request request(int b) const {
    if (per == 1) {
      const int4 r = lds.requests[b];
      return Request{uniform(r.x), uniform(r.y), uniform(r.z)};
    }
    const Request r = request_of(p, b);
    return Request{uniform(r.L), uniform(r.begin), uniform(r.n)};
  }
  // The next block of the share with something to do; false if there is none.
  __device__ __forceinline__ bool follow(Piece& w) const {
    return walk.follow(w, [&](int b) { return request(b); });
  }
  // Running sum of the units over the batch, a run of requests per thread; the thread whose requests hold a share's first unit
  // says so.  False: nothing to do for this wave.
  __device__ __forceinline__ bool begin(Piece& now) {
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
    per = (p.batch + THREADS - 1) / THREADS;
    int64_t mine = 0, cost = 0;
    for (int i = 0; i < per; ++i) {
      const int b = tid * per + i;
      if (b < p.batch) {
        const Request r = request_of(p, b);
        cost = walk.cost_of(r);
        mine += cost * p.kv_heads;
        if (per == 1) lds.requests[tid] = make_int4(r.L, r.begin, r.n, 0);
      }
    }
    int64_t sum = mine;
    if (p.few_units) {
      sum = wave_sum_up_to((int)mine);
    } else {
      for (int d = 1; d < 64; d *= 2) {
        const int64_t y = __shfl_up(sum, d);
        if (lane >= d) sum += y;
      }
    }
    if (lane == 63) lds.wave_tot[wave] = sum;
    __syncthreads();
    int64_t total = 0;
    for (int w = 0; w < THREADS / 64; ++w) {
      if (w == wave) sum += total;
      total += (int64_t)uniform64(lds.wave_tot[w]);
    }
    const Shares shares(total, gridDim.x * SHARES);
    if ((int)blockIdx.x * SHARES >= shares.U) return false;
    int64_t first = shares.bound(blockIdx.x * SHARES);
#pragma unroll
    for (int i = 0; i < SHARES; ++i) {
      const int u = blockIdx.x * SHARES + i;
      const int64_t stop = shares.bound(u + 1);
      if (u < shares.U && sum - mine <= first && first < sum) {
        lds.at[i] = tid;
        lds.off[i] = first - (sum - mine);
        lds.cost[i] = cost;
        lds.stop[i] = stop;
        lds.shares = shares;
      }
      first = stop;
    }
    __syncthreads();
    if (share() >= shares.U) return false;
    const int at = uniform(lds.at[which()]) * per;
    int64_t off = (int64_t)uniform64(lds.off[which()]);
    now.left = shares.bound(share() + 1) - shares.bound(share());
    now.b = at;
    now.rq = request(at);
    if (per == 1) {
      cost = (int64_t)uniform64(lds.cost[which()]);
    } else {
      while (off >= (cost = walk.cost_of(now.rq)) * p.kv_heads) {
        off -= cost * p.kv_heads;
        now.rq = request(++now.b);
      }
    }
    return walk.enter(now, off, cost, [&](int b) { return request(b); });
  }
  __device__ __forceinline__ int rows_of(const Piece& w) const { return min(w.rq.n * p.group - w.rb * R, R); }
  // Shares that have a part of the block of w, from this one on (which has its first page).
  __device__ __forceinline__ int partners(const Piece& w) const {
    const Shares shares = lds.shares;
    return shares.owner(lds.stop[which()] - w.left - w.off + walk.units(w.bk) - 1) - share() + 1;
  }
  // A wave's notes of blocks, in one of three places.
  __device__ __forceinline__ void keep(int place, const Piece& w) const {
    const int v[16] = {w.b, w.h, w.rb, w.rq.L, w.rq.begin, w.rq.n, w.bk.t0, w.bk.t1, w.bk.pages.ns, w.bk.pages.w0, w.bk.pages.w1, w.off, w.tile_lo, w.tile_hi,
                       (int)w.left, (int)(w.left >> 32)};
    int4* const at = (int4*)lds.pieces[uniform(threadIdx.x >> 6)][place];
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) at[i] = make_int4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
    }
  }
  __device__ __forceinline__ Piece kept(int place) const {
    const int4* const at = (const int4*)lds.pieces[uniform(threadIdx.x >> 6)][place];
    const int4 a = at[0], b = at[1], c = at[2], d = at[3];
    Piece w;
    w.b = uniform(a.x), w.h = uniform(a.y), w.rb = uniform(a.z), w.rq.L = uniform(a.w);
    w.rq.begin = uniform(b.x), w.rq.n = uniform(b.y), w.bk.t0 = uniform(b.z), w.bk.t1 = uniform(b.w);
    w.bk.pages.ns = uniform(c.x), w.bk.pages.w0 = uniform(c.y), w.bk.pages.w1 = uniform(c.z), w.off = uniform(c.w);
    w.tile_lo = uniform(d.x), w.tile_hi = uniform(d.y);
    w.left = (int64_t)(((uint64_t)(uint32_t)uniform(d.w) << 32) | (uint32_t)uniform(d.z));
    return w;
  }
};

// A wave's share of the output rows: O holds sum 2^(x - n + kLift) v_scale v_code and l sum 2^(x - m + kLift) for the row's logits x
// (log2).  Two references, so that neither a small nor a large scale of a block of values costs the weights their range.  Lane (n16,
// g) has row n16 of each row tile, and of O columns (4 g + i) D / 16 + c.
template <int D, int RT>
struct Rows {
  static constexpr int kCols = D / 16;
  f32x4 o[RT][kCols];
  float m[RT], n[RT], l[RT], ratio[RT];  // ratio = 2^(m - n)
  float saw_nan;                         // 1: value codes that are NaN have been taken for 0
  __device__ __forceinline__ void clear() {
    saw_nan = 0.f;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      m[rt] = n[rt] = -INFINITY;
      l[rt] = ratio[rt] = 0.f;
#pragma unroll
      for (int c = 0; c < kCols; ++c) o[rt][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
};

// What a weight is multiplied by.  It stays finite where a row has kept values with a scale of 0 or next to it so far, and others' is very large: the row's weights
// there are 0 or as good as that, but 0 times infinity is NaN.
__device__ __forceinline__ float value_factor(float ratio, float v_scale) { return fminf(ratio * v_scale, 0x1.fffffep+127f); }

// Weights of a tile of 32 tokens from its S^T (lane (n16, g) has tokens 16 h + 4 g + i of row n16), in two f16 terms (`low`: what
// rounding to `high` leaves), references, sums and, where a reference rises, the output.  sight: tokens that the row's query sees; full: every
// row keeps all 32 tokens, which begin at pos0.  (One term is 2^-11 of a weight: 7 to 9 in a hundred bf16 results then were the neighbour
// of the right one.  With two a bf16 result is the fp32 result rounded.  us with one / two: 1 request of 131072 56.8 / 56.9, 64 of 32768
// 713 / 714, 256 short ones of width 64 30.4 / 30.9; 64 requests of 2000 to 16000, 4 KV heads, 64 rows: width 64 75 / 86, 128 132 / 151,
// 256 238 / 270.)
template <int D, int RT, bool TREE>
__device__ __forceinline__ void weigh(const GqaDecodeParams& p, Rows<D, RT>& a, const f32x4 (&s)[RT][2], const Sight<TREE> (&sight)[RT], int text, bool full, int pos0,
                                      int g, float k_factor, float v_scale, f16x8 (&high)[RT], f16x8 (&low)[RT]) {
  [[maybe_unused]] const float given_scale = v_scale;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = s[rt][i / 4][i % 4] * k_factor;
    if (!full) {
      uint32_t nodes = 0;
      if constexpr (TREE) nodes = nodes_at(sight[rt].nodes, pos0 - text) >> (4 * g);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int pos = pos0 + 16 * (i / 4) + 4 * g + i % 4;
        bool keep = retained(pos, sight[rt].reach, p.S, p.W);
        if constexpr (TREE) keep = pos < text ? keep : nodes >> (16 * (i / 4) + i % 4) & 1;
        x[i] = keep ? x[i] : -INFINITY;
      }
    }
    float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    // (a tile that no row keeps anything of can be among a tree's, and its scale be anything)
    if constexpr (TREE) v_scale = !full && !__any(top > -INFINITY) ? 0.f : given_scale;
    const float v_log = fmaxf(__log2f(v_scale), -100.f);  // (at least 2^-100: ratio stays finite)
    if (__any(top > fminf(a.m[rt], a.n[rt] - v_log) + kSlack)) {
      top = row_max(top);
      const float next_m = top > a.m[rt] + kSlack ? top : a.m[rt];
      const float next_n = top + v_log > a.n[rt] + kSlack ? top + v_log : a.n[rt];
      a.l[rt] *= factor(a.m[rt], next_m);
      const float shrink = factor(a.n[rt], next_n);
      a.m[rt] = next_m;
      a.n[rt] = next_n;
      a.ratio[rt] = next_n == -INFINITY ? 0.f : exp2_fast(next_m - next_n);
#pragma unroll
      for (int c = 0; c < D / 16; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) a.o[rt][c][i] *= shrink;
    }
    // (a row that has kept nothing so far has reference -inf, and only masked logits)
    const float ref = a.m[rt] == -INFINITY ? 0.f : a.m[rt] - kLift, value = value_factor(a.ratio[rt], v_scale);
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[i] = exp2_fast(x[i] - ref);
      float y = w[i] * value;
      // (fixed here: the compiler may fuse the product with one of its two uses and round the other in two steps, which
      // near a tie of f16 leaves the second term for another first term)
      asm("" : "+v"(y));
      high[rt][i] = (_Float16)y;
      low[rt][i] = (_Float16)(y - (float)high[rt][i]);
    }
    a.l[rt] += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
  }
}

// A partial tile's value codes: tokens that no row of the block keeps may hold anything and become 0.  NaN in a kept one is for the rows
// that keep the token, and only for those, but a weight of 0 would not stop it in the product: it goes on as 0 too, and the block's end
// sees to it.  Lane (n16, g) has tokens 4 g + j % 4 (+ 16 from j = 4 on).
template <int D, int RT, bool TREE>
__device__ __forceinline__ void sanitize(const GqaDecodeParams& p, Rows<D, RT>& a, typename VWord<D / 64>::type (&v)[8], const Span& now, int pos0, int g) {
  constexpr int kWords = D / 64;
  const int lo = now.lo, hi = now.hi;
  uint32_t any_nan = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int pos = pos0 + (j < 4 ? 0 : 16) + 4 * g + j % 4;
    const bool keep = pos < hi && (pos < p.S || (p.W > 0 && pos >= lo - p.W) || (TREE && pos >= now.text));
    if (!keep) v[j] = typename VWord<kWords>::type{};
#pragma unroll
    for (int i = 0; i < kWords; ++i) any_nan |= nan_codes(word<kWords>(v[j], i));
  }
  if ((TREE || now.several) && __ballot(any_nan != 0) != 0) {
    a.saw_nan = 1.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = without_nan<kWords>(v[j]);
  }
}

// O^T += V^T P^T
template <int D, int RT>
__device__ __forceinline__ void add_values(Rows<D, RT>& a, const typename VWord<D / 64>::type (&v)[8], const f16x8 (&high)[RT], const f16x8 (&low)[RT]) {
  constexpr int kWords = D / 64;
#pragma unroll
  for (int wd = 0; wd < kWords; ++wd) {
#pragma unroll
    for (int col = 0; col < 4; ++col) {
      u32x4 f;
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = f16_pair(token_pair(word<kWords>(v[2 * j], wd), word<kWords>(v[2 * j + 1], wd), col / 2), col % 2);
      const f16x8 vt = __builtin_bit_cast(f16x8, f);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        f32x4& acc = a.o[rt][4 * wd + col];
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(vt, high[rt], acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(vt, low[rt], acc, 0, 0, 0);
      }
    }
  }
}

// A K operand of S^T from its codes: 8 columns of one token.
__device__ __forceinline__ bf16x8 k_operand(uint32_t lo, uint32_t hi) {
  const u32x4 w = {bf16_pair(lo, false), bf16_pair(lo, true), bf16_pair(hi, false), bf16_pair(hi, true)};
  return __builtin_bit_cast(bf16x8, w);
}

// Whether a block's query rows keep any of the 32 tokens from pos0 on, and all of them.
struct Kept {
  bool some, full;
};
template <bool TREE>
__device__ __forceinline__ Kept kept_of(const GqaDecodeParams& p, const Span& now, int pos0) {
  const int lo = now.lo, hi = now.hi;
  if constexpr (TREE)
    return Kept{pos0 < hi && (pos0 < p.S || (p.W > 0 && pos0 + kWaveTokens > lo - p.W) || pos0 + kWaveTokens > now.text),
                pos0 + kWaveTokens <= now.text && (pos0 + kWaveTokens <= p.S || pos0 >= hi - p.W)};
  return Kept{pos0 < hi && (pos0 < p.S || (p.W > 0 && pos0 + kWaveTokens > lo - p.W)),
              pos0 + kWaveTokens <= lo && (pos0 + kWaveTokens <= p.S || pos0 >= hi - p.W)};
}

// End of a block: the shares of the TG waves that hold the same rows (tokens apart) meet in LDS, references and sums first (ml: [TG][R]),
// then the outputs at the common reference, 1 / PARTS of every lane's columns at a time (o_lds: [TG][R][D / PARTS + 4]).  tg: which of the TG
// the wave is; row0: its first row.  Blocks that other work groups share too leave partial rows in `slot`.
template <int D, int RT, int R, int TG, int PARTS, int THREADS, bool OUT32, int START, bool TREE>
__device__ __forceinline__ void finish(const Dealer<R, THREADS, START, 1, TREE>& dealer, const Piece& now, Rows<D, RT>& a, float* o_lds, float4* ml,
                                       int tg, int row0, int slot) {
  constexpr int kCols = D / 16, kOStride = D / PARTS + 4;
  const int tid = threadIdx.x, lane = tid & 63, n16 = lane & 15, g = lane >> 4;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    a.l[rt] = row_sum(a.l[rt]);
    if (g == 0) ml[tg * R + row0 + rt * 16 + n16] = make_float4(a.m[rt], a.l[rt], a.n[rt], a.saw_nan);
  }
  lds_barrier();
  float shrink[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < TG; ++w) top = fmaxf(top, ml[w * R + row0 + rt * 16 + n16].z);
    // (a wave that kept nothing has zeros, or NaN that has to stay: nothing is skipped)
    shrink[rt] = factor(a.n[rt], top);
  }
  const GqaDecodeParams& end = *late_arguments();
  constexpr int kChunks = D / 8 / PARTS, kEach = 4 / PARTS;
  const int rows = dealer.rows_of(now);
  const bool whole = now.whole();
#pragma unroll
  for (int part = 0; part < PARTS; ++part) {
    if (part) lds_barrier();  // (the part before has been read)
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float* const dst = o_lds + (tg * R + row0 + rt * 16 + n16) * kOStride + g * kEach * kCols;
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        const int i = part * kEach + j;
#pragma unroll
        for (int c = 0; c < kCols; c += 4)
          *(f32x4*)(dst + j * kCols + c) = f32x4{a.o[rt][c][i] * shrink[rt], a.o[rt][c + 1][i] * shrink[rt], a.o[rt][c + 2][i] * shrink[rt], a.o[rt][c + 3][i] * shrink[rt]};
      }
    }
    lds_barrier();
    for (int k = tid; k < rows * kChunks; k += THREADS) {
      const int row = k / kChunks, in_part = k % kChunks * 8;
      const int col = in_part / (kEach * kCols) * 4 * kCols + part * kEach * kCols + in_part % (kEach * kCols);
      f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
      float top = -INFINITY, vtop = -INFINITY, sum = 0.f, nans = 0.f;
#pragma unroll
      for (int w = 0; w < TG; ++w) {
        top = fmaxf(top, ml[w * R + row].x);
        vtop = fmaxf(vtop, ml[w * R + row].z);
        nans += ml[w * R + row].w;
      }
#pragma unroll
      for (int w = 0; w < TG; ++w) {
        const float4 e = ml[w * R + row];
        sum += e.y * factor(e.x, top);
        const f32x4* src = (const f32x4*)(o_lds + (w * R + row) * kOStride + in_part);
        lo += src[0];
        hi += src[1];
      }
      const uint32_t qt = (uint32_t)(now.rb * R + row) / (uint32_t)end.group, gi = (uint32_t)(now.rb * R + row) - qt * end.group;
      if (__builtin_expect(nans != 0.f, 0)) {
        // NaN that the loop has taken for 0: the columns of the tokens that this row keeps are looked through again
        const Sight<TREE> sight = sight_of<TREE>(end, now, (int)qt, true);
#pragma unroll 1
        for (int tile = now.tile_lo; tile < now.tile_hi; ++tile) {
          const int lp = now.bk.pages.logical(tile);
          const size_t ph = (size_t)end.page_table[now.b * end.table_stride + lp] * end.kv_heads + now.h;
#pragma unroll 1
          for (int j = 0; j < kPage; ++j) {
            if (!sees<TREE>(end, sight, now.rq.L - now.rq.n, lp * kPage + j)) continue;
            const u32x2 codes = *(const u32x2*)(end.v_cache + (ph * kPage + j) * D + col);
            const uint32_t nan_lo = nan_codes(codes[0]), nan_hi = nan_codes(codes[1]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if ((nan_lo >> (8 * i)) & 0x80u) lo[i] = NAN;
              if ((nan_hi >> (8 * i)) & 0x80u) hi[i] = NAN;
            }
          }
        }
      }
      const int64_t out_row = (int64_t)(now.rq.begin + (int)qt) * end.q_heads + now.h * end.group + (int)gi;
      if (whole) {
        const float inv = sum == 0.f ? 0.f : exp2_fast(vtop - top) / sum;  // (nothing kept: 0 and -inf)
        if constexpr (OUT32) {
          f32x4* dst = (f32x4*)((float*)end.out + out_row * D + col);
          dst[0] = lo * inv;
          dst[1] = hi * inv;
        } else {
          bf16x8 y;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            y[i] = (__bf16)(lo[i] * inv);
            y[4 + i] = (__bf16)(hi[i] * inv);
          }
          *(bf16x8*)((uint16_t*)end.out + out_row * D + col) = y;
        }
        if (col == 0) {
          end.lse[out_row] = sum == 0.f ? -INFINITY : (top + __log2f(sum) - kLift) * 0.69314718055994531f;
          end.rows[out_row] = make_int2(0, 0);
        }
      } else {
        float* dst = end.part_o + ((size_t)slot * R + row) * D + col;
        ((f32x4*)dst)[0] = lo;
        ((f32x4*)dst)[1] = hi;
        if (col == 0) {
          end.part_ml[(size_t)slot * R + row] = make_float4(top, sum, vtop, 0.f);
          // the share that has a block's first page knows which ones have the others
          if (now.tile_lo == 0) end.rows[out_row] = make_int2(slot, dealer.partners(now) * 64 + row);
        }
      }
    }
  }
}

// End of a block that one wave computes by itself, one row tile: every lane has D / 4 adjacent columns of its row, and writes them.
template <int D, int THREADS, bool OUT32, int START, int SHARES, bool TREE>
__device__ __forceinline__ void finish_alone(const Dealer<16, THREADS, START, SHARES, TREE>& dealer, const Piece& now, Rows<D, 1>& a, int slot) {
  constexpr int kCols = D / 16, kQuarters = kPage / kWaveTokens;
  const int lane = threadIdx.x & 63, row = lane & 15, g = lane >> 4, col = 4 * g * kCols;
  const float sum = row_sum(a.l[0]);
  if (row >= dealer.rows_of(now)) return;
  const GqaDecodeParams& end = *late_arguments();
  const uint32_t qt = (uint32_t)(now.rb * 16 + row) / (uint32_t)end.group, gi = (uint32_t)(now.rb * 16 + row) - qt * end.group;
  if (__builtin_expect(a.saw_nan != 0.f, 0)) {  // (as in finish)
    const Sight<TREE> sight = sight_of<TREE>(end, now, (int)qt, true);
    uint32_t nans = 0;  // of the lane's columns
#pragma unroll 1
    for (int tile = now.tile_lo; tile < now.tile_hi; ++tile) {
      const int lp = now.bk.pages.logical(tile);
      const size_t ph = (size_t)end.page_table[now.b * end.table_stride + lp / kQuarters] * end.kv_heads + now.h;
#pragma unroll 1
      for (int j = 0; j < kWaveTokens; ++j) {
        if (!sees<TREE>(end, sight, now.rq.L - now.rq.n, lp * kWaveTokens + j)) continue;
        const uint32_t* codes = (const uint32_t*)(end.v_cache + (ph * kPage + lp % kQuarters * kWaveTokens + j) * D + col);
#pragma unroll 1
        for (int i = 0; i < kCols; ++i) {
          const uint32_t n = nan_codes(codes[i]);
          nans |= ((n >> 7 & 1) | (n >> 14 & 2) | (n >> 21 & 4) | (n >> 28 & 8)) << (4 * i);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < kCols; ++c)
        if (nans >> (i * kCols + c) & 1) a.o[0][c][i] = NAN;
  }
  const int64_t out_row = (int64_t)(now.rq.begin + (int)qt) * end.q_heads + now.h * end.group + (int)gi;
  if (now.whole()) {
    const float inv = sum == 0.f ? 0.f : exp2_fast(a.n[0] - a.m[0]) / sum;  // (nothing kept: 0 and -inf)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < kCols; c += 4) {
        const int64_t at = out_row * D + col + i * kCols + c;
        if constexpr (OUT32) {
          *(f32x4*)((float*)end.out + at) = f32x4{a.o[0][c][i] * inv, a.o[0][c + 1][i] * inv, a.o[0][c + 2][i] * inv, a.o[0][c + 3][i] * inv};
        } else {
          typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
          bf16x4 y;
#pragma unroll
          for (int k = 0; k < 4; ++k) y[k] = (__bf16)(a.o[0][c + k][i] * inv);
          *(bf16x4*)((uint16_t*)end.out + at) = y;
        }
      }
    if (g == 0) {
      end.lse[out_row] = sum == 0.f ? -INFINITY : (a.m[0] + __log2f(sum) - kLift) * 0.69314718055994531f;
      end.rows[out_row] = make_int2(0, 0);
    }
  } else {
    float* const dst = end.part_o + ((size_t)slot * 16 + row) * D + col;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < kCols; c += 4) *(f32x4*)(dst + i * kCols + c) = f32x4{a.o[0][c][i], a.o[0][c + 1][i], a.o[0][c + 2][i], a.o[0][c + 3][i]};
    if (g == 0) {
      end.part_ml[(size_t)slot * 16 + row] = make_float4(a.m[0], sum, a.n[0], 0.f);
      if (now.tile_lo == 0) end.rows[out_row] = make_int2(slot, dealer.partners(now) * 64 + row);
    }
  }
}

}  // namespace
}  // namespace omniattn
