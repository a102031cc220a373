// Attention of the nodes of drafted trees (see gqa_decode_kernel.hip for the formulas and how the work is dealt out) with more than 32 query
// rows to a request and KV head, heads of 128.
//
// A block has up to 128 rows.  A wave computes 32 of them, with the 32x32x16 matrix instructions: S^T = K Q^T leaves a lane 16 logits of one row, so that
// a row's maximum, sum and references are one lane's.  A block of 32 rows gives each of the four waves 32 tokens of a page; one of 64 rows gives two
// waves 64 tokens each for every half of its rows; of more, every wave all tokens of a page for its rows.  (So the codes come from memory once for all
// rows of a block: waves with other rows ask for the same ones at about the same time.)  No LDS and no barrier in the loop but for the query's
// operands, which come from LDS.
//
// What bounds it: from 96 rows on the vector and matrix instructions of the two waves of a SIMD, which take their times one after the other (of a step of 32
// rows and tokens 24 products, 32 clocks each, and 259 vector instructions, 4.3 each: codes to 16 bits, exponentials, two terms of each weight).  Where
// trees are ragged, work groups that end early too: of 64 of up to 64 nodes the vector units are at work 52 % and the matrix units 36 % of the time that compute
// units have waves, and that is four fifths of the kernel's; a wave lives for 72 % of it in the mean.
// 64 requests of 6000 tokens, 8 KV heads: 128 rows 387 us, 520 TFLOP/s (780 with the second terms of the weights); 48 rows 222 us, 3.5 TB/s.  Without
// the second terms it would be 13 in a hundred faster, and off by 2^-11 of a weight; without exponentials 5.  Heads of 256: sums of 32 rows take
// half of a wave's registers and leave room for one tile under way; so a kernel of this kind took 222 us where the wide one takes 138 (64 requests of
// 6000 tokens, 64 rows, 2 KV heads), as loads are waited for.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "gqa_common.h"

namespace omniattn {
namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16;

constexpr int kThreads = 256, kTreeStart = 2;
constexpr int kTreeRowSlots = 128;  // (a partial row says how many there are in units of this)

constexpr int D = 128;

struct TreeShape {
  static constexpr int kRowTiles = 4;                  // of 32 rows
  static constexpr int kRows = 32 * kRowTiles;
  static constexpr int kCols = D / 32;                 // columns of a lane: 32 lanes share a value row
  static constexpr int kSteps = D / 16;                // of S^T
  static constexpr int kParts = 4;                     // the output's columns meet 1 / kParts at a time
  static constexpr int kOStride = D / kParts + 4;      // floats of a row in LDS
  static constexpr size_t kQ = (size_t)kRowTiles * kSteps * 64 * 16;  // bytes of a block's query operands
  static constexpr size_t kLds = (size_t)4 * 32 * kOStride * 4 + 2 * 4 * 32 * 16 + kQ;
};

// How the four waves share a block: 2^shift of them 32 tokens apart have the same rows.
struct Roles {
  int shift;
  __device__ __forceinline__ explicit Roles(int rows) : shift(rows <= 32 ? 2 : rows <= 64 ? 1 : 0) {}
  __device__ __forceinline__ int row_tile(int wave) const { return wave >> shift; }
  __device__ __forceinline__ int tokens(int wave) const { return wave & ((1 << shift) - 1); }  // which of them the wave is
  __device__ __forceinline__ int grain() const { return kWaveTokens << shift; }                 // tokens of a unit of work (see tree_split)
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t codes_at(const uint8_t* base, uint32_t bytes) {
  const uint64_t a = uniform64((uint64_t)(uintptr_t)base);
  return __builtin_amdgcn_make_buffer_rsrc((void*)(uintptr_t)a, 0, (int)__builtin_amdgcn_readfirstlane(bytes), 0x00027000);
}

// Codes of a wave's tile.  Lane (m, h), m below 32: of K, token m's columns 32 c + 16 h + 0..15; of V, columns m D/32 + 0.. of the tokens
// 8 i + 4 h + 0..3.
struct TreeTile {
  u32x4 k[D / 32];
  uint32_t v[16];
  float ks, vs;  // scales
};
__device__ __forceinline__ void load_k(TreeTile& t, __amdgpu_buffer_rsrc_t rsrc, int at) {
#pragma unroll
  for (int c = 0; c < D / 32; ++c) t.k[c] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at + 32 * c, 0, 0));
}
__device__ __forceinline__ void load_v(TreeTile& t, __amdgpu_buffer_rsrc_t rsrc, int at) {
#pragma unroll
  for (int j = 0; j < 16; ++j)
    t.v[j] = __builtin_amdgcn_raw_buffer_load_b32(rsrc, at + (8 * (j / 4) + j % 4) * D, 0, 0);
}
__device__ __forceinline__ void settle(int& x) { asm volatile("" : "+v"(x)); }

// A wave's share of the output rows (as Rows in gqa_common.h): lane (m, h) has row m of the wave's 32, and of O columns (8 (i / 4) + 4 h + i % 4) D/32 + c.
struct TreeRows {
  static constexpr int kCols = TreeShape::kCols;
  f32x16 o[kCols];
  float m, n, l, ratio, saw_nan;
  __device__ __forceinline__ void clear() {
    m = n = -INFINITY;
    l = ratio = saw_nan = 0.f;
#pragma unroll
    for (int c = 0; c < kCols; ++c) o[c] = f32x16{};
  }
};

__device__ __forceinline__ float halves_max(float x) {  // over the two lanes that hold tokens of the same row
  float y = x;
  swap32(x, y);
  return fmaxf(x, y);
}
__device__ __forceinline__ float halves_sum(float x) {
  float y = x;
  swap32(x, y);
  return x + y;
}

typedef __attribute__((ext_vector_type(2))) float f32x2;

// Weights of a tile's 32 tokens from S^T, as weigh in gqa_common.h: references, sums, and two f16 terms (the first one rounded to zero, so that
// two conversions are an instruction; what it leaves is rounded to nearest: together 2^-22 of a weight).  Value i of a lane is token
// 8 (i / 4) + 4 h + i % 4; the terms' operand u has values 8 u + 0..7.
__device__ __forceinline__ void weigh(const GqaDecodeParams& p, TreeRows& a, f32x16& s, const Sight<true>& sight, int text, bool full, int pos0, int h,
                                      float k_factor, float v_scale, u32x4 (&high)[2], u32x4 (&low)[2]) {
  if (!full) {
    const uint32_t nodes = nodes_at(sight.nodes, pos0 - text) >> (4 * h);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int pos = pos0 + 8 * (i / 4) + 4 * h + i % 4;
      const bool node = nodes >> (8 * (i / 4) + i % 4) & 1, keep = retained(pos, sight.reach, p.S, p.W);
      s[i] = (pos < text ? keep : node) ? s[i] * k_factor : -INFINITY;
    }
    k_factor = 1.f;
  }
  float top = s[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
  top *= k_factor;
  // (a tile that no row keeps anything of can be among a tree's, and its scale be anything)
  if (!full && !__any(top > -INFINITY)) v_scale = 0.f;
  const float v_log = fmaxf(__log2f(v_scale), -100.f);
  if (__any(top > fminf(a.m, a.n - v_log) + kSlack)) {
    top = halves_max(top);
    const float next_m = top > a.m + kSlack ? top : a.m;
    const float next_n = top + v_log > a.n + kSlack ? top + v_log : a.n;
    a.l *= factor(a.m, next_m);
    const float shrink = factor(a.n, next_n);
    a.m = next_m;
    a.n = next_n;
    a.ratio = next_n == -INFINITY ? 0.f : exp2_fast(next_m - next_n);
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) a.o[c][i] *= shrink;
  }
  const float ref = a.m == -INFINITY ? 0.f : a.m - kLift, value = value_factor(a.ratio, v_scale);
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 16; i += 2) {
    const float w0 = exp2_fast(fmaf(s[i], k_factor, -ref)), w1 = exp2_fast(fmaf(s[i + 1], k_factor, -ref));
    float y0 = w0 * value, y1 = w1 * value;
    asm("" : "+v"(y0), "+v"(y1));  // (see weigh in gqa_common.h)
    const f16x2 first = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(y0, y1));
    f32x2 rest;  // (in one instruction each: y - first)
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(rest[0]) : "v"(first), "v"(y0));
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(rest[1]) : "v"(first), "v"(y1));
    high[i / 8][i / 2 % 4] = __builtin_bit_cast(uint32_t, first);
    low[i / 8][i / 2 % 4] = __builtin_bit_cast(uint32_t, __builtin_convertvector(rest, f16x2));
    sum += w0 + w1;
  }
  a.l += sum;
}

// End of a block (as finish in gqa_common.h; o_lds: [4 waves][32 rows][kOStride], ml: [4 waves][32 rows]).
template <bool OUT32, typename DEALER>
__device__ __forceinline__ void finish(const DEALER& dealer, const Piece& now, TreeRows& a, float* o_lds, float4* ml, int wave, int slot) {
  using C = TreeShape;
  constexpr int R = C::kRows, kCols = C::kCols, kChunks = D / 8 / C::kParts;
  const int tid = threadIdx.x, lane = tid & 63, m32 = lane & 31, h = lane >> 5;
  const int rows = dealer.rows_of(now);
  const Roles roles(rows);
  a.l = halves_sum(a.l);
  if (h == 0) ml[wave * 32 + m32] = make_float4(a.m, a.l, a.n, a.saw_nan);
  lds_barrier();
  float shared = -INFINITY;
  for (int w = 0; w < 1 << roles.shift; ++w) shared = fmaxf(shared, ml[((roles.row_tile(wave) << roles.shift) + w) * 32 + m32].z);
  const float shrink = factor(a.n, shared);  // (nothing is skipped: NaN has to stay)
  const GqaDecodeParams& end = *late_arguments();
  const bool whole = now.whole();
#pragma unroll
  for (int part = 0; part < C::kParts; ++part) {
    if (part) lds_barrier();
    float* const dst = o_lds + (wave * 32 + m32) * C::kOStride + 4 * h * kCols;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int c = 0; c < kCols; c += 4) {
        const int i = 4 * part + j;
        *(f32x4*)(dst + j * kCols + c) = f32x4{a.o[c][i] * shrink, a.o[c + 1][i] * shrink, a.o[c + 2][i] * shrink, a.o[c + 3][i] * shrink};
      }
    lds_barrier();
    for (int k = tid; k < rows * kChunks; k += kThreads) {
      const int row = k / kChunks, in_part = k % kChunks * 8, col = part * (D / C::kParts) + in_part;
      f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
      float top = -INFINITY, vtop = -INFINITY, sum = 0.f, nans = 0.f;
      const int first = ((row / 32) << roles.shift) * 32 + row % 32;
      for (int w = 0; w < 1 << roles.shift; ++w) {
        const float4 e = ml[first + w * 32];
        top = fmaxf(top, e.x);
        vtop = fmaxf(vtop, e.z);
        nans += e.w;
      }
      for (int w = 0; w < 1 << roles.shift; ++w) {
        const float4 e = ml[first + w * 32];
        sum += e.y * factor(e.x, top);
        const f32x4* src = (const f32x4*)(o_lds + (first + w * 32) * C::kOStride + in_part);
        lo += src[0];
        hi += src[1];
      }
      const uint32_t qt = (uint32_t)(now.rb * R + row) / (uint32_t)end.group, gi = (uint32_t)(now.rb * R + row) - qt * end.group;
      if (__builtin_expect(nans != 0.f, 0)) {
        const Sight<true> sight = sight_of<true>(end, now, (int)qt, true);
#pragma unroll 1
        for (int tile = now.tile_lo; tile < now.tile_hi; ++tile) {
          const int pos0 = now.bk.pages.logical(tile) * roles.grain();
          const size_t ph = (size_t)end.page_table[now.b * end.table_stride + pos0 / kPage] * end.kv_heads + now.h;
#pragma unroll 1
          for (int j = 0; j < roles.grain(); ++j) {
            if (!sees<true>(end, sight, now.rq.L - now.rq.n, pos0 + j)) continue;
            const u32x2 codes = *(const u32x2*)(end.v_cache + (ph * kPage + pos0 % kPage + j) * D + col);
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
          if (now.tile_lo == 0) end.rows[out_row] = make_int2(slot, dealer.partners(now) * kTreeRowSlots + row);
        }
      }
    }
  }
}

template <bool OUT32>
__global__ __launch_bounds__(kThreads, 2) void gqa_tree_kernel(GqaDecodeParams p) {
  using C = TreeShape;
  constexpr int R = C::kRows, kCols = C::kCols, kSteps = C::kSteps;
  using Deal = Dealer<R, kThreads, kTreeStart, 1, true>;
  extern __shared__ __align__(16) float lds[];
  float* const o_lds = lds;                                       // [4 waves][32][kOStride]
  float4* const ml_lds = (float4*)(lds + 4 * 32 * C::kOStride);   // [2][4 waves][32]
  bf16x8* const q_lds = (bf16x8*)(ml_lds + 2 * 4 * 32);           // [row tiles][kSteps][64 lanes]
  __shared__ typename Deal::Lds dealt;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int m32 = lane & 31, h = lane >> 5;
  Deal dealer(p, dealt);
  Piece now;
  if (!dealer.begin(now)) return;

  const int k_at = m32 * D + h * 16, v_at = 4 * h * D + m32 * kCols;
  const int blocks_per_page = kPage >> p.scale_shift;
  int parity = 0, first_partial = 0;
  // The wave's tiles: 32 tokens of every unit, of which a page has 2^split.
  int split = 0, mine = 0;
  auto take_part = [&](const Piece& w) {
    const Roles roles(uniform(dealer.rows_of(w)));
    split = 2 - roles.shift;
    mine = roles.tokens(wave) * kWaveTokens;
  };
  auto entries = [&](int b, const TileLayout& pages, int from) {
    const int last = pages.count() - 1;
    return last >= 0 ? p.page_table[b * p.table_stride + (pages.logical(min(from + lane, last)) >> split)] : 0;
  };
  // What a block's queries are to the wave: what its row sees, and whether one of its rows keeps nothing, not even of tiles that all others keep.
  Sight<true> sight;
  bool blind = false;
  auto look = [&](const Piece& w) {
    const int rows = dealer.rows_of(w), row = Roles(rows).row_tile(wave) * 32 + m32;
    const uint32_t t = (uint32_t)(w.rb * R + row) / (uint32_t)p.group;
    sight = sight_of<true>(p, w, (int)t, row < rows);
    blind = __any(row < rows && sight.reach == 0);
  };
  // The block's query operands, a quarter by each wave; all waves find them behind the next barrier.  Operand 2 c + u of lane (m, h): row m's columns
  // 32 c + 16 h + 8 u + 0..7.  Rows past the last hold zeros.
  auto bring_q = [&](const Piece& w) {
    const int rows = dealer.rows_of(w);
    for (int rt = 0; rt * 32 < rows; ++rt) {
      const int row = rt * 32 + m32;
      const uint32_t t = (uint32_t)(w.rb * R + row) / (uint32_t)p.group, gi = (uint32_t)(w.rb * R + row) - t * p.group;
      const uint16_t* src = p.q + (int64_t)(w.rq.begin + (int)t) * p.q_stride + (size_t)(w.h * p.group + (int)gi) * D + h * 16;
      bf16x8 q[kSteps / 4];
#pragma unroll
      for (int i = 0; i < kSteps / 4; ++i) {
        const int k = 4 * i + wave;
        q[i] = row < rows ? *(const bf16x8*)(src + k / 2 * 32 + k % 2 * 8) : bf16x8{};
        // (so that the softmax factor is not negative, and a row's largest product its largest logit)
        if (p.scale_log2 < 0.f) q[i] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, q[i]) ^ 0x80008000u);
      }
#pragma unroll
      for (int i = 0; i < kSteps / 4; ++i) q_lds[(rt * kSteps + 4 * i + wave) * 64 + lane] = q[i];
    }
  };
  struct Codes {
    __amdgpu_buffer_rsrc_t k, v;
  };
  const Codes none = {codes_at(p.k_cache, 0), codes_at(p.v_cache, 0)};
  auto first_of = [&](const TileLayout& pages, int tile) { return (pages.logical(tile) << (7 - split)) + mine; };
  auto aim = [&](TreeTile& t, const Span& span, int head, int tile, int ids, int held) {
    const int page = __builtin_amdgcn_readlane(ids, tile - held);
    const int pos = first_of(span.pages, tile), first = pos % kPage, live = max(min(span.hi - pos, kWaveTokens), 0);
    const size_t ph = (size_t)page * p.kv_heads + head, block = ph * blocks_per_page + (first >> p.scale_shift), code = (ph * kPage + first) * D;
    t.ks = p.k_scales[block];
    t.vs = p.v_scales[block];
    return Codes{codes_at(p.k_cache + code, live * D), codes_at(p.v_cache + code, live * D)};
  };

  // Two tiles are under way: while one is computed, the loads of the one behind the other go out as soon as their registers are free.
  TreeTile even, odd;
  int held = 0, ids = 0, tile = 0, b = 0, head = 0, row_tile = 0;
  bool idle = false;  // (a block of 65 to 96 rows: the last wave has none)
  Span span(now);
  auto begin_block = [&](const Piece& w) {
    const int rows = uniform(dealer.rows_of(w));
    take_part(w);
    look(w);
    span = Span(w);
    tile = uniform(w.tile_lo);
    b = uniform(w.b);
    head = uniform(w.h);
    row_tile = Roles(rows).row_tile(wave);
    idle = row_tile * 32 >= rows;
    held = tile;
    ids = entries(b, span.pages, held);
    settle(ids);
    Codes c = none;
    if (tile < span.tile_hi) c = aim(even, span, head, tile, ids, held);
    load_k(even, c.k, k_at);
    load_v(even, c.v, v_at);
    c = none;
    if (tile + 1 < span.tile_hi) c = aim(odd, span, head, tile + 1, ids, held);
    load_k(odd, c.k, k_at);
    load_v(odd, c.v, v_at);
  };
  begin_block(now);
  dealer.keep(0, now);
  bring_q(now);
  lds_barrier();

  while (true) {
    TreeRows a;
    a.clear();
    auto step = [&](TreeTile& t) {
      // (asked for together: one by one, each product would wait for its own)
      bf16x8 q[kSteps];
#pragma unroll
      for (int i = 0; i < kSteps; ++i) q[i] = q_lds[(row_tile * kSteps + i) * 64 + lane];
      __builtin_amdgcn_sched_barrier(0);
      const int pos0 = first_of(span.pages, tile);
      Kept kept = kept_of<true>(p, span, pos0);
      kept.full = kept.full && !blind;
      // (products before other waves' vector instructions, which they leave room for: 2 in a hundred)
      __builtin_amdgcn_s_setprio(1);
      f32x16 s = {};
#pragma unroll
      for (int i = 0; i < kSteps; ++i)
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_operand(t.k[i / 2][i % 2 * 2], t.k[i / 2][i % 2 * 2 + 1]), q[i], s, 0, 0, 0);
      __builtin_amdgcn_s_setprio(0);
      const float k_factor = fabsf(p.scale_log2) * t.ks, v_scale = kept.some ? t.vs : 0.f;
      Codes c = none;
      if (tile + 2 < span.tile_hi) {
        if (tile + 2 - held >= 64) {
          held = tile + 2;
          ids = entries(b, span.pages, held);
          settle(ids);
        }
        c = aim(t, span, head, tile + 2, ids, held);
      }
      load_k(t, c.k, k_at);
      u32x4 high[2], low[2];
      weigh(p, a, s, sight, span.text, kept.full, pos0, h, k_factor, v_scale, high, low);
      if (!kept.full) {
        // tokens that no row of the block keeps may hold anything; NaN in kept ones goes on as 0 (see sanitize in gqa_common.h)
        uint32_t any_nan = 0;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int pos = pos0 + 8 * (j / 4) + 4 * h + j % 4;
          const bool keep = pos < span.hi && (pos < p.S || (p.W > 0 && pos >= span.lo - p.W) || pos >= span.text);
          if (!keep) t.v[j] = 0;
          any_nan |= nan_codes(t.v[j]);
        }
        if (__ballot(any_nan != 0) != 0) {
          a.saw_nan = 1.f;
#pragma unroll
          for (int j = 0; j < 16; ++j) t.v[j] = without_nan<1>(t.v[j]);
        }
      }
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int col = 0; col < 4; ++col) {
          u32x4 f;
#pragma unroll
          for (int j = 0; j < 4; ++j) f[j] = f16_pair(token_pair(t.v[8 * u + 2 * j], t.v[8 * u + 2 * j + 1], col / 2), col % 2);
          const f16x8 vt = __builtin_bit_cast(f16x8, f);
          f32x16& acc = a.o[col];
          acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(vt, __builtin_bit_cast(f16x8, high[u]), acc, 0, 0, 0);
          acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(vt, __builtin_bit_cast(f16x8, low[u]), acc, 0, 0, 0);
        }
      __builtin_amdgcn_s_setprio(0);
      load_v(t, c.v, v_at);
      ++tile;
    };
    if (!idle) {
      while (tile + 1 < span.tile_hi) {
        step(even);
        step(odd);
      }
      if (tile < span.tile_hi) step(even);
    }
    Piece next = dealer.kept(0);
    const bool more_blocks = dealer.follow(next);
    if (more_blocks) {
      dealer.keep(1, next);
      begin_block(next);
    }
    finish<OUT32>(dealer, dealer.kept(0), a, o_lds, ml_lds + parity * 4 * 32, wave, 2 * (int)blockIdx.x + first_partial);
    parity ^= 1;
    first_partial = 1;
    if (!more_blocks) break;
    next = dealer.kept(1);
    dealer.keep(0, next);
    bring_q(next);  // (behind the barriers of the block's end: no wave needs the operands before any more)
    lds_barrier();
  }
}

}  // namespace

hipError_t init_gqa_tree_kernels() {
  hipError_t e = hipSuccess;
  for (const void* kernel : {(const void*)gqa_tree_kernel<false>, (const void*)gqa_tree_kernel<true>})
    if (e == hipSuccess) e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)TreeShape::kLds);
  return e;
}

hipError_t launch_gqa_tree(const GqaDecodeParams& p, int shares, hipStream_t stream) {
  if (p.out_fp32) hipLaunchKernelGGL(gqa_tree_kernel<true>, dim3(shares), dim3(kThreads), TreeShape::kLds, stream, p);
  else hipLaunchKernelGGL(gqa_tree_kernel<false>, dim3(shares), dim3(kThreads), TreeShape::kLds, stream, p);
  return hipGetLastError();
}

}  // namespace omniattn
