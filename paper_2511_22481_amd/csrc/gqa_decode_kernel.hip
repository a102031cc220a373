// Attention of grouped-query layers over the paged 8-bit cache.
//
// Query token t of a request with L tokens, n of them new, sees the keys j < L - n + t + 1 that the compression rule
// keeps (j < S, or among the last W of them): out = sum_j p_j v_j / sum_j p_j, p_j = exp(scale q.k_j), lse = ln sum p_j.
//
// Work.  The query rows (t, head of the group) of one (request, KV head) are cut into blocks of 16, 32 or 64; a block
// reads the pages that hold kept tokens.  A block counts as many units as it has pages, and two for its start (its query, the
// meeting of the waves, its results).  All units of the call, in order of request, KV head and block, are dealt out evenly: work
// group u of U takes units [u T / U, (u + 1) T / U).  Every work group finds its share by itself from the lengths on the device, so
// the host needs to know nothing but the sizes of the arrays.  A block whose pages went to several groups leaves one partial row
// each, which gqa_combine_kernel joins.
//
// A page.  The four waves take 32 of its 128 tokens each and keep a running maximum, sum and output of their own; they meet
// only at the end of a block's share.  K rows come from memory in the operand order of S^T = K Q^T (16x16x32 bf16 matrix
// instructions; an e4m3 code is exact in bf16), V rows as 8 tokens x D/16 columns per lane, which a byte permutation turns
// into the operand of O^T += V^T P^T (f16: exact for the codes, two terms and so 2^-22 for the weights, which the reference
// scales into [0, 2^15]).  The contraction's order of tokens is free, so P^T is what S^T's layout already gives each lane.
// No LDS and no barrier in the loop (width 256: the query's operands come from LDS).  A block's scale is one number per wave and
// page: K's goes into the softmax factor, V's into the weights.
//
// Many short blocks of width 64: every wave has a share of its own and takes the four tiles of a page in turn, so that the waves
// need not meet.
//
// What bounds it: up to 32 rows (64 at width 64), memory.  A work group has one tile of each wave under way (16 to 64 KB a compute
// unit), asked for as soon as the registers of the tile before are free; the loads are without conditions and every wait is for as
// many as are needed, no more.  64 requests of 32768 tokens, 8 KV heads of width 128 (4.30 GB): 733 us, 5.9 TB/s, where nothing but
// reading them in this order reaches 6.25.  One request of 131072 (268 MB): 53 us, of which 5 pass before the first product (a chain
// of four loads: lengths, table, codes, query) and 3 at the end.  93 ragged requests of 200 to 20000, 4 KV heads: 78 us, 5 TB/s.
// 64 requests of 2000 to 16000, 4 KV heads of width 128, 32 rows: 108 us, 4.4 TB/s; above, gqa_wide_kernel.hip is faster.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "gqa_common.h"

namespace omniattn {
namespace {

constexpr int kThreads = 256;
// Work groups of a compute unit, as far as their registers allow.
constexpr int groups_per_cu(int head_dim, int row_tiles) { return head_dim == 64 && row_tiles == 1 ? 4 : 2; }

// Codes of one (page, KV head): `bytes` of them may be read, behind that the loads return zeros and touch no memory.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t codes_at(const uint8_t* base, uint32_t bytes) {
  const uint64_t a = uniform64((uint64_t)(uintptr_t)base);
  return __builtin_amdgcn_make_buffer_rsrc((void*)(uintptr_t)a, 0, (int)__builtin_amdgcn_readfirstlane(bytes), 0x00027000);
}

template <int D>
struct Tile {
  static constexpr int kWords = D / 64;
  u32x4 k[2][kWords];                     // [16-token half][64-byte piece]
  typename VWord<kWords>::type v[8];      // [token of the lane]
};

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

// Waits for a load's result here, where it has just been asked for, and not where it is used on other ways too: there the wait would be
// for everything that has been asked for since.
__device__ __forceinline__ void settle(int& x) { asm volatile("" : "+v"(x)); }

template <int D, int RT>
struct Narrow {
  static constexpr int kRows = 16 * RT;
  static constexpr int kParts = D * RT == 256 ? 2 : 1;  // the output's columns meet 1 / kParts at a time, so that LDS holds two work groups
  static constexpr int kOStride = D / kParts + 4;  // floats of a row in LDS
  // Width 256: the query operands are kept in LDS (two buffers, one for the next block); in registers they would leave one work
  // group to a compute unit.
  static constexpr bool kQLds = D == 256;
  static constexpr size_t kQBytes = kQLds ? (size_t)kRows * D * 2 : 0;
  static constexpr size_t kLds = (size_t)4 * kRows * kOStride * 4 + 2 * 4 * kRows * 16 + 2 * kQBytes;
};

template <int D, int RT, bool OUT32, bool ALONE>
__global__ __launch_bounds__(kThreads, groups_per_cu(D, RT)) void gqa_decode_kernel(GqaDecodeParams p) {
  using C = Narrow<D, RT>;
  using Deal = Dealer<C::kRows, kThreads, ALONE ? 4 : 2, ALONE ? 4 : 1>;
  constexpr int kGrain = Deal::kGrain;
  static_assert(!ALONE || (D == 64 && RT == 1));
  constexpr int R = C::kRows, kCols = D / 16, kWords = D / 64;
  extern __shared__ __align__(16) float lds[];
  float* const o_lds = lds;                                    // [4 waves][R][kOStride]
  float4* const ml_lds = (float4*)(lds + 4 * R * C::kOStride); // [2][4 waves][R]
  bf16x8* const q_lds = (bf16x8*)(ml_lds + 2 * 4 * R);         // [2][operands of the products][64 lanes]
  __shared__ typename Deal::Lds dealt;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  Deal dealer(p, dealt);
  Piece now;
  if (!dealer.begin(now)) return;

  const int k_at = n16 * D + g * 16, v_at = 4 * g * D + n16 * kCols;
  const int blocks_per_page = kPage >> p.scale_shift;
  int parity = 0, first_partial = 0;  // first_partial: 1 once this work group has left its first block behind

  // Page-table entries of up to 64 of a block's pages (or quarters, if the wave is alone) from number `from` on, one per lane.
  auto entries = [&](int b, const TileLayout& pages, int from) {
    const int last = pages.count() - 1;
    return last >= 0 ? p.page_table[b * p.table_stride + pages.logical(min(from + lane, last)) / (kPage / kGrain)] : 0;
  };
  // Query rows of a block: lane n16 of every group of 16 holds one row of each row tile, the columns that its K loads bring.  Rows past
  // the last hold zeros.  reach: tokens that the row's query sees.
  constexpr int kQs = C::kQLds ? kWords / 2 : 2 * kWords;  // operands of a row tile that the wave reads: its share, or all
  bf16x8 q[RT][kQs];
  int reach[RT];
  auto load_q = [&](const Piece& w) {
    const int rows = dealer.rows_of(w);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int row = rt * 16 + n16;
      const uint32_t t = (uint32_t)(w.rb * R + row) / (uint32_t)p.group, gi = (uint32_t)(w.rb * R + row) - t * p.group;
      const bool valid = row < rows;
      reach[rt] = valid ? w.reach((int)t) : 0;
      const uint16_t* src = p.q + (int64_t)(w.rq.begin + (int)t) * p.q_stride + (size_t)(w.h * p.group + (int)gi) * D + g * 16;
      // (operand 2 c + u holds columns 64 c + 16 g + 8 u on; in LDS, the wave brings those with the remainder `wave` by 4)
#pragma unroll
      for (int i = 0; i < kQs; ++i) {
        const int k = C::kQLds ? 4 * i + wave : i;
        q[rt][i] = valid ? *(const bf16x8*)(src + k / 2 * 64 + k % 2 * 8) : bf16x8{};
      }
    }
  };
  int q_side = 0;
  auto store_q = [&](int side) {  // (all waves find them behind the next barrier)
    if constexpr (C::kQLds) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int i = 0; i < kQs; ++i) q_lds[((side * RT + rt) * 2 * kWords + 4 * i + wave) * 64 + lane] = q[rt][i];
    }
  };
  auto query = [&](int rt, int i) {
    if constexpr (C::kQLds) return q_lds[((q_side * RT + rt) * 2 * kWords + i) * 64 + lane];
    else return q[rt][i];
  };
  // A tile: the wave's quarter of a page, or the next quarter if the wave is alone.  Its first token:
  auto first_of = [&](const TileLayout& pages, int tile) { return pages.logical(tile) * kGrain + (ALONE ? 0 : wave * kWaveTokens); };
  // A tile's loads: where its codes are (scalar registers, made where they are used), and the two scales.
  struct Codes {
    __amdgpu_buffer_rsrc_t k, v;
  };
  const Codes none = {codes_at(p.k_cache, 0), codes_at(p.v_cache, 0)};
  float ks = 0.f, vs = 0.f;
  auto aim = [&](const TileLayout& pages, int h, int seen, int tile, int ids, int held) {
    const int page = __builtin_amdgcn_readlane(ids, tile - held);
    const int pos = first_of(pages, tile), first = pos % kPage, live = max(min(seen - pos, kWaveTokens), 0);
    const size_t ph = (size_t)page * p.kv_heads + h, block = ph * blocks_per_page + (first >> p.scale_shift), code = (ph * kPage + first) * D;
    ks = p.k_scales[block];
    vs = p.v_scales[block];
    return Codes{codes_at(p.k_cache + code, live * D), codes_at(p.v_cache + code, live * D)};
  };

  Tile<D> t;
  int held = now.tile_lo, ids = entries(now.b, now.bk.pages, held);
  settle(ids);
  load_q(now);
  Span span(now);
  int tile = uniform(now.tile_lo);
  {
    Codes c = none;
    if (tile < span.tile_hi) c = aim(span.pages, now.h, span.hi, tile, ids, held);
    load_k<D>(t, c.k, k_at);
    load_v<D>(t, c.v, v_at);
  }
  if constexpr (C::kQLds) {
    store_q(0);
    lds_barrier();
  }
  // Entries of the next request's first block, asked for as soon as the one before it begins: short requests come and go faster
  // than a chain of loads from the table to the codes.
  int ahead_b = -1, ahead_ids = 0;
  // Of the block that is computed, what the loop needs; the rest is the wave's note 0, and the next block's note 1.
  dealer.keep(0, now);
  int b = uniform(now.b), h = uniform(now.h);

  while (true) {
    bool more_blocks = false;
    if (ahead_b <= b) {
      ahead_b = b + 1;
      if (ahead_b < p.batch) {
        const Request r = dealer.request(ahead_b);
        if (r.n > 0) ahead_ids = entries(ahead_b, block_of<R, kGrain>(p, r, 0).pages, 0);
      }
    }
    // What the next block is (asked late, so that its description need not be kept through the loop), its query, and where its first page
    // is: its entries are the same as this block's for another KV head, or were asked for before, or are asked for now.
    auto turn_to_next = [&] {
      const Piece was = dealer.kept(0);
      Piece next = was;
      more_blocks = dealer.follow(next);
      if (!more_blocks) return none;
      dealer.keep(1, next);
      load_q(next);
      if (next.tile_lo >= next.tile_hi) return none;
      if (!(next.b == was.b && next.rb == was.rb && held == 0)) {
        held = 0;
        ids = next.b == ahead_b && next.rb == 0 ? ahead_ids : entries(next.b, next.bk.pages, 0);
        settle(ids);
      }
      return aim(next.bk.pages, next.h, next.reach(next.bk.t1), next.tile_lo, ids, held);
    };
    Rows<D, RT> a;
    a.clear();

    // A page; the loads of the one behind it go out as soon as their registers are free.  (They go out in any case, behind the share's last
    // page with nothing to read: were they conditional, the wait for K in the next pass would have to be for V's too.  And the last page
    // of a block is a copy of its own: what it has to find out would otherwise be carried through every pass.)
    auto step = [&](auto last) {
      const int pos0 = first_of(span.pages, tile);
      const Kept kept = kept_of(p, span, pos0);
      f32x4 s[RT][2];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[rt][0] = s[rt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 2 * kWords; ++i) {
        bf16x8 k[2];
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2) k[h2] = k_operand(t.k[h2][i / 2][i % 2 * 2], t.k[h2][i / 2][i % 2 * 2 + 1]);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          const bf16x8 x = query(rt, i);
#pragma unroll
          for (int h2 = 0; h2 < 2; ++h2) s[rt][h2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[h2], x, s[rt][h2], 0, 0, 0);
        }
      }
      // (the scale of a block without kept tokens may be anything)
      const float k_factor = p.scale_log2 * ks, v_scale = kept.some ? vs : 0.f;
      int seen[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) seen[rt] = reach[rt];
      Codes c;
      if constexpr (decltype(last)::value) {
        c = turn_to_next();
      } else {
        if (tile + 1 - held >= 64) {
          held = tile + 1;
          ids = entries(b, span.pages, held);
          settle(ids);
        }
        c = aim(span.pages, h, span.hi, tile + 1, ids, held);
      }
      load_k<D>(t, c.k, k_at);

      f16x8 high[RT], low[RT];
      weigh<D, RT>(p, a, s, seen, kept.full, pos0, g, k_factor, v_scale, high, low);
      if (!kept.full) sanitize<D, RT>(p, a, t.v, span, pos0, g);
      add_values<D, RT>(a, t.v, high, low);
      load_v<D>(t, c.v, v_at);
    };
    if (tile < span.tile_hi) {
      for (; tile + 1 < span.tile_hi; ++tile) step(std::false_type{});
      step(std::true_type{});
    } else {  // (nothing kept; the loads are waited for here, so that this rare way does not count where the waits of the others are set)
      const Codes c = turn_to_next();
      load_k<D>(t, c.k, k_at);
      load_v<D>(t, c.v, v_at);
#pragma unroll
      for (int i = 0; i < 2 * kWords; ++i) asm volatile("" : "+v"(t.k[i / kWords][i % kWords]));
#pragma unroll
      for (int j = 0; j < 8; ++j) asm volatile("" : "+v"(t.v[j]));
    }
    if (more_blocks) store_q(q_side ^ 1);
    q_side ^= 1;
    const int slot = 2 * dealer.share() + first_partial;
    if constexpr (ALONE) {
      finish_alone<D, kThreads, OUT32>(dealer, dealer.kept(0), a, slot);
    } else {
      finish<D, RT, R, 4, C::kParts, kThreads, OUT32>(dealer, dealer.kept(0), a, o_lds, ml_lds + parity * 4 * R, wave, 0, slot);
      parity ^= 1;
    }
    first_partial = 1;
    if (!more_blocks) break;
    const Piece next = dealer.kept(1);
    dealer.keep(0, next);
    b = next.b;
    h = next.h;
    span = Span(next);
    tile = next.tile_lo;
  }
}

// Joins the partial rows of blocks whose pages went to several work groups: o = sum_i 2^(n_i - n) o_i, l = sum_i 2^(m_i - m) l_i.  Partial i of a
// row lies in the slot of the i-th work group: the first one may have had another block before (slot 2 u + 1), the others
// begin with this one (2 u).  WAVES waves share a row, each every WAVES-th partial.
template <int D, bool OUT32, int WAVES, int BATCH>
__device__ __forceinline__ void join_row(const GqaDecodeParams& p, int64_t row, int first, int count, int in_block, int block_rows, float (*sh_o)[D], float4* sh_ml) {
  constexpr int kPer = D / 64;  // columns per lane
  typedef __attribute__((ext_vector_type(kPer))) float vec;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, u0 = first / 2;
  float m = -INFINITY, n = -INFINITY, l = 0.f;
  vec o = {};
  constexpr int kBatch = BATCH;
  for (int i0 = WAVES > 1 ? wave : 0; i0 < count; i0 += kBatch * WAVES) {
    float4 e[kBatch];
    vec x[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int i = min(i0 + k * WAVES, count - 1);
      const size_t slot = i == 0 ? first : 2 * (u0 + i);
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

// ROWS: to a wave (with one wave to a row), of which it joins those that are in parts.
template <int D, bool OUT32, int WAVES, int BATCH, int ROWS>
__global__ __launch_bounds__(64 * (WAVES > 4 ? WAVES : 4)) void gqa_combine_kernel(GqaDecodeParams p, int block_rows, int shares) {
  static_assert(WAVES == 1 || ROWS == 1);
  __shared__ float sh_o[WAVES > 1 ? WAVES : 1][D];
  __shared__ float4 sh_ml[WAVES];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t row0 = WAVES > 1 ? (int64_t)blockIdx.x : ((int64_t)blockIdx.x * 4 + wave) * ROWS, row = row0 + (ROWS > 1 ? lane : 0);
  int2 d = {0, 0};
  if (lane < ROWS || ROWS == 1) {
    if (row < (int64_t)p.num_queries * p.q_heads) {
      // (all three are asked for together)
      d = p.rows[row];
      const int token = (int)((uint32_t)row / (uint32_t)p.q_heads), first = p.q_start ? p.q_start[0] : 0, stop = p.q_start ? p.q_start[p.batch] : p.num_queries;
      const int count = d.y / 64;
      // (rows of no request: nothing was written for them)
      if (token < first || token >= stop || count <= 0 || d.x < 0 || d.x / 2 + count > shares) d.y = 0;
    }
  }
  if constexpr (ROWS == 1) {
    const int y = __builtin_amdgcn_readfirstlane(d.y);
    if (y >= 64) join_row<D, OUT32, WAVES, BATCH>(p, row, d.x, y / 64, y % 64, block_rows, sh_o, sh_ml);
  } else {
    for (uint64_t rest = __ballot(d.y >= 64); rest; rest &= rest - 1) {
      const int k = __builtin_ctzll(rest), y = __builtin_amdgcn_readlane(d.y, k);
      join_row<D, OUT32, 1, BATCH>(p, row0 + k, __builtin_amdgcn_readlane(d.x, k), y / 64, y % 64, block_rows, sh_o, sh_ml);
    }
  }
}

template <int D, bool OUT32>
hipError_t join(const GqaDecodeParams& p, int block_rows, int shares, hipStream_t stream) {
  const int64_t rows = (int64_t)p.num_queries * p.q_heads;
  // Few rows: eight waves to each.  Very many, of which few are in parts (prompts): a wave looks at 16 (524288 rows: 34 us less
  // than one to a wave).
  if (rows <= 2048) hipLaunchKernelGGL((gqa_combine_kernel<D, OUT32, 8, 4, 1>), dim3((uint32_t)rows), dim3(512), 0, stream, p, block_rows, shares);
  else if (rows <= 65536) hipLaunchKernelGGL((gqa_combine_kernel<D, OUT32, 1, 4, 1>), dim3((uint32_t)((rows + 3) / 4)), dim3(256), 0, stream, p, block_rows, shares);
  else hipLaunchKernelGGL((gqa_combine_kernel<D, OUT32, 1, 4, 16>), dim3((uint32_t)((rows + 63) / 64)), dim3(256), 0, stream, p, block_rows, shares);
  return hipGetLastError();
}

template <int D, int RT, bool OUT32, bool ALONE = false>
hipError_t narrow(const GqaDecodeParams& p, int shares, hipStream_t stream) {
  constexpr size_t lds = ALONE ? 0 : Narrow<D, RT>::kLds;
  hipLaunchKernelGGL((gqa_decode_kernel<D, RT, OUT32, ALONE>), dim3(ALONE ? shares / 4 : shares), dim3(kThreads), lds, stream, p);
  return hipGetLastError();
}

template <int D, bool OUT32>
hipError_t start(const GqaDecodeParams& p, const GqaShape& shape, int shares, hipStream_t stream) {
  hipError_t e = hipErrorInvalidValue;
  if (shape.wide) e = launch_gqa_wide(p, shape, shares, stream);
  else if (shape.shares == 4) {
    if constexpr (D == 64) e = narrow<D, 1, OUT32, true>(p, shares, stream);
  }
  else if (shape.row_tiles == 1) e = narrow<D, 1, OUT32>(p, shares, stream);
  else if constexpr (D <= 128) {
    if (shape.row_tiles == 2) e = narrow<D, 2, OUT32>(p, shares, stream);
    else if constexpr (D == 64) e = narrow<D, 4, OUT32>(p, shares, stream);
  }
  return e != hipSuccess || p.uncut ? e : join<D, OUT32>(p, shape.block_rows, shares, stream);
}

template <int D, int RT>
hipError_t allow_lds() {
  constexpr int lds = (int)Narrow<D, RT>::kLds;
  hipError_t e = hipFuncSetAttribute((const void*)gqa_decode_kernel<D, RT, false, false>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e == hipSuccess) e = hipFuncSetAttribute((const void*)gqa_decode_kernel<D, RT, true, false>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  return e;
}

}  // namespace

// By the average number of query rows of a request and KV head.  (The lengths are on the device, so the host knows no more.  All that follows was
// measured with as many new tokens for every request; a chunk of a prompt among many single tokens is cut into the few-row blocks of
// their mean, and is not measured.)  us a call, 64 requests of 2000 to 16000 tokens, 4 KV heads; "tiles": this kernel with so many row tiles
// (several blocks where the rows are more):
//   width 64   rows 16  24  32  40  64 128    width 128  rows 16  24  32  40  64 128    width 256  rows 16  24  32  40  64 128
//   1 tile          54  85  79 103 143 300    1 tile          92 149 157 220 274 553    1 tile         181 281 285 411 523 981
//   2 tiles         54  62  58  89  97 191    2 tiles         96 101 108 160 160 305    wide           178 189 183 232 262 462
//   4 tiles         80  90  82  81  87 170    wide           106 111 119 144 152 294
// (Up to 16 rows of width 256 the two are alike at these lengths; short requests end and begin faster with this kernel.)
// Waves that work alone: a block costs them 3 us less, as they need not meet, but they leave more partial rows and have less under way where
// blocks are long.  256 requests, 12 KV heads of width 64, us with them and without: 128 tokens each 14.3 / 19.8, 1 to 2000 (window 1024)
// 29.3 / 36.5, 1024 each 85 / 81, 2048 each 155 / 150; 128 requests of 500 to 8000 tokens, 8 KV heads 82 / 82.  At width 128 they lose from
// 50 to 1000 tokens on (200 requests, 8 KV heads: 44 / 41.5), and so they are for many short blocks of width 64.
// Blocks that cannot have more than a few pages go whole to a share: nothing has to be joined, which saves the second launch (2 to 3 us,
// and 3 us of the host's time).  us cut / uncut, all requests of so many pages (4 query heads to a KV head but for width 64; "wide": 40 rows):
//   requests x heads     1 page      2            3            4            6            8
//   width 128   1 x 8     8.0/6.4    9.5/7.2      9.6/8.0      9.5/8.7      9.6/10.1     9.7/11.6
//              16 x 8     9.0/7.1   12.0/9.6     13.1/11.0    13.3/12.8    13.8/16.4    15.2/19.7
//             256 x 8    23.0/20.5  29.6/27.1    46.2/43.7    58.0/55.4    81.4/78.6   103.9/101.2
//   width 64   16 x 12    8.8/7.0   11.6/9.7     11.7/8.9     13.6/13.7    14.5/17.0    14.3/19.6
//   alone     256 x 12   16.0/13.4  17.3/16.9    18.9/18.9    19.8/24.2    21.6/30.2    23.3/37.9   (lengths up to so many pages)
//   width 256   1 x 2     9.8/8.3   11.3/9.6     11.3/10.9    11.3/12.1    11.3/14.6    11.4/17.1
//   wide        1 x 2    14.9/13.4  16.0/17.3    16.1/21.1    16.0/24.7    16.0/32.2    16.3/39.6
//              64 x 2    18.0/15.9  22.5/19.9    26.2/23.7    29.7/27.5    33.4/34.7    37.3/42.2
GqaShape gqa_shape(int batch, int num_queries, int group, int kv_heads, int head_dim, int64_t pages, int cus) {
  const int64_t rows = (int64_t)((num_queries + batch - 1) / batch) * group;
  if (rows <= 16) {
    const int groups = cus * groups_per_cu(head_dim, 1);
    const bool alone = head_dim == 64 && (int64_t)batch * kv_heads >= 2 * groups && pages <= 16;
    return GqaShape{false, 1, 16, groups, alone ? 4 : 1, pages <= (alone || head_dim == 256 ? 3 : 4)};
  }
  if (head_dim == 256) return GqaShape{true, 1, 64, cus, 1, pages <= 2};
  if (rows <= 32) return GqaShape{false, 2, 32, cus * groups_per_cu(head_dim, 2), 1, pages <= 4};
  if (head_dim == 64) return GqaShape{false, 4, 64, cus * groups_per_cu(head_dim, 4), 1, pages <= 4};
  return GqaShape{true, 2, 64, cus, 1, pages <= 2};
}

hipError_t init_gqa_kernels() {
  hipError_t e = allow_lds<64, 1>();
  if (e == hipSuccess) e = allow_lds<64, 2>();
  if (e == hipSuccess) e = allow_lds<64, 4>();
  if (e == hipSuccess) e = allow_lds<128, 1>();
  if (e == hipSuccess) e = allow_lds<128, 2>();
  if (e == hipSuccess) e = allow_lds<256, 1>();
  if (e == hipSuccess) e = init_gqa_wide_kernels();
  return e;
}

hipError_t launch_gqa_decode(const GqaDecodeParams& p, const GqaShape& shape, int shares, hipStream_t stream) {
  auto with = [&](auto d) {
    return p.out_fp32 ? start<decltype(d)::value, true>(p, shape, shares, stream) : start<decltype(d)::value, false>(p, shape, shares, stream);
  };
  if (p.head_dim == 64) return with(std::integral_constant<int, 64>{});
  if (p.head_dim == 128) return with(std::integral_constant<int, 128>{});
  return with(std::integral_constant<int, 256>{});
}

}  // namespace omniattn
