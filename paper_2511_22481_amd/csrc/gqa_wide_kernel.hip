// Attention of grouped-query layers over the paged 8-bit cache for requests with many query rows: more than 32 at width 128, more than 16
// at width 256 (several new tokens, or many query heads to a KV head).  The same work as gqa_decode_kernel.hip, dealt out the same way;
// what differs is how a tile is shared.
//
// One work group of eight waves per compute unit.  A tile (32 TG tokens) is brought to LDS once by direct loads and read by RG = 8 / TG
// waves for each 32 of its tokens, each with other query rows, so a block has RG * 16 * RT = 64 rows: the codes come from memory once for
// all of them.  The tiles pass through a ring of stages, kStages - 1 of them requested ahead, over the ends of blocks too; one barrier per
// tile.
//
// What bounds it: the vector unit.  A tile of 32 tokens and 16 rows of width 256 costs a wave 192 conversions and permutations of
// codes and 130 instructions of softmax beside 48 matrix instructions, and the two waves of a SIMD take 4600 cycles for it where
// the codes would arrive in 2600.  64 requests of 2000 to 16000 tokens, 4 KV heads: width 128 152 us at 64 rows and 144 at 40 (3.0
// TB/s, 381 TFLOP/s at 64), width 256 183 at 32 rows, 232 at 40, 262 at 64.  Chunks of 512 tokens of 64 requests' prompts, 32/8 heads of 128:
// 642 us, 266 TFLOP/s (the codes are converted again for every 64 rows of a chunk).  (More row tiles to a wave would share the conversions, but
// at width 256 two leave no registers, and at width 128 four leave one wave to a SIMD.)
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gqa_common.h"

namespace omniattn {
namespace {

constexpr int kThreads = 512, kWaves = 8, kStart = 2;

template <int D, int RT>
struct Wide {
  static constexpr int kTokenGroups = D == 256 ? 2 : 4;       // TG
  static constexpr int kRowGroups = kWaves / kTokenGroups;    // RG
  static constexpr int kRows = kRowGroups * 16 * RT;
  static constexpr int kTokens = kWaveTokens * kTokenGroups;  // of a tile
  static constexpr int kTilesPerPage = kPage / kTokens;
  static constexpr int kHalf = kTokens * D;                   // bytes of a tile's K codes; V's follow
  static constexpr int kStages = 3;
  static constexpr int kLoads = 2 * kHalf / 1024 / kWaves;    // direct loads of a wave and tile (1 KB each), and one of the scales
  static constexpr int kParts = 4;                            // the output's columns meet 1 / kParts at a time
  static constexpr int kScaleBytes = 256;                     // of a wave and stage: K's and V's scale in turn, 32 times
  static constexpr size_t kRing = (size_t)kStages * (2 * kHalf + kWaves * kScaleBytes);
  static constexpr size_t kOBytes = (size_t)kTokenGroups * kRows * (D / kParts + 4) * 4;
  static constexpr size_t kLds = kRing + kOBytes + 2 * kTokenGroups * kRows * 16;
  static_assert(kLds + 10240 <= 160 * 1024, "LDS of a compute unit");
  static_assert((D == 128 || D == 256) && kLoads == 4);
};

// Where a row's 16-byte chunks lie in LDS.  Rows stand in groups of 16 (tokens 16 i ..): row r at place(r), its chunk c at c ^ twist(r), so
// that neither the 16 rows of a K operand nor the rows of a V operand meet in the same banks.  (A row is 8 or 16 chunks, 64 banks are
// 16 chunks.)
template <int D>
__device__ __forceinline__ int place(int r) {
  if constexpr (D == 128) return r ^ ((r >> 2) & 1);
  else return r;
}
template <int D>
__device__ __forceinline__ int twist(int r) {
  const int at = place<D>(r);
  if constexpr (D == 128) return (at >> 1) & 7;
  else return at & 15;
}

// The same value from memory for every lane, through the scalar cache.
__device__ __forceinline__ int scalar_load(const int32_t* at) {
  return *(const __attribute__((address_space(4))) int32_t*)(uintptr_t)uniform64((uint64_t)(uintptr_t)at);
}

// Sixteen bytes per lane at the LDS base set before, from a scalar address that went through settle_address.  (As load_lds16_at, but
// the rows may stay in L2: other blocks of query rows read them too.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <int IMM>
__device__ __forceinline__ void load_lds16_here(uint64_t base, uint32_t off) {
  asm volatile("global_load_lds_dwordx4 %0, %1 offset:%2" : : "v"(off), "s"(base), "n"(IMM) : "m0", "memory");
}
#pragma clang diagnostic pop

// Four bytes per lane from an address of its own to LDS (see load_lds16 in decode_common.h).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_lds4_each(uint32_t lds, const void* at) {
  const uint32_t m = __builtin_amdgcn_readfirstlane(lds);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dword %1, off" : : "s"(m), "v"((uint64_t)(uintptr_t)at) : "m0", "memory");
}
#pragma clang diagnostic pop

// Waits until the loads of the oldest tile are done, with one tile requested after it or none, and for all waves to get here.  (Other
// loads and stores in between only make it wait for more than it has to.)
template <int LOADS>
__device__ __forceinline__ void wait_tile(bool one_behind) {
  if (one_behind) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(LOADS) : "memory");
  else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory");
}

template <int D, int RT, bool OUT32>
__global__ __launch_bounds__(kThreads, 2) void gqa_wide_kernel(GqaDecodeParams p) {
  using C = Wide<D, RT>;
  constexpr int R = C::kRows, TG = C::kTokenGroups, kWords = D / 64, kCols = D / 16, kStages = C::kStages;
  extern __shared__ __align__(1024) uint8_t ring[];   // [stages][K codes, V codes], [stages][waves][scales], output, references
  uint8_t* const scale_ring = ring + kStages * 2 * C::kHalf;
  float* const o_lds = (float*)(ring + C::kRing);
  float4* const ml_lds = (float4*)(ring + C::kRing + C::kOBytes);
  __shared__ typename Dealer<R, kThreads, kStart>::Lds dealt;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int n16 = lane & 15, g = lane >> 4;
  const int tg = wave % TG, row0 = wave / TG * 16 * RT;
  Dealer<R, kThreads, kStart> dealer(p, dealt);
  Piece now;
  if (!dealer.begin(now)) return;
  const uint32_t ring_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)ring;

  const int blocks_per_page = kPage >> p.scale_shift;
  // Direct loads: the wave brings kLoads KB, one after the other, of K (waves 0 to 3) or V.  Lane l's 16 bytes of a KB are those of
  // chunk l % chunks ^ twist of the row that belongs to place l / chunks: whole rows of it, in another order.
  constexpr int kChunks = D / 16, kRowsPerKb = 64 / kChunks;
  // (The KB's own offset is the instruction's, on both sides.)
  uint32_t from[C::kLoads];
#pragma unroll
  for (int i = 0; i < C::kLoads; ++i) {
    const int at = (wave % 4 * C::kLoads + i) * kRowsPerKb + lane / kChunks;  // place among the tile's rows
    const int r = at % 16;
    from[i] = (at / 16 * 16 + place<D>(r)) * D + ((lane % kChunks) ^ twist<D>(place<D>(r))) * 16 - i * 1024;  // (place is its own inverse)
  }
  const uint8_t* const codes = wave < 4 ? p.k_cache : p.v_cache;

  // The tile that is asked for next: a page of a block, or a half of one.  The block's description is the wave's note 0.
  int ahead_tile = now.tile_lo, ahead_hi = now.tile_hi, ahead_half = 0, ahead_stage = 0, issued = 0, ahead_h = now.h, ahead_page = 0;
  TileLayout ahead_pages = now.bk.pages;
  const int32_t* ahead_table = p.page_table + now.b * p.table_stride;
  bool ahead_any = true;
  dealer.keep(0, now);
  auto skip_empty = [&] {
    if (ahead_tile < ahead_hi) return;
    Piece w = dealer.kept(0);
    do ahead_any = dealer.follow(w);
    while (ahead_any && w.tile_lo >= w.tile_hi);
    if (!ahead_any) return;
    dealer.keep(0, w);
    ahead_tile = w.tile_lo;
    ahead_hi = w.tile_hi;
    ahead_h = w.h;
    ahead_pages = w.bk.pages;
    ahead_table = p.page_table + w.b * p.table_stride;
  };
  skip_empty();
  const float* const my_scales = lane & 1 ? p.v_scales : p.k_scales;
  auto ask_page = [&] {
    if (ahead_any && ahead_half == 0) ahead_page = scalar_load(ahead_table + ahead_pages.logical(ahead_tile));
  };
  auto issue = [&] {
    if (!ahead_any) return;
    const size_t ph = (size_t)ahead_page * p.kv_heads + ahead_h;
    uint64_t base = (uint64_t)(uintptr_t)(codes + (ph * kPage + ahead_half * C::kTokens) * D), same = base;
    set_lds_base(ring_at + ahead_stage * 2 * C::kHalf + wave * C::kLoads * 1024);
    settle_address(base, same);
    load_lds16_here<0>(base, from[0]);
    load_lds16_here<1024>(base, from[1]);
    load_lds16_here<2 * 1024>(base, from[2]);
    load_lds16_here<3 * 1024>(base, from[3]);
    load_lds4_each(ring_at + kStages * 2 * C::kHalf + (ahead_stage * kWaves + wave) * C::kScaleBytes,
                   my_scales + ph * blocks_per_page + ((ahead_half * C::kTokens + tg * kWaveTokens) >> p.scale_shift));
    ++issued;
    if (++ahead_stage == kStages) ahead_stage = 0;
    if (++ahead_half == C::kTilesPerPage) {
      ahead_half = 0;
      ++ahead_tile;
      skip_empty();
    }
  };
  for (int i = 0; i < kStages - 1; ++i) {
    ask_page();
    issue();
  }

  bf16x8 q[RT][2 * kWords];
  int reach[RT];
  auto load_q = [&](const Piece& w) {
    const int rows = dealer.rows_of(w);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const int row = row0 + rt * 16 + n16;
      const uint32_t t = (uint32_t)(w.rb * R + row) / (uint32_t)p.group, gi = (uint32_t)(w.rb * R + row) - t * p.group;
      const bool valid = row < rows;
      reach[rt] = valid ? w.reach((int)t) : 0;
      const uint16_t* src = p.q + (int64_t)(w.rq.begin + (int)t) * p.q_stride + (size_t)(w.h * p.group + (int)gi) * D + g * 16;
#pragma unroll
      for (int i = 0; i < 2 * kWords; ++i) q[rt][i] = valid ? *(const bf16x8*)(src + i / 2 * 64 + i % 2 * 8) : bf16x8{};
    }
  };
  load_q(now);

  // Operands in LDS, from the start of a stage on: rows of the wave's 32 tokens
  const int k_row = (tg * kWaveTokens + place<D>(n16)) * D, k_twist = twist<D>(n16);
  int v_at[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int r = 4 * g + j;
    v_at[j] = C::kHalf + (tg * kWaveTokens + place<D>(r)) * D + ((n16 * kCols / 16) ^ twist<D>(r)) * 16 + n16 * kCols % 16;
  }

  int parity = 0, first_partial = 0, stage = 0, used = 0;
  dealer.keep(1, now);  // (notes 1 and 2: the block that is computed, and the one behind it)
  int tile = now.tile_lo;
  bool mine = row0 < dealer.rows_of(now);  // (a short block: waves without rows only bring their part of the tiles)
  Span span(now);
  while (true) {
    // The query is waited for here, and asked for behind the loop.  If its loads could be under way at its use in the loop, the wait
    // would stand there in every pass, and as the compiler does not count the direct loads, it would be for all tiles.
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int i = 0; i < 2 * kWords; ++i) asm volatile("" : "+v"(q[rt][i]));
    Rows<D, RT> a;
    a.clear();
    for (; tile < span.tile_hi; ++tile) {
#pragma unroll 1
      for (int half = 0; half < C::kTilesPerPage; ++half) {
        ask_page();  // (back behind the wait, which is for scalar loads too)
        wait_tile<C::kLoads + 1>(issued - used > 1);
        // (into the stage that every wave has left behind at the barrier; half of the waves later, so that one of a SIMD's two is
        // computing while the other one asks)
        if (wave < 4) issue();
        ++used;
        const uint8_t* const from_stage = ring + stage * 2 * C::kHalf;
        const float2 scale = *(const float2*)(scale_ring + (stage * kWaves + wave) * C::kScaleBytes);
        if (++stage == kStages) stage = 0;
        const int pos0 = span.pages.logical(tile) * kPage + half * C::kTokens + tg * kWaveTokens;
        const Kept kept = kept_of(p, span, pos0);
        f32x4 s[RT][2];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) s[rt][0] = s[rt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
        const bool work = mine && kept.some;
        if (work) {
#pragma unroll
          for (int c = 0; c < kWords; ++c) {
            u32x4 k[2];
#pragma unroll
            for (int h2 = 0; h2 < 2; ++h2) k[h2] = *(const u32x4*)(from_stage + k_row + h2 * 16 * D + ((4 * c + g) ^ k_twist) * 16);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
              for (int h2 = 0; h2 < 2; ++h2) {
                const bf16x8 x = k_operand(k[h2][2 * u], k[h2][2 * u + 1]);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) s[rt][h2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, q[rt][2 * c + u], s[rt][h2], 0, 0, 0);
              }
          }
        }
        if (wave >= 4) issue();
        if (work) {
          f16x8 high[RT], low[RT];
          weigh<D, RT>(p, a, s, reach, kept.full, pos0, g, p.scale_log2 * scale.x, scale.y, high, low);
          typename VWord<kWords>::type v[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = *(const typename VWord<kWords>::type*)(from_stage + v_at[j % 4] + j / 4 * 16 * D);
          if (!kept.full) sanitize<D, RT>(p, a, v, span, pos0, g);
          add_values<D, RT>(a, v, high, low);
        }
      }
    }
    // (behind the loop: see above)
    const Piece done = dealer.kept(1);
    Piece next = done;
    const bool more_blocks = dealer.follow(next);
    if (more_blocks) {
      load_q(next);
      dealer.keep(2, next);
    }
    finish<D, RT, R, TG, C::kParts, kThreads, OUT32>(dealer, done, a, o_lds, ml_lds + parity * TG * R, tg, row0, 2 * blockIdx.x + first_partial);
    parity ^= 1;
    first_partial = 1;
    if (!more_blocks) break;
    next = dealer.kept(2);
    dealer.keep(1, next);
    tile = next.tile_lo;
    mine = row0 < dealer.rows_of(next);
    span = Span(next);
  }
}

template <int D, int RT, bool OUT32>
hipError_t start(const GqaDecodeParams& p, int shares, hipStream_t stream) {
  constexpr size_t lds = Wide<D, RT>::kLds;
  hipLaunchKernelGGL((gqa_wide_kernel<D, RT, OUT32>), dim3(shares), dim3(kThreads), lds, stream, p);
  return hipGetLastError();
}
template <int D, int RT>
hipError_t allow_lds() {
  constexpr int lds = (int)Wide<D, RT>::kLds;
  hipError_t e = hipFuncSetAttribute((const void*)gqa_wide_kernel<D, RT, false>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e == hipSuccess) e = hipFuncSetAttribute((const void*)gqa_wide_kernel<D, RT, true>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  return e;
}

}  // namespace

hipError_t init_gqa_wide_kernels() {
  hipError_t e = allow_lds<128, 2>();
  if (e == hipSuccess) e = allow_lds<256, 1>();
  return e;
}

hipError_t launch_gqa_wide(const GqaDecodeParams& p, const GqaShape& shape, int shares, hipStream_t stream) {
  if (p.head_dim == 128 && shape.row_tiles == 2) return p.out_fp32 ? start<128, 2, true>(p, shares, stream) : start<128, 2, false>(p, shares, stream);
  if (p.head_dim == 256 && shape.row_tiles == 1) return p.out_fp32 ? start<256, 1, true>(p, shares, stream) : start<256, 1, false>(p, shares, stream);
  return hipErrorInvalidValue;
}

}  // namespace omniattn
