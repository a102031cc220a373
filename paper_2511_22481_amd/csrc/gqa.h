// Launch interface between the C ABI of the grouped-query part (api_gqa.cpp) and its gfx950 kernels: tables made on
// the device, the 8-bit cache with a scale for each block of tokens and KV head, and attention over it.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "plan.h"

namespace omniattn {

// Keeps the text of a HIP error for omniattn_last_hip_error and returns OMNIATTN_EHIP (api.cpp).
int hip_fail(hipError_t e, const char* what);

// Compute units of the current device; also sets its kernels' attributes, the first time (api_gqa.cpp).
int device_cus(int* cus);

struct TableParams {
  const int32_t* seq_lens;
  const int32_t* new_lens;
  const int32_t* free_pages;
  const int32_t* free_count;
  int32_t* page_table;
  int64_t stride;  // elements from one row of page_table to the next
  int32_t* seq_lens_out;
  int32_t* free_count_out;
  int32_t* q_start;
  int32_t* slot_map;
  int batch, max_pages, max_tokens;
};
hipError_t launch_table_extend(const TableParams& p, hipStream_t stream);

struct ReleaseParams {
  const int32_t* done;
  int32_t* seq_lens;
  const int32_t* page_table;
  int64_t stride;
  int32_t* free_pages;
  int32_t* free_count;
  int batch, max_pages;
  int64_t num_pages;  // entries of free_pages
};
hipError_t launch_table_release(const ReleaseParams& p, hipStream_t stream);

struct TruncateParams {
  const int32_t* seq_lens;
  const int32_t* dropped;
  const int32_t* page_table;
  int64_t stride;
  int32_t* free_pages;
  const int32_t* free_count;
  int32_t* seq_lens_out;
  int32_t* free_count_out;
  int batch, max_pages;
  int64_t num_pages;  // entries of free_pages
};
hipError_t launch_table_truncate(const TruncateParams& p, hipStream_t stream);

struct TreeMasksParams {
  const int32_t* parents;
  const int32_t* seq_lens;
  const int32_t* q_start;  // [batch + 1], or null: node b belongs to request b
  uint64_t* masks;
  int32_t* positions;      // or null
  int batch, num_tokens;
};
hipError_t launch_tree_masks(const TreeMasksParams& p, hipStream_t stream);

struct GqaKeepParams {
  const int32_t* path;
  const int32_t* seq_lens;
  const int32_t* q_start;   // [batch + 1], or null
  const int32_t* page_table;
  int64_t table_stride;
  uint8_t* cache[2];        // e4m3 [layers, num_pages, kv_heads, 128, head_dim]
  float* scales[2];         // [layers, num_pages, kv_heads, 128 / scale_tokens]
  int64_t num_pages;
  int batch, num_tokens, layers, kv_heads, head_dim, scale_tokens, max_pages;
  int run;  // layers to a wave (the launch sets it)
};
// cus: the device's compute units.
hipError_t launch_gqa_keep(GqaKeepParams p, int cus, hipStream_t stream);

struct GqaAppendParams {
  const uint16_t* rows[2];  // K and V, bf16 [tokens, kv_heads, head_dim]
  int64_t stride[2];        // elements from one token to the next
  const int32_t* slot_map;
  uint8_t* cache[2];        // e4m3 [num_pages, kv_heads, 128, head_dim]
  float* scales[2];         // [num_pages, kv_heads, 128 / scale_tokens]
  int num_tokens, kv_heads, head_dim, scale_tokens;
  uint32_t num_slots;       // num_pages * 128: other slots take nothing
};
hipError_t launch_gqa_append(const GqaAppendParams& p, hipStream_t stream);

struct GqaDecodeParams {
  const uint16_t* q;
  int64_t q_stride;         // elements from one query token to the next
  const uint8_t* k_cache;
  const uint8_t* v_cache;
  const float* k_scales;
  const float* v_scales;
  const int32_t* page_table;
  int64_t table_stride;
  const int32_t* seq_lens;
  const int32_t* q_start;   // [batch + 1], or null: query token b belongs to request b
  void* out;
  float* lse;
  int2* rows;               // per output row: first partial slot; number of partials * 64 (blocks of more rows: 128) + row inside its block (0 partials: done)
  float4* part_ml;          // [slots, block rows]: a partial row's reference (log2) and sum of weights, and its output's reference
  float* part_o;            // [slots, block rows, head_dim]: weighted sums, not yet divided
  int batch, num_queries, q_heads, kv_heads, group, head_dim;
  int max_pages, S, W, scale_shift;  // scale_shift: log2 of the tokens that share a scale
  int out_fp32;
  int few_units;            // a call's units of work (pages and blocks) are counted in 32 bits
  int uncut;                // blocks go whole to the share that has their first unit: no partial rows
  float scale_log2;         // softmax_scale * log2(e)
  const uint64_t* masks;    // [num_queries]: the nodes that each query sees; null: the queries are a request's last tokens, each seeing those before it
};
// How a call is computed: by which kernel (gqa_decode_kernel.hip, gqa_wide_kernel.hip or gqa_tree_kernel.hip), tiles of 16 query rows per wave, rows of a
// block, work groups at most, and shares of the work to each.
enum GqaKernel { kGqaNarrow, kGqaWide, kGqaTree };
struct GqaShape {
  GqaKernel kernel;
  int row_tiles, block_rows, groups, shares;
  bool uncut;               // see GqaDecodeParams
};
// pages: those that a query's kept tokens can lie in.
GqaShape gqa_shape(int batch, int num_queries, int group, int kv_heads, int head_dim, int64_t pages, int cus, bool tree);
hipError_t init_gqa_kernels();
hipError_t init_gqa_wide_kernels();
hipError_t init_gqa_tree_kernels();
// The kernel of the shape, and the one that joins partial rows.
hipError_t launch_gqa_decode(const GqaDecodeParams& p, const GqaShape& shape, int shares, hipStream_t stream);
hipError_t launch_gqa_wide(const GqaDecodeParams& p, const GqaShape& shape, int shares, hipStream_t stream);
hipError_t launch_gqa_tree(const GqaDecodeParams& p, int shares, hipStream_t stream);

}  // namespace omniattn
