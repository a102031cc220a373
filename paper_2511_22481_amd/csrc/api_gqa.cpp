// C ABI of the grouped-query part (see include/omniattn.h): tables on the device, the 8-bit cache, attention over it.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <mutex>

#include "gqa.h"

using namespace omniattn;

namespace {

#define OA_HIP(call)                                  \
  do {                                                \
    hipError_t e_ = (call);                           \
    if (e_ != hipSuccess) return hip_fail(e_, #call); \
  } while (0)

constexpr int kMaxDevices = 64;
constexpr int64_t kMaxPages = INT32_MAX / kPage;  // slots are int32
std::mutex g_mutex;
int g_cus[kMaxDevices] = {};  // compute units; 0: kernel attributes not set yet

}  // namespace

int omniattn::device_cus(int* cus) {
  int dev = 0;
  OA_HIP(hipGetDevice(&dev));
  if (dev < 0 || dev >= kMaxDevices) return OMNIATTN_EINVAL;
  std::lock_guard<std::mutex> lock(g_mutex);
  if (g_cus[dev] == 0) {
    OA_HIP(init_gqa_kernels());
    int n = 0;
    OA_HIP(hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev));
    g_cus[dev] = n > 0 ? n : 256;
  }
  *cus = g_cus[dev];
  return OMNIATTN_OK;
}

namespace {

bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// Whether two arrays of n and m int32 share memory without beginning at the same place.
bool half_overlap(const int32_t* a, const int32_t* b, size_t n) { return a != b && a < b + n && b < a + n; }

int check_table(const omniattn_table_t* t) {
  if (!t) return OMNIATTN_EINVAL;
  if (t->batch < 1 || t->max_pages_per_seq < 1 || t->max_tokens < 0 || t->num_pages < 1) return OMNIATTN_EINVAL;
  if (t->page_size != kPage) return OMNIATTN_EUNSUPPORTED;
  if (t->page_table_stride < t->max_pages_per_seq) return OMNIATTN_EINVAL;
  if (t->num_pages > kMaxPages || t->max_pages_per_seq > kMaxPages) return OMNIATTN_EUNSUPPORTED;
  return OMNIATTN_OK;
}

int check_gqa(const omniattn_gqa_t* g) {
  if (!g) return OMNIATTN_EINVAL;
  if (g->batch < 1 || g->num_q_heads < 1 || g->num_kv_heads < 1 || g->num_q_heads % g->num_kv_heads != 0) return OMNIATTN_EINVAL;
  if (g->max_pages_per_seq < 1 || g->num_pages < 1 || g->num_queries < 0) return OMNIATTN_EINVAL;
  if (g->sink < 0 || g->window < 0) return OMNIATTN_EINVAL;
  if (g->page_size != kPage) return OMNIATTN_EUNSUPPORTED;
  if (g->head_dim != 64 && g->head_dim != 128 && g->head_dim != 256) return OMNIATTN_EUNSUPPORTED;
  if (g->scale_tokens != 32 && g->scale_tokens != 64 && g->scale_tokens != 128) return OMNIATTN_EUNSUPPORTED;
  if (g->out_dtype != OMNIATTN_BF16 && g->out_dtype != OMNIATTN_FP32) return OMNIATTN_EUNSUPPORTED;
  if (g->num_pages > kMaxPages || g->max_pages_per_seq > kMaxPages) return OMNIATTN_EUNSUPPORTED;
  // (rows of the call and blocks of a request are counted in 32 bits)
  if ((int64_t)g->num_queries * g->num_q_heads > INT32_MAX / 2) return OMNIATTN_EUNSUPPORTED;
  return OMNIATTN_OK;
}

GqaShape shape_of(const omniattn_gqa_t* g, int cus, bool tree) {
  const int64_t pages = std::min<int64_t>(g->max_pages_per_seq, ((int64_t)g->sink + kPage - 1) / kPage + ((int64_t)g->window + kPage - 1) / kPage + 1);
  return gqa_shape(g->batch, g->num_queries, g->num_q_heads / g->num_kv_heads, g->num_kv_heads, g->head_dim, pages, cus, tree);
}

struct Workspace {
  size_t rows, ml, o, bytes;  // offsets, and the whole
};
size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }
Workspace workspace_of(const omniattn_gqa_t* g, const GqaShape& shape) {
  const size_t slots = (size_t)2 * shape.groups * shape.shares * shape.block_rows;
  Workspace w;
  w.rows = 0;
  w.ml = align256((size_t)g->num_queries * g->num_q_heads * sizeof(int2));
  w.o = w.ml + align256(slots * sizeof(float4));
  w.bytes = w.o + slots * g->head_dim * sizeof(float);
  return w;
}

// Enough for fewer queries too, and for any kept set and table width: the calls of a server share one.  (The number of queries decides
// by its rows to a request and KV head, up to 16, up to 32 or more; those that keep few pages have the most shares, and trees over many the
// largest blocks.)
size_t most_workspace(const omniattn_gqa_t* gqa, bool trees) {
  int cus = 0;
  if (check_gqa(gqa) != OMNIATTN_OK || device_cus(&cus) != OMNIATTN_OK) return 0;
  size_t bytes = 0;
  omniattn_gqa_t g = *gqa;
  g.sink = g.window = 0;
  const int64_t group = gqa->num_q_heads / gqa->num_kv_heads;
  for (int rows : {16, 32, INT32_MAX}) {
    g.num_queries = (int32_t)std::min<int64_t>(gqa->num_queries, std::max<int64_t>(rows / group, 1) * gqa->batch);
    bytes = std::max(bytes, workspace_of(gqa, shape_of(&g, cus, false)).bytes);
    if (trees) bytes = std::max(bytes, workspace_of(gqa, gqa_shape(g.batch, g.num_queries, (int)group, g.num_kv_heads, g.head_dim, kMaxPages, cus, true)).bytes);
  }
  return bytes;
}

// omniattn_gqa_decode, and omniattn_gqa_tree (tree).
int attend(const omniattn_gqa_t* gqa, const void* q, int64_t q_stride, const void* k_cache, const void* v_cache, const float* k_scales, const float* v_scales,
           const int32_t* page_table, const int32_t* seq_lens, const int32_t* q_start, bool tree, const uint64_t* masks, void* out, float* lse, void* workspace,
           size_t workspace_bytes, void* hip_stream) {
  int rc = check_gqa(gqa);
  if (rc != OMNIATTN_OK) return rc;
  if (gqa->page_table_stride < gqa->max_pages_per_seq) return OMNIATTN_EINVAL;
  if (!std::isfinite(gqa->softmax_scale)) return OMNIATTN_EINVAL;
  if (!q_start && gqa->num_queries != gqa->batch) return OMNIATTN_EINVAL;
  if (gqa->num_queries == 0) return OMNIATTN_OK;
  if (!q || !k_cache || !v_cache || !k_scales || !v_scales || !page_table || !seq_lens || !out || !lse) return OMNIATTN_EINVAL;
  if (tree && (!masks || !aligned(masks, 8))) return OMNIATTN_EINVAL;
  if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(out, 16)) return OMNIATTN_EINVAL;
  if (q_stride % 8 != 0 || q_stride < (int64_t)gqa->num_q_heads * gqa->head_dim) return OMNIATTN_EINVAL;
  int cus = 0;
  rc = device_cus(&cus);
  if (rc != OMNIATTN_OK) return rc;
  GqaDecodeParams p;
  p.group = gqa->num_q_heads / gqa->num_kv_heads;
  const GqaShape shape = shape_of(gqa, cus, tree);
  const Workspace w = workspace_of(gqa, shape);
  if (!workspace || workspace_bytes < w.bytes || !aligned(workspace, 256)) return OMNIATTN_EWORKSPACE;
  p.q = (const uint16_t*)q;
  p.q_stride = q_stride;
  p.k_cache = (const uint8_t*)k_cache;
  p.v_cache = (const uint8_t*)v_cache;
  p.k_scales = k_scales;
  p.v_scales = v_scales;
  p.page_table = page_table;
  p.table_stride = gqa->page_table_stride;
  p.seq_lens = seq_lens;
  p.q_start = q_start;
  p.out = out;
  p.lse = lse;
  p.rows = (int2*)((char*)workspace + w.rows);
  p.part_ml = (float4*)((char*)workspace + w.ml);
  p.part_o = (float*)((char*)workspace + w.o);
  p.batch = gqa->batch;
  p.num_queries = gqa->num_queries;
  p.q_heads = gqa->num_q_heads;
  p.kv_heads = gqa->num_kv_heads;
  p.head_dim = gqa->head_dim;
  p.max_pages = gqa->max_pages_per_seq;
  // (no request is longer than its table, 2^31 - 128 tokens at most: larger numbers mean the same, and W + 63 stays in 32 bits)
  p.S = std::min(gqa->sink, gqa->max_pages_per_seq * kPage);
  p.W = std::min(gqa->window, gqa->max_pages_per_seq * kPage);
  p.scale_shift = gqa->scale_tokens == 32 ? 5 : gqa->scale_tokens == 64 ? 6 : 7;
  p.out_fp32 = gqa->out_dtype == OMNIATTN_FP32;
  p.uncut = shape.uncut;
  p.scale_log2 = gqa->softmax_scale * 1.4426950408889634f;
  p.masks = masks;
  // Not more shares than there can be units of work (each block counts up to 2 beside its pages).
  const int64_t blocks = ((int64_t)p.num_queries * p.group + shape.block_rows - 1) / shape.block_rows + p.batch;
  const int64_t pages = std::min<int64_t>(p.max_pages, ((int64_t)p.S + kPage - 1) / kPage + ((int64_t)p.W + (tree ? p.num_queries + OMNIATTN_TREE_NODES : shape.block_rows) + kPage - 1) / kPage + 1);
  const int64_t units = blocks * p.kv_heads * (shape.shares > 1 || shape.kernel == kGqaTree ? 4 * pages + 4 : pages + 2);
  p.few_units = units <= INT32_MAX;
  const int groups = (int)std::min<int64_t>(shape.groups, (units + shape.shares - 1) / shape.shares);
  OA_HIP(launch_gqa_decode(p, shape, groups * shape.shares, (hipStream_t)hip_stream));
  return OMNIATTN_OK;
}

}  // namespace

extern "C" {

int omniattn_table_extend(const omniattn_table_t* table, const int32_t* seq_lens, const int32_t* new_lens, const int32_t* free_pages,
                          const int32_t* free_count, int32_t* page_table, int32_t* seq_lens_out, int32_t* free_count_out, int32_t* q_start,
                          int32_t* slot_map, void* hip_stream) {
  const int rc = check_table(table);
  if (rc != OMNIATTN_OK) return rc;
  if (!seq_lens || !new_lens || !free_pages || !free_count || !page_table || !seq_lens_out || !free_count_out || !q_start) return OMNIATTN_EINVAL;
  if (!slot_map && table->max_tokens > 0) return OMNIATTN_EINVAL;
  if (half_overlap(seq_lens, seq_lens_out, table->batch)) return OMNIATTN_EINVAL;
  TableParams p;
  p.seq_lens = seq_lens;
  p.new_lens = new_lens;
  p.free_pages = free_pages;
  p.free_count = free_count;
  p.page_table = page_table;
  p.stride = table->page_table_stride;
  p.seq_lens_out = seq_lens_out;
  p.free_count_out = free_count_out;
  p.q_start = q_start;
  p.slot_map = slot_map;
  p.batch = table->batch;
  p.max_pages = table->max_pages_per_seq;
  p.max_tokens = table->max_tokens;
  OA_HIP(launch_table_extend(p, (hipStream_t)hip_stream));
  return OMNIATTN_OK;
}

int omniattn_table_release(const omniattn_table_t* table, const int32_t* done, int32_t* seq_lens, const int32_t* page_table, int32_t* free_pages,
                           int32_t* free_count, void* hip_stream) {
  const int rc = check_table(table);
  if (rc != OMNIATTN_OK) return rc;
  if (!done || !seq_lens || !page_table || !free_pages || !free_count) return OMNIATTN_EINVAL;
  ReleaseParams p;
  p.done = done;
  p.seq_lens = seq_lens;
  p.page_table = page_table;
  p.stride = table->page_table_stride;
  p.free_pages = free_pages;
  p.free_count = free_count;
  p.batch = table->batch;
  p.max_pages = table->max_pages_per_seq;
  p.num_pages = table->num_pages;
  OA_HIP(launch_table_release(p, (hipStream_t)hip_stream));
  return OMNIATTN_OK;
}

int omniattn_table_truncate(const omniattn_table_t* table, const int32_t* seq_lens, const int32_t* dropped, const int32_t* page_table, int32_t* free_pages,
                            const int32_t* free_count, int32_t* seq_lens_out, int32_t* free_count_out, void* hip_stream) {
  const int rc = check_table(table);
  if (rc != OMNIATTN_OK) return rc;
  if (!seq_lens || !dropped || !page_table || !free_pages || !free_count || !seq_lens_out || !free_count_out) return OMNIATTN_EINVAL;
  if (half_overlap(seq_lens, seq_lens_out, table->batch)) return OMNIATTN_EINVAL;
  TruncateParams p;
  p.seq_lens = seq_lens;
  p.dropped = dropped;
  p.page_table = page_table;
  p.stride = table->page_table_stride;
  p.free_pages = free_pages;
  p.free_count = free_count;
  p.seq_lens_out = seq_lens_out;
  p.free_count_out = free_count_out;
  p.batch = table->batch;
  p.max_pages = table->max_pages_per_seq;
  p.num_pages = table->num_pages;
  OA_HIP(launch_table_truncate(p, (hipStream_t)hip_stream));
  return OMNIATTN_OK;
}

int omniattn_tree_masks(int32_t batch, int32_t num_tokens, const int32_t* parents, const int32_t* seq_lens, const int32_t* q_start, uint64_t* masks,
                        int32_t* positions, void* hip_stream) {
  if (batch < 1 || num_tokens < 0 || (!q_start && num_tokens != batch)) return OMNIATTN_EINVAL;
  if (num_tokens == 0) return OMNIATTN_OK;
  if (batch >= INT32_MAX >> 5) return OMNIATTN_EUNSUPPORTED;  // (a launch's threads are counted in 32 bits, as below)
  if (!parents || !seq_lens || !masks || !aligned(masks, 8)) return OMNIATTN_EINVAL;
  OA_HIP(launch_tree_masks(TreeMasksParams{parents, seq_lens, q_start, masks, positions, batch, num_tokens}, (hipStream_t)hip_stream));
  return OMNIATTN_OK;
}

int omniattn_gqa_keep(const omniattn_gqa_t* gqa, int32_t num_layers, const int32_t* path, const int32_t* seq_lens, const int32_t* q_start,
                      const int32_t* page_table, void* k_cache, void* v_cache, float* k_scales, float* v_scales, void* hip_stream) {
  const int rc = check_gqa(gqa);
  if (rc != OMNIATTN_OK) return rc;
  if (num_layers < 0 || gqa->page_table_stride < gqa->max_pages_per_seq || (!q_start && gqa->num_queries != gqa->batch)) return OMNIATTN_EINVAL;
  if (num_layers == 0 || gqa->num_queries == 0) return OMNIATTN_OK;
  if (!path || !seq_lens || !page_table || !k_cache || !v_cache || !k_scales || !v_scales) return OMNIATTN_EINVAL;
  if (!aligned(k_cache, 16) || !aligned(v_cache, 16)) return OMNIATTN_EINVAL;
  if ((int64_t)num_layers * gqa->batch >= (INT32_MAX >> 5) / gqa->num_kv_heads) return OMNIATTN_EUNSUPPORTED;
  int cus = 0;
  const int found = device_cus(&cus);
  if (found != OMNIATTN_OK) return found;
  GqaKeepParams p;
  p.path = path;
  p.seq_lens = seq_lens;
  p.q_start = q_start;
  p.page_table = page_table;
  p.table_stride = gqa->page_table_stride;
  p.cache[0] = (uint8_t*)k_cache;
  p.cache[1] = (uint8_t*)v_cache;
  p.scales[0] = k_scales;
  p.scales[1] = v_scales;
  p.num_pages = gqa->num_pages;
  p.batch = gqa->batch;
  p.num_tokens = gqa->num_queries;
  p.layers = num_layers;
  p.kv_heads = gqa->num_kv_heads;
  p.head_dim = gqa->head_dim;
  p.scale_tokens = gqa->scale_tokens;
  p.max_pages = gqa->max_pages_per_seq;
  OA_HIP(launch_gqa_keep(p, cus, (hipStream_t)hip_stream));
  return OMNIATTN_OK;
}

int omniattn_gqa_append(const omniattn_gqa_t* gqa, int32_t num_tokens, const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride,
                        const int32_t* slot_map, void* k_cache, void* v_cache, float* k_scales, float* v_scales, void* hip_stream) {
  const int rc = check_gqa(gqa);
  if (rc != OMNIATTN_OK) return rc;
  if (num_tokens < 0) return OMNIATTN_EINVAL;
  if (num_tokens == 0) return OMNIATTN_OK;
  if (!k_new || !v_new || !slot_map || !k_cache || !v_cache || !k_scales || !v_scales) return OMNIATTN_EINVAL;
  // (rows are read 16 bytes at a time)
  if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16)) return OMNIATTN_EINVAL;
  if (k_stride % 8 != 0 || v_stride % 8 != 0) return OMNIATTN_EINVAL;
  const int64_t row = (int64_t)gqa->num_kv_heads * gqa->head_dim;
  if (k_stride < row || v_stride < row) return OMNIATTN_EINVAL;
  if ((int64_t)num_tokens * gqa->num_kv_heads > INT32_MAX / 2) return OMNIATTN_EUNSUPPORTED;
  GqaAppendParams p;
  p.rows[0] = (const uint16_t*)k_new;
  p.rows[1] = (const uint16_t*)v_new;
  p.stride[0] = k_stride;
  p.stride[1] = v_stride;
  p.slot_map = slot_map;
  p.cache[0] = (uint8_t*)k_cache;
  p.cache[1] = (uint8_t*)v_cache;
  p.scales[0] = k_scales;
  p.scales[1] = v_scales;
  p.num_tokens = num_tokens;
  p.kv_heads = gqa->num_kv_heads;
  p.head_dim = gqa->head_dim;
  p.scale_tokens = gqa->scale_tokens;
  p.num_slots = (uint32_t)(gqa->num_pages * kPage);
  OA_HIP(launch_gqa_append(p, (hipStream_t)hip_stream));
  return OMNIATTN_OK;
}

size_t omniattn_gqa_workspace_bytes(const omniattn_gqa_t* gqa) { return most_workspace(gqa, true); }

size_t omniattn_gqa_decode_workspace_bytes(const omniattn_gqa_t* gqa) { return most_workspace(gqa, false); }

int omniattn_gqa_decode(const omniattn_gqa_t* gqa, const void* q, int64_t q_stride, const void* k_cache, const void* v_cache, const float* k_scales,
                        const float* v_scales, const int32_t* page_table, const int32_t* seq_lens, const int32_t* q_start, void* out, float* lse,
                        void* workspace, size_t workspace_bytes, void* hip_stream) {
  return attend(gqa, q, q_stride, k_cache, v_cache, k_scales, v_scales, page_table, seq_lens, q_start, false, nullptr, out, lse, workspace, workspace_bytes, hip_stream);
}

int omniattn_gqa_tree(const omniattn_gqa_t* gqa, const void* q, int64_t q_stride, const void* k_cache, const void* v_cache, const float* k_scales,
                      const float* v_scales, const int32_t* page_table, const int32_t* seq_lens, const int32_t* q_start, const uint64_t* masks, void* out,
                      float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return attend(gqa, q, q_stride, k_cache, v_cache, k_scales, v_scales, page_table, seq_lens, q_start, true, masks, out, lse, workspace, workspace_bytes, hip_stream);
}

}  // extern "C"
