// C ABI of draft verification (see include/omniattn.h).
#include <hip/hip_runtime.h>

#include <climits>

#include "gqa.h"
#include "verify.h"

using namespace omniattn;

namespace {

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

int parts_of(int32_t vocab) { return (int)(((int64_t)vocab + kVerifyColumns - 1) / kVerifyColumns); }

struct Workspace {
  size_t rest, rows, choices, bytes;  // offsets, and the whole
};
Workspace workspace_of(int32_t num_tokens, int32_t vocab) {
  const size_t parts = (size_t)num_tokens * parts_of(vocab);
  Workspace w;
  w.rest = align256(parts * sizeof(VerifyPart));
  w.rows = w.rest + align256(parts * sizeof(double));
  w.choices = w.rows + align256((size_t)num_tokens * sizeof(VerifyRow));
  w.bytes = w.choices + (size_t)num_tokens * sizeof(VerifyChoice);
  return w;
}

int check_verify(const omniattn_verify_t* v) {
  if (!v) return OMNIATTN_EINVAL;
  if (v->batch < 1 || v->num_tokens < 0 || v->vocab < 1) return OMNIATTN_EINVAL;
  if (v->logits_dtype != OMNIATTN_BF16 && v->logits_dtype != OMNIATTN_FP32) return OMNIATTN_EUNSUPPORTED;
  // (columns are counted in 32 bits with a wave's columns on top, a launch's threads in 32: 64 of them to a part, 512 to a request)
  if (v->vocab > INT32_MAX - kVerifyColumns || v->batch > INT32_MAX >> 8) return OMNIATTN_EUNSUPPORTED;
  if ((int64_t)v->num_tokens * parts_of(v->vocab) >= INT32_MAX >> 5) return OMNIATTN_EUNSUPPORTED;
  return OMNIATTN_OK;
}

}  // namespace

extern "C" {

size_t omniattn_tree_verify_workspace_bytes(const omniattn_verify_t* verify) {
  return check_verify(verify) == OMNIATTN_OK ? workspace_of(verify->num_tokens, verify->vocab).bytes : 0;
}

int omniattn_tree_verify(const omniattn_verify_t* verify, const void* logits, int64_t logits_stride, const float* draft_probs, int64_t draft_stride,
                         const int32_t* tokens, const int32_t* parents, const int32_t* q_start, const float* temperature, const float* uniforms,
                         int32_t* path, int32_t* out_tokens, float* logprobs, int32_t* dropped, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const int rc = check_verify(verify);
  if (rc != OMNIATTN_OK) return rc;
  if (!q_start && verify->num_tokens != verify->batch) return OMNIATTN_EINVAL;
  if (!dropped || !temperature) return OMNIATTN_EINVAL;
  if (verify->num_tokens > 0 && (!logits || !tokens || !parents || !uniforms || !path || !out_tokens)) return OMNIATTN_EINVAL;
  if (logits_stride < verify->vocab || (draft_probs && draft_stride < verify->vocab)) return OMNIATTN_EINVAL;
  const Workspace w = workspace_of(verify->num_tokens, verify->vocab);
  if (w.bytes > 0 && (!workspace || workspace_bytes < w.bytes || ((uintptr_t)workspace & 255))) return OMNIATTN_EWORKSPACE;
  int cus = 0;
  const int found = device_cus(&cus);
  if (found != OMNIATTN_OK) return found;
  VerifyParams p;
  p.logits = logits;
  p.stride = logits_stride;
  p.draft_probs = draft_probs;
  p.draft_stride = draft_stride;
  p.tokens = tokens;
  p.parents = parents;
  p.q_start = q_start;
  p.temperature = temperature;
  p.uniforms = uniforms;
  p.path = path;
  p.out_tokens = out_tokens;
  p.logprobs = logprobs;
  p.dropped = dropped;
  p.parts = (VerifyPart*)workspace;
  p.rest = (double*)((char*)workspace + w.rest);
  p.rows = (VerifyRow*)((char*)workspace + w.rows);
  p.choices = (VerifyChoice*)((char*)workspace + w.choices);
  p.batch = verify->batch;
  p.num_tokens = verify->num_tokens;
  p.vocab = verify->vocab;
  p.num_parts = parts_of(verify->vocab);
  p.logits_fp32 = verify->logits_dtype == OMNIATTN_FP32;
  const hipError_t e = launch_tree_verify(p, cus, (hipStream_t)hip_stream);
  return e == hipSuccess ? OMNIATTN_OK : hip_fail(e, "launch_tree_verify");
}

}  // extern "C"
