// Launch interface between the C ABI of draft verification (api_verify.cpp) and its gfx950 kernels (verify_kernels.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/omniattn.h"

namespace omniattn {

// Columns of a row that a wave looks at together.
constexpr int kVerifyColumns = 2048;

// Of kVerifyColumns logits of a row: the largest, the first column that has it, and the sum of exp((l - largest) / T).
struct VerifyPart {
  double sum;
  float top;
  int32_t best;
};

// Of a row: these over all columns, the node's first child (-1: none, or the request takes the likeliest token), whether it is taken, and its token's logit.
struct VerifyRow {
  double sum;
  float top;
  int32_t best, child, taken;
  float logit;
};
// Of a node: its token, the child that the walk goes to (-1: none, -2: the node was not looked at), and the logarithm of the token's probability.
struct VerifyChoice {
  int32_t token, next;
  float logprob;
};

struct VerifyParams {
  const void* logits;
  int64_t stride;          // elements from one row to the next
  const float* draft_probs;  // or null
  int64_t draft_stride;
  const int32_t* tokens;
  const int32_t* parents;
  const int32_t* q_start;  // [batch + 1], or null: node b belongs to request b
  const float* temperature;
  const float* uniforms;   // [num_tokens, 2]
  int32_t* path;
  int32_t* out_tokens;
  float* logprobs;         // or null
  int32_t* dropped;
  VerifyPart* parts;       // [num_tokens, num_parts]
  double* rest;            // the same; sums of max(p - q, 0)
  VerifyRow* rows;         // [num_tokens]
  VerifyChoice* choices;   // [num_tokens]
  int batch, num_tokens, vocab, num_parts;
  int logits_fp32;
};
// cus: the device's compute units.
hipError_t launch_tree_verify(const VerifyParams& p, int cus, hipStream_t stream);

}  // namespace omniattn
