// Internal declarations of draft verification (include/cllm_verify.h).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/cllm_verify.h"

namespace cllm {

// What the first kernel finds of a row: its largest logit and sum; of a greedy row the token.
struct alignas(16) VerifyRow {
  float max, sum;
  int verdict, top;  // kStands | kNothing | kGreedy; else top is the draft, -1: none
};
constexpr int kStands = 1, kNothing = 2, kGreedy = 4;

struct VerifyArgs {
  const void* logits;
  const int *tokens, *row_start, *seq_len;
  const float *temperature, *uniforms, *race, *draft_probs;
  int *accepted, *next;
  float* target_probs;
  long long logits_row, race_row, probs_row;
  int batch, rows, vocab;
  int splits, split_len;  // of a row in the first kernel
  int parts, part_len;    // of a request's deciding row in the second
  // scratch: a row's shares (splits > 1) and the counters of those that have come; rows; a request's
  // best key and its counter.  Counters and keys are zero between calls.
  unsigned long long* shares;
  int* row_tickets;
  VerifyRow* found;
  unsigned long long* best;
  int* request_tickets;
};

constexpr int kVerifyWarps = 32;  // of the first kernel on an SM: shares of rows, beyond one a row
cudaError_t launch_verify(const VerifyArgs& a, int dtype, int sms, cudaStream_t s);

}  // namespace cllm
