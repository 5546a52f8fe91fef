// Constraints on logits: arguments of the kernel in logits.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace aqlm {

constexpr int kMaxBiases = 2047;
constexpr int64_t kMaxHistory = (1 << 20) - 1;

struct LogitsArgs {
  const void* in;
  void* out;
  const int32_t *tokens, *token_lens, *prompt_lens;
  const float *repetition, *frequency, *presence;
  const int32_t* bias_ids;
  const float* bias_values;
  const uint32_t* mask;
  int64_t in_row, out_row, token_row, bias_row, mask_row;
  int32_t rows, vocab, history, biases;
  int32_t slices_log2;
};

hipError_t launch_logits(const LogitsArgs& a, int dtype, hipStream_t s);

}  // namespace aqlm
