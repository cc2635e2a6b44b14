// Internal launcher of the log probabilities of tokens from logits (not part of the C ABI).
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

namespace ptd {
struct TokenLogprobsParams {
  const void* logits;
  int64_t rows, row_stride;   // elements
  int vocab, k;
  int per;                    // vectors of one CTA's part of a row (the launcher's)
  float scale;                // log2(e) / temperature
  float inv_temperature;
  const int32_t* tokens;      // [rows]
  float* logprob;             // [rows]
  float* entropy;             // [rows] or NULL
  int32_t* top_idx;           // [rows][k]
  float* top_val;
  int32_t* dev_status;
};
cudaError_t launch_token_logprobs(TokenLogprobsParams p, bool bf16, int sms, cudaStream_t stream);
}  // namespace ptd
