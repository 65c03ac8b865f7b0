// Log probabilities of given tokens (logprobs.cu).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace rd {

struct LogprobArgs {
  const void* logits;         // [*][vocab], rows row_stride elements apart
  long long row_stride;
  const int32_t* row_index;   // [rows] row of the logits, or nullptr: row r; < 0: no row (NaN and -1 come out)
  const int32_t* tokens;      // [rows] or nullptr
  int rows, vocab, n_logit_rows, top;
  float inv_t;                // 1 / temperature
  float* logprob;             // [rows] or nullptr
  float* entropy;             // [rows] or nullptr
  int32_t* top_ids;           // [rows][top]
  float* top_logprobs;        // [rows][top]
};
constexpr int LOGPROB_MAX_TOP = 64;
cudaError_t launch_logprobs(int dtype, const LogprobArgs& a, cudaStream_t st);

}  // namespace rd
