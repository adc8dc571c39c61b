// Parameter block and launcher of the log probabilities (internal).
#pragma once
#include <cuda_runtime.h>
#include <cstdint>

namespace pc {

struct LogProb {
  const void* logits;                            // rows of V, `stride` elements apart
  long long stride;
  int N, V, top, group;
  float scale;
  const int* tokens;                             // [N] or null
  float *logprob, *entropy;                      // [N], each or null
  float* top_logprob;                            // [N,top]
  int* top_id;
  float* nll;                                    // [N / group] or null
};
enum { LOGITS_F32 = 0, LOGITS_BF16 = 1, LOGITS_F16 = 2 };
cudaError_t launch_token_logprobs(const LogProb& p, int type, int sm_count, cudaStream_t st);

}  // namespace pc
