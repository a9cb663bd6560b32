// Tokens drawn from rows of logits: what the host hands to the kernel.
#pragma once

#include "rlkv_internal.h"

namespace rlkv {

struct SampleCall {
  const void* logits;
  int64_t stride;
  int32_t rows, vocab;
  // for all rows, or where not null one a row
  double temperature, top_p, min_p;
  int32_t top_k;
  const float *temperatures, *top_ps, *min_ps;
  const int32_t* top_ks;
  const float* uniforms;
  int32_t* tokens;
  float* logprobs;            // or null
  void* workspace;
};
size_t sample_workspace(int rows, int vocab);
hipError_t launch_sample(const SampleCall& call, int dtype, hipStream_t stream);

}  // namespace rlkv
