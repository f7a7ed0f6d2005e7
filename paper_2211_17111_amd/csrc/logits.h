// Internal interface between the logits operators' C ABI (logits_api.cpp) and
// their HIP kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <float.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include "bevpool_logits.h"

namespace bevpool {

constexpr int kMaxAlternatives = 64;  // of logprobs
constexpr int kMaxTaught = 256;       // of distill

// scale log2 e, as one float: its rounding is a relative 2^-25 of the scale.  A scale
// for which it is infinite is refused: a row's largest logit would have exponent 0
// times infinity.
inline float exponent_factor(float scale) {
  const double c = (double)scale * 1.4426950408889634;
  return c > (double)FLT_MAX ? INFINITY : (float)c;
}

// Rows of logits and what goes with each row.
struct LogitsRows {
  int64_t rows, stride;
  const void* logits;
  const void* ids;       // of tokens: one a row in logprobs (or NULL), k in distill
  const float* teacher;  // rows x k (distill)
  float scale;
  int32_t V, k;
  int dtype, key_type;
  bool renormalise;
};

struct LogprobsOut {
  float *stats, *logprob, *lse, *entropy, *top;
  int32_t* top_ids;
};
struct LogprobsGrads {
  const float *stats, *entropy;
  const int32_t* top_ids;
  const float *logprob, *lse, *of_entropy, *top;  // outgoing, NULL where there is none
};

size_t logprobs_workspace(int64_t rows, int64_t V, int32_t k, int dtype);
hipError_t launch_logprobs_forward(const LogitsRows& in, const LogprobsOut& out, void* workspace,
                                   hipStream_t stream);
hipError_t launch_logprobs_backward(const LogitsRows& in, const LogprobsGrads& g,
                                    void* grad_logits, hipStream_t stream);

size_t distill_workspace(int64_t rows, int64_t V, int32_t k, int dtype);
hipError_t launch_distill_forward(const LogitsRows& in, float* loss, float* stats, void* workspace,
                                  hipStream_t stream);
hipError_t launch_distill_backward(const LogitsRows& in, const float* grad_loss,
                                   const float* stats, void* grad_logits, hipStream_t stream);
hipError_t launch_distill_step(const LogitsRows& in, const float* grad_loss, float* loss,
                               float* stats, void* grad_logits, void* workspace,
                               hipStream_t stream);

}  // namespace bevpool
