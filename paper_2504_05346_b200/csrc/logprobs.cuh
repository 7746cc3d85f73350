// Log probabilities of given tokens and their gradient (see logprobs.cu).
#pragma once

#include "common.cuh"

namespace thanos {

constexpr int LOGPROBS_MAX_TOP = 64;
constexpr int64_t LOGPROBS_MAX_VOCAB = 1 << 24;

struct LogprobsArgs {
  const void* Z = nullptr;          // [T, V], leading dimension ldz
  int64_t ldz = 0;
  thanos_dtype_t dtype = THANOS_BF16;
  const int64_t* target = nullptr;  // [T] or null
  float* logp = nullptr;            // [T] or null
  float* entropy = nullptr;         // [T]
  float* stats = nullptr;           // [T, 2]
  int64_t* top_index = nullptr;     // [T, k]
  float* top_logp = nullptr;
  int64_t T = 0, V = 0;
  int k = 0;
};

struct LogprobsGradArgs {
  const void* Z = nullptr;
  int64_t ldz = 0;
  void* dZ = nullptr;               // may be Z
  int64_t lddz = 0;
  thanos_dtype_t dtype = THANOS_BF16;
  const float* stats = nullptr;
  const int64_t* target = nullptr;
  const float* dlogp = nullptr;
  const float* entropy = nullptr;
  const float* dentropy = nullptr;
  const int64_t* top_index = nullptr;
  const float* dtop = nullptr;
  int64_t T = 0, V = 0;
  int k = 0;
};

thanos_status_t logprobs_impl(const LogprobsArgs& a, cudaStream_t stream);
thanos_status_t logprobs_grad_impl(const LogprobsGradArgs& a, cudaStream_t stream);

}  // namespace thanos
