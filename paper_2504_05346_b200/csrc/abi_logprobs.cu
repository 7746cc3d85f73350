// extern "C" entry points of the token log probabilities: argument checks and dispatch.
#include "logprobs.cuh"

using namespace thanos;

namespace {

constexpr int64_t MAX_TOKENS = 1 << 24;
constexpr int64_t MAX_BLOCKS = 0x7FFFFFFF;

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

thanos_status_t logits_shape(int64_t n_tok, int64_t vocab, int32_t k, thanos_dtype_t dtype) {
  if (dtype != THANOS_F32 && dtype != THANOS_BF16) return THANOS_ERR_DTYPE;
  if (n_tok < 0 || n_tok > MAX_TOKENS || vocab < 1 || vocab > LOGPROBS_MAX_VOCAB || k < 0 ||
      k > LOGPROBS_MAX_TOP || k > vocab)
    return THANOS_ERR_SHAPE;
  // what a launch's grid holds: the backward pass takes CTAs of 4096 fp32 or 8192 bf16 columns
  if (n_tok * (vocab / 4096 + 2) > MAX_BLOCKS) return THANOS_ERR_SHAPE;
  return THANOS_OK;
}

}  // namespace

extern "C" {

thanos_status_t thanos_token_logprobs(float* logp, float* entropy, float* stats, int64_t* top_index,
                                      float* top_logp, const void* Z, int64_t ldz,
                                      thanos_dtype_t dtype, const int64_t* target, int64_t n_tok,
                                      int64_t vocab, int32_t k, void* stream) {
  if (n_tok > 0 && (!Z || !entropy || !stats || (target && !logp) ||
                    (k > 0 && (!top_index || !top_logp))))
    return THANOS_ERR_INVALID_ARG;
  THANOS_TRY(logits_shape(n_tok, vocab, k, dtype));
  if (ldz < vocab) return THANOS_ERR_SHAPE;
  if (!aligned(Z, dtype == THANOS_BF16 ? 2 : 4) || !aligned(logp, 4) || !aligned(entropy, 4) ||
      !aligned(stats, 4) || !aligned(top_index, 8) || !aligned(top_logp, 4) || !aligned(target, 8))
    return THANOS_ERR_ALIGNMENT;
  if (n_tok == 0) return THANOS_OK;
  LogprobsArgs a;
  a.Z = Z;
  a.ldz = ldz;
  a.dtype = dtype;
  a.target = target;
  a.logp = target ? logp : nullptr;
  a.entropy = entropy;
  a.stats = stats;
  a.top_index = top_index;
  a.top_logp = top_logp;
  a.T = n_tok;
  a.V = vocab;
  a.k = k;
  return logprobs_impl(a, static_cast<cudaStream_t>(stream));
}

thanos_status_t thanos_token_logprobs_backward(void* dZ, int64_t lddz, const void* Z, int64_t ldz,
                                               thanos_dtype_t dtype, const float* stats,
                                               const int64_t* target, const float* dlogp,
                                               const float* entropy, const float* dentropy,
                                               const int64_t* top_index, const float* dtop,
                                               int64_t n_tok, int64_t vocab, int32_t k,
                                               void* stream) {
  if (n_tok > 0 && (!dZ || !Z || !stats || !target != !dlogp || (dentropy && !entropy) ||
                    (dtop && (!top_index || k == 0))))
    return THANOS_ERR_INVALID_ARG;
  THANOS_TRY(logits_shape(n_tok, vocab, k, dtype));
  if (ldz < vocab || lddz < vocab) return THANOS_ERR_SHAPE;
  const size_t e = dtype == THANOS_BF16 ? 2 : 4;
  if (!aligned(dZ, e) || !aligned(Z, e) || !aligned(stats, 4) || !aligned(target, 8) ||
      !aligned(dlogp, 4) || !aligned(entropy, 4) || !aligned(dentropy, 4) ||
      !aligned(top_index, 8) || !aligned(dtop, 4))
    return THANOS_ERR_ALIGNMENT;
  if (n_tok == 0) return THANOS_OK;
  LogprobsGradArgs a;
  a.Z = Z;
  a.ldz = ldz;
  a.dZ = dZ;
  a.lddz = lddz;
  a.dtype = dtype;
  a.stats = stats;
  a.target = target;
  a.dlogp = dlogp;
  a.entropy = dentropy ? entropy : nullptr;
  a.dentropy = dentropy;
  a.top_index = dtop ? top_index : nullptr;
  a.dtop = dtop;
  a.T = n_tok;
  a.V = vocab;
  a.k = dtop ? k : 0;
  return logprobs_grad_impl(a, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
