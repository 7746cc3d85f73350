// Weights in 4 bits and activations in 8 (see packed.cu), and the adapted projection on packed weights
// (packed_gemv.cu).
#pragma once

#include "recovery.cuh"

namespace thanos {

constexpr int ACT_GROUP = 32;       // columns that share an exponent

// Two codes a byte, the even column in the low half, offset by 8; scales [groups, c].
struct PackedWeights {
  const uint8_t* codes = nullptr;   // [c, ldq], rows of whole 64-column blocks
  int64_t ldq = 0;                  // bytes
  const __nv_bfloat16* scales = nullptr;
  int group = 0;
};

// x = code 2^(exponent - 127).
struct PackedActivations {
  const int8_t* codes = nullptr;    // [T, ldc]
  int64_t ldc = 0;
  const uint8_t* exps = nullptr;    // [T, lde]
  int64_t lde = 0;
};

// What is below the scales' five significant bits takes no part: a code times a scale then has at most
// eight bits, and is a bf16 number.
constexpr uint32_t SCALE_BITS = 0xFFF8u;

// The nibbles j and j + 4 of a word as the bf16 numbers whose low bits they are: 128 + nibble, or with
// another base what that has.  Both constants have to be in registers (`Nibbles`): an instruction takes one
// of its own only, and the pair would take two.
struct Nibbles {
  uint32_t mask = 0x000F000Fu, base;
  __device__ __forceinline__ explicit Nibbles(uint32_t base_ = 0x43004300u) : base(base_) {
    asm volatile("" : "+r"(mask), "+r"(base));
  }
  __device__ __forceinline__ uint32_t operator()(uint32_t w, int j) const {
    uint32_t v;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(v) : "r"(w >> (4 * j)), "r"(mask), "r"(base));
    return v;
  }
};

thanos_status_t pack_weights(uint8_t* codes, int64_t ldq, __nv_bfloat16* scales, const void* W,
                             int64_t ldw, thanos_dtype_t dtype, int64_t c, int64_t b, int group,
                             cudaStream_t stream);
// beside: starts while the launch before it in the stream runs, on whose results it does not depend, and
// is complete when both are.
thanos_status_t unpack_weights(void* W, int64_t ldw, thanos_dtype_t dtype, const PackedWeights& w,
                               int64_t c, int64_t b, cudaStream_t stream, bool beside = false);
thanos_status_t pack_activations(int8_t* codes, int64_t ldc, uint8_t* exps, int64_t lde,
                                 const void* X, int64_t ldx, thanos_dtype_t dtype, int64_t T,
                                 int64_t b, cudaStream_t stream);
thanos_status_t unpack_activations(void* X, int64_t ldx, thanos_dtype_t dtype, const int8_t* codes,
                                   int64_t ldc, const uint8_t* exps, int64_t lde, int64_t T,
                                   int64_t b, cudaStream_t stream);

// The adapted projection of few tokens, straight from the codes.  a.W is not read.
bool packed_few_tokens(const AdapterArgs& a);
size_t packed_few_workspace_bytes(int64_t T, int r);
thanos_status_t packed_forward_few(const AdapterArgs& a, const PackedWeights& w, void* workspace,
                                   cudaStream_t stream);

}  // namespace thanos
