// Shared declarations of the recovery operators (adapted projection, orthogonalised update).
#pragma once

#include "common.cuh"

namespace thanos {

struct AdapterArgs {
  // forward: out = Y [T, c], in = X [T, b]; backward: out = dX [T, b], in = dY [T, c]
  void* out = nullptr;
  int64_t ldo = 0;
  const void* in = nullptr;
  int64_t ldi = 0;
  const void* X = nullptr;      // backward: the forward input, for dA
  int64_t ldx = 0;
  const void* W = nullptr;
  int64_t ldw = 0;
  const void* A = nullptr;
  const void* B = nullptr;
  const int32_t* index = nullptr;
  const float* scale = nullptr;
  float* V = nullptr;           // forward: written (may be null)
  const float* Vin = nullptr;   // backward: read
  float* dA = nullptr;
  float* dB = nullptr;
  int accumulate = 0;
  thanos_dtype_t dtype = THANOS_BF16;
  int64_t T = 0, c = 0, b = 0, n = 0;
  int r = 0;
};

size_t adapter_workspace_bytes(bool backward, int64_t T, int64_t c, int64_t b, int64_t n, int r,
                               thanos_dtype_t dtype);
thanos_status_t adapter_forward_impl(const AdapterArgs& a, void* workspace, size_t ws_bytes,
                                     cudaStream_t stream);
thanos_status_t adapter_backward_impl(const AdapterArgs& a, void* workspace, size_t ws_bytes,
                                      cudaStream_t stream);

// fp32 operands (adapter_f32.cu)
size_t adapter_f32_workspace_bytes(bool back, int64_t T, int64_t c, int64_t b, int64_t n, int r);
thanos_status_t adapter_f32(bool back, const AdapterArgs& a, void* workspace, size_t ws_bytes,
                            cudaStream_t stream);

struct OrthogonalArgs {
  const void* G = nullptr;
  thanos_dtype_t gdtype = THANOS_F32;
  int64_t batch = 0, m = 0, n = 0;
  float coef[3] = {0.f, 0.f, 0.f};
  int steps = 0;
  float eps = 0.f;
  __nv_bfloat16* O = nullptr;   // thanos_orthogonalise
  // thanos_orthogonal_step
  void* W_out = nullptr;
  const void* W_in = nullptr;
  thanos_dtype_t wdtype = THANOS_F32;
  float* M_out = nullptr;
  const float* M_in = nullptr;
  const uint8_t* mask = nullptr;
  float keep = 1.f;             // 1 - lr * weight_decay
  float rate = 0.f;             // lr * gain
  float momentum = 0.f;
  int nesterov = 0;
};

size_t orthogonal_workspace_bytes(int64_t batch, int64_t m, int64_t n);
thanos_status_t orthogonal_impl(const OrthogonalArgs& a, void* workspace, size_t ws_bytes,
                                cudaStream_t stream);

}  // namespace thanos
