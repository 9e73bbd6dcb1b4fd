// Arguments of the differential-attention kernels, on CUDA cores and on tensor cores.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace hift {

struct DattnArgs {
  const void* qkv; const float* lam; const void* gain; const int32_t* lens;
  void* o; void* o2; void* y; float* lse;                  // forward; backward reads o, o2 and lse
  const void* dy; const void* g; const float* dsum;        // g: gradient of o (dy itself without a norm); dsum: D_1 | D_2, each [B, H, S]
  void* dqkv;
  int B, S, H, K, causal;
  int vec;                                                 // qkv and g start at 16-byte boundaries
  float scale, eps, c;
};

// Tensor-core kernels (gemm_tc.cu): bf16, heads of 64 or 128, the buffers that they move by TMA 16-byte aligned, this device set up (gemm_tc_init).
bool dattn_tc_eligible(int dtype, int D, const DattnArgs& a);
cudaError_t dattn_tc_fwd_launch(cudaStream_t st, int D, const DattnArgs& a);
cudaError_t dattn_tc_bwd_launch(cudaStream_t st, int D, const DattnArgs& a);

}  // namespace hift
