// Backward pass of the layers (lba_layer.cuh): host interface of lba_grad.cu and lba_grad_few.cu.
#pragma once
#include <cstddef>
#include <cstdint>
#include <cuda_runtime.h>

namespace lba {

struct GradCall {
  const void *grad, *pre;
  const uint8_t *A, *B, *B2;
  const float *sa, *sb, *sb2;
  const uint64_t* rng;
  void *grad_a, *grad_b, *grad_b2;      // each may be null
  float *grad_bias, *grad_bias2;
  int64_t M, N, K;
  int grad_type, pre_type, out_type, act, gated, in_m4e3, sa_per_row, sb_per_col;
  uint32_t drop_below;
  float keep_scale;
  int wait_override;  // see lba_set_wait_override
};

size_t backward_workspace(const GradCall& c);
// M, N below 2^31 and K at most 2^31 - 1; workspace 256-byte aligned, backward_workspace(c) bytes
cudaError_t launch_backward(const GradCall& c, void* workspace, cudaStream_t stream);
// lba_grad_few.cu: the same for few rows, where few_rows() holds; needs no workspace
bool few_rows(const GradCall& c, int pieces);
cudaError_t launch_backward_few(const GradCall& c, int pieces, cudaStream_t stream);

}  // namespace lba
