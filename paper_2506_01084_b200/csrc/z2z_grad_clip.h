// Global gradient norm and clipping: what z2z_api.cu hands to z2z_grad_clip.cu.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>

#include "../../include/z2z.h"

namespace z2z {

constexpr int kGradClipMaxTensors = 1 << 16;
size_t grad_clip_scratch_bytes(int n);
long long grad_clip_max_elements();              // of all tensors of 512 consecutive records together
cudaError_t launch_grad_clip(const z2z_grad_tensor* t, int n, float scale, float max_norm, float* norm, double* part, cudaStream_t s);

}  // namespace z2z
