// Cross entropy over the joint vocabulary with its gradients: what z2z_api.cu hands to z2z_xent.cu.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "z2z_common.cuh"

namespace z2z {

constexpr int kXentMaxRows = 1 << 20;
struct XentArgs {
  int N, d, dtype;
  const void* hidden;            // [N, d]
  const int32_t *row_seq, *row_nvis, *targets;
  const void *WU, *Uh;
  float *loss, *lse;             // losses: outputs; gradients alone: lse is an input, loss is NULL
  bool want_loss, want_grad;
  const float* weight;           // [N] or NULL = 1
  int grad_dtype, accumulate;
  void *g_hidden, *g_WU, *g_Uh;  // each may be NULL
  char* scratch; size_t scratch_bytes;
  int* err;                      // device error word
};
// Bytes with which a call works, and from which on more does not make it faster.  grad_dtype < 0: losses alone.
void xent_scratch_bytes(const z2z_config& c, int N, int grad_dtype, size_t* least, size_t* most);
void xent_wait_limit(unsigned long long ns);     // of calls from now on; 0: the default
cudaError_t run_xent(const CbView& cb, const z2z_config& cfg, const XentArgs& a, cudaStream_t s);

}  // namespace z2z
