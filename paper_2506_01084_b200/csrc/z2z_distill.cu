// Distillation of joint logits from a teacher's top logits.  With l the row's logits over its C columns,
// q = softmax(l / T), and p = softmax(t / T) over the teacher's entries that the row can see:
//   loss = T^2 sum_j p_j (log p_j - log q_{id_j}),     d loss / d l_c = T (q_c - sum_{id_j = c} p_j).
#include <cmath>

#include "z2z_common.cuh"
#include "z2z_internal.h"
#include "z2z_sm100.cuh"

namespace z2z {

namespace {

constexpr int kDistillMaxK = 1024;
constexpr int kDistillThreads = 512;

struct DistillArgs {
  const void* logits; int cols; long long ld;
  const int32_t* n_cols; const int32_t* ids; const float* t; int K;
  float inv_t, temperature;
  const float* weight;          // row weights (gradient), or NULL = 1
  float* loss; float* lse;      // out; the backward pass reads lse
  void* grad;                   // or NULL
};

struct Teacher { int id[kDistillMaxK]; float p[kDistillMaxK]; float red[32]; };

__device__ __forceinline__ float block_max(float v, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = threadIdx.x % 32 < blockDim.x / 32 ? red[threadIdx.x & 31] : -INFINITY;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float block_sum(float v, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = threadIdx.x % 32 < blockDim.x / 32 ? red[threadIdx.x & 31] : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

}  // namespace

// One block per row.  BACKWARD: lse is given and only the gradient is written.
template <typename T, bool BACKWARD>
__global__ void __launch_bounds__(kDistillThreads) k_distill_row(DistillArgs a) {
  __shared__ Teacher tc;
  sm100::pdl_wait();
  sm100::pdl_trigger();
  const int r = blockIdx.x, tid = threadIdx.x;
  const T* l = reinterpret_cast<const T*>(a.logits) + (size_t)r * a.ld;
  int C = a.n_cols ? a.n_cols[r] : a.cols;
  C = C < 0 ? 0 : (C > a.cols ? a.cols : C);
  const float w = a.weight ? a.weight[r] : 1.f;
  // teacher
  float tm = -INFINITY;
  for (int j = tid; j < a.K; j += kDistillThreads) {
    const int id = a.ids[(size_t)r * a.K + j];
    const float x = (unsigned)id < (unsigned)C ? a.t[(size_t)r * a.K + j] : -INFINITY;
    tc.id[j] = x == -INFINITY ? -1 : id;
    tc.p[j] = x;
    tm = fmaxf(tm, x == x ? x : INFINITY);
  }
  tm = block_max(tm, tc.red);
  const bool some = tm > -INFINITY;
  float ts = 0.f;
  for (int j = tid; j < a.K; j += kDistillThreads) if (tc.id[j] >= 0) ts += expf((tc.p[j] - tm) * a.inv_t);
  ts = block_sum(ts, tc.red);
  // student
  float m = -INFINITY, s = 0.f, lse = 0.f;
  if (!BACKWARD) {
    for (int c = tid; c < C; c += kDistillThreads) m = fmaxf(m, to_f32<T>(l[c]));
    m = block_max(m, tc.red);
    for (int c = tid; c < C; c += kDistillThreads) { const float x = to_f32<T>(l[c]); s += x == -INFINITY ? 0.f : expf((x - m) * a.inv_t); }
    s = block_sum(s, tc.red);
    lse = s == 0.f ? -INFINITY : m * a.inv_t + logf(s);
  } else {
    lse = a.lse[r];
  }
  const bool live = some && lse != -INFINITY;
  float loss = 0.f;
  for (int j = tid; j < a.K; j += kDistillThreads) {
    const float x = (tc.p[j] - tm) * a.inv_t;
    const float p = tc.id[j] >= 0 ? expf(x) / ts : 0.f;
    if (!BACKWARD && p != 0.f) loss += p * (x - logf(ts) - ((to_f32<T>(l[tc.id[j]]) - m) * a.inv_t - logf(s)));
    tc.p[j] = p;
  }
  if (!BACKWARD) {
    loss = block_sum(loss, tc.red);
    if (tid == 0) { a.loss[r] = live ? loss * a.temperature * a.temperature : 0.f; a.lse[r] = lse; }
  }
  if (!a.grad) return;
  T* out = reinterpret_cast<T*>(a.grad) + (size_t)r * a.ld;
  const bool zero = !live || w == 0.f;
  const float k = w * a.temperature;
  __syncthreads();
  // the teacher's columns: taken before the row is overwritten, written behind it
  float at[kDistillMaxK / kDistillThreads];
  int n_at = 0;
  for (int j = tid; j < a.K; j += kDistillThreads, ++n_at) {
    const int id = tc.id[j];
    float p = 0.f;
    bool first = id >= 0;
    for (int i = 0; i < a.K && first; ++i)
      if (tc.id[i] == id) { if (i < j) first = false; else p += tc.p[i]; }
    const float x = first ? to_f32<T>(l[id]) : 0.f;
    const float q = BACKWARD ? expf(fmaf(x, a.inv_t, -lse)) : expf((x - m) * a.inv_t) / s;
    at[n_at & 1] = first ? k * (q - p) : 0.f;
  }
  __syncthreads();
  for (int c = tid; c < a.cols; c += kDistillThreads) {
    float d = 0.f;
    if (!zero && c < C) {
      const float x = to_f32<T>(l[c]);
      d = k * (BACKWARD ? expf(fmaf(x, a.inv_t, -lse)) : (x == -INFINITY ? 0.f : expf((x - m) * a.inv_t)) / s);
    }
    out[c] = from_f32<T>(d);
  }
  __syncthreads();
  n_at = 0;
  if (!zero)
    for (int j = tid; j < a.K; j += kDistillThreads, ++n_at) {
      const int id = tc.id[j];
      bool first = id >= 0;
      for (int i = 0; i < j && first; ++i) if (tc.id[i] == id) first = false;
      if (first) out[id] = from_f32<T>(at[n_at & 1]);
    }
}

namespace {
int fail_arg(const char* msg) { set_last_error(msg); return Z2Z_ERR_INVALID_ARG; }

int check_distill(const void* logits, int dtype, int N, int cols, int64_t ld, const int32_t* ids, const float* t, int K, float temperature,
                  const void* grad) {
  if (dtype != Z2Z_DTYPE_FP32 && dtype != Z2Z_DTYPE_BF16) return fail_arg("unknown dtype");
  if (N < 0) return fail_arg("N < 0");
  if (cols < 1 || cols > (1 << 24)) return fail_arg("need 1 <= cols <= 2^24");
  if (ld < cols) return fail_arg("ld < cols");
  if (K < 0 || K > kDistillMaxK) return fail_arg("need 0 <= K <= 1024");
  if (!(temperature > 0.f) || !std::isfinite(temperature) || !std::isfinite(1.f / temperature)) return fail_arg("temperature must be > 0 and finite");
  if (N == 0) return Z2Z_OK;
  if (!logits) return fail_arg("d_logits is NULL");
  if (K > 0 && (!ids || !t)) return fail_arg("d_teacher_ids / d_teacher_logits is NULL");
  const uintptr_t es = dtype == Z2Z_DTYPE_BF16 ? 2 : 4;
  if (reinterpret_cast<uintptr_t>(logits) % es || reinterpret_cast<uintptr_t>(grad) % es) return fail_arg("logits and gradients must be aligned to their elements");
  return Z2Z_OK;
}

template <bool BACKWARD>
int launch_distill(const DistillArgs& a, int dtype, int N, cudaStream_t s) {
  cudaError_t e = dtype == Z2Z_DTYPE_BF16 ? launch_pdl(k_distill_row<__nv_bfloat16, BACKWARD>, dim3(N), dim3(kDistillThreads), 0, s, a)
                                          : launch_pdl(k_distill_row<float, BACKWARD>, dim3(N), dim3(kDistillThreads), 0, s, a);
  if (e != cudaSuccess) { set_last_error(cudaGetErrorString(e)); return Z2Z_ERR_CUDA; }
  return Z2Z_OK;
}
}  // namespace

}  // namespace z2z

extern "C" {

int32_t z2z_distill_loss(const void* d_logits, int32_t dtype, int32_t N, int32_t cols, int64_t ld,
                         const int32_t* d_n_cols, const int32_t* d_teacher_ids,
                         const float* d_teacher_logits, int32_t K, float temperature,
                         const float* d_row_weight, float* d_loss, float* d_lse, void* d_grad,
                         z2z_stream stream) {
  const int rc = z2z::check_distill(d_logits, dtype, N, cols, ld, d_teacher_ids, d_teacher_logits, K, temperature, d_grad);
  if (rc || N == 0) return rc;
  if (!d_loss || !d_lse) return z2z::fail_arg("d_loss / d_lse is NULL");
  z2z::DistillArgs a{d_logits, cols, ld, d_n_cols, d_teacher_ids, d_teacher_logits, K, 1.f / temperature, temperature,
                     d_row_weight, d_loss, d_lse, d_grad};
  return z2z::launch_distill<false>(a, dtype, N, reinterpret_cast<cudaStream_t>(stream));
}

int32_t z2z_distill_grad(const void* d_logits, int32_t dtype, int32_t N, int32_t cols, int64_t ld,
                         const int32_t* d_n_cols, const int32_t* d_teacher_ids,
                         const float* d_teacher_logits, int32_t K, float temperature,
                         const float* d_lse, const float* d_grad_loss, void* d_grad, z2z_stream stream) {
  const int rc = z2z::check_distill(d_logits, dtype, N, cols, ld, d_teacher_ids, d_teacher_logits, K, temperature, d_grad);
  if (rc || N == 0) return rc;
  if (!d_lse || !d_grad_loss || !d_grad) return z2z::fail_arg("d_lse / d_grad_loss / d_grad is NULL");
  z2z::DistillArgs a{d_logits, cols, ld, d_n_cols, d_teacher_ids, d_teacher_logits, K, 1.f / temperature, temperature,
                     d_grad_loss, nullptr, const_cast<float*>(d_lse), d_grad};
  return z2z::launch_distill<true>(a, dtype, N, reinterpret_cast<cudaStream_t>(stream));
}

}  // extern "C"
