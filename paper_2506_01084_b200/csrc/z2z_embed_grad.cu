// Gradient of the scaled mixed-stream lookup for its tables, by sorted tokens: the rows of the incoming gradient
// that name one target (a row of W_E, or an entry of one sequence) are brought together by a stable sort of the
// codes and added in fp32 in the order of their rows.
#include "z2z_common.cuh"
#include "z2z_internal.h"
#include "z2z_sm100.cuh"

namespace z2z {

namespace {

constexpr int kNoTarget = 0x7fffffff;

// Targets are numbered 0 .. V - 1 (rows of W_E), then V + b * cap + k.
struct GradView { int V, cap, B; void *gWE, *gEh; int d; };

template <typename T> __device__ __forceinline__ T* target_row(const GradView& v, int t) {
  return t < v.V ? reinterpret_cast<T*>(v.gWE) + (size_t)t * v.d : reinterpret_cast<T*>(v.gEh) + (size_t)(t - v.V) * v.d;
}

}  // namespace

// keys[r] = target of row r, kNoTarget without one.
__global__ void __launch_bounds__(256) k_grad_keys(CbView cb, const int32_t* __restrict__ codes, int N,
                                                   const int32_t* __restrict__ row_seq, int want_base, int want_hyper,
                                                   int32_t* __restrict__ keys) {
  sm100::pdl_wait();
  sm100::pdl_trigger();
  const int r = blockIdx.x * blockDim.x + threadIdx.x;
  if (r >= N) return;
  const int z = codes[r], b = row_seq ? row_seq[r] : r;
  int key = kNoTarget;
  if ((unsigned)b < (unsigned)cb.B) {
    if (z >= 0 && z < cb.V) { if (want_base) key = z; }
    else if (z >= cb.V && z - cb.V < cb.n[b]) { if (want_hyper) key = cb.V + b * cb.cap + (z - cb.V); }
    else if (z != Z2Z_CODE_NONE) atomicOr(&cb.status[b], Z2Z_ST_BAD_TOKEN);
  }
  keys[r] = key;
}

// Place of every row in the stable order of the keys, by counting the keys before it.
__global__ void __launch_bounds__(256) k_grad_rank(const int32_t* __restrict__ keys, int N, int32_t* __restrict__ sorted_key,
                                                   int32_t* __restrict__ sorted_row) {
  sm100::pdl_wait();
  sm100::pdl_trigger();
  __shared__ int32_t s[1024];
  const int r = blockIdx.x * blockDim.x + threadIdx.x;
  const int k = r < N ? keys[r] : 0;
  int rank = 0;
  for (int j0 = 0; j0 < N; j0 += 1024) {
    __syncthreads();
    for (int i = threadIdx.x; i < 1024; i += 256) s[i] = j0 + i < N ? keys[j0 + i] : kNoTarget;
    __syncthreads();
    const int m = N - j0 < 1024 ? N - j0 : 1024;
    for (int i = 0; i < m; ++i) rank += (s[i] < k || (s[i] == k && j0 + i < r)) ? 1 : 0;
  }
  if (r < N) { sorted_key[rank] = k; sorted_row[rank] = r; }
}

// One warp per place of the sorted list; the warp at a target's first place adds up its rows.
template <typename TG, typename TO>
__global__ void __launch_bounds__(256) k_grad_sum(GradView v, const int32_t* __restrict__ key, const int32_t* __restrict__ row, int N,
                                                  const TG* __restrict__ g, float scale, int accumulate) {
  sm100::pdl_wait();
  sm100::pdl_trigger();
  const int i = (blockIdx.x * blockDim.x + threadIdx.x) >> 5, lane = threadIdx.x & 31;
  if (i >= N) return;
  const int t = key[i];
  if (t == kNoTarget || (i > 0 && key[i - 1] == t)) return;
  TO* out = target_row<TO>(v, t);
  for (int c = lane; c < v.d; c += 32) {
    float acc = 0.f;
    for (int j = i; j < N && key[j] == t; ++j) acc += to_f32<TG>(g[(size_t)row[j] * v.d + c]);
    acc *= scale;
    if (accumulate) acc += to_f32<TO>(out[c]);
    out[c] = from_f32<TO>(acc);
  }
}

// Zero in the rows that no code names (accumulate == 0): one warp per target, found by bisection of the sorted keys.
template <typename TO>
__global__ void __launch_bounds__(256) k_grad_zero(CbView cb, GradView v, const int32_t* __restrict__ key, int N, int t_lo, int t_hi) {
  sm100::pdl_wait();
  sm100::pdl_trigger();
  const int lane = threadIdx.x & 31;
  const int warps = (gridDim.x * blockDim.x) >> 5;
  for (int t = t_lo + ((blockIdx.x * blockDim.x + threadIdx.x) >> 5); t < t_hi; t += warps) {
    if (t >= v.V) {
      const int b = (t - v.V) / v.cap, k = (t - v.V) % v.cap;
      if (k >= cb.n[b]) continue;
    }
    int lo = 0, hi = N;
    while (lo < hi) {
      const int m = (lo + hi) >> 1;
      if (key[m] < t) lo = m + 1; else hi = m;
    }
    if (lo < N && key[lo] == t) continue;
    TO* out = target_row<TO>(v, t);
    for (int c = lane; c < v.d; c += 32) out[c] = from_f32<TO>(0.f);
  }
}

size_t embed_grad_scratch_bytes(int N, int d) {
  (void)d;
  return 3 * align_up((size_t)N * 4, 256);
}

cudaError_t launch_embed_grad(const CbView& cb, const EmbedGradArgs& a, cudaStream_t s) {
  const size_t list = align_up((size_t)a.N * 4, 256);
  int32_t* keys = reinterpret_cast<int32_t*>(a.scratch);
  int32_t* sorted_key = reinterpret_cast<int32_t*>(a.scratch + list);
  int32_t* sorted_row = reinterpret_cast<int32_t*>(a.scratch + 2 * list);
  const GradView v{cb.V, cb.cap, cb.B, a.gWE, a.gEh, a.d};
  cudaError_t e = cudaSuccess;
  if (a.N > 0) {
    const dim3 rows((a.N + 255) / 256);
    e = launch_pdl(k_grad_keys, rows, dim3(256), 0, s, cb, a.codes, a.N, a.row_seq, a.gWE ? 1 : 0, a.gEh ? 1 : 0, keys);
    if (e == cudaSuccess) e = launch_pdl(k_grad_rank, rows, dim3(256), 0, s, keys, a.N, sorted_key, sorted_row);
    const dim3 warps((a.N + 7) / 8);
    const int acc = a.accumulate ? 1 : 0;
    if (e == cudaSuccess) {
      if (a.g_dtype == Z2Z_DTYPE_BF16 && a.grad_dtype == Z2Z_DTYPE_BF16)
        e = launch_pdl(k_grad_sum<__nv_bfloat16, __nv_bfloat16>, warps, dim3(256), 0, s, v, sorted_key, sorted_row, a.N, (const __nv_bfloat16*)a.g, a.scale, acc);
      else if (a.g_dtype == Z2Z_DTYPE_BF16)
        e = launch_pdl(k_grad_sum<__nv_bfloat16, float>, warps, dim3(256), 0, s, v, sorted_key, sorted_row, a.N, (const __nv_bfloat16*)a.g, a.scale, acc);
      else if (a.grad_dtype == Z2Z_DTYPE_BF16)
        e = launch_pdl(k_grad_sum<float, __nv_bfloat16>, warps, dim3(256), 0, s, v, sorted_key, sorted_row, a.N, (const float*)a.g, a.scale, acc);
      else
        e = launch_pdl(k_grad_sum<float, float>, warps, dim3(256), 0, s, v, sorted_key, sorted_row, a.N, (const float*)a.g, a.scale, acc);
    }
  }
  if (e == cudaSuccess && !a.accumulate) {
    const int lo = a.gWE ? 0 : cb.V, hi = a.gEh ? cb.V + cb.B * cb.cap : cb.V;
    const int blocks = (hi - lo + 7) / 8 < 148 * 8 ? (hi - lo + 7) / 8 : 148 * 8;
    if (hi > lo) {
      if (a.grad_dtype == Z2Z_DTYPE_BF16) e = launch_pdl(k_grad_zero<__nv_bfloat16>, dim3(blocks), dim3(256), 0, s, cb, v, sorted_key, a.N, lo, hi);
      else e = launch_pdl(k_grad_zero<float>, dim3(blocks), dim3(256), 0, s, cb, v, sorted_key, a.N, lo, hi);
    }
  }
  return e;
}

}  // namespace z2z
