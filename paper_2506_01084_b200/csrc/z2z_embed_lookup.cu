// Input embedding of a mixed base-token / hypertoken stream (Figure 2a; Section 2.3 steps 3-4):
// a base token reads its row of the embedding matrix, a hypertoken reads the hyper-embedding the
// session cached when the entry was created.  A pure gather: each output row is read once and
// written once, so the kernel is bound by HBM bandwidth (2 x N x d x element size).
//
// One warp copies one row with 16-byte accesses, several in flight per lane; warps stride over
// the rows with a grid sized to the machine.
#include "z2z_common.cuh"
#include "z2z_internal.h"
#include "z2z_sm100.cuh"

namespace z2z {

namespace {
constexpr int kLookupThreads = 256;
constexpr int kLookupUnroll = 4;
}

__global__ void __launch_bounds__(kLookupThreads) k_embed_lookup(
    CbView cb, const int32_t* codes, int N, const int32_t* row_seq, const uint4* WE, const uint4* Eh, uint4* out,
    int row_vecs /* 16-byte vectors per row */) {
  sm100::pdl_wait();                              // codes, codebook state and cache rows come from earlier kernels
  sm100::pdl_trigger();
  const int lane = threadIdx.x & 31;
  const int warps = (gridDim.x * blockDim.x) >> 5;
  for (int r = (blockIdx.x * blockDim.x + threadIdx.x) >> 5; r < N; r += warps) {
    const int z = codes[r];
    const int b = row_seq ? row_seq[r] : r;
    const uint4* src = nullptr;
    if ((unsigned)b < (unsigned)cb.B) {
      if (z >= 0 && z < cb.V) src = WE + (size_t)z * row_vecs;
      else if (z >= cb.V && z - cb.V < cb.n[b]) src = Eh + ((size_t)b * cb.cap + (z - cb.V)) * row_vecs;
    }
    uint4* dst = out + (size_t)r * row_vecs;
    if (!src) {                                   // no such token: zero row, flag the sequence
      if (lane == 0 && z != Z2Z_CODE_NONE && (unsigned)b < (unsigned)cb.B) atomicOr(&cb.status[b], Z2Z_ST_BAD_TOKEN);
      for (int i = lane; i < row_vecs; i += 32) dst[i] = make_uint4(0, 0, 0, 0);
      continue;
    }
    int i = lane;
    for (; i + 32 * (kLookupUnroll - 1) < row_vecs; i += 32 * kLookupUnroll) {
      uint4 v[kLookupUnroll];
#pragma unroll
      for (int u = 0; u < kLookupUnroll; ++u) v[u] = __ldcg(src + i + 32 * u);
#pragma unroll
      for (int u = 0; u < kLookupUnroll; ++u) __stcs(dst + i + 32 * u, v[u]);
    }
    for (; i < row_vecs; i += 32) __stcs(dst + i, __ldcg(src + i));
  }
}

namespace {
// 16 bytes of a row times a scale: the product in fp32, one rounding to the storage type.
template <typename T> __device__ __forceinline__ uint4 scaled(uint4 v, float a);
template <> __device__ __forceinline__ uint4 scaled<float>(uint4 v, float a) {
  return make_uint4(__float_as_uint(__uint_as_float(v.x) * a), __float_as_uint(__uint_as_float(v.y) * a),
                    __float_as_uint(__uint_as_float(v.z) * a), __float_as_uint(__uint_as_float(v.w) * a));
}
__device__ __forceinline__ uint32_t scaled_pair(uint32_t v, float a) {
  const __nv_bfloat162 r = __floats2bfloat162_rn(__uint_as_float(v << 16) * a, __uint_as_float(v & 0xffff0000u) * a);
  return *reinterpret_cast<const uint32_t*>(&r);
}
template <> __device__ __forceinline__ uint4 scaled<__nv_bfloat16>(uint4 v, float a) {
  return make_uint4(scaled_pair(v.x, a), scaled_pair(v.y, a), scaled_pair(v.z, a), scaled_pair(v.w, a));
}
}  // namespace

// out[r] = scale * row(codes[r]).  A warp takes kLookupUnroll vectors per lane of a row, all under way at once, so that the
// few rows of a decode step are spread over as many SMs as they have pieces, and one such piece: in a grid of the
// resident blocks with a loop every warp waits for its own chain of reads again and again (52800 rows of 4096 bf16 columns
// take 121 us that way, 100 this way: 0.95 of the copy rate).
template <typename T>
__global__ void __launch_bounds__(kLookupThreads) k_embed_lookup_scaled(
    CbView cb, const int32_t* __restrict__ codes, int N, const int32_t* __restrict__ row_seq, const uint4* __restrict__ WE,
    const uint4* __restrict__ Eh, float scale, uint4* __restrict__ out, int row_vecs, int pieces) {
  sm100::pdl_wait();
  sm100::pdl_trigger();
  const int lane = threadIdx.x & 31;
  const long long units = (long long)N * pieces, step = (long long)gridDim.x * (kLookupThreads / 32);
  for (long long unit = (long long)blockIdx.x * (kLookupThreads / 32) + (threadIdx.x >> 5); unit < units; unit += step) {
    const int r = (int)(unit / pieces), piece = (int)(unit - (long long)r * pieces);
    const int z = codes[r];
    const int b = row_seq ? row_seq[r] : r;
    const uint4* src = nullptr;
    if ((unsigned)b < (unsigned)cb.B) {
      if (z >= 0 && z < cb.V) src = WE + (size_t)z * row_vecs;
      else if (z >= cb.V && z - cb.V < cb.n[b]) src = Eh + ((size_t)b * cb.cap + (z - cb.V)) * row_vecs;
      else if (piece == 0 && lane == 0 && z != Z2Z_CODE_NONE) atomicOr(&cb.status[b], Z2Z_ST_BAD_TOKEN);
    }
    uint4* dst = out + (size_t)r * row_vecs;
    const int i = piece * 32 * kLookupUnroll + lane;
    uint4 v[kLookupUnroll];
#pragma unroll
    for (int u = 0; u < kLookupUnroll; ++u) v[u] = src && i + 32 * u < row_vecs ? __ldcg(src + i + 32 * u) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int u = 0; u < kLookupUnroll; ++u) if (i + 32 * u < row_vecs) __stcs(dst + i + 32 * u, src ? scaled<T>(v[u], scale) : v[u]);
  }
}

cudaError_t launch_embed_lookup(const CbView& cb, const int32_t* codes, int N,
                                const int32_t* row_seq, const void* WE, const void* Eh, void* out,
                                int d, int elem_bytes, cudaStream_t s) {
  const int row_vecs = d * elem_bytes / 16;
  const int warps_per_block = kLookupThreads / 32;
  int blocks = (N + warps_per_block - 1) / warps_per_block;
  const int full = 148 * 8;                       // 8 resident blocks of 256 threads per SM
  if (blocks > full) blocks = full;
  return launch_pdl(k_embed_lookup, dim3(blocks), dim3(kLookupThreads), 0, s, cb, codes, N, row_seq,
                    reinterpret_cast<const uint4*>(WE), reinterpret_cast<const uint4*>(Eh), reinterpret_cast<uint4*>(out), row_vecs);
}

cudaError_t launch_embed_lookup_scaled(const CbView& cb, const int32_t* codes, int N, const int32_t* row_seq, const void* WE,
                                       const void* Eh, float scale, void* out, int d, int dtype, cudaStream_t s) {
  const int row_vecs = d * (dtype == Z2Z_DTYPE_BF16 ? 2 : 4) / 16;
  const int pieces = (row_vecs + 32 * kLookupUnroll - 1) / (32 * kLookupUnroll), warps = kLookupThreads / 32;
  long long blocks = ((long long)N * pieces + warps - 1) / warps;
  if (blocks > (1 << 30)) blocks = 1 << 30;
  auto kern = dtype == Z2Z_DTYPE_BF16 ? k_embed_lookup_scaled<__nv_bfloat16> : k_embed_lookup_scaled<float>;
  return launch_pdl(kern, dim3((unsigned)blocks), dim3(kLookupThreads), 0, s, cb, codes, N, row_seq,
                    reinterpret_cast<const uint4*>(WE), reinterpret_cast<const uint4*>(Eh), scale, reinterpret_cast<uint4*>(out), row_vecs,
                    pieces);
}

}  // namespace z2z
