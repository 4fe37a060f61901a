// Global norm of many gradient tensors, and the tensors scaled to a largest norm.
//
//   norm = |scale| sqrt(sum over all tensors of g^2),   out = scale min(1, max_norm / (norm + 1e-6)) g
//
// Two launches: partial sums of squares, one per block; then every block adds the partial sums in the same order and
// scales its share.  Both are bound by memory: 1.9e9 bf16 elements' norm 0.63 ms, 5.9 TB/s (reads alone reach no more here);
// 3.3e8 fp32 elements to bf16 0.51 ms, 6.5 TB/s over both passes; 52 tensors of 1 MB in all 6.8 us in a graph (both passes in
// one launch, by a cluster of eight blocks that exchange their sums, took 6 to 17).  The tensors are cut into chunks of 32 KB, dealt to the blocks in turn;
// the second launch takes them from the end, where the first one's are still in L2.  Where nothing would change (in
// place, and a factor of 1) it writes nothing.
//
// Squares of 16 bytes are added in fp32 and those sums in fp64; 16 bytes whose sum of squares overflows, or is so small
// that squares may have lost bits, are scaled by a power of two and squared again, so that any finite gradient has a finite
// norm.  (In fp64 that took longer: 5.4e8 bf16 zeros,
// most of a lookup's gradient, 187 us and now 159; ordinary values 152.)
#include <cmath>

#include "z2z_common.cuh"
#include "z2z_grad_clip.h"
#include "z2z_internal.h"
#include "z2z_sm100.cuh"

namespace z2z {
using namespace sm100;

namespace {

constexpr int kClipThreads = 256;
constexpr int kVecs = 8;                         // 16-byte vectors per thread and chunk, loaded before any is used
constexpr int kChunkVecs = kClipThreads * kVecs;
constexpr int kBlocksPerSm = 4;
constexpr int kRecords = 512, kFewRecords = 64;  // tensors per launch: they are kernel parameters, which cost time to hand over

struct Record {
  const char* g;
  char* out;
  long long n;
  int first;                                     // its first chunk
  int type;                                      // bit 0: gradient is bf16, bit 1: output is
};
template <int MAX>
struct Records {
  int count, chunks;
  Record r[MAX];
};

// The tensor that holds a chunk.
template <int MAX>
__device__ __forceinline__ int record_of(const Records<MAX>& t, int chunk) {
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.r[mid].first <= chunk) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// A chunk of a tensor: whole vectors v0 .. v0 + count from the first 16-byte boundary on; the elements ahead of it go to the
// first chunk and those behind the last vector to the last one.
struct Span {
  int head;                                      // elements before the boundary
  long long v0;
  int count;                                     // vectors
  long long tail0;                               // first element of the tail, which ends with the tensor
};
__device__ __forceinline__ Span span_of(const Record& r, int chunk) {
  const int es = r.type & 1 ? 2 : 4, per = 16 / es;
  Span s;
  const int off = (int)(reinterpret_cast<uintptr_t>(r.g) & 15);
  const long long head = off ? (16 - off) / es : 0;
  s.head = (int)(head < r.n ? head : r.n);
  const long long vecs = (r.n - s.head) / per;
  s.v0 = (long long)(chunk - r.first) * kChunkVecs;
  const long long left = vecs - s.v0;
  s.count = left <= 0 ? 0 : (left < kChunkVecs ? (int)left : kChunkVecs);
  const bool last = left <= kChunkVecs && (left > 0 || chunk == r.first);
  s.tail0 = last ? s.head + vecs * per : r.n;
  if (chunk != r.first) s.head = -s.head;        // (not this chunk's)
  return s;
}

__device__ __forceinline__ float load_one(const Record& r, long long i) {
  return r.type & 1 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(r.g)[i]) : reinterpret_cast<const float*>(r.g)[i];
}
__device__ __forceinline__ void store_one(const Record& r, long long i, float x) {
  if (r.type & 2) reinterpret_cast<__nv_bfloat16*>(r.out)[i] = __float2bfloat16_rn(x);
  else reinterpret_cast<float*>(r.out)[i] = x;
}

template <bool BF16>
__device__ __forceinline__ void unpack(const uint4& v, float* x) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (BF16) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    else x[i] = __uint_as_float(w[i]);
  }
}

template <bool BF16>
__device__ __forceinline__ double squares(const uint4& v) {
  constexpr int kPer = BF16 ? 8 : 4;
  float x[kPer];
  unpack<BF16>(v, x);
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) s = fmaf(x[i], x[i], s);
  if (s > 1e-30f && s < 1e38f) return (double)s;
  // Times a power of two that brings all that counts into range: up to 1e-15, and fp32's smallest, with 2^100, and from 1e18 on with 2^-70.
  const float k = s < 1.f ? 0x1p100f : 0x1p-70f;
  float t = 0.f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) { const float y = x[i] * k; t = fmaf(y, y, t); }
  return (double)t * (s < 1.f ? 0x1p-200 : 0x1p140);
}

__device__ __forceinline__ const uint4* body(const Record& r, int head) {
  return reinterpret_cast<const uint4*>(r.g + (size_t)head * (r.type & 1 ? 2 : 4));
}

template <bool BF16>
__device__ __forceinline__ double chunk_squares(const uint4* from, int count) {
  uint4 v[kVecs];
#pragma unroll
  for (int u = 0; u < kVecs; ++u) {
    const int i = u * kClipThreads + threadIdx.x;
    v[u] = i < count ? from[i] : make_uint4(0u, 0u, 0u, 0u);
  }
  double sum = 0.0;
#pragma unroll
  for (int u = 0; u < kVecs; ++u) sum += squares<BF16>(v[u]);
  return sum;
}

// Sum over the block in an order of its own; thread 0 has it.
__device__ __forceinline__ double block_sum(double x) {
  __shared__ double s[kClipThreads / 32];
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_down_sync(0xffffffffu, x, o);
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = x;
  __syncthreads();
  if (threadIdx.x < 32) {
    x = threadIdx.x < kClipThreads / 32 ? s[threadIdx.x] : 0.0;
#pragma unroll
    for (int o = 4; o; o >>= 1) x += __shfl_down_sync(0xffffffffu, x, o);
  }
  return x;
}

template <int MAX>
__global__ void __launch_bounds__(kClipThreads, kBlocksPerSm) k_clip_norm(const __grid_constant__ Records<MAX> t, double* part) {
  pdl_wait();
  pdl_trigger();
  double sum = 0.0;
  for (int c = blockIdx.x; c < t.chunks; c += gridDim.x) {
    const Record& r = t.r[record_of(t, c)];
    const Span s = span_of(r, c);
    const uint4* from = body(r, abs(s.head)) + s.v0;
    sum += r.type & 1 ? chunk_squares<true>(from, s.count) : chunk_squares<false>(from, s.count);
    if (s.head > (int)threadIdx.x) { const double x = load_one(r, threadIdx.x); sum += x * x; }
    if (s.tail0 + threadIdx.x < r.n) { const double x = load_one(r, s.tail0 + threadIdx.x); sum += x * x; }
  }
  sum = block_sum(sum);
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// What a gradient is multiplied by: `factor`, after `pre` (1, or a power of two where the product of both is below the
// normal range, so that it keeps its bits).
struct Scale {
  float pre, factor;
  __device__ __forceinline__ float operator()(float x) const { return x * pre * factor; }
};

template <bool FROM, bool TO>
__device__ __forceinline__ void chunk_scale(const Record& r, const Span& s, const Scale& by) {
  constexpr int kPer = FROM ? 8 : 4, kOut = kPer * (TO ? 2 : 4), kAlign = kOut < 16 ? kOut : 16;
  constexpr int kBatch = 4;                      // vectors loaded before any is used
  const int head = abs(s.head);
  const uint4* from = body(r, head) + s.v0;
  char* to = r.out + (size_t)head * (TO ? 2 : 4) + s.v0 * kOut;
  const bool whole = (reinterpret_cast<uintptr_t>(to) & (kAlign - 1)) == 0;
#pragma unroll 1
  for (int i0 = threadIdx.x; i0 < s.count; i0 += kBatch * kClipThreads) {
    uint4 v[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (i0 + u * kClipThreads < s.count) v[u] = from[i0 + u * kClipThreads];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int i = i0 + u * kClipThreads;
      if (i >= s.count) break;
      float x[kPer];
      unpack<FROM>(v[u], x);
#pragma unroll
      for (int k = 0; k < kPer; ++k) x[k] = by(x[k]);
      char* at = to + (size_t)i * kOut;
      if (!whole) {
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
          if (TO) reinterpret_cast<__nv_bfloat16*>(at)[k] = __float2bfloat16_rn(x[k]);
          else reinterpret_cast<float*>(at)[k] = x[k];
        }
        continue;
      }
      uint32_t o[kOut / 4];
      if constexpr (TO) {
#pragma unroll
        for (int k = 0; k < kPer / 2; ++k) { const __nv_bfloat162 p = __floats2bfloat162_rn(x[2 * k], x[2 * k + 1]); o[k] = *reinterpret_cast<const uint32_t*>(&p); }
      } else {
#pragma unroll
        for (int k = 0; k < kPer; ++k) o[k] = __float_as_uint(x[k]);
      }
      if constexpr (kOut == 8) *reinterpret_cast<uint2*>(at) = make_uint2(o[0], o[1]);
      else {
#pragma unroll
        for (int k = 0; k < kOut / 16; ++k) reinterpret_cast<uint4*>(at)[k] = make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
      }
    }
  }
}

template <int MAX>
__global__ void __launch_bounds__(kClipThreads, kBlocksPerSm) k_clip_scale(const __grid_constant__ Records<MAX> t, const double* part, int parts, float scale, float max_norm,
                                                             float* norm_out) {
  __shared__ Scale s_by;
  __shared__ int s_write;
  pdl_wait();
  pdl_trigger();
  double sum = 0.0;
  for (int i = threadIdx.x; i < parts; i += kClipThreads) sum += part[i];
  sum = block_sum(sum);
  if (threadIdx.x == 0) {
    const float norm = (float)(fabs((double)scale) * sqrt(sum));
    if (norm_out && blockIdx.x == 0) *norm_out = norm;
    const float less = fminf(1.f, max_norm / (norm + 1e-6f));
    Scale by{1.f, scale * less};
    constexpr float kNormal = 0x1p-126f;
    if (less < kNormal || fabsf(by.factor) < kNormal) {
      // (gradients of 1e38, which a normal factor would not bring below the largest norm; 2^-100: whatever then leaves the
      // range below would be zero after the other factor, too)
      const double q = (double)scale * fmin(1.0, (double)max_norm / ((double)norm + 1e-6));
      by = fabs(q) < kNormal ? Scale{0x1p-100f, (float)(q * 0x1p100)} : Scale{1.f, (float)q};
    }
    s_by = by;
    s_write = norm < INFINITY;                   // (nor a NaN)
  }
  __syncthreads();
  if (!s_write) return;
  const Scale by = s_by;
  for (int c = t.chunks - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {
    const Record& r = t.r[record_of(t, c)];
    if (!r.out || (r.out == r.g && by.factor == 1.f)) continue;
    const Span s = span_of(r, c);
    switch (r.type) {
      case 0: chunk_scale<false, false>(r, s, by); break;
      case 1: chunk_scale<true, false>(r, s, by); break;
      case 2: chunk_scale<false, true>(r, s, by); break;
      default: chunk_scale<true, true>(r, s, by); break;
    }
    if (s.head > (int)threadIdx.x) store_one(r, threadIdx.x, by(load_one(r, threadIdx.x)));
    if (s.tail0 + threadIdx.x < r.n) store_one(r, s.tail0 + threadIdx.x, by(load_one(r, s.tail0 + threadIdx.x)));
  }
}

int clip_blocks() {
  static const int n = [] {
    int dev = 0, v = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || v <= 0) {
      cudaGetLastError();                        // (no GPU: sizes are still asked for)
      v = 148;
    }
    return kBlocksPerSm * v;
  }();
  return n;
}

int chunks_of(const z2z_grad_tensor& t) {
  const long long bytes = t.numel * (t.grad_dtype == Z2Z_DTYPE_BF16 ? 2 : 4);
  const long long c = (bytes + (long long)kChunkVecs * 16 - 1) / ((long long)kChunkVecs * 16);
  return (int)c;
}

}  // namespace

size_t grad_clip_scratch_bytes(int n) { return (size_t)((n + kRecords - 1) / kRecords) * clip_blocks() * sizeof(double); }
long long grad_clip_max_elements() { return (long long)kChunkVecs * 4 << 30; }

template <int MAX>
static cudaError_t launch_clip(const z2z_grad_tensor* t, int n, float scale, float max_norm, float* norm, double* part, cudaStream_t s) {
  const int blocks = clip_blocks();
  Records<MAX> rec;                              // filled where it is handed over, launch by launch
  auto fill = [&](int from) {
    rec.count = rec.chunks = 0;
    bool writes = false;
    for (int i = from; i < n && i < from + MAX; ++i) {
      if (t[i].numel == 0) continue;
      Record& r = rec.r[rec.count++];
      r.g = reinterpret_cast<const char*>(t[i].d_grad); r.out = reinterpret_cast<char*>(t[i].d_out); r.n = t[i].numel;
      r.first = rec.chunks;
      r.type = (t[i].grad_dtype == Z2Z_DTYPE_BF16 ? 1 : 0) | (t[i].out_dtype == Z2Z_DTYPE_BF16 ? 2 : 0);
      rec.chunks += chunks_of(t[i]);
      writes |= r.out != nullptr;
    }
    return writes;
  };
  int parts = 0;
  bool writes = false;
  for (int from = 0; from < n; from += MAX) {
    writes = fill(from);
    const int g = rec.chunks < blocks ? (rec.chunks > 0 ? rec.chunks : 1) : blocks;
    const cudaError_t e = launch_pdl(k_clip_norm<MAX>, dim3(g), dim3(kClipThreads), 0, s, rec, part + parts);
    if (e != cudaSuccess) return e;
    parts += g;
  }
  for (int from = 0; from < n || from == 0; from += MAX) {
    if (n > MAX || n == 0) writes = fill(from);
    if (!writes && from > 0) continue;
    const int g = writes ? (rec.chunks < blocks ? rec.chunks : blocks) : 1;
    if (!writes) rec.chunks = 0;
    const cudaError_t e = launch_pdl(k_clip_scale<MAX>, dim3(g), dim3(kClipThreads), 0, s, rec, part, parts, scale, max_norm, from == 0 ? norm : nullptr);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_grad_clip(const z2z_grad_tensor* t, int n, float scale, float max_norm, float* norm, double* part, cudaStream_t s) {
  return n <= kFewRecords ? launch_clip<kFewRecords>(t, n, scale, max_norm, norm, part, s) : launch_clip<kRecords>(t, n, scale, max_norm, norm, part, s);
}

}  // namespace z2z
