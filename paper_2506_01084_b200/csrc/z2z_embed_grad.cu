// Gradient of the scaled mixed-stream lookup for its tables, by sorted tokens.
//
//   dW_E[v] (+)= scale * sum of g[r] over z_r = v,      dE_h[b][k] (+)= scale * sum over the rows of b with z_r = V + k.
//
// The rows that name one target are brought together by a stable sort of the targets' numbers (row of W_E: v; entry k
// of sequence b: V + b cap + k; a row without one: the number behind the last) and added in fp32 in the order of
// their rows, so that the result does not depend on which block ran first.  No atomics touch a gradient.
//
//   k_grad_small   up to kSmallRows rows: one launch, no sort.  Every block holds all targets in shared memory; the block of
//                  a target's first row finds the others and adds them up.
//   k_grad_keys, k_grad_scatter (x passes), k_grad_sum, k_grad_finish otherwise:
//     * the sort has digits of 9 bits (two passes up to 2^18 targets) over at most kTiles tiles.  A pass is one
//       launch: every block sums the tiles' digit counts itself (a table of 2 KB per tile, from L2) instead of waiting
//       for a scan, and counts the next pass's digits at the places it scatters to;
//     * k_grad_sum reads g once, in sorted order, `chunk` places at a time (a group of threads takes 16 bytes of every
//       row).  A run inside a chunk is finished there; one that crosses chunks leaves partial sums, at most two per
//       chunk, which k_grad_finish adds in order.  A frequent token (a fifteenth of a Zipf stream) has its thousands of
//       rows spread over all SMs that way;
//     * k_grad_finish also writes the zeros of an overwriting call, so that the few long joins hide behind them.
// Bound by HBM: N d e bytes of g, and the tables' rows that are written.
#include "z2z_common.cuh"
#include "z2z_internal.h"
#include "z2z_sm100.cuh"

namespace z2z {

namespace {

constexpr int kSmallRows = 512;
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits, kMaxPasses = 3;
constexpr int kTiles = 148;              // at most one block per SM and pass
constexpr int kTileRows = 1024;          // and at least so many rows for each
constexpr int kSortThreads = 512;
constexpr int kSumThreads = 128;
constexpr int kMinChunk = 8, kMaxChunk = 128, kMinGroup = 8;
constexpr int kAhead = 4;                // rows of g that a thread has under way

// Where the targets' rows lie.
struct GradTables { int V, cap, B, d; void *gWE, *gEh; int total; };

template <typename T> __device__ __forceinline__ T* target_row(const GradTables& t, int k) {
  return k < t.V ? reinterpret_cast<T*>(t.gWE) + (size_t)k * t.d : reinterpret_cast<T*>(t.gEh) + (size_t)(k - t.V) * t.d;
}

// Target of a row; `total` without one.
__device__ __forceinline__ int target_of(const CbView& cb, const GradTables& t, int z, int b, bool* bad) {
  *bad = false;
  if ((unsigned)b >= (unsigned)cb.B) return t.total;
  if (z >= 0 && z < cb.V) return t.gWE ? z : t.total;
  if (z >= cb.V && z - cb.V < cb.n[b]) return t.gEh ? cb.V + b * cb.cap + (z - cb.V) : t.total;
  *bad = z != Z2Z_CODE_NONE;
  return t.total;
}

// 16 bytes of a row of g as fp32, and that many columns of a table's row.
template <typename T> struct Vec;
template <> struct Vec<float> { static constexpr int n = 4; };
template <> struct Vec<__nv_bfloat16> { static constexpr int n = 8; };

template <typename TG>
__device__ __forceinline__ void add_vec(float (&acc)[Vec<TG>::n], const uint4& v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (Vec<TG>::n == 4) acc[i % Vec<TG>::n] += __uint_as_float(w[i]);
    else { acc[(2 * i) % Vec<TG>::n] += __uint_as_float(w[i] << 16); acc[(2 * i + 1) % Vec<TG>::n] += __uint_as_float(w[i] & 0xffff0000u); }
  }
}

// out (+)= scale * acc, rounded once.
template <int n>
__device__ __forceinline__ void put(float* out, const float (&acc)[n], float scale, bool accumulate) {
#pragma unroll
  for (int i = 0; i < n; i += 4) {
    float4 o = accumulate ? *reinterpret_cast<const float4*>(out + i) : make_float4(0.f, 0.f, 0.f, 0.f);
    if (accumulate) { o.x = fmaf(acc[i], scale, o.x); o.y = fmaf(acc[i + 1], scale, o.y); o.z = fmaf(acc[i + 2], scale, o.z); o.w = fmaf(acc[i + 3], scale, o.w); }
    else { o.x = acc[i] * scale; o.y = acc[i + 1] * scale; o.z = acc[i + 2] * scale; o.w = acc[i + 3] * scale; }
    __stcs(reinterpret_cast<float4*>(out + i), o);
  }
}
__device__ __forceinline__ uint32_t pack(float a, float b) {
  const __nv_bfloat162 r = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&r);
}
template <int n>
__device__ __forceinline__ void put(__nv_bfloat16* out, const float (&acc)[n], float scale, bool accumulate) {
#pragma unroll
  for (int i = 0; i < n; i += 4) {
    uint2 o = accumulate ? *reinterpret_cast<const uint2*>(out + i) : make_uint2(0u, 0u);
    float f[4] = {__uint_as_float(o.x << 16), __uint_as_float(o.x & 0xffff0000u), __uint_as_float(o.y << 16), __uint_as_float(o.y & 0xffff0000u)};
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = accumulate ? fmaf(acc[i + j], scale, f[j]) : acc[i + j] * scale;
    o = make_uint2(pack(f[0], f[1]), pack(f[2], f[3]));
    __stcs(reinterpret_cast<uint2*>(out + i), o);
  }
}

// How k_grad_sum deals columns and places to groups of threads.
struct SumPlan { int vecs, slabs, per_slab, group, chunk, chunks; };

SumPlan sum_plan(int N, int d, int g_dtype) {
  SumPlan p{};
  p.vecs = d / (g_dtype == Z2Z_DTYPE_BF16 ? 8 : 4);
  p.slabs = (p.vecs + kSumThreads - 1) / kSumThreads;
  p.per_slab = (p.vecs + p.slabs - 1) / p.slabs;
  p.group = kMinGroup;
  while (p.group < p.per_slab) p.group *= 2;
  // Chunks as long as leaves every SM some 64 groups' worth of them: shorter ones are more partial sums
  p.chunk = kMinChunk;
  while (p.chunk < kMaxChunk && (long long)p.chunk * 148 * 64 < (long long)N * p.slabs) p.chunk *= 2;
  p.chunks = (N + p.chunk - 1) / p.chunk;
  return p;
}

struct SortPlan { int tiles, tile, passes; };
SortPlan sort_plan(int N, int total) {
  SortPlan p{};
  p.tiles = (N + kTileRows - 1) / kTileRows;
  if (p.tiles > kTiles) p.tiles = kTiles;
  if (p.tiles < 1) p.tiles = 1;
  p.tile = ((N + p.tiles - 1) / p.tiles + kSortThreads - 1) / kSortThreads * kSortThreads;
  p.tiles = (N + p.tile - 1) / p.tile;
  p.passes = 1;
  while (p.passes < kMaxPasses && total >> (kDigitBits * p.passes)) ++p.passes;
  return p;
}

struct GradScratch {
  int32_t* keys;        // [N]
  int2* pairs[2];       // [N] (target, row)
  int* hist;            // [kMaxPasses][kTiles][kDigits]
  int* heads;           // [0]: chunks with a run that goes on in the next one, their numbers from [1] on
  float* part;          // [chunks][2][d]
  size_t bytes;
};
GradScratch scratch_at(char* base, int N, int d) {
  GradScratch s{};
  size_t o = 0;
  auto take = [&](size_t bytes) { char* p = base + o; o = align_up(o + bytes, 256); return p; };
  if (N > kSmallRows) {
    // either type of g: the one with more chunks
    const SumPlan a = sum_plan(N, d, Z2Z_DTYPE_FP32), b = sum_plan(N, d, Z2Z_DTYPE_BF16);
    const size_t chunks = a.chunks > b.chunks ? a.chunks : b.chunks;
    s.keys = reinterpret_cast<int32_t*>(take((size_t)N * 4));
    s.pairs[0] = reinterpret_cast<int2*>(take((size_t)N * 8));
    s.pairs[1] = reinterpret_cast<int2*>(take((size_t)N * 8));
    s.hist = reinterpret_cast<int*>(take((size_t)kMaxPasses * kTiles * kDigits * 4));
    s.heads = reinterpret_cast<int*>(take((chunks + 1) * 4));
    s.part = reinterpret_cast<float*>(take(chunks * 2 * (size_t)d * 4));
  }
  s.bytes = o;
  return s;
}

}  // namespace

// ---- few rows ------------------------------------------------------------------------------------------
// Blocks [0, N * slabs): a row and a slab of its columns; behind them (an overwriting call) blocks of kZeroTargets targets.
constexpr int kZeroTargets = 64;
template <typename TG, typename TO>
__global__ void __launch_bounds__(kSumThreads) k_grad_small(CbView cb, GradTables t, const int32_t* __restrict__ codes, int N,
                                                            const int32_t* __restrict__ row_seq, const uint4* __restrict__ g, float scale,
                                                            int accumulate, int vecs, int slabs, int per_slab, int zero_lo, int zero_hi) {
  __shared__ int key[kSmallRows], list[kSmallRows];
  __shared__ int n_list, warp_n[kSumThreads / 32];
  __shared__ unsigned named[kZeroTargets / 32];
  sm100::pdl_wait();
  sm100::pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int unit = blockIdx.x;
  for (int r = tid; r < N; r += kSumThreads) {
    const int b = row_seq ? row_seq[r] : r;
    bool bad;
    key[r] = target_of(cb, t, codes[r], b, &bad);
    if (bad && unit == 0) atomicOr(&cb.status[b], Z2Z_ST_BAD_TOKEN);
  }
  if (tid < kZeroTargets / 32) named[tid] = 0u;
  __syncthreads();
  if (unit >= N * slabs) {                        // zeros
    const int t0 = zero_lo + (unit - N * slabs) * kZeroTargets;
    for (int r = tid; r < N; r += kSumThreads) {
      const int i = key[r] - t0;
      if (i >= 0 && i < kZeroTargets) atomicOr(&named[i >> 5], 1u << (i & 31));
    }
    __syncthreads();
    const int row_vecs = (int)((size_t)t.d * sizeof(TO) / 16);
    for (int i = warp; i < kZeroTargets && t0 + i < zero_hi; i += kSumThreads / 32) {
      const int k = t0 + i;
      if ((named[i >> 5] >> (i & 31)) & 1u) continue;
      if (k >= t.V && (k - t.V) % t.cap >= cb.n[(k - t.V) / t.cap]) continue;
      uint4* out = reinterpret_cast<uint4*>(target_row<TO>(t, k));
      for (int v = lane; v < row_vecs; v += 32) __stcs(out + v, make_uint4(0u, 0u, 0u, 0u));
    }
    return;
  }
  const int r = unit / slabs, slab = unit % slabs, k = key[r];
  if (k == t.total) return;
  // the rows of this target, in order; an earlier one than r has the sum
  if (tid == 0) n_list = 0;
  bool earlier = false;
  for (int j = tid; j < r; j += kSumThreads) earlier |= key[j] == k;
  if (__syncthreads_or(earlier)) return;
  for (int j0 = r; j0 < N; j0 += kSumThreads) {
    const bool hit = j0 + tid < N && key[j0 + tid] == k;
    const unsigned m = __ballot_sync(0xffffffffu, hit);
    if (lane == 0) warp_n[warp] = __popc(m);
    __syncthreads();
    int at = n_list, all = 0;
    for (int w = 0; w < kSumThreads / 32; ++w) { if (w < warp) at += warp_n[w]; all += warp_n[w]; }
    if (hit) list[at + __popc(m & ((1u << lane) - 1u))] = j0 + tid;
    __syncthreads();
    if (tid == 0) n_list += all;
  }
  __syncthreads();
  const int v = slab * per_slab + tid;
  if (tid >= per_slab || v >= vecs) return;
  float acc[Vec<TG>::n] = {};
  const int n = n_list;
  for (int i = 0; i < n; i += 8) {
    uint4 x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = i + u < n ? __ldcs(g + (size_t)list[i + u] * vecs + v) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int u = 0; u < 8; ++u) if (i + u < n) add_vec<TG>(acc, x[u]);
  }
  put(target_row<TO>(t, k) + (size_t)v * Vec<TG>::n, acc, scale, accumulate != 0);
}

// ---- the sort ----------------------------------------------------------------------------------------------
// Targets of all rows and the first pass's digit counts of every tile; clears the later passes' counts.
__global__ void __launch_bounds__(kSortThreads) k_grad_keys(CbView cb, GradTables t, const int32_t* __restrict__ codes, int N,
                                                            const int32_t* __restrict__ row_seq, int tile, int passes,
                                                            int32_t* __restrict__ keys, int* __restrict__ hist, int* __restrict__ heads) {
  __shared__ int cnt[kDigits];
  sm100::pdl_wait();
  sm100::pdl_trigger();
  const int tid = threadIdx.x;
  for (int i = tid; i < kDigits; i += kSortThreads) cnt[i] = 0;
  if (blockIdx.x == 0 && tid == 0) heads[0] = 0;
  __syncthreads();
  const int r0 = blockIdx.x * tile, r1 = min(N, r0 + tile);
  for (int r = r0 + tid; r < r1; r += kSortThreads) {
    const int b = row_seq ? row_seq[r] : r;
    bool bad;
    const int k = target_of(cb, t, codes[r], b, &bad);
    if (bad) atomicOr(&cb.status[b], Z2Z_ST_BAD_TOKEN);
    keys[r] = k;
    atomicAdd(&cnt[k & (kDigits - 1)], 1);
  }
  __syncthreads();
  for (int i = tid; i < kDigits; i += kSortThreads) {
    hist[(size_t)blockIdx.x * kDigits + i] = cnt[i];
    for (int p = 1; p < passes; ++p) hist[((size_t)p * kTiles + blockIdx.x) * kDigits + i] = 0;
  }
}

// One pass: every element goes to the place that its digit, its tile and its place in the tile give.  FIRST: the
// elements are the keys with their own places.  `next` counts the next digit at the places they go to, or is NULL.
template <bool FIRST>
__global__ void __launch_bounds__(kSortThreads) k_grad_scatter(const int32_t* __restrict__ keys, const int2* __restrict__ in, int2* __restrict__ out,
                                                               int N, int tile, int tiles, int shift, const int* __restrict__ hist,
                                                               int* __restrict__ next) {
  constexpr int kWarps = kSortThreads / 32;
  static_assert(kSortThreads == kDigits, "a thread per digit");
  __shared__ int s_base[kWarps][kDigits];                 // first place of a digit's elements of a warp
  __shared__ int s_warp[kWarps];
  sm100::pdl_wait();
  sm100::pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // where this tile's elements of digit `tid` begin: all elements of smaller digits, and those of this one in tiles before
  int before = 0, all = 0;
  for (int i = 0; i < tiles; i += 8) {
    int c[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) c[u] = i + u < tiles ? hist[(size_t)(i + u) * kDigits + tid] : 0;
#pragma unroll
    for (int u = 0; u < 8; ++u) { all += c[u]; if (i + u < (int)blockIdx.x) before += c[u]; }
  }
  int inc = all;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += x;
  }
  if (lane == 31) s_warp[warp] = inc;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) s_base[w][tid] = 0;
  __syncthreads();
  int base = inc - all + before;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) if (w < warp) base += s_warp[w];
  // a warp's share of the tile is one range; its digits are counted, then placed, in order
  const int share = tile / kWarps, e0 = blockIdx.x * tile + warp * share, e1 = min(N, e0 + share);
  auto load = [&](int i) { return FIRST ? make_int2(keys[i], i) : in[i]; };
  for (int i = e0; i < e1; i += 32) {
    const bool on = i + lane < e1;
    const int dgt = on ? (load(i + lane).x >> shift) & (kDigits - 1) : -1;
    const unsigned peers = __match_any_sync(0xffffffffu, dgt);
    if (on && (__ffs(peers) - 1) == lane) s_base[warp][dgt] += __popc(peers);
    __syncwarp();
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWarps; ++w) { const int c = s_base[w][tid]; s_base[w][tid] = base; base += c; }
  __syncthreads();
  for (int i = e0; i < e1; i += 32) {
    const bool on = i + lane < e1;
    const int2 e = on ? load(i + lane) : make_int2(0, 0);
    const int dgt = on ? (e.x >> shift) & (kDigits - 1) : -1;
    const unsigned peers = __match_any_sync(0xffffffffu, dgt);
    int at = 0;
    if (on) at = s_base[warp][dgt] + __popc(peers & ((1u << lane) - 1u));
    __syncwarp();
    if (on && (__ffs(peers) - 1) == lane) s_base[warp][dgt] += __popc(peers);
    __syncwarp();
    if (on) out[at] = e;
    if (next) {
      // (elements of one digit of this pass go to neighbouring places: mostly one tile, and for a frequent target one digit)
      const int to = on ? at / tile * kDigits + ((e.x >> (shift + kDigitBits)) & (kDigits - 1)) : -1;
      const unsigned same = __match_any_sync(0xffffffffu, to);
      if (on && (__ffs(same) - 1) == lane) atomicAdd(&next[to], __popc(same));
    }
  }
}

// ---- sums in sorted order ----------------------------------------------------------------------------------
template <typename TG, typename TO>
__global__ void __launch_bounds__(kSumThreads) k_grad_sum(GradTables t, const int2* __restrict__ sorted, int N, const uint4* __restrict__ g,
                                                          float scale, int accumulate, SumPlan p, int* __restrict__ heads,
                                                          float* __restrict__ part) {
  constexpr int kCols = Vec<TG>::n;
  extern __shared__ int2 s_sorted[];                       // per group: the place before its chunk, the chunk, the place behind
  sm100::pdl_wait();
  sm100::pdl_trigger();
  const int groups = kSumThreads / p.group, q = threadIdx.x / p.group, lane = threadIdx.x % p.group;
  const int unit = blockIdx.x * groups + q, c = unit / p.slabs, slab = unit % p.slabs;
  int2* const mine = s_sorted + q * (p.chunk + 2);
  const int i0 = c * p.chunk;
  for (int i = lane; i < p.chunk + 2; i += p.group) {
    const int at = i0 - 1 + i;
    mine[i] = at >= 0 && at < N && c < p.chunks ? sorted[at] : make_int2(-1, 0);
  }
  __syncthreads();
  const int v = slab * p.per_slab + lane;
  if (c >= p.chunks || lane >= p.per_slab || v >= p.vecs) return;
  const int n = min(p.chunk, N - i0);
  const int2* e = mine + 1;
  bool goes_on = e[-1].x == e[0].x;                        // the run began in an earlier chunk
  float acc[kCols] = {};
  for (int i = 0; i < n; i += kAhead) {
    uint4 x[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      x[u] = i + u < n && e[i + u].x < t.total ? __ldcs(g + (size_t)e[i + u].y * p.vecs + v) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (i + u >= n) break;
      const int k = e[i + u].x;
      if (k >= t.total) return;                            // rows without a target: the last ones
      add_vec<TG>(acc, x[u]);
      const bool ends = e[i + u + 1].x != k;
      if (!ends && i + u + 1 < n) continue;
      if (ends && !goes_on) {
        put(target_row<TO>(t, k) + (size_t)v * kCols, acc, scale, accumulate != 0);
      } else {
        float* to = part + ((size_t)c * 2 + (goes_on ? 0 : 1)) * t.d + (size_t)v * kCols;
#pragma unroll
        for (int j = 0; j < kCols; j += 4) *reinterpret_cast<float4*>(to + j) = make_float4(acc[j], acc[j + 1], acc[j + 2], acc[j + 3]);
        if (!goes_on && v == 0) heads[1 + atomicAdd(&heads[0], 1)] = c;
      }
      goes_on = false;
#pragma unroll
      for (int j = 0; j < kCols; ++j) acc[j] = 0.f;
    }
  }
}

// Runs over several chunks, and the zeros of an overwriting call.  A join takes 512 columns of one run: two halves of the
// block add half of the partial sums each, in order.
constexpr int kFinishThreads = 256;
constexpr int kZeroPerWarp = 8;
template <typename TO>
__global__ void __launch_bounds__(kFinishThreads) k_grad_finish(CbView cb, GradTables t, const int2* __restrict__ sorted, int N, float scale,
                                                                int accumulate, int chunk, int chunks, const int* __restrict__ heads,
                                                                const float* __restrict__ part, int zero_lo, int zero_hi) {
  __shared__ float4 s_half[kFinishThreads / 2];
  __shared__ int s_last;
  sm100::pdl_wait();
  sm100::pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, half = tid / (kFinishThreads / 2), col = tid % (kFinishThreads / 2);
  const int slabs = (t.d + 511) / 512, n_heads = heads[0];
  for (int unit = blockIdx.x; unit < n_heads * slabs; unit += gridDim.x) {
    const int c = heads[1 + unit / slabs], d0 = (unit % slabs) * 512 + 4 * col;
    const int k = sorted[(size_t)(c + 1) * chunk].x;      // (the run goes on there)
    if (tid == 0) s_last = chunks;
    __syncthreads();
    // the first chunk behind c whose first place is another target's
    for (int i = c + 1 + tid;; i += kFinishThreads) {
      const bool other = i < chunks && sorted[(size_t)i * chunk].x != k;
      if (other) atomicMin(&s_last, i);
      if (__syncthreads_or(other || i >= chunks)) break;
    }
    const int n = s_last - c;                             // partial sums: slot 1 of chunk c, slot 0 of the others
    const int a0 = half ? (n + 1) / 2 : 0, a1 = half ? n : (n + 1) / 2;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (d0 < t.d) {
      for (int i = a0; i < a1; i += 8) {
        float4 x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u)
          x[u] = i + u < a1 ? __ldcg(reinterpret_cast<const float4*>(part + ((size_t)(c + i + u) * 2 + (i + u == 0 ? 1 : 0)) * t.d + d0))
                            : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int u = 0; u < 8; ++u) if (i + u < a1) { acc.x += x[u].x; acc.y += x[u].y; acc.z += x[u].z; acc.w += x[u].w; }
      }
    }
    if (half) s_half[col] = acc;
    __syncthreads();
    if (!half && d0 < t.d) {
      const float4 o = s_half[col];
      const float sum[4] = {acc.x + o.x, acc.y + o.y, acc.z + o.z, acc.w + o.w};
      put(target_row<TO>(t, k) + d0, sum, scale, accumulate != 0);
    }
    __syncthreads();
  }
  if (zero_hi <= zero_lo) return;
  const int row_vecs = (int)((size_t)t.d * sizeof(TO) / 16);
  const int warps = gridDim.x * (kFinishThreads / 32);
  for (long long t0 = zero_lo + (long long)(blockIdx.x * (kFinishThreads / 32) + (tid >> 5)) * kZeroPerWarp; t0 < zero_hi; t0 += (long long)warps * kZeroPerWarp) {
    bool zero = false;
    const int k = (int)t0 + lane;
    if (lane < kZeroPerWarp && k < zero_hi && (k < t.V || (k - t.V) % t.cap < cb.n[(k - t.V) / t.cap])) {
      int lo = 0, hi = N;                                 // is there a row of target k?
      while (lo < hi) {
        const int m = (lo + hi) >> 1;
        if (sorted[m].x < k) lo = m + 1; else hi = m;
      }
      zero = lo >= N || sorted[lo].x != k;
    }
    unsigned todo = __ballot_sync(0xffffffffu, zero);
    while (todo) {
      const int i = __ffs(todo) - 1;
      todo &= todo - 1;
      uint4* out = reinterpret_cast<uint4*>(target_row<TO>(t, (int)t0 + i));
      for (int v = lane; v < row_vecs; v += 32) __stcs(out + v, make_uint4(0u, 0u, 0u, 0u));
    }
  }
}

size_t embed_grad_scratch_bytes(int N, int d) {
  const size_t bytes = scratch_at(nullptr, N, d).bytes;
  return N > 0 && bytes < 256 ? 256 : bytes;
}

namespace {

template <typename TG, typename TO>
cudaError_t launch_typed(const CbView& cb, const EmbedGradArgs& a, cudaStream_t s) {
  const GradTables t{cb.V, cb.cap, cb.B, a.d, a.gWE, a.gEh, cb.V + cb.B * cb.cap};
  const int acc = a.accumulate ? 1 : 0;
  const int zero_lo = acc ? 0 : (a.gWE ? 0 : cb.V), zero_hi = acc ? 0 : (a.gEh ? t.total : cb.V);
  const uint4* g = reinterpret_cast<const uint4*>(a.g);
  const SumPlan p = sum_plan(a.N, a.d, a.g_dtype);
  if (a.N <= kSmallRows) {
    const int blocks = a.N * p.slabs + (zero_hi - zero_lo + kZeroTargets - 1) / kZeroTargets;
    if (blocks == 0) return cudaSuccess;
    return launch_pdl(k_grad_small<TG, TO>, dim3(blocks), dim3(kSumThreads), 0, s, cb, t, a.codes, a.N, a.row_seq, g, a.scale, acc,
                      p.vecs, p.slabs, p.per_slab, zero_lo, zero_hi);
  }
  const GradScratch w = scratch_at(a.scratch, a.N, a.d);
  const SortPlan q = sort_plan(a.N, t.total);
  cudaError_t e = launch_pdl(k_grad_keys, dim3(q.tiles), dim3(kSortThreads), 0, s, cb, t, a.codes, a.N, a.row_seq, q.tile, q.passes, w.keys, w.hist, w.heads);
  for (int i = 0; i < q.passes && e == cudaSuccess; ++i) {
    const int* hist = w.hist + (size_t)i * kTiles * kDigits;
    int* next = i + 1 < q.passes ? w.hist + (size_t)(i + 1) * kTiles * kDigits : nullptr;
    e = launch_pdl(i == 0 ? k_grad_scatter<true> : k_grad_scatter<false>, dim3(q.tiles), dim3(kSortThreads), 0, s, w.keys, w.pairs[(i + 1) & 1],
                   w.pairs[i & 1], a.N, q.tile, q.tiles, i * kDigitBits, hist, next);
  }
  const int2* sorted = w.pairs[(q.passes - 1) & 1];
  const int groups = kSumThreads / p.group;
  if (e == cudaSuccess)
    e = launch_pdl(k_grad_sum<TG, TO>, dim3((unsigned)(((long long)p.chunks * p.slabs + groups - 1) / groups)), dim3(kSumThreads),
                   (size_t)groups * (p.chunk + 2) * sizeof(int2), s, t, sorted, a.N, g, a.scale, acc, p, w.heads, w.part);
  if (e == cudaSuccess)
    e = launch_pdl(k_grad_finish<TO>, dim3(148 * 8), dim3(kFinishThreads), 0, s, cb, t, sorted, a.N, a.scale, acc, p.chunk, p.chunks, w.heads, w.part,
                   zero_lo, zero_hi);
  return e;
}

}  // namespace

cudaError_t launch_embed_grad(const CbView& cb, const EmbedGradArgs& a, cudaStream_t s) {
  if (a.g_dtype == Z2Z_DTYPE_BF16)
    return a.grad_dtype == Z2Z_DTYPE_BF16 ? launch_typed<__nv_bfloat16, __nv_bfloat16>(cb, a, s) : launch_typed<__nv_bfloat16, float>(cb, a, s);
  return a.grad_dtype == Z2Z_DTYPE_BF16 ? launch_typed<float, __nv_bfloat16>(cb, a, s) : launch_typed<float, float>(cb, a, s);
}

}  // namespace z2z
