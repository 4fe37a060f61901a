// Gradient of the scaled mixed-stream lookup for its tables, by sorted tokens.
//
//   dW_E[v] (+)= scale * sum of g[r] over z_r = v,      dE_h[b][k] (+)= scale * sum over the rows of b with z_r = V + k.
//
// The rows that name one target are brought together by a stable sort of the targets' numbers (row of W_E: v; entry k
// of sequence b: V + b cap + k; a row without one: the number behind the last) and added in fp32 in the order of
// their rows, so that the result does not depend on which block ran first.  No atomics touch a gradient.
//
//   k_grad_small   few rows (few_rows below): one launch, no sort.  Every block holds all targets in shared memory; the block of
//                  a target's first row finds the others and adds them up.  (A single target for all rows is the worst case,
//                  1024 rows one after the other.)
//   k_grad_keys, k_grad_scatter (x passes), k_grad_sum, k_grad_finish otherwise:
//     * the sort has digits of 9 bits (two passes up to 2^18 targets) over at most kTiles tiles.  A pass is one
//       launch: every block sums the tiles' digit counts itself (a table of 2 KB per tile, from L2) instead of waiting
//       for a scan, and counts the next pass's digits at the places it scatters to;
//     * k_grad_sum reads g once, in sorted order, `chunk` places at a time (a group of threads takes 16 bytes of every
//       row).  A run inside a chunk is finished there; one that crosses chunks leaves partial sums, at most two per
//       chunk, which k_grad_finish adds in order: a warp for 128 columns of a run of a few chunks, a block for those of a
//       long one.  A frequent token (a fifteenth of a Zipf stream) has its thousands of rows spread over all SMs that way;
//     * the zeros of an overwriting call are written beside the sort, which leaves HBM idle, for the first targets
//       whether they are named or not, and beside the joins for the others.
// Bound by HBM: N d e bytes of g, and the tables' rows that are written.
#include "z2z_common.cuh"
#include "z2z_internal.h"
#include "z2z_sm100.cuh"

namespace z2z {

namespace {

constexpr int kSmallRows = 1024;
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits, kMaxPasses = 3;
constexpr int kTiles = 148;              // at most one block per SM and pass
constexpr int kTileRows = 1024;          // and at least so many rows for each
constexpr int kSortThreads = 512;
constexpr int kSumThreads = 128;
constexpr int kMinChunk = 8, kMaxChunk = 128, kMinGroup = 8;
constexpr int kAhead = 4;                // rows of g that a thread has under way
constexpr int kShortRun = 8;             // partial sums that one warp adds
constexpr int kFinishThreads = 256;
constexpr int kZeroPerBlock = 16;
constexpr size_t kZeroBeside = (size_t)40 << 20;     // bytes of zeros written beside each launch of the sort

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

// Lanes with the same digit as this one's (among those that have one): a vote per bit.
__device__ __forceinline__ unsigned same_digit(int dgt) {
  unsigned peers = __ballot_sync(0xffffffffu, dgt >= 0);
#pragma unroll
  for (int b = 0; b < kDigitBits; ++b) {
    const unsigned m = __ballot_sync(0xffffffffu, (dgt >> b) & 1);
    peers &= (dgt >> b) & 1 ? m : ~m;
  }
  return peers;
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

// The old values of n columns of a table's row, and out (+)= scale * acc, rounded once.
template <typename TO, int n> struct Old;
template <int n> struct Old<float, n> {
  float4 o[n / 4];
  __device__ __forceinline__ void load(const float* p) {
#pragma unroll
    for (int i = 0; i < n / 4; ++i) o[i] = reinterpret_cast<const float4*>(p)[i];
  }
  __device__ __forceinline__ void put(float* p, const float (&acc)[n], float scale, bool accumulate) const {
#pragma unroll
    for (int i = 0; i < n / 4; ++i) {
      const float* a = acc + 4 * i;
      const float4 r = accumulate ? make_float4(fmaf(a[0], scale, o[i].x), fmaf(a[1], scale, o[i].y), fmaf(a[2], scale, o[i].z), fmaf(a[3], scale, o[i].w))
                                  : make_float4(a[0] * scale, a[1] * scale, a[2] * scale, a[3] * scale);
      __stcs(reinterpret_cast<float4*>(p) + i, r);
    }
  }
};
__device__ __forceinline__ uint32_t pack(float a, float b) {
  const __nv_bfloat162 r = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&r);
}
template <int n> struct Old<__nv_bfloat16, n> {
  uint2 o[n / 4];
  __device__ __forceinline__ void load(const __nv_bfloat16* p) {
#pragma unroll
    for (int i = 0; i < n / 4; ++i) o[i] = reinterpret_cast<const uint2*>(p)[i];
  }
  __device__ __forceinline__ void put(__nv_bfloat16* p, const float (&acc)[n], float scale, bool accumulate) const {
#pragma unroll
    for (int i = 0; i < n / 4; ++i) {
      float f[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = acc[4 * i + j] * scale;
      if (accumulate) {
        const float q[4] = {__uint_as_float(o[i].x << 16), __uint_as_float(o[i].x & 0xffff0000u), __uint_as_float(o[i].y << 16), __uint_as_float(o[i].y & 0xffff0000u)};
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = fmaf(acc[4 * i + j], scale, q[j]);
      }
      __stcs(reinterpret_cast<uint2*>(p) + i, make_uint2(pack(f[0], f[1]), pack(f[2], f[3])));
    }
  }
};
template <typename TO, int n>
__device__ __forceinline__ void put(TO* p, const float (&acc)[n], float scale, bool accumulate) {
  Old<TO, n> old;
  if (accumulate) old.load(p);
  old.put(p, acc, scale, accumulate);
}

// Zeros in rows [k0, k1) of the targets (entries that a sequence has; the others are not the call's), by the whole block.
template <typename TO>
__device__ __forceinline__ void zero_rows(const CbView& cb, const GradTables& t, int k0, int k1) {
  const int lane = threadIdx.x & 31, row_vecs = (int)((size_t)t.d * sizeof(TO) / 16);
  for (int k = k0 + (int)(threadIdx.x >> 5); k < k1; k += (int)(blockDim.x >> 5)) {
    if (k >= t.V && (k - t.V) % t.cap >= cb.n[(k - t.V) / t.cap]) continue;
    uint4* out = reinterpret_cast<uint4*>(target_row<TO>(t, k));
    for (int v = lane; v < row_vecs; v += 32) __stcs(out + v, make_uint4(0u, 0u, 0u, 0u));
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

// Few rows: those whose blocks' looks at all targets, by N blocks for every slab and, half of them beside the writes, by those of
// the zeros, are fewer than 2^21.  One launch against the sort, us: 1000 rows of 512 bf16 columns 11.3 against 16.1; of 4096, 700
// rows (2.0 million looks) 14.9 against 16.4, 1000 rows (4 million) 26 against 17; overwriting 128256 + 10101 rows of 4096 with 400 / 700
// / 1000 rows (1.1 / 2.7 / 5.1 million) 177 / 179 / 191 against 181 / 181 / 182.
constexpr int kZeroTargets = 64;         // of a block of zeros
bool few_rows(int N, int slabs, int zeros) {
  return N <= kSmallRows && ((long long)N * slabs + zeros / kZeroTargets / 2) * N <= 1 << 21;
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
  int* heads;           // chunks with a run that goes on in the next one: [0], [1] the numbers of short and long runs, from
                        // [2] on the short runs' first chunks, from the end down the long runs'
  unsigned* named;      // a bit for every target that a row names
  float* part;          // [chunks][2][d]
  size_t bytes;
};
GradScratch scratch_at(char* base, int N, int d, int total) {
  GradScratch s{};
  size_t o = 0;
  auto take = [&](size_t bytes) { char* p = base + o; o = align_up(o + bytes, 256); return p; };
  // either type of g: the one with more chunks and slabs
  const SumPlan a = sum_plan(N, d, Z2Z_DTYPE_FP32), b = sum_plan(N, d, Z2Z_DTYPE_BF16);
  if (!few_rows(N, a.slabs, total)) {
    const size_t chunks = a.chunks > b.chunks ? a.chunks : b.chunks;
    s.keys = reinterpret_cast<int32_t*>(take((size_t)N * 4));
    s.pairs[0] = reinterpret_cast<int2*>(take((size_t)N * 8));
    s.pairs[1] = reinterpret_cast<int2*>(take((size_t)N * 8));
    s.hist = reinterpret_cast<int*>(take((size_t)kMaxPasses * kTiles * kDigits * 4));
    s.heads = reinterpret_cast<int*>(take((chunks + 2) * 4));
    s.named = reinterpret_cast<unsigned*>(take(((size_t)total + 31) / 32 * 4));
    s.part = reinterpret_cast<float*>(take(chunks * 2 * (size_t)d * 4));
  }
  s.bytes = o;
  return s;
}

}  // namespace

// ---- few rows ------------------------------------------------------------------------------------------
// Blocks [0, N * slabs): a row and a slab of its columns; behind them (an overwriting call) blocks of kZeroTargets targets.
template <typename TG, typename TO>
__global__ void __launch_bounds__(kSumThreads) k_grad_small(CbView cb, GradTables t, const int32_t* __restrict__ codes, int N,
                                                            const int32_t* __restrict__ row_seq, const uint4* __restrict__ g, float scale,
                                                            int accumulate, int vecs, int slabs, int per_slab, int zero_lo, int zero_hi) {
  __shared__ int key[kSmallRows], list[kSumThreads / 32][kSmallRows];
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
  const int r = unit / slabs, slab = unit % slabs, k = key[r], v = slab * per_slab + tid;
  if (k == t.total) return;
  const bool mine = tid < per_slab && v < vecs;
  // (row r itself and the old values are under way while the other rows are looked for)
  uint4 x0 = make_uint4(0u, 0u, 0u, 0u);
  Old<TO, Vec<TG>::n> old;
  TO* const out = target_row<TO>(t, k) + (size_t)v * Vec<TG>::n;
  if (mine) {
    x0 = __ldcs(g + (size_t)r * vecs + v);
    if (accumulate) old.load(out);
  }
  // the rows of this target, in order, by every warp for itself; an earlier one than r has the sum
  int n = 0;
  int* const rows = list[warp];
  for (int j0 = 0; j0 < N; j0 += 32) {
    const bool hit = j0 + lane < N && key[j0 + lane] == k;
    const unsigned m = __ballot_sync(0xffffffffu, hit);
    if (j0 + 31 < r ? m != 0u : j0 <= r && (m & ((1u << (r - j0)) - 1u)) != 0u) return;
    if (hit) rows[n + __popc(m & ((1u << lane) - 1u))] = j0 + lane;
    n += __popc(m);
  }
  __syncwarp();
  if (!mine) return;
  float acc[Vec<TG>::n] = {};
  add_vec<TG>(acc, x0);
  for (int i = 1; i < n; i += 8) {
    uint4 x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = i + u < n ? __ldcs(g + (size_t)rows[i + u] * vecs + v) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int u = 0; u < 8; ++u) if (i + u < n) add_vec<TG>(acc, x[u]);
  }
  old.put(out, acc, scale, accumulate != 0);
}

// ---- the sort ----------------------------------------------------------------------------------------------
// Blocks behind the sort's write zeros: kZeroSpan targets each, from zero_lo on.
constexpr int kZeroSpan = 32;

// Targets of all rows and the first pass's digit counts of every tile; clears the later passes' counts and the bits.
template <typename TO>
__global__ void __launch_bounds__(kSortThreads) k_grad_keys(CbView cb, GradTables t, const int32_t* __restrict__ codes, int N,
                                                            const int32_t* __restrict__ row_seq, int tile, int tiles, int passes, int n_words,
                                                            GradScratch w, int zero_lo, int zero_hi) {
  __shared__ int cnt[kDigits];
  sm100::pdl_wait();
  sm100::pdl_trigger();
  const int tid = threadIdx.x;
  if ((int)blockIdx.x >= tiles) {
    const int k0 = zero_lo + ((int)blockIdx.x - tiles) * kZeroSpan;
    zero_rows<TO>(cb, t, k0, min(zero_hi, k0 + kZeroSpan));
    return;
  }
  for (int i = tid; i < kDigits; i += kSortThreads) cnt[i] = 0;
  if (blockIdx.x == 0 && tid < 2) w.heads[tid] = 0;
  __syncthreads();
  const int r0 = blockIdx.x * tile, r1 = min(N, r0 + tile);
  for (int r = r0 + tid; r < r1; r += kSortThreads) {
    const int b = row_seq ? row_seq[r] : r;
    bool bad;
    const int k = target_of(cb, t, codes[r], b, &bad);
    if (bad) atomicOr(&cb.status[b], Z2Z_ST_BAD_TOKEN);
    w.keys[r] = k;
    atomicAdd(&cnt[k & (kDigits - 1)], 1);
  }
  for (int i = blockIdx.x * kSortThreads + tid; i < n_words; i += tiles * kSortThreads) w.named[i] = 0u;
  __syncthreads();
  for (int i = tid; i < kDigits; i += kSortThreads) {
    w.hist[(size_t)blockIdx.x * kDigits + i] = cnt[i];
    for (int p = 1; p < passes; ++p) w.hist[((size_t)p * kTiles + blockIdx.x) * kDigits + i] = 0;
  }
}

// One pass: every element goes to the place that its digit, its tile and its place in the tile give.  FIRST: the
// elements are the keys with their own places.  `next` counts the next digit at the places they go to, or is NULL.
// A thread keeps its first kHold elements, which are all of them up to kTiles * kTileRows rows, in registers.
constexpr int kHold = kTileRows / kSortThreads;
template <bool FIRST, typename TO>
__global__ void __launch_bounds__(kSortThreads) k_grad_scatter(CbView cb, GradTables t, const int32_t* __restrict__ keys, const int2* __restrict__ in,
                                                               int2* __restrict__ out, int N, int tile, int tiles, int shift,
                                                               const int* __restrict__ hist, int* __restrict__ next, int zero_lo, int zero_hi) {
  constexpr int kWarps = kSortThreads / 32;
  static_assert(kSortThreads == kDigits, "a thread per digit");
  __shared__ int s_base[kWarps][kDigits];                 // first place of a digit's elements of a warp
  __shared__ int s_warp[kWarps];
  sm100::pdl_wait();
  sm100::pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if ((int)blockIdx.x >= tiles) {
    const int k0 = zero_lo + ((int)blockIdx.x - tiles) * kZeroSpan;
    zero_rows<TO>(cb, t, k0, min(zero_hi, k0 + kZeroSpan));
    return;
  }
  // a warp's share of the tile is one range
  const int share = tile / kWarps, e0 = blockIdx.x * tile + warp * share, e1 = min(N, e0 + share);
  auto load = [&](int i) { return i >= e1 ? make_int2(-1, 0) : FIRST ? make_int2(keys[i], i) : in[i]; };
  int2 held[kHold];
#pragma unroll
  for (int u = 0; u < kHold; ++u) held[u] = load(e0 + 32 * u + lane);
  // where this tile's elements of digit `tid` begin: all elements of smaller digits, and those of this one in tiles before
  int before = 0, all = 0;
  for (int i = 0; i < tiles; i += 16) {
    int c[16];
#pragma unroll
    for (int u = 0; u < 16; ++u) c[u] = i + u < tiles ? hist[(size_t)(i + u) * kDigits + tid] : 0;
#pragma unroll
    for (int u = 0; u < 16; ++u) { all += c[u]; if (i + u < (int)blockIdx.x) before += c[u]; }
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
  // the warps' digits are counted, then placed, in order
  auto count = [&](int2 e) {
    const int dgt = e.x >= 0 ? (e.x >> shift) & (kDigits - 1) : -1;
    const unsigned peers = same_digit(dgt);
    if (dgt >= 0 && (__ffs(peers) - 1) == lane) s_base[warp][dgt] += __popc(peers);
    __syncwarp();
  };
#pragma unroll
  for (int u = 0; u < kHold; ++u) count(held[u]);
  for (int i = e0 + 32 * kHold; i < e1; i += 32) count(load(i + lane));
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWarps; ++w) { const int c = s_base[w][tid]; s_base[w][tid] = base; base += c; }
  __syncthreads();
  auto place = [&](int2 e) {
    const int dgt = e.x >= 0 ? (e.x >> shift) & (kDigits - 1) : -1;
    const unsigned peers = same_digit(dgt);
    int at = 0;
    if (dgt >= 0) at = s_base[warp][dgt] + __popc(peers & ((1u << lane) - 1u));
    __syncwarp();
    if (dgt >= 0 && (__ffs(peers) - 1) == lane) s_base[warp][dgt] += __popc(peers);
    __syncwarp();
    if (dgt >= 0) out[at] = e;
    if (next) {
      // (elements of one digit of this pass go to neighbouring places: mostly one tile, and for a frequent target one digit)
      const int to = dgt >= 0 ? at / tile * kDigits + ((e.x >> (shift + kDigitBits)) & (kDigits - 1)) : -1;
      const unsigned same = __match_any_sync(0xffffffffu, to);
      if (dgt >= 0 && (__ffs(same) - 1) == lane) atomicAdd(&next[to], __popc(same));
    }
  };
#pragma unroll
  for (int u = 0; u < kHold; ++u) place(held[u]);
  for (int i = e0 + 32 * kHold; i < e1; i += 32) place(load(i + lane));
}

// ---- sums in sorted order ----------------------------------------------------------------------------------
template <typename TG, typename TO, bool ACC>
__global__ void __launch_bounds__(kSumThreads) k_grad_sum(GradTables t, const int2* __restrict__ sorted, int N, const uint4* __restrict__ g,
                                                          float scale, SumPlan p, GradScratch w) {
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
    // the rows, and the old values where a run ends, all under way at once: loaded where they are added, each run would
    // wait for its own
    uint4 x[kAhead];
    Old<TO, kCols> old[ACC ? kAhead : 1];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const bool on = i + u < n && e[i + u].x < t.total;
      x[u] = on ? __ldcs(g + (size_t)e[i + u].y * p.vecs + v) : make_uint4(0u, 0u, 0u, 0u);
      if (ACC && on && e[i + u + 1].x != e[i + u].x) old[u].load(target_row<TO>(t, e[i + u].x) + (size_t)v * kCols);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (i + u >= n) break;
      const int k = e[i + u].x;
      if (k >= t.total) return;                            // rows without a target: the last ones
      add_vec<TG>(acc, x[u]);
      const bool ends = e[i + u + 1].x != k;
      if (!ends && i + u + 1 < n) continue;
      if (v == 0 && !goes_on) {
        if (!ACC) atomicOr(&w.named[k >> 5], 1u << (k & 31));
        if (!ends) {                                       // a run over several chunks begins: more than kShortRun?
          const long long far = (long long)(c + kShortRun) * p.chunk;
          if (far < N && sorted[far].x == k) w.heads[p.chunks + 1 - atomicAdd(&w.heads[1], 1)] = c;
          else w.heads[2 + atomicAdd(&w.heads[0], 1)] = c;
        }
      }
      if (ends && !goes_on) {
        old[ACC ? u : 0].put(target_row<TO>(t, k) + (size_t)v * kCols, acc, scale, ACC);
      } else {
        float* to = w.part + ((size_t)c * 2 + (goes_on ? 0 : 1)) * t.d + (size_t)v * kCols;
#pragma unroll
        for (int j = 0; j < kCols; j += 4) *reinterpret_cast<float4*>(to + j) = make_float4(acc[j], acc[j + 1], acc[j + 2], acc[j + 3]);
      }
      goes_on = false;
#pragma unroll
      for (int j = 0; j < kCols; ++j) acc[j] = 0.f;
    }
  }
}

// Runs over several chunks, and the zeros of an overwriting call.  A warp joins 128 columns of a run of at most
// kShortRun chunks, a block those of a longer one, every warp a share of its partial sums.
template <typename TO>
__global__ void __launch_bounds__(kFinishThreads) k_grad_finish(CbView cb, GradTables t, const int2* __restrict__ sorted, float scale, int accumulate,
                                                                int chunk, int chunks, GradScratch w, int join_blocks, int zero_lo, int zero_hi) {
  constexpr int kWarps = kFinishThreads / 32;
  __shared__ float4 s_sum[kWarps][32];
  sm100::pdl_wait();
  sm100::pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if ((int)blockIdx.x >= join_blocks) {                    // zeros in the rows of kZeroPerBlock targets that no row names
    const int t0 = zero_lo + ((int)blockIdx.x - join_blocks) * kZeroPerBlock, row_vecs = (int)((size_t)t.d * sizeof(TO) / 16);
    for (int k = t0 + warp; k < min(zero_hi, t0 + kZeroPerBlock); k += kWarps) {
      if (((w.named[k >> 5] >> (k & 31)) & 1u) || (k >= t.V && (k - t.V) % t.cap >= cb.n[(k - t.V) / t.cap])) continue;
      uint4* out = reinterpret_cast<uint4*>(target_row<TO>(t, k));
      for (int v = lane; v < row_vecs; v += 32) __stcs(out + v, make_uint4(0u, 0u, 0u, 0u));
    }
    return;
  }
  const int slabs = (t.d + 127) / 128, n_short = w.heads[0], n_long = w.heads[1];
  // the target of a run and how many chunks, from c on, hold a part of it: slot 1 of chunk c, slot 0 of the others
  auto extent = [&](int c, int& k) {
    int n = 1;
    for (;; n += 32) {
      const int i = c + n + lane;
      const int x = i < chunks ? sorted[(size_t)i * chunk].x : -1;
      if (n == 1) k = __shfl_sync(0xffffffffu, x, 0);
      const unsigned other = __ballot_sync(0xffffffffu, x != k);
      if (other) return n + __ffs(other) - 1;
    }
  };
  auto add = [&](int c, int i0, int i1, int d0) {
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = i0; i < i1; i += kShortRun) {
      float4 x[kShortRun];
#pragma unroll
      for (int u = 0; u < kShortRun; ++u)
        x[u] = i + u < i1 ? __ldcg(reinterpret_cast<const float4*>(w.part + ((size_t)(c + i + u) * 2 + (i + u == 0 ? 1 : 0)) * t.d + d0))
                          : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int u = 0; u < kShortRun; ++u) if (i + u < i1) { acc.x += x[u].x; acc.y += x[u].y; acc.z += x[u].z; acc.w += x[u].w; }
    }
    return acc;
  };
  for (int unit = blockIdx.x; unit < n_long * slabs; unit += join_blocks) {
    const int c = w.heads[chunks + 1 - unit / slabs], d0 = (unit % slabs) * 128 + 4 * lane;
    int k;
    const int n = extent(c, k), per = (n + kWarps - 1) / kWarps;
    if (d0 < t.d) s_sum[warp][lane] = add(c, min(n, warp * per), min(n, (warp + 1) * per), d0);
    __syncthreads();
    if (warp == 0 && d0 < t.d) {
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kWarps; ++i) { const float4 x = s_sum[i][lane]; sum[0] += x.x; sum[1] += x.y; sum[2] += x.z; sum[3] += x.w; }
      put(target_row<TO>(t, k) + d0, sum, scale, accumulate != 0);
    }
    __syncthreads();
  }
  for (long long unit = (long long)warp * join_blocks + blockIdx.x; unit < (long long)n_short * slabs; unit += (long long)join_blocks * kWarps) {
    const int c = w.heads[2 + unit / slabs], d0 = (int)(unit % slabs) * 128 + 4 * lane;
    int k;
    const int n = extent(c, k);
    if (d0 < t.d) {
      const float4 x = add(c, 0, n, d0);
      const float sum[4] = {x.x, x.y, x.z, x.w};
      put(target_row<TO>(t, k) + d0, sum, scale, accumulate != 0);
    }
  }
}

size_t embed_grad_scratch_bytes(const z2z_config& c, int N) {
  const size_t bytes = scratch_at(nullptr, N, c.d, c.V + c.B * c.cap).bytes;
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
  if (few_rows(a.N, p.slabs, zero_hi - zero_lo)) {
    const int blocks = a.N * p.slabs + (zero_hi - zero_lo + kZeroTargets - 1) / kZeroTargets;
    if (blocks == 0) return cudaSuccess;
    return launch_pdl(k_grad_small<TG, TO>, dim3(blocks), dim3(kSumThreads), 0, s, cb, t, a.codes, a.N, a.row_seq, g, a.scale, acc,
                      p.vecs, p.slabs, p.per_slab, zero_lo, zero_hi);
  }
  const GradScratch w = scratch_at(a.scratch, a.N, a.d, t.total);
  const SortPlan q = sort_plan(a.N, t.total);
  // zeros beside the sort: a share of the targets for each of its launches, the others beside the joins
  const int beside = (int)(kZeroBeside / ((size_t)a.d * sizeof(TO)));
  int at = zero_lo;
  auto zeros = [&]() { const int from = at; at = zero_hi - at < beside ? zero_hi : at + beside; return from; };
  auto blocks = [&](int from) { return dim3(q.tiles + (at - from + kZeroSpan - 1) / kZeroSpan); };
  int from = zeros();
  cudaError_t e = launch_pdl(k_grad_keys<TO>, blocks(from), dim3(kSortThreads), 0, s, cb, t, a.codes, a.N, a.row_seq, q.tile, q.tiles, q.passes,
                             acc ? 0 : (t.total + 31) / 32, w, from, at);
  for (int i = 0; i < q.passes && e == cudaSuccess; ++i) {
    const int* hist = w.hist + (size_t)i * kTiles * kDigits;
    int* next = i + 1 < q.passes ? w.hist + (size_t)(i + 1) * kTiles * kDigits : nullptr;
    from = zeros();
    e = launch_pdl(i == 0 ? k_grad_scatter<true, TO> : k_grad_scatter<false, TO>, blocks(from), dim3(kSortThreads), 0, s, cb, t, w.keys,
                   w.pairs[(i + 1) & 1], w.pairs[i & 1], a.N, q.tile, q.tiles, i * kDigitBits, hist, next, from, at);
  }
  const int2* sorted = w.pairs[(q.passes - 1) & 1];
  const int groups = kSumThreads / p.group;
  if (e == cudaSuccess)
    e = launch_pdl(acc ? k_grad_sum<TG, TO, true> : k_grad_sum<TG, TO, false>, dim3((unsigned)(((long long)p.chunks * p.slabs + groups - 1) / groups)), dim3(kSumThreads),
                   (size_t)groups * (p.chunk + 2) * sizeof(int2), s, t, sorted, a.N, g, a.scale, p, w);
  if (e == cudaSuccess)
  {
    const int joins = 148 * 8;
    e = launch_pdl(k_grad_finish<TO>, dim3(joins + (zero_hi - at + kZeroPerBlock - 1) / kZeroPerBlock), dim3(kFinishThreads), 0, s, cb, t, sorted, a.scale,
                   acc, p.chunk, p.chunks, w, joins, at, zero_hi);
  }
  return e;
}

}  // namespace

cudaError_t launch_embed_grad(const CbView& cb, const EmbedGradArgs& a, cudaStream_t s) {
  if (a.g_dtype == Z2Z_DTYPE_BF16)
    return a.grad_dtype == Z2Z_DTYPE_BF16 ? launch_typed<__nv_bfloat16, __nv_bfloat16>(cb, a, s) : launch_typed<__nv_bfloat16, float>(cb, a, s);
  return a.grad_dtype == Z2Z_DTYPE_BF16 ? launch_typed<float, __nv_bfloat16>(cb, a, s) : launch_typed<float, float>(cb, a, s);
}

}  // namespace z2z
