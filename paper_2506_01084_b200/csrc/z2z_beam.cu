// Beam search over the joint vocabularies of a session's sequences: selection and reordering.
//
// Selection: beam b offers its columns with s = score_b + (l - lse_b).  Within a beam s grows with l, so that a
// beam's best columns are its largest logits, found in fp32 without lse; s itself is taken in fp64 for those few,
// where the sum of three fp32 numbers has no rounding that could reorder beams.
//
// One launch.  A beam's columns are shared by up to 32 blocks; every block finds the `beams` best of its share:
//   1. one pass over the share with nothing but a running maximum per thread;
//   2. the `beams`-th largest of the threads' maxima bounds the best columns from below, and only the threads whose
//      maximum reaches it, `beams` of 256 unless logits are equal, have any of them: their columns are read again (from L2),
//      by a warp for each, and what reaches the bound goes to a list in shared memory;
//   3. ranks are counted among the list.
// (256 beams of 128 k columns take 32 us; where every column is offered to the list as it comes, against a bound from the first
// tile, nearly every warp has a candidate in nearly every tile: 55.)  Where the list overflows, because many
// logits are equal or the best ones lie in few threads, the bound is tightened to the `beams`-th best of what was caught, and
// step 2 done again.  The last block of a group to finish takes the best of the group's lists and deals them to the slots.
// Bound by HBM, 4 (V + n_b) bytes a beam; small calls by a chain of some ten reads, barriers and the ticket.
#include <cfloat>

#include "z2z_common.cuh"
#include "z2z_internal.h"
#include "z2z_sm100.cuh"

namespace z2z {

namespace {

constexpr int kSelThreads = 256, kSelWarps = kSelThreads / 32;
constexpr int kSelBlocks = 4;                      // on an SM
constexpr int kTileVecs = 4;                       // vectors of 4 columns that a thread has under way
constexpr int kListCap = 512;
constexpr int kMaxSplits = 32;

// A column of a beam, and a candidate of a group; `ahead` is the order that the winners come in.
struct __align__(8) BeamCand { float l; int col; };
struct GroupCand { double s; int beam; int col; float l; };
__device__ __forceinline__ bool ahead(const BeamCand& a, const BeamCand& b) { return a.l > b.l || (a.l == b.l && a.col < b.col); }
__device__ __forceinline__ bool ahead(const GroupCand& a, const GroupCand& b) {
  if (a.s != b.s) return a.s > b.s;
  if (a.beam != b.beam) return a.beam < b.beam;
  return a.l > b.l || (a.l == b.l && a.col < b.col);
}
__device__ __forceinline__ bool passes(const BeamCand& a, const BeamCand& bound) { return a.l > bound.l || (a.l == bound.l && a.col <= bound.col); }
__device__ __forceinline__ bool passes(const GroupCand& a, const GroupCand& bound) { return a.s > -INFINITY && !ahead(bound, a); }

__device__ __forceinline__ float shfl_xor(float v, int o) { return __shfl_xor_sync(0xffffffffu, v, o); }
__device__ __forceinline__ double shfl_xor(double v, int o) { return __shfl_xor_sync(0xffffffffu, v, o); }
// The k-th largest of the lanes' values.
template <typename F> __device__ __forceinline__ F kth_of_warp(F v, int k) {
  F t = v;
  for (int i = 0; i < k; ++i) {
    t = v;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) { const F x = shfl_xor(t, o); t = x > t ? x : t; }
    const unsigned at = __ballot_sync(0xffffffffu, v == t);
    if (at && (int)(threadIdx.x & 31) == __ffs(at) - 1) v = -INFINITY;
  }
  return t;
}

template <typename C> struct List {
  C* item; int* count;
  __device__ __forceinline__ void push(const C& c) const {
    const int at = atomicAdd(count, 1);
    if (at < kListCap) item[at] = c;
  }
  // By the whole block, behind a barrier: f(rank, item) for those of the first n items that have a rank below W.
  template <typename F> __device__ __forceinline__ void ranked(int n, int W, F f) const {
    for (int i = threadIdx.x; i < n; i += kSelThreads) {
      const C c = item[i];
      int rank = 0;
#pragma unroll 4
      for (int j = 0; j < n; ++j) rank += ahead(item[j], c) ? 1 : 0;
      if (rank < W) f(rank, c);
    }
  }
};

struct SelShared {
  union { BeamCand beam[kListCap]; GroupCand group[kListCap]; } list;
  GroupCand won[kMaxBeams];
  GroupCand group_bound;
  BeamCand bound;
  double warp_kth[kSelWarps];
  double score[kMaxBeams];
  float lse[kMaxBeams];
  int live[kMaxBeams];                             // 0: dead, 1: offers its columns, 2: finished, offers itself
  int hit[kSelThreads];                            // threads whose maximum reaches the bound
  int count, hits, last;
};

}  // namespace

// Grid: beams of the session x splits of a beam's columns.
__global__ void __launch_bounds__(kSelThreads, kSelBlocks) k_beam_select(CbView cb, BeamSelectArgs a, int splits, BeamCand* __restrict__ lists,
                                                             unsigned* __restrict__ tickets) {
  __shared__ SelShared sh;
  sm100::pdl_wait();
  sm100::pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int b = blockIdx.x / splits, split = blockIdx.x % splits, W = a.beams, group = b / W, g0 = group * W;
  const int per_warp = (W + kSelWarps - 1) / kSelWarps;                        // so many of every warp make W or more
  const int n_b = cb.n[b];
  if (tid < W) {
    const float score = a.scores[g0 + tid], lse = a.lse[g0 + tid];
    const int fin = a.finished ? a.finished[g0 + tid] : 0;
    sh.score[tid] = (double)score; sh.lse[tid] = lse;
    sh.live[tid] = !(score > -INFINITY) ? 0 : fin ? 2 : 1;
  }
  if (tid == 0) sh.count = sh.hits = 0;
  __syncthreads();
  auto least_of_warps = [&](double k) {
    if (lane == 0) sh.warp_kth[warp] = k;
    __syncthreads();
    double least = sh.warp_kth[0];
#pragma unroll
    for (int i = 1; i < kSelWarps; ++i) least = fmin(least, sh.warp_kth[i]);
    return least;
  };
  // ---- this block's share of the beam's columns
  if (sh.live[b - g0] == 1) {
    const float* l = a.logits + (size_t)b * ((size_t)cb.V + cb.cap);
    const int C = cb.V + n_b;
    const int off = (int)((reinterpret_cast<uintptr_t>(l) & 15) / 4), head = off ? min(C, 4 - off) : 0;
    const int vecs = (C - head) / 4, tail = C - head - 4 * vecs, share = (vecs + splits - 1) / splits;
    const int v0 = min(vecs, split * share), v1 = min(vecs, v0 + share);
    const float4* lv = reinterpret_cast<const float4*>(l + head);
    const List<BeamCand> list{sh.list.beam, &sh.count};
    // columns in front of and behind the vectors: one a thread of the first block
    auto edge_of = [&](int t) { return split != 0 ? -1 : t < head ? t : t >= 32 && t < 32 + tail ? C - tail + t - 32 : -1; };
    float top = -INFINITY;
    if (edge_of(tid) >= 0) top = fmaxf(top, l[edge_of(tid)]);
    for (int t0 = v0 + tid; t0 < v1; t0 += kSelThreads * kTileVecs) {
      float4 q[kTileVecs];
#pragma unroll
      for (int j = 0; j < kTileVecs; ++j) q[j] = t0 + j * kSelThreads < v1 ? lv[t0 + j * kSelThreads] : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
#pragma unroll
      for (int j = 0; j < kTileVecs; ++j) top = fmaxf(top, fmaxf(fmaxf(q[j].x, q[j].y), fmaxf(q[j].z, q[j].w)));
    }
    // a first bound that W threads reach, then the W-th largest maximum of those that do
    BeamCand bound{fmaxf(-FLT_MAX, (float)least_of_warps((double)kth_of_warp(top, per_warp))), 0x7fffffff};      // (-inf and NaN do not pass)
    if (top >= bound.l) list.push(BeamCand{top, tid});
    __syncthreads();
    if (sh.count > W) {
      list.ranked(sh.count, W, [&](int rank, const BeamCand& c) { if (rank == W - 1) sh.bound = c; });
      __syncthreads();
      bound.l = sh.bound.l;
    }
    __syncthreads();
    if (tid == 0) sh.count = 0;
    if (top >= bound.l) sh.hit[atomicAdd(&sh.hits, 1)] = tid;
    __syncthreads();
    const int hits = sh.hits;
    int n;
    for (;;) {
      for (int h = warp; h < hits; h += kSelWarps) {
        const int t = sh.hit[h];
        if (lane == 0 && edge_of(t) >= 0) {
          const BeamCand c{l[edge_of(t)], edge_of(t)};
          if (passes(c, bound)) list.push(c);
        }
        for (int v = v0 + t + lane * kSelThreads; v < v1; v += 32 * kSelThreads) {
          const float4 q = lv[v];
          if (fmaxf(fmaxf(q.x, q.y), fmaxf(q.z, q.w)) < bound.l) continue;
          const float x[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const BeamCand c{x[i], head + 4 * v + i};
            if (passes(c, bound)) list.push(c);
          }
        }
      }
      __syncthreads();
      n = sh.count;
      if (n <= kListCap) break;
      // (a full list holds more than W candidates, of which the new bound lets W pass: every time some 480 fewer in all)
      list.ranked(kListCap, W, [&](int rank, const BeamCand& c) { if (rank == W - 1) sh.bound = c; });
      __syncthreads();
      bound = sh.bound;
      if (tid == 0) sh.count = 0;
      __syncthreads();
    }
    BeamCand* to = lists + ((size_t)b * splits + split) * W;
    for (int i = n + tid; i < W; i += kSelThreads) __stcg(reinterpret_cast<float2*>(to + i), make_float2(-INFINITY, __int_as_float(-1)));
    list.ranked(n, W, [&](int rank, const BeamCand& c) { __stcg(reinterpret_cast<float2*>(to + rank), make_float2(c.l, __int_as_float(c.col))); });
  }
  // ---- the last block of the group deals
  __threadfence();
  __syncthreads();
  if (tid == 0) sh.last = atomicInc(tickets + group, (unsigned)(W * splits - 1)) == (unsigned)(W * splits - 1);
  __syncthreads();
  if (!sh.last) return;
  __threadfence();
  if (tid == 0) sh.count = 0;
  // Candidate i: entry i / lists of list i % lists, a list being a split of a beam.  s = -inf is none
  const int n_lists = W * splits, n_cand = n_lists * W;
  auto candidate = [&](int i) {
    const int j = i % n_lists, rank = i / n_lists;
    GroupCand c{-INFINITY, j / splits, Z2Z_CODE_NONE, 0.f};
    const int live = sh.live[c.beam];
    if (live == 2 && j % splits == 0 && rank == 0) c.s = sh.score[c.beam];
    if (live == 1) {
      const float2 q = __ldcg(reinterpret_cast<const float2*>(lists + ((size_t)g0 * splits + j) * W + rank));
      c.l = q.x; c.col = __float_as_int(q.y);
      if (c.col >= 0) c.s = sh.score[c.beam] + ((double)c.l - (double)sh.lse[c.beam]);
    }
    if (!((float)c.s > -INFINITY)) c.s = -INFINITY;                            // NaN, and what is stored as a dead slot's score
    return c;
  };
  // (the lists' best ones come first: spread over the warps they give a bound that W candidates reach)
  const int first = lane * kSelWarps + warp;
  constexpr int kMine = 4;
  GroupCand cand[kMine];
  double best = -INFINITY;
#pragma unroll
  for (int u = 0; u < kMine; ++u) {
    const int i = first + u * kSelThreads;
    cand[u] = i < n_cand ? candidate(i) : GroupCand{-INFINITY, 0, 0, 0.f};
    best = fmax(best, cand[u].s);
  }
  GroupCand bound{least_of_warps(kth_of_warp(best, per_warp)), 0x7fffffff, 0, 0.f};      // (behind every candidate of the same s)
  const List<GroupCand> list{sh.list.group, &sh.count};
  int n;
  for (;;) {
#pragma unroll
    for (int u = 0; u < kMine; ++u) if (passes(cand[u], bound)) list.push(cand[u]);
    for (int i = first + kMine * kSelThreads; i < n_cand; i += kSelThreads) {
      const GroupCand c = candidate(i);
      if (passes(c, bound)) list.push(c);
    }
    __syncthreads();
    n = sh.count;
    if (n <= kListCap) break;
    list.ranked(kListCap, W, [&](int rank, const GroupCand& c) { if (rank == W - 1) sh.group_bound = c; });
    __syncthreads();
    bound = sh.group_bound;
    if (tid == 0) sh.count = 0;
    __syncthreads();
  }
  list.ranked(n, W, [&](int rank, const GroupCand& c) { sh.won[rank] = c; });
  __syncthreads();
  if (warp != 0) return;
  // lane i: winner i, and the slot that it goes to
  const unsigned all = 0xffffffffu;
  const bool mine = lane < W, won = lane < min(n, W);
  const GroupCand c = won ? sh.won[lane] : GroupCand{-INFINITY, 64 + lane, Z2Z_CODE_NONE, 0.f};
  const bool fin = won && sh.live[c.beam] == 2;
  const unsigned peers = __match_any_sync(all, c.beam);
  const bool stays = won && (__ffs(peers) - 1) == lane;
  const unsigned taken = __reduce_or_sync(all, stays ? 1u << c.beam : 0u);
  const unsigned movers = __ballot_sync(all, mine && !stays);
  unsigned free_slots = ~taken & (W == 32 ? all : (1u << W) - 1u);
  int slot = c.beam;
  if (mine && !stays) {
    const int k = __popc(movers & ((1u << lane) - 1u));
    for (int i = 0; i < k; ++i) free_slots &= free_slots - 1u;
    slot = __ffs(free_slots) - 1;
  }
  if (mine) {
    const int o = g0 + slot;
    const bool ended = !won || fin;
    a.parent[o] = won ? g0 + c.beam : o;
    a.code[o] = c.col;
    a.next_scores[o] = (float)c.s;
    if (a.next_finished) a.next_finished[o] = ended || (a.eos >= 0 && c.col == a.eos) ? 1 : 0;
    if (a.active) a.active[o] = ended ? 0 : 1;
  }
}

// ---- reordering ---------------------------------------------------------------------------------------------
// What moves is cut into pieces of kPiece bytes, whatever it is part of, and dealt to all blocks: only the device knows
// which sequences move and how long their codebooks are, so that every block numbers the pieces for itself (two reads and a
// scan of at most 1024 sequences).  Bound by HBM, twice the bytes that move.  (96 sequences, half of
// which move, take 165 us and four 10; with sixteen blocks for every sequence of the session, most of them idle, 193 and 30.)
namespace {
constexpr int kMoveThreads = 256;
constexpr int kPiece = kMoveThreads * 4 * 16;
constexpr int kMostMoves = 1024;

// `count` pieces of 16 or 4 bytes, four under way per thread.
template <typename V>
__device__ __forceinline__ void copy_piece(V* __restrict__ dst, const V* __restrict__ src, int count) {
  int i = threadIdx.x;
  for (; i + 3 * kMoveThreads < count; i += 4 * kMoveThreads) {
    V v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = __ldcg(src + i + u * kMoveThreads);
#pragma unroll
    for (int u = 0; u < 4; ++u) __stcg(dst + i + u * kMoveThreads, v[u]);
  }
  for (; i < count; i += kMoveThreads) __stcg(dst + i, __ldcg(src + i));
}
}  // namespace

__global__ void __launch_bounds__(kMoveThreads) k_beam_reorder(CbView cb, BeamReorderArgs a) {
  __shared__ int s_to[kMostMoves], s_from[kMostMoves], s_n[kMostMoves];        // the moves
  __shared__ int s_first[kMostMoves + 1];                                      // first piece of each
  __shared__ int s_warp[2][kMoveThreads / 32];
  sm100::pdl_wait();
  sm100::pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rows0 = a.n_caches, arrays = a.n_caches + a.n_rows;                // (the hash is one of the rows)
  auto bytes_of = [&](int i, int n) { return i < rows0 ? (size_t)n * a.cache_row_bytes[i] : a.bytes[i - rows0]; };
  auto pieces_of = [&](int i, int n) { return (int)((bytes_of(i, n) + kPiece - 1) / kPiece); };
  int moves = 0, pieces = 0;
  for (int b0 = 0; b0 < cb.B; b0 += kMoveThreads) {
    const int b = b0 + tid, p = b < cb.B ? a.parent[b] : b;
    bool move = p != b;
    int n = 0, mine = 0;
    if (move) {
      if ((unsigned)p >= (unsigned)cb.B || a.parent[p] != p) {
        if (blockIdx.x == 0) atomicOr(&cb.status[b], Z2Z_ST_BAD_PARENT);
        move = false;
      } else {
        n = cb.n[p];
        for (int i = 0; i < arrays; ++i) mine += pieces_of(i, n);
      }
    }
    const unsigned m = __ballot_sync(0xffffffffu, move);
    int inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += x;
    }
    if (lane == 31) { s_warp[0][warp] = __popc(m); s_warp[1][warp] = inc; }
    __syncthreads();
    int at = moves + __popc(m & ((1u << lane) - 1u)), first = pieces + inc - mine;
    for (int w = 0; w < kMoveThreads / 32; ++w) {
      if (w < warp) { at += s_warp[0][w]; first += s_warp[1][w]; }
      moves += s_warp[0][w]; pieces += s_warp[1][w];
    }
    if (move) { s_to[at] = b; s_from[at] = p; s_n[at] = n; s_first[at] = first; }
    __syncthreads();
  }
  if (tid == 0) s_first[moves] = pieces;
  __syncthreads();
  for (int piece = blockIdx.x; piece < pieces; piece += gridDim.x) {
    int lo = 0, hi = moves;                                // the last move that begins at or before this piece and has any
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_first[mid] <= piece) lo = mid; else hi = mid;
    }
    const int to = s_to[lo], from = s_from[lo], n = s_n[lo];
    int k = piece - s_first[lo], i = 0;
    for (int q; k >= (q = pieces_of(i, n)); ++i) k -= q;
    char* base = i < rows0 ? a.cache[i] : a.rows[i - rows0];
    const size_t per = i < rows0 ? (size_t)cb.cap * a.cache_row_bytes[i] : a.stride[i - rows0];
    const size_t off = (size_t)k * kPiece, bytes = bytes_of(i, n);
    const int count = (int)(bytes - off < kPiece ? bytes - off : kPiece);
    char* dst = base + to * per + off;
    const char* src = base + from * per + off;
    if (((reinterpret_cast<uintptr_t>(dst) | reinterpret_cast<uintptr_t>(src) | (uintptr_t)count) & 15) == 0)
      copy_piece(reinterpret_cast<uint4*>(dst), reinterpret_cast<const uint4*>(src), count / 16);
    else
      copy_piece(reinterpret_cast<uint32_t*>(dst), reinterpret_cast<const uint32_t*>(src), count / 4);
  }
  // codebooks, by the blocks that have the fewest pieces; entries behind the parent's are cleared where there were more
  for (int i = (int)gridDim.x - 1 - (int)blockIdx.x; i < moves; i += gridDim.x) {
    const int b = s_to[i], p = s_from[i], rows = max(s_n[i], cb.n[b]);
    int32_t* cons = cb.cons + (size_t)b * cb.cap * cb.M;
    const int32_t* from = cb.cons + (size_t)p * cb.cap * cb.M;
    for (int v = tid; v < rows * cb.M; v += kMoveThreads) cons[v] = from[v];
    for (int v = tid; v < rows; v += kMoveThreads) cb.len[(size_t)b * cb.cap + v] = cb.len[(size_t)p * cb.cap + v];
    __syncthreads();
    if (tid == 0) {
      cb.n[b] = s_n[i]; cb.prev[b] = cb.prev[p]; cb.status[b] = cb.status[p];
      cb.n_emb[b] = cb.n_emb[p]; cb.n_emb[cb.B + b] = cb.n_emb[cb.B + p];
    }
  }
}

cudaError_t launch_beam_select(const CbView& cb, const BeamSelectArgs& a, cudaStream_t s) {
  // Blocks per beam: as many as take the fewest steps, a step being a tile of columns, when all blocks of a wave work on
  // theirs, and the bound, the second read and the ranks some two more
  const int tile = kSelThreads * kTileVecs * 4, tiles = (cb.V + cb.cap + tile - 1) / tile;
  int splits = 1;
  long long least = 0;
  for (int n = 1; n <= kMaxSplits && n <= tiles; ++n) {
    const long long waves = ((long long)cb.B * n + 148 * kSelBlocks - 1) / (148 * kSelBlocks), steps = waves * ((tiles + n - 1) / n + 2);
    if (n == 1 || steps < least) { least = steps; splits = n; }
  }
  if ((size_t)cb.B * splits * a.beams * sizeof(BeamCand) > a.lists_bytes) return cudaErrorInvalidValue;
  return launch_pdl(k_beam_select, dim3(cb.B * splits), dim3(kSelThreads), 0, s, cb, a, splits, reinterpret_cast<BeamCand*>(a.lists), a.tickets);
}

cudaError_t launch_beam_reorder(const CbView& cb, const BeamReorderArgs& a, cudaStream_t s) {
  BeamReorderArgs all = a;
  all.rows[all.n_rows] = reinterpret_cast<char*>(cb.hash);
  all.stride[all.n_rows] = all.bytes[all.n_rows] = (size_t)cb.n_slots * 8;
  ++all.n_rows;
  return launch_pdl(k_beam_reorder, dim3(148 * 8), dim3(kMoveThreads), 0, s, cb, all);
}

}  // namespace z2z
