// Beam search over the joint vocabularies of a session's sequences: selection and reordering.
//
// Selection: beam b offers its columns with s = score_b + (l - lse_b).  Within a beam s grows with l, so that a
// beam's best columns are its largest logits, found in fp32 without lse; s itself is taken in fp64 for those few,
// where the sum of three fp32 numbers has no rounding that could reorder beams.
#include "z2z_common.cuh"
#include "z2z_internal.h"
#include "z2z_sm100.cuh"

namespace z2z {

namespace {
struct __align__(8) BeamCand { float l; int col; };
// a before b in the order of a beam's columns
__device__ __forceinline__ bool ahead(float al, int ac, float bl, int bc) { return al > bl || (al == bl && ac < bc); }
}  // namespace

// One block per beam: its `beams` best columns, one after the other.  Places without a column have col = -1.
__global__ void __launch_bounds__(256) k_beam_lists(CbView cb, int W, const float* __restrict__ logits, const uint8_t* finished,
                                                    BeamCand* __restrict__ lists) {
  sm100::pdl_wait();
  sm100::pdl_trigger();
  __shared__ float s_l[8];
  __shared__ int s_c[8];
  const int b = blockIdx.x, tid = threadIdx.x;
  if (finished && finished[b]) return;
  const int C = cb.V + cb.n[b];
  const float* l = logits + (size_t)b * (cb.V + cb.cap);
  float pl = INFINITY;
  int pc = -1;
  for (int w = 0; w < W; ++w) {
    float bl = -INFINITY;
    int bc = 0x7fffffff;
    for (int c = tid; c < C; c += 256) {
      const float x = l[c];
      if (x > -INFINITY && ahead(pl, pc, x, c) && ahead(x, c, bl, bc)) { bl = x; bc = c; }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const float ol = __shfl_xor_sync(0xffffffffu, bl, o);
      const int oc = __shfl_xor_sync(0xffffffffu, bc, o);
      if (ahead(ol, oc, bl, bc)) { bl = ol; bc = oc; }
    }
    __syncthreads();
    if ((tid & 31) == 0) { s_l[tid >> 5] = bl; s_c[tid >> 5] = bc; }
    __syncthreads();
    bl = s_l[0]; bc = s_c[0];
    for (int i = 1; i < 8; ++i) if (ahead(s_l[i], s_c[i], bl, bc)) { bl = s_l[i]; bc = s_c[i]; }
    pl = bl; pc = bc;
    if (tid == 0) lists[(size_t)b * W + w] = BeamCand{bl, bc == 0x7fffffff ? -1 : bc};
    if (bc == 0x7fffffff) pl = -INFINITY;
  }
}

// One warp per group: lane i walks the list of beam i; the best head of the lists is taken W times.
__global__ void __launch_bounds__(32) k_beam_deal(CbView cb, BeamSelectArgs a, const BeamCand* __restrict__ lists) {
  sm100::pdl_wait();
  sm100::pdl_trigger();
  const unsigned all = 0xffffffffu;
  const int W = a.beams, g0 = blockIdx.x * W, lane = threadIdx.x, b = g0 + lane;
  const bool mine = lane < W;
  const float score = mine ? a.scores[b] : -INFINITY;
  const bool fin = mine && a.finished && a.finished[b];
  const double base = (double)score, lse = mine ? (double)a.lse[b] : 0.0;
  int at = 0, col = -1;
  double head = -INFINITY;
  auto next = [&]() {
    head = -INFINITY; col = -1;
    if (!mine) return;
    if (fin) { if (at == 0) head = base; }
    else if (at < W) {
      const BeamCand c = lists[(size_t)b * W + at];
      if (c.col >= 0) { head = base + ((double)c.l - lse); col = c.col; }
    }
    if (!(head > -INFINITY)) head = -INFINITY;            // NaN
  };
  next();
  int my_parent = -1, my_code = Z2Z_CODE_NONE, n_won = 0;
  double my_score = -INFINITY;
  for (int w = 0; w < W; ++w) {
    double best = head;
    int who = lane;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const double os = __shfl_xor_sync(all, best, o);
      const int ow = __shfl_xor_sync(all, who, o);
      if (os > best || (os == best && ow < who)) { best = os; who = ow; }
    }
    if (!(best > -INFINITY)) break;
    const int c = __shfl_sync(all, col, who);
    if (lane == w) { my_parent = who; my_code = c; my_score = best; }
    if (lane == who) { ++at; next(); }
    n_won = w + 1;
  }
  // the slots
  const bool won = lane < n_won;
  const unsigned peers = __match_any_sync(all, won ? my_parent : 64 + lane);
  const bool stays = won && (__ffs(peers) - 1) == lane;
  const unsigned taken = __reduce_or_sync(all, stays ? 1u << my_parent : 0u);
  const unsigned movers = __ballot_sync(all, mine && !stays);
  unsigned free_slots = ~taken & (W == 32 ? all : (1u << W) - 1u);
  int slot = my_parent;
  if (mine && !stays) {
    const int k = __popc(movers & ((1u << lane) - 1u));
    for (int i = 0; i < k; ++i) free_slots &= free_slots - 1u;
    slot = __ffs(free_slots) - 1;
  }
  const int parent_fin = __shfl_sync(all, fin ? 1 : 0, won ? my_parent : 0);
  __syncwarp();
  if (mine) {
    const int o = g0 + slot;
    a.parent[o] = won ? g0 + my_parent : o;
    a.code[o] = my_code;
    a.next_scores[o] = (float)my_score;
    const bool ended = !won || parent_fin;
    if (a.next_finished) a.next_finished[o] = ended || (a.eos >= 0 && my_code == a.eos) ? 1 : 0;
    if (a.active) a.active[o] = ended ? 0 : 1;
  }
}

// grid (slices, B): the blocks of a sequence share the rows to be copied; block 0 of them takes the codebook.
__global__ void __launch_bounds__(256) k_beam_reorder(CbView cb, BeamReorderArgs a) {
  sm100::pdl_wait();
  sm100::pdl_trigger();
  const int b = blockIdx.y, tid = threadIdx.x;
  const int p = a.parent[b];
  if (p == b) return;
  if ((unsigned)p >= (unsigned)cb.B || a.parent[p] != p) {
    if (blockIdx.x == 0 && tid == 0) atomicOr(&cb.status[b], Z2Z_ST_BAD_PARENT);
    return;
  }
  const int n = cb.n[p];
  const size_t first = (size_t)blockIdx.x * 256 + tid, step = (size_t)gridDim.x * 256;
  for (int i = 0; i < a.n_caches; ++i) {
    const size_t per = (size_t)cb.cap * a.cache_row_bytes[i], vecs = (size_t)n * a.cache_row_bytes[i] / 16;
    const uint4* src = reinterpret_cast<const uint4*>(a.cache[i] + p * per);
    uint4* dst = reinterpret_cast<uint4*>(a.cache[i] + b * per);
    for (size_t v = first; v < vecs; v += step) dst[v] = src[v];
  }
  for (int i = 0; i < a.n_rows; ++i) {
    const uint32_t* src = reinterpret_cast<const uint32_t*>(a.rows[i] + p * a.stride[i]);
    uint32_t* dst = reinterpret_cast<uint32_t*>(a.rows[i] + b * a.stride[i]);
    for (size_t v = first; v < a.bytes[i] / 4; v += step) dst[v] = src[v];
  }
  for (size_t v = first; v < (size_t)cb.n_slots; v += step) cb.hash[(size_t)b * cb.n_slots + v] = cb.hash[(size_t)p * cb.n_slots + v];
  if (blockIdx.x != 0) return;
  // entries behind the parent's are cleared where the sequence had more
  const int rows = max(n, cb.n[b]);
  for (int v = tid; v < rows * cb.M; v += 256) cb.cons[(size_t)b * cb.cap * cb.M + v] = cb.cons[(size_t)p * cb.cap * cb.M + v];
  for (int v = tid; v < rows; v += 256) cb.len[(size_t)b * cb.cap + v] = cb.len[(size_t)p * cb.cap + v];
  __syncthreads();
  if (tid == 0) {
    cb.n[b] = n; cb.prev[b] = cb.prev[p]; cb.status[b] = cb.status[p];
    cb.n_emb[b] = cb.n_emb[p]; cb.n_emb[cb.B + b] = cb.n_emb[cb.B + p];
  }
}

cudaError_t launch_beam_select(const CbView& cb, const BeamSelectArgs& a, cudaStream_t s) {
  BeamCand* lists = reinterpret_cast<BeamCand*>(a.lists);
  if ((size_t)cb.B * a.beams * sizeof(BeamCand) > a.lists_bytes) return cudaErrorInvalidValue;
  cudaError_t e = launch_pdl(k_beam_lists, dim3(cb.B), dim3(256), 0, s, cb, a.beams, a.logits, a.finished, lists);
  if (e != cudaSuccess) return e;
  return launch_pdl(k_beam_deal, dim3(cb.B / a.beams), dim3(32), 0, s, cb, a, lists);
}

cudaError_t launch_beam_reorder(const CbView& cb, const BeamReorderArgs& a, cudaStream_t s) {
  return launch_pdl(k_beam_reorder, dim3(16, cb.B), dim3(256), 0, s, cb, a);
}

}  // namespace z2z
