// Cross entropy of hidden rows over the joint vocabulary (what the model is trained on: paper Section 2.4 with the
// distribution of Section 2.3 steps 7-9), without stored logits, and its gradients.
//
//   l_rv   = h_r . W_v            v over the rows of W_U and the visible rows of U_h of the row's sequence
//   loss_r = log sum_v exp l_rv - l_rt
//   g_rv   = w_r (exp(l_rv - lse_r) - [v = t_r])
//   dh_r   = sum_v g_rv W_v       dW_v = sum_r g_rv h_r
//
// Three contractions of 2 N (V + n) d flop (the losses alone: one), all on tcgen05 with CTA pairs:
//   logits   D[v, r] = W  H^T     M = 256 vocabulary rows, N = up to 256 hidden rows, K = d
//   hidden   D[d, r] = W^T G^T    M = 256 columns,         N = up to 256 hidden rows, K = vocabulary rows
//   tables   D[v, d] = G^T H      M = 256 vocabulary rows, N = up to 256 columns,     K = hidden rows
// The vocabulary is taken in pieces: of each, G^T [v][r] is written by the epilogue of the logits, and both other
// contractions read it, with operands whose contiguous axis is the contracted one (K-major) or the other (MN-major)
// as they lie in memory: nothing is transposed.  Hidden rows are the MMA's N everywhere, so that few of them cost
// little: what is left is one pass over the tables for the logits, one for dh and the write of dW.
//
// Rows are sorted by their sequence first (stable), and rows without a target, which add nothing, are left out.
// Hypertokens are a piece per sequence: its entries against its own rows, which start at a multiple of 32 there.
//
// Numbers.  A bf16 session's g is rounded once to bf16 for gradients stored in bf16; for fp32 gradients of the tables
// it is three bf16 parts (24 bits).  An fp32 session has all operands in three parts, and takes the six products of
// parts that fp32 can hold.  Accumulators are fp32 in tensor memory.  Weights enter as w_r / max w, so that equal
// weights lose nothing to g's rounding, and the maximum multiplies the sums.  Orders of summation depend on sizes
// only: the same call gives the same bits.
#include <mutex>

#include "z2z_common.cuh"
#include "z2z_internal.h"
#include "z2z_sm100.cuh"
#include "z2z_stream.h"
#include "z2z_xent.h"

namespace z2z {
using namespace sm100;

namespace {

constexpr int kEpiWarps = 8;                     // two per tensor-memory lane quarter, which take every other 32 columns
constexpr int kThreads = 64 + 32 * kEpiWarps;
constexpr int kStages = 6;
constexpr int kTile = 256;                       // vocabulary rows or columns of a tile (128 per CTA)
constexpr int kStageBytes = 32768;               // 128 x 64 of either operand
constexpr int kMetaBytes = 2 * kTile * 16, kPartBytes = 4 * kTile * 8;
constexpr int kFrontBytes = 1024 + kMetaBytes + kPartBytes;        // a multiple of 1024
constexpr size_t kSmemBytes = 1024 + kFrontBytes + (size_t)kStages * kStageBytes;
constexpr int kHyperPad = 32;                    // a sequence's rows start at a multiple of this beside its hypertokens
constexpr int kLossRows = 8192;                  // rows whose partial sums are held at a time
constexpr int kMaxParts = 3;                     // bf16 parts of an fp32 value
constexpr int kMaxSplit = 16;
constexpr float kLog2e = 1.4426950408889634f;

struct Ctrl {
  unsigned long long full[kStages], empty[kStages], acc_full[2], acc_empty[2];
  uint32_t tmem_base;
  int abort;
};
static_assert(sizeof(Ctrl) <= 1024 && kFrontBytes % 1024 == 0, "control block");

// What the plan leaves in the scratch.
struct Plan {
  int32_t* head;             // [0] rows that take part, [1..3] jobs of hypertokens: logits, hidden, tables; [4] largest weight
  int32_t *cnt; float* wmax; // [B]
  int32_t *s0, *h0;          // [B + 1] first position of a sequence's rows, and the one beside its hypertokens
  int32_t *j1, *j2, *j3;     // [B + 1] jobs of the sequences before
  int32_t *perm, *inv;       // position -> row, row -> position or -1
  float4* meta;              // per position: lse, weight / largest, target and visible hypertokens (bits)
};

struct RowArgs {
  int N;
  const int32_t *row_seq, *row_nvis, *targets;
  const float *weight, *lse;
  float *loss_out, *lse_out;
  int th, dt;                // rows of a hypertoken tile, tiles of 256 columns
  bool hidden, tables;       // which gradients of hypertokens are wanted
};

struct Params {
  CbView cb;
  Plan pl;
  int d, dt;
  int v0, vn;                // piece: vocabulary rows v0 .. v0 + vn
  int w_row0;                // its first row in the tensor map of W
  int tr, th;                // rows per tile, and per tile of a sequence's rows
  int r_lo, r_hi;            // positions of this launch (losses: a share of the rows)
  int sb;                    // row tiles that are taken through all vocabulary tiles before the next ones
  int np1, np2, np3;         // products of parts
  int8_t a1[6], b1[6], a2[6], b2[6], a3[6], b3[6];
  bool hyper;                // with the sequences' hypertokens
  bool hyper_hidden;         // their share of dh
  int first;                 // first piece: dh's partial sums are set, not added to
  // logits
  __nv_bfloat16 *g, *gh; long long g_plane, gh_plane; int g_pitch, gh_pitch, g_parts;
  bool exact_exp;
  float2 *part, *part_h; int part_rows, part_rows_h, part0;
  float* tl;
  // gradients
  int split; long long dh_slot; float* dh;
  void *gWU, *gUh; int acc;
  int mem_cycles;            // what a tile of a table's gradient takes for its memory traffic
  int* err;
};

struct Maps {
  CUtensorMap w_k, u_k, hs_k, hh_k;              // K-major: 64 columns x 128 rows (hidden: half a tile)
  CUtensorMap w_m, u_m, ut_m, hs_m, hh_m;        // MN-major: 64 columns x 64 rows (ut: 16)
  CUtensorMap g_k, gh_k, g_m, gh_m;
};

__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

// ---- plan ------------------------------------------------------------------------------------------
struct RowState { bool mine, live, bad; int target, nvis; float w; };
__device__ __forceinline__ RowState row_state(const CbView& cb, const RowArgs& a, int r, int b) {
  RowState s{false, false, false, -1, 0, 1.f};
  if (r >= a.N) return s;
  const int seq = a.row_seq ? a.row_seq[r] : r;
  s.mine = b < cb.B ? seq == b : (seq < 0 || seq >= cb.B);
  if (!s.mine || b >= cb.B) return s;
  s.nvis = cb.n[b];
  if (a.row_nvis) { const int x = a.row_nvis[r]; s.nvis = x < s.nvis ? (x < 0 ? 0 : x) : s.nvis; }
  s.target = a.targets[r];
  s.bad = s.target != Z2Z_CODE_NONE && (s.target < 0 || s.target >= cb.V + s.nvis);
  s.live = s.target != Z2Z_CODE_NONE && !s.bad;
  if (a.weight) { s.w = a.weight[r]; if (s.w == 0.f) s.live = false; }
  return s;
}

constexpr int kScan = 8;                         // rows per lane and step: so many loads are under way

// A warp per sequence (and one for rows without): how many of its rows take part, and their largest weight.
__global__ void __launch_bounds__(128) k_xent_count(CbView cb, RowArgs a, Plan pl) {
  pdl_wait();
  pdl_trigger();
  const int b = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (b >= cb.B) return;
  int count = 0; float wmax = 0.f; bool bad = false;
  const int lo = a.row_seq ? 0 : b, hi = a.row_seq ? a.N : min(a.N, b + 1);
  for (int r0 = lo; r0 < hi; r0 += 32 * kScan) {
    RowState s[kScan];
#pragma unroll
    for (int u = 0; u < kScan; ++u) { const int r = r0 + 32 * u + lane; s[u] = row_state(cb, a, r < hi ? r : a.N, b); }
#pragma unroll
    for (int u = 0; u < kScan; ++u) {
      count += s[u].live;
      bad |= s[u].bad;
      if (s[u].live) { const float w = fabsf(s[u].w); wmax = w > wmax || w != w ? w : wmax; }
    }
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    count += __shfl_xor_sync(0xffffffffu, count, o);
    const float w = __shfl_xor_sync(0xffffffffu, wmax, o);
    wmax = w > wmax || w != w ? w : wmax;
  }
  if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(&cb.status[b], Z2Z_ST_BAD_TOKEN);
  if (lane == 0) { pl.cnt[b] = count; pl.wmax[b] = wmax; }
}

// The same warps place their rows, in order, behind those of the sequences before.
__global__ void __launch_bounds__(128) k_xent_place(CbView cb, RowArgs a, Plan pl) {
  pdl_wait();
  pdl_trigger();
  const int b = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (b > cb.B) return;
  int s0 = 0, h0 = 0, j1 = 0, j2 = 0, j3 = 0;
  float wmax = 0.f;
  for (int i = lane; i < cb.B; i += 32) {
    const float w = pl.wmax[i];
    wmax = w > wmax || w != w ? w : wmax;
    if (i >= b) continue;
    const int c = pl.cnt[i], n = cb.n[i];
    s0 += c;
    h0 += ceil_div(c, kHyperPad) * kHyperPad;
    const int rt = ceil_div(c, a.th), kt = ceil_div(n, kTile);
    j1 += rt * kt;
    if (a.hidden && n) j2 += rt * a.dt;
    if (a.tables) j3 += kt * a.dt;
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    s0 += __shfl_xor_sync(0xffffffffu, s0, o); h0 += __shfl_xor_sync(0xffffffffu, h0, o);
    j1 += __shfl_xor_sync(0xffffffffu, j1, o); j2 += __shfl_xor_sync(0xffffffffu, j2, o);
    j3 += __shfl_xor_sync(0xffffffffu, j3, o);
    const float w = __shfl_xor_sync(0xffffffffu, wmax, o);
    wmax = w > wmax || w != w ? w : wmax;
  }
  if (lane == 0) {
    pl.s0[b] = s0; pl.h0[b] = h0; pl.j1[b] = j1; pl.j2[b] = j2; pl.j3[b] = j3;
    if (b == cb.B) { pl.head[0] = s0; pl.head[1] = j1; pl.head[2] = j2; pl.head[3] = j3; pl.head[4] = __float_as_int(wmax); }
  }
  int at = s0;
  const int lo = a.row_seq || b == cb.B ? 0 : b, hi = a.row_seq ? a.N : (b == cb.B ? 0 : min(a.N, b + 1));
  for (int r0 = lo; r0 < hi; r0 += 32 * kScan) {
    RowState s[kScan];
    float lse[kScan];
#pragma unroll
    for (int u = 0; u < kScan; ++u) {
      const int r = r0 + 32 * u + lane;
      s[u] = row_state(cb, a, r < hi ? r : a.N, b);
      lse[u] = s[u].live && a.lse ? a.lse[r] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < kScan; ++u) {
      const int r = r0 + 32 * u + lane;
      const unsigned live = __ballot_sync(0xffffffffu, s[u].live);
      if (s[u].live) {
        const int p = at + __popc(live & ((1u << lane) - 1u));
        pl.perm[p] = r;
        pl.inv[r] = p;
        pl.meta[p] = make_float4(lse[u], s[u].w / wmax, __int_as_float(s[u].target), __int_as_float(s[u].nvis));
      } else if (s[u].mine) {
        pl.inv[r] = -1;
        if (a.loss_out) a.loss_out[r] = 0.f;
        if (a.lse_out) a.lse_out[r] = 0.f;
      }
      at += __popc(live);
    }
  }
}

// Sequence whose share of a prefix table holds `job`.
__device__ __forceinline__ int find_seq(const int32_t* prefix, int B, int job) {
  int lo = 0, hi = B - 1;                        // the last b with prefix[b] <= job
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (prefix[mid] <= job) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// x as the sum of bf16 values, each the rounded rest of those before.
__device__ __forceinline__ void split3(float x, __nv_bfloat16 (&p)[kMaxParts]) {
#pragma unroll
  for (int i = 0; i < kMaxParts; ++i) { p[i] = __float2bfloat16_rn(x); x -= __bfloat162float(p[i]); }
}

// A row of a matrix into bf16 (parts), zeros without one; 8 elements per thread and step.
template <typename T>
__device__ __forceinline__ void put_row(const T* src, __nv_bfloat16* dst, long long plane, int d, int tid, int threads) {
  for (int i = tid * 8; i < d; i += threads * 8) {
    if constexpr (sizeof(T) == 2) {
      uint4 v = make_uint4(0u, 0u, 0u, 0u);
      if (src) v = *reinterpret_cast<const uint4*>(src + i);
      *reinterpret_cast<uint4*>(dst + i) = v;
    } else {
      float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (src) {
        const float4 u = *reinterpret_cast<const float4*>(src + i), v = *reinterpret_cast<const float4*>(src + i + 4);
        x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w; x[4] = v.x; x[5] = v.y; x[6] = v.z; x[7] = v.w;
      }
      alignas(16) __nv_bfloat16 o[kMaxParts][8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        __nv_bfloat16 p[kMaxParts];
        split3(x[k], p);
#pragma unroll
        for (int j = 0; j < kMaxParts; ++j) o[j][k] = p[j];
      }
#pragma unroll
      for (int j = 0; j < kMaxParts; ++j) *reinterpret_cast<uint4*>(dst + (size_t)j * plane + i) = *reinterpret_cast<const uint4*>(o[j]);
    }
  }
}

struct GatherArgs {
  const void *hidden, *Uh;
  int d, positions;                              // positions: rows of the sorted copy
  __nv_bfloat16 *hs, *hh, *up, *ut;              // sorted rows; beside hypertokens; U_h in parts; its last rows
  long long hs_plane, hh_plane, up_plane, ut_plane;
};

// Hidden rows in sorted order, behind them zeros up to the next multiple of 256; the same beside their sequence's
// hypertokens, with zeros up to the next sequence.  Blocks behind them: the last n % 16 hypertokens of a sequence with
// zeros for those that do not exist (whatever lies in the cache there), and fp32 rows of U_h in parts.
template <typename T>
__global__ void __launch_bounds__(128) k_xent_gather(CbView cb, RowArgs a, Plan pl, GatherArgs g) {
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, d = g.d;
  if ((int)blockIdx.x < g.positions) {
    const int p = blockIdx.x, live = pl.head[0];
    if (p >= ceil_div(live, kTile) * kTile) return;
    const int row = p < live ? pl.perm[p] : -1;
    const T* src = row >= 0 ? reinterpret_cast<const T*>(g.hidden) + (size_t)row * d : nullptr;
    put_row(src, g.hs + (size_t)p * d, g.hs_plane, d, tid, blockDim.x);
    if (g.hh && row >= 0) {
      const int b = a.row_seq ? a.row_seq[row] : row, h = pl.h0[b] + p - pl.s0[b];
      put_row(src, g.hh + (size_t)h * d, g.hh_plane, d, tid, blockDim.x);
      if (p + 1 == pl.s0[b + 1])
        for (int i = h + 1; i < pl.h0[b + 1]; ++i) put_row<T>(nullptr, g.hh + (size_t)i * d, g.hh_plane, d, tid, blockDim.x);
    }
    return;
  }
  int i = blockIdx.x - g.positions;
  if (g.ut) {
    if (i < cb.B * 16) {
      const int b = i >> 4, n = cb.n[b], k = n / 16 * 16 + (i & 15);
      if (n % 16 == 0) return;
      put_row<T>(k < n ? reinterpret_cast<const T*>(g.Uh) + ((size_t)b * cb.cap + k) * d : nullptr, g.ut + (size_t)i * d, g.ut_plane, d, tid, blockDim.x);
      return;
    }
    i -= cb.B * 16;
  }
  const int b = i / cb.cap;
  if (i - b * cb.cap < cb.n[b]) put_row(reinterpret_cast<const T*>(g.Uh) + (size_t)i * d, g.up + (size_t)i * d, g.up_plane, d, tid, blockDim.x);
}

// Rows of an fp32 table in parts, and zeros up to the next multiple of 64 (contracted in blocks of 64).
__global__ void __launch_bounds__(128) k_xent_split(const float* __restrict__ src, __nv_bfloat16* dst, long long plane, int rows, int d) {
  pdl_wait();
  pdl_trigger();
  for (int r = blockIdx.x; r < ceil_div(rows, 64) * 64; r += gridDim.x)
    put_row(r < rows ? src + (size_t)r * d : nullptr, dst + (size_t)r * d, plane, d, threadIdx.x, blockDim.x);
}

// ---- jobs ------------------------------------------------------------------------------------------
enum JobType { kLogits, kLogitsHyper, kHidden, kHiddenHyper, kTables, kTablesHyper };
struct Job {
  int type, b;
  int m0;                    // first row of the result: vocabulary row, hypertoken or column
  int r0, n;                 // first column of the result (position, or column of the table), and how many
  int k0, k16;               // first contracted row, steps of 16
  bool tail;                 // one more step, from the copy of the last hypertokens
  int limit;                 // rows of a sequence's tile that exist (hypertokens)
  int part;                  // slot of the result
};
__device__ __forceinline__ int pad32(int n) { return (n + 31) & ~31; }

// Logits of a launch, dealt in turn: all row tiles of a share of the rows for one vocabulary tile, then the next, so
// that the clusters at work share both operands.
struct LogitsWalk {
  const Params& p;
  int c, C, idx, live, RT, VT, base, hyper;
  __device__ LogitsWalk(const Params& pp, int c_, int C_) : p(pp), c(c_), C(C_) {
    const int rows = min(p.pl.head[0], p.r_hi) - p.r_lo;
    live = rows > 0 ? rows : 0;
    RT = ceil_div(live, p.tr); VT = ceil_div(p.vn, kTile);
    base = RT * VT;
    hyper = p.hyper ? p.pl.head[1] : 0;
    idx = c;
  }
  __device__ bool next(Job& j) {
    const int at = idx;
    idx += C;
    j.tail = false; j.k0 = 0; j.k16 = ceil_div(p.d, 64) * 4;
    if (at < base) {
      const int s = at / (p.sb * VT), rem = at - s * p.sb * VT, in = min(p.sb, RT - s * p.sb), vt = rem / in;
      const int rt = s * p.sb + rem - vt * in;
      j.type = kLogits; j.b = -1; j.m0 = vt * kTile;
      j.r0 = p.r_lo + rt * p.tr;
      j.limit = min(p.tr, live - rt * p.tr);
      j.n = pad32(j.limit);
      j.part = p.part0 + 2 * vt;
      return true;
    }
    if (at - base >= hyper) return false;
    const int b = find_seq(p.pl.j1, p.cb.B, at - base), i = at - base - p.pl.j1[b];
    const int rows = p.pl.cnt[b], rt = ceil_div(rows, p.th), kt = i / rt, q = i - kt * rt;
    j.type = kLogitsHyper; j.b = b; j.m0 = kt * kTile;
    j.r0 = q * p.th;                             // (within the sequence)
    j.limit = min(p.th, rows - j.r0);
    j.n = pad32(j.limit);
    j.part = 2 * kt;
    return true;
  }
};

// Gradients of a piece.  Clusters take the tiles of dh in turn; those that are left out of the last round take tiles
// of the table's gradient meanwhile, and then all take those.
struct GradWalk {
  const Params& p;
  int c, C, live, RT, T, J2, J3, k3, rest, ahead, skip, phase, idx, jh3, jh2, kb, cost2, cost3;
  __device__ GradWalk(const Params& pp, int c_, int C_) : p(pp), c(c_), C(C_) {
    live = p.pl.head[0];
    RT = ceil_div(live, p.tr);
    T = p.dh ? RT * p.dt : 0;
    J2 = T * p.split;
    J3 = p.gWU ? ceil_div(p.vn, kTile) * p.dt : 0;
    kb = ceil_div(p.vn, 64);
    k3 = ceil_div(live, 16);
    cost2 = ceil_div(kb, p.split) * p.np2 * max(4 * 48, 2 * p.tr);
    cost3 = max(ceil_div(k3, 4) * p.np3 * 512, p.mem_cycles);
    rest = J2 % C;                               // clusters of the last round
    ahead = rest ? cost2 / cost3 : 0;
    skip = rest ? min((long long)J3, (long long)ahead * (C - rest)) : 0;
    jh3 = p.hyper && p.gUh ? p.pl.head[3] : 0;
    jh2 = p.hyper_hidden ? p.pl.head[2] : 0;
    phase = 0; idx = c;
  }
  __device__ void table_tile(Job& j, int f) {
    const int vt = f / p.dt, ct = f - vt * p.dt;
    j.type = kTables; j.b = -1; j.m0 = vt * kTile; j.r0 = ct * kTile;
    j.n = min(kTile, pad32(p.d - j.r0));
    j.k0 = 0; j.k16 = k3; j.tail = false; j.limit = 0; j.part = 0;
  }
  __device__ bool next(Job& j) {
    if (phase == 0) {
      if (idx < J2) {
        const int part = idx / T, t = idx - part * T, rt = t / p.dt;
        const int kb0 = (int)((long long)part * kb / p.split), kb1 = (int)((long long)(part + 1) * kb / p.split);
        j.type = kHidden; j.b = -1; j.m0 = (t - rt * p.dt) * kTile;
        j.r0 = rt * p.tr; j.limit = min(p.tr, live - j.r0); j.n = pad32(j.limit);
        j.k0 = kb0 * 64; j.k16 = (kb1 - kb0) * 4; j.tail = false; j.part = part;
        idx += C;
        return true;
      }
      phase = 1; idx = c - rest;
    }
    if (phase == 1) {
      if (rest && c >= rest && idx < skip) { table_tile(j, idx); idx += C - rest; return true; }
      phase = 2; idx = skip + c;
    }
    if (phase == 2) {
      if (idx < J3) { table_tile(j, idx); idx += C; return true; }
      phase = 3; idx = C - 1 - c;
    }
    const int at = idx;
    idx += C;
    if (at < jh3) {
      const int b = find_seq(p.pl.j3, p.cb.B, at), i = at - p.pl.j3[b], kt = i / p.dt;
      j.type = kTablesHyper; j.b = b; j.m0 = kt * kTile; j.r0 = (i - kt * p.dt) * kTile;
      j.n = min(kTile, pad32(p.d - j.r0));
      j.k0 = 0; j.k16 = ceil_div(p.pl.cnt[b], 16); j.tail = false; j.limit = 0; j.part = 0;
      return true;
    }
    if (at - jh3 < jh2) {
      const int b = find_seq(p.pl.j2, p.cb.B, at - jh3), i = at - jh3 - p.pl.j2[b], n = p.cb.n[b], q = i / p.dt;
      j.type = kHiddenHyper; j.b = b; j.m0 = (i - q * p.dt) * kTile;
      j.r0 = q * p.th; j.limit = min(p.th, p.pl.cnt[b] - j.r0); j.n = pad32(j.limit);
      j.k0 = 0; j.k16 = n / 16; j.tail = n % 16 != 0; j.part = p.split;
      return true;
    }
    return false;
  }
};

__device__ __forceinline__ int job_products(const Params& p, int type) {
  return type <= kLogitsHyper ? p.np1 : (type <= kHiddenHyper ? p.np2 : p.np3);
}
__device__ __forceinline__ int job_blocks(const Job& j) { return (j.k16 + 3) / 4 + (j.tail ? 1 : 0); }

// MN-major operand of 64-column boxes of 64 rows with the 128-byte swizzle: the next 8 contracted rows are 1024 bytes
// on (stride byte offset), the next 64 columns 8192 (leading byte offset).
__device__ __forceinline__ uint64_t smem_desc_mn(uint32_t addr) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(8192 >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}

// Barrier of the epilogue warps; true if `ok` was true in all their threads.
__device__ __forceinline__ bool epilogue_all(bool ok) {
  uint32_t all;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "bar.red.and.pred q, 1, %2, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(all)
      : "r"(ok ? 1u : 0u), "n"(32 * kEpiWarps)
      : "memory");
  return all != 0;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Sums over the lanes of 32 values each: lane i gets that of value i.
template <typename Op>
__device__ __forceinline__ float lanes_to_one(float (&x)[32], int lane, Op op) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const bool up = lane & o;
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const float keep = up ? x[i + o] : x[i], send = up ? x[i] : x[i + o];
      x[i] = op(keep, __shfl_xor_sync(0xffffffffu, send, o));
    }
  }
  return x[0];
}

__device__ __forceinline__ void merge_ms(float& m, float& s, float om, float os) {
  if (om == -INFINITY) return;                   // (nothing there; a NaN is in s, beside a maximum)
  if (m == -INFINITY) { m = om; s = os; return; }
  const float top = fmaxf(m, om);
  s = (m == top ? s : s * expf(m - top)) + (om == top ? os : os * expf(om - top));
  m = top;
}

enum Kind { kLoss, kGrad, kProducts };

template <int KIND, typename TO>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
k_xent(const __grid_constant__ Params p, const __grid_constant__ Maps tm) {
  using Walk = typename std::conditional<KIND == kProducts, GradWalk, LogitsWalk>::type;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* sm = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  Ctrl* ctrl = reinterpret_cast<Ctrl*>(sm);
  float4* s_meta = reinterpret_cast<float4*>(sm + 1024);
  float2* s_part = reinterpret_cast<float2*>(sm + 1024 + kMetaBytes);
  const uint32_t stage_base = smem_u32(sm + kFrontBytes);
  const int warp = uniform_warp(), lane = threadIdx.x & 31;
  const int rank = (int)cluster_ctarank();       // 0: leader (issues the MMAs), 1: peer
  const int C = gridDim.x >> 1, c = blockIdx.x >> 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) { mbar_init(smem_u32(&ctrl->full[s]), 1); mbar_init(smem_u32(&ctrl->empty[s]), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(smem_u32(&ctrl->acc_full[b]), 1); mbar_init(smem_u32(&ctrl->acc_empty[b]), 2 * kEpiWarps); }
    ctrl->abort = 0;
    mbar_init_fence();
  }
  __syncthreads();
  if (warp == 2) { tmem_alloc_pair(smem_u32(&ctrl->tmem_base), 512); tmem_relinquish_pair(); }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                            // both CTAs' barriers exist before any remote signal
  tc_fence_after();
  const uint32_t tmem_base = ctrl->tmem_base;
  pdl_wait();
  pdl_trigger();

  if (warp == 0) {
    if (lane == 0) {
      // ---------------- TMA producer (both CTAs): own 128 rows of A, own half of B's ----------------------
      const uint64_t pol = policy_evict_last();
      uint32_t full_leader[kStages];
      for (int s = 0; s < kStages; ++s) full_leader[s] = map_to_cta(smem_u32(&ctrl->full[s]), 0);
      Walk w(p, c, C);
      Job j;
      int stage = 0; uint32_t phase = 0;
      bool ok = true;
      while (ok && w.next(j)) {
        const int blocks = job_blocks(j), half = j.n >> 1, whole = (j.k16 + 3) / 4;
        const int h0 = j.b >= 0 ? p.pl.h0[j.b] : 0;
        for (int pr = 0; pr < job_products(p, j.type) && ok; ++pr) {
          for (int kb = 0; kb < blocks; ++kb) {
            if (!mbar_wait(smem_u32(&ctrl->empty[stage]), phase ^ 1u, &ctrl->abort)) { ok = false; break; }
            const uint32_t A = stage_base + (uint32_t)stage * kStageBytes, B = A + 16384u, bar = full_leader[stage];
            auto expect = [&](uint32_t bytes) { if (rank == 0) mbar_expect_tx(smem_u32(&ctrl->full[stage]), 2u * bytes); };
            if (KIND != kProducts) {
              const bool hy = j.type == kLogitsHyper;
              expect(16384u + 64u * (uint32_t)(hy ? p.th : p.tr));               // (half a tile of hidden rows, 128 bytes each)
              if (hy) {
                tma_load_3d_pair(A, &tm.u_k, kb * 64, j.b * p.cb.cap + j.m0 + rank * 128, p.a1[pr], bar, pol);
                tma_load_3d_pair(B, &tm.hh_k, kb * 64, h0 + j.r0 + rank * half, p.b1[pr], bar, pol);
              } else {
                tma_load_3d_pair(A, &tm.w_k, kb * 64, p.w_row0 + j.m0 + rank * 128, p.a1[pr], bar, pol);
                tma_load_3d_pair(B, &tm.hs_k, kb * 64, j.r0 + rank * half, p.b1[pr], bar, pol);
              }
            } else if (j.type == kHidden || j.type == kHiddenHyper) {
              const bool hy = j.type == kHiddenHyper, last = kb >= whole;
              const int nb = half > 64 ? 2 : 1;
              expect((last ? 4096u : 16384u) + 8192u * nb);
              const CUtensorMap* am = hy ? (last ? &tm.ut_m : &tm.u_m) : &tm.w_m;
              const int ay = hy ? (last ? j.b * 16 : j.b * p.cb.cap + kb * 64) : p.w_row0 + j.k0 + kb * 64;
              const CUtensorMap* bm = hy ? &tm.gh_m : &tm.g_m;
              const int by = last ? j.k16 * 16 : j.k0 + kb * 64, bx = h0 + j.r0 + rank * half;
              for (int i = 0; i < 2; ++i) tma_load_3d_pair(A + 8192u * i, am, j.m0 + rank * 128 + 64 * i, ay, p.a2[pr], bar, pol);
              for (int i = 0; i < nb; ++i) tma_load_3d_pair(B + 8192u * i, bm, bx + 64 * i, by, p.b2[pr], bar, pol);
            } else {
              const bool hy = j.type == kTablesHyper;
              const int nb = half > 64 ? 2 : 1;
              expect(16384u + 8192u * nb);
              tma_load_3d_pair(A, hy ? &tm.gh_k : &tm.g_k, h0 + kb * 64, j.m0 + rank * 128, p.a3[pr], bar, pol);
              for (int i = 0; i < nb; ++i)
                tma_load_3d_pair(B + 8192u * i, hy ? &tm.hh_m : &tm.hs_m, j.r0 + rank * half + 64 * i, h0 + kb * 64, p.b3[pr], bar, pol);
            }
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
          }
        }
      }
    }
  } else if (warp == 1) {
    if (rank == 0) {
      // ---------------- MMA issuer (leader only, the whole warp: elect_one()) ------------------------------
      Walk w(p, c, C);
      Job j;
      int stage = 0; uint32_t phase = 0, job_i = 0;
      bool ok = true;
      while (ok && w.next(j)) {
        const int blocks = job_blocks(j), products = job_products(p, j.type), whole = (j.k16 + 3) / 4;
        if (blocks == 0) continue;               // (nothing to contract: the epilogue writes zeros)
        const uint32_t buf = job_i & 1u, aph = (job_i >> 1) & 1u;
        if (!mbar_wait_warp(smem_u32(&ctrl->acc_empty[buf]), aph ^ 1u, &ctrl->abort)) { ok = false; break; }
        tc_fence_after();
        const bool a_mn = j.type == kHidden || j.type == kHiddenHyper, b_mn = KIND == kProducts;
        const uint32_t idesc = idesc_bf16_f32(kTile, j.n) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u);
        const uint32_t D = tmem_base + buf * kTile;
        uint32_t acc = 0;
        for (int pr = 0; pr < products && ok; ++pr) {
          for (int kb = 0; kb < blocks; ++kb) {
            if (!mbar_wait_warp(smem_u32(&ctrl->full[stage]), phase, &ctrl->abort)) { ok = false; break; }
            tc_fence_after();
            const uint32_t A = stage_base + (uint32_t)stage * kStageBytes, B = A + 16384u;
            const int steps = kb >= whole ? 1 : min(4, j.k16 - 4 * kb);
            if (elect_one()) {
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                if (k < steps)
                  umma_bf16_pair(D, KIND == kProducts && a_mn ? smem_desc_mn(A + k * 2048) : smem_desc_sw128(A + k * 32),
                                 b_mn ? smem_desc_mn(B + k * 2048) : smem_desc_sw128(B + k * 32), idesc, k ? 1u : acc);
              }
              umma_commit_pair(smem_u32(&ctrl->empty[stage]));
            }
            __syncwarp();
            acc = 1;
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
          }
        }
        if (!ok) break;
        if (elect_one()) umma_commit_pair(smem_u32(&ctrl->acc_full[buf]));
        __syncwarp();
        ++job_i;
      }
    }
  } else {
    // ---------------- epilogue (both CTAs): thread = row of the result (x every other 32 columns) -----------
    const int q = warp & 3, half = (warp - 2) >> 2, et = threadIdx.x - 64;
    const int in_tile = rank * 128 + q * 32 + lane;
    uint32_t acc_empty_leader[2];
    acc_empty_leader[0] = map_to_cta(smem_u32(&ctrl->acc_empty[0]), 0);
    acc_empty_leader[1] = map_to_cta(smem_u32(&ctrl->acc_empty[1]), 0);
    const float scale = __int_as_float(p.pl.head[4]);
    Walk w(p, c, C);
    Job j;
    uint32_t job_i = 0;
    bool ok = true;
    while (ok && w.next(j)) {
      const bool some = job_blocks(j) > 0;
      const uint32_t buf = job_i & 1u, aph = (job_i >> 1) & 1u;
      const uint32_t tbase = tmem_base + ((uint32_t)(q * 32) << 16) + buf * kTile;
      if constexpr (KIND != kProducts) {
        // what the tile's hidden rows are; the buffer of the job before last is free once all are at this job
        float4* meta = s_meta + (job_i & 1u) * kTile;
        const int pos0 = j.b >= 0 ? p.pl.s0[j.b] + j.r0 : j.r0;
        if (et < j.n) meta[et] = et < j.limit ? p.pl.meta[pos0 + et] : make_float4(0.f, 0.f, __int_as_float(-1), __int_as_float(-1));
        ok = mbar_wait(smem_u32(&ctrl->acc_full[buf]), aph, &ctrl->abort);
        ok = epilogue_all(ok);
        if (!ok) break;
        tc_fence_after();
        const int m = j.m0 + in_tile, limit = j.b >= 0 ? p.cb.n[j.b] : p.vn;       // row of the piece, or hypertoken
        const int id = j.b >= 0 ? p.cb.V + m : p.v0 + m;
        const bool there = m < limit;
        for (int c0 = 32 * half; c0 < j.n; c0 += 64) {
          uint32_t v[32];
          tmem_ld32(tbase + c0, v);
          tmem_ld_wait();
          if constexpr (KIND == kGrad) {
            const long long row = j.b >= 0 ? (long long)m * p.gh_pitch + p.pl.h0[j.b] + j.r0 + c0 : (long long)m * p.g_pitch + j.r0 + c0;
            __nv_bfloat16* out = (j.b >= 0 ? p.gh : p.g) + row;
            const long long plane = j.b >= 0 ? p.gh_plane : p.g_plane;
#pragma unroll
            for (int x = 0; x < 32; ++x) {
              const float4 r = meta[c0 + x];
              const float l = __uint_as_float(v[x]);
              const float e = p.exact_exp ? expf(l - r.x) : ex2((l - r.x) * kLog2e);
              const bool sees = there && r.y != 0.f && (j.b < 0 || m < __float_as_int(r.w));
              v[x] = __float_as_uint(sees ? r.y * (e - (__float_as_int(r.z) == id ? 1.f : 0.f)) : 0.f);
            }
            for (int part = 0; part < p.g_parts; ++part) {
              uint32_t o[16];
#pragma unroll
              for (int x = 0; x < 16; ++x) {
                const __nv_bfloat162 t = __floats2bfloat162_rn(__uint_as_float(v[2 * x]), __uint_as_float(v[2 * x + 1]));
                o[x] = *reinterpret_cast<const uint32_t*>(&t);
                if (part + 1 < p.g_parts) {
                  v[2 * x] = __float_as_uint(__uint_as_float(v[2 * x]) - __low2float(t));
                  v[2 * x + 1] = __float_as_uint(__uint_as_float(v[2 * x + 1]) - __high2float(t));
                }
              }
#pragma unroll
              for (int x = 0; x < 4; ++x)
                *reinterpret_cast<uint4*>(out + (size_t)part * plane + 8 * x) = make_uint4(o[4 * x], o[4 * x + 1], o[4 * x + 2], o[4 * x + 3]);
            }
          } else {
            // Sum of exponentials of 32 vocabulary rows for each of 32 hidden rows.  One reference for all of them
            // while their logits are within 40 of another: the lanes' values are then reduced once, otherwise
            // the maxima of the hidden rows are found first.
            float x[32], top = -INFINITY, low = INFINITY;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              const float4 r = meta[c0 + i];
              const float l = __uint_as_float(v[i]);
              if (there && __float_as_int(r.z) == id) p.tl[pos0 + c0 + i] = l;
              const bool sees = there && (j.b < 0 ? c0 + i < j.limit : m < __float_as_int(r.w));
              x[i] = sees ? l : -INFINITY;
              top = sees ? fmaxf(top, l) : top;
              low = sees ? fminf(low, l) : low;
            }
            bool odd = false;
#pragma unroll
            for (int i = 0; i < 32; ++i) odd |= x[i] != x[i] || x[i] == INFINITY;
#pragma unroll
            for (int o = 16; o; o >>= 1) {
              top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
              low = fminf(low, __shfl_xor_sync(0xffffffffu, low, o));
            }
            odd = __any_sync(0xffffffffu, odd);
            float ref;                                                           // of hidden row c0 + lane
            if (!odd && (top == -INFINITY || top - low < 40.f)) {
              ref = top;
#pragma unroll
              for (int i = 0; i < 32; ++i) x[i] = top == -INFINITY ? 0.f : ex2((x[i] - top) * kLog2e);
            } else {
              float y[32];
#pragma unroll
              for (int i = 0; i < 32; ++i) y[i] = x[i] != x[i] ? INFINITY : x[i];
              ref = lanes_to_one(y, lane, [](float a, float b) { return fmaxf(a, b); });
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                const float r = __shfl_sync(0xffffffffu, ref, i);
                x[i] = r == -INFINITY ? 0.f : ex2((x[i] - r) * kLog2e);                     // (+inf: inf - inf, a NaN in the sum)
              }
            }
            const float s = lanes_to_one(x, lane, [](float a, float b) { return a + b; });
            s_part[q * kTile + c0 + lane] = make_float2(ref, s);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(acc_empty_leader[buf]);
        if constexpr (KIND == kLoss) {
          epilogue_all(true);
          if (et < j.limit) {
            float m_ = -INFINITY, s_ = 0.f;
            for (int i = 0; i < 4; ++i) { const float2 v = s_part[i * kTile + et]; merge_ms(m_, s_, v.x, v.y); }
            float2* out = j.b >= 0 ? p.part_h + (size_t)(j.part + rank) * p.part_rows_h + pos0 + et
                                   : p.part + (size_t)(j.part + rank) * p.part_rows + pos0 - p.r_lo + et;
            *out = make_float2(m_, s_);
          }
        }
        ++job_i;
      } else {
        if (some) {
          if (!mbar_wait(smem_u32(&ctrl->acc_full[buf]), aph, &ctrl->abort)) { ok = false; break; }
          __syncwarp();
          tc_fence_after();
        }
        const int m = j.m0 + in_tile;
        if (j.type == kHidden || j.type == kHiddenHyper) {
          const bool set = p.first || j.type == kHiddenHyper;
          const int pos0 = j.b >= 0 ? p.pl.s0[j.b] + j.r0 : j.r0;
          float* out = p.dh + (size_t)j.part * p.dh_slot + (size_t)pos0 * p.d + m;
          for (int c0 = 32 * half; c0 < j.n && (some || set); c0 += 64) {
            uint32_t v[32];
            if (some) { tmem_ld32(tbase + c0, v); tmem_ld_wait(); }
            if (m >= p.d) continue;
            float old[32];
#pragma unroll
            for (int x = 0; x < 32; ++x) {
              if (!some) v[x] = 0u;
              old[x] = !set && c0 + x < j.limit ? out[(size_t)(c0 + x) * p.d] : 0.f;
            }
#pragma unroll
            for (int x = 0; x < 32; ++x)
              if (c0 + x < j.limit) out[(size_t)(c0 + x) * p.d] = old[x] + __uint_as_float(v[x]);
          }
        } else if (some || !p.acc) {
          const int rows = j.b >= 0 ? p.cb.n[j.b] : p.vn;
          TO* out = j.b >= 0 ? reinterpret_cast<TO*>(p.gUh) + ((size_t)j.b * p.cb.cap + m) * p.d + j.r0
                             : reinterpret_cast<TO*>(p.gWU) + (size_t)(p.v0 + m) * p.d + j.r0;
          const int cols = min(j.n, p.d - j.r0);
          for (int c0 = 32 * half; c0 < cols; c0 += 64) {
            uint32_t v[32];
            if (some) { tmem_ld32(tbase + c0, v); tmem_ld_wait(); }
            if (m >= rows) continue;
#pragma unroll
            for (int x = 0; x < 32; x += 8) {
              if (c0 + x >= cols) break;         // (columns come in eights)
              float r[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) r[i] = some ? scale * __uint_as_float(v[x + i]) : 0.f;
              TO* to = out + c0 + x;
              if constexpr (sizeof(TO) == 4) {
                float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
                if (p.acc) { a = *reinterpret_cast<const float4*>(to); b = *reinterpret_cast<const float4*>(to + 4); }
                *reinterpret_cast<float4*>(to) = make_float4(a.x + r[0], a.y + r[1], a.z + r[2], a.w + r[3]);
                *reinterpret_cast<float4*>(to + 4) = make_float4(b.x + r[4], b.y + r[5], b.z + r[6], b.w + r[7]);
              } else {
                uint4 o = make_uint4(0u, 0u, 0u, 0u);
                if (p.acc) o = *reinterpret_cast<const uint4*>(to);
                uint32_t* ow = reinterpret_cast<uint32_t*>(&o);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const __nv_bfloat162 before = *reinterpret_cast<const __nv_bfloat162*>(&ow[i]);
                  const __nv_bfloat162 t = __floats2bfloat162_rn(__low2float(before) + r[2 * i], __high2float(before) + r[2 * i + 1]);
                  ow[i] = *reinterpret_cast<const uint32_t*>(&t);
                }
                *reinterpret_cast<uint4*>(to) = o;
              }
            }
          }
        }
        if (some) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(acc_empty_leader[buf]);
          ++job_i;
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && ctrl->abort) atomicOr(p.err, 1);
  cluster_sync_all();                            // nobody leaves while the pair's MMAs may read its memory
  if (warp == 2) tmem_dealloc_pair(tmem_base, 512);
}

// Eight threads per row: the partial sums of its vocabulary and hypertoken tiles, its loss and lse.
__global__ void __launch_bounds__(256) k_xent_merge(CbView cb, RowArgs a, Plan pl, const float2* part, int part_rows, int parts,
                                                    const float2* part_h, int part_rows_h, const float* tl, int r_lo, int r_hi) {
  pdl_wait();
  pdl_trigger();
  __shared__ float2 s_ms[8][32];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, pos = r_lo + blockIdx.x * 32 + x;
  const bool live = pos < min(pl.head[0], r_hi);
  float m = -INFINITY, s = 0.f;
  int row = 0;
  if (live) {
    row = pl.perm[pos];
    const int b = a.row_seq ? a.row_seq[row] : row;
    for (int i = y; i < parts; i += 8) { const float2 v = part[(size_t)i * part_rows + pos - r_lo]; merge_ms(m, s, v.x, v.y); }
    const int hyper = 2 * ceil_div(cb.n[b], kTile);
    for (int i = y; i < hyper; i += 8) { const float2 v = part_h[(size_t)i * part_rows_h + pos]; merge_ms(m, s, v.x, v.y); }
  }
  s_ms[y][x] = make_float2(m, s);
  __syncthreads();
  if (y != 0 || !live) return;
  for (int i = 1; i < 8; ++i) merge_ms(m, s, s_ms[i][x].x, s_ms[i][x].y);
  const float ls = logf(s);
  a.lse_out[row] = m + ls;
  a.loss_out[row] = ls + (m - tl[pos]);
}

// dh of a row: its partial sums, those of the vocabulary's parts first, times the largest weight.
template <typename T>
__global__ void __launch_bounds__(128) k_xent_hidden(CbView cb, RowArgs a, Plan pl, const float* dh, long long slot, int split, T* out, int d) {
  pdl_wait();
  pdl_trigger();
  const int r = blockIdx.x, pos = pl.inv[r];
  T* to = out + (size_t)r * d;
  int slots = 0;
  if (pos >= 0) { const int b = a.row_seq ? a.row_seq[r] : r; slots = split + (cb.n[b] > 0 ? 1 : 0); }
  const float scale = __int_as_float(pl.head[4]);
  for (int i = threadIdx.x * 8; i < d; i += blockDim.x * 8) {
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < slots; ++k) {
      const float* from = dh + (size_t)k * slot + (size_t)pos * d + i;
      const float4 u = __ldcg(reinterpret_cast<const float4*>(from)), v = __ldcg(reinterpret_cast<const float4*>(from + 4));
      s[0] += u.x; s[1] += u.y; s[2] += u.z; s[3] += u.w; s[4] += v.x; s[5] += v.y; s[6] += v.z; s[7] += v.w;
    }
    if (slots) {
#pragma unroll
      for (int k = 0; k < 8; ++k) s[k] *= scale;
    }
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<float4*>(to + i) = make_float4(s[0], s[1], s[2], s[3]);
      *reinterpret_cast<float4*>(to + i + 4) = make_float4(s[4], s[5], s[6], s[7]);
    } else {
      uint32_t o[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) { const __nv_bfloat162 t = __floats2bfloat162_rn(s[2 * k], s[2 * k + 1]); o[k] = *reinterpret_cast<const uint32_t*>(&t); }
      *reinterpret_cast<uint4*>(to + i) = make_uint4(o[0], o[1], o[2], o[3]);
    }
  }
}

// Zeros of a call without rows that overwrites: W_U's rows, and the hypertokens that exist.
__global__ void __launch_bounds__(128) k_xent_zero(CbView cb, char* gWU, char* gUh, int row_bytes) {
  pdl_wait();
  pdl_trigger();
  const long long rows = (long long)cb.V + (long long)cb.B * cb.cap;
  for (long long r = blockIdx.x; r < rows; r += gridDim.x) {
    const long long k = r - cb.V;
    char* to = k < 0 ? gWU : (gUh && k % cb.cap < cb.n[k / cb.cap] ? gUh : nullptr);
    if (!to) continue;
    to += (size_t)(k < 0 ? r : k) * row_bytes;
    for (int i = threadIdx.x * 16; i < row_bytes; i += blockDim.x * 16) *reinterpret_cast<uint4*>(to + i) = make_uint4(0u, 0u, 0u, 0u);
  }
}

// ---- host ------------------------------------------------------------------------------------------
long long up_to(long long x, long long a) { return (x + a - 1) / a * a; }

int sm_count_xent() {
  static const int n = [] {
    int dev = 0, v = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || v <= 0) {
      cudaGetLastError();                        // (no GPU: sizes are still asked for)
      return 148;
    }
    return v;
  }();
  return n;
}

constexpr int kClusters = 74;                    // B200's pairs of SMs; what sizes are planned for

// Sizes of a call that the host knows.
struct Shape {
  int N, d, V, B, cap, dtype, parts;             // parts: bf16 parts of an operand
  int grad_dtype, g_parts;                       // < 0: losses alone
  int np, nh;                                    // rows of the sorted copy, and beside hypertokens
  int tr, th, dt, split;
  int pieces, vc;                                // vocabulary rows per piece, a multiple of 256
};

Shape shape_of(const z2z_config& c, int N, int grad_dtype, long long vc) {
  Shape s{};
  s.N = N; s.d = c.d; s.V = c.V; s.B = c.B; s.cap = c.cap; s.dtype = c.dtype; s.grad_dtype = grad_dtype;
  s.parts = c.dtype == Z2Z_DTYPE_FP32 ? kMaxParts : 1;
  s.g_parts = grad_dtype < 0 ? 0 : (s.parts > 1 || grad_dtype == Z2Z_DTYPE_FP32 ? kMaxParts : 1);
  s.np = (int)up_to(N, kTile);
  s.nh = (int)up_to((long long)N + (long long)(kHyperPad - 1) * (N < c.B ? N : c.B), kTile);
  // row tiles of equal height
  const int rt = (N + kTile - 1) / kTile;
  s.tr = (int)up_to((N + rt - 1) / rt, 32);
  const int mean = (int)up_to((N + c.B - 1) / c.B, 32);
  s.th = mean < 64 ? 64 : (mean > kTile ? kTile : mean);
  s.dt = (c.d + kTile - 1) / kTile;
  // with fewer tiles of dh than clusters the contracted vocabulary is split
  const int tiles = rt * s.dt;
  s.split = tiles >= kClusters ? 1 : kClusters / tiles;
  if (s.split > kMaxSplit) s.split = kMaxSplit;
  const long long whole = up_to(c.V, kTile);
  if (vc > whole) vc = whole;
  s.pieces = (int)((c.V + vc - 1) / vc);
  s.vc = (int)up_to((c.V + s.pieces - 1) / s.pieces, kTile);
  s.pieces = (c.V + s.vc - 1) / s.vc;
  return s;
}

struct Layout {
  Plan pl;
  __nv_bfloat16 *hs, *hh, *up, *ut, *wp, *g, *gh;
  float2 *part, *part_h;
  float *tl, *dh;
  size_t bytes;
};

int hyper_rows(const Shape& s) { return (int)up_to(s.cap, kTile); }

Layout layout_of(const Shape& s, char* base) {
  Layout l{};
  size_t o = 0;
  auto take = [&](size_t bytes) { char* r = base + o; o = (size_t)up_to((long long)(o + bytes), 256); return r; };
  const size_t row = (size_t)s.d * 2 * s.parts;
  l.pl.head = (int32_t*)take(32);
  l.pl.cnt = (int32_t*)take((size_t)s.B * 4); l.pl.wmax = (float*)take((size_t)s.B * 4);
  int32_t** tables[] = {&l.pl.s0, &l.pl.h0, &l.pl.j1, &l.pl.j2, &l.pl.j3};
  for (int32_t** t : tables) *t = (int32_t*)take((size_t)(s.B + 1) * 4);
  l.pl.perm = (int32_t*)take((size_t)s.np * 4); l.pl.inv = (int32_t*)take((size_t)s.np * 4);
  l.pl.meta = (float4*)take((size_t)s.np * 16);
  l.hs = (__nv_bfloat16*)take(row * s.np);
  if (s.cap > 0) {
    l.hh = (__nv_bfloat16*)take(row * s.nh);
    if (s.parts > 1) l.up = (__nv_bfloat16*)take(row * s.B * s.cap);
  }
  if (s.parts > 1) l.wp = (__nv_bfloat16*)take(row * s.vc);
  if (s.grad_dtype < 0) {
    const int vt = (s.V + kTile - 1) / kTile, rows = s.np < kLossRows ? s.np : kLossRows;
    l.part = (float2*)take((size_t)2 * vt * rows * 8);
    if (s.cap > 0) l.part_h = (float2*)take((size_t)2 * (hyper_rows(s) / kTile) * s.np * 8);
    l.tl = (float*)take((size_t)s.np * 4);
  } else {
    if (s.cap > 0) {
      l.ut = (__nv_bfloat16*)take(row * s.B * 16);
      l.gh = (__nv_bfloat16*)take((size_t)s.g_parts * hyper_rows(s) * s.nh * 2);
    }
    l.g = (__nv_bfloat16*)take((size_t)s.g_parts * s.vc * s.np * 2);
    l.dh = (float*)take((size_t)(s.split + 1) * s.np * s.d * 4);
  }
  l.bytes = o;
  return l;
}

// Vocabulary rows of a piece: G^T of 256 MB (8192 rows at least).  fp32 tables are also held in parts.
long long wanted_piece(const z2z_config& c, int N, int grad_dtype) {
  const bool f32 = c.dtype == Z2Z_DTYPE_FP32;
  if (grad_dtype < 0) return f32 ? 16384 : up_to(c.V, kTile);
  const long long per = 2ll * up_to(N, kTile) * (f32 || grad_dtype == Z2Z_DTYPE_FP32 ? kMaxParts : 1);
  long long vc = (256ll << 20) / per / kTile * kTile;
  if (vc < 8192) vc = 8192;
  if (f32 && vc > 16384) vc = 16384;
  return vc;
}
constexpr long long kLeastPiece = 2048;

size_t bytes_with(const z2z_config& c, int N, int grad_dtype, long long vc) { return layout_of(shape_of(c, N, grad_dtype, vc), nullptr).bytes; }

// The largest pieces up to the wanted ones for which the scratch suffices; 0 if none.
long long piece_for(const z2z_config& c, int N, int grad_dtype, size_t bytes) {
  long long vc = wanted_piece(c, N, grad_dtype);
  for (;;) {
    if (bytes_with(c, N, grad_dtype, vc) <= bytes) return vc;
    if (vc <= kLeastPiece) return 0;
    vc = vc / 2 < kLeastPiece ? kLeastPiece : vc / 2;
  }
}

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encode_fn() {
  static const EncodeFn fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) f = nullptr;
    return reinterpret_cast<EncodeFn>(f);
  }();
  return fn;
}

// Map over `planes` bf16 matrices [rows, cols], rows `pitch` elements apart; box = 64 columns x box_rows rows of one.
bool make_map(CUtensorMap* m, const void* base, long long rows, long long cols, long long pitch, int planes, long long plane, int box_rows) {
  const EncodeFn fn = encode_fn();
  if (!fn || rows < 1 || cols < 1) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
  const cuuint64_t strides[2] = {(cuuint64_t)pitch * 2, (cuuint64_t)(planes > 1 ? plane : rows * pitch) * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1}, es[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Products of parts, the smallest first.
void products(int parts_a, int parts_b, int* n, int8_t* a, int8_t* b) {
  *n = 0;
  for (int sum = kMaxParts - 1; sum >= 0; --sum)
    for (int i = 0; i < parts_a; ++i) {
      const int k = sum - i;
      if (k >= 0 && k < parts_b) { a[*n] = (int8_t)i; b[*n] = (int8_t)k; ++*n; }
    }
}

template <int KIND, typename TO>
cudaError_t launch_main(const Params& p, const Maps& tm, int clusters, cudaStream_t s) {
  auto kern = k_xent<KIND, TO>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes);
  if (e != cudaSuccess) return e;
  return launch_pdl(kern, dim3(2 * clusters), dim3(kThreads), kSmemBytes, s, p, tm);
}

// One of the two passes: losses, or gradients from lse.
cudaError_t run_pass(const CbView& cb, const z2z_config& cfg, const XentArgs& x, bool grad, cudaStream_t s) {
  const int gd = grad ? x.grad_dtype : -1;
  const long long vc = piece_for(cfg, x.N, gd, x.scratch_bytes);
  if (vc == 0) return cudaErrorMemoryAllocation;
  const Shape sh = shape_of(cfg, x.N, gd, vc);
  const Layout l = layout_of(sh, x.scratch);
  const int d = sh.d, clusters = sm_count_xent() / 2;
  RowArgs a{};
  a.N = x.N; a.row_seq = x.row_seq; a.row_nvis = x.row_nvis; a.targets = x.targets;
  a.th = sh.th; a.dt = sh.dt;
  if (grad) { a.weight = x.weight; a.lse = x.lse; a.hidden = x.g_hidden != nullptr; a.tables = x.g_Uh != nullptr; }
  else { a.loss_out = x.loss; a.lse_out = x.lse; }
  cudaError_t e = launch_pdl(k_xent_count, dim3((sh.B + 3) / 4), dim3(128), 0, s, cb, a, l.pl);
  if (e != cudaSuccess) return e;
  if ((e = launch_pdl(k_xent_place, dim3((sh.B + 4) / 4), dim3(128), 0, s, cb, a, l.pl)) != cudaSuccess) return e;
  GatherArgs g{};
  g.hidden = x.hidden; g.Uh = x.Uh; g.d = d; g.positions = sh.np;
  g.hs = l.hs; g.hs_plane = (long long)sh.np * d;
  g.hh = l.hh; g.hh_plane = (long long)sh.nh * d;
  g.up = l.up; g.up_plane = (long long)sh.B * sh.cap * d;
  g.ut = l.ut; g.ut_plane = (long long)sh.B * 16 * d;
  const unsigned blocks = sh.np + (l.ut ? sh.B * 16 : 0) + (l.up ? (unsigned)sh.B * sh.cap : 0);
  e = sh.dtype == Z2Z_DTYPE_FP32 ? launch_pdl(k_xent_gather<float>, dim3(blocks), dim3(128), 0, s, cb, a, l.pl, g)
                                 : launch_pdl(k_xent_gather<__nv_bfloat16>, dim3(blocks), dim3(128), 0, s, cb, a, l.pl, g);
  if (e != cudaSuccess) return e;

  Params p{};
  p.cb = cb; p.pl = l.pl; p.d = d; p.dt = sh.dt; p.tr = sh.tr; p.th = sh.th;
  products(sh.parts, sh.parts, &p.np1, p.a1, p.b1);
  // dh has the session's type: of three parts of g for fp32 tables' gradients it takes the first
  if (grad) {
    products(sh.parts, sh.parts, &p.np2, p.a2, p.b2);
    products(sh.g_parts, sh.parts, &p.np3, p.a3, p.b3);
  }
  p.g_parts = sh.g_parts; p.exact_exp = sh.g_parts > 1;
  p.g = l.g; p.g_pitch = sh.np; p.g_plane = (long long)sh.vc * sh.np;
  p.gh = l.gh; p.gh_pitch = sh.nh; p.gh_plane = (long long)hyper_rows(sh) * sh.nh;
  p.part = l.part; p.part_h = l.part_h; p.part_rows_h = sh.np; p.tl = l.tl;
  p.split = sh.split; p.dh = grad && x.g_hidden ? l.dh : nullptr; p.dh_slot = (long long)sh.np * d;
  p.gWU = x.g_WU; p.gUh = sh.cap > 0 ? x.g_Uh : nullptr; p.acc = x.accumulate ? 1 : 0;
  p.mem_cycles = kTile * kTile * (x.grad_dtype == Z2Z_DTYPE_FP32 ? 4 : 2) * (x.accumulate ? 2 : 1) / 46;
  p.err = x.err;
  // hidden rows of the row tiles that are taken through all vocabulary tiles together: a quarter of L2
  const long long tile_bytes = (long long)sh.tr * d * 2 * sh.parts;
  p.sb = (int)((32ll << 20) / tile_bytes); if (p.sb < 1) p.sb = 1;

  Maps tm{};
  const long long ur = (long long)sh.B * sh.cap;
  bool ok = make_map(&tm.hs_k, l.hs, sh.np, d, d, sh.parts, g.hs_plane, sh.tr / 2);
  if (sh.cap > 0) {
    const void* U = sh.parts > 1 ? l.up : x.Uh;
    ok = ok && make_map(&tm.u_k, U, ur, d, d, sh.parts, g.up_plane, 128) && make_map(&tm.hh_k, l.hh, sh.nh, d, d, sh.parts, g.hh_plane, sh.th / 2);
    if (grad)
      ok = ok && make_map(&tm.u_m, U, ur, d, d, sh.parts, g.up_plane, 64) && make_map(&tm.ut_m, l.ut, sh.B * 16, d, d, sh.parts, g.ut_plane, 16) &&
           make_map(&tm.hh_m, l.hh, sh.nh, d, d, sh.parts, g.hh_plane, 64) &&
           make_map(&tm.gh_k, l.gh, hyper_rows(sh), sh.nh, sh.nh, sh.g_parts, p.gh_plane, 128) &&
           make_map(&tm.gh_m, l.gh, hyper_rows(sh), sh.nh, sh.nh, sh.g_parts, p.gh_plane, 64);
  }
  if (grad)
    ok = ok && make_map(&tm.hs_m, l.hs, sh.np, d, d, sh.parts, g.hs_plane, 64) &&
         make_map(&tm.g_k, l.g, sh.vc, sh.np, sh.np, sh.g_parts, p.g_plane, 128) && make_map(&tm.g_m, l.g, sh.vc, sh.np, sh.np, sh.g_parts, p.g_plane, 64);
  const void* W = sh.parts > 1 ? l.wp : x.WU;
  const long long w_rows = sh.parts > 1 ? sh.vc : sh.V, w_plane = (long long)sh.vc * d;
  ok = ok && make_map(&tm.w_k, W, w_rows, d, d, sh.parts, w_plane, 128) && make_map(&tm.w_m, W, w_rows, d, d, sh.parts, w_plane, 64);
  if (!ok) return cudaErrorInvalidValue;

  const int share = grad ? x.N : (x.N < kLossRows ? x.N : kLossRows);
  for (int r0 = 0; r0 < x.N; r0 += share) {
    p.r_lo = r0; p.r_hi = r0 + share < x.N ? r0 + share : x.N;
    p.part_rows = (int)(sh.np < kLossRows ? sh.np : kLossRows);
    for (int i = 0; i < sh.pieces; ++i) {
      p.v0 = i * sh.vc; p.vn = sh.V - p.v0 < sh.vc ? sh.V - p.v0 : sh.vc;
      p.w_row0 = sh.parts > 1 ? 0 : p.v0;
      p.part0 = 2 * i * (sh.vc / kTile);
      p.first = i == 0;
      p.hyper = i == 0 && r0 == 0 && sh.cap > 0;
      p.hyper_hidden = p.hyper && p.dh;
      if (sh.parts > 1)
        if ((e = launch_pdl(k_xent_split, dim3(p.vn < 4096 ? p.vn : 4096), dim3(128), 0, s, reinterpret_cast<const float*>(x.WU) + (size_t)p.v0 * d, l.wp, w_plane, p.vn, d)) != cudaSuccess) return e;
      if (!grad) {
        if ((e = launch_main<kLoss, float>(p, tm, clusters, s)) != cudaSuccess) return e;
        continue;
      }
      if ((e = launch_main<kGrad, float>(p, tm, clusters, s)) != cudaSuccess) return e;
      e = x.grad_dtype == Z2Z_DTYPE_FP32 ? launch_main<kProducts, float>(p, tm, clusters, s) : launch_main<kProducts, __nv_bfloat16>(p, tm, clusters, s);
      if (e != cudaSuccess) return e;
    }
    if (!grad) {
      const int rows = p.r_hi - p.r_lo, vt = (sh.V + kTile - 1) / kTile;
      if ((e = launch_pdl(k_xent_merge, dim3((rows + 31) / 32), dim3(256), 0, s, cb, a, l.pl, l.part, p.part_rows, 2 * vt, l.part_h, sh.np, l.tl, p.r_lo, p.r_hi)) != cudaSuccess)
        return e;
    }
  }
  if (grad && x.g_hidden) {
    e = sh.dtype == Z2Z_DTYPE_FP32
            ? launch_pdl(k_xent_hidden<float>, dim3(x.N), dim3(128), 0, s, cb, a, l.pl, l.dh, p.dh_slot, sh.split, reinterpret_cast<float*>(x.g_hidden), d)
            : launch_pdl(k_xent_hidden<__nv_bfloat16>, dim3(x.N), dim3(128), 0, s, cb, a, l.pl, l.dh, p.dh_slot, sh.split, reinterpret_cast<__nv_bfloat16*>(x.g_hidden), d);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

void xent_scratch_bytes(const z2z_config& c, int N, int grad_dtype, size_t* least, size_t* most) {
  if (N <= 0) { *least = *most = 0; return; }
  // (a step needs what either pass does)
  const size_t l0 = bytes_with(c, N, -1, kLeastPiece), m0 = bytes_with(c, N, -1, wanted_piece(c, N, -1));
  const size_t l1 = grad_dtype < 0 ? 0 : bytes_with(c, N, grad_dtype, kLeastPiece);
  const size_t m1 = grad_dtype < 0 ? 0 : bytes_with(c, N, grad_dtype, wanted_piece(c, N, grad_dtype));
  *least = l0 > l1 ? l0 : l1;
  *most = m0 > m1 ? m0 : m1;
}

cudaError_t run_xent(const CbView& cb, const z2z_config& cfg, const XentArgs& a, cudaStream_t s) {
  if (a.N == 0) {
    if (!a.want_grad || a.accumulate || (!a.g_WU && !a.g_Uh)) return cudaSuccess;
    return launch_pdl(k_xent_zero, dim3(148 * 8), dim3(128), 0, s, cb, reinterpret_cast<char*>(a.g_WU), reinterpret_cast<char*>(a.g_Uh),
                      a.d * (a.grad_dtype == Z2Z_DTYPE_FP32 ? 4 : 2));
  }
  if (a.want_loss) {
    const cudaError_t e = run_pass(cb, cfg, a, false, s);
    if (e != cudaSuccess) return e;
  }
  return a.want_grad ? run_pass(cb, cfg, a, true, s) : cudaSuccess;
}

}  // namespace z2z
