// Cross entropy of hidden rows over the joint vocabulary (what the model is trained on: paper Section 2.4 with the
// distribution of Section 2.3 steps 7-9), without a matrix of fp32 logits, and its gradients.
//
//   l_rv   = h_r . W_v            v over the rows of W_U and the visible rows of U_h of the row's sequence
//   loss_r = log sum_v exp l_rv - l_rt
//   g_rv   = w_r (exp(l_rv - lse_r) - [v = t_r])
//   dh_r   = sum_v g_rv W_v       dW_v = sum_r g_rv h_r
//
// Three contractions of 2 N (V + n) d flop (the losses alone: one), all on tcgen05 with CTA pairs:
//   logits   D[r, v] = H  W^T     M = 256 hidden rows,     N = up to 256 vocabulary rows, K = d
//   hidden   D[d, r] = W^T G^T    M = 256 columns,         N = up to 256 hidden rows,     K = vocabulary rows
//   tables   D[v, d] = G^T H      M = 256 vocabulary rows, N = up to 256 columns,         K = hidden rows
// The vocabulary is taken in pieces: of each, G [r][v] is written by the epilogue of the logits, whose threads have a
// hidden row each, and both other contractions read it, with operands whose contiguous axis is the contracted one
// (K-major) or the other (MN-major) as they lie in memory: nothing is transposed.  Few rows cost little beside the
// tables: one pass over them for the logits, one for dh and the write of dW.
//
// Rows are sorted by their sequence first (stable), and rows without a target, which add nothing, are left out.
// Hypertokens are a piece per sequence: its entries against its own rows, which start at a multiple of 32 there.
// A step whose scratch has room for N (V + cap) values of 16 bits keeps its logits from the losses to the gradients, as
// distances in fixed point: three contractions then, not four (4096 rows, V = 128256, d = 4096: 9.4 ms, 11.9 without; 48 rows
// 0.70 and 0.96).
//
// Bound by the tensor cores from some hundred rows on (their power, in calls of milliseconds), below by memory: W_U is read
// twice and its gradient written once.  V = 128256, d = 4096, bf16: losses of 2047 rows (1842 with a target) 1.57 ms,
// 1.25 PFLOP/s (1.34 on a cool board); a step of 4096 (3680) rows 9.1 to 9.8 ms, 1.2 PFLOP/s of three contractions; a step of 48
// rows 0.70 to 0.75 ms, 4.2 to 4.5 TB/s of W_U twice and its gradient.
//
// Numbers.  A bf16 session's g is rounded once to bf16 for gradients stored in bf16; for fp32 gradients of the tables
// it is three bf16 parts (24 bits), of which dh takes two.  An fp32 session has all operands in three parts, and takes
// the six products of parts that fp32 can hold.  Accumulators are fp32 in tensor memory.  Weights enter as w_r / max w, so
// that equal weights lose nothing to g's rounding, and the maximum (of the finite weights) multiplies the sums.  lse
// carries what its rounding loses, and the target's p - 1 is an expm1: a row that is sure of its target keeps its gradient.
// Orders of summation depend on sizes only: the same call gives the same bits.
#include <atomic>

#include "z2z_common.cuh"
#include "z2z_internal.h"
#include "z2z_sm100.cuh"
#include "z2z_stream.h"
#include "z2z_xent.h"

namespace z2z {
using namespace sm100;

namespace {

constexpr int kEpiWarps = 8;                     // two per tensor-memory lane quarter, with 128 columns each
constexpr int kThreads = 128 + 32 * kEpiWarps;   // a warpgroup of producer, issuer and two that leave; two of the epilogue
// Registers: 384 threads are launched with 168 each; the epilogue, which holds a tile's sums, takes what the others leave
// (128 x 56 + 256 x 224 = 384 x 168; a launch with fewer is refused, since the epilogue would wait for the rest forever).
// The forms of the products spill 76 to 174 bytes a thread, those of the logits none, or 20 to 48 without chains; 190 bytes
// instead of 174 took the same time.
constexpr int kRegsFew = 56, kRegsEpi = 224;
constexpr int kRegsAtLaunch = (128 * kRegsFew + 32 * kEpiWarps * kRegsEpi) / kThreads;
constexpr int kRing = 10;                        // stages at most
constexpr int kTile = 256;                       // vocabulary rows or columns of a tile (128 per CTA)
constexpr int kTurnBytes = 32 * 128;             // a warp's 32 rows of 128 bytes on their way to memory; two of them
constexpr int kFrontBytes = 1024 + kEpiWarps * 2 * kTurnBytes;     // a multiple of 1024
constexpr size_t kSmemBytes = 232448;            // all that a block may have: control block and turns, then the ring
// A stage: 128 x 64 of either operand, or less of the hidden rows.  (The losses store no tiles.)
__host__ __device__ constexpr int front_bytes(bool turns) { return turns ? kFrontBytes : 1024; }
__host__ __device__ constexpr int ring_bytes(bool turns) { return (int)kSmemBytes - 1024 - front_bytes(turns); }
constexpr int kHyperPad = 32;                    // a sequence's rows start at a multiple of this beside its hypertokens
constexpr int kLossRows = 8192;                  // rows whose partial sums are held at a time
constexpr int kMaxParts = 3;                     // bf16 parts of an fp32 value
constexpr int kMaxSplit = 16;
constexpr float kLog2e = 1.4426950408889634f;

struct Ctrl {
  unsigned long long full[kRing], empty[kRing], acc_full[2], acc_empty[2], done;
  uint32_t tmem_base;
  uint32_t bytes[kRing];     // that this CTA has last loaded into a stage
  int issued;                // stages that it has loaded in all
  int abort, other_abort;    // a role has given up: here, in the other CTA of the pair
};
static_assert(sizeof(Ctrl) <= 1024 && kFrontBytes % 1024 == 0, "control block");

// What the plan leaves in the scratch.
struct Plan {
  int32_t* head;             // [0] rows that take part, [1..3] jobs of hypertokens: logits, hidden, tables; [4] largest finite weight, or 1;
                             // [5] a wait of this call has given up
  int32_t* cnt;              // [B] rows of a sequence that take part
  int32_t *s0, *h0;          // [B + 1] first position of a sequence's rows, and the one beside its hypertokens
  int32_t *j1, *j2, *j3;     // [B + 1] jobs of the sequences before
  int32_t *perm, *inv;       // position -> row, row -> position or -1
  int2* place;               // position -> row beside the hypertokens, and zero rows behind it (the last of a sequence)
  float4* meta;              // per position: lse, weight / largest, target and visible hypertokens (bits)
  float* rest;               // and what lse has lost to its rounding, where this call has it
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
  int cta_rows, nv;          // logits: hidden rows per CTA, vocabulary rows per tile
  int a_bytes;               // and shared memory of a stage's hidden rows
  int tr, th;                // rows per tile of dh, and per tile of a sequence's rows
  int r_lo, r_hi;            // positions of this launch (losses: a share of the rows)
  int sb;                    // row tiles that are taken through all vocabulary tiles before the next ones
  int parts;                 // bf16 parts of the session's operands
  int np2, np3;              // products of parts for dh and for the tables
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
  unsigned long long wait_ns; // after which a wait gives up
  int* err;
};

struct Maps {
  // K-major: 64 columns x 128 rows of a table, or a CTA's rows of a tile of hidden rows or of G
  CUtensorMap w_k, u_k, hs_k, hh_k, g_k, gh_k;
  // MN-major: 64 columns x 64 rows (ut: 16)
  CUtensorMap w_m, u_m, ut_m, hs_m, hh_m, g_m, gh_m;
  // stores: 32 rows x 128 bytes of G and of W_U's gradient
  CUtensorMap g_s, gh_s, o_w;
};

__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

// ---- plan ------------------------------------------------------------------------------------------
// One block: a histogram of the rows that take part over their sequences, its prefix sums, and a stable place for
// every row.  (A warp per sequence that looked through all rows took 60 us at 4096 rows of 16 sequences.)
struct PlanShared {
  int warp_sums[32];
  float wmax;
};
constexpr int kPlanThreads = 1024, kPlanFew = 256;                      // (few: up to 1024 rows of up to 32 sequences)
__host__ __device__ constexpr size_t plan_shared_bytes(int B) { return sizeof(PlanShared) + (size_t)B * 16 + (size_t)32 * B * 2; }

template <int THREADS>
__global__ void __launch_bounds__(THREADS) k_xent_plan(CbView cb, RowArgs a, Plan pl) {
  extern __shared__ unsigned char smem[];
  PlanShared& sh = *reinterpret_cast<PlanShared*>(smem);
  int* s_cnt = reinterpret_cast<int*>(smem + sizeof(PlanShared));       // rows of a sequence, then where its next ones go
  int *s_n = s_cnt + cb.B, *s_off = s_n + cb.B, *s_last = s_off + cb.B;        // hypertokens; place beside them less position; last position
  unsigned short* s_warp = reinterpret_cast<unsigned short*>(s_last + cb.B);   // [B][32] rows of a warp
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // rows of a thread whose loads are under way together; where these are all, they stay in registers
  constexpr int kBatch = 4, kBatchRows = kBatch * THREADS;
  int q[kBatch], tgt[kBatch], nv[kBatch];        // sequence, -1 where the row takes no part
  float w[kBatch], lse[kBatch];
  auto load = [&](int r0) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int r = r0 + u * THREADS + tid;
      const bool in = r < a.N;
      q[u] = in ? (a.row_seq ? a.row_seq[r] : r) : -1;
      tgt[u] = in ? a.targets[r] : Z2Z_CODE_NONE;
      nv[u] = in && a.row_nvis ? max(a.row_nvis[r], 0) : 0x7fffffff;
      w[u] = in && a.weight ? a.weight[r] : 1.f;
      lse[u] = in && a.lse ? a.lse[r] : 0.f;
    }
  };
  pdl_wait();
  pdl_trigger();
  load(0);
  for (int b = tid; b < cb.B; b += THREADS) { s_cnt[b] = 0; s_n[b] = cb.n[b]; }
  for (int i = tid; i < 32 * cb.B; i += THREADS) s_warp[i] = 0;
  if (tid == 0) sh.wmax = 0.f;
  __syncthreads();

  // whose row it is, if it takes part
  auto settle = [&](int u) {
    const int b = q[u];
    q[u] = -1;
    if (b < 0 || b >= cb.B || tgt[u] == Z2Z_CODE_NONE) return;
    nv[u] = min(nv[u], s_n[b]);
    if (tgt[u] < 0 || tgt[u] >= cb.V + nv[u]) atomicOr(&cb.status[b], Z2Z_ST_BAD_TOKEN);
    else if (w[u] != 0.f || a.loss_out) q[u] = b;
  };
  int wbits = 0;
  for (int r0 = 0; r0 < a.N; r0 += kBatchRows) {
    if (r0) load(r0);
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int r = r0 + u * THREADS + tid;
      if (r >= a.N) { q[u] = -1; continue; }
      settle(u);
      if (q[u] >= 0) {
        atomicAdd(&s_cnt[q[u]], 1);
        const float x = fabsf(w[u]);
        if (x < INFINITY) wbits = max(wbits, __float_as_int(x));
      } else {
        if (a.loss_out) a.loss_out[r] = 0.f;
        if (a.lse_out) a.lse_out[r] = 0.f;
      }
    }
  }
  // (magnitudes compare as whole numbers.  A weight that is not finite stays what it is in its own row)
  wbits = __reduce_max_sync(0xffffffffu, wbits);
  if (lane == 0) atomicMax(reinterpret_cast<int*>(&sh.wmax), wbits);
  __syncthreads();
  const float wmax = sh.wmax > 0.f ? sh.wmax : 1.f;

  // prefix sums over the sequences (B <= 1024: one each)
  const int b = tid, c = b < cb.B ? s_cnt[b] : 0, n = b < cb.B ? s_n[b] : 0;
  const int rt = ceil_div(c, a.th), kt = ceil_div(n, kTile);
  const int v[5] = {c, ceil_div(c, kHyperPad) * kHyperPad, rt * kt, a.hidden && n ? rt * a.dt : 0, a.tables ? kt * a.dt : 0};
  int32_t* const out[5] = {pl.s0, pl.h0, pl.j1, pl.j2, pl.j3};
  int x[5] = {0, 0, 0, 0, 0}, total[5];
  if (THREADS < 1024 || cb.B <= 32) {
    if (warp == 0) {
#pragma unroll
      for (int i = 0; i < 5; ++i) {
        x[i] = v[i];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const int y = __shfl_up_sync(0xffffffffu, x[i], o); if (lane >= o) x[i] += y; }
        total[i] = __shfl_sync(0xffffffffu, x[i], 31);
        x[i] -= v[i];
      }
    }
  } else if constexpr (THREADS == 1024) {
#pragma unroll
    for (int i = 0; i < 5; ++i) x[i] = block_scan_1024(v[i], sh.warp_sums, total[i]);
    __syncthreads();
  }
  if (b < cb.B) {
#pragma unroll
    for (int i = 0; i < 5; ++i) out[i][b] = x[i];
    pl.cnt[b] = c;
    s_cnt[b] = x[0]; s_off[b] = x[1] - x[0]; s_last[b] = x[0] + c - 1;
  }
  if (tid == 0) {
#pragma unroll
    for (int i = 0; i < 5; ++i) out[i][cb.B] = total[i];
    pl.head[0] = total[0]; pl.head[1] = total[2]; pl.head[2] = total[3]; pl.head[3] = total[4]; pl.head[4] = __float_as_int(wmax); pl.head[5] = 0;
  }
  __syncthreads();

  // Places, a row per thread at a time: rows of the same sequence in a warp by votes, the warps of a sequence one after another.
  for (int r0 = 0; r0 < a.N; r0 += kBatchRows) {
    if (a.N > kBatchRows) {
      load(r0);
#pragma unroll
      for (int u = 0; u < kBatch; ++u) settle(u);
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (r0 + u * THREADS >= a.N) break;
      const int r = r0 + u * THREADS + tid;
      const unsigned same = __match_any_sync(0xffffffffu, q[u]);
      const int rank = __popc(same & ((1u << lane) - 1u));
      if (q[u] >= 0 && rank == 0) s_warp[q[u] * 32 + warp] = (unsigned short)__popc(same);
      __syncthreads();
      int at = -1;
      if (q[u] >= 0) {
        at = s_cnt[q[u]] + rank;
        for (int i = 0; i < warp; ++i) at += s_warp[q[u] * 32 + i];
      }
      __syncthreads();
      if (q[u] >= 0 && rank == 0) { atomicAdd(&s_cnt[q[u]], (int)s_warp[q[u] * 32 + warp]); s_warp[q[u] * 32 + warp] = 0; }
      if (r < a.N) pl.inv[r] = at;
      if (at >= 0) {
        const int h = at + s_off[q[u]];
        pl.perm[at] = r;
        pl.place[at] = make_int2(h, at == s_last[q[u]] ? -(h + 1) & (kHyperPad - 1) : 0);
        pl.meta[at] = make_float4(lse[u], w[u] == 0.f ? 0.f : w[u] / wmax, __int_as_float(tgt[u]), __int_as_float(nv[u]));
        pl.rest[at] = 0.f;
      }
      __syncthreads();
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
#pragma unroll 4
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
    const int p = blockIdx.x, at = pl.perm[p], live = pl.head[0];
    const int2 place = pl.place[p];
    if (p >= ceil_div(live, kTile) * kTile) return;
    const int row = p < live ? at : -1;
    const T* src = row >= 0 ? reinterpret_cast<const T*>(g.hidden) + (size_t)row * d : nullptr;
    put_row(src, g.hs + (size_t)p * d, g.hs_plane, d, tid, blockDim.x);
    if (g.hh && row >= 0) {
      put_row(src, g.hh + (size_t)place.x * d, g.hh_plane, d, tid, blockDim.x);
      for (int i = 1; i <= place.y; ++i) put_row<T>(nullptr, g.hh + (size_t)(place.x + i) * d, g.hh_plane, d, tid, blockDim.x);
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
  int m0;                    // first row of the result: position (within the sequence), column, or vocabulary row
  int r0, n;                 // its first column: vocabulary row, position, or column of the table; and how many
  int k0, k16;               // first contracted row, steps of 16
  bool tail;                 // one more step, from the copy of the last hypertokens
  int limit;                 // positions of the tile that exist
  int part;                  // slot of the result
};
__host__ __device__ __forceinline__ int pad32(int n) { return (n + 31) & ~31; }
// Vocabulary tiles of a piece: up to the next multiple of 64, since G's columns are contracted in blocks of 64.
__host__ __device__ __forceinline__ int pad64(int n) { return (n + 63) & ~63; }
__host__ __device__ __forceinline__ int vocabulary_tiles(int vn, int nv) { return (pad64(vn) + nv - 1) / nv; }

// Logits of a launch, dealt in turn: all row tiles of a share of the rows for one vocabulary tile, then the next, so
// that the clusters at work share both operands.
struct LogitsWalk {
  const Params& p;
  int c, C, idx, live, RT, VT, base, hyper;
  __device__ LogitsWalk(const Params& pp, int c_, int C_) : p(pp), c(c_), C(C_) {
    const int rows = min(p.pl.head[0], p.r_hi) - p.r_lo;
    live = rows > 0 ? rows : 0;
    RT = ceil_div(live, 2 * p.cta_rows); VT = vocabulary_tiles(p.vn, p.nv);
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
      j.type = kLogits; j.b = -1; j.m0 = p.r_lo + rt * 2 * p.cta_rows;
      j.limit = min(2 * p.cta_rows, live - rt * 2 * p.cta_rows);
      j.r0 = vt * p.nv;
      j.n = min(p.nv, pad64(p.vn) - j.r0);
      j.part = p.part0 + 2 * vt;
      return true;
    }
    if (at - base >= hyper) return false;
    const int b = find_seq(p.pl.j1, p.cb.B, at - base), i = at - base - p.pl.j1[b];
    const int rows = p.pl.cnt[b], rt = ceil_div(rows, p.th), kt = i / rt, q = i - kt * rt;
    j.type = kLogitsHyper; j.b = b; j.m0 = q * p.th;
    j.limit = min(p.th, rows - j.m0);
    j.r0 = kt * kTile;
    j.n = min(kTile, pad32(p.cb.n[b] - j.r0));
    j.part = 2 * kt;
    return true;
  }
};

// Gradients of a piece.  Clusters take the tiles of dh in turn; those that are left out of the last round take tiles
// of the table's gradient meanwhile, and then all take those.
struct GradWalk {
  const Params& p;
  int c, C, live, RT, T, J2, J3, k3, rest, ahead, skip, idx, jh3, jh2, kb, cost2, cost3;
  int phase;                                     // 0: dh, 1: tables ahead, 2: tables, 3: hypertokens
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
  __device__ __forceinline__ void table_tile(Job& j, int f) {
    const int vt = f / p.dt, ct = f - vt * p.dt;
    j.type = kTables; j.b = -1; j.m0 = vt * kTile; j.r0 = ct * kTile;
    j.n = min(kTile, pad32(p.d - j.r0));
    j.k0 = 0; j.k16 = k3; j.tail = false; j.limit = 0; j.part = 0;
  }
  __device__ __forceinline__ void hidden_tile(Job& j, int f) {
    const int part = f / T, t = f - part * T, rt = t / p.dt;
    const int kb0 = (int)((long long)part * kb / p.split), kb1 = (int)((long long)(part + 1) * kb / p.split);
    j.type = kHidden; j.b = -1; j.m0 = (t - rt * p.dt) * kTile;
    j.r0 = rt * p.tr; j.limit = min(p.tr, live - j.r0); j.n = pad32(j.limit);
    j.k0 = kb0 * 64; j.k16 = (kb1 - kb0) * 4; j.tail = false; j.part = part;
  }
  __device__ __forceinline__ bool next(Job& j) {
    if (phase == 0) {
      if (idx < J2) { hidden_tile(j, idx); idx += C; return true; }
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

// Without operands in several parts: times that the contracted axis is gone through, once for each part of g.  (Gradients in
// bf16, the form without chains: one.)
__device__ __forceinline__ int job_turns(const Params& p, int type) { return type >= kTables ? p.g_parts : (type >= kHidden ? p.np2 : 1); }
__device__ __forceinline__ int job_blocks(const Job& j) { return (j.k16 + 3) / 4 + (j.tail ? 1 : 0); }
// The tensor cores' additions into an accumulator truncate: a chain of n of them is off by about n / 2 steps of 2^-24 to
// one side (losses at d = 4096 were 3e-6 off).  Where that counts an accumulator takes so many blocks of 64, and the epilogue
// adds those sums in registers, rounded to nearest, while the MMAs go on in the other accumulator.
// (dh of a bf16 session: every 256 additions for g in two parts; with one, whose rounding is up to 2^-9 of each term, the
// whole axis, 8000 additions and 2^-12 at V = 128256.)
constexpr int kChain = 8, kChainHidden = 64;
__device__ __forceinline__ int job_chain(const Params& p, const Job& j) {
  if (p.parts > 1) return 1;                     // (six products)
  return j.type <= kLogitsHyper ? kChain : (j.type <= kHiddenHyper ? kChainHidden : kChain);
}
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, volatile int* abort_flag, unsigned long long ns) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, ns));
}
// Wait for what is under way and comes to its end by itself.  Bounded by probes, of up to a microsecond each: time passes
// while a process is off the GPU, too.
constexpr int kDrainProbes = 1 << 16;
__device__ __forceinline__ void drain(uint32_t bar, uint32_t parity) {
  for (int i = 0; i < kDrainProbes; ++i)
    if (mbar_try_wait(bar, parity)) return;
}
// Loads of a pair in which a role has given up, by one thread of the leader, on whose barriers both CTAs' bytes count, once all
// roles of both have left: until they have landed, no memory of the pair may be given back.  The CTAs have issued the
// same stages in the same order, one maybe up to a whole ring of them more than the other: there the barrier still expects
// the bytes of both (the leader's stages) or none (the other's).
__device__ __forceinline__ void drain_loads(Ctrl* ctrl, int stages) {
  const int mine = ctrl->issued, theirs = (int)ld_cluster_u32(map_to_cta(smem_u32(&ctrl->issued), 1));
  const int both = min(mine, theirs), most = max(mine, theirs);
  for (int i = max(both - stages, 0); i < most; ++i) {
    const int s = i % stages;
    const uint32_t bar = smem_u32(&ctrl->full[s]);
    if (i >= mine) mbar_expect_tx(bar, ld_cluster_u32(map_to_cta(smem_u32(&ctrl->bytes[s]), 1)));
    else if (i >= theirs) mbar_complete_tx(bar, ctrl->bytes[s]);
    drain(bar, (i / stages) & 1);
  }
}

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

// Arrival at a barrier of this cluster that orders nothing: the accumulator has been read into registers when it is made
// (tcgen05.wait::ld), and a release would wait for the stores of the tile before (a tile of dW 6900 -> 5900 clocks).
__device__ __forceinline__ void mbar_arrive_relaxed(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// exp(v - lse - rest) with all roundings of the exponent made good, the difference's own (half a step of 9 is 2^-21) and
// those of log2 e among them: ex2's own error (2^-22) is what is left.
constexpr float kLog2eRest = 1.92596299e-8f;     // log2 e less kLog2e
__device__ __forceinline__ float exp_exact(float v, float lse, float rest) {
  const float x = v - lse, b = x - v, lost = (v - (x - b)) - (lse + b);      // (x + lost is the difference)
  const float y = x * kLog2e, r = fmaf(x, kLog2eRest, fmaf(x, kLog2e, -y)), e = ex2(y);
  return y > -200.f ? fmaf(e, fmaf(r, 0.69314718f, lost - rest), e) : e;     // (-inf: lost is no number)
}

__device__ __forceinline__ void merge_ms(float& m, float& s, float om, float os) {
  if (om == -INFINITY) return;                   // (nothing there; a NaN is in s, beside a maximum)
  if (m == -INFINITY) { m = om; s = os; return; }
  const float top = fmaxf(m, om);
  s = (m == top ? s : s * expf(m - top)) + (om == top ? os : os * expf(om - top));
  m = top;
}

// kKeep: the losses' sums, and every logit in 16 bits as its distance from the largest of its row and half tile, in
// steps of 2^-11 (half of one: p off by 2^-12, where g's rounding to bf16 is 2^-8); from 32 on, p < 1e-14, it is none.
enum Kind { kLoss, kGrad, kProducts, kKeep };
constexpr float kKeepSteps = 2048.f;
constexpr uint32_t kKeepNone = 65535u;

__device__ __forceinline__ void tma_store_3d(const CUtensorMap* m, uint32_t src, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(m), "r"(src), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void tma_add_3d(const CUtensorMap* m, uint32_t src, int x, int y, int z) {
  asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(m), "r"(src), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(LEFT) : "memory"); }
__device__ __forceinline__ void bulk_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// A warp's way to memory for blocks of 32 rows (one per lane) of 128 bytes: two buffers in shared memory, in which 16-byte
// groups of a row are exchanged by its row's low bits (the 128-byte swizzle), and then either one TMA store of the
// block or stores of whole lines of four rows.  (48 rows, V = 128256, d = 4096, clocks per tile of dW: stored from the lanes' own
// rows, 32 lines per instruction, 15000; lines 5900; TMA 4500, which is what 1.05 GB written at 4.2 TB/s take.)
struct Turn {
  uint4* buf;                                    // [2][32 * 8]
  int at, lane;
  __device__ __forceinline__ uint4* put(const uint32_t (&w)[32]) {
    uint4* to = buf + at * 256;
#pragma unroll
    for (int g = 0; g < 8; ++g) to[lane * 8 + (g ^ (lane & 7))] = make_uint4(w[4 * g], w[4 * g + 1], w[4 * g + 2], w[4 * g + 3]);
    return to;
  }
  // Whole blocks; what lies outside the map is left out.
  template <bool ADD>
  __device__ __forceinline__ void tma(const uint32_t (&w)[32], const CUtensorMap* m, int x, int y, int z) {
    if (lane == 0) bulk_wait_read<1>();          // the buffer's block before has left
    __syncwarp();
    uint4* from = put(w);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
      if (ADD) tma_add_3d(m, smem_u32(from), x, y, z);
      else tma_store_3d(m, smem_u32(from), x, y, z);
      bulk_commit();
    }
    at ^= 1;
  }
  // `rows` rows of `bytes` bytes (a multiple of 16), `pitch` bytes apart.
  template <bool ADD>
  __device__ __forceinline__ void lines(const uint32_t (&w)[32], char* out, long long pitch, int rows, int bytes) {
    if (lane == 0) bulk_wait_read<0>();
    __syncwarp();
    const uint4* from = put(w);
    __syncwarp();
    const int r0 = lane >> 3, g = lane & 7;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = r0 + 4 * i;
      const uint4 o = from[r * 8 + (g ^ (r & 7))];
      if (r < rows && 16 * g < bytes) {
        char* to = out + r * pitch + 16 * g;
        if (ADD) red_add_f32x4(reinterpret_cast<float*>(to), __uint_as_float(o.x), __uint_as_float(o.y), __uint_as_float(o.z), __uint_as_float(o.w));
        else *reinterpret_cast<uint4*>(to) = o;
      }
    }
    __syncwarp();
  }
};
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&t);
}
// 64 columns of a table's gradient; m: its map, for blocks that end with it or not at all, or NULL.  ADD: to what is there,
// rounded once; fp32 by reductions in L2 (every element has one writer, so that their order does not matter), bf16
// with a load ahead.
template <typename T, bool ADD>
__device__ __forceinline__ void store_columns(float (&v)[64], Turn& turn, const CUtensorMap* m, int x0, int y0, T* out, long long pitch, int rows, int cols) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (32 * h >= cols) break;
      uint32_t w[32];
#pragma unroll
      for (int x = 0; x < 32; ++x) w[x] = __float_as_uint(v[32 * h + x]);
      if (m) turn.tma<ADD>(w, m, x0 + 32 * h, y0, 0);
      else turn.lines<ADD>(w, reinterpret_cast<char*>(out + 32 * h), pitch * 4, rows, 4 * (cols - 32 * h));
    }
  } else if constexpr (!ADD) {
    uint32_t w[32];
#pragma unroll
    for (int x = 0; x < 32; ++x) w[x] = pack_bf16(v[2 * x], v[2 * x + 1]);
    if (m) turn.tma<false>(w, m, x0, y0, 0);
    else turn.lines<false>(w, reinterpret_cast<char*>(out), pitch * 2, rows, 2 * cols);
  } else {
    // four lanes per row and 32 columns; the old values are under way while the sums are turned
    const int lane = turn.lane;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (32 * h >= cols) break;
      const int r0 = lane >> 2, col = 32 * h + (lane & 3) * 8;
      uint4 old[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = r0 + 8 * i;
        old[i] = make_uint4(0u, 0u, 0u, 0u);
        if (r < rows && col < cols) old[i] = *reinterpret_cast<const uint4*>(out + r * pitch + col);
      }
      uint32_t w[32];
#pragma unroll
      for (int x = 0; x < 32; ++x) w[x] = __float_as_uint(v[32 * h + x]);
      __syncwarp();
      const float4* t4 = reinterpret_cast<const float4*>(turn.put(w));
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = r0 + 8 * i, g = 2 * (lane & 3);
        const float4 x = t4[r * 8 + (g ^ (r & 7))], y = t4[r * 8 + ((g + 1) ^ (r & 7))];
        const uint32_t o[4] = {old[i].x, old[i].y, old[i].z, old[i].w};
        const float f[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
        uint32_t t[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) t[k] = pack_bf16(__uint_as_float(o[k] << 16) + f[2 * k], __uint_as_float(o[k] & 0xffff0000u) + f[2 * k + 1]);
        if (r < rows && col < cols) *reinterpret_cast<uint4*>(out + r * pitch + col) = make_uint4(t[0], t[1], t[2], t[3]);
      }
    }
  }
}

// CHAINED: accumulators of some blocks, added in registers.  MULTI: operands of several parts, every part a stage of its own that
// all its products read (a stage per product moved twice the bytes through L2, which is what bounds it then).
template <int KIND, bool CHAINED, bool MULTI, typename TO>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
k_xent(const __grid_constant__ Params p, const __grid_constant__ Maps tm) {
  using Walk = typename std::conditional<KIND == kProducts, GradWalk, LogitsWalk>::type;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* sm = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  Ctrl* ctrl = reinterpret_cast<Ctrl*>(sm);
  const uint32_t stage_base = smem_u32(sm + front_bytes(KIND != kLoss));
  const int warp = uniform_warp(), lane = threadIdx.x & 31;
  const int rank = (int)cluster_ctarank();       // 0: leader (issues the MMAs), 1: peer
  const int C = gridDim.x >> 1, c = blockIdx.x >> 1;

  // An MMA of the logits reads 128 hidden rows from a stage's start; with fewer loaded it reads on, which only feeds rows of
  // the result that nobody looks at.
  const uint32_t b_off = KIND == kProducts ? 16384u : (uint32_t)p.a_bytes, stage_bytes = b_off + 16384u;
  const int stages = min(kRing, (int)(ring_bytes(KIND != kLoss) / (MULTI ? 16384u : stage_bytes)));

  if (threadIdx.x == 0) {
    for (int s = 0; s < kRing; ++s) { mbar_init(smem_u32(&ctrl->full[s]), 1); mbar_init(smem_u32(&ctrl->empty[s]), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(smem_u32(&ctrl->acc_full[b]), 1); mbar_init(smem_u32(&ctrl->acc_empty[b]), 2 * kEpiWarps); }
    mbar_init(smem_u32(&ctrl->done), 1);
    ctrl->issued = ctrl->abort = ctrl->other_abort = 0;
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

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsFew));
    if (warp == 0 && lane == 0) {
      // ---------------- TMA producer (both CTAs): own 128 rows of A, own half of B's ----------------------
      const uint64_t pol = policy_evict_last();
      const uint32_t full_leader = map_to_cta(smem_u32(&ctrl->full[0]), 0);
      Walk w(p, c, C);
      Job j;
      int stage = 0, issued = 0; uint32_t phase = 0;
      bool ok = true;
      auto begin = [&](uint32_t bytes) {         // the next stage, with so many bytes to come in each CTA
        ok = mbar_wait(smem_u32(&ctrl->empty[stage]), phase ^ 1u, &ctrl->abort, p.wait_ns);
        if (ok) ctrl->bytes[stage] = bytes;
        if (ok && rank == 0) mbar_expect_tx(smem_u32(&ctrl->full[stage]), 2u * bytes);
        return ok;
      };
      auto end = [&]() { ++issued; if (++stage == stages) { stage = 0; phase ^= 1u; } };
      // An operand of a job: boxes from (x, y) on, (dx, dy) further per block, with one 64 columns beside them where `two`.
      // (All of it is set up per job: with the choices made per box the thread issued a block every 600 clocks, and the
      // MMAs waited for it.)
      struct Side {
        const CUtensorMap* m;
        int x, y, dx, dy;
        bool two;
        uint32_t bytes;
      };
      auto load = [&](const Side& o, uint32_t at, uint32_t bar, int x, int y, int part) {
        tma_load_3d_pair(at, o.m, x, y, part, bar, pol);
        if (KIND == kProducts && o.two) tma_load_3d_pair(at + 8192u, o.m, x + 64, y, part, bar, pol);
      };
      while (ok && w.next(j)) {
        const int half = j.n >> 1, whole = (j.k16 + 3) / 4;
        const bool hy = j.b >= 0;
        const int h0 = hy ? p.pl.h0[j.b] : 0;
        Side A, B;
        if (KIND != kProducts) {
          const int rows = hy ? p.th >> 1 : p.cta_rows;
          A = Side{hy ? &tm.hh_k : &tm.hs_k, 0, h0 + j.m0 + rank * rows, 64, 0, false, 128u * rows};
          B = Side{hy ? &tm.u_k : &tm.w_k, 0, (hy ? j.b * p.cb.cap : p.w_row0) + j.r0 + rank * half, 64, 0, false, 16384u};
        } else if (j.type == kHidden || j.type == kHiddenHyper) {
          A = Side{hy ? &tm.u_m : &tm.w_m, j.m0 + rank * 128, hy ? j.b * p.cb.cap : p.w_row0 + j.k0, 0, 64, true, 16384u};
          B = Side{hy ? &tm.gh_k : &tm.g_k, j.k0, h0 + j.r0 + rank * half, 64, 0, false, 64u * (hy ? p.th : p.tr)};
        } else {
          A = Side{hy ? &tm.gh_m : &tm.g_m, j.m0 + rank * 128, h0, 0, 64, true, 16384u};
          B = Side{hy ? &tm.hh_m : &tm.hs_m, j.r0 + rank * half, h0, 0, 64, half > 64, half > 64 ? 16384u : 8192u};
        }
        const int turns = MULTI || !CHAINED ? 1 : job_turns(p, j.type);
        auto block = [&](int part, int ax, int ay, int bx, int by) {
          if constexpr (MULTI) {
            // (in the order in which the MMAs want them)
            auto one = [&](const Side& o, int x, int y, int i) {
              if (ok && begin(o.bytes)) { load(o, stage_base + (uint32_t)stage * 16384u, full_leader + 8u * stage, x, y, i); end(); }
            };
            one(A, ax, ay, 2); one(B, bx, by, 0); one(A, ax, ay, 0); one(B, bx, by, 2); one(A, ax, ay, 1); one(B, bx, by, 1);
          } else if (begin(A.bytes + B.bytes)) {
            const uint32_t at = stage_base + (uint32_t)stage * stage_bytes, bar = full_leader + 8u * stage;
            // (g, the tables' A and dh's B, with its smallest part first)
            load(A, at, bar, ax, ay, j.type >= kTables ? turns - 1 - part : 0);
            load(B, at + b_off, bar, bx, by, j.type >= kTables ? 0 : turns - 1 - part);
            end();
          }
        };
        for (int part = 0; part < turns && ok; ++part) {
          int ax = A.x, ay = A.y, bx = B.x, by = B.y;
          for (int kb = 0; kb < whole && ok; ++kb) {
            block(part, ax, ay, bx, by);
            ax += A.dx; ay += A.dy; bx += B.dx; by += B.dy;
          }
          if (KIND == kProducts && j.tail && ok) {
            const Side entries = A;
            A.m = &tm.ut_m; A.bytes = 4096u;
            block(part, A.x, j.b * 16, j.k16 * 16, B.y);
            A = entries;
          }
        }
      }
      ctrl->issued = issued;
    } else if (warp == 1 && rank == 0) {
      // ---------------- MMA issuer (leader only, the whole warp: elect_one()) ------------------------------
      Walk w(p, c, C);
      Job j;
      int stage = 0; uint32_t phase = 0, job_i = 0;
      bool ok = true;
      auto arrived = [&]() {
        ok = wait_warp(smem_u32(&ctrl->full[stage]), phase, &ctrl->abort, p.wait_ns);
        tc_fence_after();
        return ok;
      };
      auto advance = [&]() { if (++stage == stages) { stage = 0; phase ^= 1u; } };
      while (ok && w.next(j)) {
        const int blocks = job_blocks(j), whole = (j.k16 + 3) / 4;
        if (blocks == 0) continue;               // (nothing to contract: the epilogue writes zeros)
        const int chain = CHAINED ? job_chain(p, j) : 1 << 30;
        int left = 0;                            // blocks until the accumulator changes
        const bool a_mn = KIND == kProducts, b_mn = j.type >= kTables;
        const uint32_t idesc = idesc_bf16_f32(kTile, j.n) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u);
        uint32_t acc = 0, D = 0;
        // (a descriptor's address counts 16 bytes in its low bits: a step of 16 is 32 bytes on in a K-major operand, 2048 in
        // an MN-major one)
        const uint64_t a_kind = a_mn ? smem_desc_mn(0) : smem_desc_sw128(0), b_kind = b_mn ? smem_desc_mn(0) : smem_desc_sw128(0);
        const uint32_t a_step = a_mn ? 128u : 2u, b_step = b_mn ? 128u : 2u;
        auto mma = [&](uint32_t A, uint32_t B, int steps) {        // by one lane
          const uint64_t a = a_kind + (A >> 4), b = b_kind + (B >> 4);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (k < steps) umma_bf16_pair(D, a + k * a_step, b + k * b_step, idesc, k ? 1u : acc);
        };
        const int turns = MULTI || !CHAINED ? 1 : job_turns(p, j.type);
        for (int i = 0, kb = 0; i < blocks * turns; ++i, kb = kb + 1 == blocks ? 0 : kb + 1) {
          if (left == 0) {
            if (i) { if (elect_one()) umma_commit_pair(smem_u32(&ctrl->acc_full[job_i & 1u])); __syncwarp(); ++job_i; }
            ok = wait_warp(smem_u32(&ctrl->acc_empty[job_i & 1u]), ((job_i >> 1) & 1u) ^ 1u, &ctrl->abort, p.wait_ns);
            if (!ok) break;
            tc_fence_after();
            D = tmem_base + (job_i & 1u) * kTile;
            acc = 0;
            left = chain;
          }
          --left;
          const int steps = kb >= whole ? 1 : min(4, j.k16 - 4 * kb);
          if constexpr (MULTI) {
            // The six products of parts that fp32 can hold, the smallest first: the accumulator has its size only for the last
            // one, and what truncation there is counts from then on.
            uint32_t at[6], bar[6];
            auto take = [&](int i) {
              at[i] = stage_base + (uint32_t)stage * 16384u;
              bar[i] = smem_u32(&ctrl->empty[stage]);
              if (!arrived()) return false;
              advance();
              return true;
            };
            if (!take(0) || !take(1)) break;                                 // A2, B0
            if (elect_one()) mma(at[0], at[1], steps);
            __syncwarp();
            acc = 1;
            if (!take(2) || !take(3)) break;                                 // A0, B2
            if (elect_one()) { mma(at[2], at[3], steps); umma_commit_pair(bar[0]); umma_commit_pair(bar[3]); }
            __syncwarp();
            if (!take(4) || !take(5)) break;                                 // A1, B1
            if (elect_one()) {
              mma(at[4], at[5], steps); mma(at[4], at[1], steps); mma(at[2], at[5], steps); mma(at[2], at[1], steps);
              umma_commit_pair(bar[1]); umma_commit_pair(bar[2]); umma_commit_pair(bar[4]); umma_commit_pair(bar[5]);
            }
            __syncwarp();
          } else {
            if (!arrived()) break;
            const uint32_t at = stage_base + (uint32_t)stage * stage_bytes;
            if (elect_one()) {
              mma(at, at + b_off, steps);
              umma_commit_pair(smem_u32(&ctrl->empty[stage]));
            }
            __syncwarp();
            acc = 1;
            advance();
          }
        }
        if (!ok) break;
        if (elect_one()) umma_commit_pair(smem_u32(&ctrl->acc_full[job_i & 1u]));
        __syncwarp();
        ++job_i;
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsEpi));
    // ---------------- epilogue (both CTAs): thread = row of the result and 128 of its columns ------------------
    const int q = warp & 3, half = (warp - 4) >> 2;
    const int in_cta = q * 32 + lane, in_tile = rank * 128 + in_cta;
    Turn turn{reinterpret_cast<uint4*>(sm + 1024 + (warp - 4) * 2 * kTurnBytes), 0, lane};
    uint32_t acc_empty_leader[2];
    acc_empty_leader[0] = map_to_cta(smem_u32(&ctrl->acc_empty[0]), 0);
    acc_empty_leader[1] = map_to_cta(smem_u32(&ctrl->acc_empty[1]), 0);
    const float scale = __int_as_float(p.pl.head[4]);
    Walk w(p, c, C);
    Job j;
    uint32_t job_i = 0;
    bool ok = true;
    while (w.next(j)) {
      const int blocks = job_blocks(j) * (MULTI || !CHAINED ? 1 : job_turns(p, j.type)), chain = CHAINED ? job_chain(p, j) : 1 << 30;
      const bool some = blocks > 0;
      // the tile's sums, after which its accumulators are free
      float acc[2][64];                          // columns 128 half + 64 u + x
      if (CHAINED || !some) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int x = 0; x < 64; ++x) acc[u][x] = 0.f;
      }
      for (int at = ok ? 0 : blocks; at < blocks; at += min(chain, blocks)) {
        ok = wait_warp(smem_u32(&ctrl->acc_full[job_i & 1u]), (job_i >> 1) & 1u, &ctrl->abort, p.wait_ns);
        if (!ok) break;
        tc_fence_after();
        const uint32_t from = tmem_base + ((uint32_t)(q * 32) << 16) + (job_i & 1u) * kTile + 128 * half;
        if (CHAINED) {
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            if (128 * half + 32 * g < j.n) {
              uint32_t v[32];
              tmem_ld32(from + 32 * g, v);
              tmem_ld_wait();
#pragma unroll
              for (int x = 0; x < 32; ++x) acc[g >> 1][32 * (g & 1) + x] += __uint_as_float(v[x]);
            }
          }
        } else {
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            if (128 * half + 64 * u < j.n) {
              uint32_t v[2][32];
              tmem_ld32(from + 64 * u, v[0]);
              if (128 * half + 64 * u + 32 < j.n) tmem_ld32(from + 64 * u + 32, v[1]);
              tmem_ld_wait();
#pragma unroll
              for (int x = 0; x < 64; ++x) acc[u][x] = __uint_as_float(v[x >> 5][x & 31]);
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_relaxed(acc_empty_leader[job_i & 1u]);
        ++job_i;
      }
      if (!ok) {                                 // a wait gave up: NaN in place of this tile, and of all that follow
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int x = 0; x < 64; ++x) acc[u][x] = __int_as_float(0x7fc00000);
      }
      if constexpr (KIND != kProducts) {
        const bool hy = j.b >= 0;
        const int cta_rows = hy ? p.th >> 1 : p.cta_rows, row = rank * cta_rows + in_cta;       // of the tile
        const bool there = in_cta < cta_rows && row < j.limit;
        const int pos = (hy ? p.pl.s0[j.b] : 0) + j.m0 + row;
        float4 r = make_float4(0.f, 0.f, __int_as_float(-1), __int_as_float(0));
        if (there) r = p.pl.meta[pos];
        const int at = __float_as_int(r.z) - (hy ? p.cb.V : p.v0) - j.r0 - 128 * half;          // the target's column here, if it has it
        const int see = !there ? 0 : min((hy ? min(__float_as_int(r.w), p.cb.n[j.b]) : p.vn) - j.r0, j.n) - 128 * half;     // columns that the row sees
        // rows up to the next multiple of 32 get zeros (or none): they are contracted in steps of 16
        const int first = rank * cta_rows + q * 32;
        const int rows = min(min(32, cta_rows - q * 32), pad32(j.limit) - first);
        const int row0 = (hy ? p.pl.h0[j.b] : 0) + j.m0 + first;
        __nv_bfloat16* out = (hy ? p.gh + (size_t)row0 * p.gh_pitch : p.g + (size_t)row0 * p.g_pitch) + j.r0 + 128 * half;
        const long long pitch = 2ll * (hy ? p.gh_pitch : p.g_pitch);
        if constexpr (KIND == kGrad) {
          const long long plane = hy ? p.gh_plane : p.g_plane;
          const float lse = r.x, weight = r.y, rest = there ? p.pl.rest[pos] : 0.f;
          const int show = weight != 0.f ? see : 0;
          const bool all = __all_sync(0xffffffffu, show >= 128);
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const int cols = min(64, j.n - 128 * half - 64 * u);
            if (cols <= 0 || rows <= 0) continue;
            float (&v)[64] = acc[u];
            // (the target's, p - 1, from its logit: of a row that is sure of it p is 1 after rounding)
            const bool target = __any_sync(0xffffffffu, at >= 64 * u && at < 64 * u + 64);
            float l = 0.f;
            if (target) {
#pragma unroll
              for (int x = 0; x < 64; ++x) l = x == at - 64 * u ? v[x] : l;
            }
            if (p.exact_exp) {
#pragma unroll
              for (int x = 0; x < 64; ++x) v[x] = exp_exact(v[x], lse, rest);
            } else {
#pragma unroll
              for (int x = 0; x < 64; ++x) v[x] = ex2((v[x] - lse) * kLog2e);
            }
            if (target) {
              l = expm1f((l - lse) - rest);
#pragma unroll
              for (int x = 0; x < 64; ++x) v[x] = x == at - 64 * u ? l : v[x];
            }
#pragma unroll
            for (int x = 0; x < 64; ++x) v[x] *= weight;
            if (!all) {
#pragma unroll
              for (int x = 0; x < 64; ++x) v[x] = x < show - 64 * u ? v[x] : 0.f;
            }
            for (int part = 0; part < p.g_parts; ++part) {
              uint32_t o[32];
#pragma unroll
              for (int x = 0; x < 32; ++x) o[x] = pack_bf16(v[2 * x], v[2 * x + 1]);
              if (part + 1 < p.g_parts) {
#pragma unroll
                for (int x = 0; x < 32; ++x) {
                  v[2 * x] -= __uint_as_float(o[x] << 16);
                  v[2 * x + 1] -= __uint_as_float(o[x] & 0xffff0000u);
                }
              }
              if (rows == 32) turn.tma<false>(o, hy ? &tm.gh_s : &tm.g_s, j.r0 + 128 * half + 64 * u, row0, part);
              else turn.lines<false>(o, reinterpret_cast<char*>(out + (size_t)part * plane + 64 * u), pitch, rows, 2 * cols);
            }
          }
        } else {
          if (!__all_sync(0xffffffffu, see >= 128)) {
#pragma unroll
            for (int x = 0; x < 128; ++x) acc[x >> 6][x & 63] = x < see ? acc[x >> 6][x & 63] : -INFINITY;
          }
          if (__any_sync(0xffffffffu, at >= 0 && at < 128)) {
            float l = acc[0][0];
#pragma unroll
            for (int x = 1; x < 128; ++x) l = x == at ? acc[x >> 6][x & 63] : l;
            if (at >= 0 && at < 128 && at < see) p.tl[pos] = l;
          }
          float m = acc[0][0], s = 0.f;
#pragma unroll
          for (int x = 1; x < 128; ++x) m = fmaxf(m, acc[x >> 6][x & 63]);
          bool nan = false;
          if (m == -INFINITY) {                  // nothing here, or NaN
#pragma unroll
            for (int x = 0; x < 128; ++x) nan |= acc[x >> 6][x & 63] != acc[x >> 6][x & 63];
          } else {
            float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 0; x < 128; ++x) part[x & 3] += ex2((acc[x >> 6][x & 63] - m) * kLog2e);
            s = (part[0] + part[1]) + (part[2] + part[3]);
            nan = s != s;                        // (+inf: inf - inf)
          }
          if (there) {
            float2* ms = hy ? p.part_h + (size_t)(j.part + half) * p.part_rows_h + pos : p.part + (size_t)(j.part + half) * p.part_rows + pos - p.r_lo;
            *ms = nan ? make_float2(INFINITY, __int_as_float(0x7fc00000)) : make_float2(m, s);
          }
          if constexpr (KIND == kKeep) {
            // (a row of NaN has a NaN lse, whatever is kept of it)
            auto steps = [&](float l) { return m == -INFINITY ? kKeepNone : min(__float2uint_rn((m - l) * kKeepSteps), kKeepNone); };
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const int cols = min(64, j.n - 128 * half - 64 * u);
              if (cols <= 0 || rows <= 0) continue;
              uint32_t o[32];
#pragma unroll
              for (int x = 0; x < 32; ++x) o[x] = steps(acc[u][2 * x]) | steps(acc[u][2 * x + 1]) << 16;
              if (rows == 32) turn.tma<false>(o, hy ? &tm.gh_s : &tm.g_s, j.r0 + 128 * half + 64 * u, row0, 0);
              else turn.lines<false>(o, reinterpret_cast<char*>(out + 64 * u), pitch, rows, 2 * cols);
            }
          }
        }
      } else if (j.type == kHidden || j.type == kHiddenHyper) {
        const int m = j.m0 + in_tile, pos0 = (j.b >= 0 ? p.pl.s0[j.b] : 0) + j.r0;
        const bool set = p.first || j.type == kHiddenHyper;
        float* out = p.dh + (size_t)j.part * p.dh_slot + (size_t)(pos0 + 128 * half) * p.d + m;
        const int limit = j.limit - 128 * half;
        if (m < p.d && (some || set)) {
#pragma unroll
          for (int x0 = 0; x0 < 128; x0 += 32) {
            if (x0 >= limit) break;
            if (!set) {
              float old[32];
#pragma unroll
              for (int x = 0; x < 32; ++x) old[x] = x0 + x < limit ? __ldcg(out + (size_t)(x0 + x) * p.d) : 0.f;
#pragma unroll
              for (int x = 0; x < 32; ++x) acc[(x0 + x) >> 6][(x0 + x) & 63] += old[x];
            }
#pragma unroll
            for (int x = 0; x < 32; ++x)
              if (x0 + x < limit) out[(size_t)(x0 + x) * p.d] = acc[(x0 + x) >> 6][(x0 + x) & 63];
          }
        }
      } else if (some || !p.acc) {
        const int first = j.m0 + rank * 128 + q * 32, rows = (j.b >= 0 ? p.cb.n[j.b] : p.vn) - first;
        const float mul = some ? scale : 0.f;
        TO* out = (j.b >= 0 ? reinterpret_cast<TO*>(p.gUh) + ((size_t)j.b * p.cb.cap + first) * p.d
                            : reinterpret_cast<TO*>(p.gWU) + (size_t)(p.v0 + first) * p.d) + j.r0 + 128 * half;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int cols = min(min(j.n, p.d - j.r0) - 128 * half - 64 * u, 64);
          if (rows <= 0 || cols <= 0) continue;
#pragma unroll
          for (int x = 0; x < 64; ++x) acc[u][x] *= mul;
          const CUtensorMap* m = j.b < 0 ? &tm.o_w : nullptr;
          if (p.acc) store_columns<TO, true>(acc[u], turn, m, j.r0 + 128 * half + 64 * u, p.v0 + first, out + 64 * u, p.d, rows, cols);
          else store_columns<TO, false>(acc[u], turn, m, j.r0 + 128 * half + 64 * u, p.v0 + first, out + 64 * u, p.d, rows, cols);
        }
      }
    }
    if (lane == 0) bulk_wait_all();
  }
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && ctrl->abort) {
    atomicOr(p.err, 1);
    p.pl.head[5] = 1;
    st_cluster_u32(map_to_cta(smem_u32(&ctrl->other_abort), rank ^ 1), 1u);
  }
  __syncwarp();
  cluster_sync_all();                            // nobody leaves while the pair's MMAs may read its memory
  if (ctrl->abort | ctrl->other_abort) {
    // A role that gave up, in either CTA, has left what the others had under way: the loads land and the MMAs end first.
    if (warp == 1) {
      if (rank == 0 && elect_one()) umma_commit_pair(smem_u32(&ctrl->done));
      __syncwarp();
      if (lane == 0) drain(smem_u32(&ctrl->done), 0);
    }
    if (rank == 0 && threadIdx.x == 0) drain_loads(ctrl, stages);
    __syncthreads();
    cluster_sync_all();
  }
  if (warp == 2) tmem_dealloc_pair(tmem_base, 512);
}

// Sixteen rows per block and 64 threads each: the partial sums of its vocabulary and hypertoken tiles, its loss and lse.
// With gradients to follow (parts_of_rows > 0) lse also goes to the plan, and the copies of a hidden row without weight are
// zeroed: they are contracted with g = 0, whatever they hold.
__global__ void __launch_bounds__(1024) k_xent_merge(CbView cb, RowArgs a, Plan pl, const float2* part, int part_rows, int parts,
                                                    const float2* part_h, int part_rows_h, const float* tl, int r_lo, int r_hi,
                                                    GatherArgs g, int parts_of_rows) {
  pdl_wait();
  pdl_trigger();
  constexpr int kRows = 16, kSlices = 1024 / kRows;
  __shared__ float2 s_ms[kRows][kSlices + 1];
  // neighbouring threads read neighbouring rows
  const int x = threadIdx.x % kRows, y = threadIdx.x / kRows, p0 = r_lo + blockIdx.x * kRows, end = min(pl.head[0], r_hi);
  float m = -INFINITY, s = 0.f;
  if (p0 + x < end) {
    auto all = [&](const float2* from, size_t stride, int count) {
      constexpr int kAhead = 8;
      for (int i = y; i < count; i += kSlices * kAhead) {
        float2 v[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) v[u] = i + kSlices * u < count ? __ldcg(from + (size_t)(i + kSlices * u) * stride) : make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) merge_ms(m, s, v[u].x, v[u].y);
      }
    };
    all(part + p0 + x - r_lo, part_rows, parts);
    // (tiles beyond what the row sees have nothing for it)
    if (cb.cap > 0) all(part_h + p0 + x, part_rows_h, 2 * ceil_div(__float_as_int(pl.meta[p0 + x].w), kTile));
  }
  s_ms[x][y] = make_float2(m, s);
  __syncthreads();
  // a warp per row from here on
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, pos = p0 + w;
  if (w >= kRows || pos >= end) return;
  m = s_ms[w][lane].x; s = s_ms[w][lane].y;
  for (int i = 32; i < kSlices; i += 32) merge_ms(m, s, s_ms[w][lane + i].x, s_ms[w][lane + i].y);
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const float om = __shfl_xor_sync(0xffffffffu, m, o), os = __shfl_xor_sync(0xffffffffu, s, o);
    // (both lanes of a pair add in the same order)
    if (lane & o) { float lm = om, ls = os; merge_ms(lm, ls, m, s); m = lm; s = ls; }
    else merge_ms(m, s, om, os);
  }
  const int row = pl.perm[pos];
  if (lane == 0) {
    // (64 bits: what lse loses to its rounding is kept, and a logarithm of 8 to 16 is off by as much in 32)
    const double ls = log((double)s), sum = (double)m + ls;
    const float lse = (float)sum;
    a.lse_out[row] = lse;
    a.loss_out[row] = (float)(ls + ((double)m - (double)tl[pos]));
    if (parts_of_rows) { pl.meta[pos].x = lse; pl.rest[pos] = fabsf(lse) < INFINITY ? (float)(sum - lse) : 0.f; }
  }
  if (parts_of_rows && pl.meta[pos].y == 0.f) {
    const int h = pl.place[pos].x;
    for (int i = 0; i < parts_of_rows; ++i) {
      put_row<__nv_bfloat16>(nullptr, g.hs + (size_t)i * g.hs_plane + (size_t)pos * g.d, 0, g.d, lane, 32);
      if (g.hh) put_row<__nv_bfloat16>(nullptr, g.hh + (size_t)i * g.hh_plane + (size_t)h * g.d, 0, g.d, lane, 32);
    }
  }
}

// g from what kKeep has left, in its place: p = exp(m - steps / 2048 - lse), the target's from its own logit.  A block takes
// 32768 columns of a row, the next vectors under way while it works on the last; rows up to the next multiple of 32 become
// zeros.
struct KeptArgs { __nv_bfloat16* g; int pitch; const float2* part; int part_rows, nv; };
constexpr int kKeptThreads = 256, kKeptVecs = 2, kKeptStep = 8 * kKeptThreads * kKeptVecs, kKeptColumns = 32768;
// see: columns that the row sees; those behind them up to `cols` become zeros.  less_one: p - 1 of the target.
__device__ __forceinline__ void kept_columns(uint16_t* g, int lo, int cols, int see, const float2* part, int part_rows, int nv, const float4& r, int target,
                                             float less_one) {
  const float lse = r.x, weight = r.y, none = lse - lse;                     // (0, or NaN for a row of NaN)
  const int hi = min(cols, lo + kKeptColumns), v0 = lo + 8 * (int)threadIdx.x;
  uint4 w[kKeptVecs];
  float from[kKeptVecs];
  auto load = [&](int v) {
#pragma unroll
    for (int u = 0; u < kKeptVecs; ++u, v += 8 * kKeptThreads) {
      if (v >= hi) break;
      w[u] = *reinterpret_cast<const uint4*>(g + v);
      int slot = v >> 7;                         // half tiles of 128, unless a tile is shorter than 256
      if (nv != kTile) { const int vt = v / nv; slot = 2 * vt + ((v - vt * nv) >> 7); }
      from[u] = part[(size_t)slot * part_rows].x;
    }
  };
  load(v0);
  for (int v = v0; v < hi; v += kKeptStep) {
    uint4 now[kKeptVecs];
    float top[kKeptVecs];
#pragma unroll
    for (int u = 0; u < kKeptVecs; ++u) { now[u] = w[u]; top[u] = (from[u] - lse) * kLog2e; }
    load(v + kKeptStep);
#pragma unroll
    for (int u = 0; u < kKeptVecs; ++u) {
      const int c = v + u * 8 * kKeptThreads;
      if (c >= hi) break;
      const uint32_t in[4] = {now[u].x, now[u].y, now[u].z, now[u].w};
      float x[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint32_t q = k & 1 ? in[k >> 1] >> 16 : in[k >> 1] & 0xffffu;
        // (a whole number below 2^16 as a float: in the low bits of 2^23, less that)
        const float steps = __uint_as_float(0x4b000000u | q) - 8388608.f;
        x[k] = weight * (q == kKeepNone ? none : ex2(fmaf(steps, -kLog2e / kKeepSteps, top[u])));
      }
      if (weight == 0.f || c + 8 > see) {
#pragma unroll
        for (int k = 0; k < 8; ++k) if (weight == 0.f || c + k >= see) x[k] = 0.f;
      }
      if (target >= c && target < c + 8 && weight != 0.f) {
        const float e = weight * less_one;
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = c + k == target ? e : x[k];
      }
      *reinterpret_cast<uint4*>(g + c) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    }
  }
}
__global__ void __launch_bounds__(kKeptThreads, 5) k_xent_kept(CbView cb, RowArgs a, Plan pl, KeptArgs w, KeptArgs u, const float* tl, int chunks, int hyper) {
  pdl_wait();
  pdl_trigger();
  const int live = pl.head[0];
  const long long units = (long long)pad32(live) * (chunks + hyper);
  for (long long i = blockIdx.x; i < units; i += gridDim.x) {
    const int pos = (int)(i / (chunks + hyper)), chunk = (int)(i - (long long)pos * (chunks + hyper));
    const float4 r = pos < live ? pl.meta[pos] : make_float4(0.f, 0.f, __int_as_float(-1), 0.f);
    const float t = pos < live ? expm1f((tl[pos] - r.x) - pl.rest[pos]) : 0.f;
    const int target = __float_as_int(r.z);
    if (chunk < chunks) {
      kept_columns(reinterpret_cast<uint16_t*>(w.g) + (size_t)pos * w.pitch, chunk * kKeptColumns, pad64(cb.V), cb.V, w.part + pos, w.part_rows, w.nv, r,
                   target < cb.V ? target : -1, t);
      continue;
    }
    if (pos >= live) continue;
    // hypertokens, and the zeros up to the sequence's next multiple of 32
    const int row = pl.perm[pos], b = a.row_seq ? a.row_seq[row] : row, n = pad32(cb.n[b]), lo = (chunk - chunks) * kKeptColumns;
    if (lo >= n) continue;
    const int2 place = pl.place[pos];
    kept_columns(reinterpret_cast<uint16_t*>(u.g) + (size_t)place.x * u.pitch, lo, n, __float_as_int(r.w), u.part + pos, u.part_rows, u.nv, r, target - cb.V, t);
    for (int k = 1; k <= place.y; ++k)
      for (int v = lo + threadIdx.x * 8; v < min(n, lo + kKeptColumns); v += kKeptThreads * 8)
        *reinterpret_cast<uint4*>(u.g + (size_t)(place.x + k) * u.pitch + v) = make_uint4(0u, 0u, 0u, 0u);
  }
}

// dh of a row: its partial sums, those of the vocabulary's parts first, times the largest weight.
// The tiles of dh contract all entries of a sequence, with g = 0 for those that a row does not see; where these are not finite
// (not computed yet, maybe) the row's sum over the entries that it does see is taken here, one by one.  A call without
// such entries pays a comparison; with them 333 rows that see up to 160 entries take 43 us more (d = 1024; the step 248), 3680 rows
// of up to 760 1.2 ms (d = 4096; the step 9.1 ms).
struct SeenArgs { const __nv_bfloat16* gh; long long plane; int pitch, parts; const void* Uh; const int32_t* row_seq; };
template <typename T>
__global__ void __launch_bounds__(128) k_xent_hidden(CbView cb, Plan pl, const float* dh, long long slot, int split, SeenArgs u, T* out, int d) {
  pdl_wait();
  pdl_trigger();
  const int r = blockIdx.x, pos = pl.inv[r], i = (blockIdx.y * 128 + threadIdx.x) * 8;
  if (i >= d) return;
  // (the last: hypertokens, if it sees any.  Without weight: none, since 0 times what the tables hold may be NaN)
  const int slots = pos < 0 || pl.meta[pos].y == 0.f ? 0 : split + (__float_as_int(pl.meta[pos].w) > 0 ? 1 : 0);
  float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  const float* from = dh + (size_t)(pos < 0 ? 0 : pos) * d + i;
  constexpr int kAhead = 4;
  for (int k0 = 0; k0 < slots; k0 += kAhead) {
    float4 v[kAhead][2];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (k0 + k >= slots) break;
      v[k][0] = __ldcg(reinterpret_cast<const float4*>(from + (size_t)(k0 + k) * slot));
      v[k][1] = __ldcg(reinterpret_cast<const float4*>(from + (size_t)(k0 + k) * slot + 4));
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (k0 + k >= slots) break;
      s[0] += v[k][0].x; s[1] += v[k][0].y; s[2] += v[k][0].z; s[3] += v[k][0].w;
      s[4] += v[k][1].x; s[5] += v[k][1].y; s[6] += v[k][1].z; s[7] += v[k][1].w;
    }
  }
  if (slots > split) {
    bool finite = true;
#pragma unroll
    for (int k = 0; k < 8; ++k) finite &= fabsf(s[k]) < INFINITY;
    const float4 m = pl.meta[pos];
    if (!finite && fabsf(m.x) < INFINITY && fabsf(m.y) < INFINITY && !pl.head[5]) {
#pragma unroll
      for (int k = 0; k < 8; ++k) s[k] = 0.f;
      for (int j = 0; j < split; ++j)
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] += __ldcg(from + (size_t)j * slot + k);
      const T* entry = reinterpret_cast<const T*>(u.Uh) + (size_t)(u.row_seq ? u.row_seq[r] : r) * cb.cap * d + i;
      const __nv_bfloat16* g = u.gh + (size_t)pl.place[pos].x * u.pitch;
      const int last = u.parts > 1 ? 1 : 0;      // (one part, or three)
#pragma unroll 8
      for (int e = 0; e < __float_as_int(m.w); ++e, entry += d) {
        const float w = __bfloat162float(g[e]) + last * (__bfloat162float(g[last * u.plane + e]) + __bfloat162float(g[2 * last * u.plane + e]));
        float x[8];
        if constexpr (sizeof(T) == 4) {
          const float4 a = *reinterpret_cast<const float4*>(entry), b = *reinterpret_cast<const float4*>(entry + 4);
          x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
        } else {
          const uint4 a = *reinterpret_cast<const uint4*>(entry);
          const uint32_t o[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) { x[2 * k] = __uint_as_float(o[k] << 16); x[2 * k + 1] = __uint_as_float(o[k] & 0xffff0000u); }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] = fmaf(w, x[k], s[k]);
      }
    }
  }
  if (slots) {
    const float scale = __int_as_float(pl.head[4]);
#pragma unroll
    for (int k = 0; k < 8; ++k) s[k] *= scale;
  }
  T* to = out + (size_t)r * d + i;
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(to) = make_float4(s[0], s[1], s[2], s[3]);
    *reinterpret_cast<float4*>(to + 4) = make_float4(s[4], s[5], s[6], s[7]);
  } else {
    *reinterpret_cast<uint4*>(to) = make_uint4(pack_bf16(s[0], s[1]), pack_bf16(s[2], s[3]), pack_bf16(s[4], s[5]), pack_bf16(s[6], s[7]));
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
std::atomic<unsigned long long> g_xent_wait_ns{kWaitLimitNs};

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
  bool keep;                                     // a step whose logits are kept from the losses to the gradients
  int np, nh;                                    // rows of the sorted copy, and beside hypertokens
  int cta_rows, nv;
  int tr, th, dt, split;
  int pieces, vc;                                // vocabulary rows per piece, a multiple of 256
};

Shape shape_of(const z2z_config& c, int N, int grad_dtype, long long vc, bool keep) {
  Shape s{};
  s.N = N; s.d = c.d; s.V = c.V; s.B = c.B; s.cap = c.cap; s.dtype = c.dtype; s.grad_dtype = grad_dtype; s.keep = keep;
  s.parts = c.dtype == Z2Z_DTYPE_FP32 ? kMaxParts : 1;
  s.g_parts = grad_dtype < 0 ? 0 : (s.parts > 1 || grad_dtype == Z2Z_DTYPE_FP32 ? kMaxParts : 1);
  s.np = (int)up_to(N, kTile);
  s.nh = (int)up_to((long long)N + (long long)(kHyperPad - 1) * (N < c.B ? N : c.B), kTile);
  s.cta_rows = N > 192 ? 128 : (int)up_to((N + 1) / 2, 16);
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
  if (vc > whole || keep) vc = whole;
  s.pieces = (int)((c.V + vc - 1) / vc);
  s.vc = (int)up_to((c.V + s.pieces - 1) / s.pieces, kTile);
  s.pieces = (c.V + s.vc - 1) / s.vc;
  // Vocabulary rows per tile: the number of rounds of all clusters times the rows that a CTA loads for a tile (and something).
  // Multiples of 64, since G's tiles are stored in blocks of 64 columns.
  s.nv = kTile;
  const int row_tiles = (N + 2 * s.cta_rows - 1) / (2 * s.cta_rows);
  long long best = -1;
  for (int nv = kTile; nv >= 128; nv -= 64) {
    const long long rounds = ((long long)row_tiles * ((s.vc + nv - 1) / nv) + kClusters - 1) / kClusters, cost = rounds * (s.cta_rows + nv / 2 + 16);
    if (best < 0 || cost < best) { best = cost; s.nv = nv; }
  }
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
// Rows whose partial sums are held at a time.
int loss_rows(const Shape& s) { return s.keep || s.np < kLossRows ? s.np : kLossRows; }

// (A step's; what the gradients alone do not use is small beside the rest.)
Layout layout_of(const Shape& s, char* base) {
  Layout l{};
  size_t o = 0;
  auto take = [&](size_t bytes) { char* r = base + o; o = (size_t)up_to((long long)(o + bytes), 256); return r; };
  const size_t row = (size_t)s.d * 2 * s.parts;
  l.pl.head = (int32_t*)take(32);
  l.pl.cnt = (int32_t*)take((size_t)s.B * 4);
  int32_t** tables[] = {&l.pl.s0, &l.pl.h0, &l.pl.j1, &l.pl.j2, &l.pl.j3};
  for (int32_t** t : tables) *t = (int32_t*)take((size_t)(s.B + 1) * 4);
  l.pl.perm = (int32_t*)take((size_t)s.np * 4); l.pl.inv = (int32_t*)take((size_t)s.np * 4);
  l.pl.place = (int2*)take((size_t)s.np * 8);
  l.pl.meta = (float4*)take((size_t)s.np * 16); l.pl.rest = (float*)take((size_t)s.np * 4);
  l.hs = (__nv_bfloat16*)take(row * s.np);
  if (s.cap > 0) {
    l.hh = (__nv_bfloat16*)take(row * s.nh);
    if (s.parts > 1) l.up = (__nv_bfloat16*)take(row * s.B * s.cap);
  }
  if (s.parts > 1) l.wp = (__nv_bfloat16*)take(row * s.vc);
  l.part = (float2*)take((size_t)2 * s.pieces * vocabulary_tiles(s.vc, s.nv) * loss_rows(s) * 8);
  if (s.cap > 0) l.part_h = (float2*)take((size_t)2 * (hyper_rows(s) / kTile) * s.np * 8);
  l.tl = (float*)take((size_t)s.np * 4);
  if (s.grad_dtype >= 0) {
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

// Vocabulary rows of a piece: G of 256 MB (8192 rows at least).  fp32 tables are also held in parts.
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

// A step may keep its logits (16 bits each) instead of computing them again for the gradients, which are a quarter of its
// products: where g is a single part and the scratch has room, of which at most 4 GB are asked for.
bool may_keep(const z2z_config& c, int N, int grad_dtype) {
  return grad_dtype == Z2Z_DTYPE_BF16 && c.dtype == Z2Z_DTYPE_BF16 && up_to(N, kTile) * up_to(c.V, kTile) * 2 <= 4ll << 30;
}

size_t bytes_with(const z2z_config& c, int N, int grad_dtype, long long vc, bool keep) {
  return layout_of(shape_of(c, N, grad_dtype, vc, keep), nullptr).bytes;
}

// The largest pieces up to the wanted ones for which the scratch suffices; 0 if none.
long long piece_for(const z2z_config& c, int N, int grad_dtype, size_t bytes) {
  long long vc = wanted_piece(c, N, grad_dtype);
  for (;;) {
    if (bytes_with(c, N, grad_dtype, vc, false) <= bytes) return vc;
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

// Map over `planes` matrices [rows, cols] of bf16 (or fp32), rows `pitch` elements apart; box = 128 bytes x box_rows rows of one.
bool make_map(CUtensorMap* m, const void* base, long long rows, long long cols, long long pitch, int planes, long long plane, int box_rows,
              bool f32 = false) {
  const EncodeFn fn = encode_fn();
  if (!fn || rows < 1 || cols < 1) return false;
  const int es_ = f32 ? 4 : 2;
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
  const cuuint64_t strides[2] = {(cuuint64_t)pitch * es_, (cuuint64_t)(planes > 1 ? plane : rows * pitch) * es_};
  const cuuint32_t box[3] = {(cuuint32_t)(128 / es_), (cuuint32_t)box_rows, 1}, es[3] = {1, 1, 1};
  return fn(m, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int KIND, bool CHAINED, bool MULTI, typename TO>
cudaError_t launch_main(const Params& p, const Maps& tm, int clusters, cudaStream_t s) {
  auto kern = k_xent<KIND, CHAINED, MULTI, TO>;
  static const int regs = [&] { cudaFuncAttributes a{}; return cudaFuncGetAttributes(&a, kern) == cudaSuccess ? a.numRegs : 0; }();
  if (regs < kRegsAtLaunch) return cudaErrorInvalidConfiguration;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes);
  if (e != cudaSuccess) return e;
  return launch_pdl(kern, dim3(2 * clusters), dim3(kThreads), kSmemBytes, s, p, tm);
}
template <int KIND>
cudaError_t launch_logits(const Params& p, const Maps& tm, int clusters, cudaStream_t s) {
  if constexpr (KIND != kKeep)
    if (p.parts > 1) return launch_main<KIND, true, true, float>(p, tm, clusters, s);
  return p.d > 64 * kChain ? launch_main<KIND, true, false, float>(p, tm, clusters, s) : launch_main<KIND, false, false, float>(p, tm, clusters, s);
}

// Losses, gradients from lse, or both.
cudaError_t run_passes(const CbView& cb, const z2z_config& cfg, const XentArgs& x, cudaStream_t s) {
  const bool loss = x.want_loss, grad = x.want_grad;
  const int gd = grad ? x.grad_dtype : -1;
  const bool keep = loss && grad && may_keep(cfg, x.N, gd) && bytes_with(cfg, x.N, gd, 0, true) <= x.scratch_bytes;
  const long long vc = keep ? cfg.V : piece_for(cfg, x.N, gd, x.scratch_bytes);
  if (vc == 0) return cudaErrorMemoryAllocation;
  const Shape sh = shape_of(cfg, x.N, gd, vc, keep);
  const Layout l = layout_of(sh, x.scratch);
  const int d = sh.d, clusters = sm_count_xent() / 2;
  RowArgs a{};
  a.N = x.N; a.row_seq = x.row_seq; a.row_nvis = x.row_nvis; a.targets = x.targets;
  a.th = sh.th; a.dt = sh.dt;
  if (grad) { a.weight = x.weight; a.hidden = x.g_hidden != nullptr; a.tables = x.g_Uh != nullptr; }
  if (loss) { a.loss_out = x.loss; a.lse_out = x.lse; }
  else a.lse = x.lse;
  cudaError_t e = cudaFuncSetAttribute(k_xent_plan<kPlanThreads>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)plan_shared_bytes(1024));
  if (e != cudaSuccess) return e;
  e = sh.N <= 4 * kPlanFew && sh.B <= 32 ? launch_pdl(k_xent_plan<kPlanFew>, dim3(1), dim3(kPlanFew), plan_shared_bytes(sh.B), s, cb, a, l.pl)
                                         : launch_pdl(k_xent_plan<kPlanThreads>, dim3(1), dim3(kPlanThreads), plan_shared_bytes(sh.B), s, cb, a, l.pl);
  if (e != cudaSuccess) return e;
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
  p.cb = cb; p.pl = l.pl; p.d = d; p.dt = sh.dt; p.cta_rows = sh.cta_rows; p.nv = sh.nv; p.tr = sh.tr;
  p.a_bytes = (int)up_to(128ll * (sh.cap > 0 && sh.th / 2 > sh.cta_rows ? sh.th / 2 : sh.cta_rows), 1024); p.th = sh.th;
  p.parts = sh.parts;
  // (dh of a bf16 session is stored in bf16: of g's three parts for fp32 gradients it takes two, 16 bits)
  p.np2 = sh.parts > 1 ? 6 : (sh.g_parts > 1 ? 2 : 1); p.np3 = sh.parts > 1 ? 6 : sh.g_parts;
  p.g_parts = sh.g_parts; p.exact_exp = sh.g_parts > 1;
  p.g = l.g; p.g_pitch = sh.vc; p.g_plane = (long long)sh.vc * sh.np;
  p.gh = l.gh; p.gh_pitch = hyper_rows(sh); p.gh_plane = (long long)hyper_rows(sh) * sh.nh;
  p.part = l.part; p.part_h = l.part_h; p.part_rows = loss_rows(sh); p.part_rows_h = sh.np; p.tl = l.tl;
  p.split = sh.split; p.dh = grad && x.g_hidden ? l.dh : nullptr; p.dh_slot = (long long)sh.np * d;
  p.gWU = x.g_WU; p.gUh = sh.cap > 0 ? x.g_Uh : nullptr; p.acc = x.accumulate ? 1 : 0;
  p.mem_cycles = kTile * kTile * (x.grad_dtype == Z2Z_DTYPE_FP32 ? 4 : 2) * (x.accumulate ? 2 : 1) / 46;
  p.wait_ns = g_xent_wait_ns.load(std::memory_order_relaxed);
  p.err = x.err;
  // hidden rows of the row tiles that are taken through all vocabulary tiles together: a quarter of L2
  const long long tile_bytes = (long long)2 * sh.cta_rows * d * 2 * sh.parts;
  const long long sb = (32ll << 20) / tile_bytes;
  p.sb = (int)(sb < 1 ? 1 : (sb > 1024 ? 1024 : sb));

  Maps tm{};
  const long long ur = (long long)sh.B * sh.cap;
  bool ok = make_map(&tm.hs_k, l.hs, sh.np, d, d, sh.parts, g.hs_plane, sh.cta_rows);
  if (sh.cap > 0) {
    const void* U = sh.parts > 1 ? l.up : x.Uh;
    ok = ok && make_map(&tm.u_k, U, ur, d, d, sh.parts, g.up_plane, 128) && make_map(&tm.hh_k, l.hh, sh.nh, d, d, sh.parts, g.hh_plane, sh.th / 2);
    if (grad)
      ok = ok && make_map(&tm.u_m, U, ur, d, d, sh.parts, g.up_plane, 64) && make_map(&tm.ut_m, l.ut, sh.B * 16, d, d, sh.parts, g.ut_plane, 16) &&
           make_map(&tm.hh_m, l.hh, sh.nh, d, d, sh.parts, g.hh_plane, 64) &&
           make_map(&tm.gh_k, l.gh, sh.nh, hyper_rows(sh), hyper_rows(sh), sh.g_parts, p.gh_plane, sh.th / 2) &&
           make_map(&tm.gh_m, l.gh, sh.nh, hyper_rows(sh), hyper_rows(sh), sh.g_parts, p.gh_plane, 64) &&
           make_map(&tm.gh_s, l.gh, sh.nh, hyper_rows(sh), hyper_rows(sh), sh.g_parts, p.gh_plane, 32);
  }
  if (grad)
    ok = ok && make_map(&tm.hs_m, l.hs, sh.np, d, d, sh.parts, g.hs_plane, 64) &&
         make_map(&tm.g_k, l.g, sh.np, sh.vc, sh.vc, sh.g_parts, p.g_plane, sh.tr / 2) && make_map(&tm.g_m, l.g, sh.np, sh.vc, sh.vc, sh.g_parts, p.g_plane, 64) &&
         make_map(&tm.g_s, l.g, sh.np, sh.vc, sh.vc, sh.g_parts, p.g_plane, 32) &&
         (!x.g_WU || make_map(&tm.o_w, x.g_WU, sh.V, d, d, 1, 0, 32, x.grad_dtype == Z2Z_DTYPE_FP32));
  const void* W = sh.parts > 1 ? l.wp : x.WU;
  const long long w_rows = sh.parts > 1 ? sh.vc : sh.V, w_plane = (long long)sh.vc * d;
  ok = ok && make_map(&tm.w_k, W, w_rows, d, d, sh.parts, w_plane, 128) && make_map(&tm.w_m, W, w_rows, d, d, sh.parts, w_plane, 64);
  if (!ok) return cudaErrorInvalidValue;

  const int tiles = vocabulary_tiles(sh.vc, sh.nv);
  auto piece = [&](int i, bool again) {
    p.v0 = i * sh.vc; p.vn = sh.V - p.v0 < sh.vc ? sh.V - p.v0 : sh.vc;
    p.w_row0 = sh.parts > 1 ? 0 : p.v0;
    p.part0 = 2 * i * tiles;
    p.first = i == 0;
    if (sh.parts == 1 || (again && sh.pieces == 1)) return cudaSuccess;
    return launch_pdl(k_xent_split, dim3(p.vn < 4096 ? p.vn : 4096), dim3(128), 0, s, reinterpret_cast<const float*>(x.WU) + (size_t)p.v0 * d, l.wp, w_plane, p.vn, d);
  };
  if (loss) {
    const int share = loss_rows(sh) < x.N ? loss_rows(sh) : x.N;
    for (int r0 = 0; r0 < x.N; r0 += share) {
      p.r_lo = r0; p.r_hi = r0 + share < x.N ? r0 + share : x.N;
      for (int i = 0; i < sh.pieces; ++i) {
        p.hyper = i == 0 && r0 == 0 && sh.cap > 0;
        if ((e = piece(i, r0 > 0)) != cudaSuccess) return e;
        e = keep ? launch_logits<kKeep>(p, tm, clusters, s) : launch_logits<kLoss>(p, tm, clusters, s);
        if (e != cudaSuccess) return e;
      }
      const int parts = p.part0 + 2 * vocabulary_tiles(p.vn, sh.nv);
      e = launch_pdl(k_xent_merge, dim3((p.r_hi - p.r_lo + 15) / 16), dim3(1024), 0, s, cb, a, l.pl, l.part, p.part_rows, parts, l.part_h, sh.np, l.tl,
                     p.r_lo, p.r_hi, g, grad ? sh.parts : 0);
      if (e != cudaSuccess) return e;
    }
  }
  if (!grad) return cudaSuccess;
  if (keep) {
    const KeptArgs w{l.g, p.g_pitch, l.part, p.part_rows, sh.nv}, u{l.gh, p.gh_pitch, l.part_h, p.part_rows_h, kTile};
    const int chunks = (pad64(sh.V) + kKeptColumns - 1) / kKeptColumns, hyper = (sh.cap + kKeptColumns - 1) / kKeptColumns;
    if ((e = launch_pdl(k_xent_kept, dim3(148 * 5), dim3(kKeptThreads), 0, s, cb, a, l.pl, w, u, l.tl, chunks, hyper)) != cudaSuccess) return e;
  }
  p.r_lo = 0; p.r_hi = x.N;
  for (int i = 0; i < sh.pieces; ++i) {
    p.hyper = i == 0 && sh.cap > 0;
    p.hyper_hidden = p.hyper && p.dh;
    if ((e = piece(i, loss)) != cudaSuccess) return e;
    if (!keep && (e = launch_logits<kGrad>(p, tm, clusters, s)) != cudaSuccess) return e;
    if (x.grad_dtype == Z2Z_DTYPE_FP32)
      e = sh.parts > 1 ? launch_main<kProducts, true, true, float>(p, tm, clusters, s) : launch_main<kProducts, true, false, float>(p, tm, clusters, s);
    else
      e = sh.parts > 1 ? launch_main<kProducts, true, true, __nv_bfloat16>(p, tm, clusters, s) : launch_main<kProducts, false, false, __nv_bfloat16>(p, tm, clusters, s);
    if (e != cudaSuccess) return e;
  }
  if (!x.g_hidden) return cudaSuccess;
  const SeenArgs seen{l.gh, p.gh_plane, p.gh_pitch, p.g_parts, x.Uh, x.row_seq};
  const dim3 grid(x.N, (d + 1023) / 1024);
  return sh.dtype == Z2Z_DTYPE_FP32
             ? launch_pdl(k_xent_hidden<float>, grid, dim3(128), 0, s, cb, l.pl, l.dh, p.dh_slot, sh.split, seen, reinterpret_cast<float*>(x.g_hidden), d)
             : launch_pdl(k_xent_hidden<__nv_bfloat16>, grid, dim3(128), 0, s, cb, l.pl, l.dh, p.dh_slot, sh.split, seen, reinterpret_cast<__nv_bfloat16*>(x.g_hidden), d);
}

}  // namespace

void xent_wait_limit(unsigned long long ns) { g_xent_wait_ns.store(ns ? ns : kWaitLimitNs, std::memory_order_relaxed); }

void xent_scratch_bytes(const z2z_config& c, int N, int grad_dtype, size_t* least, size_t* most) {
  *least = *most = 0;
  if (N <= 0) return;
  *most = bytes_with(c, N, grad_dtype, wanted_piece(c, N, grad_dtype), false);
  // (smaller pieces may need more room for the losses' partial sums)
  *least = bytes_with(c, N, grad_dtype, kLeastPiece, false);
  if (*least > *most) *least = *most;
  if (may_keep(c, N, grad_dtype)) {
    const size_t kept = bytes_with(c, N, grad_dtype, 0, true);
    if (kept > *most) *most = kept;
  }
}

cudaError_t run_xent(const CbView& cb, const z2z_config& cfg, const XentArgs& a, cudaStream_t s) {
  if (a.N == 0) {
    if (!a.want_grad || a.accumulate || (!a.g_WU && !a.g_Uh)) return cudaSuccess;
    return launch_pdl(k_xent_zero, dim3(148 * 8), dim3(128), 0, s, cb, reinterpret_cast<char*>(a.g_WU), reinterpret_cast<char*>(a.g_Uh),
                      a.d * (a.grad_dtype == Z2Z_DTYPE_FP32 ? 4 : 2));
  }
  return run_passes(cb, cfg, a, s);
}

}  // namespace z2z
