// Distillation of joint logits from a teacher's top logits.  With l the row's logits over its C columns,
// q = softmax(l / T), and p = softmax(t / T) over the teacher's entries that the row can see:
//   loss = T^2 sum_j p_j (log p_j - log q_{id_j}),     d loss / d l_c = T (q_c - sum_{id_j = c} p_j).
//
// Two forms of one pass.  k_distill_stream takes many long rows (at least one for every two SMs, of 128 KB or more, with up
// to 512 entries): see there.  k_distill takes the others, a cluster of 1 to 8 blocks per row.  Every block reads its share of
// the columns once and folds it into a running maximum and sum of exponentials; every warp sends its pair to the shared
// memory of all blocks; one cluster barrier.  When the gradient is asked for, the share stays in shared memory until then (a
// thread only ever reads back what it has brought itself, so that its own copies' completion is all it waits for): the logits
// are read once and the gradient written once.  Rows longer than eight blocks hold (some 440000 fp32 columns) are read again.  The backward
// pass on its own is the same with the normaliser found anew: that is no byte more, and does not depend on what a stored
// lse has lost (2^-24 of |lse|, in every probability).
// Bound by HBM, for bf16 rows with little left: 2 exponentials a column, at 16 per clock and SM, take 0.7 of the bytes'
// time.  Hence the packed maxima, one update of the maximum per kFold vectors, and the factor of a bf16 gradient in
// the exponent.
// Exponents are kept base 2: z = c x - r with c = log2(e) / T, one fused operation, and r the rounded product of c with
// the maximum.  What r's rounding does to the terms it does to their sum, so that it drops out of q; it stays in lse, at
// one rounding of m / T.  Where |r| reaches kFar, whose rounding may be any number of powers of two, z = c (x - m) in two.
#include <cooperative_groups.h>

#include <atomic>
#include <cmath>
#include <type_traits>

#include "z2z_common.cuh"
#include "z2z_internal.h"
#include "z2z_sm100.cuh"

namespace z2z {

namespace {

constexpr int kDistillMaxK = 1024;
constexpr int kDistillThreads = 256;     // of a block, at most
constexpr int kFold = 4;                 // vectors of 16 bytes that a thread folds at once, and waits for at once
constexpr size_t kShareBytes = 72 << 10;              // of a row per block, for three blocks per SM
constexpr size_t kShareMax = 224 << 10;               // ... and at most, for one
constexpr size_t kStreamRow = 128 << 10;              // rows from here on for the persistent form
constexpr int kStreamSlots = 148;                     // its blocks

struct DistillArgs {
  const void* logits; int cols; long long ld;
  const int32_t* n_cols; const int32_t* ids; const float* t; int K;
  float inv_t, temperature, c;  // c = log2(e) / T
  const float* weight;          // row weights (gradient), or NULL = 1
  float* loss; float* lse;      // out, or NULL
  const float* old_lse;         // or NULL: rows of -inf here have nothing visible
  void* grad;                   // or NULL
  int grad_skew;                // the gradient's rows are not aligned to 16 bytes where the logits' are
  int teacher_bytes;            // of shared memory in front of the columns held there
  unsigned long long wait_ns;   // a wait gives up after
};

__device__ __forceinline__ int visible_cols(const DistillArgs& a, int r) {
  const int c = a.n_cols ? a.n_cols[r] : a.cols;
  if (a.old_lse && a.old_lse[r] == -INFINITY) return 0;
  return c < 0 ? 0 : (c > a.cols ? a.cols : c);
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
constexpr float kLn2 = 0.693147180559945f, kLog2e = 1.4426950408889634f;

template <typename T> constexpr int kPer = 16 / (int)sizeof(T);          // columns of 16 bytes
template <typename T> __device__ __forceinline__ void unpack(const uint4& v, float (&x)[kPer<T>]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (sizeof(T) == 4) x[i % kPer<T>] = __uint_as_float(w[i]);
    else { x[(2 * i) % kPer<T>] = __uint_as_float(w[i] << 16); x[(2 * i + 1) % kPer<T>] = __uint_as_float(w[i] & 0xffff0000u); }
  }
}
template <typename T> __device__ __forceinline__ uint4 packed(const float (&x)[kPer<T>]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (sizeof(T) == 4) w[i] = __float_as_uint(x[i % kPer<T>]);
    else {
      const __nv_bfloat162 r = __floats2bfloat162_rn(x[(2 * i) % kPer<T>], x[(2 * i + 1) % kPer<T>]);
      w[i] = *reinterpret_cast<const uint32_t*>(&r);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A row's columns as 16-byte vectors: `head` columns in front of the first 16-byte boundary, `vecs` vectors, `tail` columns.
struct RowSplit { int head, vecs, tail; };
template <typename T> __device__ __forceinline__ RowSplit split_row(const T* row, int cols) {
  const int off = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
  RowSplit s;
  s.head = off ? min(cols, kPer<T> - off) : 0;
  s.vecs = (cols - s.head) / kPer<T>;
  s.tail = cols - s.head - s.vecs * kPer<T>;
  return s;
}

// Maximum of the columns of some vectors (NaN does not count).
template <typename T, int n> __device__ __forceinline__ float max_of(const uint4 (&v)[n]) {
  if (sizeof(T) == 4) {
    float t = -INFINITY;
#pragma unroll
    for (int u = 0; u < n; ++u)
      t = fmaxf(t, fmaxf(fmaxf(__uint_as_float(v[u].x), __uint_as_float(v[u].y)), fmaxf(__uint_as_float(v[u].z), __uint_as_float(v[u].w))));
    return t;
  }
  auto two = [](uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); };
  __nv_bfloat162 t = two(v[0].x);
#pragma unroll
  for (int u = 0; u < n; ++u) t = __hmax2(t, __hmax2(__hmax2(two(v[u].x), two(v[u].y)), __hmax2(two(v[u].z), two(v[u].w))));
  return fmaxf(__low2float(t), __high2float(t));
}

// Running maximum m and s = sum of 2^(c x - c m).  What is at or below kMasked (the lowest value of either type, -inf) adds
// nothing; NaN and +inf make s NaN.  As long as there is nothing visible m is kMasked and s 0, or NaN.
constexpr float kMasked = -8.507059173023462e37f;          // -2^126
constexpr float kFar = 4096.f;
__device__ __forceinline__ float ref_of(float m, float c) {
  const float r = c * m;
  return !(m > kMasked) ? -INFINITY : fabsf(r) < kFar ? r : NAN;
}
struct Exponent {                                          // z of either form: the product of a near row is one operation on x itself
  float a, c, b;
  __device__ __forceinline__ float operator()(float x) const { return fmaf(x - a, c, -b); }
};
struct Fold {
  float m = kMasked, r = -INFINITY, s = 0.f;               // r = ref_of(m, c): -inf without anything visible, NaN for a far maximum
  __device__ __forceinline__ bool near() const { return fabsf(r) < kFar; }
  __device__ __forceinline__ Exponent exponent(float c) const { return near() ? Exponent{0.f, c, r} : Exponent{m, c, 0.f}; }
  // What a sum that goes by this maximum becomes by that one, not below it (near sums go by r itself).
  __device__ __forceinline__ float to(float m2, float r2, float c) const {
    if (near() && fabsf(r2) < kFar) return ex2(r - r2);
    return ex2((m - m2) * c - (near() ? fmaf(m, c, -r) : 0.f) + (fabsf(r2) < kFar ? fmaf(m2, c, -r2) : 0.f));
  }
  __device__ __forceinline__ void raise(float top, float c) {
    if (!(top > m)) return;
    float r2 = c * top;
    if (near() && fabsf(r2) < kFar) {
      s *= ex2(r - r2);
    } else {
      r2 = ref_of(top, c);
      if (m > kMasked) s *= to(top, r2, c);
    }
    m = top; r = r2;
  }
  // (behind raise: no x is above m)
  template <bool NEAR, int n> __device__ __forceinline__ void add(const float (&x)[n], float c) {
    float e[n];
#pragma unroll
    for (int i = 0; i < n; ++i) e[i] = NEAR ? ex2(fmaf(x[i], c, -r)) : m > kMasked ? ex2(exponent(c)(x[i])) : x[i] == x[i] ? 0.f : x[i];
#pragma unroll
    for (int w = n / 2; w > 0; w /= 2)
#pragma unroll
      for (int i = 0; i < w; ++i) e[i] += e[i + w];
    s += e[0];
  }
  // The vectors that `has` names, all of one kind of maximum.
  template <typename T, int n, typename H> __device__ __forceinline__ void add_vecs(const uint4 (&v)[n], float c, H has) {
    auto all = [&](auto is_near) {
#pragma unroll
      for (int u = 0; u < n; ++u)
        if (has(u)) { float x[kPer<T>]; unpack<T>(v[u], x); add<decltype(is_near)::value>(x, c); }
    };
    if (near()) all(std::true_type()); else all(std::false_type());
  }
  __device__ __forceinline__ void merge(const float2& o, float c) {            // o: another one's m and s
    const Fold b{o.x, ref_of(o.x, c), o.y};
    if (b.m > m) { s = b.s + (m > kMasked ? s * to(b.m, b.r, c) : s); m = b.m; r = b.r; }
    else s += b.m > kMasked ? b.s * b.to(m, r, c) : b.s;
  }
};
__device__ __forceinline__ float warp_max(float v) {
  float t;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(t) : "f"(v));
  return t;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// The warp's pair, in every lane.
__device__ __forceinline__ Fold warp_fold(Fold f, float c) {
  Fold t;
  t.m = warp_max(f.m);
  t.r = ref_of(t.m, c);
  t.s = warp_sum(f.m > kMasked ? f.s * f.to(t.m, t.r, c) : f.s);
  return t;
}

// The teacher's entries in shared memory: id (-1: left out), p, its base-2 logarithm, and the row's logit there; for a gradient
// also what mark_repeats needs: a table of eight slots or more per entry, and an entry's representative.
constexpr int kLater = 1 << 30;          // in id: an entry before this one has the same column; the other bits are the first one's number
constexpr int kRepeated = 1 << 29;       // in id: one behind it has; the p of all of them is in v.sum()
constexpr int kIdMask = kRepeated - 1;
struct TeacherView {
  int* id; float *p, *lp, *x; int* rep; unsigned short* table;
  // p of the column that entry j, with this id, is the first one of
  __device__ __forceinline__ float* sum() const { return reinterpret_cast<float*>(table); }
  __device__ __forceinline__ float p_of(int j, int e) const { return e & kRepeated ? sum()[j] : p[j]; }
};
__host__ __device__ __forceinline__ int table_bits(int K) {
  int b = 6;
  while ((1 << b) < 8 * K) ++b;
  return b;
}
__device__ __forceinline__ TeacherView teacher_at(char* smem, int K) {
  const int K4 = (K + 3) & ~3;
  TeacherView v;
  v.id = reinterpret_cast<int*>(smem); v.p = reinterpret_cast<float*>(smem) + K4; v.lp = v.p + K4; v.x = v.lp + K4;
  v.rep = v.id + 4 * K4; v.table = reinterpret_cast<unsigned short*>(v.rep + K4);
  return v;
}
__host__ inline size_t teacher_bytes(int K, bool grad) { return (size_t)((K + 3) & ~3) * (grad ? 20 : 16) + (grad ? (size_t)2 << table_bits(K) : 0); }

constexpr int kTeacherAhead = 8;         // entries that a lane has under way
// One warp: reads the K entries, normalises p over those that the row can see.  Returns whether there is one.
__device__ __forceinline__ bool load_teacher(const DistillArgs& a, int r, int C, const TeacherView& v) {
  const int lane = threadIdx.x & 31;
  float tm = -INFINITY;
  for (int j0 = lane; j0 < a.K; j0 += 32 * kTeacherAhead) {
    int id[kTeacherAhead];
    float t[kTeacherAhead];
#pragma unroll
    for (int u = 0; u < kTeacherAhead; ++u) {
      const size_t at = (size_t)r * a.K + min(j0 + 32 * u, a.K - 1);
      id[u] = __ldg(a.ids + at);
      t[u] = __ldg(a.t + at);
    }
#pragma unroll
    for (int u = 0; u < kTeacherAhead; ++u) {
      const int j = j0 + 32 * u;
      if ((unsigned)id[u] >= (unsigned)C || t[u] == -INFINITY) { id[u] = -1; t[u] = -INFINITY; }
      if (j < a.K) { v.id[j] = id[u]; v.p[j] = t[u]; }
      tm = fmaxf(tm, t[u] != t[u] ? INFINITY : t[u]);      // (the last entry, once more, behind the end)
    }
  }
  tm = warp_max(tm);
  if (tm == -INFINITY) { __syncwarp(); return false; }
  float s = 0.f;
  for (int j = lane; j < a.K; j += 32) s += ex2((v.p[j] - tm) * a.c);                    // (entries that are left out are -inf)
  s = warp_sum(s);
  const float lg = log2f(s), inv = 1.f / s;
  for (int j = lane; j < a.K; j += 32) {
    // (log2 p_j from the teacher's logit, which is exact where p_j is not)
    const float z = (v.p[j] - tm) * a.c;
    v.p[j] = ex2(z) * inv; v.lp[j] = z - lg;
  }
  __syncwarp();
  return true;
}
// The same warp: the row's logits at the entries that `wants` names.
template <typename T, typename W>
__device__ __forceinline__ void load_logits(const T* l, const TeacherView& v, int K, W wants) {
  for (int j0 = threadIdx.x & 31; j0 < K; j0 += 32 * kTeacherAhead) {
    float x[kTeacherAhead];
#pragma unroll
    for (int u = 0; u < kTeacherAhead; ++u) {
      const int id = v.id[min(j0 + 32 * u, K - 1)];
      x[u] = to_f32<T>(l[id >= 0 && wants(id) ? id : 0]);
    }
#pragma unroll
    for (int u = 0; u < kTeacherAhead; ++u) if (j0 + 32 * u < K) v.x[j0 + 32 * u] = x[u];
  }
}
// The same warp, when it has no more use for the ids of repeated entries: marks entries that share a column, for the gradient,
// which has one value there, and adds their p up, in order.  Every entry writes its number to a slot that its id gives, and
// looks who stands there afterwards: an entry of the same column represents it, and with one of another column both
// of that column's entries go to the next round, with other slots.  A round ends it for a column in every slot that was written.
// (1024 bf16 rows of 132352 columns with 256 / 512 entries take 128 / 148 us, some 6 / 24 of them for this; with a table filled by
// compare-and-swap it is 15 / 63, where every entry looks at all others 126 / 418.)
__device__ __forceinline__ void mark_repeats(const TeacherView& v, int K) {
  const int lane = threadIdx.x & 31, shift = 32 - table_bits(K), steps = (K + 31) / 32;
  constexpr unsigned kMul = 2654435769u;                   // (odd, as all the later rounds' are)
  constexpr int kAhead = 4;
  for (int j = lane; j < K; j += 32) if (v.id[j] >= 0) v.table[(unsigned)v.id[j] * kMul >> shift] = (unsigned short)j;
  __syncwarp();
  unsigned open = 0u;                                      // bit per entry of this lane
  bool twice = false;
  for (int b0 = 0; b0 < steps; b0 += kAhead) {
    int id[kAhead], w[kAhead], other[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) { const int j = lane + 32 * (b0 + u); id[u] = j < K ? v.id[j] : -1; }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) w[u] = id[u] >= 0 ? v.table[(unsigned)id[u] * kMul >> shift] : 0;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) other[u] = v.id[w[u]];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int j = lane + 32 * (b0 + u);
      if (id[u] < 0) continue;
      if (other[u] == id[u]) { v.rep[j] = w[u]; twice |= w[u] != j; }
      else open |= 1u << (b0 + u);
    }
  }
  for (unsigned mul = kMul; __any_sync(0xffffffffu, open != 0u);) {
    mul += 0x9e3779b8u;
    for (unsigned m = open; m; m &= m - 1u) { const int j = lane + 32 * (__ffs(m) - 1); v.table[(unsigned)v.id[j] * mul >> shift] = (unsigned short)j; }
    __syncwarp();
    for (unsigned m = open; m; m &= m - 1u) {
      const int j = lane + 32 * (__ffs(m) - 1), id = v.id[j], w = v.table[(unsigned)id * mul >> shift];
      if (v.id[w] == id) { v.rep[j] = w; twice |= w != j; open &= ~(m & (0u - m)); }
    }
    __syncwarp();
  }
  if (!__any_sync(0xffffffffu, twice)) return;
  // a column's first entry, at its representative; then the sums, at the first ones (both in the table's place)
  int* const first = reinterpret_cast<int*>(v.table) + K;
  for (int j = lane; j < K; j += 32) { first[j] = j; v.sum()[j] = v.p[j]; }
  __syncwarp();
  for (int j = lane; j < K; j += 32) if (v.id[j] >= 0 && v.rep[j] != j) atomicMin(&first[v.rep[j]], j);
  __syncwarp();
  for (int j0 = 0; j0 < K; j0 += 32) {
    const int j = j0 + lane;
    int f = -1;
    if (j < K && v.id[j] >= 0) {
      f = first[v.rep[j]];
      if (f == j) f = -1;
      else v.id[j] = kLater | f;
    }
    const unsigned peers = __match_any_sync(0xffffffffu, f);
    if (f >= 0 && __ffs(peers) - 1 == lane) {
      float p = v.sum()[f];
      for (unsigned m = peers; m; m &= m - 1u) p += v.p[j0 + __ffs(m) - 1];
      v.sum()[f] = p;
      v.id[f] |= kRepeated;
    }
    __syncwarp();
  }
}

__device__ __forceinline__ void copy_async(void* smem, const void* g) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(sm100::smem_u32(smem)), "l"(g) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// Until at most `left` groups of this thread's copies are under way.
__device__ __forceinline__ void copy_wait(int left) {
  switch (left) {
    case 0: asm volatile("cp.async.wait_group 0;" ::: "memory"); break;
    case 1: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
    case 2: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
    case 3: asm volatile("cp.async.wait_group 3;" ::: "memory"); break;
    default: asm volatile("cp.async.wait_group 4;" ::: "memory"); break;
  }
}

}  // namespace

// Many long rows: one persistent block per SM, each with a row, or clusters of a few blocks with one.  A block goes over its
// share twice, the second time for the gradient.  The rows in work at one time are held to kLiveBytes, which L2 keeps until
// they are read again, so that HBM sees the logits once.  One thread fills a ring of kStages chunks by bulk copies and runs on
// from the first pass into the second and from there into the next row.  Fifteen warps have the columns, eight vectors of
// a chunk each; one more has, a row ahead, the teacher, the columns outside the vectors and the loss, and, behind the
// barrier of the following row, the teacher's columns of the gradient.
// 2048 bf16 rows of 132352 columns, loss and gradient, 219 to 229 us by the board, of which the bytes need 163; 700 fp32 rows of
// 132347, loss and backward pass, 228 (168); the loss alone of those bf16 rows 105, half of which the exponentials need.  A row per
// block and 39 MB of live rows: two blocks per SM with a row each are 78 MB, half of whose second read misses L2 (14 % more
// time), and rows held in the shared memory of clusters of four leave a seventh of the SMs without work and a fourth of a row's
// time in its barrier (35 % more).  Fifteen warps of columns beside the two others: sixteen make the fp32 pair 5 % slower, and
// thirty with four vectors each the bf16 rows 5 %.
constexpr int kStreamWarps = 15, kStreamThreads = 32 * kStreamWarps, kStreamFold = 8, kStreamK = 512, kStages = 3;
constexpr int kPairs = kStreamWarps + 1;                   // warps that meet in a row's exchange
constexpr int kChunk = kStreamFold * kStreamThreads;       // vectors of a chunk, at most
constexpr size_t kLiveBytes = (size_t)40 << 20;

// One warp: the row's loss, T^2 sum_j p_j (log p_j - log q_j), with ls = log2 s.  The logarithm of a column of the lowest value fits
// its type, but not in base 2: a sum that becomes infinite is taken again in nats.
__device__ __forceinline__ float loss_of(const DistillArgs& a, const float* p, const float* lp, const float* x, const Fold& f, float ls) {
  const Exponent z = f.exponent(a.c);
  float loss = 0.f;
  for (int j = threadIdx.x & 31; j < a.K; j += 32) {
    const float pj = p[j], term = pj * (lp[j] - (z(x[j]) - ls));
    loss += pj != 0.f ? term : 0.f;
  }
  loss = warp_sum(loss) * kLn2;
  if (loss == INFINITY) {
    loss = 0.f;
#pragma unroll 1
    for (int j = threadIdx.x & 31; j < a.K; j += 32)
      if (p[j] != 0.f) loss += p[j] * ((lp[j] + ls) * kLn2 - (x[j] - f.m) * a.inv_t);
    loss = warp_sum(loss);
  }
  return loss * a.temperature * a.temperature;
}

struct StreamTeacher { int id[kStreamK]; float p[kStreamK], lp[kStreamK], x[kStreamK]; int some, c0, c1; };

// One warp: x becomes the gradient in this block's teacher columns, k (q - sum of p), with the sum in a column's first entry;
// id becomes -1 where nothing is to be written.
__device__ __forceinline__ void finish_teacher(const DistillArgs& a, StreamTeacher& t, const TeacherView& v, bool zero, float k, const Fold& f) {
  const int lane = threadIdx.x & 31;
  const Exponent z = f.exponent(a.c);
  unsigned write = 0u;                                     // bit per entry of this lane
  for (int j = lane, b = 0; j < a.K; j += 32, ++b) {
    const int id = t.id[j] & kIdMask;
    if (zero || t.id[j] < 0 || (t.id[j] & kLater) || id < t.c0 || id >= t.c1) continue;
    t.x[j] = k * (ex2(z(t.x[j])) / f.s - v.p_of(j, t.id[j]));
    write |= 1u << b;
  }
  __syncwarp();
  for (int j = lane, b = 0; j < a.K; j += 32, ++b) t.id[j] = (write >> b) & 1u ? t.id[j] & kIdMask : -1;
  __syncwarp();
}
template <typename T> __device__ __forceinline__ void put_teacher(const DistillArgs& a, const StreamTeacher& t, T* out) {
  for (int j = threadIdx.x & 31; j < a.K; j += 32) if (t.id[j] >= 0) out[t.id[j]] = from_f32<T>(t.x[j]);
}

// A block's part of a row: vectors [v0, v1), up to `full` columns of the row; columns [c0, c1) in all.
template <typename T> struct RowPart { const T* l; int head, v0, v1, full, c0, c1; };

template <typename T, bool GRAD>
__global__ void __launch_bounds__(kStreamThreads + 64, 1) k_distill_stream(DistillArgs a, int N, int log_g) {
  extern __shared__ __align__(128) char smem[];
  constexpr int kN = kPer<T>;
  __shared__ float2 s_all[2][8 * kPairs];
  __shared__ StreamTeacher s_teacher[2];
  __shared__ int s_rep[GRAD ? kStreamK : 1];
  __shared__ __align__(16) unsigned short s_table[GRAD ? 8 * kStreamK : 8];
  __shared__ __align__(8) unsigned long long s_full[kStages], s_empty[kStages], s_pairs[2];
  // A wait that gives up raises s_abort in all blocks of the cluster: no one waits any more, every block leaves its rows at its
  // next exchange, and behind the barrier at the end all of the cluster's rows become NaN.
  __shared__ int s_abort, s_sent[8];                       // exchanges that each block of the cluster has sent its pairs for
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  sm100::pdl_wait();
  sm100::pdl_trigger();
  const int G = 1 << log_g, rank = (int)cluster.block_rank();
  const int clusters = gridDim.x >> log_g, r0 = blockIdx.x >> log_g;
  const int rows = r0 < N ? (N - r0 + clusters - 1) / clusters : 0;
  const int tid = threadIdx.x, lane = tid & 31, warp = sm100::uniform_warp();
  auto row_at = [&](int i) { return r0 + i * clusters; };
  auto cols_of = [&](int i) { return i < rows ? visible_cols(a, row_at(i)) : 0; };
  auto part_of = [&](int i, int C) {
    RowPart<T> q;
    q.l = reinterpret_cast<const T*>(a.logits) + (size_t)row_at(i) * a.ld;
    const RowSplit sp = split_row(q.l, a.cols);
    const int share = (sp.vecs + G - 1) >> log_g;
    q.head = sp.head;
    q.v0 = min(sp.vecs, rank * share); q.v1 = min(sp.vecs, q.v0 + share);
    q.full = min(q.v1, max(q.v0, (C - sp.head) / kN));
    q.c0 = rank == 0 ? 0 : q.head + q.v0 * kN; q.c1 = rank == G - 1 ? a.cols : q.head + q.v1 * kN;
    return q;
  };
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) { sm100::mbar_init(sm100::smem_u32(&s_full[i]), 1); sm100::mbar_init(sm100::smem_u32(&s_empty[i]), kStreamWarps); }
    for (int i = 0; i < 2; ++i) sm100::mbar_init(sm100::smem_u32(&s_pairs[i]), 1);
    s_abort = 0;
    sm100::mbar_init_fence();
  }
  if (G > 1) cluster.sync();                               // all blocks are there before anything is sent to them
  else __syncthreads();
  if (rows == 0) return;
  auto to_block = [&](int* word, int value) {              // lane j: into block j's shared memory
    if (lane < G)
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(sm100::map_to_cta(sm100::smem_u32(word), lane)), "r"(value) : "memory");
  };
  auto wait = [&](unsigned long long* bar, int parity) {   // by a whole warp; false: given up, here or elsewhere
    bool ok = *reinterpret_cast<volatile int*>(&s_abort) == 0;
    ok = ok && sm100::mbar_wait(sm100::smem_u32(bar), (uint32_t)parity, &s_abort, a.wait_ns);
    ok = __all_sync(0xffffffffu, ok);
    if (!ok) to_block(&s_abort, 1);
    return ok;
  };
  auto send = [&](int i, float m, float sum) {             // (G > 1)
    if (warp == kStreamWarps && lane == 0) sm100::mbar_expect_tx(sm100::smem_u32(&s_pairs[i & 1]), (uint32_t)(G * kPairs * 8));
    if (lane < G)
      asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];"
                   ::"r"(sm100::map_to_cta(sm100::smem_u32(&s_all[i & 1][rank * kPairs + warp]), lane)), "f"(m), "f"(sum),
                     "r"(sm100::map_to_cta(sm100::smem_u32(&s_pairs[i & 1]), lane)) : "memory");
  };
  // one exchange per row: every warp's pair to all blocks of the cluster.  Behind it all that the block's warps did ahead of
  // it is done.  False, for all warps of the block alike, once s_abort is seen: all have sent their pairs for `sent` rows.
  int sent = 0;
  auto exchange = [&](int i, Fold& f) {
    f = warp_fold(f, a.c);
    if (G == 1) {
      if (lane == 0) s_all[i & 1][warp] = make_float2(f.m, f.s);
    } else {
      send(i, f.m, f.s);
    }
    sent = i + 1;
    int lost = *reinterpret_cast<volatile int*>(&s_abort);
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 p, %0, 0;\n\tbar.red.or.pred q, 1, %1, p;\n\tselp.s32 %0, 1, 0, q;\n\t}"
                 : "+r"(lost) : "n"(32 * kPairs) : "memory");
    if (lost) return false;
    if (G > 1) wait(&s_pairs[i & 1], (i >> 1) & 1);
    f = Fold();
    for (int j = lane; j < G * kPairs; j += 32) f.merge(s_all[i & 1][j], a.c);
    f = warp_fold(f, a.c);
    return true;
  };
  if (warp < kStreamWarps) {
    // ---- the columns
    const uint4* const ring = reinterpret_cast<const uint4*>(smem) + tid;
    const uint32_t none = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;                   // -inf
    int stage = 0, phase = 0;
    // This thread's vectors of the next chunk, of which the block has m.  A whole chunk is worked on without a condition;
    // what lies behind a part of one is -inf.
    using Vecs = uint4[kStreamFold];
    auto take = [&](auto whole, Vecs& v, int m) {
      const bool here = wait(&s_full[stage], phase);
      const uint4* from = ring + stage * kChunk;
#pragma unroll
      for (int u = 0; u < kStreamFold; ++u)
        v[u] = decltype(whole)::value || u * kStreamThreads + tid < m ? from[u * kStreamThreads] : make_uint4(none, none, none, none);
      __syncwarp();
      if (here && lane == 0) sm100::mbar_arrive(sm100::smem_u32(&s_empty[stage]));     // (otherwise its copy may be under way)
      if (++stage == kStages) { stage = 0; phase ^= 1; }
    };
    auto has = [&](auto whole, int u, int m) { return decltype(whole)::value || u * kStreamThreads + warp * 32 < m; };       // any of the warp
    int C1 = cols_of(1);
    RowPart<T> q = part_of(0, cols_of(0));
    bool on = true;
    for (int i = 0; i < rows; ++i) {
      const int r = row_at(i), n = q.full - q.v0;
      const float w = GRAD && a.weight ? a.weight[r] : 1.f;
      Fold f;
      auto fold = [&](auto whole, int m) {
        Vecs v;
        take(whole, v, m);
        f.raise(max_of<T>(v), a.c);
        f.add_vecs<T>(v, a.c, [&](int u) { return has(whole, u, m); });
      };
      int v0 = 0;
      for (; v0 + kChunk <= n; v0 += kChunk) fold(std::true_type(), kChunk);
      if (v0 < n || n == 0) fold(std::false_type(), n - v0);                   // (a part without columns has a chunk, too)
      if (!exchange(i, f)) { on = false; break; }
      if (GRAD) {
        const bool zero = !s_teacher[i & 1].some || f.s == 0.f || w == 0.f;
        const float k = w * a.temperature;
        // k q: in bf16 with the factor in the exponent, otherwise as a product.  (The sum of r and the factor's logarithm is rounded once
        // more than the normaliser's r: an error of 2^-24 of it, at most 2^-12 of q below kFar, to a rounding of 2^-8.)
        const bool far = !f.near(), in_exponent = sizeof(T) == 2 && k > 0.f && !far;
        const float kq = zero ? 0.f : in_exponent ? 1.f : k / f.s;
        const float off = in_exponent ? f.r + (log2f(f.s) - log2f(k)) : f.r;
        T* out = reinterpret_cast<T*>(a.grad) + (size_t)r * a.ld + q.head;
        uint4* ov = reinterpret_cast<uint4*>(out) + q.v0;
        auto put = [&](int v, const uint4& x) {
          if (!a.grad_skew) { __stcs(ov + v, x); return; }
          const T* e = reinterpret_cast<const T*>(&x);
#pragma unroll
          for (int u = 0; u < kN; ++u) out[(q.v0 + v) * kN + u] = e[u];
        };
        auto columns = [&](auto whole, auto scaled, int m) {
          Vecs v;
          take(whole, v, m);
#pragma unroll
          for (int u = 0; u < kStreamFold; ++u) {
            if (!has(whole, u, m)) break;
            float x[kN];
            unpack<T>(v[u], x);
#pragma unroll
            for (int e = 0; e < kN; ++e) {
              x[e] = ex2(!decltype(whole)::value && far ? (x[e] - f.m) * a.c : fmaf(x[e], a.c, -off));
              if (decltype(scaled)::value) x[e] *= kq;
            }
            if (!decltype(whole)::value) {
              if (zero) {
#pragma unroll
                for (int e = 0; e < kN; ++e) x[e] = 0.f;
              }
              if (u * kStreamThreads + tid < m) put(v0 + u * kStreamThreads + tid, packed<T>(x));
            } else {
              __stcs(ov + v0 + u * kStreamThreads + tid, packed<T>(x));
            }
          }
        };
        v0 = 0;
        const bool plain = !zero && !a.grad_skew && !far;  // (the other rows take the chunks in part)
        for (; plain && v0 + kChunk <= n; v0 += kChunk) {
          if (in_exponent) columns(std::true_type(), std::integral_constant<bool, sizeof(T) == 4>(), kChunk);
          else columns(std::true_type(), std::true_type(), kChunk);
        }
        for (; v0 < n || (n == 0 && v0 == 0); v0 += kChunk) columns(std::false_type(), std::true_type(), min(kChunk, n - v0));
        for (int v = max(n, 0) + tid; v < q.v1 - q.v0; v += kStreamThreads) if (q.v0 + v != q.full) put(v, make_uint4(0u, 0u, 0u, 0u));
      }
      if (i + 1 < rows) { q = part_of(i + 1, C1); C1 = cols_of(i + 2); }
    }
    if (GRAD && on) asm volatile("bar.sync 1, %0;" ::"n"(32 * kPairs) : "memory");
  } else if (warp == kStreamWarps) {
    // ---- everything else
    // columns outside the vectors, one a lane: in front of them, of the one that the row ends in, behind them
    auto edge_of = [&](const RowPart<T>& q) {
      if (lane < 8) return rank == 0 && lane < q.head ? lane : -1;
      if (lane < 16) return q.full < q.v1 && lane - 8 < kN ? q.head + q.full * kN + lane - 8 : -1;
      const int tail = a.cols - q.head - (a.cols - q.head) / kN * kN;
      return lane < 24 && rank == G - 1 && lane - 16 < tail ? a.cols - tail + lane - 16 : -1;
    };
    float edge_x = 0.f;
    // the first block takes the loss and with it the row's logits at all entries, the others those of their own columns
    auto view_of = [&](StreamTeacher& t) { return TeacherView{t.id, t.p, t.lp, t.x, s_rep, s_table}; };
    auto prepare = [&](int i, int C, const RowPart<T>& q) {
      StreamTeacher& t = s_teacher[i & 1];
      const int e = edge_of(q);
      edge_x = e >= 0 && e < C ? to_f32<T>(q.l[e]) : -INFINITY;
      const TeacherView tv = view_of(t);
      const bool some = load_teacher(a, row_at(i), C, tv);
      load_logits<T>(q.l, tv, a.K, [&](int id) { return rank == 0 || (id >= q.c0 && id < q.c1); });
      if (GRAD && some) mark_repeats(tv, a.K);
      if (lane == 0) { t.some = some; t.c0 = q.c0; t.c1 = q.c1; }
      __syncwarp();
    };
    int C = cols_of(0), C1 = cols_of(1);
    RowPart<T> q = part_of(0, C);
    prepare(0, C, q);
    bool on = true;
    for (int i = 0; i < rows; ++i) {
      const int r = row_at(i);
      const float w = GRAD && a.weight ? a.weight[r] : 1.f;
      Fold f;
      const float two[2] = {edge_x, -INFINITY};
      f.raise(edge_x, a.c);
      f.add<false>(two, a.c);
      if (!exchange(i, f)) { on = false; break; }
      // (all warps of the block have written the row before's gradient)
      if (GRAD && i > 0) put_teacher<T>(a, s_teacher[(i - 1) & 1], reinterpret_cast<T*>(a.grad) + (size_t)row_at(i - 1) * a.ld);
      StreamTeacher& t = s_teacher[i & 1];
      const bool live = t.some && f.s != 0.f;
      const float ls = log2f(f.s);
      if (rank == 0 && a.loss) {
        const float loss = live ? loss_of(a, t.p, t.lp, t.x, f, ls) : 0.f;
        if (lane == 0) { a.loss[r] = loss; a.lse[r] = f.s == 0.f ? -INFINITY : fmaf(f.m, a.inv_t, ls * kLn2); }
      }
      if (GRAD) {
        const bool zero = !live || w == 0.f;
        const float k = w * a.temperature;
        const int e = edge_of(q);
        if (e >= 0) (reinterpret_cast<T*>(a.grad) + (size_t)r * a.ld)[e] = from_f32<T>(zero || e >= C ? 0.f : k * (ex2(f.exponent(a.c)(edge_x)) / f.s));
        finish_teacher(a, t, view_of(t), zero, k, f);
      }
      if (i + 1 < rows) {
        C = C1; C1 = cols_of(i + 2);
        q = part_of(i + 1, C);
        prepare(i + 1, C, q);
      }
    }
    if (GRAD && on) {
      asm volatile("bar.sync 1, %0;" ::"n"(32 * kPairs) : "memory");
      put_teacher<T>(a, s_teacher[(rows - 1) & 1], reinterpret_cast<T*>(a.grad) + (size_t)row_at(rows - 1) * a.ld);
    }
  } else {
    // ---- the copies
    int stage = 0, phase = 1;                              // (a stage that was never filled is empty)
    int C1 = cols_of(0);
    bool on = true;
    unsigned filled = 0;                                   // chunks; chunk k is in stage k % kStages
    for (int i = 0; i < rows && on; ++i) {
      const RowPart<T> q = part_of(i, C1);
      C1 = cols_of(i + 1);
      const uint4* lv = reinterpret_cast<const uint4*>(q.l + q.head) + q.v0;
      const int n = q.full - q.v0;
      for (int pass = 0; pass < (GRAD ? 2 : 1) && on; ++pass)
        for (int v0 = 0; v0 < n || (n == 0 && v0 == 0); v0 += kChunk) {
          on = wait(&s_empty[stage], phase);
          if (!on) break;
          const int m = min(kChunk, n - v0);
          if (lane == 0) {
            const uint32_t bar = sm100::smem_u32(&s_full[stage]);
            if (m <= 0) sm100::mbar_arrive(bar);           // (a part without columns)
            else {
              sm100::mbar_expect_tx(bar, (uint32_t)m * 16u);
              asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                           ::"r"(sm100::smem_u32(smem) + (uint32_t)(stage * kChunk) * 16u), "l"(lv + v0), "r"((uint32_t)m * 16u), "r"(bar) : "memory");
            }
          }
          __syncwarp();
          ++filled;
          if (++stage == kStages) { stage = 0; phase ^= 1; }
        }
    }
    // the block's shared memory outlives the copies, whether or not the columns' warps still wait for them
    for (unsigned k = filled < kStages ? 0u : filled - kStages; k < filled; ++k) sm100::mbar_drain(sm100::smem_u32(&s_full[k % kStages]), (k / kStages) & 1u);
  }
  // ---- the end: no block leaves before all of its cluster have stopped sending to it
  __syncwarp();
  if (G > 1) {
    if (warp == 0) { to_block(&s_sent[rank], sent); __syncwarp(); }
    sm100::cluster_sync_all();
  } else {
    __syncthreads();
  }
  if (!s_abort) return;
  if (G > 1 && warp < kPairs) {
    // A block has sent its pairs for at most two rows more than another (the first of them is not waited for successfully).
    // All send what is missing, so that every exchange that was begun completes, and wait for the last two: what is
    // under way to a block then has arrived.
    int last = 0;
    for (int j = 0; j < G; ++j) last = max(last, s_sent[j]);
    for (int i = sent; i < last; ++i) {
      if (i >= 2) sm100::mbar_drain(sm100::smem_u32(&s_pairs[i & 1]), (uint32_t)((i - 2) >> 1) & 1u);
      __syncwarp();
      send(i, NAN, NAN);
    }
    for (int i = max(0, last - 2); i < last; ++i) sm100::mbar_drain(sm100::smem_u32(&s_pairs[i & 1]), (uint32_t)(i >> 1) & 1u);
  }
  for (int i = 0; i < rows; ++i) {
    const int r = row_at(i);
    const RowPart<T> q = part_of(i, 0);
    if (GRAD) for (int c = q.c0 + tid; c < q.c1; c += kStreamThreads + 64) (reinterpret_cast<T*>(a.grad) + (size_t)r * a.ld)[c] = from_f32<T>(NAN);
    if (rank == 0 && tid == 0 && a.loss) a.loss[r] = a.lse[r] = NAN;
  }
}

// Grid: rows x blocks of a cluster.  HOLD: the share stays in shared memory (behind the teacher's entries).
template <typename T, bool GRAD, bool HOLD>
__global__ void __launch_bounds__(kDistillThreads) k_distill(DistillArgs a) {
  extern __shared__ __align__(16) char smem[];
  constexpr int kN = kPer<T>, kMaxWarps = kDistillThreads / 32;
  __shared__ float2 s_all[8 * kMaxWarps];                  // (m, s) of every warp of the row
  __shared__ int s_some;                                   // the teacher has an entry
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  sm100::pdl_wait();
  sm100::pdl_trigger();
  const int G = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), r = blockIdx.x / G;
  if (G > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");       // (waited for before the first remote store)
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, warps = threads >> 5;
  const T* l = reinterpret_cast<const T*>(a.logits) + (size_t)r * a.ld;
  const int C = visible_cols(a, r);
  const RowSplit sp = split_row(l, a.cols);
  const int share = (sp.vecs + G - 1) / G, v0 = min(sp.vecs, rank * share), v1 = min(sp.vecs, v0 + share);
  const uint4* lv = reinterpret_cast<const uint4*>(l + sp.head);
  const int full = min(v1, max(v0, (C - sp.head) / kN));   // vectors [v0, full) are columns of the row; at most one behind is in part
  const int U = (full - v0 + threads - 1) / threads, groups = (U + kFold - 1) / kFold;
  uint4* hold = reinterpret_cast<uint4*>(smem + a.teacher_bytes);
  // ---- the share's columns
  if (HOLD) {
    for (int g = 0; g < groups; ++g) {
#pragma unroll
      for (int u = 0; u < kFold; ++u) {
        const int i = (g * kFold + u) * threads + tid;
        if (v0 + i < full) copy_async(hold + i, lv + v0 + i);
      }
      copy_commit();
    }
  }
  // columns outside the vectors, and those of the vector that the row ends in: one a thread
  int my_col = -1;
  if (rank == 0 && tid < sp.head) my_col = tid;
  else if (rank == G - 1 && tid >= 32 && tid < 32 + sp.tail) my_col = a.cols - sp.tail + tid - 32;
  const float my_x = my_col >= 0 && my_col < C ? to_f32<T>(l[my_col]) : -INFINITY;
  const int part = sp.head + full * kN, part_n = full < v1 ? max(0, min(kN, C - part)) : 0;
  const float part_x = tid < part_n ? to_f32<T>(l[part + tid]) : -INFINITY;
  // ---- the teacher, by one warp while the columns are under way.  The first block takes the loss and with it the row's
  // logits there; the others find those of their own columns [c0, c1) in what they hold, or here.
  const int c0 = rank == 0 ? 0 : sp.head + v0 * kN, c1 = rank == G - 1 ? a.cols : sp.head + v1 * kN;
  auto held = [&](int id) { return HOLD && id >= sp.head + v0 * kN && id < part; };
  const TeacherView tv = teacher_at(smem, a.K);
  if (warp == warps - 1 && (GRAD || rank == 0)) {
    const bool some = load_teacher(a, r, C, tv);
    load_logits<T>(l, tv, a.K, [&](int id) { return rank == 0 || (id >= c0 && id < c1 && !held(id)); });
    if (GRAD && some) mark_repeats(tv, a.K);
    if (lane == 0) s_some = some;
  }
  // ---- maximum and sum
  Fold f;
  const uint32_t none = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;                     // -inf
  {
    const float two[2] = {my_x, part_x};
    f.raise(fmaxf(my_x, part_x), a.c);
    f.add<false>(two, a.c);
  }
  for (int g = 0; g < groups; ++g) {
    uint4 v[kFold];
    if (HOLD) copy_wait(groups - 1 - g);
#pragma unroll
    for (int u = 0; u < kFold; ++u) {
      const int i = (g * kFold + u) * threads + tid;
      v[u] = v0 + i < full ? (HOLD ? hold[i] : lv[v0 + i]) : make_uint4(none, none, none, none);
    }
    f.raise(max_of<T>(v), a.c);
    f.add_vecs<T>(v, a.c, [&](int u) { return v0 + (g * kFold + u) * threads + tid < full; });
  }
  f = warp_fold(f, a.c);
  if (G > 1) {
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    if (lane < G) *cluster.map_shared_rank(&s_all[rank * warps + warp], lane) = make_float2(f.m, f.s);
    cluster.sync();                                        // (also: every logit has been read that a gradient may overwrite)
  } else {
    if (lane == 0) s_all[warp] = make_float2(f.m, f.s);
    __syncthreads();
  }
  f = Fold();
  for (int i = lane; i < G * warps; i += 32) f.merge(s_all[i], a.c);
  f = warp_fold(f, a.c);
  const bool live = f.s != 0.f && s_some;
  const float ls = log2f(f.s);
  if (rank == 0 && warp == 0 && a.loss) {
    const float loss = live ? loss_of(a, tv.p, tv.lp, tv.x, f, ls) : 0.f;
    if (lane == 0) { a.loss[r] = loss; a.lse[r] = f.s == 0.f ? -INFINITY : fmaf(f.m, a.inv_t, ls * kLn2); }
  }
  if (!GRAD) return;
  // ---- the gradient of the share
  const float w = a.weight ? a.weight[r] : 1.f, k = w * a.temperature;
  const bool zero = !live || w == 0.f;
  T* out = reinterpret_cast<T*>(a.grad) + (size_t)r * a.ld;
  // k q: in bf16 with the factor in the exponent, otherwise as a product (see k_distill_stream)
  const bool in_exponent = sizeof(T) == 2 && k > 0.f && f.near();
  const float kq = in_exponent ? 1.f : k / f.s, off = in_exponent ? f.r + (ls - log2f(k)) : f.r;
  const Exponent z = f.exponent(a.c);
  auto value = [&](float x) { return ex2(in_exponent ? fmaf(x, a.c, -off) : z(x)) * kq; };
  if (my_col >= 0) out[my_col] = from_f32<T>(zero || my_col >= C ? 0.f : value(my_x));
  if (full < v1 && tid < kN) out[part + tid] = from_f32<T>(zero || tid >= part_n ? 0.f : value(part_x));
  uint4* ov = reinterpret_cast<uint4*>(out + sp.head) + v0;
  const int n_full = zero ? 0 : full - v0;
  auto put = [&](int i, const float (&x)[kN]) {
    if (!a.grad_skew) __stcs(ov + i, packed<T>(x));
    else {
#pragma unroll
      for (int u = 0; u < kN; ++u) out[sp.head + (v0 + i) * kN + u] = from_f32<T>(x[u]);
    }
  };
  auto columns = [&](auto scaled, auto far) {
#pragma unroll 4
    for (int i = tid; i < n_full; i += threads) {
      float x[kN];
      unpack<T>(HOLD ? hold[i] : lv[v0 + i], x);
#pragma unroll
      for (int u = 0; u < kN; ++u) {
        x[u] = ex2(decltype(far)::value ? (x[u] - f.m) * a.c : fmaf(x[u], a.c, -off));
        if (decltype(scaled)::value) x[u] *= kq;
      }
      put(i, x);
    }
  };
  if (!f.near()) columns(std::true_type(), std::true_type());
  else if (in_exponent) columns(std::false_type(), std::false_type());
  else columns(std::true_type(), std::false_type());
  const float nothing[kN] = {};
  for (int i = n_full + tid; i < v1 - v0; i += threads) if (zero || v0 + i != full) put(i, nothing);
  if (zero) return;
  __syncthreads();
  // the teacher's columns, over the columns' own: k (q - sum of p), by whoever has a column's first entry
  for (int j = tid; j < a.K; j += threads) {
    const int id = tv.id[j] & kIdMask;
    if (tv.id[j] < 0 || (tv.id[j] & kLater) || id < c0 || id >= c1) continue;
    const float p = tv.p_of(j, tv.id[j]);
    const float x = rank != 0 && held(id) ? to_f32<T>(reinterpret_cast<const T*>(hold)[id - sp.head - v0 * kN]) : tv.x[j];
    out[id] = from_f32<T>(k * (ex2(z(x)) / f.s - p));
  }
}

namespace {

std::atomic<unsigned long long> g_wait_ns{sm100::kWaitLimitNs};

// c of DistillArgs
float exponent_of(float temperature) { return (float)(1.4426950408889634 / (double)temperature); }

int fail_arg(const char* msg) { set_last_error(msg); return Z2Z_ERR_INVALID_ARG; }

int check_distill(const void* logits, int dtype, int N, int cols, int64_t ld, const int32_t* ids, const float* t, int K, float temperature,
                  const void* grad) {
  if (dtype != Z2Z_DTYPE_FP32 && dtype != Z2Z_DTYPE_BF16) return fail_arg("unknown dtype");
  if (N < 0) return fail_arg("N < 0");
  if (cols < 1 || cols > (1 << 24)) return fail_arg("need 1 <= cols <= 2^24");
  if (ld < cols) return fail_arg("ld < cols");
  if (K < 0 || K > kDistillMaxK) return fail_arg("need 0 <= K <= 1024");
  if (!(temperature > 0.f) || !std::isfinite(temperature) || !std::isfinite(exponent_of(temperature))) return fail_arg("temperature must be > 0 and finite");
  if (N == 0) return Z2Z_OK;
  if (!logits) return fail_arg("d_logits is NULL");
  if (K > 0 && (!ids || !t)) return fail_arg("d_teacher_ids / d_teacher_logits is NULL");
  const uintptr_t es = dtype == Z2Z_DTYPE_BF16 ? 2 : 4;
  if (reinterpret_cast<uintptr_t>(logits) % es || reinterpret_cast<uintptr_t>(grad) % es) return fail_arg("logits and gradients must be aligned to their elements");
  return Z2Z_OK;
}

int done(cudaError_t e) {
  if (e == cudaSuccess) return Z2Z_OK;
  set_last_error(cudaGetErrorString(e));
  return Z2Z_ERR_CUDA;
}

template <typename T, bool GRAD, bool HOLD>
cudaError_t launch_loss_typed(const DistillArgs& a, int N, int G, int threads, size_t smem, cudaStream_t s) {
  auto kern = k_distill<T, GRAD, HOLD>;
  if (smem > 40 << 10) {                                   // (48 KB with the kernel's own, which is less than 8)
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3((unsigned)N * (unsigned)G);
  lc.blockDim = dim3(threads);
  lc.dynamicSmemBytes = smem;
  lc.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)G; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  lc.attrs = at; lc.numAttrs = 2;
  return cudaLaunchKernelEx(&lc, kern, a);
}

template <typename T, bool GRAD>
cudaError_t launch_stream(const DistillArgs& a, int N, int log_g, cudaStream_t s) {
  auto kern = k_distill_stream<T, GRAD>;
  constexpr int smem = kStages * kChunk * 16;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3(1u << log_g);
  lc.blockDim = dim3(kStreamThreads + 64);
  lc.dynamicSmemBytes = smem;
  lc.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = 1u << log_g; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  lc.attrs = at; lc.numAttrs = 1;
  // clusters that are resident at one time (those of four and eight leave the rest of a GPC without one); found by the first call,
  // or by each of several threads that come first
  static std::atomic<int> fit[4];
  int most = kStreamSlots >> log_g;
  if (log_g > 1) {
    int n = fit[log_g].load(std::memory_order_relaxed);
    if (!n && (e = cudaOccupancyMaxActiveClusters(&n, kern, &lc)) != cudaSuccess) return e;
    fit[log_g].store(n, std::memory_order_relaxed);
    if (n >= 1 && n < most) most = n;
  }
  lc.gridDim = dim3((unsigned)((N < most ? N : most) << log_g));
  lc.numAttrs = 2;
  return cudaLaunchKernelEx(&lc, kern, a, N, log_g);
}

template <typename T>
cudaError_t launch_loss(const DistillArgs& a, int N, cudaStream_t s) {
  const size_t row = (size_t)a.cols * sizeof(T);
  // The persistent form from rows on whose exchange is short beside their bytes, and from a row for every two SMs on.  Clusters
  // against it, us, loss alone / with the gradient, bf16: 1024 rows of 32 KB 14 / 23 against 24 / 49, of 64 KB 21 / 41 against
  // 30 / 55, of 128 KB 35 / 71 against 37 / 73, of 258 KB 63 / 138 against 55 / 117; 148 rows of 258 KB 16 / 29 against 13 / 23, 74
  // rows 11 / 17 against 10 / 16, 37 rows 9 / 13 against 11 / 17.  fp32, in the same order: 13 / 21 against 23 / 42, 20 / 38
  // against 28 / 49, 34 / 67 against 32 / 62, 59 / 124 against 44 / 102; 13 / 27 against 12 / 20, 9 / 15 against 9 / 14, 8 / 12
  // against 10 / 16.  (A longer teacher's list than kStreamK has no room beside the ring.)
  if (a.K <= kStreamK && row >= kStreamRow && N >= kStreamSlots / 2) {
    // blocks per row: so many that the rows in work stay in L2, and more where the last round would leave much of the machine idle
    int log_g = 0;
    if (a.grad) while (log_g < 3 && row * (kStreamSlots >> log_g) > kLiveBytes) ++log_g;
    auto rounds = [&](int l) { const long long m = kStreamSlots >> l; return (double)((N + m - 1) / m) / (1 << l); };
    for (int l = log_g + 1; l <= 3; ++l) if (rounds(l) < 0.9 * rounds(log_g)) log_g = l;
    return a.grad ? launch_stream<T, true>(a, N, log_g, s) : launch_stream<T, false>(a, N, log_g, s);
  }
  // Blocks per row: so many that a block's share leaves room for three on an SM, and more while all rows together do not
  // occupy the machine's SMs
  const size_t teacher = (size_t)a.teacher_bytes;
  int G = 1;
  while (G < 8 && (row / G > kShareBytes || ((long long)N * 2 * G <= 148 && row / G > 4096))) G *= 2;
  const int vecs = (int)((row / 16 + G - 1) / G);
  int threads = (vecs / 2 + 63) / 64 * 64;                 // two vectors a thread at least
  threads = threads < 64 ? 64 : (threads > kDistillThreads ? kDistillThreads : threads);
  const size_t share = (size_t)vecs * 16;
  if (!a.grad) return launch_loss_typed<T, false, false>(a, N, G, threads, teacher, s);
  if (teacher + share <= kShareMax) return launch_loss_typed<T, true, true>(a, N, G, threads, teacher + share, s);
  return launch_loss_typed<T, true, false>(a, N, G, threads, teacher, s);
}

DistillArgs distill_args(const void* logits, int cols, int64_t ld, const int32_t* n_cols, const int32_t* ids, const float* t, int K, float temperature,
                         const float* weight, float* loss, float* lse, const float* old_lse, void* grad) {
  const int skew = grad && ((reinterpret_cast<uintptr_t>(grad) ^ reinterpret_cast<uintptr_t>(logits)) & 15) ? 1 : 0;
  return DistillArgs{logits, cols, ld, n_cols, ids, t, K, 1.f / temperature, temperature, exponent_of(temperature),
                     weight, loss, lse, old_lse, grad, skew, (int)teacher_bytes(K, grad != nullptr), g_wait_ns.load(std::memory_order_relaxed)};
}
}  // namespace

}  // namespace z2z

extern "C" {

int32_t z2z_set_distill_wait_limit(int64_t ns) {
  if (ns < 0) return z2z::fail_arg("ns < 0");
  z2z::g_wait_ns.store(ns ? (unsigned long long)ns : z2z::sm100::kWaitLimitNs, std::memory_order_relaxed);
  return Z2Z_OK;
}

int32_t z2z_distill_loss(const void* d_logits, int32_t dtype, int32_t N, int32_t cols, int64_t ld,
                         const int32_t* d_n_cols, const int32_t* d_teacher_ids,
                         const float* d_teacher_logits, int32_t K, float temperature,
                         const float* d_row_weight, float* d_loss, float* d_lse, void* d_grad,
                         z2z_stream stream) {
  const int rc = z2z::check_distill(d_logits, dtype, N, cols, ld, d_teacher_ids, d_teacher_logits, K, temperature, d_grad);
  if (rc || N == 0) return rc;
  if (!d_loss || !d_lse) return z2z::fail_arg("d_loss / d_lse is NULL");
  const z2z::DistillArgs a = z2z::distill_args(d_logits, cols, ld, d_n_cols, d_teacher_ids, d_teacher_logits, K, temperature, d_row_weight, d_loss,
                                               d_lse, nullptr, d_grad);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  return z2z::done(dtype == Z2Z_DTYPE_BF16 ? z2z::launch_loss<__nv_bfloat16>(a, N, s) : z2z::launch_loss<float>(a, N, s));
}

int32_t z2z_distill_grad(const void* d_logits, int32_t dtype, int32_t N, int32_t cols, int64_t ld,
                         const int32_t* d_n_cols, const int32_t* d_teacher_ids,
                         const float* d_teacher_logits, int32_t K, float temperature,
                         const float* d_lse, const float* d_grad_loss, void* d_grad, z2z_stream stream) {
  const int rc = z2z::check_distill(d_logits, dtype, N, cols, ld, d_teacher_ids, d_teacher_logits, K, temperature, d_grad);
  if (rc || N == 0) return rc;
  if (!d_lse || !d_grad_loss || !d_grad) return z2z::fail_arg("d_lse / d_grad_loss / d_grad is NULL");
  const z2z::DistillArgs a = z2z::distill_args(d_logits, cols, ld, d_n_cols, d_teacher_ids, d_teacher_logits, K, temperature, d_grad_loss, nullptr,
                                               nullptr, d_lse, d_grad);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  return z2z::done(dtype == Z2Z_DTYPE_BF16 ? z2z::launch_loss<__nv_bfloat16>(a, N, s) : z2z::launch_loss<float>(a, N, s));
}

}  // extern "C"
