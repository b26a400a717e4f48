// Operators over rows of logits: log probabilities of given tokens with entropy and top alternatives, distillation
// from a teacher's top logits, and the gradients of both.
//
// With s_j = x_j / tau, lse = log sum_j exp(s_j), p_j = exp(s_j - lse):
//   logprob = s_y - lse          entropy H = lse - sum_j p_j s_j
//   d/dx_j (g logprob + h H) = (g ([j = y] - p_j) - h p_j (log p_j + H)) / tau
//   q = softmax of the teacher's K logits / tau;  loss = tau^2 sum_i q_i (log q_i - log p_{a_i})
//   d/dx_j (g loss) = g tau (p_j - sum_{i: a_i = j} q_i)
//
// All of them are one pass over the logits (and one over the gradient), a few operations per element and one exp, so
// device memory bounds them.  A row belongs to a group of threads: a warp (rows of up to kWarpRow elements), a block of
// 256, or a thread-block cluster of up to 8 blocks that join their partial results through distributed shared memory.
// No workspace, no atomics on device memory, and sums in a fixed order: results do not depend on timing.
//
// Element layout of a row: rows start at any element address.  The part between the first and the last 16-byte boundary
// is read as 16-byte vectors, interleaved over the group's threads; the up to EV - 1 elements before and after it ("edge"
// elements) go to one thread each.
#include <cooperative_groups.h>
#include <float.h>

#include "laq_ops.cuh"

namespace cg = cooperative_groups;

namespace laq {
namespace ops {
namespace {

constexpr int kBlock = 256;
constexpr int kWarpBlock = 128;        // block of the kernels whose rows belong to one warp each
constexpr int kWarpRow = 1024;         // longest row that one warp takes
constexpr int kMaxCluster = 8;
constexpr int kMaxTopK = 32;
constexpr int kMaxTeacher = 128;
constexpr int kBatch = 4;              // vectors of the streaming loop that a thread has in flight
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kUnset = -FLT_MAX;     // reference of a thread that has seen nothing above -inf
constexpr float kSlack = 32.f;         // a reference may lag the maximum by this many powers of two
constexpr float kEmptyLse = -1e30f;    // an lse below this belongs to a row of masks only

// ---- a group of NT threads that owns a row (or, in a cluster, a slice of it) ------------------------------------------
template <int NT>
struct Group {
  static constexpr int kWarps = NT / 32;
  static constexpr int kRowsPerBlock = NT == 32 ? kWarpBlock / 32 : 1;
  static __device__ __forceinline__ int tid() { return NT == 32 ? (int)(threadIdx.x & 31u) : (int)threadIdx.x; }
  static __device__ __forceinline__ int slot() { return NT == 32 ? (int)(threadIdx.x >> 5) : 0; }   // row within the block
  static __device__ __forceinline__ void sync() {
    if (NT == 32) __syncwarp(); else __syncthreads();
  }
};

// The share of `rank` (of `ranks`) in a row of V elements: vectors [v0, v1), i.e. elements [e0, e1) with the edges.
template <class T>
struct Slice {
  const T* row;
  int head, nvec, v0, v1, e0, e1, tail0, V;
  __device__ __forceinline__ Slice(const T* r, int V_, int rank, int ranks) : row(r), V(V_) {
    constexpr int EV = Elem<T>::EV;
    const int mis = (int)(((uintptr_t)r & 15u) / sizeof(T));
    head = mis ? min(EV - mis, V) : 0;
    nvec = (V - head) / EV;
    tail0 = head + nvec * EV;
    const int per = (nvec + ranks - 1) / ranks;
    v0 = min(rank * per, nvec);
    v1 = min(v0 + per, nvec);
    e0 = rank == 0 ? 0 : head + v0 * EV;
    e1 = rank == ranks - 1 ? V : head + v1 * EV;
  }
  __device__ __forceinline__ const T* vec(int v) const { return row + head + v * Elem<T>::EV; }
  // the edge element of thread t, or -1: the head's in the first rank (threads 0..), the tail's in the last (16..)
  __device__ __forceinline__ int edge(int t) const {
    if (t < head && e0 == 0) return t;
    const int j = tail0 + t - 16;
    return (t >= 16 && t < 32 && j < V && e1 == V) ? j : -1;
  }
};

// ---- running softmax statistics ---------------------------------------------------------------------------------------
// With d = (x - ref) c, c = log2(e) / tau:  s = sum 2^d, u = sum d 2^d.  ref is any number that no x exceeds by more than
// kSlack / c; it moves only when it must, so the common path has no rescaling.  All of it in fp32; x - ref is taken
// before the product with c, so that neither the reference nor masks at the type's lowest value lose digits.
struct Stat {
  float ref, s, u;
};

__device__ __forceinline__ void move_ref(Stat& a, float ref, float c) {    // ref >= a.ref, or NaN
  const float d = max_nan((a.ref - ref) * c, -1e4f);
  const float f = ex2(d);
  a.u = fmaf(d, a.s, a.u) * f;
  a.s *= f;
  a.ref = ref;
}

template <int N, bool ENTROPY>
__device__ __forceinline__ void add_elements(Stat& a, const float (&x)[N], float c) {
  float s0 = 0.f, s1 = 0.f, u0 = 0.f, u1 = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float d = (x[i] - a.ref) * c;
    if (ENTROPY) d = max_nan(d, -1e4f);       // -inf: 2^d is 0 and so is its share of u
    const float e = ex2(d);
    if (i & 1) {
      s1 += e;
      if (ENTROPY) u1 = fmaf(e, d, u1);
    } else {
      s0 += e;
      if (ENTROPY) u0 = fmaf(e, d, u0);
    }
  }
  a.s += s0 + s1;
  if (ENTROPY) a.u += u0 + u1;
}

__device__ __forceinline__ void follow(Stat& a, float mx, float c) {
  if (!((mx - a.ref) * c <= kSlack)) move_ref(a, mx, c);      // also taken for NaN, which then stays
}

template <class T, int N, bool ENTROPY>
__device__ __forceinline__ void add_vectors(Stat& a, float& top, const uint4 (&v)[N], float c) {
  constexpr int EV = Elem<T>::EV;
  const float mx = Elem<T>::largest(v);
  top = max_nan(top, mx);
  follow(a, mx, c);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float x[EV];
    Elem<T>::unpack(v[i], x);
    add_elements<EV, ENTROPY>(a, x, c);
  }
}

__device__ __forceinline__ Stat join(Stat a, Stat b, float c) {
  const float r = max_nan(a.ref, b.ref);
  move_ref(a, r, c);
  move_ref(b, r, c);
  a.s += b.s;
  a.u += b.u;
  return a;
}

__device__ __forceinline__ Stat warp_join(Stat a, float c) {
  float r = a.ref;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) r = max_nan(r, __shfl_xor_sync(0xffffffffu, r, o));
  move_ref(a, r, c);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
    a.u += __shfl_xor_sync(0xffffffffu, a.u, o);
  }
  return a;
}

// What a row needs of its statistics.
struct RowSum {
  float ref, log2s, lse, entropy;
  bool empty;       // nothing above -inf
  __device__ __forceinline__ RowSum(const Stat& a, float inv_tau) {
    empty = a.s == 0.f;
    ref = a.ref;
    log2s = log2f(a.s);
    lse = empty ? -INFINITY : fmaf(a.ref, inv_tau, log2s * kLn2);
    entropy = empty ? 0.f : max_nan((log2s - a.u / a.s) * kLn2, 0.f);
  }
  __device__ __forceinline__ float logp(float x, float c) const {
    if (x == -INFINITY) return log2s != log2s ? log2s : x;
    return fmaf(x - ref, c, -log2s) * kLn2;
  }
};

// ---- top alternatives -------------------------------------------------------------------------------------------------
// Candidates are 64-bit keys that order by logit, then by lowest index.  Logits at -inf are no alternatives.
constexpr uint32_t kKeyNegInf = 0x007fffffu;     // order_bits(-inf)
constexpr int kCandBlock = 1024, kCandWarp = 128;

__device__ __forceinline__ uint32_t order_bits(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);   // -0 counts as 0
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float from_order_bits(uint32_t k) {
  return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ unsigned long long cand_key(uint32_t bits, int j) {
  return ((unsigned long long)bits << 32) | (0xffffffffu - (uint32_t)j);
}

template <int NT>
struct TopShared {
  static constexpr int kCap = NT == 32 ? kCandWarp : kCandBlock;
  unsigned long long cand[kCap];
  unsigned long long best[kMaxTopK];           // the group's own k best, in order
  unsigned long long wmax[Group<NT>::kWarps];
  uint32_t wthr[Group<NT>::kWarps];
  int wcount[Group<NT>::kWarps];
  int n;
};

// Calls f(order bits, index) for every element of this thread.
template <class T, int NT, class F>
__device__ __forceinline__ void each_element(const Slice<T>& sl, F f) {
  constexpr int EV = Elem<T>::EV;
  const int t = Group<NT>::tid();
#pragma unroll 2
  for (int v = sl.v0 + t; v < sl.v1; v += NT) {
    float x[EV];
    Elem<T>::unpack(load16(sl.vec(v)), x);
#pragma unroll
    for (int i = 0; i < EV; ++i) f(order_bits(x[i]), sl.head + v * EV + i);
  }
  const int j = sl.edge(t);
  if (j >= 0) f(order_bits(Elem<T>::to_float(sl.row[j])), j);
}

// The k largest of sh.cand[0..n) in order into sh.best (0 where there are fewer): a candidate's place is the number of
// keys above it.
template <int NT>
__device__ __forceinline__ void rank_candidates(TopShared<NT>& sh, int n, int k) {
  const int t = Group<NT>::tid();
  for (int i = t; i < k; i += NT) sh.best[i] = 0ull;
  Group<NT>::sync();
  for (int i = t; i < n; i += NT) {
    const unsigned long long key = sh.cand[i];
    int place = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) place += sh.cand[j] > key;
    if (place < k && key) sh.best[place] = key;
  }
  Group<NT>::sync();
}

// The k best of the group's slice into sh.best.  `top` is this thread's largest logit (-inf if it has none).
//
// Threshold: every warp names its ceil(k / warps)-th largest of its lanes' maxima; the smallest of those has at least k
// elements at or above it, so only the elements that reach it can be among the k best, typically a few dozen: the few
// threads that own them read their part of the row again (from L2) and hand them over.  When more than kCap reach it
// (thousands of equal logits), elements above it are taken first and the ones equal to it by a scan in index order that
// ends as soon as enough are found; and when even too many lie above it, k rounds of an arg-max do it.
template <class T, int NT>
__device__ void top_of_slice(TopShared<NT>& sh, const Slice<T>& sl, float top, int k) {
  using G = Group<NT>;
  constexpr int kCap = TopShared<NT>::kCap;
  const int t = G::tid(), lane = threadIdx.x & 31, w = NT == 32 ? 0 : (int)(threadIdx.x >> 5);
  const uint32_t mine = order_bits(top);
  uint32_t left = mine, thr = 0;
  for (int i = (k + G::kWarps - 1) / G::kWarps; i > 0; --i) {
    thr = __reduce_max_sync(0xffffffffu, left);
    const uint32_t who = __ballot_sync(0xffffffffu, left == thr);
    if (lane == __ffs(who) - 1) left = 0;
  }
  if (t == 0) sh.n = 0;
  if (lane == 0) sh.wthr[w] = thr;
  G::sync();
  thr = sh.wthr[0];
#pragma unroll
  for (int i = 1; i < G::kWarps; ++i) thr = min(thr, sh.wthr[i]);
  thr = max(thr, kKeyNegInf + 1);
  if (mine >= thr)
    each_element<T, NT>(sl, [&](uint32_t b, int j) {
      if (b >= thr) {
        const int at = atomicAdd(&sh.n, 1);
        if (at < kCap) sh.cand[at] = cand_key(b, j);
      }
    });
  G::sync();
  int n = sh.n;
  if (n > kCap) {
    G::sync();
    if (t == 0) sh.n = 0;
    G::sync();
    if (mine > thr)
      each_element<T, NT>(sl, [&](uint32_t b, int j) {
        if (b > thr) {
          const int at = atomicAdd(&sh.n, 1);
          if (at < kCap) sh.cand[at] = cand_key(b, j);
        }
      });
    G::sync();
    n = sh.n;
    if (n > kCap - kMaxTopK) {
      unsigned long long last = ~0ull;
      int found = 0;
      for (; found < k; ++found) {
        unsigned long long best = 0ull;
        each_element<T, NT>(sl, [&](uint32_t b, int j) {
          const unsigned long long key = cand_key(b, j);
          if (b > kKeyNegInf && key < last && key > best) best = key;
        });
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
          const unsigned long long other = __shfl_xor_sync(0xffffffffu, best, o);
          if (other > best) best = other;
        }
        G::sync();
        if (lane == 0) sh.wmax[w] = best;
        G::sync();
        for (int i = 0; i < G::kWarps; ++i)
          if (sh.wmax[i] > best) best = sh.wmax[i];
        if (best == 0ull) break;              // uniform: every thread holds the same maximum
        if (t == 0) sh.cand[found] = best;
        last = best;
      }
      n = found;
      G::sync();
    } else {
      for (int base = sl.e0; n < k && base < sl.e1; base += NT) {     // ties at the threshold, lowest index first
        const int j = base + t;
        const bool hit = j < sl.e1 && order_bits(Elem<T>::to_float(sl.row[j])) == thr;
        const uint32_t b = __ballot_sync(0xffffffffu, hit);
        if (lane == 0) sh.wcount[w] = __popc(b);
        G::sync();
        int before = __popc(b & ((1u << lane) - 1u)), all = 0;
        for (int i = 0; i < G::kWarps; ++i) {
          if (i < w) before += sh.wcount[i];
          all += sh.wcount[i];
        }
        if (hit && n + before < k) sh.cand[n + before] = cand_key(thr, j);
        n = min(n + all, k);
        G::sync();
      }
    }
  }
  rank_candidates<NT>(sh, n, k);
}

// ---- the teacher's side of one row ------------------------------------------------------------------------------------
// One warp: entry i = lane + 32 e.  q and log q (natural), a column index or -1 where there is no entry.
struct Teacher {
  float q[kMaxTeacher / 32], logq[kMaxTeacher / 32];
  int a[kMaxTeacher / 32];
  bool any, bad;       // a live entry; an index outside the vocabulary

  __device__ __forceinline__ void read(const int32_t* idx, const float* val, int K, int V, float inv_tau) {
    const int lane = threadIdx.x & 31;
    float x[kMaxTeacher / 32];
    float mx = -INFINITY;
    bool have = false, out = false;
#pragma unroll
    for (int e = 0; e < kMaxTeacher / 32; ++e) {
      const int i = lane + 32 * e;
      a[e] = i < K ? idx[i] : -1;
      if (a[e] >= V) {
        out = true;
        a[e] = -1;
      }
      x[e] = a[e] >= 0 ? val[i] : -INFINITY;
      have |= a[e] >= 0;
      mx = max_nan(mx, x[e]);
    }
    any = __any_sync(0xffffffffu, have || out);
    bad = __any_sync(0xffffffffu, out);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    if (mx == -INFINITY && !bad) any = false;       // a teacher whose every entry is masked asks for nothing
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < kMaxTeacher / 32; ++e) {
      x[e] = x[e] == -INFINITY ? -INFINITY : (x[e] - mx) * inv_tau;
      q[e] = expf(x[e]);
      sum += q[e];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float ls = logf(sum), inv = 1.f / sum;
#pragma unroll
    for (int e = 0; e < kMaxTeacher / 32; ++e) {
      q[e] *= inv;
      logq[e] = x[e] - ls;
      if (a[e] < 0 || !any) q[e] = 0.f;
    }
  }
  // sum_i q_i (log q_i - log p_i) over the warp's entries, x: the student's logits at the entries
  __device__ __forceinline__ float divergence(const float (&x)[kMaxTeacher / 32], const RowSum& r, float c) const {
    float kl = 0.f;
#pragma unroll
    for (int e = 0; e < kMaxTeacher / 32; ++e)
      if (!(q[e] == 0.f)) kl += q[e] * (logq[e] - r.logp(x[e], c));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) kl += __shfl_xor_sync(0xffffffffu, kl, o);
    return bad ? __int_as_float(0x7fc00000) : kl;
  }
};

// ---- forward ----------------------------------------------------------------------------------------------------------
struct ForwardArgs {
  const void* x;
  long long ld, T;
  int V, ranks, k, K;
  long long ld_teacher;
  float c, inv_tau, tau;
  const int32_t* tokens;
  float *logprob, *entropy, *lse;
  int32_t* top_tokens;
  float* top_logprobs;
  const int32_t* teacher_tokens;
  const float* teacher_logits;
  float* loss;
};

// One pass over the logits: DISTILL = false for token_logprobs, true for the loss of distill without its gradient.
template <class T, int NT, bool DISTILL>
__global__ void __launch_bounds__(NT == 32 ? kWarpBlock : kBlock, NT == 32 ? 8 : 4) rows_forward_kernel(const ForwardArgs A) {
  using G = Group<NT>;
  __shared__ TopShared<NT> top_sh[G::kRowsPerBlock];
  __shared__ Stat wstat[G::kRowsPerBlock][G::kWarps];
  const int t = G::tid(), lane = threadIdx.x & 31, w = NT == 32 ? 0 : (int)(threadIdx.x >> 5);
  const int ranks = NT == 32 ? 1 : A.ranks;
  const int rank = NT == 32 ? 0 : (int)(blockIdx.x % (unsigned)ranks);
  const long long row = NT == 32 ? (long long)blockIdx.x * G::kRowsPerBlock + G::slot() : (long long)(blockIdx.x / (unsigned)ranks);
  if (NT == 32 && row >= A.T) return;
  TopShared<NT>& sh = top_sh[G::slot()];
  const T* xr = reinterpret_cast<const T*>(A.x) + row * A.ld;
  const int k = DISTILL ? 0 : A.k;

  const Slice<T> sl(xr, A.V, rank, ranks);
  const float c = A.c;
  int token = -1;
  if (!DISTILL && A.tokens) token = A.tokens[row];
  // the first batch is on its way before anything is known about the row
  int v = sl.v0 + t;
  uint4 x[kBatch];
  bool more = v + (kBatch - 1) * NT < sl.v1;
  if (more) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) x[i] = load16(sl.vec(v + i * NT));
  }
  const bool bad_token = token >= A.V;
  bool live = DISTILL || !A.tokens || token >= 0;
  Teacher te;
  if (DISTILL && w == 0 && rank == 0) {
    te.read(A.teacher_tokens + row * A.ld_teacher, A.teacher_logits + row * A.ld_teacher, A.K, A.V, A.inv_tau);
    live = te.any;                       // this warp writes the row's result; the row is read in any case
  }
  Stat a{kUnset, 0.f, 0.f};
  float top = -INFINITY;
  if (DISTILL || live) {
    while (more) {
      uint4 y[kBatch];
      v += kBatch * NT;
      more = v + (kBatch - 1) * NT < sl.v1;
      if (more) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) y[i] = load16(sl.vec(v + i * NT));
      }
      add_vectors<T, kBatch, !DISTILL>(a, top, x, c);
#pragma unroll
      for (int i = 0; i < kBatch; ++i) x[i] = y[i];
    }
    for (; v < sl.v1; v += NT) {
      uint4 y[1];
      y[0] = load16(sl.vec(v));
      add_vectors<T, 1, !DISTILL>(a, top, y, c);
    }
    const int j = sl.edge(t);
    if (j >= 0) {
      const float e[1] = {Elem<T>::to_float(xr[j])};
      top = max_nan(top, e[0]);
      follow(a, e[0], c);
      add_elements<1, !DISTILL>(a, e, c);
    }
  }
  a = warp_join(a, c);
  if (NT > 32) {
    if (lane == 0) wstat[0][w] = a;
    __syncthreads();
    a = wstat[0][0];
#pragma unroll
    for (int i = 1; i < G::kWarps; ++i) a = join(a, wstat[0][i], c);
  }
  const bool alternatives = !DISTILL && k > 0 && live;
  if (alternatives) top_of_slice<T, NT>(sh, sl, top, k);
  if (ranks > 1) {       // the first block of the cluster takes the others' results
    cg::cluster_group cluster = cg::this_cluster();
    __syncthreads();
    if (t == 0) wstat[0][0] = a;
    cluster.sync();
    if (rank == 0) {
      for (int r = 1; r < ranks; ++r) a = join(a, *cluster.map_shared_rank(&wstat[0][0], r), c);
      if (alternatives) {
        for (int i = t; i < ranks * kMaxTopK; i += NT)
          sh.cand[i] = i % kMaxTopK < k ? cluster.map_shared_rank(sh.best, i / kMaxTopK)[i % kMaxTopK] : 0ull;
        __syncthreads();
      }
    }
    cluster.sync();
    if (rank != 0) return;
    if (alternatives) rank_candidates<NT>(sh, ranks * kMaxTopK, k);
  }
  const RowSum r(a, A.inv_tau);
  if (DISTILL) {
    if (w == 0) {
      float kl = 0.f;
      if (live) {
        float xs[kMaxTeacher / 32];
#pragma unroll
        for (int e = 0; e < kMaxTeacher / 32; ++e) xs[e] = te.a[e] >= 0 ? Elem<T>::to_float(xr[te.a[e]]) : 0.f;
        kl = r.empty && !te.bad ? INFINITY : te.divergence(xs, r, c);
      }
      if (lane == 0) {
        A.loss[row] = live ? A.tau * A.tau * kl : 0.f;
        if (A.lse) A.lse[row] = live ? r.lse : 0.f;
      }
    }
    return;
  }
  if (t == 0) {
    if (A.logprob) A.logprob[row] = !live ? 0.f : bad_token ? __int_as_float(0x7fc00000) : r.logp(Elem<T>::to_float(xr[token]), c);
    if (A.entropy) A.entropy[row] = live ? r.entropy : 0.f;
    if (A.lse) A.lse[row] = live ? r.lse : 0.f;
  }
  for (int i = t; i < k; i += NT) {
    const bool nan = live && r.log2s != r.log2s;
    const unsigned long long key = live && !nan ? sh.best[i] : 0ull;
    A.top_tokens[row * k + i] = key ? (int32_t)(0xffffffffu - (uint32_t)key) : -1;
    A.top_logprobs[row * k + i] = nan ? r.log2s : key ? r.logp(from_order_bits((uint32_t)(key >> 32)), c) : -INFINITY;
  }
}

// ---- gradients --------------------------------------------------------------------------------------------------------
struct GradArgs {
  const void* x;
  void* dx;
  long long ld, ld_d, T;
  int V, ranks, K;
  long long ld_teacher;
  float c, inv_tau, inv_tau_lo, tau;
  const int32_t* tokens;
  const float *lse_in, *entropy, *d_logprob, *d_entropy;
  const int32_t* teacher_tokens;
  const float* teacher_logits;
  const float* d_loss;
  float *loss, *lse_out;
};

enum GradMode { kLogprobsGrad, kDistillGrad, kDistillStep };

template <class T>
__device__ __forceinline__ void store_vec(T* dst, const float (&y)[Elem<T>::EV], bool aligned) {
  if (aligned) {
    *reinterpret_cast<uint4*>(dst) = Elem<T>::pack(y);
  } else {
#pragma unroll
    for (int i = 0; i < Elem<T>::EV; ++i) dst[i] = Elem<T>::from_float(y[i]);
  }
}

// log p of x, natural, from an lse handed over in fp32.  For fp32 logits 1 / tau is taken as two fp32 terms: its
// rounding alone would shift every log p by 2^-24 of s, which the fp32 gradient shows.
template <class T>
__device__ __forceinline__ float logp_from_lse(float x, const GradArgs& A, float lse) {
  if (sizeof(T) == 4) return fmaf(x, A.inv_tau, fmaf(x == -INFINITY ? 0.f : x, A.inv_tau_lo, -lse));
  return fmaf(x, A.inv_tau, -lse);
}

// A thread keeps its R vectors of the row in registers, so the gradient in the same call as the loss reads the logits
// once: all loads, the statistics, their join over the group, all stores.  With the statistics handed over (kLogprobsGrad,
// kDistillGrad) there is no join and `ranks` is any number of independent pieces of the row.
template <class T, int NT, int R, int MODE>
__global__ void __launch_bounds__(NT == 32 ? kWarpBlock : kBlock, R > 8 ? 2 : R > 4 ? 3 : 4) rows_gradient_kernel(const GradArgs A) {
  using G = Group<NT>;
  constexpr int EV = Elem<T>::EV;
  constexpr bool kTeacher = MODE != kLogprobsGrad, kStep = MODE == kDistillStep;
  __shared__ Stat wstat[G::kRowsPerBlock][G::kWarps];
  __shared__ Stat cstat[kMaxCluster];
  __shared__ float sh_q[kTeacher ? G::kRowsPerBlock : 1][kMaxTeacher], sh_x[kTeacher ? G::kRowsPerBlock : 1][kMaxTeacher];
  __shared__ int sh_a[kTeacher ? G::kRowsPerBlock : 1][kMaxTeacher], sh_flags[G::kRowsPerBlock];
  const int t = G::tid(), lane = threadIdx.x & 31, w = NT == 32 ? 0 : (int)(threadIdx.x >> 5), slot = G::slot();
  const int ranks = NT == 32 ? 1 : A.ranks;
  const int rank = NT == 32 ? 0 : (int)(blockIdx.x % (unsigned)ranks);
  const long long row = NT == 32 ? (long long)blockIdx.x * G::kRowsPerBlock + slot : (long long)(blockIdx.x / (unsigned)ranks);
  if (NT == 32 && row >= A.T) return;
  const T* xr = reinterpret_cast<const T*>(A.x) + row * A.ld;
  T* dr = reinterpret_cast<T*>(A.dx) + row * A.ld_d;
  const Slice<T> sl(xr, A.V, rank, ranks);
  const bool aligned = ((((uintptr_t)xr) ^ ((uintptr_t)dr)) & 15u) == 0;   // vectors of x are vectors of dx
  const int edge = sl.edge(t);
  const float c = A.c;
  int token = -1;
  bool live = true;
  if (!kTeacher) {
    token = A.tokens[row];
    live = token >= 0;
  }
  const float lse = kStep ? 0.f : A.lse_in[row];
  if (!kStep && lse <= kEmptyLse) live = false;       // nothing left by the masks

  // the row's vectors are on their way before the teacher's entries are looked at; a row without any is read for nothing
  uint4 v[R];
  float xe = -INFINITY;
  if (kStep) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int at = sl.v0 + t + i * NT;
      if (at < sl.v1) v[i] = load16(sl.vec(at));
      else v[i] = make_uint4(Elem<T>::kNegInf, Elem<T>::kNegInf, Elem<T>::kNegInf, Elem<T>::kNegInf);
    }
    if (edge >= 0) xe = Elem<T>::to_float(xr[edge]);
  }
  float xs[kMaxTeacher / 32];
  Teacher te;
  if (kTeacher && w == 0) {
    te.read(A.teacher_tokens + row * A.ld_teacher, A.teacher_logits + row * A.ld_teacher, A.K, A.V, A.inv_tau);
    if (lane == 0) sh_flags[slot] = (te.any ? 1 : 0) | (te.bad ? 2 : 0);
    live = live && te.any;
#pragma unroll
    for (int e = 0; e < kMaxTeacher / 32; ++e) {
      // the first rank needs all of them for the loss, every rank its own slice's for the gradient
      const bool need = te.a[e] >= 0 && live && ((kStep && rank == 0) || (te.a[e] >= sl.e0 && te.a[e] < sl.e1));
      xs[e] = need ? Elem<T>::to_float(xr[te.a[e]]) : 0.f;
      sh_a[slot][lane + 32 * e] = te.a[e];
      sh_q[slot][lane + 32 * e] = te.q[e];
      sh_x[slot][lane + 32 * e] = xs[e];
    }
  }

  float ref = 0.f, log2s = 0.f;
  bool empty = false;
  if (kStep) {
    cg::cluster_group cluster = cg::this_cluster();
    if (ranks > 1) cluster.barrier_arrive();          // every block of the cluster runs before its memory is written
    Stat a{max_nan(max_nan(Elem<T>::largest(v), xe), kUnset), 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < R; ++i) {
      float x[EV];
      Elem<T>::unpack(v[i], x);
      add_elements<EV, false>(a, x, c);
    }
    const float e1[1] = {xe};
    add_elements<1, false>(a, e1, c);
    a = warp_join(a, c);
    if (NT > 32) {
      if (lane == 0) wstat[0][w] = a;
      __syncthreads();
      a = wstat[0][0];
#pragma unroll
      for (int i = 1; i < G::kWarps; ++i) a = join(a, wstat[0][i], c);
    }
    if (ranks > 1) {
      cluster.barrier_wait();
      if (t < ranks) *cluster.map_shared_rank(&cstat[rank], t) = a;
      cluster.sync();
      a = cstat[0];
      for (int i = 1; i < ranks; ++i) a = join(a, cstat[i], c);
    }
    const RowSum r(a, A.inv_tau);
    ref = r.ref;
    log2s = r.log2s;
    empty = r.empty;
    if (rank == 0 && w == 0) {
      const float kl = !live ? 0.f : empty && !te.bad ? INFINITY : te.divergence(xs, r, c);
      if (lane == 0) {
        A.loss[row] = live ? A.tau * A.tau * kl : 0.f;
        if (A.lse_out) A.lse_out[row] = live ? r.lse : 0.f;
      }
    }
  }

  // dx_j = p_j (ca + cb log p_j), then the entries that have a term of their own
  float ca, cb = 0.f, cy = 0.f;
  bool bad = false;
  if (kTeacher) {
    G::sync();
    live = live && (sh_flags[slot] & 1);
    bad = (sh_flags[slot] & 2) != 0;
    ca = bad ? __int_as_float(0x7fc00000) : A.d_loss[row] * A.tau;
  } else {
    const float g = A.d_logprob ? A.d_logprob[row] : 0.f, h = A.d_entropy ? A.d_entropy[row] : 0.f;
    cb = -h * A.inv_tau;
    ca = -(g + (A.d_entropy ? h * A.entropy[row] : 0.f)) * A.inv_tau;
    cy = g * A.inv_tau;
    if (token >= A.V) ca = __int_as_float(0x7fc00000);
  }
  const bool zero = !live || empty;
  auto grad = [&](float x) -> float {
    if (kStep) return ca * ex2(fmaf(x - ref, c, -log2s));
    float lp = logp_from_lse<T>(x, A, lse);
    if (MODE == kDistillGrad) return ca * ex2(lp * kLog2e);
    lp = max_nan(lp, -1e4f);
    return ex2(lp * kLog2e) * fmaf(cb, lp, ca);
  };
  auto put = [&](const uint4& xv, int at) {
    float x[EV], y[EV];
    Elem<T>::unpack(xv, x);
    const int j0 = sl.head + at * EV;
#pragma unroll
    for (int i = 0; i < EV; ++i) {
      y[i] = zero ? 0.f : grad(x[i]);
    }
    if (!kTeacher && !zero && (unsigned)(token - j0) < (unsigned)EV) {
#pragma unroll
      for (int i = 0; i < EV; ++i)
        if (j0 + i == token) y[i] += cy;
    }
    store_vec<T>(dr + j0, y, aligned);
  };
  if (kStep) {
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int at = sl.v0 + t + i * NT;
      if (at < sl.v1) put(v[i], at);
    }
  } else {
    for (int b = sl.v0 + t; b < sl.v1; b += R * NT) {
      if (!zero) {
#pragma unroll
        for (int i = 0; i < R; ++i)
          if (b + i * NT < sl.v1) v[i] = load16(sl.vec(b + i * NT));
      }
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (b + i * NT < sl.v1) put(v[i], b + i * NT);
    }
    if (edge >= 0 && !zero) xe = Elem<T>::to_float(xr[edge]);
  }
  if (edge >= 0) {
    float y = zero ? 0.f : grad(xe);
    if (!kTeacher && !zero && edge == token) y += cy;
    dr[edge] = Elem<T>::from_float(y);
  }
  if (kTeacher) {
    // the teacher's columns: p_j minus all of the teacher's mass there (the same column may come more than once; every
    // entry then writes the same value), over what the loop above wrote
    G::sync();
    if (zero || bad) return;
    for (int i = t; i < A.K; i += NT) {
      const int j = sh_a[slot][i];
      if (j < sl.e0 || j >= sl.e1) continue;
      float q = 0.f;
      for (int o = 0; o < A.K; ++o)
        if (sh_a[slot][o] == j) q += sh_q[slot][o];
      const float x = sh_x[slot][i];
      const float p = kStep ? ex2(fmaf(x - ref, c, -log2s)) : ex2(logp_from_lse<T>(x, A, lse) * kLog2e);
      dr[j] = Elem<T>::from_float(ca * (p - q));
    }
  }
}

// ---- host -------------------------------------------------------------------------------------------------------------
constexpr int kSMs = 148;

template <class Args>
cudaError_t launch(void (*kernel)(const Args), const Args& A, long long blocks, int threads, int cluster, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)cluster;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, A);
}

// Blocks per row of a forward pass: rows alone fill the GPU (four blocks an SM) or are split, down to two vectors a
// thread, over up to eight blocks.
int forward_ranks(long long T, long long nvec) {
  int ranks = 1;
  while (ranks < kMaxCluster && T * ranks < 4 * kSMs && nvec > (long long)ranks * 2 * kBlock) ranks *= 2;
  return ranks;
}

template <class T, bool DISTILL>
cudaError_t forward(ForwardArgs& A, cudaStream_t st) {
  if (A.V <= kWarpRow) {
    A.ranks = 1;
    return launch(rows_forward_kernel<T, 32, DISTILL>, A, (A.T + 3) / 4, kWarpBlock, 1, st);
  }
  A.ranks = forward_ranks(A.T, A.V / Elem<T>::EV);
  return launch(rows_forward_kernel<T, kBlock, DISTILL>, A, A.T * A.ranks, kBlock, A.ranks, st);
}

template <class T, int MODE>
cudaError_t gradient(GradArgs& A, cudaStream_t st) {
  const long long nvec = A.V / Elem<T>::EV;
  if (A.V <= kWarpRow) {
    A.ranks = 1;
    constexpr int R = kWarpRow / Elem<T>::EV / 32;
    return launch(rows_gradient_kernel<T, 32, R, MODE>, A, (A.T + 3) / 4, kWarpBlock, 1, st);
  }
  if constexpr (MODE != kDistillStep) {
    // pieces of 4 vectors a thread, at least one; larger where the grid would pass 2^31 blocks
    long long ranks = (nvec + 4 * kBlock - 1) / (4 * kBlock);
    while (A.T * ranks > 0x7fffffffll) ranks = (ranks + 1) / 2;
    A.ranks = ranks < 1 ? 1 : (int)ranks;
    return launch(rows_gradient_kernel<T, kBlock, 4, MODE>, A, A.T * A.ranks, kBlock, 1, st);
  } else {
    int ranks = 1;
    while (ranks < kMaxCluster &&
           (nvec > (long long)ranks * 8 * kBlock || (A.T * ranks < 3 * kSMs && nvec > (long long)ranks * 2 * kBlock)))
      ranks *= 2;
    A.ranks = ranks;
    const long long per = (nvec + ranks - 1) / ranks;
    if (per <= 4 * kBlock) return launch(rows_gradient_kernel<T, kBlock, 4, MODE>, A, A.T * ranks, kBlock, ranks, st);
    if (per <= 8 * kBlock) return launch(rows_gradient_kernel<T, kBlock, 8, MODE>, A, A.T * ranks, kBlock, ranks, st);
    return launch(rows_gradient_kernel<T, kBlock, 16, MODE>, A, A.T * ranks, kBlock, ranks, st);
  }
}

// whether a row fits the registers of eight blocks
template <class T>
bool step_fits(long long V) {
  return V / Elem<T>::EV <= (long long)kMaxCluster * 16 * kBlock;
}

template <template <class> class Call, class Args>
cudaError_t by_dtype(int dtype, Args& A, cudaStream_t st) {
  switch (dtype) {
    case LAQ_F32: return Call<float>::run(A, st);
    case LAQ_BF16: return Call<__nv_bfloat16>::run(A, st);
    default: return Call<__half>::run(A, st);
  }
}
template <class T> struct LogprobsForward { static cudaError_t run(ForwardArgs& A, cudaStream_t st) { return forward<T, false>(A, st); } };
template <class T> struct DistillForward { static cudaError_t run(ForwardArgs& A, cudaStream_t st) { return forward<T, true>(A, st); } };
template <class T> struct LogprobsGradient { static cudaError_t run(GradArgs& A, cudaStream_t st) { return gradient<T, kLogprobsGrad>(A, st); } };
template <class T> struct DistillGradient { static cudaError_t run(GradArgs& A, cudaStream_t st) { return gradient<T, kDistillGrad>(A, st); } };
template <class T> struct DistillStep { static cudaError_t run(GradArgs& A, cudaStream_t st) { return gradient<T, kDistillStep>(A, st); } };

struct Err {
  char* buf;
  size_t len;
};

laq_status check_rows(const Err& e, const void* x, int dtype, int64_t T, int64_t V, int64_t ld, float tau) {
  if (e.buf && e.len) e.buf[0] = 0;
  const int bytes = dtype_bytes(dtype);
  if (!bytes) return fail(e.buf, e.len, LAQ_EINVAL, "dtype must be LAQ_F32, LAQ_BF16 or LAQ_F16");
  if (T < 0 || T > 0x7fffffffll / kMaxCluster) return fail(e.buf, e.len, LAQ_EINVAL, "rows must be 0..2^28-1");
  if (V < 1 || V > 0x7fffff00ll) return fail(e.buf, e.len, LAQ_EINVAL, "vocab must be 1..2^31-256");
  if (ld < V) return fail(e.buf, e.len, LAQ_EINVAL, "a row stride must be at least vocab");
  if (!(tau >= 1e-4f && tau <= 1e4f)) return fail(e.buf, e.len, LAQ_EINVAL, "temperature must be 1e-4..1e4");
  if (T == 0) return LAQ_OK;
  if (!x) return fail(e.buf, e.len, LAQ_EINVAL, "null pointer");
  if (((uintptr_t)x % (uintptr_t)bytes) != 0) return fail(e.buf, e.len, LAQ_EINVAL, "logits are not aligned to their element size");
  const char* msg = wrong_device(x);
  return msg ? fail(e.buf, e.len, LAQ_EINVAL, "%s", msg) : LAQ_OK;
}

laq_status check_gradient(const Err& e, const void* x, int64_t ld, const void* dx, int64_t ld_d, int dtype, int64_t T, int64_t V) {
  const int bytes = dtype_bytes(dtype);
  if (!dx) return fail(e.buf, e.len, LAQ_EINVAL, "null pointer");
  if (((uintptr_t)dx % (uintptr_t)bytes) != 0) return fail(e.buf, e.len, LAQ_EINVAL, "the gradient is not aligned to its element size");
  if (ld_d < V) return fail(e.buf, e.len, LAQ_EINVAL, "a row stride must be at least vocab");
  const uintptr_t a0 = (uintptr_t)x, a1 = a0 + ((uintptr_t)(T - 1) * ld + V) * bytes;
  const uintptr_t b0 = (uintptr_t)dx, b1 = b0 + ((uintptr_t)(T - 1) * ld_d + V) * bytes;
  if (a0 < b1 && b0 < a1 && !(a0 == b0 && ld == ld_d))
    return fail(e.buf, e.len, LAQ_EINVAL, "the gradient overlaps the logits: it may be the same tensor or a separate one");
  return LAQ_OK;
}

laq_status done(const Err& e, cudaError_t rc) {
  const cudaError_t last = cudaGetLastError();
  if (rc == cudaSuccess) rc = last;
  return rc == cudaSuccess ? LAQ_OK : fail(e.buf, e.len, LAQ_ECUDA, "kernel launch failed: %s", cudaGetErrorString(rc));
}

void set_temperature(ForwardArgs& A, float tau) {
  A.tau = tau;
  A.inv_tau = (float)(1.0 / (double)tau);
  A.c = (float)(1.4426950408889634 / (double)tau);
}
void set_temperature(GradArgs& A, float tau) {
  A.tau = tau;
  A.inv_tau = (float)(1.0 / (double)tau);
  A.inv_tau_lo = (float)(1.0 / (double)tau - (double)A.inv_tau);
  A.c = (float)(1.4426950408889634 / (double)tau);
}

}  // namespace
}  // namespace ops
}  // namespace laq

using namespace laq::ops;

extern "C" laq_status laq_token_logprobs(const void* d_logits, int32_t dtype, int64_t rows, int64_t vocab, int64_t row_stride,
                                         float temperature, const int32_t* d_tokens, int32_t top_k, float* d_logprob,
                                         float* d_entropy, float* d_lse, int32_t* d_top_tokens, float* d_top_logprobs,
                                         void* cuda_stream, char* errbuf, size_t errbuf_len) {
  const Err e{errbuf, errbuf_len};
  const laq_status st = check_rows(e, d_logits, dtype, rows, vocab, row_stride, temperature);
  if (st != LAQ_OK) return st;
  if (top_k < 0 || top_k > kMaxTopK) return fail(errbuf, errbuf_len, LAQ_EINVAL, "top_k must be 0..32");
  if (rows == 0) return LAQ_OK;
  if (d_logprob && !d_tokens) return fail(errbuf, errbuf_len, LAQ_EINVAL, "log probabilities need tokens");
  if (top_k && (!d_top_tokens || !d_top_logprobs)) return fail(errbuf, errbuf_len, LAQ_EINVAL, "null pointer");
  ForwardArgs A = {};
  A.x = d_logits;
  A.ld = row_stride;
  A.T = rows;
  A.V = (int)vocab;
  A.k = top_k;
  set_temperature(A, temperature);
  A.tokens = d_tokens;
  A.logprob = d_logprob;
  A.entropy = d_entropy;
  A.lse = d_lse;
  A.top_tokens = d_top_tokens;
  A.top_logprobs = d_top_logprobs;
  return done(e, by_dtype<LogprobsForward>(dtype, A, (cudaStream_t)cuda_stream));
}

extern "C" laq_status laq_token_logprobs_backward(const void* d_logits, int32_t dtype, int64_t rows, int64_t vocab,
                                                  int64_t row_stride, float temperature, const int32_t* d_tokens,
                                                  const float* d_lse, const float* d_entropy, const float* d_grad_logprob,
                                                  const float* d_grad_entropy, void* d_grad_logits, int64_t grad_row_stride,
                                                  void* cuda_stream, char* errbuf, size_t errbuf_len) {
  const Err e{errbuf, errbuf_len};
  laq_status st = check_rows(e, d_logits, dtype, rows, vocab, row_stride, temperature);
  if (st != LAQ_OK || rows == 0) return st;
  if (!d_tokens || !d_lse) return fail(errbuf, errbuf_len, LAQ_EINVAL, "null pointer");
  if (d_grad_entropy && !d_entropy) return fail(errbuf, errbuf_len, LAQ_EINVAL, "the gradient of the entropy needs the entropy");
  st = check_gradient(e, d_logits, row_stride, d_grad_logits, grad_row_stride, dtype, rows, vocab);
  if (st != LAQ_OK) return st;
  GradArgs A = {};
  A.x = d_logits;
  A.dx = d_grad_logits;
  A.ld = row_stride;
  A.ld_d = grad_row_stride;
  A.T = rows;
  A.V = (int)vocab;
  set_temperature(A, temperature);
  A.tokens = d_tokens;
  A.lse_in = d_lse;
  A.entropy = d_entropy;
  A.d_logprob = d_grad_logprob;
  A.d_entropy = d_grad_entropy;
  return done(e, by_dtype<LogprobsGradient>(dtype, A, (cudaStream_t)cuda_stream));
}

static laq_status check_teacher(const Err& e, const int32_t* tokens, const float* logits, int32_t K, int64_t stride) {
  if (K < 1 || K > kMaxTeacher) return fail(e.buf, e.len, LAQ_EINVAL, "the teacher's entries per row must be 1..128");
  if (stride < K) return fail(e.buf, e.len, LAQ_EINVAL, "the teacher's row stride must be at least its entries per row");
  if (!tokens || !logits) return fail(e.buf, e.len, LAQ_EINVAL, "null pointer");
  return LAQ_OK;
}

extern "C" laq_status laq_distill(const void* d_logits, int32_t dtype, int64_t rows, int64_t vocab, int64_t row_stride,
                                  float temperature, const int32_t* d_teacher_tokens, const float* d_teacher_logits,
                                  int32_t teacher_k, int64_t teacher_stride, float* d_loss, float* d_lse,
                                  const float* d_grad_loss, void* d_grad_logits, int64_t grad_row_stride, void* cuda_stream,
                                  char* errbuf, size_t errbuf_len) {
  const Err e{errbuf, errbuf_len};
  laq_status st = check_rows(e, d_logits, dtype, rows, vocab, row_stride, temperature);
  if (st != LAQ_OK || rows == 0) return st;
  st = check_teacher(e, d_teacher_tokens, d_teacher_logits, teacher_k, teacher_stride);
  if (st != LAQ_OK) return st;
  if (!d_loss || !d_lse) return fail(errbuf, errbuf_len, LAQ_EINVAL, "null pointer");
  if ((d_grad_loss != nullptr) != (d_grad_logits != nullptr))
    return fail(errbuf, errbuf_len, LAQ_EINVAL, "the gradient needs both the gradient of the loss and a place for the result");
  if (d_grad_logits) {
    st = check_gradient(e, d_logits, row_stride, d_grad_logits, grad_row_stride, dtype, rows, vocab);
    if (st != LAQ_OK) return st;
  }
  cudaStream_t s = (cudaStream_t)cuda_stream;
  const bool fits = dtype == LAQ_F32 ? step_fits<float>(vocab) : step_fits<__half>(vocab);
  if (!d_grad_logits || !fits) {
    ForwardArgs A = {};
    A.x = d_logits;
    A.ld = row_stride;
    A.T = rows;
    A.V = (int)vocab;
    A.K = teacher_k;
    A.ld_teacher = teacher_stride;
    set_temperature(A, temperature);
    A.teacher_tokens = d_teacher_tokens;
    A.teacher_logits = d_teacher_logits;
    A.loss = d_loss;
    A.lse = d_lse;
    st = done(e, by_dtype<DistillForward>(dtype, A, s));
    if (st != LAQ_OK || !d_grad_logits) return st;
    return laq_distill_backward(d_logits, dtype, rows, vocab, row_stride, temperature, d_teacher_tokens, d_teacher_logits,
                                teacher_k, teacher_stride, d_lse, d_grad_loss, d_grad_logits, grad_row_stride, cuda_stream,
                                errbuf, errbuf_len);
  }
  GradArgs A = {};
  A.x = d_logits;
  A.dx = d_grad_logits;
  A.ld = row_stride;
  A.ld_d = grad_row_stride;
  A.T = rows;
  A.V = (int)vocab;
  A.K = teacher_k;
  A.ld_teacher = teacher_stride;
  set_temperature(A, temperature);
  A.teacher_tokens = d_teacher_tokens;
  A.teacher_logits = d_teacher_logits;
  A.d_loss = d_grad_loss;
  A.loss = d_loss;
  A.lse_out = d_lse;
  return done(e, by_dtype<DistillStep>(dtype, A, s));
}

extern "C" laq_status laq_distill_backward(const void* d_logits, int32_t dtype, int64_t rows, int64_t vocab, int64_t row_stride,
                                           float temperature, const int32_t* d_teacher_tokens, const float* d_teacher_logits,
                                           int32_t teacher_k, int64_t teacher_stride, const float* d_lse,
                                           const float* d_grad_loss, void* d_grad_logits, int64_t grad_row_stride,
                                           void* cuda_stream, char* errbuf, size_t errbuf_len) {
  const Err e{errbuf, errbuf_len};
  laq_status st = check_rows(e, d_logits, dtype, rows, vocab, row_stride, temperature);
  if (st != LAQ_OK || rows == 0) return st;
  st = check_teacher(e, d_teacher_tokens, d_teacher_logits, teacher_k, teacher_stride);
  if (st != LAQ_OK) return st;
  if (!d_lse || !d_grad_loss) return fail(errbuf, errbuf_len, LAQ_EINVAL, "null pointer");
  st = check_gradient(e, d_logits, row_stride, d_grad_logits, grad_row_stride, dtype, rows, vocab);
  if (st != LAQ_OK) return st;
  GradArgs A = {};
  A.x = d_logits;
  A.dx = d_grad_logits;
  A.ld = row_stride;
  A.ld_d = grad_row_stride;
  A.T = rows;
  A.V = (int)vocab;
  A.K = teacher_k;
  A.ld_teacher = teacher_stride;
  set_temperature(A, temperature);
  A.teacher_tokens = d_teacher_tokens;
  A.teacher_logits = d_teacher_logits;
  A.lse_in = d_lse;
  A.d_loss = d_grad_loss;
  return done(e, by_dtype<DistillGradient>(dtype, A, (cudaStream_t)cuda_stream));
}
