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
// Times in this file are device times of one call replayed as a graph, its inputs larger than the L2 cache; a call from a
// program adds its host time (13 to 18 us from Python) where the kernel does not hide it.
//
// Element layout of a row: rows start at any element address.  The part between the first and the last 16-byte boundary
// is read as 16-byte vectors, interleaved over the group's threads; the up to EV - 1 elements before and after it ("edge"
// elements) go to one thread each.
#include <cooperative_groups.h>
#include <float.h>

#include <atomic>

#include "laq_ops.cuh"

namespace cg = cooperative_groups;

namespace laq {
namespace ops {
namespace {

constexpr int kBlock = 256;
constexpr int kHalfBlock = 128;        // block of the forward pass when there are many rows
constexpr int kWarpBlock = 128;        // block of the kernels whose rows belong to one warp each
constexpr int kWarpRow = 1024;         // longest row that one warp takes
constexpr int kWarpVectors = 512;      // ... and in 16-byte vectors, where there are many rows
constexpr int kMaxCluster = 8;
constexpr int kMaxTopK = 32;
constexpr int kMaxTeacher = 128;
constexpr int kLogBatch = 2, kBatch = 1 << kLogBatch;  // vectors of the streaming loop that a thread has in flight
constexpr int kRing = 2;               // batches of the streaming loop's ring
constexpr int kForwardBlocks = 4;      // blocks of it on an SM (by shared memory: ring and alternatives)
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kUnset = -FLT_MAX;     // reference of a thread that has seen nothing above -inf
constexpr float kSlack = 8.f;          // a reference may lag the maximum by this many powers of two, see follow()
constexpr float kEmptyLse = -16777216.f;  // -2^24; an lse down here belongs to a row of masks only, see RowSum

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
  // per: vectors of a rank, at least ceil(V / EV / ranks)
  __device__ __forceinline__ Slice(const T* r, int V_, int rank, int ranks, int per) : row(r), V(V_) {
    constexpr int EV = Elem<T>::EV;
    const unsigned mis = (unsigned)((uintptr_t)r & 15u) / (unsigned)sizeof(T);
    head = min((int)((EV - mis) % EV), V);
    nvec = (int)((unsigned)(V - head) / EV);
    tail0 = head + nvec * EV;
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
// d = (x - ref) c with c = log2(e) / tau;  s = sum 2^d, u = sum d 2^d.  ref is any number that no x exceeds by more than
// kSlack / c: it moves only when it must, so the common path has no rescaling.  Two forms of d:
//   |ref c| < kNear   x c - rho with rho = fp32(ref c): one fused operation.  rho itself is the reference then, at most a
//                     quarter of a power of two from ref c; c's rounding is a change of temperature by 2^-25, the same for all.
//   otherwise         (x - ref) c, exact up to two roundings of d itself.  Such a ref is a finite mask (-1e9, -1e10, the type's
//                     lowest value: nothing else has been seen), whose product with c is rounded by many powers of two or
//                     overflows: as a reference, rho would be off by as much.  A NaN or +inf also ends here and stays.
constexpr float kNear = 4194304.f;     // 2^22
// A 16-bit gradient may bear ref c + log2 s as one rounded number up to here, where that is a factor of 2^(2^-13) at most, a sixth
// of half a step of fp16 (at a temperature of 1e-4 and logits of 20 it would be 0.5 %); beyond, the difference comes first.
constexpr float kOneNumber = 4096.f;

struct Stat {
  float ref, s, u;
};

__device__ __forceinline__ bool near_ref(float ref, float c) { return fabsf(ref * c) < kNear; }
__device__ __forceinline__ float scaled(float x, float ref, float c) {
  return near_ref(ref, c) ? fmaf(x, c, -(ref * c)) : (x - ref) * c;
}

__device__ __forceinline__ void move_ref(Stat& a, float ref, float c) {    // ref >= a.ref, or NaN
  // from where a's sums stand (rho or a.ref c, by its own form) to where the new reference's will
  float d;
  if (near_ref(ref, c)) d = near_ref(a.ref, c) ? a.ref * c - ref * c : fmaf(a.ref, c, -(ref * c));
  else d = near_ref(a.ref, c) ? -fmaf(ref, c, -(a.ref * c)) : (a.ref - ref) * c;
  d = max_nan(d, -1e4f);
  const float f = ex2(d);
  a.u = fmaf(d, a.s, a.u) * f;
  a.s *= f;
  a.ref = ref;
}

// The statistics while a thread runs over its vectors: two interleaved sums, two elements an instruction.  With ENTROPY
// the elements are first raised to a bound where 2^d is 0 but d finite (-inf would make 0 * inf of its share of u);
// `plain` is false where there is no such bound or ref is a mask, and the elements then go one by one.
template <class T, bool ENTROPY>
struct Running {
  f32x2 s2, u2, c2, rho2;
  float ref, c;
  uint32_t lo;
  bool plain;

  __device__ __forceinline__ explicit Running(float c_) : s2(0ull), u2(0ull), c2(pair_of(c_, c_)), rho2(0ull), ref(kUnset), c(c_), lo(0u), plain(false) {}
  __device__ __forceinline__ Stat get() const {
    float a, b, d, e;
    split(s2, a, b);
    split(u2, d, e);
    return Stat{ref, a + b, d + e};
  }
  __device__ __forceinline__ void set_ref(float r) {
    ref = r;
    rho2 = pair_of(-(r * c), -(r * c));
    plain = near_ref(r, c);
    if (ENTROPY) {
      lo = plain ? Elem<T>::bound(r - 200.f / c) : 0u;
      plain = plain && lo != 0u;
    }
  }
  // A lag costs precision: entropy and log probabilities are differences of numbers as large as the lag, so that a row with a
  // peak (its entropy below 1, say) shows 2^-24 of it.  With a slack of 32 powers of two peaks never moved the reference: the
  // entropy of 1400 peaked rows of 131072 was off by 1.3e-5 of its value (root mean square), with 8 by 5.6e-7; 4 gives nothing
  // more and its moves cost 1.5 %.
  __device__ __forceinline__ void follow(float mx) {
    if (!((mx - ref) * c <= kSlack)) {          // also taken for NaN
      Stat a = get();
      move_ref(a, mx, c);
      s2 = pair_of(a.s, 0.f);
      u2 = pair_of(a.u, 0.f);
      set_ref(mx);
    }
  }
  __device__ __forceinline__ void one(float x) {
    float d = scaled(x, ref, c);
    if (ENTROPY) d = max_nan(d, -1e4f);
    const float e = ex2(d);
    s2 = add2(s2, pair_of(e, 0.f));
    if (ENTROPY) u2 = add2(u2, pair_of(e * d, 0.f));
  }
  // The vectors of a call have sums of their own before they join the thread's, so that few roundings are relative to a large
  // sum (1400 peaked rows of 131072: entropy 5.6e-7 -> 9.0e-8 of its value, in the same time).
  template <int N>
  __device__ __forceinline__ void add(const uint4 (&v)[N]) {
    if (plain) {
      f32x2 bs = 0ull, bu = 0ull;          // these vectors'
#pragma unroll
      for (int i = 0; i < N; ++i) {
        f32x2 p[Elem<T>::EV / 2];
        Elem<T>::pairs(ENTROPY ? at_least<T>(v[i], lo) : v[i], p);
#pragma unroll
        for (int e = 0; e < Elem<T>::EV / 2; ++e) {
          const f32x2 d = fma2(p[e], c2, rho2), w = ex2x2(d);
          bs = i + e == 0 ? w : add2(bs, w);
          if (ENTROPY) bu = i + e == 0 ? mul2(w, d) : fma2(w, d, bu);
        }
      }
      s2 = add2(s2, bs);
      if (ENTROPY) u2 = add2(u2, bu);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float x[Elem<T>::EV];
        Elem<T>::unpack(v[i], x);
#pragma unroll
        for (int e = 0; e < Elem<T>::EV; ++e) one(x[e]);
      }
    }
  }
};

__device__ __forceinline__ Stat join(Stat a, Stat b, float c) {
  const float r = max_nan(a.ref, b.ref);
  move_ref(a, r, c);
  move_ref(b, r, c);
  a.s += b.s;
  a.u += b.u;
  return a;
}

// The joint statistics of a warp's first LANES lanes (a power of two; the others mirror them), in every lane.
template <int LANES, bool ENTROPY>
__device__ __forceinline__ Stat warp_join(Stat a, float c) {
  float r = a.ref;
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) r = max_nan(r, __shfl_xor_sync(0xffffffffu, r, o));
  move_ref(a, r, c);
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) {
    a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
    if (ENTROPY) a.u += __shfl_xor_sync(0xffffffffu, a.u, o);
  }
  return a;
}

// What a row needs of its statistics.  unit = 1 / (tau c): from powers of two back to natural logarithms, with c as it is.
struct RowSum {
  float ref, log2s, lse, entropy, c, unit, inv_tau;
  bool empty;       // nothing above -inf
  bool masked;      // nothing but masks, finite or not.  A gradient handed lse in fp32 cannot tell p where fp32 no longer
                    // holds units (at -1e9 the rounding of lse is a factor of up to e^32): all gradients are 0 then
  __device__ __forceinline__ RowSum(const Stat& a, float c_, float unit_, float inv_tau_) : c(c_), unit(unit_), inv_tau(inv_tau_) {
    empty = a.s == 0.f;
    ref = a.ref;
    log2s = log2f(a.s);
    lse = empty ? -INFINITY : near_ref(ref, c) ? (ref * c + log2s) * unit : fmaf(ref, inv_tau, log2s * unit);
    masked = lse <= kEmptyLse;
    entropy = empty ? 0.f : max_nan((log2s - a.u / a.s) * unit, 0.f);
  }
  __device__ __forceinline__ float logp(float x) const {
    if (x == -INFINITY) return log2s != log2s ? log2s : x;
    const float d = scaled(x, ref, c);
    if (d == -INFINITY) return lse == -INFINITY ? lse : fmaf(x, inv_tau, -lse);     // a mask at the type's lowest value: x c overflows
    return (d - log2s) * unit;
  }
};

// ---- top alternatives -------------------------------------------------------------------------------------------------
// Candidates are 64-bit keys that order by logit, then by lowest index.  Logits at -inf are no alternatives.
constexpr uint32_t kKeyNegInf = 0x007fffffu;     // order_bits(-inf)
constexpr int kCandBlock = 512, kCandWarp = 128;

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

constexpr int kMaxHits = 512;

template <class T, int NT>
struct TopShared {
  static constexpr int kCap = NT == 32 ? kCandWarp : kCandBlock;
  static constexpr int kSlots = NT == 32 ? 1 : 8192 / (NT * (int)sizeof(T));
  union {                                      // the slots are done with before the first candidate is named
    // largest logit of each thread's runs of batches, and behind the last of them that of its other elements
    alignas(16) T slot[NT == 32 ? 1 : kSlots + 1][NT == 32 ? 16 / sizeof(T) : NT];
    unsigned long long cand[kCap];
  };
  unsigned long long best[kMaxTopK];           // the group's own k best, in order
  unsigned long long wmax[Group<NT>::kWarps];
  uint32_t wthr[Group<NT>::kWarps];
  int wcount[Group<NT>::kWarps];
  int n, nhit;
  uint16_t hit[NT == 32 ? 1 : kMaxHits];
};

// How a thread's vectors fall into batches of kBatch (those it reads together), runs of 2^shift batches (a slot each)
// and a rest of fewer than kBatch vectors and its edge element.
template <class T, int NT>
struct Batches {
  int span, shift;
  __device__ __forceinline__ explicit Batches(const Slice<T>& sl) : span(sl.v1 - sl.v0), shift(0) {
    const int most = (span + kBatch * NT - 1) / (kBatch * NT);
    while ((max(most, 1) - 1) >> shift >= TopShared<T, NT>::kSlots) ++shift;
  }
  __device__ __forceinline__ int of(int t) const {
    const int left = span - t - (kBatch - 1) * NT;
    return left > 0 ? (left + kBatch * NT - 1) / (kBatch * NT) : 0;
  }
  __device__ __forceinline__ int slots() const { return (of(0) + (1 << shift) - 1) >> shift; }      // of any thread at most
};

// f(x, index) for the elements of a vector that are at least thr.
template <class T, class F>
__device__ __forceinline__ void pick(const uint4& v, int j0, float thr, F f) {
  constexpr int EV = Elem<T>::EV;
  const uint4 one[1] = {v};
  if (Elem<T>::largest(one) >= thr) {
    float x[EV];
    Elem<T>::unpack(v, x);
#pragma unroll
    for (int i = 0; i < EV; ++i)
      if (x[i] >= thr) f(x[i], j0 + i);
  }
}

// Hands the elements of a vector that are at least thr to the group's candidates, one reservation for all of them.
template <class T, int NT>
__device__ __forceinline__ void take_vector(TopShared<T, NT>& sh, const uint4& v, int j0, float thr) {
  constexpr int EV = Elem<T>::EV;
  float x[EV];
  Elem<T>::unpack(v, x);
  int count = 0;
#pragma unroll
  for (int i = 0; i < EV; ++i) count += x[i] >= thr;
  if (count == 0) return;
  int at = atomicAdd(&sh.n, count);
#pragma unroll
  for (int i = 0; i < EV; ++i)
    if (x[i] >= thr) {
      if (at < TopShared<T, NT>::kCap) sh.cand[at] = cand_key(order_bits(x[i]), j0 + i);
      ++at;
    }
}

// The same for all elements of this thread.
template <class T, int NT, class F>
__device__ __forceinline__ void each_element(const Slice<T>& sl, float thr, F f) {
  const int t = Group<NT>::tid();
#pragma unroll 4
  for (int v = sl.v0 + t; v < sl.v1; v += NT) pick<T>(load16(sl.vec(v)), sl.head + v * Elem<T>::EV, thr, f);
  const int j = sl.edge(t);
  if (j >= 0) {
    const float x = Elem<T>::to_float(sl.row[j]);
    if (x >= thr) f(x, j);
  }
}

// The k largest of sh.cand[0..n) in order into sh.best, which holds zeros: a candidate's place is the number of keys above
// it, counted by four lanes.
template <class T, int NT>
__device__ __forceinline__ void rank_candidates(TopShared<T, NT>& sh, int n, int k) {
  const int t = Group<NT>::tid(), part = t & 3;
  for (int i0 = 0; i0 < n; i0 += NT / 4) {
    const int i = i0 + (t >> 2);
    const unsigned long long key = i < n ? sh.cand[i] : 0ull;
    int place = 0;
#pragma unroll 4
    for (int j = part; j < n; j += 4) place += sh.cand[j] > key;
    place += __shfl_xor_sync(0xffffffffu, place, 1);
    place += __shfl_xor_sync(0xffffffffu, place, 2);
    if (part == 0 && place < k && key) sh.best[place] = key;
  }
  Group<NT>::sync();
}

// The k best of the group's slice into sh.best.  `top` is this thread's largest logit (-inf if it has none), `rest` that of
// its vectors outside the batches.
//
// Threshold: every warp names its ceil(k / warps)-th largest of its lanes' maxima; the smallest of those has at least k
// elements at or above it, so only the elements that reach it can be among the k best, typically some dozens.  The
// batches that hold them are known from the slots' maxima: the block lists those and reads them once more (from L2), a
// vector a thread, instead of every thread its whole part.  (Four vectors a thread under way at a time are slower, 16384 x
// 16384 bf16 with 20 alternatives 148 -> 160 us: what counts in a selection is its instructions.)  When more than kCap elements (or kMaxHits runs) reach the
// threshold (thousands of equal logits), elements above it are taken first and the ones equal to it by a scan in index order
// that ends as soon as enough are found; and when even too many lie above it, k rounds of an arg-max do it.
template <class T, int NT>
__device__ void top_of_slice(TopShared<T, NT>& sh, const Slice<T>& sl, const uint4* ring, float top, float rest, int k) {
  using G = Group<NT>;
  constexpr int kCap = TopShared<T, NT>::kCap;
  const int t = G::tid(), lane = threadIdx.x & 31, w = NT == 32 ? 0 : (int)(threadIdx.x >> 5);
  const uint32_t mine = order_bits(top);
  uint32_t left = mine, key = 0;
  for (int i = (k + G::kWarps - 1) / G::kWarps; i > 0; --i) {
    key = __reduce_max_sync(0xffffffffu, left);
    const uint32_t who = __ballot_sync(0xffffffffu, left == key);
    if (lane == __ffs(who) - 1) left = 0;
  }
  if (t == 0) sh.n = sh.nhit = 0;
  for (int i = t; i < k; i += NT) sh.best[i] = 0ull;
  if (lane == 0) sh.wthr[w] = key;
  G::sync();
  key = sh.wthr[0];
#pragma unroll
  for (int i = 1; i < G::kWarps; ++i) key = min(key, sh.wthr[i]);
  key = max(key, kKeyNegInf + 1);
  const float thr = from_order_bits(key);
  auto take = [&](float x, int j) {
    const int at = atomicAdd(&sh.n, 1);
    if (at < kCap) sh.cand[at] = cand_key(order_bits(x), j);
  };
  if constexpr (NT == 32) {
    if (mine >= key) each_element<T, NT>(sl, thr, take);
    G::sync();
  } else {
    const Batches<T, NT> bt(sl);
    const int slots = bt.slots();
    for (int i = t; i < (slots + 1) * (NT / Elem<T>::EV); i += NT)
      pick<T>(*reinterpret_cast<const uint4*>(&sh.slot[0][i * Elem<T>::EV]), i * Elem<T>::EV, thr, [&](float, int j) {
        const int at = atomicAdd(&sh.nhit, 1);
        if (at < kMaxHits) sh.hit[at] = (uint16_t)j;
      });
    __syncthreads();
    const int hits = sh.nhit, log_per = kLogBatch + bt.shift;
    if (hits <= kMaxHits) {
      for (int i = t; i < hits << log_per; i += NT) {
        const int h = sh.hit[i >> log_per], in = i & ((1 << log_per) - 1), who = h % NT, slot = h / NT, mb = bt.of(who);
        const int batch = slot == slots ? mb : (slot << bt.shift) + in / kBatch;
        if (slot == slots ? in >= kBatch : batch >= mb) continue;
        if (slot == slots && in == kBatch - 1) {          // the rest has at most kBatch - 1 vectors, and the edge
          const int j = sl.edge(who);
          if (j >= 0) {
            const float x = Elem<T>::to_float(sl.row[j]);
            if (x >= thr) take(x, j);
          }
          continue;
        }
        const int v = sl.v0 + who + NT * (kBatch * batch + in % kBatch);
        // the last batches are still in the ring
        if (v < sl.v1)
          take_vector<T, NT>(sh, slot != slots && batch + kRing >= mb ? ring[((batch % kRing) * kBatch + in % kBatch) * NT + who] : load16(sl.vec(v)),
                             sl.head + v * Elem<T>::EV, thr);
      }
    } else if (t == 0) {
      sh.n = kCap + 1;
    }
    __syncthreads();
  }
  int n = sh.n;
  if (n > kCap) {
    G::sync();
    if (t == 0) sh.n = 0;
    G::sync();
    if (mine > key)
      each_element<T, NT>(sl, thr, [&](float x, int j) {
        if (x > thr) take(x, j);
      });
    G::sync();
    n = sh.n;
    if (n > kCap - kMaxTopK) {
      unsigned long long last = ~0ull;
      int found = 0;
      for (; found < k; ++found) {
        unsigned long long best = 0ull;
        each_element<T, NT>(sl, -FLT_MAX, [&](float x, int j) {
          const unsigned long long c = cand_key(order_bits(x), j);
          if (c < last && c > best) best = c;
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
        const bool same = j < sl.e1 && Elem<T>::to_float(sl.row[j]) == thr;
        const uint32_t b = __ballot_sync(0xffffffffu, same);
        if (lane == 0) sh.wcount[w] = __popc(b);
        G::sync();
        int before = __popc(b & ((1u << lane) - 1u)), all = 0;
        for (int i = 0; i < G::kWarps; ++i) {
          if (i < w) before += sh.wcount[i];
          all += sh.wcount[i];
        }
        if (same && n + before < k) sh.cand[n + before] = cand_key(key, j);
        n = min(n + all, k);
        G::sync();
      }
    }
  }
  rank_candidates<T, NT>(sh, n, k);
}

// ---- the teacher's side of one row ------------------------------------------------------------------------------------
// One warp works on a row: lane holds the entries lane + 32 e.  The loads are steps of their own, so that a warp that goes
// over rows can have the next row's under way.
constexpr int kPerLane = kMaxTeacher / 32;

struct Entries {                 // column (or -1 where there is no entry) and logit
  int col[kPerLane];
  float t[kPerLane];
  __device__ __forceinline__ void load(const int32_t* idx, const float* val, int K) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int e = 0; e < kPerLane; ++e) {
      const int i = lane + 32 * e;
      col[e] = -1;
      t[e] = -INFINITY;
      if (32 * e < K && i < K) {
        col[e] = idx[i];
        t[e] = val[i];
      }
    }
  }
  // the student's logits at the columns, where need(column)
  template <class T, class F>
  __device__ __forceinline__ void student(const T* row, int K, int V, float (&x)[kPerLane], F need) const {
#pragma unroll
    for (int e = 0; e < kPerLane; ++e) {
      x[e] = 0.f;
      if (32 * e < K && col[e] >= 0 && col[e] < V && need(col[e])) x[e] = Elem<T>::to_float(row[col[e]]);
    }
  }
};

// A row's entries in shared memory: q, log q (natural) and the student's logit of all of them, for the loss, and a list of
// those whose column lies in the block's slice, for the gradient.
struct Teacher {
  float q[kMaxTeacher], logq[kMaxTeacher], x[kMaxTeacher];
  alignas(16) int col[kMaxTeacher];
  alignas(16) float colq[kMaxTeacher];
  float colx[kMaxTeacher], mass[kMaxTeacher];
  int n;               // of the list
  int any, bad;        // a live entry; a column outside the vocabulary

  // e0, e1: the slice's columns
  __device__ __forceinline__ void set(const Entries& in, const float (&xs)[kPerLane], int K, int V, float inv_tau, int e0, int e1) {
    const int lane = threadIdx.x & 31;
    float t[kPerLane];
    float mx = -INFINITY;
    bool have = false, out = false;
#pragma unroll
    for (int e = 0; e < kPerLane; ++e) {
      t[e] = -INFINITY;
      if (32 * e >= K) continue;
      out |= in.col[e] >= V;
      const bool there = in.col[e] >= 0 && in.col[e] < V;
      have |= there;
      t[e] = there ? in.t[e] : -INFINITY;
      mx = max_nan(mx, t[e]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    out = __any_sync(0xffffffffu, out);
    // a teacher whose every entry is masked asks for nothing
    have = (__any_sync(0xffffffffu, have) && mx != -INFINITY) || out;
    float sum = 0.f, e_[kPerLane];
#pragma unroll
    for (int e = 0; e < kPerLane; ++e) {
      e_[e] = 0.f;
      if (32 * e >= K) continue;
      t[e] = t[e] == -INFINITY ? -INFINITY : (t[e] - mx) * inv_tau;
      e_[e] = ex2(t[e] * kLog2e);
      sum += e_[e];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float ls = logf(sum), inv = 1.f / sum;
    int listed = 0;
#pragma unroll
    for (int e = 0; e < kPerLane; ++e) {
      if (32 * e >= K) continue;
      const int i = lane + 32 * e;
      const bool there = in.col[e] >= 0 && in.col[e] < V, mine = there && in.col[e] >= e0 && in.col[e] < e1;
      const float p = there && have ? e_[e] * inv : 0.f;
      q[i] = p;
      logq[i] = t[e] - ls;
      x[i] = xs[e];
      const uint32_t who = __ballot_sync(0xffffffffu, mine);
      if (mine) {
        const int at = listed + __popc(who & ((1u << lane) - 1u));
        col[at] = in.col[e];
        colq[at] = p;
        colx[at] = xs[e];
      }
      listed += __popc(who);
    }
    if (lane < 3 && listed + lane < kMaxTeacher) {       // the list is read four at a time
      col[listed + lane] = -1;
      colq[listed + lane] = 0.f;
    }
    if (lane == 0) {
      n = listed;
      any = have;
      bad = out;
    }
    __syncwarp();
    // mass: all of the teacher's probability in a listed entry's column, which may come more than once
    for (int i = lane; i < listed; i += 32) {
      const int j = col[i];
      float m = 0.f;
      for (int o = 0; o < listed; o += 4) {
        const int4 co = *reinterpret_cast<const int4*>(&col[o]);
        const float4 qo = *reinterpret_cast<const float4*>(&colq[o]);
        m += (co.x == j ? qo.x : 0.f) + (co.y == j ? qo.y : 0.f);
        m += (co.z == j ? qo.z : 0.f) + (co.w == j ? qo.w : 0.f);
      }
      mass[i] = m;
    }
    __syncwarp();
  }
  template <class T>
  __device__ __forceinline__ void read(const int32_t* idx, const float* val, const T* row, int K, int V, float inv_tau) {
    Entries in;
    float xs[kPerLane];
    in.load(idx, val, K);
    in.student(row, K, V, xs, [](int) { return true; });
    set(in, xs, K, V, inv_tau, 0, V);
  }
  // loss of the row / tau^2, by the warp that read it: sum_i q_i (log q_i - log p_i)
  __device__ __forceinline__ float divergence(const RowSum& r, int K) const {
    if (!any) return 0.f;
    if (bad) return __int_as_float(0x7fc00000);
    if (r.empty) return INFINITY;
    float kl = 0.f;
    for (int i = threadIdx.x & 31; i < K; i += 32)
      if (!(q[i] == 0.f)) kl += q[i] * (logq[i] - r.logp(x[i]));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) kl += __shfl_xor_sync(0xffffffffu, kl, o);
    return kl;
  }
};

// ---- forward ----------------------------------------------------------------------------------------------------------
struct ForwardArgs {
  const void* x;
  long long ld, T;
  int V, ranks, per, k, K;
  long long ld_teacher;
  float c, inv_tau, tau, unit;
  const int32_t* tokens;
  float *logprob, *entropy, *lse;
  int32_t* top_tokens;
  float* top_logprobs;
  const int32_t* teacher_tokens;
  const float* teacher_logits;
  float* loss;
};

// One pass over the logits: DISTILL = false for token_logprobs, true for the loss of distill without its gradient.
//
// Per element of 16 bits: half a comparison for the maximum, half for the bound, one unpacking, one ex2 and one and a half
// fused operations, 7.3 instructions with everything around them; memory and the special-function unit (8 cycles a warp's
// ex2) are both near their limits, so what counts is that enough is under way: eight blocks of 128 threads or four of 256 an
// SM, each thread two batches of 64 bytes through shared memory.  4096 rows of 131072 bf16: 162 us, 6.6 TB/s (1.01 of the
// measured copy rate); with 20 alternatives 181 us (0.91): the selection after a row leaves its block without loads for about
// 3 us.  (With blocks of 256, three batches and three blocks: 177 and 209 us; two vectors a batch, five blocks: 191 and 229 us;
// vectors straight to registers: 241 us.  Blocks that stay and have the next row's first batch under way during the selection:
// 204 and 225 us, since rows are then dealt out beforehand and the loop needs more instructions.)
//
// A row's selection and joins cost its block about 5 us whatever its length, and smaller blocks leave more of the others
// streaming meanwhile: where every SM has eight rows, blocks of 128 (us by 256 and by 128 threads: 4096 x 131072 bf16 168 and
// 162, with 20 alternatives 190 and 181; 6000 x 20000 bf16 65 and 53, 107 and 77; 2368 x 32000 fp32 58 and 55, 73 and 64; a
// little more than one round of them loses, 1400 x 131072 bf16 66 and 72).  Rows of one warp exist for short rows.
template <class T, int NT, bool DISTILL>
__global__ void __launch_bounds__(NT == 32 ? kWarpBlock : NT, NT == 32 ? 8 : kForwardBlocks * kBlock / NT) rows_forward_kernel(const ForwardArgs A) {
  using G = Group<NT>;
  __shared__ TopShared<T, NT> top_sh[DISTILL ? 1 : G::kRowsPerBlock];
  __shared__ Teacher teacher_sh[DISTILL ? G::kRowsPerBlock : 1];
  __shared__ Stat wstat[G::kRowsPerBlock][G::kWarps];
  const int t = G::tid(), lane = threadIdx.x & 31, w = NT == 32 ? 0 : (int)(threadIdx.x >> 5);
  const int ranks = NT == 32 ? 1 : A.ranks;
  const int rank = NT == 32 ? 0 : (int)(blockIdx.x % (unsigned)ranks);
  const long long row = NT == 32 ? (long long)blockIdx.x * G::kRowsPerBlock + G::slot() : (long long)(blockIdx.x / (unsigned)ranks);
  if (NT == 32 && row >= A.T) return;
  TopShared<T, NT>& sh = top_sh[DISTILL ? 0 : G::slot()];
  Teacher& te = teacher_sh[DISTILL ? G::slot() : 0];
  const T* xr = reinterpret_cast<const T*>(A.x) + row * A.ld;
  const int k = DISTILL ? 0 : A.k;

  const Slice<T> sl(xr, A.V, rank, ranks, A.per);
  const float c = A.c;
  int token = -1;
  if (!DISTILL && A.tokens) token = A.tokens[row];
  // The first batches are on their way before anything is known about the row.  A block's threads keep kRing batches
  // each in flight through shared memory (a warp's row is short: one batch ahead in registers).
  extern __shared__ uint4 ring[];        // [kRing][kBatch][NT], a thread's own column
  const Batches<T, NT> bt(sl);
  const int batches = bt.of(t);
  int v = sl.v0 + t;
  auto fetch = [&](int b) {              // batch b into its place of the ring
    if (b < batches) {
#pragma unroll
      for (int i = 0; i < kBatch; ++i) copy16(&ring[((b % kRing) * kBatch + i) * NT + t], sl.vec(v + (b * kBatch + i) * NT));
    }
    copy_commit();
  };
  uint4 x[kBatch];
  if constexpr (NT == 32) {
    if (batches > 0) {
#pragma unroll
      for (int i = 0; i < kBatch; ++i) x[i] = load16(sl.vec(v + i * NT));
    }
  } else {
#pragma unroll
    for (int b = 0; b < kRing - 1; ++b) fetch(b);
  }
  const bool bad_token = token >= A.V, live = DISTILL || !A.tokens || token >= 0;
  if (DISTILL && w == 0 && rank == 0)
    te.read(A.teacher_tokens + row * A.ld_teacher, A.teacher_logits + row * A.ld_teacher, xr, A.K, A.V, A.inv_tau);
  Running<T, !DISTILL> run(c);
  float top = -INFINITY, rest = -INFINITY;
  if (live) {
    float high = -INFINITY;              // of the slot
    for (int b = 0; b < batches; ++b) {
      uint4 y[NT == 32 ? kBatch : 1];
      if constexpr (NT == 32) {
        if (b + 1 < batches) {
#pragma unroll
          for (int i = 0; i < kBatch; ++i) y[i] = load16(sl.vec(v + ((b + 1) * kBatch + i) * NT));
        }
      } else {
        fetch(b + kRing - 1);
        copy_wait<kRing - 1>();
#pragma unroll
        for (int i = 0; i < kBatch; ++i) x[i] = ring[((b % kRing) * kBatch + i) * NT + t];
      }
      const float mx = Elem<T>::largest(x);
      run.follow(mx);
      run.add(x);
      if (NT > 32 && k > 0) {
        high = max_nan(high, mx);
        sh.slot[b >> bt.shift][t] = Elem<T>::from_float(high);
        if (((b + 1) & ((1 << bt.shift) - 1)) == 0) high = -INFINITY;
      }
      top = max_nan(top, mx);
      if constexpr (NT == 32) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) x[i] = y[i];
      }
    }
    v += batches * kBatch * NT;
    for (; v < sl.v1; v += NT) {
      const uint4 y[1] = {load16(sl.vec(v))};
      const float mx = Elem<T>::largest(y);
      rest = max_nan(rest, mx);
      run.follow(mx);
      run.add(y);
    }
    const int j = sl.edge(t);
    if (j >= 0) {
      const float e = Elem<T>::to_float(xr[j]);
      rest = max_nan(rest, e);
      run.follow(e);
      run.one(e);
    }
    top = max_nan(top, rest);
    if (NT > 32 && k > 0) {
      const int slots = bt.slots();
      for (int i = (batches + (1 << bt.shift) - 1) >> bt.shift; i < slots; ++i) sh.slot[i][t] = Elem<T>::from_float(-INFINITY);
      sh.slot[slots][t] = Elem<T>::from_float(rest);
    }
  }
  if (NT > 32) copy_wait<0>();           // of a row that was not looked at
  Stat a = warp_join<32, !DISTILL>(run.get(), c);
  if (NT > 32) {
    if (lane == 0) wstat[0][w] = a;
    __syncthreads();
    a = warp_join<G::kWarps, !DISTILL>(wstat[0][lane % G::kWarps], c);
  }
  const bool alternatives = !DISTILL && k > 0 && live;
  if (alternatives) top_of_slice<T, NT>(sh, sl, ring, top, rest, k);
  if (ranks > 1) {       // the first block of the cluster takes the others' results
    cg::cluster_group cluster = cg::this_cluster();
    __syncthreads();
    if (t == 0) wstat[0][0] = a;
    cluster.sync();
    if (rank == 0) {
      for (int r = 1; r < ranks; ++r) a = join(a, *cluster.map_shared_rank(&wstat[0][0], r), c);
      if (alternatives) {
        if (t < ranks * kMaxTopK && t % kMaxTopK < k)
          sh.cand[t / kMaxTopK * k + t % kMaxTopK] = cluster.map_shared_rank(sh.best, t / kMaxTopK)[t % kMaxTopK];
        __syncthreads();
        for (int i = t; i < k; i += NT) sh.best[i] = 0ull;
        __syncthreads();
      }
    }
    cluster.sync();
    if (rank != 0) return;
    if (alternatives) rank_candidates<T, NT>(sh, ranks * k, k);
  }
  const RowSum r(a, c, A.unit, A.inv_tau);
  if (DISTILL) {
    if (w == 0) {
      const float kl = te.divergence(r, A.K);
      if (lane == 0) {
        A.loss[row] = A.tau * A.tau * kl;
        A.lse[row] = te.any ? r.lse : 0.f;
      }
    }
    return;
  }
  if (t == 0) {
    if (A.logprob) A.logprob[row] = !live ? 0.f : bad_token ? __int_as_float(0x7fc00000) : r.logp(Elem<T>::to_float(xr[token]));
    if (A.entropy) A.entropy[row] = live ? r.entropy : 0.f;
    if (A.lse) A.lse[row] = live ? r.lse : 0.f;
  }
  for (int i = t; i < k; i += NT) {
    const bool nan = live && r.log2s != r.log2s;
    const unsigned long long key = live && !nan ? sh.best[i] : 0ull;
    A.top_tokens[row * k + i] = key ? (int32_t)(0xffffffffu - (uint32_t)key) : -1;
    A.top_logprobs[row * k + i] = nan ? r.log2s : key ? r.logp(from_order_bits((uint32_t)(key >> 32))) : -INFINITY;
  }
}

// ---- gradients --------------------------------------------------------------------------------------------------------
struct GradArgs {
  const void* x;
  void* dx;
  long long ld, ld_d, T;
  int V, ranks, per, K;
  long long ld_teacher;
  float c, inv_tau, inv_tau_lo, tau, unit;
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

// Gradients whose statistics are known: bound by memory, each logit read and each gradient written once (4096 rows of 100003
// bf16, starting at odd addresses: 254 us, 6.4 TB/s, 0.98 of the measured copy rate; the teacher's form, 2048 rows of 131072:
// 167 us, 0.98).  16 vectors a thread and five blocks an SM: with four vectors what a block does once made two thirds of
// its instructions (285 us).  The teacher's entries have a warp of their own, beside which the others load and store; in
// the warps' path they cost 516 instead of 333 us at 8192 rows of 65536.
//
// A thread keeps its R vectors of the row in registers, so the gradient in the same call as the loss (rows of a warp here,
// longer ones in rows_step_kernel) reads the logits once.  With the statistics handed over (kLogprobsGrad, kDistillGrad)
// `ranks` is any number of independent pieces of the row.
//
// dx_j = p_j (ca + cb log2 p_j), then the entries that have a term of their own.  16-bit logits take log2 p as one fused
// x c - kappa, two elements an instruction.  fp32 logits take (x / tau - lse) first and 1 / tau as two fp32 terms: the
// rounding of either would shift every log p by 2^-24 of s, which an fp32 gradient shows.
template <int NT, int MODE>
constexpr int kGradientThreads = MODE == kDistillGrad ? NT + 32 : NT;
template <int ID, int THREADS>
__device__ __forceinline__ void bar_sync() { asm volatile("bar.sync %0, %1;" ::"n"(ID), "n"(THREADS) : "memory"); }
template <int ID, int THREADS>
__device__ __forceinline__ void bar_arrive() { asm volatile("bar.arrive %0, %1;" ::"n"(ID), "n"(THREADS) : "memory"); }

template <class T, int NT, int R, int MODE>
__global__ void __launch_bounds__(NT == 32 ? kWarpBlock : kGradientThreads<NT, MODE>, NT == 32 ? 4 : 5) rows_gradient_kernel(const GradArgs A) {
  using G = Group<NT>;
  constexpr int EV = Elem<T>::EV;
  constexpr bool kTeacher = MODE != kLogprobsGrad, kStep = MODE == kDistillStep, kNarrow = sizeof(T) == 2;
  constexpr bool kOwnWarp = MODE == kDistillGrad && NT > 32;     // the teacher's entries have a warp of their own
  static_assert(!kStep || NT == 32, "longer rows of the step: rows_step_kernel");
  __shared__ Teacher teacher_sh[kTeacher ? G::kRowsPerBlock : 1];
  const int t = G::tid(), lane = threadIdx.x & 31, w = NT == 32 ? 0 : (int)(threadIdx.x >> 5);
  const int ranks = NT == 32 ? 1 : A.ranks;
  const int rank = NT == 32 ? 0 : (int)(blockIdx.x % (unsigned)ranks);
  const long long row = NT == 32 ? (long long)blockIdx.x * G::kRowsPerBlock + G::slot() : (long long)(blockIdx.x / (unsigned)ranks);
  if (NT == 32 && row >= A.T) return;
  Teacher& te = teacher_sh[kTeacher ? G::slot() : 0];
  const T* xr = reinterpret_cast<const T*>(A.x) + row * A.ld;
  T* dr = reinterpret_cast<T*>(A.dx) + row * A.ld_d;
  const Slice<T> sl(xr, A.V, rank, ranks, A.per);
  const bool aligned = ((((uintptr_t)xr) ^ ((uintptr_t)dr)) & 15u) == 0;   // vectors of x are vectors of dx
  const int edge = sl.edge(t);
  const float c = A.c;

  // the row's vectors are on their way before anything else of it is looked at; a row that asks for nothing is read for
  // nothing in the step, and not at all where there is a token to tell
  int token = -1;
  bool zero = false;
  float lse = 0.f;
  if (!kTeacher) {
    token = A.tokens[row];
    zero = token < 0;
  }
  if (!kStep) {
    lse = A.lse_in[row];
    zero = zero || (lse <= kEmptyLse && token < A.V);       // nothing left by the masks
  }
  constexpr int kThreads = kGradientThreads<NT, MODE>;
  const bool in_place = A.x == A.dx;
  if (kOwnWarp && w == G::kWarps) {
    // this piece's columns of the teacher: prepared while the other warps work, written over what they store
    const int32_t* idx = A.teacher_tokens + row * A.ld_teacher;
    Entries in;
    float xs[kPerLane];
    in.load(idx, A.teacher_logits + row * A.ld_teacher, A.K);
    in.student(xr, A.K, A.V, xs, [&](int j) { return j >= sl.e0 && j < sl.e1; });
    te.set(in, xs, A.K, A.V, A.inv_tau, sl.e0, sl.e1);
    if (in_place) bar_sync<1, kThreads>();          // the student's logits are read before they are written over
    bar_sync<2, kThreads>();
    const float ca = A.d_loss[row] * A.tau;
    if (zero || !te.any || te.bad) return;
    for (int i = lane; i < te.n; i += 32) {
      const float x = te.colx[i];
      const float lp = kNarrow ? fmaf(x, c, -lse * kLog2e) : fmaf(x, A.inv_tau, fmaf(x == -INFINITY ? 0.f : x, A.inv_tau_lo, -lse)) * kLog2e;
      dr[te.col[i]] = Elem<T>::from_float(ca * (ex2(lp) - te.mass[i]));
    }
    return;
  }
  uint4 v[R];
  float xe = -INFINITY;
  const int per_turn = R * NT;
  if (kTeacher || !zero) {                 // a masked row of which the teacher asks for a bad column becomes NaN
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int at = sl.v0 + t + i * NT;
      if (at < sl.v1) v[i] = load16(sl.vec(at));
      else v[i] = make_uint4(Elem<T>::kNegInf, Elem<T>::kNegInf, Elem<T>::kNegInf, Elem<T>::kNegInf);
    }
    if (edge >= 0) xe = Elem<T>::to_float(xr[edge]);
  }
  bool bad = false;
  if constexpr (kOwnWarp) {
    Entries in;                       // is there anything to learn from: every warp looks for itself
    in.load(A.teacher_tokens + row * A.ld_teacher, A.teacher_logits + row * A.ld_teacher, A.K);
    bool any = false;
#pragma unroll
    for (int e = 0; e < kPerLane; ++e) {
      bad = bad || in.col[e] >= A.V;
      any = any || (in.col[e] >= 0 && !(in.t[e] == -INFINITY));
    }
    bad = __any_sync(0xffffffffu, bad);
    zero = !bad && (zero || !__any_sync(0xffffffffu, any));
    if (in_place) bar_sync<1, kThreads>();
  }
  if (kTeacher && !kOwnWarp && w == 0)
    te.read(A.teacher_tokens + row * A.ld_teacher, A.teacher_logits + row * A.ld_teacher, xr, A.K, A.V, A.inv_tau);

  float ref = 0.f, log2s = 0.f;
  if (kStep) {
    Running<T, false> run(c);
    run.set_ref(max_nan(max_nan(Elem<T>::largest(v), xe), kUnset));
    run.add(v);
    run.one(xe);
    const Stat a = warp_join<32, false>(run.get(), c);
    const RowSum r(a, c, A.unit, A.inv_tau);
    ref = r.ref;
    log2s = r.log2s;
    zero = r.masked;
    if (rank == 0 && w == 0) {
      const float kl = te.divergence(r, A.K);
      if (lane == 0) {
        A.loss[row] = A.tau * A.tau * kl;
        A.lse_out[row] = te.any ? r.lse : 0.f;
      }
    }
  }

  float ca, cb = 0.f, cy = 0.f;
  if (kTeacher) {
    if (!kOwnWarp) {
      G::sync();
      bad = te.bad != 0;
      zero = !bad && (zero || !te.any);
    }
    ca = A.d_loss[row] * A.tau;
  } else {
    const float g = A.d_logprob ? A.d_logprob[row] : 0.f, h = A.d_entropy ? A.d_entropy[row] : 0.f;
    cb = -h * A.inv_tau;
    ca = -(g + (A.d_entropy ? h * A.entropy[row] : 0.f)) * A.inv_tau;
    cy = g * A.inv_tau;
    bad = token >= A.V;
  }
  if (bad) ca = __int_as_float(0x7fc00000);
  // log2 p = x c - kappa, for 16-bit logits whose reference is no mask
  const float kappa = kStep ? ref * c + log2s : lse * kLog2e;
  const bool packed = kNarrow && (!kStep || fabsf(kappa) < kOneNumber);
  const f32x2 c2 = pair_of(c, c), k2 = pair_of(-kappa, -kappa), ca2 = pair_of(ca, ca), cb2 = pair_of(cb * kLn2, cb * kLn2);
  // with a term in log p, -inf is raised to a bound where p is 0 and log p finite; without such a bound: one by one
  const uint32_t lo = MODE == kLogprobsGrad && kNarrow ? Elem<T>::bound((kappa - 200.f) / c) : 0u;
  auto prob = [&](float x, float& lp) -> float {       // p, and log p (natural)
    if (kStep) {
      lp = (scaled(x, ref, c) - log2s) * A.unit;
      return ex2(scaled(x, ref, c) - log2s);
    }
    lp = kNarrow ? fmaf(x, c, -kappa) * kLn2 : fmaf(x, A.inv_tau, fmaf(x == -INFINITY ? 0.f : x, A.inv_tau_lo, -lse));
    return ex2(lp * kLog2e);
  };
  auto grad = [&](float x) -> float {
    float lp;
    const float p = prob(x, lp);
    return MODE == kLogprobsGrad ? p * fmaf(cb, max_nan(lp, -1e4f), ca) : p * ca;
  };
  auto put = [&](const uint4& xv, int at) {
    const int j0 = sl.head + at * EV;
    if (zero) {
      const float y[EV] = {};
      store_vec<T>(dr + j0, y, aligned);
      return;
    }
    if constexpr (kNarrow) {
      if (packed && (MODE != kLogprobsGrad || lo) && aligned) {
        f32x2 p[EV / 2];
        Elem<T>::pairs(MODE == kLogprobsGrad ? at_least<T>(xv, lo) : xv, p);
#pragma unroll
        for (int i = 0; i < EV / 2; ++i) {
          const f32x2 lp = fma2(p[i], c2, k2), e = ex2x2(lp);
          p[i] = mul2(e, MODE == kLogprobsGrad ? fma2(cb2, lp, ca2) : ca2);
        }
        if (MODE == kLogprobsGrad && (unsigned)(token - j0) < (unsigned)EV) {
#pragma unroll
          for (int i = 0; i < EV / 2; ++i)
            p[i] = add2(p[i], pair_of(j0 + 2 * i == token ? cy : 0.f, j0 + 2 * i + 1 == token ? cy : 0.f));
        }
        *reinterpret_cast<uint4*>(dr + j0) = Elem<T>::pack_pairs(p);
        return;
      }
    }
    float x[EV], y[EV];
    Elem<T>::unpack(xv, x);
#pragma unroll
    for (int i = 0; i < EV; ++i) y[i] = grad(x[i]);
    if (MODE == kLogprobsGrad && (unsigned)(token - j0) < (unsigned)EV) {
#pragma unroll
      for (int i = 0; i < EV; ++i)
        if (j0 + i == token) y[i] += cy;
    }
    store_vec<T>(dr + j0, y, aligned);
  };
  for (int b = sl.v0 + t;;) {
#pragma unroll
    for (int i = 0; i < R; ++i)
      if (b + i * NT < sl.v1) put(v[i], b + i * NT);
    b += per_turn;
    if (kStep || b >= sl.v1) break;        // the step's plan makes a slice fit R vectors a thread
    if (!zero) {
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (b + i * NT < sl.v1) v[i] = load16(sl.vec(b + i * NT));
    }
  }
  if (edge >= 0) {
    float y = zero ? 0.f : grad(xe);
    if (!kTeacher && !zero && edge == token) y += cy;
    dr[edge] = Elem<T>::from_float(y);
  }
  if constexpr (kOwnWarp) {
    bar_arrive<2, kThreads>();
  } else if (kTeacher) {
    // the teacher's columns: p_j minus all of the teacher's mass there (the same column may come more than once; every
    // entry then writes the same value), over what the loop above wrote
    G::sync();
    if (zero || bad) return;
    for (int i = t; i < te.n; i += NT) {
      float lp;
      dr[te.col[i]] = Elem<T>::from_float(ca * (prob(te.colx[i], lp) - te.mass[i]));
    }
  }
}

// The loss and its gradient in one reading, for rows longer than a warp's.  A block goes over rows (each block of a cluster
// over its slice of them): a slice lies in shared memory, is read twice from there, for the statistics and for the gradient,
// and the next row's is on its way into each vector's place as soon as the gradient has used it.  One more warp
// prepares the next row's teacher entries while the gradient is stored, and then writes the teacher's columns over it: on
// the other warps' path that had cost as much as the whole rest.
//
// 8192 rows of 65536 bf16, 64 entries: 390 us, 5.5 TB/s (0.84 of the measured copy rate; two clusters' halves of 64 KB, three
// blocks an SM).  Two ex2 an element keep the special-function unit busy for 250 us of it, 14 instructions an element the
// schedulers for 260 us, and the two phases of a block do not overlap with themselves: other blocks have to fill the
// gaps.  Measured and dropped: slices held in registers (580 us: too few warps), 128 threads a block (510 us), part of
// the exponentials as a polynomial (no gain: the schedulers are as busy), three buffers and one block of 512 threads an SM with
// the cluster's join under the next row's statistics (592 us).
template <class T, int NT, int R>
__global__ void __launch_bounds__(NT + 32, NT > 128 ? 3 : R > 8 ? 4 : 6) rows_step_kernel(const GradArgs A) {
  constexpr int EV = Elem<T>::EV, kWarps = NT / 32, kThreads = NT + 32;
  constexpr bool kNarrow = sizeof(T) == 2;
  extern __shared__ uint4 buffer[];                // [R][NT], a thread's own column
  __shared__ Stat wstat[2][kWarps];
  __shared__ Stat cstat[2][kMaxCluster];
  __shared__ Teacher teacher[2];
  const int t = threadIdx.x, lane = t & 31, w = t >> 5, ranks = A.ranks;
  // a block stays with one rank and goes over rows
  const int rank = (int)(blockIdx.x % (unsigned)ranks);
  const int rows = (int)A.T, step = (int)(gridDim.x / (unsigned)ranks), first = (int)(blockIdx.x / (unsigned)ranks);
  const float c = A.c;
  auto slice_of = [&](int row) { return Slice<T>(reinterpret_cast<const T*>(A.x) + (long long)row * A.ld, A.V, rank, ranks, A.per); };
  // the statistics of a row, the same in every thread of the cluster
  auto row_sum = [&](int b) {
    Stat a = warp_join<kWarps, false>(wstat[b][lane % kWarps], c);
    if (ranks > 1) {
      cg::cluster_group cluster = cg::this_cluster();
      if (t < ranks) *cluster.map_shared_rank(&cstat[b][rank], t) = a;
      __syncwarp();
      // only the first warp has written to the others, and only the teacher's has read what they will write; the other warps'
      // readings of this buffer two rows ago have long been used
      if (w == 0 || w == kWarps) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
      else asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
      asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
      Stat o{kUnset, 0.f, 0.f};
      if (lane % kMaxCluster < ranks) o = cstat[b][lane % kMaxCluster];
      a = warp_join<kMaxCluster, false>(o, c);
    }
    return RowSum(a, c, A.unit, A.inv_tau);
  };
  auto prob = [&](float x, float ref, float log2s) -> float {
    return ex2(scaled(x, ref, c) - log2s);
  };
  // every block of the cluster runs before its memory is written
  if (ranks > 1) cg::this_cluster().sync();

  if (w == kWarps) {
    auto load = [&](int row, Entries& in) {
      if (row < rows) in.load(A.teacher_tokens + row * A.ld_teacher, A.teacher_logits + row * A.ld_teacher, A.K);
    };
    // the student's logits: the first rank needs all of them for the loss, every rank its own slice's for the gradient
    auto look = [&](int row, const Entries& in, float (&xs)[kPerLane]) {
      if (row >= rows) return;
      const Slice<T> sl = slice_of(row);
      in.student(sl.row, A.K, A.V, xs, [&](int j) { return rank == 0 || (j >= sl.e0 && j < sl.e1); });
    };
    auto prepare = [&](int row, const Entries& in, const float (&xs)[kPerLane], int b) {
      if (row >= rows) return;
      const Slice<T> sl = slice_of(row);
      teacher[b].set(in, xs, A.K, A.V, A.inv_tau, sl.e0, sl.e1);
    };
    Entries now, next;
    float xs[kPerLane], next_g = first < rows ? A.d_loss[first] : 0.f;
    load(first, now);
    load(first + step, next);
    look(first, now, xs);
    prepare(first, now, xs, 0);
    now = next;
    look(first + step, now, xs);
    load(first + 2 * step, next);
    int b = 0;
    for (int row = first; row < rows; row += step, b ^= 1) {
      const Teacher& te = teacher[b];
      const float ca = next_g * A.tau;
      if (row + step < rows) next_g = A.d_loss[row + step];
      bar_sync<1, kThreads>();
      const RowSum r = row_sum(b);
      if (rank == 0) {
        const float kl = te.divergence(r, A.K);
        if (lane == 0) {
          A.loss[row] = A.tau * A.tau * kl;
          A.lse_out[row] = te.any ? r.lse : 0.f;
        }
      }
      // the next row's list is made while the other warps store this row's gradient; its loads are a turn old
      prepare(row + step, now, xs, b ^ 1);
      now = next;
      look(row + 2 * step, now, xs);
      load(row + 3 * step, next);
      T* dr = reinterpret_cast<T*>(A.dx) + (long long)row * A.ld_d;
      bar_sync<2, kThreads>();
      if (te.any && !te.bad && !r.masked)
        for (int i = lane; i < te.n; i += 32)
          dr[te.col[i]] = Elem<T>::from_float(ca * (prob(te.colx[i], r.ref, r.log2s) - te.mass[i]));
      __syncwarp();
    }
    return;
  }

  // What a thread knows of a row before its turn: where its vectors lie (they are on their way to its column of the
  // buffer), the edge element and the row's scalars.
  struct Turn {
    const T* vec;          // its first vector
    int mine, edge;        // vector i is this thread's if i NT < mine; column of the edge element or -1
    float xe, g;
  } next;
  auto plan = [&](int row) {
    next.mine = 0;
    if (row >= rows) return;
    const Slice<T> sl = slice_of(row);
    next.vec = sl.vec(sl.v0 + t);
    next.mine = sl.v1 - sl.v0 - t;
    next.edge = sl.edge(t);
    next.xe = next.edge >= 0 ? Elem<T>::to_float(sl.row[next.edge]) : -INFINITY;
    next.g = A.d_loss[row];
  };
  auto fetch = [&](int i) {                        // the next row's vector i into the buffer
    if (i * NT < next.mine) copy16(&buffer[i * NT + t], next.vec + i * NT * EV);
  };
  constexpr int B = R < kBatch ? R : kBatch;
  plan(first);
#pragma unroll
  for (int i = 0; i < R; ++i) fetch(i);
  copy_commit();
  int b = 0;
  for (int row = first; row < rows; row += step, b ^= 1) {
    const Turn now = next;
    const long long row_at = (long long)row * A.ld, drow_at = (long long)row * A.ld_d;
    T* dst = reinterpret_cast<T*>(A.dx) + drow_at + (now.vec - (reinterpret_cast<const T*>(A.x) + row_at));
    const bool aligned = (((uintptr_t)dst) & 15u) == 0;          // vectors of x are vectors of dx
    float ca = now.g * A.tau;
    copy_wait<0>();
    {
      Running<T, false> run(c);
      run.follow(now.xe);
      run.one(now.xe);
#pragma unroll
      for (int i0 = 0; i0 < R; i0 += B) {
        if (i0 * NT >= now.mine) break;
        uint4 v[B];
        if ((i0 + B - 1) * NT < now.mine) {
#pragma unroll
          for (int i = 0; i < B; ++i) v[i] = buffer[(i0 + i) * NT + t];
        } else {
#pragma unroll
          for (int i = 0; i < B; ++i) {
            v[i] = make_uint4(Elem<T>::kNegInf, Elem<T>::kNegInf, Elem<T>::kNegInf, Elem<T>::kNegInf);
            if ((i0 + i) * NT < now.mine) v[i] = buffer[(i0 + i) * NT + t];
          }
        }
        run.follow(Elem<T>::largest(v));
        run.add(v);
      }
      const Stat a = warp_join<32, false>(run.get(), c);
      if (lane == 0) wstat[b][w] = a;
    }
    bar_sync<1, kThreads>();
    plan(row + step);
    if (teacher[b].bad) ca = __int_as_float(0x7fc00000);
    const RowSum r = row_sum(b);
    const float ref = r.ref, log2s = r.log2s;
    const bool zero = !teacher[b].bad && (!teacher[b].any || r.masked);
    if (aligned && !zero && fabsf(ref * c) < (kNarrow ? kOneNumber : kNear)) {
      // two elements an instruction; a 16-bit gradient bears ref c + log2 s as one rounded number, an fp32 one does not
      const float kappa = ref * c + (kNarrow ? log2s : 0.f);
      const f32x2 c2 = pair_of(c, c), k2 = pair_of(-kappa, -kappa), ca2 = pair_of(ca, ca), l2 = pair_of(-log2s, -log2s);
#pragma unroll
      for (int i = 0; i < R; ++i) {
        if (i * NT < now.mine) {
          f32x2 p[EV / 2];
          Elem<T>::pairs(buffer[i * NT + t], p);
#pragma unroll
          for (int e = 0; e < EV / 2; ++e) {
            p[e] = fma2(p[e], c2, k2);
            if (!kNarrow) p[e] = add2(p[e], l2);
            p[e] = mul2(ex2x2(p[e]), ca2);
          }
          *reinterpret_cast<uint4*>(dst + i * NT * EV) = Elem<T>::pack_pairs(p);
        }
        fetch(i);
      }
    } else {
#pragma unroll 1
      for (int i = 0; i < R; ++i) {
        if (i * NT < now.mine) {
          float x[EV];
          Elem<T>::unpack(buffer[i * NT + t], x);
#pragma unroll
          for (int e = 0; e < EV; ++e) x[e] = zero ? 0.f : ca * prob(x[e], ref, log2s);
          store_vec<T>(dst + i * NT * EV, x, aligned);
        }
        fetch(i);
      }
    }
    copy_commit();
    if (now.edge >= 0)
      reinterpret_cast<T*>(A.dx)[drow_at + now.edge] = Elem<T>::from_float(zero ? 0.f : ca * prob(now.xe, ref, log2s));
    bar_arrive<2, kThreads>();
  }
  copy_wait<0>();
}

// ---- host -------------------------------------------------------------------------------------------------------------
constexpr int kSMs = 148;

template <class Args>
cudaError_t launch(void (*kernel)(const Args), const Args& A, long long blocks, int threads, size_t smem, int cluster, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)cluster;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, A);
}

// What a kernel with dynamic shared memory needs to know of the device, found once per device: its limit is raised, and the
// blocks of it that run at the same time in clusters of 1, 2, 4 and 8.
struct Resident {
  std::atomic<int> blocks[64][4] = {};
  template <class Args>
  cudaError_t get(void (*kernel)(const Args), int threads, size_t smem, int cluster, int& out) {
    int dev = 0;
    cudaError_t rc = cudaGetDevice(&dev);
    if (rc != cudaSuccess) return rc;
    std::atomic<int>& slot = blocks[dev & 63][cluster == 8 ? 3 : cluster / 2];
    out = dev < 64 ? slot.load(std::memory_order_acquire) : 0;
    if (out > 0) return cudaSuccess;
    rc = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (rc != cudaSuccess) return rc;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(cluster * kSMs));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)cluster;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    int n = 0;
    rc = cudaOccupancyMaxActiveClusters(&n, kernel, &cfg);
    if (rc != cudaSuccess) return rc;
    out = (n < 1 ? 1 : n) * cluster;
    slot.store(out, std::memory_order_release);
    return cudaSuccess;
  }
};

// Rows that one warp takes: short ones, and longer ones when there are enough of them to fill the GPU.
template <class T>
bool warp_rows(long long T_, long long V) {
  const long long nvec = V / Elem<T>::EV;
  return V <= kWarpRow || (nvec <= kWarpVectors && T_ >= 16 * kSMs);
}

// Blocks per row of a forward pass: one where there is a row for every SM (517 rows of 50001 fp32: 23 us, with two blocks a row
// 31 us: the join costs more than the even load gives), else up to eight, down to two vectors a thread (one row of 131072
// bf16: 6.2 us by eight blocks, 11.7 us by one).
int forward_ranks(long long T, long long nvec) {
  int ranks = 1;
  while (ranks < kMaxCluster && T * ranks < kSMs && nvec > (long long)ranks * 2 * kBlock) ranks *= 2;
  return ranks;
}

template <class T, bool DISTILL>
cudaError_t forward(ForwardArgs& A, cudaStream_t st) {
  if (warp_rows<T>(A.T, A.V)) {
    A.ranks = 1;
    A.per = A.V / Elem<T>::EV;
    return launch(rows_forward_kernel<T, 32, DISTILL>, A, (A.T + 3) / 4, kWarpBlock, 0, 1, st);
  }
  const long long nvec = A.V / Elem<T>::EV;
  if (A.T >= 2 * kForwardBlocks * kSMs) {
    A.ranks = 1;
    A.per = (int)nvec;
    return launch(rows_forward_kernel<T, kHalfBlock, DISTILL>, A, A.T, kHalfBlock, (size_t)kRing * kBatch * kHalfBlock * 16, 1, st);
  }
  A.ranks = forward_ranks(A.T, nvec);
  A.per = (int)((nvec + A.ranks - 1) / A.ranks);
  return launch(rows_forward_kernel<T, kBlock, DISTILL>, A, A.T * A.ranks, kBlock, (size_t)kRing * kBatch * kBlock * 16, A.ranks, st);
}

template <class T, int NT, int R>
cudaError_t step_blocks(GradArgs& A, cudaStream_t st) {
  constexpr size_t smem = (size_t)R * NT * 16;
  static Resident resident;
  int blocks = 0;
  const cudaError_t rc = resident.get(rows_step_kernel<T, NT, R>, NT + 32, smem, A.ranks, blocks);
  if (rc != cudaSuccess) return rc;
  const long long at_once = blocks / A.ranks > 0 ? blocks / A.ranks : 1;          // rows
  return launch(rows_step_kernel<T, NT, R>, A, (A.T < at_once ? A.T : at_once) * A.ranks, NT + 32, smem, A.ranks, st);
}

template <class T, int MODE>
cudaError_t gradient(GradArgs& A, cudaStream_t st) {
  const long long nvec = A.V / Elem<T>::EV;
  if (A.V <= kWarpRow || (MODE == kLogprobsGrad && warp_rows<T>(A.T, A.V))) {
    A.ranks = 1;
    A.per = (int)nvec;
    return launch(rows_gradient_kernel<T, 32, kWarpRow / Elem<T>::EV / 32, MODE>, A, (A.T + 3) / 4, kWarpBlock, 0, 1, st);
  }
  if constexpr (MODE != kDistillStep) {
    // pieces of 16 vectors a thread, smaller ones while the rows do not fill the GPU, larger ones where the grid would pass
    // 2^31 blocks
    long long ranks = (nvec + 16 * kBlock - 1) / (16 * kBlock);
    while (A.T * ranks < 4 * kSMs && nvec > ranks * 2 * kBlock) ranks *= 2;
    while (A.T * ranks > 0x7fffffffll) ranks = (ranks + 1) / 2;
    A.ranks = ranks < 1 ? 1 : (int)ranks;
    A.per = (int)((nvec + A.ranks - 1) / A.ranks);
    return launch(rows_gradient_kernel<T, kBlock, 4, MODE>, A, A.T * A.ranks, kGradientThreads<kBlock, MODE>, 0, 1, st);
  } else {
    // a row in one block of 128 threads (up to 16 vectors a thread), or in up to eight of 256; spread wider while the rows
    // do not fill the GPU
    int ranks = 1;
    while (ranks < kMaxCluster && (nvec > (long long)ranks * 16 * kBlock || (A.T * ranks < 3 * kSMs && nvec > (long long)ranks * 2 * kHalfBlock)))
      ranks *= 2;
    A.ranks = ranks;
    A.per = (int)((nvec + ranks - 1) / ranks);
    if (A.per <= 4 * kHalfBlock) return step_blocks<T, kHalfBlock, 4>(A, st);
    if (A.per <= 8 * kHalfBlock) return step_blocks<T, kHalfBlock, 8>(A, st);
    if (A.per <= 16 * kHalfBlock) return step_blocks<T, kHalfBlock, 16>(A, st);
    return step_blocks<T, kBlock, 16>(A, st);
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
  return LAQ_OK;
}

laq_status check_gradient(const Err& e, const void* dx, int64_t ld_d, int64_t V) {
  if (!dx) return fail(e.buf, e.len, LAQ_EINVAL, "null pointer");
  if (ld_d < V) return fail(e.buf, e.len, LAQ_EINVAL, "a row stride must be at least vocab");
  return LAQ_OK;
}

template <class T>
void list_kernels(const void** list, int& n) {
  const void* all[] = {
      (const void*)rows_forward_kernel<T, 32, false>, (const void*)rows_forward_kernel<T, kHalfBlock, false>,
      (const void*)rows_forward_kernel<T, kBlock, false>, (const void*)rows_forward_kernel<T, 32, true>,
      (const void*)rows_forward_kernel<T, kHalfBlock, true>, (const void*)rows_forward_kernel<T, kBlock, true>,
      (const void*)rows_gradient_kernel<T, 32, kWarpRow / Elem<T>::EV / 32, kLogprobsGrad>,
      (const void*)rows_gradient_kernel<T, 32, kWarpRow / Elem<T>::EV / 32, kDistillGrad>,
      (const void*)rows_gradient_kernel<T, 32, kWarpRow / Elem<T>::EV / 32, kDistillStep>,
      (const void*)rows_gradient_kernel<T, kBlock, 4, kLogprobsGrad>, (const void*)rows_gradient_kernel<T, kBlock, 4, kDistillGrad>,
      (const void*)rows_step_kernel<T, kHalfBlock, 4>, (const void*)rows_step_kernel<T, kHalfBlock, 8>,
      (const void*)rows_step_kernel<T, kHalfBlock, 16>, (const void*)rows_step_kernel<T, kBlock, 16>};
  for (const void* k : all) list[n++] = k;
}

laq_status load_kernels(const Err& e) {
  static Loaded loaded;
  static const void* list[48];
  static const int n = [] {
    int count = 0;
    list_kernels<float>(list, count);
    list_kernels<__nv_bfloat16>(list, count);
    list_kernels<__half>(list, count);
    return count;
  }();
  return launched(e.buf, e.len, loaded.once(list, n));
}

laq_status done(const Err& e, cudaError_t rc) { return launched(e.buf, e.len, rc); }

void set_temperature(ForwardArgs& A, float tau) {
  A.tau = tau;
  A.inv_tau = (float)(1.0 / (double)tau);
  A.c = (float)(1.4426950408889634 / (double)tau);
  A.unit = (float)(1.0 / ((double)tau * (double)A.c));
}
void set_temperature(GradArgs& A, float tau) {
  A.tau = tau;
  A.inv_tau = (float)(1.0 / (double)tau);
  A.inv_tau_lo = (float)(1.0 / (double)tau - (double)A.inv_tau);
  A.c = (float)(1.4426950408889634 / (double)tau);
  A.unit = (float)(1.0 / ((double)tau * (double)A.c));
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
  Buffers buffers;
  buffers.in("logits", d_logits, dtype_bytes(dtype), rows, vocab, row_stride);
  buffers.in("tokens", d_tokens, 4, 1, rows, rows);
  buffers.out("logprob", d_logprob, 4, 1, rows, rows);
  buffers.out("entropy", d_entropy, 4, 1, rows, rows);
  buffers.out("lse", d_lse, 4, 1, rows, rows);
  if (top_k) {
    buffers.out("top_tokens", d_top_tokens, 4, rows, top_k, top_k);
    buffers.out("top_logprobs", d_top_logprobs, 4, rows, top_k, top_k);
  }
  laq_status ok = buffers.check(errbuf, errbuf_len);
  if (ok == LAQ_OK) ok = load_kernels(e);
  if (ok != LAQ_OK) return ok;
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
  st = check_gradient(e, d_grad_logits, grad_row_stride, vocab);
  if (st != LAQ_OK) return st;
  Buffers buffers;
  buffers.in("logits", d_logits, dtype_bytes(dtype), rows, vocab, row_stride);
  buffers.in("tokens", d_tokens, 4, 1, rows, rows);
  buffers.in("lse", d_lse, 4, 1, rows, rows);
  buffers.in("entropy", d_entropy, 4, 1, rows, rows);
  buffers.in("grad_logprob", d_grad_logprob, 4, 1, rows, rows);
  buffers.in("grad_entropy", d_grad_entropy, 4, 1, rows, rows);
  buffers.out("grad_logits", d_grad_logits, dtype_bytes(dtype), rows, vocab, grad_row_stride, "logits");
  st = buffers.check(errbuf, errbuf_len);
  if (st == LAQ_OK) st = load_kernels(e);
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
    st = check_gradient(e, d_grad_logits, grad_row_stride, vocab);
    if (st != LAQ_OK) return st;
  }
  Buffers buffers;
  buffers.in("logits", d_logits, dtype_bytes(dtype), rows, vocab, row_stride);
  buffers.in("teacher_tokens", d_teacher_tokens, 4, rows, teacher_k, teacher_stride);
  buffers.in("teacher_logits", d_teacher_logits, 4, rows, teacher_k, teacher_stride);
  buffers.out("loss", d_loss, 4, 1, rows, rows);
  buffers.out("lse", d_lse, 4, 1, rows, rows);
  buffers.in("grad_loss", d_grad_loss, 4, 1, rows, rows);
  buffers.out("grad_logits", d_grad_logits, dtype_bytes(dtype), rows, vocab, grad_row_stride, "logits");
  st = buffers.check(errbuf, errbuf_len);
  if (st == LAQ_OK) st = load_kernels(e);
  if (st != LAQ_OK) return st;
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
  st = check_gradient(e, d_grad_logits, grad_row_stride, vocab);
  if (st != LAQ_OK) return st;
  Buffers buffers;
  buffers.in("logits", d_logits, dtype_bytes(dtype), rows, vocab, row_stride);
  buffers.in("teacher_tokens", d_teacher_tokens, 4, rows, teacher_k, teacher_stride);
  buffers.in("teacher_logits", d_teacher_logits, 4, rows, teacher_k, teacher_stride);
  buffers.in("lse", d_lse, 4, 1, rows, rows);
  buffers.in("grad_loss", d_grad_loss, 4, 1, rows, rows);
  buffers.out("grad_logits", d_grad_logits, dtype_bytes(dtype), rows, vocab, grad_row_stride, "logits");
  st = buffers.check(errbuf, errbuf_len);
  if (st == LAQ_OK) st = load_kernels(e);
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
