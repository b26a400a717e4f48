// A layer's product with bias, activation and residual in its epilogue, and its gradient:
//   Z = X W^T + b,  Y = act(Z) + R            X [M][K], W [N][K], b [N], R, Y, Z [M][N]
//   dZ = dY act'(Z),  dX = dZ W,  dW = dZ^T X,  db = column sums of dZ
// bf16 or fp16 operands, fp32 accumulation on the tcgen05 tensor cores, bias, activation and residual in fp32, one
// rounding per stored value.  dZ is rounded once to the operands' type, which the two products of the gradient need
// (exact for no activation and for ReLU; with the others dX and dW carry it beside their own, in bf16 0.0023 of the result, root
// mean square, where one rounding makes 0.0017: two 16-bit parts of dZ would double both products).
//
// One kernel serves all five products, D[i][j] = sum_r A(i, r) B(j, r).  An operand is "K-major" (the summed index r is
// contiguous in memory) or "MN-major" (the free index is contiguous); TMA brings 64 values of r a stage in either form
// with the 128-byte swizzle and the matrix descriptors tell the tensor core which one it is, so nothing is transposed in
// memory.  Warp 0 loads, warp 1 issues the products, warps 2-9 run the epilogue of one tile from tensor memory while the
// next one accumulates (two accumulators).  Large products run on pairs of SMs (cta_group::2, a 256-row tile): each SM of a
// pair loads its own 128 rows of A and half of B's columns, 32 KB for the work that a lone SM loads 48 KB for, and what an
// SM takes from L2 is what bounds the lone form.  8192 x 4096 x 4096 bf16: 189 us, 1.45 PFLOP/s (0.90 of the measured library
// rate); with gelu and residual 200 us.  What is left is the L2's rate (with a quarter of the products 160 us) and the
// last wave.  One to four rows of X are plain dot products (linear_few_rows_kernel).  For some more the roles of the
// operands are swapped (W's rows fill the 128 lanes, the rows of X are the narrow side) and the summed axis is split over a
// thread-block cluster whose blocks join their partial tiles through distributed shared memory in a fixed order.
//
// Times in this file are device times of one call replayed as a graph.  Among other calls, with inputs new each time, the same call
// takes longer (8192 x 4096 x 4096 with gelu and residual 234 us), and a call from a program adds its host time (12 us from Python,
// 27 for a gradient) where the kernels do not hide it.
#include <cooperative_groups.h>

#include <atomic>
#include <type_traits>

#include "laq_ops.cuh"
#include "laq_umma_gemm.cuh"

namespace cg = cooperative_groups;

namespace laq {
namespace ops {
namespace {

using umma::kBlockK;
using umma::kTileM;

constexpr int kSMs = 148;
constexpr int kGemmThreads = 320;         // loader, tensor-core warp, eight epilogue warps
constexpr int kEpiWarps = 8;
constexpr int kFewRows = 4;               // rows of X that plain dot products take
constexpr int kFewCols = 4, kFewThreads = 128, kFewBlocks = 4;   // columns of a warp, threads of a block, blocks on an SM
constexpr int kMaxStages = 12;
constexpr int kMaxRing = 192 * 1024;      // bytes of the stage ring
constexpr int kStaging = kEpiWarps * 4096;   // ... and of the epilogue warps' pieces behind it
constexpr int kMaxSplit = 8;
constexpr uint32_t kStarvedLimit = 1u << 12;
// The tensor core's fp32 sums are cut, not rounded: every 16 terms take up to an ulp off, always towards zero (8192 terms:
// 9e-6 of the result, 512 terms: 7e-7 with bf16 operands, 2.8e-6 with fp16 ones).  fp32 results are added up in chunks of 512
// terms, which the epilogue's threads keep in registers and add with rounding while the next chunk is under way.  16-bit
// results show it in long sums alone: 65536 terms lose 6e-5, an eighth of half a step of fp16, 2^20 would lose 8e-4.  Longer
// ones are added up in chunks of 16384 terms (1.6e-5), whose sums wait in the second accumulator's tensor memory, so that
// tiles may still be 256 wide: the tensor cores stand still for it for some 2000 cycles in a chunk's 180000.  (131072 rows, dW
// of 4096 x 1024 bf16: 866 us, without chunks 845 us, with the sums in registers and tiles of 128 columns 1505 us.)
constexpr int kChunk32 = 8, kChunkLong = 256;               // k-blocks
constexpr int kLongSum = 65536;           // terms that a 16-bit result takes at once
constexpr int kGroupTiles = 16;           // tile rows that are swept together, so that operands are found in L2

struct GemmArgs {
  int I, J, nkb;                 // rows and columns of D; 64-wide blocks of the summed axis
  int nt, stages, split;         // tile width, ring depth, blocks per tile
  int tiles_i, tiles_j;
  int a_mn, b_mn;                // 1: the operand is MN-major
  int fmt;                       // operand type of the instruction descriptor: 0 fp16, 1 bf16
  int act, starve;
  long long ldo, ldz, ldr;       // row strides of out, z and residual (elements)
  void* out;
  void* z;                       // or null
  const void* bias;              // or null
  const void* residual;          // or null
  uint32_t* status;
};

__device__ __forceinline__ uint64_t desc_k_major(uint32_t addr) { return umma::smem_desc_sw128(addr); }
// MN-major tile with the 128-byte swizzle: [64 r][64 free] blocks of 128-byte rows; eight rows of r are 1024 bytes
// apart (stride offset), the next 64 values of the free index 64 rows = 8192 bytes on (leading offset).
__device__ __forceinline__ uint64_t desc_mn_major(uint32_t addr) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3ffffu) >> 4);
  d |= (uint64_t)(8192 >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
__device__ __forceinline__ uint32_t instr_desc(int fmt, int a_mn, int b_mn, int nt, int rows) {
  return (1u << 4) | ((uint32_t)fmt << 7) | ((uint32_t)fmt << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) |
         ((uint32_t)(nt >> 3) << 17) | ((uint32_t)(rows >> 4) << 24);
}

// The kernels of one call follow each other closely: each allows the next to be set up beside it as soon as all of its
// blocks run, and one that was launched so waits, before it touches anything that the one before reads or writes, until
// that one has ended (a kernel launched in the ordinary way finds nothing to wait for).  No block asks for this before it
// holds its tensor memory, so one that waits for memory held by the kernel before always gets it.  A backward pass of four
// kernels: 64 x 200 x 784 38 -> 36 us, 8192 x 4096 x 1024 154 -> 150 us.
__device__ __forceinline__ void allow_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void await_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// One lane of the (converged) warp.  The loader and the tensor-core warp are led by an elected lane and not by a fixed one:
// the compiler then knows that one thread issues and needs no loop around every copy and product, which had left the tensor
// pipe idle 45 % of the time (8192 x 4096 x 4096: 228 -> 191 us).
__device__ __forceinline__ bool elect_one() {
  uint32_t ok;
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "elect.sync _|p, 0xffffffff;\n"
      "selp.u32 %0, 1, 0, p;\n"
      "}\n"
      : "=r"(ok));
  return ok != 0;
}

// 32 or 16 columns of this warp's lanes of tensor memory
__device__ __forceinline__ void tmem_store(uint32_t taddr, const uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"r"(v[0]),
      "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]),
      "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]),
      "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]),
      "r"(taddr)
      : "memory");
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_store(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(v[0]),
      "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]),
      "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(taddr)
      : "memory");
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_load(uint32_t taddr, uint32_t (&v)[32]) { umma::tmem_load_32(taddr, v); }
__device__ __forceinline__ void tmem_load(uint32_t taddr, uint32_t (&v)[16]) { umma::tmem_load_16(taddr, v); }

// ---- the instructions of a pair of blocks -----------------------------------------------------------------------------
__device__ __forceinline__ uint32_t of_leader(uint32_t addr) {      // the same shared-memory address in the pair's first block
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
  return r;
}
// a tile into this block's memory whose bytes are counted by a barrier of either block of the pair
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
      "l"(map), "r"(bar), "r"(x), "r"(y)
      : "memory");
}
__device__ __forceinline__ void mma_pair(uint32_t d_tmem, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n"
      "}\n" ::"r"(d_tmem),
      "l"(da), "l"(db), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void commit_pair(uint32_t bar) {         // arrives at this barrier of both blocks
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
               "h"((uint16_t)3)
               : "memory");
}
__device__ __forceinline__ void arrive_at(uint32_t cluster_bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}

// gelu is the tanh form: 0.5 z (1 + tanh u) = z sigmoid(2 u), u = sqrt(2/pi) (z + 0.044715 z^3).
constexpr float kGeluC = 0.7978845608028654f, kGeluA = 0.044715f;
__device__ __forceinline__ float sigmoid(float x) {       // 0 and 1 for far x: 2^128 is +inf and its reciprocal 0
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + ex2(-1.4426950408889634f * x)));
  return r;
}
template <int N>
__device__ __forceinline__ void activate(float (&z)[N], int act) {
  if (act == LAQ_ACT_RELU) {
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] = max_nan(z[e], 0.f);
  } else if (act == LAQ_ACT_SILU) {
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] *= sigmoid(z[e]);
  } else if (act == LAQ_ACT_GELU) {
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] *= sigmoid(2.f * kGeluC * fmaf(kGeluA * z[e] * z[e], z[e], z[e]));
  }
}
__device__ __forceinline__ float slope_silu(float z) {
  const float s = sigmoid(z);
  return s * fmaf(z, 1.f - s, 1.f);
}
__device__ __forceinline__ float slope_gelu(float z) {
  const float s = sigmoid(2.f * kGeluC * fmaf(kGeluA * z * z, z, z));
  // s (1 - s) is 0 long before z^2 passes 400, so that the product stays finite however far z is
  return fmaf(z * s * (1.f - s), fmaf(6.f * kGeluC * kGeluA, fminf(z * z, 400.f), 2.f * kGeluC), s);
}

// Eight rows row0.. of column `col` of out (rows x cols): the form for transposed tiles and for tensors that allow no
// vectors.  Neighbouring lanes hold neighbouring columns.
template <class T, bool OUT32>
__device__ __forceinline__ void finish_column(const GemmArgs& A, int rows, int cols, int row0, int col, float (&x)[8]) {
  if (col >= cols || row0 >= rows) return;
  const T* res = reinterpret_cast<const T*>(A.residual);
  const int n = min(8, rows - row0);
  const float b = A.bias ? Elem<T>::to_float(reinterpret_cast<const T*>(A.bias)[col]) : 0.f;
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = res && e < n ? Elem<T>::to_float(res[(long long)(row0 + e) * A.ldr + col]) : 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] += b;
  if (A.z) {
    T* z = reinterpret_cast<T*>(A.z) + (long long)row0 * A.ldz + col;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) z[e * A.ldz] = Elem<T>::from_float(x[e]);
  }
  activate(x, A.act);
  const long long at = (long long)row0 * A.ldo + col;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (e >= n) break;
    if (OUT32) reinterpret_cast<float*>(A.out)[at + e * A.ldo] = x[e] + r[e];
    else reinterpret_cast<T*>(A.out)[at + e * A.ldo] = Elem<T>::from_float(x[e] + r[e]);
  }
}

// Eight neighbours j0.. of row i of out, for tensors that all allow 16-byte accesses at multiples of eight columns; `res8`:
// the residual's, read beforehand.
template <class T, bool OUT32>
__device__ __forceinline__ void finish_row(const GemmArgs& A, int i, int j0, float (&x)[8], const uint4& res8) {
  if (i >= A.I || j0 >= A.J) return;
  if (j0 + 8 > A.J) {                       // the last columns of rows that end within a vector
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float one[8] = {x[e]};
      finish_column<T, OUT32>(A, i + 1, A.J, i, j0 + e, one);
    }
    return;
  }
  if (A.bias) {
    float b[8];
    Elem<T>::unpack(__ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(A.bias) + j0)), b);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] += b[e];
  }
  if (A.z) *reinterpret_cast<uint4*>(reinterpret_cast<T*>(A.z) + (long long)i * A.ldz + j0) = Elem<T>::pack(x);
  activate(x, A.act);
  if (A.residual) {
    float r[8];
    Elem<T>::unpack(res8, r);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] += r[e];
  }
  if (OUT32) {
    float4* o = reinterpret_cast<float4*>(reinterpret_cast<float*>(A.out) + (long long)i * A.ldo + j0);
    o[0] = make_float4(x[0], x[1], x[2], x[3]);
    o[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    *reinterpret_cast<uint4*>(reinterpret_cast<T*>(A.out) + (long long)i * A.ldo + j0) = Elem<T>::pack(x);
  }
}
template <class T>
__device__ __forceinline__ uint4 residual8(const GemmArgs& A, int i, int j0, bool vec) {
  uint4 r = make_uint4(0u, 0u, 0u, 0u);
  if (vec && A.residual && i < A.I && j0 + 8 <= A.J) r = load16(reinterpret_cast<const T*>(A.residual) + (long long)i * A.ldr + j0);
  return r;
}

// The fp32 values of a tile row by row in shared memory, 16-byte pieces permuted within a row so that a warp writes 32 rows
// and reads along rows without bank conflicts.
__device__ __forceinline__ int piece(int row, int p, int pieces) { return row * pieces + (p ^ (row & (pieces % 8 == 0 ? 7 : 3))); }

__device__ __forceinline__ bool aligned16(const void* p, long long ld_bytes) {
  return (((uintptr_t)p | (uintptr_t)ld_bytes) & 15u) == 0;
}

__device__ __forceinline__ bool all_vectors(const GemmArgs& A, bool out32) {
  return aligned16(A.out, A.ldo * (out32 ? 4 : 2)) && (!A.z || aligned16(A.z, A.ldz * 2)) &&
         (!A.residual || aligned16(A.residual, A.ldr * 2)) && (!A.bias || aligned16(A.bias, 0));
}

// Work item `w` -> tile origin.  Tile rows are swept in groups of kGroupTiles, column by column within a group.
template <bool PAIR>
__device__ __forceinline__ void tile_of(const GemmArgs& A, int w, int& i0, int& j0) {
  constexpr int kGroup = PAIR ? kGroupTiles / 2 : kGroupTiles;
  const int group = kGroup * A.tiles_j;
  const int g = w / group, in = w - g * group;
  const int first = g * kGroup;
  const int rows = min(kGroup, A.tiles_i - first);
  i0 = (first + in % rows) * (PAIR ? 2 * kTileM : kTileM);
  j0 = (in / rows) * A.nt;
}

template <class T, bool TRANS, bool PAIR, bool OUT32, bool LONG>
__global__ void __launch_bounds__(kGemmThreads, 1) linear_gemm_kernel(const __grid_constant__ CUtensorMap tmA,
                                                                      const __grid_constant__ CUtensorMap tmB,
                                                                      const GemmArgs A) {
  extern __shared__ unsigned char gemm_smem_raw[];
  __shared__ uint64_t bars[2 * kMaxStages + 5];
  __shared__ uint32_t tmem_base_sh;
  __shared__ int abort_sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t base = umma::smem_u32(gemm_smem_raw), smem0 = (base + 1023u) & ~1023u;
  uint4* ring4 = reinterpret_cast<uint4*>(gemm_smem_raw + (smem0 - base));        // a split tile, once the ring is idle
  static_assert(!(OUT32 && (LONG || TRANS)), "fp32 results have chunks of their own, and their epilogue writes rows");
  constexpr int kChunk = OUT32 ? kChunk32 : LONG ? kChunkLong : 1 << 30;      // k-blocks that the tensor core adds up
  const int nt = A.nt, stages = A.stages, split = PAIR ? 1 : A.split;
  const int b_rows = PAIR ? nt / 2 : nt;           // columns of the tile whose part of B this block loads
  const uint32_t a_bytes = kTileM * kBlockK * 2, st_bytes = a_bytes + (uint32_t)b_rows * kBlockK * 2;
  const int half = PAIR ? (int)(blockIdx.x & 1u) : 0;
  const uint32_t full0 = umma::smem_u32(&bars[0]), empty0 = umma::smem_u32(&bars[kMaxStages]);
  const uint32_t acc_full0 = umma::smem_u32(&bars[2 * kMaxStages]), acc_empty0 = acc_full0 + 16, drain = acc_full0 + 32;
  // Two accumulators of at most 256 columns; one for a split tile, which has no successor (two of at most 128 for the chunks
  // of an fp32 result).  A long sum's chunks all go to the first, their sum is in the second.  Two blocks of a cluster on one
  // SM must be able to hold theirs at the same time (each waits for the other), and two is all that fits by shared memory (one,
  // where a split long sum is more than 128 columns wide).
  const uint32_t acc_cols = umma::tmem_cols(nt), held_cols = split > 1 && !OUT32 && !LONG ? acc_cols : 2 * acc_cols;
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      umma::mbar_init(full0 + 8 * s, 1);
      umma::mbar_init(empty0 + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      umma::mbar_init(acc_full0 + 8 * b, 1);
      umma::mbar_init(acc_empty0 + 8 * b, PAIR ? 2 * kEpiWarps : kEpiWarps);
    }
    umma::mbar_init(drain, 1);
    abort_sh = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    if (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(umma::smem_u32(&tmem_base_sh)),
                   "r"(held_cols)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(umma::smem_u32(&tmem_base_sh)),
                   "r"(held_cols)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  if (PAIR) cg::this_cluster().sync();             // both blocks' barriers are there before either signals the other's
  else __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem_base = tmem_base_sh;
  allow_next();
  await_previous();

  const int tiles = A.tiles_i * A.tiles_j;
  const int rank = split > 1 ? (int)(blockIdx.x % (unsigned)split) : 0;
  const unsigned per_tile = PAIR ? 2u : (unsigned)split;
  const int first = (int)(blockIdx.x / per_tile), step = (int)(gridDim.x / per_tile);
  const int kb_per = (A.nkb + split - 1) / split;
  const int kb0 = min(rank * kb_per, A.nkb), nkb = min(kb0 + kb_per, A.nkb) - kb0;    // > 0: the plan leaves no block idle
  const bool starved = A.starve && blockIdx.x == 0;
  const uint32_t limit = A.starve ? kStarvedLimit : umma::kWaitLimit;
  // an accumulator takes its whole sum's time: one limit for every 2^16 k-blocks (some 30 ms) of it
  const uint32_t acc_limit = A.starve ? kStarvedLimit : umma::kWaitLimit * (1u + (uint32_t)(min(nkb, kChunk) >> 16));
  volatile int* abort_flag = &abort_sh;

  if (warp == 0) {
    if (elect_one()) {
      int n = 0;                       // stages handed out so far
      bool ok = !starved;
      for (int w = first; w < tiles && ok; w += step) {
        int i0, j0;
        tile_of<PAIR>(A, w, i0, j0);
        i0 += half * kTileM;
        j0 += half * b_rows;
        for (int kb = 0; kb < nkb; ++kb, ++n) {
          const int s = n % stages;
          ok = umma::mbar_wait_abortable(empty0 + 8 * s, ((uint32_t)(n / stages) & 1u) ^ 1u, limit, abort_flag, A.status, 1u);
          if (!ok) break;
          const uint32_t sa = smem0 + s * st_bytes, sb = sa + a_bytes;
          const int r = (kb0 + kb) * kBlockK;
          if (PAIR) {
            // the pair's first block counts the bytes of both; its phase cannot end before its own arrival here
            if (half == 0) umma::mbar_expect_tx(full0 + 8 * s, 2 * st_bytes);
            const uint32_t bar = of_leader(full0 + 8 * s);
            if (A.a_mn) {
              tma_load_2d_pair(sa, &tmA, bar, i0, r);
              tma_load_2d_pair(sa + 8192, &tmA, bar, i0 + 64, r);
            } else {
              tma_load_2d_pair(sa, &tmA, bar, r, i0);
            }
            if (A.b_mn) {
              for (int b = 0; b < b_rows; b += 64) tma_load_2d_pair(sb + b * 128, &tmB, bar, j0 + b, r);
            } else {
              tma_load_2d_pair(sb, &tmB, bar, r, j0);
            }
            continue;
          }
          const uint32_t bar = full0 + 8 * s;
          umma::mbar_expect_tx(bar, st_bytes);
          if (A.a_mn) {
            umma::tma_load_2d(sa, &tmA, bar, i0, r);
            umma::tma_load_2d(sa + 8192, &tmA, bar, i0 + 64, r);
          } else {
            umma::tma_load_2d(sa, &tmA, bar, r, i0);
          }
          if (A.b_mn) {
            for (int b = 0; b < nt; b += 64) umma::tma_load_2d(sb + b * 128, &tmB, bar, j0 + b, r);
          } else {
            umma::tma_load_2d(sb, &tmB, bar, r, j0);
          }
        }
      }
      if (!ok && PAIR) {                // given up: the copies in flight still land in this block's memory, and are counted
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);        // by the other block: microseconds are enough, 2 ms ample
      } else if (!ok) {
        for (int m = n > stages ? n - stages : 0; m < n; ++m)
          for (uint32_t it = 0; it < umma::kWaitLimit && !umma::mbar_try_wait(full0 + 8 * (m % stages), (uint32_t)(m / stages) & 1u); ++it) {
          }
      }
    }
  } else if (warp == 1) {
    if (half == 0 && elect_one()) {     // the pair's first block issues the products of both
      const uint32_t idesc = instr_desc(A.fmt, A.a_mn, A.b_mn, nt, PAIR ? 2 * kTileM : kTileM);
      // 16 values of r: 32 bytes on within the rows of a K-major tile, two groups of 8 rows (2048 bytes) on in an MN-major one
      const uint32_t step_a = A.a_mn ? 128u : 2u, step_b = A.b_mn ? 128u : 2u;
      int n = 0, it = 0;
      bool ok = true;
      for (int w = first; w < tiles && ok; w += step) {
        for (int k0 = 0; k0 < nkb && ok; k0 += kChunk, ++it) {
          const int b = LONG ? 0 : it & 1, turn = LONG ? it : it >> 1, k1 = min(k0 + kChunk, nkb);
          ok = umma::mbar_wait_abortable(acc_empty0 + 8 * b, ((uint32_t)turn & 1u) ^ 1u, limit, abort_flag, A.status, 2u);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t d = tmem_base + (uint32_t)b * acc_cols;
          for (int kb = k0; kb < k1; ++kb, ++n) {
            const int s = n % stages;
            ok = umma::mbar_wait_abortable(full0 + 8 * s, (uint32_t)(n / stages) & 1u, limit, abort_flag, A.status, 4u);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t sa = smem0 + s * st_bytes, sb = sa + a_bytes;
            const uint64_t da = A.a_mn ? desc_mn_major(sa) : desc_k_major(sa), db = A.b_mn ? desc_mn_major(sb) : desc_k_major(sb);
#pragma unroll
            for (int kk = 0; kk < kBlockK / 16; ++kk) {
              const uint32_t more = kb != k0 || kk != 0 ? 1u : 0u;
              if (PAIR) mma_pair(d, da + kk * step_a, db + kk * step_b, idesc, more);
              else umma::mma_bf16_ss(d, da + kk * step_a, db + kk * step_b, idesc, more);
            }
            if (PAIR) commit_pair(empty0 + 8 * s);
            else umma::mma_commit(empty0 + 8 * s);
          }
          if (ok) {
            if (PAIR) commit_pair(acc_full0 + 8 * b);
            else umma::mma_commit(acc_full0 + 8 * b);
          }
        }
      }
      if (!ok) {                        // products under way still read the ring and write tensor memory
        if (PAIR) commit_pair(drain);
        else umma::mma_commit(drain);
        for (uint32_t i = 0; i < umma::kWaitLimit && !umma::mbar_try_wait(drain, 0u); ++i) {
        }
      }
    }
    __syncwarp();
  } else {
    const int q = warp & 3, set = (warp - 2) >> 2;
    const int row = q * 32 + lane;
    const bool vec = all_vectors(A, OUT32);
    uint4* stage4 = ring4 + (size_t)stages * st_bytes / 16 + (warp - 2) * 256;         // 4 KB of this warp
    int it = 0;
    bool ok = true;
    for (int w = first; w < tiles && ok; w += step) {
      int i0, j0;
      tile_of<PAIR>(A, w, i0, j0);
      i0 += half * kTileM;
      // a tile that lies wholly inside D and allows vectors throughout goes without any checks; its residual is read one
      // piece ahead, the first one's before the products are done
      const bool whole = !TRANS && split == 1 && vec && i0 + kTileM <= A.I && j0 + nt <= A.J && nt % 32 == 0;
      const long long row0 = i0 + q * 32 + (lane >> 2);
      const int col0 = j0 + 8 * (lane & 3);
      uint4 res[4];
      auto ahead = [&](int c0) {
        const T* p = reinterpret_cast<const T*>(A.residual) + row0 * A.ldr + col0 + c0;
#pragma unroll
        for (int k = 0; k < 4; ++k) res[k] = load16(p + 8 * k * A.ldr);
      };
      if (!OUT32 && whole && A.residual && 32 * set < nt) ahead(32 * set);
      uint32_t t0 = 0;
      // the next accumulator, and its return to the tensor-core warp
      auto acquire = [&]() {
        const int b = LONG ? 0 : it & 1, turn = LONG ? it : it >> 1;
        ok = __all_sync(0xffffffffu, umma::mbar_wait_abortable(acc_full0 + 8 * b, (uint32_t)turn & 1u, acc_limit, abort_flag, A.status, 8u));
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        t0 = tmem_base + (uint32_t)b * acc_cols + ((uint32_t)(q * 32) << 16);
      };
      auto release = [&]() {
        const int b = LONG ? 0 : it & 1;
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          if (PAIR) arrive_at(of_leader(acc_empty0 + 8 * b));
          else umma::mbar_arrive(acc_empty0 + 8 * b);
        }
        ++it;
      };
      float sum[OUT32 ? 2 : 1][32];                    // fp32 results: the chunks' sums, this lane's row
      if constexpr (OUT32) {
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int e = 0; e < 32; ++e) sum[p][e] = 0.f;
        for (int k0 = 0; k0 < nkb; k0 += kChunk) {
          acquire();
          if (!ok) break;
#pragma unroll
          for (int p = 0; p < 2; ++p)
            if (32 * set + 64 * p < nt) {
              uint32_t v[32];
              umma::tmem_load_32(t0 + (uint32_t)(32 * set + 64 * p), v);
#pragma unroll
              for (int e = 0; e < 32; ++e) sum[p][e] += __uint_as_float(v[e]);
            }
          release();
        }
        if (!ok) break;
      } else {
        if constexpr (LONG) {
          // the chunks before the last; each warp adds up the columns that it will write out
          const uint32_t total = tmem_base + acc_cols + ((uint32_t)(q * 32) << 16);
          auto add_up = [&](auto& v, int c0, bool first_chunk) {
            tmem_load(t0 + (uint32_t)c0, v);
            if (!first_chunk) {
              std::remove_reference_t<decltype(v)> sum_so_far;
              tmem_load(total + (uint32_t)c0, sum_so_far);
#pragma unroll
              for (size_t e = 0; e < sizeof(v) / 4; ++e) v[e] = __float_as_uint(__uint_as_float(sum_so_far[e]) + __uint_as_float(v[e]));
            }
            tmem_store(total + (uint32_t)c0, v);
          };
          for (int k0 = 0; k0 + kChunk < nkb; k0 += kChunk) {
            acquire();
            if (!ok) break;
            if (TRANS || split > 1) {
              uint32_t v[16];
              for (int c0 = 16 * set; c0 < nt; c0 += 32) add_up(v, c0, k0 == 0);
            } else {
              uint32_t v[32];
              for (int c0 = 32 * set; c0 < nt; c0 += 64) add_up(v, c0, k0 == 0);
            }
            release();
          }
          if (!ok) break;
        }
        acquire();
        if (!ok) break;
      }
      // the values from column c0 on of this lane's row: the accumulator's, and the sum of the chunks before it
      auto loaded = [&](int c0, auto& v) {
        tmem_load(t0 + (uint32_t)c0, v);    // past nt only where nt is no multiple of 32: not used then
        if constexpr (LONG) {
          if (nkb > kChunk) {
            std::remove_reference_t<decltype(v)> sum_so_far;
            tmem_load(tmem_base + acc_cols + ((uint32_t)(q * 32) << 16) + (uint32_t)c0, sum_so_far);
#pragma unroll
            for (size_t e = 0; e < sizeof(v) / 4; ++e) v[e] = __float_as_uint(__uint_as_float(sum_so_far[e]) + __uint_as_float(v[e]));
          }
        }
      };
      // 32 of them
      auto values = [&](int c0, uint32_t (&v)[32]) {
        if constexpr (OUT32) {
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(c0 >= 64 ? sum[1][e] : sum[0][e]);
        } else {
          loaded(c0, v);
        }
      };
      if (split > 1 && OUT32) {
        for (int c0 = 32 * set; c0 < nt; c0 += 64) {
          uint32_t v[32];
          values(c0, v);
#pragma unroll
          for (int e = 0; e < 32; e += 4)
            ring4[piece(row, (c0 + e) / 4, nt / 4)] = make_uint4(v[e], v[e + 1], v[e + 2], v[e + 3]);
        }
      } else if (split > 1) {
        for (int c0 = 16 * set; c0 < nt; c0 += 32) {
          uint32_t v[16];
          loaded(c0, v);
#pragma unroll
          for (int e = 0; e < 16; e += 4)
            ring4[piece(row, (c0 + e) / 4, nt / 4)] = make_uint4(v[e], v[e + 1], v[e + 2], v[e + 3]);
        }
      } else if (TRANS) {
        for (int c0 = 16 * set; c0 < nt; c0 += 32) {
          uint32_t v[16];
          loaded(c0, v);
          float x[2][8];
#pragma unroll
          for (int e = 0; e < 16; ++e) x[e >> 3][e & 7] = __uint_as_float(v[e]);
          finish_column<T, OUT32>(A, A.J, A.I, j0 + c0, i0 + row, x[0]);
          finish_column<T, OUT32>(A, A.J, A.I, j0 + c0 + 8, i0 + row, x[1]);
        }
      } else {
        // 32 x 32 pieces: a lane takes its row from tensor memory and hands it on; four lanes then share a row, so that
        // loads and stores of the layer's tensors are whole 64-byte stretches
#pragma unroll 1
        for (int c0 = 32 * set; c0 < nt && whole; c0 += 64) {
          const int j = col0 + c0;
          uint4 now[4];
          float bias[8] = {};
          if constexpr (!OUT32) {
#pragma unroll
            for (int k = 0; k < 4; ++k) now[k] = res[k];
            if (A.residual && c0 + 64 < nt) ahead(c0 + 64);
            if (A.bias) Elem<T>::unpack(__ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(A.bias) + j)), bias);
          }
          uint32_t v[32];
          values(c0, v);
          __syncwarp();
#pragma unroll
          for (int e = 0; e < 32; e += 4) stage4[piece(lane, e / 4, 8)] = make_uint4(v[e], v[e + 1], v[e + 2], v[e + 3]);
          __syncwarp();
          T* zp = A.z ? reinterpret_cast<T*>(A.z) + row0 * A.ldz + j : nullptr;
          T* yp = reinterpret_cast<T*>(A.out) + row0 * A.ldo + j;
          float* fp = reinterpret_cast<float*>(A.out) + row0 * A.ldo + j;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int r = 8 * k + (lane >> 2);
            const uint4 lo = stage4[piece(r, 2 * (lane & 3), 8)], hi = stage4[piece(r, 2 * (lane & 3) + 1, 8)];
            if constexpr (OUT32) {
              *reinterpret_cast<uint4*>(fp + 8 * k * A.ldo) = lo;
              *reinterpret_cast<uint4*>(fp + 8 * k * A.ldo + 4) = hi;
            } else {
              float x[8] = {__uint_as_float(lo.x), __uint_as_float(lo.y), __uint_as_float(lo.z), __uint_as_float(lo.w),
                            __uint_as_float(hi.x), __uint_as_float(hi.y), __uint_as_float(hi.z), __uint_as_float(hi.w)};
#pragma unroll
              for (int e = 0; e < 8; ++e) x[e] += bias[e];
              if (zp) *reinterpret_cast<uint4*>(zp + 8 * k * A.ldz) = Elem<T>::pack(x);
              activate(x, A.act);
              if (A.residual) {
                float y[8];
                Elem<T>::unpack(now[k], y);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] += y[e];
              }
              *reinterpret_cast<uint4*>(yp + 8 * k * A.ldo) = Elem<T>::pack(x);
            }
          }
        }
#pragma unroll 1
        for (int c0 = 32 * set; c0 < nt && !whole; c0 += 64) {
          const int jl = j0 + c0 + 8 * (lane & 3);
          uint4 some[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) some[k] = residual8<T>(A, i0 + q * 32 + 8 * k + (lane >> 2), jl, vec);
          uint32_t v[32];
          values(c0, v);
          __syncwarp();
#pragma unroll
          for (int e = 0; e < 32; e += 4) stage4[piece(lane, e / 4, 8)] = make_uint4(v[e], v[e + 1], v[e + 2], v[e + 3]);
          __syncwarp();
          if (!vec) {
            for (int k = 0; k < 32 && c0 + lane < nt; k += 8) {
              float x[8];
#pragma unroll
              for (int e = 0; e < 8; ++e)
                x[e] = __uint_as_float(reinterpret_cast<const uint32_t*>(&stage4[piece(k + e, lane >> 2, 8)])[lane & 3]);
              finish_column<T, OUT32>(A, A.I, A.J, i0 + q * 32 + k, j0 + c0 + lane, x);
            }
            continue;
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int r = 8 * k + (lane >> 2);
            const uint4 lo = stage4[piece(r, 2 * (lane & 3), 8)], hi = stage4[piece(r, 2 * (lane & 3) + 1, 8)];
            float x[8] = {__uint_as_float(lo.x), __uint_as_float(lo.y), __uint_as_float(lo.z), __uint_as_float(lo.w),
                          __uint_as_float(hi.x), __uint_as_float(hi.y), __uint_as_float(hi.z), __uint_as_float(hi.w)};
            if (c0 + 8 * (lane & 3) < nt) finish_row<T, OUT32>(A, i0 + q * 32 + r, jl, x, some[k]);
          }
        }
      }
      if (!OUT32) release();
    }
  }
  if (split > 1) {          // one tile per cluster: its blocks share the columns of the join
    cg::cluster_group cluster = cg::this_cluster();
    __syncwarp();
    cluster.sync();
    if (warp >= 2) {
      int gone = 0;
      for (int r = 0; r < split; ++r) gone |= *cluster.map_shared_rank(&abort_sh, r);
      const bool vec = all_vectors(A, OUT32);
      int i0, j0;
      tile_of<false>(A, first, i0, j0);
      // eight columns of a row at a time; lanes run along a row, or down the rows where out is transposed
      const int groups = nt / 8, tid = (int)threadIdx.x - 64;
      if (TRANS || vec) {
        for (int item = rank * 256 + tid; item < kTileM * groups && !gone; item += 256 * split) {
          const int r0 = TRANS ? item % kTileM : item / groups, g = TRANS ? item / kTileM : item % groups;
          const uint4 res = TRANS ? make_uint4(0u, 0u, 0u, 0u) : residual8<T>(A, i0 + r0, j0 + g * 8, vec);
          uint4 lo[kMaxSplit], hi[kMaxSplit];               // all blocks' parts on their way at once, added in order
#pragma unroll
          for (int r = 0; r < kMaxSplit; ++r)
            if (r < split) {
              const uint4* p = cluster.map_shared_rank(ring4, r);
              lo[r] = p[piece(r0, 2 * g, nt / 4)];
              hi[r] = p[piece(r0, 2 * g + 1, nt / 4)];
            }
          float x[8] = {};
#pragma unroll
          for (int r = 0; r < kMaxSplit; ++r)
            if (r < split) {
              x[0] += __uint_as_float(lo[r].x);
              x[1] += __uint_as_float(lo[r].y);
              x[2] += __uint_as_float(lo[r].z);
              x[3] += __uint_as_float(lo[r].w);
              x[4] += __uint_as_float(hi[r].x);
              x[5] += __uint_as_float(hi[r].y);
              x[6] += __uint_as_float(hi[r].z);
              x[7] += __uint_as_float(hi[r].w);
            }
          if (TRANS) finish_column<T, OUT32>(A, A.J, A.I, j0 + g * 8, i0 + r0, x);
          else finish_row<T, OUT32>(A, i0 + r0, j0 + g * 8, x, res);
        }
      } else {                                   // eight rows of a column: lanes run along the columns
        for (int item = rank * 256 + tid; item < kTileM / 8 * nt && !gone; item += 256 * split) {
          const int r0 = item / nt * 8, c = item % nt;
          float x[8] = {};
          for (int r = 0; r < split; ++r) {
            const uint4* p = cluster.map_shared_rank(ring4, r);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] += reinterpret_cast<const float*>(p + piece(r0 + e, c >> 2, nt / 4))[c & 3];
          }
          finish_column<T, OUT32>(A, A.I, A.J, i0 + r0, j0 + c, x);
        }
      }
    }
    __syncwarp();
    cluster.sync();
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  if (PAIR) {
    __syncwarp();
    cg::this_cluster().sync();                     // neither block's memory is used by the other any more
  } else {
    __syncthreads();
  }
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(held_cols) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(held_cols) : "memory");
  }
}

// ---- dZ and the column sums ---------------------------------------------------------------------------------------------
// Bound by memory: 8192 x 4096 with gelu 39 us, 201 MB, 5.2 TB/s (0.79; two special-function and some twenty other
// operations an element come near).  A block takes 256 columns (32 threads of eight) and a run of rows (8 threads, two rows at a time): dZ = dY act'(Z), stored
// once if dz is given, and the sum of its columns over the run, in fp32 of the UNROUNDED products, to part[run][N].
constexpr int kDzCols = 256, kDzThreads = 256;

template <class T>
__global__ void __launch_bounds__(kDzThreads, 4) linear_dz_kernel(const T* dy, long long lddy, const T* z, long long ldz, T* dz,
                                                                  long long lddz, float* part, long long M, int N, int act,
                                                                  int rows_per, int vec_ok) {
  __shared__ float sh[8][kDzCols];
  allow_next();
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const int c0 = blockIdx.x * kDzCols + tx * 8;
  const long long r0 = (long long)blockIdx.y * rows_per, r1 = min(r0 + (long long)rows_per, M);
  float sum[8] = {};
  auto row = [&](long long r, float (&g)[8], float (&x)[8]) {
    if (act == LAQ_ACT_RELU) {
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] = x[e] > 0.f ? g[e] : (x[e] == x[e] ? 0.f : x[e]);
    } else if (act == LAQ_ACT_GELU) {
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] *= slope_gelu(x[e]);
    } else if (act == LAQ_ACT_SILU) {
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] *= slope_silu(x[e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += g[e];
    // the workspace's rows are 16-byte aligned and padded to eight columns
    if (dz) *reinterpret_cast<uint4*>(dz + r * lddz + c0) = Elem<T>::pack(g);
  };
  if (c0 < N && vec_ok && c0 + 8 <= N) {
    const T* pg = dy + c0;
    const T* px = z + c0;
    for (long long r = r0 + ty; r < r1; r += 16) {
      const bool two = r + 8 < r1;
      uint4 g0 = load16(pg + r * lddy), g1 = two ? load16(pg + (r + 8) * lddy) : make_uint4(0u, 0u, 0u, 0u);
      uint4 x0 = g0, x1 = g1;
      if (act != LAQ_ACT_NONE) {
        x0 = load16(px + r * ldz);
        if (two) x1 = load16(px + (r + 8) * ldz);
      }
      float g[8], x[8];
      Elem<T>::unpack(g0, g);
      Elem<T>::unpack(x0, x);
      row(r, g, x);
      if (two) {
        Elem<T>::unpack(g1, g);
        Elem<T>::unpack(x1, x);
        row(r + 8, g, x);
      }
    }
  } else if (c0 < N) {
    for (long long r = r0 + ty; r < r1; r += 8) {
      float g[8], x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        g[e] = c0 + e < N ? Elem<T>::to_float(dy[r * lddy + c0 + e]) : 0.f;
        x[e] = act != LAQ_ACT_NONE && c0 + e < N ? Elem<T>::to_float(z[r * ldz + c0 + e]) : 0.f;
      }
      row(r, g, x);
    }
  }
  if (!part) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) sh[ty][tx * 8 + e] = sum[e];
  __syncthreads();
  const int c = blockIdx.x * kDzCols + (int)threadIdx.x;
  if (c < N) {
    float t = 0.f;
#pragma unroll
    for (int y = 0; y < 8; ++y) t += sh[y][threadIdx.x];
    part[(long long)blockIdx.y * N + c] = t;
  }
}

__global__ void __launch_bounds__(1024) linear_db_kernel(const float* part, int runs, int N, float* db) {
  __shared__ float sh[32][33];
  allow_next();
  await_previous();
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, c = blockIdx.x * 32 + tx;
  float s = 0.f;
  if (c < N) {
#pragma unroll 4
    for (int r = ty; r < runs; r += 32) s += part[(long long)r * N + c];
  }
  sh[ty][tx] = s;
  __syncthreads();
  float t = sh[tx][ty];                  // warp ty adds up column ty
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  if (tx == 0 && blockIdx.x * 32 + ty < N) db[blockIdx.x * 32 + ty] = t;
}

// One to four rows: W is read once and nothing is used twice, so memory bounds it and plain dot products keep up.  A warp
// takes four columns of Y (rows of W) and all or, of few columns, a part of the summed axis: the block's warps that share
// columns join through shared memory in a fixed order.  A warp's sums are folded so that each step halves the values a lane
// holds.  Each lane has AHEAD vectors of each of its four rows of W under way; X comes from the first-level cache.
//
// In us, by this kernel and by the tensor cores' (bias, silu and residual, weights that the L2 cache does not hold, launches
// in a row):
//   N x K        4096 x 4096    11008 x 4096    4096 x 11008    32000 x 2048    100000 x 512    200 x 784
//   1 row          7.4  12.8       16.4  25.6      16.5  23.5      22.1  30.8      19.5  24.9     2.3   7.9
//   2 rows         8.8  13.6       19.8  26.0      18.5  24.0      26.0  30.5      24.6  26.1     2.5   7.9
//   4 rows        10.5  13.6       23.9  26.0      21.6  24.3      30.6  31.2      32.8  26.2     2.7   8.0
// W is marked as read once: weights that stay in the L2 cache are not slower for it (4096 x 4096 6.3 us either way), and
// those that do not are faster (32000 x 2048, one row: 23.6 -> 22.1).
// (Blocks of 256 threads are dealt out less evenly, 11008 x 4096, one row: 19.5 us; vectors of X loaded ahead as well cost
// the registers that more vectors of W need, 4096 x 4096: 8.8 us.)
template <class T, int ROWS, int AHEAD>
__global__ void __launch_bounds__(kFewThreads, ROWS <= 2 && AHEAD == 2 ? kFewBlocks + 2 : kFewBlocks)
    linear_few_rows_kernel(const GemmArgs A, const T* x, long long ldx, const T* w, long long ldw, int K, int vec, int log_parts) {
  constexpr int kRows2 = ROWS == 3 ? 4 : ROWS, kSums = kFewCols * kRows2, kWarps = kFewThreads / 32;
  __shared__ float part[kWarps][kSums];
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5, parts = 1 << log_parts;
  const int col0 = (int)(blockIdx.x * (unsigned)(kWarps >> log_parts)) * kFewCols;
  const int first = (warp & (parts - 1)) * 32 + lane, step = 32 << log_parts;
  const T* wr[kFewCols];
#pragma unroll
  for (int c = 0; c < kFewCols; ++c) wr[c] = w + (long long)min(col0 + (warp >> log_parts) * kFewCols + c, A.J - 1) * ldw;
  f32x2 sum[kFewCols][ROWS];
#pragma unroll
  for (int c = 0; c < kFewCols; ++c)
#pragma unroll
    for (int m = 0; m < ROWS; ++m) sum[c][m] = 0ull;
  const int nv = vec ? K / 8 : 0;                  // of the summed axis in vectors
  auto batch = [&](int v0, auto whole) {           // whole: all of its vectors exist
    uint4 a[AHEAD][kFewCols];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int v = v0 + u * step;
#pragma unroll
      for (int c = 0; c < kFewCols; ++c)
        a[u][c] = decltype(whole)::value || v < nv ? __ldcs(reinterpret_cast<const uint4*>(wr[c]) + v) : make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int v = v0 + u * step;
      f32x2 q[ROWS][4];
#pragma unroll
      for (int m = 0; m < ROWS; ++m)               // nothing of X where there is nothing of W: zero times an infinity would count
        Elem<T>::pairs(decltype(whole)::value || v < nv ? __ldg(reinterpret_cast<const uint4*>(x + m * ldx) + v) : make_uint4(0u, 0u, 0u, 0u), q[m]);
#pragma unroll
      for (int c = 0; c < kFewCols; ++c) {
        f32x2 p[4];
        Elem<T>::pairs(a[u][c], p);
#pragma unroll
        for (int m = 0; m < ROWS; ++m)
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[c][m] = fma2(p[e], q[m][e], sum[c][m]);
      }
    }
  };
  int v0 = first;
  for (; v0 + (AHEAD - 1) * step < nv; v0 += AHEAD * step) batch(v0, std::true_type());
  if (v0 < nv) batch(v0, std::false_type());
  float s[kSums];
#pragma unroll
  for (int c = 0; c < kFewCols; ++c)
#pragma unroll
    for (int m = 0; m < kRows2; ++m) {
      float lo = 0.f, hi = 0.f;
      if (m < ROWS) split(sum[c][m < ROWS ? m : 0], lo, hi);
      s[c * kRows2 + m] = lo + hi;
    }
#pragma unroll 4
  for (int k = nv * 8 + first; k < K; k += step) {
    float q[ROWS];
#pragma unroll
    for (int m = 0; m < ROWS; ++m) q[m] = Elem<T>::to_float(x[m * ldx + k]);
#pragma unroll
    for (int c = 0; c < kFewCols; ++c) {
      const float p = Elem<T>::to_float(wr[c][k]);
#pragma unroll
      for (int m = 0; m < ROWS; ++m) s[c * kRows2 + m] = fmaf(p, q[m], s[c * kRows2 + m]);
    }
  }
  int o = 16;
#pragma unroll
  for (int n = kSums / 2; n > 0; n /= 2, o /= 2) {          // lanes with bit o keep the upper half of the sums
    const bool upper = lane & o;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float other = __shfl_xor_sync(0xffffffffu, upper ? s[i] : s[i + n], o);
      s[i] = (upper ? s[i + n] : s[i]) + other;
    }
  }
#pragma unroll
  for (; o > 0; o /= 2) s[0] += __shfl_xor_sync(0xffffffffu, s[0], o);
  if (lane % (32 / kSums) == 0) part[warp][lane / (32 / kSums)] = s[0];
  __syncthreads();
  if (t < kFewCols * kWarps >> log_parts) {
    float y[8] = {};
    for (int i = 0; i < parts; ++i)
#pragma unroll
      for (int m = 0; m < ROWS; ++m) y[m] += part[(t / kFewCols << log_parts) + i][t % kFewCols * kRows2 + m];
    finish_column<T, false>(A, A.I, A.J, 0, col0 + t, y);
  }
}

// Rows that a tensor map cannot describe (an address or a row pitch that is no multiple of 16 bytes) are copied once
// into the workspace with a pitch of a multiple of eight elements.
__global__ void __launch_bounds__(256) linear_pack_kernel(const uint16_t* src, long long ld, uint16_t* dst, long long pitch,
                                                          long long rows, int cols) {
  allow_next();
  const int groups = (cols + 7) / 8;
  const long long n = rows * groups, stride = (long long)gridDim.x * blockDim.x;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += stride) {
    const long long r = i / groups;
    const int c = (int)(i - r * groups) * 8;
    const uint16_t* s = src + r * ld + c;
    uint16_t v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c + e < cols ? s[e] : (uint16_t)0;
    uint4 o;
    o.x = v[0] | ((uint32_t)v[1] << 16);
    o.y = v[2] | ((uint32_t)v[3] << 16);
    o.z = v[4] | ((uint32_t)v[5] << 16);
    o.w = v[6] | ((uint32_t)v[7] << 16);
    *reinterpret_cast<uint4*>(dst + r * pitch + c) = o;
  }
}

// ---- host -----------------------------------------------------------------------------------------------------------------
size_t align256(size_t x) { return (x + 255) / 256 * 256; }
long long pad8(long long x) { return (x + 7) / 8 * 8; }
bool mappable(const void* p, long long ld) { return ((uintptr_t)p & 15u) == 0 && (ld % 8) == 0; }

struct Operand {                // a 2-byte matrix [rows][cols]
  const void* p;
  long long ld, rows, cols;
  bool mappable_() const { return mappable(p, ld); }
  size_t pack_bytes() const { return mappable_() ? 0 : align256((size_t)rows * pad8(cols) * 2); }
};

struct Plan {
  int swap, nt, split, stages, pair;
  double cost;
};

// Tile width, split, pairs and orientation by an estimate of the time in SM cycles, whose constants were fitted to all of
// these forms measured on 26 products (1 to 16384 rows): a stage costs the larger of its products (2.7 cycles per column of
// the tile, 2 at the tensor pipe's rate) and of its bytes (60 a cycle); a tile's epilogue 2000 and 9 per column, 45 where it
// writes element by element; the epilogue of one tile runs beside the products of the next.  A pair's start costs 4500
// more; the join of a split 6500 and 25 per column, and clusters of four and eight reach 136 and 128 SMs.  The form chosen by
// it is within 3 % of the fastest in 22 of the 26 and at most 25 % slower in the others.
// `swappable`: the epilogue may write the transposed tile.  An fp32 result's tile is a multiple of 64 wide (its operands are
// MN-major).
Plan make_plan(long long I, long long J, long long R, bool a_mn, bool b_mn, bool swappable, bool out32, bool long_sum) {
  Plan best{0, 128, 1, 4, 0, 1e300};
  const long long nkb = (R + kBlockK - 1) / kBlockK;
  const auto persistent = [](double waves, double main, double epi) {
    return waves * (main > epi ? main : epi) + 0.1 * (main > epi ? epi : main) + epi;
  };
  for (int swap = 0; swap <= (swappable ? 1 : 0); ++swap) {
    const long long i = swap ? J : I, j = swap ? I : J;
    const long long rows = (i + kTileM - 1) / kTileM, row_pairs = (rows + 1) / 2;
    const bool bmn = swap ? a_mn : b_mn;
    static const int widths[] = {16, 32, 64, 96, 112, 128, 160, 192, 208, 224, 256};
    for (int nt : widths) {
      if (bmn && nt % 64) continue;
      if ((swap || out32) && nt > 128) continue;     // fp32 results: 64 sums a thread
      const double mma = 2.7 * nt, epi = 2000 + (swap ? 45.0 : 9.0) * nt;
      const int stage = (kTileM + nt) * kBlockK * 2;
      const double per = mma > stage / 60.0 ? mma : stage / 60.0;
      const long long cols = (j + nt - 1) / nt, tiles = rows * cols;
      for (int log2 = 0; log2 <= 3; ++log2) {
        const int split = 1 << log2;
        const long long kb = (nkb + split - 1) >> log2;
        if (split > 1 && kb * (split - 1) >= nkb) continue;           // a block would have nothing to do
        int stages = (split > 1 ? 110 * 1024 : kMaxRing) / stage;
        if (stages > kMaxStages) stages = kMaxStages;
        if (split > 1)                                                 // the partial tile in the ring
          while (stages * stage < kTileM * nt * 4 || stages < 3) ++stages;
        if (stages * stage > kMaxRing) continue;
        // A split long sum of more than 128 columns holds all of an SM's tensor memory: only where no other split tile's block
        // (84 KB of ring at least, at 96 columns) fits beside it, since blocks of two calls could otherwise keep one another from
        // the clusters that they wait for.  256 columns (144 KB) remain.
        if (split > 1 && long_sum && nt > 128 && stages * stage <= 136 * 1024) continue;
        const double main = kb * per;
        double cost;
        if (split == 1) {
          cost = persistent((double)((tiles + kSMs - 1) / kSMs), main, epi);
        } else {
          const long long blocks = tiles << log2;
          const long long waves = split == 8 ? (blocks + 127) / 128 : split == 4 ? (blocks + 135) / 136 : (blocks + kSMs - 1) / kSMs;
          cost = 6500 + (double)waves * (main + 25.0 * nt) + epi / split;
        }
        if (cost < best.cost) best = Plan{swap, nt, split, stages, 0, cost};
      }
      // pairs of SMs: 256 rows of D
      if (!swap && nt % 128 == 0 && rows > 1) {
        const int half = (kTileM + nt / 2) * kBlockK * 2;
        int stages = kMaxRing / half;
        if (stages > kMaxStages) stages = kMaxStages;
        const double main = nkb * (mma > half / 60.0 ? mma : half / 60.0);
        const double cost = 4500 + persistent((double)((row_pairs * cols + kSMs / 2 - 1) / (kSMs / 2)), main, epi);
        if (cost < best.cost) best = Plan{0, nt, 1, stages, 1, cost};
      }
    }
  }
  return best;
}

struct Err {
  char* buf;
  size_t len;
};

template <class T, bool TRANS, bool PAIR, bool OUT32, bool LONG>
laq_status launch_gemm(const Err& e, const CUtensorMap& ma, const CUtensorMap& mb, const GemmArgs& A, bool follows,
                       cudaStream_t st) {
  auto kernel = linear_gemm_kernel<T, TRANS, PAIR, OUT32, LONG>;
  const size_t smem = (size_t)A.stages * (kTileM + (PAIR ? A.nt / 2 : A.nt)) * kBlockK * 2 + (TRANS || A.split > 1 ? 0 : kStaging) + 1024;
  const int per_tile = PAIR ? 2 : A.split;
  // the kernel's shared memory limit is raised once per device
  static std::atomic<uint64_t> raised{0};
  int dev = 0;
  cudaGetDevice(&dev);
  const uint64_t bit = 1ull << (dev & 63);
  if (dev >= 64 || !(raised.load(std::memory_order_acquire) & bit)) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxRing + kStaging + 1024) != cudaSuccess) {
      cudaGetLastError();
      return fail(e.buf, e.len, LAQ_ECUDA, "shared memory of the product kernel was refused");
    }
    raised.fetch_or(bit, std::memory_order_release);
  }
  const long long tiles = (long long)A.tiles_i * A.tiles_j;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(PAIR ? 2 * (tiles < kSMs / 2 ? tiles : kSMs / 2) : A.split > 1 ? tiles * A.split : tiles < kSMs ? tiles : kSMs));
  cfg.blockDim = dim3(kGemmThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  cfg.attrs = at;
  if (per_tile > 1) {
    at[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
    at[cfg.numAttrs].val.clusterDim.x = (unsigned)per_tile;
    at[cfg.numAttrs].val.clusterDim.y = at[cfg.numAttrs].val.clusterDim.z = 1;
    ++cfg.numAttrs;
  }
  if (follows) {
    at[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[cfg.numAttrs].val.programmaticStreamSerializationAllowed = 1;
    ++cfg.numAttrs;
  }
  return launched(e.buf, e.len, cudaLaunchKernelEx(&cfg, kernel, ma, mb, A));
}

template <class T, bool LONG>
laq_status launch_16(const Err& e, const Plan& pl, const CUtensorMap& ma, const CUtensorMap& mb, const GemmArgs& A, bool follows,
                     cudaStream_t st) {
  if (pl.pair) return launch_gemm<T, false, true, false, LONG>(e, ma, mb, A, follows, st);
  return pl.swap ? launch_gemm<T, true, false, false, LONG>(e, ma, mb, A, follows, st)
                 : launch_gemm<T, false, false, false, LONG>(e, ma, mb, A, follows, st);
}

template <class T>
laq_status launch_form(const Err& e, const Plan& pl, bool out32, bool long_sum, const CUtensorMap& ma, const CUtensorMap& mb,
                       const GemmArgs& A, bool follows, cudaStream_t st) {
  if (out32)
    return pl.pair ? launch_gemm<T, false, true, true, false>(e, ma, mb, A, follows, st)
                   : launch_gemm<T, false, false, true, false>(e, ma, mb, A, follows, st);
  return long_sum ? launch_16<T, true>(e, pl, ma, mb, A, follows, st) : launch_16<T, false>(e, pl, ma, mb, A, follows, st);
}

struct Epilogue {
  void* out = nullptr;
  long long ldo = 0;
  int out_f32 = 0, act = LAQ_ACT_NONE;
  const void *bias = nullptr, *residual = nullptr;
  long long ldr = 0;
  void* z = nullptr;
  long long ldz = 0;
};

// D[i][j] = sum_r A(i, r) B(j, r): a_mn ? A is stored [r][i] : [i][r], the same for B.  Both are mappable.  `follows`: the
// stream's last work is a kernel of the same call.
laq_status product(const Err& e, int dtype, const Operand& a, bool a_mn, const Operand& b, bool b_mn, const Epilogue& ep,
                   uint32_t* status, int starve, bool swappable, bool follows, cudaStream_t st) {
  const long long I = a_mn ? a.cols : a.rows, R = a_mn ? a.rows : a.cols, J = b_mn ? b.cols : b.rows;
  const bool out32 = ep.out_f32 != 0, long_sum = !out32 && R > kLongSum;
  const Plan pl = make_plan(I, J, R, a_mn, b_mn, swappable, out32, long_sum);
  const Operand& A0 = pl.swap ? b : a;
  const Operand& B0 = pl.swap ? a : b;
  const bool amn = pl.swap ? b_mn : a_mn, bmn = pl.swap ? a_mn : b_mn;
  CUtensorMap ma, mb;
  if (!umma::make_map_bf16_2d(&ma, A0.p, A0.rows, A0.cols, A0.ld * 2, amn ? 64 : kTileM) ||
      !umma::make_map_bf16_2d(&mb, B0.p, B0.rows, B0.cols, B0.ld * 2, bmn ? 64 : pl.pair ? pl.nt / 2 : pl.nt))
    return fail(e.buf, e.len, LAQ_ECUDA, "a tensor map was refused");
  GemmArgs A = {};
  A.I = (int)(pl.swap ? J : I);
  A.J = (int)(pl.swap ? I : J);
  A.nkb = (int)((R + kBlockK - 1) / kBlockK);
  A.nt = pl.nt;
  A.stages = pl.stages;
  A.split = pl.split;
  const int tile_rows = pl.pair ? 2 * kTileM : kTileM;
  A.tiles_i = (A.I + tile_rows - 1) / tile_rows;
  A.tiles_j = (A.J + pl.nt - 1) / pl.nt;
  A.a_mn = amn;
  A.b_mn = bmn;
  A.fmt = dtype == LAQ_BF16 ? 1 : 0;
  A.act = ep.act;
  A.starve = starve;
  A.ldo = ep.ldo;
  A.ldz = ep.ldz;
  A.ldr = ep.ldr;
  A.out = ep.out;
  A.z = ep.z;
  A.bias = ep.bias;
  A.residual = ep.residual;
  A.status = status;
  return dtype == LAQ_BF16 ? launch_form<__nv_bfloat16>(e, pl, out32, long_sum, ma, mb, A, follows, st)
                           : launch_form<__half>(e, pl, out32, long_sum, ma, mb, A, follows, st);
}

// Warps that share four columns: as many as fill the rounds of resident warps best, the fewer the better within a quarter
// (4096 x 4096, one row: two 7.4 us, four 8.2 us; 11008 x 4096: one 18.5 us, two 16.7 us).
int few_log_parts(long long groups, int items) {
  const long long resident = (long long)kFewThreads / 32 * kFewBlocks * kSMs;
  double best = 0.0;
  int pick = 0;
  for (int lp = 0; 1 << lp <= kFewThreads / 32 && (lp == 0 || items > 16 << lp); ++lp) {
    const long long warps = groups << lp, rounds = (warps + resident - 1) / resident;
    const double full = (double)warps / (double)(rounds * resident);
    if (full > 1.25 * best) {
      best = full;
      pick = lp;
    }
  }
  return pick;
}

template <class T, int ROWS>
laq_status launch_few(const Err& e, const GemmArgs& A, const Operand& x, const Operand& w, cudaStream_t st) {
  const int K = (int)x.cols, vec = x.mappable_() && w.mappable_(), items = vec ? K / 8 : K;
  const long long groups = (w.rows + kFewCols - 1) / kFewCols;
  const int log_parts = few_log_parts(groups, items), per_block = kFewThreads / 32 >> log_parts;
  const unsigned blocks = (unsigned)((groups + per_block - 1) / per_block);
  // Four vectors of each row of W under way where a lane has as many and the registers hold them (one row, 4096 x 4096: 7.4 us
  // against 8.7 us by two; 100000 x 512, where a lane has two: 26.7 us against 19.7 us).
  const auto kernel = ROWS <= 2 && items > 64 << log_parts ? linear_few_rows_kernel<T, ROWS, ROWS <= 2 ? 4 : 2> : linear_few_rows_kernel<T, ROWS, 2>;
  return launched(e.buf, e.len, launch_plain(kernel, dim3(blocks), kFewThreads, st, A, (const T*)x.p, x.ld, (const T*)w.p, w.ld, K, vec, log_parts));
}

template <class T>
laq_status few_rows(const Err& e, const Operand& x, const Operand& w, const Epilogue& ep, cudaStream_t st) {
  GemmArgs A = {};
  A.I = (int)x.rows;
  A.J = (int)w.rows;
  A.act = ep.act;
  A.out = ep.out;
  A.ldo = ep.ldo;
  A.z = ep.z;
  A.ldz = ep.ldz;
  A.bias = ep.bias;
  A.residual = ep.residual;
  A.ldr = ep.ldr;
  switch (x.rows) {
    case 1: return launch_few<T, 1>(e, A, x, w, st);
    case 2: return launch_few<T, 2>(e, A, x, w, st);
    case 3: return launch_few<T, 3>(e, A, x, w, st);
    default: return launch_few<T, 4>(e, A, x, w, st);
  }
}

// One or two rows always; three or four unless there are many short columns, where folding the sums costs more than the
// products (100000 x 512: 33 us, by the tensor cores 27 us).
bool takes_few_rows(const laq_linear_call* c) {
  if (c->flags & LAQ_LINEAR_STARVE) return false;
  return c->M <= 2 || (c->M <= kFewRows && (c->K >= 1024 || c->N <= kFewCols * kFewThreads / 32 * kFewBlocks * kSMs));
}

// Copies an operand that a tensor map cannot describe to `ws` (advanced past it).
laq_status make_mappable(const Err& e, Operand& o, char*& ws, cudaStream_t st) {
  const size_t bytes = o.pack_bytes();
  if (!bytes) return LAQ_OK;
  const long long pitch = pad8(o.cols), items = o.rows * (pitch / 8);
  const long long want = (items + 255) / 256, most = 8 * kSMs;
  const laq_status st_ = launched(e.buf, e.len, launch_plain(linear_pack_kernel, dim3((unsigned)(want < most ? want : most)), 256, st,
                                                             (const uint16_t*)o.p, o.ld, (uint16_t*)ws, pitch, o.rows, (int)o.cols));
  if (st_ != LAQ_OK) return st_;
  o.p = ws;
  o.ld = pitch;
  ws += bytes;
  return LAQ_OK;
}

bool sizes_ok(const laq_linear_call* c) {
  const long long most = 0x7fffff00ll;
  return c && c->M >= 0 && c->M <= most && c->N >= 1 && c->N <= most && c->K >= 1 && c->K <= most &&
         (c->dtype == LAQ_BF16 || c->dtype == LAQ_F16);
}

int dz_rows_per(long long M, long long N) {
  // enough blocks for four an SM, no fewer than 32 rows each, and no more than 65535 runs (a grid dimension)
  const long long cols = (N + kDzCols - 1) / kDzCols;
  long long runs = (4 * kSMs + cols - 1) / cols;
  long long per = (M + runs - 1) / runs;
  per = per < 32 ? 32 : per;
  while ((M + per - 1) / per > 65535) per *= 2;
  return (int)per;
}

// What the gradient keeps in the workspace: dZ (unless dY itself serves), the column sums' partials, packed operands.
struct BackwardNeeds {
  bool own_dz;
  size_t dz_bytes, part_bytes;
  Operand x, w, dz;
  explicit BackwardNeeds(const laq_linear_call* c) {
    const Operand dy{c->dy, c->ld_dy, c->M, c->N};
    own_dz = (c->dx || c->dw) && (c->activation != LAQ_ACT_NONE || !dy.mappable_());
    dz_bytes = own_dz ? align256((size_t)c->M * pad8(c->N) * 2) : 0;
    const int per = dz_rows_per(c->M, c->N);
    part_bytes = c->db ? align256((size_t)((c->M + per - 1) / per) * c->N * 4) : 0;
    x = Operand{c->x, c->ld_x, c->M, c->K};
    w = Operand{c->w, c->ld_w, c->N, c->K};
    dz = dy;
  }
  size_t bytes(const laq_linear_call* c) const {
    return dz_bytes + part_bytes + (c->dw ? x.pack_bytes() : 0) + (c->dx ? w.pack_bytes() : 0);
  }
};

laq_status check_call(const Err& e, const laq_linear_call* c, void* ws, size_t ws_bytes, size_t need) {
  if (e.buf && e.len) e.buf[0] = 0;
  if (!c) return fail(e.buf, e.len, LAQ_EINVAL, "null pointer");
  if (c->dtype != LAQ_BF16 && c->dtype != LAQ_F16) return fail(e.buf, e.len, LAQ_EINVAL, "dtype must be LAQ_BF16 or LAQ_F16");
  if (!sizes_ok(c)) return fail(e.buf, e.len, LAQ_EINVAL, "M must be 0..2^31-256, N and K 1..2^31-256");
  if (c->activation < LAQ_ACT_NONE || c->activation > LAQ_ACT_SILU) return fail(e.buf, e.len, LAQ_EINVAL, "unknown activation");
  if (!c->status) return fail(e.buf, e.len, LAQ_EINVAL, "status must point to a word of device memory");
  if (need && (!ws || ((uintptr_t)ws & 255u) || ws_bytes < need))
    return fail(e.buf, e.len, LAQ_EWORKSPACE, "workspace missing, misaligned (256 bytes) or too small: %zu bytes needed", need);
  if (c->flags & ~(uint32_t)LAQ_LINEAR_STARVE) return fail(e.buf, e.len, LAQ_EINVAL, "unknown flags");
  return LAQ_OK;
}

// One tensor of a call: there if it must be, rows no shorter than their length.  It is added to the buffers.
enum Access { kRead, kWritten };
laq_status check_tensor(const Err& e, Buffers& buffers, const char* name, Access access, const void* p, bool required, int64_t rows, int64_t ld,
                        int64_t cols, int bytes, const char* in_place = "") {
  if (!p) return required ? fail(e.buf, e.len, LAQ_EINVAL, "%s is null", name) : LAQ_OK;
  if (ld < cols) return fail(e.buf, e.len, LAQ_EINVAL, "the row stride of %s is shorter than its rows", name);
  if (access == kWritten) buffers.out(name, p, bytes, rows, cols, ld, in_place);
  else buffers.in(name, p, bytes, rows, cols, ld);
  return LAQ_OK;
}

#define LAQ_TRY(call)                \
  do {                               \
    const laq_status st_ = (call);   \
    if (st_ != LAQ_OK) return st_;   \
  } while (0)

template <class T>
void list_kernels(const void** list, int& n) {
  const void* all[] = {
      (const void*)linear_gemm_kernel<T, false, false, false, false>, (const void*)linear_gemm_kernel<T, true, false, false, false>,
      (const void*)linear_gemm_kernel<T, false, true, false, false>,  (const void*)linear_gemm_kernel<T, false, false, false, true>,
      (const void*)linear_gemm_kernel<T, true, false, false, true>,   (const void*)linear_gemm_kernel<T, false, true, false, true>,
      (const void*)linear_gemm_kernel<T, false, false, true, false>,  (const void*)linear_gemm_kernel<T, false, true, true, false>,
      (const void*)linear_few_rows_kernel<T, 1, 4>, (const void*)linear_few_rows_kernel<T, 1, 2>, (const void*)linear_few_rows_kernel<T, 2, 4>,
      (const void*)linear_few_rows_kernel<T, 2, 2>, (const void*)linear_few_rows_kernel<T, 3, 2>, (const void*)linear_few_rows_kernel<T, 4, 2>,
      (const void*)linear_dz_kernel<T>};
  for (const void* k : all) list[n++] = k;
}

laq_status load_kernels(const Err& e) {
  static Loaded loaded;
  static const void* list[32];
  static const int n = [] {
    int count = 0;
    list_kernels<__nv_bfloat16>(list, count);
    list_kernels<__half>(list, count);
    list[count++] = (const void*)linear_db_kernel;
    list[count++] = (const void*)linear_pack_kernel;
    return count;
  }();
  return launched(e.buf, e.len, loaded.once(list, n));
}

}  // namespace
}  // namespace ops
}  // namespace laq

using namespace laq::ops;

extern "C" size_t laq_linear_workspace_bytes(const laq_linear_call* c, int32_t backward) {
  if (!sizes_ok(c)) return 0;
  if (backward) return BackwardNeeds(c).bytes(c);
  if (takes_few_rows(c)) return 0;
  return Operand{c->x, c->ld_x, c->M, c->K}.pack_bytes() + Operand{c->w, c->ld_w, c->N, c->K}.pack_bytes();
}

extern "C" laq_status laq_linear_forward(const laq_linear_call* c, void* d_workspace, size_t workspace_bytes, void* cuda_stream,
                                         char* errbuf, size_t errbuf_len) {
  const Err e{errbuf, errbuf_len};
  const size_t need = laq_linear_workspace_bytes(c, 0);
  LAQ_TRY(check_call(e, c, d_workspace, workspace_bytes, need));
  if (c->M == 0) return LAQ_OK;
  Buffers buffers;
  buffers.out("status", c->status, 4, 1, 1, 1);
  if (need) buffers.out("the workspace", d_workspace, 1, 1, (long long)need, (long long)need);
  LAQ_TRY(check_tensor(e, buffers, "x", kRead, c->x, true, c->M, c->ld_x, c->K, 2));
  LAQ_TRY(check_tensor(e, buffers, "w", kRead, c->w, true, c->N, c->ld_w, c->K, 2));
  LAQ_TRY(check_tensor(e, buffers, "bias", kRead, c->bias, false, 1, c->N, c->N, 2));
  LAQ_TRY(check_tensor(e, buffers, "residual", kRead, c->residual, false, c->M, c->ld_residual, c->N, 2));
  LAQ_TRY(check_tensor(e, buffers, "y", kWritten, c->y, true, c->M, c->ld_y, c->N, 2, "residual"));
  LAQ_TRY(check_tensor(e, buffers, "z", kWritten, c->z, false, c->M, c->ld_z, c->N, 2));
  LAQ_TRY(buffers.check(errbuf, errbuf_len));
  LAQ_TRY(load_kernels(e));
  cudaStream_t st = (cudaStream_t)cuda_stream;
  char* ws = (char*)d_workspace;
  Operand x{c->x, c->ld_x, c->M, c->K}, w{c->w, c->ld_w, c->N, c->K};
  Epilogue ep;
  ep.out = c->y;
  ep.ldo = c->ld_y;
  ep.act = c->activation;
  ep.bias = c->bias;
  ep.residual = c->residual;
  ep.ldr = c->ld_residual;
  ep.z = c->z;
  ep.ldz = c->ld_z;
  if (takes_few_rows(c))
    return c->dtype == LAQ_BF16 ? few_rows<__nv_bfloat16>(e, x, w, ep, st) : few_rows<__half>(e, x, w, ep, st);
  LAQ_TRY(make_mappable(e, x, ws, st));
  LAQ_TRY(make_mappable(e, w, ws, st));
  return product(e, c->dtype, x, false, w, false, ep, c->status, (c->flags & LAQ_LINEAR_STARVE) != 0, true, ws != d_workspace,
                 st);
}

extern "C" laq_status laq_linear_backward(const laq_linear_call* c, void* d_workspace, size_t workspace_bytes, void* cuda_stream,
                                          char* errbuf, size_t errbuf_len) {
  const Err e{errbuf, errbuf_len};
  const size_t ws_bytes = laq_linear_workspace_bytes(c, 1);
  LAQ_TRY(check_call(e, c, d_workspace, workspace_bytes, ws_bytes));
  if (!c->dx && !c->dw && !c->db) return LAQ_OK;
  const bool act = c->activation != LAQ_ACT_NONE;
  const int dw_bytes = c->dw_dtype == LAQ_F32 ? 4 : 2;
  if (c->dw && c->dw_dtype != c->dtype && c->dw_dtype != LAQ_F32)
    return fail(errbuf, errbuf_len, LAQ_EINVAL, "dw_dtype must be the call's dtype or LAQ_F32");
  if (c->dw && c->dw_dtype == LAQ_F32 && act && c->activation != LAQ_ACT_RELU)
    return fail(errbuf, errbuf_len, LAQ_EINVAL,
                "dw in fp32 needs no activation or ReLU: with the others dZ is rounded to 16 bits before the product");
  Buffers buffers;
  buffers.out("status", c->status, 4, 1, 1, 1);
  if (ws_bytes) buffers.out("the workspace", d_workspace, 1, 1, (long long)ws_bytes, (long long)ws_bytes);
  LAQ_TRY(check_tensor(e, buffers, "dw", kWritten, c->dw, false, c->N, c->ld_dw, c->K, dw_bytes));
  LAQ_TRY(check_tensor(e, buffers, "db", kWritten, c->db, false, 1, c->N, c->N, 4));
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (c->M == 0) {               // sums over no rows
    LAQ_TRY(buffers.check(errbuf, errbuf_len));
    if (c->dw) LAQ_TRY(launched(errbuf, errbuf_len, cudaMemset2DAsync(c->dw, (size_t)c->ld_dw * dw_bytes, 0, (size_t)c->K * dw_bytes, (size_t)c->N, st)));
    if (c->db) LAQ_TRY(launched(errbuf, errbuf_len, cudaMemsetAsync(c->db, 0, (size_t)c->N * 4, st)));
    return LAQ_OK;
  }
  LAQ_TRY(check_tensor(e, buffers, "dy", kRead, c->dy, true, c->M, c->ld_dy, c->N, 2));
  if (act) LAQ_TRY(check_tensor(e, buffers, "z", kRead, c->z, true, c->M, c->ld_z, c->N, 2));
  if (c->dw) LAQ_TRY(check_tensor(e, buffers, "x", kRead, c->x, true, c->M, c->ld_x, c->K, 2));
  if (c->dx) LAQ_TRY(check_tensor(e, buffers, "w", kRead, c->w, true, c->N, c->ld_w, c->K, 2));
  LAQ_TRY(check_tensor(e, buffers, "dx", kWritten, c->dx, false, c->M, c->ld_dx, c->K, 2));
  LAQ_TRY(buffers.check(errbuf, errbuf_len));
  LAQ_TRY(load_kernels(e));
  BackwardNeeds need(c);
  char* ws = (char*)d_workspace;
  const bool starve = (c->flags & LAQ_LINEAR_STARVE) != 0;
  bool follows = false;                   // a kernel of this call was the last thing put on the stream
  if (need.own_dz || c->db) {
    void* dz = need.own_dz ? ws : nullptr;
    float* part = c->db ? (float*)(ws + need.dz_bytes) : nullptr;
    ws += need.dz_bytes + need.part_bytes;
    const int per = dz_rows_per(c->M, c->N), runs = (int)((c->M + per - 1) / per), N = (int)c->N;
    const dim3 grid((unsigned)((c->N + kDzCols - 1) / kDzCols), (unsigned)runs);
    const int vec_ok = mappable(c->dy, c->ld_dy) && (!act || mappable(c->z, c->ld_z));
    const auto launch_dz = [&](auto zero) {
      using T = decltype(zero);
      return launch_plain(linear_dz_kernel<T>, grid, kDzThreads, st, (const T*)c->dy, c->ld_dy, (const T*)c->z, c->ld_z, (T*)dz, pad8(c->N),
                          part, c->M, N, c->activation, per, vec_ok);
    };
    LAQ_TRY(launched(errbuf, errbuf_len, c->dtype == LAQ_BF16 ? launch_dz(__nv_bfloat16()) : launch_dz(__half())));
    follows = true;
    if (c->db) {
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3((unsigned)((c->N + 31) / 32));
      cfg.blockDim = dim3(1024);
      cfg.stream = st;
      cudaLaunchAttribute at[1];
      at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
      at[0].val.programmaticStreamSerializationAllowed = 1;
      cfg.attrs = at;
      cfg.numAttrs = 1;
      LAQ_TRY(launched(errbuf, errbuf_len, cudaLaunchKernelEx(&cfg, linear_db_kernel, (const float*)part, runs, N, c->db)));
    }
    if (need.own_dz) {
      need.dz.p = dz;
      need.dz.ld = pad8(c->N);
    }
  }
  if (c->dx) {
    const char* before = ws;
    LAQ_TRY(make_mappable(e, need.w, ws, st));
    follows = follows || ws != before;
    Epilogue ep;
    ep.out = c->dx;
    ep.ldo = c->ld_dx;
    LAQ_TRY(product(e, c->dtype, need.dz, false, need.w, true, ep, c->status, starve, true, follows, st));
    follows = true;
  }
  if (c->dw) {
    const char* before = ws;
    LAQ_TRY(make_mappable(e, need.x, ws, st));
    follows = follows || ws != before;
    Epilogue ep;
    ep.out = c->dw;
    ep.ldo = c->ld_dw;
    ep.out_f32 = c->dw_dtype == LAQ_F32;
    LAQ_TRY(product(e, c->dtype, need.dz, true, need.x, true, ep, c->status, starve, false, follows, st));
  }
  return LAQ_OK;
}
