// The product kernel of the layer operators (laq_ops_linear.cu, laq_ops_gated.cu, laq_ops_blocks.cu), the plan of its tiles, and
// what their host sides share.
//
// D[i][j] = sum_r A(i, r) B(j, r).  linear_gemm_kernel serves a layer's product, its gradient's two where each has a launch of its own, the
// gated block's with short or split sums, and the 8-bit product of some rows (transposed tiles); gradients_gemm_kernel (laq_ops_gradients.cu) both products of a
// gradient at once, codes_gemm_kernel (laq_ops_blocks.cu) the 8-bit product of more rows, gated_gemm_kernel (laq_ops_gated.cu) the gated block's with long sums, and without tensor memory linear_few_rows_kernel,
// linear_few_codes_kernel (laq_ops_blocks.cu) and linear_some_rows_kernel those of few rows.  An operand is "K-major" (the summed index r is
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
#pragma once

#include <cooperative_groups.h>

#include <atomic>
#include <type_traits>

#include "laq_ops.cuh"
#include "laq_umma_gemm.cuh"

namespace cg = cooperative_groups;

namespace laq {
namespace ops {

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
// results show it in long sums alone (and in numbers that fall on the other side of a rounding, which 8 bits show, so that the gated block
// has a kernel of its own where it is not split): 65536 terms lose 6e-5, an eighth of half a step of fp16, 2^20 would lose 8e-4.  Longer
// ones are added up in chunks of 16384 terms (1.6e-5), whose sums wait in the second accumulator's tensor memory, so that
// tiles may still be 256 wide: the tensor cores stand still for it for some 2000 cycles in a chunk's 180000.  (131072 rows, dW
// of 4096 x 1024 bf16: 866 us, without chunks 845 us, with the sums in registers and tiles of 128 columns 1505 us.)
constexpr int kChunk32 = 8, kChunkLong = 256;               // k-blocks
constexpr int kLongSum = 65536;           // terms that a 16-bit result takes at once
constexpr int kGroupTiles = 16;           // tile rows that are swept together, so that operands are found in L2

// What a product's operands are and what becomes of its tile.
enum Mode {
  kPlain,       // 16-bit operands
  kGated,       // 16-bit operands, B's rows are gates and then as many ups: a tile holds nt / 2 columns of each
  kCodes        // 8-bit operands with a scale for each block of 128 of the summed axis
};
constexpr int kScaleTable = 8 * 64;       // kCodes: scales that an epilogue warp has at hand
constexpr int kBlock = 128;               // columns (and, of weights, rows) that share a scale of 8-bit codes

struct GemmArgs {
  int I, J, nkb;                 // rows and columns of D; blocks of the summed axis, 64 wide (kCodes: 128)
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
// What the other modes have more.  A kernel is given no more than its mode needs: with all of it as arguments a layer's product, whose
// tiles ask for them again and again, was up to 6 % slower (9000 x 2304 x 400 37.3 us, so 39.7; 16 x 331 x 42 8.1, 8.4).
struct GatedArgs : GemmArgs {
  long long up;                  // rows of gates, so where the ups begin (columns of out)
  uint8_t* z_codes;              // z in 8 bits instead of z, or null: whole blocks of 128 columns, 8-byte aligned
  float* z_scales;
  long long ld_zc, ld_zs;
};
struct CodesArgs : GemmArgs {
  const float* sx;               // scales of X, [rows][blocks], and of W, [blocks of rows][blocks]
  const float* sw;
  long long ldsx, ldsw;
};
template <int MODE>
using ArgsOf = std::conditional_t<MODE == kGated, GatedArgs, std::conditional_t<MODE == kCodes, CodesArgs, GemmArgs>>;

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
// 8-bit codes (e4m3, 32 of the summed axis an instruction), for one block
__device__ __forceinline__ void mma_codes(uint32_t d_tmem, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n"
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
// Without a fence over the thread's other memory accesses: what is handed back has been read from tensor memory, which wait::ld and
// fence::before_thread_sync order.  (With one, which waits for the results
// that the thread has written, the 8-bit product of 8192 x 4096 x 4096 took half as long again.)
__device__ __forceinline__ void arrive_lightly(uint32_t cluster_bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
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
// Slopes, two numbers at a time.  s (1 - s) is 0 long before z^2 passes 400, so that GELU's stays finite however far z is.
__device__ __forceinline__ f32x2 times2(f32x2 a, f32x2 b) {      // mul2 without its flush of tiny products
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 both_of(float v) { return pair_of(v, v); }
__device__ __forceinline__ f32x2 sigmoid2(f32x2 x) {
  float a, b, ra, rb;
  split(add2(both_of(1.f), ex2x2(times2(both_of(-1.4426950408889634f), x))), a, b);
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(ra) : "f"(a));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(rb) : "f"(b));
  return pair_of(ra, rb);
}
__device__ __forceinline__ f32x2 one_minus2(f32x2 s) { return fma2(s, both_of(-1.f), both_of(1.f)); }
__device__ __forceinline__ f32x2 gelu_sigmoid2(f32x2 z) {
  return sigmoid2(times2(both_of(2.f * kGeluC), fma2(times2(times2(both_of(kGeluA), z), z), z, z)));
}
__device__ __forceinline__ f32x2 gelu_inner2(f32x2 z) {
  float a, b;
  split(times2(z, z), a, b);
  return fma2(both_of(6.f * kGeluC * kGeluA), pair_of(fminf(a, 400.f), fminf(b, 400.f)), both_of(2.f * kGeluC));
}
__device__ __forceinline__ f32x2 slope_silu2(f32x2 z) {
  const f32x2 s = sigmoid2(z);
  return times2(s, fma2(z, one_minus2(s), both_of(1.f)));
}
__device__ __forceinline__ f32x2 slope_gelu2(f32x2 z) {
  const f32x2 s = gelu_sigmoid2(z);
  return fma2(times2(times2(z, s), one_minus2(s)), gelu_inner2(z), s);
}

__device__ __forceinline__ float load_scale(const float* p) {      // where it stands, and not later
  float v;
  asm volatile("ld.global.nc.f32 %0, [%1];" : "=f"(v) : "l"(p));
  return v;
}

// The power of two k >= -126 with largest <= 448 2^k: 448 = 1.75 2^8.
__device__ __forceinline__ int scale_power(float largest) {
  const uint32_t b = __float_as_uint(largest);
  const int k = (int)(b >> 23) - 135 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return max(k, -126);
}
__device__ __forceinline__ float power_of_two(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }      // -126..127

__device__ __forceinline__ uint32_t encode2(float lo, float hi) {
  unsigned short two;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two) : "f"(hi), "f"(lo));
  return two;
}
__device__ __forceinline__ uint2 encode8_finite(const float (&x)[8], float inverse) {
  return make_uint2(encode2(x[0] * inverse, x[1] * inverse) | (encode2(x[2] * inverse, x[3] * inverse) << 16),
                    encode2(x[4] * inverse, x[5] * inverse) | (encode2(x[6] * inverse, x[7] * inverse) << 16));
}
// Eight codes of values times `inverse` (a power of two: exact); what is not finite becomes NaN, which e4m3 has and infinity not.
__device__ __forceinline__ uint2 encode8(const float (&x)[8], float inverse) {
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = fabsf(x[e]) < INFINITY ? x[e] * inverse : __uint_as_float(0x7fffffffu);
  return make_uint2(encode2(v[0], v[1]) | (encode2(v[2], v[3]) << 16), encode2(v[4], v[5]) | (encode2(v[6], v[7]) << 16));
}
// The largest finite magnitude of 32 values rounded to T; `finite` becomes false if one is no finite number.
template <class T>
__device__ __forceinline__ float largest_rounded(const float (&x)[32], bool& finite) {
  uint4 v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float part[8] = {x[8 * i], x[8 * i + 1], x[8 * i + 2], x[8 * i + 3], x[8 * i + 4], x[8 * i + 5], x[8 * i + 6], x[8 * i + 7]};
    v[i] = Elem<T>::pack(part);
    v[i].x &= 0x7fff7fffu, v[i].y &= 0x7fff7fffu, v[i].z &= 0x7fff7fffu, v[i].w &= 0x7fff7fffu;
  }
  float m = Elem<T>::largest(v);
  if (!(m < INFINITY)) {                     // some are not finite: one by one
    finite = false;
    m = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const float a = fabsf(Elem<T>::to_float(Elem<T>::from_float(x[i])));
      m = fmaxf(m, a < INFINITY ? a : 0.f);
    }
  }
  return m;
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
// The same of a gated block: h = act(gate + bias) (up + bias), gates and ups of A.up columns each, side by side in z and in bias.
template <class T>
__device__ __forceinline__ void finish_gated_column(const GatedArgs& A, int rows, int row0, int col, float (&g)[8], float (&u)[8]) {
  if (col >= A.up || row0 >= rows) return;
  const int n = min(8, rows - row0);
  const T* bias = reinterpret_cast<const T*>(A.bias);
  const float bg = bias ? Elem<T>::to_float(bias[col]) : 0.f, bu = bias ? Elem<T>::to_float(bias[A.up + col]) : 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    g[e] += bg;
    u[e] += bu;
  }
  if (A.z) {
    T* z = reinterpret_cast<T*>(A.z) + (long long)row0 * A.ldz + col;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) {
        z[e * A.ldz] = Elem<T>::from_float(g[e]);
        z[e * A.ldz + A.up] = Elem<T>::from_float(u[e]);
      }
  }
  activate(g, A.act);
  T* out = reinterpret_cast<T*>(A.out) + (long long)row0 * A.ldo + col;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < n) out[e * A.ldo] = Elem<T>::from_float(g[e] * u[e]);
}
template <class T>
__device__ __forceinline__ void finish_gated_row(const GatedArgs& A, int i, int j0, float (&g)[8], float (&u)[8], float inv_g = 0.f, float inv_u = 0.f,
                                                 bool finite = false) {
  if (i >= A.I || j0 >= A.up) return;              // vectors are allowed: A.up is a multiple of eight
  if (A.bias) {
    const T* bias = reinterpret_cast<const T*>(A.bias) + j0;
    float b[8];
    Elem<T>::unpack(__ldg(reinterpret_cast<const uint4*>(bias)), b);
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] += b[e];
    Elem<T>::unpack(__ldg(reinterpret_cast<const uint4*>(bias + A.up)), b);
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] += b[e];
  }
  if (A.z) {
    T* z = reinterpret_cast<T*>(A.z) + (long long)i * A.ldz + j0;
    *reinterpret_cast<uint4*>(z) = Elem<T>::pack(g);
    *reinterpret_cast<uint4*>(z + A.up) = Elem<T>::pack(u);
  }
  if (A.z_codes) {               // rounded to T first, as what is packed afterwards is
    uint8_t* z = A.z_codes + (long long)i * A.ld_zc + j0;
    float r[8];
    Elem<T>::unpack(Elem<T>::pack(g), r);
    *reinterpret_cast<uint2*>(z) = finite ? encode8_finite(r, inv_g) : encode8(r, inv_g);
    Elem<T>::unpack(Elem<T>::pack(u), r);
    *reinterpret_cast<uint2*>(z + A.up) = finite ? encode8_finite(r, inv_u) : encode8(r, inv_u);
  }
  activate(g, A.act);
#pragma unroll
  for (int e = 0; e < 8; ++e) g[e] *= u[e];
  *reinterpret_cast<uint4*>(reinterpret_cast<T*>(A.out) + (long long)i * A.ldo + j0) = Elem<T>::pack(g);
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

// The same of 32 rows of four 16-byte pieces.
__device__ __forceinline__ int narrow_piece(int row, int p) { return row * 4 + (p ^ ((row >> 1) & 3)); }

__device__ __forceinline__ bool aligned16(const void* p, long long ld_bytes) {
  return (((uintptr_t)p | (uintptr_t)ld_bytes) & 15u) == 0;
}

__device__ __forceinline__ bool all_vectors(const GemmArgs& A, bool out32) {
  return aligned16(A.out, A.ldo * (out32 ? 4 : 2)) && (!A.z || aligned16(A.z, A.ldz * 2)) &&
         (!A.residual || aligned16(A.residual, A.ldr * 2)) && (!A.bias || aligned16(A.bias, 0));
}

__device__ __forceinline__ bool all_vectors(const GatedArgs& A, bool out32) { return A.up % 8 == 0 && all_vectors(static_cast<const GemmArgs&>(A), out32); }

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

// kCodes (few rows of X, so transposed tiles alone): the tensor cores add up one block of 128, and the epilogue's threads add it, times
// its two scales, to sums in their registers while the next block is under way.
template <class T, bool TRANS, bool PAIR, bool OUT32, bool LONG, int MODE = kPlain>
__global__ void __launch_bounds__(kGemmThreads, 1) linear_gemm_kernel(const __grid_constant__ CUtensorMap tmA,
                                                                      const __grid_constant__ CUtensorMap tmB,
                                                                      const ArgsOf<MODE> A) {
  extern __shared__ unsigned char gemm_smem_raw[];
  __shared__ uint64_t bars[2 * kMaxStages + 5];
  __shared__ uint32_t tmem_base_sh;
  __shared__ int abort_sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t base = umma::smem_u32(gemm_smem_raw), smem0 = (base + 1023u) & ~1023u;
  uint4* ring4 = reinterpret_cast<uint4*>(gemm_smem_raw + (smem0 - base));        // a split tile, once the ring is idle
  static_assert(!(OUT32 && (LONG || TRANS)), "fp32 results have chunks of their own, and their epilogue writes rows");
  static_assert(MODE == kPlain || !(OUT32 || LONG), "the other modes have 16-bit results and no long sums");
  static_assert(MODE != kCodes || (TRANS && !PAIR), "8-bit tiles that are not transposed have a kernel of their own");
  constexpr int kChunk = MODE == kCodes ? 1 : OUT32 ? kChunk32 : LONG ? kChunkLong : 1 << 30;      // k-blocks that the tensor core adds up
  constexpr bool kSummed = OUT32 || MODE == kCodes;           // the epilogue's registers hold the sum of the chunks
  constexpr int kStageCols = MODE == kCodes ? kBlock : kBlockK;           // of the summed axis in a stage: 128 bytes
  const int nt = A.nt, stages = A.stages, split = PAIR ? 1 : A.split;
  // the tile is put together from shared memory: parts of the sum, or gates and ups that lie in different lanes
  const bool joined = split > 1 || (MODE == kGated && TRANS);
  const int b_rows = PAIR ? nt / 2 : nt;           // columns of the tile whose part of B this block loads
  const uint32_t a_bytes = kTileM * kBlockK * 2, st_bytes = a_bytes + (uint32_t)b_rows * kBlockK * 2;
  const int half = PAIR ? (int)(blockIdx.x & 1u) : 0;
  const uint32_t full0 = umma::smem_u32(&bars[0]), empty0 = umma::smem_u32(&bars[kMaxStages]);
  const uint32_t acc_full0 = umma::smem_u32(&bars[2 * kMaxStages]), acc_empty0 = acc_full0 + 16, drain = acc_full0 + 32;
  // Two accumulators of at most 256 columns; one for a split tile, which has no successor (two of at most 128 for the chunks
  // of an fp32 result).  A long sum's chunks all go to the first, their sum is in the second.  Two blocks of a cluster on one
  // SM must be able to hold theirs at the same time (each waits for the other), and two is all that fits by shared memory (one,
  // where a split long sum is more than 128 columns wide).
  const uint32_t acc_cols = umma::tmem_cols(nt), held_cols = joined && !kSummed && !LONG ? acc_cols : 2 * acc_cols;
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
        // a pair's second block brings the upper half of the columns: of a gated tile the ups
        if constexpr (MODE == kGated && !TRANS) j0 = j0 / 2 + half * (int)A.up;
        else j0 += half * b_rows;
        for (int kb = 0; kb < nkb; ++kb, ++n) {
          const int s = n % stages;
          ok = umma::mbar_wait_abortable(empty0 + 8 * s, ((uint32_t)(n / stages) & 1u) ^ 1u, limit, abort_flag, A.status, 1u);
          if (!ok) break;
          const uint32_t sa = smem0 + s * st_bytes, sb = sa + a_bytes;
          const int r = (kb0 + kb) * kStageCols;
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
          } else if constexpr (MODE == kGated && TRANS) {      // 64 gates and their ups
            umma::tma_load_2d(sa, &tmA, bar, r, i0 / 2);
            umma::tma_load_2d(sa + 8192, &tmA, bar, r, i0 / 2 + (int)A.up);
          } else {
            umma::tma_load_2d(sa, &tmA, bar, r, i0);
          }
          if (A.b_mn) {
            for (int b = 0; b < nt; b += 64) umma::tma_load_2d(sb + b * 128, &tmB, bar, j0 + b, r);
          } else if constexpr (MODE == kGated && !TRANS) {
            umma::tma_load_2d(sb, &tmB, bar, r, j0);
            umma::tma_load_2d(sb + nt / 2 * 128, &tmB, bar, r, j0 + (int)A.up);
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
            for (int kk = 0; kk < kBlockK / 16; ++kk) {          // 32 bytes of the summed axis: 16 values, or 32 codes
              const uint32_t more = kb != k0 || kk != 0 ? 1u : 0u;
              if (MODE == kCodes) mma_codes(d, da + kk * step_a, db + kk * step_b, idesc, more);
              else if (PAIR) mma_pair(d, da + kk * step_a, db + kk * step_b, idesc, more);
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
      const bool whole = !TRANS && MODE != kGated && split == 1 && vec && i0 + kTileM <= A.I && j0 + nt <= A.J && nt % 32 == 0;
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
      constexpr int kSums = OUT32 ? 2 : MODE == kCodes ? 4 : 1, kWide = MODE == kCodes ? 16 : 32;
      float sum[kSums][kWide];                         // the chunks' sums, this lane's row
      if constexpr (MODE == kCodes) {
#pragma unroll
        for (int p = 0; p < kSums; ++p)
#pragma unroll
          for (int e = 0; e < kWide; ++e) sum[p][e] = 0.f;
        // The scales of eight blocks of 128 at a time, of this warp's columns (rows of X) times those of W's tile: read while the eight
        // before are added, put down in shared memory, and taken from there by all lanes.  (One block's read ahead by its lanes and
        // handed round by shuffles: 128 x 4096 x 4096 in tiles of 64 rows of X and halves of the sum 20.7 us, so 17.9.)
        float* table = reinterpret_cast<float*>(ring4 + (size_t)stages * st_bytes / 16) + (warp - 2) * kScaleTable;
        float of_x[kSums][4], of_w;
        const int at = (lane & 1) * 4;                 // a lane has four blocks' of one column of each 16
        const auto read_scales = [&](int k0) {
          of_w = lane < 8 && k0 + lane < nkb ? load_scale(A.sw + (long long)(i0 / kBlock) * A.ldsw + kb0 + k0 + lane) : 0.f;
#pragma unroll
          for (int p = 0; p < kSums; ++p) {
            const float* from = A.sx + (long long)min(j0 + 16 * set + 32 * p + (lane >> 1), A.J - 1) * A.ldsx + kb0 + k0 + at;
#pragma unroll
            for (int k = 0; k < 4; ++k) of_x[p][k] = 16 * set + 32 * p < nt && k0 + at + k < nkb ? load_scale(from + k) : 0.f;
          }
        };
        read_scales(0);
        for (int k0 = 0; k0 < nkb; ++k0) {
          if (k0 % 8 == 0) {
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float w8 = __shfl_sync(0xffffffffu, of_w, at + k);
#pragma unroll
              for (int p = 0; p < kSums; ++p) table[(at + k) * 64 + 16 * p + (lane >> 1)] = of_x[p][k] * w8;
            }
            __syncwarp();
            if (k0 + 8 < nkb) read_scales(k0 + 8);
          }
          acquire();
          if (!ok) break;
#pragma unroll
          for (int p = 0; p < kSums; ++p)
            if (16 * set + 32 * p < nt) {
              uint32_t v[kWide];
              tmem_load(t0 + (uint32_t)(16 * set + 32 * p), v);
              const float4* s4 = reinterpret_cast<const float4*>(table + (k0 % 8) * 64 + 16 * p);
#pragma unroll
              for (int e = 0; e < kWide; e += 4) {
                const float4 f = s4[e / 4];
                sum[p][e] = fmaf(__uint_as_float(v[e]), f.x, sum[p][e]);
                sum[p][e + 1] = fmaf(__uint_as_float(v[e + 1]), f.y, sum[p][e + 1]);
                sum[p][e + 2] = fmaf(__uint_as_float(v[e + 2]), f.z, sum[p][e + 2]);
                sum[p][e + 3] = fmaf(__uint_as_float(v[e + 3]), f.w, sum[p][e + 3]);
              }
            }
          release();
        }
        if (!ok) break;
      } else if constexpr (OUT32) {
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
        if constexpr (MODE == kCodes) {
          const int p = c0 / (2 * kWide);          // chosen so that the sums stay in registers
#pragma unroll
          for (int e = 0; e < kWide && e < (int)(sizeof(v) / 4); ++e)
            v[e] = __float_as_uint(p == 0 ? sum[0][e] : p == 1 ? sum[1][e] : p == 2 ? sum[2][e] : sum[3][e]);
          return;
        }
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
      // ... through shared memory
      auto hand_over = [&](int c0) {
        uint32_t v[32];
        values(c0, v);
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 32; e += 4) stage4[piece(lane, e / 4, 8)] = make_uint4(v[e], v[e + 1], v[e + 2], v[e + 3]);
        __syncwarp();
      };
      if (split > 1 && kSummed && !TRANS) {
        for (int c0 = 32 * set; c0 < nt; c0 += 64) {
          uint32_t v[32];
          values(c0, v);
#pragma unroll
          for (int e = 0; e < 32; e += 4)
            ring4[piece(row, (c0 + e) / 4, nt / 4)] = make_uint4(v[e], v[e + 1], v[e + 2], v[e + 3]);
        }
      } else if (joined) {
        for (int c0 = 16 * set; c0 < nt; c0 += 32) {
          uint32_t v[16];
          loaded(c0, v);
#pragma unroll
          for (int e = 0; e < 16; e += 4)
            ring4[piece(row, (c0 + e) / 4, nt / 4)] = make_uint4(v[e], v[e + 1], v[e + 2], v[e + 3]);
        }
      } else if constexpr (MODE == kGated) {
        // 32 gates and their ups of 32 rows, handed over as below
        for (int c0 = 32 * set; c0 < nt / 2; c0 += 64) {
          float gu[2][4][8];
#pragma unroll
          for (int part = 0; part < 2; ++part) {
            hand_over(c0 + part * (nt / 2));
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              float (&x)[8] = gu[part][k];
              if (vec) {
                const int r = 8 * k + (lane >> 2);
                const uint4 lo = stage4[piece(r, 2 * (lane & 3), 8)], hi = stage4[piece(r, 2 * (lane & 3) + 1, 8)];
                x[0] = __uint_as_float(lo.x), x[1] = __uint_as_float(lo.y), x[2] = __uint_as_float(lo.z), x[3] = __uint_as_float(lo.w);
                x[4] = __uint_as_float(hi.x), x[5] = __uint_as_float(hi.y), x[6] = __uint_as_float(hi.z), x[7] = __uint_as_float(hi.w);
              } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                  x[e] = __uint_as_float(reinterpret_cast<const uint32_t*>(&stage4[piece(8 * k + e, lane >> 2, 8)])[lane & 3]);
              }
            }
          }
          const int i = i0 + q * 32, j = j0 / 2 + c0;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (vec) finish_gated_row<T>(A, i + 8 * k + (lane >> 2), j + 8 * (lane & 3), gu[0][k], gu[1][k]);
            else finish_gated_column<T>(A, A.I, i + 8 * k, j + lane, gu[0][k], gu[1][k]);
          }
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
          hand_over(c0);
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
          hand_over(c0);
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
      if (!kSummed) release();
    }
  }
  if (joined) {             // one tile per cluster: its blocks share the columns of the join
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
      if constexpr (MODE == kGated) {
        // eight rows (or, with vectors, columns) of gates and of the ups that lie 64 lanes, or half a tile's columns, on
        const auto parts_of = [&](int r0, int g, float (&x)[8]) {
          uint4 lo[kMaxSplit], hi[kMaxSplit];               // all blocks' parts on their way at once, added in order
#pragma unroll
          for (int r = 0; r < kMaxSplit; ++r)
            if (r < split) {
              const uint4* p = cluster.map_shared_rank(ring4, r);
              lo[r] = p[piece(r0, 2 * g, nt / 4)];
              hi[r] = p[piece(r0, 2 * g + 1, nt / 4)];
            }
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = 0.f;
#pragma unroll
          for (int r = 0; r < kMaxSplit; ++r)
            if (r < split) {
              x[0] += __uint_as_float(lo[r].x), x[1] += __uint_as_float(lo[r].y), x[2] += __uint_as_float(lo[r].z), x[3] += __uint_as_float(lo[r].w);
              x[4] += __uint_as_float(hi[r].x), x[5] += __uint_as_float(hi[r].y), x[6] += __uint_as_float(hi[r].z), x[7] += __uint_as_float(hi[r].w);
            }
        };
        float gate[8], up[8];
        if (TRANS) {
          for (int item = rank * 256 + tid; item < 64 * groups && !gone; item += 256 * split) {
            const int r0 = item % 64, g = item / 64;
            parts_of(r0, g, gate);
            parts_of(r0 + 64, g, up);
            finish_gated_column<T>(A, A.J, j0 + g * 8, i0 / 2 + r0, gate, up);
          }
        } else if (vec) {
          for (int item = rank * 256 + tid; item < kTileM * groups / 2 && !gone; item += 256 * split) {
            const int r0 = item / (groups / 2), g = item % (groups / 2);
            parts_of(r0, g, gate);
            parts_of(r0, g + groups / 2, up);
            finish_gated_row<T>(A, i0 + r0, j0 / 2 + g * 8, gate, up);
          }
        } else {
          for (int item = rank * 256 + tid; item < kTileM / 8 * (nt / 2) && !gone; item += 256 * split) {
            const int r0 = item / (nt / 2) * 8, c = item % (nt / 2);
#pragma unroll
            for (int e = 0; e < 8; ++e) gate[e] = up[e] = 0.f;
            for (int r = 0; r < split; ++r) {
              const uint4* p = cluster.map_shared_rank(ring4, r);
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                gate[e] += reinterpret_cast<const float*>(p + piece(r0 + e, c >> 2, nt / 4))[c & 3];
                up[e] += reinterpret_cast<const float*>(p + piece(r0 + e, (c + nt / 2) >> 2, nt / 4))[c & 3];
              }
            }
            finish_gated_column<T>(A, A.I, i0 + r0, j0 / 2 + c, gate, up);
          }
        }
      } else if (TRANS || vec) {
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

// N sums over a warp's lanes: s[0] of lane i is the one of number i / (32 / N).  Each step halves the values that a lane holds.
template <int N>
__device__ __forceinline__ void fold(float (&s)[N], int lane) {
  int o = 16;
#pragma unroll
  for (int n = N / 2; n > 0; n /= 2, o /= 2) {              // lanes with bit o keep the upper half of the sums
    const bool upper = lane & o;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float other = __shfl_xor_sync(0xffffffffu, upper ? s[i] : s[i + n], o);
      s[i] = (upper ? s[i + n] : s[i]) + other;
    }
  }
#pragma unroll
  for (; o > 0; o /= 2) s[0] += __shfl_xor_sync(0xffffffffu, s[0], o);
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
// GATED: a warp's four rows of W are two gates and their ups.
template <class T, int ROWS, int AHEAD, bool GATED = false>
__global__ void __launch_bounds__(kFewThreads, ROWS <= 2 && AHEAD == 2 ? kFewBlocks + 2 : kFewBlocks)
    linear_few_rows_kernel(const ArgsOf<GATED ? kGated : kPlain> A, const T* x, long long ldx, const T* w, long long ldw, int K, int vec, int log_parts) {
  constexpr int kOwn = GATED ? kFewCols / 2 : kFewCols;          // columns of the result that a warp has
  constexpr int kRows2 = ROWS == 3 ? 4 : ROWS, kSums = kFewCols * kRows2, kWarps = kFewThreads / 32;
  __shared__ float part[kWarps][kSums];
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5, parts = 1 << log_parts;
  const int col0 = (int)(blockIdx.x * (unsigned)(kWarps >> log_parts)) * kOwn;
  const int first = (warp & (parts - 1)) * 32 + lane, step = 32 << log_parts;
  long long up = 0;
  if constexpr (GATED) up = A.up;
  const T* wr[kFewCols];
#pragma unroll
  for (int c = 0; c < kFewCols; ++c) wr[c] = w + (min(col0 + (warp >> log_parts) * kOwn + c % kOwn, A.J - 1) + c / kOwn * up) * ldw;
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
  fold(s, lane);
  if (lane % (32 / kSums) == 0) part[warp][lane / (32 / kSums)] = s[0];
  __syncthreads();
  if constexpr (GATED) {
    if (t < kOwn * kWarps >> log_parts) {
      float g[8] = {}, u[8] = {};
      for (int i = 0; i < parts; ++i)
#pragma unroll
        for (int m = 0; m < ROWS; ++m) {
          const float* p = part[(t / kOwn << log_parts) + i];
          g[m] += p[t % kOwn * kRows2 + m];
          u[m] += p[(kOwn + t % kOwn) * kRows2 + m];
        }
      finish_gated_column<T>(A, A.I, 0, col0 + t, g, u);
    }
  } else if (t < kFewCols * kWarps >> log_parts) {
    float y[8] = {};
    for (int i = 0; i < parts; ++i)
#pragma unroll
      for (int m = 0; m < ROWS; ++m) y[m] += part[(t / kFewCols << log_parts) + i][t % kFewCols * kRows2 + m];
    finish_column<T, false>(A, A.I, A.J, 0, col0 + t, y);
  }
}

// ---- host -----------------------------------------------------------------------------------------------------------------
inline size_t align256(size_t x) { return (x + 255) / 256 * 256; }
inline long long pad8(long long x) { return (x + 7) / 8 * 8; }
inline bool mappable(const void* p, long long ld) { return ((uintptr_t)p & 15u) == 0 && (ld % 8) == 0; }

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

constexpr int kCodesRing = 160 * 1024;       // of the 8-bit product's kernel
constexpr int kWideCodesStages = 4;          // of its tiles of 256 columns, which have results of 64 KB beside the ring

// Tile width, split, pairs and orientation by an estimate of the time in SM cycles, whose constants were fitted to all of
// these forms measured on 26 products (1 to 16384 rows): a stage costs the larger of its products (2.7 cycles per column of
// the tile, 2 at the tensor pipe's rate) and of its bytes (60 a cycle); a tile's epilogue 2000 and 9 per column, 45 where it
// writes element by element; the epilogue of one tile runs beside the products of the next.  A pair's start costs 4500
// more; the join of a split 6500 and 25 per column, and clusters of four and eight reach 136 and 128 SMs.  The form chosen by
// it is within 3 % of the fastest in 22 of the 26 and at most 25 % slower in the others.
// The other modes' constants are fitted to all of their forms on 18 and 19 products each, and count a launch's 10000 cycles, which the
// transposed and split forms, whose blocks take one tile each, have in every wave.
// `swappable`: the epilogue may write the transposed tile.  `whole`: no split.  An fp32 result's tile is a multiple of 64 wide (its operands are
// MN-major).
inline Plan make_plan(long long I, long long J, long long R, bool a_mn, bool b_mn, bool swappable, bool out32, bool long_sum, Mode mode = kPlain,
                      bool whole = false) {
  Plan best{0, 128, 1, 4, 0, 1e300};
  const int stage_cols = mode == kCodes ? kBlock : kBlockK;
  const long long nkb = (R + stage_cols - 1) / stage_cols;
  const auto persistent = [](double waves, double main, double epi) {
    return waves * (main > epi ? main : epi) + 0.1 * (main > epi ? epi : main) + epi;
  };
  for (int swap = 0; swap <= (swappable ? 1 : 0); ++swap) {
    const long long i = swap ? J : I, j = swap ? I : J;
    const long long rows = (i + kTileM - 1) / kTileM, row_pairs = (rows + 1) / 2;
    const bool bmn = swap ? a_mn : b_mn;
    static const int widths[] = {16, 32, 64, 96, 112, 128, 160, 192, 208, 224, 256};
    for (int nt : widths) {
      if (mode == kCodes && !swap && nt == 256 && rows > 1) {          // pairs alone have tiles of 256 columns
        const double cost = 10000 + (double)((row_pairs * ((j + nt - 1) / nt) + kSMs / 2 - 1) / (kSMs / 2)) * (nkb * 900.0 + 6000);
        if (cost < best.cost) best = Plan{0, nt, 1, kWideCodesStages, 1, cost};
      }
      if (bmn && nt % 64) continue;
      if (mode == kGated && !swap && nt % 64) continue;          // pieces of 32 gates and as many ups
      if (mode == kCodes && !swap && nt != 128 && nt != 64) continue;
      if ((swap || out32) && nt > 128) continue;     // fp32 results: 64 sums a thread
      const double mma = 2.7 * nt, epi = 2000 + (swap ? 45.0 : 9.0) * nt;
      const int stage = (kTileM + nt) * kBlockK * 2;
      const double per = mma > stage / 60.0 ? mma : stage / 60.0;
      const long long cols = (j + nt - 1) / nt, tiles = rows * cols;
      for (int log2 = 0; log2 <= (whole ? 0 : 3); ++log2) {
        const int split = 1 << log2;
        const bool joined = split > 1 || (mode == kGated && swap);
        const long long kb = (nkb + split - 1) >> log2;
        if (mode == kCodes && !swap && split > 1) continue;          // transposed tiles alone are split
        if (split > 1 && kb * (split - 1) >= nkb) continue;           // a block would have nothing to do
        int stages = (joined ? 110 * 1024 : mode == kCodes && !swap ? kCodesRing : kMaxRing) / stage;
        if (stages > kMaxStages) stages = kMaxStages;
        if (joined)                                                    // the partial tile in the ring
          while (stages * stage < kTileM * nt * 4 || stages < 3) ++stages;
        if (stages * stage > kMaxRing) continue;
        // A split long sum of more than 128 columns holds all of an SM's tensor memory: only where no other split tile's block
        // (84 KB of ring at least, at 96 columns) fits beside it, since blocks of two calls could otherwise keep one another from
        // the clusters that they wait for.  256 columns (144 KB) remain.
        if (split > 1 && long_sum && nt > 128 && stages * stage <= 136 * 1024) continue;
        const double main = kb * per;
        double cost;
        if (mode != kPlain && (swap || joined)) {
          const long long blocks = tiles << log2;
          const long long waves = split == 8 ? (blocks + 127) / 128 : split == 4 ? (blocks + 135) / 136 : (blocks + kSMs - 1) / kSMs;
          cost = waves * (mode == kCodes ? 13000 + 112.0 * nt + kb * (700.0 + nt) : swap ? 13500 + 95.0 * nt + kb * 450.0 : 16000 + 24.0 * nt + main);
        } else if (mode == kCodes) {
          cost = 10000 + (double)((tiles + kSMs - 1) / kSMs) * (nt == 64 ? kb * 820.0 + 1800 : kb * 930.0 + 3700);
        } else if (mode == kGated) {
          cost = 10000 + persistent((double)((tiles + kSMs - 1) / kSMs), main, epi);
        } else if (!joined) {
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
        int stages = (mode == kCodes ? kCodesRing : kMaxRing) / half;
        if (stages > kMaxStages) stages = kMaxStages;
        const double main = nkb * (mma > half / 60.0 ? mma : half / 60.0);
        const double waves = (double)((row_pairs * cols + kSMs / 2 - 1) / (kSMs / 2));
        const double cost = mode == kCodes ? 10000 + waves * (nkb * 790.0 + 4500) : (mode == kGated ? 14500 : 4500) + persistent(waves, main, epi);
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

// A product kernel's shared memory limit is raised once per device.
struct Raised {
  std::atomic<uint64_t> devices{0};
};
inline laq_status raise_shared_memory(const Err& e, const void* kernel, Raised& raised, int bytes = kMaxRing + kStaging + 1024) {
  int dev = 0;
  cudaGetDevice(&dev);
  const uint64_t bit = 1ull << (dev & 63);
  if (dev >= 64 || !(raised.devices.load(std::memory_order_acquire) & bit)) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) {
      cudaGetLastError();
      return fail(e.buf, e.len, LAQ_ECUDA, "shared memory of the product kernel was refused");
    }
    raised.devices.fetch_or(bit, std::memory_order_release);
  }
  return LAQ_OK;
}
// A kernel of maps and, last, the arguments that say how many tiles there are.
template <class Args, class... Maps>
laq_status launch_tiles(const Err& e, void (*kernel)(Maps..., const Args), Raised& raised, unsigned threads, bool pair, bool joined, int staging,
                        bool follows, cudaStream_t st, const Args& A, const Maps&... maps) {
  const size_t smem = (size_t)A.stages * (kTileM + (pair ? A.nt / 2 : A.nt)) * kBlockK * 2 + staging + 1024;
  const int per_tile = pair ? 2 : A.split;
  {
    const laq_status st_ = raise_shared_memory(e, (const void*)kernel, raised);
    if (st_ != LAQ_OK) return st_;
  }
  const long long tiles = (long long)A.tiles_i * A.tiles_j;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(pair ? 2 * (tiles < kSMs / 2 ? tiles : kSMs / 2) : joined ? tiles * A.split : tiles < kSMs ? tiles : kSMs));
  cfg.blockDim = dim3(threads);
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
  return launched(e.buf, e.len, cudaLaunchKernelEx(&cfg, kernel, maps..., A));
}

template <class T, bool TRANS, bool PAIR, bool OUT32, bool LONG, int MODE = kPlain>
laq_status launch_gemm(const Err& e, const CUtensorMap& ma, const CUtensorMap& mb, const ArgsOf<MODE>& A, bool follows,
                       cudaStream_t st) {
  static Raised raised;
  const bool joined = A.split > 1 || (MODE == kGated && TRANS);
  const int staging = MODE == kCodes ? kEpiWarps * kScaleTable * 4 : TRANS || A.split > 1 ? 0 : kStaging;
  return launch_tiles<ArgsOf<MODE>, CUtensorMap, CUtensorMap>(e, linear_gemm_kernel<T, TRANS, PAIR, OUT32, LONG, MODE>, raised, kGemmThreads, PAIR, joined,
                                                              staging, follows, st, A, ma, mb);
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

// A matrix whose rows a tensor map can describe: 16-byte address and pitch.
inline bool make_map(CUtensorMap* map, Mode mode, const void* p, long long rows, long long cols, long long ld, int box_rows) {
  if (mode != kCodes) return umma::make_map_bf16_2d(map, p, rows, cols, ld * 2, box_rows);
  const umma::EncodeTiledFn fn = umma::encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld};
  const cuuint32_t box[2] = {(cuuint32_t)kBlock, (cuuint32_t)box_rows}, estr[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// X W^T in one of the other modes, X [M][K] and W [N][K] of mappable rows (kGated: N = 2 up): the tensor maps, and what the plan says
// to the kernel, added to `A`, which brings the epilogue, the scales, the status and `up`.
template <Mode mode>
struct Product {
  Plan pl;
  CUtensorMap ma, mb;
  ArgsOf<mode> A;
};
template <Mode mode>
laq_status prepare_product(const Err& e, Product<mode>& p, const Operand& x, const Operand& w, int fmt) {
  const Plan& pl = p.pl = make_plan(x.rows, w.rows, x.cols, false, false, true, false, false, mode);
  const Operand &a = pl.swap ? w : x, &b = pl.swap ? x : w;
  const int a_rows = mode == kGated && pl.swap ? kTileM / 2 : kTileM;
  const int b_rows = pl.pair || (mode == kGated && !pl.swap) ? pl.nt / 2 : pl.nt;
  if (!make_map(&p.ma, mode, a.p, a.rows, a.cols, a.ld, a_rows) || !make_map(&p.mb, mode, b.p, b.rows, b.cols, b.ld, b_rows))
    return fail(e.buf, e.len, LAQ_ECUDA, "a tensor map was refused");
  const int stage_cols = mode == kCodes ? kBlock : kBlockK, tile_rows = pl.pair ? 2 * kTileM : kTileM;
  p.A.nkb = (int)((x.cols + stage_cols - 1) / stage_cols);
  p.A.nt = pl.nt;
  p.A.stages = pl.stages;
  p.A.split = pl.split;
  p.A.tiles_i = (int)((a.rows + tile_rows - 1) / tile_rows);
  p.A.tiles_j = (int)((b.rows + pl.nt - 1) / pl.nt);
  p.A.I = (int)a.rows;
  p.A.J = (int)b.rows;
  p.A.fmt = fmt;
  return LAQ_OK;
}

// Warps that share four columns: as many as fill the rounds of resident warps best, the fewer the better within a quarter
// (4096 x 4096, one row: two 7.4 us, four 8.2 us; 11008 x 4096: one 18.5 us, two 16.7 us).
inline int few_log_parts(long long groups, int items) {
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

// One tensor of a call: there if it must be, rows no shorter than their length.  It is added to the buffers.
enum Access { kRead, kWritten };
inline laq_status check_tensor(const Err& e, Buffers& buffers, const char* name, Access access, const void* p, bool required, int64_t rows, int64_t ld,
                        int64_t cols, int bytes, const char* in_place = "") {
  if (!p) return required ? fail(e.buf, e.len, LAQ_EINVAL, "%s is null", name) : LAQ_OK;
  if (ld < cols) return fail(e.buf, e.len, LAQ_EINVAL, "the row stride of %s is shorter than its rows", name);
  if (access == kWritten) buffers.out(name, p, bytes, rows, cols, ld, in_place);
  else buffers.in(name, p, bytes, rows, cols, ld);
  return LAQ_OK;
}

#define LAQ_TRY(...)                 \
  do {                               \
    const laq_status st_ = (__VA_ARGS__); \
    if (st_ != LAQ_OK) return st_;   \
  } while (0)

// Arguments that every call of a layer has.
inline laq_status check_layer(const Err& e, int dtype, long long M, long long N, long long K, int activation, const uint32_t* status, uint32_t flags,
                              const void* ws, size_t ws_bytes, size_t need) {
  const long long most = 0x7fffff00ll;
  if (dtype != LAQ_BF16 && dtype != LAQ_F16) return fail(e.buf, e.len, LAQ_EINVAL, "dtype must be LAQ_BF16 or LAQ_F16");
  if (M < 0 || M > most || N < 1 || N > most || K < 1 || K > most)
    return fail(e.buf, e.len, LAQ_EINVAL, "M must be 0..2^31-256, N and K 1..2^31-256");
  if (activation < LAQ_ACT_NONE || activation > LAQ_ACT_SILU) return fail(e.buf, e.len, LAQ_EINVAL, "unknown activation");
  if (!status) return fail(e.buf, e.len, LAQ_EINVAL, "status must point to a word of device memory");
  if (need && (!ws || ((uintptr_t)ws & 255u) || ws_bytes < need))
    return fail(e.buf, e.len, LAQ_EWORKSPACE, "workspace missing, misaligned (256 bytes) or too small: %zu bytes needed", need);
  if (flags & ~(uint32_t)LAQ_LINEAR_STARVE) return fail(e.buf, e.len, LAQ_EINVAL, "unknown flags");
  return LAQ_OK;
}

// Defined in laq_ops_linear.cu.
// D[i][j] = sum_r A(i, r) B(j, r): a_mn ? A is stored [r][i] : [i][r], the same for B.  Both are mappable.  `whole`: the sum is not
// split.  `follows`: the stream's last work is a kernel of the same call.
laq_status product(const Err& e, int dtype, const Operand& a, bool a_mn, const Operand& b, bool b_mn, const Epilogue& ep,
                   uint32_t* status, int starve, bool swappable, bool whole, bool follows, cudaStream_t st);
// Copies an operand that a tensor map cannot describe to `ws` (advanced past it).
laq_status make_mappable(const Err& e, Operand& o, char*& ws, cudaStream_t st);
// The products of a layer's gradient, dX = dZ W and dW = dZ^T X (each if asked for); operands that are not mappable are copied
// to `ws` (advanced past them).  `whole`: where one launch for both is the faster a product that is asked for by itself has its sum whole,
// as that launch has (128 x 1024 x 256: both 15 us, by two launches with split sums 24; dW of 4528 x 2576 x 64 by itself 41 us, split 28); else
// one launch is taken only where both products have whole sums anyway.
struct Gradients {
  void* dx;
  long long ld_dx;
  void* dw;
  long long ld_dw;
  int dw_f32;
};
// Whether one launch for both (16-bit results, dZ [M][N], K inputs) is the faster by the plans' estimates, and that launch.  It splits
// no sum; a result has the same bits whether the other is asked for or not, so that it is taken only where neither product would split
// its sum by itself, or (`whole`) where the caller has the sum of a product by itself whole, too.
bool both_pay(long long M, long long N, long long K, bool whole = false);
laq_status both_products(const Err& e, int dtype, const Operand& dz, const Operand& x, const Operand& w, const Gradients& to, uint32_t* status, int starve,
                         bool follows, cudaStream_t st);
void list_both_kernels(const void** list, int& n);
laq_status gradient_products(const Err& e, int dtype, const Operand& dz, Operand x, Operand w, const Gradients& to, char*& ws, uint32_t* status,
                             int starve, bool whole, bool follows, cudaStream_t st);
// db = the sums of the columns of part [runs][N]; follows a kernel of the same call.
laq_status column_sums(const Err& e, const float* part, int runs, int N, float* db, cudaStream_t st);
laq_status zero_gradients(const Err& e, const Gradients& to, float* db, long long N, long long K, cudaStream_t st);   // of no rows
laq_status load_layer_kernels(const Err& e);

// Defined in laq_ops_blocks.cu.
// The 8-bit matrix [rows][cols] in `dtype`, rows `pitch` elements apart.
laq_status unpack_blocks(const Err& e, const laq_blocks& b, long long rows, long long cols, int dtype, void* out, long long pitch, cudaStream_t st);
laq_status pack_blocks(const Err& e, const void* x, int dtype, long long rows, long long cols, long long ld, const laq_blocks& b, cudaStream_t st);
laq_status load_block_kernels(const Err& e);
// Adds an 8-bit matrix to a call's buffers: its codes by the first name, its scales by the second.
laq_status check_blocks(const Err& e, Buffers& buffers, const char* name, const char* scales_name, Access access, const laq_blocks* b, int64_t rows,
                        int64_t cols);

size_t blocks_forward_bytes(const laq_linear_call* c, const laq_blocks* x, const laq_blocks* w);     // workspace of the 8-bit product

inline long long blocks_across(long long cols) { return (cols + kBlock - 1) / kBlock; }

// An 8-bit matrix on the device, as a kernel reads it.
struct Codes {
  const uint8_t* p;
  long long ld;
  const float* scales;
  long long lds;
  int shift;                    // rows of a block: 1 << shift
  explicit Codes(const laq_blocks* b)
      : p(b ? (const uint8_t*)b->codes : nullptr), ld(b ? b->ld_codes : 0), scales(b ? b->scales : nullptr), lds(b ? b->ld_scales : 0),
        shift(b && b->block_rows == kBlock ? 7 : 0) {}
  bool vectors(int bytes) const { return ((uintptr_t)p % bytes) == 0 && ld % bytes == 0; }
  __device__ __forceinline__ float scale(long long row, long long col) const { return __ldg(scales + (row >> shift) * lds + col / kBlock); }
};

// Two e4m3 codes in fp32.
__device__ __forceinline__ float2 decode2(uint32_t two) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)two));
  return __half22float2(*reinterpret_cast<__half2*>(&h));
}
__device__ __forceinline__ void decode8(uint2 v, float scale, float (&x)[8]) {
  const uint32_t w[4] = {v.x & 0xffffu, v.x >> 16, v.y & 0xffffu, v.y >> 16};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = decode2(w[i]);
    x[2 * i] = f.x * scale;
    x[2 * i + 1] = f.y * scale;
  }
}
// The first n (1..8) of eight codes, or of eight 16-bit numbers, or (1..16) of sixteen codes, at any address of theirs: from the aligned
// words that hold them.  What lies behind the n-th is not theirs.  `edge`: those words may reach beyond the matrix, before its first row
// or behind its last, so that single bytes are read in their place.  Between rows they may reach up to three bytes beside a row, which are
// not used.  (With single bytes at both ends of every row the blocks there set the pace, 3001 x 2050: dZ 26 us for 14.)
// AT_ONCE: the single bytes are all on their way together, which takes registers: where one branch leads there for all of a thread's loads
// (dZ so 14.8 us, word by word 16.9; unpack_kernel, 8192 x 4096, so 41 us, word by word 33).
__host__ __device__ __forceinline__ uint32_t funnel(uint32_t lo, uint32_t hi, int bits) {      // bits 0..24
#ifdef __CUDA_ARCH__
  return __funnelshift_r(lo, hi, bits);
#else
  return (uint32_t)((((uint64_t)hi << 32) | lo) >> bits);
#endif
}
// Whether words may reach beyond a matrix: from one of its rows first..last, with so many numbers of `bytes` bytes before and behind the
// ones that are read in the row.
__host__ __device__ __forceinline__ bool at_edge(long long first, long long last, long long rows, long long before, long long behind, int bytes) {
  return (first == 0 && before < 4 / bytes - 1) || (last >= rows - 1 && behind < 4 / bytes - 1);
}
template <int BYTES, bool AT_ONCE>      // so many from p on, of which the first n are there
__host__ __device__ __forceinline__ void bytes_any(const uint8_t* p, int n, bool edge, uint32_t (&v)[BYTES / 4]) {
  if (AT_ONCE && edge) {
    uint32_t b[BYTES];
#pragma unroll
    for (int i = 0; i < BYTES; ++i) b[i] = i < n ? p[i] : 0u;
#pragma unroll
    for (int k = 0; k < BYTES / 4; ++k) v[k] = b[4 * k] | b[4 * k + 1] << 8 | b[4 * k + 2] << 16 | b[4 * k + 3] << 24;
    return;
  }
  const int off = (int)((uintptr_t)p & 3u);
  const uint8_t* first = p - off;
  uint32_t w[BYTES / 4 + 1];
  if (edge) {
#pragma unroll
    for (int k = 0; k <= BYTES / 4; ++k) {
      w[k] = 0u;
#pragma unroll
      for (int i = 4 * k; i < 4 * k + 4; ++i)
        if (first + i >= p && first + i < p + n) w[k] |= (uint32_t)first[i] << (8 * (i % 4));
    }
  } else {
#pragma unroll
    for (int k = 0; k <= BYTES / 4; ++k) w[k] = 4 * k < off + n ? reinterpret_cast<const uint32_t*>(first)[k] : 0u;
  }
#pragma unroll
  for (int k = 0; k < BYTES / 4; ++k) v[k] = funnel(w[k], w[k + 1], 8 * off);
}
template <bool AT_ONCE = false>
__host__ __device__ __forceinline__ uint2 load8_any(const uint8_t* p, int n, bool edge) {
  uint32_t v[2];
  bytes_any<8, AT_ONCE>(p, n, edge, v);
  return make_uint2(v[0], v[1]);
}
template <bool AT_ONCE = false>
__host__ __device__ __forceinline__ uint4 load16_codes_any(const uint8_t* p, int n, bool edge) {
  uint32_t v[4];
  bytes_any<16, AT_ONCE>(p, n, edge, v);
  return make_uint4(v[0], v[1], v[2], v[3]);
}
template <bool AT_ONCE = false, class T>
__host__ __device__ __forceinline__ uint4 load16_any(const T* p, int n, bool edge) {
  static_assert(sizeof(T) == 2, "16-bit numbers");
  return load16_codes_any<AT_ONCE>(reinterpret_cast<const uint8_t*>(p), 2 * n, edge);
}
// The first n of eight 16-bit numbers to any address of theirs.
template <class T>
__device__ __forceinline__ void store16_any(T* p, const uint4& v, int n) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  if (n == 8 && ((uintptr_t)p & 3u) == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) reinterpret_cast<uint32_t*>(p)[i] = w[i];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) reinterpret_cast<uint16_t*>(p)[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
  }
}
__device__ __forceinline__ uint2 load8(const void* p) {
  uint2 v;
  asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p) : "memory");
  return v;
}

// ---- some rows through a layer in 8 bits or a gated block ----------------------------------------------------------------
// Three to 32 rows: W's bytes are what has to be read, and a tile in tensor memory spends most of its time on the launch, the first loads
// and the join.  Here a warp takes 16 columns (or eight gates and their ups) and every parts-th block of 128 bytes of their rows, and
// multiplies with a warp's own matrix instructions; codes are decoded to fp16 for them, exactly, and a block's sums join the others by its
// scales, as elsewhere.  Which values a lane holds as its k-th is its own affair as long as both operands agree, so a lane takes 16
// neighbouring bytes.  A warp copies its blocks to shared memory by itself, some ahead, and a thread block goes on to its next columns
// without a pause.
// Codes, 4096 x 4096, 8, 16 and 32 rows: 7.2, 7.9 and 12.4 us (by tiles 11.9, 11.9, 12.7; four by plain dot products 10.1); 11008 x 4096,
// 8 rows 13.7 (21.6); 2048 x 4096 5.8 (19.1).  Gates and ups in 16 bits, 2 x 4096 x 4096, 8 and 16 rows: 14.5 and 16.6 us (by tiles 19.0,
// 18.8; 4.6 TB/s); 2 x 1024 x 1024 3.7 (15.9).  Bound by memory and, with codes, by decoding: fp8 operands in place of fp16 are slower
// (16 rows of 11008 x 4096 31 us for 21, before the copies made it 15.4).
constexpr int kSomeThreads = 256, kSomeWarps = kSomeThreads / 32, kSomePitch = 20, kRowBytes = 128;
__host__ __device__ constexpr int some_columns(bool codes) { return codes ? 16 : 8; }
template <int EIGHTS>
struct Some {
  static constexpr int kStages = EIGHTS == 1 ? 4 : 3, kPieces = 4 + 2 * EIGHTS, kBlocks = EIGHTS <= 2 ? 2 : 1;
  static constexpr int kRing = kSomeWarps * kStages * kPieces * 32 * 16;
};
template <class T>
__device__ __forceinline__ void mma_warp(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (std::is_same<T, __half>::value)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Four codes as fp16 numbers, exactly: the lower two and the upper two.
__device__ __forceinline__ void halves_of(uint32_t codes, uint32_t& lo, uint32_t& hi) {
  asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.rn.f16x2.e4m3x2 %0, a;\ncvt.rn.f16x2.e4m3x2 %1, b;\n}" : "=r"(lo), "=r"(hi) : "r"(codes));
}
// The first n of 16 bytes to shared memory, zeros behind them.
__device__ __forceinline__ void copy_piece(uint4* to, const uint8_t* from, long long n) {
  const int bytes = n >= 16 ? 16 : n > 0 ? (int)n : 0;
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(umma::smem_u32(to)), "l"(from), "r"(bytes) : "memory");
}
// CODES: 16 columns a warp, else eight gates and their ups; ldx, ldw and K in bytes.
template <class T, int EIGHTS, bool CODES>
__global__ void __launch_bounds__(kSomeThreads, Some<EIGHTS>::kBlocks)
    linear_some_rows_kernel(const ArgsOf<CODES ? kCodes : kGated> A, const uint8_t* x, long long ldx, const uint8_t* w, long long ldw, long long K, int log_parts, int sets) {
  constexpr int kStages = Some<EIGHTS>::kStages, kPieces = Some<EIGHTS>::kPieces, kOwn = some_columns(CODES);
  extern __shared__ uint4 some_ring[];
  __shared__ float sums[kSomeWarps][8 * EIGHTS * kSomePitch];
  allow_next();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, parts = 1 << log_parts, part = warp & (parts - 1);
  const int g = lane >> 2, t = lane & 3, per_set = kSomeWarps >> log_parts;
  uint4* ring = some_ring + warp * kStages * kPieces * 32;
  // A stage: rows of eight 16-byte pieces, 16 of W and then X's; every other row's halves are exchanged, so that neither the copies (a
  // row by eight lanes) nor the reads (two rows' halves by eight lanes) meet in a bank.
  const int from_row = lane >> 3, from_piece = lane & 7, to_piece = lane ^ (from_row & 1) << 2;
  const int at_s[2] = {8 * g + (t ^ (g & 1) << 2), 8 * g + ((t + 4) ^ (g & 1) << 2)};
  const int nkb = (int)((K + kRowBytes - 1) / kRowBytes);
  // where this warp's walk over sets of columns and blocks of 128 bytes is
  struct Place {
    int set, b;
  };
  const auto next = [&](Place& p) {
    p.b += parts;
    if (p.b >= nkb) p.b = part, p.set += (int)gridDim.x;
  };
  const auto column = [&](int set) { return (set * per_set + (warp >> log_parts)) * kOwn; };
  const auto fetch = [&](const Place& p, int stage) {
    if (p.set < sets) {
      uint4* to = ring + stage * kPieces * 32 + to_piece;
      const long long k = (long long)p.b * kRowBytes + 16 * from_piece, left = K - k;
      const int col = column(p.set) + from_row;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        long long row = min(col + 4 * (CODES ? i : i & 1), A.J - 1);
        if constexpr (!CODES) row += (i >> 1) * A.up;
        copy_piece(to + 32 * i, w + row * ldw + (left > 0 ? k : 0), left);
      }
#pragma unroll
      for (int i = 0; i < 2 * EIGHTS; ++i) {
        const bool there = left > 0 && 4 * i + from_row < A.I;
        copy_piece(to + 32 * (4 + i), there ? x + (long long)(4 * i + from_row) * ldx + k : x, there ? left : 0);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  float of_x[EIGHTS][2], of_w = 0.f;
  const auto read_scales = [&](const Place& p) {
    if constexpr (CODES) {
      if (p.set >= sets) return;
      of_w = __ldg(A.sw + (long long)(min(column(p.set), A.J - 1) / kBlock) * A.ldsw + p.b);        // 16 columns lie in one tile
#pragma unroll
      for (int f = 0; f < EIGHTS; ++f)
#pragma unroll
        for (int e = 0; e < 2; ++e) of_x[f][e] = __ldg(A.sx + min(8 * f + 2 * t + e, A.I - 1) * A.ldsx + p.b);
    }
  };
  Place fetched{part < nkb ? (int)blockIdx.x : sets, part}, read = fetched;        // a warp beyond the last block has nothing to fetch
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) {
    fetch(fetched, i);
    next(fetched);
  }
  read_scales(read);
  int stage = 0;
  for (int set = blockIdx.x; set < sets; set += gridDim.x) {
    float sum[EIGHTS][4] = {};
    for (int b = part; b < nkb; b += parts) {
      float scale[EIGHTS][2];
      if constexpr (CODES) {
#pragma unroll
        for (int f = 0; f < EIGHTS; ++f) scale[f][0] = of_x[f][0] * of_w, scale[f][1] = of_x[f][1] * of_w;
        next(read);
        read_scales(read);
      }
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
      __syncwarp();
      const uint4* at = ring + stage * kPieces * 32;
      fetch(fetched, stage == 0 ? kStages - 1 : stage - 1);
      next(fetched);
      stage = stage + 1 == kStages ? 0 : stage + 1;
      if constexpr (CODES) {
        float of_block[EIGHTS][4] = {};
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const uint4 v0 = at[at_s[s]], v1 = at[64 + at_s[s]];
          const uint32_t w0[4] = {v0.x, v0.y, v0.z, v0.w}, w1[4] = {v1.x, v1.y, v1.z, v1.w};
          uint32_t h0[4][2], h1[4][2];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            halves_of(w0[i], h0[i][0], h0[i][1]);
            halves_of(w1[i], h1[i][0], h1[i][1]);
          }
#pragma unroll
          for (int f = 0; f < EIGHTS; ++f) {
            const uint4 here = at[128 + 64 * f + at_s[s]];
            const uint32_t words[4] = {here.x, here.y, here.z, here.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t lo, hi;
              halves_of(words[i], lo, hi);
              mma_warp<__half>(of_block[f], h0[i][0], h1[i][0], h0[i][1], h1[i][1], lo, hi);
            }
          }
        }
#pragma unroll
        for (int f = 0; f < EIGHTS; ++f)
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[f][e] = fmaf(of_block[f][e], scale[f][e & 1], sum[f][e]);
      } else {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const uint4 v0 = at[at_s[s]], v1 = at[64 + at_s[s]];
#pragma unroll
          for (int f = 0; f < EIGHTS; ++f) {
            const uint4 here = at[128 + 64 * f + at_s[s]];
            mma_warp<T>(sum[f], v0.x, v1.x, v0.y, v1.y, here.x, here.y);
            mma_warp<T>(sum[f], v0.z, v1.z, v0.w, v1.w, here.z, here.w);
          }
        }
      }
    }
#pragma unroll
    for (int f = 0; f < EIGHTS; ++f)
#pragma unroll
      for (int e = 0; e < 4; ++e) sums[warp][(8 * f + 2 * t + (e & 1)) * kSomePitch + g + 8 * (e >> 1)] = sum[f][e];
    __syncthreads();
    for (int i = threadIdx.x; i < per_set * EIGHTS * kOwn; i += kSomeThreads) {
      const int c = i % kOwn, f = i / kOwn % EIGHTS, group = i / (kOwn * EIGHTS), col = (set * per_set + group) * kOwn + c;
      float y[8] = {}, up[8] = {};
      for (int p = 0; p < parts; ++p) {
        const float* from = &sums[(group << log_parts) + p][8 * f * kSomePitch + c];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          y[e] += from[e * kSomePitch];
          if (!CODES) up[e] += from[e * kSomePitch + 8];
        }
      }
      if constexpr (CODES) finish_column<T, false>(A, A.I, A.J, 8 * f, col, y);
      else finish_gated_column<T>(A, A.I, 8 * f, col, y, up);
    }
    __syncthreads();
  }
}

template <class T, int EIGHTS, bool CODES>
laq_status launch_some(const Err& e, const ArgsOf<CODES ? kCodes : kGated>& A, const void* x, long long ldx, const void* w, long long ldw, long long K, cudaStream_t st) {
  static Raised raised;
  const auto kernel = linear_some_rows_kernel<T, EIGHTS, CODES>;
  LAQ_TRY(raise_shared_memory(e, (const void*)kernel, raised, Some<EIGHTS>::kRing));
  const long long groups = (A.J + some_columns(CODES) - 1) / some_columns(CODES), blocks = (K + kRowBytes - 1) / kRowBytes;
  int log_parts = 0;
  while (1 << log_parts < kSomeWarps && 1 << log_parts < blocks) ++log_parts;
  const int per_set = kSomeWarps >> log_parts;
  const long long sets = (groups + per_set - 1) / per_set, most = (long long)Some<EIGHTS>::kBlocks * kSMs;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(sets < most ? sets : most));
  cfg.blockDim = dim3(kSomeThreads);
  cfg.dynamicSmemBytes = Some<EIGHTS>::kRing;
  cfg.stream = st;
  return launched(e.buf, e.len, cudaLaunchKernelEx(&cfg, kernel, A, (const uint8_t*)x, ldx, (const uint8_t*)w, ldw, K, log_parts, (int)sets));
}
// Strides and K in bytes, multiples of 16 the former, as the addresses are.
template <class T, bool CODES>
laq_status some_rows(const Err& e, const ArgsOf<CODES ? kCodes : kGated>& A, const void* x, long long ldx, const void* w, long long ldw, long long K, cudaStream_t st) {
  return A.I <= 8    ? launch_some<T, 1, CODES>(e, A, x, ldx, w, ldw, K, st)
         : A.I <= 16 ? launch_some<T, 2, CODES>(e, A, x, ldx, w, ldw, K, st)
                     : launch_some<T, 4, CODES>(e, A, x, ldx, w, ldw, K, st);
}

}  // namespace ops
}  // namespace laq
