// Matrices in 8 bits, and the product of two of them.
//
// A matrix is e4m3 codes with an fp32 scale for each block of 128 columns of a row (activations) or for each tile of 128 rows
// and 128 columns (weights):  value = code scale.  The scale is the least power of two s >= 2^-126 with |v| <= 448 s for the
// block's finite values, so that scaling is exact, a code's own rounding (half a step: 2^-4 of the value, 2^-10 s below 2^-6 s)
// is all that is lost, and a value is a bf16 number (3 bits and a power of two).
//
//   Y = act(sum_b sx[m][b] sw[n / 128][b] (sum_{k in block b} qx[m][k] qw[n][k]) + bias) + R
//
// Products of two codes are exact and the tensor cores add up 128 of them; each block's sum is then scaled and added in fp32,
// with rounding, by the epilogue's threads (codes_gemm_kernel; of some rows linear_gemm_kernel, kCodes).
#include "laq_ops_gemm.cuh"

namespace laq {
namespace ops {
namespace {

constexpr int kPackThreads = 256;
constexpr int kLanes = 16;                // threads of a block's 128 columns, eight each
// Rows that a thread has under way: as many as keep memory busy where there are many (16-bit values four, 8192 x 4096 19.9 us, by two
// 21.9; fp32 two, 26.3 us, by four 27.5), one where the blocks are few (64 x 200: 2.3 us, by four 3.5).
template <class T>
constexpr int kMostAhead = 16 / sizeof(T) / 2;

// Eight neighbours; VEC: they lie on a 16-byte boundary and all or none exist, else the first n are read wherever they lie (`edge` as in
// load16_any).
template <class T>
struct Eight {
  static constexpr int kVectors = 8 / Elem<T>::EV;
  uint4 v[kVectors];
  template <bool VEC>
  __device__ __forceinline__ void read(const T* p, int n, bool edge) {
    if (VEC) {
#pragma unroll
      for (int i = 0; i < kVectors; ++i) v[i] = n ? load16(p + i * Elem<T>::EV) : make_uint4(0u, 0u, 0u, 0u);
      return;
    }
    float x[8];
    if constexpr (sizeof(T) == 2) {
      uint4 all = make_uint4(0u, 0u, 0u, 0u);
      if (n > 0) all = load16_any(p, n, edge);
      Elem<T>::unpack(all, x);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = e < n ? x[e] : 0.f;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = e < n ? Elem<T>::to_float(p[e]) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < kVectors; ++i) {
      float part[Elem<T>::EV];
#pragma unroll
      for (int e = 0; e < Elem<T>::EV; ++e) part[e] = x[i * Elem<T>::EV + e];
      v[i] = Elem<T>::pack(part);                    // exact: the values are of type T
    }
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int i = 0; i < kVectors; ++i) {
      float part[Elem<T>::EV];
      Elem<T>::unpack(v[i], part);
#pragma unroll
      for (int e = 0; e < Elem<T>::EV; ++e) x[i * Elem<T>::EV + e] = part[e];
    }
  }
};

// The largest magnitude of eight values, +inf or NaN where one is no finite number.
__device__ __forceinline__ float largest_of(const Eight<float>& in) {
  uint4 v[2] = {in.v[0], in.v[1]};
#pragma unroll
  for (int i = 0; i < 2; ++i) v[i].x &= 0x7fffffffu, v[i].y &= 0x7fffffffu, v[i].z &= 0x7fffffffu, v[i].w &= 0x7fffffffu;
  return Elem<float>::largest(v);
}
template <class T>
__device__ __forceinline__ float largest_of(const Eight<T>& in) {
  const uint4 v[1] = {make_uint4(in.v[0].x & 0x7fff7fffu, in.v[0].y & 0x7fff7fffu, in.v[0].z & 0x7fff7fffu, in.v[0].w & 0x7fff7fffu)};
  return Elem<T>::largest(v);
}
__device__ __forceinline__ float largest_finite(const float (&x)[8]) {
  float m = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float a = fabsf(x[e]);
    m = fmaxf(m, a < INFINITY ? a : 0.f);            // NaN compares false
  }
  return m;
}

template <bool VEC>
__device__ __forceinline__ void store_codes(uint8_t* p, uint2 codes, int n) {
  if constexpr (VEC) {
    if (n) *reinterpret_cast<uint2*>(p) = codes;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) p[e] = (uint8_t)((e < 4 ? codes.x : codes.y) >> (8 * (e & 3)));
  }
}

// A scale a row and 128 columns: 16 threads take a block.  Bound by memory.  A thread block has 16 such groups, side by side
// along a row up to 1 << log_across of them, and each has AHEAD rows under way.
// VEC: rows and their eights of columns lie on vectors.
template <class T, int AHEAD, bool VEC>
__global__ void __launch_bounds__(kPackThreads) pack_rows_kernel(const T* x, long long ld, long long rows, long long cols, uint8_t* codes, long long ldc,
                                                                 float* scales, long long lds, int log_across) {
  allow_next();
  const int group = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
  const int down = kPackThreads / kLanes >> log_across;          // groups above one another
  const long long block = ((long long)blockIdx.x << log_across) + (group & ((1 << log_across) - 1));
  const long long c0 = block * kBlock + lane * 8;
  const int n = VEC ? (c0 < cols ? 8 : 0) : (int)max(0ll, min(8ll, cols - c0));
  const bool there = block * kBlock < cols;
  const long long step = (long long)gridDim.y * down * AHEAD;
  for (long long top = (long long)blockIdx.y * down * AHEAD; top < rows; top += step) {      // the same turns for a whole warp
    const long long r0 = top + (group >> log_across);
    Eight<T> in[AHEAD];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const long long r = r0 + a * down;
      in[a].template read<VEC>(x + r * ld + c0, r < rows ? n : 0, at_edge(r, r, rows, c0, cols - c0 - 8, 2));
    }
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const long long r = r0 + a * down;
      float v[8];
      in[a].get(v);
      float m = largest_of(in[a]);
#pragma unroll
      for (int o = kLanes / 2; o > 0; o /= 2) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
      const bool finite = m < INFINITY;
      if (__any_sync(0xffffffffu, !finite)) {          // rare: the largest of those that are
        float f = largest_finite(v);
#pragma unroll
        for (int o = kLanes / 2; o > 0; o /= 2) f = fmaxf(f, __shfl_xor_sync(0xffffffffu, f, o));
        if (!finite) m = f;
      }
      const int k = scale_power(m);
      if (r < rows && there) {
        const uint2 eight = finite ? encode8_finite(v, power_of_two(-k)) : encode8(v, power_of_two(-k));
        store_codes<VEC>(codes + r * ldc + c0, eight, n);
        if (lane == 0) scales[r * lds + block] = power_of_two(k);
      }
    }
  }
}

// A scale a tile of 128 x 128: a thread block's 16 groups take eight rows each and hold them in registers.
template <class T, bool VEC>
__global__ void __launch_bounds__(kPackThreads) pack_tiles_kernel(const T* x, long long ld, long long rows, long long cols, uint8_t* codes, long long ldc,
                                                                  float* scales, long long lds, long long across) {
  __shared__ float part[kPackThreads / 32];
  allow_next();
  const long long down = blockIdx.x / across, block = blockIdx.x - down * across;
  const int group = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
  const long long c0 = block * kBlock + lane * 8, row0 = down * kBlock + group;
  const int n = (int)max(0ll, min(8ll, cols - c0));
  Eight<T> in[8];
#pragma unroll
  for (int a = 0; a < 8; ++a)
    in[a].template read<VEC>(x + (row0 + 16 * a) * ld + c0, row0 + 16 * a < rows ? n : 0, at_edge(row0 + 16 * a, row0 + 16 * a, rows, c0, cols - c0 - 8, 2));
  float m = 0.f, v[8];
#pragma unroll
  for (int a = 0; a < 8; ++a) {
    in[a].get(v);
    m = fmaxf(m, largest_finite(v));
  }
#pragma unroll
  for (int o = 16; o > 0; o /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kPackThreads / 32; ++w) m = fmaxf(m, part[w]);
  const int k = scale_power(m);
#pragma unroll
  for (int a = 0; a < 8; ++a) {
    if (row0 + 16 * a >= rows) break;
    in[a].get(v);
    store_codes<VEC>(codes + (row0 + 16 * a) * ldc + c0, encode8(v, power_of_two(-k)), n);
  }
  if (threadIdx.x == 0) scales[down * lds + block] = power_of_two(k);
}

template <class T>
__device__ __forceinline__ constexpr float largest_number() {
  return std::is_same<T, float>::value ? FLT_MAX : std::is_same<T, __half>::value ? 65504.f : 3.38953139e38f;
}
// A finite value beyond T's largest is that; NaN stays.
template <class T>
__device__ __forceinline__ float within(float v) { return fabsf(v) > largest_number<T>() ? copysignf(largest_number<T>(), v) : v; }

// Codes to values, in the same arrangement.  Bound by memory.
template <class T, int AHEAD, bool VEC>
__global__ void __launch_bounds__(kPackThreads) unpack_kernel(const Codes q, long long rows, long long cols, T* out, long long ld, int log_across) {
  allow_next();
  const int group = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
  const int down = kPackThreads / kLanes >> log_across;
  const long long block = ((long long)blockIdx.x << log_across) + (group & ((1 << log_across) - 1));
  const long long c0 = block * kBlock + lane * 8;
  const int n = (int)max(0ll, min(8ll, cols - c0));
  if (n == 0) return;
  const long long step = (long long)gridDim.y * down * AHEAD;
  for (long long r0 = (long long)blockIdx.y * down * AHEAD + (group >> log_across); r0 < rows; r0 += step) {
    uint2 in[AHEAD];
    float scale[AHEAD];
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const long long r = r0 + a * down;
      in[a] = make_uint2(0u, 0u);
      scale[a] = 0.f;
      if (r >= rows) continue;
      const uint8_t* p = q.p + r * q.ld + c0;
      in[a] = VEC ? load8(p) : load8_any(p, n, at_edge(r, r, rows, c0, cols - c0 - 8, 1));
      scale[a] = q.scale(r, c0);
    }
#pragma unroll
    for (int a = 0; a < AHEAD; ++a) {
      const long long r = r0 + a * down;
      if (r >= rows) break;
      float v[8];
      decode8(in[a], scale[a], v);
      if (!(fabsf(scale[a]) <= largest_number<T>() / 448.f)) {          // values may lie beyond T's largest
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = within<T>(v[e]);
      }
      T* o = out + r * ld + c0;
      if (VEC) {
#pragma unroll
        for (int i = 0; i < 8 / Elem<T>::EV; ++i) {
          float part[Elem<T>::EV];
#pragma unroll
          for (int e = 0; e < Elem<T>::EV; ++e) part[e] = v[i * Elem<T>::EV + e];
          *reinterpret_cast<uint4*>(o + i * Elem<T>::EV) = Elem<T>::pack(part);
        }
      } else if constexpr (sizeof(T) == 2) {
        store16_any(o, Elem<T>::pack(v), n);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < n) o[e] = v[e];
      }
    }
  }
}

// ---- one or two rows through a layer in 8 bits, or four ---------------------------------------------------------------------
// W's bytes are read once, by dot products as in linear_few_rows_kernel: a warp takes four columns and a lane 16 codes of each at
// a time, whose products it adds up and scales together.  4096 x 4096: one row 5.9 us, two 7.2 (three and four go by
// linear_some_rows_kernel, 6.7); rows of 4095 codes, which lie anywhere, 12.8, 14.4 and, four, 19.6 (code by code 16.1, 19.2 and 26.9).
constexpr int kCodesAhead = 2;
constexpr int kPlainRows = 2, kSomeRows = 32;        // of codes in order: up to these by dot products, by linear_some_rows_kernel
template <class T, int ROWS, bool VEC>
__global__ void __launch_bounds__(kFewThreads, kFewBlocks)
    linear_few_codes_kernel(const CodesArgs A, const uint8_t* x, long long ldx, const uint8_t* w, long long ldw, long long K, int log_parts) {
  constexpr int kRows2 = ROWS == 3 ? 4 : ROWS, kSums = kFewCols * kRows2, kWarps = kFewThreads / 32;
  __shared__ float part[kWarps][kSums];
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5, parts = 1 << log_parts;
  const int col0 = (int)(blockIdx.x * (unsigned)(kWarps >> log_parts)) * kFewCols;
  const int first = (warp & (parts - 1)) * 32 + lane, step = 32 << log_parts;
  const int own = min(col0 + (warp >> log_parts) * kFewCols, A.J - 1);          // four columns lie in one tile of W
  const float* sw = A.sw + (long long)(own / kBlock) * A.ldsw;
  const uint8_t* wr[kFewCols];
#pragma unroll
  for (int c = 0; c < kFewCols; ++c) wr[c] = w + (long long)min(own + c, A.J - 1) * ldw;
  float s[kSums] = {};
  // At any address sixteen codes come by the words that hold them, which may reach three codes further on both sides: the first sixteen,
  // and the last, one by one.
  constexpr int kFirst = VEC ? 0 : 1;
  const int nv = VEC ? (int)(K / 16) : max(kFirst, (int)((K - 3) / 16));
  for (int v0 = kFirst + first; v0 < nv; v0 += kCodesAhead * step) {
    uint4 a[kCodesAhead][kFewCols];
#pragma unroll
    for (int u = 0; u < kCodesAhead; ++u)
#pragma unroll
      for (int c = 0; c < kFewCols; ++c)
        a[u][c] = v0 + u * step >= nv ? make_uint4(0u, 0u, 0u, 0u)
                  : VEC               ? __ldcs(reinterpret_cast<const uint4*>(wr[c]) + v0 + u * step)
                                      : load16_codes_any(wr[c] + 16ll * (v0 + u * step), 16, false);
#pragma unroll
    for (int u = 0; u < kCodesAhead; ++u) {
      const int v = v0 + u * step;
      if (v >= nv) break;
      const float of_w = __ldg(sw + v / (kBlock / 16));
      f32x2 q[ROWS][8];
      float scale[ROWS];
#pragma unroll
      for (int m = 0; m < ROWS; ++m) {
        const uint4 b = VEC ? __ldg(reinterpret_cast<const uint4*>(x + m * ldx) + v) : load16_codes_any(x + m * ldx + 16ll * v, 16, false);
        const uint32_t words[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 f = decode2(words[i / 2] >> (16 * (i & 1)) & 0xffffu);
          q[m][i] = pair_of(f.x, f.y);
        }
        scale[m] = __ldg(A.sx + m * A.ldsx + v / (kBlock / 16)) * of_w;
      }
#pragma unroll
      for (int c = 0; c < kFewCols; ++c) {
        const uint32_t words[4] = {a[u][c].x, a[u][c].y, a[u][c].z, a[u][c].w};
        f32x2 sum[ROWS];
#pragma unroll
        for (int m = 0; m < ROWS; ++m) sum[m] = 0ull;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 f = decode2(words[i / 2] >> (16 * (i & 1)) & 0xffffu);
          const f32x2 p = pair_of(f.x, f.y);
#pragma unroll
          for (int m = 0; m < ROWS; ++m) sum[m] = fma2(p, q[m][i], sum[m]);
        }
#pragma unroll
        for (int m = 0; m < ROWS; ++m) {
          float lo, hi;
          split(sum[m], lo, hi);
          s[c * kRows2 + m] = fmaf(lo + hi, scale[m], s[c * kRows2 + m]);
        }
      }
    }
  }
  for (long long i = first, by16 = 16ll * (nv - kFirst); i < K - by16; i += step) {
    const long long k = i < 16 * kFirst ? i : i + by16;
    float q[ROWS];
#pragma unroll
    for (int m = 0; m < ROWS; ++m) q[m] = decode2(x[m * ldx + k]).x * (__ldg(A.sx + m * A.ldsx + k / kBlock) * __ldg(sw + k / kBlock));
#pragma unroll
    for (int c = 0; c < kFewCols; ++c) {
      const float p = decode2(wr[c][k]).x;
#pragma unroll
      for (int m = 0; m < ROWS; ++m) s[c * kRows2 + m] = fmaf(p, q[m], s[c * kRows2 + m]);
    }
  }
  fold(s, lane);
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

// ---- the product of two matrices of codes ----------------------------------------------------------------------------------
// A tile of 128 rows (256 on a pair of SMs) and NT columns.  The tensor cores add up one block of 128 at a time, into two accumulators
// by turns, and sixteen warps add its sums, times the block's scales, to their own: one fused multiply-add an element, since a row's
// scale and a column tile's are one number for a thread's NT / 4 columns of its row.  (Two elements an instruction are slower: their
// register pairs have to be put together first.)  The sums take up to 64
// registers of a thread; the first four warps (a loader, the tensor cores' and two that bring the scales) leave theirs to them:
// 128 x 32 + 512 x 112 of the block's 640 x 96.  The scales come through shared memory, eight blocks at a time: a load of one block's
// scale by each lane touches 32 sectors, and the adding warps' own had cost a third of the time.
constexpr int kAdders = 16, kFirstAdder = 4, kCodesThreads = 32 * (kFirstAdder + kAdders), kFewRegisters = 32, kManyRegisters = 112;
constexpr int kScaleGroup = 8;                                        // blocks whose scales come together
constexpr int kScaleFloats = kScaleGroup * (kTileM + 2);              // a group's: of 128 rows and of two column tiles
// What an adding warp hands over to itself, or its part of a result that leaves by a copy: 32 rows of 64 columns in 16 bits.
__host__ __device__ constexpr int handed_bytes(bool copies) { return copies ? 4096 : 2048; }
constexpr int codes_staging(bool copies) { return kAdders * handed_bytes(copies) + 2 * kScaleFloats * 4; }

__device__ __forceinline__ void mma_codes_pair(uint32_t d_tmem, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n"
      "}\n" ::"r"(d_tmem),
      "l"(da), "l"(db), "r"(idesc), "r"(accumulate)
      : "memory");
}
// A warp's results of 32 rows and 64 columns to memory (what lies outside Y is left out), and the end of all such copies' reading.
__device__ __forceinline__ void copy_out(const CUtensorMap* map, uint32_t from, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(from), "r"(x), "r"(y) : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
__device__ __forceinline__ void copies_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }

template <class T, bool PAIR, int NT, bool COPIES>
__global__ void __launch_bounds__(kCodesThreads, 1) codes_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                                                                      const __grid_constant__ CUtensorMap tmY, const __grid_constant__ CUtensorMap tmR,
                                                                      const CodesArgs A) {
  extern __shared__ unsigned char codes_smem_raw[];
  __shared__ uint64_t bars[2 * kMaxStages + 9], residual_bars[kAdders];
  __shared__ uint32_t tmem_base_sh;
  __shared__ int abort_sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, stages = A.stages, nkb = A.nkb;
  constexpr int kHanded = handed_bytes(COPIES);
  static_assert(!COPIES || NT == 256, "a warp's 64 columns are a copy's 128 bytes");
  const uint32_t base = umma::smem_u32(codes_smem_raw), smem0 = (base + 1023u) & ~1023u;
  constexpr int b_rows = PAIR ? NT / 2 : NT;
  constexpr uint32_t a_bytes = kTileM * kBlock, st_bytes = a_bytes + b_rows * kBlock;
  constexpr uint32_t held_cols = 2 * NT;
  const int half = PAIR ? (int)(blockIdx.x & 1u) : 0;
  const uint32_t full0 = umma::smem_u32(&bars[0]), empty0 = umma::smem_u32(&bars[kMaxStages]);
  const uint32_t acc_full0 = umma::smem_u32(&bars[2 * kMaxStages]), acc_empty0 = acc_full0 + 16, drain = acc_full0 + 32;
  const uint32_t scales_full0 = drain + 8, scales_empty0 = drain + 24;
  float* const staged = reinterpret_cast<float*>(codes_smem_raw + (smem0 - base) + stages * st_bytes + kAdders * kHanded);     // two groups' scales
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      umma::mbar_init(full0 + 8 * s, 1);
      umma::mbar_init(empty0 + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      umma::mbar_init(acc_full0 + 8 * b, 1);
      umma::mbar_init(acc_empty0 + 8 * b, PAIR ? 2 * kAdders : kAdders);
      umma::mbar_init(scales_full0 + 8 * b, 2);
      umma::mbar_init(scales_empty0 + 8 * b, kAdders);
    }
    for (int i = 0; i < kAdders; ++i) umma::mbar_init(umma::smem_u32(&residual_bars[i]), 1);
    umma::mbar_init(drain, 1);
    abort_sh = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    if (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(umma::smem_u32(&tmem_base_sh)), "r"(held_cols) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(umma::smem_u32(&tmem_base_sh)), "r"(held_cols) : "memory");
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
  const int first = (int)blockIdx.x / (PAIR ? 2 : 1), step = (int)gridDim.x / (PAIR ? 2 : 1);
  const bool starved = A.starve && blockIdx.x == 0;
  const uint32_t limit = A.starve ? kStarvedLimit : umma::kWaitLimit;
  volatile int* abort_flag = &abort_sh;

  if (warp < kFirstAdder) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFewRegisters));
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
            const int r = kb * kBlock;
            if (PAIR) {
              // the pair's first block counts the bytes of both; its phase cannot end before its own arrival here
              if (half == 0) umma::mbar_expect_tx(full0 + 8 * s, 2 * st_bytes);
              const uint32_t bar = of_leader(full0 + 8 * s);
              tma_load_2d_pair(sa, &tmA, bar, r, i0);
              tma_load_2d_pair(sb, &tmB, bar, r, j0);
            } else {
              const uint32_t bar = full0 + 8 * s;
              umma::mbar_expect_tx(bar, st_bytes);
              umma::tma_load_2d(sa, &tmA, bar, r, i0);
              umma::tma_load_2d(sb, &tmB, bar, r, j0);
            }
          }
        }
        if (!ok && PAIR) {              // given up: as in linear_gemm_kernel
          for (int i = 0; i < 2000; ++i) __nanosleep(1000);
        } else if (!ok) {
          for (int m = n > stages ? n - stages : 0; m < n; ++m)
            for (uint32_t it = 0; it < umma::kWaitLimit && !umma::mbar_try_wait(full0 + 8 * (m % stages), (uint32_t)(m / stages) & 1u); ++it) {
            }
        }
      }
    } else if (warp == 1 && half == 0) {      // the pair's first block issues the products of both
      if (elect_one()) {
        const uint32_t idesc = instr_desc(0, 0, 0, NT, PAIR ? 2 * kTileM : kTileM);
        int n = 0;
        bool ok = true;
        for (int w = first; w < tiles && ok; w += step) {
          for (int kb = 0; kb < nkb; ++kb, ++n) {
            const int b = n & 1, s = n % stages;
            ok = umma::mbar_wait_abortable(full0 + 8 * s, (uint32_t)(n / stages) & 1u, limit, abort_flag, A.status, 4u) &&
                 umma::mbar_wait_abortable(acc_empty0 + 8 * b, ((uint32_t)(n >> 1) & 1u) ^ 1u, limit, abort_flag, A.status, 2u);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t sa = smem0 + s * st_bytes, d = tmem_base + (uint32_t)b * NT;
            const uint64_t da = desc_k_major(sa), db = desc_k_major(sa + a_bytes);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {          // 32 codes are 32 bytes: two units of a descriptor's address
              if (PAIR) mma_codes_pair(d, da + 2 * kk, db + 2 * kk, idesc, kk != 0);
              else mma_codes(d, da + 2 * kk, db + 2 * kk, idesc, kk != 0);
            }
            if (PAIR) {
              commit_pair(acc_full0 + 8 * b);
              commit_pair(empty0 + 8 * s);
            } else {
              umma::mma_commit(acc_full0 + 8 * b);
              umma::mma_commit(empty0 + 8 * s);
            }
          }
        }
        if (!ok) {                      // products under way still read the ring and write tensor memory
          if (PAIR) commit_pair(drain);
          else umma::mma_commit(drain);
          for (uint32_t i = 0; i < umma::kWaitLimit && !umma::mbar_try_wait(drain, 0u); ++i) {
          }
        }
      }
    }
    if (warp >= 2) {                    // scales of 64 rows each, and (the first) of the column tiles
      const bool vec = ((uintptr_t)A.sx & 15u) == 0 && A.ldsx % 4 == 0;
      int g = 0;
      bool ok = true;
      for (int w = first; w < tiles && ok; w += step) {
        int i0, j0;
        tile_of<PAIR>(A, w, i0, j0);
        i0 += half * kTileM;
        for (int k0 = 0; k0 < nkb; k0 += kScaleGroup, ++g) {
          const int b = g & 1, n = min(kScaleGroup, nkb - k0);
          ok = __all_sync(0xffffffffu, umma::mbar_wait_abortable(scales_empty0 + 8 * b, ((uint32_t)(g >> 1) & 1u) ^ 1u, limit, abort_flag, A.status, 16u));
          if (!ok) break;
          float* to = staged + b * kScaleFloats;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int r = (warp - 2) * 64 + 32 * h + lane;
            const float* p = A.sx + (long long)min(i0 + r, A.I - 1) * A.ldsx + k0;
            if (vec && n == kScaleGroup) {
              const float4 lo = __ldg(reinterpret_cast<const float4*>(p)), hi = __ldg(reinterpret_cast<const float4*>(p) + 1);
              to[r] = lo.x, to[kTileM + r] = lo.y, to[2 * kTileM + r] = lo.z, to[3 * kTileM + r] = lo.w;
              to[4 * kTileM + r] = hi.x, to[5 * kTileM + r] = hi.y, to[6 * kTileM + r] = hi.z, to[7 * kTileM + r] = hi.w;
            } else {
              for (int k = 0; k < n; ++k) to[k * kTileM + r] = __ldg(p + k);
            }
          }
          if (warp == 2 && lane < 2 * kScaleGroup && lane % kScaleGroup < n)
            to[kScaleGroup * kTileM + lane] =
                __ldg(A.sw + (long long)(min(j0 + lane / kScaleGroup * (NT / 2), A.J - 1) / kBlock) * A.ldsw + k0 + lane % kScaleGroup);
          __syncwarp();
          if (lane == 0) umma::mbar_arrive(scales_full0 + 8 * b);
        }
      }
    }
    __syncwarp();
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyRegisters));
    constexpr int kCols = NT / 4, kPieces = kCols / 16;          // of this thread's row
    const int q = warp & 3, c_first = (warp - kFirstAdder) / 4 * kCols;
    const uint32_t mine = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)c_first;
    const uint32_t back0 = PAIR ? of_leader(acc_empty0) : acc_empty0;
    uint4* stage4 = reinterpret_cast<uint4*>(codes_smem_raw + (smem0 - base) + stages * st_bytes + (warp - kFirstAdder) * kHanded);
    // COPIES: results leave by copies of their own, and residuals come by such, in the warp's 4 KB: rows of 128 bytes, their 16-byte
    // pieces permuted by the copies' swizzle.
    const uint32_t handed = umma::smem_u32(stage4), residual_bar = umma::smem_u32(&residual_bars[warp - kFirstAdder]);
    int tile_n = 0;
    const float* my_scale = staged + q * 32 + lane;
    const float* tile_scale = staged + kScaleGroup * kTileM + (c_first >= NT / 2 ? kScaleGroup : 0);
    // The next accumulator (0 or 1) and group of scales (0 or 1), and the phases of their barriers.  What is done once for each block of
    // 128 is kept short: sixteen warps' instructions, and not the tensor cores, set the pace.
    uint32_t acc = 0, acc_phase = 0, group = 0, group_phase = 0;
    bool ok = true;
    const auto wait_for = [&](uint32_t bar, uint32_t phase, uint32_t code) {
      bool there = umma::mbar_try_wait(bar, phase);
      if (!there) there = umma::mbar_wait_abortable(bar, phase, limit, abort_flag, A.status, code);
      return (bool)__all_sync(0xffffffffu, there);
    };
    for (int w = first; w < tiles && ok; w += step) {
      float sum[kPieces][16];
#pragma unroll
      for (int p = 0; p < kPieces; ++p)
#pragma unroll
        for (int e = 0; e < 16; ++e) sum[p][e] = 0.f;
      for (int k0 = 0; k0 < nkb && ok; k0 += kScaleGroup) {
        if (COPIES && A.residual && k0 == (nkb > kScaleGroup ? kScaleGroup : 0) && lane == 0) {      // the last tile's results have left, or nearly
          int i0, j0;
          tile_of<PAIR>(A, w, i0, j0);
          copies_read();
          umma::mbar_expect_tx(residual_bar, 4096);
          umma::tma_load_2d(handed, &tmR, residual_bar, j0 + c_first, i0 + half * kTileM + q * 32);
        }
        ok = wait_for(scales_full0 + 8 * group, group_phase, 16u);
        if (!ok) break;
        const float *mine_at = my_scale + group * kScaleFloats, *tile_at = tile_scale + group * kScaleFloats;
        const int n = min(kScaleGroup, nkb - k0);
        for (int in = 0; in < n; ++in, mine_at += kTileM, ++tile_at) {
          const float scale = *mine_at * *tile_at;
          ok = wait_for(acc_full0 + 8 * acc, acc_phase, 8u);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t t0 = mine + acc * NT;
          // the accumulator goes back as soon as its last columns are in registers, before they are added
          const auto give_back = [&]() {
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
              if (PAIR) arrive_lightly(back0 + 8 * acc);
              else umma::mbar_arrive(back0 + 8 * acc);
            }
          };
          if constexpr (kPieces == 1) {
            uint32_t v[16];
            tmem_load(t0, v);
            give_back();
#pragma unroll
            for (int e = 0; e < 16; ++e) sum[0][e] = fmaf(__uint_as_float(v[e]), scale, sum[0][e]);
          } else {
#pragma unroll
            for (int p = 0; p < kPieces; p += 2) {
              uint32_t v[32];
              tmem_load(t0 + 16 * p, v);
              if (p + 2 == kPieces) give_back();
#pragma unroll
              for (int e = 0; e < 32; ++e) sum[p + e / 16][e % 16] = fmaf(__uint_as_float(v[e]), scale, sum[p + e / 16][e % 16]);
            }
          }
          acc ^= 1u;
          acc_phase ^= acc ^ 1u;
        }
        if (!ok) break;
        __syncwarp();                      // all lanes have read the group's scales
        if (lane == 0) umma::mbar_arrive(scales_empty0 + 8 * group);
        group ^= 1u;
        group_phase ^= group ^ 1u;
      }
      if (!ok) break;
      int i0, j0;
      tile_of<PAIR>(A, w, i0, j0);
      i0 += half * kTileM + q * 32;
      j0 += c_first;
      if constexpr (COPIES) {
        if (A.residual) {
          ok = __all_sync(0xffffffffu, umma::mbar_wait_abortable(residual_bar, (uint32_t)tile_n & 1u, limit, abort_flag, A.status, 32u));
          if (!ok) break;
        } else {
          if (lane == 0) copies_read();
          __syncwarp();
        }
        ++tile_n;
#pragma unroll
        for (int c = 0; c < 8; ++c) {                      // a lane's row, eight columns at a time
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = sum[c / 2][8 * (c % 2) + e];
          const int col = j0 + 8 * c;
          if (A.bias) {
            const T* bias = reinterpret_cast<const T*>(A.bias) + col;
            float b[8];
            if (col + 8 <= A.J) {
              Elem<T>::unpack(__ldg(reinterpret_cast<const uint4*>(bias)), b);
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e) b[e] = col + e < A.J ? Elem<T>::to_float(bias[e]) : 0.f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] += b[e];
          }
          activate(x, A.act);
          uint4* at = stage4 + lane * 8 + (c ^ (lane & 7));
          if (A.residual) {
            float y[8];
            Elem<T>::unpack(*at, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] += y[e];
          }
          *at = Elem<T>::pack(x);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0 && i0 < A.I && j0 < A.J) copy_out(&tmY, handed, j0, i0);
        continue;
      }
      const bool vec = all_vectors(A, false), whole = vec && i0 + 32 <= A.I && j0 + kCols <= A.J;
      // pieces of 32 x 16 through shared memory, after which two lanes share a row
      const long long row0 = i0 + (lane >> 1);
      int col = j0 + 8 * (lane & 1);
      uint4 next[2];                       // the residual of the piece after this one
      const auto ahead = [&](int c) {
        const T* rp = reinterpret_cast<const T*>(A.residual) + row0 * A.ldr + c;
        next[0] = load16(rp);
        next[1] = load16(rp + 16 * A.ldr);
      };
      if (whole && A.residual) ahead(col);
#pragma unroll 1
      for (int p = 0; p < kPieces; ++p, col += 16) {
        const uint4 res[2] = {next[0], next[1]};
        uint4 bias = make_uint4(0u, 0u, 0u, 0u);
        if (whole) {
          if (A.residual && p + 1 < kPieces) ahead(col + 16);
          if (A.bias) bias = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(A.bias) + col));
        }
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 16; e += 4)
          stage4[narrow_piece(lane, e / 4)] = make_uint4(__float_as_uint(sum[0][e]), __float_as_uint(sum[0][e + 1]), __float_as_uint(sum[0][e + 2]),
                                                         __float_as_uint(sum[0][e + 3]));
        // the next piece moves up: no register can be chosen by a number that is only known at run time
#pragma unroll
        for (int m = 0; m + 1 < kPieces; ++m)
#pragma unroll
          for (int e = 0; e < 16; ++e) sum[m][e] = sum[m + 1][e];
        __syncwarp();
        if (whole) {
          float b[8];
          Elem<T>::unpack(bias, b);
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int r = 16 * k + (lane >> 1);
            const uint4 lo = stage4[narrow_piece(r, 2 * (lane & 1))], hi = stage4[narrow_piece(r, 2 * (lane & 1) + 1)];
            float x[8] = {__uint_as_float(lo.x), __uint_as_float(lo.y), __uint_as_float(lo.z), __uint_as_float(lo.w),
                          __uint_as_float(hi.x), __uint_as_float(hi.y), __uint_as_float(hi.z), __uint_as_float(hi.w)};
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] += b[e];
            if (A.z) *reinterpret_cast<uint4*>(reinterpret_cast<T*>(A.z) + (row0 + 16 * k) * A.ldz + col) = Elem<T>::pack(x);
            activate(x, A.act);
            if (A.residual) {
              float y[8];
              Elem<T>::unpack(res[k], y);
#pragma unroll
              for (int e = 0; e < 8; ++e) x[e] += y[e];
            }
            *reinterpret_cast<uint4*>(reinterpret_cast<T*>(A.out) + (row0 + 16 * k) * A.ldo + col) = Elem<T>::pack(x);
          }
          continue;
        }
#pragma unroll 1
        for (int k = 0; k < 2; ++k) {
          float x[8];
          if (vec) {
            const int r = 16 * k + (lane >> 1);
            const uint4 lo = stage4[narrow_piece(r, 2 * (lane & 1))], hi = stage4[narrow_piece(r, 2 * (lane & 1) + 1)];
            x[0] = __uint_as_float(lo.x), x[1] = __uint_as_float(lo.y), x[2] = __uint_as_float(lo.z), x[3] = __uint_as_float(lo.w);
            x[4] = __uint_as_float(hi.x), x[5] = __uint_as_float(hi.y), x[6] = __uint_as_float(hi.z), x[7] = __uint_as_float(hi.w);
            finish_row<T, false>(A, i0 + r, col, x, residual8<T>(A, i0 + r, col, vec));
          } else {                         // half a warp has 8 rows of 16 columns
            const int r = 16 * k + 8 * (lane >> 4), c = lane & 15;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(reinterpret_cast<const uint32_t*>(&stage4[narrow_piece(r + e, c >> 2)])[c & 3]);
            finish_column<T, false>(A, A.I, A.J, i0 + r, j0 + 16 * p + c, x);
          }
        }
      }
    }
    if (COPIES && lane == 0) {
      if (!ok && A.residual) {             // given up: a residual that was asked for still lands here
        for (uint32_t it = 0; it < kStarvedLimit && !umma::mbar_try_wait(residual_bar, (uint32_t)tile_n & 1u); ++it) {
        }
      }
      asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    __syncwarp();
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

// Codes that a tensor map cannot describe are copied with a pitch of a multiple of 16 bytes, both operands' in one launch.  A warp
// takes a row, a lane 16 codes of it at a time.
struct CodeRows {
  const uint8_t* src;
  uint8_t* dst;
  long long ld, pitch, rows, cols;
};
__global__ void __launch_bounds__(256) copy_codes_kernel(const CodeRows a, const CodeRows b) {
  allow_next();
  const int lane = threadIdx.x & 31;
  const long long warps = (long long)gridDim.x * (blockDim.x / 32);
  for (long long i = ((long long)blockIdx.x * blockDim.x + threadIdx.x) / 32; i < a.rows + b.rows; i += warps) {
    const bool second = i >= a.rows;
    const long long r = second ? i - a.rows : i, cols = second ? b.cols : a.cols;
    const uint8_t* src = second ? b.src + r * b.ld : a.src + r * a.ld;
    uint8_t* dst = second ? b.dst + r * b.pitch : a.dst + r * a.pitch;
    for (long long c = lane * 16; c < cols; c += 512) {
      *reinterpret_cast<uint4*>(dst + c) = load16_codes_any(src + c, (int)min(16ll, cols - c), at_edge(r, r, second ? b.rows : a.rows, c, cols - c - 16, 1));
    }
  }
}

// ---- host -----------------------------------------------------------------------------------------------------------------
long long pad16(long long x) { return (x + 15) / 16 * 16; }
// A row by itself has no pitch that matters.
Operand codes_of(const laq_blocks* b, long long rows, long long cols) { return Operand{b->codes, rows == 1 ? pad16(cols) : b->ld_codes, rows, cols}; }
bool codes_mappable(const Operand& o) { return ((uintptr_t)o.p & 15u) == 0 && o.ld % 16 == 0; }
size_t copy_bytes(const Operand& o) { return codes_mappable(o) ? 0 : align256((size_t)o.rows * pad16(o.cols)); }

// Copies what needs it of two operands to `ws` (advanced past it).
laq_status make_codes_mappable(const Err& e, Operand& x, Operand& w, char*& ws, cudaStream_t st) {
  CodeRows rows[2] = {};
  Operand* of[2] = {&x, &w};
  long long total = 0;
  for (int i = 0; i < 2; ++i) {
    Operand& o = *of[i];
    const size_t bytes = copy_bytes(o);
    if (!bytes) continue;
    rows[i] = CodeRows{(const uint8_t*)o.p, (uint8_t*)ws, o.ld, pad16(o.cols), o.rows, o.cols};
    o.p = ws;
    o.ld = rows[i].pitch;
    ws += bytes;
    total += o.rows;
  }
  if (!total) return LAQ_OK;
  const long long want = (total + 7) / 8, most = 8 * kSMs;
  return launched(e.buf, e.len, launch_plain(copy_codes_kernel, dim3((unsigned)(want < most ? want : most)), 256, st, rows[0], rows[1]));
}

struct Spread {                // of the 16 groups of a thread block over blocks of columns and rows
  int log_across, ahead;
  dim3 grid;
  Spread(long long rows, long long cols, int most_ahead) {
    const long long across = blocks_across(cols);
    log_across = across >= 16 ? 4 : across >= 8 ? 3 : across >= 4 ? 2 : across >= 2 ? 1 : 0;
    const long long gx = (across + (1 << log_across) - 1) >> log_across, high = kPackThreads / kLanes >> log_across;
    ahead = gx * (rows / (high * most_ahead)) >= 2 * kSMs ? most_ahead : 1;
    const long long down = high * ahead, runs = (rows + down - 1) / down;
    grid = dim3((unsigned)gx, (unsigned)(runs < 65535 ? runs : 65535));
  }
};

template <class T>
laq_status pack_typed(const Err& e, const T* x, long long rows, long long cols, long long ld, const laq_blocks& b, cudaStream_t st) {
  uint8_t* codes = (uint8_t*)const_cast<void*>(b.codes);
  float* scales = const_cast<float*>(b.scales);
  const bool vec = ((uintptr_t)x & 15u) == 0 && ld * (long long)sizeof(T) % 16 == 0 && Codes(&b).vectors(8) && cols % 8 == 0;
  if (b.block_rows == kBlock) {
    const long long across = blocks_across(cols), tiles = across * ((rows + kBlock - 1) / kBlock);
    return launched(e.buf, e.len, launch_plain(vec ? pack_tiles_kernel<T, true> : pack_tiles_kernel<T, false>, dim3((unsigned)tiles), kPackThreads, st, x, ld,
                                               rows, cols, codes, b.ld_codes, scales, b.ld_scales, across));
  }
  const Spread s(rows, cols, kMostAhead<T>);
  const auto kernel = s.ahead > 1 ? (vec ? pack_rows_kernel<T, kMostAhead<T>, true> : pack_rows_kernel<T, kMostAhead<T>, false>)
                                  : (vec ? pack_rows_kernel<T, 1, true> : pack_rows_kernel<T, 1, false>);
  return launched(e.buf, e.len, launch_plain(kernel, s.grid, kPackThreads, st, x, ld, rows, cols, codes, b.ld_codes, scales, b.ld_scales, s.log_across));
}

template <class T>
laq_status unpack_typed(const Err& e, const laq_blocks& b, long long rows, long long cols, T* out, long long ld, cudaStream_t st) {
  const Spread s(rows, cols, kMostAhead<T>);
  const bool vec = ((uintptr_t)out & 15u) == 0 && ld * (long long)sizeof(T) % 16 == 0 && Codes(&b).vectors(8) && cols % 8 == 0;
  const auto kernel = s.ahead > 1 ? (vec ? unpack_kernel<T, kMostAhead<T>, true> : unpack_kernel<T, kMostAhead<T>, false>)
                                  : (vec ? unpack_kernel<T, 1, true> : unpack_kernel<T, 1, false>);
  return launched(e.buf, e.len, launch_plain(kernel, s.grid, kPackThreads, st, Codes(&b), rows, cols, out, ld, s.log_across));
}

template <class T>
void list_block_kernels(const void** list, int& n) {
  const void* all[] = {(const void*)pack_rows_kernel<T, 1, false>,   (const void*)pack_rows_kernel<T, kMostAhead<T>, false>,
                       (const void*)pack_rows_kernel<T, 1, true>,    (const void*)pack_rows_kernel<T, kMostAhead<T>, true>,
                       (const void*)pack_tiles_kernel<T, false>,     (const void*)pack_tiles_kernel<T, true>,
                       (const void*)unpack_kernel<T, 1, false>,      (const void*)unpack_kernel<T, kMostAhead<T>, false>,
                       (const void*)unpack_kernel<T, 1, true>,       (const void*)unpack_kernel<T, kMostAhead<T>, true>};
  for (const void* k : all) list[n++] = k;
}
template <class T>
void list_product_kernels(const void** list, int& n) {
  const void* all[] = {(const void*)linear_gemm_kernel<T, true, false, false, false, kCodes>, (const void*)codes_gemm_kernel<T, true, 256, true>,
                       (const void*)codes_gemm_kernel<T, true, 256, false>, (const void*)codes_gemm_kernel<T, true, 128, false>,
                       (const void*)codes_gemm_kernel<T, false, 128, false>, (const void*)codes_gemm_kernel<T, false, 64, false>,
                       (const void*)linear_few_codes_kernel<T, 1, true>, (const void*)linear_few_codes_kernel<T, 2, true>,
                       (const void*)linear_some_rows_kernel<T, 1, true>, (const void*)linear_some_rows_kernel<T, 2, true>,
                       (const void*)linear_some_rows_kernel<T, 4, true>,
                       (const void*)linear_few_codes_kernel<T, 1, false>, (const void*)linear_few_codes_kernel<T, 2, false>,
                       (const void*)linear_few_codes_kernel<T, 3, false>, (const void*)linear_few_codes_kernel<T, 4, false>};
  for (const void* k : all) list[n++] = k;
}

laq_status check_matrix(const Err& e, int64_t rows, int64_t cols) {
  const int64_t most = 0x7fffff00ll;
  if (rows < 0 || rows > most || cols < 1 || cols > most) return fail(e.buf, e.len, LAQ_EINVAL, "rows must be 0..2^31-256, cols 1..2^31-256");
  return LAQ_OK;
}

template <class T, bool PAIR, int NT, bool COPIES>
laq_status launch_codes(const Err& e, const Product<kCodes>& p, bool follows, cudaStream_t st) {
  static Raised raised;
  CUtensorMap my = p.ma, mr = p.ma;                // unused without copies or a residual
  if (COPIES && (!umma::make_map_bf16_2d(&my, p.A.out, p.A.I, p.A.J, p.A.ldo * 2, 32) ||
                 (p.A.residual && !umma::make_map_bf16_2d(&mr, p.A.residual, p.A.I, p.A.J, p.A.ldr * 2, 32))))
    return fail(e.buf, e.len, LAQ_ECUDA, "a tensor map was refused");
  return launch_tiles<CodesArgs, CUtensorMap, CUtensorMap, CUtensorMap, CUtensorMap>(e, codes_gemm_kernel<T, PAIR, NT, COPIES>, raised, kCodesThreads, PAIR, false,
                                                                          codes_staging(COPIES), follows, st, p.A, p.ma, p.mb, my, mr);
}
template <class T>
laq_status launch_product(const Err& e, const Product<kCodes>& p, bool follows, cudaStream_t st) {
  if (p.pl.swap) return launch_gemm<T, true, false, false, false, kCodes>(e, p.ma, p.mb, p.A, follows, st);
  if (!p.pl.pair) return p.pl.nt == 128 ? launch_codes<T, false, 128, false>(e, p, follows, st) : launch_codes<T, false, 64, false>(e, p, follows, st);
  if (p.pl.nt == 128) return launch_codes<T, true, 128, false>(e, p, follows, st);
  const bool copies = !p.A.z && mappable(p.A.out, p.A.ldo) && mappable(p.A.residual, p.A.ldr) && mappable(p.A.bias, 8);
  return copies ? launch_codes<T, true, 256, true>(e, p, follows, st) : launch_codes<T, true, 256, false>(e, p, follows, st);
}

bool takes_few_codes(const laq_linear_call* c) { return !(c->flags & LAQ_LINEAR_STARVE) && c->M <= kFewRows; }


template <class T>
laq_status few_codes(const Err& e, const CodesArgs& A, const Operand& x, const Operand& w, cudaStream_t st) {
  const bool vec = codes_mappable(x) && codes_mappable(w);
  const long long groups = (w.rows + kFewCols - 1) / kFewCols, items = w.cols / 16;
  const int log_parts = few_log_parts(groups, items < (1 << 30) ? (int)items : 1 << 30), per_block = kFewThreads / 32 >> log_parts;
  const auto of = [&](auto rows) {
    constexpr int kRows = decltype(rows)::value;
    if constexpr (kRows <= kPlainRows) return vec ? linear_few_codes_kernel<T, kRows, true> : linear_few_codes_kernel<T, kRows, false>;
    else return linear_few_codes_kernel<T, kRows, false>;          // aligned ones go by linear_some_rows_kernel
  };
  const auto kernel = x.rows == 1   ? of(std::integral_constant<int, 1>())
                      : x.rows == 2 ? of(std::integral_constant<int, 2>())
                      : x.rows == 3 ? of(std::integral_constant<int, 3>())
                                    : of(std::integral_constant<int, 4>());
  return launched(e.buf, e.len, launch_plain(kernel, dim3((unsigned)((groups + per_block - 1) / per_block)), kFewThreads, st, A, (const uint8_t*)x.p, x.ld,
                                             (const uint8_t*)w.p, w.ld, w.cols, log_parts));
}

// Where the tiles of tensor memory overtake: 16 rows of 8192 x 8192 22.5 us (by tiles 23.7), of 16384 x 16384 77 (72); 32 rows of
// 4096 x 4096 12.4 (12.7), of 4096 x 8192 20 (17), of 11008 x 4096 27 (22), of 16 x 65536 60 (39).  In rows longer than 8192 it is the
// columns that decide, 32 rows of 1024 x 65536 64 (79): those some microseconds are given up, and all of them go by tiles.
bool takes_some_codes(const laq_linear_call* c, const laq_blocks* xq, const laq_blocks* wq) {
  if ((c->flags & LAQ_LINEAR_STARVE) || c->M <= kPlainRows || c->M > kSomeRows) return false;
  if (c->M > 8 && c->N > (c->M > 16 ? 1ll << 24 : 1ll << 26) / c->K) return false;
  if (c->M > 16 && c->K > 8192) return false;
  return codes_mappable(codes_of(xq, c->M, c->K)) && codes_mappable(codes_of(wq, c->N, c->K));
}
}  // namespace

laq_status load_block_kernels(const Err& e) {
  static Loaded loaded;
  static const void* list[64];
  static const int n = [] {
    int count = 0;
    list_block_kernels<float>(list, count);
    list_block_kernels<__nv_bfloat16>(list, count);
    list_block_kernels<__half>(list, count);
    list_product_kernels<__nv_bfloat16>(list, count);
    list_product_kernels<__half>(list, count);
    list[count++] = (const void*)copy_codes_kernel;
    return count;
  }();
  return launched(e.buf, e.len, loaded.once(list, n));
}

laq_status pack_blocks(const Err& e, const void* x, int dtype, long long rows, long long cols, long long ld, const laq_blocks& b, cudaStream_t st) {
  return dtype == LAQ_F32    ? pack_typed(e, (const float*)x, rows, cols, ld, b, st)
         : dtype == LAQ_BF16 ? pack_typed(e, (const __nv_bfloat16*)x, rows, cols, ld, b, st)
                             : pack_typed(e, (const __half*)x, rows, cols, ld, b, st);
}

laq_status unpack_blocks(const Err& e, const laq_blocks& b, long long rows, long long cols, int dtype, void* out, long long ld, cudaStream_t st) {
  return dtype == LAQ_F32    ? unpack_typed(e, b, rows, cols, (float*)out, ld, st)
         : dtype == LAQ_BF16 ? unpack_typed(e, b, rows, cols, (__nv_bfloat16*)out, ld, st)
                             : unpack_typed(e, b, rows, cols, (__half*)out, ld, st);
}

laq_status check_blocks(const Err& e, Buffers& buffers, const char* name, const char* scales_name, Access access, const laq_blocks* b, int64_t rows,
                        int64_t cols) {
  if (!b || !b->codes || !b->scales) return fail(e.buf, e.len, LAQ_EINVAL, "the codes or the scales of %s are null", name);
  if (b->block_rows != 1 && b->block_rows != kBlock) return fail(e.buf, e.len, LAQ_EINVAL, "block_rows of %s must be 1 or 128", name);
  const int64_t down = b->block_rows == 1 ? rows : (rows + kBlock - 1) / kBlock;
  LAQ_TRY(check_tensor(e, buffers, name, access, b->codes, true, rows, b->ld_codes, cols, 1));
  return check_tensor(e, buffers, scales_name, access, b->scales, true, down, b->ld_scales, blocks_across(cols), 4);
}

}  // namespace ops
}  // namespace laq

using namespace laq::ops;

extern "C" laq_status laq_pack_blocks(const void* d_x, int32_t dtype, int64_t rows, int64_t cols, int64_t row_stride, const laq_blocks* out,
                                      void* cuda_stream, char* errbuf, size_t errbuf_len) {
  const Err e{errbuf, errbuf_len};
  if (errbuf && errbuf_len) errbuf[0] = 0;
  if (!dtype_bytes(dtype)) return fail(errbuf, errbuf_len, LAQ_EINVAL, "dtype must be LAQ_F32, LAQ_BF16 or LAQ_F16");
  LAQ_TRY(check_matrix(e, rows, cols));
  if (rows == 0) return LAQ_OK;
  Buffers buffers;
  LAQ_TRY(check_tensor(e, buffers, "x", kRead, d_x, true, rows, row_stride, cols, dtype_bytes(dtype)));
  LAQ_TRY(check_blocks(e, buffers, "out", "the scales of out", kWritten, out, rows, cols));
  LAQ_TRY(buffers.check(errbuf, errbuf_len));
  LAQ_TRY(load_block_kernels(e));
  return pack_blocks(e, d_x, dtype, rows, cols, row_stride, *out, (cudaStream_t)cuda_stream);
}

extern "C" laq_status laq_unpack_blocks(const laq_blocks* x, int64_t rows, int64_t cols, void* d_out, int32_t dtype, int64_t row_stride,
                                        void* cuda_stream, char* errbuf, size_t errbuf_len) {
  const Err e{errbuf, errbuf_len};
  if (errbuf && errbuf_len) errbuf[0] = 0;
  if (!dtype_bytes(dtype)) return fail(errbuf, errbuf_len, LAQ_EINVAL, "dtype must be LAQ_F32, LAQ_BF16 or LAQ_F16");
  LAQ_TRY(check_matrix(e, rows, cols));
  if (rows == 0) return LAQ_OK;
  Buffers buffers;
  LAQ_TRY(check_blocks(e, buffers, "x", "the scales of x", kRead, x, rows, cols));
  LAQ_TRY(check_tensor(e, buffers, "out", kWritten, d_out, true, rows, row_stride, cols, dtype_bytes(dtype)));
  LAQ_TRY(buffers.check(errbuf, errbuf_len));
  LAQ_TRY(load_block_kernels(e));
  return unpack_blocks(e, *x, rows, cols, dtype, d_out, row_stride, (cudaStream_t)cuda_stream);
}

extern "C" laq_status laq_linear_blocks_forward(const laq_linear_call* c, const laq_blocks* xq, const laq_blocks* wq, void* d_workspace,
                                                size_t workspace_bytes, void* cuda_stream, char* errbuf, size_t errbuf_len) {
  const Err e{errbuf, errbuf_len};
  if (errbuf && errbuf_len) errbuf[0] = 0;
  if (!c || !xq || !wq) return fail(errbuf, errbuf_len, LAQ_EINVAL, "null pointer");
  const size_t need = laq_linear_blocks_workspace_bytes(c, xq, wq, 0);
  LAQ_TRY(check_layer(e, c->dtype, c->M, c->N, c->K, c->activation, c->status, c->flags, d_workspace, workspace_bytes, need));
  if (c->M == 0) return LAQ_OK;
  if (xq->block_rows != 1 && c->M > 1) return fail(errbuf, errbuf_len, LAQ_EINVAL, "x must have a scale for each row (block_rows 1)");
  if (wq->block_rows != kBlock && c->N > 1) return fail(errbuf, errbuf_len, LAQ_EINVAL, "w must have a scale for each tile of 128 rows (block_rows 128)");
  Buffers buffers;
  buffers.out("status", c->status, 4, 1, 1, 1);
  if (need) buffers.out("the workspace", d_workspace, 1, 1, (long long)need, (long long)need);
  LAQ_TRY(check_blocks(e, buffers, "x", "the scales of x", kRead, xq, c->M, c->K));
  LAQ_TRY(check_blocks(e, buffers, "w", "the scales of w", kRead, wq, c->N, c->K));
  LAQ_TRY(check_tensor(e, buffers, "bias", kRead, c->bias, false, 1, c->N, c->N, 2));
  LAQ_TRY(check_tensor(e, buffers, "residual", kRead, c->residual, false, c->M, c->ld_residual, c->N, 2));
  LAQ_TRY(check_tensor(e, buffers, "y", kWritten, c->y, true, c->M, c->ld_y, c->N, 2, "residual"));
  LAQ_TRY(check_tensor(e, buffers, "z", kWritten, c->z, false, c->M, c->ld_z, c->N, 2));
  LAQ_TRY(buffers.check(errbuf, errbuf_len));
  LAQ_TRY(load_block_kernels(e));
  cudaStream_t st = (cudaStream_t)cuda_stream;
  Operand x = codes_of(xq, c->M, c->K), w = codes_of(wq, c->N, c->K);
  CodesArgs A = {};
  A.I = (int)c->M;
  A.J = (int)c->N;
  A.act = c->activation;
  A.starve = (c->flags & LAQ_LINEAR_STARVE) != 0;
  A.out = c->y;
  A.ldo = c->ld_y;
  A.z = c->z;
  A.ldz = c->ld_z;
  A.bias = c->bias;
  A.residual = c->residual;
  A.ldr = c->ld_residual;
  A.status = c->status;
  A.sx = xq->scales;
  A.ldsx = xq->ld_scales;
  A.sw = wq->scales;
  A.ldsw = wq->ld_scales;
  if (takes_some_codes(c, xq, wq))
    return c->dtype == LAQ_BF16 ? some_rows<__nv_bfloat16, true>(e, A, x.p, x.ld, w.p, w.ld, c->K, st)
                                : some_rows<__half, true>(e, A, x.p, x.ld, w.p, w.ld, c->K, st);
  if (takes_few_codes(c)) return c->dtype == LAQ_BF16 ? few_codes<__nv_bfloat16>(e, A, x, w, st) : few_codes<__half>(e, A, x, w, st);
  char* ws = (char*)d_workspace;
  LAQ_TRY(make_codes_mappable(e, x, w, ws, st));
  const bool follows = ws != d_workspace;
  Product<kCodes> p;
  p.A = A;
  LAQ_TRY(prepare_product(e, p, x, w, 0));
  return c->dtype == LAQ_BF16 ? launch_product<__nv_bfloat16>(e, p, follows, st) : launch_product<__half>(e, p, follows, st);
}

namespace laq {
namespace ops {
size_t blocks_forward_bytes(const laq_linear_call* c, const laq_blocks* xq, const laq_blocks* wq) {
  if (!xq || !wq || takes_few_codes(c) || takes_some_codes(c, xq, wq)) return 0;
  return copy_bytes(codes_of(xq, c->M, c->K)) + copy_bytes(codes_of(wq, c->N, c->K));
}
}  // namespace ops
}  // namespace laq
