// A gated feed-forward block's two projections, its activation and their product, and the gradient:
//   Z = X W^T + b,  W [2F][K]: F rows of gates G, then as many of ups U;   H = act(G) U         X [M][K], Z [M][2F], H [M][F]
//   dG = dH U act'(G),  dU = dH act(G),  dZ = [dG | dU];   dX = dZ W,  dW = dZ^T X,  db = column sums of dZ
// The forward pass is one product whose tiles hold as many columns of gates as of the ups that belong to them
// (gated_gemm_kernel; with split sums and transposed linear_gemm_kernel, kGated), so that H leaves the epilogue and Z is written only if it is asked for.  H is rounded once, from
// sums in fp32.  With W as one matrix the gradient is two products as a layer's is; dZ is rounded once to the operands' type, as there.
#include "laq_ops_gemm.cuh"

namespace laq {
namespace ops {
namespace {

// ---- both projections and their product, tiles of whole sums --------------------------------------------------------------
// A tile of 128 rows (256 on a pair of SMs) and nt columns, half of them gates and half the ups that belong to them.  The tensor cores cut
// their sums (laq_ops_gemm.cuh), which moves numbers to the other side of a rounding, and of Z in 8 bits such a one is a whole code off: they add up
// 320 to 640 terms at a time, into two accumulators by turns, and sixteen warps add those sums up with rounding.  A thread has 32 gates and their 32
// ups of a row, 64 sums (eight warps would need 128 each, more than there are registers); the first four warps, a loader and the tensor
// cores' among them, leave theirs to them as in codes_gemm_kernel.  Both accumulators are free while a tile's results are written.
// Packed Z of 2048 x (2 x 2048) x 2048 and x 4096 is 1.7e-4 and 1.9e-4 off the codes of its fp64 values (from sums cut throughout 3.4e-4 and 5.9e-4, from plain fp32 sums
// 1.3e-4 and 1.8e-4).  8192 x 4096 x 4096 419 us (cut throughout 434), 4096 x 5504 x 2048 144 (139), with Z 175 (166), with Z in 8 bits 182 (175).
constexpr int kAdders = 16, kFirstAdder = 4, kGatedThreads = 32 * (kFirstAdder + kAdders), kFewRegisters = 32, kManyRegisters = 112;
constexpr int kChunk = 10, kShortSum = 16;             // k-blocks: 640 and 1024 terms
// A sum's chunk that begins at k0: all of a short sum, which linear_gemm_kernel does not cut up either, so that Z in 8 bits is that of the call without.  The
// first two of a long one are what the tensor cores can do while the last tile's results are written (of 384 terms 4096 x 5504 x 2048 with Z in 8 bits
// 190 us for 160).  Those after them are shorter in sums that have few of them, for each costs an accumulator's way there and back
// (8192 x 4096 x 4096 by chunks of 320 terms 438 us for 402, and no nearer than plain fp32 sums in either way).
__device__ __forceinline__ int chunk_at(int k0, int nkb) {
  return nkb <= kShortSum ? kShortSum : k0 < 2 * kChunk ? kChunk : max(kChunk / 2, min(kChunk, nkb / 6));
}
// What an adding warp hands over to itself: 32 rows of W columns.  16 leave the ring its six stages, and 32 make whole 64-byte stretches of what
// is written, which pays where Z is written too (4096 x 5504 x 2048 with Z in 8 bits 161 us, by 16 columns 181; 512 x 4096 x 4096 without Z 33.7, by 32 34.5).
__host__ __device__ constexpr int handed_bytes(int w) { return 32 * 4 * w; }

template <class T, bool PAIR, int W>
__global__ void __launch_bounds__(kGatedThreads, 1) gated_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                                                                      const GatedArgs A) {
  extern __shared__ unsigned char gated_smem_raw[];
  __shared__ uint64_t bars[2 * kMaxStages + 9];
  __shared__ signed char powers[kAdders][64];          // of the scales that each warp's columns ask for: 32 rows' gates and ups
  __shared__ uint32_t tmem_base_sh;
  __shared__ int abort_sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, nt = A.nt, stages = A.stages, nkb = A.nkb;
  const uint32_t base = umma::smem_u32(gated_smem_raw), smem0 = (base + 1023u) & ~1023u;
  const int b_rows = PAIR ? nt / 2 : nt;           // of W that this block loads: a pair's first block the gates', its second the ups'
  const uint32_t a_bytes = kTileM * kBlockK * 2, st_bytes = a_bytes + (uint32_t)b_rows * kBlockK * 2;
  const int half = PAIR ? (int)(blockIdx.x & 1u) : 0;
  const uint32_t full0 = umma::smem_u32(&bars[0]), empty0 = umma::smem_u32(&bars[kMaxStages]);
  const uint32_t acc_full0 = umma::smem_u32(&bars[2 * kMaxStages]), acc_empty0 = acc_full0 + 16, drain = acc_full0 + 32, told0 = drain + 8;
  const uint32_t acc_cols = umma::tmem_cols(nt), held_cols = 2 * acc_cols;
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      umma::mbar_init(full0 + 8 * s, 1);
      umma::mbar_init(empty0 + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      umma::mbar_init(acc_full0 + 8 * b, 1);
      umma::mbar_init(acc_empty0 + 8 * b, PAIR ? 2 * kAdders : kAdders);
    }
    umma::mbar_init(drain, 1);
    for (int q = 0; q < 4; ++q) umma::mbar_init(told0 + 8 * q, kAdders / 4);
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
  const uint32_t limit = A.starve ? kStarvedLimit : umma::kWaitLimit;
  volatile int* abort_flag = &abort_sh;

  if (warp < kFirstAdder) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kFewRegisters));
    if (warp == 0) {
      if (elect_one()) {
        int n = 0;                       // stages handed out so far
        bool ok = !(A.starve && blockIdx.x == 0);
        for (int w = first; w < tiles && ok; w += step) {
          int i0, j0;
          tile_of<PAIR>(A, w, i0, j0);
          i0 += half * kTileM;
          j0 = j0 / 2 + half * (int)A.up;
          for (int kb = 0; kb < nkb; ++kb, ++n) {
            const int s = n % stages;
            ok = umma::mbar_wait_abortable(empty0 + 8 * s, ((uint32_t)(n / stages) & 1u) ^ 1u, limit, abort_flag, A.status, 1u);
            if (!ok) break;
            const uint32_t sa = smem0 + s * st_bytes, sb = sa + a_bytes;
            const int r = kb * kBlockK;
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
              umma::tma_load_2d(sb + nt / 2 * 128, &tmB, bar, r, j0 + (int)A.up);
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
        const uint32_t idesc = instr_desc(A.fmt, 0, 0, nt, PAIR ? 2 * kTileM : kTileM);
        int n = 0, it = 0;
        bool ok = true;
        for (int w = first; w < tiles && ok; w += step) {
          for (int k0 = 0, k1; k0 < nkb && ok; k0 = k1, ++it) {
            const int b = it & 1;
            k1 = min(k0 + chunk_at(k0, nkb), nkb);
            ok = umma::mbar_wait_abortable(acc_empty0 + 8 * b, ((uint32_t)(it >> 1) & 1u) ^ 1u, limit, abort_flag, A.status, 2u);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t d = tmem_base + (uint32_t)b * acc_cols;
            for (int kb = k0; kb < k1; ++kb, ++n) {
              const int s = n % stages;
              ok = umma::mbar_wait_abortable(full0 + 8 * s, (uint32_t)(n / stages) & 1u, limit, abort_flag, A.status, 4u);
              if (!ok) break;
              asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
              const uint32_t sa = smem0 + s * st_bytes;
              const uint64_t da = desc_k_major(sa), db = desc_k_major(sa + a_bytes);
#pragma unroll
              for (int kk = 0; kk < kBlockK / 16; ++kk) {          // 32 bytes of the summed axis: two units of a descriptor's address
                const uint32_t more = kb != k0 || kk != 0 ? 1u : 0u;
                if (PAIR) mma_pair(d, da + 2 * kk, db + 2 * kk, idesc, more);
                else umma::mma_bf16_ss(d, da + 2 * kk, db + 2 * kk, idesc, more);
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
        if (!ok) {                      // products under way still read the ring and write tensor memory
          if (PAIR) commit_pair(drain);
          else umma::mma_commit(drain);
          for (uint32_t i = 0; i < umma::kWaitLimit && !umma::mbar_try_wait(drain, 0u); ++i) {
          }
        }
      }
    }
    __syncwarp();
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kManyRegisters));
    const int q = warp & 3, c0 = (warp - kFirstAdder) / 4 * 32;          // this warp's rows, and its first column of the gates and of the ups
    const bool there = c0 < nt / 2, vec = all_vectors(A, false);
    const uint32_t mine = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)c0;
    const uint32_t back0 = PAIR ? of_leader(acc_empty0) : acc_empty0, told = told0 + 8 * q;
    unsigned char* const staging = gated_smem_raw + (smem0 - base) + stages * st_bytes;
    uint4* stage4 = reinterpret_cast<uint4*>(staging + (warp - kFirstAdder) * handed_bytes(W));
    int it = 0;
    uint32_t told_phase = 0;
    bool ok = true;
    const auto wait_for = [&](uint32_t bar, uint32_t phase, uint32_t code) {
      bool done = umma::mbar_try_wait(bar, phase);
      if (!done) done = umma::mbar_wait_abortable(bar, phase, limit, abort_flag, A.status, code);
      return (bool)__all_sync(0xffffffffu, done);
    };
    for (int w = first; w < tiles && ok; w += step) {
      float sum[2][32];                      // of this lane's row: gates, ups
#pragma unroll
      for (int part = 0; part < 2; ++part)
#pragma unroll
        for (int e = 0; e < 32; ++e) sum[part][e] = 0.f;
      for (int k0 = 0; k0 < nkb; k0 += chunk_at(k0, nkb), ++it) {
        const int b = it & 1;
        ok = wait_for(acc_full0 + 8 * b, (uint32_t)(it >> 1) & 1u, 8u);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (there) {
#pragma unroll
          for (int part = 0; part < 2; ++part) {
            uint32_t v[32];
            umma::tmem_load_32(mine + (uint32_t)b * acc_cols + (uint32_t)(part * (nt / 2)), v);
#pragma unroll
            for (int e = 0; e < 32; ++e) sum[part][e] += __uint_as_float(v[e]);
          }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          if (PAIR) arrive_lightly(back0 + 8 * b);
          else umma::mbar_arrive(back0 + 8 * b);
        }
      }
      if (!ok) break;
      int i0, j0;
      tile_of<PAIR>(A, w, i0, j0);
      i0 += half * kTileM + q * 32;
      j0 = j0 / 2 + c0;
      // Z in 8 bits: a tile of 256 columns has a block of gates and one of ups.  A lane looks its row's through for their scales; the three
      // other warps of these rows have the other columns, and they tell one another what they found.
      float inv_g = 0.f, inv_u = 0.f;
      bool finite = true;
      if (A.z_codes) {
        float largest[2];
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          float x[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] = sum[part][e];
          if (A.bias) {
            const uint4* bias = reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(A.bias) + part * A.up + j0);
#pragma unroll
            for (int b8 = 0; b8 < 4; ++b8) {
              float b[8];
              Elem<T>::unpack(__ldg(bias + b8), b);
#pragma unroll
              for (int e = 0; e < 8; ++e) x[8 * b8 + e] += b[e];
            }
          }
          largest[part] = largest_rounded<T>(x, finite);
        }
        finite = __all_sync(0xffffffffu, finite);
        const int wi = warp - kFirstAdder;
        const auto all_four = [&]() {
          __syncwarp();
          if (lane == 0) umma::mbar_arrive(told);
          const bool done = wait_for(told, told_phase, 16u);
          told_phase ^= 1u;
          return done;
        };
        powers[wi][lane] = (signed char)scale_power(largest[0]);
        powers[wi][32 + lane] = (signed char)scale_power(largest[1]);
        ok = all_four();
        if (!ok) break;
        int kg = -126, ku = -126;
#pragma unroll
        for (int other = 0; other < 4; ++other) {
          kg = max(kg, (int)powers[4 * other + (wi & 3)][lane]);
          ku = max(ku, (int)powers[4 * other + (wi & 3)][32 + lane]);
        }
        // The next tile's are written behind its last chunk, which of three or more comes only when all warps have given back its first, and so
        // have read these; else they wait for one another.
        if (nkb <= 2 * kChunk) {
          ok = all_four();
          if (!ok) break;
        }
        inv_g = power_of_two(-kg);
        inv_u = power_of_two(-ku);
        if (c0 == 0 && i0 + lane < A.I) {
          float* to = A.z_scales + (long long)(i0 + lane) * A.ld_zs + j0 / kBlock;
          to[0] = power_of_two(kg);
          to[A.up / kBlock] = power_of_two(ku);
        }
      }
      if (!there) continue;
      // W gates and their ups of 32 rows through shared memory, after which W / 8 lanes share a row, or W neighbouring lanes have neighbouring
      // columns of eight rows
      constexpr int kRow = W / 8, kDown = 32 / kRow;          // lanes that share a row, rows at a time
      const auto at = [](int r, int p) { return W == 32 ? piece(r, p, 8) : narrow_piece(r, p); };
#pragma unroll
      for (int h = 0; h < 32; h += W) {
        float gu[2][kRow][8];
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          __syncwarp();
#pragma unroll
          for (int e = 0; e < W; e += 4)
            stage4[at(lane, e / 4)] = make_uint4(__float_as_uint(sum[part][h + e]), __float_as_uint(sum[part][h + e + 1]), __float_as_uint(sum[part][h + e + 2]),
                                                 __float_as_uint(sum[part][h + e + 3]));
          __syncwarp();
#pragma unroll
          for (int k = 0; k < kRow; ++k) {
            float (&x)[8] = gu[part][k];
            if (vec) {
              const int r = kDown * k + lane / kRow, p = 2 * (lane % kRow);
              const uint4 lo = stage4[at(r, p)], hi = stage4[at(r, p + 1)];
              x[0] = __uint_as_float(lo.x), x[1] = __uint_as_float(lo.y), x[2] = __uint_as_float(lo.z), x[3] = __uint_as_float(lo.w);
              x[4] = __uint_as_float(hi.x), x[5] = __uint_as_float(hi.y), x[6] = __uint_as_float(hi.z), x[7] = __uint_as_float(hi.w);
            } else {
              const int r = kDown * k + 8 * (lane / W), c = lane % W;
#pragma unroll
              for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(reinterpret_cast<const uint32_t*>(&stage4[at(r + e, c >> 2)])[c & 3]);
            }
          }
        }
#pragma unroll
        for (int k = 0; k < kRow; ++k) {
          const int r = kDown * k + lane / kRow;
          const float ig = __shfl_sync(0xffffffffu, inv_g, r), iu = __shfl_sync(0xffffffffu, inv_u, r);
          if (vec) finish_gated_row<T>(A, i0 + r, j0 + h + 8 * (lane % kRow), gu[0][k], gu[1][k], ig, iu, finite);
          else finish_gated_column<T>(A, A.I, i0 + kDown * k + 8 * (lane / W), j0 + h + lane % W, gu[0][k], gu[1][k]);
        }
      }
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

// ---- the gradient of Z ---------------------------------------------------------------------------------------------------
// dZ and its column sums.  Bound by memory.  A block takes 256 columns of the gates and of the ups (32 threads of eight) and a run
// of rows (8 threads); sums in fp32 of the unrounded products, to part[run][2F].  CODES: Z comes in 8 bits.
// At odd sizes and addresses (not VEC) 8-bit codes are read by the aligned words that hold a thread's eight columns (3001 x 2050: 34 us
// by single codes, 14 us so), 16-bit numbers one by one by neighbouring lanes (14 us; by words 26 us).
constexpr int kCols = 256, kThreads = 256;
// Blocks that an SM holds: codes at odd places need more registers (3001 x 2050: 17.4 us by three, 13.9 by two; 16-bit numbers in
// order, 8192 x 4096 with the product behind it: three 91 us, two 96, four 100).
__host__ __device__ constexpr int blocks_at_once(bool codes, bool vec) { return codes && !vec ? 2 : 3; }

template <class T, bool CODES, bool VEC>
__global__ void __launch_bounds__(kThreads, blocks_at_once(CODES, VEC)) gated_dz_kernel(const T* dh, long long lddh, const T* z, long long ldz, const Codes zq, T* dz, long long lddz,
                                                               float* part, long long M, long long F, int act, int rows_per) {
  __shared__ float sh[8][2 * kCols];
  allow_next();
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const long long base = (long long)blockIdx.x * kCols;
  const long long r0 = (long long)blockIdx.y * rows_per, r1 = min(r0 + (long long)rows_per, M);
  float sum[2][8] = {};
  // dG and dU of eight pairs, in place of the gates and the ups
  const auto slopes = [&](const float (&d)[8], float (&g)[8], float (&u)[8]) {
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const f32x2 gate = pair_of(g[e], g[e + 1]), up = pair_of(u[e], u[e + 1]), grad = pair_of(d[e], d[e + 1]);
      f32x2 value = gate, slope = both_of(1.f);
      if (act == LAQ_ACT_RELU) {
        float a[2], b[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          a[i] = g[e + i] > 0.f ? 1.f : (g[e + i] == g[e + i] ? 0.f : g[e + i]);
          b[i] = max_nan(g[e + i], 0.f);
        }
        slope = pair_of(a[0], a[1]);
        value = pair_of(b[0], b[1]);
      } else if (act == LAQ_ACT_GELU) {
        const f32x2 s = gelu_sigmoid2(gate);
        value = times2(gate, s);
        slope = fma2(times2(value, one_minus2(s)), gelu_inner2(gate), s);
      } else if (act == LAQ_ACT_SILU) {
        const f32x2 s = sigmoid2(gate);
        value = times2(gate, s);
        slope = times2(s, fma2(gate, one_minus2(s), both_of(1.f)));
      }
      split(times2(times2(grad, up), slope), g[e], g[e + 1]);
      split(times2(grad, value), u[e], u[e + 1]);
      sum[0][e] += g[e], sum[0][e + 1] += g[e + 1];
      sum[1][e] += u[e], sum[1][e + 1] += u[e + 1];
    }
  };
  constexpr bool kEights = VEC || CODES;          // a thread's columns are neighbours; else 32 apart, so that lanes are
  if constexpr (kEights) {
    const long long c0 = base + tx * 8;
    const int n = VEC ? (c0 < F ? 8 : 0) : (int)max(0ll, min(8ll, F - c0));            // of this thread's columns there are
    const bool up_vec = VEC || F % 8 == 0;
    const int here = kBlock - (int)((F + c0) % kBlock);                                // ups before the next block
    const auto rows = [&](long long r, auto edge) {          // r and, if it is there, r + 8
      const bool two = r + 8 < r1;
      uint4 d[2];
      [[maybe_unused]] uint4 g[2], u[2];                    // 16-bit projections, or
      [[maybe_unused]] uint2 qg[2], qu[2];                  // codes and their scales
      [[maybe_unused]] float sg[2], su[2], su_next[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const long long row = two || i == 0 ? r + 8 * i : r;             // a row is read twice rather than beyond the last
        const T* pd = dh + row * lddh + c0;
        d[i] = VEC ? load16(pd) : load16_any<true>(pd, n, decltype(edge)::value);
        if constexpr (CODES) {
          const uint8_t* p = zq.p + row * zq.ld + c0;
          qg[i] = VEC ? load8(p) : load8_any<true>(p, n, decltype(edge)::value);
          qu[i] = VEC ? load8(p + F) : load8_any<true>(p + F, n, decltype(edge)::value);
          sg[i] = zq.scale(row, c0);
          su[i] = zq.scale(row, F + c0);
          if (!VEC) su_next[i] = zq.scale(row, F + c0 + n - 1);        // eight ups may lie in two blocks
        } else {
          const T* p = z + row * ldz + c0;
          g[i] = load16(p);
          u[i] = load16(p + F);
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (i == 1 && !two) break;
        float df[8], gf[8], uf[8];
        Elem<T>::unpack(d[i], df);
        if constexpr (CODES) {
          decode8(qg[i], sg[i], gf);
          decode8(qu[i], VEC ? su[i] : 1.f, uf);
          if (!VEC) {
#pragma unroll
            for (int e = 0; e < 8; ++e) uf[e] *= e < here ? su[i] : su_next[i];
          }
        } else {
          Elem<T>::unpack(g[i], gf);
          Elem<T>::unpack(u[i], uf);
        }
        slopes(df, gf, uf);
        if (dz) {
          T* o = dz + (r + 8 * i) * lddz + c0;
          const uint4 dg = Elem<T>::pack(gf), du = Elem<T>::pack(uf);
          if (n == 8) *reinterpret_cast<uint4*>(o) = dg;                      // rows and eights of them are aligned
          else store16_any(o, dg, n);
          if (n == 8 && up_vec) *reinterpret_cast<uint4*>(o + F) = du;
          else store16_any(o + F, du, n);
        }
      }
    };
    if (n > 0) {
      for (long long r = r0 + ty; r < r1; r += 16) {
        if (!VEC && at_edge(r, r + 8, M, c0, F - c0 - 8, 1)) rows(r, std::true_type());
        else rows(r, std::false_type());
      }
    }
  } else {
    for (long long r = r0 + ty; r < r1; r += 8) {
      float df[8], gf[8], uf[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const long long c = base + tx + 32 * e;
        const bool there = c < F;
        df[e] = there ? Elem<T>::to_float(dh[r * lddh + c]) : 0.f;
        gf[e] = there ? Elem<T>::to_float(z[r * ldz + c]) : 0.f;
        uf[e] = there ? Elem<T>::to_float(z[r * ldz + F + c]) : 0.f;
      }
      slopes(df, gf, uf);
      if (dz) {
        T* o = dz + r * lddz;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const long long c = base + tx + 32 * e;
          if (c < F) {
            o[c] = Elem<T>::from_float(gf[e]);
            o[F + c] = Elem<T>::from_float(uf[e]);
          }
        }
      }
    }
  }
  if (!part) return;
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int e = 0; e < 8; ++e) sh[ty][h * kCols + (kEights ? tx * 8 + e : tx + 32 * e)] = sum[h][e];
  __syncthreads();
  const long long c = base + threadIdx.x;
  if (c >= F) return;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float t = 0.f;
#pragma unroll
    for (int y = 0; y < 8; ++y) t += sh[y][h * kCols + threadIdx.x];
    part[(long long)blockIdx.y * 2 * F + h * F + c] = t;
  }
}

// ---- host -----------------------------------------------------------------------------------------------------------------
constexpr long long kLongestSum = 65536;       // terms that a 16-bit result takes without chunks

laq_status check_call(const Err& e, const laq_gated_call* c, void* ws, size_t ws_bytes, size_t need) {
  if (e.buf && e.len) e.buf[0] = 0;
  if (!c) return fail(e.buf, e.len, LAQ_EINVAL, "null pointer");
  if (c->F < 1 || c->F > 0x3fffff00ll) return fail(e.buf, e.len, LAQ_EINVAL, "F must be 1..2^30-256");
  if (c->K > kLongestSum) return fail(e.buf, e.len, LAQ_EINVAL, "K must be 1..65536");
  return check_layer(e, c->dtype, c->M, 2 * c->F, c->K, c->activation, c->status, c->flags, ws, ws_bytes, need);
}

bool sizes_ok(const laq_gated_call* c) {
  return c && c->M >= 0 && c->M <= 0x7fffff00ll && c->F >= 1 && c->F <= 0x3fffff00ll && c->K >= 1 && c->K <= kLongestSum &&
         (c->dtype == LAQ_BF16 || c->dtype == LAQ_F16);
}

// Plain dot products, by the same rule as a layer's (laq_ops_linear.cu), for as many rows of W, but three and four rows of a large W
// that lies in order go as below (2 x 11008 x 4096: 38 us, so 32; 2 x 512 x 2048: 3.5 us, 4.1).
bool some_in_order(const laq_gated_call* c) { return mappable(c->x, c->ld_x) && mappable(c->w, c->ld_w); }
bool takes_few_rows(const laq_gated_call* c) {
  if (c->flags & LAQ_LINEAR_STARVE) return false;
  if (c->M > 2 && c->F >= (1ll << 24) / c->K && some_in_order(c)) return false;
  return c->M <= 2 || (c->M <= kFewRows && (c->K >= 1024 || 2 * c->F <= kFewCols * kFewThreads / 32 * kFewBlocks * kSMs));
}
// linear_some_rows_kernel.  Where the tiles of tensor memory overtake: 16 rows of 2 x 11008 x 4096 38.3 us (by tiles 38.4), of 2 x 4096 x
// 4096 16.6 (18.8); 32 rows of 2 x 4096 x 4096 26 us (20), of 2 x 4096 x 1024 12.4 (12.1), of 2 x 1501 x 1000 8.4 (10.9).
bool takes_some_rows(const laq_gated_call* c) {
  if ((c->flags & LAQ_LINEAR_STARVE) || takes_few_rows(c) || c->M > 32) return false;
  if (c->M > 8 && c->F > (c->M > 16 ? 1ll << 21 : 1ll << 25) / c->K) return false;
  if (c->M > 16 && c->K > 4096) return false;
  return some_in_order(c);
}

// Z in 8 bits leaves the epilogue where a tile has whole blocks of gates and of ups: 128 of each, not split, and vectors throughout.
// Else it is packed from 16 bits afterwards, with the same result.  4096 x 5504 x 2048: 147 us and 26 to pack it, 153 us in the epilogue.
bool packs_in_epilogue(const laq_gated_call* c) {
  if (!c->z_blocks || takes_few_rows(c) || takes_some_rows(c) || c->F % kBlock || !mappable(c->h, c->ld_h) || (c->bias && !mappable(c->bias, 8)) ||
      c->z_blocks->block_rows != 1 || !Codes(c->z_blocks).vectors(8))
    return false;
  const Plan pl = make_plan(c->M, 2 * c->F, c->K, false, false, true, false, false, kGated);
  return !pl.swap && pl.nt == 2 * kBlock && pl.split == 1;
}

struct ForwardNeeds {
  Operand x, w;
  size_t z_bytes;               // Z in 16 bits, before it is packed
  explicit ForwardNeeds(const laq_gated_call* c) : x{c->x, c->ld_x, c->M, c->K}, w{c->w, c->ld_w, 2 * c->F, c->K} {
    z_bytes = c->z_blocks && !packs_in_epilogue(c) ? align256((size_t)c->M * pad8(2 * c->F) * 2) : 0;
  }
  size_t bytes(const laq_gated_call* c) const { return z_bytes + (takes_few_rows(c) || takes_some_rows(c) ? 0 : x.pack_bytes() + w.pack_bytes()); }
};

bool dz_vectors(const laq_gated_call* c) {
  return c->F % 8 == 0 && mappable(c->dh, c->ld_dh) && (c->z_blocks ? Codes(c->z_blocks).vectors(8) : mappable(c->z, c->ld_z));
}

// Rows of a run: no more blocks than the SMs hold at once (8192 x 4096 with the product behind it: 592 blocks for 444 places 103 us, so
// 91 us), or as many rounds of them as leave a tenth less of the places empty; no fewer than 32 rows each, and no more than 2048, so that
// a thread adds up 256 numbers at most, one after another.
int rows_of_a_run(const laq_gated_call* c) {
  const long long M = c->M, cols = (c->F + kCols - 1) / kCols, places = blocks_at_once(c->z_blocks != nullptr, dz_vectors(c)) * kSMs;
  const long long least = M > 2048 ? (M + 2047) / 2048 : 1, first = (cols * least + places - 1) / places;
  long long runs = first * places / cols, rounds = first;
  for (long long k = first + 1; k < first + 8; ++k)
    if (10 * k * runs < 9 * rounds * (k * places / cols)) rounds = k, runs = k * places / cols;
  long long per = (M + runs - 1) / runs;
  per = per < 32 ? 32 : per;
  while ((M + per - 1) / per > 65535) per *= 2;
  return (int)per;
}

struct BackwardNeeds {
  size_t dz_bytes, part_bytes, x_bytes;
  Operand x, w, dz;
  explicit BackwardNeeds(const laq_gated_call* c)
      : x{c->x, c->ld_x, c->M, c->K}, w{c->w, c->ld_w, 2 * c->F, c->K}, dz{nullptr, pad8(2 * c->F), c->M, 2 * c->F} {
    const int per = rows_of_a_run(c);
    dz_bytes = c->dx || c->dw ? align256((size_t)c->M * dz.ld * 2) : 0;
    part_bytes = c->db ? align256((size_t)((c->M + per - 1) / per) * 2 * c->F * 4) : 0;
    if (c->x_blocks) x = Operand{nullptr, pad8(c->K), c->M, c->K};
    x_bytes = c->x_blocks && c->dw ? align256((size_t)c->M * x.ld * 2) : 0;
  }
  size_t bytes(const laq_gated_call* c) const {
    return dz_bytes + part_bytes + x_bytes + (c->dw ? x.pack_bytes() : 0) + (c->dx ? w.pack_bytes() : 0);
  }
};

template <class T, int ROWS>
laq_status launch_few(const Err& e, const GatedArgs& A, const Operand& x, const Operand& w, cudaStream_t st) {
  const int K = (int)x.cols, vec = x.mappable_() && w.mappable_(), items = vec ? K / 8 : K;
  const long long groups = (A.up + kFewCols / 2 - 1) / (kFewCols / 2);
  const int log_parts = few_log_parts(groups, items), per_block = kFewThreads / 32 >> log_parts;
  const auto kernel = ROWS <= 2 && items > 64 << log_parts ? linear_few_rows_kernel<T, ROWS, ROWS <= 2 ? 4 : 2, true>
                                                          : linear_few_rows_kernel<T, ROWS, 2, true>;
  return launched(e.buf, e.len, launch_plain(kernel, dim3((unsigned)((groups + per_block - 1) / per_block)), kFewThreads, st, A, (const T*)x.p, x.ld,
                                             (const T*)w.p, w.ld, K, vec, log_parts));
}

template <class T>
laq_status few_rows(const Err& e, const GatedArgs& A, const Operand& x, const Operand& w, cudaStream_t st) {
  switch (x.rows) {
    case 1: return launch_few<T, 1>(e, A, x, w, st);
    case 2: return launch_few<T, 2>(e, A, x, w, st);
    case 3: return launch_few<T, 3>(e, A, x, w, st);
    default: return launch_few<T, 4>(e, A, x, w, st);
  }
}

template <class T, bool PAIR, int W>
laq_status launch_whole(const Err& e, const Product<kGated>& p, bool follows, cudaStream_t st) {
  static Raised raised;
  GatedArgs A = p.A;
  const int stage = (kTileM + (PAIR ? A.nt / 2 : A.nt)) * kBlockK * 2, most = (kMaxRing + kStaging - kAdders * handed_bytes(W)) / stage;
  if (A.stages > most) A.stages = most;
  return launch_tiles<GatedArgs, CUtensorMap, CUtensorMap>(e, gated_gemm_kernel<T, PAIR, W>, raised, kGatedThreads, PAIR, false, kAdders * handed_bytes(W), follows,
                                                           st, A, p.ma, p.mb);
}
// Whole sums of more than 1024 terms, or Z in 8 bits, take gated_gemm_kernel; shorter ones are up to a tenth faster by linear_gemm_kernel's fewer
// threads (300 x 64 x 64 5.8 us, 6.6; 517 x 1501 x 1000 14.5, 15.8), and their cuts do not show in 16 bits.
template <class T>
laq_status launch_product(const Err& e, const Product<kGated>& p, bool follows, cudaStream_t st) {
  const bool adds = !p.pl.swap && p.pl.split == 1 && (p.A.nkb > kShortSum || p.A.z_codes);
  if (p.pl.pair)
    return !adds                      ? launch_gemm<T, false, true, false, false, kGated>(e, p.ma, p.mb, p.A, follows, st)
           : p.A.z || p.A.z_codes ? launch_whole<T, true, 32>(e, p, follows, st)
                                      : launch_whole<T, true, 16>(e, p, follows, st);
  if (p.pl.swap) return launch_gemm<T, true, false, false, false, kGated>(e, p.ma, p.mb, p.A, follows, st);
  return adds ? launch_whole<T, false, 16>(e, p, follows, st) : launch_gemm<T, false, false, false, false, kGated>(e, p.ma, p.mb, p.A, follows, st);
}

template <class T>
void list_kernels(const void** list, int& n) {
  const void* all[] = {(const void*)linear_gemm_kernel<T, false, false, false, false, kGated>, (const void*)linear_gemm_kernel<T, true, false, false, false, kGated>,
                       (const void*)gated_gemm_kernel<T, true, 16>, (const void*)gated_gemm_kernel<T, true, 32>, (const void*)gated_gemm_kernel<T, false, 16>,
                       (const void*)linear_gemm_kernel<T, false, true, false, false, kGated>,
                       (const void*)linear_few_rows_kernel<T, 1, 4, true>, (const void*)linear_few_rows_kernel<T, 1, 2, true>,
                       (const void*)linear_few_rows_kernel<T, 2, 4, true>, (const void*)linear_few_rows_kernel<T, 2, 2, true>,
                       (const void*)linear_few_rows_kernel<T, 3, 2, true>, (const void*)linear_few_rows_kernel<T, 4, 2, true>,
                       (const void*)linear_some_rows_kernel<T, 1, false>, (const void*)linear_some_rows_kernel<T, 2, false>,
                       (const void*)linear_some_rows_kernel<T, 4, false>,
                       (const void*)gated_dz_kernel<T, false, false>, (const void*)gated_dz_kernel<T, false, true>,
                       (const void*)gated_dz_kernel<T, true, false>, (const void*)gated_dz_kernel<T, true, true>};
  for (const void* k : all) list[n++] = k;
}

// Its own kernels, and those of the products and of the 8-bit matrices that its calls may use.
laq_status load_kernels(const Err& e) {
  static Loaded loaded;
  static const void* list[64];
  static const int n = [] {
    int count = 0;
    list_kernels<__nv_bfloat16>(list, count);
    list_kernels<__half>(list, count);
    return count;
  }();
  LAQ_TRY(launched(e.buf, e.len, loaded.once(list, n)));
  LAQ_TRY(load_layer_kernels(e));
  return load_block_kernels(e);
}

}  // namespace
}  // namespace ops
}  // namespace laq

using namespace laq::ops;

extern "C" size_t laq_gated_workspace_bytes(const laq_gated_call* c, int32_t backward) {
  if (!sizes_ok(c)) return 0;
  return backward ? BackwardNeeds(c).bytes(c) : ForwardNeeds(c).bytes(c);
}

extern "C" laq_status laq_gated_forward(const laq_gated_call* c, void* d_workspace, size_t workspace_bytes, void* cuda_stream, char* errbuf,
                                        size_t errbuf_len) {
  const Err e{errbuf, errbuf_len};
  const size_t ws_bytes = laq_gated_workspace_bytes(c, 0);
  LAQ_TRY(check_call(e, c, d_workspace, workspace_bytes, ws_bytes));
  if (c->z && c->z_blocks) return fail(errbuf, errbuf_len, LAQ_EINVAL, "z and z_blocks are both given");
  if (c->M == 0) return LAQ_OK;
  const long long N = 2 * c->F;
  Buffers buffers;
  buffers.out("status", c->status, 4, 1, 1, 1);
  if (ws_bytes) buffers.out("the workspace", d_workspace, 1, 1, (long long)ws_bytes, (long long)ws_bytes);
  LAQ_TRY(check_tensor(e, buffers, "x", kRead, c->x, true, c->M, c->ld_x, c->K, 2));
  LAQ_TRY(check_tensor(e, buffers, "w", kRead, c->w, true, N, c->ld_w, c->K, 2));
  LAQ_TRY(check_tensor(e, buffers, "bias", kRead, c->bias, false, 1, N, N, 2));
  LAQ_TRY(check_tensor(e, buffers, "h", kWritten, c->h, true, c->M, c->ld_h, c->F, 2));
  if (c->z_blocks) LAQ_TRY(check_blocks(e, buffers, "z", "the scales of z", kWritten, c->z_blocks, c->M, N));
  else LAQ_TRY(check_tensor(e, buffers, "z", kWritten, c->z, false, c->M, c->ld_z, N, 2));
  LAQ_TRY(buffers.check(errbuf, errbuf_len));
  LAQ_TRY(load_kernels(e));
  cudaStream_t st = (cudaStream_t)cuda_stream;
  ForwardNeeds need(c);
  char* ws = (char*)d_workspace;
  GatedArgs A = {};
  A.I = (int)c->M;
  A.J = (int)c->F;
  A.up = c->F;
  A.act = c->activation;
  A.starve = (c->flags & LAQ_LINEAR_STARVE) != 0;
  A.out = c->h;
  A.ldo = c->ld_h;
  A.z = c->z;
  A.ldz = c->ld_z;
  A.bias = c->bias;
  A.status = c->status;
  if (need.z_bytes) {
    A.z = ws;
    A.ldz = pad8(N);
    ws += need.z_bytes;
  } else if (c->z_blocks) {
    A.z_codes = (uint8_t*)const_cast<void*>(c->z_blocks->codes);
    A.z_scales = const_cast<float*>(c->z_blocks->scales);
    A.ld_zc = c->z_blocks->ld_codes;
    A.ld_zs = c->z_blocks->ld_scales;
  }
  const bool bf16 = c->dtype == LAQ_BF16;
  if (takes_some_rows(c)) {
    LAQ_TRY(bf16 ? some_rows<__nv_bfloat16, false>(e, A, c->x, 2 * c->ld_x, c->w, 2 * c->ld_w, 2 * c->K, st)
                 : some_rows<__half, false>(e, A, c->x, 2 * c->ld_x, c->w, 2 * c->ld_w, 2 * c->K, st));
  } else if (takes_few_rows(c)) {
    LAQ_TRY(bf16 ? few_rows<__nv_bfloat16>(e, A, need.x, need.w, st) : few_rows<__half>(e, A, need.x, need.w, st));
  } else {
    const char* before = ws;
    LAQ_TRY(make_mappable(e, need.x, ws, st));
    LAQ_TRY(make_mappable(e, need.w, ws, st));
    const bool follows = ws != before;
    Product<kGated> p;
    p.A = A;
    LAQ_TRY(prepare_product(e, p, need.x, need.w, bf16 ? 1 : 0));
    LAQ_TRY(bf16 ? launch_product<__nv_bfloat16>(e, p, follows, st) : launch_product<__half>(e, p, follows, st));
  }
  if (need.z_bytes) return pack_blocks(e, A.z, c->dtype, c->M, N, A.ldz, *c->z_blocks, st);
  return LAQ_OK;
}

extern "C" laq_status laq_gated_backward(const laq_gated_call* c, void* d_workspace, size_t workspace_bytes, void* cuda_stream, char* errbuf,
                                         size_t errbuf_len) {
  const Err e{errbuf, errbuf_len};
  const size_t ws_bytes = laq_gated_workspace_bytes(c, 1);
  LAQ_TRY(check_call(e, c, d_workspace, workspace_bytes, ws_bytes));
  if (!c->dx && !c->dw && !c->db) return LAQ_OK;
  if (c->z && c->z_blocks) return fail(errbuf, errbuf_len, LAQ_EINVAL, "z and z_blocks are both given");
  if (c->x && c->x_blocks) return fail(errbuf, errbuf_len, LAQ_EINVAL, "x and x_blocks are both given");
  const long long N = 2 * c->F;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  Buffers buffers;
  buffers.out("status", c->status, 4, 1, 1, 1);
  if (ws_bytes) buffers.out("the workspace", d_workspace, 1, 1, (long long)ws_bytes, (long long)ws_bytes);
  LAQ_TRY(check_tensor(e, buffers, "dw", kWritten, c->dw, false, N, c->ld_dw, c->K, 2));
  LAQ_TRY(check_tensor(e, buffers, "db", kWritten, c->db, false, 1, N, N, 4));
  const Gradients to{c->dx, c->ld_dx, c->dw, c->ld_dw, 0};
  if (c->M == 0) {
    LAQ_TRY(buffers.check(errbuf, errbuf_len));
    return zero_gradients(e, to, c->db, N, c->K, st);
  }
  LAQ_TRY(check_tensor(e, buffers, "dh", kRead, c->dh, true, c->M, c->ld_dh, c->F, 2));
  if (c->z_blocks) LAQ_TRY(check_blocks(e, buffers, "z", "the scales of z", kRead, c->z_blocks, c->M, N));
  else LAQ_TRY(check_tensor(e, buffers, "z", kRead, c->z, true, c->M, c->ld_z, N, 2));
  if (c->dw) {
    if (c->x_blocks) LAQ_TRY(check_blocks(e, buffers, "x", "the scales of x", kRead, c->x_blocks, c->M, c->K));
    else LAQ_TRY(check_tensor(e, buffers, "x", kRead, c->x, true, c->M, c->ld_x, c->K, 2));
  }
  if (c->dx) LAQ_TRY(check_tensor(e, buffers, "w", kRead, c->w, true, N, c->ld_w, c->K, 2));
  LAQ_TRY(check_tensor(e, buffers, "dx", kWritten, c->dx, false, c->M, c->ld_dx, c->K, 2));
  LAQ_TRY(buffers.check(errbuf, errbuf_len));
  LAQ_TRY(load_kernels(e));
  BackwardNeeds need(c);
  char* ws = (char*)d_workspace;
  void* dz = need.dz_bytes ? ws : nullptr;
  float* part = c->db ? (float*)(ws + need.dz_bytes) : nullptr;
  ws += need.dz_bytes + need.part_bytes;
  const int per = rows_of_a_run(c), runs = (int)((c->M + per - 1) / per);
  const dim3 grid((unsigned)((c->F + kCols - 1) / kCols), (unsigned)runs);
  const Codes zq(c->z_blocks);
  const bool vec = dz_vectors(c);
  const auto launch_dz = [&](auto zero) {
    using T = decltype(zero);
    const auto kernel = c->z_blocks ? (vec ? gated_dz_kernel<T, true, true> : gated_dz_kernel<T, true, false>)
                                    : (vec ? gated_dz_kernel<T, false, true> : gated_dz_kernel<T, false, false>);
    return launch_plain(kernel, grid, kThreads, st, (const T*)c->dh, c->ld_dh, (const T*)c->z, c->ld_z, zq, (T*)dz, need.dz.ld, part, c->M, c->F,
                        c->activation, per);
  };
  LAQ_TRY(launched(errbuf, errbuf_len, c->dtype == LAQ_BF16 ? launch_dz(__nv_bfloat16()) : launch_dz(__half())));
  if (c->db) LAQ_TRY(column_sums(e, part, runs, (int)N, c->db, st));
  need.dz.p = dz;
  if (need.x_bytes) {
    need.x.p = ws;
    ws += need.x_bytes;
    LAQ_TRY(unpack_blocks(e, *c->x_blocks, c->M, c->K, c->dtype, const_cast<void*>(need.x.p), need.x.ld, st));
  }
  return gradient_products(e, c->dtype, need.dz, need.x, need.w, to, ws, c->status, (c->flags & LAQ_LINEAR_STARVE) != 0, true, true, st);
}
