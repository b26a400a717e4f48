// Both products of a layer's gradient in one launch:  dX = dZ W  and  dW = dZ^T X,  of 16-bit operands, to 16 bits.
//
// Pairs of SMs take tiles of 256 x NT of either product, one after another.  By themselves the products leave the last round of
// tiles partly empty (8192 x 2048 of a sum over 8192: 256 tiles for 74 pairs, four rounds for 3.5), together they have one such
// round between them, and no start in the middle.  A tile's sum runs in the same order as in linear_gemm_kernel, with the same result.
// With the operands as they lie, the summed index of dX is contiguous in dZ alone and that of dW in neither operand.
#include "laq_ops_gemm.cuh"

namespace laq {
namespace ops {
namespace {

struct OneProduct {
  int I, J, nkb, tiles_i, tiles_j, a_mn;
  long long ldo;
  void* out;
};
struct BothArgs {
  OneProduct of[2];              // the one with the longer sum first
  int nt, stages, fmt, starve;
  uint32_t* status;
};

// As tile_of: tile rows are swept in groups, so that operands are found in L2.
__device__ __forceinline__ void tile_at(const OneProduct& P, int nt, int w, int& i0, int& j0) {
  constexpr int kGroup = kGroupTiles / 2;
  const int group = kGroup * P.tiles_j, g = w / group, in = w - g * group, top = g * kGroup, rows = min(kGroup, P.tiles_i - top);
  i0 = (top + in % rows) * 2 * kTileM;
  j0 = in / rows * nt;
}

template <class T>
__global__ void __launch_bounds__(kGemmThreads, 1)
    gradients_gemm_kernel(const __grid_constant__ CUtensorMap tmA0, const __grid_constant__ CUtensorMap tmB0, const __grid_constant__ CUtensorMap tmA1,
                          const __grid_constant__ CUtensorMap tmB1, const __grid_constant__ BothArgs A) {
  extern __shared__ unsigned char both_smem_raw[];
  __shared__ uint64_t bars[2 * kMaxStages + 5];
  __shared__ uint32_t tmem_base_sh;
  __shared__ int abort_sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, nt = A.nt, stages = A.stages, b_rows = nt / 2;
  const uint32_t base = umma::smem_u32(both_smem_raw), smem0 = (base + 1023u) & ~1023u;
  const uint32_t a_bytes = kTileM * kBlockK * 2, st_bytes = a_bytes + (uint32_t)b_rows * kBlockK * 2;
  const int half = (int)(blockIdx.x & 1u);
  const uint32_t full0 = umma::smem_u32(&bars[0]), empty0 = umma::smem_u32(&bars[kMaxStages]);
  const uint32_t acc_full0 = umma::smem_u32(&bars[2 * kMaxStages]), acc_empty0 = acc_full0 + 16, drain = acc_full0 + 32;
  const uint32_t acc_cols = umma::tmem_cols(nt), held_cols = 2 * acc_cols;
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      umma::mbar_init(full0 + 8 * s, 1);
      umma::mbar_init(empty0 + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      umma::mbar_init(acc_full0 + 8 * b, 1);
      umma::mbar_init(acc_empty0 + 8 * b, 2 * kEpiWarps);
    }
    umma::mbar_init(drain, 1);
    abort_sh = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(umma::smem_u32(&tmem_base_sh)), "r"(held_cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  cg::this_cluster().sync();                       // both blocks' barriers are there before either signals the other's
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem_base = tmem_base_sh;
  allow_next();
  await_previous();

  const int split_at = A.of[0].tiles_i * A.of[0].tiles_j, tiles = split_at + A.of[1].tiles_i * A.of[1].tiles_j;
  const int first = (int)(blockIdx.x / 2), step = (int)(gridDim.x / 2);
  const uint32_t limit = A.starve ? kStarvedLimit : umma::kWaitLimit;
  volatile int* abort_flag = &abort_sh;

  if (warp == 0) {
    if (elect_one()) {
      int n = 0;                       // stages handed out so far
      bool ok = !(A.starve && blockIdx.x == 0);
      for (int w = first; w < tiles && ok; w += step) {
        const int which = w >= split_at;
        const OneProduct& P = A.of[which];
        const CUtensorMap *ma = which ? &tmA1 : &tmA0, *mb = which ? &tmB1 : &tmB0;
        int i0, j0;
        tile_at(P, nt, which ? w - split_at : w, i0, j0);
        i0 += half * kTileM;
        j0 += half * b_rows;
        const int nkb = P.nkb, a_mn = P.a_mn;
        for (int kb = 0; kb < nkb; ++kb, ++n) {
          const int s = n % stages;
          ok = umma::mbar_wait_abortable(empty0 + 8 * s, ((uint32_t)(n / stages) & 1u) ^ 1u, limit, abort_flag, A.status, 1u);
          if (!ok) break;
          const uint32_t sa = smem0 + s * st_bytes, sb = sa + a_bytes;
          const int r = kb * kBlockK;
          // the pair's first block counts the bytes of both; its phase cannot end before its own arrival here
          if (half == 0) umma::mbar_expect_tx(full0 + 8 * s, 2 * st_bytes);
          const uint32_t bar = of_leader(full0 + 8 * s);
          if (a_mn) {
            tma_load_2d_pair(sa, ma, bar, i0, r);
            tma_load_2d_pair(sa + 8192, ma, bar, i0 + 64, r);
          } else {
            tma_load_2d_pair(sa, ma, bar, r, i0);
          }
          for (int b = 0; b < b_rows; b += 64) tma_load_2d_pair(sb + b * 128, mb, bar, j0 + b, r);
        }
      }
      if (!ok)                          // given up: as in linear_gemm_kernel
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    }
  } else if (warp == 1) {
    if (half == 0 && elect_one()) {     // the pair's first block issues the products of both
      int n = 0, it = 0;
      bool ok = true;
      for (int w = first; w < tiles && ok; w += step, ++it) {
        const OneProduct& P = A.of[w >= split_at];
        const int nkb = P.nkb, a_mn = P.a_mn;
        const uint32_t idesc = instr_desc(A.fmt, a_mn, 1, nt, 2 * kTileM), step_a = a_mn ? 128u : 2u, step_b = 128u;
        const int b = it & 1;
        ok = umma::mbar_wait_abortable(acc_empty0 + 8 * b, ((uint32_t)(it >> 1) & 1u) ^ 1u, limit, abort_flag, A.status, 2u);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t d = tmem_base + (uint32_t)b * acc_cols;
        for (int kb = 0; kb < nkb; ++kb, ++n) {
          const int s = n % stages;
          ok = umma::mbar_wait_abortable(full0 + 8 * s, (uint32_t)(n / stages) & 1u, limit, abort_flag, A.status, 4u);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t sa = smem0 + s * st_bytes;
          const uint64_t da = a_mn ? desc_mn_major(sa) : desc_k_major(sa), db = desc_mn_major(sa + a_bytes);
#pragma unroll
          for (int kk = 0; kk < kBlockK / 16; ++kk) mma_pair(d, da + kk * step_a, db + kk * step_b, idesc, kb != 0 || kk != 0 ? 1u : 0u);
          commit_pair(empty0 + 8 * s);
        }
        if (ok) commit_pair(acc_full0 + 8 * b);
      }
      if (!ok) {                        // products under way still read the ring and write tensor memory
        commit_pair(drain);
        for (uint32_t i = 0; i < umma::kWaitLimit && !umma::mbar_try_wait(drain, 0u); ++i) {
        }
      }
    }
    __syncwarp();
  } else {
    const int q = warp & 3, set = (warp - 2) >> 2;
    uint4* stage4 = reinterpret_cast<uint4*>(both_smem_raw + (smem0 - base) + (size_t)stages * st_bytes) + (warp - 2) * 256;         // 4 KB of this warp
    int it = 0;
    for (int w = first; w < tiles; w += step, ++it) {
      const int which = w >= split_at;
      const OneProduct& P = A.of[which];
      int i0, j0;
      tile_at(P, nt, which ? w - split_at : w, i0, j0);
      i0 += half * kTileM + q * 32;
      const int I = P.I, J = P.J;
      const long long ldo = P.ldo;
      T* const out = reinterpret_cast<T*>(P.out);
      const bool vec = aligned16(out, ldo * 2), pairs = (((uintptr_t)out | (uintptr_t)(ldo * 2)) & 3u) == 0;
      const int b = it & 1;
      const uint32_t acc_limit = A.starve ? kStarvedLimit : umma::kWaitLimit;
      const bool ok = __all_sync(0xffffffffu, umma::mbar_wait_abortable(acc_full0 + 8 * b, (uint32_t)(it >> 1) & 1u, acc_limit, abort_flag, A.status, 8u));
      if (!ok) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t t0 = tmem_base + (uint32_t)b * acc_cols + ((uint32_t)(q * 32) << 16);
#pragma unroll 1
      for (int c0 = 32 * set; c0 < nt; c0 += 64) {
        uint32_t v[32];
        umma::tmem_load_32(t0 + (uint32_t)c0, v);
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 32; e += 4) stage4[piece(lane, e / 4, 8)] = make_uint4(v[e], v[e + 1], v[e + 2], v[e + 3]);
        __syncwarp();
        if (vec) {                      // four lanes share a row
          const int j = j0 + c0 + 8 * (lane & 3);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int r = 8 * k + (lane >> 2), i = i0 + r;
            const uint4 lo = stage4[piece(r, 2 * (lane & 3), 8)], hi = stage4[piece(r, 2 * (lane & 3) + 1, 8)];
            const float x[8] = {__uint_as_float(lo.x), __uint_as_float(lo.y), __uint_as_float(lo.z), __uint_as_float(lo.w),
                                __uint_as_float(hi.x), __uint_as_float(hi.y), __uint_as_float(hi.z), __uint_as_float(hi.w)};
            T* to = out + (long long)i * ldo + j;
            if (i < I && j + 8 <= J) {
              *reinterpret_cast<uint4*>(to) = Elem<T>::pack(x);
            } else if (i < I) {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (j + e < J) to[e] = Elem<T>::from_float(x[e]);
            }
          }
        } else if (pairs) {             // rows that allow four bytes: sixteen lanes share a row
          const int j = j0 + c0 + 2 * (lane & 15);
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            const int r = 2 * k + (lane >> 4), i = i0 + r;
            const float* x = reinterpret_cast<const float*>(&stage4[piece(r, (lane & 15) >> 1, 8)]) + 2 * (lane & 1);
            T* to = out + (long long)i * ldo + j;
            if (i < I && j + 2 <= J) {
              const T two[2] = {Elem<T>::from_float(x[0]), Elem<T>::from_float(x[1])};
              *reinterpret_cast<uint32_t*>(to) = *reinterpret_cast<const uint32_t*>(two);
            } else if (i < I && j < J) {
              to[0] = Elem<T>::from_float(x[0]);
            }
          }
        } else {
          const int j = j0 + c0 + lane;
#pragma unroll 8
          for (int r = 0; r < 32; ++r)
            if (i0 + r < I && j < J)
              out[(long long)(i0 + r) * ldo + j] = Elem<T>::from_float(reinterpret_cast<const float*>(&stage4[piece(r, lane >> 2, 8)])[lane & 3]);
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) arrive_at(of_leader(acc_empty0 + 8 * b));
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncwarp();
  cg::this_cluster().sync();                       // neither block's memory is used by the other any more
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(held_cols) : "memory");
  }
}

// ---- host -----------------------------------------------------------------------------------------------------------------
struct Form {
  int nt;
  double cost;
};
// By make_plan's constants for a pair's tiles: its first pair has the most of the tiles that come first.
Form both_form(long long M, long long N, long long K) {
  Form best{256, 1e300};
  for (int nt = 128; nt <= 256; nt += 128) {
    const double per = 2.7 * nt > (kTileM + nt / 2) * kBlockK * 2 / 60.0 ? 2.7 * nt : (kTileM + nt / 2) * kBlockK * 2 / 60.0;
    const long long cols = (K + nt - 1) / nt, P = kSMs / 2;
    const long long nx = (M + 255) / 256 * cols, nw = (N + 255) / 256 * cols;          // tiles of dX and of dW
    const double kx = (double)((N + kBlockK - 1) / kBlockK), kw = (double)((M + kBlockK - 1) / kBlockK);
    const long long n0 = kx >= kw ? nx : nw, rounds0 = (n0 + P - 1) / P, rounds = (nx + nw + P - 1) / P;
    const double k0 = kx >= kw ? kx : kw, k1 = kx >= kw ? kw : kx, epi = 2000 + 9.0 * nt;
    const auto tile = [&](double k) { return k * per > epi ? k * per : epi; };
    const double cost = 4500 + rounds0 * tile(k0) + (rounds - rounds0) * tile(k1) + epi;
    if (cost < best.cost) best = Form{nt, cost};
  }
  return best;
}

template <class T>
laq_status launch_both(const Err& e, const CUtensorMap (&m)[4], const BothArgs& A, bool follows, cudaStream_t st) {
  static Raised raised;
  const auto kernel = gradients_gemm_kernel<T>;
  LAQ_TRY(raise_shared_memory(e, (const void*)kernel, raised));
  const long long tiles = (long long)A.of[0].tiles_i * A.of[0].tiles_j + (long long)A.of[1].tiles_i * A.of[1].tiles_j;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * (tiles < kSMs / 2 ? tiles : kSMs / 2)));
  cfg.blockDim = dim3(kGemmThreads);
  cfg.dynamicSmemBytes = (size_t)A.stages * (kTileM + A.nt / 2) * kBlockK * 2 + kStaging + 1024;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  cfg.attrs = at;
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = 2;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.numAttrs = follows ? 2 : 1;
  return launched(e.buf, e.len, cudaLaunchKernelEx(&cfg, kernel, m[0], m[1], m[2], m[3], A));
}

}  // namespace

bool both_pay(long long M, long long N, long long K, bool whole) {
  if (M > kLongSum || N > kLongSum) return false;
  const Plan dx = make_plan(M, K, N, false, true, true, false, false), dw = make_plan(N, K, M, true, true, false, false, false);
  if (!whole && (dx.split > 1 || dw.split > 1)) return false;
  // The second launch costs 4000 cycles at least.  The estimates compare tiles of one width well and those of two widths badly: where a
  // product takes wider tiles by itself, one launch has to promise 15 % less.  Measured against two launches, 509 gradients of 16 to
  // 16384 rows that the estimates alone would join: with tiles as wide as theirs (442) all take 3 to 38 % less (8192 x 4096 x 2048
  // 235 us apart, 227 together, 4096 x 4096 x 512 71 and 44); with narrower ones that promise as much 12 take 13 % less to 1 % more,
  // of the 55 others 23 took up to 35 % more (8192 x 11008 x 784 363 and 491) and none took more than 16 % less.
  const Form form = both_form(M, N, K);
  return form.cost < (form.nt >= dx.nt && form.nt >= dw.nt ? 1.0 : 0.85) * (dx.cost + dw.cost + 4000);
}

laq_status both_products(const Err& e, int dtype, const Operand& dz, const Operand& x, const Operand& w, const Gradients& to, uint32_t* status, int starve,
                         bool follows, cudaStream_t st) {
  const long long M = dz.rows, N = dz.cols, K = x.cols;
  BothArgs A = {};
  A.nt = both_form(M, N, K).nt;
  A.fmt = dtype == LAQ_BF16 ? 1 : 0;
  A.starve = starve;
  A.status = status;
  A.stages = kMaxRing / ((kTileM + A.nt / 2) * kBlockK * 2);
  const auto product_of = [&](long long rows, long long sum, int a_mn, void* out, long long ldo) {
    return OneProduct{(int)rows, (int)K, (int)((sum + kBlockK - 1) / kBlockK), (int)((rows + 255) / 256), (int)((K + A.nt - 1) / A.nt), a_mn, ldo, out};
  };
  const int x_first = N >= M ? 1 : 0;                // dX's sum is over N, dW's over M
  A.of[x_first ? 0 : 1] = product_of(M, N, 0, to.dx, to.ld_dx);
  A.of[x_first ? 1 : 0] = product_of(N, M, 1, to.dw, to.ld_dw);
  CUtensorMap m[4];
  const int ix = x_first ? 0 : 2, iw = x_first ? 2 : 0;
  if (!umma::make_map_bf16_2d(&m[ix], dz.p, dz.rows, dz.cols, dz.ld * 2, kTileM) || !umma::make_map_bf16_2d(&m[ix + 1], w.p, w.rows, w.cols, w.ld * 2, 64) ||
      !umma::make_map_bf16_2d(&m[iw], dz.p, dz.rows, dz.cols, dz.ld * 2, 64) || !umma::make_map_bf16_2d(&m[iw + 1], x.p, x.rows, x.cols, x.ld * 2, 64))
    return fail(e.buf, e.len, LAQ_ECUDA, "a tensor map was refused");
  return dtype == LAQ_BF16 ? launch_both<__nv_bfloat16>(e, m, A, follows, st) : launch_both<__half>(e, m, A, follows, st);
}

void list_both_kernels(const void** list, int& n) {
  list[n++] = (const void*)gradients_gemm_kernel<__nv_bfloat16>;
  list[n++] = (const void*)gradients_gemm_kernel<__half>;
}

}  // namespace ops
}  // namespace laq
