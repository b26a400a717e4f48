// A layer's product with bias, activation and residual in its epilogue, and its gradient:
//   Z = X W^T + b,  Y = act(Z) + R            X [M][K], W [N][K], b [N], R, Y, Z [M][N]
//   dZ = dY act'(Z),  dX = dZ W,  dW = dZ^T X,  db = column sums of dZ
// bf16 or fp16 operands, fp32 accumulation on the tcgen05 tensor cores, bias, activation and residual in fp32, one
// rounding per stored value.  dZ is rounded once to the operands' type, which the two products of the gradient need
// (exact for no activation and for ReLU; with the others dX and dW carry it beside their own, in bf16 0.0023 of the result, root
// mean square, where one rounding makes 0.0017: two 16-bit parts of dZ would double both products).
//
// The products are linear_gemm_kernel (laq_ops_gemm.cuh); both of a gradient are gradients_gemm_kernel (laq_ops_gradients.cu) where that
// is the faster; one to four rows of X are plain dot products.
#include "laq_ops_gemm.cuh"

namespace laq {
namespace ops {
namespace {

// ---- dZ and the column sums ---------------------------------------------------------------------------------------------
// Bound by memory: 8192 x 4096 with gelu 39 us, 201 MB, 5.2 TB/s (0.79; two special-function and some twenty other
// operations an element come near).  A block takes 256 columns (32 threads of eight) and a run of rows (8 threads, two rows at a time): dZ = dY act'(Z), stored
// once if dz is given, and the sum of its columns over the run, in fp32 of the UNROUNDED products, to part[run][N].
constexpr int kDzCols = 256, kDzThreads = 256;

// CODES: Z comes in 8 bits (`zq`), 8 codes and their scale for a thread's columns.
template <class T, bool CODES>
__global__ void __launch_bounds__(kDzThreads, 4) linear_dz_kernel(const T* dy, long long lddy, const T* z, long long ldz, const Codes zq, T* dz,
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
      for (int e = 0; e < 8; e += 2) split(times2(pair_of(g[e], g[e + 1]), slope_gelu2(pair_of(x[e], x[e + 1]))), g[e], g[e + 1]);
    } else if (act == LAQ_ACT_SILU) {
#pragma unroll
      for (int e = 0; e < 8; e += 2) split(times2(pair_of(g[e], g[e + 1]), slope_silu2(pair_of(x[e], x[e + 1]))), g[e], g[e + 1]);
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
      float g[8], x[8];
      if constexpr (CODES) {
        const uint2 q0 = load8(zq.p + r * zq.ld + c0), q1 = two ? load8(zq.p + (r + 8) * zq.ld + c0) : make_uint2(0u, 0u);
        const float s0 = zq.scale(r, c0), s1 = two ? zq.scale(r + 8, c0) : 0.f;
        Elem<T>::unpack(g0, g);
        decode8(q0, s0, x);
        row(r, g, x);
        if (two) {
          Elem<T>::unpack(g1, g);
          decode8(q1, s1, x);
          row(r + 8, g, x);
        }
        continue;
      }
      uint4 x0 = g0, x1 = g1;
      if (act != LAQ_ACT_NONE) {
        x0 = load16(px + r * ldz);
        if (two) x1 = load16(px + (r + 8) * ldz);
      }
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
      if constexpr (CODES) decode8(load8_any(zq.p + r * zq.ld + c0, min(8, N - c0), at_edge(r, r, M, c0, N - c0 - 8, 1)), zq.scale(r, c0), x);
      // all sixteen numbers before the first is converted (8192 x 4097, SiLU: 51 us, one by one 59)
      const T *pg = dy + r * lddy + c0, *px = z + r * ldz + c0;
      T gs[8], xs[8];
      const bool also = !CODES && act != LAQ_ACT_NONE;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        gs[e] = c0 + e < N ? pg[e] : T(0.f);
        xs[e] = also && c0 + e < N ? px[e] : T(0.f);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        g[e] = Elem<T>::to_float(gs[e]);
        if constexpr (CODES) x[e] = c0 + e < N ? x[e] : 0.f;
        else x[e] = Elem<T>::to_float(xs[e]);
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

// Rows that a tensor map cannot describe (an address or a row pitch that is no multiple of 16 bytes) are copied once
// into the workspace with a pitch of a multiple of eight elements.
__global__ void __launch_bounds__(256) linear_pack_kernel(const uint16_t* src, long long ld, uint16_t* dst, long long pitch,
                                                          long long rows, int cols) {
  allow_next();
  const int groups = (cols + 7) / 8;
  const long long n = rows * groups, stride = (long long)gridDim.x * blockDim.x;
  const bool few = n <= 256 * kSMs;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += stride) {
    const long long r = i / groups;
    const int c = (int)(i - r * groups) * 8;
    const uint16_t* s = src + r * ld + c;
    // What lies behind a row's last number is never looked at: the tensor map ends with the row.  Numbers one by one at the matrix's
    // two ends, and where the copy is short and takes its latency (16 x 331 x 42 7.8 us, by words 8.2; 8192 x 1001 x 4095 93 us, so 86).
    if (few || at_edge(r, r, rows, c, cols - c - 8, 2)) {
      uint32_t v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = c + e < cols ? s[e] : 0u;
      *reinterpret_cast<uint4*>(dst + r * pitch + c) = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
    } else {
      *reinterpret_cast<uint4*>(dst + r * pitch + c) = load16_any(s, min(8, cols - c), false);
    }
  }
}

// ---- host -----------------------------------------------------------------------------------------------------------------
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

}  // namespace

laq_status product(const Err& e, int dtype, const Operand& a, bool a_mn, const Operand& b, bool b_mn, const Epilogue& ep,
                   uint32_t* status, int starve, bool swappable, bool whole, bool follows, cudaStream_t st) {
  const long long I = a_mn ? a.cols : a.rows, R = a_mn ? a.rows : a.cols, J = b_mn ? b.cols : b.rows;
  const bool out32 = ep.out_f32 != 0, long_sum = !out32 && R > kLongSum;
  const Plan pl = make_plan(I, J, R, a_mn, b_mn, swappable, out32, long_sum, kPlain, whole);
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

namespace {

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

}  // namespace

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

int dz_rows_per(long long M, long long N) {
  // enough blocks for four an SM, no fewer than 32 rows each, and no more than 65535 runs (a grid dimension)
  const long long cols = (N + kDzCols - 1) / kDzCols;
  long long runs = (4 * kSMs + cols - 1) / cols;
  long long per = (M + runs - 1) / runs;
  per = per < 32 ? 32 : per;
  while ((M + per - 1) / per > 65535) per *= 2;
  return (int)per;
}

namespace {

bool sizes_ok(const laq_linear_call* c) {
  const long long most = 0x7fffff00ll;
  return c && c->M >= 0 && c->M <= most && c->N >= 1 && c->N <= most && c->K >= 1 && c->K <= most &&
         (c->dtype == LAQ_BF16 || c->dtype == LAQ_F16);
}

// What the gradient keeps in the workspace: dZ (unless dY itself serves), the column sums' partials, packed operands.
struct BackwardNeeds {
  bool own_dz;
  size_t dz_bytes, part_bytes;
  Operand x, w, dz;
  size_t x_bytes = 0, w_bytes = 0;          // operands that come in 8 bits, in the call's type
  explicit BackwardNeeds(const laq_linear_call* c, const laq_blocks* xq = nullptr, const laq_blocks* wq = nullptr) {
    const Operand dy{c->dy, c->ld_dy, c->M, c->N};
    own_dz = (c->dx || c->dw) && (c->activation != LAQ_ACT_NONE || !dy.mappable_());
    dz_bytes = own_dz ? align256((size_t)c->M * pad8(c->N) * 2) : 0;
    const int per = dz_rows_per(c->M, c->N);
    part_bytes = c->db ? align256((size_t)((c->M + per - 1) / per) * c->N * 4) : 0;
    x = Operand{c->x, c->ld_x, c->M, c->K};
    w = Operand{c->w, c->ld_w, c->N, c->K};
    dz = dy;
    if (xq) x = Operand{nullptr, pad8(c->K), c->M, c->K};
    if (wq) w = Operand{nullptr, pad8(c->K), c->N, c->K};
    if (xq && c->dw) x_bytes = align256((size_t)c->M * pad8(c->K) * 2);
    if (wq && c->dx) w_bytes = align256((size_t)c->N * pad8(c->K) * 2);
  }
  size_t bytes(const laq_linear_call* c) const {
    return dz_bytes + part_bytes + x_bytes + w_bytes + (c->dw ? x.pack_bytes() : 0) + (c->dx ? w.pack_bytes() : 0);
  }
};

laq_status check_call(const Err& e, const laq_linear_call* c, void* ws, size_t ws_bytes, size_t need) {
  if (e.buf && e.len) e.buf[0] = 0;
  if (!c) return fail(e.buf, e.len, LAQ_EINVAL, "null pointer");
  return check_layer(e, c->dtype, c->M, c->N, c->K, c->activation, c->status, c->flags, ws, ws_bytes, need);
}

template <class T>
void list_kernels(const void** list, int& n) {
  const void* all[] = {
      (const void*)linear_gemm_kernel<T, false, false, false, false>, (const void*)linear_gemm_kernel<T, true, false, false, false>,
      (const void*)linear_gemm_kernel<T, false, true, false, false>,  (const void*)linear_gemm_kernel<T, false, false, false, true>,
      (const void*)linear_gemm_kernel<T, true, false, false, true>,   (const void*)linear_gemm_kernel<T, false, true, false, true>,
      (const void*)linear_gemm_kernel<T, false, false, true, false>,  (const void*)linear_gemm_kernel<T, false, true, true, false>,
      (const void*)linear_few_rows_kernel<T, 1, 4>, (const void*)linear_few_rows_kernel<T, 1, 2>, (const void*)linear_few_rows_kernel<T, 2, 4>,
      (const void*)linear_few_rows_kernel<T, 2, 2>, (const void*)linear_few_rows_kernel<T, 3, 2>, (const void*)linear_few_rows_kernel<T, 4, 2>,
      (const void*)linear_dz_kernel<T, false>, (const void*)linear_dz_kernel<T, true>};
  for (const void* k : all) list[n++] = k;
}

}  // namespace

laq_status load_layer_kernels(const Err& e) {
  static Loaded loaded;
  static const void* list[64];
  static const int n = [] {
    int count = 0;
    list_kernels<__nv_bfloat16>(list, count);
    list_kernels<__half>(list, count);
    list_both_kernels(list, count);
    list[count++] = (const void*)linear_db_kernel;
    list[count++] = (const void*)linear_pack_kernel;
    return count;
  }();
  return launched(e.buf, e.len, loaded.once(list, n));
}

laq_status column_sums(const Err& e, const float* part, int runs, int N, float* db, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(((long long)N + 31) / 32));
  cfg.blockDim = dim3(1024);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return launched(e.buf, e.len, cudaLaunchKernelEx(&cfg, linear_db_kernel, part, runs, N, db));
}

laq_status gradient_products(const Err& e, int dtype, const Operand& dz, Operand x, Operand w, const Gradients& to, char*& ws, uint32_t* status,
                             int starve, bool whole, bool follows, cudaStream_t st) {
  const bool together = (whole || (to.dx && to.dw && !to.dw_f32)) && both_pay(dz.rows, dz.cols, x.cols, whole);
  whole = whole && together;
  if (together && to.dx && to.dw) {
    const char* before = ws;
    LAQ_TRY(make_mappable(e, w, ws, st));
    LAQ_TRY(make_mappable(e, x, ws, st));
    return both_products(e, dtype, dz, x, w, to, status, starve, follows || ws != before, st);
  }
  if (to.dx) {
    const char* before = ws;
    LAQ_TRY(make_mappable(e, w, ws, st));
    follows = follows || ws != before;
    Epilogue ep;
    ep.out = to.dx;
    ep.ldo = to.ld_dx;
    LAQ_TRY(product(e, dtype, dz, false, w, true, ep, status, starve, true, whole, follows, st));
    follows = true;
  }
  if (to.dw) {
    const char* before = ws;
    LAQ_TRY(make_mappable(e, x, ws, st));
    follows = follows || ws != before;
    Epilogue ep;
    ep.out = to.dw;
    ep.ldo = to.ld_dw;
    ep.out_f32 = to.dw_f32;
    LAQ_TRY(product(e, dtype, dz, true, x, true, ep, status, starve, false, whole, follows, st));
  }
  return LAQ_OK;
}

laq_status zero_gradients(const Err& e, const Gradients& to, float* db, long long N, long long K, cudaStream_t st) {
  const size_t bytes = to.dw_f32 ? 4 : 2;
  if (to.dw) LAQ_TRY(launched(e.buf, e.len, cudaMemset2DAsync(to.dw, (size_t)to.ld_dw * bytes, 0, (size_t)K * bytes, (size_t)N, st)));
  if (db) LAQ_TRY(launched(e.buf, e.len, cudaMemsetAsync(db, 0, (size_t)N * 4, st)));
  return LAQ_OK;
}

namespace {

// A layer's gradient; operands that come in 8 bits replace the call's own.
laq_status layer_backward(const Err& e, const laq_linear_call* c, const laq_blocks* xq, const laq_blocks* wq, const laq_blocks* zq, void* d_workspace,
                          size_t workspace_bytes, size_t ws_bytes, cudaStream_t st) {
  LAQ_TRY(check_call(e, c, d_workspace, workspace_bytes, ws_bytes));
  if (!c->dx && !c->dw && !c->db) return LAQ_OK;
  const bool act = c->activation != LAQ_ACT_NONE;
  const int dw_bytes = c->dw_dtype == LAQ_F32 ? 4 : 2;
  if (c->dw && c->dw_dtype != c->dtype && c->dw_dtype != LAQ_F32)
    return fail(e.buf, e.len, LAQ_EINVAL, "dw_dtype must be the call's dtype or LAQ_F32");
  if (c->dw && c->dw_dtype == LAQ_F32 && act && c->activation != LAQ_ACT_RELU)
    return fail(e.buf, e.len, LAQ_EINVAL,
                "dw in fp32 needs no activation or ReLU: with the others dZ is rounded to 16 bits before the product");
  Buffers buffers;
  buffers.out("status", c->status, 4, 1, 1, 1);
  if (ws_bytes) buffers.out("the workspace", d_workspace, 1, 1, (long long)ws_bytes, (long long)ws_bytes);
  LAQ_TRY(check_tensor(e, buffers, "dw", kWritten, c->dw, false, c->N, c->ld_dw, c->K, dw_bytes));
  LAQ_TRY(check_tensor(e, buffers, "db", kWritten, c->db, false, 1, c->N, c->N, 4));
  const Gradients to{c->dx, c->ld_dx, c->dw, c->ld_dw, c->dw_dtype == LAQ_F32};
  if (c->M == 0) {               // sums over no rows
    LAQ_TRY(buffers.check(e.buf, e.len));
    return zero_gradients(e, to, c->db, c->N, c->K, st);
  }
  LAQ_TRY(check_tensor(e, buffers, "dy", kRead, c->dy, true, c->M, c->ld_dy, c->N, 2));
  if (act) LAQ_TRY(zq ? check_blocks(e, buffers, "z", "the scales of z", kRead, zq, c->M, c->N)
                      : check_tensor(e, buffers, "z", kRead, c->z, true, c->M, c->ld_z, c->N, 2));
  if (c->dw) LAQ_TRY(xq ? check_blocks(e, buffers, "x", "the scales of x", kRead, xq, c->M, c->K)
                        : check_tensor(e, buffers, "x", kRead, c->x, true, c->M, c->ld_x, c->K, 2));
  if (c->dx) LAQ_TRY(wq ? check_blocks(e, buffers, "w", "the scales of w", kRead, wq, c->N, c->K)
                        : check_tensor(e, buffers, "w", kRead, c->w, true, c->N, c->ld_w, c->K, 2));
  LAQ_TRY(check_tensor(e, buffers, "dx", kWritten, c->dx, false, c->M, c->ld_dx, c->K, 2));
  LAQ_TRY(buffers.check(e.buf, e.len));
  LAQ_TRY(load_layer_kernels(e));
  if (xq || wq || zq) LAQ_TRY(load_block_kernels(e));
  BackwardNeeds need(c, xq, wq);
  char* ws = (char*)d_workspace;
  const bool starve = (c->flags & LAQ_LINEAR_STARVE) != 0;
  bool follows = false;                   // a kernel of this call was the last thing put on the stream
  if (need.own_dz || c->db) {
    void* dz = need.own_dz ? ws : nullptr;
    float* part = c->db ? (float*)(ws + need.dz_bytes) : nullptr;
    ws += need.dz_bytes + need.part_bytes;
    const int per = dz_rows_per(c->M, c->N), runs = (int)((c->M + per - 1) / per), N = (int)c->N;
    const dim3 grid((unsigned)((c->N + kDzCols - 1) / kDzCols), (unsigned)runs);
    const bool coded = act && zq;
    const int vec_ok = mappable(c->dy, c->ld_dy) && (!act || (coded ? Codes(zq).vectors(8) : mappable(c->z, c->ld_z)));
    const auto launch_dz = [&](auto zero) {
      using T = decltype(zero);
      return launch_plain(coded ? linear_dz_kernel<T, true> : linear_dz_kernel<T, false>, grid, kDzThreads, st, (const T*)c->dy, c->ld_dy,
                          (const T*)c->z, c->ld_z, Codes(zq), (T*)dz, pad8(c->N), part, c->M, N, c->activation, per, vec_ok);
    };
    LAQ_TRY(launched(e.buf, e.len, c->dtype == LAQ_BF16 ? launch_dz(__nv_bfloat16()) : launch_dz(__half())));
    follows = true;
    if (c->db) LAQ_TRY(column_sums(e, part, runs, N, c->db, st));
    if (need.own_dz) {
      need.dz.p = dz;
      need.dz.ld = pad8(c->N);
    }
  }
  // operands in 8 bits are restored first
  const auto restored = [&](const laq_blocks* q, Operand& o, size_t bytes) {
    if (!bytes) return LAQ_OK;
    o.p = ws;
    ws += bytes;
    follows = true;
    return unpack_blocks(e, *q, o.rows, o.cols, c->dtype, const_cast<void*>(o.p), o.ld, st);
  };
  LAQ_TRY(restored(wq, need.w, need.w_bytes));
  LAQ_TRY(restored(xq, need.x, need.x_bytes));
  return gradient_products(e, c->dtype, need.dz, need.x, need.w, to, ws, c->status, starve, false, follows, st);
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

extern "C" size_t laq_linear_blocks_workspace_bytes(const laq_linear_call* c, const laq_blocks* x, const laq_blocks* w, int32_t backward) {
  if (!sizes_ok(c)) return 0;
  return backward ? BackwardNeeds(c, x, w).bytes(c) : blocks_forward_bytes(c, x, w);
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
  LAQ_TRY(load_layer_kernels(e));
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
  return product(e, c->dtype, x, false, w, false, ep, c->status, (c->flags & LAQ_LINEAR_STARVE) != 0, true, false, ws != d_workspace,
                 st);
}

extern "C" laq_status laq_linear_backward(const laq_linear_call* c, void* d_workspace, size_t workspace_bytes, void* cuda_stream,
                                          char* errbuf, size_t errbuf_len) {
  const Err e{errbuf, errbuf_len};
  return layer_backward(e, c, nullptr, nullptr, nullptr, d_workspace, workspace_bytes, laq_linear_workspace_bytes(c, 1), (cudaStream_t)cuda_stream);
}

extern "C" laq_status laq_linear_blocks_backward(const laq_linear_call* c, const laq_blocks* x, const laq_blocks* w, const laq_blocks* z,
                                                 void* d_workspace, size_t workspace_bytes, void* cuda_stream, char* errbuf, size_t errbuf_len) {
  const Err e{errbuf, errbuf_len};
  return layer_backward(e, c, x, w, z, d_workspace, workspace_bytes, laq_linear_blocks_workspace_bytes(c, x, w, 1), (cudaStream_t)cuda_stream);
}
