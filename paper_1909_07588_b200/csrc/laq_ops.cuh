// What the context-free operators (laq_ops_rows.cu, laq_ops_linear.cu) share: element types, argument checks that end
// in a status and a text, and the checks of a call's buffers.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <float.h>
#include <stdint.h>

#include <atomic>
#include <cstdarg>
#include <cstdio>
#include <cstring>

#include "laq.h"

namespace laq {
namespace ops {

inline laq_status fail(char* errbuf, size_t errlen, laq_status st, const char* fmt, ...) {
  if (errbuf && errlen) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(errbuf, errlen, fmt, ap);
    va_end(ap);
  }
  return st;
}

inline int dtype_bytes(int dtype) { return dtype == LAQ_F32 ? 4 : (dtype == LAQ_BF16 || dtype == LAQ_F16) ? 2 : 0; }

// The status of a launch by its own return value: an error that an earlier call of this thread has left behind is neither taken for
// this one's nor cleared.
inline laq_status launched(char* errbuf, size_t errlen, cudaError_t rc) {
  if (rc == cudaSuccess) return LAQ_OK;
  cudaGetLastError();
  return fail(errbuf, errlen, LAQ_ECUDA, "kernel launch failed: %s", cudaGetErrorString(rc));
}
template <class... Params, class... Args>
cudaError_t launch_plain(void (*kernel)(Params...), dim3 grid, unsigned threads, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.stream = st;
  return cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
}

// The runtime loads a kernel's code on its first use, which may take device memory for it.  The first call on a device has all
// of a file's kernels loaded (some 0.05 ms each), so that no later call takes any, whichever forms it needs.
class Loaded {
 public:
  cudaError_t once(const void* const* kernels, int n) {
    int dev = 0;
    cudaError_t rc = cudaGetDevice(&dev);
    if (rc != cudaSuccess) return rc;
    const uint64_t bit = 1ull << (dev & 63);
    if (dev < 64 && (devices_.load(std::memory_order_acquire) & bit)) return cudaSuccess;
    for (int i = 0; i < n; ++i) {
      cudaFuncAttributes fa;
      rc = cudaFuncGetAttributes(&fa, kernels[i]);
      if (rc != cudaSuccess) return rc;
    }
    devices_.fetch_or(bit, std::memory_order_release);
    return cudaSuccess;
  }

 private:
  std::atomic<uint64_t> devices_{0};
};

// The driver's query of several properties of a pointer in one call (0.03 us; a call asks for up to 14 pointers), and that of
// the calling thread's context.
struct Driver {
  CUresult (*pointer_attributes)(unsigned int, CUpointer_attribute*, void**, CUdeviceptr) = nullptr;
  CUresult (*current_context)(CUcontext*) = nullptr;
  Driver() {
    find("cuPointerGetAttributes", (void**)&pointer_attributes);
    find("cuCtxGetCurrent", (void**)&current_context);
  }
  static void find(const char* name, void** fn) {
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint(name, fn, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      *fn = nullptr;
    }
  }
};
inline const Driver& driver() {
  static const Driver d;
  return d;
}

// Bytes in rows: [p + i pitch, p + i pitch + width) for i < rows.
struct Extent {
  uintptr_t p;
  unsigned long long rows, pitch, width;
  uintptr_t end() const { return p + (rows - 1) * pitch + width; }
  bool meets(uintptr_t a, uintptr_t b) const {      // a row of it and [a, b)
    if (b <= p || end() <= a) return false;
    const unsigned long long i = a < p + width ? 0 : (a - p - width) / pitch + 1;      // the first row that ends behind a
    return i < rows && p + i * pitch < b;
  }
  // Rows of two matrices may lie between each other (halves of the columns of one, every other row): exact.
  bool meets(const Extent& o) const {
    if (!rows || !o.rows || !width || !o.width || o.end() <= p || end() <= o.p) return false;
    if (pitch == o.pitch && rows > 1 && o.rows > 1) {      // all rows lie alike: o's row 0 is q rows and r bytes into this one
      const bool behind = o.p >= p;
      const unsigned long long d = behind ? o.p - p : p - o.p, q = d / pitch, r = d % pitch;
      const Extent &a = behind ? *this : o, &b = behind ? o : *this;
      // b's row i meets a's row q + i (r < a.width) or q + i + 1 (r + b.width > pitch)
      return (r < a.width && q < a.rows) || (r + b.width > pitch && q + 1 < a.rows);
    }
    const Extent &few = rows <= o.rows ? *this : o, &many = rows <= o.rows ? o : *this;
    for (unsigned long long i = 0; i < few.rows; ++i)
      if (many.meets(few.p + i * few.pitch, few.p + i * few.pitch + few.width)) return true;
    return false;
  }
};

// The buffers of a call, all of which are looked at before its first kernel runs: each must be aligned to its elements and lie
// in the memory of the current device, where the kernels run, and one that is written may share no byte with any other.  A
// null pointer (an optional buffer) is left out.
class Buffers {
 public:
  // rows x cols elements of `bytes` bytes, rows ld elements apart.  in_place: the name of the one buffer that an output may be
  void in(const char* name, const void* p, int bytes, long long rows, long long cols, long long ld) { add(name, p, bytes, rows, cols, ld, false, ""); }
  void out(const char* name, const void* p, int bytes, long long rows, long long cols, long long ld, const char* in_place = "") {
    add(name, p, bytes, rows, cols, ld, true, in_place);
  }
  laq_status check(char* errbuf, size_t errlen) const {
    for (int i = 0; i < count_; ++i) {
      const Buffer& b = list_[i];
      if (b.p % (uintptr_t)b.bytes) return fail(errbuf, errlen, LAQ_EINVAL, "%s is not aligned to its element size", b.name);
      if ((double)b.x.rows * (double)b.x.pitch > kAddressable) return fail(errbuf, errlen, LAQ_EINVAL, "the rows of %s reach beyond any memory", b.name);
    }
    for (int i = 0; i < count_; ++i)
      for (int j = 0; j < count_; ++j) {
        const Buffer &a = list_[i], &b = list_[j];
        if (!a.written || i == j || (b.written && j < i)) continue;
        const bool itself = a.p == b.p && a.x.pitch == b.x.pitch && !strcmp(a.in_place, b.name);
        if (!itself && a.x.meets(b.x)) return fail(errbuf, errlen, LAQ_EINVAL, "%s and %s overlap", a.name, b.name);
      }
    int dev = -1;
    const Driver& drv = driver();
    if (cudaGetDevice(&dev) != cudaSuccess || !drv.pointer_attributes || !drv.current_context) {
      cudaGetLastError();
      return fail(errbuf, errlen, LAQ_EINVAL, "no current CUDA device");
    }
    // A thread that has made no call yet has no context, and without one the driver answers no question and encodes no tensor map.
    CUcontext context = nullptr;
    if (drv.current_context(&context) != CUDA_SUCCESS || !context) {
      const cudaError_t rc = cudaSetDevice(dev);
      if (rc != cudaSuccess) {
        cudaGetLastError();
        return fail(errbuf, errlen, LAQ_ECUDA, "the device cannot be used: %s", cudaGetErrorString(rc));
      }
    }
    for (int i = 0; i < count_; ++i) {
      CUmemorytype type = (CUmemorytype)0;
      int on = -1;
      CUpointer_attribute what[2] = {CU_POINTER_ATTRIBUTE_MEMORY_TYPE, CU_POINTER_ATTRIBUTE_DEVICE_ORDINAL};
      void* out[2] = {&type, &on};
      const bool known = drv.pointer_attributes(2, what, out, (CUdeviceptr)list_[i].p) == CUDA_SUCCESS;
      if (known && type == CU_MEMORYTYPE_DEVICE && on == dev) continue;
      unsigned managed = 0;                  // managed memory serves wherever it lies
      what[0] = CU_POINTER_ATTRIBUTE_IS_MANAGED;
      out[0] = &managed;
      if (known && drv.pointer_attributes(1, what, out, (CUdeviceptr)list_[i].p) == CUDA_SUCCESS && managed) continue;
      if (!known || type != CU_MEMORYTYPE_DEVICE)
        return fail(errbuf, errlen, LAQ_EINVAL, "%s is not device memory", list_[i].name);
      return fail(errbuf, errlen, LAQ_EINVAL, "%s lives on another GPU than the current device: make its device current for the call", list_[i].name);
    }
    return LAQ_OK;
  }

 private:
  struct Buffer {
    const char* name;
    uintptr_t p;
    int bytes;
    bool written;
    const char* in_place;
    Extent x;
  };
  void add(const char* name, const void* p, int bytes, long long rows, long long cols, long long ld, bool written, const char* in_place) {
    if (!p || count_ == kMost) return;
    const long long pitch = rows <= 1 ? cols : ld < kAddressable ? ld : (long long)kAddressable;
    list_[count_++] = Buffer{name, (uintptr_t)p, bytes, written, in_place,
                             Extent{(uintptr_t)p, (unsigned long long)rows, (unsigned long long)pitch * bytes, (unsigned long long)cols * bytes}};
  }
  static constexpr int kMost = 16;       // more than any call has
  static constexpr double kAddressable = 1.4e17;      // 2^57 bytes
  Buffer list_[kMost];
  int count_ = 0;
};

// One element type each: conversion, 16-byte vectors of EV elements, the largest of a vector (a NaN wins).
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// Two fp32 numbers in a register pair: one instruction for both.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair_of(float a, float b) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void split(f32x2 p, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.ftz.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 ex2x2(f32x2 p) {
  float a, b;
  split(p, a, b);
  return pair_of(ex2(a), ex2(b));
}

template <class T>
struct Elem;

template <>
struct Elem<float> {
  static constexpr int EV = 4;
  static constexpr uint32_t kNegInf = 0xff800000u;     // 32 bits of -inf elements
  static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[4]) {
    x[0] = __uint_as_float(v.x);
    x[1] = __uint_as_float(v.y);
    x[2] = __uint_as_float(v.z);
    x[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
  static __device__ __forceinline__ void pairs(const uint4& v, f32x2 (&p)[2]) {
    p[0] = pair_of(__uint_as_float(v.x), __uint_as_float(v.y));
    p[1] = pair_of(__uint_as_float(v.z), __uint_as_float(v.w));
  }
  static __device__ __forceinline__ uint4 pack_pairs(const f32x2 (&p)[2]) {
    float a, b, d, e;
    split(p[0], a, b);
    split(p[1], d, e);
    return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(d), __float_as_uint(e));
  }
  // a bound no larger than `lo`, as a word of elements; 0 if the type has no finite one
  static __device__ __forceinline__ uint32_t bound(float lo) { return fabsf(lo) < FLT_MAX ? __float_as_uint(lo) : 0u; }
  static __device__ __forceinline__ uint32_t at_least1(uint32_t w, uint32_t lo) {
    return __float_as_uint(max_nan(__uint_as_float(w), __uint_as_float(lo)));
  }
  static __device__ __forceinline__ float to_float(float v) { return v; }
  static __device__ __forceinline__ float from_float(float v) { return v; }
  template <int N>
  static __device__ __forceinline__ float largest(const uint4 (&v)[N]) {
    float m = __uint_as_float(v[0].x);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      m = max_nan(max_nan(m, __uint_as_float(v[i].x)), __uint_as_float(v[i].y));
      m = max_nan(max_nan(m, __uint_as_float(v[i].z)), __uint_as_float(v[i].w));
    }
    return m;
  }
};

template <>
struct Elem<__nv_bfloat16> {
  static constexpr int EV = 8;
  static constexpr uint32_t kNegInf = 0xff80ff80u;
  static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ void pairs(const uint4& v, f32x2 (&p)[4]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = pair_of(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  }
  static __device__ __forceinline__ uint4 pack_pairs(const f32x2 (&p)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a, b;
      split(p[i], a, b);
      const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ uint32_t bound(float lo) {
    const __nv_bfloat16 h = __float2bfloat16_rd(lo);
    const uint32_t b = *reinterpret_cast<const uint16_t*>(&h);
    return fabsf(__bfloat162float(h)) < INFINITY ? b | (b << 16) : 0u;
  }
  static __device__ __forceinline__ uint32_t at_least1(uint32_t w, uint32_t lo) {
    const __nv_bfloat162 r = __hmax2_nan(pair(w), pair(lo));
    return *reinterpret_cast<const uint32_t*>(&r);
  }
  static __device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
  static __device__ __forceinline__ __nv_bfloat16 from_float(float v) { return __float2bfloat16_rn(v); }
  static __device__ __forceinline__ __nv_bfloat162 pair(uint32_t w) { return *reinterpret_cast<__nv_bfloat162*>(&w); }
  template <int N>
  static __device__ __forceinline__ float largest(const uint4 (&v)[N]) {
    __nv_bfloat162 m = pair(v[0].x);
#pragma unroll
    for (int i = 0; i < N; ++i)
      m = __hmax2_nan(__hmax2_nan(m, __hmax2_nan(pair(v[i].x), pair(v[i].y))), __hmax2_nan(pair(v[i].z), pair(v[i].w)));
    return max_nan(__low2float(m), __high2float(m));
  }
};

template <>
struct Elem<__half> {
  static constexpr int EV = 8;
  static constexpr uint32_t kNegInf = 0xfc00fc00u;
  static __device__ __forceinline__ __half2 pair(uint32_t w) { return *reinterpret_cast<__half2*>(&w); }
  static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(pair(w[i]));
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2 h = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ void pairs(const uint4& v, f32x2 (&p)[4]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(pair(w[i]));
      p[i] = pair_of(f.x, f.y);
    }
  }
  static __device__ __forceinline__ uint4 pack_pairs(const f32x2 (&p)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a, b;
      split(p[i], a, b);
      const __half2 h = __floats2half2_rn(a, b);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ uint32_t bound(float lo) {
    const __half h = __float2half_rd(lo);
    const uint32_t b = *reinterpret_cast<const uint16_t*>(&h);
    return fabsf(__half2float(h)) < INFINITY ? b | (b << 16) : 0u;
  }
  static __device__ __forceinline__ uint32_t at_least1(uint32_t w, uint32_t lo) {
    const __half2 r = __hmax2_nan(pair(w), pair(lo));
    return *reinterpret_cast<const uint32_t*>(&r);
  }
  static __device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
  static __device__ __forceinline__ __half from_float(float v) { return __float2half_rn(v); }
  template <int N>
  static __device__ __forceinline__ float largest(const uint4 (&v)[N]) {
    __half2 m = pair(v[0].x);
#pragma unroll
    for (int i = 0; i < N; ++i)
      m = __hmax2_nan(__hmax2_nan(m, __hmax2_nan(pair(v[i].x), pair(v[i].y))), __hmax2_nan(pair(v[i].z), pair(v[i].w)));
    return max_nan(__low2float(m), __high2float(m));
  }
};

// Every element of a vector raised to at least the bound of Elem<T>::bound (a NaN stays).
template <class T>
__device__ __forceinline__ uint4 at_least(const uint4& v, uint32_t lo) {
  return make_uint4(Elem<T>::at_least1(v.x, lo), Elem<T>::at_least1(v.y, lo), Elem<T>::at_least1(v.z, lo), Elem<T>::at_least1(v.w, lo));
}

// Plain (coherent) 16-byte load and store: a gradient may be written over the tensor that it is computed from.
__device__ __forceinline__ uint4 load16(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}

// 16 bytes from global to shared memory in the background; a thread waits for its own copies and reads only those, so no
// barrier is involved.  Commits group the copies; wait<N> returns when all but the last N groups have landed.
__device__ __forceinline__ void copy16(void* smem, const void* p) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(p) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

}  // namespace ops
}  // namespace laq
