// What the serving operators (pages, rotary positions, paged cache, decode attention) share: refusals with a reason,
// launches with programmatic stream serialisation, and element types.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <cstdio>

#include "amap_serve.h"

namespace amap_serve {

// the reason of this thread's last refusal (amap_serve_error); a fixed buffer, so that failing cannot itself fail
char *error_text();
constexpr int kErrorText = 256;

inline int refuse(int code, const char *why) {
  snprintf(error_text(), kErrorText, "%s", why);
  return code;
}
inline int accept() {
  error_text()[0] = 0;
  return AMAP_OK;
}

#define SERVE_REQUIRE(cond, code, why) \
  do {                                 \
    if (!(cond)) return refuse(code, why); \
  } while (0)

// multiprocessors of the current device
int device_sms();

// cluster: blocks of a cluster, 1 for none
template <typename... P, typename... A>
int launch_clusters(void (*kernel)(P...), dim3 grid, int cluster, int threads, size_t smem, void *stream, const A &...args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
  if (e != cudaSuccess) {
    cudaGetLastError();  // a refused launch leaves no error behind for the caller's next CUDA call
    return refuse(AMAP_ECUDA, cudaGetErrorString(e));
  }
  return accept();
}
template <typename... P, typename... A>
int launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, void *stream, const A &...args) {
  return launch_clusters(kernel, grid, 1, threads, smem, stream, args...);
}

// EVERY thread of every kernel calls both, in this order, before it touches a buffer: a block that returned without
// waiting could let its grid finish before the grid ahead of it has, and the grid behind it start too early.
__device__ __forceinline__ void pdl_begin() {
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

// ---- elements ----
template <int DT> struct Elem;
template <> struct Elem<AMAP_BF16> {
  using T = __nv_bfloat16;
  static __device__ __forceinline__ float to(T v) { return __bfloat162float(v); }
  static __device__ __forceinline__ T from(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Elem<AMAP_FP16> {
  using T = __half;
  static __device__ __forceinline__ float to(T v) { return __half2float(v); }
  static __device__ __forceinline__ T from(float v) { return __float2half_rn(v); }
};
template <> struct Elem<AMAP_FP32> {
  using T = float;
  static __device__ __forceinline__ float to(T v) { return v; }
  static __device__ __forceinline__ T from(float v) { return v; }
};
__device__ __forceinline__ uint8_t to_e4m3(float v) { return (uint8_t)__nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3); }

template <int BYTES> struct Raw;
template <> struct Raw<1> { using T = uint8_t; };
template <> struct Raw<2> { using T = uint16_t; };
template <> struct Raw<4> { using T = uint32_t; };
template <> struct Raw<8> { using T = uint2; };
template <> struct Raw<16> { using T = uint4; };

inline int dtype_bytes(int dt) { return dt == AMAP_FP32 ? 4 : dt == AMAP_E4M3 ? 1 : (dt == AMAP_BF16 || dt == AMAP_FP16) ? 2 : 0; }
inline bool aligned(const void *p, int64_t bytes) { return (reinterpret_cast<uintptr_t>(p) % (uint64_t)bytes) == 0; }

// [lo, hi) of the bytes that a strided tensor spans, relative to its pointer (strides may be negative or zero)
struct Span {
  int64_t lo = 0, hi = 0;
  void add(int64_t extent, int64_t stride, int64_t es) {
    const int64_t d = (extent - 1) * stride * es;
    if (d < 0) lo += d;
    else hi += d;
  }
};
inline bool overlap(const void *a, const Span &sa, const void *b, const Span &sb) {
  const int64_t pa = (int64_t)reinterpret_cast<uintptr_t>(a), pb = (int64_t)reinterpret_cast<uintptr_t>(b);
  return pa + sa.lo < pb + sb.hi && pb + sb.lo < pa + sa.hi;
}

// checks of a cache's description that every operator on it makes; AMAP_OK, or the refusal
int check_cache(const amap_cache &c);

}  // namespace amap_serve
