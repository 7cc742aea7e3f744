// Host state and checks shared by the serving operators.
#include <cmath>
#include <cuda_runtime_api.h>

#include <atomic>

#include "serve_common.cuh"

namespace amap_serve {

char *error_text() {
  static thread_local char text[kErrorText] = "";
  return text;
}

int device_sms() {
  static std::atomic<int> known[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
  int sms = known[dev].load(std::memory_order_relaxed);
  if (sms == 0) {
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1) {
      cudaGetLastError();
      return 148;
    }
    known[dev].store(sms, std::memory_order_relaxed);
  }
  return sms;
}

int check_cache(const amap_cache &c) {
  SERVE_REQUIRE(c.k && c.v, AMAP_EINVAL, "cache: null pointer");
  SERVE_REQUIRE(c.dtype == AMAP_BF16 || c.dtype == AMAP_FP16 || c.dtype == AMAP_E4M3, AMAP_EINVAL, "cache: type is bf16, fp16 or e4m3");
  SERVE_REQUIRE(c.n_pages >= 1 && c.page_size >= 1 && c.heads >= 1 && c.head_dim >= 1, AMAP_EINVAL, "cache: pages, page size, heads and head size are at least 1");
  SERVE_REQUIRE((int64_t)c.n_pages * c.page_size <= 0x7FFFFFFF, AMAP_EOVERFLOW, "cache: more than 2^31-1 slots");
  SERVE_REQUIRE(std::isfinite(c.k_scale) && std::isfinite(c.v_scale) && c.k_scale > 0 && c.v_scale > 0, AMAP_EINVAL, "cache: scales are positive and finite");
  SERVE_REQUIRE(c.dtype == AMAP_E4M3 || (c.k_scale == 1.0f && c.v_scale == 1.0f), AMAP_EINVAL, "cache: a 16-bit cache has scales of 1");
  return AMAP_OK;
}

}  // namespace amap_serve

extern "C" const char *amap_serve_error(void) { return amap_serve::error_text(); }
