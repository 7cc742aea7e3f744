// Attention of one new token per request over a paged cache.
#include <algorithm>
#include <cmath>

#include "serve_common.cuh"

using namespace amap_serve;

namespace {

constexpr int kThreads = 128;

__device__ __forceinline__ float to_float(const char *p, int64_t at, int dtype) {
  if (dtype == AMAP_BF16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(p)[at]);
  if (dtype == AMAP_FP16) return __half2float(reinterpret_cast<const __half *>(p)[at]);
  return __half2float(__half(__nv_cvt_fp8_to_halfraw(reinterpret_cast<const uint8_t *>(p)[at], __NV_E4M3)));
}

// One block per request and q head; 128 tokens a round: a thread scores one token, then owns columns of the output.
__global__ void __launch_bounds__(kThreads) attend_kernel(const __grid_constant__ amap_attend_args A) {
  __shared__ float q[256], score[kThreads], part[kThreads / 32];
  __shared__ int64_t where[kThreads];
  pdl_begin();
  const int r = blockIdx.y, h = blockIdx.x, tid = threadIdx.x;
  const amap_cache &C = A.cache;
  const int group = A.q_heads / C.heads, kvh = h / group, D = C.head_dim;
  for (int d = tid; d < D; d += kThreads) q[d] = to_float(static_cast<const char *>(A.q), r * A.q_row + h * A.q_head + d, A.dtype);
  const int n = (int)min((int64_t)max(A.seq_lens[r], 0), (int64_t)A.max_pages * C.page_size);
  const int low = A.window > 0 ? max(0, n - A.window) : 0;
  float top = -INFINITY, sum = 0.0f, o[2] = {0.0f, 0.0f};
  __syncthreads();
  for (int base = low; base < n; base += kThreads) {
    const int t = base + tid;
    float s = -INFINITY;
    int64_t v_at = -1;
    if (t < n) {
      const int page = A.block_table[r * A.table_stride + t / C.page_size], off = t % C.page_size;
      if (page >= 0 && page < C.n_pages) {
        const int64_t k_at = page * C.k_page + off * C.k_token + kvh * C.k_head;
        v_at = page * C.v_page + off * C.v_token + kvh * C.v_head;
        s = 0.0f;
        for (int d = 0; d < D; ++d) s += q[d] * to_float(static_cast<const char *>(C.k), k_at + d, C.dtype);
        s *= A.scale * C.k_scale;
        if (A.softcap > 0) s = A.softcap * tanhf(s / A.softcap);
      }
    }
    where[tid] = v_at;
    float m = s;
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
    if ((tid & 31) == 0) part[tid >> 5] = m;
    __syncthreads();
    m = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
    const float now = fmaxf(top, m);
    const float keep = now == -INFINITY ? 1.0f : expf(top - now);
    score[tid] = v_at < 0 ? 0.0f : expf(s - now);
    top = now;
    __syncthreads();
    sum *= keep;
    o[0] *= keep;
    o[1] *= keep;
    for (int i = 0; i < kThreads; ++i) {
      if (where[i] < 0) continue;
      sum += score[i];
      for (int k = 0; k < 2; ++k) {
        const int d = tid + k * kThreads;
        if (d < D) o[k] += score[i] * to_float(static_cast<const char *>(C.v), where[i] + d, C.dtype);
      }
    }
    __syncthreads();
  }
  for (int k = 0; k < 2; ++k) {
    const int d = tid + k * kThreads;
    if (d >= D) break;
    const float y = sum > 0 ? o[k] / sum * C.v_scale : sum == 0 ? 0.0f : sum;
    const int64_t at = r * A.out_row + h * A.out_head + d;
    if (A.dtype == AMAP_BF16) static_cast<__nv_bfloat16 *>(A.out)[at] = __float2bfloat16_rn(y);
    else static_cast<__half *>(A.out)[at] = __float2half_rn(y);
  }
  if (A.lse && tid == 0) A.lse[r * A.lse_row + h] = sum == 0 ? -INFINITY : top + logf(sum);
}

}  // namespace

extern "C" int amap_attend_workspace(int32_t n_requests, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int64_t *bytes) {
  SERVE_REQUIRE(bytes, AMAP_EINVAL, "null pointer");
  SERVE_REQUIRE(n_requests >= 1 && q_heads >= 1 && kv_heads >= 1 && q_heads % kv_heads == 0, AMAP_EINVAL, "q heads: a multiple of the cache's heads");
  SERVE_REQUIRE(head_dim >= 8 && head_dim <= 256 && head_dim % 8 == 0, AMAP_EUNSUPPORTED, "head size: a multiple of 8, up to 256");
  *bytes = 256;
  return accept();
}

extern "C" int amap_attend(const amap_attend_args *a, void *cuda_stream) {
  SERVE_REQUIRE(a, AMAP_EINVAL, "null pointer");
  if (const int rc = check_cache(a->cache)) return rc;
  const amap_cache &c = a->cache;
  int64_t need = 0;
  if (const int rc = amap_attend_workspace(a->n_requests, a->q_heads, c.heads, c.head_dim, &need)) return rc;
  SERVE_REQUIRE(a->n_requests <= 0xFFFF, AMAP_EINVAL, "at most 65535 requests");
  SERVE_REQUIRE(a->dtype == AMAP_BF16 || a->dtype == AMAP_FP16, AMAP_EINVAL, "type: bf16 or fp16");
  SERVE_REQUIRE(c.dtype == AMAP_E4M3 || c.dtype == a->dtype, AMAP_EINVAL, "a 16-bit cache has the type of q");
  SERVE_REQUIRE(a->q && a->out && a->block_table && a->seq_lens && a->workspace, AMAP_EINVAL, "null pointer");
  SERVE_REQUIRE(a->max_pages >= 1 && a->table_stride >= a->max_pages, AMAP_EINVAL, "table rows overlap");
  SERVE_REQUIRE((int64_t)a->max_pages * c.page_size <= 0x7FFFFFFF, AMAP_EOVERFLOW, "a table row holds more than 2^31-1 tokens");
  SERVE_REQUIRE(std::isfinite(a->scale) && std::isfinite(a->softcap) && a->softcap >= 0 && a->window >= 0 && a->reserved == 0, AMAP_EINVAL,
                "scale is finite, softcap and window are not negative");
  SERVE_REQUIRE(a->workspace_bytes >= need, AMAP_EINVAL, "workspace too small");
  const int es = dtype_bytes(c.dtype), per16 = 16 / es;
  SERVE_REQUIRE(c.head_dim % per16 == 0, AMAP_EUNSUPPORTED, "head size: whole 16-byte chunks");
  for (const int64_t s : {c.k_page, c.k_token, c.k_head, c.v_page, c.v_token, c.v_head})
    SERVE_REQUIRE(s % per16 == 0, AMAP_EALIGN, "cache strides: whole 16-byte chunks");
  SERVE_REQUIRE(aligned(c.k, 16) && aligned(c.v, 16), AMAP_EALIGN, "cache: aligned to 16 bytes");
  SERVE_REQUIRE(aligned(a->q, 2) && aligned(a->out, 2) && aligned(a->lse, 4) && aligned(a->block_table, 4) && aligned(a->seq_lens, 4) &&
                    aligned(a->workspace, 256), AMAP_EALIGN, "misaligned pointer");
  Span qs, os;
  qs.hi = os.hi = (int64_t)c.head_dim * 2;
  qs.add(a->n_requests, a->q_row, 2);
  qs.add(a->q_heads, a->q_head, 2);
  os.add(a->n_requests, a->out_row, 2);
  os.add(a->q_heads, a->out_head, 2);
  SERVE_REQUIRE(!overlap(a->q, qs, a->out, os), AMAP_EINVAL, "q and out overlap");
  return launch(attend_kernel, dim3(a->q_heads, a->n_requests), kThreads, 0, cuda_stream, *a);
}
