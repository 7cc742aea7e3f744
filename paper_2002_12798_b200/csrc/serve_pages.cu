// Block tables, slot maps and positions of a serving step, built on the GPU from the requests' lengths.
//
// Everything follows from two running sums over the requests (pages needed, tokens wanted).  Every block computes the
// sums for itself, 1024 requests at a time, and then writes the tokens of its own range: one launch, no block waits
// for another, and whole-number sums make the answer independent of timing.  Bound: latency (three dependent loads
// and two block scans: 64 requests 4.5 us) until the tokens are many; then the 12 bytes written per token and their binary
// searches (1024 requests, 102 thousand tokens: 8.1 us, of which 0.3 are bytes).
#include <algorithm>
#include <cstdint>

#include "serve_common.cuh"

using namespace amap_serve;

namespace {

constexpr int kThreads = 256;
constexpr int kPerThread = 4;
constexpr int kChunk = kThreads * kPerThread;   // requests per round of the scan
constexpr int kTokensPerBlock = 1024;

// exclusive sums over the block of two values per thread; totals in *ta, *tb
__device__ __forceinline__ void block_scan(int64_t &a, int64_t &b, int64_t *ta, int64_t *tb, int64_t (*part)[2]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t a0 = a, b0 = b;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t ua = __shfl_up_sync(~0u, a, d), ub = __shfl_up_sync(~0u, b, d);
    if (lane >= d) a += ua, b += ub;
  }
  __syncthreads();  // the previous scan's sums have been read
  if (lane == 31) part[warp][0] = a, part[warp][1] = b;
  __syncthreads();
  int64_t sa = 0, sb = 0, la = 0, lb = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) la += part[w][0], lb += part[w][1];
    sa += part[w][0], sb += part[w][1];
  }
  a += la - a0;
  b += lb - b0;
  *ta = sa;
  *tb = sb;
}

__global__ void __launch_bounds__(kThreads) extend_kernel(const __grid_constant__ amap_pages_extend_args A) {
  __shared__ int64_t part[kThreads / 32][2];
  __shared__ int32_t start[kChunk + 1], old[kChunk], first[kChunk];
  pdl_begin();
  const int64_t room = (int64_t)A.max_pages * A.page_size;
  const int32_t count = min(max(*A.free_count, 0), A.free_capacity);
  const int64_t t0 = (int64_t)blockIdx.x * kTokensPerBlock, t1 = min(t0 + kTokensPerBlock, (int64_t)A.max_tokens);
  int64_t pages_before = 0, tokens_before = 0;  // of all requests that fit their table row
  int64_t granted_before = 0, popped = 0;
  for (int base = 0; base < A.n_requests; base += kChunk) {
    int32_t new_len[kPerThread], len[kPerThread], need[kPerThread];
    bool fits[kPerThread];
    int64_t np = 0, nt = 0;
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
      const int r = base + threadIdx.x * kPerThread + k;
      new_len[k] = r < A.n_requests ? A.new_lens[r] : 0;
      len[k] = r < A.n_requests ? A.seq_lens[r] : 0;
    }
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
      fits[k] = new_len[k] >= 0 && len[k] >= 0 && (int64_t)len[k] + new_len[k] <= room;
      if (!fits[k]) new_len[k] = 0;
      const uint32_t page = A.page_size, has = fits[k] ? ((uint32_t)len[k] + page - 1) / page : 0;
      need[k] = fits[k] ? ((uint32_t)len[k] + new_len[k] + page - 1) / page - has : 0;
      np += need[k];
      nt += new_len[k];
    }
    int64_t p = np, t = nt, all_pages, all_tokens;
    block_scan(p, t, &all_pages, &all_tokens, part);
    p += pages_before;
    t += tokens_before;
    int64_t g = 0, gp = 0;
    int32_t status[kPerThread], page_first[kPerThread];
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
      page_first[k] = (int32_t)min(p, (int64_t)0x7FFFFFFF);  // used only where it is below `count`
      p += need[k];
      t += new_len[k];
      status[k] = !fits[k] ? 1 : need[k] > 0 && p > count ? 2 : new_len[k] > 0 && t > A.max_tokens ? 3 : 0;
      if (status[k] != 0) new_len[k] = 0, need[k] = 0;
      g += new_len[k];
      gp += need[k];
    }
    int64_t at = g, unused = gp, all_granted, all_popped;
    block_scan(at, unused, &all_granted, &all_popped, part);
    at += granted_before;
    const bool mine = base / kChunk % gridDim.x == blockIdx.x;  // this block reports on these requests
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
      const int i = threadIdx.x * kPerThread + k, r = base + i;
      start[i] = (int32_t)at;
      old[i] = len[k];
      first[i] = page_first[k];
      if (mine && r < A.n_requests) {
        A.query_start[r] = (int32_t)at;
        A.seq_lens_out[r] = len[k] + new_len[k];
        A.status[r] = status[k];
      }
      at += new_len[k];
    }
    if (threadIdx.x == kThreads - 1) start[kChunk] = (int32_t)at;
    __syncthreads();
    // tokens of these requests that are in the block's range
    const int64_t lo = max(t0, granted_before), hi = min(t1, granted_before + all_granted);
    for (int64_t i = lo + threadIdx.x; i < hi; i += kThreads) {
      int a = 0, b = kChunk;  // the last request whose start is at or before i: start[a] <= i < start[b]
      while (b - a > 1) {
        const int m = (a + b) >> 1;
        if (start[m] <= i) a = m;
        else b = m;
      }
      const int r = base + a;
      const uint32_t page = A.page_size, pos = (uint32_t)(old[a] + ((int32_t)i - start[a]));
      const int32_t j = (int32_t)(pos / page), off = (int32_t)(pos % page), has = (int32_t)(((uint32_t)old[a] + page - 1) / page);
      int32_t *entry = A.block_table + r * A.table_stride + j;
      int32_t number;
      if (j >= has) {
        number = A.free_pages[count - 1 - (first[a] + j - has)];
        if (off == 0) *entry = number;  // a new page's first token enters it; no token reads it back in this step
      } else {
        number = *entry;
      }
      A.slots[i] = number >= 0 && number < A.n_pages ? number * A.page_size + off : -1;
      A.positions[i] = (int32_t)pos;
      A.requests[i] = r;
    }
    pages_before += all_pages;
    tokens_before += all_tokens;
    granted_before += all_granted;
    popped += all_popped;
    __syncthreads();  // start, old, first are free again
  }
  for (int64_t i = max(t0, granted_before) + threadIdx.x; i < t1; i += kThreads) {
    A.slots[i] = -1;
    A.positions[i] = 0;
    A.requests[i] = -1;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    A.query_start[A.n_requests] = (int32_t)granted_before;
    *A.free_count_out = count - (int32_t)popped;
  }
}

// The pages of finished requests behind one another on the stack, without the holes of their table rows: where a request's
// go is known once the rows before it have been counted.  A cluster counts them all: its warps take neighbouring requests,
// eight rows under way at once, and its blocks tell each other their sums through shared memory.  Where a warp has several
// rows, as many clusters do the same and each copies its part of them: the copies are more instructions than the counting.
// Bound by latency (lengths, rows, the cluster's barrier, rows again) and by what eight multiprocessors count: 4 requests
// 4.5 us, 64 5.6, 1024 of which a third has finished 7.0 (one cluster: 9.5), of which all 8.4, 2000 of which 0.6 10.9.
// (Without holes to look for, lengths alone would say where pages go: 5.6, 5.1, 5.1 and 8.9 for the last four.)
constexpr int kCluster = 8, kMostClusters = 8, kReleaseThreads = 512, kReleaseWarps = kReleaseThreads / 32;
constexpr int kBatch = 8;  // rows whose loads are under way together
constexpr int kAhead = 2;  // fours of a row that a lane asks for together

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int64_t of_rank(const int64_t *mine, uint32_t rank) {
  uint32_t at;
  int64_t v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(mine)), "r"(rank));
  asm volatile("ld.shared::cluster.s64 %0, [%1];" : "=l"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ int64_t warp_sum(int64_t v) {
#pragma unroll
  for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(~0u, v, d);
  return v;
}

__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kReleaseThreads)
    release_kernel(const __grid_constant__ amap_pages_release_args A, const int32_t n_pages) {
  __shared__ int64_t of_warp[kReleaseWarps], sums[2];
  pdl_begin();
  const uint32_t rank = cluster_rank();
  const int cluster = blockIdx.x / kCluster, clusters = gridDim.x / kCluster;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int32_t count = min(max(*A.free_count, 0), A.free_capacity);
  const int64_t room = (int64_t)A.max_pages * A.page_size;
  const bool fours = (reinterpret_cast<uintptr_t>(A.block_table) % 16 | A.table_stride % 4) == 0;
  auto page = [&](int32_t e) { return e >= 0 && e < n_pages; };
  int64_t before = 0;
  int round = 0;
  constexpr int kWarps = kCluster * kReleaseWarps;
  for (int64_t base = 0; base < A.n_requests; base += kWarps * 32, round ^= 1) {
    const int requests = (int)min((int64_t)(kWarps * 32), A.n_requests - base), rows = (requests + kWarps - 1) / kWarps;  // to a warp
    const int first = ((int)rank * kReleaseWarps + warp) * rows, live = max(0, min(rows, requests - first));
    const int64_t r0 = base + first;
    uint32_t entries = 0;  // of the lane's row
    if (lane < live) {
      const int32_t raw = A.seq_lens[r0 + lane];
      const bool done = A.done[r0 + lane] != 0;
      const uint32_t len = (uint32_t)min((int64_t)max(raw, 0), room);
      if (done) entries = (len + (uint32_t)A.page_size - 1) / (uint32_t)A.page_size;
      if (cluster == 0) A.seq_lens_out[r0 + lane] = done ? 0 : raw;
    }
    // four entries of row i from j on; -1 behind its end
    auto four = [&](int i, uint32_t n, uint32_t j, int32_t (&e)[4]) {
      const int32_t *row = A.block_table + (r0 + i) * A.table_stride;
      if (fours && j + 4 <= n) {
        const int4 v = *reinterpret_cast<const int4 *>(row + j);
        e[0] = v.x, e[1] = v.y, e[2] = v.z, e[3] = v.w;
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) e[k] = j + k < n ? row[j + k] : -1;
      }
    };
    int32_t held = 0;  // pages among them
    for (uint32_t todo = __ballot_sync(~0u, entries > 0); todo;) {
      int32_t e[kBatch][kAhead][4];
      int i[kBatch];
      uint32_t n[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        i[b] = todo ? __ffs(todo) - 1 : 0;
        n[b] = __shfl_sync(~0u, entries, i[b]);
        if (!todo) n[b] = 0;
        todo &= todo - 1;
#pragma unroll
        for (int j = 0; j < kAhead; ++j) four(i[b], n[b], 128 * j + 4 * lane, e[b][j]);
      }
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        if (n[b] == 0) break;
        int32_t own = 0;
#pragma unroll
        for (int j = 0; j < kAhead; ++j) own += page(e[b][j][0]) + page(e[b][j][1]) + page(e[b][j][2]) + page(e[b][j][3]);
        for (uint32_t j = 128 * kAhead + 4 * lane; j < n[b]; j += 128) {
          int32_t more[4];
          four(i[b], n[b], j, more);
          own += page(more[0]) + page(more[1]) + page(more[2]) + page(more[3]);
        }
        own = __reduce_add_sync(~0u, own);
        if (lane == i[b]) held = own;
      }
    }
    int64_t upto = held;  // with the warp's rows before
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t v = __shfl_up_sync(~0u, upto, d);
      if (lane >= d) upto += v;
    }
    if (lane == 31) of_warp[warp] = upto;
    __syncthreads();
    const int64_t of_lane = lane < kReleaseWarps ? of_warp[lane] : 0, ahead = warp_sum(lane < warp ? of_lane : 0), all = warp_sum(of_lane);
    if (threadIdx.x == 0) sums[round] = all;
    cluster_sync();  // a round's sums are written again two rounds on, behind the next round's barrier
    const int64_t sum = lane < kCluster ? of_rank(&sums[round], lane) : 0;
    const int64_t start = count + before + ahead + warp_sum(lane < rank ? sum : 0);
    before += warp_sum(sum);
    for (int i = cluster; i < live; i += clusters) {
      const uint32_t n = __shfl_sync(~0u, entries, i);
      if (n == 0) continue;
      int64_t to = start + __shfl_sync(~0u, upto - held, i);
      for (uint32_t j0 = 0; j0 < n; j0 += 128 * kAhead) {
        int32_t e[kAhead][4];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) four(i, n, j0 + 128 * j + 4 * lane, e[j]);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          int64_t place = to;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t pages = __ballot_sync(~0u, page(e[j][k]));
            place += __popc(pages & ((1u << lane) - 1));
            to += __popc(pages);
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (page(e[j][k]) && place < A.free_capacity) A.free_pages[place] = e[j][k];
            place += page(e[j][k]);
          }
        }
      }
    }
  }
  cluster_sync();  // no block ends while another reads its sums
  if (blockIdx.x == 0 && threadIdx.x == 0) *A.free_count_out = (int32_t)min((int64_t)A.free_capacity, count + before);
}

bool apart(const void *a, int64_t an, const void *b, int64_t bn) {
  Span sa, sb;
  sa.hi = an;
  sb.hi = bn;
  return !overlap(a, sa, b, sb);
}

int check_shape(int32_t requests, int32_t max_pages, int32_t page_size, int32_t capacity, int64_t stride) {
  SERVE_REQUIRE(requests >= 1 && max_pages >= 1 && page_size >= 1 && capacity >= 0, AMAP_EINVAL, "requests, table entries and page size are at least 1");
  SERVE_REQUIRE((int64_t)max_pages * page_size <= 0x7FFFFFFF, AMAP_EOVERFLOW, "a table row holds more than 2^31-1 tokens");
  SERVE_REQUIRE(stride >= max_pages, AMAP_EINVAL, "table rows overlap");
  return AMAP_OK;
}

}  // namespace

extern "C" int amap_pages_extend(const amap_pages_extend_args *a, void *cuda_stream) {
  SERVE_REQUIRE(a, AMAP_EINVAL, "null pointer");
  if (const int rc = check_shape(a->n_requests, a->max_pages, a->page_size, a->free_capacity, a->table_stride)) return rc;
  SERVE_REQUIRE(a->n_pages >= 1 && a->max_tokens >= 1, AMAP_EINVAL, "pages and max_tokens are at least 1");
  SERVE_REQUIRE((int64_t)a->n_pages * a->page_size <= 0x7FFFFFFF, AMAP_EOVERFLOW, "more than 2^31-1 slots");
  const void *all[] = {a->new_lens, a->seq_lens, a->block_table, a->free_count, a->query_start, a->slots, a->positions, a->requests,
                       a->seq_lens_out, a->free_count_out, a->status};
  for (const void *p : all) {
    SERVE_REQUIRE(p, AMAP_EINVAL, "null pointer");
    SERVE_REQUIRE(aligned(p, 4), AMAP_EALIGN, "misaligned pointer");
  }
  SERVE_REQUIRE(a->free_pages || a->free_capacity == 0, AMAP_EINVAL, "null pointer");
  SERVE_REQUIRE(aligned(a->free_pages, 4), AMAP_EALIGN, "misaligned pointer");
  const int64_t R = a->n_requests, T = a->max_tokens;
  const struct { const void *p; int64_t n; bool out; } b[] = {
      {a->new_lens, 4 * R, false}, {a->seq_lens, 4 * R, false}, {a->free_pages, 4 * (int64_t)a->free_capacity, false}, {a->free_count, 4, false},
      {a->block_table, 4 * ((R - 1) * a->table_stride + a->max_pages), true}, {a->query_start, 4 * (R + 1), true}, {a->slots, 4 * T, true},
      {a->positions, 4 * T, true}, {a->requests, 4 * T, true}, {a->seq_lens_out, 4 * R, true}, {a->free_count_out, 4, true}, {a->status, 4 * R, true}};
  for (const auto &x : b)
    for (const auto &y : b)
      SERVE_REQUIRE(&x == &y || !x.out || apart(x.p, x.n, y.p, y.n), AMAP_EINVAL, "an output overlaps another buffer");
  const unsigned blocks = (unsigned)((T + kTokensPerBlock - 1) / kTokensPerBlock);
  return launch(extend_kernel, dim3(blocks), kThreads, 0, cuda_stream, *a);
}

extern "C" int amap_pages_release_within(const amap_pages_release_args *a, int32_t n_pages, void *cuda_stream) {
  SERVE_REQUIRE(a, AMAP_EINVAL, "null pointer");
  SERVE_REQUIRE(n_pages >= 1, AMAP_EINVAL, "pages are at least 1");
  if (const int rc = check_shape(a->n_requests, a->max_pages, a->page_size, a->free_capacity, a->table_stride)) return rc;
  const void *all[] = {a->seq_lens, a->block_table, a->free_count, a->seq_lens_out, a->free_count_out};
  SERVE_REQUIRE(a->done, AMAP_EINVAL, "null pointer");
  for (const void *p : all) {
    SERVE_REQUIRE(p, AMAP_EINVAL, "null pointer");
    SERVE_REQUIRE(aligned(p, 4), AMAP_EALIGN, "misaligned pointer");
  }
  SERVE_REQUIRE(a->free_pages || a->free_capacity == 0, AMAP_EINVAL, "null pointer");
  SERVE_REQUIRE(aligned(a->free_pages, 4), AMAP_EALIGN, "misaligned pointer");
  const int64_t R = a->n_requests;
  const struct { const void *p; int64_t n; bool out; } b[] = {
      {a->done, R, false}, {a->seq_lens, 4 * R, false}, {a->block_table, 4 * ((R - 1) * a->table_stride + a->max_pages), false}, {a->free_count, 4, false},
      {a->free_pages, 4 * (int64_t)a->free_capacity, true}, {a->seq_lens_out, 4 * R, true}, {a->free_count_out, 4, true}};
  for (const auto &x : b)
    for (const auto &y : b)
      SERVE_REQUIRE(&x == &y || !x.out || apart(x.p, x.n, y.p, y.n), AMAP_EINVAL, "an output overlaps another buffer");
  // a cluster for each row of a warp
  const int64_t rows = (R + kCluster * kReleaseWarps - 1) / (kCluster * kReleaseWarps);
  const unsigned clusters = (unsigned)std::min<int64_t>(kMostClusters, rows);
  return launch(release_kernel, dim3(clusters * kCluster), kReleaseThreads, 0, cuda_stream, *a, n_pages);
}

extern "C" int amap_pages_release(const amap_pages_release_args *a, void *cuda_stream) { return amap_pages_release_within(a, INT32_MAX, cuda_stream); }
