// The cache of 4 bits: its description, and reading tokens back in 16 or 32 bits.
//
// Reading.  A thread has eight elements of K and the same eight of V of a token, of two heads: a word and two 16-bit halves of codes,
// the two words of numbers, and two stores of 16 bytes each.  A block has 16 tokens of these heads, so that where they are a cell's (the tokens
// of a prompt) the halves of V, which lie apart, are served by the cell's lines in the first-level cache.
// Bound: memory, of which three quarters are the stores: 65537 tokens of 8 heads of 128 fp16 elements in groups of 32 (353 MB) 62 us
// = 5.6 TB/s (one head a thread, 64-bit index arithmetic: 85); 700 tokens 5.2 us, latency.
#include <algorithm>

#include "serve_alias.hpp"
#include "serve_common.cuh"
#include "serve_packed.cuh"

using namespace amap_serve;

namespace {

constexpr int kThreads = 256;

struct ReadParams {
  const char *data;
  int64_t page, head;
  char *k, *v;
  int64_t k_row, k_head, v_row, v_head;  // elements
  const int32_t *slots;
  int64_t rows;
  int32_t heads, page_size, n_slots, group_shift, head_blocks;
  uint32_t div_mul, div_shift;  // slot / page_size (0 mul: a power of two)
};

__device__ __forceinline__ float low_of(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ float step_of(uint32_t w) { return __uint_as_float(w << 16); }

// the i-th four bits of the lower half of a word as it lies in a cell, which with the half's bytes exchanged is `other`: masked out
// where they are, beside 2^23, which goes together with the scale
__device__ __forceinline__ float code_of(uint32_t w, uint32_t other, int i) {
  const int at = kTurn + 4 * (i & 1);
  return fmaf(__uint_as_float(((i < 2 ? w : other) & (15u << at)) | 0x4B000000u), 1.0f / (1 << at), -0x1p23f / (1 << at));
}
__device__ __forceinline__ uint32_t bytes_exchanged(uint32_t w) { return __byte_perm(w, 0, 0x2301); }

template <int DT>
__device__ __forceinline__ void put(char *p, int64_t at, const float (&x)[8], bool wide) {
  using T = typename Elem<DT>::T;
  T *to = reinterpret_cast<T *>(p) + at;
  union {
    T e[8];
    uint4 four[sizeof(T) / 2];
  } u;
#pragma unroll
  for (int i = 0; i < 8; ++i) u.e[i] = Elem<DT>::from(x[i]);
  if (wide) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4 *>(to)[i] = u.four[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) to[i] = u.e[i];
  }
}

// A block: 256 / chunks rows (16 at least or all that fit) of kHeads heads, their loads under way together.
constexpr int kHeads = 2;
template <int NS> constexpr int kRows = kThreads / (4 * NS) >= 16 ? kThreads / (4 * NS) / 16 * 16 : kThreads / (4 * NS);

template <int DT, int NS, bool WIDE>
__global__ void __launch_bounds__(kThreads) read_kernel(const __grid_constant__ ReadParams P) {
  constexpr int CHUNKS = 4 * NS;
  const int c = threadIdx.x % CHUNKS, in_block = threadIdx.x / CHUNKS;
  const uint32_t block = blockIdx.x / P.head_blocks;
  const int head0 = (blockIdx.x - block * P.head_blocks) * kHeads;
  const int64_t row = (int64_t)block * kRows<NS> + in_block;
  pdl_begin();
  if (in_block >= kRows<NS> || row >= P.rows) return;
  const int32_t slot = P.slots[row];
  const bool there = slot >= 0 && slot < P.n_slots;
  uint32_t kw[kHeads] = {}, v0[kHeads] = {}, v1[kHeads] = {};
  uint2 numbers[kHeads] = {};
  if (there) {
    const uint32_t page = P.div_mul ? __umulhi((uint32_t)slot, P.div_mul) >> P.div_shift : (uint32_t)slot >> P.div_shift;
    const int in = slot - (int)page * P.page_size, token = in % kCell, groups = CHUNKS * 8 >> P.group_shift;
    const char *const cell = P.data + (int64_t)page * P.page + (int64_t)(in / kCell) * cell_bytes(NS, groups);
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
      if (head0 + h >= P.heads) break;
      const char *const own = cell + (int64_t)(head0 + h) * P.head;
      kw[h] = *reinterpret_cast<const uint32_t *>(own + k_word_at(NS, token, c));
      v0[h] = *reinterpret_cast<const uint16_t *>(own + v_half_at(NS, token, 2 * c));
      v1[h] = *reinterpret_cast<const uint16_t *>(own + v_half_at(NS, token, 2 * c + 1));
      numbers[h] = *reinterpret_cast<const uint2 *>(own + numbers_at(NS, token, c * 8 >> P.group_shift));
    }
  }
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    if (head0 + h >= P.heads) break;
    float k[8], v[8];
    const uint32_t kx = bytes_exchanged(kw[h]), x0 = bytes_exchanged(v0[h]), x1 = bytes_exchanged(v1[h]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      k[i] = fmaf(step_of(numbers[h].x), i & 1 ? code_of(kw[h] >> 16, kx >> 16, i >> 1) : code_of(kw[h], kx, i >> 1), low_of(numbers[h].x));
      v[i] = fmaf(step_of(numbers[h].y), i < 4 ? code_of(v0[h], x0, i) : code_of(v1[h], x1, i - 4), low_of(numbers[h].y));
    }
    put<DT>(P.k, row * P.k_row + (head0 + h) * P.k_head + c * 8, k, WIDE);
    put<DT>(P.v, row * P.v_row + (head0 + h) * P.v_head + c * 8, v, WIDE);
  }
}

template <int DT, int NS>
int run(ReadParams &P, bool wide, void *stream) {
  P.head_blocks = (P.heads + kHeads - 1) / kHeads;
  const int64_t blocks = (P.rows + kRows<NS> - 1) / kRows<NS> * P.head_blocks;
  SERVE_REQUIRE(blocks <= 0x7FFFFFFF, AMAP_EOVERFLOW, "too many rows");
  const dim3 grid((unsigned)blocks);
  return wide ? launch(read_kernel<DT, NS, true>, grid, kThreads, 0, stream, P) : launch(read_kernel<DT, NS, false>, grid, kThreads, 0, stream, P);
}

template <int DT>
int run_dim(ReadParams &P, int head_dim, bool wide, void *stream) {
  switch (head_dim) {
    case 64: return run<DT, 2>(P, wide, stream);
    case 96: return run<DT, 3>(P, wide, stream);
    case 128: return run<DT, 4>(P, wide, stream);
    default: return run<DT, 8>(P, wide, stream);
  }
}

}  // namespace

int amap_serve::check_packed(const amap_packed &c) {
  SERVE_REQUIRE(c.data, AMAP_EINVAL, "cache: null pointer");
  SERVE_REQUIRE(c.n_pages >= 1 && c.heads >= 1 && c.heads <= 0xFFFF && c.reserved == 0, AMAP_EINVAL, "cache: pages and heads are at least 1, heads 65535 at most");
  const int64_t bytes = amap_packed_bytes(c.page_size, c.head_dim, c.group);
  if (bytes == 0) return AMAP_EUNSUPPORTED;  // its reason stands
  SERVE_REQUIRE((int64_t)c.n_pages * c.page_size <= 0x7FFFFFFF, AMAP_EOVERFLOW, "cache: more than 2^31-1 slots");
  SERVE_REQUIRE(aligned(c.data, 16) && c.page % 16 == 0 && c.head % 16 == 0, AMAP_EALIGN, "cache: data and strides in whole 16 bytes");
  // pages of heads lie apart: one stride steps over all that the other reaches
  const __int128 page = c.page < 0 ? -(__int128)c.page : c.page, head = c.head < 0 ? -(__int128)c.head : c.head;
  const bool pages = c.n_pages > 1, heads = c.heads > 1;
  SERVE_REQUIRE(page * c.n_pages + head * c.heads < ((__int128)1 << 60), AMAP_EOVERFLOW, "cache: strides beyond any memory");
  SERVE_REQUIRE((!pages || page >= bytes) && (!heads || head >= bytes) &&
                    (!pages || !heads || page >= (c.heads - 1) * head + bytes || head >= (c.n_pages - 1) * page + bytes),
                AMAP_EINVAL, "cache: pages overlap");
  return AMAP_OK;
}

extern "C" int64_t amap_packed_bytes(int32_t page_size, int32_t head_dim, int32_t group) {
  const char *why = nullptr;
  if (page_size < kCell || page_size % kCell) why = "cache: page_size is a multiple of 16";
  else if (head_dim != 64 && head_dim != 96 && head_dim != 128 && head_dim != 256) why = "cache: heads of 64, 96, 128 or 256 elements";
  else if ((group != 32 && group != 64) || head_dim % group) why = "cache: groups of 32 elements, or of 64 where they divide a head";
  if (why) {
    refuse(AMAP_EUNSUPPORTED, why);
    return 0;
  }
  accept();
  return (int64_t)(page_size / kCell) * cell_bytes(head_dim / kSlab, head_dim / group);
}

extern "C" int amap_packed_read(const amap_packed_read_args *a, void *cuda_stream) {
  SERVE_REQUIRE(a, AMAP_EINVAL, "null pointer");
  SERVE_REQUIRE(a->dtype == AMAP_BF16 || a->dtype == AMAP_FP16 || a->dtype == AMAP_FP32, AMAP_EINVAL, "type: bf16, fp16 or fp32");
  SERVE_REQUIRE(a->rows >= 0 && a->rows <= 0x7FFFFFFF && a->reserved == 0, AMAP_EINVAL, "rows: 0 .. 2^31-1");
  const amap_packed &c = a->cache;
  if (const int rc = check_packed(c)) return rc;
  if (a->rows == 0) return accept();
  SERVE_REQUIRE(a->k && a->v && a->slots, AMAP_EINVAL, "null pointer");
  const int es = dtype_bytes(a->dtype);
  SERVE_REQUIRE(aligned(a->k, es) && aligned(a->v, es) && aligned(a->slots, 4), AMAP_EALIGN, "misaligned pointer");
  SERVE_REQUIRE((a->rows == 1 || (a->k_row && a->v_row)) && (c.heads == 1 || (a->k_head && a->v_head)), AMAP_EINVAL, "rows of k or v lie on one another");
  const int64_t width = (int64_t)c.head_dim * es;
  const Runs k = {(int64_t) reinterpret_cast<uintptr_t>(a->k), a->rows, a->k_row * es, c.heads, a->k_head * es};
  const Runs v = {(int64_t) reinterpret_cast<uintptr_t>(a->v), a->rows, a->v_row * es, c.heads, a->v_head * es};
  SERVE_REQUIRE(!share(k, v, width), AMAP_EINVAL, "k and v share elements");
  Span held, ks, vs;
  held.hi = amap_packed_bytes(c.page_size, c.head_dim, c.group);
  held.add(c.n_pages, c.page, 1);
  held.add(c.heads, c.head, 1);
  ks.hi = vs.hi = width;
  ks.add(a->rows, a->k_row, es), ks.add(c.heads, a->k_head, es);
  vs.add(a->rows, a->v_row, es), vs.add(c.heads, a->v_head, es);
  SERVE_REQUIRE(!overlap(a->k, ks, c.data, held) && !overlap(a->v, vs, c.data, held), AMAP_EINVAL, "k or v overlaps the cache");
  ReadParams P = {};
  P.data = static_cast<const char *>(c.data), P.page = c.page, P.head = c.head;
  P.k = static_cast<char *>(a->k), P.v = static_cast<char *>(a->v);
  P.k_row = a->k_row, P.k_head = a->k_head, P.v_row = a->v_row, P.v_head = a->v_head;
  P.slots = a->slots;
  P.rows = a->rows;
  P.heads = c.heads, P.page_size = c.page_size, P.n_slots = c.n_pages * c.page_size, P.group_shift = c.group == 64 ? 6 : 5;
  // the high word of a product with ceil(2^(32+s) / page_size), s = floor(log2 page_size): exact for slots below 2^31
  int s = 0;
  while ((2u << s) <= (uint32_t)c.page_size) ++s;
  P.div_shift = s;
  if (c.page_size != 1 << s) P.div_mul = (uint32_t)((((uint64_t)1 << (32 + s)) + c.page_size - 1) / c.page_size);
  const int per16 = 16 / es;
  const bool wide = aligned(a->k, 16) && aligned(a->v, 16) && a->k_row % per16 == 0 && a->k_head % per16 == 0 && a->v_row % per16 == 0 && a->v_head % per16 == 0;
  switch (a->dtype) {
    case AMAP_BF16: return run_dim<AMAP_BF16>(P, c.head_dim, wide, cuda_stream);
    case AMAP_FP16: return run_dim<AMAP_FP16>(P, c.head_dim, wide, cuda_stream);
    default: return run_dim<AMAP_FP32>(P, c.head_dim, wide, cuda_stream);
  }
}
