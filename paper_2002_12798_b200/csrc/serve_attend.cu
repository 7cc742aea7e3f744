// Attention of one new token per request over a paged cache, split over the cache's length and joined in one launch.
//
// Mathematics.  For a cache head and the (up to 8 NT) q heads that share it, with S^T = K Q^T (tokens x heads) and the
// running maximum m, sum l and O^T = V^T P^T (head elements x heads) of a softmax in base 2:
//   m' = max(m, max S),  P = 2^(S - m'),  l' = l 2^(m-m') + sum P,  O' = O 2^(m-m') + P V;  parts with their own
//   (m, l, O) join the same way, and out = O / l, lse = (m + log2 l) ln 2.
//
// Bound: HBM.  Every K and V element of a live token is read once and meets 2 x group multiply-adds; the tokens take the
// M side of the matrix instructions (K as it lies, V through transposing loads), so that 8 q heads fill the N side
// whatever the group size and the tensor pipe stays a small part of the time.  The matrix instructions are warp-wide
// mma.sync: a product of 16 tokens by 8 heads is far below the 128 rows a tcgen05 tile wants, and at 2 x 8 multiply-adds
// per element the legacy rate is several times what HBM can feed.
//
// Split.  The tiles (64 or 128 tokens) of all requests form one line, cut into equal pieces: balanced to a tile whatever the
// lengths are, and computed by every block for itself from seq_lens (no plan, no host).  A piece belongs to a team of
// blocks, one per cache head (or a divisor of their number, where more teams then fill the device better): what they
// read lies side by side in caches ordered by token, and they read it at about the same time.
// An item is a request's tiles of one head.  A block that has a part of an item writes it to the workspace; the last to
// arrive joins the parts in the order of the tokens (very many of them in groups first), so the result does not depend
// on who that is.  The part a block begins with is, where it has few others, joined by the producer warp meanwhile.
//
// Pipeline.  A producer warp looks up pages, one tile ahead, and fills a ring of tiles; four warps take a quarter of each
// tile.  Pages of 8 n tokens arrive by tensor copies (TMA) of whole 8 to 64 token boxes, others row by row with 16-byte
// asynchronous copies; both lay 128-byte rows out with the same swizzle, chunk ^ (row mod 8), so that the matrix loads
// meet every bank once.  Only the end of an item synchronises the four warps.
//
// Measured: one request of 131009 tokens over 8 heads of 128 fp16 elements (537 MB) 89.6 us = 6.0 TB/s; 32 requests of up
// to 16384 tokens in bf16 6.5 TB/s; 128 of up to 4096 over an e4m3 cache, 8 q heads to each, 5.2; 33 tokens 5.5 us.
#include <cuda.h>

#include <algorithm>
#include <atomic>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <type_traits>

#include "serve_common.cuh"

using namespace amap_serve;

namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps, kBlock = kThreads + 32;  // the last warp is the producer
// tokens per warp and step, in sixteens: two where a token's row is 128 bytes, so that a step moves 32 KB either way and two
// independent products hide each other's latency (128 e4m3 requests: 103 us with one, 100 with two)
template <int ROW_BYTES> constexpr int kSixteens = ROW_BYTES == 128 ? 2 : 1;
constexpr int kMostBlocksPerSm = 2;
constexpr int kGroup = 8;               // teams whose parts are joined first, where an item has more than kDirect of them
constexpr int kDirect = 12;
constexpr int kAside = 4;               // parts that the producer warp joins
template <int DP> constexpr int kJoined = 2 * (DP + 4);  // parts, or groups of them, that the four warps have room to join
static_assert(kDirect <= kJoined<64>, "parts joined without groups");
constexpr int kMostMembers = 32;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Params {
  alignas(64) CUtensorMap k_map, v_map;  // [page][head][token][element], boxes of 128 bytes x 2^box_shift tokens
  amap_attend_args a;
  int32_t group, blocks_per_head, items_per_request;  // q heads per cache head; blocks of 8 NT of them; cache heads x blocks
  int32_t members, rounds;                            // blocks of a team; items_per_request / members
  uint32_t div_mul, div_shift;                        // token / page_size (0 mul: a power of two)
  int32_t tensor_copies, box_shift;
  int32_t q_pairs, out_pairs;                         // two elements at a time are aligned
  float *part_o, *part_ml;
  int32_t *failed, *grouped, *arrived;
};

// Blocks resident per multiprocessor: two where their registers allow (O and q of 8 heads of up to 128 elements); with 16
// heads held to half the registers, what spills costs more than the second block brings (32 requests of 8k tokens, 16 q
// heads per cache head, P in two terms: 131 us against 117; in three 129 with one block).
template <int DP, int NT> constexpr int kResident = DP == 256 || NT >= 2 ? 1 : 2;
// Stages of the ring: 192 KB a multiprocessor, of which about two thirds are in flight (latency times bandwidth is 50).
template <int ROW_BYTES, int RESIDENT> constexpr int kStages = 192 * 1024 / RESIDENT / (2 * 16 * kSixteens<ROW_BYTES> * kWarps * ROW_BYTES);

__device__ __forceinline__ uint32_t smem_at(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool live) {
  const int n = live ? 16 : 0;  // nothing is read where the row is not live: the 16 bytes become zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void copies_arrive(uint32_t bar) {  // when this thread's copies so far have landed
  asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tensor_copy(uint32_t dst, const CUtensorMap *map, int x, int token, int head, int page, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
               "l"(map), "r"(x), "r"(token), "r"(head), "r"(page), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void bar_init(uint32_t bar, int n) { asm volatile("mbarrier.init.shared.b64 [%0], %1;" ::"r"(bar), "r"(n) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void bar_arrive_bytes(uint32_t bar, int n) {
  asm volatile("mbarrier.arrive.expect_tx.shared.b64 _, [%0], %1;" ::"r"(bar), "r"(n) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// Every wait ends: after two seconds it gives up, marks the workspace, and later waits of the warp return at once, so that
// the block still walks through its steps and barriers (on what lies in shared memory) and ends.
__device__ __noinline__ bool bar_wait_slow(uint32_t bar, uint32_t parity, int32_t *failed) {
  uint64_t begin, now;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(begin));
  do {
    if (bar_try(bar, parity)) return true;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(now));
  } while (now - begin < 2000000000ull);
  *failed = 1;
  return false;
}
__device__ __forceinline__ void bar_wait(uint32_t bar, uint32_t parity, int32_t *failed, bool &alive) {
  if (!bar_try(bar, parity) && alive) alive = bar_wait_slow(bar, parity, failed);
}
// What a warp that has given up does before it ends: it waits, as long again for each stage, for the last copies into the
// ring, which a block must not leave behind it.  Stages before `stage` were filled last in the lap whose phase has `parity`,
// the others in the lap before (there is none before the first, and then this wait is over at once).
__device__ __noinline__ void settle(uint32_t full, int stages, int stage, uint32_t parity, int32_t *failed) {
  for (int s = 0; s < stages; ++s) bar_wait_slow(full + 8 * s, s < stage ? parity : parity ^ 1, failed);
}
__device__ __forceinline__ void sync_consumers() { asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory"); }

__device__ __forceinline__ void load4(uint32_t at, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void load4_transposed(uint32_t at, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t transposed(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
template <int CT>
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (CT == AMAP_BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_of(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// tanh: 1 - 2 / (e^2x + 1), whose error is some 2^-23 however small x is; below 0.3 therefore its series, to x^9 (what is
// left out is less than 2^-24 of it).  Within 2^-20 of itself.
__device__ __forceinline__ float tanh_of(float x) {
  const float y = x * x;
  const float series = x + x * y * (-1.0f / 3 + y * (2.0f / 15 + y * (-17.0f / 315 + y * (62.0f / 2835))));
  const float closed = 1.0f - __fdividef(2.0f, exp2_of(x * (2.0f * kLog2e)) + 1.0f);
  return fabsf(x) < 0.3f ? series : closed;
}
// four e4m3 as four fp16: exact
__device__ __forceinline__ void halves_of(uint32_t four, uint32_t *low, uint32_t *high) {
  asm("{ .reg .b16 l, h; mov.b32 {l, h}, %2; cvt.rn.f16x2.e4m3x2 %0, l; cvt.rn.f16x2.e4m3x2 %1, h; }" : "=r"(*low), "=r"(*high) : "r"(four));
}

// P in 16-bit terms, each what the ones before it leave over, so that P V has the precision of 32-bit P: three terms of
// bf16's 8 bits, or two of fp16's 11.  A remainder is no less than `least`, nor (BANDED) is the first term: above zero where
// V can hold an infinity, so that it meets no zero that P has not got.
// P is taken relative to a maximum that is renewed only when a score passes it by more than kSlack (in powers of 2): the
// true one moves in most of the early steps, and O would be rescaled each time.  fp16 terms carry P times 2^kLift, out of
// the way of fp16's smallest numbers; 2^(kLift + kSlack) is below its largest.  A step with a score further than kDeep
// below the maximum (beside a token that has nearly all the weight, every one) would still come too near them: such a
// step goes by bands of kBand powers of 2 from its own highest score down, each lifted to 2^(kLift + kSlack) and scaled
// back in 32 bits.  In all others P is 2^(kLift - kDeep) at least, 2^12 of fp16's smallest steps.  The three numbers share
// fp16's 40 powers of 2 out so that bands are rare: with scores of 2.9 (standard deviation, powers of 2) 16 q heads per
// cache head take 80 us for 32 requests up to 8192 tokens, with 8 + 7, 17 in place of 6 + 9, 21 94 us, without bands 78.  With
// scores of 11.6 nearly every step goes by bands: 128 e4m3 requests 119 -> 182 us, 32 of fp16 195 -> 276.
constexpr float kSlack = 6.0f, kDeep = 21.0f, kBand = 24.0f;
template <int CT> constexpr float kLift = CT == AMAP_FP16 ? 9.0f : 0.0f;
template <int CT> constexpr int kTerms = CT == AMAP_BF16 ? 3 : 2;
template <int CT, bool BANDED>
__device__ __forceinline__ void split(float p0, float p1, float least, uint32_t (&term)[kTerms<CT>]) {
  if constexpr (CT == AMAP_BF16) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint32_t u0 = __float_as_uint(p0), u1 = __float_as_uint(p1);
      term[k] = __byte_perm(u0, u1, 0x7632);
      p0 = fmaxf(p0 - __uint_as_float(u0 & 0xFFFF0000u), least);
      p1 = fmaxf(p1 - __uint_as_float(u1 & 0xFFFF0000u), least);
    }
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(term[2]) : "f"(p1), "f"(p0));
  } else {
    asm("cvt.rz.f16x2.f32 %0, %1, %2;" : "=r"(term[0]) : "f"(p1), "f"(p0));
    __half2 h = *reinterpret_cast<const __half2 *>(&term[0]);
    if constexpr (BANDED) {
      h = __hmax2_nan(h, __float2half2_rn(least));
      term[0] = *reinterpret_cast<const uint32_t *>(&h);
    }
    const float r0 = fmaxf(p0 - __low2float(h), least), r1 = fmaxf(p1 - __high2float(h), least);
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(term[1]) : "f"(r1), "f"(r0));
  }
}

// The line of tiles of TILE tokens: request by request, its heads round by round (a round is a team's), a round's tiles in
// order.  A request without tokens counts one tile, so that somebody writes its zeros.  Every item (a round of a request)
// is longer by kEntry places, for what it costs to put the item before it away and to take it up; its tiles are the
// places behind those.
constexpr int kEntry = 2;

template <int TILE>
struct Cursor {
  int r, h, n, low, t, left, n_next;  // h: the round
  int rest;                           // places from the tile at hand to the end of the piece

  static __device__ __forceinline__ int clamped(const Params &P, int len) {
    return (int)min((int64_t)max(len, 0), (int64_t)P.a.max_pages * P.a.cache.page_size);
  }
  static __device__ __forceinline__ int lowest(const Params &P, int n) { return P.a.window > 0 ? max(0, n - P.a.window) : 0; }
  static __device__ __forceinline__ int tiles(const Params &P, int n) {
    return max(1, n / TILE + (n % TILE != 0) - lowest(P, n) / TILE);  // n may be 2^31 - 1
  }
  __device__ __forceinline__ void enter(const Params &P) {
    low = lowest(P, n);
    t = low & ~(TILE - 1);
    left = tiles(P, n);
  }
  __device__ __forceinline__ void start(const Params &P, int r0, int h0, int tile, int64_t first_place, int64_t end) {
    r = r0;
    h = h0;
    n = clamped(P, P.a.seq_lens[r]);
    n_next = P.a.seq_lens[min(r + 1, P.a.n_requests - 1)];
    enter(P);
    t += tile * TILE;
    left -= tile;
    rest = (int)(end - first_place) - tile;
  }
  __device__ __forceinline__ int stride() const { return left > 1 ? 1 : 1 + kEntry; }
  __device__ __forceinline__ bool more() const { return rest > stride(); }
  __device__ __forceinline__ void advance(const Params &P) {
    rest -= stride();
    if (--left > 0) {
      t += TILE;
      return;
    }
    if (++h == P.rounds) {
      h = 0;
      ++r;
      n = clamped(P, n_next);
      n_next = P.a.seq_lens[min(r + 1, P.a.n_requests - 1)];  // read an item ahead of its use
    }
    enter(P);
  }
};

__device__ __forceinline__ void write_pair(const Params &P, int64_t at, float x, float y) {
  if (P.a.dtype == AMAP_BF16) {
    __nv_bfloat16 *out = static_cast<__nv_bfloat16 *>(P.a.out) + at;
    const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
    if (P.out_pairs) *reinterpret_cast<__nv_bfloat162 *>(out) = v;
    else out[0] = v.x, out[1] = v.y;
  } else {
    __half *out = static_cast<__half *>(P.a.out) + at;
    const __half2 v = __floats2half2_rn(x, y);
    if (P.out_pairs) *reinterpret_cast<__half2 *>(out) = v;
    else out[0] = v.x, out[1] = v.y;
  }
}

// Threads that work together: the four warps, or the producer's.
struct Consumers {
  static constexpr int kCount = kThreads;
  static __device__ __forceinline__ int index() { return threadIdx.x; }
  static __device__ __forceinline__ void sync() { sync_consumers(); }
};
struct Producer {
  static constexpr int kCount = 32;
  static __device__ __forceinline__ int index() { return threadIdx.x & 31; }
  static __device__ __forceinline__ void sync() { __syncwarp(); }
};

// Joins n parts of an item, the i-th in slot slot_of(i), in this order: into the output, or (final: false) into slot
// slot_of(0), which nobody else reads before this block has arrived for it.  ml: room for n x 8, free again on return:
// the four warps' lies in `joint`, where the next item's (m, l) go without a barrier ahead of them (with heads of 64
// elements, those of warp 0's second head over part 8's of the third, which warp 1 reads).
template <typename T, int CT, int DP, int HB, typename F>
__device__ void join(const Params &P, float2 (*ml)[8], int n, F slot_of, int heads, bool final, int r, int first_head) {
  const int tid = T::index(), D = P.a.cache.head_dim;
  for (int h0 = 0; h0 < heads; h0 += 8) {
    const int items = min(8, heads - h0) * (DP / 4);
    float4 v[8];
    auto ask = [&](int item, int i0) {
      const float4 *part = reinterpret_cast<const float4 *>(P.part_o + (int64_t)(h0 + item / (DP / 4)) * DP) + item % (DP / 4);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        v[j] = item < items && i0 + j < n ? __ldcg(part + (int64_t)slot_of(i0 + j) * (HB * DP / 4)) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    };
    ask(tid, 0);  // under way while the parts' (m, l) are shared out
    T::sync();
    for (int i = tid >> 3; i < n; i += T::kCount / 8) ml[i][tid & 7] = __ldcg(reinterpret_cast<const float2 *>(P.part_ml) + (int64_t)slot_of(i) * HB + h0 + (tid & 7));
    T::sync();
    for (int item = tid; item < items; item += T::kCount) {
      const int in = item / (DP / 4), d = item % (DP / 4) * 4;
      float top = -INFINITY;
      for (int i = 0; i < n; ++i) top = fmaxf(top, ml[i][in].x);
      float sum = 0.0f;
      float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      for (int i0 = 0; i0 < n; i0 += 8) {
        if (item != tid || i0) ask(item, i0);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (i0 + j >= n) break;
          const float2 own = ml[i0 + j][in];
          const float f = top == -INFINITY ? 1.0f : exp2_of(own.x - top);
          sum += own.y * f;
          y.x += v[j].x * f;
          y.y += v[j].y * f;
          y.z += v[j].z * f;
          y.w += v[j].w * f;
        }
      }
      if (d >= D) continue;
      if (final) {
        const float f = sum == 0.0f ? 0.0f : P.a.cache.v_scale / sum;
        const int64_t to = (int64_t)r * P.a.out_row + (int64_t)(first_head + h0 + in) * P.a.out_head + d;
        write_pair(P, to, y.x * f, y.y * f);
        write_pair(P, to + 2, y.z * f, y.w * f);
        if (d == 0 && P.a.lse) P.a.lse[(int64_t)r * P.a.lse_row + first_head + h0 + in] = sum == 0.0f ? -INFINITY : (top - kLift<CT> + log2f(sum)) * kLn2;
      } else {
        const int64_t to = (int64_t)slot_of(0) * HB + h0 + in;
        *reinterpret_cast<float4 *>(P.part_o + to * DP + d) = y;
        if (d == 0) reinterpret_cast<float2 *>(P.part_ml)[to] = make_float2(top, sum);
      }
    }
  }
  T::sync();
}

// Whether this block is the last of n to arrive at the counter, which then is ready for the next call.  What the threads
// have written before is seen by whoever arrives later: the barrier orders it before thread 0's arrival, which releases
// it and acquires what the others have released.
template <typename T>
__device__ __forceinline__ bool last_of(int32_t *counter, int n, int *told) {
  T::sync();
  if (T::index() == 0) {
    int before;
    asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(counter) : "memory");
    if (before == n - 1) *counter = 0;
    *told = before == n - 1;
  }
  T::sync();
  return *told != 0;
}

template <int S, int TILE> struct Small {
  uint64_t full[S], empty[S];
  int64_t sums[kWarps], first_place;
  uint32_t rows_there[S][TILE / 32];  // rows of a stage whose page is there
  int begin[3], told, told_aside;
  float2 aside[kAside][8];
};

template <int CT, bool FP8, int DP, int NT>
__global__ void __launch_bounds__(kBlock, (kResident<DP, NT>)) attend_kernel(const __grid_constant__ Params P) {
  constexpr int ES = FP8 ? 1 : 2, RB = DP * ES, NB = RB / 128, S = kStages<RB, kResident<DP, NT>>;
  constexpr int U = kSixteens<RB>, ROWS = 16 * U, TILE = ROWS * kWarps;  // tokens per warp and step, and per tile
  constexpr int MT = DP / 16;                  // 16-element steps of a head
  constexpr int HB = 8 * NT;                   // q heads of a block
  constexpr int kBox = TILE * 128;             // bytes of a tile's rows of 128
  constexpr int kStage = 2 * NB * kBox;        // K then V
  constexpr int kPitch = DP + 4;               // floats between heads in `joint`: the writes of a warp meet all banks once,
                                               // and a warp's (m, l) of a head has room behind its O
  extern __shared__ __align__(1024) char smem[];
  float *joint = reinterpret_cast<float *>(smem + S * kStage);  // [warps][8][kPitch]
  // all in one piece: static shared memory ahead of it would cost its 1024-byte alignment, and with it the second block
  using Line = Cursor<TILE>;
  Small<S, TILE> &small = *reinterpret_cast<Small<S, TILE> *>(joint + kWarps * 8 * kPitch);
  float2(*const joined)[8] = reinterpret_cast<float2(*)[8]>(joint);  // [kJoined<DP>][8], while `joint` is idle
  static_assert(sizeof(float2) * 8 * kJoined<DP> <= sizeof(float) * kWarps * 8 * kPitch, "room for the parts of an item");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
  const amap_cache &C = P.a.cache;
  const int D = C.head_dim;
  if (tid == 0) {
    for (int i = 0; i < S; ++i) {
      bar_init(smem_at(&small.full[i]), P.tensor_copies ? 1 : 33);
      bar_init(smem_at(&small.empty[i]), kWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (!P.tensor_copies && D < DP) {  // what lies behind a head's end is never copied over: zeros (tensor copies bring their own)
    for (int i = tid; i < S * kStage / 16; i += kBlock) reinterpret_cast<uint4 *>(smem)[i] = make_uint4(0, 0, 0, 0);
  }
  pdl_begin();

  // ---- where this block's piece of the line begins ----
  const int R = P.a.n_requests, per = (R + kThreads - 1) / kThreads, r_first = warp < kWarps ? min(R, tid * per) : R, r_last = min(R, r_first + per);
  int64_t mine = 0;
  for (int r = r_first; r < r_last; ++r) mine += kEntry + Line::tiles(P, Line::clamped(P, P.a.seq_lens[r]));
  mine *= P.rounds;
  int64_t upto = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t v = __shfl_up_sync(~0u, upto, d);
    if (lane >= d) upto += v;
  }
  if (lane == 31 && warp < kWarps) small.sums[warp] = upto;
  __syncthreads();
  int64_t total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) upto += small.sums[w];
    total += small.sums[w];
  }
  const int team = blockIdx.x / P.members, member = blockIdx.x - team * P.members;
  const int64_t pieces = min((int64_t)(gridDim.x / P.members), total);  // none of them empty
  if (team >= pieces) return;
  const int64_t u0 = total * team / pieces, u1 = total * (team + 1) / pieces;
  if (warp < kWarps && upto > u0 && upto - mine <= u0) {
    int64_t u = upto - mine;
    for (int r = r_first; r < r_last; ++r) {
      const int tiles = Line::tiles(P, Line::clamped(P, P.a.seq_lens[r]));
      const int64_t places = (int64_t)(kEntry + tiles) * P.rounds;
      if (u + places > u0) {
        const int64_t in = u0 - u;
        const int round = in <= 0x7FFFFFFF ? (int)in / (kEntry + tiles) : (int)(in / (kEntry + tiles));
        const int tile = max(0, (int)(in - (int64_t)round * (kEntry + tiles)) - kEntry);
        small.begin[0] = r;
        small.begin[1] = round;
        small.begin[2] = tile;
        small.first_place = u + (int64_t)round * (kEntry + tiles) + kEntry;  // of the item that u0 is in
        break;
      }
      u += places;
    }
  }
  __syncthreads();
  Line at;
  at.start(P, small.begin[0], small.begin[1], small.begin[2], small.first_place, u1);
  if (at.rest <= 0) return;  // a piece between two items
  bool alive = true;
  // the parts of the item that the piece begins in: those of the teams `from` to `to`, of which the first began it in its
  // second slot, the others go on with it in their first
  const int64_t first_place = small.first_place, first_last = first_place + Line::tiles(P, at.n) - 1;
  auto team_of = [&](int64_t place) { return (int)(((place + 1) * pieces - 1) / total); };
  const int first_from = team_of(first_place), first_to = team_of(first_last);
  const bool aside = first_place < u0 && first_last + 1 + kEntry < u1 && first_to - first_from < kAside;

  if (warp == kWarps) {
    // ---- the producer ----
    const int boxes = TILE >> P.box_shift;
    int entry = -1, offset = 0, there = 0;
    auto look = [&](int row) {  // the page of a row of the tile at `at`, if any of the row's box takes part
      const int token = at.t + row;
      there = token < at.n && token > at.low - (P.tensor_copies ? 1 << P.box_shift : 1);
      if (there) {
        const uint32_t page = P.div_mul ? __umulhi((uint32_t)token, P.div_mul) >> P.div_shift : (uint32_t)token >> P.div_shift;
        offset = token - (int)page * C.page_size;
        entry = P.a.block_table[(int64_t)at.r * P.a.table_stride + page];
      }
    };
    int stage = 0;
    uint32_t parity = 1;  // the first round of waits finds every stage empty
    if (P.tensor_copies) {
      const int row = lane << P.box_shift;
      if (lane < boxes) look(row);
      for (bool more = true; more;) {
        const int head = (at.h * P.members + member) / P.blocks_per_head;
        const bool live = lane < boxes && there && (uint32_t)entry < (uint32_t)C.n_pages;
        const int page = live ? entry : C.n_pages;  // a page beyond the last: zeros, and nothing is read
        const int token = live ? offset : 0;
        uint32_t rows[TILE / 32];
#pragma unroll
        for (int k = 0; k < TILE / 32; ++k) rows[k] = __ballot_sync(~0u, __shfl_sync(~0u, live, (lane + 32 * k) >> P.box_shift));
        more = at.more();
        if (more) {
          at.advance(P);
          there = 0;
          if (lane < boxes) look(row);
        }
        bar_wait(smem_at(&small.empty[stage]), parity, P.failed, alive);
        if (!__all_sync(~0u, alive)) break;
        const uint32_t bar = smem_at(&small.full[stage]), to = smem_at(smem + stage * kStage) + row * 128;
        if (lane == 0) {
#pragma unroll
          for (int k = 0; k < TILE / 32; ++k) small.rows_there[stage][k] = rows[k];
          bar_arrive_bytes(bar, kStage);
        }
        __syncwarp();
        if (lane < boxes) {
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            tensor_copy(to + b * kBox, &P.k_map, b * (128 / ES), token, head, page, bar);
            tensor_copy(to + (NB + b) * kBox, &P.v_map, b * (128 / ES), token, head, page, bar);
          }
        }
        if (++stage == S) stage = 0, parity ^= 1;
      }
    } else {
      // a lane looks up every 32nd row; the copies of a row are 8 lanes' 16 bytes of its 128
      int entries[TILE / 32], offsets[TILE / 32];
      bool theres[TILE / 32];
      auto look_all = [&]() {
#pragma unroll
        for (int k = 0; k < TILE / 32; ++k) {
          look(lane + 32 * k);
          entries[k] = entry, offsets[k] = offset, theres[k] = there;
        }
      };
      look_all();
      for (bool more = true; more;) {
        const int head = (at.h * P.members + member) / P.blocks_per_head;
        int64_t k_at[TILE / 32], v_at[TILE / 32];
        uint32_t mask[TILE / 32];
#pragma unroll
        for (int k = 0; k < TILE / 32; ++k) {
          const bool live = theres[k] && (uint32_t)entries[k] < (uint32_t)C.n_pages;
          mask[k] = __ballot_sync(~0u, live);
          k_at[k] = live ? (int64_t)entries[k] * C.k_page + (int64_t)offsets[k] * C.k_token + (int64_t)head * C.k_head : 0;
          v_at[k] = live ? (int64_t)entries[k] * C.v_page + (int64_t)offsets[k] * C.v_token + (int64_t)head * C.v_head : 0;
        }
        more = at.more();
        if (more) {
          at.advance(P);
          look_all();
        }
        bar_wait(smem_at(&small.empty[stage]), parity, P.failed, alive);
        if (!__all_sync(~0u, alive)) break;
        const uint32_t bar = smem_at(&small.full[stage]), to = smem_at(smem + stage * kStage);
#pragma unroll
        for (int k = 0; k < TILE / 32; ++k) {
#pragma unroll 2
          for (int i = 0; i < 8; ++i) {
            const int src = i * 4 + (lane >> 3), row = 32 * k + src;
            const int64_t k_row = __shfl_sync(~0u, k_at[k], src), v_row = __shfl_sync(~0u, v_at[k], src);
            const bool live = (mask[k] >> src) & 1;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
              const int c = b * 128 + (lane & 7) * 16;
              const uint32_t dst = to + b * kBox + row * 128 + (((lane & 7) ^ (row & 7)) * 16);
              if (c < D * ES) {
                copy16(dst, static_cast<const char *>(C.k) + k_row * ES + c, live);
                copy16(dst + NB * kBox, static_cast<const char *>(C.v) + v_row * ES + c, live);
              }
            }
          }
        }
        copies_arrive(bar);
        if (lane == 0) {
#pragma unroll
          for (int k = 0; k < TILE / 32; ++k) small.rows_there[stage][k] = mask[k];
          bar_arrive(bar);
        }
        if (++stage == S) stage = 0, parity ^= 1;
      }
    }
    if (!__all_sync(~0u, alive)) {
      settle(smem_at(&small.full[0]), S, stage, parity ^ 1, P.failed);
      return;
    }
    if (aside) {
      asm volatile("bar.sync 2, %0;" ::"n"(kBlock) : "memory");  // the four warps have written the first item's part
      const int h = small.begin[1] * P.members + member, r = small.begin[0], in_group = h % P.blocks_per_head * HB;
      auto slot_of = [&](int i) { return 2 * ((first_from + i) * P.members + member) + (i == 0 ? 1 : 0); };
      if (last_of<Producer>(P.arrived + (int64_t)r * P.items_per_request + h, first_to - first_from + 1, &small.told_aside))
        join<Producer, CT, DP, HB>(P, small.aside, first_to - first_from + 1, slot_of, min(HB, P.group - in_group), true, r,
                                   h / P.blocks_per_head * P.group + in_group);
    }
    return;
  }

  // ---- q of an item, as the B operand: element pairs (2 t4, +8) of head g; e4m3: 4 t4 .. +3, K's order there ----
  uint32_t q[NT][MT][2];
  float to_log2[NT][2];  // scores times this are exponents of 2 (before a softcap: the score itself)
  const float unit = (P.a.softcap > 0 ? 1.0f : kLog2e) * P.a.scale * C.k_scale;
  auto ask_q = [&](int r, int h) {
    const int first = h / P.blocks_per_head * P.group, in_group = h % P.blocks_per_head * HB;
    const uint16_t *row = static_cast<const uint16_t *>(P.a.q) + (int64_t)r * P.a.q_row;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int head = in_group + nt * 8 + g;
      const bool there = head < P.group;
      const uint16_t *x = row + (int64_t)(first + (there ? head : 0)) * P.a.q_head;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int d = m * 16 + (FP8 ? 4 * t4 + 2 * k : 2 * t4 + 8 * k);
          uint32_t v = 0;
          if (there && d < D) {
            if (P.q_pairs) v = *reinterpret_cast<const uint32_t *>(x + d);
            else v = x[d] | (uint32_t)x[d + 1] << 16;
          }
          q[nt][m][k] = v;
        }
      }
    }
  };
  auto take_q = [&]() {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      to_log2[nt][0] = to_log2[nt][1] = unit;
      // q as fp16 times a power of two that brings its largest element near fp16's largest: elements down to 2^-31 of it are
      // exact (of fp16's 11 bits, down to 2^-28)
      if constexpr (FP8) {
        float big = 0.0f;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float2 f;
            if (P.a.dtype == AMAP_BF16) f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&q[nt][m][k]));
            else f = __half22float2(*reinterpret_cast<const __half2 *>(&q[nt][m][k]));
            big = fmaxf(big, fmaxf(fabsf(f.x), fabsf(f.y)));
          }
        }
        big = fmaxf(big, __shfl_xor_sync(~0u, big, 1));
        big = fmaxf(big, __shfl_xor_sync(~0u, big, 2));
        // 2^14 2^e <= big < 2^15 2^e; e within what 2^-e and 2^e are normal numbers for
        const int e = min(max((int)(__float_as_uint(big) >> 23) - 127 - 14, -120), 120);
        const float down = __uint_as_float((uint32_t)(127 - e) << 23), up = __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float2 f;
            if (P.a.dtype == AMAP_BF16) f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&q[nt][m][k]));
            else f = __half22float2(*reinterpret_cast<const __half2 *>(&q[nt][m][k]));
            const __half2 h2 = __floats2half2_rn(f.x * down, f.y * down);
            q[nt][m][k] = *reinterpret_cast<const uint32_t *>(&h2);
          }
        }
        to_log2[nt][0] *= __shfl_sync(~0u, up, 8 * t4);  // of heads 2 t4 and 2 t4 + 1: the columns of S^T here
        to_log2[nt][1] *= __shfl_sync(~0u, up, 8 * t4 + 4);
      }
    }
  };

  float o[NT][MT][4], m[NT][2], l[NT][2];
  auto clear = [&]() {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      m[nt][0] = m[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = 0.0f;
#pragma unroll
      for (int i = 0; i < MT; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.0f;
    }
  };

  ask_q(at.r, at.h * P.members + member);
  take_q();
  clear();
  int64_t item_first = first_place;
  // where a lane's row of the matrix loads lies in a tile, and its chunk 2j (+1 for the upper lanes) swizzled
  uint32_t lane_at[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) lane_at[j] = (warp * ROWS + (lane & 15)) * 128 + (((2 * j) ^ ((lane >> 4) ^ (lane & 7))) * 16);
  const uint32_t ring = smem_at(smem);

  int stage = 0;
  uint32_t parity = 0;
  bool more = true;
#pragma unroll 1
  while (more) {
    // tokens of mine that take part: a range of rows, without those of pages that are not there
    const int row0 = at.t + warp * ROWS, upper = min(max(at.n - row0, 0), ROWS), lower = min(max(at.low - row0, 0), ROWS);
    constexpr uint32_t kAll = ~0u >> (32 - ROWS);
    uint32_t rows = (upper ? kAll >> (ROWS - upper) : 0) & ~(lower ? kAll >> (ROWS - lower) : 0);
    bar_wait(smem_at(&small.full[stage]), parity, P.failed, alive);
    const uint32_t k_at = ring + stage * kStage, v_at = k_at + NB * kBox;
    rows &= small.rows_there[stage][warp * ROWS / 32] >> (warp * ROWS % 32);
    if (rows) {
      if (rows != kAll) {
        // P is zero in the other rows, but what lies there may be anything: zeros to V
        for (int i = lane; i < ROWS * 8 * NB; i += 32) {
          const int row = (i >> 3) & (ROWS - 1);
          if (!((rows >> row) & 1))
            asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(v_at + (i / (ROWS * 8)) * kBox + (warp * ROWS + row) * 128 + (i & 7) * 16), "r"(0) : "memory");
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // before the tensor copies that come to lie there
        __syncwarp();
      }
      // S^T, sixteen tokens by eight heads each, in two sums where there is but one sixteen: a product then need not wait
      // for the one before it
      constexpr int CHAINS = U == 1 ? 2 : 1;
      float s[U][NT][4], other[CHAINS == 2 ? NT : 1][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
#pragma unroll
          for (int u = 0; u < U; ++u) s[u][nt][c] = 0.0f;
          if constexpr (CHAINS == 2) other[nt][c] = 0.0f;
        }
      }
      if constexpr (!FP8) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
          for (int u = 0; u < U; ++u) {
            uint32_t a[4];
            load4(k_at + lane_at[i & 3] + u * 2048 + (i >> 2) * kBox, a);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma<CT>(CHAINS == 2 && (i & 1) ? other[nt] : s[u][nt], a[0], a[1], a[2], a[3], q[nt][i][0], q[nt][i][1]);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < MT; i += 2) {
#pragma unroll
          for (int u = 0; u < U; ++u) {
            uint32_t a[4];
            load4(k_at + lane_at[(i >> 1) & 3] + u * 2048 + (i >> 3) * kBox, a);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              uint32_t a0, a1, a2, a3;
              halves_of(a[2 * j], &a0, &a2);
              halves_of(a[2 * j + 1], &a1, &a3);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma<CT>(CHAINS == 2 && j ? other[nt] : s[u][nt], a0, a1, a2, a3, q[nt][i + j][0], q[nt][i + j][1]);
            }
          }
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int c = 0; c < 4; ++c) s[u][nt][c] = (CHAINS == 2 ? s[u][nt][c] + other[nt][c] : s[u][nt][c]) * to_log2[nt][c & 1];
        }
      }
      if (P.a.softcap > 0) {
        const float in = fminf(1.0f / P.a.softcap, FLT_MAX), out = P.a.softcap * kLog2e;
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int c = 0; c < 4; ++c) s[u][nt][c] = tanh_of(s[u][nt][c] * in) * out;
          }
        }
      }
      if (rows != kAll) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const bool live0 = (rows >> (u * 16 + g)) & 1, live1 = (rows >> (u * 16 + g + 8)) & 1;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int c = 0; c < 4; ++c) s[u][nt][c] = (c < 2 ? live0 : live1) ? s[u][nt][c] : -INFINITY;
          }
        }
      }
      auto highest = [&](int nt, int c) {
        float top = fmaxf(s[0][nt][c], s[0][nt][c + 2]);
        if constexpr (U == 2) top = fmaxf(top, fmaxf(s[U - 1][nt][c], s[U - 1][nt][c + 2]));
        return top;
      };
      bool higher = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) higher |= highest(nt, 0) > m[nt][0] + kSlack || highest(nt, 1) > m[nt][1] + kSlack;
      if (__any_sync(~0u, higher)) {  // seldom after the first tile
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float top = highest(nt, c);
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 4));
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 8));
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 16));
            top = fmaxf(top, m[nt][c]);
            const float keep = top == -INFINITY ? 1.0f : exp2_of(m[nt][c] - top);
            m[nt][c] = top;
            l[nt][c] *= keep;
#pragma unroll
            for (int i = 0; i < MT; ++i) {
              o[nt][i][c] *= keep;
              o[nt][i][c + 2] *= keep;
            }
          }
        }
      }
      uint32_t p[U][NT][2][kTerms<CT>];
      // P V of this step onto O, as it is or (banded: true_type) times `back`
      auto weigh = [&](auto banded, const float (&back)[NT][2]) {
        auto add = [&](int u, int nt, int i, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
          if constexpr (decltype(banded)::value) {
            float part[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < kTerms<CT>; ++w) mma<CT>(part, a0, a1, a2, a3, p[u][nt][0][w], p[u][nt][1][w]);
#pragma unroll
            for (int c = 0; c < 4; ++c) o[nt][i][c] += part[c] * back[nt][c & 1];
          } else {
#pragma unroll
            for (int w = 0; w < kTerms<CT>; ++w) mma<CT>(o[nt][i], a0, a1, a2, a3, p[u][nt][0][w], p[u][nt][1][w]);
          }
        };
        if constexpr (!FP8) {
#pragma unroll
          for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
              uint32_t a[4];
              load4_transposed(v_at + lane_at[i & 3] + u * 2048 + (i >> 2) * kBox, a);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) add(u, nt, i, a[0], a[2], a[1], a[3]);
            }
          }
        } else {  // rows g and g + 8 of the product are elements 2g and 2g + 1
#pragma unroll
          for (int i = 0; i < MT; i += 2) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
              uint32_t a[4];
              load4_transposed(v_at + lane_at[(i >> 1) & 3] + u * 2048 + (i >> 3) * kBox, a);
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                uint32_t a0, a1, a2, a3;
                halves_of(__byte_perm(a[2 * j], 0, 0x3120), &a0, &a1);
                halves_of(__byte_perm(a[2 * j + 1], 0, 0x3120), &a2, &a3);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) add(u, nt, i + j, a0, a1, a2, a3);
              }
            }
          }
        }
      };
      auto terms = [&](auto banded, int u, int nt, const float (&e)[4], float least) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          split<CT, decltype(banded)::value>(e[2 * k], e[2 * k + 1], least, p[u][nt][k]);
#pragma unroll
          for (int w = 0; w < kTerms<CT>; ++w) p[u][nt][k][w] = transposed(p[u][nt][k][w]);
        }
      };
      bool deep = false;
      if constexpr (CT == AMAP_FP16) {
        auto lowest = [&](int nt, int c) {
          float low = fminf(s[0][nt][c], s[0][nt][c + 2]);
          if constexpr (U == 2) low = fminf(low, fminf(s[U - 1][nt][c], s[U - 1][nt][c + 2]));
          return low;
        };
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) deep |= lowest(nt, 0) < m[nt][0] - kDeep || lowest(nt, 1) < m[nt][1] - kDeep;
        deep = __any_sync(~0u, deep);
        if (deep && rows != kAll) {  // or is it only what takes no part
          deep = false;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
              for (int c = 0; c < 4; ++c) deep |= s[u][nt][c] < m[nt][c & 1] - kDeep && s[u][nt][c] > -INFINITY;
            }
          }
          deep = __any_sync(~0u, deep);
        }
      }
      float back[NT][2] = {};
      if (!deep) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float from[2] = {(m[nt][0] == -INFINITY ? 0.0f : m[nt][0]) - kLift<CT>, (m[nt][1] == -INFINITY ? 0.0f : m[nt][1]) - kLift<CT>};
#pragma unroll
          for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int c = 0; c < 4; ++c) s[u][nt][c] = exp2_of(s[u][nt][c] - from[c & 1]);
            l[nt][0] += s[u][nt][0] + s[u][nt][2];
            l[nt][1] += s[u][nt][1] + s[u][nt][3];
            terms(std::false_type(), u, nt, s[u][nt], CT == AMAP_BF16 ? 0x1p-126f : FP8 ? 0.0f : 0x1p-24f);
          }
        }
        weigh(std::false_type(), back);
      } else if constexpr (CT == AMAP_FP16) {
        float least = 0.0f;
        if constexpr (!FP8) {  // what is in no band is zero, unless an infinity is there to meet it
          uint32_t infinite = 0;
          for (int i = lane; i < ROWS * 8 * NB; i += 32) {
            uint32_t x[4];
            asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];"
                         : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3])
                         : "r"(v_at + (i / (ROWS * 8)) * kBox + (warp * ROWS + ((i >> 3) & (ROWS - 1))) * 128 + (i & 7) * 16)
                         : "memory");
#pragma unroll
            for (int w = 0; w < 4; ++w) infinite |= __vcmpeq2(x[w] & 0x7FFF7FFFu, 0x7C007C00u);
          }
          if (__any_sync(~0u, infinite != 0)) least = 0x1p-24f;
        }
        float high[NT][2];  // the band's highest score
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float top = highest(nt, c);
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 4));
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 8));
            high[nt][c] = fmaxf(top, __shfl_xor_sync(~0u, top, 16));
          }
        }
        bool below = true;
#pragma unroll 1
        for (int band = 0; below && band < 6; ++band) {  // down to 2^-144 of the highest
          below = false;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int c = 0; c < 2; ++c)
              back[nt][c] = high[nt][c] == -INFINITY ? 0.0f : exp2_of(high[nt][c] - m[nt][c] - kSlack);
#pragma unroll
            for (int u = 0; u < U; ++u) {
              float e[4];
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                const float x = s[u][nt][c], top = high[nt][c & 1], bottom = top - kBand;
                const bool in = !(x <= bottom) && (band == 0 || x <= top);  // NaN: in the first
                below |= x <= bottom && x > -INFINITY && bottom > -INFINITY;
                e[c] = in ? exp2_of(x - top + (kLift<CT> + kSlack)) : 0.0f;
              }
              l[nt][0] += (e[0] + e[2]) * back[nt][0];
              l[nt][1] += (e[1] + e[3]) * back[nt][1];
              terms(std::true_type(), u, nt, e, least);
            }
            high[nt][0] -= kBand;
            high[nt][1] -= kBand;
          }
          weigh(std::true_type(), back);
          below = __any_sync(~0u, below);
        }
      }
    }
    __syncwarp();
    if (lane == 0) bar_arrive(smem_at(&small.empty[stage]));
    if (++stage == S) stage = 0, parity ^= 1;

    more = at.more();
    if (at.left > 1 && more) {
      at.advance(P);
      continue;
    }
    // ---- the end of an item, or of this block's part of it: join the warps ----
    const int r = at.r, h = at.h * P.members + member, tiles = Line::tiles(P, at.n);
    if (more) {
      at.advance(P);
      ask_q(at.r, at.h * P.members + member);  // the next item's, under way while this one is put away
    }
    const int64_t item_last = item_first + tiles - 1;
    const bool whole = item_first >= u0 && item_last < u1;
    const int first = h / P.blocks_per_head * P.group, in_group = h % P.blocks_per_head * HB;
    const int heads = min(HB, P.group - in_group);
    const int slot = 2 * (team * P.members + member) + (item_first >= u0 ? 1 : 0);  // a block has at most two parts: its first item's and its last's
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if (nt * 8 >= heads) break;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float sum = l[nt][c];
        sum += __shfl_xor_sync(~0u, sum, 4);
        sum += __shfl_xor_sync(~0u, sum, 8);
        sum += __shfl_xor_sync(~0u, sum, 16);
        if (g == 0) *reinterpret_cast<float2 *>(joint + (warp * 8 + 2 * t4 + c) * kPitch + DP) = make_float2(m[nt][c], sum);
      }
      sync_consumers();
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const float *ml = joint + (2 * t4 + c) * kPitch + DP;
        const float top = fmaxf(fmaxf(ml[0], ml[8 * kPitch]), fmaxf(ml[16 * kPitch], ml[24 * kPitch]));
        const float f = top == -INFINITY ? 1.0f : exp2_of(m[nt][c] - top);
        float *to = joint + (warp * 8 + 2 * t4 + c) * kPitch;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          to[i * 16 + (FP8 ? 2 * g : g)] = o[nt][i][c] * f;
          to[i * 16 + (FP8 ? 2 * g + 1 : g + 8)] = o[nt][i][c + 2] * f;
        }
      }
      sync_consumers();
      const int n_heads = min(8, heads - nt * 8);
      for (int i = tid; i < n_heads * (DP / 2); i += kThreads) {
        const int in = i / (DP / 2), d = i % (DP / 2) * 2, head = nt * 8 + in;
        if (d >= D) continue;
        const float *ml = joint + in * kPitch + DP;
        const float top = fmaxf(fmaxf(ml[0], ml[8 * kPitch]), fmaxf(ml[16 * kPitch], ml[24 * kPitch]));
        float sum = 0.0f;
        float2 y = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          sum += ml[w * 8 * kPitch + 1] * (top == -INFINITY ? 1.0f : exp2_of(ml[w * 8 * kPitch] - top));
          const float2 v = *reinterpret_cast<const float2 *>(joint + (w * 8 + in) * kPitch + d);
          y.x += v.x;
          y.y += v.y;
        }
        if (whole) {
          const float f = sum == 0.0f ? 0.0f : C.v_scale / sum;
          write_pair(P, (int64_t)r * P.a.out_row + (int64_t)(first + in_group + head) * P.a.out_head + d, y.x * f, y.y * f);
          if (d == 0 && P.a.lse)
            P.a.lse[(int64_t)r * P.a.lse_row + first + in_group + head] = sum == 0.0f ? -INFINITY : (top - kLift<CT> + log2f(sum)) * kLn2;
        } else {
          *reinterpret_cast<float2 *>(P.part_o + ((int64_t)slot * HB + head) * DP + d) = y;
          if (d == 0) reinterpret_cast<float2 *>(P.part_ml)[(int64_t)slot * HB + head] = make_float2(top, sum);
        }
      }
      sync_consumers();
    }
    if (!whole) {  // uniform over the block
      if (aside && item_first < u0) {
        asm volatile("bar.arrive 2, %0;" ::"n"(kBlock) : "memory");
      } else {
        const int from = team_of(item_first), to = team_of(item_last);
        auto slot_of_team = [&](int b) { return 2 * (b * P.members + member) + (b == from ? 1 : 0); };
        int32_t *item = P.arrived + (int64_t)r * P.items_per_request + h;
        if (to - from < kDirect) {
          if (last_of<Consumers>(item, to - from + 1, &small.told))
            join<Consumers, CT, DP, HB>(P, joined, to - from + 1, [&](int i) { return slot_of_team(from + i); }, heads, true, r, first + in_group);
        } else {
          // of the items with parts in a group of teams, one at most began before the group and one at most, among those
          // with more than kDirect parts, begins in it: two counters
          const int group = team / kGroup, b0 = max(from, group * kGroup), b1 = min(to, group * kGroup + kGroup - 1);
          if (last_of<Consumers>(P.grouped + 2 * (group * P.members + member) + (from >= group * kGroup ? 1 : 0), b1 - b0 + 1, &small.told)) {
            join<Consumers, CT, DP, HB>(P, joined, b1 - b0 + 1, [&](int i) { return slot_of_team(b0 + i); }, heads, false, r, first + in_group);
            const int g0 = from / kGroup, g1 = to / kGroup;
            if (last_of<Consumers>(item, g1 - g0 + 1, &small.told))
              join<Consumers, CT, DP, HB>(P, joined, g1 - g0 + 1, [&](int i) { return slot_of_team(max(from, (g0 + i) * kGroup)); }, heads, true, r,
                                          first + in_group);
          }
        }
      }
    }
    if (more) {
      item_first = u1 - at.rest;
      take_q();
      clear();
    }
  }
  if (!alive) settle(smem_at(&small.full[0]), S, stage, parity, P.failed);
}

template <int CT, bool FP8, int DP, int NT>
int run(Params &P, void *stream) {
  constexpr int RB = DP * (FP8 ? 1 : 2);
  constexpr int TILE = 16 * kSixteens<RB> * kWarps;
  constexpr int S = kStages<RB, kResident<DP, NT>>;
  constexpr size_t smem = (size_t)S * 2 * TILE * RB + sizeof(float) * kWarps * 8 * (DP + 4) + sizeof(Small<S, TILE>);
  // the block's shared memory is asked for, and how many blocks a multiprocessor then holds, once per device
  static std::atomic<int> known[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess || dev >= 64) {
    cudaGetLastError();
    return refuse(AMAP_ECUDA, e != cudaSuccess ? cudaGetErrorString(e) : "device number");
  }
  int blocks = known[dev].load(std::memory_order_relaxed);
  if (blocks == 0) {
    int per_sm = 0;
    e = cudaFuncSetAttribute(attend_kernel<CT, FP8, DP, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, attend_kernel<CT, FP8, DP, NT>, kBlock, smem);
    if (e != cudaSuccess || per_sm < 1) {
      cudaGetLastError();
      return refuse(AMAP_ECUDA, e != cudaSuccess ? cudaGetErrorString(e) : "the kernel does not fit a multiprocessor");
    }
    blocks = device_sms() * std::min(per_sm, kMostBlocksPerSm);
    SERVE_REQUIRE((blocks + kGroup - 1) / kGroup <= kJoined<DP>, AMAP_EUNSUPPORTED, "more multiprocessors than an item's parts can be joined from");
    known[dev].store(blocks, std::memory_order_relaxed);
  }
  // a team's blocks: the largest divisor of the items of a request that leaves no more than a fiftieth of the device idle
  for (int members = 1; members <= std::min(P.items_per_request, kMostMembers); ++members)
    if (P.items_per_request % members == 0 && blocks / members * members * 50 >= blocks * 49) P.members = members;
  P.rounds = P.items_per_request / P.members;
  const int64_t most = (int64_t)P.a.n_requests * P.rounds * std::max<int64_t>(1, ((int64_t)P.a.max_pages * P.a.cache.page_size + TILE - 1) / TILE);
  SERVE_REQUIRE((int64_t)P.a.n_requests * P.rounds * (((int64_t)P.a.max_pages * P.a.cache.page_size) / TILE + 1 + kEntry) / (blocks / P.members) < 0x7FFFFFFF,
                AMAP_EOVERFLOW, "more tokens than a block can count");
  return launch(attend_kernel<CT, FP8, DP, NT>, dim3((unsigned)(std::min<int64_t>(blocks / P.members, most) * P.members)), kBlock, smem, stream, P);
}

template <int CT, bool FP8, int DP>
int run_heads(Params &P, int nt, void *stream) {
  switch (nt) {
    case 1: return run<CT, FP8, DP, 1>(P, stream);
    case 2: return run<CT, FP8, DP, 2>(P, stream);
    default:
      if constexpr (DP < 256) return run<CT, FP8, DP, 4>(P, stream);
      else return run<CT, FP8, DP, 2>(P, stream);
  }
}

template <int CT, bool FP8>
int run_dim(Params &P, int dp, int nt, void *stream) {
  switch (dp) {
    case 64:
      if constexpr (!FP8) return run_heads<CT, FP8, 64>(P, nt, stream);
    case 128: return run_heads<CT, FP8, 128>(P, nt, stream);
    default: return run_heads<CT, FP8, 256>(P, nt, stream);
  }
}

// head sizes are padded to what a kernel is built for (in shared memory only: no more is read): whole rows of 128 bytes
int padded_dim(int d, int es) { return d * es <= 128 ? 128 / es : d <= 128 ? 128 : 256; }
// eights of q heads that share a pass over the cache: all of a group where its accumulators fit the registers
int eights(int group, int dp) {
  const int most = dp < 256 ? 4 : 2;
  return group <= 8 ? 1 : group <= 16 || most == 2 ? 2 : 4;
}



int check_shape(int32_t n_requests, int32_t q_heads, int32_t kv_heads, int32_t head_dim) {
  SERVE_REQUIRE(n_requests >= 1 && n_requests <= 0xFFFF, AMAP_EINVAL, "requests: 1 .. 65535");
  SERVE_REQUIRE(q_heads >= 1 && q_heads <= 0xFFFF && kv_heads >= 1 && q_heads % kv_heads == 0, AMAP_EINVAL, "q heads: a multiple of the cache's heads");
  SERVE_REQUIRE(head_dim >= 8 && head_dim <= 256 && head_dim % 8 == 0, AMAP_EUNSUPPORTED, "head size: a multiple of 8, up to 256");
  return AMAP_OK;
}

struct Workspace {
  int64_t ml, failed, grouped, arrived, bytes;  // offsets; the partial outputs come first
};
Workspace workspace(int32_t n_requests, int32_t q_heads, int32_t kv_heads, int32_t head_dim) {
  const int dp = head_dim <= 128 ? 128 : 256, group = q_heads / kv_heads, hb = 8 * eights(group, dp);
  const int64_t blocks = (int64_t)device_sms() * kMostBlocksPerSm, items = (int64_t)n_requests * kv_heads * ((group + hb - 1) / hb);
  Workspace w;
  w.ml = 2 * blocks * hb * dp * 4;
  w.failed = w.ml + 2 * blocks * hb * 8;
  w.grouped = w.failed + 16;
  w.arrived = w.grouped + (blocks / kGroup + kMostMembers) * 2 * 4;
  w.bytes = (w.arrived + items * 4 + 255) / 256 * 256;
  return w;
}

using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                            const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

Encode encoder() {
  static std::atomic<Encode> known{nullptr};
  Encode f = known.load(std::memory_order_relaxed);
  if (!f) {
    void *p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      return nullptr;
    }
    f = reinterpret_cast<Encode>(p);
    known.store(f, std::memory_order_relaxed);
  }
  return f;
}

bool encode(const amap_cache &c, void *base, int64_t page, int64_t token, int64_t head, int box, CUtensorMap *out) {
  const Encode f = encoder();
  if (!f) return false;
  const int64_t es = dtype_bytes(c.dtype), row = c.head_dim * es;
  const cuuint64_t dims[4] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.page_size, (cuuint64_t)c.heads, (cuuint64_t)c.n_pages};
  cuuint64_t strides[3];
  const int64_t given[3] = {token * es, head * es, page * es};
  for (int i = 0; i < 3; ++i) {
    if (dims[i + 1] == 1) strides[i] = (cuuint64_t)row;  // a stride that no element uses
    else if (given[i] <= 0 || given[i] >= ((int64_t)1 << 40)) return false;
    else strides[i] = (cuuint64_t)given[i];
  }
  const cuuint32_t boxes[4] = {(cuuint32_t)(128 / es), (cuuint32_t)box, 1, 1}, ones[4] = {1, 1, 1, 1};
  const CUtensorMapDataType type = c.dtype == AMAP_E4M3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : c.dtype == AMAP_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  return f(out, type, 4, base, dims, strides, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int check_readable(const amap_cache &c) {
  if (const int rc = check_cache(c)) return rc;
  const int es = dtype_bytes(c.dtype), per16 = 16 / es;
  SERVE_REQUIRE(c.head_dim >= 8 && c.head_dim <= 256 && c.head_dim % per16 == 0, AMAP_EUNSUPPORTED, "head size: whole 16-byte chunks, up to 256 elements");
  for (const int64_t s : {c.k_page, c.k_token, c.k_head, c.v_page, c.v_token, c.v_head})
    SERVE_REQUIRE(s % per16 == 0, AMAP_EALIGN, "cache strides: whole 16-byte chunks");
  SERVE_REQUIRE(aligned(c.k, 16) && aligned(c.v, 16), AMAP_EALIGN, "cache: aligned to 16 bytes");
  return AMAP_OK;
}

void encode_both(const amap_cache &c, amap_cache_maps *out) {
  static_assert(sizeof(out->k_map) == sizeof(CUtensorMap), "a tensor map is 128 bytes");
  memset(out, 0, sizeof *out);
  if (c.page_size % 8) return;
  int shift = 3;
  while (shift < 6 && c.page_size % (2 << shift) == 0) ++shift;
  CUtensorMap k, v;  // aligned to 64 bytes, as the encoder wants them
  if (!encode(c, c.k, c.k_page, c.k_token, c.k_head, 1 << shift, &k) || !encode(c, c.v, c.v_page, c.v_token, c.v_head, 1 << shift, &v)) return;
  memcpy(out->k_map, &k, sizeof k);
  memcpy(out->v_map, &v, sizeof v);
  out->box_shift = shift;
  out->usable = 1;
}

}  // namespace

extern "C" int amap_attend_workspace(int32_t n_requests, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int64_t *bytes, int64_t *failed) {
  SERVE_REQUIRE(bytes, AMAP_EINVAL, "null pointer");
  if (const int rc = check_shape(n_requests, q_heads, kv_heads, head_dim)) return rc;
  const Workspace w = workspace(n_requests, q_heads, kv_heads, head_dim);
  *bytes = w.bytes;
  if (failed) *failed = w.failed;
  return accept();
}

extern "C" int amap_cache_encode(const amap_cache *cache, amap_cache_maps *out) {
  SERVE_REQUIRE(cache && out, AMAP_EINVAL, "null pointer");
  if (const int rc = check_readable(*cache)) return rc;
  encode_both(*cache, out);
  return accept();
}

extern "C" int amap_attend(const amap_attend_args *a, void *cuda_stream) {
  SERVE_REQUIRE(a, AMAP_EINVAL, "null pointer");
  if (const int rc = check_readable(a->cache)) return rc;
  const amap_cache &c = a->cache;
  if (const int rc = check_shape(a->n_requests, a->q_heads, c.heads, c.head_dim)) return rc;
  SERVE_REQUIRE(a->dtype == AMAP_BF16 || a->dtype == AMAP_FP16, AMAP_EINVAL, "type: bf16 or fp16");
  SERVE_REQUIRE(c.dtype == AMAP_E4M3 || c.dtype == a->dtype, AMAP_EINVAL, "a 16-bit cache has the type of q");
  SERVE_REQUIRE(a->q && a->out && a->block_table && a->seq_lens && a->workspace, AMAP_EINVAL, "null pointer");
  SERVE_REQUIRE(a->max_pages >= 1 && a->table_stride >= a->max_pages, AMAP_EINVAL, "table rows overlap");
  SERVE_REQUIRE((int64_t)a->max_pages * c.page_size <= 0x7FFFFFFF, AMAP_EOVERFLOW, "a table row holds more than 2^31-1 tokens");
  SERVE_REQUIRE(std::isfinite(a->scale) && std::isfinite(a->softcap) && a->softcap >= 0 && a->window >= 0 && a->reserved == 0, AMAP_EINVAL,
                "scale is finite, softcap and window are not negative");
  SERVE_REQUIRE(aligned(a->q, 2) && aligned(a->out, 2) && aligned(a->lse, 4) && aligned(a->block_table, 4) && aligned(a->seq_lens, 4) &&
                    aligned(a->workspace, 256), AMAP_EALIGN, "misaligned pointer");
  Span qs, os;
  qs.hi = os.hi = (int64_t)c.head_dim * 2;
  qs.add(a->n_requests, a->q_row, 2);
  qs.add(a->q_heads, a->q_head, 2);
  os.add(a->n_requests, a->out_row, 2);
  os.add(a->q_heads, a->out_head, 2);
  SERVE_REQUIRE(!overlap(a->q, qs, a->out, os), AMAP_EINVAL, "q and out overlap");

  const Workspace w = workspace(a->n_requests, a->q_heads, c.heads, c.head_dim);
  SERVE_REQUIRE(a->workspace_bytes >= w.bytes, AMAP_EINVAL, "workspace too small");
  const int dp = padded_dim(c.head_dim, dtype_bytes(c.dtype));
  Params P = {};
  P.a = *a;
  P.group = a->q_heads / c.heads;
  const int nt = eights(P.group, dp);
  P.blocks_per_head = (P.group + 8 * nt - 1) / (8 * nt);
  P.items_per_request = c.heads * P.blocks_per_head;
  SERVE_REQUIRE((int64_t)a->n_requests * P.items_per_request <= 0x7FFFFFFF, AMAP_EOVERFLOW, "more than 2^31-1 pairs of request and head");
  // token / page_size for tokens below 2^31: a shift, or the high word of a product with ceil(2^(32+s) / page_size),
  // s = floor(log2 page_size), whose excess over 2^(32+s) is at most page_size - 1 < 2^(s+1): exact up to 2^31
  int s = 0;
  while ((2u << s) <= (uint32_t)c.page_size) ++s;
  P.div_shift = s;
  if (c.page_size != 1 << s) P.div_mul = (uint32_t)((((uint64_t)1 << (32 + s)) + c.page_size - 1) / c.page_size);
  P.q_pairs = aligned(a->q, 4) && a->q_row % 2 == 0 && a->q_head % 2 == 0;
  P.out_pairs = aligned(a->out, 4) && a->out_row % 2 == 0 && a->out_head % 2 == 0;
  char *ws = static_cast<char *>(a->workspace);
  P.part_o = reinterpret_cast<float *>(ws);
  P.part_ml = reinterpret_cast<float *>(ws + w.ml);
  P.failed = reinterpret_cast<int32_t *>(ws + w.failed);
  P.grouped = reinterpret_cast<int32_t *>(ws + w.grouped);
  P.arrived = reinterpret_cast<int32_t *>(ws + w.arrived);
  amap_cache_maps made;
  const amap_cache_maps *maps = a->maps;
  if (!maps) {
    encode_both(c, &made);
    maps = &made;
  }
  P.tensor_copies = maps->usable;
  P.box_shift = maps->box_shift;
  if (maps->usable) {
    SERVE_REQUIRE(maps->box_shift >= 3 && maps->box_shift <= 6 && c.page_size % (1 << maps->box_shift) == 0, AMAP_EINVAL, "maps of another cache");
    memcpy(&P.k_map, maps->k_map, sizeof P.k_map);
    memcpy(&P.v_map, maps->v_map, sizeof P.v_map);
  }
  if (c.dtype == AMAP_E4M3) return run_dim<AMAP_FP16, true>(P, dp, nt, cuda_stream);
  return c.dtype == AMAP_BF16 ? run_dim<AMAP_BF16, false>(P, dp, nt, cuda_stream) : run_dim<AMAP_FP16, false>(P, dp, nt, cuda_stream);
}
