// Attention of one new token per request over a paged cache of 4 bits (amap_packed).
//
// Mathematics.  That of serve_attend.cu with K = low_K + step_K c and V = low_V + step_V d by groups of elements:
//   s_t = scale sum_g (step_K <q_g, c_tg> + low_K sum(q_g)),   O = sum_t sum_g (P_t step_V) d_tg + P_t low_V
// so the matrix instructions see the codes themselves.  A code's four bits, masked out where they lie in a 16-bit half, are
// an fp16 number: code x 2^-21 in bits 3 .. 6, code x 2^-17 in bits 7 .. 10 (fp16 counts evenly from 0 to 2^11 of its
// smallest steps), exact in the products: no conversion.  q's elements that meet the lower kind of K's codes are taken 16
// times as large; of O the lower kind's rows are scaled at the end.  Five operations for eight codes: four masks, and the
// halves' bytes exchanged for the last two of four.  Tokens are the M side of both products; P is transposed in between.
//
// Precision.  q is fp16 times a power of two that brings its largest element near 2^11 (2^15 where it meets the lower kind):
// elements down to 2^-27 of it are exact (of fp16's 11 bits, down to 2^-24).  P step_V enters as two fp16 terms of 11 bits, the
// second what the first leaves over.  They are taken relative to a reference R that follows the largest WEIGHT of a token so
// far, P times its largest |low_V| or step_V, rather than the largest P: so the products lie near fp16's upper end for values of
// any size (2^-110 and more), and an element is off by 2^-30 of the largest weight of a token, over all groups of the head, at most:
// a token is cut off only where its weight is 2^-24 of that, and so are a group's codes whose steps are 2^-24 of another group's (down
// to 2^-18 a 16-bit output does not show it).  A lift of its own for each group would be 8 more multiplications for two.  P itself, l and the sums of P low_V are in 32 bits, where R may be far from the largest score; values above 2^24 are
// scaled, so that neither end of their range is met (kLarge).  The matrix
// unit cuts its sums off to 24 bits, counted from the largest of the exponent FIELDS: fp16 numbers below 2^-14 stand in line as if
// they were 2^-14.  So codes in bits 0 .. 3 and 4 .. 7 lost up to four bits (sums of 16 products off by 2^-21.8 of the largest one,
// in the bits 3 .. 10 by 2^-26.2 as with codes that are ordinary numbers; root mean squares): lse was off by 4e-7, relative,
// for keys of 16 times the variance of one channel, and is by 4e-8 (products and sums in 32 bits: 3e-8).  V's codes are counted
// down in every second cell, so that what is summed over a long request stays small beside what is cut off at every step.
//
// Bound: a warp's own chain, with two computing warps to a scheduler.  A cell of 16 tokens (2304 bytes of 128 elements in groups of
// 64) is 300 instructions of a warp, of them 135 on the half-rate integer pipe, 90 on the multipliers and 24 products of 16 x 8 x 16
// (2.03 clocks of a multiprocessor each): at full issue some 115 clocks, where the cell takes 99 to come from HBM and is
// there after 165.  No unit is at its limit (issue slots 49 %, integer pipe 46, products 31, DRAM 45); warps wait for their own
// last instruction first, for one another and the pipes next, and a quarter as long for instructions to come: the loop with its
// rare branches is larger than the nearest instruction memory, and ptxas' order of it is worth some 4 % either way.  Copies alone
// take 116 us of the 162 of 64 requests; a third block a multiprocessor (128 registers) brings nothing.
//
// Split, ring and join are serve_attend.cu's.  A tile is 128 tokens: eight cells, copied in bulk in runs that every page divides into.
//
// Measured: 64 requests of up to 16384 tokens, 32 q heads over 8 of 128 elements, bf16, groups of 64 (605 MB) 162 us = 3.7
// TB/s; one request of 131009 tokens, fp16, groups of 32 (168 MB) 53 us = 3.2; 128 requests of up to 4096, 64 q heads over 4
// (155 MB) 95 us; 33 tokens 6.3 us.
#define AMAP_ATTEND_PARTS_ONLY
#include "serve_attend.cu"
#include "serve_packed.cuh"

namespace {

constexpr int kPackedTile = 128, kCells = kPackedTile / kCell, kOwn = kCells / kWarps;  // cells of a tile; of a warp
constexpr int kLook = 32 / kCells;                                                      // tiles whose pages are looked up at a time
static_assert(kOwn == 2, "a warp's cells of a tile");
constexpr float kUp = 0x1p9f, kTop = 0x1p15f;  // P is kUp times what it stands for; P step_V above kTop renews the reference
constexpr float kNone = -3e38f;            // the reference before the first token
constexpr float kLeast = 0x1p-90f;         // a smaller |low| or step counts as this much
constexpr float kMost = 0x1p72f;           // a sum of P above this renews the reference, too (tokens whose V is constant have no step)
// Where a |low| or step is above kLarge the item's numbers of V are taken times a power of 2 from then on, which brings the largest
// below 1.  So P |low| is below kMost kLarge (and below 2 kUp where the reference is new), with room for a sum of 2^27 of them, and the
// most probable token's P is 2^-24 at least, far enough from 2^-126 for 32 bits to hold what l adds up.
constexpr float kLarge = 0x1p24f;
// O is handed over as this much of itself, so that a sum of the largest values has room; what divides it by l takes that off
constexpr float kRoom = 0x1p-24f;

template <int NS> constexpr int kPackedResident = NS >= 8 ? 1 : 2;
// Stages of the ring: what a multiprocessor's shared memory has room for beside the rest of its blocks, up to eight.
constexpr int least(int a, int b) { return a < b ? a : b; }
template <int NS, int NG, int RESIDENT>
constexpr int kPackedStages = least(8, (226 * 1024 / RESIDENT - 3 * 1024 - (int)sizeof(float) * kWarps * 8 * (32 * NS + 4)) / (kCells * cell_bytes(NS, NG)));

struct PackedParams {
  Params p;
  const char *data;
  int64_t page, head;  // bytes
  int32_t run;         // cells that every page divides into, up to a tile's: 1, 2, 4 or 8
};

__device__ __forceinline__ void bulk_copy(uint32_t dst, const void *src, int bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
template <int WORDS>
__device__ __forceinline__ void load_words(const char *at, uint32_t *r) {
  if constexpr (WORDS == 4) {
    const uint4 v = *reinterpret_cast<const uint4 *>(at);
    r[0] = v.x, r[1] = v.y, r[2] = v.z, r[3] = v.w;
  } else if constexpr (WORDS == 2) {
    const uint2 v = *reinterpret_cast<const uint2 *>(at);
    r[0] = v.x, r[1] = v.y;
  } else {
    r[0] = *reinterpret_cast<const uint32_t *>(at);
  }
}
// the first of a sum of products: nothing has to be set to zero ahead of it
__device__ __forceinline__ void mma_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}
// K codes of a lane: slabs side by side, four at a time; three are single words (their rows are 12 bytes)
template <int NS>
__device__ __forceinline__ void load_k(const char *at, int token, int t4, uint32_t (&r)[NS]) {
#pragma unroll
  for (int first = 0; first < NS; first += 4) {
    const int wide = NS - first < 4 ? NS - first : 4;
    const char *from = at + first * 256 + (token * 4 + t4) * 4 * wide;
    if (wide == 4) load_words<4>(from, &r[first]);
    else if (wide == 2) load_words<2>(from, &r[first]);
    else
      for (int i = 0; i < wide; ++i) load_words<1>(from + 4 * i, &r[first + i]);
  }
}
// V codes of the COUNT (1 or 2) slabs from `slab` on, which lie side by side where they are two
template <int NS, int COUNT>
__device__ __forceinline__ void load_v(const char *at, int lane, int slab, uint32_t (&r)[COUNT][2]) {
  const int first = slab & ~1, wide = NS - first < 2 ? 1 : 2;
  const char *from = at + first * 256 + lane * 8 * wide + (slab - first) * 8;
  if constexpr (COUNT == 2) load_words<4>(from, &r[0][0]);
  else load_words<2>(from, &r[0][0]);
}
__device__ __forceinline__ float step_of(uint32_t w) { return __uint_as_float(w * 0x10000u); }
__device__ __forceinline__ float low_of(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// a lower and an upper code of both halves (kTurn); with the halves' bytes exchanged, the other two
constexpr uint32_t kLower = 0x00780078u, kUpper = 0x07800780u;
__device__ __forceinline__ uint32_t bytes_exchanged(uint32_t w) { return __byte_perm(w, 0, 0x2301); }

__device__ __forceinline__ float power_of_2(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }  // -126 .. 127
// low and step times 2^e
__device__ __forceinline__ uint32_t scaled(uint32_t w, int e) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"((uint32_t)(127 + e) * (0x10001u << 7)));
  return r;
}
// the larger step, and the larger |low| with one sign or the other; NaN counts for nothing
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// a and b as fp16 in one word, and what that leaves over, likewise
__device__ __forceinline__ void two_terms(float a, float b, uint32_t (&term)[2]) {
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(term[0]) : "f"(b), "f"(a));
  float x, y;
  asm("{ .reg .b16 l, h; mov.b32 {l, h}, %2; sub.f32.f16 %0, l, %3; sub.f32.f16 %1, h, %4; }" : "=f"(x), "=f"(y) : "r"(term[0]), "f"(a), "f"(b));
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(term[1]) : "f"(-y), "f"(-x));
}

// NS: slabs of 32 elements of a head; SG: slabs of a group.  A block has eight q heads: with sixteen, whose sums leave room for one
// block a multiprocessor, 128 requests of 64 q heads to 4 take 106 us instead of 90, although the codes are then unpacked once.
template <int NS, int SG>
__global__ void __launch_bounds__(kBlock, (kPackedResident<NS>)) attend_packed_kernel(const __grid_constant__ PackedParams PP) {
  const Params &P = PP.p;
  constexpr int NG = NS / SG, D = 32 * NS, C = cell_bytes(NS, NG), kStage = kCells * C;
  constexpr int S = kPackedStages<NS, NG, kPackedResident<NS>>;
  constexpr int HB = 8;
  constexpr int kPair = NG % 2 == 0 ? 2 : 1;     // groups whose products are summed at a time
  constexpr int kPitch = D + 4;
  extern __shared__ __align__(1024) char smem[];
  float *joint = reinterpret_cast<float *>(smem + S * kStage);  // [warps][8][kPitch]
  using Line = Cursor<kPackedTile>;
  Small<S, kPackedTile> &small = *reinterpret_cast<Small<S, kPackedTile> *>(joint + kWarps * 8 * kPitch);
  float2(*const joined)[8] = reinterpret_cast<float2(*)[8]>(joint);  // [kJoined<D>][8], while `joint` is idle
  static_assert(sizeof(float2) * 8 * kJoined<D> <= sizeof(float) * kWarps * 8 * kPitch, "room for the parts of an item");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
  const amap_cache &cache = P.a.cache;
  if (tid == 0) {
    for (int i = 0; i < S; ++i) {
      bar_init(smem_at(&small.full[i]), 1);
      bar_init(smem_at(&small.empty[i]), kWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  pdl_begin();
  Piece<kPackedTile> piece;
  if (!piece.find(P, small)) return;
  Line &at = piece.at;
  const int team = piece.team, member = piece.member;
  const int64_t u0 = piece.u0, u1 = piece.u1;
  bool alive = true;

  if (warp == kWarps) {
    // ---- the producer: it looks pages up for kLook tiles of an item at a time, a group of them ahead (a look takes about as
    // long as four tiles take to come: with one at a time 64 requests were 172 us); a lane has a run of cells that lie
    // side by side in a page, as many as every page divides into ----
    const int run = PP.run, ahead = lane / kCells, cell0 = lane % kCells;
    int entry = -1, offset = 0, from_cell = 0, n_cells = 0, tiles = 0;
    auto look = [&]() {
      tiles = min(kLook, min(at.left, at.rest));
      const int token = at.t + ahead * kPackedTile + cell0 * kCell;
      n_cells = 0;
      if (ahead < tiles && cell0 % run == 0 && token < at.n && token + run * kCell > at.low) {
        const uint32_t page = P.div_mul ? __umulhi((uint32_t)token, P.div_mul) >> P.div_shift : (uint32_t)token >> P.div_shift;
        offset = token - (int)page * cache.page_size;
        entry = P.a.block_table[(int64_t)at.r * P.a.table_stride + page];
        from_cell = max(at.low - token, 0) / kCell;
        n_cells = min(run, (at.n - token + kCell - 1) / kCell) - from_cell;
      }
    };
    int stage = 0;
    uint32_t parity = 1;  // the first round of waits finds every stage empty
    look();
    for (bool more = true; more && __all_sync(~0u, alive);) {
      const int head = (at.h * P.members + member) / P.blocks_per_head;
      if ((uint32_t)entry >= (uint32_t)cache.n_pages) n_cells = 0;
      const int count = n_cells, first = cell0 + from_cell, t = at.t, n = at.n, low = at.low, there = tiles;
      const uint32_t cells = __reduce_or_sync(~0u, count > 0 ? ((1u << count) - 1) << (ahead * kCells + first) : 0u);
      const char *from = PP.data + (count > 0 ? (int64_t)entry * PP.page + (int64_t)head * PP.head + (int64_t)(offset / kCell + from_cell) * C : 0);
      at.t += (there - 1) * kPackedTile;
      at.left -= there - 1;
      at.rest -= there - 1;
      more = at.more();
      if (more) {
        at.advance(P);
        look();
      }
      for (int k = 0; k < there; ++k) {
        // of the lane-th warp: its tokens that take part
        const int row0 = t + k * kPackedTile + lane * 32, upper = min(max(n - row0, 0), 32), lower = min(max(low - row0, 0), 32);
        const uint32_t in_tile = cells >> (k * kCells) & ((1u << kCells) - 1), own = in_tile >> (lane * kOwn & 31);
        const uint32_t rows = (upper ? ~0u >> (32 - upper) : 0) & ~(lower ? ~0u >> (32 - lower) : 0) & ((own & 1 ? 0xFFFFu : 0u) | (own & 2 ? 0xFFFF0000u : 0u));
        bar_wait(smem_at(&small.empty[stage]), parity, P.failed, alive);
        if (!__all_sync(~0u, alive)) break;
        const uint32_t bar = smem_at(&small.full[stage]);
        if (lane < kWarps) small.rows_there[stage][lane] = rows;
        __syncwarp();
        if (lane == 0) bar_arrive_bytes(bar, __popc(in_tile) * C);
        __syncwarp();
        if (count > 0 && ahead == k) bulk_copy(smem_at(smem + stage * kStage) + first * C, from, count * C, bar);
        if (++stage == S) stage = 0, parity ^= 1;
      }
    }
    if (!__all_sync(~0u, alive)) {
      settle(smem_at(&small.full[0]), S, stage, parity ^ 1, P.failed);
      return;
    }
    if (piece.aside) join_aside<D, HB>(P, small, piece, 0.0f);
    return;
  }

  // ---- q of an item, as the B operand: of head g, of each slab the elements 8 t4 .. +7 ----
  uint32_t q[NS][4];
  // of heads 2 t4 and 2 t4 + 1, S^T's columns here: what makes exponents of 2 of the products' sums, never zero (with a softcap
  // it makes scores, which are brought back to the products' unit once they are capped); sums of q over a group, as the products count it
  float to_log2[2], sums[NG][2];
  const float unit = (P.a.softcap > 0 ? 1.0f : kLog2e) * P.a.scale;
  auto ask_q = [&](int r, int h) {
    const int first = h / P.blocks_per_head * P.group, in_group = h % P.blocks_per_head * HB;
    const uint16_t *row = static_cast<const uint16_t *>(P.a.q) + (int64_t)r * P.a.q_row;
    const int head = in_group + g;
    const bool there = head < P.group;
    const uint16_t *x = row + (int64_t)(first + (there ? head : 0)) * P.a.q_head;
#pragma unroll
    for (int j = 0; j < NS; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int d = j * 32 + t4 * 8 + i * 2;
        uint32_t v = 0;
        if (there) v = P.q_pairs ? *reinterpret_cast<const uint32_t *>(x + d) : x[d] | (uint32_t)x[d + 1] << 16;
        q[j][i] = v;
      }
    }
  };
  auto as_floats = [&](uint32_t v) {
    return P.a.dtype == AMAP_BF16 ? make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u)) : __half22float2(*reinterpret_cast<const __half2 *>(&v));
  };
  auto take_q = [&]() {
    float big = 0.0f;
#pragma unroll
    for (int j = 0; j < NS; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 f = as_floats(q[j][i]);
        big = fmaxf(big, fmaxf(fabsf(f.x), fabsf(f.y)));
      }
    }
    big = fmaxf(big, __shfl_xor_sync(~0u, big, 1));
    big = fmaxf(big, __shfl_xor_sync(~0u, big, 2));
    // 2^10 2^e <= big < 2^11 2^e; e within what 2^-e and 2^e are normal numbers for
    const int e = min(max((int)(__float_as_uint(big) >> 23) - 127 - 10, -120), 120);
    const float down = __uint_as_float((uint32_t)(127 - e) << 23);
    float up = unit * __uint_as_float((uint32_t)(127 + e) << 23);
    up = copysignf(fminf(fmaxf(fabsf(up) * 0x1p17f, FLT_MIN), FLT_MAX), up);
    to_log2[0] = __shfl_sync(~0u, up, 8 * t4);
    to_log2[1] = __shfl_sync(~0u, up, 8 * t4 + 4);
#pragma unroll
    for (int n = 0; n < NG; ++n) {
      float sum = 0.0f;
#pragma unroll
      for (int j = n * SG; j < (n + 1) * SG; ++j) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float2 f = as_floats(q[j][i]);
          f.x *= down;
          f.y *= down;
          sum += f.x + f.y;
          const float kind = i & 1 ? 1.0f : 16.0f;
          const __half2 h2 = __floats2half2_rn(f.x * kind, f.y * kind);
          q[j][i] = *reinterpret_cast<const uint32_t *>(&h2);
        }
      }
      sum += __shfl_xor_sync(~0u, sum, 1);
      sum += __shfl_xor_sync(~0u, sum, 2);
      sum *= 0x1p-17f;
      sums[n][0] = __shfl_sync(~0u, sum, 8 * t4);
      sums[n][1] = __shfl_sync(~0u, sum, 8 * t4 + 4);
    }
  };

  // o: codes' part of O^T, elements by heads 2 t4 and 2 t4 + 1; of these heads: low's part of a group over this lane's tokens,
  // the same of l, and the reference
  float o[2 * NS][4], lows[NG][2], l[2], ref[2];
  bool fresh;   // nothing is in them yet
  int scale_v;  // V's numbers are taken times 2^scale_v
  auto clear = [&]() {
    fresh = true;
    scale_v = 0;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      l[c] = 0.0f;
      ref[c] = kNone;
#pragma unroll
      for (int n = 0; n < NG; ++n) lows[n][c] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 2 * NS; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
  };

  ask_q(at.r, at.h * P.members + member);
  take_q();
  clear();
  int64_t item_first = piece.first_place;
  int stage = 0;
  uint32_t parity = 0;
  const int numbers = NS * 512 + g * 8;  // where this lane finds those of token g (of g + 8: 64 bytes behind)
  bool more = true;
#pragma unroll 1
  while (more) {
    const int here = min(at.left, at.rest);  // tiles of the item in this piece
#pragma unroll 1
    for (int tile = here; tile > 0; --tile) {
      bar_wait(smem_at(&small.full[stage]), parity, P.failed, alive);
      const uint32_t rows = small.rows_there[stage][warp];
      char *const base = smem + stage * kStage + warp * kOwn * C;
      if (rows) {
        if (scale_v != 0) {  // where they lie: it is seldom
#pragma unroll 1
          for (int i = lane; i < kOwn * NG * kCell; i += 32) {
            uint32_t *const at = reinterpret_cast<uint32_t *>(base + i / (NG * kCell) * C + NS * 512 + i % (NG * kCell) * 8 + 4);
            *at = scaled(*at, scale_v);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // ahead of the copy that overwrites them
          __syncwarp();
        }
        float s[kOwn][4];    // tokens g, g + 8 of a cell by heads 2 t4, 2 t4 + 1
        uint32_t w[kOwn][2][NG];  // V's numbers
        uint32_t k[kOwn][2][NS];
#pragma unroll
        for (int u = 0; u < kOwn; ++u) {
          load_k<NS>(base + u * C, g, t4, k[u][0]);
          load_k<NS>(base + u * C, g + 8, t4, k[u][1]);
        }
#pragma unroll
        for (int n0 = 0; n0 < NG; n0 += kPair) {
          float acc[kOwn][kPair][4];  // products that need not wait for one another, by turns
#pragma unroll
          for (int j = 0; j < SG; ++j) {
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
#pragma unroll
              for (int n = 0; n < kPair; ++n) {
#pragma unroll
                for (int u = 0; u < kOwn; ++u) {
                  const int slab = (n0 + n) * SG + j;
                  const uint32_t w0 = i ? bytes_exchanged(k[u][0][slab]) : k[u][0][slab], w1 = i ? bytes_exchanged(k[u][1][slab]) : k[u][1][slab];
                  const uint32_t a0 = w0 & kLower, a1 = w1 & kLower, a2 = w0 & kUpper, a3 = w1 & kUpper;
                  if (j == 0 && i == 0) mma_first(acc[u][n], a0, a1, a2, a3, q[slab][i], q[slab][i + 1]);
                  else mma<AMAP_FP16>(acc[u][n], a0, a1, a2, a3, q[slab][i], q[slab][i + 1]);
                }
              }
            }
          }
#pragma unroll
          for (int u = 0; u < kOwn; ++u) {
#pragma unroll
            for (int n = 0; n < kPair; ++n) {
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const uint2 both = *reinterpret_cast<const uint2 *>(base + u * C + numbers + (n0 + n) * 128 + e * 64);
                w[u][e][n0 + n] = both.y;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                  float &x = s[u][2 * e + c];
                  x = n0 + n ? fmaf(low_of(both.x), sums[n0 + n][c], x) : low_of(both.x) * sums[n0 + n][c];
                  x = fmaf(step_of(both.x), acc[u][n][2 * e + c], x);
                }
              }
            }
          }
        }
        if (P.a.softcap > 0) {
          const float in = fminf(1.0f / P.a.softcap, FLT_MAX), out = P.a.softcap * kLog2e;
#pragma unroll
          for (int u = 0; u < kOwn; ++u) {
#pragma unroll
            for (int i = 0; i < 4; ++i) s[u][i] = tanh_of(s[u][i] * to_log2[i & 1] * in) * out / to_log2[i & 1];
          }
        }
        if (rows != ~0u) {  // what lies there of tokens that take no part may be anything: their P is zero, and so are V's numbers
#pragma unroll
          for (int u = 0; u < kOwn; ++u) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              if ((rows >> (u * kCell + e * 8 + g)) & 1) continue;
#pragma unroll
              for (int c = 0; c < 2; ++c) s[u][2 * e + c] = copysignf(INFINITY, -to_log2[c]);
#pragma unroll
              for (int n = 0; n < NG; ++n) w[u][e][n] = 0;
            }
          }
        }
        float step[kOwn][2];  // a token's largest
        uint32_t all;         // the largest of all of these
        auto look_over = [&]() {
          all = 0;
#pragma unroll
          for (int u = 0; u < kOwn; ++u) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              uint32_t most = w[u][e][0];
#pragma unroll
              for (int n = 1; n < NG; ++n) most = larger(most, w[u][e][n]);
              step[u][e] = step_of(most);
              all = larger(all, most);
            }
          }
        };
        look_over();
        float p[kOwn][4], sum[2];
        auto weigh = [&]() {
          bool beyond = fresh || fmaxf(fabsf(low_of(all)), step_of(all)) > kLarge;
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float most = 0.0f;
#pragma unroll
            for (int u = 0; u < kOwn; ++u) {
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                p[u][2 * e + c] = exp2_of(fmaf(s[u][2 * e + c], to_log2[c], -ref[c])) * kUp;  // the exponent is exact where P is large
                most = fmaxf(most, p[u][2 * e + c] * step[u][e]);
              }
            }
            sum[c] = p[0][c] + p[0][c + 2] + (p[1][c] + p[1][c + 2]);
            beyond |= most > kTop || sum[c] > kMost;
          }
          return beyond;
        };
        // seldom after the first tile: the reference, and all that is relative to it, go by this step's weights, too
        auto renew = [&]() {
          int down = 0;  // V's new scale is 2^-down of the one so far
          const float size = __uint_as_float(__reduce_max_sync(~0u, __float_as_uint(fmaxf(fabsf(low_of(all)), step_of(all)))));
          if (size > kLarge) {
            down = min((int)(__float_as_uint(size) >> 23) - 126, 126 + scale_v);
            scale_v -= down;
#pragma unroll
            for (int i = 0; i < 2 * kOwn * NG; ++i) w[i / (2 * NG)][i / NG % 2][i % NG] = scaled(w[i / (2 * NG)][i / NG % 2][i % NG], -down);
            look_over();
          }
          float weight[kOwn][2];  // log2 of the larger of |low| and step
#pragma unroll
          for (int u = 0; u < kOwn; ++u) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float x = fmaxf(kLeast, step[u][e]);
#pragma unroll
              for (int n = 0; n < NG; ++n) x = fmaxf(x, fabsf(low_of(w[u][e][n])));
              weight[u][e] = __log2f(x);
            }
          }
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float top = ref[c] + __log2f(l[c]) - 100.0f;  // l has room
#pragma unroll
            for (int u = 0; u < kOwn; ++u) top = fmaxf(top, fmaxf(fmaf(s[u][c], to_log2[c], weight[u][0]), fmaf(s[u][c + 2], to_log2[c], weight[u][1])));
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 4));
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 8));
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 16));
            top = fmaxf(top, ref[c] - (float)down);  // weights so far are smaller by this, too
            const float keep = exp2_of(ref[c] - top), keep_o = keep * power_of_2(-down);
            ref[c] = top;
            l[c] *= keep;
#pragma unroll
            for (int n = 0; n < NG; ++n) lows[n][c] *= keep_o;
#pragma unroll
            for (int i = 0; i < 2 * NS; ++i) {
              o[i][c] *= keep_o;
              o[i][c + 2] *= keep_o;
            }
          }
          fresh = false;
        };
        if (__any_sync(~0u, weigh())) {
          renew();
          weigh();
        }
        l[0] += sum[0];
        l[1] += sum[1];
#pragma unroll
        for (int n = 0; n < NG; ++n) {
#pragma unroll
          for (int u = 0; u < kOwn; ++u) {
            // the second cell's codes are counted down from 15, low + step c = (low + 15 step) - step (15 - c): what the matrix
            // unit sums then goes up and down by turns, and stays small beside what it cuts off at every step
            uint32_t b[2][2];  // P step_V, [term][eight tokens]
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float own = step_of(w[u][e][n]), by = u ? -own : own, low = u ? fmaf(15.0f, own, low_of(w[u][e][n])) : low_of(w[u][e][n]);
              uint32_t term[2];
              two_terms(p[u][2 * e] * by, p[u][2 * e + 1] * by, term);
              b[0][e] = transposed(term[0]), b[1][e] = transposed(term[1]);
#pragma unroll
              for (int c = 0; c < 2; ++c) lows[n][c] = fmaf(p[u][2 * e + c], low, lows[n][c]);
            }
            uint32_t v[SG][2], a[2 * SG][4];
            load_v<NS, SG>(base + u * C + NS * 256, lane, n * SG, v);
#pragma unroll
            for (int j = 0; j < SG; ++j) {
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const uint32_t x0 = i ? bytes_exchanged(v[j][0]) : v[j][0], x1 = i ? bytes_exchanged(v[j][1]) : v[j][1];
                a[2 * j + i][0] = (u ? ~x0 : x0) & kLower;
                a[2 * j + i][1] = (u ? ~x0 : x0) & kUpper;
                a[2 * j + i][2] = (u ? ~x1 : x1) & kLower;
                a[2 * j + i][3] = (u ? ~x1 : x1) & kUpper;
              }
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) {
#pragma unroll
              for (int i = 0; i < 2 * SG; ++i) {
                mma<AMAP_FP16>(o[2 * n * SG + i], a[i][0], a[i][1], a[i][2], a[i][3], b[t][0], b[t][1]);
              }
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) bar_arrive(smem_at(&small.empty[stage]));
      if (++stage == S) stage = 0, parity ^= 1;
    }
    at.left -= here - 1;
    at.rest -= here - 1;
    more = at.more();
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
    for (int c = 0; c < 2; ++c) {
      float sum = l[c];
      sum += __shfl_xor_sync(~0u, sum, 4);
      sum += __shfl_xor_sync(~0u, sum, 8);
      sum += __shfl_xor_sync(~0u, sum, 16);
      if (ref[c] == kNone) ref[c] = -INFINITY;
      if (g == 0) *reinterpret_cast<float2 *>(joint + (warp * 8 + 2 * t4 + c) * kPitch + D) = make_float2(ref[c], sum / kUp);
    }
    sync_consumers();
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const float *ml = joint + (2 * t4 + c) * kPitch + D;
      const float top = fmaxf(fmaxf(ml[0], ml[8 * kPitch]), fmaxf(ml[16 * kPitch], ml[24 * kPitch]));
      const float f = (top == -INFINITY ? 1.0f : exp2_of(ref[c] - top)) / kUp, unscale = power_of_2(-scale_v);
      float *to = joint + (warp * 8 + 2 * t4 + c) * kPitch;
#pragma unroll
      for (int n = 0; n < NG; ++n) {
        float low = lows[n][c];
        low += __shfl_xor_sync(~0u, low, 4);
        low += __shfl_xor_sync(~0u, low, 8);
        low += __shfl_xor_sync(~0u, low, 16);
        low *= kRoom;
#pragma unroll
        for (int i = 2 * n * SG; i < 2 * (n + 1) * SG; ++i)  // rows g and g + 8 are elements 4g + 2 (i mod 2) and the one behind it
          *reinterpret_cast<float2 *>(to + i / 2 * 32 + 4 * g + 2 * (i & 1)) =
              make_float2(fmaf(o[i][c], 0x1p21f * kRoom, low) * f * unscale, fmaf(o[i][c + 2], 0x1p17f * kRoom, low) * f * unscale);
      }
    }
    sync_consumers();
    sum_warps<D, HB>(P, joint, 0, heads, whole, r, first + in_group, slot, 0.0f);
    sync_consumers();
    if (!whole) hand_in<D, HB>(P, small, joined, piece, item_first, item_last, heads, r, h, first + in_group, 0.0f);  // uniform over the block
    if (more) {
      item_first = u1 - at.rest;
      take_q();
      clear();
    }
  }
  if (!alive) settle(smem_at(&small.full[0]), S, stage, parity, P.failed);
}

template <int NS, int SG>
int run_packed(PackedParams &P, void *stream) {
  constexpr int S = kPackedStages<NS, NS / SG, kPackedResident<NS>>, D = 32 * NS;
  constexpr size_t smem = (size_t)S * kCells * cell_bytes(NS, NS / SG) + sizeof(float) * kWarps * 8 * (D + 4) + sizeof(Small<S, kPackedTile>);
  static std::atomic<int> known[64];
  return launch_split<D, kPackedTile>(attend_packed_kernel<NS, SG>, known, P.p, P, smem, stream);
}

}  // namespace

extern "C" int amap_packed_attend(const amap_attend_args *a, const amap_packed *packed, void *cuda_stream) {
  SERVE_REQUIRE(a && packed, AMAP_EINVAL, "null pointer");
  const amap_packed &c = *packed;
  if (const int rc = check_packed(c)) return rc;
  if (const int rc = check_call(*a, c.heads, c.head_dim, c.page_size)) return rc;
  PackedParams PP = {};
  Params &P = PP.p;
  P.a = *a;
  P.a.maps = nullptr;
  P.a.cache = {};
  P.a.cache.n_pages = c.n_pages, P.a.cache.page_size = c.page_size, P.a.cache.heads = c.heads, P.a.cache.head_dim = c.head_dim;
  P.a.cache.k_scale = 1.0f, P.a.cache.v_scale = 1.0f / kRoom;
  PP.data = static_cast<const char *>(c.data), PP.page = c.page, PP.head = c.head;
  PP.run = 1;
  while (PP.run < kCells && c.page_size / kCell % (2 * PP.run) == 0) PP.run *= 2;
  if (const int rc = place(P, 1)) return rc;
  switch (c.head_dim * 2 + (c.group == 64)) {
    case 128: return run_packed<2, 1>(PP, cuda_stream);
    case 129: return run_packed<2, 2>(PP, cuda_stream);
    case 192: return run_packed<3, 1>(PP, cuda_stream);
    case 256: return run_packed<4, 1>(PP, cuda_stream);
    case 257: return run_packed<4, 2>(PP, cuda_stream);
    case 512: return run_packed<8, 1>(PP, cuda_stream);
    default: return run_packed<8, 2>(PP, cuda_stream);  // check_packed has refused everything else
  }
}
