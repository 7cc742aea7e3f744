// Attention of one new token per request over a paged cache of 4 bits (amap_packed).
//
// Mathematics.  That of serve_attend.cu with K = low_K + step_K c and V = low_V + step_V d by groups of elements:
//   s_t = scale sum_g (step_K <q_g, c_tg> + low_K sum(q_g)),   O = sum_t sum_g (P_t step_V) d_tg + P_t low_V
// so the matrix instructions see the codes themselves.  A code's four bits, masked out where they lie in a 16-bit half, are
// an fp16 number: code x 2^-24 in bits 0 .. 3, code x 2^-20 in bits 4 .. 7 (fp16 counts evenly from 0 to 2^11 of its
// smallest steps), exact in the products.  Eight codes cost a shift and four masks, no conversion; q's elements that meet
// the lower kind are taken 16 times as large, and the two kinds of O's rows are scaled at the end.
//
// Precision.  q is fp16 times a power of two that brings its largest element near 2^11 (2^15 where it meets the lower kind):
// elements down to 2^-27 of it are exact (of fp16's 11 bits, down to 2^-24).  P step_V enters as two fp16 terms of 11 bits, the
// second what the first leaves over.  They are taken relative to a reference R that follows the largest WEIGHT of a token so far,
// P times its largest |low_V| or step_V, rather than the largest P: so the products lie within 2^15 of fp16's range from above
// whatever the values' size is, and a token is cut off only where its weight is 2^-24 of the largest or less (and then by
// 2^-40 of that).  P itself, l and the sums of P low_V are in 32 bits, where R may be far from the largest score.
//
// Bound: HBM; a cell of 16 tokens (2304 bytes of 128 elements in groups of 64) is about 290 instructions of a warp and 32
// products of 16 x 8 x 16, where a multiprocessor has 400 issue slots in the time that the cell takes to come.  The q heads are the M side of the first
// product (so that P comes out as the second one wants it, without a transposition) and the N side of the second.
//
// Split, ring and join are serve_attend.cu's.  A tile is 128 tokens: eight cells, each one bulk copy.
#define AMAP_ATTEND_PARTS_ONLY
#include "serve_attend.cu"
#include "serve_packed.cuh"

namespace {

constexpr int kPackedTile = 128, kCells = kPackedTile / kCell, kOwn = kCells / kWarps;  // cells of a tile; of a warp
static_assert(kOwn == 2, "a warp's cells of a tile");
constexpr float kUp = 9.0f, kTop = 0x1p15f;  // P is 2^kUp times what it stands for; a weight above kTop renews the reference
constexpr float kNone = -3e38f;            // the reference before the first token

template <int NS, int NT> constexpr int kPackedResident = NS * NT >= 8 ? 1 : 2;
// Stages of the ring: what a multiprocessor's shared memory has room for beside the rest of its blocks, up to eight.
constexpr int least(int a, int b) { return a < b ? a : b; }
template <int NS, int NG, int RESIDENT>
constexpr int kPackedStages = least(8, (226 * 1024 / RESIDENT - 3072 - (int)sizeof(float) * kWarps * 8 * (32 * NS + 4)) / (kCells * cell_bytes(NS, NG)));

struct PackedParams {
  Params p;
  const char *data;
  int64_t page, head;
};

__device__ __forceinline__ void bulk_copy(uint32_t dst, const void *src, int bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
template <int WORDS>
__device__ __forceinline__ void load_words(uint32_t at, uint32_t *r) {
  if constexpr (WORDS == 4) asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
  else if constexpr (WORDS == 2) asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(at) : "memory");
  else asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r[0]) : "r"(at) : "memory");
}
// K codes of a lane: slabs side by side, four at a time; three are single words (their rows are 12 bytes)
template <int NS>
__device__ __forceinline__ void load_k(uint32_t at, int token, int t4, uint32_t (&r)[NS]) {
#pragma unroll
  for (int first = 0; first < NS; first += 4) {
    constexpr int kAll = 4;
    const int wide = NS - first < kAll ? NS - first : kAll;
    const uint32_t from = at + first * 256 + (token * 4 + t4) * 4 * wide;
    if (wide == 4) load_words<4>(from, &r[first]);
    else if (wide == 2) load_words<2>(from, &r[first]);
    else
      for (int i = 0; i < wide; ++i) load_words<1>(from + 4 * i, &r[first + i]);
  }
}
template <int NS>
__device__ __forceinline__ void load_v(uint32_t at, int lane, uint32_t (&r)[NS][2]) {
#pragma unroll
  for (int first = 0; first < NS; first += 2) {
    if (NS - first >= 2) {
      load_words<4>(at + first * 256 + lane * 16, &r[first][0]);
    } else {
      load_words<2>(at + first * 256 + lane * 8, &r[first][0]);
    }
  }
}
__device__ __forceinline__ float step_of(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float low_of(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// a and b as fp16 in one word, and what that leaves over, likewise
__device__ __forceinline__ void two_terms(float a, float b, uint32_t (&term)[2]) {
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(term[0]) : "f"(b), "f"(a));
  const float2 h = __half22float2(*reinterpret_cast<const __half2 *>(&term[0]));
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(term[1]) : "f"(b - h.y), "f"(a - h.x));
}

// NS: slabs of 32 elements of a head; SG: slabs of a group; NT: eights of q heads
template <int NS, int SG, int NT>
__global__ void __launch_bounds__(kBlock, (kPackedResident<NS, NT>)) attend_packed_kernel(const __grid_constant__ PackedParams PP) {
  const Params &P = PP.p;
  constexpr int NG = NS / SG, D = 32 * NS, C = cell_bytes(NS, NG), kStage = kCells * C;
  constexpr int S = kPackedStages<NS, NG, kPackedResident<NS, NT>>;
  constexpr int HB = 8 * NT, NM = (NT + 1) / 2;  // sixteens of q heads
  constexpr int kRows = NT == 1 ? 1 : 2;         // rows of a sixteen that a lane has: heads g, and g + 8
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
    // ---- the producer: lane i has cell i of the tile ----
    int entry = -1, offset = 0;
    bool there = false;
    auto look = [&]() {
      const int token = at.t + lane * kCell;
      there = lane < kCells && token < at.n && token > at.low - kCell;
      if (there) {
        const uint32_t page = P.div_mul ? __umulhi((uint32_t)token, P.div_mul) >> P.div_shift : (uint32_t)token >> P.div_shift;
        offset = token - (int)page * cache.page_size;
        entry = P.a.block_table[(int64_t)at.r * P.a.table_stride + page];
      }
    };
    int stage = 0;
    uint32_t parity = 1;  // the first round of waits finds every stage empty
    look();
    for (bool more = true; more;) {
      const int head = (at.h * P.members + member) / P.blocks_per_head;
      const bool live = there && (uint32_t)entry < (uint32_t)cache.n_pages;
      const uint32_t cells = __ballot_sync(~0u, live);
      const char *from = PP.data + (live ? (int64_t)entry * PP.page + (int64_t)head * PP.head + (int64_t)(offset / kCell) * C : 0);
      more = at.more();
      if (more) {
        at.advance(P);
        look();
      }
      bar_wait(smem_at(&small.empty[stage]), parity, P.failed, alive);
      if (!__all_sync(~0u, alive)) break;
      const uint32_t bar = smem_at(&small.full[stage]);
      if (lane == 0) {
        small.rows_there[stage][0] = cells;
        bar_arrive_bytes(bar, __popc(cells) * C);
      }
      __syncwarp();
      if (live) bulk_copy(smem_at(smem + stage * kStage) + lane * C, from, C, bar);
      if (++stage == S) stage = 0, parity ^= 1;
    }
    if (!__all_sync(~0u, alive)) {
      settle(smem_at(&small.full[0]), S, stage, parity ^ 1, P.failed);
      return;
    }
    if (piece.aside) join_aside<D, HB>(P, small, piece, kUp);
    return;
  }

  // ---- q of an item, as the A operand: a lane has heads g and g + 8 of a sixteen, of each slab the elements 8 t4 .. +7 ----
  uint32_t q[NM][kRows][NS][4];
  float to_log2[NM][kRows], sums[NM][kRows][NG];  // sums of q over a group, as the products count it
  const float unit = (P.a.softcap > 0 ? 1.0f : kLog2e) * P.a.scale;
  auto ask_q = [&](int r, int h) {
    const int first = h / P.blocks_per_head * P.group, in_group = h % P.blocks_per_head * HB;
    const uint16_t *row = static_cast<const uint16_t *>(P.a.q) + (int64_t)r * P.a.q_row;
#pragma unroll
    for (int m = 0; m < NM; ++m) {
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        const int head = in_group + m * 16 + k * 8 + g;
        const bool there = head < P.group;
        const uint16_t *x = row + (int64_t)(first + (there ? head : 0)) * P.a.q_head;
#pragma unroll
        for (int j = 0; j < NS; ++j) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int d = j * 32 + t4 * 8 + i * 2;
            uint32_t v = 0;
            if (there) v = P.q_pairs ? *reinterpret_cast<const uint32_t *>(x + d) : x[d] | (uint32_t)x[d + 1] << 16;
            q[m][k][j][i] = v;
          }
        }
      }
    }
  };
  auto as_floats = [&](uint32_t v) {
    return P.a.dtype == AMAP_BF16 ? make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u)) : __half22float2(*reinterpret_cast<const __half2 *>(&v));
  };
  auto take_q = [&]() {
#pragma unroll
    for (int m = 0; m < NM; ++m) {
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        float big = 0.0f;
#pragma unroll
        for (int j = 0; j < NS; ++j) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 f = as_floats(q[m][k][j][i]);
            big = fmaxf(big, fmaxf(fabsf(f.x), fabsf(f.y)));
          }
        }
        big = fmaxf(big, __shfl_xor_sync(~0u, big, 1));
        big = fmaxf(big, __shfl_xor_sync(~0u, big, 2));
        // 2^10 2^e <= big < 2^11 2^e; e within what 2^-e and 2^e are normal numbers for
        const int e = min(max((int)(__float_as_uint(big) >> 23) - 127 - 10, -120), 120);
        const float down = __uint_as_float((uint32_t)(127 - e) << 23);
        to_log2[m][k] = unit * __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
        for (int n = 0; n < NG; ++n) {
          float sum = 0.0f;
#pragma unroll
          for (int j = n * SG; j < (n + 1) * SG; ++j) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float2 f = as_floats(q[m][k][j][i]);
              f.x *= down;
              f.y *= down;
              sum += f.x + f.y;
              const float kind = i & 1 ? 1.0f : 16.0f;
              const __half2 h2 = __floats2half2_rn(f.x * kind, f.y * kind);
              q[m][k][j][i] = *reinterpret_cast<const uint32_t *>(&h2);
            }
          }
          sum += __shfl_xor_sync(~0u, sum, 1);
          sum += __shfl_xor_sync(~0u, sum, 2);
          sums[m][k][n] = sum * 0x1p-20f;
        }
      }
    }
  };

  // o: codes' part of O^T, elements by heads 2 t4 and 2 t4 + 1; of head g (nt eights on): low's part of a group over this
  // lane's tokens, the same of l, and the reference
  float o[NT][2 * NS][4], lows[NT][NG], l[NT], ref[NT];
  auto clear = [&]() {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      l[nt] = 0.0f;
      ref[nt] = kNone;
#pragma unroll
      for (int n = 0; n < NG; ++n) lows[nt][n] = 0.0f;
#pragma unroll
      for (int i = 0; i < 2 * NS; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.0f;
    }
  };

  ask_q(at.r, at.h * P.members + member);
  take_q();
  clear();
  int64_t item_first = piece.first_place;
  int stage = 0;
  uint32_t parity = 0;
  bool more = true;
#pragma unroll 1
  while (more) {
    // this warp's tokens that take part
    const int row0 = at.t + warp * 32, upper = min(max(at.n - row0, 0), 32), lower = min(max(at.low - row0, 0), 32);
    uint32_t rows = (upper ? ~0u >> (32 - upper) : 0) & ~(lower ? ~0u >> (32 - lower) : 0);
    bar_wait(smem_at(&small.full[stage]), parity, P.failed, alive);
    const uint32_t cells = small.rows_there[stage][0] >> (warp * kOwn);
    rows &= (cells & 1 ? 0xFFFFu : 0u) | (cells & 2 ? 0xFFFF0000u : 0u);
    const uint32_t base = smem_at(smem + stage * kStage) + warp * kOwn * C;
    if (rows) {
      const bool all = rows == ~0u;
      float s[kOwn][NT][4];   // head g (+ 8 nt); tokens 2 t4, 2 t4 + 1, + 8, + 9 of a cell
      float most[kOwn][4];    // of these tokens, the largest |low_V| or step_V
#pragma unroll
      for (int u = 0; u < kOwn; ++u) {
        const uint32_t cell = base + u * C;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          most[u][i] = 0x1p-60f;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) s[u][nt][i] = 0.0f;
        }
        uint32_t k[2][NS];
        load_k<NS>(cell, g, t4, k[0]);
        load_k<NS>(cell, g + 8, t4, k[1]);
#pragma unroll
        for (int n = 0; n < NG; ++n) {
          float acc[NM][2][4];
#pragma unroll
          for (int m = 0; m < NM; ++m) {
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[m][0][c] = acc[m][1][c] = 0.0f;
          }
#pragma unroll
          for (int j = n * SG; j < (n + 1) * SG; ++j) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {  // eight tokens
              const uint32_t w = k[e][j], w8 = w >> 8;
#pragma unroll
              for (int m = 0; m < NM; ++m) {
                mma<AMAP_FP16>(acc[m][e], q[m][0][j][0], kRows == 2 ? q[m][kRows - 1][j][0] : 0u, q[m][0][j][1], kRows == 2 ? q[m][kRows - 1][j][1] : 0u,
                               w & 0x000F000Fu, w & 0x00F000F0u);
                mma<AMAP_FP16>(acc[m][e], q[m][0][j][2], kRows == 2 ? q[m][kRows - 1][j][2] : 0u, q[m][0][j][3], kRows == 2 ? q[m][kRows - 1][j][3] : 0u,
                               w8 & 0x000F000Fu, w8 & 0x00F000F0u);
              }
            }
          }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            uint32_t w[4];
            load_words<4>(cell + NS * 512 + n * 128 + e * 64 + t4 * 16, w);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const float step = step_of(w[c]), low = low_of(w[c]);
              most[u][2 * e + c] = fmaxf(most[u][2 * e + c], fmaxf(step_of(w[2 + c]), fabsf(low_of(w[2 + c]))));
#pragma unroll
              for (int m = 0; m < NM; ++m) {
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                  if (2 * m + r >= NT) continue;
                  float &x = s[u][2 * m + r][2 * e + c];
                  x = fmaf(step, acc[m][e][2 * r + c], fmaf(low, sums[m][r][n], x));
                }
              }
            }
          }
        }
      }
#pragma unroll
      for (int u = 0; u < kOwn; ++u) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int i = 0; i < 4; ++i) s[u][nt][i] = s[u][nt][i] * 0x1p20f * to_log2[nt / 2][kRows == 2 ? nt & 1 : 0];
        }
      }
      if (P.a.softcap > 0) {
        const float in = fminf(1.0f / P.a.softcap, FLT_MAX), out = P.a.softcap * kLog2e;
#pragma unroll
        for (int u = 0; u < kOwn; ++u) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int i = 0; i < 4; ++i) s[u][nt][i] = tanh_of(s[u][nt][i] * in) * out;
          }
        }
      }
      auto live = [&](int u, int i) { return (rows >> (u * kCell + (i >> 1) * 8 + 2 * t4 + (i & 1))) & 1; };
      if (!all) {  // what lies there of tokens that take no part may be anything
#pragma unroll
        for (int u = 0; u < kOwn; ++u) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (live(u, i)) continue;
            most[u][i] = 0x1p-60f;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[u][nt][i] = -INFINITY;
          }
        }
      }
      float p[kOwn][NT][4];
      auto weigh = [&]() {
        bool higher = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float from = ref[nt] - kUp;
#pragma unroll
          for (int u = 0; u < kOwn; ++u) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              p[u][nt][i] = exp2_of(s[u][nt][i] - from);
              higher |= p[u][nt][i] * most[u][i] > kTop;
            }
          }
        }
        return __any_sync(~0u, higher);
      };
      if (weigh()) {  // seldom after the first tile
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float top = kNone;
#pragma unroll
          for (int u = 0; u < kOwn; ++u) {
#pragma unroll
            for (int i = 0; i < 4; ++i) top = fmaxf(top, s[u][nt][i] + __log2f(most[u][i]));
          }
          top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
          top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
          top = fmaxf(top, ref[nt]);
          const float keep = exp2_of(ref[nt] - top);
          ref[nt] = top;
          l[nt] *= keep;
#pragma unroll
          for (int n = 0; n < NG; ++n) lows[nt][n] *= keep;
          const float keep0 = __shfl_sync(~0u, keep, 8 * t4), keep1 = __shfl_sync(~0u, keep, 8 * t4 + 4);
#pragma unroll
          for (int i = 0; i < 2 * NS; ++i) {
            o[nt][i][0] *= keep0;
            o[nt][i][1] *= keep1;
            o[nt][i][2] *= keep0;
            o[nt][i][3] *= keep1;
          }
        }
        weigh();
      }
#pragma unroll
      for (int u = 0; u < kOwn; ++u) {
        const uint32_t cell = base + u * C;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) l[nt] += (p[u][nt][0] + p[u][nt][1]) + (p[u][nt][2] + p[u][nt][3]);
        uint32_t v[NS][2];
        load_v<NS>(cell + NS * 256, lane, v);
#pragma unroll
        for (int n = 0; n < NG; ++n) {
          uint32_t w[2][2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            load_words<2>(cell + NS * 512 + n * 128 + e * 64 + t4 * 16 + 8, w[e]);
            if (!all) {
#pragma unroll
              for (int c = 0; c < 2; ++c) w[e][c] = live(u, 2 * e + c) ? w[e][c] : 0;
            }
          }
          uint32_t b[NT][2][2];  // [eight tokens][term]
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float p0 = p[u][nt][2 * e], p1 = p[u][nt][2 * e + 1];
              lows[nt][n] = fmaf(p0, low_of(w[e][0]), fmaf(p1, low_of(w[e][1]), lows[nt][n]));
              two_terms(p0 * step_of(w[e][0]), p1 * step_of(w[e][1]), b[nt][e]);
            }
          }
#pragma unroll
          for (int j = n * SG; j < (n + 1) * SG; ++j) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const uint32_t w0 = v[j][0] >> (8 * i), w1 = v[j][1] >> (8 * i);
              const uint32_t a0 = w0 & 0x000F000Fu, a1 = w0 & 0x00F000F0u, a2 = w1 & 0x000F000Fu, a3 = w1 & 0x00F000F0u;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                mma<AMAP_FP16>(o[nt][2 * j + i], a0, a1, a2, a3, b[nt][0][0], b[nt][1][0]);
                mma<AMAP_FP16>(o[nt][2 * j + i], a0, a1, a2, a3, b[nt][0][1], b[nt][1][1]);
              }
            }
          }
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
      float sum = l[nt];
      sum += __shfl_xor_sync(~0u, sum, 1);
      sum += __shfl_xor_sync(~0u, sum, 2);
      const float own = ref[nt] == kNone ? -INFINITY : ref[nt];
      if (t4 == 0) *reinterpret_cast<float2 *>(joint + (warp * 8 + g) * kPitch + D) = make_float2(own, sum);
      sync_consumers();
      const float *ml = joint + g * kPitch + D;
      const float top = fmaxf(fmaxf(ml[0], ml[8 * kPitch]), fmaxf(ml[16 * kPitch], ml[24 * kPitch]));
      const float f = top == -INFINITY ? 1.0f : exp2_of(own - top);
      const float f0 = __shfl_sync(~0u, f, 8 * t4), f1 = __shfl_sync(~0u, f, 8 * t4 + 4);
      float *to = joint + (warp * 8 + 2 * t4) * kPitch;
#pragma unroll
      for (int n = 0; n < NG; ++n) {
        float low = lows[nt][n];
        low += __shfl_xor_sync(~0u, low, 1);
        low += __shfl_xor_sync(~0u, low, 2);
        const float low0 = __shfl_sync(~0u, low, 8 * t4), low1 = __shfl_sync(~0u, low, 8 * t4 + 4);
#pragma unroll
        for (int i = 2 * n * SG; i < 2 * (n + 1) * SG; ++i) {  // rows g and g + 8 are elements 4g + 2 (i mod 2) and the one behind it
          const int d = i / 2 * 32 + 4 * g + 2 * (i & 1);
          *reinterpret_cast<float2 *>(to + d) = make_float2(fmaf(o[nt][i][0], 0x1p24f, low0) * f0, fmaf(o[nt][i][2], 0x1p20f, low0) * f0);
          *reinterpret_cast<float2 *>(to + kPitch + d) = make_float2(fmaf(o[nt][i][1], 0x1p24f, low1) * f1, fmaf(o[nt][i][3], 0x1p20f, low1) * f1);
        }
      }
      sync_consumers();
      sum_warps<D, HB>(P, joint, nt, heads, whole, r, first + in_group, slot, kUp);
      sync_consumers();
    }
    if (!whole) hand_in<D, HB>(P, small, joined, piece, item_first, item_last, heads, r, h, first + in_group, kUp);  // uniform over the block
    if (more) {
      item_first = u1 - at.rest;
      take_q();
      clear();
    }
  }
  if (!alive) settle(smem_at(&small.full[0]), S, stage, parity, P.failed);
}

template <int NS, int SG, int NT>
int run_packed(PackedParams &P, void *stream) {
  constexpr int S = kPackedStages<NS, NS / SG, kPackedResident<NS, NT>>, D = 32 * NS;
  constexpr size_t smem = (size_t)S * kCells * cell_bytes(NS, NS / SG) + sizeof(float) * kWarps * 8 * (D + 4) + sizeof(Small<S, kPackedTile>);
  static std::atomic<int> known[64];
  return launch_split<D, kPackedTile>(attend_packed_kernel<NS, SG, NT>, known, P.p, P, smem, stream);
}

template <int NS, int SG>
int run_packed_heads(PackedParams &P, int nt, void *stream) {
  switch (nt) {
    case 1: return run_packed<NS, SG, 1>(P, stream);
    case 2: return run_packed<NS, SG, 2>(P, stream);
    default:
      if constexpr (NS < 8) return run_packed<NS, SG, 4>(P, stream);
      else return run_packed<NS, SG, 2>(P, stream);
  }
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
  P.a.cache.k_scale = P.a.cache.v_scale = 1.0f;
  PP.data = static_cast<const char *>(c.data), PP.page = c.page, PP.head = c.head;
  const int nt = eights(a->q_heads / c.heads, c.head_dim <= 128 ? 128 : 256);
  if (const int rc = place(P, nt)) return rc;
  switch (c.head_dim * 2 + (c.group == 64)) {
    case 128: return run_packed_heads<2, 1>(PP, nt, cuda_stream);
    case 129: return run_packed_heads<2, 2>(PP, nt, cuda_stream);
    case 192: return run_packed_heads<3, 1>(PP, nt, cuda_stream);
    case 256: return run_packed_heads<4, 1>(PP, nt, cuda_stream);
    case 257: return run_packed_heads<4, 2>(PP, nt, cuda_stream);
    case 512: return run_packed_heads<8, 1>(PP, nt, cuda_stream);
    default: return run_packed_heads<8, 2>(PP, nt, cuda_stream);  // check_packed has refused everything else
  }
}
