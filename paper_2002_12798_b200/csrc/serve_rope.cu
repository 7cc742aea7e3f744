// Rotary positions with several axes, and their fusion with the write into a paged cache.
//
// Pair i of a token at position p (along the pair's axis) turns by p * f_i radians.  The plan keeps f_i / 2pi as a
// 64-bit fraction of a turn; p times that fraction wraps modulo a full turn exactly, so the angle's error is
// p * 2^-65 turns whatever p is, and `turn` takes it from there in 32 bits.
//
// Bound: memory, every element is read and written once.  A block takes a few tokens of one part (q, k or v): its
// threads issue their loads, compute the tokens' cos and sin once for all heads while those are under way, and turn
// and store.  An item is VEC pairs (two 16-byte accesses each way where alignment allows), two per thread: few, so that
// blocks are short and many overlap (8192 tokens of 40 heads of 128 bf16 elements: 32.2 us = 5.2 TB/s; four items 33.3 us,
// one item at more blocks 36).  Beside a copy of the same bytes (26 us) it pays for the arithmetic and for the angles,
// which stand between a block's loads and its stores.  16 tokens into the cache: 1.9 us, latency alone.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "serve_alias.hpp"
#include "serve_common.cuh"

using namespace amap_serve;

struct amap_rope_t {
  int32_t head_dim, half, n_axes, pairs;
  float scale;
  uint64_t phase[AMAP_ROPE_MAX_DIM / 2];
  uint8_t axis[AMAP_ROPE_MAX_DIM / 2];
};

namespace {

constexpr int kThreads = 256;
constexpr int kMaxHalf = AMAP_ROPE_MAX_DIM / 2;
constexpr int kUnroll = 2;      // items per thread whose loads are issued together
constexpr int kBlocks = 4;      // resident per multiprocessor
constexpr int kMaxTokens = 16;  // per block

// where a part's rows go
enum { kRows = 0, kCacheTurned = 1, kCacheCopied = 2 };

// n / d for n below 2^31: the high word of a product with ceil(2^(32+s) / d), s = floor(log2 d)
struct Div {
  uint32_t mul, shift, d;
};
Div div_by(uint32_t d) {
  Div f = {0, 0, d};
  while ((2ull << f.shift) <= d) ++f.shift;
  if (d != 1u << f.shift) f.mul = (uint32_t)((((uint64_t)1 << (32 + f.shift)) + d - 1) / d);
  return f;
}
__device__ __forceinline__ uint32_t quotient(uint32_t n, const Div &f) { return f.mul ? __umulhi(n, f.mul) >> f.shift : n >> f.shift; }

// v / d in 32 bits, correctly rounded where it is a normal number that 8 bits can hold, by Markstein's correction (IBM
// Journal of Research and Development 34, 1990): with r the rounded reciprocal of d, q = v r is within one unit of the
// quotient and q + (v - q d) r is the quotient rounded.  d is taken times a power of 2 that brings it near 1, so that any
// positive number will do.  (A division in the kernel costs the 16-bit caches, which have none, 8 % for its registers.)
struct Divisor {
  float pre, d, r;
};
Divisor divide_by(float d) {
  int e = 0;
  frexpf(d, &e);  // 2^(e-1) <= d < 2^e
  e = std::max(-126, std::min(126, e - 1));
  Divisor f;
  f.pre = ldexpf(1.0f, -e);
  f.d = d * f.pre;  // exact
  f.r = 1.0f / f.d;
  return f;
}
__device__ __forceinline__ float quotient(float v, const Divisor &f) {
  const float x = v * f.pre, q = x * f.r;
  // outside: zeros of either sign, and what is clamped, infinities and NaN among them
  return fabsf(q) > 0x1p-20f && fabsf(q) < 1024.0f ? fmaf(fmaf(-q, f.d, x), f.r, q) : q;
}

struct Part {
  const char *x;
  char *y;
  int64_t x_row, x_head, y_row, y_head;  // elements; cache: y_row is the page stride
  int64_t y_token;
  int32_t heads;
  int32_t kind;
  Divisor scale;         // cache: what an element of 8 bits is to be multiplied by
  int32_t tokens;        // per block
  uint32_t first_block;  // blocks of the parts before this one
  Div by_heads;
};

struct Params {
  uint64_t phase[kMaxHalf];
  uint8_t axis[kMaxHalf];
  Part part[4];
  const void *positions;
  const int32_t *slots;
  int64_t position_axis, position_row;
  int64_t rows;
  int32_t n_parts;
  int32_t half, head_dim;
  Div by_items, by_half, by_page;  // items of a head: half/VEC chunks of pairs, then the chunks behind rotary_dim two at a time
  int32_t wide_positions, n_slots, e4m3;
  float scale, sign;
};

template <int DT, int VEC>
__device__ __forceinline__ void unpack(const typename Raw<VEC * sizeof(typename Elem<DT>::T)>::T &raw, float (&v)[VEC]) {
  using E = Elem<DT>;
  union {
    typename Raw<VEC * sizeof(typename E::T)>::T raw;
    typename E::T e[VEC];
  } u;
  u.raw = raw;
#pragma unroll
  for (int j = 0; j < VEC; ++j) v[j] = E::to(u.e[j]);
}

// two values as two elements in one word: the packed conversion runs on the arithmetic pipes, the single one on the
// special-function unit at a quarter of their rate
template <int DT>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  uint32_t r;
  if constexpr (DT == AMAP_BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
  return r;
}

template <int DT, int VEC>
__device__ __forceinline__ void store(char *p, int64_t at, const float (&v)[VEC], bool e4m3, const Divisor &scale) {
  using E = Elem<DT>;
  constexpr int ES = sizeof(typename E::T);
  if (e4m3) {
    union {
      typename Raw<VEC>::T raw;
      uint16_t two[(VEC + 1) / 2];
    } u;
    if constexpr (VEC == 1) {
      u.raw = to_e4m3(quotient(v[0], scale));
    } else {
#pragma unroll
      for (int j = 0; j < VEC; j += 2) u.two[j / 2] = __nv_cvt_float2_to_fp8x2(make_float2(quotient(v[j], scale), quotient(v[j + 1], scale)), __NV_SATFINITE, __NV_E4M3);
    }
    *reinterpret_cast<typename Raw<VEC>::T *>(p + at) = u.raw;
  } else {
    union {
      typename Raw<VEC * ES>::T raw;
      typename E::T e[VEC];
      uint32_t two[(VEC + 1) / 2];
    } u;
    if constexpr (ES == 4 || VEC == 1) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) u.e[j] = E::from(v[j]);
    } else {
#pragma unroll
      for (int j = 0; j < VEC; j += 2) u.two[j / 2] = pack2<DT>(v[j], v[j + 1]);
    }
    *reinterpret_cast<typename Raw<VEC * ES>::T *>(p + at * ES) = u.raw;
  }
}

// sin and cos of a fraction of a turn in units of 2^-64.  For 16-bit elements the nearest half turn is left to sincospif: its
// argument, a float near half a turn at most, is within 2^-24 pi.  fp32 elements would show that; the nearest quarter turn
// is taken off in integers for them, which leaves an argument eight times smaller and as much closer.
template <int DT>
__device__ __forceinline__ void turn(uint64_t turns, float *s, float *c) {
  if constexpr (DT != AMAP_FP32) {
    sincospif((float)(int32_t)(turns >> 32) * 0x1p-31f, s, c);
  } else {
    const uint32_t quarter = ((uint32_t)(turns >> 32) + 0x20000000u) >> 30;
    const int64_t rest = (int64_t)(turns - ((uint64_t)quarter << 62));  // [-1/8, 1/8) turn
    float x, y;
    sincospif((float)(int32_t)(rest >> 30) * 0x1p-33f, &x, &y);
    const float a = quarter & 1 ? y : x, b = quarter & 1 ? x : y;
    *s = quarter & 2 ? -a : a;
    *c = (quarter + 1) & 2 ? -b : b;
  }
}

// Where pair i's cos (and sin) of a token is kept: the VEC values of a chunk in fours, a four of all chunks side by side,
// so that neighbouring lanes read neighbouring 16 bytes.
template <int VEC>
__device__ __forceinline__ int place(int i, int half) {
  if constexpr (VEC < 4) return i;
  else return (i % VEC) / 4 * (half / VEC * 4) + i / VEC * 4 + i % 4;
}

template <int VEC>
__device__ __forceinline__ void fetch(const float *row, int c, int half, float (&v)[VEC]) {
#pragma unroll
  for (int j = 0; j < VEC; j += VEC < 4 ? 1 : 4) {
    if constexpr (VEC < 4) {
      v[j] = row[c * VEC + j];
    } else {
      const float4 f = *reinterpret_cast<const float4 *>(row + j / 4 * (half / VEC * 4) + c * 4);
      v[j] = f.x, v[j + 1] = f.y, v[j + 2] = f.z, v[j + 3] = f.w;
    }
  }
}

template <int DT, int VEC, int PAIRS>
__global__ void __launch_bounds__(kThreads, kBlocks) rope_kernel(const __grid_constant__ Params P) {
  __shared__ __align__(16) float turn_cos[kMaxTokens * kMaxHalf], turn_sin[kMaxTokens * kMaxHalf];
  constexpr int ES = sizeof(typename Elem<DT>::T);
  using Chunk = typename Raw<VEC * ES>::T;
  int k = 0;
  while (k + 1 < P.n_parts && blockIdx.x >= P.part[k + 1].first_block) ++k;
  const Part part = P.part[k];  // a copy: the fields stay in registers
  const int half = P.half, chunks = half / VEC, items = P.by_items.d;
  const int64_t row0 = (int64_t)(blockIdx.x - part.first_block) * part.tokens;
  const int tokens = (int)min((int64_t)part.tokens, P.rows - row0), n = tokens * part.heads * items;
  const bool turns = part.kind != kCacheCopied;
  const char *const x0 = part.x + row0 * part.x_row * ES;
  char *const y0 = part.kind == kRows ? part.y + row0 * part.y_row * ES : part.y;
  pdl_begin();

  Chunk a[kUnroll], b[kUnroll];
  int64_t to[kUnroll];  // of the head's first element
  int chunk[kUnroll], token[kUnroll];
  bool live[kUnroll];
  auto load = [&](int base) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int item = base + u * kThreads;
      live[u] = item < n;
      if (!live[u]) continue;
      const uint32_t row = quotient(item, P.by_items);
      chunk[u] = item - row * items;
      token[u] = quotient(row, part.by_heads);
      const uint32_t head = row - token[u] * part.heads;
      if (part.kind == kRows) {
        to[u] = (uint32_t)token[u] * part.y_row + head * part.y_head;
      } else {
        const int32_t slot = P.slots[row0 + token[u]];
        live[u] = slot >= 0 && slot < P.n_slots;
        if (!live[u]) continue;
        const uint32_t page = quotient(slot, P.by_page);
        to[u] = page * part.y_row + (uint32_t)(slot - page * P.by_page.d) * part.y_token + head * part.y_head;
      }
      const bool tail = chunk[u] >= chunks;
      const int first = tail ? 2 * half + 2 * (chunk[u] - chunks) * VEC : PAIRS == AMAP_PAIRS_HALF ? chunk[u] * VEC : 2 * chunk[u] * VEC;
      const int gap = tail || PAIRS != AMAP_PAIRS_HALF ? VEC : half;
      const char *p = x0 + ((uint32_t)token[u] * part.x_row + head * part.x_head + first) * ES;
      a[u] = *reinterpret_cast<const Chunk *>(p);
      if (first + gap < P.head_dim) b[u] = *reinterpret_cast<const Chunk *>(p + gap * ES);
    }
  };
  auto finish = [&]() {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (!live[u]) continue;
      float v[VEC], w[VEC];
      unpack<DT, VEC>(a[u], v);
      unpack<DT, VEC>(b[u], w);
      const bool tail = chunk[u] >= chunks;
      const int first = tail ? 2 * half + 2 * (chunk[u] - chunks) * VEC : PAIRS == AMAP_PAIRS_HALF ? chunk[u] * VEC : 2 * chunk[u] * VEC;
      const int gap = tail || PAIRS != AMAP_PAIRS_HALF ? VEC : half;
      if (turns && !tail) {
        float c[VEC], s[VEC];
        fetch<VEC>(turn_cos + token[u] * half, chunk[u], half, c);
        fetch<VEC>(turn_sin + token[u] * half, chunk[u], half, s);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          float &e0 = PAIRS == AMAP_PAIRS_HALF ? v[j] : 2 * j < VEC ? v[(2 * j) % VEC] : w[(2 * j) % VEC];
          float &e1 = PAIRS == AMAP_PAIRS_HALF ? w[j] : 2 * j + 1 < VEC ? v[(2 * j + 1) % VEC] : w[(2 * j + 1) % VEC];
          const float p = e0, q = e1;
          e0 = p * c[j] - q * s[j];
          e1 = q * c[j] + p * s[j];
        }
      }
      const bool e4m3 = part.kind != kRows && P.e4m3;
      store<DT, VEC>(y0, to[u] + first, v, e4m3, part.scale);
      if (first + gap < P.head_dim) store<DT, VEC>(y0, to[u] + first + gap, w, e4m3, part.scale);
    }
  };

  load(threadIdx.x);
  if (turns) {
    // the tables lie in the kernel's parameters; read as constants, a warp's 32 addresses would be served one by one,
    // as memory they are two lines
    const uint64_t *phases = P.phase;
    const uint8_t *axes = P.axis;
    asm volatile("" : "+l"(phases), "+l"(axes));
    for (int i = threadIdx.x; i < tokens * half; i += kThreads) {
      const int at = quotient(i, P.by_half), pair = i - at * half;
      const int64_t from = axes[pair] * P.position_axis + (row0 + at) * P.position_row;
      const int64_t pos = P.wide_positions ? static_cast<const int64_t *>(P.positions)[from] : static_cast<const int32_t *>(P.positions)[from];
      const uint64_t turns = (uint64_t)pos * phases[pair];  // in units of 2^-64 turns
      float s, c;
      turn<DT>(turns, &s, &c);
      turn_cos[at * half + place<VEC>(pair, half)] = c * P.scale;
      turn_sin[at * half + place<VEC>(pair, half)] = s * P.scale * P.sign;
    }
    __syncthreads();
  }
  finish();
  for (int base = threadIdx.x + kUnroll * kThreads; base < n; base += kUnroll * kThreads) {  // many heads a token
    load(base);
    finish();
  }
}

template <int DT, int VEC>
int run(const amap_rope_t &plan, Params &P, void *stream) {
  const int items = P.half / VEC + ((P.head_dim - 2 * P.half) / VEC + 1) / 2;
  P.by_items = div_by(items);
  P.by_half = div_by(std::max(P.half, 1));
  // tokens per block: two items a thread, but no fewer than two blocks a multiprocessor where there is that much work
  const int sms = device_sms();
  int64_t all = 0;
  for (int k = 0; k < P.n_parts; ++k) all += P.rows * P.part[k].heads * items;
  const int64_t per_block = std::min<int64_t>(kUnroll * kThreads, std::max<int64_t>(all / (2 * sms), 1));
  int64_t blocks = 0;
  for (int k = 0; k < P.n_parts; ++k) {
    Part &part = P.part[k];
    part.by_heads = div_by(part.heads);
    part.tokens = (int32_t)std::max<int64_t>(1, std::min<int64_t>(kMaxTokens, per_block / ((int64_t)part.heads * items)));
    part.first_block = (uint32_t)blocks;
    blocks += (P.rows + part.tokens - 1) / part.tokens;
  }
  SERVE_REQUIRE(blocks <= 0x7FFFFFFF, AMAP_EOVERFLOW, "too many rows");
  const dim3 grid((unsigned)blocks);
  return plan.pairs == AMAP_PAIRS_HALF ? launch(rope_kernel<DT, VEC, AMAP_PAIRS_HALF>, grid, kThreads, 0, stream, P)
                                       : launch(rope_kernel<DT, VEC, AMAP_PAIRS_ADJACENT>, grid, kThreads, 0, stream, P);
}

// the widest access, in elements, that every chunk of every part allows
int widest(const Params &P, int es, int heads_es) {
  int vec = 16 / es;
  auto fits = [&](int v) {
    if (P.half % v || (P.head_dim - 2 * P.half) % v) return false;
    for (int k = 0; k < P.n_parts; ++k) {
      const Part &p = P.part[k];
      const int ys = p.kind == kRows ? es : heads_es;
      if (!aligned(p.x, (int64_t)v * es) || !aligned(p.y, (int64_t)v * ys)) return false;
      for (const int64_t s : {p.x_row, p.x_head, p.y_row, p.y_head, p.y_token})
        if (s % v) return false;
    }
    return true;
  };
  while (vec > 1 && !fits(vec)) vec >>= 1;
  return vec;
}

int run_typed(const amap_rope_t &plan, Params &P, int dtype, int cache_es, void *stream) {
  memcpy(P.phase, plan.phase, sizeof P.phase);
  memcpy(P.axis, plan.axis, sizeof P.axis);
  P.half = plan.half;
  P.head_dim = plan.head_dim;
  P.scale = plan.scale;
  const int vec = widest(P, dtype_bytes(dtype), cache_es);
  if (dtype == AMAP_FP32) {
    switch (vec) {
      case 4: return run<AMAP_FP32, 4>(plan, P, stream);
      case 2: return run<AMAP_FP32, 2>(plan, P, stream);
      default: return run<AMAP_FP32, 1>(plan, P, stream);
    }
  }
  if (dtype == AMAP_BF16) {
    switch (vec) {
      case 8: return run<AMAP_BF16, 8>(plan, P, stream);
      case 4: return run<AMAP_BF16, 4>(plan, P, stream);
      case 2: return run<AMAP_BF16, 2>(plan, P, stream);
      default: return run<AMAP_BF16, 1>(plan, P, stream);
    }
  }
  switch (vec) {
    case 8: return run<AMAP_FP16, 8>(plan, P, stream);
    case 4: return run<AMAP_FP16, 4>(plan, P, stream);
    case 2: return run<AMAP_FP16, 2>(plan, P, stream);
    default: return run<AMAP_FP16, 1>(plan, P, stream);
  }
}

int check_rows(int64_t rows, const void *positions, int32_t bits) {
  SERVE_REQUIRE(rows >= 0 && rows <= 0x7FFFFFFF, AMAP_EINVAL, "rows: 0 .. 2^31-1");
  SERVE_REQUIRE(bits == 32 || bits == 64, AMAP_EINVAL, "positions: 32 or 64 bits");
  SERVE_REQUIRE(rows == 0 || positions, AMAP_EINVAL, "positions: null pointer");
  SERVE_REQUIRE(aligned(positions, bits / 8), AMAP_EALIGN, "positions: misaligned");
  return AMAP_OK;
}

Span rows_span(int64_t rows, int64_t row, int heads, int64_t head, int dim, int es) {
  Span s;
  s.hi = (int64_t)dim * es;
  s.add(rows, row, es);
  s.add(heads, head, es);
  return s;
}

Runs runs(const void *at, int64_t rows, int64_t row, int heads, int64_t head, int es) {
  return {(int64_t) reinterpret_cast<uintptr_t>(at), rows, row * es, heads, head * es};
}

}  // namespace

extern "C" int amap_rope_plan(int32_t head_dim, int32_t rotary_dim, const double *inv_freq, const int32_t *axis, int32_t n_axes,
                              int32_t pairs, float scale, amap_rope_t **out) {
  SERVE_REQUIRE(out, AMAP_EINVAL, "out: null pointer");
  SERVE_REQUIRE(head_dim >= 1 && head_dim <= AMAP_ROPE_MAX_DIM, AMAP_EINVAL, "head_dim: 1 .. 256");
  SERVE_REQUIRE(rotary_dim >= 0 && rotary_dim <= head_dim && rotary_dim % 2 == 0, AMAP_EINVAL, "rotary_dim: even, 0 .. head_dim");
  SERVE_REQUIRE(rotary_dim == 0 || inv_freq, AMAP_EINVAL, "inv_freq: null pointer");
  SERVE_REQUIRE(n_axes >= 1 && n_axes <= AMAP_ROPE_MAX_AXES, AMAP_EINVAL, "n_axes: 1 .. 4");
  SERVE_REQUIRE(pairs == AMAP_PAIRS_HALF || pairs == AMAP_PAIRS_ADJACENT, AMAP_EINVAL, "pairs: half or adjacent");
  SERVE_REQUIRE(std::isfinite(scale), AMAP_EINVAL, "scale: finite");
  for (int i = 0; i < rotary_dim / 2; ++i) {
    SERVE_REQUIRE(std::isfinite(inv_freq[i]), AMAP_EINVAL, "inv_freq: finite values");
    SERVE_REQUIRE(!axis || (axis[i] >= 0 && axis[i] < n_axes), AMAP_EINVAL, "axis: values in [0, n_axes)");
  }
  amap_rope_t *p = new (std::nothrow) amap_rope_t();
  SERVE_REQUIRE(p, AMAP_ENOMEM, "out of host memory");
  p->head_dim = head_dim;
  p->half = rotary_dim / 2;
  p->n_axes = n_axes;
  p->pairs = pairs;
  p->scale = scale;
  for (int i = 0; i < rotary_dim / 2; ++i) {
    const long double turns = (long double)inv_freq[i] / (2.0L * 3.14159265358979323846264338327950288L);
    const long double part = turns - floorl(turns);  // [0, 1]
    const long double fixed = floorl(part * 0x1p64L + 0.5L);
    p->phase[i] = fixed >= 0x1p64L ? 0 : (uint64_t)fixed;
    p->axis[i] = axis ? (uint8_t)axis[i] : 0;
  }
  *out = p;
  return accept();
}

extern "C" void amap_rope_destroy(amap_rope_t *plan) { delete plan; }

extern "C" int amap_rope_rotate(const amap_rope_t *plan, const amap_rope_args *a, void *cuda_stream) {
  SERVE_REQUIRE(plan && a, AMAP_EINVAL, "null pointer");
  SERVE_REQUIRE(a->n_parts >= 1 && a->n_parts <= 4, AMAP_EINVAL, "n_parts: 1 .. 4");
  SERVE_REQUIRE(a->dtype == AMAP_BF16 || a->dtype == AMAP_FP16 || a->dtype == AMAP_FP32, AMAP_EINVAL, "type: bf16, fp16 or fp32");
  if (const int rc = check_rows(a->rows, a->positions, a->position_bits)) return rc;
  if (a->rows == 0) return accept();
  const int es = dtype_bytes(a->dtype);
  Params P = {};
  for (int k = 0; k < a->n_parts; ++k) {
    const amap_rope_part &s = a->part[k];
    SERVE_REQUIRE(s.x && s.y, AMAP_EINVAL, "part: null pointer");
    SERVE_REQUIRE(s.heads >= 1 && s.heads <= 0xFFFF && s.reserved == 0, AMAP_EINVAL, "part: 1 .. 65535 heads");
    SERVE_REQUIRE(aligned(s.x, es) && aligned(s.y, es), AMAP_EALIGN, "part: misaligned");
    SERVE_REQUIRE((a->rows == 1 || s.y_row != 0) && (s.heads == 1 || s.y_head != 0), AMAP_EINVAL, "part: rows of y lie on one another");
    P.part[k] = {static_cast<const char *>(s.x), static_cast<char *>(s.y), s.x_row, s.x_head, s.y_row, s.y_head, 0,
                 s.heads, kRows, {}, 0, 0, {}};
  }
  // an output laid over an input is a race, unless the part is turned in place; parts turned in place may interleave in
  // one buffer (q and k of a fused projection), whose byte ranges overlap without sharing an element
  const int64_t width = (int64_t)plan->head_dim * es;
  for (int k = 0; k < a->n_parts; ++k) {
    const amap_rope_part &s = a->part[k];
    const bool in_place = s.x == s.y && s.x_row == s.y_row && s.x_head == s.y_head;
    const Span ys = rows_span(a->rows, s.y_row, s.heads, s.y_head, plan->head_dim, es);
    const Runs y = runs(s.y, a->rows, s.y_row, s.heads, s.y_head, es);
    for (int j = 0; j < a->n_parts; ++j) {
      const amap_rope_part &r = a->part[j];
      if (!in_place)
        SERVE_REQUIRE(!overlap(s.y, ys, r.x, rows_span(a->rows, r.x_row, r.heads, r.x_head, plan->head_dim, es)), AMAP_EINVAL,
                      "part: y overlaps an x that is not its own");
      else
        SERVE_REQUIRE(j == k || !share(y, runs(r.x, a->rows, r.x_row, r.heads, r.x_head, es), width), AMAP_EINVAL,
                      "parts: a y shares elements with an x that is not its own");
      SERVE_REQUIRE(j <= k || !share(y, runs(r.y, a->rows, r.y_row, r.heads, r.y_head, es), width), AMAP_EINVAL, "parts: two y share elements");
    }
  }
  P.n_parts = a->n_parts;
  P.rows = a->rows;
  P.positions = a->positions;
  P.position_axis = a->position_axis;
  P.position_row = a->position_row;
  P.wide_positions = a->position_bits == 64;
  P.sign = a->inverse ? -1.0f : 1.0f;
  return run_typed(*plan, P, a->dtype, es, cuda_stream);
}

extern "C" int amap_rope_append(const amap_rope_t *plan, const amap_append_args *a, void *cuda_stream) {
  SERVE_REQUIRE(plan && a, AMAP_EINVAL, "null pointer");
  SERVE_REQUIRE(a->dtype == AMAP_BF16 || a->dtype == AMAP_FP16, AMAP_EINVAL, "type: bf16 or fp16");
  if (const int rc = check_rows(a->rows, a->positions, a->position_bits)) return rc;
  if (const int rc = check_cache(a->cache)) return rc;
  SERVE_REQUIRE(a->cache.dtype == AMAP_E4M3 || a->cache.dtype == a->dtype, AMAP_EINVAL, "a 16-bit cache has the type of q, k and v");
  SERVE_REQUIRE(a->cache.head_dim == plan->head_dim, AMAP_EINVAL, "the cache's head size differs from the plan's");
  SERVE_REQUIRE(a->q_heads >= 0 && a->q_heads <= 0xFFFF && a->cache.heads <= 0xFFFF && a->reserved == 0, AMAP_EINVAL, "at most 65535 heads");
  if (a->rows == 0) return accept();
  SERVE_REQUIRE(a->k && a->v && a->slots && (a->q_heads == 0 || (a->q && a->q_out)), AMAP_EINVAL, "null pointer");
  const int es = dtype_bytes(a->dtype), ces = dtype_bytes(a->cache.dtype);
  SERVE_REQUIRE(aligned(a->q, es) && aligned(a->k, es) && aligned(a->v, es) && aligned(a->q_out, es) && aligned(a->slots, 4) &&
                    aligned(a->cache.k, ces) && aligned(a->cache.v, ces), AMAP_EALIGN, "misaligned pointer");
  const amap_cache &c = a->cache;
  SERVE_REQUIRE((c.n_pages == 1 || (c.k_page && c.v_page)) && (c.page_size == 1 || (c.k_token && c.v_token)) && (c.heads == 1 || (c.k_head && c.v_head)),
                AMAP_EINVAL, "the cache's rows lie on one another");
  SERVE_REQUIRE(a->q_heads == 0 || ((a->rows == 1 || a->q_out_row) && (a->q_heads == 1 || a->q_out_head)), AMAP_EINVAL, "rows of q_out lie on one another");
  const bool e4m3 = c.dtype == AMAP_E4M3;
  Params P = {};
  int n = 0;
  if (a->q_heads) {
    if (a->q_out != a->q || a->q_row != a->q_out_row || a->q_head != a->q_out_head) {
      const Span xs = rows_span(a->rows, a->q_row, a->q_heads, a->q_head, plan->head_dim, es);
      const Span ys = rows_span(a->rows, a->q_out_row, a->q_heads, a->q_out_head, plan->head_dim, es);
      SERVE_REQUIRE(!overlap(a->q, xs, a->q_out, ys) &&
                        !overlap(a->k, rows_span(a->rows, a->k_row, c.heads, a->k_head, plan->head_dim, es), a->q_out, ys) &&
                        !overlap(a->v, rows_span(a->rows, a->v_row, c.heads, a->v_head, plan->head_dim, es), a->q_out, ys),
                    AMAP_EINVAL, "q_out overlaps q, k or v");
    } else {  // in place: beside k and v in one buffer, but not over them
      const Runs y = runs(a->q_out, a->rows, a->q_out_row, a->q_heads, a->q_out_head, es);
      const int64_t width = (int64_t)plan->head_dim * es;
      SERVE_REQUIRE(!share(y, runs(a->k, a->rows, a->k_row, c.heads, a->k_head, es), width) &&
                        !share(y, runs(a->v, a->rows, a->v_row, c.heads, a->v_head, es), width), AMAP_EINVAL, "q_out overlaps k or v");
    }
    P.part[n++] = {static_cast<const char *>(a->q), static_cast<char *>(a->q_out), a->q_row, a->q_head, a->q_out_row, a->q_out_head, 0, a->q_heads, kRows,
                   {}, 0, 0, {}};
  }
  P.part[n++] = {static_cast<const char *>(a->k), static_cast<char *>(c.k), a->k_row, a->k_head, c.k_page, c.k_head, c.k_token, c.heads,
                 kCacheTurned, e4m3 ? divide_by(c.k_scale) : Divisor(), 0, 0, {}};
  P.part[n++] = {static_cast<const char *>(a->v), static_cast<char *>(c.v), a->v_row, a->v_head, c.v_page, c.v_head, c.v_token,
                 c.heads, kCacheCopied, e4m3 ? divide_by(c.v_scale) : Divisor(), 0, 0, {}};
  P.n_parts = n;
  P.rows = a->rows;
  P.positions = a->positions;
  P.position_axis = a->position_axis;
  P.position_row = a->position_row;
  P.wide_positions = a->position_bits == 64;
  P.sign = 1.0f;
  P.slots = a->slots;
  P.by_page = div_by(c.page_size);
  P.n_slots = c.n_pages * c.page_size;
  P.e4m3 = e4m3;
  return run_typed(*plan, P, a->dtype, ces, cuda_stream);
}
