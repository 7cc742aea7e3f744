// Rotary positions with several axes, and their fusion with the write into a paged cache.
//
// Pair i of a token at position p (along the pair's axis) turns by p * f_i radians.  The plan keeps f_i / 2pi as a
// 64-bit fraction of a turn; p times that fraction wraps modulo a full turn exactly, so the angle's error is
// p * 2^-65 turns whatever p is, and sincospi takes it from there in 32 bits.
//
// Bound: memory, every element is read and written once (a cos/sin pair serves all heads of a token, so the angles
// are 1/heads of the work and never leave the chip).
#include <cmath>
#include <cstring>
#include <new>

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

// where a part's rows go
enum { kRows = 0, kCacheTurned = 1, kCacheCopied = 2 };

struct Part {
  const char *x;
  char *y;
  int64_t x_row, x_head, y_row, y_head;  // elements; cache: y_row is the page stride
  int64_t y_token;
  int32_t first_head;  // heads of the parts before this one
  int32_t kind;
  float inv_scale;
};

struct Params {
  uint64_t phase[kMaxHalf];
  uint8_t axis[kMaxHalf];
  Part part[4];
  const void *positions;
  const int32_t *slots;
  int64_t position_axis, position_row;
  int64_t rows;
  int32_t n_parts, heads;  // heads of all parts together
  int32_t half, head_dim;
  int32_t items;  // per head: half/VEC chunks of pairs, then the chunks behind rotary_dim two at a time
  int32_t wide_positions, page_size, n_slots, e4m3;
  float scale, sign;
};

template <int DT, int VEC>
__device__ __forceinline__ void load(const char *p, int64_t at, float (&v)[VEC]) {
  using E = Elem<DT>;
  constexpr int ES = sizeof(typename E::T);
  union {
    typename Raw<VEC * ES>::T raw;
    typename E::T e[VEC];
  } u;
  u.raw = *reinterpret_cast<const typename Raw<VEC * ES>::T *>(p + at * ES);
#pragma unroll
  for (int j = 0; j < VEC; ++j) v[j] = E::to(u.e[j]);
}

template <int DT, int VEC>
__device__ __forceinline__ void store(char *p, int64_t at, const float (&v)[VEC], bool e4m3, float inv_scale) {
  using E = Elem<DT>;
  constexpr int ES = sizeof(typename E::T);
  if (e4m3) {
    union {
      typename Raw<VEC>::T raw;
      uint8_t e[VEC];
    } u;
#pragma unroll
    for (int j = 0; j < VEC; ++j) u.e[j] = to_e4m3(v[j] * inv_scale);
    *reinterpret_cast<typename Raw<VEC>::T *>(p + at) = u.raw;
  } else {
    union {
      typename Raw<VEC * ES>::T raw;
      typename E::T e[VEC];
    } u;
#pragma unroll
    for (int j = 0; j < VEC; ++j) u.e[j] = E::from(v[j]);
    *reinterpret_cast<typename Raw<VEC * ES>::T *>(p + at * ES) = u.raw;
  }
}

// One block per token: the threads first compute the token's cos and sin once, then walk its heads.  An item is VEC
// pairs: two chunks of VEC elements, half a rotary dimension apart (PAIRS_HALF) or side by side.
template <int DT, int VEC, int PAIRS>
__global__ void __launch_bounds__(kThreads) rope_kernel(const __grid_constant__ Params P) {
  __shared__ float2 turn[kMaxHalf];
  pdl_begin();
  const int64_t row = blockIdx.x;
  for (int i = threadIdx.x; i < P.half; i += kThreads) {
    const int64_t at = P.axis[i] * P.position_axis + row * P.position_row;
    const int64_t pos = P.wide_positions ? static_cast<const int64_t *>(P.positions)[at] : static_cast<const int32_t *>(P.positions)[at];
    const int32_t turns = (int32_t)(((uint64_t)pos * P.phase[i]) >> 32);  // in units of 2^-32 turns, [-1/2, 1/2)
    float s, c;
    sincospif((float)turns * 0x1p-31f, &s, &c);
    turn[i] = make_float2(c * P.scale, s * P.scale * P.sign);
  }
  __syncthreads();
  int64_t slot = -1;
  if (P.slots) {
    slot = P.slots[row];
    if (slot < 0 || slot >= P.n_slots) slot = -1;
  }
  const int chunks = P.half / VEC;
  for (int item = threadIdx.x; item < P.heads * P.items; item += kThreads) {
    const int head = item / P.items, c = item - head * P.items;
    int k = 0;
    while (k + 1 < P.n_parts && head >= P.part[k + 1].first_head) ++k;
    const Part &part = P.part[k];
    const int h = head - part.first_head;
    const int64_t x = row * part.x_row + h * part.x_head;
    int64_t y;
    bool e4m3 = false;
    if (part.kind == kRows) {
      y = row * part.y_row + h * part.y_head;
    } else {
      if (slot < 0) continue;
      y = slot / P.page_size * part.y_row + slot % P.page_size * part.y_token + h * part.y_head;
      e4m3 = P.e4m3;
    }
    if (c < chunks) {
      const int first = PAIRS == AMAP_PAIRS_HALF ? c * VEC : 2 * c * VEC;
      const int second = PAIRS == AMAP_PAIRS_HALF ? P.half + c * VEC : first + VEC;
      float a[VEC], b[VEC];
      load<DT, VEC>(part.x, x + first, a);
      load<DT, VEC>(part.x, x + second, b);
      if (part.kind != kCacheCopied) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float2 t = turn[c * VEC + j];
          if constexpr (PAIRS == AMAP_PAIRS_HALF) {
            const float u = a[j], w = b[j];
            a[j] = u * t.x - w * t.y;
            b[j] = w * t.x + u * t.y;
          } else {
            float &e0 = 2 * j < VEC ? a[(2 * j) % VEC] : b[(2 * j) % VEC];
            float &e1 = 2 * j + 1 < VEC ? a[(2 * j + 1) % VEC] : b[(2 * j + 1) % VEC];
            const float u = e0, w = e1;
            e0 = u * t.x - w * t.y;
            e1 = w * t.x + u * t.y;
          }
        }
      }
      store<DT, VEC>(part.y, y + first, a, e4m3, part.inv_scale);
      store<DT, VEC>(part.y, y + second, b, e4m3, part.inv_scale);
    } else {
      for (int q = 0; q < 2; ++q) {
        const int at = 2 * P.half + (2 * (c - chunks) + q) * VEC;
        if (at >= P.head_dim) break;
        float a[VEC];
        load<DT, VEC>(part.x, x + at, a);
        store<DT, VEC>(part.y, y + at, a, e4m3, part.inv_scale);
      }
    }
  }
}

template <int DT, int VEC>
int run(const amap_rope_t &plan, Params &P, void *stream) {
  P.items = P.half / VEC + ((P.head_dim - 2 * P.half) / VEC + 1) / 2;
  const dim3 grid((unsigned)P.rows);
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
  int64_t heads = 0;
  for (int k = 0; k < a->n_parts; ++k) {
    const amap_rope_part &s = a->part[k];
    SERVE_REQUIRE(s.x && s.y, AMAP_EINVAL, "part: null pointer");
    SERVE_REQUIRE(s.heads >= 1 && s.heads <= 0xFFFF && s.reserved == 0, AMAP_EINVAL, "part: 1 .. 65535 heads");
    SERVE_REQUIRE(aligned(s.x, es) && aligned(s.y, es), AMAP_EALIGN, "part: misaligned");
    SERVE_REQUIRE((a->rows == 1 || s.y_row != 0) && (s.heads == 1 || s.y_head != 0), AMAP_EINVAL, "part: rows of y lie on one another");
    P.part[k] = {static_cast<const char *>(s.x), static_cast<char *>(s.y), s.x_row, s.x_head, s.y_row, s.y_head, 0,
                 (int32_t)heads, kRows, 1.0f};
    heads += s.heads;
  }
  // an output laid over an input is a race, unless the part is turned in place; parts turned in place may interleave in
  // one buffer (q and k of a fused projection), whose byte ranges overlap without sharing an element
  for (int k = 0; k < a->n_parts; ++k) {
    const amap_rope_part &s = a->part[k];
    if (s.x == s.y && s.x_row == s.y_row && s.x_head == s.y_head) continue;
    const Span ys = rows_span(a->rows, s.y_row, s.heads, s.y_head, plan->head_dim, es);
    for (int j = 0; j < a->n_parts; ++j) {
      const amap_rope_part &r = a->part[j];
      SERVE_REQUIRE(!overlap(s.y, ys, r.x, rows_span(a->rows, r.x_row, r.heads, r.x_head, plan->head_dim, es)), AMAP_EINVAL,
                    "part: y overlaps an x that is not its own");
    }
  }
  P.n_parts = a->n_parts;
  P.heads = (int32_t)heads;
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
    }
    P.part[n++] = {static_cast<const char *>(a->q), static_cast<char *>(a->q_out), a->q_row, a->q_head, a->q_out_row, a->q_out_head, 0, 0, kRows, 1.0f};
  }
  P.part[n++] = {static_cast<const char *>(a->k), static_cast<char *>(c.k), a->k_row, a->k_head, c.k_page, c.k_head, c.k_token, a->q_heads,
                 kCacheTurned, 1.0f / c.k_scale};
  P.part[n++] = {static_cast<const char *>(a->v), static_cast<char *>(c.v), a->v_row, a->v_head, c.v_page, c.v_head, c.v_token,
                 a->q_heads + c.heads, kCacheCopied, 1.0f / c.v_scale};
  P.n_parts = n;
  P.heads = a->q_heads + 2 * c.heads;
  P.rows = a->rows;
  P.positions = a->positions;
  P.position_axis = a->position_axis;
  P.position_row = a->position_row;
  P.wide_positions = a->position_bits == 64;
  P.sign = 1.0f;
  P.slots = a->slots;
  P.page_size = c.page_size;
  P.n_slots = c.n_pages * c.page_size;
  P.e4m3 = c.dtype == AMAP_E4M3;
  return run_typed(*plan, P, a->dtype, ces, cuda_stream);
}
