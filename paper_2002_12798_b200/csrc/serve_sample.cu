// Sampling: temperature, top-k, min-p and top-p, and a token from one uniform number per row (amap_sample).
//
// Mathematics.  A token's weight is w = 2^y, y = (x - max) log2(e) / temperature, held as a whole number W of units of 2^-44: y
// comes out of one 64-bit multiply-add as a fixed-point number with 45 fractional bits, 2^y by table and a polynomial in
// integers (Tang, ACM Transactions on Mathematical Software 15, 1989): 2^-40 of itself.  Sums of W are whole numbers, so
// their order does not matter, and the answer is the 64-bit definition's for all but about one row in 10^7: with weights of
// 24 bits the borders between 10^5 tokens would move by a percent of the distance between them.
//
// What the settings keep is a beginning of the order by (logit, index), given by a last logit and how many of the tokens
// that have it are kept.  It is found by histograms of counts and sums: first over y (bins of 2^-6), then over the bits
// of the logits in the bin where the bound falls, until that holds one logit.  The draw takes the sums of each warp's run of
// the row, and goes through one of them.
//
// Bound: memory for many rows; the logits are read once from HBM and two to five times from the second-level cache.  A row
// is a cluster's, of as many blocks as fill the device, which exchange sums through shared memory.
#include <cooperative_groups.h>

#include <algorithm>
#include <atomic>
#include <cfloat>
#include <cmath>

#include "serve_common.cuh"

using namespace amap_serve;
namespace cg = cooperative_groups;

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMostBlocks = 8;          // of a cluster
constexpr int kBins = 2944;             // 46 powers of two in 64 bins each: all weights that are not zero
constexpr int kKeyBins = 2048;
constexpr int kPoints = 1024;           // of the table of 2^x
constexpr int kUnit = 44;               // W is in units of 2^-44

struct Params {
  amap_sample_args a;
  int32_t blocks;  // of a row
};

struct Tally {  // of the elements before a bound
  uint64_t mass;
  uint32_t count;
};

struct Shared {
  uint64_t table[kPoints];
  uint32_t count[kBins], low[kBins], high[kBins];  // a bin's tokens and the sum of their W
  uint64_t share_mass[kBins / 2];                  // the cluster's sums of this block's share of the bins
  uint32_t share_count[kBins / 2];
  // exchanged with the other blocks; every step has its own
  uint64_t block_mass, warp_mass[kWarps];
  uint32_t block_count, warp_equal[kWarps];
  float block_max;
  int32_t block_first;
  uint32_t block_least, block_most;
  uint64_t found_mass;
  uint32_t found_count, found_bin;
  // this block's
  uint64_t scan_mass[kWarps];
  uint32_t scan_count[kWarps];
  float warp_max[kWarps];
  int32_t warp_first[kWarps];
  uint32_t warp_least[kWarps], warp_most[kWarps];
  uint64_t all_mass[kMostBlocks * kWarps];
  uint32_t all_equal[kMostBlocks * kWarps];
  uint64_t pick_before;
  uint32_t pick_equal;
  int32_t pick_warp;
};

// order of floats as whole numbers
__device__ __forceinline__ uint32_t key_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);  // -0 is 0
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

// floor(f * m) for f in [0, 1)
__device__ __forceinline__ uint64_t share_of(float f, uint64_t m) {
  const uint32_t b = __float_as_uint(f), e = b >> 23;
  if (!(f > 0.0f)) return 0;
  const uint64_t mant = e ? (b & 0x7FFFFFu) | 0x800000u : b & 0x7FFFFFu;
  const int down = 150 - (int)(e ? e : 1);  // f = mant * 2^-down
  const uint64_t hi = __umul64hi(mant, m), lo = mant * m;
  if (down >= 128) return 0;
  return down >= 64 ? (down == 64 ? hi : hi >> (down - 64)) : hi << (64 - down) | lo >> down;
}
// ceil(f * m) likewise
__device__ __forceinline__ uint64_t share_up(float f, uint64_t m) {
  const uint64_t whole = share_of(f, m);
  if (!(f > 0.0f)) return 0;
  const uint32_t b = __float_as_uint(f), e = b >> 23;
  const uint64_t mant = e ? (b & 0x7FFFFFu) | 0x800000u : b & 0x7FFFFFu;
  const int down = 150 - (int)(e ? e : 1);
  const uint64_t hi = __umul64hi(mant, m), lo = mant * m;
  const bool rest = down >= 128 ? (hi | lo) != 0 : down >= 64 ? lo != 0 || (down > 64 && hi << (128 - down) != 0) : lo << (64 - down) != 0;
  return whole + rest;
}

template <int DT>
struct Sampler {
  using T = typename Elem<DT>::T;
  static constexpr int VEC = 16 / sizeof(T), kAhead = 16 / VEC;  // vectors under way in a thread
  Shared &S;
  const T *x;
  int vocab, shift;      // shift: elements between the 16-byte boundary at or before x and x
  int begin, end;        // this warp's vectors, counted from that boundary
  int blocks, rank;
  float top;             // the largest logit
  bool infinite;         // it is +infinity
  double by;             // y = (x - top) by
  float range;           // weights of logits further than this below it are zero
  uint64_t least;        // smaller weights count as zero (min_p)

  __device__ __forceinline__ void load(int j, float (&v)[VEC]) const {
    const int first = j * VEC - shift;
    if (j < end && first >= 0 && first + VEC <= vocab) {
      union {
        uint4 raw;
        T e[VEC];
      } u;
      u.raw = *reinterpret_cast<const uint4 *>(x + first);
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[i] = Elem<DT>::to(u.e[i]);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[i] = j < end && first + i >= 0 && first + i < vocab ? Elem<DT>::to(x[first + i]) : __uint_as_float(0x7FC00000u);
    }
  }
  // f(index, value) for every element of this lane's vectors; NaN for those that are none
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    for (int j = begin + (threadIdx.x & 31); j < end; j += 32 * kAhead) {
      float v[kAhead][VEC];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) load(j + 32 * k, v[k]);
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) f((j + 32 * k) * VEC - shift + i, v[k][i]);
      }
    }
  }

  // y + 64 with 45 fractional bits; 0 for what has no weight
  __device__ __forceinline__ uint64_t place_of(float v) const {
    if (infinite) return v == top ? 64ull << 45 : 0;
    if (!(top - v <= range)) return 0;  // NaN and -infinity among them
    // 192 + y lies between 128 and 256, where a double's last bit is 2^-45
    return (uint64_t)__double_as_longlong(fma((double)v - (double)top, by, 192.0)) & ((1ull << 52) - 1);
  }
  __device__ __forceinline__ uint64_t weight_of(uint64_t place) const {
    const uint32_t whole = (uint32_t)(place >> 45), point = (uint32_t)(place >> 35) & (kPoints - 1), rest = (uint32_t)(place >> 3);
    // rest: 32 bits of what is beyond the point, d = rest 2^-42; 2^d - 1 = e + e^2/2 + e^3/6 with e = d ln 2, in units of 2^-42
    const uint32_t e = __umulhi(rest, 2977044472u), e2 = __umulhi(e, e), e3 = __umulhi(e2, e);
    const uint32_t p = e + (e2 >> 11) + (__umulhi(e3, 715827883u) >> 20);
    if (whole < 20) return 0;
    const uint64_t t = S.table[point];
    const uint64_t w = (t + ((uint64_t)__umulhi((uint32_t)(t >> 13), p) << 3)) >> (64 - whole);
    return w >= least ? w : 0;
  }
  __device__ __forceinline__ uint64_t weight(float v) const { return weight_of(place_of(v)); }
  static __device__ __forceinline__ int bin_of(uint64_t place) { return (int)(((64ull << 45) - place) >> 39); }

  __device__ __forceinline__ void clear_bins(int n) const {
    for (int i = threadIdx.x; i < n; i += kThreads) S.count[i] = S.low[i] = S.high[i] = 0;
    __syncthreads();
  }
  __device__ __forceinline__ void add(int bin, uint64_t w) const {
    atomicAdd(&S.count[bin], 1u);
    const uint32_t lo = (uint32_t)w, before = atomicAdd(&S.low[bin], lo);
    const uint32_t hi = (uint32_t)(w >> 32) + (before + lo < lo);
    if (hi) atomicAdd(&S.high[bin], hi);
  }

  // Sums over the block (every thread gets them)
  __device__ __forceinline__ Tally block_sum(Tally t) const {
#pragma unroll
    for (int d = 16; d; d >>= 1) {
      t.mass += __shfl_xor_sync(~0u, t.mass, d);
      t.count += __shfl_xor_sync(~0u, t.count, d);
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) S.scan_mass[threadIdx.x >> 5] = t.mass, S.scan_count[threadIdx.x >> 5] = t.count;
    __syncthreads();
    Tally all = {0, 0};
#pragma unroll
    for (int w = 0; w < kWarps; ++w) all.mass += S.scan_mass[w], all.count += S.scan_count[w];
    return all;
  }

  // The first bin at whose end the tokens so far (by_count) are `want` or more, or their sum `target` or more, and the tally
  // before it.  Adds the cluster's histograms up on the way: a block has a share of the bins.  There is such a bin.
  __device__ Tally find_bin(int n, bool by_count, uint32_t want, uint64_t target, int *bin) const {
    cg::cluster_group cluster = cg::this_cluster();
    const int per = (n + blocks - 1) / blocks, first = rank * per, mine = max(0, min(per, n - first));
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (blocks > 1) cluster.sync();
    else __syncthreads();
    auto get = [&](int i, Tally *t) {  // bin first + i, of the whole cluster
      if (blocks > 1) *t = {S.share_mass[i], S.share_count[i]};
      else *t = {(uint64_t)S.high[i] << 32, S.count[i]}, t->mass += S.low[i];
    };
    Tally sum = {0, 0};
    if (blocks > 1) {
      for (int i = tid; i < mine; i += kThreads) {
        Tally t = {0, 0};
        for (int b = 0; b < blocks; ++b) {
          const Shared *o = cluster.map_shared_rank(&S, b);
          t.mass += ((uint64_t)o->high[first + i] << 32) + o->low[first + i];
          t.count += o->count[first + i];
        }
        S.share_mass[i] = t.mass, S.share_count[i] = t.count;
      }
      __syncthreads();
    }
    // runs of bins: a thread's, side by side
    const int run = (mine + kThreads - 1) / kThreads, i0 = min(mine, tid * run), i1 = min(mine, i0 + run);
    for (int i = i0; i < i1; ++i) {
      Tally t;
      get(i, &t);
      sum.mass += t.mass, sum.count += t.count;
    }
    Tally upto = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint64_t m = __shfl_up_sync(~0u, upto.mass, d);
      const uint32_t c = __shfl_up_sync(~0u, upto.count, d);
      if (lane >= d) upto.mass += m, upto.count += c;
    }
    __syncthreads();
    if (lane == 31) S.scan_mass[warp] = upto.mass, S.scan_count[warp] = upto.count;
    __syncthreads();
    Tally whole = {0, 0};
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) upto.mass += S.scan_mass[w], upto.count += S.scan_count[w];
      whole.mass += S.scan_mass[w], whole.count += S.scan_count[w];
    }
    if (blocks > 1) {
      if (tid == 0) S.block_mass = whole.mass, S.block_count = whole.count, S.found_bin = ~0u;
      cluster.sync();
      for (int b = 0; b < rank; ++b) {
        const Shared *o = cluster.map_shared_rank(&S, b);
        upto.mass += o->block_mass, upto.count += o->block_count;
      }
    } else {
      if (tid == 0) S.found_mass = 0, S.found_count = 0, S.found_bin = 0;
      __syncthreads();
    }
    auto enough = [&](const Tally &t) { return by_count ? t.count >= want : t.mass >= target; };
    Tally before = {upto.mass - sum.mass, upto.count - sum.count};
    if (enough(upto) && !enough(before)) {  // one thread of the cluster
      for (int i = i0; i < i1; ++i) {
        Tally t;
        get(i, &t);
        t.mass += before.mass, t.count += before.count;
        if (enough(t)) {
          S.found_mass = before.mass, S.found_count = before.count, S.found_bin = first + i;
          break;
        }
        before = t;
      }
    }
    if (blocks > 1) {
      cluster.sync();
      Tally t = {0, 0};
      *bin = 0;
      for (int b = 0; b < blocks; ++b) {
        const Shared *o = cluster.map_shared_rank(&S, b);
        if (o->found_bin != ~0u) *bin = (int)o->found_bin, t = {o->found_mass, o->found_count};
      }
      cluster.sync();  // before anybody writes to these again
      return t;
    }
    __syncthreads();
    *bin = (int)S.found_bin;
    const Tally t = {S.found_mass, S.found_count};
    __syncthreads();
    return t;
  }

  // Among the tokens of a bin of y: the logit (as a key) at which `want` tokens or the sum `target` are reached, and the tally
  // before it.
  __device__ Tally refine(int bin, bool by_count, uint32_t want, uint64_t target, uint32_t *key) const {
    cg::cluster_group cluster = cg::this_cluster();
    uint32_t lo = ~0u, hi = 0;
    each([&](int, float v) {
      const uint64_t place = place_of(v);
      if (place && bin_of(place) == bin && weight_of(place)) lo = min(lo, key_of(v)), hi = max(hi, key_of(v));
    });
    lo = __reduce_min_sync(~0u, lo), hi = __reduce_max_sync(~0u, hi);
    if ((threadIdx.x & 31) == 0) S.warp_least[threadIdx.x >> 5] = lo, S.warp_most[threadIdx.x >> 5] = hi;
    __syncthreads();
    lo = ~0u, hi = 0;
    for (int w = 0; w < kWarps; ++w) lo = min(lo, S.warp_least[w]), hi = max(hi, S.warp_most[w]);
    if (blocks > 1) {
      if (threadIdx.x == 0) S.block_least = lo, S.block_most = hi;
      cluster.sync();
      for (int b = 0; b < blocks; ++b) {
        const Shared *o = cluster.map_shared_rank(&S, b);
        lo = min(lo, o->block_least), hi = max(hi, o->block_most);
      }
      cluster.sync();
    }
    Tally all = {0, 0};
    for (int pass = 0; pass < 3 && lo < hi; ++pass) {  // 11 bits each
      const int down = max(0, 32 - __clz(hi - lo) - 11);  // hi - lo >> down is below kKeyBins
      __syncthreads();
      clear_bins(kKeyBins);
      each([&](int, float v) {
        const uint64_t place = place_of(v);
        if (!place || bin_of(place) != bin) return;
        const uint32_t k = key_of(v);
        const uint64_t w = weight_of(place);
        if (w && k >= lo && k <= hi) add((hi - k) >> down, w);
      });
      int at;
      const Tally t = find_bin(kKeyBins, by_count, want - all.count, target - all.mass, &at);
      all.mass += t.mass, all.count += t.count;
      hi -= (uint32_t)at << down;
      lo = max(lo, hi - min(hi, (1u << down) - 1));
    }
    *key = hi;
    return all;
  }
};

template <int DT>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const __grid_constant__ Params P) {
  extern __shared__ __align__(16) char smem[];
  Shared &S = *reinterpret_cast<Shared *>(smem);
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, row = blockIdx.x / P.blocks;
  for (int i = tid; i < kPoints; i += kThreads) S.table[i] = (uint64_t)rint(exp2((double)i / kPoints) * (double)(1ull << kUnit));
  pdl_begin();
  using Z = Sampler<DT>;
  Z z{S};
  z.blocks = P.blocks, z.rank = blockIdx.x - row * P.blocks;
  z.x = static_cast<const typename Z::T *>(P.a.logits) + (int64_t)row * P.a.row;
  z.vocab = P.a.vocab;
  z.shift = (int)((reinterpret_cast<uintptr_t>(z.x) % 16) / sizeof(typename Z::T));
  const int vectors = (z.vocab + z.shift + Z::VEC - 1) / Z::VEC, warps = P.blocks * kWarps, per = (vectors + 32 * warps - 1) / (32 * warps) * 32;
  z.begin = min(vectors, (z.rank * kWarps + warp) * per), z.end = min(vectors, z.begin + per);
  const float temperature = P.a.by_row & 1 ? P.a.temperatures[row] : P.a.temperature;
  const int top_k = P.a.by_row & 2 ? P.a.top_ks[row] : P.a.top_k;
  const float top_p = P.a.by_row & 4 ? P.a.top_ps[row] : P.a.top_p, min_p = P.a.by_row & 8 ? P.a.min_ps[row] : P.a.min_p;

  // ---- the largest logit, the first of them ----
  float best = -INFINITY;
  int first = 0x7FFFFFFF;
  z.each([&](int i, float v) {
    if (v > best) best = v, first = i;
  });
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    const float v = __shfl_xor_sync(~0u, best, d);
    const int i = __shfl_xor_sync(~0u, first, d);
    if (v > best || (v == best && i < first)) best = v, first = i;
  }
  if (lane == 0) S.warp_max[warp] = best, S.warp_first[warp] = first;
  __syncthreads();
  auto better = [&](float v, int i) {
    if (v > best || (v == best && i < first)) best = v, first = i;
  };
  for (int w = 0; w < kWarps; ++w) better(S.warp_max[w], S.warp_first[w]);
  if (P.blocks > 1) {
    if (tid == 0) S.block_max = best, S.block_first = first;
    cluster.sync();
    for (int b = 0; b < P.blocks; ++b) {
      const Shared *o = cluster.map_shared_rank(&S, b);
      better(o->block_max, o->block_first);
    }
  }
  if (!(temperature > 0.0f) || best == -INFINITY) {
    if (z.rank == 0 && tid == 0) {
      P.a.tokens[row] = best == -INFINITY ? -1 : first;
      if (P.a.logprobs) P.a.logprobs[row] = best == -INFINITY ? -INFINITY : 0.0f;
    }
    if (P.blocks > 1) cluster.sync();  // nobody leaves while its shared memory is read
    return;
  }
  z.top = best;
  z.infinite = best == INFINITY;
  z.by = 1.4426950408889634 / (double)temperature;
  z.range = fminf(40.0f * temperature, FLT_MAX);  // 2^-57.7
  z.least = min_p > 0.0f ? (uint64_t)ceil((double)fminf(min_p, 1.0f) * (double)(1ull << kUnit)) : 1;

  // ---- what is kept: tokens with a larger key than `last`, and the first `equal` of those that have it ----
  uint32_t last = 0, equal = ~0u;
  uint64_t last_weight = 0;
  const bool by_k = top_k > 0 && top_k < z.vocab, by_p = top_p < 1.0f;
  if (by_k || by_p) {
    z.clear_bins(kBins);
    Tally all = {0, 0};
    z.each([&](int, float v) {
      const uint64_t place = z.place_of(v);
      if (!place) return;
      const uint64_t w = z.weight_of(place);
      if (!w) return;
      z.add(Z::bin_of(place), w);
      all.mass += w, ++all.count;
    });
    all = z.block_sum(all);
    if (P.blocks > 1) {
      if (tid == 0) S.block_mass = all.mass, S.block_count = all.count;
      cluster.sync();
      all = {0, 0};
      for (int b = 0; b < P.blocks; ++b) {
        const Shared *o = cluster.map_shared_rank(&S, b);
        all.mass += o->block_mass, all.count += o->block_count;
      }
      cluster.sync();
    }
    uint64_t base = all.mass;  // what top_p is a part of
    int bin_k = 0, bin_p = 0;
    Tally k = {0, 0}, p = {0, 0};
    const bool cut = by_k && (uint32_t)top_k < all.count;
    // the bins' sums are needed for both bounds, before refining writes over them: top_p's bin is looked for among
    // the sums that top_k leaves, which refining its bin gives; so the histogram is made anew in between
    if (cut) {
      k = z.find_bin(kBins, true, top_k, 0, &bin_k);
      const Tally in = z.refine(bin_k, true, top_k - k.count, 0, &last);
      last_weight = z.weight(of_key(last));
      equal = top_k - k.count - in.count;
      base = k.mass + in.mass + equal * last_weight;
    }
    if (by_p) {
      const uint64_t target = max(share_up(fmaxf(top_p, 0.0f), base), (uint64_t)1);
      if (cut) {
        __syncthreads();
        z.clear_bins(kBins);
        z.each([&](int, float v) {
          const uint64_t place = z.place_of(v);
          if (!place || key_of(v) < last) return;
          const uint64_t w = z.weight_of(place);
          if (w) z.add(Z::bin_of(place), w);
        });
      }
      p = z.find_bin(kBins, false, 0, target, &bin_p);
      const Tally in = z.refine(bin_p, false, 0, target - p.mass, &last);
      last_weight = z.weight(of_key(last));
      const uint64_t left = target - p.mass - in.mass;
      equal = (uint32_t)((left + last_weight - 1) / last_weight);
    }
  }

  // ---- the draw ----
  uint64_t mass = 0;
  uint32_t same = 0;
  z.each([&](int, float v) {
    const uint64_t place = z.place_of(v);
    if (!place) return;
    const uint32_t k = key_of(v);
    if (k > last) mass += z.weight_of(place);
    else same += k == last;
  });
#pragma unroll
  for (int d = 16; d; d >>= 1) mass += __shfl_xor_sync(~0u, mass, d);
  same = __reduce_add_sync(~0u, same);
  if (lane == 0) S.warp_mass[warp] = mass, S.warp_equal[warp] = same;
  if (P.blocks > 1) cluster.sync();
  else __syncthreads();
  if (tid < warps) {
    const Shared *o = P.blocks > 1 ? cluster.map_shared_rank(&S, tid / kWarps) : &S;
    S.all_mass[tid] = o->warp_mass[tid % kWarps], S.all_equal[tid] = o->warp_equal[tid % kWarps];
  }
  __syncthreads();
  if (warp == 0) {
    // four warps' runs to a lane
    constexpr int kEach = kMostBlocks * kWarps / 32;
    uint64_t m[kEach];
    uint32_t e[kEach], equals = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int w = lane * kEach + i;
      m[i] = w < warps ? S.all_mass[w] : 0, e[i] = w < warps ? S.all_equal[w] : 0;
      equals += e[i];
    }
    uint32_t before_equal = equals;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint32_t v = __shfl_up_sync(~0u, before_equal, d);
      if (lane >= d) before_equal += v;
    }
    before_equal -= equals;
    uint64_t sum = 0;
    uint32_t b = before_equal;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      m[i] += last_weight * (uint64_t)min(e[i], equal - min(equal, b));
      b += e[i];
      sum += m[i];
    }
    uint64_t upto = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint64_t v = __shfl_up_sync(~0u, upto, d);
      if (lane >= d) upto += v;
    }
    const uint64_t all = __shfl_sync(~0u, upto, 31);
    const float u = P.a.uniform[row];
    const uint64_t target = share_of(u > 0.0f ? fminf(u, 0x1.fffffep-1f) : 0.0f, all);
    uint64_t before = upto - sum;
    b = before_equal;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (before <= target && target < before + m[i]) S.pick_warp = lane * kEach + i, S.pick_before = target - before, S.pick_equal = b;
      before += m[i];
      b += e[i];
    }
    if (lane == 0) S.all_mass[0] = all;
  }
  __syncthreads();
  if (S.pick_warp / kWarps == z.rank && S.pick_warp % kWarps == warp) {
    const uint64_t target = S.pick_before, all = S.all_mass[0];
    uint64_t before = 0;
    uint32_t seen = S.pick_equal;
    for (int j0 = z.begin; j0 < z.end; j0 += 32) {
      float v[Z::VEC];
      z.load(j0 + lane, v);
      uint32_t equals = 0;
#pragma unroll
      for (int i = 0; i < Z::VEC; ++i) equals += z.place_of(v[i]) && key_of(v[i]) == last;
      uint32_t rank = equals;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t t = __shfl_up_sync(~0u, rank, d);
        if (lane >= d) rank += t;
      }
      const uint32_t row_equals = __shfl_sync(~0u, rank, 31);
      rank += seen - equals;
      uint64_t w[Z::VEC], sum = 0;
#pragma unroll
      for (int i = 0; i < Z::VEC; ++i) {
        w[i] = 0;
        if (z.place_of(v[i])) {
          const uint32_t k = key_of(v[i]);
          if (k > last) w[i] = z.weight(v[i]);
          else if (k == last && rank++ < equal) w[i] = last_weight;
        }
        sum += w[i];
      }
      uint64_t upto = sum;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint64_t t = __shfl_up_sync(~0u, upto, d);
        if (lane >= d) upto += t;
      }
      const uint64_t step = __shfl_sync(~0u, upto, 31);
      upto += before;
      if (target < before + step) {
        if (target < upto && target >= upto - sum) {
          uint64_t at = upto - sum;
#pragma unroll
          for (int i = 0; i < Z::VEC; ++i) {
            if (target >= at && target < at + w[i]) {
              P.a.tokens[row] = (j0 + lane) * Z::VEC - z.shift + i;
              if (P.a.logprobs) P.a.logprobs[row] = (float)log((double)w[i] / (double)all);
            }
            at += w[i];
          }
        }
        break;
      }
      before += step;
      seen += row_equals;
    }
  }
  if (P.blocks > 1) cluster.sync();  // nobody leaves while its shared memory is read
}

template <int DT>
int run(const Params &P, void *stream) {
  static std::atomic<bool> known[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && dev < 64 && !known[dev].load(std::memory_order_relaxed)) {
    e = cudaFuncSetAttribute(sample_kernel<DT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared));
    if (e == cudaSuccess) known[dev].store(true, std::memory_order_relaxed);
  }
  if (e != cudaSuccess || dev >= 64) {
    cudaGetLastError();
    return refuse(AMAP_ECUDA, e != cudaSuccess ? cudaGetErrorString(e) : "device number");
  }
  return launch_clusters(sample_kernel<DT>, dim3((unsigned)(P.a.rows * P.blocks)), P.blocks, kThreads, sizeof(Shared), stream, P);
}

}  // namespace

extern "C" int amap_sample(const amap_sample_args *a, void *cuda_stream) {
  SERVE_REQUIRE(a, AMAP_EINVAL, "null pointer");
  SERVE_REQUIRE(a->rows >= 1 && a->rows <= 0xFFFF, AMAP_EINVAL, "rows: 1 .. 65535");
  SERVE_REQUIRE(a->vocab >= 1 && a->vocab <= 1 << 20, AMAP_EINVAL, "vocab: 1 .. 2^20");
  SERVE_REQUIRE(a->dtype == AMAP_BF16 || a->dtype == AMAP_FP16 || a->dtype == AMAP_FP32, AMAP_EINVAL, "type: bf16, fp16 or fp32");
  SERVE_REQUIRE((a->by_row & ~15) == 0, AMAP_EINVAL, "by_row: bits 0 .. 3");
  SERVE_REQUIRE(a->logits && a->uniform && a->tokens && (!(a->by_row & 1) || a->temperatures) && (!(a->by_row & 2) || a->top_ks) &&
                    (!(a->by_row & 4) || a->top_ps) && (!(a->by_row & 8) || a->min_ps), AMAP_EINVAL, "null pointer");
  SERVE_REQUIRE((a->by_row & 1) || std::isfinite(a->temperature), AMAP_EINVAL, "temperature: finite");
  SERVE_REQUIRE((a->by_row & 4) || (a->top_p >= 0 && a->top_p <= 1), AMAP_EINVAL, "top_p: 0 .. 1");
  SERVE_REQUIRE((a->by_row & 8) || (a->min_p >= 0 && a->min_p <= 1), AMAP_EINVAL, "min_p: 0 .. 1");
  SERVE_REQUIRE(aligned(a->logits, dtype_bytes(a->dtype)) && aligned(a->uniform, 4) && aligned(a->tokens, 4) && aligned(a->logprobs, 4) &&
                    aligned(a->temperatures, 4) && aligned(a->top_ks, 4) && aligned(a->top_ps, 4) && aligned(a->min_ps, 4), AMAP_EALIGN, "misaligned pointer");
  Params P = {};
  P.a = *a;
  // blocks of a row: as many as fill the device twice over, but none with less than two vectors of 16 bytes a thread
  const int64_t vectors = (int64_t)a->vocab * dtype_bytes(a->dtype) / 16;
  P.blocks = 1;
  while (P.blocks < kMostBlocks && (int64_t)a->rows * P.blocks * 2 <= 2 * device_sms() && vectors >= P.blocks * 4 * kThreads) P.blocks *= 2;
  switch (a->dtype) {
    case AMAP_BF16: return run<AMAP_BF16>(P, cuda_stream);
    case AMAP_FP16: return run<AMAP_FP16>(P, cuda_stream);
    default: return run<AMAP_FP32>(P, cuda_stream);
  }
}
