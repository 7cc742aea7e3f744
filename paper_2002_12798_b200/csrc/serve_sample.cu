// Sampling: temperature, top-k, min-p and top-p, and a token from one uniform number per row (amap_sample).
//
// Mathematics.  A token's weight w = 2^y, y = (x - max) log2(e) / temperature, by a table of 2^(i/1024) and a polynomial of degree 3
// in 64 bits (Tang, ACM Transactions on Mathematical Software 15, 1989), is rounded to a whole number W of units of 2^-44.
// Sums of W are whole numbers, so their order does not matter.  W is off by half a unit at most, and weights below 2^-45 are none: a
// sum is off by 2^-45 of the largest weight for each token, 2^-26 of it at most (2^19 tokens just below 2^-45), as a rule by
// far less, since roundings go either way.  The answer is the 64-bit definition's where the uniform number is further than that from
// a border between two tokens: with weights of 24 bits, rows of 10^5 tokens would often come out otherwise.
//
// What the settings keep is a beginning of the order by (logit, index), given by a last logit and how many of the tokens
// that have it are kept.  A first bound is cheap: min_p gives one; for top_k the top_k-th largest of the threads' own
// maxima; for top_p alone the weight that all tokens together would need to make up the rest.  The tokens above it, few as
// a rule, are listed by each warp, and if there are 1024 at most one block sorts them and is done.  More of them, or a row
// whose lists overflow, go by histograms of counts and sums: first over y (64 bins to a power of two), then over the bits
// of the logits in the bin where a bound falls, until that holds one logit.  bf16 logits, of which some thousand different
// ones have a weight, are counted in a bin of their own each, and weighed once.  The draw takes the sums of each warp's run
// of the row (or of its list), and goes through one of them.
//
// Bound: latency.  Where all tokens are weighed one by one (about 25 instructions, nine of them in 64 bits) no unit is near its
// limit: 128 x 131072 fp32 have 49 % of the issue slots, 15 % of the 64-bit pipe, and wait for loads first, for one another
// and for barriers next; 64 registers a thread, for two blocks of 16 warps, leave 56 to 76 bytes of spills (240 to 316 read back).  The largest logit's
// pass is memory's.  The rest are chains: one row, of 1000 logits in one block or of 32000 in eight, is 15 to 19 us of bins
// cleared and scanned for a bound, two sorts of 15 barriers and more, and scans, with exchanges of one to four us where
// there are blocks to exchange with.  The logits come from HBM once, and from the second-level cache once or twice more.  A row is a
// cluster's, of as many blocks as fill the device, which exchange sums through shared memory.
//
// Measured: one row of 32000 fp32 logits, 50 largest, top_p 0.95, 20 us; 64 rows of 100003 bf16, top_p 0.9, 61; 128 of 131072
// fp32, nothing cut off, 62 (67 MB: 10 from HBM); 256 of 150001 bf16 with settings of their own 130 to 142, by the settings drawn.
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
constexpr int kBins = 4096;             // bins of y: 64 to a power of two, in all 45 of which weights are not zero; or bf16 logits
constexpr int kKeyBins = 2048;
constexpr int kPoints = 1024;           // of the table of 2^x
constexpr int kUnit = 44;               // W is in units of 2^-44
constexpr int kListBytes = 2560;        // of a warp's list
constexpr int kSorted = 1024;           // tokens that one block sorts

struct Params {
  amap_sample_args a;
  int32_t blocks;  // of a row
};

struct Tally {  // of the elements before a bound
  uint64_t mass;
  uint32_t count;
};

struct Shared {
  double table[kPoints];
  union {
    struct {
      uint32_t count[kBins], low[kBins], high[kBins];  // a bin's tokens and the sum of their W
    };
    uint64_t order[kSorted];     // key and index of the tokens to be sorted
    uint64_t weight_of[kBins];   // of a bf16 logit
  };
  char lists[kWarps][kListBytes];
  // exchanged with the other blocks
  uint64_t run_mass[kThreads];  // of the bins that a thread adds up
  uint32_t run_count[kThreads];
  Tally block_tally[2];
  uint64_t warp_mass[kWarps];
  uint32_t warp_equal[kWarps], warp_listed[kWarps];
  float block_max;
  int32_t block_first;
  uint32_t block_least, block_most;
  // this block's
  Tally found;
  uint32_t found_run, found_bin;
  uint64_t scan_mass[kWarps];
  uint32_t scan_count[kWarps];
  float warp_max[kWarps];
  int32_t warp_first[kWarps];
  uint32_t warp_least[kWarps], warp_most[kWarps];
  uint64_t all_mass[kMostBlocks * kWarps];
  uint32_t all_equal[kMostBlocks * kWarps];
  uint64_t pick_before, total;
  uint32_t pick_equal;
  int32_t pick_warp, kept;
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
  // a token of a list: its logit, and its place in the warp's run of the row (65536 tokens at most)
  struct Entry {
    uint16_t at;
    T logit;
  };
  static constexpr int kListed = kListBytes / sizeof(Entry);
  static constexpr int VEC = 16 / sizeof(T), kAhead = 3;  // elements of a vector; vectors under way in a thread
  Shared &S;
  const T *x;
  int vocab, shift;      // shift: elements between the 16-byte boundary at or before x and x
  int begin, end;        // this warp's vectors, counted from that boundary
  int blocks, rank;
  bool alone;            // only tokens with the largest logit have a weight, as it is +infinity or next to the lowest float: they count as 0,
                         // the others as -1
  float largest;
  double top, by;        // y = (x - top) by / 1024
  float least_value;     // smaller logits, and NaN, have no weight, and are taken to be this one
  uint64_t least;        // smaller W count as zero (min_p)
  bool listed;           // the tokens are those of the warps' lists
  int n_listed;

  union Vector {
    uint4 raw;
    T e[VEC];
  };
  // the j-th vector before `until`; NaN for what lies outside the row
  __device__ __forceinline__ Vector load(int j, int until) const {
    const int first = j * VEC - shift;
    Vector u;
    if (j < until && first >= 0 && first + VEC <= vocab) {
      u.raw = *reinterpret_cast<const uint4 *>(x + first);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) u.e[i] = j < until && first + i >= 0 && first + i < vocab ? x[first + i] : Elem<DT>::from(__uint_as_float(0x7FC00000u));
    }
    return u;
  }
  // f(index of the first, logits) for this lane's vectors among those from `from` to `until`; NaN for what is no element of the row
  template <typename F>
  __device__ __forceinline__ void each_vector(int from, int until, F f) const {
    int j = from + (threadIdx.x & 31);
    Vector ahead[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) ahead[k] = load(j + 32 * k, until);
#pragma unroll 1
    for (; j - (int)(threadIdx.x & 31) < until; j += 32) {
      const Vector u = ahead[0];
#pragma unroll
      for (int k = 0; k + 1 < kAhead; ++k) ahead[k] = ahead[k + 1];
      ahead[kAhead - 1] = load(j + 32 * kAhead, until);
      float v[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[i] = Elem<DT>::to(u.e[i]);
      f(j * VEC - shift, v);
    }
  }
  // f(index, logit) for each element
  template <typename F>
  __device__ __forceinline__ void each_between(int from, int until, F f) const {
    each_vector(from, until, [&](int first, const float (&v)[VEC]) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) f(first + i, v[i]);
    });
  }
  template <typename F>
  __device__ __forceinline__ void each_of_row(F f) const { each_between(begin, end, f); }
  __device__ __forceinline__ float value(float v) const { return fmaxf(alone ? (v == largest ? 0.0f : -1.0f) : v, least_value); }
  __device__ __forceinline__ Entry *list() const { return reinterpret_cast<Entry *>(S.lists[threadIdx.x >> 5]); }
  __device__ __forceinline__ int index_of(const Entry &e) const { return begin * VEC - shift + e.at; }
  // f(value) for every token, of the row or of the lists
  template <typename F>
  __device__ __forceinline__ void each(F f) const {
    if (listed) {
      for (int i = threadIdx.x & 31; i < n_listed; i += 32) f(value(Elem<DT>::to(list()[i].logit)));
    } else {
      each_of_row([&](int, float v) { f(value(v)); });
    }
  }

  // W of a token, and 1024 y rounded
  __device__ __forceinline__ uint64_t weight(float v, int *y) const {
    constexpr double kMagic = 0x1.8p52, kBase = 0x1.8p8;
    constexpr double c1 = 6.769015435155716e-4, c2 = 2.290978498068816e-7, c3 = 5.169222938345892e-11;  // (ln 2 / 1024)^n / n!
    const double d = (double)v - top, t = fma(d, by, kMagic), r = fma(d, by, kMagic - t), p = r * fma(r, fma(r, c3, c2), c1);
    const int i = __double2loint(t);
    *y = i;
    const double two = S.table[i & (kPoints - 1)], power = __hiloint2double(__double2hiint(two) + (i >> 10) * (1 << 20), __double2loint(two));
    // beside 384 the last bit is 2^-44
    const uint64_t w = (uint64_t)(__double_as_longlong(fma(power, p, power) + kBase) - __double_as_longlong(kBase));
    return w >= least ? w : 0;
  }
  __device__ __forceinline__ uint64_t weight(float v) const {
    int y;
    return weight(v, &y);
  }
  // of the draw of a token with logit v where the kept ones' W add up to `all`: by its weight unrounded, which may be a few units
  __device__ __forceinline__ float log_probability(float v, uint64_t all) const {
    constexpr double kLn2 = 0.6931471805599453;
    return (float)(((double)v - top) * by * (kLn2 / 1024) - log((double)all / (double)(1ull << kUnit)));
  }
  static __device__ __forceinline__ int bin_of(int y) { return -y >> 4; }
  // a value that every token with a bin up to this one reaches
  __device__ __forceinline__ float value_of_bin(int bin) const { return fmaxf(__double2float_rd(top - (16.0 * (bin + 1) + 1.0) / by), least_value); }

  // ---- bf16: few logits are near enough to the largest to have a weight, and every one can have a bin of its own, counted down
  // from the largest; those below 2^-7, of either sign, share one ----
  static constexpr int kTiny = 0x4400;  // its place in the order: 0x4400 logits are below, 0x4400 above
  int top_place;
  static __device__ __forceinline__ int place_of(float v) {
    const uint32_t b = __float_as_uint(v), o = (int32_t)b < 0 ? ~b >> 16 : b >> 16 | 0x8000u;
    return (int)(o >= 0xBC00u ? o - 0x77FFu : min(o, (uint32_t)kTiny));
  }
  __device__ __forceinline__ int logit_bin(float v) const { return top_place - place_of(v); }
  __device__ __forceinline__ int tiny_bin() const { return top_place - kTiny; }
  __device__ __forceinline__ float logit_of(int bin) const {
    const uint32_t c = top_place - bin, o = c > (uint32_t)kTiny ? c + 0x77FFu : c;
    return __uint_as_float((o & 0x8000u ? o & 0x7FFFu : ~o & 0xFFFFu) << 16);
  }
  __device__ __forceinline__ void make_table() const {  // with nobody looking into the bins
    const int bins = min(kBins, logit_bin(least_value) + 1);
    for (int i = threadIdx.x; i < bins; i += kThreads) S.weight_of[i] = i == tiny_bin() ? 0 : weight(value(logit_of(i)));
    __syncthreads();
  }

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

  __device__ __forceinline__ const Shared *block(int b) const { return blocks > 1 ? cg::this_cluster().map_shared_rank(&S, b) : &S; }
  __device__ __forceinline__ void sync_row() const {
    if (blocks > 1) cg::this_cluster().sync();
    else __syncthreads();
  }

  // The first bin at whose end the row's tokens so far (by_count) are `want` or more, or their sum `target` or more, and the
  // tally before it; there is such a bin.  The blocks exchange sums of runs of bins, and look into the bins of one run.
  // Between this and what writes to the bins next lies a barrier of the row's blocks.
  __device__ Tally find_bin(int n, bool by_count, uint32_t want, uint64_t target, int *bin) const {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, run = (n + kThreads - 1) / kThreads;  // at most 8
    __syncthreads();
    Tally sum = {0, 0};
    for (int i = min(n, tid * run); i < min(n, (tid + 1) * run); ++i) {
      sum.mass += ((uint64_t)S.high[i] << 32) + S.low[i];
      sum.count += S.count[i];
    }
    S.run_mass[tid] = sum.mass, S.run_count[tid] = sum.count;
    if (tid == 0) S.found = {0, 0}, S.found_run = 0, S.found_bin = 0;
    sync_row();
    if (blocks > 1) {
      sum = {0, 0};
#pragma unroll
      for (int b = 0; b < kMostBlocks; ++b) {
        if (b < blocks) sum.mass += block(b)->run_mass[tid], sum.count += block(b)->run_count[tid];
      }
    }
    Tally upto = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint64_t m = __shfl_up_sync(~0u, upto.mass, d);
      const uint32_t c = __shfl_up_sync(~0u, upto.count, d);
      if (lane >= d) upto.mass += m, upto.count += c;
    }
    if (lane == 31) S.scan_mass[warp] = upto.mass, S.scan_count[warp] = upto.count;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) upto.mass += S.scan_mass[w], upto.count += S.scan_count[w];
    }
    auto enough = [&](const Tally &t) { return by_count ? t.count >= want : t.mass >= target; };
    const Tally before = {upto.mass - sum.mass, upto.count - sum.count};
    if (enough(upto) && !enough(before)) S.found = before, S.found_run = tid;
    __syncthreads();
    if (warp == 0) {  // a bin to each of eight lanes, a block to each of four eights
      const int i = S.found_run * run + (lane & 7);
      Tally t = {0, 0};
      if ((lane & 7) < run && i < n) {
        for (int b = lane >> 3; b < blocks; b += 4) {
          const Shared *o = block(b);
          t.mass += ((uint64_t)o->high[i] << 32) + o->low[i];
          t.count += o->count[i];
        }
      }
#pragma unroll
      for (int d = 8; d < 32; d <<= 1) t.mass += __shfl_xor_sync(~0u, t.mass, d), t.count += __shfl_xor_sync(~0u, t.count, d);
      Tally at = S.found, own = t;
#pragma unroll
      for (int d = 1; d < 8; d <<= 1) {
        const uint64_t m = __shfl_up_sync(~0u, t.mass, d, 8);
        const uint32_t c = __shfl_up_sync(~0u, t.count, d, 8);
        if ((lane & 7) >= d) t.mass += m, t.count += c;
      }
      at.mass += t.mass, at.count += t.count;
      const Tally ahead = {at.mass - own.mass, at.count - own.count};
      __syncwarp();
      if (lane < 8 && enough(at) && !enough(ahead)) S.found = ahead, S.found_bin = i;
    }
    __syncthreads();
    *bin = (int)S.found_bin;
    return S.found;
  }

  // Among the tokens of a bin of y: the logit (as a key) at which `want` tokens or the sum `target` are reached, and the tally
  // before it.
  __device__ Tally refine(int bin, bool by_count, uint32_t want, uint64_t target, uint32_t *key) const {
    uint32_t lo = ~0u, hi = 0;
    each([&](float v) {
      int y;
      if (weight(v, &y) && bin_of(y) == bin) lo = min(lo, key_of(v)), hi = max(hi, key_of(v));
    });
    lo = __reduce_min_sync(~0u, lo), hi = __reduce_max_sync(~0u, hi);
    if ((threadIdx.x & 31) == 0) S.warp_least[threadIdx.x >> 5] = lo, S.warp_most[threadIdx.x >> 5] = hi;
    __syncthreads();
    lo = ~0u, hi = 0;
    for (int w = 0; w < kWarps; ++w) lo = min(lo, S.warp_least[w]), hi = max(hi, S.warp_most[w]);
    if (threadIdx.x == 0) S.block_least = lo, S.block_most = hi;
    sync_row();
    for (int b = 0; b < blocks; ++b) lo = min(lo, block(b)->block_least), hi = max(hi, block(b)->block_most);
    Tally all = {0, 0};
    for (int pass = 0; pass < 3 && lo < hi; ++pass) {  // 11 bits each
      const int down = max(0, 32 - __clz(hi - lo) - 11);  // hi - lo >> down is below kKeyBins
      if (pass) sync_row();
      clear_bins(kKeyBins);
      each([&](float v) {
        int y;
        const uint32_t k = key_of(v);
        const uint64_t w = weight(v, &y);
        if (w && bin_of(y) == bin && k >= lo && k <= hi) add((hi - k) >> down, w);
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
  for (int i = tid; i < kPoints; i += kThreads) S.table[i] = exp2((double)i / kPoints);
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

  z.listed = false;
  // ---- the largest logit ----
  float own = -INFINITY;
  z.each_of_row([&](int, float v) { own = fmaxf(own, v); });
  float best = own;
#pragma unroll
  for (int d = 16; d; d >>= 1) best = fmaxf(best, __shfl_xor_sync(~0u, best, d));
  if (lane == 0) S.warp_max[warp] = best;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWarps; ++w) best = fmaxf(best, S.warp_max[w]);
  if (P.blocks > 1) {
    if (tid == 0) S.block_max = best;
    z.sync_row();
    for (int b = 0; b < P.blocks; ++b) best = fmaxf(best, z.block(b)->block_max);
  }
  if (!(temperature > 0.0f) || best == -INFINITY) {
    int first = 0x7FFFFFFF;
    z.each_of_row([&](int i, float v) {
      if (v == best && i < first && i >= 0 && i < z.vocab) first = i;
    });
    first = __reduce_min_sync(~0u, first);
    if (lane == 0) S.warp_first[warp] = first;
    __syncthreads();
    if (tid == 0) {
      for (int w = 0; w < kWarps; ++w) first = min(first, S.warp_first[w]);
      S.block_first = first;
    }
    z.sync_row();
    if (z.rank == 0 && tid == 0) {
      for (int b = 0; b < P.blocks; ++b) first = min(first, z.block(b)->block_first);
      P.a.tokens[row] = best == -INFINITY ? -1 : first;
      if (P.a.logprobs) P.a.logprobs[row] = best == -INFINITY ? -INFINITY : 0.0f;
    }
    z.sync_row();  // nobody leaves while its shared memory is read
    return;
  }
  // ---- weights ----
  // kHottest: least_value lies above -FLT_MAX, which stands for -infinity and NaN, unless the largest logit itself is within 40 of
  // them of it (in fp32 the two next to the lowest number)
  constexpr double kHottest = 1e30;
  z.alone = best == INFINITY || best < (float)(41 * kHottest - FLT_MAX);
  z.largest = best;
  const double t = fmin((double)temperature, kHottest);
  z.top = z.alone ? 0.0f : best;
  z.by = 1024 * 1.4426950408889634 / t;
  z.least_value = fmaxf(__double2float_rd(z.top - (z.alone ? 1.0 : 40.0 * t)), -FLT_MAX);  // 2^-57.7
  if (z.least_value >= (float)z.top) z.least_value = nextafterf((float)z.top, -INFINITY);
  if (z.alone) z.by = 1024.0 * 100;
  // where the next smaller float is further away than that, y stays within what `weight` can take
  z.by = fmin(z.by, 1024.0 * 1000 / (z.top - z.least_value));
  z.least = min_p > 0.0f ? (uint64_t)ceil((double)fminf(min_p, 1.0f) * (double)(1ull << kUnit)) : 1;

  // bf16, and all logits that have a weight are among the bins
  z.top_place = Z::place_of(best);
  const bool by_logit = DT == AMAP_BF16 && !z.alone && z.logit_bin(z.least_value) < kBins;

  // ---- what is kept: tokens with a larger key than `last`, and the first `equal` of those that have it ----
  uint32_t last = 0, equal = ~0u;
  uint64_t last_weight = 0;
  const bool by_k = top_k > 0 && top_k < z.vocab, by_p = top_p < 1.0f;
  int turn = 0;
  auto total = [&](Tally all) {  // over the row's blocks
    all = z.block_sum(all);
    if (P.blocks > 1) {
      turn ^= 1;  // what is read here is not written to before the next barrier but one
      if (tid == 0) S.block_tally[turn] = all;
      z.sync_row();
      all = {0, 0};
      for (int b = 0; b < P.blocks; ++b) all.mass += z.block(b)->block_tally[turn].mass, all.count += z.block(b)->block_tally[turn].count;
    }
    return all;
  };
  if (by_k || min_p > 0.0f || (by_p && !by_logit)) {
    // a bound that is easily had
    float bound = z.least_value;
    if (min_p > 0.0f) bound = fmaxf(bound, __double2float_rd(z.top + 1024 * (log2((double)fminf(min_p, 1.0f)) - 1e-6) / z.by));
    if (by_k && top_k <= P.blocks * kThreads) {
      // the top_k-th largest of the threads' own maxima
      z.clear_bins(kBins);
      int y;
      const uint64_t w = z.weight(z.value(own), &y);
      if (w) z.add(Z::bin_of(y), w);
      if (total({w, w != 0}).count >= (uint32_t)top_k) {
        int bin;
        z.find_bin(kBins, true, top_k, 0, &bin);
        bound = fmaxf(bound, z.value_of_bin(bin));
      }
    } else if (!by_k && !(min_p > 0.0f)) {
      Tally all = {0, 0};
      z.each([&](float v) {
        const uint64_t w = z.weight(v);
        all.mass += w, all.count += w != 0;
      });
      all = total(all);
      if (tid == 0) S.total = all.mass;
      // a token that is kept last has no less than its share of what is to be left out: a thousandth less, for the roundings, and
      // half a unit, by which W may be above the weight (with less than that left there is no bound, and log2 gives a NaN)
      const double share = (1.0 - (double)fmaxf(top_p, 0.0f)) * (double)all.mass / all.count * 0.999 - 0.5;
      bound = fmaxf(bound, __double2float_rd(z.top + 1024 * (log2(fmin(share / (double)(1ull << kUnit), 1.0)) - 1e-6) / z.by));
    }
    // the tokens that reach it, in their order
    int n = 0;
    typename Z::Vector next = z.load(z.begin + lane, z.end);
#pragma unroll 1
    for (int j0 = z.begin; j0 < z.end; j0 += 32) {
      const typename Z::Vector u = next;
      next = z.load(j0 + 32 + lane, z.end);
      float v[Z::VEC];
      uint32_t mine = 0;
#pragma unroll
      for (int i = 0; i < Z::VEC; ++i) {
        v[i] = z.value(Elem<DT>::to(u.e[i]));
        mine |= (v[i] >= bound && v[i] > z.least_value ? 1u : 0u) << i;
      }
      if (!__any_sync(~0u, mine)) continue;
      const int count = __popc(mine);
      int at = count;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(~0u, at, d);
        if (lane >= d) at += o;
      }
      const int all = __shfl_sync(~0u, at, 31);
      at += n - count;
#pragma unroll
      for (int i = 0; i < Z::VEC; ++i) {
        if (!(mine >> i & 1)) continue;
        if (at < Z::kListed) z.list()[at] = {(uint16_t)((j0 - z.begin + lane) * Z::VEC + i), u.e[i]};
        ++at;
      }
      n += all;
    }
    if (lane == 0) S.warp_listed[warp] = n;
    __syncwarp();
    z.sync_row();
    // how many there are ahead of this warp's and in all, and whether every list has room
    int ahead = 0, count = 0;
    bool room = per * Z::VEC <= 65536;
    for (int w = lane; w < warps; w += 32) {
      const int c = z.block(w / kWarps)->warp_listed[w % kWarps];
      room &= c <= Z::kListed;
      count += c;
      ahead += w < z.rank * kWarps + warp ? c : 0;
    }
    room = __all_sync(~0u, room);
    count = __reduce_add_sync(~0u, count);
    ahead = __reduce_add_sync(~0u, ahead);
    z.listed = room;
    z.n_listed = n;

    if (room && count <= kSorted) {
      // ---- few: one block sorts them by key, largest first, then index ----
      Shared *home = P.blocks > 1 ? cluster.map_shared_rank(&S, 0) : &S;
      for (int i = lane; i < n; i += 32) home->order[ahead + i] = (uint64_t)key_of(z.value(Elem<DT>::to(z.list()[i].logit))) << 32 | (0xFFFFFFFFu - z.index_of(z.list()[i]));
      z.sync_row();
      if (z.rank == 0) {
        int size = 32;
        while (size < count) size *= 2;
        for (int i = count + tid; i < size; i += kThreads) S.order[i] = 0;
        auto sort = [&]() {  // bitonic, descending
          for (int run = 2; run <= size; run *= 2) {
            for (int d = run / 2; d; d /= 2) {
              __syncthreads();
              for (int i = tid; i < size / 2; i += kThreads) {
                const int lo = 2 * i - (i & (d - 1)), hi = lo + d;
                const uint64_t x = S.order[lo], y = S.order[hi];
                if ((x < y) == !(lo & run)) S.order[lo] = y, S.order[hi] = x;
              }
            }
          }
          __syncthreads();
        };
        // sums up to each: two to a thread
        auto scan = [&](uint64_t (&w)[2]) {
          uint64_t upto = w[0] + w[1];
#pragma unroll
          for (int d = 1; d < 32; d <<= 1) {
            const uint64_t o = __shfl_up_sync(~0u, upto, d);
            if (lane >= d) upto += o;
          }
          __syncthreads();
          if (lane == 31) S.scan_mass[warp] = upto;
          __syncthreads();
          uint64_t all = 0;
#pragma unroll
          for (int v = 0; v < kWarps; ++v) {
            if (v < warp) upto += S.scan_mass[v];
            all += S.scan_mass[v];
          }
          w[0] = upto - w[1];
          w[1] = upto;
          return all;
        };
        sort();
        const int most = by_k ? min(count, top_k) : count;
        uint64_t w[2], upto[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) w[i] = upto[i] = 2 * tid + i < most ? z.weight(of_key((uint32_t)(S.order[2 * tid + i] >> 32))) : 0;
        const uint64_t base = scan(upto);
        // of the whole row's, where neither top_k nor min_p leave anything out: the first pass has it (top_p alone)
        const uint64_t target = by_p ? max(share_up(fmaxf(top_p, 0.0f), by_k || min_p > 0.0f ? base : S.total), (uint64_t)1) : ~0ull;
        if (tid == 0) S.kept = 0;
        __syncthreads();
        int kept = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) kept += w[i] != 0 && upto[i] - w[i] < target;
        kept = __reduce_add_sync(~0u, kept);
        if (lane == 0) atomicAdd(&S.kept, kept);
        __syncthreads();
        kept = S.kept;
        // the kept ones, by index (largest first: the sums are taken from the other end)
        const int size_before = size;
        size = 32;
        while (size < kept) size *= 2;
        for (int i = tid; i < size_before; i += kThreads) {
          const uint64_t k = S.order[i];
          if (i < size) S.order[i] = i < kept ? k << 32 | k >> 32 : 0;
        }
        sort();
#pragma unroll
        for (int i = 0; i < 2; ++i) w[i] = upto[i] = 2 * tid + i < kept ? z.weight(of_key((uint32_t)S.order[2 * tid + i])) : 0;
        const uint64_t all = scan(upto);
        const float u = P.a.uniform[row];
        const uint64_t draw = share_of(u > 0.0f ? fminf(u, 0x1.fffffep-1f) : 0.0f, all);
        // S.order has ~index in its upper half, largest first, so the lowest index comes first
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (w[i] && draw >= upto[i] - w[i] && draw < upto[i]) {
            P.a.tokens[row] = (int32_t)(0xFFFFFFFFu - (uint32_t)(S.order[2 * tid + i] >> 32));
            if (P.a.logprobs) P.a.logprobs[row] = z.log_probability(of_key((uint32_t)S.order[2 * tid + i]), all);
          }
        }
      }
      z.sync_row();  // nobody leaves while its shared memory is read
      return;
    }
  }
  // ---- many: histograms ----
  if (by_k || by_p) {
    const bool logits = by_logit && !z.listed;
    bool found = false;
    Tally all = {0, 0};
    int bin;
    if (logits) {
      z.clear_bins(kBins);
      z.each_vector(z.begin, z.end, [&](int, const float (&x)[Z::VEC]) {
        uint32_t tiny = 0;
#pragma unroll
        for (int i = 0; i < Z::VEC; ++i) {
          const float v = z.value(x[i]);
          const int at = z.logit_bin(v);
          const bool own = at != z.tiny_bin();
          if (v > z.least_value && own) atomicAdd(&S.count[at], 1u);
          tiny |= own ? 0u : 1u << i;
        }
        if (tiny) {
#pragma unroll
          for (int i = 0; i < Z::VEC; ++i) {
            const uint64_t w = tiny >> i & 1 ? z.weight(z.value(x[i])) : 0;
            if (w) z.add(z.tiny_bin(), w);
          }
        }
      });
      __syncthreads();
      for (int i = tid; i < kBins; i += kThreads) {
        const uint64_t w = z.weight(z.value(z.logit_of(i))), m = w * S.count[i];
        if (i != z.tiny_bin()) {
          if (!w) S.count[i] = 0;
          S.low[i] = (uint32_t)m, S.high[i] = (uint32_t)(m >> 32);
        }
        all.mass += ((uint64_t)S.high[i] << 32) + S.low[i], all.count += S.count[i];
      }
      all = total(all);
      found = true;
      uint64_t base = all.mass;
      auto settle = [&](bool by_count, uint32_t want, uint64_t target) {  // last and equal; what is ahead of them
        const Tally t = z.find_bin(kBins, by_count, want, target, &bin);
        found = found && bin != z.tiny_bin();
        if (!found) return t;
        const float v = z.logit_of(bin);
        last = key_of(v);
        last_weight = z.weight(v);
        equal = by_count ? want - t.count : (uint32_t)((target - t.mass + last_weight - 1) / max(last_weight, (uint64_t)1));
        return t;
      };
      if (by_k && (uint32_t)top_k < all.count) {
        const Tally t = settle(true, top_k, 0);
        base = t.mass + equal * last_weight;
      }
      if (by_p && found) {
        z.sync_row();
        settle(false, 0, max(share_up(fmaxf(top_p, 0.0f), base), (uint64_t)1));
      }
      if (!found) {  // a bound falls among the logits that share a bin
        z.sync_row();
        last = 0, equal = ~0u, last_weight = 0, all = {0, 0};
      }
    }
    if (!found) {
      z.clear_bins(kBins);  // a barrier of the row's blocks lies behind what looked into them last
      auto tally = [&](uint32_t from) {
        z.each([&](float v) {
          int y;
          const uint64_t w = z.weight(v, &y);
          if (!w || key_of(v) < from) return;
          z.add(Z::bin_of(y), w);
          all.mass += w, ++all.count;
        });
      };
      tally(0);
      all = total(all);
      uint64_t base = by_k || min_p > 0.0f || by_logit ? all.mass : S.total;  // what top_p is a part of
      const bool cut = by_k && (uint32_t)top_k < all.count;
      if (cut) {
        const Tally k = z.find_bin(kBins, true, top_k, 0, &bin);
        const Tally in = z.refine(bin, true, top_k - k.count, 0, &last);
        last_weight = z.weight(of_key(last));
        equal = top_k - k.count - in.count;
        base = k.mass + in.mass + equal * last_weight;
      }
      if (by_p) {
        const uint64_t target = max(share_up(fmaxf(top_p, 0.0f), base), (uint64_t)1);
        if (cut) {  // refining has written over the histogram
          z.sync_row();
          z.clear_bins(kBins);
          tally(last);
        }
        const Tally p = z.find_bin(kBins, false, 0, target, &bin);
        const Tally in = z.refine(bin, false, 0, target - p.mass, &last);
        last_weight = z.weight(of_key(last));
        equal = (uint32_t)((target - p.mass - in.mass + last_weight - 1) / max(last_weight, (uint64_t)1));
      }
    }
  }

  // ---- the draw ----
  const bool by_table = by_logit && !z.listed;
  if (by_table) {
    if (by_k || by_p) z.sync_row();  // the table comes to lie over the bins
    z.make_table();
  }
  uint64_t mass = 0;
  uint32_t same = 0;
  // least_value has no weight, though the 16-bit logit whose bin it is in may have one (below zero a bin's logit is its upper end)
  const float last_value = last ? of_key(last) : z.least_value;
  auto weigh = [&](float v) {
    const uint64_t w = z.weight(v);
    mass += v > last_value ? w : 0;
    same += v == last_value;
  };
  auto weigh_vectors = [&](int from, int until) {
    z.each_vector(from, until, [&](int, const float (&x)[Z::VEC]) {
      if (!by_table) {
#pragma unroll
        for (int i = 0; i < Z::VEC; ++i) weigh(z.value(x[i]));
        return;
      }
      uint32_t tiny = 0;
#pragma unroll
      for (int i = 0; i < Z::VEC; ++i) {
        const float v = z.value(x[i]);
        const int at = z.logit_bin(v);
        const bool own = at != z.tiny_bin();
        if (v > last_value && own) mass += S.weight_of[at];
        same += v == last_value;
        tiny |= own || !(v > last_value) ? 0u : 1u << i;
      }
      if (tiny) {
#pragma unroll
        for (int i = 0; i < Z::VEC; ++i) mass += tiny >> i & 1 ? z.weight(z.value(x[i])) : 0;
      }
    });
  };
  auto over_warp = [&]() {
#pragma unroll
    for (int d = 16; d; d >>= 1) mass += __shfl_xor_sync(~0u, mass, d);
    same = __reduce_add_sync(~0u, same);
  };
  if (z.listed) z.each(weigh);
  else weigh_vectors(z.begin, z.end);
  over_warp();
  if (lane == 0) S.warp_mass[warp] = mass, S.warp_equal[warp] = same;
  z.sync_row();
  if (tid < warps) {
    const Shared *o = z.block(tid / kWarps);
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
  if (S.pick_warp / kWarps == z.rank) {
    // the run of that warp, a part of it to each warp; a list is short enough for one
    uint64_t target = S.pick_before, before = 0;
    const uint64_t all = S.all_mass[0];
    uint32_t seen = S.pick_equal;
    int from = 0, until = 0, chosen = S.pick_warp % kWarps;
    if (!z.listed) {
      const int run = min(vectors, S.pick_warp * per), end = min(vectors, run + per), part = (per / 32 + kWarps - 1) / kWarps * 32;
      mass = 0, same = 0;
      weigh_vectors(min(end, run + warp * part), min(end, run + (warp + 1) * part));
      over_warp();
      if (lane == 0) S.scan_mass[warp] = mass, S.scan_count[warp] = same;
      __syncthreads();
      for (chosen = 0; chosen + 1 < kWarps; ++chosen) {
        const uint64_t m = S.scan_mass[chosen] + last_weight * (uint64_t)min(S.scan_count[chosen], equal - min(equal, seen));
        if (target < before + m) break;
        before += m;
        seen += S.scan_count[chosen];
      }
      from = min(end, run + chosen * part), until = min(end, run + (chosen + 1) * part);
    }
    if (warp == chosen) {
    // N tokens of each lane, in order: those of a vector, or one of the list
    auto go = [&](auto width, int from, int to, auto get, auto index) {
      constexpr int N = decltype(width)::value;
      for (int j0 = from; j0 < to; j0 += 32) {
        float v[N];
        get(j0 + lane, v);
        uint32_t equals = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) equals += key_of(v[i]) == last;
        uint32_t rank = equals;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const uint32_t o = __shfl_up_sync(~0u, rank, d);
          if (lane >= d) rank += o;
        }
        const uint32_t row_equals = __shfl_sync(~0u, rank, 31);
        rank += seen - equals;
        uint64_t w[N], sum = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const uint32_t k = key_of(v[i]);
          w[i] = k > last ? z.weight(v[i]) : k == last && rank++ < equal ? last_weight : 0;
          sum += w[i];
        }
        uint64_t upto = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const uint64_t o = __shfl_up_sync(~0u, upto, d);
          if (lane >= d) upto += o;
        }
        const uint64_t step = __shfl_sync(~0u, upto, 31);
        upto += before;
        if (target < before + step) {
          if (target < upto && target >= upto - sum) {
            uint64_t at = upto - sum;
#pragma unroll
            for (int i = 0; i < N; ++i) {
              if (target >= at && target < at + w[i]) {
                P.a.tokens[row] = index(j0 + lane, i);
                if (P.a.logprobs) P.a.logprobs[row] = z.log_probability(v[i], all);
              }
              at += w[i];
            }
          }
          return;
        }
        before += step;
        seen += row_equals;
      }
    };
    if (z.listed) {
      go(std::integral_constant<int, 1>(), 0, z.n_listed, [&](int j, float (&v)[1]) { v[0] = j < z.n_listed ? z.value(Elem<DT>::to(z.list()[j].logit)) : z.least_value; },
         [&](int j, int) { return z.index_of(z.list()[j]); });
    } else {
      go(std::integral_constant<int, Z::VEC>(), from, until,
         [&](int j, float (&v)[Z::VEC]) {
           const typename Z::Vector u = z.load(j, until);
#pragma unroll
           for (int i = 0; i < Z::VEC; ++i) v[i] = z.value(Elem<DT>::to(u.e[i]));
         },
         [&](int j, int i) { return j * Z::VEC - z.shift + i; });
    }
    }
  }
  z.sync_row();  // nobody leaves while its shared memory is read
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
  SERVE_REQUIRE(a->vocab >= 1 && a->vocab <= 1 << 19, AMAP_EINVAL, "vocab: 1 .. 2^19");
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
  // blocks of a row: as many as fill the device twice over, but none with less than a vector of 16 bytes a thread.  More rows
  // than multiprocessors that have settings of their own differ in work, and get twice as many, to even out (256 x 150001
  // bf16, settings mixed: 154 -> 130 us; all alike, 40 largest of 150001: 60 -> 80)
  const int64_t vectors = (int64_t)a->vocab * dtype_bytes(a->dtype) / 16, sms = device_sms();
  const int64_t most = (a->rows > sms && a->by_row ? 4 : 2) * sms;
  P.blocks = 1;
  while (P.blocks < kMostBlocks && (int64_t)a->rows * P.blocks * 2 <= most && vectors >= P.blocks * 2 * kThreads) P.blocks *= 2;
  switch (a->dtype) {
    case AMAP_BF16: return run<AMAP_BF16>(P, cuda_stream);
    case AMAP_FP16: return run<AMAP_FP16>(P, cuda_stream);
    default: return run<AMAP_FP32>(P, cuda_stream);
  }
}
