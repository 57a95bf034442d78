// sample.cuh -- one token per row of logits after temperature, top-k, top-p and min-p, drawn with the
// caller's uniform (the target's side of section 3.1 when it decodes with these filters).
//
// Mathematics.  With z = x / T and the ids ordered by (z descending, id ascending): the first k stay;
// of those, the ones whose predecessors in that order hold less than p of the mass; of those, the ones
// with exp(z - max z) >= min_p; the first always.  The token is the first kept id, in id order, whose
// cumulative mass exceeds u times the kept mass.
//
// Weights are integers: 2^44 exp(z - max z), rounded.  At most 2^19 of them fit 63 bits, so their sums are
// exact and the same in any order: splitting a row over CTAs, atomics and the order of threads change
// nothing.  A weight above 2^-11 of the greatest is computed to about 2^-38 of its value (fine_weight()),
// one below in fp32.  (z, id) is one 64-bit integer (order_of()), so every cut is a bound on it.  Under
// top-p the mass of the ids that cannot stay is added up in fp32, a thread's share at a time.
//
// A cluster of CTAs takes a row, a slice each.  Bound by DRAM for many rows (one read of the logits), by the
// chain of exchanges for few.
//   Sampled pass (rows that a filter thins out, vocabularies of some ten thousand ids on).  A few units of 16
//   bytes a thread, spread over the slice, give a value above which the ids that can stay should lie: under
//   top-k the sample's value of a rank a little above its share of k; under top-p where the sample's mass below
//   is a part of what may be left out, by half octaves of weight; under min-p its definition.  The row is then
//   read once: the ids above go to the first CTA, and under top-p the mass below is added up, which tells
//   whether the guess held; if not, it is lowered by what that pass found, once.
//   Two passes (short vocabularies, guesses that failed).  The row maximum and a safe bound from the maxima of
//   groups of elements: under top-k where every CTA has k / SP groups that reach a value; under top-p where V
//   ids of its weight would carry less than 1 - p of what the maxima carry, or, first, a nearer one that the
//   pass checks.  The second read comes from L2: what is in flight on the chip (at V = 151936, fp32, 46 MB with eight
//   CTAs a row, 92 MB with four) fits it, and a re-read of such slices ran at 11 TB/s against 7 from DRAM; holding
//   them in shared memory left two CTAs an SM, waiting for each other (512 rows with top-p: 249 us against 173).
//   The first CTA sorts up to kSort candidates by preference, scans their weights, sorts what stays by id and
//   draws, while the others have left (one row 2.7 us, against 7.4 for radix selections over the list); more of
//   them it thins out by bins of value first.
//   More candidates than kListCap under top-p: their weights are added up by value in kBins bins over the
//   cluster, and the candidates down to the bin that holds the border are gathered, or those in it, which decide
//   it.  What else leaves too many is cut by a radix selection over the whole row.  Then, and without any
//   filter, the cluster scans the kept weights in id order.
// What it measured (device time): V = 151936, one fp32 row with top-k and top-p 12.0 us; 512 fp32 rows with top-k 80
// us, 3.9 TB/s, with min-p 81, with top-p 120; 1088 bf16 rows with top-k and top-p 107 us, 3.1 TB/s; temperature
// alone, which reads the row twice and weighs every element, 64 fp32 rows 38 us, 512 of them 199.  For many rows the
// waves of CTAs end unevenly (3.4 of them at 512 rows) and the first CTA's 6 us stay; more CTAs an SM (48 and 40
// registers) gave 77 and 81 us for the first.
// One translation unit an element type (sample_f32.cu, sample_bf16.cu, sample_f16.cu); sample.cu dispatches.
#pragma once

#include <math.h>

#include "kernels.h"
#include "rows.cuh"

namespace dm {

constexpr int kDrawThreads = 256;   // threads of a CTA
constexpr int kWarps = kDrawThreads / 32;
constexpr int kDrawBatch = 4;       // 16-byte loads a thread has in flight
constexpr int kLocalCap = 2048;     // candidates a CTA holds, a segment of them a warp
constexpr int kSeg = kLocalCap / kWarps;
constexpr int kListCap = 3040;      // candidates the cluster's first CTA can take
constexpr int kMaxSliceBytes = 256 << 10;  // the launch's rule: 524288 fp32 ids over eight CTAs, and no more by any halving
constexpr int kMaxSteps = ((kMaxSliceBytes / 16 + 1 + kWarps - 1) / kWarps + 31) / 32;  // of 32 units, a warp's of a slice
constexpr int kBins = 512;          // of values, or of ids
constexpr int kSubCap = 256;        // entries of one bin that are ranked against each other
constexpr int kSort = 512;          // entries that are sorted, two a thread
constexpr int kSlots = 256;         // half octaves of weight on a grid of its own
constexpr int kOctaves = 64;        // half octaves of weight in which the groups' maxima are added up
constexpr int kWeightBits = 44;     // the greatest weight is 2^44
constexpr float kNoWeight = -45.f;  // log2 of a relative weight that rounds to nothing
constexpr float kCoarse = -11.f;    // below this (log2) a weight is computed in fp32

using u64 = unsigned long long;

// 2^44 * 2^(i/32), rounded, i = 0..31.
__constant__ u64 c_pow2[32] = {
    0x100000000000ull, 0x1059b0d31585ull, 0x10b5586cf989ull, 0x111301d0125bull, 0x1172b83c7d51ull, 0x11d4873168baull,
    0x12387a6e7562ull, 0x129e9df51fdfull, 0x1306fe0a31b7ull, 0x1371a7373aaaull, 0x13dea64c1234ull, 0x144e08606189ull,
    0x14bfdad5362aull, 0x15342b569d50ull, 0x15ab07dd4854ull, 0x16247eb03a56ull, 0x16a09e667f3cull, 0x171f75e8ec5full,
    0x17a11473eb02ull, 0x182589994cceull, 0x18ace5422aa1ull, 0x193737b0cdc6ull, 0x19c49182a3f1ull, 0x1a5503b23e25ull,
    0x1ae89f995ad4ull, 0x1b7f76f2fb5eull, 0x1c199bdd8553ull, 0x1cb720dcef90ull, 0x1d5818dcfba5ull, 0x1dfc97337b9bull,
    0x1ea4afa2a491ull, 0x1f50765b6e45ull};

// What the weights of a row depend on: the row maximum and log2(e) / T as a sum of two floats.
struct Scale {
  float m, k_hi, k_lo;
  bool inf;  // the maximum is +inf: all mass on the ids that share it
};

// round(2^44 exp((x - m) / T)); 0 for NaN and -inf.  t = (x - m) log2(e) / T is carried as a sum of two
// floats (x - m exactly, by Knuth's two-sum), split into an integer, a multiple of 1/32 looked up in
// `pow2`, and a remainder |r| <= 1/64 whose 2^r - 1 is the Taylor sum of exp(r ln 2), its first term
// again in two floats; the product is formed in integers.
static __device__ __noinline__ u64 fine_weight(float x, float m, float k_hi, float k_lo, const u64* pow2) {
  const float d = x - m;
  const float t = d * k_hi;
  // x - m = d + d_lo
  const float xv = d + m;
  const float mv = d - xv;
  const float d_lo = (x - xv) + (-m - mv);
  const float t_lo = fmaf(d, k_hi, -t) + fmaf(d, k_lo, d_lo * k_hi);
  const int j = __float2int_rn(t * 32.f);
  const float r = fmaf(static_cast<float>(j), -1.f / 32.f, t);
  constexpr float kLn2Hi = 0.693147182f, kLn2Lo = -1.90465430e-9f;
  const float p = r * kLn2Hi;
  const float p_lo = fmaf(r, kLn2Hi, -p) + fmaf(r, kLn2Lo, t_lo * kLn2Hi);
  const float y = p + p_lo;
  const float q = fmaf(y * y, fmaf(y, fmaf(y, fmaf(y, 1.f / 120.f, 1.f / 24.f), 1.f / 6.f), 0.5f), p_lo);
  constexpr float kFix = 137438953472.f;  // 2^37
  const int s = __float2int_rn(p * kFix) + __float2int_rn(q * kFix);
  const u64 base = pow2[j & 31];
  const long long add = static_cast<long long>(base >> 13) * s;
  const u64 v = base + static_cast<u64>(add >> 24);
  const int n = -(j >> 5);
  return (v + ((1ull << n) >> 1)) >> n;
}

__device__ __forceinline__ u64 weight(float x, const Scale& sc, const u64* pow2) {
  if (sc.inf) return x == sc.m ? 1ull << kWeightBits : 0ull;
  const float t = (x - sc.m) * sc.k_hi;
  if (!(t >= kNoWeight)) return 0ull;
  // below 2^33: 32 bits and a doubling
  if (t < kCoarse) return static_cast<u64>(__float2uint_rn(ex2(t + static_cast<float>(kWeightBits - 1)))) << 1;
  return fine_weight(x, sc.m, sc.k_hi, sc.k_lo, pow2);
}

// log(w / all) of the element x, whose weight w is.  More than half of the mass: by what the others have, so that a
// log-probability near 0 is good to its own size; less: by the logit, of which more digits are there than of a small weight.
static __device__ __noinline__ float log_prob(float x, u64 w, u64 all, const Scale& sc, float temp) {
  const u64 others = all - w;
  if (w > others) return -log1pf(static_cast<float>(others) / static_cast<float>(w));
  return (sc.inf ? 0.f : (x - sc.m) / temp) - logf(static_cast<float>(all) * 0x1p-44f);
}

// The order of preference as integers: greater value, greater key (-0 as +0, NaN last); equal values: the lower id.
__device__ __forceinline__ uint32_t value_key(float x) { return x != x ? 0u : f32_ord(x + 0.f); }
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ u64 order_of(uint32_t key, uint32_t id) { return (static_cast<u64>(key) << 32) | (~id); }
__device__ __forceinline__ u64 order_of(float x, uint32_t id) { return order_of(value_key(x), id); }

// The bin of a value at most `top`, counted from there down; monotone, and in range whatever is rounded.
__device__ __forceinline__ int value_bin(float x, float top, float scale) {
  return min(max(static_cast<int>((top - x) * scale), 0), kBins - 1);
}

struct Settings {
  float temp, top_p, u;
  int top_k;
  bool use_k, use_p, use_m;
};

struct DrawShared {  // dynamic shared memory
  union {
    uint2 local[kLocalCap];  // this CTA's candidates (value, id), a segment a warp; later, in the first CTA, those
                             // of the list that are left
    struct {                // the radix selection, which has no candidates
      u64 digit[2][256];    // a round's histogram, by round parity (read by the cluster)
      u64 total[256];
    };
  };
  union {
    uint2 list[kListCap];   // the first CTA: the cluster's candidates
    u64 step[kWarps * kMaxSteps];  // the totals of the slice's steps, a share of them a warp
  };
  union {
    struct {                // what is sorted, its weights and values
      u64 sort[kSort], sort_amount[kSort];
      float value[kSort];
    };
    struct {
      uint4 bins[kBins];    // count and weights (three limbs of 15 bits) by value or id
      u64 sub_order[kSubCap], sub_amount[kSubCap];  // the entries of a bin
    };
  };
  u64 pow2[32];
  u64 scan[kWarps];
  u64 sum;                // kept mass of this CTA (read by the cluster)
  u64 tail[5], mass[5];   // the first CTA: mass of the ids that are no candidates, and of those that are, by gathering
  u64 need, result, below;
  u64 cut;                // the first CTA: the border of top-p (read by the cluster)
  double floor;           // T log(min_p)
  float group[256];       // maxima of groups of threads
  uint32_t octave[kOctaves];  // the threads' maxima's mass by half octaves of weight (read by the cluster)
  float red[kWarps], red2[kWarps];
  float max, aux;         // this CTA's maximum, and its part of the candidates' bound (read by the cluster)
  float k_hi, k_lo;
  float m, top, tau, guess, below_guess, lowest;  // lowest: the least value that min-p keeps
  uint32_t key;
  int n_warp[kWarps];  // entries of the warps' segments of local; more than a segment: not all are there
  uint32_t n_list[6];     // the first CTA: the cluster's candidates, by gathering
  float best[8 * kWarps]; // the greatest values of every warp's sample (read by the cluster)
  uint32_t slot[kSlots];  // the sample's mass by half octaves (read by the cluster)
  int n_sub, bin, n_upto, n_in, by_min_p;
};

// A row's slice: ids [lo, lo + len), read in units of 16 bytes aligned in global memory.  Whole units are one load;
// the first and the last unit, which may hold what is not the row's, are read element by element.
template <typename T>
struct Slice {
  static constexpr int N = Vec<T>::kN;

  const T* src;
  int lo, len, shift, units, first, last;
  __device__ __forceinline__ Slice(const T* row, int from, int n) : src(row + from), lo(from), len(n) {
    shift = row_shift(src);
    units = row_units<T>(shift, len);
    first = shift ? 1 : 0;
    last = (shift + len) / N;
  }
  __device__ __forceinline__ Vec<T> load(int q) const {
    Vec<T> f;
    if (q >= first && q < last) {
      f.raw = __ldcg(reinterpret_cast<const uint4*>(src + (q * N - shift)));
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int at = q * N + i - shift;
        if (at >= 0 && at < len) f.e[i] = src[at];
        else from_f32(-INFINITY, &f.e[i]);
      }
    }
    return f;
  }
  __device__ __forceinline__ bool holds(int q, int i) const {
    const int at = q * N + i - shift;
    return at >= 0 && at < len;
  }
  __device__ __forceinline__ uint32_t id(int q, int i) const { return static_cast<uint32_t>(lo + q * N + i - shift); }
  // f(unit, its index) for every unit, by whole warps (lanes past the end: -inf, and an index that holds nothing),
  // kDrawBatch loads of a thread at a time
  template <typename F>
  __device__ __forceinline__ void each(F&& f) const {
    const int lane = threadIdx.x & 31;
    const uint4* unit = reinterpret_cast<const uint4*>(src - shift);
    Vec<T> none;
#pragma unroll
    for (int i = 0; i < N; ++i) from_f32(-INFINITY, &none.e[i]);
    int q0 = first + static_cast<int>(threadIdx.x) - lane;
    Vec<T> v[kDrawBatch];
    for (; q0 + (kDrawBatch - 1) * kDrawThreads + 31 < last; q0 += kDrawBatch * kDrawThreads) {
#pragma unroll
      for (int j = 0; j < kDrawBatch; ++j) v[j].raw = __ldcg(unit + (q0 + lane) + j * kDrawThreads);
#pragma unroll
      for (int j = 0; j < kDrawBatch; ++j) f(v[j], q0 + lane + j * kDrawThreads);
    }
    if (q0 < last) {
#pragma unroll
      for (int j = 0; j < kDrawBatch; ++j) {
        v[j] = none;
        if (q0 + lane + j * kDrawThreads < last) v[j].raw = __ldcg(unit + (q0 + lane) + j * kDrawThreads);
      }
#pragma unroll
      for (int j = 0; j < kDrawBatch; ++j)
        if (q0 + j * kDrawThreads < last) f(v[j], q0 + lane + j * kDrawThreads < last ? q0 + lane + j * kDrawThreads : units);
    }
    if (threadIdx.x < 32 && (first || units > last)) {  // the two units that are not whole
      const int q = lane == 0 && first ? 0 : (lane == 1 && units > last && last >= first ? last : units);
      f(q < units ? load(q) : none, q);
    }
  }
  // the units of this warp's share of the slice, in id order: [*q0, *q1)
  __device__ __forceinline__ void warp_share(int* q0, int* q1) const {
    const int per = (units + kWarps - 1) / kWarps;
    *q0 = min(units, static_cast<int>(threadIdx.x >> 5) * per);
    *q1 = min(units, *q0 + per);
  }
};

// floor(f * all), or the ceiling, for 0 <= f < 1 (f's bits below 2^-64 are dropped)
__device__ __forceinline__ u64 share_of(float f, u64 all, bool up) {
  const uint32_t b = __float_as_uint(f);
  const int e = static_cast<int>(b >> 23);  // f = (mantissa) 2^(e - 150)
  const u64 mant = e ? (b & 0x7fffffu) | 0x800000u : 0u;
  const int by = e - 150 + 64;
  const u64 f64 = by >= 0 ? mant << by : (by > -64 ? mant >> -by : 0);
  return __umul64hi(f64, all) + (up && f64 * all != 0);
}

// A lower bound (16 bits of the key) on the j-th greatest of the warp's 32 * PER values.
template <int PER>
__device__ __forceinline__ float jth_greatest(const float (&v)[PER], int j) {
  uint32_t key[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) key[i] = value_key(v[i]) >> 16;
  uint32_t prefix = 0;
  for (int bit = 15; bit >= 0; --bit) {
    const uint32_t c = prefix | (1u << bit);
    int n = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) n += __popc(__ballot_sync(0xffffffffu, key[i] >= c));
    if (n >= j) prefix = c;
  }
  return prefix <= 0x7fu ? -INFINITY : key_value(prefix << 16);  // keys up to 0x7fffff: -inf and NaN
}

__device__ __forceinline__ void add_to_bin(uint4* bin, u64 w) {
  atomicAdd(&bin->x, 1u);
  atomicAdd(&bin->y, static_cast<uint32_t>(w) & 0x7fffu);
  atomicAdd(&bin->z, static_cast<uint32_t>(w >> 15) & 0x7fffu);
  atomicAdd(&bin->w, static_cast<uint32_t>(w >> 30));
}
__device__ __forceinline__ u64 bin_mass(const uint4& b) {
  return static_cast<u64>(b.y) + (static_cast<u64>(b.z) << 15) + (static_cast<u64>(b.w) << 30);
}

__device__ __forceinline__ u64 block_total(u64 v, DrawShared& sh) {
  u64 all;
  __syncthreads();
  block_scan<u64, kDrawThreads>(v, sh.scan, threadIdx.x, &all);
  return all;
}

// ------------------------------------------------------------------ the first CTA: searches over its list
// The entry at which the amounts (1, or the weights) of the list's entries, from the first in the order on, reach
// `need`: its order.  Entries below `cut` do not count; the order is that of preference, or that of ids.
struct ListView {
  const uint2* list;
  int n;
  u64 cut;
  const Scale& sc;
  const u64* pow2;
  __device__ __forceinline__ bool entry(int e, bool weighted, bool by_id, u64* order, u64* amount) const {
    const uint2 v = list[e];
    const u64 o = order_of(__uint_as_float(v.x), v.y);
    if (o < cut) return false;
    *order = by_id ? static_cast<u64>(~v.y) : o;
    *amount = weighted ? weight(__uint_as_float(v.x), sc, pow2) : 1ull;
    return true;
  }
};

template <bool WEIGHTED, bool BY_ID>
__device__ u64 find_border(const ListView& l, u64 need, float top, float scale, uint32_t id_width, DrawShared& sh) {
  const int tid = threadIdx.x;
  u64 o = 0, a = 0;
  __syncthreads();
  if (tid == 0) sh.n_sub = 0;
  for (int i = tid; i < kBins; i += kDrawThreads) sh.bins[i] = make_uint4(0, 0, 0, 0);
  __syncthreads();
  auto bin_of = [&](int e) {
    const uint2 v = l.list[e];
    return BY_ID ? static_cast<int>(v.y / id_width) : value_bin(__uint_as_float(v.x), top, scale);
  };
  for (int e = tid; e < l.n; e += kDrawThreads)
    if (l.entry(e, WEIGHTED, BY_ID, &o, &a)) {
      if (WEIGHTED) add_to_bin(&sh.bins[bin_of(e)], a);
      else atomicAdd(&sh.bins[bin_of(e)].y, 1u);
    }
  __syncthreads();
  constexpr int kPer = kBins / kDrawThreads;
  u64 mine[kPer], sum = 0, all;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    mine[i] = bin_mass(sh.bins[tid * kPer + i]);
    sum += mine[i];
  }
  u64 before = block_scan<u64, kDrawThreads>(sum, sh.scan, tid, &all) - sum;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (before < need && need <= before + mine[i]) {
      sh.bin = tid * kPer + i;
      sh.need = need - before;
    }
    before += mine[i];
  }
  __syncthreads();
  const int bin = sh.bin;
  for (int e = tid; e < l.n; e += kDrawThreads)
    if (bin_of(e) == bin && l.entry(e, WEIGHTED, BY_ID, &o, &a)) {
      const int at = atomicAdd(&sh.n_sub, 1);
      if (at < kSubCap) {
        sh.sub_order[at] = o;
        sh.sub_amount[at] = a;
      }
    }
  __syncthreads();
  const int c = sh.n_sub;
  if (c <= kSubCap) {  // each against each
    const u64 want = sh.need;
    const bool pairs = c <= kDrawThreads / 2;  // two threads an entry
    const int e = pairs ? tid >> 1 : tid;
    o = e < c ? sh.sub_order[e] : ~0ull;
    u64 before = 0;
#pragma unroll 4
    for (int j = pairs ? tid & 1 : 0; j < c; j += pairs ? 2 : 1) {
      const u64 oj = sh.sub_order[j], a = sh.sub_amount[j];
      before += oj > o ? a : 0ull;
    }
    if (pairs) before += __shfl_xor_sync(0xffffffffu, before, 1);
    if (e < c && before < want && want <= before + sh.sub_amount[e]) sh.result = o;
  } else {  // hundreds of equal values: one bit of the order at a time, the greatest order from which on the amounts reach `need`
    u64 prefix = 0;
    for (int bit = BY_ID ? 31 : 63; bit >= 0; --bit) {
      const u64 c2 = prefix | (1ull << bit);
      u64 sum = 0;
      for (int i = tid; i < l.n; i += kDrawThreads)
        if (l.entry(i, WEIGHTED, BY_ID, &o, &a) && o >= c2) sum += a;
      if (block_total(sum, sh) >= need) prefix = c2;
    }
    if (tid == 0) sh.result = prefix;
  }
  __syncthreads();
  return sh.result;
}

// Sorts np2 (a power of two, at most kSort) integers, descending, thread t holding elements 2 t and 2 t + 1 before and
// after: bitonic, steps of 64 and more through shared memory.
__device__ __forceinline__ void sort_pairs(u64& a, u64& b, int np2, u64* s) {
  const int tid = threadIdx.x;
  for (int size = 2; size <= np2; size *= 2) {
    const bool up = (2 * tid & size) == 0;  // this run: descending
    for (int stride = size / 2; stride >= 64; stride /= 2) {
      __syncthreads();
      if (2 * tid < np2) reinterpret_cast<ulonglong2*>(s)[tid] = make_ulonglong2(a, b);
      __syncthreads();
      if (2 * tid < np2) {
        const ulonglong2 o = reinterpret_cast<const ulonglong2*>(s)[tid ^ (stride / 2)];
        const bool low = (2 * tid & stride) == 0;  // this element is the pair's first
        a = (low == up) == (o.x > a) ? o.x : a;
        b = (low == up) == (o.y > b) ? o.y : b;
      }
    }
    if (2 * tid < np2) {  // whole warps: np2 >= 64
      for (int stride = min(size / 2, 32); stride >= 2; stride /= 2) {
        const u64 x = __shfl_xor_sync(0xffffffffu, a, stride / 2), y = __shfl_xor_sync(0xffffffffu, b, stride / 2);
        const bool low = (2 * tid & stride) == 0;
        a = (low == up) == (x > a) ? x : a;
        b = (low == up) == (y > b) ? y : b;
      }
      if ((a < b) == up) {
        const u64 t = a;
        a = b;
        b = t;
      }
    }
  }
}

// floor(mass * w / 2^44), w at most 2^44.
__device__ __forceinline__ u64 rescaled(u64 mass, u64 w) {
  return w >> kWeightBits ? mass : __umul64hi(mass, w << (64 - kWeightBits));
}

// The mass that top-p asks for, of what is there.
__device__ __forceinline__ u64 top_p_need(const Settings& set, u64 all) {
  return set.top_p > 0.f ? max(share_of(set.top_p, all, true), 1ull) : 1ull;
}

// The end of a row with at most kSort candidates: sorted by preference, and what stays of them by id.  `need`: the mass
// that top-p asks for, 0 where it goes by what top-k leaves and `tail`, which is relative to sc.m.  The list holds the
// row's maximum, which sc.m need not be.
__device__ __forceinline__ void finish_sorted(const uint2* list, int n, u64 need, u64 tail, const Settings& set, Scale sc,
                                              DrawShared& sh, int32_t* token, float* logp) {
  const int tid = threadIdx.x;
  int np2 = 64;
  while (np2 < n) np2 *= 2;
  u64 o[2], w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int e = 2 * tid + i;
    o[i] = 0;  // behind every candidate
    if (e < n) o[i] = order_of(__uint_as_float(list[e].x), list[e].y);
  }
  sort_pairs(o[0], o[1], np2, sh.sort);
  __syncthreads();
  if (tid == 0) {
    const float top = key_value(static_cast<uint32_t>(o[0] >> 32));
    sh.top = top;
    if (set.use_m) sh.lowest = top == INFINITY ? INFINITY : __double2float_ru(top + sh.floor);
  }
  __syncthreads();
  const float was = sc.m;
  sc.m = sh.top;
  sc.inf = sc.m == INFINITY;
  if (tail && was != sc.m) tail = rescaled(tail, weight(was, sc, sh.pow2));
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int e = 2 * tid + i;  // its rank
    w[i] = 0;
    if (e < n && !(set.use_k && e >= set.top_k)) w[i] = weight(key_value(static_cast<uint32_t>(o[i] >> 32)), sc, sh.pow2);
  }
  u64 all;
  __syncthreads();
  const u64 before = block_scan<u64, kDrawThreads>(w[0] + w[1], sh.scan, tid, &all) - w[0] - w[1];
  if (set.use_p) {
    if (need == 0) need = top_p_need(set, all + tail);
    if (before + w[0] >= need) w[1] = 0;
    if (before >= need) w[0] = 0;
  }
  if (set.use_m) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (!(key_value(static_cast<uint32_t>(o[i] >> 32)) >= sh.lowest)) w[i] = 0;
  }
  // by id: the kept entries first, lowest id first, each with its rank
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int e = 2 * tid + i;
    sh.sort_amount[e] = w[i];
    sh.value[e] = key_value(static_cast<uint32_t>(o[i] >> 32));
    o[i] = w[i] ? (o[i] << 32) | static_cast<uint32_t>(e) : 0ull;  // the order's low half is ~id
  }
  // (what stays stands first: the second sort takes no more of it)
  const int kept = __syncthreads_count(w[0] != 0) + __syncthreads_count(w[1] != 0);
  while (np2 > 64 && np2 / 2 >= kept) np2 /= 2;
  sort_pairs(o[0], o[1], np2, sh.sort);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) w[i] = o[i] ? sh.sort_amount[static_cast<uint32_t>(o[i])] : 0ull;
  u64 at = block_scan<u64, kDrawThreads>(w[0] + w[1], sh.scan, tid, &all) - w[0] - w[1];
  const u64 goal = share_of(set.u, all, false);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (at <= goal && goal < at + w[i]) {
      const uint32_t y = ~static_cast<uint32_t>(o[i] >> 32);
      *token = static_cast<int32_t>(y);
      if (logp) *logp = log_prob(sh.value[static_cast<uint32_t>(o[i])], w[i], all, sc, set.temp);
    }
    at += w[i];
  }
}

// The end of a row in the cluster's first CTA: n candidates, every id that can stay among them; `tail`: the mass of
// the others, where top-p goes by it.
__device__ __forceinline__ void finish_list(int n, u64 tail, const Settings& set, const Scale& sc, int V, DrawShared& sh,
                                            int32_t* token, float* logp) {
  const int tid = threadIdx.x;
  if (n <= kSort) return finish_sorted(sh.list, n, 0, tail, set, sc, sh, token, logp);
  const float scale = sh.tau > -INFINITY && sc.m > sh.tau ? static_cast<float>(kBins) / (sc.m - sh.tau) * 0.9999f : 0.f;
  const uint32_t id_width = static_cast<uint32_t>((V + kBins - 1) / kBins);

  // more of them: by value first, down to the bin that holds the border of top-k, else of top-p
  for (int i = tid; i < kBins; i += kDrawThreads) sh.bins[i] = make_uint4(0, 0, 0, 0);
  __syncthreads();
  for (int e = tid; e < n; e += kDrawThreads) {
    const float x = __uint_as_float(sh.list[e].x);
    add_to_bin(&sh.bins[value_bin(x, sc.m, scale)], set.use_k ? 0ull : weight(x, sc, sh.pow2));
  }
  __syncthreads();
  constexpr int kPer = kBins / kDrawThreads;
  u64 amount[kPer], sum = 0, all;
  int count[kPer], num = 0, n_all;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const uint4 b = sh.bins[tid * kPer + i];
    count[i] = static_cast<int>(b.x);
    amount[i] = set.use_k ? static_cast<u64>(b.x) : bin_mass(b);
    sum += amount[i];
    num += count[i];
  }
  u64 before = block_scan<u64, kDrawThreads>(sum, sh.scan, tid, &all) - sum;
  __syncthreads();
  int upto = block_scan<int, kDrawThreads>(num, reinterpret_cast<int*>(sh.scan), tid, &n_all) - num;
  const u64 need = set.use_k ? min(static_cast<u64>(set.top_k), all) : (set.use_p ? min(top_p_need(set, all + tail), all) : all);
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    upto += count[i];
    if (before < need && need <= before + amount[i]) {
      sh.bin = tid * kPer + i;
      sh.n_upto = upto;
    }
    before += amount[i];
  }
  if (tid == 0) sh.n_sub = 0;
  __syncthreads();
  if (sh.n_upto <= kSort) {
    const int bin = sh.bin;
    for (int e = tid; e < n; e += kDrawThreads) {
      const uint2 v = sh.list[e];
      if (value_bin(__uint_as_float(v.x), sc.m, scale) <= bin) sh.local[atomicAdd(&sh.n_sub, 1)] = v;
    }
    __syncthreads();
    return finish_sorted(sh.local, sh.n_sub, set.use_k ? 0 : need, 0, set, sc, sh, token, logp);
  }

  // still more (top-k of several hundreds, min-p on a flat row): border by border
  ListView l{sh.list, n, 0, sc, sh.pow2};
  auto kept = [&] {  // the mass from the cut on
    u64 mass = 0;
    for (int e = tid; e < n; e += kDrawThreads) {
      const float x = __uint_as_float(sh.list[e].x);
      if (order_of(x, sh.list[e].y) >= l.cut) mass += weight(x, sc, sh.pow2);
    }
    return block_total(mass, sh);
  };
  if (set.use_k && set.top_k < n)
    l.cut = find_border<false, false>(l, static_cast<u64>(set.top_k), sc.m, scale, 1, sh);
  all = kept();
  if (set.use_p) {
    const u64 share = top_p_need(set, all + tail);
    if (share < all) {
      l.cut = max(l.cut, find_border<true, false>(l, share, sc.m, scale, 1, sh));
      all = kept();
    }
  }
  if (set.use_m) {
    const u64 low = static_cast<u64>(value_key(sh.lowest)) << 32;
    if (low > l.cut) {
      l.cut = low;
      all = kept();
    }
  }
  const u64 goal = share_of(set.u, all, false);
  const uint32_t y = ~static_cast<uint32_t>(find_border<true, true>(l, goal + 1, sc.m, scale, id_width, sh));
  for (int e = tid; e < n; e += kDrawThreads)
    if (sh.list[e].y == y) {
      *token = static_cast<int32_t>(y);
      if (logp) {
        const float x = __uint_as_float(sh.list[e].x);
        *logp = log_prob(x, weight(x, sc, sh.pow2), all, sc, set.temp);
      }
    }
}

// ------------------------------------------------------------------ the whole cluster
// The warp's candidates, n of them, into the first CTA's list (as far as they fit); more than a segment: not all are
// there, and the list counts as full.
__device__ __forceinline__ void push(DrawShared& sh, int n, int round) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (!n) return;
  int to = 0;
  if (lane == 0) to = static_cast<int>(atom_add_cluster(&sh.n_list[round], 0, n > kSeg ? kListCap + 1 : n));
  to = __shfl_sync(0xffffffffu, to, 0);
  __syncwarp();
  const int fit = min(min(n, kSeg), kListCap - to);
  for (int i = lane; i < fit; i += 32) st_cluster(&sh.list[to + i], 0, sh.local[warp * kSeg + i]);
}

// The warp's part of the masses that are no candidates and that are, in units of 2^-44, to the first CTA.
__device__ __forceinline__ void add_masses(DrawShared& sh, int round, float rest, float hits) {
  u64 t = static_cast<u64>(rest * 0x1p44f), h = static_cast<u64>(fminf(hits, 0x1p8f) * 0x1p44f);
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    t += __shfl_xor_sync(0xffffffffu, t, o);
    h += __shfl_xor_sync(0xffffffffu, h, o);
  }
  if ((threadIdx.x & 31) == 0) {
    red_add_cluster(&sh.tail[round], 0, t);
    red_add_cluster(&sh.mass[round], 0, h);
  }
}

// After every warp's push: the cluster's number of candidates.
__device__ __forceinline__ int gathered(DrawShared& sh, int round) {
  cluster_sync();
  return static_cast<int>(ld_cluster(&sh.n_list[round], 0));
}

// Appends the elements of a unit that `wanted` says to the warp's segment `seg` of a list; *n: how many it has.
template <typename T, typename W>
__device__ __forceinline__ void append(const Slice<T>& sl, const Vec<T>& f, int q, int* n, uint2* seg, int cap, W&& wanted) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < Vec<T>::kN; ++i) {
    const float x = to_f32(f.e[i]);
    const bool hit = wanted(x) && sl.holds(q, i);
    const unsigned who = __ballot_sync(0xffffffffu, hit);
    const int at = *n + __popc(who & ((1u << lane) - 1u));
    if (hit && at < cap) seg[at] = make_uint2(__float_as_uint(x), sl.id(q, i));
    *n += __popc(who);
  }
}

// Of amounts a(value, id) over the slice, in id order: every warp's total into sh.scan, and the total of each of its
// steps (32 units) into sh.step; returns the CTA's.
template <typename T, typename A>
__device__ u64 slice_total(const Slice<T>& sl, DrawShared& sh, A&& amount) {
  constexpr int kAhead = 4;  // steps whose loads are under way together
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int q0, q1;
  sl.warp_share(&q0, &q1);
  u64* step = sh.step + warp * kMaxSteps;
  u64 all = 0;
  for (int q = q0; q < q1; q += 32 * kAhead) {
    Vec<T> v[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (q + 32 * j < q1) v[j] = sl.load(q + 32 * j + lane);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (q + 32 * j >= q1) break;
      const int mine = q + 32 * j + lane;
      u64 sum = 0;
#pragma unroll
      for (int i = 0; i < Vec<T>::kN; ++i)
        if (mine < q1 && sl.holds(mine, i)) sum += amount(to_f32(v[j].e[i]), sl.id(mine, i));
#pragma unroll
      for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (lane == 0) step[(q - q0) / 32 + j] = sum;
      all += sum;
    }
  }
  __syncthreads();
  if (lane == 0) sh.scan[warp] = all;
  __syncthreads();
  all = 0;
  for (int w = 0; w < kWarps; ++w) all += sh.scan[w];
  return all;
}

// After slice_total, with the same amounts: calls f(value, id) for the element at which the amounts pass `target`
// (their sum before it is at most `target`, with it more); `target` is below the CTA's total.
template <typename T, typename A, typename F>
__device__ void slice_locate(const Slice<T>& sl, u64 target, DrawShared& sh, A&& amount, F&& f) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  u64 at = 0;
  for (int w = 0; w < warp; ++w) at += sh.scan[w];
  if (target < at || target >= at + sh.scan[warp]) return;
  int q0, q1;
  sl.warp_share(&q0, &q1);
  const u64* step = sh.step + warp * kMaxSteps;
  const int steps = (q1 - q0 + 31) / 32;
  for (int s0 = 0; s0 < steps; s0 += 32) {
    const u64 mine = s0 + lane < steps ? step[s0 + lane] : 0ull;
    const u64 incl = warp_scan(mine, lane);
    const unsigned passed = __ballot_sync(0xffffffffu, target < at + incl);
    if (!passed) {
      at += __shfl_sync(0xffffffffu, incl, 31);
      continue;
    }
    const int s1 = __ffs(passed) - 1;  // the step that holds the element
    at += __shfl_sync(0xffffffffu, incl - mine, s1);
    const int q = q0 + 32 * (s0 + s1) + lane;
    const Vec<T> v = sl.load(q);
    u64 w[Vec<T>::kN], sum = 0;
#pragma unroll
    for (int i = 0; i < Vec<T>::kN; ++i) {
      w[i] = q < q1 && sl.holds(q, i) ? amount(to_f32(v.e[i]), sl.id(q, i)) : 0ull;
      sum += w[i];
    }
    u64 before = at + warp_scan(sum, lane) - sum;
#pragma unroll
    for (int i = 0; i < Vec<T>::kN; ++i) {
      if (before <= target && target < before + w[i]) f(to_f32(v.e[i]), sl.id(q, i));
      before += w[i];
    }
    return;
  }
}

// Radix selection across the cluster, for rows whose candidates no bound thins out.  Every element from `old` on
// carries `amount` (1, or its weight); the cut is the order at which the amounts, from the first on, reach `need`
// >= 1 (at most what they carry together).  Ties are cut by id, CTA by CTA: the result holds for this CTA's ids.
template <typename T, int SP, bool WEIGHTED>
__device__ u64 radix_cut(const Slice<T>& sl, u64 need, u64 old, const Scale& sc, DrawShared& sh, uint32_t part) {
  const int tid = threadIdx.x;
  uint32_t prefix = 0, mask = 0;
  int round = 0;
  for (int bit = 24; bit >= 0; bit -= 8, ++round) {
    u64* hist = sh.digit[round & 1];
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    sl.each([&](const Vec<T>& f, int q) {
#pragma unroll
      for (int i = 0; i < Vec<T>::kN; ++i) {
        const float x = to_f32(f.e[i]);
        const uint32_t k = value_key(x);
        const bool in = (k & mask) == prefix && sl.holds(q, i) && order_of(k, sl.id(q, i)) >= old;
        const uint32_t digit = (k >> bit) & 255;
        const u64 amount = !in ? 0ull : (WEIGHTED ? weight(x, sc, sh.pow2) : 1ull);
        // where the warp's elements share a digit (rows of equal values do throughout), one addition for all of them
        const unsigned who = __ballot_sync(0xffffffffu, in);
        if (!who) continue;
        const int one = __ffs(who) - 1;
        const uint32_t shared = __shfl_sync(0xffffffffu, digit, one);
        if (__all_sync(0xffffffffu, !in || digit == shared)) {
          u64 sum = amount;
#pragma unroll
          for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
          if ((tid & 31) == one) atomicAdd(&hist[digit], sum);
        } else if (in) {
          atomicAdd(&hist[digit], amount);
        }
      }
    });
    cluster_sync();  // every CTA's histogram is in place
    if (tid < 256) {
      u64 all = 0;
#pragma unroll
      for (int c = 0; c < SP; ++c) all += ld_cluster(&hist[tid], c);
      sh.total[tid] = all;
    }
    __syncthreads();
    if (tid < 32) {  // the digit at which the amounts, from the greatest digit down, reach `need`
      u64 mine[8], sum = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        mine[j] = sh.total[255 - (8 * tid + j)];
        sum += mine[j];
      }
      u64 above = warp_scan(sum, tid) - sum;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (above < need && need <= above + mine[j]) {
          sh.key = prefix | (static_cast<uint32_t>(255 - (8 * tid + j)) << bit);
          sh.need = need - above;
        }
        above += mine[j];
      }
    }
    __syncthreads();
    prefix = sh.key;
    need = sh.need;
    mask |= 255u << bit;
  }
  // ties: `need` of what the equal elements carry goes to the ones of lowest id.  They weigh the same, so the last
  // histogram gives every CTA the number of them before its slice.
  const u64* hist = sh.digit[(round - 1) & 1];
  const u64 each = WEIGHTED ? max(weight(key_value(prefix), sc, sh.pow2), 1ull) : 1ull;
  const u64 count = (need + each - 1) / each;  // equal elements that stay, over the cluster
  u64 before = 0, own = 0;
#pragma unroll
  for (int c = 0; c < SP; ++c) {
    const u64 n = ld_cluster(&hist[prefix & 255], c) / each;
    if (c < static_cast<int>(part)) before += n;
    if (c == static_cast<int>(part)) own = n;
  }
  cluster_sync();  // the histograms may be written again
  u64 cut = order_of(prefix, 0u) + 1;  // none of the equal ones
  if (before + own <= count) {
    cut = order_of(prefix, 0xffffffffu);  // all of them
  } else if (before < count) {
    auto equal = [&](float x, uint32_t id) { return static_cast<u64>(value_key(x) == prefix && order_of(prefix, id) >= old); };
    slice_total(sl, sh, equal);
    slice_locate(sl, count - before - 1, sh, equal, [&](float, uint32_t id) { sh.result = order_of(prefix, id); });
    __syncthreads();
    cut = sh.result;
  }
  return max(cut, old);
}

// The half octave of weight that a value lies in, on a grid that does not depend on the row's maximum.
__device__ __forceinline__ int half_octave(float x, float k) {
  return static_cast<int>(fminf(fmaxf(floorf(2.f * x * k), -1e9f), 1e9f));
}

// By one warp: the value below which the sample's mass, in units of 2^(-16 + half_octave(m) / 2), is at most `most`, or,
// if that is negative, at most its share -most of the sample's whole mass.
template <int SP>
__device__ float sampled_bound(DrawShared& sh, float m, float k, float most) {
  const int lane = threadIdx.x & 31;
  const int top = half_octave(m, k);
  float a[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {  // half octaves 2 lane and 2 lane + 1 from the top
    a[h] = 0.f;
#pragma unroll
    for (int c = 0; c < SP; ++c) a[h] += static_cast<float>(ld_cluster(&sh.slot[(top - 2 * lane - h) & (kSlots - 1)], c));
    a[h] *= ex2(-0.5f * static_cast<float>(2 * lane + h));
  }
  float below = a[0] + a[1];  // this lane's and all lower weights
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const float y = __shfl_down_sync(0xffffffffu, below, o);
    if (lane + o < 32) below += y;
  }
  if (most < 0.f) most *= -__shfl_sync(0xffffffffu, below, 0);
  const unsigned whole = __ballot_sync(0xffffffffu, below <= most);
  const unsigned half = __ballot_sync(0xffffffffu, below - a[0] <= most);
  const int from = min(whole ? 2 * (__ffs(whole) - 1) : kOctaves, half ? 2 * (__ffs(half) - 1) + 1 : kOctaves);
  return 0.5f * static_cast<float>(top - from + 1) / k;
}

// One pass over the row, for rows that some filter thins out: a value above which the ids that can stay lie is
// guessed from a sample (`v`: kSample units a thread, in whole warps, spread over the slice), the row is read once, and
// the guess is checked by what was found.  False (the same in every CTA): it was wrong, or too many ids lie above it.
template <typename T, int SP>
__device__ bool draw_from_sample(const Slice<T>& sl, const Vec<T> (&v)[8 / SP], const Settings& set, float min_p,
                                 const DrawParams& p, unsigned row, uint32_t part, DrawShared& sh) {
  constexpr int N = Vec<T>::kN;
  constexpr int kSample = 8 / SP;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const bool with_tail = set.use_p && !set.use_k;
  // top-k: of the k greatest about `e` are in the sample; a few more than that
  constexpr int kBest = 16 / SP, kValues = kBest * kWarps * SP;  // values of a warp, and of the cluster
  const float e = static_cast<float>(set.top_k) * (static_cast<float>(SP * kDrawThreads * kSample * N) / static_cast<float>(p.V));
  const int nth = static_cast<int>(fminf(e, 1e6f) + 3.f * sqrtf(fmaxf(e, 0.f)) + 2.5f);
  if (set.use_k && nth > kValues / 4) return false;
  float mx = -INFINITY;
#pragma unroll
  for (int j = 0; j < kSample; ++j) mx = fmaxf(mx, vec_max(v[j]));
  const float first = warp_max(mx);
  float next = first, left = mx;
#pragma unroll
  for (int i = 0; i < kBest; ++i) {  // of equal ones, one
    if (lane == 0) sh.best[kBest * warp + i] = next;
    left = left < next ? left : -INFINITY;
    if (i + 1 < kBest) next = warp_max(left);
  }
  const float k = sh.k_hi;
  // top-p: the sample's mass by half octaves, 32 octaves from the warp's maximum down: slot i mod kSlots holds the sum
  // of 2^(x k - i / 2) over the values of half octave i
  if (with_tail) {
    const int top = half_octave(first, k);
#pragma unroll
    for (int j = 0; j < kSample; ++j)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float x = to_f32(v[j].e[i]);
        const int h = half_octave(x, k);
        if (h > top - kOctaves)
          atomicAdd(&sh.slot[h & (kSlots - 1)], static_cast<uint32_t>(ex2(fmaf(x, k, -0.5f * static_cast<float>(h))) * 65536.f));
      }
  }
  if (tid == 32 && set.use_m) {
    const double d = static_cast<double>(set.temp) * log(fmin(static_cast<double>(min_p), 1.0));
    sh.floor = d == d ? d : -INFINITY;
  }
  cluster_sync();
  if (warp == 0) {
    constexpr int kPer = kValues / 32;
    float b[kPer], m = -INFINITY;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int at = i * 32 + lane;
      b[i] = ld_cluster(&sh.best[at % (kBest * kWarps)], at / (kBest * kWarps));
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) m = fmaxf(m, b[i]);
    m = warp_max(m);
    float tau = -INFINITY;
    if (set.use_k) {
      tau = jth_greatest<kPer>(b, nth);
    } else if (set.use_p) {
      tau = sampled_bound<SP>(sh, m, k, -0.6f * (1.f - set.top_p));  // a part of what may be left out of the sample
    }
    if (lane == 0) {
      // under min-p nothing below m + T log(min_p) stays, m being at most the maximum (with top-k and top-p, top-p
      // still goes by what top-k leaves)
      const float low = set.use_m && !(set.use_k && set.use_p) ? __double2float_rd(m + sh.floor) : -INFINITY;
      sh.by_min_p = low >= tau;
      tau = fmaxf(tau, low);
      sh.m = m;
      sh.tau = fminf(tau, m);
    }
  }
  __syncthreads();
  const float m = sh.m;
  float tau = sh.tau;
  if (!(tau > -INFINITY) || !(m < INFINITY)) {
    cluster_sync();
    return false;
  }

  int n = 0;
  u64 tail = 0;
  for (int attempt = 0;; ++attempt) {
    float rest = 0.f, hits = 0.f;
    int n_own = 0;
    sl.each([&](const Vec<T>& f, int q) {
      if (with_tail) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float x = to_f32(f.e[i]);
          const float e = ex2((x - m) * k);
          rest += x < tau ? e : 0.f;
          hits += x >= tau ? e : 0.f;
        }
      }
      if (__any_sync(0xffffffffu, vec_max(f) >= tau)) append<T>(sl, f, q, &n_own, sh.local + warp * kSeg, kSeg, [&](float x) { return x >= tau; });
    });
    if (with_tail) add_masses(sh, 3 + attempt, rest, hits);
    push(sh, n_own, 4 + attempt);
    n = gathered(sh, 4 + attempt);
    bool good = n >= 1 && n <= kListCap && (!set.use_k || sh.by_min_p || n >= set.top_k);
    if (with_tail) {
      tail = ld_cluster(&sh.tail[3 + attempt], 0);
      const float t = static_cast<float>(tail), h = static_cast<float>(ld_cluster(&sh.mass[3 + attempt], 0));
      const bool held = sh.by_min_p || t * 1.0001f <= (1.f - set.top_p) * (t + h);
      if (!held && attempt == 0) {
        // The sample missed what carries the mass: its lower part, scaled up to the row, against the row's own mass.
        if (warp == 0) {
          const float unit = static_cast<float>(p.V) / (static_cast<float>(SP * kDrawThreads * kSample * N) * 65536.f) *
                             ex2(fmaf(-m, k, 0.5f * static_cast<float>(half_octave(m, k))));
          const float next = sampled_bound<SP>(sh, m, k, (1.f - set.top_p) * 0.2f * (t + h) * 0x1p-44f / unit);
          if (lane == 0) sh.tau = fminf(next, tau);
        }
        __syncthreads();
        tau = sh.tau;
        if (tau > -INFINITY) continue;
      }
      good = good && held;
    }
    if (!good) {
      cluster_sync();  // done with the counts
      return false;
    }
    break;
  }
  if (part != 0) return true;

  // ---- the first CTA: the true maximum is in the list
  int32_t* token = p.tokens + row;
  float* logp = p.logp ? p.logp + row : nullptr;
  if (!with_tail) tail = 0;
  if (n <= kSort) {
    finish_sorted(sh.list, n, 0, tail, set, Scale{m, k, sh.k_lo, false}, sh, token, logp);
  } else {
    float top = -INFINITY;
    for (int e = tid; e < n; e += kDrawThreads) top = fmaxf(top, __uint_as_float(sh.list[e].x));
    top = warp_max(top);
    if (lane == 0) sh.red[warp] = top;
    __syncthreads();
    top = warp_max(lane < kWarps ? sh.red[lane] : -INFINITY);
    const Scale sc{top, k, sh.k_lo, top == INFINITY};
    if (tid == 0 && set.use_m) sh.lowest = sc.inf ? INFINITY : __double2float_ru(top + sh.floor);
    if (tail && m != top) tail = rescaled(tail, weight(m, sc, sh.pow2));
    __syncthreads();
    finish_list(n, tail, set, sc, p.V, sh, token, logp);
  }
  cluster_sync();  // this CTA stays until the others, which read its counts, have left
  return true;
}

// By one warp: the value below which the groups' maxima carry at most `most` (in units of 2^-20), or, if that is
// negative, at most its share -most of what they carry together; sh.below_guess: what they do carry below it.
template <int SP>
__device__ float maxima_bound(DrawShared& sh, const Scale& sc, float most) {
  const int lane = threadIdx.x & 31;
  float a = 0.f, b = 0.f;  // half octaves 2 lane and 2 lane + 1
#pragma unroll
  for (int c = 0; c < SP; ++c) {
    a += static_cast<float>(ld_cluster(&sh.octave[2 * lane], c));
    b += static_cast<float>(ld_cluster(&sh.octave[2 * lane + 1], c));
  }
  float below = a + b;  // this lane's and all lower weights
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const float y = __shfl_down_sync(0xffffffffu, below, o);
    if (lane + o < 32) below += y;
  }
  if (most < 0.f) most *= -__shfl_sync(0xffffffffu, below, 0);
  const unsigned whole = __ballot_sync(0xffffffffu, below <= most), half = __ballot_sync(0xffffffffu, below - a <= most);
  const int first = min(whole ? 2 * (__ffs(whole) - 1) : kOctaves, half ? 2 * (__ffs(half) - 1) + 1 : kOctaves);
  const float left = __shfl_sync(0xffffffffu, first & 1 ? below - a : below, min(first, kOctaves - 1) / 2);
  if (lane == 0) sh.below_guess = first < kOctaves ? left : 0.f;
  return sc.m - 0.5f * static_cast<float>(first) / sc.k_hi;
}

template <typename T, int SP>
__global__ void __launch_bounds__(kDrawThreads, 4) filtered_draw_kernel(const DrawParams p) {
  extern __shared__ __align__(16) unsigned char s_raw[];
  DrawShared& sh = *reinterpret_cast<DrawShared*>(s_raw);
  const unsigned row = blockIdx.x / SP;
  const uint32_t part = cluster_ctarank();  // == blockIdx.x % SP
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int lo = min(p.V, static_cast<int>(part) * p.slice);
  const Slice<T> sl(static_cast<const T*>(p.logits) + row * static_cast<size_t>(p.stride), lo,
                    min(p.V, lo + p.slice) - lo);
  constexpr int N = Vec<T>::kN;
  constexpr int kSample = 8 / SP;  // units a thread

  // the slice, on its way into L2
  if (tid == 0 && sl.last > sl.first)
    l2_prefetch_bulk(sl.src + (sl.first * N - sl.shift), static_cast<uint32_t>(sl.last - sl.first) * 16);

  // ---- the sample, on its way while the settings are read
  Vec<T> v[kSample];
  const bool sampled = p.slice >= 4 * kDrawThreads * kSample * N;
  if (sampled) {
    int q0, q1;
    sl.warp_share(&q0, &q1);
#pragma unroll
    for (int j = 0; j < kSample; ++j) v[j] = sl.load(q0 + (q1 - q0) / kSample * j + lane);
  }
  sh.slot[tid] = 0;

  // ---- the row's settings
  const unsigned at_set = row / p.rows_per_set;
  Settings set;
  set.temp = p.temperature ? __ldg(p.temperature + at_set) : 1.f;
  set.top_k = p.top_k ? __ldg(p.top_k + at_set) : 0;
  set.top_p = p.top_p ? __ldg(p.top_p + at_set) : 1.f;
  const float min_p = p.min_p ? __ldg(p.min_p + at_set) : 0.f;
  set.u = __ldg(p.uniforms + row);
  if (!(set.u >= 0.f)) set.u = 0.f;
  if (set.u >= 1.f) set.u = 0x1.fffffep-1f;  // the largest float below 1

  if (!(set.temp > 0.f)) {  // greedy
    set.temp = 1.f;
    set.top_k = 1;
  }
  set.use_k = set.top_k >= 1 && set.top_k < p.V;
  set.use_p = set.top_p < 1.f;
  set.use_m = min_p > 0.f;
  const bool with_tail = set.use_p && !set.use_k;
  if (tid < 32) sh.pow2[tid] = c_pow2[tid];
  if (tid == 32) {
    constexpr float kLog2eHi = 1.44269502f, kLog2eLo = 1.92596300e-8f;
    const float k = fminf(kLog2eHi / set.temp, 3.0e38f);  // a T so small leaves the maximum alone either way
    sh.k_hi = k;
    sh.k_lo = k > 0.f && k < 1.0e38f ? (fmaf(-k, set.temp, kLog2eHi) + kLog2eLo) / set.temp : 0.f;
#pragma unroll
    for (int i = 0; i < 6; ++i) sh.n_list[i] = 0;
#pragma unroll
    for (int i = 0; i < 5; ++i) sh.tail[i] = sh.mass[i] = 0;
  }
  __syncthreads();
  if (sampled && (set.use_k || set.use_p || set.use_m))
    if (draw_from_sample<T, SP>(sl, v, set, min_p, p, row, part, sh)) return;

  // ---- the row maximum (NaN never is)
  float mx = -INFINITY;
  sl.each([&](const Vec<T>& f, int) { mx = fmaxf(mx, vec_max(f)); });

  if (tid == 32 && set.use_m) {
    const double d = static_cast<double>(set.temp) * log(fmin(static_cast<double>(min_p), 1.0));
    sh.floor = d == d ? d : -INFINITY;  // an infinite T makes all ids alike
  }

  // ---- what bounds the candidates from below
  // top-k: where every CTA has ceil(k / 8) groups of elements whose maxima reach a value, k elements do
  const int in_cta = set.use_k ? (set.top_k + SP - 1) / SP : 0;
  const bool small_k = in_cta <= 64;
  const bool bound_k = set.use_k && in_cta <= 128;
  if (bound_k) {  // 128 groups, or 256
    float g = mx;
    for (int o = 1; o < (small_k ? kDrawThreads / 128 : kDrawThreads / 256); o *= 2) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, o));
    const int per = small_k ? kDrawThreads / 128 : kDrawThreads / 256;
    if (tid % per == 0) sh.group[tid / per] = g;
  }
  const float wmx = warp_max(mx);
  if (lane == 0) sh.red[warp] = wmx;
  __syncthreads();
  float own_max = sh.red[0];
#pragma unroll
  for (int w = 1; w < kWarps; ++w) own_max = fmaxf(own_max, sh.red[w]);
  if (with_tail) {  // top-p: the maxima's own mass is a lower bound of the whole
    const float e = warp_sum(mx > -INFINITY ? ex2((mx - own_max) * sh.k_hi) : 0.f);
    if (lane == 0) sh.red2[warp] = e;
    __syncthreads();
  }
  if (warp == 0) {
    float aux = -INFINITY;
    if (bound_k) {
      float g[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = i < 4 || !small_k ? sh.group[i * 32 + lane] : -INFINITY;
      aux = jth_greatest<8>(g, in_cta);
    }
    if (with_tail) aux = warp_sum(lane < kWarps ? sh.red2[lane] : 0.f);
    if (lane == 0) {
      sh.max = own_max;
      sh.aux = aux;
    }
  }
  cluster_sync();
  if (warp == 0) {
    const float cm = lane < SP ? ld_cluster(&sh.max, lane) : -INFINITY;
    const float ca = lane < SP ? ld_cluster(&sh.aux, lane) : INFINITY;
    const float m = warp_max(cm);
    float tau = -INFINITY;
    if (set.use_k) {
      tau = set.top_k == 1 ? m : -warp_max(-ca);
    } else if (set.use_p) {
      // mass below tau <= V exp((tau - m) / T) <= (1 - p) * mass
      const float z = warp_sum(cm > -INFINITY && lane < SP ? ca * ex2((cm - m) * sh.k_hi) : 0.f);
      tau = m + log2f((1.f - set.top_p) * z / static_cast<float>(p.V) * 0.999f) / sh.k_hi;
    }
    float lowest = -INFINITY;
    if (set.use_m) {
      if (lane == 0) {
        const double d = m + sh.floor;
        lowest = m == INFINITY ? INFINITY : __double2float_ru(d);
        if (!(set.use_k && set.use_p)) tau = fmaxf(tau, __double2float_rd(d));
      }
    }
    if (lane == 0) {
      sh.m = m;
      sh.tau = sh.guess = fminf(tau, m);
      sh.lowest = lowest;
    }
  }
  __syncthreads();
  const Scale sc{sh.m, sh.k_hi, sh.k_lo, sh.m == INFINITY};
  float* logp = p.logp ? p.logp + row : nullptr;
  if (sc.m == -INFINITY) {  // nothing to draw from: the same in every CTA of the cluster
    if (part == 0 && tid == 0) {
      p.tokens[row] = 0;
      if (logp) *logp = -INFINITY;
    }
    cluster_sync();  // no CTA leaves while another may still read its maximum
    return;
  }

  // ---- the candidates, to the first CTA if they are few
  u64 cut = 0;  // the order of the last id that stays
  bool cut_k = set.use_k, cut_p = set.use_p;  // still to be found
  if ((sh.tau > -INFINITY || p.V <= 1024) && !sc.inf) {
    if (with_tail && sh.tau > -INFINITY) {
      // That bound is safe but low.  A nearer one, to be checked: where the groups' maxima below it carry a third of
      // what top-p may leave out.
      if (tid < kOctaves) sh.octave[tid] = 0;
      __syncthreads();
      const float t = (mx - sc.m) * sc.k_hi;
      if (t > -0.5f * kOctaves)
        atomicAdd(&sh.octave[min(static_cast<int>(-2.f * t), kOctaves - 1)], static_cast<uint32_t>(ex2(t) * 0x1p20f));
      cluster_sync();
      if (warp == 0) {
        const float guess = maxima_bound<SP>(sh, sc, -(1.f - set.top_p) * (1.f / 3.f));
        if (lane == 0) sh.guess = fmaxf(sh.tau, guess);
      }
      __syncthreads();
    }
    float tau = sh.guess;
    int n = 0;
    u64 tail = 0;
    for (int attempt = 0;; ++attempt) {
      float rest = 0.f, hits = 0.f;
      int n_own = 0;
      sl.each([&](const Vec<T>& f, int q) {
        if (with_tail) {
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const float x = to_f32(f.e[i]);
            const float e = ex2((x - sc.m) * sc.k_hi);
            rest += x < tau ? e : 0.f;
            hits += x >= tau ? e : 0.f;
          }
        }
        if (__any_sync(0xffffffffu, vec_max(f) >= tau)) append<T>(sl, f, q, &n_own, sh.local + warp * kSeg, kSeg, [&](float x) { return x >= tau; });
      });
      if (lane == 0) sh.n_warp[warp] = n_own;
      if (with_tail) add_masses(sh, attempt, rest, hits);
      push(sh, n_own, attempt);
      n = gathered(sh, attempt);
      if (!with_tail) break;
      tail = ld_cluster(&sh.tail[attempt], 0);
      const float t = static_cast<float>(tail), h = static_cast<float>(ld_cluster(&sh.mass[attempt], 0));
      if (tau == sh.tau || t * 1.0001f <= (1.f - set.top_p) * (t + h)) break;  // every id that can stay is above tau
      // too high: lower by what the maxima below it turned out to stand for; then the safe bound
      if (attempt == 0 && warp == 0) {
        const float next = maxima_bound<SP>(sh, sc, sh.below_guess * 0.4f * (1.f - set.top_p) * (t + h) / t);
        if (lane == 0) sh.guess = fmaxf(sh.tau, fminf(next, tau));
      }
      __syncthreads();
      tau = attempt == 0 && sh.guess < tau ? sh.guess : sh.tau;
    }
    const float scale = tau > -INFINITY && sc.m > tau ? static_cast<float>(kBins) / (sc.m - tau) * 0.9999f : 0.f;
    bool fits = n <= kListCap;
    if (!fits && with_tail) {
      const int n_own = sh.n_warp[warp];
      const bool listed = __syncthreads_and(n_own <= kSeg);  // the local list has them all
      // the candidates' weights by value (from the list, or from the slice where it has more than the list holds)
      for (int i = tid; i < kBins; i += kDrawThreads) sh.bins[i] = make_uint4(0, 0, 0, 0);
      __syncthreads();
      if (listed) {
        for (int e = lane; e < n_own; e += 32) {
          const float x = __uint_as_float(sh.local[warp * kSeg + e].x);
          add_to_bin(&sh.bins[value_bin(x, sc.m, scale)], weight(x, sc, sh.pow2));
        }
      } else {
        // (gathered by the warp first, so that whole warps compute weights; the list's memory is free meanwhile)
        constexpr int kPart = kListCap / kWarps;
        uint2* part_list = sh.list + warp * kPart;
        int held = 0;
        auto flush = [&] {
          __syncwarp();
          for (int e = lane; e < held; e += 32) {
            const float x = __uint_as_float(part_list[e].x);
            add_to_bin(&sh.bins[value_bin(x, sc.m, scale)], weight(x, sc, sh.pow2));
          }
          __syncwarp();
          held = 0;
        };
        sl.each([&](const Vec<T>& f, int q) {
          if (!__any_sync(0xffffffffu, vec_max(f) >= tau)) return;
          append<T>(sl, f, q, &held, part_list, kPart, [&](float x) { return x >= tau; });
          if (held > kPart - 32 * N) flush();
        });
        flush();
      }
      cluster_sync();
      // the bin that holds top-p's border, found by the first CTA
      if (part == 0) {
        constexpr int kPer = kBins / kDrawThreads;
        u64 mass[kPer], sum = 0, all;
        int count[kPer], num = 0, n_all;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          mass[i] = 0;
          count[i] = 0;
          uint4 b[SP];
#pragma unroll
          for (int c = 0; c < SP; ++c) b[c] = ld_cluster(&sh.bins[tid * kPer + i], c);
#pragma unroll
          for (int c = 0; c < SP; ++c) {
            mass[i] += bin_mass(b[c]);
            count[i] += static_cast<int>(b[c].x);
          }
          sum += mass[i];
          num += count[i];
        }
        u64 before = block_scan<u64, kDrawThreads>(sum, sh.scan, tid, &all) - sum;
        __syncthreads();
        int upto = block_scan<int, kDrawThreads>(num, reinterpret_cast<int*>(sh.scan), tid, &n_all) - num;
        const u64 need = min(top_p_need(set, all + tail), all);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          if (before < need && need <= before + mass[i]) {
            sh.bin = tid * kPer + i;
            sh.need = need - before;
            sh.n_upto = upto + count[i];
            sh.n_in = count[i];
            sh.below = all + tail - before - mass[i];  // the mass after the bin
          }
          before += mass[i];
          upto += count[i];
        }
      }
      cluster_sync();
      const int bin = static_cast<int>(ld_cluster(reinterpret_cast<uint32_t*>(&sh.bin), 0));
      const int n_upto = static_cast<int>(ld_cluster(reinterpret_cast<uint32_t*>(&sh.n_upto), 0));
      const int n_in = static_cast<int>(ld_cluster(reinterpret_cast<uint32_t*>(&sh.n_in), 0));
      // Down to the border they are gathered if they can be sorted, else those in its bin are (as many as the warps'
      // segments hold where the ids lie anyhow: five eighths of them): the first CTA alone takes longer over a long list
      // than the cluster over two more passes (1500 of 151936 ids kept: 160 us against 100).
      constexpr int kSafe = kListCap < kLocalCap / 8 * 5 * SP ? kListCap : kLocalCap / 8 * 5 * SP;
      fits = n_upto <= kSort;
      if (fits || n_in <= kSafe) {
        auto wanted = [&](float x) {
          const int b = value_bin(x, sc.m, scale);
          return b == bin || (fits && b < bin);
        };
        int left = 0;
        if (listed) {  // in place: what stays of a warp's segment moves to its front
          for (int e0 = 0; e0 < n_own; e0 += 32) {
            const bool on = e0 + lane < n_own;
            const uint2 v = on ? sh.local[warp * kSeg + e0 + lane] : make_uint2(0, 0);
            const bool hit = on && wanted(__uint_as_float(v.x));
            const unsigned who = __ballot_sync(0xffffffffu, hit);
            if (hit) sh.local[warp * kSeg + left + __popc(who & ((1u << lane) - 1u))] = v;
            left += __popc(who);
            __syncwarp();
          }
        } else {
          sl.each([&](const Vec<T>& f, int q) {
            if (__any_sync(0xffffffffu, vec_max(f) >= tau))
              append<T>(sl, f, q, &left, sh.local + warp * kSeg, kSeg, [&](float x) { return x >= tau && wanted(x); });
          });
        }
        push(sh, left, 3);
        n = gathered(sh, 3);
        fits = fits && n <= kListCap;
        if (!fits && n <= kListCap) {  // the border's bin decides the border
          if (part == 0) {
            const u64 need = sh.need;
            const float top = sc.m - static_cast<float>(bin) / scale;  // of the bin, which is binned again
            const u64 border = find_border<true, false>(ListView{sh.list, n, 0, sc, sh.pow2}, need, top,
                                                        scale * static_cast<float>(kBins), 1, sh);
            if (tid == 0) sh.cut = border;
          }
          cluster_sync();
          cut = ld_cluster(&sh.cut, 0);
          cut_p = false;
        } else if (part == 0) {
          tail = sh.below;
        }
      }
    }
    if (fits) {
      if (part != 0) return;
      __syncthreads();
      if (sh.tau != tau && tid == 0) sh.tau = tau;
      __syncthreads();
      finish_list(n, tail, set, sc, p.V, sh, p.tokens + row, logp);
      cluster_sync();  // this CTA stays until the others, which read its counts, have left
      return;
    }
  }

  // ---- the cluster goes on together: what is left to cut
  if (cut_k) cut = radix_cut<T, SP, false>(sl, static_cast<u64>(set.top_k), cut, sc, sh, part);
  auto kept_weight = [&](float x, uint32_t id) { return order_of(x, id) >= cut ? weight(x, sc, sh.pow2) : 0ull; };
  if (cut_p) {
    const u64 own = slice_total(sl, sh, kept_weight);
    if (tid == 0) sh.sum = own;
    cluster_sync();
    u64 all = 0;
    for (int c = 0; c < SP; ++c) all += ld_cluster(&sh.sum, c);
    cluster_sync();
    const u64 need = top_p_need(set, all);
    cut = radix_cut<T, SP, true>(sl, need, cut, sc, sh, part);
  }
  if (set.use_m) cut = max(cut, static_cast<u64>(value_key(sh.lowest)) << 32);

  // ---- the draw, in id order
  const u64 own = slice_total(sl, sh, kept_weight);
  if (tid == 0) sh.sum = own;
  cluster_sync();
  u64 all = 0, before = 0;
#pragma unroll
  for (int c = 0; c < SP; ++c) {
    const u64 n = ld_cluster(&sh.sum, c);
    if (c < static_cast<int>(part)) before += n;
    all += n;
  }
  cluster_arrive();  // done with the other CTAs' shared memory
  const u64 goal = share_of(set.u, all, false);
  if (before <= goal && goal < before + own)
    slice_locate(sl, goal - before, sh, kept_weight, [&](float x, uint32_t id) {
      p.tokens[row] = static_cast<int32_t>(id);
      if (logp) *logp = log_prob(x, weight(x, sc, sh.pow2), all, sc, set.temp);
    });
  cluster_wait();
}

template <typename T, int SP>
static cudaError_t launch_draw(DrawParams p, int rows, cudaStream_t stream) {
  constexpr size_t smem = sizeof(DrawShared);
  p.slice = ((p.V + SP - 1) / SP + 7) & ~7;
  cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(filtered_draw_kernel<T, SP>), smem, false);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(rows) * SP);
  cfg.blockDim = dim3(kDrawThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = SP;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, filtered_draw_kernel<T, SP>, p);
  return e != cudaSuccess ? e : cudaGetLastError();
}

// CTAs a row: eight, so that few rows use many SMs; halved while the rows alone keep four CTAs an SM busy and a slice is
// shorter than 128 KB, for what a CTA does besides reading does not shrink with its slice.
template <typename T>
cudaError_t launch_draw_type(const DrawParams& p, int rows, cudaStream_t stream) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  int split = 8;
  while (split > 2 && static_cast<long long>(rows) * split > 4 * sms && p.V / split * sizeof(T) < (128 << 10)) split /= 2;
  if (split == 8) return launch_draw<T, 8>(p, rows, stream);
  return split == 4 ? launch_draw<T, 4>(p, rows, stream) : launch_draw<T, 2>(p, rows, stream);
}

}  // namespace dm
