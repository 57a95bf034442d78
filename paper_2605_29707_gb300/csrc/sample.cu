// sample.cu -- one token per row of logits after temperature, top-k, top-p and min-p, drawn with the
// caller's uniform (the target's side of section 3.1 when it decodes with these filters).
//
// Mathematics.  With z = x / T and the ids ordered by (z descending, id ascending): the first k stay;
// of those, the ones whose predecessors in that order hold less than p of the mass; of those, the ones
// with exp(z - max z) >= min_p; the first always.  The token is the first kept id, in id order, whose
// cumulative mass exceeds u times the kept mass.
//
// Weights are integers: 2^44 exp(z - max z), rounded.  At most 2^19 of them fit 63 bits, so every sum
// is exact and the same in any order: splitting a row over CTAs, atomics and the order of threads
// change nothing.  A weight above 2^-14 of the greatest is computed to about 2^-38 of its value
// (weight()), one below in fp32.  (z, id) is one 64-bit integer (Order), so every cut is a bound on it.
//
// A cluster of eight CTAs takes a row, an eighth each, and reads it twice, the second time from L2: eight
// slices of 76 KB (V = 151936, fp32) per SM would not fit its shared memory, while what is in flight on
// the whole chip fits L2, and a plain re-read of L2-resident slices ran at 11 TB/s against 7 from DRAM.
//   1. the row maximum, and a value below which no id can stay: with top-k, where every CTA has k / 8
//      groups of elements whose maxima reach it; with top-p, where V ids of its weight would carry less
//      than 1 - p of what those maxima carry already; with min-p, from its definition;
//   2. the ids above it, the candidates, go to the first CTA, which finishes the row alone while the
//      others leave; with top-p the weights of the other ids are added up on the way, in fp32.
// Too many candidates (more than kListCap) under top-p: the candidates' weights are added up by value
// in kBins bins, the bin that holds the border is found, and either the candidates down to it are few
// enough, or those in it are and decide the border.  What else leaves too many is cut by a radix selection
// over the whole row.  Then, and without any filter, the cluster scans the kept weights in id order.
#include <math.h>

#include "kernels.h"
#include "rows.cuh"

namespace dm {

constexpr int kDrawThreads = 256;
constexpr int kDrawWarps = kDrawThreads / 32;
constexpr int kDrawBatch = 4;       // 16-byte loads a thread has in flight
constexpr int kListCap = 2048;      // candidates the cluster's first CTA can take
constexpr int kBins = 512;          // of values, or of ids
constexpr int kSubCap = 256;        // entries of one bin that are ranked against each other
constexpr int kDirect = 128;        // entries that are ranked without bins
constexpr int kWeightBits = 44;     // the greatest weight is 2^44
constexpr float kNoWeight = -45.f;  // log2 of a relative weight that rounds to nothing
constexpr float kCoarse = -14.f;    // below this (log2) a weight is computed in fp32

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
__device__ __forceinline__ u64 weight(float x, const Scale& sc, const u64* pow2) {
  if (sc.inf) return x == sc.m ? 1ull << kWeightBits : 0ull;
  const float d = x - sc.m;
  const float t = d * sc.k_hi;
  if (!(t >= kNoWeight)) return 0ull;
  if (t < kCoarse) return static_cast<u64>(__float2uint_rn(ex2(t + static_cast<float>(kWeightBits))));
  // x - m = d + d_lo
  const float xv = d + sc.m;
  const float mv = d - xv;
  const float d_lo = (x - xv) + (-sc.m - mv);
  const float t_lo = fmaf(d, sc.k_hi, -t) + fmaf(d, sc.k_lo, d_lo * sc.k_hi);
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
  uint2 local[kListCap];  // this CTA's candidates (value, id); in the first CTA, later, the list's weights
  uint2 list[kListCap];   // the first CTA: the cluster's candidates
  uint4 bins[kBins];      // count and weights (three limbs of 15 bits) by value or id
  u64 pow2[32];
  u64 sub_order[kSubCap];
  u64 sub_amount[kSubCap];
  u64 scan[kDrawWarps];
  u64 digit[2][256];      // a radix round's histogram, by round parity (read by the cluster)
  u64 total[256];
  u64 sum;                // kept mass of this CTA (read by the cluster)
  u64 tail;               // the first CTA: mass of the ids that are no candidates
  u64 need, result;
  u64 cut;                // the first CTA: the border of top-p (read by the cluster)
  double floor;           // T log(min_p)
  float group[kDrawThreads];
  float red[kDrawWarps], red2[kDrawWarps];
  float max, aux;         // this CTA's maximum, and its part of the candidates' bound (read by the cluster)
  float k_hi, k_lo;
  float m, tau, lowest;   // lowest: the least value that min-p keeps
  uint32_t key;
  int n_local;            // entries of local
  uint32_t n_list[2];     // the first CTA: the cluster's candidates, of the first and the second gathering
  int base, n_sub, bin, n_upto, n_in, before;
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
  // f(unit, its index) for every unit, a batch of loads at a time
  template <typename F>
  __device__ __forceinline__ void each(F&& f) const {
    for (int q0 = threadIdx.x; q0 < units; q0 += kDrawThreads * kDrawBatch) {
      Vec<T> v[kDrawBatch];
#pragma unroll
      for (int j = 0; j < kDrawBatch; ++j)
        if (q0 + j * kDrawThreads < units) v[j] = load(q0 + j * kDrawThreads);
#pragma unroll
      for (int j = 0; j < kDrawBatch; ++j)
        if (q0 + j * kDrawThreads < units) f(v[j], q0 + j * kDrawThreads);
    }
  }
  // the units of this warp's share of the slice, in id order: [*q0, *q1)
  __device__ __forceinline__ void warp_share(int* q0, int* q1) const {
    const int per = (units + kDrawWarps - 1) / kDrawWarps;
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
__device__ __forceinline__ float jth_greatest(const float* v, int j, int lane) {
  uint32_t key[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) key[i] = value_key(v[i * 32 + lane]) >> 16;
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
  const u64* wt;
  int n;
  u64 cut;
  __device__ __forceinline__ bool entry(int e, bool weighted, bool by_id, u64* order, u64* amount) const {
    const uint2 v = list[e];
    const u64 o = order_of(__uint_as_float(v.x), v.y);
    if (o < cut) return false;
    *order = by_id ? static_cast<u64>(~v.y) : o;
    *amount = weighted ? wt[e] : 1ull;
    return true;
  }
};

template <bool WEIGHTED, bool BY_ID>
__device__ u64 find_border(const ListView& l, u64 need, float top, float scale, uint32_t id_width, DrawShared& sh) {
  const int tid = threadIdx.x;
  u64 o = 0, a = 0;
  __syncthreads();
  if (tid == 0) sh.n_sub = 0;
  if (l.n <= kDirect) {
    if (tid < l.n) {
      if (!l.entry(tid, WEIGHTED, BY_ID, &o, &a)) o = a = 0;
      sh.sub_order[tid] = o;
      sh.sub_amount[tid] = a;
    }
    __syncthreads();
    if (tid == 0) sh.n_sub = l.n;
  } else {
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
    u64 mine[kBins / kDrawThreads], sum = 0, all;
#pragma unroll
    for (int i = 0; i < kBins / kDrawThreads; ++i) {
      mine[i] = bin_mass(sh.bins[tid * (kBins / kDrawThreads) + i]);
      sum += mine[i];
    }
    u64 before = block_scan<u64, kDrawThreads>(sum, sh.scan, tid, &all) - sum;
#pragma unroll
    for (int i = 0; i < kBins / kDrawThreads; ++i) {
      if (before < need && need <= before + mine[i]) {
        sh.bin = tid * (kBins / kDrawThreads) + i;
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
  }
  __syncthreads();
  const int c = sh.n_sub;
  if (c <= kSubCap) {  // each against each
    const u64 want = l.n <= kDirect ? need : sh.need;
    const bool pairs = c <= kDrawThreads / 2;  // two threads an entry
    const int e = pairs ? tid >> 1 : tid;
    o = e < c ? sh.sub_order[e] : ~0ull;
    u64 before = 0;
    for (int j = pairs ? tid & 1 : 0; j < c; j += pairs ? 2 : 1)
      if (sh.sub_order[j] > o) before += sh.sub_amount[j];
    if (pairs) before += __shfl_xor_sync(0xffffffffu, before, 1);
    if (e < c && before < want && want <= before + sh.sub_amount[e]) sh.result = o;
  } else {  // one bit of the order at a time: the greatest order from which on the amounts reach `need`
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

// The end of a row in the cluster's first CTA: n candidates, every id that can stay among them; `tail`: the mass of
// the others, where top-p goes by it.
__device__ void finish_list(int n, u64 tail, const Settings& set, const Scale& sc, int V, DrawShared& sh, int32_t* token,
                            float* logp) {
  const int tid = threadIdx.x;
  u64* wt = reinterpret_cast<u64*>(sh.local);
  ListView l{sh.list, wt, n, 0};
  const float scale = sh.tau > -INFINITY && sc.m > sh.tau ? static_cast<float>(kBins) / (sc.m - sh.tau) * 0.9999f : 0.f;
  const uint32_t id_width = static_cast<uint32_t>((V + kBins - 1) / kBins);
  u64 mine = 0;
  for (int e = tid; e < n; e += kDrawThreads) {
    const u64 w = weight(__uint_as_float(sh.list[e].x), sc, sh.pow2);
    wt[e] = w;
    mine += w;
  }
  u64 all = block_total(mine, sh);
  auto kept = [&] {  // the mass from the cut on
    u64 sum = 0;
    for (int e = tid; e < n; e += kDrawThreads)
      if (order_of(__uint_as_float(sh.list[e].x), sh.list[e].y) >= l.cut) sum += wt[e];
    return block_total(sum, sh);
  };
  if (set.use_k && set.top_k < n) {
    l.cut = find_border<false, false>(l, static_cast<u64>(set.top_k), sc.m, scale, 1, sh);
    all = kept();
  }
  if (set.use_p) {
    const u64 need = set.top_p > 0.f ? max(share_of(set.top_p, all + tail, true), 1ull) : 1ull;
    if (need < all) {
      l.cut = max(l.cut, find_border<true, false>(l, need, sc.m, scale, 1, sh));
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
      if (logp) *logp = (__uint_as_float(sh.list[e].x) - sc.m) / set.temp - logf(static_cast<float>(all) * 0x1p-44f);
    }
}

// ------------------------------------------------------------------ the whole cluster
// This CTA's candidates into the first CTA's list (as far as they fit); the cluster's number of them.
__device__ int gather(DrawShared& sh, int round) {
  const int tid = threadIdx.x;
  __syncthreads();
  const int n = sh.n_local;
  if (tid == 0) sh.base = static_cast<int>(atom_add_cluster(&sh.n_list[round], 0, static_cast<uint32_t>(n)));
  __syncthreads();
  const int base = sh.base;
  const int fit = min(min(n, kListCap), kListCap - base);
  for (int i = tid; i < fit; i += kDrawThreads) st_cluster(&sh.list[base + i], 0, sh.local[i]);
  cluster_sync();
  return static_cast<int>(ld_cluster(&sh.n_list[round], 0));
}

// Of amounts a(value, id) over the slice, in id order: every warp's total into sh.scan; returns the CTA's.
template <typename T, typename A>
__device__ u64 slice_total(const Slice<T>& sl, DrawShared& sh, A&& amount) {
  int q0, q1;
  sl.warp_share(&q0, &q1);
  u64 sum = 0;
#pragma unroll 2
  for (int q = q0 + (threadIdx.x & 31); q < q1; q += 32) {
    const Vec<T> f = sl.load(q);
#pragma unroll
    for (int i = 0; i < Vec<T>::kN; ++i)
      if (sl.holds(q, i)) sum += amount(to_f32(f.e[i]), sl.id(q, i));
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh.scan[threadIdx.x >> 5] = sum;
  __syncthreads();
  u64 all = 0;
  for (int w = 0; w < kDrawWarps; ++w) all += sh.scan[w];
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
  for (int q = q0 + lane; q - lane < q1; q += 32) {
    Vec<T> v;
    u64 sum = 0;
    if (q < q1) {
      v = sl.load(q);
#pragma unroll
      for (int i = 0; i < Vec<T>::kN; ++i)
        if (sl.holds(q, i)) sum += amount(to_f32(v.e[i]), sl.id(q, i));
    }
    const u64 incl = warp_scan(sum, lane);
    const u64 all = __shfl_sync(0xffffffffu, incl, 31);
    if (target < at + all) {
      u64 mine = at + incl - sum;
      if (sum && mine <= target && target < mine + sum) {
        bool done = false;
#pragma unroll
        for (int i = 0; i < Vec<T>::kN; ++i) {
          if (done || !sl.holds(q, i)) continue;
          mine += amount(to_f32(v.e[i]), sl.id(q, i));
          if (target < mine) {
            f(to_f32(v.e[i]), sl.id(q, i));
            done = true;
          }
        }
      }
      return;
    }
    at += all;
  }
}

// Radix selection across the cluster, for rows whose candidates no bound thins out.  Every element from `old` on
// carries `amount` (1, or its weight); the cut is the order at which the amounts, from the first on, reach `need`
// >= 1 (at most what they carry together).  Ties are cut by id, CTA by CTA: the result holds for this CTA's ids.
template <typename T, bool WEIGHTED>
__device__ u64 radix_cut(const Slice<T>& sl, u64 need, u64 old, const Scale& sc, DrawShared& sh, uint32_t part) {
  const int tid = threadIdx.x;
  uint32_t prefix = 0, mask = 0;
  int round = 0;
  for (int bit = 24; bit >= 0; bit -= 8, ++round) {
    u64* hist = sh.digit[round & 1];
    hist[tid] = 0;
    __syncthreads();
    sl.each([&](const Vec<T>& f, int q) {
#pragma unroll
      for (int i = 0; i < Vec<T>::kN; ++i) {
        const float x = to_f32(f.e[i]);
        const uint32_t k = value_key(x);
        if ((k & mask) == prefix && sl.holds(q, i) && order_of(k, sl.id(q, i)) >= old)
          atomicAdd(&hist[(k >> bit) & 255], WEIGHTED ? weight(x, sc, sh.pow2) : 1ull);
      }
    });
    cluster_sync();  // every CTA's histogram is in place
    u64 all = 0;
#pragma unroll
    for (int c = 0; c < kRowSplit; ++c) all += ld_cluster(&hist[tid], c);
    sh.total[tid] = all;
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
  for (int c = 0; c < kRowSplit; ++c) {
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

template <typename T>
__global__ void __launch_bounds__(kDrawThreads, 4) filtered_draw_kernel(const DrawParams p) {
  extern __shared__ __align__(16) unsigned char s_raw[];
  DrawShared& sh = *reinterpret_cast<DrawShared*>(s_raw);
  const unsigned row = blockIdx.x / kRowSplit;
  const uint32_t part = cluster_ctarank();  // == blockIdx.x % kRowSplit
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int lo = min(p.V, static_cast<int>(part) * p.slice);
  const Slice<T> sl(static_cast<const T*>(p.logits) + row * static_cast<size_t>(p.stride), lo,
                    min(p.V, lo + p.slice) - lo);
  constexpr int N = Vec<T>::kN;

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

  // ---- the row maximum (NaN never is)
  float mx = -INFINITY;
  sl.each([&](const Vec<T>& f, int) { mx = fmaxf(mx, vec_max(f)); });

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
    const double k = 1.4426950408889634 / static_cast<double>(set.temp);
    sh.k_hi = static_cast<float>(fmin(k, 3.0e38));  // a T so small leaves the maximum alone either way
    sh.k_lo = k < 3.0e38 ? static_cast<float>(k - static_cast<double>(sh.k_hi)) : 0.f;
    sh.n_local = 0;
    sh.n_list[0] = sh.n_list[1] = 0;
    sh.tail = 0;
  }
  if (tid == 64 && set.use_m) {
    const double d = static_cast<double>(set.temp) * log(fmin(static_cast<double>(min_p), 1.0));
    sh.floor = d == d ? d : -INFINITY;  // an infinite T makes all ids alike
  }
  if (with_tail)
    for (int i = tid; i < kBins; i += kDrawThreads) sh.bins[i] = make_uint4(0, 0, 0, 0);

  // ---- what bounds the candidates from below
  // top-k: where every CTA has ceil(k / 8) groups of elements whose maxima reach a value, k elements do
  const int in_cta = (set.top_k + kRowSplit - 1) / kRowSplit;
  const bool small_k = in_cta <= kDrawThreads / 4;
  const bool bound_k = set.use_k && in_cta <= kDrawThreads / 2;
  if (bound_k) {
    const float g = small_k ? fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1)) : mx;
    if (!small_k) sh.group[tid] = g;
    else if ((tid & 1) == 0) sh.group[tid >> 1] = g;
  }
  const float wmx = warp_max(mx);
  if (lane == 0) sh.red[warp] = wmx;
  __syncthreads();
  float own_max = sh.red[0];
#pragma unroll
  for (int w = 1; w < kDrawWarps; ++w) own_max = fmaxf(own_max, sh.red[w]);
  if (with_tail) {  // top-p: the maxima's own mass is a lower bound of the whole
    const float e = warp_sum(mx > -INFINITY ? ex2((mx - own_max) * sh.k_hi) : 0.f);
    if (lane == 0) sh.red2[warp] = e;
    __syncthreads();
  }
  if (warp == 0) {
    float aux = -INFINITY;
    if (bound_k)
      aux = small_k ? jth_greatest<kDrawWarps / 2>(sh.group, in_cta, lane) : jth_greatest<kDrawWarps>(sh.group, in_cta, lane);
    if (with_tail) aux = warp_sum(lane < kDrawWarps ? sh.red2[lane] : 0.f);
    if (lane == 0) {
      sh.max = own_max;
      sh.aux = aux;
    }
  }
  cluster_sync();
  if (warp == 0) {
    const float cm = lane < kRowSplit ? ld_cluster(&sh.max, lane) : -INFINITY;
    const float ca = lane < kRowSplit ? ld_cluster(&sh.aux, lane) : INFINITY;
    const float m = warp_max(cm);
    float tau = -INFINITY;
    if (set.use_k) {
      tau = set.top_k == 1 ? m : -warp_max(-ca);
    } else if (set.use_p) {
      // mass below tau <= V exp((tau - m) / T) <= (1 - p) * mass
      const float z = warp_sum(cm > -INFINITY && lane < kRowSplit ? ca * ex2((cm - m) * sh.k_hi) : 0.f);
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
      sh.tau = fminf(tau, m);
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
  const float tau = sh.tau;
  u64 cut = 0;  // the order of the last id that stays
  bool cut_k = set.use_k, cut_p = set.use_p;  // still to be found
  if ((tau > -INFINITY || p.V <= kListCap) && !sc.inf) {
    const float scale = tau > -INFINITY && sc.m > tau ? static_cast<float>(kBins) / (sc.m - tau) * 0.9999f : 0.f;
    float rest = 0.f;
    sl.each([&](const Vec<T>& f, int q) {
      if (with_tail) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float x = to_f32(f.e[i]);
          const float e = ex2((x - sc.m) * sc.k_hi);
          rest += x < tau ? e : 0.f;
        }
      }
      if (vec_max(f) >= tau) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float x = to_f32(f.e[i]);
          if (x >= tau && sl.holds(q, i)) {
            const int at = atomicAdd(&sh.n_local, 1);
            if (at < kListCap) sh.local[at] = make_uint2(__float_as_uint(x), sl.id(q, i));
            if (with_tail) add_to_bin(&sh.bins[value_bin(x, sc.m, scale)], weight(x, sc, sh.pow2));
          }
        }
      }
    });
    if (with_tail) {
      const u64 t = block_total(static_cast<u64>(rest * 0x1p44f), sh);
      if (tid == 0) red_add_cluster(&sh.tail, 0, t);
    }
    int n = gather(sh, 0);
    bool fits = n <= kListCap;
    if (!fits && with_tail) {
      // the bin that holds top-p's border, found by the first CTA
      if (part == 0) {
        constexpr int kPer = kBins / kDrawThreads;
        u64 mass[kPer], sum = 0, all;
        int count[kPer], num = 0, n_all;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          mass[i] = 0;
          count[i] = 0;
          for (int c = 0; c < kRowSplit; ++c) {
            const uint4 b = ld_cluster(&sh.bins[tid * kPer + i], c);
            mass[i] += bin_mass(b);
            count[i] += static_cast<int>(b.x);
          }
          sum += mass[i];
          num += count[i];
        }
        u64 before = block_scan<u64, kDrawThreads>(sum, sh.scan, tid, &all) - sum;
        __syncthreads();
        int upto = block_scan<int, kDrawThreads>(num, reinterpret_cast<int*>(sh.scan), tid, &n_all) - num;
        const u64 need = min(set.top_p > 0.f ? max(share_of(set.top_p, all + sh.tail, true), 1ull) : 1ull, all);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          if (before < need && need <= before + mass[i]) {
            sh.bin = tid * kPer + i;
            sh.need = need - before;
            sh.n_upto = upto + count[i];
            sh.n_in = count[i];
            sh.total[0] = all + sh.tail - before - mass[i];  // below the bin
          }
          before += mass[i];
          upto += count[i];
        }
      }
      if (tid == 0) sh.n_local = 0;
      cluster_sync();
      const int bin = static_cast<int>(ld_cluster(reinterpret_cast<uint32_t*>(&sh.bin), 0));
      const int n_upto = static_cast<int>(ld_cluster(reinterpret_cast<uint32_t*>(&sh.n_upto), 0));
      const int n_in = static_cast<int>(ld_cluster(reinterpret_cast<uint32_t*>(&sh.n_in), 0));
      fits = n_upto <= kListCap;
      if (fits || n_in <= kListCap) {
        sl.each([&](const Vec<T>& f, int q) {
          if (!(vec_max(f) >= tau)) return;
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const float x = to_f32(f.e[i]);
            if (!(x >= tau) || !sl.holds(q, i)) continue;
            const int b = value_bin(x, sc.m, scale);
            if (b == bin || (fits && b < bin))
              sh.local[atomicAdd(&sh.n_local, 1)] = make_uint2(__float_as_uint(x), sl.id(q, i));
          }
        });
        n = gather(sh, 1);
        if (!fits) {  // the border's bin decides the border
          if (part == 0) {
            u64* wt = reinterpret_cast<u64*>(sh.local);
            const u64 need = sh.need;
            for (int e = tid; e < n; e += kDrawThreads) wt[e] = weight(__uint_as_float(sh.list[e].x), sc, sh.pow2);
            const float top = sc.m - static_cast<float>(bin) / scale;  // of the bin, which is binned again
            const u64 border = find_border<true, false>(ListView{sh.list, wt, n, 0}, need, top,
                                                        scale * static_cast<float>(kBins), 1, sh);
            if (tid == 0) sh.cut = border;
          }
          cluster_sync();
          cut = ld_cluster(&sh.cut, 0);
          cut_p = false;
        } else if (part == 0 && tid == 0) {
          sh.tail = sh.total[0];
        }
      }
    }
    if (fits) {
      if (part != 0) return;
      __syncthreads();
      finish_list(n, sh.tail, set, sc, p.V, sh, p.tokens + row, logp);
      cluster_sync();  // this CTA stays until the others, which read its counts, have left
      return;
    }
  }

  // ---- the cluster goes on together: what is left to cut
  if (cut_k) cut = radix_cut<T, false>(sl, static_cast<u64>(set.top_k), cut, sc, sh, part);
  auto kept_weight = [&](float x, uint32_t id) { return order_of(x, id) >= cut ? weight(x, sc, sh.pow2) : 0ull; };
  if (cut_p) {
    const u64 own = slice_total(sl, sh, kept_weight);
    if (tid == 0) sh.sum = own;
    cluster_sync();
    u64 all = 0;
    for (int c = 0; c < kRowSplit; ++c) all += ld_cluster(&sh.sum, c);
    cluster_sync();
    const u64 need = set.top_p > 0.f ? max(share_of(set.top_p, all, true), 1ull) : 1ull;
    cut = radix_cut<T, true>(sl, need, cut, sc, sh, part);
  }
  if (set.use_m) cut = max(cut, static_cast<u64>(value_key(sh.lowest)) << 32);

  // ---- the draw, in id order
  const u64 own = slice_total(sl, sh, kept_weight);
  if (tid == 0) sh.sum = own;
  cluster_sync();
  u64 all = 0, before = 0;
#pragma unroll
  for (int c = 0; c < kRowSplit; ++c) {
    const u64 n = ld_cluster(&sh.sum, c);
    if (c < static_cast<int>(part)) before += n;
    all += n;
  }
  cluster_arrive();  // done with the other CTAs' shared memory
  const u64 goal = share_of(set.u, all, false);
  if (before <= goal && goal < before + own)
    slice_locate(sl, goal - before, sh, kept_weight, [&](float x, uint32_t id) {
      p.tokens[row] = static_cast<int32_t>(id);
      if (logp) *logp = (sc.inf ? 0.f : (x - sc.m) / set.temp) - logf(static_cast<float>(all) * 0x1p-44f);
    });
  cluster_wait();
}

template <typename T>
static cudaError_t launch_draw(const DrawParams& p, int rows, cudaStream_t stream) {
  constexpr size_t smem = sizeof(DrawShared);
  cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(filtered_draw_kernel<T>), smem, false);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(rows) * kRowSplit);
  cfg.blockDim = dim3(kDrawThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kRowSplit;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, filtered_draw_kernel<T>, p);
  return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_filtered_draw(DrawParams p, int dtype, int rows, cudaStream_t stream) {
  if (rows <= 0 || rows > 0x7fffffff / kRowSplit) return cudaErrorInvalidValue;
  if (p.V > kMaxDrawVocab) return cudaErrorInvalidValue;
  p.slice = ((p.V + kRowSplit - 1) / kRowSplit + 7) & ~7;
  if (dtype == kF32) return launch_draw<float>(p, rows, stream);
  if (dtype == kBf16) return launch_draw<__nv_bfloat16>(p, rows, stream);
  return launch_draw<__half>(p, rows, stream);
}

}  // namespace dm
