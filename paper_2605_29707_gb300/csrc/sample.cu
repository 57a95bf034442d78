// sample.cu -- one token per row of logits after temperature, top-k, top-p and min-p, drawn with the
// caller's uniform (the target's side of section 3.1 when it decodes with these filters).
//
// Mathematics.  With z = x / T and the ids ordered by (z descending, id ascending): the first k stay;
// of those, the ones whose predecessors in that order hold less than p of the mass; of those, the ones
// with exp(z - max z) >= min_p; the first always.  The token is the first kept id, in id order, whose
// cumulative mass exceeds u times the kept mass.
//
// Weights are integers: 2^44 exp(z - max z), rounded.  At most 2^19 of them fit 64 bits, so every sum
// is exact and the same in any order: splitting a row over CTAs, atomics and the order of threads
// change nothing.  Where a weight can move a border (above 2^-14 of the greatest) it is computed to
// about 2^-38 of its value (weight()), below that in fp32: a border then lies where 64-bit arithmetic
// puts it but for about 1e-11 of the mass.
//
// A cluster of eight CTAs holds a row in shared memory, one DRAM read.  The cut by top-k and the cut by
// top-p are each a radix selection over the order-preserving integer of the value, 8 bits a round,
// with a histogram of counts (top-k) or of weights (top-p) per CTA that the cluster adds up; ties at the
// cut are resolved by id from the CTAs' counts of them.  The draw scans the kept weights in id order.
#include <math.h>

#include "kernels.h"
#include "rows.cuh"

namespace dm {

constexpr int kDrawThreads = 512;
constexpr int kWeightBits = 44;    // the greatest weight is 2^44
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

// The order of preference as integers: greater value, greater key; -0 as +0, NaN last.
__device__ __forceinline__ uint32_t value_key(float x) { return x != x ? 0u : f32_ord(x + 0.f); }

__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float((k & 0x80000000u) ? k & 0x7fffffffu : ~k);
}

struct DrawShared {
  u64 pow2[32];
  u64 mass[2][256];      // a round's histogram, by round parity (read by the cluster)
  u64 scan[kDrawThreads / 32];
  u64 sum;               // kept mass of this CTA (read by the cluster)
  u64 total[256];        // the cluster's histogram
  u64 need;
  double floor;          // T log(min_p)
  float group[kDrawThreads];  // maxima of groups of threads
  float red[kDrawThreads / 32];
  float red2[kDrawThreads / 32];
  float max, aux;        // this CTA's maximum, and its bound on where the candidates begin (read by the cluster)
  float k_hi, k_lo;
  float m, tau;
  uint32_t prefix;
  int cut;
  uint32_t count[2];     // this CTA's candidates, before and after their bound is raised (read by the cluster)
  u64 tail[2];           // mass of its other ids (read by the cluster)
  int last_bin;
};

// The cut that a selection leaves: an element stays when its key is greater, or when it is equal and its
// place in this CTA's slice lies below `cut`.
struct Cut {
  uint32_t key;
  int at;
  __device__ __forceinline__ bool keeps(uint32_t k, int i) const { return k > key || (k == key && i < at); }
};

// Radix selection across the cluster.  Every element that `old` keeps carries `amount` (1, or its weight);
// the new cut keeps the elements whose predecessors in the order of preference carry less than `need`.
// The amounts of all of them add up to at least `need` >= 1.
template <typename T, bool WEIGHTED>
__device__ Cut radix_cut(const T* s, int shift, int len, u64 need, const Cut& old, const Scale& sc, DrawShared& sh,
                         uint32_t part) {
  const int tid = threadIdx.x;
  uint32_t prefix = 0, mask = 0;
  int round = 0;
  for (int bit = 24; bit >= 0; bit -= 8, ++round) {
    u64* hist = sh.mass[round & 1];
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    for (int i = tid; i < len; i += kDrawThreads) {
      const float x = to_f32(s[shift + i]);
      const uint32_t k = value_key(x);
      if ((k & mask) == prefix && old.keeps(k, i))
        atomicAdd(&hist[(k >> bit) & 255], WEIGHTED ? weight(x, sc, sh.pow2) : 1ull);
    }
    cluster_sync();  // every CTA's histogram is in place
    if (tid < 256) {
      u64 all = 0;
#pragma unroll
      for (int c = 0; c < kRowSplit; ++c) all += ld_cluster(&hist[tid], c);
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
          sh.prefix = prefix | (static_cast<uint32_t>(255 - (8 * tid + j)) << bit);
          sh.need = need - above;
        }
        above += mine[j];
      }
    }
    __syncthreads();
    prefix = sh.prefix;
    need = sh.need;
    mask |= 255u << bit;
  }
  // ties: `need` of what the equal elements carry goes to the ones of lowest id.  They weigh the same, so
  // the last histogram gives every CTA the number of them before its slice.
  const u64* hist = sh.mass[(round - 1) & 1];
  u64 each = 1;
  if (WEIGHTED) {
    each = weight(key_value(prefix), sc, sh.pow2);
  }
  const u64 count = (need + each - 1) / each;  // equal elements that stay, over the cluster
  u64 before = 0, own = 0;
#pragma unroll
  for (int c = 0; c < kRowSplit; ++c) {
    const u64 n = ld_cluster(&hist[prefix & 255], c) / each;
    if (c < static_cast<int>(part)) before += n;
    if (c == static_cast<int>(part)) own = n;
  }
  Cut cut{prefix, len};
  const long long stay = static_cast<long long>(count) - static_cast<long long>(before);
  if (stay <= 0) {
    cut.at = 0;
  } else if (stay < static_cast<long long>(own)) {  // the place of the stay-th equal element
    const int run = (len + kDrawThreads - 1) / kDrawThreads;
    const int i0 = min(len, tid * run), i1 = min(len, i0 + run);
    int n = 0;
    for (int i = i0; i < i1; ++i) {
      const uint32_t k = value_key(to_f32(s[shift + i]));
      n += k == prefix && old.keeps(k, i);
    }
    int all;
    int seen = block_scan<int, kDrawThreads>(n, reinterpret_cast<int*>(sh.scan), tid, &all) - n;
    if (seen < stay && stay <= seen + n) {
      for (int i = i0; i < i1; ++i) {
        const uint32_t k = value_key(to_f32(s[shift + i]));
        if (k == prefix && old.keeps(k, i) && ++seen == stay) sh.cut = i + 1;
      }
    }
    __syncthreads();
    cut.at = sh.cut;
  }
  if (old.key == prefix) cut.at = min(cut.at, old.at);
  cluster_sync();  // the histograms may be written again
  return cut;
}

// ------------------------------------------------------------------ few candidates: one CTA finishes the row
constexpr int kListCap = 2048;                            // candidates the cluster's first CTA can take
constexpr int kPerThread = kListCap / kDrawThreads;
constexpr int kBins = 512;                                // of the candidates' values
constexpr int kGroupsSmall = 128;                         // groups whose maxima bound the k-th greatest

// Bits of an element type's keys that say nothing (an order-preserving shift of the key drops them).
template <typename T>
constexpr int kKeyShift = sizeof(T) == 4 ? 0 : 13;
template <>
constexpr int kKeyShift<__nv_bfloat16> = 16;

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

// Radix selection within the block, over the list entries (4 a thread at most, in id order) that `kept` has bits
// for; `amount` as in radix_cut.  Returns the bits that stay.  `range`: the entries' keys differ in bits below it.
template <bool WEIGHTED>
__device__ __forceinline__ unsigned block_cut(const uint32_t (&key)[kPerThread], const u64 (&w)[kPerThread],
                                              unsigned kept, u64 need, int range, DrawShared& sh) {
  const int tid = threadIdx.x;
  uint32_t prefix = 0, mask = 0;
  int bit = range;
  while (bit > 0) {
    const int width = min(8, bit);
    bit -= width;
    u64* hist = sh.mass[0];
    __syncthreads();
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPerThread; ++i)
      if ((kept >> i & 1) && (key[i] & mask) == prefix)
        atomicAdd(&hist[(key[i] >> bit) & ((1u << width) - 1u)], WEIGHTED ? w[i] : 1ull);
    __syncthreads();
    if (tid < 32) {
      u64 mine[8], sum = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        mine[j] = hist[255 - (8 * tid + j)];
        sum += mine[j];
      }
      u64 above = warp_scan(sum, tid) - sum;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (above < need && need <= above + mine[j]) {
          sh.prefix = static_cast<uint32_t>(255 - (8 * tid + j)) << bit;
          sh.need = need - above;
        }
        above += mine[j];
      }
    }
    __syncthreads();
    prefix |= sh.prefix;
    need = sh.need;
    mask |= ((1u << width) - 1u) << bit;
  }
  // greater: stay; equal: the first in id order whose predecessors carry less than `need`
  unsigned stay = 0, equal = 0;
  u64 each = 0;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    if (!(kept >> i & 1)) continue;
    const uint32_t k = key[i] & mask;
    if (k > prefix) stay |= 1u << i;
    if (k == prefix) {
      equal |= 1u << i;
      each = WEIGHTED ? w[i] : 1ull;
    }
  }
  u64 all;
  const u64 own = each * __popc(equal);
  __syncthreads();
  u64 before = block_scan<u64, kDrawThreads>(own, sh.scan, tid, &all) - own;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i)
    if (equal >> i & 1) {
      if (before < need) stay |= 1u << i;
      before += each;
    }
  return stay;
}

__device__ __forceinline__ u64 share_of(float f, u64 all, bool up) {  // floor or ceil of f * all, 0 <= f < 1
  const u64 f64 = static_cast<u64>(static_cast<double>(f) * 18446744073709551616.0);
  return __umul64hi(f64, all) + (up && f64 * all != 0);
}

__device__ __forceinline__ float clamped_uniform(float u) {
  if (!(u >= 0.f)) return 0.f;
  return u >= 1.f ? 0x1.fffffep-1f : u;  // the largest float below 1
}

struct Settings {
  float temp, top_p, min_p, u;
  int top_k;
  bool use_k, use_p, use_m;
};

// The first CTA's end of a row: n candidates (values and ids, in id order), every id of the row that can stay among
// them; `tail`: the mass of the others, where top-p goes by it.
template <typename T>
__device__ void finish_list(const uint2* list, int n, u64 tail, const Settings& set, const Scale& sc, DrawShared& sh,
                            int32_t* token, float* logp) {
  const int tid = threadIdx.x;
  const int per = (n + kDrawThreads - 1) / kDrawThreads;  // <= kPerThread
  float x[kPerThread];
  uint32_t key[kPerThread];
  u64 w[kPerThread];
  unsigned kept = 0;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    const int at = tid * per + i;
    x[i] = -INFINITY;
    if (i < per && at < n) {
      x[i] = __uint_as_float(list[at].x);
      kept |= 1u << i;
    }
    key[i] = value_key(x[i]) >> kKeyShift<T>;
    w[i] = 0;
  }
  const int range = 32 - __clz((value_key(sc.m) >> kKeyShift<T>) ^ (value_key(sh.tau) >> kKeyShift<T>));
  if (set.use_k && set.top_k < n)
    kept = block_cut<false>(key, w, kept, static_cast<u64>(set.top_k), range, sh);
  u64 mine = 0;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i)
    if (kept >> i & 1) {
      w[i] = weight(x[i], sc, sh.pow2);
      mine += w[i];
    }
  if (set.use_p) {
    u64 all;
    __syncthreads();
    block_scan<u64, kDrawThreads>(mine, sh.scan, tid, &all);
    const u64 need = set.top_p > 0.f ? share_of(set.top_p, all + tail, true) : 0;
    if (need < all) kept = block_cut<true>(key, w, kept, max(need, 1ull), range, sh);
  }
  mine = 0;
  const float floor = set.use_m ? __double2float_ru(sc.m + sh.floor) : -INFINITY;
#pragma unroll
  for (int i = 0; i < kPerThread; ++i) {
    if (!(kept >> i & 1) || !(x[i] >= floor)) w[i] = 0;
    mine += w[i];
  }
  u64 all;
  __syncthreads();
  u64 at = block_scan<u64, kDrawThreads>(mine, sh.scan, tid, &all) - mine;
  const u64 goal = share_of(set.u, all, false);
  if (at <= goal && goal < at + mine) {
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
      if (at <= goal && goal < at + w[i]) {
        *token = static_cast<int32_t>(list[tid * per + i].y);
        if (logp) *logp = (x[i] - sc.m) / set.temp - logf(static_cast<float>(all) * 0x1p-44f);
      }
      at += w[i];
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kDrawThreads) filtered_draw_kernel(const DrawParams p) {
  extern __shared__ __align__(16) unsigned char s_raw[];
  __shared__ DrawShared sh;
  T* s = reinterpret_cast<T*>(s_raw);
  const size_t row = blockIdx.x / kRowSplit;
  const uint32_t part = cluster_ctarank();  // == blockIdx.x % kRowSplit
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int lo = min(p.V, static_cast<int>(part) * p.slice);
  const int len = min(p.V, lo + p.slice) - lo;
  const T* src = static_cast<const T*>(p.logits) + row * static_cast<size_t>(p.stride) + lo;
  const int shift = row_shift(src);
  stage_slice<T, kDrawThreads>(s, src, len, tid);

  // ---- the row's settings
  const unsigned at_set = static_cast<unsigned>(row) / p.rows_per_set;
  Settings set;
  set.temp = p.temperature ? __ldg(p.temperature + at_set) : 1.f;
  set.top_k = p.top_k ? __ldg(p.top_k + at_set) : 0;
  set.top_p = p.top_p ? __ldg(p.top_p + at_set) : 1.f;
  set.min_p = p.min_p ? __ldg(p.min_p + at_set) : 0.f;
  set.u = clamped_uniform(__ldg(p.uniforms + row));
  if (!(set.temp > 0.f)) {  // greedy
    set.temp = 1.f;
    set.top_k = 1;
  }
  set.use_k = set.top_k >= 1 && set.top_k < p.V;
  set.use_p = set.top_p < 1.f;
  set.use_m = set.min_p > 0.f;
  const int mask_words = (p.slice + 16 + 31) / 32;
  uint32_t* mask = reinterpret_cast<uint32_t*>(s + p.slice + 16);  // one bit per staged element: a candidate
  uint2* list = reinterpret_cast<uint2*>(mask + ((mask_words + 3) & ~3));
  for (int i = tid; i < mask_words; i += kDrawThreads) mask[i] = 0;
  if (tid < 32) sh.pow2[tid] = c_pow2[tid];
  if (tid == 0) {
    const double k = 1.4426950408889634 / static_cast<double>(set.temp);
    sh.k_hi = static_cast<float>(fmin(k, 3.0e38));  // a T so small leaves the maximum alone either way
    sh.k_lo = k < 3.0e38 ? static_cast<float>(k - static_cast<double>(sh.k_hi)) : 0.f;
    const double d = set.use_m ? static_cast<double>(set.temp) * log(fmin(static_cast<double>(set.min_p), 1.0)) : 0.0;
    sh.floor = d == d ? d : -INFINITY;  // an infinite T makes all ids alike
  }

  // ---- the row maximum (NaN never is), and what bounds the candidates from below
  cp_async_wait_all();
  __syncthreads();
  constexpr int N = Vec<T>::kN;
  const Vec<T>* v = reinterpret_cast<const Vec<T>*>(s);
  const int units = row_units<T>(shift, len);
  float mx = -INFINITY;
  for (int q = tid; q < units; q += kDrawThreads) {
    Vec<T> f;
    f.raw = v[q].raw;
    mx = fmaxf(mx, vec_max(f));
  }
  // top-k: where every CTA has ceil(k / 8) groups of elements whose maxima reach a value, k elements do
  const int in_cta = (set.top_k + kRowSplit - 1) / kRowSplit;
  const bool small_k = in_cta <= kGroupsSmall / 2;
  const bool bound_k = set.use_k && in_cta <= kDrawThreads / 2;
  if (bound_k) {
    float g = mx;
    if (small_k) {
      g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 1));
      g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, 2));
      if ((tid & 3) == 0) sh.group[tid >> 2] = g;
    } else {
      sh.group[tid] = g;
    }
  }
  const float wmx = warp_max(mx);
  if (lane == 0) sh.red[warp] = wmx;
  __syncthreads();
  float own_max = sh.red[0];
#pragma unroll
  for (int w = 1; w < kDrawThreads / 32; ++w) own_max = fmaxf(own_max, sh.red[w]);
  if (set.use_p && !set.use_k) {  // top-p: the maxima's own mass is a lower bound of the whole
    float e = warp_sum(mx > -INFINITY ? ex2((mx - own_max) * sh.k_hi) : 0.f);
    if (lane == 0) sh.red2[warp] = e;
    __syncthreads();
  }
  if (warp == 0) {
    float aux = -INFINITY;
    if (bound_k)
      aux = small_k ? jth_greatest<kGroupsSmall / 32>(sh.group, in_cta, lane)
                    : jth_greatest<kDrawThreads / 32>(sh.group, in_cta, lane);
    if (set.use_p && !set.use_k) aux = warp_sum(lane < kDrawThreads / 32 ? sh.red2[lane] : 0.f);
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
    if (set.use_m && !(set.use_k && set.use_p)) tau = fmaxf(tau, __double2float_rd(m + sh.floor));
    if (lane == 0) {
      sh.m = m;
      sh.tau = fminf(tau, m);
    }
  }
  __syncthreads();
  const Scale sc{sh.m, sh.k_hi, sh.k_lo, sh.m == INFINITY};
  if (sc.m == -INFINITY) {  // nothing to draw from: the same in every CTA of the cluster
    if (part == 0 && tid == 0) {
      p.tokens[row] = 0;
      if (p.logp) p.logp[row] = -INFINITY;
    }
    cluster_sync();  // no CTA leaves while another may still read its maximum
    return;
  }

  // ---- the candidates: marked in every slice, gathered by the first CTA if they are few
  const float tau = sh.tau;
  if ((tau > -INFINITY || p.V <= kListCap) && !sc.inf) {
    const bool with_tail = set.use_p && !set.use_k;
    float rest = 0.f;
    for (int q = tid; q < units; q += kDrawThreads) {
      Vec<T> f;
      f.raw = v[q].raw;
      if (with_tail) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float x = to_f32(f.e[i]);
          const float e = ex2((x - sc.m) * sc.k_hi);
          rest += x < tau ? e : 0.f;
        }
      }
      if (vec_max(f) >= tau) {
        unsigned bits = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int at = q * N + i - shift;
          if (to_f32(f.e[i]) >= tau && at >= 0 && at < len) bits |= 1u << i;
        }
        if (bits) atomicOr(&mask[q * N / 32], bits << (q * N % 32));
      }
    }
    __syncthreads();
    const int words = (units * N + 31) / 32;
    const int per = (words + kDrawThreads - 1) / kDrawThreads;
    int place = 0, n = 0;
    u64 tail = 0;
    bool fits = false;
    for (int round = 0; round < 2; ++round) {
      int mine = 0;
      for (int i = tid * per; i < min(words, tid * per + per); ++i) mine += __popc(mask[i]);
      int own;
      place = block_scan<int, kDrawThreads>(mine, reinterpret_cast<int*>(sh.scan), tid, &own) - mine;
      __syncthreads();
      if (with_tail && round == 0) {
        u64 t;
        block_scan<u64, kDrawThreads>(static_cast<u64>(rest * 0x1p44f), sh.scan, tid, &t);
        if (tid == 0) sh.tail[0] = t;
      }
      if (tid == 0) sh.count[round] = static_cast<uint32_t>(own);
      cluster_sync();
      int before = 0;
      n = 0;
      tail = 0;
#pragma unroll
      for (int c = 0; c < kRowSplit; ++c) {
        const int y = static_cast<int>(ld_cluster(&sh.count[round], c));
        if (c < static_cast<int>(part)) before += y;
        n += y;
        if (with_tail) tail += ld_cluster(&sh.tail[round], c);
      }
      place += before;
      fits = n <= kListCap;
      if (fits || !with_tail || round) break;

      // top-p with too many candidates: count them by value, and raise tau to where the mass above it surely holds
      // the share.  A bin's mass lies between its count times the weights at its two ends.
      uint32_t* bins = reinterpret_cast<uint32_t*>(sh.mass);
      const float scale = static_cast<float>(kBins) / (sc.m - tau) * 0.9999f;
      if (tid < kBins) bins[tid] = 0;
      __syncthreads();
      for (int i = tid; i < words; i += kDrawThreads)
        for (uint32_t w = mask[i]; w; w &= w - 1) {
          const float x = to_f32(s[i * 32 + __ffs(w) - 1]);
          atomicAdd(&bins[static_cast<int>((sc.m - x) * scale)], 1u);
        }
      cluster_sync();
      uint32_t count = 0;
      for (int c = 0; c < kRowSplit; ++c) count += ld_cluster(&bins[tid], c);
      const float hi_w = ex2(-static_cast<float>(tid) / scale * sc.k_hi);
      const float lo_w = ex2(-static_cast<float>(tid + 1) / scale * sc.k_hi);
      if (tid == 0) sh.last_bin = kBins - 1;
      u64 hi_all, lo_all;
      __syncthreads();
      const u64 hi = block_scan<u64, kDrawThreads>(static_cast<u64>(static_cast<float>(count) * hi_w * 0x1p40f), sh.scan,
                                                   tid, &hi_all);
      __syncthreads();
      const u64 lo = block_scan<u64, kDrawThreads>(static_cast<u64>(static_cast<float>(count) * lo_w * 0x1p40f), sh.scan,
                                                   tid, &lo_all);
      const float below = static_cast<float>(hi_all - hi + (tail >> 4));
      if ((1.f - set.top_p) * static_cast<float>(lo) >= 1.001f * set.top_p * below) atomicMin(&sh.last_bin, tid);
      __syncthreads();
      const int last_bin = sh.last_bin;
      u64 mid = 0, t;
      for (int i = tid; i < words; i += kDrawThreads) {
        uint32_t left = 0;
        for (uint32_t w = mask[i]; w; w &= w - 1) {
          const float x = to_f32(s[i * 32 + __ffs(w) - 1]);
          if (static_cast<int>((sc.m - x) * scale) <= last_bin) left |= w & -w;
          else mid += weight(x, sc, sh.pow2);
        }
        mask[i] = left;
      }
      block_scan<u64, kDrawThreads>(mid, sh.scan, tid, &t);
      if (tid == 0) sh.tail[1] = sh.tail[0] + t;
      __syncthreads();
    }
    if (fits) {
      for (int i = tid * per; i < min(words, tid * per + per); ++i)
        for (uint32_t w = mask[i]; w; w &= w - 1) {
          const int e = i * 32 + __ffs(w) - 1;
          st_cluster(&list[place++], 0, make_uint2(__float_as_uint(to_f32(s[e])), static_cast<uint32_t>(lo + e - shift)));
        }
      cluster_sync();
      if (part == 0)
        finish_list<T>(list, n, tail, set, sc, sh, p.tokens + row, p.logp ? p.logp + row : nullptr);
      return;
    }
    cluster_sync();  // done with the counts before their memory is used again
  }

  // ---- the three cuts
  Cut cut{0u, len};
  if (set.use_k) cut = radix_cut<T, false>(s, shift, len, static_cast<u64>(set.top_k), cut, sc, sh, part);
  if (set.use_p) {
    u64 mine = 0;
    for (int i = tid; i < len; i += kDrawThreads) {
      const float x = to_f32(s[shift + i]);
      if (cut.keeps(value_key(x), i)) mine += weight(x, sc, sh.pow2);
    }
    u64 sum;
    block_scan<u64, kDrawThreads>(mine, sh.scan, tid, &sum);
    if (tid == 0) sh.sum = sum;
    cluster_sync();
    u64 all = 0;
    for (int c = 0; c < kRowSplit; ++c) all += ld_cluster(&sh.sum, c);
    cluster_sync();
    const u64 need = set.top_p > 0.f ? share_of(set.top_p, all, true) : 0;
    cut = radix_cut<T, true>(s, shift, len, max(need, 1ull), cut, sc, sh, part);
  }
  if (set.use_m) {
    const float floor = sc.inf ? INFINITY : __double2float_ru(sc.m + sh.floor);
    const uint32_t key = value_key(floor);
    if (key > cut.key) cut = Cut{key, len};
  }

  // ---- the draw, in id order
  const int run = ((len + kDrawThreads - 1) / kDrawThreads) | 1;
  const int i0 = min(len, tid * run), i1 = min(len, i0 + run);
  u64 mine = 0;
  for (int i = i0; i < i1; ++i) {
    const float x = to_f32(s[shift + i]);
    if (cut.keeps(value_key(x), i)) mine += weight(x, sc, sh.pow2);
  }
  u64 sum;
  const u64 incl = block_scan<u64, kDrawThreads>(mine, sh.scan, tid, &sum);
  if (tid == 0) sh.sum = sum;
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
  u64 at = before + incl - mine;
  if (mine && at <= goal && goal < at + mine) {
    for (int i = i0; i < i1; ++i) {
      const float x = to_f32(s[shift + i]);
      if (!cut.keeps(value_key(x), i)) continue;
      const u64 w = weight(x, sc, sh.pow2);
      at += w;
      if (goal < at) {
        p.tokens[row] = lo + i;
        if (p.logp) {
          const float z = sc.inf ? 0.f : (x - sc.m) / set.temp;
          p.logp[row] = z - logf(static_cast<float>(all) * 0x1p-44f);
        }
        break;
      }
    }
  }
  cluster_wait();
}

template <typename T>
static cudaError_t launch_draw(const DrawParams& p, int rows, cudaStream_t stream) {
  const int mask_words = (p.slice + 16 + 31) / 32;
  const size_t smem = (static_cast<size_t>(p.slice) + 16) * sizeof(T) + ((mask_words + 3) & ~3) * 4 + kListCap * 8;
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
  p.slice = ((p.V + kRowSplit - 1) / kRowSplit + 7) & ~7;
  if (p.V > kMaxRowVocab) return cudaErrorInvalidValue;
  if (dtype == kF32) return launch_draw<float>(p, rows, stream);
  if (dtype == kBf16) return launch_draw<__nv_bfloat16>(p, rows, stream);
  return launch_draw<__half>(p, rows, stream);
}

}  // namespace dm
