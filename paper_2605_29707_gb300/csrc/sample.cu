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
  if (t < kCoarse) return static_cast<u64>(__float2uint_rn(exp2f(t + static_cast<float>(kWeightBits))));
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

struct DrawShared {
  u64 pow2[32];
  u64 mass[2][256];      // a round's histogram, by round parity (read by the cluster)
  u64 scan[kDrawThreads / 32];
  u64 sum;               // kept mass of this CTA (read by the cluster)
  u64 total[256];        // the cluster's histogram
  u64 need;
  float red[kDrawThreads / 32];
  float max;             // this CTA's maximum (read by the cluster)
  float k_hi, k_lo, floor;
  float m;
  uint32_t prefix;
  uint32_t equal;        // this CTA's elements at the cut (read by the cluster)
  int cut;
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
    const uint32_t b = (prefix & 0x80000000u) ? prefix & 0x7fffffffu : ~prefix;
    each = weight(__uint_as_float(b), sc, sh.pow2);
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
  const size_t set = row / p.rows_per_set;
  float temp = p.temperature ? __ldg(p.temperature + set) : 1.f;
  int top_k = p.top_k ? __ldg(p.top_k + set) : 0;
  const float top_p = p.top_p ? __ldg(p.top_p + set) : 1.f;
  const float min_p = p.min_p ? __ldg(p.min_p + set) : 0.f;
  if (!(temp > 0.f)) {  // greedy
    temp = 1.f;
    top_k = 1;
  }
  if (tid < 32) sh.pow2[tid] = c_pow2[tid];
  if (tid == 0) {
    const double k = 1.4426950408889634 / static_cast<double>(temp);
    sh.k_hi = static_cast<float>(fmin(k, 3.0e38));  // a T so small leaves the maximum alone either way
    sh.k_lo = k < 3.0e38 ? static_cast<float>(k - static_cast<double>(sh.k_hi)) : 0.f;
    sh.floor = -INFINITY;  // of x - max
  }

  // ---- the row maximum (NaN never is)
  cp_async_wait_all();
  __syncthreads();
  float mx = -INFINITY;
  for (int i = tid; i < len; i += kDrawThreads) mx = fmaxf(mx, to_f32(s[shift + i]));
  mx = warp_max(mx);
  if (lane == 0) sh.red[warp] = mx;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kDrawThreads / 32; ++w) mx = fmaxf(mx, sh.red[w]);
    sh.max = mx;
  }
  cluster_sync();
  if (warp == 0) {
    const float m = warp_max(lane < kRowSplit ? ld_cluster(&sh.max, lane) : -INFINITY);
    if (lane == 0) sh.m = m;
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

  // ---- the three cuts
  Cut cut{0u, len};
  if (top_k >= 1 && top_k < p.V)
    cut = radix_cut<T, false>(s, shift, len, static_cast<u64>(top_k), cut, sc, sh, part);
  if (top_p < 1.f) {
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
    // mass before < p * all, in integers: before < ceil(p * all)
    u64 need = 1;
    if (top_p > 0.f) {
      const u64 p64 = static_cast<u64>(static_cast<double>(top_p) * 18446744073709551616.0);
      need = __umul64hi(p64, all) + (p64 * all != 0);
    }
    cut = radix_cut<T, true>(s, shift, len, max(need, 1ull), cut, sc, sh, part);
  }
  if (min_p > 0.f) {
    if (tid == 0) {
      const double d = static_cast<double>(temp) * log(static_cast<double>(min_p));
      sh.floor = sc.inf ? INFINITY : __double2float_ru(fmin(static_cast<double>(sc.m) + d, static_cast<double>(sc.m)));
    }
    __syncthreads();
    const uint32_t key = value_key(sh.floor);
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
  float u = __ldg(p.uniforms + row);
  if (!(u >= 0.f)) u = 0.f;
  if (u >= 1.f) u = 0x1.fffffep-1f;  // the largest float below 1
  const u64 goal = __umul64hi(static_cast<u64>(static_cast<double>(u) * 18446744073709551616.0), all);
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
          const float z = sc.inf ? 0.f : (x - sc.m) / temp;
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
  const size_t smem = (static_cast<size_t>(p.slice) + 16) * sizeof(T);
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
