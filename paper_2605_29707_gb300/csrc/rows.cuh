// rows.cuh -- building blocks of the kernels that work on rows of vocabulary logits split over a
// cluster of CTAs (sample.cuh, distill.cu): element types, units of 16 bytes, accesses to the cluster's
// shared memory, and reductions and scans over a block.  The operators on a paged cache (cache.cu, attend.cu,
// attend_rows.cu) take the element types and units from here.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include "kernels.h"
#include "ptx.cuh"

namespace dm {

// ------------------------------------------------------------------ element types
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }

// One rounding, to nearest even, of a value computed in fp32 to the element type.
__device__ __forceinline__ void from_f32(float v, float* out) { *out = v; }
__device__ __forceinline__ void from_f32(float v, __nv_bfloat16* out) { *out = __float2bfloat16_rn(v); }
__device__ __forceinline__ void from_f32(float v, __half* out) { *out = __float2half_rn(v); }

template <typename T>
struct Vec {  // 16 bytes of elements
  static constexpr int kN = 16 / sizeof(T);
  union {
    uint4 raw;
    T e[kN];
  };
  __device__ __forceinline__ Vec() {}
  __device__ __forceinline__ Vec(const Vec& o) : raw(o.raw) {}
  __device__ __forceinline__ Vec& operator=(const Vec& o) {
    raw = o.raw;
    return *this;
  }
};

// 2^x by the special function unit (relative error below 2^-22; results below 2^-126 are 0).
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The unit's elements in fp32, and back with one rounding each (pairs of 16-bit elements share an instruction).
__device__ __forceinline__ void unpack(const Vec<float>& f, float (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = f.e[i];
}
__device__ __forceinline__ void unpack(const Vec<__nv_bfloat16>& f, float (&v)[8]) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(f.e);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack(const Vec<__half>& f, float (&v)[8]) {
  const __half2* h = reinterpret_cast<const __half2*>(f.e);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 t = __half22float2(h[i]);
    v[2 * i] = t.x;
    v[2 * i + 1] = t.y;
  }
}
__device__ __forceinline__ void pack(const float (&v)[4], Vec<float>* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) f->e[i] = v[i];
}
__device__ __forceinline__ void pack(const float (&v)[8], Vec<__nv_bfloat16>* f) {
  __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(f->e);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
}
__device__ __forceinline__ void pack(const float (&v)[8], Vec<__half>* f) {
  __half2* h = reinterpret_cast<__half2*>(f->e);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
}

// The greatest of the unit's elements; NaN never is (-inf if there is nothing else).
__device__ __forceinline__ float vec_max(const Vec<float>& f) {
  return fmaxf(fmaxf(f.e[0], f.e[1]), fmaxf(f.e[2], f.e[3]));
}
template <typename T, typename T2>
__device__ __forceinline__ float vec_max_pairs(const Vec<T>& f) {
  const T2* h = reinterpret_cast<const T2*>(f.e);
  const T2 a = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
  return fmaxf(to_f32(a.x), to_f32(a.y));
}
__device__ __forceinline__ float vec_max(const Vec<__nv_bfloat16>& f) {
  return vec_max_pairs<__nv_bfloat16, __nv_bfloat162>(f);
}
__device__ __forceinline__ float vec_max(const Vec<__half>& f) { return vec_max_pairs<__half, __half2>(f); }

// ------------------------------------------------------------------ units
// Elements between the 16-byte boundary at or below `src` and src itself.
template <typename T>
__device__ __forceinline__ int row_shift(const T* src) {
  return static_cast<int>((reinterpret_cast<uintptr_t>(src) & 15) / sizeof(T));
}

// Units of 16 bytes, aligned, that hold `len` elements from `shift` elements past a boundary on.
template <typename T>
__device__ __forceinline__ int row_units(int shift, int len) {
  return len > 0 ? (shift + len + Vec<T>::kN - 1) / Vec<T>::kN : 0;
}

// ------------------------------------------------------------------ clusters
__device__ __forceinline__ uint32_t ld_cluster(const uint32_t* local, uint32_t rank) {
  return ld_cluster_u32(cluster_addr(local, rank));
}
__device__ __forceinline__ float ld_cluster(const float* local, uint32_t rank) {
  return __uint_as_float(ld_cluster_u32(cluster_addr(local, rank)));
}
__device__ __forceinline__ unsigned long long ld_cluster(const unsigned long long* local, uint32_t rank) {
  unsigned long long v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(cluster_addr(local, rank)) : "memory");
  return v;
}

__device__ __forceinline__ void st_cluster(uint2* local, uint32_t rank, uint2 v) {
  asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(cluster_addr(local, rank)), "r"(v.x), "r"(v.y)
               : "memory");
}

__device__ __forceinline__ uint4 ld_cluster(const uint4* local, uint32_t rank) {
  uint4 v;
  asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(cluster_addr(local, rank))
               : "memory");
  return v;
}
__device__ __forceinline__ uint32_t atom_add_cluster(uint32_t* local, uint32_t rank, uint32_t v) {
  uint32_t old;
  asm volatile("atom.relaxed.cluster.shared::cluster.add.u32 %0, [%1], %2;"
               : "=r"(old)
               : "r"(cluster_addr(local, rank)), "r"(v)
               : "memory");
  return old;
}
__device__ __forceinline__ void red_add_cluster(unsigned long long* local, uint32_t rank, unsigned long long v) {
  asm volatile("red.relaxed.cluster.shared::cluster.add.u64 [%0], %1;" ::"r"(cluster_addr(local, rank)), "l"(v) : "memory");
}

// ------------------------------------------------------------------ block reductions and scans
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
template <typename I>
__device__ __forceinline__ I warp_scan(I v, int lane) {  // inclusive, integers
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const I y = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += y;
  }
  return v;
}

// Inclusive scan of one integer a thread, in thread order; *total: the block's sum.  `s` holds one
// value a warp; the caller's next use of it needs a barrier in between.
template <typename I, int THREADS>
__device__ __forceinline__ I block_scan(I v, I* s, int tid, I* total) {
  const int warp = tid >> 5, lane = tid & 31;
  I x = warp_scan(v, lane);
  if (lane == 31) s[warp] = x;
  __syncthreads();
  const I sums = warp_scan(lane < THREADS / 32 ? s[lane] : I(0), lane);  // every warp scans the warps' sums
  const I before = __shfl_sync(0xffffffffu, sums, warp > 0 ? warp - 1 : 0);
  *total = __shfl_sync(0xffffffffu, sums, 31);
  return warp > 0 ? x + before : x;
}

}  // namespace dm
