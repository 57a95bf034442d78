// distill.cu -- distillation of a teacher's top logits into rows of student logits: the loss of every
// row, its gradient, or both in one pass over the logits.
//
// Mathematics.  Row x[V], temperature T, z = x / T, list (id_j, t_j), j < kt (a negative id is an empty
// place), weight w, upstream gradient g.  p = softmax(z); q_j = softmax(t / T) over the list, and nothing
// for the other ids ("renorm"), or q_j = exp(t_j) and rest = max(0, 1 - sum q) for all other ids together
// ("tail").  With log Z the log-sum-exp of z over every id, log R over the ids not listed:
//   loss     = w [ sum_j q_j (log q_j - z_j + log Z) + rest (log rest - log R + log Z) ]
//   dx_v     = (g w / T) [ exp(z_v - log Z) - sum_{j: id_j = v} q_j ]                       v listed
//            = (g w / T) exp(z_v - log R) [ R / Z - rest ]                                  v not listed
// The sum over the ids not listed is taken directly, with its own maximum: 1 - sum p_j would lose it where
// the student agrees with the teacher.  Terms with q = 0 or rest = 0 are 0; a row of weight 0 has loss and
// gradient 0 whatever its logits hold.
//
// Bound by DRAM.  For the loss, and for loss and gradient together, a cluster of eight CTAs holds the row
// in shared memory: every logit is read once, and written once as a gradient.  The gradient alone, from the
// two sums that the loss left, is one pass without a cluster.
#include <math.h>

#include "kernels.h"
#include "rows.cuh"

namespace dm {

constexpr int kDistillThreads = 256;
constexpr int kGradThreads = 256;
constexpr int kGradChunk = 16384;  // elements of a row per CTA of the gradient pass
static_assert(kMaxTeacher <= kDistillThreads && kMaxTeacher <= kGradThreads, "one list entry a thread");

// Sum over the block in a fixed order; `s` holds one value a warp.
template <int THREADS>
__device__ __forceinline__ float block_sum(float v, float* s, int tid) {
  v = warp_sum(v);
  __syncthreads();
  if ((tid & 31) == 0) s[tid >> 5] = v;
  __syncthreads();
  float all = 0.f;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) all += s[w];
  return all;
}
template <int THREADS>
__device__ __forceinline__ float block_max(float v, float* s, int tid) {
  v = warp_max(v);
  __syncthreads();
  if ((tid & 31) == 0) s[tid >> 5] = v;
  __syncthreads();
  float all = s[0];
#pragma unroll
  for (int w = 1; w < THREADS / 32; ++w) all = fmaxf(all, s[w]);
  return all;
}

// One place of the teacher's list, thread j's.
struct Place {
  int id;       // -1: empty, or past the list
  float x;      // the student's logit
  float q;      // the teacher's probability
  bool first;   // no earlier place has the same id
  float q_all;  // first: the sum of q over the places with this id
};

// Reads the row's list (thread j < kt: place j; the logits of ids in [lo, hi) alone) and gives the
// teacher's mass outside it.  s_id, s_q: [kt].
template <typename T, int THREADS>
__device__ __forceinline__ Place teacher_place(const DistillParams& p, size_t row, const T* x, int lo, int hi, int* s_id,
                                               float* s_q, float* s_red, float* rest) {
  const int tid = threadIdx.x;
  Place e{-1, -INFINITY, 0.f, false, 0.f};
  float t = -INFINITY;
  if (tid < p.kt) {
    const int id = __ldg(p.ids + row * p.kt + tid);
    if (id >= 0 && id < p.V) {
      e.id = id;
      t = __ldg(p.scores + row * p.kt + tid);
      if (id >= lo && id < hi) e.x = to_f32(x[id]);
    }
  }
  if (p.tail) {
    e.q = expf(t);
  } else {
    t *= p.inv_t;
    const float top = block_max<THREADS>(t, s_red, tid);
    e.q = t > -INFINITY ? expf(t - top) : 0.f;
  }
  const float sum = block_sum<THREADS>(e.q, s_red, tid);
  if (p.tail) {
    *rest = fmaxf(0.f, 1.f - sum);
  } else {
    e.q = sum > 0.f ? e.q / sum : 0.f;
    *rest = 0.f;
  }
  if (tid < p.kt) {
    s_id[tid] = e.id;
    s_q[tid] = e.q;
  }
  __syncthreads();
  if (e.id >= 0) {
    e.first = true;
    for (int j = 0; j < p.kt; ++j) {
      if (s_id[j] != e.id) continue;
      if (j < tid) e.first = false;
      e.q_all += s_q[j];
    }
  }
  if (p.tail && p.kt >= p.V && __syncthreads_count(e.first) == p.V) *rest = 0.f;  // every id is listed
  return e;
}

template <typename T, bool GRAD>
__global__ void __launch_bounds__(kDistillThreads) distill_kernel(const DistillParams p) {
  extern __shared__ __align__(16) unsigned char s_raw[];
  __shared__ int s_id[kMaxTeacher];
  __shared__ float s_q[kMaxTeacher];
  __shared__ float s_red[kDistillThreads / 32];
  __shared__ float s_part;     // this CTA's maximum, then (s_part2) its sum: read by the cluster
  __shared__ float s_part2;
  T* s = reinterpret_cast<T*>(s_raw);
  constexpr int N = Vec<T>::kN;
  const size_t row = blockIdx.x / kRowSplit;
  const uint32_t part = cluster_ctarank();  // == blockIdx.x % kRowSplit
  const int tid = threadIdx.x;
  const int lo = min(p.V, static_cast<int>(part) * p.slice);
  const int len = min(p.V, lo + p.slice) - lo;
  const T* x = static_cast<const T*>(p.logits) + row * static_cast<size_t>(p.stride);
  const int shift = row_shift(x + lo);
  const int units = row_units<T>(shift, len);
  stage_slice<T, kDistillThreads>(s, x + lo, len, tid);
  const float w = p.weights ? __ldg(p.weights + row) : 1.f;
  float rest;
  const Place e = teacher_place<T, kDistillThreads>(p, row, x, 0, p.V, s_id, s_q, s_red, &rest);
  cp_async_wait_all();
  __syncthreads();

  // ---- the listed ids leave the slice: what is left is the rest
  T none;
  from_f32(-INFINITY, &none);
  if (e.id >= lo && e.id < lo + len) s[shift + e.id - lo] = none;
  __syncthreads();
  const Vec<T>* v = reinterpret_cast<const Vec<T>*>(s);
  float mx = -INFINITY;
  for (int q = tid; q < units; q += kDistillThreads) {
    Vec<T> f;
    f.raw = v[q].raw;
#pragma unroll
    for (int i = 0; i < N; ++i) mx = fmaxf(mx, to_f32(f.e[i]));
  }
  mx = block_max<kDistillThreads>(mx, s_red, tid);
  if (tid == 0) s_part = mx;
  cluster_sync();
  float m = -INFINITY;  // of the ids not listed
#pragma unroll
  for (int c = 0; c < kRowSplit; ++c) m = fmaxf(m, ld_cluster(&s_part, c));
  const float base = m > -INFINITY ? m : 0.f;
  float sum = 0.f;
  for (int q = tid; q < units; q += kDistillThreads) {
    Vec<T> f;
    f.raw = v[q].raw;
#pragma unroll
    for (int i = 0; i < N; ++i) sum += ex2((to_f32(f.e[i]) - base) * p.k2);
  }
  sum = block_sum<kDistillThreads>(sum, s_red, tid);
  if (tid == 0) s_part2 = sum;
  cluster_sync();
  float r = 0.f;  // sum over the ids not listed, relative to their maximum
#pragma unroll
  for (int c = 0; c < kRowSplit; ++c) r += ld_cluster(&s_part2, c);
  cluster_arrive();  // done with the other CTAs' shared memory

  // ---- every id: the rest and the listed ones, relative to the row's maximum
  const float top = block_max<kDistillThreads>(fmaxf(e.x, m), s_red, tid);
  const bool empty = !(top > -INFINITY) && !isnan(top);  // every logit is -inf
  const float ref = empty ? 0.f : top;
  const float mine = e.first ? ex2((e.x - ref) * p.k2) : 0.f;
  const float listed = block_sum<kDistillThreads>(mine, s_red, tid);
  const float m_top = m > -INFINITY ? m - ref : 0.f;
  const float r_top = r * ex2(m_top * p.k2);
  const float z = r_top + listed;
  const float log_z = logf(z);  // relative to ref
  const float log_r = m_top * p.inv_t + logf(r);
  if (part == 0) {
    float l = 0.f;
    if (e.q > 0.f) l = empty ? INFINITY : e.q * (logf(e.q) - ((e.x - ref) * p.inv_t - log_z));
    l = block_sum<kDistillThreads>(l, s_red, tid);
    if (tid == 0) {
      if (rest > 0.f) l += empty ? INFINITY : rest * (logf(rest) - (log_r - log_z));
      p.loss[row] = w == 0.f ? 0.f : w * l;
      if (p.lse) {
        p.lse[2 * row] = empty ? -INFINITY : ref * p.inv_t + log_z;
        p.lse[2 * row + 1] = ref * p.inv_t + log_r;
      }
    }
  }
  if (GRAD) {
    const float up = p.grad_loss ? __ldg(p.grad_loss + row) : 1.f;
    const float scale = w == 0.f ? 0.f : up * w * p.inv_t;
    const float inv_z = z == 0.f ? 0.f : 1.f / z;
    // exp(z_v - log R) (R / Z - rest), with 2^((x - base) k2) = exp(z_v - log R) r
    const float a = r == 0.f ? 0.f : scale * (r_top * inv_z - rest) / r;
    T* dx = static_cast<T*>(p.dlogits) + row * static_cast<size_t>(p.grad_stride) + lo;
    const bool zero = w == 0.f;
    auto grad = [&](T xv) {
      T g;
      from_f32(zero ? 0.f : a * ex2((to_f32(xv) - base) * p.k2), &g);
      return g;
    };
    if (row_shift(dx) == shift) {
      for (int q = tid; q < units; q += kDistillThreads) {
        Vec<T> f, g;
        f.raw = v[q].raw;
#pragma unroll
        for (int i = 0; i < N; ++i) g.e[i] = grad(f.e[i]);
        const int i0 = q * N - shift;
        if (i0 >= 0 && i0 + N <= len) {
          *reinterpret_cast<uint4*>(dx + i0) = g.raw;
        } else {
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (i0 + i >= 0 && i0 + i < len) dx[i0 + i] = g.e[i];
        }
      }
    } else {
      for (int i = tid; i < len; i += kDistillThreads) dx[i] = grad(s[shift + i]);
    }
    __syncthreads();  // the listed ids' places are written again
    if (e.first && e.id >= lo && e.id < lo + len) {
      T g;
      from_f32(zero ? 0.f : scale * (mine * inv_z - e.q_all), &g);
      dx[e.id - lo] = g;
    }
  }
  cluster_wait();
}

// The gradient from the sums that the loss left: one CTA per chunk of a row.
template <typename T>
__global__ void __launch_bounds__(kGradThreads) distill_grad_kernel(const DistillParams p, int chunks) {
  __shared__ int s_id[kMaxTeacher];
  __shared__ float s_q[kMaxTeacher];
  __shared__ float s_red[kGradThreads / 32];
  constexpr int N = Vec<T>::kN;
  const size_t row = blockIdx.x / chunks;
  const int tid = threadIdx.x;
  const int lo = static_cast<int>(blockIdx.x % chunks) * kGradChunk;
  const int len = min(p.V - lo, kGradChunk);
  const T* x = static_cast<const T*>(p.logits) + row * static_cast<size_t>(p.stride);
  T* dx = static_cast<T*>(p.dlogits) + row * static_cast<size_t>(p.grad_stride) + lo;
  const float w = p.weights ? __ldg(p.weights + row) : 1.f;
  if (w == 0.f) {
    T none;
    from_f32(0.f, &none);
    for (int i = tid; i < len; i += kGradThreads) dx[i] = none;
    return;
  }
  float rest;
  const Place e = teacher_place<T, kGradThreads>(p, row, x, lo, lo + len, s_id, s_q, s_red, &rest);
  __syncthreads();  // the listed logits are read before any gradient is written (they may share memory)
  const float lse = p.lse[2 * row], lse_rest = p.lse[2 * row + 1];
  const float scale = (p.grad_loss ? __ldg(p.grad_loss + row) : 1.f) * w * p.inv_t;
  const bool some = lse_rest > -INFINITY || isnan(lse_rest);
  const float a = some ? scale * (expf(lse_rest - lse) - rest) : 0.f;
  const float base = some ? lse_rest : 0.f;
  auto grad = [&](T xv) {
    T g;
    from_f32(some ? a * expf(fmaf(to_f32(xv), p.inv_t, -base)) : 0.f, &g);
    return g;
  };
  x += lo;
  const int shift = row_shift(x);
  if (row_shift(dx) == shift) {
    const int units = row_units<T>(shift, len);
    for (int q = tid; q < units; q += kGradThreads) {
      const int i0 = q * N - shift;
      if (i0 >= 0 && i0 + N <= len) {
        Vec<T> f, g;
        f.raw = *reinterpret_cast<const uint4*>(x + i0);
#pragma unroll
        for (int i = 0; i < N; ++i) g.e[i] = grad(f.e[i]);
        *reinterpret_cast<uint4*>(dx + i0) = g.raw;
      } else {
        for (int i = max(0, i0); i < min(len, i0 + N); ++i) dx[i] = grad(x[i]);
      }
    }
  } else {
    for (int i = tid; i < len; i += kGradThreads) dx[i] = grad(x[i]);
  }
  __syncthreads();  // the listed ids' places are written again
  if (e.first && e.id >= lo && e.id < lo + len) {
    const float pv = lse > -INFINITY || isnan(lse) ? expf(fmaf(e.x, p.inv_t, -lse)) : 0.f;
    T g;
    from_f32(scale * (pv - e.q_all), &g);
    dx[e.id - lo] = g;
  }
}

template <typename T, bool GRAD>
static cudaError_t launch_rows(const DistillParams& p, int rows, cudaStream_t stream) {
  const size_t smem = (static_cast<size_t>(p.slice) + 16) * sizeof(T);
  cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(distill_kernel<T, GRAD>), smem, false);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(rows) * kRowSplit);
  cfg.blockDim = dim3(kDistillThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kRowSplit;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, distill_kernel<T, GRAD>, p);
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <typename T>
static cudaError_t launch_type(const DistillParams& p, int rows, cudaStream_t stream) {
  if (p.loss) return p.dlogits ? launch_rows<T, true>(p, rows, stream) : launch_rows<T, false>(p, rows, stream);
  const int chunks = (p.V + kGradChunk - 1) / kGradChunk;
  if (static_cast<long long>(rows) * chunks > 0x7fffffffLL) return cudaErrorInvalidValue;
  distill_grad_kernel<T><<<static_cast<unsigned>(rows) * chunks, kGradThreads, 0, stream>>>(p, chunks);
  return cudaGetLastError();
}

cudaError_t launch_distill(DistillParams p, int dtype, int rows, cudaStream_t stream) {
  if (rows <= 0 || rows > 0x7fffffff / kRowSplit) return cudaErrorInvalidValue;
  p.slice = ((p.V + kRowSplit - 1) / kRowSplit + 7) & ~7;
  if (p.V > kMaxDistillVocab) return cudaErrorInvalidValue;
  if (dtype == kF32) return launch_type<float>(p, rows, stream);
  if (dtype == kBf16) return launch_type<__nv_bfloat16>(p, rows, stream);
  return launch_type<__half>(p, rows, stream);
}

}  // namespace dm
