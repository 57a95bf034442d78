// distill.cu -- distillation of a teacher's top logits into rows of student logits: the loss of every
// row, its gradient, or both in one pass over the logits.
//
// Mathematics.  Row x[V], temperature T, z = x / T, list (id_j, t_j), j < kt (a negative id is an empty
// place), weight w, upstream gradient g.  p = softmax(z); q_j = softmax(t / T) over the list, and nothing
// for the other ids ("renorm"), or q_j = exp(t_j) and rest = max(0, 1 - sum q) for all other ids together
// ("tail").  With log Z the log-sum-exp of z over every id, log R over the ids not listed, Q = sum q + rest (1, but where
// the list teaches nothing, its probabilities add up to more, or every id is listed and they add up to less):
//   loss     = w [ sum_j q_j (log q_j - z_j + log Z) + rest (log rest - log R + log Z) ]
//   dx_v     = (g w / T) [ Q exp(z_v - log Z) - sum_{j: id_j = v} q_j ]                     v listed
//            = (g w / T) exp(z_v - log R) [ Q R / Z - rest ]                                v not listed
// The loss's terms are of the size of log Z and cancel where the student agrees with the teacher, so it is formed as
//   loss / w = sum_b q_b h(p_b / q_b - 1) + sum_b (q_b - p_b),   h(d) = d - log(1 + d) >= 0,
// b over the distinct listed ids (q_b: the sum of their places' q_j) and, with a tail, the rest; places that share an
// id add q_j log(q_j / q_b).  The second sum is 0 where a rest is left (everything on both sides), R / Z under renorm
// and sum q - 1 + R / Z without a rest.  1 - sum q, which is small where the teacher is sure of an id, is -expm1(t)
// of the list's greatest score less the q of the other places: good to its own size, not to that of 1.  Relative
// error of the loss of 151936 ids, T = 4, eight places: 1e-6; of the terms added as they stand 2e-3.
// The sum over the ids not listed is taken directly, with its own maximum: 1 - sum p_j would lose it where
// the student agrees with the teacher.  Terms with q = 0 or rest = 0 are 0; a row of weight 0 has loss and
// gradient 0 whatever its logits hold.
//
// The gradient alone is bound by DRAM; with the loss, many rows are bound by DRAM at six tenths of its rate and by the barriers
// around the list and the exchange, few rows by the chain of one.
// For the loss, and for loss and gradient together, a cluster of CTAs takes a row, a slice each.
// A thread keeps the maximum of what it reads and the sum relative to it; warps, the CTA and, with one exchange,
// the cluster join such pairs.  The teacher's list is one warp's work; the ids that it names are marked in shared
// memory, a bit an element, and pass for -inf on the way through.  The gradient reads the slice again, from L2:
// what is in flight on the chip (58 MB at V = 151936, bf16) fits it.  The gradient alone, from the two sums that the loss
// left, is one pass without a cluster, but for rows whose sums are too far from zero to tell their logits apart.
// What it measured (device time): loss and gradient of 4096 bf16 rows, V = 151936, 530 us, 4.7 TB/s (522 with the
// rest as 1 - sum q); with the slices held in shared memory, 38 KB and five CTAs an SM, 568 us, for there they could
// not be longer.  Slices from 64 KB on; from 32 KB 657 us, from 128 KB, which no longer fit L2, 636.  Vocabularies
// just below a power of two have the longest, up to 128 KB, 100 MB in flight: as many bytes at V = 65535, 131071 or
// 262143 take 615 us (540 at 140000).  Gradient alone of 512 fp32 rows 96.7 us, 6.4 TB/s, 0.95 of the measured copy
// rate, of 512 bf16 rows 61; loss of 1023 fp16 rows, V = 41511, 30.7 us; loss of 16 bf16 rows 8.1 us.  Gradient rows
// of another 16-byte alignment than the logits' are written element by element: 165 us for the 512 fp32 rows, and 390
// instead of 145 for loss and gradient of 1024 bf16 rows.  A list of 64 places costs 10 us in 90 (512 bf16 rows), of
// 256, where every place looks at every other, 97 in 177.
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

// Q, from the sum of the list's weights (as exponentials: their quotients by it are q under renorm).  A NaN shows.
__device__ __forceinline__ float teacher_mass(int tail, float sum, float rest) {
  if (tail) return rest > 0.f ? 1.f : sum;
  return sum == 0.f ? 0.f : sum / sum;
}

// What a list of log-probabilities leaves, 1 - sum q (negative where the q add up to more): `top` the greatest score,
// `others` the sum of q over all places but one that has it.
__device__ __forceinline__ float unlisted_mass(float top, float others) { return -expm1f(top) - others; }

// One place of the teacher's list, thread j's.
struct Place {
  int id;       // -1: empty, or past the list
  float x;      // the student's logit
  float q;      // the teacher's probability
  bool first;   // no earlier place has the same id
  float q_all;  // first: the sum of q over the places with this id
};

// The row's list, place j (thread j < kt) with what it holds; gives the teacher's mass outside it, and all of it.  The
// logits of ids in [lo, hi) alone are read.  s_id, s_q: [kt].
template <typename T, int THREADS>
__device__ __forceinline__ Place teacher_place(const DistillParams& p, int id, float score, const T* x, int lo, int hi,
                                               int* s_id, float* s_q, float* s_red, float* rest, float* mass) {
  const int tid = threadIdx.x;
  Place e{-1, -INFINITY, 0.f, false, 0.f};
  float t = -INFINITY;
  if (id >= 0 && id < p.V) {
    e.id = id;
    t = score;
    if (id >= lo && id < hi) e.x = to_f32(x[id]);
  }
  const float top = block_max<THREADS>(t, s_red, tid);
  float sum;
  if (p.tail) {
    e.q = expf(t);
    const int count = __syncthreads_count(t == top);
    float others = block_sum<THREADS>(t == top ? 0.f : e.q, s_red, tid);
    others += static_cast<float>(count - 1) * expf(top);
    sum = others + expf(top);
    *rest = fmaxf(0.f, unlisted_mass(top, others));
  } else {
    e.q = t > -INFINITY || isnan(t) ? expf((t - top) * p.inv_t) : 0.f;  // (a NaN score shows)
    sum = block_sum<THREADS>(e.q, s_red, tid);
    e.q = sum == 0.f ? 0.f : e.q / sum;
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
  *mass = teacher_mass(p.tail, sum, *rest);
  return e;
}

// A maximum and the sum of 2^((x - m) k2) over what it is the maximum of; m = -inf: nothing.
struct MaxSum {
  float m, s;
};
__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b, float k2) {
  const float m = fmaxf(a.m, b.m);
  // (a NaN sum stays one; an empty side adds nothing)
  const float sa = a.m == m ? a.s : a.s * ex2((a.m - m) * k2);
  const float sb = b.m == m ? b.s : b.s * ex2((b.m - m) * k2);
  return MaxSum{m, sa + sb};
}
__device__ __forceinline__ MaxSum warp_join(MaxSum v, float k2) {
#pragma unroll
  for (int o = 16; o; o >>= 1)
    v = join(v, MaxSum{__shfl_xor_sync(0xffffffffu, v.m, o), __shfl_xor_sync(0xffffffffu, v.s, o)}, k2);
  return v;
}

// 2^((x - base) k2) of a unit's elements, but for a factor that all of them share, exp_factor(base, k2).  fp32
// logits: the difference first, which keeps the argument to 2.5 roundings of itself; the factor is 1.  16-bit logits:
// one multiply-add with -base k2 rounded, one instruction less of ten.  What that rounding adds to every argument is
// known exactly, and the factor takes it out where the terms have been added up.  Beyond kFusedMost (a row of masked
// places alone: -1e10 times k2 is rounded by hundreds) the difference first, as for fp32; the rounding is 2^-9 at
// most below it.
constexpr float kFusedMost = 65536.f;
template <typename T>
__device__ __forceinline__ void unit_exp(const Vec<T>& f, float base, float k2, float (&e)[Vec<T>::kN]) {
  float x[Vec<T>::kN];
  unpack(f, x);
  const float c = -base * k2;
  if (sizeof(T) == 2 && fabsf(c) < kFusedMost) {
#pragma unroll
    for (int i = 0; i < Vec<T>::kN; ++i) e[i] = ex2(fmaf(x[i], k2, c));
  } else {
#pragma unroll
    for (int i = 0; i < Vec<T>::kN; ++i) e[i] = ex2((x[i] - base) * k2);
  }
}
template <typename T>
__device__ __forceinline__ float exp_factor(float base, float k2) {
  const float c = -base * k2;
  return sizeof(T) == 2 && fabsf(c) < kFusedMost ? ex2(-fmaf(base, k2, c)) : 1.f;
}

// q log(q / p) + p - q = q h(p / q - 1).  Near p = q by the series of log(1 + d) = 2 artanh(s), s = d / (2 + d): an error of
// p then counts by p - q alone; up to a factor of two by log1p; further off by the logarithms, p's being `log_p`.
__device__ __forceinline__ float excess(float q, float p, float log_p) {
  if (q == 0.f) return p;
  const float gap = p - q, d = gap / q;
  if (fabsf(gap) <= 0.25f * q) {  // |s| <= 1 / 7: the series' next term is below 2^-28 of h
    const float s = d / (2.f + d), s2 = s * s;
    return q * (s * d - 2.f * s * s2 * fmaf(s2, fmaf(s2, fmaf(s2, 1.f / 9.f, 1.f / 7.f), 1.f / 5.f), 1.f / 3.f));
  }
  return gap - q * (p > 0.5f * q && p < 2.f * q ? log1pf(d) : log_p - logf(q));
}

constexpr int kLanePlaces = kMaxTeacher / 32;  // places of the list that a lane of the list's warp has

constexpr int kDistillBatch = 4;  // 16-byte loads a thread has in flight

// A row's slice x[lo .. lo + len), in units of 16 bytes aligned in global memory; `listed` has a byte a unit, whose bits
// say which of its elements the teacher lists.
template <typename T>
struct Part {
  static constexpr int N = Vec<T>::kN;
  const T* src;
  int len, shift, units, first, last;
  const unsigned char* listed;
  __device__ __forceinline__ Part(const T* p, int n, const unsigned char* marks) : src(p), len(n), listed(marks) {
    shift = row_shift(p);
    units = row_units<T>(shift, len);
    first = shift ? 1 : 0;       // whole units: [first, last)
    last = (shift + len) / N;
  }
  // The listed elements, and what is not the row's, carry no weight.
  __device__ __forceinline__ void strike(Vec<T>* f, int q) const {
    const unsigned bits = listed[q];
    if (bits) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (bits >> i & 1) from_f32(-INFINITY, &f->e[i]);
    }
  }
  __device__ __forceinline__ Vec<T> edge(int q) const {
    Vec<T> f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = q * N + i - shift;
      if (at >= 0 && at < len) f.e[i] = src[at];
      else from_f32(-INFINITY, &f.e[i]);
    }
    return f;
  }
  // f(unit, index) for whole units, kDistillBatch loads of a thread at a time, and g(unit, index) for the first and
  // the last where they are not whole
  template <typename F, typename G>
  __device__ __forceinline__ void each(F&& f, G&& g) const {
    const uint4* unit = reinterpret_cast<const uint4*>(src - shift);
    Vec<T> v[kDistillBatch];
    for (int q = first + threadIdx.x; q < last; q += kDistillBatch * kDistillThreads) {
#pragma unroll
      for (int j = 0; j < kDistillBatch; ++j)
        if (q + j * kDistillThreads < last) v[j].raw = __ldcg(unit + q + j * kDistillThreads);
#pragma unroll
      for (int j = 0; j < kDistillBatch; ++j)
        if (q + j * kDistillThreads < last) {
          strike(&v[j], q + j * kDistillThreads);
          f(v[j], q + j * kDistillThreads);
        }
    }
    if (threadIdx.x < 2 && units > 0) {
      const int q = threadIdx.x == 0 ? 0 : last;
      if (threadIdx.x == 0 ? shift != 0 : last < units && (last > 0 || !shift)) {
        Vec<T> e = edge(q);
        strike(&e, q);
        g(e, q);
      }
    }
  }
};

template <typename T, int SP, bool GRAD>
__global__ void __launch_bounds__(kDistillThreads, 5) distill_kernel(const DistillParams p) {
  extern __shared__ __align__(16) unsigned char s_listed[];  // a byte a unit
  __shared__ int s_id[kMaxTeacher];
  __shared__ float s_q[kMaxTeacher], s_x[kMaxTeacher];  // later, in s_x, the listed ids' gradients
  __shared__ float s_all[kMaxTeacher];                  // the sum of q over the places with the place's id
  __shared__ MaxSum s_warp[kDistillThreads / 32];
  __shared__ MaxSum s_part[SP];  // every CTA's ids that are not listed (written by the cluster)
  __shared__ float s_a, s_base;
  constexpr int N = Vec<T>::kN;
  const unsigned row = blockIdx.x / SP;
  const uint32_t part = SP > 1 ? cluster_ctarank() : 0;  // == blockIdx.x % SP
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (SP > 1) cluster_arrive();  // this CTA runs: the others may store into its shared memory
  const int lo = min(p.V, static_cast<int>(part) * p.slice);
  const int len = min(p.V, lo + p.slice) - lo;
  const T* x = static_cast<const T*>(p.logits) + row * static_cast<size_t>(p.stride);
  const Part<T> slice(x + lo, len, s_listed);
  const int shift = slice.shift;
  if (tid == 32 && slice.last > slice.first)  // on its way into L2 while the list is read
    l2_prefetch_bulk(slice.src + (slice.first * N - shift), static_cast<uint32_t>(slice.last - slice.first) * 16);
  for (int i = tid; i < (slice.units + 4) / 4; i += kDistillThreads) reinterpret_cast<uint32_t*>(s_listed)[i] = 0;
  const float w = p.weights ? __ldg(p.weights + row) : 1.f;

  // ---- the teacher's list, by warp 0: the student's logits, the teacher's probabilities, and what it leaves to the rest
  float rest = 0.f, taught = 0.f, left = 0.f;  // (warp 0's) the teacher's mass outside and inside the list, 1 - inside
  const int places = (p.kt + 31) / 32;  // of a lane: 32 i + lane
  if (warp == 0) {
    float t[kLanePlaces], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kLanePlaces; ++i) {
      const int j = 32 * i + lane;
      t[i] = -INFINITY;
      if (j < p.kt) {
        const int id = __ldg(p.ids + row * static_cast<size_t>(p.kt) + j);
        const bool on = id >= 0 && id < p.V;
        if (on) t[i] = __ldg(p.scores + row * static_cast<size_t>(p.kt) + j);
        s_id[j] = on ? id : -1;
        s_x[j] = on ? to_f32(x[id]) : -INFINITY;
      }
      top = fmaxf(top, t[i]);
    }
    top = warp_max(top);
#pragma unroll
    for (int i = 0; i < kLanePlaces; ++i) {
      t[i] = t[i] > -INFINITY || isnan(t[i]) ? expf(p.tail ? t[i] : (t[i] - top) * p.inv_t) : 0.f;
      taught += t[i];
    }
    taught = warp_sum(taught);
    if (p.tail) {
      const float q_top = expf(top);
      float others = 0.f;
      int count = 0;
#pragma unroll
      for (int i = 0; i < kLanePlaces; ++i) {
        others += t[i] == q_top ? 0.f : t[i];
        count += __popc(__ballot_sync(0xffffffffu, t[i] == q_top));
      }
      left = unlisted_mass(top, warp_sum(others) + static_cast<float>(count - 1) * q_top);
      rest = fmaxf(0.f, left);
    }
#pragma unroll
    for (int i = 0; i < kLanePlaces; ++i)
      if (32 * i + lane < p.kt) s_q[32 * i + lane] = p.tail ? t[i] : (taught == 0.f ? 0.f : t[i] / taught);  // (NaN shows)
  }
  __syncthreads();

  // ---- the listed ids leave the slice: what is left is the rest
  if (warp == 0) {
    for (int j = lane; j < p.kt; j += 32) {
      const int at = s_id[j] - lo;
      if (at >= 0 && at < len)  // (a byte's word at a time: two places may share a unit)
        atomicOr(reinterpret_cast<uint32_t*>(s_listed) + (at + shift) / N / 4,
                 1u << ((at + shift) / N % 4 * 8 + (at + shift) % N));
    }
  }
  __syncthreads();
  MaxSum mine{-INFINITY, 0.f};
  float factor = 1.f;  // mine.m's
  auto take = [&](const Vec<T>& f, int) {
    const float top = vec_max(f);
    if (top > mine.m) {
      mine.s *= mine.m > -INFINITY ? ex2((mine.m - top) * p.k2) : 1.f;  // (nothing but a NaN sum yet)
      mine.m = top;
      factor = exp_factor<T>(top, p.k2);
    }
    float e2[N];
    unit_exp(f, mine.m > -INFINITY ? mine.m : 0.f, p.k2, e2);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) sum += e2[i];
    mine.s = fmaf(sum, factor, mine.s);
  };
  slice.each(take, take);
  mine = warp_join(mine, p.k2);
  if (lane == 0) s_warp[warp] = mine;
  __syncthreads();
  if (SP > 1) cluster_wait();  // every CTA of the cluster runs (what was read since the arrival hides the wait)
  if (warp == 0) {
    MaxSum all = s_warp[0];
#pragma unroll
    for (int i = 1; i < kDistillThreads / 32; ++i) all = join(all, s_warp[i], p.k2);
    if (SP == 1) {
      if (lane == 0) s_part[0] = all;
    } else if (lane < SP) {
      st_cluster(reinterpret_cast<uint2*>(&s_part[part]), lane, make_uint2(__float_as_uint(all.m), __float_as_uint(all.s)));
    }
  }
  if (SP > 1) cluster_sync();
  else __syncthreads();

  // ---- every id: the rest and the listed ones, relative to the row's maximum
  if (warp == 0) {
    MaxSum r = s_part[0];
#pragma unroll
    for (int c = 1; c < SP; ++c) r = join(r, s_part[c], p.k2);
    float top = r.m, loss = 0.f;
    int distinct = 0;
    unsigned firsts = 0;  // places whose id no earlier place has
    for (int i = 0; i < places; ++i) {
      const int j = 32 * i + lane;
      const int id = j < p.kt ? s_id[j] : -1;
      bool first = id >= 0;
      if (first) {
        top = fmaxf(top, s_x[j]);
        float all = 0.f;
        for (int k = 0; k < p.kt; ++k)
          if (s_id[k] == id) {
            all += s_q[k];
            if (k < j) first = false;
          }
        s_all[j] = all;
        if (s_q[j] > 0.f && s_q[j] != all) loss += s_q[j] * logf(s_q[j] / all);  // a shared id
      }
      if (first) firsts |= 1u << i;
      distinct += __popc(__ballot_sync(0xffffffffu, first));
    }
    top = warp_max(top);
    if (distinct == p.V) rest = 0.f;                            // every id is listed
    const bool empty = !(top > -INFINITY) && !isnan(r.s);       // every logit is -inf
    const float ref = top > -INFINITY ? top : 0.f;
    float listed = 0.f;
    for (int i = 0; i < places; ++i)
      if (firsts >> i & 1) listed += ex2((s_x[32 * i + lane] - ref) * p.k2);
    listed = warp_sum(listed);
    const float m_top = r.m > -INFINITY ? r.m - ref : 0.f;
    const float r_top = r.s * ex2(m_top * p.k2);
    const float z = r_top + listed;
    const float inv_z = z == 0.f ? 0.f : 1.f / z;
    const float log_z = logf(z), log_r = m_top * p.inv_t + logf(r.s);  // relative to ref
    float scale = 0.f;
    const float mass = teacher_mass(p.tail, taught, rest);
    if (GRAD) {
      scale = w == 0.f ? 0.f : (p.grad_loss ? __ldg(p.grad_loss + row) : 1.f) * w * p.inv_t;
      if (lane == 0) {
        // exp(z_v - log R) (Q R / Z - rest), with 2^((x - base) k2) = exp(z_v - log R) R
        s_a = r.s == 0.f ? 0.f : scale * (mass * r_top * inv_z - rest) / r.s;
        s_base = r.m > -INFINITY ? r.m : 0.f;
      }
    }
    for (int i = 0; i < places; ++i) {  // each first place's part of the loss, and its gradient
      const int j = 32 * i + lane;
      if (!(firsts >> i & 1)) continue;
      const float pj = ex2((s_x[j] - ref) * p.k2) * inv_z, q = s_all[j];
      if (part == 0) loss += excess(q, pj, (s_x[j] - ref) * p.inv_t - log_z);
      if (GRAD) s_x[j] = w == 0.f ? 0.f : scale * (mass * pj - q);
    }
    if (part == 0) {
      loss = warp_sum(loss);
      if (lane == 0) {
        const float p_rest = r_top / z;
        if (rest > 0.f) loss += excess(rest, p_rest, log_r - log_z);
        else loss += p.tail ? p_rest - left : p_rest;
        if (taught == 0.f && rest == 0.f) loss = 0.f;  // nothing is taught
        else if (empty) loss = INFINITY;
        p.loss[row] = w == 0.f ? 0.f : w * loss;
        if (p.lse) {
          p.lse[2 * static_cast<size_t>(row)] = empty ? -INFINITY : ref * p.inv_t + log_z;
          p.lse[2 * static_cast<size_t>(row) + 1] = ref * p.inv_t + log_r;
        }
      }
    }
    if (GRAD) {
      __syncwarp();
      for (int i = 0; i < places; ++i)
        if (!(firsts >> i & 1) && 32 * i + lane < p.kt) s_id[32 * i + lane] = -1;
    }
  }
  if (GRAD) {
    __syncthreads();
    const float base = s_base, a = s_a * exp_factor<T>(base, p.k2);
    T* dx = static_cast<T*>(p.dlogits) + row * static_cast<size_t>(p.grad_stride) + lo;
    const bool zero = w == 0.f;
    auto grads = [&](const Vec<T>& f) {
      float e2[N];
      if (zero) {
#pragma unroll
        for (int i = 0; i < N; ++i) e2[i] = 0.f;
      } else {
        unit_exp(f, base, p.k2, e2);
#pragma unroll
        for (int i = 0; i < N; ++i) e2[i] *= a;
      }
      Vec<T> g;
      pack(e2, &g);
      return g;
    };
    auto scatter = [&](const Vec<T>& f, int q) {
      const Vec<T> g = grads(f);
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (q * N + i >= shift && q * N + i < shift + len) dx[q * N + i - shift] = g.e[i];
    };
    if (row_shift(dx) == shift)
      slice.each([&](const Vec<T>& f, int q) { __stcs(reinterpret_cast<uint4*>(dx + (q * N - shift)), grads(f).raw); },
                 scatter);
    else
      slice.each(scatter, scatter);
    __syncthreads();  // the listed ids' places are written again
    for (int j = tid; j < p.kt; j += kDistillThreads) {
      const int at = s_id[j] - lo;
      if (at >= 0 && at < len) {
        T g;
        from_f32(s_x[j], &g);
        dx[at] = g;
      }
    }
  }
}

// A stored log-sum-exp beyond this does not tell the row's logits apart any more: half its last place is more than 2^-14
// (of -1e10, where every id that is not listed is masked so: hundreds).
constexpr float kFarSum = 1024.f;
__device__ __forceinline__ bool far_sum(float lse) { return fabsf(lse) > kFarSum && fabsf(lse) < INFINITY; }

// Join over the block; `s` holds one pair a warp.
__device__ __forceinline__ MaxSum block_join(MaxSum v, float k2, MaxSum* s, int tid) {
  v = warp_join(v, k2);
  __syncthreads();
  if ((tid & 31) == 0) s[tid >> 5] = v;
  __syncthreads();
  MaxSum all = s[0];
#pragma unroll
  for (int w = 1; w < kGradThreads / 32; ++w) all = join(all, s[w], k2);
  return all;
}

// The gradient of a whole row, by one CTA, with sums of its own, as distill_kernel takes them: they lie relative to the
// logits that they are sums of.  Rows like that are few, so this reads element by element (one row of 151936 fp32 ids:
// 250 us; 512 of them 630).  The logits and the gradient may share memory: everything is read before anything is written.
template <typename T>
__device__ __noinline__ void far_row(const DistillParams& p, size_t row, int id, float score, const T* x, T* dx, float w,
                                     int* s_id, float* s_q, float* s_red) {
  __shared__ uint32_t s_mark[kGradChunk / 32];  // the listed ids of a chunk, a bit each
  __shared__ MaxSum s_pair[kGradThreads / 32];
  const int tid = threadIdx.x;
  float rest, mass;
  const Place e = teacher_place<T, kGradThreads>(p, id, score, x, 0, p.V, s_id, s_q, s_red, &rest, &mass);
  MaxSum mine{-INFINITY, 0.f};
  for (int lo = 0; lo < p.V; lo += kGradChunk) {
    __syncthreads();
    for (int i = tid; i < kGradChunk / 32; i += kGradThreads) s_mark[i] = 0;
    __syncthreads();
    if (e.first && e.id >= lo && e.id - lo < kGradChunk) atomicOr(&s_mark[(e.id - lo) / 32], 1u << (e.id - lo) % 32);
    __syncthreads();
    const int end = min(p.V - lo, kGradChunk);
    for (int i = tid; i < end; i += kGradThreads) {
      const float v = to_f32(x[lo + i]);
      if (s_mark[i / 32] >> i % 32 & 1 || v == -INFINITY) continue;
      if (v > mine.m) {
        mine.s *= mine.m > -INFINITY ? ex2((mine.m - v) * p.k2) : 1.f;  // (nothing but a NaN sum yet)
        mine.m = v;
      }
      mine.s += ex2((v - mine.m) * p.k2);
    }
  }
  const MaxSum r = block_join(mine, p.k2, s_pair, tid);
  const MaxSum l = block_join(MaxSum{e.first ? e.x : -INFINITY, e.first && e.x != -INFINITY ? 1.f : 0.f}, p.k2, s_pair, tid);
  const MaxSum all = join(r, l, p.k2);
  const float scale = (p.grad_loss ? __ldg(p.grad_loss + row) : 1.f) * w * p.inv_t;
  const float inv_z = all.s == 0.f ? 0.f : 1.f / all.s;
  const float r_top = r.m > -INFINITY ? r.s * ex2((r.m - all.m) * p.k2) : r.s;
  const float a = r.s == 0.f ? 0.f : scale * (mass * r_top * inv_z - rest) / r.s;
  const float base = r.m > -INFINITY ? r.m : 0.f;
  for (int i = tid; i < p.V; i += kGradThreads) {
    T g;
    from_f32(a * ex2((to_f32(x[i]) - base) * p.k2), &g);
    dx[i] = g;
  }
  __syncthreads();  // the listed ids' places are written again
  if (e.first) {
    T g;
    from_f32(scale * (mass * (e.x > -INFINITY || isnan(e.x) ? ex2((e.x - all.m) * p.k2) * inv_z : 0.f) - e.q_all), &g);
    dx[e.id] = g;
  }
}

// The gradient from the sums that the loss left: one CTA per chunk of a row.
template <typename T>
__global__ void __launch_bounds__(kGradThreads) distill_grad_kernel(const __grid_constant__ DistillParams p, int chunks) {
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
  const float lse = p.lse[2 * row], lse_rest = p.lse[2 * row + 1];
  const int id = tid < p.kt ? __ldg(p.ids + row * p.kt + tid) : -1;  // (on the way before anything is asked of the others)
  const float score = tid < p.kt ? __ldg(p.scores + row * p.kt + tid) : -INFINITY;
  if (w == 0.f) {
    T none;
    from_f32(0.f, &none);
    for (int i = tid; i < len; i += kGradThreads) dx[i] = none;
    return;
  }
  if (far_sum(lse) || far_sum(lse_rest)) {
    if (lo == 0) far_row(p, row, id, score, x, dx, w, s_id, s_q, s_red);
    return;
  }
  float rest, mass;
  const Place e = teacher_place<T, kGradThreads>(p, id, score, x, lo, lo + len, s_id, s_q, s_red, &rest, &mass);
  __syncthreads();  // the listed logits are read before any gradient is written (they may share memory)
  const float scale = (p.grad_loss ? __ldg(p.grad_loss + row) : 1.f) * w * p.inv_t;
  const bool some = lse_rest > -INFINITY || isnan(lse_rest);
  const float a = some ? scale * (mass * expf(lse_rest - lse) - rest) : 0.f;
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
    from_f32(scale * (mass * pv - e.q_all), &g);
    dx[e.id - lo] = g;
  }
}

template <typename T, int SP, bool GRAD>
static cudaError_t launch_rows(DistillParams p, int rows, cudaStream_t stream) {
  p.slice = ((p.V + SP - 1) / SP + 7) & ~7;
  const size_t smem = (static_cast<size_t>(p.slice) * sizeof(T) / 16 + 16) / 16 * 16 + 16;
  cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(distill_kernel<T, SP, GRAD>), smem, false);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(rows) * SP);
  cfg.blockDim = dim3(kDistillThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = SP;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = SP > 1 ? 1 : 0;
  e = cudaLaunchKernelEx(&cfg, distill_kernel<T, SP, GRAD>, p);
  return e != cudaSuccess ? e : cudaGetLastError();
}

// CTAs a row: eight, so that few rows use many SMs; halved while the rows alone keep four CTAs an SM busy and a slice is
// shorter than 64 KB, for what a CTA does besides reading does not shrink with its slice.
template <typename T, bool GRAD>
static cudaError_t launch_split(const DistillParams& p, int rows, cudaStream_t stream) {
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  int split = 8;
  while (split > 1 && static_cast<long long>(rows) * split > 4 * sms && p.V / split * sizeof(T) < (64 << 10)) split /= 2;
  switch (split) {
    case 8: return launch_rows<T, 8, GRAD>(p, rows, stream);
    case 4: return launch_rows<T, 4, GRAD>(p, rows, stream);
    case 2: return launch_rows<T, 2, GRAD>(p, rows, stream);
  }
  return launch_rows<T, 1, GRAD>(p, rows, stream);
}

template <typename T>
static cudaError_t launch_type(const DistillParams& p, int rows, cudaStream_t stream) {
  if (p.loss) return p.dlogits ? launch_split<T, true>(p, rows, stream) : launch_split<T, false>(p, rows, stream);
  const int chunks = (p.V + kGradChunk - 1) / kGradChunk;
  if (static_cast<long long>(rows) * chunks > 0x7fffffffLL) return cudaErrorInvalidValue;
  distill_grad_kernel<T><<<static_cast<unsigned>(rows) * chunks, kGradThreads, 0, stream>>>(p, chunks);
  return cudaGetLastError();
}

cudaError_t launch_distill(const DistillParams& p, int dtype, int rows, cudaStream_t stream) {
  if (rows <= 0 || rows > 0x7fffffff / 8) return cudaErrorInvalidValue;
  if (p.V > kMaxRowVocab) return cudaErrorInvalidValue;
  if (dtype == kF32) return launch_type<float>(p, rows, stream);
  if (dtype == kBf16) return launch_type<__nv_bfloat16>(p, rows, stream);
  return launch_type<__half>(p, rows, stream);
}

}  // namespace dm
