// attend_rows.cu -- attention over a paged cache for every element type, page size, stride and head size: a block a row.
//
// Row (token, query head) with query x: s_j = scale x . k_j over the keys it sees, out = sum_j e^(s_j - m) v_j / sum_j
// e^(s_j - m), lse = m + log of that sum.  One pass with a running maximum m for each of eight warps, 32 keys at a time: a lane a
// key for the scores and a lane D / 32 elements for the values; the warps' sums are added up in their order.  Everything in
// fp32; hidden keys are not read.  It is bound by the latency of a warp's chain and, with many rows, by L1, which every row's keys
// pass: one token over 1000 keys 69 us (bf16, pages of 15; 425 with one warp a row), 64 tokens over up to 8192 keys 1.7 ms (bf16
// pages of 65, or fp32), 2.5 ms with heads of 256 elements, ragged fp32 chunks of up to 701 tokens 11.6 ms.  The layouts that the
// tensor cores take (13 us, 176 us, 64 us) never come here.
#include <math.h>

#include "kernels.h"
#include "paged.cuh"
#include "rows.cuh"

namespace dm {
namespace {

constexpr int kRowWarps = 8;
constexpr int kLaneElems = kMaxHeadDim / 32;

template <typename T, bool VEC>
__global__ void __launch_bounds__(32 * kRowWarps) attend_rows_kernel(const AttendParams p) {
  __shared__ float s_q[kMaxHeadDim], s_o[kRowWarps][kMaxHeadDim], s_m[kRowWarps], s_sum[kRowWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned row = blockIdx.x;
  const int token = row / p.hq, head = row - token * p.hq;
  const PagedCache& c = p.cache;
  const int seq = find_sequence(p.batch, token);
  if (seq < 0) return;
  const Sequence s = load_sequence(c, p.batch, p.tokens, seq);
  const int i = token - s.row;
  if (i < 0 || i >= s.n) return;
  const long long first = s.first;
  const int32_t* const parent = p.parent ? p.parent + static_cast<long long>(seq) * p.N : nullptr;
  const T* const q = static_cast<const T*>(p.q) + token * p.q_stride + static_cast<long long>(head) * c.D;
  for (int d = threadIdx.x; d < c.D; d += 32 * kRowWarps) s_q[d] = to_f32(q[d]);
  __syncthreads();
  const long long head_off = (head / p.group) * c.head_stride;
  const T* const k = static_cast<const T*>(c.k) + head_off;
  const T* const v = static_cast<const T*>(c.v) + head_off;
  const int32_t* const table = p.batch.table + seq * p.batch.table_stride;

  float m = -INFINITY, sum = 0.f, o[kLaneElems];
#pragma unroll
  for (int e = 0; e < kLaneElems; ++e) o[e] = 0.f;
  const long long end = p.mask == kMaskCausal ? min(first + i + 1, static_cast<long long>(s.kv)) : s.kv;
  for (long long j0 = 32 * warp; j0 < end; j0 += 32 * kRowWarps) {
    const int j = static_cast<int>(j0) + lane;
    long long off = -1;
    if (j0 + lane < end && sees(p.mask, parent, p.N, i, first, j)) {
      const int pi = j / c.page, pg = table[pi];
      if (pg >= 0 && pg < c.pages) off = pg * c.page_stride + (j - pi * c.page) * c.token_stride;
      else set_status(p.status, kStatusBadPage);
    }
    float z = -INFINITY;
    if (off >= 0) {
      float dot = 0.f;
      if constexpr (VEC) {
        for (int d = 0; d < c.D; d += Vec<T>::kN) {
          Vec<T> r;
          r.raw = *reinterpret_cast<const uint4*>(k + off + d);
          float x[Vec<T>::kN];
          unpack(r, x);
#pragma unroll
          for (int e = 0; e < Vec<T>::kN; ++e) dot = fmaf(s_q[d + e], x[e], dot);
        }
      } else {
        for (int d = 0; d < c.D; ++d) dot = fmaf(s_q[d], to_f32(k[off + d]), dot);
      }
      z = dot * p.scale;
    }
    float top = z;
#pragma unroll
    for (int w = 16; w; w >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, w));
    top = fmaxf(top, m);
    const float base = top == -INFINITY ? 0.f : top;
    const float w = off >= 0 ? expf(z - base) : 0.f;
    const float keep = expf(m - base);
    m = top;
    float add = w;
#pragma unroll
    for (int x = 16; x; x >>= 1) add += __shfl_xor_sync(~0u, add, x);
    sum = fmaf(sum, keep, add);
#pragma unroll
    for (int e = 0; e < kLaneElems; ++e) o[e] *= keep;
    unsigned live = __ballot_sync(~0u, off >= 0);
    while (live) {
      const int l = __ffs(live) - 1;
      live &= live - 1;
      const float wl = __shfl_sync(~0u, w, l);
      const T* const x = v + __shfl_sync(~0u, off, l);
#pragma unroll
      for (int e = 0; e < kLaneElems; ++e)
        if (lane + 32 * e < c.D) o[e] = fmaf(wl, to_f32(x[lane + 32 * e]), o[e]);
    }
  }
#pragma unroll
  for (int e = 0; e < kLaneElems; ++e)
    if (lane + 32 * e < c.D) s_o[warp][lane + 32 * e] = o[e];
  if (lane == 0) {
    s_m[warp] = m;
    s_sum[warp] = sum;
  }
  __syncthreads();
  m = s_m[0];
#pragma unroll
  for (int w = 1; w < kRowWarps; ++w) m = fmaxf(m, s_m[w]);
  const float base = m == -INFINITY ? 0.f : m;
  float f[kRowWarps];
  sum = 0.f;
#pragma unroll
  for (int w = 0; w < kRowWarps; ++w) {
    f[w] = expf(s_m[w] - base);
    sum = fmaf(s_sum[w], f[w], sum);
  }
  T* const out = static_cast<T*>(p.out) + token * p.out_stride + static_cast<long long>(head) * c.D;
  for (int d = threadIdx.x; d < c.D; d += 32 * kRowWarps) {
    float y = 0.f;
#pragma unroll
    for (int w = 0; w < kRowWarps; ++w)
      if (s_m[w] != -INFINITY) y = fmaf(s_o[w][d], f[w], y);
    from_f32(sum == 0.f ? 0.f : y / sum, out + d);
  }
  if (p.lse && threadIdx.x == 0) p.lse[row] = sum == 0.f ? -INFINITY : m + logf(sum);
}

template <typename T>
cudaError_t launch_rows(const AttendParams& p, bool vector, cudaStream_t stream) {
  const unsigned grid = static_cast<unsigned>(p.tokens) * static_cast<unsigned>(p.hq);  // below 2^31
  if (vector) attend_rows_kernel<T, true><<<grid, 32 * kRowWarps, 0, stream>>>(p);
  else attend_rows_kernel<T, false><<<grid, 32 * kRowWarps, 0, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attend_rows(const AttendParams& p, int dtype, bool vector, cudaStream_t stream) {
  if (dtype == kF32) return launch_rows<float>(p, vector, stream);
  if (dtype == kBf16) return launch_rows<__nv_bfloat16>(p, vector, stream);
  return launch_rows<__half>(p, vector, stream);
}

}  // namespace dm
