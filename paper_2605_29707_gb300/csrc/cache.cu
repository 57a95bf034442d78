// cache.cu -- what stands around the attention over a paged cache: rotary positions, alone or with the write of new
// keys and values into the cache, and the accepted nodes' move after a verification.
//
// Rotary positions.  Pair i of a token at position p turns by a = p f_i, cos and sin times an amplitude:
//   (y0, y1) = (x0 cos a - x1 sin a, x1 cos a + x0 sin a).
// At p = 2^20 the fp32 product p f_i is wrong by 0.03 radians, so the angle is kept as a fraction of a turn in 64-bit
// fixed point: F_i = f_i / (2 pi) modulo 1, from f_i's 24-bit mantissa and 64 bits of 1 / (2 pi), in integers; p F_i
// modulo 2^64 is the angle, exact but for F_i's last bit, 2^-33 of a turn at p = 2^31.  The nearest quarter turn comes off in
// integers too, and cos and sin of the rest, at most an eighth of a turn, are taken in fp32.
#include <math.h>

#include "kernels.h"
#include "paged.cuh"
#include "rows.cuh"

namespace dm {
namespace {

constexpr int kRopeThreads = 256;

// f / (2 pi) in units of 2^-64 of a turn, modulo a turn: f = m 2^e with m below 2^24, |f| <= 1024.
__device__ __forceinline__ uint64_t turn_speed(float f) {
  constexpr uint64_t kInv2Pi = 0x28BE60DB9391054AULL;  // floor(2^64 / (2 pi))
  const uint32_t bits = __float_as_uint(f);
  const int be = (bits >> 23) & 0xff;
  const uint64_t m = be ? (bits & 0x7fffffu) | 0x800000u : bits & 0x7fffffu;
  const int down = 150 - (be ? be : 1);  // f = m 2^-down
  const uint64_t lo = kInv2Pi * m, hi = __umul64hi(kInv2Pi, m);
  uint64_t F;
  if (down <= 0) F = -down < 64 ? lo << -down : 0;
  else if (down < 64) F = (lo >> down) | (hi << (64 - down));
  else F = down < 128 ? hi >> (down - 64) : 0;
  return (bits >> 31) ? 0 - F : F;
}

// cos and sin of p turns of speed F, times the amplitude.
__device__ __forceinline__ void turn(int p, uint64_t F, float amplitude, float* co, float* si) {
  const uint64_t t = static_cast<uint64_t>(static_cast<int64_t>(p)) * F;
  const uint64_t quarter = (t + (1ULL << 61)) >> 62;
  const int64_t rest = static_cast<int64_t>(t - (quarter << 62));  // [-1/8, 1/8) of a turn
  float s, c;
  sincospif(static_cast<float>(rest) * 0x1p-63f, &s, &c);
  const float a = (quarter & 1) ? s : c, b = (quarter & 1) ? c : s;  // up to signs
  *co = (((quarter + 1) & 2) ? -a : a) * amplitude;
  *si = ((quarter & 2) ? -b : b) * amplitude;
}

// N elements in one access of 16 or 8 bytes, or one element.
template <typename T, int N>
struct Unit {
  float v[N];
  static constexpr int kBytes = N * static_cast<int>(sizeof(T));
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (kBytes == 16) {
      Vec<T> r;
      r.raw = *reinterpret_cast<const uint4*>(p);
      unpack(r, v);
    } else if constexpr (kBytes == 8 && N > 1) {
      alignas(8) T e[N];
      *reinterpret_cast<uint2*>(e) = *reinterpret_cast<const uint2*>(p);
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = to_f32(e[i]);
    } else {
      v[0] = to_f32(*p);
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (kBytes == 16) {
      Vec<T> r;
      pack(v, &r);
      *reinterpret_cast<uint4*>(p) = r.raw;
    } else if constexpr (kBytes == 8 && N > 1) {
      alignas(8) T e[N];
#pragma unroll
      for (int i = 0; i < N; ++i) from_f32(v[i], e + i);
      *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(e);
    } else {
      from_f32(v[0], p);
    }
  }
};

// A thread keeps one share of a token's head, its angles in registers, and takes it through the heads h0 .. h1 - 1:
// the heads of x, then those of k.  Values have no angles; their units go round the token's threads.
//   shares: rot / 2 / N of N pairs each (halves: a unit of each half; neighbours: two units), then (D - rot) / N units
//   that are copied.
template <typename T, int N>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const RopeParams p, int shares, int heads_a_block) {
  using U = Unit<T, N>;
  const long long at = static_cast<long long>(blockIdx.x) * kRopeThreads + threadIdx.x;
  const int token = static_cast<int>(at / shares), share = static_cast<int>(at - static_cast<long long>(token) * shares);
  if (token >= p.tokens) return;
  const int turned = p.rot / 2 / N;
  const bool append = p.k != nullptr;

  int place = -1, pos = 0, seq = -1;
  long long dst = -1;
  if (append) {
    seq = find_sequence(p.batch, token);
    if (seq < 0) return;  // a row behind the last sequence
    const Sequence s = load_sequence(p.cache, p.batch, p.tokens, seq);
    const int i = token - s.row, first = s.kv - s.n;
    place = first + i;
    dst = place_offset(p.cache, p.batch, seq, place);
    pos = place;
    if (p.depth && i >= 1 && i <= p.N) pos = first + p.depth[static_cast<long long>(seq) * p.N + i - 1];
  }
  if (p.positions) pos = p.positions[token];

  const int h0 = blockIdx.y * heads_a_block, all = p.heads + (append ? 2 * p.cache.heads : 0);
  const int h1 = min(h0 + heads_a_block, all), spun = p.heads + (append ? p.cache.heads : 0);
  T* const ck = static_cast<T*>(p.cache.k);
  T* const cv = static_cast<T*>(p.cache.v);
  auto source = [&](int h) {
    return h < p.heads ? static_cast<const T*>(p.x) + token * p.x_token + h * p.x_head
                       : static_cast<const T*>(p.k) + token * p.k_token + static_cast<long long>(h - p.heads) * p.D;
  };
  auto target = [&](int h) -> T* {
    if (h < p.heads) return static_cast<T*>(p.y) + token * p.y_token + h * p.y_head;
    return dst < 0 ? nullptr : ck + dst + (h - p.heads) * p.cache.head_stride;
  };

  if (share < turned) {
    if (h0 < spun) {
      float co[N], si[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        turn(pos, turn_speed(p.freq[share * N + i]), p.amplitude, &co[i], &si[i]);
        if (p.back) si[i] = -si[i];
      }
      const int o0 = p.pairs ? 2 * share * N : share * N;
      const int o1 = p.pairs ? o0 + N : o0 + p.rot / 2;
#pragma unroll 4
      for (int h = h0; h < min(h1, spun); ++h) {
        const T* const x = source(h);
        T* const y = target(h);
        U a, b;
        a.load(x + o0);
        b.load(x + o1);
        if (p.pairs) {
#pragma unroll
          for (int i = 0; i < N; ++i) {  // pair i of the share: elements 2 i and 2 i + 1 of the two units in a row
            float& x0 = 2 * i < N ? a.v[2 * i < N ? 2 * i : 0] : b.v[2 * i < N ? 0 : 2 * i - N];
            float& x1 = 2 * i + 1 < N ? a.v[2 * i + 1 < N ? 2 * i + 1 : 0] : b.v[2 * i + 1 < N ? 0 : 2 * i + 1 - N];
            const float y0 = fmaf(x0, co[i], -(x1 * si[i])), y1 = fmaf(x1, co[i], x0 * si[i]);
            x0 = y0;
            x1 = y1;
          }
        } else {
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const float y0 = fmaf(a.v[i], co[i], -(b.v[i] * si[i])), y1 = fmaf(b.v[i], co[i], a.v[i] * si[i]);
            a.v[i] = y0;
            b.v[i] = y1;
          }
        }
        if (y) {
          a.store(y + o0);
          b.store(y + o1);
        }
      }
    }
  } else {
    const int o = p.rot + (share - turned) * N;
#pragma unroll 4
    for (int h = h0; h < min(h1, spun); ++h) {
      T* const y = target(h);
      U a;
      a.load(source(h) + o);
      if (y) a.store(y + o);
    }
  }
  if (!append || dst < 0) return;
  const int units = p.D / N;
#pragma unroll 2
  for (int h = max(h0, spun) - spun; h < h1 - spun; ++h) {
    const T* const x = static_cast<const T*>(p.v) + token * p.v_token + static_cast<long long>(h) * p.D;
    T* const y = cv + dst + h * p.cache.head_stride;
    for (int u = share; u < units; u += shares) {
      U a;
      a.load(x + u * N);
      a.store(y + u * N);
    }
  }
}

template <typename T, int N>
cudaError_t launch_rope_units(const RopeParams& p, int sms, cudaStream_t stream) {
  const int shares = p.rot / 2 / N + (p.D - p.rot) / N;
  const int heads = p.heads + (p.k ? 2 * p.cache.heads : 0);
  const long long blocks = (static_cast<long long>(p.tokens) * shares + kRopeThreads - 1) / kRopeThreads;
  // Angles cost as much as several heads, so a thread takes all of them where the tokens fill the chip four blocks an SM
  // deep; fewer tokens spread their heads over the blocks.
  long long split = (4LL * sms + blocks - 1) / blocks;
  split = split < 1 ? 1 : split > heads ? heads : split;
  const int each = static_cast<int>((heads + split - 1) / split);
  const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>((heads + each - 1) / each));
  rope_kernel<T, N><<<grid, kRopeThreads, 0, stream>>>(p, shares, each);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_rope_type(const RopeParams& p, int unit_bytes, int sms, cudaStream_t stream) {
  constexpr int kElem = static_cast<int>(sizeof(T));
  if (unit_bytes == 16) return launch_rope_units<T, 16 / kElem>(p, sms, stream);
  if (unit_bytes == 8) return launch_rope_units<T, 8 / kElem>(p, sms, stream);
  return launch_rope_units<T, 1>(p, sms, stream);
}

// ---------------------------------------------------------------- accepted nodes
constexpr int kCommitThreads = 256;
constexpr int kMovesAhead = 8;

// A block takes a sequence's keys, or values, of one layer; a thread one unit of every node.  The list rises, so node
// j's source lies behind the targets of all moves before it: moves may read ahead of the earlier ones' writes, and a
// thread that reads eight before it writes them leaves every unit what one move after the other would.
template <typename U>
__global__ void __launch_bounds__(kCommitThreads) commit_kernel(const CommitParams p, int units) {
  const int b = blockIdx.x, layer = blockIdx.y >> 1, tid = threadIdx.x;
  const bool values = blockIdx.y & 1;
  const PagedCache& c = p.cache;
  const int s0 = p.batch.start[b], s1 = p.batch.start[b + 1], kv = p.batch.kv_len[b], count = p.count[b];
  const int tree = min(p.N, s1 - s0 - 1);  // nodes
  const long long first = static_cast<long long>(kv) - (static_cast<long long>(s1) - s0 - 1);  // node 0's place
  const int32_t* const nodes = p.nodes + static_cast<long long>(b) * p.N;
  bool good = s0 >= 0 && s1 >= s0 && kv >= 0 && kv <= table_places(c, p.batch);
  if (s1 == s0) good = good && count == 0;
  else good = good && first >= 1 && count >= 0 && count <= tree;
  if (good)
    for (int j = tid; j < count; j += kCommitThreads) {
      const int node = nodes[j];
      good = good && node >= 0 && node < tree && (j == 0 || node > nodes[j - 1]);
      if (good) {
        good = place_offset(c, p.batch, b, static_cast<int>(first) + node) >= 0 &&
               place_offset(c, p.batch, b, static_cast<int>(first) + j) >= 0;
      }
    }
  good = __syncthreads_and(good);
  if (blockIdx.y == 0 && tid == 0)
    p.new_len[b] = !good ? -1 : s1 == s0 ? kv : static_cast<int>(first) + count;
  if (!good) return;
  const int f = static_cast<int>(first);
  using E = typename U::elem;
  E* const e = static_cast<E*>(values ? c.v : c.k) + layer * p.layer_stride;
  const int per_head = c.D / U::kN;
  for (int u = tid; u < units; u += kCommitThreads) {
    const int head = u / per_head;
    const long long o = head * c.head_stride + static_cast<long long>(u - head * per_head) * U::kN;
    for (int j0 = 0; j0 < count; j0 += kMovesAhead) {
      typename U::type r[kMovesAhead];
      long long to[kMovesAhead];
#pragma unroll
      for (int i = 0; i < kMovesAhead; ++i) {
        const int j = j0 + i;
        to[i] = -1;
        if (j < count && nodes[j] != j) {
          to[i] = place_offset(c, p.batch, b, f + j) + o;
          r[i] = *reinterpret_cast<const typename U::type*>(e + place_offset(c, p.batch, b, f + nodes[j]) + o);
        }
      }
#pragma unroll
      for (int i = 0; i < kMovesAhead; ++i)
        if (to[i] >= 0) *reinterpret_cast<typename U::type*>(e + to[i]) = r[i];
    }
  }
}

template <typename E, typename V, int N>
struct MoveUnit {
  using elem = E;
  using type = V;
  static constexpr int kN = N;
};

}  // namespace

cudaError_t launch_rope(const RopeParams& p, int dtype, int unit_bytes, int sms, cudaStream_t stream) {
  if (dtype == kF32) return launch_rope_type<float>(p, unit_bytes, sms, stream);
  if (dtype == kBf16) return launch_rope_type<__nv_bfloat16>(p, unit_bytes, sms, stream);
  return launch_rope_type<__half>(p, unit_bytes, sms, stream);
}

cudaError_t launch_commit(const CommitParams& p, int elem_bytes, bool vector, cudaStream_t stream) {
  const dim3 grid(static_cast<unsigned>(p.batch.B), static_cast<unsigned>(2 * p.layers));
  const int elems = p.cache.heads * p.cache.D;
  if (vector && elem_bytes == 2)
    commit_kernel<MoveUnit<uint16_t, uint4, 8>><<<grid, kCommitThreads, 0, stream>>>(p, elems / 8);
  else if (vector)
    commit_kernel<MoveUnit<uint32_t, uint4, 4>><<<grid, kCommitThreads, 0, stream>>>(p, elems / 4);
  else if (elem_bytes == 2)
    commit_kernel<MoveUnit<uint16_t, uint16_t, 1>><<<grid, kCommitThreads, 0, stream>>>(p, elems);
  else
    commit_kernel<MoveUnit<uint32_t, uint32_t, 1>><<<grid, kCommitThreads, 0, stream>>>(p, elems);
  return cudaGetLastError();
}

}  // namespace dm
