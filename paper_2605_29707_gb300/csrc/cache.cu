// cache.cu -- what stands around the attention over a paged cache: rotary positions, alone or with the write of new
// keys and values into the cache, and the accepted nodes' move after a verification.
//
// Rotary positions.  Pair i of a token at position p turns by a = p f_i, cos and sin times an amplitude:
//   (y0, y1) = (x0 cos a - x1 sin a, x1 cos a + x0 sin a).
// At p = 2^20 the fp32 product p f_i is wrong by 0.03 radians, so the angle is kept as a fraction of a turn in 64-bit
// fixed point: F_i = f_i / (2 pi) modulo 1, from f_i's 24-bit mantissa and 96 bits of 1 / (2 pi), in integers; p F_i
// modulo 2^64 is the angle, exact but for F_i's last bit, 2^-33 of a turn at p = 2^31, at any speed.  The nearest quarter turn comes off in
// integers too, and cos and sin of the rest, at most an eighth of a turn, are taken in fp32.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "kernels.h"
#include "paged.cuh"
#include "rows.cuh"

namespace dm {
namespace {

constexpr int kRopeThreads = 256;

// f / (2 pi) in units of 2^-64 of a turn, modulo a turn: f = m 2^e with m below 2^24, |f| <= 1024.
__device__ __forceinline__ uint64_t turn_speed(float f) {
  constexpr uint64_t kInv2Pi = 0x28BE60DB9391054AULL;  // floor(2^64 / (2 pi)), and its next 32 bits
  constexpr uint32_t kInv2PiNext = 0x7F09D5F4u;
  const uint32_t bits = __float_as_uint(f);
  const int be = (bits >> 23) & 0xff;
  const uint64_t m = be ? (bits & 0x7fffffu) | 0x800000u : bits & 0x7fffffu;
  const int down = 150 - (be ? be : 1);  // f = m 2^-down
  const uint32_t next = __umulhi(kInv2PiNext, static_cast<uint32_t>(m));  // what speeds above 1 bring up
  const uint64_t lo = kInv2Pi * m + next, hi = __umul64hi(kInv2Pi, m) + (lo < next ? 1 : 0);
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
  static constexpr int kBytes = N * static_cast<int>(sizeof(T));
  using Raw = typename std::conditional<kBytes == 16, uint4, typename std::conditional<kBytes == 8, uint2, T>::type>::type;
  Raw raw;
  __device__ __forceinline__ void load(const T* p) { raw = *reinterpret_cast<const Raw*>(p); }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<Raw*>(p) = raw; }
  __device__ __forceinline__ void get(float (&v)[N]) const {
    const T* const e = reinterpret_cast<const T*>(&raw);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = to_f32(e[i]);
  }
  __device__ __forceinline__ void put(const float (&v)[N]) {
    T* const e = reinterpret_cast<T*>(&raw);
#pragma unroll
    for (int i = 0; i < N; ++i) from_f32(v[i], e + i);
  }
};

// Loads of a thread in flight, and blocks an SM that share the heads out: neighbours in one unit, or two units that pair up.
// us at 4 / 8 / 16 loads (8 blocks) and 4 / 8 / 16 blocks (the loads as chosen): 12003 tokens x 48 fp16 heads in a cache, pairs
// of neighbours, 50.5 / 49.6 / 56.8 and 52.8 / 49.6 / 50.3; 16384 x 32 bf16 heads, halves, 47.4 / 53.5 / 73.3 and 45.9 / 47.4 / 48.6.
// Units of 16 bytes take 54 to 68 registers, so 3 or 4 blocks of the 4 or 6 are on an SM at once; that was weighed on these
// large calls alone, and small ones end unevenly (3001 x 14 fp32 heads: 940 blocks, a wave and a half).
__host__ __device__ constexpr int units_ahead(bool inside) { return inside ? 8 : 4; }
__host__ __device__ constexpr int rope_blocks(bool inside) { return inside ? 6 : 4; }

// A thread keeps one share of a token's head, its angles in registers, and takes it through the heads h0 .. h1 - 1: those
// of x, then those of k, then those of v.  A share is a unit of N elements that holds pairs of neighbours (INSIDE), or
// two units whose elements pair up; the units behind the turned ones, and all of v's, are copied.  The first heads are on
// their way while the angles are computed.
// Bound by DRAM where there are many tokens, by one thread's chain of latencies (sequence, page, heads) where there are few:
// 12003 tokens of 48 fp16 heads into a cache 49.3 us, 6.0 TB/s; the gradient of 16384 x 32 bf16 heads 46.4 us, 5.8 TB/s; 3001 x
// 14 heads of 80 fp32 elements 5.9 us from L2 (9.4 from DRAM, 1.5 TB/s); 17 tokens of 48 heads 4.7 us.  Angles in shared memory, or a thread for every head,
// were not needed: a thread's angles are some 480 instructions among 2000.
template <typename T, int N, bool INSIDE>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const RopeParams p, int shares, int heads_a_block) {
  constexpr int kUnits = INSIDE ? 1 : 2, kHeads = units_ahead(INSIDE) / kUnits, kAngles = INSIDE ? N / 2 : N;
  const long long at = static_cast<long long>(blockIdx.x) * kRopeThreads + threadIdx.x;
  const int token = static_cast<int>(at / shares), share = static_cast<int>(at - static_cast<long long>(token) * shares);
  if (token >= p.tokens) return;
  const bool append = p.k != nullptr;

  int pos = 0;
  long long dst = -1;
  if (append) {
    const int seq = find_sequence(p.batch, token);
    if (seq < 0) return;  // a row behind the last sequence
    const Sequence s = load_sequence(p.cache, p.batch, p.tokens, seq);
    const int i = token - s.row, first = s.first;
    pos = first + i;
    dst = place_offset(p.cache, p.batch, seq, pos);
    if (p.depth && i >= 1 && i <= p.N) pos = first + p.depth[static_cast<long long>(seq) * p.N + i - 1];
  }
  if (p.positions) pos = p.positions[token];

  // the share's elements: o0, and o1 where there is a second unit
  const int turned = INSIDE ? p.rot / N : p.rot / 2 / N, behind = share - turned;
  int o0 = share * N, o1 = p.D;
  if (!INSIDE) {
    if (behind >= 0) {
      o0 = p.rot + 2 * N * behind;
      o1 = o0 + N;
    } else if (p.pairs) {  // N is 1
      o0 = 2 * share;
      o1 = o0 + 1;
    } else {
      o1 = o0 + p.rot / 2;
    }
  }
  const bool second = !INSIDE && o1 < p.D;
  const int spun = p.heads + (append ? p.cache.heads : 0), all = spun + (append ? p.cache.heads : 0);
  const int h0 = blockIdx.y * heads_a_block, h1 = min(h0 + heads_a_block, all);
  auto source = [&](int h) {
    if (h < p.heads) return static_cast<const T*>(p.x) + token * p.x_token + h * p.x_head;
    if (h < spun) return static_cast<const T*>(p.k) + token * p.k_token + static_cast<long long>(h - p.heads) * p.D;
    return static_cast<const T*>(p.v) + token * p.v_token + static_cast<long long>(h - spun) * p.D;
  };
  auto target = [&](int h) -> T* {
    if (h < p.heads) return static_cast<T*>(p.y) + token * p.y_token + h * p.y_head;
    if (dst < 0) return nullptr;  // no place in the cache
    if (h < spun) return static_cast<T*>(p.cache.k) + dst + (h - p.heads) * p.cache.head_stride;
    return static_cast<T*>(p.cache.v) + dst + (h - spun) * p.cache.head_stride;
  };
  Unit<T, N> u[kHeads][kUnits];
  auto load = [&](int h) {
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
      if (h + i >= h1) break;
      const T* const x = source(h + i);
      u[i][0].load(x + o0);
      if (second) u[i][kUnits - 1].load(x + o1);
    }
  };
  load(h0);

  float co[kAngles], si[kAngles];
  if (behind < 0) {
#pragma unroll
    for (int i = 0; i < kAngles; ++i) {
      turn(pos, turn_speed(p.freq[share * kAngles + i]), p.amplitude, &co[i], &si[i]);
      if (p.back) si[i] = -si[i];
    }
  }
  for (int h = h0;;) {
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
      if (h + i >= h1) break;
      if (behind < 0 && h + i < spun) {
        float a[N];
        u[i][0].get(a);
        if constexpr (INSIDE) {
#pragma unroll
          for (int e = 0; e < kAngles; ++e) {
            const float x0 = a[2 * e], x1 = a[2 * e + 1];
            a[2 * e] = fmaf(x0, co[e], -(x1 * si[e]));
            a[2 * e + 1] = fmaf(x1, co[e], x0 * si[e]);
          }
        } else {
          float b[N];
          u[i][kUnits - 1].get(b);
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const float x0 = a[e], x1 = b[e];
            a[e] = fmaf(x0, co[e], -(x1 * si[e]));
            b[e] = fmaf(x1, co[e], x0 * si[e]);
          }
          u[i][kUnits - 1].put(b);
        }
        u[i][0].put(a);
      }
      T* const y = target(h + i);
      if (y) {
        u[i][0].store(y + o0);
        if (second) u[i][kUnits - 1].store(y + o1);
      }
    }
    h += kHeads;
    if (h >= h1) break;
    load(h);
  }
}

template <typename T, int N, bool INSIDE>
cudaError_t launch_rope_units(const RopeParams& p, int sms, cudaStream_t stream) {
  const int rest = (p.D - p.rot) / N;
  const int shares = INSIDE ? p.D / N : p.rot / 2 / N + (rest + 1) / 2;
  const int heads = p.heads + (p.k ? 2 * p.cache.heads : 0);
  const long long blocks = (static_cast<long long>(p.tokens) * shares + kRopeThreads - 1) / kRopeThreads;
  // Angles cost as much as several heads, so a thread takes all of them where the tokens fill the chip that many blocks an
  // SM; fewer tokens spread their heads over the blocks.
  long long split = (static_cast<long long>(rope_blocks(INSIDE)) * sms + blocks - 1) / blocks;
  split = split < 1 ? 1 : split > heads ? heads : split;
  const int each = static_cast<int>((heads + split - 1) / split);
  const dim3 grid(static_cast<unsigned>(blocks), static_cast<unsigned>((heads + each - 1) / each));
  rope_kernel<T, N, INSIDE><<<grid, kRopeThreads, 0, stream>>>(p, shares, each);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_rope_type(const RopeParams& p, int unit_bytes, int sms, cudaStream_t stream) {
  constexpr int kElem = static_cast<int>(sizeof(T));
  if (unit_bytes == 16 && p.pairs) return launch_rope_units<T, 16 / kElem, true>(p, sms, stream);
  if (unit_bytes == 8 && p.pairs) return launch_rope_units<T, 8 / kElem, true>(p, sms, stream);
  if (unit_bytes == 16) return launch_rope_units<T, 16 / kElem, false>(p, sms, stream);
  if (unit_bytes == 8) return launch_rope_units<T, 8 / kElem, false>(p, sms, stream);
  return launch_rope_units<T, 1, false>(p, sms, stream);
}

// ---------------------------------------------------------------- accepted nodes
constexpr int kCommitThreads = 256;
constexpr int kCommitBlocks = 8;  // blocks an SM that share the layers out
constexpr int kMoves = 256;       // moves looked up at a time
constexpr int kMovesAhead = 8;

template <typename E, typename V, int N>
struct MoveUnit {
  using elem = E;
  using type = V;
  static constexpr int kN = N;
};

// A block takes some layers of a sequence, keys and values.  It looks the whole list through, then the moves' places, once
// for all layers; a thread takes one unit of a place through all moves.  The list rises, so node j's source lies behind
// the targets of all moves before it: moves may read ahead of the earlier ones' writes, and a thread that reads eight
// before it writes them leaves every unit what one move after the other would.
// Bound by the chain of look-ups (sequence, list, table, keys) where little moves, by a thread's loads in flight where much
// does (a layer's moves of a sequence, 0 to 8, before the next layer's): 64 sequences' nodes in 64 layers 18.0 us with the
// rows in DRAM, 4.0 TB/s of the 73 MB that move, and 13.4 us with them in L2, which holds them when the call is repeated;
// 28 layers of one sequence 3.0 us.  With the places looked up by every thread for itself, and a block a layer's keys or
// values, the two took 38 and 5.4 us (repeated).
template <typename U>
__global__ void __launch_bounds__(kCommitThreads) commit_kernel(const CommitParams p, int units, int layers_a_block) {
  using E = typename U::elem;
  using V = typename U::type;
  __shared__ long long s_from[kMoves], s_to[kMoves];
  const int b = blockIdx.x, tid = threadIdx.x;
  const PagedCache& c = p.cache;
  const int s0 = p.batch.start[b], s1 = p.batch.start[b + 1], kv = p.batch.kv_len[b], count = p.count[b];
  const int tree = min(p.N, s1 - s0 - 1);  // nodes
  const long long first = static_cast<long long>(kv) - (static_cast<long long>(s1) - s0 - 1);  // node 0's place
  const int32_t* const nodes = p.nodes + static_cast<long long>(b) * p.N;
  bool good = s0 >= 0 && s1 >= s0 && kv >= 0 && kv <= table_places(c, p.batch);
  if (s1 == s0) good = good && count == 0;
  else good = good && first >= 1 && count >= 0 && count <= tree;
  const int f = static_cast<int>(first);
  // move j's element offsets, -1 where nothing moves; false where it cannot be made
  auto look = [&](int j, long long* from, long long* to) {
    const int node = nodes[j];
    if (node < 0 || node >= tree || (j > 0 && node <= nodes[j - 1])) return false;
    *from = place_offset(c, p.batch, b, f + node);
    *to = place_offset(c, p.batch, b, f + j);
    const bool is = *from >= 0 && *to >= 0;
    if (node == j) *from = -1;
    return is;
  };
  if (good)
    for (int j = tid; j < count; j += kCommitThreads) {
      long long from, to;
      good = look(j, &from, &to) && good;
      if (j < kMoves) {
        s_from[j] = from;
        s_to[j] = to;
      }
    }
  good = __syncthreads_and(good);
  if (blockIdx.y == 0 && tid == 0) p.new_len[b] = !good ? -1 : s1 == s0 ? kv : f + count;
  if (!good) return;
  const int l0 = blockIdx.y * layers_a_block, layers = min(layers_a_block, p.layers - l0), per_head = c.D / U::kN;
  for (int m0 = 0; m0 < count; m0 += kMoves) {
    const int moves = min(kMoves, count - m0);
    if (m0 > 0) {
      __syncthreads();
      if (tid < moves) look(m0 + tid, &s_from[tid], &s_to[tid]);
      __syncthreads();
    }
    for (int x = tid; x < 2 * units * layers; x += kCommitThreads) {
      const int slice = x / units, u = x - slice * units, head = u / per_head;  // slice: layer, keys or values
      E* const e = static_cast<E*>(slice & 1 ? c.v : c.k) + (l0 + (slice >> 1)) * p.layer_stride + head * c.head_stride +
                   static_cast<long long>(u - head * per_head) * U::kN;
      for (int j0 = 0; j0 < moves; j0 += kMovesAhead) {
        V r[kMovesAhead];
#pragma unroll
        for (int i = 0; i < kMovesAhead; ++i)
          if (j0 + i < moves && s_from[j0 + i] >= 0) r[i] = *reinterpret_cast<const V*>(e + s_from[j0 + i]);
#pragma unroll
        for (int i = 0; i < kMovesAhead; ++i)
          if (j0 + i < moves && s_from[j0 + i] >= 0) *reinterpret_cast<V*>(e + s_to[j0 + i]) = r[i];
      }
    }
  }
}

template <typename U>
cudaError_t launch_commit_units(const CommitParams& p, int sms, cudaStream_t stream) {
  const long long slots = static_cast<long long>(kCommitBlocks) * sms;
  const long long each = (static_cast<long long>(p.layers) * p.batch.B + slots - 1) / slots;
  const int units = p.cache.heads * p.cache.D / U::kN, most = (1 << 30) / (2 * units);  // a block counts units in 32 bits
  const int layers = static_cast<int>(std::min({each, static_cast<long long>(p.layers), static_cast<long long>(most)}));
  const dim3 grid(static_cast<unsigned>(p.batch.B), static_cast<unsigned>((p.layers + layers - 1) / layers));
  commit_kernel<U><<<grid, kCommitThreads, 0, stream>>>(p, units, layers);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_rope(const RopeParams& p, int dtype, int unit_bytes, int sms, cudaStream_t stream) {
  if (dtype == kF32) return launch_rope_type<float>(p, unit_bytes, sms, stream);
  if (dtype == kBf16) return launch_rope_type<__nv_bfloat16>(p, unit_bytes, sms, stream);
  return launch_rope_type<__half>(p, unit_bytes, sms, stream);
}

cudaError_t launch_commit(const CommitParams& p, int elem_bytes, bool vector, int sms, cudaStream_t stream) {
  if (vector && elem_bytes == 2) return launch_commit_units<MoveUnit<uint16_t, uint4, 8>>(p, sms, stream);
  if (vector) return launch_commit_units<MoveUnit<uint32_t, uint4, 4>>(p, sms, stream);
  if (elem_bytes == 2) return launch_commit_units<MoveUnit<uint16_t, uint16_t, 1>>(p, sms, stream);
  return launch_commit_units<MoveUnit<uint32_t, uint32_t, 1>>(p, sms, stream);
}

}  // namespace dm
