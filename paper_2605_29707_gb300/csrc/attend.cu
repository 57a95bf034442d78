// attend.cu -- attention of new tokens over a paged cache on the tensor cores, bf16 and fp16.
//
// Mathematics.  Query x of a row, keys k_j and values v_j that it sees:  s_j = x . k_j,  out = sum_j 2^(c (s_j - m)) v_j /
// sum_j 2^(c (s_j - m)),  lse = scale m + log of that sum, with c = scale log2(e) and any m; one pass over the keys, 128 at
// a time, with m the running maximum.
//
// The query heads of a group share their keys, so a tile of 128 rows holds 128 / group tokens with all of the group's heads,
// and a group of queries (a sequence's tokens, one head of keys) has one or two tiles.  Each of two warpgroups owns an S and an
// O accumulator in tensor memory, and keeps one row a thread: with two tiles of queries each has its own and both take
// every tile of keys; with one, the warpgroups take the tiles of keys in turn and add up at the end.  S = X K^T runs
// with both operands in shared memory; the weights replace S in tensor memory and are the first operand of O += W V
// there, half of the keys as soon as their weights stand.  While one warpgroup takes its exponentials, the tensor core works
// for the other.  O is scaled down only where
// the maximum has grown by more than 2^8 since m was set: the weights stay below 2^8, whose sums fp32 holds.
//
// Work is the line of all (sequence, head, group of queries, tile of keys), cut into equal stretches, one a CTA (one an SM):
// whatever the lengths, which the host does not know, no SM idles.  A stretch that begins or ends inside a group leaves its
// unnormalised sums, maxima and masses in the workspace, two slots a CTA; a second kernel joins them in order.
//
// Masks only touch tiles that reach past the first key that some row does not see.  There the weights' 0 would meet
// values nobody vouches for (places behind the last key, tokens of other branches), so in such tiles whatever is not
// finite, or lies behind the last key, is set to 0 in shared memory, and rows that do see such a value get it added at the
// end from the cache.
//
// Warps: eight for the softmax, one that brings keys, one values (TMA, a copy a piece of a page and 64 elements), one that
// issues the products, one that walks the line, describes the segments to the others and brings the next one's queries.
//
// What bounds it (device time; floors at the measured copy and cuBLAS rates).  Single tokens: DRAM; 64 sequences of up to 8192
// keys 176 us, 6.1 TB/s.  Long chunks: the tensor core and, over seconds, the power limit; 4096 tokens over 32768 keys 1310-1380
// us in short runs, 1.50-1.57 PFLOP/s, 1465 when repeated for a second.  There two tiles of queries take 2700 cycles a tile of
// keys without any softmax (the products' operands and the incoming tiles are 126 of the 128 bytes a cycle that shared
// memory gives) and 3000 with it.  Trees and short chunks: what a segment costs besides its tiles, some 13000 cycles (queries,
// masks, the last products, the results), and with the one token that a tree of 2^k nodes has over, a second group that reads
// all keys again: 64 trees of 32 nodes, 64 heads on 8, 230 us at 5 TB/s, twice their bytes.  One short call: the chain of launch,
// lengths, page, keys, softmax and join, 13 us.
//
// Tried and left out, us of the long chunk at the time: steering the products by one thread alone 1849 (the whole warp 1309); one
// loop for both kinds of group 1460 (written out 1319); reading the scores twice from tensor memory 1583 (once 1370); two
// threads a row 1440 (one 1372); queries as whole tiles with zeros, results through shared memory, keys backwards in every other
// group (no gain).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include <atomic>
#include <type_traits>

#include "kernels.h"
#include "paged.cuh"
#include "ptx.cuh"
#include "rows.cuh"

namespace dm {
namespace {

constexpr int kStages = 4;          // tiles of keys or values in flight: 128 KB beside 64 KB of queries
constexpr int kHalfBytes = 16384;   // 128 rows of 64 elements
constexpr int kTileBytes = 2 * kHalfBytes;
constexpr int kSoftThreads = 256;
constexpr int kThreads = kSoftThreads + 128;  // and two warps for keys and values, one for queries, one that multiplies
// Registers a thread: 168 at launch (384 threads share 65536); rows of 128 scores take more, the other warps less:
// 2 x 128 x 192 + 128 x 120 = 384 x 168.
constexpr int kSoftRegs = 192, kOtherRegs = 120;
constexpr int kS = 0, kO = 256;     // tensor memory columns: S of warpgroup w at 128 w, O at 256 + 128 w
// log2 of what a maximum may grow before O is scaled.  fp16 weights of 2^8 are far from 65504, bf16's and the sums' range is
// fp32's; scaling at every growth would wait for the products in most of the first tiles.  (Leaving small growths to the
// end's division is a published method.)
constexpr float kGrowth = 8.f;

constexpr int kSegments = 2;        // segments described ahead
constexpr int kTreeWords = 3;       // a token's ancestors among the first 96 new tokens, a bit each
constexpr int kConsumers = kSoftThreads / 32 + 3;  // warps that follow the segments: the softmax's, two loads, the products

struct Segment {
  Sequence s;
  int seq, head;
  int tok0, tokens;    // the group's, in the sequence
  int t0, t1, tiles;   // tiles of keys here, of all; none: the end of the line
  int last;            // the unit at which the last tile begins
};

struct Shared {
  uint64_t full[kStages], empty[kStages], s_full[2], w_half[2], w_ready[2], o_done[2], q_ready[2], q_free[2];
  uint64_t seg_ready[kSegments], seg_done[kSegments], met;
  uint32_t tmem;
  int abort, code;
  unsigned used[2][kStages];  // keys, values: the last copy into a stage, plus 1
  unsigned odd[2];  // by the segment's parity: the segment, from 1 on, that met a value that is not finite in a masked tile
  float norm[2][2][kAttendRows];  // accumulator: maximum, sum
  Segment seg[kSegments];
  uint32_t above[kSegments][2 * kAttendRows][kTreeWords];  // a tree's tokens: themselves and their ancestors
  int before[kAttendSeqs + 1];  // units of work before a sequence
  Sequence seq[kAttendSeqs];
};
constexpr size_t kSharedBytes = 1024 + static_cast<size_t>(2 + kStages) * kTileBytes + sizeof(Shared);
static_assert(kSharedBytes <= 232448, "a CTA's shared memory");

// Descriptors of 128-byte swizzled tiles differ in their low word alone (start address and, MN-major, the distance of
// blocks): 32-bit sums step them.
constexpr uint32_t kDescHigh = (1024 >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_low(uint32_t addr, uint32_t block) {
  return ((addr & 0x3FFFFu) >> 4) | ((block >> 4) << 16);
}

// D[tmem] (+)= A[smem] B[smem]^T, and D[tmem] (+)= A[tmem] B[smem], 16-bit operands, by their low words.
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\t"
      "mov.b64 x, {%1, %5};\n\tmov.b64 y, {%2, %5};\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(add), "n"(kDescHigh)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 y;\n\t"
      "mov.b64 y, {%2, %5};\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(add), "n"(kDescHigh)
      : "memory");
}
__device__ __forceinline__ bool elect_one() {
  uint32_t yes;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(yes));
  return yes != 0;
}

// Each thread of the warp writes 16 / 32 consecutive 32-bit columns of its TMEM lane.
__device__ __forceinline__ void tc_st_x16(uint32_t taddr, const float (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])), "r"(__float_as_uint(v[3])),
      "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])), "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7])),
      "r"(__float_as_uint(v[8])), "r"(__float_as_uint(v[9])), "r"(__float_as_uint(v[10])), "r"(__float_as_uint(v[11])),
      "r"(__float_as_uint(v[12])), "r"(__float_as_uint(v[13])), "r"(__float_as_uint(v[14])), "r"(__float_as_uint(v[15]))
      : "memory");
}

__device__ __forceinline__ void tc_st_x32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
      "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
      "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}

__device__ __forceinline__ void tc_wait_st() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// 16 bytes from global to shared memory, or zeros; cp.async.wait_all waits for the thread's.
__device__ __forceinline__ void copy_async(void* dst, const void* src, bool full) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(full ? 16 : 0) : "memory");
}
// One arrival for a warp, after what its threads did before.
__device__ __forceinline__ void warp_arrive(uint64_t* bar) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

template <int N>
__device__ __forceinline__ void regs_up() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void regs_down() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

__device__ __forceinline__ void fma2(float& x0, float& x1, float a, float b) {  // x = x a + b
  asm("{\n\t.reg .b64 x, y, z;\n\t"
      "mov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %2};\n\tmov.b64 z, {%3, %3};\n\t"
      "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "+f"(x0), "+f"(x1)
      : "f"(a), "f"(b));
}
__device__ __forceinline__ void add2(float& s0, float& s1, float x0, float x1) {
  asm("{\n\t.reg .b64 x, y;\n\t"
      "mov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\t"
      "add.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "+f"(s0), "+f"(s1)
      : "f"(x0), "f"(x1));
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi, __nv_bfloat16) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __half) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// ---------------------------------------------------------------- the line of work
// Keys that some token below `last` of a sequence sees, in tiles; a group that sees none still has one, for its rows'
// zeros.
__device__ __forceinline__ int key_tiles(int mask, const Sequence& s, int last) {
  const int seen = mask == kMaskCausal ? min(max(s.first + last, 0), s.kv) : s.kv;
  return max(1, seen / kAttendKeys + (seen % kAttendKeys != 0));
}

// What a group from token tok0 on counts: kAttendGroupCost for its queries and its end, and for every tile of keys what
// two tiles of queries, or one, cost there.
__device__ __forceinline__ int tile_cost(const AttendSplit& sp, int tokens) {
  return tokens > sp.tile_tokens ? kAttendTwoCost : kAttendOneCost;
}
__device__ __forceinline__ int group_units(const AttendParams& p, const AttendSplit& sp, const Sequence& s, int tok0) {
  const int tokens = min(2 * sp.tile_tokens, s.n - tok0);
  return kAttendGroupCost + key_tiles(p.mask, s, tok0 + tokens) * tile_cost(sp, tokens);
}

// A CTA's stretch of the line.  A tile of keys belongs to the stretch in which it begins.
struct Line {
  int at, end;
  int seq, head, tok0, u;  // u: units of the group before `at`

  __device__ __forceinline__ void begin(const Shared* sh, const AttendParams& p, const AttendSplit& sp, int from, int to) {
    at = from;
    end = to;
    if (at >= end) return;
    int lo = 0, hi = p.batch.B;
#pragma unroll 1
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (sh->before[mid] <= at) lo = mid; else hi = mid;
    }
    seq = lo;
    const int each = (sh->before[lo + 1] - sh->before[lo]) / p.cache.heads;
    u = at - sh->before[lo];
    head = u / each;
    u -= head * each;
    const Sequence s = sh->seq[seq];
    const int step = 2 * sp.tile_tokens, groups = (s.n + step - 1) / step;
    int g = 0;
    if (groups > 1 && p.mask != kMaskCausal) {  // all but the last alike
      const int n = group_units(p, sp, s, 0);
      g = min(u / n, groups - 1);
      u -= g * n;
    } else if (groups > 1) {  // every lane of the warp adds up a part of them; the one where u lies goes through its own
      const int lane = threadIdx.x & 31, share = (groups + 31) / 32;
      const int mine = min(groups, lane * share), stop = min(groups, mine + share);
      int sum = 0;
#pragma unroll 1
      for (int i = mine; i < stop; ++i) sum += group_units(p, sp, s, i * step);
      int upto = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(~0u, upto, o);
        if (lane >= o) upto += y;
      }
      const int owner = __ffs(__ballot_sync(~0u, u < upto)) - 1;
      u -= __shfl_sync(~0u, upto - sum, owner);
#pragma unroll 1
      for (g = owner * share;; ++g) {
        const int n = group_units(p, sp, s, g * step);
        if (u < n) break;
        u -= n;
      }
    }
    tok0 = g * step;
  }

  __device__ __forceinline__ bool next(const Shared* sh, const AttendParams& p, const AttendSplit& sp, Segment* g) {
#pragma unroll 1
    while (at < end) {
      while (sh->seq[seq].n == 0) ++seq;
      g->s = sh->seq[seq];
      g->seq = seq;
      g->head = head;
      g->tok0 = tok0;
      g->tokens = min(2 * sp.tile_tokens, g->s.n - tok0);
      g->tiles = key_tiles(p.mask, g->s, tok0 + g->tokens);
      const int cost = tile_cost(sp, g->tokens), all = kAttendGroupCost + g->tiles * cost;
      const int n = min(all - u, end - at);
      g->t0 = (max(u - kAttendGroupCost, 0) + cost - 1) / cost;
      u += n;
      at += n;
      g->t1 = (max(u - kAttendGroupCost, 0) + cost - 1) / cost;
      g->last = at - u + all - cost;
      if (u == all) {
        u = 0;
        tok0 += 2 * sp.tile_tokens;
        if (tok0 >= g->s.n) {
          tok0 = 0;
          if (++head == p.cache.heads) {
            head = 0;
            ++seq;
          }
        }
      }
      if (g->t1 > g->t0) return true;
    }
    return false;
  }
};

// A sequence's units; -1 where a causal one has several groups, each of its own length.
__device__ __forceinline__ int sequence_units(const AttendParams& p, const AttendSplit& sp, const Sequence& s) {
  const int step = 2 * sp.tile_tokens, groups = (s.n + step - 1) / step;
  if (p.mask == kMaskCausal && groups > 1) return -1;
  if (groups == 0) return 0;
  return ((groups - 1) * group_units(p, sp, s, 0) + group_units(p, sp, s, (groups - 1) * step)) * p.cache.heads;
}

// The first key that some token from tok0 on may not see.
__device__ __forceinline__ int masked_from(const AttendParams& p, const Sequence& s, int tok0) {
  if (p.mask == kMaskFull) return s.kv;
  return min(max(s.first + (p.mask == kMaskCausal ? tok0 + 1 : 0), 0), s.kv);
}

// Whether a tree's tokens have their ancestors in `above`.
__device__ __forceinline__ bool tree_in_words(const AttendParams& p, const Segment& g) {
  return p.mask == kMaskTree && g.s.n <= 32 * kTreeWords;
}

// Which of 128 keys from key0 on token i sees, a bit each.
__device__ __forceinline__ void seen_bits(const AttendParams& p, const Segment& g, const uint32_t* above, int i, int key0,
                                          uint32_t (&bits)[4]) {
  const int first = g.s.first;
  int limit = g.s.kv;  // every key below it is seen
  if (p.mask == kMaskCausal) limit = min(max(first + i + 1, 0), g.s.kv);
  if (p.mask == kMaskTree) limit = i > p.N ? 0 : min(max(first, 0), g.s.kv);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const int n = limit - key0 - 32 * w;
    bits[w] = n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1;
  }
  if (p.mask != kMaskTree || i > p.N) return;
  if (tree_in_words(p, g)) {  // (places before 0 are nobody's)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int t = key0 + 32 * w - first, word = t >> 5;  // the word of keys begins at new token t
      const uint32_t lo = word >= 0 && word < kTreeWords ? above[word] : 0;
      const uint32_t hi = word >= -1 && word < kTreeWords - 1 ? above[word + 1] : 0;
      bits[w] |= __funnelshift_r(lo, hi, t & 31);
      const int n = g.s.kv - key0 - 32 * w;  // new tokens past the table have no key
      if (n < 32) bits[w] &= n <= 0 ? 0u : (1u << n) - 1;
    }
    return;
  }
  const int32_t* const parent = p.parent + static_cast<long long>(g.seq) * p.N;
  for (int a = i;; a = tree_up(parent, a)) {
    const int at = first + a - key0;
    if (at < 0) break;
    const uint32_t bit = 1u << (at & 31);
#pragma unroll
    for (int w = 0; w < 4; ++w)
      if (at >> 5 == w && key0 + at < g.s.kv) bits[w] |= bit;
    if (a == 0) break;
  }
}

// A wait of its own limit for what is in flight when the others have given up.
__device__ __forceinline__ void drain_wait(uint64_t* bar, uint32_t parity) {
  const long long t0 = clock64();
  while (!mbar_try_wait(bar, parity) && clock64() - t0 < kWaitCycles) {
  }
}

// ---------------------------------------------------------------- warps
// The whole warp waits; false: somebody has given up.
__device__ __forceinline__ bool warp_wait(Shared* sh, uint64_t* bar, uint32_t parity) {
  return __all_sync(~0u, mbar_wait(bar, parity, &sh->abort, &sh->code));
}
// The warp's segment number `index`, or nullptr at the end of the line.
__device__ __forceinline__ const Segment* next_segment(Shared* sh, unsigned index) {
  if (!warp_wait(sh, &sh->seg_ready[index % kSegments], index / kSegments & 1)) return nullptr;
  const Segment* const g = &sh->seg[index % kSegments];
  return g->t1 > g->t0 ? g : nullptr;
}
__device__ __forceinline__ void segment_done(Shared* sh, unsigned index) { warp_arrive(&sh->seg_done[index % kSegments]); }

// Tiles of a segment with n of them pass the ring as K_0 .. K_(a-1), then V_j and K_(j+a) in turn: the order in which the
// products want them, a = 1 where both warpgroups take every tile, 2 where they alternate.
__device__ __forceinline__ int value_place(int j, int n, int ahead) { return min(ahead, n) + j + min(j, max(0, n - ahead)); }
__device__ __forceinline__ int key_place(int j, int n, int ahead) { return j < ahead ? j : value_place(j - ahead, n, ahead) + 1; }

// One warp brings the keys, one the values: a copy a piece (what a page has in common with a tile) and half of the
// elements.  A lane a piece keeps the piece's place and looks its page up a tile ahead.
__device__ void load_warp(Shared* sh, uint8_t* ring, const CUtensorMap* map, bool values, const AttendParams& p,
                          const AttendSplit& sp) {
  const int lane = threadIdx.x & 31;
  const int pieces = kAttendKeys / sp.piece, page_size = p.cache.page;
  const bool two_halves = p.cache.D > 64;
  const uint32_t bytes = two_halves ? kTileBytes : kHalfBytes;
  const int pages_on = kAttendKeys / page_size, places_on = kAttendKeys % page_size;
  const uint64_t keep = l2_policy_evict_last(), drop = l2_policy_evict_first();
  const unsigned held = !values && sp.held == static_cast<int>(blockIdx.x) ? 0u : ~0u;  // test hook: the copy withheld
  unsigned base = 0, used[kStages] = {};
  bool ok = true;
  const Segment* g;
  for (unsigned index = 0; ok && (g = next_segment(sh, index)) != nullptr; ++index) {
    const int n = g->t1 - g->t0, ahead = g->tokens > sp.tile_tokens ? 1 : 2, kv = g->s.kv, head = g->head;
    const int32_t* const table = p.batch.table + g->seq * p.batch.table_stride;
    const uint64_t policy = g->tok0 + g->tokens < g->s.n ? keep : drop;  // the next group of queries reads the same tiles
    int place = g->t0 * kAttendKeys + lane * sp.piece, entry = place / page_size, token = place - entry * page_size;
    auto inside = [&]() { return lane < pieces && static_cast<unsigned>(place) < static_cast<unsigned>(kv); };
    int found = inside() ? table[entry] : 0;
    for (int j = 0; j < n; ++j) {
      int page = found;
      const int here = token;
      if (!inside()) {
        page = p.cache.pages;  // past the last page: reads as zeros
      } else if (page < 0 || page >= p.cache.pages) {
        sh->code = kStatusBadPage;
        page = p.cache.pages;
      }
      place += kAttendKeys;
      entry += pages_on;
      token += places_on;
      if (token >= page_size) {
        token -= page_size;
        ++entry;
      }
      if (j + 1 < n && inside()) found = table[entry];
      const unsigned at = base + (values ? value_place(j, n, ahead) : key_place(j, n, ahead));
      const int stage = at % kStages;
      ok = at < kStages || warp_wait(sh, &sh->empty[stage], (at / kStages - 1) & 1);
      if (!ok) break;
      uint8_t* dst = ring + stage * kTileBytes;
      if (at != held && elect_one()) mbar_arrive_expect_tx(&sh->full[stage], bytes);
      __syncwarp();
#pragma unroll 1
      for (int q = at != held ? 0 : pieces; q < pieces; ++q, dst += sp.piece * 128) {
        const int y = __shfl_sync(~0u, here, q), w = __shfl_sync(~0u, page, q);
        if (elect_one()) {
          tma_load_4d(dst, map, &sh->full[stage], 0, y, head, w, policy);
          if (two_halves) tma_load_4d(dst + kHalfBytes, map, &sh->full[stage], 64, y, head, w, policy);
        }
      }
#pragma unroll
      for (int i = 0; i < kStages; ++i) used[i] = i == stage ? at + 1 : used[i];
    }
    base += 2 * n;
    segment_done(sh, index);
  }
  if (lane == 0)
#pragma unroll
    for (int i = 0; i < kStages; ++i) sh->used[values][i] = used[i];
}

// The whole warp follows the segments, one thread issues: what steers the products stays in uniform registers.  The tensor core
// waits for little else than this warp, so the loops are written out for either kind of group.
template <typename T>
__device__ void multiply_warp(Shared* sh, uint32_t q_addr, uint32_t ring_addr, const AttendParams& p, const AttendSplit& sp) {
  constexpr bool kBf = !std::is_same<T, __half>::value;
  const int steps = (p.cache.D + 15) / 16;
  const uint32_t tmem = sh->tmem;
  const uint32_t qk = idesc_16_f32(kBf, kAttendRows, kAttendKeys, false), wv = idesc_16_f32(kBf, kAttendRows, 16 * steps, true);
  unsigned it = 0, turns[2] = {0, 0}, queries[2] = {0, 0};  // tiles, weights of an accumulator, tiles of queries
  auto take = [&]() {
    const unsigned stage = it % kStages;
    const bool ok = warp_wait(sh, &sh->full[stage], (it / kStages) & 1);
    ++it;
    return ok ? static_cast<int>(stage) : -1;
  };
  // S of accumulator w from query tile `tile` and the keys in `stage`; last: nobody else wants them; free: nor the queries
  auto scores = [&](int w, int tile, int stage, bool last, bool free) {
    tc_fence_after();
    const uint32_t a = desc_low(q_addr + tile * kTileBytes, 16), b = desc_low(ring_addr + stage * kTileBytes, 16);
    if (elect_one()) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint32_t step = (k >> 2) * (kHalfBytes >> 4) + (k & 3) * 2;
        if (k < steps) mma_ss(tmem + kS + 128 * w, a + step, b + step, qk, k > 0);
      }
      tc_commit(&sh->s_full[w]);
      if (last) tc_commit(&sh->empty[stage]);
      if (free) tc_commit(&sh->q_free[tile]);
    }
    __syncwarp();
  };
  // Half of O of accumulator w, from its weights of 64 keys and the values in `stage`
  auto weigh = [&](int w, int half, int stage, bool add, bool last) {
    tc_fence_after();
    const uint32_t b = desc_low(ring_addr + stage * kTileBytes + half * (kHalfBytes / 2), kHalfBytes);
    if (elect_one()) {
#pragma unroll
      for (int k = 0; k < kAttendKeys / 32; ++k)
        mma_ts(tmem + kO + 128 * w, tmem + kS + 128 * w + 32 * half + 8 * k, b + k * (2048 >> 4), wv, k > 0 ? 1 : add);
      if (half) tc_commit(&sh->o_done[w]);
      if (half && last) tc_commit(&sh->empty[stage]);
    }
    __syncwarp();
  };
  auto halves = [&](int w) { return warp_wait(sh, &sh->w_half[w], turns[w] & 1); };
  auto weights = [&](int w) { return warp_wait(sh, &sh->w_ready[w], turns[w]++ & 1); };
  auto queried = [&](int tile) { return warp_wait(sh, &sh->q_ready[tile], queries[tile]++ & 1); };
  const Segment* g;
  for (unsigned index = 0; (g = next_segment(sh, index)) != nullptr; ++index) {
    const bool two = g->tokens > sp.tile_tokens;
    const int n = g->t1 - g->t0;
    segment_done(sh, index);
    if (!queried(0)) return;
    if (two) {
      int k = take();
      if (k < 0) return;
      scores(0, 0, k, false, n == 1);
      if (!queried(1)) return;
      scores(1, 1, k, true, n == 1);
      for (int j = 0; j < n; ++j) {
        if (!halves(0)) return;
        const int v = take();
        if (v < 0) return;
        weigh(0, 0, v, j > 0, false);
        if (!weights(0)) return;
        weigh(0, 1, v, true, false);
        if (j + 1 < n) {
          k = take();
          if (k < 0) return;
          scores(0, 0, k, false, j + 2 == n);
        }
        if (!halves(1)) return;
        weigh(1, 0, v, j > 0, true);
        if (!weights(1)) return;
        weigh(1, 1, v, true, true);
        if (j + 1 < n) scores(1, 1, k, true, j + 2 == n);
      }
    } else {
      for (int w = 0; w < 2 && w < n; ++w) {
        const int k = take();
        if (k < 0) return;
        scores(w, 0, k, true, n <= 2 && w + 1 == n);
      }
      for (int j = 0; j < n; ++j) {
        const int w = j & 1;
        if (!halves(w)) return;
        const int v = take();
        if (v < 0) return;
        weigh(w, 0, v, j >= 2, true);
        if (!weights(w)) return;
        weigh(w, 1, v, true, true);
        if (j + 2 < n) {
          const int k = take();
          if (k < 0) return;
          scores(w, 0, k, true, j + 3 == n);
        }
      }
    }
  }
}

// Sets what is not finite among two elements to 0; true if something was.
template <typename T>
__device__ __forceinline__ bool drop_odd(uint32_t* w) {
  constexpr uint32_t kExp = std::is_same<T, __half>::value ? 0x7C00u : 0x7F80u;  // all ones: infinity or NaN
  const uint32_t keep = ((*w & kExp) == kExp ? 0 : 0xFFFFu) | ((*w & kExp << 16) == kExp << 16 ? 0 : 0xFFFF0000u);
  *w &= keep;
  return keep != ~0u;
}

// Byte offset of a row's 16-byte unit in a 128-byte swizzled tile.
__device__ __forceinline__ uint32_t unit_offset(int row, int unit) {
  return (unit >> 3) * kHalfBytes + row * 128 + (((unit & 7) ^ (row & 7)) << 4);
}

// A tile's queries into shared memory, by `threads` threads of which this is number `tid`: 16 bytes each, zeros behind the
// last element.  Rows without a query keep what they hold: it reaches nobody.
template <typename T>
__device__ __forceinline__ void bring_queries(uint8_t* dst, int tile, const AttendParams& p, const AttendSplit& sp,
                                              const Segment& g, int tid, int threads) {
  const int G = p.group, units = (p.cache.D + 15) / 16 * 2, step = threads / units;
  const int unit = tid % units, tok0 = tile * sp.tile_tokens, rows = min(sp.tile_tokens, g.tokens - tok0) * G;
  const int inv_group = (65536 + G - 1) / G;  // row / G, rows below 128
  if (tid / units < step)
#pragma unroll 2
    for (int row = tid / units; row < rows; row += step) {
      const int tk = row * inv_group >> 16;
      const T* const src = static_cast<const T*>(p.q) + (g.s.row + g.tok0 + tok0 + tk) * p.q_stride +
                           static_cast<int64_t>(g.head * G + row - tk * G) * p.cache.D + 8 * unit;
      const bool is = 8 * unit < p.cache.D;
      copy_async(dst + unit_offset(row, unit), is ? src : static_cast<const T*>(p.q), is);
    }
  asm volatile("cp.async.wait_all;" ::: "memory");
  fence_async_smem();
}

// A warp that walks the line: describes the segments, brings their queries (but the first's) as soon as the products are
// done with the ones before, and notes the group that goes on behind this stretch for the kernel that joins.
template <typename T>
__device__ void line_warp(Shared* sh, uint8_t* q_smem, const AttendParams& p, const AttendSplit& sp, Line line, int each) {
  const int lane = threadIdx.x & 31;
  unsigned queries[2] = {0, 0};
  AttendTail tail{-1, 0, 0, 0};
  Segment g;
  for (unsigned index = 0;; ++index) {
    const bool more = line.next(sh, p, sp, &g);
    const unsigned slot = index % kSegments;
    if (index >= kSegments && !warp_wait(sh, &sh->seg_done[slot], (index / kSegments - 1) & 1)) break;
    if (!more) g.t0 = g.t1 = 0;
    if (more && tree_in_words(p, g)) {
      const int32_t* const parent = p.parent + static_cast<long long>(g.seq) * p.N;
      for (int t = lane; t < g.tokens; t += 32) {
        uint32_t words[kTreeWords] = {};
        for (int a = min(g.tok0 + t, p.N);; a = tree_up(parent, a)) {  // (tokens past the tree see nothing anyway)
#pragma unroll
          for (int w = 0; w < kTreeWords; ++w) words[w] |= a >> 5 == w ? 1u << (a & 31) : 0u;
          if (a == 0) break;
        }
#pragma unroll
        for (int w = 0; w < kTreeWords; ++w) sh->above[slot][t][w] = words[w];
      }
    }
    if (lane == 0) sh->seg[slot] = g;
    warp_arrive(&sh->seg_ready[slot]);
    if (!more) break;
    const bool two = g.tokens > sp.tile_tokens;
    if (g.t0 == 0 && g.t1 < g.tiles) tail = AttendTail{g.last / each, g.s.row + g.tok0, g.head, g.tokens};
#pragma unroll 1
    for (int tile = 0; tile < (two ? 2 : 1); ++tile) {
      const unsigned use = queries[tile]++;
      if (index == 0 || sh->abort) continue;
      if (use > 0 && !warp_wait(sh, &sh->q_free[tile], (use - 1) & 1)) continue;
      bring_queries<T>(q_smem + tile * kTileBytes, tile, p, sp, g, lane, 32);
      warp_arrive(&sh->q_ready[tile]);
    }
  }
  if (lane == 0) sp.tails[blockIdx.x] = tail;
}

// One warpgroup: a row's softmax, the end of a segment.
template <typename T>
__device__ void soft_group(Shared* sh, uint8_t* q_smem, uint8_t* ring, const AttendParams& p, const AttendSplit& sp) {
  const int w = threadIdx.x >> 7, r = threadIdx.x & 127, lane_base = (threadIdx.x >> 5 & 3) * 32;
  const int D = p.cache.D, G = p.group, steps = (D + 15) / 16, units = 2 * steps;
  const uint32_t tmem = sh->tmem + (static_cast<uint32_t>(lane_base) << 16);
  const uint32_t s_col = tmem + kS + 128 * w, o_col = tmem + kO + 128 * w;
  const float c = p.scale_log2;
  const int tile_rows = sp.tile_tokens * G;
  const int my_tok = r / G, my_head = r - my_tok * G;  // of a tile
  const int row_step = 128 / units, unit_row = r / units, unit = r - unit_row * units;  // 16 bytes a thread
  unsigned segment = 0, turn = 0, base = 0, meetings = 0;
  auto meet = [&]() {  // all warps of both accumulators
    warp_arrive(&sh->met);
    return warp_wait(sh, &sh->met, meetings++ & 1);
  };
  bool crossed = false;
  const Segment* seg;
  for (; (seg = next_segment(sh, segment)) != nullptr; ++segment) {
    const Segment& g = *seg;
    const bool two = g.tokens > sp.tile_tokens;
    const int n = g.t1 - g.t0, ahead = two ? 1 : 2;
    const int tile = two ? w : 0;
    if (segment == 0) {  // everybody brings the first queries
      bring_queries<T>(q_smem + tile * kTileBytes, tile, p, sp, g, two ? r : threadIdx.x, two ? 128 : kSoftThreads);
      if (!meet()) return;
      if (threadIdx.x == 0) mbar_arrive(&sh->q_ready[0]);
      if (threadIdx.x == 128 && two) mbar_arrive(&sh->q_ready[1]);
      __syncwarp();
    } else if (crossed) {  // the other accumulator's warps have read ours
      if (!meet()) return;
    }
    crossed = !two;
    const int tok = tile * sp.tile_tokens + my_tok;  // in the group
    const bool valid = r < tile_rows && tok < g.tokens;
    const bool busy = __any_sync(~0u, valid);  // a warp without rows only keeps time: what its lanes hold reaches nobody
    const int i = g.tok0 + tok;
    const int from = masked_from(p, g.s, g.tok0 + tile * sp.tile_tokens);
    float m = -INFINITY, l = 0.f;
    for (int j = two ? 0 : w; j < n; j += two ? 1 : 2, ++turn) {
      const bool started = j >= (two ? 1 : 2);
      const int key0 = (g.t0 + j) * kAttendKeys;
      const bool masked = key0 + kAttendKeys > from;
      if (!warp_wait(sh, &sh->s_full[w], turn & 1)) return;
      tc_fence_after();
      if (masked) {  // values that weights of 0 must not meet
        const unsigned place = base + value_place(j, n, ahead);
        const int stage = place % kStages, row0 = max(from - key0, 0);
        if (!warp_wait(sh, &sh->full[stage], (place / kStages) & 1)) return;
        if (unit_row < row_step)
#pragma unroll 2
          for (int row = row0 + unit_row; row < kAttendKeys; row += row_step) {
            uint4* const at = reinterpret_cast<uint4*>(ring + stage * kTileBytes + unit_offset(row, unit));
            if (key0 + row >= g.s.kv) {
              *at = make_uint4(0, 0, 0, 0);
            } else {
              uint4 v = *at;
              if (drop_odd<T>(&v.x) | drop_odd<T>(&v.y) | drop_odd<T>(&v.z) | drop_odd<T>(&v.w)) {
                *reinterpret_cast<volatile unsigned*>(&sh->odd[segment & 1]) = segment + 1;
                __threadfence_block();
                *at = v;
              }
            }
          }
        fence_async_smem();
        __syncwarp();
      }
      auto softmax = [&](auto Masked) {
        constexpr bool kMasked = decltype(Masked)::value;
        float s[4][32], top[4];
        uint32_t bits[4] = {0, 0, 0, 0};
#pragma unroll
        for (int x = 0; x < 4; ++x) tc_ld_x32(s_col + 32 * x, s[x]);
        if constexpr (kMasked) {
          if (valid) seen_bits(p, g, sh->above[segment % kSegments][tok], i, key0, bits);
          __syncwarp();
        }
        tc_wait_ld();
        if constexpr (kMasked) {
#pragma unroll
          for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int y = 0; y < 32; ++y) s[x][y] = bits[x] >> y & 1 ? s[x][y] : -INFINITY;
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          top[x] = fmaxf(s[x][0], s[x][1]);
#pragma unroll
          for (int y = 2; y < 32; y += 2) top[x] = fmaxf(fmaxf(top[x], s[x][y]), s[x][y + 1]);
        }
        const float seen = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
        if (!started) {
          m = seen;
        } else {
          const float up = fmaxf(m, seen);
          if (__any_sync(~0u, valid && (up - m) * c > kGrowth)) {
            const float keep = m == up ? 1.f : ex2((m - up) * c);
            mbar_wait(&sh->o_done[w], (turn - 1) & 1, &sh->abort, &sh->code);
            tc_fence_after();
#pragma unroll 1
            for (int d = 0; d < steps; ++d) {
              float o[16];
              tc_ld_x16(o_col + 16 * d, o);
              tc_wait_ld();
#pragma unroll
              for (int x = 0; x < 16; ++x) o[x] *= keep;
              tc_st_x16(o_col + 16 * d, o);
            }
            l *= keep;
            m = up;
          }
        }
        const float mc = m == -INFINITY ? 0.f : -m * c;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < 4; x += 2) {
          uint32_t pk[32];
#pragma unroll
          for (int y = 0; y < 64; y += 2) {
            float a = s[x + y / 32][y % 32], b = s[x + y / 32][y % 32 + 1];
            fma2(a, b, c, mc);
            a = ex2(a);
            b = ex2(b);
            add2(sum[y & 2], sum[(y & 2) + 1], a, b);
            pk[y / 2] = pack2(a, b, T());
          }
          tc_st_x32(s_col + 16 * x, pk);
          if (x == 0) {
            tc_wait_st();
            tc_fence_before();
            warp_arrive(&sh->w_half[w]);
          }
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        tc_wait_st();
      };
      if (busy) {
        if (masked) softmax(std::true_type());
        else softmax(std::false_type());
      } else {
        tc_fence_before();
        warp_arrive(&sh->w_half[w]);
      }
      tc_fence_before();
      warp_arrive(&sh->w_ready[w]);
    }

    // the segment's end: sums into the output, or into the workspace where the group's keys go on elsewhere
    const bool any = n > (two ? 0 : w);
    if (any && !warp_wait(sh, &sh->o_done[w], (turn - 1) & 1)) return;
    tc_fence_after();
    float f0 = 1.f, f1 = 0.f;  // one tile of queries: the warpgroups' weights
    if (!two) {
      sh->norm[w][0][r] = m;
      sh->norm[w][1][r] = l;
      tc_fence_before();
      if (!meet()) return;
      tc_fence_after();
      const float m0 = sh->norm[0][0][r], m1 = sh->norm[1][0][r];
      m = fmaxf(m0, m1);
      f0 = m0 == -INFINITY ? 0.f : m0 == m ? 1.f : ex2((m0 - m) * c);
      f1 = m1 == -INFINITY ? 0.f : m1 == m ? 1.f : ex2((m1 - m) * c);
      l = sh->norm[0][1][r] * f0 + sh->norm[1][1][r] * f1;
    }
    if (p.mask == kMaskTree && i > p.N) {  // past the tree: nothing seen, though tiles before the new tokens ask no mask
      m = -INFINITY;
      l = 0.f;
    }
    const bool odd = *reinterpret_cast<volatile unsigned*>(&sh->odd[segment & 1]) == segment + 1;
    const bool whole = g.t0 == 0 && g.t1 == g.tiles;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int slot = 2 * blockIdx.x + (g.t0 == 0 ? 1 : 0), slot_row = tile * kAttendRows + r;
    const long long row = g.s.row + i;
    const int head = g.head * G + my_head;
    T* const out = static_cast<T*>(p.out) + row * p.out_stride + static_cast<long long>(head) * D;
    float* const part = sp.parts + static_cast<long long>(slot) * D * sp.slot_rows + slot_row;
    const int share = two ? 0 : w, shares = two ? 1 : 2;  // of the blocks of 16 elements
    if (busy)
#pragma unroll 1
      for (int d = 16 * share; d < D; d += 16 * shares) {
        float o[16];
        if (two) {
          tc_ld_x16(o_col + d, o);
          tc_wait_ld();
        } else {
          float o1[16];
          tc_ld_x16(tmem + kO + d, o);
          tc_ld_x16(tmem + kO + 128 + d, o1);
          tc_wait_ld();
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            if (f0 == 0.f) o[x] = 0.f;
            if (f1 == 0.f) o1[x] = 0.f;
            o[x] = fmaf(o[x], f0, o1[x] * f1);
          }
        }
        if (valid) {
#pragma unroll
          for (int x = 0; x < 16; x += 8) {
            if (d + x >= D) break;
            if (whole) {
              float y[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) y[e] = o[x + e] * inv;
              Vec<T> v;
              pack(y, &v);
              if (l == 0.f) v.raw = make_uint4(0, 0, 0, 0);
              *reinterpret_cast<uint4*>(out + d + x) = v.raw;
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e) part[static_cast<long long>(d + x + e) * sp.slot_rows] = o[x + e];
            }
          }
        }
        __syncwarp();  // the loads of tensor memory are the whole warp's
      }
    if (odd && valid) {  // what was left out of the products, where this row sees it
      const int end = min(g.s.kv, g.t1 * kAttendKeys);
      const int32_t* const parent = p.parent ? p.parent + static_cast<long long>(g.seq) * p.N : nullptr;
#pragma unroll 1
      for (int key = max(masked_from(p, g.s, g.tok0), g.t0 * kAttendKeys); key < end; ++key) {
        if (!sees(p.mask, parent, p.N, i, g.s.first, key)) continue;
        const long long off = place_offset(p.cache, p.batch, g.seq, key);
        if (off < 0) continue;
        const T* const v = static_cast<const T*>(p.cache.v) + off + g.head * p.cache.head_stride;
#pragma unroll 1
        for (int d = 0; d < D; ++d) {
          const float f = to_f32(v[d]);
          if (isfinite(f) || (d >> 4) % shares != share) continue;
          if (whole)
            from_f32(to_f32(out[d]) + f, out + d);
          else
            part[static_cast<long long>(d) * sp.slot_rows] += f;
        }
      }
    }
    if (valid && (two || w == 0)) {
      if (!whole) {
        float* const norm = sp.norms + static_cast<long long>(slot) * 2 * sp.slot_rows + slot_row;
        norm[0] = m;
        norm[sp.slot_rows] = l;
      } else if (p.lse) {
        p.lse[row * p.hq + head] = l == 0.f ? -INFINITY : fmaf(m, p.scale, logf(l));
      }
    }
    tc_fence_before();
    base += 2 * n;
    segment_done(sh, segment);
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 1)
    attend_kernel(const __grid_constant__ CUtensorMap keys, const __grid_constant__ CUtensorMap values, const AttendParams p,
                  const AttendSplit sp) {
  extern __shared__ uint8_t raw[];
  uint8_t* const tiles = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);  // queries, then the ring
  uint8_t* const ring = tiles + 2 * kTileBytes;
  Shared* const sh = reinterpret_cast<Shared*>(ring + kStages * kTileBytes);
  const int tid = threadIdx.x, warp = tid >> 5;
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&sh->full[i], 1);
      mbar_init(&sh->empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh->s_full[i], 1);
      mbar_init(&sh->w_half[i], 4);
      mbar_init(&sh->w_ready[i], 4);  // a warp each
      mbar_init(&sh->o_done[i], 1);
      mbar_init(&sh->q_ready[i], 1);
      mbar_init(&sh->q_free[i], 1);
      sh->odd[i] = 0;
    }
    for (int i = 0; i < kSegments; ++i) {
      mbar_init(&sh->seg_ready[i], 1);
      mbar_init(&sh->seg_done[i], kConsumers);
    }
    mbar_init(&sh->met, kSoftThreads / 32);
    fence_mbar_init();
    sh->abort = 0;
    sh->code = 0;
    tma_prefetch_desc(&keys);
    tma_prefetch_desc(&values);
  }
  if (warp == kSoftThreads / 32) {
    tmem_alloc(&sh->tmem, 512);
    tmem_relinquish();
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  bool several = false;
#pragma unroll 1
  for (int b = tid; b < p.batch.B; b += kThreads) {
    const Sequence s = load_sequence(p.cache, p.batch, p.tokens, b);
    const int n = sequence_units(p, sp, s);
    several = several || n < 0;
    sh->seq[b] = s;
    sh->before[b + 1] = n;
  }
  if (tid == 0) sh->before[0] = 0;
  tc_fence_before();
  several = __syncthreads_or(several);
  tc_fence_after();
  const int lane = tid & 31;
  if (several) {  // a warp a sequence, a lane a group
    const int step = 2 * sp.tile_tokens;
    for (int b = warp; b < p.batch.B; b += kThreads / 32) {
      if (sh->before[b + 1] >= 0) continue;
      const Sequence s = sh->seq[b];
      int n = 0;
#pragma unroll 1
      for (int t = lane * step; t < s.n; t += 32 * step) n += group_units(p, sp, s, t);
#pragma unroll
      for (int o = 16; o; o >>= 1) n += __shfl_xor_sync(~0u, n, o);
      __syncwarp();
      if (lane == 0) sh->before[b + 1] = n * p.cache.heads;
    }
    __syncthreads();
  }
  if (warp == 0) {
    int carry = 0;
#pragma unroll 1
    for (int b = 0; b < p.batch.B; b += 32) {
      int x = b + tid < p.batch.B ? sh->before[b + tid + 1] : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(~0u, x, o);
        if (tid >= o) x += y;
      }
      x += carry;
      if (b + tid < p.batch.B) sh->before[b + tid + 1] = x;
      carry = __shfl_sync(~0u, x, 31);
    }
  }
  __syncthreads();
  const int units = sh->before[p.batch.B], ctas = gridDim.x, cta = blockIdx.x;
  const int each = max(kAttendLeast, (units + ctas - 1) / ctas), from = cta < (units + each - 1) / each ? cta * each : units;
  Line line;
  line.begin(sh, p, sp, from, from + min(each, units - from));
  if (tid < kSoftThreads) {
    regs_up<kSoftRegs>();
    soft_group<T>(sh, tiles, ring, p, sp);
  } else {
    regs_down<kOtherRegs>();
    if (warp == kSoftThreads / 32 || warp == kSoftThreads / 32 + 2) {
      const bool v = warp == kSoftThreads / 32 + 2;
      load_warp(sh, ring, v ? &values : &keys, v, p, sp);
    }
    if (warp == kSoftThreads / 32 + 1) {
      multiply_warp<T>(sh, smem_u32(tiles), smem_u32(ring), p, sp);
      if (sh->abort) {  // products in flight read the tiles and write the accumulators: they take microseconds
        const long long t0 = clock64();
        while (clock64() - t0 < kWaitCycles / 1024) {
        }
      }
    }
    if (warp == kSoftThreads / 32 + 3) line_warp<T>(sh, tiles, p, sp, line, each);
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (tid == 0) {
    sp.codes[blockIdx.x] = sh->code;
    if (sh->abort)  // copies that nobody has waited for write into this CTA's memory
      for (int i = 0; i < kStages; ++i) {
        const unsigned last = max(sh->used[0][i], sh->used[1][i]);
        if (last) drain_wait(&sh->full[i], ((last - 1) / kStages) & 1);
      }
  }
  if (warp == kSoftThreads / 32) {
    tc_fence_after();
    tmem_dealloc(sh->tmem, 512);
  }
}

// ---------------------------------------------------------------- joining
constexpr int kJoinThreads = 256;
constexpr int kJoinRows = 32;  // rows a block: a lane a row
constexpr int kJoinAhead = 4;  // partial results in flight
constexpr int kJoinElems = 4;  // elements a thread

// Bound by the latency of its loads: 2.5 us for one token's 8 parts of 8 heads, some 4 for 8 groups of 19 parts (5.7 with one way),
// 15-20 for 152 groups of two or three parts of 256 rows.
// The group that CTA blockIdx.x began and others went on with: 32 of its rows' sums over all of them, in a fixed order.  Rows
// lie side by side in the slots: a lane takes a row, a warp four elements and every WAYS-th part; the ways meet and the
// results turn round in shared memory.  Few rows have many parts: four ways.
template <typename T, int WAYS>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const AttendParams p, const AttendSplit sp) {
  constexpr int kCols = kJoinThreads / 32 / WAYS * kJoinElems;  // elements a block
  __shared__ float s_o[WAYS][kJoinRows][kCols + 1], s_m[WAYS][kJoinRows], s_l[WAYS][kJoinRows];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, way = warp % WAYS, cols = warp / WAYS * kJoinElems;
  if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0 && warp == 0) {
    int code = 0;
    for (unsigned i = lane; i < gridDim.x; i += 32) {
      const int x = sp.codes[i];
      code = x != 0 ? x : code;
    }
    const unsigned bad = __ballot_sync(~0u, code != 0);
    if (bad) code = __shfl_sync(~0u, code, __ffs(bad) - 1);
    if (lane == 0 && (sp.first || code != 0)) *p.status = code;
  }
  const AttendTail tail = sp.tails[blockIdx.x];
  const int D = p.cache.D, G = p.group, rows = tail.tokens * G, first = blockIdx.x, row0 = blockIdx.y * kJoinRows;
  const int col0 = blockIdx.z * kCols, d = col0 + cols;  // D is a multiple of 8: four elements, or none
  if (tail.last < 0 || row0 >= rows) return;
  const long long slot_rows = sp.slot_rows;
  const int at = min(row0 + lane, rows - 1), tok = at / G;
  const int slot_row = tok < sp.tile_tokens ? at : kAttendRows + at - sp.tile_tokens * G;
  float m = -INFINITY, l = 0.f, o[kJoinElems];
#pragma unroll
  for (int e = 0; e < kJoinElems; ++e) o[e] = 0.f;
  for (int i0 = first + way; i0 <= tail.last; i0 += WAYS * kJoinAhead) {
    float mi[kJoinAhead], li[kJoinAhead], v[kJoinAhead][kJoinElems];
#pragma unroll
    for (int i = 0; i < kJoinAhead; ++i) {
      const int cta = i0 + WAYS * i;
      if (cta > tail.last) {
        mi[i] = -INFINITY;
        li[i] = 0.f;
        continue;
      }
      const long long slot = cta == first ? 2 * first + 1 : 2 * cta;
      const float* const norm = sp.norms + slot * 2 * slot_rows + slot_row;
      const float* const part = sp.parts + (slot * D + d) * slot_rows + slot_row;
      mi[i] = norm[0];
      li[i] = norm[slot_rows];
#pragma unroll
      for (int e = 0; e < kJoinElems; ++e) v[i][e] = d < D ? part[e * slot_rows] : 0.f;
    }
    float up = m;
#pragma unroll
    for (int i = 0; i < kJoinAhead; ++i) up = fmaxf(up, mi[i]);
    const float keep = m == up ? 1.f : ex2((m - up) * p.scale_log2);
    m = up;
    l *= keep;
#pragma unroll
    for (int e = 0; e < kJoinElems; ++e) o[e] *= keep;
#pragma unroll
    for (int i = 0; i < kJoinAhead; ++i) {
      // no part, or one that saw nothing: sums of 0.  (A NaN score is no maximum: it shows in the sum alone.)
      if (mi[i] == -INFINITY && li[i] == 0.f) continue;
      const float f = mi[i] == m ? 1.f : ex2((mi[i] - m) * p.scale_log2);
      l = fmaf(li[i], f, l);
#pragma unroll
      for (int e = 0; e < kJoinElems; ++e) o[e] = fmaf(v[i][e], f, o[e]);
    }
  }
  if (cols == 0) {
    s_m[way][lane] = m;
    s_l[way][lane] = l;
  }
#pragma unroll
  for (int e = 0; e < kJoinElems; ++e) s_o[way][lane][cols + e] = o[e];
  __syncthreads();
  const int r = threadIdx.x / (kCols / 8), x = threadIdx.x % (kCols / 8) * 8;
  if (r >= kJoinRows || row0 + r >= rows || col0 + x >= D) return;
  m = s_m[0][r];
#pragma unroll
  for (int w = 1; w < WAYS; ++w) m = fmaxf(m, s_m[w][r]);
  float y[8] = {};
  l = 0.f;
#pragma unroll
  for (int w = 0; w < WAYS; ++w) {
    const float mw = s_m[w][r];
    if (mw == -INFINITY && s_l[w][r] == 0.f) continue;
    const float f = mw == m ? 1.f : ex2((mw - m) * p.scale_log2);
    l = fmaf(s_l[w][r], f, l);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = fmaf(s_o[w][r][x + e], f, y[e]);
  }
  const float inv = 1.f / l;
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = l == 0.f ? 0.f : y[e] * inv;
  const int tk = (row0 + r) / G, head = tail.head * G + row0 + r - tk * G;
  const long long row = tail.row + tk;
  Vec<T> v;
  pack(y, &v);
  *reinterpret_cast<uint4*>(static_cast<T*>(p.out) + row * p.out_stride + static_cast<long long>(head) * D + col0 + x) = v.raw;
  if (p.lse && col0 + x == 0) p.lse[row * p.hq + head] = l == 0.f ? -INFINITY : fmaf(m, p.scale, logf(l));
}

template <typename T, int WAYS>
cudaError_t launch_join(cudaLaunchConfig_t cfg, const AttendParams& p, const AttendSplit& s, int grid) {
  constexpr int kCols = kJoinThreads / 32 / WAYS * kJoinElems;
  cfg.gridDim = dim3(grid, (s.slot_rows + kJoinRows - 1) / kJoinRows, (p.cache.D + kCols - 1) / kCols);
  cfg.blockDim = dim3(kJoinThreads);
  cfg.dynamicSmemBytes = 0;
  return cudaLaunchKernelEx(&cfg, join_kernel<T, WAYS>, p, s);
}

template <typename T>
cudaError_t launch_tc_type(const CUtensorMap& keys, const CUtensorMap& values, const AttendParams& p, const AttendSplit& s,
                           int grid, cudaStream_t stream) {
  cudaError_t e = ensure_smem_attr(reinterpret_cast<const void*>(&attend_kernel<T>), kSharedBytes, false);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSharedBytes;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, attend_kernel<T>, keys, values, p, s);
  if (e != cudaSuccess) return e;
  return s.slot_rows <= kAttendRows ? launch_join<T, 4>(cfg, p, s, grid) : launch_join<T, 1>(cfg, p, s, grid);
}

}  // namespace

// Test hook state (domino_debug_hold): the CTA of the next launch that withholds its first tile of keys; -1: none.
static std::atomic<int> g_held_cta{-1};
void arm_attend_hold(int cta) { g_held_cta = cta; }

cudaError_t launch_attend_tc(const CUtensorMap& keys, const CUtensorMap& values, const AttendParams& p,
                             const AttendSplit& split, int dtype, int grid, cudaStream_t stream) {
  AttendSplit s = split;
  s.held = g_held_cta.load(std::memory_order_relaxed) < 0 ? -1 : g_held_cta.exchange(-1);
  if (dtype == kBf16) return launch_tc_type<__nv_bfloat16>(keys, values, p, s, grid, stream);
  return launch_tc_type<__half>(keys, values, p, s, grid, stream);
}

}  // namespace dm
