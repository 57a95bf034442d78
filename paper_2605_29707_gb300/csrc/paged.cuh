// paged.cuh -- places of a paged cache and the sequences of a batch, as the device reads them.
#pragma once

#include "kernels.h"

namespace dm {

// The places that the table holds, cut off a tile below 2^31.
__device__ __forceinline__ int table_places(const PagedCache& c, const PagedBatch& b) {
  const long long n = static_cast<long long>(b.table_width) * c.page;
  return n > 0x7fffff80LL ? 0x7fffff80 : static_cast<int>(n);
}

constexpr int kNoLength = 1 << 30;

struct Sequence {
  int row;    // its first new token's row
  int n;      // new tokens
  int kv;     // keys, the new ones among them
  int first;  // its first new token's place: kv - n, or more where the last ones lie past the table
};

// What the batch says of sequence b, cut off at the tensors' ends.  Keys end with the table, and new tokens keep their
// places even so; only what is no length, 2^30 and more past a table that holds fewer, is taken for the table's end.
__device__ __forceinline__ Sequence load_sequence(const PagedCache& c, const PagedBatch& b, int tokens, int seq) {
  const int s0 = b.start[seq], s1 = b.start[seq + 1], kv = b.kv_len[seq];
  Sequence s;
  s.row = min(max(s0, 0), tokens);
  s.n = min(max(s1, s.row), tokens) - s.row;
  const int places = table_places(c, b), first = max(kv, 0) - s.n;
  s.kv = min(max(kv, 0), places);
  s.first = first <= places || kv < kNoLength ? first : s.kv - s.n;
  return s;
}

// The sequence that row `token` belongs to, or -1.
__device__ __forceinline__ int find_sequence(const PagedBatch& b, int token) {
  int lo = 0, hi = b.B;  // start[lo] <= token < start[hi]
  if (token < b.start[0] || token >= b.start[hi]) return -1;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (b.start[mid] <= token) lo = mid; else hi = mid;
  }
  return lo;
}

// Element offset of (place, head 0), or -1 where the place has no page.
__device__ __forceinline__ long long place_offset(const PagedCache& c, const PagedBatch& b, int seq, int place) {
  if (place < 0 || place >= table_places(c, b)) return -1;
  const int i = place / c.page, pg = b.table[seq * b.table_stride + i];
  if (pg < 0 || pg >= c.pages) return -1;
  return pg * c.page_stride + (place - i * c.page) * c.token_stride;
}

// The token that token a > 0 of a sequence follows in its tree (parents given by node: token a is node a - 1).
__device__ __forceinline__ int tree_up(const int32_t* parent, int a) {
  const int up = parent[a - 1];
  return up < -1 || up >= a - 1 ? 0 : up + 1;  // a parent is an earlier node, or the anchor
}

// Whether token i of a sequence (keys of new tokens from `first` on) sees the key at `place`, below its kv.
__device__ __forceinline__ bool sees(int mask, const int32_t* parent, int N, int i, long long first, int place) {
  if (mask == kMaskFull) return true;
  const long long t = place - first;  // the key's new token, or negative
  if (mask == kMaskCausal) return t <= i;
  if (i > N) return false;
  if (t < 0) return true;
  int a = i;
  while (a > t && a > 0) a = tree_up(parent, a);
  return a == t;
}

}  // namespace dm
