// Packed documents: rows off[d] .. off[d + 1] - 1 of a matrix belong to document d.  Device code that finds a document by row or
// by tile from the offsets alone, so that the host needs no copy of them.
#pragma once
#include <hip/hip_runtime.h>

namespace br {

struct DocSpan {
  int doc;         // -1: rows of no document (in front of the first one, behind the last)
  int first, end;  // its rows
};

// Rows of item i of the list [rows in front of document 0, document 0, ..., document n - 1, rows behind it], held within [0, rows].
__device__ inline DocSpan doc_item(const int* __restrict__ off, int n, int rows, int i) {
  DocSpan s;
  s.doc = i >= 1 && i <= n ? i - 1 : -1;
  const int a = i == 0 ? 0 : off[min(i - 1, n)], b = i > n ? rows : off[min(i, n)];
  s.first = min(max(a, 0), rows);
  s.end = min(max(b, s.first), rows);
  return s;
}

// The longest list of tiles of `tile` rows that n documents of `rows` rows give (and what doc_tile_of searches).
__host__ __device__ inline long long doc_tiles_most(int n, long long rows, int tile) { return rows / tile + n + 2; }

// Sums over the lanes up to this one.
__device__ inline int lanes_up_to(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr:1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31
  return x;
}

// How many of 0 .. n - 1 come before the first that pred is false of, by a whole wavefront, 64 places at a time: one round up to 64, two up to 4096.  (pred: true up to some
// place and false from there on; else some number of 0 .. n.)
template <typename PRED>
__device__ inline int leading(int n, PRED pred) {
  const int lane = threadIdx.x & 63;
  int at = 0;
  for (int left = n; left > 0;) {
    const int step = (left + 63) >> 6, last = (lane + 1) * step - 1;  // a lane's places: `step` of those left, the last one is asked for
    const unsigned long long all = __builtin_amdgcn_ballot_w64(last < left && pred(at + min(last, left - 1)));
    const int k = all == ~0ull ? 64 : __builtin_ctzll(~all);
    at += k * step;
    left = k == 64 ? 0 : min(step - 1, left - k * step);
  }
  return at;
}

// A tile of the list of all items' tiles: its item, and its first row (whole wavefronts; uniform).  pick(number of tiles) says which, -1: none.
// Up to DOC_SCAN items their tiles are counted, 64 items at a time, a lane each.  More are not: item i has the places from floor(its first row / tile) + i on, of which one may
// hold no tile, so that a search finds the item and no workgroup's time grows with the documents.  us counted / searched, forward, 16 heads of 64 in bf16: documents of 85 tokens,
// 100 of them 20.2 / 20.3, 300 55 / 46, 1023 311 / 194; of 128 tokens, where every second place is empty, 100 26 / 36, 400 126 / 166, 1023 388 / 416, 2000 1000 / 822; of 16 tokens, 4000 1616 / 311.
constexpr int DOC_SCAN = 1024;
template <typename PICK>
__device__ inline bool doc_tile_of(const int* __restrict__ off, int n, int rows, int tile, PICK pick, DocSpan* span, int* row) {
  const int lane = threadIdx.x & 63, items = n + 2;
  auto tiles_of = [&](const DocSpan& s) { return (s.end - s.first + tile - 1) / tile; };
  if (items > DOC_SCAN) {
    const int t = pick(rows / tile + items);
    if (t < 0) return false;
    auto before = [&](int i) { return (i == 0 ? 0 : min(max(off[i - 1], 0), rows) / tile) + i; };  // places of the items in front of item i
    const int i = max(leading(items, [&](int i) { return before(i) <= t; }) - 1, 0), k = t - before(i);
    *span = doc_item(off, n, rows, i);
    if (k < 0 || k >= tiles_of(*span)) return false;
    *row = span->first + k * tile;
    return true;
  }
  auto item = [&](int i) { return i < items ? doc_item(off, n, rows, i) : DocSpan{-1, 0, 0}; };
  DocSpan s = item(lane);
  int mine = tiles_of(s), sum = lanes_up_to(mine), total;
  if (items <= 64) {
    total = __builtin_amdgcn_readlane(sum, 63);
  } else {
    int all = mine;
#pragma unroll 4
    for (int i = lane + 64; i < items + 63; i += 64) all += tiles_of(item(i));
    total = __builtin_amdgcn_readlane(lanes_up_to(all), 63);
  }
  int t = pick(total);
  if (t < 0) return false;
  for (int base = 0;;) {
    const unsigned long long beyond = __builtin_amdgcn_ballot_w64(sum > t);
    if (beyond) {
      const int at = __builtin_ctzll(beyond);
      span->doc = __builtin_amdgcn_readlane(s.doc, at);
      span->first = __builtin_amdgcn_readlane(s.first, at);
      span->end = __builtin_amdgcn_readlane(s.end, at);
      *row = span->first + (t - __builtin_amdgcn_readlane(sum - mine, at)) * tile;
      return true;
    }
    t -= __builtin_amdgcn_readlane(sum, 63);
    base += 64;
    if (base >= items) return false;
    s = item(base + lane);
    mine = tiles_of(s);
    sum = lanes_up_to(mine);
  }
}
__device__ inline bool doc_tile(const int* __restrict__ off, int n, int rows, int tile, int t, DocSpan* span, int* row) {
  return doc_tile_of(off, n, rows, tile, [&](int total) { return t < total ? t : -1; }, span, row);
}

}  // namespace br
