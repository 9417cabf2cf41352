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

// The longest list of tiles of `tile` rows that n documents of `rows` rows give.
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

// A tile of the list of all items' tiles: its item, and its first row (whole wavefronts; uniform).  pick(number of tiles) says which, -1: none.  64 items at a
// time, a lane each; more than 64 are counted first.
template <typename PICK>
__device__ inline bool doc_tile_of(const int* __restrict__ off, int n, int rows, int tile, PICK pick, DocSpan* span, int* row) {
  const int lane = threadIdx.x & 63, items = n + 2;
  auto tiles_of = [&](const DocSpan& s) { return (s.end - s.first + tile - 1) / tile; };
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
