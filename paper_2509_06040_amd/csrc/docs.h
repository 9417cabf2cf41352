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

// Tile t of the list of all items' tiles: its item, and its first row (whole wavefronts; uniform).  64 items at a time, a lane each.  False: there are fewer.
__device__ inline bool doc_tile(const int* __restrict__ off, int n, int rows, int tile, int t, DocSpan* span, int* row) {
  const int lane = threadIdx.x & 63;
  for (int base = 0; base < n + 2; base += 64) {
    const int i = base + lane;
    DocSpan s{-1, 0, 0};
    if (i < n + 2) s = doc_item(off, n, rows, i);
    const int mine = (s.end - s.first + tile - 1) / tile;
    int sum = mine;  // of the lanes up to this one
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(sum, d, 64);
      if (lane >= d) sum += o;
    }
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
  }
  return false;
}

}  // namespace br
