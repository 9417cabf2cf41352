// What the kernels of attention over packed documents share: arguments, the rows of a workgroup, operands.
#pragma once
#include "dit.h"
#include "docs.h"
#include "train.h"

namespace br {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct AttnArgs {
  br_attn_shape s;
  float scale;
  int tiles;  // of a head
  const void *q, *k, *v, *out, *dout;
  float *lse, *ref, *delta;  // ref: lse in powers of two, infinite for a query without keys (its probabilities are zero); delta: dout . out
  void *o, *dq, *dk, *dv;
};

__device__ inline float quarters_max(float x) {
  x = __builtin_elementwise_maximum(x, __shfl_xor(x, 16, 64));
  return __builtin_elementwise_maximum(x, __shfl_xor(x, 32, 64));
}
__device__ inline float quarters_sum(float x) {
  x += __shfl_xor(x, 16, 64);
  return x + __shfl_xor(x, 32, 64);
}

// The rows on the other side of `span`'s document.
__device__ inline DocSpan other_rows(const int* off, int n, int rows, const DocSpan& span) {
  DocSpan o{-1, 0, 0};
  if (span.doc >= 0) o = doc_item(off, n, rows, span.doc + 1);
  return o;
}

// Workgroup -> (head, tile of the head).  Workgroups go round-robin over the 8 XCDs: g = gcd(heads, 8) heads are in work at a time, each on 8 / g XCDs, so
// that the tiles of a document's head find what they share in their XCD's L2.
__host__ __device__ inline int heads_at_a_time(int heads) { return heads % 8 == 0 ? 8 : heads % 4 == 0 ? 4 : heads % 2 == 0 ? 2 : 1; }
__host__ __device__ inline long long head_tile_blocks(int heads, int tiles) {
  const int g = heads_at_a_time(heads), each = (tiles + 8 / g - 1) / (8 / g);
  return (long long)heads / g * each * 8;
}
__device__ inline bool head_tile(int heads, int tiles, int* head, int* tile) {
  const int g = heads_at_a_time(heads), dies = 8 / g, each = (tiles + dies - 1) / dies, x = blockIdx.x & 7, t = blockIdx.x >> 3;
  *head = t / each * g + x % g;
  *tile = (t - t / each * each) * dies + x / g;
  return *tile < tiles;
}

// Tiles of `rows` own rows over all heads: sets a.tiles; workgroups of the launch.
inline br_status attn_grid(AttnArgs& a, int tokens, int heads, int rows, unsigned* blocks) {
  const long long tiles = doc_tiles_most(a.s.n_docs, tokens, rows);
  a.tiles = (int)tiles;
  const long long n = tiles < 0x7FFFFFFFLL ? head_tile_blocks(heads, a.tiles) : 0x7FFFFFFFLL;
  BR_REQUIRE(n < 0x7FFFFFFFLL, BR_ESHAPE, "attention: too many workgroups for one launch");
  *blocks = (unsigned)n;
  return BR_OK;
}

// ---- attn_packed_bf16.hip
bool attn_packed_bf16_fits(const br_attn_shape& s);
br_status launch_attn_forward_bf16(AttnArgs a, hipStream_t st);
br_status launch_attn_grad_bf16(AttnArgs a, hipStream_t st);

}  // namespace br
