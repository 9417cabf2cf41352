// What the kernels of attention over packed documents share: arguments, the rows of a workgroup, operands.
#pragma once
#include <algorithm>
#include <cmath>

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
  const void *q, *k, *v, *out, *dout;
  float *lse, *ref, *delta;  // ref: lse in powers of two, infinite for a query without keys (its probabilities are zero); delta: -dout . out
  void *o, *dq, *dk, *dv;
  // Launches of few own rows cut the other side's rows of each document in `parts`, a workgroup each, whose sums (fp32, as they stand) a launch behind joins.
  int parts;
  unsigned blocks;       // workgroups of a part
  int slots;             // workgroups that the units of a compute die take at once, where the last ones may be cut in halves; else 0
  float *part, *part2;   // [parts][tokens][heads][head_dim]: o, dq or dk; dv
  float *part_ref, *part_sum;  // forward: [parts][heads][tokens]
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
// This workgroup's part of them, in whole tiles.
__device__ inline void take_part(DocSpan* rows, int parts, int part, int tile) {
  if (parts == 1) return;
  const long long each = (((long long)rows->end - rows->first + tile - 1) / tile + parts - 1) / parts * tile;
  const int end = rows->end;
  rows->first = (int)min<long long>(rows->first + part * each, end);
  rows->end = (int)min<long long>(rows->first + each, end);
}
template <typename T>
__device__ inline T* part_row(T* base, int part, int tokens, int row, int heads, int head, int dh) { return base + (((size_t)part * tokens + row) * heads + head) * dh; }

// Workgroup -> (head, tile of the head).  Workgroups go round-robin over the 8 XCDs: g = gcd(heads, 8) heads are in work at a time, each on 8 / g XCDs, so
// that the tiles of a document's head find what they share in their XCD's L2.
//
// Halves (a.slots > 0): where at most half of a die's slots are left for its last tiles, these are cut in two (16 own rows a wave instead of 32), which take 0.6
// of a tile's time.
__host__ __device__ inline int heads_at_a_time(int heads) { return heads % 8 == 0 ? 8 : heads % 4 == 0 ? 4 : heads % 2 == 0 ? 2 : 1; }
__host__ __device__ inline long long head_tile_blocks(int heads, long long tiles, int slots) {
  const int g = heads_at_a_time(heads);
  return (heads / g * ((tiles + 8 / g - 1) / (8 / g)) + slots / 2) * 8;
}
struct OwnRows {
  DocSpan span;
  int row, head, part;
  bool half;
};
__device__ inline bool own_place(const AttnArgs& a, const int* off, int tokens, int heads, int rows, OwnRows* o) {
  o->part = a.parts == 1 ? 0 : blockIdx.x / a.blocks;
  const unsigned block = blockIdx.x - o->part * a.blocks;  // (a part's workgroups are a multiple of 8)
  const int x = block & 7;
  int second = 0;
  o->half = false;
  const bool found = doc_tile_of(off, a.s.n_docs, tokens, rows, [&](int total) {
    const int g = heads_at_a_time(heads), dies = 8 / g, each = (total + dies - 1) / dies, n = heads / g * each;
    int t = block >> 3;
    if (a.slots > 0) {
      const int whole = n / a.slots * a.slots;
      if (t >= whole && (n - whole) * 2 <= a.slots) {
        second = (t - whole) & 1;
        t = whole + (t - whole) / 2;
        o->half = true;
      }
    }
    if (t >= n) return -1;
    const int k = t / each, tile = (t - k * each) * dies + x / g;
    o->head = k * g + x % g;
    return tile < total ? tile : -1;
  }, &o->span, &o->row);
  if (!found) return false;
  o->row += second * (rows / 2);
  return o->row < o->span.end;
}

// Tiles of `rows` own rows over all heads, in `parts`, `per_cu` workgroups a unit that may be halved (0: not): sets the fields of a; workgroups of the launch.
inline br_status attn_grid(AttnArgs& a, int tokens, int heads, int rows, int parts, int per_cu, unsigned* blocks) {
  const long long tiles = doc_tiles_most(a.s.n_docs, tokens, rows);
  a.parts = parts;
  // Halves, by the tiles that documents of average length give: where the last round is at most half full, and the first or the second; up to the fourth where a
  // workgroup has a unit for itself (where two or three share one, those that are left run faster by themselves).  The code of both sizes costs launches that need
  // one 1 to 2 %.  us without / with: backward, heads of 128, two documents of 4350, 12 heads 766 / 748, six of 1050, 16 heads 251 / 244, two of 525, 8 heads 44 / 32;
  // of 64, the same 27.6 / 21.5, one of 325, 4 heads 21 / 17; forward, three of 2025, 12 heads of 128 97.4 / 93.5, six of 1050, 16 of 64 48.8 / 45; not: eight of
  // 2025, 8 heads of 128, 2.04 rounds 142 / 147.
  const int slots = per_cu * device_cu_count() / 8;
  const double rounds = (double)heads * ((double)tokens / rows + 0.5 * std::min(a.s.n_docs, tokens)) / 8.0 / std::max(slots, 1);
  a.slots = parts == 1 && rounds < (per_cu == 1 ? 4.0 : 1.2) && rounds - floor(rounds) <= 0.55 ? slots : 0;
  const long long n = tiles < 0x7FFFFFFFLL ? head_tile_blocks(heads, tiles, a.slots) : 0x7FFFFFFFLL;
  BR_REQUIRE(n * parts < 0x7FFFFFFFLL, BR_ESHAPE, "attention: too many workgroups for one launch");
  a.blocks = (unsigned)n;
  *blocks = (unsigned)(n * parts);
  return BR_OK;
}

// Parts of a launch whose own rows make fewer workgroups than the units take at once (`per_cu` each).  They save the time of the steps that others take (step_us for 32
// rows of an average document, `heads` times over for keys that several heads of queries share) and cost the join: 4 us, and `outputs` fp32 values of every
// own row's channel written and read by each part (3 TB/s together).  us in one part / as many as this rule gives: bf16 backward, 8 heads on two, two documents of 750,
// heads of 64 73 / 38, of 128 116 / 56; 4 heads, one of 1060, 41 / 30 and 64 / 45; four of 1024 queries on 77 keys, heads of 128 47 / 32; fp32 forward, 20 queries on
// 1800 keys, heads of 128 24 / 15.
inline int attn_parts(const br_attn_shape& s, long long own_tokens, int own_heads, int own_rows, long long other_tokens, int heads, int per_cu, float step_us, int outputs) {
  if (own_tokens == 0 || other_tokens == 0 || s.n_docs == 0) return 1;
  const int tiles = cdiv(cdiv(other_tokens, s.n_docs), 32);
  if ((float)heads * tiles * step_us <= 7.f) return 1;  // (no number of parts can save 3 us)
  const long long blocks = std::max<long long>(cdiv(own_tokens, own_rows), std::min<long long>(s.n_docs, own_tokens)) * own_heads;
  const int most = (int)std::min<long long>({(long long)per_cu * device_cu_count() / blocks, (long long)heads * tiles / 4, tiles, 64});
  int best = 1;
  float gain = 3.f;
  for (int n = 2; n <= most; ++n) {
    const float g = (float)heads * tiles * step_us * (1.f - 1.f / n) - 4.f - (float)n * own_tokens * own_heads * s.head_dim * outputs * 8.f / 3e6f;
    if (g > gain) {
      gain = g;
      best = n;
    }
  }
  return best;
}

// ---- attn_packed_bf16.hip
bool attn_packed_bf16_fits(const br_attn_shape& s);
br_status launch_attn_forward_bf16(AttnArgs a, int parts, hipStream_t st);
br_status launch_attn_grad_bf16(AttnArgs a, int parts_q, int parts_k, hipStream_t st);
// ---- attn_train.hip: what the parts leave, into the outputs
br_status launch_attn_join_forward(const AttnArgs& a, hipStream_t st);
br_status launch_attn_join_dq(const AttnArgs& a, hipStream_t st);
br_status launch_attn_join_dkv(const AttnArgs& a, hipStream_t st);
// own rows of a workgroup and workgroups a unit of the bf16 kernels: forward, dq, dk and dv
constexpr int PACK_OWN = 128;
inline int pack_per_cu(int head_dim, int pass) { return head_dim == 128 ? (pass == 2 ? 1 : 2) : pass == 2 ? 2 : pass == 1 ? 3 : 4; }

}  // namespace br
