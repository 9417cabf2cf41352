// bf16 attention over packed documents: the forward pass, dq (own rows: queries, tiles of keys), and dk with dv (own rows: keys, tiles of queries).
//
// A wavefront keeps 32 rows of its side in registers (column operands of the score products) and their sums in accumulators, and walks tiles of 32
// rows of the other side in LDS.  Tile j of the backward pass: scores S = Y1 X1 and X = Y2 X2 (X1, X2: own q and dout, or own k and v), probabilities P = exp2(S - ref), dS = P
// (X - delta), and the products with the tile's rows, dk += Y1^T dS (dq the same) and dv += Y2^T P.  These wait for the next tile: between its scores' last
// matrix instructions and theirs stand the exponentials of the tile itself.
//
// Both kernels of the backward pass take scores anew from q, k and the log-sum-exp: seven products where the formulas have five, nothing of a tile's size in memory and every sum in one
// wavefront's registers in a fixed order (dq added up over the workgroups of the keys instead would be 85 MB of fp32 for a head of a document of 4600 tokens).
//
// Bound by the matrix pipe, the exponentials issued beside it, and the clock that the chip's power leaves (2.0 to 2.3 GHz with random inputs; with inputs of zero
// 20 to 30 % faster).  Measured: forward, 16 heads of 64, 16 documents of 1025 to 1101 tokens 96 us, 768 TFLOP/s (matrix pipe 32 % busy, VALU 54 %); backward of eight of them 155
// us, 600 TFLOP/s by the formulas' five products, 840 by the seven; backward, 12 heads of 128, two documents of 4096 to 4608 716 to 737 us by machine, 735 to 755 and 1030 to 1060 (matrix pipe 52 % busy for
// dq, 40 % for dk and dv, VALU 36 and 31 %); eight documents of 2001, 16 heads, forward 834 at heads of 64 and 1003 at 128, backward 1080 and
// 1096 by the seven.  A library product of 8192^3 reaches 1570 on the same card, both operands along the contraction (1340 with the second as it lies, 1520 over large shapes).
//
// Rounded to bf16: P and dS, which the matrix instruction takes as bf16 operands, and the results; scores, sums, references and delta stay fp32.
//
// Tiles come straight from global memory into LDS, rows as they lie, 16-byte chunks permuted per row so that both the fragments of 16 rows
// and the transposed reads (eight rows, two chunks) spread over the banks.
#include "attn_packed.h"
#include "static_for.h"

namespace br {

#define BR_LPTR(p) ((void __attribute__((address_space(3)))*)(p))

extern __shared__ __attribute__((aligned(1024))) char g_packed_tiles[];

constexpr int PACK_TILE = 32;  // rows of a tile

// Waves a SIMD, buffers, and tiles between two barriers.
enum class Pass { FORWARD, QUERIES, KEYS };
template <int DH, Pass PASS>
struct PackForm {
  static constexpr int WPE = DH == 128 ? (PASS == Pass::KEYS ? 1 : 2) : PASS == Pass::KEYS ? 2 : PASS == Pass::FORWARD ? 4 : 3;  // (pack_per_cu)
  static constexpr int NB = DH == 128 ? (PASS == Pass::KEYS ? 6 : 4) : PASS == Pass::FORWARD ? 4 : 6, EACH = NB >= 6 ? 2 : 1;
  static constexpr int LDS = NB * (2 * PACK_TILE * DH * 2 + (PASS == Pass::KEYS ? 2 * PACK_TILE * 4 : 0));
};

static __device__ inline u32x4 buffer_rows(const void* p, unsigned bytes) {
  const unsigned long long v = reinterpret_cast<unsigned long long>(p);
  return u32x4{(unsigned)__builtin_amdgcn_readfirstlane((unsigned)v), (unsigned)__builtin_amdgcn_readfirstlane((unsigned)(v >> 32)) & 0xffffu,
               (unsigned)__builtin_amdgcn_readfirstlane(bytes), 0x00020000u};
}

// Slot permutation of a tile's rows: 16-byte chunk c of row r sits in slot c ^ tile_swz(r).  Transposed 8-byte reads are served 32 lanes at a time (eight rows
// and two chunks: the rows, or with 128-byte rows the row pairs, take different pairs of slots).  16-byte reads are served in groups of lanes
// {0-3, 12-15, 20-27} and {4-11, 16-19, 28-31} (and 32 further): with even permutations the quarters' neighbouring chunks fill the odd slots.  (Permutations that are
// free of conflicts for 16 consecutive lanes instead: a third of the LDS's cycles were conflicts.)
template <int DH>
__device__ inline int tile_swz(int r) { return DH == 128 ? (r & 7) << 1 : (r >> 1 & 3) << 1; }

// Two matrices' rows on their way into LDS in tiles of PACK_TILE rows, those of the second behind those of the first: 1 KB an instruction, lane i fills bytes
// 16 i .. 16 i + 15, so the permutation is applied on the global side; rows past the document's end lie past the buffer's and arrive as zeros.
template <int DH>
struct TilePair {
  static constexpr int CH = DH / 8, RPI = 64 / CH, LPW = PACK_TILE / RPI / 4, ROW_B = DH * 2, TILE_B = PACK_TILE * ROW_B, BUF_B = 2 * TILE_B;
  static_assert(LPW >= 1, "");
  u32x4 rows1, rows2;
  unsigned lb1, lb2, off1[LPW], off2[LPW], lds_w;
  int n_rows;
  // `heads` heads of DH values side by side, from y1 and y2 on
  __device__ __forceinline__ void open(const bf16* y1, long long ld1, const bf16* y2, long long ld2, int n, int heads, const char* lds, int wv) {
    n_rows = n;
    lb1 = (unsigned)(ld1 * 2);
    lb2 = (unsigned)(ld2 * 2);
    rows1 = buffer_rows(y1, (unsigned)(n - 1) * lb1 + heads * ROW_B);
    rows2 = buffer_rows(y2, (unsigned)(n - 1) * lb2 + heads * ROW_B);
    lds_w = (unsigned)(uintptr_t)BR_LPTR(const_cast<char*>(lds)) + wv * LPW * 1024;
    rewind(0, wv);
  }
  __device__ __forceinline__ void rewind(int head, int wv) {  // to the first tile of a head
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int t = 0; t < LPW; ++t) {
      const int r = (wv * LPW + t) * RPI + lane / CH;
      const unsigned c = head * ROW_B + ((lane % CH ^ tile_swz<DH>(r)) << 4);
      off1[t] = r < n_rows ? r * lb1 + c : 0xFFFFFFFFu;
      off2[t] = r < n_rows ? r * lb2 + c : 0xFFFFFFFFu;
    }
  }
  __device__ __forceinline__ void next(int buf) {  // this wave's share of the next tile, into the buffer `buf` bytes on
#pragma unroll
    for (int t = 0; t < LPW; ++t) {
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds_w + buf + t * 1024), "v"(off1[t]), "s"(rows1) : "memory", "m0");
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds_w + buf + TILE_B + t * 1024), "v"(off2[t]), "s"(rows2) : "memory", "m0");
      off1[t] = __builtin_elementwise_add_sat(off1[t], PACK_TILE * lb1);
      off2[t] = __builtin_elementwise_add_sat(off2[t], PACK_TILE * lb2);
    }
  }
};

// This lane's fragments of a tile: 16 rows from 16 blk on (row operand, channels of step ks), or 16 channels (row operand transposed, all 32 rows: slot (quarter g, e) of
// the contraction is row 16 (e / 4) + 4 g + e % 4).
template <int DH>
struct TileFrags {
  static constexpr int KS = DH / 32, DB = DH / 16, ROW_B = DH * 2;
  typedef const char __attribute__((address_space(3)))* lptr;
  lptr l0;
  unsigned raddr[KS], caddr[DB];
  __device__ __forceinline__ void open(const char* lds) {
    const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4, crow = 4 * g + (l16 >> 2);
    l0 = (lptr)BR_LPTR(const_cast<char*>(lds));
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) raddr[ks] = l16 * ROW_B + (((ks * 4 + g) ^ tile_swz<DH>(l16)) << 4);
#pragma unroll
    for (int d = 0; d < DB; ++d) caddr[d] = crow * ROW_B + (((2 * d + ((l16 & 3) >> 1)) ^ tile_swz<DH>(crow)) << 4) + 8 * (l16 & 1);
  }
  __device__ __forceinline__ bf16x8 rows(int blk, int ks, int at) const { return *(const bf16x8 __attribute__((address_space(3)))*)(l0 + raddr[ks] + (at + blk * 16 * ROW_B)); }
  __device__ __forceinline__ bf16x8 cols(int d, int at) const {
    const lptr p = l0 + caddr[d] + at;
    union { s16x4 s[2]; bf16x8 v; } u;
    u.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)p);
    u.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(p + 16 * ROW_B));
    return u.v;
  }
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ unsigned two_bf16(float lo, float hi) { return __builtin_bit_cast(unsigned, __builtin_convertvector(f32x2{lo, hi}, bf16x2)); }

__device__ __forceinline__ f32x4 mma(bf16x8 x, bf16x8 y, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0); }

// Behind every EACH-th step j: the tiles asked for at the last turn have landed, every wave is done with those before tile j, whose buffers take the tiles
// from j + NB - EACH on.
__device__ __forceinline__ void tile_turn() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// What tile -1 is read as in the first step: finite, with operands of zero beside it.
template <int DH, int NB>
static __device__ __forceinline__ void clear_last_buffer(char* lds) {
  constexpr int BUF_B = TilePair<DH>::BUF_B;
  for (int at = threadIdx.x * 16; at < BUF_B; at += 256 * 16) *reinterpret_cast<u32x4*>(lds + (NB - 1) * BUF_B + at) = u32x4{0, 0, 0, 0};
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

constexpr float REF_LIMIT = 2048.f;  // a query's reference moves when eight of its probabilities add up to more

// Output and log-sum-exp of 128 queries.  Which reference is subtracted from the scores of a query does not matter, as long as it is the same for all it
// sums: it is the maximum of some tile, and moves only when a lane's eight probabilities of a tile add up to more than REF_LIMIT, so that no maximum is taken
// on the way.
template <int DH, int QB>
static __device__ __forceinline__ void packed_forward_rows(const AttnArgs& a, const OwnRows& place) {
  using F = PackForm<DH, Pass::FORWARD>;
  using TP = TilePair<DH>;
  constexpr int NB = F::NB, EACH = F::EACH;
  constexpr int KS = DH / 32, DB = DH / 16, BUF_B = TP::BUF_B, TILE_B = TP::TILE_B;
  constexpr int NA = 2 * KS, NC = DB, NS = NA + NC, FR = 4, RA = FR - 1;
  static_assert(NS % FR == 0 && NB % 2 == 0 && NB % EACH == 0 && NB >= 2 + 2 * EACH, "");
  char* lds = g_packed_tiles;
  const int head = place.head, part_of = place.part;
  const DocSpan own = place.span;
  DocSpan keys = other_rows(a.s.k_off, a.s.n_docs, a.s.k_tokens, own);
  take_part(&keys, a.parts, part_of, PACK_TILE);
  const int kv = head / (a.s.n_heads / a.s.n_kv_heads), lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row0 = place.row + wv * (16 * QB);
  const bool active = row0 < own.end;  // (uniform over the wave)
  const int n_keys = keys.end - keys.first, N = (n_keys + PACK_TILE - 1) / PACK_TILE;

  bf16x8 q[QB][KS];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
      q[qb][ks] = *reinterpret_cast<const bf16x8*>((const bf16*)a.q + (size_t)min(row0 + qb * 16 + l16, own.end - 1) * a.s.q_stride + (size_t)head * DH + ks * 32 + g * 8);
  f32x4 o[DB][QB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) o[d][qb] = f32x4{0.f, 0.f, 0.f, 0.f};
  float ref[QB], sum[QB];  // reference, in powers of two; sum of this lane's probabilities
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    ref[qb] = -3.4028235e38f;  // (the first score above -inf moves it)
    sum[qb] = 0.f;
  }
  if (N > 0) {
    TP tiles;
    tiles.open((const bf16*)a.k + (size_t)kv * DH + (size_t)keys.first * a.s.k_stride, a.s.k_stride, (const bf16*)a.v + (size_t)kv * DH + (size_t)keys.first * a.s.v_stride, a.s.v_stride,
               n_keys, 1, lds, wv);
    int asked = 0;
    auto issue = [&](int b) __attribute__((always_inline)) {
      if (asked < N) tiles.next(b * BUF_B);
      ++asked;
    };
#pragma unroll
    for (int b = 0; b + 1 < NB; ++b) issue(b);
    clear_last_buffer<DH, NB>(lds);
    tile_turn();
    if (!active) {  // a wave without rows only keeps up its share of the tile traffic
      for (int j = EACH - 1, b = NB - 1; j + 1 < N; j += EACH) {
        tile_turn();
#pragma unroll
        for (int i = 0; i < EACH; ++i, b = b + 1 == NB ? 0 : b + 1) issue(b);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      return;
    }
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(q[qb][ks]));
    TileFrags<DH> frags;
    frags.open(lds);
    auto frag_of = [&](auto Nc, int ao, int co) __attribute__((always_inline)) {  // n < NA: scores (block of 16 keys, step of the channels), else values
      constexpr int n = decltype(Nc)::value;
      if constexpr (n < NA) return frags.rows(n / KS, n % KS, ao);
      else return frags.cols(n - NA, co + TILE_B);
    };
    const float unit = a.scale * LOG2E;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    f32x4 s[2][QB];      // [block of 16 keys][block of queries]
    bf16x8 pf[2][QB];    // [parity of the tile][block of queries]
    float part[QB];      // sum of this lane's probabilities of the tile
    bf16x8 fr[FR];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int e = 0; e < 8; ++e) pf[1][qb][e] = (bf16)0.f;  // (tile -1)
    auto use = [&](auto Nc, auto Pc, auto QBc, const bf16x8& f) __attribute__((always_inline)) {  // Pc: parity of the values' tile
      constexpr int n = decltype(Nc)::value, P = decltype(Pc)::value, qb = decltype(QBc)::value;
      if constexpr (n < NA) s[n / KS][qb] = mma(f, q[qb][n % KS], n % KS == 0 ? zero : s[n / KS][qb]);
      else o[n - NA][qb] = mma(f, pf[P][qb], o[n - NA][qb]);
    };
    auto prob = [&](auto Pc, int e) __attribute__((always_inline)) {  // element e: block of keys, block of queries, key
      constexpr int P = decltype(Pc)::value;
      const int b = e / (4 * QB), qb = (e >> 2) % QB, r = e & 3;
      const float p = __builtin_amdgcn_exp2f(fmaf(s[b][qb][r], unit, -ref[qb]));
      part[qb] = b == 0 && r == 0 ? p : part[qb] + p;
      pf[P][qb][b * 4 + r] = (bf16)p;
    };
    auto step = [&](auto Pc, auto Bc, int j, auto LASTc) __attribute__((always_inline)) {  // LASTc: may be the last one
      constexpr int P = decltype(Pc)::value, B = decltype(Bc)::value, BP = (B + NB - 1) % NB, BN = (B + 1) % NB;
      constexpr int NE = 8 * QB;
      constexpr bool LAST = decltype(LASTc)::value;
      const bool tail = LAST && j == N - 1 && n_keys % PACK_TILE != 0;
      static_for<NS>([&](auto Nc) __attribute__((always_inline)) {
        constexpr int n = decltype(Nc)::value;
        if constexpr (n + RA < NS) fr[(n + RA) % FR] = frag_of(std::integral_constant<int, n + RA>{}, B * BUF_B, BP * BUF_B);
        else fr[(n + RA) % FR] = frag_of(std::integral_constant<int, n + RA - NS>{}, BN * BUF_B, B * BUF_B);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (LAST && n == NA) {
          if (tail) {  // keys past the end
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
              for (int qb = 0; qb < QB; ++qb)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                  if (j * PACK_TILE + b * 16 + 4 * g + r >= n_keys) s[b][qb][r] = -INFINITY;
          }
        }
        static_for<QB>([&](auto Qc) __attribute__((always_inline)) {
          use(Nc, std::integral_constant<int, P ^ 1>{}, Qc, fr[n % FR]);
          __builtin_amdgcn_sched_barrier(0);
          if constexpr (decltype(Qc)::value == 0 && n >= NA) {
#pragma unroll
            for (int e = NE * (n - NA) / NC; e < NE * (n - NA + 1) / NC; ++e) prob(Pc, e);
            __builtin_amdgcn_sched_barrier(0);
          }
        });
      });
      // (each query moves for itself: its result does not depend on which queries share its wave; a score that is not a number makes its own sum one)
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(part[0] <= REF_LIMIT && part[QB - 1] <= REF_LIMIT)) != 0, 0)) {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          const bool over = quarters_max(part[qb] <= REF_LIMIT ? 0.f : 1.f) != 0.f;
          const f32x4 m = __builtin_elementwise_maximum(s[0][qb], s[1][qb]);
          const float most = quarters_max(__builtin_elementwise_maximum(__builtin_elementwise_maximum(m[0], m[1]), __builtin_elementwise_maximum(m[2], m[3])));
          const float next = over ? __builtin_elementwise_maximum(ref[qb], most * unit) : ref[qb], shrink = __builtin_amdgcn_exp2f(ref[qb] - next);
          ref[qb] = next;
          sum[qb] *= shrink;
#pragma unroll
          for (int d = 0; d < DB; ++d) o[d][qb] *= shrink;
        }
#pragma unroll
        for (int e = 0; e < NE; ++e) prob(Pc, e);
      }
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) sum[qb] += part[qb];
    };
    auto behind = [&](auto Bc) __attribute__((always_inline)) {  // the step in buffer B
      constexpr int B = decltype(Bc)::value;
      if constexpr (B % EACH == EACH - 1) {
        tile_turn();
#pragma unroll
        for (int i = EACH; i > 0; --i) issue((B + NB - i) % NB);
      }
    };
    static_for<RA>([&](auto Nc) __attribute__((always_inline)) { fr[decltype(Nc)::value] = frag_of(Nc, 0, 0); });
    int j = 0;
    for (; j + NB < N; j += NB)  // (whole rounds of the buffers with more behind them: no questions in between; 2 %.  The backward pass loses 1 to 4 % to that much code)
      static_for<NB>([&](auto Bc) __attribute__((always_inline)) {
        constexpr int B = decltype(Bc)::value;
        step(std::integral_constant<int, B & 1>{}, Bc, 0, std::false_type{});
        behind(Bc);
      });
    bool more = true;
    while (more) {
      static_for<NB>([&](auto Bc) __attribute__((always_inline)) {
        if (!more) return;
        constexpr int B = decltype(Bc)::value, P = B & 1;
        step(std::integral_constant<int, P>{}, Bc, j, std::true_type{});
        more = ++j < N;
        if (more) behind(Bc);
      });
    }
    auto last = [&](auto Pc, int at) __attribute__((always_inline)) {  // values of the last tile, `at` bytes on
      static_for<NC>([&](auto Ic) __attribute__((always_inline)) {
        using Nc = std::integral_constant<int, NA + decltype(Ic)::value>;
        const bf16x8 f = frag_of(Nc{}, 0, at);
        static_for<QB>([&](auto Qc) __attribute__((always_inline)) { use(Nc{}, Pc, Qc, f); });
      });
    };
    const int at = (N - 1) % NB * BUF_B;
    if (N & 1) last(std::integral_constant<int, 0>{}, at);
    else last(std::integral_constant<int, 1>{}, at);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }
  if (!active) return;
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const float total = quarters_sum(sum[qb]), inv = total == 0.f ? 0.f : 1.f / total;
    const int row = row0 + qb * 16 + l16;
    if (row >= own.end) continue;
    if (a.parts > 1) {
      float* to = part_row(a.part, part_of, a.s.q_tokens, row, a.s.n_heads, head, DH) + 4 * g;
#pragma unroll
      for (int d = 0; d < DB; ++d) *reinterpret_cast<f32x4*>(to + 16 * d) = o[d][qb];
      if (g == 0) {
        const size_t at = ((size_t)part_of * a.s.n_heads + head) * a.s.q_tokens + row;
        a.part_ref[at] = ref[qb];
        a.part_sum[at] = total;
      }
      continue;
    }
    bf16* out = (bf16*)a.o + (size_t)row * a.s.o_stride + (size_t)head * DH + 4 * g;
#pragma unroll
    for (int d = 0; d < DB; ++d) store4(out + 16 * d, o[d][qb][0] * inv, o[d][qb][1] * inv, o[d][qb][2] * inv, o[d][qb][3] * inv);
    if (g == 0) a.lse[(size_t)head * a.s.q_tokens + row] = total == 0.f ? -INFINITY : (ref[qb] + __builtin_amdgcn_logf(total)) * LN2;
  }
}

template <int DH, bool HALVES>
__global__ __launch_bounds__(256, (PackForm<DH, Pass::FORWARD>::WPE)) void packed_forward_bf16_kernel(AttnArgs a) {
  OwnRows place;
  if (!own_place(a, a.s.q_off, a.s.q_tokens, a.s.n_heads, PACK_OWN, &place)) return;
  if constexpr (HALVES) {
    if (place.half) return packed_forward_rows<DH, 1>(a, place);
  }
  packed_forward_rows<DH, 2>(a, place);
}

// (dk and dv of head dim 128: 128 accumulators and 64 operands a lane, one wave a SIMD)
template <int DH, Pass PASS, int QB>
static __device__ __forceinline__ void packed_grad_rows(const AttnArgs& a, const OwnRows& place) {
  using F = PackForm<DH, PASS>;
  using TP = TilePair<DH>;
  constexpr bool KEYS = PASS == Pass::KEYS;
  constexpr int NB = F::NB, EACH = F::EACH;
  constexpr int KS = DH / 32, DB = DH / 16, BUF_B = TP::BUF_B, TILE_B = TP::TILE_B;
  constexpr int NA = 4 * KS, NC = KEYS ? 2 * DB : DB, NS = NA + NC, FR = DH == 128 && KEYS ? 8 : 4, RA = FR - 1;
  constexpr int REFS = NB * BUF_B, REF_B = 2 * PACK_TILE * 4;  // ref and delta of a tile's rows, behind the tiles
  static_assert(NS % FR == 0 && NB % 2 == 0 && NB % EACH == 0 && NB >= 2 + 2 * EACH, "");
  char* lds = g_packed_tiles;
  const int share = a.s.n_heads / a.s.n_kv_heads, head = place.head, part_of = place.part;
  const DocSpan own = place.span;
  DocSpan other = other_rows(KEYS ? a.s.q_off : a.s.k_off, a.s.n_docs, KEYS ? a.s.q_tokens : a.s.k_tokens, own);
  // Documents of one tile of keys take delta from the probabilities (sum of p X): that from the output carries the output's rounding to bf16, which few keys
  // do not average out (2 to 4 keys: dq and dk 0.0031 off the formula instead of 0.0023; from 30 on no difference).
  const bool brief = !KEYS && other.end - other.first <= PACK_TILE;
  take_part(&other, a.parts, part_of, PACK_TILE);
  const int kv = KEYS ? head : head / share, h0 = KEYS ? head * share : head;
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row0 = place.row + wv * (16 * QB);
  const bool active = row0 < own.end;  // (uniform over the wave)

  // ---- own rows
  const bf16* x1 = KEYS ? (const bf16*)a.k + (size_t)kv * DH : (const bf16*)a.q + (size_t)head * DH;
  const bf16* x2 = KEYS ? (const bf16*)a.v + (size_t)kv * DH : (const bf16*)a.dout + (size_t)head * DH;
  const size_t ld1 = KEYS ? a.s.k_stride : a.s.q_stride, ld2 = KEYS ? a.s.v_stride : a.s.o_stride;
  bf16x8 f1[QB][KS], f2[QB][KS];
  float ref[QB] = {}, delta[QB] = {};
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const int row = min(row0 + qb * 16 + l16, own.end - 1);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      f1[qb][ks] = *reinterpret_cast<const bf16x8*>(x1 + (size_t)row * ld1 + ks * 32 + g * 8);
      f2[qb][ks] = *reinterpret_cast<const bf16x8*>(x2 + (size_t)row * ld2 + ks * 32 + g * 8);
    }
    if constexpr (!KEYS) {  // delta and ref of the own queries, for the kernel of dk and dv too
      float d = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8 o = *reinterpret_cast<const bf16x8*>((const bf16*)a.out + (size_t)row * a.s.o_stride + (size_t)head * DH + ks * 32 + g * 8);
#pragma unroll
        for (int e = 0; e < 8; ++e) d = fmaf((float)o[e], (float)f2[qb][ks][e], d);
      }
      const size_t at = (size_t)head * a.s.q_tokens + row;
      const float lse = a.lse[at];
      delta[qb] = brief ? 0.f : quarters_sum(d);
      ref[qb] = lse == -INFINITY ? INFINITY : lse * LOG2E;
      if (g == 0 && row0 + qb * 16 + l16 < own.end && part_of == 0) {
        a.ref[at] = ref[qb];
        if (!brief) a.delta[at] = -delta[qb];
      }
    }
  }
  f32x4 acc1[DB][QB], acc2[KEYS ? DB : 1][QB];  // dq or dk; dv
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      acc1[d][qb] = f32x4{0.f, 0.f, 0.f, 0.f};
      if constexpr (KEYS) acc2[d][qb] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

  const int n_rows = other.end - other.first, nt = (n_rows + PACK_TILE - 1) / PACK_TILE, N = KEYS ? nt * share : nt;
  if (N > 0) {
    const long long ld_y1 = KEYS ? a.s.q_stride : a.s.k_stride, ld_y2 = KEYS ? a.s.o_stride : a.s.v_stride;
    TP tiles;
    tiles.open((KEYS ? (const bf16*)a.q + (size_t)h0 * DH : (const bf16*)a.k + (size_t)kv * DH) + (size_t)other.first * ld_y1, ld_y1,
               (KEYS ? (const bf16*)a.dout + (size_t)h0 * DH : (const bf16*)a.v + (size_t)kv * DH) + (size_t)other.first * ld_y2, ld_y2, n_rows, KEYS ? share : 1, lds, wv);
    const unsigned lds0 = (unsigned)(uintptr_t)BR_LPTR(lds);
    int asked = 0, asked_head = 0, asked_tile = 0;
    auto issue = [&](int b) __attribute__((always_inline)) {  // the next tile into buffer b
      if (asked < N) {
        tiles.next(b * BUF_B);
        if constexpr (KEYS) {  // ref (wave 0) and delta (wave 1) of the tile's queries
          if (wv < 2) {
            const u32x4 d = buffer_rows((wv == 0 ? a.ref : a.delta) + (size_t)(h0 + asked_head) * a.s.q_tokens + other.first, (unsigned)n_rows * 4);
            if (lane < PACK_TILE)
              asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds0 + REFS + b * REF_B + wv * (PACK_TILE * 4)),
                           "v"((unsigned)(asked_tile * PACK_TILE + lane) * 4u), "s"(d) : "memory", "m0");
          }
          if (++asked_tile == nt) {
            asked_tile = 0;
            tiles.rewind(++asked_head, wv);
          }
        }
        ++asked;
      }
    };
#pragma unroll
    for (int b = 0; b + 1 < NB; ++b) issue(b);
    clear_last_buffer<DH, NB>(lds);
    tile_turn();
    if (!active) {  // a wave without rows only keeps up its share of the tile traffic
      for (int j = EACH - 1, b = NB - 1; j + 1 < N; j += EACH) {
        tile_turn();
#pragma unroll
        for (int i = 0; i < EACH; ++i, b = b + 1 == NB ? 0 : b + 1) issue(b);
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      return;
    }
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        asm volatile("" : "+v"(f1[qb][ks]), "+v"(f2[qb][ks]));
      }

    TileFrags<DH> frags;
    frags.open(lds);
    // Slot n of a step: a fragment of the scores (n < NA: block of 16 rows, step of the channels, S or X) or of the products behind them.
    auto frag_of = [&](auto Nc, int ao, int co) __attribute__((always_inline)) {  // ao, co: the buffers
      constexpr int n = decltype(Nc)::value, i = n - NA;
      if constexpr (n < NA) return frags.rows(n / (2 * KS), (n >> 1) % KS, ao + (n & 1) * TILE_B);
      else return frags.cols(KEYS ? i >> 1 : i, co + (KEYS ? 1 - (i & 1) : 0) * TILE_B);
    };
    f32x4 s[2][2][QB];               // [S | X][block of 16 rows][own block]
    u32x4 pf[2][QB], df[2][QB];      // P and dS, two bf16 values a word [parity of the tile][own block]
    bf16x8 fr[FR];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) pf[1][qb] = df[1][qb] = u32x4{0, 0, 0, 0};  // (tile -1)
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    const float unit = a.scale * LOG2E;
    f32x4 rv[2], dl[2];  // ref and -delta of the tile's rows (KEYS)
    f32x4 cd[QB];        // -delta of the own queries, four times: what X starts from
    if constexpr (!KEYS) {
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        cd[qb] = f32x4{-delta[qb], -delta[qb], -delta[qb], -delta[qb]};
        asm volatile("" : "+v"(cd[qb]));
      }
    }
    // The probabilities of a tile in 5 operations for each two of a lane's: exponents, exponential, exponential, dS, conversions.
    constexpr int OPS = 5 * 4 * QB;
    float p0 = 0.f, p1 = 0.f, ds0 = 0.f, ds1 = 0.f;  // (of the two in work)
    auto prob = [&](auto Pc, auto Ic) __attribute__((always_inline)) {
      constexpr int P = decltype(Pc)::value, op = decltype(Ic)::value % 5, two = decltype(Ic)::value / 5, b = two / (2 * QB), qb = (two >> 1) % QB, r = 2 * (two & 1);
      if constexpr (op == 0) {
        p0 = fmaf(s[0][b][qb][r], unit, KEYS ? -rv[b][r] : -ref[qb]);
        p1 = fmaf(s[0][b][qb][r + 1], unit, KEYS ? -rv[b][r + 1] : -ref[qb]);
        asm volatile("" : "+v"(p0), "+v"(p1));
      } else if constexpr (op == 1) {
        p0 = __builtin_amdgcn_exp2f(p0);
        asm volatile("" : "+v"(p0));
      } else if constexpr (op == 2) {
        p1 = __builtin_amdgcn_exp2f(p1);
        asm volatile("" : "+v"(p1));
      } else if constexpr (op == 3) {
        ds0 = p0 * s[1][b][qb][r];
        ds1 = p1 * s[1][b][qb][r + 1];
        asm volatile("" : "+v"(ds0), "+v"(ds1));
      } else {
        if constexpr (KEYS) pf[P][qb][b * 2 + r / 2] = two_bf16(p0, p1);
        df[P][qb][b * 2 + r / 2] = two_bf16(ds0, ds1);
      }
    };
    auto use = [&](auto Nc, auto Pc, auto QBc, const bf16x8& f) __attribute__((always_inline)) {  // Pc: parity of the products' tile
      constexpr int n = decltype(Nc)::value, P = decltype(Pc)::value, qb = decltype(QBc)::value;
      if constexpr (n < NA) {
        constexpr int kind = n & 1, b = n / (2 * KS), ks = (n >> 1) % KS;
        s[kind][b][qb] = mma(f, kind == 0 ? f1[qb][ks] : f2[qb][ks], ks > 0 ? s[kind][b][qb] : kind == 0 ? zero : KEYS ? dl[b] : cd[qb]);
      } else {
        constexpr int i = n - NA, d = KEYS ? i >> 1 : i;
        if constexpr (KEYS && (i & 1) == 0) acc2[d][qb] = mma(f, __builtin_bit_cast(bf16x8, pf[P][qb]), acc2[d][qb]);
        else acc1[d][qb] = mma(f, __builtin_bit_cast(bf16x8, df[P][qb]), acc1[d][qb]);
      }
    };
    // Step of tile j (parity P, buffer B): its scores, its probabilities behind the first block's, the products of tile j - 1.
    auto step = [&](auto Pc, auto Bc) __attribute__((always_inline)) {
      constexpr int P = decltype(Pc)::value, B = decltype(Bc)::value, BP = (B + NB - 1) % NB, BN = (B + 1) % NB;
      // Behind each product from G0 on, as many of the operations on the probabilities as spread them evenly: one or two ordinary instructions hide in a product's 16
      // cycles, eight behind one product and none behind the next three cost a wave 20 cycles.
      constexpr int G0 = QB * (NA / 2 + 1), GN = QB * NS;
      static_assert((G0 + GN) / 2 >= QB * NA, "the second block's scores come first");
      if constexpr (KEYS) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          rv[b] = *(const f32x4 __attribute__((address_space(3)))*)(frags.l0 + (REFS + B * REF_B + b * 64) + g * 16);
          dl[b] = *(const f32x4 __attribute__((address_space(3)))*)(frags.l0 + (REFS + B * REF_B + PACK_TILE * 4 + b * 64) + g * 16);
        }
      }
      static_for<NS>([&](auto Nc) __attribute__((always_inline)) {
        constexpr int n = decltype(Nc)::value;
        // (the scores in front: 1 % over both kernels)
        if constexpr (n == 0) __builtin_amdgcn_s_setprio(1);
        if constexpr (n == NA) __builtin_amdgcn_s_setprio(0);
        static_for<QB>([&](auto Qc) __attribute__((always_inline)) {
          use(Nc, std::integral_constant<int, P ^ 1>{}, Qc, fr[n % FR]);
          __builtin_amdgcn_sched_barrier(0);
          if constexpr (decltype(Qc)::value == 0) {
            if constexpr (n + RA < NS) fr[(n + RA) % FR] = frag_of(std::integral_constant<int, n + RA>{}, B * BUF_B, BP * BUF_B);
            else fr[(n + RA) % FR] = frag_of(std::integral_constant<int, n + RA - NS>{}, BN * BUF_B, B * BUF_B);
            __builtin_amdgcn_sched_barrier(0);
          }
          constexpr int gap = n * QB + decltype(Qc)::value;
          if constexpr (gap >= G0) {
            constexpr int from = OPS * (gap - G0) / (GN - G0), to = OPS * (gap - G0 + 1) / (GN - G0);
            static_for<to - from>([&](auto Ic) __attribute__((always_inline)) { prob(Pc, std::integral_constant<int, from + decltype(Ic)::value>{}); });
            __builtin_amdgcn_sched_barrier(0);
          }
        });
      });
      // (used in the next step only: left to itself, the compiler moves every second step's exponentials there, where no matrix instruction runs beside them)
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        u32x4 &x = pf[P][qb], &y = df[P][qb];
        if constexpr (KEYS) asm volatile("" : "+v"(x));
        asm volatile("" : "+v"(y));
      }
    };
    auto behind = [&](auto Bc) __attribute__((always_inline)) {  // the step in buffer B
      constexpr int B = decltype(Bc)::value;
      if constexpr (B % EACH == EACH - 1) {
        tile_turn();
#pragma unroll
        for (int i = EACH; i > 0; --i) issue((B + NB - i) % NB);
      }
    };
    static_for<RA>([&](auto Nc) __attribute__((always_inline)) { fr[decltype(Nc)::value] = frag_of(Nc, 0, 0); });
    u32x4 there;  // ones where the lane's queries of a head's last tile are below the end
    if constexpr (KEYS) {
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const int row = (nt - 1) * PACK_TILE + (e >> 2) * 16 + 4 * g + (e & 3);
        there[e >> 1] = (row < n_rows ? 0x0000FFFFu : 0u) | (row + 1 < n_rows ? 0xFFFF0000u : 0u);
      }
    }
    int j = 0, left = n_rows % PACK_TILE != 0 ? nt : -1;  // (tiles up to a head's last one, if that has rows past the end)
    bool more = true;
    while (more) {
      static_for<NB>([&](auto Bc) __attribute__((always_inline)) {
        if (!more) return;
        constexpr int B = decltype(Bc)::value, P = B & 1;
        step(std::integral_constant<int, P>{}, Bc);
        // rows past the end (zeros, which an infinite own row makes scores of that are not numbers) count as none
        if constexpr (KEYS) {
          if (--left == 0) {
            left = nt;
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
              df[P][qb] &= there;
              pf[P][qb] &= there;
            }
          }
        } else if (j == N - 1) {
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (j * PACK_TILE + (e >> 2) * 16 + 4 * g + (e & 3) >= n_rows) df[P][qb][e >> 1] &= e & 1 ? 0x0000FFFFu : 0xFFFF0000u;
        }
        more = ++j < N;
        if (more) behind(Bc);
      });
    }
    if constexpr (!KEYS) {
      if (brief) {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
          float p[8], d = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            p[e] = (e >> 2) * 16 + 4 * g + (e & 3) < n_rows ? __builtin_amdgcn_exp2f(fmaf(s[0][e >> 2][qb][e & 3], unit, -ref[qb])) : 0.f;
            d = fmaf(p[e], s[1][e >> 2][qb][e & 3], d);
          }
          d = quarters_sum(d);
#pragma unroll
          for (int e = 0; e < 8; e += 2) df[0][qb][e >> 1] = two_bf16(p[e] * (s[1][e >> 2][qb][e & 3] - d), p[e + 1] * (s[1][e >> 2][qb][(e & 3) + 1] - d));
          if (g == 0 && row0 + qb * 16 + l16 < own.end) a.delta[(size_t)head * a.s.q_tokens + row0 + qb * 16 + l16] = -d;
        }
      }
    }
    auto last = [&](auto Pc, int at) __attribute__((always_inline)) {  // products of the last tile, `at` bytes on
      static_for<NC>([&](auto Ic) __attribute__((always_inline)) {
        using Nc = std::integral_constant<int, NA + decltype(Ic)::value>;
        const bf16x8 f = frag_of(Nc{}, 0, at);
        static_for<QB>([&](auto Qc) __attribute__((always_inline)) { use(Nc{}, Pc, Qc, f); });
      });
    };
    const int at = (N - 1) % NB * BUF_B;
    if (N & 1) last(std::integral_constant<int, 0>{}, at);
    else last(std::integral_constant<int, 1>{}, at);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }
  if (!active) return;
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const int row = row0 + qb * 16 + l16;
    if (row >= own.end) continue;
    if (a.parts > 1) {
      const int tokens = KEYS ? a.s.k_tokens : a.s.q_tokens, heads = KEYS ? a.s.n_kv_heads : a.s.n_heads;
      float* to = part_row(a.part, part_of, tokens, row, heads, head, DH) + 4 * g;
#pragma unroll
      for (int d = 0; d < DB; ++d) *reinterpret_cast<f32x4*>(to + 16 * d) = acc1[d][qb];
      if constexpr (KEYS) {
        to = part_row(a.part2, part_of, tokens, row, heads, head, DH) + 4 * g;
#pragma unroll
        for (int d = 0; d < DB; ++d) *reinterpret_cast<f32x4*>(to + 16 * d) = acc2[d][qb];
      }
      continue;
    }
    bf16* to1 = KEYS ? (bf16*)a.dk + (size_t)row * a.s.dk_stride + (size_t)kv * DH + 4 * g : (bf16*)a.dq + (size_t)row * a.s.dq_stride + (size_t)head * DH + 4 * g;
#pragma unroll
    for (int d = 0; d < DB; ++d) store4(to1 + 16 * d, acc1[d][qb][0] * a.scale, acc1[d][qb][1] * a.scale, acc1[d][qb][2] * a.scale, acc1[d][qb][3] * a.scale);
    if constexpr (KEYS) {
      bf16* to2 = (bf16*)a.dv + (size_t)row * a.s.dv_stride + (size_t)kv * DH + 4 * g;
#pragma unroll
      for (int d = 0; d < DB; ++d) store4(to2 + 16 * d, acc2[d][qb][0], acc2[d][qb][1], acc2[d][qb][2], acc2[d][qb][3]);
    }
  }
}

template <int DH, Pass PASS, bool HALVES>
__global__ __launch_bounds__(256, (PackForm<DH, PASS>::WPE)) void packed_grad_bf16_kernel(AttnArgs a) {
  constexpr bool KEYS = PASS == Pass::KEYS;
  OwnRows place;
  if (!own_place(a, KEYS ? a.s.k_off : a.s.q_off, KEYS ? a.s.k_tokens : a.s.q_tokens, KEYS ? a.s.n_kv_heads : a.s.n_heads, PACK_OWN, &place)) return;
  if constexpr (HALVES) {
    if (place.half) return packed_grad_rows<DH, PASS, 1>(a, place);
  }
  packed_grad_rows<DH, PASS, 2>(a, place);
}

br_status launch_attn_forward_bf16(AttnArgs a, int parts, hipStream_t st) {
  unsigned n;
  const br_status ok = attn_grid(a, a.s.q_tokens, a.s.n_heads, PACK_OWN, parts, pack_per_cu(a.s.head_dim, 0), &n);
  if (ok != BR_OK) return ok;
  auto run = [&](auto Dc) {
    constexpr int DH = decltype(Dc)::value;
    if (a.slots > 0) hipLaunchKernelGGL((packed_forward_bf16_kernel<DH, true>), dim3(n), dim3(256), (PackForm<DH, Pass::FORWARD>::LDS), st, a);
    else hipLaunchKernelGGL((packed_forward_bf16_kernel<DH, false>), dim3(n), dim3(256), (PackForm<DH, Pass::FORWARD>::LDS), st, a);
  };
  if (a.s.head_dim == 64) run(std::integral_constant<int, 64>{});
  else run(std::integral_constant<int, 128>{});
  BR_LAUNCH_CHECK();
  return parts > 1 ? launch_attn_join_forward(a, st) : BR_OK;
}

template <int DH>
static br_status grad_launch(AttnArgs a, int parts_q, int parts_k, hipStream_t st) {
  unsigned n;
  if (a.s.q_tokens > 0) {
    br_status ok = attn_grid(a, a.s.q_tokens, a.s.n_heads, PACK_OWN, parts_q, pack_per_cu(DH, 1), &n);
    if (ok != BR_OK) return ok;
    if (a.slots > 0) hipLaunchKernelGGL((packed_grad_bf16_kernel<DH, Pass::QUERIES, true>), dim3(n), dim3(256), (PackForm<DH, Pass::QUERIES>::LDS), st, a);
    else hipLaunchKernelGGL((packed_grad_bf16_kernel<DH, Pass::QUERIES, false>), dim3(n), dim3(256), (PackForm<DH, Pass::QUERIES>::LDS), st, a);
    BR_LAUNCH_CHECK();
    if (parts_q > 1 && (ok = launch_attn_join_dq(a, st)) != BR_OK) return ok;
  }
  if (a.s.k_tokens > 0) {
    br_status ok = attn_grid(a, a.s.k_tokens, a.s.n_kv_heads, PACK_OWN, parts_k, pack_per_cu(DH, 2), &n);
    if (ok != BR_OK) return ok;
    if (a.slots > 0) hipLaunchKernelGGL((packed_grad_bf16_kernel<DH, Pass::KEYS, true>), dim3(n), dim3(256), (PackForm<DH, Pass::KEYS>::LDS), st, a);
    else hipLaunchKernelGGL((packed_grad_bf16_kernel<DH, Pass::KEYS, false>), dim3(n), dim3(256), (PackForm<DH, Pass::KEYS>::LDS), st, a);
    BR_LAUNCH_CHECK();
    if (parts_k > 1 && (ok = launch_attn_join_dkv(a, st)) != BR_OK) return ok;
  }
  return BR_OK;
}

br_status launch_attn_grad_bf16(AttnArgs a, int parts_q, int parts_k, hipStream_t st) {
  return a.s.head_dim == 64 ? grad_launch<64>(a, parts_q, parts_k, st) : grad_launch<128>(a, parts_q, parts_k, st);
}

// Rows of a document are addressed with 32-bit byte offsets from its first one; the host knows the matrices' size only.  Past it, eight documents of 1063 tokens, 16 heads of 64,
// forward and backward: 94 and 249 us in the general form, 53 and 165 here.
bool attn_packed_bf16_fits(const br_attn_shape& s) {
  auto fits = [](int64_t tokens, int64_t stride) { return tokens * stride * 2 < (1LL << 32); };
  return s.dtype == BR_BF16 && fits(s.q_tokens, s.q_stride) && fits(s.q_tokens, s.o_stride) && fits(s.k_tokens, s.k_stride) && fits(s.k_tokens, s.v_stride);
}

}  // namespace br
