// The backward pass of bf16 attention over packed documents: dq (own rows: queries, tiles of keys), and dk with dv (own rows: keys, tiles of queries).
//
// A wavefront keeps 32 rows of its side in registers (column operands of both score products) and their gradients in accumulators, and walks tiles of 32
// rows of the other side in LDS.  Tile j: scores S = Y1 X1 and X = Y2 X2 (X1, X2: own q and dout, or own k and v), probabilities P = exp2(S - ref), dS = P
// (X - delta), and the products with the tile's rows, dk += Y1^T dS (dq the same) and dv += Y2^T P.  These wait for the next tile: between its scores' last
// matrix instructions and theirs stand the exponentials of the tile itself.
//
// Tiles come straight from global memory into LDS (four buffers), rows as they lie, 16-byte chunks permuted per row so that both the fragments of 16 rows
// and the transposed reads (eight rows, two chunks) spread over the banks.
#include "attn_packed.h"
#include "static_for.h"

namespace br {

#define BR_LPTR(p) ((void __attribute__((address_space(3)))*)(p))

extern __shared__ __attribute__((aligned(1024))) char g_grad_tiles[];

constexpr int GRAD_TILE = 32, GRAD_NB = 4, GRAD_OWN = 128;  // rows of a tile, buffers, own rows of a workgroup

static __device__ inline u32x4 buffer_rows(const void* p, unsigned bytes) {
  const unsigned long long v = reinterpret_cast<unsigned long long>(p);
  return u32x4{(unsigned)__builtin_amdgcn_readfirstlane((unsigned)v), (unsigned)__builtin_amdgcn_readfirstlane((unsigned)(v >> 32)) & 0xffffu,
               (unsigned)__builtin_amdgcn_readfirstlane(bytes), 0x00020000u};
}

template <int DH>
constexpr int GRAD_LDS = GRAD_NB * (2 * GRAD_TILE * DH * 2 + 2 * GRAD_TILE * 4);

// Waves a SIMD: dk and dv of head dim 128 have 128 accumulators and 64 operands a lane.
template <int DH, bool KEYS>
__global__ __launch_bounds__(256, DH == 128 && KEYS ? 1 : 2) void packed_grad_bf16_kernel(AttnArgs a) {
  constexpr int CH = DH / 8, KS = DH / 32, DB = DH / 16, RPI = 64 / CH, LPW = GRAD_TILE / RPI / 4;
  constexpr int ROW_B = DH * 2, TILE_B = GRAD_TILE * ROW_B, BUF_B = 2 * TILE_B, QB = 2;
  constexpr int NA = 4 * KS, NC = KEYS ? 2 * DB : DB, NS = NA + NC, FR = DH == 128 && KEYS ? 8 : 4, RA = FR - 1;
  constexpr int REFS = GRAD_NB * BUF_B, REF_B = 2 * GRAD_TILE * 4;  // ref and delta of a tile's rows, behind the tiles
  static_assert(NS % FR == 0 && LPW >= 1, "");
  char* lds = g_grad_tiles;

  const int share = a.s.n_heads / a.s.n_kv_heads;
  int head, tile, own0;
  DocSpan own;
  const int* own_off = KEYS ? a.s.k_off : a.s.q_off;
  if (!head_tile(KEYS ? a.s.n_kv_heads : a.s.n_heads, a.tiles, &head, &tile) ||
      !doc_tile(own_off, a.s.n_docs, KEYS ? a.s.k_tokens : a.s.q_tokens, GRAD_OWN, tile, &own, &own0))
    return;
  const DocSpan other = other_rows(KEYS ? a.s.q_off : a.s.k_off, a.s.n_docs, KEYS ? a.s.q_tokens : a.s.k_tokens, own);
  const int kv = KEYS ? head : head / share, h0 = KEYS ? head * share : head;
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row0 = own0 + wv * 32;
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
      delta[qb] = quarters_sum(d);
      ref[qb] = lse == -INFINITY ? INFINITY : lse * LOG2E;
      if (g == 0 && row0 + qb * 16 + l16 < own.end) {
        a.ref[at] = ref[qb];
        a.delta[at] = delta[qb];
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

  const int n_rows = other.end - other.first, nt = (n_rows + GRAD_TILE - 1) / GRAD_TILE, N = KEYS ? nt * share : nt;
  if (N > 0) {
    // ---- tiles: 1 KB an instruction, lane i fills bytes 16 i .. 16 i + 15, so the permutation is applied on the global side; rows past the document's end
    // lie past the buffer's and arrive as zeros
    const bf16* y1 = (KEYS ? (const bf16*)a.q + (size_t)h0 * DH : (const bf16*)a.k + (size_t)kv * DH) + (size_t)other.first * (KEYS ? a.s.q_stride : a.s.k_stride);
    const bf16* y2 = (KEYS ? (const bf16*)a.dout + (size_t)h0 * DH : (const bf16*)a.v + (size_t)kv * DH) + (size_t)other.first * (KEYS ? a.s.o_stride : a.s.v_stride);
    const unsigned lb1 = (unsigned)((KEYS ? a.s.q_stride : a.s.k_stride) * 2), lb2 = (unsigned)((KEYS ? a.s.o_stride : a.s.v_stride) * 2);
    const unsigned width = (KEYS ? share : 1) * ROW_B;
    const u32x4 rows1 = buffer_rows(y1, (unsigned)(n_rows - 1) * lb1 + width), rows2 = buffer_rows(y2, (unsigned)(n_rows - 1) * lb2 + width);
    auto swz = [](int r) { return DH == 128 ? ((r & 7) << 1 | (r >> 3 & 1)) : ((r >> 1 & 3) << 1 | (r >> 3 & 1)); };
    unsigned off1[LPW], off2[LPW];
    const int lrow = lane / CH, slot = lane % CH;
    auto rewind = [&](int h) __attribute__((always_inline)) {  // first tile of head h0 + h
#pragma unroll
      for (int t = 0; t < LPW; ++t) {
        const int r = (wv * LPW + t) * RPI + lrow;
        const unsigned c = h * ROW_B + ((slot ^ swz(r)) << 4);
        off1[t] = r < n_rows ? r * lb1 + c : 0xFFFFFFFFu;
        off2[t] = r < n_rows ? r * lb2 + c : 0xFFFFFFFFu;
      }
    };
    rewind(0);
    const unsigned lds0 = (unsigned)(uintptr_t)BR_LPTR(lds), lds_w = lds0 + wv * LPW * 1024;
    int asked = 0, asked_head = 0, asked_tile = 0;
    auto issue = [&](int b) __attribute__((always_inline)) {  // the next tile into buffer b
      if (asked < N) {
        const int buf = b * BUF_B;
#pragma unroll
        for (int t = 0; t < LPW; ++t) {
          asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds_w + buf + t * 1024), "v"(off1[t]), "s"(rows1) : "memory", "m0");
          asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds_w + buf + TILE_B + t * 1024), "v"(off2[t]), "s"(rows2) : "memory", "m0");
          off1[t] = __builtin_elementwise_add_sat(off1[t], GRAD_TILE * lb1);
          off2[t] = __builtin_elementwise_add_sat(off2[t], GRAD_TILE * lb2);
        }
        if constexpr (KEYS) {  // ref (wave 0) and delta (wave 1) of the tile's queries
          if (wv < 2) {
            const u32x4 d = buffer_rows((wv == 0 ? a.ref : a.delta) + (size_t)(h0 + asked_head) * a.s.q_tokens + other.first, (unsigned)n_rows * 4);
            if (lane < GRAD_TILE)
              asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds0 + REFS + b * REF_B + wv * (GRAD_TILE * 4)),
                           "v"((unsigned)(asked_tile * GRAD_TILE + lane) * 4u), "s"(d) : "memory", "m0");
          }
          if (++asked_tile == nt) {
            asked_tile = 0;
            rewind(++asked_head);
          }
        }
        ++asked;
      }
    };
    // Behind step j: tile j + 2 has landed, every wave is done with tile j - 1, whose buffer takes tile j + 3.
    auto turn = [&]() __attribute__((always_inline)) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    };
    issue(0);
    issue(1);
    issue(2);
    // Tile -1, whose gradients are zeros, lies in the last buffer: finite rows there
    for (int at = tid * 16; at < BUF_B; at += 256 * 16) *reinterpret_cast<u32x4*>(lds + (GRAD_NB - 1) * BUF_B + at) = u32x4{0, 0, 0, 0};
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    turn();
    if (!active) {  // a wave without rows only keeps up its share of the tile traffic
      for (int j = 0; j + 1 < N; ++j) {
        turn();
        issue((j + 3) % GRAD_NB);
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

    unsigned raddr[KS], caddr[DB];  // this lane's fragments in buffer 0
    static_for<KS>([&](auto Kc) __attribute__((always_inline)) {
      constexpr int ks = decltype(Kc)::value;
      raddr[ks] = l16 * ROW_B + (((ks * 4 + g) ^ swz(l16)) << 4);
    });
    const int crow = 4 * g + (l16 >> 2);
    static_for<DB>([&](auto Dc) __attribute__((always_inline)) {
      constexpr int d = decltype(Dc)::value;
      caddr[d] = crow * ROW_B + (((2 * d + ((l16 & 3) >> 1)) ^ swz(crow)) << 4) + 8 * (l16 & 1);
    });
    typedef const char __attribute__((address_space(3)))* lptr;
    const lptr l0 = (lptr)BR_LPTR(lds);
    // Slot n of a step: a fragment of the scores (n < NA: block of 16 rows, step of the channels, S or X) or of the products behind them.
    auto frag_of = [&](auto Nc, int ao, int co) __attribute__((always_inline)) {  // ao, co: the buffers
      constexpr int n = decltype(Nc)::value;
      if constexpr (n < NA) {
        return *(const bf16x8 __attribute__((address_space(3)))*)(l0 + raddr[(n >> 1) % KS] + (ao + (n & 1) * TILE_B + n / (2 * KS) * 16 * ROW_B));
      } else {
        constexpr int i = n - NA, d = KEYS ? i >> 1 : i, y = KEYS ? 1 - (i & 1) : 0;
        const lptr p = l0 + caddr[d] + (co + y * TILE_B);
        union { s16x4 s[2]; bf16x8 v; } u;
        u.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)p);
        u.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(p + 16 * ROW_B));
        return u.v;
      }
    };
    f32x4 s[2][2][QB];               // [S | X][block of 16 rows][own block]
    bf16x8 pf[2][QB], df[2][QB];     // [parity of the tile][own block]
    bf16x8 fr[FR];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
      for (int e = 0; e < 8; ++e) pf[1][qb][e] = df[1][qb][e] = (bf16)0.f;  // (tile -1)
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    auto mma = [](bf16x8 x, bf16x8 y, f32x4 c) __attribute__((always_inline)) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0); };
    const float unit = a.scale * LOG2E;
    f32x4 rv[2], dl[2];  // ref and delta of the tile's rows (KEYS)
    auto prob = [&](auto Pc, int e) __attribute__((always_inline)) {
      constexpr int P = decltype(Pc)::value;
      const int b = e / (4 * QB), qb = (e >> 2) % QB, r = e & 3;
      const float p = __builtin_amdgcn_exp2f(fmaf(s[0][b][qb][r], unit, KEYS ? -rv[b][r] : -ref[qb]));
      const float ds = p * (s[1][b][qb][r] - (KEYS ? dl[b][r] : delta[qb]));
      if constexpr (KEYS) pf[P][qb][b * 4 + r] = (bf16)p;
      df[P][qb][b * 4 + r] = (bf16)ds;
    };
    auto use = [&](auto Nc, auto Pc, auto QBc, const bf16x8& f) __attribute__((always_inline)) {  // Pc: parity of the products' tile
      constexpr int n = decltype(Nc)::value, P = decltype(Pc)::value, qb = decltype(QBc)::value;
      if constexpr (n < NA) {
        constexpr int kind = n & 1, b = n / (2 * KS), ks = (n >> 1) % KS;
        s[kind][b][qb] = mma(f, kind == 0 ? f1[qb][ks] : f2[qb][ks], ks == 0 ? zero : s[kind][b][qb]);
      } else {
        constexpr int i = n - NA, d = KEYS ? i >> 1 : i;
        if constexpr (KEYS && (i & 1) == 0) acc2[d][qb] = mma(f, pf[P][qb], acc2[d][qb]);
        else acc1[d][qb] = mma(f, df[P][qb], acc1[d][qb]);
      }
    };
    // Step of tile j (parity P, buffer B): its scores, its probabilities behind the first block's, the products of tile j - 1.
    auto step = [&](auto Pc, auto Bc) __attribute__((always_inline)) {
      constexpr int P = decltype(Pc)::value, B = decltype(Bc)::value, BP = (B + GRAD_NB - 1) % GRAD_NB, BN = (B + 1) % GRAD_NB;
      constexpr int E0 = NA / 2 + 2, EN = NS - 1, NE = 8 * QB;  // the probabilities are taken in these slots
      constexpr int E1 = NA + 1;                                // those of the second block from here on
      if constexpr (KEYS) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          rv[b] = *(const f32x4 __attribute__((address_space(3)))*)(l0 + (REFS + B * REF_B + b * 64) + g * 16);
          dl[b] = *(const f32x4 __attribute__((address_space(3)))*)(l0 + (REFS + B * REF_B + GRAD_TILE * 4 + b * 64) + g * 16);
        }
      }
      static_for<NS>([&](auto Nc) __attribute__((always_inline)) {
        constexpr int n = decltype(Nc)::value;
        if constexpr (n + RA < NS) fr[(n + RA) % FR] = frag_of(std::integral_constant<int, n + RA>{}, B * BUF_B, BP * BUF_B);
        else fr[(n + RA) % FR] = frag_of(std::integral_constant<int, n + RA - NS>{}, BN * BUF_B, B * BUF_B);
        __builtin_amdgcn_sched_barrier(0);
        static_for<QB>([&](auto Qc) __attribute__((always_inline)) {
          use(Nc, std::integral_constant<int, P ^ 1>{}, Qc, fr[n % FR]);
          __builtin_amdgcn_sched_barrier(0);
          if constexpr (decltype(Qc)::value == 0) {
            if constexpr (n >= E0 && n < E1) {
#pragma unroll
              for (int e = NE / 2 * (n - E0) / (E1 - E0); e < NE / 2 * (n - E0 + 1) / (E1 - E0); ++e) prob(Pc, e);
            } else if constexpr (n >= E1 && n < EN) {
#pragma unroll
              for (int e = NE / 2 * (n - E1) / (EN - E1); e < NE / 2 * (n - E1 + 1) / (EN - E1); ++e) prob(Pc, NE / 2 + e);
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        });
      });
    };
    static_for<RA>([&](auto Nc) __attribute__((always_inline)) { fr[decltype(Nc)::value] = frag_of(Nc, 0, 0); });
    int j = 0;
    bool more = true;
    while (more) {
      static_for<GRAD_NB>([&](auto Bc) __attribute__((always_inline)) {
        if (!more) return;
        constexpr int B = decltype(Bc)::value, P = B & 1;
        step(std::integral_constant<int, P>{}, Bc);
        if (!KEYS && j == N - 1) {  // keys past the end
#pragma unroll
          for (int qb = 0; qb < QB; ++qb)
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (j * GRAD_TILE + (e >> 2) * 16 + 4 * g + (e & 3) >= n_rows) df[P][qb][e] = (bf16)0.f;
        }
        more = ++j < N;
        if (more) {
          turn();
          issue((B + 3) % GRAD_NB);
        } else {  // products of the last tile
          static_for<NC>([&](auto Ic) __attribute__((always_inline)) {
            using Nc = std::integral_constant<int, NA + decltype(Ic)::value>;
            const bf16x8 f = frag_of(Nc{}, 0, B * BUF_B);
            static_for<QB>([&](auto Qc) __attribute__((always_inline)) { use(Nc{}, std::integral_constant<int, P>{}, Qc, f); });
          });
        }
      });
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }
  if (!active) return;
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const int row = row0 + qb * 16 + l16;
    if (row >= own.end) continue;
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

// Rows of a document are addressed with 32-bit byte offsets from its first one.
bool attn_grad_bf16_fits(const br_attn_shape& s) {
  auto fits = [](int64_t tokens, int64_t stride) { return tokens * stride * 2 < (1LL << 32); };
  return s.dtype == BR_BF16 && fits(s.q_tokens, s.q_stride) && fits(s.q_tokens, s.o_stride) && fits(s.k_tokens, s.k_stride) && fits(s.k_tokens, s.v_stride);
}

template <int DH>
static br_status grad_launch(AttnArgs a, hipStream_t st) {
  auto run = [&](auto KEYSc, int tokens, int heads) -> br_status {
    constexpr bool KEYS = decltype(KEYSc)::value;
    if (tokens == 0) return BR_OK;
    a.tiles = (int)doc_tiles_most(a.s.n_docs, tokens, GRAD_OWN);
    hipLaunchKernelGGL((packed_grad_bf16_kernel<DH, KEYS>), dim3((unsigned)head_tile_blocks(heads, a.tiles)), dim3(256), GRAD_LDS<DH>, st, a);
    BR_LAUNCH_CHECK();
    return BR_OK;
  };
  const br_status ok = run(std::false_type{}, a.s.q_tokens, a.s.n_heads);
  return ok != BR_OK ? ok : run(std::true_type{}, a.s.k_tokens, a.s.n_kv_heads);
}

br_status launch_attn_grad_bf16(AttnArgs a, hipStream_t st) { return a.s.head_dim == 64 ? grad_launch<64>(a, st) : grad_launch<128>(a, st); }

}  // namespace br
