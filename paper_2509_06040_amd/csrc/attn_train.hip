// Attention over packed documents with its backward pass: the forms that hold for every type and head dim (fp32; bf16 where offsets pass 32 bits).
//
// A wavefront keeps 16 rows of one side in registers (queries forward and for dq, keys for dk and dv) and walks the rows of the other side in tiles of 64
// that the workgroup stages in LDS, the next tile on its way in registers meanwhile.  Scores are taken so that a lane holds four rows of the tile for ONE row of
// its own per block of 16 (C layout of the 16x16 matrix instructions); exponentiated, these registers are, without moving, the column operand of the
// products that contract over the tile's rows, whose row operand is read from LDS transposed.
//
// WIDE: the four wavefronts have 16 own rows each and all of the tile.  Otherwise (fp32 launches that would leave compute units empty) they share 16 own rows and
// take 16 rows of the tile each; their sums are joined through LDS at the end.
//
// Bound by the fp32 matrix instructions (154 TFLOP/s in a library product) where there are rows for all units: 16 heads, documents of 1001 tokens, eight with heads of 64: forward 315 us, 104
// TFLOP/s, backward 1014 us, 81 by the formulas' five products, 113 by the seven taken; four with heads of 128: 105, 72 and 101.  By latency below: eight heads of 64 on two, six documents of 5 to 404
// tokens 22 us for dq, 29 for dk and dv, 4.5 for their join (each wavefront staging its own rows without barriers: 21, 30).
#include "attn_packed.h"

namespace br {

// Operands of a type.  A fragment holds EPL consecutive contraction indices of quarter g of the lanes: a step contracts 4 EPL of them.
template <typename T>
struct Op;
template <>
struct Op<bf16> {
  using Frag = bf16x8;
  static constexpr int EPL = 8;
  static __device__ inline f32x4 mma(const Frag& a, const Frag& b, const f32x4& c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Op<float> {
  using Frag = f32x4;
  static constexpr int EPL = 4;
  static __device__ inline f32x4 mma(const Frag& a, const Frag& b, f32x4 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);  // (each takes index 4 g + e from quarter g)
    return c;
  }
};

// A tile of 64 rows of DH values in LDS.  Rows of bf16 lie as they are, their 16-byte chunks permuted per row so that fragments of 16 consecutive rows and
// transposed reads of eight rows and two chunks both spread over the banks; rows of fp32 are 16 bytes further apart.
constexpr int TILE_ROWS = 64;
template <typename T, int DH>
struct Tile {
  static constexpr int ROW = DH * (int)sizeof(T) + (sizeof(T) == 4 ? 16 : 0), BYTES = TILE_ROWS * ROW, CH = DH * (int)sizeof(T) / 16;
  static __device__ inline int chunk(int r, int c) {
    if constexpr (sizeof(T) == 4) return r * ROW + c * 16;
    const int f = DH == 128 ? (r & 7) << 1 : (r >> 1 & 3) << 1;
    return r * ROW + ((c ^ f) << 4);
  }
  static constexpr int EACH = TILE_ROWS * CH / 256;  // 16-byte chunks a thread
  static_assert(TILE_ROWS * CH % 256 == 0, "");
  struct Regs {
    f32x4 v[EACH];
  };
  // rows first .. first + 63 (those from `end` on: zeros) of a matrix with `stride` elements a row
  static __device__ inline void fetch(Regs& r, const T* p, size_t stride, int first, int end) {
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int i = k * 256 + threadIdx.x, row = i / CH, c = i - row * CH;
      r.v[k] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (first + row < end) r.v[k] = *reinterpret_cast<const f32x4*>(reinterpret_cast<const char*>(p + (size_t)(first + row) * stride) + c * 16);
    }
  }
  static __device__ inline void put(char* lds, const Regs& r) {
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int i = k * 256 + threadIdx.x, row = i / CH, c = i - row * CH;
      *reinterpret_cast<f32x4*>(lds + chunk(row, c)) = r.v[k];
    }
  }
  // row operand: rows 16 blk + lane % 16, contraction over the channels of step ks
  static __device__ inline typename Op<T>::Frag rows(const char* lds, int blk, int ks) {
    const int lane = threadIdx.x & 63;
    return *reinterpret_cast<const typename Op<T>::Frag*>(lds + chunk(blk * 16 + (lane & 15), ks * 4 + (lane >> 4)));
  }
  // row operand: channels 16 d + lane % 16, contraction over the rows of step ks: rows 4 g + e of its blocks of 16
  static __device__ inline typename Op<T>::Frag cols(const char* lds, int ks, int d) {
    const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
    if constexpr (sizeof(T) == 2) {
      // in a group of 16 lanes, lane 4 r + q supplies the address of 8 bytes (4 values of row r) and lane j receives element j of rows 0..3
      const int r = 4 * g + (l16 >> 2), at = chunk(ks * 32 + r, 2 * d + ((l16 & 3) >> 1)) + 8 * (l16 & 1), at2 = chunk(ks * 32 + 16 + r, 2 * d + ((l16 & 3) >> 1)) + 8 * (l16 & 1);
      union { s16x4 s[2]; bf16x8 v; } u;
      u.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(lds + at));
      u.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(lds + at2));
      return u.v;
    } else {
      f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<const float*>(lds + (ks * 16 + 4 * g + e) * ROW + (16 * d + l16) * 4);
      return v;
    }
  }
};

// Column operands from registers: row `row` of a matrix (below `end`, else zeros), all channels.
template <typename T, int DH>
static __device__ inline void own_rows(typename Op<T>::Frag (&f)[DH / (4 * Op<T>::EPL)], const T* p, size_t stride, int row, int end) {
#pragma unroll
  for (int ks = 0; ks < DH / (4 * Op<T>::EPL); ++ks) {
    f[ks] = typename Op<T>::Frag{};
    if (row < end) f[ks] = *reinterpret_cast<const typename Op<T>::Frag*>(p + (size_t)row * stride + ks * 4 * Op<T>::EPL + (threadIdx.x >> 4 & 3) * Op<T>::EPL);
  }
}
// Step ks of a contraction over the tile's rows: blocks of 16 rows in the C layout, in the type of the operands.
template <typename T>
static __device__ inline typename Op<T>::Frag step_of(const f32x4* p, int ks) {
  if constexpr (sizeof(T) == 2) {
    bf16x8 f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (bf16)p[2 * ks + (e >> 2)][e & 3];
    return f;
  } else {
    return p[ks];
  }
}

// WIDE: each wavefront's blocks d of 16 channels, else their sums over the four wavefronts (in their order; block d by wavefront d % 4).  f(d, values).
template <int DB, bool WIDE, typename F>
static __device__ inline void joined(char* lds, const f32x4 (&acc)[DB], F f) {
  if constexpr (WIDE) {
#pragma unroll
    for (int d = 0; d < DB; ++d) f(d, acc[d]);
  } else {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    f32x4* to = reinterpret_cast<f32x4*>(lds);
    __syncthreads();
#pragma unroll
    for (int d = 0; d < DB; ++d) to[(wave * DB + d) * 64 + lane] = acc[d];
    __syncthreads();
#pragma unroll
    for (int d = 0; d < DB; ++d)
      if (d % 4 == wave) f(d, (to[d * 64 + lane] + to[(DB + d) * 64 + lane]) + (to[(2 * DB + d) * 64 + lane] + to[(3 * DB + d) * 64 + lane]));
  }
}

template <typename T, int DH, bool WIDE>
struct Kernel {  // sizes of the kernels below
  using O = Op<T>;
  using L = Tile<T, DH>;
  static constexpr int KS = DH / (4 * O::EPL), DB = DH / 16, OWN = WIDE ? 64 : 16;
  static constexpr int NB = WIDE ? 4 : 1, PS = 16 * NB / (4 * O::EPL);  // blocks of 16 rows of the tile a wavefront takes, steps over them
  static_assert(WIDE || O::EPL == 4, "");
};

template <typename T, int DH, bool WIDE>
__global__ __launch_bounds__(256) void packed_attention_kernel(AttnArgs a) {
  using K = Kernel<T, DH, WIDE>;
  using O = Op<T>;
  using L = Tile<T, DH>;
  constexpr int KS = K::KS, PS = K::PS, DB = K::DB, NB = K::NB;
  __shared__ __attribute__((aligned(16))) char lds[2 * L::BYTES];
  __shared__ float tops[4][16], sums[4][16];
  OwnRows place;
  if (!own_place(a, a.s.q_off, a.s.q_tokens, a.s.n_heads, K::OWN, &place)) return;
  const DocSpan span = place.span;
  const int first = place.row, head = place.head, part_of = place.part;
  DocSpan keys = other_rows(a.s.k_off, a.s.n_docs, a.s.k_tokens, span);
  take_part(&keys, a.parts, part_of, TILE_ROWS);
  const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kv = head / (a.s.n_heads / a.s.n_kv_heads);
  const int row = first + (WIDE ? wave * 16 : 0) + l16, b0 = WIDE ? 0 : wave;
  const T *k = (const T*)a.k + (size_t)kv * DH, *v = (const T*)a.v + (size_t)kv * DH;
  typename O::Frag q[KS];
  own_rows<T, DH>(q, (const T*)a.q + (size_t)head * DH, a.s.q_stride, row, span.end);
  f32x4 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  float top = -INFINITY, sum = 0.f;
  const float unit = a.scale * LOG2E;  // scores in powers of two
  typename L::Regs nk, nv;
  L::fetch(nk, k, a.s.k_stride, keys.first, keys.end);
  L::fetch(nv, v, a.s.v_stride, keys.first, keys.end);
  for (int k0 = keys.first; k0 < keys.end; k0 += TILE_ROWS) {
    __syncthreads();
    L::put(lds, nk);
    L::put(lds + L::BYTES, nv);
    __syncthreads();
    L::fetch(nk, k, a.s.k_stride, k0 + TILE_ROWS, keys.end);
    L::fetch(nv, v, a.s.v_stride, k0 + TILE_ROWS, keys.end);
    f32x4 p[NB];
    float most = -INFINITY;
#pragma unroll
    for (int b = 0; b < NB; ++b) p[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int b = 0; b < NB; ++b) p[b] = O::mma(L::rows(lds, b0 + b, ks), q[ks], p[b]);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[b][r] = k0 + (b0 + b) * 16 + 4 * g + r < keys.end ? p[b][r] * unit : -INFINITY;
        most = __builtin_elementwise_maximum(most, p[b][r]);
      }
    const float next = __builtin_elementwise_maximum(top, quarters_max(most)), ref = next == -INFINITY ? 0.f : next;
    const float shrink = __builtin_amdgcn_exp2f(top - ref);
    float part = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[b][r] = __builtin_amdgcn_exp2f(p[b][r] - ref);
        part += p[b][r];
      }
    sum = sum * shrink + part;
    top = next;
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] *= shrink;
#pragma unroll
    for (int ks = 0; ks < PS; ++ks) {
      const typename O::Frag pf = step_of<T>(p, ks);
#pragma unroll
      for (int d = 0; d < DB; ++d) o[d] = O::mma(L::cols(lds + L::BYTES, b0 + ks, d), pf, o[d]);
    }
  }
  sum = quarters_sum(sum);
  if constexpr (!WIDE) {  // one reference for the four wavefronts
    if (g == 0) {
      tops[wave][l16] = top;
      sums[wave][l16] = sum;
    }
    __syncthreads();
    const float most = __builtin_elementwise_maximum(__builtin_elementwise_maximum(tops[0][l16], tops[1][l16]), __builtin_elementwise_maximum(tops[2][l16], tops[3][l16]));
    const float ref = most == -INFINITY ? 0.f : most, shrink = __builtin_amdgcn_exp2f(top - ref);
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] *= shrink;
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) sum += sums[w][l16] * __builtin_amdgcn_exp2f(tops[w][l16] - ref);
    top = most;
  }
  if (a.parts > 1) {
    float* to = part_row(a.part, part_of, a.s.q_tokens, row, a.s.n_heads, head, DH) + 4 * g;
    joined<DB, WIDE>(lds, o, [&](int d, f32x4 x) {
      if (row < span.end) *reinterpret_cast<f32x4*>(to + 16 * d) = x;
    });
    if (row < span.end && g == 0 && (WIDE || wave == 0)) {
      const size_t at = ((size_t)part_of * a.s.n_heads + head) * a.s.q_tokens + row;
      a.part_ref[at] = top;
      a.part_sum[at] = sum;
    }
    return;
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  T* out = (T*)a.o + (size_t)row * a.s.o_stride + (size_t)head * DH + 4 * g;
  joined<DB, WIDE>(lds, o, [&](int d, f32x4 x) {
    if (row < span.end) store4(out + 16 * d, x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
  });
  if (row < span.end && g == 0 && (WIDE || wave == 0)) a.lse[(size_t)head * a.s.q_tokens + row] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * LN2;
}

// dq, and ref and delta for the kernel of dk and dv.
template <typename T, int DH, bool WIDE>
__global__ __launch_bounds__(256) void packed_attention_dq_kernel(AttnArgs a) {
  using K = Kernel<T, DH, WIDE>;
  using O = Op<T>;
  using L = Tile<T, DH>;
  constexpr int KS = K::KS, PS = K::PS, DB = K::DB, NB = K::NB;
  __shared__ __attribute__((aligned(16))) char lds[2 * L::BYTES];
  OwnRows place;
  if (!own_place(a, a.s.q_off, a.s.q_tokens, a.s.n_heads, K::OWN, &place)) return;
  const DocSpan span = place.span;
  const int first = place.row, head = place.head, part_of = place.part;
  DocSpan keys = other_rows(a.s.k_off, a.s.n_docs, a.s.k_tokens, span);
  // bf16, documents of one tile of keys: delta from the probabilities (sum of p X), as in the other bf16 form: that from the output carries the output's rounding (documents of 2
  // to 4 keys: dk 0.0035 off the formula instead of 0.0023).
  const bool brief = sizeof(T) == 2 && keys.end - keys.first <= TILE_ROWS;
  take_part(&keys, a.parts, part_of, TILE_ROWS);
  const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kv = head / (a.s.n_heads / a.s.n_kv_heads);
  const int row = first + (WIDE ? wave * 16 : 0) + l16, b0 = WIDE ? 0 : wave;
  const T *k = (const T*)a.k + (size_t)kv * DH, *v = (const T*)a.v + (size_t)kv * DH;
  typename L::Regs nk, nv;
  L::fetch(nk, k, a.s.k_stride, keys.first, keys.end);
  L::fetch(nv, v, a.s.v_stride, keys.first, keys.end);
  typename O::Frag q[KS], dout[KS];
  own_rows<T, DH>(q, (const T*)a.q + (size_t)head * DH, a.s.q_stride, row, span.end);
  own_rows<T, DH>(dout, (const T*)a.dout + (size_t)head * DH, a.s.o_stride, row, span.end);
  float delta = 0.f, ref = INFINITY;  // (a query without keys, or that is not there: probabilities of zero)
  {
    typename O::Frag out[KS];
    own_rows<T, DH>(out, (const T*)a.out + (size_t)head * DH, a.s.o_stride, row, span.end);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int e = 0; e < O::EPL; ++e) delta = fmaf((float)dout[ks][e], (float)out[ks][e], delta);
    delta = quarters_sum(delta);
    if (row < span.end) {
      const size_t at = (size_t)head * a.s.q_tokens + row;
      const float lse = a.lse[at];
      if (lse != -INFINITY) ref = lse * LOG2E;
      if (g == 0 && (WIDE || wave == 0) && part_of == 0) {
        a.ref[at] = ref;
        a.delta[at] = -delta;
      }
    }
  }
  f32x4 dq[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) dq[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float unit = a.scale * LOG2E;
  for (int k0 = keys.first; k0 < keys.end; k0 += TILE_ROWS) {
    __syncthreads();
    L::put(lds, nk);
    L::put(lds + L::BYTES, nv);
    __syncthreads();
    L::fetch(nk, k, a.s.k_stride, k0 + TILE_ROWS, keys.end);
    L::fetch(nv, v, a.s.v_stride, k0 + TILE_ROWS, keys.end);
    f32x4 s[NB], ds[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) s[b] = ds[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        s[b] = O::mma(L::rows(lds, b0 + b, ks), q[ks], s[b]);
        ds[b] = O::mma(L::rows(lds + L::BYTES, b0 + b, ks), dout[ks], ds[b]);
      }
    if (brief) {
      delta = 0.f;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (k0 + (b0 + b) * 16 + 4 * g + r < keys.end) delta = fmaf(__builtin_amdgcn_exp2f(fmaf(s[b][r], unit, -ref)), ds[b][r], delta);
      delta = quarters_sum(delta);
      if (row < span.end && g == 0) a.delta[(size_t)head * a.s.q_tokens + row] = -delta;
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[b][r], unit, -ref));
        ds[b][r] = k0 + (b0 + b) * 16 + 4 * g + r < keys.end ? p * (ds[b][r] - delta) : 0.f;
      }
#pragma unroll
    for (int ks = 0; ks < PS; ++ks) {
      const typename O::Frag f = step_of<T>(ds, ks);
#pragma unroll
      for (int d = 0; d < DB; ++d) dq[d] = O::mma(L::cols(lds, b0 + ks, d), f, dq[d]);
    }
  }
  if (a.parts > 1) {
    float* to = part_row(a.part, part_of, a.s.q_tokens, row, a.s.n_heads, head, DH) + 4 * g;
    joined<DB, WIDE>(lds, dq, [&](int d, f32x4 x) {
      if (row < span.end) *reinterpret_cast<f32x4*>(to + 16 * d) = x;
    });
    return;
  }
  T* to = (T*)a.dq + (size_t)row * a.s.dq_stride + (size_t)head * DH + 4 * g;
  joined<DB, WIDE>(lds, dq, [&](int d, f32x4 x) {
    if (row < span.end) store4(to + 16 * d, x[0] * a.scale, x[1] * a.scale, x[2] * a.scale, x[3] * a.scale);
  });
}

// dk and dv, over the queries of all heads that share the keys.
template <typename T, int DH, bool WIDE>
__global__ __launch_bounds__(256) void packed_attention_dkv_kernel(AttnArgs a) {
  using K = Kernel<T, DH, WIDE>;
  using O = Op<T>;
  using L = Tile<T, DH>;
  constexpr int KS = K::KS, PS = K::PS, DB = K::DB, NB = K::NB;
  __shared__ __attribute__((aligned(16))) char lds[2 * L::BYTES];
  __shared__ __attribute__((aligned(16))) float refs[2 * TILE_ROWS];  // ref (infinite where there is no query), -delta
  OwnRows place;
  if (!own_place(a, a.s.k_off, a.s.k_tokens, a.s.n_kv_heads, K::OWN, &place)) return;
  const DocSpan span = place.span;
  const int first = place.row, kv = place.head, part_of = place.part;
  DocSpan queries = other_rows(a.s.q_off, a.s.n_docs, a.s.q_tokens, span);
  take_part(&queries, a.parts, part_of, TILE_ROWS);
  const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), share = a.s.n_heads / a.s.n_kv_heads;
  const int row = first + (WIDE ? wave * 16 : 0) + l16, b0 = WIDE ? 0 : wave;
  typename L::Regs nq, nd;
  float next_ref = 0.f;
  auto fetch = [&](int head, int q0) {
    L::fetch(nq, (const T*)a.q + (size_t)head * DH, a.s.q_stride, q0, queries.end);
    L::fetch(nd, (const T*)a.dout + (size_t)head * DH, a.s.o_stride, q0, queries.end);
    if (threadIdx.x < 2 * TILE_ROWS) {
      const int i = q0 + (threadIdx.x & (TILE_ROWS - 1));
      next_ref = threadIdx.x < TILE_ROWS ? INFINITY : 0.f;
      if (i < queries.end) next_ref = (threadIdx.x < TILE_ROWS ? a.ref : a.delta)[(size_t)head * a.s.q_tokens + i];
    }
  };
  const bool some = queries.first < queries.end;
  if (some) fetch(kv * share, queries.first);
  typename O::Frag k[KS], v[KS];
  own_rows<T, DH>(k, (const T*)a.k + (size_t)kv * DH, a.s.k_stride, row, span.end);
  own_rows<T, DH>(v, (const T*)a.v + (size_t)kv * DH, a.s.v_stride, row, span.end);
  f32x4 dk[DB], dv[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) dk[d] = dv[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float unit = a.scale * LOG2E;
  int head = kv * share, q0 = queries.first;
  while (some && head < (kv + 1) * share) {
    __syncthreads();
    L::put(lds, nq);
    L::put(lds + L::BYTES, nd);
    if (threadIdx.x < 2 * TILE_ROWS) refs[threadIdx.x] = next_ref;
    __syncthreads();
    const int there = queries.end - q0;  // rows of the tile below the end; those past it (zeros, which an infinite key makes scores of that are not numbers) count as none
    q0 += TILE_ROWS;
    if (q0 >= queries.end) {
      q0 = queries.first;
      ++head;
    }
    if (head < (kv + 1) * share) fetch(head, q0);
    f32x4 p[NB], ds[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) p[b] = ds[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        p[b] = O::mma(L::rows(lds, b0 + b, ks), k[ks], p[b]);
        ds[b] = O::mma(L::rows(lds + L::BYTES, b0 + b, ks), v[ks], ds[b]);
      }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const f32x4 ref = *reinterpret_cast<const f32x4*>(refs + (b0 + b) * 16 + 4 * g), delta = *reinterpret_cast<const f32x4*>(refs + TILE_ROWS + (b0 + b) * 16 + 4 * g);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p[b][r] = __builtin_amdgcn_exp2f(fmaf(p[b][r], unit, -ref[r]));
        ds[b][r] = p[b][r] * (ds[b][r] + delta[r]);
      }
    }
    if (there < TILE_ROWS) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if ((b0 + b) * 16 + 4 * g + r >= there) p[b][r] = ds[b][r] = 0.f;
    }
#pragma unroll
    for (int ks = 0; ks < PS; ++ks) {
      const typename O::Frag pf = step_of<T>(p, ks), df = step_of<T>(ds, ks);
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        dv[d] = O::mma(L::cols(lds + L::BYTES, b0 + ks, d), pf, dv[d]);
        dk[d] = O::mma(L::cols(lds, b0 + ks, d), df, dk[d]);
      }
    }
  }
  if (a.parts > 1) {
    float* pk = part_row(a.part, part_of, a.s.k_tokens, row, a.s.n_kv_heads, kv, DH) + 4 * g;
    float* pv = part_row(a.part2, part_of, a.s.k_tokens, row, a.s.n_kv_heads, kv, DH) + 4 * g;
    joined<DB, WIDE>(lds, dk, [&](int d, f32x4 x) {
      if (row < span.end) *reinterpret_cast<f32x4*>(pk + 16 * d) = x;
    });
    joined<DB, WIDE>(lds, dv, [&](int d, f32x4 x) {
      if (row < span.end) *reinterpret_cast<f32x4*>(pv + 16 * d) = x;
    });
    return;
  }
  T* tk = (T*)a.dk + (size_t)row * a.s.dk_stride + (size_t)kv * DH + 4 * g;
  T* tv = (T*)a.dv + (size_t)row * a.s.dv_stride + (size_t)kv * DH + 4 * g;
  joined<DB, WIDE>(lds, dk, [&](int d, f32x4 x) {
    if (row < span.end) store4(tk + 16 * d, x[0] * a.scale, x[1] * a.scale, x[2] * a.scale, x[3] * a.scale);
  });
  joined<DB, WIDE>(lds, dv, [&](int d, f32x4 x) {
    if (row < span.end) store4(tv + 16 * d, x[0], x[1], x[2], x[3]);
  });
}

// ---- joins of the parts, four channels a thread, in the parts' order
template <typename T>
__global__ __launch_bounds__(256) void packed_join_kernel(const float* __restrict__ part, const float* __restrict__ part2, T* __restrict__ to, T* __restrict__ to2, long long stride,
                                                          long long stride2, int parts, long long quads, int row_quads, float scale, float scale2) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= quads) return;
  const bool second = blockIdx.y == 1;
  const f32x4* p = reinterpret_cast<const f32x4*>(second ? part2 : part) + i;
  f32x4 x = p[0];
#pragma unroll 4
  for (int k = 1; k < parts; ++k) x += p[k * quads];
  x *= second ? scale2 : scale;
  store4((second ? to2 : to) + i / row_quads * (second ? stride2 : stride) + i % row_quads * 4, x[0], x[1], x[2], x[3]);
}

template <typename T>
__global__ __launch_bounds__(256) void packed_join_forward_kernel(AttnArgs a, long long quads) {
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
  if (i >= quads) return;
  const int dq = a.s.head_dim / 4, row_quads = a.s.n_heads * dq, row = (int)(i / row_quads), head = (int)(i % row_quads) / dq;
  const size_t at = (size_t)head * a.s.q_tokens + row, each = (size_t)a.s.n_heads * a.s.q_tokens;
  float most = -INFINITY;
  for (int k = 0; k < a.parts; ++k) most = __builtin_elementwise_maximum(most, a.part_ref[k * each + at]);
  const float ref = most == -INFINITY ? 0.f : most;
  const f32x4* p = reinterpret_cast<const f32x4*>(a.part) + i;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  float sum = 0.f;
#pragma unroll 4
  for (int k = 0; k < a.parts; ++k) {
    const float w = __builtin_amdgcn_exp2f(a.part_ref[k * each + at] - ref);
    x += p[k * quads] * w;
    sum += a.part_sum[k * each + at] * w;
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  store4((T*)a.o + (size_t)row * a.s.o_stride + i % row_quads * 4, x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
  if (i % dq == 0) a.lse[at] = sum == 0.f ? -INFINITY : (most + __builtin_amdgcn_logf(sum)) * LN2;
}

br_status launch_attn_join_forward(const AttnArgs& a, hipStream_t st) {
  const long long quads = (long long)a.s.q_tokens * a.s.n_heads * a.s.head_dim / 4;
  if (a.s.dtype == BR_BF16) hipLaunchKernelGGL(packed_join_forward_kernel<bf16>, dim3(cdiv(quads, 256)), dim3(256), 0, st, a, quads);
  else hipLaunchKernelGGL(packed_join_forward_kernel<float>, dim3(cdiv(quads, 256)), dim3(256), 0, st, a, quads);
  BR_LAUNCH_CHECK();
  return BR_OK;
}
static br_status join(const AttnArgs& a, int tokens, int heads, void* to, void* to2, long long stride, long long stride2, float scale, float scale2, hipStream_t st) {
  const int row_quads = heads * a.s.head_dim / 4;
  const long long quads = (long long)tokens * row_quads;
  const dim3 grid(cdiv(quads, 256), to2 ? 2 : 1);
  if (a.s.dtype == BR_BF16)
    hipLaunchKernelGGL(packed_join_kernel<bf16>, grid, dim3(256), 0, st, a.part, a.part2, (bf16*)to, (bf16*)to2, stride, stride2, a.parts, quads, row_quads, scale, scale2);
  else
    hipLaunchKernelGGL(packed_join_kernel<float>, grid, dim3(256), 0, st, a.part, a.part2, (float*)to, (float*)to2, stride, stride2, a.parts, quads, row_quads, scale, scale2);
  BR_LAUNCH_CHECK();
  return BR_OK;
}
br_status launch_attn_join_dq(const AttnArgs& a, hipStream_t st) { return join(a, a.s.q_tokens, a.s.n_heads, a.dq, nullptr, a.s.dq_stride, 0, a.scale, 1.f, st); }
br_status launch_attn_join_dkv(const AttnArgs& a, hipStream_t st) { return join(a, a.s.k_tokens, a.s.n_kv_heads, a.dk, a.dv, a.s.dk_stride, a.s.dv_stride, a.scale, 1.f, st); }

static AttnArgs attn_args(const br_attn_shape& s) {
  AttnArgs a{};
  a.s = s;
  a.scale = s.scale > 0.f ? s.scale : (float)(1.0 / sqrt((double)s.head_dim));
  a.parts = 1;
  return a;
}

// fp32: 64 own rows a workgroup where that gives one workgroup a compute unit (backward: two), else 16.  us with 64 / 16, heads of 64: forward 7200 own rows over all
// heads 16.4 / 14.1, 17 600 32.1 / 32.8, 35 200 44.3 / 51.2; backward 17 600 94.5 / 84.9, 35 200 137 / 138, 70 400 224 / 253; heads of 128 the same way.
static bool attn_f32_wide(long long rows_heads, bool backward) { return rows_heads >= (backward ? 2LL : 1LL) * 64 * device_cu_count(); }

// Parts of the launches of a call.
struct AttnPlan {
  int forward, dq, dkv;
};
static AttnPlan attn_plan(const br_attn_shape& s) {
  const int share = s.n_heads / s.n_kv_heads, d = s.head_dim;
  const bool bf = s.dtype == BR_BF16;
  if (bf && !attn_packed_bf16_fits(s)) return {1, 1, 1};
  const long long q = (long long)s.q_tokens * s.n_heads, k = (long long)s.k_tokens * s.n_kv_heads;
  const int own = bf ? PACK_OWN : 16;
  // (time of 32 rows of the other side in a workgroup, us)
  auto queries = [&](bool backward) {
    if (!bf && attn_f32_wide(q, backward)) return 1;
    const float step = bf ? (backward ? 0.4f : 0.3f) + 0.0015f * d : d / (backward ? 70.f : 90.f);
    return attn_parts(s, s.q_tokens, s.n_heads, own, s.k_tokens, 1, bf ? pack_per_cu(d, backward ? 1 : 0) : 2, step, 1);
  };
  const int keys = !bf && attn_f32_wide(k, true) ? 1 : attn_parts(s, s.k_tokens, s.n_kv_heads, own, s.q_tokens, share, bf ? pack_per_cu(d, 2) : 2, bf ? 0.4f + 0.005f * d : d / 50.f, 2);
  return {queries(false), queries(true), keys};
}

// f(T, DH, WIDE)
template <typename F>
static void attn_form(const br_attn_shape& s, bool wide, F f) {
#define BR_D(n) std::integral_constant<int, n>{}
  if (s.dtype == BR_BF16) {
    if (s.head_dim == 64) f(bf16{}, BR_D(64), std::true_type{});
    else f(bf16{}, BR_D(128), std::true_type{});
    return;
  }
  auto with = [&](auto D) {
    if (wide) f(float{}, D, std::true_type{});
    else f(float{}, D, std::false_type{});
  };
  if (s.head_dim == 16) with(BR_D(16));
  else if (s.head_dim == 32) with(BR_D(32));
  else if (s.head_dim == 64) with(BR_D(64));
  else with(BR_D(128));
#undef BR_D
}

// Workspace: ref and delta of the backward pass, then what the parts of one launch leave.
static size_t attn_rows_bytes(const br_attn_shape& s) { return align_up((size_t)s.n_heads * s.q_tokens * 4, 256); }
size_t attn_train_workspace(const br_attn_shape& s, bool backward) {
  const AttnPlan p = attn_plan(s);
  const size_t q = align_up((size_t)s.q_tokens * s.n_heads * s.head_dim * 4, 256), k = align_up((size_t)s.k_tokens * s.n_kv_heads * s.head_dim * 4, 256);
  if (!backward) return p.forward > 1 ? p.forward * (q + 2 * attn_rows_bytes(s)) : 0;
  return 2 * attn_rows_bytes(s) + std::max(p.dq > 1 ? p.dq * q : 0, p.dkv > 1 ? 2 * p.dkv * k : 0);
}

br_status launch_attn_train_forward(const br_attn_shape& s, const void* q, const void* k, const void* v, void* out, float* lse, void* ws, hipStream_t st) {
  AttnArgs a = attn_args(s);
  const AttnPlan plan = attn_plan(s);
  a.q = q;
  a.k = k;
  a.v = v;
  a.o = out;
  a.lse = lse;
  a.part = reinterpret_cast<float*>(ws);
  a.part_ref = a.part + (size_t)plan.forward * s.q_tokens * s.n_heads * s.head_dim;
  a.part_sum = a.part_ref + (size_t)plan.forward * s.q_tokens * s.n_heads;
  if (attn_packed_bf16_fits(s)) return launch_attn_forward_bf16(a, plan.forward, st);
  br_status ok = BR_OK;
  attn_form(s, attn_f32_wide((long long)s.q_tokens * s.n_heads, false), [&](auto Tc, auto Dc, auto Wc) {
    using T = decltype(Tc);
    constexpr int DH = decltype(Dc)::value;
    constexpr bool WIDE = decltype(Wc)::value;
    unsigned n;
    if ((ok = attn_grid(a, s.q_tokens, s.n_heads, Kernel<T, DH, WIDE>::OWN, plan.forward, 0, &n)) != BR_OK) return;
    hipLaunchKernelGGL((packed_attention_kernel<T, DH, WIDE>), dim3(n), dim3(256), 0, st, a);
  });
  if (ok != BR_OK) return ok;
  BR_LAUNCH_CHECK();
  return plan.forward > 1 ? launch_attn_join_forward(a, st) : BR_OK;
}

br_status launch_attn_train_backward(const br_attn_shape& s, const void* dout, const void* q, const void* k, const void* v, const void* out, const float* lse, void* dq, void* dk,
                                     void* dv, void* ws, hipStream_t st) {
  AttnArgs a = attn_args(s);
  const AttnPlan plan = attn_plan(s);
  a.q = q;
  a.k = k;
  a.v = v;
  a.out = out;
  a.dout = dout;
  a.lse = const_cast<float*>(lse);
  char* w = reinterpret_cast<char*>(ws);
  a.ref = reinterpret_cast<float*>(w);
  a.delta = reinterpret_cast<float*>(w + attn_rows_bytes(s));
  a.part = reinterpret_cast<float*>(w + 2 * attn_rows_bytes(s));
  a.part2 = a.part + (size_t)plan.dkv * s.k_tokens * s.n_kv_heads * s.head_dim;
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  if (attn_packed_bf16_fits(s)) return launch_attn_grad_bf16(a, plan.dq, plan.dkv, st);
  br_status ok = BR_OK;
  if (s.q_tokens > 0) {
    attn_form(s, attn_f32_wide((long long)s.q_tokens * s.n_heads, true), [&](auto Tc, auto Dc, auto Wc) {
      using T = decltype(Tc);
      constexpr int DH = decltype(Dc)::value;
      constexpr bool WIDE = decltype(Wc)::value;
      unsigned n;
      if ((ok = attn_grid(a, s.q_tokens, s.n_heads, Kernel<T, DH, WIDE>::OWN, plan.dq, 0, &n)) != BR_OK) return;
      hipLaunchKernelGGL((packed_attention_dq_kernel<T, DH, WIDE>), dim3(n), dim3(256), 0, st, a);
    });
    if (ok != BR_OK) return ok;
    BR_LAUNCH_CHECK();
    if (plan.dq > 1 && (ok = launch_attn_join_dq(a, st)) != BR_OK) return ok;
  }
  if (s.k_tokens > 0) {
    attn_form(s, attn_f32_wide((long long)s.k_tokens * s.n_kv_heads, true), [&](auto Tc, auto Dc, auto Wc) {
      using T = decltype(Tc);
      constexpr int DH = decltype(Dc)::value;
      constexpr bool WIDE = decltype(Wc)::value;
      unsigned n;
      if ((ok = attn_grid(a, s.k_tokens, s.n_kv_heads, Kernel<T, DH, WIDE>::OWN, plan.dkv, 0, &n)) != BR_OK) return;
      hipLaunchKernelGGL((packed_attention_dkv_kernel<T, DH, WIDE>), dim3(n), dim3(256), 0, st, a);
    });
    if (ok != BR_OK) return ok;
    BR_LAUNCH_CHECK();
    if (plan.dkv > 1 && (ok = launch_attn_join_dkv(a, st)) != BR_OK) return ok;
  }
  return BR_OK;
}

}  // namespace br
