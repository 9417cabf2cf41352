// Forward and backward pass of the modulated LayerNorm over packed documents (memory-bound).
//   y = (x - mean) rstd,  out = y (1 + scale) + shift
//   dx = residual + rstd (g - mean(g) - y mean(g y)),  g = dout (1 + scale);  dshift = sum of dout, dscale = sum of dout y
//
// A row lies in the registers of TPR threads (a wavefront up to 2048 columns, a workgroup of 256 above), in VPL pieces of four columns a
// thread.  Statistics are taken in two passes over these registers, as the network's LayerNorm takes them.
//
// Every matrix is read or written once.  Measured: forward, 17 000 rows of 1024, bf16 out, 23 us, 4.5 TB/s; backward, 33 000 rows of 1536, fp32 residual and bf16 dout, 156 us,
// 4.5 TB/s (a copy of 4 GB: 4.75), 6.6 us of them the launch that joins the tiles' column sums.
#include "dit.h"
#include "docs.h"
#include "train.h"

namespace br {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

template <typename T>
__device__ inline float4 load4(const T* p) {
  if constexpr (sizeof(T) == 4) {
    return *reinterpret_cast<const float4*>(p);
  } else {
    const bf16x4 v = *reinterpret_cast<const bf16x4*>(p);
    return make_float4((float)v[0], (float)v[1], (float)v[2], (float)v[3]);
  }
}

// Sums of two values over the threads of a row.  `red`: 2 x 8 floats of LDS, used in turn (`turn`).
template <int TPR>
__device__ inline void row_sums(float* a, float* b, float* red, int turn) {
  *a = lanes_sum<64>(*a);
  *b = lanes_sum<64>(*b);
  if constexpr (TPR > 64) {
    float* r = red + (turn & 1) * 8;
    if ((threadIdx.x & 63) == 0) {
      r[threadIdx.x >> 6] = *a;
      r[4 + (threadIdx.x >> 6)] = *b;
    }
    __syncthreads();
    *a = (r[0] + r[1]) + (r[2] + r[3]);
    *b = (r[4] + r[5]) + (r[6] + r[7]);
  }
}

// Group of the document that holds `row` (-1: none), and the first row behind that document.
__device__ inline int row_group(const br_norm_shape& s, int row, int* end) {
  const int before = leading(s.n_docs + 1, [&](int i) { return s.row_off[i] <= row; });  // offsets up to `row`
  const int next = before <= s.n_docs ? s.row_off[before] : s.rows;
  *end = min(max(next, row + 1), s.rows);
  const int g = before >= 1 && before <= s.n_docs ? s.group[before - 1] : -1;
  return g < s.n_groups ? g : -1;
}

template <typename T, int VPL, int TPR>
__global__ __launch_bounds__(256) void norm_forward_kernel(br_norm_shape s, int rows_each, const float* __restrict__ x, const float* __restrict__ mods, T* __restrict__ out,
                                                           float* __restrict__ mean_out, float* __restrict__ rstd_out) {
  __shared__ float red[16];
  const int tid = threadIdx.x % TPR, H = s.hidden;
  const long long begin = ((long long)blockIdx.x * (256 / TPR) + (TPR == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0)) * rows_each;
  if (begin >= s.rows) return;
  int row = (int)begin;
  const int stop = (int)min<long long>(begin + rows_each, s.rows);
  const float inv_h = 1.f / (float)H;
  auto fetch = [&](int r, float4 (&v)[VPL]) {
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const int c = (i * TPR + tid) * 4;
      v[i] = c < H ? load4(x + (size_t)r * H + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  };
  float4 v[VPL], next[VPL], sc[VPL], sh[VPL];
  fetch(row, v);
  int end = row, group = -1, turn = 0;
  for (; row < stop; ++row) {
    if (row >= end) {
      const int before = group;
      group = row_group(s, row, &end);
      if (group >= 0 && group != before) {
        const float* m = mods + (size_t)group * s.mods_stride;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
          const int c = min((i * TPR + tid) * 4, H - 4);
          sc[i] = load4(m + s.scale_off + c);
          sh[i] = load4(m + s.shift_off + c);
        }
      }
    }
    if (row + 1 < stop) fetch(row + 1, next);
    if (group >= 0) {
      float sum = 0.f, sq = 0.f;
#pragma unroll
      for (int i = 0; i < VPL; ++i) sum += (v[i].x + v[i].y) + (v[i].z + v[i].w);
      row_sums<TPR>(&sum, &sq, red, turn++);
      const float mean = sum * inv_h;
#pragma unroll
      for (int i = 0; i < VPL; ++i)
        if ((i * TPR + tid) * 4 < H) sq += sum_sq4(v[i], mean);
      sum = 0.f;
      row_sums<TPR>(&sq, &sum, red, turn++);
      const float rstd = 1.f / sqrtf(sq * inv_h + 1e-6f);
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        const int c = (i * TPR + tid) * 4;
        if (c < H)
          store4(out + (size_t)row * H + c, fmaf((v[i].x - mean) * rstd, 1.f + sc[i].x, sh[i].x), fmaf((v[i].y - mean) * rstd, 1.f + sc[i].y, sh[i].y),
                 fmaf((v[i].z - mean) * rstd, 1.f + sc[i].z, sh[i].z), fmaf((v[i].w - mean) * rstd, 1.f + sc[i].w, sh[i].w));
      }
      if (tid == 0 && mean_out) {
        mean_out[row] = mean;
        rstd_out[row] = rstd;
      }
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i) v[i] = next[i];
  }
}

// A workgroup takes a tile of consecutive rows of one document, each of its row groups every (256 / TPR)-th of them, and leaves the tile's column sums in
// part[tile][dout | dout y][H] and its group in tile_group[tile].
// Workgroups a compute unit that the registers of the backward pass allow.
template <int VPL, int TPR>
constexpr int NORM_PER_CU = TPR == 64 ? (VPL <= 1 ? 8 : VPL <= 2 ? 5 : VPL <= 3 ? 4 : VPL <= 4 ? 3 : 2) : VPL <= 3 ? 4 : VPL <= 4 ? 3 : 1;

template <typename T, int VPL, int TPR>
__global__ __launch_bounds__(256, (NORM_PER_CU<VPL, TPR>)) void norm_backward_kernel(br_norm_shape s, int tile, const T* __restrict__ dout, const float* __restrict__ x, const float* __restrict__ mean,
                                                            const float* __restrict__ rstd, const float* __restrict__ mods, const float* residual, float* dx,
                                                            float* __restrict__ part, int* __restrict__ tile_group) {
  __shared__ float red[16];
  __shared__ float4 cols[TPR == 64 ? 2 * 256 : 1];
  const int tid = threadIdx.x % TPR, H = s.hidden;
  DocSpan span;
  int row;
  const bool there = doc_tile(s.row_off, s.n_docs, s.rows, tile, blockIdx.x, &span, &row);
  int group = there && span.doc >= 0 ? s.group[span.doc] : -1;
  if (group >= s.n_groups) group = -1;
  if (threadIdx.x == 0) tile_group[blockIdx.x] = group;
  if (group < 0) return;
  const int stop = min(row + tile, span.end);
  const float inv_h = 1.f / (float)H;
  float4 sc[VPL], a[VPL], b[VPL];  // a: sum of dout, b: of dout y
  const float* m = mods + (size_t)group * s.mods_stride + s.scale_off;
#pragma unroll
  for (int i = 0; i < VPL; ++i) {
    const int c = (i * TPR + tid) * 4;
    sc[i] = load4(m + min(c, H - 4));
    a[i] = b[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  int turn = 0;
  for (int r = row + (TPR == 64 ? (int)(threadIdx.x >> 6) : 0); r < stop; r += 256 / TPR) {
    float4 y[VPL], d[VPL], res[VPL];
    const float mu = mean[r], rs = rstd[r];
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const int c = (i * TPR + tid) * 4;
      const size_t at = (size_t)r * H + c;
      y[i] = c < H ? load4(x + at) : make_float4(mu, mu, mu, mu);
      d[i] = c < H ? load4(dout + at) : make_float4(0.f, 0.f, 0.f, 0.f);
      res[i] = residual && c < H ? load4(residual + at) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    float sg = 0.f, sgy = 0.f;
    auto take = [&](float& yy, float& dd, float scale, float& sa, float& sb) {
      yy = (yy - mu) * rs;
      sa += dd;
      sb = fmaf(dd, yy, sb);
      dd *= 1.f + scale;
      sg += dd;
      sgy = fmaf(dd, yy, sgy);
    };
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      take(y[i].x, d[i].x, sc[i].x, a[i].x, b[i].x);
      take(y[i].y, d[i].y, sc[i].y, a[i].y, b[i].y);
      take(y[i].z, d[i].z, sc[i].z, a[i].z, b[i].z);
      take(y[i].w, d[i].w, sc[i].w, a[i].w, b[i].w);
    }
    row_sums<TPR>(&sg, &sgy, red, turn++);
    const float c1 = sg * inv_h, c2 = sgy * inv_h;
    auto give = [&](float yy, float dd, float rr) { return fmaf(rs, dd - c1 - yy * c2, rr); };
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const int c = (i * TPR + tid) * 4;
      if (c < H)
        store4(dx + (size_t)r * H + c, give(y[i].x, d[i].x, res[i].x), give(y[i].y, d[i].y, res[i].y), give(y[i].z, d[i].z, res[i].z), give(y[i].w, d[i].w, res[i].w));
    }
  }
  float* p = part + (size_t)blockIdx.x * 2 * H;
#pragma unroll
  for (int i = 0; i < VPL; ++i) {
    const int c = (i * TPR + tid) * 4;
    if constexpr (TPR == 64) {  // the four wavefronts' sums of the same 256 columns
      cols[threadIdx.x] = a[i];
      cols[256 + threadIdx.x] = b[i];
      __syncthreads();
      if (threadIdx.x < 128 && c < H) {
        const float4* q = cols + (threadIdx.x >> 6) * 256 + tid;
        const float4 u = q[0], v = q[64], w = q[128], z = q[192];
        store4(p + (threadIdx.x >> 6) * H + c, (u.x + v.x) + (w.x + z.x), (u.y + v.y) + (w.y + z.y), (u.z + v.z) + (w.z + z.z), (u.w + v.w) + (w.w + z.w));
      }
      __syncthreads();
    } else if (c < H) {
      store4(p + c, a[i].x, a[i].y, a[i].z, a[i].w);
      store4(p + H + c, b[i].x, b[i].y, b[i].z, b[i].w);
    }
  }
}

// dmods of group blockIdx.y, 64 of the 2 H columns: 64 slices of the tiles, joined in their order.  (6.6 us for 512 tiles of 2 x 1536: the latency of each slice's loads.)
__global__ __launch_bounds__(1024) void norm_columns_kernel(br_norm_shape s, int n_tiles, const float* __restrict__ part, const int* __restrict__ tile_group, float* __restrict__ dmods) {
  __shared__ float4 sums[1024];
  const int H = s.hidden, group = blockIdx.y, c = (blockIdx.x * 16 + (threadIdx.x & 15)) * 4, slice = threadIdx.x >> 4;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  if (c < 2 * H) {
    constexpr int U = 8;
    for (int t0 = slice; t0 < n_tiles; t0 += 64 * U) {
      float4 v[U];
      bool in[U];
#pragma unroll
      for (int u = 0; u < U; ++u) in[u] = t0 + 64 * u < n_tiles && tile_group[min(t0 + 64 * u, n_tiles - 1)] == group;
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = in[u] ? load4(part + (size_t)(t0 + 64 * u) * 2 * H + c) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        acc.x += v[u].x;
        acc.y += v[u].y;
        acc.z += v[u].z;
        acc.w += v[u].w;
      }
    }
  }
  auto add = [](float4& x, const float4& y) {
    x.x += y.x;
    x.y += y.y;
    x.z += y.z;
    x.w += y.w;
  };
  sums[threadIdx.x] = acc;
  __syncthreads();
  if (slice < 8) {
#pragma unroll
    for (int k = 1; k < 8; ++k) add(acc, sums[threadIdx.x + k * 128]);
    sums[threadIdx.x] = acc;
  }
  __syncthreads();
  if (slice == 0 && c < 2 * H) {
#pragma unroll
    for (int k = 1; k < 8; ++k) add(acc, sums[threadIdx.x + k * 16]);
    store4(dmods + (size_t)group * s.mods_stride + (c < H ? s.shift_off + c : s.scale_off + c - H), acc.x, acc.y, acc.z, acc.w);
  }
}

// f(columns a thread in pieces of four, threads a row)
template <typename F>
static void norm_form(int H, F f) {
  auto with = [&](auto V, auto TPR) { f(V, TPR); };
  using W = std::integral_constant<int, 64>;
  using G = std::integral_constant<int, 256>;
#define BR_V(n) std::integral_constant<int, n>{}
  const int w = cdiv(H, 256), g = cdiv(H, 1024);
  if (w <= 1) with(BR_V(1), W{});
  else if (w <= 2) with(BR_V(2), W{});
  else if (w <= 3) with(BR_V(3), W{});
  else if (w <= 4) with(BR_V(4), W{});
  else if (w <= 6) with(BR_V(6), W{});
  else if (w <= 8) with(BR_V(8), W{});
  else if (g <= 3) with(BR_V(3), G{});
  else if (g <= 4) with(BR_V(4), G{});
  else if (g <= 8) with(BR_V(8), G{});
  else with(BR_V(16), G{});
#undef BR_V
}

// Rows of a tile of the backward pass: as many workgroups as the units hold at once, four rows at least, and no more column sums in the workspace than the header says.
static int norm_tile(const br_norm_shape& s) {
  int per_cu = 1;
  norm_form(s.hidden, [&](auto Vc, auto Tc) { per_cu = NORM_PER_CU<decltype(Vc)::value, decltype(Tc)::value>; });
  return std::max({4, cdiv(s.rows, (long long)per_cu * device_cu_count()), cdiv(s.rows, s.rows / 16 + 960)});
}

size_t norm_train_workspace(const br_norm_shape& s) {
  const long long tiles = doc_tiles_most(s.n_docs, s.rows, norm_tile(s));
  return align_up((size_t)tiles * 2 * s.hidden * 4, 256) + (size_t)tiles * 4;
}

br_status launch_norm_forward(const br_norm_shape& s, const float* x, const float* mods, void* out, float* mean, float* rstd, hipStream_t st) {
  norm_form(s.hidden, [&](auto Vc, auto Tc) {
    constexpr int VPL = decltype(Vc)::value, TPR = decltype(Tc)::value, PER = 256 / TPR;
    const int each = std::max(1, std::min(8, cdiv(s.rows, 8LL * PER * device_cu_count())));
    const dim3 g(cdiv(s.rows, (long long)PER * each));
    if (s.dtype == BR_BF16) hipLaunchKernelGGL((norm_forward_kernel<bf16, VPL, TPR>), g, dim3(256), 0, st, s, each, x, mods, (bf16*)out, mean, rstd);
    else hipLaunchKernelGGL((norm_forward_kernel<float, VPL, TPR>), g, dim3(256), 0, st, s, each, x, mods, (float*)out, mean, rstd);
  });
  BR_LAUNCH_CHECK();
  return BR_OK;
}

br_status launch_norm_backward(const br_norm_shape& s, const void* dout, const float* x, const float* mean, const float* rstd, const float* mods, const float* residual, float* dx,
                               float* dmods, void* ws, hipStream_t st) {
  const int tile = norm_tile(s), tiles = (int)doc_tiles_most(s.n_docs, s.rows, tile);
  float* part = reinterpret_cast<float*>(ws);
  int* tile_group = reinterpret_cast<int*>(reinterpret_cast<char*>(ws) + align_up((size_t)tiles * 2 * s.hidden * 4, 256));
  norm_form(s.hidden, [&](auto Vc, auto Tc) {
    constexpr int VPL = decltype(Vc)::value, TPR = decltype(Tc)::value;
    if (s.dtype == BR_BF16)
      hipLaunchKernelGGL((norm_backward_kernel<bf16, VPL, TPR>), dim3(tiles), dim3(256), 0, st, s, tile, (const bf16*)dout, x, mean, rstd, mods, residual, dx, part, tile_group);
    else hipLaunchKernelGGL((norm_backward_kernel<float, VPL, TPR>), dim3(tiles), dim3(256), 0, st, s, tile, (const float*)dout, x, mean, rstd, mods, residual, dx, part, tile_group);
  });
  BR_LAUNCH_CHECK();
  hipLaunchKernelGGL(norm_columns_kernel, dim3(cdiv(2LL * s.hidden, 64), s.n_groups), dim3(1024), 0, st, s, tiles, part, tile_group, dmods);
  BR_LAUNCH_CHECK();
  return BR_OK;
}

}  // namespace br
