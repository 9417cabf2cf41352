// The clipped objective over kept edges and its gradient with respect to the velocities (memory-bound).
//   mu_r = a_z z_parent + a_v v_r,  logp_e = c0 - h |z_e - mu_r|^2,  rho_e = exp(logp_e - logp_old_e)
//   d(-J)/dv_r = sum_e w_e (z_e - mu_r),  w_e = -rho_e A_e / n * 2 h a_v, 0 where the clipped term is the smaller one
// Two launches: squares of the differences by slices of a latent, then, once every slice is known, the gradient.  The second reads again what the
// first read, for edges that are not clipped; up to 256 MB of it comes out of the memory-side cache.
// Measured: four trees of 16 leaves, latents of 65 536, half of the edges kept: 40 us for the squares (172 MB, 4.3 TB/s), 27 for the gradient (169 MB, 6.2 TB/s).  One launch whose
// last slice of a row goes on to the gradient: 110 us, its workgroups' round trips follow one another.
#include "dispatch.h"
#include "dit.h"
#include "train.h"

namespace br {

constexpr int OBJ_THREADS = 256;

__device__ inline double wave_sum_d(double x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d, 64);
  return x;
}

struct ObjRow {
  float a_z, a_v;
  double h, c0;
  const float *z, *v;
  int e0, e1;
};
__device__ inline int in_range(int i, int n) { return min(max(i, 0), n - 1); }
__device__ inline ObjRow obj_row(const br_edge_set& s, const float* z, const float* v, int r) {
  ObjRow o;
  o.a_z = (float)s.row_coef[4 * (size_t)r];
  o.a_v = (float)s.row_coef[4 * (size_t)r + 1];
  o.h = s.row_coef[4 * (size_t)r + 2];
  o.c0 = s.row_coef[4 * (size_t)r + 3];
  o.z = z + (size_t)in_range(s.row_parent[r], s.n_nodes) * s.D;
  o.v = v + (size_t)r * s.D;
  o.e0 = min(max(s.row_first[r], 0), s.n_edges);
  o.e1 = min(max(s.row_first[r + 1], o.e0), s.n_edges);
  return o;
}
__device__ inline float4 obj_mean(const ObjRow& o, long long at) {
  const float4 a = *reinterpret_cast<const float4*>(o.z + at), b = *reinterpret_cast<const float4*>(o.v + at);
  return make_float4(fmaf(o.a_z, a.x, o.a_v * b.x), fmaf(o.a_z, a.y, o.a_v * b.y), fmaf(o.a_z, a.z, o.a_v * b.z), fmaf(o.a_z, a.w, o.a_v * b.w));
}

__device__ inline float obj_square(const float4& x, const float4& m) {
  const float a = x.x - m.x, b = x.y - m.y, c = x.z - m.z, d = x.w - m.w;
  return fmaf(a, a, b * b) + fmaf(c, c, d * d);
}
__device__ inline void add_weighted(float4& g, float w, const float4& x, const float4& m) {
  g.x = fmaf(w, x.x - m.x, g.x);
  g.y = fmaf(w, x.y - m.y, g.y);
  g.z = fmaf(w, x.z - m.z, g.z);
  g.w = fmaf(w, x.w - m.w, g.w);
}
// The row that holds edge e: row_first[row] <= e < row_first[row + 1].
__device__ inline int obj_row_of(const br_edge_set& s, int e) {
  int lo = 0, hi = s.n_rows;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (s.row_first[mid] <= e) lo = mid;
    else hi = mid;
  }
  return lo;
}

// part[e * slices + slice] = sum over the slice of (z_e - mu)^2
template <int Q>
__global__ __launch_bounds__(OBJ_THREADS) void objective_squares_kernel(br_edge_set s, int slices, const float* __restrict__ z, const float* __restrict__ v, double* __restrict__ part) {
  __shared__ double red[4];
  const int r = blockIdx.x / slices, slice = blockIdx.x - r * slices;
  const ObjRow o = obj_row(s, z, v, r);
  const long long base = (long long)slice * (OBJ_THREADS * 4 * Q) + threadIdx.x * 4;
  float4 m[Q];
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const long long at = base + q * (OBJ_THREADS * 4);
    m[q] = at < s.D ? obj_mean(o, at) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  for (int e = o.e0; e < o.e1; ++e) {
    const float* c = z + (size_t)in_range(s.edge_ids[e], s.n_nodes) * s.D;
    float4 x[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const long long at = base + q * (OBJ_THREADS * 4);
      x[q] = at < s.D ? *reinterpret_cast<const float4*>(c + at) : m[q];
    }
    float acc = 0.f;
#pragma unroll
    for (int q = 0; q < Q; ++q) acc += obj_square(x[q], m[q]);
    const double w = wave_sum_d((double)acc);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = w;
    __syncthreads();
    if (threadIdx.x == 0) part[(size_t)e * slices + slice] = (red[0] + red[1]) + (red[2] + red[3]);
  }
}

struct ObjTerm {
  double logp, term, weight;  // weight: of dlogp in d(-J)
  bool clipped;
};
__device__ inline ObjTerm obj_term(const br_edge_set& s, double squares, double h, double c0, float logp_old, float adv, double inv_n) {
  ObjTerm t;
  t.logp = c0 - h * squares;
  const double rho = exp(t.logp - (double)logp_old), a = adv, eps = s.clip_eps;
  const double term = rho * a, held = fmin(fmax(rho, 1.0 - eps), 1.0 + eps) * a;
  t.clipped = held < term;
  t.term = (t.clipped ? held : term) * inv_n;  // (not their minimum, which drops a term that is not a number)
  t.weight = t.clipped ? 0.0 : -term * inv_n;
  return t;
}

__device__ inline float obj_weight(const ObjTerm& t, const ObjRow& o) { return (float)(t.weight * 2.0 * o.h * (double)o.a_v); }

// Workgroup 0: J and the log-densities, an edge a thread.  The others: a slice of a row's gradient.
template <int Q>
__global__ __launch_bounds__(OBJ_THREADS) void objective_grad_kernel(br_edge_set s, int slices, double inv_n, const float* __restrict__ z, const float* __restrict__ v,
                                                                     const float* __restrict__ logp_old, const float* __restrict__ adv, const double* __restrict__ part,
                                                                     float* __restrict__ J, float* __restrict__ logp_new, float* __restrict__ grad, unsigned char* __restrict__ clipped) {
  if (blockIdx.x == 0) {
    __shared__ double red[4];
    double sum = 0.0;
    for (int e = threadIdx.x; e < s.n_edges; e += OBJ_THREADS) {
      const int lo = obj_row_of(s, e);
      double sq = 0.0;
#pragma unroll 8
      for (int i = 0; i < slices; ++i) sq += part[(size_t)e * slices + i];
      const int node = in_range(s.edge_ids[e], s.n_nodes);
      const ObjTerm t = obj_term(s, sq, s.row_coef[4 * (size_t)lo + 2], s.row_coef[4 * (size_t)lo + 3], logp_old[node], adv[node], inv_n);
      sum += t.term;
      logp_new[e] = (float)t.logp;
      if (clipped) clipped[e] = t.clipped;
    }
    sum = wave_sum_d(sum);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) J[0] = (float)((red[0] + red[1]) + (red[2] + red[3]));
    return;
  }
  const int block = blockIdx.x - 1, r = block / slices, slice = block - r * slices;
  const ObjRow o = obj_row(s, z, v, r);
  const long long base = (long long)slice * (OBJ_THREADS * 4 * Q) + threadIdx.x * 4;
  float4 m[Q], g[Q];
#pragma unroll
  for (int q = 0; q < Q; ++q) m[q] = g[q] = make_float4(0.f, 0.f, 0.f, 0.f);
  bool have = false;  // the mean: read for the first edge that counts (a row whose edges are all clipped reads nothing)
  for (int e = o.e0; e < o.e1; ++e) {
    double sq = 0.0;
    for (int i = 0; i < slices; ++i) sq += part[(size_t)e * slices + i];  // (the same order as above: the same rho)
    const int node = in_range(s.edge_ids[e], s.n_nodes);
    const ObjTerm t = obj_term(s, sq, o.h, o.c0, logp_old[node], adv[node], inv_n);
    if (t.weight == 0.0) continue;
    const float w = obj_weight(t, o);
    const float* c = z + (size_t)node * s.D;
    float4 x[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const long long at = base + q * (OBJ_THREADS * 4);
      x[q] = at < s.D ? *reinterpret_cast<const float4*>(c + at) : make_float4(0.f, 0.f, 0.f, 0.f);
      if (!have && at < s.D) m[q] = obj_mean(o, at);
    }
    have = true;
#pragma unroll
    for (int q = 0; q < Q; ++q) add_weighted(g[q], w, x[q], m[q]);
  }
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const long long at = base + q * (OBJ_THREADS * 4);
    if (at < s.D) *reinterpret_cast<float4*>(grad + (size_t)r * s.D + at) = g[q];
  }
}

// Small sets (rule::objective_one_launch) in one launch of one workgroup, an edge, then a row, a wavefront at a time.
__global__ __launch_bounds__(1024) void objective_small_kernel(br_edge_set s, double inv_n, const float* __restrict__ z, const float* __restrict__ v,
                                                               const float* __restrict__ logp_old, const float* __restrict__ adv, float* __restrict__ J, float* __restrict__ logp_new,
                                                               float* __restrict__ grad, unsigned char* __restrict__ clipped) {
  __shared__ double squares[rule::OBJECTIVE_SMALL_EDGES], red[16];
  __shared__ float weight[rule::OBJECTIVE_SMALL_EDGES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int e = wave; e < s.n_edges; e += 16) {
    const ObjRow o = obj_row(s, z, v, obj_row_of(s, e));
    const float* c = z + (size_t)in_range(s.edge_ids[e], s.n_nodes) * s.D;
    double acc = 0.0;
    for (long long at = lane * 4; at < s.D; at += 256) acc += obj_square(*reinterpret_cast<const float4*>(c + at), obj_mean(o, at));
    acc = wave_sum_d(acc);
    if (lane == 0) squares[e] = acc;
  }
  __syncthreads();
  double sum = 0.0;
  for (int e = threadIdx.x; e < s.n_edges; e += 1024) {
    const ObjRow o = obj_row(s, z, v, obj_row_of(s, e));
    const int node = in_range(s.edge_ids[e], s.n_nodes);
    const ObjTerm t = obj_term(s, squares[e], o.h, o.c0, logp_old[node], adv[node], inv_n);
    sum += t.term;
    weight[e] = obj_weight(t, o);
    logp_new[e] = (float)t.logp;
    if (clipped) clipped[e] = t.clipped;
  }
  sum = wave_sum_d(sum);
  if (lane == 0) red[wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int k = 1; k < 16; ++k) sum += red[k];
    J[0] = (float)sum;
  }
  for (int r = wave; r < s.n_rows; r += 16) {
    const ObjRow o = obj_row(s, z, v, r);
    for (long long at = lane * 4; at < s.D; at += 256) {
      const float4 m = obj_mean(o, at);
      float4 g = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int e = o.e0; e < o.e1; ++e)
        if (weight[e] != 0.f) add_weighted(g, weight[e], *reinterpret_cast<const float4*>(z + (size_t)in_range(s.edge_ids[e], s.n_nodes) * s.D + at), m);
      *reinterpret_cast<float4*>(grad + (size_t)r * s.D + at) = g;
    }
  }
}

// Quads a thread: four, where that leaves two workgroups a compute unit, else one.
static int obj_quads(const br_edge_set& e) { return (long long)e.n_rows * cdiv(e.D, OBJ_THREADS * 16) >= 2LL * device_cu_count() ? 4 : 1; }
static int obj_slices(const br_edge_set& e) { return cdiv(e.D, OBJ_THREADS * 4LL * obj_quads(e)); }

size_t objective_grad_workspace(const br_edge_set& e) { return std::max<size_t>(256, (size_t)e.n_edges * obj_slices(e) * 8); }

br_status launch_objective_grad(const br_edge_set& e, const float* z, const float* v, const float* logp_old, const float* adv, float* J, float* logp_new, float* grad,
                                unsigned char* clipped, void* ws, hipStream_t st) {
  const int slices = obj_slices(e);
  const long long n = (long long)e.n_rows * slices;
  BR_REQUIRE(n < 0x7FFFFFFFLL, BR_ESHAPE, "br_grpo_backward: too many rows for one launch");
  const double inv_n = 1.0 / (double)(e.n_total > 0 ? e.n_total : e.n_edges);
  double* part = reinterpret_cast<double*>(ws);
  if (rule::objective_one_launch(e.n_edges, e.D)) {
    hipLaunchKernelGGL(objective_small_kernel, dim3(1), dim3(1024), 0, st, e, inv_n, z, v, logp_old, adv, J, logp_new, grad, clipped);
    BR_LAUNCH_CHECK();
    return BR_OK;
  }
  auto run = [&](auto Qc) {
    constexpr int Q = decltype(Qc)::value;
    hipLaunchKernelGGL(objective_squares_kernel<Q>, dim3((unsigned)n), dim3(OBJ_THREADS), 0, st, e, slices, z, v, part);
    hipLaunchKernelGGL(objective_grad_kernel<Q>, dim3((unsigned)n + 1), dim3(OBJ_THREADS), 0, st, e, slices, inv_n, z, v, logp_old, adv, part, J, logp_new, grad, clipped);
  };
  if (obj_quads(e) == 4) run(std::integral_constant<int, 4>{});
  else run(std::integral_constant<int, 1>{});
  BR_LAUNCH_CHECK();
  return BR_OK;
}

}  // namespace br
