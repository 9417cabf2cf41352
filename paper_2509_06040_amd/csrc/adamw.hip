// One AdamW step over many tensors (memory-bound): 48 tensors a launch, their pointers in the kernel's arguments, so that a step needs
// no table on the device.  A wavefront takes 256 consecutive elements of a tensor, four a lane: the block of one scale of
// the states in 8 bits, whose largest value is then a maximum over the wavefront.
//
// 240 M parameters with bf16 gradients and copies: states in 32 bits 1150 us, 5.66 TB/s; in 8 bits 650 to 700 us (664 in a long run, 696 in the first passes of one), 5.4 to 5.8 TB/s, and the read-out of their values 411 us, 5.85.
// A step in 8 bits has the chip's VALU nearly full (generator, root, quotient, codes): with scales by four quotients, maxima by way of LDS and codes taken apart with integer
// arithmetic it took 747 to 812.
//
// fp32 quads (parameters, gradients, states) are loaded and stored past the caches, and codes are stored so: nothing here is read twice (states in 32 bits: plain 1223 us, stores past
// the caches 1227, loads too 1151).  bf16 gradients and codes are loaded plainly, bf16 copies, which the network reads next, stored so.
//
// Every product, sum, quotient and root is rounded by itself (no contraction): states in 8 bits are the same bits wherever they are computed.
#include "dit.h"
#include "philox.h"
#include "train.h"

#pragma clang fp contract(off)

namespace br {

constexpr uint32_t TAG_ADAMW = 4;
constexpr int ADAMW_TENSORS = 48, ADAMW_GROUP = 256;
constexpr int ADAMW_EACH = 2;  // groups a wavefront, read before the first is worked on (four 1 to 4 % slower, as one after the other)
constexpr int ADAMW_BLOCK = 4 * ADAMW_EACH * ADAMW_GROUP;

struct AdamwEntry {
  float* p;
  const void* g;
  void *m, *v;
  float *m_scale, *v_scale;
  void* copy;
  long long n;
  float decay;    // 1 - lr weight_decay
  unsigned block0;  // first workgroup
  unsigned index;   // of the tensor
  unsigned wide;    // whole quads are aligned
};
struct AdamwArgs {
  AdamwEntry t[ADAMW_TENSORS];
  int n;
  float b1, c1, b2, c2, eps, rate, root_scale;  // c = 1 - b; rate = lr / (1 - b1^step); root_scale = 1 / sqrt(1 - b2^step)
  unsigned step;
  const float* grad_scale;
  uint64_t seed;
};
static_assert(sizeof(AdamwArgs) <= 4096 - 64, "kernel arguments");

typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef unsigned char u8x4 __attribute__((ext_vector_type(4)));

// A quad of a tensor: elements at .. at + 3, those from n on read as 0 and not written.
template <typename T>
__device__ inline float4 quad_load(const T* p, long long at, long long n, bool wide) {
  if (wide && at + 4 <= n) {
    if constexpr (sizeof(T) == 4) {
      const f32x4_t x = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t*>(p + at));
      return make_float4(x[0], x[1], x[2], x[3]);
    } else {
      const bf16x4 v = *reinterpret_cast<const bf16x4*>(p + at);
      return make_float4((float)v[0], (float)v[1], (float)v[2], (float)v[3]);
    }
  }
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (at < n) v.x = (float)p[at];
  if (at + 1 < n) v.y = (float)p[at + 1];
  if (at + 2 < n) v.z = (float)p[at + 2];
  if (at + 3 < n) v.w = (float)p[at + 3];
  return v;
}
template <typename T>
__device__ inline void quad_store(T* p, long long at, long long n, bool wide, const float4& v) {
  if (wide && at + 4 <= n) {
    if constexpr (sizeof(T) == 4) {
      __builtin_nontemporal_store(f32x4_t{v.x, v.y, v.z, v.w}, reinterpret_cast<f32x4_t*>(p + at));
    } else {
      store4(p + at, v.x, v.y, v.z, v.w);
    }
    return;
  }
  if (at < n) p[at] = (T)v.x;
  if (at + 1 < n) p[at + 1] = (T)v.y;
  if (at + 2 < n) p[at + 2] = (T)v.z;
  if (at + 3 < n) p[at + 3] = (T)v.w;
}
__device__ inline unsigned quad_codes(const unsigned char* p, long long at, long long n, bool wide) {
  if (wide && at + 4 <= n) return *reinterpret_cast<const unsigned*>(p + at);
  unsigned v = 0;
  for (int i = 0; i < 4; ++i)
    if (at + i < n) v |= (unsigned)p[at + i] << (8 * i);
  return v;
}
__device__ inline void quad_codes_store(unsigned char* p, long long at, long long n, bool wide, unsigned v) {
  if (wide && at + 4 <= n) {
    __builtin_nontemporal_store(v, reinterpret_cast<unsigned*>(p + at));
    return;
  }
  for (int i = 0; i < 4; ++i)
    if (at + i < n) p[at + i] = (unsigned char)(v >> (8 * i));
}

// Codes of 4 bits of exponent e and M of mantissa f: f at e = 0, else (f + 2^M) 2^(e - 1).
template <int M>
constexpr float CODE_MOST = (float)(((2 << M) - 1) << 14);
template <int M>
__device__ inline float code_value(unsigned code) {  // without a sign: as e and f stand in fp32, subnormal numbers among them, a power of two below
  return ldexpf(__builtin_bit_cast(float, code << (23 - M)), 126 + M);
}
// The code below y (0 <= y <= CODE_MOST), or the one above it where 16 random bits, as a fraction, reach over.
template <int M>
__device__ inline unsigned code_of(float y, unsigned random16) {
  const int e = max((int)(__builtin_bit_cast(unsigned, y) >> 23) - 127 - M, 0);
  return ((unsigned)e << M) + (unsigned)fmaf((float)random16, 1.f / 65536.f, ldexpf(y, -e));  // (the product is exact)
}

// Scales of a block of m and one of sqrt(v) and the factors that take values to codes.  Lower half of the wavefront: m, upper half: sqrt(v); a quarter then each of the four quotients.
// Magnitudes are compared as numbers' bits, so that one that is not finite is the largest.  Blocks without a value above 2^-96 are held as zeros (their scale would leave fp32).
struct BlockScales {
  float m, v, m_up, v_up;
};
__device__ inline BlockScales block_scales(const float4& m, const float4& v) {
  auto mag = [](float x) { return __builtin_bit_cast(unsigned, x) & 0x7FFFFFFFu; };
  auto four = [&](const float4& x) { return max(max(mag(x.x), mag(x.y)), max(mag(x.z), mag(x.w))); };
  auto p = __builtin_amdgcn_permlane32_swap(four(m), four(v), false, false);
  unsigned t = max((unsigned)p[0], (unsigned)p[1]);
  p = __builtin_amdgcn_permlane16_swap(t, t, false, false);
  t = max((unsigned)p[0], (unsigned)p[1]);
  auto with = [&](auto CTRL) { t = max(t, (unsigned)__builtin_amdgcn_update_dpp(0, (int)t, decltype(CTRL)::value, 0xf, 0xf, true)); };
  with(std::integral_constant<int, 0x128>{});  // row_ror:8
  with(std::integral_constant<int, 0x124>{});  // row_ror:4
  with(std::integral_constant<int, 0x4E>{});   // quad_perm [2,3,0,1]
  with(std::integral_constant<int, 0xB1>{});   // quad_perm [1,0,3,2]
  const int lane = threadIdx.x & 63;
  const float top = __builtin_bit_cast(float, t), most = lane & 32 ? CODE_MOST<4> : CODE_MOST<3>;
  const bool fine = top < INFINITY, some = top > 1.2621774e-29f, up = lane & 16;
  const float q = (up ? most : top) / (up ? top : most), r = fine ? (some ? q : 0.f) : up ? 0.f : __builtin_nanf("");
  auto of = [&](int l) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, r), l)); };
  return {of(0), of(32), of(16), of(48)};
}

// What a lane reads of a group: a quad of each tensor, as it lies in memory.
template <int BITS>
struct AdamwQuad {
  float4 p, g, m, v;
  unsigned cm, cv;
  float sm, sv;
};

template <typename G, int BITS>
__global__ __launch_bounds__(256) void adamw_kernel(AdamwArgs a) {
  int lo = 0, hi = a.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.t[mid].block0 <= blockIdx.x) lo = mid;
    else hi = mid;
  }
  const AdamwEntry& t = a.t[lo];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long n = t.n, base = (long long)(blockIdx.x - t.block0) * ADAMW_BLOCK + wave * (ADAMW_EACH * ADAMW_GROUP);
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  PhiloxKey key;
  if constexpr (BITS == 8) key = philox_key(a.seed);
  auto load = [&](AdamwQuad<BITS>& q, long long first, bool wide) __attribute__((always_inline)) {
    const long long at = first + lane * 4;
    q.p = quad_load(t.p, at, n, wide);
    q.g = quad_load(reinterpret_cast<const G*>(t.g), at, n, wide);
    if constexpr (BITS == 32) {
      q.m = quad_load(reinterpret_cast<const float*>(t.m), at, n, wide);
      q.v = quad_load(reinterpret_cast<const float*>(t.v), at, n, wide);
    } else {
      q.cm = quad_codes(reinterpret_cast<const unsigned char*>(t.m), at, n, wide);
      q.cv = quad_codes(reinterpret_cast<const unsigned char*>(t.v), at, n, wide);
      q.sm = t.m_scale[first / ADAMW_GROUP];
      q.sv = t.v_scale[first / ADAMW_GROUP];
    }
  };
  auto update = [&](AdamwQuad<BITS>& q, long long first, bool wide) __attribute__((always_inline)) {
    const long long at = first + lane * 4;
    if constexpr (BITS == 8) {
      auto mom = [&](int i) { const unsigned c = q.cm >> (8 * i) & 255; const float x = code_value<3>(c & 127); return (c & 128 ? -x : x) * q.sm; };
      auto sec = [&](int i) { const float x = code_value<4>(q.cv >> (8 * i) & 255) * q.sv; return x * x; };
      q.m = make_float4(mom(0), mom(1), mom(2), mom(3));
      q.v = make_float4(sec(0), sec(1), sec(2), sec(3));
    }
    float4 root;
    auto one = [&](float& pp, float gg, float& mm, float& vv, float& rr) {
      if (a.grad_scale) gg = gg * gs;
      mm = mm * a.b1 + gg * a.c1;
      vv = vv * a.b2 + (gg * a.c2) * gg;
      rr = sqrtf(vv);
      pp = pp * t.decay - (mm / (rr * a.root_scale + a.eps)) * a.rate;
    };
    one(q.p.x, q.g.x, q.m.x, q.v.x, root.x);
    one(q.p.y, q.g.y, q.m.y, q.v.y, root.y);
    one(q.p.z, q.g.z, q.m.z, q.v.z, root.z);
    one(q.p.w, q.g.w, q.m.w, q.v.w, root.w);
    if constexpr (BITS == 32) {
      quad_store(reinterpret_cast<float*>(t.m), at, n, wide, q.m);
      quad_store(reinterpret_cast<float*>(t.v), at, n, wide, q.v);
    } else {
      if (at >= n) q.m = root = make_float4(0.f, 0.f, 0.f, 0.f);  // (with eps = 0 a quotient of zeros; the states of what is not there are 0 as they are)
      const BlockScales scales = block_scales(q.m, root);
      uint32_t w[4];
      philox4x32_10(key, (uint32_t)(at >> 2), t.index, a.step, TAG_ADAMW, w);
      unsigned cm = 0, cv = 0;
      auto pack = [&](int i, float mm, float rr) {
        const unsigned c = code_of<3>(fminf(fabsf(mm) * scales.m_up, CODE_MOST<3>), w[i] & 0xFFFF) | (mm < 0.f ? 128u : 0u);
        cm |= c << (8 * i);
        cv |= code_of<4>(fminf(rr * scales.v_up, CODE_MOST<4>), w[i] >> 16) << (8 * i);
      };
      pack(0, q.m.x, root.x);
      pack(1, q.m.y, root.y);
      pack(2, q.m.z, root.z);
      pack(3, q.m.w, root.w);
      quad_codes_store(reinterpret_cast<unsigned char*>(t.m), at, n, wide, cm);
      quad_codes_store(reinterpret_cast<unsigned char*>(t.v), at, n, wide, cv);
      if (lane == 0) {
        t.m_scale[first / ADAMW_GROUP] = scales.m;
        t.v_scale[first / ADAMW_GROUP] = scales.v;
      }
    }
    quad_store(t.p, at, n, wide, q.p);
    if (t.copy) quad_store(reinterpret_cast<bf16*>(t.copy), at, n, wide, q.p);
  };
  if (t.wide && base + ADAMW_EACH * ADAMW_GROUP <= n) {  // all of them read first
    AdamwQuad<BITS> q[ADAMW_EACH];
#pragma unroll
    for (int k = 0; k < ADAMW_EACH; ++k) load(q[k], base + k * ADAMW_GROUP, true);
#pragma unroll
    for (int k = 0; k < ADAMW_EACH; ++k) update(q[k], base + k * ADAMW_GROUP, true);
  } else {
    for (int k = 0; k < ADAMW_EACH && base + k * ADAMW_GROUP < n; ++k) {
      AdamwQuad<BITS> q;
      load(q, base + k * ADAMW_GROUP, t.wide);
      update(q, base + k * ADAMW_GROUP, t.wide);
    }
  }
}

__global__ __launch_bounds__(256) void adamw_values_kernel(AdamwArgs a) {  // p: values of m, copy: values of v (fp32)
  int lo = 0, hi = a.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.t[mid].block0 <= blockIdx.x) lo = mid;
    else hi = mid;
  }
  const AdamwEntry& t = a.t[lo];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long n = t.n, base = (long long)(blockIdx.x - t.block0) * ADAMW_BLOCK + wave * (ADAMW_EACH * ADAMW_GROUP);
  const bool wide = t.wide;
#pragma unroll
  for (int k = 0; k < ADAMW_EACH; ++k) {
    const long long first = base + k * ADAMW_GROUP, at = first + lane * 4;
    if (first >= n) break;
    const unsigned cm = quad_codes(reinterpret_cast<const unsigned char*>(t.m), at, n, wide), cv = quad_codes(reinterpret_cast<const unsigned char*>(t.v), at, n, wide);
    const float sm = t.m_scale[first / ADAMW_GROUP], sv = t.v_scale[first / ADAMW_GROUP];
    auto mom = [&](int i) { const unsigned c = cm >> (8 * i) & 255; const float x = code_value<3>(c & 127); return (c & 128 ? -x : x) * sm; };
    auto sec = [&](int i) { const float x = code_value<4>(cv >> (8 * i) & 255) * sv; return x * x; };
    quad_store(t.p, at, n, wide, make_float4(mom(0), mom(1), mom(2), mom(3)));
    quad_store(reinterpret_cast<float*>(t.copy), at, n, wide, make_float4(sec(0), sec(1), sec(2), sec(3)));
  }
}

// Launches of up to ADAMW_TENSORS tensors with elements; fill(entry, tensor number).
template <typename FILL, typename LAUNCH>
static br_status adamw_launches(AdamwArgs& a, const br_adamw_tensor* t, int n, FILL fill, LAUNCH launch) {
  for (int i = 0; i < n;) {
    long long blocks = 0;
    a.n = 0;
    for (; i < n && a.n < ADAMW_TENSORS; ++i) {
      if (t[i].n == 0) continue;
      const long long more = (t[i].n + ADAMW_BLOCK - 1) / ADAMW_BLOCK;
      if (blocks + more > 0x7FFFFFFFLL) break;
      AdamwEntry& e = a.t[a.n++];
      e = AdamwEntry{t[i].param, t[i].grad, t[i].m, t[i].v, t[i].m_scale, t[i].v_scale, t[i].copy, t[i].n, 0.f, (unsigned)blocks, (unsigned)i, 0};
      fill(e, i);
      blocks += more;
    }
    if (a.n == 0) continue;
    launch((unsigned)blocks);
    BR_LAUNCH_CHECK();
  }
  return BR_OK;
}

static bool on(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

br_status launch_adamw(const br_adamw_cfg& c, const br_adamw_tensor* t, int n, hipStream_t st) {
  AdamwArgs a;
  a.b1 = (float)c.beta1;
  a.c1 = (float)(1.0 - c.beta1);
  a.b2 = (float)c.beta2;
  a.c2 = (float)(1.0 - c.beta2);
  a.eps = (float)c.eps;
  a.rate = (float)(c.lr / (1.0 - pow(c.beta1, (double)c.step)));
  a.root_scale = (float)(1.0 / sqrt(1.0 - pow(c.beta2, (double)c.step)));
  a.step = (unsigned)c.step;
  a.grad_scale = c.grad_scale;
  a.seed = c.seed;
  const uintptr_t g = c.grad_dtype == BR_F32 ? 16 : 8, s = c.state_bits == 32 ? 16 : 4;
  return adamw_launches(
      a, t, n,
      [&](AdamwEntry& e, int i) {
        e.decay = (float)(1.0 - c.lr * t[i].weight_decay);
        e.wide = on(e.p, 16) && on(e.g, g) && on(e.m, s) && on(e.v, s) && on(e.copy, 8);
      },
      [&](unsigned blocks) {
        if (c.state_bits == 32) {
          if (c.grad_dtype == BR_F32) hipLaunchKernelGGL((adamw_kernel<float, 32>), dim3(blocks), dim3(256), 0, st, a);
          else hipLaunchKernelGGL((adamw_kernel<bf16, 32>), dim3(blocks), dim3(256), 0, st, a);
        } else {
          if (c.grad_dtype == BR_F32) hipLaunchKernelGGL((adamw_kernel<float, 8>), dim3(blocks), dim3(256), 0, st, a);
          else hipLaunchKernelGGL((adamw_kernel<bf16, 8>), dim3(blocks), dim3(256), 0, st, a);
        }
      });
}

br_status launch_adamw_values(const br_adamw_tensor* t, int n, float* const* m, float* const* v, hipStream_t st) {
  AdamwArgs a{};
  return adamw_launches(
      a, t, n,
      [&](AdamwEntry& e, int i) {
        e.p = m[i];
        e.copy = v[i];
        e.wide = on(e.p, 16) && on(e.copy, 16) && on(e.m, 4) && on(e.v, 4);
      },
      [&](unsigned blocks) { hipLaunchKernelGGL(adamw_values_kernel, dim3(blocks), dim3(256), 0, st, a); });
}

}  // namespace br
