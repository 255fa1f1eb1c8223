// qk_norm_rope.cu -- from a {q, k, v} projection's outputs to what the attention
// reads, in one pass: per head of q and k (if asked for) the norm
// y = x / sqrt(mean(x^2) + eps) * w, then the rotation of the pairs (a, b) by the
// token's angle, (a cos - b sin, b cos + a sin); q rounded to 16 bits, k and v
// rounded into the token's slot of the cache.  All arithmetic is in fp32; each
// value is rounded once, when it is stored.
//
// Bound by HBM: an fp32 value is read and a 16-bit one written once (6 bytes a
// value, and the token's cosines and sines).  A head is D / 8 lanes.  A lane has two
// runs of four values, chosen so that both values of every pair are its own: of the
// rotated values run 4l and run rot / 2 + 4l, of the others two that follow one
// another.  So the rotation needs no exchange between lanes, and the norm a sum over
// the head's lanes only.  A warp takes a run of a token's heads, two groups of them at
// a time with the next two's loads in flight, and keeps the token's cosines and sines
// in registers.  8191 tokens of 64 + 16 heads of 128: 90 us, 5.6
// TB/s, 84 % of the copy rate (four lanes' worth of exchange per value and no loads ahead:
// 110 us; more heads at a time: 91 to 104 us).  Of 16-bit inputs 116 us, 2.9 TB/s: a lane
// then loads 8 bytes at a time, and the loads ahead are half as many bytes.
#include <algorithm>

#include "sss_internal.cuh"

namespace sss {
namespace {

constexpr int kThreads = 128;
constexpr int kCtas = 7;    // per SM: 72 registers a thread hold the loads ahead (8 bytes
                            // spill; more CTAs with fewer registers: 91 to 131 us)
constexpr int kUnroll = 2;

struct RopeArgs {
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;  // elements from a token to the next
  const int32_t *positions, *slots;
  const float *cos, *sin, *wq, *wk;
  void *q_out, *k_out, *v_out;
  int64_t slots_n, kv_stride, max_pos;
  uint32_t* status;
  int tokens, hq, hkv, rot, pairs;
  float eps;
  int run;  // groups of heads that a warp takes
  int runs; // of a token
};

template <typename T>
__device__ __forceinline__ float4 load4(const T* p) {
  if constexpr (sizeof(T) == 4) {
    return __ldcs(reinterpret_cast<const float4*>(p));
  } else {
    const uint2 u = __ldcs(reinterpret_cast<const uint2*>(p));
    T h[4];
    memcpy(h, &u, 8);
    return make_float4(static_cast<float>(h[0]), static_cast<float>(h[1]),
                       static_cast<float>(h[2]), static_cast<float>(h[3]));
  }
}
template <typename T>
__device__ __forceinline__ void store4(T* p, float4 v) {
  T h[4];
  if constexpr (sizeof(T) == 2) {
    const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same<T, __half>::value) h[i] = __float2half_rn(f[i]);
      else h[i] = __float2bfloat16_rn(f[i]);
    }
  }
  uint2 u;
  memcpy(&u, h, 8);
  *reinterpret_cast<uint2*>(p) = u;
}

// (x, y) * c + (y, x) * s of two runs: the rotation where y is x's other half
__device__ __forceinline__ float4 axpy4(float4 a, float4 c, float4 b, float4 s) {
  return make_float4(a.x * c.x + b.x * s.x, a.y * c.y + b.y * s.y, a.z * c.z + b.z * s.z,
                     a.w * c.w + b.w * s.w);
}
__device__ __forceinline__ float4 swapped(float4 a) { return make_float4(a.y, a.x, a.w, a.z); }
__device__ __forceinline__ float4 scaled(float4 a, float r, float4 w) {
  return make_float4(a.x * r * w.x, a.y * r * w.y, a.z * r * w.z, a.w * r * w.w);
}

template <typename IN, typename OUT, int D>
__global__ void __launch_bounds__(kThreads, kCtas) qk_norm_rope_kernel(const RopeArgs a) {
  constexpr int LANES = D / 8;       // of a head
  constexpr int GH = 32 / LANES;     // heads of a warp at a time
  const int lane = threadIdx.x & 31;
  const int sub = lane / LANES, l = lane % LANES;
  const int64_t item = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) >> 5;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int64_t t = item / a.runs;
  if (t >= a.tokens) return;
  const int h0 = static_cast<int>(item % a.runs) * a.run * GH;
  const int heads = a.hq + 2 * a.hkv;
  const int h1 = min(heads, h0 + a.run * GH);

  uint32_t flags = 0;
  int64_t slot = a.slots ? a.slots[t] : t;
  if (slot >= a.slots_n) flags |= SSS_FLAG_INDEX;
  const bool keep = slot >= 0 && slot < a.slots_n;  // -1: the token is not kept
  // the lane's runs, and what turns them: y0 = x0 c0 + o0 s0, y1 = x1 c1 + o1 s1 with
  // o0 = x1 and o1 = x0 (halves), or the neighbours in the run (pairs)
  const int half = a.rot / 2;
  const bool turned = 8 * l < a.rot;
  const int d0 = turned ? 4 * l : 8 * l;
  const int d1 = turned ? half + 4 * l : 8 * l + 4;
  const float4 one = make_float4(1.f, 1.f, 1.f, 1.f), none = make_float4(0.f, 0.f, 0.f, 0.f);
  float4 c0 = one, s0 = none, c1 = one, s1 = none;
  if (a.rot > 0) {
    int64_t pos = a.positions[t];
    if (pos < 0 || pos >= a.max_pos) {
      flags |= SSS_FLAG_INDEX;
      pos = pos < 0 ? 0 : a.max_pos - 1;
    }
    const float* cr = a.cos + pos * half;
    const float* sr = a.sin + pos * half;
    if (turned && a.pairs) {
      const float2 ca = __ldg(reinterpret_cast<const float2*>(cr + d0 / 2));
      const float2 sa = __ldg(reinterpret_cast<const float2*>(sr + d0 / 2));
      const float2 cb = __ldg(reinterpret_cast<const float2*>(cr + d1 / 2));
      const float2 sb = __ldg(reinterpret_cast<const float2*>(sr + d1 / 2));
      c0 = make_float4(ca.x, ca.x, ca.y, ca.y);
      s0 = make_float4(-sa.x, sa.x, -sa.y, sa.y);
      c1 = make_float4(cb.x, cb.x, cb.y, cb.y);
      s1 = make_float4(-sb.x, sb.x, -sb.y, sb.y);
    } else if (turned) {
      c0 = c1 = __ldg(reinterpret_cast<const float4*>(cr + d0));
      s1 = __ldg(reinterpret_cast<const float4*>(sr + d0));
      s0 = make_float4(-s1.x, -s1.y, -s1.z, -s1.w);
    }
  }
  // heads hb, hb + GH, ... of the lane's place in the warp
  auto fetch = [&](int hb, float4 (&x0)[kUnroll], float4 (&x1)[kUnroll]) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = hb + u * GH + sub;
      x0[u] = x1[u] = none;
      if (h < h1) {
        const IN* src;
        if (h < a.hq) src = static_cast<const IN*>(a.q) + t * a.q_stride + h * D;
        else if (h < a.hq + a.hkv) src = static_cast<const IN*>(a.k) + t * a.k_stride + (h - a.hq) * D;
        else src = static_cast<const IN*>(a.v) + t * a.v_stride + (h - a.hq - a.hkv) * D;
        x0[u] = load4(src + d0);
        x1[u] = load4(src + d1);
      }
    }
  };
  float4 n0[kUnroll], n1[kUnroll];
  fetch(h0, n0, n1);
#pragma unroll 1
  for (int hb = h0; hb < h1; hb += kUnroll * GH) {
    float4 x0[kUnroll], x1[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      x0[u] = n0[u];
      x1[u] = n1[u];
    }
    if (hb + kUnroll * GH < h1) fetch(hb + kUnroll * GH, n0, n1);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = hb + u * GH + sub;
      const bool is_q = h < a.hq, is_v = h >= a.hq + a.hkv;
      float4 y0 = x0[u], y1 = x1[u];
      if (a.wq != nullptr || a.wk != nullptr) {
        float ss = y0.x * y0.x + y0.y * y0.y + y0.z * y0.z + y0.w * y0.w + y1.x * y1.x +
                   y1.y * y1.y + y1.z * y1.z + y1.w * y1.w;
#pragma unroll
        for (int m = LANES / 2; m > 0; m >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
        const float* w = is_q ? a.wq : a.wk;
        if (!is_v && w != nullptr) {
          const float r = 1.0f / sqrtf(ss / D + a.eps);
          y0 = scaled(y0, r, __ldg(reinterpret_cast<const float4*>(w + d0)));
          y1 = scaled(y1, r, __ldg(reinterpret_cast<const float4*>(w + d1)));
        }
      }
      if (!is_v) {
        const float4 o0 = a.pairs ? swapped(y0) : y1, o1 = a.pairs ? swapped(y1) : y0;
        if (turned) {
          y0 = axpy4(y0, c0, o0, s0);
          y1 = axpy4(y1, c1, o1, s1);
        }
      }
      if (h >= h1) continue;
      OUT* dst = nullptr;
      if (is_q) {
        dst = static_cast<OUT*>(a.q_out) + (t * a.hq + h) * D;
      } else if (keep) {
        const int kh = h - a.hq - (is_v ? a.hkv : 0);
        dst = static_cast<OUT*>(is_v ? a.v_out : a.k_out) + slot * a.kv_stride + kh * D;
      }
      if (dst != nullptr) {
        store4(dst + d0, y0);
        store4(dst + d1, y1);
      }
    }
  }
  if (flags && a.status) atomicOr(a.status, flags);
}

template <typename IN, typename OUT, int D>
cudaError_t run(RopeArgs& a, cudaStream_t stream) {
  constexpr int GH = 256 / D;
  const int groups = (a.hq + 2 * a.hkv + GH - 1) / GH;
  // A run's groups share their cosines and sines; the shortest runs, up to 8, whose warps
  // are on the SMs all at once (200 tokens of 80 heads: 6.8 us in a wave and a half, 4.4 in
  // one; 512 of 48 heads: 5.8 and 4.8; 48: 2.5 at any length).
  a.run = 1;
  while (a.run < 8 && static_cast<int64_t>(a.tokens) * ((groups + a.run - 1) / a.run) >
                          kCtas * (kThreads / 32) * device_sm_count())
    ++a.run;
  a.runs = (groups + a.run - 1) / a.run;
  const int64_t warps = static_cast<int64_t>(a.tokens) * a.runs;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((warps * 32 + kThreads - 1) / kThreads));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, qk_norm_rope_kernel<IN, OUT, D>, a);
}

template <typename IN, typename OUT>
cudaError_t run_dim(RopeArgs& a, int dim, cudaStream_t stream) {
  return dim == 64 ? run<IN, OUT, 64>(a, stream) : run<IN, OUT, 128>(a, stream);
}
template <typename OUT>
cudaError_t run_in(RopeArgs& a, int in_dtype, int dim, cudaStream_t stream) {
  switch (in_dtype) {
    case SSS_OUT_F16: return run_dim<__half, OUT>(a, dim, stream);
    case SSS_OUT_BF16: return run_dim<__nv_bfloat16, OUT>(a, dim, stream);
    default: return run_dim<float, OUT>(a, dim, stream);
  }
}

}  // namespace

cudaError_t launch_qk_norm_rope(const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                const void* v, int64_t v_stride, int in_dtype, int64_t tokens,
                                int heads, const sss_rope_t& r, const int32_t* positions,
                                void* q_out, const sss_kv_cache_t& cache, const int32_t* slots,
                                uint32_t* status, cudaStream_t stream) {
  RopeArgs a = {};
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.positions = positions;
  a.slots = slots;
  a.cos = r.cos;
  a.sin = r.sin;
  a.wq = r.q_norm;
  a.wk = r.k_norm;
  a.q_out = q_out;
  a.k_out = cache.k;
  a.v_out = cache.v;
  a.slots_n = cache.slots;
  a.kv_stride = cache.stride;
  a.max_pos = r.max_pos;
  a.status = status;
  a.tokens = static_cast<int>(tokens);
  a.hq = heads;
  a.hkv = cache.heads;
  a.rot = r.rot_dim;
  a.pairs = r.style == SSS_ROPE_PAIRS;
  a.eps = r.eps;
  return cache.dtype == SSS_OUT_F16 ? run_in<__half>(a, in_dtype, cache.dim, stream)
                                    : run_in<__nv_bfloat16>(a, in_dtype, cache.dim, stream);
}

}  // namespace sss
