// qk_norm_rope.cu -- from a {q, k, v} projection's outputs to what the attention
// reads, in one pass: per head of q and k (if asked for) the norm
// y = x / sqrt(mean(x^2) + eps) * w, then the rotation of the pairs (a, b) by the
// token's angle, (a cos - b sin, b cos + a sin); q rounded to 16 bits, k and v
// rounded into the token's slot of the cache.  All arithmetic is in fp32; each
// value is rounded once, when it is stored.
//
// Bound by HBM: an fp32 value is read and a 16-bit one written once (6 bytes a
// value, and the token's cosines and sines).  A head is D / 4 lanes with four
// consecutive values each, so a warp holds 128 / D heads; the norm is a sum over
// the head's lanes, and the other value of a pair (a, a + rot / 2) one shuffle
// away.  A warp takes a run of a token's heads, four groups of them in flight at a
// time, and keeps the token's cosines and sines and the norm's weights in
// registers.
#include <algorithm>

#include "sss_internal.cuh"

namespace sss {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;

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

template <typename IN, typename OUT, int D>
__global__ void __launch_bounds__(kThreads) qk_norm_rope_kernel(const RopeArgs a) {
  constexpr int LANES = D / 4;       // of a head
  constexpr int GH = 32 / LANES;     // heads of a warp at a time
  const int lane = threadIdx.x & 31;
  const int sub = lane / LANES, l = lane % LANES, d = 4 * l;
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
  float4 c = make_float4(1.f, 1.f, 1.f, 1.f), s = make_float4(0.f, 0.f, 0.f, 0.f);
  int other = lane;  // the lane of the other halves of this lane's pairs
  if (a.rot > 0) {
    int64_t pos = a.positions[t];
    if (pos < 0 || pos >= a.max_pos) {
      flags |= SSS_FLAG_INDEX;
      pos = pos < 0 ? 0 : a.max_pos - 1;
    }
    const int half = a.rot / 2;
    const float* cr = a.cos + pos * half;
    const float* sr = a.sin + pos * half;
    if (d < a.rot) {
      if (a.pairs) {
        const float2 c2 = __ldg(reinterpret_cast<const float2*>(cr + d / 2));
        const float2 s2 = __ldg(reinterpret_cast<const float2*>(sr + d / 2));
        c = make_float4(c2.x, c2.x, c2.y, c2.y);
        s = make_float4(-s2.x, s2.x, -s2.y, s2.y);
      } else {
        const bool low = d < half;
        c = __ldg(reinterpret_cast<const float4*>(cr + (low ? d : d - half)));
        s = __ldg(reinterpret_cast<const float4*>(sr + (low ? d : d - half)));
        if (low) s = make_float4(-s.x, -s.y, -s.z, -s.w);
        other = lane + (low ? half / 4 : -(half / 4));
      }
    }
  }
  const float4 one = make_float4(1.f, 1.f, 1.f, 1.f);
  const float4 wq = a.wq ? __ldg(reinterpret_cast<const float4*>(a.wq + d)) : one;
  const float4 wk = a.wk ? __ldg(reinterpret_cast<const float4*>(a.wk + d)) : one;

  for (int hb = h0; hb < h1; hb += kUnroll * GH) {
    float4 x[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = hb + u * GH + sub;
      x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (h < h1) {
        const IN* src;
        if (h < a.hq) src = static_cast<const IN*>(a.q) + t * a.q_stride + h * D;
        else if (h < a.hq + a.hkv) src = static_cast<const IN*>(a.k) + t * a.k_stride + (h - a.hq) * D;
        else src = static_cast<const IN*>(a.v) + t * a.v_stride + (h - a.hq - a.hkv) * D;
        x[u] = load4(src + d);
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = hb + u * GH + sub;
      const bool is_q = h < a.hq, is_v = h >= a.hq + a.hkv;
      float4 y = x[u];
      float ss = y.x * y.x + y.y * y.y + y.z * y.z + y.w * y.w;
#pragma unroll
      for (int m = LANES / 2; m > 0; m >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, m);
      if (!is_v && (is_q ? a.wq : a.wk) != nullptr) {
        const float r = 1.0f / sqrtf(ss / D + a.eps);
        const float4 w = is_q ? wq : wk;
        y = make_float4(y.x * r * w.x, y.y * r * w.y, y.z * r * w.z, y.w * r * w.w);
      }
      float4 o;  // the other halves
      if (a.pairs) {
        o = make_float4(y.y, y.x, y.w, y.z);
      } else {
        o.x = __shfl_sync(0xffffffffu, y.x, other);
        o.y = __shfl_sync(0xffffffffu, y.y, other);
        o.z = __shfl_sync(0xffffffffu, y.z, other);
        o.w = __shfl_sync(0xffffffffu, y.w, other);
      }
      if (!is_v && d < a.rot)
        y = make_float4(y.x * c.x + o.x * s.x, y.y * c.y + o.y * s.y, y.z * c.z + o.z * s.z,
                        y.w * c.w + o.w * s.w);
      if (h >= h1) continue;
      if (is_q) {
        store4(static_cast<OUT*>(a.q_out) + (t * a.hq + h) * D + d, y);
      } else if (keep) {
        const int kh = h - a.hq - (is_v ? a.hkv : 0);
        store4(static_cast<OUT*>(is_v ? a.v_out : a.k_out) + slot * a.kv_stride + kh * D + d, y);
      }
    }
  }
  if (flags && a.status) atomicOr(a.status, flags);
}

template <typename IN, typename OUT, int D>
cudaError_t run(RopeArgs& a, cudaStream_t stream) {
  constexpr int GH = 128 / D;
  const int groups = (a.hq + 2 * a.hkv + GH - 1) / GH;
  // a run of 16 groups shares its cosines and sines; fewer while the warps of
  // the call would not fill the SMs (8 CTAs of 8 warps each)
  a.run = 16;
  while (a.run > kUnroll &&
         static_cast<int64_t>(a.tokens) * ((groups + a.run - 1) / a.run) < 64 * device_sm_count())
    a.run /= 2;
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
