// kv_q4.cu -- keys and values into the 4-bit cache and out of it.
//
// Store: per group of 32 values of a head M = max |x|, s = -+M/8 by the sign rule, c =
// clip(RNE(x / s), -8, 7) of the exact quotient (rne.cuh), as the weights' quantizer.
// A head is D / 8 lanes of eight consecutive values: a group is four lanes, whose
// extremes meet in two exchanges; each lane packs its codes and three more exchanges make
// words of the cache's layout of them (kv_q4.cuh).  Fetch goes the same way back.
//
// Bound by HBM: 2 or 4 bytes a value in and 9/16 out, or the other way round.  A warp takes
// a run of a token's heads, keys then values, kUnroll groups of them at a time, with the
// slot read beside them.
#include <algorithm>

#include "kv_q4.cuh"
#include "rne.cuh"

namespace sss {
namespace {

constexpr int kThreads = 128;
constexpr int kUnroll = 4;

struct StoreArgs {
  const void *k, *v;
  int64_t k_stride, v_stride;  // elements
  const int32_t* slots;
  Q4Cache cache;
  uint32_t* status;
  int64_t tokens;
  int run, runs;  // groups of heads that a warp takes, and such runs of a token
};

// eight consecutive values
template <typename T>
__device__ __forceinline__ void load8(const T* p, uint64_t (&x)[4]) {
  if constexpr (sizeof(T) == 4) {
    const float4 a = __ldcs(reinterpret_cast<const float4*>(p));
    const float4 b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
    x[0] = pack2(a.x, a.y);
    x[1] = pack2(a.z, a.w);
    x[2] = pack2(b.x, b.y);
    x[3] = pack2(b.z, b.w);
  } else {
    const uint4 u = __ldcs(reinterpret_cast<const uint4*>(p));
    T h[8];
    memcpy(h, &u, 16);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      x[i] = pack2(static_cast<float>(h[2 * i]), static_cast<float>(h[2 * i + 1]));
  }
}

// The codes of a lane's eight values, packed, and the scale of its group (four lanes).
__device__ __forceinline__ uint32_t quantize8(uint64_t (&x)[4], uint16_t& s16, uint32_t& flags) {
  float mx, mn, x0, x1;
  unpack2(x[0], x0, x1);
  mx = mn = x0;
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    unpack2(x[p], x0, x1);
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(mx) : "f"(x0));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(mx) : "f"(x1));
    mn = fminf(mn, fminf(x0, x1));
  }
#pragma unroll
  for (int m = 1; m <= 2; m <<= 1) {
    const float o = __shfl_xor_sync(0xffffffffu, mx, m);
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(mx) : "f"(o));
    mn = fminf(mn, __shfl_xor_sync(0xffffffffu, mn, m));
  }
  const bool bad = is_nonfinite(mx) || is_nonfinite(mn);
  if (bad) flags |= SSS_FLAG_NONFINITE;
  const float M = fmaxf(mx, -mn);
  const float alpha = __fmul_rn(M, 0.125f);  // exact unless subnormal
  const bool zero = alpha == 0.f || bad;
  const float s = zero ? 0.f : mx > -mn ? -alpha : alpha;
  s16 = __half_as_ushort(__float2half_rn(s));
  if ((s16 & 0x7fffu) == 0x7c00u) {  // (kept finite: the value of a key that a row does not
    s16 -= 1;                        // see is multiplied by zero)
    flags |= SSS_FLAG_RANGE;
  }
  if (zero) return 0x88888888u;
  float ss = s, sig = 1.f;
  const bool far = M < 0x1p-96f || M > 0x1p+96f;
  if (far) {  // keep 1/s normal
    sig = M < 1.f ? 0x1p+64f : 0x1p-64f;
    ss = __fmul_rn(s, sig);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      unpack2(x[p], x0, x1);
      x[p] = pack2(__fmul_rn(x0, sig), __fmul_rn(x1, sig));
    }
  }
  float u[8];
  codes_of<8>(x, ss, __frcp_rn(ss), u, [&](int e) {
    float a, b;
    unpack2(x[e / 2], a, b);
    return (e & 1) ? b : a;
  });
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float t = fminf(u[e], kMagic + 15.f);
    if (far) t = fmaxf(t, kMagic);  // (a subnormal alpha is rounded: both ends may clip)
    w |= (static_cast<uint32_t>(__float_as_int(t)) & 15u) << (4 * e);
  }
  return w;
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads) kv_store_q4_kernel(const __grid_constant__ StoreArgs a) {
  using B = Q4Block<D>;
  constexpr int LANES = D / 8, GH = 32 / LANES;
  const int lane = threadIdx.x & 31, sub = lane / LANES, l = lane % LANES;
  const int64_t item = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) >> 5;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int64_t t = item / a.runs;
  if (t >= a.tokens) return;
  const int h0 = static_cast<int>(item - t * a.runs) * a.run * GH, heads = 2 * a.cache.heads;
  const int h1 = min(heads, h0 + a.run * GH);
  uint32_t flags = 0;
  const int64_t slot = a.slots ? a.slots[t] : t;
  if (slot >= a.cache.slots) flags |= SSS_FLAG_INDEX;
  const bool keep = slot >= 0 && slot < a.cache.slots;
  if (keep) {
    const int j = static_cast<int>(slot) & 15;
    for (int hb = h0; hb < h1; hb += kUnroll * GH) {
      uint64_t x[kUnroll][4];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int h = hb + u * GH + sub;
        const bool is_v = h >= a.cache.heads;
        const T* src = is_v ? static_cast<const T*>(a.v) + t * a.v_stride + (h - a.cache.heads) * D
                            : static_cast<const T*>(a.k) + t * a.k_stride + h * D;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[u][i] = 0;
        if (h < h1) load8(src + 8 * l, x[u]);
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (hb + u * GH >= h1) break;
        const int h = hb + u * GH + sub;
        uint16_t s16;
        const uint32_t w = q4_transpose<D>(quantize8(x[u], s16, flags), l);
        if (h >= h1) continue;
        const bool is_v = h >= a.cache.heads;
        char* b = q4_block<D>(a.cache, slot, is_v ? h - a.cache.heads : h);
        const int at = q4_word<D>(l);
        reinterpret_cast<uint32_t*>(b + (is_v ? B::kV : B::kK) + j * B::kRow)[is_v ? q4_value_word<D>(at, j) : at] = w;
        if ((l & 3) == 0)
          reinterpret_cast<uint16_t*>(b + (is_v ? B::kVS : B::kKS) + j * B::kScales)[l >> 2] = s16;
      }
    }
  }
  if (flags && a.status) atomicOr(a.status, flags);
}

struct FetchArgs {
  Q4Cache cache;
  const int32_t* slots;
  void *k, *v;
  uint32_t* status;
  int64_t rows;
  int run, runs;
  Q4Stage stage;
};

template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&f)[8]) {
  if constexpr (sizeof(T) == 4) {
    __stcs(reinterpret_cast<float4*>(p), make_float4(f[0], f[1], f[2], f[3]));
    __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(f[4], f[5], f[6], f[7]));
  } else {
    T h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (std::is_same<T, __half>::value) h[i] = __float2half_rn(f[i]);
      else h[i] = __float2bfloat16_rn(f[i]);
    }
    uint4 u;
    memcpy(&u, h, 16);
    *reinterpret_cast<uint4*>(p) = u;
  }
}

// STAGE: blockIdx.y is a request; row t of the copy is its key t, in a page of its own.
template <typename T, int D, bool STAGE>
__global__ void __launch_bounds__(kThreads) kv_fetch_q4_kernel(const __grid_constant__ FetchArgs a) {
  using B = Q4Block<D>;
  constexpr int LANES = D / 8, GH = 32 / LANES;
  const int lane = threadIdx.x & 31, sub = lane / LANES, l = lane % LANES;
  const int64_t item = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) >> 5;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int64_t t = item / a.runs;
  if (t >= a.rows) return;
  const int h0 = static_cast<int>(item - t * a.runs) * a.run * GH, heads = 2 * a.cache.heads;
  const int h1 = min(heads, h0 + a.run * GH);
  uint32_t flags = 0;
  int64_t slot, row = t;
  if constexpr (STAGE) {
    const Q4Stage& s = a.stage;
    const int b = blockIdx.y, shift = a.cache.shift;
    const int64_t p = t >> shift;
    const int32_t page = s.table[static_cast<int64_t>(b) * s.table_width + p];
    const bool real = page >= 0 && static_cast<int64_t>(page) + 1 <= a.cache.slots >> shift;
    row = static_cast<int64_t>(b) * s.pages * (1 << shift) + t;
    if (h0 == 0 && lane == 0 && (t & ((1 << shift) - 1)) == 0)
      s.new_table[static_cast<int64_t>(b) * s.pages + p] = real ? b * s.pages + static_cast<int32_t>(p) : -1;
    // (what is no page, and keys past the request's, are the attention's to flag)
    if (!real || t >= s.kv_len[b] || t >= s.max_kv) return;
    slot = (static_cast<int64_t>(page) << shift) + (t & ((1 << shift) - 1));
  } else {
    slot = a.slots ? a.slots[t] : t;
    if (slot >= a.cache.slots) {
      flags |= SSS_FLAG_INDEX;
      slot = -1;
    }
  }
  const int j = static_cast<int>(slot) & 15, at = q4_word<D>(l);
  for (int hb = h0; hb < h1; hb += kUnroll * GH) {
    uint32_t w[kUnroll];
    uint16_t s16[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = hb + u * GH + sub;
      const bool is_v = h >= a.cache.heads;
      w[u] = 0x88888888u;
      s16[u] = 0;
      if (h < h1 && slot >= 0) {
        const char* b = q4_block<D>(a.cache, slot, is_v ? h - a.cache.heads : h);
        w[u] = __ldg(reinterpret_cast<const uint32_t*>(b + (is_v ? B::kV : B::kK) + j * B::kRow) +
                     (is_v ? q4_value_word<D>(at, j) : at));
        s16[u] = __ldg(reinterpret_cast<const uint16_t*>(b + (is_v ? B::kVS : B::kKS) + j * B::kScales) + (l >> 2));
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (hb + u * GH >= h1) break;
      const int h = hb + u * GH + sub;
      const uint32_t c = q4_transpose<D>(w[u], l);
      const float s = __half2float(__ushort_as_half(s16[u]));
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e)
        f[e] = s * static_cast<float>(static_cast<int>(c >> (4 * e) & 15u) - 8);
      if (h >= h1) continue;
      const bool is_v = h >= a.cache.heads;
      T* out = static_cast<T*>(is_v ? a.v : a.k);
      if (out) store8(out + (row * a.cache.heads + (is_v ? h - a.cache.heads : h)) * D + 8 * l, f);
    }
  }
  if (flags && a.status) atomicOr(a.status, flags);
}

template <typename K, typename A>
cudaError_t launch(K kern, A& a, int64_t rows, int dim, int batch, cudaStream_t stream) {
  // The longest runs, up to kUnroll, that leave every SM eight warps.
  const int gh = 256 / dim, groups = (2 * a.cache.heads + gh - 1) / gh;
  a.run = 1;
  while (a.run < kUnroll && rows * batch * ((groups + a.run) / (a.run + 1)) >= 8 * device_sm_count())
    ++a.run;
  a.runs = (groups + a.run - 1) / a.run;
  const int64_t blocks = (rows * a.runs * 32 + kThreads - 1) / kThreads;
  if (blocks > INT32_MAX) return cudaErrorNotSupported;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(blocks), static_cast<unsigned>(batch));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, a);
}

template <typename T>
cudaError_t store(StoreArgs& a, int dim, cudaStream_t stream) {
  return dim == 64 ? launch(kv_store_q4_kernel<T, 64>, a, a.tokens, dim, 1, stream)
                   : launch(kv_store_q4_kernel<T, 128>, a, a.tokens, dim, 1, stream);
}
template <typename T, bool STAGE>
cudaError_t fetch(FetchArgs& a, int dim, int batch, cudaStream_t stream) {
  return dim == 64 ? launch(kv_fetch_q4_kernel<T, 64, STAGE>, a, a.rows, dim, batch, stream)
                   : launch(kv_fetch_q4_kernel<T, 128, STAGE>, a, a.rows, dim, batch, stream);
}

}  // namespace

cudaError_t launch_kv_store_q4(const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                               int in_dtype, int64_t tokens, const sss_kv_cache_q4_t& cache,
                               const int32_t* slots, uint32_t* status, cudaStream_t stream) {
  StoreArgs a = {k, v, k_stride, v_stride, slots, q4_cache(cache), status, tokens, 1, 1};
  switch (in_dtype) {
    case SSS_OUT_F16: return store<__half>(a, cache.dim, stream);
    case SSS_OUT_BF16: return store<__nv_bfloat16>(a, cache.dim, stream);
    default: return store<float>(a, cache.dim, stream);
  }
}

cudaError_t launch_kv_fetch_q4(const sss_kv_cache_q4_t& cache, const int32_t* slots, int64_t count,
                               void* k, void* v, int out_dtype, uint32_t* status,
                               cudaStream_t stream) {
  FetchArgs a = {q4_cache(cache), slots, k, v, status, count, 1, 1, {}};
  switch (out_dtype) {
    case SSS_OUT_F16: return fetch<__half, false>(a, cache.dim, 1, stream);
    case SSS_OUT_BF16: return fetch<__nv_bfloat16, false>(a, cache.dim, 1, stream);
    default: return fetch<float, false>(a, cache.dim, 1, stream);
  }
}

cudaError_t launch_kv_stage_q4(const Q4Cache& c, int dim, int dtype, const Q4Stage& s,
                               cudaStream_t stream) {
  FetchArgs a = {c, nullptr, s.k, s.v, nullptr, static_cast<int64_t>(s.pages) << c.shift, 1, 1, s};
  return dtype == SSS_OUT_F16 ? fetch<__half, true>(a, dim, s.batch, stream)
                              : fetch<__nv_bfloat16, true>(a, dim, s.batch, stream);
}

}  // namespace sss
