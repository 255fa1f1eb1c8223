// kv_q4.cu -- keys and values into the 4-bit cache and out of it.
//
// Store: per group of 32 values of a head M = max |x|, s = -+M/8 by the sign rule, c =
// clip(RNE(x / s), -8, 7) of the exact quotient (rne.cuh), as the weights' quantizer.
// A head is D / 8 lanes of eight consecutive values: a group is four lanes, whose
// extremes meet in two exchanges; each lane packs its codes and three more exchanges make
// words of the cache's layout of them (kv_q4.cuh).  Fetch goes the same way back.
//
// Bound by HBM: 2 or 4 bytes a value in and 9/16 out, or the other way round.  A warp takes
// a run of a token's heads, keys then values, then that of a later token, kUnroll groups of
// heads at a time with the next ones' loads in flight.
#include <algorithm>
#include <numeric>

#include "kv_q4.cuh"
#include "rne.cuh"

namespace sss {
namespace {

constexpr int kThreads = 128;

struct StoreArgs {
  const void *k, *v;
  int64_t k_stride, v_stride;  // elements
  const int32_t* slots;
  Q4Cache cache;
  uint32_t* status;
  int64_t tokens;
  int run, runs;  // groups of heads that a warp takes, and such runs of a token
};

// A lane's eight consecutive values, as they come.
template <typename T>
struct Raw;
template <>
struct Raw<float> {
  float4 a, b;
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void load(const float* p) {
    a = __ldcs(reinterpret_cast<const float4*>(p));
    b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
  }
};
template <typename T>
struct Raw {
  uint4 a;
  __device__ __forceinline__ void zero() { a = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ void load(const T* p) { a = __ldcs(reinterpret_cast<const uint4*>(p)); }
};

// A group's scale and its reciprocal, from its largest value and its smallest one's negative.
struct Scale {
  float s, r;  // s and 1 / s, both times 2^+-64 where far
  uint16_t s16;
  bool zero, far;
};
__device__ __forceinline__ Scale scale_of(float mx, float mn, uint32_t& flags) {
  Scale q;
  const bool bad = is_nonfinite(mx) || is_nonfinite(mn);
  if (bad) flags |= SSS_FLAG_NONFINITE;
  const float M = fmaxf(mx, mn), alpha = __fmul_rn(M, 0.125f);  // exact unless subnormal
  q.zero = alpha == 0.f || bad;
  q.s = q.zero ? 0.f : mx > mn ? -alpha : alpha;
  q.s16 = __half_as_ushort(__float2half_rn(q.s));
  if ((q.s16 & 0x7fffu) == 0x7c00u) {  // (kept finite: an unseen key's is multiplied by zero)
    q.s16 -= 1;
    flags |= SSS_FLAG_RANGE;
  }
  q.far = M < 0x1p-96f || M > 0x1p+96f;  // keep 1/s normal
  if (q.far) q.s = __fmul_rn(q.s, M < 1.f ? 0x1p+64f : 0x1p-64f);
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(q.r) : "f"(q.zero ? 1.f : q.s));  // within 2^-23
  return q;
}

// u: the stored codes as kMagic + 0 .. 16 (a little past both ends where far), clipped and
// packed.  The low byte of such a number is the code: four to a register, 16 made 15.
__device__ __forceinline__ uint32_t packed(const float (&u)[8], bool far) {
  uint32_t t[8], w[2];
#pragma unroll
  for (int e = 0; e < 8; ++e) t[e] = __float_as_uint(u[e]);
  if (far) {  // (a subnormal alpha is rounded)
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = __float_as_uint(fminf(fmaxf(u[e], kMagic), kMagic + 15.f));
  }
#pragma unroll
  for (int o = 0; o < 2; ++o) {  // even codes, odd codes
    w[o] = __byte_perm(__byte_perm(t[o], t[o + 2], 0x0040), __byte_perm(t[o + 4], t[o + 6], 0x0040), 0x5410);
    w[o] -= w[o] >> 4 & 0x01010101u;
  }
  return w[0] + (w[1] << 4);
}

// The codes of a lane's eight values, packed, and the scale of its group (four lanes).
__device__ __forceinline__ uint32_t quantize8(const Raw<float>& v, uint16_t& s16, uint32_t& flags) {
  uint64_t x[4] = {pack2(v.a.x, v.a.y), pack2(v.a.z, v.a.w), pack2(v.b.x, v.b.y), pack2(v.b.z, v.b.w)};
  const float f[8] = {v.a.x, v.a.y, v.a.z, v.a.w, v.b.x, v.b.y, v.b.z, v.b.w};
  float mx = f[0], mn = f[0];
#pragma unroll
  for (int e = 1; e < 8; ++e) {
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(mx) : "f"(f[e]));
    mn = fminf(mn, f[e]);
  }
#pragma unroll
  for (int m = 1; m <= 2; m <<= 1) {
    const float o = __shfl_xor_sync(0xffffffffu, mx, m);
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(mx) : "f"(o));
    mn = fminf(mn, __shfl_xor_sync(0xffffffffu, mn, m));
  }
  const Scale q = scale_of(mx, -mn, flags);
  s16 = q.s16;
  if (q.zero) return 0x88888888u;
  if (q.far) {
    const float sig = fmaxf(mx, -mn) < 1.f ? 0x1p+64f : 0x1p-64f;
#pragma unroll
    for (int p = 0; p < 4; ++p) x[p] = pack2(__fmul_rn(f[2 * p], sig), __fmul_rn(f[2 * p + 1], sig));
  }
  float u[8];
  codes_of<8>(x, q.s, q.r, u, [&](int e) {
    float a, b;
    unpack2(x[e / 2], a, b);
    return (e & 1) ? b : a;
  });
  return packed(u, q.far);
}

template <typename T>
struct Two;
template <>
struct Two<__half> {
  using V = __half2;
  static __device__ __forceinline__ float2 f(V v) { return __half22float2(v); }
};
template <>
struct Two<__nv_bfloat16> {
  using V = __nv_bfloat162;
  static __device__ __forceinline__ float2 f(V v) { return __bfloat1622float2(v); }
};

// 16-bit values.  With significands of 11 bits at most, x / s = 8 x / M is a half-integer or at
// least 2^-13 away from one (8 a / b 2^e - (n + 1/2) = (16 a 2^e - (2 n + 1) b) / 2 b with a, b <
// 2^11, and e >= -5 where the quotient comes near 1/2 at all).  x r is within 2^-19 of it, so
// rounded to multiples of 2^-14 first it is a tie where the quotient is one and on the
// quotient's side of one elsewhere: no exact remainder is needed.
template <typename T>
__device__ __forceinline__ uint32_t quantize8(const Raw<T>& v, uint16_t& s16, uint32_t& flags) {
  using V = typename Two<T>::V;
  V x[4];
  memcpy(x, &v.a, 16);
  // (largest, smallest's negative) in one register: NaN where one is
  const V a = __hmax2_nan(__hmax2_nan(x[0], x[1]), __hmax2_nan(x[2], x[3]));
  const V b = __hneg2(__hmin2_nan(__hmin2_nan(x[0], x[1]), __hmin2_nan(x[2], x[3])));
  uint32_t a32, b32;
  memcpy(&a32, &a, 4);
  memcpy(&b32, &b, 4);
  uint32_t lo = __byte_perm(a32, b32, 0x5410), hi = __byte_perm(a32, b32, 0x7632);
  V m, n;
  memcpy(&m, &lo, 4);
  memcpy(&n, &hi, 4);
  m = __hmax2_nan(m, n);
#pragma unroll
  for (int d = 1; d <= 2; d <<= 1) m = __hmax2_nan(m, __shfl_xor_sync(0xffffffffu, m, d));
  const float2 top = Two<T>::f(m);
  const Scale q = scale_of(top.x, top.y, flags);
  s16 = q.s16;
  if (q.zero) return 0x88888888u;
  const float sig = !q.far ? 1.f : fmaxf(top.x, top.y) < 1.f ? 0x1p+64f : 0x1p-64f;
  constexpr float kSnap = 768.f;  // 1.5 2^9: its last place is 2^-14
  const uint64_t r2 = pack2(q.r, q.r), snap = pack2(kSnap, kSnap), one = pack2(1.f, 1.f);
  const uint64_t magic = pack2(kMagic + 8.f - kSnap, kMagic + 8.f - kSnap);
  float u[8];
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    float2 f = Two<T>::f(x[p]);
    if (q.far) f = make_float2(__fmul_rn(f.x, sig), __fmul_rn(f.y, sig));
    // (snapped + kSnap) + (kMagic + 8 - kSnap): one rounding to an integer, ties to even
    unpack2(fma2(fma2(pack2(f.x, f.y), r2, snap), one, magic), u[2 * p], u[2 * p + 1]);
  }
  return packed(u, q.far);
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 8) kv_store_q4_kernel(const __grid_constant__ StoreArgs a) {
  using B = Q4Block<D>;
  constexpr int LANES = D / 8, GH = 32 / LANES;
  constexpr int U = sizeof(T) == 4 ? 1 : 2;  // groups of heads at a time
  const int lane = threadIdx.x & 31, sub = lane / LANES, l = lane % LANES;
  const int warp = (blockIdx.x * kThreads + threadIdx.x) >> 5;
  const int H = a.cache.heads, heads = 2 * H;
  int64_t t = warp / a.runs;
  const int h0 = (warp - static_cast<int>(t) * a.runs) * a.run * GH, h1 = min(heads, h0 + a.run * GH);
  const int64_t step = gridDim.x * (kThreads / 32) / a.runs;  // (a multiple of runs)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (t >= a.tokens) return;
  const auto load = [&](int64_t tt, int hb, Raw<T> (&x)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = hb + u * GH + sub;
      const T* src = h >= H ? static_cast<const T*>(a.v) + tt * a.v_stride + (h - H) * D
                            : static_cast<const T*>(a.k) + tt * a.k_stride + h * D;
      x[u].zero();
      if (h < h1) x[u].load(src + 8 * l);
    }
  };
  const auto slot_of = [&](int64_t tt) { return a.slots ? static_cast<int64_t>(a.slots[tt]) : tt; };
  uint32_t flags = 0;
  const int word = q4_word<D>(l);
  const int per_head = B::kBytes << (a.cache.shift - 4);  // bytes of a head's blocks in a page
  int64_t slot = slot_of(t);
  int hb = h0;
  Raw<T> next[U];
  load(t, hb, next);
  while (true) {
    Raw<T> x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = next[u];
    const int64_t at_slot = slot;
    const int at_h = hb;
    hb += U * GH;
    if (hb >= h1) {
      hb = h0;
      t += step;
      if (t < a.tokens) slot = slot_of(t);
    }
    const bool more = t < a.tokens;
    if (more) load(t, hb, next);
    if (at_slot >= a.cache.slots) flags |= SSS_FLAG_INDEX;
    if (at_slot >= 0 && at_slot < a.cache.slots) {
      const int in = static_cast<int>(at_slot) & ((1 << a.cache.shift) - 1), j = in & 15;
      char* page = a.cache.blocks + (at_slot >> a.cache.shift) * a.cache.page_stride + (in >> 4) * B::kBytes;
      const int vword = q4_value_word<D>(word, j);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = at_h + u * GH + sub;
        uint16_t s16;
        const uint32_t w = q4_transpose<D>(quantize8(x[u], s16, flags), l);
        if (h >= h1) continue;
        const bool is_v = h >= H;
        char* b = page + static_cast<int64_t>(is_v ? h - H : h) * per_head + (is_v ? B::kV : B::kK);
        reinterpret_cast<uint32_t*>(b + j * B::kRow)[is_v ? vword : word] = w;
        if ((l & 3) == 0)  // (the scales follow the codes)
          reinterpret_cast<uint16_t*>(b + B::kKS + j * B::kScales)[l >> 2] = s16;
      }
    }
    if (!more) break;
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
__global__ void __launch_bounds__(kThreads, 8) kv_fetch_q4_kernel(const __grid_constant__ FetchArgs a) {
  using B = Q4Block<D>;
  constexpr int LANES = D / 8, GH = 32 / LANES;
  constexpr int U = 2;  // groups of heads at a time
  const int lane = threadIdx.x & 31, sub = lane / LANES, l = lane % LANES;
  const int warp = (blockIdx.x * kThreads + threadIdx.x) >> 5;
  const int H = a.cache.heads, heads = 2 * H, shift = a.cache.shift;
  int64_t t = warp / a.runs;
  const int h0 = (warp - static_cast<int>(t) * a.runs) * a.run * GH, h1 = min(heads, h0 + a.run * GH);
  const int64_t step = gridDim.x * (kThreads / 32) / a.runs;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  uint32_t flags = 0;
  int64_t rows = a.rows, first = 0;
  const int32_t* table = nullptr;
  if constexpr (STAGE) {
    const Q4Stage& s = a.stage;
    const int b = blockIdx.y;
    table = s.table + static_cast<int64_t>(b) * s.table_width;
    first = static_cast<int64_t>(b) * s.pages << shift;
    // the copy's table, of the pages that are real; (what is none, and keys past the
    // request's, are the attention's to flag)
    for (int p = blockIdx.x * kThreads + threadIdx.x; p < s.pages; p += gridDim.x * kThreads) {
      const int32_t page = table[p];
      s.new_table[static_cast<int64_t>(b) * s.pages + p] =
          page >= 0 && page < a.cache.slots >> shift ? b * s.pages + p : -1;
    }
    rows = min(rows, min(static_cast<int64_t>(s.kv_len[b]), s.max_kv));
  }
  if (t >= rows) return;
  const auto slot_of = [&](int64_t tt) -> int64_t {
    if constexpr (STAGE) {
      const int32_t page = __ldg(table + (tt >> shift));
      return page >= 0 && page < a.cache.slots >> shift
                 ? (static_cast<int64_t>(page) << shift) + (tt & ((1 << shift) - 1)) : -1;
    } else {
      return a.slots ? static_cast<int64_t>(a.slots[tt]) : tt;
    }
  };
  const int word = q4_word<D>(l), per_head = B::kBytes << (shift - 4);
  const auto load = [&](int64_t slot, int hb, uint32_t (&w)[U], uint16_t (&s16)[U]) {
    const int in = static_cast<int>(slot) & ((1 << shift) - 1), j = in & 15;
    const char* page = a.cache.blocks + (slot >> shift) * a.cache.page_stride + (in >> 4) * B::kBytes;
    const bool real = slot >= 0 && slot < a.cache.slots;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = hb + u * GH + sub;
      const bool is_v = h >= H;
      const char* b = page + static_cast<int64_t>(is_v ? h - H : h) * per_head + (is_v ? B::kV : B::kK);
      w[u] = 0x88888888u;
      s16[u] = 0;
      if (real && h < h1) {
        w[u] = __ldg(reinterpret_cast<const uint32_t*>(b + j * B::kRow) + (is_v ? q4_value_word<D>(word, j) : word));
        s16[u] = __ldg(reinterpret_cast<const uint16_t*>(b + B::kKS + j * B::kScales) + (l >> 2));
      }
    }
  };
  // the slot of the row after the next is read beside the next one's words
  int64_t slot = slot_of(t), ahead = t + step < rows ? slot_of(t + step) : 0;
  int hb = h0;
  uint32_t nw[U];
  uint16_t ns[U];
  load(slot, hb, nw, ns);
  while (true) {
    uint32_t w[U];
    float s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      w[u] = nw[u];
      s[u] = __half2float(__ushort_as_half(ns[u]));
    }
    const int64_t row = first + t;
    const int at_h = hb;
    if (slot >= a.cache.slots) flags |= SSS_FLAG_INDEX;
    const bool skip = STAGE && slot < 0;
    hb += U * GH;
    if (hb >= h1) {
      hb = h0;
      t += step;
      slot = ahead;
      if (t + step < rows) ahead = slot_of(t + step);
    }
    const bool more = t < rows;
    if (more) load(slot, hb, nw, ns);
    if (!skip) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = at_h + u * GH + sub;
        const uint32_t c = q4_transpose<D>(w[u], l);
        float f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)  // (2^23 + u) - (2^23 + 8), without a conversion
          f[e] = s[u] * (__uint_as_float((c >> (4 * e) & 15u) | 0x4B000000u) - 8388616.f);
        if (h >= h1) continue;
        const bool is_v = h >= H;
        T* out = static_cast<T*>(is_v ? a.v : a.k);
        if (out) store8(out + (row * H + (is_v ? h - H : h)) * D + 8 * l, f);
      }
    }
    if (!more) break;
  }
  if (flags && a.status) atomicOr(a.status, flags);
}

template <typename K, typename A>
cudaError_t launch(K kern, A& a, int64_t rows, int dim, int batch, cudaStream_t stream) {
  // All of a token's heads to a warp while that gives every SM 32 warps, else as many runs
  // as do; then as many warps as run at a time.
  const int gh = 256 / dim, groups = (2 * a.cache.heads + gh - 1) / gh;
  const int64_t all = int64_t{64} * device_sm_count();
  a.runs = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(groups, all / std::max<int64_t>(1, rows * batch))));
  a.run = (groups + a.runs - 1) / a.runs;
  a.runs = (groups + a.run - 1) / a.run;
  // (whole CTAs of whole tokens' runs)
  const int64_t unit = std::lcm<int64_t>(a.runs, kThreads / 32) / (kThreads / 32);
  const int64_t want = (rows * a.runs * 32 + kThreads - 1) / kThreads;
  const int64_t most = std::max<int64_t>(1, all / (kThreads / 32) / batch);
  const int64_t blocks = (std::min(want, most) + unit - 1) / unit * unit;
  if (blocks > INT32_MAX / kThreads) return cudaErrorNotSupported;
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
