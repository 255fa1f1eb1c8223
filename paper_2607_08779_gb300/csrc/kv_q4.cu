// kv_q4.cu -- keys and values into the 4-bit cache and out of it.
//
// Store: per group of 32 values of a head M = max |x|, s = -+M/8 by the sign rule, c =
// clip(RNE(x / s), -8, 7) of the exact quotient (rne.cuh), as the weights' quantizer.
// A head is D / 8 lanes of eight consecutive values: a group is four lanes, whose
// extremes meet in two exchanges; each lane packs its codes and three more exchanges make
// words of the cache's layout of them (kv_q4.cuh).  Fetch goes the same way back.
//
// Bound by instruction issue and by HBM (2 or 4 bytes a value in and 9/16 out, or the other way
// round), so an item has little around its values: a warp takes 256 / D tokens' keys or their
// values, kUnroll heads with all of their loads in flight, and steps from head to head by
// adding to two addresses.  (Tokens beside each other and not heads: no lane is idle whatever
// their number, and slots in order share sectors.)
//
// 8191 tokens of 8 heads of 128 in bf16: store 10.9 us, 3.9 TB/s (issue slots 69 % taken, the
// integer pipe 64 %), fetch 6.9 us, 6.2 TB/s; in fp32 13.5 and 10.3 us.  16 tokens: 1.8
// and 1.5 us, a launch.  With the next token's loads in flight in resident warps 18.4 and 14.0.
#include <algorithm>

#include "kv_q4.cuh"
#include "rne.cuh"

namespace sss {
namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;
constexpr int kUnroll = 4;

struct StoreArgs {
  const void *k, *v;
  int64_t k_stride, v_stride;  // elements
  const int32_t* slots;
  Q4Cache cache;
  uint32_t* status;
  int64_t tokens;
  int run;   // heads that a warp takes
  int runs;  // of them
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

// Grid: tokens, kWarps times 256 / D to a CTA; runs of heads, of the keys and then of the values.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) kv_store_q4_kernel(const __grid_constant__ StoreArgs a) {
  using B = Q4Block<D>;
  constexpr int LANES = D / 8, TOKENS = 32 / LANES;
  constexpr int U = sizeof(T) == 4 ? kUnroll / 2 : kUnroll;
  const int lane = threadIdx.x & 31, l = lane % LANES;
  const int64_t first = (static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5)) * TOKENS;
  const int64_t t = first + lane / LANES;
  const int runs = a.runs;
  const bool is_v = blockIdx.y >= runs;
  const int h0 = (blockIdx.y - (is_v ? runs : 0)) * a.run, h1 = min(a.cache.heads, h0 + a.run);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (first >= a.tokens) return;
  const bool in = t < a.tokens;
  const T* src = (is_v ? static_cast<const T*>(a.v) + t * a.v_stride : static_cast<const T*>(a.k) + t * a.k_stride) +
                 h0 * D + 8 * l;
  const int64_t slot = !in ? -1 : a.slots ? a.slots[t] : t;
  const bool keep = slot >= 0 && slot < a.cache.slots;
  uint32_t flags = slot >= a.cache.slots ? SSS_FLAG_INDEX : 0u;
  const int at = static_cast<int>(slot) & ((1 << a.cache.shift) - 1), j = at & 15;
  const int per_head = B::kBytes << (a.cache.shift - 4);  // bytes of a head's blocks in a page
  const int word = q4_word<D>(l);
  char* head = a.cache.blocks + (slot >> a.cache.shift) * a.cache.page_stride + (at >> 4) * B::kBytes +
               static_cast<int64_t>(h0) * per_head + (is_v ? B::kV : B::kK);
  const int code_at = j * B::kRow + 4 * (is_v ? q4_value_word<D>(word, j) : word);
  const int scale_at = B::kKS + j * B::kScales + 2 * (l >> 2);  // (the scales follow the codes)
  for (int h = h0; h < h1; h += U) {
    Raw<T> x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      x[u].zero();
      if (keep && h + u < h1) x[u].load(src + u * D);
    }
    src += U * D;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (h + u >= h1) break;
      uint16_t s16;
      const uint32_t w = q4_transpose<D>(quantize8(x[u], s16, flags), l);
      if (keep) {
        *reinterpret_cast<uint32_t*>(head + code_at) = w;
        if ((l & 3) == 0) *reinterpret_cast<uint16_t*>(head + scale_at) = s16;
      }
      head += per_head;
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

// Eight consecutive values of a lane; of fp32 ones a store is 32 bytes of a pair of lanes, so
// the even lane takes the first halves of both runs, the odd one the second (15.6 us a fetch of
// 8191 tokens where each writes its own).  Called by whole warps; `in`: the run is written.
template <typename T>
__device__ __forceinline__ void store8(T* p, float (&f)[8], bool in) {
  if constexpr (sizeof(T) == 4) {
    const bool odd = threadIdx.x & 1;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float o = __shfl_xor_sync(0xffffffffu, odd ? f[i] : f[4 + i], 1);
      if (odd) f[i] = o;
      else f[4 + i] = o;
    }
    p += odd ? -4 : 0;
    if (!in) return;
    __stcs(reinterpret_cast<float4*>(p), make_float4(f[0], f[1], f[2], f[3]));
    __stcs(reinterpret_cast<float4*>(p + 8), make_float4(f[4], f[5], f[6], f[7]));
  } else {
    if (!in) return;
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

// the same as fp16 values, 65504 at most
__device__ __forceinline__ void store8_finite(__half* p, const float (&f)[8], bool in) {
  uint32_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(h[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
  if (in) *reinterpret_cast<uint4*>(p) = make_uint4(h[0], h[1], h[2], h[3]);
}

// Queries for the copy (see Q4Stage): a row of D values is D / 8 lanes.  CTA `cta` of `ctas`.
template <int D>
__device__ __forceinline__ void stage_queries(const Q4Stage& a, int64_t cta, int64_t ctas) {
  constexpr int LANES = D / 8;
  const int l = threadIdx.x % LANES, heads = a.q_heads;
  const int64_t rows = a.tokens * heads;
  for (int64_t r0 = cta * (kThreads / LANES); r0 < rows; r0 += ctas * (kThreads / LANES)) {
    const int64_t row = r0 + threadIdx.x / LANES, t = row / heads;
    const bool in = row < rows;
    uint4 u = make_uint4(0u, 0u, 0u, 0u);
    if (in)
      u = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q) + t * a.q_stride +
                                               (row - t * heads) * D + 8 * l));
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    float f[8], top = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      top = fmaxf(top, fmaxf(fabsf(f[2 * i]), fabsf(f[2 * i + 1])));
    }
#pragma unroll
    for (int m = LANES / 2; m > 0; m >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
    // (a row of infinities or NaN keeps them)
    const int E = min(max(static_cast<int>(__float_as_uint(top) >> 23 & 255u) - 127, -112), 127);
    const float up = __int_as_float((14 - E + 127) << 23);
    __half2 h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(f[2 * i] * up, f[2 * i + 1] * up);
    memcpy(&u, h, 16);
    if (!in) continue;
    *reinterpret_cast<uint4*>(static_cast<__half*>(a.q_out) + row * D + 8 * l) = u;
    // (kept above zero and below infinity, for what is multiplied by an infinity or zero)
    if (l == 0)
      a.scales[row] = fminf(fmaxf(a.scale_log2 * __int_as_float((E - 14 + 127) << 23), 1e-37f), 3e38f);
  }
}

// Whether one of a lane's values of these heads is beyond fp16's range, by whole warps.  (Inlined, or as a
// test of each value where it is written, prompts of 4000 tokens and 32 heads took 123 us, so 120.)
template <int D>
__device__ __noinline__ uint32_t range_flags(const char* head, int per_head, int heads, int code_at,
                                             int scale_at, bool in) {
  const int l = threadIdx.x % (D / 8);
  uint32_t flags = 0;
#pragma unroll 1
  for (int h = 0; h < heads; ++h, head += per_head) {
    uint32_t c = in ? __ldg(reinterpret_cast<const uint32_t*>(head + code_at)) : 0x88888888u;
    const float s = in ? __half2float(__ushort_as_half(__ldg(reinterpret_cast<const uint16_t*>(head + scale_at)))) : 0.f;
    c = q4_transpose<D>(c, l);
#pragma unroll 1
    for (int e = 0; e < 8; ++e)
      if (fabsf(s) * fabsf(static_cast<float>(c >> (4 * e) & 15u) - 8.f) > 65504.f) flags |= SSS_FLAG_RANGE;
  }
  return flags;
}

// As the store's grid, of rows.  STAGE: blockIdx.z is a request, t its key t, in a page of its own
// of the copy, or in the cache's place.  QUERIES: the grid's rows behind the 2 * runs are the queries' (a variant
// of its own, as the others take 1 us more with it).
template <typename T, int D, bool STAGE, bool QUERIES>
__global__ void __launch_bounds__(kThreads) kv_fetch_q4_kernel(const __grid_constant__ FetchArgs a) {
  using B = Q4Block<D>;
  constexpr int LANES = D / 8, TOKENS = 32 / LANES;
  const int lane = threadIdx.x & 31, l = lane % LANES;
  const int64_t first = (static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5)) * TOKENS;
  const int64_t t = first + lane / LANES;
  const int runs = a.runs, shift = a.cache.shift;
  const bool is_v = blockIdx.y >= runs;
  const int h0 = (blockIdx.y - (is_v ? runs : 0)) * a.run, h1 = min(a.cache.heads, h0 + a.run);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if constexpr (QUERIES) {
    if (blockIdx.y >= 2 * runs) {
      const int64_t layer = static_cast<int64_t>(gridDim.x) * gridDim.z;
      stage_queries<D>(a.stage, (blockIdx.y - 2 * runs) * layer + static_cast<int64_t>(blockIdx.z) * gridDim.x + blockIdx.x,
                       (gridDim.y - 2 * runs) * layer);
      return;
    }
  }
  if (first >= a.rows) return;
  bool in = t < a.rows;  // the row is written
  uint32_t flags = 0;
  int64_t slot = -1, row = t;
  if constexpr (STAGE) {
    const Q4Stage& s = a.stage;
    const int b = blockIdx.z;
    const int64_t p = first >> shift;  // (a warp's rows are of one page)
    const int32_t page = __ldg(s.table + static_cast<int64_t>(b) * s.table_width + p);
    const bool real = page >= 0 && page < a.cache.slots >> shift;
    // the copy's table, of the pages that are real (what is none, and keys past the
    // request's, are the attention's to flag; what fp16 does not hold is flagged here)
    if (s.new_table != nullptr && blockIdx.y == 0 && lane == 0 && (first & ((1 << shift) - 1)) == 0)
      s.new_table[static_cast<int64_t>(b) * s.pages + p] = real ? b * s.pages + static_cast<int32_t>(p) : -1;
    const int64_t keys = min(static_cast<int64_t>(s.kv_len[b]), s.max_kv);
    if (!real || first >= keys) return;
    in = t < keys;
    slot = (static_cast<int64_t>(page) << shift) + (t & ((1 << shift) - 1));
    // (a page that requests share is copied by each of them: the same bytes)
    row = s.new_table != nullptr ? row + (static_cast<int64_t>(b) * s.pages << shift) : slot;
  } else if (in) {
    slot = a.slots ? a.slots[t] : t;
    if (slot >= a.cache.slots) {
      flags |= SSS_FLAG_INDEX;
      slot = -1;
    }
  }
  T* out = static_cast<T*>(is_v ? a.v : a.k);
  if (out != nullptr) {
    out += (row * a.cache.heads + h0) * D + 8 * l;
    const int at = static_cast<int>(slot) & ((1 << shift) - 1), j = at & 15;
    const int per_head = B::kBytes << (shift - 4), word = q4_word<D>(l);
    const char* head = a.cache.blocks + (slot >> shift) * a.cache.page_stride + (at >> 4) * B::kBytes +
                       static_cast<int64_t>(h0) * per_head + (is_v ? B::kV : B::kK);
    const int code_at = j * B::kRow + 4 * (is_v ? q4_value_word<D>(word, j) : word);
    const int scale_at = B::kKS + j * B::kScales + 2 * (l >> 2);
    uint32_t most = 0;  // of the scales' sizes (of the copy's alone)
    for (int h = h0; h < h1; h += kUnroll) {
      uint32_t w[kUnroll];
      uint16_t s16[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        w[u] = 0x88888888u;
        s16[u] = 0;
        if (in && slot >= 0 && h + u < h1) {
          w[u] = __ldg(reinterpret_cast<const uint32_t*>(head + code_at));
          s16[u] = __ldg(reinterpret_cast<const uint16_t*>(head + scale_at));
        }
        head += per_head;
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (h + u >= h1) break;
        const uint32_t c = q4_transpose<D>(w[u], l);
        const float s = __half2float(__ushort_as_half(s16[u]));
        // A nibble at bits 4 n of a float of 2^23 and more is 2^23 + 16^n u: times s / 16^n, less
        // s (2^23 / 16^n + 8).  For n = 2, 3 and 4 that constant is exact in fp32, and so is the
        // result of one multiply-add.
        const uint32_t part[3] = {c << 8, c >> 4, c >> 16};
        float f[8], by[3], less[3];
#pragma unroll
        for (int n = 0; n < 3; ++n) {
          by[n] = s * (1.f / (1 << (4 * (n + 2))));
          less[n] = -s * ((1 << 23 >> (4 * (n + 2))) + 8.f);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
          f[e] = __fmaf_rn(__uint_as_float((part[e / 3] & (15u << (4 * (e % 3 + 2)))) | 0x4B000000u),
                           by[e % 3], less[e % 3]);
        if constexpr (STAGE) {
          most = max(most, s16[u] & 0x7fffu);
          store8_finite(out, f, in);
        } else {
          store8(out, f, in);
        }
        out += D;
      }
    }
    // a scale of 8188 or less keeps the copy in fp16's range; else the warp looks for what was cut
    if (STAGE && __any_sync(0xffffffffu, most > 0x6FFFu)) {
      const int steps = (h1 - h0 + kUnroll - 1) / kUnroll;
      flags |= range_flags<D>(head - static_cast<int64_t>(steps) * kUnroll * per_head, per_head, h1 - h0, code_at, scale_at, in);
    }
  }
  if (flags && a.status) atomicOr(a.status, flags);
}

template <typename K, typename A>
cudaError_t launch(K kern, A& a, int64_t rows, int dim, int batch, cudaStream_t stream, int64_t queries = 0) {
  // All heads to a warp, or where that gives an SM fewer than 16 warps as many runs of them as do.
  const int64_t all = int64_t{16} * device_sm_count(), tokens = kWarps * 256 / dim;  // of a CTA
  const int64_t warps = std::max<int64_t>(1, 2 * batch * ((rows + 256 / dim - 1) / (256 / dim)));
  const int heads = a.cache.heads;
  int runs = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(heads, all / warps)));
  a.run = (heads + runs - 1) / runs;
  runs = (heads + a.run - 1) / a.run;
  cudaLaunchConfig_t cfg = {};
  a.runs = runs;
  // (the queries: as many more rows of the grid as give them eight CTAs an SM or all they need; in a
  // launch of their own two prompts of 14 to 83 tokens, 12 heads, took 12.2 us, so 10.8; one of 4000, 32 heads, 123 and 120)
  const unsigned ctas = static_cast<unsigned>((rows + tokens - 1) / tokens);
  const int64_t of_queries = std::min<int64_t>((queries * (dim / 8) + kThreads - 1) / kThreads, 8 * device_sm_count());
  const int64_t layer = std::max<int64_t>(1, static_cast<int64_t>(ctas) * batch);
  cfg.gridDim = dim3(ctas, static_cast<unsigned>(2 * runs + (of_queries + layer - 1) / layer), static_cast<unsigned>(batch));
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
template <typename T, bool STAGE, bool QUERIES = false>
cudaError_t fetch(FetchArgs& a, int dim, int batch, cudaStream_t stream) {
  const int64_t queries = QUERIES ? a.stage.tokens * a.stage.q_heads : 0;
  return dim == 64 ? launch(kv_fetch_q4_kernel<T, 64, STAGE, QUERIES>, a, a.rows, dim, batch, stream, queries)
                   : launch(kv_fetch_q4_kernel<T, 128, STAGE, QUERIES>, a, a.rows, dim, batch, stream, queries);
}

}  // namespace

cudaError_t launch_kv_store_q4(const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                               int in_dtype, int64_t tokens, const sss_kv_cache_q4_t& cache,
                               const int32_t* slots, uint32_t* status, cudaStream_t stream) {
  StoreArgs a = {k, v, k_stride, v_stride, slots, q4_cache(cache), status, tokens, 1};
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

cudaError_t launch_kv_stage_q4(const Q4Cache& c, int dim, const Q4Stage& s, cudaStream_t stream) {
  FetchArgs a = {c, nullptr, s.k, s.v, s.status, static_cast<int64_t>(s.pages) << c.shift, 1, 1, s};
  return s.q ? fetch<__half, true, true>(a, dim, s.batch, stream) : fetch<__half, true>(a, dim, s.batch, stream);
}

}  // namespace sss
