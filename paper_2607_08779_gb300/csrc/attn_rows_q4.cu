// attn_rows_q4.cu -- attention of few rows over the cache in 4 bits.
//
//   o_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = 2^(c q_i.k_j - m_i),  c = scale log2(e)
//
// A warp to a token and head.  A key is D / 8 lanes, one code word each, so a warp takes
// 256 / D keys at a time and keeps a running maximum, sum and output for each of them.
#include <algorithm>

#include "attn.cuh"
#include "kv_q4.cuh"

namespace sss {
namespace {

constexpr int kWarps = 4;

template <typename T, int D>
__global__ void __launch_bounds__(32 * kWarps) attn_rows_q4_kernel(const __grid_constant__ AttnArgs a,
                                                                  const __grid_constant__ Q4Cache c) {
  using B = Q4Block<D>;
  constexpr int W = D / 8, KEYS = 32 / W;
  const int lane = threadIdx.x & 31, w = lane % W, sub = lane / W;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  if (row >= static_cast<int64_t>(a.tokens) * a.heads) return;
  const int t = static_cast<int>(row / a.heads), head = static_cast<int>(row - static_cast<int64_t>(t) * a.heads);
  const int kh = head / a.group;
  int lo = 0, hi = a.batch;  // the token's request: the last whose first token is not behind it
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.cu_q[mid] <= t) lo = mid;
    else hi = mid;
  }
  uint32_t flags = 0;
  const AttnRequest rq = attn_request(a, lo, flags);
  const int i = t - rq.q0;
  const bool mine = i >= 0 && i < rq.n;
  const int lim = mine ? attn_limit(rq, i) : 0;
  const int32_t* table = a.table + static_cast<int64_t>(lo) * a.table_width;
  float q[8], o[8];
  float m = -INFINITY, sum = 0.f;
#pragma unroll
  for (int n = 0; n < 8; ++n) {
    q[n] = static_cast<float>(static_cast<const T*>(a.q)[t * a.q_stride + head * D + 2 * W * (n & 3) + W * (n >> 2) + w]);
    o[n] = 0.f;
  }
  for (int k0 = 0; k0 < lim; k0 += KEYS) {
    const int key = k0 + sub;
    uint32_t kw = 0x88888888u, vw = kw;
    float ks[8], vs[8];
#pragma unroll
    for (int n = 0; n < 8; ++n) ks[n] = vs[n] = 0.f;
    if (key < lim) {
      const int page = table[key >> a.page_shift];
      const int64_t slot = attn_slot(a, page, key);
      if (slot < 0) {
        flags |= SSS_FLAG_INDEX;
      } else {
        const int j = key & 15;
        const char* b = q4_block<D>(c, slot, kh);
        kw = reinterpret_cast<const uint32_t*>(b + B::kK + j * B::kRow)[w];
        vw = reinterpret_cast<const uint32_t*>(b + B::kV + j * B::kRow)[q4_value_word<D>(w, j)];
        const __half* kss = reinterpret_cast<const __half*>(b + B::kKS + j * B::kScales);
        const __half* vss = reinterpret_cast<const __half*>(b + B::kVS + j * B::kScales);
#pragma unroll
        for (int n = 0; n < 8; ++n) {
          const int g = (2 * W * (n & 3) + W * (n >> 2) + w) / 32;
          ks[n] = __half2float(kss[g]);
          vs[n] = __half2float(vss[g]);
        }
      }
    }
    float x = 0.f;
#pragma unroll
    for (int n = 0; n < 8; ++n) x += q[n] * (ks[n] * static_cast<float>(static_cast<int>(kw >> (4 * n) & 15u) - 8));
#pragma unroll
    for (int d = W / 2; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    if (key >= lim) continue;
    x *= a.scale_log2;
    const float top = fmaxf(m, x);
    const float f = top == -INFINITY ? 1.f : ex2(m - top), p = ex2(x - (top == -INFINITY ? 0.f : top));
    m = top;
    sum = sum * f + p;
#pragma unroll
    for (int n = 0; n < 8; ++n)
      o[n] = o[n] * f + p * (vs[n] * static_cast<float>(static_cast<int>(vw >> (4 * n) & 15u) - 8));
  }
  __syncwarp();
#pragma unroll
  for (int d = W; d < 32; d <<= 1) {
    const float om = __shfl_xor_sync(0xffffffffu, m, d), top = fmaxf(m, om);
    const float f = top == -INFINITY ? 1.f : ex2(m - top), g = top == -INFINITY ? 1.f : ex2(om - top);
    sum = sum * f + __shfl_xor_sync(0xffffffffu, sum, d) * g;
    m = top;
#pragma unroll
    for (int n = 0; n < 8; ++n) o[n] = o[n] * f + __shfl_xor_sync(0xffffffffu, o[n], d) * g;
  }
  if (flags && a.status) atomicOr(a.status, flags);
  if (!mine || sub != 0) return;
  const float r = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int n = 0; n < 8; ++n) {
    const uint32_t v = Pair<T>::pack(o[n] * r, 0.f);
    reinterpret_cast<uint16_t*>(a.out)[row * D + 2 * W * (n & 3) + W * (n >> 2) + w] = static_cast<uint16_t>(v);
  }
}

template <typename T, int D>
cudaError_t run(const AttnArgs& a, const Q4Cache& c, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((static_cast<int64_t>(a.tokens) * a.heads + kWarps - 1) / kWarps));
  cfg.blockDim = dim3(32 * kWarps);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, attn_rows_q4_kernel<T, D>, a, c);
}

}  // namespace

cudaError_t launch_attn_rows_q4(const AttnArgs& a, const Q4Cache& c, int dtype, int dim, cudaStream_t stream) {
  if (dtype == SSS_OUT_F16) return dim == 64 ? run<__half, 64>(a, c, stream) : run<__half, 128>(a, c, stream);
  return dim == 64 ? run<__nv_bfloat16, 64>(a, c, stream) : run<__nv_bfloat16, 128>(a, c, stream);
}

}  // namespace sss
