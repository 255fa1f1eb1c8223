// attn.cuh -- what the kernels of sss_attention share: their arguments, how a
// launch's work is laid out over requests, rows and keys, and the joining of
// partial results.
//
// Rows.  Token i of request b (n tokens, of kv that it then has) sees its keys
// 0 .. kv - n + i.  The `group` query heads that share a key/value head see the same
// keys, so a tile takes tokens x heads as its rows: `tpt` tokens of `hpt` heads
// of one key/value head (a group of more heads than a tile takes goes in
// `hchunks` tiles).
//
// Keys.  A tile's keys may be cut into splits.  With few rows they are the CTAs of a
// cluster of nsplit, which join there; with many rows each split of `chunk` keys leaves
// its normalised fp32 rows and the log2 of their sums in the workspace, and
// attn_join_kernel adds them.
#pragma once

#include "sss_internal.cuh"

namespace sss {

struct AttnArgs {
  const void* q;
  void* out;  // [tokens][heads][dim]
  const void *k, *v;
  const int32_t *cu_q, *kv_len, *table;
  int64_t q_stride, slots, kv_stride;  // strides in elements
  float* part;      // [nsplit][tokens][heads][dim]
  float* part_lse;  // [nsplit][tokens][heads]
  uint32_t* status;
  int batch, tokens, max_q, max_kv;
  int heads, kv_heads, group;
  int hpt, hchunks, tpt;
  int hpt_inverse;  // row * hpt_inverse >> 16 = row / hpt for rows < 32
  int tiles;        // an upper bound of the call's token tiles
  int tile0;        // the launch's first (a grid holds 65535)
  int one_tile;     // max_q <= tpt: tile b is request b's only one
  int table_width, page_shift;
  int chunk, nsplit;
  int rows;         // of the row form's tiles: 16 or 32
  int warps;        // of its CTAs, over 4 bits: 4 or 8
  int stall;        // test hook
  int box_rows;     // of an output box of the prompt form
  float scale_log2;  // scale * log2(e)
  const float* row_scale;  // nullable [tokens][heads]: in its place, of fp16 operands for bf16 outputs
};

// A request, with lengths that are safe to index by whatever cu_q and kv_len hold
// (what had to be cut raises SSS_FLAG_INDEX).
struct AttnRequest {
  int q0, n, kv;
};
__device__ __forceinline__ AttnRequest attn_request(const AttnArgs& a, int64_t q0, int64_t q1,
                                                    int64_t kv, uint32_t& flags) {
  AttnRequest r;
  int64_t n = q1 - q0;
  if (q0 < 0 || n < 0 || q1 > a.tokens) {
    n = 0;
    flags |= SSS_FLAG_INDEX;
  }
  if (n > a.max_q) {
    n = a.max_q;
    flags |= SSS_FLAG_INDEX;
  }
  // keys that the request can have: those the table has pages for, or without a
  // table its own rows
  int64_t most = a.table ? static_cast<int64_t>(a.table_width) << a.page_shift
                         : min(n, a.slots - q0);
  if (most > a.max_kv) most = a.max_kv;
  if (!a.kv_len) kv = n;
  if (kv < 0 || kv > most) {
    kv = kv < 0 || most < 0 ? 0 : most;
    flags |= SSS_FLAG_INDEX;
  }
  r.q0 = static_cast<int>(q0);
  r.n = static_cast<int>(n);
  r.kv = static_cast<int>(kv);
  return r;
}
__device__ __forceinline__ AttnRequest attn_request(const AttnArgs& a, int b, uint32_t& flags) {
  return attn_request(a, a.cu_q[b], a.cu_q[b + 1], a.kv_len ? a.kv_len[b] : 0, flags);
}

// keys that token i of the request sees
__device__ __forceinline__ int attn_limit(const AttnRequest& r, int i) {
  return max(0, min(r.kv, r.kv - r.n + i + 1));
}

// Token tile `tile` of the launch, found by a whole warp: its request and first
// token.  A request's tiles run from its last tokens, which see the most keys, to
// its first.  False behind the last tile.  The flags may differ by lane.  (Each lane brings all of a request's
// lengths at once: where they are not in the caches, one trip to memory.)
__device__ __forceinline__ bool attn_tile(const AttnArgs& a, int tile, int& b, int& i0,
                                          AttnRequest& rq, uint32_t& flags) {
  if (a.one_tile) {
    b = tile;
    i0 = 0;
    if (tile >= a.batch) return false;
    rq = attn_request(a, b, flags);
    return true;
  }
  const int lane = threadIdx.x & 31;
  int before = 0;
  for (int base = 0; base < a.batch; base += 32) {
    int q0 = 0, q1 = 0, kv = 0, nt = 0;
    if (base + lane < a.batch) {
      q0 = a.cu_q[base + lane];
      q1 = a.cu_q[base + lane + 1];
      kv = a.kv_len ? a.kv_len[base + lane] : 0;
      const int64_t n = static_cast<int64_t>(q1) - q0;
      if (n < 0) flags |= SSS_FLAG_INDEX;
      if (n > 0) nt = static_cast<int>((min(n, static_cast<int64_t>(a.max_q)) + a.tpt - 1) / a.tpt);
    }
    int sum = nt;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, sum, d);
      if (lane >= d) sum += o;
    }
    const uint32_t behind = __ballot_sync(0xffffffffu, before + sum > tile);
    if (behind) {
      const int w = __ffs(behind) - 1;
      b = base + w;
      const int first = before + __shfl_sync(0xffffffffu, sum - nt, w);
      const int count = __shfl_sync(0xffffffffu, nt, w);
      i0 = (count - 1 - (tile - first)) * a.tpt;
      rq = attn_request(a, __shfl_sync(0xffffffffu, q0, w), __shfl_sync(0xffffffffu, q1, w),
                        __shfl_sync(0xffffffffu, kv, w), flags);
      return true;
    }
    before += __shfl_sync(0xffffffffu, sum, 31);
  }
  return false;
}

// The slot of the request's key `key` (a multiple of a step that no page splits),
// or -1 where the table has no valid page for it.
__device__ __forceinline__ int64_t attn_slot(const AttnArgs& a, int page, int key) {
  const int64_t first = static_cast<int64_t>(page) << a.page_shift;
  if (page < 0 || first + (int64_t{1} << a.page_shift) > a.slots) return -1;
  return first + (key & ((1 << a.page_shift) - 1));
}

template <typename T>
struct Pair;  // two 16-bit values in a register
template <>
struct Pair<__half> {
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static constexpr uint32_t kExp = 0x7C00u;
  static __device__ __forceinline__ float value(uint16_t b) { return __half2float(__ushort_as_half(b)); }
};
template <>
struct Pair<__nv_bfloat16> {
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static constexpr uint32_t kExp = 0x7F80u;
  static __device__ __forceinline__ float value(uint16_t b) {
    return __bfloat162float(__ushort_as_bfloat16(b));
  }
};
// whether one of the word's two values is infinite or NaN
template <typename T>
__device__ __forceinline__ bool pair_nonfinite(uint32_t w) {
  constexpr uint32_t lo = Pair<T>::kExp, hi = lo << 16;
  return (w & lo) == lo || (w & hi) == hi;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The forms of the attention.
cudaError_t launch_attn_rows(const AttnArgs& a, int dtype, int dim, cudaStream_t stream);
cudaError_t launch_attn_prompt(const AttnArgs& a, int dtype, int dim, cudaStream_t stream);
cudaError_t launch_attn_join(const AttnArgs& a, int dtype, int dim, cudaStream_t stream);

}  // namespace sss
