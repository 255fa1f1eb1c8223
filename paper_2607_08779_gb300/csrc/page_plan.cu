// page_plan.cu -- what a step of a serving loop needs to know of its paged
// key/value cache, from the requests' lengths: which pages the new tokens take,
// the block table with them, and every token's position and slot.
//
// With P tokens to a page, request b holds ceil(past / P) pages and needs
// ceil((past + fresh) / P).  The pages that it takes start at the sum of what the
// requests before it take (an exclusive scan), its tokens at the sum of their
// tokens.  Token i of request b lies at position past + i, in page
// table[b][position / P] at place position % P.
//
// Bound by latency: 16 requests read and write 400 bytes, 64 requests with 30,000
// new tokens a quarter of a megabyte.  So it is one launch without a grid-wide
// wait: every CTA scans all lengths by itself (256 requests at a time, one per
// thread) and places its share of the tokens by a binary search among them.  A
// table entry below ceil(past / P) is only read, the others only written (by the
// page's first token), so the order of the CTAs does not matter.  16 requests of one
// token: 2.2 us; 64 with up to 2048 new tokens each: 2.4 us.
#include <algorithm>

#include "sss_internal.cuh"

namespace sss {
namespace {

constexpr int kThreads = 256;

struct PlanArgs {
  const int32_t *past, *fresh, *free_pages;
  int32_t* table;
  int32_t *cu_q, *kv_len, *positions, *slots, *used;
  uint32_t* status;
  int64_t tokens;  // size of positions and slots
  int batch, nfree, width, shift;
};

// inclusive sums over the CTA's threads
__device__ __forceinline__ int64_t warp_scan(int64_t v, int lane) {
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t o = __shfl_up_sync(0xffffffffu, v, d);
    if (lane >= d) v += o;
  }
  return v;
}

__global__ void __launch_bounds__(kThreads) page_plan_kernel(const PlanArgs a) {
  constexpr int kWarps = kThreads / 32;
  __shared__ int64_t first_token[kThreads + 1];  // of the chunk's requests
  __shared__ int64_t first_page[kThreads];       // index into free_pages
  __shared__ int past_of[kThreads];
  __shared__ int64_t warp_tokens[kWarps], warp_pages[kWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int P = 1 << a.shift;
  const bool writer = blockIdx.x == 0;
  uint32_t flags = 0;
  int64_t tokens0 = 0, pages0 = 0;  // of the chunks before this one
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  for (int b0 = 0; b0 < a.batch; b0 += kThreads) {
    const int b = b0 + tid;
    int64_t past = 0, fresh = 0;
    if (b < a.batch) {
      past = a.past[b];
      fresh = a.fresh[b];
      if (past < 0 || fresh < 0 || past + fresh > INT32_MAX) {
        flags |= SSS_FLAG_INDEX;
        past = past < 0 ? 0 : past;
        fresh = fresh < 0 ? 0 : min(fresh, static_cast<int64_t>(INT32_MAX) - past);
      }
    }
    const int64_t need = ((past + fresh + P - 1) >> a.shift) - ((past + P - 1) >> a.shift);
    const int64_t ts = warp_scan(fresh, lane), ps = warp_scan(need, lane);
    if (lane == 31) {
      warp_tokens[warp] = ts;
      warp_pages[warp] = ps;
    }
    __syncthreads();
    int64_t t0 = tokens0, p0 = pages0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const int64_t t = warp_tokens[w], p = warp_pages[w];
      t0 += w < warp ? t : 0;
      p0 += w < warp ? p : 0;
      tokens0 += t;
      pages0 += p;
    }
    first_token[tid] = t0 + ts - fresh;
    first_page[tid] = p0 + ps - need;
    past_of[tid] = static_cast<int>(past);
    if (tid == 0) first_token[kThreads] = tokens0;
    if (writer && b < a.batch) {
      // (never past the buffers of a token's row, whatever the lengths say: a request that
      // they cut has the keys of the tokens that are left)
      const int64_t from = min(t0 + ts - fresh, a.tokens), to = min(t0 + ts, a.tokens);
      a.cu_q[b] = static_cast<int32_t>(from);
      a.kv_len[b] = static_cast<int32_t>(past + to - from);
    }
    __syncthreads();
    const int64_t begin = first_token[0], end = min(tokens0, a.tokens);
    const int64_t step = static_cast<int64_t>(gridDim.x) * kThreads;
    for (int64_t t = begin + static_cast<int64_t>(blockIdx.x) * kThreads + tid; t < end; t += step) {
      int r = 0;  // the last request whose first token is not behind t
#pragma unroll
      for (int s = kThreads / 2; s > 0; s >>= 1)
        if (first_token[r + s] <= t) r += s;
      const int64_t pos = past_of[r] + (t - first_token[r]);
      const int64_t c = pos >> a.shift, held = (static_cast<int64_t>(past_of[r]) + P - 1) >> a.shift;
      int32_t page = -1;
      if (c < a.width) {
        int32_t* entry = a.table + static_cast<int64_t>(b0 + r) * a.width + c;
        if (c < held) {
          page = *entry;
          if (page < 0) flags |= SSS_FLAG_INDEX;
        } else {
          const int64_t at = first_page[r] + (c - held);
          if (at < a.nfree) page = a.free_pages[at];
          if (page < 0) flags |= SSS_FLAG_PAGES;
          if ((pos & (P - 1)) == 0) *entry = page;
        }
      } else {
        flags |= SSS_FLAG_PAGES;
      }
      const int64_t slot = (static_cast<int64_t>(page) << a.shift) + (pos & (P - 1));
      if (slot > INT32_MAX) flags |= SSS_FLAG_INDEX;
      a.positions[t] = static_cast<int32_t>(pos);
      a.slots[t] = page < 0 || slot > INT32_MAX ? -1 : static_cast<int32_t>(slot);
    }
    __syncthreads();
  }
  // rows of the step's buffers that hold no token
  for (int64_t t = tokens0 + static_cast<int64_t>(blockIdx.x) * kThreads + tid; t < a.tokens;
       t += static_cast<int64_t>(gridDim.x) * kThreads) {
    a.positions[t] = 0;
    a.slots[t] = -1;
  }
  if (writer && tid == 0) {
    if (tokens0 > a.tokens) flags |= SSS_FLAG_INDEX;
    a.cu_q[a.batch] = static_cast<int32_t>(min(tokens0, a.tokens));
    *a.used = static_cast<int32_t>(min(pages0, static_cast<int64_t>(a.nfree)));
  }
  if (flags && a.status) atomicOr(a.status, flags);
}

}  // namespace

cudaError_t launch_page_plan(const int32_t* past, const int32_t* fresh, int batch, int page_size,
                             const int32_t* free_pages, int nfree, int32_t* table, int width,
                             int32_t* cu_q, int32_t* kv_len, int32_t* positions, int32_t* slots,
                             int64_t tokens, int32_t* used, uint32_t* status, cudaStream_t stream) {
  PlanArgs a = {past, fresh, free_pages, table, cu_q, kv_len, positions, slots, used,
                status, tokens, batch, nfree, width, 0};
  while ((1 << a.shift) < page_size) ++a.shift;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(std::max<int64_t>(
      1, std::min<int64_t>((tokens + kThreads - 1) / kThreads, device_sm_count()))));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, page_plan_kernel, a);
}

}  // namespace sss
