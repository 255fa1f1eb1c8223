// attention.cu -- how a call of sss_attention is laid out: which form, its row
// tiles, and how its keys are split.
#include <algorithm>

#include "attn.cuh"

namespace sss {

AttnPlan plan_attention(int64_t tokens, int heads, const sss_kv_cache_t& c, int batch, int max_q,
                        int64_t max_kv) {
  AttnPlan p = {};
  const int group = heads / c.heads;
  const int64_t sms = device_sm_count();
  // the row form while a request's tokens and heads are one tile of it (and without
  // a cache to make a tensor map of)
  p.prompt = static_cast<int64_t>(group) * max_q > 32 && max_q > 1 && c.slots > 0;
  int64_t splits, step;
  if (p.prompt) {
    // two row tiles of 128 rows: `tt` tokens (a multiple of 8, as its box in swizzled
    // shared memory needs) of up to 16 heads each
    p.hpt = std::min(group, 16);
    p.tpt = 2 * (128 / p.hpt / 8 * 8);
  } else {
    // 16 rows while they hold a request's tokens and heads
    p.row_tiles16 = static_cast<int64_t>(group) * max_q <= 16 ? 1 : 2;
    p.hpt = std::min(group, 16 * p.row_tiles16);
    p.tpt = std::min(16 * p.row_tiles16 / p.hpt, max_q);
  }
  p.hchunks = (group + p.hpt - 1) / p.hpt;
  p.one_tile = max_q <= p.tpt;
  p.tiles = p.one_tile ? batch : std::min(tokens / p.tpt + batch,
                                          static_cast<int64_t>(batch) * ((max_q + p.tpt - 1) / p.tpt));
  const int64_t items = std::max<int64_t>(1, p.tiles * c.heads * p.hchunks);
  if (p.prompt) {
    step = 128;
    splits = std::min(sms / items, (max_kv + 511) / 512);
  } else {
    step = 64;
    splits = std::min(4 * sms / items, (max_kv + 255) / 256);
  }
  splits = std::max<int64_t>(1, splits);
  p.chunk = std::max<int64_t>(step, ((max_kv + splits - 1) / splits + step - 1) / step * step);
  p.nsplit = std::max<int64_t>(1, (max_kv + p.chunk - 1) / p.chunk);
  if (p.nsplit > 1) {
    const size_t rowsz = static_cast<size_t>(tokens) * heads;
    p.part_bytes = (p.nsplit * rowsz * c.dim * 4 + 255) / 256 * 256;
    p.ws_bytes = p.part_bytes + p.nsplit * rowsz * 4;
  }
  return p;
}

cudaError_t launch_attention(const AttnPlan& p, const void* q, int64_t q_stride, int heads,
                             const sss_kv_cache_t& c, const int32_t* cu_q, const int32_t* kv_len,
                             const int32_t* table, int width, int batch, int64_t tokens, int max_q,
                             int64_t max_kv, float scale, void* out, void* workspace,
                             uint32_t* status, cudaStream_t stream) {
  AttnArgs a = {};
  a.q = q;
  a.out = out;
  a.k = c.k;
  a.v = c.v;
  a.cu_q = cu_q;
  a.kv_len = kv_len;
  a.table = table;
  a.q_stride = q_stride;
  a.slots = c.slots;
  a.kv_stride = c.stride;
  a.part = static_cast<float*>(workspace);
  a.part_lse = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.part_bytes);
  a.status = status;
  a.batch = batch;
  a.tokens = static_cast<int>(tokens);
  a.max_q = max_q;
  a.max_kv = static_cast<int>(max_kv);
  a.heads = heads;
  a.kv_heads = c.heads;
  a.group = heads / c.heads;
  a.hpt = p.hpt;
  a.hchunks = p.hchunks;
  a.tpt = p.tpt;
  a.tiles = static_cast<int>(p.tiles);
  a.one_tile = p.one_tile ? 1 : 0;
  a.table_width = width;
  while (table && (1 << a.page_shift) < c.page_size) ++a.page_shift;
  a.chunk = static_cast<int>(p.chunk);
  a.nsplit = static_cast<int>(p.nsplit);
  a.scale_log2 = scale * 1.4426950408889634f;
  a.stall = (test_stall_mask() & SSS_TEST_STALL_ATTENTION) ? 1 : 0;
  cudaError_t e = p.prompt ? launch_attn_prompt(a, c.dtype, c.dim, stream)
                           : launch_attn_rows(a, c.dtype, c.dim, p.row_tiles16, stream);
  if (e == cudaSuccess && p.nsplit > 1) e = launch_attn_join(a, c.dtype, c.dim, stream);
  return e;
}

}  // namespace sss
