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
  if (p.prompt) {
    // two row tiles of 128 rows: `tt` tokens (a multiple of 8, as its box in swizzled
    // shared memory needs) of up to 16 heads each
    p.hpt = std::min(group, 16);
    p.tpt = 2 * (128 / p.hpt / 8 * 8);
  } else {
    // 16 rows while they hold a request's tokens and heads
    p.rows = static_cast<int64_t>(group) * max_q <= 16 ? 16 : 32;
    p.hpt = std::min(group, p.rows);
    p.tpt = std::min(p.rows / p.hpt, max_q);
  }
  p.hchunks = (group + p.hpt - 1) / p.hpt;
  p.one_tile = max_q <= p.tpt;
  p.tiles = p.one_tile ? batch : std::min(tokens / p.tpt + batch,
                                          static_cast<int64_t>(batch) * ((max_q + int64_t{p.tpt} - 1) / p.tpt));
  const int64_t per_tile = static_cast<int64_t>(c.heads) * p.hchunks;
  const int64_t items = std::max<int64_t>(1, p.tiles * per_tile);
  if (p.prompt) {
    // Split for SMs that the tiles leave idle, down to one key tile, where it pays: a key
    // tile takes about 1.4 us of an item, the join 2.7 us and what the outputs of `n`
    // splits, written and read in fp32, take at 5 TB/s (5000 bytes in a ns).  30 tokens of
    // 8 heads after 1000: 16.4 us whole, 10.5 in eight; 30 of 32 heads after 500: 14.2
    // whole, 13.2 in five; 500 of 16 heads after 3000: 50.4 whole, 26.9 in five; 512 of 32
    // heads: 12.3 whole, 19.1 in two; 700 of 8 heads: 15.2 whole, 16.3 in six.
    const int64_t kt = std::max<int64_t>(1, (max_kv + 127) / 128);
    const int64_t most = std::max<int64_t>(1, std::min(sms / items, kt));
    int64_t steps = kt, least = kt * 1400;
    for (int64_t n = 2; n <= most; ++n) {
      const int64_t of = (kt + n - 1) / n;
      const int64_t cost = of * 1400 + 2700 + n * tokens * heads * c.dim * 8 / 5000;
      if (cost >= least) continue;
      least = cost;
      steps = of;
    }
    p.chunk = steps * 128;
    p.nsplit = std::max<int64_t>(1, (max_kv + p.chunk - 1) / p.chunk);
    p.join = p.nsplit > 1;
    if (p.join) {
      const size_t rows = static_cast<size_t>(p.nsplit) * tokens * heads;
      p.lse_at = rows * c.dim * 4;
      p.ws_bytes = p.lse_at + rows * 4;
    }
    return p;
  }
  // Few rows: a cluster of as many CTAs as run at a time (two an SM, and whole
  // clusters in a cluster of SMs: 8 of 16 CTAs, 32 of 8), halved until all of them but one
  // have 128 keys: 2 above 128 keys, 4 above 384, 8 above 896, 16 above 1920 (one request of
  // 500 keys: 5.8 us in pairs, 4.8 in fours; of 900: 5.8 in fours, 4.9 in eights).  A second wave costs more than it evens out (24
  // requests of 150 to 1200 keys: 15.7 us whole, 17.5 in pairs; 32 of 256 to 2000: 24.6 in
  // pairs, 31.2 in fours), but where keys are many (20 requests of 400 to 3000: 30.6 us
  // whole, 23.0 in pairs; 16 of 130 to 16384: 89 us in pairs, 59 in fours; 64 of 12000 to
  // 16384: 548 us whole, 530 in fours).
  constexpr int64_t kLeast = 128;
  const int64_t fit = items <= 8 ? 16 : items <= 32 ? 8 : items <= 2 * sms / 4 ? 4 : items <= sms ? 2 : 1;
  int64_t cluster = std::max<int64_t>(fit, max_kv >= 4096 ? 4 : max_kv >= 2048 ? 2 : 1);
  while (cluster > 1 && (cluster - 1) * kLeast >= max_kv) cluster /= 2;
  p.nsplit = cluster;
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
  a.part_lse = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.lse_at);
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
  a.hpt_inverse = 65536 / p.hpt + 1;
  a.tpt = p.tpt;
  a.tiles = static_cast<int>(p.tiles);
  a.one_tile = p.one_tile ? 1 : 0;
  a.table_width = width;
  while (table && (1 << a.page_shift) < c.page_size) ++a.page_shift;
  a.chunk = static_cast<int>(p.chunk);
  a.nsplit = static_cast<int>(p.nsplit);
  a.rows = p.rows;
  a.scale_log2 = scale * 1.4426950408889634f;
  const uint32_t stall = p.prompt ? SSS_TEST_STALL_ATTENTION : SSS_TEST_STALL_ATTENTION_ROWS;
  a.stall = (test_stall_mask() & stall) ? 1 : 0;
  cudaError_t e = p.prompt ? launch_attn_prompt(a, c.dtype, c.dim, stream)
                           : launch_attn_rows(a, c.dtype, c.dim, stream);
  if (e == cudaSuccess && p.join) e = launch_attn_join(a, c.dtype, c.dim, stream);
  return e;
}

}  // namespace sss
