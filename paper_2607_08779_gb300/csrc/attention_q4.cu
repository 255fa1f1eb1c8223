// attention_q4.cu -- how a call of sss_attention_q4 is laid out.
//
// Few rows (single or drafted tokens) read the cache as it is: attn_rows_q4.cu.  Many rows
// would unpack each key and value once for every tile of rows; they are unpacked once for
// the call instead, into the workspace, and go the way of a 16-bit cache.  That writes and
// reads 2 bytes a value, next to 4 flops a value and row: a few per cent of a batch of prompts.
// (Of a step that mixes a chunk with single tokens it is more: max_q says which way the whole
// call goes, so the single tokens' keys are copied too.)
//
// The copy is fp16 for both types of q: fp16(s) c has 14 significant bits at most, of which fp16
// keeps 11 and bf16 would keep 8 (error of the outputs, against 64 bits: 2.8e-3 to 3.4e-3 with a
// bf16 copy, where their own rounding is 1.6e-3).  bf16 queries then go with it as fp16 numbers of
// the same digits: each row gives off a power of two, which its scores' scale takes back.  They are
// staged by the launch that copies the keys.  Small values lose nothing: fp16(s) c is a multiple of
// 2^-24, fp16's least number, and is rounded where it has more than 11 bits, never below.  Large
// ones (beyond 65504, a scale above 8188) are cut and flagged; a copy of a 16th of them, which holds
// them all, lost four bits of what is below 2^-10 (values of about 1e-4: an error of 3e-3 against 2e-4).
#include <algorithm>

#include "attn.cuh"
#include "kv_q4.cuh"

namespace sss {

namespace {
size_t rounded(size_t bytes) { return (bytes + 255) / 256 * 256; }

// the copy in the workspace as a cache
sss_kv_cache_t staged(const AttnQ4Plan& p, const sss_kv_cache_q4_t& c, int batch, void* ws) {
  sss_kv_cache_t s = {};
  char* at = static_cast<char*>(ws);
  s.k = at + p.k_at;
  s.v = at + p.v_at;
  s.slots = (p.whole ? c.pages : static_cast<int64_t>(batch) * p.pages) * c.page_size;
  s.stride = static_cast<int64_t>(c.heads) * c.dim;
  s.page_size = c.page_size;
  s.heads = c.heads;
  s.dim = c.dim;
  s.dtype = SSS_OUT_F16;
  return s;
}

// Row tiles of 8 or 16 tokens x heads, and the splits of their keys.
void plan_rows(AttnPlan& p, int64_t tokens, int group, int kv_heads, int dim, int batch,
               int max_q, int64_t max_kv) {
  // (The figures below compare layouts; the kernels are 1 to 3 % slower by now, all alike.)
  const int64_t sms = device_sm_count();
  p.rows = static_cast<int64_t>(group) * max_q <= 8 ? 8 : 16;
  p.hpt = std::min(group, p.rows);
  p.tpt = std::min(p.rows / p.hpt, max_q);
  p.hchunks = (group + p.hpt - 1) / p.hpt;
  p.one_tile = max_q <= p.tpt;
  p.tiles = p.one_tile ? batch : std::min(tokens / p.tpt + batch,
                                          static_cast<int64_t>(batch) * ((max_q + int64_t{p.tpt} - 1) / p.tpt));
  const int64_t items = std::max<int64_t>(1, p.tiles * kv_heads * p.hchunks);
  // How many CTAs (a cluster of them) share a tile's keys, and of how many warps.  Few tiles: one
  // CTA of 8 warps an SM, as many as that leaves room for (one request of 8192 keys and one
  // key/value head: 6.2 us, 7.5 with 4 warps; 4 of 1400 to 4096 and 8 heads 8.4 and 9.6; 8 of 500 to
  // 1500 7.1 and 8.4), but for 9 to 16 tiles of long requests, where clusters of 16 (or 8) CTAs of 4
  // warps find room, four CTAs of 8 being half a wave (up to 8192 keys, 9, 10, 12, 16 and 16 tiles: 8.4, 8.6,
  // 10.4, 10.4 and 11.9 us so, 12.6, 12.6, 12.6, 12.5 and 13.0 with 8; up to 4096 6.4 to 8.8 and 8.3 to
  // 8.6; up to 3000 and 16 tiles 7.3 to 8.5 and 7.2 to 7.5; 8 tiles of up to 4096 6.4 to 7.2 and 6.3 to 6.5, 24
  // and 32 12.0 and 13.0, and 8.4 and 8.7).  More tiles: CTAs of 4 warps, three
  // an SM; more waves of them cost 2 to 5 us each (64 requests of 300 to 500 keys and 8
  // heads: 12.5 us whole, 20.4 in pairs; 32 of 256 to 2000: 21.0 whole, 17.6 in pairs; 16 of 270 to
  // 800: 8.4 in pairs, 10.8 in fours).  Each CTA but one has 128 keys (one request of 500:
  // 4.2 us in fours, 4.7 in eights).
  constexpr int64_t kLeast = 128;
  int64_t cluster;
  p.warps = max_kv >= 1024 && items <= 64 ? 8 : 4;
  if (p.warps == 8 && items > 8 && items <= 16 && max_kv >= 4096) {
    p.warps = 4;
    cluster = p.rows == 8 ? 16 : 8;
  } else if (p.warps == 8) {
    cluster = items <= 4 ? 16 : items <= 8 ? 8 : items <= 32 ? 4 : 2;
  } else {
    cluster = items <= 8 ? 16 : items <= 32 ? 8 : items <= sms ? (max_kv >= 2048 ? 4 : 2) : items <= 2 * sms ? 2 : 1;
    if (max_kv >= 4096) cluster = std::max<int64_t>(cluster, 2);
  }
  while (cluster > 1 && (cluster - 1) * kLeast >= max_kv) cluster /= 2;
  p.nsplit = cluster;
  // Long requests in chunks of 1024 to 2048 keys, about 256 CTAs of them or more, joined by a
  // second kernel (2.5 us): no cluster then waits for room on one part of the chip, and lengths
  // that differ even out (16 requests of 130 to 16384 keys and 64 heads: 37.5 us in clusters,
  // 30.9 in chunks; 64 of 12000 to 16384: 209 and 185; one of 32768: 21.4 and 14.4; 20 of 400 to
  // 3000: 19.4 and 25.7).  Where the keys take half the time (heads of 64) or tiles are fewer at
  // a time (16 rows) from twice that length on; with 8 warps from 12 steps of a warp on (4 of 2700
  // to 8192, 8 steps: 12.7 us so, 14.6 in chunks).
  const int64_t chunk = std::min<int64_t>(2048, std::max<int64_t>(1024, (max_kv * items / 256 + 127) / 128 * 128));
  const int64_t least = chunk * (p.rows == 8 && dim == 128 ? 4 : 8);
  const bool many = p.warps == 8 ? max_kv / (cluster * 256) >= 12 : max_kv * items >= 1024 * 256;
  if (max_kv >= least && many && items <= 1024) {
    p.chunk = chunk;
    p.nsplit = (max_kv + chunk - 1) / chunk;
    p.join = true;
    const size_t rows = static_cast<size_t>(p.nsplit) * tokens * group * kv_heads;
    p.lse_at = rows * dim * 4;
    p.ws_bytes = p.lse_at + rows * 4;
  }
}
}  // namespace

AttnQ4Plan plan_attention_q4(int64_t tokens, int heads, const sss_kv_cache_q4_t& c, int width,
                             int batch, int max_q, int64_t max_kv) {
  AttnQ4Plan p = {};
  p.pages = static_cast<int>(std::min<int64_t>(width, (max_kv + c.page_size - 1) / c.page_size));
  // Four row tiles read the cache four times, mostly in L2; the copy is written and read at
  // 2 bytes a value.
  const int group = heads / c.heads;
  if (static_cast<int64_t>(group) * max_q <= 64 || max_q == 1 || p.pages == 0) {
    plan_rows(p.of, tokens, group, c.heads, c.dim, batch, max_q, max_kv);
    p.ws_bytes = p.of.ws_bytes;
  } else {
    // `pages` for each request, as many as the bounds allow, or the cache's where those are fewer (the
    // bounds of a captured step are far above its lengths: 64 requests of up to 131072 keys and 8 heads of
    // 128 would take 32 GB, over a cache of 200,000 slots 0.8)
    p.whole = batch > 1 && c.pages > 0 && c.pages < static_cast<int64_t>(batch) * p.pages;
    const sss_kv_cache_t copy = staged(p, c, batch, nullptr);
    p.of = plan_attention(tokens, heads, copy, batch, max_q, max_kv);
    const size_t bytes = static_cast<size_t>(copy.slots) * c.heads * c.dim * 2;
    p.table_at = rounded(p.of.ws_bytes);
    p.k_at = p.table_at + (p.whole ? 0 : rounded(static_cast<size_t>(batch) * p.pages * 4));
    p.v_at = p.k_at + rounded(bytes);
    p.q_at = p.v_at + rounded(bytes);
    p.scale_at = p.q_at + rounded(static_cast<size_t>(tokens) * heads * c.dim * 2);
    p.ws_bytes = p.scale_at + rounded(static_cast<size_t>(tokens) * heads * 4);
  }
  return p;
}

cudaError_t launch_attention_q4(const AttnQ4Plan& p, const void* q, int64_t q_stride, int heads,
                                int dtype, const sss_kv_cache_q4_t& c, const int32_t* cu_q,
                                const int32_t* kv_len, const int32_t* table, int width, int batch,
                                int64_t tokens, int max_q, int64_t max_kv, float scale, void* out,
                                void* workspace, uint32_t* status, cudaStream_t stream) {
  if (p.of.prompt) {
    char* ws = static_cast<char*>(workspace);
    int32_t* to = p.whole ? nullptr : reinterpret_cast<int32_t*>(ws + p.table_at);
    const bool bf16 = dtype == SSS_OUT_BF16;
    float* const scales = reinterpret_cast<float*>(ws + p.scale_at);
    Q4Stage s = {kv_len, table, width, batch, p.pages, max_kv, to, ws + p.k_at, ws + p.v_at, status};
    if (bf16) {
      s.q = q;
      s.q_stride = q_stride;
      s.tokens = tokens;
      s.q_heads = heads;
      s.scale_log2 = scale * 1.4426950408889634f;
      s.q_out = ws + p.q_at;
      s.scales = scales;
      q = ws + p.q_at;
      q_stride = static_cast<int64_t>(heads) * c.dim;
    }
    const cudaError_t e = launch_kv_stage_q4(q4_cache(c), c.dim, s, stream);
    if (e != cudaSuccess) return e;
    return launch_attention(p.of, q, q_stride, heads, staged(p, c, batch, ws), cu_q, kv_len,
                            p.whole ? table : to, p.whole ? width : p.pages, batch, tokens, max_q, max_kv,
                            scale, out, ws, status, stream, bf16 ? scales : nullptr);
  }
  AttnArgs a = {};
  a.q = q;
  a.out = out;
  a.cu_q = cu_q;
  a.kv_len = kv_len;
  a.table = table;
  a.q_stride = q_stride;
  a.slots = c.pages * c.page_size;
  a.status = status;
  a.batch = batch;
  a.tokens = static_cast<int>(tokens);
  a.max_q = max_q;
  a.max_kv = static_cast<int>(max_kv);
  a.heads = heads;
  a.kv_heads = c.heads;
  a.group = heads / c.heads;
  a.table_width = width;
  while ((1 << a.page_shift) < c.page_size) ++a.page_shift;
  a.hpt = p.of.hpt;
  a.hchunks = p.of.hchunks;
  a.hpt_inverse = 65536 / p.of.hpt + 1;
  a.tpt = p.of.tpt;
  a.tiles = static_cast<int>(p.of.tiles);
  a.one_tile = p.of.one_tile ? 1 : 0;
  a.nsplit = static_cast<int>(p.of.nsplit);
  a.chunk = static_cast<int>(p.of.chunk);
  a.part = static_cast<float*>(workspace);
  a.part_lse = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.of.lse_at);
  a.rows = p.of.rows;
  a.warps = p.of.warps;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.stall = (test_stall_mask() & SSS_TEST_STALL_ATTENTION_ROWS) ? 1 : 0;
  const cudaError_t e = launch_attn_rows_q4(a, q4_cache(c), dtype, c.dim, stream);
  return e == cudaSuccess && p.of.join ? launch_attn_join(a, dtype, c.dim, stream) : e;
}

}  // namespace sss
