// attention_q4.cu -- how a call of sss_attention_q4 is laid out.
//
// Few rows (single or drafted tokens) read the cache as it is: attn_rows_q4.cu.  Many rows
// would unpack each key and value once for every tile of rows; they are unpacked once for
// the call instead, into the workspace, and go the way of a 16-bit cache.  That writes and
// reads 2 bytes a value, next to 4 flops a value and row: a few per cent.
#include <algorithm>

#include "attn.cuh"
#include "kv_q4.cuh"

namespace sss {

namespace {
size_t rounded(size_t bytes) { return (bytes + 255) / 256 * 256; }

// the copy in the workspace as a cache
sss_kv_cache_t staged(const AttnQ4Plan& p, const sss_kv_cache_q4_t& c, int batch, int dtype, void* ws) {
  sss_kv_cache_t s = {};
  char* at = static_cast<char*>(ws);
  s.k = at + p.k_at;
  s.v = at + p.v_at;
  s.slots = static_cast<int64_t>(batch) * p.pages * c.page_size;
  s.stride = static_cast<int64_t>(c.heads) * c.dim;
  s.page_size = c.page_size;
  s.heads = c.heads;
  s.dim = c.dim;
  s.dtype = dtype;
  return s;
}
}  // namespace

AttnQ4Plan plan_attention_q4(int64_t tokens, int heads, const sss_kv_cache_q4_t& c, int width,
                             int batch, int max_q, int64_t max_kv) {
  AttnQ4Plan p = {};
  p.pages = static_cast<int>(std::min<int64_t>(width, (max_kv + c.page_size - 1) / c.page_size));
  p.of = plan_attention(tokens, heads, staged(p, c, batch, SSS_OUT_BF16, nullptr), batch, max_q, max_kv);
  if (p.of.prompt) {
    const size_t bytes = static_cast<size_t>(batch) * p.pages * c.page_size * c.heads * c.dim * 2;
    p.table_at = rounded(p.of.ws_bytes);
    p.k_at = p.table_at + rounded(static_cast<size_t>(batch) * p.pages * 4);
    p.v_at = p.k_at + rounded(bytes);
    p.ws_bytes = p.v_at + rounded(bytes);
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
    int32_t* to = reinterpret_cast<int32_t*>(ws + p.table_at);
    const Q4Stage s = {kv_len, table, width, batch, p.pages, max_kv, to, ws + p.k_at, ws + p.v_at};
    cudaError_t e = launch_kv_stage_q4(q4_cache(c), c.dim, dtype, s, stream);
    if (e != cudaSuccess) return e;
    return launch_attention(p.of, q, q_stride, heads, staged(p, c, batch, dtype, ws), cu_q, kv_len,
                            to, p.pages, batch, tokens, max_q, max_kv, scale, out, ws, status, stream);
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
  a.scale_log2 = scale * 1.4426950408889634f;
  return launch_attn_rows_q4(a, q4_cache(c), dtype, c.dim, stream);
}

}  // namespace sss
