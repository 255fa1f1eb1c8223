// kv_q4.cuh -- the layout of the key/value cache in 4 bits (see sss_kv_cache_q4_t), and
// the transposition between a head's values in order and its code words.
#pragma once

#include "sss_internal.cuh"

namespace sss {

constexpr int kQ4Slots = 16;  // of a block: what one bulk copy brings, and a tile's keys

// Where the parts of a block lie.  A head of D values has D / 8 code words and D / 32
// scales a slot.
template <int D>
struct Q4Block {
  static constexpr int kRow = D / 2;                          // bytes of a slot's codes
  static constexpr int kScales = D / 16;                      // bytes of its scales
  static constexpr int kK = 0, kKS = kQ4Slots * kRow;         // keys
  static constexpr int kV = kKS + kQ4Slots * kScales, kVS = kV + kQ4Slots * kRow;
  static constexpr int kBytes = kVS + kQ4Slots * kScales;     // 18 D
};

// Word w of slot j's values: halves swapped for every other pair of slots where a row is
// 64 bytes, so that the eight-byte reads of four slots by a warp meet 32 distinct banks.
template <int D>
__device__ __forceinline__ int q4_value_word(int w, int j) {
  return D == 128 ? w ^ ((j & 2) << 2) : w;
}

struct Q4Cache {
  char* blocks;
  int64_t page_stride;
  int64_t slots;
  int shift, heads;  // of the page size; key/value heads
};
inline Q4Cache q4_cache(const sss_kv_cache_q4_t& c) {
  Q4Cache q = {static_cast<char*>(c.blocks), c.page_stride, c.pages * c.page_size, 0, c.heads};
  while ((1 << q.shift) < c.page_size) ++q.shift;
  return q;
}
// the block that holds `slot` of head h
template <int D>
__device__ __forceinline__ char* q4_block(const Q4Cache& c, int64_t slot, int h) {
  const int64_t page = slot >> c.shift;
  const int in = static_cast<int>(slot) & ((1 << c.shift) - 1);
  return c.blocks + page * c.page_stride +
         ((static_cast<int64_t>(h) << (c.shift - 4)) + (in >> 4)) * Q4Block<D>::kBytes;
}

// A head is D / 8 lanes; lane l has the nibbles of dimensions 8 l .. 8 l + 7 (nibble e of
// its register) on one side, and a code word on the other: word q4_word(l), whose nibble n
// = a + 4 h is dimension 2 W a + W h + w, W = D / 8.  With l's bits (a1 a0 h p), or (a1 a0 h)
// for 64, and lane rank n = (h a1 a0), word w = 8 p + e of the eight lanes with the same p
// is made of their nibbles e: an 8 x 8 transposition, three exchanges.  It is its own
// inverse.
template <int D>
__device__ __forceinline__ int q4_word(int l) {
  return D == 128 ? 8 * (l & 1) + 2 * (l & 2) + (l >> 2) : 4 * (l & 1) + (l >> 1);
}
template <int D>
__device__ __forceinline__ uint32_t q4_transpose(uint32_t v, int l) {
  constexpr int M2 = D == 128 ? 2 : 1, M1 = D == 128 ? 8 : 4, M0 = D == 128 ? 4 : 2;
  uint32_t o = __shfl_xor_sync(0xffffffffu, v, M2);
  v = __byte_perm(v, o, (l & M2) ? 0x3276 : 0x5410);
  o = __shfl_xor_sync(0xffffffffu, v, M1);
  v = __byte_perm(v, o, (l & M1) ? 0x3715 : 0x6240);
  // (moved by a nibble before it is sent: one rotation)
  o = __shfl_xor_sync(0xffffffffu, __funnelshift_l(v, v, (l & M0) ? 4 : 28), M0);
  const uint32_t keep = (l & M0) ? 0xF0F0F0F0u : 0x0F0F0F0Fu;
  return (v & keep) | (o & ~keep);
}

// What sss_attention_q4 leaves of its requests' keys and values for the form of many rows:
// 16-bit values in pages of its own, request b's from page b * pages on, and their table; or in
// the cache's pages, where the cache has fewer.
struct Q4Stage {
  const int32_t *kv_len, *table;
  int table_width, batch;
  int pages;          // of a request
  int64_t max_kv;
  int32_t* new_table; // [batch][pages], or null: the cache's pages
  void *k, *v;        // [slots][heads][dim] fp16, 65504 at most (else flagged)
  uint32_t* status;
  // bf16 queries (else null) as fp16 ones, dense, each row (token, head) with a power of two of
  // its own taken off so that its largest value is between 2^14 and 2^15; and `scale_log2`
  // times that for each row.
  const void* q;
  int64_t q_stride, tokens;
  int q_heads;
  float scale_log2;
  void* q_out;        // [tokens][q_heads][dim]
  float* scales;      // [tokens][q_heads]
};
cudaError_t launch_kv_stage_q4(const Q4Cache& c, int dim, const Q4Stage& s, cudaStream_t stream);

// Attention of few rows over the cache.
struct AttnArgs;
cudaError_t launch_attn_rows_q4(const AttnArgs& a, const Q4Cache& c, int dtype, int dim,
                                cudaStream_t stream);

}  // namespace sss
