// attn_prompt.cu -- attention of many rows (prompts and chunks of prompts) on the
// 5th-generation tensor cores: tcgen05 + tensor memory + TMA.
//
//   o_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = 2^(c q_i.k_j - c m_i),  c = scale log2(e)
//
// in one pass over the keys, m_i a running maximum.  Bound by the tensor pipe: a
// tile of 128 rows and 128 keys takes two products of 128 x 128 x D (1024 cycles at
// D = 128), and the softmax between them 128 exponentials a row.  So a CTA holds two
// row tiles (A and B) that share every key and value tile, and while the softmax
// warps work on one tile's scores the tensor core multiplies for the other:
//   warps 0-3, 4-7  softmax of row tile A, B: a thread owns a row.  It reads the
//             row's 128 scores from tensor memory, takes the maximum, writes p as
//             16-bit pairs over the scores' columns (the second product's A
//             operand) and keeps the row's sum; at the end it scales the row's
//             output and stores it;
//   warp 8    issues the products: scores S = Q K^T (both from shared memory), then
//             O += P V with P from tensor memory.  It takes A and B in turn, which keeps
//             them half a step apart;
//   warps 9, 11  TMA producers of Q and K, and of V (a box per page, or per 128 packed
//             keys; the boxes of a warp are issued one after another, 16 of them at pages
//             of 16 keys: one warp for both lost 5 to 10 % there);
//   warp 10   scheduler: says what the CTA works on next;
//   warps 12-15  look through V tiles that some row does not see whole.
//
// The grid has a CTA for every item (two row tiles and a split of the keys); those
// that run take the items of those that do not yet (cluster launch control), so
// that an item's loads, its first scores and the search for its request run
// while the one before is finished.  Within a request the items with the most keys
// come first.
// Rows are tokens x the heads that share a key/value head (head-major, so that a TMA
// box brings a head's tokens): all heads of a group see almost the same keys, a
// tile spans few tokens, and little of the last key tile is masked.
//
// The maximum is raised only where a score passes it by 8 powers of two: until then
// p stays within 2^8 and nothing has to be rescaled.  (O of the tile lies in
// tensor memory, and a row's thread rescales it there between the scores' arrival,
// which says that the previous product has completed, and the next one's start.)  A
// warp's rows are raised together, by a vote in which only rows of the request have a
// say: the others hold the next request's queries, or what shared memory happened to
// hold, and a request's result must not depend on either.
//
// p is rounded to the cache's type, the tensor core's operand (both operands of a product
// are of one type, and values are read as the cache holds them); the row's sum is that of
// p in fp32, taken as the exponentials come, where a sum of the rounded ones would unpack
// them again in the step's longest chain.  Error against 64 bits, of the output's norm:
// 1.9e-3 to 2.3e-3 in bf16, 2.5e-4 to 2.9e-4 in fp16 (rounded once at the end: 1.6e-3,
// 2.1e-4).
//
// A value that is infinite or NaN must not reach rows that do not see its key (0 x
// NaN would).  In tiles that every row of the CTA sees it cannot do harm; in the others
// warps 12-15 replace it by zero and note the first key of each kind for its
// column, and the rows that see that key add it at the end.
//
// Measured: 8192 tokens of 32 heads of 128 over 8 key/value heads, bf16: 353 us in a
// stream, 1.56 PFLOP/s of what the causal rows need, 82 % of the measured bf16 rate; a few
// calls alone, before the power cap lowers the clock (at 1.91 GHz), 324 us, 1.70 PFLOP/s.  A
// step of both row tiles takes about 2600 cycles where its products take 2048: a row
// tile's softmax is a chain of about 1300 (read the scores, the maximum, 128
// exponentials, write p), longer than the other tile's products that cover it.  10
// ragged prompts: 84 us, 2.1 times their products' time: an item's end and start cost
// 4100 to 6000 cycles, against 1 to 16 steps, and a tile of which rows see a part 1000
// more; this code runs once an item, a quarter of it waiting for instructions.  512
// tokens: 11.7 us, 4.6 of them up to the first scores, then four steps in a row.
// Other divisions of the work that were slower at 8192 tokens: an issuing warp per row
// tile (426 us free-running, 342 in turns), two threads to a row (357), p handed over
// in halves (437), outputs written by warps of their own (339; ragged 106) or straight from
// registers in 32-byte pieces (333; ragged 91), partly seen tiles 32 keys at a time in a
// loop (353; ragged 97).
//
// Tensor memory: scores (then p) of A and B, 128 columns each; outputs of A and B,
// D columns each.  Every wait is bounded (about one second); on expiry the CTA
// raises SSS_FLAG_TIMEOUT, all roles leave their loops and the memory is released.
#include <cuda.h>

#include <algorithm>

#include "attn.cuh"
#include "tc.cuh"

namespace sss {
namespace {

constexpr int kThreads = 512;
constexpr int kKeys = 128;      // of a tile
constexpr float kRaise = 8.0f;  // powers of two
constexpr int kTmemCols = 512;  // one CTA per SM
constexpr int kConsumers = 15;  // warps that read an item

__device__ __forceinline__ void tma_load_3d(const CUtensorMap* map, uint64_t* bar, void* dst, int x,
                                            int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
      : "memory");
}

struct AttnMaps {
  CUtensorMap q, k, v;
  CUtensorMap out;  // boxes of 64 columns of what a warp's 32 rows hold of tokens x heads
};

template <int D>
struct PromptSmem {
  static constexpr int HALVES = D / 64;             // 128-byte wide parts of a row
  static constexpr int PART = 128 * 128;            // a part of 128 rows
  static constexpr int Q_TILE = HALVES * PART;
  static constexpr int KV_TILE = HALVES * PART;
  static constexpr int KS = D == 128 ? 2 : 4;       // key and value tiles in flight
  // (a stage is asked for 2T - 1536 cycles before its use, T = 2048 at best: two do)
  static constexpr int VS = KS;
  static constexpr int K_OFF = 2 * Q_TILE;
  static constexpr int V_OFF = K_OFF + KS * KV_TILE;
  static constexpr int OUT_OFF = V_OFF + VS * KV_TILE;    // 32 rows of 128 bytes per warp
  static constexpr int WORK_OFF = OUT_OFF + 8 * 4096;     // two items, and a 16-byte answer
  static constexpr int FIRST_OFF = WORK_OFF + 2 * 64 + 16;  // uint32 [2][D]
  static constexpr int BAR_OFF = FIRST_OFF + 2 * D * 4;
  static constexpr int NBAR = 4 + 2 * KS + 3 * VS + 4 * 2 + 4 + 2;
  static constexpr int TOTAL = BAR_OFF + NBAR * 8 + 16 + 1024;  // + align slack
  static_assert(TOTAL <= 227 * 1024, "shared memory per CTA");
};

// Instruction descriptor, kind::f16: D fp32, A and B of one 16-bit type, A K-major, B
// K-major or (keys x d, d contiguous) MN-major.
template <typename T>
constexpr uint32_t idesc_of(int n, bool b_mn) {
  const uint32_t fmt = std::is_same<T, __half>::value ? 0u : 1u;
  return (1u << 4) | (fmt << 7) | (fmt << 10) | (b_mn ? 1u << 16 : 0u) |
         (static_cast<uint32_t>(n >> 3) << 17) | (8u << 24);
}

// Shared-memory operands.  All have 128-byte swizzled rows in atoms of 8 rows, 1024
// bytes apart, so the upper words of their descriptors are the same: only the lower
// word is handed about.  Q and K are K-major (d contiguous).  V is MN-major: 64 values of
// d are one row of an atom of 8 keys, and the next 64 values lie a part further.
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_low(uint32_t saddr, uint32_t part) {
  return ((saddr & 0x3FFFFu) >> 4) | (part >> 4) << 16;
}
// Four products of 16 deep in one block, the first of them from zero unless acc.  A and
// B from shared memory, 32 bytes further along d each.
__device__ __forceinline__ void mma4_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc,
                                        uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b32 x, y;\n .reg .b64 a, b;\n setp.ne.b32 p, %4, 0;\n"
      " mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %5};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n"
      " add.u32 x, %1, 2;\n add.u32 y, %2, 2;\n mov.b64 a, {x, %5};\n mov.b64 b, {y, %5};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, 1;\n"
      " add.u32 x, %1, 4;\n add.u32 y, %2, 4;\n mov.b64 a, {x, %5};\n mov.b64 b, {y, %5};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, 1;\n"
      " add.u32 x, %1, 6;\n add.u32 y, %2, 6;\n mov.b64 a, {x, %5};\n mov.b64 b, {y, %5};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, 1;\n}\n" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(acc), "r"(kDescHigh)
      : "memory");
}
// A from tensor memory, 8 columns further each; B 16 keys (2048 bytes) further.
__device__ __forceinline__ void mma4_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc,
                                        uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b32 x, y;\n .reg .b64 b;\n setp.ne.b32 p, %4, 0;\n"
      " mov.b64 b, {%2, %5};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n"
      " add.u32 x, %1, 8;\n add.u32 y, %2, 128;\n mov.b64 b, {y, %5};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [x], b, %3, 1;\n"
      " add.u32 x, %1, 16;\n add.u32 y, %2, 256;\n mov.b64 b, {y, %5};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [x], b, %3, 1;\n"
      " add.u32 x, %1, 24;\n add.u32 y, %2, 384;\n mov.b64 b, {y, %5};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [x], b, %3, 1;\n}\n" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(acc), "r"(kDescHigh)
      : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_wait_st() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// (x0, x1) * s + t
__device__ __forceinline__ float2 fma2(float x0, float x1, float s, float t) {
  float2 r;
  asm("{\n .reg .b64 a, b, c, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %4};\n"
      " mov.b64 c, {%5, %5};\n fma.rn.f32x2 d, a, b, c;\n mov.b64 {%0, %1}, d;\n}\n"
      : "=f"(r.x), "=f"(r.y)
      : "f"(x0), "f"(x1), "f"(s), "f"(t));
  return r;
}
__device__ __forceinline__ float2 mul2(float x0, float x1, float s) {
  float2 r;
  asm("{\n .reg .b64 a, b, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %4};\n"
      " mul.rn.f32x2 d, a, b;\n mov.b64 {%0, %1}, d;\n}\n"
      : "=f"(r.x), "=f"(r.y)
      : "f"(x0), "f"(x1), "f"(s));
  return r;
}
__device__ __forceinline__ float2 add2(float2 x, float2 y) {
  float2 r;
  asm("{\n .reg .b64 a, b, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n"
      " add.rn.f32x2 d, a, b;\n mov.b64 {%0, %1}, d;\n}\n"
      : "=f"(r.x), "=f"(r.y)
      : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y));
  return r;
}

// An item, as the scheduler leaves it in shared memory.
struct __align__(16) Work {
  int live;      // 0: there is no further item
  int b;         // request
  int q0, n, kv; // its AttnRequest
  int kh, g0, nh;  // key/value head; first head of the group and number of heads
  int i0;        // first token of row tile A (row tile B's: i0 + tt)
  int k0;        // first key of the split
  int lim0;      // keys that the first token sees
  int n0, n1;    // key tiles of A, B
  int z;
  int alone;     // no other split has keys
  int pad;
};
static_assert(sizeof(Work) == 64, "");

// The grid's next CTA that has not started, kept from starting: its index in x (-1:
// all have).  To be called by one thread; not again after -1.
__device__ __forceinline__ void next_cta_ask(uint32_t answer, uint64_t* bar) {
  mbar_arrive_expect_tx(bar, 16);
  asm volatile(
      "clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 "
      "[%0], [%1];" ::"r"(answer),
      "r"(smem_u32(bar))
      : "memory");
}
__device__ __forceinline__ int next_cta(uint32_t answer) {
  uint32_t ok, x;
  asm volatile(
      "{\n .reg .pred p;\n .reg .b128 h;\n ld.shared.b128 h, [%2];\n"
      " clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\n"
      " selp.u32 %0, 1, 0, p;\n mov.u32 %1, 0;\n"
      " @p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%1, _, _, _}, h;\n}\n"
      : "=r"(ok), "=r"(x)
      : "r"(answer)
      : "memory");
  // (the answer has been read before the next one is written)
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  return ok ? static_cast<int>(x) : -1;
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 1)
    attn_prompt_kernel(const __grid_constant__ AttnMaps maps, const __grid_constant__ AttnArgs a) {
  using S = PromptSmem<D>;
  extern __shared__ unsigned char smem_raw[];
  // 1024-byte alignment for the swizzle atoms
  unsigned char* smem = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  Work* works = reinterpret_cast<Work*>(smem + S::WORK_OFF);
  // By item parity and column, ten bits each: the first key (from the first tile that
  // some row does not see whole) whose value is +inf, -inf, NaN.
  uint32_t* first = reinterpret_cast<uint32_t*>(smem + S::FIRST_OFF);
  constexpr uint32_t kNone = 0x3FFFFFFFu;
  const uint32_t answer = smem_u32(smem + S::WORK_OFF + 2 * sizeof(Work));
  uint64_t* full_q = reinterpret_cast<uint64_t*>(smem + S::BAR_OFF);
  uint64_t* empty_q = full_q + 2;
  uint64_t* full_k = empty_q + 2;
  uint64_t* empty_k = full_k + S::KS;
  uint64_t* full_v = empty_k + S::KS;
  // the value tile has been looked through, and the next key tile of the item is there
  uint64_t* seen = full_v + S::VS;
  uint64_t* empty_v = seen + S::VS;
  uint64_t* full_s = empty_v + S::VS;   // scores are there (and earlier products done)
  uint64_t* full_p = full_s + 2;
  uint64_t* done = full_p + 2;          // the row tile's output is complete
  uint64_t* free_o = done + 2;          // it has been read
  uint64_t* full_w = free_o + 2;        // an item
  uint64_t* empty_w = full_w + 2;
  uint64_t* asked = empty_w + 2;
  uint64_t* retired = asked + 1;        // used when a wait has run out
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(retired + 1);
  volatile int* abort = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile int* odd = reinterpret_cast<volatile int*>(tmem_slot + 2);  // [2]: `first` holds something

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (warp == 9 && lane < 4) {
    const CUtensorMap* m = &maps.q + lane;
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(m)) : "memory");
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < 2; ++s) {
      mbar_init(&full_q[s], 1);
      mbar_init(&empty_q[s], 1);
      mbar_init(&full_s[s], 1);
      mbar_init(&full_p[s], 4);
      mbar_init(&done[s], 1);
      mbar_init(&free_o[s], 4);
      mbar_init(&full_w[s], 1);
      mbar_init(&empty_w[s], kConsumers);
      odd[s] = 0;
    }
    for (int s = 0; s < S::KS; ++s) {
      mbar_init(&full_k[s], 1);
      mbar_init(&empty_k[s], 2);  // the issuer's, and the warp's that sees every key tile
    }
    for (int s = 0; s < S::VS; ++s) {
      mbar_init(&full_v[s], 1);
      mbar_init(&seen[s], 4);
      mbar_init(&empty_v[s], 1);
    }
    mbar_init(asked, 1);
    mbar_init(retired, 1);
    *abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  for (int i = threadIdx.x; i < 2 * D; i += kThreads) first[i] = kNone;
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     smem_u32(tmem_slot)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int tt = a.tpt / 2;  // tokens of a row tile

  // A wait of the roles whose work is safe to go on with whatever it finds (a wait
  // that ran out raised *abort, and all later ones give up at once).
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    if (!mbar_try_wait(bar, parity)) (void)mbar_wait(bar, parity, abort);
    __syncwarp();
  };

  // The next item, into w: false where there is none (or a wait ran out, ok).  The
  // softmax warps give its place back when they have finished it: an item reaches the
  // others when all is done with the one before the last.
  auto take = [&](int item, Work& w, bool& ok) -> bool {
    ok = __all_sync(0xffffffffu, mbar_wait(&full_w[item & 1], (item >> 1) & 1, abort));
    if (!ok) return false;
    const int4* src = reinterpret_cast<const int4*>(&works[item & 1]);
    int4* dst = reinterpret_cast<int4*>(&w);
#pragma unroll
    for (int i = 0; i < 4; ++i) dst[i] = src[i];
    __syncwarp();
    if (lane == 0 && warp >= 8) mbar_arrive(&empty_w[item & 1]);
    return __reduce_or_sync(0xffffffffu, w.live) != 0;  // (a uniform register)
  };

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == 10) {
      // ---------------- scheduler ----------------
      int x = blockIdx.x, item = 0, asks = 0;
      const int per = a.kv_heads * a.hchunks;
      bool ok = true;
      while (ok) {
        if (x >= 0 && lane == 0) next_cta_ask(answer, asked);
        Work w = {};
        bool live = false;
        uint32_t flags = 0;
        if (x >= 0) {
          int tile = x / per, hx = x - tile * per;
          if (a.nsplit > 1) {
            w.z = tile % a.nsplit;
            tile /= a.nsplit;
          }
          w.kh = hx;
          if (a.hchunks > 1) {
            w.kh = hx / a.hchunks;
            w.g0 = (hx - w.kh * a.hchunks) * a.hpt;
          }
          w.nh = min(a.hpt, a.group - w.g0);
          AttnRequest rq;
          if (attn_tile(a, tile, w.b, w.i0, rq, flags)) {
            w.q0 = rq.q0;
            w.n = rq.n;
            w.kv = rq.kv;
            if (w.i0 < rq.n) {
              w.k0 = w.z * a.chunk;
              w.lim0 = attn_limit(rq, w.i0);
              int lim1 = w.lim0, n[2] = {0, 0};  // lim1: keys that the last token sees
#pragma unroll
              for (int s = 0; s < 2; ++s) {
                const int i = w.i0 + s * tt, last = min(i + tt, rq.n) - 1;
                if (last < i) continue;
                lim1 = attn_limit(rq, last);
                n[s] = max(0, (min(lim1, w.k0 + a.chunk) - w.k0 + kKeys - 1) / kKeys);
              }
              w.n0 = n[0];
              w.n1 = n[1];
              w.alone = lim1 <= a.chunk;
              live = n[0] + n[1] > 0 || w.z == 0;
            }
          }
        }
        if (flags && a.status) atomicOr(a.status, flags);
        if (live || x < 0) {
          ok = __all_sync(0xffffffffu,
                          mbar_wait(&empty_w[item & 1], ((item >> 1) & 1) ^ 1, abort));
          if (!ok) break;
          w.live = live;
          if (lane == 0) {
            works[item & 1] = w;
            mbar_arrive(&full_w[item & 1]);
          }
          __syncwarp();
          ++item;
        }
        if (x < 0) break;
        ok = __all_sync(0xffffffffu, mbar_wait(asked, asks & 1, abort));
        if (!ok) break;
        ++asks;
        x = next_cta(answer);
        __syncwarp();
      }
      if (!ok && x >= 0) {  // the answer in flight lands before the CTA's memory goes
        int drain = 0;
        (void)mbar_wait(asked, asks & 1, &drain);
      }
    } else if (warp == 9 || warp == 11) {
      // ---------------- TMA producers: of Q and K, and of V ----------------
      const bool vals = warp == 11;
      const CUtensorMap* const map = vals ? &maps.v : &maps.k;
      uint64_t* const full = vals ? full_v : full_k;
      uint64_t* const empty = vals ? empty_v : empty_k;
      unsigned char* const tiles = smem + (vals ? S::V_OFF : S::K_OFF);
      const int box = a.table ? min(kKeys, 1 << a.page_shift) : kKeys;  // keys of a box
      const int boxes = kKeys / box * S::HALVES;
      const int my = lane / S::HALVES, half = lane % S::HALVES;
      uint32_t flags = 0;
      int count = 0, qc[2] = {0, 0};  // tiles asked for
      Work w;
      bool ok;
      for (int item = 0; take(item, w, ok); ++item) {
        const int n[2] = {w.n0, w.n1}, nt = max(w.n0, w.n1);
        const int32_t* table =
            a.table ? a.table + static_cast<int64_t>(w.b) * a.table_width : nullptr;
        // Lane l brings box l of a tile: its first slot.  Boxes behind the keys, or of
        // a page that is none, lie past the cache and read as zeros.
        auto entry = [&](int j) -> int {
          const int key = w.k0 + kKeys * j + my * box;
          return table && lane < boxes && j < nt && key < w.kv
                     ? __ldg(table + (key >> a.page_shift))
                     : -1;
        };
        auto slot_of = [&](int page, int j) -> int {
          const int key = w.k0 + kKeys * j + my * box;
          if (key >= w.kv || lane >= boxes) return static_cast<int>(a.slots);
          if (!table) return w.q0 + key;
          const int64_t s = attn_slot(a, page, key);
          if (s < 0) flags |= SSS_FLAG_INDEX;
          return static_cast<int>(s < 0 ? a.slots : s);
        };
        int page = entry(0);
        for (int j = 0; j < nt && ok; ++j) {
          const int slot = slot_of(page, j);
          page = entry(j + 1);
          const int st = count % S::KS;
          ok = ok && __all_sync(0xffffffffu,
                                mbar_wait(empty + st, ((count / S::KS) & 1) ^ 1, abort));
          if (!ok) break;
          if (lane == 0) mbar_arrive_expect_tx(full + st, S::KV_TILE);
          __syncwarp();
          if (lane < boxes)
            tma_load_2d(map, full + st, tiles + st * S::KV_TILE + half * S::PART + my * box * 128,
                        w.kh * D + 64 * half, slot);
          __syncwarp();
          ++count;
          if (j > 0 || vals) continue;
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            if (n[s] == 0 || !ok) continue;
            ok = __all_sync(0xffffffffu, mbar_wait(&empty_q[s], (qc[s] & 1) ^ 1, abort));
            if (!ok) continue;
            if (lane == 0) mbar_arrive_expect_tx(&full_q[s], a.hpt * tt * 128 * S::HALVES);
            __syncwarp();
            if (lane < S::HALVES)
              tma_load_3d(&maps.q, &full_q[s], smem + s * S::Q_TILE + lane * S::PART, 64 * lane,
                          w.q0 + w.i0 + s * tt, w.kh * a.group + w.g0);
            __syncwarp();
            ++qc[s];
          }
        }
        if (!ok) break;
      }
      if (flags && a.status) atomicOr(a.status, flags);
      if (!ok) {  // let this CTA's copies still in flight land
        int drain = 0;
        for (int s = 0; s < 2; ++s)
          if (qc[s] > 0) (void)mbar_wait(&full_q[s], (qc[s] - 1) & 1, &drain);
        for (int i = max(0, count - S::KS); i < count; ++i)
          (void)mbar_wait(full + i % S::KS, (i / S::KS) & 1, &drain);
      }
    } else if (warp == 8) {
      // ---------------- issuer of the products ----------------
      // What it costs beside the products is its waits (a few dependent instructions
      // each, beside two softmax warps on the same scheduler): three a step.  Its
      // control flow and operands are kept in uniform registers: a product then issues
      // in the 64 cycles that it takes, else in 80 to 110.
      constexpr uint32_t id_s = idesc_of<T>(kKeys, false), id_o = idesc_of<T>(D, true);
      const uint32_t tm = __reduce_or_sync(0xffffffffu, tmem);
      const uint32_t base = smem_u32(smem);
      const uint32_t q_desc = desc_low(base, 0), k_desc = desc_low(base + S::K_OFF, 0);
      const uint32_t v_desc = desc_low(base + S::V_OFF, S::PART);
      constexpr uint32_t kStage = S::KV_TILE >> 4, kQ = S::Q_TILE >> 4, kPart = S::PART >> 4;
      uint32_t count = 0;  // key tiles before
      uint32_t qph = 0, pph = 0, oph = 3;  // bit s: the parities of row tile s
      auto scores = [&](int s, uint32_t st) {  // S_s = Q_s K^T of stage st
#pragma unroll
        for (int h = 0; h < S::HALVES; ++h)
          mma4_ss(tm + s * kKeys, q_desc + s * kQ + h * kPart, k_desc + st * kStage + h * kPart,
                  id_s, h > 0);
        umma_commit(&full_s[s]);
      };
      auto outputs = [&](int s, uint32_t st, uint32_t acc) {  // O_s += P_s V
        mma4_ts(tm + 2 * kKeys + s * D, tm + s * kKeys, v_desc + st * kStage, id_o, acc);
        mma4_ts(tm + 2 * kKeys + s * D, tm + s * kKeys + 32, v_desc + st * kStage + 512, id_o, 1);
      };
      for (uint32_t item = 0;; ++item) {
        if (!__all_sync(0xffffffffu, mbar_wait(&full_w[item & 1], item >> 1 & 1, abort))) break;
        const volatile Work* w = &works[item & 1];
        const uint32_t n0 = __reduce_or_sync(0xffffffffu, w->n0);
        const uint32_t n1 = __reduce_or_sync(0xffffffffu, w->n1);
        const uint32_t live = __reduce_or_sync(0xffffffffu, w->live);
        if (lane == 0) mbar_arrive(&empty_w[item & 1]);
        __syncwarp();
        if (live == 0) break;
        const uint32_t nt = max(n0, n1);
        if (nt == 0) continue;
        wait(&full_k[count % S::KS], count / S::KS & 1);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const uint32_t n = s ? n1 : n0;
          if (n == 0) continue;
          wait(&full_q[s], qph >> s & 1);
          qph ^= 1u << s;
          tc_fence_after();
          if (elect_one()) {
            scores(s, count % S::KS);
            if (n == 1) umma_commit(&empty_q[s]);
          }
          __syncwarp();
        }
        if (elect_one()) umma_commit(&empty_k[count % S::KS]);
        __syncwarp();
#pragma unroll
        for (int s = 0; s < 2; ++s) {  // the outputs of the item before have been read
          if ((s ? n1 : n0) == 0) continue;
          wait(&free_o[s], oph >> s & 1);
          oph ^= 1u << s;
        }
        // while both row tiles have at least two key tiles ahead
        const uint32_t both = min(n0, n1) > 2 ? min(n0, n1) - 2 : 0;
        uint32_t j = 0;
#pragma unroll 1
        for (; j < both; ++j, ++count) {
          const uint32_t st = count % S::KS, st1 = (count + 1) % S::KS;
          wait(&seen[st], count / S::KS & 1);
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            wait(&full_p[s], pph >> s & 1);
            tc_fence_after();
            if (elect_one()) {
              outputs(s, st, j > 0);
              scores(s, st1);
              if (s == 1) {
                umma_commit(&empty_v[st]);
                umma_commit(&empty_k[st1]);
              }
            }
            __syncwarp();
          }
          pph ^= 3;
        }
#pragma unroll 1
        for (; j < nt; ++j, ++count) {
          const uint32_t st = count % S::KS, st1 = (count + 1) % S::KS;
          wait(&seen[st], count / S::KS & 1);
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            const uint32_t n = s ? n1 : n0;
            if (j >= n) continue;
            wait(&full_p[s], pph >> s & 1);
            pph ^= 1u << s;
            tc_fence_after();
            if (elect_one()) {
              outputs(s, st, j > 0);
              if (j + 1 == n) umma_commit(&done[s]);
              if (j + 1 < n) scores(s, st1);
              if (j + 2 == n) umma_commit(&empty_q[s]);
            }
            __syncwarp();
          }
          if (elect_one()) {
            umma_commit(&empty_v[st]);
            if (j + 1 < nt) umma_commit(&empty_k[st1]);
          }
          __syncwarp();
        }
      }
      if (*abort) {  // products still in flight must retire before the memory goes
        int drain = 0;
        if (elect_one()) umma_commit(retired);
        __syncwarp();
        (void)mbar_wait(retired, 0u, &drain);
      }
    } else if (warp >= 12) {
      // ---------------- values that are infinite or NaN ----------------
      // (also with nothing to look for these warps see every tile's phase in turn)
      constexpr uint32_t kExp2 = Pair<T>::kExp * 0x10001u;
      constexpr uint32_t kOne2 = (Pair<T>::kExp & (~Pair<T>::kExp + 1)) * 0x10001u;
      const int t128 = threadIdx.x - 384;
      int vs = 0;
      uint32_t vph = 0;
      bool ok = true;
      Work w;
      for (int item = 0;; ++item) {
        const bool live = ok && take(item, w, ok);
        // (the four warps leave together, and clear together the notes of the item
        // before the last)
        uint32_t stop;
        asm volatile(
            "{\n .reg .pred p, q;\n setp.eq.u32 q, %1, 0;\n bar.red.or.pred p, 1, 128, q;\n"
            " selp.u32 %0, 1, 0, p;\n}\n"
            : "=r"(stop)
            : "r"(live ? 1u : 0u)
            : "memory");
        if (stop) break;
        const int used = odd[item & 1];
        asm volatile("bar.sync 1, 128;" ::: "memory");
        if (used) {
          if (t128 < D) first[(item & 1) * D + t128] = kNone;
          odd[item & 1] = 0;
        }
        asm volatile("bar.sync 1, 128;" ::: "memory");
        const int nt = max(w.n0, w.n1), from = max(w.lim0 - w.k0, 0) / kKeys;
        for (int j = 0; j < nt && ok; ++j) {
          ok = __all_sync(0xffffffffu, mbar_wait(&full_v[vs], vph, abort));
          // (one warp also sees every key tile)
          if (warp == 12 && ok) {
            if (j == 0) {
              ok = __all_sync(0xffffffffu, mbar_wait(&full_k[vs], vph, abort));
              if (lane == 0) mbar_arrive(&empty_k[vs]);
            }
            const int vs1 = vs + 1 == S::VS ? 0 : vs + 1;
            if (j + 1 < nt && ok) {
              ok = __all_sync(0xffffffffu,
                              mbar_wait(&full_k[vs1], vph ^ (vs1 == 0 ? 1 : 0), abort));
              if (lane == 0) mbar_arrive(&empty_k[vs1]);
            }
          }
          if (!ok) break;
          if (j >= from) {
            unsigned char* tile = smem + S::V_OFF + vs * S::KV_TILE;
            constexpr int PIECES = S::KV_TILE / 16 / 128;  // of a thread
            uint32_t found = 0;
#pragma unroll 4
            for (int i = 0; i < PIECES; ++i) {
              const uint4 u = *reinterpret_cast<const uint4*>(tile + (t128 + 128 * i) * 16);
              // an exponent of all ones carries into the sign's place
              found |= ((u.x & kExp2) + kOne2) | ((u.y & kExp2) + kOne2) |
                       ((u.z & kExp2) + kOne2) | ((u.w & kExp2) + kOne2);
            }
            if (found & 0x80008000u) {
              for (int i = 0; i < PIECES; ++i) {
                const int p = t128 + 128 * i, row = p / 8 % kKeys, half = p / (8 * kKeys);
                uint16_t* v16 = reinterpret_cast<uint16_t*>(tile + p * 16);
                for (int e = 0; e < 8; ++e) {
                  const uint16_t x = v16[e];
                  if ((x & Pair<T>::kExp) != Pair<T>::kExp) continue;
                  const int d = 64 * half + 8 * ((p & 7) ^ (row & 7)) + e;
                  const bool nan = (x & 0x7FFFu) != Pair<T>::kExp;
                  const uint32_t key = kKeys * (j - from) + row;  // < 128 + 256 + 128
                  const int at = nan ? 20 : 10 * (x >> 15);
                  uint32_t* word = &first[(item & 1) * D + d];
                  uint32_t old = *word;
                  while (key < ((old >> at) & 1023u)) {
                    const uint32_t have =
                        atomicCAS(word, old, (old & ~(1023u << at)) | key << at);
                    if (have == old) break;
                    old = have;
                  }
                  v16[e] = 0;
                }
              }
              odd[item & 1] = 1;
              __threadfence_block();
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          }
          __syncwarp();
          if (lane == 0 && !(a.stall && item == 0 && j == 0 && warp == 15)) mbar_arrive(&seen[vs]);
          if (++vs == S::VS) {
            vs = 0;
            vph ^= 1;
          }
        }
      }
    }
  } else {
    // ---------------- softmax ----------------
    asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    const int s = warp >> 2;  // row tile
    const int row = 32 * (warp & 3) + lane;
    const int g = row / tt;   // head, and token of the row tile
    const int ti = s * tt + row - g * tt;
    const uint32_t lanes = tmem + (static_cast<uint32_t>(32 * (warp & 3)) << 16);
    const uint32_t sc_col = lanes + s * kKeys, o_col = lanes + 2 * kKeys + s * D;
    uint32_t sph = 0, dph = 0;
    // of an item: its first key, the row tile's key tiles, and the keys that the row
    // sees and that all rows of the row tile see (the rest stays in shared memory, which
    // the item keeps until these warps have finished it); by how much a score must pass
    // the row's maximum to raise it
    int k0, n, lim, whole;
    float pass;
    bool more;
    auto begin = [&](int item) {
      Work w;
      bool ok;
      more = take(item, w, ok);
      const AttnRequest rq = {w.q0, w.n, w.kv};
      k0 = w.k0;
      n = s ? w.n1 : w.n0;
      const bool in = g < w.nh && w.i0 + ti < w.n;
      lim = in ? attn_limit(rq, w.i0 + ti) : 0;
      pass = in ? kRaise : INFINITY;  // (a row of no token has no say)
      whole = attn_limit(rq, min(w.i0 + s * tt, w.n - 1));
    };
    begin(0);
    for (int item = 0; more; ++item) {
      float mx = -INFINITY;
      float2 sum[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) sum[x] = make_float2(0.f, 0.f);
      for (int j = 0; j < n; ++j) {
        wait(&full_s[s], sph);
        sph ^= 1;
        tc_fence_after();
        uint32_t v[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld_async<32>(sc_col + 32 * c, v[c]);
        tmem_wait_ld();
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int x = 0; x < 32; ++x) asm volatile("" : "+r"(v[c][x]));  // (not before the wait)
        const int key0 = k0 + kKeys * j;
        if (key0 + kKeys > whole) {
          const int left = lim - key0;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            if (key0 + 32 * c + 32 <= whole) continue;
            const int m = min(max(left - 32 * c, 0), 32);
            const uint32_t keep = m == 32 ? 0xFFFFFFFFu : (1u << m) - 1u;
#pragma unroll
            for (int x = 0; x < 32; ++x)
              if (!(keep & (1u << x))) v[c][x] = 0xFF800000u;
          }
        }
        float t[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          t[c] = __uint_as_float(v[c][0]);
#pragma unroll
          for (int x = 1; x < 31; x += 2)
            t[c] = max3(t[c], __uint_as_float(v[c][x]), __uint_as_float(v[c][x + 1]));
          t[c] = fmaxf(t[c], __uint_as_float(v[c][31]));
        }
        const float top = fmaxf(max3(t[0], t[1], t[2]), t[3]);
        if (__any_sync(0xffffffffu, (top - mx) * a.scale_log2 > pass)) {
          const float to = fmaxf(mx, top);
          const float f = to == -INFINITY ? 1.f : ex2((mx - to) * a.scale_log2);
          mx = to;
#pragma unroll
          for (int x = 0; x < 4; ++x) sum[x] = make_float2(sum[x].x * f, sum[x].y * f);
          if (j > 0) {
#pragma unroll 1
            for (int c = 0; c < D / 16; ++c) {
              uint32_t o[16];
              tmem_ld_async<16>(o_col + 16 * c, o);
              tmem_wait_ld();
#pragma unroll
              for (int x = 0; x < 16; ++x) {
                asm volatile("" : "+r"(o[x]));
                o[x] = __float_as_uint(__uint_as_float(o[x]) * f);
              }
              tmem_st16(o_col + 16 * c, o);
            }
          }
        }
        const float neg = mx == -INFINITY ? 0.f : -mx * a.scale_log2;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t p[16];
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            float2 y = fma2(__uint_as_float(v[c][2 * x]), __uint_as_float(v[c][2 * x + 1]),
                            a.scale_log2, neg);
            y.x = ex2(y.x);
            y.y = ex2(y.y);
            sum[x & 3] = add2(sum[x & 3], y);
            p[x] = Pair<T>::pack(y.x, y.y);
          }
          tmem_st16(sc_col + 16 * c, p);
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&full_p[s]);
      }
      // the row's output: all that can be is got ready while the last product runs, the
      // next item among it
      const Work& w = works[item & 1];
      const int i = w.i0 + ti, keys = n;
      const bool in = g < w.nh && i < w.n;
      const float2 s01 = add2(add2(sum[0], sum[1]), add2(sum[2], sum[3]));
      const float total = s01.x + s01.y;
      const float r = total == 0.f ? 0.f : 1.f / total;  // a row without keys: zeros
      const int64_t at = static_cast<int64_t>(w.q0 + i) * a.heads + w.kh * a.group + w.g0 + g;
      const int64_t zat = static_cast<int64_t>(w.z) * a.tokens * a.heads + at;
      const uint32_t rows_in = __ballot_sync(0xffffffffu, in);
      const bool alone = w.alone;
      char* base = alone ? static_cast<char*>(a.out) + at * (D * 2)
                         : reinterpret_cast<char*>(a.part) + zat * (D * 4);
      const int out_x = w.kh * a.group + w.g0 + g, out_y = w.q0 + i;
      // the notes' keys are counted from there
      const int seen_keys = lim - w.k0 - max(w.lim0 - w.k0, 0) / kKeys * kKeys;
      begin(item + 1);
      if (keys > 0) {
        wait(&done[s], dph);
        dph ^= 1;
        tc_fence_after();
      }
      // 128 bytes of each of the warp's rows at a time, through shared memory (rows in
      // swizzled atoms of eight).  The 32 rows are a box of tokens x heads, or up to four
      // (each is issued by itself, 130 cycles): a TMA store takes it while the warp goes
      // on; those at a request's end, and partial results, are stored by the warp, four
      // rows at a time.
      unsigned char* stage = smem + S::OUT_OFF + warp * 4096;
      const uint32_t mine = smem_u32(stage) + lane * 128;
      auto put = [&](const uint32_t (&o)[32], int off, int c, bool boxes) {
        asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");  // (of this stage)
        __syncwarp();
#pragma unroll
        for (int x = 0; x < 8; ++x)
          asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(mine + ((x ^ (lane & 7)) * 16)),
                       "r"(o[4 * x]), "r"(o[4 * x + 1]), "r"(o[4 * x + 2]), "r"(o[4 * x + 3])
                       : "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        uint32_t left = rows_in;
        if (boxes) {
          const uint32_t all = a.box_rows == 32 ? ~0u : (1u << a.box_rows) - 1;
          const int b0 = lane & ~(a.box_rows - 1);
          const bool whole = (rows_in >> b0 & all) == all;  // all are tokens of the request
          if (lane == b0 && whole)
            asm volatile(
                "cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(
                    reinterpret_cast<uint64_t>(&maps.out)),
                "r"(64 * c), "r"(out_y), "r"(out_x), "r"(mine)
                : "memory");
          asm volatile("cp.async.bulk.commit_group;" ::: "memory");
          const uint32_t some = __ballot_sync(0xffffffffu, !whole);
          left &= some;
          if (left == 0) return;
        }
        const uint32_t from = smem_u32(stage) + (lane >> 3) * 128;
#pragma unroll 1
        for (int x = 0; x < 8; ++x) {
          const int row = 4 * x + (lane >> 3);
          uint4 u;
          asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                       : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w)
                       : "r"(from + x * 512 + (((lane & 7) ^ (row & 7)) * 16))
                       : "memory");
          char* dst = reinterpret_cast<char*>(
              __shfl_sync(0xffffffffu, reinterpret_cast<uintptr_t>(base), row));
          if (left >> row & 1) *reinterpret_cast<uint4*>(dst + off + (lane & 7) * 16) = u;
        }
      };
      const uint32_t keep = keys > 0 ? 0xFFFFFFFFu : 0u;  // (else nothing was added up there)
      // (Compact code, each path in a loop of its own: it runs once an item, out of
      // the instruction caches.)
      if (alone) {
#pragma unroll 1
        for (int c = 0; c < D / 64; ++c) {
          uint32_t o[2][32];
          tmem_ld_async<32>(o_col + 64 * c, o[0]);
          tmem_ld_async<32>(o_col + 64 * c + 32, o[1]);
          tmem_wait_ld();
          uint32_t p[32];
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int x = 0; x < 16; ++x) {
              asm volatile("" : "+r"(o[h][2 * x]), "+r"(o[h][2 * x + 1]));
              const float2 y = mul2(__uint_as_float(o[h][2 * x]), __uint_as_float(o[h][2 * x + 1]), r);
              p[16 * h + x] = Pair<T>::pack(y.x, y.y) & keep;
            }
          if (keys > 0 && c == D / 64 - 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&free_o[s]);
          }
          put(p, 128 * c, c, true);
        }
      } else {
#pragma unroll 1
        for (int c = 0; c < D / 32; ++c) {
          uint32_t o[32];
          tmem_ld32(o_col + 32 * c, o);
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            asm volatile("" : "+r"(o[2 * x]), "+r"(o[2 * x + 1]));
            const float2 y = mul2(__uint_as_float(o[2 * x]), __uint_as_float(o[2 * x + 1]), r);
            o[2 * x] = __float_as_uint(y.x) & keep;
            o[2 * x + 1] = __float_as_uint(y.y) & keep;
          }
          if (keys > 0 && c == D / 32 - 1) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&free_o[s]);
          }
          put(o, 128 * c, c, false);
        }
        if (in) a.part_lse[zat] = total == 0.f ? -INFINITY : mx * a.scale_log2 + log2f(total);
      }
      if (odd[item & 1]) {  // infinite and NaN values that the row sees
        const uint32_t* notes = first + (item & 1) * D;
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");  // (the rows are stored)
        asm volatile("fence.proxy.async;" ::: "memory");
        __syncwarp();
#pragma unroll 1
        for (int d = 0; d < D && in; ++d) {
          const uint32_t f = notes[d];
          float y = 0.f;
          if (static_cast<int>(f & 1023u) < seen_keys) y += INFINITY;
          if (static_cast<int>((f >> 10) & 1023u) < seen_keys) y -= INFINITY;
          if (static_cast<int>(f >> 20) < seen_keys) y = NAN;
          if (y == 0.f) continue;
          if (alone) {
            uint16_t* at16 = reinterpret_cast<uint16_t*>(base) + d;
            *at16 = static_cast<uint16_t>(Pair<T>::pack(y + Pair<T>::value(*at16), 0.f));
          } else {
            reinterpret_cast<float*>(base)[d] += y;
          }
        }
        __syncwarp();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&empty_w[item & 1]);
    }
    asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  if (*abort && threadIdx.x == 0 && a.status != nullptr) atomicOr(a.status, SSS_FLAG_TIMEOUT);
  if (warp == 8) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem),
                 "r"(kTmemCols)
                 : "memory");
  }
}

CUresult encode(EncodeTiledFn enc, CUtensorMap* map, CUtensorMapDataType type, const void* base,
                int64_t width, int64_t rows, int64_t stride, int box_rows) {
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(width), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(stride) * 2};
  const cuuint32_t box[2] = {64, static_cast<cuuint32_t>(box_rows)};
  const cuuint32_t estr[2] = {1, 1};
  return enc(map, type, 2, const_cast<void*>(base), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

// boxes of 64 columns x tokens x heads
CUresult encode_heads(EncodeTiledFn enc, CUtensorMap* map, CUtensorMapDataType type,
                      const void* base, int heads, int dim, int64_t tokens, int64_t stride,
                      int box_tokens, int box_heads) {
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(dim), static_cast<cuuint64_t>(tokens),
                              static_cast<cuuint64_t>(heads)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(stride) * 2,
                                 static_cast<cuuint64_t>(dim) * 2};
  const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(box_tokens),
                             static_cast<cuuint32_t>(box_heads)};
  const cuuint32_t estr[3] = {1, 1, 1};
  return enc(map, type, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

template <typename T, int D>
cudaError_t run_prompt(AttnArgs a, cudaStream_t stream) {
  EncodeTiledFn enc = tensor_map_encoder();
  if (enc == nullptr) return cudaErrorNotSupported;
  const CUtensorMapDataType type = std::is_same<T, __half>::value
                                       ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                       : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  const int box = a.table ? std::min(kKeys, 1 << a.page_shift) : kKeys;
  AttnMaps maps;
  const int tt = a.tpt / 2;
  // the output's boxes: tokens (a power of two that divides a row tile's) x heads
  const int bt = std::min(tt & -tt, 32), bh = bt == tt ? 32 / bt : 1;
  a.box_rows = bt * bh;
  if (encode_heads(enc, &maps.q, type, a.q, a.heads, D, a.tokens, a.q_stride, tt, a.hpt) !=
          CUDA_SUCCESS ||
      encode(enc, &maps.k, type, a.k, static_cast<int64_t>(a.kv_heads) * D, a.slots, a.kv_stride,
             box) != CUDA_SUCCESS ||
      encode(enc, &maps.v, type, a.v, static_cast<int64_t>(a.kv_heads) * D, a.slots, a.kv_stride,
             box) != CUDA_SUCCESS ||
      encode_heads(enc, &maps.out, type, a.out, a.heads, D, a.tokens,
                   static_cast<int64_t>(a.heads) * D, bt, bh) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;
  auto kern = attn_prompt_kernel<T, D>;
  cudaError_t e = ensure_smem(kern, PromptSmem<D>::TOTAL);
  if (e != cudaSuccess) return e;
  const int64_t blocks = static_cast<int64_t>(a.tiles) * a.kv_heads * a.hchunks * a.nsplit;
  if (blocks < 1 || blocks > INT32_MAX) return cudaErrorNotSupported;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(blocks));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = PromptSmem<D>::TOTAL;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, maps, a);
}

}  // namespace

cudaError_t launch_attn_prompt(const AttnArgs& a, int dtype, int dim, cudaStream_t stream) {
  if (dtype == SSS_OUT_F16)
    return dim == 64 ? run_prompt<__half, 64>(a, stream) : run_prompt<__half, 128>(a, stream);
  return dim == 64 ? run_prompt<__nv_bfloat16, 64>(a, stream)
                   : run_prompt<__nv_bfloat16, 128>(a, stream);
}

}  // namespace sss
