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
//             O += P V with P from tensor memory;
//   warp 9    TMA producer of Q, K and V (a box per page, or per 128 packed keys);
//   warps 10-11  look through V tiles that some row does not see whole.
// Rows are tokens x the heads that share a key/value head (head-major, so that a TMA
// box brings a head's tokens): all heads of a group see almost the same keys, a
// tile spans few tokens, and little of the last key tile is masked.
//
// The maximum is raised only where a score passes it by 8 powers of two: until then
// p stays within 2^8 and nothing has to be rescaled.  (O of the tile lies in
// tensor memory, and a row's thread rescales it there between the scores' arrival,
// which says that the previous product has completed, and the next one's start.)
//
// A value that is infinite or NaN must not reach rows that do not see its key (0 x
// NaN would).  In tiles that every row of the CTA sees it cannot do harm; in the others
// warps 10-11 replace it by zero and note the first key of each kind for its
// column, and the rows that see that key add it at the end.
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

constexpr int kThreads = 384;
constexpr int kKeys = 128;      // of a tile
constexpr float kRaise = 8.0f;  // powers of two
constexpr int kTmemCols = 512;  // one CTA per SM

struct AttnMaps {
  CUtensorMap q, k, v;
};

template <int D>
struct PromptSmem {
  static constexpr int HALVES = D / 64;             // 128-byte wide parts of a row
  static constexpr int PART = 128 * 128;            // a part of 128 rows
  static constexpr int Q_TILE = HALVES * PART;
  static constexpr int KV_TILE = HALVES * PART;
  static constexpr int KS = D == 128 ? 2 : 4;       // key and value tiles in flight
  static constexpr int VS = D == 128 ? 3 : 4;
  static constexpr int K_OFF = 2 * Q_TILE;
  static constexpr int V_OFF = K_OFF + KS * KV_TILE;
  static constexpr int FIRST_OFF = V_OFF + VS * KV_TILE;  // int [3][D]
  static constexpr int BAR_OFF = FIRST_OFF + 3 * D * 4;
  static constexpr int NBAR = 2 + 2 * KS + 3 * VS + 3 * 2 + 1;
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

// V as a B operand: 64 values of d are one 128-byte row of a swizzled part, 8 keys an
// atom of 1024 bytes; the next 64 values lie a part further.
__device__ __forceinline__ uint64_t mn_desc(uint32_t saddr, uint32_t part) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
  d |= static_cast<uint64_t>(part >> 4) << 16;
  d |= static_cast<uint64_t>(1024 >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(2) << 61;
  return d;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                       uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(acc)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc,
                                       uint32_t acc) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(acc)
      : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_wait_st() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
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
__device__ __forceinline__ float2 add2(float2 x, float2 y) {
  float2 r;
  asm("{\n .reg .b64 a, b, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n"
      " add.rn.f32x2 d, a, b;\n mov.b64 {%0, %1}, d;\n}\n"
      : "=f"(r.x), "=f"(r.y)
      : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y));
  return r;
}

// What the CTA works on: two row tiles of `tt` tokens each.
struct PromptWork {
  AttnRequest rq;
  int b, kh, g0, nh, i0, tt, z;
  int k0;        // first key of the split
  int lim0;      // keys that the first token sees
  int n[2];      // key tiles of A, B
};

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 1)
    attn_prompt_kernel(const __grid_constant__ AttnMaps maps, const __grid_constant__ AttnArgs a) {
  using S = PromptSmem<D>;
  extern __shared__ unsigned char smem_raw[];
  // 1024-byte alignment for the swizzle atoms
  unsigned char* smem = reinterpret_cast<unsigned char*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  int* first = reinterpret_cast<int*>(smem + S::FIRST_OFF);  // [+inf, -inf, NaN][D]
  uint64_t* full_q = reinterpret_cast<uint64_t*>(smem + S::BAR_OFF);
  uint64_t* full_k = full_q + 2;
  uint64_t* empty_k = full_k + S::KS;
  uint64_t* full_v = empty_k + S::KS;
  uint64_t* seen_v = full_v + S::VS;   // looked through
  uint64_t* empty_v = seen_v + S::VS;
  uint64_t* full_s = empty_v + S::VS;  // scores are there (and earlier products done)
  uint64_t* full_p = full_s + 2;
  uint64_t* done = full_p + 2;         // the row tile's output is complete
  uint64_t* retired = done + 2;        // used when a wait has run out
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(retired + 1);
  volatile int* abort = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* odd = reinterpret_cast<int*>(tmem_slot + 2);  // `first` holds something

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  // this CTA's work
  uint32_t flags = 0;
  PromptWork w;
  const int hx = (blockIdx.x / a.nsplit) % (a.kv_heads * a.hchunks);
  w.z = blockIdx.x % a.nsplit;
  w.kh = hx / a.hchunks;
  w.g0 = hx % a.hchunks * a.hpt;
  w.nh = min(a.hpt, a.group - w.g0);
  w.tt = a.tpt / 2;
  if (!attn_tile(a, blockIdx.x / (a.nsplit * a.kv_heads * a.hchunks), w.b, w.i0)) return;
  w.rq = attn_request(a, w.b, flags);
  if (flags && a.status && threadIdx.x == 0) atomicOr(a.status, flags);
  flags = 0;
  if (w.i0 >= w.rq.n) return;
  w.k0 = w.z * a.chunk;
  w.lim0 = attn_limit(w.rq, w.i0);
  int lim1 = w.lim0;  // keys that the last token sees
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const int i = w.i0 + s * w.tt, last = min(i + w.tt, w.rq.n) - 1;
    w.n[s] = 0;
    if (last < i) continue;
    lim1 = attn_limit(w.rq, last);
    w.n[s] = max(0, (min(lim1, w.k0 + a.chunk) - w.k0 + kKeys - 1) / kKeys);
  }
  const bool alone = lim1 <= a.chunk;  // no other split has keys
  const int nt = max(w.n[0], w.n[1]);
  if (nt == 0 && w.z > 0) return;

  if (threadIdx.x == 0) {
    for (int s = 0; s < 2; ++s) {
      mbar_init(&full_q[s], 1);
      mbar_init(&full_s[s], 1);
      mbar_init(&full_p[s], 4);
      mbar_init(&done[s], 1);
    }
    for (int s = 0; s < S::KS; ++s) {
      mbar_init(&full_k[s], 1);
      mbar_init(&empty_k[s], 1);
    }
    for (int s = 0; s < S::VS; ++s) {
      mbar_init(&full_v[s], 1);
      mbar_init(&seen_v[s], 2);
      mbar_init(&empty_v[s], 1);
    }
    mbar_init(retired, 1);
    *abort = 0;
    *odd = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  for (int i = threadIdx.x; i < 3 * D; i += kThreads) first[i] = INT32_MAX;
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

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == 9) {
      // ---------------- TMA producer ----------------
      const int box = a.table ? min(kKeys, 1 << a.page_shift) : kKeys;  // keys of a box
      const int boxes = kKeys / box * S::HALVES;
      const int my = lane / S::HALVES, half = lane % S::HALVES;
      const int32_t* table =
          a.table ? a.table + static_cast<int64_t>(w.b) * a.table_width : nullptr;
      // Lane l brings box l of a tile: its first slot.  Boxes behind the keys, or of
      // a page that is none, lie past the cache and read as zeros.
      auto entry = [&](int j) -> int {
        const int key = w.k0 + kKeys * j + my * box;
        return table && lane < boxes && j < nt && key < w.rq.kv
                   ? __ldg(table + (key >> a.page_shift))
                   : -1;
      };
      auto slot_of = [&](int page, int j) -> int {
        const int key = w.k0 + kKeys * j + my * box;
        if (key >= w.rq.kv || lane >= boxes) return static_cast<int>(a.slots);
        if (!table) return w.rq.q0 + key;
        const int64_t s = attn_slot(a, page, key);
        if (s < 0) flags |= SSS_FLAG_INDEX;
        return static_cast<int>(s < 0 ? a.slots : s);
      };
      if (elect_one()) {
        for (int s = 0; s < 2; ++s) {
          if (w.n[s] == 0) continue;
          mbar_arrive_expect_tx(&full_q[s], w.nh * w.tt * 128 * S::HALVES);
          for (int g = 0; g < w.nh; ++g)
            for (int h = 0; h < S::HALVES; ++h)
              tma_load_2d(&maps.q, &full_q[s],
                          smem + s * S::Q_TILE + h * S::PART + g * w.tt * 128,
                          (w.kh * a.group + w.g0 + g) * D + 64 * h, w.rq.q0 + w.i0 + s * w.tt);
        }
      }
      __syncwarp();
      int page = entry(0), j = 0;
      bool ok = true;
      for (; j < nt; ++j) {
        const int slot = slot_of(page, j);
        page = entry(j + 1);
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          const int stages = kv ? S::VS : S::KS, st = j % stages;
          uint64_t* full = (kv ? full_v : full_k) + st;
          ok = ok && __all_sync(0xffffffffu, mbar_wait((kv ? empty_v : empty_k) + st,
                                                       ((j / stages) & 1) ^ 1, abort));
          if (!ok) break;
          if (lane == 0) mbar_arrive_expect_tx(full, S::KV_TILE);
          __syncwarp();
          if (lane < boxes)
            tma_load_2d(kv ? &maps.v : &maps.k, full,
                        smem + (kv ? S::V_OFF : S::K_OFF) + st * S::KV_TILE + half * S::PART +
                            my * box * 128,
                        w.kh * D + 64 * half, slot);
          __syncwarp();
        }
        if (!ok) break;
      }
      if (flags && a.status) atomicOr(a.status, flags);
      if (!ok) {
        // let this CTA's copies still in flight land (of a barrier never used, the
        // phase before its first counts as completed); tile j may have its keys only
        int drain = 0;
        for (int s = 0; s < 2; ++s)
          if (w.n[s] > 0) (void)mbar_wait(&full_q[s], 0, &drain);
        for (int i = max(0, j - S::KS + 1); i <= j; ++i) {
          const uint32_t par = (i / S::KS) & 1;
          // (tile j's keys, where they were not asked for, are the stage's last ones)
          if (i < j || mbar_test_wait(&empty_k[i % S::KS], par ^ 1u))
            (void)mbar_wait(&full_k[i % S::KS], par, &drain);
        }
        for (int i = max(0, j - S::VS); i < j; ++i)
          (void)mbar_wait(&full_v[i % S::VS], (i / S::VS) & 1, &drain);
      }
    } else if (warp == 8) {
      // ---------------- issuer of the products ----------------
      constexpr uint32_t id_s = idesc_of<T>(kKeys, false), id_o = idesc_of<T>(D, true);
      const uint32_t tm = __reduce_or_sync(0xffffffffu, tmem);
      const uint32_t base = smem_u32(smem);
      auto wait = [&](uint64_t* bar, uint32_t parity) -> bool {
        return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort));
      };
      auto scores = [&](int s, int j) {  // S_s = Q_s K_j^T
        if (elect_one()) {
#pragma unroll
          for (int h = 0; h < S::HALVES; ++h) {
            const uint64_t qd = sw128_desc(base + s * S::Q_TILE + h * S::PART);
            const uint64_t kd =
                sw128_desc(base + S::K_OFF + (j % S::KS) * S::KV_TILE + h * S::PART);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              mma_ss(tm + s * kKeys, qd + 2 * kk, kd + 2 * kk, id_s, h + kk > 0);
          }
          umma_commit(&full_s[s]);
        }
        __syncwarp();
      };
      bool go = true;
      for (int s = 0; s < 2; ++s)
        if (w.n[s] > 0) go = go && wait(&full_q[s], 0);
      if (nt > 0) go = go && wait(&full_k[0], 0);
      tc_fence_after();
      if (go && nt > 0) {
        for (int s = 0; s < 2; ++s)
          if (w.n[s] > 0) scores(s, 0);
        if (elect_one()) umma_commit(&empty_k[0]);
        __syncwarp();
      }
      for (int j = 0; j < nt && go; ++j) {
        go = wait(&seen_v[j % S::VS], (j / S::VS) & 1);
        const uint32_t vbase = base + S::V_OFF + (j % S::VS) * S::KV_TILE;
        bool have_k = false;
        for (int s = 0; s < 2 && go; ++s) {
          if (j >= w.n[s]) continue;
          go = wait(&full_p[s], j & 1);
          if (!go) break;
          tc_fence_after();
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < kKeys / 16; ++kk)  // O_s += P_s V_j
              mma_ts(tm + 2 * kKeys + s * D, tm + s * kKeys + 8 * kk,
                     mn_desc(vbase + kk * 2048, S::PART), id_o, j + kk > 0);
            if (j + 1 == w.n[s]) umma_commit(&done[s]);
          }
          __syncwarp();
          if (j + 1 < w.n[s]) {
            if (!have_k) {
              go = wait(&full_k[(j + 1) % S::KS], ((j + 1) / S::KS) & 1);
              if (!go) break;
              tc_fence_after();
              have_k = true;
            }
            scores(s, j + 1);
          }
        }
        if (!go) break;
        if (elect_one()) {
          umma_commit(&empty_v[j % S::VS]);
          if (j + 1 < nt) umma_commit(&empty_k[(j + 1) % S::KS]);
        }
        __syncwarp();
      }
      if (*abort) {  // products still in flight must retire before the memory goes
        int drain = 0;
        if (elect_one()) umma_commit(retired);
        __syncwarp();
        (void)mbar_wait(retired, 0u, &drain);
      }
    } else {
      // ---------------- values that are infinite or NaN ----------------
      // (also with nothing to look for these warps see every tile's phase in turn)
      constexpr uint32_t kExp2 = Pair<T>::kExp * 0x10001u;
      constexpr uint32_t kOne2 = (Pair<T>::kExp & (~Pair<T>::kExp + 1)) * 0x10001u;
      const int t64 = threadIdx.x - 320;
      for (int j = 0; j < nt; ++j) {
        const int st = j % S::VS;
        if (!__all_sync(0xffffffffu, mbar_wait(&full_v[st], (j / S::VS) & 1, abort))) break;
        const int key0 = w.k0 + kKeys * j;
        if (key0 + kKeys > w.lim0) {
          unsigned char* tile = smem + S::V_OFF + st * S::KV_TILE;
          constexpr int PIECES = S::KV_TILE / 16 / 64;  // of a thread
          uint32_t found = 0;
#pragma unroll 8
          for (int i = 0; i < PIECES; ++i) {
            const uint4 u = *reinterpret_cast<const uint4*>(tile + (t64 + 64 * i) * 16);
            // an exponent of all ones carries into the sign's place
            found |= ((u.x & kExp2) + kOne2) | ((u.y & kExp2) + kOne2) |
                     ((u.z & kExp2) + kOne2) | ((u.w & kExp2) + kOne2);
          }
          if (found & 0x80008000u) {
            for (int i = 0; i < PIECES; ++i) {
              const int p = t64 + 64 * i, row = p / 8 % kKeys, half = p / (8 * kKeys);
              uint16_t* v16 = reinterpret_cast<uint16_t*>(tile + p * 16);
              for (int e = 0; e < 8; ++e) {
                const uint16_t x = v16[e];
                if ((x & Pair<T>::kExp) != Pair<T>::kExp) continue;
                const int d = 64 * half + 8 * ((p & 7) ^ (row & 7)) + e;
                const bool nan = (x & 0x7FFFu) != Pair<T>::kExp;
                atomicMin(&first[(nan ? 2 : x >> 15) * D + d], key0 + row);
                v16[e] = 0;
              }
            }
            *odd = 1;
            __threadfence_block();
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        __syncwarp();
        if (lane == 0 && !(a.stall && j == 0 && warp == 11)) mbar_arrive(&seen_v[st]);
      }
    }
  } else {
    // ---------------- softmax ----------------
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    const int s = warp >> 2;  // row tile
    const int row = 32 * (warp & 3) + lane;
    const int g = row / w.tt, i = w.i0 + s * w.tt + row - g * w.tt;
    const bool in = g < w.nh && i < w.rq.n;
    const int lim = in ? attn_limit(w.rq, i) : 0;
    // keys that all rows of the row tile see
    const int whole = attn_limit(w.rq, min(w.i0 + s * w.tt, w.rq.n - 1));
    const uint32_t lanes = tmem + (static_cast<uint32_t>(32 * (warp & 3)) << 16);
    const uint32_t sc_col = lanes + s * kKeys, o_col = lanes + 2 * kKeys + s * D;
    float mx = -INFINITY;
    float2 sum = make_float2(0.f, 0.f);
    bool ok = true;
    const int n = w.n[s];
    for (int j = 0; j < n; ++j) {
      ok = __all_sync(0xffffffffu, mbar_wait(&full_s[s], j & 1, abort));
      if (!ok) break;
      tc_fence_after();
      uint32_t v[4][32];
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld_async<32>(sc_col + 32 * c, v[c]);
      tmem_wait_ld();
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int x = 0; x < 32; ++x) asm volatile("" : "+r"(v[c][x]));  // (not before the wait)
      const int key0 = w.k0 + kKeys * j;
      if (key0 + kKeys > whole) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int x = 0; x < 32; ++x)
            if (key0 + 32 * c + x >= lim) v[c][x] = 0xFF800000u;
      }
      float t[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        t[c] = __uint_as_float(v[c][0]);
#pragma unroll
        for (int x = 1; x < 32; ++x) t[c] = fmaxf(t[c], __uint_as_float(v[c][x]));
      }
      const float top = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
      if (__any_sync(0xffffffffu, (top - mx) * a.scale_log2 > kRaise)) {
        const float to = fmaxf(mx, top);
        const float f = to == -INFINITY ? 1.f : ex2((mx - to) * a.scale_log2);
        mx = to;
        sum.x *= f;
        sum.y *= f;
        if (j > 0) {
#pragma unroll
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
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          uint32_t p[8];
#pragma unroll
          for (int x = 0; x < 8; ++x) {
            float2 y = fma2(__uint_as_float(v[c][16 * hf + 2 * x]),
                            __uint_as_float(v[c][16 * hf + 2 * x + 1]), a.scale_log2, neg);
            y.x = ex2(y.x);
            y.y = ex2(y.y);
            sum = add2(sum, y);
            p[x] = Pair<T>::pack(y.x, y.y);
          }
#pragma unroll
          for (int x = 0; x < 8; ++x) v[c][8 * hf + x] = p[x];
        }
        uint32_t st[16];
#pragma unroll
        for (int x = 0; x < 16; ++x) st[x] = v[c][x];
        tmem_st16(sc_col + 16 * c, st);
      }
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&full_p[s]);
    }
    // the row's output
    if (n > 0 && ok) ok = __all_sync(0xffffffffu, mbar_wait(&done[s], 0, abort));
    if (ok) {
      tc_fence_after();
      const float total = sum.x + sum.y;
      const float r = total == 0.f ? 0.f : 1.f / total;  // a row without keys: zeros
      const int64_t at = static_cast<int64_t>(w.rq.q0 + i) * a.heads + w.kh * a.group + w.g0 + g;
      const int64_t zat = static_cast<int64_t>(w.z) * a.tokens * a.heads + at;
      const bool mark = *reinterpret_cast<volatile int*>(odd) != 0;
#pragma unroll 1
      for (int c = 0; c < D / 32; ++c) {
        uint32_t o[32];
        if (n > 0) {
          tmem_ld32(o_col + 32 * c, o);
#pragma unroll
          for (int x = 0; x < 32; ++x) asm volatile("" : "+r"(o[x]));
        } else {
#pragma unroll
          for (int x = 0; x < 32; ++x) o[x] = 0;
        }
        if (in) {
#pragma unroll
          for (int x = 0; x < 32; ++x) {
            float y = __uint_as_float(o[x]) * r;
            if (mark) {
              const int d = 32 * c + x;
              if (first[d] < lim) y += INFINITY;
              if (first[D + d] < lim) y -= INFINITY;
              if (first[2 * D + d] < lim) y = NAN;
            }
            o[x] = __float_as_uint(y);
          }
          if (alone) {
            uint4* dst = reinterpret_cast<uint4*>(static_cast<T*>(a.out) + at * D + 32 * c);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const uint32_t* y = o + 8 * x;
              dst[x] = make_uint4(Pair<T>::pack(__uint_as_float(y[0]), __uint_as_float(y[1])),
                                  Pair<T>::pack(__uint_as_float(y[2]), __uint_as_float(y[3])),
                                  Pair<T>::pack(__uint_as_float(y[4]), __uint_as_float(y[5])),
                                  Pair<T>::pack(__uint_as_float(y[6]), __uint_as_float(y[7])));
            }
          } else {
            uint4* dst = reinterpret_cast<uint4*>(a.part + zat * D + 32 * c);
#pragma unroll
            for (int x = 0; x < 8; ++x)
              dst[x] = make_uint4(o[4 * x], o[4 * x + 1], o[4 * x + 2], o[4 * x + 3]);
          }
        }
        __syncwarp();
      }
      if (in && !alone)
        a.part_lse[zat] = total == 0.f ? -INFINITY : mx * a.scale_log2 + log2f(total);
    }
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

template <typename T, int D>
cudaError_t run_prompt(const AttnArgs& a, cudaStream_t stream) {
  EncodeTiledFn enc = tensor_map_encoder();
  if (enc == nullptr) return cudaErrorNotSupported;
  const CUtensorMapDataType type = std::is_same<T, __half>::value
                                       ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                       : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  const int box = a.table ? std::min(kKeys, 1 << a.page_shift) : kKeys;
  AttnMaps maps;
  if (encode(enc, &maps.q, type, a.q, static_cast<int64_t>(a.heads) * D, a.tokens, a.q_stride,
             a.tpt / 2) != CUDA_SUCCESS ||
      encode(enc, &maps.k, type, a.k, static_cast<int64_t>(a.kv_heads) * D, a.slots, a.kv_stride,
             box) != CUDA_SUCCESS ||
      encode(enc, &maps.v, type, a.v, static_cast<int64_t>(a.kv_heads) * D, a.slots, a.kv_stride,
             box) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;
  auto kern = attn_prompt_kernel<T, D>;
  cudaError_t e = ensure_smem(kern, PromptSmem<D>::TOTAL);
  if (e != cudaSuccess) return e;
  const int64_t blocks = static_cast<int64_t>(a.tiles) * a.kv_heads * a.hchunks * a.nsplit;
  if (blocks > INT32_MAX) return cudaErrorNotSupported;
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
