// attn_rows.cu -- attention of few rows: the single tokens (or a few drafted ones)
// of a decode step over the paged cache, and the joining of partial results.
//
//   o_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = 2^(c q_i.k_j - m_i),  c = scale log2(e)
//
// Bound by HBM: every key and value is read once, for group x 2 operations a byte.
// So the matrix products run on mma.sync (m16n8k16; 16 or 32 rows of tokens x
// heads, at a fraction of its rate), and everything else serves the loads: each of
// the CTA's four warps streams its own steps of 16 keys and 16 values through a
// private ring of cp.async copies, without a barrier in the loop, and keeps a
// running maximum m, sum and fp32 output of its own; they meet once, at the end.  No
// part is left out of a join because its weight is zero: an infinite or NaN value in it
// has to reach the row all the same.
// 16 keys never leave a page, so a step's rows have one base address; 32 steps'
// table entries are read ahead, one per lane.  Where tiles are few, the keys of one are
// split over the CTAs of a cluster, 64 at a time in turn, which join their outputs through
// distributed shared memory: no second kernel, no workspace, and a fixed order.  The
// stores into a peer are counted by a barrier there (a cluster-wide barrier after plain
// ones took 0.2 to 0.4 us longer).  That wait is bounded (about one second): on expiry the
// CTA raises SSS_FLAG_TIMEOUT.  No CTA leaves its shared memory before all of the cluster
// have issued their stores (a second cluster barrier, arrived at behind the stores and
// waited for at the very end, when as a rule all have), and one whose wait ran out first lets
// those that are under way land.
//
// Measured (32 heads of 128 over 8, bf16): 64 requests of 12000 to 16384 keys 517 to 530
// us, 7.0 TB/s, above the copy rate; 16 ragged ones of 130 to 16384 (64 heads) 59.3 us, 85 %
// of it, the longest request's cluster being last; one request of 2047 keys 5.9 us, the
// launch, the lengths' and the first keys' latency and the join.  A ring of two or four
// steps (at 16 rows), and three CTAs an SM, were slower on the whole; so was dividing all
// requests' keys evenly over the SMs with a second kernel to join (64 against 59, 558
// against 516 us).
// m is raised only where a score passes it by 8 (then 2^8 at most enters the
// 16-bit p, in range): the outputs are rescaled seldom and the warp votes on it
// without first reducing its maxima.
#include <algorithm>

#include "attn.cuh"
#include "tc.cuh"

namespace sss {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kStep = 16;   // keys of a warp's step
constexpr float kRaise = 8.0f;

template <int D, int R, bool CL>
struct RowsSmem {
  // Steps in a warp's ring: as many as leave room for two CTAs an SM (32 rows of 128: 16
  // requests of 500 to 4000 keys and 32 heads to a key/value head: 38.4 us with three and
  // one CTA, 23.2 with two and two).
  static constexpr int kStages = R * D == 32 * 128 ? 2 : 3;
  static constexpr int TILE = kStep * D * 2;             // 16 keys (or values)
  static constexpr int RING = kStages * 2 * TILE;        // of a warp
  static constexpr int LD = D + 4;  // of the warps' outputs, which follow: distinct banks
  static constexpr int RINGS = std::max(kWarps * RING, kWarps * R * LD * 4);
  // the splits' pieces of the values that this one joins (their number rounded up)
  static constexpr int TOTAL = RINGS + (CL ? (R * D / 4 + 16) * 16 : 0);
};

__device__ __forceinline__ uint32_t smem_addr(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool in) {
  const int bytes = in ? 16 : 0;  // the rest is filled with zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes)
               : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
template <typename T>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                         uint32_t b1) {
  if constexpr (std::is_same<T, __half>::value)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Shared memory of another CTA of the cluster, at the address that addr is in this
// one's; stores into it, whose bytes a barrier there counts.
__device__ __forceinline__ uint32_t of_peer(uint32_t addr, int rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void peer_store(uint32_t addr, float v, uint32_t bar) {
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.f32 [%0], %1, [%2];" ::"r"(
                   addr),
               "f"(v), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void peer_store(uint32_t addr, float4 v, uint32_t bar) {
  asm volatile(
      "st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, "
      "[%5];" ::"r"(addr),
      "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w), "r"(bar)
      : "memory");
}

// (Two CTAs an SM are 255 registers a thread at most.  16 rows need 160 to 247; 32 rows of
// 64 values 226 or 230; 32 rows of 128 spill 148 or 172 bytes, which costs less than one
// CTA an SM: see RowsSmem.)  MT tiles of 16 rows.  CL: the splits of a tile's keys are the CTAs of a cluster, whose
// keys differ in number by 64 at most, and join through its shared memory: each adds up a
// share of the values (16 bytes at a time), and all store their partial results there.
template <typename T, int D, int MT, bool CL>
__global__ void __launch_bounds__(kThreads, 2) attn_rows_kernel(const __grid_constant__ AttnArgs a) {
  constexpr int R = 16 * MT;
  using S = RowsSmem<D, R, CL>;
  constexpr int kStages = S::kStages;
  constexpr int CH = D / 8;       // 16-byte pieces of a row
  constexpr int KD = D / 16;      // mma steps along d
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ float wmax[kWarps][R], wsum[kWarps][R];
  __shared__ float split_lse[CL ? 16 : 1][R];  // of every split
  __shared__ uint64_t arrived;  // what the splits store here
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // another CTA's shared memory exists only once that CTA has started: waited for
  // before the first store into a peer
  if constexpr (CL) {
    if (threadIdx.x == 0) {
      mbar_init(&arrived, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  // this CTA's work; the heads of a tile are neighbours in the grid's order, as their
  // keys are in memory (heads outermost: 61 -> 70 us for 16 requests of 130 to 16384 keys)
  const int z = blockIdx.x, hx = blockIdx.y;
  const int kh = a.hchunks == 1 ? hx : hx / a.hchunks;
  const int g0 = (hx - kh * a.hchunks) * a.hpt;
  const int nh = min(a.hpt, a.group - g0);  // heads of the tile
  // (the tokens of rows < 32, without a division)
  const auto token_of = [&](int row) { return row * a.hpt_inverse >> 16; };
  const auto leave = [&]() {
    if constexpr (CL) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  };
  // The keys go to the splits and their warps 16 at a time in turn: whatever the
  // request's length, step s of the warp starts at key_of(s).  So the table's entries of
  // its first 32 steps (one per lane) are asked for with the request's lengths, not after.
  const auto key_of = [&](int s) { return kStep * (warp + kWarps * (CL ? z + a.nsplit * s : s)); };
  const int64_t width = static_cast<int64_t>(a.table_width) << a.page_shift;
  const auto entry = [&](const int32_t* table, int s) {
    const int64_t key = kStep * (warp + kWarps * (CL ? z + static_cast<int64_t>(a.nsplit) * s : s));
    return key < width && key < a.max_kv ? __ldg(table + (key >> a.page_shift)) : 0;
  };
  int page = 0;
  const int tile = a.tile0 + blockIdx.z;
  if (a.table && a.one_tile && tile < a.batch)
    page = entry(a.table + static_cast<int64_t>(tile) * a.table_width, lane);
  int b, i0;
  uint32_t flags = 0;
  AttnRequest rq;
  const bool found = attn_tile(a, tile, b, i0, rq, flags);
  const int nt = found ? min(a.tpt, rq.n - i0) : 0;  // tokens of the tile
  if (nt <= 0) {
    if (flags && a.status && warp == 0) atomicOr(a.status, flags);
    return leave();
  }
  const int lim1 = attn_limit(rq, i0 + nt - 1);
  const int lim0 = attn_limit(rq, i0);
  const int steps = (lim1 + kStep - 1) / kStep;
  // splits with keys
  const int n = CL ? max(1, min(a.nsplit, (steps + kWarps - 1) / kWarps)) : 1;
  const bool alone = n == 1;  // the tile has no other split
  if (CL && alone && z > 0) return leave();
  const int first = warp + kWarps * z;
  const int turn = CL ? 31 - __clz(kWarps * a.nsplit) : 2;  // (a cluster is a power of two)
  static_assert(kWarps == 4, "turn");
  const int mine = first < steps ? (steps - first - 1 >> turn) + 1 : 0;  // steps of the warp
  const int32_t* table = a.table ? a.table + static_cast<int64_t>(b) * a.table_width : nullptr;
  unsigned char* ring = smem + warp * S::RING;
  const uint32_t ring_addr = smem_addr(ring);
  const int64_t row_bytes = a.kv_stride * 2;
  // each split adds up `per` of the tile's 16-byte pieces: piece x belongs to split x / per
  constexpr int PIECES = D / 4;  // of a row
  const int rows = nt * a.hpt;  // (with those of heads that a last group of heads lacks)
  const int per = CL ? (rows * PIECES + n - 1) / n : 1;
  const int per_inverse = CL ? (1 << 20) / per + 1 : 1;  // (exact: x < 1024, per <= 512)
  auto issue = [&](int s) {
    if (s < mine) {
      if (table && (s & 31) == 0 && (s > 0 || !a.one_tile)) page = entry(table, s + lane);
      const int key = key_of(s);
      int64_t slot = rq.q0 + key;
      if (table) slot = attn_slot(a, __shfl_sync(0xffffffffu, page, s & 31), key);
      if (slot < 0) flags |= SSS_FLAG_INDEX;
      const uint32_t dst = ring_addr + (s % kStages) * 2 * S::TILE;
      const int64_t at = (slot < 0 ? 0 : slot) * row_bytes + kh * D * 2;
      const char* ksrc = static_cast<const char*>(a.k) + at;
      const char* vsrc = static_cast<const char*>(a.v) + at;
#pragma unroll
      for (int i = 0; i < kStep * CH / 32; ++i) {
        const int row = (lane + 32 * i) / CH, c = (lane + 32 * i) % CH;
        const bool in = slot >= 0 && key + row < lim1;
        const int64_t off = in ? row * row_bytes + c * 16 : 0;
        const uint32_t to = dst + row * (D * 2) + ((c ^ (row & 7)) * 16);
        copy16(to, ksrc + off, in);
        copy16(to + S::TILE, vsrc + off, in);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  for (int s = 0; s < kStages - 1; ++s) issue(s);

  // the rows' queries as mma operands, and how many keys each row sees
  uint32_t qf[MT][KD][4];
  int lim[MT][2];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int row = 16 * m + 8 * e + (lane >> 2);
      const int i = token_of(row), g = row - i * a.hpt;
      const bool in = i < nt && g < nh;
      lim[m][e] = in ? attn_limit(rq, i0 + i) : 0;
      const T* src = static_cast<const T*>(a.q) + (rq.q0 + i0 + (in ? i : 0)) * a.q_stride +
                     (kh * a.group + g0 + (in ? g : 0)) * D + 2 * (lane & 3);
#pragma unroll
      for (int kk = 0; kk < KD; ++kk) {
        qf[m][kk][e] = in ? __ldg(reinterpret_cast<const uint32_t*>(src + 16 * kk)) : 0u;
        qf[m][kk][2 + e] = in ? __ldg(reinterpret_cast<const uint32_t*>(src + 16 * kk + 8)) : 0u;
      }
    }

  // The sums are those of the rounded p, by one more product with ones: what
  // rounding takes off all of a row's p alike then cancels.
  constexpr uint32_t kOnes = std::is_same<T, __half>::value ? 0x3C003C00u : 0x3F803F80u;
  float o[MT][D / 8][4];
  float mx[MT][2], sum[MT][4];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
#pragma unroll
    for (int e = 0; e < 2; ++e) mx[m][e] = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[m][i] = 0.f;
#pragma unroll
    for (int n = 0; n < D / 8; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[m][n][i] = 0.f;
  }

  for (int s = 0; s < mine; ++s) {
    issue(s + kStages - 1);
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
    __syncwarp();
    const uint32_t kt = ring_addr + (s % kStages) * 2 * S::TILE, vt = kt + S::TILE;
    const int key0 = key_of(s);

    // scores: two tiles of 8 keys, each in two sums (shorter chains of products)
    float sc[MT][2][4], odd_sc[MT][2][4];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[m][n][i] = odd_sc[m][n][i] = 0.f;
#pragma unroll
    for (int kk = 0; kk < KD; ++kk) {
      const int row = (lane & 7) + ((lane >> 4) << 3), c = 2 * kk + ((lane >> 3) & 1);
      uint32_t kf[4];
      ldsm4(kf, kt + row * (D * 2) + ((c ^ (row & 7)) * 16));
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        mma16816<T>(kk & 1 ? odd_sc[m][0] : sc[m][0], qf[m][kk], kf[0], kf[1]);
        mma16816<T>(kk & 1 ? odd_sc[m][1] : sc[m][1], qf[m][kk], kf[2], kf[3]);
      }
    }
    // scale, mask, and raise the maxima where a score passes them by much
    bool raise = false;
    const bool cut = key0 + kStep > lim0;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x = (sc[m][n][i] + odd_sc[m][n][i]) * a.scale_log2;
          if (cut && key0 + 8 * n + 2 * (lane & 3) + (i & 1) >= lim[m][i >> 1]) x = -INFINITY;
          sc[m][n][i] = x;
          raise = raise || x > mx[m][i >> 1] + kRaise;
        }
    if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float t = fmaxf(fmaxf(sc[m][0][2 * e], sc[m][0][2 * e + 1]),
                          fmaxf(sc[m][1][2 * e], sc[m][1][2 * e + 1]));
          t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 1));
          t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 2));
          t = fmaxf(t, mx[m][e]);
          const float f = t == -INFINITY ? 1.f : ex2(mx[m][e] - t);
          mx[m][e] = t;
          sum[m][2 * e] *= f;
          sum[m][2 * e + 1] *= f;
#pragma unroll
          for (int n = 0; n < D / 8; ++n) {
            o[m][n][2 * e] *= f;
            o[m][n][2 * e + 1] *= f;
          }
        }
    }
    uint32_t pf[MT][4];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float ref = mx[m][i >> 1];
          const float p = ex2(sc[m][n][i] - (ref == -INFINITY ? 0.f : ref));
          sc[m][n][i] = p;
        }
      pf[m][0] = Pair<T>::pack(sc[m][0][0], sc[m][0][1]);
      pf[m][1] = Pair<T>::pack(sc[m][0][2], sc[m][0][3]);
      pf[m][2] = Pair<T>::pack(sc[m][1][0], sc[m][1][1]);
      pf[m][3] = Pair<T>::pack(sc[m][1][2], sc[m][1][3]);
      mma16816<T>(sum[m], pf[m], kOnes, kOnes);
    }
    // A value that is infinite or NaN reaches the rows that see its key and no
    // other: 0 x NaN would reach all.  Where a step's keys are not seen by every
    // row, such values are added by hand and leave the tile.
    if (cut && lim0 < lim1) {
      bool odd = false;
#pragma unroll
      for (int i = 0; i < kStep * CH / 32; ++i) {
        uint32_t w[4];
        const uint32_t at = vt + (lane + 32 * i) * 16;
        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                     : "r"(at)
                     : "memory");
#pragma unroll
        for (int j = 0; j < 4; ++j) odd = odd || pair_nonfinite<T>(w[j]);
      }
      if (__any_sync(0xffffffffu, odd)) {
        for (int key = 0; key < kStep; ++key) {
          const int from = (lane & ~3) | ((key & 7) >> 1);
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            float pk[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float lo = (key & 1) ? sc[m][0][2 * e + 1] : sc[m][0][2 * e];
              const float hi = (key & 1) ? sc[m][1][2 * e + 1] : sc[m][1][2 * e];
              pk[e] = __shfl_sync(0xffffffffu, key < 8 ? lo : hi, from);
            }
#pragma unroll
            for (int n = 0; n < D / 8; ++n) {
              uint32_t w;
              const uint32_t at = vt + key * (D * 2) + ((n ^ (key & 7)) * 16) + 4 * (lane & 3);
              asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w) : "r"(at) : "memory");
#pragma unroll
              for (int x = 0; x < 2; ++x) {
                const uint16_t bits = static_cast<uint16_t>(x ? w >> 16 : w & 0xFFFFu);
                if ((bits & Pair<T>::kExp) != Pair<T>::kExp) continue;
#pragma unroll
                for (int e = 0; e < 2; ++e)
                  if (key0 + key < lim[m][e]) o[m][n][2 * e + x] += pk[e] * Pair<T>::value(bits);
              }
            }
          }
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kStep * CH / 32; ++i) {
          unsigned char* at = ring + (s % kStages) * 2 * S::TILE + S::TILE + (lane + 32 * i) * 16;
          uint16_t* v16 = reinterpret_cast<uint16_t*>(at);
          for (int j = 0; j < 8; ++j)
            if ((v16[j] & Pair<T>::kExp) == Pair<T>::kExp) v16[j] = 0;
        }
        __syncwarp();
      }
    }
#pragma unroll
    for (int n2 = 0; n2 < D / 16; ++n2) {
      const int row = lane & 15, c = 2 * n2 + (lane >> 4);
      uint32_t vf[4];
      ldsm4_t(vf, vt + row * (D * 2) + ((c ^ (row & 7)) * 16));
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        mma16816<T>(o[m][2 * n2], pf[m], vf[0], vf[1]);
        mma16816<T>(o[m][2 * n2 + 1], pf[m], vf[2], vf[3]);
      }
    }
    __syncwarp();  // the stage is read; the next issue may overwrite it
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  if (flags && a.status) atomicOr(a.status, flags);

  // join the warps
  constexpr int LD = S::LD;
  float* part = reinterpret_cast<float*>(smem);
  __syncthreads();
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if (16 * m + 8 * e >= rows) continue;
      const int row = 16 * m + 8 * e + (lane >> 2);
      if ((lane & 3) == 0) {
        wmax[warp][row] = mx[m][e];
        wsum[warp][row] = sum[m][2 * e];
      }
      float* dst = part + (warp * R + row) * LD + 2 * (lane & 3);
#pragma unroll
      for (int n = 0; n < D / 8; ++n)
        *reinterpret_cast<float2*>(dst + 8 * n) = make_float2(o[m][n][2 * e], o[m][n][2 * e + 1]);
    }
  __syncthreads();
  // pieces of 16 bytes; with CL those of a split follow one another in `gather`
  const uint32_t gather = smem_addr(smem + S::RINGS), lse0 = smem_addr(&split_lse[0][0]);
  if (CL && !alone) {
    if (threadIdx.x == 0) {  // from each split this one's pieces and their rows' sums
      const int end = min(z * per + per, rows * PIECES);
      const int bytes = (end - z * per) * 16 + ((end - 1) / PIECES - z * per / PIECES + 1) * 4;
      // (the test hook: 16 bytes that nobody stores)
      if (z < n) mbar_arrive_expect_tx(&arrived, (z * per < end ? n * bytes : 0) + (a.stall ? 16 : 0));
    }
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  for (int x = threadIdx.x; x < rows * PIECES; x += kThreads) {
    const int row = x / PIECES, d = 4 * (x % PIECES);
    const int i = token_of(row), g = row - i * a.hpt;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, wmax[w][row]);
    const float ref = top == -INFINITY ? 0.f : top;
    float total = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float f = ex2(wmax[w][row] - ref);  // (0 of a warp without keys)
      const float4 v = *reinterpret_cast<const float4*>(part + (w * R + row) * LD + d);
      total += f * wsum[w][row];
      acc.x += f * v.x;
      acc.y += f * v.y;
      acc.z += f * v.z;
      acc.w += f * v.w;
    }
    const float r = total == 0.f ? 0.f : 1.f / total;  // a row without keys: zeros
    acc = make_float4(acc.x * r, acc.y * r, acc.z * r, acc.w * r);
    const float lse = total == 0.f ? -INFINITY : top + log2f(total);
    const int64_t at = static_cast<int64_t>(rq.q0 + i0 + i) * a.heads + kh * a.group + g0 + g;
    if (alone) {
      const uint2 u = make_uint2(Pair<T>::pack(acc.x, acc.y), Pair<T>::pack(acc.z, acc.w));
      if (g < nh) *reinterpret_cast<uint2*>(static_cast<T*>(a.out) + at * D + d) = u;
    } else if constexpr (CL) {
      if (z < n) {
        const int to = x * per_inverse >> 20;
        const uint32_t bar = of_peer(smem_addr(&arrived), to);
        peer_store(of_peer(gather + (z * per + x - to * per) * 16, to), acc, bar);
        // (the row's pieces belong to a few of the splits: each gets its sum)
        if (d == 0 || x == to * per) peer_store(of_peer(lse0 + (z * R + row) * 4, to), lse, bar);
      }
    }
  }
  if constexpr (CL) {
    if (alone) return leave();
    __syncwarp();
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    bool ok = z < n;  // this CTA has pieces to join
    if (ok) {
      int abort = 0;
      ok = __all_sync(0xffffffffu, mbar_wait(&arrived, 0, &abort));
      if (!ok && a.status && lane == 0) atomicOr(a.status, SSS_FLAG_TIMEOUT);
    }
    // a lane per split and piece (a cluster is a power of two)
    const int cl = a.nsplit, w = threadIdx.x & (cl - 1);
    for (int y0 = 0; ok && y0 < per; y0 += kThreads / cl) {
      const int y = y0 + threadIdx.x / cl, x = z * per + y, row = x / PIECES, d = 4 * (x % PIECES);
      const int i = token_of(row), g = row - i * a.hpt;
      const bool in = y < per && row < rows;
      const float l = in && w < n ? split_lse[w][row] : -INFINITY;
      float top = l;
      for (int m = cl / 2; m > 0; m >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
      float total = l == -INFINITY ? 0.f : ex2(l - top);
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (in && w < n) {
        v = *reinterpret_cast<const float4*>(smem + S::RINGS + (w * per + y) * 16);
        v = make_float4(v.x * total, v.y * total, v.z * total, v.w * total);
      }
      for (int m = cl / 2; m > 0; m >>= 1) {
        total += __shfl_xor_sync(0xffffffffu, total, m);
        v.x += __shfl_xor_sync(0xffffffffu, v.x, m);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, m);
        v.z += __shfl_xor_sync(0xffffffffu, v.z, m);
        v.w += __shfl_xor_sync(0xffffffffu, v.w, m);
      }
      if (!in || w != 0 || g >= nh) continue;
      const float r = total == 0.f ? 0.f : 1.f / total;
      const int64_t at = static_cast<int64_t>(rq.q0 + i0 + i) * a.heads + kh * a.group + g0 + g;
      const uint2 u = make_uint2(Pair<T>::pack(v.x * r, v.y * r), Pair<T>::pack(v.z * r, v.w * r));
      *reinterpret_cast<uint2*>(static_cast<T*>(a.out) + at * D + d) = u;
    }
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (z < n && !ok) {
      int drain = 0;
      (void)mbar_wait(&arrived, 0, &drain);
    }
  }
}

// The rows whose tile has more than one split: the splits' outputs, weighted by
// 2^lse, in split order.  WARPS to a row, of which each takes every WARPS-th split.
constexpr int kJoinWarps = 4;  // of a CTA
template <typename T, int D, int WARPS>
__global__ void __launch_bounds__(32 * kJoinWarps) attn_join_kernel(const __grid_constant__ AttnArgs a) {
  __shared__ float4 sums[kJoinWarps][D / 4];
  __shared__ float totals[kJoinWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, first = warp % WARPS;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (kJoinWarps / WARPS) + warp / WARPS;
  const int64_t rows = static_cast<int64_t>(a.tokens) * a.heads;
  if (row >= rows) return;
  const int t = static_cast<int>(row / a.heads);
  // the token's request: the last whose first token is not behind it
  int lo = 0, hi = a.batch;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.cu_q[mid] <= t) lo = mid;
    else hi = mid;
  }
  uint32_t flags = 0;
  const AttnRequest rq = attn_request(a, lo, flags);
  const int i = t - rq.q0;
  if (i < 0 || i >= rq.n) return;
  const int lim = attn_limit(rq, min(i / a.tpt * a.tpt + a.tpt, rq.n) - 1);
  if (lim <= a.chunk) return;
  const int n = (lim + a.chunk - 1) / a.chunk;
  float top = -INFINITY;
  for (int z = lane; z < n; z += 32) top = fmaxf(top, a.part_lse[z * rows + row]);
#pragma unroll
  for (int m = 16; m > 0; m >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
  const float ref = top == -INFINITY ? 0.f : top;
  constexpr int LANES = D / 4;  // that hold the row
  float total = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int z = first; z < n; z += WARPS) {
    const float lse = a.part_lse[z * rows + row];
    const float4 v = lane < LANES ? reinterpret_cast<const float4*>(a.part + (z * rows + row) * D)[lane]
                                  : make_float4(0.f, 0.f, 0.f, 0.f);
    const float f = ex2(lse - ref);
    total += f;
    acc.x += f * v.x;
    acc.y += f * v.y;
    acc.z += f * v.z;
    acc.w += f * v.w;
  }
  if constexpr (WARPS > 1) {
    static_assert(WARPS == kJoinWarps, "a CTA's row");
    if (lane < LANES) sums[warp][lane] = acc;
    if (lane == 0) totals[warp] = total;
    __syncthreads();
    if (warp != 0) return;
#pragma unroll
    for (int w = 1; w < WARPS; ++w) {
      const float4 v = sums[w][lane % LANES];
      total += totals[w];
      acc = make_float4(acc.x + v.x, acc.y + v.y, acc.z + v.z, acc.w + v.w);
    }
  }
  if (lane >= LANES) return;
  const float r = total == 0.f ? 0.f : 1.f / total;
  reinterpret_cast<uint2*>(static_cast<T*>(a.out) + row * D)[lane] =
      make_uint2(Pair<T>::pack(acc.x * r, acc.y * r), Pair<T>::pack(acc.z * r, acc.w * r));
}

template <typename K>
cudaError_t launch(K kern, const AttnArgs& a, dim3 grid, int threads, int smem,
                   cudaStream_t stream, int cluster = 1) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, a);
}

template <typename T, int D, int MT, bool CL>
cudaError_t run_rows(AttnArgs a, cudaStream_t stream) {
  auto kern = attn_rows_kernel<T, D, MT, CL>;
  constexpr int smem = RowsSmem<D, 16 * MT, CL>::TOTAL;
  cudaError_t e = ensure_smem(kern, smem);
  if (e != cudaSuccess) return e;
  if (CL && a.nsplit > 8) {
    e = ensure_large_cluster(kern);
    if (e != cudaSuccess) return e;
  }
  constexpr int kMost = 65535;  // of a grid's z (more tiles than requests: only over a cache without slots)
  for (; e == cudaSuccess && a.tile0 < a.tiles; a.tile0 += kMost)
    e = launch(kern, a, dim3(a.nsplit, a.kv_heads * a.hchunks, std::min(kMost, a.tiles - a.tile0)), kThreads,
               smem, stream, a.nsplit);
  return e;
}
template <typename T, int D, int MT>
cudaError_t rows_mode(const AttnArgs& a, cudaStream_t stream) {
  return a.nsplit > 1 ? run_rows<T, D, MT, true>(a, stream) : run_rows<T, D, MT, false>(a, stream);
}
template <typename T>
cudaError_t rows_dim(const AttnArgs& a, int dim, cudaStream_t stream) {
  if (dim == 64)
    return a.rows == 16 ? rows_mode<T, 64, 1>(a, stream) : rows_mode<T, 64, 2>(a, stream);
  return a.rows == 16 ? rows_mode<T, 128, 1>(a, stream) : rows_mode<T, 128, 2>(a, stream);
}
template <typename T, int D>
cudaError_t run_join(const AttnArgs& a, cudaStream_t stream) {
  const bool wide = a.nsplit > 8;  // a CTA to a row
  const int64_t rows = static_cast<int64_t>(a.tokens) * a.heads;
  const int64_t blocks = wide ? rows : (rows + kJoinWarps - 1) / kJoinWarps;
  if (blocks > INT32_MAX) return cudaErrorNotSupported;
  const dim3 grid(static_cast<unsigned>(blocks));
  return wide ? launch(attn_join_kernel<T, D, kJoinWarps>, a, grid, 32 * kJoinWarps, 0, stream)
              : launch(attn_join_kernel<T, D, 1>, a, grid, 32 * kJoinWarps, 0, stream);
}
template <typename T>
cudaError_t join_dim(const AttnArgs& a, int dim, cudaStream_t stream) {
  return dim == 64 ? run_join<T, 64>(a, stream) : run_join<T, 128>(a, stream);
}

}  // namespace

cudaError_t launch_attn_rows(const AttnArgs& a, int dtype, int dim, cudaStream_t stream) {
  return dtype == SSS_OUT_F16 ? rows_dim<__half>(a, dim, stream)
                              : rows_dim<__nv_bfloat16>(a, dim, stream);
}
cudaError_t launch_attn_join(const AttnArgs& a, int dtype, int dim, cudaStream_t stream) {
  return dtype == SSS_OUT_F16 ? join_dim<__half>(a, dim, stream)
                              : join_dim<__nv_bfloat16>(a, dim, stream);
}

}  // namespace sss
