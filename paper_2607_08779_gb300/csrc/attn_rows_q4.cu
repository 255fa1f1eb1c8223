// attn_rows_q4.cu -- attention of few rows (the single tokens, or a few drafted ones, of a
// decode step) over the cache in 4 bits.
//
//   o_i = sum_j p_ij v_j / sum_j p_ij,   p_ij = 2^(c q_i.k_j - m_i),  c = scale log2(e)
//
// with k_jd = s_jg k'_jd, v_jd = t_jg v'_jd: codes k', v' in -8 .. 7, a scale for each group g of
// 32 dimensions.  The products run on mma.sync over the codes alone, keys (and then
// dimensions) as its 16 rows, tokens x heads as its 8 columns:
//   scores   x_ij = sum_g s_jg (sum_{d in g} q_id k'_jd),  scaled in fp32 group by group;
//   outputs  o_id = sum_j (p_ij t_jg) v'_jd, with p t rounded to fp16 for the product (for
//            bf16 outputs p is rounded first: the product of two halves is one instruction for
//            two rows, and an error of 2^-10 at most is a quarter of the output's own).
// p is 2^10 where a row's score is its largest, so that p t is a normal number of fp16 down to p t =
// 2^-24 of that: the cache's least scale.  (With p of 1 there values of 1e-4 lost up to 2 %, and many
// keys of little weight all they had.)  Where a row sees a scale of 32 or more its p is lowered, and what
// it has added up with it, as where its maximum is raised.  To look at a step's scales costs 1 to 2 %
// (64 requests of 12000 to 16384 keys: 185 us without, 187).
// A nibble u = code + 8 becomes a 16-bit operand by one AND: in bits 0-3 of a half it is the
// (subnormal) number u 2^-24, in bits 4-7 u 2^-20, exactly.  For the keys the 8 that are too
// much are taken off by what the sums start from, -8 times q's sums; for the values by a
// subtraction, exact as well (by a product with constants instead: 237 us against 229, and by
// numbers 1024 + u: 250).  q is made fp16 with a power of two of its row's own (|q'| <
// 2^15: what is 2^-28 of the row's largest or less is rounded), whatever its type; the odd nibbles' q' is
// a 16th.  So the type of q and out hardly matters inside.
//
// Bound by the issue of its instructions, not far from HBM: 16 keys and values of a head of
// 128 are 2304 bytes, which an SM's share of the bandwidth brings in 96 cycles.  Four
// schedulers have 384 issue slots in that time; the step takes about 280 with 8 columns, 16 of
// them products that keep a scheduler for 7 cycles each.  64 requests of 12000 to 16384 keys (32
// heads of 128 over 8): 187 us, 5.6 TB/s, 83 % of the copy rate (the copies without the
// arithmetic run at 105 %); 16 of 130 to 16384 (64 heads) 30.9, the longest ones' chunks and the
// second kernel being last; one of 2047 keys 5.1.  With 16 columns 32 requests of 16384 keys
// and 4 heads take 99 us, 45 % of that rate; heads of 64 (64 requests of 8000 to 16384 keys) 102, a CTA
// more an SM having taken 7 % off.  What did not help: the next step's scores beside
// this one's outputs (236 us against 233 at the time), four CTAs an SM with shorter rings (249),
// 16 keys a step (244 against 216).
// A block of the cache is one bulk copy into a ring that each warp has for itself, with a
// barrier for each stage and no other wait in the loop.  The codes lie so that each lane's are
// vector loads without bank conflicts (the keys' order in a tile, key_slot below, is chosen for
// that), and that neighbours in an operand are the halves of a word (keys) or one byte
// permutation apart (values).  The rest is as in attn_rows.cu: 32 blocks' table entries
// read ahead, splits of a tile's keys joined in a cluster, or chunks of them by
// attn_join_kernel, in a fixed order.
#include <algorithm>

#include "attn.cuh"
#include "kv_q4.cuh"
#include "tc.cuh"

namespace sss {
namespace {

// How a tile's keys are split over CTAs: not; over those of a cluster, in turn, which join them
// there; or in chunks, whose results attn_join_kernel joins.
enum Split { kWhole, kCluster, kChunks };

// A warp's steps: long chunks go 64 keys at a time (64 requests of 12000 to 16384 keys: 202 us
// by 32, 190 by 64), with fewer votes, branches and waits a key; else 32 spread a request's keys
// over more warps (one of 2047: 5.2 us, 6.4 by 64).
template <Split SPLIT>
struct Ring {
  static constexpr int kBlocks = SPLIT == kChunks ? 4 : 2;  // of the cache in a step
  static constexpr int kStages = SPLIT == kChunks ? 2 : 3;  // steps
};

template <int D, int R, Split SPLIT, int WARPS>
struct RowsQ4Smem {
  static constexpr int kBlocks = Ring<SPLIT>::kBlocks, kStages = Ring<SPLIT>::kStages;
  static constexpr bool CL = SPLIT == kCluster;
  static constexpr int STAGE = kBlocks * Q4Block<D>::kBytes;
  static constexpr int RING = kStages * STAGE;  // of a warp
  static constexpr int LD = D + 4;  // of the warps' outputs, which follow
  static constexpr int RINGS = WARPS * std::max(RING, R * LD * 4);
  // the splits' pieces of the values that this one joins (their number rounded up)
  static constexpr int TOTAL = RINGS + (CL ? (R * D / 4 + 16) * 16 : 0);
};

// The power of two of a row's largest p, at most kTop: lowered (to -1 at least) for a scale of 32 and more,
// whose bits without the sign these take, so that p times a scale is below 2^15; and the
// largest scale that leaves it as it is.
constexpr int kTop = 10;
__device__ __forceinline__ int top_for(int top, uint32_t scale) {
  return min(top, 29 - min(static_cast<int>(scale >> 10), 30));
}
__device__ __forceinline__ uint32_t scale_for(int top) {
  return (static_cast<uint32_t>(30 - top) << 10) - 1u;
}
// the larger of each half's sizes, the first not negative (a NaN counts for nothing)
__device__ __forceinline__ uint32_t larger2(uint32_t a, uint32_t b) {
  const __half2 v = __hmax2(*reinterpret_cast<const __half2*>(&a), __habs2(*reinterpret_cast<const __half2*>(&b)));
  return *reinterpret_cast<const uint32_t*>(&v);
}

// The slot of a step that is row (or operand column) i of a tile: four slots in order for the
// even ones, four in reverse for the odd.
__device__ __forceinline__ int key_slot(int i) {
  return (i & 8) + ((i & 1) ? 4 + ((i >> 1 & 3) ^ 3) : (i >> 1 & 3));
}

// d = A B + c, or d += A B
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                        uint32_t a3, uint32_t b0, uint32_t b1, const float (&c)[4]) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%10,%11,%12,%13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                        uint32_t a3, uint32_t b0, uint32_t b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// an 8 x 8 matrix of 16-bit values, two of a row to a lane, transposed
__device__ __forceinline__ uint32_t transposed(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
// The lower (e = 0, 1) or upper nibble of the lower byte of both halves as subnormal numbers:
// u 2^-24, or u 2^-20 where e is odd.  (The upper bytes come down by a byte permutation, which
// costs half of what a shift does.)
__device__ __forceinline__ uint32_t nibbles(uint32_t w, int e) {
  return w & (e & 1 ? 0x00F000F0u : 0x000F000Fu);
}
// the same less 8 of that unit
__device__ __forceinline__ uint32_t codes(uint32_t w, int e) {
  uint32_t r = nibbles(w, e);
  asm("sub.rn.f16x2 %0, %0, %1;" : "+r"(r) : "r"(e & 1 ? 0x00800080u : 0x00080008u));
  return r;
}
template <typename V>
__device__ __forceinline__ void lds(V& v, const unsigned char* at) {
  v = *reinterpret_cast<const V*>(at);
}
// both halves of p times the lower or upper half of w
__device__ __forceinline__ uint32_t times_half(uint32_t p, uint32_t w, bool upper) {
  const __half2 t = *reinterpret_cast<const __half2*>(&w);
  const __half2 v = __hmul2(*reinterpret_cast<const __half2*>(&p), upper ? __high2half2(t) : __low2half2(t));
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float2 halves(uint32_t w) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
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

// NT tiles of 8 rows (tokens x heads).
template <typename T, int D, int NT, Split SPLIT, int WARPS>
__global__ void __launch_bounds__(32 * WARPS, WARPS == 8 ? 1 : (NT == 1 ? 3 : 2) + (D == 64 ? 1 : 0))
    attn_rows_q4_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ Q4Cache c4) {
  constexpr int R = 8 * NT;
  constexpr bool CL = SPLIT == kCluster;
  constexpr int kWarps = WARPS, kThreads = 32 * WARPS;
  using S = RowsQ4Smem<D, R, SPLIT, WARPS>;
  constexpr int kBlocks = S::kBlocks, kStages = S::kStages;
  constexpr int kStep = kBlocks * kQ4Slots;  // keys of a step
  constexpr int kAhead = 32 / kBlocks;       // steps whose blocks the lanes hold
  using B = Q4Block<D>;
  constexpr int W = D / 8;      // words of a slot
  constexpr int KW = W / 4;     // that a lane has of a key's
  constexpr int VW = W / 8;     // and of a value's
  constexpr int G = D / 32;     // groups
  constexpr int PER = 4 / G;    // nibble places to a group
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ float wmax[kWarps][R], wsum[kWarps][R];
  __shared__ int lims[kWarps][R];
  __shared__ float split_lse[CL ? 16 : 1][R];  // of every split
  __shared__ uint64_t arrived;                 // what the splits store here
  __shared__ uint64_t full[kWarps][kStages];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int r = lane >> 2, c = lane & 3;  // of the operands' layouts
  if (lane < kStages) mbar_init(&full[warp][lane], kBlocks);
  if (CL && threadIdx.x == 0) mbar_init(&arrived, 1);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  __syncwarp();
  // another CTA's shared memory exists only once that CTA has started: waited for
  // before the first store into a peer
  if constexpr (CL) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  const int z = blockIdx.x, hx = blockIdx.y;
  const int kh = a.hchunks == 1 ? hx : hx / a.hchunks;
  const int g0 = (hx - kh * a.hchunks) * a.hpt;
  const int nh = min(a.hpt, a.group - g0);  // heads of the tile
  const auto token_of = [&](int row) { return row * a.hpt_inverse >> 16; };
  const auto leave = [&]() {
    if constexpr (CL) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  };
  // the keys go to the splits of a cluster and their warps a step at a time in turn
  const int chunk0 = SPLIT == kChunks ? z * a.chunk : 0;
  const auto key_of = [&](int s) { return chunk0 + kStep * (warp + kWarps * (CL ? z + a.nsplit * s : s)); };
  const int64_t width = static_cast<int64_t>(a.table_width) << a.page_shift;
  // the lane's block among those of steps s .. s + kAhead - 1
  const auto lane_key = [&](int s) {
    const int64_t t = s + lane / kBlocks;
    return chunk0 + kStep * (warp + kWarps * (CL ? z + a.nsplit * t : t)) + kQ4Slots * (lane % kBlocks);
  };
  const auto entry = [&](const int32_t* table, int s) {
    const int64_t key = lane_key(s);
    return key < width && key < a.max_kv ? __ldg(table + (key >> a.page_shift)) : 0;
  };
  int page = 0;
  const int tile = a.tile0 + blockIdx.z;
  if (a.one_tile && tile < a.batch)
    page = entry(a.table + static_cast<int64_t>(tile) * a.table_width, 0);
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
  if (SPLIT == kChunks && z > 0 && chunk0 >= lim1) return;
  const int keys = SPLIT == kChunks ? min(a.chunk, lim1 - chunk0) : lim1;  // of the CTA's splits
  const int steps = (keys + kStep - 1) / kStep;
  // splits with keys
  const int n = CL ? max(1, min(a.nsplit, (steps + kWarps - 1) / kWarps)) : 1;
  const bool alone = SPLIT == kChunks ? lim1 <= a.chunk : n == 1;  // the tile has no other split
  if (CL && alone && z > 0) return leave();
  const int first = CL ? warp + kWarps * z : warp;
  const int turn = 31 - __clz(CL ? kWarps * a.nsplit : kWarps);  // (powers of two)
  const int mine = first < steps ? (steps - first - 1 >> turn) + 1 : 0;  // steps of the warp
  const int32_t* table = a.table + static_cast<int64_t>(b) * a.table_width;
  unsigned char* ring = smem + warp * S::RING;
  // each split adds up `per` of the tile's 16-byte pieces: piece x belongs to split x / per
  constexpr int PIECES = D / 4;  // of a row
  const int rows = nt * a.hpt;   // (with those of heads that a last group of heads lacks)
  const int per = CL ? (rows * PIECES + n - 1) / n : 1;
  const int per_inverse = CL ? (1 << 20) / per + 1 : 1;  // (exact: x < 1024, per <= 512)

  // kAhead steps' blocks, one to a lane, which issues their copies; and which of them are
  // not there: without keys that a row sees, or without a page in the table.
  const char* block = nullptr;
  uint32_t pageless = 0;
  const auto look_up = [&](int s) {
    const int64_t key = lane_key(s);
    const int64_t slot = key < lim1 ? attn_slot(a, page, static_cast<int>(key)) : -1;
    if (slot < 0 && key < lim1) flags |= SSS_FLAG_INDEX;
    block = q4_block<D>(c4, slot < 0 ? 0 : slot, kh);
    pageless = __ballot_sync(0xffffffffu, slot < 0);
  };
  if (!a.one_tile) page = entry(table, 0);
  look_up(0);
  // A step's blocks into its stage; of one that is not there a bit of `none` (kBlocks to a
  // stage), and only an arrival.
  uint32_t none = 0;
  const auto issue = [&](int s, int stage) {
    if (s >= mine) return;
    const int at = s % kAhead;
    if (at == 0 && s > 0) {
      page = entry(table, s);
      look_up(s);
    }
    constexpr uint32_t kAll = (1u << kBlocks) - 1;
    const uint32_t bad = pageless >> (kBlocks * at) & kAll;
    none = (none & ~(kAll << (kBlocks * stage))) | bad << (kBlocks * stage);
    if (lane / kBlocks == at) {
      uint64_t* bar = &full[warp][stage];
      if (pageless >> lane & 1u) {
        mbar_arrive(bar);
      } else {
        mbar_arrive_expect_tx(bar, B::kBytes);
        asm volatile(
            "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, "
            "[%3];" ::"r"(smem_u32(ring) + stage * S::STAGE + lane % kBlocks * B::kBytes),
            "l"(block), "r"(B::kBytes), "r"(smem_u32(bar))
            : "memory");
      }
    }
  };
#pragma unroll 1
  for (int s = 0; s < kStages; ++s) issue(s, s);

  // q' as operands, what the scores' sums start from, and the rows' scales and limits: of
  // the accumulators' rows 2 c and 2 c + 1 of each tile
  uint32_t qf[NT][4][KW];
  float start[NT][G][4], rscale[NT][2];
  int lim[NT][2];
#pragma unroll
  for (int m = 0; m < NT; ++m) {
    const int row = 8 * m + r;
    const int i = token_of(row), g = row - i * a.hpt;
    const bool in = i < nt && g < nh;
    const T* src = static_cast<const T*>(a.q) + (rq.q0 + i0 + (in ? i : 0)) * a.q_stride +
                   (kh * a.group + g0 + (in ? g : 0)) * D;
    // the lane's dimensions: 2 W e + W h + w for its words w = KW c .. KW c + KW - 1
    float x[4][2][KW];
    float top = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t v[KW / 2];
        const T* at = src + 2 * W * e + W * h + KW * c;
        if constexpr (KW == 4) {
          const uint2 u = in ? __ldg(reinterpret_cast<const uint2*>(at)) : make_uint2(0u, 0u);
          v[0] = u.x;
          v[1] = u.y;
        } else {
          v[0] = in ? __ldg(reinterpret_cast<const uint32_t*>(at)) : 0u;
        }
#pragma unroll
        for (int w = 0; w < KW; ++w) {
          x[e][h][w] = Pair<T>::value(static_cast<uint16_t>(w & 1 ? v[w / 2] >> 16 : v[w / 2]));
          top = fmaxf(top, fabsf(x[e][h][w]));
        }
      }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    // 2^(14 - E) for a largest size of 2^E and more
    const int E = max(static_cast<int>(__float_as_uint(top) >> 23 & 255u) - 127, -112);
    const float up = __int_as_float((14 - min(E, 127) + 127) << 23);
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        const float f = e & 1 ? up * 0.0625f : up;
        const __half2 v = __floats2half2_rn(x[e][0][w] * f, x[e][1][w] * f);
        qf[m][e][w] = *reinterpret_cast<const uint32_t*>(&v);
      }
    // 2^(E - 14) of the scale, and the 2^24 of the nibbles'
    const float rs = fminf(fmaxf(1e-37f, a.scale_log2 * __int_as_float((min(E, 127) - 14 + 127) << 23) * 0x1p24f), 3e38f);  // (for what is multiplied by infinities)
    const int limit = in ? attn_limit(rq, i0 + i) : 0;
    if (c == 0) lims[warp][row] = limit;
    // -8 times q's sums: products with codes that are all -8
#pragma unroll
    for (int g = 0; g < G; ++g) {
#pragma unroll
      for (int k = 0; k < 4; ++k) start[m][g][k] = 0.f;
#pragma unroll
      for (int e = g * PER; e < g * PER + PER; ++e)
#pragma unroll
        for (int w = 0; w < KW; w += 2) {
          const uint32_t less = e & 1 ? 0x80808080u : 0x80088008u;
          mma_f16(start[m][g], less, less, less, less, qf[m][e][w], qf[m][e][w + 1]);
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int from = 4 * (2 * c + k);
      rscale[m][k] = __shfl_sync(0xffffffffu, rs, from);
      lim[m][k] = __shfl_sync(0xffffffffu, limit, from);
    }
  }

  float o[NT][4][VW][4];  // rows 2 c, 2 c + 1 of dimensions 2 W e + w and 2 W e + W + w
  // ref: what scaled scores are added to, -mx scaled and the row's power of two, or 0
  float mx[NT][2], ref[NT][2], sum[NT][2];
  // The rows' powers of two are in wmax until the warps are joined, and are looked up there once one
  // was lowered; fits2: the largest scale, twice, that leaves all of them as they are.
  constexpr uint32_t kFits2 = ((30u - kTop) << 10) * 0x10001u - 0x10001u;
  if (lane < R) wmax[warp][lane] = kTop;
  __syncwarp();
  uint32_t fits2 = kFits2;
#pragma unroll
  for (int m = 0; m < NT; ++m) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      mx[m][k] = -INFINITY;
      ref[m][k] = sum[m][k] = 0.f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int w = 0; w < VW; ++w)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[m][e][w][i] = 0.f;
  }
  // the lane's keys of the scores are slots j0 and j0 + 8 of a block, of the values v0, v1
  // and those + 8
  const int j0 = key_slot(r), v0 = key_slot(2 * c), v1 = key_slot(2 * c + 1);
  const uint32_t k_at = j0 * B::kRow + 4 * KW * c, s_at = j0 * B::kScales;
  const uint32_t v0_at = B::kV + v0 * B::kRow + 4 * q4_value_word<D>(VW * r, v0);
  const uint32_t v1_at = B::kV + v1 * B::kRow + 4 * q4_value_word<D>(VW * r, v1);
  int stage = 0;
  uint32_t parity = 0;
  bool waited = true;
#pragma unroll 1
  for (int s = 0; s < mine; ++s) {
    if (!__all_sync(0xffffffffu, mbar_try_wait(&full[warp][stage], parity))) {
      int abort = 0;
      waited = __all_sync(0xffffffffu, mbar_wait(&full[warp][stage], parity, &abort));
      if (!waited) break;
    }
    const unsigned char* at = ring + stage * S::STAGE;
    const int key0 = key_of(s);
    const uint32_t blank = none >> (kBlocks * stage) & ((1u << kBlocks) - 1);
    const bool rare = key0 + kStep > lim0 || blank != 0;  // (rows that are no token's see nothing then)
    // the values' scales: is one too large for p?  (two to a lane; for heads of 64 each to two lanes)
    uint32_t most2 = fits2;
#pragma unroll
    for (int u = 0; u < kBlocks; ++u) {
      uint32_t w;
      lds(w, at + u * B::kBytes + B::kVS + 4 * (lane % (kQ4Slots * G / 2)));
      most2 = larger2(most2, w);
    }

    // scores
    float x[kBlocks][NT][4];
#pragma unroll
    for (int u = 0; u < kBlocks; ++u) {
      uint32_t kw[2][KW];
      float ks[2][G];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const unsigned char* k = at + u * B::kBytes + B::kK + k_at + e * 8 * B::kRow;
        const unsigned char* f = at + u * B::kBytes + B::kKS + s_at + e * 8 * B::kScales;
        if constexpr (KW == 4) {
          uint4 w;
          lds(w, k);
          kw[e][0] = w.x; kw[e][1] = w.y; kw[e][2] = w.z; kw[e][3] = w.w;
          uint2 h;
          lds(h, f);
          const float2 lo = halves(h.x), hi = halves(h.y);
          ks[e][0] = lo.x; ks[e][1] = lo.y; ks[e][2] = hi.x; ks[e][3] = hi.y;
        } else {
          uint2 w;
          lds(w, k);
          kw[e][0] = w.x; kw[e][1] = w.y;
          uint32_t h;
          lds(h, f);
          const float2 lo = halves(h);
          ks[e][0] = lo.x; ks[e][1] = lo.y;
        }
      }
      // bytes 0 and 2 of the words, then 1 and 3
      uint32_t ku[2][KW];
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int w = 0; w < KW; ++w) ku[e][w] = __byte_perm(kw[e][w], 0u, 0x3311);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        float acc[NT][4];
#pragma unroll
        for (int e = g * PER; e < g * PER + PER; ++e)
#pragma unroll
          for (int w = 0; w < KW; w += 2) {
            const uint32_t(&from)[2][KW] = e < 2 ? kw : ku;
            const uint32_t a0 = nibbles(from[0][w], e), a1 = nibbles(from[1][w], e);
            const uint32_t a2 = nibbles(from[0][w + 1], e), a3 = nibbles(from[1][w + 1], e);
#pragma unroll
            for (int m = 0; m < NT; ++m) {
              if (e == g * PER && w == 0)
                mma_f16(acc[m], a0, a1, a2, a3, qf[m][e][w], qf[m][e][w + 1], start[m][g]);
              else
                mma_f16(acc[m], a0, a1, a2, a3, qf[m][e][w], qf[m][e][w + 1]);
            }
          }
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            x[u][m][i] = g == 0 ? ks[i >> 1][g] * acc[m][i] : x[u][m][i] + ks[i >> 1][g] * acc[m][i];
      }
    }
    // mask, and raise the maxima (not yet scaled, as the scores) where a score passes them
    if (rare) {  // no page: zeros (what the stage holds is of any kind); not seen: -inf
#pragma unroll
      for (int u = 0; u < kBlocks; ++u)
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (blank >> u & 1u) x[u][m][i] = 0.f;
            if (key0 + kQ4Slots * u + j0 + 8 * (i >> 1) >= lim[m][i & 1]) x[u][m][i] = -INFINITY;
          }
    }
    float top[NT][2];
    bool raise = most2 != fits2;
#pragma unroll
    for (int m = 0; m < NT; ++m)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        top[m][k] = fmaxf(x[0][m][k], x[0][m][2 + k]);
#pragma unroll
        for (int u = 1; u < kBlocks; ++u) top[m][k] = fmaxf(top[m][k], fmaxf(x[u][m][k], x[u][m][2 + k]));
        raise = raise || top[m][k] > mx[m][k];
      }
    if (__any_sync(0xffffffffu, raise)) {
      // the step's largest scales of keys before `end`, the lane's two
      const auto seen2 = [&](int end) {
        uint32_t w = 0;
#pragma unroll 1
        for (int u = 0; u < kBlocks; ++u) {
          const int word = lane % (kQ4Slots * G / 2), slot = word / (G / 2);
          uint32_t v;
          lds(v, at + u * B::kBytes + B::kVS + 4 * word);
          if (!(blank >> u & 1u) && key0 + kQ4Slots * u + slot < end) w = larger2(w, v);
        }
        return w;
      };
      if (__any_sync(0xffffffffu, most2 != fits2) &&
          __any_sync(0xffffffffu, larger2(fits2, seen2(lim1)) != fits2)) {  // lower p for the rows that see it
        uint32_t high = 0;
#pragma unroll 1
        for (int row = 0; row < R; ++row) {
          const uint32_t w = seen2(lims[warp][row]);
          const uint32_t big = __reduce_max_sync(0xffffffffu, max(w & 0xFFFFu, w >> 16));
          const int now = top_for(static_cast<int>(wmax[warp][row]), big);
          high = max(high, static_cast<uint32_t>(now + 1));
          __syncwarp();
          if (lane == 0) wmax[warp][row] = static_cast<float>(now);
        }
        __syncwarp();
        fits2 = scale_for(static_cast<int>(high) - 1) * 0x10001u - 1u;  // (not kFits2 again)
      }
#pragma unroll
      for (int m = 0; m < NT; ++m)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float t = fmaxf(top[m][k], mx[m][k]);
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, d));
          // (rounded down: no p passes its power of two, however large the scores)
          float power = kTop;
          if (fits2 != kFits2) power = wmax[warp][8 * m + 2 * c + k];
          const float to = t == -INFINITY ? 0.f : __fmaf_rd(-t, rscale[m][k], power);
          const float f = mx[m][k] == -INFINITY ? 1.f : ex2(to - ref[m][k]);
          mx[m][k] = t;
          ref[m][k] = to;
          sum[m][k] *= f;
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int w = 0; w < VW; ++w) {
              o[m][e][w][k] *= f;
              o[m][e][w][2 + k] *= f;
            }
        }
    }
#pragma unroll
    for (int u = 0; u < kBlocks; ++u)
#pragma unroll
      for (int m = 0; m < NT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[u][m][i] = ex2(__fmaf_rn(x[u][m][i], rscale[m][i & 1], ref[m][i & 1]));
          sum[m][i & 1] += x[u][m][i];
        }
    // outputs
#pragma unroll
    for (int u = 0; u < kBlocks; ++u) {
      uint32_t p[G][NT][2];  // p t of the lane's two keys
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const unsigned char* f = at + u * B::kBytes + B::kVS + s_at + e * 8 * B::kScales;
        uint32_t h[G / 2];
        if constexpr (G == 4) {
          uint2 w;
          lds(w, f);
          h[0] = w.x; h[1] = w.y;
        } else {
          lds(h[0], f);
        }
        if constexpr (std::is_same<T, __half>::value) {
#pragma unroll
          for (int g = 0; g < G; ++g) {
            const float2 t2 = halves(h[g / 2]);
            const float t = g & 1 ? t2.y : t2.x;
#pragma unroll
            for (int m = 0; m < NT; ++m) p[g][m][e] = Pair<__half>::pack(x[u][m][2 * e] * t, x[u][m][2 * e + 1] * t);
          }
        } else {
#pragma unroll
          for (int m = 0; m < NT; ++m) {
            const uint32_t p2 = Pair<__half>::pack(x[u][m][2 * e], x[u][m][2 * e + 1]);
#pragma unroll
            for (int g = 0; g < G; ++g) p[g][m][e] = times_half(p2, h[g / 2], g & 1);
          }
        }
      }
      if (rare) {  // what a row does not see may be of any scale
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int key = key0 + kQ4Slots * u + j0 + 8 * e;
            const uint32_t seen = (key < lim[m][0] ? 0xFFFFu : 0u) | (key < lim[m][1] ? 0xFFFF0000u : 0u);
#pragma unroll
            for (int g = 0; g < G; ++g) p[g][m][e] &= seen;
          }
      }
      if (blank >> u & 1u) continue;  // (the values are zeros)
      uint32_t vw[4][VW];  // of the operand's columns 2 c, 2 c + 1, 2 c + 8, 2 c + 9
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const unsigned char* v = at + u * B::kBytes + (e & 1 ? v1_at : v0_at) + (e >> 1) * 8 * B::kRow;
        if constexpr (VW == 2) {
          uint2 w;
          lds(w, v);
          vw[e][0] = w.x; vw[e][1] = w.y;
        } else {
          lds(vw[e][0], v);
        }
      }
#pragma unroll
      for (int g = 0; g < G; ++g) {
#pragma unroll
        for (int m = 0; m < NT; ++m)
#pragma unroll
          for (int e = 0; e < 2; ++e) p[g][m][e] = transposed(p[g][m][e]);
#pragma unroll
        for (int w = 0; w < VW; ++w) {
#pragma unroll
          for (int e = g * PER; e < g * PER + PER; ++e) {
            // neighbours' bytes side by side
            const uint32_t lo = e < 2 ? 0x5410u : 0x5511u, hi = e < 2 ? 0x7632u : 0x7733u;
            const uint32_t a0 = codes(__byte_perm(vw[0][w], vw[1][w], lo), e);
            const uint32_t a1 = codes(__byte_perm(vw[0][w], vw[1][w], hi), e);
            const uint32_t a2 = codes(__byte_perm(vw[2][w], vw[3][w], lo), e);
            const uint32_t a3 = codes(__byte_perm(vw[2][w], vw[3][w], hi), e);
#pragma unroll
            for (int m = 0; m < NT; ++m) mma_f16(o[m][e][w], a0, a1, a2, a3, p[g][m][0], p[g][m][1]);
          }
        }
      }
    }
    __syncwarp();  // the stage is read
    issue(s + kStages, stage);
    if (++stage == kStages) {
      stage = 0;
      parity ^= 1u;
    }
  }
  if (!waited) {  // what is under way has to land before the ring is used again
    flags |= SSS_FLAG_TIMEOUT;
    for (int i = 0; i < kStages; ++i) {  // (a stage without copies under way: no harm)
      int drain = 0;
      (void)mbar_wait(&full[warp][stage], parity, &drain);
      if (++stage == kStages) {
        stage = 0;
        parity ^= 1u;
      }
    }
  }
  if (flags && a.status) atomicOr(a.status, flags);

  // join the warps
  constexpr int LD = S::LD;
  float* part = reinterpret_cast<float*>(smem);
  __syncthreads();
#pragma unroll
  for (int m = 0; m < NT; ++m)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int row = 8 * m + 2 * c + k;
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) sum[m][k] += __shfl_xor_sync(0xffffffffu, sum[m][k], d);
      if (r == 0) {
        wmax[warp][row] = mx[m][k] == -INFINITY ? -INFINITY : -ref[m][k];
        wsum[warp][row] = sum[m][k];
      }
      float* dst = part + (warp * R + row) * LD + VW * r;
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int h = 0; h < 2; ++h)
        {
          constexpr float kUnit[2] = {0x1p24f, 0x1p20f};
          float* to = dst + 2 * W * e + W * h;
          if constexpr (VW == 2)
            *reinterpret_cast<float2*>(to) = make_float2(o[m][e][0][2 * h + k] * kUnit[e & 1], o[m][e][1][2 * h + k] * kUnit[e & 1]);
          else
            *to = o[m][e][0][2 * h + k] * kUnit[e & 1];
        }
    }
  __syncthreads();
  // pieces of 16 bytes; with CL those of a split follow one another in `gather`
  const uint32_t gather = smem_u32(smem + S::RINGS), lse0 = smem_u32(&split_lse[0][0]);
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
    } else if constexpr (SPLIT == kChunks) {
      const int64_t of = z * static_cast<int64_t>(a.tokens) * a.heads + at;
      if (g < nh) {
        *reinterpret_cast<float4*>(a.part + of * D + d) = acc;
        if (d == 0) a.part_lse[of] = lse;
      }
    } else if constexpr (CL) {
      if (z < n) {
        const int to = x * per_inverse >> 20;
        const uint32_t bar = of_peer(smem_u32(&arrived), to);
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

template <typename T, int D, int NT, Split SPLIT, int WARPS>
cudaError_t run(AttnArgs a, const Q4Cache& c, cudaStream_t stream) {
  constexpr bool CL = SPLIT == kCluster;
  auto kern = attn_rows_q4_kernel<T, D, NT, SPLIT, WARPS>;
  constexpr int smem = RowsQ4Smem<D, 8 * NT, SPLIT, WARPS>::TOTAL;
  cudaError_t e = ensure_smem(kern, smem);
  if (e != cudaSuccess) return e;
  if (CL && a.nsplit > 8) {
    e = ensure_large_cluster(kern);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(32 * WARPS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = CL ? a.nsplit : 1;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = CL ? 2 : 1;
  constexpr int kMost = 65535;  // of a grid's z
  for (; e == cudaSuccess && a.tile0 < a.tiles; a.tile0 += kMost) {
    cfg.gridDim = dim3(a.nsplit, a.kv_heads * a.hchunks, std::min(kMost, a.tiles - a.tile0));
    e = cudaLaunchKernelEx(&cfg, kern, a, c);
  }
  return e;
}
template <typename T, int D, Split SPLIT, int WARPS = 4>
cudaError_t tiles(const AttnArgs& a, const Q4Cache& c, cudaStream_t stream) {
  return a.rows == 8 ? run<T, D, 1, SPLIT, WARPS>(a, c, stream) : run<T, D, 2, SPLIT, WARPS>(a, c, stream);
}
template <typename T, int D>
cudaError_t splits(const AttnArgs& a, const Q4Cache& c, cudaStream_t stream) {
  if (a.nsplit == 1) return tiles<T, D, kWhole>(a, c, stream);
  if (a.chunk > 0) return tiles<T, D, kChunks>(a, c, stream);
  return a.warps == 8 ? tiles<T, D, kCluster, 8>(a, c, stream) : tiles<T, D, kCluster>(a, c, stream);
}

}  // namespace

cudaError_t launch_attn_rows_q4(const AttnArgs& a, const Q4Cache& c, int dtype, int dim, cudaStream_t stream) {
  if (dtype == SSS_OUT_F16) return dim == 64 ? splits<__half, 64>(a, c, stream) : splits<__half, 128>(a, c, stream);
  return dim == 64 ? splits<__nv_bfloat16, 64>(a, c, stream) : splits<__nv_bfloat16, 128>(a, c, stream);
}

}  // namespace sss
