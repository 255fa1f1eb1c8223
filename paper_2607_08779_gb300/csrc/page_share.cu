// page_share.cu -- pages that several rows of a block table hold: forking rows, finding
// the free pages again (and moving held ones down), and copying pages.
//
// Nothing keeps counts of a page's holders: the table says who holds what.  Forking reads
// rows and writes rows; the free pages are those that no row names.  So a request ends, a
// beam is dropped or a length cut by changing the table's rows and lengths alone.  (A row that
// was cut into a page which others hold goes through a fork, of itself if need be, before it
// gets new tokens: that is where pages are given their writers.)
#include <algorithm>

#include "kv_q4.cuh"

namespace sss {
namespace {

// ---------------------------------------------------------------------------
// Fork.  Row r takes the pages of past[p] tokens of its parent p: all shared, but a last
// one that is partly filled, which one row alone may hold: the first of those that end in
// it, unless a row holds all of it (a length may have been cut into a page that other
// rows share, so it is the page that counts and not the parent).  The free pages that the others
// take are numbered by an exclusive sum over the rows.
//
// Bound by latency where rows are few, by the tables' bytes where they are long (each
// parent's entries are looked at, each row's read and written).  One launch.  Its first cluster
// says who ends in what: each of its CTAs puts the rows' last pages in a hash table of its own, with the
// first row of each, and looks up its share of the parents' full pages in it; what it finds is a bit
// for that first row in every CTA.  The first CTA then numbers the rows.  The other CTAs write the new
// table meanwhile, all of it but those last pages' entries, which the first CTA writes.
// 16 rows of 128 entries: 3.9 us; 64 of 513 from 64 parents 5.2; 512 of 2049 7.6; 1024 of 257 from 256
// parents 7.1.  Looking at an entry costs a dozen instructions and a read of shared memory at a place of
// its own: 49,000 of them take one SM 8 us.
// ---------------------------------------------------------------------------

constexpr int kForkThreads = 1024;     // 256 where rows and tables are small
constexpr int kForkCtas = 16;          // of the first cluster
constexpr int kForkPiece = 256;        // entries that a warp takes at a time
constexpr int kMaxRows = 65536;
constexpr int kForkChunk = 8192;       // rows whose pages are in the hash table at a time
constexpr int32_t kNoKey = INT32_MIN;  // (of it: free)

struct ForkArgs {
  const int32_t *parents, *past, *free_pages, *table;
  int32_t *new_table, *new_past, *src, *dst, *used;
  uint32_t* status;
  int rows, batch, nfree, width, shift;
  int slots;    // of the hash table, a power of two
  int cluster;  // CTAs of the first cluster
};

__device__ __forceinline__ int warp_sum_to(int v, int lane) {
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int o = __shfl_up_sync(0xffffffffu, v, d);
    if (lane >= d) v += o;
  }
  return v;
}
__device__ __forceinline__ void cluster_meet() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t of_rank(const uint32_t* p, int rank) {
  uint32_t addr = static_cast<uint32_t>(__cvta_generic_to_shared(p));
  asm("mapa.shared::cluster.u32 %0, %0, %1;" : "+r"(addr) : "r"(rank));
  return addr;
}

// row r's parent and its tokens, whatever the call holds; -1 and 0 of an empty row
__device__ __forceinline__ int parent_of_row(const ForkArgs& a, int r, int64_t& past, uint32_t& flags) {
  past = 0;
  int parent = a.parents[r];
  if (parent >= a.batch) {
    flags |= SSS_FLAG_INDEX;
    parent = -1;
  }
  if (parent < 0) return -1;
  past = a.past[parent];
  const int64_t most = static_cast<int64_t>(a.width) << a.shift;
  if (past < 0 || past > most) {
    flags |= SSS_FLAG_INDEX;
    past = past < 0 ? 0 : most;
  }
  return parent;
}
// what a row ends in: its last page where that is partly filled (an entry that is none: another
// negative number for each parent), or kNoKey
__device__ __forceinline__ int32_t last_page(const ForkArgs& a, int parent, int64_t past) {
  if (parent < 0 || (past & ((1 << a.shift) - 1)) == 0) return kNoKey;
  const int32_t page = a.table[static_cast<int64_t>(parent) * a.width + (past >> a.shift)];
  return page >= 0 ? page : -2 - parent;
}
// where a key is looked for first in the hash table; its slot there, from that one on, `add`: it is
// put there, else -1 where it is not
__device__ __forceinline__ int first_slot(int slots, int32_t key) {
  const uint32_t h = static_cast<uint32_t>(key) * 2654435761u;
  return static_cast<int>((h ^ h >> 15) & (slots - 1));
}
__device__ __forceinline__ int slot_of(int32_t* keys, int slots, int32_t key, int h, bool add) {
  for (int i = 0; i < slots; ++i) {  // (at most half of them are taken)
    const int at = (h + i) & (slots - 1);
    const int32_t old = add ? atomicCAS(&keys[at], kNoKey, key) : keys[at];
    if (old == key) return at;
    if (old == kNoKey) return add ? at : -1;
  }
  return -1;
}
// The new table but for the entries of partly filled last pages: CTA `cta` of `ctas`.
__device__ __forceinline__ void write_rows(const ForkArgs& a, int cta, int ctas) {
  const int lane = threadIdx.x & 31, warps = blockDim.x / 32;
  const uint32_t pieces = (a.width + int64_t{kForkPiece} - 1) / kForkPiece;
  const uint32_t items = static_cast<uint32_t>(a.rows) * pieces;  // (2^32 are more than fit in memory)
  for (uint32_t i = cta * warps + (threadIdx.x >> 5); i < items; i += ctas * warps) {
    const int r = static_cast<int>(i / pieces), c0 = static_cast<int>(i - r * pieces) * kForkPiece;
    int64_t past;
    uint32_t said = 0;
    const int parent = parent_of_row(a, r, past, said);
    const int whole = static_cast<int>(past >> a.shift);
    const int open = (past & ((1 << a.shift) - 1)) != 0 ? whole : -1;
    const int32_t* in = a.table + static_cast<int64_t>(max(parent, 0)) * a.width;
    int32_t* out = a.new_table + static_cast<int64_t>(r) * a.width;
    int32_t v[kForkPiece / 32];
#pragma unroll
    for (int k = 0; k < kForkPiece / 32; ++k) {
      const int c = c0 + 32 * k + lane;
      v[k] = c < whole ? __ldg(in + c) : -1;
    }
#pragma unroll
    for (int k = 0; k < kForkPiece / 32; ++k) {
      const int c = c0 + 32 * k + lane;
      if (c < a.width && c != open) out[c] = v[k];
    }
  }
}

__global__ void __launch_bounds__(kForkThreads, 1) page_fork_kernel(const __grid_constant__ ForkArgs a) {
  extern __shared__ __align__(16) int32_t hashed[];  // the hash table: keys, then first rows
  __shared__ uint32_t met[kMaxRows / 32];    // parents of a row
  __shared__ uint32_t full[kMaxRows / 32];   // first rows whose page some row holds all of
  __shared__ uint32_t keeps[kMaxRows / 32];  // rows that keep their last page
  __shared__ int warp_takes[kForkThreads / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int threads = blockDim.x, warps = threads / 32;
  const int ctas = a.cluster, me = blockIdx.x;
  const bool looks = me < ctas;  // a CTA of the first cluster
  int32_t *keys = hashed, *firsts = hashed + a.slots;
  uint32_t flags = 0;
  if (looks) {
    for (int i = tid; i < (a.batch + 31) / 32; i += threads) met[i] = 0;
    for (int i = tid; i < (a.rows + 31) / 32; i += threads) full[i] = keeps[i] = 0;
    for (int i = tid; i < a.slots; i += threads) {
      keys[i] = kNoKey;
      firsts[i] = INT32_MAX;
    }
    if (ctas > 1) cluster_meet();  // (before a peer's first bit)
    else __syncthreads();
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (!looks) {
    write_rows(a, me - ctas, gridDim.x - ctas);
    return;
  }
  // a row's parent, tokens and last page; a thread looks once where it has one row
  const bool one = a.rows <= threads;
  int parent = -1;
  int64_t past = 0;
  int32_t key = kNoKey;
  const auto look = [&](int r) {
    parent = parent_of_row(a, r, past, flags);
    key = last_page(a, parent, past);
  };
  // the parents' full pages, a warp to a piece of them, the next one's entries under way
  const uint32_t pieces = (a.width + int64_t{kForkPiece} - 1) / kForkPiece;
  const uint32_t items = static_cast<uint32_t>(a.batch) * pieces;
  struct Piece {
    int b, c0, past;
    int32_t v[kForkPiece / 32];
  };
  const auto load = [&](Piece& p, uint32_t i) {
    if (i >= items) return;
    p.b = static_cast<int>(i / pieces);
    p.c0 = static_cast<int>(i - p.b * pieces) * kForkPiece;
    p.past = a.past[p.b];
    const int32_t* row = a.table + static_cast<int64_t>(p.b) * a.width;
#pragma unroll
    for (int k = 0; k < kForkPiece / 32; ++k) {
      const int c = p.c0 + 32 * k + lane;
      p.v[k] = c < a.width ? row[c] : -1;
    }
  };
  const uint32_t item0 = me * warps + warp;
  for (int chunk = 0; chunk < a.rows; chunk += kForkChunk) {
    const int end = min(a.rows, chunk + kForkChunk);
    Piece p, next;
    load(next, item0);
    // the chunk's rows into the table; then the others, for what of it they end in too
    for (int r = chunk + tid; r < end; r += threads) {
      look(r);
      if (parent >= 0) atomicOr(&met[parent >> 5], 1u << (parent & 31));
      if (key != kNoKey) atomicMin(&firsts[slot_of(keys, a.slots, key, first_slot(a.slots, key), true)], r);
    }
    if (a.rows > kForkChunk) {
      __syncthreads();
      for (int r = tid; r < a.rows; r += threads) {
        if (r >= chunk && r < end) continue;
        look(r);
        if (parent >= 0) atomicOr(&met[parent >> 5], 1u << (parent & 31));
        const int at = key == kNoKey ? -1 : slot_of(keys, a.slots, key, first_slot(a.slots, key), false);
        if (at >= 0) atomicMin(&firsts[at], r);
      }
    }
    __syncthreads();
    for (uint32_t i = item0; i < items; i += ctas * warps) {
      p = next;
      load(next, i + ctas * warps);
      if (!(met[p.b >> 5] >> (p.b & 31) & 1u)) continue;
      const int left = (max(0, p.past) >> a.shift) - p.c0 - lane;  // full pages from the lane's first on
      uint32_t hit = 0;  // entries whose first slot is not free (few: most slots are)
#pragma unroll
      for (int k = 0; k < kForkPiece / 32; ++k)
        if (keys[first_slot(a.slots, p.v[k])] != kNoKey && p.v[k] >= 0 && 32 * k < left) hit |= 1u << k;
#pragma unroll
      for (int k = 0; k < kForkPiece / 32; ++k) {
        if (!(hit >> k & 1u)) continue;
        const int at = slot_of(keys, a.slots, p.v[k], first_slot(a.slots, p.v[k]), false);
        if (at < 0) continue;
        const int first = firsts[at];
        if (ctas == 1) {
          atomicOr(&full[first >> 5], 1u << (first & 31));
          continue;
        }
        for (int c = 0; c < ctas; ++c)
          asm volatile("red.relaxed.cluster.shared::cluster.or.b32 [%0], %1;" ::"r"(of_rank(&full[first >> 5], c)),
                       "r"(1u << (first & 31))
                       : "memory");
      }
    }
    if (ctas > 1) cluster_meet();
    else __syncthreads();
    if (me == 0) {
      for (int r = chunk + tid; r < end; r += threads) {
        if (!one) look(r);
        if (key == kNoKey || firsts[slot_of(keys, a.slots, key, first_slot(a.slots, key), false)] != r) continue;
        if (!(full[r >> 5] >> (r & 31) & 1u)) atomicOr(&keeps[r >> 5], 1u << (r & 31));
      }
    }
    __syncthreads();
    if (end == a.rows) break;
    for (int i = tid; i < a.slots; i += threads) {
      keys[i] = kNoKey;
      firsts[i] = INT32_MAX;
    }
    __syncthreads();
  }
  if (me > 0) return;
  // the rows in order: which pages they end with
  int taken = 0;
  for (int r0 = 0; r0 < a.rows; r0 += threads) {
    const int r = r0 + tid;
    bool take = false;
    if (r < a.rows) {
      if (!one) look(r);
      take = key != kNoKey && !(keeps[r >> 5] >> (r & 31) & 1u);
    }
    const bool none = take && key < 0;  // nothing to copy
    if (none) {
      flags |= SSS_FLAG_INDEX;
      take = false;
    }
    const int upto = warp_sum_to(take ? 1 : 0, lane);
    if (lane == 31) warp_takes[warp] = upto;
    __syncthreads();
    const int takes = lane < warps ? warp_takes[lane] : 0;
    const int sums = warp_sum_to(takes, lane);
    const int at = taken + __shfl_sync(0xffffffffu, sums - takes, warp) + upto - 1;
    taken += __shfl_sync(0xffffffffu, sums, 31);
    if (r < a.rows) {
      int from = -1, to = -1, held = static_cast<int>(past);
      const int whole = held >> a.shift;
      int32_t* last = a.new_table + static_cast<int64_t>(r) * a.width + whole;
      if (take) {
        to = at < a.nfree ? a.free_pages[at] : -1;
        if (to >= 0) from = key;
        else flags |= SSS_FLAG_PAGES;
        to = max(to, -1);
      }
      if (none || (take && to < 0)) held = whole << a.shift;  // it ends with its last full page
      if (key != kNoKey) *last = take || none ? to : key >= 0 ? key : a.table[static_cast<int64_t>(parent) * a.width + whole];
      a.new_past[r] = held;
      a.src[r] = from;
      a.dst[r] = to;
    }
    __syncthreads();
  }
  if (tid == 0) *a.used = min(taken, a.nfree);
  if (flags && a.status) atomicOr(a.status, flags);
}

// ---------------------------------------------------------------------------
// Reclaim.  One cluster: each CTA sets the bits of the pages that its share of the table
// names in a map of its own, the CTAs join their maps (each a slice of it from all, then
// every slice from its CTA), and every CTA counts the map's words.  With rk(x) held pages
// below x, m in all and k moves, the free page x is the (x - rk(x))-th and the held one the
// (m - 1 - rk(x))-th from above: both say by themselves which move they belong to
// and where in the list what is free afterwards stands:
//   a free page that stays free: its number less the k that are taken, and the held pages
//     below it that moved away, max(0, rk(x) - (m - k));
//   one that moved away: rk(x) - (m - k), and the x - rk(x) - k free ones below it.
// Bound by latency: a few waits of the cluster, and the table's entries, whose bits are set and
// (with moves) looked up in shared memory.  16 requests, 4000 pages: 4.6 us; 256 requests of up
// to 1024 entries, 51,000 pages, with moves: 13.6 us.
// ---------------------------------------------------------------------------

constexpr int kMapThreads = 1024;
constexpr int kMapCtas = 16;
constexpr int kSpan = 8;  // words of the map to one running count
constexpr int kMapPiece = 512;  // entries that a warp takes at a time (128: 16.0 us for the last case above)

struct MapArgs {
  const int32_t *table, *past;
  int32_t *free_pages, *free_count, *new_table, *src, *dst, *moves;
  uint32_t* status;
  int batch, width, shift, pages, most;
};

__device__ __forceinline__ uint32_t peer_word(const uint32_t* p, int rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(of_rank(p, rank)) : "memory");
  return v;
}
// the entries of row b that hold pages
__device__ __forceinline__ int held_entries(const MapArgs& a, int b, uint32_t& flags) {
  int64_t past = a.past[b];
  const int64_t most = static_cast<int64_t>(a.width) << a.shift;
  if (past < 0 || past > most) {
    flags |= SSS_FLAG_INDEX;
    past = past < 0 ? 0 : most;
  }
  return static_cast<int>((past + (1 << a.shift) - 1) >> a.shift);
}

__global__ void __launch_bounds__(kMapThreads, 1) page_map_kernel(const __grid_constant__ MapArgs a) {
  extern __shared__ __align__(16) uint32_t map[];  // [words], then the counts [spans] and [words]
  __shared__ int warp_held[32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int ctas = gridDim.x, me = blockIdx.x;  // (one cluster)
  const int spans = (a.pages + 32 * kSpan - 1) / (32 * kSpan), words = spans * kSpan;
  int* count = reinterpret_cast<int*>(map + words);
  uint8_t* in_span = reinterpret_cast<uint8_t*>(count + spans);  // of each word, from its span's first
  uint32_t flags = 0;
  for (int i = tid; i < words; i += kMapThreads) map[i] = 0;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  __syncthreads();
  // the rows' entries, a warp to a piece of them
  constexpr int kWarps = kMapThreads / 32, kPiece = kMapPiece;
  const int pieces = (a.width + kPiece - 1) / kPiece;
  const int64_t items = static_cast<int64_t>(a.batch) * pieces;
  for (int64_t i = static_cast<int64_t>(me) * kWarps + warp; i < items; i += static_cast<int64_t>(ctas) * kWarps) {
    const int b = static_cast<int>(i / pieces), c0 = static_cast<int>(i - static_cast<int64_t>(b) * pieces) * kPiece;
    const int held = held_entries(a, b, flags);
    const int32_t* row = a.table + static_cast<int64_t>(b) * a.width;
    int32_t v[kPiece / 32];
#pragma unroll
    for (int k = 0; k < kPiece / 32; ++k) {
      const int c = c0 + 32 * k + lane;
      v[k] = c < held ? row[c] : 0;
    }
#pragma unroll
    for (int k = 0; k < kPiece / 32; ++k) {
      if (c0 + 32 * k + lane >= held) continue;
      if (v[k] < 0 || v[k] >= a.pages) flags |= SSS_FLAG_INDEX;
      else atomicOr(&map[v[k] >> 5], 1u << (v[k] & 31));
    }
  }
  if (ctas > 1) {
    cluster_meet();
    const int slice = (words + ctas - 1) / ctas;
    for (int i = me * slice + tid; i < min(words, (me + 1) * slice); i += kMapThreads) {
      uint32_t v = 0, of[kMapCtas];
#pragma unroll
      for (int c = 0; c < kMapCtas; ++c) of[c] = c < ctas ? peer_word(map + i, c) : 0u;
#pragma unroll
      for (int c = 0; c < kMapCtas; ++c) v |= of[c];
      map[i] = v;
    }
    cluster_meet();
    for (int i = tid; i < words; i += kMapThreads)
      if (i / slice != me) map[i] = peer_word(map + i, i / slice);
  }
  __syncthreads();
  // counts: of the spans, then their sums
  int m = 0;
  for (int s0 = 0; s0 < spans; s0 += kMapThreads) {
    const int s = s0 + tid;
    int n = 0;
    if (s < spans)
#pragma unroll
      for (int w = 0; w < kSpan; ++w) {
        in_span[s * kSpan + w] = static_cast<uint8_t>(n);  // (224 at most)
        n += __popc(map[s * kSpan + w]);
      }
    const int upto = warp_sum_to(n, lane);
    if (lane == 31) warp_held[warp] = upto;
    __syncthreads();
    const int of = warp_held[lane];
    const int sums = warp_sum_to(of, lane);
    const int before = __shfl_sync(0xffffffffu, sums - of, warp);
    if (s < spans) count[s] = m + before + upto - n;
    m += __shfl_sync(0xffffffffu, sums, 31);
    __syncthreads();
  }
  const auto rank_of = [&](int x) {  // held pages below x
    const int w = x >> 5;
    return count[w / kSpan] + in_span[w] + __popc(map[w] & ((1u << (x & 31)) - 1));
  };
  // moves: as many as there are free pages below m
  int k = 0;
  if (a.moves && m < a.pages) k = min(a.most, m - rank_of(m));
  // the lists, a warp to a span
  for (int s = me * kWarps + warp; s < spans; s += ctas * kWarps) {
    int below = count[s];
#pragma unroll
    for (int i = 0; i < kSpan; ++i) {
      const uint32_t bits = map[s * kSpan + i];
      const int x = 32 * (s * kSpan + i) + lane;
      const int rk = below + __popc(bits & ((1u << lane) - 1));
      below += __popc(bits);
      if (x >= a.pages) continue;
      int pos = -1;
      if (bits >> lane & 1u) {
        const int j = m - 1 - rk;
        if (j < k) {
          a.src[j] = x;
          pos = rk - (m - k) + (x - rk) - k;
        }
      } else {
        const int j = x - rk;
        if (j < k) a.dst[j] = x;
        else pos = j - k + max(0, rk - (m - k));
      }
      if (pos >= 0) a.free_pages[pos] = x;
      if (x >= a.pages - m) a.free_pages[x] = -1;
    }
  }
  if (me == 0 && tid == 0) {
    *a.free_count = a.pages - m;
    if (a.moves) *a.moves = k;
  }
  if (a.moves) {
    for (int i = k + me * kMapThreads + tid; i < a.most; i += ctas * kMapThreads) a.src[i] = a.dst[i] = -1;
    // the moves of all CTAs; pages from the last one's source on are moved
    if (ctas > 1) cluster_meet();
    else __syncthreads();
    const int lowest = k > 0 ? __ldcg(a.src + k - 1) : INT32_MAX;
    for (int64_t i = static_cast<int64_t>(me) * kWarps + warp; i < items; i += static_cast<int64_t>(ctas) * kWarps) {
      const int b = static_cast<int>(i / pieces), c0 = static_cast<int>(i - static_cast<int64_t>(b) * pieces) * kPiece;
      uint32_t said = 0;
      const int held = held_entries(a, b, said);
      const int64_t at = static_cast<int64_t>(b) * a.width;
      int32_t v[kPiece / 32];
#pragma unroll
      for (int e = 0; e < kPiece / 32; ++e) {
        const int c = c0 + 32 * e + lane;
        v[e] = c < held ? a.table[at + c] : -1;
      }
#pragma unroll
      for (int e = 0; e < kPiece / 32; ++e)
        if (v[e] >= lowest && v[e] < a.pages) v[e] = __ldcg(a.dst + (m - 1 - rank_of(v[e])));
#pragma unroll
      for (int e = 0; e < kPiece / 32; ++e) {
        const int c = c0 + 32 * e + lane;
        if (c < held) a.new_table[at + c] = v[e];
      }
    }
  }
  if (flags && a.status) atomicOr(a.status, flags);
  // nobody leaves while a peer may still read its map
  if (ctas > 1) cluster_meet();
}

// ---------------------------------------------------------------------------
// Copy.  Each CTA takes pieces of the pages that are to be copied, of one cache after the
// other.  Bound by HBM, or by the launch where pages are few: all layers go in one.  500 pages of
// 128 KB, keys and values: 42.3 us, 6.2 TB/s, 92 % of the copy rate; 12 pages of 18 KB in 32 layers:
// 4.1 us.
// ---------------------------------------------------------------------------

constexpr int kCopyThreads = 256;
constexpr int kCopyCtas = 4;      // an SM
constexpr int kCopyUnroll = 4;    // 16-byte loads in flight a thread

struct CopyArgs {
  char* base[2 * kMaxCopyCaches];      // keys and values, or blocks
  int64_t stride[2 * kMaxCopyCaches];  // bytes from a page to the next
  const int32_t *src, *dst;
  uint32_t* status;
  int64_t pages;
  int parts, n;
  int rows, row16;  // evenly spaced rows of a page (a power of two), 16-byte units of a row
  int row_shift;
  int pieces;       // of a page
};

__global__ void __launch_bounds__(kCopyThreads, kCopyCtas) page_copy_kernel(const __grid_constant__ CopyArgs a) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  constexpr int kPiece = kCopyThreads * kCopyUnroll;  // units
  const int64_t items = static_cast<int64_t>(a.n) * a.parts * a.pieces;
  const int units = a.rows * a.row16;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t e = it / a.pieces;
    const int piece = static_cast<int>(it - e * a.pieces);
    const int part = static_cast<int>(e / a.n), i = static_cast<int>(e - static_cast<int64_t>(part) * a.n);
    const int64_t from = a.src[i], to = a.dst[i];
    if (from < 0 || to < 0 || from >= a.pages || to >= a.pages) {
      if ((from >= 0 || to >= 0) && threadIdx.x == 0 && a.status) atomicOr(a.status, SSS_FLAG_INDEX);
      continue;
    }
    const int64_t stride = a.stride[part], row_stride = stride >> a.row_shift;
    const char* in = a.base[part] + from * stride;
    char* out = a.base[part] + to * stride;
    uint4 v[kCopyUnroll];
    int64_t at[kCopyUnroll];
#pragma unroll
    for (int u = 0; u < kCopyUnroll; ++u) {
      const int x = piece * kPiece + u * kCopyThreads + threadIdx.x;
      const int row = x / a.row16;
      at[u] = row * row_stride + static_cast<int64_t>(x - row * a.row16) * 16;
      if (x < units) v[u] = __ldcs(reinterpret_cast<const uint4*>(in + at[u]));
    }
#pragma unroll
    for (int u = 0; u < kCopyUnroll; ++u)
      if (piece * kPiece + u * kCopyThreads + threadIdx.x < units) *reinterpret_cast<uint4*>(out + at[u]) = v[u];
  }
}

template <typename K, typename A>
cudaError_t launch(K kern, const A& a, int64_t ctas, int threads, int smem, int cluster, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(ctas));
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

int shift_of(int page_size) {
  int s = 0;
  while ((1 << s) < page_size) ++s;
  return s;
}

cudaError_t copy(CopyArgs& a, cudaStream_t stream) {
  const int units = a.rows * a.row16;
  a.row_shift = shift_of(a.rows);
  a.pieces = (units + kCopyThreads * kCopyUnroll - 1) / (kCopyThreads * kCopyUnroll);
  const int64_t items = static_cast<int64_t>(a.n) * a.parts * a.pieces;
  return launch(page_copy_kernel, a, std::min<int64_t>(items, int64_t{kCopyCtas} * device_sm_count()),
                kCopyThreads, 0, 1, stream);
}

}  // namespace

cudaError_t launch_page_fork(const int32_t* parents, int rows, const int32_t* past, int batch,
                             int page_size, const int32_t* free_pages, int nfree,
                             const int32_t* table, int width, int32_t* new_table,
                             int32_t* new_past, int32_t* src, int32_t* dst, int32_t* used,
                             uint32_t* status, cudaStream_t stream) {
  ForkArgs a = {parents, past, free_pages, table, new_table, new_past, src, dst, used,
                status, rows, batch, nfree, width, shift_of(page_size), 64, 1};
  while (a.slots < 2 * kForkChunk && a.slots < 8 * rows) a.slots *= 2;
  cudaError_t e = ensure_smem(page_fork_kernel, 2 * kForkChunk * 8);
  if (e != cudaSuccess) return e;
  const int64_t pieces = (width + int64_t{kForkPiece} - 1) / kForkPiece;
  const int64_t parts = batch * pieces, items = rows * pieces;
  // A thread to a row, and CTAs until a warp has one piece to look at (64 rows of 513 from 64 parents, 8
  // CTAs of 512 threads: 5.2 us, 16 of 256 5.9, 8 of 1024 6.0, two pieces a warp 6.2; 1024 of 257 from 256
  // parents, 8 of 1024 threads 7.0, 16 of 512 10.5, two pieces a warp 8.6; 4 of 20 from one, 256 threads 3.1,
  // 512 3.3, 1024 3.6).
  const int threads = rows <= 256 && parts <= 8 ? 256 : rows <= 512 ? 512 : kForkThreads, warps = threads / 32;
  while (a.cluster < kForkCtas && parts > int64_t{a.cluster} * warps) a.cluster *= 2;
  if (a.cluster > 8) {
    e = ensure_large_cluster(page_fork_kernel);
    if (e != cudaSuccess) return e;
  }
  // (CTAs that write: about one an SM, in whole clusters)
  const int64_t writers = std::min<int64_t>((items + warps - 1) / warps, device_sm_count());
  const int64_t ctas = (1 + (writers + a.cluster - 1) / a.cluster) * a.cluster;
  return launch(page_fork_kernel, a, ctas, threads, a.slots * 8, a.cluster, stream);
}

cudaError_t launch_page_reclaim(const int32_t* table, int width, const int32_t* past, int batch,
                                int page_size, int pages, int32_t* free_pages, int32_t* free_count,
                                int32_t* new_table, int32_t* src, int32_t* dst, int most,
                                int32_t* moves, uint32_t* status, cudaStream_t stream) {
  const MapArgs a = {table, past, free_pages, free_count, new_table, src, dst, moves,
                     status, batch, width, shift_of(page_size), pages, most};
  const int spans = (pages + 32 * kSpan - 1) / (32 * kSpan);
  const int smem = spans * (kSpan * 4 + 4 + kSpan);
  cudaError_t e = ensure_smem(page_map_kernel, kMaxMapPages / (32 * kSpan) * (kSpan * 4 + 4 + kSpan));
  if (e != cudaSuccess) return e;
  // CTAs until three of four of their warps, at most, have a piece of the table, or a span of the map
  // (16 requests of up to 4096 tokens: 4.6 us with one CTA, 6.1 with two.  64 of up to 8192 with moves: 33.2,
  // 21.3, 13.5, 12.4 and 12.0 us with 1, 2, 4, 8 and 16; 256 of up to 16384: 91.7, 53.2, 30.7, 19.1 and
  // 13.6.  From 48 pieces a CTA on instead: 256 of up to 1000 tokens 10.9 us, so 10.1; 8 of up to 32768
  // 18.5, so 14.4.)
  const int64_t work = std::max<int64_t>(static_cast<int64_t>(batch) * ((width + kMapPiece - 1) / kMapPiece), spans);
  int ctas = 1;
  while (ctas < kMapCtas && work > ctas * 24) ctas *= 2;
  if (ctas > 8) {
    e = ensure_large_cluster(page_map_kernel);
    if (e != cudaSuccess) return e;
  }
  return launch(page_map_kernel, a, ctas, kMapThreads, smem, ctas, stream);
}

cudaError_t launch_page_copy(const sss_kv_cache_t* const* caches, int count, const int32_t* src,
                             const int32_t* dst, int n, uint32_t* status, cudaStream_t stream) {
  CopyArgs a = {};
  const sss_kv_cache_t& c = *caches[0];
  const bool dense = std::all_of(caches, caches + count, [](const sss_kv_cache_t* x) {
    return x->stride == static_cast<int64_t>(x->heads) * x->dim;
  });
  a.rows = dense ? 1 : c.page_size;
  a.row16 = c.heads * c.dim / 8 * (dense ? c.page_size : 1);
  for (int i = 0; i < count; ++i)
    for (int v = 0; v < 2; ++v) {
      a.base[2 * i + v] = static_cast<char*>(v ? caches[i]->v : caches[i]->k);
      a.stride[2 * i + v] = caches[i]->stride * 2 * c.page_size;
    }
  a.src = src;
  a.dst = dst;
  a.status = status;
  a.pages = c.slots / c.page_size;
  a.parts = 2 * count;
  a.n = n;
  return copy(a, stream);
}

cudaError_t launch_page_copy_q4(const sss_kv_cache_q4_t* const* caches, int count,
                                const int32_t* src, const int32_t* dst, int n, uint32_t* status,
                                cudaStream_t stream) {
  CopyArgs a = {};
  const sss_kv_cache_q4_t& c = *caches[0];
  a.rows = 1;
  a.row16 = c.heads * (c.page_size / 16) * (18 * c.dim / 16);
  for (int i = 0; i < count; ++i) {
    a.base[i] = static_cast<char*>(caches[i]->blocks);
    a.stride[i] = caches[i]->page_stride;
  }
  a.src = src;
  a.dst = dst;
  a.status = status;
  a.pages = c.pages;
  a.parts = count;
  a.n = n;
  return copy(a, stream);
}

}  // namespace sss
