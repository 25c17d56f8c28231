// What the kernels of the attention over the paged cache share: arguments, the slots that a row tile looks
// at, and how the work is cut into equal shares.
//
// The query rows of a sequence that share a KV head (row r = query r / G, head r % G of the group) are cut
// into row tiles, and the slots that a row tile sees into tiles of 128.  Row tile by row tile, KV head by KV
// head, slot tile by slot tile, the tiles of a launch form one line, in which every (row tile, head) also takes
// kItemCost places for what it costs by itself; CTA c of g walks places T c / g .. T (c + 1) / g - 1.  So
// every CTA has the same work to a tile, whatever the lengths are, and at most its first and its last (row
// tile, head) are shared with others: those leave a normalised partial output and its log-sum-exp per row
// (slot 2 c: it begins inside, 2 c + 1: it begins there and goes on elsewhere), which kv_attn_combine weighs
// together.  The log-sum-exp stays in two terms, a score and the logarithm of a sum relative to it: of large scores 32 bits
// would not hold the sum of both (at 2^20 to an eighth).
//
// The kernels have a second form, TREE, for queries that are nodes of a tree of drafted tokens: a node sees the slots before the tree
// (as far as the window around its position, base + its depth, lets it) and of the tree's those whose bits kv_tree.cu has set for it.
#pragma once
#include <cuda.h>

#include "pace_kv.cuh"
#include "pace_ptx.cuh"

namespace pace {

constexpr int kKvTile = 128;      // slots of one tile
constexpr float kNone = -0x1p127f;   // a row's maximum before its first slot, below any score (and finite: x - kNone is never NaN)
constexpr int kManyRows = 256;    // rows of a tile of the form for many
constexpr int kItemCost = 3;      // slot tiles that the queries and the output of a (row tile, head) are worth (pace.h states both: the size of a launch),
constexpr int kTreeCost = 6;      // of trees of many rows (with 5, 6, 7: 16 ragged ones of dim 64 24.0, 24.9, 26.2 us; 32 of 128 rows on 700-9000 slots 103, 101, 96)
constexpr int kPlanCtas = 152;    // CTAs of a launch at most: an SM each (the size queries need no device)

// The launch's sequences, those without queries left out.
struct KvSeqs {
  int nb;
  int seq[kKvMaxB];        // number in the call
  int q0[kKvMaxB];         // first query
  int nq[kKvMaxB];
  int tile0[kKvMaxB + 1];  // row tiles before it
};

// Written by CTA c where its last (row tile, head) goes on in CTAs c + 1 .. c + followers.
struct KvSplit {
  int i, row_tile, head, followers;
};

struct KvAttnArgs {
  KvView c;
  const uint16_t* Q;
  uint16_t* out;
  float* lse;
  int64_t q_stride, table_stride;
  const int32_t* lens;
  const int32_t* table;
  KvSplit* split;       // [CTAs]
  float2* part_lse;     // [2 CTAs][rows of a tile], base 2: score, logarithm relative to it (-inf: saw nothing)
  float* part;          // [2 CTAs][rows of a tile][D]
  float scale2;         // scale * log2(e)
  int q_heads, group, window, sinks, max_len;
  FastDiv by_group;
  KvSeqs s;
  // of a tree, else null:
  const int32_t* depth;     // [queries] a node's ancestors
  const uint32_t* family;   // [queries][words]: word k stands for slots 32 (base / 32 + k) .., rounded down
  int words;
  int after_tree;           // the launch follows kv_tree_kernel, and waits for it only where it reads depth and family
};

__device__ __forceinline__ bool kv_sees(int j, int p, int window, int sinks) {
  return j <= p && (window <= 0 || j > p - window || j < sinks);
}

// The slot tiles that queries at slots p_first .. p_last look at: n of them, the i-th being i for i < head, else i + skip.
struct KvSpan {
  int n, head, skip;
  __device__ __forceinline__ int tile(int i) const { return i < head ? i : i + skip; }
};
__device__ __forceinline__ KvSpan kv_span(int p_first, int p_last, int window, int sinks) {
  KvSpan s{0, 0, 0};
  if (p_last < 0) return s;
  const int end = p_last / kKvTile + 1;
  s.n = s.head = end;
  if (window > 0) {
    const int from = max(p_first - window + 1, 0) / kKvTile;             // first tile of the window
    const int few = min((min(sinks, p_last + 1) + kKvTile - 1) / kKvTile, end);   // tiles that hold the first slots
    if (few < from) s = KvSpan{few + end - from, few, from - few};
  }
  return s;
}

// One (row tile, KV head) of the line, of which this CTA walks slot tiles t0 .. t1 - 1.
struct KvItem {
  int i, row_tile, head, t0, t1;
  int row0, rows;           // its query rows
  int p0;                   // slot of the sequence's query 0
  int p_first, p_last;      // slots of the tile's first and last query (of a tree: of its node 0, a position that none is before, and of the last)
  int p_all;                // the last slot that all rows see, as far as the window lets them
  KvSpan span;
};

template <int ROWS, bool TREE>
__device__ __forceinline__ void kv_item_rows(const KvAttnArgs& a, int i, int row_tile, KvItem& it) {
  it.i = i;
  it.row_tile = row_tile;
  it.p0 = min(max(a.lens[a.s.seq[i]], 0), a.max_len) - a.s.nq[i];
  it.row0 = row_tile * ROWS;
  it.rows = min(a.s.nq[i] * a.group - it.row0, ROWS);
  it.p_first = TREE ? it.p0 : it.p0 + static_cast<int>(a.by_group(it.row0));
  it.p_all = TREE ? it.p0 - 1 : it.p_first;
  it.p_last = it.p0 + static_cast<int>(a.by_group(it.row0 + it.rows - 1));
  it.span = kv_span(it.p_first, it.p_last, a.window, a.sinks);
}

// Output row of the item's row r, (query, head) flattened.
__device__ __forceinline__ int64_t kv_out_row(const KvAttnArgs& a, const KvItem& it, int r) {
  const int row = it.row0 + r, token = static_cast<int>(a.by_group(row));
  return static_cast<int64_t>(a.s.q0[it.i] + token) * a.q_heads + it.head * a.group + row - token * a.group;
}
// Its query.
__device__ __forceinline__ const uint16_t* kv_query(const KvAttnArgs& a, const KvItem& it, int r, int D) {
  const int row = it.row0 + r, token = static_cast<int>(a.by_group(row));
  return a.Q + (a.s.q0[it.i] + token) * a.q_stride + static_cast<int64_t>(it.head * a.group + row - token * a.group) * D;
}

// Bits of a number of columns up to m (0 .. m - 1) out of 32.
__device__ __forceinline__ uint32_t below(int m) { return m >= 32 ? 0xFFFFFFFFu : m <= 0 ? 0u : (1u << m) - 1u; }

// Of slots at .. at + 31 (at >= 0, a multiple of 32) those that a node sees: `node` its query, p its position.
__device__ __forceinline__ uint32_t kv_tree_sees(const KvAttnArgs& a, int base, int64_t node, int p, int at) {
  const uint32_t near = a.window > 0 ? ~below(p - a.window + 1 - at) | below(a.sinks - at) : 0xFFFFFFFFu;
  const int k = (at >> 5) - (base >> 5);
  return (below(base - at) & near) | (k >= 0 && k < a.words ? a.family[node * a.words + k] : 0u);
}

// Where a CTA's share lies; the same for all its threads.  CTA c of a line of total = each * ctas + more tiles begins at
// c * each + min(c, more).  (The call keeps a launch below 2^31 tiles.)
struct KvShare {
  int pos, end;             // its tiles of the line
  int each, more, ctas;
  int cost;                 // places of an item besides its tiles
  int base;                 // first tile of (i, row_tile)
  int i, row_tile;
};

// Walks a share (item) by item.
template <int ROWS, bool TREE>
struct KvWalk {
  KvShare s;
  KvItem it;
  bool have;
  __device__ __forceinline__ void begin(const KvShare& share) {
    s = share;
    have = false;
  }
  __device__ __forceinline__ bool next(const KvAttnArgs& a) {
    if (s.pos >= s.end) return false;
#pragma unroll 1
    while (true) {
      if (!have) {
        kv_item_rows<ROWS, TREE>(a, s.i, s.row_tile, it);
        have = true;
      }
      const uint32_t off = s.pos - s.base, n = it.span.n > 0 ? it.span.n + s.cost : 0;
      if (off < n * a.c.heads) {
        it.head = off / n;
        const int from = off - it.head * n, to = min(static_cast<int>(n), from + (s.end - s.pos));
        s.pos += to - from;
        it.t0 = max(from - s.cost, 0);
        it.t1 = max(to - s.cost, 0);
        if (it.t0 < it.t1) return true;
        if (s.pos >= s.end) return false;
        continue;
      }
      s.base += n * a.c.heads;
      have = false;
      if (++s.row_tile >= a.s.tile0[s.i + 1] - a.s.tile0[s.i]) {
        s.row_tile = 0;
        ++s.i;
      }
    }
  }
};

constexpr int kShareWarps = 12;      // warps of a block at most

// Every thread of the block (whole warps, at most kShareWarps) calls this once; `buf` holds two ints per warp.  Row tiles that see
// nothing get their zeros here.
template <int ROWS, int D, bool TREE>
__device__ __forceinline__ KvShare kv_share(const KvAttnArgs& a, int* buf, KvShare* found, int* status) {
  const int threads = blockDim.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int tiles = a.s.tile0[a.s.nb], per = (tiles + threads - 1) / threads;
  const int first = min(tid * per, tiles), last = min(first + per, tiles);
  int i0 = 0, hi = a.s.nb - 1;      // the sequence of row tile `first`
#pragma unroll 1
  while (i0 < hi) {
    const int mid = (i0 + hi + 1) >> 1;
    if (a.s.tile0[mid] <= first) i0 = mid;
    else hi = mid - 1;
  }
  KvShare s{};
  int mine = 0, items = 0, before = 0;      // of this thread's row tiles: slot tiles, items; places before them
#pragma unroll 1
  for (int round = 0; round < 2; ++round) {      // how many there are; where this CTA's begin
    if (round == 1) {
      int sum = mine, num = items;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, sum, o), y = __shfl_up_sync(0xffffffffu, num, o);
        if (lane >= o) {
          sum += x;
          num += y;
        }
      }
      if (lane == 31) {
        buf[2 * warp] = sum;
        buf[2 * warp + 1] = num;
      }
      __syncthreads();
      int total = 0, total_items = 0, before_items = 0;
#pragma unroll
      for (int w = 0; w < kShareWarps; ++w) {
        if (w >= threads / 32) break;
        if (w == warp) {
          before = total;
          before_items = total_items;
        }
        total += buf[2 * w];
        total_items += buf[2 * w + 1];
      }
      s.ctas = min(static_cast<int>(gridDim.x), total);
      const int c = blockIdx.x;
      if (c >= s.ctas) return s;      // nothing to do (the whole block)
      // (few tiles: one each, however dear the rest is; unless items are so few that a CTA need not have parts of two)
      constexpr int COST = TREE && ROWS == kManyRows ? kTreeCost : kItemCost;
      // (Trees: as soon as a CTA has more than one.  A batch of one long tree and seven short ones, 636 tiles of 52 items, took 68 us where
      // several short items came to one CTA, and takes 33.)
      if (TREE && ROWS == kManyRows) s.cost = total > s.ctas ? COST : 0;
      else s.cost = total >= COST * s.ctas || (total > s.ctas && total >= 4 * COST * total_items) ? COST : 0;
      total += s.cost * total_items;
      before += sum - mine + s.cost * (before_items + num - items);
      mine += s.cost * items;
      s.each = total / s.ctas;
      s.more = total - s.each * s.ctas;
      s.pos = c * s.each + min(c, s.more);
      s.end = s.pos + s.each + (c < s.more ? 1 : 0);
      if (s.pos < before || s.pos >= before + mine) break;
    }
    int i = i0;
#pragma unroll 1
    for (int t = first; t < last; ++t) {
#pragma unroll 1
      while (t >= a.s.tile0[i + 1]) ++i;
      KvItem it;
      kv_item_rows<ROWS, TREE>(a, i, t - a.s.tile0[i], it);
      const int n = it.span.n > 0 ? (it.span.n + s.cost) * a.c.heads : 0;
      if (round == 1) {
        if (s.pos < before + n) {
          s.base = before;
          s.i = i;
          s.row_tile = it.row_tile;
          *found = s;
          break;
        }
        before += n;
        continue;
      }
      mine += n;
      items += n > 0 ? a.c.heads : 0;
      if (blockIdx.x == 0 && it.row_tile == 0 && static_cast<uint32_t>(a.lens[a.s.seq[i]]) > static_cast<uint32_t>(a.max_len)) record_error(status, PACE_ERR_INVALID_ARG, K_KV_ATTN);
      if (n == 0 && t % gridDim.x == blockIdx.x) {
#pragma unroll 1
        for (it.head = 0; it.head < a.c.heads; ++it.head)
#pragma unroll 1
          for (int r = 0; r < it.rows; ++r) {
            const int64_t at = kv_out_row(a, it, r);
#pragma unroll 1
            for (int d = 0; d < D; d += 8) *reinterpret_cast<uint4*>(a.out + at * D + d) = make_uint4(0, 0, 0, 0);
            if (a.lse != nullptr) a.lse[at] = -INFINITY;
          }
      }
    }
  }
  __syncthreads();
  return *found;
}

// What CTA c tells the combine kernel: how many later CTAs its last item goes on in.
__device__ __forceinline__ void kv_write_split(const KvAttnArgs& a, const KvShare& s, const KvItem& it) {
  KvSplit sp{it.i, it.row_tile, it.head, 0};
  if (it.t0 == 0 && it.t1 > 0 && it.t1 < it.span.n) {   // CTA j takes part iff it begins before the item's end
    const int c = blockIdx.x, end = (c + 1) * s.each + min(c + 1, s.more) + it.span.n - it.t1, wide = s.more * (s.each + 1);
    const int last = end <= wide ? (end + s.each) / (s.each + 1) : s.more + (end - wide + s.each - 1) / s.each;
    sp.followers = last - 1 - c;
  }
  a.split[blockIdx.x] = sp;
}

struct KvMaps {
  CUtensorMap k, v;
};

// The start of a launch.  kv_tree_kernel, which needs some microseconds for what is read last, starts when all work before it is
// complete: a launch that follows it need not wait for that again, and waits for it only in threads that come to read what it writes, and
// once before it ends (so what waits for this launch has waited for that one too).
template <bool TREE>
__device__ __forceinline__ void kv_begin(const KvAttnArgs& a) {
  if (!TREE || !a.after_tree) ptx::begin_call();
}
template <bool TREE>
__device__ __forceinline__ void kv_tree_ready(const KvAttnArgs& a) {
  if (TREE && a.after_tree) ptx::begin_call();
}

// mbar_wait with its limit counted in tries (2^18; the hardware holds one that has to wait for about 4 us, which makes a second): a
// few instructions, where the kernels here wait in many places and instructions that are not run push those that are out of the
// instruction cache.
__device__ __forceinline__ bool kv_wait(uint32_t bar, uint32_t parity) {
  int left = 1 << 18;
#pragma unroll 1
  while (!ptx::mbar_try_wait(bar, parity))
    if (--left == 0) return false;
  return true;
}

// A warp's wait, which leaves it converged.
__device__ __forceinline__ bool kv_wait_warp(uint32_t bar, uint32_t parity) {
  int left = 1 << 18;
#pragma unroll 1
  while (!__all_sync(0xffffffffu, ptx::mbar_try_wait(bar, parity)))
    if (--left == 0) return false;
  return true;
}

// A role that gives up on a wait says so here; the others leave as their own waits run out.
__device__ __forceinline__ bool stopped(const int* abort) { return *reinterpret_cast<const volatile int*>(abort) != 0; }
__device__ __forceinline__ void stop(int* abort, int* status) {
  *reinterpret_cast<volatile int*>(abort) = 1;
  record_error(status, PACE_ERR_TIMEOUT, K_KV_ATTN);
}

// N columns of this warp's 32 lanes, ready to use.
template <int N>
__device__ __forceinline__ void load_cols(uint32_t addr, uint32_t (&v)[N]) {
  if constexpr (N == 64) {
    ptx::tmem_ld_32x32b_x64(addr, v);
    ptx::tmem_wait_ld();
    ptx::reg_fence64(v);
  } else {
    ptx::tmem_ld_32x32b(addr, v);
    ptx::tmem_wait_ld();
    ptx::reg_fence(v);
  }
}

// The rings that warp 0 fills: ST places of a K tile, SV of a V tile, `stride` bytes apart.  JOINT: one ring of ST + SV places, K and V of
// a tile one after the other (`k`, `empty`; two arrivals free a place).
struct KvRings {
  uint8_t* k;
  uint8_t* v;
  int stride;
  uint64_t* full;        // [ST] the tile's bytes, their announcement and 32 lanes' copies (33 arrivals)
  uint64_t* empty;       // [ST]
  uint64_t* v_empty;     // [SV] (null: as `empty`, SV = ST)
  float (*scales)[16];   // [ST] a tile's K scales, then its V scales
};

// Warp 0 of a CTA: fetches the slot tiles of its share, K and V in boxes of a page, at most 128 rows, each by TMA; the tile's 8 K
// and 8 V scales by 4-byte copies.
template <int D, int ST, int SV, bool JOINT = false, typename Walk>
__device__ __forceinline__ void kv_fetch(const KvMaps& maps, const KvAttnArgs& a, Walk& walk, const KvRings& ring, int* abort,
                                         int* status) {
  using namespace ptx;
  const int lane = threadIdx.x & 31;
  const int shift = min(a.c.page_shift, 7), box_rows = 1 << shift, boxes = kKvTile >> shift;
  const int tiles_per_load = 32 / boxes;     // a lane holds the page of one box
  int t = 0;                                 // tiles so far
  while (!stopped(abort) && walk.next(a)) {
    const KvItem& it = walk.it;
    const int32_t* table = a.table + static_cast<int64_t>(a.s.seq[it.i]) * a.table_stride;
    // (slots that no query of the item sees: behind the last one's own, and from the first ones to the first query's window)
    const int last = it.p_last, before = a.window > 0 ? it.p_first - a.window : -1;
    auto page_of = [&](int tile_i) {         // of box lane % boxes of tile tile_i + lane / boxes
      const int i = tile_i + lane / boxes;
      if (i >= it.t1) return -2;
      const int slot = it.span.tile(i) * kKvTile + (lane % boxes) * box_rows;
      if (slot > last || (slot >= a.sinks && slot + box_rows - 1 <= before)) return -2;      // nothing there that counts
      const int page = table[slot >> a.c.page_shift];
      return page >= 0 && page < a.c.n_pages ? page : -1;
    };
    int mine = page_of(it.t0), next = -2;
#pragma unroll 1
    for (int i = it.t0; i < it.t1; ++i, ++t) {
      const int k = (i - it.t0) & (tiles_per_load - 1);
      if (k == 0) {
        if (i > it.t0) mine = next;
        next = page_of(i + tiles_per_load);
      }
      int page = __shfl_sync(0xffffffffu, mine, k * boxes + lane % boxes);
      const bool there = page != -2;
      if (page == -1) {
        if (lane < boxes) record_error(status, PACE_ERR_INVALID_ARG, K_KV_ATTN);
        page = 0;      // (the sequence's results mean nothing then; the copy stays inside the cache)
      }
      const int s = t % ST, v = t % SV;
      constexpr int PLACES = ST + SV;
      static_assert(!JOINT || 2 * ST > PLACES, "a tile's barrier is not used again before the tile that had it is done with");
      bool ok;
      if constexpr (JOINT) {
        ok = 2 * t < PLACES || kv_wait(smem_u32(&ring.empty[2 * t % PLACES]), (2 * t / PLACES - 1) & 1);
        ok = ok && (2 * t + 1 < PLACES || kv_wait(smem_u32(&ring.empty[(2 * t + 1) % PLACES]), ((2 * t + 1) / PLACES - 1) & 1));
      } else {
        ok = t < ST || kv_wait(smem_u32(&ring.empty[s]), (t / ST - 1) & 1);
        if (ring.v_empty != nullptr) ok = ok && (t < SV || kv_wait(smem_u32(&ring.v_empty[v]), (t / SV - 1) & 1));
      }
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) {
        if (lane == 0) stop(abort, status);
        break;
      }
      const int slot0 = it.span.tile(i) * kKvTile;
      const int n_there = __popc(__ballot_sync(0xffffffffu, there && lane < boxes));
      if (lane == 0) mbar_arrive_expect_tx(smem_u32(&ring.full[s]), 2 * n_there * box_rows * D);
      // scale j (K: 0-7, V: 8-15) of the tile: block j % 8, in box (j % 8) * 16 / box_rows
      const int blk = lane & 7;
      const int bpage = __shfl_sync(0xffffffffu, page, blk * kKvBlock >> shift);
      const int row = (slot0 + blk * kKvBlock) & ((1 << a.c.page_shift) - 1);
      if (lane < 16 && bpage >= 0 && slot0 + blk * kKvBlock <= last)
        cp_async4(smem_u32(&ring.scales[s][lane]),
                  (lane < 8 ? a.c.ks : a.c.vs) + bpage * a.c.scale_stride + (static_cast<int64_t>(it.head) << (a.c.page_shift - 4)) + row / kKvBlock);
      cp_async_arrive(smem_u32(&ring.full[s]));
      __syncwarp();
      if (lane < boxes && there) {
        const int y = (it.head << a.c.page_shift) + ((slot0 + lane * box_rows) & ((1 << a.c.page_shift) - 1));
        uint8_t* k_to = ring.k + (JOINT ? 2 * t % PLACES : s) * ring.stride;
        uint8_t* v_to = JOINT ? ring.k + (2 * t + 1) % PLACES * ring.stride : ring.v + v * ring.stride;
        tma_load_3d(smem_u32(k_to + lane * box_rows * D), &maps.k, 0, y, page, smem_u32(&ring.full[s]));
        tma_load_3d(smem_u32(v_to + lane * box_rows * D), &maps.v, 0, y, page, smem_u32(&ring.full[s]));
      }
    }
  }
}

// Launches of the two forms (rows of a tile: 8, 16 or 32, and kManyRows; nodes of trees where a.family is set); `grid` CTAs, then the
// combine kernel.
pace_status_t launch_kv_decode(const KvMaps& maps, const KvAttnArgs& a, int D, int rows, unsigned grid, int* status, cudaStream_t stream);
pace_status_t launch_kv_prefill(const KvMaps& maps, const KvAttnArgs& a, int D, unsigned grid, int* status, cudaStream_t stream);
pace_status_t launch_kv_combine(const KvAttnArgs& a, int D, int rows, unsigned grid, int64_t items, cudaStream_t stream);

// Depths and family bits of the nodes of trees (host prefix cu_q), as KvAttnArgs has them.
struct KvTree {
  const int32_t* parents;
  int32_t* depth;
  uint32_t* family;
  int words;
};
pace_status_t launch_kv_tree(const KvTree& t, const int32_t* cu_q, int B, const int32_t* lens, int max_len, int window, int sinks, int* status,
                             cudaStream_t stream);

}  // namespace pace
