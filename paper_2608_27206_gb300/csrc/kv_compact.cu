// Serve: kept tokens of the paged 8-bit cache moved together, in place or to other pages, in several layers at once.
//
// Slot base + i takes the kept token i, from slot base + r_i with r_i >= i.  A block of 16 slots gets a scale of its own: with c the
// codes and s the scales that its tokens come from, s' is the smallest power of two with |c| s <= 448 s' for all of them, and c' is
// c s / s' rounded to e4m3.  s' is at most the largest s, so c' = c wherever the scale stays (most blocks of one source block, and those are
// copied as they are); a token from under a smaller scale loses bits only below 2^-6 of s', as it would have had it been appended there.
//
// What bounds it is HBM: a kept token's codes once in and once out.  A warp takes a head's 16 rows of K or V, 16 bytes per lane and
// load; a block's 16 source rows are looked up (list, page table: a chain of loads) once for all heads and layers.  To other pages the
// written blocks of all sequences form a line, block by block and in it layer by layer, of which every CTA takes an equal
// share, as the lengths and counts on the device have it.  In place, blocks are written in order: what block i overwrites are
// sources of blocks up to i, which have been read, since r_i >= i.  So a warp goes over a sequence's blocks of one head by itself, with the rows of
// the next blocks on their way (reading ahead takes nothing away: only earlier blocks have been written), and needs no other order; where there are
// many blocks a CTA takes sixteen at a time.
//
// Measured, 28 layers of 4 heads of 128: 4260 of 10589 tokens to other pages 44.5 us, 5.5 TB/s (a plain copy of as many bytes 41; 64 when
// every block had its CTA, 56 with as many instructions for the largest code and the ratio as that took: 600 of a warp per block and head, 460
// now, of which one in two issue slots is used), in place 75 us; the accepted tokens of 64 trees of 26 14 us, in place 13, which is
// latency (in place, trees of 50 nodes and more: 137, as the kernel goes by the room of their lists).
#include <cuda_fp16.h>

#include <algorithm>

#include "pace_kv.cuh"
#include "pace_ptx.cuh"

namespace pace {
namespace {

constexpr int kMoveThreads = 256, kMoveCtas = 4;      // to other pages: threads of a CTA, CTAs of an SM
constexpr int kSlideThreads = 128;                    // in place, a warp per head's K or V
constexpr int kSlideBlocks = 4;                       // ... with so many blocks of a sequence at most
constexpr int kWideWarps = 16;                        // in place, a CTA per head's K or V
constexpr int kMaxLayers = 64;                        // of one launch

struct CompactArgs {
  uint8_t* codes[2][kMaxLayers];      // K and V of each layer
  float* scales[2][kMaxLayers];
  int64_t page_stride, scale_stride, src_stride, dst_stride;
  int n_pages, page_shift, heads, layers;
  FastDiv by_tasks;                   // 2 heads
  const int32_t* lens;
  const int32_t* src_table;
  const int32_t* dst_table;
  const int32_t* rows;
  const int32_t* counts;
  int32_t* new_lens;                  // null: another launch writes them
  int b0, nb;
  int cu[kKvMaxB + 1];                // newest tokens of each sequence
  int cu_rows[kKvMaxB + 1];           // its list
};

// Where a sequence's newest tokens begin, and how many of them are kept; -1: what its numbers say cannot be.
struct Kept {
  int base, count;
};
__device__ __forceinline__ Kept kept_of(const CompactArgs& a, int b) {
  const int len = a.lens[a.b0 + b], n = a.cu[b + 1] - a.cu[b], room = a.cu_rows[b + 1] - a.cu_rows[b];
  const int count = a.counts != nullptr ? a.counts[a.b0 + b] : room;
  return len < n || count < 0 || count > room ? Kept{len, -1} : Kept{len - n, count};
}
// Its new length, which one thread of the launch writes.
__device__ __forceinline__ void put_length(const CompactArgs& a, int b, const Kept& k, int* status) {
  if (k.count < 0) record_error(status, PACE_ERR_INVALID_ARG, K_KV_COMPACT);
  if (a.new_lens != nullptr) a.new_lens[a.b0 + b] = k.base + max(k.count, 0);
}

// Where slot `slot` of a sequence gets its token from: places of its codes and scale in head 0; code -1: zeros, -2: nothing goes there.
struct alignas(16) Source {
  int64_t code, scale;
};
__device__ __forceinline__ Source place_of(const CompactArgs& a, int page, int64_t slot, int D) {
  const int at = static_cast<int>(slot) & ((1 << a.page_shift) - 1);
  return Source{page * a.page_stride + at * D, page * a.scale_stride + at / kKvBlock};
}
__device__ __forceinline__ Source source_of(const CompactArgs& a, int b, const Kept& k, int64_t slot, int dst_page, int D, int* status) {
  const int64_t i = slot - k.base;      // which of the kept tokens
  if (i < 0) return dst_page < 0 ? Source{-1, 0} : place_of(a, dst_page, slot, D);      // there already
  if (i >= k.count) return Source{-2, 0};
  int64_t row = i;
  bool ok = true;
  if (a.rows != nullptr) {
    const int32_t* list = a.rows + a.cu_rows[b];
    const int mine = list[i], before = i > 0 ? list[i - 1] : -1;
    row = static_cast<int64_t>(mine) - a.cu[b];
    ok = row >= i && row < a.cu[b + 1] - a.cu[b] && mine > before;
  }
  const int64_t s = k.base + row, pi = s >> a.page_shift;
  const int page = ok && pi < a.src_stride ? a.src_table[(a.b0 + b) * a.src_stride + pi] : -1;
  if (page >= 0 && page < a.n_pages) return place_of(a, page, s, D);
  record_error(status, PACE_ERR_INVALID_ARG, K_KV_COMPACT);
  return Source{-1, 0};
}
// The page that a block goes to; -1: none.
__device__ __forceinline__ int target_of(const CompactArgs& a, int b, int64_t block, int* status, bool say) {
  const int64_t pi = block * kKvBlock >> a.page_shift;
  const int page = pi < a.dst_stride ? a.dst_table[(a.b0 + b) * a.dst_stride + pi] : -1;
  if (page >= 0 && page < a.n_pages) return page;
  if (say) record_error(status, PACE_ERR_INVALID_ARG, K_KV_COMPACT);
  return -1;
}

// Codes times a ratio, rounded again.
__device__ __forceinline__ uint32_t times(uint32_t u, float ratio) {
  const uint32_t f0 = e4m3x2_to_f16x2(u & 0xFFFFu), f1 = e4m3x2_to_f16x2(u >> 16);
  const float2 g0 = __half22float2(*reinterpret_cast<const __half2*>(&f0)), g1 = __half22float2(*reinterpret_cast<const __half2*>(&f1));
  return e4m3x4(g0.x * ratio, g0.y * ratio, g1.x * ratio, g1.y * ratio);
}
// The same for 2^e, -24 <= e <= 18, in f16, which holds every product of a code down to its last bit at 2^-24, 2^-14 of half a step of
// the smallest codes: what is lost below decides nothing.
__device__ __forceinline__ uint4 times_pow2(uint4 u, int e) {
  const int e0 = min(max(e, -14), 15), e1 = e - e0;      // (f16 has no larger powers, and no smaller ones without its shift)
  const uint32_t f = static_cast<uint32_t>(15 + e0) * 0x04000400u;
  auto two = [&](uint32_t codes) {
    uint32_t x = e4m3x2_to_f16x2(codes);
    uint16_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(x) : "r"(x), "r"(f));
    if (e1 != 0) asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(x) : "r"(x), "r"(static_cast<uint32_t>(15 + e1) * 0x04000400u));
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(x));
    return static_cast<uint32_t>(r);
  };
  auto four = [&](uint32_t codes) { return two(codes & 0xFFFFu) | two(codes >> 16) << 16; };
  return make_uint4(four(u.x), four(u.y), four(u.z), four(u.w));
}

// The largest magnitude of sixteen codes: of their low seven bits, 0x7F a NaN.  (Sixteen bits at a time the upper byte decides; the
// lower bytes go by themselves.)
__device__ __forceinline__ uint32_t largest(const uint4& x) {
  const uint32_t up = __vmaxu2(__vimax3_u16x2(x.x & 0x7F7F7F7Fu, x.y & 0x7F7F7F7Fu, x.z & 0x7F7F7F7Fu), x.w & 0x7F7F7F7Fu);
  const uint32_t lo = __vmaxu2(__vimax3_u16x2(x.x & 0x007F007Fu, x.y & 0x007F007Fu, x.z & 0x007F007Fu), x.w & 0x007F007Fu);
  const uint32_t m = __vmaxu2(up >> 8 & 0x007F007Fu, lo);
  return max(m & 0xFFFFu, m >> 16);
}

// A block's rows of one head, K or V, as a warp holds them: 16 codes of PASS rows in a lane, and their scales.
template <int D>
struct Rows {
  static constexpr int LPR = D / 16, RPP = 32 / LPR, PASS = kKvBlock / RPP;      // lanes per row, rows per pass
  uint4 x[PASS];
  float s[PASS];
};
struct HeadOf {      // of a layer
  uint8_t* codes;
  float* scales;
  int head;
};
__device__ __forceinline__ HeadOf head_of(const CompactArgs& a, int layer, int task) {
  const bool is_v = task >= a.heads;
  return HeadOf{a.codes[is_v][layer], a.scales[is_v][layer], is_v ? task - a.heads : task};
}

template <int D>
__device__ __forceinline__ void get_rows(const CompactArgs& a, const HeadOf& h, const Source* from, Rows<D>& r) {
  using R = Rows<D>;
  const int lane = threadIdx.x & 31, col = lane % R::LPR * 16, row0 = lane / R::LPR;
  const uint8_t* codes = h.codes + (static_cast<int64_t>(h.head) << a.page_shift) * D + col;
  const float* scales = h.scales + (static_cast<int64_t>(h.head) << (a.page_shift - 4));
#pragma unroll
  for (int p = 0; p < R::PASS; ++p) {
    const Source f = from[p * R::RPP + row0];
    r.x[p] = make_uint4(0, 0, 0, 0);
    r.s[p] = 1.f;
    if (f.code >= 0) {
      r.x[p] = *reinterpret_cast<const uint4*>(codes + f.code);
      r.s[p] = scales[f.scale];
    }
  }
}

// ... to the slots of a page that begin at `to_place` (in head 0), `n` of them, under their scale.
template <int D>
__device__ __forceinline__ void put_rows(const CompactArgs& a, const HeadOf& h, Rows<D>& r, const Source& to_place, int n, int* status) {
  using R = Rows<D>;
  const int lane = threadIdx.x & 31, col = lane % R::LPR * 16, row0 = lane / R::LPR;
  float amax = 0.f;
  auto bad_scale = [](float x) { return !(x > 0.f && x < INFINITY); };
  auto value = [](uint32_t m) {
    const uint32_t f = e4m3x2_to_f16x2(m);
    return __low2float(*reinterpret_cast<const __half2*>(&f));
  };
  bool bad = false;
#pragma unroll
  for (int p = 0; p < R::PASS; ++p) {
    const uint32_t m = largest(r.x[p]);
    bad = bad || m == 0x7Fu || bad_scale(r.s[p]);
    amax = fmaxf(amax, value(m) * r.s[p]);
  }
  if (__any_sync(0xffffffffu, bad)) {      // rows (of LPR lanes) with a NaN or a scale that is none become zeros
    if (bad) record_error(status, PACE_ERR_INVALID_ARG, K_KV_COMPACT);
    amax = 0.f;
#pragma unroll
    for (int p = 0; p < R::PASS; ++p) {
      uint32_t m = bad_scale(r.s[p]) ? 0x7Fu : largest(r.x[p]);
#pragma unroll
      for (int o = 1; o < R::LPR; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
      if (m == 0x7Fu) {
        r.x[p] = make_uint4(0, 0, 0, 0);
        r.s[p] = 1.f;
        m = 0;
      }
      amax = fmaxf(amax, value(m) * r.s[p]);
    }
  }
  amax = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(amax)));      // (none is negative; the lanes have their rows and scales)
  const float to = scale_for(amax);
  uint8_t* codes = h.codes + to_place.code + (static_cast<int64_t>(h.head) << a.page_shift) * D + col;
#pragma unroll
  for (int p = 0; p < R::PASS; ++p) {
    const int at = p * R::RPP + row0;
    uint4 x = r.x[p];
    const uint32_t was = __float_as_uint(r.s[p]), now = __float_as_uint(to);
    if (was != now) {
      if ((was & 0x7FFFFFu) == 0) {      // (above 2^18 every code is 0, as none passes 448; from 2^-24 on nothing is left of any)
        x = times_pow2(x, min(max(static_cast<int>(was >> 23) - static_cast<int>(now >> 23), -24), 18));
      } else {      // (a scale that this library has not made, or below 2^-126)
        const float ratio = __fdiv_rn(r.s[p], to);
        x = make_uint4(times(x.x, ratio), times(x.y, ratio), times(x.z, ratio), times(x.w, ratio));
      }
    }
    if (at < n) *reinterpret_cast<uint4*>(codes + at * D) = x;
  }
  if (lane == 0) h.scales[to_place.scale + (static_cast<int64_t>(h.head) << (a.page_shift - 4))] = to;
}

// Of a block's slots those that hold a token when it is written.
__device__ __forceinline__ int slots_of(const Kept& k, int64_t block) {
  return static_cast<int>(min(static_cast<int64_t>(k.base) + k.count - block * kKvBlock, static_cast<int64_t>(kKvBlock)));
}

// To other pages.
template <int D>
__global__ void __launch_bounds__(kMoveThreads, kMoveCtas) kv_move_kernel(const __grid_constant__ CompactArgs a, int* status) {
  static_assert(kMoveThreads >= kKvMaxB, "a thread per sequence");
  __shared__ int s_base[kKvMaxB], s_count[kKvMaxB], s_end[kKvMaxB], s_warp[kMoveThreads / 32], s_page;
  __shared__ Source s_from[kKvBlock];
  ptx::begin_call();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, warps = kMoveThreads / 32;
  {      // the line: blocks up to each sequence's end
    int blocks = 0;
    if (tid < a.nb) {
      const Kept k = kept_of(a, tid);
      if (blockIdx.x == 0) put_length(a, tid, k, status);
      s_base[tid] = k.base;
      s_count[tid] = k.count;
      if (k.count > 0) blocks = (k.base + k.count - 1) / kKvBlock - k.base / kKvBlock + 1;
    }
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, blocks, o);
      if (lane >= o) blocks += x;
    }
    if (lane == 31) s_warp[warp] = blocks;
    __syncthreads();
    for (int w = 0; w < warp; ++w) blocks += s_warp[w];
    if (tid < a.nb) s_end[tid] = blocks;
    __syncthreads();
  }
  const int64_t total = static_cast<int64_t>(s_end[a.nb - 1]) * a.layers;
  int64_t u = total * blockIdx.x / gridDim.x;
  const int64_t end = total * (blockIdx.x + 1) / gridDim.x;
#pragma unroll 1
  while (u < end) {
    const int at = static_cast<int>(u / a.layers), from_layer = static_cast<int>(u - static_cast<int64_t>(at) * a.layers);
    const int n_layers = static_cast<int>(min(static_cast<int64_t>(a.layers - from_layer), end - u));
    int b = 0, hi = a.nb - 1;      // the first sequence whose end is past it
    while (b < hi) {
      const int mid = (b + hi) >> 1;
      if (s_end[mid] > at) hi = mid;
      else b = mid + 1;
    }
    const Kept k{s_base[b], s_count[b]};
    const int64_t block = k.base / kKvBlock + at - (b > 0 ? s_end[b - 1] : 0);
    if (tid < kKvBlock) {
      const int page = target_of(a, b, block, status, tid == 0);
      s_from[tid] = source_of(a, b, k, block * kKvBlock + tid, page, D, status);
      if (tid == 0) s_page = page;
    }
    __syncthreads();
    const Source to = place_of(a, max(s_page, 0), block * kKvBlock, D);
    const int tasks = s_page >= 0 ? n_layers * 2 * a.heads : 0, n = slots_of(k, block);
#pragma unroll 1
    for (int t = warp; t < tasks; t += warps) {
      const int l = static_cast<int>(a.by_tasks(t));
      const HeadOf h = head_of(a, from_layer + l, t - l * 2 * a.heads);
      Rows<D> r;
      get_rows<D>(a, h, s_from, r);
      put_rows<D>(a, h, r, to, n, status);
    }
    __syncthreads();      // (the rows' sources have been used)
    u += n_layers;
  }
}

// In place, kSlideBlocks blocks of a sequence at most (the call's lists have room for no more): a warp per head's K or V.
template <int D>
__global__ void __launch_bounds__(kSlideThreads) kv_slide_kernel(const __grid_constant__ CompactArgs a, int* status) {
  constexpr int WARPS = kSlideThreads / 32;
  __shared__ Source s_from[kSlideBlocks][kKvBlock];
  __shared__ int s_page[kSlideBlocks];
  ptx::begin_call();
  const int b = blockIdx.x, tid = threadIdx.x;
  const Kept k = kept_of(a, b);
  if (blockIdx.y == 0 && tid == 0) put_length(a, b, k, status);
  if (k.count <= 0) return;
  const int64_t first = k.base / kKvBlock, last = (static_cast<int64_t>(k.base) + k.count - 1) / kKvBlock;
  const int n = static_cast<int>(last - first) + 1;
  for (int i = tid; i < n * kKvBlock; i += kSlideThreads) {
    const int64_t block = first + i / kKvBlock;
    const int page = target_of(a, b, block, status, i % kKvBlock == 0);
    s_from[i / kKvBlock][i % kKvBlock] = source_of(a, b, k, first * kKvBlock + i, page, D, status);
    if (i % kKvBlock == 0) s_page[i / kKvBlock] = page;
  }
  __syncthreads();
  const int task = blockIdx.y * WARPS + (tid >> 5), layer = static_cast<int>(a.by_tasks(task));
  if (layer >= a.layers) return;
  const HeadOf h = head_of(a, layer, task - layer * 2 * a.heads);
  Rows<D> r[2];
  get_rows<D>(a, h, s_from[0], r[0]);
#pragma unroll
  for (int j = 0; j < kSlideBlocks; ++j) {
    if (j >= n) break;
    if (j + 1 < n) get_rows<D>(a, h, s_from[j + 1], r[(j + 1) & 1]);
    if (s_page[j] >= 0) put_rows<D>(a, h, r[j & 1], place_of(a, s_page[j], (first + j) * kKvBlock, D), slots_of(k, first + j), status);
  }
}

// In place, many blocks: a CTA per head's K or V, a warp per block of a round of kWideWarps.  All read a round's rows before one
// writes them, and the next round's before they write: what a round overwrites are sources of rounds up to it.
template <int D, int CTAS>
__global__ void __launch_bounds__(32 * kWideWarps, CTAS) kv_slide_wide_kernel(const __grid_constant__ CompactArgs a, int* status) {
  __shared__ Source s_from[3][kWideWarps][kKvBlock];
  __shared__ int s_page[3][kWideWarps];
  ptx::begin_call();
  const int b = blockIdx.x, tid = threadIdx.x, warp = tid >> 5;
  const Kept k = kept_of(a, b);
  if (blockIdx.y == 0 && tid == 0) put_length(a, b, k, status);
  if (k.count <= 0) return;
  const int layer = static_cast<int>(a.by_tasks(blockIdx.y));
  const HeadOf h = head_of(a, layer, static_cast<int>(blockIdx.y) - layer * 2 * a.heads);
  const int64_t first = k.base / kKvBlock, last = (static_cast<int64_t>(k.base) + k.count - 1) / kKvBlock;
  const int rounds = static_cast<int>((last - first) / kWideWarps) + 1;
  auto look_up = [&](int round) {      // (three rounds' places: one is written, the next one's rows are fetched, and the one after is looked up)
    if (round >= rounds || tid >= kWideWarps * kKvBlock) return;
    const int64_t block = first + static_cast<int64_t>(round) * kWideWarps + tid / kKvBlock;
    if (block > last) return;
    const int page = target_of(a, b, block, status, tid % kKvBlock == 0);
    s_from[round % 3][tid / kKvBlock][tid % kKvBlock] = source_of(a, b, k, block * kKvBlock + tid % kKvBlock, page, D, status);
    if (tid % kKvBlock == 0) s_page[round % 3][tid / kKvBlock] = page;
  };
  auto block_of = [&](int round) { return first + static_cast<int64_t>(round) * kWideWarps + warp; };
  Rows<D> r, next;
  look_up(0);
  look_up(1);
  __syncthreads();
  if (block_of(0) <= last) get_rows<D>(a, h, s_from[0][warp], next);
#pragma unroll 1
  for (int round = 0; round < rounds; ++round) {
    r = next;
    __syncthreads();      // every warp has this round's rows, and the next one's places are known
    if (round + 1 < rounds && block_of(round + 1) <= last) get_rows<D>(a, h, s_from[(round + 1) % 3][warp], next);
    look_up(round + 2);
    const int64_t block = block_of(round);
    const int page = block <= last ? s_page[round % 3][warp] : -1;
    if (page >= 0) put_rows<D>(a, h, r, place_of(a, page, block * kKvBlock, D), slots_of(k, block), status);
  }
}

}  // namespace
}  // namespace pace

using namespace pace;

extern "C" pace_status_t pace_kv_compact(const pace_kv_cache* layers, int n_layers, const int32_t* cu_new, int B, const int32_t* seq_lens,
                                         const int32_t* block_table, int64_t table_stride, const int32_t* cu_rows, const int32_t* rows,
                                         const int32_t* counts, const int32_t* dst_table, int64_t dst_stride, int32_t* new_lens,
                                         pace_stream_t stream) {
  if (B < 0 || n_layers < 1) return PACE_ERR_INVALID_ARG;
  if (B == 0) return PACE_OK;
  if (layers == nullptr) return PACE_ERR_INVALID_ARG;
  for (int l = 0; l < n_layers; ++l) {
    PACE_CHECK(check_cache(layers + l));
    const pace_kv_cache &c = layers[l], &f = layers[0];
    if (c.n_pages != f.n_pages || c.page_stride != f.page_stride || c.scale_stride != f.scale_stride || c.page_size != f.page_size ||
        c.n_kv_heads != f.n_kv_heads || c.head_dim != f.head_dim)
      return PACE_ERR_INVALID_ARG;
  }
  PACE_CHECK(check_prefix(cu_new, B));
  if (cu_rows == nullptr) cu_rows = cu_new;
  PACE_CHECK(check_prefix(cu_rows, B));
  for (int b = 0; b < B; ++b)
    if (cu_rows[b + 1] - cu_rows[b] > cu_new[b + 1] - cu_new[b]) return PACE_ERR_INVALID_ARG;
  if (seq_lens == nullptr || block_table == nullptr || table_stride < 1 || table_stride > INT32_MAX || new_lens == nullptr) return PACE_ERR_INVALID_ARG;
  if (dst_table != nullptr && (dst_stride < 1 || dst_stride > INT32_MAX || (dst_table == block_table && dst_stride != table_stride)))
    return PACE_ERR_INVALID_ARG;
  for (const int32_t* p : {seq_lens, block_table, rows, counts, dst_table, static_cast<const int32_t*>(new_lens)})
    if (reinterpret_cast<uintptr_t>(p) % 4 != 0) return PACE_ERR_INVALID_ARG;
  if (overlap(new_lens, B, seq_lens, B) || (counts != nullptr && overlap(new_lens, B, counts, B)) ||
      (rows != nullptr && overlap(new_lens, B, rows, cu_rows[B])) || overlap(new_lens, B, block_table, B * table_stride) ||
      (dst_table != nullptr && overlap(new_lens, B, dst_table, B * dst_stride)))
    return PACE_ERR_INVALID_ARG;
  PACE_CHECK(check_device());
  const bool in_place = dst_table == nullptr || dst_table == block_table;
  CompactArgs a{};
  const KvView v = kv_view(layers);
  a.page_stride = v.page_stride;
  a.scale_stride = v.scale_stride;
  a.n_pages = v.n_pages;
  a.page_shift = v.page_shift;
  a.heads = v.heads;
  a.by_tasks = fast_div(2 * static_cast<uint32_t>(v.heads));
  a.src_stride = table_stride;
  a.dst_stride = in_place ? table_stride : dst_stride;
  a.lens = seq_lens;
  a.src_table = block_table;
  a.dst_table = in_place ? block_table : dst_table;
  a.rows = rows;
  a.counts = counts;
  int* status = device_status_word();
  int sms = 0;
  PACE_CHECK(sm_count(&sms));
  for (int l0 = 0; l0 < n_layers; l0 += kMaxLayers) {
    a.layers = std::min(kMaxLayers, n_layers - l0);
    for (int l = 0; l < a.layers; ++l) {
      const pace_kv_cache& c = layers[l0 + l];
      a.codes[0][l] = static_cast<uint8_t*>(c.k);
      a.codes[1][l] = static_cast<uint8_t*>(c.v);
      a.scales[0][l] = c.k_scale;
      a.scales[1][l] = c.v_scale;
    }
    a.new_lens = l0 == 0 ? new_lens : nullptr;
    for (int b0 = 0; b0 < B; b0 += kKvMaxB) {
      a.b0 = b0;
      a.nb = std::min(kKvMaxB, B - b0);
      for (int i = 0; i <= a.nb; ++i) {
        a.cu[i] = cu_new[b0 + i];
        a.cu_rows[i] = cu_rows[b0 + i];
      }
      if (in_place) {
        // A warp by itself moves a block in a microsecond, a round of a CTA takes little more: few blocks of many sequences go by warps, which
        // waste none, where a list may reach more than kSlideBlocks (wherever in a block its first token lands) by CTAs.
        int most = 0;
        for (int i = 0; i < a.nb; ++i) most = std::max(most, a.cu_rows[i + 1] - a.cu_rows[i]);
        const unsigned tasks = static_cast<unsigned>(a.layers * 2 * a.heads), warps = kSlideThreads / 32, nb = static_cast<unsigned>(a.nb);
        if (most <= (kSlideBlocks - 1) * kKvBlock + 1)
          PACE_CHECK(launch_dependent(layers->head_dim == 128 ? kv_slide_kernel<128> : kv_slide_kernel<64>, dim3(nb, (tasks + warps - 1) / warps),
                                      kSlideThreads, 0, 1, stream, a, status));
        else
          // (28 layers of 4 heads: 75 us with two CTAs to an SM, 88 with one and more registers; 2 layers: 42 and 36)
          PACE_CHECK(launch_dependent(layers->head_dim == 64 ? kv_slide_wide_kernel<64, 2> : nb * static_cast<int64_t>(tasks) > sms ? kv_slide_wide_kernel<128, 2> : kv_slide_wide_kernel<128, 1>,
                                      dim3(nb, tasks), 32 * kWideWarps, 0, 1, stream, a, status));
      } else {
        int64_t blocks = 0;      // at most, wherever in a block a sequence's first token lands
        for (int i = 0; i < a.nb; ++i)
          if (a.cu_rows[i + 1] > a.cu_rows[i]) blocks += (a.cu_rows[i + 1] - a.cu_rows[i] + 2 * (kKvBlock - 1)) / kKvBlock;
        const unsigned grid = static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>(blocks * a.layers, static_cast<int64_t>(sms) * kMoveCtas)));
        PACE_CHECK(launch_dependent(layers->head_dim == 128 ? kv_move_kernel<128> : kv_move_kernel<64>, grid, kMoveThreads, 0, 1, stream, a, status));
      }
    }
  }
  return PACE_OK;
}
