// Serve: kept tokens of the paged 8-bit cache moved together, in place or to other pages, in several layers at once.
//
// Slot base + i takes the kept token i, from slot base + r_i with r_i >= i.  A block of 16 slots gets a scale of its own: with c the
// codes and s the scales that its tokens come from, s' is the smallest power of two with |c| s <= 448 s' for all of them, and c' is
// c s / s' rounded to e4m3.  s' is at most the largest s, so c' = c wherever the scale stays (most blocks of one source block, and those are
// copied as they are); a token from under a smaller scale loses bits only below 2^-6 of s', as it would have had it been appended there.
//
// What bounds it is HBM: a kept token's codes once in and once out.  One CTA per written block and layer finds its 16 source rows once for
// all heads (length, list, page table: a chain of loads that other CTAs of the SM hide); a warp takes a head's 16 rows of K or V, 16 bytes
// per lane and load.  In place, blocks are written in order: what block i overwrites are sources of blocks up to i, which have
// been read, since r_i >= i.  So a CTA goes over a sequence's blocks by itself, a head's K or V always in the same warp, and needs no other order.
#include <cuda_fp16.h>

#include <algorithm>

#include "pace_kv.cuh"
#include "pace_ptx.cuh"

namespace pace {
namespace {

constexpr int kCompactThreads = 256;
constexpr int kMaxLayers = 64;        // of one launch

struct CompactArgs {
  uint8_t* codes[2][kMaxLayers];      // K and V of each layer
  float* scales[2][kMaxLayers];
  int64_t page_stride, scale_stride, src_stride, dst_stride;
  int n_pages, page_shift, heads;
  const int32_t* lens;
  const int32_t* src_table;
  const int32_t* dst_table;
  const int32_t* rows;
  const int32_t* counts;
  int32_t* new_lens;                  // null: another launch writes them
  int b0, nb;
  int cu[kKvMaxB + 1];                // newest tokens of each sequence
  int cu_rows[kKvMaxB + 1];           // its list
  int block_prefix[kKvMaxB + 1];      // blocks that it may write (in place: 1 where it may write any)
};

// Codes times a ratio, rounded again.
__device__ __forceinline__ uint32_t times(uint32_t u, float ratio) {
  const uint32_t f0 = e4m3x2_to_f16x2(u & 0xFFFFu), f1 = e4m3x2_to_f16x2(u >> 16);
  const float2 g0 = __half22float2(*reinterpret_cast<const __half2*>(&f0)), g1 = __half22float2(*reinterpret_cast<const __half2*>(&f1));
  return e4m3x4(g0.x * ratio, g0.y * ratio, g1.x * ratio, g1.y * ratio);
}

template <int D, bool IN_PLACE>
__global__ void __launch_bounds__(kCompactThreads) kv_compact_kernel(const __grid_constant__ CompactArgs a, int* status) {
  constexpr int LPR = D / 16, RPP = 32 / LPR, PASS = kKvBlock / RPP;      // lanes per row, rows per pass
  __shared__ int src_page[kKvBlock], src_slot[kKvBlock];      // of each slot of the block; page -1: zeros, -2: nothing there
  ptx::begin_call();
  // the kept tokens of a sequence; -1: what its numbers say cannot be
  auto kept = [&](int b, int64_t len, int n) {
    const int room = a.cu_rows[b + 1] - a.cu_rows[b], count = a.counts != nullptr ? a.counts[a.b0 + b] : room;
    return len < n || count < 0 || count > room ? -1 : count;
  };
  if (a.new_lens != nullptr && blockIdx.x == 0 && blockIdx.y == 0) {
    for (int b = threadIdx.x; b < a.nb; b += kCompactThreads) {
      const int len = a.lens[a.b0 + b], n = a.cu[b + 1] - a.cu[b], count = kept(b, len, n);
      if (count < 0) record_error(status, PACE_ERR_INVALID_ARG, K_KV_COMPACT);
      a.new_lens[a.b0 + b] = count < 0 ? len : len - n + count;
    }
  }
  int lo = 0, hi = a.nb - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.block_prefix[mid] <= static_cast<int>(blockIdx.x)) lo = mid;
    else hi = mid - 1;
  }
  const int b = lo, n = a.cu[b + 1] - a.cu[b];
  if (static_cast<int>(blockIdx.x) >= a.block_prefix[a.nb]) return;      // (a launch for the lengths alone)
  // (a length may be anything: slots in 64 bits until they are known to be in the table)
  const int64_t len = a.lens[a.b0 + b], base = len - n;
  const int count = kept(b, len, n);
  if (count <= 0) return;
  const int64_t first = base / kKvBlock, last = (base + count - 1) / kKvBlock;
  const int64_t begin = IN_PLACE ? first : first + (blockIdx.x - a.block_prefix[b]), end = IN_PLACE ? last : min(begin, last);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = kCompactThreads / 32, layer = blockIdx.y;
  const int col = (lane % LPR) * 16, row0 = lane / LPR, blocks = 1 << (a.page_shift - 4), page_slots = 1 << a.page_shift;
#pragma unroll 1
  for (int64_t block = begin; block <= end; ++block) {
    const int64_t slot0 = block * kKvBlock, pi = slot0 >> a.page_shift;
    const int slot = static_cast<int>(slot0) & (page_slots - 1);      // of row 0, in its page
    int page = pi < a.dst_stride ? a.dst_table[(a.b0 + b) * a.dst_stride + pi] : -1;
    if (page < 0 || page >= a.n_pages) {
      if (threadIdx.x == 0) record_error(status, PACE_ERR_INVALID_ARG, K_KV_COMPACT);
      page = -1;
    }
    if (threadIdx.x < kKvBlock) {
      const int r = threadIdx.x;
      const int64_t i = slot0 + r - base;      // which of the kept tokens
      int from = -2, at = slot + r;
      if (i < 0) {
        from = page;      // there already
      } else if (i < count) {
        int64_t row = i;
        bool ok = true;
        if (a.rows != nullptr) {
          const int32_t* list = a.rows + a.cu_rows[b];
          row = static_cast<int64_t>(list[i]) - a.cu[b];
          ok = row >= i && row < n && (i == 0 || list[i] > list[i - 1]);
        }
        const int64_t s = base + row, sp = s >> a.page_shift;
        at = static_cast<int>(s) & (page_slots - 1);
        from = ok && sp < a.src_stride ? a.src_table[(a.b0 + b) * a.src_stride + sp] : -1;
        if (from < 0 || from >= a.n_pages) {
          record_error(status, PACE_ERR_INVALID_ARG, K_KV_COMPACT);
          from = -1;
        }
      }
      src_page[r] = from;
      src_slot[r] = at;
    }
    __syncthreads();
    if (page >= 0) {
#pragma unroll 1
      for (int task = warp; task < 2 * a.heads; task += warps) {
        const bool is_v = task >= a.heads;
        const int head = is_v ? task - a.heads : task;
        uint8_t* codes = a.codes[is_v][layer];
        float* scales = a.scales[is_v][layer];
        uint4 x[PASS];
        float s[PASS];
#pragma unroll
        for (int p = 0; p < PASS; ++p) {
          const int r = p * RPP + row0, from = src_page[r], at = src_slot[r];
          x[p] = make_uint4(0, 0, 0, 0);
          s[p] = 1.f;
          if (from >= 0) {
            x[p] = *reinterpret_cast<const uint4*>(codes + from * a.page_stride + ((static_cast<int64_t>(head) << a.page_shift) + at) * D + col);
            s[p] = scales[from * a.scale_stride + head * blocks + at / kKvBlock];
          }
        }
        float amax = 0.f;
        bool bad = false;
#pragma unroll
        for (int p = 0; p < PASS; ++p) {
          // the largest magnitude of sixteen codes is the largest of their low seven bits, 0x7F a NaN
          uint32_t m = __vmaxu4(__vmaxu4(x[p].x & 0x7F7F7F7Fu, x[p].y & 0x7F7F7F7Fu), __vmaxu4(x[p].z & 0x7F7F7F7Fu, x[p].w & 0x7F7F7F7Fu));
          m = __vmaxu4(m, m >> 16);
          m = max(m & 0xFFu, m >> 8 & 0xFFu);
#pragma unroll
          for (int o = 1; o < LPR; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
          if (m == 0x7Fu || !(s[p] > 0.f && s[p] < INFINITY)) {      // the whole row (its LPR lanes)
            bad = true;
            x[p] = make_uint4(0, 0, 0, 0);
            m = 0;
            s[p] = 1.f;
          }
          const uint32_t f = e4m3x2_to_f16x2(m);
          amax = fmaxf(amax, __low2float(*reinterpret_cast<const __half2*>(&f)) * s[p]);
        }
#pragma unroll
        for (int o = LPR; o < 32; o <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
        if (bad) record_error(status, PACE_ERR_INVALID_ARG, K_KV_COMPACT);
        const float to = scale_for(amax);
        __syncwarp();      // every lane has its rows and their scales: in place they may go
#pragma unroll
        for (int p = 0; p < PASS; ++p) {
          const int r = p * RPP + row0;
          if (src_page[r] == -2) continue;
          if (s[p] != to) {
            const float ratio = __fdiv_rn(s[p], to);
            x[p] = make_uint4(times(x[p].x, ratio), times(x[p].y, ratio), times(x[p].z, ratio), times(x[p].w, ratio));
          }
          *reinterpret_cast<uint4*>(codes + page * a.page_stride + ((static_cast<int64_t>(head) << a.page_shift) + slot + r) * D + col) = x[p];
        }
        if (lane == 0) scales[page * a.scale_stride + head * blocks + slot / kKvBlock] = to;
      }
    }
    if (IN_PLACE) __syncthreads();      // (the rows' sources have been used)
  }
}

// Whether [p, p + np) and [q, q + nq), in int32, have a part in common.
bool overlap(const int32_t* p, int64_t np, const int32_t* q, int64_t nq) {
  const auto a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return np > 0 && nq > 0 && a < b + 4 * static_cast<uintptr_t>(nq) && b < a + 4 * static_cast<uintptr_t>(np);
}

}  // namespace
}  // namespace pace

using namespace pace;

extern "C" pace_status_t pace_kv_compact(const pace_kv_cache* layers, int n_layers, const int32_t* cu_new, int B, const int32_t* seq_lens,
                                         const int32_t* block_table, int64_t table_stride, const int32_t* cu_rows, const int32_t* rows,
                                         const int32_t* counts, const int32_t* dst_table, int64_t dst_stride, int32_t* new_lens,
                                         pace_stream_t stream) {
  if (B < 0 || n_layers < 0) return PACE_ERR_INVALID_ARG;
  if (B == 0 || n_layers == 0) return PACE_OK;
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
  a.src_stride = table_stride;
  a.dst_stride = in_place ? table_stride : dst_stride;
  a.lens = seq_lens;
  a.src_table = block_table;
  a.dst_table = in_place ? block_table : dst_table;
  a.rows = rows;
  a.counts = counts;
  int* status = device_status_word();
  for (int l0 = 0; l0 < n_layers; l0 += kMaxLayers) {
    const int nl = std::min(kMaxLayers, n_layers - l0);
    for (int l = 0; l < nl; ++l) {
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
      int64_t blocks = 0;
      for (int i = 0; i <= a.nb; ++i) {
        a.cu[i] = cu_new[b0 + i];
        a.cu_rows[i] = cu_rows[b0 + i];
        a.block_prefix[i] = static_cast<int>(blocks);
        if (i == a.nb) break;
        const int most = cu_rows[b0 + i + 1] - cu_rows[b0 + i];
        if (most > 0) blocks += in_place ? 1 : (most + 2 * (kKvBlock - 1)) / kKvBlock;      // wherever in a block the first one lands
      }
      if (blocks == 0 && l0 > 0) continue;
      auto* kernel = layers->head_dim == 128 ? (in_place ? kv_compact_kernel<128, true> : kv_compact_kernel<128, false>)
                                             : (in_place ? kv_compact_kernel<64, true> : kv_compact_kernel<64, false>);
      PACE_CHECK(launch_dependent(kernel, dim3(static_cast<unsigned>(std::max<int64_t>(blocks, 1)), static_cast<unsigned>(nl)), kCompactThreads, 0, 1,
                                  stream, a, status));
    }
  }
  return PACE_OK;
}
