// Serve: causal attention of the newest tokens over the paged 8-bit cache.
//
// out = sum_j softmax_j(scale q . k_j) v_j over the slots that a query sees, in one pass over them:
// with the running maximum m and sum l of the weights so far, a block of 16 slots with scores x_j gives
//   m' = max(m, max_j x_j),  l' = l 2^(m - m') + sum_j 2^(x_j - m'),  o' = o 2^(m - m') + sum_j 2^(x_j - m') v_j
// (scores in base 2, sums in fp32), and out = o / l.
//
// One CTA takes 16 of the query rows that share a KV head (row r = query r / G, head r % G of the
// group) and walks the blocks of slots that any of them sees.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include <cudaTypedefs.h>

#include "kv_attn.cuh"
#include "pace_ptx.cuh"

namespace pace {
namespace {

constexpr int kRows = 16, kAttnThreads = 128;

template <int D>
__global__ void __launch_bounds__(kAttnThreads) kv_attn_rows(const __grid_constant__ KvAttnArgs a, int* status) {
  __shared__ float q[kRows][D + 1], kv[kKvBlock][D + 1], p[kRows][kKvBlock], m[kRows], l[kRows], f[kRows];
  ptx::begin_call();
  int lo = 0, hi = a.s.nb - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.s.tile0[mid] <= static_cast<int>(blockIdx.x)) lo = mid;
    else hi = mid - 1;
  }
  const int b = lo, n = a.s.nq[b], head = blockIdx.y, tid = threadIdx.x;
  const int row0 = (static_cast<int>(blockIdx.x) - a.s.tile0[b]) * kRows, rows = min(n * a.group - row0, kRows);
  int len = max(a.lens[a.s.seq[b]], 0);
  if (len > a.max_len) {
    if (tid == 0) record_error(status, PACE_ERR_INVALID_ARG, K_KV_ATTN);
    len = a.max_len;
  }
  const int p0 = len - n;   // slot of query 0
  auto token = [&](int r) { return a.s.q0[b] + (row0 + r) / a.group; };
  auto qhead = [&](int r) { return head * a.group + (row0 + r) % a.group; };
  for (int i = tid; i < kRows * D; i += kAttnThreads) {
    const int r = i / D, d = i % D;
    q[r][d] = r < rows ? __uint_as_float(static_cast<uint32_t>(a.Q[token(r) * a.q_stride + qhead(r) * D + d]) << 16) : 0.f;
  }
  if (tid < kRows) {
    m[tid] = -INFINITY;
    l[tid] = 0.f;
  }
  float o[D / 8];   // row tid / 8, columns tid % 8 + 8 i
#pragma unroll
  for (int i = 0; i < D / 8; ++i) o[i] = 0.f;
  const int p_first = p0 + row0 / a.group, p_last = p0 + (row0 + rows - 1) / a.group;
  const int from = a.window > 0 ? max(p_first - a.window + 1, 0) / kKvBlock : 0;   // first block of the window
  const int mr = tid / 8;
  for (int blk = 0; blk * kKvBlock <= p_last; ++blk) {
    if (blk < from && blk * kKvBlock >= a.sinks) blk = from;
    const int slot = blk * kKvBlock;
    const int page = a.table[a.s.seq[b] * a.table_stride + (slot >> a.c.page_shift)];
    const bool ok = page >= 0 && page < a.c.n_pages;
    if (!ok && tid == 0) record_error(status, PACE_ERR_INVALID_ARG, K_KV_ATTN);
    const int at = slot & ((1 << a.c.page_shift) - 1);
    const int64_t sc = page * a.c.scale_stride + (static_cast<int64_t>(head) << (a.c.page_shift - 4)) + at / kKvBlock;
    const int64_t co = page * a.c.page_stride + ((static_cast<int64_t>(head) << a.c.page_shift) + at) * D;
    auto fetch = [&](const uint8_t* codes, const float* scales) {
      const float s = ok ? scales[sc] : 0.f;
      for (int i = tid; i < kKvBlock * D / 2; i += kAttnThreads) {
        const int j = 2 * i / D, d = 2 * i % D;
        float2 x = make_float2(0.f, 0.f);
        if (ok && kv_sees(slot + j, p_last, 0, 0) && (a.window <= 0 || slot + j < a.sinks || slot + j > p_first - a.window)) {
          const uint32_t h = e4m3x2_to_f16x2(*reinterpret_cast<const uint16_t*>(codes + co + 2 * i));
          x = __half22float2(*reinterpret_cast<const __half2*>(&h));
          x.x *= s;
          x.y *= s;
        }
        kv[j][d] = x.x;
        kv[j][d + 1] = x.y;
      }
    };
    __syncthreads();
    fetch(a.c.k, a.c.ks);
    __syncthreads();
    for (int i = tid; i < kRows * kKvBlock; i += kAttnThreads) {
      const int r = i / kKvBlock, j = i % kKvBlock;
      float s = 0.f;
      for (int d = 0; d < D; ++d) s = fmaf(q[r][d], kv[j][d], s);
      const bool see = r < rows && kv_sees(slot + j, p0 + (row0 + r) / a.group, a.window, a.sinks);
      p[r][j] = see ? s * a.scale2 : -INFINITY;
    }
    __syncthreads();
    fetch(a.c.v, a.c.vs);
    if (tid < kRows) {
      float mx = m[tid];
      for (int j = 0; j < kKvBlock; ++j) mx = fmaxf(mx, p[tid][j]);
      const float base = mx == -INFINITY ? 0.f : mx;
      const float k = exp2f(m[tid] - base);
      float sum = 0.f;
      for (int j = 0; j < kKvBlock; ++j) {
        const float e = exp2f(p[tid][j] - base);
        p[tid][j] = e;
        sum += e;
      }
      l[tid] = l[tid] * k + sum;
      m[tid] = mx;
      f[tid] = k;
    }
    __syncthreads();
    const float k = f[mr];
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      float s = o[i] * k;
      for (int j = 0; j < kKvBlock; ++j) {
        const float w = p[mr][j];
        if (w != 0.f) s = fmaf(w, kv[j][tid % 8 + 8 * i], s);
      }
      o[i] = s;
    }
  }
  __syncthreads();
  if (mr < rows) {
    const float sum = l[mr], inv = sum != 0.f ? 1.f / sum : 0.f;
    uint16_t* dst = a.out + (static_cast<int64_t>(token(mr)) * a.q_heads + qhead(mr)) * D;
#pragma unroll
    for (int i = 0; i < D / 8; ++i) dst[tid % 8 + 8 * i] = __bfloat16_as_ushort(__float2bfloat16_rn(o[i] * inv));
    if (a.lse != nullptr && tid % 8 == 0)
      a.lse[static_cast<int64_t>(token(mr)) * a.q_heads + qhead(mr)] =
          sum != 0.f ? (m[mr] + log2f(sum)) * 0.69314718055994531f : -INFINITY;
  }
}

// 3-D map over the codes: D bytes x the rows of all heads of a page x pages; a box is 16 to 128 rows of one page.
pace_status_t make_map(CUtensorMap* m, const pace_kv_cache* c, void* codes) {
  auto enc = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(tensor_map_encoder());
  if (enc == nullptr) return set_cuda_error(cudaErrorNotSupported);
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(c->head_dim), static_cast<cuuint64_t>(c->n_kv_heads) * c->page_size,
                              static_cast<cuuint64_t>(c->n_pages)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(c->head_dim), static_cast<cuuint64_t>(c->page_stride)};
  const cuuint32_t box[3] = {static_cast<cuuint32_t>(c->head_dim), static_cast<cuuint32_t>(std::min(c->page_size, kKvTile)), 1};
  const cuuint32_t step[3] = {1, 1, 1};
  const CUresult r = enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, codes, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         c->head_dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                         CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? PACE_OK : PACE_ERR_INVALID_ARG;
}

pace_status_t check_attention(const pace_kv_cache* cache, const int32_t* cu_q, int B, int n_q_heads, int max_len) {
  PACE_CHECK(check_cache(cache));
  PACE_CHECK(check_prefix(cu_q, B));
  if (n_q_heads < 1 || n_q_heads % cache->n_kv_heads != 0 || n_q_heads / cache->n_kv_heads > 64) return PACE_ERR_INVALID_ARG;
  if (max_len < 0 || max_len > (1 << 30)) return PACE_ERR_INVALID_ARG;
  if (cu_q[B] > (1 << 30) / (n_q_heads / cache->n_kv_heads)) return PACE_ERR_INVALID_ARG;
  return PACE_OK;
}

// Sequences of at most kFewRows query rows per KV head take the transposed products of kv_decode.cu.
constexpr int kFewRows = 32;

// Rows of a tile for few-row sequences: 8, 16 or 32, what the largest needs (0: there are none).
int few_rows(const int32_t* cu_q, int B, int group) {
  int most = 0;
  for (int b = 0; b < B; ++b) {
    const int64_t rows = static_cast<int64_t>(cu_q[b + 1] - cu_q[b]) * group;
    if (rows <= kFewRows) most = std::max(most, static_cast<int>(rows));
  }
  return most == 0 ? 0 : most <= 8 ? 8 : most <= 16 ? 16 : 32;
}

struct Workspace {
  size_t lse, part, total;
};
Workspace workspace(int rows, int D) {
  Workspace w{};
  w.lse = align_up(kPlanCtas * sizeof(KvSplit), 256);
  w.part = w.lse + align_up(static_cast<size_t>(2) * kPlanCtas * rows * sizeof(float), 256);
  w.total = w.part + static_cast<size_t>(2) * kPlanCtas * rows * D * sizeof(float);
  return w;
}

}  // namespace
}  // namespace pace

using namespace pace;

extern "C" size_t pace_kv_attention_workspace_size(const pace_kv_cache* cache, const int32_t* cu_q, int B, int n_q_heads,
                                                   int max_len) {
  if (B <= 0 || check_attention(cache, cu_q, B, n_q_heads, max_len) != PACE_OK) return 0;
  return workspace(few_rows(cu_q, B, n_q_heads / cache->n_kv_heads), cache->head_dim).total;
}

extern "C" pace_status_t pace_kv_attention(const pace_kv_cache* cache, const void* Q, int64_t q_row_stride, const int32_t* cu_q,
                                           int B, int n_q_heads, const int32_t* seq_lens, const int32_t* block_table,
                                           int64_t table_stride, int max_len, float scale, int window, int sinks, void* out,
                                           float* lse, void* ws, size_t ws_bytes, pace_stream_t stream) {
  if (B < 0) return PACE_ERR_INVALID_ARG;
  if (B == 0) return PACE_OK;
  PACE_CHECK(check_attention(cache, cu_q, B, n_q_heads, max_len));
  if (cu_q[B] == 0) return PACE_OK;
  const int D = cache->head_dim, group = n_q_heads / cache->n_kv_heads;
  if (!rows_ok(Q, q_row_stride, n_q_heads, D) || out == nullptr || reinterpret_cast<uintptr_t>(out) % 16 != 0)
    return PACE_ERR_INVALID_ARG;
  if (seq_lens == nullptr || block_table == nullptr || table_stride < 1 || table_stride > INT32_MAX || sinks < 0) return PACE_ERR_INVALID_ARG;
  if (max_len > table_stride * cache->page_size) return PACE_ERR_INVALID_ARG;
  if (!(scale > 0.f) || !std::isfinite(scale)) return PACE_ERR_INVALID_ARG;
  const int few = few_rows(cu_q, B, group);
  const Workspace w = workspace(few, D);
  if (ws == nullptr || reinterpret_cast<uintptr_t>(ws) % 16 != 0 || ws_bytes < w.total) return PACE_ERR_WORKSPACE;
  PACE_CHECK(check_device());
  KvMaps maps;
  PACE_CHECK(make_map(&maps.k, cache, cache->k));
  PACE_CHECK(make_map(&maps.v, cache, cache->v));
  KvAttnArgs a{};
  a.c = kv_view(cache);
  a.Q = static_cast<const uint16_t*>(Q);
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.q_stride = q_row_stride;
  a.table_stride = table_stride;
  a.lens = seq_lens;
  a.table = block_table;
  a.split = static_cast<KvSplit*>(ws);
  a.part_lse = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + w.lse);
  a.part = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + w.part);
  a.scale2 = static_cast<float>(static_cast<double>(scale) * 1.4426950408889634);
  a.q_heads = n_q_heads;
  a.group = group;
  a.window = window;
  a.sinks = sinks;
  a.max_len = max_len;
  int* status = device_status_word();
  int sms = 0;
  PACE_CHECK(sm_count(&sms));
  const int64_t slot_tiles = std::max(1, (max_len + kKvTile - 1) / kKvTile);
  for (const bool is_few : {true, false}) {
    const int rows = is_few ? few : kRows;
    for (int b = 0; b < B;) {
      a.s.nb = 0;
      a.s.tile0[0] = 0;
      int64_t tiles = 0;
      for (; b < B && a.s.nb < kKvMaxB; ++b) {
        const int n = cu_q[b + 1] - cu_q[b];
        const int64_t r = static_cast<int64_t>(n) * group;
        if (n == 0 || (r <= kFewRows) != is_few) continue;
        const int i = a.s.nb++;
        a.s.seq[i] = b;
        a.s.q0[i] = cu_q[b];
        a.s.nq[i] = n;
        tiles += (r + rows - 1) / rows;
        a.s.tile0[i + 1] = static_cast<int>(tiles);
      }
      if (a.s.nb == 0) break;
      if (is_few) {
        const int64_t most = tiles * cache->n_kv_heads * slot_tiles;
        const unsigned grid = static_cast<unsigned>(std::min<int64_t>({most, sms, kPlanCtas}));
        PACE_CHECK(launch_kv_decode(maps, a, D, rows, grid, status, stream));
        if (slot_tiles > 1) PACE_CHECK(launch_kv_combine(a, D, rows, grid, stream));
      } else {
        auto* kernel = D == 128 ? kv_attn_rows<128> : kv_attn_rows<64>;
        PACE_CHECK(launch_dependent(kernel, dim3(static_cast<unsigned>(tiles), static_cast<unsigned>(cache->n_kv_heads)), kAttnThreads,
                                    0, 1, stream, a, status));
      }
    }
  }
  return PACE_OK;
}
