// Serve: causal attention of the newest tokens over the paged 8-bit cache: the call, its checks and its plan.
//
// out = sum_j softmax_j(scale q . k_j) v_j over the slots that a query sees, in one pass over them with running maximum and
// sum.  Two forms: sequences of at most 32 query rows per KV head (kv_decode.cu, bound by HBM) and the others (kv_prefill.cu,
// bound by the tensor pipe); a batch of both takes a launch of each.
#include <cudaTypedefs.h>

#include <algorithm>
#include <cmath>

#include "kv_attn.cuh"

namespace pace {
namespace {

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

// Rows of the call's largest tile.
int most_rows(const int32_t* cu_q, int B, int group) {
  for (int b = 0; b < B; ++b)
    if (static_cast<int64_t>(cu_q[b + 1] - cu_q[b]) * group > kFewRows) return kManyRows;
  return few_rows(cu_q, B, group);
}

int64_t slot_tiles(int max_len) { return std::max(1, (max_len + kKvTile - 1) / kKvTile); }

// The sequences of a form that the next launch takes, from b on (b: the first that it leaves); its row tiles.
int64_t next_launch(const int32_t* cu_q, int B, int group, bool is_few, int rows, int& b, KvSeqs* s) {
  int64_t tiles = 0;
  int nb = 0;
  for (; b < B && nb < kKvMaxB; ++b) {
    const int n = cu_q[b + 1] - cu_q[b];
    const int64_t r = static_cast<int64_t>(n) * group;
    if (n == 0 || (r <= kFewRows) != is_few) continue;
    tiles += (r + rows - 1) / rows;
    if (s != nullptr) {
      s->seq[nb] = b;
      s->q0[nb] = cu_q[b];
      s->nq[nb] = n;
      s->tile0[nb + 1] = static_cast<int>(tiles);
    }
    ++nb;
  }
  if (s != nullptr) {
    s->nb = nb;
    s->tile0[0] = 0;
  }
  return tiles;
}

// What the size query and the call refuse alike, and before anything is launched.
pace_status_t check_attention(const pace_kv_cache* cache, const int32_t* cu_q, int B, int n_q_heads, int max_len) {
  PACE_CHECK(check_cache(cache));
  PACE_CHECK(check_prefix(cu_q, B));
  if (n_q_heads < 1 || n_q_heads % cache->n_kv_heads != 0 || n_q_heads / cache->n_kv_heads > kKvMaxGroup) return PACE_ERR_INVALID_ARG;
  if (max_len < 0 || max_len > (1 << 30)) return PACE_ERR_INVALID_ARG;
  const int group = n_q_heads / cache->n_kv_heads;
  if (cu_q[B] > (1 << 30) / group) return PACE_ERR_INVALID_ARG;
  const int64_t most = INT32_MAX / (cache->n_kv_heads * (slot_tiles(max_len) + kItemCost));      // row tiles of a launch
  for (const bool is_few : {true, false})
    for (int b = 0; b < B;)
      if (next_launch(cu_q, B, group, is_few, is_few ? few_rows(cu_q, B, group) : kManyRows, b, nullptr) > most) return PACE_ERR_INVALID_ARG;
  return PACE_OK;
}

struct Workspace {
  size_t lse, part, total;
};
Workspace workspace(int rows, int D) {
  Workspace w{};
  w.lse = align_up(kPlanCtas * sizeof(KvSplit), 256);
  w.part = w.lse + align_up(static_cast<size_t>(2) * kPlanCtas * rows * sizeof(float2), 256);
  w.total = w.part + static_cast<size_t>(2) * kPlanCtas * rows * D * sizeof(float);
  return w;
}

}  // namespace
}  // namespace pace

using namespace pace;

extern "C" size_t pace_kv_attention_workspace_size(const pace_kv_cache* cache, const int32_t* cu_q, int B, int n_q_heads,
                                                   int max_len) {
  if (B <= 0 || check_attention(cache, cu_q, B, n_q_heads, max_len) != PACE_OK) return 0;
  return workspace(most_rows(cu_q, B, n_q_heads / cache->n_kv_heads), cache->head_dim).total;
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
  const Workspace w = workspace(most_rows(cu_q, B, group), D);
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
  a.part_lse = reinterpret_cast<float2*>(static_cast<uint8_t*>(ws) + w.lse);
  a.part = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + w.part);
  a.scale2 = static_cast<float>(static_cast<double>(scale) * 1.4426950408889634);
  a.q_heads = n_q_heads;
  a.group = group;
  a.by_group = fast_div(static_cast<uint32_t>(group));
  a.window = window < max_len ? window : 0;      // (one of max_len leaves nothing out; smaller ones keep slot - window within 32 bits)
  a.sinks = sinks;
  a.max_len = max_len;
  int* status = device_status_word();
  int sms = 0;
  PACE_CHECK(sm_count(&sms));
  for (const bool is_few : {true, false}) {
    const int rows = is_few ? few : kManyRows;
    for (int b = 0; b < B;) {
      const int64_t tiles = next_launch(cu_q, B, group, is_few, rows, b, &a.s);
      if (tiles == 0) break;
      const unsigned grid = static_cast<unsigned>(std::min<int64_t>({tiles * cache->n_kv_heads * slot_tiles(max_len), sms, kPlanCtas}));
      if (is_few) PACE_CHECK(launch_kv_decode(maps, a, D, rows, grid, status, stream));
      else PACE_CHECK(launch_kv_prefill(maps, a, D, grid, status, stream));
      if (slot_tiles(max_len) > 1) PACE_CHECK(launch_kv_combine(a, D, rows, grid, stream));
    }
  }
  return PACE_OK;
}
