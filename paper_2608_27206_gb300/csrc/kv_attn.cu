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

// Sequences of at most so many query rows per KV head take the transposed products of kv_decode.cu, trees up to kFewNodes of them: with 17
// to 32 the two halves of a CTA of kv_prefill.cu are faster (64 trees of 28 rows on 5001-28007 slots 211 us against 424, 8 on
// 700-9000 25 against 36), below they are not (8 of 14 rows 22 us against 30 then).
constexpr int kFewRows = 32, kFewNodes = 16;
// Trees of few rows go with the others in one launch where that gives the others this many slot tiles more at most, were all of them as
// long as max_len: a launch of their own and its join cost 14 to 20 us, of a long row tile of one to eight rows a slot tile 0.3 us more of a CTA than
// there (64 single nodes on 5001-28007 slots 150 us, 21 rows each 208).  Mean of 699 ragged batches of both kinds 27.3 us with 16 for 64 here,
// 25.4 with 48, 24.8 without a limit.
constexpr int kAlong = 64 * kPlanCtas;

// Rows of a tile for few-row sequences: 8, 16 or 32, what the largest needs (0: there are none).
int few_rows(const int32_t* cu_q, int B, int group, int limit) {
  int most = 0;
  for (int b = 0; b < B; ++b) {
    const int64_t rows = static_cast<int64_t>(cu_q[b + 1] - cu_q[b]) * group;
    if (rows <= limit) most = std::max(most, static_cast<int>(rows));
  }
  return most == 0 ? 0 : most <= 8 ? 8 : most <= 16 ? 16 : 32;
}

// Rows of the call's largest tile.
int most_rows(const int32_t* cu_q, int B, int group, int limit) {
  for (int b = 0; b < B; ++b)
    if (static_cast<int64_t>(cu_q[b + 1] - cu_q[b]) * group > limit) return kManyRows;
  return few_rows(cu_q, B, group, limit);
}

int64_t slot_tiles(int max_len) { return std::max(1, (max_len + kKvTile - 1) / kKvTile); }

// Most rows of the sequences that kv_decode.cu takes in a call.
int few_limit(const int32_t* cu_q, int B, int group, int heads, int max_len, bool tree) {
  if (!tree) return kFewRows;
  int64_t few = 0, many = 0;
  for (int b = 0; b < B; ++b) {
    const int64_t rows = static_cast<int64_t>(cu_q[b + 1] - cu_q[b]) * group;
    few += rows > 0 && rows <= kFewNodes;
    many += rows > kFewNodes;
  }
  return many > 0 && few * heads * slot_tiles(max_len) <= kAlong ? 0 : kFewNodes;
}

// The sequences of a form that the next launch takes, from b on (b: the first that it leaves); its row tiles.
int64_t next_launch(const int32_t* cu_q, int B, int group, int limit, bool is_few, int rows, int& b, KvSeqs* s) {
  int64_t tiles = 0;
  int nb = 0;
  for (; b < B && nb < kKvMaxB; ++b) {
    const int n = cu_q[b + 1] - cu_q[b];
    const int64_t r = static_cast<int64_t>(n) * group;
    if (n == 0 || (r <= limit) != is_few) continue;
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
pace_status_t check_attention(const pace_kv_cache* cache, const int32_t* cu_q, int B, int n_q_heads, int max_len, bool tree) {
  PACE_CHECK(check_cache(cache));
  PACE_CHECK(check_prefix(cu_q, B));
  if (n_q_heads < 1 || n_q_heads % cache->n_kv_heads != 0 || n_q_heads / cache->n_kv_heads > kKvMaxGroup) return PACE_ERR_INVALID_ARG;
  if (max_len < 0 || max_len > (1 << 30)) return PACE_ERR_INVALID_ARG;
  const int group = n_q_heads / cache->n_kv_heads;
  if (cu_q[B] > (1 << 30) / group) return PACE_ERR_INVALID_ARG;
  const int limit = few_limit(cu_q, B, group, cache->n_kv_heads, max_len, tree);
  const int64_t most = INT32_MAX / (cache->n_kv_heads * (slot_tiles(max_len) + (tree ? kTreeCost : kItemCost)));      // row tiles of a launch
  for (const bool is_few : {true, false})
    for (int b = 0; b < B;)
      if (next_launch(cu_q, B, group, limit, is_few, is_few ? few_rows(cu_q, B, group, limit) : kManyRows, b, nullptr) > most) return PACE_ERR_INVALID_ARG;
  return PACE_OK;
}

struct Workspace {
  size_t lse, part, depth, family, total;
  int words;
};
Workspace workspace(int rows, int D, const int32_t* cu_q, int B, bool tree) {
  Workspace w{};
  w.lse = align_up(kPlanCtas * sizeof(KvSplit), 256);
  w.part = w.lse + align_up(static_cast<size_t>(2) * kPlanCtas * rows * sizeof(float2), 256);
  w.total = w.part + static_cast<size_t>(2) * kPlanCtas * rows * D * sizeof(float);
  if (tree) {
    int most = 1;
    for (int b = 0; b < B; ++b) most = std::max(most, cu_q[b + 1] - cu_q[b]);
    w.words = (most + 62) / 32;      // (wherever in a word the first bit lands)
    w.depth = w.total;
    w.family = w.depth + align_up(static_cast<size_t>(cu_q[B]) * sizeof(int32_t), 256);
    w.total = w.family + static_cast<size_t>(cu_q[B]) * w.words * sizeof(uint32_t);
  }
  return w;
}

// Trees have at most PACE_TREE_MAX nodes.
pace_status_t check_tree(const int32_t* cu_q, int B) {
  for (int b = 0; b < B; ++b)
    if (cu_q[b + 1] - cu_q[b] > PACE_TREE_MAX) return PACE_ERR_INVALID_ARG;
  return PACE_OK;
}

size_t workspace_size(const pace_kv_cache* cache, const int32_t* cu_q, int B, int n_q_heads, int max_len, bool tree) {
  if (B <= 0 || check_attention(cache, cu_q, B, n_q_heads, max_len, tree) != PACE_OK || (tree && check_tree(cu_q, B) != PACE_OK)) return 0;
  const int group = n_q_heads / cache->n_kv_heads, limit = few_limit(cu_q, B, group, cache->n_kv_heads, max_len, tree);
  return workspace(most_rows(cu_q, B, group, limit), cache->head_dim, cu_q, B, tree).total;
}

// Both calls; parents null: the queries follow one another.
pace_status_t attend(const pace_kv_cache* cache, const void* Q, int64_t q_row_stride, const int32_t* cu_q, int B, int n_q_heads,
                     const int32_t* parents, bool tree, const int32_t* seq_lens, const int32_t* block_table, int64_t table_stride, int max_len,
                     float scale, int window, int sinks, void* out, float* lse, void* ws, size_t ws_bytes, cudaStream_t stream) {
  if (B < 0) return PACE_ERR_INVALID_ARG;
  if (B == 0) return PACE_OK;
  PACE_CHECK(check_attention(cache, cu_q, B, n_q_heads, max_len, tree));
  if (tree) PACE_CHECK(check_tree(cu_q, B));
  if (cu_q[B] == 0) return PACE_OK;
  if (tree && (parents == nullptr || reinterpret_cast<uintptr_t>(parents) % 4 != 0)) return PACE_ERR_INVALID_ARG;
  const int D = cache->head_dim, group = n_q_heads / cache->n_kv_heads;
  if (!rows_ok(Q, q_row_stride, n_q_heads, D) || out == nullptr || reinterpret_cast<uintptr_t>(out) % 16 != 0)
    return PACE_ERR_INVALID_ARG;
  if (seq_lens == nullptr || block_table == nullptr || table_stride < 1 || table_stride > INT32_MAX || sinks < 0) return PACE_ERR_INVALID_ARG;
  if (max_len > table_stride * cache->page_size) return PACE_ERR_INVALID_ARG;
  if (!(scale > 0.f) || !std::isfinite(scale)) return PACE_ERR_INVALID_ARG;
  const int limit = few_limit(cu_q, B, group, cache->n_kv_heads, max_len, tree), few = few_rows(cu_q, B, group, limit);
  const Workspace w = workspace(most_rows(cu_q, B, group, limit), D, cu_q, B, tree);
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
  a.sinks = std::min(sinks, max_len);      // (no position reaches max_len; sums with it stay within 32 bits)
  a.max_len = max_len;
  int* status = device_status_word();
  int sms = 0;
  PACE_CHECK(sm_count(&sms));
  if (tree) {
    KvTree t{parents, reinterpret_cast<int32_t*>(static_cast<uint8_t*>(ws) + w.depth), reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(ws) + w.family), w.words};
    PACE_CHECK(launch_kv_tree(t, cu_q, B, seq_lens, max_len, a.window, a.sinks, status, stream));
    a.depth = t.depth;
    a.family = t.family;
    a.words = t.words;
    a.after_tree = 1;
  }
  for (const bool is_few : {true, false}) {
    const int rows = is_few ? few : kManyRows;
    for (int b = 0; b < B;) {
      const int64_t tiles = next_launch(cu_q, B, group, limit, is_few, rows, b, &a.s);
      if (tiles == 0) break;
      const unsigned grid = static_cast<unsigned>(std::min<int64_t>({tiles * cache->n_kv_heads * slot_tiles(max_len), sms, kPlanCtas}));
      if (is_few) PACE_CHECK(launch_kv_decode(maps, a, D, rows, grid, status, stream));
      else PACE_CHECK(launch_kv_prefill(maps, a, D, grid, status, stream));
      a.after_tree = 0;
      if (slot_tiles(max_len) > 1) PACE_CHECK(launch_kv_combine(a, D, rows, grid, tiles * cache->n_kv_heads, stream));
    }
  }
  return PACE_OK;
}

}  // namespace
}  // namespace pace

using namespace pace;

extern "C" size_t pace_kv_attention_workspace_size(const pace_kv_cache* cache, const int32_t* cu_q, int B, int n_q_heads,
                                                   int max_len) {
  return workspace_size(cache, cu_q, B, n_q_heads, max_len, false);
}

extern "C" size_t pace_kv_tree_attention_workspace_size(const pace_kv_cache* cache, const int32_t* cu_q, int B, int n_q_heads,
                                                        int max_len) {
  return workspace_size(cache, cu_q, B, n_q_heads, max_len, true);
}

extern "C" pace_status_t pace_kv_attention(const pace_kv_cache* cache, const void* Q, int64_t q_row_stride, const int32_t* cu_q,
                                           int B, int n_q_heads, const int32_t* seq_lens, const int32_t* block_table,
                                           int64_t table_stride, int max_len, float scale, int window, int sinks, void* out,
                                           float* lse, void* ws, size_t ws_bytes, pace_stream_t stream) {
  return attend(cache, Q, q_row_stride, cu_q, B, n_q_heads, nullptr, false, seq_lens, block_table, table_stride, max_len, scale, window, sinks, out,
                lse, ws, ws_bytes, stream);
}

extern "C" pace_status_t pace_kv_tree_attention(const pace_kv_cache* cache, const void* Q, int64_t q_row_stride, const int32_t* cu_q,
                                                int B, int n_q_heads, const int32_t* parents, const int32_t* seq_lens,
                                                const int32_t* block_table, int64_t table_stride, int max_len, float scale, int window,
                                                int sinks, void* out, float* lse, void* ws, size_t ws_bytes, pace_stream_t stream) {
  return attend(cache, Q, q_row_stride, cu_q, B, n_q_heads, parents, true, seq_lens, block_table, table_stride, max_len, scale, window, sinks, out,
                lse, ws, ws_bytes, stream);
}
