// Serve: trees of drafted tokens: who sees whom, and the walk along the tokens that are accepted.
//
// kv_tree_kernel: of every node its depth and, as bits over the tree's slots, which of them it sees: its ancestors and itself, as far
// as the window around its position lets it.  The attention kernels read a word of bits where they would compare slots.  A thread goes
// up from a node twice, for its depth and for its bits, in shared memory and run by run: nodes whose parent is the one before them follow
// each other in slots and positions, so that a line of drafts is one step and a tree takes as many as it branches on the way.  All latency: a
// tree of 26 nodes takes 3 us, most of it the launch; the attention starts beside it.
//
// draft_accept_kernel: a warp walks a tree.  A child comes after its parent, so one pass over the nodes in order finds the path: of each
// 32 nodes, those that agree with what was picked after their parent are known at once, and a ballot finds the first child of the node
// that the walk has come to.
#include <algorithm>

#include "kv_attn.cuh"

namespace pace {
namespace {

struct TreeArgs {
  KvTree t;
  const int32_t* lens;
  int max_len, window, sinks;
  int b0;                      // the launch's first sequence
  int cu[kKvMaxB + 1];
};

constexpr int kTreeThreads = 256;

__global__ void __launch_bounds__(kTreeThreads) kv_tree_kernel(const __grid_constant__ TreeArgs a, int* status) {
  constexpr int WORDS = PACE_TREE_MAX / 32;
  __shared__ int16_t up[PACE_TREE_MAX], head[PACE_TREE_MAX];      // parents; where the run of a node begins
  __shared__ uint32_t begins[WORDS];                              // nodes that begin one
  ptx::begin_call();
  const int b = blockIdx.x, at = a.cu[b], n = a.cu[b + 1] - at, lane = threadIdx.x & 31;
  const int base = min(max(a.lens[a.b0 + b], 0), a.max_len) - n;
  for (int t0 = threadIdx.x - lane; t0 < n; t0 += kTreeThreads) {
    const int t = t0 + lane;
    int p = t < n ? a.t.parents[at + t] : -1;
    if (p < -1 || p >= t) {
      record_error(status, PACE_ERR_INVALID_ARG, K_KV_TREE);
      p = -1;
    }
    up[t] = static_cast<int16_t>(p);
    const uint32_t bits = __ballot_sync(0xffffffffu, p != t - 1 || t == 0);
    if (lane == 0) begins[t0 / 32] = bits;
  }
  __syncthreads();
  for (int t = threadIdx.x; t < n; t += kTreeThreads) {
    int w = t / 32;
    uint32_t bits = begins[w] & (0xFFFFFFFFu >> (31 - t % 32));
    while (bits == 0) bits = begins[--w];      // (node 0 begins one)
    head[t] = static_cast<int16_t>(32 * w + 31 - __clz(bits));
  }
  __syncthreads();
  for (int t = threadIdx.x; t < n; t += kTreeThreads) {
    int depth = 0;
    for (int x = t;;) {
      depth += x - head[x];
      x = up[head[x]];
      if (x < 0) break;
      ++depth;
    }
    a.t.depth[at + t] = depth;
    // runs come in falling order, and so do the words of their slots
    uint32_t* row = a.t.family + static_cast<int64_t>(at + t) * a.t.words;
    int k = a.t.words - 1;
    uint32_t bits = 0;
    auto see = [&](int from, int to) {      // slots from .. to - 1
      from = max(from, 0);
      if (from >= to) return;
      for (int word = ((to - 1) >> 5) - (base >> 5), low = (from >> 5) - (base >> 5); word >= low; --word) {
        for (; k > word; --k) {
          row[k] = bits;
          bits = 0;
        }
        const int slot0 = 32 * (word + (base >> 5));
        bits |= below(to - slot0) & ~below(from - slot0);
      }
    };
    int place = base + depth, far = 0;      // position of x, generations from t
    for (int x = t; x >= 0;) {
      const int h = head[x], first = base + h, end = base + x + 1;      // the run's slots, positions up to `place`
      if (a.window > 0) {
        const int near = max(end - max(a.window - far, 0), first), sink = min(max(end - 1 - place + a.sinks, first), near);
        see(near, end);
        see(first, sink);
      } else {
        see(first, end);
      }
      far += x - h + 1;
      place -= x - h + 1;
      x = up[h];
    }
    for (; k >= 0; --k) {
      row[k] = bits;
      bits = 0;
    }
  }
}

constexpr int kAcceptMaxB = 1024;     // sequences of one launch
constexpr int kAcceptWarps = 4;

struct AcceptArgs {
  const int32_t* tokens;
  const int32_t* parents;
  const int32_t* picked;
  int32_t* rows;
  int32_t* counts;
  int32_t* next;
  int b0, nb;
  int cu[kAcceptMaxB + 1];
};

__global__ void __launch_bounds__(32 * kAcceptWarps) draft_accept_kernel(const __grid_constant__ AcceptArgs a, int* status) {
  ptx::begin_call();
  const int b = blockIdx.x * kAcceptWarps + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (b >= a.nb) return;
  const int at = a.cu[b], n = a.cu[b + 1] - at;
  int now = 0, count = 0;        // the node that the walk has come to; how many have been accepted
  if (n > 0) {
    if (lane == 0) a.rows[at] = at;
    count = 1;
  }
  constexpr int U = 4;           // 32 nodes each, loaded together
#pragma unroll 1
  for (int t0 = 0; t0 < n; t0 += 32 * U) {
    int parent[U];
    bool agrees[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + 32 * u + lane;
      parent[u] = t < n ? a.parents[at + t] : -1;
      if (parent[u] < -1 || parent[u] >= t) {
        record_error(status, PACE_ERR_INVALID_ARG, K_DRAFT_ACCEPT);
        parent[u] = -1;
      }
      agrees[u] = t < n && parent[u] >= 0 && a.tokens[at + t] == a.picked[at + parent[u]];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      uint32_t child;
      while ((child = __ballot_sync(0xffffffffu, agrees[u] && parent[u] == now)) != 0) {
        now = t0 + 32 * u + __ffs(child) - 1;
        if (lane == 0) a.rows[at + count] = at + now;
        ++count;
      }
    }
  }
  for (int i = count + lane; i < n; i += 32) a.rows[at + i] = -1;
  if (lane == 0) {
    a.counts[a.b0 + b] = count;
    a.next[a.b0 + b] = n > 0 ? a.picked[at + now] : -1;
  }
}

}  // namespace

pace_status_t launch_kv_tree(const KvTree& t, const int32_t* cu_q, int B, const int32_t* lens, int max_len, int window, int sinks, int* status,
                             cudaStream_t stream) {
  TreeArgs a{};
  a.t = t;
  a.lens = lens;
  a.max_len = max_len;
  a.window = window;
  a.sinks = sinks;
  for (int b0 = 0; b0 < B; b0 += kKvMaxB) {
    const int nb = std::min(kKvMaxB, B - b0);
    a.b0 = b0;
    for (int i = 0; i <= nb; ++i) a.cu[i] = cu_q[b0 + i];
    if (a.cu[nb] == a.cu[0]) continue;
    PACE_CHECK(launch_dependent(kv_tree_kernel, static_cast<unsigned>(nb), kTreeThreads, 0, 1, stream, a, status));
  }
  return PACE_OK;
}

}  // namespace pace

using namespace pace;

extern "C" pace_status_t pace_draft_accept(const int32_t* tokens, const int32_t* parents, const int32_t* picked, const int32_t* cu_nodes, int B,
                                           int32_t* rows, int32_t* counts, int32_t* next_tokens, pace_stream_t stream) {
  if (B < 0) return PACE_ERR_INVALID_ARG;
  if (B == 0) return PACE_OK;
  PACE_CHECK(check_prefix(cu_nodes, B));
  const int64_t n = cu_nodes[B];
  if (n > 0 && (tokens == nullptr || parents == nullptr || picked == nullptr || rows == nullptr)) return PACE_ERR_INVALID_ARG;
  if (counts == nullptr || next_tokens == nullptr) return PACE_ERR_INVALID_ARG;
  for (const int32_t* p : {tokens, parents, picked, static_cast<const int32_t*>(rows), static_cast<const int32_t*>(counts),
                           static_cast<const int32_t*>(next_tokens)})
    if (reinterpret_cast<uintptr_t>(p) % 4 != 0) return PACE_ERR_INVALID_ARG;
  for (const int32_t* p : {tokens, parents, picked})
    if (overlap(rows, n, p, n) || overlap(counts, B, p, n) || overlap(next_tokens, B, p, n)) return PACE_ERR_INVALID_ARG;
  if (overlap(rows, n, counts, B) || overlap(rows, n, next_tokens, B) || overlap(counts, B, next_tokens, B)) return PACE_ERR_INVALID_ARG;
  PACE_CHECK(check_device());
  int* status = device_status_word();
  AcceptArgs a{};
  a.tokens = tokens;
  a.parents = parents;
  a.picked = picked;
  a.rows = rows;
  a.counts = counts;
  a.next = next_tokens;
  for (int b0 = 0; b0 < B; b0 += kAcceptMaxB) {
    a.b0 = b0;
    a.nb = std::min(kAcceptMaxB, B - b0);
    for (int i = 0; i <= a.nb; ++i) a.cu[i] = cu_nodes[b0 + i];
    PACE_CHECK(launch_dependent(draft_accept_kernel, static_cast<unsigned>((a.nb + kAcceptWarps - 1) / kAcceptWarps), 32 * kAcceptWarps, 0, 1,
                                stream, a, status));
  }
  return PACE_OK;
}
