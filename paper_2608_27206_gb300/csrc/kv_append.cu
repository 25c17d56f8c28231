// Serve: new keys and values into the paged 8-bit cache, rotated on the way, and the rotation table.
//
// A pair (x1, x2) = (x[i], x[i + D/2]) of a key turns by its position's angle,
//   y1 = x1 c - x2 s,  y2 = x2 c + x1 s,
// and a block of 16 slots and one head is stored as e4m3 codes round(y / s) with the smallest power
// of two s that covers the block.  The power costs e4m3 nothing (it is a floating format) and makes
// the growth of a block's scale, when a later token needs more, an exact factor on its older codes.
//
// What bounds it is HBM: a token's rows once in, its codes and turned queries once out; what stands in the way is the chain of loads
// before them (length, row, position, angles).  One CTA per touched block, three to an SM: it stages the tokens' (cos, sin) once
// for all heads while the first rows are on their way; a warp takes a head's 16 rows of K or V, 16 bytes per lane and load, both halves
// of a pair in one lane, 16 bits wide until they are used.  For the queries a lane keeps its row's angles in registers
// and goes over heads, four in flight.  16 prompts, 44000 tokens of 28 + 8 heads of 128: 137 us, 5.9 TB/s (two CTAs per SM 145,
// four 149: registers).  A decode step is latency: 64 tokens in 9 us.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cmath>

#include "pace_kv.cuh"
#include "pace_ptx.cuh"

namespace pace {
namespace {

constexpr int kAppendThreads = 256;

struct AppendArgs {
  KvView c;
  const uint16_t* K;
  const uint16_t* V;
  const uint16_t* Q;
  uint16_t* q_out;
  int64_t k_stride, v_stride, q_stride, n_src, table_stride;
  const int32_t* lens;
  const int32_t* table;
  const int32_t* rows;
  const float2* rope;
  const int32_t* pos;
  int64_t n_pos, pos_stride;
  int sec0, sec01, q_heads;
  int b0, nb;                      // the launch's sequences
  int cu[kKvMaxB + 1];             // first token of each
  int block_prefix[kKvMaxB + 1];   // blocks that a sequence's tokens may touch, at most
};

// Eight elements of either half of a row: a[i] and b[i] are a pair.
struct Raw {
  uint4 a, b;
};
struct Pairs {
  float2 a[4], b[4];
};
__device__ __forceinline__ void widen(const uint4& u, float2 (&f)[4]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
}
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint4 pack_bf16(const float2 (&f)[4]) {
  return make_uint4(bf16x2(f[0].x, f[0].y), bf16x2(f[1].x, f[1].y), bf16x2(f[2].x, f[2].y), bf16x2(f[3].x, f[3].y));
}

// (cos, sin) of eight pairs, two at a time.
struct Turn {
  float2 c[4], s[4];
};
__device__ __forceinline__ Turn load_turn(const float2* cs) {
  Turn t;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 u = *reinterpret_cast<const float4*>(cs + 2 * i);
    t.c[i] = make_float2(u.x, u.z);
    t.s[i] = make_float2(u.y, u.w);
  }
  return t;
}
// Products and sums rounded one by one, so that a result does not hang on the contraction into FMAs.  The sums are scalar: ptxas joins a
// packed sum (add, or an FMA by 1) with the packed product before it, rounding modifiers or not.
__device__ __forceinline__ void turn(Pairs& x, const Turn& t) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 ac = ptx::fmul2(x.a[i], t.c[i]), bs = ptx::fmul2(x.b[i], t.s[i]);
    const float2 bc = ptx::fmul2(x.b[i], t.c[i]), as = ptx::fmul2(x.a[i], t.s[i]);
    x.a[i] = make_float2(__fsub_rn(ac.x, bs.x), __fsub_rn(ac.y, bs.y));
    x.b[i] = make_float2(__fadd_rn(bc.x, as.x), __fadd_rn(bc.y, as.y));
  }
}
// Adds a NaN to `all` if an element is not finite, else zeros.
__device__ __forceinline__ void see_finite(const Pairs& x, float2& all) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    all = ptx::ffma2(x.a[i], make_float2(0.f, 0.f), all);
    all = ptx::ffma2(x.b[i], make_float2(0.f, 0.f), all);
  }
}
__device__ __forceinline__ void drop_infinite(Pairs& x) {
  auto fix = [](float& v) { v = fabsf(v) < INFINITY ? v : 0.f; };
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    fix(x.a[i].x);
    fix(x.a[i].y);
    fix(x.b[i].x);
    fix(x.b[i].y);
  }
}

template <int D>
__global__ void __launch_bounds__(kAppendThreads, 3) kv_append_kernel(const __grid_constant__ AppendArgs a, int* status) {
  constexpr int H = D / 2, LPR = D / 16, RPP = 32 / LPR, PASS = kKvBlock / RPP;   // lanes per row, rows per pass
  __shared__ __align__(16) float2 cs[kKvBlock][H];
  __shared__ int64_t src[kKvBlock];   // source row of each slot; -1: no (valid) new token there
  __shared__ int pos[3][kKvBlock];
  ptx::begin_call();
  int lo = 0, hi = a.nb - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.block_prefix[mid] <= static_cast<int>(blockIdx.x)) lo = mid;
    else hi = mid - 1;
  }
  const int b = lo, n = a.cu[b + 1] - a.cu[b];
  // (a length may be anything: slots in 64 bits until they are known to be in the table)
  const int64_t len = a.lens[a.b0 + b], first = len - n;
  if (first < 0) {
    if (threadIdx.x == 0) record_error(status, PACE_ERR_INVALID_ARG, K_KV_APPEND);
  }
  // (of a sequence shorter than its new tokens those before its first slot are dropped)
  const int64_t slot0 = (first < 0 ? 0 : first / kKvBlock * kKvBlock) + static_cast<int64_t>(blockIdx.x - a.block_prefix[b]) * kKvBlock;
  if (slot0 >= len) return;
  const int r_lo = static_cast<int>(max(first - slot0, int64_t{0})), r_hi = static_cast<int>(min(len - slot0, int64_t{kKvBlock}));
  const int64_t pi = slot0 >> a.c.page_shift;
  const int slot = static_cast<int>(slot0) & ((1 << a.c.page_shift) - 1);      // of row 0, in its page
  int page = -1;
  if (pi < a.table_stride) page = a.table[(a.b0 + b) * a.table_stride + pi];
  const int token0 = a.cu[b] + static_cast<int>(slot0 - first);   // of row 0, where that is a new token
  if (threadIdx.x < kKvBlock) {
    const int r = threadIdx.x;
    int64_t s = -1;
    if (r >= r_lo && r < r_hi) {
      s = a.rows != nullptr ? a.rows[token0 + r] : token0 + r;
      bool ok = s >= 0 && s < a.n_src;
      if (ok && a.rope != nullptr) {
        const int n_rows = a.sec01 < H ? 3 : a.sec0 < a.sec01 ? 2 : 1;
        int p[3] = {0, 0, 0};
#pragma unroll
        for (int c = 0; c < 3; ++c)
          if (c < n_rows) p[c] = a.pos[c * a.pos_stride + s];
#pragma unroll
        for (int c = 0; c < 3; ++c) {
          ok = ok && p[c] >= 0 && p[c] < a.n_pos;
          pos[c][r] = p[c];
        }
      }
      if (!ok) {
        record_error(status, PACE_ERR_INVALID_ARG, K_KV_APPEND);
        s = -1;
      }
    }
    src[r] = s;
  }
  if (page < 0 || page >= a.c.n_pages) {
    if (threadIdx.x == 0) record_error(status, PACE_ERR_INVALID_ARG, K_KV_APPEND);
    page = -1;
  }
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = kAppendThreads / 32;
  const int col = (lane % LPR) * 8, row0 = lane / LPR;
  const bool turned = a.rope != nullptr;
  auto load = [&](const uint16_t* from) { return Raw{*reinterpret_cast<const uint4*>(from), *reinterpret_cast<const uint4*>(from + H)}; };
  // ---- the cache: a warp takes a head's 16 rows of K or V
  bool staged = !turned;
#pragma unroll 1
  for (int task = warp;; task += warps) {
    const bool is_v = task >= a.c.heads, mine = task < 2 * a.c.heads && page >= 0;
    const int head = is_v ? task - a.c.heads : task;
    Raw x[PASS];
    if (mine) {
      const uint16_t* base = (is_v ? a.V : a.K) + static_cast<int64_t>(head) * D + col;
      const int64_t stride = is_v ? a.v_stride : a.k_stride;
#pragma unroll
      for (int p = 0; p < PASS; ++p) {
        const int64_t s = src[p * RPP + row0];
        x[p] = Raw{};
        if (s >= 0) x[p] = load(base + s * stride);
      }
    }
    if (!staged) {      // (while the first rows are on their way)
      staged = true;
#pragma unroll 4
      for (int i = threadIdx.x; i < kKvBlock * H; i += kAppendThreads) {
        const int r = i / H, p = i % H;
        if (src[r] < 0) continue;
        cs[r][p] = a.rope[static_cast<int64_t>(pos[p < a.sec0 ? 0 : p < a.sec01 ? 1 : 2][r]) * H + p];
      }
      __syncthreads();
    }
    if (!mine) break;
    auto get = [&](int p, bool strict) {      // pass p's elements as they are to be stored
      Pairs e;
      widen(x[p].a, e.a);
      widen(x[p].b, e.b);
      if (!is_v && turned && src[p * RPP + row0] >= 0) turn(e, load_turn(&cs[p * RPP + row0][col]));
      if (strict) drop_infinite(e);
      return e;
    };
    // The rows stay 16 bits wide and are turned twice, for their maximum and for their codes: 32 registers instead of 64
    float amax = 0.f;
    bool strict = false;
#pragma unroll 1
    while (true) {
      float2 all = make_float2(0.f, 0.f);
      amax = 0.f;
#pragma unroll
      for (int p = 0; p < PASS; ++p) {
        const Pairs e = get(p, strict);
        see_finite(e, all);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          amax = ptx::max3(amax, fabsf(e.a[i].x), fabsf(e.a[i].y));
          amax = ptx::max3(amax, fabsf(e.b[i].x), fabsf(e.b[i].y));
        }
      }
      if (!__any_sync(0xffffffffu, !(all.x + all.y == 0.f))) break;
      if (lane == 0) record_error(status, PACE_ERR_INVALID_ARG, K_KV_APPEND);
      strict = true;      // what is not finite counts as 0
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
    const int blocks = 1 << (a.c.page_shift - 4);
    float* scale = (is_v ? a.c.vs : a.c.ks) + page * a.c.scale_stride + head * blocks + slot / kKvBlock;
    uint8_t* codes = (is_v ? a.c.v : a.c.k) + page * a.c.page_stride +
                     ((static_cast<int64_t>(head) << a.c.page_shift) + slot) * D + col;
    float s = scale_for(amax), ratio = 1.f;
    if (r_lo > 0) {
      const float old = *scale;
      if (old > 0.f && old < INFINITY) {
        s = fmaxf(s, old);
        ratio = __fdiv_rn(old, s);
      }
      __syncwarp();   // every lane has read the scale
    }
    if (lane == 0) *scale = s;
    const float inv = __frcp_rn(s);   // exact: a power of two from 2^-120 to 2^64
    const float2 inv2 = make_float2(inv, inv);
#pragma unroll
    for (int p = 0; p < PASS; ++p) {
      const int r = p * RPP + row0;
      uint8_t* o = codes + r * D;
      if (src[r] >= 0) {
        Pairs e = get(p, strict);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          e.a[i] = ptx::fmul2(e.a[i], inv2);
          e.b[i] = ptx::fmul2(e.b[i], inv2);
        }
        *reinterpret_cast<uint2*>(o) = make_uint2(e4m3x4(e.a[0].x, e.a[0].y, e.a[1].x, e.a[1].y), e4m3x4(e.a[2].x, e.a[2].y, e.a[3].x, e.a[3].y));
        *reinterpret_cast<uint2*>(o + H) = make_uint2(e4m3x4(e.b[0].x, e.b[0].y, e.b[1].x, e.b[1].y), e4m3x4(e.b[2].x, e.b[2].y, e.b[3].x, e.b[3].y));
      } else if (r < r_lo && ratio != 1.f) {   // an older token under the grown scale
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
          const uint2 w = *reinterpret_cast<const uint2*>(o + h * H);
          uint32_t z[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t u = i == 0 ? w.x : w.y;
            const uint32_t f0 = e4m3x2_to_f16x2(u & 0xFFFFu), f1 = e4m3x2_to_f16x2(u >> 16);
            const float2 g0 = __half22float2(*reinterpret_cast<const __half2*>(&f0));
            const float2 g1 = __half22float2(*reinterpret_cast<const __half2*>(&f1));
            z[i] = e4m3x4(g0.x * ratio, g0.y * ratio, g1.x * ratio, g1.y * ratio);
          }
          *reinterpret_cast<uint2*>(o + h * H) = make_uint2(z[0], z[1]);
        }
      }
    }
  }
  if (a.q_heads == 0) return;
  // ---- the queries: a warp keeps a pass of rows, with their angles, and goes over heads; warps share out the passes that have rows
  const int p_lo = r_lo / RPP, live = (r_hi - 1) / RPP - p_lo + 1, over = live > 2 ? 4 : live;
  const int p = p_lo + warp % over, r = p * RPP + row0;
  if (p >= PASS || r < r_lo || r >= r_hi) return;
  const int64_t s = src[r];
  uint16_t* to = a.q_out + static_cast<int64_t>(token0 + r) * a.q_heads * D + col;
  const uint16_t* from = a.Q + max(s, static_cast<int64_t>(0)) * a.q_stride + col;
  Turn t{};
  if (turned && s >= 0) t = load_turn(&cs[r][col]);
  float2 all = make_float2(0.f, 0.f);
  const int step = warps / over;
#pragma unroll 1
  for (int h0 = warp / over; h0 < a.q_heads; h0 += 4 * step) {
    Raw x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[k] = Raw{};      // (the query of a token that could not be found is zero)
      if (h0 + k * step < a.q_heads && s >= 0) x[k] = load(from + static_cast<int64_t>(h0 + k * step) * D);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (h0 + k * step >= a.q_heads) break;
      Pairs e;
      widen(x[k].a, e.a);
      widen(x[k].b, e.b);
      if (turned) turn(e, t);
      see_finite(e, all);
      uint16_t* o = to + static_cast<int64_t>(h0 + k * step) * D;
      *reinterpret_cast<uint4*>(o) = turned ? pack_bf16(e.a) : x[k].a;
      *reinterpret_cast<uint4*>(o + H) = turned ? pack_bf16(e.b) : x[k].b;
    }
  }
  if (!(all.x + all.y == 0.f)) record_error(status, PACE_ERR_INVALID_ARG, K_KV_APPEND);
}

__global__ void __launch_bounds__(256) rope_table_kernel(float2* table, int64_t n_positions, int half, double step) {
  ptx::begin_call();
  const int64_t total = n_positions * half;
  for (int64_t i = blockIdx.x * static_cast<int64_t>(blockDim.x) + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * blockDim.x) {
    double s, c;
    sincos(static_cast<double>(i / half) * exp(step * static_cast<double>(i % half)), &s, &c);
    table[i] = make_float2(static_cast<float>(c), static_cast<float>(s));
  }
}

}  // namespace
}  // namespace pace

using namespace pace;

extern "C" pace_status_t pace_rope_table(float* table, int64_t n_positions, int head_dim, double base, pace_stream_t stream) {
  if (n_positions < 0 || n_positions > INT32_MAX || (head_dim != 64 && head_dim != 128) || !(base > 0.0) || !std::isfinite(base))
    return PACE_ERR_INVALID_ARG;
  if (n_positions == 0) return PACE_OK;
  if (table == nullptr || reinterpret_cast<uintptr_t>(table) % 16 != 0) return PACE_ERR_INVALID_ARG;
  PACE_CHECK(check_device());
  const int half = head_dim / 2;
  const unsigned grid = static_cast<unsigned>(std::min<int64_t>((n_positions * half + 255) / 256, 4096));
  return launch_dependent(rope_table_kernel, grid, 256, 0, 1, stream, reinterpret_cast<float2*>(table), n_positions, half,
                          -2.0 * std::log(base) / head_dim);
}

extern "C" pace_status_t pace_kv_append(const pace_kv_cache* cache, const void* K, const void* V, int64_t k_row_stride,
                                        int64_t v_row_stride, int64_t n_src_rows, const int32_t* cu_new, int B,
                                        const int32_t* seq_lens, const int32_t* block_table, int64_t table_stride,
                                        const int32_t* rows, const pace_rope* rope, const void* Q, int64_t q_row_stride,
                                        int n_q_heads, void* q_out, pace_stream_t stream) {
  if (B < 0) return PACE_ERR_INVALID_ARG;
  if (B == 0) return PACE_OK;
  PACE_CHECK(check_cache(cache));
  PACE_CHECK(check_prefix(cu_new, B));
  if (cu_new[B] == 0) return PACE_OK;
  const int D = cache->head_dim;
  if (!rows_ok(K, k_row_stride, cache->n_kv_heads, D) || !rows_ok(V, v_row_stride, cache->n_kv_heads, D)) return PACE_ERR_INVALID_ARG;
  if (seq_lens == nullptr || block_table == nullptr || table_stride < 1 || n_src_rows < 1 || n_src_rows > INT32_MAX)
    return PACE_ERR_INVALID_ARG;
  if (rows == nullptr && n_src_rows < cu_new[B]) return PACE_ERR_INVALID_ARG;
  if ((Q == nullptr) != (q_out == nullptr)) return PACE_ERR_INVALID_ARG;
  if (Q != nullptr && (n_q_heads < 1 || n_q_heads > kKvMaxQHeads || !rows_ok(Q, q_row_stride, n_q_heads, D) ||
                       reinterpret_cast<uintptr_t>(q_out) % 16 != 0))
    return PACE_ERR_INVALID_ARG;
  AppendArgs a{};
  if (rope != nullptr) {
    const int32_t* s = rope->sections;
    if (rope->table == nullptr || rope->positions == nullptr || reinterpret_cast<uintptr_t>(rope->table) % 16 != 0 ||
        rope->n_positions < 1 || rope->positions_stride < 0 || s[0] < 0 || s[1] < 0 || s[2] < 0 ||
        static_cast<int64_t>(s[0]) + s[1] + s[2] != D / 2)
      return PACE_ERR_INVALID_ARG;
    a.rope = reinterpret_cast<const float2*>(rope->table);
    a.pos = rope->positions;
    a.n_pos = rope->n_positions;
    a.pos_stride = rope->positions_stride;
    a.sec0 = s[0];
    a.sec01 = s[0] + s[1];
  }
  PACE_CHECK(check_device());
  a.c = kv_view(cache);
  a.K = static_cast<const uint16_t*>(K);
  a.V = static_cast<const uint16_t*>(V);
  a.Q = static_cast<const uint16_t*>(Q);
  a.q_out = static_cast<uint16_t*>(q_out);
  a.k_stride = k_row_stride;
  a.v_stride = v_row_stride;
  a.q_stride = q_row_stride;
  a.n_src = n_src_rows;
  a.table_stride = table_stride;
  a.lens = seq_lens;
  a.table = block_table;
  a.rows = rows;
  a.q_heads = Q != nullptr ? n_q_heads : 0;
  int* status = device_status_word();
  for (int b0 = 0; b0 < B; b0 += kKvMaxB) {
    a.b0 = b0;
    a.nb = std::min(kKvMaxB, B - b0);
    int64_t blocks = 0;
    for (int i = 0; i <= a.nb; ++i) {
      a.cu[i] = cu_new[b0 + i];
      a.block_prefix[i] = static_cast<int>(blocks);
      if (i < a.nb) {
        const int n = cu_new[b0 + i + 1] - cu_new[b0 + i];
        if (n > 0) blocks += (n + 2 * (kKvBlock - 1)) / kKvBlock;   // wherever in a block the first one lands
      }
    }
    if (blocks == 0) continue;
    auto* kernel = D == 128 ? kv_append_kernel<128> : kv_append_kernel<64>;
    PACE_CHECK(launch_dependent(kernel, static_cast<unsigned>(blocks), kAppendThreads, 0, 1, stream, a, status));
  }
  return PACE_OK;
}
