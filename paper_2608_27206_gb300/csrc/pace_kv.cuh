// What the calls on the paged 8-bit cache share: argument checks, the table of sequences, the scale rule.
#pragma once
#include <cstdint>

#include "pace_common.cuh"

namespace pace {

constexpr int kKvMaxB = 256;          // sequences of one launch
constexpr int kKvBlock = PACE_KV_BLOCK;
constexpr int kKvMaxGroup = 64, kKvMaxQHeads = 256 * kKvMaxGroup;      // query heads per KV head, in all

// The cache as the kernels take it.
struct KvView {
  uint8_t* k;
  uint8_t* v;
  float* ks;
  float* vs;
  int64_t page_stride, scale_stride;
  int n_pages, page_shift, heads;
};

inline pace_status_t check_cache(const pace_kv_cache* c) {
  if (c == nullptr || c->k == nullptr || c->v == nullptr || c->k_scale == nullptr || c->v_scale == nullptr)
    return PACE_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return PACE_ERR_INVALID_ARG;
  if (c->n_kv_heads < 1 || c->n_kv_heads > 256) return PACE_ERR_INVALID_ARG;
  const int p = c->page_size;
  if (p != 16 && p != 32 && p != 64 && p != 128 && p != 256) return PACE_ERR_INVALID_ARG;
  if (c->n_pages < 1 || c->n_pages > INT32_MAX) return PACE_ERR_INVALID_ARG;
  const int64_t page = static_cast<int64_t>(c->n_kv_heads) * p * c->head_dim;
  if (c->page_stride < page || c->page_stride % 16 != 0 || c->page_stride > INT64_MAX / c->n_pages) return PACE_ERR_INVALID_ARG;
  if (c->scale_stride < static_cast<int64_t>(c->n_kv_heads) * (p / kKvBlock)) return PACE_ERR_INVALID_ARG;
  if (c->scale_stride > INT64_MAX / 4 / c->n_pages) return PACE_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v)) % 16 != 0) return PACE_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(c->k_scale) | reinterpret_cast<uintptr_t>(c->v_scale)) % 4 != 0) return PACE_ERR_INVALID_ARG;
  return PACE_OK;
}

inline KvView kv_view(const pace_kv_cache* c) {
  int shift = 4;
  while ((1 << shift) < c->page_size) ++shift;
  return KvView{static_cast<uint8_t*>(c->k), static_cast<uint8_t*>(c->v), c->k_scale, c->v_scale, c->page_stride,
                c->scale_stride, static_cast<int>(c->n_pages), shift, c->n_kv_heads};
}

// A host prefix of tokens per sequence: starts at 0, never falls, below 2^30 tokens.
inline pace_status_t check_prefix(const int32_t* cu, int B) {
  if (cu == nullptr || cu[0] != 0) return PACE_ERR_INVALID_ARG;
  for (int b = 0; b < B; ++b)
    if (cu[b + 1] < cu[b]) return PACE_ERR_INVALID_ARG;
  return cu[B] <= (1 << 30) ? PACE_OK : PACE_ERR_INVALID_ARG;
}

// Rows `stride` elements apart of `heads` heads of D bf16: 16-byte aligned, no overlap.
inline bool rows_ok(const void* p, int64_t stride, int heads, int D) {
  return p != nullptr && reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % 8 == 0 &&
         stride >= static_cast<int64_t>(heads) * D && stride <= (int64_t{1} << 31);
}

// Exponent bits of the smallest power of two s with amax <= 448 s, from 2^-64 to 2^120 (448 = 1.75 * 2^8).
__device__ __forceinline__ float scale_for(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = static_cast<int>(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return __uint_as_float(static_cast<uint32_t>(max(min(e, 127 + 120), 127 - 64)) << 23);
}

// Two e4m3 codes (ties to even, saturating at 448, NaN stays NaN), `lo` in the low byte.
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  return e4m3x2(a, b) | (e4m3x2(c, d) << 16);
}
// The values of two codes, exactly, as f16.
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t two) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(static_cast<uint16_t>(two)));
  return r;
}

}  // namespace pace
