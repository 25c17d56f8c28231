// Serve: attention over the paged cache for few query rows per KV head (decode steps, drafted tokens).
//
// K and V cross HBM once and go to the tensor cores as the 8-bit codes they are.  With so few rows the
// codes are the large operand of both products, so both are formed transposed:
//   S^T [128 slots x rows] = K [slots x D] q^T         O^T [D x rows] += V^T [D x slots] P^T
// A 16-bit factor enters as two e4m3 terms side by side, x = hi + lo / 16: to 8 bits for the weights P; of bf16 q (8
// significant bits are two times 4; each row is first brought under 256 by a power of two, to 128 at least) exactly for elements
// of 2^-6 and more, smaller ones, those under 2^-13 of the row's largest, are off by 2^-14 at most.  Terms are columns of the same product, so they cost little while N is small.
// Two terms hold 8 bits of P from 2^-5 to 448 only, 2^-9 to 1 of the largest weight.  A context of tens of thousands of slots of which
// one draws half of the weight has nearly all of its others below that, and they make up the output where that one's value is
// small: held to a floor of 2^-18 of the largest they cost it percents.  So weights below 2^-5 go into two more columns, times 2^13: 8
// bits down to 2^-22 of the largest, and an absolute error of 2^-31 below.
//
// A TMEM lane of S^T is a slot.  Its thread applies the block's K scale and the mask, and turns the score x
// (base 2) of row q into the weight 2^(x - m_q), which it sums, and into P = 16 * 2^(x - m_q) vs 2^-r_q,
// vs being the block's V scale.  m_q and m_q + r_q stand for the largest x and the largest x + log2(vs) so far, but lag
// behind: they move only when a weight would pass 2^60 or P 256 (e4m3 ends at 448).  So the usual tile has no maximum and no
// exchange between threads but one barrier's vote, and O^T stays in TMEM untouched.  Whatever x is, log2(vs) is only ever added to
// a difference of scores: added to a score of 2^24 and more it would be rounded.
//
// What bounds it is HBM where rows are few: per slot and head 2 D bytes.  From S of a tile to its P takes a group of four warps more than
// a microsecond, one and a half times what a tile of 32 KB takes an SM to fetch; so two groups take every other tile, each with its own
// m, r, l and O^T, and join them at the item's end.  64 sequences of 5001-28007 slots, 4 heads of 128, 7 rows: 156 us, 5.6 TB/s (with one
// pair of columns for P 153; one group took 210 against 150).  With 32 rows it is the groups: 463 us, 34 us of it the second pair's
// stores and products of twice the columns.
// Roles of a CTA (one per SM): warp 0 fetches tiles of 128 slots (TMA boxes of a page each, scales by 4-byte copies) through a
// ring of stages, warp 1 issues the MMAs, warps 2-5 and 6-9 own the 128 lanes of even and odd tiles.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "kv_attn.cuh"

namespace pace {
namespace {

using namespace ptx;

constexpr int kWarps = 10, kThreads = 32 * kWarps;
constexpr float kFar = 60.f;         // how far a score may pass m_q
constexpr float kOver = 4.f;         // ... and x + log2(vs) may pass m_q + r_q
constexpr float kUnit = 4.f;         // log2 of P at m_q + r_q
constexpr float kSmall = 0x1p-5f, kTimes = 0x1p13f;      // P below the first takes the second pair of columns, times the second

template <int D, int NQ>
struct DecodeCfg {
  static constexpr int TILE = kKvTile * D;              // bytes of a K or V tile
  static constexpr int STAGES = D == 128 ? (NQ == 8 ? 6 : NQ == 16 ? 5 : 4) : (NQ == 8 ? 12 : NQ == 16 ? 11 : 9);      // what fits
  static constexpr int QBYTES = 2 * NQ * D;             // hi rows, then lo rows
  static constexpr int PBYTES = 4 * NQ * kKvTile;       // 16 columns of every slot, then the next 16
  static constexpr uint32_t SWIZZLE = D == 128 ? 2 : 4;
  static constexpr uint32_t GROUP = 8 * D;              // bytes of 8 rows
  static constexpr int COLS = 2 * NQ, OCOLS = 4 * NQ;   // TMEM: four S, then O of either group
  static constexpr uint32_t O_AT = 4 * COLS;
  static constexpr uint32_t TMEM = NQ == 8 ? 128 : NQ == 16 ? 256 : 512;
  static constexpr uint32_t IDESC_S = idesc_e4m3_f32(128, COLS, false, false);
  static constexpr uint32_t IDESC_O = idesc_e4m3_f32(128, OCOLS, true, true);
};

struct Stat {
  float m, r, over, g;     // m_q, r_q, r_q + kOver, 2^(kUnit - r_q)
};

template <int D, int NQ>
struct alignas(16) DecodeCtl {
  uint64_t full[DecodeCfg<D, NQ>::STAGES], empty[DecodeCfg<D, NQ>::STAGES], s_full[4], p_full[4], pv_done[4], q_full;
  Stat stat[2][NQ];
  float qc[NQ];             // scale2 * the row's power of two
  int slot_of[NQ];          // slot of the row's query
  float2 fac[2][NQ];
  int64_t out_at[NQ];
  float2 red[2][4][NQ];
  float scales[DecodeCfg<D, NQ>::STAGES][16];   // a tile's K scales, then its V scales
  int scan[2 * kWarps];
  KvShare share;
  uint32_t tmem;
  int abort;
};

// Largest of the warp's values (a NaN counts only where all are).
__device__ __forceinline__ float warp_max(float x) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}

template <int D, int NQ>
__global__ void __launch_bounds__(kThreads, 1) kv_decode_kernel(const __grid_constant__ KvMaps maps, const __grid_constant__ KvAttnArgs a,
                                                                int* status) {
  using C = DecodeCfg<D, NQ>;
  constexpr int ST = C::STAGES;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sKV = smem;                         // stages of a K tile and a V tile
  uint8_t* sQ = sKV + ST * 2 * C::TILE;
  uint8_t* sP = sQ + C::QBYTES;                // four
  auto* ctl = reinterpret_cast<DecodeCtl<D, NQ>*>(sP + 4 * C::PBYTES);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto full = [&](int s) { return smem_u32(&ctl->full[s]); };
  auto empty = [&](int s) { return smem_u32(&ctl->empty[s]); };
  auto s_full = [&](int p) { return smem_u32(&ctl->s_full[p]); };
  auto p_full = [&](int p) { return smem_u32(&ctl->p_full[p]); };
  auto pv_done = [&](int p) { return smem_u32(&ctl->pv_done[p]); };
  const uint32_t q_full = smem_u32(&ctl->q_full);

  begin_call();
  const KvShare share = kv_share<NQ, D>(a, ctl->scan, &ctl->share, status);
  if (static_cast<int>(blockIdx.x) >= share.ctas) {
    if (threadIdx.x == 0) a.split[blockIdx.x] = KvSplit{0, 0, 0, 0};
    return;
  }
  if (warp == 0 && lane == 0) {
    prefetch_tensormap(&maps.k);
    prefetch_tensormap(&maps.v);
    for (int s = 0; s < ST; ++s) {
      mbar_init(full(s), 33);      // the byte count's arrival and 32 lanes' scales
      mbar_init(empty(s), 1);
    }
    for (int p = 0; p < 4; ++p) {
      mbar_init(s_full(p), 1);
      mbar_init(p_full(p), 4);
      mbar_init(pv_done(p), 1);
    }
    mbar_init(q_full, 8);
    fence_mbar_init();
    ctl->abort = 0;
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&ctl->tmem), C::TMEM);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = ctl->tmem;
  KvWalk<NQ> walk;
  walk.begin(share);

  if (warp == 0) {
    kv_fetch<D, ST, ST>(maps, a, walk, KvRings{sKV, sKV + C::TILE, 2 * C::TILE, ctl->full, ctl->empty, nullptr, ctl->scales}, &ctl->abort, status);
  } else if (warp == 1) {
    // ---- products ----------------------------------------------------------------------------
    if (lane == 0) {
      const uint64_t dq = smem_desc(smem_u32(sQ), 16, C::GROUP, C::SWIZZLE);
      // V^T: 8 slots of D contiguous codes per repeat.  (D = 64 fills lanes 0-63; the other half of the 128 rows reads
      // the same codes again and is not used.)
      const uint64_t dk = smem_desc(smem_u32(sKV), 16, C::GROUP, C::SWIZZLE);
      const uint64_t dv = smem_desc(smem_u32(sKV + C::TILE), 0, C::GROUP, C::SWIZZLE);
      const uint64_t dp = smem_desc(smem_u32(sP), 8 * 16, 16 * kKvTile, 0);
      int t = 0, items = 0;
      bool ok = true;
      auto weigh = [&](int u, bool first) {     // O += V^T P of tile u
        if (!kv_wait(p_full(u & 3), (u >> 2) & 1)) return false;
        tc_fence_after_sync();
        const uint64_t v = dv + static_cast<uint64_t>((u % ST) * 2 * (C::TILE >> 4)), p = dp + static_cast<uint64_t>((u & 3) * (C::PBYTES >> 4));
#pragma unroll
        for (int k = 0; k < kKvTile / 32; ++k)
          mma_f8_ss(tmem + C::O_AT + (u & 1) * C::OCOLS, v + static_cast<uint64_t>(k * (32 * D >> 4)), p + static_cast<uint64_t>(k * (32 * 16 >> 4)),
                    C::IDESC_O, !first || k > 0);
        mma_commit(empty(u % ST));
        mma_commit(pv_done(u & 3));
        return true;
      };
      // S goes two tiles ahead, so that a group finds its next one when it is done with one.  (S and P of tile t are in place t % 4, and so is the barrier of its P V: a
      // parity names one of two phases, and of the group's last two products the first need not be complete.
      // S of tile t comes after P V of tile t - 3, which waited for P of that tile: who sees it complete may overwrite P of tile t - 4.)
      while (ok && walk.next(a)) {
        ok = kv_wait(q_full, items & 1);
        ++items;
        const int n = walk.it.t1 - walk.it.t0;
#pragma unroll 1
        for (int i = 0; ok && i < n + 2; ++i) {
          if (i < n) {
            const int u = t + i;
            ok = kv_wait(full(u % ST), (u / ST) & 1);
            if (!ok) break;
            tc_fence_after_sync();
            const uint64_t k0 = dk + static_cast<uint64_t>((u % ST) * 2 * (C::TILE >> 4));
#pragma unroll
            for (int k = 0; k < D / 32; ++k)
              mma_f8_ss(tmem + (u & 3) * C::COLS, k0 + static_cast<uint64_t>(2 * k), dq + static_cast<uint64_t>(2 * k), C::IDESC_S, k > 0);
            mma_commit(s_full(u & 3));
          }
          if (i >= 2) ok = weigh(t + i - 2, i < 4);
        }
        t += n;
      }
      if (!ok) stop(&ctl->abort, status);
    }
    __syncwarp();
  } else {
    // ---- weights -----------------------------------------------------------------------------
    const int grp = warp >= 6, quad = warp & 3, me = quad * 32 + lane;    // TMEM lane: slot of the tile, then column of the output
    const uint32_t lanes = tmem + (static_cast<uint32_t>(quad * 32) << 16);
    Stat* stat = ctl->stat[grp];
    int t = 0;
    while (walk.next(a)) {
      const KvItem& it = walk.it;
      bool bad = false;
      named_barrier_sync(3, 256);      // the last item's shared statistics have been read
      // q: rows of this item as hi and lo codes (rows past it are zero), the power of two of each
#pragma unroll 1
      for (int q = warp - 2; q < NQ; q += 8) {
        constexpr int E = D / 32;      // elements of a lane
        float x[E];
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = 0.f;
        if (q < it.rows) {
          const uint16_t* src = kv_query(a, it, q, D) + lane * E;
          uint32_t w[E / 2];
          if constexpr (E == 4) {
            const uint2 u = *reinterpret_cast<const uint2*>(src);
            w[0] = u.x;
            w[1] = u.y;
          } else {
            w[0] = *reinterpret_cast<const uint32_t*>(src);
          }
#pragma unroll
          for (int e = 0; e < E; ++e) x[e] = __uint_as_float(e & 1 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
        }
        float top = 0.f;
        bool fin = true;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          top = fmaxf(top, fabsf(x[e]));
          fin = fin && fabsf(x[e]) < INFINITY;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        fin = __all_sync(0xffffffffu, fin);
        const int e2 = fin ? max(static_cast<int>(__float_as_uint(top) >> 23) - 127 - 7, -110) : 0;   // top 2^-e2 in [128, 256)
        const float inv = __uint_as_float(static_cast<uint32_t>(127 - e2) << 23);
        uint32_t hi = 0x7F7F7F7Fu, lo = 0;      // a row that is not finite: NaN throughout
        if (fin) {
          float y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int e = 0; e < E; ++e) y[e] = x[e] * inv;
          hi = e4m3x4(y[0], y[1], y[2], y[3]);
          const uint32_t f0 = e4m3x2_to_f16x2(hi & 0xFFFFu), f1 = e4m3x2_to_f16x2(hi >> 16);
          const float2 g0 = __half22float2(*reinterpret_cast<const __half2*>(&f0)), g1 = __half22float2(*reinterpret_cast<const __half2*>(&f1));
          lo = e4m3x4((y[0] - g0.x) * 16.f, (y[1] - g0.y) * 16.f, (y[2] - g1.x) * 16.f, (y[3] - g1.y) * 16.f);
        }
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          const int row = part * NQ + q, byte = lane * E, chunk = byte / 16 ^ (D == 128 ? row & 7 : (row >> 1) & 3);
          uint8_t* dst = sQ + row * D + chunk * 16 + byte % 16;
          if constexpr (E == 4) *reinterpret_cast<uint32_t*>(dst) = part ? lo : hi;
          else *reinterpret_cast<uint16_t*>(dst) = static_cast<uint16_t>(part ? lo : hi);
        }
        if (lane == 0) {
          const bool real = q < it.rows;
          ctl->qc[q] = real ? a.scale2 * __uint_as_float(static_cast<uint32_t>(127 + e2) << 23) : 0.f;
          ctl->slot_of[q] = real ? it.p0 + static_cast<int>(a.by_group(it.row0 + q)) : -1;
          // (rows past the item score 0 and must not ask for anything)
          ctl->stat[0][q] = ctl->stat[1][q] = real ? Stat{kNone, kNone, kNone, 0.f} : Stat{-kNone, -kNone, -kNone, 0.f};
        }
      }
      fence_proxy_async_shared();
      __syncwarp();
      if (lane == 0) mbar_arrive(q_full);
      named_barrier_sync(3, 256);
      float l[NQ];
#pragma unroll
      for (int q = 0; q < NQ; ++q) l[q] = 0.f;
#pragma unroll 1
      for (int i = it.t0 + ((t ^ grp) & 1); i < it.t1; i += 2) {      // the tiles whose number in the CTA's order is the group's, modulo 2
        const int u = t + i - it.t0, s = u % ST, p = u & 3;
        const bool begun = i >= it.t0 + 2;
        const int slot0 = it.span.tile(i) * kKvTile, slot = slot0 + me;
        bool ok = kv_wait(full(s), (u / ST) & 1);        // the tile's scales (and V, below)
        ok = __all_sync(0xffffffffu, ok && kv_wait(s_full(p), (u >> 2) & 1));
        if (!ok) {
          if (lane == 0) stop(&ctl->abort, status);
          bad = true;
        }
        tc_fence_after_sync();
        // every row sees the whole tile?
        const bool whole = slot0 + kKvTile - 1 <= it.p_first &&
                           (a.window <= 0 || slot0 > it.p_last - a.window || slot0 + kKvTile <= a.sinks);
        float ks = ctl->scales[s][me >> 4], vs = ctl->scales[s][8 + (me >> 4)];
        float x[NQ];
        {
          uint32_t sv[C::COLS];
          load_cols(lanes + p * C::COLS, sv);
          bool any = whole;
          if (!whole) {
#pragma unroll
            for (int q = 0; q < NQ; ++q) any = any || kv_sees(slot, ctl->slot_of[q], a.window, a.sinks);
            if (!any) ks = vs = 0.f;     // (what is there may be NaN)
            // 0 * NaN is NaN: a slot of V that some row does not see must not hold one.  Slots that nobody sees are
            // cleared; where rows differ, a slot with a NaN code is cleared and those that see it get a NaN weight.
            uint4* v = reinterpret_cast<uint4*>(sKV + (2 * s + 1) * C::TILE + me * D);
            bool nan = false;
            if (any) {
#pragma unroll
              for (int e = 0; e < D / 16; ++e) {
                const uint4 u = v[e ^ (me & (D / 16 - 1))];      // (any order: lanes side by side would meet in one bank)
                const uint32_t w = (((u.x & 0x7F7F7F7Fu) + 0x01010101u) | ((u.y & 0x7F7F7F7Fu) + 0x01010101u) | ((u.z & 0x7F7F7F7Fu) + 0x01010101u) |
                                    ((u.w & 0x7F7F7F7Fu) + 0x01010101u)) & 0x80808080u;
                nan = nan || w != 0;
              }
            }
            if (!any || nan) {
#pragma unroll
              for (int e = 0; e < D / 16; ++e) v[e ^ (me & (D / 16 - 1))] = make_uint4(0, 0, 0, 0);
            }
            if (nan) vs = NAN;
          }
          if (vs != vs) ks = vs;      // (by way of its score: the products below drop a NaN scale)
#pragma unroll
          for (int q = 0; q < NQ; ++q) {
            x[q] = fmaf(__uint_as_float(sv[NQ + q]), 0.0625f, __uint_as_float(sv[q])) * (ks * ctl->qc[q]);
            if (!whole && !kv_sees(slot, ctl->slot_of[q], a.window, a.sinks)) x[q] = -INFINITY;
          }
        }
        const float lv = static_cast<float>(static_cast<int>(__float_as_uint(vs) >> 23) - 127);   // log2(vs), far down for 0
        bool ask = bad;
#pragma unroll
        for (int q = 0; q < NQ; ++q) ask = ask || x[q] - stat[q].m > fminf(kFar, stat[q].over - lv);
        if (named_barrier_any(1 + grp, 128, ask)) {
          // some row's m or r has to move: the tile's maxima over all slots (a warp's second one relative to its first), new values,
          // factors for l and O
#pragma unroll
          for (int q = 0; q < NQ; ++q) {
            const float mx = fmaxf(warp_max(x[q]), kNone), mw = warp_max(x[q] - mx + lv);
            if (lane == 0) ctl->red[grp][quad][q] = make_float2(mx, mw);
          }
          named_barrier_sync(1 + grp, 128);
          if (me < NQ) {
            const Stat st = stat[me];
            float mx = kNone;
#pragma unroll
            for (int w = 0; w < 4; ++w) mx = fmaxf(mx, ctl->red[grp][w][me].x);
            auto weighted = [&](float base) {      // largest x + log2(vs) of the tile, less base
              float r = -INFINITY;
#pragma unroll
              for (int w = 0; w < 4; ++w) r = fmaxf(r, ctl->red[grp][w][me].x - base + ctl->red[grp][w][me].y);
              return r;
            };
            const bool move = mx - st.m > kFar || weighted(st.m) > st.over;     // (each row by itself)
            float2 fac = make_float2(1.f, 1.f);
            if (move) {
              const float m = fmaxf(st.m, mx), r = fmaxf(st.m - m + st.r, weighted(m));
              fac = make_float2(exp2f(st.m - m), exp2f((st.m - m) + (st.r - r)));
              stat[me] = Stat{m, r, r + kOver, exp2f(kUnit - r)};
            }
            ctl->fac[grp][me] = fac;
          }
          if (begun && !kv_wait(pv_done((u - 2) & 3), ((u - 2) >> 2) & 1)) stop(&ctl->abort, status);
          named_barrier_sync(1 + grp, 128);
          bad = named_barrier_any(1 + grp, 128, stopped(&ctl->abort));
          if (bad) break;
#pragma unroll
          for (int q = 0; q < NQ; ++q) l[q] *= ctl->fac[grp][q].x;
          if (begun) {
            tc_fence_after_sync();
#pragma unroll 1
            for (int c = 0; c < C::OCOLS; c += 16) {
              uint32_t o[16];
              load_cols(lanes + C::O_AT + grp * C::OCOLS + c, o);
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * ctl->fac[grp][(c + e) % NQ].y);
              tmem_st_32x32b(lanes + C::O_AT + grp * C::OCOLS + c, o);
            }
            tmem_wait_st();
          }
        }
        // weights, and P as hi and lo codes, in the columns of its size: 16 columns of this slot at a time
        uint32_t w[4 * NQ / 4];
#pragma unroll
        for (int q = 0; q < NQ; q += 4) {
          float y[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float pr = ex2_approx(x[q + e] - stat[q + e].m);
            l[q + e] += pr;
            y[e] = pr * fminf(vs * stat[q + e].g, 0x1p100f);      // (the bound: pr is 0 or all but 0 there, and 0 times infinity)
          }
          uint32_t small = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (y[e] < kSmall) {
              y[e] *= kTimes;
              small |= 0xFFu << 8 * e;
            }
          }
          const uint32_t hi = e4m3x4(y[0], y[1], y[2], y[3]);
          const uint32_t f0 = e4m3x2_to_f16x2(hi & 0xFFFFu), f1 = e4m3x2_to_f16x2(hi >> 16);
          const float2 g0 = __half22float2(*reinterpret_cast<const __half2*>(&f0)), g1 = __half22float2(*reinterpret_cast<const __half2*>(&f1));
          const uint32_t lo = e4m3x4((y[0] - g0.x) * 16.f, (y[1] - g0.y) * 16.f, (y[2] - g1.x) * 16.f, (y[3] - g1.y) * 16.f);
          w[q / 4] = hi & ~small;
          w[NQ / 4 + q / 4] = lo & ~small;
          w[2 * NQ / 4 + q / 4] = hi & small;
          w[3 * NQ / 4 + q / 4] = lo & small;
        }
        uint8_t* dst = sP + p * C::PBYTES + me * 16;
#pragma unroll
        for (int c = 0; c < C::OCOLS / 16; ++c)
          *reinterpret_cast<uint4*>(dst + c * 16 * kKvTile) = make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
        fence_proxy_async_shared();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full(p));
      }
      // ---- the item's (part of the) output, joined from the groups' ---------------------------
      t += it.t1 - it.t0;
      const int last = t - 1 - ((t - 1 ^ grp) & 1);      // the group's last tile (not of this item, if it had none)
      if (!bad && last >= t - (it.t1 - it.t0) && !kv_wait(pv_done(last & 3), (last >> 2) & 1)) stop(&ctl->abort, status);
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        float v = l[q];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (lane == 0) ctl->red[grp][quad][q].x = v;
      }
      if (named_barrier_any(3, 256, bad || stopped(&ctl->abort))) break;
      const bool complete = it.t0 == 0 && it.t1 == it.span.n;
      const int64_t slot = (2 * static_cast<int64_t>(blockIdx.x) + (it.t0 == 0 ? 1 : 0)) * NQ;
      if (me < it.rows) {
        float l2[2], m = kNone;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          l2[k] = (ctl->red[k][0][me].x + ctl->red[k][1][me].x) + (ctl->red[k][2][me].x + ctl->red[k][3][me].x);
          if (l2[k] != 0.f) m = fmaxf(m, ctl->stat[k][me].m);      // (a group that saw nothing has no say)
        }
        const float f0 = l2[0] == 0.f ? 0.f : exp2f(ctl->stat[0][me].m - m), f1 = l2[1] == 0.f ? 0.f : exp2f(ctl->stat[1][me].m - m);
        const float sum = l2[0] * f0 + l2[1] * f1;
        const float f = grp == 0 ? f0 : f1;
        // out = sum over the groups of O f / (g sum); 0 says that the group saw nothing (else O counts however small f is: it may be NaN)
        float by = f / (stat[me].g * sum);
        if (by == 0.f) by = 1e-37f;
        ctl->fac[grp][me].x = (grp == 0 ? l2[0] : l2[1]) == 0.f ? 0.f : by;
        if (grp == 0) {
          const int64_t at = complete ? kv_out_row(a, it, me) : slot + me;
          ctl->out_at[me] = at * D;
          const float rel = sum == 0.f ? -INFINITY : log2f(sum);
          if (!complete) a.part_lse[at] = make_float2(m, rel);
          else if (a.lse != nullptr) a.lse[at] = (m + rel) * 0.69314718055994531f;
        }
      }
      named_barrier_sync(1 + grp, 128);
      tc_fence_after_sync();
      float v[NQ];
#pragma unroll
      for (int q = 0; q < NQ; ++q) v[q] = 0.f;
#pragma unroll
      for (int c = 0; c < C::OCOLS; c += 16) {
        uint32_t o[16];
        load_cols(lanes + C::O_AT + grp * C::OCOLS + c, o);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          constexpr float unit[4] = {1.f, 0.0625f, 1.f / kTimes, 0.0625f / kTimes};
          v[(c + e) % NQ] = fmaf(__uint_as_float(o[e]), unit[(c + e) / NQ], v[(c + e) % NQ]);
        }
      }
      tc_fence_before_sync();
      // each group ends half of the rows, with the other's sums by way of P's places (all products have completed)
      float* join = reinterpret_cast<float*>(sP);
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const float f = ctl->fac[grp][q].x;
        v[q] = f == 0.f ? 0.f : v[q] * f;
        if (q / (NQ / 2) != grp && q < it.rows && me < D) join[q * D + me] = v[q];
      }
      named_barrier_sync(3, 256);
      if (me < D) {
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          if (q / (NQ / 2) != grp || q >= it.rows) continue;
          const float sum = v[q] + join[q * D + me];
          if (complete) a.out[ctl->out_at[q] + me] = __bfloat16_as_ushort(__float2bfloat16_rn(sum));
          else a.part[ctl->out_at[q] + me] = sum;
        }
      }
    }
    if (threadIdx.x == 64) kv_write_split(a, share, walk.it);
  }
  // everything issued has completed: the last tile's commit has been waited for, unless the CTA gave up
  tc_fence_before_sync();
  __syncthreads();
  if (stopped(&ctl->abort)) {
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 100000ull) {
    }
    __syncthreads();
  }
  tc_fence_after_sync();
  if (warp == 1) tmem_dealloc(tmem, C::TMEM);
}

// The items that several CTAs walked: out = sum_c 2^(lse_c - max) o_c / sum_c 2^(lse_c - max), parts in a fixed order; lse_c = b_c + r_c,
// and differences are of b by itself first, which leaves them exact where the scores b are close.  What it
// takes is latency, so a warp's loads go out together, PARTS parts of ROWS rows at a time.  Where rows are few a row has 8 warps (a
// sequence alone makes as many parts as there are tiles: 38 of them took 8 us with one warp); where they are many and a row has few
// parts, a warp has 4 rows (2 us less in a call of 517 tokens than with one row).
template <int D, int ROWS, int PARTS, int SPLIT>
__global__ void __launch_bounds__(256) kv_attn_combine(const __grid_constant__ KvAttnArgs a, int tile_rows) {
  constexpr int E = D / 32;      // elements of a lane
  static_assert(ROWS == 1 || SPLIT == 1, "a warp has several rows or a row several warps");
  __shared__ float s_base[8], s_top[8], s_sum[8];
  __shared__ __align__(16) float s_o[SPLIT > 1 ? 8 : 1][D];
  launch_dependents();
  grid_dependency_wait();
  const int c = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int4 raw = __ldcg(reinterpret_cast<const int4*>(a.split + c));
  const KvSplit sp{raw.x, raw.y, raw.z, raw.w};
  if (sp.followers == 0) return;
  const int q0 = (blockIdx.y * (8 / SPLIT) + warp / SPLIT) * ROWS;
  const int live = min(ROWS, a.s.nq[sp.i] * a.group - sp.row_tile * tile_rows - q0);      // rows of this warp
  if (live <= 0) return;      // (a row's warps all)
  auto at = [&](int j, int r) { return static_cast<int64_t>(j == 0 ? 2 * c + 1 : 2 * (c + j)) * tile_rows + q0 + r; };
  const int parts = sp.followers + 1;
  // of row lane / PARTS (the same in its PARTS lanes): the largest b, the largest lse relative to it, the sum; of every row o
  float base = -INFINITY, top = -INFINITY, sum = 0.f, o[ROWS][E];
  auto finite = [](float x) { return x == -INFINITY ? 0.f : x; };      // (where nothing was seen: 2^(-inf - 0), no NaN)
#pragma unroll
  for (int r = 0; r < ROWS; ++r)
#pragma unroll
    for (int e = 0; e < E; ++e) o[r][e] = 0.f;
#pragma unroll 1
  for (int j0 = warp % SPLIT; j0 < parts; j0 += PARTS * SPLIT) {      // parts j0, j0 + SPLIT, ...
    const int j_mine = j0 + lane % PARTS * SPLIT, r_mine = lane / PARTS;
    float2 lse = make_float2(-INFINITY, -INFINITY);
    if (j_mine < parts && r_mine < live) lse = __ldcg(a.part_lse + at(j_mine, r_mine));
    if (lse.y == -INFINITY) lse.x = -INFINITY;
    float v[ROWS][PARTS][E];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
      for (int k = 0; k < PARTS; ++k) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[r][k][e] = 0.f;
        if (j0 + k * SPLIT >= parts || r >= live) continue;
        const float* p = a.part + at(j0 + k * SPLIT, r) * D + lane * E;
        if constexpr (E == 4) {
          const float4 u = __ldcg(reinterpret_cast<const float4*>(p));
          v[r][k][0] = u.x;
          v[r][k][1] = u.y;
          v[r][k][2] = u.z;
          v[r][k][3] = u.w;
        } else {
          const float2 u = __ldcg(reinterpret_cast<const float2*>(p));
          v[r][k][0] = u.x;
          v[r][k][1] = u.y;
        }
      }
    float b = fmaxf(lse.x, base);
#pragma unroll
    for (int s = PARTS / 2; s > 0; s >>= 1) b = fmaxf(b, __shfl_xor_sync(0xffffffffu, b, s));
    const float rel = lse.x - finite(b) + lse.y, was = base - finite(b) + top;
    float now = fmaxf(rel, was);
#pragma unroll
    for (int s = PARTS / 2; s > 0; s >>= 1) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, s));
    const float f = exp2f(was - finite(now)), mine = exp2f(rel - finite(now));
    base = b;
    top = now;
    sum *= f;
    float all = mine;
#pragma unroll
    for (int s = PARTS / 2; s > 0; s >>= 1) all += __shfl_xor_sync(0xffffffffu, all, s);
    sum += all;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const float fr = __shfl_sync(0xffffffffu, f, r * PARTS);
#pragma unroll
      for (int e = 0; e < E; ++e) o[r][e] *= fr;
#pragma unroll
      for (int k = 0; k < PARTS; ++k) {
        const float w = __shfl_sync(0xffffffffu, mine, r * PARTS + k);
#pragma unroll
        for (int e = 0; e < E; ++e) o[r][e] = fmaf(w, v[r][k][e], o[r][e]);
      }
    }
  }
  if constexpr (SPLIT > 1) {
    if (lane == 0) {
      s_base[warp] = base;
      s_top[warp] = top;
      s_sum[warp] = sum;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) s_o[warp][lane * E + e] = o[0][e];
    __syncthreads();
    if (warp > 0) return;
    base = s_base[0];
#pragma unroll
    for (int k = 1; k < SPLIT; ++k) base = fmaxf(base, s_base[k]);
    top = -INFINITY;
#pragma unroll
    for (int k = 0; k < SPLIT; ++k) top = fmaxf(top, s_base[k] - finite(base) + s_top[k]);
    sum = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) o[0][e] = 0.f;
#pragma unroll
    for (int k = 0; k < SPLIT; ++k) {
      const float f = exp2f(s_base[k] - finite(base) + s_top[k] - finite(top));
      sum = fmaf(f, s_sum[k], sum);
#pragma unroll
      for (int e = 0; e < E; ++e) o[0][e] = fmaf(f, s_o[k][lane * E + e], o[0][e]);
    }
  }
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    if (r >= live) break;
    const float s = __shfl_sync(0xffffffffu, sum, r * PARTS), m = __shfl_sync(0xffffffffu, base + top, r * PARTS);
    const float inv = s == 0.f ? 0.f : 1.f / s;
    const int row = sp.row_tile * tile_rows + q0 + r, token = static_cast<int>(a.by_group(row));
    const int64_t dst = static_cast<int64_t>(a.s.q0[sp.i] + token) * a.q_heads + sp.head * a.group + row - token * a.group;
    uint32_t w[E / 2];
#pragma unroll
    for (int e = 0; e < E / 2; ++e)
      w[e] = static_cast<uint32_t>(__bfloat16_as_ushort(__float2bfloat16_rn(o[r][2 * e] * inv))) |
             static_cast<uint32_t>(__bfloat16_as_ushort(__float2bfloat16_rn(o[r][2 * e + 1] * inv))) << 16;
    if constexpr (E == 4) *reinterpret_cast<uint2*>(a.out + dst * D + lane * E) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(a.out + dst * D + lane * E) = w[0];
    if (lane == 0 && a.lse != nullptr) a.lse[dst] = s == 0.f ? -INFINITY : (m + log2f(s)) * 0.69314718055994531f;
  }
}

template <int D, int NQ>
pace_status_t run_decode(const KvMaps& maps, const KvAttnArgs& a, unsigned grid, int* status, cudaStream_t stream) {
  using C = DecodeCfg<D, NQ>;
  constexpr size_t smem = 1024 + C::STAGES * 2 * C::TILE + C::QBYTES + 4 * C::PBYTES + sizeof(DecodeCtl<D, NQ>);
  static_assert(smem <= 227 * 1024, "shared memory");
  static DeviceOnce once;
  int dev = 0;
  PACE_CUDA(cudaGetDevice(&dev));
  if (!once.done(dev)) {
    PACE_CUDA(cudaFuncSetAttribute(kv_decode_kernel<D, NQ>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
    once.mark(dev);
  }
  return launch_dependent(kv_decode_kernel<D, NQ>, grid, kThreads, smem, 1, stream, maps, a, status);
}

}  // namespace

pace_status_t launch_kv_decode(const KvMaps& maps, const KvAttnArgs& a, int D, int rows, unsigned grid, int* status, cudaStream_t stream) {
  if (D == 128)
    return rows == 8 ? run_decode<128, 8>(maps, a, grid, status, stream) : rows == 16 ? run_decode<128, 16>(maps, a, grid, status, stream)
                                                                                   : run_decode<128, 32>(maps, a, grid, status, stream);
  return rows == 8 ? run_decode<64, 8>(maps, a, grid, status, stream) : rows == 16 ? run_decode<64, 16>(maps, a, grid, status, stream)
                                                                                 : run_decode<64, 32>(maps, a, grid, status, stream);
}

pace_status_t launch_kv_combine(const KvAttnArgs& a, int D, int rows, unsigned grid, cudaStream_t stream) {
  if (rows == kManyRows)
    return launch_dependent(D == 128 ? kv_attn_combine<128, 4, 4, 1> : kv_attn_combine<64, 4, 4, 1>, dim3(grid, static_cast<unsigned>(rows / 32)),
                            256, 0, 1, stream, a, rows);
  return launch_dependent(D == 128 ? kv_attn_combine<128, 1, 8, 8> : kv_attn_combine<64, 1, 8, 8>, dim3(grid, static_cast<unsigned>(rows)), 256, 0, 1,
                          stream, a, rows);
}

}  // namespace pace
