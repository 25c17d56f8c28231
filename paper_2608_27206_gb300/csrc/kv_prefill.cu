// Serve: attention over the paged cache for many query rows per KV head (prefill, whole or in chunks).
//
//   S [128 rows x 128 slots] = q K^T        O [128 rows x D] += P V
// S is formed in 8 bits: K as the codes it is stored as, bf16 q as an e4m3 term and an e5m2 term for what is left of it.  Each row is
// first brought under 256 by a power of two, to 128 at least; of an element of 2^-6 or more the first term then takes 4 of its 8
// significant bits, what is left are 8 units of its last bit at most, and e5m2 holds that exactly (3 significant bits, down to 2^-16; e4m3,
// which ends at 2^-9, would lose bits from 2^-3 on).  Smaller elements, those under 2^-13 of the row's largest, are off by 2^-14 at most, 2^-21 of
// it.  Two 8-bit products cost what one of 16 bits would, at half the shared memory and with no work on K.  P V is formed in f16,
// which holds every e4m3 number, and a weight to 11 bits.
//
// A TMEM lane of S is a query row and one thread's.  With x the score in base 2 and vs the V scale of a slot's block, the row's
// weights are P = 2^(x + log2(vs) - w) and l = sum P / vs; both scales are constants of 16 columns, so a weight costs
// one multiply-add, one exponential, one addition and half a conversion.  w is a whole number, the maximum of the row's first
// 64 slots rounded up, and then stays: f16 has room for weights up to 2^15 above it, and below it 14 binary orders keep all their bits
// and what is lost is under 2^-25.  Only when the weights of 64 columns sum up to more does w move, and O, l and the tile's weights so
// far with it, to where that sum is 2^5 to 2^6: then, as at first, the largest weight is 1/2 at least, and what is lost under 2^-24 of it.
// (Down to a sum of 1 a row would move less often, but 64 equal weights would be 2^-6 each: a call of 517 tokens 98-100 us, so 101-102; with the
// largest weight at 2^4 instead it would be 108.)  There is no maximum in the common path.  (Weights of blocks whose V scale is below
// 2^-110 of the largest are lost to l.)
//
// The tensor pipe needs 2048 clocks per slot tile of 2 x 128 rows at D = 128 (1024 at D = 64), the exponentials 1024 at either, and in a
// long prompt a slot tile takes 4060 all told: what bounds it is the chain from S to P to P V, 50 % tensor active (a call of 517 tokens
// 43 %, prompts of D = 64 with a window 18 %, where items are short and change often).  Two row tiles A and B share every K and V tile (a V
// tile turned into f16 once for both) and take turns: while one's weights are worked out, the other's products run.  P overwrites its
// S in TMEM.  Measured: a prompt of 10825 tokens, 28 + 4 heads of 128: 815-830 us, 1.01-1.03 PFLOP/s; 517 tokens at the end of 11342:
// 102 us.  Tried and slower, when these were 790-815 and 97: S by halves of 64 columns (A is read twice as often: 844 us), two threads per
// row on four warps per scheduler (908), a warp of MMAs per row tile (872), a single row tile with S ahead (1013; the short call 89).
//
// Nodes of trees (TREE) have few rows to an item, so that a slot tile is bound by the chain alone; what differs for them:
//   S of the next slot tile is formed half by half, each as soon as P of that half has been used up (q crosses shared memory twice as often,
//   but a half's owners find the next one ready: 40 trees of 182 rows on 5001-28007 slots 257 us with S whole, 238 by halves);
//   of an item of one row tile and kPairTiles slot tiles or more, A and B take every other slot tile and join at the end (64 such trees
//   of 63 rows 278 us with B idle, 220); K and V tiles then share one ring, as S runs two tiles ahead;
//   parts of full tiles go out by way of shared memory, and warps without rows only keep step.
// Measured: those 40 trees 233 us, 855 TFLOP/s and 2.4 TB/s; 64 of 63 rows 220 us, 4.0 TB/s.  In the former a slot tile takes 3600 clocks, 2600 of
// them shared memory's (S by halves 1540, P V 510, V's conversion and the fetch 640), the rest hand-overs from P to products to S; tensor pipe
// 52 % active.  One item alone costs 20000 clocks besides its tiles: the plan 4000, q 4500-7000, its first tile 1500 more, its output 2500-6000.
// Tried: A's two halves before B's (250 us instead of 238), a pair's halves in step instead of in turn (275 instead of 235).
// Roles of a CTA (one per SM): warp 0 fetches, warp 1 issues the MMAs, warps 2-3 turn V into f16 (they also see to NaN that must
// not reach rows that do not look at it), warps 4-7 and 8-11 own the rows of A and B.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "kv_attn.cuh"

namespace pace {
namespace {

using namespace ptx;

constexpr int kThreads = 384;
constexpr int kHalf = 64;          // columns of S at a time
constexpr float kMost = 32768.f;   // sum of 64 weights at which w moves
constexpr int kAfter = 6;          // log2 of what that sum is when w has moved, at most (so the largest weight is 2^-1 at least)
constexpr float kFar = 0x1p22f;    // a row's maximum from which on its scores are taken relative to one of them; of trees, whose halves and parts are
constexpr float kTreeFar = 0x1p12f;      // more often joined where one is past it and the other not: a score rounded there is 2^-12 off, at 2^22 a quarter
constexpr uint32_t kTmem = 512;    // S of A and B, then O of A and B, 128 columns each

template <int D>
struct PrefillCfg {
  static constexpr int TILE = kKvTile * D;
  static constexpr int STAGES = D == 128 ? 3 : 6;       // places of K tiles,
  static constexpr int VSTAGES = D == 128 ? 2 : 4;      // of V tiles
  static constexpr int QTILE = 128 * D;                 // hi or lo codes of a row tile
  static constexpr int VCHUNK = kKvTile * 128;          // f16 V: 64 columns of every slot, 128 bytes each
  static constexpr int VTILE = VCHUNK * D / 64;
  static constexpr uint32_t SWIZZLE = D == 128 ? 2 : 4;
  static constexpr uint32_t GROUP = 8 * D;
  static constexpr uint32_t IDESC_HI = idesc_e4m3_f32(128, kKvTile, false, false), IDESC_LO = idesc_e4m3_f32(128, kKvTile, false, false, true);
  static constexpr uint32_t HALF_HI = idesc_e4m3_f32(128, kHalf, false, false), HALF_LO = idesc_e4m3_f32(128, kHalf, false, false, true);
  static constexpr uint32_t IDESC_O = idesc_f16_mn_f32(128, D);
};

template <int D>
struct alignas(16) PrefillCtl {
  static constexpr int ST = PrefillCfg<D>::STAGES, SV = PrefillCfg<D>::VSTAGES;
  uint64_t full[ST], empty[ST + SV], v_empty[SV], known[4], ready[2], vfree[2], s_full[2][2], p_full[2][2], q_full[2], o_done[2][2], x_full[2], x_read[2];
  float scales[ST][16];
  float4 block[4][8];           // of the last tiles, per block of 16 slots: K scale, log2(V scale), 1 / V scale
  uint32_t nan[2][4];           // slots of which some row sees a NaN value
  float4 state[2][128];         // of the rows of a pair's halves: m, w, l, far
  int scan[2 * kThreads / 32];
  KvShare share;
  uint32_t tmem;
  int abort;
};

// A tile that rows at slots up to p_last, which see every slot up to p_all but for the window, all see whole.
__device__ __forceinline__ bool kv_whole(int slot0, int p_all, int p_last, int window, int sinks) {
  return slot0 + kKvTile - 1 <= p_all && (window <= 0 || slot0 > p_last - window || slot0 + kKvTile <= sinks);
}

// Of a tree: whether A and B take every other slot tile of an item that has one row tile.  (Joining them costs what two or three slot tiles
// take: with 4 for 8, 32 trees of 128 rows on 700-9000 slots 112 us instead of 108; with 16, 64 of dim 64 110 instead of 105.)
constexpr int kPairTiles = 8;
template <bool TREE>
__device__ __forceinline__ bool kv_pair(const KvItem& it) { return TREE && it.rows <= 128 && it.t1 - it.t0 >= kPairTiles; }

__device__ __forceinline__ uint32_t f16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// Two bf16 times a power of two, as f16.
__device__ __forceinline__ uint32_t pair_f16(uint32_t two, float by) {
  return f16x2(__uint_as_float(two << 16) * by, __uint_as_float(two & 0xFFFF0000u) * by);
}
// Four f16 as two terms: e4m3, and what is left of them in e5m2.
__device__ __forceinline__ void split_8bit(uint32_t a, uint32_t b, uint32_t& hi, uint32_t& lo) {
  auto code = [](uint32_t two) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(two));
    return static_cast<uint32_t>(r);
  };
  auto rest = [](uint32_t two, uint32_t codes) {
    uint32_t d;
    uint16_t r;
    asm("sub.f16x2 %0, %1, %2;" : "=r"(d) : "r"(two), "r"(e4m3x2_to_f16x2(codes)));
    asm("cvt.rn.satfinite.e5m2x2.f16x2 %0, %1;" : "=h"(r) : "r"(d));
    return static_cast<uint32_t>(r);
  };
  const uint32_t ca = code(a), cb = code(b);
  hi = ca | cb << 16;
  lo = rest(a, ca) | rest(b, cb) << 16;
}

template <int D, bool TREE>
__global__ void __launch_bounds__(kThreads, 1) kv_prefill_kernel(const __grid_constant__ KvMaps maps, const __grid_constant__ KvAttnArgs a,
                                                                 int* status) {
  using C = PrefillCfg<D>;
  constexpr int ST = C::STAGES, PLACES = ST + C::VSTAGES;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sK = smem;                              // K tiles, as codes
  uint8_t* sC = sK + ST * C::TILE;                 // V tiles, as codes
  uint8_t* sV = sC + C::VSTAGES * C::TILE;         // two V tiles in f16
  uint8_t* sQ = sV + 2 * C::VTILE;                 // A hi, A lo, B hi, B lo
  auto* ctl = reinterpret_cast<PrefillCtl<D>*>(sQ + 4 * C::QTILE);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto full = [&](int s) { return smem_u32(&ctl->full[s]); };
  auto empty = [&](int s) { return smem_u32(&ctl->empty[s]); };
  auto known = [&](int b) { return smem_u32(&ctl->known[b]); };
  auto ready = [&](int b) { return smem_u32(&ctl->ready[b]); };
  auto vfree = [&](int b) { return smem_u32(&ctl->vfree[b]); };
  auto s_full = [&](int i, int h) { return smem_u32(&ctl->s_full[i][h]); };
  auto p_full = [&](int i, int h) { return smem_u32(&ctl->p_full[i][h]); };
  auto q_full = [&](int i) { return smem_u32(&ctl->q_full[i]); };
  auto o_done = [&](int i, int h) { return smem_u32(&ctl->o_done[i][h]); };
  auto x_full = [&](int i) { return smem_u32(&ctl->x_full[i]); };
  auto x_read = [&](int i) { return smem_u32(&ctl->x_read[i]); };

  kv_begin<TREE>(a);
  const KvShare share = kv_share<kManyRows, D, TREE>(a, ctl->scan, &ctl->share, status);
  if (static_cast<int>(blockIdx.x) >= share.ctas) {
    kv_tree_ready<TREE>(a);      // (a launch does not end before the one that it follows)
    if (threadIdx.x == 0) a.split[blockIdx.x] = KvSplit{0, 0, 0, 0};
    return;
  }
  if (warp == 0 && lane == 0) {
    prefetch_tensormap(&maps.k);
    prefetch_tensormap(&maps.v);
    for (int s = 0; s < ST; ++s) mbar_init(full(s), 33);
    for (int s = 0; s < (TREE ? PLACES : ST); ++s) mbar_init(empty(s), TREE ? 2 : 1);
    for (int s = 0; s < C::VSTAGES; ++s) mbar_init(smem_u32(&ctl->v_empty[s]), 2);
    for (int b = 0; b < 4; ++b) mbar_init(known(b), 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(ready(i), 2);
      mbar_init(vfree(i), 1);
      for (int h = 0; h < 2; ++h) {
        mbar_init(s_full(i, h), 1);
        mbar_init(p_full(i, h), 4);
        mbar_init(o_done(i, h), 1);
      }
      mbar_init(q_full(i), 4);
      mbar_init(x_full(i), 4);
      mbar_init(x_read(i), 4);
    }
    fence_mbar_init();
    ctl->abort = 0;
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(&ctl->tmem), kTmem);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = ctl->tmem;

  if (warp == 0) {
    KvWalk<kManyRows, TREE> walk;
    walk.begin(share);
    kv_fetch<D, ST, C::VSTAGES, TREE>(maps, a, walk, KvRings{sK, sC, C::TILE, ctl->full, ctl->empty, ctl->v_empty, ctl->scales}, &ctl->abort, status);
  } else if (warp == 1) {
    // ---- products: P V of a slot tile, half by half as the weights come, then S of the next; A and B in turn ----------
    // The warp stays converged: operands of these instructions are registers of the whole warp, and in one lane's branch each took 80
    // clocks.
    KvWalk<kManyRows, TREE> walk;
    walk.begin(share);
    const KvItem& it = walk.it;
    const uint32_t issue = elect_one();
    const uint64_t dq = smem_desc(smem_u32(sQ), 16, C::GROUP, C::SWIZZLE);
    const uint64_t dk = smem_desc(smem_u32(sK), 16, C::GROUP, C::SWIZZLE);
    const uint64_t dv = smem_desc(smem_u32(sV), C::VCHUNK, 1024, 2);
    int t = 0, done_a = 0, done_b = 0, items_a = 0, items_b = 0;      // slot tiles; of a row tile: slot tiles, items
    bool ok = true;
    auto wait = [&](uint32_t bar, int round) {
      ok = kv_wait_warp(bar, round & 1);
      return ok;
    };
    auto commit = [&](uint32_t bar) {
      if (issue) mma_commit(bar);
    };
    auto release = [&](int u) {      // the place of K of slot tile u
      if constexpr (TREE) {
        commit(empty(2 * u % PLACES));
        commit(empty(2 * u % PLACES));
      } else {
        commit(empty(u % ST));
      }
    };
    auto scores = [&](int i, int u) {      // S of slot tile u
      const uint64_t q = dq + static_cast<uint64_t>(i * 2 * (C::QTILE >> 4));
      const uint64_t k0 = dk + static_cast<uint64_t>((TREE ? 2 * u % PLACES : u % ST) * (C::TILE >> 4));
#pragma unroll
      for (int part = 0; part < 2; ++part)
#pragma unroll
        for (int k = 0; k < D / 32; ++k)
          mma_f8_ss(tmem + i * 128, q + static_cast<uint64_t>(part * (C::QTILE >> 4) + 2 * k), k0 + static_cast<uint64_t>(2 * k),
                    part == 0 ? C::IDESC_HI : C::IDESC_LO, part > 0 || k > 0, issue);
      commit(s_full(i, 0));
    };
    auto half_scores = [&](int i, int h, int u) {      // 64 columns of it
      const uint64_t q = dq + static_cast<uint64_t>(i * 2 * (C::QTILE >> 4));
      const uint64_t k0 = dk + static_cast<uint64_t>((TREE ? 2 * u % PLACES : u % ST) * (C::TILE >> 4) + h * (kHalf * D >> 4));
#pragma unroll
      for (int part = 0; part < 2; ++part)
#pragma unroll
        for (int k = 0; k < D / 32; ++k)
          mma_f8_ss(tmem + i * 128 + h * kHalf, q + static_cast<uint64_t>(part * (C::QTILE >> 4) + 2 * k), k0 + static_cast<uint64_t>(2 * k),
                    part == 0 ? C::HALF_HI : C::HALF_LO, part > 0 || k > 0, issue);
      commit(s_full(i, h));
    };
    auto both_scores = [&](int i, int u) {      // whole, for owners who wait for halves
      scores(i, u);
      commit(s_full(i, 1));
    };
    auto weigh = [&](int i, int h, int u, int round, bool first) {      // O += P V of half a slot tile
      if (!wait(p_full(i, h), round)) return;
      tc_fence_after_sync();
      const uint64_t v = dv + static_cast<uint64_t>((u & 1) * (C::VTILE >> 4));
#pragma unroll
      for (int k = 0; k < kHalf / 16; ++k)
        mma_f16_ts(tmem + 256 + i * 128, tmem + i * 128 + h * kHalf + k * 8, v + static_cast<uint64_t>((h * 4 + k) * (2048 >> 4)), C::IDESC_O,
                   !first || h > 0 || k > 0, issue);
      commit(o_done(i, h));
    };
    while (ok && walk.next(a)) {
      const int n = it.t1 - it.t0, two = it.rows > 128;
      if (kv_pair<TREE>(it)) {
        if (!wait(full(t % ST), t / ST) || !wait(q_full(0), items_a++)) break;
        tc_fence_after_sync();
        both_scores(0, t);
        release(t);
        if (!wait(full((t + 1) % ST), (t + 1) / ST) || !wait(q_full(1), items_b++)) break;
        tc_fence_after_sync();
        both_scores(1, t + 1);
        release(t + 1);
#pragma unroll 1
        for (int u = t; ok && u < t + n; ++u) {
          const bool more = u + 2 < t + n;
          const int k = u - t, i = k & 1, round = (i == 0 ? done_a : done_b) + (k >> 1);
          if (!wait(ready(u & 1), u >> 1)) break;
          weigh(i, 0, u, round, k < 2);
          if (more && (!ok || !wait(full((u + 2) % ST), (u + 2) / ST))) break;
          if (more) half_scores(i, 0, u + 2);
          if (ok) weigh(i, 1, u, round, k < 2);
          if (!ok) break;
          commit(vfree(u & 1));
          if (more) {
            half_scores(i, 1, u + 2);
            release(u + 2);
          }
        }
        t += n;
        done_a += (n + 1) >> 1;
        done_b += n >> 1;
        continue;
      }
      if (!wait(full(t % ST), t / ST)) break;
#pragma unroll 1
      for (int i = 0; i <= two; ++i) {
        if (!wait(q_full(i), i == 0 ? items_a++ : items_b++)) break;
        tc_fence_after_sync();
        if constexpr (TREE) {
          half_scores(i, 0, t);
          half_scores(i, 1, t);
        } else {
          scores(i, t);
        }
      }
      if (!ok) break;
      release(t);
      if ((n > 1 && !wait(full((t + 1) % ST), (t + 1) / ST)) || !wait(ready(t & 1), t >> 1)) break;
#pragma unroll 1
      for (int u = t; ok && u < t + n; ++u) {
        const bool more = u + 1 < t + n;
        if constexpr (TREE) {
#pragma unroll
          for (int part = 0; part < 4; ++part) {
            const int i = part & 1, h = part >> 1;
            if (!ok || i > two) continue;
            weigh(i, h, u, (i == 0 ? done_a : done_b) + u - t, u == t);
            if (ok && more) half_scores(i, h, u + 1);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (!ok || i > two) break;
            weigh(i, 0, u, (i == 0 ? done_a : done_b) + u - t, u == t);
            if (ok) weigh(i, 1, u, (i == 0 ? done_a : done_b) + u - t, u == t);
            if (ok && more) scores(i, u + 1);
          }
        }
        if (!ok) break;
        commit(vfree(u & 1));
        if (more) {
          release(u + 1);
          if ((u + 2 < t + n && !wait(full((u + 2) % ST), (u + 2) / ST)) || !wait(ready((u + 1) & 1), (u + 1) >> 1)) break;
        }
      }
      t += n;
      done_a += n;
      if (two) done_b += n;
    }
    if (!ok && lane == 0) stop(&ctl->abort, status);
    __syncwarp();
  } else if (warp < 4) {
    // ---- V of a slot tile as f16, and the tile's constants ---------------------------------------
    KvWalk<kManyRows, TREE> walk;
    walk.begin(share);
    const KvItem& it = walk.it;
    int t = 0;
    bool ok = true;
    while (ok && walk.next(a)) {
#pragma unroll 1
      for (int j = it.t0; ok && j < it.t1; ++j, ++t) {
        const int s = t % ST, b = t & 1, slot0 = it.span.tile(j) * kKvTile;
        ok = __all_sync(0xffffffffu, kv_wait(full(s), (t / ST) & 1));
        if (!ok) break;
        // 0 * NaN is NaN: no slot of V that some row does not see may hold one.  Slots that nobody sees become zero; where rows
        // differ, so does a slot with a NaN, and rows that see it take a NaN weight for it.
        const bool whole = kv_whole(slot0, it.p_all, it.p_last, a.window, a.sinks);
        auto usable = [](float x) { return x >= 0x1p-120f && x <= 0x1p124f; };      // (1 / x and log2 x are finite)
        if (warp == 2 && lane < 8) {      // (where the slots are not there, or rows differ, no scale may be NaN either)
          float ks = ctl->scales[s][lane], vs = ctl->scales[s][8 + lane];
          if (!whole && (slot0 + lane * kKvBlock > it.p_last || !usable(ks) || !usable(vs))) ks = vs = 1.f;
          ctl->block[t & 3][lane] = make_float4(ks, log2f(vs), 1.f / vs, 0.f);
        }
        // (known before V is: the rows' owners need it first.  Their last use of this place, four tiles ago, was over when `vfree` of
        // the tile before the last but one was waited for)
        __syncwarp();
        if (warp == 2 && lane == 0) mbar_arrive(known(t & 3));
        ok = __all_sync(0xffffffffu, t < 2 || kv_wait(vfree(b), ((t >> 1) - 1) & 1));
        if (!ok) break;
#pragma unroll 1
        for (int part = warp - 2; part < 4; part += 2) {
          const int row = part * 32 + lane, slot = slot0 + row;      // a slot of the tile
          const bool any = slot <= it.p_last && (a.window <= 0 || slot > it.p_first - a.window || slot < a.sinks);
          const uint8_t* src = (TREE ? sK + (2 * t + 1) % PLACES * C::TILE : sC + (t % C::VSTAGES) * C::TILE) + row * D;
          uint4 u[D / 16];
#pragma unroll
          for (int e = 0; e < D / 16; ++e) u[e] = *reinterpret_cast<const uint4*>(src + (e ^ (D == 128 ? row & 7 : (row >> 1) & 3)) * 16);
          if (!whole) {
            bool nan = false;
            if (any) {
#pragma unroll
              for (int e = 0; e < D / 16; ++e)
                nan = nan || ((((u[e].x & 0x7F7F7F7Fu) + 0x01010101u) | ((u[e].y & 0x7F7F7F7Fu) + 0x01010101u) |
                               ((u[e].z & 0x7F7F7F7Fu) + 0x01010101u) | ((u[e].w & 0x7F7F7F7Fu) + 0x01010101u)) & 0x80808080u) != 0;
              nan = nan || !usable(ctl->scales[s][row >> 4]) || !usable(ctl->scales[s][8 + (row >> 4)]);
            }
            if (!any || nan) {
#pragma unroll
              for (int e = 0; e < D / 16; ++e) u[e] = make_uint4(0, 0, 0, 0);
            }
            const uint32_t bits = __ballot_sync(0xffffffffu, nan);
            if (lane == 0) ctl->nan[b][part] = bits;
          }
          uint8_t* dst = sV + b * C::VTILE + row * 128;
#pragma unroll
          for (int e = 0; e < D / 16; ++e) {
            uint8_t* d = dst + (e >> 2) * C::VCHUNK;
            const int c = (e & 3) * 2;
            *reinterpret_cast<uint4*>(d + ((c ^ (row & 7)) * 16)) =
                make_uint4(e4m3x2_to_f16x2(u[e].x), e4m3x2_to_f16x2(u[e].x >> 16), e4m3x2_to_f16x2(u[e].y), e4m3x2_to_f16x2(u[e].y >> 16));
            *reinterpret_cast<uint4*>(d + (((c + 1) ^ (row & 7)) * 16)) =
                make_uint4(e4m3x2_to_f16x2(u[e].z), e4m3x2_to_f16x2(u[e].z >> 16), e4m3x2_to_f16x2(u[e].w), e4m3x2_to_f16x2(u[e].w >> 16));
          }
        }
        fence_proxy_async_shared();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(ready(b));
          mbar_arrive(TREE ? empty((2 * t + 1) % PLACES) : smem_u32(&ctl->v_empty[t % C::VSTAGES]));
        }
      }
    }
    if (!ok && lane == 0) stop(&ctl->abort, status);
  } else {
    // ---- weights: a thread owns a row -------------------------------------------------------------
    const int i = (warp - 4) >> 2, quad = warp & 3, me = quad * 32 + lane;
    const uint32_t sS = tmem + (static_cast<uint32_t>(quad * 32) << 16) + i * 128, sO = sS + 256;
    KvWalk<kManyRows, TREE> walk;
    walk.begin(share);
    const KvItem& it = walk.it;
    constexpr float FAR = TREE ? kTreeFar : kFar;
    int t = 0, mine = 0, joins = 0;      // slot tiles of the CTA, of this row tile; pairs joined
    bool ok = true;
    while (ok && walk.next(a)) {
      const int n = it.t1 - it.t0;
      const bool pair = kv_pair<TREE>(it);
      if (i == 1 && it.rows <= 128 && !pair) {
        t += n;
        continue;
      }
      // (a pair's B has rows 64 on first: of up to 64 rows, A's and B's are then on different schedulers)
      const int row0 = pair ? 0 : i * 128, row = row0 + (pair ? me ^ (i * 64) : me);
      const bool real = row < it.rows;
      const int n_mine = pair ? (n + 1 - i) >> 1 : n;
      if (TREE && row - lane >= it.rows) {      // a warp without rows: whatever its lanes of P hold, nobody reads what comes of it
        if (lane == 0) mbar_arrive(q_full(i));
#pragma unroll 1
        for (int g = 0; ok && g < 2 * n_mine; ++g) {
          ok = __all_sync(0xffffffffu, kv_wait(s_full(i, g & 1), (mine + (g >> 1)) & 1));
          if (ok && lane == 0) mbar_arrive(p_full(i, g & 1));
        }
        t += n;
        mine += n_mine;
        if (pair && ok) {
          if (lane == 0) mbar_arrive(x_full(i));
          if (lane == 0) mbar_arrive(x_read(1 - i));
          ok = __all_sync(0xffffffffu, kv_wait(x_read(i), joins & 1));
          ++joins;
        }
        continue;
      }
      auto slot_of = [&](int r) { return it.p0 + static_cast<int>(a.by_group(it.row0 + min(r, it.rows - 1))); };
      int p = slot_of(row);      // of the row (of a tree's node: its position)
      const int p_lo = TREE ? it.p_all : slot_of(row0), p_hi = slot_of(row0 + 127);      // of the tile's first and last
      int64_t node = 0;
      if constexpr (TREE) {
        node = a.s.q0[it.i] + p - it.p0;
        if (a.window > 0) {
          kv_tree_ready<TREE>(a);
          p = it.p0 + a.depth[node];
        }
      }
      constexpr int LANES = D / 8, STEP = 32 / LANES;      // lanes that move a row, rows at a time
      const int sub = lane / LANES, part = lane % LANES;
      uint8_t* tile = sQ + i * 2 * C::QTILE + quad * 32 * D;
      auto place = [&](int r, int chunk) {      // of a row's 16-byte chunk: the swizzle of the operand tiles, the second half in the lo tile
        constexpr int PER = D / 16;
        return tile + (chunk >= PER ? C::QTILE : 0) + r * D + ((chunk % PER) ^ (D == 128 ? r & 7 : (r >> 1) & 3)) * 16;
      };
      float c;                  // scale2 * the row's power of two
      {
        // q as hi and lo codes.  A row waits in its places until its owner turns it into them, 16 elements at a time and in place: of a
        // pair of chunks the first is in the hi tile and the second in the lo tile
        {
          const unsigned long long from = real ? reinterpret_cast<unsigned long long>(kv_query(a, it, row, D)) : 0;
          uint4 u[32 / STEP];
#pragma unroll
          for (int k = 0; k < 32 / STEP; ++k) {
            const unsigned long long src = __shfl_sync(0xffffffffu, from, k * STEP + sub);
            u[k] = src != 0 ? *(reinterpret_cast<const uint4*>(src) + part) : make_uint4(0, 0, 0, 0);
          }
#pragma unroll
          for (int k = 0; k < 32 / STEP; ++k) *reinterpret_cast<uint4*>(place(k * STEP + sub, part / 2 + (part & 1) * (D / 16))) = u[k];
        }
        __syncwarp();
        uint32_t most = 0;      // largest magnitude, as the bits of two bf16 without their signs
#pragma unroll 4
        for (int e = 0; e < D / 8; ++e) {
          const uint4 u = *reinterpret_cast<const uint4*>(place(lane, e));
          most = __vmaxu2(__vmaxu2(most, __vmaxu2(u.x & 0x7FFF7FFFu, u.y & 0x7FFF7FFFu)), __vmaxu2(u.z & 0x7FFF7FFFu, u.w & 0x7FFF7FFFu));
        }
        const uint32_t top = max(most & 0xFFFFu, most >> 16);
        const bool fin = top < 0x7F80u;
        const int e2 = fin ? max(static_cast<int>(top >> 7) - 127 - 7, -110) : 0;      // top 2^-e2 in [128, 256)
        const float inv = fin ? __uint_as_float(static_cast<uint32_t>(127 - e2) << 23) : NAN;      // (a row that is not finite: NaN throughout)
        c = a.scale2 * __uint_as_float(static_cast<uint32_t>(127 + e2) << 23);
#pragma unroll 2
        for (int e = 0; e < D / 16; ++e) {      // by way of f16, which holds them (and 2^-24 where e5m2 ends at 2^-16)
          const uint4 u0 = *reinterpret_cast<const uint4*>(place(lane, e)), u1 = *reinterpret_cast<const uint4*>(place(lane, e + D / 16));
          const uint32_t w[8] = {u0.x, u0.y, u0.z, u0.w, u1.x, u1.y, u1.z, u1.w};
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) split_8bit(pair_f16(w[2 * k], inv), pair_f16(w[2 * k + 1], inv), hi[k], lo[k]);
          *reinterpret_cast<uint4*>(place(lane, e)) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
          *reinterpret_cast<uint4*>(place(lane, e + D / 16)) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
        fence_proxy_async_shared();
        __syncwarp();
        if (lane == 0) mbar_arrive(q_full(i));
      }
      float w = kNone, l = 0.f, peak = 0.f;      // peak: the largest sum of 64 weights under w
      // A maximum below FAR is a whole number, and so are the logarithms of the scales: x + (log2(vs) - w) has one rounding, of
      // a small result.  Beyond it log2(vs) - w would lose bits, scores that are equal come out different, and weights under a w that
      // is their maximum pass 1 by any factor.  There (`far`) S of the half tile is first turned into x - m, x rounded like any score
      // and m a score of the row that is the largest so far to within FAR / 4, so that what w is about is small again.
      bool far = false;
      float m = 0.f;      // (0 of other rows)
      int slot0 = 0;
      bool whole = true;
#pragma unroll 1
      for (int g = 0; g < 2 * n_mine; ++g) {      // half tiles
        const int h = g & 1, v = pair ? i + (g & ~1) : g >> 1, u = t + v, b = u & 1;
        const uint32_t sX = sS + h * kHalf;
        if (h == 0) {
          slot0 = it.span.tile(it.t0 + v) * kKvTile;
          whole = kv_whole(slot0, p_lo, p_hi, a.window, a.sinks);
          // (S first: a row tile that left items out may be rounds ahead of the others until its products run)
          ok = kv_wait(s_full(i, 0), (mine + (g >> 1)) & 1) && kv_wait(known(u & 3), (u >> 2) & 1) && (whole || kv_wait(ready(b), (u >> 1) & 1));
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc_fence_after_sync();
        } else if (TREE) {
          ok = __all_sync(0xffffffffu, kv_wait(s_full(i, 1), (mine + (g >> 1)) & 1));
          if (!ok) break;
          tc_fence_after_sync();
        }
        const float4* block = &ctl->block[u & 3][4 * h];
        if (!whole) {      // what the row does not see becomes -inf
          kv_tree_ready<TREE>(a);
          // (it sees slots up to p that are past `from` or before `few`)
          const int from = a.window > 0 ? p - a.window : -1, few = a.window > 0 ? a.sinks : INT32_MAX;
#pragma unroll 1
          for (int q = 0; q < 2; ++q) {
            const int at = slot0 + kHalf * h + 32 * q;
            const uint32_t see = TREE ? kv_tree_sees(a, it.p0, node, p, at) : below(p + 1 - at) & (~below(from + 1 - at) | below(few - at));
            const uint32_t nan = ctl->nan[b][2 * h + q] & see;
            if (__all_sync(0xffffffffu, (see & ~nan) == 0xFFFFFFFFu)) continue;
            uint32_t x[32];
            load_cols(sX + 32 * q, x);
#pragma unroll
            for (int e = 0; e < 32; ++e) x[e] = see >> e & 1 ? x[e] : 0xFF800000u;
            if (__any_sync(0xffffffffu, nan != 0)) {
#pragma unroll
              for (int e = 0; e < 32; ++e) x[e] = nan >> e & 1 ? 0x7FC00000u : x[e];
            }
            tmem_st_32x32b(sX + 32 * q, x);
          }
          tmem_wait_st();
        }
        float back = 0.f;        // old m less new
        auto level = [&](bool mine, float least) {      // S of rows that are `mine` becomes x - m, m the largest x if that is far above `least`
          float top = -INFINITY;
#pragma unroll 1
          for (int e0 = 0; e0 < 8; ++e0) {      // four times 16 columns for the largest, and again
            uint32_t y[16];
            load_cols(sX + 16 * (e0 & 3), y);
            const float mul = fmaxf(block[e0 & 3].x * c, 1e-37f);
            if (e0 == 4 && mine) {
              const float to = top > least + FAR / 4 ? top : least;
              back = m - to;
              m = to;
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float x = __fmul_rn(__uint_as_float(y[e]), mul);
              top = fmaxf(top, x);
              y[e] = mine ? __float_as_uint(x - m) : y[e];
            }
            if (e0 >= 4) tmem_st_32x32b(sX + 16 * (e0 & 3), y);
          }
          tmem_wait_st();
        };
        if (__any_sync(0xffffffffu, far)) level(far, m);
        uint32_t words[32];
        bool over = g == 0 || back != 0.f;      // the row's w has to move
        float sum = INFINITY;                   // (by how much: not known)
        // Two rounds at most: a move leaves a sum of 64 weights of at most 2^0.5 each.  (Below FAR the largest weight's exponent is
        // exact to 2^-1; of a far row x - m is at most 0 where m has just moved, else below FAR / 4.)
        int rounds = 4;
#pragma unroll 1
        while (true) {
          if (--rounds == 0) {
            ok = false;
            break;
          }
          if (__any_sync(0xffffffffu, over)) {
            // w moves in the rows that need it, and O (once its products have completed) and l with it: to a power that covers the sum
            // of the weights, or to the scores' maximum where that is not known.  The weights start (again) from S, which is whole.
            // (A move costs the same for a row and for 32: those that have outgrown their w by less come along, which leaves them
            // further from the next)
            peak = over ? sum : peak;
            float now = peak >= static_cast<float>(2 << kAfter) ? w + static_cast<float>(static_cast<int>(__float_as_uint(peak) >> 23) - 126 - kAfter) : w;
            bool find = over && !(sum < INFINITY && fabsf(now) < FAR);
            if (!over && !(fabsf(now) < FAR)) now = w;
#pragma unroll 1
            while (__any_sync(0xffffffffu, find)) {
              float top = kNone;
#pragma unroll 1
              for (int e0 = 0; e0 < 4; ++e0) {
                uint32_t y[16];
                load_cols(sX + 16 * e0, y);
                const float4 k = block[e0];
                const float mul = far ? 1.f : fmaxf(k.x * c, 1e-37f);
#pragma unroll
                for (int e = 0; e < 16; ++e) top = fmaxf(top, fmaf(__uint_as_float(y[e]), mul, k.y));
              }
              if (find) now = ceilf(top);
              find = find && !far && top > kNone && !(fabsf(top) < FAR);
              if (!__any_sync(0xffffffffu, find)) break;
              level(find, -INFINITY);      // (once: these are far now)
              far = far || find;
            }
            const float f = ex2_approx((w + back) - now);
            back = 0.f;
            w = now;
            l *= f;
            peak = 0.f;
            if (g > 0) {
              // (S of the tile is complete, so the products of the tiles before are; of half a tile, those of the half before it need not be)
              if (h == 1) ok = __all_sync(0xffffffffu, kv_wait(o_done(i, 0), (mine + (g >> 1)) & 1));
              else if (TREE) ok = __all_sync(0xffffffffu, kv_wait(o_done(i, 1), (mine + (g >> 1) - 1) & 1));
              if (!ok) break;
              tc_fence_after_sync();
#pragma unroll 1
              for (int e0 = 0; e0 < D / 64; ++e0) {
                uint32_t y[32], z[32];
                tmem_ld_32x32b(sO + 64 * e0, y);
                load_cols(sO + 64 * e0 + 32, z);
                reg_fence(y);
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                  y[e] = __float_as_uint(__uint_as_float(y[e]) * f);
                  z[e] = __float_as_uint(__uint_as_float(z[e]) * f);
                }
                tmem_st_32x32b(sO + 64 * e0, y);
                tmem_st_32x32b(sO + 64 * e0 + 32, z);
              }
              tmem_wait_st();
            }
          }
          uint32_t x[64];
          load_cols(sX, x);
          float dl = 0.f;
          sum = 0.f;
#pragma unroll
          for (int e0 = 0; e0 < 4; ++e0) {      // a block's columns
            const float4 k = block[e0];
            const float mul = far ? 1.f : fmaxf(k.x * c, 1e-37f), add = k.y - w;      // (not 0: -inf stays what it is)
            const float2 mul2 = make_float2(mul, mul), add2 = make_float2(add, add);
            float2 s0 = make_float2(0.f, 0.f), s1 = s0;
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
              const uint32_t* v = x + 16 * e0 + e;
              float2 y0 = ffma2(make_float2(__uint_as_float(v[0]), __uint_as_float(v[1])), mul2, add2);
              float2 y1 = ffma2(make_float2(__uint_as_float(v[2]), __uint_as_float(v[3])), mul2, add2);
              y0 = make_float2(ex2_approx(y0.x), ex2_approx(y0.y));
              y1 = make_float2(ex2_approx(y1.x), ex2_approx(y1.y));
              s0 = fadd2(s0, y0);
              s1 = fadd2(s1, y1);
              words[8 * e0 + e / 2] = f16x2(y0.x, y0.y);
              words[8 * e0 + e / 2 + 1] = f16x2(y1.x, y1.y);
            }
            s0 = fadd2(s0, s1);
            const float all = s0.x + s0.y;
            sum += all;
            dl = fmaf(all, k.z, dl);
          }
          over = sum >= kMost;
          if (!__any_sync(0xffffffffu, over)) {
            l += dl;
            peak = fmaxf(peak, sum);
            break;
          }
        }
        if (!ok) break;
        tmem_st_32x32b(sX, words);
        tmem_wait_st();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full(i, h));
      }
      if (!ok) break;
      t += n;
      mine += n_mine;
      // ---- the item's (part of the) output -----------------------------------------------------
      ok = __all_sync(0xffffffffu, kv_wait(o_done(i, 1), (mine - 1) & 1));
      if (!ok) break;
      tc_fence_after_sync();
      const bool complete = it.t0 == 0 && it.t1 == it.span.n;
      const int64_t slot = (2 * static_cast<int64_t>(blockIdx.x) + (it.t0 == 0 ? 1 : 0)) * kManyRows + row;
      const int64_t at = complete ? kv_out_row(a, it, real ? row : 0) : slot;
      if (pair) {
        // A ends the first half of the columns and B the second, each with what the other leaves of them in its q tile (its products have
        // completed): out = (O f + O' f') / (l f + l' f'), f = 2^(its base less the larger one)
        constexpr int HALF = D / 2, CHUNKS = HALF / 4;      // columns, and their 16-byte chunks in a row
        auto left = [&](int whose, int r, int chunk) { return reinterpret_cast<float4*>(sQ + whose * 2 * C::QTILE + r * HALF * 4 + ((chunk ^ (r & (CHUNKS - 1))) * 16)); };
#pragma unroll 1
        for (int q = 0; q < HALF / 32; ++q) {
          uint32_t o[32];
          load_cols(sO + (1 - i) * HALF + 32 * q, o);
#pragma unroll
          for (int e = 0; e < 32; e += 4)
            *left(i, row, 8 * q + e / 4) = make_float4(__uint_as_float(o[e]), __uint_as_float(o[e + 1]), __uint_as_float(o[e + 2]), __uint_as_float(o[e + 3]));
        }
        ctl->state[i][row] = make_float4(m, w, l, far ? 1.f : 0.f);
        __syncwarp();
        if (lane == 0) mbar_arrive(x_full(i));
        ok = __all_sync(0xffffffffu, kv_wait(x_full(1 - i), joins & 1));
        if (!ok) break;
        const float4 its = ctl->state[1 - i][row];
        const float apart = l == 0.f ? -INFINITY : its.z == 0.f ? INFINITY : (m - its.x) + (w - its.y);      // (one that saw nothing has no say)
        const bool first = !(apart < 0.f);
        const float f = first ? 1.f : exp2f(apart), f2 = first ? exp2f(-apart) : 1.f;
        const float sum = (l == 0.f ? 0.f : l * f) + (its.z == 0.f ? 0.f : its.z * f2);
        const float by = l == 0.f ? 0.f : f / sum, by2 = its.z == 0.f ? 0.f : f2 / sum;
#pragma unroll 1
        for (int q = 0; q < HALF / 32; ++q) {
          uint32_t o[32];
          load_cols(sO + i * HALF + 32 * q, o);
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            const float4 x = *left(1 - i, row, 8 * q + e / 4);
            const float y[4] = {x.x, x.y, x.z, x.w};
            // (a half that saw nothing is zero, whatever its accumulator holds)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              o[e + k] = __float_as_uint((l == 0.f ? 0.f : __uint_as_float(o[e + k]) * by) + (its.z == 0.f ? 0.f : y[k] * by2));
          }
          if (real && complete) {
#pragma unroll
            for (int e = 0; e < 32; e += 8)
              *reinterpret_cast<uint4*>(a.out + at * D + i * HALF + 32 * q + e) =
                  make_uint4(bf16x2(__uint_as_float(o[e]), __uint_as_float(o[e + 1])), bf16x2(__uint_as_float(o[e + 2]), __uint_as_float(o[e + 3])),
                             bf16x2(__uint_as_float(o[e + 4]), __uint_as_float(o[e + 5])), bf16x2(__uint_as_float(o[e + 6]), __uint_as_float(o[e + 7])));
          } else if (real) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) *reinterpret_cast<uint4*>(a.part + slot * D + i * HALF + 32 * q + e) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
          }
        }
        if (real && i == 0) {
          const float rel = sum == 0.f ? -INFINITY : log2f(sum), base = first ? w : its.y, top = first ? m : its.x;
          const bool high = first ? far : its.w != 0.f;
          if (!complete) a.part_lse[slot] = high ? make_float2(top, base + rel) : make_float2(base, rel);
          else if (a.lse != nullptr) a.lse[at] = (top + (base + rel)) * 0.69314718055994531f;
        }
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(x_read(1 - i));
        ok = __all_sync(0xffffffffu, kv_wait(x_read(i), joins & 1));      // (the next q goes where the other reads)
        if (!ok) break;
        ++joins;
        continue;
      }
      const float inv = l == 0.f ? 0.f : 1.f / l, rel = l == 0.f ? -INFINITY : log2f(l);
      // complete rows go out by way of the q tile, which is done with (this warp's rows), so that lanes write side by side; parts of
      // trees too where all eight warps have some, half of the columns at a time (5000 clocks; row by row 8000, where few have some 2500)
#pragma unroll 1
      for (int q = 0; q < D / 32; ++q) {
        uint32_t o[32];
        load_cols(sO + 32 * q, o);
        // (a row that saw nothing here is zero, whatever its accumulator holds)
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = l == 0.f ? 0u : __float_as_uint(__uint_as_float(o[e]) * inv);
        if (complete) {
#pragma unroll
          for (int e = 0; e < 32; e += 8) {
            uint32_t x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
              asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(x[k]) : "f"(__uint_as_float(o[e + 2 * k + 1])), "f"(__uint_as_float(o[e + 2 * k])));
            *reinterpret_cast<uint4*>(place(lane, 4 * q + e / 8)) = make_uint4(x[0], x[1], x[2], x[3]);
          }
        } else if (TREE && it.rows > 128) {
          constexpr int PER_HALF = D / 64;      // rounds of 32 columns
          const int mine = q % PER_HALF * 8;
#pragma unroll
          for (int e = 0; e < 32; e += 4) *reinterpret_cast<uint4*>(place(lane, mine + e / 4)) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
          if (q % PER_HALF == PER_HALF - 1) {
            __syncwarp();
            constexpr int WIDE = D / 8;      // lanes of a row's half
            float* to = a.part + (slot - lane + lane / WIDE) * D + q / PER_HALF * (D / 2) + lane % WIDE * 4;
#pragma unroll 2
            for (int r = lane / WIDE; r < min(32, it.rows - (row - lane)); r += 32 / WIDE, to += 32 / WIDE * D)
              *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(place(r, lane % WIDE));
            __syncwarp();
          }
        } else if (real) {
#pragma unroll
          for (int e = 0; e < 32; e += 4) *reinterpret_cast<uint4*>(a.part + slot * D + 32 * q + e) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
        }
      }
      tc_fence_before_sync();
      if (complete) {
        __syncwarp();
        const unsigned long long to = real ? reinterpret_cast<unsigned long long>(a.out + at * D) : 0;
#pragma unroll 4
        for (int k = 0; k < 32; k += STEP) {
          const unsigned long long dst = __shfl_sync(0xffffffffu, to, k + sub);
          if (dst != 0) *(reinterpret_cast<uint4*>(dst) + part) = *reinterpret_cast<const uint4*>(place(k + sub, part));
        }
        __syncwarp();
      }
      if (real) {
        if (!complete) a.part_lse[slot] = far ? make_float2(m, w + rel) : make_float2(w, rel);
        else if (a.lse != nullptr) a.lse[at] = (m + (w + rel)) * 0.69314718055994531f;
      }
    }
    if (!ok && lane == 0) stop(&ctl->abort, status);
    kv_tree_ready<TREE>(a);
    if (threadIdx.x == 4 * 32) kv_write_split(a, share, it);
  }
  tc_fence_before_sync();
  __syncthreads();
  if (stopped(&ctl->abort)) {
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 100000ull) {
    }
    __syncthreads();
  }
  tc_fence_after_sync();
  if (warp == 1) tmem_dealloc(tmem, kTmem);
}

template <int D, bool TREE>
pace_status_t run_prefill(const KvMaps& maps, const KvAttnArgs& a, unsigned grid, int* status, cudaStream_t stream) {
  using C = PrefillCfg<D>;
  constexpr size_t smem = 1024 + (C::STAGES + C::VSTAGES) * C::TILE + 2 * C::VTILE + 4 * C::QTILE + sizeof(PrefillCtl<D>);
  static_assert(smem <= 227 * 1024, "shared memory");
  static DeviceOnce once;
  int dev = 0;
  PACE_CUDA(cudaGetDevice(&dev));
  if (!once.done(dev)) {
    PACE_CUDA(cudaFuncSetAttribute(kv_prefill_kernel<D, TREE>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
    once.mark(dev);
  }
  return launch_dependent(kv_prefill_kernel<D, TREE>, grid, kThreads, smem, 1, stream, maps, a, status);
}

}  // namespace

pace_status_t launch_kv_prefill(const KvMaps& maps, const KvAttnArgs& a, int D, unsigned grid, int* status, cudaStream_t stream) {
  if (a.family != nullptr) return D == 128 ? run_prefill<128, true>(maps, a, grid, status, stream) : run_prefill<64, true>(maps, a, grid, status, stream);
  return D == 128 ? run_prefill<128, false>(maps, a, grid, status, stream) : run_prefill<64, false>(maps, a, grid, status, stream);
}

}  // namespace pace
