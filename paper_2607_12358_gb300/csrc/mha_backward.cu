// The gradient of attention in bf16 on tcgen05 (acid_mha_backward).
//
// Two kernels, each with one side stationary, form
//     dv = P^T g,  dk = scale dS^T q      (keys stationary: S^T = k q^T, dP^T = v g^T)
//     dq = scale dS k                     (queries stationary: S = q k^T, dP = g v^T)
// with P = 2^(scale log2(e) S - lse log2(e)) and dS = P (dP - sum(g out)).  P and dS
// go through the same registers and tensor memory as the forward pass's probabilities:
// written over S and dP as bf16 they are the A operand of the next product, and both
// sums stay in tensor memory until a tile's last step.
//   One kernel with all three sums would need five products instead of seven, but has
// to add dq into memory from every key tile: 64 KB of fp32 a step, through shared
// memory, in an order that changes results (or waits on other CTAs), and dS a second
// time in shared memory.  At head dim 128 a step's operands already take what shared
// memory delivers (128 bytes a clock feed an M128 N128 product of two shared operands
// exactly): 3840 clocks for its five products, against 2050 + 1800 for the two kernels.
#include <algorithm>
#include <type_traits>

#include "attention.cuh"
#include "mha.cuh"

namespace acid {

unsigned int take_device_error_mha_backward();
ACID_DEVICE_FLAG_READER(take_device_error_mha_backward)
BoundsRecord take_bounds_mha_backward();
ACID_BOUNDS_READER(take_bounds_mha_backward)

namespace {

constexpr int kTile = 128;     // rows of a tile on either side
constexpr int kThreads = 320;  // TMA warp, MMA warp, eight warps of elementwise work
constexpr int kWorkers = 256;
constexpr int kStatBytes = 2 * kStatRows * 4;

struct BwdArgs {
  MhaShape s;
  const float* stats;
  __nv_bfloat16 *out1, *out2;  // keys stationary: dk, dv (either may be null); queries stationary: dq
  int64_t ld1, ld2;
  float scale, scale_log2;
  int slots, stat_slots, heads;  // of the stationary side
  int full, splits, units;       // as in the forward pass: units from `full` on are shares of an item
  float* part;                   // [split units][1 or 2][D / 4][128 rows][4]
};

// A CTA's unit: a stationary tile with the streamed tiles that see it.
struct BwdUnit {
  int head;         // of the stationary side
  int row0, rows;   // first stationary row, rows left in its sequence
  int j0, tiles;    // streamed tiles [j0, j0 + tiles) of the sequence, for each head of the group
  int n0, steps;    // steps [n0, n0 + steps) of group * tiles
  int part;         // slot of a share's partial sums, or -1
  int tile, index;  // of and in the sequence
  MhaSeq seq;
};

template <bool KEYS>
__device__ __forceinline__ bool bwd_unit(const BwdArgs& a, int u, BwdUnit& x) {
  int item = u, split = 0, slot;
  x.part = -1;
  if (u >= a.full) {
    x.part = u - a.full;
    item = a.full + x.part / a.splits;
    split = x.part % a.splits;
  }
  if (a.s.frame == 0) {
    slot = item % a.slots;
    x.head = item / a.slots;
  } else {  // longest first under a causal window: the first keys, the last queries
    slot = item / a.heads;
    if (!KEYS) slot = a.slots - 1 - slot;
    x.head = item % a.heads;
  }
  if (!mha_slot<kTile, KEYS>(a.s, slot, x.seq, x.index, x.tile)) return false;
  const int r0 = x.tile * kTile, n = KEYS ? x.seq.nk : x.seq.nq;
  x.row0 = (KEYS ? x.seq.k0 : x.seq.q0) + r0;
  x.rows = n - r0;
  int lo, hi, none;
  const int last = r0 + min(x.rows, kTile) - 1;
  if (KEYS) {
    mha_queries_of(a.s, x.seq, r0, lo, none);
    mha_queries_of(a.s, x.seq, last, none, hi);
  } else {
    mha_keys_of(a.s, x.seq, r0, lo, none);
    mha_keys_of(a.s, x.seq, last, none, hi);
  }
  x.j0 = lo / kTile;
  x.tiles = hi > lo ? (hi + kTile - 1) / kTile - x.j0 : 0;
  const int total = x.tiles * (KEYS ? a.s.group : 1);
  x.n0 = 0;
  x.steps = total;
  if (x.part >= 0) {
    x.n0 = (int)((int64_t)split * total / a.splits);
    x.steps = (int)((int64_t)(split + 1) * total / a.splits) - x.n0;
  }
  return true;
}
template <bool KEYS>
__device__ __forceinline__ bool next_bwd_unit(const BwdArgs& a, int& u, BwdUnit& x) {
  for (; u < a.units; u += gridDim.x)
    if (bwd_unit<KEYS>(a, u, x) && x.steps > 0) return true;
  return false;
}

// Shared memory: the two stationary tiles, rings of the two streamed operands, the
// rows' statistics beside them, barriers.  Y1 (q or k) is read by the first product of
// a step and the last one of an earlier step, so its ring is longer by the steps that
// the first product runs ahead.
template <int HEAD_DIM, bool KEYS_>
struct BwdCfg {
  static constexpr int D = HEAD_DIM;
  static constexpr bool KEYS = KEYS_;
  static constexpr int CH = D / 64, CHUNK = kTile * 128, T_BYTES = CH * CHUNK;
  // S regions in tensor memory: with two, the next step's S is formed while this one's is
  // worked on.  Keys stationary at head dim 128: S, dP and two sums fill the 512 columns.
  static constexpr int NS = KEYS && D == 128 ? 1 : 2;
  static constexpr int Y1S = D == 64 ? 4 : NS + 1, Y2S = D == 64 ? 4 : 2;
  static constexpr int SUMS = KEYS ? 2 : 1;
  static constexpr int OFF_X = 0, OFF_Y1 = 2 * T_BYTES, OFF_Y2 = OFF_Y1 + Y1S * T_BYTES;
  static constexpr int OFF_STAT = OFF_Y2 + Y2S * T_BYTES;
  static constexpr int OFF_BAR = OFF_STAT + (KEYS ? Y1S * kStatBytes : 0);
  static constexpr int SMEM = OFF_BAR + 512 + 1024;
  static_assert(SMEM <= 227 * 1024, "shared memory");
  static constexpr uint32_t S_COL = 0, DP_COL = NS * 128, SUM_COL = DP_COL + 128;
  static_assert(SUM_COL + SUMS * D <= 512, "tensor memory");
  static constexpr uint32_t TMEM_COLS = 512;
};

template <class C>
struct BwdBars {
  uint64_t *x_full, *x_empty, *y1_full, *y1_empty, *y2_full, *y2_empty;
  uint64_t *s_full, *dp_full, *dp_read, *p_full, *ds_full, *sum_full, *sum_empty, *edge, *drain;
  uint32_t* tmem_slot;
  static constexpr int kCount = 2 + 2 * C::Y1S + 2 * C::Y2S + C::NS + 8;
  static_assert(kCount * 8 + 4 <= 512, "barrier area");
  __device__ __forceinline__ explicit BwdBars(uint8_t* at) {
    uint64_t* b = reinterpret_cast<uint64_t*>(at);
    auto take = [&](int n) { uint64_t* r = b; b += n; return r; };
    x_full = take(1);
    x_empty = take(1);
    y1_full = take(C::Y1S);
    y1_empty = take(C::Y1S);
    y2_full = take(C::Y2S);
    y2_empty = take(C::Y2S);
    s_full = take(C::NS);
    dp_full = take(1);
    dp_read = take(1);
    p_full = take(1);
    ds_full = take(1);
    sum_full = take(1);
    sum_empty = take(1);
    edge = take(1);
    drain = take(1);
    tmem_slot = reinterpret_cast<uint32_t*>(b);
  }
  __device__ __forceinline__ void init() const {
    mbar_init(x_full, 1);
    mbar_init(x_empty, 1);
    for (int i = 0; i < C::Y1S; ++i) {
      mbar_init(&y1_full[i], 1);
      mbar_init(&y1_empty[i], 1);
    }
    for (int i = 0; i < C::Y2S; ++i) {
      mbar_init(&y2_full[i], 1);
      mbar_init(&y2_empty[i], 1);
    }
    for (int i = 0; i < C::NS; ++i) mbar_init(&s_full[i], 1);
    mbar_init(dp_full, 1);
    mbar_init(dp_read, kWorkers);
    mbar_init(p_full, kWorkers);
    mbar_init(ds_full, kWorkers);
    mbar_init(sum_full, 1);
    mbar_init(sum_empty, kWorkers);
    mbar_init(edge, 1);
    mbar_init(drain, 1);
    mbar_fence_init();
  }
};

// `bytes` (a multiple of 16, both addresses 16-byte aligned) counted on `bar`.
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                   smem_u32(dst)),
               "l"(src), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

// Four consecutive floats as two packed pairs.  (Through a generic pointer, which is
// what the aligned base of dynamic shared memory is to the compiler, the same loads
// take the path of global memory: 4726 rows, 30 x 64, keys stationary STEP1A us instead of
// STEP1B.)
__device__ __forceinline__ void lds_pairs(uint32_t addr, uint64_t& a, uint64_t& b) {
  asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(a), "=l"(b) : "r"(addr));
}

// D[128 x 128] = A B^T over D columns, both K-major in shared memory.
template <class C>
__device__ __forceinline__ void mma_scores(uint32_t d, uint64_t adesc, uint64_t bdesc) {
  constexpr uint32_t idesc = idesc_bf16_f32(128, 128, false, false);
#pragma unroll
  for (int kk = 0; kk < C::D / 16; ++kk) {
    const uint64_t off = (uint64_t)(((kk >> 2) * C::CHUNK + (kk & 3) * 32) >> 4);
    mma_bf16_ss(d, adesc + off, bdesc + off, idesc, kk != 0);
  }
}
// D[128 x D] (+)= A B over the 128 streamed rows: A in tensor memory as the workers
// leave it (bf16 pairs, rows 0-63 from column a on, rows 64-127 from a + 64 on), B
// MN-major in shared memory.
template <class C>
__device__ __forceinline__ void mma_sum(uint32_t d, uint32_t a, uint64_t bdesc, bool accumulate) {
  constexpr uint32_t idesc = idesc_bf16_f32(128, C::D, false, true);
#pragma unroll
  for (int kk = 0; kk < 8; ++kk)
    mma_bf16_ts(d, a + (kk >> 2) * 64 + (kk & 3) * 8, bdesc + (uint64_t)((kk * 16 * 128) >> 4), idesc,
                accumulate || kk != 0);
}

// Rows [valid, 128) of a loaded tile are set to zero (rows of another sequence or of
// none, which a product over rows would meet with weight 0).  By a whole warp.
template <class C>
__device__ __forceinline__ void clear_tile_rows(uint8_t* tile, int valid, int lane) {
  for (int c = 0; c < C::CH; ++c) {
    uint4* p = reinterpret_cast<uint4*>(tile + c * C::CHUNK);
    for (int i = valid * 8 + lane; i < kTile * 8; i += 32) p[i] = make_uint4(0, 0, 0, 0);
  }
  fence_proxy_async_smem();
  __syncwarp();
}

// X1, X2: the stationary operands (k, v or q, g); Y1, Y2: the streamed ones (q, g or
// k, v).
template <class C>
__global__ void __launch_bounds__(kThreads, 1)
    mha_backward_kernel(const __grid_constant__ CUtensorMap tmX1, const __grid_constant__ CUtensorMap tmX2,
                        const __grid_constant__ CUtensorMap tmY1, const __grid_constant__ CUtensorMap tmY2,
                        const __grid_constant__ BwdArgs a) {
  constexpr bool KEYS = C::KEYS;
  constexpr int D = C::D;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sX = smem + C::OFF_X;
  uint8_t* sY1 = smem + C::OFF_Y1;
  uint8_t* sY2 = smem + C::OFF_Y2;
  const BwdBars<C> bar(smem + C::OFF_BAR);
  const int warp = warp_index(), lane = threadIdx.x & 31;
  if (warp == 0 && lane == 0) {
    tma_prefetch_desc(&tmX1);
    tma_prefetch_desc(&tmX2);
    tma_prefetch_desc(&tmY1);
    tma_prefetch_desc(&tmY2);
    bar.init();
  }
  if (warp == 1) tmem_alloc(bar.tmem_slot, C::TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *bar.tmem_slot;
  pdl_wait();

  if (warp == 0) {  // -------------------------------------------- TMA producer
    bool ok = true;
    int y1_done = 0, y2_done = 0, x_done = 0, edges = 0;
    BwdUnit x;
    int u = blockIdx.x, g = 0;
    for (; ok && next_bwd_unit<KEYS>(a, u, x); u += gridDim.x, ++x_done) {
      if (x_done > 0 && !mbar_wait_warp(bar.x_empty, (x_done - 1) & 1)) { ok = false; break; }
      if (lane == 0) {
        mbar_expect_tx(bar.x_full, 2 * C::T_BYTES);
        for (int c = 0; c < C::CH; ++c) {
          tma_load_2d(sX + c * C::CHUNK, &tmX1, bar.x_full, x.head * D + c * 64, x.row0);
          tma_load_2d(sX + C::T_BYTES + c * C::CHUNK, &tmX2, bar.x_full, x.head * D + c * 64, x.row0);
        }
      }
      const int seq0 = KEYS ? x.seq.q0 : x.seq.k0, n = KEYS ? x.seq.nq : x.seq.nk, all = KEYS ? a.s.nq : a.s.nk;
      const int stat0 = KEYS ? mha_slot0(a.s.qb, x.index, x.seq.q0, kStatRows) : 0;
      for (int i = 0; ok && i < x.steps; ++i, ++g) {
        const int j = x.j0 + (x.n0 + i) % x.tiles;
        const int head = KEYS ? x.head * a.s.group + (x.n0 + i) / x.tiles : x.head / a.s.group;
        const int valid = n - j * kTile, row = seq0 + j * kTile;
        const bool clear = valid < kTile && seq0 + n < all;
        // (the statistics of a tile's queries come with it: one kilobyte)
        auto load = [&](uint8_t* dst, const CUtensorMap* map, uint64_t* full, uint8_t* stat_dst) -> bool {
          uint64_t* to = clear ? bar.edge : full;
          if (lane == 0) {
            mbar_expect_tx(to, C::T_BYTES + (stat_dst != nullptr ? kStatBytes : 0));
            for (int c = 0; c < C::CH; ++c) tma_load_2d(dst + c * C::CHUNK, map, to, head * D + c * 64, row);
            if (stat_dst != nullptr)
              bulk_load(stat_dst, a.stats + mha_stat_offset(head, a.stat_slots, stat0 + j), kStatBytes, to);
          }
          if (clear) {
            if (!mbar_wait_warp(bar.edge, edges++ & 1)) return false;
            clear_tile_rows<C>(dst, valid, lane);
            if (lane == 0) mbar_arrive(full);
          }
          return true;
        };
        const int s1 = g % C::Y1S, s2 = g % C::Y2S;
        const int r1 = g / C::Y1S, r2 = g / C::Y2S;
        if (r1 > 0 && !mbar_wait_warp(&bar.y1_empty[s1], (r1 - 1) & 1)) { ok = false; break; }
        if (!load(sY1 + s1 * C::T_BYTES, &tmY1, &bar.y1_full[s1],
                  KEYS ? smem + C::OFF_STAT + s1 * kStatBytes : nullptr)) { ok = false; break; }
        y1_done = g + 1;
        if (r2 > 0 && !mbar_wait_warp(&bar.y2_empty[s2], (r2 - 1) & 1)) { ok = false; break; }
        if (!load(sY2 + s2 * C::T_BYTES, &tmY2, &bar.y2_full[s2], nullptr)) { ok = false; break; }
        y2_done = g + 1;
      }
    }
    if (!ok && lane == 0) {  // a wait ran out: the loads issued so far have landed before the CTA leaves
      mbar_wait(bar.x_full, x_done & 1);
      for (int i = std::max(0, y1_done - C::Y1S); i < y1_done; ++i) mbar_wait(&bar.y1_full[i % C::Y1S], (i / C::Y1S) & 1);
      for (int i = std::max(0, y2_done - C::Y2S); i < y2_done; ++i) mbar_wait(&bar.y2_full[i % C::Y2S], (i / C::Y2S) & 1);
    }
  } else if (warp == 1) {  // ------------------------------------- MMA issuer
    const bool leader = elect_one();
    const uint64_t x1 = smem_desc_sw128(smem_u32(sX), 16, 1024);
    const uint64_t x2 = smem_desc_sw128(smem_u32(sX + C::T_BYTES), 16, 1024);
    const uint64_t y1k = smem_desc_sw128(smem_u32(sY1), 16, 1024), y2k = smem_desc_sw128(smem_u32(sY2), 16, 1024);
    const uint64_t y1m = smem_desc_sw128(smem_u32(sY1), C::CHUNK, 1024);
    const uint64_t y2m = smem_desc_sw128(smem_u32(sY2), C::CHUNK, 1024);
    auto at = [](uint64_t desc, int slot) { return desc + (uint64_t)((slot * C::T_BYTES) >> 4); };
    bool ok = true;
    int u = blockIdx.x, units = 0, g0 = 0;
    BwdUnit x;
    for (; ok && next_bwd_unit<KEYS>(a, u, x); u += gridDim.x, ++units) {
      if (!mbar_wait_warp(bar.x_full, units & 1)) { ok = false; break; }
      auto scores = [&](int i) -> bool {  // S of step i
        const int g = g0 + i;
        if (i >= x.steps) return true;
        if (!mbar_wait_warp(&bar.y1_full[g % C::Y1S], (g / C::Y1S) & 1)) return false;
        tc_fence_after();
        if (leader) {
          mma_scores<C>(tmem + C::S_COL + (g % C::NS) * 128, x1, at(y1k, g % C::Y1S));
          mma_commit(&bar.s_full[g % C::NS]);
        }
        __syncwarp();
        return true;
      };
      auto grads = [&](int i) -> bool {  // dP of step i
        const int g = g0 + i;
        if (i >= x.steps) return true;
        if (!mbar_wait_warp(&bar.y2_full[g % C::Y2S], (g / C::Y2S) & 1)) return false;
        tc_fence_after();
        if (leader) {
          mma_scores<C>(tmem + C::DP_COL, x2, at(y2k, g % C::Y2S));
          mma_commit(bar.dp_full);
          if (!KEYS) mma_commit(&bar.y2_empty[g % C::Y2S]);
          if (i == x.steps - 1) mma_commit(bar.x_empty);
        }
        __syncwarp();
        return true;
      };
      ok = scores(0) && grads(0) && (C::NS == 1 || scores(1));
      for (int i = 0; ok && i < x.steps; ++i) {
        const int g = g0 + i;
        if (i == 0 && units > 0 && !mbar_wait_warp(bar.sum_empty, (units - 1) & 1)) { ok = false; break; }
        if constexpr (KEYS) {
          // dv += P^T g, over S; then the next S may take the region
          if (!mbar_wait_warp(bar.p_full, g & 1)) { ok = false; break; }
          tc_fence_after();
          if (leader) {
            mma_sum<C>(tmem + C::SUM_COL + D, tmem + C::S_COL + (g % C::NS) * 128, at(y2m, g % C::Y2S), i != 0);
            mma_commit(&bar.y2_empty[g % C::Y2S]);
          }
          __syncwarp();
          if (!scores(i + C::NS)) { ok = false; break; }
          if (!mbar_wait_warp(bar.ds_full, g & 1)) { ok = false; break; }
          tc_fence_after();
          if (leader) {
            mma_sum<C>(tmem + C::SUM_COL, tmem + C::DP_COL, at(y1m, g % C::Y1S), i != 0);
            mma_commit(&bar.y1_empty[g % C::Y1S]);
            if (i == x.steps - 1) mma_commit(bar.sum_full);
          }
          __syncwarp();
          if (!grads(i + 1)) { ok = false; break; }
        } else {
          // the next dP as soon as this one has been read; dq += dS k, over S
          if (i + 1 < x.steps) {
            if (!mbar_wait_warp(bar.dp_read, g & 1) || !grads(i + 1)) { ok = false; break; }
          }
          if (!mbar_wait_warp(bar.ds_full, g & 1)) { ok = false; break; }
          tc_fence_after();
          if (leader) {
            mma_sum<C>(tmem + C::SUM_COL, tmem + C::S_COL + (g % C::NS) * 128, at(y1m, g % C::Y1S), i != 0);
            mma_commit(&bar.y1_empty[g % C::Y1S]);
            if (i == x.steps - 1) mma_commit(bar.sum_full);
          }
          __syncwarp();
          if (!scores(i + C::NS)) { ok = false; break; }
        }
      }
      g0 += x.steps;
    }
    if (!ok && leader) drain_mmas(bar.drain);
  } else {  // ------------------------------------------- workers
    // Warps 2-5 have the first 64 streamed rows (columns) of a step, warps 6-9 the others;
    // a thread has one stationary row, its TMEM lane.
    const int half = (warp - 2) >> 2, q = warp & 3, r = q * 32 + lane;
    const uint32_t base = tmem + ((uint32_t)(q * 32) << 16);
    const uint64_t sc2 = f2_pack(a.scale_log2, a.scale_log2);
    bool ok = true;
    int g = 0, sums = 0;
    for (int u = blockIdx.x; ok && u < a.units; u += gridDim.x) {
      BwdUnit x;
      if (!bwd_unit<KEYS>(a, u, x)) continue;
      const int last = (KEYS ? x.seq.nk : x.seq.nq) - 1, r0 = x.tile * kTile;
      auto seen = [&](int row, int& lo, int& hi) {
        if (KEYS) mha_queries_of(a.s, x.seq, min(row, last), lo, hi);
        else mha_keys_of(a.s, x.seq, min(row, last), lo, hi);
      };
      int lo, hi, all_lo, all_hi, none;
      seen(r0 + r, lo, hi);
      seen(r0, none, all_hi);
      seen(r0 + kTile - 1, all_lo, none);
      float nlse = 0.f, ndelta = 0.f;
      if (!KEYS) {
        const int slot = mha_slot0(a.s.qb, x.index, x.seq.q0, kStatRows) + x.tile;
        const float* st = a.stats + mha_stat_offset(x.head, a.stat_slots, slot);
        nlse = st[r];
        ndelta = st[kStatRows + r];
      }
      // One step; MASK: some row does not see some streamed row.
      auto step = [&](int i, auto mask) -> bool {
        constexpr bool MASK = decltype(mask)::value;
        const int c0 = (x.j0 + (x.n0 + i) % x.tiles) * kTile + half * 64;
        const uint32_t s_at = base + C::S_COL + (g % C::NS) * 128 + half * 64, dp_at = base + C::DP_COL + half * 64;
        const uint32_t st = smem_u32(smem + C::OFF_STAT + (KEYS ? g % C::Y1S : 0) * kStatBytes) + half * 256;
        if (!mbar_wait(&bar.s_full[g % C::NS], (g / C::NS) & 1)) return false;
        // (the statistics were written by the copy that the scores' operand came with: its own barrier
        // makes them visible to this thread; completed long before)
        if (KEYS && !mbar_wait(&bar.y1_full[g % C::Y1S], (g / C::Y1S) & 1)) return false;
        tc_fence_after();
        float p[64];
#pragma unroll
        for (int c = 0; c < 2; ++c) tmem_ld32(s_at + c * 32, reinterpret_cast<uint32_t*>(p + c * 32));
        tmem_wait_ld();
#pragma unroll
        for (int c = 0; c < 64; c += 4) {
          uint64_t n01, n23;
          if (KEYS) lds_pairs(st + c * 4, n01, n23);
          else n01 = n23 = f2_pack(nlse, nlse);
          f2_unpack(f2_fma(f2_pack(p[c], p[c + 1]), sc2, n01), p[c], p[c + 1]);
          f2_unpack(f2_fma(f2_pack(p[c + 2], p[c + 3]), sc2, n23), p[c + 2], p[c + 3]);
        }
        float dp[64];
        // dP is read behind P where it comes later than S, and beside the exponentials where
        // it is there by then (queries stationary)
        auto read_dp = [&]() -> bool {
          if (!mbar_wait(bar.dp_full, g & 1)) return false;
          tc_fence_after();
#pragma unroll
          for (int c = 0; c < 2; ++c) tmem_ld32(dp_at + c * 32, reinterpret_cast<uint32_t*>(dp + c * 32));
          return true;
        };
        if (!KEYS && !read_dp()) return false;
#pragma unroll
        for (int c = 0; c < 64; ++c) {
          p[c] = ex2_approx(p[c]);
          if (MASK && (c0 + c < lo || c0 + c >= hi)) p[c] = 0.f;
        }
        if constexpr (KEYS) {
          uint32_t pk[32];
#pragma unroll
          for (int c = 0; c < 32; ++c) pk[c] = pack_bf16(p[2 * c], p[2 * c + 1]);
          tmem_st32(s_at, pk);
          tmem_wait_st();
          tc_fence_before();
          mbar_arrive(bar.p_full);
          if (!read_dp()) return false;
        }
        tmem_wait_ld();
        if constexpr (!KEYS) {
          tc_fence_before();
          mbar_arrive(bar.dp_read);
        }
        uint32_t pk[32];
#pragma unroll
        for (int c = 0; c < 64; c += 4) {
          uint64_t d01, d23;
          if (KEYS) lds_pairs(st + kStatRows * 4 + c * 4, d01, d23);
          else d01 = d23 = f2_pack(ndelta, ndelta);
          float v[4];
          f2_unpack(f2_mul(f2_pack(p[c], p[c + 1]), f2_add(f2_pack(dp[c], dp[c + 1]), d01)), v[0], v[1]);
          f2_unpack(f2_mul(f2_pack(p[c + 2], p[c + 3]), f2_add(f2_pack(dp[c + 2], dp[c + 3]), d23)), v[2], v[3]);
          if (MASK)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (c0 + c + k < lo || c0 + c + k >= hi) v[k] = 0.f;  // (0 times what may not be finite)
          pk[c / 2] = pack_bf16(v[0], v[1]);
          pk[c / 2 + 1] = pack_bf16(v[2], v[3]);
        }
        tmem_st32(KEYS ? dp_at : s_at, pk);
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(bar.ds_full);
        return true;
      };
      for (int i = 0; i < x.steps; ++i, ++g) {
        const int c0 = (x.j0 + (x.n0 + i) % x.tiles) * kTile;
        // (streamed queries behind the sequence have probability 0 by their statistics)
        const bool plain = c0 >= all_lo && (c0 + kTile <= all_hi || (KEYS && all_hi == x.seq.nq));
        if (!(plain ? step(i, std::false_type{}) : step(i, std::true_type{}))) {
          ok = false;
          break;
        }
      }
      // ------------------------------------------------ sums
      if (ok && x.steps > 0) ok = mbar_wait(bar.sum_full, sums++ & 1);
      ok = __all_sync(0xffffffffu, ok);
      tc_fence_after();
      const bool mine = ok && r < x.rows;
#pragma unroll 1
      for (int w = 0; w < C::SUMS; ++w) {
        __nv_bfloat16* out = w == 0 ? a.out1 : a.out2;
        const int64_t ld = w == 0 ? a.ld1 : a.ld2;
        const float by = w == 0 ? a.scale : 1.0f;
#pragma unroll 1
        for (int c = half * (D / 2); c < (half + 1) * (D / 2); c += 32) {
          uint32_t o[32];
          if (x.steps > 0) {
            tmem_ld32(base + C::SUM_COL + w * D + c, o);
            tmem_wait_ld();
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = 0;
          }
          if (!ok) continue;
          if (x.part >= 0) {
            float* to = a.part + (((int64_t)x.part * C::SUMS + w) * (D / 4) + c / 4) * (kTile * 4) + r * 4;
#pragma unroll
            for (int i = 0; i < 8; ++i)
              *reinterpret_cast<uint4*>(to + i * kTile * 4) = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
            continue;
          }
          const int64_t at = (int64_t)(x.row0 + r) * ld + x.head * D + c;
          if (!mine || out == nullptr || !ACID_IN_BOUNDS(kSiteMha, at + 31, (KEYS ? a.s.nk : a.s.nq) * ld)) continue;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            auto v = [&](int k) { return __uint_as_float(o[8 * i + k]) * by; };
            reinterpret_cast<uint4*>(out + at)[i] =
                make_uint4(pack_bf16(v(0), v(1)), pack_bf16(v(2), v(3)), pack_bf16(v(4), v(5)), pack_bf16(v(6), v(7)));
          }
        }
      }
      if (ok && x.steps > 0) {
        tc_fence_before();
        mbar_arrive(bar.sum_empty);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, C::TMEM_COLS);
  }
}

// Adds the shares of the split items in their order.  A thread has four columns of a
// row; a warp 32 rows.
template <int D, bool KEYS>
__global__ void __launch_bounds__(256) mha_backward_join_kernel(const __grid_constant__ BwdArgs a) {
  constexpr int SUMS = KEYS ? 2 : 1;
  pdl_wait();
  const int it = blockIdx.x, row = threadIdx.x & 127;
  BwdUnit x;
  if (!bwd_unit<KEYS>(a, a.full + it * a.splits, x) || row >= x.rows) return;
  const int idx = blockIdx.y * 2 + (threadIdx.x >> 7);  // quad of columns, of dk and then dv
  const int w = idx / (D / 4), c = idx % (D / 4) * 4;
  __nv_bfloat16* out = w == 0 ? a.out1 : a.out2;
  if (out == nullptr) return;
  const float* p = a.part + ((int64_t)it * a.splits * SUMS * (D / 4) + idx) * (kTile * 4) + row * 4;
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s = 0; s < a.splits; ++s) {
    const float4 v = *reinterpret_cast<const float4*>(p + (int64_t)s * SUMS * (D / 4) * (kTile * 4));
    sum.x += v.x;
    sum.y += v.y;
    sum.z += v.z;
    sum.w += v.w;
  }
  const float by = w == 0 ? a.scale : 1.0f;
  const int64_t ld = w == 0 ? a.ld1 : a.ld2, at = (int64_t)(x.row0 + row) * ld + x.head * D + c;
  if (!ACID_IN_BOUNDS(kSiteMha, at + 3, (int64_t)(KEYS ? a.s.nk : a.s.nq) * ld)) return;
  *reinterpret_cast<uint2*>(out + at) = make_uint2(pack_bf16(sum.x * by, sum.y * by), pack_bf16(sum.z * by, sum.w * by));
}

struct BwdPlan {
  int slots, items, full, splits;
};
// As the forward pass: a few items are shared out so that they fill the GPU, and so is
// the last wave of many where all are alike.
BwdPlan bwd_plan(const MhaShape& s, bool keys, int sms) {
  BwdPlan p;
  p.slots = mha_slots(keys ? s.nk : s.nq, s.seqs, (keys ? s.kb : s.qb) != nullptr, kTile);
  p.items = p.slots * (keys ? s.kv_heads : s.heads);
  p.full = p.items;
  p.splits = 1;
  const int steps = ((keys ? s.nq : s.nk) / s.seqs + kTile - 1) / kTile * (keys ? s.group : 1);
  const int whole = p.items / sms * sms, tail = p.items - whole;
  const bool alike = s.seqs == 1 && s.frame == 0;
  const int splits = tail > 0 ? std::min(sms / tail, steps / 2) : 1;
  if ((whole == 0 || alike) && splits >= 2) {
    p.full = whole;
    p.splits = splits;
  }
  return p;
}
size_t bwd_part_bytes(const BwdPlan& p, int sums, int d) {
  return p.full < p.items ? (size_t)(p.items - p.full) * p.splits * sums * kTile * d * sizeof(float) : 0;
}

template <int D, bool KEYS>
acid_status launch(const MhaArgs& x, cudaStream_t s) {
  using C = BwdCfg<D, KEYS>;
  static PerContext allowed;
  ACID_TRY(allow_smem(allowed, mha_backward_kernel<C>, C::SMEM));
  const MhaShape& m = x.shape;
  const int64_t nq = std::max(m.nq, 1), nk = std::max(m.nk, 1);  // (without rows nothing is loaded)
  const int64_t wq = (int64_t)m.heads * D, wk = (int64_t)m.kv_heads * D;
  const void* any = KEYS ? x.k : x.q;
  CUtensorMap tq, tg, tk, tv;
  ACID_TRY(make_tmap_bf16(&tq, m.nq > 0 ? x.q : any, nq, wq, x.ldq, kTile));
  ACID_TRY(make_tmap_bf16(&tg, m.nq > 0 ? x.dout : any, nq, wq, x.lddo, kTile));
  ACID_TRY(make_tmap_bf16(&tk, m.nk > 0 ? x.k : any, nk, wk, x.ldk, kTile));
  ACID_TRY(make_tmap_bf16(&tv, m.nk > 0 ? x.v : any, nk, wk, x.ldv, kTile));
  const BwdPlan p = bwd_plan(m, KEYS, num_sms());
  BwdArgs a = {};
  a.s = m;
  a.stats = x.stats;
  a.out1 = static_cast<__nv_bfloat16*>(KEYS ? x.dk : x.dq);
  a.ld1 = KEYS ? x.lddk : x.lddq;
  a.out2 = static_cast<__nv_bfloat16*>(x.dv);
  a.ld2 = x.lddv;
  a.scale = x.scale;
  a.scale_log2 = x.scale * 1.4426950408889634f;
  a.slots = p.slots;
  a.stat_slots = mha_slots(m.nq, m.seqs, m.qb != nullptr, kStatRows);
  a.heads = KEYS ? m.kv_heads : m.heads;
  a.full = p.full;
  a.splits = p.splits;
  a.units = p.full + (p.items - p.full) * p.splits;
  a.part = static_cast<float*>(x.part);
  launch_pdl(mha_backward_kernel<C>, std::min(a.units, num_sms()), kThreads, C::SMEM, s, KEYS ? tk : tq, KEYS ? tv : tg,
             KEYS ? tq : tk, KEYS ? tg : tv, a);
  ACID_CHECK_LAUNCH();
  if (p.full < p.items) {
    launch_pdl(mha_backward_join_kernel<D, KEYS>, dim3(p.items - p.full, C::SUMS * D / 8), 256, 0, s, a);
    ACID_CHECK_LAUNCH();
  }
  return ACID_OK;
}

}  // namespace

size_t mha_backward_tc_bytes(const MhaArgs& x) {
  const int sms = num_sms();
  return std::max(bwd_part_bytes(bwd_plan(x.shape, true, sms), 2, x.head_dim),
                  bwd_part_bytes(bwd_plan(x.shape, false, sms), 1, x.head_dim));
}

acid_status mha_backward_tc(const MhaArgs& x, cudaStream_t s) {
  if (x.dk != nullptr || x.dv != nullptr) ACID_TRY(x.head_dim == 128 ? (launch<128, true>(x, s)) : (launch<64, true>(x, s)));
  if (x.dq != nullptr) ACID_TRY(x.head_dim == 128 ? (launch<128, false>(x, s)) : (launch<64, false>(x, s)));
  return ACID_OK;
}

}  // namespace acid
