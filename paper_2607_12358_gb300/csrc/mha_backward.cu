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
// exactly): 3840 clocks for its five products, against about 2000 + 1500 that the two
// kernels take (32760 rows, 12 heads: 1.36 + 1.01 us a step at the power cap's 1.45 GHz).
#include <algorithm>
#include <type_traits>

#include "attention.cuh"
#include "mha.cuh"
#include "mha_shares.h"

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
  int items;      // stationary tiles and heads
  int full;       // items [0, full) go to the CTAs whole, one in turn; the others' steps are shared out
  int alike;      // every item has the same steps
  int order;      // of the items (MhaOrder)
  float* part;    // [2 CTAs][1 or 2][D / 4][128 rows][4]: sums of an item's share
  int4* record;   // [CTAs][2]: the item that begins in a CTA's share and ends in another's
  int64_t part_floats;  // room for parts
};

// What a CTA does at a time: a stationary tile, or a share of its steps.
struct BwdUnit {
  int head;        // of the stationary side
  int row0, rows;  // first stationary row, rows of the tile
  int r0, nq, nk;  // that row in its sequence, the sequence's rows
  int y0;          // the sequence's first streamed row
  int j0, tiles;   // streamed tiles [j0, j0 + tiles) of the sequence, for each head of the group
  int n0, steps;   // steps [n0, n0 + steps) of group * tiles, which come back to 0 at their end
  int part;        // slot of a share's partial sums, or -1
  int stat;        // keys stationary: slot of the sequence's first queries; else of this tile's
};

// An item with all its steps (which may be none); false: an empty slot.
template <bool KEYS>
__device__ __forceinline__ bool bwd_item(const BwdArgs& a, int slot, int head, BwdUnit& x) {
  MhaSeq seq;
  int index, tile;
  x.steps = 0;
  if (!mha_slot<kTile, KEYS>(a.s, slot, seq, index, tile)) return false;
  const int n = KEYS ? seq.nk : seq.nq;
  x.head = head;
  x.r0 = tile * kTile;
  x.row0 = (KEYS ? seq.k0 : seq.q0) + x.r0;
  x.rows = min(n - x.r0, kTile);
  x.nq = seq.nq;
  x.nk = seq.nk;
  x.y0 = KEYS ? seq.q0 : seq.k0;
  x.stat = mha_slot0(a.s.qb, index, seq.q0, kStatRows) + (KEYS ? 0 : tile);
  int lo, hi, none;
  if (KEYS) {
    mha_queries_of(a.s, seq, x.r0, lo, none);
    mha_queries_of(a.s, seq, x.r0 + x.rows - 1, none, hi);
  } else {
    mha_keys_of(a.s, seq, x.r0, lo, none);
    mha_keys_of(a.s, seq, x.r0 + x.rows - 1, none, hi);
  }
  x.j0 = lo / kTile;
  x.tiles = hi > lo ? (hi + kTile - 1) / kTile - x.j0 : 0;
  x.n0 = 0;
  x.steps = x.tiles * (KEYS ? a.s.group : 1);
  x.part = -1;
  return true;
}

// The units of this CTA, in order, by its producer warp.  First whole items, one in
// turn.  Then the steps of all other items, laid end to end head by head, in equal
// shares: a share begins and ends inside an item as a rule, whose parts are joined by
// mha_backward_join_kernel.  `scratch` holds a head's steps up to and with each slot
// (uneven items are shared out only where they are fewer than the SMs).
constexpr int kLeastSteps = 4;  // of a share
struct BwdUpto {
  const int64_t* scratch;
  int64_t per;  // of every slot, or -1: see scratch
  __device__ __forceinline__ int64_t operator()(int slot) const { return per >= 0 ? (slot + 1) * per : scratch[slot]; }
};
template <bool KEYS>
struct BwdWalk {
  const BwdArgs& a;
  int64_t* scratch;
  int lane;
  int turn = 0;    // of the whole items
  int next = 0;    // shared item
  bool shared = false;
  int64_t s, from, to;  // first step of `next`; this share's steps
  StepShares<BwdUpto> share;
  int units = 0;
  __device__ __forceinline__ BwdWalk(const BwdArgs& a_, int64_t* scratch_, int lane_)
      : a(a_), scratch(scratch_), lane(lane_) {}

  __device__ __forceinline__ void share_out() {
    shared = true;
    BwdUnit x;
    int per = -1;
    if (a.alike) {
      bwd_item<KEYS>(a, 0, 0, x);
      per = x.steps;
    } else {
      int64_t total = 0;
      for (int i = 0; i < a.slots; i += 32) {
        int64_t sum = 0;
        if (i + lane < a.slots) {
          bwd_item<KEYS>(a, i + lane, 0, x);
          sum = x.steps;
        }
#pragma unroll
        for (int off = 1; off < 32; off *= 2) {
          const int64_t t = __shfl_up_sync(0xffffffffu, (long long)sum, off);
          if (lane >= off) sum += t;
        }
        if (i + lane < a.slots) scratch[i + lane] = total + sum;
        total += __shfl_sync(0xffffffffu, (long long)sum, 31);
      }
      __syncwarp();
    }
    share = StepShares<BwdUpto>(BwdUpto{scratch, per}, a.heads, a.slots, a.full, gridDim.x, kLeastSteps);
    if ((int)blockIdx.x >= share.shares) {
      next = a.items;
      from = to = 0;
      return;
    }
    from = share.bound(blockIdx.x);
    to = share.bound(blockIdx.x + 1);
    share.begin(blockIdx.x, next, s);
    fence_proxy_async_smem();  // the scratch becomes a target of copies
    __syncwarp();
  }

  // Gradients of rows that nothing sees, or that see nothing.
  __device__ __forceinline__ void clear(const BwdUnit& x, int d) const {
    for (int w = 0; w < (KEYS ? 2 : 1); ++w) {
      __nv_bfloat16* out = w == 0 ? a.out1 : a.out2;
      const int64_t ld = w == 0 ? a.ld1 : a.ld2;
      for (int i = lane; out != nullptr && i < x.rows * (d / 8); i += 32) {
        const int64_t at = (int64_t)(x.row0 + i / (d / 8)) * ld + x.head * d + i % (d / 8) * 8;
        if (ACID_IN_BOUNDS(kSiteMha, at + 7, (KEYS ? a.s.nk : a.s.nq) * ld))
          *reinterpret_cast<uint4*>(out + at) = make_uint4(0, 0, 0, 0);
      }
    }
  }

  // The next unit with steps; false: none.
  __device__ __forceinline__ bool operator()(BwdUnit& x, int d) {
    int slot, head;
    while (!shared && turn * (int)gridDim.x < a.full) {
      next = mha_turn(turn++);
      if (next >= a.full) break;
      mha_item(a.order, a.slots, a.heads, next, slot, head);
      if (!bwd_item<KEYS>(a, slot, head, x)) continue;
      if (x.steps > 0) return true;
      clear(x, d);
    }
    if (a.full == a.items) return false;
    if (!shared) share_out();
    for (; next < a.items; ++next) {
      mha_item(a.order, a.slots, a.heads, next, slot, head);
      if (!bwd_item<KEYS>(a, slot, head, x)) continue;
      if (x.steps == 0) {
        clear(x, d);
        continue;
      }
      if (s >= to) return false;
      const int n = x.steps, n0 = (int)max((int64_t)0, from - s), n1 = (int)min((int64_t)n, to - s);
      // An item's tiles are taken round its end, the first one where the first share inside
      // the item begins: the CTAs that work on a head then stream the same tiles at a time,
      // all but one out of L2 (32760 queries, 301 and 512 keys, 12 x 128: 709 MB from HBM in
      // 140 us without, 220 MB in 121 us with it).
      int64_t c = (s - share.base) * share.shares / share.work;
      while (share.bound(c) < s) ++c;
      const int turn = share.bound(c) < s + n ? (int)(share.bound(c) - s) : 0;
      x.n0 = n0 >= turn ? n0 - turn : n0 - turn + n;
      x.steps = n1 - n0;
      if (n0 > 0 || n1 < n) x.part = 2 * blockIdx.x + (units > 0);
      if (n0 == 0 && n1 < n && lane == 0) {
        int last = blockIdx.x;
        while (share.bound(last + 1) < s + n) ++last;
        a.record[2 * blockIdx.x] = make_int4(x.rows, x.row0, x.head, x.part);
        a.record[2 * blockIdx.x + 1] = make_int4(last, 0, 0, 0);
      }
      ++units;
      s += n;
      ++next;
      return true;
    }
    return false;
  }
};

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
  static_assert(KEYS || NS == 2, "queries stationary: two regions");
  static constexpr int Y1S = D == 64 ? 4 : NS + 1, Y2S = D == 64 ? 4 : 2;
  static constexpr int SUMS = KEYS ? 2 : 1;
  static constexpr int OFF_X = 0, OFF_Y1 = 2 * T_BYTES, OFF_Y2 = OFF_Y1 + Y1S * T_BYTES;
  static constexpr int OFF_STAT = OFF_Y2 + Y2S * T_BYTES;
  static constexpr int UNITS = 4, UNIT_BYTES = 64;
  static constexpr int OFF_UNIT = OFF_STAT + (KEYS ? Y1S * kStatBytes : 0);
  static constexpr int OFF_BAR = OFF_UNIT + UNITS * UNIT_BYTES;
  static constexpr int SMEM = OFF_BAR + 512 + 1024;
  static_assert(SMEM <= 227 * 1024, "shared memory");
  static constexpr uint32_t S_COL = 0, DP_COL = NS * 128, SUM_COL = DP_COL + 128;
  static_assert(SUM_COL + SUMS * D <= 512, "tensor memory");
  static constexpr uint32_t TMEM_COLS = 512;
};

template <class C>
struct BwdBars {
  uint64_t *unit_full, *x_full, *x_empty, *y1_full, *y1_empty, *y2_full, *y2_empty;
  uint64_t *s_full, *dp_full, *dp_read, *p_full, *ds_full, *sum_full, *sum_empty, *edge, *drain;
  uint32_t* tmem_slot;
  static constexpr int kCount = 2 + 2 * C::Y1S + 2 * C::Y2S + C::NS + 10 + C::UNITS;
  static_assert(kCount * 8 + 4 <= 512, "barrier area");
  __device__ __forceinline__ explicit BwdBars(uint8_t* at) {
    uint64_t* b = reinterpret_cast<uint64_t*>(at);
    auto take = [&](int n) { uint64_t* r = b; b += n; return r; };
    unit_full = take(C::UNITS);
    x_full = take(1);
    x_empty = take(1);
    y1_full = take(C::Y1S);
    y1_empty = take(C::Y1S);
    y2_full = take(C::Y2S);
    y2_empty = take(C::Y2S);
    s_full = take(C::NS);
    dp_full = take(1);
    dp_read = take(1);
    // (two each: the workers may be a step ahead of the MMA warp, which can be held up by a
    // tile that is still on its way)
    p_full = take(2);
    ds_full = take(2);
    sum_full = take(1);
    sum_empty = take(1);
    edge = take(1);
    drain = take(1);
    tmem_slot = reinterpret_cast<uint32_t*>(b);
  }
  __device__ __forceinline__ void init() const {
    for (int i = 0; i < C::UNITS; ++i) mbar_init(&unit_full[i], 1);
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
    for (int i = 0; i < 2; ++i) {
      mbar_init(&p_full[i], kWorkers);
      mbar_init(&ds_full[i], kWorkers);
    }
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

// 16 columns of 32-bit registers a lane to tensor memory.
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(
          taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

// Four consecutive floats as two packed pairs.  (Through a generic pointer, which is
// what the aligned base of dynamic shared memory is to the compiler, the same loads
// take the path of global memory: keys stationary, 4726 rows, 30 x 64 348 us instead of
// 305.)
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

// 64 bytes of a row, a lane's own, by whole sectors where the address allows it.
__device__ __forceinline__ void store_64_bytes(void* p, const uint32_t* w) {
  if ((reinterpret_cast<uintptr_t>(p) & 31) == 0) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(static_cast<uint8_t*>(p) + 32 * i),
                   "r"(w[8 * i]), "r"(w[8 * i + 1]), "r"(w[8 * i + 2]), "r"(w[8 * i + 3]), "r"(w[8 * i + 4]),
                   "r"(w[8 * i + 5]), "r"(w[8 * i + 6]), "r"(w[8 * i + 7])
                   : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      static_cast<uint4*>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  }
}

// Columns [lo, hi) of 32 as bits.
__device__ __forceinline__ uint32_t column_bits(int lo, int hi) {
  lo = max(lo, 0);
  hi = min(hi, 32);
  return lo < hi ? (0xffffffffu >> (32 - hi)) & (0xffffffffu << lo) : 0u;
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
  int4* const entries = reinterpret_cast<int4*>(smem + C::OFF_UNIT);
  auto entry = [&](int n) { return entries + n % C::UNITS * (C::UNIT_BYTES / 16); };
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
  if (threadIdx.x == 0 && a.full < a.items) a.record[2 * blockIdx.x] = make_int4(0, 0, 0, 0);

  if (warp == 0) {  // -------------------------------------------- TMA producer
    bool ok = true;
    int y1_done = 0, y2_done = 0, x_done = 0, edges = 0, g = 0;
    BwdWalk<KEYS> walk(a, reinterpret_cast<int64_t*>(sY1), lane);
    BwdUnit x;
    for (; ok; ++x_done) {
      const bool more = walk(x, D);
      if (lane == 0) {
        int4* e = entry(x_done);
        e[0] = make_int4(more ? x.steps : 0, x.head, x.row0, x.rows);
        e[1] = make_int4(x.r0, x.nq, x.nk, x.part);
        e[2] = make_int4(x.j0, x.tiles, more ? x.n0 % x.tiles : 0, x.stat);
        mbar_arrive(&bar.unit_full[x_done % C::UNITS]);
      }
      if (!more) break;
      if (x_done > 0 && !mbar_wait_warp(bar.x_empty, (x_done - 1) & 1)) { ok = false; break; }
      if (lane == 0) {
        mbar_expect_tx(bar.x_full, 2 * C::T_BYTES);
        for (int c = 0; c < C::CH; ++c) {
          tma_load_2d(sX + c * C::CHUNK, &tmX1, bar.x_full, x.head * D + c * 64, x.row0);
          tma_load_2d(sX + C::T_BYTES + c * C::CHUNK, &tmX2, bar.x_full, x.head * D + c * 64, x.row0);
        }
      }
      const int rows = KEYS ? x.nq : x.nk, all = KEYS ? a.s.nq : a.s.nk;
      int jt = x.n0 % x.tiles, head = KEYS ? x.head * a.s.group + x.n0 / x.tiles : x.head / a.s.group;
      const int heads_end = (x.head + 1) * a.s.group;  // of a key head's queries
      for (int i = 0; ok && i < x.steps; ++i, ++g) {
        const int j = x.j0 + jt;
        const int valid = rows - j * kTile, row = x.y0 + j * kTile;
        const bool clear = valid < kTile && x.y0 + rows < all;
        // (the statistics of a tile's queries come with it: one kilobyte)
        auto load = [&](uint8_t* dst, const CUtensorMap* map, uint64_t* full, uint8_t* stat_dst) -> bool {
          uint64_t* to = clear ? bar.edge : full;
          if (lane == 0) {
            mbar_expect_tx(to, C::T_BYTES + (stat_dst != nullptr ? kStatBytes : 0));
            for (int c = 0; c < C::CH; ++c) tma_load_2d(dst + c * C::CHUNK, map, to, head * D + c * 64, row);
            if (stat_dst != nullptr) {
              const int64_t at = mha_stat_offset(head, a.stat_slots, x.stat + j);
              const bool in = ACID_IN_BOUNDS(kSiteMha, at + 2 * kStatRows - 1, mha_stat_offset(a.s.heads, a.stat_slots, 0));
              bulk_load(stat_dst, a.stats + (in ? at : 0), kStatBytes, to);  // (the barrier counts its bytes)
            }
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
        if (++jt == x.tiles) {
          jt = 0;
          if (KEYS && ++head == heads_end) head -= a.s.group;
        }
      }
    }
    if (!ok && lane == 0) {  // a wait ran out: the loads issued so far have landed before the CTA leaves
      mbar_wait(bar.x_full, x_done & 1);  // (of a unit whose load was not issued: runs out too)
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
    // Conditions that depend on a unit are votes here and in the workers: behind a branch that
    // the compiler does not know to be the same in all lanes descriptors, ring slots and
    // counters leave the uniform registers (dq 32760 rows, 12 x 128 5660 us instead of 5271;
    // 4726 rows, 30 x 64 dk and dv 276 instead of 267, dq 214 instead of 198).
    for (int units = 0, g = 0; ok; ++units) {
      if (!mbar_wait_warp(&bar.unit_full[units % C::UNITS], (units / C::UNITS) & 1)) { ok = false; break; }
      const int steps = static_cast<const volatile int*>(&entry(units)->x)[0];
      auto has = [&](int i) -> bool { return __any_sync(0xffffffffu, i < steps); };
      if (!has(0)) break;
      if (!mbar_wait_warp(bar.x_full, units & 1)) { ok = false; break; }
      auto scores = [&](int gs) -> bool {  // S of step gs
        if (!mbar_wait_warp(&bar.y1_full[gs % C::Y1S], (gs / C::Y1S) & 1)) return false;
        tc_fence_after();
        if (leader) {
          mma_scores<C>(tmem + C::S_COL + (gs % C::NS) * 128, x1, at(y1k, gs % C::Y1S));
          mma_commit(&bar.s_full[gs % C::NS]);
        }
        __syncwarp();
        return true;
      };
      auto grads = [&](int gs, bool last) -> bool {  // dP of step gs; last: of the unit
        if (!mbar_wait_warp(&bar.y2_full[gs % C::Y2S], (gs / C::Y2S) & 1)) return false;
        tc_fence_after();
        if (leader) {
          mma_scores<C>(tmem + C::DP_COL, x2, at(y2k, gs % C::Y2S));
          mma_commit(bar.dp_full);
          if (!KEYS) mma_commit(&bar.y2_empty[gs % C::Y2S]);
          if (last) mma_commit(bar.x_empty);
        }
        __syncwarp();
        return true;
      };
      bool more = has(1), first = true;  // a step behind this one
      ok = scores(g) && grads(g, !more) && (C::NS == 1 || !more || scores(g + 1));
      if (ok && units > 0) ok = mbar_wait_warp(bar.sum_empty, (units - 1) & 1);
      for (int i = 0; ok; ++i, ++g) {
        const bool more2 = has(i + 2);
        if constexpr (KEYS) {
          // dv += P^T g, over S; then the next S may take the region
          if (!mbar_wait_warp(&bar.p_full[g & 1], (g >> 1) & 1)) { ok = false; break; }
          tc_fence_after();
          if (leader) {
            mma_sum<C>(tmem + C::SUM_COL + D, tmem + C::S_COL + (g % C::NS) * 128, at(y2m, g % C::Y2S), !first);
            mma_commit(&bar.y2_empty[g % C::Y2S]);
          }
          __syncwarp();
          if ((C::NS == 1 ? more : more2) && !scores(g + C::NS)) { ok = false; break; }
          if (!mbar_wait_warp(&bar.ds_full[g & 1], (g >> 1) & 1)) { ok = false; break; }
          tc_fence_after();
          if (leader) {
            mma_sum<C>(tmem + C::SUM_COL, tmem + C::DP_COL, at(y1m, g % C::Y1S), !first);
            mma_commit(&bar.y1_empty[g % C::Y1S]);
            if (!more) mma_commit(bar.sum_full);
          }
          __syncwarp();
          if (more && !grads(g + 1, !more2)) { ok = false; break; }
        } else {
          // the next dP as soon as this one has been read; dq += dS k, over S
          if (more) {
            if (!mbar_wait_warp(bar.dp_read, g & 1) || !grads(g + 1, !more2)) { ok = false; break; }
          }
          if (!mbar_wait_warp(&bar.ds_full[g & 1], (g >> 1) & 1)) { ok = false; break; }
          tc_fence_after();
          if (leader) {
            mma_sum<C>(tmem + C::SUM_COL, tmem + C::S_COL + (g % C::NS) * 128, at(y1m, g % C::Y1S), !first);
            mma_commit(&bar.y1_empty[g % C::Y1S]);
            if (!more) mma_commit(bar.sum_full);
          }
          __syncwarp();
          if (more2 && !scores(g + C::NS)) { ok = false; break; }
        }
        first = false;
        if (!more) {
          ++g;
          break;
        }
        more = more2;
      }
    }
    if (!ok && leader) drain_mmas(bar.drain);
  } else {  // ------------------------------------------- workers
    // Warps 2-5 have the first 64 streamed rows (columns) of a step, warps 6-9 the others;
    // a thread has one stationary row, its TMEM lane.
    const int half = (warp - 2) >> 2, q = warp & 3, r = q * 32 + lane;
    const uint32_t base = tmem + ((uint32_t)(q * 32) << 16);
    const uint64_t sc2 = f2_pack(a.scale_log2, a.scale_log2);
    bool ok = true;
    int g = 0, steps = 0;
    float nlse = 0.f, ndelta = 0.f;
    // the unit's steps; queries stationary: its rows' statistics are on their way
    auto fetch = [&](int n) -> bool {
      if (!mbar_wait(&bar.unit_full[n % C::UNITS], (n / C::UNITS) & 1)) return false;
      steps = entry(n)[0].x;
      if (!KEYS && steps > 0) {
        const float* st = a.stats + mha_stat_offset(entry(n)[0].y, a.stat_slots, entry(n)[2].w);
        if (ACID_IN_BOUNDS(kSiteMha, st + kStatRows + r - a.stats, mha_stat_offset(a.s.heads, a.stat_slots, 0))) {
          nlse = st[r];
          ndelta = st[kStatRows + r];
        }
      }
      return true;
    };
    ok = __all_sync(0xffffffffu, fetch(0));
    for (int n = 0; ok && __any_sync(0xffffffffu, steps > 0); ++n) {
      const int4 e0 = entry(n)[0], e1 = entry(n)[1], e2 = entry(n)[2];
      const int rows = e0.w, part = e1.w;
      const MhaSeq seq{0, e1.y, 0, e1.z};
      auto seen = [&](int row, int& lo, int& hi) {
        if (KEYS) mha_queries_of(a.s, seq, e1.x + min(row, rows - 1), lo, hi);
        else mha_keys_of(a.s, seq, e1.x + min(row, rows - 1), lo, hi);
      };
      int lo, hi, all_lo, all_hi, none;
      seen(r, lo, hi);
      seen(0, none, all_hi);
      seen(kTile - 1, all_lo, none);
      // One step; MASK: some row does not see some streamed row.
      auto step = [&](int cc, auto mask) -> bool {
        constexpr bool MASK = decltype(mask)::value;
        uint32_t bits[2] = {~0u, ~0u};
        if (MASK) {
          const int first = cc + half * 64;
          bits[0] = column_bits(lo - first, hi - first);
          bits[1] = column_bits(lo - first - 32, hi - first - 32);
        }
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
        if constexpr (!KEYS && MASK) {  // (32 columns at a time: with the masks' registers more would spill)
          if (!mbar_wait(bar.dp_full, g & 1)) return false;
          tc_fence_after();
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            uint32_t pk[32];
            tmem_ld32(dp_at + 32 * k, reinterpret_cast<uint32_t*>(dp));
            tmem_wait_ld();
            if (k == 1) {
              tc_fence_before();
              mbar_arrive(bar.dp_read);
            }
#pragma unroll
            for (int c = 0; c < 32; ++c) p[32 * k + c] = bits[k] >> c & 1 ? ex2_approx(p[32 * k + c]) : 0.f;
#pragma unroll
            for (int c = 0; c < 32; c += 2) {
              float v0, v1;
              f2_unpack(f2_mul(f2_pack(p[32 * k + c], p[32 * k + c + 1]),
                               f2_add(f2_pack(dp[c], dp[c + 1]), f2_pack(ndelta, ndelta))), v0, v1);
              pk[c / 2] = pack_bf16(v0, v1);
            }
            tmem_st16(s_at + 16 * k, pk);
          }
          tmem_wait_st();
          tc_fence_before();
          mbar_arrive(&bar.ds_full[g & 1]);
          return true;
        }
        if (!KEYS && !read_dp()) return false;
#pragma unroll
        for (int c = 0; c < 64; ++c) {
          p[c] = ex2_approx(p[c]);
          if (MASK && !(bits[c / 32] >> (c % 32) & 1)) p[c] = 0.f;
        }
        if constexpr (KEYS) {
          uint32_t pk[32];
#pragma unroll
          for (int c = 0; c < 32; ++c) pk[c] = pack_bf16(p[2 * c], p[2 * c + 1]);
          tmem_st32(s_at, pk);
          tmem_wait_st();
          tc_fence_before();
          mbar_arrive(&bar.p_full[g & 1]);
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
          pk[c / 2] = pack_bf16(v[0], v[1]);
          pk[c / 2 + 1] = pack_bf16(v[2], v[3]);
        }
        tmem_st32(KEYS ? dp_at : s_at, pk);
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&bar.ds_full[g & 1]);
        return true;
      };
      const int begin0 = e2.x * kTile, end0 = begin0 + e2.y * kTile;
      int cc = begin0 + e2.z * kTile;
      for (int i = 0; __any_sync(0xffffffffu, i < steps); ++i, ++g) {
        const int c0 = cc;
        // (streamed queries behind the sequence have probability 0 by their statistics)
        const bool plain = c0 >= all_lo && (c0 + kTile <= all_hi || (KEYS && all_hi == seq.nq));
        if (!(__any_sync(0xffffffffu, plain) ? step(cc, std::false_type{}) : step(cc, std::true_type{}))) {
          ok = false;
          break;
        }
        cc = cc + kTile == end0 ? begin0 : cc + kTile;
      }
      // ------------------------------------------------ sums
      if (ok) ok = fetch(n + 1) && mbar_wait(bar.sum_full, n & 1);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      constexpr int kChunks = C::SUMS * D / 64;  // of 32 columns, for each half
#pragma unroll 1
      for (int k = 0; k < kChunks; ++k) {
        const int w = (half * kChunks + k) / (D / 32), c = (half * kChunks + k) % (D / 32) * 32;
        __nv_bfloat16* out = w == 0 ? a.out1 : a.out2;
        const int64_t ld = w == 0 ? a.ld1 : a.ld2;
        const float by = w == 0 ? a.scale : 1.0f;
        uint32_t o[32];
        tmem_ld32(base + C::SUM_COL + w * D + c, o);
        tmem_wait_ld();
        if (k == kChunks - 1) {  // the sums have been read: the next unit's may begin
          tc_fence_before();
          mbar_arrive(bar.sum_empty);
        }
        if (__any_sync(0xffffffffu, part >= 0)) {
          float* to = a.part + (((int64_t)part * C::SUMS + w) * (D / 4) + c / 4) * (kTile * 4) + r * 4;
          if (!ACID_IN_BOUNDS(kSiteMha, to + 7 * kTile * 4 + 3 - a.part, a.part_floats)) continue;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            *reinterpret_cast<uint4*>(to + i * kTile * 4) = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
          continue;
        }
        const int64_t at = (int64_t)(e0.z + r) * ld + e0.y * D + c;
        if (r >= rows || out == nullptr || !ACID_IN_BOUNDS(kSiteMha, at + 31, (KEYS ? a.s.nk : a.s.nq) * ld)) continue;
        uint32_t w16[16];
#pragma unroll
        for (int i = 0; i < 16; ++i)
          w16[i] = pack_bf16(__uint_as_float(o[2 * i]) * by, __uint_as_float(o[2 * i + 1]) * by);
        store_64_bytes(out + at, w16);
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

// Adds the parts of the items that lie in several shares, in the shares' order: the
// first in the share where the item begins, the others the first units of theirs.  A
// thread has 16 columns of a row.
template <int D, bool KEYS>
__global__ void __launch_bounds__(256) mha_backward_join_kernel(const __grid_constant__ BwdArgs a) {
  constexpr int SUMS = KEYS ? 2 : 1;
  pdl_wait();
  const int cta = blockIdx.x, row = threadIdx.x & 127;
  const int4 e = a.record[2 * cta];  // {rows, row0, head, part}
  if (row >= e.x) return;            // (no rows: no such item)
  const int last = a.record[2 * cta + 1].x;
  const int idx = blockIdx.y * 2 + (threadIdx.x >> 7);  // 16 columns, of dk and then dv
  const int w = idx / (D / 16), c = idx % (D / 16) * 16;
  __nv_bfloat16* out = w == 0 ? a.out1 : a.out2;
  if (out == nullptr) return;
  constexpr int64_t kPart = (int64_t)SUMS * (D / 4) * (kTile * 4);
  const float* p = a.part + (int64_t)idx * (kTile * 16) + row * 4;
  if (!ACID_IN_BOUNDS(kSiteMha, p + max(e.w, 2 * last) * kPart + 3 * kTile * 4 + 3 - a.part, a.part_floats)) return;
  float4 sum[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) sum[k] = *reinterpret_cast<const float4*>(p + e.w * kPart + k * kTile * 4);
  for (int s = cta + 1; s <= last; ++s) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float4 v = *reinterpret_cast<const float4*>(p + 2 * s * kPart + k * kTile * 4);
      sum[k].x += v.x;
      sum[k].y += v.y;
      sum[k].z += v.z;
      sum[k].w += v.w;
    }
  }
  const float by = w == 0 ? a.scale : 1.0f;
  const int64_t ld = w == 0 ? a.ld1 : a.ld2, at = (int64_t)(e.y + row) * ld + e.z * D + c;
  if (!ACID_IN_BOUNDS(kSiteMha, at + 15, (int64_t)(KEYS ? a.s.nk : a.s.nq) * ld)) return;
  auto two = [&](const float4& v) { return make_uint2(pack_bf16(v.x * by, v.y * by), pack_bf16(v.z * by, v.w * by)); };
#pragma unroll
  for (int k = 0; k < 4; k += 2) {
    const uint2 lo = two(sum[k]), hi = two(sum[k + 1]);
    *reinterpret_cast<uint4*>(out + at + 4 * k) = make_uint4(lo.x, lo.y, hi.x, hi.y);
  }
}

// Which items go to the CTAs whole.  Fewer items than SMs: none, all their steps are
// shared out evenly.  More: the CTAs take whole items, of one head after the other, so
// that those at work at a time stream the same tiles out of L2 (8190 rows, 24 on 8 heads,
// windows of five frames: 255 us, shared out evenly head by head 284); the last, partial
// wave is shared out where all items are alike.  With sequences and windows lengths
// differ, and many items even out.  Items of a few steps stay whole: a join takes as
// long as three of them.
struct BwdPlan {
  int slots, items, full;
  bool alike;
  int order;
};
BwdPlan bwd_plan(const MhaShape& s, int d, bool keys, int sms) {
  BwdPlan p;
  const bool bounded = (keys ? s.kb : s.qb) != nullptr;
  p.slots = mha_slots(keys ? s.nk : s.nq, s.seqs, bounded, kTile);
  p.items = p.slots * (keys ? s.kv_heads : s.heads);
  p.alike = s.qb == nullptr && s.kb == nullptr && s.frame == 0;
  const int64_t steps = ((int64_t)(keys ? s.nq : s.nk) / s.seqs + kTile - 1) / kTile * (keys ? s.group : 1);
  p.full = p.items;
  p.order = kByHead;
  if (steps > 2 * kLeastSteps) {
    if (p.items < sms) p.full = 0;
    else if (p.alike) p.full = p.items / sms * sms;
  }
  if (p.full == p.items) p.order = mha_order(s, d, keys, keys);
  return p;
}
size_t bwd_part_bytes(const BwdPlan& p, int sms, int sums, int d) {
  return p.full < p.items ? (size_t)sms * (2 * sums * kTile * d * sizeof(float) + 2 * sizeof(int4)) : 0;
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
  const int sms = num_sms();
  const BwdPlan p = bwd_plan(m, D, KEYS, sms);
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
  a.items = p.items;
  a.full = p.full;
  a.alike = p.alike;
  a.order = p.order;
  const bool shared = p.full < p.items;
  const int ctas = shared ? sms : std::min(p.items, sms);
  a.part = static_cast<float*>(x.part);
  a.part_floats = (int64_t)sms * 2 * C::SUMS * kTile * D;
  a.record = reinterpret_cast<int4*>(a.part + a.part_floats);
  launch_pdl(mha_backward_kernel<C>, ctas, kThreads, C::SMEM, s, KEYS ? tk : tq, KEYS ? tv : tg, KEYS ? tq : tk,
             KEYS ? tg : tv, a);
  ACID_CHECK_LAUNCH();
  if (shared) {
    launch_pdl(mha_backward_join_kernel<D, KEYS>, dim3(ctas, C::SUMS * D / 32), 256, 0, s, a);
    ACID_CHECK_LAUNCH();
  }
  return ACID_OK;
}

}  // namespace

size_t mha_backward_tc_bytes(const MhaArgs& x) {
  const int sms = num_sms();
  return std::max(bwd_part_bytes(bwd_plan(x.shape, x.head_dim, true, sms), sms, 2, x.head_dim),
                  bwd_part_bytes(bwd_plan(x.shape, x.head_dim, false, sms), sms, 1, x.head_dim));
}

acid_status mha_backward_tc(const MhaArgs& x, cudaStream_t s) {
  if (x.dk != nullptr || x.dv != nullptr) ACID_TRY(x.head_dim == 128 ? (launch<128, true>(x, s)) : (launch<64, true>(x, s)));
  if (x.dq != nullptr) ACID_TRY(x.head_dim == 128 ? (launch<128, false>(x, s)) : (launch<64, false>(x, s)));
  return ACID_OK;
}

}  // namespace acid
