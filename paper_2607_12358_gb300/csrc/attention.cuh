// The pieces of the tcgen05 attention kernels: tile and ring layout, barriers, the
// softmax of a tile and the MMAs of a step.  What a kernel does with them stands
// with the kernels (attention.cu, mha_forward.cu).
#pragma once

#include <cudaTypedefs.h>
#include <math.h>

#include "common.cuh"
#include "internal.h"

namespace acid {

acid_status make_tmap_bf16(CUtensorMap* map, const void* base, int64_t rows, int64_t cols, int64_t ld, int box_rows);
acid_status make_tmap_bf16_box(CUtensorMap* map, const void* base, int64_t rows, int64_t cols, int64_t ld,
                               int box_cols, int box_rows, CUtensorMapSwizzle swizzle);

namespace {

constexpr int kTileQ = 128;  // query rows per tile (two tiles per CTA)
constexpr int kBQ = 2 * kTileQ;
constexpr int kAttnThreads = 320;
constexpr float kRescaleLog2 = 8.0f, kRescale = 256.0f;
constexpr int kAttnPartCtas = kAttnSplitCtas;  // CTAs of a split tail wave (partials workspace capacity)

// Head dim and keys per K/V tile of a kernel.
template <int HEAD_DIM, int KEYS>
struct AttnCfg {
  static constexpr int D = HEAD_DIM, BKV = KEYS;
  // S regions in TMEM.  Step n of a CTA (2 * key-tile step + query tile: the
  // tiles alternate) uses region n % NB, and S(n + NB) is issued right after
  // PV(n), which reads P(n) from it.  Head dim 128: S and O of both query tiles
  // fill TMEM.  Head dim 64: O needs half the columns, and a third region lets
  // the tensor cores run ahead of the softmax warps, which set the pace at this
  // head dim: a step costs them about 630 clocks whatever its keys and 9.4 more
  // per key (4726 tokens, 30 heads: 197.6 us in 64-key tiles on four regions,
  // 163.1 in 96-key tiles on four, 146.6 in 128-key tiles on these three).
  // 64-key tiles are for the shortest key ranges, where starting and ending
  // items weighs most: 256 columns, two CTAs on an SM.
  static constexpr int CTAS_PER_SM = BKV == 64 ? 2 : 1;
  static constexpr int NB = D <= 64 && BKV == 128 ? 3 : 2;
  static constexpr int KVS = NB == 3 ? 4 : 2;        // K and V ring depth
  // Whether a tile's row max is formed before its exponentials or only where the
  // row sum asks for it (softmax_tile).  At head dim 128 the MMAs and power set
  // the pace and the two take the same time; two CTAs on an SM leave too few
  // registers to keep a row until its sum is known.
  static constexpr bool MAX_FIRST = !(D == 64 && BKV == 128);
  static constexpr int CH = D / 64;                  // 64-column chunks per row
  static constexpr int CHUNK_Q = 128 * 128;          // 128 rows x 128 bytes
  static constexpr int CHUNK_KV = BKV * 128;         // BKV rows x 128 bytes
  static constexpr int T_BYTES = CH * CHUNK_Q;       // one 128-row tile of Q
  static constexpr int KV_BYTES = CH * CHUNK_KV;     // one K or V tile
  static constexpr int OFF_Q = 0;                    // Q_a, Q_b
  static constexpr int OFF_K = OFF_Q + 2 * T_BYTES;  // rings
  static constexpr int OFF_V = OFF_K + KVS * KV_BYTES;
  static constexpr int OFF_BAR = OFF_V + KVS * KV_BYTES;
  static constexpr int BAR_BYTES = 512;
  static constexpr int SMEM = OFF_BAR + BAR_BYTES + 1024;
  // attn_persist_kernel adds the output staging: per softmax warp two
  // 32-row x 32-column bf16 boxes (64-byte swizzle) for TMA stores
  static constexpr int STAGE_BOX = 32 * 64;
  static constexpr int OFF_STAGE_P = OFF_V + KVS * KV_BYTES;
  static constexpr int OFF_BAR_P = OFF_STAGE_P + 8 * 2 * STAGE_BOX;
  static constexpr int SMEM_P = OFF_BAR_P + BAR_BYTES + 1024;
  // TMEM columns: the S regions (P over the first BKV / 2 columns of each), O_a, O_b
  static constexpr uint32_t O_COL = NB * BKV, TMEM_COLS = O_COL + 2 * D;
  static_assert(TMEM_COLS * CTAS_PER_SM == 512, "the CTAs of an SM take all of TMEM");
  __host__ __device__ static constexpr uint32_t o_col(int t) { return O_COL + t * D; }
  // Region of step g of tile t, and the parity of its use.
  static __device__ __forceinline__ int sb(int t, int g) { return NB == 2 ? t : (2 * g + t) % NB; }
  static __device__ __forceinline__ uint32_t sp(int t, int g) { return (uint32_t)(NB == 2 ? g : (2 * g + t) / NB) & 1; }
  static __device__ __forceinline__ int slot(int g) { return g & (KVS - 1); }
  static __device__ __forceinline__ uint32_t round(int g) { return (uint32_t)(g / KVS); }
};

// The barriers of a CTA.
template <class C>
struct AttnBars {
  uint64_t *q_full, *q_empty;  // [2] per query tile
  uint64_t *k_full, *k_empty, *v_full, *v_empty;  // [KVS]
  uint64_t *s_full, *p_full, *pv_done;  // [NB] per S region
  uint64_t* drain;  // failure path: the MMAs issued so far have completed
  uint32_t* tmem_slot;
  static constexpr int kCount = 4 + 4 * C::KVS + 3 * C::NB + 1;
  static_assert(kCount * 8 + 4 <= C::BAR_BYTES, "barrier area");
  __device__ __forceinline__ explicit AttnBars(uint8_t* at) {
    uint64_t* b = reinterpret_cast<uint64_t*>(at);
    auto take = [&](int n) { uint64_t* r = b; b += n; return r; };
    q_full = take(2);
    q_empty = take(2);
    k_full = take(C::KVS);
    k_empty = take(C::KVS);
    v_full = take(C::KVS);
    v_empty = take(C::KVS);
    s_full = take(C::NB);
    p_full = take(C::NB);
    pv_done = take(C::NB);
    drain = take(1);
    tmem_slot = reinterpret_cast<uint32_t*>(b);
  }
  __device__ __forceinline__ void init() const {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&q_full[i], 1);
      mbar_init(&q_empty[i], 1);
    }
    for (int i = 0; i < C::KVS; ++i) {
      mbar_init(&k_full[i], 1);
      mbar_init(&k_empty[i], 1);
      mbar_init(&v_full[i], 1);
      mbar_init(&v_empty[i], 1);
    }
    for (int i = 0; i < C::NB; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&p_full[i], 128);
      mbar_init(&pv_done[i], 1);
    }
    mbar_init(drain, 1);
    mbar_fence_init();
  }
};

// Softmax of one key tile for this thread's query row (row r of tile t is
// TMEM lane r): waits for S_t, writes P_t = 2^(s * scale - m) over the S
// region as bf16 pairs, updates the running reference max m and sum l,
// rescales O_t when the reference moves, and hands P_t to the MMA warp.
// g: this tile's step count in the CTA; first: the row has no reference max yet (the
// item's first key tile, or no key seen so far);
// MASK: kNoMask, kTail (the keys of a partial last tile are those below hi) or
// kRange (those in [lo, hi), which may be none: the row's reference max then stays
// -inf and its probabilities are 0).
enum : int { kNoMask = 0, kTail = 1, kRange = 2 };
template <class C, int MASK>
__device__ __forceinline__ bool softmax_tile(const AttnBars<C>& bar, int t, int g, bool first, int lo, int hi,
                                             uint32_t s_base, uint32_t o_addr, float scale_log2, float& m_run,
                                             float& l_run) {
  const uint32_t s_addr = s_base + C::sb(t, g) * C::BKV;
  // The lanes of a warp wait on the same phase, so they give up together
  // (after the wait limit) and the warp-collective tcgen05.ld / st below stay
  // convergent; a vote here would rule out a phase that completes exactly at
  // the limit for some lanes only, but costs 2-3% in this loop.
  if (!mbar_wait(&bar.s_full[C::sb(t, g)], C::sp(t, g))) return false;
  tc_fence_after();
  float s[C::BKV];
#pragma unroll
  for (int c = 0; c < C::BKV / 32; ++c) tmem_ld32(s_addr + c * 32, reinterpret_cast<uint32_t*>(s + c * 32));
  tmem_wait_ld();
  bool resc = false;
  float f = 1.0f;
  if constexpr (MASK == kTail) {
#pragma unroll
    for (int i = 0; i < C::BKV; ++i)
      if (i >= hi) s[i] = -INFINITY;
  }
  // (after the scaling: a scale of 0 or less must not meet an infinity)
  auto mask_pair = [&](int i) {
    if constexpr (MASK == kRange) {
      if (2 * i < lo || 2 * i >= hi) s[2 * i] = -INFINITY;
      if (2 * i + 1 < lo || 2 * i + 1 >= hi) s[2 * i + 1] = -INFINITY;
    }
  };
  const uint64_t sc2 = f2_pack(scale_log2, scale_log2);
  const float mref = first ? 0.f : m_run;
  const uint64_t nm2 = f2_pack(-mref, -mref);
  auto row_max = [](const float* m4) { return fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])); };
  auto shift = [&](float me) {
    const uint64_t sh2 = f2_pack(-me, -me);
#pragma unroll
    for (int i = 0; i < C::BKV / 2; ++i)
      f2_unpack(f2_add(f2_pack(s[2 * i], s[2 * i + 1]), sh2), s[2 * i], s[2 * i + 1]);
  };
  // P = 2^e as bf16 pairs over the first BKV/2 columns of S_t, and the row sum
  // as packed fp32 pairs
  auto exps = [&]() -> float {
    uint64_t acc0 = f2_pack(0.f, 0.f), acc1 = acc0;
#pragma unroll
    for (int half = 0; half < C::BKV / 64; ++half) {
      uint32_t pk[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        const float p0 = ex2_approx(s[half * 64 + 2 * i]), p1 = ex2_approx(s[half * 64 + 2 * i + 1]);
        if (i & 1)
          acc1 = f2_add(acc1, f2_pack(p0, p1));
        else
          acc0 = f2_add(acc0, f2_pack(p0, p1));
        pk[i] = pack_bf16(p0, p1);
      }
      tmem_st32(s_addr + half * 32, pk);
    }
    float a0, a1, b0, b1;
    f2_unpack(acc0, a0, a1);
    f2_unpack(acc1, b0, b1);
    return (a0 + a1) + (b0 + b1);
  };
  // e = s * scale - m_run in place (packed pairs; the first tile uses 0 as the
  // reference); the row max of e in four independent 3-input max chains on the
  // ALU pipe.  The P_t region is free here: the MMAs run in order, and S_t(g)
  // follows the PV that read it.  Lazy rescaling: the reference max moves only
  // on the first tile or when the row max exceeds it by more than 2^8; then e
  // is shifted in place.
  float ls;
  if constexpr (C::MAX_FIRST) {
    float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int i = 0; i < C::BKV / 2; ++i) {
      f2_unpack(f2_fma(f2_pack(s[2 * i], s[2 * i + 1]), sc2, nm2), s[2 * i], s[2 * i + 1]);
      mask_pair(i);
      m4[i & 3] = fmax3(m4[i & 3], s[2 * i], s[2 * i + 1]);
    }
    const float me = row_max(m4);
    if ((first && (MASK != kRange || me != -INFINITY)) || me > kRescaleLog2) {
      if (!first) {
        resc = true;
        f = ex2_approx(-me);
        l_run *= f;
      }
      m_run = mref + me;
      shift(me);
    }
    ls = exps();
  } else {
    // An element above 2^8 makes the row sum larger than 2^8 (or NaN), so the
    // max is formed on a row's first tile and then only for such a sum.  Where
    // it moves the reference, the warp writes its P again.  Without the max the
    // exponentials start as the scores are scaled: 4726 tokens, 30 heads 172.9 ->
    // 158.9 us (with 96-key tiles).  A row that moves at every tile pays its
    // exponentials twice: with scores that rise by 2^10 from tile to tile 290 us,
    // where the max first takes 207 to 228 (64-key tiles).  A flag that lets a
    // tile behind a move form its max first takes 211 there, but ordinary scores
    // 151 instead of 147 and peaked ones 171 instead of 162, so there is none.
    auto max_of_e = [&] {
      float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int i = 0; i < C::BKV / 2; ++i) m4[i & 3] = fmax3(m4[i & 3], s[2 * i], s[2 * i + 1]);
      return row_max(m4);
    };
#pragma unroll
    for (int i = 0; i < C::BKV / 2; ++i) {
      f2_unpack(f2_fma(f2_pack(s[2 * i], s[2 * i + 1]), sc2, nm2), s[2 * i], s[2 * i + 1]);
      mask_pair(i);
    }
    if (first) {
      m_run = max_of_e();
      if (MASK != kRange || m_run != -INFINITY) shift(m_run);
    }
    ls = exps();
    if (!first && !(ls <= kRescale)) {
      const float me = max_of_e();
      if (me > kRescaleLog2) {
        resc = true;
        f = ex2_approx(-me);
        l_run *= f;
        m_run += me;
        shift(me);
      }
    }
    if (__any_sync(0xffffffffu, resc)) {
      tmem_wait_st();  // the first P has been written
      ls = exps();
    }
  }
  l_run += ls;
  if (__any_sync(0xffffffffu, resc)) {
    // (no later use of that region can have completed: the MMAs of step (t, g) wait for this warp)
    if (!mbar_wait(&bar.pv_done[C::sb(t, g - 1)], C::sp(t, g - 1))) return false;
    tc_fence_after();
#pragma unroll 1
    for (int c = 0; c < C::D; c += 32) {
      uint32_t o[32];
      tmem_ld32(o_addr + c, o);
      tmem_wait_ld();
#pragma unroll
      for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
      tmem_st32(o_addr + c, o);
    }
  }
  tmem_wait_st();
  tc_fence_before();
  mbar_arrive(&bar.p_full[C::sb(t, g)]);
  return true;
}

// S_t = Q_t K^T for one key tile: D/16 MMAs (M128, N = BKV, K16) into TMEM
// column d; qdesc_t / kdesc_slot: shared-memory descriptors of Q_t and of the
// K ring slot (an operand at byte offset o is the descriptor plus o >> 4).
template <class C>
__device__ __forceinline__ void issue_s_mma(uint32_t d, uint64_t qdesc_t, uint64_t kdesc_slot) {
  constexpr uint32_t idesc_s = idesc_bf16_f32(128, C::BKV, false, false);
#pragma unroll
  for (int kk = 0; kk < C::D / 16; ++kk) {
    const uint64_t off_a = (uint64_t)(((kk >> 2) * C::CHUNK_Q + (kk & 3) * 32) >> 4);
    const uint64_t off_b = (uint64_t)(((kk >> 2) * C::CHUNK_KV + (kk & 3) * 32) >> 4);
    mma_bf16_ss(d, qdesc_t + off_a, kdesc_slot + off_b, idesc_s, kk != 0);
  }
}

// O_t (+)= P_t V for one key tile: BKV/16 MMAs (M128, N = D, K16), P_t from
// TMEM at column p (bf16 pairs over the S region), V MN-major from the ring
// slot; accumulate is false on an item's first key tile.
template <class C>
__device__ __forceinline__ void issue_pv_mma(uint32_t d, uint32_t p, uint64_t vdesc_slot, bool accumulate) {
  constexpr uint32_t idesc_o = idesc_bf16_f32(128, C::D, false, true);
#pragma unroll
  for (int kk = 0; kk < C::BKV / 16; ++kk)
    mma_bf16_ts(d, p + kk * 8, vdesc_slot + (uint64_t)((kk * 16 * 128) >> 4), idesc_o, accumulate || kk != 0);
}

// TMA loads of one K or V tile (D / 64 chunks of 64 columns) into a ring slot.
template <class C>
__device__ __forceinline__ void load_kv_tile(uint8_t* dst, const CUtensorMap* map, uint64_t* bar, int col, int row) {
  mbar_expect_tx(bar, C::KV_BYTES);
  for (int c = 0; c < C::CH; ++c) tma_load_2d(dst + c * C::CHUNK_KV, map, bar, col + c * 64, row);
}

// Failure path (a wait ran out): the producer waits, bounded, until the last K
// and V loads of each ring have landed, so that no copy writes into the shared
// memory of a CTA that has left; the MMA thread waits, bounded, for the MMAs it
// has issued before tensor memory is freed.  Never called on the normal path.
template <class C>
__device__ __noinline__ void drain_loads(const AttnBars<C>& bar, int nk, int nv) {
  for (int j = nk > C::KVS ? nk - C::KVS : 0; j < nk; ++j) mbar_wait(&bar.k_full[C::slot(j)], C::round(j) & 1);
  for (int j = nv > C::KVS ? nv - C::KVS : 0; j < nv; ++j) mbar_wait(&bar.v_full[C::slot(j)], C::round(j) & 1);
}
__device__ __noinline__ void drain_mmas(uint64_t* drain) {
  mma_commit(drain);
  mbar_wait(drain, 0);
}

// The MMA warp's commits and operands.
template <class C>
struct AttnMma {
  const AttnBars<C>& bar;
  uint32_t tmem;
  uint64_t qdesc, kdesc, vdesc;
  __device__ __forceinline__ AttnMma(const AttnBars<C>& b, uint32_t tm, uint8_t* sQ, uint8_t* sK, uint8_t* sV)
      : bar(b), tmem(tm) {
    // Descriptors are built once; an operand at byte offset o from a base is
    // the base descriptor plus o >> 4 (the 14-bit address field cannot
    // overflow: shared memory ends below 256 KB).
    qdesc = smem_desc_sw128(smem_u32(sQ), 16, 1024);
    kdesc = smem_desc_sw128(smem_u32(sK), 16, 1024);
    vdesc = smem_desc_sw128(smem_u32(sV), C::CHUNK_KV, 1024);
  }
  // S_t = Q_t K^T of step g into its S region of tile t
  __device__ __forceinline__ void s_step(int t, int g) const {
    issue_s_mma<C>(tmem + C::sb(t, g) * C::BKV, qdesc + (uint64_t)((t * C::T_BYTES) >> 4),
                   kdesc + (uint64_t)((C::slot(g) * C::KV_BYTES) >> 4));
    mma_commit(&bar.s_full[C::sb(t, g)]);
    if (t == 1) mma_commit(&bar.k_empty[C::slot(g)]);
  }
  // O_t += P_t V of step g; accumulate is false on an item's first key tile
  __device__ __forceinline__ void pv_step(int t, int g, bool accumulate) const {
    issue_pv_mma<C>(tmem + C::o_col(t), tmem + C::sb(t, g) * C::BKV,
                    vdesc + (uint64_t)((C::slot(g) * C::KV_BYTES) >> 4), accumulate);
    mma_commit(&bar.pv_done[C::sb(t, g)]);
    if (t == 1) mma_commit(&bar.v_empty[C::slot(g)]);
  }
};

}  // namespace
}  // namespace acid
