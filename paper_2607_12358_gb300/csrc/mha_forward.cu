// Attention with row sums in bf16 on tcgen05 (acid_mha_forward): the flash kernel of
// attention.cu over sequences, shared key heads and windows of frames.
//
// An item is two 128-row query tiles of one head and sequence; its key tiles are
// those that the 256 rows see.  A tile that every row of a query tile sees runs the
// softmax without a mask; the others mask each row by its own range of keys.  Roles
// and pipeline are those of attn_persist_kernel.
#include <algorithm>

#include "attention.cuh"
#include "mha.cuh"

namespace acid {

unsigned int take_device_error_mha_forward();
ACID_DEVICE_FLAG_READER(take_device_error_mha_forward)
BoundsRecord take_bounds_mha_forward();
ACID_BOUNDS_READER(take_bounds_mha_forward)

namespace {

struct FwdArgs {
  MhaShape s;
  __nv_bfloat16* out;
  float* lse;
  int64_t ldo;
  float scale_log2;
  int slots;   // of query-tile pairs
  int order;   // of the items (MhaOrder)
  int full;    // items that one CTA takes whole; the rest are split along their keys
  int splits;  // CTAs to a split item
  int units;
  float* part_o;   // [split units][256][D]: unnormalised output
  float* part_ml;  // [split units][256][2]: reference max and sum
  int64_t part_rows;  // rows of parts that the scratch has room for
};

constexpr int kBarBytes = 768;  // barriers, units

// What a CTA does at a time: an item, or a share of its key tiles.
struct FwdUnit {
  int head, q0, rows, q_end;  // first row of the pair, rows left in the sequence from there, its last row's successor
  int k0, nk, j0, tiles;      // first key row and keys of the sequence; key tiles [j0, j0 + tiles)
  int part;                   // slot of a split unit's partial result, or -1
  int tile;                   // of the sequence
  MhaSeq seq;
};

// False: nothing there (an empty slot).
template <class C>
__device__ __forceinline__ bool fwd_unit(const FwdArgs& a, int u, FwdUnit& x) {
  int item = u, split = 0, slot, index;
  x.part = -1;
  if (u >= a.full) {
    x.part = u - a.full;
    item = a.full + x.part / a.splits;
    split = x.part % a.splits;
  }
  mha_item(a.order, a.slots, a.s.heads, item, slot, x.head);
  if (!mha_slot<kBQ, false>(a.s, slot, x.seq, index, x.tile)) return false;
  const int r0 = x.tile * kBQ;
  x.q0 = x.seq.q0 + r0;
  x.rows = x.seq.nq - r0;
  x.q_end = x.seq.q0 + x.seq.nq;
  x.k0 = x.seq.k0;
  x.nk = x.seq.nk;
  int lo, hi, none;
  mha_keys_of(a.s, x.seq, r0, lo, none);
  mha_keys_of(a.s, x.seq, r0 + min(x.rows, kBQ) - 1, none, hi);
  x.j0 = lo / C::BKV;
  x.tiles = hi > lo ? (hi + C::BKV - 1) / C::BKV - x.j0 : 0;
  if (x.part >= 0) {
    const int first = (int)((int64_t)split * x.tiles / a.splits);
    x.tiles = (int)((int64_t)(split + 1) * x.tiles / a.splits) - first;
    x.j0 += first;
  }
  return true;
}
// A unit without key tiles: rows that see no key.  By the producer's warp.
template <class C>
__device__ __forceinline__ void write_empty(const FwdArgs& a, const FwdUnit& x, int lane) {
  const int rows = min(x.rows, kBQ);
  for (int r = lane; r < rows; r += 32) {
    if (x.part >= 0) {
      const int64_t at = (int64_t)x.part * kBQ + r;
      if (ACID_IN_BOUNDS(kSiteMha, at, a.part_rows)) *reinterpret_cast<float2*>(a.part_ml + at * 2) = make_float2(-INFINITY, 0.f);
    } else if (ACID_IN_BOUNDS(kSiteMha, x.head * (int64_t)a.s.nq + x.q0 + r, (int64_t)a.s.heads * a.s.nq)) {
      a.lse[(int64_t)x.head * a.s.nq + x.q0 + r] = -INFINITY;
    }
  }
  if (x.part >= 0) return;
  for (int i = lane; i < rows * (C::D / 8); i += 32) {
    const int64_t at = (int64_t)(x.q0 + i / (C::D / 8)) * a.ldo + x.head * C::D + i % (C::D / 8) * 8;
    if (ACID_IN_BOUNDS(kSiteMha, at + 7, (int64_t)a.s.nq * a.ldo))
      *reinterpret_cast<uint4*>(a.out + at) = make_uint4(0, 0, 0, 0);
  }
}

// The units of a CTA that have key tiles, as its producer warp finds them, in a ring in
// shared memory: {key tiles (0: no more units), head, q0, q_end}, {first query row, queries
// and keys of the sequence, first key tile}, {part}.  The other warps read what they need
// when they need it, and every branch that goes by it is a vote.  With each warp forming its
// units by itself, and branches on loaded values, which the compiler cannot know to be the
// same in all lanes, descriptors, ring slots and loop counts left the uniform registers for
// those beside a row's 128 scores: 4726 rows, 30 heads of 64 205 us instead of 164, 8192
// rows, 12 heads of 128 330 instead of 271 (of that, votes alone 170 to 164 and 303 to 271).
struct UnitRing {
  static constexpr int kEntries = 4, kBytes = kEntries * (48 + 16);
  int4* entries;
  uint64_t *full, *empty;
  __device__ __forceinline__ explicit UnitRing(uint8_t* at)
      : entries(reinterpret_cast<int4*>(at)),
        full(reinterpret_cast<uint64_t*>(at + kEntries * 48)),
        empty(full + kEntries) {}
  __device__ __forceinline__ void init() const {
    for (int i = 0; i < kEntries; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 9);  // eight softmax warps, the MMA warp
    }
  }
  __device__ __forceinline__ const volatile int* at(int n) const {
    return reinterpret_cast<const volatile int*>(entries + n % kEntries * 3);
  }
  __device__ __forceinline__ bool wait(int n) const { return mbar_wait_warp(&full[n % kEntries], (n / kEntries) & 1); }
  // By one lane, behind the warp's last read.
  __device__ __forceinline__ void done(int n) const { mbar_arrive(&empty[n % kEntries]); }
  // By the producer's warp: unit n, or that there is none.
  __device__ __forceinline__ bool publish(int n, bool any, const FwdUnit& x, int lane) const {
    if (n >= kEntries && !mbar_wait_warp(&empty[n % kEntries], (n / kEntries - 1) & 1)) return false;
    if (lane == 0) {
      int4* e = entries + n % kEntries * 3;
      e[0] = any ? make_int4(x.tiles, x.head, x.q0, x.q_end) : make_int4(0, 0, 0, 0);
      if (any) {
        e[1] = make_int4(x.tile * kBQ, x.seq.nq, x.nk, x.j0);
        e[2] = make_int4(x.part, 0, 0, 0);
      }
      mbar_arrive(&full[n % kEntries]);
    }
    __syncwarp();
    return true;
  }
};

// Rows [valid, ROWS) of a loaded tile (128-byte swizzled chunks of 64 columns) are
// set to zero: rows of another sequence, or of none, that a product over keys would
// meet with weight 0, and may hold anything.  By a whole warp.
template <int ROWS, int CHUNKS>
__device__ __forceinline__ void clear_rows(uint8_t* tile, int valid, int lane) {
  for (int c = 0; c < CHUNKS; ++c) {
    uint4* p = reinterpret_cast<uint4*>(tile + c * ROWS * 128);
    for (int i = valid * 8 + lane; i < ROWS * 8; i += 32) p[i] = make_uint4(0, 0, 0, 0);
  }
  fence_proxy_async_smem();
  __syncwarp();
}

template <class C>
__global__ void __launch_bounds__(kAttnThreads, C::CTAS_PER_SM)
    mha_forward_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                       const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmO,
                       const __grid_constant__ FwdArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sQ = smem + C::OFF_Q;
  uint8_t* sK = smem + C::OFF_K;
  uint8_t* sV = smem + C::OFF_V;
  const AttnBars<C> bar(smem + C::OFF_BAR_P);
  constexpr int kOffRing = (AttnBars<C>::kCount * 8 + 4 + 15) / 16 * 16;
  static_assert(kOffRing + UnitRing::kBytes + 8 <= kBarBytes, "barrier area");
  const UnitRing ring(smem + C::OFF_BAR_P + kOffRing);
  uint64_t* edge = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR_P + kBarBytes - 8);  // a V tile to be cleared
  static_assert(AttnBars<C>::kCount * 8 + 16 <= C::BAR_BYTES, "barrier area");

  const int warp = warp_index(), lane = threadIdx.x & 31;
  if (warp == 0 && lane == 0) {
    tma_prefetch_desc(&tmQ);
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
    tma_prefetch_desc(&tmO);
    mbar_init(edge, 1);
    ring.init();
    bar.init();
  }
  if (warp == 1) tmem_alloc(bar.tmem_slot, C::TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *bar.tmem_slot;
  pdl_wait();  // the set-up above overlaps the tail of the kernel before

  if (warp == 0) {  // -------------------------------------------- TMA producer
    bool ok = true;
    int k_done = 0, v_done = 0, edges = 0;
    FwdUnit x, next;
    int turn = 0, n = 0;  // n: the unit's number among those with key tiles
    auto find = [&](FwdUnit& y) -> bool {
      for (int u; (u = mha_turn(turn)) < a.units; ) {
        ++turn;
        if (!fwd_unit<C>(a, u, y)) continue;
        if (y.tiles > 0) return true;
        write_empty<C>(a, y, lane);
      }
      return false;
    };
    // a unit is published while the one before it is loaded, behind its first tile
    bool more = find(x);
    ok = ring.publish(0, more, x, lane);
    for (int g = 0; ok && more; x = next, ++n) {
      const int kcol = x.head / a.s.group * C::D;
      auto load_q = [&](int t) -> bool {
        if (n > 0 && !mbar_wait_warp(&bar.q_empty[t], (n - 1) & 1)) return false;
        if (lane == 0) {
          mbar_expect_tx(&bar.q_full[t], C::T_BYTES);
          for (int c = 0; c < C::CH; ++c)
            tma_load_2d(sQ + t * C::T_BYTES + c * C::CHUNK_Q, &tmQ, &bar.q_full[t], x.head * C::D + c * 64,
                        x.q0 + t * kTileQ);
        }
        return true;
      };
      if (!load_q(0)) { ok = false; break; }
      for (int j = 0; j < x.tiles; ++j, ++g) {
        const int st = C::slot(g), row = (x.j0 + j) * C::BKV;  // of the sequence
        const uint32_t round = C::round(g);
        if (round > 0 && !mbar_wait_warp(&bar.k_empty[st], (round - 1) & 1)) { ok = false; break; }
        if (lane == 0) load_kv_tile<C>(sK + st * C::KV_BYTES, &tmK, &bar.k_full[st], kcol, x.k0 + row);
        k_done = g + 1;
        if (j == 0 && !load_q(1)) { ok = false; break; }
        if (round > 0 && !mbar_wait_warp(&bar.v_empty[st], (round - 1) & 1)) { ok = false; break; }
        const int valid = x.nk - row;
        if (valid < C::BKV && x.k0 + x.nk < a.s.nk) {  // rows behind the sequence: P is 0 there, V must be finite
          if (lane == 0) load_kv_tile<C>(sV + st * C::KV_BYTES, &tmV, edge, kcol, x.k0 + row);
          if (!mbar_wait_warp(edge, edges++ & 1)) { ok = false; break; }
          clear_rows<C::BKV, C::CH>(sV + st * C::KV_BYTES, valid, lane);
          if (lane == 0) mbar_arrive(&bar.v_full[st]);
        } else if (lane == 0) {
          load_kv_tile<C>(sV + st * C::KV_BYTES, &tmV, &bar.v_full[st], kcol, x.k0 + row);
        }
        v_done = g + 1;
        if (j == 0) {
          more = find(next);
          if (!ring.publish(n + 1, more, next, lane)) { ok = false; break; }
        }
      }
    }
    // after a wait ran out: the last K and V loads of each ring have landed
    // (a tile on `edge` has been waited for; Q loads are waited for by the MMA warp)
    if (!ok && lane == 0) drain_loads<C>(bar, k_done, v_done);
  } else if (warp == 1) {  // ------------------------------------- MMA issuer
    const bool leader = elect_one();
    const AttnMma<C> mma(bar, tmem, sQ, sK, sV);
    // The unit whose S is to be issued next, and its tile js.  `last` keeps for the latest
    // 32 steps whether a unit ends there: PV runs up to two steps behind.  The query tile is
    // known where a step is issued, and with it the descriptors.
    int js = 0, ns = 0, tiles = 0, end = 0;  // end: steps that there are, so far
    bool more = false;
    uint32_t last = 0;
    auto read_unit = [&]() -> bool {
      if (!ring.wait(ns)) return false;
      tiles = ring.at(ns)[0];
      more = __any_sync(0xffffffffu, tiles > 0);
      if (leader) ring.done(ns);
      return true;
    };
    auto issue_s = [&](int t, int g) -> bool {
      if (!more) return true;
      if (t == 0 && !mbar_wait_warp(&bar.k_full[C::slot(g)], C::round(g) & 1)) return false;
      if (js == 0 && !mbar_wait_warp(&bar.q_full[t], ns & 1)) return false;
      tc_fence_after();
      const bool ends = __all_sync(0xffffffffu, js == tiles - 1);
      if (leader) {
        mma.s_step(t, g);
        if (ends) mma_commit(&bar.q_empty[t]);
      }
      __syncwarp();
      if (t == 0) {
        end = g + 1;
        last = (last & ~(1u << (g & 31))) | ((uint32_t)ends << (g & 31));
      } else if (!ends) {
        ++js;
      } else {
        js = 0;
        ++ns;
        return read_unit();
      }
      return true;
    };
    bool ok = read_unit();
#pragma unroll
    for (int n = 0; n < C::NB; ++n) ok = ok && issue_s(n & 1, n >> 1);
    bool first = true;
    for (int g = 0; ok && g < end; ++g) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (!mbar_wait_warp(&bar.p_full[C::sb(t, g)], C::sp(t, g))) { ok = false; break; }
        if (t == 0 && !mbar_wait_warp(&bar.v_full[C::slot(g)], C::round(g) & 1)) { ok = false; break; }
        tc_fence_after();
        if (leader) mma.pv_step(t, g, !first);
        __syncwarp();
        if (!issue_s((t + C::NB) & 1, g + (t + C::NB) / 2)) { ok = false; break; }
      }
      first = (last >> (g & 31)) & 1;
    }
    if (!ok && leader) drain_mmas(bar.drain);
  } else {  // ------------------- softmax: warps 2-5 tile a, 6-9 tile b
    const int t = (warp - 2) >> 2;
    const int q = warp & 3;
    const int r = t * kTileQ + q * 32 + lane;  // row of the pair
    const uint32_t lane_base = (uint32_t)(q * 32) << 16;
    const uint32_t s_base = tmem + lane_base;
    const uint32_t o_addr = tmem + lane_base + C::o_col(t);
    uint8_t* stage = smem + C::OFF_STAGE_P + (warp - 2) * 2 * C::STAGE_BOX;
    int n_st = 0, g = 0;
    bool ok = true;
    for (int n = 0;; ++n) {
      if (!ring.wait(n)) { ok = false; break; }
      const volatile int* e = ring.at(n);
      auto word = [&](int i) { return __shfl_sync(0xffffffffu, e[i], 0); };
      const int tiles = word(0);
      if (__any_sync(0xffffffffu, tiles == 0)) break;
      // keys that all rows of the query tile see
      const int r0 = word(4), last = word(5) - 1;
      const MhaSeq seq{0, last + 1, 0, word(6)};
      int all_lo, all_hi, none, c0 = word(7) * C::BKV;
      mha_keys_of(a.s, seq, min(r0 + t * kTileQ, last), none, all_hi);
      mha_keys_of(a.s, seq, min(r0 + t * kTileQ + kTileQ - 1, last), all_lo, none);
      float m_run = -INFINITY, l_run = 0.f;
      for (int j = 0; j < tiles; ++j, ++g, c0 += C::BKV) {
        const bool fresh = m_run == -INFINITY;
        bool ok_j;
        if (c0 >= all_lo && c0 + C::BKV <= all_hi) {
          ok_j = softmax_tile<C, kNoMask>(bar, t, g, fresh, 0, 0, s_base, o_addr, a.scale_log2, m_run, l_run);
        } else {  // the keys that this row sees (formed here, they are not kept through the other tiles)
          const int nq = e[5];
          int lo, hi;
          mha_keys_of(a.s, MhaSeq{0, nq, 0, e[6]}, min(e[4] + r, nq - 1), lo, hi);
          ok_j = softmax_tile<C, kRange>(bar, t, g, fresh, lo - c0, hi - c0, s_base, o_addr, a.scale_log2, m_run, l_run);
        }
        if (!ok_j) {
          ok = false;
          break;
        }
      }
      // ------------------------------------------------ output: O_t / l
      if (ok) ok = mbar_wait(&bar.pv_done[C::sb(t, g - 1)], C::sp(t, g - 1));
      ok = __all_sync(0xffffffffu, ok);  // the unit loop continues for the whole warp or not at all
      if (!ok) break;
      tc_fence_after();
      const int head = e[1], q0 = e[2], q_end = e[3], part = e[8];
      __syncwarp();
      if (lane == 0) ring.done(n);
      const int row = q0 + r, row0 = q0 + t * kTileQ + q * 32;  // this warp's 32 rows start at row0
      const bool mine = row < q_end;
      if (__any_sync(0xffffffffu, part >= 0)) {
        const int64_t slot = (int64_t)part * kBQ + r;
        const bool keep = mine && ACID_IN_BOUNDS(kSiteMha, slot, a.part_rows);
        if (keep) *reinterpret_cast<float2*>(a.part_ml + slot * 2) = make_float2(m_run, l_run);
#pragma unroll 1
        for (int c = 0; c < C::D; c += 32) {
          uint32_t o[32];
          tmem_ld32(o_addr + c, o);
          tmem_wait_ld();
          if (!keep) continue;
          float* pp = a.part_o + slot * C::D + c;
#pragma unroll
          for (int i = 0; i < 32; i += 4)
            *reinterpret_cast<uint4*>(pp + i) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
        }
        continue;
      }
      const float inv = l_run == 0.f ? 0.f : 1.0f / l_run;
      if (mine && ACID_IN_BOUNDS(kSiteMha, head * (int64_t)a.s.nq + row, (int64_t)a.s.heads * a.s.nq))
        a.lse[(int64_t)head * a.s.nq + row] =
            l_run == 0.f ? -INFINITY : (m_run + log2f(l_run)) * 0.6931471805599453f;
      // The warp's 32 x 32 box leaves through shared memory and one TMA store where its
      // rows end with the matrix's (which clips it) or lie in the sequence; else row by row.
      const bool box_ok = __any_sync(0xffffffffu, row0 + 32 <= q_end || q_end == a.s.nq);
#pragma unroll 1
      for (int c = 0; c < C::D; c += 32) {
        uint32_t o[32];
        tmem_ld32(o_addr + c, o);
        tmem_wait_ld();
        if (__any_sync(0xffffffffu, row0 >= q_end)) continue;  // warp-uniform
        uint4 w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          // (a row without a sum has O = 0 times P = 0 of values that may not be finite)
          auto v = [&](int i) { return l_run == 0.f ? 0.f : __uint_as_float(o[8 * k + i]) * inv; };
          w[k] = make_uint4(pack_bf16(v(0), v(1)), pack_bf16(v(2), v(3)), pack_bf16(v(4), v(5)), pack_bf16(v(6), v(7)));
        }
        if (!box_ok) {
          const int64_t at = (int64_t)row * a.ldo + head * C::D + c;
          if (mine && ACID_IN_BOUNDS(kSiteMha, at + 31, (int64_t)a.s.nq * a.ldo))
#pragma unroll
            for (int k = 0; k < 4; ++k) reinterpret_cast<uint4*>(a.out + at)[k] = w[k];
          continue;
        }
        uint8_t* box = stage + (n_st & 1) * C::STAGE_BOX;
        if (lane == 0 && n_st >= 2) bulk_wait_group_read<1>();
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 4; ++k) *reinterpret_cast<uint4*>(box + lane * 64 + ((k ^ ((lane >> 1) & 3)) << 4)) = w[k];
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          tma_store_2d(&tmO, box, head * C::D + c, row0);
          bulk_commit_group();
        }
        ++n_st;
      }
    }
    if (lane == 0) bulk_wait_group<0>();  // output stores complete before the CTA ends
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, C::TMEM_COLS);
  }
}

// Joins the parts of the split items: O = sum 2^(m_s - M) O_s / sum 2^(m_s - M) l_s
// with M = max m_s, in the parts' order.  One warp a row, D / 32 columns a lane.
template <int D>
__global__ void __launch_bounds__(256) mha_merge_kernel(const __grid_constant__ FwdArgs a, int rows) {
  pdl_wait();
  const int wrow = (int)(blockIdx.x * 8 + (threadIdx.x >> 5)), lane = threadIdx.x & 31;
  if (wrow >= rows) return;
  const int it = wrow / kBQ, rr = wrow % kBQ;
  int slot, head, index, tile;
  MhaSeq seq;
  mha_item(a.order, a.slots, a.s.heads, a.full + it, slot, head);
  if (!mha_slot<kBQ, false>(a.s, slot, seq, index, tile) || tile * kBQ + rr >= seq.nq) return;
  const int64_t row = seq.q0 + tile * kBQ + rr;
  const float* ml = a.part_ml + ((int64_t)it * a.splits * kBQ + rr) * 2;
  if (!ACID_IN_BOUNDS(kSiteMha, ((int64_t)it * a.splits + a.splits - 1) * kBQ + rr, a.part_rows)) return;
  float M = -INFINITY;
  for (int sp = 0; sp < a.splits; ++sp) M = fmaxf(M, ml[(int64_t)sp * kBQ * 2]);
  float acc[D / 32] = {}, L = 0.f;
  for (int sp = 0; sp < a.splits; ++sp) {
    const float m = ml[(int64_t)sp * kBQ * 2], l = ml[(int64_t)sp * kBQ * 2 + 1];
    if (l == 0.f) continue;  // saw no key: nothing was written, or zeros
    const float w = ex2_approx(m - M);
    L = fmaf(w, l, L);
    const float* o = a.part_o + ((int64_t)(it * a.splits + sp) * kBQ + rr) * D + lane;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) acc[i] = fmaf(w, o[i * 32], acc[i]);
  }
  const float inv = L == 0.f ? 0.f : 1.0f / L;
  const int64_t at = row * a.ldo + head * D;
  if (!ACID_IN_BOUNDS(kSiteMha, at + D - 1, (int64_t)a.s.nq * a.ldo)) return;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) a.out[at + i * 32 + lane] = __float2bfloat16_rn(acc[i] * inv);
  if (lane == 0 && ACID_IN_BOUNDS(kSiteMha, head * (int64_t)a.s.nq + row, (int64_t)a.s.heads * a.s.nq))
    a.lse[(int64_t)head * a.s.nq + row] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
}

// How a call's items go to CTAs (of `sms` SMs): whole ones, and how many shares each of
// the rest is split into.
struct FwdPlan {
  int slots, items, full, splits;
  size_t part_bytes(int d) const { return (size_t)(items - full) * splits * kBQ * (d + 2) * sizeof(float); }
};
// Keys to a tile: as acid_attention_forward.
int key_tile(const MhaArgs& x) { return x.head_dim == 64 && x.shape.nk <= 448 ? 64 : 128; }

FwdPlan plan(const MhaArgs& x, int sms) {
  FwdPlan p;
  const MhaShape& s = x.shape;
  const int bkv = key_tile(x), cap = bkv == 64 ? 2 * sms : sms;
  p.slots = mha_slots(s.nq, s.seqs, s.qb != nullptr, kBQ);
  p.items = p.slots * s.heads;
  p.full = p.items;
  p.splits = 1;
  if (bkv == 64) return p;
  const int tiles = (s.nk / s.seqs + bkv - 1) / bkv;  // of a sequence, on average
  const int whole = p.items / cap * cap, tail = p.items - whole;
  // A few items are split so that they fill the GPU.  So is the last, partial wave of
  // many items over a long key range where all items are alike; with sequences or
  // windows the items' lengths differ, and the CTAs even out by themselves.
  const bool alike = s.seqs == 1 && s.frame == 0;
  const bool split = whole == 0 || (alike && s.nk > 8 * x.head_dim);
  const int splits = tail > 0 ? std::min(cap / tail, tiles / 2) : 1;
  if (split && splits >= 2) {
    p.full = whole;
    p.splits = splits;
  }
  return p;
}

template <class C>
constexpr int kSmem = C::SMEM_P - C::BAR_BYTES + kBarBytes;

template <class C>
acid_status launch(const MhaArgs& x, cudaStream_t s) {
  constexpr int D = C::D;
  static PerContext allowed;
  ACID_TRY(allow_smem(allowed, mha_forward_kernel<C>, kSmem<C>));
  const MhaShape& m = x.shape;
  CUtensorMap tq, tk, tv, to;
  const int64_t wq = (int64_t)m.heads * D, wk = (int64_t)m.kv_heads * D;
  const int64_t nk = std::max(m.nk, 1);  // (without keys nothing is loaded)
  ACID_TRY(make_tmap_bf16(&tq, x.q, m.nq, wq, x.ldq, kTileQ));
  ACID_TRY(make_tmap_bf16(&tk, m.nk > 0 ? x.k : x.q, nk, wk, x.ldk, C::BKV));
  ACID_TRY(make_tmap_bf16(&tv, m.nk > 0 ? x.v : x.q, nk, wk, x.ldv, C::BKV));
  ACID_TRY(make_tmap_bf16_box(&to, x.out, m.nq, wq, x.ldo, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B));
  const FwdPlan p = plan(x, num_sms());
  FwdArgs a = {};
  a.s = m;
  a.out = static_cast<__nv_bfloat16*>(x.out);
  a.lse = x.lse;
  a.ldo = x.ldo;
  a.scale_log2 = x.scale * 1.4426950408889634f;
  a.slots = p.slots;
  a.order = mha_order(m, D, false, false);
  a.full = p.full;
  a.splits = p.splits;
  a.units = p.full + (p.items - p.full) * p.splits;
  a.part_o = static_cast<float*>(x.part);
  a.part_ml = a.part_o + (size_t)(p.items - p.full) * p.splits * kBQ * D;
  a.part_rows = (int64_t)(x.part_bytes / ((D + 2) * sizeof(float)));
  launch_pdl(mha_forward_kernel<C>, std::min(a.units, num_sms() * C::CTAS_PER_SM), kAttnThreads, kSmem<C>, s, tq, tk, tv,
             to, a);
  ACID_CHECK_LAUNCH();
  if (p.full < p.items) {
    const int rows = (p.items - p.full) * kBQ;
    launch_pdl(mha_merge_kernel<D>, (rows + 7) / 8, 256, 0, s, a, rows);
    ACID_CHECK_LAUNCH();
  }
  return ACID_OK;
}

}  // namespace

size_t mha_forward_tc_bytes(const MhaArgs& x) {
  const FwdPlan p = plan(x, num_sms());
  return p.full < p.items ? p.part_bytes(x.head_dim) : 0;
}

acid_status mha_forward_tc(const MhaArgs& x, cudaStream_t s) {
  if (x.head_dim == 128) return launch<AttnCfg<128, 128>>(x, s);
  return key_tile(x) == 64 ? launch<AttnCfg<64, 64>>(x, s) : launch<AttnCfg<64, 128>>(x, s);
}

}  // namespace acid
