// What the kernels of acid_mha_forward and acid_mha_backward share: the shape of
// a call as the device sees it, its sequences, and which rows see which.
#pragma once

#include <stdint.h>

#include "common.cuh"
#include "internal.h"

namespace acid {

// Rows are 32-bit (at most kMhaMaxRows); offsets into matrices are 64-bit.
constexpr int64_t kMhaMaxRows = (int64_t)1 << 30;
constexpr int kStatRows = 128;  // query rows of a slot of the row statistics (MhaStats)

struct MhaShape {
  int nq, nk, heads, kv_heads, group;  // group: query heads that share a key head
  int seqs;
  const int2 *qb, *kb;  // [seqs] {first row, row past the last}; null: all rows
  int frame, before, after, q_first;
};

// One sequence's rows: queries [q0, q0 + nq), keys [k0, k0 + nk).
struct MhaSeq {
  int q0, nq, k0, nk;
};

// A bound as the device reads it: inside the matrix and in order, whatever the
// array holds, so that no access leaves the operands.
__device__ __forceinline__ void mha_bound(const int2* b, int i, int seqs, int n, int& first, int& rows) {
  const int2 v = b != nullptr && ACID_IN_BOUNDS(kSiteMha, i, seqs) ? __ldg(b + i) : make_int2(0, n);
  first = min(max(v.x, 0), n);
  rows = min(max(v.y, first), n) - first;
}
__device__ __forceinline__ MhaSeq mha_seq(const MhaShape& s, int i) {
  MhaSeq q;
  mha_bound(s.qb, i, s.seqs, s.nq, q.q0, q.nq);
  mha_bound(s.kb, i, s.seqs, s.nk, q.k0, q.nk);
  return q;
}

// The last sequence that begins at or before a row: its own, if it is of one.
__device__ __forceinline__ int mha_sequence_of(const int2* b, int seqs, int64_t row) {
  int lo = 0;
  if (b != nullptr)
    for (int hi = seqs; hi - lo > 1;) {
      const int mid = (lo + hi) >> 1;
      if (__ldg(b + mid).x <= row) lo = mid;
      else hi = mid;
    }
  return lo;
}

// Slots of tiles of `tile` rows.  Sequence i begins at slot first / tile + i, so
// that each has as many slots as it can need (and one may stay empty) without a
// table or a scan of the lengths before it: ceil(len / tile) <=
// (first + len) / tile - first / tile + 1.
__host__ __device__ __forceinline__ int mha_slots(int rows, int seqs, bool bounded, int tile) {
  return bounded ? rows / tile + seqs : (rows + tile - 1) / tile;
}
// First slot of sequence i, whose first row is `first`.
__device__ __forceinline__ int mha_slot0(const int2* b, int i, int first, int tile) {
  return b != nullptr ? first / tile + i : 0;
}
// The sequence and its tile at a slot of the queries or keys; false: an empty slot.
template <int TILE, bool KEYS>
__device__ __forceinline__ bool mha_slot(const MhaShape& s, int slot, MhaSeq& seq, int& index, int& tile) {
  const int2* b = KEYS ? s.kb : s.qb;
  int lo = 0;
  if (b != nullptr) {
    const int n = KEYS ? s.nk : s.nq;
    for (int hi = s.seqs; hi - lo > 1;) {
      const int mid = (lo + hi) >> 1;
      if (min(max(__ldg(b + mid).x, 0), n) / TILE + mid <= slot) lo = mid;
      else hi = mid;
    }
  }
  index = lo;
  seq = mha_seq(s, lo);
  tile = slot - mha_slot0(b, lo, KEYS ? seq.k0 : seq.q0, TILE);
  const int rows = KEYS ? seq.nk : seq.nq;
  return tile >= 0 && tile < (rows + TILE - 1) / TILE;
}

// Order in which CTAs take the items, one of `heads` and a slot each, in turn.
//   By head: those at work at a time stream the same keys (or queries) out of L2.
//   By slot, all heads of a slot together: a round of CTAs then has items of one
// sequence or one frame, which are as long as each other, so that the rounds come out
// even (4726, 2501 and 1013 rows, 30 heads: the longest CTA has 196 tiles instead of 225,
// 184.5 on average).  Under a window the items with the most tiles come first: a causal
// one's last queries, its first keys.
enum MhaOrder : int { kByHead = 0, kBySlot = 1, kBySlotDown = 2 };
__host__ __device__ __forceinline__ void mha_item(int order, int slots, int heads, int item, int& slot, int& head) {
  if (order == kByHead) {
    slot = item % slots;
    head = item / slots;
  } else {
    slot = item / heads;
    if (order == kBySlotDown) slot = slots - 1 - slot;
    head = item % heads;
  }
}
// By slot all heads' streamed rows are in use together; with sequences, whose items have
// all of them to read, only where L2 holds them.
inline int mha_order(const MhaShape& s, int d, bool queries_streamed, bool first_longest) {
  const int64_t bytes = queries_streamed ? (int64_t)s.nq * s.heads * d * 4 : (int64_t)s.nk * s.kv_heads * d * 4;
  if (s.frame != 0) return first_longest ? kBySlot : kBySlotDown;
  return s.seqs > 1 && bytes <= (int64_t)80 << 20 ? kBySlot : kByHead;
}

// The item that this CTA takes in a turn: the turns go through the CTAs forwards and
// backwards alternately, so that items which get shorter from one to the next come out
// even (32760 rows causal in 21 frames, 12 heads: 1988 us, always forwards 2087).
__device__ __forceinline__ int mha_turn(int turn) {
  const int n = gridDim.x;
  return turn * n + (turn & 1 ? n - 1 - (int)blockIdx.x : (int)blockIdx.x);
}

__device__ __forceinline__ int floor_div(int a, int b) { return a >= 0 ? a / b : -((b - 1 - a) / b); }
__device__ __forceinline__ int clamp_row(int64_t v, int n) { return (int)min(max(v, (int64_t)0), (int64_t)n); }

// Position of a sequence's first query among its keys.
__device__ __forceinline__ int mha_first(const MhaShape& s, const MhaSeq& q) {
  return s.q_first >= 0 ? s.q_first : q.nk - q.nq;
}
// Keys [lo, hi) of the sequence that its query row i sees, and queries [lo, hi)
// that see its key row j.  Both bounds grow with the row.
__device__ __forceinline__ void mha_keys_of(const MhaShape& s, const MhaSeq& q, int i, int& lo, int& hi) {
  lo = 0;
  hi = q.nk;
  if (s.frame == 0) return;
  const int64_t at = floor_div(i + mha_first(s, q), s.frame);
  if (s.before >= 0) lo = clamp_row((at - s.before) * s.frame, q.nk);
  if (s.after >= 0) hi = clamp_row((at + s.after + 1) * s.frame, q.nk);
}
__device__ __forceinline__ void mha_queries_of(const MhaShape& s, const MhaSeq& q, int j, int& lo, int& hi) {
  lo = 0;
  hi = q.nq;
  if (s.frame == 0) return;
  const int64_t at = j / s.frame, first = mha_first(s, q);
  if (s.after >= 0) lo = clamp_row((at - s.after) * s.frame - first, q.nq);
  if (s.before >= 0) hi = clamp_row((at + s.before + 1) * s.frame - first, q.nq);
}

// Row statistics of the backward pass, [heads][slots][2][kStatRows] floats: -lse
// (in the unit of the kernels' exponential) and less the sum of dout out over the
// head's columns.  Rows past a sequence's end and rows that see no key hold -inf and 0,
// which makes their probabilities 0.
__host__ __device__ __forceinline__ int64_t mha_stat_offset(int head, int slots, int slot) {
  return ((int64_t)head * slots + slot) * (2 * kStatRows);
}

// 8 columns of a row as they are loaded, and as fp32.
template <typename T> struct MhaRaw;
template <> struct MhaRaw<__nv_bfloat16> {
  uint4 u;
  __device__ __forceinline__ void zero() { u = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { u = __ldg(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void get(float* v) const {
    v[0] = bf16_lo(u.x); v[1] = bf16_hi(u.x); v[2] = bf16_lo(u.y); v[3] = bf16_hi(u.y);
    v[4] = bf16_lo(u.z); v[5] = bf16_hi(u.z); v[6] = bf16_lo(u.w); v[7] = bf16_hi(u.w);
  }
};
template <> struct MhaRaw<float> {
  float4 a, b;
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void load(const float* p) {
    a = __ldg(reinterpret_cast<const float4*>(p));
    b = __ldg(reinterpret_cast<const float4*>(p + 4));
  }
  __device__ __forceinline__ void get(float* v) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
};

// A call of either direction.
struct MhaArgs {
  MhaShape shape;
  int dtype, head_dim;
  float scale;
  const void *q, *k, *v;
  int64_t ldq, ldk, ldv;
  void* out;  // forward: written; backward: read
  int64_t ldo;
  float* lse;
  const void* dout;
  int64_t lddo;
  void *dq, *dk, *dv;
  int64_t lddq, lddk, lddv;
  float* stats;
  void* part;  // scratch behind the statistics
  size_t part_bytes;
};

// mha_few.cu: a few query rows.  Whether a call is one, and its bytes of scratch.
bool mha_few(const MhaArgs& a);
size_t mha_few_bytes(const MhaArgs& a);
acid_status mha_forward_few(const MhaArgs& a, cudaStream_t s);
// mha_forward.cu: bf16 on tcgen05.  Bytes of scratch (part) that the call needs.
size_t mha_forward_tc_bytes(const MhaArgs& a);
acid_status mha_forward_tc(const MhaArgs& a, cudaStream_t s);
// mha_backward.cu: the same of the gradient.
size_t mha_backward_tc_bytes(const MhaArgs& a);
acid_status mha_backward_tc(const MhaArgs& a, cudaStream_t s);
// mha_f32.cu: the FP32 pipes
acid_status mha_forward_f32(const MhaArgs& a, cudaStream_t s);
acid_status mha_backward_f32(const MhaArgs& a, cudaStream_t s);

}  // namespace acid
