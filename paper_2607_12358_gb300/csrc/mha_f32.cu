// Attention with row sums, and its gradient, on the FP32 pipes.
#include <math.h>

#include <algorithm>

#define ACID_UNIT_WITHOUT_WAITS
#include "mha.cuh"

namespace acid {

BoundsRecord take_bounds_mha_f32();
ACID_BOUNDS_READER(take_bounds_mha_f32)

namespace {

constexpr int kGroups = 4, kCols = 32, kThreads = 128 * kGroups;  // groups of four warps; rows of a streamed tile

// A matrix in memory: [rows, ..] with row stride ld.
struct Rows {
  const float* p;
  int64_t ld;
  int rows;
};
// N rows of D values from (row, col) on their way (cp.async) to shared memory (row stride
// lds there); rows outside [0, valid) are zeros.
template <int D, int N>
__device__ __forceinline__ void load_rows(float* dst, int lds, const Rows& m, int64_t row, int col, int valid, int tid,
                                          int threads) {
  const float* src = m.p + row * m.ld + col;
  const int64_t ld = m.ld;
  for (int i = tid; i < N * (D / 4); i += threads) {
    const int r = i / (D / 4), c = (i % (D / 4)) * 4;
    const bool on = r < valid && ACID_IN_BOUNDS(kSiteMha, (row + r) * ld + col + c + 3, m.rows * ld);
    cp_async<16>(dst + r * lds + c, src + (on ? (int64_t)r * ld + c : 0), on);
  }
}

// Products of R rows of a (row stride lds) with the two rows kg and kg + 16 of b.
template <int D, int R>
__device__ __forceinline__ void products(const float* a, const float* b, int lds, int kg, float (&s)[R][2]) {
#pragma unroll
  for (int i = 0; i < R; ++i) s[i][0] = s[i][1] = 0.f;
#pragma unroll 4
  for (int d = 0; d < D; d += 4) {
    float4 bv[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) bv[c] = *reinterpret_cast<const float4*>(b + (kg + 16 * c) * lds + d);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const float4 av = *reinterpret_cast<const float4*>(a + i * lds + d);
#pragma unroll
      for (int c = 0; c < 2; ++c)
        s[i][c] += fmaf(av.y, bv[c].y, av.x * bv[c].x) + fmaf(av.w, bv[c].w, av.z * bv[c].z);
    }
  }
}

// acc[i][..] += sum over the 32 streamed rows of p[i][row] b[row][columns of this lane]
template <int D, int R>
__device__ __forceinline__ void accumulate(const float* p, int ldp, const float* b, int lds, int kg,
                                           float (&acc)[R][D / 16]) {
#pragma unroll 2
  for (int k0 = 0; k0 < kCols; k0 += 4) {
    float4 pv[R];
#pragma unroll
    for (int i = 0; i < R; ++i) pv[i] = *reinterpret_cast<const float4*>(p + i * ldp + k0);
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      float2 bv[D / 32];
#pragma unroll
      for (int c = 0; c < D / 32; ++c) bv[c] = *reinterpret_cast<const float2*>(b + (k0 + kk) * lds + 32 * c + 2 * kg);
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const float w = kk == 0 ? pv[i].x : kk == 1 ? pv[i].y : kk == 2 ? pv[i].z : pv[i].w;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          acc[i][2 * c] = fmaf(w, bv[c].x, acc[i][2 * c]);
          acc[i][2 * c + 1] = fmaf(w, bv[c].y, acc[i][2 * c + 1]);
        }
      }
    }
  }
}

struct F32Args {
  MhaShape s;
  const float *q, *k, *v, *dout;
  int64_t ldq, ldk, ldv, lddo;
  void *out1, *out2, *out3;  // forward: out; backward: dk, dv, dq
  int64_t ld1, ld2, ld3;
  float *lse, *stats;
  float scale;
  int stat_slots;
};

// Shared memory, in floats: two stationary tiles; for each group BUFS buffers of two
// streamed tiles and their rows' statistics, and NP tiles of products.  Up to head dim 64
// the next tiles are on their way while a group works on its own.
template <int D, int ROWS, int NP>
struct F32Cfg {
  static constexpr int LD = D + 4, LDP = kCols + 4, BUFS = D <= 64 ? 2 : 1;
  static constexpr int OFF_STREAM = 2 * ROWS * LD;
  static constexpr int BUF = 2 * kCols * LD + 2 * kCols, STREAM = BUFS * BUF + NP * ROWS * LDP;
  static constexpr int FLOATS = OFF_STREAM + kGroups * STREAM;
  static_assert(kGroups * ROWS * (D + 2) <= kGroups * STREAM, "the parts fit over the streamed tiles");
  static_assert(FLOATS * 4 <= 227 * 1024, "shared memory");
};

// ----------------------------------------------------------------- forward
// A CTA has 16 query rows of a head; its groups of four warps walk the key tiles
// in turn with a running maximum and sum each, and their parts are joined through
// shared memory.  A half-warp has two rows.
template <int D>
__global__ void __launch_bounds__(kThreads) mha_forward_f32_kernel(const F32Args a) {
  constexpr int ROWS = 16, R = 2;
  using C = F32Cfg<D, ROWS, 1>;
  extern __shared__ __align__(16) float sm[];
  pdl_wait();
  const int g = threadIdx.x >> 7, t = threadIdx.x & 127, hw = t >> 4, kg = t & 15;
  const int h = blockIdx.y, hk = h / a.s.group;
  MhaSeq seq;
  int index, tile;
  if (!mha_slot<ROWS, false>(a.s, blockIdx.x, seq, index, tile)) return;
  const int r0 = tile * ROWS, rows = min(ROWS, seq.nq - r0);
  float* sq = sm;
  float* bufs = sm + C::OFF_STREAM + g * C::STREAM;
  float* sp = bufs + C::BUFS * C::BUF + hw * R * C::LDP;
  const Rows q{a.q, a.ldq, a.s.nq}, k{a.k, a.ldk, a.s.nk}, v{a.v, a.ldv, a.s.nk};
  load_rows<D, ROWS>(sq, C::LD, q, (int64_t)seq.q0 + r0, h * D, rows, threadIdx.x, kThreads);
  int lo[R], hi[R], first, last, none;
  mha_keys_of(a.s, seq, r0, first, none);
  mha_keys_of(a.s, seq, r0 + rows - 1, none, last);
#pragma unroll
  for (int i = 0; i < R; ++i) mha_keys_of(a.s, seq, r0 + min(hw * R + i, rows - 1), lo[i], hi[i]);
  float m[R], l[R], o[R][D / 16] = {};
#pragma unroll
  for (int i = 0; i < R; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
  }
  auto fetch = [&](int j, int buf) {  // tile j's keys and values, if there is one
    float* to = bufs + buf * C::BUF;
    if (j * kCols < last) {
      const int64_t row = (int64_t)seq.k0 + j * kCols;
      load_rows<D, kCols>(to, C::LD, k, row, hk * D, seq.nk - j * kCols, t, 128);
      load_rows<D, kCols>(to + kCols * C::LD, C::LD, v, row, hk * D, seq.nk - j * kCols, t, 128);
    }
    cp_async_commit();
  };
  int buf = 0;
  fetch(first / kCols + g, 0);
  cp_async_wait<0>();
  __syncthreads();  // the query rows, and every group's first tiles
  for (int j = first / kCols + g; j * kCols < last; j += kGroups) {
    if (C::BUFS == 2) fetch(j + kGroups, buf ^ 1);
    const float* sk = bufs + buf * C::BUF;
    const float* sv = sk + kCols * C::LD;
    float s[R][2];
    products<D, R>(sq + hw * R * C::LD, sk, C::LD, kg, s);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      float mt = -INFINITY;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int key = j * kCols + kg + 16 * c;
        s[i][c] = key >= lo[i] && key < hi[i] ? s[i][c] * a.scale : -INFINITY;
        mt = fmaxf(mt, s[i][c]);
      }
#pragma unroll
      for (int off = 8; off > 0; off >>= 1) mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, off));
      const float mn = fmaxf(m[i], mt), ref = mn == -INFINITY ? 0.f : mn;
      const float corr = expf(m[i] - ref);
      m[i] = mn;
      l[i] *= corr;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) o[i][c] *= corr;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const float p = expf(s[i][c] - ref);
        l[i] += p;
        sp[i * C::LDP + kg + 16 * c] = p;
      }
    }
    __syncwarp();
    accumulate<D, R>(sp, C::LDP, sv, C::LD, kg, o);
    group_sync(1 + g, 128);  // the tiles have been read
    if (C::BUFS == 1) fetch(j + kGroups, 0);
    cp_async_wait<0>();
    group_sync(1 + g, 128);  // the next are there
    if (C::BUFS == 2) buf ^= 1;
  }
  // ---- join: [group][ROWS][D] parts over the streamed tiles, then {m, l}
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], off);
  __syncthreads();
  float* mo = sm + C::OFF_STREAM;
  float2* ml = reinterpret_cast<float2*>(mo + kGroups * ROWS * D);
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int at = g * ROWS + hw * R + i;
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
      *reinterpret_cast<float2*>(mo + at * D + 32 * c + 2 * kg) = make_float2(o[i][2 * c], o[i][2 * c + 1]);
    if (kg == 0) ml[at] = make_float2(m[i], l[i]);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < rows * D; i += kThreads) {
    const int r = i / D, c = i % D;
    float mx = -INFINITY, acc = 0.f, den = 0.f;
    for (int gg = 0; gg < kGroups; ++gg) mx = fmaxf(mx, ml[gg * ROWS + r].x);
    const float ref = mx == -INFINITY ? 0.f : mx;
    for (int gg = 0; gg < kGroups; ++gg) {
      const float2 e = ml[gg * ROWS + r];
      const float w = expf(e.x - ref);
      den = fmaf(w, e.y, den);
      acc = fmaf(w, mo[(gg * ROWS + r) * D + c], acc);
    }
    const int64_t row = seq.q0 + r0 + r, at = row * a.ld1 + h * D + c;
    if (!ACID_IN_BOUNDS(kSiteMha, at, (int64_t)a.s.nq * a.ld1)) continue;
    static_cast<float*>(a.out1)[at] = den > 0.f ? acc / den : den == 0.f ? 0.f : den;
    if (c == 0 && ACID_IN_BOUNDS(kSiteMha, h * (int64_t)a.s.nq + row, (int64_t)a.s.heads * a.s.nq))
      a.lse[(int64_t)h * a.s.nq + row] = den == 0.f ? -INFINITY : mx + logf(den);
  }
}

// ---------------------------------------------------------------- gradient
// One kernel for both halves.  A CTA keeps 16 rows and streams tiles of 32:
//   KEYS   keeps keys and values, streams q and dout of every query head of the
//          group: rows are keys, columns queries; dk += ds^T q, dv += p^T dout;
//   else   keeps q and dout, streams keys and values: dq += ds k.
// The groups of four warps take the tiles in turn and their sums are joined in order.
template <int D, bool KEYS>
__device__ __forceinline__ void mha_backward_f32(const F32Args& a) {
  constexpr int ROWS = 16, R = 2;
  using C = F32Cfg<D, ROWS, 2>;
  extern __shared__ __align__(16) float sm[];
  const int g = threadIdx.x >> 7, t = threadIdx.x & 127, hw = t >> 4, kg = t & 15;
  const int hb = blockIdx.y;  // head of the rows that stay
  MhaSeq seq;
  int index, tile;
  if (hb >= (KEYS ? a.s.kv_heads : a.s.heads) || !mha_slot<ROWS, KEYS>(a.s, blockIdx.x, seq, index, tile)) return;
  const int n_rows = KEYS ? seq.nk : seq.nq, r0 = tile * ROWS, rows = min(ROWS, n_rows - r0);
  const int slot0 = mha_slot0(a.s.qb, index, seq.q0, kStatRows);
  float* x1 = sm;
  float* x2 = sm + ROWS * C::LD;
  float* bufs = sm + C::OFF_STREAM + g * C::STREAM;
  float* sp = bufs + C::BUFS * C::BUF;
  float* sd = sp + ROWS * C::LDP;
  const Rows q{a.q, a.ldq, a.s.nq}, dout{a.dout, a.lddo, a.s.nq}, k{a.k, a.ldk, a.s.nk}, v{a.v, a.ldv, a.s.nk};
  const int64_t x0 = (KEYS ? seq.k0 : seq.q0) + (int64_t)r0, y0 = KEYS ? seq.q0 : seq.k0;  // rows in memory
  if (KEYS) {
    load_rows<D, ROWS>(x1, C::LD, k, x0, hb * D, rows, threadIdx.x, kThreads);
    load_rows<D, ROWS>(x2, C::LD, v, x0, hb * D, rows, threadIdx.x, kThreads);
  } else {
    load_rows<D, ROWS>(x1, C::LD, q, x0, hb * D, rows, threadIdx.x, kThreads);
    load_rows<D, ROWS>(x2, C::LD, dout, x0, hb * D, rows, threadIdx.x, kThreads);
  }
  auto seen = [&](int row, int& lo, int& hi) {
    if (KEYS) mha_queries_of(a.s, seq, row, lo, hi);
    else mha_keys_of(a.s, seq, row, lo, hi);
  };
  int lo[R], hi[R], first, last, none;
  seen(r0, first, none);
  seen(r0 + rows - 1, none, last);
  float nl[R], dl[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int row = r0 + min(hw * R + i, rows - 1);
    seen(row, lo[i], hi[i]);
    if (!KEYS) {
      const int64_t at = mha_stat_offset(hb, a.stat_slots, slot0 + row / kStatRows) + row % kStatRows;
      const bool in = ACID_IN_BOUNDS(kSiteMha, at + kStatRows, mha_stat_offset(a.s.heads, a.stat_slots, 0));
      nl[i] = in ? a.stats[at] : -INFINITY;
      dl[i] = in ? a.stats[at + kStatRows] : 0.f;
    }
  }
  const int j0 = first / kCols, tiles = last > j0 * kCols ? (last + kCols - 1) / kCols - j0 : 0;
  const int total = tiles * (KEYS ? a.s.group : 1);
  float acc1[R][D / 16] = {}, acc2[R][D / 16] = {};
  // step n: tile j0 + n % tiles of the n / tiles-th head of the group
  auto fetch = [&](int n, int buf) {
    if (n < total) {
      const int c0 = (j0 + n % tiles) * kCols, h = KEYS ? hb * a.s.group + n / tiles : hb / a.s.group;
      float* y1 = bufs + buf * C::BUF;
      float* y2 = y1 + kCols * C::LD;
      if (KEYS) {
        load_rows<D, kCols>(y1, C::LD, q, y0 + c0, h * D, seq.nq - c0, t, 128);
        load_rows<D, kCols>(y2, C::LD, dout, y0 + c0, h * D, seq.nq - c0, t, 128);
        if (t < 2 * kCols) {  // the streamed rows' statistics
          const int64_t at = mha_stat_offset(h, a.stat_slots, slot0 + c0 / kStatRows) + c0 % kStatRows +
                             (t / kCols) * kStatRows + t % kCols;
          if (ACID_IN_BOUNDS(kSiteMha, at, mha_stat_offset(a.s.heads, a.stat_slots, 0)))
            cp_async<4>(y2 + kCols * C::LD + t, a.stats + at, true);
        }
      } else {
        load_rows<D, kCols>(y1, C::LD, k, y0 + c0, h * D, seq.nk - c0, t, 128);
        load_rows<D, kCols>(y2, C::LD, v, y0 + c0, h * D, seq.nk - c0, t, 128);
      }
    }
    cp_async_commit();
  };
  int buf = 0;
  fetch(g, 0);
  cp_async_wait<0>();
  __syncthreads();  // the stationary rows, and every group's first tiles
  for (int n = g; n < total; n += kGroups) {
    if (C::BUFS == 2) fetch(n + kGroups, buf ^ 1);
    const float* y1 = bufs + buf * C::BUF;
    const float* y2 = y1 + kCols * C::LD;
    const float* st = y2 + kCols * C::LD;
    const int c0 = (j0 + n % tiles) * kCols;
    float s[R][2], dp[R][2];
    products<D, R>(x1 + hw * R * C::LD, y1, C::LD, kg, s);
    products<D, R>(x2 + hw * R * C::LD, y2, C::LD, kg, dp);
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int col = kg + 16 * c;
        const float nlse = KEYS ? st[col] : nl[i], ndelta = KEYS ? st[kCols + col] : dl[i];
        const bool on = c0 + col >= lo[i] && c0 + col < hi[i];
        const float p = on ? expf(fmaf(s[i][c], a.scale, nlse)) : 0.f;
        if (KEYS) sp[(hw * R + i) * C::LDP + col] = p;
        sd[(hw * R + i) * C::LDP + col] = on ? p * (dp[i][c] + ndelta) : 0.f;
      }
    __syncwarp();
    accumulate<D, R>(sd + hw * R * C::LDP, C::LDP, y1, C::LD, kg, acc1);
    if (KEYS) accumulate<D, R>(sp + hw * R * C::LDP, C::LDP, y2, C::LD, kg, acc2);
    group_sync(1 + g, 128);  // the tiles have been read
    if (C::BUFS == 1) fetch(n + kGroups, 0);
    cp_async_wait<0>();
    group_sync(1 + g, 128);  // the next are there
    if (C::BUFS == 2) buf ^= 1;
  }
  auto join = [&](const float (&acc)[R][D / 16], void* out, int64_t ld, int row0, float by) {
    __syncthreads();
    float* mo = sm + C::OFF_STREAM;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int c = 0; c < D / 32; ++c)
        *reinterpret_cast<float2*>(mo + (g * ROWS + hw * R + i) * D + 32 * c + 2 * kg) =
            make_float2(acc[i][2 * c], acc[i][2 * c + 1]);
    __syncthreads();
    if (out == nullptr) return;
    for (int i = threadIdx.x; i < rows * D; i += kThreads) {
      float sum = 0.f;
      for (int gg = 0; gg < kGroups; ++gg) sum += mo[gg * ROWS * D + i];
      const int64_t at = (int64_t)(row0 + i / D) * ld + hb * D + i % D;
      if (!ACID_IN_BOUNDS(kSiteMha, at, (int64_t)(KEYS ? a.s.nk : a.s.nq) * ld)) continue;
      static_cast<float*>(out)[at] = sum * by;
    }
  };
  if (KEYS) {
    join(acc1, a.out1, a.ld1, seq.k0 + r0, a.scale);
    join(acc2, a.out2, a.ld2, seq.k0 + r0, 1.f);
  } else {
    join(acc1, a.out3, a.ld3, seq.q0 + r0, a.scale);
  }
}

// Both halves in one launch (blockIdx.z: `first` of them on): neither fills the GPU at the
// sizes of the fp32 mode (256 rows, 4 heads of 64: 64 CTAs each; one after the other 35.7
// us with the statistics, so 19).
template <int D>
__global__ void __launch_bounds__(kThreads) mha_backward_f32_kernel(const F32Args a, int first) {
  pdl_wait();
  if (blockIdx.z + first == 0) mha_backward_f32<D, true>(a);
  else mha_backward_f32<D, false>(a);
}

template <int D>
acid_status forward(const MhaArgs& x, const F32Args& base, cudaStream_t s) {
  static PerContext allowed;
  constexpr size_t smem = (size_t)F32Cfg<D, 16, 1>::FLOATS * 4;
  ACID_TRY(allow_smem(allowed, mha_forward_f32_kernel<D>, smem));
  F32Args a = base;
  a.out1 = x.out;
  a.ld1 = x.ldo;
  const dim3 grid(mha_slots(a.s.nq, a.s.seqs, a.s.qb != nullptr, 16), a.s.heads);
  launch_pdl(mha_forward_f32_kernel<D>, grid, kThreads, smem, s, a);
  ACID_CHECK_LAUNCH();
  return ACID_OK;
}

template <int D>
acid_status backward(const MhaArgs& x, const F32Args& base, cudaStream_t s) {
  static PerContext allowed;
  constexpr size_t smem = (size_t)F32Cfg<D, 16, 2>::FLOATS * 4;
  ACID_TRY(allow_smem(allowed, mha_backward_f32_kernel<D>, smem));
  F32Args a = base;
  a.out1 = x.dk;
  a.ld1 = x.lddk;
  a.out2 = x.dv;
  a.ld2 = x.lddv;
  a.out3 = x.dq;
  a.ld3 = x.lddq;
  const bool keys = x.dk != nullptr || x.dv != nullptr, queries = x.dq != nullptr;
  if (!keys && !queries) return ACID_OK;
  const int kx = keys ? mha_slots(a.s.nk, a.s.seqs, a.s.kb != nullptr, 16) : 0;
  const int qx = queries ? mha_slots(a.s.nq, a.s.seqs, a.s.qb != nullptr, 16) : 0;
  const dim3 grid(std::max(kx, qx), queries ? a.s.heads : a.s.kv_heads, keys && queries ? 2 : 1);
  launch_pdl(mha_backward_f32_kernel<D>, grid, kThreads, smem, s, a, keys ? 0 : 1);
  ACID_CHECK_LAUNCH();
  return ACID_OK;
}

F32Args base_args(const MhaArgs& x) {
  F32Args a = {};
  a.s = x.shape;
  a.q = static_cast<const float*>(x.q);
  a.k = static_cast<const float*>(x.k);
  a.v = static_cast<const float*>(x.v);
  a.dout = static_cast<const float*>(x.dout);
  a.ldq = x.ldq;
  a.ldk = x.ldk;
  a.ldv = x.ldv;
  a.lddo = x.lddo;
  a.lse = x.lse;
  a.stats = x.stats;
  a.scale = x.scale;
  a.stat_slots = mha_slots(a.s.nq, a.s.seqs, a.s.qb != nullptr, kStatRows);
  return a;
}

}  // namespace

acid_status mha_forward_f32(const MhaArgs& x, cudaStream_t s) {
  const F32Args a = base_args(x);
  switch (x.head_dim) {
    case 32: return forward<32>(x, a, s);
    case 64: return forward<64>(x, a, s);
    case 96: return forward<96>(x, a, s);
    default: return forward<128>(x, a, s);
  }
}

acid_status mha_backward_f32(const MhaArgs& x, cudaStream_t s) {
  const F32Args a = base_args(x);
  switch (x.head_dim) {
    case 32: return backward<32>(x, a, s);
    case 64: return backward<64>(x, a, s);
    case 96: return backward<96>(x, a, s);
    default: return backward<128>(x, a, s);
  }
}

}  // namespace acid
