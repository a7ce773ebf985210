// Attention with row sums, and its gradient, on the FP32 pipes.
#include <math.h>

#define ACID_UNIT_WITHOUT_WAITS
#include "mha.cuh"

namespace acid {

BoundsRecord take_bounds_mha_f32();
ACID_BOUNDS_READER(take_bounds_mha_f32)

namespace {

constexpr int kGroups = 4, kCols = 32, kThreads = 128 * kGroups;  // groups of four warps; rows of a streamed tile

// N rows of D values (row stride lds in shared memory); rows outside [0, valid) are
// zeros.
template <int D, int N>
__device__ __forceinline__ void load_rows(float* dst, int lds, const float* src, int64_t ld, int valid, int tid,
                                          int threads) {
  for (int i = tid; i < N * (D / 8); i += threads) {
    const int r = i / (D / 8), c = (i % (D / 8)) * 8;
    float v[8] = {};
    if (r < valid) load8(src + (int64_t)r * ld + c, v);
    *reinterpret_cast<float4*>(dst + r * lds + c) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(dst + r * lds + c + 4) = make_float4(v[4], v[5], v[6], v[7]);
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
  for (int k = 0; k < kCols; ++k) {
    float bv[D / 16];
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      const float2 t = *reinterpret_cast<const float2*>(b + k * lds + 32 * c + 2 * kg);
      bv[2 * c] = t.x;
      bv[2 * c + 1] = t.y;
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const float w = p[i * ldp + k];
#pragma unroll
      for (int c = 0; c < D / 16; ++c) acc[i][c] = fmaf(w, bv[c], acc[i][c]);
    }
  }
}

struct F32Args {
  MhaShape s;
  const void *q, *k, *v, *o, *dout;
  int64_t ldq, ldk, ldv, ldo, lddo;
  void *out1, *out2;  // forward: out; keys: dk, dv; queries: dq
  int64_t ld1, ld2;
  float *lse, *stats;
  float scale;
  int stat_slots;
};

template <int D, int ROWS, int NSTREAM, int NP>
struct F32Cfg {
  static constexpr int LD = D + 4, LDP = kCols + 4;
  static constexpr int OFF_STREAM = 2 * ROWS * LD;                        // after the two stationary tiles
  static constexpr int STREAM = NSTREAM * kCols * LD + NP * ROWS * LDP + 2 * kCols;  // of one group
  static constexpr int FLOATS = OFF_STREAM + kGroups * STREAM;
};

// ----------------------------------------------------------------- forward
// A CTA has 16 query rows of a head; its groups of four warps walk the key tiles
// in turn with a running maximum and sum each, and their parts are joined through
// shared memory.  A half-warp has two rows.
template <int D>
__global__ void __launch_bounds__(kThreads) mha_forward_f32_kernel(const F32Args a) {
  constexpr int ROWS = 16, R = 2;
  using C = F32Cfg<D, ROWS, 2, 1>;
  extern __shared__ __align__(16) float sm[];
  pdl_wait();
  const int g = threadIdx.x >> 7, t = threadIdx.x & 127, hw = t >> 4, kg = t & 15;
  const int h = blockIdx.y, hk = h / a.s.group;
  MhaSeq seq;
  int index, tile;
  if (!mha_slot<ROWS, false>(a.s, blockIdx.x, seq, index, tile)) return;
  const int r0 = tile * ROWS, rows = min(ROWS, seq.nq - r0);
  float* sq = sm;
  float* sk = sm + C::OFF_STREAM + g * C::STREAM;
  float* sv = sk + kCols * C::LD;
  float* sp = sv + kCols * C::LD + hw * R * C::LDP;
  const float* q = static_cast<const float*>(a.q) + (int64_t)(seq.q0 + r0) * a.ldq + h * D;
  const float* k = static_cast<const float*>(a.k) + (int64_t)seq.k0 * a.ldk + hk * D;
  const float* v = static_cast<const float*>(a.v) + (int64_t)seq.k0 * a.ldv + hk * D;
  load_rows<D, ROWS>(sq, C::LD, q, a.ldq, rows, threadIdx.x, kThreads);
  __syncthreads();
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
  for (int j = first / kCols + g; j * kCols < last; j += kGroups) {
    group_sync(1 + g, 128);  // the tiles before have been read
    load_rows<D, kCols>(sk, C::LD, k + (int64_t)j * kCols * a.ldk, a.ldk, seq.nk - j * kCols, t, 128);
    load_rows<D, kCols>(sv, C::LD, v + (int64_t)j * kCols * a.ldv, a.ldv, seq.nk - j * kCols, t, 128);
    group_sync(1 + g, 128);
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
    if (c == 0) a.lse[(int64_t)h * a.s.nq + row] = den == 0.f ? -INFINITY : mx + logf(den);
  }
}

// ---------------------------------------------------------------- gradient
// One kernel for both halves.  A CTA keeps 16 rows and streams tiles of 32:
//   KEYS   keeps keys and values, streams q and dout of every query head of the
//          group: rows are keys, columns queries; dk += ds^T q, dv += p^T dout;
//   else   keeps q and dout, streams keys and values: dq += ds k.
// The groups of four warps take the tiles in turn and their sums are joined in order.
template <int D, bool KEYS>
__global__ void __launch_bounds__(kThreads) mha_backward_f32_kernel(const F32Args a) {
  constexpr int ROWS = 16, R = 2;
  using C = F32Cfg<D, ROWS, 2, 2>;
  extern __shared__ __align__(16) float sm[];
  pdl_wait();
  const int g = threadIdx.x >> 7, t = threadIdx.x & 127, hw = t >> 4, kg = t & 15;
  const int hb = blockIdx.y;  // head of the rows that stay
  MhaSeq seq;
  int index, tile;
  if (!mha_slot<ROWS, KEYS>(a.s, blockIdx.x, seq, index, tile)) return;
  const int n_rows = KEYS ? seq.nk : seq.nq, r0 = tile * ROWS, rows = min(ROWS, n_rows - r0);
  const int slot0 = mha_slot0(a.s.qb, index, seq.q0, kStatRows);
  float* x1 = sm;
  float* x2 = sm + ROWS * C::LD;
  float* y1 = sm + C::OFF_STREAM + g * C::STREAM;
  float* y2 = y1 + kCols * C::LD;
  float* sp = y2 + kCols * C::LD;
  float* sd = sp + ROWS * C::LDP;
  float* st = sd + ROWS * C::LDP;  // KEYS: the streamed rows' statistics
  const float* q = static_cast<const float*>(a.q) + (int64_t)seq.q0 * a.ldq;
  const float* k = static_cast<const float*>(a.k) + (int64_t)seq.k0 * a.ldk;
  const float* v = static_cast<const float*>(a.v) + (int64_t)seq.k0 * a.ldv;
  const float* dout = static_cast<const float*>(a.dout) + (int64_t)seq.q0 * a.lddo;
  if (KEYS) {
    load_rows<D, ROWS>(x1, C::LD, k + (int64_t)r0 * a.ldk + hb * D, a.ldk, rows, threadIdx.x, kThreads);
    load_rows<D, ROWS>(x2, C::LD, v + (int64_t)r0 * a.ldv + hb * D, a.ldv, rows, threadIdx.x, kThreads);
  } else {
    load_rows<D, ROWS>(x1, C::LD, q + (int64_t)r0 * a.ldq + hb * D, a.ldq, rows, threadIdx.x, kThreads);
    load_rows<D, ROWS>(x2, C::LD, dout + (int64_t)r0 * a.lddo + hb * D, a.lddo, rows, threadIdx.x, kThreads);
  }
  __syncthreads();
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
      const float* at = a.stats + mha_stat_offset(hb, a.stat_slots, slot0 + row / kStatRows) + row % kStatRows;
      nl[i] = at[0];
      dl[i] = at[kStatRows];
    }
  }
  const int j0 = first / kCols, tiles = last > j0 * kCols ? (last + kCols - 1) / kCols - j0 : 0;
  const int total = tiles * (KEYS ? a.s.group : 1);
  float acc1[R][D / 16] = {}, acc2[R][D / 16] = {};
  for (int n = g; n < total; n += kGroups) {
    const int j = j0 + n % tiles, h = KEYS ? hb * a.s.group + n / tiles : hb / a.s.group, c0 = j * kCols;
    group_sync(1 + g, 128);  // the tiles before have been read
    if (KEYS) {
      load_rows<D, kCols>(y1, C::LD, q + (int64_t)c0 * a.ldq + h * D, a.ldq, seq.nq - c0, t, 128);
      load_rows<D, kCols>(y2, C::LD, dout + (int64_t)c0 * a.lddo + h * D, a.lddo, seq.nq - c0, t, 128);
      if (t < 2 * kCols) {
        const float* at = a.stats + mha_stat_offset(h, a.stat_slots, slot0 + c0 / kStatRows) + c0 % kStatRows;
        st[t] = at[(t / kCols) * kStatRows + t % kCols];
      }
    } else {
      load_rows<D, kCols>(y1, C::LD, k + (int64_t)c0 * a.ldk + h * D, a.ldk, seq.nk - c0, t, 128);
      load_rows<D, kCols>(y2, C::LD, v + (int64_t)c0 * a.ldv + h * D, a.ldv, seq.nk - c0, t, 128);
    }
    group_sync(1 + g, 128);
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
  join(acc1, a.out1, a.ld1, (KEYS ? seq.k0 : seq.q0) + r0, a.scale);
  if (KEYS) join(acc2, a.out2, a.ld2, seq.k0 + r0, 1.f);
}

template <int D>
acid_status forward(const MhaArgs& x, const F32Args& base, cudaStream_t s) {
  static PerContext allowed;
  constexpr size_t smem = (size_t)F32Cfg<D, 16, 2, 1>::FLOATS * 4;
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
  static PerContext allowed_k, allowed_q;
  constexpr size_t smem = (size_t)F32Cfg<D, 16, 2, 2>::FLOATS * 4;
  F32Args a = base;
  if (x.dk != nullptr || x.dv != nullptr) {
    ACID_TRY(allow_smem(allowed_k, mha_backward_f32_kernel<D, true>, smem));
    a.out1 = x.dk;
    a.ld1 = x.lddk;
    a.out2 = x.dv;
    a.ld2 = x.lddv;
    const dim3 grid(mha_slots(a.s.nk, a.s.seqs, a.s.kb != nullptr, 16), a.s.kv_heads);
    launch_pdl(mha_backward_f32_kernel<D, true>, grid, kThreads, smem, s, a);
    ACID_CHECK_LAUNCH();
  }
  if (x.dq != nullptr) {
    ACID_TRY(allow_smem(allowed_q, mha_backward_f32_kernel<D, false>, smem));
    a.out1 = x.dq;
    a.ld1 = x.lddq;
    const dim3 grid(mha_slots(a.s.nq, a.s.seqs, a.s.qb != nullptr, 16), a.s.heads);
    launch_pdl(mha_backward_f32_kernel<D, false>, grid, kThreads, smem, s, a);
    ACID_CHECK_LAUNCH();
  }
  return ACID_OK;
}

F32Args base_args(const MhaArgs& x) {
  F32Args a = {};
  a.s = x.shape;
  a.q = x.q;
  a.k = x.k;
  a.v = x.v;
  a.o = x.out;
  a.dout = x.dout;
  a.ldq = x.ldq;
  a.ldk = x.ldk;
  a.ldv = x.ldv;
  a.ldo = x.ldo;
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
