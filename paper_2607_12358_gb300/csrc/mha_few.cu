// Attention of a few query rows over many keys (acid_mha_forward): single tokens, or one
// for each of many sequences, whose products are too few to fill a tile of the tensor
// cores.  A query row's keys and values are read for it alone, once for up to four of the
// query heads that share a key head.
#include <math.h>

#include <algorithm>

#define ACID_UNIT_WITHOUT_WAITS
#include "mha.cuh"

namespace acid {

BoundsRecord take_bounds_mha_few();
ACID_BOUNDS_READER(take_bounds_mha_few)

namespace {

constexpr int kWarps = 8;  // of a CTA

struct FewArgs {
  MhaShape s;
  const void *q, *k, *v;
  int64_t ldq, ldk, ldv, ldo;
  void* out;
  float* lse;
  float scale;   // of the scores, in the exponential's unit
  int splits, chunks;  // shares of a row's keys; groups of R heads that share a key head
  float* part;   // [row][head][split][D + 2]: unnormalised output, reference max, sum
  int64_t part_floats;
};

// Exponential and logarithm of a type's scores: base 2 by the hardware for bf16, e for fp32.
template <typename T> struct Base;
template <> struct Base<__nv_bfloat16> {
  static constexpr float kUnit = 1.4426950408889634f;
  static __device__ __forceinline__ float exp(float x) { return ex2_approx(x); }
  static __device__ __forceinline__ float lse(float m, float l) { return (m + log2f(l)) * 0.6931471805599453f; }
};
template <> struct Base<float> {
  static constexpr float kUnit = 1.0f;
  static __device__ __forceinline__ float exp(float x) { return expf(x); }
  static __device__ __forceinline__ float lse(float m, float l) { return m + logf(l); }
};

// Running maximum, sum and output of R heads over a lane's 8 columns.
template <typename T, int R>
struct Running {
  float m[R], l[R], o[R][8];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int h = 0; h < R; ++h) {
      m[h] = -INFINITY;
      l[h] = 0.f;
#pragma unroll
      for (int c = 0; c < 8; ++c) o[h][c] = 0.f;
    }
  }
  // Another part of the same rows joins: (m2, l2, o2), which may be empty (l2 = 0).
  __device__ __forceinline__ void join(int h, float m2, float l2, const float* o2) {
    const float mn = fmaxf(m[h], m2), ref = mn == -INFINITY ? 0.f : mn;
    const float a = Base<T>::exp(m[h] - ref), b = Base<T>::exp(m2 - ref);
    m[h] = mn;
    l[h] = a * l[h] + b * l2;
#pragma unroll
    for (int c = 0; c < 8; ++c) o[h][c] = a * o[h][c] + b * o2[c];
  }
};

// CTA (split, key head and chunk of its query heads, query row).  LANES lanes have a key
// row, 8 columns each; a lane has the next BATCH key and value rows on their way, as they
// are stored, while it works on the ones before.  One query head to a key head is HBM
// bound: 32760 keys, 12 heads of 128 35 us with the join, 84% of the copy bandwidth.  With
// more heads or rows to a key the products set the pace, 8 columns a lane and three or four
// shuffles a key (mha_few's table).
template <typename T, int D, int R>
__global__ void __launch_bounds__(32 * kWarps, 2) mha_few_kernel(const __grid_constant__ FewArgs a) {
  constexpr int LANES = D == 32 ? 4 : D == 64 ? 8 : 16, KEYS = 32 / LANES;  // keys a warp has at a time
  constexpr int BATCH = (sizeof(T) == 2 ? 4 : 2) / (R == 4 ? 2 : 1);  // two CTAs to an SM
  __shared__ float joined[kWarps][R][D + 2];
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane / LANES, col = lane % LANES * 8;
  const bool on = col < D;  // (head dim 96: 12 of 16 lanes)
  const int row = blockIdx.z, hk = blockIdx.y / a.chunks, h0 = hk * a.s.group + blockIdx.y % a.chunks * R;
  const int heads = min(R, (hk + 1) * a.s.group - h0);
  const MhaSeq seq = mha_seq(a.s, mha_sequence_of(a.s.qb, a.s.seqs, row));
  if (row < seq.q0 || row >= seq.q0 + seq.nq) return;  // of no sequence
  int first, last;
  mha_keys_of(a.s, seq, row - seq.q0, first, last);
  const int n = max(last - first, 0);
  const int begin = first + (int)((int64_t)n * blockIdx.x / a.splits), end = first + (int)((int64_t)n * (blockIdx.x + 1) / a.splits);
  float q[R][8];
#pragma unroll
  for (int h = 0; h < R; ++h) {
#pragma unroll
    for (int c = 0; c < 8; ++c) q[h][c] = 0.f;
    const int64_t at = (int64_t)row * a.ldq + (h0 + h) * D + col;
    if (on && h < heads && ACID_IN_BOUNDS(kSiteMha, at + 7, (int64_t)a.s.nq * a.ldq))
      load8(static_cast<const T*>(a.q) + at, q[h]);
#pragma unroll
    for (int c = 0; c < 8; ++c) q[h][c] *= a.scale;
  }
  Running<T, R> run;
  run.clear();
  const T* kp = static_cast<const T*>(a.k) + (int64_t)seq.k0 * a.ldk + hk * D + col;
  const T* vp = static_cast<const T*>(a.v) + (int64_t)seq.k0 * a.ldv + hk * D + col;
  constexpr int kStep = kWarps * KEYS * BATCH;
  MhaRaw<T> kr[BATCH], vr[BATCH];
  auto fetch = [&](int j0) {
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const int j = j0 + b * KEYS;
      kr[b].zero();
      vr[b].zero();
      if (on && j < end && ACID_IN_BOUNDS(kSiteMha, (int64_t)(seq.k0 + j) * a.ldk + hk * D + col + 7, a.s.nk * a.ldk) &&
          ACID_IN_BOUNDS(kSiteMha, (int64_t)(seq.k0 + j) * a.ldv + hk * D + col + 7, a.s.nk * a.ldv)) {
        kr[b].load(kp + (int64_t)j * a.ldk);
        vr[b].load(vp + (int64_t)j * a.ldv);
      }
    }
  };
  int j0 = begin + warp * KEYS * BATCH + sub;
  fetch(j0);
  for (; j0 - sub < end; j0 += kStep) {
    MhaRaw<T> kc[BATCH], vc[BATCH];
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      kc[b] = kr[b];
      vc[b] = vr[b];
    }
    fetch(j0 + kStep);
#pragma unroll
    for (int h = 0; h < R; ++h) {
      float s[BATCH], top = -INFINITY;
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        float k[8];
        kc[b].get(k);
        s[b] = 0.f;
#pragma unroll
        for (int c = 0; c < 8; ++c) s[b] = fmaf(q[h][c], k[c], s[b]);
#pragma unroll
        for (int off = LANES / 2; off > 0; off >>= 1) s[b] += __shfl_xor_sync(0xffffffffu, s[b], off);
        if (j0 + b * KEYS >= end) s[b] = -INFINITY;
        top = fmaxf(top, s[b]);
      }
      const float mn = fmaxf(run.m[h], top), ref = mn == -INFINITY ? 0.f : mn;
      const float down = Base<T>::exp(run.m[h] - ref);
      run.m[h] = mn;
      run.l[h] *= down;
#pragma unroll
      for (int c = 0; c < 8; ++c) run.o[h][c] *= down;
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        const float p = Base<T>::exp(s[b] - ref);
        run.l[h] += p;
        float v[8];
        vc[b].get(v);
#pragma unroll
        for (int c = 0; c < 8; ++c) run.o[h][c] = fmaf(p, v[c], run.o[h][c]);
      }
    }
  }
  // the warp's key groups, then the CTA's warps, each in a fixed order
#pragma unroll
  for (int off = LANES; off < 32; off *= 2)
#pragma unroll
    for (int h = 0; h < R; ++h) {
      float o2[8];
      const float m2 = __shfl_xor_sync(0xffffffffu, run.m[h], off), l2 = __shfl_xor_sync(0xffffffffu, run.l[h], off);
#pragma unroll
      for (int c = 0; c < 8; ++c) o2[c] = __shfl_xor_sync(0xffffffffu, run.o[h][c], off);
      run.join(h, m2, l2, o2);
    }
  if (sub == 0)
#pragma unroll
    for (int h = 0; h < R; ++h) {
      if (on)
#pragma unroll
        for (int c = 0; c < 8; ++c) joined[warp][h][col + c] = run.o[h][c];
      if (col == 0) {
        joined[warp][h][D] = run.m[h];
        joined[warp][h][D + 1] = run.l[h];
      }
    }
  __syncthreads();
  for (int h = 0; h < heads; ++h) {
    float m = -INFINITY, l = 0.f;
    for (int w = 0; w < kWarps; ++w) m = fmaxf(m, joined[w][h][D]);
    const float ref = m == -INFINITY ? 0.f : m;
    float by[kWarps];
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      by[w] = Base<T>::exp(joined[w][h][D] - ref);
      l += by[w] * joined[w][h][D + 1];
    }
    const int64_t hr = (int64_t)row * a.s.heads + h0 + h;
    for (int c = threadIdx.x; c < D; c += 32 * kWarps) {
      float o = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) o += by[w] * joined[w][h][c];
      if (a.splits > 1) {
        const int64_t at = (hr * a.splits + blockIdx.x) * (D + 2) + c;
        if (ACID_IN_BOUNDS(kSiteMha, at, a.part_floats)) a.part[at] = o;
      } else {
        const int64_t at = (int64_t)row * a.ldo + (h0 + h) * D + c;
        if (ACID_IN_BOUNDS(kSiteMha, at, (int64_t)a.s.nq * a.ldo))
          io<T>::st(static_cast<T*>(a.out) + at, l == 0.f ? 0.f : o / l);
      }
    }
    if (threadIdx.x == 0) {
      if (a.splits > 1) {
        const int64_t at = (hr * a.splits + blockIdx.x) * (D + 2) + D;
        if (ACID_IN_BOUNDS(kSiteMha, at + 1, a.part_floats)) {
          a.part[at] = m;
          a.part[at + 1] = l;
        }
      } else if (ACID_IN_BOUNDS(kSiteMha, (h0 + h) * (int64_t)a.s.nq + row, (int64_t)a.s.heads * a.s.nq)) {
        a.lse[(int64_t)(h0 + h) * a.s.nq + row] = l == 0.f ? -INFINITY : Base<T>::lse(m, l);
      }
    }
  }
}

// Joins the shares of a row and head: a CTA's warps take them in turn, and their sums
// are added in the warps' order.
constexpr int kJoinWarps = 8;
template <typename T, int D>
__global__ void __launch_bounds__(32 * kJoinWarps) mha_few_join_kernel(const __grid_constant__ FewArgs a) {
  __shared__ float sums[kJoinWarps][D + 1], tops[kJoinWarps];
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int row = blockIdx.x / a.s.heads, h = blockIdx.x % a.s.heads;
  if (a.s.qb != nullptr) {  // rows of no sequence stay as they are
    const MhaSeq seq = mha_seq(a.s, mha_sequence_of(a.s.qb, a.s.seqs, row));
    if (row < seq.q0 || row >= seq.q0 + seq.nq) return;
  }
  const float* p = a.part + (int64_t)blockIdx.x * a.splits * (D + 2);
  if (!ACID_IN_BOUNDS(kSiteMha, (blockIdx.x + (int64_t)1) * a.splits * (D + 2) - 1, a.part_floats)) return;
  float m = -INFINITY;
  for (int s = threadIdx.x; s < a.splits; s += 32 * kJoinWarps) m = fmaxf(m, p[(int64_t)s * (D + 2) + D]);
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
  if (lane == 0) tops[warp] = m;
  __syncthreads();
  for (int w = 0; w < kJoinWarps; ++w) m = fmaxf(m, tops[w]);
  const float ref = m == -INFINITY ? 0.f : m;
  float l = 0.f, o[D / 32] = {};
#pragma unroll 4
  for (int s = warp; s < a.splits; s += kJoinWarps) {
    const float* part = p + (int64_t)s * (D + 2);
    const float by = Base<T>::exp(part[D] - ref);
    l = fmaf(by, part[D + 1], l);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] = fmaf(by, part[i * 32 + lane], o[i]);
  }
#pragma unroll
  for (int i = 0; i < D / 32; ++i) sums[warp][i * 32 + lane] = o[i];
  if (lane == 0) sums[warp][D] = l;
  __syncthreads();
  const int c = threadIdx.x;
  if (c >= D) return;
  float sum = 0.f;
  l = 0.f;
#pragma unroll
  for (int w = 0; w < kJoinWarps; ++w) {
    sum += sums[w][c];
    l += sums[w][D];
  }
  const int64_t at = (int64_t)row * a.ldo + h * D + c;
  if (!ACID_IN_BOUNDS(kSiteMha, at, (int64_t)a.s.nq * a.ldo)) return;
  io<T>::st(static_cast<T*>(a.out) + at, l == 0.f ? 0.f : sum / l);
  if (c == 0 && ACID_IN_BOUNDS(kSiteMha, h * (int64_t)a.s.nq + row, (int64_t)a.s.heads * a.s.nq))
    a.lse[(int64_t)h * a.s.nq + row] = l == 0.f ? -INFINITY : Base<T>::lse(m, l);
}

// Query heads of a key head that a CTA takes.
int heads_at_once(const MhaShape& s) { return s.group >= 4 ? 4 : s.group >= 2 ? 2 : 1; }
// Shares of a row's keys: one wave of two CTAs an SM, of 128 keys or more.
int few_splits(const MhaShape& s) {
  const int64_t r = heads_at_once(s), ctas = (int64_t)s.nq * s.kv_heads * ((s.group + r - 1) / r);
  const int64_t most = std::max<int64_t>(1, s.nk / s.seqs / 128);
  return (int)std::max<int64_t>(1, std::min<int64_t>({most, 2 * (int64_t)num_sms() / ctas, 128}));
}

template <typename T, int D, int R>
acid_status launch(const MhaArgs& x, cudaStream_t s) {
  FewArgs a = {};
  a.s = x.shape;
  a.q = x.q;
  a.k = x.k;
  a.v = x.v;
  a.ldq = x.ldq;
  a.ldk = x.ldk;
  a.ldv = x.ldv;
  a.out = x.out;
  a.ldo = x.ldo;
  a.lse = x.lse;
  a.scale = x.scale * Base<T>::kUnit;
  a.splits = few_splits(a.s);
  a.chunks = (a.s.group + R - 1) / R;
  a.part = static_cast<float*>(x.part);
  a.part_floats = (int64_t)(x.part_bytes / sizeof(float));
  launch_pdl(mha_few_kernel<T, D, R>, dim3(a.splits, a.s.kv_heads * a.chunks, a.s.nq), 32 * kWarps, 0, s, a);
  ACID_CHECK_LAUNCH();
  if (a.splits > 1) {
    launch_pdl(mha_few_join_kernel<T, D>, (unsigned)(a.s.nq * a.s.heads), 32 * kJoinWarps, 0, s, a);
    ACID_CHECK_LAUNCH();
  }
  return ACID_OK;
}
template <typename T, int D>
acid_status by_heads(const MhaArgs& x, cudaStream_t s) {
  switch (heads_at_once(x.shape)) {
    case 1: return launch<T, D, 1>(x, s);
    case 2: return launch<T, D, 2>(x, s);
    default: return launch<T, D, 4>(x, s);
  }
}

}  // namespace

// Whether a call goes to this kernel.  Its time grows with the rows and heads, where a tile
// of the tensor cores (256 rows; fp32: 16) takes the same for one as for all of its rows.
// us here / on tiles, cold caches, replayed from a graph, which adds about 8 to both:
//                                         1 row    2 rows     4 rows a sequence
//   12 x 128, 512 keys                    11 / 17  11 / 18    13 / 18
//   12 x 128, 4726 keys                   18 / 26  20 / 26    24 / 26
//   24 x 128, 4726 keys                   24 / 30  28 / 30    36 / 30
//   12 x 128, 32760 keys                  50 / 59  61 / 58    85 / 59
//   24 on 8 x 128, 32760 keys             48 / 75  75 / 75   161 / 75
//   16 on 1 x 128, 32760 keys             28 / 56  40 / 55    67 / 55
//   30 x 64, 32760 keys                   61 / 70  72 / 70   120 / 71
//   8 sequences, 12 x 128, 512 keys       18 / 20  18 / 20    26 / 19
//   64 sequences, 12 x 128, 64 keys       20 / 38  26 / 38    40 / 38
//   64 sequences, 24 on 8 x 128, 4096    274 / 505 511 / 511 971 / 519
//   fp32, 4 x 64, 256 keys                13 / 16  13 / 16    12 / 16
//   fp32, 12 x 128, 2048 keys             18 / 120 18 / 120   22 / 120
//   fp32, 16 sequences, 4 x 64, 512 keys  18 / 26             18 / 26
// One row a sequence is always faster here, two where query heads share the loads.  Else up to
// four in bf16 as long as all rows' products with the keys are few.  Lengths are on the device,
// so the rule goes by their averages: what it keeps from here is also a batch of 63 sequences of
// one row and one of 190 rows against 32760 keys (3094 / 392).  fp32 products take as long on
// tiles as here, and few rows leave most SMs without a tile.
bool mha_few(const MhaArgs& a) {
  const MhaShape& s = a.shape;
  if (s.nk == 0 || s.nq > 65535 || s.heads > 4096) return false;
  const int64_t seqs = s.seqs;
  if (s.nq <= (s.group > 1 ? 2 : 1) * seqs) return true;
  const int64_t products = (int64_t)s.nq * s.heads * a.head_dim * (s.nk / seqs);
  return s.nq <= 4 * seqs && (a.dtype == ACID_FP32 || products <= 1 << 25);
}

size_t mha_few_bytes(const MhaArgs& x) {
  const int splits = few_splits(x.shape);
  return splits > 1 ? (size_t)x.shape.nq * x.shape.heads * splits * (x.head_dim + 2) * sizeof(float) : 0;
}

acid_status mha_forward_few(const MhaArgs& x, cudaStream_t s) {
  if (x.dtype == ACID_BF16) return x.head_dim == 64 ? by_heads<__nv_bfloat16, 64>(x, s) : by_heads<__nv_bfloat16, 128>(x, s);
  switch (x.head_dim) {
    case 32: return by_heads<float, 32>(x, s);
    case 64: return by_heads<float, 64>(x, s);
    case 96: return by_heads<float, 96>(x, s);
    default: return by_heads<float, 128>(x, s);
  }
}

}  // namespace acid
