// Norm sites: the gate, residual, norms and modulation between two branches of
// a block, and their gradients (acid_norm_site_*).
#include <algorithm>
#include <string>

#define ACID_UNIT_WITHOUT_WAITS
#include "common.cuh"
#include "internal.h"

namespace acid {

BoundsRecord take_bounds_site();
ACID_BOUNDS_READER(take_bounds_site)

namespace {

using bf16 = __nv_bfloat16;
constexpr int kMaxWidth = 4096;           // 8 warps of 16 columns a lane
constexpr int kMaxWarps = kMaxWidth / 512;

// What both directions read, as the kernels see it.
struct Site {
  int64_t rows, first, group;  // group >= 1
  int d, post, pre, tanh;
  float eps, res, branch;
  const float *gate, *scale, *shift, *post_w, *pre_w;
  int64_t ld_mod, groups;
};
__device__ __forceinline__ int64_t group_of(const Site& s, int64_t row) {
  return row < s.first ? 0 : (s.first > 0) + (row - s.first) / s.group;
}
// First row of group g, and of the one after it.
__device__ __forceinline__ int64_t group_begin(const Site& s, int64_t g) {
  if (s.first > 0) {
    if (g == 0) return 0;
    --g;
  }
  return s.first + g * s.group;
}
__device__ __forceinline__ int64_t group_end(const Site& s, int64_t g) {
  return s.first > 0 && g == 0 ? s.first : min(s.rows, group_begin(s, g) + s.group);
}

struct SiteFwd {
  Site s;
  const void *x, *y;
  void *r, *u;
  int64_t ldx, ldy, ldr, ldu;
};
struct SiteBwd {
  Site s;
  const void *du, *r, *y, *dr;
  int64_t lddu, ldr, ldy, lddr;
  void *dx, *dy;
  int64_t lddx, lddy;
  float *dgate, *dscale, *dshift, *dpost_w, *dpre_w;
  int64_t ld_dmod;
  float* part;   // [2 ctas][3][d]: sums of a group's rows that lie in one CTA
  float* wpart;  // [ctas][2][d]: the CTA's share of dpre_w and dpost_w
  int64_t per;   // rows of a CTA
};

// A thread's 16 columns: two octets, 8 (tid + j blockDim) ..., as eight fp32
// pairs, so that one instruction does the arithmetic of two columns.  Octets
// past the row's end hold zeros all through.
struct Cols {
  uint64_t v[8];
};
#define FOR_PAIRS _Pragma("unroll") for (int i = 0; i < 8; ++i)
__device__ __forceinline__ uint64_t f2_same(float x) { return f2_pack(x, x); }
__device__ __forceinline__ float f2_total(uint64_t x) {
  float a, b;
  f2_unpack(x, a, b);
  return a + b;
}
// Sum of the pairs.
__device__ __forceinline__ float total(const uint64_t (&p)[8]) {
  return f2_total(f2_add(f2_add(f2_add(p[0], p[1]), f2_add(p[2], p[3])), f2_add(f2_add(p[4], p[5]), f2_add(p[6], p[7]))));
}
__device__ __forceinline__ float total(const Cols& a) { return total(a.v); }
// Sum of the products.
__device__ __forceinline__ float dot(const Cols& a, const Cols& b) {
  uint64_t s = f2_mul(a.v[0], b.v[0]), t = f2_mul(a.v[1], b.v[1]);
#pragma unroll
  for (int i = 2; i < 8; i += 2) {
    s = f2_fma(a.v[i], b.v[i], s);
    t = f2_fma(a.v[i + 1], b.v[i + 1], t);
  }
  return f2_total(f2_add(s, t));
}

struct Place {
  int c[2], d;  // first column of each octet
  bool on[2];
};
__device__ __forceinline__ Place place(int d) {
  const int c0 = threadIdx.x * 8, c1 = c0 + blockDim.x * 8;
  return {{c0, c1}, d, {c0 < d, c1 < d}};
}
__device__ __forceinline__ void fill(Cols& a, int j, float x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) a.v[4 * j + i] = f2_same(x);
}
// Columns of a vector; `none` in all of the row's where there is none.
__device__ __forceinline__ Cols vec(const float* p, const Place& at, float none) {
  Cols a;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    if (!at.on[j] || p == nullptr) {
      fill(a, j, at.on[j] ? none : 0.f);
    } else if (ACID_IN_BOUNDS(kSiteNormSite, at.c[j] + 7, at.d)) {
      const float4 lo = *reinterpret_cast<const float4*>(p + at.c[j]);
      const float4 hi = *reinterpret_cast<const float4*>(p + at.c[j] + 4);
      a.v[4 * j] = f2_pack(lo.x, lo.y);
      a.v[4 * j + 1] = f2_pack(lo.z, lo.w);
      a.v[4 * j + 2] = f2_pack(hi.x, hi.y);
      a.v[4 * j + 3] = f2_pack(hi.z, hi.w);
    }
  }
  return a;
}
__device__ __forceinline__ void times(Cols& a, const Cols& b) { FOR_PAIRS a.v[i] = f2_mul(a.v[i], b.v[i]); }
__device__ __forceinline__ void plus(Cols& a, float x, const Place& at) {
  FOR_PAIRS a.v[i] = f2_add(a.v[i], f2_same(at.on[i >> 2] ? x : 0.f));
}
// branch_scale times the gate's columns of a group.
__device__ __forceinline__ Cols gate_cols(const Site& s, int64_t m, const Place& at) {
  Cols g = vec(s.gate ? s.gate + m : nullptr, at, 1.f);
  FOR_PAIRS {
    if (s.tanh && s.gate) {
      float lo, hi;
      f2_unpack(g.v[i], lo, hi);
      g.v[i] = f2_pack(tanhf(lo), tanhf(hi));
    }
    g.v[i] = f2_mul(g.v[i], f2_same(s.branch));
  }
  return g;
}
// 1 + scale of a group.
__device__ __forceinline__ Cols scale_cols(const Site& s, int64_t m, const Place& at) {
  Cols a = vec(s.scale ? s.scale + m : nullptr, at, 0.f);
  plus(a, 1.f, at);
  return a;
}

template <typename T>
__device__ __forceinline__ void store_pairs(T* p, const uint64_t* v) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) f2_unpack(v[i], f[2 * i], f[2 * i + 1]);
  store8(p, f);
}
// To a row of the operand, whose first element is `row`.
template <typename T>
__device__ __forceinline__ void put(T* row, const Place& at, const Cols& a, int64_t r, int64_t rows) {
#pragma unroll
  for (int j = 0; j < 2; ++j)
    if (at.on[j] && ACID_IN_BOUNDS(kSiteNormSite, r, rows)) store_pairs(row + at.c[j], a.v + 4 * j);
}

// Sums of N values over the CTA; every thread gets them.  The first shuffles
// hand half of the values to half of the lanes, so that four sums take six
// shuffles and not twenty.  Rounds alternate between two buffers, so that one
// barrier a round is enough: a thread writes a buffer again behind the other
// one's barrier.  Slots of warps that the CTA does not have are zero.
struct Reducer {
  float4 (*red)[kMaxWarps];
  int round, warps, warp, lane;
  template <int N>
  __device__ __forceinline__ float4 sum(float a, float b = 0.f, float c = 0.f, float e = 0.f) {
    float* out = reinterpret_cast<float*>(&red[round][warp]);
    if constexpr (N > 2) {
      const bool hi = lane & 16, mid = lane & 8;
      float p = hi ? c : a, q = hi ? e : b;
      p += __shfl_xor_sync(0xffffffffu, hi ? a : c, 16);
      q += __shfl_xor_sync(0xffffffffu, hi ? b : e, 16);
      a = mid ? q : p;
      a += __shfl_xor_sync(0xffffffffu, mid ? p : q, 8);
    } else if constexpr (N == 2) {
      const bool hi = lane & 16;
      const float p = hi ? b : a;
      a = p + __shfl_xor_sync(0xffffffffu, hi ? a : b, 16);
      a += __shfl_xor_sync(0xffffffffu, a, 8);
    } else {
      a += __shfl_xor_sync(0xffffffffu, a, 16);
      a += __shfl_xor_sync(0xffffffffu, a, 8);
    }
    a += __shfl_xor_sync(0xffffffffu, a, 4);
    a += __shfl_xor_sync(0xffffffffu, a, 2);
    a += __shfl_xor_sync(0xffffffffu, a, 1);
    constexpr int kOwn = N > 2 ? 8 : N == 2 ? 16 : 32;  // lanes that hold one of the sums
    if ((lane & (kOwn - 1)) == 0) out[lane / kOwn] = a;
    __syncthreads();
    const float4* t = red[round];
    round ^= 1;
    auto add = [](float4 x, float4 y) { return make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w); };
    float4 v = add(add(t[0], t[1]), add(t[2], t[3]));
    if (warps > 4) v = add(v, add(add(t[4], t[5]), add(t[6], t[7])));
    return v;
  }
};
__device__ __forceinline__ Reducer reducer(float4 (*red)[kMaxWarps]) {
  if (threadIdx.x < 2 * kMaxWarps) red[0][threadIdx.x] = make_float4(0.f, 0.f, 0.f, 0.f);
  __syncthreads();
  return {red, 0, (int)(blockDim.x >> 5), (int)(threadIdx.x >> 5), (int)(threadIdx.x & 31)};
}

// A thread's own ring of row pieces in shared memory: it copies the columns
// that it will work on and nobody else reads them, so that waiting for its own
// copies is all the synchronisation there is.  A stage is planes of 16 bytes a
// thread.
template <typename T>
constexpr int kPlanes = sizeof(T);  // of 16 columns
template <typename T>
__device__ __forceinline__ void stage(uint8_t* mine, int plane, const T* row, const Place& at, int64_t r, int64_t rows) {
  constexpr int kOctet = kPlanes<T> / 2;
#pragma unroll
  for (int j = 0; j < 2; ++j)
    if (at.on[j] && ACID_IN_BOUNDS(kSiteNormSite, r, rows))
#pragma unroll
      for (int i = 0; i < kOctet; ++i)
        cp_async<16>(mine + (plane + j * kOctet + i) * blockDim.x * 16,
                     reinterpret_cast<const uint8_t*>(row + at.c[j]) + 16 * i, true);
}
template <typename T>
__device__ __forceinline__ Cols unstage(const uint8_t* mine, int plane, const Place& at) {
  constexpr int kOctet = kPlanes<T> / 2;
  Cols a;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    if (!at.on[j]) {
      fill(a, j, 0.f);
      continue;
    }
    const uint8_t* q = mine + (plane + j * kOctet) * blockDim.x * 16;
    uint64_t* v = a.v + 4 * j;
    if constexpr (sizeof(T) == 2) {
      const uint4 u = *reinterpret_cast<const uint4*>(q);
      v[0] = f2_pack(bf16_lo(u.x), bf16_hi(u.x));
      v[1] = f2_pack(bf16_lo(u.y), bf16_hi(u.y));
      v[2] = f2_pack(bf16_lo(u.z), bf16_hi(u.z));
      v[3] = f2_pack(bf16_lo(u.w), bf16_hi(u.w));
    } else {
      const ulonglong2 lo = *reinterpret_cast<const ulonglong2*>(q);
      const ulonglong2 hi = *reinterpret_cast<const ulonglong2*>(q + blockDim.x * 16);
      v[0] = lo.x;
      v[1] = lo.y;
      v[2] = hi.x;
      v[3] = hi.y;
    }
  }
  return a;
}

// A CTA takes a row at a time; row k of CTA b is b start + k step, k < count.
constexpr int kFwdStages = 4;
template <typename TS, typename TB, bool BRANCH>
__global__ void __launch_bounds__(32 * kMaxWarps, 2) site_forward_kernel(SiteFwd a, int64_t start, int64_t step,
                                                                        uint32_t count) {
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ float4 red[2][kMaxWarps];
  pdl_wait();
  const Site& s = a.s;
  const Place at = place(s.d);
  Reducer sums = reducer(red);
  const float d = (float)s.d, per_d = 1.f / d;
  int64_t row = blockIdx.x * start;
  const uint32_t n = row < s.rows ? (uint32_t)min((int64_t)count, (s.rows - 1 - row) / step + 1) : 0;
  constexpr int kStage = kPlanes<TS> + (BRANCH ? kPlanes<TB> : 0);
  uint8_t* mine = ring + threadIdx.x * 16;
  const int stride = kStage * blockDim.x * 16;
  int64_t ahead = row;  // the next row to be copied
  uint32_t copied = 0;
  int to = 0;
  auto issue = [&] {
    if (copied < n) {
      stage(mine + to * stride, 0, static_cast<const TS*>(a.x) + ahead * a.ldx, at, ahead, s.rows);
      if constexpr (BRANCH)
        stage(mine + to * stride, kPlanes<TS>, static_cast<const TB*>(a.y) + ahead * a.ldy, at, ahead, s.rows);
      ahead += step;
      ++copied;
    }
    to = to + 1 == kFwdStages ? 0 : to + 1;
    cp_async_commit();
  };
  for (int k = 0; k < kFwdStages - 1; ++k) issue();
  const bool wants_mean = s.pre == ACID_NORM_LAYER && a.u != nullptr;
  int st = 0;
  for (uint32_t k = 0; k < n;) {
    // the rows of one group
    const int64_t g = group_of(s, row), m = g * s.ld_mod;
    const uint32_t stop = (uint32_t)min((int64_t)n, k + (group_end(s, g) - 1 - row) / step + 1);
    Cols gw, sc = scale_cols(s, m, at);  // gate and post_w, (1 + scale) and pre_w, shift
    const Cols sh = vec(s.shift ? s.shift + m : nullptr, at, 0.f);
    times(sc, vec(s.pre_w, at, 1.f));
    if constexpr (BRANCH) {
      gw = gate_cols(s, m, at);
      times(gw, vec(s.post_w, at, 1.f));
    }
    for (; k < stop; ++k, row += step) {
      cp_async_wait<kFwdStages - 2>();
      Cols r = unstage<TS>(mine + st * stride, 0, at);
      FOR_PAIRS r.v[i] = f2_mul(r.v[i], f2_same(s.res));
      float mean = 0.f;
      if constexpr (BRANCH) {
        Cols y = unstage<TB>(mine + st * stride, kPlanes<TS>, at);
        issue();
        if (s.post == ACID_NORM_LAYER) plus(y, -(sums.sum<1>(total(y)).x / d), at);
        // the sum of r comes with the branch's sum of squares, from those of x and of g w y
        const float sq = dot(y, y);
        times(y, gw);
        float inv = 1.f;
        if (s.post != ACID_NORM_NONE || wants_mean) {
          const float4 t = sums.sum<3>(sq, total(y), total(r));
          if (s.post != ACID_NORM_NONE) inv = rsqrtf(fmaf(t.x, per_d, s.eps));
          mean = fmaf(inv, t.y, t.z) / d;
        }
        FOR_PAIRS r.v[i] = f2_fma(f2_same(inv), y.v[i], r.v[i]);
      } else {
        issue();
        if (wants_mean) mean = sums.sum<1>(total(r)).x / d;
      }
      st = st + 1 == kFwdStages ? 0 : st + 1;
      if (a.r != nullptr) put(static_cast<TS*>(a.r) + row * a.ldr, at, r, row, s.rows);
      if (a.u == nullptr) continue;
      if (s.pre != ACID_NORM_NONE) {
        if (s.pre == ACID_NORM_LAYER) plus(r, -mean, at);
        const float inv = rsqrtf(fmaf(sums.sum<1>(dot(r, r)).x, per_d, s.eps));
        FOR_PAIRS r.v[i] = f2_mul(r.v[i], f2_same(inv));
      }
      FOR_PAIRS r.v[i] = f2_fma(r.v[i], sc.v[i], sh.v[i]);
      put(static_cast<TB*>(a.u) + row * a.ldu, at, r, row, s.rows);
    }
  }
}

// Gradients of the site's vectors for one group from the raw sums
// sum du, sum du n and sum dr p over its rows (which = 0, 1, 2): one column.
__device__ __forceinline__ void put_sum(const SiteBwd& a, int which, int64_t g, int c, float v) {
  const Site& s = a.s;
  float* out = which == 0 ? a.dshift : which == 1 ? a.dscale : a.dgate;
  if (out == nullptr || !ACID_IN_BOUNDS(kSiteNormSite, c, s.d)) return;
  if (which == 1 && s.pre_w != nullptr) v *= s.pre_w[c];
  if (which == 2) {
    const float th = s.tanh && s.gate ? tanhf(s.gate[g * s.ld_mod + c]) : 0.f;
    v *= s.branch * (1.f - th * th) * (s.post_w != nullptr ? s.post_w[c] : 1.f);
  }
  out[g * a.ld_dmod + c] = v;
}
// The same for a thread's columns.
__device__ __forceinline__ void put_sums(const SiteBwd& a, int which, int64_t g, int64_t m, const Place& at, Cols v) {
  const Site& s = a.s;
  float* out = which == 0 ? a.dshift : which == 1 ? a.dscale : a.dgate;
  if (out == nullptr) return;
  if (which == 1) times(v, vec(s.pre_w, at, 1.f));
  if (which == 2) {
    times(v, vec(s.post_w, at, 1.f));
    const Cols t = vec(s.tanh && s.gate ? s.gate + m : nullptr, at, 0.f);
    FOR_PAIRS {
      float lo, hi;
      f2_unpack(t.v[i], lo, hi);
      lo = tanhf(lo);
      hi = tanhf(hi);
      v.v[i] = f2_mul(v.v[i], f2_pack(s.branch * (1.f - lo * lo), s.branch * (1.f - hi * hi)));
    }
  }
  put(out + g * a.ld_dmod, at, v, g, s.groups);
}

// The gradients.  CTA b takes the rows [b per, (b + 1) per) and keeps the sums
// over the rows of its group in registers.  A group that lies in the CTA's rows
// is finished here; of one that reaches over their edge the sums go to the
// CTA's slot 2 b (the group began earlier) or 2 b + 1 (it begins here), and
// site_join_kernel adds the slots.
// (two stages where four fp32 rows of 4096 columns have to fit)
template <typename TS, typename TB>
constexpr int kBwdStages = sizeof(TS) + sizeof(TB) == 8 ? 2 : 3;
template <typename TS, typename TB>
__global__ void __launch_bounds__(384, 1) site_backward_kernel(SiteBwd a) {
  constexpr int kStages = kBwdStages<TS, TB>;
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ float4 red[2][kMaxWarps];
  pdl_wait();
  const Site& s = a.s;
  const Place at = place(s.d);
  Reducer sums = reducer(red);
  const float d = (float)s.d, per_d = 1.f / d;
  const int64_t begin = blockIdx.x * a.per, end = min(s.rows, begin + a.per);
  constexpr int kR = 0, kDr = kPlanes<TS>, kY = 2 * kPlanes<TS>, kDu = kY + kPlanes<TB>, kStage = kDu + kPlanes<TB>;
  uint8_t* mine = ring + threadIdx.x * 16;
  const int stride = kStage * blockDim.x * 16;
  ulonglong2* wsum = reinterpret_cast<ulonglong2*>(ring + kStages * stride) + threadIdx.x;  // 8 planes of 4 columns
  int64_t ahead = begin;
  int to = 0;
  auto issue = [&] {
    if (ahead < end) {
      uint8_t* p = mine + to * stride;
      if (a.du != nullptr) {
        stage(p, kR, static_cast<const TS*>(a.r) + ahead * a.ldr, at, ahead, s.rows);
        stage(p, kDu, static_cast<const TB*>(a.du) + ahead * a.lddu, at, ahead, s.rows);
      }
      if (a.dr != nullptr) stage(p, kDr, static_cast<const TS*>(a.dr) + ahead * a.lddr, at, ahead, s.rows);
      if (a.y != nullptr) stage(p, kY, static_cast<const TB*>(a.y) + ahead * a.ldy, at, ahead, s.rows);
      ++ahead;
    }
    to = to + 1 == kStages ? 0 : to + 1;
    cp_async_commit();
  };
  for (int k = 0; k < kStages - 1; ++k) issue();
  const bool weights = a.dpre_w != nullptr || a.dpost_w != nullptr;
  for (int i = 0; weights && i < 8; ++i) wsum[i * blockDim.x] = make_ulonglong2(0, 0);
  const Cols zero = {};
  int st = 0;
  for (int64_t row = begin; row < end;) {
    const int64_t g = group_of(s, row), m = g * s.ld_mod, from = row, last = min(end, group_end(s, g));
    Cols A = {}, S = {}, T = {}, sc = scale_cols(s, m, at), gw = gate_cols(s, m, at);
    times(sc, vec(s.pre_w, at, 1.f));
    times(gw, vec(s.post_w, at, 1.f));
    for (; row < last; ++row) {
      cp_async_wait<kStages - 2>();
      const uint8_t* p = mine + st * stride;
      Cols n = a.du != nullptr ? unstage<TS>(p, kR, at) : zero, du = a.du != nullptr ? unstage<TB>(p, kDu, at) : zero;
      Cols y = a.y != nullptr ? unstage<TB>(p, kY, at) : zero, dr = a.dr != nullptr ? unstage<TS>(p, kDr, at) : zero;
      issue();
      st = st + 1 == kStages ? 0 : st + 1;
      if (s.pre == ACID_NORM_LAYER || s.post == ACID_NORM_LAYER) {
        const float4 t = sums.sum<2>(total(n), total(y));
        if (s.pre == ACID_NORM_LAYER) plus(n, -(t.x / d), at);
        if (s.post == ACID_NORM_LAYER) plus(y, -(t.y / d), at);
      }
      FOR_PAIRS A.v[i] = f2_add(A.v[i], du.v[i]);
      // S takes du n before du becomes dn = du (1 + scale) pre_w, so the root comes first
      Cols dn = du;
      times(dn, sc);
      float in = 1.f, ip = 1.f, mean = 0.f, along = 0.f;
      if (s.pre != ACID_NORM_NONE || s.post != ACID_NORM_NONE) {
        const float4 t = sums.sum<4>(dot(n, n), dot(y, y), total(dn), dot(dn, n));
        if (s.pre != ACID_NORM_NONE) {
          in = rsqrtf(fmaf(t.x, per_d, s.eps));
          mean = s.pre == ACID_NORM_LAYER ? t.z * per_d : 0.f;
          along = t.w * in * in * per_d;
        }
        if (s.post != ACID_NORM_NONE) ip = rsqrtf(fmaf(t.y, per_d, s.eps));
      }
      FOR_PAIRS {
        S.v[i] = f2_fma(f2_mul(du.v[i], f2_same(in)), n.v[i], S.v[i]);
        dn.v[i] = f2_fma(n.v[i], f2_same(-along), dn.v[i]);
      }
      plus(dn, -mean, at);
      FOR_PAIRS {
        dr.v[i] = f2_fma(f2_same(in), dn.v[i], dr.v[i]);
        y.v[i] = f2_mul(y.v[i], f2_same(ip));
        T.v[i] = f2_fma(dr.v[i], y.v[i], T.v[i]);
      }
      if (a.dx != nullptr) {
        Cols o;
        FOR_PAIRS o.v[i] = f2_mul(dr.v[i], f2_same(s.res));
        put(static_cast<TS*>(a.dx) + row * a.lddx, at, o, row, s.rows);
      }
      if (a.dy == nullptr) continue;
      times(dr, gw);
      if (s.post != ACID_NORM_NONE) {
        const float4 t = sums.sum<2>(total(dr), dot(dr, y));
        FOR_PAIRS dr.v[i] = f2_fma(y.v[i], f2_same(-t.y * per_d), dr.v[i]);
        if (s.post == ACID_NORM_LAYER) plus(dr, -t.x * per_d, at);
        FOR_PAIRS dr.v[i] = f2_mul(dr.v[i], f2_same(ip));
      }
      put(static_cast<TB*>(a.dy) + row * a.lddy, at, dr, row, s.rows);
    }
    if (weights) {  // dpre_w gathers (1 + scale) S, dpost_w branch_scale gate T
      const Cols f = scale_cols(s, m, at), h = gate_cols(s, m, at);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ulonglong2& p = wsum[i * blockDim.x];
        ulonglong2& q = wsum[(4 + i) * blockDim.x];
        p = make_ulonglong2(f2_fma(f.v[2 * i], S.v[2 * i], p.x), f2_fma(f.v[2 * i + 1], S.v[2 * i + 1], p.y));
        q = make_ulonglong2(f2_fma(h.v[2 * i], T.v[2 * i], q.x), f2_fma(h.v[2 * i + 1], T.v[2 * i + 1], q.y));
      }
    }
    const bool starts = group_begin(s, g) == from, ends = group_end(s, g) == last;
    if (starts && ends) {
      put_sums(a, 0, g, m, at, A);
      put_sums(a, 1, g, m, at, S);
      put_sums(a, 2, g, m, at, T);
    } else {
      const int64_t i = 2 * (int64_t)blockIdx.x + starts, slots = 2 * (int64_t)gridDim.x;
      float* slot = a.part + i * 3 * s.d;
      put(slot, at, A, i, slots);
      put(slot + s.d, at, S, i, slots);
      put(slot + 2 * s.d, at, T, i, slots);
    }
  }
  if (!weights) return;
  float* wp = a.wpart + (int64_t)blockIdx.x * 2 * s.d;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    Cols v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const ulonglong2 p = wsum[(4 * w + i) * blockDim.x];
      v.v[2 * i] = p.x;
      v.v[2 * i + 1] = p.y;
    }
    put(wp + w * s.d, at, v, blockIdx.x, gridDim.x);
  }
}

// Adds the CTAs' slots in the CTAs' order.  A job is one vector of one group
// that reaches over an edge (jobs counted by groups, or by CTAs where these are
// fewer: the group that begins in the CTA and leaves it), or one of the two
// weights' gradients.  `segs` warps share a job's slots, a lane takes a column.
constexpr int kJoinWarps = 16;
__global__ void __launch_bounds__(32 * kJoinWarps) site_join_kernel(SiteBwd a, int ctas, int jobs, int segs,
                                                                   bool by_cta) {
  __shared__ float part[kJoinWarps][32];
  pdl_wait();
  const Site& s = a.s;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, seg = warp % segs;
  const int c = blockIdx.x * 32 + lane, d = s.d, job = blockIdx.y * (kJoinWarps / segs) + warp / segs;
  const int which = job / jobs;  // 0 .. 2: dshift, dscale, dgate; 3, 4: dpre_w, dpost_w
  int64_t g = 0, lo = 0, hi = -1;  // slots lo .. hi
  if (which < 3) {
    const int64_t i = job - which * jobs;
    g = by_cta ? group_of(s, min(s.rows, (i + 1) * a.per) - 1) : i;
    lo = group_begin(s, g) / a.per;
    hi = (group_end(s, g) - 1) / a.per;
    if (lo == hi || (by_cta && lo != i)) hi = lo - 1;  // finished by its CTA, or another job's
  } else if (job - 3 * jobs < 2) {
    hi = ctas - 1;
  }
  float v = 0.f;
  if (c < d) {
    const float* base = which < 3 ? a.part + which * d : a.wpart + (job - 3 * jobs) * d;
    const int64_t width = which < 3 ? 6 * (int64_t)d : 2 * (int64_t)d;
#pragma unroll 8
    for (int64_t k = lo + seg; k <= hi; k += segs)
      v += base[k * width + (which < 3 && k == lo ? 3 * d : 0) + c];
  }
  part[warp][lane] = v;
  __syncthreads();
  if (seg != 0 || c >= d || hi < lo) return;
  float t = 0.f;
  for (int i = 0; i < segs; ++i) t += part[warp + i][lane];
  if (which < 3) {
    put_sum(a, which, g, c, t);
  } else {
    float* out = job - 3 * jobs == 0 ? a.dpre_w : a.dpost_w;
    if (out != nullptr) out[c] = t;
  }
}

constexpr int kMaxCtas = 2048;  // of the backward pass (workspace)

int64_t num_groups(const acid_norm_site& s) {
  const int64_t rest = s.rows - s.first_rows;
  const int64_t group = s.group_rows > 0 ? s.group_rows : std::max<int64_t>(rest, 1);
  return (s.first_rows > 0) + (rest + group - 1) / group;
}

bool known_dtype(int t) { return t == ACID_BF16 || t == ACID_FP32; }
bool known_norm(int k) { return k == ACID_NORM_NONE || k == ACID_NORM_RMS || k == ACID_NORM_LAYER; }
size_t bytes_of(int dtype) { return dtype == ACID_BF16 ? 2 : 4; }

acid_status check_site(const acid_norm_site* s) {
  ACID_REQUIRE(s != nullptr, ACID_ERR_INVALID_ARG, "norm_site: null site");
  ACID_REQUIRE(known_dtype(s->stream_dtype) && known_dtype(s->branch_dtype), ACID_ERR_INVALID_ARG,
               "norm_site: unknown dtype");
  ACID_REQUIRE(known_norm(s->post_norm) && known_norm(s->pre_norm), ACID_ERR_INVALID_ARG, "norm_site: unknown norm");
  ACID_REQUIRE(s->rows >= 0 && s->d > 0 && s->rows <= (int64_t(1) << 39), ACID_ERR_INVALID_ARG, "norm_site: bad shape");
  ACID_REQUIRE(s->d % 8 == 0 && s->d <= kMaxWidth, ACID_ERR_UNSUPPORTED,
               "norm_site: d must be a multiple of 8, <= 4096");
  ACID_REQUIRE(s->first_rows >= 0 && s->first_rows <= s->rows && s->group_rows >= 0, ACID_ERR_INVALID_ARG,
               "norm_site: need 0 <= first_rows <= rows and group_rows >= 0");
  ACID_REQUIRE(s->eps >= 0.f, ACID_ERR_INVALID_ARG, "norm_site: eps must be >= 0");
  const bool mods = s->gate || s->scale || s->shift;
  if (mods && num_groups(*s) > 1)
    ACID_REQUIRE(s->ld_mod >= s->d && s->ld_mod % 4 == 0, ACID_ERR_INVALID_ARG,
                 "norm_site: ld_mod must be a multiple of 4, >= d");
  ACID_REQUIRE(aligned(s->gate, 16) && aligned(s->scale, 16) && aligned(s->shift, 16) && aligned(s->post_w, 16) &&
                   aligned(s->pre_w, 16),
               ACID_ERR_UNSUPPORTED, "norm_site: vectors must be 16-byte aligned");
  return ACID_OK;
}

// A [rows, d] operand, or none.
acid_status check_rows(const acid_norm_site& s, const void* p, int64_t ld, const char* name) {
  if (p == nullptr) return ACID_OK;
  ACID_REQUIRE(ld >= s.d, ACID_ERR_INVALID_ARG, std::string("norm_site: row stride of ") + name + " smaller than d");
  ACID_REQUIRE(aligned(p, 16) && ld % 8 == 0, ACID_ERR_UNSUPPORTED,
               std::string("norm_site: ") + name + " must be 16-byte aligned, its row stride a multiple of 8");
  return ACID_OK;
}

Site site_args(const acid_norm_site& s) {
  Site a;
  a.rows = s.rows;
  a.first = s.first_rows;
  a.group = s.group_rows > 0 ? s.group_rows : std::max<int64_t>(s.rows - s.first_rows, 1);
  a.d = s.d;
  a.post = s.post_norm;
  a.pre = s.pre_norm;
  a.tanh = s.gate_tanh != 0;
  a.eps = s.eps;
  a.res = s.res_scale;
  a.branch = s.branch_scale;
  a.gate = s.gate;
  a.scale = s.scale;
  a.shift = s.shift;
  a.post_w = s.post_w;
  a.pre_w = s.pre_w;
  a.groups = num_groups(s);
  a.ld_mod = s.ld_mod;
  return a;
}

int threads_for(int d) { return (d + 511) / 512 * 32; }

constexpr size_t kMaxSmem = 200 * 1024;
// CTAs that an SM keeps of a kernel with so much shared memory; sets the kernel
// up in the context.  (An occupancy query at each launch would take longer than
// the smallest kernels.)
template <typename K>
acid_status ctas_per_sm(PerContext& known, K kernel, int threads, size_t smem, int* ctas) {
  int regs = 0;
  ACID_TRY(known.get(&regs, [&](int* v) {
    ACID_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMaxSmem));
    cudaFuncAttributes f = {};
    ACID_CUDA(cudaFuncGetAttributes(&f, kernel));
    *v = f.numRegs > 0 ? (f.numRegs + 7) / 8 * 8 : 256;
    return ACID_OK;
  }));
  const size_t warps = 4 * (512 / (size_t)regs);  // each of the four schedulers holds 512 registers of 32 lanes
  *ctas = (int)std::max<size_t>(1, std::min<size_t>({warps * 32 / threads, 224 * 1024 / (smem + 1536), 24}));
  return ACID_OK;
}
size_t part_bytes(int d, int ctas) { return (size_t)ctas * 2 * 3 * d * sizeof(float); }

template <template <typename, typename> class F, typename A>
acid_status by_types(const acid_norm_site& s, const A& a) {
  using H = __nv_bfloat16;
  if (s.stream_dtype == ACID_BF16) return s.branch_dtype == ACID_BF16 ? F<H, H>::run(a) : F<H, float>::run(a);
  return s.branch_dtype == ACID_BF16 ? F<float, H>::run(a) : F<float, float>::run(a);
}

struct FwdLaunch {
  SiteFwd a;
  cudaStream_t s;
};
template <typename TS, typename TB>
struct RunFwd {
  static acid_status run(const FwdLaunch& l) { return l.a.y != nullptr ? go<true>(l) : go<false>(l); }
  template <bool BRANCH>
  static acid_status go(const FwdLaunch& l) {
    static PerContext known;
    const Site& s = l.a.s;
    const int threads = threads_for(s.d);
    const size_t smem = (size_t)kFwdStages * threads * 16 * (kPlanes<TS> + (BRANCH ? kPlanes<TB> : 0));
    int fit;
    ACID_TRY(ctas_per_sm(known, site_forward_kernel<TS, TB, BRANCH>, threads, smem, &fit));
    const int64_t most = (int64_t)num_sms() * fit;
    const int64_t ctas = std::min(s.rows, most), per = (s.rows + ctas - 1) / ctas;
    const bool strided = s.groups == 1;
    launch_pdl(site_forward_kernel<TS, TB, BRANCH>, (unsigned)(strided ? ctas : (s.rows + per - 1) / per), threads,
               smem, l.s, l.a, strided ? int64_t(1) : per, strided ? ctas : int64_t(1), (uint32_t)per);
    ACID_CHECK_LAUNCH();
    return ACID_OK;
  }
};
struct BwdLaunch {
  SiteBwd a;
  cudaStream_t s;
};
template <typename TS, typename TB>
struct RunBwd {
  static acid_status run(const BwdLaunch& l) {
    static PerContext known;
    SiteBwd a = l.a;
    const Site& s = a.s;
    const int threads = threads_for(s.d);
    const size_t smem = (size_t)threads * (kBwdStages<TS, TB> * 16 * 2 * (kPlanes<TS> + kPlanes<TB>) + 128);
    int fit;
    ACID_TRY(ctas_per_sm(known, site_backward_kernel<TS, TB>, threads, smem, &fit));
    const int64_t most = std::min<int64_t>(kMaxCtas, (int64_t)num_sms() * fit);
    a.per = std::max<int64_t>(1, (s.rows + most - 1) / most);
    const int ctas = (int)((s.rows + a.per - 1) / a.per);
    a.wpart = a.part + part_bytes(s.d, ctas) / sizeof(float);
    launch_pdl(site_backward_kernel<TS, TB>, ctas, threads, smem, l.s, a);
    ACID_CHECK_LAUNCH();
    const bool weights = a.dpre_w != nullptr || a.dpost_w != nullptr;
    const bool vectors = a.dgate != nullptr || a.dscale != nullptr || a.dshift != nullptr;
    // does any group reach over an edge?
    const int64_t head = s.first > 0 ? s.first : 0, longest = std::max(head, std::min(s.group, s.rows - head));
    if (!weights && (!vectors || (longest == 1))) return ACID_OK;
    const bool by_cta = s.groups > ctas;
    const int jobs = by_cta ? ctas : (int)s.groups;
    const int64_t span = std::max<int64_t>(longest / a.per + 2, weights ? ctas : 0);
    int segs = 1;
    while (segs < kJoinWarps && segs * 8 < span) segs *= 2;
    const int per_cta = kJoinWarps / segs;
    launch_pdl(site_join_kernel, dim3((s.d + 31) / 32, (3 * jobs + 2 + per_cta - 1) / per_cta), 32 * kJoinWarps, 0, l.s, a,
               ctas, jobs, segs, by_cta);
    ACID_CHECK_LAUNCH();
    return ACID_OK;
  }
};

size_t workspace_bytes(const acid_norm_site& s) {
  const int ctas = (int)std::min<int64_t>(kMaxCtas, std::max<int64_t>(s.rows, 1));
  return part_bytes(s.d, ctas) + (size_t)ctas * 2 * s.d * sizeof(float);
}

}  // namespace
}  // namespace acid

using namespace acid;

extern "C" acid_status acid_norm_site_groups(const acid_norm_site* site, int64_t* groups) {
  clear_error();
  ACID_TRY(check_site(site));
  ACID_REQUIRE(groups != nullptr, ACID_ERR_INVALID_ARG, "acid_norm_site_groups: groups is null");
  *groups = num_groups(*site);
  return ACID_OK;
}

extern "C" acid_status acid_norm_site_forward(const acid_norm_site* site, const void* x, int64_t ldx, const void* y,
                                              int64_t ldy, void* r, int64_t ldr, void* u, int64_t ldu,
                                              acid_stream_t stream) {
  clear_error();
  ACID_TRY(check_site(site));
  if (site->rows == 0) return ACID_OK;
  ACID_REQUIRE(x != nullptr && (r != nullptr || u != nullptr), ACID_ERR_INVALID_ARG,
               "acid_norm_site_forward: need x, and r or u");
  ACID_TRY(check_rows(*site, x, ldx, "x"));
  ACID_TRY(check_rows(*site, y, ldy, "y"));
  ACID_TRY(check_rows(*site, r, ldr, "r"));
  ACID_TRY(check_rows(*site, u, ldu, "u"));
  const FwdLaunch l{{site_args(*site), x, y, r, u, ldx, ldy, ldr, ldu}, (cudaStream_t)stream};
  return by_types<RunFwd>(*site, l);
}

extern "C" acid_status acid_norm_site_workspace_size(const acid_norm_site* site, size_t* bytes) {
  clear_error();
  ACID_TRY(check_site(site));
  ACID_REQUIRE(bytes != nullptr, ACID_ERR_INVALID_ARG, "acid_norm_site_workspace_size: bytes is null");
  *bytes = workspace_bytes(*site);
  return ACID_OK;
}

extern "C" acid_status acid_norm_site_backward(const acid_norm_site* site, const void* du, int64_t lddu, const void* r,
                                               int64_t ldr, const void* y, int64_t ldy, const void* dr, int64_t lddr,
                                               const acid_norm_site_grads* grads, void* ws, size_t ws_bytes,
                                               acid_stream_t stream) {
  clear_error();
  ACID_TRY(check_site(site));
  ACID_REQUIRE(grads != nullptr, ACID_ERR_INVALID_ARG, "acid_norm_site_backward: null gradients");
  const acid_norm_site_grads& o = *grads;
  const int64_t groups = num_groups(*site);
  cudaStream_t s = (cudaStream_t)stream;
  if (groups > 1 && (o.dgate || o.dscale || o.dshift))
    ACID_REQUIRE(o.ld_dmod >= site->d && o.ld_dmod % 4 == 0, ACID_ERR_INVALID_ARG,
                 "acid_norm_site_backward: ld_dmod must be a multiple of 4, >= d");
  ACID_REQUIRE(aligned(o.dgate, 16) && aligned(o.dscale, 16) && aligned(o.dshift, 16) && aligned(o.dpost_w, 16) &&
                   aligned(o.dpre_w, 16),
               ACID_ERR_UNSUPPORTED, "acid_norm_site_backward: vectors must be 16-byte aligned");
  if (site->rows == 0) {  // no groups; the weights' sums are empty
    if (o.dpost_w) ACID_CUDA(cudaMemsetAsync(o.dpost_w, 0, site->d * sizeof(float), s));
    if (o.dpre_w) ACID_CUDA(cudaMemsetAsync(o.dpre_w, 0, site->d * sizeof(float), s));
    return ACID_OK;
  }
  ACID_REQUIRE(du != nullptr || dr != nullptr, ACID_ERR_INVALID_ARG, "acid_norm_site_backward: need du or dr");
  ACID_REQUIRE(du != nullptr || !(o.dscale || o.dshift || o.dpre_w), ACID_ERR_INVALID_ARG,
               "acid_norm_site_backward: dscale, dshift and dpre_w need du");
  ACID_REQUIRE(du == nullptr || r != nullptr, ACID_ERR_INVALID_ARG, "acid_norm_site_backward: du needs r");
  ACID_REQUIRE(y != nullptr || !(o.dy || o.dgate || o.dpost_w), ACID_ERR_INVALID_ARG,
               "acid_norm_site_backward: dy, dgate and dpost_w need y");
  ACID_TRY(check_rows(*site, du, lddu, "du"));
  ACID_TRY(check_rows(*site, r, ldr, "r"));
  ACID_TRY(check_rows(*site, y, ldy, "y"));
  ACID_TRY(check_rows(*site, dr, lddr, "dr"));
  ACID_TRY(check_rows(*site, o.dx, o.lddx, "dx"));
  ACID_TRY(check_rows(*site, o.dy, o.lddy, "dy"));
  ACID_REQUIRE(ws != nullptr && aligned(ws, 16), ACID_ERR_WORKSPACE,
               "acid_norm_site_backward: workspace null or not 16-byte aligned");
  const size_t need = workspace_bytes(*site);
  ACID_REQUIRE(ws_bytes >= need, ACID_ERR_WORKSPACE,
               "acid_norm_site_backward: workspace too small (need " + std::to_string(need) + ")");
  const BwdLaunch l{{site_args(*site), du, r, y, dr, lddu, ldr, ldy, lddr, o.dx, o.dy, o.lddx, o.lddy, o.dgate, o.dscale,
                     o.dshift, o.dpost_w, o.dpre_w, o.ld_dmod, static_cast<float*>(ws), nullptr, 1},
                    s};
  return by_types<RunBwd>(*site, l);
}
