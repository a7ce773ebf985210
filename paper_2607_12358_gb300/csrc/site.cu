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
constexpr int kMaxWidth = 4096;  // 8 warps of 16 columns a lane
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

// A thread's columns: 8 V of them in runs of E, E (tid + j blockDim) ..., as fp32
// pairs, so that one instruction does the arithmetic of two columns.  E is such
// that a warp's loads and stores of a run are contiguous: 8 where both types are
// bf16, else 4 (with fp32 in runs of 8 each access takes half of its 32-byte sectors:
// 32760 x 1536 fp32 stream 114 us, its gradient 226).  Runs past the row's end hold
// zeros all through.
//   V is 2; 1 for rows of at most 256 columns, which are one warp's then (26 Mi elements
// of 256 columns, bf16: 68 us, 82 with half of the warp's lanes; their gradient 132,
// 178).
template <int V>
struct Cols {
  uint64_t v[4 * V];
};
template <int V>
constexpr int kMostThreads = V == 1 ? 32 : kMaxWidth / 16;
#define FOR_PAIRS _Pragma("unroll") for (int i = 0; i < 4 * V; ++i)
__device__ __forceinline__ uint64_t f2_same(float x) { return f2_pack(x, x); }
__device__ __forceinline__ float f2_total(uint64_t x) {
  float a, b;
  f2_unpack(x, a, b);
  return a + b;
}
// Sum of the pairs.
template <int V>
__device__ __forceinline__ float total(const Cols<V>& a) {
  uint64_t s[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) s[i] = V == 2 ? f2_add(a.v[i], a.v[4 * V - 4 + i]) : a.v[i];
  return f2_total(f2_add(f2_add(s[0], s[1]), f2_add(s[2], s[3])));
}
// Sum of the products.
template <int V>
__device__ __forceinline__ float dot(const Cols<V>& a, const Cols<V>& b) {
  uint64_t s = f2_mul(a.v[0], b.v[0]), t = f2_mul(a.v[1], b.v[1]);
#pragma unroll
  for (int i = 2; i < 4 * V; i += 2) {
    s = f2_fma(a.v[i], b.v[i], s);
    t = f2_fma(a.v[i + 1], b.v[i + 1], t);
  }
  return f2_total(f2_add(s, t));
}

template <int V, int E>
struct Place {
  static constexpr int kRuns = 8 * V / E;
  int c[kRuns], d;  // first column of each run
  bool on[kRuns];
};
template <int V, int E>
__device__ __forceinline__ Place<V, E> place(int d) {
  Place<V, E> at;
  at.d = d;
#pragma unroll
  for (int j = 0; j < at.kRuns; ++j) {
    at.c[j] = (threadIdx.x + j * blockDim.x) * E;
    at.on[j] = at.c[j] < d;
  }
  return at;
}
// Columns of a vector; `none` in all of the row's where there is none.
template <int V, int E>
__device__ __forceinline__ Cols<V> vec(const float* p, const Place<V, E>& at, float none) {
  Cols<V> a;
#pragma unroll
  for (int j = 0; j < at.kRuns; ++j) {
    uint64_t* v = a.v + j * (E / 2);
    const float fill = at.on[j] ? none : 0.f;
#pragma unroll
    for (int i = 0; i < E / 2; ++i) v[i] = f2_same(fill);
    if (!at.on[j] || p == nullptr || !ACID_IN_BOUNDS(kSiteNormSite, at.c[j] + E - 1, at.d)) continue;
#pragma unroll
    for (int i = 0; i < E / 4; ++i) {
      const float4 x = *reinterpret_cast<const float4*>(p + at.c[j] + 4 * i);
      v[2 * i] = f2_pack(x.x, x.y);
      v[2 * i + 1] = f2_pack(x.z, x.w);
    }
  }
  return a;
}
template <int V>
__device__ __forceinline__ void times(Cols<V>& a, const Cols<V>& b) { FOR_PAIRS a.v[i] = f2_mul(a.v[i], b.v[i]); }
template <int V, int E>
__device__ __forceinline__ void plus(Cols<V>& a, float x, const Place<V, E>& at) {
  FOR_PAIRS a.v[i] = f2_add(a.v[i], f2_same(at.on[i / (E / 2)] ? x : 0.f));
}
// branch_scale times the gate's columns of a group.
template <int V, int E>
__device__ __forceinline__ Cols<V> gate_cols(const Site& s, int64_t m, const Place<V, E>& at) {
  Cols<V> g = vec(s.gate ? s.gate + m : nullptr, at, 1.f);
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
template <int V, int E>
__device__ __forceinline__ Cols<V> scale_cols(const Site& s, int64_t m, const Place<V, E>& at) {
  Cols<V> a = vec(s.scale ? s.scale + m : nullptr, at, 0.f);
  plus(a, 1.f, at);
  return a;
}

// To a row of the operand, whose first element is `row`.
template <typename T, int V, int E>
__device__ __forceinline__ void put(T* row, const Place<V, E>& at, const Cols<V>& a, int64_t r, int64_t rows) {
#pragma unroll
  for (int j = 0; j < at.kRuns; ++j) {
    float f[E];
#pragma unroll
    for (int i = 0; i < E / 2; ++i) f2_unpack(a.v[j * (E / 2) + i], f[2 * i], f[2 * i + 1]);
    if (!at.on[j] || !ACID_IN_BOUNDS(kSiteNormSite, r, rows)) continue;
    T* p = row + at.c[j];
    if constexpr (E == 8) {
      store8(p, f);
    } else if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    } else {
      *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]));
    }
  }
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
// copies is all the synchronisation there is.  A stage is a plane for each run of
// each operand: a warp's copies go to consecutive addresses (with a thread's pieces
// side by side they took longer: 32760 x 1536 128 us, not 112).  Pieces of runs past the
// row's end are zeros from the start.
template <typename T, int V>
constexpr int kBytes = 8 * V * sizeof(T);  // of a thread's columns
template <typename T, int V, int E>
__device__ __forceinline__ void stage(uint8_t* plane, const T* row, const Place<V, E>& at, int64_t r, int64_t rows) {
  constexpr int kRun = E * sizeof(T);
#pragma unroll
  for (int j = 0; j < at.kRuns; ++j)
    if (at.on[j] && ACID_IN_BOUNDS(kSiteNormSite, r, rows)) {
      const uint32_t to = smem_u32(plane + (threadIdx.x + j * blockDim.x) * kRun);
      if constexpr (kRun == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(row + at.c[j]) : "memory");
      else
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(row + at.c[j]) : "memory");
    }
}
template <typename T, int V, int E>
__device__ __forceinline__ Cols<V> unstage(const uint8_t* plane) {
  constexpr int kRun = E * sizeof(T), kRuns = 8 * V / E;
  Cols<V> a;
#pragma unroll
  for (int j = 0; j < kRuns; ++j) {
    const uint8_t* q = plane + (threadIdx.x + j * blockDim.x) * kRun;
    uint64_t* v = a.v + j * (E / 2);
    if constexpr (sizeof(T) == 4) {
      const ulonglong2 x = *reinterpret_cast<const ulonglong2*>(q);
      v[0] = x.x;
      v[1] = x.y;
    } else if constexpr (E == 8) {
      const uint4 u = *reinterpret_cast<const uint4*>(q);
      v[0] = f2_pack(bf16_lo(u.x), bf16_hi(u.x));
      v[1] = f2_pack(bf16_lo(u.y), bf16_hi(u.y));
      v[2] = f2_pack(bf16_lo(u.z), bf16_hi(u.z));
      v[3] = f2_pack(bf16_lo(u.w), bf16_hi(u.w));
    } else {
      const uint2 u = *reinterpret_cast<const uint2*>(q);
      v[0] = f2_pack(bf16_lo(u.x), bf16_hi(u.x));
      v[1] = f2_pack(bf16_lo(u.y), bf16_hi(u.y));
    }
  }
  return a;
}
// Zeros in the thread's pieces of an operand.
template <typename T, int V, int E>
__device__ __forceinline__ void clear_plane(uint8_t* plane) {
  constexpr int kRun = E * sizeof(T);
#pragma unroll
  for (int j = 0; j < 8 * V / E; ++j) {
    uint8_t* q = plane + (threadIdx.x + j * blockDim.x) * kRun;
    *reinterpret_cast<uint2*>(q) = make_uint2(0, 0);
    if constexpr (kRun == 16) *reinterpret_cast<uint2*>(q + 8) = make_uint2(0, 0);
  }
}
template <typename TS, typename TB>
constexpr int kRunOf = sizeof(TS) + sizeof(TB) == 4 ? 8 : 4;

// r = res x + branch gate (N_post(y) post_w), u = N_pre(r) pre_w (1 + scale) + shift.
// A CTA takes a row at a time; row k of CTA b is b start + k step, k < count: rows that
// lie apart where there is one group (the CTAs then work on one stretch of memory),
// adjoining ones where a CTA would change its group's vectors at each row otherwise.
// Each operand passes once, so the bytes bound it; a few rows in flight a CTA and two or
// more CTAs an SM keep the memory busy through the two or three sums of a row.  fp32
// stream, bf16 branch, RMS and layer norm: 32760 x 1536 105 us (85% of a copy's rate),
// 67576 x 3072, both bf16, a group of 2040 rows a frame, 252 us (97%); one row 3.5 us, which is a
// launch and three sums' latency.
constexpr int kFwdStages = 4;
template <typename TS, typename TB, bool BRANCH, int V>
__global__ void __launch_bounds__(kMostThreads<V>, V == 1 ? 16 : 2) site_forward_kernel(SiteFwd a, int64_t start, int64_t step, uint32_t count) {
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ float4 red[2][kMaxWarps];
  constexpr int E = kRunOf<TS, TB>, kX = kBytes<TS, V>, kStage = kX + (BRANCH ? kBytes<TB, V> : 0);
  const Site& s = a.s;
  const Place<V, E> at = place<V, E>(s.d);
  uint8_t* mine = ring;
  const int unit = blockDim.x, stage_bytes = kStage * unit;
  if (!at.on[at.kRuns - 1])
    for (int k = 0; k < kFwdStages; ++k) {
      clear_plane<TS, V, E>(ring + k * stage_bytes);
      if constexpr (BRANCH) clear_plane<TB, V, E>(ring + k * stage_bytes + kX * unit);
    }
  Reducer sums = reducer(red);
  pdl_wait();
  const float d = (float)s.d, per_d = 1.f / d;
  int64_t row = blockIdx.x * start;
  const uint32_t n = row < s.rows ? (uint32_t)min((int64_t)count, (s.rows - 1 - row) / step + 1) : 0;
  int64_t ahead = row;  // the next row to be copied
  const TS* xp = static_cast<const TS*>(a.x) + row * a.ldx;
  const TB* yp = static_cast<const TB*>(a.y) + (BRANCH ? row * a.ldy : 0);
  uint32_t copied = 0;
  uint8_t* to = mine;
  auto issue = [&] {
    if (copied < n) {
      stage<TS, V, E>(to, xp, at, ahead, s.rows);
      xp += step * a.ldx;
      if constexpr (BRANCH) {
        stage<TB, V, E>(to + kX * unit, yp, at, ahead, s.rows);
        yp += step * a.ldy;
      }
      ahead += step;
      ++copied;
    }
    to = to == mine + (kFwdStages - 1) * stage_bytes ? mine : to + stage_bytes;
    cp_async_commit();
  };
  for (int k = 0; k < kFwdStages - 1; ++k) issue();
  const bool wants_mean = s.pre == ACID_NORM_LAYER && a.u != nullptr;
  const uint8_t* from = mine;
  TS* rp = static_cast<TS*>(a.r) + (a.r != nullptr ? row * a.ldr : 0);
  TB* up = static_cast<TB*>(a.u) + (a.u != nullptr ? row * a.ldu : 0);
  for (uint32_t k = 0; k < n;) {
    // the rows of one group
    const int64_t g = group_of(s, row), m = g * s.ld_mod;
    const uint32_t stop = (uint32_t)min((int64_t)n, k + (group_end(s, g) - 1 - row) / step + 1);
    Cols<V> gw, sc = scale_cols(s, m, at);  // gate and post_w, (1 + scale) and pre_w, shift
    const Cols<V> sh = vec(s.shift ? s.shift + m : nullptr, at, 0.f);
    times(sc, vec(s.pre_w, at, 1.f));
    if constexpr (BRANCH) {
      gw = gate_cols(s, m, at);
      times(gw, vec(s.post_w, at, 1.f));
    }
    for (; k < stop; ++k, row += step) {
      cp_async_wait<kFwdStages - 2>();
      Cols<V> r = unstage<TS, V, E>(from);
      float mean = 0.f;
      if constexpr (BRANCH) {
        Cols<V> y = unstage<TB, V, E>(from + kX * unit);
        issue();
        FOR_PAIRS r.v[i] = f2_mul(r.v[i], f2_same(s.res));
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
        FOR_PAIRS r.v[i] = f2_mul(r.v[i], f2_same(s.res));
        if (wants_mean) mean = sums.sum<1>(total(r)).x / d;
      }
      from = from == mine + (kFwdStages - 1) * stage_bytes ? mine : from + stage_bytes;
      if (a.r != nullptr) {
        put(rp, at, r, row, s.rows);
        rp += step * a.ldr;
      }
      if (a.u == nullptr) continue;
      if (s.pre != ACID_NORM_NONE) {
        if (s.pre == ACID_NORM_LAYER) plus(r, -mean, at);
        const float inv = rsqrtf(fmaf(sums.sum<1>(dot(r, r)).x, per_d, s.eps));
        FOR_PAIRS r.v[i] = f2_mul(r.v[i], f2_same(inv));
      }
      FOR_PAIRS r.v[i] = f2_fma(r.v[i], sc.v[i], sh.v[i]);
      put(up, at, r, row, s.rows);
      up += step * a.ldu;
    }
  }
}

// The slope 1 - tanh^2 of a gate, 4 e / (1 + e)^2 with e = exp(-2 |x|): 1 - tanh^2 itself has
// nothing left of it where the gate is past 9.
__device__ __forceinline__ float tanh_slope(float x) {
  const float e = expf(-2.f * fabsf(x)), f = 1.f + e;
  return __fdividef(4.f * e, f * f);
}

// Gradients of the site's vectors for one group from the raw sums
// sum du, sum du n and sum dr p over its rows (which = 0, 1, 2): one column.
__device__ __forceinline__ void put_sum(const SiteBwd& a, int which, int64_t g, int c, float v) {
  const Site& s = a.s;
  float* out = which == 0 ? a.dshift : which == 1 ? a.dscale : a.dgate;
  if (out == nullptr || !ACID_IN_BOUNDS(kSiteNormSite, c, s.d)) return;
  if (which == 1 && s.pre_w != nullptr) v *= s.pre_w[c];
  if (which == 2) {
    v *= s.branch * (s.tanh && s.gate ? tanh_slope(s.gate[g * s.ld_mod + c]) : 1.f) * (s.post_w != nullptr ? s.post_w[c] : 1.f);
  }
  out[g * a.ld_dmod + c] = v;
}
// The same for a thread's columns.
template <int V, int E>
__device__ __forceinline__ void put_sums(const SiteBwd& a, int which, int64_t g, int64_t m, const Place<V, E>& at, Cols<V> v) {
  const Site& s = a.s;
  float* out = which == 0 ? a.dshift : which == 1 ? a.dscale : a.dgate;
  if (out == nullptr) return;
  if (which == 1) times(v, vec(s.pre_w, at, 1.f));
  if (which == 2) {
    times(v, vec(s.post_w, at, 1.f));
    FOR_PAIRS v.v[i] = f2_mul(v.v[i], f2_same(s.branch));
    if (s.tanh && s.gate) {
      const Cols<V> t = vec(s.gate + m, at, 0.f);
      FOR_PAIRS {
        float lo, hi;
        f2_unpack(t.v[i], lo, hi);
        v.v[i] = f2_mul(v.v[i], f2_pack(tanh_slope(lo), tanh_slope(hi)));
      }
    }
  }
  put(out + g * a.ld_dmod, at, v, g, s.groups);
}

// The gradients.  CTA b takes the rows [b per, (b + 1) per) and keeps the sums
// over the rows of its group in registers.  A group that lies in the CTA's rows
// is finished here; of one that reaches over their edge the sums go to the
// CTA's slot 2 b (the group began earlier) or 2 b + 1 (it begins here), and
// site_join_kernel adds the slots.  A row's four sums go together, so that it waits for
// the CTA two or three times.  The bytes bound it from some thousand rows on: 32760 x 1536,
// fp32 stream, bf16 branch, a group of 1560 rows 145 us (92% of a copy's rate), with the
// second kernel 155; 226 x 1920 5 and 12.6 us, of which the launches' and the sums'
// latency is nearly all.
constexpr int kBwdStages = 3;
template <typename TS, typename TB, int V>
__global__ void __launch_bounds__(kMostThreads<V>, V == 1 ? 12 : 1) site_backward_kernel(SiteBwd a) {
  extern __shared__ __align__(16) uint8_t ring[];
  __shared__ float4 red[2][kMaxWarps];
  constexpr int E = kRunOf<TS, TB>, kS = kBytes<TS, V>, kB = kBytes<TB, V>, kR = 0, kDr = kS, kY = 2 * kS, kDu = kY + kB;
  constexpr int kStage = kDu + kB;
  const Site& s = a.s;
  const Place<V, E> at = place<V, E>(s.d);
  uint8_t* mine = ring;
  const int unit = blockDim.x, stage_bytes = kStage * unit;
  ulonglong2* wsum = reinterpret_cast<ulonglong2*>(ring + kBwdStages * stage_bytes) + threadIdx.x;  // [4 V]
  const bool weights = a.dpre_w != nullptr || a.dpost_w != nullptr;
  // absent operands and columns past the row are zeros
  if (!at.on[at.kRuns - 1] || a.du == nullptr || a.dr == nullptr || a.y == nullptr)
    for (int k = 0; k < kBwdStages; ++k) {
      uint8_t* p = ring + k * stage_bytes;
      clear_plane<TS, V, E>(p + kR * unit);
      clear_plane<TS, V, E>(p + kDr * unit);
      clear_plane<TB, V, E>(p + kY * unit);
      clear_plane<TB, V, E>(p + kDu * unit);
    }
  for (int i = 0; weights && i < 4 * V; ++i) wsum[i * blockDim.x] = make_ulonglong2(0, 0);
  Reducer sums = reducer(red);
  pdl_wait();
  const float d = (float)s.d, per_d = 1.f / d;
  const int64_t begin = blockIdx.x * a.per, end = min(s.rows, begin + a.per);
  int64_t ahead = begin;
  const TS *rp = static_cast<const TS*>(a.r) + (a.du ? begin * a.ldr : 0), *drp = static_cast<const TS*>(a.dr) + (a.dr ? begin * a.lddr : 0);
  const TB *dup = static_cast<const TB*>(a.du) + (a.du ? begin * a.lddu : 0), *yp = static_cast<const TB*>(a.y) + (a.y ? begin * a.ldy : 0);
  TS* dxp = static_cast<TS*>(a.dx) + (a.dx ? begin * a.lddx : 0);
  TB* dyp = static_cast<TB*>(a.dy) + (a.dy ? begin * a.lddy : 0);
  uint8_t* to = mine;
  auto issue = [&] {
    if (ahead < end) {
      if (a.du != nullptr) {
        stage<TS, V, E>(to + kR * unit, rp, at, ahead, s.rows);
        stage<TB, V, E>(to + kDu * unit, dup, at, ahead, s.rows);
        rp += a.ldr;
        dup += a.lddu;
      }
      if (a.dr != nullptr) {
        stage<TS, V, E>(to + kDr * unit, drp, at, ahead, s.rows);
        drp += a.lddr;
      }
      if (a.y != nullptr) {
        stage<TB, V, E>(to + kY * unit, yp, at, ahead, s.rows);
        yp += a.ldy;
      }
      ++ahead;
    }
    to = to == mine + (kBwdStages - 1) * stage_bytes ? mine : to + stage_bytes;
    cp_async_commit();
  };
  for (int k = 0; k < kBwdStages - 1; ++k) issue();
  const uint8_t* from = mine;
  for (int64_t row = begin; row < end;) {
    const int64_t g = group_of(s, row), m = g * s.ld_mod, first = row, last = min(end, group_end(s, g));
    Cols<V> A = {}, S = {}, T = {}, sc = scale_cols(s, m, at), gw = gate_cols(s, m, at);
    times(sc, vec(s.pre_w, at, 1.f));
    times(gw, vec(s.post_w, at, 1.f));
    for (; row < last; ++row) {
      cp_async_wait<kBwdStages - 2>();
      Cols<V> n = unstage<TS, V, E>(from + kR * unit), du = unstage<TB, V, E>(from + kDu * unit);
      Cols<V> y = unstage<TB, V, E>(from + kY * unit), dr = unstage<TS, V, E>(from + kDr * unit);
      issue();
      from = from == mine + (kBwdStages - 1) * stage_bytes ? mine : from + stage_bytes;
      if (s.pre == ACID_NORM_LAYER || s.post == ACID_NORM_LAYER) {
        const float4 t = sums.sum<2>(total(n), total(y));
        if (s.pre == ACID_NORM_LAYER) plus(n, -(t.x / d), at);
        if (s.post == ACID_NORM_LAYER) plus(y, -(t.y / d), at);
      }
      FOR_PAIRS A.v[i] = f2_add(A.v[i], du.v[i]);
      Cols<V> dn = du;
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
      // dr += in (dn - mean - along n); S takes du in n
      FOR_PAIRS {
        S.v[i] = f2_fma(f2_mul(du.v[i], f2_same(in)), n.v[i], S.v[i]);
        dn.v[i] = f2_fma(n.v[i], f2_same(-along), dn.v[i]);
      }
      if (s.pre == ACID_NORM_LAYER) plus(dn, -mean, at);
      FOR_PAIRS {
        dr.v[i] = f2_fma(f2_same(in), dn.v[i], dr.v[i]);
        y.v[i] = f2_mul(y.v[i], f2_same(ip));
        T.v[i] = f2_fma(dr.v[i], y.v[i], T.v[i]);
      }
      if (a.dx != nullptr) {
        Cols<V> o;
        FOR_PAIRS o.v[i] = f2_mul(dr.v[i], f2_same(s.res));
        put(dxp, at, o, row, s.rows);
        dxp += a.lddx;
      }
      if (a.dy == nullptr) continue;
      times(dr, gw);
      if (s.post != ACID_NORM_NONE) {
        const float4 t = sums.sum<2>(total(dr), dot(dr, y));
        FOR_PAIRS dr.v[i] = f2_fma(y.v[i], f2_same(-t.y * per_d), dr.v[i]);
        if (s.post == ACID_NORM_LAYER) plus(dr, -t.x * per_d, at);
        FOR_PAIRS dr.v[i] = f2_mul(dr.v[i], f2_same(ip));
      }
      put(dyp, at, dr, row, s.rows);
      dyp += a.lddy;
    }
    if (weights) {  // dpre_w gathers (1 + scale) S, dpost_w branch_scale gate T
      const Cols<V> f = scale_cols(s, m, at), h = gate_cols(s, m, at);
#pragma unroll
      for (int i = 0; i < 2 * V; ++i) {
        ulonglong2& p = wsum[i * blockDim.x];
        ulonglong2& q = wsum[(2 * V + i) * blockDim.x];
        p = make_ulonglong2(f2_fma(f.v[2 * i], S.v[2 * i], p.x), f2_fma(f.v[2 * i + 1], S.v[2 * i + 1], p.y));
        q = make_ulonglong2(f2_fma(h.v[2 * i], T.v[2 * i], q.x), f2_fma(h.v[2 * i + 1], T.v[2 * i + 1], q.y));
      }
    }
    const bool starts = group_begin(s, g) == first, ends = group_end(s, g) == last;
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
    Cols<V> v;
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) {
      const ulonglong2 p = wsum[(2 * V * w + i) * blockDim.x];
      v.v[2 * i] = p.x;
      v.v[2 * i + 1] = p.y;
    }
    put(wp + w * s.d, at, v, blockIdx.x, gridDim.x);
  }
}

// Adds the CTAs' slots in the CTAs' order.  A job is one vector of one group that
// reaches over an edge (counted by groups, or by CTAs where these are fewer: the
// group that begins in the CTA and leaves it), or one of the two weights' gradients.
// `segs` warps share a job's slots, a lane takes a column.  The groups' jobs come first,
// in `ctas_v` CTAs down the grid, and share by the CTAs that a group reaches over; the
// weights' by all CTAs.  (As many warps for each group's as for the weights': 700 rows of
// 1536, each its own group, 170 us in all, now 19.)
constexpr int kJoinWarps = 16;
struct Join {
  int jobs, segs;  // of each vector
  int ctas_v, segs_w;
  int ctas;        // of site_backward_kernel
  bool by_cta;
};
__global__ void __launch_bounds__(32 * kJoinWarps) site_join_kernel(SiteBwd a, Join n) {
  __shared__ float part[kJoinWarps][32];
  pdl_wait();
  const Site& s = a.s;
  const bool rows = blockIdx.y < n.ctas_v;
  const int segs = rows ? n.segs : n.segs_w, y = rows ? blockIdx.y : blockIdx.y - n.ctas_v;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, seg = warp % segs;
  const int c = blockIdx.x * 32 + lane, d = s.d, job = y * (kJoinWarps / segs) + warp / segs;
  const int which = rows ? job / n.jobs : 3 + job;  // 0 .. 2: dshift, dscale, dgate; 3, 4: dpre_w, dpost_w
  int64_t g = 0, lo = 0, hi = -1;  // slots lo .. hi
  if (which < 3) {
    const int64_t i = job - which * n.jobs;
    g = n.by_cta ? group_of(s, min(s.rows, (i + 1) * a.per) - 1) : i;
    lo = group_begin(s, g) / a.per;
    hi = (group_end(s, g) - 1) / a.per;
    if (lo == hi || (n.by_cta && lo != i)) hi = lo - 1;  // finished by its CTA, or another job's
  } else if (!rows && which < 5) {
    hi = n.ctas - 1;
  }
  float v = 0.f;
  if (c < d) {
    const float* base = which < 3 ? a.part + which * d : a.wpart + (which - 3) * d;
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
    float* out = which == 3 ? a.dpre_w : a.dpost_w;
    if (out != nullptr) out[c] = t;
  }
}

// Rows of a group after the first rows: no more than there are, so that sums with it stay in range.
int64_t group_length(const acid_norm_site& s) {
  const int64_t rest = std::max<int64_t>(s.rows - s.first_rows, 1);
  return s.group_rows > 0 ? std::min(s.group_rows, rest) : rest;
}
int64_t num_groups(const acid_norm_site& s) {
  const int64_t rest = s.rows - s.first_rows, group = group_length(s);
  return (s.first_rows > 0) + (rest + group - 1) / group;
}

bool known_dtype(int t) { return t == ACID_BF16 || t == ACID_FP32; }
bool known_norm(int k) { return k == ACID_NORM_NONE || k == ACID_NORM_RMS || k == ACID_NORM_LAYER; }

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
  a.group = group_length(s);
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

int threads_for(int d, int v) { return (d + 256 * v - 1) / (256 * v) * 32; }
// Columns of a thread in eights (Cols).
int eights_for(int d) { return d <= 256 ? 1 : 2; }
// CTAs of the backward pass that a workspace has slots for: 13 warps an SM (registers leave room for 8 to 12).
int max_ctas(int d) { return 2048 / (threads_for(d, eights_for(d)) / 32); }

constexpr size_t kMaxSmem = 224 * 1024;
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
  static acid_status run(const FwdLaunch& l) {
    if (eights_for(l.a.s.d) == 1) return l.a.y != nullptr ? go<true, 1>(l) : go<false, 1>(l);
    return l.a.y != nullptr ? go<true, 2>(l) : go<false, 2>(l);
  }
  template <bool BRANCH, int V>
  static acid_status go(const FwdLaunch& l) {
    static PerContext known;
    const Site& s = l.a.s;
    const int threads = threads_for(s.d, V);
    const size_t smem = (size_t)threads * kFwdStages * (kBytes<TS, V> + (BRANCH ? kBytes<TB, V> : 0));
    const auto kernel = site_forward_kernel<TS, TB, BRANCH, V>;
    int fit;
    ACID_TRY(ctas_per_sm(known, kernel, threads, smem, &fit));
    const int64_t most = (int64_t)num_sms() * fit;
    const int64_t ctas = std::min(s.rows, most), per = (s.rows + ctas - 1) / ctas;
    const bool strided = s.groups == 1;
    launch_pdl(kernel, (unsigned)(strided ? ctas : (s.rows + per - 1) / per), threads, smem, l.s, l.a,
               strided ? int64_t(1) : per, strided ? ctas : int64_t(1), (uint32_t)per);
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
  static acid_status run(const BwdLaunch& l) { return eights_for(l.a.s.d) == 1 ? go<1>(l) : go<2>(l); }
  template <int V>
  static acid_status go(const BwdLaunch& l) {
    static PerContext known;
    SiteBwd a = l.a;
    const Site& s = a.s;
    const int threads = threads_for(s.d, V);
    const size_t smem = (size_t)threads * (kBwdStages * 2 * (kBytes<TS, V> + kBytes<TB, V>) + 64 * V);
    int fit;
    ACID_TRY(ctas_per_sm(known, site_backward_kernel<TS, TB, V>, threads, smem, &fit));
    const int64_t most = std::min<int64_t>(max_ctas(s.d), (int64_t)num_sms() * fit);
    a.per = std::max<int64_t>(1, (s.rows + most - 1) / most);
    const int ctas = (int)((s.rows + a.per - 1) / a.per);
    a.wpart = a.part + part_bytes(s.d, ctas) / sizeof(float);
    launch_pdl(site_backward_kernel<TS, TB, V>, ctas, threads, smem, l.s, a);
    ACID_CHECK_LAUNCH();
    const bool weights = a.dpre_w != nullptr || a.dpost_w != nullptr;
    const bool vectors = a.dgate != nullptr || a.dscale != nullptr || a.dshift != nullptr;
    // does any group reach over an edge?
    const int64_t head = s.first > 0 ? s.first : 0, longest = std::max(head, std::min(s.group, s.rows - head));
    const bool over = vectors && longest > 1;
    if (!weights && !over) return ACID_OK;
    auto share = [](int64_t slots) {  // warps for so many slots
      int segs = 1;
      while (segs < kJoinWarps && segs * 8 < slots) segs *= 2;
      return segs;
    };
    Join n{1, 1, 0, share(ctas), ctas, s.groups > ctas};
    if (over) {
      n.jobs = n.by_cta ? ctas : (int)s.groups;
      n.segs = share(std::min<int64_t>(ctas, longest / a.per + 2));
      n.ctas_v = (3 * n.jobs * n.segs + kJoinWarps - 1) / kJoinWarps;
    }
    const int ctas_w = weights ? (2 * n.segs_w + kJoinWarps - 1) / kJoinWarps : 0;
    launch_pdl(site_join_kernel, dim3((s.d + 31) / 32, n.ctas_v + ctas_w), 32 * kJoinWarps, 0, l.s, a, n);
    ACID_CHECK_LAUNCH();
    return ACID_OK;
  }
};

size_t workspace_bytes(const acid_norm_site& s) {
  const int ctas = (int)std::min<int64_t>(max_ctas(s.d), std::max<int64_t>(s.rows, 1));
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
  acid_norm_site used = *site;
  // Without du or y their norms have no part in the gradients: the kernel finds zeros there, whose norm is none at eps 0.
  if (du == nullptr) used.pre_norm = ACID_NORM_NONE;
  if (y == nullptr) used.post_norm = ACID_NORM_NONE;
  const BwdLaunch l{{site_args(used), du, r, y, dr, lddu, ldr, ldy, lddr, o.dx, o.dy, o.lddx, o.lddy, o.dgate, o.dscale,
                     o.dshift, o.dpost_w, o.dpre_w, o.ld_dmod, static_cast<float*>(ws), nullptr, 1},
                    s};
  return by_types<RunBwd>(*site, l);
}
