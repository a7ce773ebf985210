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

constexpr int kMaxWidth = 4096;           // 16 warps of 8 columns a lane
constexpr int kMaxWarps = kMaxWidth / 256;

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

// 8 columns of a vector, or 8 times the same value where there is none.
__device__ __forceinline__ void vec8(const float* p, int c, int d, float none, float* v) {
  if (p != nullptr && ACID_IN_BOUNDS(kSiteNormSite, c + 7, d)) {
    load8(p + c, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = none;
  }
}
template <typename T>
__device__ __forceinline__ void row8(const void* p, int64_t ld, int64_t row, int64_t rows, int c, float* v) {
  if (ACID_IN_BOUNDS(kSiteNormSite, row, rows)) load8(static_cast<const T*>(p) + row * ld + c, v);
}
template <typename T>
__device__ __forceinline__ void put8(void* p, int64_t ld, int64_t row, int64_t rows, int c, const float* v) {
  if (ACID_IN_BOUNDS(kSiteNormSite, row, rows)) store8(static_cast<T*>(p) + row * ld + c, v);
}

// Sums of N values over the CTA; every thread gets them.  Rounds alternate
// between two buffers, so that one barrier a round is enough: a thread writes a
// buffer again behind the other one's barrier.
template <int N>
__device__ __forceinline__ void cta_sum(float (&v)[N], float (*red)[kMaxWarps][4], int& round) {
  static_assert(N <= 4, "a warp's slot holds four sums");
  const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  if (warps == 1) return;
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) red[round][warp][i] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = 0.f;
  for (int w = 0; w < warps; ++w)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += red[round][w][i];
  round ^= 1;
}

// v (0 in the columns past the row) becomes N(v); returns 1 / the root.
__device__ __forceinline__ float norm_row(float (&v)[8], int kind, bool on, int d, float eps,
                                          float (*red)[kMaxWarps][4], int& round) {
  if (kind == ACID_NORM_NONE) return 1.f;
  if (kind == ACID_NORM_LAYER) {
    float s[1] = {0.f};
#pragma unroll
    for (int j = 0; j < 8; ++j) s[0] += v[j];
    cta_sum(s, red, round);
    const float mean = s[0] / d;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = on ? v[j] - mean : 0.f;
  }
  float q[1] = {0.f};
#pragma unroll
  for (int j = 0; j < 8; ++j) q[0] = fmaf(v[j], v[j], q[0]);
  cta_sum(q, red, round);
  const float inv = rsqrtf(q[0] / d + eps);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] *= inv;
  return inv;
}

// One row at a time, 8 columns a thread.
template <typename TS, typename TB>
__global__ void __launch_bounds__(32 * kMaxWarps) site_forward_kernel(SiteFwd a) {
  __shared__ float red[2][kMaxWarps][4];
  pdl_wait();
  const Site& s = a.s;
  const int c = threadIdx.x * 8, d = s.d;
  const bool on = c < d;
  int round = 0;
  for (int64_t row = blockIdx.x; row < s.rows; row += gridDim.x) {
    const int64_t m = group_of(s, row) * s.ld_mod;
    float r[8] = {}, t[8];
    if (on) {
      row8<TS>(a.x, a.ldx, row, s.rows, c, r);
#pragma unroll
      for (int j = 0; j < 8; ++j) r[j] *= s.res;
    }
    if (a.y != nullptr) {
      float y[8] = {};
      if (on) row8<TB>(a.y, a.ldy, row, s.rows, c, y);
      norm_row(y, s.post, on, d, s.eps, red, round);
      if (on) {
        vec8(s.post_w, c, d, 1.f, t);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] *= t[j];
        vec8(s.gate ? s.gate + m : nullptr, c, d, 1.f, t);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float g = s.tanh && s.gate ? tanhf(t[j]) : t[j];
          r[j] = fmaf(s.branch * g, y[j], r[j]);
        }
      }
    }
    if (on && a.r != nullptr) put8<TS>(a.r, a.ldr, row, s.rows, c, r);
    if (a.u == nullptr) continue;
    norm_row(r, s.pre, on, d, s.eps, red, round);
    if (!on) continue;
    vec8(s.pre_w, c, d, 1.f, t);
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] *= t[j];
    vec8(s.scale ? s.scale + m : nullptr, c, d, 0.f, t);
    float h[8];
    vec8(s.shift ? s.shift + m : nullptr, c, d, 0.f, h);
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = fmaf(r[j], 1.f + t[j], h[j]);
    put8<TB>(a.u, a.ldu, row, s.rows, c, r);
  }
}

// The gradient of a norm's input from dn, that of its output n.
__device__ __forceinline__ void norm_back(float (&dn)[8], const float (&n)[8], float inv, int kind, bool on, int d,
                                          float (*red)[kMaxWarps][4], int& round) {
  if (kind == ACID_NORM_NONE) return;
  float s[2] = {0.f, 0.f};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    s[0] += dn[j];
    s[1] = fmaf(dn[j], n[j], s[1]);
  }
  cta_sum(s, red, round);
  const float mean = kind == ACID_NORM_LAYER ? s[0] / d : 0.f, along = s[1] / d;
#pragma unroll
  for (int j = 0; j < 8; ++j) dn[j] = on ? (dn[j] - mean - n[j] * along) * inv : 0.f;
}

// Gradients of the site's vectors for one group from the raw sums
// A = sum du, S = sum du n, T = sum dr p over its rows.
__device__ __forceinline__ void put_group(const SiteBwd& a, int64_t g, int c, const float (&A)[8], const float (&S)[8],
                                          const float (&T)[8]) {
  const Site& s = a.s;
  float w[8], o[8];
  const int64_t at = g * a.ld_dmod + c, m = g * s.ld_mod;
  if (a.dshift != nullptr) store8(a.dshift + at, A);
  if (a.dscale != nullptr) {
    vec8(s.pre_w, c, s.d, 1.f, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = w[j] * S[j];
    store8(a.dscale + at, o);
  }
  if (a.dgate != nullptr) {
    vec8(s.post_w, c, s.d, 1.f, w);
    float t[8];
    vec8(s.gate ? s.gate + m : nullptr, c, s.d, 1.f, t);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float th = s.tanh && s.gate ? tanhf(t[j]) : 0.f;
      o[j] = s.branch * w[j] * T[j] * (1.f - th * th);
    }
    store8(a.dgate + at, o);
  }
}

// CTA b takes the rows [b per, (b + 1) per).  A group that lies in it is
// finished here; of one that reaches over its edge the sums go to the CTA's
// slot 2 b (the group began earlier) or 2 b + 1 (it begins here).
template <typename TS, typename TB>
__global__ void __launch_bounds__(32 * kMaxWarps) site_backward_kernel(SiteBwd a) {
  __shared__ float red[2][kMaxWarps][4];
  pdl_wait();
  const Site& s = a.s;
  const int c = threadIdx.x * 8, d = s.d;
  const bool on = c < d;
  int round = 0;
  const int64_t begin = blockIdx.x * a.per, end = min(s.rows, begin + a.per);
  float W[2][8] = {};
  for (int64_t row = begin; row < end;) {
    const int64_t g = group_of(s, row), m = g * s.ld_mod, from = row, to = min(end, group_end(s, g));
    float A[8] = {}, S[8] = {}, T[8] = {}, sc[8] = {}, gp[8] = {}, w[8];
    if (on) {
      vec8(s.scale ? s.scale + m : nullptr, c, d, 0.f, sc);
      vec8(s.gate ? s.gate + m : nullptr, c, d, 1.f, gp);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        sc[j] += 1.f;
        gp[j] = s.branch * (s.tanh && s.gate ? tanhf(gp[j]) : gp[j]);
      }
    }
    for (; row < to; ++row) {
      float dr[8] = {};
      if (on && a.dr != nullptr) row8<TS>(a.dr, a.lddr, row, s.rows, c, dr);
      if (a.du != nullptr) {
        float n[8] = {}, du[8] = {};
        if (on) {
          row8<TS>(a.r, a.ldr, row, s.rows, c, n);
          row8<TB>(a.du, a.lddu, row, s.rows, c, du);
        }
        const float inv = norm_row(n, s.pre, on, d, s.eps, red, round);
        if (on) vec8(s.pre_w, c, d, 1.f, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          A[j] += du[j];
          S[j] = fmaf(du[j], n[j], S[j]);
          du[j] = on ? du[j] * sc[j] * w[j] : 0.f;
        }
        norm_back(du, n, inv, s.pre, on, d, red, round);
#pragma unroll
        for (int j = 0; j < 8; ++j) dr[j] += du[j];
      }
      if (on && a.dx != nullptr) {
        float o[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = s.res * dr[j];
        put8<TS>(a.dx, a.lddx, row, s.rows, c, o);
      }
      if (a.y == nullptr) continue;
      float p[8] = {};
      if (on) row8<TB>(a.y, a.ldy, row, s.rows, c, p);
      const float inv = norm_row(p, s.post, on, d, s.eps, red, round);
      if (on) vec8(s.post_w, c, d, 1.f, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        T[j] = fmaf(dr[j], p[j], T[j]);
        dr[j] = on ? dr[j] * gp[j] * w[j] : 0.f;
      }
      if (a.dy == nullptr) continue;
      norm_back(dr, p, inv, s.post, on, d, red, round);
      if (on) put8<TB>(a.dy, a.lddy, row, s.rows, c, dr);
    }
    if (!on) continue;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      W[0][j] = fmaf(sc[j], S[j], W[0][j]);
      W[1][j] = fmaf(gp[j], T[j], W[1][j]);
    }
    const bool starts = group_begin(s, g) == from, ends = group_end(s, g) == to;
    if (starts && ends) {
      put_group(a, g, c, A, S, T);
    } else {
      float* slot = a.part + (2 * (int64_t)blockIdx.x + starts) * 3 * d + c;
      store8(slot, A);
      store8(slot + d, S);
      store8(slot + 2 * d, T);
    }
  }
  if (!on) return;
  float* wp = a.wpart + (int64_t)blockIdx.x * 2 * d + c;
  store8(wp, W[0]);
  store8(wp + d, W[1]);
}

// Joins the CTAs' sums in the CTAs' order: blockIdx.y < ctas: the group that
// begins in that CTA and reaches past its end (if there is one); y = ctas: the
// weights' gradients.
__global__ void __launch_bounds__(128) site_join_kernel(SiteBwd a, int ctas) {
  pdl_wait();
  const Site& s = a.s;
  const int c = (blockIdx.x * 128 + threadIdx.x) * 8, d = s.d;
  if (c >= d) return;
  float v[3][8] = {}, t[8];
  if ((int)blockIdx.y == ctas) {
    for (int b = 0; b < ctas; ++b)
      for (int i = 0; i < 2; ++i) {
        load8(a.wpart + ((int64_t)b * 2 + i) * d + c, t);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] += t[j];
      }
    if (a.dpre_w != nullptr) store8(a.dpre_w + c, v[0]);
    if (a.dpost_w != nullptr) store8(a.dpost_w + c, v[1]);
    return;
  }
  const int64_t b = blockIdx.y, end = min(s.rows, (b + 1) * a.per), g = group_of(s, end - 1);
  if (group_end(s, g) <= end || group_begin(s, g) < b * a.per) return;
  const int64_t last = (group_end(s, g) - 1) / a.per;
  for (int64_t k = b; k <= last; ++k)
    for (int i = 0; i < 3; ++i) {
      load8(a.part + ((2 * k + (k == b)) * 3 + i) * d + c, t);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] += t[j];
    }
  put_group(a, g, c, v[0], v[1], v[2]);
}

constexpr int kMaxCtas = 1024;

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
  ACID_REQUIRE(s->rows >= 0 && s->d > 0 && s->rows <= (int64_t(1) << 40), ACID_ERR_INVALID_ARG, "norm_site: bad shape");
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

int threads_for(int d) { return (d + 255) / 256 * 32; }

// Rows of a CTA of the backward pass, and the CTAs.
struct Split {
  int64_t per;
  int ctas;
};
Split split_rows(int64_t rows, int most) {
  const int64_t per = std::max<int64_t>(1, (rows + most - 1) / most);
  return {per, (int)((rows + per - 1) / per)};
}

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
    const unsigned grid = (unsigned)std::min<int64_t>(l.a.s.rows, (int64_t)num_sms() * 8);
    launch_pdl(site_forward_kernel<TS, TB>, grid, threads_for(l.a.s.d), 0, l.s, l.a);
    ACID_CHECK_LAUNCH();
    return ACID_OK;
  }
};
struct BwdLaunch {
  SiteBwd a;
  int ctas;
  cudaStream_t s;
};
template <typename TS, typename TB>
struct RunBwd {
  static acid_status run(const BwdLaunch& l) {
    launch_pdl(site_backward_kernel<TS, TB>, l.ctas, threads_for(l.a.s.d), 0, l.s, l.a);
    ACID_CHECK_LAUNCH();
    return ACID_OK;
  }
};

size_t part_bytes(int d, int ctas) { return (size_t)ctas * 2 * 3 * d * sizeof(float); }
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
  const Split sp = split_rows(site->rows, std::min(kMaxCtas, num_sms() * 2));
  BwdLaunch l{{site_args(*site), du, r, y, dr, lddu, ldr, ldy, lddr, o.dx, o.dy, o.lddx, o.lddy, o.dgate, o.dscale,
               o.dshift, o.dpost_w, o.dpre_w, o.ld_dmod, static_cast<float*>(ws), nullptr, sp.per},
              sp.ctas, s};
  l.a.wpart = l.a.part + part_bytes(site->d, sp.ctas) / sizeof(float);
  ACID_TRY(by_types<RunBwd>(*site, l));
  launch_pdl(site_join_kernel, dim3((site->d / 8 + 127) / 128, sp.ctas + 1), 128, 0, s, l.a, sp.ctas);
  ACID_CHECK_LAUNCH();
  return ACID_OK;
}
