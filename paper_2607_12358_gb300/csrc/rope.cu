// Rotary positions with several axes, and the rotation taken back, which is its
// gradient (acid_rope_*).
#include <math.h>

#include <algorithm>

#define ACID_UNIT_WITHOUT_WAITS
#include "common.cuh"
#include "internal.h"

namespace acid {

BoundsRecord take_bounds_rope();
ACID_BOUNDS_READER(take_bounds_rope)

namespace {

using bf16 = __nv_bfloat16;
constexpr int kAxes = 4, kMaxPairs = 128, kMaxRows = 4, kThreads = 256;

struct Rope {
  const void* x;
  void* out;
  int64_t ldx, ldo, rows, first;
  int heads, d, pairs;  // pairs of columns that are turned; the rest of a head passes through
  int copy_first;       // 0: in place, the first rows stay as they are
  float sign;           // -1: backwards
  const float* positions;
  int64_t ld_pos;
  uint32_t grid_rows;  // (rows are at most 2^31: a larger grid is cut to 2^32 - 1)
  int axes, grid[kAxes];
  float origin[kAxes];
  // Turns of pair p at position 1 as two floats, hi + lo, and its axis.
  float hi[kMaxPairs], lo[kMaxPairs];
  uint8_t axis[kMaxPairs];
};

// Angle of pair p at a position, as a fraction of half a turn.  pos hi is split
// into the product and its rounding error (one FMA each), so the whole turns drop
// out exactly and the angle is right to 2^-23 of a turn at any position up to 2^24 (of
// pairs that turn by up to a radian a place; by f radians: up to 2^24 / f, from where on
// the rounding error is itself whole turns and more); in fp32 radians the rounding of the angle itself is 2^-24 of it: 0.01 rad at 2e5.
__device__ __forceinline__ float half_turns(float pos, float hi, float lo) {
  const float t = pos * hi, e = fmaf(pos, hi, -t);
  return 2.0f * ((t - rintf(t)) + fmaf(pos, lo, e));
}

// (cos, sin) of all pairs of the CTA's rows.  A part's pairs are read two at a time, 16
// bytes: the first two of all parts lie side by side, then the next two, so that the
// lanes of a warp read without bank conflicts.
template <int PAIRS>
__device__ __forceinline__ void fill_table(const Rope& a, int64_t row0, int n, float2* table) {
  for (int i = threadIdx.x; i < n * a.pairs; i += kThreads) {
    const int r = i / a.pairs, p = i - r * a.pairs, ax = a.axis[p];
    const int64_t row = row0 + r;
    if (row < a.first) continue;
    float pos;
    if (a.positions != nullptr) {
      const int64_t at = row * a.ld_pos + ax;
      if (!ACID_IN_BOUNDS(kSiteRope, at, a.rows * a.ld_pos)) continue;
      pos = a.positions[at];
    } else {
      uint32_t place = (uint32_t)(row - a.first) % a.grid_rows;  // row-major over the grid, the last axis fastest
      for (int k = a.axes - 1; k > ax; --k) place /= (uint32_t)a.grid[k];
      pos = (float)(place % (uint32_t)a.grid[ax]) + a.origin[ax];
    }
    float s, c;
    sincospif(half_turns(pos, a.hi[p], a.lo[p]), &s, &c);
    const int in = p % PAIRS;
    table[r * a.pairs + in / 2 * (a.pairs / PAIRS * 2) + p / PAIRS * 2 + in % 2] = make_float2(c, a.sign * s);
  }
}

// One thread's part of a head: 8 columns (4 interleaved pairs), or, where the pairs are
// (p, p + pairs), 8 columns of each half; held as they are loaded.
template <typename T, bool HALVES>
struct Part {
  static constexpr int kWords = (int)sizeof(T) / 2, kVectors = HALVES ? 2 * kWords : kWords;  // 16 bytes each
  uint4 u[kVectors];
  __device__ __forceinline__ void load(const T* p, int pairs, bool turned) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) u[i] = reinterpret_cast<const uint4*>(p)[i];
    if constexpr (HALVES) {
      if (turned)
#pragma unroll
        for (int i = 0; i < kWords; ++i) u[kWords + i] = reinterpret_cast<const uint4*>(p + pairs)[i];
    }
  }
  __device__ __forceinline__ void get(float* v, int half) const {
    const uint4* w = u + half * kWords;
    if constexpr (sizeof(T) == 2) {
      v[0] = bf16_lo(w->x); v[1] = bf16_hi(w->x); v[2] = bf16_lo(w->y); v[3] = bf16_hi(w->y);
      v[4] = bf16_lo(w->z); v[5] = bf16_hi(w->z); v[6] = bf16_lo(w->w); v[7] = bf16_hi(w->w);
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        v[4 * i] = __uint_as_float(w[i].x); v[4 * i + 1] = __uint_as_float(w[i].y);
        v[4 * i + 2] = __uint_as_float(w[i].z); v[4 * i + 3] = __uint_as_float(w[i].w);
      }
    }
  }
  static constexpr int kPairs = HALVES ? 8 : 4;
  // Turned by the pairs' (cos, sin), and stored.
  __device__ __forceinline__ void turn(T* p, int pairs, const float2* t) const {
    float a[8], b[8];
    get(a, 0);
    if constexpr (HALVES) get(b, 1);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const float2 cs = t[i / 2 * (pairs / kPairs * 2) + i % 2];
      float& x = HALVES ? a[i] : a[2 * i];
      float& y = HALVES ? b[i] : a[2 * i + 1];
      const float x0 = x, y0 = y;
      x = fmaf(x0, cs.x, -y0 * cs.y);
      y = fmaf(x0, cs.y, y0 * cs.x);
    }
    store8(p, a);
    if constexpr (HALVES) store8(p + pairs, b);
  }
  __device__ __forceinline__ void keep(T* p, int pairs, bool turned) const {
#pragma unroll
    for (int i = 0; i < kWords; ++i) reinterpret_cast<uint4*>(p)[i] = u[i];
    if constexpr (HALVES) {
      if (turned)
#pragma unroll
        for (int i = 0; i < kWords; ++i) reinterpret_cast<uint4*>(p + pairs)[i] = u[kWords + i];
    }
  }
};

// A CTA has up to kMaxRows rows: it forms their angles' cosines and sines once, one a
// thread, and then its threads sweep over the rows' heads, each on the same columns of
// every head it meets.  HBM bound; what keeps loads in flight is eight CTAs an SM with two
// 16-byte loads a thread.  (One load a thread: 90 us at 32760 rows, 24 heads of 128; four,
// which leaves six CTAs, 96; two 80.  A row's cosines and sines kept in registers over
// its heads, and so row by row: 88.)
template <typename T, bool HALVES>
__global__ void __launch_bounds__(kThreads) rope_kernel(const __grid_constant__ Rope a, int rows_per_cta) {
  extern __shared__ __align__(16) float2 table[];
  using P = Part<T, HALVES>;
  const int64_t row0 = (int64_t)blockIdx.x * rows_per_cta;
  const int n = (int)min((int64_t)rows_per_cta, a.rows - row0);
  if (a.positions != nullptr) pdl_wait();
  fill_table<P::kPairs>(a, row0, n, table);
  if (a.positions == nullptr) pdl_wait();
  __syncthreads();
  const int turned_parts = a.pairs / P::kPairs;
  const int parts = turned_parts + (a.d - 2 * a.pairs) / 8;  // threads to a head
  const int heads_at_once = kThreads / parts;
  const int part = threadIdx.x % parts, lane = threadIdx.x / parts;
  if (lane >= heads_at_once) return;
  const bool turned = part < turned_parts;
  const int col = HALVES && !turned ? 2 * a.pairs + (part - turned_parts) * 8 : part * 8;
  constexpr int kAhead = P::kVectors <= 2 ? 2 : 1;
  const int total = n * a.heads;
  for (int i = lane; i < total; i += kAhead * heads_at_once) {
    P p[kAhead];
    int64_t from[kAhead], to[kAhead];
    int rows[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int at = i + k * heads_at_once;
      rows[k] = at < total ? at / a.heads : -1;
      if (rows[k] < 0) continue;
      const int64_t row = row0 + rows[k], c = (int64_t)(at - rows[k] * a.heads) * a.d + col;
      from[k] = row * a.ldx + c;
      to[k] = row * a.ldo + c;
      // (in place the columns and rows that are not turned are left alone)
      if (!a.copy_first && !(turned && row >= a.first)) rows[k] = -1;
      if (!ACID_IN_BOUNDS(kSiteRope, from[k] + (HALVES && turned ? a.pairs : 0) + 7, a.rows * a.ldx) ||
          !ACID_IN_BOUNDS(kSiteRope, to[k] + (HALVES && turned ? a.pairs : 0) + 7, a.rows * a.ldo))
        rows[k] = -1;
      if (rows[k] >= 0) p[k].load(static_cast<const T*>(a.x) + from[k], a.pairs, turned);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (rows[k] < 0) continue;
      T* out = static_cast<T*>(a.out) + to[k];
      if (turned && row0 + rows[k] >= a.first) p[k].turn(out, a.pairs, table + rows[k] * a.pairs + part * 2);
      else p[k].keep(out, a.pairs, turned);
    }
  }
}

acid_status rope_entry(const acid_rope* r, const void* x, int64_t ldx, void* out, int64_t ldo, float sign,
                       cudaStream_t s) {
  ACID_REQUIRE(r != nullptr, ACID_ERR_INVALID_ARG, "rope: null description");
  ACID_REQUIRE(r->dtype == ACID_BF16 || r->dtype == ACID_FP32, ACID_ERR_INVALID_ARG, "rope: unknown dtype");
  ACID_REQUIRE(r->rows >= 0 && r->heads > 0 && r->head_dim > 0, ACID_ERR_INVALID_ARG, "rope: bad rows, heads or head_dim");
  ACID_REQUIRE(r->first_rows >= 0 && r->first_rows <= r->rows, ACID_ERR_INVALID_ARG,
               "rope: need 0 <= first_rows <= rows");
  ACID_REQUIRE(r->axes >= 1 && r->axes <= kAxes, ACID_ERR_INVALID_ARG, "rope: need 1 to 4 axes");
  ACID_REQUIRE(r->head_dim % 8 == 0 && r->head_dim <= 2 * kMaxPairs, ACID_ERR_UNSUPPORTED,
               "rope: head_dim must be a multiple of 8, <= 256");
  Rope a = {};
  for (int ax = 0; ax < r->axes; ++ax) {
    const int n = r->axis_dim[ax];
    ACID_REQUIRE(n > 0 && n % 2 == 0 && 2 * a.pairs + n <= r->head_dim, ACID_ERR_INVALID_ARG,
                 "rope: axes must have an even number of columns, no more than head_dim in all");
    ACID_REQUIRE(r->theta[ax] > 0 && isfinite(r->theta[ax]), ACID_ERR_INVALID_ARG,
                 "rope: theta must be positive and finite");
    // (a product a pair: 64 powers would take longer than the smallest calls' kernel)
    const double ratio = pow((double)r->theta[ax], -2.0 / n);
    double turns = 1.0 / 6.283185307179586476925286766559;
    for (int j = 0; j < n / 2; ++j, ++a.pairs, turns *= ratio) {
      a.hi[a.pairs] = (float)turns;
      a.lo[a.pairs] = (float)(turns - (double)a.hi[a.pairs]);
      a.axis[a.pairs] = (uint8_t)ax;
    }
  }
  const bool halves = r->halves != 0;
  ACID_REQUIRE(a.pairs % (halves ? 8 : 4) == 0, ACID_ERR_UNSUPPORTED,
               "rope: the axes' columns must be a multiple of 8 in all, 16 with halves");
  int64_t places = 1;
  a.axes = r->axes;
  for (int ax = 0; r->positions == nullptr && ax < r->axes; ++ax) {
    ACID_REQUIRE(r->grid[ax] > 0 && places <= ((int64_t)1 << 40) / r->grid[ax], ACID_ERR_INVALID_ARG,
                 "rope: need positions, or a grid of at least 1 and at most 2^40 places");
    ACID_REQUIRE(isfinite(r->origin[ax]), ACID_ERR_INVALID_ARG, "rope: origin must be finite");
    a.grid[ax] = r->grid[ax];
    a.origin[ax] = r->origin[ax];
    places *= r->grid[ax];
  }
  a.grid_rows = (uint32_t)std::min<int64_t>(places, UINT32_MAX);
  ACID_REQUIRE(r->positions == nullptr || (r->ld_pos >= r->axes && aligned(r->positions, 4)), ACID_ERR_INVALID_ARG,
               "rope: positions need a row stride of at least the axes, and 4-byte alignment");
  const int64_t width = (int64_t)r->heads * r->head_dim;
  ACID_REQUIRE(width <= INT32_MAX / kMaxRows && r->rows <= (int64_t)1 << 31, ACID_ERR_UNSUPPORTED, "rope: too large");
  ACID_REQUIRE(ldx >= width && ldo >= width, ACID_ERR_INVALID_ARG, "rope: row stride smaller than heads * head_dim");
  if (r->rows == 0) return ACID_OK;
  ACID_REQUIRE(x != nullptr && out != nullptr, ACID_ERR_INVALID_ARG, "rope: null pointer");
  ACID_REQUIRE(aligned(x, 16) && aligned(out, 16) && ldx % 8 == 0 && ldo % 8 == 0, ACID_ERR_UNSUPPORTED,
               "rope: operands must be 16-byte aligned, their row strides multiples of 8");
  ACID_REQUIRE(x != out || ldx == ldo, ACID_ERR_INVALID_ARG, "rope: in place needs one row stride");
  a.x = x;
  a.out = out;
  a.ldx = ldx;
  a.ldo = ldo;
  a.rows = r->rows;
  a.first = r->first_rows;
  a.heads = r->heads;
  a.d = r->head_dim;
  a.copy_first = x != out;
  a.sign = sign;
  a.positions = r->positions;
  a.ld_pos = r->ld_pos;
  const int per = (int)std::min<int64_t>(kMaxRows, std::max<int64_t>(1, r->rows / (8 * num_sms())));
  const int64_t ctas = (r->rows + per - 1) / per;
  const auto kernel = r->dtype == ACID_BF16 ? (halves ? rope_kernel<bf16, true> : rope_kernel<bf16, false>)
                                            : (halves ? rope_kernel<float, true> : rope_kernel<float, false>);
  launch_pdl(kernel, (unsigned)ctas, kThreads, (size_t)per * a.pairs * sizeof(float2), s, a, per);
  ACID_CHECK_LAUNCH();
  return ACID_OK;
}

}  // namespace
}  // namespace acid

using namespace acid;

extern "C" acid_status acid_rope_forward(const acid_rope* rope, const void* x, int64_t ldx, void* out, int64_t ldo,
                                         acid_stream_t stream) {
  clear_error();
  return rope_entry(rope, x, ldx, out, ldo, 1.0f, (cudaStream_t)stream);
}

extern "C" acid_status acid_rope_backward(const acid_rope* rope, const void* dout, int64_t lddo, void* dx, int64_t lddx,
                                          acid_stream_t stream) {
  clear_error();
  return rope_entry(rope, dout, lddo, dx, lddx, -1.0f, (cudaStream_t)stream);
}
