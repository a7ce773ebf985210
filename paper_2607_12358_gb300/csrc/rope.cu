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
  int64_t grid_rows;
  int axes, grid[kAxes];
  float origin[kAxes];
  // Turns of pair p at position 1 as two floats, hi + lo, and its axis.
  float hi[kMaxPairs], lo[kMaxPairs];
  uint8_t axis[kMaxPairs];
};

// Angle of pair p at a position, as a fraction of half a turn.  pos hi is split
// into the product and its rounding error (one FMA each), so the whole turns drop
// out exactly and the angle is right to 2^-23 of a turn at any position up to 2^24;
// in fp32 radians the rounding of the angle itself is 2^-24 of it: 0.01 rad at 2e5.
__device__ __forceinline__ float half_turns(float pos, float hi, float lo) {
  const float t = pos * hi, e = fmaf(pos, hi, -t);
  return 2.0f * ((t - rintf(t)) + fmaf(pos, lo, e));
}

// (cos, sin) of all pairs of the CTA's rows.
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
      int64_t n_ax = (row - a.first) % a.grid_rows;  // row-major over the grid, the last axis fastest
      for (int k = a.axes - 1; k > ax; --k) n_ax /= a.grid[k];
      pos = (float)(n_ax % a.grid[ax]) + a.origin[ax];
    }
    float s, c;
    sincospif(half_turns(pos, a.hi[p], a.lo[p]), &s, &c);
    table[i] = make_float2(c, a.sign * s);
  }
}

// One thread's part of a head: 8 columns (4 interleaved pairs), or, where the
// pairs are (p, p + pairs), 8 columns of each half.
template <typename T, bool HALVES>
struct Part {
  float v[HALVES ? 16 : 8];
  __device__ __forceinline__ void load(const T* p, int pairs, bool turned) {
    load8(p, v);
    if constexpr (HALVES) {
      if (turned) load8(p + pairs, v + 8);
    }
  }
  __device__ __forceinline__ void turn(const float2* t) {
#pragma unroll
    for (int i = 0; i < (HALVES ? 8 : 4); ++i) {
      const float2 cs = t[i];
      float& a = v[HALVES ? i : 2 * i];
      float& b = v[HALVES ? i + 8 : 2 * i + 1];
      const float x = a, y = b;
      a = fmaf(x, cs.x, -y * cs.y);
      b = fmaf(x, cs.y, y * cs.x);
    }
  }
  __device__ __forceinline__ void store(T* p, int pairs, bool turned) const {
    store8(p, v);
    if constexpr (HALVES) {
      if (turned) store8(p + pairs, v + 8);
    }
  }
};

// A CTA has up to kMaxRows rows: it forms their angles' cosines and sines once,
// one a thread, and then its threads sweep over the rows' heads, each on the same
// columns of every head it meets.
template <typename T, bool HALVES>
__global__ void __launch_bounds__(kThreads) rope_kernel(const __grid_constant__ Rope a, int rows_per_cta) {
  extern __shared__ __align__(16) float2 table[];
  const int64_t row0 = (int64_t)blockIdx.x * rows_per_cta;
  const int n = (int)min((int64_t)rows_per_cta, a.rows - row0);
  if (a.positions != nullptr) pdl_wait();
  fill_table(a, row0, n, table);
  if (a.positions == nullptr) pdl_wait();
  __syncthreads();
  const int turned_parts = HALVES ? a.pairs / 8 : a.pairs / 4;
  const int parts = turned_parts + (a.d - 2 * a.pairs) / 8;  // threads to a head
  const int heads_at_once = kThreads / parts;
  const int part = threadIdx.x % parts, lane = threadIdx.x / parts;
  if (lane >= heads_at_once) return;
  const bool turned = part < turned_parts;
  const int col = HALVES && !turned ? 2 * a.pairs + (part - turned_parts) * 8 : part * 8;
  for (int i = lane; i < n * a.heads; i += heads_at_once) {
    const int r = i / a.heads, h = i - r * a.heads;
    const int64_t row = row0 + r;
    const bool turn = turned && row >= a.first;
    if (!turn && !a.copy_first) continue;  // in place: nothing to do
    const int64_t c = (int64_t)h * a.d + col;
    if (!ACID_IN_BOUNDS(kSiteRope, row * a.ldx + c + 7, a.rows * a.ldx) ||
        !ACID_IN_BOUNDS(kSiteRope, row * a.ldo + c + 7, a.rows * a.ldo))
      continue;
    Part<T, HALVES> p;
    p.load(static_cast<const T*>(a.x) + row * a.ldx + c, a.pairs, turned);
    if (turn) p.turn(table + r * a.pairs + part * (HALVES ? 8 : 4));
    p.store(static_cast<T*>(a.out) + row * a.ldo + c, a.pairs, turned);
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
  a.grid_rows = 1;
  a.axes = r->axes;
  for (int ax = 0; r->positions == nullptr && ax < r->axes; ++ax) {
    ACID_REQUIRE(r->grid[ax] > 0 && a.grid_rows <= ((int64_t)1 << 40) / r->grid[ax], ACID_ERR_INVALID_ARG,
                 "rope: need positions, or a grid of at least 1 and at most 2^40 places");
    ACID_REQUIRE(isfinite(r->origin[ax]), ACID_ERR_INVALID_ARG, "rope: origin must be finite");
    a.grid[ax] = r->grid[ax];
    a.origin[ax] = r->origin[ax];
    a.grid_rows *= r->grid[ax];
  }
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
