// Modulation projections with 4-bit weights: quantiser, values, product and
// input gradient (acid_q4_*).
#include <algorithm>
#include <string>

#define ACID_UNIT_WITHOUT_WAITS
#include "common.cuh"
#include "internal.h"

namespace acid {

BoundsRecord take_bounds_q4();
ACID_BOUNDS_READER(take_bounds_q4)

namespace {

constexpr int kThreads = 256;
using bf16 = __nv_bfloat16;

// A weight as the kernels see it.
struct Q4 {
  const uint32_t* packed;  // [n][16 slabs] words
  const void* scales;
  const uint8_t* zeros;
  int64_t n;
  int k, slabs, group_log, groups;  // group = 1 << group_log columns; groups = ceil(k / group)
};
// First of the eight columns that word `w` of a row holds.
__device__ __forceinline__ int word_column(int w) { return (w >> 4) * 128 + (w & 3) * 32 + ((w >> 2) & 3) * 8; }
// The word that holds the columns 8 o .. 8 o + 7.
__device__ __forceinline__ int column_word(int o) { return (o & ~15) + ((o & 3) << 2) + ((o >> 2) & 3); }

template <typename TS>
__device__ __forceinline__ float scale_at(const Q4& w, int64_t row, int col) {
  const int64_t i = row * w.groups + (col >> w.group_log);
  return ACID_IN_BOUNDS(kSiteQ4, i, w.n * w.groups) ? io<TS>::ld(static_cast<const TS*>(w.scales) + i) : 0.f;
}
__device__ __forceinline__ int zero_at(const Q4& w, int64_t row, int col) {
  const int64_t i = row * w.groups + (col >> w.group_log);
  return w.zeros != nullptr && ACID_IN_BOUNDS(kSiteQ4, i, w.n * w.groups) ? w.zeros[i] : 8;
}
__device__ __forceinline__ uint32_t word_at(const Q4& w, int64_t row, int i) {
  const int64_t at = row * w.slabs * 16 + i;
  return ACID_IN_BOUNDS(kSiteQ4, at, w.n * w.slabs * 16) ? w.packed[at] : 0u;
}

__device__ __forceinline__ float value_at(int dtype, const void* p, int64_t i) {
  return dtype == ACID_BF16 ? __bfloat162float(static_cast<const bf16*>(p)[i]) : static_cast<const float*>(p)[i];
}
__device__ __forceinline__ void put_value(int dtype, void* p, int64_t i, float v) {
  if (dtype == ACID_BF16)
    static_cast<bf16*>(p)[i] = __float2bfloat16_rn(v);
  else
    static_cast<float*>(p)[i] = v;
}

struct Fwd {
  Q4 w;
  const void* x;
  int64_t ldx, m;
  int x_dtype, silu, out_dtype;
  const float* bias;
  void* out;
  int64_t ldo;
};

// A warp forms one output column of up to 4 rows.
constexpr int kRows = 4;
template <typename TS>
__global__ void __launch_bounds__(kThreads) q4_forward_kernel(Fwd a) {
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), m0 = (int64_t)blockIdx.y * kRows;
  if (row >= a.w.n) return;
  float acc[kRows] = {};
  for (int i = lane; i < a.w.slabs * 16; i += 32) {
    const int col = word_column(i);
    if (col >= a.w.k) continue;
    const uint32_t word = word_at(a.w, row, i);
    const float s = scale_at<TS>(a.w, row, col);
    const int z = zero_at(a.w, row, col);
    for (int j = 0; j < 8 && col + j < a.w.k; ++j) {
      const float v = s * (float)((int)(word >> (4 * j) & 15u) - z);
      for (int m = 0; m < kRows; ++m) {
        if (m0 + m >= a.m) break;
        float x = value_at(a.x_dtype, a.x, (m0 + m) * a.ldx + col + j);
        if (a.silu) x = silu(x);
        acc[m] = fmaf(x, v, acc[m]);
      }
    }
  }
  for (int m = 0; m < kRows; ++m) {
    for (int o = 16; o > 0; o >>= 1) acc[m] += __shfl_xor_sync(0xffffffffu, acc[m], o);
    if (lane == 0 && m0 + m < a.m)
      put_value(a.out_dtype, a.out, (m0 + m) * a.ldo + row, acc[m] + (a.bias ? a.bias[row] : 0.f));
  }
}

struct Bwd {
  Q4 w;
  const void *g, *x;
  int64_t ldg, ldx, m;
  int g_dtype, x_dtype, silu;
  void* dx;
  int64_t lddx;
  float* dbias;
  float* part;  // [splits][m][128 slabs]
  int splits;
};

// A thread sums its word's eight columns over a share of the weight's rows.
template <typename TS>
__global__ void __launch_bounds__(kThreads) q4_backward_kernel(Bwd a) {
  pdl_wait();
  const int i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= a.w.slabs * 16) return;
  const int col = word_column(i);
  const int64_t m0 = (int64_t)blockIdx.z * kRows;
  const int64_t per = (a.w.n + a.splits - 1) / a.splits;
  const int64_t begin = blockIdx.y * per, end = min(a.w.n, begin + per);
  float acc[kRows][8] = {};
  if (col < a.w.k)
    for (int64_t row = begin; row < end; ++row) {
      const uint32_t word = word_at(a.w, row, i);
      const float s = scale_at<TS>(a.w, row, col);
      const int z = zero_at(a.w, row, col);
      for (int m = 0; m < kRows; ++m) {
        if (m0 + m >= a.m) break;
        const float g = value_at(a.g_dtype, a.g, (m0 + m) * a.ldg + row) * s;
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[m][j] = fmaf(g, (float)((int)(word >> (4 * j) & 15u) - z), acc[m][j]);
      }
    }
  for (int m = 0; m < kRows; ++m)
    if (m0 + m < a.m) store8(a.part + ((int64_t)blockIdx.y * a.m + m0 + m) * a.w.slabs * 128 + col, acc[m]);
}

// Joins the shares in their order and takes the activation's gradient.
__global__ void __launch_bounds__(kThreads) q4_backward_join_kernel(Bwd a) {
  pdl_wait();
  const int c = blockIdx.x * kThreads + threadIdx.x;
  const int64_t m = blockIdx.y;
  if (c >= a.w.k) return;
  float v = 0.f;
  for (int b = 0; b < a.splits; ++b) v += a.part[((int64_t)b * a.m + m) * a.w.slabs * 128 + c];
  if (a.silu) {
    const float x = value_at(a.x_dtype, a.x, m * a.ldx + c), e = 1.f / (1.f + expf(-x));
    v *= e * (1.f + x * (1.f - e));
  }
  put_value(a.x_dtype, a.dx, m * a.lddx + c, v);
}

__global__ void __launch_bounds__(kThreads) q4_bias_kernel(Bwd a) {
  pdl_wait();
  const int64_t n = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (n >= a.w.n) return;
  float v = 0.f;
  for (int64_t m = 0; m < a.m; ++m) v += value_at(a.g_dtype, a.g, m * a.ldg + n);
  a.dbias[n] = v;
}

// ---------------------------------------------------------------- quantiser
// max of two values; a NaN wins
__device__ __forceinline__ float max_or_nan(float a, float b) { return a != a ? a : b != b ? b : fmaxf(a, b); }

// A warp takes 128 columns of a row, four a lane; a group is 8, 16 or 32 lanes.
template <typename TW, typename TS>
__global__ void __launch_bounds__(kThreads) q4_quantize_kernel(const TW* W, int64_t ldw, Q4 w, uint32_t* packed,
                                                               TS* scales, uint8_t* zeros) {
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const int64_t unit = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  if (unit >= w.n * w.slabs) return;
  const int64_t row = unit / w.slabs;
  const int slab = (int)(unit - row * w.slabs), col = slab * 128 + lane * 4;
  float v[4], hi = 0.f, lo = 0.f;  // lo: -min(w, 0)
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[j] = col + j < w.k ? io<TW>::ld(W + row * ldw + col + j) : 0.f;
    hi = max_or_nan(hi, v[j]);
    lo = max_or_nan(lo, -v[j]);
  }
  const int span = 1 << (w.group_log - 2);  // lanes of a group
  for (int o = span >> 1; o > 0; o >>= 1) {
    hi = max_or_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    lo = max_or_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
  }
  const bool asym = zeros != nullptr;
  TS st;
  io<TS>::st(&st, asym ? (hi + lo) / 15.f : max_or_nan(hi, lo) / 7.f);
  const float s = io<TS>::ld(&st), div = s == 0.f ? 1.f : s;
  const float z = asym ? fminf(fmaxf(rintf(lo / div), 0.f), 15.f) : 8.f;
  uint32_t q = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) q |= (uint32_t)fminf(fmaxf(rintf(v[j] / div) + z, 0.f), 15.f) << (4 * j);
  const uint32_t other = __shfl_down_sync(0xffffffffu, q, 1);
  if ((lane & 1) == 0) {
    const int64_t at = row * w.slabs * 16 + column_word(col >> 3);
    if (ACID_IN_BOUNDS(kSiteQ4, at, w.n * w.slabs * 16)) packed[at] = q | other << 16;
  }
  if ((lane & (span - 1)) == 0 && col < w.k) {
    const int64_t at = row * w.groups + (col >> w.group_log);
    if (ACID_IN_BOUNDS(kSiteQ4, at, w.n * w.groups)) {
      scales[at] = st;
      if (asym) zeros[at] = (uint8_t)z;
    }
  }
}

template <typename TS, typename TO>
__global__ void __launch_bounds__(kThreads) q4_dequantize_kernel(Q4 w, TO* out, int64_t ldo, bool wide) {
  pdl_wait();
  const int octets = (w.k + 7) / 8;
  const int64_t unit = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (unit >= w.n * octets) return;
  const int64_t row = unit / octets;
  const int o = (int)(unit - row * octets), col = o * 8;
  const uint32_t word = word_at(w, row, column_word(o));
  const float s = scale_at<TS>(w, row, col);
  const int z = zero_at(w, row, col);
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = s * (float)((int)(word >> (4 * j) & 15u) - z);
  TO* p = out + row * ldo + col;
  if (wide && col + 8 <= w.k) {
    store8(p, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (col + j < w.k) io<TO>::st(p + j, v[j]);
  }
}

// --------------------------------------------------------------------- host
bool known_dtype(int t) { return t == ACID_BF16 || t == ACID_FP32; }

constexpr int64_t kMostRows = 32768;  // of x in one call (grid limits)

acid_status check_weight(const acid_q4_weight* w) {
  ACID_REQUIRE(w != nullptr, ACID_ERR_INVALID_ARG, "q4: null weight");
  ACID_REQUIRE(w->n >= 1 && w->n < (int64_t(1) << 31) && w->k >= 1 && w->k <= 65536, ACID_ERR_INVALID_ARG,
               "q4: need 1 <= n < 2^31 and 1 <= k <= 65536");
  ACID_REQUIRE(w->n * ((w->k + 127) / 128) <= (int64_t(1) << 32), ACID_ERR_UNSUPPORTED, "q4: weight too large");
  ACID_REQUIRE(w->group == 32 || w->group == 64 || w->group == 128, ACID_ERR_UNSUPPORTED,
               "q4: group must be 32, 64 or 128");
  ACID_REQUIRE(known_dtype(w->scale_dtype), ACID_ERR_INVALID_ARG, "q4: unknown scale dtype");
  return ACID_OK;
}
acid_status check_pointers(const acid_q4_weight& w) {
  ACID_REQUIRE(w.packed != nullptr && w.scales != nullptr, ACID_ERR_INVALID_ARG, "q4: null weight pointer");
  ACID_REQUIRE(aligned(w.packed, 16) && aligned(w.scales, w.scale_dtype == ACID_BF16 ? 2 : 4), ACID_ERR_UNSUPPORTED,
               "q4: packed must be 16-byte aligned, scales aligned to their type");
  return ACID_OK;
}
acid_status check_matrix(int dtype, const void* p, int64_t ld, int64_t cols, const char* name) {
  ACID_REQUIRE(known_dtype(dtype), ACID_ERR_INVALID_ARG, std::string("q4: unknown dtype of ") + name);
  ACID_REQUIRE(p != nullptr, ACID_ERR_INVALID_ARG, std::string("q4: ") + name + " is null");
  ACID_REQUIRE(aligned(p, dtype == ACID_BF16 ? 2 : 4), ACID_ERR_UNSUPPORTED,
               std::string("q4: ") + name + " must be aligned to its type");
  ACID_REQUIRE(ld >= cols, ACID_ERR_INVALID_ARG, std::string("q4: row stride of ") + name + " smaller than the row");
  return ACID_OK;
}

Q4 q4_args(const acid_q4_weight& w) {
  const int log = w.group == 32 ? 5 : w.group == 64 ? 6 : 7;
  return {static_cast<const uint32_t*>(w.packed), w.scales, w.zeros, w.n, w.k, (w.k + 127) / 128, log,
          (w.k + w.group - 1) >> log};
}

int bwd_splits(int64_t n) { return (int)std::min<int64_t>(64, (n + 63) / 64); }
size_t bwd_part_bytes(const acid_q4_weight& w, int64_t m) {
  return (size_t)bwd_splits(w.n) * m * ((w.k + 127) / 128 * 128) * sizeof(float);
}

}  // namespace
}  // namespace acid

using namespace acid;

extern "C" acid_status acid_q4_row_bytes(int32_t k, size_t* bytes) {
  clear_error();
  ACID_REQUIRE(bytes != nullptr && k >= 1 && k <= 65536, ACID_ERR_INVALID_ARG, "acid_q4_row_bytes: bad argument");
  *bytes = (size_t)(k + 127) / 128 * 64;
  return ACID_OK;
}

extern "C" acid_status acid_q4_quantize(int32_t w_dtype, const void* W, int64_t ldw, const acid_q4_weight* weight,
                                        acid_stream_t stream) {
  clear_error();
  ACID_TRY(check_weight(weight));
  ACID_TRY(check_pointers(*weight));
  ACID_TRY(check_matrix(w_dtype, W, ldw, weight->k, "W"));
  cudaStream_t s = (cudaStream_t)stream;
  const Q4 w = q4_args(*weight);
  const unsigned grid = (unsigned)((w.n * w.slabs + kThreads / 32 - 1) / (kThreads / 32));
  auto packed = static_cast<uint32_t*>(const_cast<void*>(weight->packed));
  auto scales = const_cast<void*>(weight->scales);
  auto zeros = const_cast<uint8_t*>(weight->zeros);
  auto launch = [&](auto* src, auto* sc) {
    launch_pdl(q4_quantize_kernel<std::remove_const_t<std::remove_pointer_t<decltype(src)>>,
                                  std::remove_pointer_t<decltype(sc)>>,
               grid, kThreads, 0, s, src, ldw, w, packed, sc, zeros);
  };
  auto by_scale = [&](auto* src) {
    if (weight->scale_dtype == ACID_BF16)
      launch(src, static_cast<bf16*>(scales));
    else
      launch(src, static_cast<float*>(scales));
  };
  if (w_dtype == ACID_BF16)
    by_scale(static_cast<const bf16*>(W));
  else
    by_scale(static_cast<const float*>(W));
  ACID_CHECK_LAUNCH();
  return ACID_OK;
}

extern "C" acid_status acid_q4_dequantize(const acid_q4_weight* weight, int32_t out_dtype, void* out, int64_t ldo,
                                          acid_stream_t stream) {
  clear_error();
  ACID_TRY(check_weight(weight));
  ACID_TRY(check_pointers(*weight));
  ACID_TRY(check_matrix(out_dtype, out, ldo, weight->k, "out"));
  cudaStream_t s = (cudaStream_t)stream;
  const Q4 w = q4_args(*weight);
  const unsigned grid = (unsigned)((w.n * ((w.k + 7) / 8) + kThreads - 1) / kThreads);
  const bool wide = aligned(out, 16) && ldo % 8 == 0;
  const bool h = weight->scale_dtype == ACID_BF16;
  if (out_dtype == ACID_BF16)
    launch_pdl(h ? q4_dequantize_kernel<bf16, bf16> : q4_dequantize_kernel<float, bf16>, grid, kThreads, 0, s, w,
               static_cast<bf16*>(out), ldo, wide);
  else
    launch_pdl(h ? q4_dequantize_kernel<bf16, float> : q4_dequantize_kernel<float, float>, grid, kThreads, 0, s, w,
               static_cast<float*>(out), ldo, wide);
  ACID_CHECK_LAUNCH();
  return ACID_OK;
}

extern "C" acid_status acid_q4_linear_forward(int32_t x_dtype, const void* x, int64_t ldx, int64_t M,
                                              const acid_q4_weight* weight, const float* bias, int32_t silu_input,
                                              int32_t out_dtype, void* out, int64_t ldo, acid_stream_t stream) {
  clear_error();
  ACID_TRY(check_weight(weight));
  ACID_REQUIRE(M >= 0 && M <= kMostRows, ACID_ERR_INVALID_ARG, "acid_q4_linear_forward: need 0 <= M <= 32768");
  if (M == 0) return ACID_OK;
  ACID_TRY(check_pointers(*weight));
  ACID_TRY(check_matrix(x_dtype, x, ldx, weight->k, "x"));
  ACID_TRY(check_matrix(out_dtype, out, ldo, weight->n, "out"));
  ACID_REQUIRE(aligned(bias, 4), ACID_ERR_UNSUPPORTED, "acid_q4_linear_forward: bias must be 4-byte aligned");
  const Fwd a{q4_args(*weight), x, ldx, M, x_dtype, silu_input != 0, out_dtype, bias, out, ldo};
  const dim3 grid((unsigned)((a.w.n + kThreads / 32 - 1) / (kThreads / 32)), (unsigned)((M + kRows - 1) / kRows));
  launch_pdl(weight->scale_dtype == ACID_BF16 ? q4_forward_kernel<bf16> : q4_forward_kernel<float>, grid, kThreads, 0,
             (cudaStream_t)stream, a);
  ACID_CHECK_LAUNCH();
  return ACID_OK;
}

extern "C" acid_status acid_q4_linear_workspace_size(const acid_q4_weight* weight, int64_t M, size_t* bytes) {
  clear_error();
  ACID_TRY(check_weight(weight));
  ACID_REQUIRE(bytes != nullptr && M >= 0 && M <= kMostRows, ACID_ERR_INVALID_ARG,
               "acid_q4_linear_workspace_size: bad argument");
  *bytes = std::max<size_t>(16, bwd_part_bytes(*weight, M));
  return ACID_OK;
}

extern "C" acid_status acid_q4_linear_backward(int32_t g_dtype, const void* g, int64_t ldg, int64_t M,
                                               const acid_q4_weight* weight, int32_t x_dtype, const void* x,
                                               int64_t ldx, int32_t silu_input, void* dx, int64_t lddx, float* dbias,
                                               void* ws, size_t ws_bytes, acid_stream_t stream) {
  clear_error();
  ACID_TRY(check_weight(weight));
  ACID_REQUIRE(M >= 0 && M <= kMostRows, ACID_ERR_INVALID_ARG, "acid_q4_linear_backward: need 0 <= M <= 32768");
  ACID_REQUIRE(dx != nullptr || dbias != nullptr, ACID_ERR_INVALID_ARG, "acid_q4_linear_backward: need dx or dbias");
  ACID_REQUIRE(aligned(dbias, 4), ACID_ERR_UNSUPPORTED, "acid_q4_linear_backward: dbias must be 4-byte aligned");
  cudaStream_t s = (cudaStream_t)stream;
  if (M == 0) {
    if (dbias) ACID_CUDA(cudaMemsetAsync(dbias, 0, weight->n * sizeof(float), s));
    return ACID_OK;
  }
  ACID_TRY(check_matrix(g_dtype, g, ldg, weight->n, "g"));
  if (dx != nullptr) {
    ACID_TRY(check_pointers(*weight));
    ACID_TRY(check_matrix(x_dtype, dx, lddx, weight->k, "dx"));
    if (silu_input) ACID_TRY(check_matrix(x_dtype, x, ldx, weight->k, "x"));
    ACID_REQUIRE(ws != nullptr && aligned(ws, 16), ACID_ERR_WORKSPACE,
                 "acid_q4_linear_backward: workspace null or not 16-byte aligned");
    const size_t need = bwd_part_bytes(*weight, M);
    ACID_REQUIRE(ws_bytes >= need, ACID_ERR_WORKSPACE,
                 "acid_q4_linear_backward: workspace too small (need " + std::to_string(need) + ")");
  }
  const Bwd a{q4_args(*weight), g, x, ldg, ldx, M, g_dtype, x_dtype, silu_input != 0, dx, lddx, dbias,
              static_cast<float*>(ws), bwd_splits(weight->n)};
  if (dx != nullptr) {
    const dim3 grid((a.w.slabs * 16 + kThreads - 1) / kThreads, a.splits, (unsigned)((M + kRows - 1) / kRows));
    launch_pdl(weight->scale_dtype == ACID_BF16 ? q4_backward_kernel<bf16> : q4_backward_kernel<float>, grid, kThreads,
               0, s, a);
    ACID_CHECK_LAUNCH();
    launch_pdl(q4_backward_join_kernel, dim3((a.w.k + kThreads - 1) / kThreads, (unsigned)M), kThreads, 0, s, a);
    ACID_CHECK_LAUNCH();
  }
  if (dbias != nullptr) {
    launch_pdl(q4_bias_kernel, (unsigned)((a.w.n + kThreads - 1) / kThreads), kThreads, 0, s, a);
    ACID_CHECK_LAUNCH();
  }
  return ACID_OK;
}
