// 4-bit weights as the kernels see them, and what the units that use them share.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"
#include "internal.h"

namespace acid {

// A weight as the kernels see it.
struct Q4 {
  const uint32_t* packed;  // [n][16 slabs] words
  const void* scales;
  const uint8_t* zeros;
  int64_t n;
  int k, slabs, group_log, groups;  // group = 1 << group_log columns; groups = ceil(k / group)
};

__device__ __forceinline__ float value_at(int dtype, const void* p, int64_t i) {
  return dtype == ACID_BF16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]) : static_cast<const float*>(p)[i];
}
__device__ __forceinline__ void put_value(int dtype, void* p, int64_t i, float v) {
  if (dtype == ACID_BF16)
    static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
  else
    static_cast<float*>(p)[i] = v;
}
template <typename H2>
__device__ __forceinline__ uint32_t bits(H2 h) {
  return *reinterpret_cast<uint32_t*>(&h);
}
__device__ __forceinline__ __half2 half2_of(uint32_t u) { return *reinterpret_cast<__half2*>(&u); }

// The product's operands.  The activated input enters as two halves, high and
// low part, after a power of two that brings the largest value of each row (a few
// rows: of each 128 columns of it) to 2^13 .. 2^14: together 22 bits of that value, and of
// any down to 2^-16 of it.
struct Q4Fwd {
  Q4 w;
  const void* x;
  int64_t ldx, m;
  int x_dtype, silu, out_dtype;
  const float* bias;
  void* out;
  int64_t ldo;
  uint8_t* parts;  // past a few rows: the parts as the tensor cores read them
  float* back;     // [m], and the powers of two taken back
  int kw;          // few rows: warps of a CTA that share a row's columns
};
// The power of two that brings `top` to 2^13 .. 2^14 (2^127 at most).
__device__ __forceinline__ float up_to_half(float top) {
  return __uint_as_float(min(267u - (__float_as_uint(top) >> 23), 254u) << 23);
}
// The activated octet's eight values; returns their largest (finite) magnitude.
__device__ __forceinline__ float octet_values(const Q4Fwd& a, int64_t m, int col, float (&v)[8]) {
  float top = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    v[j] = 0.f;
    if (m < a.m && col + j < a.w.k) {
      v[j] = value_at(a.x_dtype, a.x, m * a.ldx + col + j);
      if (a.silu) v[j] = silu(v[j]);
    }
    if (isfinite(v[j])) top = fmaxf(top, fabsf(v[j]));
  }
  return top;
}
// High and low parts of an octet, columns j and j + 4 to a register.
__device__ __forceinline__ void split_octet(const float (&v)[8], float by, uint4& hi, uint4& lo) {
  uint32_t h[4], l[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float x = v[j] * by, y = v[j + 4] * by;
    const __half2 p = __floats2half2_rn(x, y);
    const float2 f = __half22float2(p);
    h[j] = bits(p);
    // nothing is left of an infinity or a NaN
    l[j] = bits(__floats2half2_rn(isfinite(f.x) ? x - f.x : 0.f, isfinite(f.y) ? y - f.y : 0.f));
  }
  hi = make_uint4(h[0], h[1], h[2], h[3]);
  lo = make_uint4(l[0], l[1], l[2], l[3]);
}
// The four pairs (columns j and j + 4) of a word as halves q - z; z1 = 1024 + z and
// z64 = 64 + z in both halves.  A code in the low bits of the half 1024 (or in
// the next four bits, worth 16) is read without a conversion.
__device__ __forceinline__ void halves_of(uint32_t w, uint32_t z1, uint32_t z64, uint32_t (&d)[4]) {
  const __half2 sixteenth = __float2half2_rn(0.0625f);
  const uint32_t v = w >> 8;
  d[0] = bits(__hsub2(half2_of((w & 0x000f000fu) | 0x64006400u), half2_of(z1)));
  d[1] = bits(__hfma2(half2_of((w & 0x00f000f0u) | 0x64006400u), sixteenth, __hneg2(half2_of(z64))));
  d[2] = bits(__hsub2(half2_of((v & 0x000f000fu) | 0x64006400u), half2_of(z1)));
  d[3] = bits(__hfma2(half2_of((v & 0x00f000f0u) | 0x64006400u), sixteenth, __hneg2(half2_of(z64))));
}
// The same for zero point z (0 .. 15).
__device__ __forceinline__ void halves_of(uint32_t w, uint32_t z, uint32_t (&d)[4]) {
  const uint32_t both = z * 0x00010001u;
  halves_of(w, 0x64006400u | both, 0x54005400u | both << 4, d);
}

// The input gradient's operands.
struct Q4Bwd {
  Q4 w;
  const void *g, *x;
  int64_t ldg, ldx, m;
  int g_dtype, x_dtype, scale_dtype, silu;
  void* dx;
  int64_t lddx;
  float* dbias;
  // of the call's workspace
  float* part;     // [shares][m][128 slabs]: sums, joined in their order
  uint8_t* parts;  // g as the tensor cores read it
  float* back;     // [shares / 2][m]: the powers of two taken back; negative: g has values there that are not finite
  uint32_t* top;   // largest scales
  int shares;
  int64_t per;     // rows of the weight to a CTA
};
constexpr int kQ4Chunk = 64;  // rows of x that a kernel of many rows takes at a time

// q4_rows.cu: tcgen05 kernels.
size_t q4_rows_forward_bytes(const Q4& w, int64_t m);
acid_status q4_rows_forward(Q4Fwd a, void* workspace, int scale_dtype, cudaStream_t s);
size_t q4_backward_bytes(const Q4& w, int64_t m);
acid_status q4_backward(Q4Bwd a, void* workspace, cudaStream_t s);

}  // namespace acid
