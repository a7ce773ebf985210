// Modulation projections with 4-bit weights: quantiser, values, product and
// input gradient (acid_q4_*).
#include <algorithm>
#include <string>

#define ACID_UNIT_WITHOUT_WAITS
#include <cuda_fp16.h>

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

// D += A B of one 16 x 8 x 16 tile of the warp-wide tensor instruction.  Lane
// 4 g + t holds of A the rows g, g + 8 and the columns 2 t, 2 t + 1 (a0, a1) and
// 2 t + 8, 2 t + 9 (a2, a3), of B the same columns (as its rows) of column g, and
// of D the rows g (d0, d1) and g + 8 (d2, d3) of the columns 2 t, 2 t + 1.  A
// contraction index is a name only: both operands may take any order of it.
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same from zero: D = A B.
__device__ __forceinline__ void mma_f16_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                              uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <typename H2>
__device__ __forceinline__ uint32_t bits(H2 h) {
  return *reinterpret_cast<uint32_t*>(&h);
}
__device__ __forceinline__ __half2 half2_of(uint32_t u) { return *reinterpret_cast<__half2*>(&u); }
__device__ __forceinline__ __nv_bfloat162 bf162_of(uint32_t u) { return *reinterpret_cast<__nv_bfloat162*>(&u); }

__device__ __forceinline__ uint4 load_stream(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

// ------------------------------------------------------------------ product
// out^T = W a(x)^T on the tensor cores, the codes as the exact halves q - z
// (16 rows of the weight to a tile) against the rows of a(x), 8 to a tile.  a(x)
// enters as two halves, high and low part, after a power of two that brings
// the largest value of each 128 columns of a row to 2^13 .. 2^14: together 22 bits
// of it.  Products are exact, a group's sum is formed by the tensor cores in
// fp32 and multiplied by the group's scale in fp32.
// Up to kPackedRows rows: the parts of row m are columns 2 m and 2 m + 1 of one
// tile, prepared by each CTA in its shared memory.  More rows: q4_parts_kernel
// prepares them once, in the order in which the lanes read them.
struct Fwd {
  Q4 w;
  const void* x;
  int64_t ldx, m;
  int x_dtype, silu, out_dtype;
  const float* bias;
  void* out;
  int64_t ldo;
  uint4* parts;  // [chunks of 64 rows][slab][4 words][2 parts][8 NT columns][4 lanes]
  float* back;   // [m][slabs]: the powers of two taken back
  int kw;        // warps of a CTA that share a row's columns
};
constexpr int kPackedRows = 4, kChunk = 64;

// The activated octet's eight values and the factor of their slab; 16 lanes in a
// row hold a slab's octets.
__device__ __forceinline__ float octet_of(const Fwd& a, int64_t m, int col, float (&v)[8]) {
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
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  return __uint_as_float(min(267u - (__float_as_uint(top) >> 23), 254u) << 23);
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

template <int NT>
__global__ void __launch_bounds__(kThreads) q4_parts_kernel(Fwd a) {
  pdl_wait();
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int per_row = a.w.slabs * 16;
  const int64_t m = i / per_row;
  const int o = (int)(i - m * per_row), slab = o >> 4;
  float v[8];
  const float by = octet_of(a, m, o * 8, v);
  if (m >= a.m) return;
  uint4 hi, lo;
  split_octet(v, by, hi, lo);
  const int64_t chunk = m / kChunk;
  const int n = (int)(m - chunk * kChunk), word = (o >> 2) & 3, t = o & 3;
  uint4* p = a.parts + (((chunk * a.w.slabs + slab) * 4 + word) * 2 * NT * 8 + n) * 4 + t;
  p[0] = hi;
  p[NT * 8 * 4] = lo;
  if ((o & 15) == 0) a.back[m * a.w.slabs + slab] = 1.f / by;
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

// The four pairs of a word as halves q - 8: what halves_of gives without a zero
// point, which the few-rows kernel takes into account by the sum of a(x) over
// the group, sum x (q - z) = sum x (q - 8) + (8 - z) sum x.
__device__ __forceinline__ void halves_of(uint32_t w, uint32_t (&d)[4]) { halves_of(w, 0x64086408u, 0x54805480u, d); }

// Where a warp reads its row tile: 32 rows g, g + 8, g + 16, g + 24 of a lane, rows
// past the end as the last one.
struct TileRows {
  const uint4* q[4];
  int64_t s[4];
};
__device__ __forceinline__ TileRows tile_rows(const Q4& w, int64_t tile, int g, int t) {
  TileRows r;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int64_t row = min(tile * 32 + g + 8 * q, w.n - 1);
    r.q[q] = reinterpret_cast<const uint4*>(w.packed) + row * w.slabs * 4 + t;
    r.s[q] = row * w.groups;
  }
  return r;
}

// A few rows: a CTA's warps split a row tile's slabs among kw of them, and 8 / kw
// row tiles are neighbours.  A lane reads 16 bytes of four rows: word i of them
// holds its columns of the slab's 32 columns i, so that four lanes' words make a
// tile's step of 16 columns twice.
template <typename TS, bool ZEROS>
__global__ void __launch_bounds__(kThreads, 2) q4_few_kernel(Fwd a) {
  extern __shared__ __align__(16) uint8_t smem[];
  const Q4& w = a.w;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, warp = warp_index();
  const int kw = a.kw, rw = kThreads / 32 / kw, kwarp = warp % kw, rwarp = warp / kw;
  const int rows = (int)a.m, cols = 2 * rows;
  uint4* frag = reinterpret_cast<uint4*>(smem);                                   // [slab][word][column][t]
  float* back = reinterpret_cast<float*>(smem + (size_t)w.slabs * 16 * cols * 16);  // [slab][row]
  float* xsum = back + w.slabs * kPackedRows;                                     // [slab][32 columns][row]
  float* red = xsum + (ZEROS ? 4 * w.slabs * kPackedRows : 0);                    // [8 warps][row][33]
  const int64_t tiles = (w.n + 31) / 32, sets = (tiles + rw - 1) / rw;
  const int mine = (w.slabs - kwarp + kw - 1) / kw;  // slabs of this warp
  const int per_slab = 128 >> w.group_log, lane_group = t >> (w.group_log - 5);
  struct Load {
    uint4 q[4];
    float s[4];
    uint8_t z[4];
  };
  pdl_wait();
  // this warp's steps (row set, slab), two fetched ahead
  int64_t set = blockIdx.x, fset = set;
  int k = 0, fslab = kwarp;
  TileRows at = tile_rows(w, fset * rw + rwarp, g, t);
  auto next = [&](Load& l) {
    if (fset < sets) {
      const int group = min(fslab * per_slab + lane_group, w.groups - 1);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint4* p = at.q[q] + fslab * 4;
        if (ACID_IN_BOUNDS(kSiteQ4, (p - reinterpret_cast<const uint4*>(w.packed)) * 4 + 3, w.n * w.slabs * 16))
          l.q[q] = load_stream(p);
        if (ACID_IN_BOUNDS(kSiteQ4, at.s[q] + group, w.n * w.groups)) {
          l.s[q] = io<TS>::ld(static_cast<const TS*>(w.scales) + at.s[q] + group);
          if constexpr (ZEROS) l.z[q] = w.zeros[at.s[q] + group];
        }
      }
    }
    fslab += kw;
    if (fslab >= w.slabs) {
      fslab = kwarp;
      fset += gridDim.x;
      if (fset < sets) at = tile_rows(w, fset * rw + rwarp, g, t);
    }
  };
  Load l[2];
  next(l[0]);
  next(l[1]);
  // a(x) in parts, while the first weights are on their way
  {
    const int per_row = w.slabs * 16, all = per_row * rows;
    for (int base = threadIdx.x & ~31; base < all; base += kThreads) {
      const int i = base + lane, m = i / per_row, o = i - m * per_row;
      float v[8];
      const float by = octet_of(a, m, o * 8, v);
      float sum = 0.f;
      if constexpr (ZEROS) {
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += v[j];
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      }
      if (m >= rows) continue;
      uint4 hi, lo;
      split_octet(v, by, hi, lo);
      uint4* p = frag + ((o >> 2) * cols + 2 * m) * 4 + (o & 3);
      p[0] = hi;
      p[4] = lo;
      if ((o & 15) == 0) back[(o >> 4) * kPackedRows + m] = 1.f / by;
      if (ZEROS && (o & 3) == 0) xsum[(o >> 2) * kPackedRows + m] = sum;
    }
    __syncthreads();
  }
  float sum[2][2];  // row t of the input, rows g + 8 h + 16 r of the tile
  auto clear = [&] { sum[0][0] = sum[0][1] = sum[1][0] = sum[1][1] = 0.f; };
  const uint4* mine_b = frag + (g < cols ? g * 4 + t : 0);
  auto compute = [&](const Load& l, int slab) {
    const float bk = back[slab * kPackedRows + t];
    float acc[2][4], xs = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint4 b = mine_b[(slab * 4 + i) * cols * 4];
      if (g >= cols) b = make_uint4(0, 0, 0, 0);
      const bool first = (i << 5 & ((1 << w.group_log) - 1)) == 0;
      if (ZEROS) xs = (first ? 0.f : xs) + xsum[(slab * 4 + i) * kPackedRows + t];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        uint32_t d[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint4& v = l.q[2 * r + h];
          halves_of(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w, d[h]);
        }
        if (first)
          mma_f16_first(acc[r], d[0][0], d[1][0], d[0][1], d[1][1], b.x, b.y);
        else
          mma_f16(acc[r], d[0][0], d[1][0], d[0][1], d[1][1], b.x, b.y);
        mma_f16(acc[r], d[0][2], d[1][2], d[0][3], d[1][3], b.z, b.w);
      }
      if (((i + 1) << 5 & ((1 << w.group_log) - 1)) == 0) {  // the group ends
        const int from = (lane & ~3) | (i >> (w.group_log - 5) << (w.group_log - 5));  // a lane that has its scale
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int q = 2 * r + h;
            const float s = __shfl_sync(0xffffffffu, l.s[q], from);
            float v = (acc[r][2 * h] + acc[r][2 * h + 1]) * bk;  // both parts of row t are in this lane
            if constexpr (ZEROS)
              v = fmaf((float)(8 - (int)__shfl_sync(0xffffffffu, (uint32_t)l.z[q], from)), xs, v);
            sum[r][h] = fmaf(s, v, sum[r][h]);
          }
      }
    }
  };
  auto put = [&](int64_t row, int m, float v) {
    if (row < w.n && m < rows)
      put_value(a.out_dtype, a.out, m * a.ldo + row, v + (a.bias != nullptr ? a.bias[row] : 0.f));
  };
  auto finish = [&] {
    if (kw == 1) {
#pragma unroll
      for (int q = 0; q < 4; ++q) put((set * rw + rwarp) * 32 + 8 * q + g, t, sum[q >> 1][q & 1]);
      return;
    }
    __syncthreads();  // the buffer's last readers are done
#pragma unroll
    for (int q = 0; q < 4; ++q) red[(warp * kPackedRows + t) * 33 + 8 * q + g] = sum[q >> 1][q & 1];
    __syncthreads();
    for (int i = threadIdx.x; i < rw * rows * 32; i += kThreads) {
      const int row = i & 31, m = (i >> 5) % rows, rt = (i >> 5) / rows;
      float v = 0.f;
      for (int j = 0; j < kw; ++j) v += red[((rt * kw + j) * kPackedRows + m) * 33 + row];
      put((set * rw + rt) * 32 + row, m, v);
    }
  };
  clear();
  auto step = [&](Load& cur) {
    if (set >= sets) return;
    compute(cur, kwarp + k * kw);
    next(cur);
    if (++k == mine) {
      finish();
      clear();
      k = 0;
      set += gridDim.x;
    }
  };
  while (set < sets) {
    step(l[0]);
    step(l[1]);
  }
}

// More rows: the same tiles of the weight against 8 NT columns of parts.
template <int NT, typename TS>
__global__ void __launch_bounds__(kThreads, NT <= 2 ? 2 : 1) q4_forward_kernel(Fwd a) {
  extern __shared__ __align__(16) uint8_t smem[];
  pdl_wait();
  const Q4& w = a.w;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, warp = warp_index();
  const int kw = a.kw, rw = kThreads / 32 / kw, kwarp = warp % kw, rwarp = warp / kw;
  const int64_t chunk = blockIdx.y, m0 = chunk * kChunk;
  constexpr int kCols = NT * 8;
  float* red = reinterpret_cast<float*>(smem);  // [8 warps][column][33]: sums of the warps that share rows

  const int64_t tiles = (w.n + 31) / 32, sets = (tiles + rw - 1) / rw;
  const int mine = (w.slabs - kwarp + kw - 1) / kw;  // slabs of this warp
  struct Load {
    uint4 q[4];
    float s[4];
    uint32_t z[4];
  };
  const int per_slab = 128 >> w.group_log, lane_group = t >> (w.group_log - 5);
  auto fetch = [&](Load& l, int64_t set, int slab) {
    const int64_t row0 = (set * rw + rwarp) * 32 + g;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t row = min(row0 + 8 * q, w.n - 1);
      const int64_t at = row * w.slabs + slab;
      if (ACID_IN_BOUNDS(kSiteQ4, at, w.n * w.slabs)) l.q[q] = load_stream(reinterpret_cast<const uint4*>(w.packed) + at * 4 + t);
      const int64_t i = row * w.groups + min(slab * per_slab + lane_group, w.groups - 1);
      if (ACID_IN_BOUNDS(kSiteQ4, i, w.n * w.groups)) {
        l.s[q] = io<TS>::ld(static_cast<const TS*>(w.scales) + i);
        l.z[q] = w.zeros != nullptr ? w.zeros[i] : 8u;
      }
    }
  };
  float acc[2][NT][4], sum[2][NT][4];
  auto compute = [&](const Load& l, int slab) {
    float bk[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        bk[n][e] = m0 + 8 * n + 2 * t + e < a.m ? a.back[(m0 + 8 * n + 2 * t + e) * w.slabs + slab] : 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int from = (lane & ~3) | (i >> (w.group_log - 5) << (w.group_log - 5));  // a lane that has the group's scale
      uint32_t d[4][4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t z = w.zeros != nullptr ? __shfl_sync(0xffffffffu, l.z[q], from) * 0x00010001u : 0x00080008u;
        const uint32_t word = i == 0 ? l.q[q].x : i == 1 ? l.q[q].y : i == 2 ? l.q[q].z : l.q[q].w;
        halves_of(word, 0x64006400u | z, 0x54005400u | z << 4, d[q]);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const uint4* p = a.parts + (((chunk * w.slabs + slab) * 4 + i) * 2 * NT * 8 + n * 8 + g) * 4 + t;
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          const uint4 b = p[part * NT * 8 * 4];
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            mma_f16(acc[r][n], d[2 * r][0], d[2 * r + 1][0], d[2 * r][1], d[2 * r + 1][1], b.x, b.y);
            mma_f16(acc[r][n], d[2 * r][2], d[2 * r + 1][2], d[2 * r][3], d[2 * r + 1][3], b.z, b.w);
          }
        }
      }
      if (((i + 1) << 5 & ((1 << w.group_log) - 1)) == 0) {  // the group ends
        float sc[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) sc[q] = __shfl_sync(0xffffffffu, l.s[q], from);
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              sum[r][n][e] = fmaf(sc[2 * r + (e >> 1)], acc[r][n][e] * bk[n][e & 1], sum[r][n][e]);
              acc[r][n][e] = 0.f;
            }
      }
    }
  };
  auto put = [&](int64_t row, int m, float v) {
    if (row < w.n && m0 + m < a.m)
      put_value(a.out_dtype, a.out, (m0 + m) * a.ldo + row, v + (a.bias != nullptr ? a.bias[row] : 0.f));
  };
  auto each = [&](auto&& f) {  // f(sum, row of the tile, column)
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) f(sum[r][n][e], 16 * r + 8 * (e >> 1) + g, 8 * n + 2 * t + (e & 1));
  };
  auto finish = [&](int64_t set) {
    const int64_t row0 = (set * rw + rwarp) * 32;
    if (kw == 1) {
      each([&](float v, int row, int m) { put(row0 + row, m, v); });
      return;
    }
    __syncthreads();  // the buffer's last readers are done
    each([&](float v, int row, int m) { red[(warp * kCols + m) * 33 + row] = v; });
    __syncthreads();
    for (int i = threadIdx.x; i < rw * kCols * 32; i += kThreads) {
      const int row = i & 31, m = (i >> 5) % kCols, rt = (i >> 5) / kCols;
      float v = 0.f;
      for (int k = 0; k < kw; ++k) v += red[((rt * kw + k) * kCols + m) * 33 + row];
      put((set * rw + rt) * 32 + row, m, v);
    }
  };
  auto clear = [&] {
#pragma unroll
    for (int r = 0; r < 2; ++r)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[r][n][e] = sum[r][n][e] = 0.f;
  };
  // this warp's steps (row set, slab), two fetched ahead
  int64_t set = blockIdx.x, fset = set;
  int k = 0, fk = 0;
  auto advance = [&](int64_t& st, int& i) {
    if (++i == mine) {
      i = 0;
      st += gridDim.x;
    }
  };
  Load l[2];
  auto next = [&](Load& into) {
    if (fset < sets) fetch(into, fset, kwarp + fk * kw);
    advance(fset, fk);
  };
  next(l[0]);
  next(l[1]);
  clear();
  auto step = [&](Load& cur) {
    if (set >= sets) return;
    compute(cur, kwarp + k * kw);
    next(cur);
    if (k == mine - 1) {
      finish(set);
      clear();
    }
    advance(set, k);
  };
  while (set < sets) {
    step(l[0]);
    step(l[1]);
  }
}

// ----------------------------------------------------------- input gradient
// dx^T = W^T g^T on the tensor cores: tiles of 16 columns of the weight by 16 of
// its rows, the codes as the exact bf16 values q - z, against 8 columns of
// (g s)^T, whose fp32 values enter as three bf16 parts (24 bits).  A CTA takes one
// slab of columns and a share of the rows, and leaves its sums for the join.
struct Bwd {
  Q4 w;
  const void *g, *x;
  int64_t ldg, ldx, m;
  int g_dtype, x_dtype, scale_dtype, silu;
  void* dx;
  int64_t lddx;
  float* dbias;
  float* part;   // [splits][m][128 slabs]
  int splits;
  int64_t per;   // rows of the weight to a CTA, a multiple of 16
};
constexpr int kBwdPackedRows = 2;  // three parts of two rows fit eight columns
// rows of the weight whose g and scales are staged at a time
template <bool PACKED>
constexpr int kStageRows = PACKED ? 768 : 256;
template <int NT, bool PACKED>
constexpr int kStageCols = PACKED ? kBwdPackedRows : NT * 8;
constexpr int larger(int a, int b) { return a > b ? a : b; }
template <int NT, int IW, bool PACKED>
constexpr int kBwdSmem = larger((kStageCols<NT, PACKED> + 4) * kStageRows<PACKED> * 4, 2 * IW * NT * 8 * 128 * 4);
// IW words of a lane's four (32 columns each) are this warp's: 4 / IW warps share
// a block of 16 rows, and the 2 IW groups of such warps take blocks in turn.
template <int NT, int IW, bool PACKED>
__global__ void __launch_bounds__(kThreads, NT <= 2 ? 2 : 1) q4_backward_kernel(Bwd a) {
  extern __shared__ __align__(16) uint8_t smem[];
  constexpr int kShare = 4 / IW, kTurns = 2 * IW, kRows = kStageRows<PACKED>, kBlocks = kRows / 16;
  constexpr int kStaged = kStageCols<NT, PACKED>;
  pdl_wait();
  const Q4& w = a.w;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, warp = warp_index();
  const int first_word = (warp % kShare) * IW, turn = warp / kShare;
  const int slab = blockIdx.x;
  const int64_t chunk = blockIdx.z, m0 = chunk * kChunk;
  const int64_t begin = blockIdx.y * a.per, end = min(w.n, begin + a.per);
  if (a.dbias != nullptr && slab == 0 && chunk == 0)
    for (int64_t n = begin + threadIdx.x; n < end; n += kThreads) {
      float v = 0.f;
      for (int64_t m = 0; m < a.m; ++m) v += value_at(a.g_dtype, a.g, m * a.ldg + n);
      a.dbias[n] = v;
    }
  if (a.dx == nullptr) return;
  float4* gs = reinterpret_cast<float4*>(smem);           // [block][column][t]: rows 2 t, 2 t + 1, 2 t + 8, 2 t + 9
  float4* ss = gs + kBlocks * kStaged * 4;  // [block][word][t]
  float acc[IW][2][NT][4];
#pragma unroll
  for (int i = 0; i < IW; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][j][n][e] = 0.f;
  struct Load {
    uint32_t q[4][IW];
    uint32_t z[4];  // zero points of the words, a byte each
  };
  const int per_slab = 128 >> w.group_log;
  auto row_of = [&](int64_t block, int r) { return block * 16 + 2 * t + (r & 1) + (r >> 1) * 8; };
  const int64_t blocks_end = (end + 15) / 16;
  auto fetch = [&](Load& l, int64_t block) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t row = min(row_of(block, r), w.n - 1);
      const int64_t at = (row * w.slabs + slab) * 16 + 4 * (g & 3) + first_word;
      if (ACID_IN_BOUNDS(kSiteQ4, at + IW - 1, w.n * w.slabs * 16)) {
        const uint32_t* p = w.packed + at;
        if constexpr (IW == 4) {
          const uint4 v = *reinterpret_cast<const uint4*>(p);
          l.q[r][0] = v.x; l.q[r][1] = v.y; l.q[r][2] = v.z; l.q[r][3] = v.w;
        } else if constexpr (IW == 2) {
          const uint2 v = *reinterpret_cast<const uint2*>(p);
          l.q[r][0] = v.x; l.q[r][1] = v.y;
        } else {
          l.q[r][0] = *p;
        }
      }
      if (w.zeros != nullptr) {
        l.z[r] = 0;
#pragma unroll
        for (int i = 0; i < IW; ++i) {
          const int64_t z = row * w.groups + min(slab * per_slab + ((first_word + i) >> (w.group_log - 5)), w.groups - 1);
          if (ACID_IN_BOUNDS(kSiteQ4, z, w.n * w.groups)) l.z[r] |= (uint32_t)w.zeros[z] << (8 * i);
        }
      }
    }
  };
  // eight halves of a word's columns of two rows: which half the lane takes
  const uint32_t half = g < 4 ? 0x5410u : 0x7632u;
  auto compute = [&](const Load& l, int block) {
#pragma unroll
    for (int i = 0; i < IW; ++i) {
      uint32_t b[NT][3][2];
      const float4 s = ss[(block * 4 + first_word + i) * 4 + t];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (!PACKED || g < 3 * kBwdPackedRows) v = gs[(block * kStaged + (PACKED ? g / 3 : n * 8 + g)) * 4 + t];
        float f[4] = {v.x * s.x, v.y * s.y, v.z * s.z, v.w * s.w};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int part = 0; part < 3; ++part) {
            const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * h], f[2 * h + 1]);
            const float lo = __low2float(p), hi = __high2float(p);
            b[n][part][h] = bits(p);
            f[2 * h] = isfinite(lo) ? f[2 * h] - lo : 0.f;
            f[2 * h + 1] = isfinite(hi) ? f[2 * h + 1] - hi : 0.f;
          }
          if constexpr (PACKED) {  // column 3 m + part
            const int part = g % 3;
            b[n][0][h] = part == 0 ? b[n][0][h] : part == 1 ? b[n][1][h] : b[n][2][h];
          }
        }
      }
      uint32_t q01 = __byte_perm(l.q[0][i], l.q[1][i], half), q89 = __byte_perm(l.q[2][i], l.q[3][i], half);
      uint32_t z01 = 0x43084308u, z89 = 0x43084308u;  // 128 + z
      if (w.zeros != nullptr) {
        z01 = 0x43004300u | (l.z[0] >> (8 * i) & 15u) | (l.z[1] >> (8 * i) & 15u) << 16;
        z89 = 0x43004300u | (l.z[2] >> (8 * i) & 15u) | (l.z[3] >> (8 * i) & 15u) << 16;
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        uint32_t d[4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {  // the code in the low bits of the bf16 128
          d[e] = bits(__hsub2(bf162_of((q01 & 0x000f000fu) | 0x43004300u), bf162_of(z01)));
          d[2 + e] = bits(__hsub2(bf162_of((q89 & 0x000f000fu) | 0x43004300u), bf162_of(z89)));
          q01 >>= 4;
          q89 >>= 4;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int part = 0; part < (PACKED ? 1 : 3); ++part)
            mma_bf16(acc[i][j][n], d[0], d[1], d[2], d[3], b[n][part][0], b[n][part][1]);
      }
    }
  };
  constexpr int kAhead = PACKED ? 3 : IW == 4 ? 2 : 4;
  static_assert(kBlocks % (kTurns * kAhead) == 0, "a stage is a whole number of rounds of every warp's ring");
  Load l[kAhead];
  int64_t fetched = begin / 16 + turn;
#pragma unroll
  for (int k = 0; k < kAhead; ++k, fetched += kTurns)
    if (fetched < blocks_end) fetch(l[k], fetched);
  for (int64_t base = begin; base < end; base += kRows) {
    __syncthreads();
    // g and scales of the next rows; zeros past the end
    for (int i = threadIdx.x; i < kStaged * kRows; i += kThreads) {
      const int col = i / kRows, r = i % kRows;
      const int64_t n = base + r, m = m0 + col;
      const float v = n < end && m < a.m ? value_at(a.g_dtype, a.g, m * a.ldg + n) : 0.f;
      const int b = r / 16, q = r % 8 / 2, e = r % 2 + (r % 16) / 8 * 2;
      reinterpret_cast<float*>(gs + (b * kStaged + col) * 4 + q)[e] = v;
    }
    for (int i = threadIdx.x; i < 4 * kRows; i += kThreads) {
      const int word = i % 4, r = i / 4;
      const int64_t n = base + r;
      float v = 0.f;
      if (n < end) {
        const int64_t at = n * w.groups + min(slab * per_slab + (word >> (w.group_log - 5)), w.groups - 1);
        if (ACID_IN_BOUNDS(kSiteQ4, at, w.n * w.groups)) v = value_at(a.scale_dtype, w.scales, at);
      }
      const int b = r / 16, q = r % 8 / 2, e = r % 2 + (r % 16) / 8 * 2;
      reinterpret_cast<float*>(ss + (b * 4 + word) * 4 + q)[e] = v;
    }
    __syncthreads();
    const int blocks = (int)(min((int64_t)kRows, end - base) + 15) / 16;  // kAhead of them are fetched
#pragma unroll 1
    for (int k0 = turn; k0 < kBlocks; k0 += kTurns * kAhead)
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (k0 + k * kTurns < blocks) compute(l[k], k0 + k * kTurns);
        if (fetched < blocks_end) fetch(l[k], fetched);
        fetched += kTurns;
      }
  }
  // the turns' sums, then the CTA's share
  __syncthreads();
  constexpr int kCols = NT * 8;
  float* red = reinterpret_cast<float*>(smem);  // [turn][column][128]
#pragma unroll
  for (int i = 0; i < IW; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int c = 32 * (first_word + i) + 8 * (g & 3) + 4 * (g >> 2) + 2 * j;
          *reinterpret_cast<float2*>(red + (turn * kCols + n * 8 + 2 * t + e) * 128 + c) =
              make_float2(acc[i][j][n][e], acc[i][j][n][2 + e]);
        }
  __syncthreads();
  const int rows = (int)min((int64_t)(PACKED ? kBwdPackedRows : kCols), a.m - m0);
  for (int i = threadIdx.x; i < rows * 128; i += kThreads) {
    const int m = i / 128, c = i % 128;
    float v = 0.f;
    for (int u = 0; u < kTurns; ++u)
#pragma unroll
      for (int part = 0; part < (PACKED ? 3 : 1); ++part) v += red[(u * kCols + (PACKED ? 3 * m + part : m)) * 128 + c];
    const int64_t at = (blockIdx.y * a.m + m0 + m) * w.slabs * 128 + slab * 128 + c;
    if (ACID_IN_BOUNDS(kSiteQ4, at, a.splits * a.m * w.slabs * 128)) a.part[at] = v;
  }
}

// Joins the shares in their order and takes the activation's gradient.
__global__ void __launch_bounds__(kThreads) q4_backward_join_kernel(Bwd a) {
  pdl_wait();
  const int c = blockIdx.x * kThreads + threadIdx.x;
  const int64_t m = blockIdx.y, width = (int64_t)a.w.slabs * 128;
  if (c >= a.w.k) return;
  float v = 0.f;
#pragma unroll 8
  for (int b = 0; b < a.splits; ++b) v += a.part[(b * a.m + m) * width + c];
  if (a.silu) {
    const float x = value_at(a.x_dtype, a.x, m * a.ldx + c), e = 1.f / (1.f + expf(-x));
    v *= e * (1.f + x * (1.f - e));
  }
  put_value(a.x_dtype, a.dx, m * a.lddx + c, v);
}

// ---------------------------------------------------------------- quantiser
// A lane takes eight columns of a row (one word), a warp 32 such octets of one
// row at a time: two slabs, whose groups are 4, 8 or 16 lanes.
constexpr int kUnits = 4;  // octet runs of a warp, all loaded before the first is worked on
struct Runs {
  int64_t n;    // runs: n rows of per_row
  int per_row;
};
__host__ __device__ inline Runs runs_of(int64_t rows, int k) {
  const int per_row = (k + 255) / 256;
  return {rows * per_row, per_row};
}

// the larger of two values; a NaN wins
__device__ __forceinline__ float max_or_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// Code of v in 0 .. 15: rint(v / s) + z.  The quotient comes from a product with
// inv = 1 / s, off by less than 2^-22 of it, and is rounded to even by the sum with
// 1.5 2^23; only within 1e-4 of the middle of two codes (and where inv is no use)
// does the division decide.
__device__ __forceinline__ uint32_t code_of(float v, float s, float inv, int z) {
  constexpr float kRound = 12582912.f;
  float q = v * inv, r = q + kRound;
  if (!(fabsf(q - (r - kRound)) < 0.4999f)) {
    q = fminf(fmaxf(rintf(v / s), -64.f), 64.f);  // (a NaN becomes -64)
    r = q + kRound;
  }
  return (uint32_t)min(max((int)(__float_as_uint(r) - __float_as_uint(kRound)) + z, 0), 15);
}

template <typename TW, typename TS>
__global__ void __launch_bounds__(kThreads) q4_quantize_kernel(const TW* W, int64_t ldw, Q4 w, uint32_t* packed,
                                                               TS* scales, uint8_t* zeros, bool wide) {
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const Runs runs = runs_of(w.n, w.k);
  const int64_t first = ((int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5)) * kUnits;
  const bool asym = zeros != nullptr;
  const int span = 1 << (w.group_log - 3);  // lanes of a group
  float v[kUnits][8];
  int64_t row = first / runs.per_row;
  int at = (int)(first - row * runs.per_row);
  const int64_t row0 = row;
  const int at0 = at;
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const int col = (at * 32 + lane) * 8;
    const bool in = first + u < runs.n;
    if (in && wide && col + 8 <= w.k && ACID_IN_BOUNDS(kSiteQ4, row, w.n)) {
      load8(W + row * ldw + col, v[u]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[u][j] = in && col + j < w.k ? io<TW>::ld(W + row * ldw + col + j) : 0.f;
    }
    if (++at == runs.per_row) {
      at = 0;
      ++row;
    }
  }
  row = row0;
  at = at0;
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    if (first + u >= runs.n) break;
    const int octet = at * 32 + lane, col = octet * 8;
    float hi = 0.f, lo = 0.f;  // max(w, 0) and -min(w, 0), or max |w|
#pragma unroll
    for (int j = 0; j < 8; ++j) hi = max_or_nan(hi, asym ? v[u][j] : fabsf(v[u][j]));
    if (asym)
#pragma unroll
      for (int j = 0; j < 8; ++j) lo = max_or_nan(lo, -v[u][j]);
    for (int o = span >> 1; o > 0; o >>= 1) {
      hi = max_or_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
      if (asym) lo = max_or_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    }
    TS st;
    io<TS>::st(&st, asym ? (hi + lo) / 15.f : hi / 7.f);
    const float s = io<TS>::ld(&st), div = s == 0.f ? 1.f : s, inv = 1.f / div;
    const int z = asym ? (int)fminf(fmaxf(rintf(lo / div), 0.f), 15.f) : 8;
    uint32_t q = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) q |= code_of(v[u][j], div, inv, z) << (4 * j);
    if (octet < w.slabs * 16) {
      const int64_t p = row * w.slabs * 16 + column_word(octet);
      if (ACID_IN_BOUNDS(kSiteQ4, p, w.n * w.slabs * 16)) packed[p] = q;
    }
    if ((lane & (span - 1)) == 0 && col < w.k) {
      const int64_t p = row * w.groups + (col >> w.group_log);
      if (ACID_IN_BOUNDS(kSiteQ4, p, w.n * w.groups)) {
        scales[p] = st;
        if (asym) zeros[p] = (uint8_t)z;
      }
    }
    if (++at == runs.per_row) {
      at = 0;
      ++row;
    }
  }
}

// 32 bytes with one store where the address allows it: a lane's own sector.
__device__ __forceinline__ void store_octet(float* p, const float* v, bool sector) {
  if (sector) {
    asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]),
                 "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
                 : "memory");
  } else {
    store8(p, v);
  }
}
__device__ __forceinline__ void store_octet(bf16* p, const float* v, bool) { store8(p, v); }

template <typename TS, typename TO>
__global__ void __launch_bounds__(kThreads) q4_dequantize_kernel(Q4 w, TO* out, int64_t ldo, bool wide, bool sector) {
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const Runs runs = runs_of(w.n, w.k);
  const int64_t first = ((int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5)) * kUnits;
  int64_t row = first / runs.per_row;
  int at = (int)(first - row * runs.per_row);
  uint32_t word[kUnits];
  float s[kUnits];
  int z[kUnits];
  const int64_t row0 = row;
  const int at0 = at;
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const int octet = at * 32 + lane;
    word[u] = 0;
    s[u] = 0.f;
    z[u] = 8;
    if (first + u < runs.n && octet * 8 < w.k) {
      word[u] = word_at(w, row, column_word(octet));
      s[u] = scale_at<TS>(w, row, octet * 8);
      z[u] = zero_at(w, row, octet * 8);
    }
    if (++at == runs.per_row) {
      at = 0;
      ++row;
    }
  }
  row = row0;
  at = at0;
#pragma unroll
  for (int u = 0; u < kUnits; ++u) {
    const int col = (at * 32 + lane) * 8;
    if (first + u < runs.n && col < w.k) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)  // 2^23 + q is the float with q in its last bits
        v[j] = s[u] * (__uint_as_float((word[u] >> (4 * j) & 15u) | 0x4B000000u) - (8388608.f + (float)z[u]));
      TO* p = out + row * ldo + col;
      if (wide && col + 8 <= w.k) {
        if (ACID_IN_BOUNDS(kSiteQ4, row, w.n)) store_octet(p, v, sector);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (col + j < w.k) io<TO>::st(p + j, v[j]);
      }
    }
    if (++at == runs.per_row) {
      at = 0;
      ++row;
    }
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

// n tiles that a kernel is built for
int tiles_for(int64_t m) {
  const int nt = (int)((std::min<int64_t>(m, kChunk) + 7) / 8);
  return nt <= 3 ? nt : nt <= 5 ? 5 : 8;
}
int64_t chunks_of(int64_t m) { return (m + kChunk - 1) / kChunk; }

// Whether the CTAs prepare a(x) themselves: few rows, whose parts fit their shared memory twice an SM.
bool packed_rows(int64_t m, int k) { return m <= kPackedRows && m * k <= 16384; }
// Workspace of the product: the parts of a(x), then the powers of two.
size_t parts_bytes(const acid_q4_weight& w, int64_t m) {
  return packed_rows(m, w.k) ? 0 : (size_t)chunks_of(m) * ((w.k + 127) / 128) * tiles_for(m) * 4096;
}
size_t fwd_bytes(const acid_q4_weight& w, int64_t m) {
  return packed_rows(m, w.k) ? 0 : parts_bytes(w, m) + (size_t)m * ((w.k + 127) / 128) * sizeof(float);
}

// CTAs that share a slab's rows in the input gradient.
int bwd_splits(int64_t n, int slabs) {
  const int64_t want = (304 + slabs - 1) / slabs, most = (n + 127) / 128;
  return (int)std::max<int64_t>(1, std::min(want, most));
}
int64_t bwd_per(int64_t n, int slabs) {
  const int64_t splits = bwd_splits(n, slabs);
  return ((n + splits - 1) / splits + 15) / 16 * 16;
}
size_t bwd_bytes(const acid_q4_weight& w, int64_t m) {
  const int slabs = (w.k + 127) / 128;
  return (size_t)bwd_splits(w.n, slabs) * m * slabs * 128 * sizeof(float);
}

size_t workspace_bytes(const acid_q4_weight& w, int64_t m) {
  return std::max<size_t>({16, fwd_bytes(w, m), bwd_bytes(w, m)});
}

// Warps of a CTA that share a row's columns: as many as give every SM eight warps
// where the rows alone would not.
int sharing_warps(const Q4& w) {
  int kw = 1;
  while (kw < 8 && 2 * kw <= w.slabs && (w.n + 31) / 32 * kw < 8 * num_sms()) kw *= 2;
  return kw;
}
template <typename TS, bool ZEROS>
acid_status launch_few(Fwd a, cudaStream_t s) {
  static PerContext allowed;
  a.kw = sharing_warps(a.w);
  const int rw = kThreads / 32 / a.kw;
  const size_t smem = (size_t)a.w.slabs * (512 * a.m + 4 * kPackedRows * (ZEROS ? 5 : 1)) +
                      (a.kw == 1 ? 0 : 8 * kPackedRows * 33 * sizeof(float));
  ACID_TRY(allow_smem(allowed, q4_few_kernel<TS, ZEROS>, 110 * 1024));
  const int64_t sets = ((a.w.n + 31) / 32 + rw - 1) / rw;
  launch_pdl(q4_few_kernel<TS, ZEROS>, (unsigned)std::min<int64_t>(sets, (int64_t)num_sms() * 2), kThreads, smem, s, a);
  ACID_CHECK_LAUNCH();
  return ACID_OK;
}
template <int NT, typename TS>
acid_status launch_forward(Fwd a, cudaStream_t s) {
  static PerContext allowed;
  a.kw = sharing_warps(a.w);
  const int rw = kThreads / 32 / a.kw;
  const size_t smem = a.kw == 1 ? 0 : (size_t)8 * NT * 8 * 33 * sizeof(float);
  ACID_TRY(allow_smem(allowed, q4_forward_kernel<NT, TS>, 8 * NT * 8 * 33 * sizeof(float)));
  const int64_t sets = ((a.w.n + 31) / 32 + rw - 1) / rw;
  const dim3 grid((unsigned)std::min<int64_t>(sets, (int64_t)num_sms() * (NT <= 2 ? 2 : 1)), (unsigned)chunks_of(a.m));
  launch_pdl(q4_forward_kernel<NT, TS>, grid, kThreads, smem, s, a);
  ACID_CHECK_LAUNCH();
  return ACID_OK;
}
template <int NT>
acid_status launch_parts_forward(const Fwd& a, bool half_scales, cudaStream_t s) {
  const int64_t octets = a.m * a.w.slabs * 16;
  launch_pdl(q4_parts_kernel<NT>, (unsigned)((octets + kThreads - 1) / kThreads), kThreads, 0, s, a);
  ACID_CHECK_LAUNCH();
  return half_scales ? launch_forward<NT, bf16>(a, s) : launch_forward<NT, float>(a, s);
}

template <int NT, int IW, bool PACKED>
acid_status launch_backward(const Bwd& a, cudaStream_t s) {
  static PerContext allowed;
  const auto kernel = q4_backward_kernel<NT, IW, PACKED>;
  ACID_TRY(allow_smem(allowed, kernel, kBwdSmem<NT, IW, PACKED>));
  const dim3 grid(a.dx != nullptr ? a.w.slabs : 1, a.splits, a.dx != nullptr ? (unsigned)chunks_of(a.m) : 1);
  launch_pdl(kernel, grid, kThreads, kBwdSmem<NT, IW, PACKED>, s, a);
  ACID_CHECK_LAUNCH();
  return ACID_OK;
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
  const bool wide = aligned(W, 16) && ldw % 8 == 0;
  const int64_t per_cta = kThreads / 32 * kUnits;
  const unsigned grid = (unsigned)((runs_of(w.n, w.k).n + per_cta - 1) / per_cta);
  auto packed = static_cast<uint32_t*>(const_cast<void*>(weight->packed));
  auto scales = const_cast<void*>(weight->scales);
  auto zeros = const_cast<uint8_t*>(weight->zeros);
  auto launch = [&](auto* src, auto* sc) {
    launch_pdl(q4_quantize_kernel<std::remove_const_t<std::remove_pointer_t<decltype(src)>>,
                                  std::remove_pointer_t<decltype(sc)>>,
               grid, kThreads, 0, s, src, ldw, w, packed, sc, zeros, wide);
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
  const int64_t per_cta = kThreads / 32 * kUnits;
  const unsigned grid = (unsigned)((runs_of(w.n, w.k).n + per_cta - 1) / per_cta);
  const bool wide = aligned(out, 16) && ldo % 8 == 0, sector = wide && aligned(out, 32);
  const bool h = weight->scale_dtype == ACID_BF16;
  if (out_dtype == ACID_BF16)
    launch_pdl(h ? q4_dequantize_kernel<bf16, bf16> : q4_dequantize_kernel<float, bf16>, grid, kThreads, 0, s, w,
               static_cast<bf16*>(out), ldo, wide, sector);
  else
    launch_pdl(h ? q4_dequantize_kernel<bf16, float> : q4_dequantize_kernel<float, float>, grid, kThreads, 0, s, w,
               static_cast<float*>(out), ldo, wide, sector);
  ACID_CHECK_LAUNCH();
  return ACID_OK;
}

extern "C" acid_status acid_q4_linear_forward(int32_t x_dtype, const void* x, int64_t ldx, int64_t M,
                                              const acid_q4_weight* weight, const float* bias, int32_t silu_input,
                                              int32_t out_dtype, void* out, int64_t ldo, void* ws, size_t ws_bytes,
                                              acid_stream_t stream) {
  clear_error();
  ACID_TRY(check_weight(weight));
  ACID_REQUIRE(M >= 0 && M <= kMostRows, ACID_ERR_INVALID_ARG, "acid_q4_linear_forward: need 0 <= M <= 32768");
  if (M == 0) return ACID_OK;
  ACID_TRY(check_pointers(*weight));
  ACID_TRY(check_matrix(x_dtype, x, ldx, weight->k, "x"));
  ACID_TRY(check_matrix(out_dtype, out, ldo, weight->n, "out"));
  ACID_REQUIRE(aligned(bias, 4), ACID_ERR_UNSUPPORTED, "acid_q4_linear_forward: bias must be 4-byte aligned");
  const size_t need = fwd_bytes(*weight, M);
  ACID_REQUIRE(need == 0 || (ws != nullptr && aligned(ws, 16)), ACID_ERR_WORKSPACE,
               "acid_q4_linear_forward: workspace null or not 16-byte aligned");
  ACID_REQUIRE(ws_bytes >= need, ACID_ERR_WORKSPACE,
               "acid_q4_linear_forward: workspace too small (need " + std::to_string(need) + ")");
  Fwd a{q4_args(*weight), x, ldx, M, x_dtype, silu_input != 0, out_dtype, bias, out, ldo, static_cast<uint4*>(ws), nullptr, 1};
  a.back = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + parts_bytes(*weight, M));
  const bool h = weight->scale_dtype == ACID_BF16;
  cudaStream_t s = (cudaStream_t)stream;
  if (need == 0) {
    if (weight->zeros != nullptr) return h ? launch_few<bf16, true>(a, s) : launch_few<float, true>(a, s);
    return h ? launch_few<bf16, false>(a, s) : launch_few<float, false>(a, s);
  }
  switch (tiles_for(M)) {
    case 1: return launch_parts_forward<1>(a, h, s);
    case 2: return launch_parts_forward<2>(a, h, s);
    case 3: return launch_parts_forward<3>(a, h, s);
    case 5: return launch_parts_forward<5>(a, h, s);
    default: return launch_parts_forward<8>(a, h, s);
  }
}

extern "C" acid_status acid_q4_linear_workspace_size(const acid_q4_weight* weight, int64_t M, size_t* bytes) {
  clear_error();
  ACID_TRY(check_weight(weight));
  ACID_REQUIRE(bytes != nullptr && M >= 0 && M <= kMostRows, ACID_ERR_INVALID_ARG,
               "acid_q4_linear_workspace_size: bad argument");
  *bytes = workspace_bytes(*weight, M);
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
    const size_t need = workspace_bytes(*weight, M);
    ACID_REQUIRE(ws_bytes >= need, ACID_ERR_WORKSPACE,
                 "acid_q4_linear_backward: workspace too small (need " + std::to_string(need) + ")");
  }
  const int slabs = (weight->k + 127) / 128;
  Bwd a{q4_args(*weight), g, x, ldg, ldx, M, g_dtype, x_dtype, weight->scale_dtype, silu_input != 0, dx, lddx, dbias,
        static_cast<float*>(ws), 0, bwd_per(weight->n, slabs)};
  a.splits = (int)((weight->n + a.per - 1) / a.per);
  if (M <= kBwdPackedRows) {
    ACID_TRY((launch_backward<1, 4, true>(a, s)));
  } else {
    switch (tiles_for(M)) {
      case 1: ACID_TRY((launch_backward<1, 4, false>(a, s))); break;
      case 2: ACID_TRY((launch_backward<2, 4, false>(a, s))); break;
      case 3: ACID_TRY((launch_backward<3, 2, false>(a, s))); break;
      case 5: ACID_TRY((launch_backward<5, 1, false>(a, s))); break;
      default: ACID_TRY((launch_backward<8, 1, false>(a, s)));
    }
  }
  if (dx == nullptr) return ACID_OK;
  launch_pdl(q4_backward_join_kernel, dim3((a.w.k + kThreads - 1) / kThreads, (unsigned)M), kThreads, 0, s, a);
  ACID_CHECK_LAUNCH();
  return ACID_OK;
}
