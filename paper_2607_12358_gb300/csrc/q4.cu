// Modulation projections with 4-bit weights: quantiser, values, product and
// input gradient (acid_q4_*).
#include <algorithm>
#include <string>

#define ACID_UNIT_WITHOUT_WAITS
#include "q4.cuh"

namespace acid {

BoundsRecord take_bounds_q4();
ACID_BOUNDS_READER(take_bounds_q4)

namespace {

constexpr int kThreads = 256;
using bf16 = __nv_bfloat16;

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
__device__ __forceinline__ uint4 load_stream(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

// ------------------------------------------------- product with a few rows
// out^T = W a(x)^T on the tensor cores, the codes as the exact halves q - z (16
// rows of the weight to a tile) against the two parts of a(x).  Products are
// exact, a group's sum is formed by the tensor cores in fp32 and multiplied by
// the group's scale in fp32.  The parts of row m are columns 2 m and 2 m + 1 of one
// tile of eight, prepared by each CTA in its shared memory.
using Fwd = Q4Fwd;
constexpr int kPackedRows = 4;

// The activated octet's values and the factor of their slab; 16 lanes in a row
// hold a slab's octets.
__device__ __forceinline__ float octet_of(const Fwd& a, int64_t m, int col, float (&v)[8]) {
  float top = octet_values(a, m, col, v);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  return up_to_half(top);
}

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

// Row m of a(x) times a row of the weight, value by value.
template <typename TS>
__device__ __noinline__ float plain_product(const Fwd& a, int64_t m, int64_t row) {
  float sum = 0.f;
  for (int col = 0; col < a.w.k; col += 32) {
    float part = 0.f;
    for (int o = col / 8; o < col / 8 + 4 && o * 8 < a.w.k; ++o) {
      float v[8];
      octet_values(a, m, o * 8, v);
      const uint32_t word = word_at(a.w, row, column_word(o));
      const float s = scale_at<TS>(a.w, row, col);
      const int z = zero_at(a.w, row, col);
      for (int j = 0; j < 8 && o * 8 + j < a.w.k; ++j) part += v[j] * (s * (float)((int)(word >> (4 * j) & 15u) - z));
    }
    sum += part;
  }
  return sum;
}
// Values that the kernels' sums cannot serve: not finite, or so large that a sum may pass the
// largest number where the result does not.  Each warp notes what it met, one entry a warp.
enum Special { kInfinite = 1, kLarge = 2 };
__device__ __forceinline__ void note_special(int* noted, bool infinite, float by) {
  // (by, the least power of two that a value was brought down with; 65536 values below 2^82
  // times 15 stay far from the largest number)
  const int it = (infinite ? kInfinite : 0) | (by < 0x1p-60f ? kLarge : 0), all = __reduce_or_sync(0xffffffffu, it);
  if ((threadIdx.x & 31) == 0) noted[threadIdx.x >> 5] = all;
}
// Behind the kernels' loops: the CTA's results that are not finite, or should not be, value by value.
template <typename TS>
__device__ __noinline__ void special_results(const Fwd& a, int rw, bool infinite) {
  __syncthreads();
  const int rows = (int)a.m;
  const int64_t tiles = (a.w.n + 31) / 32, sets = (tiles + rw - 1) / rw;
  for (int64_t set = blockIdx.x; set < sets; set += gridDim.x)
    for (int i = threadIdx.x; i < rw * rows * 32; i += kThreads) {
      const int64_t row = (set * rw + i / (rows * 32)) * 32 + (i & 31), m = (i >> 5) % rows, at = m * a.ldo + row;
      if (row >= a.w.n) continue;
      const bool bad = !isfinite(value_at(a.out_dtype, a.out, at));
      if (!infinite && !bad) continue;
      const float v = plain_product<TS>(a, m, row);
      if (bad || !isfinite(v)) put_value(a.out_dtype, a.out, at, v + (a.bias != nullptr ? a.bias[row] : 0.f));
    }
}
template <typename TS>
__device__ __forceinline__ void look_at_special(const Fwd& a, int rw, const int* noted) {
  const int all = __reduce_or_sync(0xffffffffu, noted[threadIdx.x & 7]);
  if (all != 0) special_results<TS>(a, rw, all & kInfinite);
}

// Two to four rows: the codes enter as q - 8 and a zero point by the sum of a(x) over
// the group, sum x (q - z) = sum x (q - 8) + (8 - z) sum x (without values that are not
// finite, whose two shares may have either sign: special_results).  A CTA's warps split a
// row tile's slabs among kw of them, and 8 / kw row tiles are neighbours.  A lane reads 16
// bytes of four rows: word i of them holds its columns of the slab's 32 columns i, so
// that four lanes' words make a tile's step of 16 columns twice.
//   Instructions bound it, 425 a warp for 32 rows of 128 columns, of which 144 convert codes
// (two rows: issue 61 to 66% busy, the integer pipe 60 to 63%, DRAM 42 to 46%): 276480 x 1536,
// groups of 128, two rows 56 us, four 57 to 58 (56% of a copy's rate); groups of 64 with zero
// points 66 and 67 us.
template <typename TS, bool ZEROS, int LOG>
__global__ void __launch_bounds__(kThreads, 2) q4_few_kernel(Fwd a) {
  constexpr int kWords = 1 << (LOG - 5);  // of 32 columns, to a group
  extern __shared__ __align__(16) uint8_t smem[];
  const Q4& w = a.w;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, warp = warp_index();
  const int kw = a.kw, rw = kThreads / 32 / kw, kwarp = warp % kw, rwarp = warp / kw;
  const int rows = (int)a.m, cols = 2 * rows;
  uint4* frag = reinterpret_cast<uint4*>(smem);                                   // [slab][word][column][t]
  float* back = reinterpret_cast<float*>(smem + (size_t)w.slabs * 16 * cols * 16);  // [slab][row]
  float* xsum = back + w.slabs * kPackedRows;                                     // [slab][32 columns][row]
  uint4* none = reinterpret_cast<uint4*>(xsum + (ZEROS ? 4 * w.slabs * kPackedRows : 0));  // zeros
  int* noted = reinterpret_cast<int*>(none + 1);                                  // [8 warps]
  float* red = reinterpret_cast<float*>(none + 3);                                // [8 warps][row][33]
  const int64_t tiles = (w.n + 31) / 32, sets = (tiles + rw - 1) / rw;
  const int mine = (w.slabs - kwarp + kw - 1) / kw;  // slabs of this warp
  constexpr int per_slab = 4 / kWords;
  const int lane_group = t / kWords;
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
    bool infinite = false;  // (with zero points; else such values go through the sums)
    float least = 1.f;
    const int per_row = w.slabs * 16, all = per_row * rows;
    for (int base = threadIdx.x & ~31; base < all; base += kThreads) {
      const int i = base + lane, m = i / per_row, o = i - m * per_row;
      float v[8];
      const float by = octet_of(a, m, o * 8, v);
      least = fminf(least, by);
      float sum = 0.f;
      if constexpr (ZEROS) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (!isfinite(v[j])) {
            infinite = true;
            v[j] = 0.f;
          }
          sum += v[j];
        }
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
    if (threadIdx.x == 0) *none = make_uint4(0, 0, 0, 0);
    note_special(noted, infinite, least);
    __syncthreads();
  }
  float sum[2][2];  // row t of the input, rows g + 8 h + 16 r of the tile
  auto clear = [&] { sum[0][0] = sum[0][1] = sum[1][0] = sum[1][1] = 0.f; };
  const uint4* mine_b = g < cols ? frag + g * 4 + t : none;  // columns past the parts are zeros
  const int word_b = g < cols ? cols * 4 : 0;
  auto compute = [&](const Load& l, int slab) {
    const float bk = back[slab * kPackedRows + t];
    const uint4* pb = mine_b + slab * 4 * word_b;
    float acc[2][4], xs = 0.f, z[4];
    if constexpr (ZEROS)
#pragma unroll
      for (int q = 0; q < 4; ++q) z[q] = 8.f - (float)l.z[q];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 b = pb[i * word_b];
      if (ZEROS) xs = (i % kWords == 0 ? 0.f : xs) + xsum[(slab * 4 + i) * kPackedRows + t];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        uint32_t d[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint4& v = l.q[2 * r + h];
          halves_of(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w, 8u, d[h]);
        }
        if (i % kWords == 0)
          mma_f16_first(acc[r], d[0][0], d[1][0], d[0][1], d[1][1], b.x, b.y);
        else
          mma_f16(acc[r], d[0][0], d[1][0], d[0][1], d[1][1], b.x, b.y);
        mma_f16(acc[r], d[0][2], d[1][2], d[0][3], d[1][3], b.z, b.w);
      }
      if ((i + 1) % kWords == 0) {  // the group ends
        const int from = (lane & ~3) | i / kWords * kWords;  // a lane that has its scale
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int q = 2 * r + h;
            const float s = kWords == 4 ? l.s[q] : __shfl_sync(0xffffffffu, l.s[q], from);
            float v = (acc[r][2 * h] + acc[r][2 * h + 1]) * bk;  // both parts of row t are in this lane
            if constexpr (ZEROS) v = fmaf(kWords == 4 ? z[q] : __shfl_sync(0xffffffffu, z[q], from), xs, v);
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
  look_at_special<TS>(a, rw, noted);
}

// ------------------------------------------------------- product with one row
// One row on whole numbers.  The activated values of 128 columns, times the power of two
// that brings the largest to 2^22 .. 2^23, are rounded to v = 2^16 h + 2^8 m + l (h signed,
// m and l unsigned bytes: to within 2^-23 of the largest), and four codes meet four
// bytes of each in one instruction (dot product of bytes).  A lane's part of a group's sum
// of v (q - z) is exact: it has 31 bits up to 16 columns, where the three sums may wrap on
// the way, and is put together from two parts in fp32 beyond.  What is not finite is left
// out there (special_results).
//   The tensor cores' tile has room for four rows; for one, most of it is empty, and its
// codes have to become halves first: 9 instructions for eight codes, here 3, and 6 for
// their products.  276480 x 1536, groups of 128 43 us (76% of a copy's rate; by the kernel
// above 54), of 64 with zero points 53 us (65%; 65).  No unit is full there: the pipe of the
// byte products is 61% busy, issue 62 to 64%, DRAM (under a profiler) 60 and 52%; sixteen
// warps an SM with two loads ahead each wait for memory and for that pipe in turn.
// 9216 x 1536 5 us, a launch and the loads' latency.
struct OneSmem {
  size_t low, sums, back, red, noted, all;  // behind the high bytes, uint4 [16 slabs]
};
__host__ __device__ inline OneSmem one_smem(int slabs, int groups_of_slab) {
  OneSmem o;
  o.low = (size_t)slabs * 16 * 16;              // uint2 [16 slabs]
  o.sums = o.low + (size_t)slabs * 16 * 8;      // int2 [slab][group][4]
  o.back = o.sums + (size_t)slabs * groups_of_slab * 32;
  o.red = o.back + (size_t)slabs * 4;
  o.noted = o.red + 8 * 33 * 4;
  o.all = o.noted + 32;
  return o;
}
template <typename TS, bool ZEROS, int LOG>
__global__ void __launch_bounds__(kThreads, 2) q4_one_kernel(Fwd a) {
  constexpr int kWords = 1 << (LOG - 5), per_slab = 4 / kWords;  // words of 32 columns to a group; groups to a slab
  extern __shared__ __align__(16) uint8_t smem[];
  const Q4& w = a.w;
  const OneSmem at_smem = one_smem(w.slabs, per_slab);
  uint4* high = reinterpret_cast<uint4*>(smem);                     // [octet]: h and m of the even columns and the odd ones
  uint2* low = reinterpret_cast<uint2*>(smem + at_smem.low);        // [octet]: l
  int2* vsum = reinterpret_cast<int2*>(smem + at_smem.sums);        // [slab][group][t]: sums of h, and of 2^8 m + l
  float* back = reinterpret_cast<float*>(smem + at_smem.back);      // [slab]
  float* red = reinterpret_cast<float*>(smem + at_smem.red);        // [8 warps][33]
  int* noted = reinterpret_cast<int*>(smem + at_smem.noted);        // [8 warps]
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, warp = warp_index();
  const int kw = a.kw, rw = kThreads / 32 / kw, kwarp = warp % kw, rwarp = warp / kw;
  const int64_t tiles = (w.n + 31) / 32, sets = (tiles + rw - 1) / rw;
  const int mine = (w.slabs - kwarp + kw - 1) / kw;  // slabs of this warp
  const int lane_group = t / kWords;
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
  // the bytes of a(x), while the first weights are on their way
  bool infinite = false;
  float least = 1.f;
  for (int base = threadIdx.x & ~31; base < w.slabs * 16; base += kThreads) {
    const int o = base + lane;  // the octet 4 i + t of a slab's 16 lanes
    float v[8];
    float top = octet_values(a, 0, o * 8, v);
#pragma unroll
    for (int x = 8; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
    const float by = __uint_as_float(min(276u - (__float_as_uint(top) >> 23), 254u) << 23);
    least = fminf(least, by);
    uint32_t d[6] = {};  // h, m, l of the even columns and of the odd ones
    int sh = 0, sl = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      infinite = infinite || !isfinite(v[j]);
      const int n = isfinite(v[j]) ? min(__float2int_rn(v[j] * by), (1 << 23) - 1) : 0;
      sh += n >> 16;
      sl += n & 0xffff;
#pragma unroll
      for (int b = 0; b < 3; ++b) d[2 * b + j % 2] |= ((uint32_t)n >> (16 - 8 * b) & 255u) << (8 * (j / 2));
    }
#pragma unroll
    for (int x = 4; x < 4 * kWords; x <<= 1) {
      sh += __shfl_xor_sync(0xffffffffu, sh, x);
      sl += __shfl_xor_sync(0xffffffffu, sl, x);
    }
    if (o < w.slabs * 16) {
      high[o] = make_uint4(d[0], d[1], d[2], d[3]);
      low[o] = make_uint2(d[4], d[5]);
      const int i = (o >> 2) & 3, slab = o >> 4;
      if (i % kWords == 0) vsum[(slab * per_slab + i / kWords) * 4 + (o & 3)] = make_int2(sh, sl);
      if ((o & 15) == 0) back[slab] = 1.f / by;
    }
  }
  note_special(noted, infinite, least);
  __syncthreads();
  float sum[4] = {};  // rows g + 8 q of the tile, this lane's columns
  auto compute = [&](const Load& l, int slab) {
    const float bk = back[slab];
    int h[4], m[4], lw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 hm = high[(slab * 4 + i) * 4 + t];
      const uint2 lo = low[(slab * 4 + i) * 4 + t];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t word = i == 0 ? l.q[q].x : i == 1 ? l.q[q].y : i == 2 ? l.q[q].z : l.q[q].w;
        const uint32_t even = word & 0x0f0f0f0fu, uneven = word >> 4 & 0x0f0f0f0fu;
        if (i % kWords == 0) h[q] = m[q] = lw[q] = 0;
        h[q] = __dp4a((int)uneven, (int)hm.y, __dp4a((int)even, (int)hm.x, h[q]));
        m[q] = (int)__dp4a(uneven, hm.w, __dp4a(even, hm.z, (uint32_t)m[q]));
        lw[q] = (int)__dp4a(uneven, lo.y, __dp4a(even, lo.x, (uint32_t)lw[q]));
      }
      if ((i + 1) % kWords == 0) {  // the group ends
        const int from = (lane & ~3) | i / kWords * kWords;  // a lane that has its scale
        const int2 vs = vsum[(slab * per_slab + i / kWords) * 4 + t];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float s = kWords == 4 ? l.s[q] : __shfl_sync(0xffffffffu, l.s[q], from);
          const int z = !ZEROS ? 8 : kWords == 4 ? l.z[q] : __shfl_sync(0xffffffffu, (int)l.z[q], from);
          const int r = m[q] * 256 + lw[q] - z * vs.y;
          float v;
          if constexpr (kWords == 4)
            v = fmaf((float)(h[q] - z * vs.x), 65536.f, (float)r);
          else
            v = (float)(int)((uint32_t)(h[q] - z * vs.x) * 65536u + (uint32_t)r);
          sum[q] = fmaf(s, v * bk, sum[q]);
        }
      }
    }
  };
  auto put = [&](int64_t row, float v) {
    if (row < w.n) put_value(a.out_dtype, a.out, row, v + (a.bias != nullptr ? a.bias[row] : 0.f));
  };
  auto finish = [&] {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      sum[q] += __shfl_xor_sync(0xffffffffu, sum[q], 1);
      sum[q] += __shfl_xor_sync(0xffffffffu, sum[q], 2);
    }
    const float v = t == 0 ? sum[0] : t == 1 ? sum[1] : t == 2 ? sum[2] : sum[3];
    sum[0] = sum[1] = sum[2] = sum[3] = 0.f;
    if (kw == 1) {
      put((set * rw + rwarp) * 32 + 8 * t + g, v);
      return;
    }
    __syncthreads();  // the buffer's last readers are done
    red[warp * 33 + 8 * t + g] = v;
    __syncthreads();
    for (int i = threadIdx.x; i < rw * 32; i += kThreads) {
      float all = 0.f;
      for (int j = 0; j < kw; ++j) all += red[((i >> 5) * kw + j) * 33 + (i & 31)];
      put((set * rw + (i >> 5)) * 32 + (i & 31), all);
    }
  };
  auto step = [&](Load& cur) {
    if (set >= sets) return;
    compute(cur, kwarp + k * kw);
    next(cur);
    if (++k == mine) {
      finish();
      k = 0;
      set += gridDim.x;
    }
  };
  while (set < sets) {
    step(l[0]);
    step(l[1]);
  }
  look_at_special<TS>(a, rw, noted);
}

// ---------------------------------------------------------------- quantiser
// the larger of two values; a NaN wins
__device__ __forceinline__ float max_or_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// Codes of eight values in 0 .. 15, rint(v / s) + z, by divisions.
__device__ __noinline__ uint32_t divided_codes(float4 lo, float4 hi, float s, int z) {
  const float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  uint32_t word = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j)  // (a NaN becomes the lowest code)
    word |= (uint32_t)fminf(fmaxf(rintf(v[j] / s) + (float)z, 0.f), 15.f) << (4 * j);
  return word;
}
// The same with one division a group: the quotient comes from a product with
// inv = 1 / s, off by less than 2^-22 of it, and is rounded to even by the sum with 1.5 2^23,
// whose last bits are then the code's; the eight are gathered by one addition each,
// the constant bits above them taken out at the end.
//   A quotient near the middle of two codes depends on its last bits (they are corrected by
// the remainder, after Markstein).  Where value and
// scale are bf16 (SHORT) it is the middle m or at least 2^-9 off it (v - m s is a multiple
// of half the last place of s), and the middle itself is met often; the remainder v - q s
// (one fma, exact) takes the product's error out, so that it comes out exactly.  Otherwise a
// word with a value within 1e-4 of a middle is formed by divisions, as are those whose
// scale is no ordinary number.
//   Quotients lie in -7.03 .. 7.03 without zero points (s may be rounded down by 2^-8):
// no code is clamped; with them the largest may come out as 16.
template <bool ZEROS, bool SHORT>
__device__ __forceinline__ uint32_t codes_of(const float (&v)[8], float s, float inv, int z) {
  constexpr float kRound = 12582912.f;
  const uint64_t inv2 = f2_pack(inv, inv), up = f2_pack(kRound, kRound), down = f2_pack(-kRound, -kRound);
  const uint64_t minus = f2_pack(-1.f, -1.f), minus_s = f2_pack(-s, -s);
  const float most = kRound + (float)(15 - z);
  uint32_t word = 0;
  float off = 0.f;
#pragma unroll
  for (int j = 6; j >= 0; j -= 2) {
    const uint64_t v2 = f2_pack(v[j], v[j + 1]);
    uint64_t q = f2_mul(v2, inv2);
    if (SHORT) q = f2_fma(f2_fma(q, minus_s, v2), inv2, q);
    const uint64_t r = f2_add(q, up);
    float x, y;
    if (!SHORT) {
      f2_unpack(f2_fma(f2_add(r, down), minus, q), x, y);
      off = max_or_nan(off, max_or_nan(fabsf(x), fabsf(y)));
    }
    f2_unpack(r, x, y);
    if (ZEROS) {
      x = fminf(x, most);
      y = fminf(y, most);
    }
    word = word * 16u + __float_as_uint(y);
    word = word * 16u + __float_as_uint(x);
  }
  const bool sure = SHORT ? s >= 0x1p-90f && s <= 0x1p90f : off < 0.4999f;
  if (sure) return word - (0x4B400000u - (uint32_t)z) * 0x11111111u;
  return divided_codes(make_float4(v[0], v[1], v[2], v[3]), make_float4(v[4], v[5], v[6], v[7]), s, z);
}

// 8 values of the weight as they lie in memory, zeros past its columns.
template <typename TW>
struct Octet {
  uint4 bits[sizeof(TW) / 2];
  __device__ __forceinline__ void load(const TW* p, int cols, bool wide) {
    if (wide && cols >= 8) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(TW) / 2; ++i) bits[i] = reinterpret_cast<const uint4*>(p)[i];
      return;
    }
    uint32_t u[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (sizeof(TW) == 4)
        u[j] = j < cols ? __float_as_uint(p[j]) : 0u;
      else
        u[j] = j < cols ? __bfloat16_as_ushort(p[j]) : 0u;
    }
    if constexpr (sizeof(TW) == 4) {
      bits[0] = make_uint4(u[0], u[1], u[2], u[3]);
      bits[1] = make_uint4(u[4], u[5], u[6], u[7]);
    } else {
      bits[0] = make_uint4(u[0] | u[1] << 16, u[2] | u[3] << 16, u[4] | u[5] << 16, u[6] | u[7] << 16);
    }
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
    const uint32_t* u = reinterpret_cast<const uint32_t*>(bits);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      v[j] = sizeof(TW) == 4 ? __uint_as_float(u[j]) : j % 2 ? bf16_hi(u[j / 2]) : bf16_lo(u[j / 2]);
  }
};
// Four lanes take 128 columns of a row, each of them the octets t, t + 4, t + 8 and t + 12:
// their loads lie together and a lane's four words do too (with 32 adjoining columns a
// lane, 16-byte pieces 64 bytes apart, 36864 x 3072 took 88 us).  The four share 128 >> LOG
// groups: the exchange that finds the largest values hands each group to lanes that do its
// two divisions, once for 32 columns, and hand them round.
//   A CTA's threads go on by `rows` rows and `slabs` slabs, with the next columns' loads
// ahead of the work (without: 70 us).  HBM bounds it: 36864 x 3072, groups of 128, from bf16
// 45 us (93% of a copy's rate), from fp32 80 us (94%); with fp32 scales of bf16 values,
// whose middles are divided out, 91 us.
template <typename TW, typename TS, bool ZEROS, int LOG>
__global__ void __launch_bounds__(kThreads) q4_quantize_kernel(const TW* W, int64_t ldw, Q4 w, uint32_t* packed,
                                                               TS* scales, uint8_t* zeros, bool wide, int64_t rows,
                                                               int slabs) {
  pdl_wait();
  constexpr int kGroups = 128 >> LOG;
  const int t = threadIdx.x & 3;
  int64_t next_row = (blockIdx.x * (kThreads / 4) + (threadIdx.x >> 2)) / w.slabs;
  int next_slab = (int)((blockIdx.x * (kThreads / 4) + (threadIdx.x >> 2)) - next_row * w.slabs);
  Octet<TW> next[4];
  auto fetch = [&] {
    const int col = next_slab * 128 + 8 * t;
    const bool in = next_row < w.n && ACID_IN_BOUNDS(kSiteQ4, next_row, w.n);
    const TW* src = W + (in ? next_row * ldw + col : 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) next[i].load(src + 32 * i, in ? w.k - col - 32 * i : 0, wide);
  };
  fetch();
  // whole warps go on together: the shuffles need all lanes
  for (;;) {
    const int64_t row = next_row;
    const int slab = next_slab;
    const bool in = row < w.n;
    if (!__any_sync(0xffffffffu, in)) break;
    float v[4][8], hi[kGroups], lo[kGroups];  // max(w, 0) and -min(w, 0), or max |w|
#pragma unroll
    for (int i = 0; i < 4; ++i) next[i].values(v[i]);
    next_row += rows;
    next_slab += slabs;
    if (next_slab >= w.slabs) {
      next_slab -= w.slabs;
      ++next_row;
    }
    fetch();
#pragma unroll
    for (int g = 0; g < kGroups; ++g) hi[g] = lo[g] = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float &h = hi[i >> (LOG - 5)], &l = lo[i >> (LOG - 5)];
        h = max_or_nan(h, ZEROS ? v[i][j] : fabsf(v[i][j]));
        if (ZEROS) l = max_or_nan(l, -v[i][j]);
      }
    // lane t ends with group t & (kGroups - 1)
    auto largest = [&](float (&x)[kGroups]) {
      if constexpr (kGroups == 4) {
        const bool up = t & 2;
        const float a = __shfl_xor_sync(0xffffffffu, up ? x[0] : x[2], 2), b = __shfl_xor_sync(0xffffffffu, up ? x[1] : x[3], 2);
        x[0] = max_or_nan(up ? x[2] : x[0], a);
        x[1] = max_or_nan(up ? x[3] : x[1], b);
      }
      if constexpr (kGroups >= 2) {
        const bool up = t & 1;
        const float a = __shfl_xor_sync(0xffffffffu, up ? x[0] : x[1], 1);
        x[0] = max_or_nan(up ? x[1] : x[0], a);
      } else {
        x[0] = max_or_nan(x[0], __shfl_xor_sync(0xffffffffu, x[0], 1));
      }
      if constexpr (kGroups <= 2) x[0] = max_or_nan(x[0], __shfl_xor_sync(0xffffffffu, x[0], 2));
      return x[0];
    };
    const float top = largest(hi), low = ZEROS ? largest(lo) : 0.f;
    TS st;
    io<TS>::st(&st, ZEROS ? (top + low) / 15.f : top / 7.f);
    const float s = io<TS>::ld(&st), div = s == 0.f ? 1.f : s, inv = 1.f / div;
    const int z = ZEROS ? (int)fminf(fmaxf(rintf(low / div), 0.f), 15.f) : 8;
    // word 4 t + i of the slab holds the octet t of its 32 columns i
    constexpr bool kShort = sizeof(TW) == 2 && sizeof(TS) == 2;
    uint32_t words[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      constexpr uint32_t kAll = 0xffffffffu;
      const int of = i >> (LOG - 5);
      if (kGroups == 1)
        words[i] = codes_of<ZEROS, kShort>(v[i], div, inv, z);
      else
        words[i] = codes_of<ZEROS, kShort>(v[i], __shfl_sync(kAll, div, of, 4), __shfl_sync(kAll, inv, of, 4),
                                   ZEROS ? __shfl_sync(kAll, z, of, 4) : 8);
    }
    if (!in) continue;
    const int64_t at = (row * w.slabs + slab) * 16 + 4 * t;
    if (ACID_IN_BOUNDS(kSiteQ4, at + 3, w.n * w.slabs * 16))
      *reinterpret_cast<uint4*>(packed + at) = make_uint4(words[0], words[1], words[2], words[3]);
    const int group = slab * kGroups + t;
    if (t < kGroups && group < w.groups) {
      const int64_t p = row * w.groups + group;
      if (ACID_IN_BOUNDS(kSiteQ4, p, w.n * w.groups)) {
        scales[p] = st;
        if (ZEROS) zeros[p] = (uint8_t)z;
      }
    }
  }
}

// ------------------------------------------------------------------- values
// A lane takes eight columns of a row (one word), a warp 32 such octets of one
// row at a time.  HBM bounds it: 36864 x 3072 to fp32 in 75 us (89% of a copy's rate).
constexpr int kUnits = 4;  // octet runs of a warp, all loaded before the first is worked on
struct Runs {
  int64_t n;    // runs: n rows of per_row
  int per_row;
};
__host__ __device__ inline Runs runs_of(int64_t rows, int k) {
  const int per_row = (k + 255) / 256;
  return {rows * per_row, per_row};
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

// Whether the CTAs prepare a(x) themselves: few rows, whose parts fit their shared memory twice an SM.
bool few_rows(int64_t m, int k) { return m <= kPackedRows && m * k <= 16384; }
size_t fwd_bytes(const Q4& w, int64_t m) { return few_rows(m, w.k) ? 0 : q4_rows_forward_bytes(w, m); }
size_t workspace_bytes(const Q4& w, int64_t m) {
  return std::max<size_t>({16, fwd_bytes(w, m), m > 0 ? q4_backward_bytes(w, m) : 0});
}

// Warps of a CTA that share a row's columns: as many as give every SM eight warps where
// the rows alone would not, and up to four while an SM's sixteen warps have less than two
// turns each, which then come out more evenly (a row of x, groups of 128: 46080 x 1536
// with four 10.9 us, with one 13.5; 80000 x 1920 with two 20.4, with one 25.4; beyond, the
// sums' exchange costs more than it gains: 138240 x 3072 48.2 and 44.1).
int sharing_warps(const Q4& w) {
  const int64_t tiles = (w.n + 31) / 32, sms = num_sms();
  int kw = 1;
  while (kw < 8 && 2 * kw <= w.slabs && (tiles * kw < 8 * sms || (kw < 4 && tiles * kw < 28 * sms))) kw *= 2;
  return kw;
}
template <typename TS, bool ZEROS, int LOG>
acid_status launch_few(Fwd a, cudaStream_t s) {
  a.kw = sharing_warps(a.w);
  const int rw = kThreads / 32 / a.kw;
  const int64_t sets = ((a.w.n + 31) / 32 + rw - 1) / rw;
  const unsigned grid = (unsigned)std::min<int64_t>(sets, (int64_t)num_sms() * 2);
  if (a.m == 1) {
    static PerContext allowed;
    ACID_TRY(allow_smem(allowed, q4_one_kernel<TS, ZEROS, LOG>, 110 * 1024));
    launch_pdl(q4_one_kernel<TS, ZEROS, LOG>, grid, kThreads, one_smem(a.w.slabs, 128 >> LOG).all, s, a);
  } else {
    static PerContext allowed;
    const size_t smem = (size_t)a.w.slabs * (512 * a.m + 4 * kPackedRows * (ZEROS ? 5 : 1)) + 48 +
                        (a.kw == 1 ? 0 : 8 * kPackedRows * 33 * sizeof(float));
    ACID_TRY(allow_smem(allowed, q4_few_kernel<TS, ZEROS, LOG>, 110 * 1024));
    launch_pdl(q4_few_kernel<TS, ZEROS, LOG>, grid, kThreads, smem, s, a);
  }
  ACID_CHECK_LAUNCH();
  return ACID_OK;
}
template <typename TS, bool ZEROS>
acid_status launch_few(const Fwd& a, cudaStream_t s) {
  return a.w.group_log == 5   ? launch_few<TS, ZEROS, 5>(a, s)
         : a.w.group_log == 6 ? launch_few<TS, ZEROS, 6>(a, s)
                              : launch_few<TS, ZEROS, 7>(a, s);
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
  const int64_t units = kThreads / 4, all = (w.n * w.slabs + units - 1) / units;  // 128 columns of a row, by four threads
  const int64_t most = (int64_t)num_sms() * (w_dtype == ACID_BF16 ? 3 : 2), turns = (all + most - 1) / most;
  const unsigned grid = (unsigned)((all + turns - 1) / turns);
  const int64_t step = grid * units, rows = step / w.slabs;
  const int slabs = (int)(step - rows * w.slabs);
  auto packed = static_cast<uint32_t*>(const_cast<void*>(weight->packed));
  auto scales = const_cast<void*>(weight->scales);
  auto zeros = const_cast<uint8_t*>(weight->zeros);
  auto launch = [&](auto* src, auto* sc) {
    using TW = std::remove_const_t<std::remove_pointer_t<decltype(src)>>;
    using TS = std::remove_pointer_t<decltype(sc)>;
    auto with = [&](auto log) {
      constexpr int LOG = decltype(log)::value;
      launch_pdl(zeros != nullptr ? q4_quantize_kernel<TW, TS, true, LOG> : q4_quantize_kernel<TW, TS, false, LOG>, grid,
                 kThreads, 0, s, src, ldw, w, packed, sc, zeros, wide, rows, slabs);
    };
    w.group_log == 5   ? with(std::integral_constant<int, 5>())
    : w.group_log == 6 ? with(std::integral_constant<int, 6>())
                       : with(std::integral_constant<int, 7>());
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
  const Q4 w = q4_args(*weight);
  const size_t need = fwd_bytes(w, M);
  ACID_REQUIRE(need == 0 || (ws != nullptr && aligned(ws, 16)), ACID_ERR_WORKSPACE,
               "acid_q4_linear_forward: workspace null or not 16-byte aligned");
  ACID_REQUIRE(ws_bytes >= need, ACID_ERR_WORKSPACE,
               "acid_q4_linear_forward: workspace too small (need " + std::to_string(need) + ")");
  Fwd a{w, x, ldx, M, x_dtype, silu_input != 0, out_dtype, bias, out, ldo, nullptr, nullptr, 1};
  cudaStream_t s = (cudaStream_t)stream;
  if (need != 0) return q4_rows_forward(a, ws, weight->scale_dtype, s);
  const bool h = weight->scale_dtype == ACID_BF16;
  if (weight->zeros != nullptr) return h ? launch_few<bf16, true>(a, s) : launch_few<float, true>(a, s);
  return h ? launch_few<bf16, false>(a, s) : launch_few<float, false>(a, s);
}

extern "C" acid_status acid_q4_linear_forward_workspace_size(const acid_q4_weight* weight, int64_t M, size_t* bytes) {
  clear_error();
  ACID_TRY(check_weight(weight));
  ACID_REQUIRE(bytes != nullptr && M >= 0 && M <= kMostRows, ACID_ERR_INVALID_ARG,
               "acid_q4_linear_forward_workspace_size: bad argument");
  *bytes = fwd_bytes(q4_args(*weight), M);
  return ACID_OK;
}

extern "C" acid_status acid_q4_linear_workspace_size(const acid_q4_weight* weight, int64_t M, size_t* bytes) {
  clear_error();
  ACID_TRY(check_weight(weight));
  ACID_REQUIRE(bytes != nullptr && M >= 0 && M <= kMostRows, ACID_ERR_INVALID_ARG,
               "acid_q4_linear_workspace_size: bad argument");
  *bytes = workspace_bytes(q4_args(*weight), M);
  return ACID_OK;
}

extern "C" acid_status acid_q4_linear_backward(int32_t g_dtype, const void* g, int64_t ldg, int64_t M,
                                               const acid_q4_weight* weight, int32_t x_dtype, const void* x,
                                               int64_t ldx, int32_t silu_input, void* dx, int64_t lddx, float* dbias,
                                               void* ws, size_t ws_bytes, acid_stream_t stream) {
  clear_error();
  ACID_TRY(check_weight(weight));
  ACID_REQUIRE(M >= 0 && M <= kMostRows, ACID_ERR_INVALID_ARG, "acid_q4_linear_backward: need 0 <= M <= 32768");
  ACID_REQUIRE(M == 0 || dx != nullptr || dbias != nullptr, ACID_ERR_INVALID_ARG,
               "acid_q4_linear_backward: need dx or dbias");
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
    const size_t need = workspace_bytes(q4_args(*weight), M);
    ACID_REQUIRE(ws_bytes >= need, ACID_ERR_WORKSPACE,
                 "acid_q4_linear_backward: workspace too small (need " + std::to_string(need) + ")");
  }
  const Q4Bwd a{q4_args(*weight), g, x, ldg, ldx, M, g_dtype, x_dtype, weight->scale_dtype, silu_input != 0, dx, lddx, dbias};
  return q4_backward(a, ws, s);
}
