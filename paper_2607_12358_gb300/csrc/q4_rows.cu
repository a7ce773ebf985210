// 4-bit weights against many rows (tens of timestep embeddings: frames, branches
// or steps): the product and its input gradient on tcgen05; the gradient of one row.
#include <algorithm>
#include <string>
#include <type_traits>

#include "q4.cuh"

namespace acid {

unsigned int take_device_error_q4_rows();
BoundsRecord take_bounds_q4_rows();
ACID_DEVICE_FLAG_READER(take_device_error_q4_rows)
ACID_BOUNDS_READER(take_bounds_q4_rows)

namespace {

using bf16 = __nv_bfloat16;
constexpr int kThreads = 256;

// Instruction descriptor of kind::f16 with fp16 A and B, fp32 accumulator.
__host__ __device__ constexpr uint32_t idesc_f16_f32(int M, int N, bool b_mn) {
  return (1u << 4) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
// One arrival for the warp, after what all its lanes did.
__device__ __forceinline__ void arrive_warp(uint64_t* bar, bool leader) {
  __syncwarp();
  if (leader) mbar_arrive(bar);
}
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                   smem_u32(dst)),
               "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

// How a value s (q - z) enters the gradient's product, by what its bits need.
enum Values {
  kOneHalf,     // bf16 scale, z = 8: 8 bits times 3 (q - 8 is -8 .. 7): exact in a half
  kTwoHalves,   // bf16 scale, any z: 12 bits: a half and what is left of it
  kThreeTerms   // fp32 scale, itself two halves sh + sl
};
// A word's eight columns: the product with sh rounded to a half, and what is left of
// it (exact: sh (q - z) has 15 bits at most) with sl's part: 22 bits together.
template <Values KIND>
__device__ __forceinline__ void scaled_halves(uint32_t word, uint32_t z1, uint32_t z64, uint32_t sh, uint32_t sl,
                                              uint32_t (&hi)[4], uint32_t (&lo)[4]) {
  uint32_t d[4];
  halves_of(word, z1, z64, d);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const __half2 c = half2_of(d[j]), h = __hmul2(c, half2_of(sh));
    hi[j] = bits(h);
    if constexpr (KIND != kOneHalf) {
      __half2 l = __hfma2(c, half2_of(sh), __hneg2(h));
      if constexpr (KIND == kThreeTerms) l = __hfma2(c, half2_of(sl), l);
      lo[j] = bits(l);
    }
  }
}
// sh and, in the upper half, sl of a scale after its power of two.
__device__ __forceinline__ uint32_t split_scale(float s) {
  const __half h = __float2half_rn(s);
  return bits(__halves2half2(h, __float2half_rn(s - __half2float(h))));
}
// The power of two that brings the largest scale, `top` in bits, to 2^10 .. 2^11 (2^127
// at most): values below 2^15, and what is left of them far above a half's least.
__device__ __forceinline__ float up_to_scale(uint32_t top) {
  return __uint_as_float((uint32_t)min(264 - (int)(top >> 23), 254) << 23);
}
__device__ __forceinline__ uint32_t finite_bits(float v) { return isfinite(v) ? __float_as_uint(fabsf(v)) : 0u; }

// ------------------------------------------------------------------ product
// D[128 rows of the weight, 16 NB] = codes x parts^T for each group of columns, the
// codes as the exact halves q - z in tensor memory (a row to a lane, where the lane's
// threads write them), the parts of a(x) in shared memory (16 NB rows of high parts,
// then of low parts, which go first into the same sums).  The same threads read the
// group's sums back and add them in fp32 to the row's totals, times its scale.  (The scale as part of the operand, a
// value in two halves, would spare that only where sums may stay in tensor memory: the
// tensor cores' sums lose up to 2^-23 of themselves at each addition, always towards
// zero, 1.7e-4 over 65536 columns.  It costs more instructions and twice the MMAs.)
//   A CTA has two tiles of 128 rows, or one.  Each of their lanes belongs to two threads,
// which take the codes of every other slab of 128 columns (with half of each slab's the
// same waits and fences came twice as often) and half of the columns of all sums.  The
// chain of waits from a slab's codes to its sums bounds it, then the instructions that
// make the operands.  34 rows, 36864 x 3072: groups of 128 27 us (35% of a copy's rate), of
// 64 33 us, of 32 56 us; 8 rows 23 us; 18432 x 3072, groups of 64 22 us.  (One thread
// issuing for both tiles in steps of 64 columns, two tiles always: 37, 44, 75, 32, 43 us.)
constexpr int kFwdRing = 4;   // slabs of parts in shared memory
constexpr int kCodeRing = 2;  // a warp's slabs of its 32 rows of codes
// Bytes of a slab's parts: two boxes of 64 columns, rows of 128 bytes whose
// 16-byte units are swizzled as the tensor cores read them.
template <int NB>
constexpr int kSlabBytes = 32 * NB * 256;
template <int NB>
constexpr int kFwdSmem = kFwdRing * kSlabBytes<NB> + 16 * kCodeRing * 2048 + 512 + 1024;
// Of a CTA with so many tiles: to each eight warps that make operands and one for MMAs; one that copies parts.
constexpr int fwd_threads(int tiles) { return (9 * tiles + 1) * 32; }

// One CTA to a row of a(x).
constexpr int kPartThreads = 512;
template <int NB>
__global__ void __launch_bounds__(kPartThreads) q4_parts_kernel(Q4Fwd a) {
  __shared__ uint32_t largest;
  pdl_wait();
  pdl_trigger();
  const int64_t m = blockIdx.x, chunk = m / kQ4Chunk;
  const int n = (int)(m - chunk * kQ4Chunk), octets = a.w.slabs * 16;
  if (threadIdx.x == 0) largest = 0;
  __syncthreads();
  float v[8], top = 0.f;
  for (int o = threadIdx.x; o < octets; o += kPartThreads) top = fmaxf(top, octet_values(a, m, o * 8, v));
  const uint32_t t = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
  if ((threadIdx.x & 31) == 0) atomicMax(&largest, t);
  __syncthreads();
  const float by = up_to_half(__uint_as_float(largest));
  if (threadIdx.x == 0) a.back[m] = 1.f / by;
  for (int o = threadIdx.x; o < octets; o += kPartThreads) {
    if (octets > kPartThreads) octet_values(a, m, o * 8, v);  // (else they are still there)
    uint4 hi, lo;
    split_octet(v, by, hi, lo);
    const int slab = o >> 4, word = (o >> 2) & 3, unit = (word & 1) * 4 + (o & 3);
    // octets in the order of the codes in a lane: words 32 columns by 32, in them the lanes' quarters
    uint8_t* p = a.parts + (chunk * a.w.slabs + slab) * kSlabBytes<NB> + (word >> 1) * (32 * NB * 128);
    *reinterpret_cast<uint4*>(p + n * 128 + ((unit ^ (n & 7)) << 4)) = hi;
    *reinterpret_cast<uint4*>(p + (16 * NB + n) * 128 + ((unit ^ (n & 7)) << 4)) = lo;
  }
}

template <int NB, int LOG, int TILES>
__global__ void __launch_bounds__(fwd_threads(TILES), 1) q4_rows_forward_kernel(Q4Fwd a, int scale_dtype) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* ring = smem;
  uint8_t* codes = ring + kFwdRing * kSlabBytes<NB>;
  constexpr int kCols = 16 * NB;
  constexpr int kGroups = 128 >> LOG;  // of a slab
  // tensor memory: codes [tile][2 buffers][64], sums [tile][buffers]
  constexpr int kSums = NB <= 2 ? 4 : 2, kDStride = 128 / kSums;
  constexpr uint32_t kACol = 0, kDCol = 256;
  uint64_t* bars = reinterpret_cast<uint64_t*>(codes + 16 * kCodeRing * 2048);
  uint64_t *b_full = bars, *b_empty = bars + kFwdRing;                 // [ring]
  uint64_t *a_full = b_empty + kFwdRing, *a_empty = a_full + 4;        // [tile][2]
  uint64_t *d_full = a_empty + 4, *d_empty = d_full + 2 * kSums;       // [tile][buffer]
  uint64_t* drain = d_empty + 2 * kSums;                               // [tile]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 2);
  const Q4& w = a.w;
  const int warp = warp_index(), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kFwdRing; ++i) {
      mbar_init(&b_full[i], 1);
      mbar_init(&b_empty[i], TILES);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(&a_full[i], 4);
      mbar_init(&a_empty[i], 1);
    }
    for (int i = 0; i < 2 * kSums; ++i) {
      mbar_init(&d_full[i], 1);
      mbar_init(&d_empty[i], 8);
    }
    mbar_init(&drain[0], 1);
    mbar_init(&drain[1], 1);
    mbar_fence_init();
  }
  if (warp == 8 * TILES) tmem_alloc(tmem_slot, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();

  constexpr int kSetRows = 128 * TILES;
  const int64_t sets = (w.n + kSetRows - 1) / kSetRows, chunk = blockIdx.y, m0 = chunk * kQ4Chunk;
  const uint8_t* parts = a.parts + chunk * w.slabs * kSlabBytes<NB>;

  if (warp == 9 * TILES) {
    if (lane == 0) {  // ------------------------------------------ copies of the parts
      int issued = 0;
      bool ok = true;
      for (int64_t set = blockIdx.x; ok && set < sets; set += gridDim.x)
        for (int slab = 0; slab < w.slabs; ++slab, ++issued) {
          const int st = issued % kFwdRing;
          if (issued >= kFwdRing && !mbar_wait(&b_empty[st], (issued / kFwdRing - 1) & 1)) { ok = false; break; }
          mbar_expect_tx(&b_full[st], kSlabBytes<NB>);
          bulk_load(ring + st * kSlabBytes<NB>, parts + (int64_t)slab * kSlabBytes<NB>, kSlabBytes<NB>, &b_full[st]);
        }
      // after a wait ran out: the last copies have landed before the CTA leaves
      if (!ok)
        for (int j = issued > kFwdRing ? issued - kFwdRing : 0; j < issued; ++j)
          mbar_wait(&b_full[j % kFwdRing], (j / kFwdRing) & 1);
    }
  } else if (warp >= 8 * TILES) {
    // ------------------------------------------------------------- MMA issuers, a tile each
    if (elect_one()) {
      const int tile = warp - 8 * TILES;
      constexpr uint32_t idesc = idesc_f16_f32(128, kCols, false);
      const uint64_t bdesc = smem_desc_sw128(smem_u32(ring), 16, 1024);
      bool ok = true;
      uint32_t v = 0, e = 0;  // slabs, groups
      for (int64_t set = blockIdx.x; ok && set < sets; set += gridDim.x)
        for (int slab = 0; ok && slab < w.slabs; ++slab, ++v) {
          const int st = v % kFwdRing, ab = tile * 2 + (v & 1);
          ok = mbar_wait(&b_full[st], (v / kFwdRing) & 1) && mbar_wait(&a_full[ab], (v >> 1) & 1);
          const uint64_t slot = bdesc + (uint64_t)((st * kSlabBytes<NB>) >> 4);
#pragma unroll
          for (int g = 0; g < kGroups; ++g, ++e) {
            const int db = tile * kSums + e % kSums;
            if (ok && e >= kSums) ok = mbar_wait(&d_empty[db], (e / kSums - 1) & 1);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int part = 1; part >= 0; --part)  // the low parts first, on smaller sums
#pragma unroll
              for (int k = g * (8 / kGroups); k < (g + 1) * (8 / kGroups); ++k)  // 16 columns of the slab
                mma_bf16_ts(tmem + kDCol + db * kDStride, tmem + kACol + ab * 64 + k * 8,
                            slot + (uint64_t)(((k >> 2) * (2 * kCols * 128) + part * (kCols * 128) + (k & 3) * 32) >> 4), idesc,
                            part == 0 || k != g * (8 / kGroups));
            mma_commit(&d_full[db]);
          }
          if (ok) {
            mma_commit(&a_empty[ab]);
            mma_commit(&b_empty[st]);
          }
        }
      if (!ok) {
        mma_commit(&drain[tile]);
        mbar_wait(&drain[tile], 0);
      }
    }
    __syncwarp();
  } else {
    // ------------------- codes into tensor memory, sums out of it: warps 0-7 tile 0, 8-15 tile 1; in a tile two warps
    // to a quarter of the lanes, which take every other slab's codes and share the columns of all sums
    const int tile = warp >> 3, half = (warp >> 2) & 1;
    const bool leader = elect_one();
    const uint32_t quad = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t c_addr = tmem + quad + kACol + tile * 128 + half * 64;
    const uint32_t d_addr = tmem + quad + kDCol + tile * 128 + half * 8 * NB;
    uint64_t *my_full = &a_full[tile * 2 + half], *my_empty = &a_empty[tile * 2 + half];
    uint8_t* mine = codes + warp * kCodeRing * 2048;
    const int row_in_set = tile * 128 + (warp & 3) * 32;
    // A lane copies 16 bytes of four of the warp's 32 rows (64 bytes of a row together) and reads its own row back; the
    // units change places from pair to pair of rows, so that eight rows' reads lie in different banks.
    auto place = [](int row, int unit) { return row * 64 + ((unit ^ ((row >> 1) & 3)) << 4); };
    int64_t fset = blockIdx.x;
    int fslab = 0, fst = 0, st = 0;
    const uint32_t* src[4] = {};
    auto aim = [&] {  // the copies' rows in set fset; those past the end are the last one
#pragma unroll
      for (int q = 0; q < 4; ++q)
        src[q] = w.packed + min(fset * kSetRows + row_in_set + (lane >> 2) + 8 * q, w.n - 1) * w.slabs * 16 + 4 * (lane & 3);
    };
    // The warp's next slab: every other one of all that the CTA has.
    auto forward = [&](int by) {
      fslab += by;
      while (fslab >= w.slabs && fset < sets) {
        fslab -= w.slabs;
        fset += gridDim.x;
        aim();
      }
    };
    aim();
    forward(half);
    auto copy = [&] {
      if (fset < sets) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t* from = src[q] + fslab * 16;
          const bool in = ACID_IN_BOUNDS(kSiteQ4, from - w.packed + 3, w.n * w.slabs * 16);
          cp_async<16>(mine + fst * 2048 + place((lane >> 2) + 8 * q, lane & 3), in ? from : w.packed, in);
        }
        forward(2);
      }
      cp_async_commit();
      fst ^= 1;
    };
    copy();
    copy();
    bool ok = true;
    uint32_t v = 0, taken = 0;  // slabs; groups whose sums were read back
    constexpr int kEarly = kGroups > kSums ? kGroups - kSums : 0;
    uint64_t total[NB][4];  // pairs of the row's sums: half of the columns
    // Adds the oldest group's sums, whose scale is s.
    auto take = [&](float s) {
      const int db = taken % kSums;
      ok = mbar_wait_warp(&d_full[tile * kSums + db], (taken / kSums) & 1);
      ++taken;
      if (!ok) return;
      tc_fence_after();
      const uint64_t s2 = f2_pack(s, s);
      uint32_t r[NB][8];
#pragma unroll
      for (int n = 0; n < NB; ++n) tmem_ld8(d_addr + db * kDStride + n * 8, r[n]);
      tmem_wait_ld();
      tc_fence_before();
      arrive_warp(&d_empty[tile * kSums + db], leader);
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          total[n][e] = f2_fma(s2, f2_pack(__uint_as_float(r[n][2 * e]), __uint_as_float(r[n][2 * e + 1])), total[n][e]);
    };
    for (int64_t set = blockIdx.x; ok && set < sets; set += gridDim.x) {
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) total[n][e] = 0;
      const int64_t row = set * kSetRows + row_in_set + lane, at = min(row, w.n - 1) * w.groups;
      // scales and zero points of a slab's groups, a slab ahead
      float scales[kGroups];
      uint8_t zeros[kGroups];
      auto look = [&](int slab) {
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
          const int64_t p = at + min(slab * kGroups + i, w.groups - 1);
          if (!ACID_IN_BOUNDS(kSiteQ4, p, w.n * w.groups)) continue;
          scales[i] = value_at(scale_dtype, w.scales, p);
          if (w.zeros != nullptr) zeros[i] = w.zeros[p];
        }
      };
      look(0);
      float s[kGroups] = {};
      for (int slab = 0; ok && slab < w.slabs; ++slab, ++v) {
        float before[kGroups];  // the scales of the slab whose sums are not taken yet
        uint32_t z1[kGroups], z64[kGroups];
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
          const uint32_t z = (w.zeros != nullptr ? zeros[i] & 15u : 8u) * 0x00010001u;
          before[i] = s[i];
          s[i] = scales[i];
          z1[i] = 0x64006400u | z;
          z64[i] = 0x54005400u | z << 4;
        }
        if (slab + 1 < w.slabs) look(slab + 1);
        // the sums of the slab before, while this one's are formed: the groups whose buffers that slab's others wait for
        // come ahead of the codes
        if (slab > 0)
#pragma unroll
          for (int i = 0; i < kEarly; ++i)
            if (ok) take(before[i]);
        if (!ok) break;
        if ((v & 1) == half) {
          cp_async_wait<kCodeRing - 1>();
          __syncwarp();
          uint4 q[4];  // words of the columns 32 i + 8 c
#pragma unroll
          for (int c = 0; c < 4; ++c) q[c] = *reinterpret_cast<const uint4*>(mine + st * 2048 + place(lane, c));
          __syncwarp();
          copy();
          st ^= 1;
          if (v >= 2) ok = mbar_wait_warp(my_empty, ((v >> 1) - 1) & 1);
          if (!ok) break;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int of = i >> (LOG - 5);
            uint32_t d[16];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              uint32_t x[4];
              halves_of(i == 0 ? q[c].x : i == 1 ? q[c].y : i == 2 ? q[c].z : q[c].w, z1[of], z64[of], x);
#pragma unroll
              for (int j = 0; j < 4; ++j) d[4 * c + j] = x[j];
            }
            tmem_st16(c_addr + i * 16, d);
          }
          tmem_wait_st();
          tc_fence_before();
          arrive_warp(my_full, leader);
        }
        if (slab > 0)
#pragma unroll
          for (int i = kEarly; i < kGroups; ++i)
            if (ok) take(before[i]);
      }
#pragma unroll
      for (int i = 0; i < kGroups; ++i)
        if (ok) take(s[i]);
      if (!ok || row >= w.n) continue;
      const float bias = a.bias != nullptr ? a.bias[row] : 0.f;
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int64_t m = m0 + 8 * (half * NB + n) + 2 * e;
          float x, y;
          f2_unpack(total[n][e], x, y);
          if (m < a.m) put_value(a.out_dtype, a.out, m * a.ldo + row, fmaf(x, a.back[m], bias));
          if (m + 1 < a.m) put_value(a.out_dtype, a.out, (m + 1) * a.ldo + row, fmaf(y, a.back[m + 1], bias));
        }
    }
    cp_async_wait<0>();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 8 * TILES) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// ----------------------------------------------------------- input gradient
// D[2 x 64 parts of g, 128 columns] += parts x values for 128 rows of the weight at a
// time.  The parts of g (row m: lane m its high halves, lane 64 + m its low halves)
// come from q4_back_parts_kernel and go to tensor memory; the values, two halves
// each, are written to shared memory, where they are the second operand as they lie
// (columns together).  A block's sums are read back and added up in fp32, as in the
// product, while the next block's are formed.
//   A block's values are 64 KB written to shared memory and 64 KB read, and its MMAs take
// 1024 clocks; the instructions that make the values and the chain of waits around them
// bound it, at about twice that: 34 rows, 18432 x 3072, groups of 64 with fp32 scales and
// zero points 40 us, 36864 x 3072, groups of 128 with bf16 scales 54 us, with the kernels
// before and after it.  (The scales, a line of memory to each row, loaded by the warps
// that use them: 47 and 69 us.)
constexpr int kBackThreads = 640;  // 16 warps that make operands and read sums, one for MMAs, one for g's parts, two for scales
constexpr int kBackRing = 3;  // blocks of a warp's eight rows of codes
struct BackSmem {
  static constexpr int kPart = 128 * 256;    // [box of 64 columns][128 rows][128 bytes]
  static constexpr int kBuffer = 2 * kPart;  // high, low
  static constexpr int kParts = 16 * 2 * kQ4Chunk * 16;  // a block of g's parts
  static constexpr int kOffParts = 2 * kBuffer, kOffCodes = kOffParts + 2 * kParts;
  static constexpr int kOffScales = kOffCodes + 16 * kBackRing * 512;  // of two blocks
  static constexpr int kOffBar = kOffScales + 2 * 128 * 4 * 8, kBytes = kOffBar + 256 + 1024;
};
constexpr int kTopRuns = 32;  // parts of a share's scales that are scanned by a CTA each

// What each addition rounds off is added up beside the sum (exact: the difference of the
// operands' and the sum's parts), so that terms that cancel leave a sum as good as its terms.
__device__ __forceinline__ void bias_of(const Q4Bwd& a, int64_t n) {
  float sum = 0.f, off = 0.f;
#pragma unroll 8
  for (int64_t m = 0; m < a.m; ++m) {
    const float v = value_at(a.g_dtype, a.g, m * a.ldg + n), t = sum + v, part = t - sum;
    off += (sum - (t - part)) + (v - part);
    sum = t;
  }
  a.dbias[n] = isfinite(sum) ? sum + off : sum;
}
// The bias's gradient alone.
__global__ void __launch_bounds__(kThreads) q4_bias_kernel(Q4Bwd a) {
  pdl_wait();
  for (int64_t n = (int64_t)blockIdx.x * kThreads + threadIdx.x; n < a.w.n; n += (int64_t)gridDim.x * kThreads) bias_of(a, n);
}

// For each share of the weight's rows (blockIdx.x): the parts of a row of g, after
// a power of two of the row and share (y < m); the largest scale of a part of the share
// (the next kTopRuns); the bias's gradient of 256 rows (the rest).  What is not finite in g
// has parts of 0 (an infinity times a value's low half, mostly 0, would be NaN): the power
// of two is negative then, and plain_gradient adds it.
//   parts: [chunk][run of 8 rows of the weight][2][rows of the chunk][8]
__global__ void __launch_bounds__(kThreads) q4_back_parts_kernel(Q4Bwd a) {
  __shared__ uint32_t largest;
  __shared__ bool odd;
  pdl_wait();
  const int64_t begin = blockIdx.x * a.per, end = min(a.w.n, begin + a.per), y = blockIdx.y;
  if (y >= a.m + kTopRuns) {
    const int64_t step = (gridDim.y - a.m - kTopRuns) * kThreads;
    for (int64_t n = begin + (y - a.m - kTopRuns) * kThreads + threadIdx.x; n < end; n += step) bias_of(a, n);
    return;
  }
  if (threadIdx.x == 0) {
    largest = 0;
    odd = false;
  }
  __syncthreads();
  uint32_t top = 0;
  auto join = [&] {
    top = __reduce_max_sync(0xffffffffu, top);
    if ((threadIdx.x & 31) == 0) atomicMax(&largest, top);
    __syncthreads();
  };
  if (y >= a.m) {
    const int64_t run = y - a.m, all = (end - begin) * a.w.groups, per = (all + kTopRuns - 1) / kTopRuns;
    const int64_t i0 = begin * a.w.groups + run * per, i1 = begin * a.w.groups + min(all, (run + 1) * per);
#pragma unroll 8
    for (int64_t i = i0 + threadIdx.x; i < i1; i += kThreads)
      if (ACID_IN_BOUNDS(kSiteQ4, i, a.w.n * a.w.groups)) top = max(top, finite_bits(value_at(a.scale_dtype, a.w.scales, i)));
    join();
    if (threadIdx.x == 0) a.top[blockIdx.x * kTopRuns + run] = largest;
    return;
  }
  const int64_t m = y, chunk = m / kQ4Chunk, rows = min((int64_t)kQ4Chunk, a.m - chunk * kQ4Chunk), r = m - chunk * kQ4Chunk;
#pragma unroll 8
  for (int64_t n = begin + threadIdx.x; n < end; n += kThreads) {
    const float v = value_at(a.g_dtype, a.g, m * a.ldg + n);
    top = max(top, finite_bits(v));
    if (!isfinite(v)) odd = true;
  }
  join();
  const float up = up_to_half(__uint_as_float(largest));
  if (threadIdx.x == 0) a.back[blockIdx.x * a.m + m] = odd ? -1.f / up : 1.f / up;
  // runs of eight rows of the weight; the last block of a share is filled with zeros
  const int64_t runs = (min(begin + a.per, (a.w.n + 127) / 128 * 128) - begin) / 8, all_runs = (a.w.n + 127) / 128 * 16;
  for (int64_t i = threadIdx.x; i < runs; i += kThreads) {
    const int64_t n0 = begin + i * 8;
    uint32_t h[4], l[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float v0 = n0 + 2 * j < end ? value_at(a.g_dtype, a.g, m * a.ldg + n0 + 2 * j) * up : 0.f;
      float v1 = n0 + 2 * j + 1 < end ? value_at(a.g_dtype, a.g, m * a.ldg + n0 + 2 * j + 1) * up : 0.f;
      if (!isfinite(v0)) v0 = 0.f;
      if (!isfinite(v1)) v1 = 0.f;
      const __half2 p = __floats2half2_rn(v0, v1);
      const float2 f = __half22float2(p);
      h[j] = bits(p);
      l[j] = bits(__floats2half2_rn(v0 - f.x, v1 - f.y));
    }
    uint4* out = reinterpret_cast<uint4*>(a.parts) + chunk * all_runs * 2 * kQ4Chunk + (n0 / 8) * 2 * rows + r;
    out[0] = make_uint4(h[0], h[1], h[2], h[3]);
    out[rows] = make_uint4(l[0], l[1], l[2], l[3]);
  }
}

// Column c of row m of g W over a share's rows of the weight, value by value: all of them, or those of g that are not
// finite alone.
__device__ __noinline__ float plain_gradient(const Q4Bwd& a, int64_t m, int c, int64_t begin, int64_t end, bool all) {
  const Q4& w = a.w;
  const int in_slab = c & 127, word = (c >> 7) * 16 + 4 * (in_slab % 32 / 8) + in_slab / 32, shift = 4 * (c % 8);
  float sum = 0.f, part = 0.f;
  for (int64_t n = begin; n < end && !isnan(sum + part); ++n) {
    const float v = value_at(a.g_dtype, a.g, m * a.ldg + n);
    if (!all && isfinite(v)) continue;
    const int64_t i = n * w.groups + (c >> w.group_log), p = n * w.slabs * 16 + word;
    if (!ACID_IN_BOUNDS(kSiteQ4, i, w.n * w.groups) || !ACID_IN_BOUNDS(kSiteQ4, p, w.n * w.slabs * 16)) continue;
    const int z = w.zeros != nullptr ? w.zeros[i] : 8;
    part += v * (value_at(a.scale_dtype, w.scales, i) * (float)((int)(w.packed[p] >> shift & 15u) - z));
    if ((n & 63) == 63) {
      sum += part;
      part = 0.f;
    }
  }
  return sum + part;
}

template <Values KIND, int LOG>
__global__ void __launch_bounds__(kBackThreads, 1) q4_rows_backward_kernel(Q4Bwd a) {
  using TS = std::conditional_t<KIND == kThreeTerms, float, bf16>;
  constexpr int kGroups = 128 >> LOG;
  extern __shared__ uint8_t smem_raw[];
  using L = BackSmem;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::kOffBar);
  uint64_t *full = bars, *empty = bars + 2, *d_empty = bars + 4, *p_full = bars + 6, *p_empty = bars + 8, *s_full = bars + 10;  // [buffer]
  uint64_t* drain = bars + 12;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 13);
  const Q4& w = a.w;
  const int warp = warp_index(), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&full[i], 16);
      mbar_init(&empty[i], 1);
      mbar_init(&d_empty[i], 16);
      mbar_init(&p_full[i], 1);
      mbar_init(&p_empty[i], 16);
      mbar_init(&s_full[i], 2);
    }
    mbar_init(drain, 1);
    mbar_fence_init();
  }
  if (warp == 16) tmem_alloc(tmem_slot, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();

  const int slab = blockIdx.x;
  const int64_t begin = blockIdx.y * a.per, end = min(w.n, begin + a.per), chunk = blockIdx.z, m0 = chunk * kQ4Chunk;
  const int rows = (int)min((int64_t)kQ4Chunk, a.m - m0), blocks = (int)((end - begin + 127) / 128);
  constexpr uint32_t kDCol = 0, kACol = 256;  // tensor memory: sums [2 buffers][128], parts [2 buffers][64]
  const float one = up_to_scale(__reduce_max_sync(0xffffffffu, a.top[blockIdx.y * kTopRuns + lane]));

  const int64_t all_runs = (w.n + 127) / 128 * 16;
  if (warp == 17) {
    if (lane == 0) {  // ------------------------------------------ copies of g's parts
      const uint8_t* src = a.parts + (chunk * all_runs * 2 * kQ4Chunk + begin / 8 * 2 * rows) * 16;
      const uint32_t bytes = 16 * 2 * rows * 16;
      int b = 0;
      for (; b < blocks; ++b) {
        const int i = b & 1;
        if (b >= 2 && !mbar_wait(&p_empty[i], ((b >> 1) - 1) & 1)) break;
        mbar_expect_tx(&p_full[i], bytes);
        bulk_load(smem + L::kOffParts + i * L::kParts, src + (int64_t)b * bytes, bytes, &p_full[i]);
      }
      // after a wait ran out: the last copies have landed before the CTA leaves
      if (b < blocks)
        for (int j = b > 2 ? b - 2 : 0; j < b; ++j) mbar_wait(&p_full[j & 1], (j >> 1) & 1);
    }
  } else if (warp >= 18) {
    // ------------------- a block's scales in their two halves, and its zero points: half of the rows to a warp, a lane has
    // one of the slab's groups, two blocks ahead in its registers
    constexpr int kMine = 2 * kGroups, kApart = 32 / kGroups;  // rows of a lane, and between them
    struct Look {
      float s[kMine];
      uint8_t z[kMine];
    };
    const int64_t apart = (int64_t)kApart * w.groups;
    int64_t row = begin + (warp - 18) * 64 + lane / kGroups;
    int64_t at = row * w.groups + min(slab * kGroups + lane % kGroups, w.groups - 1);
    auto look = [&](Look& l) {  // the next block's
#pragma unroll
      for (int j = 0; j < kMine; ++j) {
        const bool in = row + j * kApart < w.n;
        const int64_t p = in ? at + j * apart : 0;
        if (!ACID_IN_BOUNDS(kSiteQ4, p, w.n * w.groups)) continue;
        l.s[j] = io<TS>::ld(static_cast<const TS*>(w.scales) + p);
        // (rows past the end meet parts of zero; another row's scale may be far above the share's, and not fit a half)
        if (!in) l.s[j] = 0.f;
        if (KIND != kOneHalf && w.zeros != nullptr) l.z[j] = w.zeros[p];
      }
      row += 128;
      at += (int64_t)128 * w.groups;
    };
    uint2* to = reinterpret_cast<uint2*>(smem + L::kOffScales) + (warp - 18) * 64 * kGroups + lane;
    bool ok = true;
    auto put = [&](Look& l, int b) {
      // (the block before last has been read when its values are there)
      if (b >= 2) ok = mbar_wait_warp(&full[b & 1], ((b >> 1) - 1) & 1);
      if (!ok) return;
#pragma unroll
      for (int j = 0; j < kMine; ++j)
        to[(b & 1) * 128 * kGroups + 32 * j] =
            make_uint2(split_scale(l.s[j] * one), KIND != kOneHalf && w.zeros != nullptr ? l.z[j] & 15u : 8u);
      if (b + 2 < blocks) look(l);
      arrive_warp(&s_full[b & 1], lane == 0);
    };
    Look l[2];
    look(l[0]);
    if (blocks > 1) look(l[1]);
    for (int b = 0; ok && b < blocks; b += 2) {
      put(l[0], b);
      if (ok && b + 1 < blocks) put(l[1], b + 1);
    }
  } else if (warp == 16) {
    // ------------------------------------------------------------- MMA issuer
    const bool leader = elect_one();
    constexpr uint32_t idesc = idesc_f16_f32(128, 128, true);
    const uint64_t bdesc = smem_desc_sw128(smem_u32(smem), L::kPart / 2, 1024);
    bool ok = true;
    for (int b = 0; ok && b < blocks; ++b) {
      const int i = b & 1;
      if (!mbar_wait_warp(&full[i], (b >> 1) & 1)) { ok = false; break; }
      if (b >= 2 && !mbar_wait_warp(&d_empty[i], ((b >> 1) - 1) & 1)) { ok = false; break; }
      tc_fence_after();
      if (leader) {
#pragma unroll
        for (int part = KIND == kOneHalf ? 0 : 1; part >= 0; --part) {  // the low values first, on small sums
          const uint64_t slot = bdesc + (uint64_t)((i * L::kBuffer + part * L::kPart) >> 4);
#pragma unroll
          for (int k = 0; k < 8; ++k)
            mma_bf16_ts(tmem + kDCol + i * 128, tmem + kACol + i * 64 + k * 8, slot + (uint64_t)((k * 16 * 128) >> 4), idesc,
                        (part == 0 && KIND != kOneHalf) || k != 0);
        }
        mma_commit(&empty[i]);
      }
      __syncwarp();
    }
    if (!ok && leader) {
      mma_commit(drain);
      mbar_wait(drain, 0);
    }
  } else {
    // ------------------- a warp's eight rows of a block's values into shared memory, a quarter of its lanes' parts into
    // tensor memory, and a quarter of the columns of their sums out of it
    const int quarter = warp >> 2, m = (warp & 1) * 32 + lane, g = lane >> 2, t = lane & 3, odd = g & 1;
    const bool low = (warp & 2) != 0, active = (warp & 1) * 32 < rows, leader = elect_one();
    const uint32_t quad = (uint32_t)((warp & 3) * 32) << 16;
    uint8_t* mine = smem + L::kOffCodes + warp * kBackRing * 512;
    // a lane's own 16 bytes of its row, some blocks ahead
    int64_t crow = begin + warp * 8 + g;
    const uint32_t* src = w.packed + (crow * w.slabs + slab) * 16 + 4 * t;
    const int64_t src_step = (int64_t)128 * 16 * w.slabs;
    int fetched = 0, fst = 0;
    auto copy = [&] {
      if (fetched < blocks) {
        // (rows past the end, against parts of zero, are the first one)
        const uint32_t* from = crow < w.n ? src : w.packed;
        const bool in = ACID_IN_BOUNDS(kSiteQ4, from - w.packed + 3, w.n * w.slabs * 16);
        cp_async<16>(mine + fst * 512 + lane * 16, in ? from : w.packed, in);
        crow += 128;
        src += src_step;
        ++fetched;
      }
      cp_async_commit();
      fst = fst + 1 == kBackRing ? 0 : fst + 1;
    };
    for (int i = 0; i < kBackRing - 1; ++i) copy();
    bool ok = true;
    int st = 0;
    uint64_t total[16];  // pairs of a quarter of the slab's columns
#pragma unroll
    for (int i = 0; i < 16; ++i) total[i] = 0;
    auto take = [&](int b) {  // the sums of block b
      ok = mbar_wait_warp(&empty[b & 1], (b >> 1) & 1);
      if (!ok) return;
      tc_fence_after();
      if (active) {
        uint32_t r[4][8];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld8(tmem + quad + kDCol + (b & 1) * 128 + quarter * 32 + c * 8, r[c]);
        tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < 16; ++i)
          total[i] = f2_add(total[i], f2_pack(__uint_as_float(r[i >> 2][2 * (i & 3)]), __uint_as_float(r[i >> 2][2 * (i & 3) + 1])));
      }
      tc_fence_before();
      arrive_warp(&d_empty[b & 1], leader);
    };
    auto block = [&](int b) {
      const int i = b & 1;
      if (b >= 2) take(b - 2);  // the tensor cores are done with these buffers
      if (ok) ok = mbar_wait_warp(&p_full[i], (b >> 1) & 1);
      if (!ok) return;
      if (active) {
        const uint4* p = reinterpret_cast<const uint4*>(smem + L::kOffParts + i * L::kParts) +
                         quarter * 4 * 2 * rows + (low ? rows : 0) + min(m, rows - 1);
        uint32_t d[16];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint4 x = p[j * 2 * rows];
          d[4 * j] = x.x;
          d[4 * j + 1] = x.y;
          d[4 * j + 2] = x.z;
          d[4 * j + 3] = x.w;
        }
        tmem_st16(tmem + quad + kACol + i * 64 + quarter * 16, d);
      }
      arrive_warp(&p_empty[i], leader);
      cp_async_wait<kBackRing - 2>();
      const uint4 q = *reinterpret_cast<const uint4*>(mine + st * 512 + lane * 16);
      st = st + 1 == kBackRing ? 0 : st + 1;
      copy();
      uint32_t sh[kGroups], sl[kGroups], z1[kGroups], z64[kGroups];
      ok = mbar_wait_warp(&s_full[i], (b >> 1) & 1);
      if (!ok) return;
#pragma unroll
      for (int v = 0; v < kGroups; ++v) {
        const uint2 x = reinterpret_cast<const uint2*>(smem + L::kOffScales)[(i * 128 + warp * 8 + g) * kGroups + v];
        sh[v] = __byte_perm(x.x, 0, 0x1010);
        sl[v] = __byte_perm(x.x, 0, 0x3232);
        z1[v] = 0x64006400u | x.y * 0x00010001u;
        z64[v] = 0x54005400u | x.y * 0x00100010u;
      }
      // neighbouring rows take their words in another order, so that their units lie in different banks
      const uint4 v = odd ? make_uint4(q.y, q.x, q.w, q.z) : q;
      const int row = warp * 8 + g;
      uint8_t* to = smem + i * L::kBuffer;
      const int at = row * 128 + (((odd * 4 + t) ^ (row & 7)) << 4);  // unit of word 0 or 1
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        // word s ^ odd: its group, and the unit beside the first one's for the second of a box
        const int even_of = s >> (LOG - 5), odd_of = (s ^ 1) >> (LOG - 5);
        const bool other = odd != 0 && even_of != odd_of;
        uint32_t hi[4], lo[4];
        scaled_halves<KIND>(s == 0 ? v.x : s == 1 ? v.y : s == 2 ? v.z : v.w, other ? z1[odd_of] : z1[even_of],
                            other ? z64[odd_of] : z64[even_of], other ? sh[odd_of] : sh[even_of],
                            other ? sl[odd_of] : sl[even_of], hi, lo);
        uint8_t* p = to + (at ^ ((s & 1) * 64)) + (s >> 1) * (L::kPart / 2);
        *reinterpret_cast<uint4*>(p) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        if constexpr (KIND != kOneHalf) *reinterpret_cast<uint4*>(p + L::kPart) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
      }
      tmem_wait_st();
      tc_fence_before();
      fence_proxy_async_smem();
      arrive_warp(&full[i], leader);
    };
    for (int b = 0; ok && b < blocks; ++b) block(b);
    cp_async_wait<0>();
    if (ok && blocks > 1) take(blocks - 2);
    if (ok) take(blocks - 1);
    if (ok && m < rows) {
      const float back = a.back[blockIdx.y * a.m + m0 + m], per_s = 1.f / one;
      const float less = fminf(fabsf(back), per_s), more = fmaxf(fabsf(back), per_s);  // (the other way a large g overflows)
      const int64_t at = ((blockIdx.y * 2 + low) * a.m + m0 + m) * w.slabs * 128 + slab * 128 + quarter * 32;
      if (ACID_IN_BOUNDS(kSiteQ4, at + 31, a.shares * a.m * w.slabs * 128)) {
#pragma unroll
        for (int o = 0; o < 4; ++o) {  // an octet's columns j and j + 4 lie side by side
          float f[8];
#pragma unroll
          for (int j = 0; j < 4; ++j) f2_unpack(total[4 * o + j], f[2 * j], f[2 * j + 1]);
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j] = f[j] * less * more;
          *reinterpret_cast<float4*>(a.part + at + o * 8) = make_float4(f[0], f[2], f[4], f[6]);
          *reinterpret_cast<float4*>(a.part + at + o * 8 + 4) = make_float4(f[1], f[3], f[5], f[7]);
        }
        const int c0 = slab * 128 + quarter * 32;
        if (back < 0.f && !low)
          for (int c = 0; c < min(32, w.k - c0); ++c) a.part[at + c] += plain_gradient(a, m0 + m, c0 + c, begin, end, false);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 16) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// --------------------------------------------- input gradient of one row
// dx of one row of g on the FP32 pipes: a lane takes a row's 32 columns of a slab (16
// bytes), eight rows to a warp, and keeps the columns' sums over its rows.  A code in bits
// 4 e .. 4 e + 3 of the last bits of 2^23 is 16^e q without a conversion; 2^23 + 16^e z is
// taken off (exact), and the column's 16^e at the end.  The lanes', the warps' and
// (q4_backward_join_kernel) the shares' sums are added in order.
//   In the kernel above one row of g fills 2 of 128 lanes, and there are three launches for
// two: 276480 x 1536, groups of 64 with zero points 113 to 119 us over several GPUs (29 to
// 31% of a copy's rate; 194 above), of 128 without 96, 9216 x 1536, groups of 128 10 us (14).
// The instructions bound it, two a code and 50 a row for its scales and places (the integer
// pipe 68% busy, issue 55 to 60%, DRAM 26 to 28%); two rows took as long as above.
constexpr int kOneBackCtas = 2;  // of an SM
template <typename TS, bool ZEROS, int LOG>
__global__ void __launch_bounds__(kThreads, kOneBackCtas) q4_one_backward_kernel(Q4Bwd a) {
  constexpr int kGroups = 128 >> LOG, kAhead = 4;
  __shared__ float red[kThreads / 32][128];
  pdl_wait();
  const Q4& w = a.w;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, slab = blockIdx.x;
  const int64_t begin = blockIdx.y * a.per, end = min(w.n, begin + a.per);
  struct Load {
    uint4 q;
    float s[kGroups], g;
    uint8_t z[kGroups];
  };
  // this lane's next row: rows past the end are the first one against 0
  int64_t row = begin + warp * 8 + g;
  const int64_t q0 = (begin * w.slabs + slab) * 16 + 4 * t, s0 = begin * w.groups;
  int64_t qi = q0 + (int64_t)(warp * 8 + g) * w.slabs * 16, si = s0 + (int64_t)(warp * 8 + g) * w.groups;
  int group[kGroups];
#pragma unroll
  for (int v = 0; v < kGroups; ++v) group[v] = min(slab * kGroups + v, w.groups - 1);
  auto look = [&](Load& l) {
    const bool in = row < end;
    const int64_t q = in ? qi : q0, s = in ? si : s0;
    if (ACID_IN_BOUNDS(kSiteQ4, q + 3, w.n * w.slabs * 16)) {
      const uint32_t* p = w.packed + q;
      asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                   : "=r"(l.q.x), "=r"(l.q.y), "=r"(l.q.z), "=r"(l.q.w)
                   : "l"(p));
    }
#pragma unroll
    for (int v = 0; v < kGroups; ++v) {
      if (!ACID_IN_BOUNDS(kSiteQ4, s + group[v], w.n * w.groups)) continue;
      l.s[v] = io<TS>::ld(static_cast<const TS*>(w.scales) + s + group[v]);
      if constexpr (ZEROS) l.z[v] = w.zeros[s + group[v]];
    }
    l.g = in ? value_at(a.g_dtype, a.g, row) : 0.f;
    row += 64;
    qi += (int64_t)64 * w.slabs * 16;
    si += (int64_t)64 * w.groups;
  };
  constexpr float kOne = 8388608.f;  // 2^23
  const uint64_t one2 = f2_pack(kOne, kOne), minus = f2_pack(-1.f, -1.f);
  // 16^e of a word's pairs of columns: fields 0 .. 4, and 5 .. 7 shifted down
  const uint64_t power[4] = {f2_pack(1.f, 16.f), f2_pack(256.f, 4096.f), f2_pack(65536.f, 1.f), f2_pack(16.f, 256.f)};
  uint64_t sum[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[i][j] = 0;
  auto add = [&](const Load& l) {
    uint64_t off[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int v = i >> (LOG - 5);
      if (i == 0 || (ZEROS && i % (1 << (LOG - 5)) == 0)) {  // -(2^23 + 16^e z)
        const float z = ZEROS ? (float)l.z[v] : 8.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) off[j] = f2_mul(f2_fma(f2_pack(z, z), power[j], one2), minus);
      }
      const float c = l.s[v] * l.g;
      const uint64_t c2 = f2_pack(c, c);
      const uint32_t x = i == 0 ? l.q.x : i == 1 ? l.q.y : i == 2 ? l.q.z : l.q.w, y = x >> 20;
      auto code = [](uint32_t u, int e) { return __uint_as_float((u & (15u << (4 * e))) | 0x4B000000u); };
      const uint64_t q[4] = {f2_pack(code(x, 0), code(x, 1)), f2_pack(code(x, 2), code(x, 3)), f2_pack(code(x, 4), code(y, 0)),
                             f2_pack(code(y, 1), code(y, 2))};
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[i][j] = f2_fma(c2, f2_add(q[j], off[j]), sum[i][j]);
    }
  };
  Load l[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) look(l[i]);
  const int64_t steps = (end - begin + 63) / 64;
  for (int64_t i = 0; i < steps; i += kAhead)
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {  // (steps past the last one add zeros)
      add(l[j]);
      look(l[j]);
    }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float x, y, px, py;
      f2_unpack(sum[i][j], x, y);
      f2_unpack(power[j], px, py);
      x /= px;  // (powers of two)
      y /= py;
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        x += __shfl_xor_sync(0xffffffffu, x, o);
        y += __shfl_xor_sync(0xffffffffu, y, o);
      }
      if (g == 0) {
        red[warp][32 * i + 8 * t + 2 * j] = x;
        red[warp][32 * i + 8 * t + 2 * j + 1] = y;
      }
    }
  __syncthreads();
  if (threadIdx.x < 128) {
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) v += red[i][threadIdx.x];
    // (16^e times a sum may pass the largest number where the sum does not)
    if (!isfinite(v) && slab * 128 + threadIdx.x < w.k) v = plain_gradient(a, 0, slab * 128 + threadIdx.x, begin, end, true);
    const int64_t at = ((int64_t)blockIdx.y * w.slabs + slab) * 128 + threadIdx.x;
    if (ACID_IN_BOUNDS(kSiteQ4, at, (int64_t)a.shares * w.slabs * 128)) a.part[at] = v;
  }
  if (a.dbias != nullptr && slab == 0)
    for (int64_t n = begin + threadIdx.x; n < end; n += kThreads) bias_of(a, n);
}

// Joins the shares in their order and takes the activation's gradient.
__global__ void __launch_bounds__(128) q4_backward_join_kernel(Q4Bwd a) {
  pdl_wait();
  const int c = blockIdx.x * 128 + threadIdx.x;
  const int64_t m = blockIdx.y, width = (int64_t)a.w.slabs * 128;
  if (c >= a.w.k) return;
  float v = 0.f;
#pragma unroll 8
  for (int b = 0; b < a.shares; ++b) v += a.part[(b * a.m + m) * width + c];
  if (a.silu) {
    const float x = value_at(a.x_dtype, a.x, m * a.ldx + c), e = 1.f / (1.f + expf(-x));
    v *= e * (1.f + x * (1.f - e));
  }
  put_value(a.x_dtype, a.dx, m * a.lddx + c, v);
}

// --------------------------------------------------------------------- host
// Sixteens of rows of x that the product's kernel takes at a time.
int sixteens_of(int64_t m) { return (int)((std::min<int64_t>(m, kQ4Chunk) + 15) / 16); }
int64_t chunks_of(int64_t m) { return (m + kQ4Chunk - 1) / kQ4Chunk; }

template <int NB, int LOG, int TILES>
acid_status launch_forward(const Q4Fwd& a, int scale_dtype, cudaStream_t s) {
  static PerContext allowed;
  ACID_TRY(allow_smem(allowed, q4_rows_forward_kernel<NB, LOG, TILES>, kFwdSmem<NB>));
  const int64_t sets = (a.w.n + 128 * TILES - 1) / (128 * TILES);
  const dim3 grid((unsigned)std::min<int64_t>(sets, num_sms()), (unsigned)chunks_of(a.m));
  launch_pdl(q4_rows_forward_kernel<NB, LOG, TILES>, grid, fwd_threads(TILES), kFwdSmem<NB>, s, a, scale_dtype);
  ACID_CHECK_LAUNCH();
  return ACID_OK;
}
// One tile to a CTA where every tile has an SM to itself (34 rows, 4608 x 3072, groups of
// 64: 21 us, with two tiles 32), else two (36864 x 3072, groups of 128 27 us, one by one 33).
template <int NB, int LOG>
acid_status launch_forward(const Q4Fwd& a, int scale_dtype, cudaStream_t s) {
  return (a.w.n + 127) / 128 <= num_sms() ? launch_forward<NB, LOG, 1>(a, scale_dtype, s)
                                          : launch_forward<NB, LOG, 2>(a, scale_dtype, s);
}
template <int NB>
acid_status launch_forward(const Q4Fwd& a, int scale_dtype, cudaStream_t s) {
  launch_pdl(q4_parts_kernel<NB>, (unsigned)a.m, kPartThreads, 0, s, a);
  ACID_CHECK_LAUNCH();
  return a.w.group_log == 5   ? launch_forward<NB, 5>(a, scale_dtype, s)
         : a.w.group_log == 6 ? launch_forward<NB, 6>(a, scale_dtype, s)
                              : launch_forward<NB, 7>(a, scale_dtype, s);
}

template <Values KIND, int LOG>
acid_status launch_backward(const Q4Bwd& a, cudaStream_t s) {
  static PerContext allowed;
  ACID_TRY(allow_smem(allowed, q4_rows_backward_kernel<KIND, LOG>, BackSmem::kBytes));
  const dim3 grid(a.w.slabs, (unsigned)((a.w.n + a.per - 1) / a.per), (unsigned)chunks_of(a.m));
  launch_pdl(q4_rows_backward_kernel<KIND, LOG>, grid, kBackThreads, BackSmem::kBytes, s, a);
  ACID_CHECK_LAUNCH();
  return ACID_OK;
}
template <Values KIND>
acid_status launch_backward(const Q4Bwd& a, cudaStream_t s) {
  return a.w.group_log == 5   ? launch_backward<KIND, 5>(a, s)
         : a.w.group_log == 6 ? launch_backward<KIND, 6>(a, s)
                              : launch_backward<KIND, 7>(a, s);
}

// Rows of the weight to a CTA of the gradient, in whole blocks of 128, and the
// CTAs that share a slab's rows: as many CTAs as an SM each has.  (152 and not the device's
// SMs: the workspace and the order of the sums go by the weight's shape alone.)
int64_t share_rows(const Q4& w) {
  const int64_t want = std::max(1, 152 / w.slabs), per = (w.n + want - 1) / want;
  return (per + 127) / 128 * 128;
}
int64_t shares_of(const Q4& w) { return (w.n + share_rows(w) - 1) / share_rows(w); }

// Rows of the weight to a CTA of one row's gradient.
int64_t one_share_rows(const Q4& w) {
  const int64_t want = std::max(1, kOneBackCtas * 152 / w.slabs), per = (w.n + want - 1) / want;
  return (per + 63) / 64 * 64;
}
template <typename TS, bool ZEROS>
acid_status launch_one_backward(const Q4Bwd& a, cudaStream_t s) {
  const dim3 grid(a.w.slabs, (unsigned)a.shares);
  const auto kernel = a.w.group_log == 5   ? q4_one_backward_kernel<TS, ZEROS, 5>
                      : a.w.group_log == 6 ? q4_one_backward_kernel<TS, ZEROS, 6>
                                           : q4_one_backward_kernel<TS, ZEROS, 7>;
  launch_pdl(kernel, grid, kThreads, 0, s, a);
  ACID_CHECK_LAUNCH();
  return ACID_OK;
}

// Workspace of the gradient: sums of each share, parts of g, powers of two, largest scales.
struct BackSpace {
  size_t parts, back, top, all;
};
BackSpace back_space(const Q4& w, int64_t m) {
  BackSpace b;
  const size_t shares = (size_t)shares_of(w), runs = (size_t)(w.n + 127) / 128 * 16;
  b.parts = shares * 2 * m * w.slabs * 128 * sizeof(float);
  const int64_t last = m - (chunks_of(m) - 1) * kQ4Chunk;  // rows of the last chunk
  b.back = b.parts + ((size_t)(chunks_of(m) - 1) * kQ4Chunk + last) * runs * 2 * 16;
  b.top = b.back + shares * m * sizeof(float);
  b.all = b.top + shares * kTopRuns * sizeof(uint32_t);
  if (m == 1) b.all = (size_t)((w.n + one_share_rows(w) - 1) / one_share_rows(w)) * w.slabs * 128 * sizeof(float);
  return b;
}

}  // namespace

size_t q4_rows_parts_bytes(const Q4& w, int64_t m) {
  return (size_t)chunks_of(m) * w.slabs * sixteens_of(m) * kSlabBytes<1>;
}
size_t q4_rows_forward_bytes(const Q4& w, int64_t m) { return q4_rows_parts_bytes(w, m) + (size_t)m * sizeof(float); }

acid_status q4_rows_forward(Q4Fwd a, void* workspace, int scale_dtype, cudaStream_t s) {
  a.parts = static_cast<uint8_t*>(workspace);
  a.back = reinterpret_cast<float*>(a.parts + q4_rows_parts_bytes(a.w, a.m));
  switch (sixteens_of(a.m)) {
    case 1: return launch_forward<1>(a, scale_dtype, s);
    case 2: return launch_forward<2>(a, scale_dtype, s);
    case 3: return launch_forward<3>(a, scale_dtype, s);
    default: return launch_forward<4>(a, scale_dtype, s);
  }
}

size_t q4_backward_bytes(const Q4& w, int64_t m) { return back_space(w, m).all; }

acid_status q4_backward(Q4Bwd a, void* workspace, cudaStream_t s) {
  if (a.dx == nullptr) {
    launch_pdl(q4_bias_kernel, (unsigned)std::min<int64_t>((a.w.n + kThreads - 1) / kThreads, 1 << 16), kThreads, 0, s, a);
    ACID_CHECK_LAUNCH();
    return ACID_OK;
  }
  const BackSpace b = back_space(a.w, a.m);
  uint8_t* base = static_cast<uint8_t*>(workspace);
  a.part = static_cast<float*>(workspace);
  a.parts = base + b.parts;
  a.back = reinterpret_cast<float*>(base + b.back);
  a.top = reinterpret_cast<uint32_t*>(base + b.top);
  a.per = share_rows(a.w);
  const int64_t shares = shares_of(a.w);
  a.shares = (int)shares * 2;
  if (a.m == 1) {
    a.per = one_share_rows(a.w);
    a.shares = (int)((a.w.n + a.per - 1) / a.per);
    const bool h = a.scale_dtype == ACID_BF16;
    ACID_TRY(a.w.zeros != nullptr ? (h ? launch_one_backward<bf16, true>(a, s) : launch_one_backward<float, true>(a, s))
                                  : (h ? launch_one_backward<bf16, false>(a, s) : launch_one_backward<float, false>(a, s)));
    launch_pdl(q4_backward_join_kernel, dim3((a.w.k + 127) / 128, (unsigned)a.m), 128, 0, s, a);
    ACID_CHECK_LAUNCH();
    return ACID_OK;
  }
  const int64_t bias_ctas = a.dbias != nullptr ? std::min<int64_t>((a.per + kThreads - 1) / kThreads, 1024) : 0;
  launch_pdl(q4_back_parts_kernel, dim3((unsigned)shares, (unsigned)(a.m + kTopRuns + bias_ctas)), kThreads, 0, s, a);
  ACID_CHECK_LAUNCH();
  ACID_TRY(a.scale_dtype != ACID_BF16     ? launch_backward<kThreeTerms>(a, s)
           : a.w.zeros != nullptr ? launch_backward<kTwoHalves>(a, s)
                                  : launch_backward<kOneHalf>(a, s));
  launch_pdl(q4_backward_join_kernel, dim3((a.w.k + 127) / 128, (unsigned)a.m), 128, 0, s, a);
  ACID_CHECK_LAUNCH();
  return ACID_OK;
}

}  // namespace acid
