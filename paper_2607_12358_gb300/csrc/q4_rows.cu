// 4-bit weights against many rows (tens of timestep embeddings: frames, branches
// or steps): the product and its input gradient on tcgen05.
#include <algorithm>
#include <string>

#include "q4.cuh"

namespace acid {

unsigned int take_device_error_q4_rows();
BoundsRecord take_bounds_q4_rows();
ACID_DEVICE_FLAG_READER(take_device_error_q4_rows)
ACID_BOUNDS_READER(take_bounds_q4_rows)

namespace {

using bf16 = __nv_bfloat16;
constexpr int kThreads = 256;
constexpr int kRowsThreads = 320;  // product: eight warps that make operands, an MMA warp and a copying warp
constexpr int kBackThreads = 416;  // gradient: eight and four warps that make operands, and an MMA warp

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
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                   smem_u32(dst)),
               "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

// ------------------------------------------------------------------ product
// D[128 rows of the weight, 16 NT] = codes x parts^T for each group of columns,
// the codes as the exact halves q - z in tensor memory (a row to a lane, where the
// lane's thread writes them), the parts of a(x) in shared memory (8 NT rows of high
// parts, then of low parts).  The same threads read the group's sums back, a row to a
// thread, and add them to the row's totals times its scale and the parts' powers of
// two.  A CTA has two tiles of 128 rows, whose four warps each run on their own.
constexpr int kFwdRing = 4;   // slabs of parts in shared memory
constexpr int kCodeRing = 3;  // slabs of a warp's 32 rows of codes
// Bytes of a slab's parts: two boxes of 64 columns, rows of 128 bytes whose
// 16-byte units are swizzled as the tensor cores read them.
template <int NT>
constexpr int kSlabBytes = 16 * NT * 256;
template <int NT>
constexpr int kFwdSmem = kFwdRing * kSlabBytes<NT> + 8 * kCodeRing * 2048 + 256 + 1024;

// One CTA to a row of a(x).
template <int NT>
__global__ void __launch_bounds__(kThreads) q4_parts_kernel(Q4Fwd a) {
  __shared__ uint32_t largest;
  pdl_wait();
  const int64_t m = blockIdx.x, chunk = m / kQ4Chunk;
  const int n = (int)(m - chunk * kQ4Chunk), octets = a.w.slabs * 16;
  if (threadIdx.x == 0) largest = 0;
  __syncthreads();
  float v[8], top = 0.f;
  for (int o = threadIdx.x; o < octets; o += kThreads) top = fmaxf(top, octet_values(a, m, o * 8, v));
  const uint32_t t = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
  if ((threadIdx.x & 31) == 0) atomicMax(&largest, t);
  __syncthreads();
  const float by = up_to_half(__uint_as_float(largest));
  if (threadIdx.x == 0) a.back[m] = 1.f / by;
  for (int o = threadIdx.x; o < octets; o += kThreads) {
    if (octets > kThreads) octet_values(a, m, o * 8, v);  // (else they are still there)
    uint4 hi, lo;
    split_octet(v, by, hi, lo);
    const int slab = o >> 4, word = (o >> 2) & 3, unit = (word & 1) * 4 + (o & 3);
    // octets in the order of the codes in a lane: words 32 columns by 32, in them the lanes' quarters
    uint8_t* p = a.parts + (chunk * a.w.slabs + slab) * kSlabBytes<NT> + (word >> 1) * (16 * NT * 128);
    *reinterpret_cast<uint4*>(p + n * 128 + ((unit ^ (n & 7)) << 4)) = hi;
    *reinterpret_cast<uint4*>(p + (8 * NT + n) * 128 + ((unit ^ (n & 7)) << 4)) = lo;
  }
}

template <int NT, typename TS>
__global__ void __launch_bounds__(kRowsThreads, 1) q4_rows_forward_kernel(Q4Fwd a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* ring = smem;
  uint8_t* codes = ring + kFwdRing * kSlabBytes<NT>;
  uint64_t* bars = reinterpret_cast<uint64_t*>(codes + 8 * kCodeRing * 2048);
  uint64_t *b_full = bars, *b_empty = bars + kFwdRing;                           // [ring]
  uint64_t *a_full = b_empty + kFwdRing, *d_full = a_full + 4, *d_empty = d_full + 2;  // [tile][2], [tile], [tile]
  uint64_t* drain = d_empty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  constexpr int kCols = 16 * NT, kHalf = 8 * NT;
  constexpr uint32_t kACol = 0, kDCol = 256;  // tensor memory: codes [tile][2][64], sums [tile][<= 128]
  const Q4& w = a.w;
  const int warp = warp_index(), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kFwdRing; ++i) {
      mbar_init(&b_full[i], 1);
      mbar_init(&b_empty[i], 1);
    }
    for (int i = 0; i < 4; ++i) mbar_init(&a_full[i], 128);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&d_full[i], 1);
      mbar_init(&d_empty[i], 128);
    }
    mbar_init(drain, 1);
    mbar_fence_init();
  }
  if (warp == 8) tmem_alloc(tmem_slot, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();

  const int64_t sets = (w.n + 255) / 256, chunk = blockIdx.y, m0 = chunk * kQ4Chunk;
  const int group = 1 << w.group_log, per_slab = 128 >> w.group_log;
  const int words = group / 32;  // of 32 columns, to a group
  const uint8_t* parts = a.parts + chunk * w.slabs * kSlabBytes<NT>;

  if (warp == 9) {
    if (lane == 0) {  // ------------------------------------------ copies of the parts
      int issued = 0;
      bool ok = true;
      for (int64_t set = blockIdx.x; ok && set < sets; set += gridDim.x)
        for (int slab = 0; slab < w.slabs; ++slab, ++issued) {
          const int st = issued % kFwdRing;
          if (issued >= kFwdRing && !mbar_wait(&b_empty[st], (issued / kFwdRing - 1) & 1)) { ok = false; break; }
          mbar_expect_tx(&b_full[st], kSlabBytes<NT>);
          bulk_load(ring + st * kSlabBytes<NT>, parts + (int64_t)slab * kSlabBytes<NT>, kSlabBytes<NT>, &b_full[st]);
        }
      // after a wait ran out: the last copies have landed before the CTA leaves
      if (!ok)
        for (int j = issued > kFwdRing ? issued - kFwdRing : 0; j < issued; ++j)
          mbar_wait(&b_full[j % kFwdRing], (j / kFwdRing) & 1);
    }
  } else if (warp == 8) {
    // ------------------------------------------------------------- MMA issuer
    const bool leader = elect_one();
    constexpr uint32_t idesc = idesc_f16_f32(128, kCols, false);
    const uint64_t bdesc = smem_desc_sw128(smem_u32(ring), 16, 1024);
    bool ok = true;
    uint32_t u = 0;  // steps (groups of columns)
    int v = 0;       // slabs
    for (int64_t set = blockIdx.x; ok && set < sets; set += gridDim.x)
      for (int slab = 0; ok && slab < w.slabs; ++slab, ++v) {
        const int st = v % kFwdRing;
        if (!mbar_wait_warp(&b_full[st], (v / kFwdRing) & 1)) { ok = false; break; }
        const uint64_t slot = bdesc + (uint64_t)((st * kSlabBytes<NT>) >> 4);
        for (int i = 0; ok && i < per_slab; ++i, ++u)
          for (int tile = 0; tile < 2; ++tile) {
            if (!mbar_wait_warp(&a_full[tile * 2 + (u & 1)], (u >> 1) & 1)) { ok = false; break; }
            if (u > 0 && !mbar_wait_warp(&d_empty[tile], (u - 1) & 1)) { ok = false; break; }
            tc_fence_after();
            if (leader) {
              const uint32_t d = tmem + kDCol + tile * 128, c = tmem + kACol + tile * 128 + (u & 1) * 64;
              for (int k = 0; k < group / 16; ++k) {
                const int kk = i * (group / 16) + k;  // 16 columns of the slab
                mma_bf16_ts(d, c + k * 8, slot + (uint64_t)(((kk >> 2) * (kCols * 128) + (kk & 3) * 32) >> 4), idesc, k != 0);
              }
              if (i == per_slab - 1 && tile == 1) mma_commit(&b_empty[st]);
              mma_commit(&d_full[tile]);
            }
            __syncwarp();
          }
      }
    if (!ok && leader) {
      mma_commit(drain);
      mbar_wait(drain, 0);
    }
  } else {
    // ----------------------- codes into tensor memory, sums out of it: warps 0-3 tile 0, 4-7 tile 1
    const int tile = warp >> 2, g = lane >> 2, t = lane & 3;
    const uint32_t quad = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t c_addr = tmem + quad + kACol + tile * 128, d_addr = tmem + quad + kDCol + tile * 128;
    uint8_t* mine = codes + warp * kCodeRing * 2048;
    // A lane copies 16 bytes of the rows g, g + 8, g + 16, g + 24 of the warp's 32 (64 bytes of a row together) and
    // reads its own row back; the units of a row are exchanged so that eight rows' reads lie in different banks.
    auto place = [](int row, int unit) { return row * 64 + ((unit ^ ((row >> 1) & 3)) << 4); };
    int64_t fset = blockIdx.x;
    int fslab = 0, fst = 0;
    auto copy = [&] {
      if (fset < sets) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int64_t row = min(fset * 256 + warp * 32 + g + 8 * q, w.n - 1);
          const int64_t at = (row * w.slabs + fslab) * 16 + 4 * t;
          const bool in = ACID_IN_BOUNDS(kSiteQ4, at + 3, w.n * w.slabs * 16);
          cp_async<16>(mine + fst * 2048 + place(g + 8 * q, t), w.packed + (in ? at : 0), in);
        }
        if (++fslab == w.slabs) {
          fslab = 0;
          fset += gridDim.x;
        }
      }
      cp_async_commit();
      fst = fst + 1 == kCodeRing ? 0 : fst + 1;
    };
    for (int i = 0; i < kCodeRing - 1; ++i) copy();
    uint64_t total[NT][4];  // pairs of the row's sums
    bool ok = true;
    uint32_t u = 0;
    // Adds the sums of step `step`, whose scale is s.
    auto take = [&](uint32_t step, float s) -> bool {
      if (!mbar_wait_warp(&d_full[tile], step & 1)) return false;
      tc_fence_after();
      constexpr int kBatch = NT <= 5 ? NT : 4;
#pragma unroll
      for (int n0 = 0; n0 < NT; n0 += kBatch) {
        uint32_t hi[kBatch][8], lo[kBatch][8];
#pragma unroll
        for (int n = 0; n < kBatch; ++n) {
          tmem_ld8(d_addr + (n0 + n) * 8, hi[n]);
          tmem_ld8(d_addr + kHalf + (n0 + n) * 8, lo[n]);
        }
        tmem_wait_ld();
        if (n0 + kBatch == NT) {
          tc_fence_before();
          mbar_arrive(&d_empty[tile]);
        }
        const uint64_t s2 = f2_pack(s, s);
#pragma unroll
        for (int n = 0; n < kBatch; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint64_t x = f2_add(f2_pack(__uint_as_float(hi[n][2 * e]), __uint_as_float(hi[n][2 * e + 1])),
                                      f2_pack(__uint_as_float(lo[n][2 * e]), __uint_as_float(lo[n][2 * e + 1])));
            total[n0 + n][e] = f2_fma(x, s2, total[n0 + n][e]);
          }
      }
      return true;
    };
    int st = 0;
    for (int64_t set = blockIdx.x; ok && set < sets; set += gridDim.x) {
      const int64_t row = set * 256 + warp * 32 + lane, at = min(row, w.n - 1) * w.groups;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) total[n][e] = 0;
      // scales and zero points of a slab's groups, a slab ahead
      float scales[4];
      uint8_t zeros[4];
      auto look = [&](int slab) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (i >= per_slab) break;
          const int64_t p = at + min(slab * per_slab + i, w.groups - 1);
          if (!ACID_IN_BOUNDS(kSiteQ4, p, w.n * w.groups)) continue;
          scales[i] = io<TS>::ld(static_cast<const TS*>(w.scales) + p);
          if (w.zeros != nullptr) zeros[i] = w.zeros[p];
        }
      };
      look(0);
      float scale = 0.f;  // of the step whose sums are not taken yet
      bool pending = false;
      for (int slab = 0; ok && slab < w.slabs; ++slab) {
        cp_async_wait<kCodeRing - 2>();
        __syncwarp();
        uint4 q[4];  // q[t]: words of the columns 32 i + 8 t
#pragma unroll
        for (int c = 0; c < 4; ++c) q[c] = *reinterpret_cast<const uint4*>(mine + st * 2048 + place(lane, c));
        copy();
        st = st + 1 == kCodeRing ? 0 : st + 1;
        float s[4];
        uint32_t z[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[i] = scales[i];
          z[i] = w.zeros != nullptr ? zeros[i] : 8u;
        }
        if (slab + 1 < w.slabs) look(slab + 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int within = i & (words - 1), of = words == 4 ? 0 : words == 2 ? i >> 1 : i;
          const uint32_t zero = of == 0 ? z[0] : of == 1 ? z[1] : of == 2 ? z[2] : z[3];
          uint32_t d[16];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            uint32_t h[4];
            halves_of(i == 0 ? q[c].x : i == 1 ? q[c].y : i == 2 ? q[c].z : q[c].w, zero, h);
#pragma unroll
            for (int j = 0; j < 4; ++j) d[4 * c + j] = h[j];
          }
          tmem_st16(c_addr + (u & 1) * 64 + within * 16, d);
          if (within != words - 1) continue;
          tmem_wait_st();
          tc_fence_before();
          mbar_arrive(&a_full[tile * 2 + (u & 1)]);
          // the sums of the step before, while this one's are formed
          if (pending && ok) ok = take(u - 1, scale);
          pending = true;
          scale = of == 0 ? s[0] : of == 1 ? s[1] : of == 2 ? s[2] : s[3];
          ++u;
        }
      }
      if (ok) ok = take(u - 1, scale);
      if (!ok || row >= w.n) continue;
      const float bias = a.bias != nullptr ? a.bias[row] : 0.f;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int64_t m = m0 + 8 * n + 2 * e;
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
  if (warp == 8) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// ----------------------------------------------------------- input gradient
// D[2 x 64 parts of g s, 128 columns] += parts x codes for 128 rows of the weight at a
// time.  (g s), a power of two that brings its largest value below 2^15, and
// two halves of it are formed by the threads of a lane of tensor memory (row m of
// g: lane m its high parts, lane 64 + m its low parts), once for each of the slab's
// groups; the codes, exact halves q - z, are written to shared memory, where they
// are the second operand as they lie (columns together).  Sums stay in tensor memory
// over all of a CTA's rows.
struct BwdSmem {
  static constexpr int kCodes = 128 * 256;                // [box of 64 columns][128 rows][128 bytes]
  static constexpr int kGStride = 132;                    // floats of a row of g: 128 and a shift of the banks
  static constexpr int kG = kQ4Chunk * kGStride * 4;
  static constexpr int kOffG = 2 * kCodes, kOffS = kOffG + 2 * kG, kOffBar = kOffS + 2 * 4 * 128 * 4;
  static constexpr int kBytes = kOffBar + 256 + 1024;
};

// Largest scale and largest |g| of each row over runs of kQ4ScanRows rows of the
// weight (blockIdx.y: a chunk of g's rows), and the bias's gradient.
__global__ void __launch_bounds__(kThreads) q4_scan_kernel(Q4Bwd a) {
  __shared__ uint32_t top[1 + kQ4Chunk];  // bits of non-negative floats
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const bool first = blockIdx.y == 0;
  const int64_t n0 = (int64_t)blockIdx.x * kQ4ScanRows, n1 = min(a.w.n, n0 + kQ4ScanRows);
  const int64_t m0 = (int64_t)blockIdx.y * kQ4Chunk, m1 = min(a.m, m0 + kQ4Chunk);
  if (threadIdx.x <= kQ4Chunk) top[threadIdx.x] = 0;
  __syncthreads();
  auto bits_of = [](float v) { return isfinite(v) ? __float_as_uint(fabsf(v)) : 0u; };
  if (first) {
    uint32_t s = 0;
    for (int64_t i = n0 * a.w.groups + threadIdx.x; i < n1 * a.w.groups; i += kThreads)
      if (ACID_IN_BOUNDS(kSiteQ4, i, a.w.n * a.w.groups)) s = max(s, bits_of(value_at(a.scale_dtype, a.w.scales, i)));
    s = __reduce_max_sync(0xffffffffu, s);
    if (lane == 0) atomicMax(&top[0], s);
  }
  constexpr int kPer = kQ4ScanRows / kThreads;
  float sum[kPer] = {};
#pragma unroll 4
  for (int64_t m = m0; m < m1; ++m) {
    uint32_t t = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int64_t n = n0 + j * kThreads + threadIdx.x;
      const float v = n < n1 ? value_at(a.g_dtype, a.g, m * a.ldg + n) : 0.f;
      sum[j] += v;
      t = max(t, bits_of(v));
    }
    t = __reduce_max_sync(0xffffffffu, t);
    if (lane == 0) atomicMax(&top[1 + m - m0], t);
  }
  if (first && a.dbias != nullptr)
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int64_t n = n0 + j * kThreads + threadIdx.x;
      if (n >= n1) continue;
      for (int64_t m = m1; m < a.m; ++m) sum[j] += value_at(a.g_dtype, a.g, m * a.ldg + n);
      a.dbias[n] = sum[j];
    }
  __syncthreads();
  float* out = a.top + blockIdx.x * (a.m + 1);
  if (first && threadIdx.x == 0) out[0] = __uint_as_float(top[0]);
  if (threadIdx.x < m1 - m0) out[1 + m0 + threadIdx.x] = __uint_as_float(top[1 + threadIdx.x]);
}

template <typename TG, typename TS>
__global__ void __launch_bounds__(kBackThreads, 1) q4_rows_backward_kernel(Q4Bwd a) {
  extern __shared__ uint8_t smem_raw[];
  using L = BwdSmem;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  float* gs = reinterpret_cast<float*>(smem + L::kOffG);  // [2][64][kGStride]
  float* ss = reinterpret_cast<float*>(smem + L::kOffS);  // [2][group of the slab][128]
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::kOffBar);
  uint64_t *a_full = bars, *a_empty = bars + 2, *w_full = bars + 4, *w_empty = bars + 6, *done = bars + 8, *drain = bars + 9;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 10);
  const Q4& w = a.w;
  const int warp = warp_index(), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&a_full[i], 256);
      mbar_init(&a_empty[i], 1);
      mbar_init(&w_full[i], 128);
      mbar_init(&w_empty[i], 1);
    }
    mbar_init(done, 1);
    mbar_init(drain, 1);
    mbar_fence_init();
  }
  if (warp == 12) tmem_alloc(tmem_slot, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();

  const int slab = blockIdx.x, variants = 128 >> w.group_log;
  const int64_t begin = blockIdx.y * a.per, end = min(w.n, begin + a.per), m0 = (int64_t)blockIdx.z * kQ4Chunk;
  const int rows = (int)min((int64_t)kQ4Chunk, a.m - m0), blocks = (int)((end - begin + 127) / 128);
  // tensor memory: sums [128], or [4][64] of which half is used; parts [buffer][group][64]
  const int a_bufs = variants == 4 ? 1 : 2;
  const uint32_t kDCol = 0, kACol = variants == 4 ? 256 : 128;
  const int d_step = variants == 1 ? 0 : 64;  // a group's sums are 128 columns, or the 64 of its box

  if (warp == 12) {
    // ------------------------------------------------------------- MMA issuer
    const bool leader = elect_one();
    const uint32_t idesc = idesc_f16_f32(128, variants == 1 ? 128 : 64, true);
    const uint64_t bdesc = smem_desc_sw128(smem_u32(smem), L::kCodes / 2, 1024);
    bool ok = true;
    for (int b = 0; ok && b < blocks; ++b) {
      const int ab = b % a_bufs, wb = b & 1;
      if (!mbar_wait_warp(&a_full[ab], (b / a_bufs) & 1)) { ok = false; break; }
      if (!mbar_wait_warp(&w_full[wb], (b >> 1) & 1)) { ok = false; break; }
      tc_fence_after();
      if (leader) {
        for (int v = 0; v < variants; ++v) {
          const int box = variants == 1 ? 0 : variants == 2 ? v : v >> 1;
          const uint64_t slot = bdesc + (uint64_t)((wb * L::kCodes + box * (L::kCodes / 2)) >> 4);
          for (int k = 0; k < 8; ++k)
            mma_bf16_ts(tmem + kDCol + v * d_step, tmem + kACol + (ab * variants + v) * 64 + k * 8,
                        slot + (uint64_t)((k * 16 * 128) >> 4), idesc, b != 0 || k != 0);
        }
        mma_commit(&a_empty[ab]);
        mma_commit(&w_empty[wb]);
        if (b == blocks - 1) mma_commit(done);
      }
      __syncwarp();
    }
    if (!ok && leader) {
      mma_commit(drain);
      mbar_wait(drain, 0);
    }
  } else if (warp >= 8) {
    // ------------------------------------------- codes into shared memory, 32 rows of a block to a warp
    const int g = lane >> 2, t = lane & 3, odd = g & 1;
    struct Load {
      uint4 q[4];
      uint8_t z[4][4];  // zero points of the slab's groups
    };
    auto fetch = [&](Load& l, int b) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int64_t row = min(begin + b * 128 + (warp - 8) * 32 + g + 8 * q, w.n - 1);
        const int64_t at = (row * w.slabs + slab) * 16 + 4 * t;
        if (ACID_IN_BOUNDS(kSiteQ4, at + 3, w.n * w.slabs * 16)) l.q[q] = *reinterpret_cast<const uint4*>(w.packed + at);
        if (w.zeros == nullptr) continue;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          if (v >= variants) break;
          const int64_t z = row * w.groups + min(slab * variants + v, w.groups - 1);
          if (ACID_IN_BOUNDS(kSiteQ4, z, w.n * w.groups)) l.z[q][v] = w.zeros[z];
        }
      }
    };
    const int word_log = w.group_log - 5;
    bool ok = true;
    Load l;
    fetch(l, 0);
    for (int b = 0; ok && b < blocks; ++b) {
      const int wb = b & 1;
      if (b >= 2 && !mbar_wait_warp(&w_empty[wb], ((b >> 1) - 1) & 1)) { ok = false; break; }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int row = (warp - 8) * 32 + g + 8 * q;
        // neighbouring rows take their words in another order, so that their units lie in different banks
        const uint4 v = odd ? make_uint4(l.q[q].y, l.q[q].x, l.q[q].w, l.q[q].z) : l.q[q];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const int i = s ^ odd, unit = (i & 1) * 4 + t;
          uint32_t h[4];
          uint32_t z = 8;
          if (w.zeros != nullptr) {
            const int of = i >> word_log;
            z = (of == 0 ? l.z[q][0] : of == 1 ? l.z[q][1] : of == 2 ? l.z[q][2] : l.z[q][3]) & 15u;
          }
          halves_of(s == 0 ? v.x : s == 1 ? v.y : s == 2 ? v.z : v.w, z, h);
          *reinterpret_cast<uint4*>(smem + wb * L::kCodes + (i >> 1) * (L::kCodes / 2) + row * 128 + ((unit ^ (row & 7)) << 4)) =
              make_uint4(h[0], h[1], h[2], h[3]);
        }
      }
      if (b + 1 < blocks) fetch(l, b + 1);
      fence_proxy_async_smem();
      mbar_arrive(&w_full[wb]);
    }
  } else {
    // ----------------------------------------------- parts of g s, then the sums: two warps to a quarter of the lanes,
    // half of the block's rows each
    const int tid = threadIdx.x & 127, half = warp >> 2, m = (warp & 1) * 32 + lane;
    const bool low = (warp & 2) != 0, active = (warp & 1) * 32 < rows;
    // the powers of two
    float gt = 0.f, st = 0.f;
    for (int i = 0; i < a.scans; ++i) {
      st = fmaxf(st, a.top[(int64_t)i * (a.m + 1)]);
      if (m < rows) gt = fmaxf(gt, a.top[(int64_t)i * (a.m + 1) + 1 + m0 + m]);
    }
    const float up = up_to_half(gt);                                                       // |g| to 2^13 .. 2^14
    const float one = __uint_as_float(max(254 - (int)(__float_as_uint(st) >> 23), 1) << 23);  // scales to 1 .. 2
    // Row n of the block to thread n, or n + 128: g by its rows (every other one), scales by groups (the same).  Scales
    // are looked at a block before they are stored.
    auto copy = [&](int b) {
      const int64_t n = begin + b * 128 + tid;
      float* gd = gs + (b & 1) * (L::kG / 4) + tid;
      if constexpr (sizeof(TG) == 4) {
        const float* src = static_cast<const float*>(a.g) + m0 * a.ldg + (n < end ? n : begin);
#pragma unroll 4
        for (int i = half; i < rows; i += 2) cp_async<4>(gd + i * L::kGStride, src + i * a.ldg, n < end);
      } else {
#pragma unroll 8
        for (int i = half; i < rows; i += 2)
          gd[i * L::kGStride] = n < end ? io<TG>::ld(static_cast<const TG*>(a.g) + (m0 + i) * a.ldg + n) : 0.f;
      }
      cp_async_commit();
    };
    float sv[2];
    auto look = [&](int b) {
      const int64_t n = begin + b * 128 + tid;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int v = half + 2 * j;
        sv[j] = 0.f;
        if (v >= variants || n >= end || b >= blocks) continue;
        const int64_t at = n * w.groups + min(slab * variants + v, w.groups - 1);
        if (ACID_IN_BOUNDS(kSiteQ4, at, w.n * w.groups)) sv[j] = io<TS>::ld(static_cast<const TS*>(w.scales) + at);
      }
    };
    auto store = [&](int b) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (half + 2 * j < variants) ss[((b & 1) * 4 + half + 2 * j) * 128 + tid] = sv[j] * one;
    };
    copy(0);
    look(0);
    store(0);
    look(1);
    const uint32_t quad = (uint32_t)((warp & 3) * 32) << 16;
    bool ok = true;
    const uint64_t up2 = f2_pack(up, up);
    for (int b = 0; b < blocks; ++b) {
      cp_async_wait<0>();
      // block b is there, and nobody reads the other buffer any more; after a wait ran out the eight warps leave together
      if (!group_all(1, 256, ok)) {
        ok = false;
        break;
      }
      if (b + 1 < blocks) {
        copy(b + 1);
        store(b + 1);
        look(b + 2);
      }
      const int ab = b % a_bufs;
      if (b >= a_bufs) ok = mbar_wait_warp(&a_empty[ab], (b / a_bufs - 1) & 1);
      if (active && ok) {
        const float* gr = gs + (b & 1) * (L::kG / 4) + m * L::kGStride;
        for (int v = 0; v < variants; ++v) {
          const float* sr = ss + ((b & 1) * 4 + v) * 128;
          const uint32_t to = tmem + quad + kACol + (ab * variants + v) * 64;
#pragma unroll
          for (int e4 = 0; e4 < 2; ++e4) {
            const int c = 2 * half + e4;
            uint32_t d[16];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float4 x = *reinterpret_cast<const float4*>(gr + c * 32 + j * 4);
              const float4 y = *reinterpret_cast<const float4*>(sr + c * 32 + j * 4);
              const uint64_t p[2] = {f2_mul(f2_mul(f2_pack(x.x, x.y), up2), f2_pack(y.x, y.y)),
                                     f2_mul(f2_mul(f2_pack(x.z, x.w), up2), f2_pack(y.z, y.w))};
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                float f0, f1;
                f2_unpack(p[e], f0, f1);
                __half2 h = __floats2half2_rn(f0, f1);
                if (low) {
                  const float2 f = __half22float2(h);
                  h = __floats2half2_rn(f0 - f.x, f1 - f.y);
                }
                d[2 * j + e] = bits(h);
              }
            }
            tmem_st16(to + c * 16, d);
          }
        }
        tmem_wait_st();
      }
      tc_fence_before();
      mbar_arrive(&a_full[ab]);
    }
    cp_async_wait<0>();
    if (ok) ok = mbar_wait_warp(done, 0);
    tc_fence_after();
    if (ok && active) {
      const float down = 1.f / up, per_s = 1.f / one;
      float* out = a.part + ((blockIdx.y * 2 + low) * a.m + m0 + m) * w.slabs * 128 + slab * 128;
#pragma unroll
      for (int e = 0; e < 2; ++e) {  // 32 columns
        const int c = 2 * half + e, v = variants == 4 ? c : 0;
        uint32_t r[32];
        tmem_ld32(tmem + quad + kDCol + (variants == 4 ? v * 64 + (c & 1) * 32 : c * 32), r);
        tmem_wait_ld();
        const int64_t at = ((blockIdx.y * 2 + low) * a.m + m0 + m) * w.slabs * 128 + slab * 128 + c * 32;
        if (m < rows && ACID_IN_BOUNDS(kSiteQ4, at + 31, a.shares * a.m * w.slabs * 128)) {
#pragma unroll
          for (int o = 0; o < 4; ++o) {  // an octet's columns j and j + 4 lie side by side
            float f[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(r[8 * o + j]) * down * per_s;
            *reinterpret_cast<float4*>(out + c * 32 + o * 8) = make_float4(f[0], f[2], f[4], f[6]);
            *reinterpret_cast<float4*>(out + c * 32 + o * 8 + 4) = make_float4(f[1], f[3], f[5], f[7]);
          }
        }
        __syncwarp();
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 12) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// --------------------------------------------------------------------- host
// Column tiles of eight that the product's kernel is built for.
int tiles_for(int64_t m) {
  const int nt = (int)((std::min<int64_t>(m, kQ4Chunk) + 7) / 8);
  return nt <= 3 ? nt : nt <= 5 ? 5 : 8;
}
int64_t chunks_of(int64_t m) { return (m + kQ4Chunk - 1) / kQ4Chunk; }

template <int NT, typename TS>
acid_status launch_forward(const Q4Fwd& a, cudaStream_t s) {
  static PerContext allowed;
  ACID_TRY(allow_smem(allowed, q4_rows_forward_kernel<NT, TS>, kFwdSmem<NT>));
  const int64_t sets = (a.w.n + 255) / 256;
  const dim3 grid((unsigned)std::min<int64_t>(sets, num_sms()), (unsigned)chunks_of(a.m));
  launch_pdl(q4_rows_forward_kernel<NT, TS>, grid, kRowsThreads, kFwdSmem<NT>, s, a);
  ACID_CHECK_LAUNCH();
  return ACID_OK;
}
template <int NT>
acid_status launch_forward(const Q4Fwd& a, int scale_dtype, cudaStream_t s) {
  launch_pdl(q4_parts_kernel<NT>, (unsigned)a.m, kThreads, 0, s, a);
  ACID_CHECK_LAUNCH();
  return scale_dtype == ACID_BF16 ? launch_forward<NT, bf16>(a, s) : launch_forward<NT, float>(a, s);
}

template <typename TG, typename TS>
acid_status launch_backward(const Q4Bwd& a, cudaStream_t s) {
  static PerContext allowed;
  ACID_TRY(allow_smem(allowed, q4_rows_backward_kernel<TG, TS>, BwdSmem::kBytes));
  const dim3 grid(a.w.slabs, (unsigned)((a.w.n + a.per - 1) / a.per), (unsigned)chunks_of(a.m));
  launch_pdl(q4_rows_backward_kernel<TG, TS>, grid, kBackThreads, BwdSmem::kBytes, s, a);
  ACID_CHECK_LAUNCH();
  return ACID_OK;
}

}  // namespace

size_t q4_rows_parts_bytes(const Q4& w, int64_t m) {
  return (size_t)chunks_of(m) * w.slabs * tiles_for(m) * kSlabBytes<1>;
}
size_t q4_rows_back_bytes(const Q4&, int64_t m) {
  return (size_t)m * sizeof(float);
}

acid_status q4_rows_forward(const Q4Fwd& a, int scale_dtype, cudaStream_t s) {
  switch (tiles_for(a.m)) {
    case 1: return launch_forward<1>(a, scale_dtype, s);
    case 2: return launch_forward<2>(a, scale_dtype, s);
    case 3: return launch_forward<3>(a, scale_dtype, s);
    case 5: return launch_forward<5>(a, scale_dtype, s);
    default: return launch_forward<8>(a, scale_dtype, s);
  }
}

// As many CTAs as an SM each has, in whole blocks of 128 rows.
int64_t q4_rows_share(const Q4& w) {
  const int64_t want = std::max(1, 152 / w.slabs), per = (w.n + want - 1) / want;
  return (per + 127) / 128 * 128;
}

acid_status q4_rows_backward(const Q4Bwd& a, cudaStream_t s) {
  launch_pdl(q4_scan_kernel, dim3(a.scans, (unsigned)chunks_of(a.m)), kThreads, 0, s, a);
  ACID_CHECK_LAUNCH();
  if (a.g_dtype == ACID_BF16)
    return a.scale_dtype == ACID_BF16 ? launch_backward<bf16, bf16>(a, s) : launch_backward<bf16, float>(a, s);
  return a.scale_dtype == ACID_BF16 ? launch_backward<float, bf16>(a, s) : launch_backward<float, float>(a, s);
}

}  // namespace acid
