// Attention with row sums, and its gradient: the entry points (acid_mha_*) and the
// statistics that the backward kernels read.
#include <math.h>

#include <algorithm>
#include <string>

#define ACID_UNIT_WITHOUT_WAITS
#include "mha.cuh"

namespace acid {

BoundsRecord take_bounds_mha();
ACID_BOUNDS_READER(take_bounds_mha)

namespace {

constexpr int kThreads = 256;

struct StatArgs {
  MhaShape s;
  const void *out, *dout;
  int64_t ldo, lddo;
  const float* lse;
  float* stats;
  int d, slots;
  float unit;  // of the kernels' exponential: 1 for e, log2(e) for 2
};

// -lse and -sum(dout out) of a slot's rows for one head (mha_stat_offset).  A row is
// `lanes` lanes of 8 columns.  It reads out and dout once: 202 MB (32760 rows, 12 x 128) in
// 37.6 us, 79% of the copy bandwidth, issue 60%; 39 in a call, 44 with L2 full of lines that
// have to be written back first.  (8190 rows, 24 x 128, L2 full of such lines: 23.9 us, eight
// rows ahead 30.5, two 23.8, heads side by side 23.6, six CTAs an SM, which spill, 28.7.)
template <typename T>
__global__ void __launch_bounds__(kThreads) mha_stats_kernel(const StatArgs a, int lanes) {
  pdl_wait();
  MhaSeq seq;
  int index, tile;
  if (!mha_slot<kStatRows, false>(a.s, blockIdx.x, seq, index, tile)) return;
  const int h = blockIdx.y, part = threadIdx.x % lanes, step = kThreads / lanes;
  float* to = a.stats + mha_stat_offset(h, a.slots, blockIdx.x);
  constexpr int kAhead = sizeof(T) == 2 ? 4 : 2;  // rows whose loads are on the way together
  for (int r0 = threadIdx.x / lanes; r0 < kStatRows; r0 += kAhead * step) {
    MhaRaw<T> o[kAhead], g[kAhead];
    float lse[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int i = tile * kStatRows + r0 + k * step;
      o[k].zero();
      g[k].zero();
      lse[k] = -INFINITY;
      if (i >= seq.nq || r0 + k * step >= kStatRows) continue;
      const int64_t row = seq.q0 + i;
      const int64_t at = row * a.ldo + h * a.d + part * 8, from = row * a.lddo + h * a.d + part * 8;
      if (part * 8 < a.d && ACID_IN_BOUNDS(kSiteMha, at + 7, (int64_t)a.s.nq * a.ldo) &&
          ACID_IN_BOUNDS(kSiteMha, from + 7, (int64_t)a.s.nq * a.lddo)) {
        o[k].load(static_cast<const T*>(a.out) + at);
        g[k].load(static_cast<const T*>(a.dout) + from);
      }
      if (ACID_IN_BOUNDS(kSiteMha, h * (int64_t)a.s.nq + row, (int64_t)a.s.heads * a.s.nq))
        lse[k] = a.lse[(int64_t)h * a.s.nq + row];
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      float x[8], y[8], sum = 0.f;
      o[k].get(x);
      g[k].get(y);
#pragma unroll
      for (int c = 0; c < 8; ++c) sum = fmaf(x[c], y[c], sum);
      for (int off = lanes / 2; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
      const int r = r0 + k * step;
      if (part == 0 && r < kStatRows &&
          ACID_IN_BOUNDS(kSiteMha, mha_stat_offset(h, a.slots, blockIdx.x) + kStatRows + r,
                         mha_stat_offset(a.s.heads, a.slots, 0))) {
        to[r] = lse[k] == -INFINITY ? -INFINITY : -lse[k] * a.unit;  // (a row that sees no key: probability 0)
        to[kStatRows + r] = lse[k] == -INFINITY ? 0.f : -sum;
      }
    }
  }
}

// Zeros in the rows of no sequence, a warp a row.  Results that a caller has not allocated
// are zero there; zeroing them whole wrote 33 MB and took 10 us of 234 at 4726 + 2501 + 1013
// rows, 30 heads of 64.
struct PaddingArgs {
  const int2* bounds;
  int seqs, rows, heads;
  int width;  // bytes of a row
  uint8_t *a, *b;
  int64_t lda, ldb;  // bytes
  float* lse;
};
__global__ void __launch_bounds__(kThreads) mha_padding_kernel(const PaddingArgs p) {
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  if (row >= p.rows) return;
  int first, n;
  mha_bound(p.bounds, mha_sequence_of(p.bounds, p.seqs, row), p.seqs, p.rows, first, n);
  if (row >= first && row < (int64_t)first + n) return;
  for (int i = lane * 16; i < p.width; i += 512) {
    if (p.a != nullptr && ACID_IN_BOUNDS(kSiteMha, row * p.lda + i + 15, p.rows * p.lda))
      *reinterpret_cast<uint4*>(p.a + row * p.lda + i) = make_uint4(0, 0, 0, 0);
    if (p.b != nullptr && ACID_IN_BOUNDS(kSiteMha, row * p.ldb + i + 15, p.rows * p.ldb))
      *reinterpret_cast<uint4*>(p.b + row * p.ldb + i) = make_uint4(0, 0, 0, 0);
  }
  if (p.lse != nullptr)
    for (int h = lane; h < p.heads; h += 32)
      if (ACID_IN_BOUNDS(kSiteMha, h * (int64_t)p.rows + row, (int64_t)p.heads * p.rows)) p.lse[(int64_t)h * p.rows + row] = 0.f;
}

acid_status check_mha(const acid_mha* m) {
  ACID_REQUIRE(m != nullptr, ACID_ERR_INVALID_ARG, "mha: null description");
  ACID_REQUIRE(m->dtype == ACID_BF16 || m->dtype == ACID_FP32, ACID_ERR_INVALID_ARG, "mha: unknown dtype");
  ACID_REQUIRE(m->nq >= 0 && m->nk >= 0, ACID_ERR_INVALID_ARG, "mha: rows must be >= 0");
  ACID_REQUIRE(m->nq <= kMhaMaxRows && m->nk <= kMhaMaxRows, ACID_ERR_UNSUPPORTED, "mha: more than 2^30 rows");
  ACID_REQUIRE(m->heads > 0 && m->kv_heads > 0 && m->heads % m->kv_heads == 0, ACID_ERR_INVALID_ARG,
               "mha: heads must be a multiple of kv_heads, both > 0");
  ACID_REQUIRE(m->heads <= 65535, ACID_ERR_UNSUPPORTED, "mha: more than 65535 heads");
  if (m->dtype == ACID_BF16)
    ACID_REQUIRE(m->head_dim == 64 || m->head_dim == 128, ACID_ERR_UNSUPPORTED, "mha bf16: head_dim must be 64 or 128");
  else
    ACID_REQUIRE(m->head_dim > 0 && m->head_dim % 32 == 0 && m->head_dim <= 128, ACID_ERR_UNSUPPORTED,
                 "mha fp32: head_dim must be 32, 64, 96 or 128");
  ACID_REQUIRE(isfinite(m->scale), ACID_ERR_INVALID_ARG, "mha: scale must be finite");
  ACID_REQUIRE(m->sequences >= 1 && m->sequences <= 65535, ACID_ERR_INVALID_ARG, "mha: need 1 to 65535 sequences");
  ACID_REQUIRE((std::max(m->nq, m->nk) / 64 + m->sequences + 1) * m->heads <= (int64_t)1 << 30, ACID_ERR_UNSUPPORTED,
               "mha: too many rows and heads");
  ACID_REQUIRE(m->sequences == 1 || (m->q_bounds != nullptr && m->k_bounds != nullptr), ACID_ERR_INVALID_ARG,
               "mha: several sequences need the bounds of both queries and keys");
  ACID_REQUIRE(aligned(m->q_bounds, 8) && aligned(m->k_bounds, 8), ACID_ERR_UNSUPPORTED,
               "mha: bounds must be 8-byte aligned");
  ACID_REQUIRE(m->frame_rows >= 0 && m->frame_rows <= kMhaMaxRows, ACID_ERR_INVALID_ARG,
               "mha: frame_rows must be 0 .. 2^30");
  ACID_REQUIRE(m->frames_before >= -1 && m->frames_after >= -1, ACID_ERR_INVALID_ARG,
               "mha: frames_before and frames_after must be >= -1");
  ACID_REQUIRE(m->q_first >= -1 && m->q_first <= kMhaMaxRows, ACID_ERR_INVALID_ARG, "mha: q_first must be -1 .. 2^30");
  return ACID_OK;
}

// A [rows, heads head_dim] operand.
acid_status check_operand(const acid_mha& m, const void* p, int64_t ld, int64_t rows, int heads, const char* name) {
  ACID_REQUIRE(p != nullptr || rows == 0, ACID_ERR_INVALID_ARG, std::string("mha: ") + name + " is null");
  ACID_REQUIRE(ld >= (int64_t)heads * m.head_dim, ACID_ERR_INVALID_ARG,
               std::string("mha: row stride of ") + name + " smaller than its heads");
  ACID_REQUIRE(aligned(p, 16) && ld % 8 == 0, ACID_ERR_UNSUPPORTED,
               std::string("mha: ") + name + " must be 16-byte aligned, its row stride a multiple of 8");
  return ACID_OK;
}
// The same of an output that may be left out.
acid_status check_gradient(const acid_mha& m, const void* p, int64_t ld, int64_t rows, int heads, const char* name) {
  return p == nullptr ? ACID_OK : check_operand(m, p, ld, rows, heads, name);
}

MhaArgs common_args(const acid_mha& m) {
  MhaArgs a = {};
  MhaShape& s = a.shape;
  s.nq = (int)m.nq;
  s.nk = (int)m.nk;
  s.heads = m.heads;
  s.kv_heads = m.kv_heads;
  s.group = m.heads / m.kv_heads;
  s.seqs = m.sequences;
  s.qb = reinterpret_cast<const int2*>(m.q_bounds);
  s.kb = reinterpret_cast<const int2*>(m.k_bounds);
  s.frame = (int)m.frame_rows;
  s.before = m.frames_before;
  s.after = m.frames_after;
  s.q_first = (int)m.q_first;
  if (s.before < 0 && s.after < 0) s.frame = 0;  // every frame sees every other
  a.dtype = m.dtype;
  a.head_dim = m.head_dim;
  a.scale = m.scale;
  return a;
}

int stat_slots(const acid_mha& m) { return mha_slots((int)m.nq, m.sequences, m.q_bounds != nullptr, kStatRows); }
size_t stat_bytes(const acid_mha& m) { return (size_t)mha_stat_offset(m.heads, stat_slots(m), 0) * sizeof(float); }

size_t forward_bytes(const acid_mha& m) {
  const MhaArgs a = common_args(m);
  if (m.nq == 0) return 0;
  if (mha_few(a)) return mha_few_bytes(a);
  return m.dtype == ACID_BF16 ? mha_forward_tc_bytes(a) : 0;
}
size_t backward_bytes(const acid_mha& m) {
  return stat_bytes(m) + (m.dtype == ACID_BF16 ? mha_backward_tc_bytes(common_args(m)) : 0);
}

acid_status check_workspace(const void* ws, size_t bytes, size_t need, const char* call) {
  if (need == 0) return ACID_OK;
  ACID_REQUIRE(ws != nullptr && aligned(ws, 16), ACID_ERR_WORKSPACE,
               std::string(call) + ": workspace null or not 16-byte aligned");
  ACID_REQUIRE(bytes >= need, ACID_ERR_WORKSPACE,
               std::string(call) + ": workspace too small (need " + std::to_string(need) + ")");
  return ACID_OK;
}

}  // namespace
}  // namespace acid

using namespace acid;

extern "C" acid_status acid_mha_forward_workspace_size(const acid_mha* mha, size_t* bytes) {
  clear_error();
  ACID_TRY(check_mha(mha));
  ACID_REQUIRE(bytes != nullptr, ACID_ERR_INVALID_ARG, "acid_mha_forward_workspace_size: bytes is null");
  *bytes = forward_bytes(*mha);
  return ACID_OK;
}

extern "C" acid_status acid_mha_backward_workspace_size(const acid_mha* mha, size_t* bytes) {
  clear_error();
  ACID_TRY(check_mha(mha));
  ACID_REQUIRE(bytes != nullptr, ACID_ERR_INVALID_ARG, "acid_mha_backward_workspace_size: bytes is null");
  *bytes = backward_bytes(*mha);
  return ACID_OK;
}

extern "C" acid_status acid_mha_forward(const acid_mha* mha, const void* q, int64_t ldq, const void* k, int64_t ldk,
                                        const void* v, int64_t ldv, void* out, int64_t ldo, float* lse, void* ws,
                                        size_t ws_bytes, acid_stream_t stream) {
  clear_error();
  ACID_TRY(check_mha(mha));
  const acid_mha& m = *mha;
  ACID_TRY(check_operand(m, q, ldq, m.nq, m.heads, "q"));
  ACID_TRY(check_operand(m, k, ldk, m.nk, m.kv_heads, "k"));
  ACID_TRY(check_operand(m, v, ldv, m.nk, m.kv_heads, "v"));
  ACID_TRY(check_operand(m, out, ldo, m.nq, m.heads, "out"));
  if (m.nq == 0) return ACID_OK;
  ACID_REQUIRE(lse != nullptr && aligned(lse, 4), ACID_ERR_INVALID_ARG, "acid_mha_forward: lse is null or not aligned");
  ACID_TRY(check_workspace(ws, ws_bytes, forward_bytes(m), "acid_mha_forward"));
  MhaArgs a = common_args(m);
  a.q = q;
  a.ldq = ldq;
  a.k = k;
  a.ldk = ldk;
  a.v = v;
  a.ldv = ldv;
  a.out = out;
  a.ldo = ldo;
  a.lse = lse;
  a.part = ws;
  a.part_bytes = ws_bytes;
  if (mha_few(a)) return mha_forward_few(a, (cudaStream_t)stream);
  return m.dtype == ACID_BF16 ? mha_forward_tc(a, (cudaStream_t)stream) : mha_forward_f32(a, (cudaStream_t)stream);
}

extern "C" acid_status acid_mha_backward(const acid_mha* mha, const void* dout, int64_t lddo, const void* q, int64_t ldq,
                                         const void* k, int64_t ldk, const void* v, int64_t ldv, const void* out,
                                         int64_t ldo, const float* lse, const acid_mha_grads* grads, void* ws,
                                         size_t ws_bytes, acid_stream_t stream) {
  clear_error();
  ACID_TRY(check_mha(mha));
  const acid_mha& m = *mha;
  cudaStream_t s = (cudaStream_t)stream;
  ACID_REQUIRE(grads != nullptr, ACID_ERR_INVALID_ARG, "acid_mha_backward: null gradients");
  const acid_mha_grads& o = *grads;
  ACID_REQUIRE(o.dq || o.dk || o.dv || (m.nq == 0 && m.nk == 0), ACID_ERR_INVALID_ARG,
               "acid_mha_backward: need dq, dk or dv");
  ACID_TRY(check_operand(m, dout, lddo, m.nq, m.heads, "dout"));
  ACID_TRY(check_operand(m, q, ldq, m.nq, m.heads, "q"));
  ACID_TRY(check_operand(m, k, ldk, m.nk, m.kv_heads, "k"));
  ACID_TRY(check_operand(m, v, ldv, m.nk, m.kv_heads, "v"));
  ACID_TRY(check_operand(m, out, ldo, m.nq, m.heads, "out"));
  ACID_TRY(check_gradient(m, o.dq, o.lddq, m.nq, m.heads, "dq"));
  ACID_TRY(check_gradient(m, o.dk, o.lddk, m.nk, m.kv_heads, "dk"));
  ACID_TRY(check_gradient(m, o.dv, o.lddv, m.nk, m.kv_heads, "dv"));
  ACID_REQUIRE(m.nq == 0 || (lse != nullptr && aligned(lse, 4)), ACID_ERR_INVALID_ARG,
               "acid_mha_backward: lse is null or not aligned");
  if (m.nq == 0 && m.nk == 0) return ACID_OK;
  ACID_TRY(check_workspace(ws, ws_bytes, backward_bytes(m), "acid_mha_backward"));
  MhaArgs a = common_args(m);
  a.q = q;
  a.ldq = ldq;
  a.k = k;
  a.ldk = ldk;
  a.v = v;
  a.ldv = ldv;
  a.out = const_cast<void*>(out);
  a.ldo = ldo;
  a.lse = const_cast<float*>(lse);
  a.dout = dout;
  a.lddo = lddo;
  a.dq = m.nq > 0 ? o.dq : nullptr;
  a.lddq = o.lddq;
  a.dk = m.nk > 0 ? o.dk : nullptr;
  a.lddk = o.lddk;
  a.dv = m.nk > 0 ? o.dv : nullptr;
  a.lddv = o.lddv;
  a.stats = static_cast<float*>(ws);
  a.part = static_cast<uint8_t*>(ws) + stat_bytes(m);
  a.part_bytes = ws_bytes - stat_bytes(m);
  if (m.nq > 0) {
    const StatArgs t{a.shape, out, dout, ldo, lddo, lse, a.stats, m.head_dim, stat_slots(m),
                     m.dtype == ACID_BF16 ? 1.4426950408889634f : 1.0f};
    int lanes = 4;
    while (lanes * 8 < m.head_dim) lanes *= 2;
    launch_pdl(m.dtype == ACID_BF16 ? mha_stats_kernel<__nv_bfloat16> : mha_stats_kernel<float>,
               dim3(t.slots, m.heads), kThreads, 0, s, t, lanes);
    ACID_CHECK_LAUNCH();
  }
  return m.dtype == ACID_BF16 ? mha_backward_tc(a, s) : mha_backward_f32(a, s);
}

extern "C" acid_status acid_mha_clear_padding(const acid_mha* mha, int32_t keys, void* a, int64_t lda, void* b,
                                              int64_t ldb, float* lse, acid_stream_t stream) {
  clear_error();
  ACID_TRY(check_mha(mha));
  const acid_mha& m = *mha;
  const int64_t rows = keys ? m.nk : m.nq;
  const int heads = keys ? m.kv_heads : m.heads;
  ACID_TRY(check_gradient(m, a, lda, rows, heads, "a"));
  ACID_TRY(check_gradient(m, b, ldb, rows, heads, "b"));
  ACID_REQUIRE(aligned(lse, 4) && (lse == nullptr || !keys), ACID_ERR_INVALID_ARG,
               "acid_mha_clear_padding: lse not aligned, or with the keys' rows");
  const int32_t* bounds = keys ? m.k_bounds : m.q_bounds;
  if (bounds == nullptr || rows == 0 || (a == nullptr && b == nullptr && lse == nullptr)) return ACID_OK;
  const int64_t size = m.dtype == ACID_BF16 ? 2 : 4;
  ACID_REQUIRE(heads * m.head_dim * size <= INT32_MAX, ACID_ERR_UNSUPPORTED, "acid_mha_clear_padding: rows too wide");
  const PaddingArgs p{reinterpret_cast<const int2*>(bounds), m.sequences, (int)rows, heads, (int)(heads * m.head_dim * size),
                      static_cast<uint8_t*>(a), static_cast<uint8_t*>(b), lda * size, ldb * size, lse};
  launch_pdl(mha_padding_kernel, (unsigned)((rows + kThreads / 32 - 1) / (kThreads / 32)), kThreads, 0,
             (cudaStream_t)stream, p);
  ACID_CHECK_LAUNCH();
  return ACID_OK;
}
