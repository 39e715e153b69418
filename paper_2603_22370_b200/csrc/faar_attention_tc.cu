// Attention for head_dim 64 and 128 on the tcgen05 tensor cores (sm_100a).  Forward: attn_fwd_tc_kernel for whole causal sequences,
// attn_fwd_scored_kernel for key ranges with capped or biased scores, a kernel of its own.  Backward: attn_dq_tc_kernel and
// attn_dkv_tc_kernel are compiled for either (FORM), attn_scored_rows_kernel prepares the forms over ranges.  They are built like the
// causal forward kernel and described where they start.
//
// Causal forward.  One CTA takes 128 queries of one head and sweeps the keys in tiles of 64 (one sweep):
//   S   = Q K_j^T       tcgen05.mma  M = 128, N = 64, K = d    -> 64 FP32 columns of tensor memory
//   P_j = 2^(c S - m)   four warps, one query row per thread (its tensor-memory lane): no shuffles; the row
//                       goes back to tensor memory as BF16 pairs, 32 columns (tcgen05.st)
//   O  += P_j V_j       tcgen05.mma  M = 128, N = d, K = 64    accumulating in d more columns over the whole sweep;
//                       P_j is the A operand, read from tensor memory; V_j is read from shared memory as it lies
//                       in memory (keys as rows: a B operand with its N index contiguous)
//   m is the row's reference, not its running maximum: it moves to a tile's maximum only when that exceeds it by
//   more than 2^8 (probabilities stay below 2^8, the final division by their sum and lse = m + log2(sum) are
//   exact either way); only then is O rescaled, in tensor memory, between two P V products.
// Q, K_j, V_j arrive by TMA (two stages for K and V).  A fifth warp issues every copy and every MMA (by one lane of a
// converged warp: fwd 145.5 -> 140.6 us, bwd 385 -> 354 us at 4 x 2048 tokens, 32 heads, against a lane-0 branch); the
// scores have two buffers in tensor memory, so S of tile j + 1 is formed while the warps work on tile j, and two
// CTAs per SM overlap what remains serial (softmax -> P V).
// Rows of a tile beyond the sequence end arrive as zeros (the copies' maps have the sequence as a dimension of its own): a
// probability of 0 for a masked key would not keep an infinity or NaN of the next sequence's rows out of a product.  Query
// rows beyond the end are not stored; keys beyond it are masked.
// Every barrier wait is bounded; a wait that gives up records a code in a status word of this module (read by
// faar_attention_status), raises the CTA's abort flag and all roles leave.
#include <cuda.h>
#include <limits.h>

#include <type_traits>

#include "faar_internal.cuh"

namespace {

constexpr int QT = 128, KT = 64;
constexpr int CTL = 256;
// Rows are staged in panels of 64 columns (128 bytes, one swizzle row): a head of 128 has two panels per tile.
constexpr int Q_PANEL = QT * 128, KV_PANEL = KT * 128;
// Forward.  Tensor memory, 256 columns and two CTAs per SM for both head sizes: S of even / odd tiles in columns 0..63 /
// 64..127, O from 128.  head_dim 64 leaves room for P of its own (192..223 / 224..255); with head_dim 128 O takes the
// rest, and P_j is written over the first half of S_j, which its thread has just read.
// Measured against the fragment kernels that head_dim 128 took before (16 / 8 heads): 2 x 1000 tokens forward 292 -> 23 us,
// backward 798 -> 87 us; 4 x 2048 tokens 1681 -> 90 us (761 TFLOP/s) and 4253 -> 363 us.  Bound by the row threads (one 2^x
// per score on the special-function unit and the instructions around it), not by the tensor pipe.
template <int HD> struct Fwd {
  static constexpr int NP = HD / 64, Q_BYTES = NP * Q_PANEL, KV_BYTES = NP * KV_PANEL;
  static constexpr int OFF_K = Q_BYTES, OFF_V = OFF_K + 2 * KV_BYTES, OFF_CTL = OFF_V + 2 * KV_BYTES;
  static constexpr int SMEM = OFF_CTL + CTL + 1024;
  static constexpr bool P_OVER_S = HD == 128;
  static constexpr int COL_O = 128;
  static __device__ __forceinline__ uint32_t col_p(int j) { return P_OVER_S ? 64u * (uint32_t)(j & 1) : 192u + 32u * (uint32_t)(j & 1); }
};
constexpr int THREADS = 160;
constexpr int TMEM_COLS = 256;
constexpr float FWD_SLACK = 8.0f;                  // log2 of how far a tile's maximum may exceed the row's reference
constexpr unsigned long long LIMIT_NS = 2000000000ull;

__device__ uint32_t g_attn_status;                 // 0 = no wait has given up since the last read-and-clear

// The forms of a kernel's scores.  CAUSAL is whole causal sequences, compiled without anything of the others; all others go by
// a range of keys per query, and may cap the scores, bias them by distance, or both.
enum { CAUSAL = 0, RANGES = 1, CAPPED = 2, BIASED = 4 };

// tanh(t) / t as a polynomial in t^2, for |t| <= CAP_NEAR: the least maximum of the relative error among those of degree 5 (1.3e-7),
// found by iteratively reweighted least squares on Chebyshev points.
constexpr int CAP_TERMS = 6;
constexpr float CAP_NEAR = 0.8660254f;             // t^2 <= 0.75
constexpr double CAP_SERIES[CAP_TERMS] = {0.999999866180388, -0.33332032839016174, 0.13312545291211608, -0.05272645227582916,
                                          0.01837978821405255, -0.003900106715071943};

struct ScoreArgs {
  float cap_in, cap_out;           // t = cap_in S, capped score = cap_out tanh(t): in units of log2, as all scores here
  float cap_series[CAP_TERMS];     // times cap_out
  float tanh_series[CAP_TERMS];
  const float* slopes;             // [H]
  const int* key_lo; const int* key_hi;      // [B, S]
  const int4* tiles;               // backward: of every 64 queries, see attn_scored_rows_kernel
};

struct TcParams {
  __nv_bfloat16* out; float* lse;
  long long ldo;
  int B, S, H, Hkv;
  float scale_log2;
  ScoreArgs sc;
};

__device__ __forceinline__ uint32_t s32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint32_t b, uint32_t n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(b), "r"(n)); }
__device__ __forceinline__ void bar_arrive(uint32_t b) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(b) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t b, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(b), "r"(bytes) : "memory");
}
__device__ __forceinline__ uint32_t bar_try(uint32_t b, uint32_t parity) {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}"
               : "=r"(ok) : "r"(b), "r"(parity) : "memory");
  return ok;
}
__device__ __forceinline__ unsigned long long now_ns() {
  unsigned long long t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
__device__ __noinline__ bool bar_wait_slow(uint32_t b, uint32_t parity, volatile int* abort_flag, uint32_t code) {
  const unsigned long long t0 = now_ns();
  for (uint32_t spin = 1;; ++spin) {
    if (bar_try(b, parity)) return true;
    if ((spin & 0xFF) == 0) {
      if (*abort_flag) return false;
      if (now_ns() - t0 > LIMIT_NS) { atomicCAS(&g_attn_status, 0u, code); *abort_flag = 1; return false; }
    }
  }
}
__device__ __forceinline__ bool bar_wait(uint32_t b, uint32_t parity, volatile int* abort_flag, uint32_t code) {
  return bar_try(b, parity) ? true : bar_wait_slow(b, parity, abort_flag, code);
}
__device__ __forceinline__ void tma_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// Operand with the contraction index contiguous: rows of 128 bytes, 128-byte swizzle, 8-row groups 1024 B apart.
__device__ __forceinline__ uint64_t desc_k_major(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3FFFF) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) |
         ((uint64_t)2 << 61);
}
// Operand with its N index contiguous (64 of them = one 128-byte row per contraction index): groups of 8
// contraction indices 1024 B apart; the second 64-wide group along N (head_dim 128) is the next 64-row panel, 8192 B on.
__device__ __forceinline__ uint64_t desc_n_major(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3FFFF) >> 4) | ((uint64_t)(8192 >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
         ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// D = F32, A = B = BF16, M = 128; bit 16: B has its N index contiguous.
__device__ __forceinline__ constexpr uint32_t idesc(int n, int b_n_major) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)b_n_major << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(QT >> 4) << 24);
}
__device__ __forceinline__ void mma(uint32_t d, uint64_t da, uint64_t db, uint32_t id, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d), "l"(da), "l"(db), "r"(id), "r"(acc) : "memory");
}
// 32 consecutive FP32 columns of this thread's tensor-memory lane
__device__ __forceinline__ void ld32(uint32_t taddr, float (&r)[32]) {
  uint32_t u[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
      "%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]),
        "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]),
        "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]),
        "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
      : "r"(taddr) : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) r[i] = __uint_as_float(u[i]);
}
// Two such loads in flight together (one wait for both)
__device__ __forceinline__ void ld32x2(uint32_t ta, uint32_t tb, float (&a)[32], float (&b)[32]) {
  uint32_t u[32], v[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%64];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,%48,%49,%50,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63}, [%65];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31]),
        "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(ta), "r"(tb) : "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) { a[i] = __uint_as_float(u[i]); b[i] = __uint_as_float(v[i]); }
}
// Loads and stores of tensor memory are instructions of the whole warp.  Rows beyond the end of a sequence store nothing, so where
// another load follows such stores a __syncwarp brings the lanes together: nothing else does.
__device__ __forceinline__ void ld16(uint32_t ta, float (&a)[16]) {
  uint32_t u[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]), "=r"(u[10]),
        "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
      : "r"(ta) : "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) a[i] = __uint_as_float(u[i]);
}
__device__ __forceinline__ void ld16x2(uint32_t ta, uint32_t tb, float (&a)[16], float (&b)[16]) {
  uint32_t u[16], v[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%32];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%33];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]), "=r"(u[10]),
        "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]),
        "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(ta), "r"(tb) : "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) { a[i] = __uint_as_float(u[i]); b[i] = __uint_as_float(v[i]); }
}
// 32 consecutive 32-bit columns of this thread's tensor-memory lane, written (BF16 pairs of an A operand)
__device__ __forceinline__ void st32(uint32_t taddr, const uint32_t (&u)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
      "%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
      ::"r"(taddr), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]),
        "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]), "r"(u[16]), "r"(u[17]), "r"(u[18]), "r"(u[19]),
        "r"(u[20]), "r"(u[21]), "r"(u[22]), "r"(u[23]), "r"(u[24]), "r"(u[25]), "r"(u[26]), "r"(u[27]), "r"(u[28]), "r"(u[29]),
        "r"(u[30]), "r"(u[31])
      : "memory");
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void st16(uint32_t taddr, const uint32_t (&u)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
      ::"r"(taddr), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]),
        "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15])
      : "memory");
}
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// D = A B^T over d contraction elements, both operands staged row by row (panels of 64 elements, pa / pb bytes apart)
template <int HD>
__device__ __forceinline__ void mma_rows(uint32_t d, uint32_t sa, uint32_t pa, uint32_t sb, uint32_t pb, uint32_t id) {
#pragma unroll
  for (int k = 0; k < HD / 16; ++k)
    mma(d, desc_k_major(sa + (k >> 2) * pa) + 2u * (k & 3), desc_k_major(sb + (k >> 2) * pb) + 2u * (k & 3), id, k != 0 ? 1u : 0u);
}
// D (+)= A B with A read from tensor memory (128 lanes = rows, two BF16 contraction elements per 32-bit column,
// the lower index in the lower half) and B from shared memory
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a_tmem, uint64_t db, uint32_t id, uint32_t acc) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
               ::"r"(d), "r"(a_tmem), "l"(db), "r"(id), "r"(acc) : "memory");
}
// 2^x on the special-function unit, one instruction (relative error about 2^-22; -inf gives 0; results below the
// normal range are flushed to zero, which is what a probability that small should be)
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// max of three in one instruction
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}

// NP boxes of 64 columns, rows from `row` of sequence b (rows beyond the sequence arrive as zeros)
template <int HD>
__device__ __forceinline__ void tma_head(uint32_t dst, uint32_t panel, const CUtensorMap* map, int x, int row, int b, uint32_t bar) {
#pragma unroll
  for (int c = 0; c < HD / 64; ++c) tma_3d(dst + c * panel, map, x + 64 * c, row, b, bar);
}

// ---- scores beyond the causal form -------------------------------------------------------------------------------
// A query's keys, cut to its sequence.  An empty range gives bounds that any other undoes in a minimum or maximum; sequences of
// up to 2^30 tokens leave room for differences of positions.
constexpr int EMPTY_LO = 0x40000000, EMPTY_HI = 0;
__device__ __forceinline__ int2 key_range(const ScoreArgs& a, int b, int q, int S) {
  const long long at = (long long)b * S + q;
  const int lo = a.key_lo ? max(a.key_lo[at], 0) : 0, hi = a.key_hi ? min(a.key_hi[at], S) : q + 1;
  return lo < hi ? make_int2(lo, hi) : make_int2(EMPTY_LO, EMPTY_HI);
}
// Bit i: key k0 + i is in the range
__device__ __forceinline__ uint32_t bits_below(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; }
__device__ __forceinline__ uint32_t range_bits(int2 r, int k0) { return bits_below(r.y - k0) & ~bits_below(r.x - k0); }

// What the 128 queries of a tile see together: keys from `lo` on and before `hi` are seen by one at least, from `all_lo` on and
// before `all_hi` by every one.  `r`: the calling thread's query, where it has one (warps 0 .. 3: one each); `slots`: 16 ints of
// shared memory.  All threads of the CTA call it.
struct Span { int lo, hi, all_lo, all_hi; };
__device__ __forceinline__ Span tile_span(int2 r, bool row, volatile int* slots) {
  const int warp = threadIdx.x >> 5;
  const bool some = row && r.x < r.y;
  const int lo = __reduce_min_sync(0xffffffffu, some ? r.x : EMPTY_LO), hi = __reduce_max_sync(0xffffffffu, some ? r.y : EMPTY_HI);
  const int all_lo = __reduce_max_sync(0xffffffffu, row ? r.x : 0), all_hi = __reduce_min_sync(0xffffffffu, row ? r.y : INT_MAX);
  if (warp < 4 && (threadIdx.x & 31) == 0) { slots[4 * warp] = lo; slots[4 * warp + 1] = hi; slots[4 * warp + 2] = all_lo; slots[4 * warp + 3] = all_hi; }
  __syncthreads();
  Span s = {slots[0], slots[1], slots[2], slots[3]};
#pragma unroll
  for (int w = 1; w < 4; ++w) {
    s.lo = min(s.lo, slots[4 * w]); s.hi = max(s.hi, slots[4 * w + 1]);
    s.all_lo = max(s.all_lo, slots[4 * w + 2]); s.all_hi = min(s.all_hi, slots[4 * w + 3]);
  }
  return s;
}

__device__ __forceinline__ float2 pair(float x) { return make_float2(x, x); }
// tanh(t) cap_out + o, of two values: a polynomial for |t| <= CAP_NEAR, and beyond it 1 - 2 / (1 + 2^(2 t
// log2 e)) on the special-function units.  Which one goes by the value alone, so that a score is the same bits whatever lies next
// to it; a warp without any beyond skips the second.
__device__ __forceinline__ float2 cap_near(float2 t, const ScoreArgs& a, float2 o) {
  const float2 y = __fmul2_rn(t, t);
  float2 q = pair(a.cap_series[CAP_TERMS - 1]);
#pragma unroll
  for (int k = CAP_TERMS - 2; k >= 0; --k) q = __ffma2_rn(q, y, pair(a.cap_series[k]));
  return __ffma2_rn(t, q, o);
}
__device__ __forceinline__ float cap_far(float t, const ScoreArgs& a, float o) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + ex2(t * 2.885390081777927f)));
  return fmaf(-2.0f * a.cap_out, r, a.cap_out + o);
}
// Whether some value of the warp's is beyond the polynomial (one that is no number is, or ends as none)
template <int N>
__device__ __forceinline__ bool cap_any_far(const float (&s)[N], const ScoreArgs& a) {
  float m[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    m[0] = max3(m[0], fabsf(s[i]), fabsf(s[i + 1]));
    m[1] = max3(m[1], fabsf(s[i + 2]), fabsf(s[i + 3]));
  }
  return __any_sync(0xffffffffu, !(fmaxf(m[0], m[1]) * a.cap_in <= CAP_NEAR));
}
// Products S -> scores in units of log2 minus `ref`, in place: 32 values of a row whose partners lie side by side, the first at
// distance `first` (query - key), each further one STEP (-1 along keys, +1 along queries) from it.  The bias is linear along the
// values on either side of distance 0.  PLAIN: all lie on one side (`slope` negated where that is the negative one), and none
// is beyond the cap's polynomial; a value is the same bits either way.
template <int FORM, int STEP, bool PLAIN>
__device__ __forceinline__ void score_values(float (&s)[32], const ScoreArgs& a, float scale_log2, float slope, int first, float ref) {
  const float2 start = pair(fmaf(-slope, (float)first, -ref));
  auto offsets = [&](int i) {                                  // minus the reference, minus the bias
    if constexpr ((FORM & BIASED) == 0) return pair(-ref);
    const float2 at = make_float2((float)i, (float)(i + 1));
    float2 o = __ffma2_rn(pair(-slope * (float)STEP), at, start);
    if (!PLAIN) {
      const float2 other = __ffma2_rn(pair(slope * (float)STEP), at, pair(fmaf(slope, (float)first, -ref)));
      if (first + STEP * i < 0) o.x = other.x;
      if (first + STEP * (i + 1) < 0) o.y = other.y;
    }
    return o;
  };
  auto all = [&](auto far) {
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
      float2 r;
      if constexpr ((FORM & CAPPED) != 0) {
        const float2 t = __fmul2_rn(make_float2(s[i], s[i + 1]), pair(a.cap_in)), o = offsets(i);
        r = cap_near(t, a, o);
        if constexpr (decltype(far)::value) {
          const float2 f = make_float2(cap_far(t.x, a, o.x), cap_far(t.y, a, o.y));
          r.x = fabsf(t.x) <= CAP_NEAR ? r.x : f.x;
          r.y = fabsf(t.y) <= CAP_NEAR ? r.y : f.y;
        }
      } else {
        r = __ffma2_rn(make_float2(s[i], s[i + 1]), pair(scale_log2), offsets(i));
      }
      s[i] = r.x; s[i + 1] = r.y;
    }
  };
  if ((FORM & CAPPED) && !PLAIN && cap_any_far(s, a)) all(std::true_type{}); else all(std::false_type{});
}
// The backward kernels need tanh itself, in place of products S: cap_out tanh is the score, 1 - tanh^2 its slope.
__device__ __forceinline__ void tanh_values(float (&s)[32], const ScoreArgs& a) {
  auto beyond = [](float t) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + ex2(t * 2.885390081777927f)));
    return fmaf(-2.0f, r, 1.0f);
  };
  auto all = [&](auto far) {
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
      const float2 t = __fmul2_rn(make_float2(s[i], s[i + 1]), pair(a.cap_in)), y = __fmul2_rn(t, t);
      float2 q = pair(a.tanh_series[CAP_TERMS - 1]);
#pragma unroll
      for (int k = CAP_TERMS - 2; k >= 0; --k) q = __ffma2_rn(q, y, pair(a.tanh_series[k]));
      float2 r = __fmul2_rn(t, q);
      if constexpr (decltype(far)::value) {
        const float2 f = make_float2(beyond(t.x), beyond(t.y));
        r.x = fabsf(t.x) <= CAP_NEAR ? r.x : f.x;
        r.y = fabsf(t.y) <= CAP_NEAR ? r.y : f.y;
      }
      s[i] = r.x; s[i + 1] = r.y;
    }
  };
  if (cap_any_far(s, a)) all(std::true_type{}); else all(std::false_type{});
}
// x plus the bias of distances d and d + STEP; nb: minus the head's slope in units of log2
template <int STEP>
__device__ __forceinline__ float2 add_bias(float2 x, float nb, float d) {
  return __ffma2_rn(pair(nb), make_float2(fabsf(d), fabsf(d + (float)STEP)), x);
}

// Rows of an operand that some of the rows working with it may not see: what is not finite there would reach them all, as 0 times
// an infinity is no 0.  Such values of a staged tile are set to 0 (`units` 16-byte units from `base` on, of which the calling thread
// takes every `threads`-th from `first` on; `found`: a word in shared memory that gets `bits` where there are any, or 0); the generic
// writes are made visible to the tensor cores.
__device__ __forceinline__ bool not_finite(uint4 v) {        // all exponent bits of one of eight BF16 values set
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t acc = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) acc |= (w[i] & 0x7F807F80u) + 0x00800080u;
  return (acc & 0x80008000u) != 0;
}
__device__ __forceinline__ uint32_t only_finite(uint32_t w) {
  if ((w & 0x7F80u) == 0x7F80u) w &= 0xFFFF0000u;
  if ((w & 0x7F800000u) == 0x7F800000u) w &= 0x0000FFFFu;
  return w;
}
__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __noinline__ void scrub(uint32_t base, int units, int first, int threads, uint32_t found, uint32_t bits) {
  for (int u = first; u < units; u += threads) {
    const uint32_t at = base + 16u * (uint32_t)u;
    const uint4 v = lds128(at);
    if (!not_finite(v)) continue;
    if (found) asm volatile("red.shared.or.b32 [%0], %1;" ::"r"(found), "r"(bits) : "memory");
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(only_finite(v.x)), "r"(only_finite(v.y)), "r"(only_finite(v.z)),
                 "r"(only_finite(v.w)) : "memory");
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}
// Tiles of KT rows where something was found: a bit each, modulo 32
__device__ __forceinline__ uint32_t tile_bit(int tile) { return 1u << (tile & 31); }
__device__ __forceinline__ uint32_t found_tiles(uint32_t found) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(found) : "memory");
  return v;
}
// Whether a row of HD values in memory holds one that is not finite
template <int HD>
__device__ __forceinline__ bool row_not_finite(const __nv_bfloat16* row) {
  bool any = false;
#pragma unroll 4
  for (int c = 0; c < HD; c += 8) any |= not_finite(*reinterpret_cast<const uint4*>(row + c));
  return any;
}
// NaN if one of N products is not finite, else 0 (+ acc)
template <int N>
__device__ __forceinline__ float2 finite_probe(const float (&s)[N], float2 acc) {
#pragma unroll
  for (int i = 0; i < N; i += 2) acc = __ffma2_rn(make_float2(s[i], s[i + 1]), pair(0.f), acc);
  return acc;
}

template <int HD>
__global__ void __launch_bounds__(THREADS, 2)
attn_fwd_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                     const __grid_constant__ CUtensorMap tmV, const TcParams p) {
  using F = Fwd<HD>;
  constexpr int KV_BYTES = F::KV_BYTES, Q_BYTES = F::Q_BYTES, OFF_CTL = F::OFF_CTL, OFF_K = F::OFF_K, OFF_V = F::OFF_V;
  extern __shared__ uint8_t raw[];
  const uint32_t base = (s32(raw) + 1023u) & ~1023u;
  uint8_t* smem = raw + (base - s32(raw));
  const uint32_t ctl = base + OFF_CTL;
  const uint32_t bar_q = ctl;
  // Tiles alternate between two barriers each for P written and P V complete.  With one, a phase could be over before it is waited
  // for (the row threads announce P_j before they look for P V_{j-1}), and its parity be taken for that of the next but one.  4 x 2048
  // tokens, us, one barrier each -> two: 32 heads of 64 130.5 -> 133.0, 16 of 128 86.8 -> 87.8.
  auto bar_p = [&](int j) { return ctl + 72u + 32u * (j & 1); };
  auto bar_o = [&](int j) { return ctl + 80u + 32u * (j & 1); };
  auto kfull = [&](int s) { return ctl + 8u + 8u * s; };
  auto vfull = [&](int s) { return ctl + 24u + 8u * s; };
  auto bar_s = [&](int s) { return ctl + 40u + 8u * s; };         // scores of a tile in buffer s are complete
  auto bar_sfree = [&](int s) { return ctl + 56u + 8u * s; };     // ... have been read by all 128 rows
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem + OFF_CTL + 96);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + OFF_CTL + 100);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  // one-dimensional grid, query tile slowest and descending: CTAs start in order of decreasing work
  const int hb = p.H * p.B;
  const int qt = (int)(gridDim.x / hb) - 1 - (int)(blockIdx.x / hb);
  const int h = (blockIdx.x % hb) % p.H, b = (blockIdx.x % hb) / p.H;
  const int g = h / (p.H / p.Hkv);
  const long long seq0 = (long long)b * p.S;
  const int q0 = qt * QT;
  const int last_q = min(q0 + QT, p.S) - 1;
  const int n_kt = last_q / KT + 1;                          // key tiles that some query of this tile sees

  if (threadIdx.x == 0) {
    bar_init(bar_q, 1);
    for (int s = 0; s < 2; ++s) { bar_init(kfull(s), 1); bar_init(vfull(s), 1); }
    for (int s = 0; s < 2; ++s) { bar_init(bar_s(s), 1); bar_init(bar_sfree(s), 128); }
    for (int s = 0; s < 2; ++s) { bar_init(bar_o(s), 1); bar_init(bar_p(s), 128); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 4) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(s32(const_cast<uint32_t*>(tmem_slot))),
                 "r"((uint32_t)TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = *tmem_slot;
  faar_pdl_sync();                                          // set-up done; now wait for the previous kernel's data
  const uint32_t sQ = base;
  auto sK = [&](int s) { return base + OFF_K + (uint32_t)s * KV_BYTES; };
  auto sV = [&](int s) { return base + OFF_V + (uint32_t)s * KV_BYTES; };

  if (warp == 4) {
    // ---------------- copies and MMAs: one lane of this warp, which stays converged (see faar_elect_one; copies issued under
    // `if (lane == 0)` cost the 64-element heads' backward pass 3 %) ----------
    auto wait = [&](uint32_t bar, uint32_t parity, uint32_t code) {
      return __all_sync(0xffffffffu, bar_wait(bar, parity, abort_flag, code)) != 0;
    };
    auto load_k = [&](int j) {
      if (faar_elect_one()) { bar_expect(kfull(j & 1), KV_BYTES); tma_head<HD>(sK(j & 1), KV_PANEL, &tmK, g * HD, j * KT, b, kfull(j & 1)); }
      __syncwarp();
    };
    auto load_v = [&](int j) {
      if (faar_elect_one()) { bar_expect(vfull(j & 1), KV_BYTES); tma_head<HD>(sV(j & 1), KV_PANEL, &tmV, g * HD, j * KT, b, vfull(j & 1)); }
      __syncwarp();
    };
    if (faar_elect_one()) {
      bar_expect(bar_q, Q_BYTES);
      tma_head<HD>(sQ, Q_PANEL, &tmQ, h * HD, q0, b, bar_q);
    }
    load_k(0); load_v(0);
    if (n_kt > 1) { load_k(1); load_v(1); }
    bool ok = wait(bar_q, 0u, 0xA01u);
    constexpr uint32_t id_s = idesc(KT, 0), id_pv = idesc(HD, 1);
    // S of tile j into score buffer j & 1.  The scores of tile j + 1 are issued before this warp waits for the
    // probabilities of tile j, so the tensor cores form them while the four warps work on tile j.
    auto issue_s = [&](int j) {
      if (faar_elect_one()) {
        mma_rows<HD>(tmem + 64u * (uint32_t)(j & 1), sQ, Q_PANEL, sK(j & 1), KV_PANEL, id_s);
        commit(bar_s(j & 1));
      }
      __syncwarp();
    };
    if (ok) ok = wait(kfull(0), 0u, 0xA10u);
    if (ok) { fence_after(); issue_s(0); }
    for (int j = 0; j < n_kt && ok; ++j) {
      const int st = j & 1;
      const uint32_t ph = (uint32_t)((j >> 1) & 1);
      if (j + 1 < n_kt) {
        ok = wait(kfull((j + 1) & 1), (uint32_t)(((j + 1) >> 1) & 1), 0xA10u | ((j + 1) & 1));
        // its score buffer last held tile j - 1: read by all rows (or, holding P_{j-1} by now, consumed by P V_{j-1})
        if (ok && j >= 1)
          ok = F::P_OVER_S ? wait(bar_o(j - 1), (uint32_t)(((j - 1) >> 1) & 1), 0xA20u) : wait(bar_sfree((j + 1) & 1), (uint32_t)(((j - 1) >> 1) & 1), 0xA20u);
        if (!ok) break;
        fence_after();
        issue_s(j + 1);
      }
      // P_j written (into P buffer j & 1): S_j has been read, so its K stage is free
      ok = wait(bar_p(j), ph, 0xA30u);
      if (!ok) break;
      if (j + 2 < n_kt) load_k(j + 2);
      ok = wait(vfull(st), ph, 0xA40u | st);
      // P V_{j-1} complete: its V stage is free
      if (ok && j > 0) ok = wait(bar_o(j - 1), (uint32_t)(((j - 1) >> 1) & 1), 0xA50u);
      if (!ok) break;
      if (j >= 1 && j + 1 < n_kt) load_v(j + 1);
      fence_after();
      const uint64_t db = desc_n_major(sV(st));
      const uint32_t ta = tmem + F::col_p(j);                        // P_j: 16 contraction steps = 8 columns
      if (faar_elect_one()) {
#pragma unroll
        for (int k = 0; k < KT / 16; ++k) mma_ts(tmem + (uint32_t)F::COL_O, ta + 8u * k, db + 128u * k, id_pv, (j | k) != 0 ? 1u : 0u);
        commit(bar_o(j));
      }
      __syncwarp();
    }
    if (!ok) { const unsigned long long t0 = now_ns(); while (now_ns() - t0 < 2000000ull) {} }   // copies in flight
  } else {
    // ---------------- softmax: thread = query row = tensor-memory lane ----------------
    const int row = 32 * warp + lane;
    const int qi = q0 + row;
    const uint32_t t_lane = tmem + ((uint32_t)(32 * warp) << 16), t_o = t_lane + (uint32_t)F::COL_O;
    float m = -INFINITY, l = 0.f;                             // the reference the row's probabilities are relative to; their sum
    bool ok = true;
    for (int j = 0; j < n_kt; ++j) {
      const int k0 = j * KT;
      const uint32_t t_s = t_lane + 64u * (uint32_t)(j & 1);
      ok = bar_wait(bar_s(j & 1), (uint32_t)((j >> 1) & 1), abort_flag, 0xB10u);
      if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
      fence_after();
      float s[KT];
      {
        float t[32], t2[32];
        ld32x2(t_s, t_s + 32u, t, t2);
#pragma unroll
        for (int i = 0; i < 32; ++i) { s[i] = t[i]; s[32 + i] = t2[i]; }
      }
      if (!F::P_OVER_S) {
        fence_before();
        bar_arrive(bar_sfree(j & 1));
      }
      if (k0 + KT - 1 > q0 || k0 + KT > p.S) {                // the tile crosses some row's diagonal, or the sequence end
#pragma unroll
        for (int i = 0; i < KT; ++i)
          if (!(k0 + i <= qi && k0 + i < p.S)) s[i] = -INFINITY;
      }
      float mx4[4] = {s[0], s[1], s[2], s[3]};                   // four independent chains, two scores per instruction
#pragma unroll
      for (int i = 4; i < KT; i += 8) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (i + 2 * c + 1 < KT) mx4[c] = max3(mx4[c], s[i + 2 * c], s[i + 2 * c + 1]);
      }
      const float m_tile = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * p.scale_log2;
      // The output accumulates in tensor memory over the whole sweep.  The row's reference moves only when a tile's
      // maximum exceeds it by more than 2^FWD_SLACK: until then the probabilities (at most 2^FWD_SLACK) and their sum
      // stay relative to the old one, which the final division and lse = m + log2(l) undo exactly, and the
      // accumulated output needs no rescaling.
      const float m_new = m_tile > m + FWD_SLACK ? m_tile : m;
      const float ref = m_new == -INFINITY ? 0.f : m_new;     // a row beyond the sequence may have seen no key
      const float alpha = ex2(m - ref);                       // 1 while the reference stays
      const bool moved = m_new != m && j > 0;
      bool prev_done = j == 0;                                // P V_{j-1} known to be complete
      if (__any_sync(0xffffffffu, moved)) {                   // O = O * 2^(m_old - m_new), between P V_{j-1} and P V_j
        ok = bar_wait(bar_o(j - 1), (uint32_t)(((j - 1) >> 1) & 1), abort_flag, 0xB20u);
        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
        prev_done = true;
        fence_after();
        const float a = moved ? alpha : 1.0f;
#pragma unroll
        for (int half = 0; half < HD / 32; ++half) {
          float t[32];
          uint32_t u[32];
          ld32(t_o + 32u * half, t);
#pragma unroll
          for (int i = 0; i < 32; ++i) u[i] = __float_as_uint(t[i] * a);
          st32(t_o + 32u * half, u);
        }
      }
      // exponent arguments and sums two at a time (packed FP32 multiply-add and add: the same roundings)
      const float2 sc2 = make_float2(p.scale_log2, p.scale_log2), nr2 = make_float2(-ref, -ref);
      float2 sum2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
      uint32_t pk[KT / 2];
#pragma unroll
      for (int w = 0; w < KT / 2; ++w) {
        const float2 x = __ffma2_rn(make_float2(s[2 * w], s[2 * w + 1]), sc2, nr2);
        const float2 e = make_float2(ex2(x.x), ex2(x.y));
        sum2[w & 1] = __fadd2_rn(sum2[w & 1], e);
        pk[w] = pack2(e.x, e.y);
      }
      st32(t_lane + F::col_p(j), pk);             // this row of P_j, an A operand in tensor memory
      fence_before();
      bar_arrive(bar_p(j));
      l = l * alpha + ((sum2[0].x + sum2[0].y) + (sum2[1].x + sum2[1].y));
      m = m_new;
      // every completion of P V is observed in order (it has had this tile's softmax to happen): P buffer j & 1 is
      // then free for tile j + 2
      if (!prev_done) {
        ok = bar_wait(bar_o(j - 1), (uint32_t)(((j - 1) >> 1) & 1), abort_flag, 0xB21u);
        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
      }
    }
    if (ok) {
      ok = bar_wait(bar_o(n_kt - 1), (uint32_t)(((n_kt - 1) >> 1) & 1), abort_flag, 0xB30u);
      ok = __all_sync(0xffffffffu, ok);
    }
    if (ok) {
      fence_after();
      const float inv = l > 0.f ? 1.0f / l : 0.f;
      uint4* dst = reinterpret_cast<uint4*>(p.out + (seq0 + qi) * p.ldo + h * HD);
#pragma unroll
      for (int pair = 0; pair < HD / 64; ++pair) {
        float t[2][32];
        ld32x2(t_o + 64u * pair, t_o + 64u * pair + 32u, t[0], t[1]);
        if (qi < p.S) {
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            const float* v = &t[c >> 2][8 * (c & 3)];
            dst[8 * pair + c] = make_uint4(pack2(v[0] * inv, v[1] * inv), pack2(v[2] * inv, v[3] * inv), pack2(v[4] * inv, v[5] * inv),
                                           pack2(v[6] * inv, v[7] * inv));
          }
        }
        if (pair + 1 < HD / 64) __syncwarp();
      }
      if (qi < p.S) p.lse[((long long)b * p.H + h) * p.S + qi] = m + log2f(l);
    }
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  if (warp == 4) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)TMEM_COLS) : "memory");
  }
}

// ---- forward over key ranges ----------------------------------------------------------------------------------------
// The products and buffers are the causal kernel's with heads of 128 (P_j over S_j), for both head sizes; one thread a query.
// No unit is full.  By counters, of the cycles that an SM is at work (heads of 64, documents of 700, capped; heads of 128, 8192 tokens, biased):
// instruction issue 43 / 44 %, FMA 37 / 23, 2^x 31 / 50, tensor pipe 15 / 50, with ten warps an SM: each of a scheduler's two or three
// row warps takes its scores' multiply-adds (a capped score takes eight), 2^x, packing and stores one after the other, and a product of 64 keys
// reads both operands from shared memory, 6 KB per 16 contraction steps, for half as long again as its tensor work.  So FMAs and 2^x come one
// after the other where a tile's maximum has to be known before its first 2^x.  So a tile is taken relative to the query's reference
// as it stands, scores and 2^x in one sweep, the maximum along with them; only where it turns out to lie above the reference by more
// than 2^SCORED_SLACK (or where there is none yet) the tile is read again and taken in two sweeps, with a new reference.  The keys'
// tiles come from the queries' own back to the first, then the later ones: next to the query a bias by distance is least, so that the
// first reference lasts, and where ranges end at the query itself the tile without a reference is one that has keys to mask, too.
// An infinity or NaN in V reaches all of a tile's queries in the product, those that do not see it by a probability of 0.  So a CTA
// that finds something in its output that is no finite number goes over its tiles once more, and this time rids V of such values where
// a tile has keys to mask, noting which keys they belong to.
// 4 x 2048 tokens, us (TFLOP/s of what is visible): 32 / 8 heads of 64, causal 132 (521; the causal kernel 133), biased 143 (481), capped
// 195 (353); 16 / 8 heads of 128 87 (790), 91 (755), 115 (598).  1 x 8192, 16 heads of 128, biased, one document: 262-268 (1026-1049);
// behind prefixes of up to 0.4 of the sequence, which it sees whole, 301-335.
template <int HD> struct FwdScored {
  static constexpr int NP = HD / 64, Q_BYTES = NP * Q_PANEL, KV_BYTES = NP * KV_PANEL;
  static constexpr int OFF_K = Q_BYTES, OFF_V = OFF_K + 2 * KV_BYTES, OFF_CTL = OFF_V + 2 * KV_BYTES;
  static constexpr int SMEM = OFF_CTL + CTL + 1024;
  static constexpr uint32_t COL_O = 128;                     // S_j, then P_j: 64 (j & 1)
  static_assert(2 * (SMEM + 1024) <= 228 * 1024, "two CTAs per SM");
};
constexpr float SCORED_SLACK = 32.0f;              // far from what overflows; sums, probabilities and outputs are floating point

template <int HD, int FORM>
__global__ void __launch_bounds__(THREADS, 2)
attn_fwd_scored_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                       const __grid_constant__ CUtensorMap tmV, const TcParams p) {
  using F = FwdScored<HD>;
  constexpr int KV_BYTES = F::KV_BYTES;
  extern __shared__ uint8_t raw[];
  const uint32_t base = (s32(raw) + 1023u) & ~1023u;
  uint8_t* smem = raw + (base - s32(raw));
  const uint32_t ctl = base + F::OFF_CTL;
  const uint32_t bar_q = ctl, bar_v = ctl + 88;                  // bar_v: V of an edge tile has been looked through
  auto kfull = [&](int s) { return ctl + 8u + 8u * s; };
  auto vfull = [&](int s) { return ctl + 24u + 8u * s; };
  auto bar_s = [&](int s) { return ctl + 40u + 8u * s; };         // scores of a tile in buffer s are complete
  auto bar_p = [&](int s) { return ctl + 56u + 8u * s; };         // probabilities of a tile in buffer s are written
  auto bar_o = [&](int s) { return ctl + 72u + 8u * s; };         // ... and their product with V has run
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem + F::OFF_CTL + 96);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + F::OFF_CTL + 100);
  uint32_t* const bad_keys = reinterpret_cast<uint32_t*>(smem + F::OFF_CTL + 192);        // 3 x 2
  const int warp = threadIdx.x >> 5;

  const int hb = p.H * p.B;
  const int qt = (int)(gridDim.x / hb) - 1 - (int)(blockIdx.x / hb);
  const int h = (blockIdx.x % hb) % p.H, b = (blockIdx.x % hb) / p.H;
  const int g = h / (p.H / p.Hkv);
  const long long seq0 = (long long)b * p.S;
  const int q0 = qt * QT, row = threadIdx.x, qi = q0 + row;      // (of the row threads)

  if (threadIdx.x == 0) {
    bar_init(bar_q, 1);
    for (int s = 0; s < 2; ++s) { bar_init(kfull(s), 1); bar_init(vfull(s), 1); bar_init(bar_s(s), 1); bar_init(bar_p(s), 128); bar_init(bar_o(s), 1); }
    bar_init(bar_v, 128);
    for (int i = 0; i < 6; ++i) bad_keys[i] = 0u;
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 4) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(s32(const_cast<uint32_t*>(tmem_slot))),
                 "r"((uint32_t)TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  faar_pdl_sync();                                          // the ranges may be the previous kernel's
  int2 range = {0, INT_MAX};                                // this thread's query (one beyond the end: anything will do)
  const bool is_row = warp < 4 && qi < p.S;
  if (is_row) range = key_range(p.sc, b, qi, p.S);
  fence_before();
  const Span span = tile_span(range, is_row, reinterpret_cast<volatile int*>(smem + F::OFF_CTL + 112));      // and the set-up, for all
  fence_after();
  const uint32_t tmem = *tmem_slot;
  const int kt0 = span.lo / KT, kt1 = (span.hi - 1) / KT, n_kt = span.lo < span.hi ? kt1 + 1 - kt0 : 0;      // key tiles that some query of this tile sees
  const int own = min(max((q0 + QT - 1) / KT, kt0), kt1), n_back = own - kt0 + 1;
  auto tile_at = [&](int j) { return j < n_back ? own - j : kt0 + j; };
  const uint32_t sQ = base;
  auto sK = [&](int s) { return base + F::OFF_K + (uint32_t)s * KV_BYTES; };
  auto sV = [&](int s) { return base + F::OFF_V + (uint32_t)s * KV_BYTES; };

  if (warp == 4) {
    // ---------------- copies and MMAs ----------------
    auto wait = [&](uint32_t bar, uint32_t parity, uint32_t code) {
      return __all_sync(0xffffffffu, bar_wait(bar, parity, abort_flag, code)) != 0;
    };
    // Tiles are counted on over both sweeps: u = sweep * n_kt + j, in buffers and stages u & 1
    auto load_k = [&](int u, int j) {
      if (faar_elect_one()) { bar_expect(kfull(u & 1), KV_BYTES); tma_head<HD>(sK(u & 1), KV_PANEL, &tmK, g * HD, tile_at(j) * KT, b, kfull(u & 1)); }
      __syncwarp();
    };
    auto load_v = [&](int u, int j) {
      if (faar_elect_one()) { bar_expect(vfull(u & 1), KV_BYTES); tma_head<HD>(sV(u & 1), KV_PANEL, &tmV, g * HD, tile_at(j) * KT, b, vfull(u & 1)); }
      __syncwarp();
    };
    constexpr uint32_t id_s = idesc(KT, 0), id_pv = idesc(HD, 1);
    auto issue_s = [&](int u) {
      if (faar_elect_one()) {
        mma_rows<HD>(tmem + 64u * (uint32_t)(u & 1), sQ, Q_PANEL, sK(u & 1), KV_PANEL, id_s);
        commit(bar_s(u & 1));
      }
      __syncwarp();
    };
    auto phase = [](int u) { return (uint32_t)((u >> 1) & 1); };
    bool ok = n_kt > 0;
    if (ok && faar_elect_one()) {
      bar_expect(bar_q, F::Q_BYTES);
      tma_head<HD>(sQ, Q_PANEL, &tmQ, h * HD, q0, b, bar_q);
    }
    __syncwarp();
    for (int u0 = 0;; u0 += n_kt) {
      if (ok) {
        load_k(u0, 0); load_v(u0, 0);
        if (n_kt > 1) { load_k(u0 + 1, 1); load_v(u0 + 1, 1); }
        if (u0 == 0) ok = wait(bar_q, 0u, 0xA01u);
        if (ok) ok = wait(kfull(u0 & 1), phase(u0), 0xA10u);
        if (ok) { fence_after(); issue_s(u0); }
        for (int j = 0; j < n_kt && ok; ++j) {
          const int u = u0 + j, st = u & 1;
          // P V of the tile before complete: its V stage and its buffer of tensor memory are free, for V of tile j + 1 and S_{j+1}
          if (j > 0) ok = wait(bar_o(st ^ 1), phase(u - 1), 0xA20u);
          if (ok && j + 1 < n_kt) {
            if (j >= 1) load_v(u + 1, j + 1);
            ok = wait(kfull(st ^ 1), phase(u + 1), 0xA10u | (st ^ 1));
            if (!ok) break;
            fence_after();
            issue_s(u + 1);
          }
          if (ok && j + 2 < n_kt) {                           // S_j complete: its K stage is free (K would come too late once P_j is there)
            ok = wait(bar_s(st), phase(u), 0xA25u);
            if (!ok) break;
            load_k(u + 2, j + 2);
          }
          if (ok) ok = wait(bar_p(st), phase(u), 0xA30u | st);
          if (ok) ok = wait(vfull(st), phase(u), 0xA40u | st);
          if (!ok) break;
          fence_after();
          const uint64_t db = desc_n_major(sV(st));
          if (faar_elect_one()) {
#pragma unroll
            for (int k = 0; k < KT / 16; ++k)
              mma_ts(tmem + F::COL_O, tmem + 64u * (uint32_t)st + 8u * k, db + 128u * k, id_pv, (j | k) != 0 ? 1u : 0u);
            commit(bar_o(st));
          }
          __syncwarp();
        }
        if (!ok) { const unsigned long long t0 = now_ns(); while (now_ns() - t0 < 2000000ull) {} }   // copies in flight
      }
      if (!__syncthreads_or(0) || u0 > 0) break;
    }
  } else {
    const uint32_t t_lane = tmem + ((uint32_t)(32 * warp) << 16), t_o = t_lane + F::COL_O;
    const float slope = (FORM & BIASED) ? 1.4426950408889634f * p.sc.slopes[h] : 0.f;
    __nv_bfloat16* const out = p.out + (seq0 + qi) * p.ldo + h * HD;
    float* const lse = p.lse + ((long long)b * p.H + h) * p.S + qi;
    bool ok = true;
    for (int sweep = 0;; ++sweep) {
      float m = -INFINITY, l = 0.f;                             // the reference the probabilities are relative to; their sum
      bool poison = false;                                      // this row sees a V that is not finite
      int edges = 0;                                            // tiles looked through so far
      for (int j = 0; j < n_kt; ++j) {
        const int k0 = tile_at(j) * KT, u = sweep * n_kt + j, st = u & 1;
        const uint32_t t_s = t_lane + 64u * (uint32_t)st, ph = (uint32_t)((u >> 1) & 1);
        if (sweep && (k0 < span.all_lo || k0 + KT > span.all_hi)) {      // some row does not see some key: no infinity or NaN of its V may reach it
          ok = bar_wait(vfull(st), ph, abort_flag, 0xB15u);
          if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
          // keys of the tile with such a V: three sets of bits in turn; the next edge tile's was read two edge tiles ago, by threads
          // that have all come to the last one's barrier since
          if (threadIdx.x < 2) bad_keys[2 * ((edges + 1) % 3) + threadIdx.x] = 0u;
          uint32_t* const seen = bad_keys + 2 * (edges % 3);
          for (int i = 0; i < KV_BYTES / 2048; ++i) {
            const uint32_t off = 16u * (uint32_t)(threadIdx.x + 128 * i), key = (off % KV_PANEL) / 128u;
            if (not_finite(lds128(sV(st) + off))) atomicOr(seen + (key >> 5), 1u << (key & 31));
          }
          bar_arrive(bar_v);
          ok = bar_wait(bar_v, (uint32_t)(edges & 1), abort_flag, 0xB16u);
          if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
          ++edges;
          const uint32_t low = reinterpret_cast<volatile uint32_t*>(seen)[0], high = reinterpret_cast<volatile uint32_t*>(seen)[1];
          if (low | high) {
            poison |= ((low & range_bits(range, k0)) | (high & range_bits(range, k0 + 32))) != 0u;
            scrub(sV(st), KV_BYTES / 16, threadIdx.x, 128, 0u, 0u);
          }
        }
        // S_j complete, and with it all products issued before, P V_{j-2} among them: of the two barriers for P V the one of tile j - 1
        // has seen all its phases but that one, so a wait for it cannot mistake the parity
        ok = bar_wait(bar_s(st), ph, abort_flag, 0xB10u);
        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
        fence_after();
        // The short way: whoever sees a key of the tile has a reference, and it lies in the past of all of the warp, or in the future
        const bool full = __all_sync(0xffffffffu, range.x <= k0 && range.y >= k0 + KT);
        bool plain = __all_sync(0xffffffffu, m != -INFINITY || range.x >= k0 + KT || range.y <= k0);
        const bool past = k0 + KT - 1 <= q0 + 32 * warp;
        if (FORM & BIASED) plain = plain && (past || k0 >= q0 + 32 * warp + 31);
        const float side = past ? slope : -slope;
        auto mask = [&](float (&s)[32], int half) {
          const uint32_t bits = range_bits(range, k0 + 32 * half);
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (!((bits >> i) & 1u)) s[i] = -INFINITY;
        };
        const float ref = m == -INFINITY ? 0.f : m;
        auto maximum = [&](const float (&s)[32]) {
          float mx[2] = {s[0], s[1]};                             // two chains, two scores per instruction
#pragma unroll
          for (int i = 2; i + 3 < 32; i += 4) { mx[0] = max3(mx[0], s[i], s[i + 1]); mx[1] = max3(mx[1], s[i + 2], s[i + 3]); }
          return fmaxf(max3(mx[0], s[30], s[31]), mx[1]);
        };
        uint32_t pk[KT / 2];
        auto powers = [&](const float (&s)[32], int half) {       // probabilities, packed; their sum
          float2 sum2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
          for (int w = 0; w < 16; ++w) {
            const float2 e = make_float2(ex2(s[2 * w]), ex2(s[2 * w + 1]));
            sum2[w & 1] = __fadd2_rn(sum2[w & 1], e);
            pk[16 * half + w] = pack2(e.x, e.y);
          }
          return (sum2[0].x + sum2[0].y) + (sum2[1].x + sum2[1].y);
        };
        float sum = 0.f;
        if (plain) {
          float s[2][32];
          ld32x2(t_s, t_s + 32u, s[0], s[1]);
          if constexpr ((FORM & CAPPED) != 0) plain = !cap_any_far(s[0], p.sc) && !cap_any_far(s[1], p.sc);
          if (plain) {
            float top = -INFINITY;                              // of the tile's scores, relative to the reference
            auto sweep_tile = [&](auto whole) {
#pragma unroll
              for (int half = 0; half < 2; ++half) {
                score_values<FORM, -1, true>(s[half], p.sc, p.scale_log2, side, qi - k0 - 32 * half, ref);
                if constexpr (!decltype(whole)::value) mask(s[half], half);
                top = fmaxf(top, maximum(s[half]));
                sum += powers(s[half], half);
              }
            };
            if (full) sweep_tile(std::true_type{}); else sweep_tile(std::false_type{});
            plain = !__any_sync(0xffffffffu, top > SCORED_SLACK);
          }
        }
        if (!plain) {
          float s[2][32];
          ld32x2(t_s, t_s + 32u, s[0], s[1]);
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            score_values<FORM, -1, false>(s[half], p.sc, p.scale_log2, slope, qi - k0 - 32 * half, ref);
            if (!full) mask(s[half], half);
          }
          const float top = fmaxf(maximum(s[0]), maximum(s[1]));
          const bool moved = m == -INFINITY ? top > -INFINITY : top > SCORED_SLACK;
          const float by = moved ? top : 0.f;
          const float alpha = m == -INFINITY ? 0.f : ex2(-by);  // of what has been summed (nothing, before the first reference)
          const bool any = __any_sync(0xffffffffu, moved);
          if (any) {
            if (moved) m = ref + by;
            l *= alpha;
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
              for (int i = 0; i < 32; i += 2) {
                const float2 r = __fadd2_rn(make_float2(s[half][i], s[half][i + 1]), pair(-by));
                s[half][i] = r.x; s[half][i + 1] = r.y;
              }
          }
          sum = powers(s[0], 0) + powers(s[1], 1);
          if (any && j > 0) {                                    // O = O * 2^(m_old - m_new), between P V_{j-1} and P V_j
            ok = bar_wait(bar_o(st ^ 1), (uint32_t)(((u - 1) >> 1) & 1), abort_flag, 0xB20u);
            if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
            fence_after();
            const float a = moved ? alpha : 1.0f;
#pragma unroll 1
            for (int c = 0; c < HD; c += 16) {
              float t[16];
              uint32_t u[16];
              ld16(t_o + (uint32_t)c, t);
#pragma unroll
              for (int i = 0; i < 16; ++i) u[i] = __float_as_uint(t[i] * a);
              st16(t_o + (uint32_t)c, u);
            }
            wait_st();
          }
        }
        l += sum;
        st32(t_s, pk);                                          // this row of P_j, an A operand in tensor memory, over S_j
        fence_before();
        bar_arrive(bar_p(st));
      }
      bool broken = false;                                      // something in this row's output is no finite number
      if (n_kt == 0) {                                          // no query of this tile sees a key
        if (qi < p.S) {
          for (int c = 0; c < HD / 8; ++c) reinterpret_cast<uint4*>(out)[c] = make_uint4(0u, 0u, 0u, 0u);
          *lse = -INFINITY;
        }
      } else if (ok) {
        const int u = sweep * n_kt + n_kt - 1;
        ok = bar_wait(bar_o(u & 1), (uint32_t)((u >> 1) & 1), abort_flag, 0xB30u);
        ok = __all_sync(0xffffffffu, ok);
        if (ok) {
          fence_after();
          float inv = l > 0.f ? 1.0f / l : 0.f;
          if (poison) inv = __int_as_float(0x7FFFFFFF);
#pragma unroll
          for (int c0 = 0; c0 < HD; c0 += 64) {
            float t[2][32];
            ld32x2(t_o + (uint32_t)c0, t_o + (uint32_t)(c0 + 32), t[0], t[1]);
            if (qi < p.S) {
#pragma unroll
              for (int c = 0; c < 8; ++c) {
                const float* v = &t[c >> 2][8 * (c & 3)];
                const uint4 w = make_uint4(pack2(v[0] * inv, v[1] * inv), pack2(v[2] * inv, v[3] * inv), pack2(v[4] * inv, v[5] * inv),
                                           pack2(v[6] * inv, v[7] * inv));
                broken |= not_finite(w);
                reinterpret_cast<uint4*>(out + c0)[c] = w;
              }
            }
            __syncwarp();                                       // the next load wants the whole warp (see ld16)
          }
          if (qi < p.S) *lse = m + log2f(l);
        }
      }
      fence_before();                                           // these loads before the second sweep's products
      if (!__syncthreads_or(broken) || sweep) break;
    }
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  if (warp == 4) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)TMEM_COLS) : "memory");
  }
}

// ---- backward, dQ: one CTA per 128 queries of a head, sweeping the key tiles up to the diagonal ---------------
//   S_j = Q K_j^T, dP_j = dO V_j^T     two MMAs into 64 + 64 columns of tensor memory
//   dS_j = P_j (dP_j - delta) / sqrt(d), P_j = 2^(c S_j - lse)     one query row per thread, written as BF16
//                                                                   pairs into 32 columns of tensor memory, the
//                                                                   third product's A operand
//   dQ += dS_j K_j                       third MMA, accumulating in 64 more columns over the whole sweep (K_j read
//                                        as it lies in memory: keys as contraction rows, d contiguous)
// The dQ product of tile j - 1 is issued after the score products of tile j, so it runs while the rows work on
// tile j; K / V tiles come through three TMA stages.  Only the final dQ leaves tensor memory.
// head_dim 128: 160 KB of operands allow one CTA per SM, whose 512 columns then hold two S and two dP buffers, so that the
// score products of tile j + 1 run while the rows work on tile j; dS_j is written over the S columns its threads have
// read, and the buffer pair is free again when dQ += dS_j K_j has run.
// Over key ranges (FORM != CAUSAL) this kernel comes before dK / dV's, and makes good what delta lacks.  delta = dO . O is taken from the
// stored BF16 output; where a query's softmax is peaked, dP - delta nearly cancels, and half a step of O was half of the gradients'
// error (0.0041 of their norm instead of 0.0024).  As P's sum is 1, sum over keys of P (dP - delta') is delta - delta': its sum along the
// row gives the exact delta, which is written back for the dK / dV kernel, and dQ's own correction is that difference times R = sum
// of P K (P times the cap's slope), a fourth product.  R's operand is written over dP, dS over S, as with heads of 128.  It costs the
// fourth product and its operand's stores, dK / dV next to dQ, and with heads of 64 the overlap of a tile's score products with the
// rows of the one before: forward and backward, 4 x 2048 tokens, 32 / 8 heads of 64, documents of 700, capped, 470 -> 501 us; 333 tokens, 4 / 2 heads
// of 128, 24 -> 32.  Backward call, causal ranges, 408 us (the causal kernels 341), heads of 128 358 (332).  By counters, heads of 64, documents
// of 700, capped: dQ / dK, dV issue 51 / 46 % of their cycles, FMA 47 / 34, tensor pipe 24 / 18; the long scoreboard, loads of
// tensor memory among it, holds warps up longest.
template <int HD> struct Dq {
  static constexpr int NP = HD / 64, Q_BYTES = NP * Q_PANEL, KV_BYTES = NP * KV_PANEL, STAGE = 2 * KV_BYTES, STAGES = 3;
  static constexpr int OFF_DO = Q_BYTES, OFF_KV = 2 * Q_BYTES, OFF_CTL = OFF_KV + STAGES * STAGE;
  static constexpr int SMEM = OFF_CTL + CTL + 1024;
  static constexpr bool TWO = HD == 128;                     // two score buffers
  static constexpr int TMEM = TWO ? 512 : 256;
  static constexpr int COL_DP = TWO ? 128 : 64, COL_DQ = TWO ? 256 : 128, COL_R = COL_DQ + HD;
  static constexpr int CTAS = TWO ? 1 : 2;
};
// The backward kernels have no reduction along a row, so two threads share a row (32 of the 64 columns each:
// warps w and w + 4 read the same tensor-memory lanes): eight row warps, the ninth issues copies and MMAs.
constexpr int BWD_THREADS = 288, ROW_THREADS = 256;

struct TcBwdParams {
  const __nv_bfloat16* q; const __nv_bfloat16* k; const __nv_bfloat16* dout;       // as the copies' maps have them: looked at again where something was not finite
  long long ldo;
  const float* lse; const float* dsum;
  __nv_bfloat16* dq; __nv_bfloat16* dk; __nv_bfloat16* dv;
  long long ldq, ldk;
  int B, S, H, Hkv;
  float scale_log2, inv_sqrt_d;
  const float2* rope;              // dq and dk turn back by their row's angles (null: not)
  int parts;                       // dK / dV: CTAs of a cluster that share a key tile's items (1, 2 or 4)
  int sum_parts;                   // delta's parts: of (b, h, query), part j lies at dsum + j sum_part + h sum_head + b sum_batch + query
  long long sum_part, sum_head, sum_batch;
  int apart;                       // dQ: its memory may hold what the dK / dV kernel reads, so it waits for that one
  ScoreArgs sc;
};

// delta of a query, its parts asked for together (8 at most: heads of 128 in units of 16 columns)
__device__ __forceinline__ float delta_of(const TcBwdParams& p, int b, int h, int q) {
  const float* at = p.dsum + (long long)h * p.sum_head + (long long)b * p.sum_batch + q;
  float s = at[0];
  if (p.sum_parts > 1) {
    float v[7];
#pragma unroll
    for (int j = 0; j < 7; ++j) v[j] = j + 1 < p.sum_parts ? at[(j + 1) * p.sum_part] : 0.f;
    s = ((s + v[0]) + (v[1] + v[2])) + ((v[3] + v[4]) + (v[5] + v[6]));      // a binary tree, as within the parts
  }
  return s;
}

// A gradient's row towards a head before the rotary embedding: this thread's HD / 4 pairs (elements i and i + HD / 2, from
// i = HD / 4 * half on), turned back from FP32 accumulators in tensor memory (`t`: the head's first column) by the row's `angles`.
// 4 x 2048 tokens, 32 / 8 heads of 64, us: dK / dV 217 and a pass over dq and dk 17.4 more -> 218.5, dQ 157 -> 160; 2 x 1000, 16 / 8
// heads of 128: 49.5 + 8.3 -> 51.3, 28.2 -> 30.  (Sines and cosines formed here: dQ 174 and 37; a row's angles side by side: 168, 33.)
// The first 16 angles are requested before the last product is waited for.
struct Angles { float2 sc[16]; };
__device__ __forceinline__ void load_angles(const float2* angles, long long tokens, int c, Angles& v) {
#pragma unroll
  for (int j = 0; j < 16; ++j) v.sc[j] = angles[(c + j) * tokens];
}
template <int HD>
__device__ __forceinline__ void turn_back(const float2* angles, long long tokens, Angles& v, uint32_t t, int half, bool valid, __nv_bfloat16* row) {
#pragma unroll
  for (int c = HD / 4 * half; c < HD / 4 * (half + 1); c += 16) {
    float a[16], b[16];
    ld16x2(t + (uint32_t)c, t + (uint32_t)(c + HD / 2), a, b);
#pragma unroll
    for (int j = 0; j < 16; ++j) faar_rope_turn(a[j], b[j], -v.sc[j].x, v.sc[j].y);
    if (valid) {
      if (c + 16 < HD / 4 * (half + 1)) load_angles(angles, tokens, c + 16, v);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        reinterpret_cast<uint4*>(row + c)[h] = make_uint4(pack2(a[8 * h], a[8 * h + 1]), pack2(a[8 * h + 2], a[8 * h + 3]),
                                                          pack2(a[8 * h + 4], a[8 * h + 5]), pack2(a[8 * h + 6], a[8 * h + 7]));
        reinterpret_cast<uint4*>(row + HD / 2 + c)[h] = make_uint4(pack2(b[8 * h], b[8 * h + 1]), pack2(b[8 * h + 2], b[8 * h + 3]),
                                                                   pack2(b[8 * h + 4], b[8 * h + 5]), pack2(b[8 * h + 6], b[8 * h + 7]));
      }
    }
    __syncwarp();                                           // the next load wants the whole warp (see ld16)
  }
}

// Barriers of the row threads; the second says whether one of them has x
__device__ __forceinline__ void row_threads_sync() { asm volatile("barrier.cta.sync 1, %0;" ::"n"(ROW_THREADS) : "memory"); }
__device__ __forceinline__ bool row_threads_any(bool x) {
  uint32_t any;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %1, 0;\n\tbarrier.cta.red.or.pred p, 1, %2, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
               : "=r"(any) : "r"((uint32_t)x), "n"(ROW_THREADS) : "memory");
  return any != 0;
}

// What was taken out of a staged row of K for those who do not see it, those who do get all the same: a row of dS K with such a key is no
// number, whatever dS is (0 times an infinity, too).  Tiles that all of a CTA's queries see get there by themselves; where an edge tile's
// were set to 0 (`found`), this looks at the keys of the CTA's span in those tiles once more, in memory: whether one that the thread's query
// (`range`) sees has one.  All row threads call it; `words`: 8 ints of shared memory.
template <int HD>
__device__ __noinline__ bool sees_bad_key(const __nv_bfloat16* k, long long ldk, Span span, int2 range, uint32_t found,
                                          volatile uint32_t* words) {
  bool sees = false;
  for (int k0 = span.lo / KT * KT; k0 < span.hi; k0 += ROW_THREADS) {
    if (!(__funnelshift_r(found, found, k0 / KT) & ((1u << (ROW_THREADS / KT)) - 1u))) continue;
    const int key = k0 + (int)threadIdx.x;
    const uint32_t bad = __ballot_sync(0xffffffffu, key < span.hi && row_not_finite<HD>(k + key * ldk));
    row_threads_sync();                                     // the words of the keys before have been read
    if ((threadIdx.x & 31) == 0) words[threadIdx.x >> 5] = bad;
    row_threads_sync();
#pragma unroll 1
    for (int w = 0; w < ROW_THREADS / 32; ++w) sees |= (words[w] & range_bits(range, k0 + 32 * w)) != 0u;
  }
  return sees;
}

template <int HD, int FORM>
__global__ void __launch_bounds__(BWD_THREADS, Dq<HD>::CTAS)
attn_dq_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmDO,
                    const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const TcBwdParams p) {
  using C = Dq<HD>;
  constexpr int KV_BYTES = C::KV_BYTES, Q_BYTES = C::Q_BYTES;
  extern __shared__ uint8_t raw[];
  const uint32_t base = (s32(raw) + 1023u) & ~1023u;
  uint8_t* smem = raw + (base - s32(raw));
  const uint32_t ctl = base + C::OFF_CTL;
  const uint32_t bar_qd = ctl, bar_sfree = ctl + 48;
  // TWO: one barrier of each kind per buffer (tiles alternate); otherwise one, passed once per tile
  auto bar_s = [&](int j) { return C::TWO ? ctl + 104u + 8u * (j & 1) : ctl + 40u; };
  auto bar_ds = [&](int j) { return C::TWO ? ctl + 120u + 8u * (j & 1) : ctl + 56u; };
  auto bar_done = [&](int j) { return C::TWO ? ctl + 136u + 8u * (j & 1) : ctl + 64u; };
  auto parity = [&](int j) { return (uint32_t)(C::TWO ? (j >> 1) & 1 : j & 1); };
  auto kvfull = [&](int s) { return ctl + 8u + 8u * s; };
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem + C::OFF_CTL + 96);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::OFF_CTL + 100);
  const uint32_t scrubbed = ctl + 224;                       // over ranges: tiles of K that had something not finite
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  // one-dimensional grid, query tile slowest and descending: CTAs start in order of decreasing work
  const int hb = p.H * p.B;
  const int qt = (int)(gridDim.x / hb) - 1 - (int)(blockIdx.x / hb);
  const int h = (blockIdx.x % hb) % p.H, b = (blockIdx.x % hb) / p.H;
  const int g = h / (p.H / p.Hkv);
  const long long seq0 = (long long)b * p.S;
  const int q0 = qt * QT;
  const int last_q = min(q0 + QT, p.S) - 1;
  int kt0 = 0, n_kt = last_q / KT + 1;

  if (threadIdx.x == 0) {
    bar_init(bar_qd, 1);
    for (int s = 0; s < C::STAGES; ++s) bar_init(kvfull(s), 1);
    for (int s = 0; s < (C::TWO ? 2 : 1); ++s) { bar_init(bar_s(s), 1); bar_init(bar_done(s), 1); bar_init(bar_ds(s), ROW_THREADS); }
    bar_init(bar_sfree, ROW_THREADS);
    *abort_flag = 0;
    asm volatile("st.shared.u32 [%0], 0;" ::"r"(scrubbed) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(s32(const_cast<uint32_t*>(tmem_slot))),
                 "r"((uint32_t)C::TMEM) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  // head_dim 64: S in columns 0..63, dP: 64..127, dQ: 128..191; causal: dS (BF16 pairs) in 192..223; over ranges: dS over S, R's operand
  // over dP, R in 192..255.  head_dim 128: two S in 0..127, two dP in 128..255, dQ 256..383, over ranges R in 384..511; dS over S
  const uint32_t tmem = *tmem_slot;
  if (FORM != CAUSAL || p.apart) faar_pdl_sync();
  else faar_pdl_launch();                                   // needs nothing of the dK / dV kernel, next to which it runs
  int2 range = {0, INT_MAX};                                // this thread's query
  Span span = {};
  if constexpr (FORM != CAUSAL) {
    const int q = q0 + 32 * (warp & 3) + lane;
    const bool is_row = warp < 8 && q < p.S;
    if (is_row) range = key_range(p.sc, b, q, p.S);
    span = tile_span(range, is_row, reinterpret_cast<volatile int*>(smem + C::OFF_CTL + 160));
    kt0 = span.lo / KT;
    n_kt = span.lo < span.hi ? (span.hi - 1) / KT + 1 - kt0 : 0;
  }
  const uint32_t sQ = base, sDO = base + C::OFF_DO;
  auto sK = [&](int s) { return base + C::OFF_KV + (uint32_t)s * C::STAGE; };
  auto sV = [&](int s) { return sK(s) + KV_BYTES; };
  auto col_s = [&](int j) { return C::TWO ? 64u * (uint32_t)(j & 1) : 0u; };
  auto col_dp = [&](int j) { return (uint32_t)C::COL_DP + col_s(j); };
  // dS_j as 64 BF16 pairs' columns: 8 per contraction step; over S each thread half's 16 columns start at its own 32
  constexpr bool OVER = C::TWO || FORM != CAUSAL;
  auto col_ds = [&](int j, int step) { return OVER ? col_s(j) + (uint32_t)(32 * (step >> 1) + 8 * (step & 1)) : 192u + 8u * (uint32_t)step; };

  if (warp == 8) {
    auto wait = [&](uint32_t bar, uint32_t parity, uint32_t code) {
      return __all_sync(0xffffffffu, bar_wait(bar, parity, abort_flag, code)) != 0;
    };
    auto load_kv = [&](int j) {
      const int st = j % C::STAGES;
      if (faar_elect_one()) {
        bar_expect(kvfull(st), 2 * KV_BYTES);
        tma_head<HD>(sK(st), KV_PANEL, &tmK, g * HD, (kt0 + j) * KT, b, kvfull(st));
        tma_head<HD>(sV(st), KV_PANEL, &tmV, g * HD, (kt0 + j) * KT, b, kvfull(st));
      }
      __syncwarp();
    };
    const bool some = FORM == CAUSAL || n_kt > 0;
    if (some) {
      if (faar_elect_one()) {
        bar_expect(bar_qd, 2 * Q_BYTES);
        tma_head<HD>(sQ, Q_PANEL, &tmQ, h * HD, q0, b, bar_qd);
        tma_head<HD>(sDO, Q_PANEL, &tmDO, h * HD, q0, b, bar_qd);
      }
      load_kv(0);
      if (n_kt > 1) load_kv(1);
      if (OVER && n_kt > 2) load_kv(2);
    }
    bool ok = some && wait(bar_qd, 0u, 0xC01u);
    constexpr uint32_t id_k = idesc(KT, 0), id_n = idesc(HD, 1);
    auto issue_s = [&](int j) {                               // S_j, dP_j
      const int st = j % C::STAGES;
      if (faar_elect_one()) {
        mma_rows<HD>(tmem + col_s(j), sQ, Q_PANEL, sK(st), KV_PANEL, id_k);
        mma_rows<HD>(tmem + col_dp(j), sDO, Q_PANEL, sV(st), KV_PANEL, id_k);
        commit(bar_s(j));
      }
      __syncwarp();
    };
    auto issue_dq = [&](int j) {                              // dQ += dS_j K_j
      const uint64_t db = desc_n_major(sK(j % C::STAGES));
      if (faar_elect_one()) {
#pragma unroll
        for (int k = 0; k < KT / 16; ++k)
          mma_ts(tmem + (uint32_t)C::COL_DQ, tmem + col_ds(j, k), db + 128u * k, id_n, (j | k) != 0 ? 1u : 0u);
        if constexpr (FORM != CAUSAL) {                       // R += P K_j
#pragma unroll
          for (int k = 0; k < KT / 16; ++k)
            mma_ts(tmem + (uint32_t)C::COL_R, tmem + (uint32_t)C::COL_DP + col_ds(j, k), db + 128u * k, id_n, (j | k) != 0 ? 1u : 0u);
        }
        commit(bar_done(j));
      }
      __syncwarp();
    };
    if constexpr (C::TWO) {
      if (ok) ok = wait(kvfull(0), 0u, 0xC20u);
      if (ok) { fence_after(); issue_s(0); }
      for (int j = 0; j < n_kt && ok; ++j) {
        if (j >= 1 && j + 1 < n_kt) ok = wait(bar_done(j - 1), parity(j - 1), 0xC10u);   // buffers and stage of tile j - 1 are free
        if (ok && j >= 1 && j + 2 < n_kt) load_kv(j + 2);
        if (ok && j + 1 < n_kt) {
          ok = wait(kvfull((j + 1) % C::STAGES), (uint32_t)(((j + 1) / C::STAGES) & 1), 0xC20u | ((j + 1) % C::STAGES));
          if (!ok) break;
          fence_after();
          issue_s(j + 1);
        }
        if (ok) ok = wait(bar_ds(j), parity(j), 0xC40u);
        if (!ok) break;
        fence_after();
        issue_dq(j);
      }
    } else if constexpr (OVER) {
      if (ok) ok = wait(kvfull(0), 0u, 0xC20u);
      if (ok) { fence_after(); issue_s(0); }
      for (int j = 0; j < n_kt && ok; ++j) {
        ok = wait(bar_ds(j), parity(j), 0xC40u);
        if (!ok) break;
        fence_after();
        issue_dq(j);
        if (j + 1 < n_kt) {                                   // S and dP of the next tile lie over what this product reads
          ok = wait(kvfull((j + 1) % C::STAGES), (uint32_t)(((j + 1) / C::STAGES) & 1), 0xC20u | ((j + 1) % C::STAGES));
          if (ok) ok = wait(bar_done(j), parity(j), 0xC10u);
          if (!ok) break;
          fence_after();
          issue_s(j + 1);
          if (j + 3 < n_kt) load_kv(j + 3);
        }
      }
    } else {
      for (int j = 0; j < n_kt && ok; ++j) {
        const int st = j % C::STAGES;
        if (j >= 1 && j + 1 < n_kt) {                         // stage of tile j + 1 last held tile j - 2
          if (j >= 2) ok = wait(bar_done(j - 2), parity(j - 2), 0xC10u);
          if (!ok) break;
          load_kv(j + 1);
        }
        ok = wait(kvfull(st), (uint32_t)((j / C::STAGES) & 1), 0xC20u | st);
        if (ok && j > 0) ok = wait(bar_sfree, (uint32_t)((j - 1) & 1), 0xC30u);
        if (!ok) break;
        fence_after();
        issue_s(j);
        if (j > 0) {
          ok = wait(bar_ds(j - 1), parity(j - 1), 0xC40u);
          if (!ok) break;
          fence_after();
          issue_dq(j - 1);
        }
      }
      if (ok) ok = wait(bar_ds(n_kt - 1), parity(n_kt - 1), 0xC50u);
      if (ok) { fence_after(); issue_dq(n_kt - 1); }
    }
    if (FORM != CAUSAL) __syncthreads();                      // the row warps' (their sums)
    if (!ok && some) { const unsigned long long t0 = now_ns(); while (now_ns() - t0 < 2000000ull) {} }
  } else {
    const int row = 32 * (warp & 3) + lane, half = warp >> 2;    // this thread: columns 32 half .. 32 half + 31 of its row
    const int qi = q0 + row;
    const uint32_t t_lane = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
    const long long ro = ((long long)b * p.H + h) * p.S;
    const float lse = qi < p.S ? p.lse[ro + qi] : 0.f;
    const float nd = qi < p.S ? -delta_of(p, b, h, qi) * p.inv_sqrt_d : 0.f;
    bool ok = true;
    float2 lack = make_float2(0.f, 0.f);                      // over ranges: this thread's share of the row's sum of P (dP - delta) / sqrt(d)
    const float nb = (FORM & BIASED) ? -1.4426950408889634f * p.sc.slopes[h] : 0.f;
    for (int j = 0; j < n_kt; ++j) {
      const int k0 = (kt0 + j) * KT;
      ok = bar_wait(bar_s(j), parity(j), abort_flag, 0xD10u);
      if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
      fence_after();
      float s[32];
      uint32_t pr_pk[16];                                     // over ranges: R's operand
      auto tile = [&](auto diag_tag) {                        // P (dP - delta) / sqrt(d); the mask only where needed
        constexpr bool DIAG = decltype(diag_tag)::value;
        float t[32], d[32];
        ld32x2(t_lane + col_s(j) + 32u * half, t_lane + col_dp(j) + 32u * half, t, d);
        uint32_t bits = 0;
        if constexpr (FORM != CAUSAL && DIAG) {
          bits = range_bits(range, k0 + 32 * half);
          // an infinity or NaN in a row of K makes its whole column of S no finite number, in every row: where one shows, the tile's
          // half (these 128 threads') is rid of it before the third product, S having been formed
          const float2 f = finite_probe(t, pair(0.f));
          if (__any_sync(0xffffffffu, !(f.x + f.y == 0.f))) {
            const int st = j % C::STAGES;
            ok = bar_wait(kvfull(st), (uint32_t)((j / C::STAGES) & 1), abort_flag, 0xD15u);
#pragma unroll
            for (int c = 0; c < C::NP; ++c) scrub(sK(st) + (uint32_t)(c * KV_PANEL + 4096 * half), 256, 32 * (warp & 3) + lane, 128, scrubbed,
                                                tile_bit(kt0 + j));
          }
        }
        if constexpr ((FORM & CAPPED) != 0) tanh_values(t, p.sc);
        [[maybe_unused]] const float dist = (float)(qi - (k0 + 32 * half));
        const float2 sc2 = make_float2(p.scale_log2, p.scale_log2), nl2 = make_float2(-lse, -lse);
        const float2 is2 = make_float2(p.inv_sqrt_d, p.inv_sqrt_d), nd2 = make_float2(nd, nd);
#pragma unroll
        for (int i = 0; i < 32; i += 2) {                        // two elements per multiply-add
          float2 x = __ffma2_rn(make_float2(t[i], t[i + 1]), (FORM & CAPPED) ? pair(p.sc.cap_out) : sc2, nl2);
          if constexpr ((FORM & BIASED) != 0) x = add_bias<-1>(x, nb, dist - (float)i);
          float2 pr = make_float2(ex2(x.x), ex2(x.y));
          if (DIAG && FORM == CAUSAL) {                          // above the diagonal (and beyond the sequence end)
            if (k0 + 32 * half + i > qi) pr.x = 0.f;
            if (k0 + 32 * half + i + 1 > qi) pr.y = 0.f;
          }
          float2 r = __fmul2_rn(pr, __ffma2_rn(make_float2(d[i], d[i + 1]), is2, nd2));
          if constexpr (FORM != CAUSAL) {
            float2 w = pr, flat = r;
            if constexpr ((FORM & CAPPED) != 0) {
              const float2 slope = __ffma2_rn(make_float2(-t[i], -t[i + 1]), make_float2(t[i], t[i + 1]), pair(1.0f));
              w = __fmul2_rn(w, slope);
              r = __fmul2_rn(r, slope);
            }
            if (DIAG) {                                          // also where what is masked is no number
              if (!((bits >> i) & 1u)) r.x = flat.x = w.x = 0.f;
              if (!((bits >> (i + 1)) & 1u)) r.y = flat.y = w.y = 0.f;
            }
            lack = __fadd2_rn(lack, flat);
            pr_pk[i / 2] = pack2(w.x, w.y);
          }
          s[i] = r.x; s[i + 1] = r.y;
        }
      };
      // some key of the tile above some row; some row does not see some key
      const bool edge = FORM == CAUSAL ? k0 + KT - 1 > q0 : k0 < span.all_lo || k0 + KT > span.all_hi;
      if (edge) tile(std::true_type{}); else tile(std::false_type{});
      if (FORM != CAUSAL && !__all_sync(0xffffffffu, ok)) { ok = false; break; }
      if (!OVER) {
        fence_before();
        bar_arrive(bar_sfree);
        if (j > 0) {                                          // the dS buffer is free once dQ of tile j - 1 has run
          ok = bar_wait(bar_done(j - 1), parity(j - 1), abort_flag, 0xD20u);
          if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
        }
      }
      uint32_t pk[16];
#pragma unroll
      for (int w = 0; w < 16; ++w) pk[w] = pack2(s[2 * w], s[2 * w + 1]);
      st16(t_lane + col_ds(j, 2 * half), pk);                 // this thread's half of the row of dS_j: an A operand
      if constexpr (FORM != CAUSAL) st16(t_lane + (uint32_t)C::COL_DP + col_ds(j, 2 * half), pr_pk);
      wait_st();
      fence_before();
      bar_arrive(bar_ds(j));
    }
    const long long tokens = (long long)p.B * p.S;
    const float2* const angles = p.rope ? p.rope + seq0 + qi : nullptr;
    Angles first;
    if (angles && qi < p.S) load_angles(angles, tokens, HD / 4 * half, first);
    if (FORM != CAUSAL && n_kt == 0) {                        // no query of this tile sees a key
      if (qi < p.S) {
        uint4* dst = reinterpret_cast<uint4*>(p.dq + (seq0 + qi) * p.ldq + h * HD + (HD / 2) * half);
        for (int c = 0; c < HD / 16; ++c) dst[c] = make_uint4(0u, 0u, 0u, 0u);
      }
      ok = false;
    }
    if (ok) {
      ok = bar_wait(bar_done(n_kt - 1), parity(n_kt - 1), abort_flag, 0xD30u);
      ok = __all_sync(0xffffffffu, ok);
    }
    float by = 0.f;                                           // of R
    if constexpr (FORM != CAUSAL) {                           // the two halves' sums, through the operands' memory, which nobody reads any more
      float* const sums = reinterpret_cast<float*>(smem);
      const float mine = lack.x + lack.y;
      if (ok) sums[half * QT + row] = mine;
      __syncthreads();
      if (ok) by = half == 0 ? mine + sums[QT + row] : sums[row] + mine;
      if (ok && half == 0 && qi < p.S) const_cast<float*>(p.dsum)[ro + qi] = (by - nd) / p.inv_sqrt_d;
      const uint32_t found = found_tiles(scrubbed);
      if (found && sees_bad_key<HD>(p.k + seq0 * p.ldk + g * HD, p.ldk, span, range, found, reinterpret_cast<volatile uint32_t*>(sums + 2 * QT)))
        by = __int_as_float(0x7FFFFFFF);
    }
    if (ok) {
      fence_after();
      uint4* dst = reinterpret_cast<uint4*>(p.dq + (seq0 + qi) * p.ldq + h * HD);
      if (angles) turn_back<HD>(angles, tokens, first, t_lane + (uint32_t)C::COL_DQ, half, qi < p.S, reinterpret_cast<__nv_bfloat16*>(dst));
      else
#pragma unroll
      for (int q = 0; q < C::NP; ++q) {                       // this thread's half of the row
        float t[32];
        const int c0 = (HD / 2) * half + 32 * q;
        ld32(t_lane + (uint32_t)(C::COL_DQ + c0), t);
        if constexpr (FORM != CAUSAL) {
          float r[32];
          ld32(t_lane + (uint32_t)(C::COL_R + c0), r);
#pragma unroll
          for (int i = 0; i < 32; ++i) t[i] = fmaf(-by, r[i], t[i]);
        }
        if (qi < p.S) {
#pragma unroll
          for (int c = 0; c < 4; ++c)
            dst[c0 / 8 + c] = make_uint4(pack2(t[8 * c], t[8 * c + 1]), pack2(t[8 * c + 2], t[8 * c + 3]),
                                         pack2(t[8 * c + 4], t[8 * c + 5]), pack2(t[8 * c + 6], t[8 * c + 7]));
        }
        __syncwarp();
      }
    }
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  if (warp == 8) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)C::TMEM) : "memory");
  }
  if (FORM == CAUSAL && threadIdx.x == 0) faar_pdl_join();
}

// ---- backward, dK and dV: one CTA per 128 keys of a key / value head ------------------------------------------
// The keys are the rows (tensor-memory lanes); the CTA sweeps the (head, 64-query tile) pairs that see them:
//   S^T = K Q_i^T, dP^T = V dO_i^T          two MMAs into 64 + 64 columns of tensor memory
//   P^T = 2^(c S^T - lse_q), dS^T = P^T (dP^T - delta_q) / sqrt(d)    one key row per thread; both written as BF16
//                                            pairs over the columns the thread has just read (its half of S^T, of
//                                            dP^T), from where they are the A operands of the accumulating products
//   dV += P^T dO_i, dK += dS^T Q_i           two MMAs that accumulate in 64 + 64 columns over the whole sweep
//                                            (dO_i and Q_i read as they lie in memory: queries as contraction rows)
// 256 columns of tensor memory and under 100 KB of shared memory: two CTAs per SM, which overlap each other's serial
// chain (score products -> rows -> accumulating products -> next item's score products, which overwrite P^T / dS^T
// and so wait for the accumulating products).  Q / dO tiles come through four TMA stages (requested three items
// ahead), lse and delta of a tile's 64 queries are staged in shared memory by the row threads themselves.  Queries
// beyond the sequence end are masked.
// head_dim 128: dV and dK take 256 columns and the operands 162 KB, so one CTA per SM with all 512 columns: two S^T and two
// dP^T buffers, the score products of item i + 1 run while the rows work on item i; three stages.
template <int HD> struct Dkv {
  static constexpr int NP = HD / 64, KEY_BYTES = NP * Q_PANEL, QD_BYTES = NP * KV_PANEL, STAGE = 2 * QD_BYTES;
  static constexpr bool TWO = HD == 128;
  static constexpr int STAGES = TWO ? 3 : 4;
  static constexpr int OFF_V = KEY_BYTES, OFF_QD = 2 * KEY_BYTES, OFF_ROWV = OFF_QD + STAGES * STAGE, OFF_CTL = OFF_ROWV + 2 * 2 * KT * 4;
  static constexpr int OFF_RANGE = OFF_CTL + CTL;            // [2][KT] ranges of an item's queries, where scores go by them
  static constexpr int SMEM = OFF_RANGE + 2 * KT * 8 + 1024;
  static constexpr int CTAS = TWO ? 1 : 2;
  // head_dim 64: S^T in columns 0..63, dP^T: 64..127, dV: 128..191, dK: 192..255.  The thread of row half h reads columns
  // 32 h .. 32 h + 31 of S^T (dP^T) and writes its 32 values of P^T (dS^T) as 16 BF16 pairs to columns 32 h .. 32 h + 15
  // of the same buffer.
  static constexpr int TMEM = TWO ? 512 : 256;
  static constexpr int COL_DP = TWO ? 128 : 64, COL_DV = TWO ? 256 : 128, COL_DK = COL_DV + HD;
  static_assert(CTAS * (SMEM + 1024) <= 228 * 1024, "shared memory budget");
};

// Few key tiles leave SMs idle while one CTA sweeps every query tile of every head of its group, so the items of a key tile are
// then dealt over the CTAs of a cluster.  Each ends with partial dV and dK; of their 2 HD columns each CTA finishes a part:
// the others' values for it come through distributed shared memory, over the operands, which all have been read by then.
// A part is 16-column chunks from the lower half of dV's (or dK's) columns and their partners HD / 2 further on, which the
// rotary embedding pairs.  Values lie in 16-byte units, [sender][chunk][4 columns][row].
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
template <int HD>
__device__ __noinline__ void finish_parts(uint32_t base, uint32_t t_acc, int row, int half, int parts, int rank, bool has, bool valid,
                                          __nv_bfloat16* dk, __nv_bfloat16* dv, const float2* angles, long long tokens) {
  const int per = parts / 2, pairs = HD / 32 / per;             // CTAs for each of dV and dK; pairs of chunks a CTA finishes
  auto column = [&](int owner, int pair, int partner) {         // of the accumulators, dV's columns first
    return (owner >= per ? HD : 0) + 16 * ((owner % per) * pairs + pair) + partner * (HD / 2);
  };
  auto unit = [&](int sender, int pair, int partner, int u) {
    return base + (uint32_t)(((((sender * pairs + pair) * 2 + partner) * 4 + u) * QT + row) << 4);
  };
  cluster_sync();                                               // nobody's operands are read any more
  for (int d = 1; d < parts; ++d) {
    const int owner = (rank + d) % parts, slot = rank < owner ? rank : rank - 1;
    for (int pair = half; pair < pairs * 2; pair += 2) {        // (pair, partner) one after the other
      float v[16];
      ld16(t_acc + (uint32_t)column(owner, pair >> 1, pair & 1), v);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        uint32_t dst;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(dst) : "r"(unit(slot, pair >> 1, pair & 1, u)), "r"(owner));
        asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "f"(has ? v[4 * u] : 0.f), "f"(has ? v[4 * u + 1] : 0.f),
                     "f"(has ? v[4 * u + 2] : 0.f), "f"(has ? v[4 * u + 3] : 0.f) : "memory");
      }
    }
  }
  cluster_sync();
  const bool is_k = rank >= per;
  __nv_bfloat16* const out = is_k ? dk : dv;
  for (int pair = half; pair < pairs; pair += 2) {
    float v[2][16];
#pragma unroll
    for (int partner = 0; partner < 2; ++partner) {
      ld16(t_acc + (uint32_t)column(rank, pair, partner), v[partner]);
#pragma unroll
      for (int j = 0; j < 16; ++j) v[partner][j] = has ? v[partner][j] : 0.f;
      for (int sender = 0; sender < parts - 1; ++sender) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          float4 x;
          asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(unit(sender, pair, partner, u)) : "memory");
          v[partner][4 * u] += x.x; v[partner][4 * u + 1] += x.y; v[partner][4 * u + 2] += x.z; v[partner][4 * u + 3] += x.w;
        }
      }
    }
    const int c = column(rank, pair, 0) - (is_k ? HD : 0);
    if (valid) {
      if (is_k && angles) {
        Angles a;
        load_angles(angles, tokens, c, a);
#pragma unroll
        for (int j = 0; j < 16; ++j) faar_rope_turn(v[0][j], v[1][j], -a.sc[j].x, a.sc[j].y);
      }
#pragma unroll
      for (int partner = 0; partner < 2; ++partner) {
        uint4* dst = reinterpret_cast<uint4*>(out + c + partner * (HD / 2));
#pragma unroll
        for (int q = 0; q < 2; ++q)
          dst[q] = make_uint4(pack2(v[partner][8 * q], v[partner][8 * q + 1]), pack2(v[partner][8 * q + 2], v[partner][8 * q + 3]),
                              pack2(v[partner][8 * q + 4], v[partner][8 * q + 5]), pack2(v[partner][8 * q + 6], v[partner][8 * q + 7]));
      }
    }
    __syncwarp();                                           // the next load wants the whole warp (see ld16)
  }
}

// HD / 2 columns of accumulators of this thread's lane, from `t` on: no numbers where `bad` (the whole warp calls it)
template <int HD>
__device__ __forceinline__ void spoil(uint32_t t, bool bad) {
#pragma unroll 1
  for (int c = 0; c < HD / 2; c += 16) {
    float v[16];
    uint32_t u[16];
    ld16(t + (uint32_t)c, v);
#pragma unroll
    for (int i = 0; i < 16; ++i) u[i] = bad ? 0x7FFFFFFFu : __float_as_uint(v[i]);
    st16(t + (uint32_t)c, u);
  }
  wait_st();
}
// As sees_bad_key: what was taken out of staged rows of Q or dO for the keys that they do not see makes dK or dV of those that they do
// no number.  Goes through the queries that see a key of this CTA's, in the tiles where that was, once more, in memory, and spoils the
// accumulators of the keys that one with such a row sees.  All row threads call it, the products being through.  It finds anew what it
// works on: with arguments whole and dealt key tiles of heads of 64 kept their registers for them (4 x 2048 tokens, capped, backward call
// 597 -> 615 us).  Sequences that end in 100 tokens of padding, finite -> NaN, backward call, us: 4 x 2048 tokens, heads of 64 409 -> 442, of 128
// 350 -> 394, 1 x 8192 capped 1965 -> 2154 (all tiles looked through: 1283, 1212, 8721).
template <int HD, bool DEALT>
__device__ __noinline__ void spoil_seen(const TcBwdParams& p) {
  extern __shared__ uint8_t raw[];
  uint8_t* const smem = raw + (((s32(raw) + 1023u) & ~1023u) - s32(raw));
  int4* const list = reinterpret_cast<int4*>(smem);         // over the operands, which have been read
  const uint32_t t_lane = *reinterpret_cast<volatile uint32_t*>(smem + Dkv<HD>::OFF_CTL + 128) + ((threadIdx.x & 96) << 16);
  const int groups = p.Hkv * p.B, rep = p.H / p.Hkv, tile = (int)(blockIdx.x / (unsigned)(DEALT ? p.parts : 1));
  const int g = (tile % groups) % p.Hkv, b = (tile % groups) / p.Hkv, row = (int)threadIdx.x & (QT - 1), half = (int)threadIdx.x >> 7;
  const int k0 = tile / groups * QT, kj = k0 + row;
  const uint32_t found = found_tiles(s32(smem) + Dkv<HD>::OFF_CTL + 136);
  int seen = 0;                                             // by a query whose q (1), whose dO (2) is not finite
  for (int q0 = 0; q0 < p.S; q0 += ROW_THREADS) {
    if (!(__funnelshift_r(found, found, q0 / KT) & ((1u << (ROW_THREADS / KT)) - 1u))) continue;
    const int q = q0 + (int)threadIdx.x;
    const int2 r = q < p.S ? key_range(p.sc, b, q, p.S) : make_int2(EMPTY_LO, EMPTY_HI);
    const bool near = r.x < k0 + QT && r.y > k0;            // sees a key of the tile
    const long long at = (long long)b * p.S + q;
    for (int h = g * rep; h < (g + 1) * rep; ++h) {
      int4 mine = make_int4(r.x, r.y - r.x, 0, 0);          // first key, how many, which of the two is not finite
      if (near) mine.z = row_not_finite<HD>(p.q + at * p.ldq + h * HD) + 2 * row_not_finite<HD>(p.dout + at * p.ldo + h * HD);
      if (!row_threads_any(mine.z != 0)) continue;          // (the list before has been read)
      list[threadIdx.x] = mine;
      row_threads_sync();
#pragma unroll 1
      for (int i = 0; i < ROW_THREADS; ++i) {
        const int4 v = list[i];
        if (v.z && (uint32_t)(kj - v.x) < (uint32_t)v.y) seen |= v.z;
      }
    }
  }
  fence_after();
  const uint32_t t_half = t_lane + (uint32_t)(HD / 2 * half);
  if (__any_sync(0xffffffffu, seen & 1)) spoil<HD>(t_half + (uint32_t)Dkv<HD>::COL_DK, seen & 1);
  if (__any_sync(0xffffffffu, seen & 2)) spoil<HD>(t_half + (uint32_t)Dkv<HD>::COL_DV, seen & 2);
  fence_before();
  row_threads_sync();                                       // a row's two threads may read one another's columns (finish_parts)
}

// DEALT: p.parts CTAs share a key tile (compiled in: as a choice at run time it cost whole key tiles 1 %)
template <int HD, bool DEALT, int FORM>
__global__ void __launch_bounds__(BWD_THREADS, Dkv<HD>::CTAS)
attn_dkv_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmDO,
                     const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ TcBwdParams p) {
  using C = Dkv<HD>;
  extern __shared__ uint8_t raw[];
  const uint32_t base = (s32(raw) + 1023u) & ~1023u;
  uint8_t* smem = raw + (base - s32(raw));
  const uint32_t ctl = base + C::OFF_CTL;
  const uint32_t bar_kv = ctl;
  auto qfull = [&](int s) { return ctl + 8u + 8u * s; };          // 4
  auto bar_s = [&](int s) { return ctl + 40u + 8u * s; };         // 2 (items alternate): the score products of an item are complete
  auto bar_pds = [&](int s) { return ctl + 72u + 8u * s; };       // 2: P^T / dS^T of an item written by all rows
  auto bar_done = [&](int s) { return ctl + 88u + 8u * s; };      // 2: the accumulating MMAs of an item have run
  auto bar_rv = [&](int s) { return ctl + 112u + 8u * s; };       // 2: lse / delta of an item staged, previous use read by all
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem + C::OFF_CTL + 128);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::OFF_CTL + 132);
  const uint32_t scrubbed = ctl + 136;                   // over ranges: tiles of Q or dO that had something not finite
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  // one-dimensional grid, key tile slowest: CTAs start in order of decreasing work (the first key tiles see the
  // most queries), so the short ones fill the end of the launch
  const int groups = p.Hkv * p.B;
  const int parts = DEALT ? p.parts : 1, rank = (int)(blockIdx.x % (unsigned)parts), tile = (int)(blockIdx.x / (unsigned)parts);
  const int kt = tile / groups, g = (tile % groups) % p.Hkv, b = (tile % groups) / p.Hkv;
  const int rep = p.H / p.Hkv;
  const long long seq0 = (long long)b * p.S;
  const int k0 = kt * QT;
  const int n_qt = (p.S + KT - 1) / KT;
  int qt0 = k0 / KT;                                               // first query tile that sees a key of this tile
  int per_head = n_qt - qt0;
  auto items = [&] { const int n_all = rep * per_head; return n_all > rank ? (n_all - rank + parts - 1) / parts : 0; };
  int n_it = items();                                              // this CTA's: rank, rank + parts, ...

  if (threadIdx.x == 0) {
    bar_init(bar_kv, 1);
    for (int s = 0; s < C::STAGES; ++s) bar_init(qfull(s), 1);
    for (int s = 0; s < 2; ++s) {
      bar_init(bar_s(s), 1); bar_init(bar_done(s), 1); bar_init(bar_pds(s), ROW_THREADS); bar_init(bar_rv(s), ROW_THREADS);
    }
    *abort_flag = 0;
    asm volatile("st.shared.u32 [%0], 0;" ::"r"(scrubbed) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(s32(const_cast<uint32_t*>(tmem_slot))),
                 "r"((uint32_t)C::TMEM) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = *tmem_slot;
  faar_pdl_wait_first();                                    // set-up done; now wait for the previous kernel's data, then let dQ's start
  const int4* const tiles = FORM != CAUSAL ? p.sc.tiles + (long long)b * n_qt : nullptr;
  if constexpr (FORM != CAUSAL) {                           // from the first query tile to the last one that sees a key of this tile
    int first = INT_MAX, last = -1;
    for (int t = lane; t < n_qt; t += 32) {
      const int4 v = tiles[t];
      if (v.x < k0 + QT && v.y > k0 && v.x < v.y) { first = min(first, t); last = t; }
    }
    qt0 = __reduce_min_sync(0xffffffffu, first);
    per_head = __reduce_max_sync(0xffffffffu, last) - qt0 + 1;
    if (per_head <= 0) qt0 = per_head = 0;
    n_it = items();
  }
  const uint32_t sKt = base, sVt = base + C::OFF_V;
  auto sQ = [&](int s) { return base + C::OFF_QD + (uint32_t)s * C::STAGE; };
  auto sDO = [&](int s) { return sQ(s) + C::QD_BYTES; };
  auto col_s = [&](int i) { return C::TWO ? 64u * (uint32_t)(i & 1) : 0u; };
  auto col_dp = [&](int i) { return (uint32_t)C::COL_DP + col_s(i); };
  // Item after item without divisions: head of the group, query tile from qt0 on
  struct Item { int h, t; };
  auto advance = [&](Item& x) {
    x.t += parts;
    while (x.t >= per_head) { x.t -= per_head; ++x.h; }
  };
  auto first_item = [&] {
    Item x = {0, rank - parts};
    if (FORM != CAUSAL && n_it > 0) advance(x);
    return x;
  };
  auto head_of = [&](int i) { return g * rep + (i * parts + rank) / per_head; };
  auto q0_of = [&](int i) { return (qt0 + (i * parts + rank) % per_head) * KT; };

  if (warp == 8) {
    auto wait = [&](uint32_t bar, uint32_t parity, uint32_t code) {
      return __all_sync(0xffffffffu, bar_wait(bar, parity, abort_flag, code)) != 0;
    };
    Item to_load = first_item();                               // items are loaded in their order
    auto load_item = [&](int i) {
      const int st = i % C::STAGES;
      const int hd = FORM == CAUSAL ? head_of(i) : g * rep + to_load.h, q0 = FORM == CAUSAL ? q0_of(i) : (qt0 + to_load.t) * KT;
      if (faar_elect_one()) {
        bar_expect(qfull(st), 2 * C::QD_BYTES);
        tma_head<HD>(sQ(st), KV_PANEL, &tmQ, hd * HD, q0, b, qfull(st));
        tma_head<HD>(sDO(st), KV_PANEL, &tmDO, hd * HD, q0, b, qfull(st));
      }
      __syncwarp();
      if (FORM != CAUSAL) advance(to_load);
    };
    if (n_it > 0 && faar_elect_one()) {
      bar_expect(bar_kv, 2 * C::KEY_BYTES);
      tma_head<HD>(sKt, Q_PANEL, &tmK, g * HD, k0, b, bar_kv);
      tma_head<HD>(sVt, Q_PANEL, &tmV, g * HD, k0, b, bar_kv);
    }
    if (n_it > 0) load_item(0);
    if (n_it > 1) load_item(1);
    if (n_it > 2) load_item(2);
    bool ok = n_it > 0 && wait(bar_kv, 0u, 0xE01u);
    constexpr uint32_t id_k = idesc(KT, 0), id_n = idesc(HD, 1);
    auto issue_s = [&](int i) {                                // S^T and dP^T of item i
      const int st = i % C::STAGES;
      if (faar_elect_one()) {
        mma_rows<HD>(tmem + col_s(i), sKt, Q_PANEL, sQ(st), KV_PANEL, id_k);
        mma_rows<HD>(tmem + col_dp(i), sVt, Q_PANEL, sDO(st), KV_PANEL, id_k);
        commit(bar_s(i & 1));
      }
      __syncwarp();
    };
    // dV += P^T dO_i, dK += dS^T Q_i.  A operands from tensor memory: contraction steps 0, 1 (queries 0..31) in columns
    // 0..15 of the buffer, steps 2, 3 (queries 32..63) in columns 32..47
    auto accumulate = [&](int i) {
      const int st = i % C::STAGES;
      const uint64_t dd = desc_n_major(sDO(st)), dq_ = desc_n_major(sQ(st));
      if (faar_elect_one()) {
#pragma unroll
        for (int k = 0; k < KT / 16; ++k)
          mma_ts(tmem + (uint32_t)C::COL_DV, tmem + col_s(i) + (uint32_t)(32 * (k >> 1) + 8 * (k & 1)), dd + 128u * k, id_n, (i | k) != 0 ? 1u : 0u);
#pragma unroll
        for (int k = 0; k < KT / 16; ++k)
          mma_ts(tmem + (uint32_t)C::COL_DK, tmem + col_dp(i) + (uint32_t)(32 * (k >> 1) + 8 * (k & 1)), dq_ + 128u * k, id_n, (i | k) != 0 ? 1u : 0u);
        commit(bar_done(i & 1));
      }
      __syncwarp();
    };
    if (ok) ok = wait(qfull(0), 0u, 0xE10u);
    if (ok) { fence_after(); issue_s(0); }
    for (int i = 0; i < n_it && ok; ++i) {
      if constexpr (C::TWO) {
        if (i >= 1 && i + 1 < n_it) ok = wait(bar_done((i - 1) & 1), (uint32_t)(((i - 1) >> 1) & 1), 0xE40u);   // buffers, stage of item i - 1
        if (ok && i >= 1 && i + 2 < n_it) load_item(i + 2);
        if (ok && i + 1 < n_it) {
          ok = wait(qfull((i + 1) % C::STAGES), (uint32_t)(((i + 1) / C::STAGES) & 1), 0xE10u);
          if (!ok) break;
          fence_after();
          issue_s(i + 1);
        }
        if (ok) ok = wait(bar_pds(i & 1), (uint32_t)((i >> 1) & 1), 0xE30u);
        if (!ok) break;
        fence_after();
        accumulate(i);
      } else {
        if (i + 3 < n_it) {                                    // its stage last held item i - 1: wait for that item's
          if (i >= 1) ok = wait(bar_done((i - 1) & 1), (uint32_t)(((i - 1) >> 1) & 1), 0xE40u);   // MMAs
          if (!ok) break;
          load_item(i + 3);
        }
        ok = wait(bar_pds(i & 1), (uint32_t)((i >> 1) & 1), 0xE30u);
        if (!ok) break;
        fence_after();
        accumulate(i);
        if (i + 1 < n_it) {
          // the next item's score products overwrite P^T / dS^T: after the accumulating products have read them
          ok = wait(qfull((i + 1) % C::STAGES), (uint32_t)(((i + 1) / C::STAGES) & 1), 0xE10u);
          if (ok) ok = wait(bar_done(i & 1), (uint32_t)((i >> 1) & 1), 0xE20u);
          if (!ok) break;
          fence_after();
          issue_s(i + 1);
        }
      }
    }
    if (!ok && n_it > 0) { const unsigned long long t0 = now_ns(); while (now_ns() - t0 < 2000000ull) {} }
    __syncwarp();
    if (DEALT) { cluster_sync(); cluster_sync(); }      // the row warps' (finish_parts)
  } else {
    const int row = 32 * (warp & 3) + lane, half = warp >> 2;    // this thread: queries 32 half .. 32 half + 31 of an item
    const int kj = k0 + row;
    const uint32_t t_lane = tmem + ((uint32_t)(32 * (warp & 3)) << 16);
    float* rowv_all = reinterpret_cast<float*>(smem + C::OFF_ROWV);      // [2][2][KT]: lse, delta / sqrt(d) negated
    bool ok = true;
    // this thread's share of an item's 64 lse values (rows 0..63) or 64 negated, scaled delta values (rows 64..127);
    // the value for item i + 1 is requested at the start of item i, so its latency is off the per-item path
    auto row_value = [&](int i) {
      const long long ro = ((long long)b * p.H + head_of(i)) * p.S;
      const int q = q0_of(i) + (row & (KT - 1));
      if (q >= p.S) return 0.f;
      return row < KT ? p.lse[ro + q] : -delta_of(p, b, head_of(i), q) * p.inv_sqrt_d;
    };
    float rv_next = 0.f;
    if (FORM == CAUSAL && half == 0 && n_it > 0) rv_next = row_value(0);
    // Over ranges: an item's values likewise, and by the other half's threads its queries' ranges (first key; how many) and what they
    // see together.  All is kept as it was read until it is staged: a value that is worked on at once is waited for at once, which
    // took 800 to 2000 clocks an item.
    int2* range_all = reinterpret_cast<int2*>(smem + C::OFF_RANGE);
    Item ahead = first_item();
    float raw_next = 0.f;
    int2 range_next = {};
    int4 tile_next = {};
    auto request = [&] {                                         // what item `ahead` needs, then on to the next one
      const int q = min((qt0 + ahead.t) * KT + (row & (KT - 1)), p.S - 1), hd = g * rep + ahead.h;
      if (half == 0) {
        const long long at = ((long long)b * p.H + hd) * p.S + q;
        raw_next = row < KT ? p.lse[at] : p.dsum[at];
      } else if (row < KT) {
        const long long at = (long long)b * p.S + q;
        range_next.x = p.sc.key_lo ? p.sc.key_lo[at] : 0;
        range_next.y = p.sc.key_hi ? p.sc.key_hi[at] : q + 1;
      }
      tile_next = tiles[qt0 + ahead.t];
      advance(ahead);
    };
    if (FORM != CAUSAL && n_it > 0) request();
    Item now = first_item();
    for (int i = 0; i < n_it; ++i) {
      const int q0 = FORM == CAUSAL ? q0_of(i) : (qt0 + now.t) * KT;
      float* rowv = rowv_all + (i & 1) * 2 * KT;
      int2* rowr = range_all + (i & 1) * KT;
      const int4 tile_now = tile_next;
      const float nb = (FORM & BIASED) ? -1.4426950408889634f * p.sc.slopes[g * rep + now.h] : 0.f;
      if constexpr (FORM == CAUSAL) {
        if (half == 0) {                                         // the first four warps stage the 128 values
          rowv[row] = rv_next;
          if (i + 1 < n_it) rv_next = row_value(i + 1);
        }
      } else {
        const bool in = q0 + (row & (KT - 1)) < p.S;
        if (half == 0) {
          rowv[row] = !in ? 0.f : row < KT ? raw_next : -raw_next * p.inv_sqrt_d;
        } else if (row < KT) {
          const int lo = max(range_next.x, 0), hi = min(range_next.y, p.S);
          rowr[row] = in && lo < hi ? make_int2(lo, hi - lo) : make_int2(EMPTY_LO, 0);
        }
        if (i + 1 < n_it) request();
        advance(now);
      }
      // every row thread arrives: the buffer of item i + 2 is then written only after all have read item i's
      bar_arrive(bar_rv(i & 1));
      ok = bar_wait(bar_rv(i & 1), (uint32_t)((i >> 1) & 1), abort_flag, 0xF05u);
      if (ok) ok = bar_wait(bar_s(i & 1), (uint32_t)((i >> 1) & 1), abort_flag, 0xF10u);
      if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
      fence_after();
      // the item crosses the diagonal or the sequence end; some query does not see some key
      const bool edge = FORM == CAUSAL ? q0 < k0 + QT || q0 + KT > p.S : tile_now.z > k0 || tile_now.w < k0 + QT || q0 + KT > p.S;
      // the mask costs three instructions per element: only items that need it take that path
      auto item = [&](auto edge_tag) {
        constexpr bool EDGE = decltype(edge_tag)::value;
        float t[32], d[32];
        ld32x2(t_lane + col_s(i) + 32u * half, t_lane + col_dp(i) + 32u * half, t, d);
        if constexpr (FORM != CAUSAL && EDGE) {
          // a row of Q or dO that is not finite shows in its whole column of S^T or dP^T; see the dQ kernel
          const float2 f = finite_probe(d, finite_probe(t, pair(0.f)));
          if (__any_sync(0xffffffffu, !(f.x + f.y == 0.f))) {
            const int st = i % C::STAGES;
            ok = bar_wait(qfull(st), (uint32_t)((i / C::STAGES) & 1), abort_flag, 0xF15u);
#pragma unroll
            for (int c = 0; c < C::NP; ++c) {
              scrub(sQ(st) + (uint32_t)(c * KV_PANEL + 4096 * half), 256, row, 128, scrubbed, tile_bit(q0 / KT));
              scrub(sDO(st) + (uint32_t)(c * KV_PANEL + 4096 * half), 256, row, 128, scrubbed, tile_bit(q0 / KT));
            }
          }
        }
        if constexpr ((FORM & CAPPED) != 0) tanh_values(t, p.sc);
        [[maybe_unused]] const float dist = (float)(q0 + 32 * half - kj);
#pragma unroll
        for (int j4 = 0; j4 < 32; j4 += 4) {
          const float4 l4 = *reinterpret_cast<const float4*>(rowv + 32 * half + j4);          // the same address in every lane
          const float4 n4 = *reinterpret_cast<const float4*>(rowv + KT + 32 * half + j4);
          const float lq[4] = {l4.x, l4.y, l4.z, l4.w}, nq[4] = {n4.x, n4.y, n4.z, n4.w};
#pragma unroll
          for (int e = 0; e < 4; e += 2) {                       // two elements per multiply-add
            const int j = j4 + e, c = 32 * half + j;
            const float2 nl2 = make_float2(-lq[e], -lq[e + 1]);
            float2 x = __ffma2_rn(make_float2(t[j], t[j + 1]), (FORM & CAPPED) ? pair(p.sc.cap_out) : make_float2(p.scale_log2, p.scale_log2), nl2);
            if constexpr ((FORM & BIASED) != 0) x = add_bias<1>(x, nb, dist + (float)j);
            float2 pr = make_float2(ex2(x.x), ex2(x.y));
            if (EDGE && FORM == CAUSAL) {
              if (!(kj <= q0 + c && q0 + c < p.S)) pr.x = 0.f;
              if (!(kj <= q0 + c + 1 && q0 + c + 1 < p.S)) pr.y = 0.f;
            }
            float2 r = __fmul2_rn(pr, __ffma2_rn(make_float2(d[j], d[j + 1]), make_float2(p.inv_sqrt_d, p.inv_sqrt_d),
                                                 make_float2(nq[e], nq[e + 1])));
            if constexpr ((FORM & CAPPED) != 0) r = __fmul2_rn(r, __ffma2_rn(make_float2(-t[j], -t[j + 1]), make_float2(t[j], t[j + 1]), pair(1.0f)));
            if constexpr (EDGE && FORM != CAUSAL) {              // also where what is masked is no number
              const int4 rg = *reinterpret_cast<const int4*>(rowr + c);
              if (!((uint32_t)(kj - rg.x) < (uint32_t)rg.y)) pr.x = r.x = 0.f;
              if (!((uint32_t)(kj - rg.z) < (uint32_t)rg.w)) pr.y = r.y = 0.f;
            }
            t[j] = pr.x; t[j + 1] = pr.y;
            d[j] = r.x; d[j + 1] = r.y;
          }
        }
        // this thread's half of the rows of P^T and dS^T: A operands in tensor memory
        uint32_t pk[16];
#pragma unroll
        for (int w = 0; w < 16; ++w) pk[w] = pack2(t[2 * w], t[2 * w + 1]);
        st16(t_lane + col_s(i) + 32u * half, pk);                // over the first half of the columns just read
#pragma unroll
        for (int w = 0; w < 16; ++w) pk[w] = pack2(d[2 * w], d[2 * w + 1]);
        st16(t_lane + col_dp(i) + 32u * half, pk);
      };
      if (edge) item(std::true_type{}); else item(std::false_type{});
      if (FORM != CAUSAL && !__all_sync(0xffffffffu, ok)) { ok = false; break; }
      wait_st();
      fence_before();
      bar_arrive(bar_pds(i & 1));
    }
    const long long tokens = (long long)p.B * p.S;
    const float2* const angles = p.rope ? p.rope + seq0 + kj : nullptr;
    Angles first;
    if (angles && kj < p.S && !DEALT) load_angles(angles, tokens, HD / 4 * half, first);
    if (ok && n_it > 0) {
      ok = bar_wait(bar_done((n_it - 1) & 1), (uint32_t)(((n_it - 1) >> 1) & 1), abort_flag, 0xF30u);
      ok = __all_sync(0xffffffffu, ok);
    }
    if constexpr (FORM != CAUSAL) {
      row_threads_sync();                                     // all have come to the end: the flag is final, the operands have been read
      if (found_tiles(scrubbed)) spoil_seen<HD, DEALT>(p);
    }
    if constexpr (DEALT) {
      fence_after();
      const long long at = (seq0 + kj) * p.ldk + g * HD;
      finish_parts<HD>(base, t_lane + (uint32_t)C::COL_DV, row, half, parts, rank, n_it > 0, kj < p.S, p.dk + at, p.dv + at, angles, tokens);
    } else if (FORM != CAUSAL && n_it == 0) {                // no query sees a key of this tile
      if (kj < p.S)
        for (int c = 0; c < HD / 16; ++c) {
          const long long at = (seq0 + kj) * p.ldk + g * HD + (HD / 2) * half + 8 * c;
          *reinterpret_cast<uint4*>(p.dk + at) = *reinterpret_cast<uint4*>(p.dv + at) = make_uint4(0u, 0u, 0u, 0u);
        }
    } else if (ok) {
      fence_after();
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        uint4* dst = reinterpret_cast<uint4*>((which ? p.dk : p.dv) + (seq0 + kj) * p.ldk + g * HD);
        if (which && angles) {
          turn_back<HD>(angles, tokens, first, t_lane + (uint32_t)C::COL_DK, half, kj < p.S, reinterpret_cast<__nv_bfloat16*>(dst));
          break;
        }
#pragma unroll
        for (int q = 0; q < C::NP; ++q) {                      // this thread's half of the row
          float t[32];
          const int c0 = (HD / 2) * half + 32 * q;
          ld32(t_lane + (uint32_t)(C::COL_DV + HD * which + c0), t);
          if (kj < p.S) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
              dst[c0 / 8 + c] = make_uint4(pack2(t[8 * c], t[8 * c + 1]), pack2(t[8 * c + 2], t[8 * c + 3]),
                                           pack2(t[8 * c + 4], t[8 * c + 5]), pack2(t[8 * c + 6], t[8 * c + 7]));
          }
          __syncwarp();
        }
      }
    }
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  if (warp == 8) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)C::TMEM) : "memory");
  }
}

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                             const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                             CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// B sequences of [S, cols] BF16, row stride ld elements: boxes of 64 columns x box_rows rows of one sequence, 128-byte swizzle
int head_map(faar_ctx* ctx, CUtensorMap* map, const void* ptr, int B, int S, int cols, long long ld, int box_rows) {
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)S, (cuuint64_t)B};
  cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)S * (cuuint64_t)ld * 2};
  cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1};
  cuuint32_t es[3] = {1, 1, 1};
  CUresult r = reinterpret_cast<EncodeFn>(ctx->encode_tiled)(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(ptr), dims,
                                                             strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                                             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                                             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? 0 : (int)cudaErrorInvalidValue;
}

template <int HD>
int launch_fwd(faar_ctx* ctx, const TcParams& p, const void* q, int64_t ldq, const void* k, const void* v, int64_t ldk) {
  using F = Fwd<HD>;
  static_assert(2 * (F::SMEM + 1024) <= 228 * 1024, "two CTAs per SM");
  CUtensorMap tmQ, tmK, tmV;
  int e = head_map(ctx, &tmQ, q, p.B, p.S, p.H * HD, ldq, QT);
  if (!e) e = head_map(ctx, &tmK, k, p.B, p.S, p.Hkv * HD, ldk, KT);
  if (!e) e = head_map(ctx, &tmV, v, p.B, p.S, p.Hkv * HD, ldk, KT);
  if (!e) e = faar_allow_smem(ctx, (const void*)attn_fwd_tc_kernel<HD>, F::SMEM);
  if (e) return e;
  faar_launch_pdl(ctx, attn_fwd_tc_kernel<HD>, dim3(((p.S + QT - 1) / QT) * p.H * p.B, 1, 1), dim3(THREADS), F::SMEM, tmQ, tmK, tmV, p);
  return (int)cudaGetLastError();
}

template <int HD, int FORM>
int launch_fwd_scored(faar_ctx* ctx, const TcParams& p, const void* q, int64_t ldq, const void* k, const void* v, int64_t ldk) {
  using F = FwdScored<HD>;
  CUtensorMap tmQ, tmK, tmV;
  int e = head_map(ctx, &tmQ, q, p.B, p.S, p.H * HD, ldq, QT);
  if (!e) e = head_map(ctx, &tmK, k, p.B, p.S, p.Hkv * HD, ldk, KT);
  if (!e) e = head_map(ctx, &tmV, v, p.B, p.S, p.Hkv * HD, ldk, KT);
  if (!e) e = faar_allow_smem(ctx, (const void*)attn_fwd_scored_kernel<HD, FORM>, F::SMEM);
  if (e) return e;
  faar_launch_pdl(ctx, attn_fwd_scored_kernel<HD, FORM>, dim3(((p.S + QT - 1) / QT) * p.H * p.B, 1, 1), dim3(THREADS), F::SMEM, tmQ, tmK, tmV, p);
  return (int)cudaGetLastError();
}

// Over how many CTAs the items of a key tile are dealt: up to `most` CTAs in all (four an SM with heads of 64, of which two run at
// a time; one with heads of 128, where dQ next to this kernel has use for what is left), while the first key tile leaves each two
// items.  Backward call, one CTA a key tile -> two -> four, us: 32 / 8 heads of 64, 2 x 1000 tokens (128 key tiles) 112 -> 73 -> 70,
// 1 x 300 36 -> 24.6 -> 19, 4 x 2048 (512; one) 338 -> 361 -> 408; 16 / 8 heads of 128, 2 x 1000 (128; one) 64 -> 62.4 -> 81, in an
// alignment step 2882 -> 2905 with two; 3 x 2048 (384; one) 250 -> 275 -> 343.
int pick_parts(int most, int tiles, int longest) {
  int parts = 1;
  while (parts < 4 && 2 * parts * tiles <= most && longest >= 4 * parts) parts *= 2;
  return parts;
}

template <int HD, int FORM>
int launch_bwd(faar_ctx* ctx, TcBwdParams& p, const void* q, int64_t ldq, const void* k, const void* v, int64_t ldk,
               const void* dout, int64_t ldo) {
  CUtensorMap tmQ, tmDO, tmK, tmV, tmQk, tmDOk, tmKk, tmVk;      // boxes of 128 rows / of 64 rows
  int e = head_map(ctx, &tmQ, q, p.B, p.S, p.H * HD, ldq, QT);
  if (!e) e = head_map(ctx, &tmDO, dout, p.B, p.S, p.H * HD, ldo, QT);
  if (!e) e = head_map(ctx, &tmK, k, p.B, p.S, p.Hkv * HD, ldk, QT);
  if (!e) e = head_map(ctx, &tmV, v, p.B, p.S, p.Hkv * HD, ldk, QT);
  if (!e) e = head_map(ctx, &tmQk, q, p.B, p.S, p.H * HD, ldq, KT);
  if (!e) e = head_map(ctx, &tmDOk, dout, p.B, p.S, p.H * HD, ldo, KT);
  if (!e) e = head_map(ctx, &tmKk, k, p.B, p.S, p.Hkv * HD, ldk, KT);
  if (!e) e = head_map(ctx, &tmVk, v, p.B, p.S, p.Hkv * HD, ldk, KT);
  if (!e) e = faar_allow_smem(ctx, (const void*)attn_dkv_tc_kernel<HD, false, FORM>, Dkv<HD>::SMEM);
  if (!e) e = faar_allow_smem(ctx, (const void*)attn_dkv_tc_kernel<HD, true, FORM>, Dkv<HD>::SMEM);
  if (!e) e = faar_allow_smem(ctx, (const void*)attn_dq_tc_kernel<HD, FORM>, Dq<HD>::SMEM);
  if (e) return e;
  const int tiles = (p.S + QT - 1) / QT;
  // Ranges make key tiles of any work, the longest of which the others wait for: with capped scores, whose items are long against what
  // the exchange costs, heads of 64 deal up to twice as many.  Backward call, one CTA a key tile -> two (where not said otherwise 4 x 2048
  // tokens, 32 / 8 heads of 64), us: capped, documents of 700 tokens 534 -> 507, of 200 315 -> 286, one each 591 -> 587; 1 x 8192, documents of
  // 700 634 -> 544, of 3000 1153 -> 920; 8 x 1000, of 300 323 -> 295; 3 x 2048, 8 / 8 heads, of 700 150 -> 136; biased too, of 700 587 ->
  // 555, one each 642 -> 648.  Not capped, where it is left at one: of 700 377 -> 364, of 200 228 -> 210, one each 408 -> 420.  Heads of 128:
  // capped, of 700 334 -> 376, one each 386 -> 424, not capped, of 200 171 -> 204.
  const int more = HD == 64 && (FORM & CAPPED) && (p.sc.key_lo || p.sc.key_hi) ? 2 : 1;
  p.parts = pick_parts(more * ctx->num_sms * Dkv<HD>::CTAS * Dkv<HD>::CTAS, tiles * p.Hkv * p.B, p.H / p.Hkv * ((p.S + KT - 1) / KT));
  auto launch_dq = [&] {
    faar_launch_pdl(ctx, attn_dq_tc_kernel<HD, FORM>, dim3(tiles * p.H * p.B, 1, 1), dim3(BWD_THREADS), Dq<HD>::SMEM, tmQ, tmDO, tmKk, tmVk, p);
    return (int)cudaGetLastError();
  };
  if (FORM != CAUSAL) {                                    // dK and dV take delta as this kernel leaves it
    e = launch_dq();
    if (e) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = p.parts;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3(tiles * p.Hkv * p.B * p.parts);
  cfg.blockDim = dim3(BWD_THREADS);
  cfg.dynamicSmemBytes = Dkv<HD>::SMEM;
  cfg.stream = ctx->stream;
  cfg.attrs = attr;
  cfg.numAttrs = p.parts > 1 ? 2 : 1;
  e = (int)cudaLaunchKernelEx(&cfg, p.parts > 1 ? attn_dkv_tc_kernel<HD, true, FORM> : attn_dkv_tc_kernel<HD, false, FORM>, tmQk, tmDOk, tmK, tmV, p);
  if (!e) e = (int)cudaGetLastError();
  return e || FORM != CAUSAL ? e : launch_dq();
}

// Whether dq (rows of ldq elements) lies over something that the dK / dV kernel reads
bool over_inputs(int B, int S, int H, int Hkv, int D, const void* dq, const void* q, int64_t ldq, const void* k, const void* v, int64_t ldk,
                 const void* dout, int64_t ldo) {
  const uintptr_t dq0 = reinterpret_cast<uintptr_t>(dq), rows = (uintptr_t)B * S - 1, dq1 = dq0 + (rows * ldq + (uintptr_t)H * D) * 2;
  auto meets = [&](const void* a, int64_t ld, int heads) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a);
    return x < dq1 && dq0 < x + (rows * ld + (uintptr_t)heads * D) * 2;
  };
  return meets(q, ldq, H) || meets(dout, ldo, H) || meets(k, ldk, Hkv) || meets(v, ldk, Hkv);
}

// What the scored backward kernels need of every row first, one warp a job: delta[b, h, q] = sum of dO * O over the head, 256 / D rows
// a job (the first `head_jobs` jobs), and for every 64 queries what they see together: keys from x on and before y are seen by one
// at least (x >= y: by none), from z on and before w by every one.  Bound by reading out and dout.  In the dQ kernel, whose CTAs have these
// rows, it would be a launch less but a wait more in each: 4 x 2048 tokens, 32 / 8 heads of 64, causal 414 -> 434 us, documents of 700 capped 484 -> 516;
// 333 tokens, a step, 32.2 -> 33.0.
template <int D>
__global__ void __launch_bounds__(128)
attn_scored_rows_kernel(const __nv_bfloat16* out, const __nv_bfloat16* dout, long long ldo, int B, int S, int H, const ScoreArgs sc, float* delta,
                        int4* tiles, long long head_jobs, long long jobs) {
  faar_pdl_sync();
  constexpr int LPR = D / 8, ROWS = 32 / LPR;               // lanes a row, rows at once
  const int lane = threadIdx.x & 31, chunks = (S + ROWS - 1) / ROWS, n_qt = (S + KT - 1) / KT;
  for (long long job = blockIdx.x * 4ll + (threadIdx.x >> 5); job < jobs; job += gridDim.x * 4ll) {
    if (job < head_jobs) {
      const int h = (int)(job % H);                         // heads fastest: the rows' lines are read whole
      const long long rest = job / H;
      const int b = (int)(rest / chunks), q = (int)(rest % chunks) * ROWS + lane / LPR;
      float acc = 0.f;
      if (q < S) {
        const long long at = ((long long)b * S + q) * ldo + h * D + 8 * (lane % LPR);
        float x[8], y[8];
        faar_unpack8(*reinterpret_cast<const uint4*>(out + at), x);
        faar_unpack8(*reinterpret_cast<const uint4*>(dout + at), y);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc = fmaf(x[i], y[i], acc);
      }
#pragma unroll
      for (int o = LPR / 2; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
      if (q < S && lane % LPR == 0) delta[((long long)b * H + h) * S + q] = acc;
    } else {
      const long long t = job - head_jobs;
      const int b = (int)(t / n_qt), q0 = (int)(t % n_qt) * KT;
      int4 v = make_int4(EMPTY_LO, EMPTY_HI, 0, INT_MAX);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int q = q0 + lane + 32 * i;
        if (q >= S) continue;
        const int2 r = key_range(sc, b, q, S);
        v.x = min(v.x, r.x); v.y = max(v.y, r.y); v.z = max(v.z, r.x); v.w = min(v.w, r.y);
      }
      v.x = __reduce_min_sync(0xffffffffu, v.x); v.y = __reduce_max_sync(0xffffffffu, v.y);
      v.z = __reduce_max_sync(0xffffffffu, v.z); v.w = __reduce_min_sync(0xffffffffu, v.w);
      if (lane == 0) tiles[t] = v;
    }
  }
}

ScoreArgs score_args(const faar_attention_scores* s, float scale) {
  ScoreArgs a = {};
  if (s->softcap > 0.f) {
    const double out = (double)s->softcap * 1.4426950408889634;
    a.cap_in = (float)((double)scale / s->softcap);
    a.cap_out = (float)out;
    for (int i = 0; i < CAP_TERMS; ++i) {
      a.cap_series[i] = (float)(CAP_SERIES[i] * out);
      a.tanh_series[i] = (float)CAP_SERIES[i];
    }
  }
  a.slopes = s->slopes; a.key_lo = s->key_lo; a.key_hi = s->key_hi;
  return a;
}
// The kernels compiled for a form of scores
template <class Fn> int by_form(const faar_attention_scores* s, Fn&& fn) {
  using std::integral_constant;
  if (s->softcap > 0.f)
    return s->slopes ? fn(integral_constant<int, RANGES | CAPPED | BIASED>{}) : fn(integral_constant<int, RANGES | CAPPED>{});
  return s->slopes ? fn(integral_constant<int, RANGES | BIASED>{}) : fn(integral_constant<int, RANGES>{});
}

}  // namespace

// Scratch of a scored backward call: delta [B, H, S] floats, then a record for every 64 queries
static size_t delta_bytes(int B, int S, int H) { return ((size_t)B * H * S * sizeof(float) + 15) / 16 * 16; }
size_t faar_attention_scored_scratch(int B, int S, int H) {
  return delta_bytes(B, S, H) + (size_t)B * (((size_t)S + KT - 1) / KT) * sizeof(int4);
}

int faar_launch_attention_scored_fwd(faar_ctx* ctx, int B, int S, int H, int Hkv, int D, const void* q, int64_t ldq, const void* k, const void* v,
                                     int64_t ldk, const faar_attention_scores* scores, void* out, int64_t ldo, float* lse) {
  faar_prof_scope ps(ctx, FAAR_K_ATTENTION);
  const float scale = scores->scale > 0.f ? scores->scale : 1.0f / sqrtf((float)D);
  TcParams p = {};
  p.out = reinterpret_cast<__nv_bfloat16*>(out); p.lse = lse; p.ldo = ldo; p.B = B; p.S = S; p.H = H; p.Hkv = Hkv;
  p.scale_log2 = scale * 1.4426950408889634f;
  p.sc = score_args(scores, scale);
  return by_form(scores, [&](auto form) {
    constexpr int F = decltype(form)::value;
    return D == 64 ? launch_fwd_scored<64, F>(ctx, p, q, ldq, k, v, ldk) : launch_fwd_scored<128, F>(ctx, p, q, ldq, k, v, ldk);
  });
}

int faar_launch_attention_scored_bwd(faar_ctx* ctx, int B, int S, int H, int Hkv, int D, const void* q, int64_t ldq, const void* k, const void* v,
                                     int64_t ldk, const faar_attention_scores* scores, const void* out, const void* dout, int64_t ldo,
                                     const float* lse, void* scratch, void* dq, void* dk, void* dv) {
  faar_prof_scope ps(ctx, FAAR_K_ATTENTION);
  const float scale = scores->scale > 0.f ? scores->scale : 1.0f / sqrtf((float)D);
  float* delta = reinterpret_cast<float*>(scratch);
  int4* tiles = reinterpret_cast<int4*>(reinterpret_cast<uint8_t*>(scratch) + delta_bytes(B, S, H));
  TcBwdParams p = {};
  p.lse = lse; p.dsum = delta;
  p.sum_parts = 1; p.sum_head = S; p.sum_batch = (long long)H * S;
  p.dq = reinterpret_cast<__nv_bfloat16*>(dq); p.dk = reinterpret_cast<__nv_bfloat16*>(dk); p.dv = reinterpret_cast<__nv_bfloat16*>(dv);
  p.q = reinterpret_cast<const __nv_bfloat16*>(q); p.k = reinterpret_cast<const __nv_bfloat16*>(k); p.dout = reinterpret_cast<const __nv_bfloat16*>(dout); p.ldo = ldo;
  p.ldq = ldq; p.ldk = ldk; p.B = B; p.S = S; p.H = H; p.Hkv = Hkv;
  p.scale_log2 = scale * 1.4426950408889634f; p.inv_sqrt_d = scale;
  p.sc = score_args(scores, scale);
  p.sc.tiles = tiles;
  const int rows = 256 / D;
  const long long head_jobs = (long long)B * H * ((S + rows - 1) / rows), jobs = head_jobs + (long long)B * ((S + KT - 1) / KT);
  long long blocks = (jobs + 3) / 4;
  if (blocks > (long long)ctx->num_sms * 16) blocks = (long long)ctx->num_sms * 16;
  faar_launch_pdl(ctx, D == 64 ? attn_scored_rows_kernel<64> : attn_scored_rows_kernel<128>, dim3((unsigned)blocks), dim3(128), 0,
                  reinterpret_cast<const __nv_bfloat16*>(out), reinterpret_cast<const __nv_bfloat16*>(dout), (long long)ldo, B, S, H, p.sc, delta,
                  tiles, head_jobs, jobs);
  return by_form(scores, [&](auto form) {
    constexpr int F = decltype(form)::value;
    return D == 64 ? launch_bwd<64, F>(ctx, p, q, ldq, k, v, ldk, dout, ldo) : launch_bwd<128, F>(ctx, p, q, ldq, k, v, ldk, dout, ldo);
  });
}

int faar_launch_attention_fwd_tc(faar_ctx* ctx, int B, int S, int H, int Hkv, int D, const void* q, int64_t ldq, const void* k,
                                 const void* v, int64_t ldk, void* out, int64_t ldo, float* lse, float scale_log2) {
  if ((long long)B * S > 0x7FFFFFFFll) return (int)cudaErrorInvalidValue;
  TcParams p = {};
  p.out = reinterpret_cast<__nv_bfloat16*>(out); p.lse = lse; p.ldo = ldo; p.B = B; p.S = S; p.H = H; p.Hkv = Hkv;
  p.scale_log2 = scale_log2;
  return D == 64 ? launch_fwd<64>(ctx, p, q, ldq, k, v, ldk) : launch_fwd<128>(ctx, p, q, ldq, k, v, ldk);
}

int faar_launch_attention_bwd_tc(faar_ctx* ctx, int B, int S, int H, int Hkv, int D, const void* q, int64_t ldq, const void* k,
                                 const void* v, int64_t ldk, const void* dout, int64_t ldo, const float* lse,
                                 const float* dsum, int sum_parts, void* dq, void* dk, void* dv, float scale_log2, const float2* rope) {
  if ((long long)B * S > 0x7FFFFFFFll) return (int)cudaErrorInvalidValue;
  TcBwdParams p = {};
  p.rope = rope;
  p.lse = lse; p.dsum = dsum;
  // attn_dsum_kernel: [B, H, S]; the product that wrote dO: [parts, H, B S]
  p.sum_parts = sum_parts ? sum_parts : 1;
  p.sum_head = sum_parts ? (long long)B * S : S; p.sum_batch = sum_parts ? S : (long long)H * S; p.sum_part = (long long)B * S * H;
  p.dq = reinterpret_cast<__nv_bfloat16*>(dq); p.dk = reinterpret_cast<__nv_bfloat16*>(dk); p.dv = reinterpret_cast<__nv_bfloat16*>(dv);
  p.ldq = ldq; p.ldk = ldk; p.B = B; p.S = S; p.H = H; p.Hkv = Hkv; p.scale_log2 = scale_log2;
  p.inv_sqrt_d = scale_log2 / 1.4426950408889634f;
  p.apart = over_inputs(B, S, H, Hkv, D, dq, q, ldq, k, v, ldk, dout, ldo);
  return D == 64 ? launch_bwd<64, CAUSAL>(ctx, p, q, ldq, k, v, ldk, dout, ldo) : launch_bwd<128, CAUSAL>(ctx, p, q, ldq, k, v, ldk, dout, ldo);
}

// Reads and clears the status word of this module (synchronous copy: call after the stream has been synchronised).
int faar_attention_tc_status(uint32_t* code_out) {
  uint32_t v = 0, zero = 0;
  cudaError_t e = cudaMemcpyFromSymbol(&v, g_attn_status, sizeof(v));
  if (e == cudaSuccess && v) e = cudaMemcpyToSymbol(g_attn_status, &zero, sizeof(zero));
  *code_out = v;
  return (int)e;
}
