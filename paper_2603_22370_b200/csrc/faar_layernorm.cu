// Layer norm of a decoder block whose norms have a mean and a bias: forward, alone or behind a residual sum, and backward
// with the gradients of weight and bias.  BF16 rows in and out, FP32 statistics, weights and weight gradients.
//   y = (x - m) r g + b,  m = mean(x),  r = 1 / sqrt(mean((x - m)^2) + eps)
//   with h = (x - m) r and w = g dy:  dx = r (w - mean(w) - h mean(w h)),  dg = sum over rows of dy h,  db = of dy
// The variance is the mean square of what is left after the mean has been taken off (two passes over values that are on
// the chip): the difference of mean squares would lose every digit of a row whose mean is large against its spread.
#include "faar_internal.cuh"

namespace {


__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

// ---- how both passes go over the rows -------------------------------------------------------------------------
// A group of threads (whole warps) takes a row: a thread holds the same 8 VPT columns of every row that its group takes, so the
// norm's weights and the columns' gradients stay in registers (a warp a row would read the FP32 weights from L1 for every row, four
// times the row's own traffic: 8192 x 2048 forward 23.4 us).  R rows at a time: their sums go through shuffles and
// shared memory together, with one barrier of the group, while copies into shared memory run ahead, of which a thread reads only what
// it has copied itself: they need no barrier.  A CTA holds up to 512 threads, of one group or of several with rows of their own,
// and an SM one CTA.
constexpr int MAX_THREADS = 512;
template <int VPT, int TENSORS> constexpr int ROWS_AT_ONCE = VPT == 4 ? 1 : (TENSORS == 3 ? 2 : 4) / VPT;
// TENSORS inputs come through the ring: 16-byte units a thread and stage, stages (196 KB in all at the most), bytes a thread
template <int VPT, int TENSORS> constexpr int STAGE_UNITS = ROWS_AT_ONCE<VPT, TENSORS> * VPT * TENSORS;
template <int VPT, int TENSORS> constexpr int RING_STAGES = STAGE_UNITS<VPT, TENSORS> <= 4 ? 4 : STAGE_UNITS<VPT, TENSORS> <= 8 ? 3 : 2;
template <int VPT, int TENSORS> constexpr int RING_BYTES = RING_STAGES<VPT, TENSORS> * STAGE_UNITS<VPT, TENSORS> * 16;

struct Group {
  int tpr, id, t, lane, warp, warps;     // threads a row; which group of the CTA; thread, lane, warp of the group; its warps
  __device__ explicit Group(int tpr_) : tpr(tpr_), id(threadIdx.x / tpr_), t(threadIdx.x - id * tpr_), lane(threadIdx.x & 31), warp(t >> 5), warps(tpr_ >> 5) {}
  __device__ void sync() const { asm volatile("barrier.cta.sync %0, %1;" ::"r"(1 + id), "r"(tpr) : "memory"); }
};
// V sums over the group, all at once: lane l gets number l % V.  `slots` [warps][V] is free again once the group has come to the
// next barrier.
template <int V>
__device__ __forceinline__ float group_sums(float (&sum)[V], const Group& g, float* slots) {
  // halves of the values change places with halves of the lanes until a lane has one: lane l that of number l / (32 / V)
#pragma unroll
  for (int n = V / 2, o = 16; n > 0; n /= 2, o /= 2)
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const bool up = g.lane & o;
      const float send = up ? sum[i] : sum[i + n], keep = up ? sum[i + n] : sum[i];
      sum[i] = keep + __shfl_xor_sync(0xffffffffu, send, o);
    }
#pragma unroll
  for (int o = 16 / V; o > 0; o /= 2) sum[0] += __shfl_xor_sync(0xffffffffu, sum[0], o);
  if (g.warps == 1) return __shfl_sync(0xffffffffu, sum[0], g.lane % V * (32 / V));
  if (g.lane % (32 / V) == 0) slots[g.warp * V + g.lane / (32 / V)] = sum[0];
  g.sync();
  float total = 0.f;
  for (int w = g.lane / V; w < g.warps; w += 32 / V) total += slots[w * V + g.lane % V];
#pragma unroll
  for (int o = V; o < 32; o *= 2) total += __shfl_xor_sync(0xffffffffu, total, o);
  return total;
}

// The ring: copies of R rows' columns of up to three matrices; what is not there arrives as zeros
template <int VPT, int TENSORS>
struct Ring {
  static constexpr int R = ROWS_AT_ONCE<VPT, TENSORS>, STAGES = RING_STAGES<VPT, TENSORS>;
  uint4* mine;                           // [STAGES][STAGE_UNITS][threads of the CTA]
  const __nv_bfloat16* p[TENSORS];
  int64_t ld[TENSORS];
  int rows, cols, column0, column_step;
  __device__ __forceinline__ uint4* unit(int stage, int tensor, int r, int k) const {
    return mine + (stage * STAGE_UNITS<VPT, TENSORS> + (tensor * R + r) * VPT + k) * (int)blockDim.x;
  }
  __device__ __forceinline__ void request(int stage, int64_t row0) const {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int k = 0; k < VPT; ++k) {
        const int c = column0 + column_step * k;
        const bool there = row0 + r < rows && c < cols;
        const uint32_t bytes = there ? 16u : 0u;
#pragma unroll
        for (int t = 0; t < TENSORS; ++t)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                       ::"r"((uint32_t)__cvta_generic_to_shared(unit(stage, t, r, k))), "l"(p[t] + (there ? (row0 + r) * ld[t] + c : 0)), "r"(bytes) : "memory");
      }
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  __device__ __forceinline__ void wait() const { asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory"); }
  static __device__ __forceinline__ int before(int stage) { return stage == 0 ? STAGES - 1 : stage - 1; }
  static __device__ __forceinline__ int after(int stage) { return stage == STAGES - 1 ? 0 : stage + 1; }
};

// ---- forward: with SUM the row is first formed as the BF16-rounded sum x + b and written to `sum_out` -------------
template <int VPT, bool SUM>
__global__ void __launch_bounds__(MAX_THREADS)
layernorm_kernel(const __nv_bfloat16* x, int64_t ldx, const __nv_bfloat16* b, int64_t ldb, __nv_bfloat16* sum_out, int64_t lds,
                 const float* __restrict__ g, const float* __restrict__ bias, float eps, __nv_bfloat16* y, int64_t ldy, float* mean_out,
                 float* rstd_out, int rows, int cols, int tpr) {
  using RingT = Ring<VPT, SUM ? 2 : 1>;
  constexpr int R = RingT::R;
  extern __shared__ uint4 ring_memory[];
  __shared__ float slots[2][MAX_THREADS / 32 * R];
  faar_pdl_sync();
  const Group grp(tpr);
  RingT ring;
  ring.mine = ring_memory + threadIdx.x;
  ring.p[0] = x; ring.ld[0] = ldx;
  if constexpr (SUM) { ring.p[1] = b; ring.ld[1] = ldb; }
  ring.rows = rows; ring.cols = cols; ring.column0 = 8 * grp.t; ring.column_step = 8 * tpr;
  auto column = [&](int k) { return 8 * (grp.t + tpr * k); };
  const int groups = blockDim.x / tpr;
  const int64_t first = ((int64_t)blockIdx.x * groups + grp.id) * R, step = (int64_t)gridDim.x * groups * R;
#pragma unroll
  for (int st = 0; st < RingT::STAGES - 1; ++st) ring.request(st, first + st * step);
  float gg[VPT][8] = {}, bb[VPT][8] = {};
#pragma unroll
  for (int k = 0; k < VPT; ++k)
    if (column(k) < cols) {
      load8(g + column(k), gg[k]);
      if (bias) load8(bias + column(k), bb[k]);
    }
  float* const slot0 = slots[0] + grp.id * grp.warps * R;
  float* const slot1 = slots[1] + grp.id * grp.warps * R;
  int stage = 0;
  for (int64_t row0 = first; row0 < rows; row0 += step, stage = RingT::after(stage)) {
    ring.wait();
    uint4 v[R][VPT];
    float sum[R], mean[R], rstd[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      sum[r] = 0.f;
#pragma unroll
      for (int k = 0; k < VPT; ++k) {
        v[r][k] = *ring.unit(stage, 0, r, k);                 // zeros behind the last column
        float a[8];
        faar_unpack8(v[r][k], a);
        if constexpr (SUM) {
          float u[8];
          faar_unpack8(*ring.unit(stage, 1, r, k), u);
#pragma unroll
          for (int i = 0; i < 8; ++i) a[i] += u[i];
          v[r][k] = faar_pack8(a);
          faar_unpack8(v[r][k], a);
          if (row0 + r < rows && column(k) < cols) *reinterpret_cast<uint4*>(sum_out + (row0 + r) * lds + column(k)) = v[r][k];
        }
        sum[r] += ((a[0] + a[1]) + (a[2] + a[3])) + ((a[4] + a[5]) + (a[6] + a[7]));
      }
    }
    ring.request(RingT::before(stage), row0 + (RingT::STAGES - 1) * step);       // the stage of the turn before, which has been read
    float total = group_sums<R>(sum, grp, slot0) / (float)cols;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      mean[r] = __shfl_sync(0xffffffffu, total, r);
      sum[r] = 0.f;
#pragma unroll
      for (int k = 0; k < VPT; ++k) {
        if (column(k) >= cols) continue;
        float a[8];
        faar_unpack8(v[r][k], a);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[r] = fmaf(a[i] - mean[r], a[i] - mean[r], sum[r]);
      }
    }
    total = 1.0f / sqrtf(group_sums<R>(sum, grp, slot1) / (float)cols + eps);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      rstd[r] = __shfl_sync(0xffffffffu, total, r);
      if (row0 + r >= rows) continue;
      if (grp.t == 0) {
        if (mean_out) mean_out[row0 + r] = mean[r];
        if (rstd_out) rstd_out[row0 + r] = rstd[r];
      }
#pragma unroll
      for (int k = 0; k < VPT; ++k) {
        if (column(k) >= cols) continue;
        float a[8];
        faar_unpack8(v[r][k], a);
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = fmaf((a[i] - mean[r]) * rstd[r], gg[k][i], bb[k][i]);
        *reinterpret_cast<uint4*>(y + (row0 + r) * ldy + column(k)) = faar_pack8(a);
      }
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

// Forward of rows too long for that: one CTA a row, which it reads three times, twice from L2 (the threads read back what they wrote)
template <bool SUM>
__global__ void __launch_bounds__(MAX_THREADS)
layernorm_long_kernel(const __nv_bfloat16* x, int64_t ldx, const __nv_bfloat16* b, int64_t ldb, __nv_bfloat16* sum_out, int64_t lds,
                      const float* __restrict__ g, const float* __restrict__ bias, float eps, __nv_bfloat16* y, int64_t ldy, float* mean_out,
                      float* rstd_out, int cols) {
  __shared__ float slots[2][MAX_THREADS / 32];
  faar_pdl_sync();
  const Group grp(MAX_THREADS);
  const int64_t row = blockIdx.x;
  const __nv_bfloat16* src = SUM ? sum_out + row * lds : x + row * ldx;
  float s[1] = {0.f}, ss[1] = {0.f};
  for (int c = 8 * threadIdx.x; c < cols; c += 8 * MAX_THREADS) {
    float a[8];
    uint4 v = *reinterpret_cast<const uint4*>(x + row * ldx + c);
    faar_unpack8(v, a);
    if (SUM) {
      float r[8];
      faar_unpack8(*reinterpret_cast<const uint4*>(b + row * ldb + c), r);
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] += r[i];
      v = faar_pack8(a);
      *reinterpret_cast<uint4*>(sum_out + row * lds + c) = v;
      faar_unpack8(v, a);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) s[0] += a[i];
  }
  const float mean = group_sums<1>(s, grp, slots[0]) / (float)cols;
  for (int c = 8 * threadIdx.x; c < cols; c += 8 * MAX_THREADS) {
    float a[8];
    faar_unpack8(*reinterpret_cast<const uint4*>(src + c), a);
#pragma unroll
    for (int i = 0; i < 8; ++i) ss[0] = fmaf(a[i] - mean, a[i] - mean, ss[0]);
  }
  const float rstd = 1.0f / sqrtf(group_sums<1>(ss, grp, slots[1]) / (float)cols + eps);
  if (threadIdx.x == 0) {
    if (mean_out) mean_out[row] = mean;
    if (rstd_out) rstd_out[row] = rstd;
  }
  for (int c = 8 * threadIdx.x; c < cols; c += 8 * MAX_THREADS) {
    float a[8], gg[8], bb[8];
    faar_unpack8(*reinterpret_cast<const uint4*>(src + c), a);
    load8(g + c, gg);
    if (bias) load8(bias + c, bb);
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = fmaf((a[i] - mean) * rstd, gg[i], bias ? bb[i] : 0.f);
    *reinterpret_cast<uint4*>(y + row * ldy + c) = faar_pack8(a);
  }
}

// ---- backward: one pass over x and dy for all three results ------------------------------------------------------
// The columns' weight gradients stay in registers over all of a group's rows; a CTA's groups add theirs up in shared memory, and
// the CTAs' sums ([slabs][2][cols]) are added by a second kernel, in an order that the launch shape alone decides.
template <int VPT, bool ADD>
__global__ void __launch_bounds__(MAX_THREADS)
layernorm_bwd_kernel(const __nv_bfloat16* dy, int64_t lddy, const __nv_bfloat16* x, int64_t ldx, const float* __restrict__ g,
                     const float* __restrict__ mean_in, const float* __restrict__ rstd_in, const __nv_bfloat16* add, int64_t ldadd,
                     __nv_bfloat16* dx, int64_t lddx, float* partials, int rows, int cols, int tpr) {
  using RingT = Ring<VPT, ADD ? 3 : 2>;
  constexpr int R = RingT::R, V = 2 * R;
  constexpr bool KEEP = VPT < 4;                             // room for the norm's weights in registers
  extern __shared__ uint4 ring_memory[];
  __shared__ float slots[2][MAX_THREADS / 32 * V];
  faar_pdl_sync();
  const Group grp(tpr);
  RingT ring;
  ring.mine = ring_memory + threadIdx.x;
  ring.p[0] = x; ring.ld[0] = ldx; ring.p[1] = dy; ring.ld[1] = lddy;
  if constexpr (ADD) { ring.p[2] = add; ring.ld[2] = ldadd; }
  ring.rows = rows; ring.cols = cols; ring.column0 = 8 * grp.t; ring.column_step = 8 * tpr;
  auto column = [&](int k) { return 8 * (grp.t + tpr * k); };
  const int groups = blockDim.x / tpr;
  const int64_t first = ((int64_t)blockIdx.x * groups + grp.id) * R, step = (int64_t)gridDim.x * groups * R;
#pragma unroll
  for (int st = 0; st < RingT::STAGES - 1; ++st) ring.request(st, first + st * step);
  float gg[KEEP ? VPT : 1][8], dg[VPT][8] = {}, db[VPT][8] = {};
  if constexpr (KEEP) {
#pragma unroll
    for (int k = 0; k < VPT; ++k)
      if (column(k) < cols) load8(g + column(k), gg[k]);
  }
  // the norm's weights of the k-th vector
  auto weights = [&](int k) -> float (&)[8] {
    if constexpr (!KEEP) load8(g + column(k), gg[0]);
    return gg[KEEP ? k : 0];
  };
  float mean_next[R], rstd_next[R];
  auto request_stats = [&](int64_t row0) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      mean_next[r] = row0 + r < rows ? mean_in[row0 + r] : 0.f;
      rstd_next[r] = row0 + r < rows ? rstd_in[row0 + r] : 0.f;
    }
  };
  request_stats(first);
  int turn = 0, stage = 0;
  for (int64_t row0 = first; row0 < rows; row0 += step, turn ^= 1, stage = RingT::after(stage)) {
    ring.wait();
    uint4 xv[R][VPT], dv[R][VPT];
    float mean[R], rstd[R], sum[V];
#pragma unroll
    for (int r = 0; r < R; ++r) { mean[r] = mean_next[r]; rstd[r] = rstd_next[r]; }
    request_stats(row0 + step);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float sw = 0.f, swh = 0.f;
#pragma unroll
      for (int k = 0; k < VPT; ++k) {
        xv[r][k] = *ring.unit(stage, 0, r, k);
        dv[r][k] = *ring.unit(stage, 1, r, k);
        if (column(k) >= cols) continue;
        float a[8], d[8];
        faar_unpack8(xv[r][k], a);
        faar_unpack8(dv[r][k], d);
        const float(&gk)[8] = weights(k);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float h = (a[i] - mean[r]) * rstd[r], w = d[i] * gk[i];
          sw += w;
          swh = fmaf(w, h, swh);
          dg[k][i] = fmaf(d[i], h, dg[k][i]);
          db[k][i] += d[i];
        }
      }
      sum[2 * r] = sw;
      sum[2 * r + 1] = swh;
    }
    ring.request(RingT::before(stage), row0 + (RingT::STAGES - 1) * step);       // the stage of the turn before, which has been read
    const float total = group_sums<V>(sum, grp, slots[turn] + grp.id * grp.warps * V) / (float)cols;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float mw = __shfl_sync(0xffffffffu, total, 2 * r), mwh = __shfl_sync(0xffffffffu, total, 2 * r + 1);
      if (row0 + r >= rows) continue;
#pragma unroll
      for (int k = 0; k < VPT; ++k) {
        if (column(k) >= cols) continue;
        float a[8], d[8];
        faar_unpack8(xv[r][k], a);
        faar_unpack8(dv[r][k], d);
        const float(&gk)[8] = weights(k);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float h = (a[i] - mean[r]) * rstd[r];
          a[i] = rstd[r] * (fmaf(-h, mwh, d[i] * gk[i]) - mw);
        }
        if constexpr (ADD) {
          faar_unpack8(*ring.unit(stage, 2, r, k), d);
#pragma unroll
          for (int i = 0; i < 8; ++i) a[i] += d[i];
        }
        *reinterpret_cast<uint4*>(dx + (row0 + r) * lddx + column(k)) = faar_pack8(a);
      }
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  if (!partials) return;
  if (groups > 1) {                                          // over the ring: [vector][half][groups][tpr], eight columns' halves side by side
    __syncthreads();
    float4* all = reinterpret_cast<float4*>(ring_memory);
    auto at = [&](int k, int part, int id) { return all + ((k * 4 + part) * groups + id) * tpr + grp.t; };
#pragma unroll
    for (int k = 0; k < VPT; ++k)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        *at(k, h, grp.id) = make_float4(dg[k][4 * h], dg[k][4 * h + 1], dg[k][4 * h + 2], dg[k][4 * h + 3]);
        *at(k, 2 + h, grp.id) = make_float4(db[k][4 * h], db[k][4 * h + 1], db[k][4 * h + 2], db[k][4 * h + 3]);
      }
    __syncthreads();
    if (grp.id != 0) return;
    for (int id = 1; id < groups; ++id)
#pragma unroll
      for (int k = 0; k < VPT; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float4 u = *at(k, h, id), w = *at(k, 2 + h, id);
          dg[k][4 * h] += u.x; dg[k][4 * h + 1] += u.y; dg[k][4 * h + 2] += u.z; dg[k][4 * h + 3] += u.w;
          db[k][4 * h] += w.x; db[k][4 * h + 1] += w.y; db[k][4 * h + 2] += w.z; db[k][4 * h + 3] += w.w;
        }
  }
  float* out = partials + (int64_t)blockIdx.x * 2 * cols;
#pragma unroll
  for (int k = 0; k < VPT; ++k) {
    if (column(k) >= cols) continue;
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      *reinterpret_cast<float4*>(out + column(k) + i) = make_float4(dg[k][i], dg[k][i + 1], dg[k][i + 2], dg[k][i + 3]);
      *reinterpret_cast<float4*>(out + cols + column(k) + i) = make_float4(db[k][i], db[k][i + 1], db[k][i + 2], db[k][i + 3]);
    }
  }
}

// The slabs' sums: 32 columns a CTA, 32 threads a column
__global__ void __launch_bounds__(1024)
layernorm_dw_sum_kernel(const float* partials, int slabs, float* dg, float* db, int cols) {
  __shared__ float part[32][33];
  faar_pdl_sync();
  const int c = blockIdx.x * 32 + threadIdx.x;
  float s = 0.f;
  if (c < 2 * cols)
    for (int k = threadIdx.y; k < slabs; k += 32) s += partials[(int64_t)k * 2 * cols + c];
  part[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  s = faar_warp_sum(part[threadIdx.x][threadIdx.y]);         // of column threadIdx.y
  const int mine = blockIdx.x * 32 + threadIdx.y;
  if (threadIdx.x == 0 && mine < 2 * cols) {
    float* out = mine < cols ? dg : db;
    if (out) out[mine < cols ? mine : mine - cols] = s;
  }
}

// Launch shape: vectors of 8 columns a thread, threads a row, groups a CTA (no more than give every SM a CTA), CTAs.  Two vectors a
// thread make more groups, whose turns (a sum's latency, then another's work) overlap; a short row has no use for them.  Behind a sum
// or not, the same shape: the same bits.  us, one vector -> two (-> four): forward 8192 x 2048 20.6 -> 18.2, 8192 x 4096 37.5 -> 31.8 (33.2), 16384 x
// 1024 20.8 -> 18.1, with the sum 8192 x 4096 45.8 -> 49.6; backward 8192 x 2048 29.4 -> 27.3 (37.3), 8192 x 4096 49.0 -> 46.1 (61.4).
// A plain copy of as many bytes as 8192 x 4096 forward takes 24.9-28.3.  With a residual (forward) or its gradient (backward), 8192 x 2048
// 24.0 and 32.8, 8192 x 4096 49.9 and 58.6, 777 x 1040 4.5 and 7.5.  By counters (8192 x 4096 forward, backward): instruction issue 63 and 67 %
// of the cycles at work, ALU 33 and 44, FMA 31 and 37, DRAM 30 and 46: none is full, with 16 warps an SM that wait for their group's sums,
// twice a row forward and once backward.
struct Shape { int vpt, tpr, groups, ctas; };
static_assert(4 * 8 * MAX_THREADS == FAAR_LAYERNORM_COLS, "four vectors a thread at the most");
Shape shape(const faar_ctx* ctx, int rows, int cols) {
  Shape s;
  const int vectors = cols / 8;
  s.vpt = vectors <= 64 ? 1 : vectors <= 2 * MAX_THREADS ? 2 : 4;
  s.tpr = ((vectors + s.vpt - 1) / s.vpt + 31) / 32 * 32;
  const int64_t turns = ((int64_t)rows * s.vpt + 3) / 4;     // of four rows, two or one
  const int64_t even = (turns + ctx->num_sms - 1) / ctx->num_sms;
  s.groups = MAX_THREADS / s.tpr;
  if (s.groups > even) s.groups = (int)even;
  const int64_t ctas = (turns + s.groups - 1) / s.groups;
  s.ctas = (int)(ctas < ctx->num_sms ? ctas : ctx->num_sms);
  return s;
}

}  // namespace

int faar_layernorm_slabs(const faar_ctx* ctx, int rows, int cols) { return shape(ctx, rows, cols).ctas; }

int faar_launch_layernorm(faar_ctx* ctx, int rows, int cols, const void* x, int64_t ldx, const void* b, int64_t ldb, void* sum_out, int64_t lds,
                          const float* g, const float* bias, float eps, void* y, int64_t ldy, float* mean, float* rstd) {
  faar_prof_scope ps(ctx, FAAR_K_GLUE);
  auto* xp = reinterpret_cast<const __nv_bfloat16*>(x);
  auto* bp = reinterpret_cast<const __nv_bfloat16*>(b);
  auto* sp = reinterpret_cast<__nv_bfloat16*>(sum_out);
  auto* yp = reinterpret_cast<__nv_bfloat16*>(y);
  if (cols > FAAR_LAYERNORM_COLS) {
    faar_launch_pdl(ctx, bp ? layernorm_long_kernel<true> : layernorm_long_kernel<false>, dim3((unsigned)rows), dim3(MAX_THREADS), 0, xp, ldx, bp, ldb,
                    sp, lds, g, bias, eps, yp, ldy, mean, rstd, cols);
    return (int)cudaGetLastError();
  }
  const Shape s = shape(ctx, rows, cols);
  auto launch = [&](auto* kernel, int bytes) {
    const int e = faar_allow_smem(ctx, (const void*)kernel, bytes * MAX_THREADS);
    if (e) return e;
    const int threads = s.tpr * s.groups;
    faar_launch_pdl(ctx, kernel, dim3(s.ctas), dim3(threads), bytes * threads, xp, ldx, bp, ldb, sp, lds, g, bias, eps, yp, ldy, mean, rstd, rows, cols,
                    s.tpr);
    return (int)cudaGetLastError();
  };
  if (s.vpt == 1) return bp ? launch(layernorm_kernel<1, true>, RING_BYTES<1, 2>) : launch(layernorm_kernel<1, false>, RING_BYTES<1, 1>);
  if (s.vpt == 2) return bp ? launch(layernorm_kernel<2, true>, RING_BYTES<2, 2>) : launch(layernorm_kernel<2, false>, RING_BYTES<2, 1>);
  return bp ? launch(layernorm_kernel<4, true>, RING_BYTES<4, 2>) : launch(layernorm_kernel<4, false>, RING_BYTES<4, 1>);
}

int faar_launch_layernorm_bwd(faar_ctx* ctx, int rows, int cols, const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* g,
                              const float* mean, const float* rstd, const void* add, int64_t ldadd, void* dx, int64_t lddx, float* dg,
                              float* db, float* partials) {
  faar_prof_scope ps(ctx, FAAR_K_GLUE);
  const Shape s = shape(ctx, rows, cols);
  if (!dg && !db) partials = nullptr;
  auto launch = [&](auto* kernel, int bytes) {
    const int e = faar_allow_smem(ctx, (const void*)kernel, bytes * MAX_THREADS);
    if (e) return e;
    const int threads = s.tpr * s.groups;
    faar_launch_pdl(ctx, kernel, dim3(s.ctas), dim3(threads), bytes * threads, reinterpret_cast<const __nv_bfloat16*>(dy), lddy,
                    reinterpret_cast<const __nv_bfloat16*>(x), ldx, g, mean, rstd, reinterpret_cast<const __nv_bfloat16*>(add), ldadd,
                    reinterpret_cast<__nv_bfloat16*>(dx), lddx, partials, rows, cols, s.tpr);
    return (int)cudaGetLastError();
  };
  int e;
  if (s.vpt == 1) e = add ? launch(layernorm_bwd_kernel<1, true>, RING_BYTES<1, 3>) : launch(layernorm_bwd_kernel<1, false>, RING_BYTES<1, 2>);
  else if (s.vpt == 2) e = add ? launch(layernorm_bwd_kernel<2, true>, RING_BYTES<2, 3>) : launch(layernorm_bwd_kernel<2, false>, RING_BYTES<2, 2>);
  else e = add ? launch(layernorm_bwd_kernel<4, true>, RING_BYTES<4, 3>) : launch(layernorm_bwd_kernel<4, false>, RING_BYTES<4, 2>);
  if (e || !partials) return e;
  faar_launch_pdl(ctx, layernorm_dw_sum_kernel, dim3((2 * cols + 31) / 32), dim3(32, 32), 0, (const float*)partials, s.ctas, dg, db, cols);
  return (int)cudaGetLastError();
}
