// Layer norm over the rows of x [T, D], the step in front of a block's linears:
//   forward   m = mean(x), v = mean((x - m)^2), r = 1 / sqrt(v + eps), y = (x - m) r gamma + beta, optionally with the checkpoint of x
//   backward  xh = (x - m) r, h = dy gamma:  dx = r (h - mean(h) - xh mean(h xh)),  dgamma = sum_t dy xh,  dbeta = sum_t dy
// with x itself or its 8-bit checkpoint in backward. One pass over memory each: a group of TPR threads holds a row in registers, eight
// neighbouring elements at a time, so that mean, centred squares and result need x once. Groups walk over rows and load the next row while they
// work on this one; the parameters stay in registers (forward) or, as FP32, in shared memory (backward, whose registers hold the two sums of
// the thread's columns). At the end the groups of a CTA add their column sums up in shared memory, the CTAs through a small FP32 matrix that a
// second launch sums. Every sum has a fixed order.
//
// Measured (us, inputs from HBM, replayed from a graph; in brackets the share of the copy bandwidth), forward / backward: 16384 x 1024 BF16 14.1
// (0.73) / 23.5 (0.66), with the checkpoint 17.6 (0.74) / 22.2 (0.58), 4096 x 4096 so 19.1 (0.68) / 23.6 (0.55), 2048 x 8192 so 20.7 (0.62) / 26.3
// (0.49), FP32 4095 x 4096 19.4 (0.80) / 34.3 (0.75). A row's chain through its sums bounds it, at 0.54 of the issue slots with a quarter of an
// SM's warps; of backward about 4 us are the second launch. Registers decide the rest: forward gains from warps (FP32 4095 x 4096 22.2 with 512
// threads on an SM, 19.6 with 1024), backward loses more by spilling than they bring (16384 x 1024 23.6 with 128 registers, 52 with 85), and a
// row in one warp there holds too many sums (41.7). Where shapes spill it shows (2^24 elements as rows of so many columns, with the checkpoint):
//   columns             1024   1500 (rows cut short)  2048   2816   4096   5120   8192   12288   16384
//   BF16 forward        15.7   35.5                   18.8   20.6   18.8   22.5   20.0   22.4    38.2
//   FP32 forward        24.2   36.1                   20.8   37.6   21.9   40.9   23.3   40.1    56.2
//   BF16 backward       21.9   36.7                   22.5   25.9   23.5   28.7   26.2   35.8    54.2
#include "../../include/nvfp4.h"

#include "act8.cuh"
#include "nvfp4_internal.h"

namespace nvfp4 {

namespace {

constexpr int kMaxD = 16384;  // TPR 512, four vectors of eight a thread
// Backward: threads of a CTA (one per SM, 128 registers each) and CTAs, at most. Tuning constants, not hardware queries: the workspace size
// derived from them must not depend on the device.
constexpr int kBwdThreads = 512, kBwdCtas = 148;

template <int TPR>
constexpr int kFwdThreadsOf = TPR < 128 ? 128 : TPR;  // of a CTA
// Forward's threads per SM, and so its registers a thread: 1024 threads have 64, 640 have 96. Shapes of three vectors (1025 to 1536, 2049 to 3072,
// 4097 to 6144 columns) spill at 64, with BF16 rows 8 to 80 bytes, with FP32 rows 24 to 172, and the largest of four up to 276: see the times.
template <int NV, int TPR>
constexpr int kFwdThreadsPerSm = TPR == 32 && NV > 2 ? 640 : 1024;

constexpr int kSlots = kBwdThreads / 32;  // of group_sum2, one set

// eight parameters from column c on, 0 past D
__device__ __forceinline__ void params8(const void* p, int f32, int c, int D, f32x2 (&v)[4]) {
  if (f32) {
    Raw8<kSrcF32> r;
    load_f32x8(static_cast<const float*>(p), c, D, r.lo, r.hi);
    values8(r, v);
  } else {
    values8(Raw8<kSrcBf16>{load_bf16x8(static_cast<const uint16_t*>(p), c, D)}, v);
  }
}

template <int TPR>
__device__ __forceinline__ void group_barrier(int group) {
  if constexpr (TPR == 512)  // (the whole CTA)
    __syncthreads();
  else
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(TPR) : "memory");
}
// Sum over the group's threads, in all of them. `slot`: shared memory that no thread of the group may still be reading from an earlier call
// (calls alternate between two, a barrier in each).
template <int TPR>
__device__ __forceinline__ float group_sum(float v, float* slot, int group, int lane) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  if constexpr (TPR > 32) {
    if ((lane & 31) == 0) slot[lane >> 5] = v;
    group_barrier<TPR>(group);
    v = slot[0];
#pragma unroll
    for (int w = 1; w < TPR / 32; ++w) v += slot[w];
  }
  return v;
}
// Two sums at once: the half warps exchange, so that each adds up one of the two.
template <int TPR>
__device__ __forceinline__ float2 group_sum2(float x, float y, float2* slot, int group, int lane) {
  const bool upper = lane & 16;
  float v = (upper ? y : x) + __shfl_xor_sync(0xFFFFFFFFu, upper ? x : y, 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  if constexpr (TPR > 32) {
    if ((lane & 15) == 0) reinterpret_cast<float*>(slot)[lane >> 4] = v;
    group_barrier<TPR>(group);
    float2 s = slot[0];
#pragma unroll
    for (int w = 1; w < TPR / 32; ++w) {
      s.x += slot[w].x;
      s.y += slot[w].y;
    }
    return s;
  } else {
    const float other = __shfl_xor_sync(0xFFFFFFFFu, v, 16);
    return upper ? make_float2(other, v) : make_float2(v, other);
  }
}

__device__ __forceinline__ void store_grad(void* out, int f32, int c, float v) {  // (a gradient of a parameter may lie on any address of its type)
  if (f32)
    static_cast<float*>(out)[c] = v;
  else
    static_cast<uint16_t*>(out)[c] = (uint16_t)bf16x2_of(v, 0.0f);
}

struct NormFwdArgs {
  ActSrc x;
  int64_t T;
  int D, params_f32;
  const void *gamma, *beta;
  float eps;
  uint16_t* y;
  int64_t ldy;
  float2* stats;  // (m, r) of a row; optional
  uint8_t *codes, *scales;
};

// FULL: D is a multiple of eight, so that no piece of eight is cut short (1999 x 1000 forward 5.0 us against 5.5).
template <int SRC, bool CK, int NV, int TPR, bool FULL>
__global__ void __launch_bounds__(kFwdThreadsOf<TPR>, kFwdThreadsPerSm<NV, TPR> / kFwdThreadsOf<TPR>) norm_fwd_kernel(NormFwdArgs a) {
  pdl_prologue();
  constexpr int GROUPS = kFwdThreadsOf<TPR> / TPR;
  __shared__ float slots[2][GROUPS][TPR / 32];
  extern __shared__ __align__(16) uint8_t smem[];
  ulonglong2* const params = reinterpret_cast<ulonglong2*>(smem);  // [gamma, beta][NV][2][TPR], four values each
  const int group = threadIdx.x / TPR, lane = threadIdx.x % TPR, D = a.D, ldc = (D + 31) & ~31;
  const float inv_D = 1.0f / (float)D;
  const f32x2 minus_one = pair_of(-1.0f);
  Raw8<SRC> next[NV];
  int64_t row = (int64_t)blockIdx.x * GROUPS + group;
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  // this thread's first elements of its rows; the pointers move from row to row
  constexpr int SIZE = SRC == kSrcF32 ? 4 : 2;
  const uint8_t* x = static_cast<const uint8_t*>(a.x.p) + (row * a.x.ld + lane * 8) * SIZE;
  uint16_t* y = a.y + row * a.ldy + lane * 8;
  uint8_t *codes = CK ? a.codes + row * ldc + lane * 8 : nullptr, *scales = CK ? a.scales + row * (ldc >> 5) + (lane >> 2) : nullptr;
  const int64_t x_step = step * a.x.ld * SIZE, y_step = step * a.ldy, c_step = step * ldc, s_step = step * (ldc >> 5);
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + lane) * 8;
      next[i] = Raw8<SRC>{};
      if (c < D && row < a.T) next[i] = load8_at<SRC>(x + (size_t)i * TPR * 8 * SIZE, nullptr, FULL ? 8 : D - c);
    }
    x += x_step;
  };
  fetch(row);
  for (int j = group; j < 2 * NV; j += GROUPS) {
    const int c = ((j >> 1) * TPR + lane) * 8;
    f32x2 p[4] = {};
    if (c < D && (j & 1) == 0) params8(a.gamma, a.params_f32, c, D, p);
    if (c < D && (j & 1) && a.beta) params8(a.beta, a.params_f32, c, D, p);
#pragma unroll
    for (int e = 0; e < 2; ++e) params[(((j & 1) * NV + (j >> 1)) * 2 + e) * TPR + lane] = make_ulonglong2(p[2 * e], p[2 * e + 1]);
  }
  __syncthreads();
  for (; row < a.T; row += step) {
    f32x2 v[NV][4];
    float amax[NV];
    f32x2 sum = pair_of(0.0f);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      values8(next[i], v[i]);
      if (CK) amax[i] = amax8(next[i]);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum = add2(sum, v[i][e]);
    }
    fetch(row + step);
    if (CK) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + lane) * 8;
        ckpt8_store(v[i], amax[i], codes + i * TPR * 8, scales + i * TPR / 4, (lane & 3) == 0, c < ldc);
      }
      codes += c_step;
      scales += s_step;
    }
    const float mean = group_sum<TPR>(sum_of(sum), slots[0][group], group, lane) * inv_D;
    f32x2 sq = pair_of(0.0f);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + lane) * 8;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i][e] = fma2(minus_one, pair_of(mean), v[i][e]);  // x - m, rounded once
      if (c + 8 <= D) {
#pragma unroll
        for (int e = 0; e < 4; ++e) sq = fma2(v[i][e], v[i][e], sq);
      } else if (!FULL) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 d = values_of(v[i][e]);
          sq = add2(sq, pair_of(c + 2 * e < D ? d.x * d.x : 0.0f, c + 2 * e + 1 < D ? d.y * d.y : 0.0f));
        }
      }
    }
    const float var = group_sum<TPR>(sum_of(sq), slots[1][group], group, lane) * inv_D;
    const float rstd = rsqrtf(var + a.eps);  // (off by 2 units in the last place at most)
    if (a.stats && lane == 0) a.stats[row] = make_float2(mean, rstd);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + lane) * 8;
      if (c >= D) continue;
      f32x2 o[4];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const ulonglong2 g = params[(i * 2 + e) * TPR + lane], b = params[((NV + i) * 2 + e) * TPR + lane];
        o[2 * e] = fma2(mul2(v[i][2 * e], pair_of(rstd)), g.x, b.x);
        o[2 * e + 1] = fma2(mul2(v[i][2 * e + 1], pair_of(rstd)), g.y, b.y);
      }
      store_bf16x8(y + i * TPR * 8, 0, FULL ? 8 : D - c, o);
    }
    y += y_step;
  }
}

struct NormBwdArgs {
  ActSrc dy, x;
  int64_t T;
  int D, params_f32, dx_f32, has_beta;
  const void* gamma;
  const float2* stats;
  void* dx;
  int64_t lddx;
  float* partial;  // [CTA][dgamma, dbeta][columns up to a multiple of 8]; unused by a single CTA, which writes the gradients
  void *dgamma, *dbeta;
  int grads_f32;
};

template <int SRC, int NV, int TPR, bool FULL>
__global__ void __launch_bounds__(kBwdThreads, 1) norm_bwd_kernel(NormBwdArgs a) {
  pdl_prologue();
  constexpr int GROUPS = kBwdThreads / TPR;
  extern __shared__ __align__(16) uint8_t smem[];
  const int group = threadIdx.x / TPR, lane = threadIdx.x % TPR, D = a.D;
  float2* const slots = reinterpret_cast<float2*>(smem) + group * (TPR / 32);  // and again kSlots further on
  ulonglong2* const gamma = reinterpret_cast<ulonglong2*>(reinterpret_cast<f32x2*>(smem) + 2 * kSlots);  // [NV][2][TPR], four values each
  f32x2* const sums = reinterpret_cast<f32x2*>(gamma);                            // and at the end, GROUPS / 2 times [dgamma, dbeta][NV][4][TPR]
  const float inv_D = 1.0f / (float)D;
  Raw8<kSrcBf16> dy_next[NV];
  Raw8<SRC> x_next[NV];
  float2 st_next = make_float2(0.0f, 0.0f);
  int64_t row = (int64_t)blockIdx.x * GROUPS + group;
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  // this thread's first elements of its rows; the pointers move from row to row
  constexpr int SIZE = SRC == kSrcF32 ? 4 : SRC == kSrcBf16 ? 2 : 1;
  const uint8_t* dy = static_cast<const uint8_t*>(a.dy.p) + (row * a.dy.ld + lane * 8) * 2;
  const uint8_t* x = static_cast<const uint8_t*>(a.x.p) + (row * a.x.ld + lane * 8) * SIZE;
  const uint8_t* scales = SRC == kSrcCkpt8 ? a.x.scales + row * (a.x.ld >> 5) + (lane >> 2) : nullptr;
  const float2* stats = a.stats + row;
  const int dx_size = a.dx_f32 ? 4 : 2;
  uint8_t* dx = static_cast<uint8_t*>(a.dx) + (row * a.lddx + lane * 8) * dx_size;
  const int64_t dy_step = step * a.dy.ld * 2, x_step = step * a.x.ld * SIZE, s_step = step * (a.x.ld >> 5), dx_step = step * a.lddx * dx_size;
  auto fetch = [&](int64_t row) {
    if (row >= a.T) return;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + lane) * 8;
      dy_next[i] = Raw8<kSrcBf16>{};
      x_next[i] = Raw8<SRC>{};
      if (c < D) {
        dy_next[i] = load8_at<kSrcBf16>(dy + i * TPR * 16, nullptr, FULL ? 8 : D - c);
        x_next[i] = load8_at<SRC>(x + i * TPR * 8 * SIZE, SRC == kSrcCkpt8 ? scales + i * TPR / 4 : nullptr, FULL ? 8 : D - c);
      }
    }
    st_next = *stats;
    dy += dy_step;
    x += x_step;
    if (SRC == kSrcCkpt8) scales += s_step;
    stats += step;
  };
  fetch(row);
  if (group == 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + lane) * 8;
      f32x2 g[4] = {};
      if (c < D) params8(a.gamma, a.params_f32, c, D, g);
#pragma unroll
      for (int e = 0; e < 2; ++e) gamma[(i * 2 + e) * TPR + lane] = make_ulonglong2(g[2 * e], g[2 * e + 1]);
    }
  }
  __syncthreads();
  f32x2 dg[NV][4] = {}, db[NV][4] = {};
  const f32x2 minus_one = pair_of(-1.0f);
  int parity = 0;
  for (; row < a.T; row += step, parity ^= 1) {
    f32x2 h[NV][4], xh[NV][4], s1 = pair_of(0.0f), s2 = s1;  // (past D dy and gamma are 0)
    const float2 st = st_next;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      values8(dy_next[i], h[i]);
      if constexpr (SRC == kSrcCkpt8) {  // code * (scale r) - m r: one rounding of 2^-24 of m r and one of the result
        ckpt8_decode(x_next[i].q, xh[i]);
        const f32x2 k = pair_of(ckpt8_scale(x_next[i].byte) * st.y), c = pair_of(-(st.x * st.y));
#pragma unroll
        for (int e = 0; e < 4; ++e) xh[i][e] = fma2(xh[i][e], k, c);
      } else {
        values8(x_next[i], xh[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) xh[i][e] = mul2(fma2(minus_one, pair_of(st.x), xh[i][e]), pair_of(st.y));
      }
    }
    fetch(row + step);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if ((i * TPR + lane) * 8 >= D) continue;
      const ulonglong2 g01 = gamma[i * 2 * TPR + lane], g23 = gamma[(i * 2 + 1) * TPR + lane];
      const f32x2 gam[4] = {g01.x, g01.y, g23.x, g23.y};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        dg[i][e] = fma2(h[i][e], xh[i][e], dg[i][e]);
        db[i][e] = add2(h[i][e], db[i][e]);
        h[i][e] = mul2(h[i][e], gam[e]);
        s1 = add2(s1, h[i][e]);
        s2 = fma2(h[i][e], xh[i][e], s2);
      }
    }
    const float2 s = group_sum2<TPR>(sum_of(s1), sum_of(s2), slots + parity * kSlots, group, lane);
    const f32x2 c1 = pair_of(-(s.x * inv_D)), c2 = pair_of(-(s.y * inv_D)), r = pair_of(st.y);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + lane) * 8;
      if (c >= D) continue;
      f32x2 o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = mul2(add2(fma2(xh[i][e], c2, h[i][e]), c1), r);
      if (a.dx_f32)
        store_f32x8(reinterpret_cast<float*>(dx) + i * TPR * 8, 0, FULL ? 8 : D - c, o);
      else
        store_bf16x8(reinterpret_cast<uint16_t*>(dx) + i * TPR * 8, 0, FULL ? 8 : D - c, o);
    }
    dx += dx_step;
  }
  // the groups' sums: the upper half of them adds to the lower one until one is left
  __syncthreads();  // (gamma is done with)
#pragma unroll
  for (int half = GROUPS / 2; half > 0; half >>= 1) {
    f32x2* mine = sums + (size_t)(group - (group >= half ? half : 0)) * (2 * NV * 4 * TPR) + lane;
    if (group >= half && group < 2 * half) {
#pragma unroll
      for (int i = 0; i < NV * 4; ++i) {
        mine[i * TPR] = dg[i >> 2][i & 3];
        mine[(NV * 4 + i) * TPR] = db[i >> 2][i & 3];
      }
    }
    __syncthreads();
    if (group < half) {
#pragma unroll
      for (int i = 0; i < NV * 4; ++i) {
        dg[i >> 2][i & 3] = add2(dg[i >> 2][i & 3], mine[i * TPR]);
        db[i >> 2][i & 3] = add2(db[i >> 2][i & 3], mine[(NV * 4 + i) * TPR]);
      }
    }
    __syncthreads();
  }
  if (group != 0) return;
  if (gridDim.x == 1) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + lane) * 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (c + e >= D) continue;
        const float2 g = values_of(dg[i][e >> 1]), b = values_of(db[i][e >> 1]);
        store_grad(a.dgamma, a.grads_f32, c + e, e & 1 ? g.y : g.x);
        if (a.has_beta) store_grad(a.dbeta, a.grads_f32, c + e, e & 1 ? b.y : b.x);
      }
    }
    return;
  }
  const int Dp = (D + 7) & ~7;
  float* out = a.partial + (size_t)blockIdx.x * 2 * Dp;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * TPR + lane) * 8;
    if (c >= D) continue;
    store_f32x8(out, c, Dp, dg[i]);
    if (a.has_beta) store_f32x8(out + Dp, c, Dp, db[i]);
  }
}

// Column sums of the CTAs' partial sums: a CTA takes 32 columns of one of the two, each of its warps every n-th row, then the warps' sums of
// a column are added in order.
__global__ void __launch_bounds__(1024) norm_bwd_finish_kernel(const float* __restrict__ partial, int rows, int D, int f32, void* __restrict__ dgamma,
                                                              void* __restrict__ dbeta) {
  pdl_prologue();
  __shared__ float red[32][32];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, Dp = (D + 7) & ~7;
  constexpr int PER = (kBwdCtas + 31) / 32;  // rows of a warp, at most: all loads at once
  float v[PER], s = 0.0f;
#pragma unroll
  for (int k = 0; k < PER; ++k) v[k] = c < D && wid + 32 * k < rows ? partial[((size_t)(wid + 32 * k) * 2 + blockIdx.y) * Dp + c] : 0.0f;
#pragma unroll
  for (int k = 0; k < PER; ++k) s += v[k];
  red[wid][lane] = s;
  __syncthreads();
  if (wid != 0 || c >= D) return;
  float t = 0.0f;
#pragma unroll
  for (int w = 0; w < 32; ++w) t += red[w][lane];
  store_grad(blockIdx.y ? dbeta : dgamma, f32, c, t);
}

template <int N>
using Int = std::integral_constant<int, N>;

// The shape of a row's group, as (vectors of eight a thread, threads): as few threads as hold the row in three vectors each, in up to four vectors
// up to 1024 elements, which one warp holds, so that most rows need no barrier, and in the largest rows.
template <typename F>
auto with_fwd_shape(int D, F&& f) {
  const int n8 = (D + 7) / 8;
  if (n8 <= 32) return f(Int<1>{}, Int<32>{});
  if (n8 <= 64) return f(Int<2>{}, Int<32>{});
  if (n8 <= 96) return f(Int<3>{}, Int<32>{});
  if (n8 <= 128) return f(Int<4>{}, Int<32>{});
  if (n8 <= 192) return f(Int<3>{}, Int<64>{});
  if (n8 <= 256) return f(Int<2>{}, Int<128>{});
  if (n8 <= 384) return f(Int<3>{}, Int<128>{});
  if (n8 <= 512) return f(Int<2>{}, Int<256>{});
  if (n8 <= 768) return f(Int<3>{}, Int<256>{});
  if (n8 <= 1024) return f(Int<2>{}, Int<512>{});
  if (n8 <= 1536) return f(Int<3>{}, Int<512>{});
  return f(Int<4>{}, Int<512>{});
}

// Backward's: in two vectors, since its registers hold the columns' sums too, more in the largest rows.
template <typename F>
auto with_bwd_shape(int D, F&& f) {
  const int n8 = (D + 7) / 8;
  if (n8 <= 32) return f(Int<1>{}, Int<32>{});
  if (n8 <= 64) return f(Int<2>{}, Int<32>{});
  if (n8 <= 128) return f(Int<2>{}, Int<64>{});
  if (n8 <= 256) return f(Int<2>{}, Int<128>{});
  if (n8 <= 512) return f(Int<2>{}, Int<256>{});
  if (n8 <= 1024) return f(Int<2>{}, Int<512>{});
  if (n8 <= 1536) return f(Int<3>{}, Int<512>{});
  return f(Int<4>{}, Int<512>{});
}

template <int SRC, bool CK>
cudaError_t launch_norm_fwd(const NormFwdArgs& a, cudaStream_t st) {
  return with_fwd_shape(a.D, [&](auto nv, auto tpr) {
    constexpr int NV = decltype(nv)::value, TPR = decltype(tpr)::value, THREADS = kFwdThreadsOf<TPR>, GROUPS = THREADS / TPR;
    constexpr size_t smem = (size_t)2 * NV * 2 * TPR * sizeof(ulonglong2);
    auto kernel = a.D % 8 ? norm_fwd_kernel<SRC, CK, NV, TPR, false> : norm_fwd_kernel<SRC, CK, NV, TPR, true>;
    const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), smem + 1024);
    if (e != cudaSuccess) return e;
    const int64_t ctas = std::min<int64_t>((a.T + GROUPS - 1) / GROUPS, (int64_t)device_sm_count() * (kFwdThreadsPerSm<NV, TPR> / THREADS));
    return launch_kernel(kernel, dim3((unsigned)ctas), dim3(THREADS), smem, st, a);
  });
}

int bwd_ctas(int64_t T, int D) {
  return with_bwd_shape(D, [&](auto, auto tpr) {
    constexpr int GROUPS = kBwdThreads / decltype(tpr)::value;
    // (up to two rows a group, one CTA without the second launch: us from Python, 16 x 1024 7.4 against 10.8)
    return T <= 2 * GROUPS ? 1 : (int)std::min<int64_t>((T + GROUPS - 1) / GROUPS, kBwdCtas);
  });
}

template <int SRC>
cudaError_t launch_norm_bwd(const NormBwdArgs& a, int ctas, cudaStream_t st) {
  return with_bwd_shape(a.D, [&](auto nv, auto tpr) {
    constexpr int NV = decltype(nv)::value, TPR = decltype(tpr)::value, GROUPS = kBwdThreads / TPR;
    constexpr size_t smem = (2 * kSlots + (size_t)GROUPS * NV * 4 * TPR) * sizeof(f32x2);  // slots; gamma, or the sums of half the groups
    auto kernel = a.D % 8 ? norm_bwd_kernel<SRC, NV, TPR, false> : norm_bwd_kernel<SRC, NV, TPR, true>;
    const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), smem);
    if (e != cudaSuccess) return e;
    return launch_kernel(kernel, dim3((unsigned)ctas), dim3(kBwdThreads), smem, st, a);
  });
}

}  // namespace

}  // namespace nvfp4

using namespace nvfp4;

extern "C" {

nvfp4_status nvfp4_layernorm_fwd(const void* X, int32_t x_dtype, int64_t ldx, int64_t T, int64_t D, const void* gamma, const void* beta, int32_t param_dtype,
                                 float eps, void* Y, int64_t ldy, float* stats, const nvfp4_ckpt8* x8, void* stream) {
  if (x_dtype < 0 || x_dtype > 1 || param_dtype < 0 || param_dtype > 1) return NVFP4_ERR_ENUM;
  if (T < 0 || D <= 0 || !(eps >= 0.0f)) return NVFP4_ERR_SHAPE;
  if (D > kMaxD || T > 0x7FFFFFFF) return NVFP4_ERR_LIMIT;
  nvfp4_status s;
  if (x8 && (s = check_ckpt8(x8, T, D)) != NVFP4_OK) return s;
  if (T == 0) return NVFP4_OK;
  if (!X || !gamma || !Y) return NVFP4_ERR_NULL;
  if (bad_matrix(X, ldx, D, x_dtype == NVFP4_DT_F32 ? 4 : 2) || bad_matrix(Y, ldy, D, 2) || !aligned(gamma, 16) || !aligned(beta, 16) || !aligned(stats, 8))
    return NVFP4_ERR_ALIGN;
  if (!device_is_sm100()) return NVFP4_ERR_ARCH;
  NormFwdArgs a{};
  a.x = ActSrc{X, nullptr, ldx};
  a.T = T;
  a.D = (int)D;
  a.params_f32 = param_dtype == NVFP4_DT_F32;
  a.gamma = gamma;
  a.beta = beta;
  a.eps = eps;
  a.y = static_cast<uint16_t*>(Y);
  a.ldy = ldy;
  a.stats = reinterpret_cast<float2*>(stats);
  if (x8) {
    a.codes = x8->codes;
    a.scales = x8->scales;
  }
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = x_dtype == NVFP4_DT_F32 ? (x8 ? launch_norm_fwd<kSrcF32, true>(a, st) : launch_norm_fwd<kSrcF32, false>(a, st))
                                                : (x8 ? launch_norm_fwd<kSrcBf16, true>(a, st) : launch_norm_fwd<kSrcBf16, false>(a, st));
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? NVFP4_OK : NVFP4_ERR_CUDA;
}

size_t nvfp4_layernorm_bwd_workspace_bytes(int64_t T, int64_t D) {
  if (T <= 0 || D <= 0 || D > kMaxD) return 256;
  return (size_t)bwd_ctas(T, (int)D) * 2 * ((D + 7) / 8 * 8) * sizeof(float);
}

nvfp4_status nvfp4_layernorm_bwd(const void* dY, int64_t lddy, const void* X, int32_t x_dtype, int64_t ldx, const nvfp4_ckpt8* x8, int64_t T, int64_t D,
                                 const void* gamma, int32_t param_dtype, const float* stats, void* dX, int64_t lddx, void* dgamma, void* dbeta,
                                 int32_t dparam_dtype, void* workspace, size_t ws_bytes, void* stream) {
  if (x_dtype < 0 || x_dtype > 1 || param_dtype < 0 || param_dtype > 1 || dparam_dtype < 0 || dparam_dtype > 1) return NVFP4_ERR_ENUM;
  if (T < 0 || D <= 0) return NVFP4_ERR_SHAPE;
  if (D > kMaxD || T > 0x7FFFFFFF) return NVFP4_ERR_LIMIT;
  nvfp4_status s;
  if (x8 && (s = check_ckpt8(x8, T, D)) != NVFP4_OK) return s;
  if (!gamma || !dgamma || (T > 0 && (!dY || (!x8 && !X) || !stats || !dX))) return NVFP4_ERR_NULL;
  const int dx_bytes = x_dtype == NVFP4_DT_F32 ? 4 : 2, dp_align = dparam_dtype == NVFP4_DT_F32 ? 4 : 2;
  if ((T > 0 && (bad_matrix(dY, lddy, D, 2) || bad_matrix(dX, lddx, D, dx_bytes) || (!x8 && bad_matrix(X, ldx, D, dx_bytes)) || !aligned(stats, 8))) || !aligned(gamma, 16) ||
      !aligned(dgamma, dp_align) || !aligned(dbeta, dp_align))
    return NVFP4_ERR_ALIGN;
  if (!workspace || !aligned(workspace, 16) || ws_bytes < nvfp4_layernorm_bwd_workspace_bytes(T, D)) return NVFP4_ERR_WORKSPACE;
  if (!device_is_sm100()) return NVFP4_ERR_ARCH;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int ctas = bwd_ctas(T, (int)D);
  if (T > 0) {
    NormBwdArgs a{};
    a.dy = ActSrc{dY, nullptr, lddy};
    a.x = x8 ? ActSrc{x8->codes, x8->scales, (D + 31) / 32 * 32} : ActSrc{X, nullptr, ldx};
    a.T = T;
    a.D = (int)D;
    a.params_f32 = param_dtype == NVFP4_DT_F32;
    a.dx_f32 = x_dtype == NVFP4_DT_F32;
    a.has_beta = dbeta != nullptr;
    a.gamma = gamma;
    a.stats = reinterpret_cast<const float2*>(stats);
    a.dx = dX;
    a.lddx = lddx;
    a.partial = static_cast<float*>(workspace);
    a.dgamma = dgamma;
    a.dbeta = dbeta;
    a.grads_f32 = dparam_dtype == NVFP4_DT_F32;
    const cudaError_t e = x8 ? launch_norm_bwd<kSrcCkpt8>(a, ctas, st)
                             : x_dtype == NVFP4_DT_F32 ? launch_norm_bwd<kSrcF32>(a, ctas, st) : launch_norm_bwd<kSrcBf16>(a, ctas, st);
    if (e != cudaSuccess || cudaGetLastError() != cudaSuccess) return NVFP4_ERR_CUDA;
    if (ctas == 1) return NVFP4_OK;
  }
  launch_kernel(norm_bwd_finish_kernel, dim3((unsigned)((D + 31) / 32), dbeta ? 2u : 1u), dim3(1024), 0, st, static_cast<const float*>(workspace), T > 0 ? ctas : 0, (int)D,
                (int)(dparam_dtype == NVFP4_DT_F32), dgamma, dbeta);
  return cudaGetLastError() == cudaSuccess ? NVFP4_OK : NVFP4_ERR_CUDA;
}

}  // extern "C"
