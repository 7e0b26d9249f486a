// Layer norm over the rows of x [T, D], the step in front of a block's linears:
//   forward   m = mean(x), v = mean((x - m)^2), r = 1 / sqrt(v + eps), y = (x - m) r gamma + beta, optionally with the checkpoint of x
//   backward  xh = (x - m) r, h = dy gamma:  dx = r (h - mean(h) - xh mean(h xh)),  dgamma = sum_t dy xh,  dbeta = sum_t dy
// with x itself or its 8-bit checkpoint in backward. One pass over memory each: a group of TPR threads holds a whole row in registers, eight
// neighbouring elements at a time, so that mean, centred squares and result need x once. Backward's groups walk over rows and keep the two
// column sums of their columns in registers; the groups of a CTA add theirs up in shared memory, the CTAs through a small FP32 matrix that a
// second launch sums. Every sum has a fixed order.
#include "../../include/nvfp4.h"

#include "act8.cuh"
#include "nvfp4_internal.h"

namespace nvfp4 {

namespace {

constexpr int kMaxD = 16384;  // TPR 512, four vectors of eight a thread
// CTAs of backward, at most. A tuning constant, not a hardware query: the workspace size derived from it must not depend on the device.
constexpr int kBwdCtas = 592;

template <int TPR>
constexpr int kThreadsOf = TPR < 256 ? 256 : TPR;  // of a CTA

// eight parameters from column c on, 0 past D
__device__ __forceinline__ void params8(const void* p, int f32, int c, int D, float (&v)[8]) {
  if (f32) {
    Raw8<kSrcF32> r;
    load_f32x8(static_cast<const float*>(p), c, D, r.lo, r.hi);
    values8(r, v);
  } else {
    bf16x8_values(load_bf16x8(static_cast<const uint16_t*>(p), c, D), v);
  }
}

template <int TPR>
__device__ __forceinline__ void group_barrier(int group) {
  if constexpr (kThreadsOf<TPR> == TPR)
    __syncthreads();
  else
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(TPR) : "memory");
}
// Sums of two values over the group's threads, in all of them. `slot`: shared memory that no thread of the group may still be reading from
// an earlier call (calls alternate between two, a barrier in each).
template <int TPR>
__device__ __forceinline__ float2 group_sum2(float2 v, float2* slot, int group, int lane) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, o);
    v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, o);
  }
  if constexpr (TPR > 32) {
    if ((lane & 31) == 0) slot[lane >> 5] = v;
    group_barrier<TPR>(group);
    v = slot[0];
#pragma unroll
    for (int w = 1; w < TPR / 32; ++w) {
      v.x += slot[w].x;
      v.y += slot[w].y;
    }
  }
  return v;
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

template <int SRC, bool CK, int NV, int TPR>
__global__ void __launch_bounds__(kThreadsOf<TPR>) norm_fwd_kernel(NormFwdArgs a) {
  pdl_prologue();
  constexpr int GROUPS = kThreadsOf<TPR> / TPR;
  __shared__ float2 slots[2][GROUPS][TPR / 32];
  const int group = threadIdx.x / TPR, lane = threadIdx.x % TPR, D = a.D;
  const int64_t row = (int64_t)blockIdx.x * GROUPS + group;
  if (row >= a.T) return;  // (the whole group)
  float v[NV][8];
  float sum = 0.0f;
  {
    Raw8<SRC> raw[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + lane) * 8;
      if (c < D) raw[i] = load8<SRC>(a.x, row, c, D);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + lane) * 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = 0.0f;
      if (c < D) values8(raw[i], v[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += v[i][e];
    }
  }
  const float inv_D = 1.0f / (float)D;
  const float mean = group_sum2<TPR>(make_float2(sum, 0.0f), slots[0][group], group, lane).x * inv_D;
  float sq = 0.0f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * TPR + lane) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = v[i][e] - mean;
      if (c + e < D) sq = fmaf(d, d, sq);
    }
  }
  const float var = group_sum2<TPR>(make_float2(sq, 0.0f), slots[1][group], group, lane).x * inv_D;
  const float rstd = 1.0f / sqrtf(var + a.eps);
  if (a.stats && lane == 0) a.stats[row] = make_float2(mean, rstd);
  const int ldc = (D + 31) & ~31;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * TPR + lane) * 8;
    if (CK) ckpt8_store(v[i], a.codes + row * ldc, a.scales + row * (ldc >> 5), c, c < ldc);
    if (c < D) {
      float g[8], b[8] = {}, o[8];
      params8(a.gamma, a.params_f32, c, D, g);
      if (a.beta) params8(a.beta, a.params_f32, c, D, b);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = fmaf((v[i][e] - mean) * rstd, g[e], b[e]);
      store_bf16x8(a.y + row * a.ldy, c, D, o);
    }
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
  float* partial;  // [CTA][dgamma, dbeta][columns up to a multiple of 8]
};

template <int SRC, int NV, int TPR>
__global__ void __launch_bounds__(kThreadsOf<TPR>) norm_bwd_kernel(NormBwdArgs a) {
  pdl_prologue();
  constexpr int GROUPS = kThreadsOf<TPR> / TPR;
  __shared__ float2 slots[2][GROUPS][TPR / 32];
  extern __shared__ float sums[];  // GROUPS / 2 times [dgamma, dbeta][NV][8][TPR]
  const int group = threadIdx.x / TPR, lane = threadIdx.x % TPR, D = a.D;
  const float inv_D = 1.0f / (float)D;
  float dg[NV][8] = {}, db[NV][8] = {};
  int parity = 0;
  for (int64_t row = (int64_t)blockIdx.x * GROUPS + group; row < a.T; row += (int64_t)gridDim.x * GROUPS, parity ^= 1) {
    Raw8<kSrcBf16> dyr[NV];
    Raw8<SRC> xr[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + lane) * 8;
      if (c < D) {
        dyr[i] = load8<kSrcBf16>(a.dy, row, c, D);
        xr[i] = load8<SRC>(a.x, row, c, D);
      }
    }
    const float2 st = a.stats[row];
    float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + lane) * 8;
      if (c >= D) continue;
      float dy[8], x[8], g[8];
      values8(dyr[i], dy);
      values8(xr[i], x);
      params8(a.gamma, a.params_f32, c, D, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) {  // (past D dy and gamma are 0)
        const float xh = (x[e] - st.x) * st.y, h = dy[e] * g[e];
        dg[i][e] = fmaf(dy[e], xh, dg[i][e]);
        db[i][e] += dy[e];
        s.x += h;
        s.y = fmaf(h, xh, s.y);
      }
    }
    s = group_sum2<TPR>(s, slots[parity][group], group, lane);
    const float c1 = s.x * inv_D, c2 = s.y * inv_D;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (i * TPR + lane) * 8;
      if (c >= D) continue;
      float dy[8], x[8], g[8], o[8];
      values8(dyr[i], dy);
      values8(xr[i], x);
      params8(a.gamma, a.params_f32, c, D, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float xh = (x[e] - st.x) * st.y;
        o[e] = st.y * (fmaf(-xh, c2, dy[e] * g[e]) - c1);
      }
      if (a.dx_f32)
        store_f32x8(static_cast<float*>(a.dx) + row * a.lddx, c, D, o);
      else
        store_bf16x8(static_cast<uint16_t*>(a.dx) + row * a.lddx, c, D, o);
    }
  }
  // the groups' sums: the upper half of them adds to the lower one until one is left
#pragma unroll
  for (int half = GROUPS / 2; half > 0; half >>= 1) {
    float* mine = sums + (size_t)(group - (group >= half ? half : 0)) * (2 * NV * 8 * TPR) + lane;
    if (group >= half && group < 2 * half) {
#pragma unroll
      for (int i = 0; i < NV * 8; ++i) {
        mine[i * TPR] = dg[i >> 3][i & 7];
        mine[(NV * 8 + i) * TPR] = db[i >> 3][i & 7];
      }
    }
    __syncthreads();
    if (group < half) {
#pragma unroll
      for (int i = 0; i < NV * 8; ++i) {
        dg[i >> 3][i & 7] += mine[i * TPR];
        db[i >> 3][i & 7] += mine[(NV * 8 + i) * TPR];
      }
    }
    __syncthreads();
  }
  if (group != 0) return;
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
  float s = 0.0f;
  if (c < D) {
#pragma unroll 4
    for (int k = wid; k < rows; k += 32) s += partial[((size_t)k * 2 + blockIdx.y) * Dp + c];
  }
  red[wid][lane] = s;
  __syncthreads();
  if (wid != 0 || c >= D) return;
  float t = 0.0f;
#pragma unroll
  for (int w = 0; w < 32; ++w) t += red[w][lane];
  void* out = blockIdx.y ? dbeta : dgamma;
  if (f32)
    static_cast<float*>(out)[c] = t;
  else
    static_cast<uint16_t*>(out)[c] = (uint16_t)bf16x2_of(t, 0.0f);
}

// The shape of a row's group: as few threads as hold the row in at most four vectors each.
template <typename F>
cudaError_t with_shape(int D, F&& f) {
  const int n8 = (D + 7) / 8;
  auto nv = [&](auto tpr) {
    constexpr int TPR = decltype(tpr)::value;
    const int n = (n8 + TPR - 1) / TPR;
    if constexpr (TPR == 32) {
      if (n <= 1) return f(std::integral_constant<int, 1>{}, tpr);
      if (n <= 2) return f(std::integral_constant<int, 2>{}, tpr);
    }
    if (n <= 3) return f(std::integral_constant<int, 3>{}, tpr);
    return f(std::integral_constant<int, 4>{}, tpr);
  };
  if (n8 <= 128) return nv(std::integral_constant<int, 32>{});
  if (n8 <= 256) return nv(std::integral_constant<int, 64>{});
  if (n8 <= 512) return nv(std::integral_constant<int, 128>{});
  if (n8 <= 1024) return nv(std::integral_constant<int, 256>{});
  return nv(std::integral_constant<int, 512>{});
}

template <int SRC, bool CK>
cudaError_t launch_norm_fwd(const NormFwdArgs& a, cudaStream_t st) {
  return with_shape(a.D, [&](auto nv, auto tpr) {
    constexpr int NV = decltype(nv)::value, TPR = decltype(tpr)::value, GROUPS = kThreadsOf<TPR> / TPR;
    return launch_kernel(norm_fwd_kernel<SRC, CK, NV, TPR>, dim3((unsigned)((a.T + GROUPS - 1) / GROUPS)), dim3(kThreadsOf<TPR>), 0, st, a);
  });
}

int bwd_ctas(int64_t T, int D) {
  const int groups = D <= 1024 ? 8 : D <= 2048 ? 4 : D <= 4096 ? 2 : 1;
  return (int)std::min<int64_t>((T + groups - 1) / groups, kBwdCtas);
}

template <int SRC>
cudaError_t launch_norm_bwd(const NormBwdArgs& a, int ctas, cudaStream_t st) {
  return with_shape(a.D, [&](auto nv, auto tpr) {
    constexpr int NV = decltype(nv)::value, TPR = decltype(tpr)::value, GROUPS = kThreadsOf<TPR> / TPR;
    constexpr size_t smem = (size_t)(GROUPS / 2) * 2 * NV * 8 * TPR * sizeof(float);
    auto kernel = norm_bwd_kernel<SRC, NV, TPR>;
    const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), smem);
    if (e != cudaSuccess) return e;
    return launch_kernel(kernel, dim3((unsigned)ctas), dim3(kThreadsOf<TPR>), smem, st, a);
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
    const cudaError_t e = x8 ? launch_norm_bwd<kSrcCkpt8>(a, ctas, st)
                             : x_dtype == NVFP4_DT_F32 ? launch_norm_bwd<kSrcF32>(a, ctas, st) : launch_norm_bwd<kSrcBf16>(a, ctas, st);
    if (e != cudaSuccess || cudaGetLastError() != cudaSuccess) return NVFP4_ERR_CUDA;
  }
  launch_kernel(norm_bwd_finish_kernel, dim3((unsigned)((D + 31) / 32), dbeta ? 2u : 1u), dim3(1024), 0, st, static_cast<const float*>(workspace), T > 0 ? ctas : 0, (int)D,
                (int)(dparam_dtype == NVFP4_DT_F32), dgamma, dbeta);
  return cudaGetLastError() == cudaSuccess ? NVFP4_OK : NVFP4_ERR_CUDA;
}

}  // extern "C"
