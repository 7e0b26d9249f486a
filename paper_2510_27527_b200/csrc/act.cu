// The activations of a block in 8 bits, and SwiGLU, the step between its linears:
//   nvfp4_ckpt8_pack / _unpack   a matrix of activations as E4M3 codes under a power-of-two scale per 32 elements, and back
//   nvfp4_swiglu_fwd             h = g s u, s = 1 / (1 + exp(-g)), optionally with the checkpoints of g and u
//   nvfp4_swiglu_bwd             dg = dh u s (1 + g (1 - s)), du = dh g s, with g and u from their BF16 values or their checkpoints
// All of them stream: a thread takes eight neighbouring elements of a row, so that every load and store of a warp is contiguous.
#include "../../include/nvfp4.h"

#include "act8.cuh"
#include "nvfp4_internal.h"

namespace nvfp4 {

namespace {

// n / d for 0 <= n < total, in 32-bit arithmetic where that is enough
__device__ __forceinline__ int64_t quotient(int64_t n, int64_t d, int64_t total) {
  return total <= 0xFFFFFFFFll ? (int64_t)((uint32_t)n / (uint32_t)d) : n / d;
}

template <int SRC>
__global__ void __launch_bounds__(256) ckpt8_pack_kernel(ActSrc x, int64_t R, int D, int ldc, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  pdl_prologue();
  const int64_t n8 = ldc >> 3, total = R * n8;
  const int64_t gid = (int64_t)blockIdx.x * 256 + threadIdx.x;  // (a group's four threads are in one warp: n8 is a multiple of 4)
  const bool live = gid < total;
  const int64_t row = live ? quotient(gid, n8, total) : 0;
  const int c = (int)(gid - row * n8) << 3;
  float v[8] = {};
  if (live && c < D) values8(load8<SRC>(x, row, c, D), v);
  ckpt8_store(v, codes + row * ldc, scales + row * (ldc >> 5), c, live);
}

template <bool F32>
__global__ void __launch_bounds__(256) ckpt8_unpack_kernel(ActSrc x, int64_t R, int D, void* __restrict__ out, int64_t ld) {
  pdl_prologue();
  const int64_t n8 = (D + 7) >> 3, total = R * n8;
  const int64_t gid = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (gid >= total) return;
  const int64_t row = quotient(gid, n8, total);
  const int c = (int)(gid - row * n8) << 3;
  float v[8];
  values8(load8<kSrcCkpt8>(x, row, c, D), v);
  if (F32)
    store_f32x8(static_cast<float*>(out) + row * ld, c, D, v);
  else
    store_bf16x8(static_cast<uint16_t*>(out) + row * ld, c, D, v);
}

// 1 / (1 + exp(-g)): 1 at +inf, 0 at -inf
__device__ __forceinline__ float sigmoid(float g) { return __fdividef(1.0f, 1.0f + __expf(-g)); }

struct CkptOut {
  uint8_t *codes, *scales;
};

template <bool CK>
__global__ void __launch_bounds__(256) swiglu_fwd_kernel(ActSrc g, ActSrc u, int64_t T, int D, int ldc, uint16_t* __restrict__ h, int64_t ldh, CkptOut cg, CkptOut cu) {
  pdl_prologue();
  const int64_t n8 = CK ? ldc >> 3 : (D + 7) >> 3, total = T * n8;
  const int64_t gid = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const bool live = gid < total;
  const int64_t row = live ? quotient(gid, n8, total) : 0;
  const int c = (int)(gid - row * n8) << 3;
  float gv[8] = {}, uv[8] = {};
  if (live && c < D) {
    const Raw8<kSrcBf16> gr = load8<kSrcBf16>(g, row, c, D), ur = load8<kSrcBf16>(u, row, c, D);
    values8(gr, gv);
    values8(ur, uv);
    float o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = gv[i] * sigmoid(gv[i]) * uv[i];
    store_bf16x8(h + row * ldh, c, D, o);
  }
  if (CK) {
    ckpt8_store(gv, cg.codes + row * ldc, cg.scales + row * (ldc >> 5), c, live);
    ckpt8_store(uv, cu.codes + row * ldc, cu.scales + row * (ldc >> 5), c, live);
  }
}

template <int SRC>
__global__ void __launch_bounds__(256) swiglu_bwd_kernel(ActSrc dh, ActSrc g, ActSrc u, int64_t T, int D, uint16_t* __restrict__ dg, int64_t lddg, uint16_t* __restrict__ du,
                                                        int64_t lddu) {
  pdl_prologue();
  const int64_t n8 = (D + 7) >> 3, total = T * n8;
  const int64_t gid = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (gid >= total) return;
  const int64_t row = quotient(gid, n8, total);
  const int c = (int)(gid - row * n8) << 3;
  const Raw8<kSrcBf16> hr = load8<kSrcBf16>(dh, row, c, D);
  const Raw8<SRC> gr = load8<SRC>(g, row, c, D), ur = load8<SRC>(u, row, c, D);
  float hv[8], gv[8], uv[8], a[8], b[8];
  values8(hr, hv);
  values8(gr, gv);
  values8(ur, uv);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float s = sigmoid(gv[i]);
    a[i] = hv[i] * uv[i] * (s * (1.0f + gv[i] * (1.0f - s)));
    b[i] = hv[i] * (gv[i] * s);
  }
  store_bf16x8(dg + row * lddg, c, D, a);
  store_bf16x8(du + row * lddu, c, D, b);
}

constexpr int64_t kMaxCols = (int64_t)1 << 24;  // columns are 32-bit in the kernels
// CTAs of 256 threads for `threads` threads, 0: more than a grid has
unsigned ctas(int64_t threads) {
  const int64_t n = (threads + 255) / 256;
  return n <= 0x7FFFFFFF ? (unsigned)n : 0u;
}
nvfp4_status launched() { return cudaGetLastError() == cudaSuccess ? NVFP4_OK : NVFP4_ERR_CUDA; }

}  // namespace

nvfp4_status check_ckpt8(const nvfp4_ckpt8* c, int64_t R, int64_t K) {
  if (!c) return NVFP4_ERR_NULL;
  if (c->R != R || c->K != K) return NVFP4_ERR_SHAPE;
  if (R == 0) return NVFP4_OK;
  if (!c->codes || !c->scales) return NVFP4_ERR_NULL;
  return aligned(c->codes, 16) ? NVFP4_OK : NVFP4_ERR_ALIGN;
}

}  // namespace nvfp4

using namespace nvfp4;

extern "C" {

int64_t nvfp4_ckpt8_ld(int64_t K) { return (K + 31) / 32 * 32; }

nvfp4_status nvfp4_ckpt8_pack(const void* X, int32_t x_dtype, int64_t ldx, int64_t R, int64_t K, const nvfp4_ckpt8* out, void* stream) {
  if (!out) return NVFP4_ERR_NULL;
  if (x_dtype < 0 || x_dtype > 1) return NVFP4_ERR_ENUM;
  if (R < 0 || K <= 0) return NVFP4_ERR_SHAPE;
  if (K > kMaxCols) return NVFP4_ERR_LIMIT;
  nvfp4_status s = check_ckpt8(out, R, K);
  if (s != NVFP4_OK) return s;
  if (R == 0) return NVFP4_OK;
  if (!X) return NVFP4_ERR_NULL;
  if (bad_matrix(X, ldx, K, x_dtype == NVFP4_DT_F32 ? 4 : 2)) return NVFP4_ERR_ALIGN;
  const int64_t ldc = nvfp4_ckpt8_ld(K);
  const unsigned grid = ctas(R * (ldc / 8));
  if (!grid) return NVFP4_ERR_LIMIT;
  if (!device_is_sm100()) return NVFP4_ERR_ARCH;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const ActSrc x{X, nullptr, ldx};
  launch_kernel(x_dtype == NVFP4_DT_F32 ? ckpt8_pack_kernel<kSrcF32> : ckpt8_pack_kernel<kSrcBf16>, dim3(grid), dim3(256), 0, st, x, R, (int)K, (int)ldc, out->codes, out->scales);
  return launched();
}

nvfp4_status nvfp4_ckpt8_unpack(const nvfp4_ckpt8* in, void* X, int32_t x_dtype, int64_t ldx, void* stream) {
  if (!in) return NVFP4_ERR_NULL;
  if (x_dtype < 0 || x_dtype > 1) return NVFP4_ERR_ENUM;
  if (in->R < 0 || in->K <= 0) return NVFP4_ERR_SHAPE;
  if (in->K > kMaxCols) return NVFP4_ERR_LIMIT;
  nvfp4_status s = check_ckpt8(in, in->R, in->K);
  if (s != NVFP4_OK) return s;
  if (in->R == 0) return NVFP4_OK;
  if (!X) return NVFP4_ERR_NULL;
  if (bad_matrix(X, ldx, in->K, x_dtype == NVFP4_DT_F32 ? 4 : 2)) return NVFP4_ERR_ALIGN;
  const unsigned grid = ctas(in->R * ((in->K + 7) / 8));
  if (!grid) return NVFP4_ERR_LIMIT;
  if (!device_is_sm100()) return NVFP4_ERR_ARCH;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const ActSrc x{in->codes, in->scales, nvfp4_ckpt8_ld(in->K)};
  launch_kernel(x_dtype == NVFP4_DT_F32 ? ckpt8_unpack_kernel<true> : ckpt8_unpack_kernel<false>, dim3(grid), dim3(256), 0, st, x, in->R, (int)in->K, X, ldx);
  return launched();
}

nvfp4_status nvfp4_swiglu_fwd(const void* G, int64_t ldg, const void* U, int64_t ldu, int64_t T, int64_t D, void* H, int64_t ldh, const nvfp4_ckpt8* g8,
                              const nvfp4_ckpt8* u8, void* stream) {
  if (T < 0 || D <= 0 || (g8 == nullptr) != (u8 == nullptr)) return NVFP4_ERR_SHAPE;
  if (D > kMaxCols) return NVFP4_ERR_LIMIT;
  nvfp4_status s;
  if (g8 && ((s = check_ckpt8(g8, T, D)) != NVFP4_OK || (s = check_ckpt8(u8, T, D)) != NVFP4_OK)) return s;
  if (T == 0) return NVFP4_OK;
  if (!G || !U || !H) return NVFP4_ERR_NULL;
  if (bad_matrix(G, ldg, D, 2) || bad_matrix(U, ldu, D, 2) || bad_matrix(H, ldh, D, 2)) return NVFP4_ERR_ALIGN;
  const int64_t ldc = nvfp4_ckpt8_ld(D);
  const unsigned grid = ctas(T * (g8 ? ldc / 8 : (D + 7) / 8));
  if (!grid) return NVFP4_ERR_LIMIT;
  if (!device_is_sm100()) return NVFP4_ERR_ARCH;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const ActSrc g{G, nullptr, ldg}, u{U, nullptr, ldu};
  const CkptOut cg{g8 ? g8->codes : nullptr, g8 ? g8->scales : nullptr}, cu{u8 ? u8->codes : nullptr, u8 ? u8->scales : nullptr};
  launch_kernel(g8 ? swiglu_fwd_kernel<true> : swiglu_fwd_kernel<false>, dim3(grid), dim3(256), 0, st, g, u, T, (int)D, (int)ldc, static_cast<uint16_t*>(H), ldh, cg, cu);
  return launched();
}

nvfp4_status nvfp4_swiglu_bwd(const void* dH, int64_t lddh, const void* G, int64_t ldg, const void* U, int64_t ldu, const nvfp4_ckpt8* g8, const nvfp4_ckpt8* u8,
                              int64_t T, int64_t D, void* dG, int64_t lddg, void* dU, int64_t lddu, void* stream) {
  if (T < 0 || D <= 0 || (g8 == nullptr) != (u8 == nullptr)) return NVFP4_ERR_SHAPE;
  if (D > kMaxCols) return NVFP4_ERR_LIMIT;
  nvfp4_status s;
  if (g8 && ((s = check_ckpt8(g8, T, D)) != NVFP4_OK || (s = check_ckpt8(u8, T, D)) != NVFP4_OK)) return s;
  if (T == 0) return NVFP4_OK;
  if (!dH || !dG || !dU || (!g8 && (!G || !U))) return NVFP4_ERR_NULL;
  if (bad_matrix(dH, lddh, D, 2) || bad_matrix(dG, lddg, D, 2) || bad_matrix(dU, lddu, D, 2) || (!g8 && (bad_matrix(G, ldg, D, 2) || bad_matrix(U, ldu, D, 2))))
    return NVFP4_ERR_ALIGN;
  const unsigned grid = ctas(T * ((D + 7) / 8));
  if (!grid) return NVFP4_ERR_LIMIT;
  if (!device_is_sm100()) return NVFP4_ERR_ARCH;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const ActSrc dh{dH, nullptr, lddh};
  const ActSrc g = g8 ? ActSrc{g8->codes, g8->scales, nvfp4_ckpt8_ld(D)} : ActSrc{G, nullptr, ldg};
  const ActSrc u = g8 ? ActSrc{u8->codes, u8->scales, nvfp4_ckpt8_ld(D)} : ActSrc{U, nullptr, ldu};
  launch_kernel(g8 ? swiglu_bwd_kernel<kSrcCkpt8> : swiglu_bwd_kernel<kSrcBf16>, dim3(grid), dim3(256), 0, st, dh, g, u, T, (int)D, static_cast<uint16_t*>(dG), lddg,
                static_cast<uint16_t*>(dU), lddu);
  return launched();
}

}  // extern "C"
