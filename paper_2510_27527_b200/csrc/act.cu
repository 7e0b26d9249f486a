// The activations of a block in 8 bits, and SwiGLU, the step between its linears:
//   nvfp4_ckpt8_pack / _unpack   a matrix of activations as E4M3 codes under a power-of-two scale per 32 elements, and back
//   nvfp4_swiglu_fwd             h = g s u, s = 1 / (1 + exp(-g)), optionally with the checkpoints of g and u
//   nvfp4_swiglu_bwd             dg = dh u s (1 + g (1 - s)), du = dh g s, with g and u from their BF16 values or their checkpoints
// All of them stream: a thread takes eight neighbouring elements of a row, so that every load and store of a warp is contiguous.
// Measured (us, inputs from HBM; in brackets the share of the copy bandwidth): 16384 x 8192 BF16 packed 59.1 (1.06), unpacked 62.7 (1.00); SwiGLU
// 16384 x 2816 forward 40.8 (1.04), with checkpoints 60.0 (0.96), backward 68.5 (1.03), from checkpoints 57.7 (0.99). Memory bounds them.
#include "../../include/nvfp4.h"

#include <type_traits>

#include "act8.cuh"
#include "nvfp4_internal.h"

namespace nvfp4 {

namespace {

// n / d for 0 <= n < total, in 32-bit arithmetic where that is enough
__device__ __forceinline__ int64_t quotient(int64_t n, int64_t d, int64_t total) {
  return total <= 0xFFFFFFFFll ? (int64_t)((uint32_t)n / (uint32_t)d) : n / d;
}

// FLAT, of every kernel here: matrices without gaps (leading dimensions that are D, and D a multiple of the group where there are checkpoints),
// whose pieces of eight need no row and column: fewer instructions for what is bound by them and by memory alike (SwiGLU forward with
// checkpoints, 16384 x 2816: 66.6 us with rows and columns, 60.0 without).
//
// NB pieces of eight elements a thread, one CTA's next to one another: one piece's loads of all threads of an SM (32 KB from BF16, 16 KB of
// codes) are fewer than memory needs in flight.
template <int SRC, int NB, bool FLAT>
__global__ void __launch_bounds__(256) ckpt8_pack_kernel(ActSrc x, int64_t R, int D, int ldc, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  pdl_prologue();
  const int64_t n8 = ldc >> 3, total = R * n8;
  const int64_t first = (int64_t)blockIdx.x * (256 * NB) + threadIdx.x;  // (a group's four threads are in one warp: n8 is a multiple of 4)
  Raw8<SRC> r[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int64_t gid = first + j * 256;
    r[j] = Raw8<SRC>{};
    if (gid >= total) continue;
    if (FLAT) {
      r[j] = load8_flat<SRC>(x, gid);
    } else {
      const int64_t row = quotient(gid, n8, total);
      const int c = (int)(gid - row * n8) << 3;
      if (c < D) r[j] = load8<SRC>(x, row, c, D);
    }
  }
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int64_t gid = first + j * 256;  // (a checkpoint has no gaps)
    f32x2 v[4];
    values8(r[j], v);
    ckpt8_store(v, amax8(r[j]), codes + gid * 8, scales + (gid >> 2), (gid & 3) == 0, gid < total);
  }
}

template <bool F32, int NB, bool FLAT>
__global__ void __launch_bounds__(256) ckpt8_unpack_kernel(ActSrc x, int64_t R, int D, void* __restrict__ out, int64_t ld) {
  pdl_prologue();
  const int64_t n8 = (D + 7) >> 3, total = R * n8;
  const int64_t first = (int64_t)blockIdx.x * (256 * NB) + threadIdx.x;
  Raw8<kSrcCkpt8> r[NB];
  int64_t row[NB];
  int c[NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int64_t gid = first + j * 256;
    if (gid >= total) break;
    if (FLAT) {
      r[j] = load8_flat<kSrcCkpt8>(x, gid);
    } else {
      row[j] = quotient(gid, n8, total);
      c[j] = (int)(gid - row[j] * n8) << 3;
      r[j] = load8<kSrcCkpt8>(x, row[j], c[j], D);
    }
  }
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    const int64_t gid = first + j * 256;
    if (gid >= total) break;
    f32x2 v[4];
    values8(r[j], v);
    if (F32)
      store_f32x8(FLAT ? static_cast<float*>(out) + gid * 8 : static_cast<float*>(out) + row[j] * ld, FLAT ? 0 : c[j], FLAT ? 8 : D, v);
    else if (FLAT)
      store_bf16x8(static_cast<uint16_t*>(out) + gid * 8, v);
    else
      store_bf16x8(static_cast<uint16_t*>(out) + row[j] * ld, c[j], D, v);
  }
}

// 1 / (1 + exp(-g)), exp(-g) = 2^(-g log2 e): 1 at +inf, 0 at -inf. The quotient of a quarter of the denominator, a quarter of it: in range for
// every finite one, where the fast division gives 0 for those above 2^126, whose quotients are subnormal numbers that make normal products with a
// large u (g = -88, u = 2^20: 2^-101). Below g = -88.72 the power is infinite and the result 0; a power below 2^-126 is nothing beside 1.
__device__ __forceinline__ float power2(float t) {
  float p;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(p) : "f"(t));
  return p;
}
__device__ __forceinline__ f32x2 sigmoid2(f32x2 g) {
  const float2 t = values_of(mul2(g, pair_of(-1.44269504f)));
  const float2 y = values_of(fma2(pair_of(power2(t.x), power2(t.y)), pair_of(0.25f), pair_of(0.25f)));
  return mul2(pair_of(__fdividef(1.0f, y.x), __fdividef(1.0f, y.y)), pair_of(0.25f));
}

struct CkptOut {
  uint8_t *codes, *scales;
};

template <bool CK, bool FLAT>
__global__ void __launch_bounds__(256) swiglu_fwd_kernel(ActSrc g, ActSrc u, int64_t T, int D, int ldc, uint16_t* h, int64_t ldh, CkptOut cg, CkptOut cu) {
  pdl_prologue();
  const int64_t n8 = CK ? ldc >> 3 : (D + 7) >> 3, total = T * n8;
  const int64_t gid = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const bool live = gid < total;
  int64_t row = 0;
  int c = 0;
  Raw8<kSrcBf16> gr{}, ur{};
  if (FLAT && live) {
    gr = load8_flat<kSrcBf16>(g, gid);
    ur = load8_flat<kSrcBf16>(u, gid);
  }
  if (!FLAT && live) {
    row = quotient(gid, n8, total);
    c = (int)(gid - row * n8) << 3;
    if (c < D) {
      gr = load8<kSrcBf16>(g, row, c, D);
      ur = load8<kSrcBf16>(u, row, c, D);
    }
  }
  f32x2 gv[4], uv[4];
  values8(gr, gv);
  values8(ur, uv);
  if (live && c < D) {
    f32x2 o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = mul2(mul2(gv[i], sigmoid2(gv[i])), uv[i]);
    if (FLAT)
      store_bf16x8(h + gid * 8, o);
    else
      store_bf16x8(h + row * ldh, c, D, o);
  }
  if (CK) {
    ckpt8_store(gv, amax8(gr), cg.codes + gid * 8, cg.scales + (gid >> 2), (gid & 3) == 0, live);
    ckpt8_store(uv, amax8(ur), cu.codes + gid * 8, cu.scales + (gid >> 2), (gid & 3) == 0, live);
  }
}

template <int SRC, bool FLAT>
__global__ void __launch_bounds__(256) swiglu_bwd_kernel(ActSrc dh, ActSrc g, ActSrc u, int64_t T, int D, uint16_t* dg, int64_t lddg, uint16_t* du,
                                                        int64_t lddu) {
  pdl_prologue();
  const int64_t n8 = (D + 7) >> 3, total = T * n8;
  const int64_t gid = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (gid >= total) return;
  int64_t row = 0;
  int c = 0;
  Raw8<kSrcBf16> hr;
  Raw8<SRC> gr, ur;
  if (FLAT) {
    hr = load8_flat<kSrcBf16>(dh, gid);
    gr = load8_flat<SRC>(g, gid);
    ur = load8_flat<SRC>(u, gid);
  } else {
    row = quotient(gid, n8, total);
    c = (int)(gid - row * n8) << 3;
    hr = load8<kSrcBf16>(dh, row, c, D);
    gr = load8<SRC>(g, row, c, D);
    ur = load8<SRC>(u, row, c, D);
  }
  f32x2 hv[4], gv[4], uv[4], a[4], b[4];
  values8(hr, hv);
  values8(gr, gv);
  values8(ur, uv);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 s = sigmoid2(gv[i]), one = pair_of(1.0f), rest = fma2(s, pair_of(-1.0f), one);
    a[i] = mul2(mul2(hv[i], uv[i]), mul2(s, fma2(gv[i], rest, one)));
    b[i] = mul2(hv[i], mul2(gv[i], s));
  }
  if (FLAT) {
    store_bf16x8(dg + gid * 8, a);
    store_bf16x8(du + gid * 8, b);
  } else {
    store_bf16x8(dg + row * lddg, c, D, a);
    store_bf16x8(du + row * lddu, c, D, b);
  }
}

constexpr int64_t kMaxCols = (int64_t)1 << 24, kMaxRows = (int64_t)1 << 38;  // columns are 32-bit in the kernels; pieces do not pass 64 bits
// CTAs of 256 threads for `pieces` pieces, nb a thread; 0: more than a grid has
unsigned ctas(int64_t pieces, int nb = 1) {
  const int64_t n = (pieces + 256 * nb - 1) / (256 * nb);
  return n <= 0x7FFFFFFF ? (unsigned)n : 0u;
}
// Up to here a call's pieces are all in flight at once, one a thread.
int64_t few_pieces() { return (int64_t)device_sm_count() * 2048; }
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
  if (K > kMaxCols || R > kMaxRows) return NVFP4_ERR_LIMIT;
  nvfp4_status s = check_ckpt8(out, R, K);
  if (s != NVFP4_OK) return s;
  if (R == 0) return NVFP4_OK;
  if (!X) return NVFP4_ERR_NULL;
  if (bad_matrix(X, ldx, K, x_dtype == NVFP4_DT_F32 ? 4 : 2)) return NVFP4_ERR_ALIGN;
  const int64_t ldc = nvfp4_ckpt8_ld(K);
  const int64_t pieces = R * (ldc / 8);
  const int nb = pieces > few_pieces() ? 2 : 1;
  const unsigned grid = ctas(pieces, nb);
  if (!grid) return NVFP4_ERR_LIMIT;
  if (!device_is_sm100()) return NVFP4_ERR_ARCH;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const ActSrc x{X, nullptr, ldx};
  const bool f32 = x_dtype == NVFP4_DT_F32;
  auto kernel = [&](auto flat) {
    constexpr bool FLAT = decltype(flat)::value;
    return nb == 1 ? (f32 ? ckpt8_pack_kernel<kSrcF32, 1, FLAT> : ckpt8_pack_kernel<kSrcBf16, 1, FLAT>)
                   : (f32 ? ckpt8_pack_kernel<kSrcF32, 2, FLAT> : ckpt8_pack_kernel<kSrcBf16, 2, FLAT>);
  };
  launch_kernel(ldx == ldc && K == ldc ? kernel(std::true_type{}) : kernel(std::false_type{}), dim3(grid), dim3(256), 0, st, x, R, (int)K, (int)ldc, out->codes, out->scales);
  return launched();
}

nvfp4_status nvfp4_ckpt8_unpack(const nvfp4_ckpt8* in, void* X, int32_t x_dtype, int64_t ldx, void* stream) {
  if (!in) return NVFP4_ERR_NULL;
  if (x_dtype < 0 || x_dtype > 1) return NVFP4_ERR_ENUM;
  if (in->R < 0 || in->K <= 0) return NVFP4_ERR_SHAPE;
  if (in->K > kMaxCols || in->R > kMaxRows) return NVFP4_ERR_LIMIT;
  nvfp4_status s = check_ckpt8(in, in->R, in->K);
  if (s != NVFP4_OK) return s;
  if (in->R == 0) return NVFP4_OK;
  if (!X) return NVFP4_ERR_NULL;
  if (bad_matrix(X, ldx, in->K, x_dtype == NVFP4_DT_F32 ? 4 : 2)) return NVFP4_ERR_ALIGN;
  const int64_t pieces = in->R * ((in->K + 7) / 8);
  const int nb = pieces > few_pieces() ? 4 : 1;
  const unsigned grid = ctas(pieces, nb);
  if (!grid) return NVFP4_ERR_LIMIT;
  if (!device_is_sm100()) return NVFP4_ERR_ARCH;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const ActSrc x{in->codes, in->scales, nvfp4_ckpt8_ld(in->K)};
  const bool f32 = x_dtype == NVFP4_DT_F32;
  auto kernel = [&](auto flat) {
    constexpr bool FLAT = decltype(flat)::value;
    return nb == 1 ? (f32 ? ckpt8_unpack_kernel<true, 1, FLAT> : ckpt8_unpack_kernel<false, 1, FLAT>)
                   : (f32 ? ckpt8_unpack_kernel<true, 4, FLAT> : ckpt8_unpack_kernel<false, 4, FLAT>);
  };
  launch_kernel(ldx == in->K && in->K % 32 == 0 ? kernel(std::true_type{}) : kernel(std::false_type{}), dim3(grid), dim3(256), 0, st, x, in->R, (int)in->K, X, ldx);
  return launched();
}

nvfp4_status nvfp4_swiglu_fwd(const void* G, int64_t ldg, const void* U, int64_t ldu, int64_t T, int64_t D, void* H, int64_t ldh, const nvfp4_ckpt8* g8,
                              const nvfp4_ckpt8* u8, void* stream) {
  if (T < 0 || D <= 0 || (g8 == nullptr) != (u8 == nullptr)) return NVFP4_ERR_SHAPE;
  if (D > kMaxCols || T > kMaxRows) return NVFP4_ERR_LIMIT;
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
  const bool flat = ldg == D && ldu == D && ldh == D && D % (g8 ? 32 : 8) == 0;
  launch_kernel(g8 ? (flat ? swiglu_fwd_kernel<true, true> : swiglu_fwd_kernel<true, false>) : (flat ? swiglu_fwd_kernel<false, true> : swiglu_fwd_kernel<false, false>), dim3(grid), dim3(256), 0, st, g, u, T, (int)D, (int)ldc, static_cast<uint16_t*>(H), ldh, cg, cu);
  return launched();
}

nvfp4_status nvfp4_swiglu_bwd(const void* dH, int64_t lddh, const void* G, int64_t ldg, const void* U, int64_t ldu, const nvfp4_ckpt8* g8, const nvfp4_ckpt8* u8,
                              int64_t T, int64_t D, void* dG, int64_t lddg, void* dU, int64_t lddu, void* stream) {
  if (T < 0 || D <= 0 || (g8 == nullptr) != (u8 == nullptr)) return NVFP4_ERR_SHAPE;
  if (D > kMaxCols || T > kMaxRows) return NVFP4_ERR_LIMIT;
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
  const bool flat = g.ld == D && u.ld == D && lddh == D && lddg == D && lddu == D;  // (a checkpoint's ld is a multiple of 32, another's of 8)
  launch_kernel(g8 ? (flat ? swiglu_bwd_kernel<kSrcCkpt8, true> : swiglu_bwd_kernel<kSrcCkpt8, false>)
                   : (flat ? swiglu_bwd_kernel<kSrcBf16, true> : swiglu_bwd_kernel<kSrcBf16, false>), dim3(grid), dim3(256), 0, st, dh, g, u, T, (int)D, static_cast<uint16_t*>(dG), lddg,
                static_cast<uint16_t*>(dU), lddu);
  return launched();
}

}  // extern "C"
