// Activations in rows of BF16, FP32 or 8-bit checkpoints, eight neighbouring elements to a thread: loads, stores and the checkpoint's
// format (nvfp4_ckpt8 in the ABI header). A group of 32 elements is four such threads next to one another.
#pragma once
#include "../../include/nvfp4.h"
#include "nvfp4_device.cuh"

namespace nvfp4 {

// checks of arguments, on the host
inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline bool bad_matrix(const void* p, int64_t ld, int64_t cols, int elem_bytes) { return !aligned(p, 16) || ld < cols || (ld * elem_bytes) % 16 != 0; }
nvfp4_status check_ckpt8(const nvfp4_ckpt8* c, int64_t R, int64_t K);  // a checkpoint for a matrix [R, K]

constexpr int kSrcBf16 = 0, kSrcF32 = 1, kSrcCkpt8 = 2;

// ---------------------------------------------------------------------------------------------------------
// the checkpoint's format
// ---------------------------------------------------------------------------------------------------------
// E4M3 has no infinity: x, or NaN where x is not finite (inf * 0 is NaN; x + 0 keeps the sign of a zero, since x * 0 has it too).
__device__ __forceinline__ float finite_or_nan(float x) { return __fmaf_rn(x, 0.0f, x); }
// Byte of the group's scale 2^(byte - 127) from its largest finite magnitude a: the smallest power of two with a <= 448 * scale. 448 is
// 1.75 * 2^8, so the exponent is a's less 8, one more where a's mantissa is above 1.75 (the addition carries into the exponent then). From
// 2^-117 up: there the smallest code, 2^-9, is still a normal BF16 number.
__device__ __forceinline__ uint32_t ckpt8_scale_byte(float a) {
  return (uint32_t)max((int)((__float_as_uint(a) + 0x1FFFFFu) >> 23) - 8, 10);
}
__device__ __forceinline__ float ckpt8_scale(uint32_t byte) { return __uint_as_float(byte << 23); }            // byte in 10 .. 247
__device__ __forceinline__ float ckpt8_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }  // 1 / scale, exactly

// The eight codes of v at a group's scale (the product is exact unless it lies far below the smallest code), lowest element first.
__device__ __forceinline__ uint2 ckpt8_encode(const float (&v)[8], float inverse) {
  uint16_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(h[i]) : "f"(__fmul_rn(v[2 * i + 1], inverse)), "f"(__fmul_rn(v[2 * i], inverse)));
  return make_uint2((uint32_t)h[0] | (uint32_t)h[1] << 16, (uint32_t)h[2] | (uint32_t)h[3] << 16);
}
__device__ __forceinline__ void ckpt8_decode(const uint2& q, float scale, float (&v)[8]) {  // exact
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = i < 2 ? q.x : q.y;
    uint32_t h2;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"((uint16_t)((i & 1) ? w >> 16 : w & 0xFFFFu)));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h2));
    v[2 * i] = __fmul_rn(f.x, scale);
    v[2 * i + 1] = __fmul_rn(f.y, scale);
  }
}
// Stores the checkpoint of the eight elements v at column c of a row (c < ld, a multiple of 8; elements past the row's end are 0).
// All four threads of a group call this together, whether they have elements or not; `store` says whether this one writes.
__device__ __forceinline__ void ckpt8_store(const float (&x)[8], uint8_t* codes_row, uint8_t* scales_row, int c, bool store) {
  float v[8], a = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    v[i] = finite_or_nan(x[i]);
    a = fmaxf(a, fabsf(v[i]));  // (the maximum of a number and NaN is the number)
  }
  a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 1));
  a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 2));
  const uint32_t byte = ckpt8_scale_byte(a);
  if (!store) return;
  *reinterpret_cast<uint2*>(codes_row + c) = ckpt8_encode(v, ckpt8_inverse(byte));
  if ((c & 31) == 0) scales_row[c >> 5] = (uint8_t)byte;
}

// ---------------------------------------------------------------------------------------------------------
// eight elements of a row, as they lie in memory and as binary32
// ---------------------------------------------------------------------------------------------------------
template <int SRC>
struct Raw8;
template <>
struct Raw8<kSrcBf16> {
  uint4 w;
};
template <>
struct Raw8<kSrcF32> {
  float4 lo, hi;
};
template <>
struct Raw8<kSrcCkpt8> {
  uint2 q;
  float scale;
};

__device__ __forceinline__ void bf16x8_values(const uint4& w, float (&v)[8]) {
  v[0] = bf16_lo(w.x); v[1] = bf16_hi(w.x);
  v[2] = bf16_lo(w.y); v[3] = bf16_hi(w.y);
  v[4] = bf16_lo(w.z); v[5] = bf16_hi(w.z);
  v[6] = bf16_lo(w.w); v[7] = bf16_hi(w.w);
}
__device__ __forceinline__ void values8(const Raw8<kSrcBf16>& r, float (&v)[8]) { bf16x8_values(r.w, v); }
__device__ __forceinline__ void values8(const Raw8<kSrcF32>& r, float (&v)[8]) {
  v[0] = r.lo.x; v[1] = r.lo.y; v[2] = r.lo.z; v[3] = r.lo.w;
  v[4] = r.hi.x; v[5] = r.hi.y; v[6] = r.hi.z; v[7] = r.hi.w;
}
__device__ __forceinline__ void values8(const Raw8<kSrcCkpt8>& r, float (&v)[8]) { ckpt8_decode(r.q, r.scale, v); }

// Elements c .. c + 7 of a row of D (c a multiple of 8; the row starts on a 16-byte boundary). Elements from D on are 0 and not read.
__device__ __forceinline__ uint4 load_bf16x8(const uint16_t* row, int c, int D) {
  if (c + 8 <= D) return *reinterpret_cast<const uint4*>(row + c);
  uint32_t h[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) h[i] = c + i < D ? row[c + i] : 0u;
  return make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
}
__device__ __forceinline__ void load_f32x8(const float* row, int c, int D, float4& lo, float4& hi) {
  if (c + 8 <= D) {
    lo = *reinterpret_cast<const float4*>(row + c);
    hi = *reinterpret_cast<const float4*>(row + c + 4);
    return;
  }
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = c + i < D ? row[c + i] : 0.0f;
  lo = make_float4(v[0], v[1], v[2], v[3]);
  hi = make_float4(v[4], v[5], v[6], v[7]);
}

// A matrix of activations: BF16 or FP32 with a leading dimension, or a checkpoint (ld its padded row length).
struct ActSrc {
  const void* p;          // values, or the checkpoint's codes
  const uint8_t* scales;  // of a checkpoint
  int64_t ld;
};
template <int SRC>
__device__ __forceinline__ Raw8<SRC> load8(const ActSrc& s, int64_t row, int c, int D) {
  Raw8<SRC> r;
  if constexpr (SRC == kSrcBf16) {
    r.w = load_bf16x8(static_cast<const uint16_t*>(s.p) + row * s.ld, c, D);
  } else if constexpr (SRC == kSrcF32) {
    load_f32x8(static_cast<const float*>(s.p) + row * s.ld, c, D, r.lo, r.hi);
  } else {  // (codes past D are 0)
    r.q = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(s.p) + row * s.ld + c);
    r.scale = ckpt8_scale(s.scales[row * (s.ld >> 5) + (c >> 5)]);
  }
  return r;
}

// Eight values to a row of BF16 or FP32, those before D.
__device__ __forceinline__ uint32_t bf16x2_of(float lo, float hi) {
  uint32_t w;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  return w;
}
__device__ __forceinline__ void store_bf16x8(uint16_t* row, int c, int D, const float (&v)[8]) {
  const uint4 w = make_uint4(bf16x2_of(v[0], v[1]), bf16x2_of(v[2], v[3]), bf16x2_of(v[4], v[5]), bf16x2_of(v[6], v[7]));
  if (c + 8 <= D) {
    *reinterpret_cast<uint4*>(row + c) = w;
    return;
  }
  const uint32_t h[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (c + i < D) row[c + i] = (uint16_t)(h[i >> 1] >> (16 * (i & 1)));
}
__device__ __forceinline__ void store_f32x8(float* row, int c, int D, const float (&v)[8]) {
  if (c + 8 <= D) {
    *reinterpret_cast<float4*>(row + c) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(row + c + 4) = make_float4(v[4], v[5], v[6], v[7]);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (c + i < D) row[c + i] = v[i];
}

}  // namespace nvfp4
