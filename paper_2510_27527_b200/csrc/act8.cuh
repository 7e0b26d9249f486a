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

// Two binary32 values in a register pair; one packed instruction each. The kernels around the linears issue about as many instructions as
// they have time for beside memory, and most of them are such.
using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 pair_of(float lo, float hi) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ f32x2 pair_of(float v) { return pair_of(v, v); }
__device__ __forceinline__ float2 values_of(f32x2 p) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(p));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ float sum_of(f32x2 p) {
  const float2 v = values_of(p);
  return v.x + v.y;
}

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

// The eight codes of v at a group's scale (the product is exact unless it lies far below the smallest code), lowest element first. NaN has
// a code of its own, infinities would saturate.
__device__ __forceinline__ uint2 ckpt8_encode(const f32x2 (&v)[4], float inverse) {
  uint16_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 y = values_of(mul2(v[i], pair_of(inverse)));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(h[i]) : "f"(y.y), "f"(y.x));
  }
  return make_uint2((uint32_t)h[0] | (uint32_t)h[1] << 16, (uint32_t)h[2] | (uint32_t)h[3] << 16);
}
// The codes' own values, without the group's scale.
__device__ __forceinline__ void ckpt8_decode(const uint2& q, f32x2 (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = i < 2 ? q.x : q.y;
    uint32_t h2;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"((uint16_t)((i & 1) ? w >> 16 : w & 0xFFFFu)));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h2));
    v[i] = pair_of(f.x, f.y);
  }
}
// Stores the checkpoint of the eight elements v, whose largest finite-or-infinite magnitude is a (elements past a row's end are 0). All four
// threads of a group call this together, whether they have elements or not; `store` says whether this one writes, `first` whether it is the
// group's first, which writes the scale.
__device__ __forceinline__ void ckpt8_store(const f32x2 (&v)[4], float a, uint8_t* codes, uint8_t* scale, bool first, bool store) {
  a = fmaxf(a, 0.0f);  // (only NaN: 0)
  a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 1));
  a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 2));
  uint32_t byte = ckpt8_scale_byte(a);
  uint2 q;
  if (__any_sync(0xFFFFFFFFu, a == __uint_as_float(0x7F800000u))) {  // an infinity in one of the warp's groups: it becomes NaN and does not count
    f32x2 u[4];
    a = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = values_of(v[i]);
      const float lo = finite_or_nan(f.x), hi = finite_or_nan(f.y);
      a = fmaxf(a, fmaxf(fabsf(lo), fabsf(hi)));  // (the maximum of a number and NaN is the number)
      u[i] = pair_of(lo, hi);
    }
    a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 1));
    a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 2));
    byte = ckpt8_scale_byte(a);
    q = ckpt8_encode(u, ckpt8_inverse(byte));
  } else {
    q = ckpt8_encode(v, ckpt8_inverse(byte));
  }
  if (!store) return;
  *reinterpret_cast<uint2*>(codes) = q;
  if (first) *scale = (uint8_t)byte;
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
  uint32_t byte;  // of the scale (as it was loaded: arithmetic on it would wait for the load)
};

__device__ __forceinline__ f32x2 bf16_pair(uint32_t w) { return pair_of(bf16_lo(w), bf16_hi(w)); }
__device__ __forceinline__ void values8(const Raw8<kSrcBf16>& r, f32x2 (&v)[4]) {
  v[0] = bf16_pair(r.w.x);
  v[1] = bf16_pair(r.w.y);
  v[2] = bf16_pair(r.w.z);
  v[3] = bf16_pair(r.w.w);
}
__device__ __forceinline__ void values8(const Raw8<kSrcF32>& r, f32x2 (&v)[4]) {
  v[0] = pair_of(r.lo.x, r.lo.y);
  v[1] = pair_of(r.lo.z, r.lo.w);
  v[2] = pair_of(r.hi.x, r.hi.y);
  v[3] = pair_of(r.hi.z, r.hi.w);
}
__device__ __forceinline__ void values8(const Raw8<kSrcCkpt8>& r, f32x2 (&v)[4]) {  // exact
  ckpt8_decode(r.q, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = mul2(v[i], pair_of(ckpt8_scale(r.byte)));
}
// The largest magnitude of the eight, NaN left out (NaN where there is nothing else).
__device__ __forceinline__ float amax8(const Raw8<kSrcBf16>& r) {
  const uint32_t m = amax16x2(amax16x2(r.w.x, r.w.y), amax16x2(r.w.z, r.w.w));
  return fmaxf(fabsf(bf16_lo(m)), fabsf(bf16_hi(m)));
}
__device__ __forceinline__ float amax8(const Raw8<kSrcF32>& r) {
  return fmaxf(fmaxf(fmaxf(fabsf(r.lo.x), fabsf(r.lo.y)), fmaxf(fabsf(r.lo.z), fabsf(r.lo.w))),
               fmaxf(fmaxf(fabsf(r.hi.x), fabsf(r.hi.y)), fmaxf(fabsf(r.hi.z), fabsf(r.hi.w))));
}

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
// The eight from an address on (and their group's scale), of which `left` belong to the row.
template <int SRC>
__device__ __forceinline__ Raw8<SRC> load8_at(const void* p, const uint8_t* scale, int left) {
  Raw8<SRC> r;
  if constexpr (SRC == kSrcBf16) {
    r.w = load_bf16x8(static_cast<const uint16_t*>(p), 0, left);
  } else if constexpr (SRC == kSrcF32) {
    load_f32x8(static_cast<const float*>(p), 0, left, r.lo, r.hi);
  } else {  // (codes past the row's end are 0)
    r.q = *static_cast<const uint2*>(p);
    r.byte = *scale;
  }
  return r;
}
template <int SRC>
__device__ __forceinline__ Raw8<SRC> load8(const ActSrc& s, int64_t row, int c, int D) {
  constexpr int SIZE = SRC == kSrcF32 ? 4 : SRC == kSrcBf16 ? 2 : 1;
  return load8_at<SRC>(static_cast<const uint8_t*>(s.p) + (row * s.ld + c) * SIZE, SRC == kSrcCkpt8 ? s.scales + row * (s.ld >> 5) + (c >> 5) : nullptr, D - c);
}

// Elements 8 i .. 8 i + 7 of a matrix without gaps between its rows (and, of a checkpoint, in its last groups).
template <int SRC>
__device__ __forceinline__ Raw8<SRC> load8_flat(const ActSrc& s, int64_t i) {
  Raw8<SRC> r;
  if constexpr (SRC == kSrcBf16) {
    r.w = static_cast<const uint4*>(s.p)[i];
  } else if constexpr (SRC == kSrcF32) {
    r.lo = static_cast<const float4*>(s.p)[2 * i];
    r.hi = static_cast<const float4*>(s.p)[2 * i + 1];
  } else {
    r.q = static_cast<const uint2*>(s.p)[i];
    r.byte = s.scales[i >> 2];
  }
  return r;
}

// Eight values to a row of BF16 or FP32, those before D.
__device__ __forceinline__ uint32_t bf16x2_of(float lo, float hi) {
  uint32_t w;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
  return w;
}
__device__ __forceinline__ uint32_t bf16x2_of(f32x2 p) {
  const float2 v = values_of(p);
  return bf16x2_of(v.x, v.y);
}
__device__ __forceinline__ void store_bf16x8(uint16_t* row, int c, int D, const f32x2 (&v)[4]) {
  const uint32_t w[4] = {bf16x2_of(v[0]), bf16x2_of(v[1]), bf16x2_of(v[2]), bf16x2_of(v[3])};
  if (c + 8 <= D) {
    *reinterpret_cast<uint4*>(row + c) = make_uint4(w[0], w[1], w[2], w[3]);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (c + i < D) row[c + i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
}
__device__ __forceinline__ void store_bf16x8(uint16_t* at, const f32x2 (&v)[4]) {
  *reinterpret_cast<uint4*>(at) = make_uint4(bf16x2_of(v[0]), bf16x2_of(v[1]), bf16x2_of(v[2]), bf16x2_of(v[3]));
}
__device__ __forceinline__ void store_f32x8(float* row, int c, int D, const f32x2 (&v)[4]) {
  const float2 a = values_of(v[0]), b = values_of(v[1]), d = values_of(v[2]), e = values_of(v[3]);
  if (c + 8 <= D) {
    *reinterpret_cast<float4*>(row + c) = make_float4(a.x, a.y, b.x, b.y);
    *reinterpret_cast<float4*>(row + c + 4) = make_float4(d.x, d.y, e.x, e.y);
    return;
  }
  const float f[8] = {a.x, a.y, b.x, b.y, d.x, d.y, e.x, e.y};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (c + i < D) row[c + i] = f[i];
}

}  // namespace nvfp4
