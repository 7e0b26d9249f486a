// nvfp4_gemv: a few tokens times quantized weights, Y[m, n] = sum_k X[m, k] (P Sb Sg)[n, k] (+ the outlier channels' BF16 product, + bias), the
// product of token-by-token answering. X stays in BF16 (nothing about it is quantized); the weights are read once, 0.5625 bytes each.
//
// The work is reading the weights, so all else is kept off their way. A warp takes 16 weight rows x 128 k at a time, 16 bytes (32 codes) of two
// rows per lane, and multiplies them on the tensor cores (mma m16n8k16: 8 tokens cost what one costs): E2M1 pairs become FP16 pairs in one
// conversion each, times the block scale exactly (P * Sb has at most 7 significant bits and lies within FP16's normal range). Which k stand
// in which slot of an instruction is free as long as both operands agree, so the codes are used as they lie in memory and X is staged in
// shared memory in that order. FP16 also holds X: a token's 128 values are scaled by the power of two that brings their largest magnitude to
// [2^14, 2^15); a BF16 value has 8 significant bits, so the scaling is exact for all down to 2^-28 of the largest, and what is below loses less
// than 2^-39 of it. Every 128 k the FP32 result of the instructions is added to FP32 sums with the product of that power of two and the
// weights' global scale, which is constant there in every scale mode.
// The outlier channels go through BF16 instructions, 32 of them per step, with the same rows.
// A CTA takes 64 rows: 16 of each 32 of a 128-row tile, because that is whose scale bytes lie together. The k axis is split over the warps of a CTA
// and over the CTAs of a cluster, whose sums are added through distributed shared memory in a fixed order, one that M does not change.
#include "../../include/nvfp4.h"

#include "act8.cuh"
#include "nvfp4_internal.h"

namespace nvfp4 {

namespace {

constexpr int kRows = 64;        // weight rows of a CTA
constexpr int kKWarps = 2;       // warps along k
constexpr int kThreads = 4 * kKWarps * 32;
constexpr int kPrefetch = 4;     // items in flight per warp
constexpr int kMaxTokens = 32;   // of one pass over the weights
constexpr int kMaxCluster = 8;
constexpr int kXBytes = 64 * 1024;  // of staged X, at most

struct GemvArgs {
  const uint16_t* X;
  int64_t ldx, M;
  int D, K;  // columns of X, of the operand
  const int32_t *keep, *outl;
  int n_out, Kh;
  const uint16_t* W_out;
  const uint8_t *codes, *sf;
  const float* gscale;
  int64_t N;
  int gs_mode, tiled;
  const uint16_t* bias;
  void* Y;
  int y_f32;
  int64_t ldy;
  int n_codes, n_items;  // 128-k pieces of the codes; those and the 32-channel steps of the outliers
  int seg;               // items staged at a time
};

struct Item {  // what a lane holds of one item
  uint4 w0, w1;
  uint32_t s0, s1;  // two scale bytes each
  float g0, g1;
};

__device__ __forceinline__ uint4 load_stream(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// eight codes times the scale pair (both halves equal), as FP16 pairs in order
__device__ __forceinline__ void weights8(uint32_t word, uint32_t scale2, uint32_t (&h)[4]) {
  asm("{\n"
      ".reg .b8 b0, b1, b2, b3;\n"
      "mov.b32 {b0, b1, b2, b3}, %4;\n"
      "cvt.rn.f16x2.e2m1x2 %0, b0;\n"
      "cvt.rn.f16x2.e2m1x2 %1, b1;\n"
      "cvt.rn.f16x2.e2m1x2 %2, b2;\n"
      "cvt.rn.f16x2.e2m1x2 %3, b3;\n"
      "}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(word));
  const __half2 s = *reinterpret_cast<const __half2*>(&scale2);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 p = __hmul2(*reinterpret_cast<const __half2*>(&h[i]), s);
    h[i] = *reinterpret_cast<const uint32_t*>(&p);
  }
}
// the values of two E4M3 bytes, each in both halves of a word
__device__ __forceinline__ void scales2(uint32_t bytes, uint32_t (&s)[2]) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)bytes));
  s[0] = __byte_perm(h, h, 0x1010);
  s[1] = __byte_perm(h, h, 0x3232);
}
__device__ __forceinline__ float load_cluster(const float* p, uint32_t rank) {
  uint32_t at;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}

// Column `c` of the source that the operand's (or the outliers') column k stands for; -1 where it has none.
__device__ __forceinline__ uint32_t x_bits(const uint16_t* row, const int32_t* cols, int k, int n, int D) {
  if (k >= n) return 0u;
  const int c = cols ? cols[k] : k;
  return (uint32_t)c < (uint32_t)D ? row[c] : 0x7FC0u;  // a column that X does not have: NaN
}
__device__ __forceinline__ uint4 x8(const uint16_t* row, const int32_t* cols, int k, int n, int D) {
  if (!cols && k + 8 <= n) return *reinterpret_cast<const uint4*>(row + k);
  uint32_t h[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) h[i] = x_bits(row, cols, k + i, n, D);
  return make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
}

template <int MT>  // instructions' widths of eight tokens
__global__ void __launch_bounds__(kThreads) gemv_kernel(GemvArgs a) {
  pdl_prologue();
  extern __shared__ __align__(16) uint8_t smem[];
  constexpr int TOK = 8 * MT;
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int rowset = wid & 3, kw = wid >> 2;
  const int S = (int)cluster_ctas(), rank = (int)(blockIdx.x % (uint32_t)S);
  const int64_t rb = blockIdx.x / (uint32_t)S;
  const int64_t m0 = (int64_t)blockIdx.y * kMaxTokens;
  const int Mg = (int)min((int64_t)kMaxTokens, a.M - m0);
  const int64_t row0 = (rb >> 1) * 128 + rowset * 32 + (rb & 1) * 16 + g;
  const int64_t r0 = min(row0, a.N - 1), r1 = min(row0 + 8, a.N - 1);  // (rows past the end repeat the last one and are not stored)
  const int Kp = (a.K + 127) & ~127;
  const int64_t nb = Kp >> 4, nbp = (nb + 15) & ~(int64_t)15;

  uint8_t* xs = smem;                                                       // [item][4][token][4] 16 bytes
  float* xscale = reinterpret_cast<float*>(smem + (size_t)a.seg * 256 * Mg);  // [item][TOK]
  float* red = xscale + a.seg * TOK;                                        // [kw][TOK][kRows]

  const int i_begin = (int)((int64_t)rank * a.n_items / S), i_end = (int)((int64_t)(rank + 1) * a.n_items / S);
  const uint8_t *c0 = a.codes + r0 * (Kp >> 1) + t * 16, *c1 = a.codes + r1 * (Kp >> 1) + t * 16;
  const uint16_t *o0 = a.W_out + r0 * a.Kh + t * 8, *o1 = a.W_out + r1 * a.Kh + t * 8;
  const uint8_t* sf0 = a.tiled ? a.sf + sf_tiled_offset(r0, 2 * t, nbp) : a.sf + r0 * nb + 2 * t;
  const uint8_t* sf1 = a.tiled ? a.sf + sf_tiled_offset(r1, 2 * t, nbp) : a.sf + r1 * nb + 2 * t;
  const int sf_step = a.tiled ? 1024 : 8;  // bytes from one item to the next
  const bool b128 = a.gs_mode == kGsBlock128;
  const float* gs0 = a.gscale + (b128 ? r0 * (Kp >> 7) : a.gs_mode == kGsRow ? r0 : 0);
  const float* gs1 = a.gscale + (b128 ? r1 * (Kp >> 7) : a.gs_mode == kGsRow ? r1 : 0);

  auto load = [&](Item& q, int i) {
    if (i < a.n_codes) {
      q.w0 = load_stream(c0 + (int64_t)i * 64);
      q.w1 = load_stream(c1 + (int64_t)i * 64);
      q.s0 = *reinterpret_cast<const uint16_t*>(sf0 + (int64_t)i * sf_step);
      q.s1 = *reinterpret_cast<const uint16_t*>(sf1 + (int64_t)i * sf_step);
      q.g0 = gs0[b128 ? i : 0];
      q.g1 = gs1[b128 ? i : 0];
    } else {
      q.w0 = load_stream(o0 + (int64_t)(i - a.n_codes) * 32);
      q.w1 = load_stream(o1 + (int64_t)(i - a.n_codes) * 32);
    }
  };

  float acc[MT][4] = {};
  Item q[kPrefetch];
  for (int s0 = i_begin; s0 < i_end; s0 += a.seg) {
    const int n_seg = min(a.seg, i_end - s0);
#pragma unroll
    for (int p = 0; p < kPrefetch; ++p)
      if (kw + p * kKWarps < n_seg) load(q[p], s0 + kw + p * kKWarps);
    // X: 16 lanes take a token's 128 values of a piece (or the 32 of a step: 4 lanes of them), eight each
    {
      const int l16 = lane & 15;
      for (int u0 = wid * 2; u0 < n_seg * Mg; u0 += kThreads / 16) {  // (a warp's two halves stay together)
        const int u = u0 + (lane >> 4);
        const bool live = u < n_seg * Mg;
        const int it = live ? u / Mg : 0, m = live ? u - it * Mg : 0, i = s0 + it;
        const uint16_t* row = a.X + (m0 + m) * a.ldx;
        const bool code = i < a.n_codes;
        uint4 w = make_uint4(0, 0, 0, 0);
        if (live && code) w = x8(row, a.keep, i * 128 + l16 * 8, a.K, a.D);
        if (live && !code && l16 < 4) w = x8(row, a.outl, (i - a.n_codes) * 32 + l16 * 8, a.n_out, a.D);
        uint32_t m2 = amax16x2(amax16x2(w.x, w.y), amax16x2(w.z, w.w));
        float v[8], big = fmaxf(fabsf(bf16_lo(m2)), fabsf(bf16_hi(m2)));
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) big = fmaxf(big, __shfl_xor_sync(0xFFFFFFFFu, big, o));
        const uint32_t e = max(__float_as_uint(big) >> 23, 15u);
        if (code) {
          const float to = __uint_as_float((268u - e) << 23);  // 2^(141 - e)
          bf16x8_values(w, v);
          uint32_t h[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const __half2 p = __floats2half2_rn(v[2 * j] * to, v[2 * j + 1] * to);
            h[j] = *reinterpret_cast<const uint32_t*>(&p);
          }
          w = make_uint4(h[0], h[1], h[2], h[3]);
        }
        if (live) {
          uint8_t* at = xs + (size_t)it * 256 * Mg;
          if (code) {
            *reinterpret_cast<uint4*>(at + (((l16 & 3) * Mg + m) * 4 + (l16 >> 2)) * 16) = w;
            if (l16 == 0) xscale[it * TOK + m] = __uint_as_float((e - 14u) << 23);  // 2^(e - 141)
          } else if (l16 < 4) {
            *reinterpret_cast<uint4*>(at + (m * 4 + l16) * 16) = w;
          }
        }
      }
    }
    __syncthreads();
    for (int j = kw; j < n_seg; j += kPrefetch * kKWarps) {
#pragma unroll
      for (int p = 0; p < kPrefetch; ++p) {
        const int it = j + p * kKWarps;
        if (it < n_seg) {
          const uint8_t* at = xs + (size_t)it * 256 * Mg;
          float d[MT][4] = {};
          if (s0 + it < a.n_codes) {
            uint32_t sa[2], sb[2];
            scales2(q[p].s0, sa);
            scales2(q[p].s1, sb);
            const uint32_t wa[4] = {q[p].w0.x, q[p].w0.y, q[p].w0.z, q[p].w0.w}, wb[4] = {q[p].w1.x, q[p].w1.y, q[p].w1.z, q[p].w1.w};
#pragma unroll
            for (int wd = 0; wd < 4; ++wd) {
              uint32_t ha[4], hb[4];
              weights8(wa[wd], sa[wd >> 1], ha);
              weights8(wb[wd], sb[wd >> 1], hb);
#pragma unroll
              for (int n = 0; n < MT; ++n) {
                uint4 b = make_uint4(0, 0, 0, 0);
                if (n * 8 + g < Mg) b = *reinterpret_cast<const uint4*>(at + ((wd * Mg + n * 8 + g) * 4 + t) * 16);
                mma_f16(d[n], ha[0], hb[0], ha[1], hb[1], b.x, b.y);
                mma_f16(d[n], ha[2], hb[2], ha[3], hb[3], b.z, b.w);
              }
            }
#pragma unroll
            for (int n = 0; n < MT; ++n) {
              const float2 xsc = *reinterpret_cast<const float2*>(xscale + it * TOK + n * 8 + 2 * t);
              acc[n][0] = fmaf(d[n][0], xsc.x * q[p].g0, acc[n][0]);
              acc[n][1] = fmaf(d[n][1], xsc.y * q[p].g0, acc[n][1]);
              acc[n][2] = fmaf(d[n][2], xsc.x * q[p].g1, acc[n][2]);
              acc[n][3] = fmaf(d[n][3], xsc.y * q[p].g1, acc[n][3]);
            }
          } else {
#pragma unroll
            for (int n = 0; n < MT; ++n) {
              uint4 b = make_uint4(0, 0, 0, 0);
              if (n * 8 + g < Mg) b = *reinterpret_cast<const uint4*>(at + ((n * 8 + g) * 4 + t) * 16);
              mma_bf16(d[n], q[p].w0.x, q[p].w1.x, q[p].w0.y, q[p].w1.y, b.x, b.y);
              mma_bf16(d[n], q[p].w0.z, q[p].w1.z, q[p].w0.w, q[p].w1.w, b.z, b.w);
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[n][e] += d[n][e];
            }
          }
          if (it + kPrefetch * kKWarps < n_seg) load(q[p], s0 + it + kPrefetch * kKWarps);
        }
      }
    }
    __syncthreads();
  }

  // the warps' sums, then the cluster's
#pragma unroll
  for (int n = 0; n < MT; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) red[(kw * TOK + n * 8 + 2 * t + (e & 1)) * kRows + rowset * 16 + g + (e >> 1) * 8] = acc[n][e];
  __syncthreads();
  if (kKWarps > 1) {
    for (int i = threadIdx.x; i < Mg * kRows; i += kThreads) {
      float s = red[i];
#pragma unroll
      for (int k = 1; k < kKWarps; ++k) s += red[k * TOK * kRows + i];
      red[i] = s;
    }
    __syncthreads();
  }
  if (S > 1) {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  const int rows = kRows / S;  // that this CTA finishes
  for (int i = threadIdx.x; i < Mg * rows; i += kThreads) {
    const int m = i / rows, r = rank * rows + (i - m * rows);
    const float* p = red + m * kRows + r;
    float s = 0.0f;
    if (S == 1)
      s = *p;
    else
      for (int k = 0; k < S; ++k) s += load_cluster(p, (uint32_t)k);
    const int64_t n = (rb >> 1) * 128 + (r >> 4) * 32 + (rb & 1) * 16 + (r & 15);
    if (n < a.N) {
      if (a.bias) s += bf16_bits_to_float(a.bias[n]);
      if (a.y_f32)
        static_cast<float*>(a.Y)[(m0 + m) * a.ldy + n] = s;
      else
        static_cast<uint16_t*>(a.Y)[(m0 + m) * a.ldy + n] = (uint16_t)bf16x2_of(s, 0.0f);
    }
  }
  if (S > 1) {  // (the others may still read from here)
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
}

template <int MT>
cudaError_t launch_gemv(GemvArgs a, int64_t row_ctas, int S, cudaStream_t st) {
  const int Mg = (int)std::min<int64_t>(a.M, kMaxTokens);
  const int per_cta = (a.n_items + S - 1) / S;
  a.seg = std::max(1, std::min(per_cta, kXBytes / (256 * Mg)));
  const size_t smem = (size_t)a.seg * (256 * Mg + 8 * MT * 4) + (size_t)kKWarps * 8 * MT * kRows * 4;
  const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(gemv_kernel<MT>), smem);
  if (e != cudaSuccess) return e;
  return launch_kernel_cluster_smem(gemv_kernel<MT>, dim3((unsigned)(row_ctas * S), (unsigned)((a.M + kMaxTokens - 1) / kMaxTokens)), (unsigned)S, dim3(kThreads), smem, st, a);
}

}  // namespace

}  // namespace nvfp4

using namespace nvfp4;

extern "C" {

nvfp4_status nvfp4_gemv(const void* X_bf16, int64_t ldx, int64_t M, int64_t D, const nvfp4_operand* W, const int32_t* keep_cols, const int32_t* outlier_cols,
                        int64_t n_out, const void* W_out, const void* bias_bf16, void* Y, int32_t y_dtype, int64_t ldy, void* stream) {
  if (!W) return NVFP4_ERR_NULL;
  if (W->gs_mode < 0 || W->gs_mode > 2 || W->sf_layout < 0 || W->sf_layout > 1 || y_dtype < 0 || y_dtype > 1) return NVFP4_ERR_ENUM;
  if (M < 0 || D <= 0 || n_out < 0 || W->R < 0 || W->K <= 0 || W->K + n_out != D) return NVFP4_ERR_SHAPE;
  if (D > ((int64_t)1 << 30) || W->R > ((int64_t)1 << 31) || M > 65535ll * kMaxTokens) return NVFP4_ERR_LIMIT;
  if (M == 0 || W->R == 0) return NVFP4_OK;
  if (!X_bf16 || !Y || !W->codes || !W->sf || !W->gscale || (n_out > 0 && (!keep_cols || !outlier_cols || !W_out))) return NVFP4_ERR_NULL;
  if (bad_matrix(X_bf16, ldx, D, 2) || bad_matrix(Y, ldy, W->R, y_dtype == NVFP4_DT_F32 ? 4 : 2) || !aligned(W->codes, 16) || !aligned(W->sf, 16) || !aligned(W->gscale, 4) ||
      !aligned(bias_bf16, 2) || (n_out > 0 && (!aligned(W_out, 16) || !aligned(keep_cols, 4) || !aligned(outlier_cols, 4))))
    return NVFP4_ERR_ALIGN;
  if (!device_is_sm100()) return NVFP4_ERR_ARCH;
  GemvArgs a{};
  a.X = static_cast<const uint16_t*>(X_bf16);
  a.ldx = ldx;
  a.M = M;
  a.D = (int)D;
  a.K = (int)W->K;
  a.keep = n_out > 0 ? keep_cols : nullptr;
  a.outl = n_out > 0 ? outlier_cols : nullptr;
  a.n_out = (int)n_out;
  a.Kh = (int)nvfp4_outlier_pad(n_out);
  a.W_out = static_cast<const uint16_t*>(W_out);
  a.codes = W->codes;
  a.sf = W->sf;
  a.gscale = W->gscale;
  a.N = W->R;
  a.gs_mode = W->gs_mode;
  a.tiled = W->sf_layout == NVFP4_SF_TILED128x4;
  a.bias = static_cast<const uint16_t*>(bias_bf16);
  a.Y = Y;
  a.y_f32 = y_dtype == NVFP4_DT_F32;
  a.ldy = ldy;
  a.n_codes = (int)(nvfp4_padded_k(W->K) / 128);
  a.n_items = a.n_codes + (n_out > 0 ? a.Kh / 32 : 0);
  // CTAs along k: as many as give every SM up to four of them, while every warp keeps an item
  const int64_t row_ctas = (W->R + 127) / 128 * 2, most = (int64_t)device_sm_count() * 4;
  int S = 1;
  while (S < kMaxCluster && row_ctas * S * 2 <= most && a.n_items >= 2 * S * kKWarps) S *= 2;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = M <= 8 ? launch_gemv<1>(a, row_ctas, S, st) : M <= 16 ? launch_gemv<2>(a, row_ctas, S, st) : launch_gemv<4>(a, row_ctas, S, st);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? NVFP4_OK : NVFP4_ERR_CUDA;
}

}  // extern "C"
