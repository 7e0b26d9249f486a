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
// A CTA is four warps of 32 rows, a 128-row tile, because that is whose scale bytes lie together. A warp brings its rows' codes and scales
// through a ring of its own in shared memory (asynchronous copies, kStages pieces ahead, no barrier between warps).
// The k axis is split over the CTAs of a cluster, whose sums are added through distributed shared memory in a fixed order, one that M does
// not change.
#include "../../include/nvfp4.h"

#include "act8.cuh"
#include "nvfp4_internal.h"

namespace nvfp4 {

namespace {

constexpr int kRows = 128;       // weight rows of a CTA, 32 of a warp
constexpr int kThreads = 128;
constexpr int kStages = 4;       // pieces in flight per warp
constexpr int kStageBytes = 2048 + 256 + 128;  // 32 rows of 64 bytes, their scales, their global scales
constexpr int kSfAt = 2048, kGsAt = kSfAt + 256;
constexpr int kRingBytes = 4 * kStages * kStageBytes;
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

__device__ __forceinline__ void copy16(uint32_t to, const void* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void copy4(uint32_t to, const void* from) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ uint4 shared16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t shared_u16(uint32_t at) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ float shared_f32(uint32_t at) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
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

template <int MT, bool B128, bool TILED>  // MT: instructions' widths of eight tokens
__global__ void __launch_bounds__(kThreads) gemv_kernel(GemvArgs a) {
  pdl_prologue();
  extern __shared__ __align__(16) uint8_t smem[];
  constexpr int TOK = 8 * MT;
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  uint32_t S, rank, rb;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(S));
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%clusterid.x;" : "=r"(rb));
  const int64_t m0 = (int64_t)blockIdx.y * kMaxTokens;
  const int Mg = (int)min((int64_t)kMaxTokens, a.M - m0);
  const int64_t row_w = (int64_t)rb * kRows + wid * 32;  // the warp's first row
  const int64_t last = a.N - 1;                          // (rows past the end repeat the last one and are not stored)
  const int64_t rs = min(row_w + lane, last);            // whose scales this lane brings
  const int Kp = (a.K + 127) & ~127;
  const int64_t nb = Kp >> 4, nbp = (nb + 15) & ~(int64_t)15;

  uint8_t* xs = smem + kRingBytes;                                             // [piece][4][token][4] 16 bytes, then one piece of zeros
  float* xscale = reinterpret_cast<float*>(xs + (size_t)(a.seg + 1) * 256 * Mg);  // [piece][TOK]
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + wid * (kStages * kStageBytes);
  const uint32_t xs_at = (uint32_t)__cvta_generic_to_shared(xs), xscale_at = (uint32_t)__cvta_generic_to_shared(xscale);

  const int i_begin = (int)(rank * (uint32_t)a.n_items / S), i_end = (int)((rank + 1) * (uint32_t)a.n_items / S);
  const uint8_t *c[4], *o[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t r = min(row_w + g + 8 * j, last);
    c[j] = a.codes + r * (Kp >> 1) + t * 16;
    o[j] = reinterpret_cast<const uint8_t*>(a.W_out) + r * a.Kh * 2 + t * 16;
  }
  const uint8_t* sf = a.sf + (TILED ? (int64_t)sf_tiled_offset(rs, 0, nbp) : rs * nb);
  const float* gs = a.gscale + (B128 ? rs * (Kp >> 7) : 0);
  float gv[4] = {};
  if (!B128)
#pragma unroll
    for (int j = 0; j < 4; ++j) gv[j] = a.gscale[a.gs_mode == kGsRow ? min(row_w + g + 8 * j, last) : 0];

  // piece i into its place in the ring; one group of copies, empty past the end
  auto fetch = [&](int i) {
    if (i < i_end) {
      const uint32_t to = ring + (uint32_t)(i & (kStages - 1)) * kStageBytes;
      if (i < a.n_codes) {
#pragma unroll
        for (int j = 0; j < 4; ++j) copy16(to + j * 512 + lane * 16, c[j] + (int64_t)i * 64);
        copy4(to + kSfAt + lane * 8, sf + (int64_t)i * (TILED ? 1024 : 8));  // four blocks' scales, and the next four's
        copy4(to + kSfAt + lane * 8 + 4, sf + (int64_t)i * (TILED ? 1024 : 8) + (TILED ? 512 : 4));
        if (B128) copy4(to + kGsAt + lane * 4, gs + i);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) copy16(to + j * 512 + lane * 16, o[j] + (int64_t)(i - a.n_codes) * 64);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int p = 0; p < kStages; ++p) fetch(i_begin + p);
  for (int i = threadIdx.x; i < 16 * Mg; i += kThreads) *reinterpret_cast<uint4*>(xs + (size_t)a.seg * 256 * Mg + i * 16) = make_uint4(0, 0, 0, 0);

  // where this lane's X lies in a piece, for each eight tokens; tokens that do not exist are read from the zeros
  uint32_t b_at[MT], b_step[MT];
#pragma unroll
  for (int n = 0; n < MT; ++n) {
    const bool live = n * 8 + g < Mg;
    b_at[n] = xs_at + (live ? ((n * 8 + g) * 4 + t) * 16 : a.seg * 256 * Mg);
    b_step[n] = live ? 256 * Mg : 0;
  }

  float acc[2][MT][4] = {};
  for (int s0 = i_begin; s0 < i_end; s0 += a.seg) {
    const int n_seg = min(a.seg, i_end - s0);
    if (s0 > i_begin) __syncthreads();
    // X: 16 lanes take a token's 128 values of a piece (or the 32 of an outlier step: 4 lanes of them), eight each; kAhead loads at a time
    {
      constexpr int kAhead = 4;
      const int l16 = lane & 15, n_units = n_seg * Mg;
      for (int u0 = wid * 2 + (lane >> 4); u0 - (lane >> 4) < n_units; u0 += kAhead * (kThreads / 16)) {  // (a warp's two halves stay together)
        uint4 w[kAhead];
        int it[kAhead], m[kAhead];
#pragma unroll
        for (int p = 0; p < kAhead; ++p) {
          const int u = u0 + p * (kThreads / 16);
          w[p] = make_uint4(0, 0, 0, 0);
          it[p] = m[p] = 0;
          if (u < n_units) {
            it[p] = Mg == 1 ? u : u / Mg;
            m[p] = u - it[p] * Mg;
            const int i = s0 + it[p];
            const uint16_t* row = a.X + (m0 + m[p]) * a.ldx;
            if (i < a.n_codes)
              w[p] = x8(row, a.keep, i * 128 + l16 * 8, a.K, a.D);
            else if (l16 < 4)
              w[p] = x8(row, a.outl, (i - a.n_codes) * 32 + l16 * 8, a.n_out, a.D);
          }
        }
#pragma unroll
        for (int p = 0; p < kAhead; ++p) {
          const int u = u0 + p * (kThreads / 16);
          const uint32_t m2 = amax16x2(amax16x2(w[p].x, w[p].y), amax16x2(w[p].z, w[p].w));
          uint32_t big = max(m2 & 0x7FFFu, (m2 >> 16) & 0x7FFFu);  // (bit patterns of magnitudes are ordered like them)
#pragma unroll
          for (int o = 1; o < 16; o <<= 1) big = max(big, __shfl_xor_sync(0xFFFFFFFFu, big, o));
          if (u >= n_units) continue;
          const uint32_t e = max(big >> 7, 15u);
          uint8_t* at = xs + (size_t)it[p] * 256 * Mg;
          if (s0 + it[p] < a.n_codes) {
            const float to = __uint_as_float((268u - e) << 23);  // 2^(141 - e)
            const uint32_t wj[4] = {w[p].x, w[p].y, w[p].z, w[p].w};
            uint32_t h[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float2 v = values_of(mul2(bf16_pair(wj[j]), pair_of(to)));
              const __half2 q = __floats2half2_rn(v.x, v.y);
              h[j] = *reinterpret_cast<const uint32_t*>(&q);
            }
            *reinterpret_cast<uint4*>(at + (((l16 & 3) * Mg + m[p]) * 4 + (l16 >> 2)) * 16) = make_uint4(h[0], h[1], h[2], h[3]);
            if (l16 == 0) xscale[it[p] * TOK + m[p]] = __uint_as_float((e - 14u) << 23);  // 2^(e - 141)
          } else if (l16 < 4) {
            *reinterpret_cast<uint4*>(at + (m[p] * 4 + l16) * 16) = w[p];
          }
        }
      }
    }
    __syncthreads();
    uint32_t b_now[MT];
#pragma unroll
    for (int n = 0; n < MT; ++n) b_now[n] = b_at[n];
    uint32_t xsc_now = xscale_at + 8 * t;
    const int s_codes = min(s0 + n_seg, a.n_codes);
    int i = s0;
#pragma unroll 1
    for (; i < s_codes; ++i) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
      __syncwarp();
      const uint32_t at = ring + (uint32_t)(i & (kStages - 1)) * kStageBytes;
      uint32_t wv[4][4], sc[4][2];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint4 w = shared16(at + j * 512 + lane * 16);
        wv[j][0] = w.x; wv[j][1] = w.y; wv[j][2] = w.z; wv[j][3] = w.w;
        scales2(shared_u16(at + kSfAt + (g + 8 * j) * 8 + t * 2), sc[j]);
        if (B128) gv[j] = shared_f32(at + kGsAt + (g + 8 * j) * 4);
      }
      __syncwarp();
      fetch(i + kStages);
      float d[2][MT][4] = {};
#pragma unroll
      for (int wd = 0; wd < 4; ++wd) {
        uint32_t h[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) weights8(wv[j][wd], sc[j][wd >> 1], h[j]);
#pragma unroll
        for (int n = 0; n < MT; ++n) {
          const uint4 b = shared16(b_now[n] + (uint32_t)(wd * Mg) * 64);
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            mma_f16(d[k][n], h[2 * k][0], h[2 * k + 1][0], h[2 * k][1], h[2 * k + 1][1], b.x, b.y);
            mma_f16(d[k][n], h[2 * k][2], h[2 * k + 1][2], h[2 * k][3], h[2 * k + 1][3], b.z, b.w);
          }
        }
      }
#pragma unroll
      for (int n = 0; n < MT; ++n) {
        const float x0 = shared_f32(xsc_now + n * 32), x1 = shared_f32(xsc_now + n * 32 + 4);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          acc[k][n][0] = fmaf(d[k][n][0], x0 * gv[2 * k], acc[k][n][0]);
          acc[k][n][1] = fmaf(d[k][n][1], x1 * gv[2 * k], acc[k][n][1]);
          acc[k][n][2] = fmaf(d[k][n][2], x0 * gv[2 * k + 1], acc[k][n][2]);
          acc[k][n][3] = fmaf(d[k][n][3], x1 * gv[2 * k + 1], acc[k][n][3]);
        }
        b_now[n] += b_step[n];
      }
      xsc_now += TOK * 4;
    }
#pragma unroll 1
    for (; i < s0 + n_seg; ++i) {  // outlier channels
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
      __syncwarp();
      const uint32_t at = ring + (uint32_t)(i & (kStages - 1)) * kStageBytes;
      uint4 w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = shared16(at + j * 512 + lane * 16);
      __syncwarp();
      fetch(i + kStages);
#pragma unroll
      for (int n = 0; n < MT; ++n) {
        const uint4 b = shared16(b_now[n]);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float d[4] = {};
          mma_bf16(d, w[2 * k].x, w[2 * k + 1].x, w[2 * k].y, w[2 * k + 1].y, b.x, b.y);
          mma_bf16(d, w[2 * k].z, w[2 * k + 1].z, w[2 * k].w, w[2 * k + 1].w, b.z, b.w);
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[k][n][e] += d[e];
        }
        b_now[n] += b_step[n];
      }
    }
  }

  // the cluster's sums, where the rings were
  __syncthreads();
  float* red = reinterpret_cast<float*>(smem);  // [TOK][kRows]
#pragma unroll
  for (int n = 0; n < MT; ++n)
#pragma unroll
    for (int e = 0; e < 8; ++e) red[(n * 8 + 2 * t + (e & 1)) * kRows + wid * 32 + g + (e >> 1) * 8] = acc[e >> 2][n][e & 3];
  __syncthreads();
  if (S > 1) {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  for (int i = rank * kThreads + threadIdx.x; i < Mg * kRows; i += S * kThreads) {
    const int m = i / kRows, r = i % kRows;
    const float* p = red + m * kRows + r;
    float s = 0.0f;
    if (S == 1)
      s = *p;
    else
      for (uint32_t k = 0; k < S; ++k) s += load_cluster(p, k);
    const int64_t n = (int64_t)rb * kRows + r;
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

template <int MT, bool B128, bool TILED>
cudaError_t launch_gemv(GemvArgs a, int64_t row_ctas, int S, cudaStream_t st) {
  const int Mg = (int)std::min<int64_t>(a.M, kMaxTokens);
  const int per_cta = (a.n_items + S - 1) / S;
  a.seg = std::max(1, std::min(per_cta, kXBytes / (256 * Mg)));
  const size_t smem = kRingBytes + (size_t)(a.seg + 1) * 256 * Mg + (size_t)a.seg * 8 * MT * 4;
  auto kernel = gemv_kernel<MT, B128, TILED>;
  const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), smem);
  if (e != cudaSuccess) return e;
  return launch_kernel_cluster_smem(kernel, dim3((unsigned)(row_ctas * S), (unsigned)((a.M + kMaxTokens - 1) / kMaxTokens)), (unsigned)S, dim3(kThreads), smem, st, a);
}
template <int MT>
cudaError_t launch_gemv(const GemvArgs& a, int64_t row_ctas, int S, cudaStream_t st) {
  if (a.gs_mode == kGsBlock128) return a.tiled ? launch_gemv<MT, true, true>(a, row_ctas, S, st) : launch_gemv<MT, true, false>(a, row_ctas, S, st);
  return a.tiled ? launch_gemv<MT, false, true>(a, row_ctas, S, st) : launch_gemv<MT, false, false>(a, row_ctas, S, st);
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
  // CTAs along k
  const int64_t row_ctas = (W->R + kRows - 1) / kRows, sms = device_sm_count();
  int S = 1;
  while (S < kMaxCluster && row_ctas * S * 2 <= sms * 4 && a.n_items >= 2 * S) S *= 2;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = M <= 8 ? launch_gemv<1>(a, row_ctas, S, st) : M <= 16 ? launch_gemv<2>(a, row_ctas, S, st) : launch_gemv<4>(a, row_ctas, S, st);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? NVFP4_OK : NVFP4_ERR_CUDA;
}

}  // extern "C"
