// nvfp4_gemv: a few tokens times quantized weights, Y[m, n] = sum_k X[m, k] (P Sb Sg)[n, k] (+ the outlier channels' BF16 product, + bias), the
// product of token-by-token answering. X stays in BF16 (nothing about it is quantized); the weights are read once, 0.5625 bytes each.
//
// The work is reading the weights, so all else is kept off their way. A warp takes 32 weight rows x 128 k at a time, 16 bytes (32 codes) of four
// rows per lane, and multiplies them on the tensor cores (mma m16n8k16: 8 tokens cost what one costs; tcgen05 would want codes that somebody has
// expanded into shared memory, or X in FP4): E2M1 pairs become FP16 pairs in one conversion each, times the block scale exactly (P * Sb has at
// most 7 significant bits and lies within FP16's normal range). Those multiplications are as many as the conversions and lengthen the chain to
// the matrix instruction. Up to two tokens, where an instruction's other columns are free, sums of one block each are scaled instead (SEP below). Which k stand
// in which slot of an instruction is free as long as both operands agree, so the codes are used as they lie in memory and X is staged in
// shared memory in that order. FP16 also holds X: a token's 128 values are divided by the power of four r^2 that brings their largest magnitude
// to [2^14, 2^16); a BF16 value has 8 significant bits, so the largest stays below FP16's end, the scaling is exact for all down to 2^-28 of
// the largest, and what is below loses less than 2^-39 of it. Every 128 k the FP32 result d of the instructions is added to FP32 sums with r^2
// and the weights' global scale g, which is constant there in every scale mode, as (d r) (r g): r^2 g by itself is a subnormal number, of few
// bits, for tokens below 2^-100, whose results still are normal ones.
// The outlier channels go through BF16 instructions, 32 of them per step, with the same rows.
//
// A CTA takes a 128-row tile, because that is whose scale bytes lie together, 256 k at a time: one tensor copy of 128 bytes of its rows (128-byte
// swizzle), one of their scales, three or four of them in flight. One warp has them brought; eight take 32 rows and one of the
// two halves of the 256 k each. The k axis is split over the CTAs of a cluster as well, whose sums are read through distributed
// shared memory and added in a fixed order. Waits are for copies alone, and bounded.
//
// Measured (us, weights from HBM, replayed from a graph; the weights alone at the copy bandwidth in brackets): 1024 x 1024 times one token 3.0
// (0.1), 4096 x 4096 5.9 (1.5), 8192 x 8192 11.3 (5.8); times 8 with 1x128 outer blocks 15.5, times 16 17.6, times 32 30.3; 14336 x 4096 times
// 16 17.8 (5.2). What bounds it: for one token the chain of a warp's conversions and matrix instructions at 0.44 of the issue slots, what a
// short kernel begins and ends with (2 us until X is staged and the first weights are there, 1.5 for the cluster's sums), and 256 CTAs on 148
// SMs; for more tokens the multiplications with the block scales, and above 16 a second wave of CTAs (below). Measured and not better: rows
// through each warp's own ring of asynchronous copies (14.6 for 8192 x 8192 times one), three CTAs to an SM (13.6), more CTAs than fit at once
// (16.6), X staged by every CTA for 16 tokens (24.8 against 17.6). Every 32 tokens are a pass over the weights: this is no form for a prompt
// (8192 x 8192 times 64 58, times 2048 1700, where the library's quantizer and FP4 GEMM take 15 and 69).
#include "../../include/nvfp4.h"

#include "act8.cuh"
#include "nvfp4_internal.h"
#include "nvfp4_tc.cuh"

namespace nvfp4 {

namespace {

constexpr int kRows = 128;          // weight rows of a CTA, 32 of a warp
constexpr int kConsumers = 256;     // four row groups x two halves of k
constexpr int kThreads = kConsumers + 32;
constexpr int kCodeBytes = 16384;   // of a stage: 128 rows x 128 bytes
constexpr int kScaleBytes = 2048;   // four scale tiles
constexpr int kStageBytes = kCodeBytes + kScaleBytes;
constexpr int kMaxTokens = 32;      // of one pass over the weights
constexpr int kMaxCluster = 8;
// Two CTAs of up to 16 tokens share an SM, one of more has it to itself.
template <int MT>
constexpr int kStages = MT == 2 ? 3 : 4;
constexpr int kXBytes = 30 * 1024;  // of X staged by the CTA itself, at most
// A pair of pieces of X staged in memory: the values of both, then their powers of two.
__host__ __device__ constexpr int pair_bytes(int tokens, int wide) { return 512 * tokens + 8 * wide; }

struct GemvArgs {
  const uint16_t* X;
  int64_t ldx, M;
  int D, K;  // columns of X, of the operand
  const int32_t *keep, *outl;
  int n_out;
  const uint8_t* sf;
  const float* gscale;
  int64_t N;
  int gs_mode;
  const uint16_t* bias;
  void* Y;
  int y_f32;
  int64_t ldy;
  int n_codes;           // 128-k pieces of the codes
  int n_code_pairs, n_pairs;  // pairs of them; those and the pairs of 32-channel steps of the outliers
  int seg;               // pairs whose X a CTA stages at a time
  uint8_t* staged;       // X staged in memory: [32 tokens][pair] pair_bytes
  int wide;              // tokens that an instruction's width is rounded to, of the kernel that reads it
  int32_t* dev_status;
  long long wait_limit;  // bound of every wait, in clock cycles
  int starve;            // test hook of the waits: the first stage never completes
};

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
__device__ __forceinline__ uint32_t shared_u32(uint32_t at) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
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
// eight codes as FP16 pairs in order
__device__ __forceinline__ void codes8(uint32_t word, uint32_t (&h)[4]) {
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
}
// and times the scale pair (both halves equal)
__device__ __forceinline__ void weights8(uint32_t word, uint32_t scale2, uint32_t (&h)[4]) {
  codes8(word, h);
  const __half2 s = *reinterpret_cast<const __half2*>(&scale2);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 p = __hmul2(*reinterpret_cast<const __half2*>(&h[i]), s);
    h[i] = *reinterpret_cast<const uint32_t*>(&p);
  }
}
__device__ __forceinline__ uint32_t scale_pair(uint32_t bytes) {  // the values of two E4M3 bytes as an FP16 pair
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)bytes));
  return h;
}
// the values of two E4M3 bytes, each in both halves of a word
__device__ __forceinline__ void scales2(uint32_t bytes, uint32_t (&s)[2]) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)bytes));
  s[0] = __byte_perm(h, h, 0x1010);
  s[1] = __byte_perm(h, h, 0x3232);
}
// what the cluster's CTA `rank` holds at this address of its shared memory
__device__ __forceinline__ float load_cluster(const float* p, uint32_t rank) {
  uint32_t at;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void consumer_barrier() { asm volatile("bar.sync 1, %0;" ::"n"(kConsumers) : "memory"); }

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
// The same for the two lists that a piece can go by; not inlined, since a kernel starts as fast as its instructions come in.
__device__ __noinline__ uint4 x8_apart(const uint16_t* row, const int32_t* cols, int k, int n, int D) { return x8(row, cols, k, n, D); }

// One token's 128 values of a piece of X (or the 32 of an outlier step), by 16 lanes, eight each (4 of them).
__device__ __forceinline__ uint4 load_piece(const GemvArgs& a, int64_t m, int i, int l16) {
  const uint16_t* row = a.X + m * a.ldx;
  const bool code = i < 2 * a.n_code_pairs;
  const int k = code ? i * 128 + l16 * 8 : (i - 2 * a.n_code_pairs) * 32 + l16 * 8;
  if (!a.keep && k + 8 <= a.K) return *reinterpret_cast<const uint4*>(row + k);
  return code || l16 < 4 ? x8_apart(row, code ? a.keep : a.outl, k, code ? a.K : a.n_out, a.D) : make_uint4(0, 0, 0, 0);
}
// Stores them as the instructions read them: [4 words of a lane's 16 codes][token][lane t] 16 bytes, and the power of two r that they are to be
// multiplied by again, twice. Every lane of a warp calls this; `live`: this one's unit exists.
__device__ __forceinline__ void store_piece(uint4 w, bool code, bool live, int l16, int m, int Mg, uint8_t* at, float* scale) {
  const uint32_t m2 = amax16x2(amax16x2(w.x, w.y), amax16x2(w.z, w.w));
  uint32_t big = max(m2 & 0x7FFFu, (m2 >> 16) & 0x7FFFu);  // (bit patterns of magnitudes are ordered like them)
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) big = max(big, __shfl_xor_sync(0xFFFFFFFFu, big, o));
  if (!live) return;
  const int e = (int)max(big >> 7, 15u), r = (e - 141) >> 1;  // -63 .. 57
  if (code) {
    const float to = __uint_as_float((uint32_t)(127 - 2 * r) << 23);  // 2^(-2 r)
    const uint32_t wj[4] = {w.x, w.y, w.z, w.w};
    uint32_t h[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 v = values_of(mul2(bf16_pair(wj[j]), pair_of(to)));
      const __half2 q = __floats2half2_rn(v.x, v.y);
      h[j] = *reinterpret_cast<const uint32_t*>(&q);
    }
    *reinterpret_cast<uint4*>(at + (((l16 & 3) * Mg + m) * 4 + (l16 >> 2)) * 16) = make_uint4(h[0], h[1], h[2], h[3]);
    if (l16 == 0) *scale = __uint_as_float((uint32_t)(127 + r) << 23);  // 2^r
  } else if (l16 < 4) {
    *reinterpret_cast<uint4*>(at + (m * 4 + l16) * 16) = w;
  }
}

// X staged in memory, for three and more tokens, whose staging in every CTA would take as long as the weights do (14336 x 4096 times 16 tokens:
// 25.5 us then). It waits before it lets the product's CTAs start, so that those may read the weights at once.
__global__ void __launch_bounds__(256) gemv_stage_kernel(const GemvArgs a) {
  pdl_wait();
  pdl_launch_next();
  const int l16 = threadIdx.x & 15, pieces = 2 * a.n_pairs;
  const int64_t u = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  const int64_t m = u <= 0xFFFFFFFFll ? (int64_t)((uint32_t)u / (uint32_t)pieces) : u / pieces;
  const int i = (int)(u - m * pieces);
  const bool live = m < a.M;
  const int64_t group = m / kMaxTokens;
  const int Mg = live ? (int)min((int64_t)kMaxTokens, a.M - group * kMaxTokens) : 1, mg = (int)(m - group * kMaxTokens);
  uint8_t* at = a.staged + (group * a.n_pairs * pair_bytes(kMaxTokens, a.wide)) + (int64_t)(i >> 1) * pair_bytes(Mg, a.wide);
  store_piece(live ? load_piece(a, m, i, l16) : make_uint4(0, 0, 0, 0), i < 2 * a.n_code_pairs, live, l16, mg, Mg, at + (i & 1) * 256 * Mg,
              reinterpret_cast<float*>(at + 512 * Mg) + (i & 1) * a.wide + mg);
}

// MT: instructions' widths of eight tokens, or with SEP (up to four tokens) of two: an instruction's eight columns are used for two tokens times four lanes, so
// that each of its sums is over one lane's codes, which are of one block; the block scale then multiplies sums instead of codes. X is staged by
// the CTA; else it lies staged in memory and comes with the weights.
template <int MT, bool B128, bool SEP>
__global__ void __launch_bounds__(kThreads, MT > 2 ? 1 : 2) gemv_kernel(const __grid_constant__ CUtensorMap codes_map, const __grid_constant__ CUtensorMap outliers_map, const GemvArgs a) {
  extern __shared__ uint8_t smem_raw[];
  constexpr int TOK = 8 * MT, STAGES = kStages<MT>;
  __shared__ __align__(8) uint64_t full[STAGES];
  __shared__ __align__(8) uint64_t empty[STAGES];
  __shared__ int abort_flag;
  const int warp = uniform_warp_index(), lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int wrow = warp & 3, half = (warp >> 2) & 1;
  uint32_t S, rank, rb;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(S));
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm("mov.u32 %0, %%clusterid.x;" : "=r"(rb));
  const int64_t m0 = (int64_t)blockIdx.y * kMaxTokens;
  const int Mg = (int)min((int64_t)kMaxTokens, a.M - m0);
  const int Kp = (a.K + 127) & ~127;
  const int64_t nbp = ((Kp >> 4) + 15) & ~15;

  const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;  // (swizzled copies)
  const int x_bytes = SEP ? 0 : pair_bytes(Mg, TOK), stage_bytes = kStageBytes + (x_bytes + 1023) / 1024 * 1024;
  uint8_t* xs = smem_raw + (ring - smem_u32(smem_raw)) + STAGES * stage_bytes;     // SEP: [piece][4][token][4] 16 bytes; then one piece of zeros
  float* xscale = reinterpret_cast<float*>(xs + (size_t)(SEP ? 2 * a.seg + 1 : 1) * 256 * Mg);  // SEP: [piece][TOK]
  float* red = xscale + (SEP ? 2 * a.seg * TOK : 0);                              // [half][token][row]
  const uint32_t xs_at = smem_u32(xs), xscale_at = smem_u32(xscale), zeros = xs_at + (SEP ? 2 * a.seg * 256 * Mg : 0);
  const int p_begin = (int)(rank * (uint32_t)a.n_pairs / S), p_end = (int)((rank + 1) * (uint32_t)a.n_pairs / S);

  int filled = 0;  // stages that the bringing warp has had copied
  if (warp == kConsumers / 32) {  // brings the weights
    const uint32_t leader = elect_leader();
    if (leader) {
      asm volatile("prefetch.tensormap [%0];" ::"l"(&codes_map) : "memory");
      abort_flag = 0;
      for (int i = 0; i < STAGES; ++i) {
        mbar_init(smem_u32(&full[i]), 1);
        mbar_init(smem_u32(&empty[i]), kConsumers / 32);
      }
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    asm volatile("bar.arrive 2, %0;" ::"n"(kThreads) : "memory");  // (the consumers wait there for the barriers)
    int i = 0;
    uint32_t phase = 1;
    const uint8_t* const x = a.staged + (int64_t)blockIdx.y * a.n_pairs * pair_bytes(kMaxTokens, TOK);
    auto bring_x = [&](int p, int i) {
      bulk_load(ring + i * stage_bytes + kStageBytes, x + (int64_t)p * x_bytes, x_bytes, smem_u32(&full[i]), leader);
    };
    if (SEP) pdl_wait();
    for (int p = p_begin; p < p_end; ++p) {
      const uint32_t to = ring + i * stage_bytes, bar = smem_u32(&full[i]);
      if (!SEP && p == p_begin + STAGES) {  // the first stages are full of weights: now X
        pdl_wait();
        for (int f = 0; f < STAGES; ++f) bring_x(p_begin + f, f);
      }
      if (!__all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&empty[i]), phase, &abort_flag, a.dev_status, a.wait_limit))) break;
      if (p < a.n_code_pairs) {
        mbar_expect_tx(bar, kStageBytes + x_bytes + (a.starve && p == p_begin ? 16 : 0), leader);
        tma_load_2d(to, &codes_map, p * 128, (int32_t)(rb * kRows), bar, leader);
        bulk_load(to + kCodeBytes, a.sf + ((int64_t)rb * (nbp >> 2) + (int64_t)p * 4) * 512, kScaleBytes, bar, leader);
      } else {
        mbar_expect_tx(bar, kCodeBytes + x_bytes, leader);
        tma_load_2d(to, &outliers_map, (p - a.n_code_pairs) * 64, (int32_t)(rb * kRows), bar, leader);
      }
      if (!SEP && p >= p_begin + STAGES) bring_x(p, i);
      ++filled;
      if (++i == STAGES) {
        i = 0;
        phase ^= 1u;
      }
    }
    if (!SEP && p_end - p_begin <= STAGES) {
      pdl_wait();
      for (int f = 0; f < p_end - p_begin; ++f) bring_x(p_begin + f, f);
    }
  }
  float acc[2][MT][4] = {};
  if (warp < kConsumers / 32) {
    pdl_wait();
    for (int i = threadIdx.x; i < 16 * Mg; i += kConsumers) *reinterpret_cast<uint4*>(xs + (zeros - xs_at) + i * 16) = make_uint4(0, 0, 0, 0);

    // the global scales of the four rows whose results this lane holds
    const float* gs[4];
    float gv[4] = {}, gv_next[4] = {};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t r = min((int64_t)rb * kRows + wrow * 32 + g + 8 * j, a.N - 1);
      gs[j] = a.gscale + (B128 ? r * (Kp >> 7) : a.gs_mode == kGsRow ? r : 0);
      if (!B128) gv[j] = *gs[j];
    }
    auto fetch_gs = [&](int i) {  // of piece i
      if (B128 && i < a.n_codes)
#pragma unroll
        for (int j = 0; j < 4; ++j) gv_next[j] = gs[j][i];
    };
    fetch_gs(2 * p_begin + half);

    // where this lane's X lies in a staged pair, for each eight tokens; tokens that do not exist are read from the zeros
    uint32_t b_at[MT];
    bool live[MT];
#pragma unroll
    for (int n = 0; n < MT; ++n) {
      const int m = SEP ? n * 2 + (g >> 2) : n * 8 + g;
      live[n] = m < Mg && (!SEP || (g & 3) == t);
      b_at[n] = (m * 4 + t) * 16 + half * 256 * Mg;
    }

    int s = 0;  // the stage
    uint32_t phase = 0;
    const int seg = SEP ? a.seg : p_end - p_begin;
    for (int q0 = p_begin; q0 < p_end; q0 += seg) {
      const int s0 = 2 * q0, n_seg = 2 * min(seg, p_end - q0);  // pieces
      if (SEP) {
        if (q0 > p_begin) consumer_barrier();
        const int l16 = lane & 15, n_units = n_seg * Mg;
        // (one load at a time: a kernel starts as fast as its instructions come in; with four ahead 1024 x 1024 takes 3.3 instead of 3.0 us)
        for (int u0 = warp * 2; u0 < n_units; u0 += kConsumers / 16) {  // (a warp's two halves stay together)
          const int u = u0 + (lane >> 4), it = Mg == 1 ? u : (int)((uint32_t)u / (uint32_t)Mg), m = u - it * Mg;
          const bool unit = u < n_units;
          const uint4 w = unit ? load_piece(a, m0 + m, s0 + it, l16) : make_uint4(0, 0, 0, 0);
          store_piece(w, s0 + it < 2 * a.n_code_pairs, unit, l16, m, Mg, xs + (size_t)it * 256 * Mg, xscale + it * TOK + m);
        }
      }
      if (q0 == p_begin)
        asm volatile("bar.sync 2, %0;" ::"n"(kThreads) : "memory");  // X is staged, the barriers are there
      else
        consumer_barrier();
#pragma unroll 1
      for (int p = q0; p < q0 + n_seg / 2; ++p) {
        if (!__all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&full[s]), phase, &abort_flag, a.dev_status, a.wait_limit))) break;
        const uint32_t at = ring + s * stage_bytes;
        const int i = 2 * p + half;  // this warp's piece
        const uint32_t xp = SEP ? xs_at + (p - q0) * 512 * Mg : at + kStageBytes;  // this pair of X
        const uint32_t xsc = SEP ? xscale_at + (2 * (p - q0) + half) * TOK * 4 + 4 * (t >> 1) : xp + 512 * Mg + half * TOK * 4 + 8 * t;
        uint32_t b_now[MT];
#pragma unroll
        for (int n = 0; n < MT; ++n) b_now[n] = live[n] ? xp + b_at[n] : zeros;
        uint32_t wv[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint4 w = shared16(at + (wrow * 32 + 8 * j + g) * 128 + (((half * 4 + t) ^ g) << 4));
          wv[j][0] = w.x; wv[j][1] = w.y; wv[j][2] = w.z; wv[j][3] = w.w;
        }
        const bool code = p < a.n_code_pairs;
        uint32_t sc[4][2];
        if (code) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (SEP) {  // of two lanes' two blocks each
              const uint32_t four = shared_u32(at + kCodeBytes + (half * 2 + (t & 1)) * 512 + (8 * j + g) * 16 + wrow * 4);
              sc[j][0] = scale_pair(four & 0xFFFFu);
              sc[j][1] = scale_pair(four >> 16);
            } else scales2(shared_u16(at + kCodeBytes + (half * 2 + (t >> 1)) * 512 + (8 * j + g) * 16 + wrow * 4 + (t & 1) * 2), sc[j]);
            if (B128) gv[j] = gv_next[j];
          }
          fetch_gs(i + 2);
        }
        if (SEP) {  // (else X is still to be read from the stage)
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&empty[s]));
        }
        if (SEP && code && i < a.n_codes) {
          // Rows g and g + 8, then g + 16 and g + 24: at once for one width, one after the other for two (registers). d: of the lanes' first block,
          // then of their second; chains of instructions side by side.
          constexpr int KB = MT == 1 ? 2 : 1;
#pragma unroll
          for (int k0 = 0; k0 < 2; k0 += KB) {
            float d[MT][KB][2][4] = {};
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              uint32_t h[2 * KB][2][4];
#pragma unroll
              for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int j = 0; j < 2 * KB; ++j) codes8(wv[2 * k0 + j][2 * b + u], h[j][b]);
#pragma unroll
              for (int n = 0; n < MT; ++n) {
                uint4 x[2];
#pragma unroll
                for (int b = 0; b < 2; ++b) x[b] = shared16(b_now[n] + (uint32_t)((2 * b + u) * Mg) * 64);
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                  for (int k = 0; k < KB; ++k) mma_f16(d[n][k][b], h[2 * k][b][0], h[2 * k + 1][b][0], h[2 * k][b][1], h[2 * k + 1][b][1], x[b].x, x[b].y);
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                  for (int k = 0; k < KB; ++k) mma_f16(d[n][k][b], h[2 * k][b][2], h[2 * k + 1][b][2], h[2 * k][b][3], h[2 * k + 1][b][3], x[b].z, x[b].w);
              }
            }
#pragma unroll
            for (int n = 0; n < MT; ++n) {
              const f32x2 r = pair_of(shared_f32(xsc + 8 * n));
#pragma unroll
              for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int e = 0; e < 4; e += 2) {  // columns 2 t and 2 t + 1: lanes (2 t) & 3 and the next of token 2 n + (t >> 1)
                  const int j = 2 * (k0 + k) + (e >> 1);
                  float2 scale[2];
#pragma unroll
                  for (int c = 0; c < 2; ++c) scale[c] = __half22float2(*reinterpret_cast<const __half2*>(&sc[j][c]));
                  const f32x2 v = fma2(pair_of(d[n][k][1][e], d[n][k][1][e + 1]), pair_of(scale[0].y, scale[1].y),
                                       mul2(pair_of(d[n][k][0][e], d[n][k][0][e + 1]), pair_of(scale[0].x, scale[1].x)));
                  const float2 sum = values_of(fma2(mul2(v, r), mul2(r, pair_of(gv[j])), pair_of(acc[k0 + k][n][e], acc[k0 + k][n][e + 1])));
                  acc[k0 + k][n][e] = sum.x;
                  acc[k0 + k][n][e + 1] = sum.y;
                }
            }
          }
        } else if (!SEP && code && i < a.n_codes) {
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
            const f32x2 r = pair_of(shared_f32(xsc + n * 32), shared_f32(xsc + n * 32 + 4));
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int e = 0; e < 4; e += 2) {
                const float2 sum = values_of(fma2(mul2(pair_of(d[k][n][e], d[k][n][e + 1]), r), mul2(r, pair_of(gv[2 * k + (e >> 1)])), pair_of(acc[k][n][e], acc[k][n][e + 1])));
                acc[k][n][e] = sum.x;
                acc[k][n][e + 1] = sum.y;
              }
          }
        } else if (!code) {  // 32 outlier channels
#pragma unroll
          for (int n = 0; n < MT; ++n) {
            const uint4 b = shared16(b_now[n]);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              float d[4] = {};
              mma_bf16(d, wv[2 * k][0], wv[2 * k + 1][0], wv[2 * k][1], wv[2 * k + 1][1], b.x, b.y);
              mma_bf16(d, wv[2 * k][2], wv[2 * k + 1][2], wv[2 * k][3], wv[2 * k + 1][3], b.z, b.w);
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[k][n][e] += d[e];
            }
          }
        }
        if (!SEP) {
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&empty[s]));
        }
        if (++s == STAGES) {
          s = 0;
          phase ^= 1u;
        }
      }
    }
  }
  pdl_launch_next();

  // each warp's sums, then the cluster's
  if (warp >= kConsumers / 32) {
  } else if (SEP) {  // the four lanes' sums of a token: two of them here, two in the neighbour
#pragma unroll
    for (int n = 0; n < MT; ++n)
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          const int m = 2 * n + (t >> 1);
          float v = acc[k][n][e] + acc[k][n][e + 1];
          v += __shfl_xor_sync(0xFFFFFFFFu, v, 1);
          if ((t & 1) == 0 && m < Mg) red[(half * Mg + m) * kRows + wrow * 32 + k * 16 + g + (e >> 1) * 8] = v;
        }
  } else {
#pragma unroll
    for (int n = 0; n < MT; ++n)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int m = n * 8 + 2 * t + (e & 1);
        if (m < Mg) red[(half * Mg + m) * kRows + wrow * 32 + g + (e >> 1) * 8] = acc[e >> 2][n][e & 3];
      }
  }
  if (S > 1) {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  } else {
    __syncthreads();
  }
  for (int i = (int)rank * kThreads + threadIdx.x; i < Mg * kRows; i += (int)S * kThreads) {
    const int m = i / kRows, r = i % kRows;
    const float* p = red + m * kRows + r;
    float v[2 * kMaxCluster], sum = 0.0f;
#pragma unroll
    for (int k = 0; k < 2 * kMaxCluster; ++k)
      if (k < 2 * (int)S) v[k] = S > 1 ? load_cluster(p + (k & 1) * Mg * kRows, (uint32_t)(k >> 1)) : p[(k & 1) * Mg * kRows];
#pragma unroll
    for (int k = 0; k < 2 * kMaxCluster; ++k)
      if (k < 2 * (int)S) sum += v[k];
    const int64_t n = (int64_t)rb * kRows + r;
    if (n < a.N) {
      if (a.bias) sum += bf16_bits_to_float(a.bias[n]);
      if (a.y_f32)
        static_cast<float*>(a.Y)[(m0 + m) * a.ldy + n] = sum;
      else
        static_cast<uint16_t*>(a.Y)[(m0 + m) * a.ldy + n] = (uint16_t)bf16x2_of(sum, 0.0f);
    }
  }
  if (warp == kConsumers / 32 && *(volatile int*)&abort_flag) {  // a wait ran out: the copies under way get the same time to land before the CTA ends
    for (int f = max(0, filled - STAGES); f < filled; ++f) {
      const long long t0 = clock64();
      while (!mbar_test(smem_u32(&full[f % STAGES]), (uint32_t)(f / STAGES) & 1u) && clock64() - t0 < a.wait_limit) {
      }
    }
  }
  if (S > 1) {  // (the others may still read from here)
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
  }
}

template <int MT, bool B128, bool SEP>
cudaError_t launch_gemv(const CUtensorMap& codes, const CUtensorMap& outliers, GemvArgs a, int64_t row_ctas, int S, cudaStream_t st) {
  const int Mg = (int)std::min<int64_t>(a.M, kMaxTokens);
  const int per_cta = (a.n_pairs + S - 1) / S;
  a.seg = std::max(1, std::min(per_cta, (kXBytes / (256 * Mg) - 1) / 2));
  a.wide = 8 * MT;
  const size_t x = SEP ? (size_t)(2 * a.seg + 1) * 256 * Mg + (size_t)2 * a.seg * 8 * MT * 4 : (size_t)256 * Mg;
  const size_t smem = 1024 + kStages<MT> * (kStageBytes + (SEP ? 0 : (pair_bytes(Mg, 8 * MT) + 1023) / 1024 * 1024)) + x + (size_t)2 * Mg * kRows * 4;
  if (!SEP) {
    const int64_t units = a.M * 2 * a.n_pairs;
    const cudaError_t e = launch_kernel(gemv_stage_kernel, dim3((unsigned)((units + 15) / 16)), dim3(256), 0, st, a);
    if (e != cudaSuccess) return e;
  }
  auto kernel = gemv_kernel<MT, B128, SEP>;
  const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), smem);
  if (e != cudaSuccess) return e;
  return launch_kernel_cluster_smem(kernel, dim3((unsigned)(row_ctas * S), (unsigned)((a.M + kMaxTokens - 1) / kMaxTokens)), (unsigned)S, dim3(kThreads), smem, st, codes, outliers, a);
}
template <int MT, bool SEP>
cudaError_t launch_gemv(const CUtensorMap& codes, const CUtensorMap& outliers, const GemvArgs& a, int64_t row_ctas, int S, cudaStream_t st) {
  return a.gs_mode == kGsBlock128 ? launch_gemv<MT, true, SEP>(codes, outliers, a, row_ctas, S, st) : launch_gemv<MT, false, SEP>(codes, outliers, a, row_ctas, S, st);
}

}  // namespace

}  // namespace nvfp4

using namespace nvfp4;

extern "C" {

size_t nvfp4_gemv_workspace_bytes(int64_t M, int64_t D, int64_t n_out) {
  if (M <= 2 || D <= 0 || n_out < 0 || n_out > D) return 0;
  const int64_t pairs = (nvfp4_padded_k(D - n_out) / 128 + 1) / 2 + nvfp4_outlier_pad(n_out) / 64;
  const int wide = M <= 8 ? 8 : M <= 16 ? 16 : 32;
  return (size_t)(pairs * (M / kMaxTokens * pair_bytes(kMaxTokens, wide) + (M % kMaxTokens ? pair_bytes((int)(M % kMaxTokens), wide) : 0)));
}

nvfp4_status nvfp4_gemv(const void* X_bf16, int64_t ldx, int64_t M, int64_t D, const nvfp4_operand* W, const int32_t* keep_cols, const int32_t* outlier_cols,
                        int64_t n_out, const void* W_out, const void* bias_bf16, void* Y, int32_t y_dtype, int64_t ldy, int32_t* dev_status, void* workspace, size_t ws_bytes,
                        void* stream) {
  return nvfp4_gemv_ex(X_bf16, ldx, M, D, W, keep_cols, outlier_cols, n_out, W_out, bias_bf16, Y, y_dtype, ldy, dev_status, nullptr, workspace, ws_bytes, stream);
}

nvfp4_status nvfp4_gemv_ex(const void* X_bf16, int64_t ldx, int64_t M, int64_t D, const nvfp4_operand* W, const int32_t* keep_cols, const int32_t* outlier_cols,
                           int64_t n_out, const void* W_out, const void* bias_bf16, void* Y, int32_t y_dtype, int64_t ldy, int32_t* dev_status, const nvfp4_gemm_opts* opts,
                           void* workspace, size_t ws_bytes, void* stream) {
  if (!W) return NVFP4_ERR_NULL;
  if (opts && (opts->variant != NVFP4_GEMM_AUTO || opts->wait_limit_cycles < 0)) return NVFP4_ERR_ENUM;
  if (W->gs_mode < 0 || W->gs_mode > 2 || W->sf_layout != NVFP4_SF_TILED128x4 || y_dtype < 0 || y_dtype > 1) return NVFP4_ERR_ENUM;
  if (M < 0 || D <= 0 || n_out < 0 || W->R < 0 || W->K <= 0 || W->K + n_out != D) return NVFP4_ERR_SHAPE;
  if (D > ((int64_t)1 << 24) || W->R > ((int64_t)1 << 31) || M > 65535ll * kMaxTokens) return NVFP4_ERR_LIMIT;
  if (M == 0 || W->R == 0) return NVFP4_OK;
  if (!X_bf16 || !Y || !W->codes || !W->sf || !W->gscale || (n_out > 0 && (!keep_cols || !outlier_cols || !W_out))) return NVFP4_ERR_NULL;
  if (bad_matrix(X_bf16, ldx, D, 2) || bad_matrix(Y, ldy, W->R, y_dtype == NVFP4_DT_F32 ? 4 : 2) || !aligned(W->codes, 16) || !aligned(W->sf, 16) || !aligned(W->gscale, 4) ||
      !aligned(bias_bf16, 2) || (n_out > 0 && (!aligned(W_out, 16) || !aligned(keep_cols, 4) || !aligned(outlier_cols, 4))))
    return NVFP4_ERR_ALIGN;
  const int64_t n_code_pairs = (nvfp4_padded_k(W->K) / 128 + 1) / 2, n_pairs = n_code_pairs + nvfp4_outlier_pad(n_out) / 64;
  if (M * 2 * n_pairs > 16 * (int64_t)0x7FFFFFFF) return NVFP4_ERR_LIMIT;  // (the grid that stages X)
  if (M > 2 && (!workspace || !aligned(workspace, 16) || ws_bytes < nvfp4_gemv_workspace_bytes(M, D, n_out))) return NVFP4_ERR_WORKSPACE;
  if (!device_is_sm100()) return NVFP4_ERR_ARCH;
  GemvArgs a{};
  a.staged = static_cast<uint8_t*>(workspace);
  a.X = static_cast<const uint16_t*>(X_bf16);
  a.ldx = ldx;
  a.M = M;
  a.D = (int)D;
  a.K = (int)W->K;
  a.keep = n_out > 0 ? keep_cols : nullptr;
  a.outl = n_out > 0 ? outlier_cols : nullptr;
  a.n_out = (int)n_out;
  a.sf = W->sf;
  a.gscale = W->gscale;
  a.N = W->R;
  a.gs_mode = W->gs_mode;
  a.bias = static_cast<const uint16_t*>(bias_bf16);
  a.Y = Y;
  a.y_f32 = y_dtype == NVFP4_DT_F32;
  a.ldy = ldy;
  a.n_codes = (int)(nvfp4_padded_k(W->K) / 128);
  a.n_code_pairs = (int)n_code_pairs;
  a.n_pairs = (int)n_pairs;
  a.dev_status = dev_status;
  a.wait_limit = opts && opts->wait_limit_cycles > 0 ? opts->wait_limit_cycles : DEFAULT_WAIT_LIMIT_CYCLES;
  a.starve = opts && opts->starve_first_stage;
  CUtensorMap codes{}, outliers{};
  if (!encode_codes_map(&codes, W->codes, W->R, nvfp4_padded_k(W->K)) || (n_out > 0 && !encode_outliers_map(&outliers, W_out, W->R, nvfp4_outlier_pad(n_out)))) return NVFP4_ERR_CUDA;
  // CTAs along k: as many as leave every CTA a pair and are two to an SM together. (Of more than 16 tokens an SM holds one, so that they are up to
  // two waves there: 256 for 8192 x 8192.)
  const int64_t row_ctas = (W->R + kRows - 1) / kRows, most = (int64_t)device_sm_count() * 2;
  const int S = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(kMaxCluster, a.n_pairs), most / row_ctas));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  // Three and four tokens: as one and two (in two columns of instructions each) where one wave of CTAs has two pairs each at most and a launch more is
  // what counts: us from Python / on the device, times three, 1024 x 2816 5.4 / 5.0 against 6.8 / 5.1 with the launch, 1024 x 4096 5.6 / 5.1 against
  // 6.5 / 5.2; with four pairs 1024 x 8192 7.7 / 7.6 against 7.1 / 6.9, with fifteen 128 x 30000 18.4 / 18.3 against 13.0 / 12.6.
  const bool few = M <= 4 && row_ctas * a.n_pairs <= most && a.n_pairs <= 2 * S;
  const cudaError_t e = M <= 2    ? launch_gemv<1, true>(codes, outliers, a, row_ctas, S, st)
                        : few     ? launch_gemv<2, true>(codes, outliers, a, row_ctas, S, st)
                        : M <= 8  ? launch_gemv<1, false>(codes, outliers, a, row_ctas, S, st)
                        : M <= 16 ? launch_gemv<2, false>(codes, outliers, a, row_ctas, S, st)
                                  : launch_gemv<4, false>(codes, outliers, a, row_ctas, S, st);
  return e == cudaSuccess && cudaGetLastError() == cudaSuccess ? NVFP4_OK : NVFP4_ERR_CUDA;
}

}  // extern "C"
