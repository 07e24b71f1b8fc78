// Product of two e4m3 matrices with a scale for each block of 128 along the sum, sm_100a:
//   y[r, f] = sum over blocks b of  sx[r, b] sw[f / 128, b]  sum over k in block b of  xq[r, k] wq[f, k]
// the forward product of a fully connected layer (wq [features, K]), in fp32 until y is rounded.
//
// The scales are any fp32 numbers, so a block's sum has to be multiplied before it is added to the next one's: the tensor cores sum a block
// of 128 into one of several accumulators in tensor memory, while other warps take an earlier one's sums out, multiply them by the product of
// the two scales and add them to sums in registers. Where that product is no normal number - infinite, subnormal or zero, though the block's
// share of y need not be -, the sum is multiplied by one scale and then by the other. No ordinary scales are like that, so the rows that have such
// a block are computed again behind the tensor cores' work, by plain multiply-adds (recompute_rows; 1024 rows of 4096 features, K = 4096: one
// such row 167 us instead of 20, all of them 10 ms). (Two factors for each sum in the loop itself, behind a test of four blocks' products: 284 us
// for 16384 rows instead of 258.) Two kernels:
//
// Pairs of CTAs (fp8_pair_kernel), for many rows: a pair computes 256 rows of y and 128 features - those of one weight block, so that a row
// has one scale a block. tcgen05.mma with 256 rows reads both CTAs' halves of the features.
//   warp 0 TMA producer; warp 1 MMA issuer (first CTA); warps 2, 3 products of scales; warps 4-11 take, scale and store: a thread owns one
//   row and 64 features, two sums an instruction.
// What bounds it: 16384 x 4096 . 4096 x 4096 takes 254-262 us (2.1 PFLOP/s, 63 % of twice the measured burst bf16 rate; 300 us when the chip is
// power-limited, 66 % of twice the sustained one). With the scaling warps doing nothing but hand accumulators back, the same MMAs take 186
// us; what they add is their instructions on the schedulers that the issuing threads share (single multiply-adds instead of pairs: 273 us).
//
// Features as rows of the MMA (fp8_rows_kernel), for few rows of x (one generated token for each of a batch's sequences): 128 features meet T
// rows of x, so the weights stream through shared memory once and only T - rows columns are wasted on absent rows of x. The sum over K is
// split over a cluster of CTAs so that all multiprocessors pull weights; partial sums meet through distributed shared memory in a
// fixed order. One row, 4096 x 4096: 5.1 us; the weights' bytes alone are 2.6.
#include <float.h>

#include "dgrad_common.cuh"

namespace sdgp {
namespace {

constexpr int kBlockK = 128;            // bytes of a stage's row: one scale block, one 128-byte swizzle row
constexpr int kTileBytes = 128 * kBlockK;

struct Fp8Params {
  const uint8_t *xq, *wq;  // [rows, K], [features, K]
  int64_t K;
  const float* sx;  // [rows, blocks]
  const float* sw;  // [feature blocks, blocks]
  void* y;          // [rows, features]
  int64_t rows, features;
  int blocks;
  int tiles_n, tiles;  // pair kernel: feature tiles, all tiles; rows kernel: feature blocks
  int stages;
  int dtype;
};

// Instruction descriptor of kind::f8f6f4: fp32 sums, e4m3 A and B (format 0), both K-major.
__host__ __device__ constexpr uint32_t fp8_idesc(int m, int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24); }

__device__ __forceinline__ void mma_fp8_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void mma_fp8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// Waits for this thread's loads from tensor memory; names the registers so that nothing that reads them moves before it.
__device__ __forceinline__ void tmem_ld_wait_for(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]),
                 "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]),
                 "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]),
                 "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
               :
               : "memory");
}

// 16 columns, for the narrowest accumulators.
__device__ __forceinline__ void tmem_ld_32x16(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
#pragma unroll
  for (int i = 16; i < 32; ++i) r[i] = 0u;
}

__device__ __forceinline__ uint64_t float_pair(float a, float b) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ void float_pair(uint64_t p, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
// (x, y) times a pair of scales, added to a pair of sums.
__device__ __forceinline__ void fma_pair(uint64_t& sums, uint32_t x, uint32_t y, uint64_t scale) {
  asm("{\n\t.reg .b64 v;\n\tmov.b64 v, {%1, %2};\n\tfma.rn.f32x2 %0, v, %3, %0;\n\t}" : "+l"(sums) : "r"(x), "r"(y), "l"(scale));
}

// Whether all of some products of scales are normal numbers or NaN, from their least and largest magnitude.
template <int N>
__device__ __forceinline__ bool all_normal(const float (&x)[N]) {
  float least = fabsf(x[0]), most = least;
#pragma unroll
  for (int i = 1; i < N; ++i) {
    least = fminf(least, fabsf(x[i]));
    most = fmaxf(most, fabsf(x[i]));
  }
  return !(least < FLT_MIN) && !(most > FLT_MAX);
}
// What a block's sum v is multiplied by, as (v * first) * second: (1, the scales' product), which leaves v as it is, wherever that product
// is a normal number or NaN, or a scale is zero. Else the larger scale comes first. Sums of e4m3 products are 0 or from 2^-18 to 2^25: where the
// scales' product is too large both are above 1 and v * first is no larger than the result; where it is too small, v * first is a normal number
// if the result is not zero.
struct Factors {
  float first, second;
};
__device__ __forceinline__ Factors factors_of(float x, float w) {
  const float product = x * w;
  if (!(fabsf(product) < FLT_MIN || fabsf(product) > FLT_MAX) || x == 0.0f || w == 0.0f) return {1.0f, product};
  const bool x_first = fabsf(x) > fabsf(w);
  return {x_first ? x : w, x_first ? w : x};
}

// Sixteen products of e4m3 numbers, added up in order.
__device__ __forceinline__ float add_products(const uint4& a, const uint4& b, float sum) {
  const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, bw[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    uint32_t x, w;  // pairs of binary16, exact
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(x) : "h"((uint16_t)(aw[i / 2] >> 16 * (i & 1))));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(w) : "h"((uint16_t)(bw[i / 2] >> 16 * (i & 1))));
    sum = fmaf(lane_lo<true>(x), lane_lo<true>(w), sum);
    sum = fmaf(lane_hi<true>(x), lane_hi<true>(w), sum);
  }
  return sum;
}

// Of y's rows [row0, row0 + rows) and `count` features of a block of 128, the rows with a block whose scales want two factors, by `warps` warps
// of which this is number `warp`.
__device__ __forceinline__ void recompute_rows(const Fp8Params& p, int64_t row0, int rows, int64_t feature0, int count, int warp, int warps) {
  const int lane = threadIdx.x & 31;
  const float* sw = p.sw + feature0 / 128 * p.blocks;
  for (int r = warp; r < rows; r += warps) {
    const int64_t row = row0 + r;
    if (row >= p.rows) break;
    const float* sx = p.sx + row * p.blocks;
    bool two = false;
    for (int b = lane; b < p.blocks; b += 32) two |= factors_of(sx[b], sw[b]).first != 1.0f;
    if (!__any_sync(0xFFFFFFFFu, two)) continue;
    for (int i = lane; i < count; i += 32) {
      const int64_t feature = feature0 + i;
      if (feature >= p.features) break;
      const uint8_t *x = p.xq + row * p.K, *w = p.wq + feature * p.K;
      float sum = 0.0f;
      for (int b = 0; b < p.blocks; ++b) {
        float v = 0.0f;
        const int64_t end = min(p.K, (int64_t)(b + 1) * kBlockK);
        for (int64_t k = (int64_t)b * kBlockK; k < end; k += 16) v = add_products(*(const uint4*)(x + k), *(const uint4*)(w + k), v);
        const Factors f = factors_of(sx[b], sw[b]);
        sum = fmaf(v * f.first, f.second, sum);
      }
      const int64_t at = row * p.features + feature;
      if (p.dtype == SDGP_FP32) ((float*)p.y)[at] = sum;
      else ((uint16_t*)p.y)[at] = (uint16_t)(p.dtype == SDGP_FP16 ? f32_to_f16_bits(sum) : f32_to_bf16_bits(sum));
    }
  }
}

// The same as a call, where the code inlined made the kernel's loops slower (the kernel of 64 rows 63 instead of 58 us, pairs of CTAs 278 instead of 261).
__device__ __noinline__ void call_recompute_rows(const Fp8Params p, int64_t row0, int rows, int64_t feature0, int count, int warp, int warps) {
  recompute_rows(p, row0, rows, feature0, count, warp, warps);
}

__device__ __forceinline__ void st_cluster_u32(uint32_t addr, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// ------------------------------------------------------------------------------------------------ pairs of CTAs

constexpr int kPairThreads = 384;
constexpr int kPairMaxStages = 8;
constexpr int kPairFeatures = 128;                        // features of a tile: one weight block
constexpr int kHalf = kPairFeatures / 2;                  // rows of wq that a CTA stages; features of a scaling thread
constexpr int kPairStage = kTileBytes + kHalf * kBlockK;
constexpr int kPairBufs = 4;                              // accumulators
constexpr int kScaleGroup = 4;                            // blocks whose scales are multiplied at a time
constexpr int kScaleFloats = kScaleGroup * 128;
constexpr int kStagedBytes = 8 * 4096;  // 32 rows of 128 bytes of y for each multiplying warp
constexpr int kPairSlack = kSmemSlack + 2 * kScaleFloats * 4 + kStagedBytes;

__global__ void __launch_bounds__(kPairThreads, 1)
fp8_pair_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmY,
                const __grid_constant__ Fp8Params p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + (-ptx::smem_u32(smem_raw) & 1023u);
  uint8_t* staged = smem + p.stages * kPairStage;
  uint64_t* full = (uint64_t*)(staged + kStagedBytes);
  uint64_t* empty = full + kPairMaxStages;
  uint64_t* acc_full = empty + kPairMaxStages;
  uint64_t* acc_empty = acc_full + kPairBufs;
  uint64_t* scale_full = acc_empty + kPairBufs;
  uint64_t* scale_empty = scale_full + 2;
  uint32_t* tmem_slot = (uint32_t*)(scale_empty + 2);
  volatile uint32_t* again = tmem_slot + 1;               // some rows are to be computed again
  float* scales = (float*)(staged + kStagedBytes + 256);  // [2][kScaleGroup][128]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = ptx::cluster_ctarank();
  unsigned int* err = &g_device_error;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kPairMaxStages; ++s) {
      ptx::mbar_init(&full[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < kPairBufs; ++a) {
      ptx::mbar_init(&acc_full[a], 1);
      ptx::mbar_init(&acc_empty[a], 16);  // eight warps of each CTA
    }
    for (int g = 0; g < 2; ++g) {
      ptx::mbar_init(&scale_full[g], 2);
      ptx::mbar_init(&scale_empty[g], 8);
    }
    *again = 0u;
    ptx::fence_mbar_init();
    ptx::prefetch_tensormap(&tmX);
    ptx::prefetch_tensormap(&tmW);
  }
  if (warp == 1) {
    ptx::tmem_alloc_pair(tmem_slot, kTmemCols);
    ptx::tmem_relinquish_pair();
  }
  ptx::tc_fence_before_sync();
  ptx::cluster_sync();
  ptx::tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  ptx::wait_for_previous_grid();
  ptx::launch_dependents();

  const int pairs = gridDim.x >> 1, first = blockIdx.x >> 1;
  if (warp < 4) {
    fewer_registers<64>();
    if (warp == 0) {
      if (ptx::elect_one()) {
        int st = 0;
        uint32_t ph = 0;
        bool alive = true;
        for (int t = first; alive && t < p.tiles; t += pairs) {
          const int x_row = (t / p.tiles_n) * 256 + (int)rank * 128, w_row = (t % p.tiles_n) * kPairFeatures + (int)rank * kHalf;
          for (int b = 0; b < p.blocks; ++b) {
            if (!ptx::mbar_wait(&empty[st], ph ^ 1u, err, 0x100u + st)) { alive = false; break; }
            if (rank == 0) ptx::mbar_arrive_expect_tx(&full[st], 2u * kPairStage);
            ptx::tma_load_2d_pair(smem + st * kPairStage, &tmX, &full[st], b * kBlockK, x_row);
            ptx::tma_load_2d_pair(smem + st * kPairStage + kTileBytes, &tmW, &full[st], b * kBlockK, w_row);
            if (++st == p.stages) { st = 0; ph ^= 1u; }
          }
        }
      }
    } else if (warp == 1 && rank == 0) {
      if (ptx::elect_one()) {
        constexpr uint32_t idesc = fp8_idesc(256, kPairFeatures);
        const uint64_t desc0 = ptx::make_smem_desc(0, 16, 1024, 2);
        int st = 0, buf = 0;
        uint32_t ph = 0, aph = 0;
        bool alive = true;
        for (int t = first; alive && t < p.tiles; t += pairs) {
          for (int b = 0; b < p.blocks; ++b) {
            if (!ptx::mbar_wait(&acc_empty[buf], aph ^ 1u, err, 0x200u + buf) || !ptx::mbar_wait(&full[st], ph, err, 0x300u + st)) {
              alive = false;
              break;
            }
            ptx::tc_fence_after_sync();
            const uint64_t a = desc0 + (ptx::smem_u32(smem + st * kPairStage) >> 4);
            const uint64_t w = a + (kTileBytes >> 4);
#pragma unroll
            for (int k = 0; k < 4; ++k)  // 32 elements an instruction
              mma_fp8_pair(tmem_base + (uint32_t)(buf * kPairFeatures), a + 2 * k, w + 2 * k, idesc, k != 0);
            ptx::tc_commit_pair(&empty[st], 3);
            ptx::tc_commit_pair(&acc_full[buf], 3);
            if (++st == p.stages) { st = 0; ph ^= 1u; }
            if (++buf == kPairBufs) { buf = 0; aph ^= 1u; }
          }
        }
      }
    } else if (warp >= 2) {
      // The scales' products, four blocks at a time, into shared memory. Loaded by the scaling warps themselves - 32 lines a warp and block, from
      // L2 since the stages leave next to no L1 - they slowed the products down by a tenth.
      const int i = threadIdx.x - 64;  // rows i and i + 64
      int g = 0;
      uint32_t gph = 0;
      bool alive = true;
      for (int t = first; alive && t < p.tiles; t += pairs) {
        const int64_t row = (int64_t)(t / p.tiles_n) * 256 + (int)rank * 128 + i;
        const float* sx0 = p.sx + (row < p.rows ? row : 0) * p.blocks;
        const float* sx1 = p.sx + (row + 64 < p.rows ? row + 64 : 0) * p.blocks;
        const float* sw = p.sw + (int64_t)(t % p.tiles_n) * p.blocks;
        for (int b = 0; b < p.blocks; b += kScaleGroup) {
          float x0[kScaleGroup], x1[kScaleGroup], w[kScaleGroup];
#pragma unroll
          for (int k = 0; k < kScaleGroup; ++k) {
            const int at = min(b + k, p.blocks - 1);
            x0[k] = sx0[at];
            x1[k] = sx1[at];
            w[k] = sw[at];
          }
          if (!ptx::mbar_wait<kIdleWaitNs>(&scale_empty[g], gph ^ 1u, err, 0x900u + g)) { alive = false; break; }
          float* to = scales + g * kScaleFloats + i;
          float product[2 * kScaleGroup];
#pragma unroll
          for (int k = 0; k < kScaleGroup; ++k) {
            to[k * 128] = product[2 * k] = x0[k] * w[k];
            to[k * 128 + 64] = product[2 * k + 1] = x1[k] * w[k];
          }
          if (!all_normal(product)) {  // (zero, it may be, because a scale is)
            bool two = false;
#pragma unroll
            for (int k = 0; k < kScaleGroup; ++k) two |= factors_of(x0[k], w[k]).first != 1.0f || factors_of(x1[k], w[k]).first != 1.0f;
            if (two) *again = 1u;
          }
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&scale_full[g]);
          if (++g == 2) { g = 0; gph ^= 1u; }
        }
      }
    }
  } else {
    more_registers<216>();
    const int half = (warp - 4) >> 2;   // which features of the tile
    const uint32_t lanes = tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(half * kHalf);
    const float* my_scales = scales + (warp & 3) * 32 + lane;
    int buf = 0, group = 0;
    uint32_t aph = 0, gph = 0;
    bool alive = true;
    for (int t = first; alive && t < p.tiles; t += pairs) {
      const int64_t row = (int64_t)(t / p.tiles_n) * 256 + (int)rank * 128 + (warp & 3) * 32 + lane;
      const int64_t feature = (int64_t)(t % p.tiles_n) * kPairFeatures + half * kHalf;
      uint64_t sums[kHalf / 2];  // pairs of features
#pragma unroll
      for (int c = 0; c < kHalf / 2; ++c) sums[c] = 0u;
      for (int b = 0; b < p.blocks; ++b) {
        const int k = b % kScaleGroup;
        if (k == 0 && !ptx::mbar_wait(&scale_full[group], gph, err, 0xA00u + group)) { alive = false; break; }
        const float scale = my_scales[group * kScaleFloats + k * 128];
        const uint64_t scale2 = float_pair(scale, scale);
        if (!ptx::mbar_wait(&acc_full[buf], aph, err, 0x400u + buf)) { alive = false; break; }
        ptx::tc_fence_after_sync();
        const uint32_t from = lanes + (uint32_t)(buf * kPairFeatures);
        uint32_t v[kHalf / 32][32];
#pragma unroll
        for (int c = 0; c < kHalf / 32; ++c) ptx::tmem_ld_32x32(from + 32u * c, v[c]);
#pragma unroll
        for (int c = 0; c < kHalf / 32; ++c) tmem_ld_wait_for(v[c]);
        ptx::tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive_cluster(&acc_empty[buf], 0);
#pragma unroll
        for (int c = 0; c < kHalf / 32; ++c)
#pragma unroll
          for (int e = 0; e < 16; ++e) fma_pair(sums[16 * c + e], v[c][2 * e], v[c][2 * e + 1], scale2);
        if (k == kScaleGroup - 1 || b + 1 == p.blocks) {
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&scale_empty[group]);
          if (++group == 2) { group = 0; gph ^= 1u; }
        }
        if (++buf == kPairBufs) { buf = 0; aph ^= 1u; }
      }
      if (!alive) break;
      // y through shared memory, in slabs of 32 rows x 128 bytes that a TMA store each takes away (clipped at the edges)
      float acc[kHalf];
#pragma unroll
      for (int c = 0; c < kHalf / 2; ++c) float_pair(sums[c], acc[2 * c], acc[2 * c + 1]);
      uint8_t* slab = staged + (warp - 4) * 4096;
      constexpr int kMost = kHalf / 32;  // slabs of fp32
#pragma unroll
      for (int c = 0; c < kMost; ++c) {
        const bool wide = p.dtype == SDGP_FP32;
        if (!wide && (c & 1)) continue;
        if (lane == 0) ptx::bulk_wait_group_read<0>();  // the store before has read the slab
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          uint4 w;
          if (wide) {
            const int e = 32 * c + 4 * k;
            w = make_uint4(__float_as_uint(acc[e]), __float_as_uint(acc[e + 1]), __float_as_uint(acc[e + 2]), __float_as_uint(acc[e + 3]));
          } else {
            const int e = (32 * c + 8 * k) % kHalf;
            if (p.dtype == SDGP_FP16)
              w = make_uint4(pack_pair_rn<true>(acc[e], acc[e + 1]), pack_pair_rn<true>(acc[e + 2], acc[e + 3]),
                             pack_pair_rn<true>(acc[e + 4], acc[e + 5]), pack_pair_rn<true>(acc[e + 6], acc[e + 7]));
            else
              w = make_uint4(pack_pair_rn<false>(acc[e], acc[e + 1]), pack_pair_rn<false>(acc[e + 2], acc[e + 3]),
                             pack_pair_rn<false>(acc[e + 4], acc[e + 5]), pack_pair_rn<false>(acc[e + 6], acc[e + 7]));
          }
          *(uint4*)(slab + lane * 128 + ((k ^ (lane & 7)) << 4)) = w;  // 128-byte swizzle
        }
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          if (row < p.rows && feature + 32 * c < p.features) ptx::tma_store_2d(&tmY, slab, (int)feature + 32 * c, (int)row);
          ptx::bulk_commit_group();
        }
      }
    }
    if (lane == 0) ptx::bulk_wait_group_read<0>();
    if (*again && alive) {  // (written before the products that the last tile's sums were multiplied by)
      if (lane == 0) ptx::bulk_wait_group<0>();  // what this warp has stored is in memory
      __syncwarp();
      for (int t = first; t < p.tiles; t += pairs)
        call_recompute_rows(p, (int64_t)(t / p.tiles_n) * 256 + (int)rank * 128 + (warp & 3) * 32, 32,
                            (int64_t)(t % p.tiles_n) * kPairFeatures + half * kHalf, kHalf, 0, 1);
    }
  }
  ptx::tc_fence_before_sync();
  ptx::cluster_sync();
  ptx::tc_fence_after_sync();
  if (warp == 1) ptx::tmem_dealloc_pair(tmem_base, kTmemCols);
}

// ------------------------------------------------------------------------------------------------ features as rows

constexpr int kRowsThreads = 192;
constexpr int kRowsMaxStages = 12;
constexpr int kMostSplit = 8;                            // CTAs that share a sum
constexpr int kRowsGroup = 8;                             // blocks whose scales are fetched at a time
constexpr int kRowsSlack = 1024 + 512 + 2 * kRowsGroup * 64 * 4;  // alignment, barriers, products of scales

template <int T>
__global__ void __launch_bounds__(kRowsThreads)
fp8_rows_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmW, const Fp8Params p) {
  constexpr int kStageBytes = kTileBytes + T * kBlockK;
  constexpr int kBufs = 8;                         // accumulators: so many blocks' products may wait to be scaled
  constexpr uint32_t kCols = kBufs * T;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + (-ptx::smem_u32(smem_raw) & 1023u);  // (an offset: a pointer put together from integers is no longer known to be shared)
  uint64_t* full = (uint64_t*)(smem + p.stages * kStageBytes);
  uint64_t* empty = full + kRowsMaxStages;
  uint64_t* acc_full = empty + kRowsMaxStages;
  uint64_t* acc_empty = acc_full + kBufs;
  uint32_t* tmem_slot = (uint32_t*)(acc_empty + kBufs);
  volatile uint32_t* again = tmem_slot + 1;        // some rows are to be computed again
  float* scales = (float*)((uint8_t*)full + 512);  // [2][kRowsGroup][T]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int split = (int)ptx::cluster_nctarank(), rank = (int)ptx::cluster_ctarank();
  unsigned int* err = &g_device_error;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kRowsMaxStages; ++s) {
      ptx::mbar_init(&full[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < kBufs; ++a) {
      ptx::mbar_init(&acc_full[a], 1);
      ptx::mbar_init(&acc_empty[a], 4);
    }
    *again = 0u;
    ptx::fence_mbar_init();
    ptx::prefetch_tensormap(&tmX);
    ptx::prefetch_tensormap(&tmW);
  }
  if (warp == 1) {
    ptx::tmem_alloc(tmem_slot, kCols);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  ptx::wait_for_previous_grid();
  ptx::launch_dependents();

  const int tile = (int)(blockIdx.x / (unsigned)split);
  const int feature_block = tile % p.tiles_n;
  const int64_t row0 = (int64_t)(tile / p.tiles_n) * T;
  const int b0 = (int)((int64_t)p.blocks * rank / split), b1 = (int)((int64_t)p.blocks * (rank + 1) / split);
  uint64_t sums[T / 2];  // (of the multiplying warps) pairs of rows of x
  const int f = (warp & 3) * 32 + lane;  // their feature of the block
  bool alive = true, normal = true;  // normal: no block wants two factors

  if (warp == 0) {
    if (ptx::elect_one()) {
      int st = 0;
      uint32_t ph = 0;
      for (int b = b0; b < b1; ++b) {
        if (!ptx::mbar_wait(&empty[st], ph ^ 1u, err, 0x500u + st)) break;
        ptx::mbar_arrive_expect_tx(&full[st], kStageBytes);
        ptx::tma_load_2d(smem + st * kStageBytes, &tmW, &full[st], b * kBlockK, feature_block * 128);
        ptx::tma_load_2d(smem + st * kStageBytes + kTileBytes, &tmX, &full[st], b * kBlockK, (int)row0);
        if (++st == p.stages) { st = 0; ph ^= 1u; }
      }
    }
  } else if (warp == 1) {
    if (ptx::elect_one()) {
      constexpr uint32_t idesc = fp8_idesc(128, T);
      const uint64_t desc0 = ptx::make_smem_desc(0, 16, 1024, 2);
      int st = 0, buf = 0;
      uint32_t ph = 0, aph = 0;
      for (int b = b0; b < b1; ++b) {
        if (!ptx::mbar_wait(&acc_empty[buf], aph ^ 1u, err, 0x600u + buf) || !ptx::mbar_wait(&full[st], ph, err, 0x700u + st)) break;
        ptx::tc_fence_after_sync();
        const uint64_t w = desc0 + (ptx::smem_u32(smem + st * kStageBytes) >> 4);
        const uint64_t x = w + (kTileBytes >> 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) mma_fp8(tmem_base + (uint32_t)(buf * T), w + 2 * k, x + 2 * k, idesc, k != 0);
        ptx::tc_commit(&empty[st]);
        ptx::tc_commit(&acc_full[buf]);
        if (++st == p.stages) { st = 0; ph ^= 1u; }
        if (++buf == kBufs) { buf = 0; aph ^= 1u; }
      }
    }
  } else {
    const uint32_t lanes = tmem_base + ((uint32_t)((warp & 3) * 32) << 16);
    // the products of the two scales, eight blocks at a time, loaded while the eight before are in use: value j of a thread is row
    // (tid + 128 j) % T of block (tid + 128 j) / T
    constexpr int kEach = T * kRowsGroup / 128;
    const int tid = threadIdx.x - 64;
    const float* sw = p.sw + (int64_t)feature_block * p.blocks;
    float ahead_x[kEach], ahead_w[kEach];  // (1 where there is no row or block)
    auto load = [&](int first) {
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        const int64_t row = row0 + (tid + 128 * j) % T;
        const int b = first + (tid + 128 * j) / T;
        const bool there = row < p.rows && b < b1;
        ahead_x[j] = there ? p.sx[row * p.blocks + b] : 1.0f;
        ahead_w[j] = there ? sw[b] : 1.0f;
      }
    };
#pragma unroll
    for (int c = 0; c < T / 2; ++c) sums[c] = 0u;
    load(b0);
    int buf = 0;
    uint32_t aph = 0;
    for (int b = b0; b < b1; ++b) {
      const int k = (b - b0) % kRowsGroup, which = ((b - b0) / kRowsGroup) & 1;
      if (k == 0) {
        float* to = scales + which * kRowsGroup * T + tid;
        float product[kEach];
#pragma unroll
        for (int j = 0; j < kEach; ++j) to[128 * j] = product[j] = ahead_x[j] * ahead_w[j];
        if (!all_normal(product)) {  // (zero, it may be, because a scale is)
#pragma unroll
          for (int j = 0; j < kEach; ++j) normal &= factors_of(ahead_x[j], ahead_w[j]).first == 1.0f;
        }
        load(b + kRowsGroup);
        ptx::named_bar_sync(1, 128);  // (who writes the other group's has passed this barrier, so all have read it)
      }
      alive = ptx::mbar_wait(&acc_full[buf], aph, err, 0x800u + buf) && alive;  // (all four warps stay in step for that)
      ptx::tc_fence_after_sync();
      const float* s = scales + (which * kRowsGroup + k) * T;
#pragma unroll
      for (int c = 0; c < T; c += 32) {
        uint32_t v[32];
        if constexpr (T == 16) tmem_ld_32x16(lanes + (uint32_t)(buf * T), v);
        else ptx::tmem_ld_32x32(lanes + (uint32_t)(buf * T + c), v);
        tmem_ld_wait_for(v);
        if (c + 32 >= T) {
          ptx::tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&acc_empty[buf]);
        }
#pragma unroll
        for (int e = 0; e < (T < 32 ? T : 32); e += 4) {
          const float4 k = *(const float4*)(s + c + e);
          fma_pair(sums[(c + e) / 2], v[e], v[e + 1], float_pair(k.x, k.y));
          fma_pair(sums[(c + e) / 2 + 1], v[e + 2], v[e + 3], float_pair(k.z, k.w));
        }
      }
      if (++buf == kBufs) { buf = 0; aph ^= 1u; }
    }
  }

  const int64_t feature = (int64_t)feature_block * 128 + f;
  const int rows = (int)min((int64_t)T, p.rows - row0);
  float acc[T];
#pragma unroll
  for (int c = 0; c < T / 2; ++c) float_pair(sums[c], acc[2 * c], acc[2 * c + 1]);
  auto store = [&](int c, float x) {
    const int64_t at = (row0 + c) * p.features + feature;
    if (p.dtype == SDGP_FP32) ((float*)p.y)[at] = x;
    else ((uint16_t*)p.y)[at] = (uint16_t)(p.dtype == SDGP_FP16 ? f32_to_f16_bits(x) : f32_to_bf16_bits(x));
  };
  if (split == 1) {
    if (warp >= 2 && alive && feature < p.features) {
#pragma unroll
      for (int c = 0; c < T; ++c)
        if (c < rows) store(c, acc[c]);
    }
    if (!normal) *again = 1u;
  } else {
    // partial sums [T][128] over the stages, which every multiplication has read to the end; each CTA adds and stores its share of the rows of
    // x, in the order of the CTAs
    float* partial = (float*)smem;
    if (warp >= 2) {
#pragma unroll
      for (int c = 0; c < T; ++c) partial[c * 128 + f] = acc[c];
    }
    ptx::cluster_sync();
    if (warp >= 2 && alive && feature < p.features) {
      for (int c = T * rank / split; c < min(rows, T * (rank + 1) / split); ++c) {
        float v[kMostSplit];
#pragma unroll
        for (int r = 0; r < kMostSplit; ++r) v[r] = r < split ? ptx::ld_cluster_f32(ptx::map_to_cta(&partial[c * 128 + f], (uint32_t)r)) : 0.0f;
        float sum = v[0];
#pragma unroll
        for (int r = 1; r < kMostSplit; ++r) sum += v[r];
        store(c, sum);
      }
    }
    if (!normal) st_cluster_u32(ptx::map_to_cta((const void*)again, 0), 1u);
    ptx::cluster_sync();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  if (rank == 0 && *again && alive) {
    if constexpr (T == 64) call_recompute_rows(p, row0, rows, (int64_t)feature_block * 128, 128, warp, kRowsThreads / 32);
    else recompute_rows(p, row0, rows, (int64_t)feature_block * 128, 128, warp, kRowsThreads / 32);
  }
  if (warp == 1) ptx::tmem_dealloc(tmem_base, kCols);
}

// ------------------------------------------------------------------------------------------------ host

bool encode_rows(CUtensorMap* map, const void* base, int64_t rows, int64_t K, int box_rows) {
  const uint64_t dims[2] = {(uint64_t)K, (uint64_t)rows}, strides[1] = {(uint64_t)K};
  const uint32_t box[2] = {kBlockK, (uint32_t)box_rows};
  return encode_fresh(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

sdgp_status launch_pair(const void* xq, const void* wq, Fp8Params p, int64_t K, cudaStream_t stream) {
  static bool done[kMaxDevices] = {};
  if (!configure_once(fp8_pair_kernel, done)) return SDGP_ERR_CUDA;
  CUtensorMap tx, tw, ty;
  if (!encode_rows(&tx, xq, p.rows, K, 128) || !encode_rows(&tw, wq, p.features, K, kHalf)) return SDGP_ERR_CUDA;
  // y [rows, features] in boxes of 32 rows x 128 bytes
  const uint64_t size = p.dtype == SDGP_FP32 ? 4 : 2, dims[2] = {(uint64_t)p.features, (uint64_t)p.rows}, strides[1] = {(uint64_t)p.features * size};
  const uint32_t box[2] = {(uint32_t)(128 / size), 32};
  if (!encode_fresh(&ty, p.dtype == SDGP_FP32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, p.y, dims, strides, box,
                    CU_TENSOR_MAP_SWIZZLE_128B))
    return SDGP_ERR_CUDA;
  p.stages = (kSmemLimit - kPairSlack) / kPairStage;
  if (p.stages > kPairMaxStages) p.stages = kPairMaxStages;
  p.tiles_n = (int)((p.features + kPairFeatures - 1) / kPairFeatures);
  const int64_t tiles = (p.rows + 255) / 256 * p.tiles_n;
  if (tiles > 0x7FFFFFFF) return SDGP_ERR_UNSUPPORTED;
  p.tiles = (int)tiles;
  return launch_pairs(fp8_pair_kernel, pairs_for(p.tiles), kPairThreads, p.stages * kPairStage + kPairSlack, stream, tx, tw, ty, p);
}

template <int T>
sdgp_status launch_rows(const void* xq, const void* wq, Fp8Params p, int64_t K, cudaStream_t stream) {
  static bool done[kMaxDevices] = {};
  if (!configure_once(fp8_rows_kernel<T>, done)) return SDGP_ERR_CUDA;
  CUtensorMap tx, tw;
  if (!encode_rows(&tx, xq, p.rows, K, T) || !encode_rows(&tw, wq, p.features, K, 128)) return SDGP_ERR_CUDA;
  constexpr int stage = kTileBytes + T * kBlockK;
  p.tiles_n = (int)((p.features + 127) / 128);
  const int64_t tiles = (p.rows + T - 1) / T * p.tiles_n;
  // CTAs that share a tile's sum: as long as they are all resident at once and each has two blocks at least
  int split = 1;
  while (split < kMostSplit && 2 * split * tiles <= sm_count() && 4 * split <= p.blocks) split *= 2;
  if (tiles * split > 0x7FFFFFFF) return SDGP_ERR_UNSUPPORTED;
  p.stages = (kSmemLimit - kRowsSlack) / stage;
  if (p.stages > kRowsMaxStages) p.stages = kRowsMaxStages;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * split));
  cfg.blockDim = dim3(kRowsThreads);
  cfg.dynamicSmemBytes = (size_t)(p.stages * stage + kRowsSlack);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)split;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, fp8_rows_kernel<T>, tx, tw, p) == cudaSuccess ? SDGP_OK : SDGP_ERR_CUDA;
}

}  // namespace

cudaError_t take_error_fp8(unsigned int* word) { return take_error_word(word); }

sdgp_status launch_fp8_linear(const void* xq, const float* x_scale, const void* wq, const float* w_scale, void* y, int64_t rows,
                              int64_t features, int64_t K, int dtype, cudaStream_t stream) {
  Fp8Params p = {};
  p.xq = (const uint8_t*)xq;
  p.wq = (const uint8_t*)wq;
  p.K = K;
  p.sx = x_scale;
  p.sw = w_scale;
  p.y = y;
  p.rows = rows;
  p.features = features;
  p.blocks = (int)((K + kBlockK - 1) / kBlockK);
  p.dtype = dtype;
  // Few rows: the weights' bytes count, and the sum over K can be split. From 33 rows the pair kernel was level or ahead (4096 features, K =
  // 4096: 33 rows 10.9 us on either, 64: 11.1 and 11.3, 256: 11.7 and 16.1, 1024: 20.5 and 58.9); its TMA stores want rows of y of
  // whole 16 bytes.
  if (rows <= 16) return launch_rows<16>(xq, wq, p, K, stream);
  if (rows <= 32) return launch_rows<32>(xq, wq, p, K, stream);
  if (features * (dtype == SDGP_FP32 ? 4 : 2) % 16 != 0) return launch_rows<64>(xq, wq, p, K, stream);
  return launch_pair(xq, wq, p, K, stream);
}

}  // namespace sdgp
