// Product of two e4m3 matrices with a scale for each block of 128 along the sum, sm_100a:
//   y[r, f] = sum over blocks b of  sx[r, b] sw[f / 128, b]  sum over k in block b of  xq[r, k] wq[f, k]
// the forward product of a fully connected layer (wq [features, K]), in fp32 until y is rounded.
//
// The scales are any fp32 numbers, so a block's sum has to be multiplied before it is added to the next one's: the tensor cores sum one block
// of 128 into one of two accumulators in tensor memory while other warps take the other one's sums out, multiply them by the two
// scales and add them to sums in registers. Two kernels:
//
// Pairs of CTAs (fp8_pair_kernel), for many rows: a pair computes 256 rows of y and BN features; tcgen05.mma with 256 rows reads both CTAs' halves.
// A thread of the eight multiplying warps owns one row and BN / 2 features of one weight block: both scales are numbers of that thread,
// one fused multiply-add a sum.
//   warp 0 TMA producer; warp 1 MMA issuer (first CTA); warps 4-11 take, scale and store.
// What bounds it: the MMAs of a block take 512 clocks a pair (BN = 256), taking and scaling its sums about as long.
//
// Features as rows of the MMA (fp8_rows_kernel), for few rows of x (one generated token for each of a batch's sequences): 128 features meet T
// rows of x, so the weights stream through shared memory once and nothing is wasted on absent rows of x but T - rows columns. The sum is
// split over a cluster of CTAs so that all multiprocessors pull weights; partial sums meet through distributed shared memory in a
// fixed order. Bound by the weights' bytes.
#include "dgrad_common.cuh"

namespace sdgp {
namespace {

constexpr int kBlockK = 128;            // bytes of a stage's row: one scale block, one 128-byte swizzle row
constexpr int kTileBytes = 128 * kBlockK;

struct Fp8Params {
  const float* sx;  // [rows, blocks]
  const float* sw;  // [feature blocks, blocks]
  void* y;          // [rows, features]
  int64_t rows, features;
  int blocks;
  int tiles_n, tiles;  // pair kernel: feature tiles, all tiles; rows kernel: feature blocks
  int stages;
  int dtype;
  int aligned32;    // every row of y starts on a 32-byte boundary
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

template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// COLS consecutive features of one row of y, `left` of them inside it.
template <int COLS>
__device__ __forceinline__ void store_features(void* y, int64_t at, int64_t left, const float (&acc)[COLS], int dtype, bool aligned32) {
  if (dtype == SDGP_FP32) {
    float* out = (float*)y + at;
    if (aligned32 && left >= COLS) {
#pragma unroll
      for (int c = 0; c < COLS; c += 8) ptx::st_global_256(out + c, (const uint32_t*)&acc[c]);
    } else {
#pragma unroll
      for (int c = 0; c < COLS; ++c)
        if (c < left) out[c] = acc[c];
    }
    return;
  }
  uint16_t* out = (uint16_t*)y + at;
#pragma unroll
  for (int c = 0; c < COLS; c += 16) {
    uint32_t packed[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      packed[e] = dtype == SDGP_FP16 ? pack_pair_rn<true>(acc[c + 2 * e], acc[c + 2 * e + 1]) : pack_pair_rn<false>(acc[c + 2 * e], acc[c + 2 * e + 1]);
    if (aligned32 && c + 16 <= left) {
      ptx::st_global_256(out + c, packed);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (c + 2 * e < left) out[c + 2 * e] = (uint16_t)packed[e];
        if (c + 2 * e + 1 < left) out[c + 2 * e + 1] = (uint16_t)(packed[e] >> 16);
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ pairs of CTAs

constexpr int kPairThreads = 384;
constexpr int kPairMaxStages = 8;

template <int BN>
__global__ void __launch_bounds__(kPairThreads, 1)
fp8_pair_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmW, const Fp8Params p) {
  constexpr int kBufs = 512 / BN;                // accumulators in tensor memory
  constexpr int kHalf = BN / 2;                  // rows of wq that a CTA stages; features of a multiplying thread
  constexpr int kStageBytes = kTileBytes + kHalf * kBlockK;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint64_t* full = (uint64_t*)(smem + p.stages * kStageBytes);
  uint64_t* empty = full + kPairMaxStages;
  uint64_t* acc_full = empty + kPairMaxStages;
  uint64_t* acc_empty = acc_full + kBufs;
  uint32_t* tmem_slot = (uint32_t*)(acc_empty + kBufs);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = ptx::cluster_ctarank();
  unsigned int* err = &g_device_error;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kPairMaxStages; ++s) {
      ptx::mbar_init(&full[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < kBufs; ++a) {
      ptx::mbar_init(&acc_full[a], 1);
      ptx::mbar_init(&acc_empty[a], 16);  // eight warps of each CTA
    }
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
          const int x_row = (t / p.tiles_n) * 256 + (int)rank * 128, w_row = (t % p.tiles_n) * BN + (int)rank * kHalf;
          for (int b = 0; b < p.blocks; ++b) {
            if (!ptx::mbar_wait(&empty[st], ph ^ 1u, err, 0x100u + st)) { alive = false; break; }
            if (rank == 0) ptx::mbar_arrive_expect_tx(&full[st], 2u * kStageBytes);
            ptx::tma_load_2d_pair(smem + st * kStageBytes, &tmX, &full[st], b * kBlockK, x_row);
            ptx::tma_load_2d_pair(smem + st * kStageBytes + kTileBytes, &tmW, &full[st], b * kBlockK, w_row);
            if (++st == p.stages) { st = 0; ph ^= 1u; }
          }
        }
      }
    } else if (warp == 1 && rank == 0) {
      if (ptx::elect_one()) {
        constexpr uint32_t idesc = fp8_idesc(256, BN);
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
            const uint64_t a = desc0 + (ptx::smem_u32(smem + st * kStageBytes) >> 4);
            const uint64_t w = a + (kTileBytes >> 4);
#pragma unroll
            for (int k = 0; k < 4; ++k)  // 32 elements an instruction
              mma_fp8_pair(tmem_base + (uint32_t)(buf * BN), a + 2 * k, w + 2 * k, idesc, k != 0);
            ptx::tc_commit_pair(&empty[st], 3);
            ptx::tc_commit_pair(&acc_full[buf], 3);
            if (++st == p.stages) { st = 0; ph ^= 1u; }
            if (++buf == kBufs) { buf = 0; aph ^= 1u; }
          }
        }
      }
    }
  } else {
    more_registers<216>();
    const int half = (warp - 4) >> 2;   // which features of the tile
    const uint32_t lanes = tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(half * kHalf);
    int buf = 0;
    uint32_t aph = 0;
    bool alive = true;
    for (int t = first; alive && t < p.tiles; t += pairs) {
      const int64_t row = (int64_t)(t / p.tiles_n) * 256 + (int)rank * 128 + (warp & 3) * 32 + lane;
      const int64_t feature = (int64_t)(t % p.tiles_n) * BN + half * kHalf;
      const float* sx = p.sx + (row < p.rows ? row : 0) * p.blocks;
      const float* sw = p.sw + (feature < p.features ? feature / 128 : 0) * p.blocks;
      float acc[kHalf];
#pragma unroll
      for (int c = 0; c < kHalf; ++c) acc[c] = 0.0f;
      float next = sx[0] * sw[0];
      for (int b = 0; b < p.blocks; ++b) {
        const float scale = next;
        if (b + 1 < p.blocks) next = sx[b + 1] * sw[b + 1];
        if (!ptx::mbar_wait(&acc_full[buf], aph, err, 0x400u + buf)) { alive = false; break; }
        ptx::tc_fence_after_sync();
        const uint32_t from = lanes + (uint32_t)(buf * BN);
        uint32_t v[2][32];
        ptx::tmem_ld_32x32(from, v[0]);
#pragma unroll
        for (int c = 0; c < kHalf / 32; ++c) {
          tmem_ld_wait_for(v[c & 1]);
          if (c + 1 < kHalf / 32) {
            ptx::tmem_ld_32x32(from + 32u * (c + 1), v[(c + 1) & 1]);
          } else {  // all of it is in registers
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive_cluster(&acc_empty[buf], 0);
          }
#pragma unroll
          for (int e = 0; e < 32; ++e) acc[32 * c + e] = fmaf(__uint_as_float(v[c & 1][e]), scale, acc[32 * c + e]);
        }
        if (++buf == kBufs) { buf = 0; aph ^= 1u; }
      }
      if (alive && row < p.rows && feature < p.features)
        store_features<kHalf>(p.y, row * p.features + feature, p.features - feature, acc, p.dtype, p.aligned32 != 0);
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
constexpr int kRowsSlack = 1024 + 256 + 2 * 128 * 4;  // alignment, barriers, the scales of two blocks

template <int T>
__global__ void __launch_bounds__(kRowsThreads)
fp8_rows_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmW, const Fp8Params p) {
  constexpr int kStageBytes = kTileBytes + T * kBlockK;
  constexpr uint32_t kCols = T < 16 ? 32 : 2 * T;  // two accumulators
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint64_t* full = (uint64_t*)(smem + p.stages * kStageBytes);
  uint64_t* empty = full + kRowsMaxStages;
  uint64_t* acc_full = empty + kRowsMaxStages;
  uint64_t* acc_empty = acc_full + 2;
  uint32_t* tmem_slot = (uint32_t*)(acc_empty + 2);
  float* scales = (float*)(acc_empty + 4);  // [2][T]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int split = (int)ptx::cluster_nctarank(), rank = (int)ptx::cluster_ctarank();
  unsigned int* err = &g_device_error;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kRowsMaxStages; ++s) {
      ptx::mbar_init(&full[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      ptx::mbar_init(&acc_full[a], 1);
      ptx::mbar_init(&acc_empty[a], 4);
    }
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
  float acc[T];  // (of the multiplying warps)
  const int f = (warp & 3) * 32 + lane;  // their feature of the block
  bool alive = true;

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
        if (++buf == 2) { buf = 0; aph ^= 1u; }
      }
    }
  } else {
    const uint32_t lanes = tmem_base + ((uint32_t)((warp & 3) * 32) << 16);
    const int i = threadIdx.x - 64;  // the row of x whose scale this thread fetches
    const bool mine = i < T && row0 + i < p.rows;
    const float* sx = p.sx + (mine ? row0 + i : 0) * p.blocks;
    const float* sw = p.sw + (int64_t)feature_block * p.blocks;
#pragma unroll
    for (int c = 0; c < T; ++c) acc[c] = 0.0f;
    float next = mine ? sx[b0] * sw[b0] : 0.0f;
    int buf = 0;
    uint32_t aph = 0;
    for (int b = b0; b < b1; ++b) {
      if (i < T) scales[buf * T + i] = next;
      if (mine && b + 1 < b1) next = sx[b + 1] * sw[b + 1];
      alive = ptx::mbar_wait(&acc_full[buf], aph, err, 0x800u + buf) && alive;  // (all four warps stay in step: the barrier below)
      ptx::named_bar_sync(1, 128);
      ptx::tc_fence_after_sync();
      const float* s = scales + buf * T;
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
          acc[c + e] = fmaf(__uint_as_float(v[e]), k.x, acc[c + e]);
          acc[c + e + 1] = fmaf(__uint_as_float(v[e + 1]), k.y, acc[c + e + 1]);
          acc[c + e + 2] = fmaf(__uint_as_float(v[e + 2]), k.z, acc[c + e + 2]);
          acc[c + e + 3] = fmaf(__uint_as_float(v[e + 3]), k.w, acc[c + e + 3]);
        }
      }
      buf ^= 1;
      if (buf == 0) aph ^= 1u;
    }
  }

  const int64_t feature = (int64_t)feature_block * 128 + f;
  auto store = [&](int64_t row, float x) {
    if (row >= p.rows || feature >= p.features) return;
    const int64_t at = row * p.features + feature;
    if (p.dtype == SDGP_FP32) ((float*)p.y)[at] = x;
    else ((uint16_t*)p.y)[at] = (uint16_t)(p.dtype == SDGP_FP16 ? f32_to_f16_bits(x) : f32_to_bf16_bits(x));
  };
  if (split == 1) {
    if (warp >= 2 && alive) {
#pragma unroll
      for (int c = 0; c < T; ++c) store(row0 + c, acc[c]);
    }
  } else {
    // partial sums [T][128] over the stages, which every multiplication has read to the end
    float* partial = (float*)smem;
    if (warp >= 2) {
#pragma unroll
      for (int c = 0; c < T; ++c) partial[c * 128 + f] = acc[c];
    }
    ptx::cluster_sync();
    if (warp >= 2 && alive) {
      const int c0 = T * rank / split, c1 = T * (rank + 1) / split;
      for (int c = c0; c < c1; ++c) {
        float sum = 0.0f;
        for (int r = 0; r < split; ++r) sum += ptx::ld_cluster_f32(ptx::map_to_cta(&partial[c * 128 + f], (uint32_t)r));
        store(row0 + c, sum);
      }
    }
    ptx::cluster_sync();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  if (warp == 1) ptx::tmem_dealloc(tmem_base, kCols);
}

// ------------------------------------------------------------------------------------------------ host

bool encode_rows(CUtensorMap* map, const void* base, int64_t rows, int64_t K, int box_rows) {
  const uint64_t dims[2] = {(uint64_t)K, (uint64_t)rows}, strides[1] = {(uint64_t)K};
  const uint32_t box[2] = {kBlockK, (uint32_t)box_rows};
  return encode_fresh(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, base, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

template <int BN>
sdgp_status launch_pair(const void* xq, const void* wq, Fp8Params p, int64_t K, cudaStream_t stream) {
  static bool done[kMaxDevices] = {};
  if (!configure_once(fp8_pair_kernel<BN>, done)) return SDGP_ERR_CUDA;
  CUtensorMap tx, tw;
  if (!encode_rows(&tx, xq, p.rows, K, 128) || !encode_rows(&tw, wq, p.features, K, BN / 2)) return SDGP_ERR_CUDA;
  constexpr int stage = kTileBytes + BN / 2 * kBlockK;
  p.stages = (kSmemLimit - kSmemSlack) / stage;
  if (p.stages > kPairMaxStages) p.stages = kPairMaxStages;
  p.tiles_n = (int)((p.features + BN - 1) / BN);
  const int64_t tiles = (p.rows + 255) / 256 * p.tiles_n;
  if (tiles > 0x7FFFFFFF) return SDGP_ERR_UNSUPPORTED;
  p.tiles = (int)tiles;
  return launch_pairs(fp8_pair_kernel<BN>, pairs_for(p.tiles), kPairThreads, p.stages * stage + kSmemSlack, stream, tx, tw, p);
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
  while (split < 8 && 2 * split * tiles <= sm_count() && 4 * split <= p.blocks) split *= 2;
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
  p.sx = x_scale;
  p.sw = w_scale;
  p.y = y;
  p.rows = rows;
  p.features = features;
  p.blocks = (int)((K + kBlockK - 1) / kBlockK);
  p.dtype = dtype;
  p.aligned32 = (((uintptr_t)y | (uint64_t)features * (dtype == SDGP_FP32 ? 4 : 2)) & 31u) == 0;
  if (rows <= 16) return launch_rows<16>(xq, wq, p, K, stream);
  if (rows <= 32) return launch_rows<32>(xq, wq, p, K, stream);
  if (rows <= 64) return launch_rows<64>(xq, wq, p, K, stream);
  const int64_t pair_tiles = (rows + 255) / 256 * ((features + 255) / 256);
  if (rows <= 128 || !p.aligned32 || pair_tiles * 4 < sm_count()) return launch_rows<128>(xq, wq, p, K, stream);
  return launch_pair<256>(xq, wq, p, K, stream);
}

}  // namespace sdgp
