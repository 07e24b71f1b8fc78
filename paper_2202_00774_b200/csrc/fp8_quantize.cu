// Quantisation to e4m3 with a scale for each block of 128 columns of a row (activations) or of 128 x 128 elements (weights), sm_100a.
//
// The scale of a block is the power of two s with max|x| / s in (224, 448] (448 is the largest e4m3 number; 1 for a block of zeros, at
// least 2^-126): x / s is exact in fp32, so an element is rounded once. A scale that is no power of two would use the last half of a
// binade of range more, and round twice. A block with a NaN or an infinity gets the scale NaN and NaN elements: the product it
// enters is NaN, not a wrong number.
//
// Both kernels are a pure stream, one read and one write of half the size (a quarter, of fp32): a thread takes 16 elements in two wide
// loads, eight neighbouring lanes a row of a block.
#include "elements.cuh"
#include "ptx.cuh"
#include "sdgp_internal.cuh"

namespace sdgp {
namespace {

constexpr int kThreads = 256;

// Bit pattern of the scale and of its reciprocal, from the bits of max|x|.
__device__ __forceinline__ void scale_of(uint32_t most, float& scale, float& inverse) {
  if (most >= 0x7F800000u) {
    scale = inverse = __uint_as_float(0x7FC00000u);
    return;
  }
  // max|x| = 1.f 2^e; 448 = 1.75 2^8
  const int e = max((int)(most >> 23) - 8 + ((most & 0x7FFFFFu) > 0x600000u ? 1 : 0), 1);
  const int biased = most == 0u ? 127 : e;
  scale = __uint_as_float((uint32_t)biased << 23);
  inverse = __uint_as_float((uint32_t)(254 - biased) << 23);
}

__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return (uint32_t)lo | (uint32_t)hi << 16;
}

template <int DT>
struct Sixteen {
  typename Element<DT>::Raw r[2];
};
template <int DT>
__device__ __forceinline__ Sixteen<DT> load16(const void* x, int64_t at, bool live) {
  Sixteen<DT> s;
  if (live) {
    s.r[0] = Element<DT>::load8(x, at);
    s.r[1] = Element<DT>::load8(x, at + 8);
  } else {
    s.r[0].a = s.r[0].b = s.r[1].a = s.r[1].b = make_uint4(0u, 0u, 0u, 0u);
  }
  return s;
}
// Bits of the largest magnitude (NaN above infinity above numbers).
template <int DT>
__device__ __forceinline__ uint32_t largest16(const Sixteen<DT>& s) {
  uint32_t most = 0;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float x[8];
    Element<DT>::widen(s.r[h], x);
#pragma unroll
    for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(x[e]) & 0x7FFFFFFFu);
  }
  return most;
}
template <int DT>
__device__ __forceinline__ uint4 quantize16(const Sixteen<DT>& s, float inverse) {
  float x[2][8];
  Element<DT>::widen(s.r[0], x[0]);
  Element<DT>::widen(s.r[1], x[1]);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    x[0][e] *= inverse;
    x[1][e] *= inverse;
  }
  return make_uint4(to_e4m3x4(x[0][0], x[0][1], x[0][2], x[0][3]), to_e4m3x4(x[0][4], x[0][5], x[0][6], x[0][7]),
                    to_e4m3x4(x[1][0], x[1][1], x[1][2], x[1][3]), to_e4m3x4(x[1][4], x[1][5], x[1][6], x[1][7]));
}

// A scale for each row: eight lanes a block, `kRounds` blocks of each in flight.
constexpr int kRounds = 2;
template <int DT>
__global__ void __launch_bounds__(kThreads)
quantize_rows_kernel(const void* __restrict__ x, int64_t blocks, int K, int row_blocks, uint8_t* __restrict__ q, float* __restrict__ scale) {
  ptx::wait_for_previous_grid();
  ptx::launch_dependents();
  const int lane8 = threadIdx.x & 7;
  const int64_t first = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 3, stride = (int64_t)gridDim.x * (kThreads / 8);
  Sixteen<DT> s[kRounds];
  int64_t at[kRounds];
  bool live[kRounds];
#pragma unroll
  for (int i = 0; i < kRounds; ++i) {
    const int64_t b = first + i * stride;
    const int64_t row = blocks <= 0xFFFFFFFFll ? (int64_t)((uint32_t)b / (uint32_t)row_blocks) : b / row_blocks;
    const int col = (int)(b - row * row_blocks) * 128 + lane8 * 16;
    live[i] = b < blocks && col < K;
    at[i] = row * K + col;
    s[i] = load16<DT>(x, at[i], live[i]);
  }
#pragma unroll
  for (int i = 0; i < kRounds; ++i) {
    uint32_t most = largest16(s[i]);
#pragma unroll
    for (int d = 4; d > 0; d >>= 1) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
    float sc, inverse;
    scale_of(most, sc, inverse);
    if (live[i]) *(uint4*)(q + at[i]) = quantize16(s[i], inverse);
    const int64_t b = first + i * stride;
    if (lane8 == 0 && b < blocks) scale[b] = sc;
  }
}

// A scale for each 128 x 128 block: one CTA, four rows' parts of 16 a thread, kept in registers between the maximum and the rounding.
template <int DT>
__global__ void __launch_bounds__(kThreads)
quantize_squares_kernel(const void* __restrict__ x, int64_t rows, int K, int row_blocks, uint8_t* __restrict__ q, float* __restrict__ scale) {
  __shared__ uint32_t found[kThreads / 32];
  ptx::wait_for_previous_grid();
  ptx::launch_dependents();
  const int64_t block_row = blockIdx.x / row_blocks;
  const int col = (int)(blockIdx.x - block_row * row_blocks) * 128 + (threadIdx.x & 7) * 16;
  Sixteen<DT> s[4];
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t row = block_row * 128 + i * 32 + (threadIdx.x >> 3);
    s[i] = load16<DT>(x, row * K + col, row < rows && col < K);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) most = max(most, largest16(s[i]));
  most = __reduce_max_sync(0xFFFFFFFFu, most);
  if ((threadIdx.x & 31) == 0) found[threadIdx.x >> 5] = most;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) most = max(most, found[w]);
  float sc, inverse;
  scale_of(most, sc, inverse);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t row = block_row * 128 + i * 32 + (threadIdx.x >> 3);
    if (row < rows && col < K) *(uint4*)(q + row * K + col) = quantize16(s[i], inverse);
  }
  if (threadIdx.x == 0) scale[blockIdx.x] = sc;
}

template <typename... Params, typename... Args>
cudaError_t launch(void (*kernel)(Params...), int64_t ctas, cudaStream_t stream, Args... args) {
  if (ctas > 0x7FFFFFFF) return cudaErrorInvalidValue;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
}

template <int DT>
cudaError_t launch_typed(const void* x, int64_t rows, int64_t K, int block_rows, void* q, float* scale, cudaStream_t stream) {
  const int64_t row_blocks = (K + 127) / 128;
  if (block_rows == 128)
    return launch(quantize_squares_kernel<DT>, (rows + 127) / 128 * row_blocks, stream, x, rows, K, row_blocks, q, scale);
  const int64_t blocks = rows * row_blocks, per_cta = kThreads / 8 * kRounds;
  return launch(quantize_rows_kernel<DT>, (blocks + per_cta - 1) / per_cta, stream, x, blocks, K, row_blocks, q, scale);
}

}  // namespace

cudaError_t launch_fp8_quantize(const void* x, int64_t rows, int64_t K, int block_rows, int dtype, void* q, float* scale, cudaStream_t stream) {
  if (dtype == SDGP_BF16) return launch_typed<SDGP_BF16>(x, rows, K, block_rows, q, scale, stream);
  if (dtype == SDGP_FP16) return launch_typed<SDGP_FP16>(x, rows, K, block_rows, q, scale, stream);
  return launch_typed<SDGP_FP32>(x, rows, K, block_rows, q, scale, stream);
}

}  // namespace sdgp
