// Elements of the tensors of the language-model kernels (logprob.cu, norm.cu, fp8_quantize.cu): bf16, binary16 or fp32 in memory, fp32 in
// registers, eight at a time.
#pragma once
#include "prune_core.cuh"
#include "ptx.cuh"

namespace sdgp {
namespace {

template <int DT>
struct Element {  // DT: sdgp_dtype
  static constexpr bool kF16 = DT == SDGP_FP16;
  static constexpr bool k32 = DT == SDGP_FP32;
  static constexpr int kBytes = k32 ? 4 : 2;

  static __device__ __forceinline__ float load(const void* p, int64_t i) {
    if constexpr (k32) return ((const float*)p)[i];
    else return lane_lo<kF16>((uint32_t)((const uint16_t*)p)[i]);
  }
  static __device__ __forceinline__ void store(void* p, int64_t i, float x) {
    if constexpr (k32) ((float*)p)[i] = x;
    else ((uint16_t*)p)[i] = (uint16_t)f32_to_elem_bits<kF16>(x);
  }
  // Eight elements as they lie in memory (16 bytes, or 32 of fp32); `i` a multiple of 8 and the tensor 16-byte aligned.
  struct Raw {
    uint4 a, b;  // b: fp32 only
  };
  static __device__ __forceinline__ Raw load8(const void* p, int64_t i) {
    Raw r;
    const uint4* q = (const uint4*)((const uint8_t*)p + i * kBytes);
    r.a = q[0];
    r.b = k32 ? q[1] : make_uint4(0u, 0u, 0u, 0u);
    return r;
  }
  // Eight times -infinity.
  static __device__ __forceinline__ Raw lowest8() {
    const uint32_t w = k32 ? 0xFF800000u : kF16 ? 0xFC00FC00u : 0xFF80FF80u;
    Raw r;
    r.a = r.b = make_uint4(w, w, w, w);
    return r;
  }
  static __device__ __forceinline__ void widen(const Raw& r, float (&x)[8]) {
    if constexpr (k32) {
      const uint32_t w[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(w[e]);
    } else {
      const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[2 * e] = lane_lo<kF16>(w[e]);
        x[2 * e + 1] = lane_hi<kF16>(w[e]);
      }
    }
  }
  // The largest of eight; NaN is passed over (-infinity or NaN if there is nothing else).
  static __device__ __forceinline__ float largest(const Raw& r, const float (&x)[8]) {
    if constexpr (k32) {
      return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    } else {  // two at a time
      uint32_t m;
      if constexpr (kF16) {
        const __half2 h = __hmax2(__hmax2(*(const __half2*)&r.a.x, *(const __half2*)&r.a.y), __hmax2(*(const __half2*)&r.a.z, *(const __half2*)&r.a.w));
        m = *(const uint32_t*)&h;
      } else {
        const __nv_bfloat162 h = __hmax2(__hmax2(*(const __nv_bfloat162*)&r.a.x, *(const __nv_bfloat162*)&r.a.y),
                                         __hmax2(*(const __nv_bfloat162*)&r.a.z, *(const __nv_bfloat162*)&r.a.w));
        m = *(const uint32_t*)&h;
      }
      return fmaxf(lane_lo<kF16>(m), lane_hi<kF16>(m));
    }
  }
  // Rounded to nearest even.
  static __device__ __forceinline__ Raw narrow(const float (&x)[8]) {
    Raw r;
    if constexpr (k32) {
      r.a = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
      r.b = make_uint4(__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7]));
    } else {
      r.a = make_uint4(pack_pair_rn<kF16>(x[0], x[1]), pack_pair_rn<kF16>(x[2], x[3]), pack_pair_rn<kF16>(x[4], x[5]),
                       pack_pair_rn<kF16>(x[6], x[7]));
      r.b = make_uint4(0u, 0u, 0u, 0u);
    }
    return r;
  }
  static __device__ __forceinline__ void store8(void* p, int64_t i, const Raw& r) {
    uint4* q = (uint4*)((uint8_t*)p + i * kBytes);
    if (k32 && ((uintptr_t)q & 31u) == 0) {  // a whole sector at once
      const uint32_t w[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
      ptx::st_global_256(q, w);
      return;
    }
    q[0] = r.a;
    if (k32) q[1] = r.b;
  }
};

// The larger of two numbers; NaN if one of them is.
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}

// Two fp32 operations in one instruction: half the issue slots of kernels that memory should bound.
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 w, {%6, %7};\n\t"
      "fma.rn.f32x2 z, x, y, w;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
  return x;
}

__device__ __forceinline__ float exp2_approx(float x) {  // 2^x, relative error about 2^-22; subnormal results are zero
  float d;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(x));
  return d;
}

}  // namespace
}  // namespace sdgp
