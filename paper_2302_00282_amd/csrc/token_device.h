// Device-side vocabulary of the token kernels: reductions over a wavefront, and the rounding that quantised rows share.
#pragma once
#include "device_common.h"
#include "token_kernels.h"

namespace xenos {

typedef __attribute__((ext_vector_type(4))) int i32x4_t;
typedef __attribute__((ext_vector_type(16))) int i32x16_t;

// The largest |value| by its bits: a NaN's are above infinity's, so that it stays.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = umax(v, (uint32_t)__shfl_xor((int)v, o));
  return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

// The bare instruction, as fmx_raw: for values from loads and plain arithmetic (the compiler adds no waits for what an instruction in assembly reads)
__device__ __forceinline__ float max3_raw(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// The step of a row whose largest magnitude has the bits m: q = rint(v inv), and q times scale() stands for v.
struct RowStep {
  float amp, inv;
  __device__ __forceinline__ explicit RowStep(uint32_t m) : amp(__uint_as_float(umax(m, __float_as_uint(kTinyAmplitude)))), inv(127.f / amp) {}
  __device__ __forceinline__ float scale() const { return amp / 127.f; }
  __device__ __forceinline__ int operator()(float v) const { return (int)rintf(v * inv); }
};

}  // namespace xenos
