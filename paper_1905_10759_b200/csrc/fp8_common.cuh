// Device helpers shared by the kernels of 8-bit operands: e4m3 conversions, and loads that stay where they are written (a kernel
// launched with launch_pdl lives before the data it reads does: plain loads behind pdl_wait, never the read-only kind).
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

namespace hbmm {
namespace fp8 {

constexpr int kGroup = 128;                   // elements along a row per scale

__device__ __forceinline__ uint4 load16(const void* p) {
  uint4 v;
  asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 load8(const void* p) {
  uint2 v;
  asm volatile("ld.global.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}
__device__ __forceinline__ uint32_t load4(const void* p) {
  uint32_t v;
  asm volatile("ld.global.u32 %0, [%1];" : "=r"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ uint32_t load1(const void* p) {
  uint32_t v;
  asm volatile("ld.global.u8 %0, [%1];" : "=r"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ float loadf(const float* p) { return __uint_as_float(load4(p)); }

// A walk over the (row, chunk) pairs of a matrix, row by row, `step` pairs at a time: without the division per turn that the pair's
// number would take (64-bit, 80 instructions; a third of what the quantizer executed).
struct RowWalk {
  int64_t row, chunk, chunks, step_rows, step_chunks;
  __device__ __forceinline__ RowWalk(int64_t first, int64_t step, int64_t chunks_) : chunks(chunks_) {
    row = first / chunks; chunk = first - row * chunks;
    step_rows = step / chunks; step_chunks = step - step_rows * chunks;
  }
  __device__ __forceinline__ void next() {
    row += step_rows; chunk += step_chunks;
    if (chunk >= chunks) { chunk -= chunks; row++; }
  }
};

// Two fp32 -> two codes (lo in the low byte), nearest even; magnitudes above 448 saturate, NaN gives the NaN code.
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
  unsigned short r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t to_e4m3x4(float a, float b, float c, float d) { return to_e4m3x2(a, b) | to_e4m3x2(c, d) << 16; }

// Two codes (in the low 16 bits) -> their values, exact (every e4m3 number is an fp16 number).
__device__ __forceinline__ float2 from_e4m3x2(uint32_t codes) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<unsigned short>(codes)));
  float2 f;
  asm("{\n\t.reg .b16 l, u;\n\tmov.b32 {l, u}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, u;\n\t}" : "=f"(f.x), "=f"(f.y) : "r"(h));
  return f;
}

__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// The scale of a group from the bits of its largest finite magnitude: the smallest power of two s with amax / s <= 448, at
// least 2^-117 (448 = 1.75 * 2^8).  Exponent fields only, so exact for subnormal amax too (their field is 0: the floor).
__device__ __forceinline__ uint32_t scale_exponent(uint32_t amax_bits) {
  const int e = static_cast<int>(amax_bits >> 23) - 8 + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return static_cast<uint32_t>(e < 10 ? 10 : e);
}
__device__ __forceinline__ float pow2_of(uint32_t exponent) { return __uint_as_float(exponent << 23); }
__device__ __forceinline__ float pow2_inverse(uint32_t exponent) { return __uint_as_float((254u - exponent) << 23); }

// x / s for the conversion; + 0 so that -0 leaves as +0 (a tiny negative product rounds to -0 and keeps its sign bit).
__device__ __forceinline__ float scaled(float x, float inverse) { return fmaf(x, inverse, 0.0f); }

}  // namespace fp8
}  // namespace hbmm
