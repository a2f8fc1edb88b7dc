// Products of few rows of an 8-bit operand (single tokens and small batches): C = A^ W^^T for at most 16 rows of A.
//
// Bound by reading W once.  A CTA takes 16 rows of W; its warps take the groups of 128 elements in turn, so that what is in flight is
// 2 KB per warp and group.  A warp forms the group's 16 x 8 dot products with four m16n8k32 e4m3 mma.sync (rows of W are the
// instruction's rows, rows of A its columns), scales them into fp32 registers and the warps' sums are added in warp order at the end.
// Each lane reads 32 consecutive bytes of two rows of W (and of its row of A); which 32 elements of the group meet in which
// instruction does not matter as long as both operands agree, so lane t of a quad takes bytes 32 t .. 32 t + 31.
// MEASURED
#include <cuda_bf16.h>
#include "fp8_common.cuh"
#include "kernels.h"
#include "pdl.cuh"

namespace hbmm {
namespace {

using namespace fp8;

constexpr int kRowsW = 16;

struct Args {
  const uint8_t* a; int64_t ld_a;
  const float* a_s; int64_t ld_as;
  const uint8_t* w; int64_t ld_w;
  const float* w_s; int64_t ld_ws;
  void* c; int64_t ldc; int32_t c_bf16;
  int32_t M;
  int64_t N, K, groups;
};

__device__ __forceinline__ void mma_e4m3(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 16 codes of a row from column k on; zeros past its end.
__device__ __forceinline__ uint4 codes16(const uint8_t* row, int64_t k, int64_t K, bool in) {
  if (in && k + 16 <= K) return load16(row + k);
  uint32_t w[4] = {0, 0, 0, 0};
  if (in)
    for (int e = 0; e < 16; e++)
      if (k + e < K) w[e / 4] |= load1(row + k + e) << (8 * (e % 4));
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// COLS: columns of A rows in eights (1: up to 8 rows of A, 2: up to 16).
template <int COLS, int WARPS>
__global__ void __launch_bounds__(WARPS * 32)
fp8_gemv_kernel(const Args g) {
  __shared__ float part[WARPS][kRowsW][8 * COLS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = lane >> 2, quad = lane & 3;
  const int64_t n0 = static_cast<int64_t>(blockIdx.x) * kRowsW;
  pdl_wait();
  const bool in0 = n0 + row < g.N, in1 = n0 + row + 8 < g.N;
  const uint8_t *w0 = g.w + (in0 ? n0 + row : 0) * g.ld_w, *w1 = g.w + (in1 ? n0 + row + 8 : 0) * g.ld_w;
  const float* ws = g.w_s + n0 / kGroup * g.ld_ws;       // 16 rows lie in one block of 128
  float acc[COLS][4];
#pragma unroll
  for (int t = 0; t < COLS; t++)
#pragma unroll
    for (int e = 0; e < 4; e++) acc[t][e] = 0.0f;
  for (int64_t gr = warp; gr < g.groups; gr += WARPS) {
    const int64_t k = gr * kGroup + quad * 32;
    const uint4 x0 = codes16(w0, k, g.K, in0), x1 = codes16(w0, k + 16, g.K, in0);
    const uint4 y0 = codes16(w1, k, g.K, in1), y1 = codes16(w1, k + 16, g.K, in1);
    const uint32_t x[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w}, y[8] = {y0.x, y0.y, y0.z, y0.w, y1.x, y1.y, y1.z, y1.w};
    const float sw = loadf(ws + gr);
#pragma unroll
    for (int t = 0; t < COLS; t++) {
      const int m = 8 * t + row;                         // this lane's row of A as an operand
      const bool in = m < g.M;
      const uint8_t* ar = g.a + (in ? m : 0) * g.ld_a;
      const uint4 b0 = codes16(ar, k, g.K, in), b1 = codes16(ar, k + 16, g.K, in);
      const uint32_t b[8] = {b0.x, b0.y, b0.z, b0.w, b1.x, b1.y, b1.z, b1.w};
      const int c0 = 8 * t + 2 * quad;                   // this lane's rows of A in the result
      const float s0 = c0 < g.M ? loadf(g.a_s + c0 * g.ld_as + gr) * sw : 0.0f, s1 = c0 + 1 < g.M ? loadf(g.a_s + (c0 + 1) * g.ld_as + gr) * sw : 0.0f;
      float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int q = 0; q < 4; q++) {
        const uint32_t a[4] = {x[2 * q], y[2 * q], x[2 * q + 1], y[2 * q + 1]};
        mma_e4m3(d, a, b[2 * q], b[2 * q + 1]);
      }
      acc[t][0] = fmaf(s0, d[0], acc[t][0]);
      acc[t][1] = fmaf(s1, d[1], acc[t][1]);
      acc[t][2] = fmaf(s0, d[2], acc[t][2]);
      acc[t][3] = fmaf(s1, d[3], acc[t][3]);
    }
  }
#pragma unroll
  for (int t = 0; t < COLS; t++) {
    part[warp][row][8 * t + 2 * quad] = acc[t][0];
    part[warp][row][8 * t + 2 * quad + 1] = acc[t][1];
    part[warp][row + 8][8 * t + 2 * quad] = acc[t][2];
    part[warp][row + 8][8 * t + 2 * quad + 1] = acc[t][3];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < kRowsW * 8 * COLS; i += WARPS * 32) {
    const int n = i % kRowsW, m = i / kRowsW;
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < WARPS; w++) sum += part[w][n][m];
    if (m < g.M && n0 + n < g.N) {
      if (g.c_bf16) static_cast<__nv_bfloat16*>(g.c)[m * g.ldc + n0 + n] = __float2bfloat16_rn(sum);
      else static_cast<float*>(g.c)[m * g.ldc + n0 + n] = sum;
    }
  }
}

}  // namespace

bool fp8_gemv_supported(const Fp8View& A) { return A.rows <= 16; }

cudaError_t launch_fp8_gemv(const Fp8View& A, const Fp8View& W, void* C, bool c_bf16, int64_t ldc, cudaStream_t stream) {
  const Args g{A.codes, A.ld, A.scales, A.ld_s, W.codes, W.ld, W.scales, W.ld_s, C, ldc, c_bf16 ? 1 : 0, static_cast<int32_t>(A.rows), W.rows, A.K,
               (A.K + kGroup - 1) / kGroup};
  const dim3 grid(static_cast<unsigned>((W.rows + kRowsW - 1) / kRowsW));
  if (A.rows > 8) return launch_pdl(fp8_gemv_kernel<2, 16>, grid, dim3(16 * 32), 0, stream, g);
  return launch_pdl(fp8_gemv_kernel<1, 16>, grid, dim3(16 * 32), 0, stream, g);
}

}  // namespace hbmm
