// Products of few rows of an 8-bit operand (single tokens and small batches): C = A^ W^^T for at most 16 rows of A.
//
// Bound by reading W once.  A CTA takes 16 rows of W; its warps take the groups of 128 elements in turn, so that what is in flight is
// 2 KB per warp and group.  A warp forms the group's 16 x 8 dot products with four m16n8k32 e4m3 mma.sync (rows of W are the
// instruction's rows, rows of A its columns), scales them into fp32 registers and the warps' sums are added in warp order at the end.
// Each lane reads 32 consecutive bytes of two rows of W (and of its row of A); which 32 elements of the group meet in which
// instruction does not matter as long as both operands agree, so lane t of a quad takes bytes 32 t .. 32 t + 31.
#include <cuda_bf16.h>
#include <type_traits>
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
// 16 codes of a row from column k on; zeros past its end (WHOLE: it does not end before).
template <bool WHOLE>
__device__ __forceinline__ uint4 codes16(const uint8_t* row, int64_t k, int64_t K) {
  if (WHOLE || k + 16 <= K) return load16(row + k);
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < 16; e++)
    if (k + e < K) w[e / 4] |= load1(row + k + e) << (8 * (e % 4));
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// COLS: rows of A in eights.  WARPS, DEEP: warps per CTA and groups that a warp loads at a time.  Weights from memory, launch included:
// 1 x 4096 x 9216 9.2 us, 1 x 8192 x 8192 14.9 (4.5 TB/s), 1 x 4096 x 4096 5.7, 1 x 1000 x 4096 3.6; 16 x 8192 x 8192 20.6.  How the
// choices compared, before the loads of whole groups lost their checks (16 warps with single groups / 8 with two / 8 with three): 1 x
// 4096 x 9216 15.6 / 13.5 / 12.4 us, 1 x 4096 x 4096 8.2 / 7.0 / 7.5, 1 x 1000 x 4096 (63 CTAs) 4.2 / 5.6 / 5.7, 16 with two 4.1; 16 rows
// of A, 4096 x 9216, from L2, 17.6 us with 16 and 1, 12.5 with 8 and 2.  Groups kept in flight in a ring instead: 1 x 4096 x 9216 14.7.
template <int COLS, int WARPS, int DEEP>
__global__ void __launch_bounds__(WARPS * 32, WARPS == 16 ? 1 : 2)
fp8_gemv_kernel(const Args g) {
  __shared__ float part[WARPS][kRowsW][8 * COLS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = lane >> 2, quad = lane & 3;
  const int64_t n0 = static_cast<int64_t>(blockIdx.x) * kRowsW;
  pdl_wait();
  // a row past the end of an operand reads the first one: what comes of it is not stored
  const uint8_t *w0 = g.w + (n0 + row < g.N ? n0 + row : 0) * g.ld_w, *w1 = g.w + (n0 + row + 8 < g.N ? n0 + row + 8 : 0) * g.ld_w;
  const float* ws = g.w_s + n0 / kGroup * g.ld_ws;       // 16 rows lie in one block of 128
  const uint8_t* ar[COLS];
  const float *s0[COLS], *s1[COLS];
#pragma unroll
  for (int t = 0; t < COLS; t++) {
    const int m = 8 * t + row, c = 8 * t + 2 * quad;     // this lane's row of A as an operand, its two in the result
    ar[t] = g.a + (m < g.M ? m : 0) * g.ld_a;
    s0[t] = g.a_s + (c < g.M ? c : 0) * g.ld_as;
    s1[t] = g.a_s + (c + 1 < g.M ? c + 1 : 0) * g.ld_as;
  }
  float acc[COLS][4];
#pragma unroll
  for (int t = 0; t < COLS; t++)
#pragma unroll
    for (int e = 0; e < 4; e++) acc[t][e] = 0.0f;
  struct Loads { uint4 w[4], a[COLS][2]; float s[COLS][2], sw; };
  const auto fetch = [&](auto whole, int64_t gr, Loads& l) {
    constexpr bool WHOLE = decltype(whole)::value;
    const int64_t k = gr * kGroup + quad * 32;
    l.w[0] = codes16<WHOLE>(w0, k, g.K); l.w[1] = codes16<WHOLE>(w0, k + 16, g.K);
    l.w[2] = codes16<WHOLE>(w1, k, g.K); l.w[3] = codes16<WHOLE>(w1, k + 16, g.K);
    l.sw = loadf(ws + gr);
#pragma unroll
    for (int t = 0; t < COLS; t++) {
      l.a[t][0] = codes16<WHOLE>(ar[t], k, g.K); l.a[t][1] = codes16<WHOLE>(ar[t], k + 16, g.K);
      l.s[t][0] = loadf(s0[t] + gr);
      l.s[t][1] = loadf(s1[t] + gr);
    }
  };
  const auto add = [&](const Loads& l) {
    const uint32_t x[8] = {l.w[0].x, l.w[0].y, l.w[0].z, l.w[0].w, l.w[1].x, l.w[1].y, l.w[1].z, l.w[1].w};
    const uint32_t y[8] = {l.w[2].x, l.w[2].y, l.w[2].z, l.w[2].w, l.w[3].x, l.w[3].y, l.w[3].z, l.w[3].w};
#pragma unroll
    for (int t = 0; t < COLS; t++) {
      const uint32_t b[8] = {l.a[t][0].x, l.a[t][0].y, l.a[t][0].z, l.a[t][0].w, l.a[t][1].x, l.a[t][1].y, l.a[t][1].z, l.a[t][1].w};
      const float f0 = l.s[t][0] * l.sw, f1 = l.s[t][1] * l.sw;
      float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int q = 0; q < 4; q++) {
        const uint32_t a[4] = {x[2 * q], y[2 * q], x[2 * q + 1], y[2 * q + 1]};
        mma_e4m3(d, a, b[2 * q], b[2 * q + 1]);
      }
      acc[t][0] = fmaf(f0, d[0], acc[t][0]);
      acc[t][1] = fmaf(f1, d[1], acc[t][1]);
      acc[t][2] = fmaf(f0, d[2], acc[t][2]);
      acc[t][3] = fmaf(f1, d[3], acc[t][3]);
    }
  };
  const int64_t full = g.K / kGroup;
  int64_t gr = warp;
  for (; gr + (DEEP - 1) * WARPS < full; gr += DEEP * WARPS) {
    Loads l[DEEP];
#pragma unroll
    for (int i = 0; i < DEEP; i++) fetch(std::true_type(), gr + i * WARPS, l[i]);
#pragma unroll
    for (int i = 0; i < DEEP; i++) add(l[i]);
  }
  Loads rest[DEEP];                                      // fewer than DEEP groups of this warp, the last one perhaps short
#pragma unroll
  for (int i = 0; i < DEEP; i++) {
    const int64_t at = gr + i * WARPS;
    if (at < full) fetch(std::true_type(), at, rest[i]);
    else if (at < g.groups) fetch(std::false_type(), at, rest[i]);
  }
#pragma unroll
  for (int i = 0; i < DEEP; i++)
    if (gr + i * WARPS < g.groups) add(rest[i]);
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
  int dev = 0, sms = 0;
  const cudaError_t e = current_device(&dev, &sms);
  if (e != cudaSuccess) return e;
  if (A.rows > 8) return launch_pdl(fp8_gemv_kernel<2, 8, 2>, grid, dim3(8 * 32), 0, stream, g);
  // one CTA per SM or fewer: more warps each; else two per SM, the longer rows with three groups in flight
  if (static_cast<int>(grid.x) <= sms) return launch_pdl(fp8_gemv_kernel<1, 16, 2>, grid, dim3(16 * 32), 0, stream, g);
  if (g.groups <= 32) return launch_pdl(fp8_gemv_kernel<1, 8, 2>, grid, dim3(8 * 32), 0, stream, g);
  return launch_pdl(fp8_gemv_kernel<1, 8, 3>, grid, dim3(8 * 32), 0, stream, g);
}

}  // namespace hbmm
