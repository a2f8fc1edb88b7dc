// Products of 8-bit operands: C = A^ W^^T and C = A^ W^ (see include/hbmm.h), and the weight gradient gy^T X^ (+ base).
// One thread per output, sums in fp32: a group's dot product first, then its scales.
#include <cuda_bf16.h>
#include "fp8_common.cuh"
#include "kernels.h"
#include "pdl.cuh"

namespace hbmm {
namespace {

using namespace fp8;

constexpr int kThreads = 256;

__device__ __forceinline__ float value(const uint8_t* p) { return from_e4m3x2(load1(p)).x; }

__global__ void __launch_bounds__(kThreads)
fp8_gemm_plain(const Fp8View A, const Fp8View W, int transposed, void* C, int c_bf16, int64_t ldc) {
  pdl_wait();
  const int64_t N = transposed ? W.K : W.rows, total = A.rows * N;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * kThreads) {
    const int64_t m = i / N, n = i - m * N;
    float sum = 0.0f;
    for (int64_t k0 = 0; k0 < A.K; k0 += kGroup) {
      const int64_t k1 = k0 + kGroup < A.K ? k0 + kGroup : A.K;
      float dot = 0.0f;
      for (int64_t k = k0; k < k1; k++) dot += value(A.codes + m * A.ld + k) * value(transposed ? W.codes + k * W.ld + n : W.codes + n * W.ld + k);
      const int64_t g = k0 / kGroup, nb = n / kGroup;
      sum += dot * (loadf(A.scales + m * A.ld_s + g) * loadf(transposed ? W.scales + g * W.ld_s + nb : W.scales + nb * W.ld_s + g));
    }
    if (c_bf16) static_cast<__nv_bfloat16*>(C)[m * ldc + n] = __float2bfloat16_rn(sum);
    else static_cast<float*>(C)[m * ldc + n] = sum;
  }
}

__global__ void __launch_bounds__(kThreads)
fp8_weight_grad_plain(const __nv_bfloat16* gy, int64_t N, int64_t ldg, const Fp8View X, const float* base, int64_t ld_base, float* gw, int64_t ldw) {
  pdl_wait();
  const int64_t total = N * X.K;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * kThreads) {
    const int64_t n = i / X.K, k = i - n * X.K;
    float sum = 0.0f;
    for (int64_t m = 0; m < X.rows; m++) {
      const float x = __bfloat162float(__float2bfloat16_rn(value(X.codes + m * X.ld + k) * loadf(X.scales + m * X.ld_s + k / kGroup)));
      sum += load_elem<__nv_bfloat16>(gy + m * ldg + n) * x;
    }
    gw[n * ldw + k] = base ? loadf(base + n * ld_base + k) + sum : sum;
  }
}

dim3 grid_of(int64_t total, int sms) {
  const int64_t n = (total + kThreads - 1) / kThreads, cap = static_cast<int64_t>(sms) * 8;
  return dim3(static_cast<unsigned>(n < cap ? n : cap));
}

}  // namespace

cudaError_t launch_fp8_gemm(const Fp8View& A, const Fp8View& W, bool transposed, void* C, bool c_bf16, int64_t ldc, cudaStream_t stream) {
  int dev = 0, sms = 0;
  const cudaError_t e = current_device(&dev, &sms);
  if (e != cudaSuccess) return e;
  return launch_pdl(fp8_gemm_plain, grid_of(A.rows * (transposed ? W.K : W.rows), sms), dim3(kThreads), 0, stream, A, W, transposed ? 1 : 0, C,
                    c_bf16 ? 1 : 0, ldc);
}

cudaError_t launch_fp8_weight_grad(const void* gy, int64_t N, int64_t ldg, const Fp8View& X, const float* base, int64_t ld_base, float* gw,
                                   int64_t ldw, cudaStream_t stream) {
  int dev = 0, sms = 0;
  const cudaError_t e = current_device(&dev, &sms);
  if (e != cudaSuccess) return e;
  return launch_pdl(fp8_weight_grad_plain, grid_of(N * X.K, sms), dim3(kThreads), 0, stream, static_cast<const __nv_bfloat16*>(gy), N, ldg, X,
                    base, ld_base, gw, ldw);
}

}  // namespace hbmm
