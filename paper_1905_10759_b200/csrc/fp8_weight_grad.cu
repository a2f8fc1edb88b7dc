// Weight gradient from the 8-bit copy of the activations: GW = gy^T X^ (+ base) (see include/hbmm.h).
// One thread per output, sums in fp32.
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

}  // namespace

cudaError_t launch_fp8_weight_grad(const void* gy, int64_t N, int64_t ldg, const Fp8View& X, const float* base, int64_t ld_base, float* gw,
                                   int64_t ldw, cudaStream_t stream) {
  int dev = 0, sms = 0;
  const cudaError_t e = current_device(&dev, &sms);
  if (e != cudaSuccess) return e;
  const int64_t n = (N * X.K + kThreads - 1) / kThreads, cap = static_cast<int64_t>(sms) * 8;
  return launch_pdl(fp8_weight_grad_plain, dim3(static_cast<unsigned>(n < cap ? n : cap)), dim3(kThreads), 0, stream,
                    static_cast<const __nv_bfloat16*>(gy), N, ldg, X, base, ld_base, gw, ldw);
}

}  // namespace hbmm
