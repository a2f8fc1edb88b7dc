// Quantization to e4m3 with a power-of-two scale per 128 row elements, or per block of 128 x 128 elements.
//
//   s = 2^ceil(log2(amax / 448)),  code = rne(x / s)
//
// Streams, HBM bound: 4 or 2 bytes read and 1 written per element.  The scale comes from the exponent field of amax alone, x / s
// is a product with a power of two, so no step but the conversion rounds.
// Rows: a warp takes four loads of 16 bytes per lane, 512 (fp32) or 1024 (bf16) consecutive elements of a row; a load covers one
// group (fp32: the whole warp) or two (bf16: half a warp each), whose maximum is a shuffle tree over exponent-ordered integers.
// Blocks: one CTA per block keeps its 128 x 128 elements in registers (64 per thread) between the maximum and the conversion.
#include <cuda_bf16.h>
#include "fp8_common.cuh"
#include "kernels.h"
#include "pdl.cuh"

namespace hbmm {
namespace {

using namespace fp8;

constexpr int kThreads = 256;

// EPT consecutive elements from column k on; columns >= K read as zeros.  VEC: the row allows loads of whole vectors.
template <bool BF16, int EPT, bool VEC>
__device__ __forceinline__ void load_run(const void* row, int64_t k, int64_t K, float (&v)[EPT]) {
  const char* p = static_cast<const char*>(row) + k * (BF16 ? 2 : 4);
  if (VEC && k + EPT <= K) {
    uint32_t w[EPT * (BF16 ? 2 : 4) / 4];
    if constexpr (sizeof(w) == 16) { const uint4 q = load16(p); w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w; }
    else { const uint2 q = load8(p); w[0] = q.x; w[1] = q.y; }
    if constexpr (BF16) {
#pragma unroll
      for (int i = 0; i < EPT / 2; i++) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < EPT; i++) v[i] = __uint_as_float(w[i]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < EPT; e++) {
      v[e] = 0.0f;
      if (k + e < K) {
        if constexpr (BF16) v[e] = load_elem<__nv_bfloat16>(p + 2 * e);
        else v[e] = load_elem<float>(p + 4 * e);
      }
    }
  }
}

// The codes of EPT (4 or 8) consecutive elements; the row starts on 16 bytes and k is a multiple of EPT.
template <int EPT>
__device__ __forceinline__ void store_codes(uint8_t* row, int64_t k, int64_t K, const float (&v)[EPT], float inverse) {
  uint32_t c[EPT / 4];
#pragma unroll
  for (int i = 0; i < EPT / 4; i++)
    c[i] = to_e4m3x4(scaled(v[4 * i], inverse), scaled(v[4 * i + 1], inverse), scaled(v[4 * i + 2], inverse), scaled(v[4 * i + 3], inverse));
  if (k + EPT <= K) {
    if constexpr (EPT == 8) *reinterpret_cast<uint2*>(row + k) = make_uint2(c[0], c[1]);
    else *reinterpret_cast<uint32_t*>(row + k) = c[0];
  } else {
#pragma unroll
    for (int e = 0; e < EPT; e++)
      if (k + e < K) row[k + e] = static_cast<uint8_t>(c[e / 4] >> (8 * (e % 4)));
  }
}

// Largest magnitude that is no NaN (infinite where an element is).
template <int EPT>
__device__ __forceinline__ float largest(const float (&v)[EPT]) {
  float top = 0.0f;
#pragma unroll
  for (int e = 0; e < EPT; e++) top = fmaxf(top, fabsf(v[e]));
  return top;
}
// An infinity counts as NaN does: as no number.  (A group's maximum shows whether it holds one, so that most groups skip this.)
template <int EPT>
__device__ __forceinline__ void drop_infinities(float (&v)[EPT]) {
#pragma unroll
  for (int e = 0; e < EPT; e++)
    if (isinf(v[e])) v[e] = __uint_as_float(0x7FC00000u);
}

template <bool BF16, bool VEC>
__global__ void __launch_bounds__(kThreads)
fp8_quantize_rows(const void* x, int64_t rows, int64_t K, int64_t ldx, uint8_t* codes, int64_t ld, float* scales, int64_t ld_s) {
  constexpr int EPT = BF16 ? 8 : 4, LANES = kGroup / EPT, PER_LOAD = 32 * EPT, LOADS = 4;
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const int64_t chunks = (K + LOADS * PER_LOAD - 1) / (LOADS * PER_LOAD), items = rows * chunks;
  const int64_t nwarps = static_cast<int64_t>(gridDim.x) * (kThreads / 32);
  for (int64_t it = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) >> 5; it < items; it += nwarps) {     // warp-uniform
    const int64_t r = it / chunks, k0 = (it - r * chunks) * (LOADS * PER_LOAD) + lane * EPT;
    const char* row = static_cast<const char*>(x) + r * ldx * (BF16 ? 2 : 4);
    float v[LOADS][EPT];
#pragma unroll
    for (int j = 0; j < LOADS; j++) load_run<BF16, EPT, VEC>(row, k0 + j * PER_LOAD, K, v[j]);
#pragma unroll
    for (int j = 0; j < LOADS; j++) {
      const auto group_top = [&] {                      // magnitudes order as their bits do
        uint32_t top = __float_as_uint(largest<EPT>(v[j]));
        if constexpr (LANES == 32) return __reduce_max_sync(0xffffffffu, top);
#pragma unroll
        for (int off = 1; off < LANES; off <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, off));
        return top;
      };
      uint32_t top = group_top();
      if (__any_sync(0xffffffffu, top >= 0x7F800000u)) {
        drop_infinities<EPT>(v[j]);
        top = group_top();
      }
      const uint32_t ex = scale_exponent(top);
      const int64_t k = k0 + j * PER_LOAD;
      if (k < K) {
        store_codes<EPT>(codes + r * ld, k, K, v[j], pow2_inverse(ex));
        if (lane % LANES == 0) scales[r * ld_s + k / kGroup] = pow2_of(ex);
      }
    }
  }
}

template <bool BF16, bool VEC>
__global__ void __launch_bounds__(kThreads)
fp8_quantize_blocks(const void* x, int64_t rows, int64_t K, int64_t ldx, uint8_t* codes, int64_t ld, float* scales, int64_t ld_s) {
  constexpr int WARPS = kThreads / 32, PER_WARP = kGroup / WARPS;      // a warp's 16 rows, four elements per lane and row
  __shared__ uint32_t tops[2][WARPS];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_wait();
  const int64_t G = (K + kGroup - 1) / kGroup, items = (rows + kGroup - 1) / kGroup * G;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t br = it / G, g = it - br * G, r0 = br * kGroup + warp * PER_WARP, k = g * kGroup + lane * 4;
    float v[PER_WARP][4];
#pragma unroll
    for (int i = 0; i < PER_WARP; i++)
      load_run<BF16, 4, VEC>(static_cast<const char*>(x) + (r0 + i) * ldx * (BF16 ? 2 : 4), k, r0 + i < rows ? K : 0, v[i]);
    const auto block_top = [&](int at) {
      float top = 0.0f;
#pragma unroll
      for (int i = 0; i < PER_WARP; i++) top = fmaxf(top, largest<4>(v[i]));
      const uint32_t bits = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
      if (lane == 0) tops[at][warp] = bits;
      __syncthreads();
      uint32_t all = 0;
#pragma unroll
      for (int w = 0; w < WARPS; w++) all = max(all, tops[at][w]);
      return all;
    };
    uint32_t top = block_top(0);
    if (top >= 0x7F800000u) {                           // the same in every thread
#pragma unroll
      for (int i = 0; i < PER_WARP; i++) drop_infinities<4>(v[i]);
      top = block_top(1);
    }
    const uint32_t ex = scale_exponent(top);
#pragma unroll
    for (int i = 0; i < PER_WARP; i++)
      if (r0 + i < rows && k < K) store_codes<4>(codes + (r0 + i) * ld, k, K, v[i], pow2_inverse(ex));
    if (threadIdx.x == 0) scales[br * ld_s + g] = pow2_of(ex);
    __syncthreads();                                    // every thread has read the maxima
  }
}

}  // namespace

cudaError_t launch_fp8_quantize(const void* x, bool x_bf16, int64_t rows, int64_t K, int64_t ldx, uint8_t* codes, int64_t ld, float* scales,
                                int64_t ld_s, bool blocks, cudaStream_t stream) {
  int dev = 0, sms = 0;
  const cudaError_t e = current_device(&dev, &sms);
  if (e != cudaSuccess) return e;
  // whole vectors: 16 bytes, but 8 where a lane takes four bf16 (blocks)
  const int64_t size = x_bf16 ? 2 : 4, vec_bytes = blocks && x_bf16 ? 8 : 16;
  const bool vec = reinterpret_cast<uintptr_t>(x) % vec_bytes == 0 && ldx * size % vec_bytes == 0;
  int64_t ctas;
  if (blocks) {
    ctas = (rows + kGroup - 1) / kGroup * ((K + kGroup - 1) / kGroup);
  } else {
    const int64_t per_warp = x_bf16 ? 1024 : 512, items = rows * ((K + per_warp - 1) / per_warp);
    ctas = (items + kThreads / 32 - 1) / (kThreads / 32);
  }
  const int64_t cap = static_cast<int64_t>(sms) * 64;
  const dim3 grid(static_cast<unsigned>(ctas < cap ? ctas : cap));
#define HBMM_Q(KERNEL, B, V) return launch_pdl(KERNEL<B, V>, grid, dim3(kThreads), 0, stream, x, rows, K, ldx, codes, ld, scales, ld_s)
  if (blocks) {
    if (x_bf16) { if (vec) HBMM_Q(fp8_quantize_blocks, true, true); HBMM_Q(fp8_quantize_blocks, true, false); }
    if (vec) HBMM_Q(fp8_quantize_blocks, false, true);
    HBMM_Q(fp8_quantize_blocks, false, false);
  }
  if (x_bf16) { if (vec) HBMM_Q(fp8_quantize_rows, true, true); HBMM_Q(fp8_quantize_rows, true, false); }
  if (vec) HBMM_Q(fp8_quantize_rows, false, true);
  HBMM_Q(fp8_quantize_rows, false, false);
#undef HBMM_Q
}

}  // namespace hbmm
