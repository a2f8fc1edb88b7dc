// Quantization to e4m3 with a power-of-two scale per 128 row elements, or per block of 128 x 128 elements.
//
//   s = 2^ceil(log2(amax / 448)),  code = rne(x / s)
//
// Streams, HBM bound: 4 or 2 bytes read and 1 written per element.  The scale comes from the exponent field of amax alone, x / s
// is a product with a power of two, so no step but the conversion rounds.
// Rows: a warp takes four loads of 16 bytes per lane, 512 (fp32) or 1024 (bf16) consecutive elements of a row; a load covers one
// group (fp32: the whole warp) or two (bf16: half a warp each), whose maximum is a tree over the raw bits (magnitudes order as their
// bits do).  The next four loads are in flight meanwhile.
// Blocks: one CTA per block keeps its raw elements in registers between the maximum and the conversion.
// Measured: rows, 8192 x 8192 bf16 (203 MB) 38 us, 5.3 TB/s, fp32 (338 MB) 57, 5.9; blocks, 4096 x 9216 fp32 (189 MB) 32, 5.8 TB/s.  Two CTAs of the row
// kernel more per SM with fewer loads each: 41 us and up.
#include <cuda_bf16.h>
#include "fp8_common.cuh"
#include "kernels.h"
#include "pdl.cuh"

namespace hbmm {
namespace {

using namespace fp8;

constexpr int kThreads = 256;

// 16 raw bytes of a row: 4 fp32 or 8 bf16 elements from column k on; columns >= K read as zeros.  VEC: the row starts on 16 bytes.
template <bool BF16, bool VEC>
__device__ __forceinline__ uint4 load_raw(const void* row, int64_t k, int64_t K) {
  constexpr int EPT = BF16 ? 8 : 4;
  const char* p = static_cast<const char*>(row) + k * (BF16 ? 2 : 4);
  if (VEC && k + EPT <= K) return load16(p);
  uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < EPT; e++)
    if (k + e < K) {
      if constexpr (BF16) w[e / 2] |= __float_as_uint(load_elem<__nv_bfloat16>(p + 2 * e)) >> (e % 2 ? 0 : 16);
      else w[e] = __float_as_uint(load_elem<float>(p + 4 * e));
    }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// Largest magnitude of 16 raw bytes, as the bits of an fp32 (magnitudes order as their bits do; what is not finite comes last).
template <bool BF16>
__device__ __forceinline__ uint32_t raw_top(const uint4 v) {
  if constexpr (BF16) {
    constexpr uint32_t kMag = 0x7FFF7FFFu;
    const uint32_t m = __vmaxu2(__vimax3_u16x2(v.x & kMag, v.y & kMag, v.z & kMag), v.w & kMag);
    return max(m << 16, m & 0xFFFF0000u);
  } else {
    constexpr uint32_t kMag = 0x7FFFFFFFu;
    return max(__vimax3_u32(v.x & kMag, v.y & kMag, v.z & kMag), v.w & kMag);
  }
}
// Elements that are not finite become NaN and leave the maximum (rare: a maximum shows whether there are any).
template <bool BF16>
__device__ __noinline__ uint4 raw_without(const uint4 v) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; i++) {
    if constexpr (BF16) {
      if ((w[i] & 0x7F80u) == 0x7F80u) w[i] = (w[i] & 0xFFFF0000u) | 0x7FFFu;
      if ((w[i] & 0x7F800000u) == 0x7F800000u) w[i] = (w[i] & 0xFFFFu) | 0x7FFF0000u;
    } else if ((w[i] & 0x7F800000u) == 0x7F800000u) {
      w[i] = 0x7FFFFFFFu;
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <bool BF16>
__device__ __noinline__ uint32_t finite_top(const uint4 v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const uint32_t a = (BF16 ? w[i] << 16 : w[i]) & 0x7FFFFFFFu, b = BF16 ? w[i] & 0x7FFF0000u : 0u;
    if (a < 0x7F800000u) top = max(top, a);
    if (b < 0x7F800000u) top = max(top, b);
  }
  return top;
}
// The codes of 16 raw bytes to their row (which starts on 16 bytes; k a multiple of the elements).
template <bool BF16>
__device__ __forceinline__ void store_codes(uint8_t* row, int64_t k, int64_t K, const uint4 v, float inverse) {
  constexpr int EPT = BF16 ? 8 : 4;
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t c[EPT / 4];
#pragma unroll
  for (int i = 0; i < EPT / 4; i++) {
    if constexpr (BF16)
      c[i] = to_e4m3x4(scaled(__uint_as_float(w[2 * i] << 16), inverse), scaled(__uint_as_float(w[2 * i] & 0xFFFF0000u), inverse),
                       scaled(__uint_as_float(w[2 * i + 1] << 16), inverse), scaled(__uint_as_float(w[2 * i + 1] & 0xFFFF0000u), inverse));
    else
      c[i] = to_e4m3x4(scaled(__uint_as_float(w[0]), inverse), scaled(__uint_as_float(w[1]), inverse), scaled(__uint_as_float(w[2]), inverse),
                       scaled(__uint_as_float(w[3]), inverse));
  }
  if (k + EPT <= K) {
    if constexpr (BF16) *reinterpret_cast<uint2*>(row + k) = make_uint2(c[0], c[1]);
    else *reinterpret_cast<uint32_t*>(row + k) = c[0];
  } else {
#pragma unroll
    for (int e = 0; e < EPT; e++)
      if (k + e < K) row[k + e] = static_cast<uint8_t>(c[e / 4] >> (8 * (e % 4)));
  }
}

constexpr int kLoads = 4;             // of 16 bytes per lane and turn
constexpr int kResident = 4;          // CTAs per SM of the row kernel's walk

template <bool BF16, bool VEC>
__global__ void __launch_bounds__(kThreads, kResident)
fp8_quantize_rows(const void* x, int64_t rows, int64_t K, int64_t ldx, uint8_t* codes, int64_t ld, float* scales, int64_t ld_s) {
  constexpr int EPT = BF16 ? 8 : 4, LANES = kGroup / EPT, PER_LOAD = 32 * EPT;
  pdl_wait();
  const int lane = threadIdx.x & 31;
  const int64_t chunks = (K + kLoads * PER_LOAD - 1) / (kLoads * PER_LOAD);
  RowWalk ahead((static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) >> 5, static_cast<int64_t>(gridDim.x) * (kThreads / 32), chunks);   // of a warp
  uint4 next[kLoads];
  const auto fetch = [&](uint4 (&v)[kLoads]) {
    const int64_t k0 = ahead.chunk * (kLoads * PER_LOAD) + lane * EPT;
    const char* row = static_cast<const char*>(x) + ahead.row * ldx * (BF16 ? 2 : 4);
#pragma unroll
    for (int j = 0; j < kLoads; j++) v[j] = load_raw<BF16, VEC>(row, k0 + j * PER_LOAD, K);
  };
  const auto over_group = [&](uint32_t top) {
    if constexpr (LANES == 32) {
      return __reduce_max_sync(0xffffffffu, top);
    } else {
#pragma unroll
      for (int off = 1; off < LANES; off <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, off));
      return top;
    }
  };
  if (ahead.row < rows) fetch(next);
  while (ahead.row < rows) {
    uint4 v[kLoads];
    const int64_t r = ahead.row, k0 = ahead.chunk * (kLoads * PER_LOAD) + lane * EPT;
#pragma unroll
    for (int j = 0; j < kLoads; j++) v[j] = next[j];
    ahead.next();
    if (ahead.row < rows) fetch(next);                  // in flight while this one is worked on
#pragma unroll
    for (int j = 0; j < kLoads; j++) {
      uint32_t top = over_group(raw_top<BF16>(v[j]));
      if (__any_sync(0xffffffffu, top >= 0x7F800000u)) {
        top = over_group(finite_top<BF16>(v[j]));
        v[j] = raw_without<BF16>(v[j]);
      }
      const uint32_t ex = scale_exponent(top);
      const int64_t k = k0 + j * PER_LOAD;
      if (k < K) {
        store_codes<BF16>(codes + r * ld, k, K, v[j], pow2_inverse(ex));
        if (lane % LANES == 0) scales[r * ld_s + k / kGroup] = pow2_of(ex);
      }
    }
  }
}

template <bool BF16, bool VEC>
__global__ void __launch_bounds__(kThreads, BF16 ? 4 : 3)
fp8_quantize_blocks(const void* x, int64_t rows, int64_t K, int64_t ldx, uint8_t* codes, int64_t ld, float* scales, int64_t ld_s) {
  // a load covers one row of the block (fp32) or two (bf16); the CTA's eight warps take its rows in turn
  constexpr int EPT = BF16 ? 8 : 4, LANES = kGroup / EPT, ROWS = 32 / LANES, WARPS = kThreads / 32, LOADS = kGroup / WARPS / ROWS;
  __shared__ uint32_t tops[2][WARPS];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_wait();
  const int64_t G = (K + kGroup - 1) / kGroup, items = (rows + kGroup - 1) / kGroup * G;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t br = it / G, g = it - br * G, r0 = br * kGroup + warp * ROWS + lane / LANES, k = g * kGroup + lane % LANES * EPT;
    const char* from = static_cast<const char*>(x) + r0 * ldx * (BF16 ? 2 : 4);
    uint4 v[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; i++)
      v[i] = load_raw<BF16, VEC>(from + i * (WARPS * ROWS * ldx * (BF16 ? 2 : 4)), k, r0 + i * WARPS * ROWS < rows ? K : 0);
    const auto over_block = [&](int at, uint32_t top) {
      top = __reduce_max_sync(0xffffffffu, top);
      if (lane == 0) tops[at][warp] = top;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < WARPS; w++) top = max(top, tops[at][w]);
      return top;
    };
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < LOADS; i++) top = max(top, raw_top<BF16>(v[i]));
    top = over_block(0, top);
    if (top >= 0x7F800000u) {                           // the same in every thread
      top = 0;
#pragma unroll
      for (int i = 0; i < LOADS; i++) {
        top = max(top, finite_top<BF16>(v[i]));
        v[i] = raw_without<BF16>(v[i]);
      }
      top = over_block(1, top);
    }
    const uint32_t ex = scale_exponent(top);
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      const int64_t r = r0 + i * WARPS * ROWS;
      if (r < rows && k < K) store_codes<BF16>(codes + r * ld, k, K, v[i], pow2_inverse(ex));
    }
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
  const bool vec = reinterpret_cast<uintptr_t>(x) % 16 == 0 && ldx * (x_bf16 ? 2 : 4) % 16 == 0;
  int64_t ctas;
  if (blocks) {
    ctas = (rows + kGroup - 1) / kGroup * ((K + kGroup - 1) / kGroup);
  } else {
    const int64_t per_warp = x_bf16 ? 1024 : 512, items = rows * ((K + per_warp - 1) / per_warp);
    ctas = (items + kThreads / 32 - 1) / (kThreads / 32);
  }
  const int64_t cap = static_cast<int64_t>(sms) * (blocks ? 64 : kResident);      // rows: all at once, a warp reads ahead along its walk
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
