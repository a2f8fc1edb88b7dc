// C-ABI layer of the 8-bit operands: argument validation on the host, then dispatch (see include/hbmm.h for the contract).
#include <cstddef>
#include <cstdint>
#include "../../include/hbmm.h"
#include "kernels.h"

using namespace hbmm;

namespace {

constexpr int64_t kGroup = 128;
constexpr int64_t kMaxExtent = int64_t{1} << 31;        // rows and columns are tensor-copy coordinates
constexpr int64_t kMaxPitch = int64_t{1} << 40;         // bytes between rows that a tensor map can hold; every matrix's here

inline bool on16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline int64_t up(int64_t v, int64_t a) { return (v + a - 1) / a * a; }
inline int64_t groups(int64_t n) { return (n + kGroup - 1) / kGroup; }
inline bool valid_dtype(int32_t d) { return d == HBMM_F32 || d == HBMM_BF16; }

hbmm_status check_operand(const hbmm_fp8_operand* op, int32_t block_rows = 0) {
  if (!op || op->rows <= 0 || op->K <= 0) return HBMM_ERR_INVALID_ARG;
  if (op->block_rows != 1 && op->block_rows != kGroup) return HBMM_ERR_UNSUPPORTED;
  if (block_rows != 0 && op->block_rows != block_rows) return HBMM_ERR_UNSUPPORTED;
  if (op->rows >= kMaxExtent || op->K >= kMaxExtent || op->ld_codes >= kMaxPitch || op->ld_scales >= kMaxPitch) return HBMM_ERR_UNSUPPORTED;
  if (!op->codes || !op->scales || op->ld_codes < op->K || op->ld_scales < groups(op->K)) return HBMM_ERR_INVALID_ARG;
  if (!on16(op->codes) || !on16(op->scales) || op->ld_codes % 16 != 0 || op->ld_scales % 4 != 0) return HBMM_ERR_ALIGNMENT;
  return HBMM_OK;
}

Fp8View view_of(const hbmm_fp8_operand* op) { return {op->codes, op->scales, op->rows, op->K, op->ld_codes, op->ld_scales}; }

// A matrix whose rows start on 16-byte boundaries, or wherever its elements may.
hbmm_status check_rows(const void* p, int64_t cols, int64_t ld, int64_t size, bool rows16 = true) {
  if (!p || ld < cols) return HBMM_ERR_INVALID_ARG;
  if (ld >= kMaxPitch / size) return HBMM_ERR_UNSUPPORTED;
  if (!rows16) return reinterpret_cast<uintptr_t>(p) % size == 0 ? HBMM_OK : HBMM_ERR_ALIGNMENT;
  return on16(p) && ld * size % 16 == 0 ? HBMM_OK : HBMM_ERR_ALIGNMENT;
}
inline int64_t size_of(int32_t dtype) { return dtype == HBMM_BF16 ? 2 : 4; }
inline hbmm_status status_of(cudaError_t e) { return e == cudaSuccess ? HBMM_OK : HBMM_ERR_CUDA; }

}  // namespace

extern "C" {

hbmm_status hbmm_fp8_operand_bytes(int64_t rows, int64_t K, int32_t block_rows, size_t* codes_bytes, size_t* scales_bytes,
                                   int64_t* ld_codes, int64_t* ld_scales) {
  if (rows <= 0 || K <= 0) return HBMM_ERR_INVALID_ARG;
  if ((block_rows != 1 && block_rows != kGroup) || rows >= kMaxExtent || K >= kMaxExtent) return HBMM_ERR_UNSUPPORTED;
  const int64_t lc = up(K, 16), ls = up(groups(K), 4);
  if (codes_bytes) *codes_bytes = static_cast<size_t>(rows * lc);
  if (scales_bytes) *scales_bytes = static_cast<size_t>((rows + block_rows - 1) / block_rows * ls * 4);
  if (ld_codes) *ld_codes = lc;
  if (ld_scales) *ld_scales = ls;
  return HBMM_OK;
}

hbmm_status hbmm_fp8_quantize(const void* x, int32_t x_dtype, int64_t rows, int64_t K, int64_t ldx, const hbmm_fp8_operand* out,
                              void* stream) {
  hbmm_status st = check_operand(out);
  if (st != HBMM_OK) return st;
  if (!valid_dtype(x_dtype) || rows != out->rows || K != out->K) return HBMM_ERR_INVALID_ARG;
  if ((st = check_rows(x, K, ldx, size_of(x_dtype), false)) != HBMM_OK) return st;
  return status_of(launch_fp8_quantize(x, x_dtype == HBMM_BF16, rows, K, ldx, out->codes, out->ld_codes, out->scales, out->ld_scales,
                                       out->block_rows != 1, static_cast<cudaStream_t>(stream)));
}

hbmm_status hbmm_fp8_gemm(const hbmm_fp8_operand* A, const hbmm_fp8_operand* W, void* C, int32_t c_dtype, int64_t ldc, void* stream) {
  hbmm_status st = check_operand(A, 1);
  if (st == HBMM_OK) st = check_operand(W, kGroup);
  if (st != HBMM_OK) return st;
  if (A->K != W->K || !valid_dtype(c_dtype)) return HBMM_ERR_INVALID_ARG;
  if ((st = check_rows(C, W->rows, ldc, size_of(c_dtype))) != HBMM_OK) return st;
  if (fp8_gemv_supported(view_of(A)))
    return status_of(launch_fp8_gemv(view_of(A), view_of(W), C, c_dtype == HBMM_BF16, ldc, static_cast<cudaStream_t>(stream)));
  return status_of(launch_fp8_gemm(view_of(A), view_of(W), false, C, c_dtype == HBMM_BF16, ldc, static_cast<cudaStream_t>(stream)));
}

hbmm_status hbmm_fp8_input_grad(const hbmm_fp8_operand* GY, const hbmm_fp8_operand* W, void* GX, int32_t gx_dtype, int64_t ldgx,
                                void* stream) {
  hbmm_status st = check_operand(GY, 1);
  if (st == HBMM_OK) st = check_operand(W, kGroup);
  if (st != HBMM_OK) return st;
  if (GY->K != W->rows || !valid_dtype(gx_dtype)) return HBMM_ERR_INVALID_ARG;
  if ((st = check_rows(GX, W->K, ldgx, size_of(gx_dtype))) != HBMM_OK) return st;
  return status_of(launch_fp8_gemm(view_of(GY), view_of(W), true, GX, gx_dtype == HBMM_BF16, ldgx, static_cast<cudaStream_t>(stream)));
}

hbmm_status hbmm_fp8_weight_grad(const void* gy, int32_t gy_dtype, int64_t N, int64_t ldg, const hbmm_fp8_operand* X, const float* base,
                                 int64_t ld_base, float* GW, int64_t ldw, void* stream) {
  hbmm_status st = check_operand(X, 1);
  if (st != HBMM_OK) return st;
  if (N <= 0 || !valid_dtype(gy_dtype)) return HBMM_ERR_INVALID_ARG;
  if (gy_dtype != HBMM_BF16 || N >= kMaxExtent) return HBMM_ERR_UNSUPPORTED;
  if ((st = check_rows(gy, N, ldg, 2)) != HBMM_OK) return st;
  if ((st = check_rows(GW, X->K, ldw, 4)) != HBMM_OK) return st;
  if (base && (st = check_rows(base, X->K, ld_base, 4)) != HBMM_OK) return st;
  if (base == GW && ld_base != ldw && N > 1) return HBMM_ERR_INVALID_ARG;
  return status_of(launch_fp8_weight_grad(gy, N, ldg, view_of(X), base, ld_base, GW, ldw, static_cast<cudaStream_t>(stream)));
}

hbmm_status hbmm_fp8_binarize_backward(const hbmm_fp8_operand* X, const void* gy, int32_t dtype, int64_t ldg, int32_t beta, void* gx,
                                       int64_t ldo, void* stream) {
  hbmm_status st = check_operand(X, 1);
  if (st != HBMM_OK) return st;
  if (beta < 1 || !valid_dtype(dtype)) return HBMM_ERR_INVALID_ARG;
  if ((st = check_rows(gy, X->K, ldg, size_of(dtype), false)) != HBMM_OK) return st;
  if ((st = check_rows(gx, X->K, ldo, size_of(dtype), false)) != HBMM_OK) return st;
  return status_of(launch_fp8_binarize_backward(view_of(X), gy, dtype == HBMM_BF16, ldg, beta, gx, ldo, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
