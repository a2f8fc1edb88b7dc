// Gradient through the Hadamard binarization (Eq. 6, straight-through estimator of Eq. 5) from an 8-bit copy of x:
//   gx[i] = (1/n_g) s_i sum_{j in group(i)} gy[j] s_j  +  delta_g gy[i] [|x^_i| <= 1],
// x^ = code * scale (exact in fp32 for the quantizer's scales), s the code's sign bit, delta_g the mean |x^| of the group.  Only |x^|
// enters besides s, so a scale's sign leaves with the bit that holds it.
// A stream: 1 + 4 + 4 bytes per element (1 + 2 + 2 in bf16) where the fp32 form of backward.cu moves 12.
//
// Groups of a power of two up to 128 elements: the 128 elements that share a scale belong to 32 lanes of four (fp32) or 16 lanes
// of eight (bf16): 16-byte gradients either way; group sums are shuffle trees inside them.
// Other groups: four lanes, a warp, or (more than 1024 elements) a CTA per group, two walks over the group with one element per load.
// Measured: 8192 x 8192, groups of 32, bf16 (338 MB) 68 us, 5.0 TB/s; with five or six CTAs per SM 76 and 98; fp32 (606 MB) 119, 5.1.
// The other groups are bound by their small loads, not by memory: bf16, a group per row 210 us (1.6 TB/s), groups of 256 235, of 48
// 526, of 3 697; fp32 212 and 522 for a group per row and of 48.
#include <cuda_bf16.h>
#include "fp8_common.cuh"
#include "kernels.h"
#include "pdl.cuh"

namespace hbmm {
namespace {

using namespace fp8;

constexpr int kThreads = 256;
constexpr int kResident = 4;          // CTAs per SM of the walk below (64 registers a thread)

struct BackArgs {
  const uint8_t* codes; const float* scales;
  int64_t rows, K, ld, ld_s;
  const void* gy; int64_t ldg;
  void* gx; int64_t ldo;
};

__device__ __forceinline__ float with_sign(float v, uint32_t code) { return __uint_as_float(__float_as_uint(v) ^ ((code & 0x80u) << 24)); }
template <typename T> __device__ __forceinline__ T rounded(float v);
template <> __device__ __forceinline__ float rounded<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 rounded<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Elements per lane.
template <typename T> struct Per { static constexpr int N = 16 / sizeof(T); };

// What a lane reads of a run: codes, gradients (raw), the run's scale.
template <int E> struct Item { uint32_t c[E / 4]; uint4 g; float scale; };

// The largest magnitude of a code whose product with the scale's is at most 1 in fp32: [|x^| <= 1] is one comparison of the code's own
// value.  A power of two: its inverse.
__device__ __forceinline__ float clip_limit(float scale) {
  const uint32_t bits = __float_as_uint(scale);
  if ((bits & 0x807FFFFFu) == 0 && bits - 0x00800000u < 0x7E000000u) return __uint_as_float((254u << 23) - bits);
  scale = fabsf(scale);
  const uint32_t code = to_e4m3x2(1.0f / scale, 0.0f) & 0x7Fu;        // nearest; the one below where that is too large
  const float v = from_e4m3x2(code).x;
  return v * scale > 1.0f && code != 0 ? from_e4m3x2(code - 1).x : v;
}

template <typename T, int BETA, bool VEC>
__global__ void __launch_bounds__(kThreads)
fp8_binarize_backward_rows(const BackArgs a) {
  constexpr int E = Per<T>::N, RUN = 32 * E;                         // a warp's run: one scale group (fp32) or two (bf16)
  constexpr int IN = BETA < E ? BETA : E, LANES = BETA > E ? BETA / E : 1;
  constexpr bool BF16 = E == 8;
  pdl_wait();
  const int lane = threadIdx.x & 31;
  RowWalk ahead((static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) >> 5, static_cast<int64_t>(gridDim.x) * (kThreads / 32),
                (a.K + RUN - 1) / RUN);                              // of a warp
  const auto fetch = [&](Item<E>& l) {
    const int64_t r = ahead.row, k = ahead.chunk * RUN + lane * E;
    const T* gy = static_cast<const T*>(a.gy) + r * a.ldg;
    const uint8_t* codes = a.codes + r * a.ld;
    l.scale = k < a.K ? loadf(a.scales + r * a.ld_s + k / kGroup) : 0.0f;
    const bool whole = k + E <= a.K;
    if (whole) {                                                     // codes start on 16 bytes and k is a multiple of E
      if constexpr (BF16) { const uint2 q = load8(codes + k); l.c[0] = q.x; l.c[1] = q.y; }
      else l.c[0] = load4(codes + k);
    } else {
#pragma unroll
      for (int e = 0; e < E / 4; e++) l.c[e] = 0;
#pragma unroll
      for (int e = 0; e < E; e++)
        if (k + e < a.K) l.c[e / 4] |= load1(codes + k + e) << (8 * (e % 4));
    }
    if (VEC && whole) {
      l.g = load16(gy + k);
    } else {
      uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
      for (int e = 0; e < E; e++)
        if (k + e < a.K) {
          const uint32_t v = __float_as_uint(load_elem<T>(gy + k + e));
          if constexpr (BF16) w[e / 2] |= e % 2 ? v : v >> 16;
          else w[e] = v;
        }
      l.g = make_uint4(w[0], w[1], w[2], w[3]);
    }
  };
  Item<E> next;
  if (ahead.row < a.rows) fetch(next);
  while (ahead.row < a.rows) {
    const Item<E> l = next;
    const int64_t r = ahead.row, k0 = ahead.chunk * RUN, k = k0 + lane * E;
    ahead.next();
    if (ahead.row < a.rows) fetch(next);                             // in flight while this one is worked on
    const uint32_t gw[4] = {l.g.x, l.g.y, l.g.z, l.g.w};
    float mag[E], back[E];                                           // the code's magnitude (without its scale) and gy s
    uint32_t sign[4];                                                // the signs where gw's are
#pragma unroll
    for (int e = 0; e < E; e += 2) {
      const float2 f = from_e4m3x2((l.c[e / 4] & 0x7F7F7F7Fu) >> (8 * (e % 4)) & 0xFFFFu);
      mag[e] = f.x; mag[e + 1] = f.y;
    }
#pragma unroll
    for (int i = 0; i < 4; i++) {
      if constexpr (BF16) {
        sign[i] = __byte_perm(l.c[i / 2], 0u, i % 2 ? 0x3424 : 0x1404) & 0x80008000u;
        const uint32_t w = gw[i] ^ sign[i];
        back[2 * i] = __uint_as_float(w << 16);
        back[2 * i + 1] = __uint_as_float(w & 0xFFFF0000u);
      } else {
        sign[i] = l.c[0] << (24 - 8 * i) & 0x80000000u;
        back[i] = __uint_as_float(gw[i] ^ sign[i]);
      }
    }
    const float limit = clip_limit(l.scale);
    const bool inside = k0 + RUN <= a.K;                             // warp-uniform: every group of the run is whole or ends with it
    float o[E];
#pragma unroll
    for (int q = 0; q < E; q += IN) {                                // the groups of this lane
      float m[IN], b[IN];
#pragma unroll
      for (int e = 0; e < IN; e++) { m[e] = mag[q + e]; b[e] = back[q + e]; }
#pragma unroll
      for (int w = 1; w < IN; w <<= 1)
#pragma unroll
        for (int e = 0; e < IN; e += 2 * w) { m[e] += m[e + w]; b[e] += b[e + w]; }
      float sm = m[0], sb = b[0];
#pragma unroll
      for (int off = 1; off < LANES; off <<= 1) {
        sm += __shfl_xor_sync(0xffffffffu, sm, off);
        sb += __shfl_xor_sync(0xffffffffu, sb, off);
      }
      float dm, db;
      sm *= fabsf(l.scale);                                          // one scale: a group lies in one run of 128
      if (inside) {
        dm = sm * (1.0f / BETA); db = sb * (1.0f / BETA);
      } else {
        const int64_t left = a.K - (k + q) / BETA * BETA;            // elements from the group's start on
        const float n = static_cast<float>(left >= BETA ? BETA : left > 0 ? left : 1);
        dm = sm / n; db = sb / n;
      }
      // s db + delta gy = s (db + delta gy s)
#pragma unroll
      for (int e = q; e < q + IN; e++) o[e] = db + (mag[e] <= limit ? dm * back[e] : 0.0f);
    }
    T* gx = static_cast<T*>(a.gx) + r * a.ldo;
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; i++) w[i] = (BF16 ? bf16x2(o[2 * i % E], o[(2 * i + 1) % E]) : __float_as_uint(o[i])) ^ sign[i];
    if (VEC && k + E <= a.K) {
      *reinterpret_cast<uint4*>(gx + k) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int e = 0; e < E; e++)
        if (k + e < a.K) {
          if constexpr (BF16) reinterpret_cast<unsigned short*>(gx)[k + e] = static_cast<unsigned short>(w[e / 2] >> (16 * (e % 2)));
          else reinterpret_cast<uint32_t*>(gx)[k + e] = w[e];
        }
    }
  }
}

__device__ __forceinline__ float magnitude(uint32_t code, float scale) { return from_e4m3x2(code & 0x7Fu).x * fabsf(scale); }

// A team of TEAM threads (at most a warp, or the whole CTA) per (row, group), any group length.
template <typename T, int TEAM>
__global__ void __launch_bounds__(kThreads)
fp8_binarize_backward_teams(const BackArgs a, int64_t beta) {
  constexpr int WARPS = kThreads / 32;
  __shared__ float part[2][WARPS];
  pdl_wait();
  const int64_t G = (a.K + beta - 1) / beta, items = a.rows * G;
  const int me = threadIdx.x % TEAM;
  constexpr int TEAMS = kThreads / TEAM;
  const int64_t step = static_cast<int64_t>(gridDim.x) * TEAMS;
  // whole CTAs walk together (the shuffles need every lane, the barriers every warp): the bound is rounded up
  for (int64_t first = static_cast<int64_t>(blockIdx.x) * TEAMS; first < items; first += step) {
    const int64_t it = first + threadIdx.x / TEAM;
    const bool live = it < items;
    const int64_t r = live ? it / G : 0, k0 = live ? (it - r * G) * beta : 0;
    const int64_t k1 = live ? (k0 + beta < a.K ? k0 + beta : a.K) : 0;
    const T* gy = static_cast<const T*>(a.gy) + r * a.ldg;
    T* gx = static_cast<T*>(a.gx) + r * a.ldo;
    const uint8_t* codes = a.codes + r * a.ld;
    const float* scales = a.scales + r * a.ld_s;
    float sm = 0.0f, sb = 0.0f;
    for (int64_t k = k0 + me; k < k1; k += TEAM) {
      const uint32_t c = load1(codes + k);
      sm += magnitude(c, loadf(scales + k / kGroup));
      sb += with_sign(load_elem<T>(gy + k), c);
    }
#pragma unroll
    for (int off = 1; off < (TEAM < 32 ? TEAM : 32); off <<= 1) {
      sm += __shfl_xor_sync(0xffffffffu, sm, off);
      sb += __shfl_xor_sync(0xffffffffu, sb, off);
    }
    if constexpr (TEAM > 32) {
      __syncthreads();                                               // the group before has been read
      if (threadIdx.x % 32 == 0) { part[0][threadIdx.x / 32] = sm; part[1][threadIdx.x / 32] = sb; }
      __syncthreads();
      sm = sb = 0.0f;
#pragma unroll
      for (int w = 0; w < WARPS; w++) { sm += part[0][w]; sb += part[1][w]; }
    }
    const float n = static_cast<float>(k1 > k0 ? k1 - k0 : 1), dm = sm / n, db = sb / n;
    for (int64_t k = k0 + me; k < k1; k += TEAM) {
      const uint32_t c = load1(codes + k);
      const float ste = magnitude(c, loadf(scales + k / kGroup)) <= 1.0f ? dm * load_elem<T>(gy + k) : 0.0f;
      gx[k] = rounded<T>(with_sign(db, c) + ste);
    }
  }
}

template <typename T>
cudaError_t launch(const BackArgs& a, int64_t beta, int sms, cudaStream_t stream) {
  const auto grid = [&](int64_t work, int64_t per, int ctas = 32) {
    const int64_t n = (work + per - 1) / per, cap = static_cast<int64_t>(sms) * ctas;
    return dim3(static_cast<unsigned>(n < cap ? n : cap));
  };
  // group sizes a warp takes by shuffles (a row shorter than its group has a last group of its own length like any other)
  if ((beta & (beta - 1)) == 0 && beta <= 128) {
    const int64_t run = 32 * Per<T>::N;
    const dim3 g = grid(a.rows * ((a.K + run - 1) / run), kThreads / 32, kResident);     // all at once: a warp reads ahead along its walk
    const bool vec = reinterpret_cast<uintptr_t>(a.gy) % 16 == 0 && reinterpret_cast<uintptr_t>(a.gx) % 16 == 0 &&
                     a.ldg * static_cast<int64_t>(sizeof(T)) % 16 == 0 && a.ldo * static_cast<int64_t>(sizeof(T)) % 16 == 0;
#define HBMM_B(B)                                                                                                                   \
  case B:                                                                                                                           \
    return vec ? launch_pdl(fp8_binarize_backward_rows<T, B, true>, g, dim3(kThreads), 0, stream, a)                                 \
               : launch_pdl(fp8_binarize_backward_rows<T, B, false>, g, dim3(kThreads), 0, stream, a);
    switch (beta) { HBMM_B(1) HBMM_B(2) HBMM_B(4) HBMM_B(8) HBMM_B(16) HBMM_B(32) HBMM_B(64) HBMM_B(128) }
#undef HBMM_B
  }
  if (beta > a.K) beta = a.K;
  const int64_t items = a.rows * ((a.K + beta - 1) / beta);
  if (beta > 1024) return launch_pdl(fp8_binarize_backward_teams<T, kThreads>, grid(items, 1), dim3(kThreads), 0, stream, a, beta);
  if (beta > 16) return launch_pdl(fp8_binarize_backward_teams<T, 32>, grid(items, kThreads / 32), dim3(kThreads), 0, stream, a, beta);
  return launch_pdl(fp8_binarize_backward_teams<T, 4>, grid(items, kThreads / 4), dim3(kThreads), 0, stream, a, beta);
}

}  // namespace

cudaError_t launch_fp8_binarize_backward(const Fp8View& X, const void* gy, bool bf16, int64_t ldg, int64_t beta, void* gx, int64_t ldo,
                                         cudaStream_t stream) {
  int dev = 0, sms = 0;
  const cudaError_t e = current_device(&dev, &sms);
  if (e != cudaSuccess) return e;
  const BackArgs a{X.codes, X.scales, X.rows, X.K, X.ld, X.ld_s, gy, ldg, gx, ldo};
  return bf16 ? launch<__nv_bfloat16>(a, beta, sms, stream) : launch<float>(a, beta, sms, stream);
}

}  // namespace hbmm
