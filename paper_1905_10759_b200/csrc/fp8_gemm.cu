// Products of 8-bit operands on the 5th-generation tensor cores (tcgen05 / TMEM): C = A^ W^^T and C = A^ W^.
//
//   C[m,n] = sum_g (sA[m,g] sW[n/128,g]) D_g[m,n],   D_g[m,n] = sum_{k in group g} A[m,k] W[n,k]
//
// A pair of CTAs forms D_g of a 256 x 256 tile with four 256 x 256 x 32 MMAs (kind::f8f6f4, cta_group::2) into one of two
// accumulators in tensor memory; eight epilogue warps per CTA add it, times the two scales, to fp32 registers (128 columns of one
// row per thread: both scales are one number per thread and group, so the scaling is one fma per output, two per instruction),
// while the tensor cores fill the other accumulator.  512 clk of MMA against 256 of fma and 256 of tensor-memory reads per group.
// The scales are fp32 numbers of any value: they are applied to fp32 sums, no power of two is assumed.
//
// C = A^ W^ (the input gradient; the contraction runs along the rows of W) reads the same W: its tiles arrive as 128 rows of the
// contraction x 128 columns and enter the MMA as an MN-major operand.  Nothing is transposed in memory.
//
// Per CTA and group 16 KB of A (its own 128 rows) and 16 KB of W (its half of the 256 columns) arrive by tensor copies (128-byte
// swizzle, zeros outside the matrices, so no edge needs a case of its own); six stages in flight.
//   warps 0-7 : epilogue (TMEM lanes 32 * (w % 4).., columns 128 * (w / 4)..)
//   warp  8   : one thread issues this CTA's copies;  warp 9 : TMEM allocation, and in the first CTA the MMA-issuing thread (10, 11 hand over registers)
// Products of few tiles: a cluster of two or four pairs shares each tile in equal parts of K (fp8_tile.cuh).
#include <cuda_bf16.h>
#include "fp8_tile.cuh"
#include "kernels.h"
#include "pdl.cuh"
#include "tensor_map.h"

namespace hbmm {
namespace {

using namespace fp8;

constexpr int TN = 256, COLS = TN / 2;         // columns of a pair's tile; of an epilogue warp
constexpr int kThreads = 12 * 32, kLoaderWarp = 8, kMmaWarp = 9, kEpilogueWarps = 8;
constexpr int kRegsEpilogue = 208, kRegsOthers = 80;     // 256 x 208 + 128 x 80 of the 384 x 168 registers at launch
constexpr int kTile = 128 * 128;               // bytes of an operand's part of a stage
constexpr int STAGE = 2 * kTile, STAGES = 6;
constexpr int OFF_A = 0, OFF_B = STAGES * kTile, OFF_OUT = STAGES * STAGE, OFF_BAR = OFF_OUT + kEpilogueWarps * 4096;
constexpr int kBytes = OFF_BAR + (2 * STAGES + 5) * 8 + 16;
constexpr int kMostParts = 4;                  // pairs that share a tile
static_assert(kBytes <= 227 * 1024 && TM * TN * 4 <= STAGES * STAGE, "shared memory");

struct Args {
  const float* a_s; int64_t ld_as;
  const float* w_s; int64_t w_step_n, w_step_g;        // scale of (column block, group): w_s[block * w_step_n + group * w_step_g]
  Out out;
  int32_t groups;                              // of the contraction
  int32_t parts;                               // pairs (of one cluster) that share a tile
};

template <bool TRANS>
__global__ void __launch_bounds__(kThreads, 1)
fp8_gemm_kernel(const Args g, const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap w_map) {
  extern __shared__ __align__(1024) unsigned char smem[];
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + OFF_BAR);
  uint64_t* empty = full + STAGES;
  uint64_t* tfull = empty + STAGES;
  uint64_t* tempty = tfull + 2;
  uint64_t* drained = tempty + 2;
  uint32_t* tmem_base_ptr = reinterpret_cast<uint32_t*>(drained + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_base_ptr + 1);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_ctarank(), lead = rank & ~1u, half = rank & 1u;      // the pair's first CTA; this CTA's rows of the tile
  const int64_t tiles_m = (g.out.M + 2 * TM - 1) / (2 * TM), tiles_n = (g.out.N + TN - 1) / TN, n_tiles = tiles_m * tiles_n;
  const int part = static_cast<int>(rank >> 1);
  // the pair's walk: tiles of its own, or one tile's groups [g0, g1) of `parts`
  const int64_t walker = blockIdx.x / (2 * g.parts), walkers = gridDim.x / (2 * g.parts);
  const int g0 = static_cast<int>(static_cast<int64_t>(part) * g.groups / g.parts), g1 = static_cast<int>(static_cast<int64_t>(part + 1) * g.groups / g.parts);

  pdl_launch_dependents();
  if (tid == 0) {
    for (int s = 0; s < STAGES; s++) {
      mbar_init(&full[s], 1);           // first CTA: its loader's expect_tx arrival; the copies of both CTAs complete the bytes
      mbar_init(&empty[s], 1);          // MMA commit (to both CTAs)
    }
    for (int b = 0; b < 2; b++) { mbar_init(&tfull[b], 1); mbar_init(&tempty[b], 2 * kEpilogueWarps); }
    mbar_init(drained, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    tmem_alloc_pair(tmem_base_ptr, 512);
    tmem_relinquish_pair();
  }
  pdl_wait();
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();                  // every CTA's barriers exist before another signals them
  tc_fence_after();
  const uint32_t tmem_base = *tmem_base_ptr;

  if (warp >= kEpilogueWarps) reg_dec<kRegsOthers>();
  if (warp == kLoaderWarp) {
    // =========================== loader (both CTAs) ===========================
    if (elect_one()) {
      asm volatile("prefetch.tensormap [%0];" ::"l"(&a_map) : "memory");
      asm volatile("prefetch.tensormap [%0];" ::"l"(&w_map) : "memory");
      const uint32_t full0 = mapa_rank(smem_u32(full), lead);
      int s = 0;
      uint32_t round = 0;
      int64_t issued = 0;
      bool ok = true;
      for (int64_t tile = walker; tile < n_tiles && ok; tile += walkers) {
        int64_t tm, tn;
        tile_at(tile, tiles_m, tiles_n, &tm, &tn);
        const int32_t a_row = static_cast<int32_t>(tm * 2 * TM + half * TM), w_at = static_cast<int32_t>(tn * TN + half * (TN / 2));
        for (int kb = g0; kb < g1; kb++) {
          if (round > 0 && !mbar_wait(&empty[s], (round & 1) ^ 1, abort_flag, 1)) { ok = false; break; }
          if (half == 0) mbar_arrive_expect_tx(&full[s], 2 * STAGE);
          const uint32_t bar = full0 + s * 8;
          tma_load_2d_pair(smem + OFF_A + s * kTile, &a_map, kb * kGroup, a_row, bar);
          if (TRANS) tma_load_2d_pair(smem + OFF_B + s * kTile, &w_map, w_at, kb * kGroup, bar);
          else tma_load_2d_pair(smem + OFF_B + s * kTile, &w_map, kb * kGroup, w_at, bar);
          issued++;
          if (++s == STAGES) { s = 0; round++; }
        }
      }
      if (!ok || *abort_flag) {
        // aborted: copies already issued must land before this CTA's shared memory goes away.  The first CTA can watch its
        // barriers; the second cannot see them and gives its copies a fixed time that is far longer than a copy.
        if (half == 0) {
          const int64_t pending = issued < STAGES ? issued : STAGES;
          for (int64_t q = 1; q <= pending; q++) {
            const int64_t idx = issued - q;
            mbar_wait_quiet(&full[idx % STAGES], static_cast<uint32_t>((idx / STAGES) & 1), kDrainPolls);
          }
        } else {
          for (int q = 0; q < 64; q++) __nanosleep(1000);
        }
      }
    }
    __syncwarp();
  } else if (warp == kMmaWarp) {
    // =========================== MMA issuer (first CTA of the pair) ===========================
    if (half == 0 && elect_one()) {
      constexpr uint32_t idesc = instr_desc_pair(TN, kFmtE4M3) | (TRANS ? kTransposeB : 0u);
      // 32 elements of the contraction: 32 bytes along K-major rows, 32 rows of 128 bytes of an MN-major tile
      constexpr uint32_t kStepA = 32 >> 4, kStepB = (TRANS ? 32 * 128 : 32) >> 4;
      const uint16_t both = static_cast<uint16_t>(3u << lead);
      const uint64_t da0 = smem_desc(smem_u32(smem + OFF_A)), db0 = smem_desc(smem_u32(smem + OFF_B));
      const uint64_t da_hi = da0 & 0xFFFFFFFF00000000ull, db_hi = db0 & 0xFFFFFFFF00000000ull;
      const uint32_t da_lo = static_cast<uint32_t>(da0), db_lo = static_cast<uint32_t>(db0);
      const uint32_t full_a = smem_u32(full), empty_a = smem_u32(empty), tfull_a = smem_u32(tfull), tempty_a = smem_u32(tempty);
      uint32_t s = 0, full_par = 0, it = 0;
      bool ok = true;
      for (int64_t tile = walker; tile < n_tiles && ok; tile += walkers) {
        for (int kb = g0; kb < g1; kb++, it++) {
          const uint32_t buf = it & 1;
          if (it >= 2 && !mbar_wait_a(tempty_a + buf * 8, ((it >> 1) & 1) ^ 1, abort_flag, 3)) { ok = false; break; }
          if (!mbar_wait_a(full_a + s * 8, full_par, abort_flag, 2)) { ok = false; break; }
          tc_fence_after();
          const uint32_t a_lo = da_lo + s * (kTile >> 4), b_lo = db_lo + s * (kTile >> 4);
#pragma unroll
          for (uint32_t ks = 0; ks < kGroup / 32; ks++)
            umma_f8_pair(tmem_base + buf * TN, da_hi | (a_lo + ks * kStepA), db_hi | (b_lo + ks * kStepB), idesc, ks != 0 ? 1u : 0u);
          umma_commit_pair_mc(empty_a + s * 8, both);
          umma_commit_pair_mc(tfull_a + buf * 8, both);
          if (++s == STAGES) { s = 0; full_par ^= 1; }
        }
      }
      // every MMA issued so far has retired (in both CTAs) before tensor memory is released -- also after an abort
      umma_commit_pair(smem_u32(drained));
      if (!mbar_wait_quiet(drained, 0, g_spin_limit < kDrainPolls ? kDrainPolls : g_spin_limit)) {
        atomicCAS(&g_error_word, 0, 4);
        *abort_flag = 1;
      }
    }
    __syncwarp();
  } else if (warp < kEpilogueWarps) {
    // =========================== epilogue (both CTAs) ===========================
    reg_inc<kRegsEpilogue>();
    const int row = (warp & 3) * 32 + lane, col0 = (warp >> 2) * COLS;
    const uint32_t tmem_at = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16) + col0;
    const uint32_t tempty0 = mapa_rank(smem_u32(tempty), lead);
    unsigned char* stage = smem + OFF_OUT + warp * 4096;
    constexpr int AHEAD = 4;                     // groups whose scales are loaded at a time, while those before are used
    float na[AHEAD], nw[AHEAD];
    int64_t tm = 0, tn = 0;
    const auto fetch = [&](int64_t tile, int kb) {
      if (tile >= n_tiles) return;
      tile_at(tile, tiles_m, tiles_n, &tm, &tn);
      const int64_t m = tm * 2 * TM + half * TM + row, n = tn * TN + col0;
      const float* ap = g.a_s + m * g.ld_as;
      const float* wp = g.w_s + n / kGroup * g.w_step_n;
#pragma unroll
      for (int j = 0; j < AHEAD; j++) {
        const bool in = kb + j < g1 && m < g.out.M && n < g.out.N;
        na[j] = in ? loadf(ap + kb + j) : 0.0f;
        nw[j] = in ? loadf(wp + (kb + j) * g.w_step_g) : 0.0f;
      }
    };
    uint32_t it = 0;
    bool ok = true;
    fetch(walker, g0);
    for (int64_t tile = walker; tile < n_tiles && ok; tile += walkers) {
      uint64_t acc[COLS / 2];
#pragma unroll
      for (int j = 0; j < COLS / 2; j++) acc[j] = 0ull;
      const int64_t m0 = tm * 2 * TM + half * TM, n0 = tn * TN;
      for (int kb0 = g0; kb0 < g1 && ok; kb0 += AHEAD) {
        float fa[AHEAD], fw[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; j++) { fa[j] = na[j]; fw[j] = nw[j]; }
        if (kb0 + AHEAD < g1) fetch(tile, kb0 + AHEAD);
        else fetch(tile + walkers, g0);
        const int n = g1 - kb0 < AHEAD ? g1 - kb0 : AHEAD;
#pragma unroll 1
        for (int j = 0; j < n; j++, it++) {
          const uint32_t buf = it & 1;
          const float f = j == 0 ? fa[0] * fw[0] : j == 1 ? fa[1] * fw[1] : j == 2 ? fa[2] * fw[2] : fa[3] * fw[3];
          if (!mbar_wait(&tfull[buf], (it >> 1) & 1, abort_flag, 5)) { ok = false; break; }
          tc_fence_after();
          drain<COLS>(tmem_at + buf * TN, acc, f, [&] {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(tempty0 + buf * 8);
          });
        }
      }
      if (!ok) break;
      if (g.parts == 1) store_tile<COLS>(g.out, stage, acc, m0 + (warp & 3) * 32, n0 + col0, lane);
      // every copy of this CTA's only tile has been read: its partial sums take the stages' place
      else stage_part<TN, COLS>(smem, acc, row, col0);
    }
  }

  if (g.parts > 1) {
    __syncwarp();
    cluster_sync_all();
    if (warp < kEpilogueWarps) {
      int64_t tm, tn;
      tile_at(walker, tiles_m, tiles_n, &tm, &tn);
      finish_parts<TN, kMostParts>(g.out, smem, part, g.parts, half, tm * 2 * TM + half * TM, tn * TN, tid, kEpilogueWarps * 32);
    }
    __syncwarp();
  }
  // No CTA may leave while another can still reach into it (the MMAs read the second CTA's shared memory and write its tensor
  // memory; copies and epilogue warps signal the first one's barriers; partial sums are read by the whole cluster).
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc_pair(tmem_base, 512);
  }
}

// Byte matrix [rows, cols] in boxes of 128 rows x 128 bytes.
bool make_map(const Fp8View& v, CUtensorMap* map) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(v.K), static_cast<cuuint64_t>(v.rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(v.ld)};
  const cuuint32_t box[2] = {128, 128}, elem[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(v.codes), dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Pairs per tile: as many (1, 2, 4) as keep every cluster resident, two groups at least for each.
int choose_parts(int64_t tiles, int64_t pairs, int groups) {
  int parts = 1;
  while (parts < kMostParts && tiles * parts * 2 <= pairs && groups >= parts * 2 * 2) parts *= 2;
  return parts;
}

template <bool TRANS>
cudaError_t launch(Args g, const Fp8View& A, const Fp8View& W, int dev, int sms, cudaStream_t stream) {
  static DeviceOnce configured;
  if (configured.pending(dev)) {
    const cudaError_t e = cudaFuncSetAttribute(fp8_gemm_kernel<TRANS>, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    if (e != cudaSuccess) return e;
    configured.mark(dev);
  }
  CUtensorMap a_map, w_map;
  if (!make_map(A, &a_map) || !make_map(W, &w_map)) return cudaErrorNotSupported;
  const int64_t tiles = ((g.out.M + 2 * TM - 1) / (2 * TM)) * ((g.out.N + TN - 1) / TN), pairs = sms / 2;
  g.parts = choose_parts(tiles, pairs, g.groups);
  const int64_t clusters = g.parts > 1 ? tiles : (tiles < pairs ? tiles : pairs);
  return launch_pdl_cluster(fp8_gemm_kernel<TRANS>, dim3(static_cast<unsigned>(clusters * 2 * g.parts)), dim3(kThreads),
                            static_cast<unsigned>(2 * g.parts), kBytes, stream, g, a_map, w_map);
}

}  // namespace

cudaError_t launch_fp8_gemm(const Fp8View& A, const Fp8View& W, bool transposed, void* C, bool c_bf16, int64_t ldc, cudaStream_t stream) {
  int dev = 0, sms = 0;
  const cudaError_t e = current_device(&dev, &sms);
  if (e != cudaSuccess) return e;
  Args g{};
  g.a_s = A.scales; g.ld_as = A.ld_s; g.w_s = W.scales;
  g.w_step_n = transposed ? 1 : W.ld_s; g.w_step_g = transposed ? W.ld_s : 1;
  g.out = Out{C, ldc, c_bf16 ? 1 : 0, nullptr, 0, A.rows, transposed ? W.K : W.rows};
  g.groups = static_cast<int32_t>((A.K + kGroup - 1) / kGroup);
  return transposed ? launch<true>(g, A, W, dev, sms, stream) : launch<false>(g, A, W, dev, sms, stream);
}

cudaError_t fp8_gemm_health(int op, int* value) {
  switch (op) {
    case kHealthRead: return umma::read_error_word(value);
    case kHealthClear: return umma::clear_error_word();
    case kHealthSetSpinLimit: return umma::set_spin_limit(static_cast<uint32_t>(*value));
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace hbmm
