// Weight gradient from the 8-bit copy of the activations on the 5th-generation tensor cores: GW = gy^T X^ (+ base).
//
//   GW[n,k] = base[n,k] + sum_m gy[m,n] x^[m,k],   x^[m,k] = s[m, k/128] code[m,k]
//
// The contraction runs along the rows of both operands, and the scale changes with it: x^ has to be formed before the product.  For a
// power-of-two scale code * s is a bf16 number (e4m3 has four significant bits), so one bf16 product per pair is exact; any other
// scale costs a rounding to bf16.  gy and x^ enter the MMA as MN-major operands, as they lie in memory: nothing is transposed.
//
// A pair of CTAs takes a 256 x 256 tile of GW (cta_group::2, 256 x 256 x 16 MMAs, kind::f16) and walks along m in stages of 64 rows:
// per CTA 16 KB of gy (its 128 columns) and 8 KB of codes (its half of the 256 columns of X) by tensor copies; eight warps convert
// the codes into the 16 KB of bf16 that the MMA reads (128-byte-swizzled, conflict-free 16-byte stores).  512 clk of MMA per stage
// against 32 elements per converting thread.  The two accumulators of 256 columns let a tile's epilogue run beside the next one's MMAs.
//   warps 0-7   : epilogue (TMEM lanes 32 * (w % 4).., columns 128 * (w / 4)..)
//   warp  8     : this CTA's copies;  warp 9 : TMEM allocation, MMA issue in the first CTA;  warp 10 : scales, up to 16 stages ahead
//   warps 12-19 : converters;  warp 11, in the second CTA : tells the first that a stage is converted
// The first CTA's MMAs read what the second one's converters wrote.  These arrive at a barrier of their own CTA; a thread that waits
// there announces the stage by an asynchronous store, whose completion is a release at cluster scope and holds nobody up.  (8192 x
// 4096 x 4096: 250 us; with that store from the converters 280, with releasing arrivals 443, from the waiting thread 361 to 465.)
// Measured: 8192 x 4096 x 4096 250 us in a run of a few milliseconds, 1.1 PFLOP/s, 290 in one of seconds, where the 1000 W hold the SMs
// at 1630 of 1965 MHz (zeros: 239 at 1965, the same clocks).  Tensor pipe half of the time active: the converters take 930 clk per
// stage, and copies, conversion and MMA want 160 bytes of shared memory per clock at full rate, of 128.  256 x 4096 x 9216 46 us, 151
// MB written; 72 us with a base, 302 MB.
// Few tiles: a cluster of two to four pairs shares each tile in equal parts of m (fp8_tile.cuh).
#include <cuda_bf16.h>
#include "fp8_tile.cuh"
#include "kernels.h"
#include "pdl.cuh"
#include "tensor_map.h"

namespace hbmm {
namespace {

using namespace fp8;

constexpr int TN = 256, ROWS = 64;             // columns of a pair's tile; rows of the contraction per stage
constexpr int kThreads = 20 * 32, kEpilogueWarps = 8, kLoaderWarp = 8, kMmaWarp = 9, kScaleWarp = 10, kRelayWarp = 11, kConvertWarp = 12, kConvertWarps = 8;
constexpr int kOperand = 128 * ROWS * 2, kCodes = 128 * ROWS, STAGES = 5;          // bytes per stage of gy and of converted X; of codes
constexpr int kChunkBytes = ROWS * 128;        // 64 columns of an operand: 128 bytes per row
constexpr int kSlots = 16;                     // stages of scales
constexpr int OFF_A = 0, OFF_B = STAGES * kOperand, OFF_CODES = 2 * STAGES * kOperand, OFF_OUT = OFF_CODES + STAGES * kCodes;
constexpr int OFF_SCALES = OFF_OUT + kEpilogueWarps * kStoreBytes, OFF_BAR = OFF_SCALES + kSlots * ROWS * 4;
constexpr int kBars = 6 * STAGES + 2 * kSlots + 5;
constexpr int OFF_SENT = OFF_BAR + kBars * 8, kBytes = OFF_SENT + 8 + 4 + STAGES * 4 + 8;
// An accumulator in tensor memory takes 512 rows, the epilogue adds it to fp32 registers: the tensor cores' additions truncate, always
// towards zero, and with 8192 rows of sizes from 2^-8 to 2^8 in one accumulator the result was 9e-6 off.
constexpr int kChunkStages = 512 / ROWS;
constexpr int kRegsEpilogue = 176, kRegsOthers = 40;         // 256 x 176 + 384 x 40 of the 640 x 96 registers at launch
static_assert(kBytes <= 227 * 1024 && TM * TN * 4 <= OFF_CODES, "shared memory");

struct Args {
  const float* x_s; int64_t ld_xs;
  Out out;                                     // M: rows of GW (columns of gy), N: columns of GW (of X)
  int64_t rows;                                // of gy and X
  int32_t stages, parts;
};

__global__ void __launch_bounds__(kThreads, 1)
fp8_weight_grad_kernel(const Args g, const __grid_constant__ CUtensorMap gy_map, const __grid_constant__ CUtensorMap x_map) {
  extern __shared__ __align__(1024) unsigned char smem[];
  uint64_t* afull = reinterpret_cast<uint64_t*>(smem + OFF_BAR);     // first CTA: gy of both CTAs
  // this CTA's codes: two barriers per stage, as two halves of the converters take turns and the number of stages is odd (with one,
  // a half would wait for the same parity at every visit, and pass when the other half's codes have not come yet)
  uint64_t* cfull = afull + STAGES;
  uint64_t* bfull = cfull + 2 * STAGES;        // first CTA: converted, in both CTAs
  uint64_t* bdone = bfull + STAGES;            // second CTA: converted here
  uint64_t* empty = bdone + STAGES;
  uint64_t* sfull = empty + STAGES;            // scales of a stage
  uint64_t* sempty = sfull + kSlots;
  uint64_t* tfull = sempty + kSlots;
  uint64_t* tempty = tfull + 2;
  uint64_t* drained = tempty + 2;
  int64_t* issued = reinterpret_cast<int64_t*>(smem + OFF_SENT);     // stages that this CTA's loader has issued, in the end
  uint32_t* announced = reinterpret_cast<uint32_t*>(issued + 1);     // second CTA: stages that it has announced, in the end
  uint32_t* told = announced + 1;              // first CTA, [STAGES]: where the announcements land, the number of the stage (from 1)
  uint32_t* tmem_base_ptr = told + STAGES;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_base_ptr + 1);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_ctarank(), lead = rank & ~1u, half = rank & 1u;
  const int64_t tiles_m = (g.out.M + 2 * TM - 1) / (2 * TM), tiles_n = (g.out.N + TN - 1) / TN, n_tiles = tiles_m * tiles_n;
  const int part = static_cast<int>(rank >> 1);
  const int64_t walker = blockIdx.x / (2 * g.parts), walkers = gridDim.x / (2 * g.parts);
  const int s0 = static_cast<int>(static_cast<int64_t>(part) * g.stages / g.parts), s1 = static_cast<int>(static_cast<int64_t>(part + 1) * g.stages / g.parts);

  pdl_launch_dependents();
  if (tid == 0) {
    for (int s = 0; s < STAGES; s++) {
      mbar_init(&afull[s], 1);
      mbar_init(&cfull[s], 1);
      mbar_init(&cfull[STAGES + s], 1);
      mbar_init(&bfull[s], kConvertWarps / 2 + 1);          // one half of this CTA's converters; its loader's expect_tx for the other CTA's word
      mbar_init(&bdone[s], kConvertWarps / 2);
      mbar_init(&empty[s], 1);
    }
    for (int s = 0; s < kSlots; s++) { mbar_init(&sfull[s], 32); mbar_init(&sempty[s], kConvertWarps / 2); }
    for (int b = 0; b < 2; b++) { mbar_init(&tfull[b], 1); mbar_init(&tempty[b], 2 * kEpilogueWarps); }
    mbar_init(drained, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid < STAGES) told[tid] = 0;
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
  const Waiter wait{g_spin_limit, abort_flag};

  if (warp >= kEpilogueWarps) reg_dec<kRegsOthers>();
  if (warp == kLoaderWarp) {
    // =========================== loader (both CTAs) ===========================
    if (elect_one()) {
      asm volatile("prefetch.tensormap [%0];" ::"l"(&gy_map) : "memory");
      asm volatile("prefetch.tensormap [%0];" ::"l"(&x_map) : "memory");
      const uint32_t afull0 = mapa_rank(smem_u32(afull), lead);
      int s = 0, c = 0;
      uint32_t par = 1;                                  // the first round waits for nobody
      int64_t n_issued = 0;
      bool ok = true;
      for (int64_t tile = walker; tile < n_tiles && ok; tile += walkers) {
        int64_t tm, tn;
        tile_at(tile, tiles_m, tiles_n, &tm, &tn);
        const int32_t n_at = static_cast<int32_t>(tm * 2 * TM + half * TM), k_at = static_cast<int32_t>(tn * TN + half * (TN / 2));
        for (int st = s0; st < s1; st++) {
          if (!wait(smem_u32(&empty[s]), par, 1)) { ok = false; break; }
          if (half == 0) {
            mbar_arrive_expect_tx(&afull[s], 2 * kOperand);
            mbar_arrive_expect_tx(&bfull[s], 4);
          }
          mbar_arrive_expect_tx(&cfull[c], kCodes);
          tma_load_2d(smem + OFF_CODES + s * kCodes, &x_map, k_at, st * ROWS, &cfull[c]);
          if (++c == 2 * STAGES) c = 0;
          unsigned char* a = smem + OFF_A + s * kOperand;
          tma_load_2d_pair(a, &gy_map, n_at, st * ROWS, afull0 + s * 8);
          tma_load_2d_pair(a + kChunkBytes, &gy_map, n_at + 64, st * ROWS, afull0 + s * 8);
          n_issued++;
          if (++s == STAGES) { s = 0; par ^= 1; }
        }
      }
      *issued = n_issued;
    }
    __syncwarp();
  } else if (warp == kScaleWarp) {
    // =========================== scale loader (both CTAs) ===========================
    uint32_t f = 0, par = 1;
    bool ok = true;
    for (int64_t tile = walker; tile < n_tiles && ok; tile += walkers) {
      int64_t tm, tn;
      tile_at(tile, tiles_m, tiles_n, &tm, &tn);
      const int64_t block = tn * 2 + half;
      for (int st = s0; st < s1; st++) {
        if (!wait(smem_u32(&sempty[f]), par, 8)) { ok = false; break; }
        const uint32_t slot = smem_u32(smem + OFF_SCALES + f * ROWS * 4);
#pragma unroll
        for (int i = 0; i < ROWS / 32; i++) {
          const int64_t m = static_cast<int64_t>(st) * ROWS + 32 * i + lane;
          const bool in = m < g.rows && block * kGroup < g.out.N;
          cp_async4(slot + (32 * i + lane) * 4, g.x_s + (in ? m * g.ld_xs + block : 0), in ? 4 : 0);
        }
        cp_async_arrive(&sfull[f]);
        if (++f == kSlots) { f = 0; par ^= 1; }
      }
    }
    cp_async_wait_all();                                 // also after an abort
    __syncwarp();
  } else if (warp == kRelayWarp) {
    // =========================== announcements (second CTA) ===========================
    if (half != 0 && elect_one()) {
      const uint32_t bfull0 = mapa_rank(smem_u32(bfull), lead), told0 = mapa_rank(smem_u32(told), lead);
      uint32_t s = 0, par = 0, n = 0;
      bool ok = true;
      for (int64_t tile = walker; tile < n_tiles && ok; tile += walkers)
        for (int st = s0; st < s1; st++) {
          if (!wait(smem_u32(&bdone[s]), par, 7)) { ok = false; break; }
          st_async_u32(told0 + s * 4, ++n, bfull0 + s * 8);
          if (++s == STAGES) { s = 0; par ^= 1; }
        }
      *announced = n;
    }
    __syncwarp();
  } else if (warp >= kConvertWarp) {
    // =========================== converters (both CTAs) ===========================
    // Four warps per stage, the other four on the next one: a warp's waits and its fence come once per four items of work.
    const int me = tid - kConvertWarp * 32 & 127;
    const uint32_t mine = (warp - kConvertWarp) / 4;
    const uint32_t converted = smem_u32(half == 0 ? bfull : bdone);
    const int q = me & 7;                                // 16 codes from column 16 q, rows me / 8 + 16 i
    uint32_t s = 0, c = 0, c_par = 0, f = 0, f_par = 0, turn = 0;
    bool ok = true;
    for (int64_t tile = walker; tile < n_tiles && ok; tile += walkers) {
      for (int st = s0; st < s1; st++, turn ^= 1) {
        if (turn == mine) {
          if (!wait(smem_u32(&sfull[f]), f_par, 7) || !wait(smem_u32(&cfull[c]), c_par, 7)) { ok = false; break; }
          const float* scales = reinterpret_cast<const float*>(smem + OFF_SCALES + f * ROWS * 4) + (me >> 3);
          const unsigned char* codes = smem + OFF_CODES + s * kCodes + me * 16;
          // two 16-byte pieces of the row's 64 columns; lanes of the second 64 columns store theirs in the other order, so that the
          // eight lanes of a row hit different banks (rows 16 apart share their swizzle)
          const bool swap = (q & 4) != 0;
          unsigned char* rows64 = smem + OFF_B + s * kOperand + (q >> 2) * kChunkBytes;
          unsigned char* to0 = swz(rows64, me >> 3, 2 * (q & 3) + (swap ? 1 : 0));
          unsigned char* to1 = swz(rows64, me >> 3, 2 * (q & 3) + (swap ? 0 : 1));
#pragma unroll
          for (int i = 0; i < ROWS / 16; i++) {
            const uint4 x = *reinterpret_cast<const uint4*>(codes + i * 16 * 128);
            const float sc = scales[i * 16];
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
            uint32_t o[8];
#pragma unroll
            for (int e = 0; e < 4; e++) {
              const float2 lo = from_e4m3x2(w[e] & 0xFFFFu), hi = from_e4m3x2(w[e] >> 16);
              o[2 * e] = bf16x2(lo.x * sc, lo.y * sc);
              o[2 * e + 1] = bf16x2(hi.x * sc, hi.y * sc);
            }
            *reinterpret_cast<uint4*>(to0 + i * 16 * 128) = swap ? make_uint4(o[4], o[5], o[6], o[7]) : make_uint4(o[0], o[1], o[2], o[3]);
            *reinterpret_cast<uint4*>(to1 + i * 16 * 128) = swap ? make_uint4(o[0], o[1], o[2], o[3]) : make_uint4(o[4], o[5], o[6], o[7]);
          }
          fence_async_proxy();                           // the stores are the tensor core's to read
          __syncwarp();
          if (lane == 0) {
            mbar_arrive_a(converted + s * 8);
            mbar_arrive(&sempty[f]);
          }
        }
        if (++s == STAGES) s = 0;
        if (++c == 2 * STAGES) { c = 0; c_par ^= 1; }
        if (++f == kSlots) { f = 0; f_par ^= 1; }
      }
    }
  } else if (warp == kMmaWarp) {
    // =========================== MMA issuer (first CTA of the pair) ===========================
    if (half == 0 && elect_one()) {
      constexpr uint32_t idesc = instr_desc_pair(TN, kFmtBF16) | kTransposeA | kTransposeB;
      constexpr uint32_t kStepRows = (16 * 128) >> 4;                      // 16 rows of the contraction
      const uint16_t both = static_cast<uint16_t>(3u << lead);
      const uint64_t da0 = smem_desc_mn(smem_u32(smem + OFF_A), kChunkBytes), db0 = smem_desc_mn(smem_u32(smem + OFF_B), kChunkBytes);
      const uint64_t da_hi = da0 & 0xFFFFFFFF00000000ull, db_hi = db0 & 0xFFFFFFFF00000000ull;
      const uint32_t da_lo = static_cast<uint32_t>(da0), db_lo = static_cast<uint32_t>(db0);
      const uint32_t afull_a = smem_u32(afull), bfull_a = smem_u32(bfull), empty_a = smem_u32(empty), tfull_a = smem_u32(tfull), tempty_a = smem_u32(tempty);
      uint32_t s = 0, par = 0, acc = 0;
      bool ok = true;
      for (int64_t tile = walker; tile < n_tiles && ok; tile += walkers) {
        for (int c0 = s0; c0 < s1 && ok; c0 += kChunkStages, acc++) {
          const int c1 = s1 - c0 < kChunkStages ? s1 : c0 + kChunkStages;
          const uint32_t buf = acc & 1;
          if (acc >= 2 && !wait(tempty_a + buf * 8, ((acc >> 1) & 1) ^ 1, 3)) { ok = false; break; }
          for (int st = c0; st < c1; st++) {
            if (!wait(afull_a + s * 8, par, 2) || !wait.cluster(bfull_a + s * 8, par, 2)) { ok = false; break; }
            tc_fence_after();
            const uint32_t a_lo = da_lo + s * (kOperand >> 4), b_lo = db_lo + s * (kOperand >> 4);
#pragma unroll
            for (uint32_t ks = 0; ks < ROWS / 16; ks++)
              umma_bf16_pair(tmem_base + buf * TN, da_hi | (a_lo + ks * kStepRows), db_hi | (b_lo + ks * kStepRows), idesc, st != c0 || ks != 0 ? 1u : 0u);
            umma_commit_pair_mc(empty_a + s * 8, both);
            if (++s == STAGES) { s = 0; par ^= 1; }
          }
          if (ok) umma_commit_pair_mc(tfull_a + buf * 8, both);
        }
      }
      // every MMA issued so far has retired (in both CTAs) before tensor memory is released -- also after an abort
      umma_commit_pair(smem_u32(drained));
      if (!mbar_wait_quiet(drained, 0, wait.limit < kDrainPolls ? kDrainPolls : wait.limit)) {
        atomicCAS(&g_error_word, 0, 4);
        *abort_flag = 1;
      }
    }
    __syncwarp();
  } else if (warp < kEpilogueWarps) {
    // =========================== epilogue (both CTAs) ===========================
    reg_inc<kRegsEpilogue>();
    const int row = (warp & 3) * 32 + lane, col0 = (warp >> 2) * (TN / 2);
    const uint32_t tmem_at = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16) + col0;
    const uint32_t tempty0 = mapa_rank(smem_u32(tempty), lead);
    unsigned char* stage = smem + OFF_OUT + warp * kStoreBytes;
    uint32_t n = 0;
    bool ok = true;
    for (int64_t tile = walker; tile < n_tiles && ok; tile += walkers) {
      uint64_t acc[kRun];
#pragma unroll
      for (int j = 0; j < kRun; j++) acc[j] = 0ull;
      int64_t tm, tn;
      tile_at(tile, tiles_m, tiles_n, &tm, &tn);
      const int64_t m0 = tm * 2 * TM + half * TM + (warp & 3) * 32, n0 = tn * TN + col0;
      if (g.parts == 1) prefetch_base(g.out, m0, n0, lane);
      for (int c0 = s0; c0 < s1; c0 += kChunkStages, n++) {
        const uint32_t buf = n & 1;
        if (!wait(smem_u32(&tfull[buf]), (n >> 1) & 1, 5)) { ok = false; break; }
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < 8; c++) {
          uint32_t d[16];
          tmem_ld16(tmem_at + buf * TN + c * 16, d);
          tmem_ld_wait(d);
#pragma unroll
          for (int j = 0; j < 16; j += 2) acc[c * 8 + j / 2] = add2(pack2(d[j], d[j + 1]), acc[c * 8 + j / 2]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster_read(tempty0 + buf * 8);
      }
      if (!ok) break;
      if (g.parts == 1) store_tile<true>(g.out, stage, acc, m0, n0, n0 + kRun, lane);
      // every stage of this CTA's only tile has been read: its partial sums take their place
      else stage_part<TN>(smem, acc, row, col0, col0 + kRun);
    }
  }

  if (g.parts > 1) {
    __syncwarp();
    cluster_sync_all();
    if (warp < kEpilogueWarps) {
      int64_t tm, tn;
      tile_at(walker, tiles_m, tiles_n, &tm, &tn);
      finish_parts<TN>(g.out, smem, part, g.parts, half, tm * 2 * TM + half * TM, tn * TN, tid, kEpilogueWarps * 32);
    }
  }
  leave_cluster(abort_flag, 2 * g.parts, [&](uint32_t me) {
    const int64_t n = *issued;
    for (int64_t i = n > STAGES ? n - STAGES : 0; i < n; i++)
      mbar_wait_quiet(&cfull[i % (2 * STAGES)], static_cast<uint32_t>((i / (2 * STAGES)) & 1), kDrainPolls);
    if ((me & 1) == 0) {
      drain_pair_copies<STAGES>(afull, n, ld_cluster_s64(mapa_rank(smem_u32(issued), me + 1)), kOperand);
    } else {
      const uint32_t m = *announced;
      for (uint32_t i = m > STAGES ? m - STAGES : 0; i < m; i++) wait_word(mapa_rank(smem_u32(told + i % STAGES), me - 1), ~0u, i + 1);
    }
  });
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc_pair(tmem_base, 512);
  }
}

std::atomic<int> g_resident[64][kMostParts + 1];          // per device

bool make_map(const void* p, bool bf16, int64_t rows, int64_t cols, int64_t pitch, CUtensorMap* map) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(pitch)};
  const cuuint32_t box[2] = {bf16 ? 64u : 128u, ROWS}, elem[2] = {1, 1};
  return fn(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(p), dims, strides, box, elem,
            CU_TENSOR_MAP_INTERLEAVE_NONE, bf16 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

cudaError_t launch_fp8_weight_grad(const void* gy, int64_t N, int64_t ldg, const Fp8View& X, const float* base, int64_t ld_base, float* gw,
                                   int64_t ldw, cudaStream_t stream) {
  static DeviceOnce configured;
  int dev = 0, sms = 0;
  cudaError_t e = current_device(&dev, &sms);
  if (e != cudaSuccess) return e;
  if (configured.pending(dev)) {
    e = cudaFuncSetAttribute(fp8_weight_grad_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kBytes);
    if (e != cudaSuccess) return e;
    configured.mark(dev);
  }
  CUtensorMap gy_map, x_map;
  if (!make_map(gy, true, X.rows, N, ldg * 2, &gy_map) || !make_map(X.codes, false, X.rows, X.K, X.ld, &x_map)) return cudaErrorNotSupported;
  Args g{};
  g.x_s = X.scales; g.ld_xs = X.ld_s;
  g.out = Out{gw, ldw, 0, base, ld_base, N, X.K};
  g.rows = X.rows;
  g.stages = static_cast<int32_t>((X.rows + ROWS - 1) / ROWS);
  const int64_t tiles = ((N + 2 * TM - 1) / (2 * TM)) * ((X.K + TN - 1) / TN), pairs = sms / 2;
  g.parts = dev >= 0 && dev < 64 ? choose_parts(fp8_weight_grad_kernel, kThreads, kBytes, g_resident[dev], tiles, pairs, g.stages, 4) : 1;
  const int64_t clusters = g.parts > 1 ? tiles : (tiles < pairs ? tiles : pairs);
  return launch_pdl_cluster(fp8_weight_grad_kernel, dim3(static_cast<unsigned>(clusters * 2 * g.parts)), dim3(kThreads), static_cast<unsigned>(2 * g.parts),
                            kBytes, stream, g, gy_map, x_map);
}

cudaError_t fp8_weight_grad_expire_wait(cudaStream_t stream) { return launch_wait_expiry(stream); }

cudaError_t fp8_weight_grad_health(int op, int* value) {
  switch (op) {
    case kHealthRead: return umma::read_error_word(value);
    case kHealthClear: return umma::clear_error_word();
    case kHealthSetSpinLimit: return umma::set_spin_limit(static_cast<uint32_t>(*value));
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace hbmm
