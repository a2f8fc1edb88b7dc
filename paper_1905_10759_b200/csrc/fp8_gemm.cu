// Products of 8-bit operands on the 5th-generation tensor cores (tcgen05 / TMEM): C = A^ W^^T and C = A^ W^.
//
//   C[m,n] = sum_g (sA[m,g] sW[n/128,g]) D_g[m,n],   D_g[m,n] = sum_{k in group g} A[m,k] W[n,k]
//
// A pair of CTAs takes a 256 x 256 tile (cta_group::2, 256 x N x 32 MMAs); how it sums the groups goes by their scales, four groups
// (a step) at a time:
//   * all of them powers of two (what hbmm_fp8_quantize writes): the tensor cores apply them (kind::mxf8f6f4, block scales: a UE8M0
//     byte per row and 32 elements, here the same byte for the four instructions of a group) and a run along K (kChunk below) is
//     one accumulation in tensor memory, 256 columns;
//   * otherwise each group's dot products go to one of three units of 128 columns, and the epilogue adds them, times the two scales,
//     to fp32 registers.  The accumulation in tensor memory is left where it stands and taken first.
// The second way costs 560 clk per 128 columns and group, MMA to epilogue and back (8192^3 with scales of any value 0.57 ms in short
// runs, 1.94 PFLOP/s, 0.69 in long ones; in seven units of 64 columns 1.17 ms).  The first is bound by the tensor cores' power: 8192^3
// to bf16 0.38 to 0.39 ms in a run of a few milliseconds, 0.46 (2.4 PFLOP/s) in one of seconds, where the 1000 W hold the SMs at 1160
// of 1965 MHz; with operands of zeros, which take less, 0.29.  To fp32 0.41 to 0.51.  Tensor pipe 82 % active on 2048 x 8192 x 8192.
//
// C = A^ W^ (the input gradient; the contraction runs along the rows of W) reads the same W: its tiles arrive as 128 rows of the
// contraction x 128 columns and enter the MMA as an MN-major operand.  Nothing is transposed in memory.
//
// Per CTA and group 16 KB of A (its own 128 rows) and 16 KB of W (its half of the 256 columns) arrive by tensor copies (128-byte
// swizzle, zeros outside the matrices, so no edge needs a case of its own); six stages in flight.
//   warps 0-7   : epilogue (TMEM lanes 32 * (w % 4)..; columns 64 h .. and 128 + 64 h .. with h = w / 4)
//   warp  8     : one thread issues this CTA's copies;  warp 9 : TMEM allocation, and in the first CTA the MMA-issuing thread
//   warp  10    : copies each step's scales to shared memory, up to eight steps ahead (11 hands over registers)
//   warps 12-15 : scouts: look the scales over and write their exponents to tensor memory
// What one CTA writes and the other depends on (the factors, which the first CTA's MMAs take from both tensor memories, and the kind
// of the scales) is announced by asynchronous stores that complete on the barrier the readers wait at, a release at cluster scope;
// the arrivals across the pair release nothing but reads.  (Store and releasing arrival: 2600 clk beside the copies, 0.53 ms.)
// Products of few tiles: a cluster of two to four pairs shares each tile in equal parts of K (fp8_tile.cuh).
#include <cuda_bf16.h>
#include "fp8_tile.cuh"
#include "kernels.h"
#include "pdl.cuh"
#include "tensor_map.h"

namespace hbmm {
namespace {

using namespace fp8;

constexpr int TN = 256;                        // columns of a pair's tile
constexpr int kThreads = 16 * 32, kEpilogueWarps = 8, kLoaderWarp = 8, kMmaWarp = 9, kScaleWarp = 10, kScoutWarp = 12;
constexpr int kRegsEpilogue = 200, kRegsIssue = 56, kRegsScout = 56;      // 256 x 200 + 128 x 56 + 128 x 56 = 64 K registers
constexpr int kTile = 128 * 128;               // bytes of an operand's part of a stage
constexpr int STAGE = 2 * kTile, STAGES = 6;
// A step is four groups: its scales arrive together, beside the stages.  Shared memory of a slot: 128 rows x 4 scales of A, then W's.
constexpr int kStep = 4, kSlots = 8, kScalesA = 128 * kStep * 4, kSlotBytes = kScalesA + 128;
// Tensor memory: three units of 128 columns for partial sums (a whole accumulator takes the first two), then the factors of each
// slot, 16 columns (4 of A, 8 of W).
// A whole accumulator takes a run of kChunk steps, then the epilogue adds it to fp32 registers.  An instruction cuts its 32 products and
// the sum so far below 2^-25 of the largest of them and truncates what they add up to (always towards zero), so the error of a run
// grows with its length where nothing cancels.  Positive operands, groups of sizes from 2^-12 to 2^12, K = 16384, relative to the
// norm: 1.3e-5 with runs of 8192 elements, 5.4e-6 with 4096, 2.9e-6 with 2048, 1.5e-6 with 1024, 8e-7 with 512; random signs and
// one size, K = 8192: 1.2e-7, 7.6e-8 with 1024.  Taking an accumulator holds the MMAs up: 8192^3 381 us with runs of 8192, 390 with
// 4096, 408 with 2048, 444 with 1024; 8192 x 4096 x 4096 99, 99, 103, 119.  An fp32 result gets 2048, as below that the time grows
// faster than the error falls; a bf16 result, whose own rounding is up to 3.9e-3, gets 8192.
constexpr int kChunkF32 = 4, kChunkBF16 = 16;
constexpr int kUnit = 128, kUnits = 3, kTurns = 2 * kUnits, kFactorCols = 384, kFactorSlot = 16;
constexpr int OFF_A = 0, OFF_B = STAGES * kTile, OFF_OUT = STAGES * STAGE, OFF_SCALES = OFF_OUT + kEpilogueWarps * kStoreBytes;
constexpr int OFF_BAR = OFF_SCALES + kSlots * kSlotBytes;
constexpr int kBars = 2 * STAGES + 2 * kTurns + 2 + 3 * kSlots + 1;
constexpr int kScouts = 4, kFlags = 2 * kScouts;                             // words of a slot: one from each scout of both CTAs
// In such a word.  Tested by the sign: with the lowest bit in its place, masked out, scales of any value took 580 us at 8192^3, not 562
// (the same work otherwise; by how the compiler arranged the epilogue).
constexpr uint32_t kNoFactors = 1u << 31;
constexpr int OFF_FLAGS = OFF_BAR + kBars * 8, OFF_SENT = OFF_FLAGS + kSlots * kFlags * 4, kBytes = OFF_SENT + 8 + kScouts * 4 + 8;
static_assert(kBytes <= 227 * 1024 && TM * TN * 4 <= STAGES * STAGE && kFactorCols + kSlots * kFactorSlot <= 512, "shared and tensor memory");

struct Args {
  const float* a_s; int64_t ld_as;
  const float* w_s; int64_t w_step_n, w_step_g;        // scale of (column block, group): w_s[block * w_step_n + group * w_step_g]
  Out out;
  int32_t groups;                              // of the contraction
  int32_t parts;                               // pairs (of one cluster) that share a tile
};

// A normal power of two: what the tensor cores' own factors can be.
__device__ __forceinline__ bool is_factor(uint32_t bits) { return (bits & 0x807FFFFFu) == 0 && bits - 0x00800000u < 0x7F000000u; }

// The scale of the tile's block b (0, 1) of columns in the step's group j.
template <bool TRANS>
__device__ __forceinline__ float w_scale(const unsigned char* at, int b, int j) {
  return *reinterpret_cast<const float*>(at + (TRANS ? j * 2 + b : b * 4 + j) * 4);
}

template <bool TRANS>
__global__ void __launch_bounds__(kThreads, 1)
fp8_gemm_kernel(const Args g, const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap w_map) {
  extern __shared__ __align__(1024) unsigned char smem[];
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + OFF_BAR);
  uint64_t* empty = full + STAGES;
  // units of partial sums: partial sum i lies in unit i % 3, is read by warpgroup i % 2 and has barrier i % 6, so that a warpgroup
  // meets a barrier of its own at its visits, one parity after the other
  uint64_t* ufull = empty + STAGES;
  uint64_t* uempty = ufull + kTurns;
  uint64_t* xfull = uempty + kTurns;           // the whole accumulator
  uint64_t* xempty = xfull + 1;
  uint64_t* scales = xempty + 1;               // a step's scales are in this CTA's shared memory
  uint64_t* sfull = scales + kSlots;           // its factors are in both CTAs' tensor memory, and how it is summed is known
  uint64_t* sempty = sfull + kSlots;           // its slot is free in both CTAs
  uint64_t* drained = sempty + kSlots;
  // [kSlots][CTA of the pair][scout]: the number of the step (from 1), and the topmost bit where its scales are no factors
  uint32_t* flags = reinterpret_cast<uint32_t*>(smem + OFF_FLAGS);
  int64_t* issued = reinterpret_cast<int64_t*>(smem + OFF_SENT);               // stages that this CTA's loader has issued, in the end
  uint32_t* looked = reinterpret_cast<uint32_t*>(issued + 1);                  // steps that each of its scouts has announced
  uint32_t* tmem_base_ptr = looked + kScouts;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_base_ptr + 1);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_ctarank(), lead = rank & ~1u, half = rank & 1u;      // the pair's first CTA; this CTA's rows of the tile
  const int64_t tiles_m = (g.out.M + 2 * TM - 1) / (2 * TM), tiles_n = (g.out.N + TN - 1) / TN, n_tiles = tiles_m * tiles_n;
  const int part = static_cast<int>(rank >> 1);
  // the pair's walk: tiles of its own, or one tile's groups [g0, g1) of `parts`
  const int64_t walker = blockIdx.x / (2 * g.parts), walkers = gridDim.x / (2 * g.parts);
  const int steps = (g.groups + kStep - 1) / kStep, chunk = g.out.bf16 ? kChunkBF16 : kChunkF32;
  const int g0 = static_cast<int>(static_cast<int64_t>(part) * steps / g.parts) * kStep;
  const int g_end = static_cast<int>(static_cast<int64_t>(part + 1) * steps / g.parts) * kStep, g1 = g_end < g.groups ? g_end : g.groups;

  pdl_launch_dependents();
  if (tid == 0) {
    for (int s = 0; s < STAGES; s++) {
      mbar_init(&full[s], 1);           // first CTA: its loader's expect_tx arrival; the copies of both CTAs complete the bytes
      mbar_init(&empty[s], 1);          // MMA commit (to both CTAs)
    }
    for (int u = 0; u < kTurns; u++) { mbar_init(&ufull[u], 1); mbar_init(&uempty[u], kEpilogueWarps); }    // one warpgroup of each CTA
    mbar_init(xfull, 1);
    mbar_init(xempty, 2 * kEpilogueWarps);
    for (int f = 0; f < kSlots; f++) {
      mbar_init(&scales[f], 32);                            // the scale loader's lanes
      mbar_init(&sfull[f], kScouts);                        // this CTA's scouts; the words of both CTAs' complete the bytes
      mbar_init(&sempty[f], 2 * kEpilogueWarps + 1);        // epilogue warps of both CTAs, MMA commit
    }
    mbar_init(drained, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid < kSlots * kFlags) flags[tid] = 0;            // no step's number
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
  const auto are_factors = [&](uint32_t f) {           // behind sfull; a CTA's scouts have looked at the same scales
    const volatile uint32_t* v = flags + f * kFlags;
    return static_cast<int32_t>(v[0] | v[kScouts]) >= 0;
  };

  if (warp >= kScoutWarp) reg_dec<kRegsScout>();
  else if (warp >= kEpilogueWarps) reg_dec<kRegsIssue>();
  if (warp == kLoaderWarp) {
    // =========================== loader (both CTAs) ===========================
    if (elect_one()) {
      asm volatile("prefetch.tensormap [%0];" ::"l"(&a_map) : "memory");
      asm volatile("prefetch.tensormap [%0];" ::"l"(&w_map) : "memory");
      const uint32_t full0 = mapa_rank(smem_u32(full), lead);
      int s = 0;
      uint32_t round = 0;
      int64_t n_issued = 0;
      bool ok = true;
      for (int64_t tile = walker; tile < n_tiles && ok; tile += walkers) {
        int64_t tm, tn;
        tile_at(tile, tiles_m, tiles_n, &tm, &tn);
        const int32_t a_row = static_cast<int32_t>(tm * 2 * TM + half * TM), w_at = static_cast<int32_t>(tn * TN + half * (TN / 2));
        for (int kb = g0; kb < g1; kb++) {
          if (round > 0 && !wait(smem_u32(&empty[s]), (round & 1) ^ 1, 1)) { ok = false; break; }
          if (half == 0) mbar_arrive_expect_tx(&full[s], 2 * STAGE);
          const uint32_t bar = full0 + s * 8;
          tma_load_2d_pair(smem + OFF_A + s * kTile, &a_map, kb * kGroup, a_row, bar);
          if (TRANS) tma_load_2d_pair(smem + OFF_B + s * kTile, &w_map, w_at, kb * kGroup, bar);
          else tma_load_2d_pair(smem + OFF_B + s * kTile, &w_map, kb * kGroup, w_at, bar);
          n_issued++;
          if (++s == STAGES) { s = 0; round++; }
        }
      }
      *issued = n_issued;
    }
    __syncwarp();
  } else if (warp == kScaleWarp) {
    // =========================== scale loader (both CTAs) ===========================
    // As far ahead of the stages as there are slots.  16 bytes of every row: by lanes, as a tensor copy takes such short rows one by
    // one and holds up the stages behind it.
    uint32_t f = 0, f_par = 1;                           // the first round waits for nobody
    bool ok = true;
    for (int64_t tile = walker; tile < n_tiles && ok; tile += walkers) {
      int64_t tm, tn;
      tile_at(tile, tiles_m, tiles_n, &tm, &tn);
      const int64_t m0 = tm * 2 * TM + half * TM, rows = g.out.M - m0;
      for (int kb = g0; kb < g1; kb += kStep) {
        if (!wait(smem_u32(&sempty[f]), f_par, 8)) { ok = false; break; }
        const uint32_t slot = smem_u32(smem + OFF_SCALES + f * kSlotBytes);
        const int bytes = 4 * (g1 - kb < kStep ? g1 - kb : kStep);
#pragma unroll
        for (int c = 0; c < 4; c++) {
          const int row = 32 * c + lane;
          const bool in = row < rows;
          cp_async16(slot + row * 16, g.a_s + (in ? (m0 + row) * g.ld_as + kb : 0), in ? bytes : 0);
        }
        // W's, [block][group] or [group][block]: one by one (the two blocks need not lie in one aligned 16 bytes)
        const int b = TRANS ? lane & 1 : lane >> 2, j = TRANS ? lane >> 1 : lane & 3;
        if (lane < 8) {
          const bool in = kb + j < g1 && (tn * 2 + b) * kGroup < g.out.N;
          cp_async4(slot + kScalesA + lane * 4, g.w_s + (in ? (tn * 2 + b) * g.w_step_n + (kb + j) * g.w_step_g : 0), in ? 4 : 0);
        }
        cp_async_arrive(&scales[f]);
        if (++f == kSlots) { f = 0; f_par ^= 1; }
      }
    }
    cp_async_wait_all();                                 // also after an abort
    __syncwarp();
  } else if (warp == kMmaWarp) {
    // =========================== MMA issuer (first CTA of the pair) ===========================
    if (half == 0 && elect_one()) {
      constexpr uint32_t kMajor = TRANS ? kTransposeB : 0u;
      // 32 elements of the contraction: 32 bytes along K-major rows, 32 rows of 128 bytes of an MN-major tile
      constexpr uint32_t kStepA = 32 >> 4, kStepB = (TRANS ? 32 * 128 : 32) >> 4;
      constexpr uint32_t kHalfB = (TRANS ? 64 : 64 * 128) >> 4;            // 64 columns further
      const uint16_t both = static_cast<uint16_t>(3u << lead);
      const uint64_t da0 = smem_desc(smem_u32(smem + OFF_A)), db0 = smem_desc(smem_u32(smem + OFF_B));
      const uint64_t da_hi = da0 & 0xFFFFFFFF00000000ull, db_hi = db0 & 0xFFFFFFFF00000000ull;
      const uint32_t da_lo = static_cast<uint32_t>(da0), db_lo = static_cast<uint32_t>(db0);
      const uint32_t full_a = smem_u32(full), empty_a = smem_u32(empty), ufull_a = smem_u32(ufull), uempty_a = smem_u32(uempty);
      const uint32_t sempty_a = smem_u32(sempty);
      uint32_t s = 0, full_par = 0;            // stage
      uint32_t u = 0, u_round = 0;             // barrier of the next partial sum, and how often the ring of six went round
      uint32_t x = 0;                          // whole accumulators so far
      uint32_t f = 0, f_par = 0;               // slot of scales
      bool ok = true;
      // the accumulator's columns are free: the units' last partial sums and the last whole accumulator have been read
      const auto accumulator_free = [&] {
        if (x > 0 && !wait(smem_u32(xempty), (x & 1) ^ 1, 3)) return false;
        for (uint32_t i = 0; i < kTurns; i++) {
          const uint32_t uses = u_round + (u > i ? 1 : 0);
          if (i % kUnits < 2 && uses > 0 && !wait(uempty_a + i * 8, (uses & 1) ^ 1, 3)) return false;
        }
        return true;
      };
      for (int64_t tile = walker; tile < n_tiles && ok; tile += walkers) {
        int open = 0;                          // steps in the accumulator
        const auto close = [&] {
          umma_commit_pair_mc(smem_u32(xfull), both);
          x++;
          open = 0;
        };
        for (int kb0 = g0; kb0 < g1 && ok; kb0 += kStep) {
          if (!wait.cluster(smem_u32(&sfull[f]), f_par, 7)) { ok = false; break; }
          tc_fence_after();
          const int n = g1 - kb0 < kStep ? g1 - kb0 : kStep;
          if (are_factors(f)) {
            if (open == 0 && !accumulator_free()) { ok = false; break; }
            const uint32_t sa = tmem_base + kFactorCols + f * kFactorSlot;
            uint32_t idesc = instr_desc_mx_pair(TN) | kMajor;
            for (int j = 0; j < n; j++) {
              if (!wait(full_a + s * 8, full_par, 2)) { ok = false; break; }
              tc_fence_after();
              const uint32_t a_lo = da_lo + s * (kTile >> 4), b_lo = db_lo + s * (kTile >> 4);
#pragma unroll
              for (uint32_t ks = 0; ks < kGroup / 32; ks++)
                umma_mxf8_pair(tmem_base, da_hi | (a_lo + ks * kStepA), db_hi | (b_lo + ks * kStepB), idesc, sa, sa + 4,
                               open != 0 || j != 0 || ks != 0 ? 1u : 0u);
              umma_commit_pair_mc(empty_a + s * 8, both);
              if (++s == STAGES) { s = 0; full_par ^= 1; }
              idesc += instr_desc_mx_byte(1);
            }
            if (ok && ++open == chunk) close();
          } else {
            if (open != 0) close();
            constexpr uint32_t idesc = instr_desc_pair(kUnit, kFmtE4M3) | kMajor;
            for (int j = 0; j < n && ok; j++) {
              for (uint32_t h = 0; h < 2; h++) {
                const uint32_t unit = u < kUnits ? u : u - kUnits, before = u < kUnits ? u + kUnits : u - kUnits;      // the unit's last sum
                const uint32_t uses = u < kUnits ? u_round : u_round + 1;
                if (unit < 2 && x > 0 && !wait(smem_u32(xempty), (x & 1) ^ 1, 3)) { ok = false; break; }
                if (uses > 0 && !wait(uempty_a + before * 8, (uses & 1) ^ 1, 3)) { ok = false; break; }
                if (h == 0 && !wait(full_a + s * 8, full_par, 2)) { ok = false; break; }
                tc_fence_after();
                const uint32_t a_lo = da_lo + s * (kTile >> 4), b_lo = db_lo + s * (kTile >> 4) + h * kHalfB;
#pragma unroll
                for (uint32_t ks = 0; ks < kGroup / 32; ks++)
                  umma_f8_pair(tmem_base + unit * kUnit, da_hi | (a_lo + ks * kStepA), db_hi | (b_lo + ks * kStepB), idesc, ks != 0 ? 1u : 0u);
                umma_commit_pair_mc(ufull_a + u * 8, both);
                if (++u == kTurns) { u = 0; u_round++; }
              }
              if (!ok) break;
              umma_commit_pair_mc(empty_a + s * 8, both);
              if (++s == STAGES) { s = 0; full_par ^= 1; }
            }
          }
          if (!ok) break;
          umma_commit_pair_mc(sempty_a + f * 8, both);
          if (++f == kSlots) { f = 0; f_par ^= 1; }
        }
        if (ok && open != 0) close();
      }
      // every MMA issued so far has retired (in both CTAs) before tensor memory is released -- also after an abort
      umma_commit_pair(smem_u32(drained));
      if (!mbar_wait_quiet(drained, 0, wait.limit < kDrainPolls ? kDrainPolls : wait.limit)) {
        atomicCAS(&g_error_word, 0, 4);
        *abort_flag = 1;
      }
    }
    __syncwarp();
  } else if (warp >= kScoutWarp) {
    // =========================== scouts (both CTAs) ===========================
    // A step's scales as they arrive: whether all of them are powers of two, and their exponents into tensor memory.  (Nobody loads
    // them when they are needed: a load waits behind the copies in flight, 2 to 3 us for the 192 KB of an SM's stages.)
    const int quarter = warp - kScoutWarp;
    const uint32_t factor_at = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + kFactorCols;
    uint32_t f = 0, f_par = 0, n_looked = 0;
    bool ok = true;
    for (int64_t tile = walker; tile < n_tiles && ok; tile += walkers) {
      int64_t tm, tn;
      tile_at(tile, tiles_m, tiles_n, &tm, &tn);
      const int64_t rows = g.out.M - (tm * 2 * TM + half * TM);            // of this CTA's half tile on
      const bool second = tn * TN + kGroup < g.out.N;                      // the tile has a second block of columns
      for (int kb = g0; kb < g1; kb += kStep) {
        if (!wait(smem_u32(&scales[f]), f_par, 8)) { ok = false; break; }
        const unsigned char* slot = smem + OFF_SCALES + f * kSlotBytes;
        const int n = g1 - kb < kStep ? g1 - kb : kStep;
        constexpr uint32_t kOne = 0x3F800000u;
        bool good = true;
        uint32_t a[4], w[2] = {0, 0};
#pragma unroll
        for (int c = 0; c < 4; c++) {                                      // rows 32 c + lane
          const uint4 v = *reinterpret_cast<const uint4*>(slot + (32 * c + lane) * 16);
          const bool in = 32 * c + lane < rows;
          const uint32_t e[4] = {in ? v.x : kOne, in && n > 1 ? v.y : kOne, in && n > 2 ? v.z : kOne, in && n > 3 ? v.w : kOne};
          a[c] = 0;
#pragma unroll
          for (int j = 0; j < kStep; j++) { good &= is_factor(e[j]); a[c] |= (e[j] >> 23) << (8 * j); }
        }
#pragma unroll
        for (int b = 0; b < 2; b++)
#pragma unroll
          for (int j = 0; j < kStep; j++) {
            const uint32_t e = j < n && (b == 0 || second) ? __float_as_uint(w_scale<TRANS>(slot + kScalesA, b, j)) : kOne;
            good &= is_factor(e);
            w[b] |= (e >> 23 & 0xFFu) << (8 * j);
          }
        good = __all_sync(0xffffffffu, good);
        tc_fence_after();                                                  // the slot's last MMAs, through the scale loader's wait
        const uint32_t at = factor_at + f * kFactorSlot, w0[4] = {w[0], w[0], w[0], w[0]}, w1[4] = {w[1], w[1], w[1], w[1]};
        tmem_st4(at, a);
        tmem_st4(at + 4, w0);
        tmem_st4(at + 8, w1);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        n_looked++;
        if (lane == 0) {
          // the verdict to both CTAs, and with it that this scout's factors are written
          for (uint32_t c = 0; c < 2; c++)
            st_async_u32(mapa_rank(smem_u32(flags + f * kFlags + half * kScouts + quarter), lead + c), n_looked | (good ? 0u : kNoFactors),
                         mapa_rank(smem_u32(&sfull[f]), lead + c));
          if (quarter == 0) mbar_arrive_expect_tx(&sfull[f], kFlags * 4);
          else mbar_arrive(&sfull[f]);
        }
        __syncwarp();
        if (++f == kSlots) { f = 0; f_par ^= 1; }
      }
    }
    if (lane == 0) looked[quarter] = n_looked;
  } else if (warp < kEpilogueWarps) {
    // =========================== epilogue (both CTAs) ===========================
    reg_inc<kRegsEpilogue>();
    const int row = (warp & 3) * 32 + lane;
    const uint32_t h = warp >> 2;                // columns 64 h .. and 128 + 64 h .. of the tile
    const uint32_t tmem_at = tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const uint32_t uempty0 = mapa_rank(smem_u32(uempty), lead), xempty0 = mapa_rank(smem_u32(xempty), lead);
    unsigned char* stage = smem + OFF_OUT + warp * kStoreBytes;
    uint32_t u = h, u_par = 0;                   // barrier of this warpgroup's next partial sum: every second one is its own
    uint32_t x_par = 0, f = 0, f_par = 0;
    uint64_t acc[kRun];
    bool ok = true;
    for (int64_t tile = walker; tile < n_tiles && ok; tile += walkers) {
      int64_t tm, tn;
      tile_at(tile, tiles_m, tiles_n, &tm, &tn);
      const int64_t m0 = tm * 2 * TM + half * TM, n0 = tn * TN;
#pragma unroll
      for (int j = 0; j < kRun; j++) acc[j] = 0ull;
      int open = 0;
      const auto take_accumulator = [&] {
        if (!wait(smem_u32(xfull), x_par, 5)) return false;
        tc_fence_after();
        drain(tmem_at + 64 * h, tmem_at + 128 + 64 * h, acc, 1.0f, 1.0f, [&] {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster_read(xempty0);
        });
        x_par ^= 1;
        open = 0;
        return true;
      };
      // `open` counts as the MMA issuer's does; a full accumulator is taken at the next step or at the tile's end
      for (int kb0 = g0; kb0 < g1 && ok; kb0 += kStep) {
        if (!wait.cluster(smem_u32(&sfull[f]), f_par, 6)) { ok = false; break; }
        const bool factors = are_factors(f);
        const int n = g1 - kb0 < kStep ? g1 - kb0 : kStep;
        if (open != 0 && (!factors || open == chunk) && !take_accumulator()) { ok = false; break; }
        if (factors) {
          open++;
        } else {
          const unsigned char* slot = smem + OFF_SCALES + f * kSlotBytes;
#pragma unroll 1
          for (int j = 0; j < n; j++) {
            const float sa = *reinterpret_cast<const float*>(slot + row * 16 + j * 4);
            const float f0 = sa * w_scale<TRANS>(slot + kScalesA, 0, j), f1 = sa * w_scale<TRANS>(slot + kScalesA, 1, j);
            if (!wait(smem_u32(&ufull[u]), u_par, 5)) { ok = false; break; }
            tc_fence_after();
            const uint32_t at = tmem_at + (u < kUnits ? u : u - kUnits) * kUnit;
            drain(at, at + 64, acc, f0, f1, [&] {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive_cluster_read(uempty0 + u * 8);
            });
            u += 2;
            if (u >= kTurns) { u -= kTurns; u_par ^= 1; }
          }
          if (!ok) break;
        }
        __syncwarp();
        if (lane == 0) {
          mbar_arrive_cluster_read(mapa_rank(smem_u32(&sempty[f]), lead));
          mbar_arrive_cluster_read(mapa_rank(smem_u32(&sempty[f]), lead + 1));
        }
        if (++f == kSlots) { f = 0; f_par ^= 1; }
      }
      if (ok && open != 0 && !take_accumulator()) ok = false;
      if (!ok) break;
      if (g.parts == 1) store_tile<false>(g.out, stage, acc, m0 + (warp & 3) * 32, n0 + 64 * h, n0 + 128 + 64 * h, lane);
    }
    if (g.parts > 1) {
      // The partial sums of this CTA's only tile take the stages' place, once both warpgroups have seen their last unit: the MMAs
      // of the other one's may still read the last stage.
      asm volatile("bar.sync 1, 256;" ::: "memory");
      if (ok) stage_part<TN>(smem, acc, row, 64 * h, 128 + 64 * h);
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
    __syncwarp();
  }
  // The MMAs read the second CTA's shared memory and write its tensor memory; copies, scouts and epilogue warps signal barriers of
  // both; partial sums are read by the whole cluster.
  leave_cluster(abort_flag, 2 * g.parts, [&](uint32_t me) {
    for (uint32_t q = 0; q < kScouts; q++) {
      const uint32_t n = looked[q];
      for (uint32_t i = n > kSlots ? n - kSlots : 0; i < n; i++)
        for (uint32_t c = 0; c < 2; c++)
          wait_word(mapa_rank(smem_u32(flags + i % kSlots * kFlags + (me & 1) * kScouts + q), (me & ~1u) + c), ~kNoFactors, i + 1);
    }
    if ((me & 1) == 0) drain_pair_copies<STAGES>(full, *issued, ld_cluster_s64(mapa_rank(smem_u32(issued), me + 1)), STAGE);
  });
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc_pair(tmem_base, 512);
  }
}

// Byte matrix [rows, cols] in boxes of 128 rows x 128 bytes; zeros outside.
bool make_map(const Fp8View& v, CUtensorMap* map) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(v.K), static_cast<cuuint64_t>(v.rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(v.ld)};
  const cuuint32_t box[2] = {128, 128}, elem[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(v.codes), dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

std::atomic<int> g_resident[64][kMostParts + 1];          // per device; both instantiations take a whole SM per CTA

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
  g.parts = dev >= 0 && dev < 64 ? choose_parts(fp8_gemm_kernel<TRANS>, kThreads, kBytes, g_resident[dev], tiles, pairs, (g.groups + kStep - 1) / kStep, 2) : 1;
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

cudaError_t fp8_gemm_expire_wait(cudaStream_t stream) { return launch_wait_expiry(stream); }

cudaError_t fp8_gemm_health(int op, int* value) {
  switch (op) {
    case kHealthRead: return umma::read_error_word(value);
    case kHealthClear: return umma::clear_error_word();
    case kHealthSetSpinLimit: return umma::set_spin_limit(static_cast<uint32_t>(*value));
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace hbmm
