// Epilogue of the 8-bit operands' tensor-core products: partial sums of a run of the contraction leave tensor memory into fp32
// registers (one row per thread), finished tiles leave through shared memory in whole lines, and the parts of a tile that several
// CTA pairs of a cluster share are added over distributed shared memory in rank order (no atomics: the same sum in every run).
#pragma once
#include <atomic>
#include <cuda_bf16.h>
#include "fp8_common.cuh"
#include "umma_common.cuh"

namespace hbmm {
namespace fp8 {

using namespace umma;

// Where a product goes: [M, N] fp32 or bf16, rows on 16-byte boundaries; base (fp32, may be null) is added to an fp32 product.
struct Out {
  void* c; int64_t ldc; int32_t bf16;
  const float* base; int64_t ld_base;
  int64_t M, N;
};

// The loads of 16 columns have landed.  The registers pass through the statement, so that nothing that reads them can move above it.
__device__ __forceinline__ void tmem_ld_wait(uint32_t (&v)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]),
                 "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
               :: "memory");
}

// A thread's accumulators are two runs of 64 columns of its row, two columns per register pair.
constexpr int kRun = 64;

// acc += f0 * D for the run at at0 and f1 * D for the run at at1; 16 columns load while the ones before are added.  release() runs
// once all of them are in registers.
template <typename Release>
__device__ __forceinline__ void drain(uint32_t at0, uint32_t at1, uint64_t (&acc)[kRun], float f0, float f1, Release release) {
  uint32_t d[2][16];
  const uint64_t ff[2] = {pack2(__float_as_uint(f0), __float_as_uint(f0)), pack2(__float_as_uint(f1), __float_as_uint(f1))};
  tmem_ld16(at0, d[0]);
  tmem_ld_wait(d[0]);
#pragma unroll
  for (int c = 0; c < 8; c++) {
    if (c + 1 < 8) tmem_ld16((c + 1 < 4 ? at0 : at1) + ((c + 1) % 4) * 16, d[(c + 1) & 1]);
    else release();
#pragma unroll
    for (int j = 0; j < 16; j += 2) acc[c * 8 + j / 2] = fma2(ff[c / 4], pack2(d[c & 1][j], d[c & 1][j + 1]), acc[c * 8 + j / 2]);
    if (c + 1 < 8) tmem_ld_wait(d[(c + 1) & 1]);
  }
}

// Four consecutive outputs (column n a multiple of four) to their row, as the row's end allows.
__device__ __forceinline__ void store_out4(const Out& o, int64_t m, int64_t n, float4 v) {
  if (m >= o.M || n >= o.N) return;
  const bool whole = n + 4 <= o.N;
  if (o.bf16) {
    __nv_bfloat16* p = static_cast<__nv_bfloat16*>(o.c) + m * o.ldc + n;
    if (whole) {
      *reinterpret_cast<uint2*>(p) = make_uint2(bf16x2(v.x, v.y), bf16x2(v.z, v.w));
      return;
    }
    const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 3; i++)
      if (n + i < o.N) p[i] = __float2bfloat16_rn(e[i]);
    return;
  }
  float* p = static_cast<float*>(o.c) + m * o.ldc + n;
  if (o.base) {
    const float* b = o.base + m * o.ld_base + n;
    if (whole) {
      const uint4 q = load16(b);
      v.x += __uint_as_float(q.x); v.y += __uint_as_float(q.y); v.z += __uint_as_float(q.z); v.w += __uint_as_float(q.w);
    } else {
      v.x += loadf(b);
      if (n + 1 < o.N) v.y += loadf(b + 1);
      if (n + 2 < o.N) v.z += loadf(b + 2);
    }
  }
  if (whole) { *reinterpret_cast<float4*>(p) = v; return; }
  p[0] = v.x;
  if (n + 1 < o.N) p[1] = v.y;
  if (n + 2 < o.N) p[2] = v.z;
}

// A warp's 32 rows (row m0 + lane in this lane's registers) of the runs at columns n0 and n1 to memory through shared memory: lanes write
// their own rows and read the rows of a store instruction side by side.  Pieces of 16 bytes lie where neither conflicts.
//   narrow: eight rows of 64 bytes at a time, 16 columns in fp32, 32 in bf16 (rounded on the way in);
//   wide (fp32): 16 rows at a time, four rows of whole 128-byte lines per store, and the base, if any, half a step ahead of its use.
//   (blocks that lie inside the matrix only: with a check per piece 256 x 4096 x 9216 outputs took 82 us instead of 45).
// Elsewhere rows and columns that the matrix lacks are skipped piece by piece; a piece that it ends in goes element by element.
constexpr int kStoreBytes = 2048;             // per warp
__device__ __forceinline__ unsigned char* store_piece(unsigned char* stage, int row, int piece) { return stage + row * 64 + ((piece ^ (row >> 1 & 3)) << 4); }
// The base's lines of a warp's 32 rows x 128 columns into L2, some time before store_tile reads them.
__device__ __forceinline__ void prefetch_base(const Out& o, int64_t m0, int64_t n0, int lane) {
  if (!o.base || m0 + lane >= o.M) return;
#pragma unroll
  for (int c = 0; c < 4; c++)
    if (n0 + c * 32 < o.N) asm volatile("prefetch.global.L2 [%0];" ::"l"(o.base + (m0 + lane) * o.ld_base + n0 + c * 32));
}
template <bool WIDE>
__device__ __forceinline__ void store_tile(const Out& o, unsigned char* stage, const uint64_t (&acc)[kRun], int64_t m0, int64_t n0, int64_t n1, int lane) {
  if (m0 >= o.M) return;
  const int rows = o.M - m0 < 32 ? static_cast<int>(o.M - m0) : 32;
  const auto left = [&](int64_t n) { return o.N - n < 64 ? static_cast<int>(o.N - n) : 64; };       // columns from n on, 0 or less: none
  const auto words = [&](int j) {                       // four consecutive columns of this lane's row, raw
    return make_uint4(static_cast<uint32_t>(acc[j]), static_cast<uint32_t>(acc[j] >> 32), static_cast<uint32_t>(acc[j + 1]), static_cast<uint32_t>(acc[j + 1] >> 32));
  };
  if (WIDE && rows == 32 && n0 + kRun <= o.N && n1 + kRun <= o.N) {
    const int sub = lane / 8, piece = lane % 8;
    const int64_t r0 = m0 + sub;
    float* out = static_cast<float*>(o.c) + r0 * o.ldc + n0 + piece * 4;
    const bool base = o.base != nullptr;
    const float* from = base ? o.base + r0 * o.ld_base + n0 + piece * 4 : nullptr;
    uint4 ahead[4];
    if (base) {
#pragma unroll
      for (int i = 0; i < 4; i++) ahead[i] = load16(from + i * 4 * o.ld_base);
    }
#pragma unroll
    for (int c = 0; c < 4; c++) {
      const int64_t on = c == 1 ? n1 - n0 - 32 : 32;
#pragma unroll
      for (int hf = 0; hf < 2; hf++) {                  // 16 of the rows at a time
        __syncwarp();
        if (lane / 16 == hf) {
#pragma unroll
          for (int p = 0; p < 8; p++) *reinterpret_cast<uint4*>(swz(stage, lane % 16, p)) = words(c * 16 + 2 * p);
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 4; i++) {
          float4 v = *reinterpret_cast<const float4*>(swz(stage, i * 4 + sub, piece));
          if (base) {
            v.x += __uint_as_float(ahead[i].x); v.y += __uint_as_float(ahead[i].y);
            v.z += __uint_as_float(ahead[i].z); v.w += __uint_as_float(ahead[i].w);
          }
          *reinterpret_cast<float4*>(out + (hf * 4 + i) * 4 * o.ldc) = v;
        }
        if (base && (c < 3 || hf == 0)) {
          if (hf == 1) from += on;
#pragma unroll
          for (int i = 0; i < 4; i++) ahead[i] = load16(from + ((1 - hf) * 4 + i) * 4 * o.ld_base);
        }
      }
      out += on;
    }
    return;
  }
  const int sub = lane / 4, piece = lane % 4;
  const int64_t r0 = m0 + sub;
  if (!WIDE && o.bf16) {                                // 32 columns at a time, rounded on the way in
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(o.c) + r0 * o.ldc + n0 + piece * 8;
#pragma unroll
    for (int c = 0; c < 4; c++) {
      const int64_t n = (c < 2 ? n0 : n1) + c % 2 * 32;
      __syncwarp();
#pragma unroll
      for (int p = 0; p < 4; p++) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; e++) {
          float lo, hi;
          unpack2(acc[c * 16 + p * 4 + e], lo, hi);
          w[e] = bf16x2(lo, hi);
        }
        *reinterpret_cast<uint4*>(store_piece(stage, lane, p)) = make_uint4(w[0], w[1], w[2], w[3]);
      }
      __syncwarp();
      const int cols = left(n + piece * 8);
#pragma unroll
      for (int i = 0; i < 4; i++) {
        if (i * 8 + sub >= rows) continue;
        const uint4 v = *reinterpret_cast<const uint4*>(store_piece(stage, i * 8 + sub, piece));
        __nv_bfloat16* to = out + i * 8 * o.ldc;
        if (cols >= 8) {
          *reinterpret_cast<uint4*>(to) = v;
        } else {
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int e = 0; e < 7; e++)
            if (e < cols) reinterpret_cast<unsigned short*>(to)[e] = static_cast<unsigned short>(w[e / 2] >> (16 * (e % 2)));
        }
      }
      out += c == 1 ? n1 - n0 - 32 : 32;
    }
    return;
  }
  float* out = static_cast<float*>(o.c) + r0 * o.ldc + n0 + piece * 4;
#pragma unroll
  for (int c = 0; c < 8; c++) {
    const int64_t n = (c < 4 ? n0 : n1) + c % 4 * 16;
    __syncwarp();                                       // the columns before have been read
#pragma unroll
    for (int p = 0; p < 4; p++) *reinterpret_cast<uint4*>(store_piece(stage, lane, p)) = words(c * 8 + 2 * p);
    __syncwarp();
    const int cols = left(n + piece * 4);
#pragma unroll
    for (int i = 0; i < 4; i++) {
      if (i * 8 + sub >= rows) continue;
      const float4 v = *reinterpret_cast<const float4*>(store_piece(stage, i * 8 + sub, piece));
      if (cols >= 4 && !(WIDE && o.base)) *reinterpret_cast<float4*>(out + i * 8 * o.ldc) = v;
      else if (cols > 0) store_out4(o, r0 + i * 8, n + piece * 4, v);
    }
    out += c == 3 ? n1 - n0 - kRun + 16 : 16;
  }
}

// ---- tiles shared by several CTAs of a cluster
constexpr int kMostParts = 4;                 // pairs of a cluster that may share a tile
// The 16-byte piece u of a row of TN fp32 partial sums.
template <int TN>
__device__ __forceinline__ int part_offset(int row, int u) { return row * (TN * 4) + ((u ^ (row & 7)) << 4); }

// A thread's runs at columns c0 and c1 of the tile.
template <int TN>
__device__ __forceinline__ void stage_part(unsigned char* base, const uint64_t (&acc)[kRun], int row, int c0, int c1) {
#pragma unroll
  for (int p = 0; p < 32; p++) {
    float v[4];
    unpack2(acc[2 * p], v[0], v[1]);
    unpack2(acc[2 * p + 1], v[2], v[3]);
    *reinterpret_cast<float4*>(base + part_offset<TN>(row, (p < 16 ? c0 : c1) / 4 + p % 16)) = make_float4(v[0], v[1], v[2], v[3]);
  }
}
__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.volatile.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ int64_t ld_cluster_s64(uint32_t addr) {
  int64_t v;
  asm volatile("ld.volatile.shared::cluster.s64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void st_cluster_u32(uint32_t addr, uint32_t v) {
  asm volatile("st.volatile.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ float4 ld_cluster16(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}
// This CTA's share (part `mine` of `parts`) of the 128 rows of a tile whose partial sums lie in the CTAs `rank0`, `rank0` + 2, ...
template <int TN>
__device__ __forceinline__ void finish_parts(const Out& o, unsigned char* base, int mine, int parts, uint32_t rank0, int64_t m0, int64_t n0, int tid,
                                             int threads) {
  const int r0 = mine * TM / parts, r1 = (mine + 1) * TM / parts;
  for (int i = tid; i < (r1 - r0) * (TN / 4); i += threads) {
    const int row = r0 + i / (TN / 4), u = i % (TN / 4);
    if (m0 + row >= o.M || n0 + 4 * u >= o.N) continue;
    const uint32_t at = smem_u32(base + part_offset<TN>(row, u));
    float4 v[kMostParts];
#pragma unroll
    for (int q = 0; q < kMostParts; q++)
      if (q < parts) v[q] = ld_cluster16(mapa_rank(at, rank0 + 2 * q));
    float4 sum = v[0];
#pragma unroll
    for (int q = 1; q < kMostParts; q++)
      if (q < parts) { sum.x += v[q].x; sum.y += v[q].y; sum.z += v[q].z; sum.w += v[q].w; }
    store_out4(o, m0 + row, n0 + 4 * u, sum);
  }
}

// How many pairs (one cluster) share a tile: as many, up to four, as leave every tile's cluster resident at once (a B200 with 74 pairs
// holds 33 clusters of two, 22 of three and 15 of four pairs of such CTAs; 16 tiles in clusters of four took twice the time of one
// turn) and each at least `least` of a tile's `units` of the contraction.  known: what the device answered before, plus one; a
// failure is not kept and costs this call the split.
template <typename Kernel>
int choose_parts(Kernel kernel, int threads, int bytes, std::atomic<int> (&known)[kMostParts + 1], int64_t tiles, int64_t pairs, int units, int least) {
  for (int parts = kMostParts; parts >= 2; parts--) {
    if (tiles * parts > pairs || units < parts * least) continue;
    int n = known[parts].load(std::memory_order_relaxed);
    if (n == 0) {
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3(static_cast<unsigned>(2 * parts * pairs));
      cfg.blockDim = dim3(static_cast<unsigned>(threads));
      cfg.dynamicSmemBytes = static_cast<size_t>(bytes);
      cudaLaunchAttribute attr[1];
      attr[0].id = cudaLaunchAttributeClusterDimension;
      attr[0].val.clusterDim.x = static_cast<unsigned>(2 * parts);
      attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
      cfg.attrs = attr;
      cfg.numAttrs = 1;
      int clusters = 0;
      if (cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg) != cudaSuccess) {
        cudaGetLastError();                             // this answer's failure is not the launch's
        continue;
      }
      n = clusters + 1;
      known[parts].store(n, std::memory_order_relaxed);
    }
    if (tiles <= n - 1) return parts;
  }
  return 1;
}

// ---- the end of a kernel
// Returns when no CTA of the cluster reaches into this one any more; every thread of every CTA comes here behind its role.  Where a
// wait gave up in one of them, copies and announcements may still be on their way: drain, which every CTA's first thread then runs
// while all of them are there, waits for those of its CTA, whose number it knows by then (each wait bounded as the others).
template <typename Drain>
__device__ __forceinline__ void leave_cluster(volatile int* abort_flag, uint32_t ctas, Drain drain) {
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (*abort_flag != 0 && threadIdx.x < ctas) st_cluster_u32(mapa_rank(smem_u32(const_cast<int*>(abort_flag)), threadIdx.x), 1u);
  __syncwarp();
  cluster_sync_all();
  if (*abort_flag != 0) {                               // the same in every CTA
    if (threadIdx.x == 0) drain(cluster_ctarank());     // read again: kept from the start it costs registers that spill
    __syncwarp();
    __syncthreads();
    cluster_sync_all();
  }
}
// Copies that both CTAs of a pair issue, STAGES ahead at most, complete on the first one's barriers, `bytes` from each and one arrival,
// which expects both.  The first CTA waits for the last of them: issued and other are the copies of the two.
template <int STAGES>
__device__ __forceinline__ void drain_pair_copies(uint64_t* full, int64_t issued, int64_t other, uint32_t bytes) {
  const int64_t last = issued > other ? issued : other;
  for (int64_t i = last > STAGES ? last - STAGES : 0; i < last; i++) {
    uint64_t* bar = &full[i % STAGES];
    if (i >= issued) mbar_arrive_expect_tx(bar, bytes);              // the other CTA went further
    else if (i >= other) mbar_complete_tx(bar, bytes);               // this one did
    mbar_wait_quiet(bar, static_cast<uint32_t>((i / STAGES) & 1), kDrainPolls);
  }
}
// A word that st_async_u32 is bringing to this address of the cluster (where the kernel wrote another one at its start).
__device__ __forceinline__ void wait_word(uint32_t cluster_addr, uint32_t mask, uint32_t value) {
  for (uint32_t it = 0; it < kDrainPolls; it++)
    if ((ld_cluster_u32(cluster_addr) & mask) == value) return;
}

// Test only: a thread each in two blocks waits, in the two ways that the kernels' roles do, on a barrier that nobody arrives at and
// that guards nothing (no copy, no MMA in flight).  The waits run out after the limit in force and record code 9.
static __global__ void wait_expiry_kernel() {
  __shared__ uint64_t bar;
  __shared__ int flag;
  if (threadIdx.x != 0) return;
  mbar_init(&bar, 1);
  flag = 0;
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  const Waiter wait{g_spin_limit, &flag};
  if (blockIdx.x == 0) wait(smem_u32(&bar), 0, 9);
  else wait.cluster(smem_u32(&bar), 0, 9);
}
static inline cudaError_t launch_wait_expiry(cudaStream_t stream) {
  wait_expiry_kernel<<<2, 32, 0, stream>>>();
  return cudaGetLastError();
}

// Output tiles are walked in blocks of eight rows of tiles, column by column, so that the tiles in flight at one time cover about as
// many rows of one operand as of the other (fewest bytes read for the products of a wave).
__device__ __forceinline__ void tile_at(int64_t i, int64_t tiles_m, int64_t tiles_n, int64_t* tm, int64_t* tn) {
  constexpr int64_t kRows = 8;
  const int64_t block = i / (kRows * tiles_n), in = i - block * (kRows * tiles_n);
  const int64_t rows = tiles_m - block * kRows < kRows ? tiles_m - block * kRows : kRows;
  *tn = in / rows;
  *tm = block * kRows + (in - *tn * rows);
}

}  // namespace fp8
}  // namespace hbmm
