// Expert products on 4-bit microscaled operands: tcgen05.mma kind::mxf4 with a scale per block of 32, over groups of rows of any length.
//
//   C[r, :] = act(A[r, :] . B[e]^T + bias[e]),  offsets[e] <= r < offsets[e + 1]
//
// The weights' columns (rows of B[e]) are the 128 rows of an MMA and NT rows of A its columns, at every size: a tile of few rows of A is
// then a narrow MMA with nothing computed on fill, and one kernel serves one token and thousands.  A lane of tensor memory is a column
// of C, a column of it a row.
//
// Per CTA (persistent, one per SM):
//   warp 0       TMA: stages of 256 of the contraction, 128 x 128 bytes of B and NT x 128 bytes of A, and their scales, 1024 of the
//                contraction (32 bytes of a row's scales) at a time
//   warp 1       the MMAs, 64 of the contraction each
//   warps 2-13   epilogue, three for each quarter of tensor memory's lanes
//   warps 14-17  scales: a stage's from shared through registers into tensor memory, where every quarter of the lanes wants its own
//                copy: row 32 c + l of a tile in lane l, column c, four blocks' bytes to a column.  Rows start anywhere, so no
//                prepared layout could serve them.
// Few rows leave few tiles: then a cluster of CTAs shares each (SPLIT), each a stretch of the contraction, and the first adds up the others'
// accumulators, which they write into its shared memory, in the order of the stretches.
// MT = 2: two MMAs side by side, 256 columns of C, for long contractions (see wide()); the one accumulator's halves are handed over one by one
// (32768 rows, 4096 x 16384, at the power cap: 1432 us, both at once 1471).
// What bounds it: few rows, the reading of the weights (64 experts of 4096 x 16384, 32 rows each, 377 us, 92 % of the copy rate; eight rows of eight
// experts 51 us, 84 %, of which 8 us do not grow with the experts: a call without rows takes 2, one with a single tile 10); many
// rows, the issuing warps and the 54 bytes a clock an SM receives from L2, then the board's 1000 W (32768 rows: 1190 to 1330 us
// alone, 1430 in a loop, 3.0 to 3.7 PFLOP/s); short contractions, the epilogue (16384 rows, 768 x 2048, bf16 results 31 us, with GeLU 53, of which
// 17 are the multiply-adds of the polynomial at full rate; to 4 bits 46, with GeLU 65).
// Two accumulators of NT columns, and as many buffers of scales as there are stages: a stage is full when its operands have landed and
// its scales are in tensor memory, and one commit frees both.  (A wait that is over at once still takes the MMA warp 100 cycles, a commit
// 60 to 100, issuing an MMA 80: with barriers of their own for the scales a stage took 815 cycles beside the MMAs' 384.)
#include "../../include/ecmoe.h"
#include "gelu.cuh"
#include "internal.h"
#include "mx.cuh"
#include "tc_ptx.cuh"

#include <cudaTypedefs.h>
#include <math.h>
#include <string.h>

namespace ecmoe {

namespace {

constexpr int kM = 128;                              // columns of C per tile
constexpr int kStageK = 256, kRowBytes = kStageK / 2;
constexpr int kBBytes = kM * kRowBytes;              // 16 KiB
constexpr int kEpi = 12, kScaleWarps = 4;
constexpr int kChunk = 16;                           // rows an epilogue warp takes at a time
constexpr int kThreads = 32 * (2 + kEpi + kScaleWarps);
constexpr int kMaxE = 256;
constexpr int kTmemCols = 512;
constexpr int kScaleStages = 2, kScaleStageK = 1024, kScaleRow = kScaleStageK / 32;
constexpr int kSmemBudget = 221 * 1024;

// mt: MMAs side by side, 128 columns of C each
__host__ __device__ constexpr int stage_bytes(int nt, int mt) { return mt * kBBytes + nt * kRowBytes; }
__host__ __device__ constexpr int scale_stage_bytes(int nt, int mt) { return (mt * kM + nt) * kScaleRow; }
// Most CTAs to a tile, and what the first of them keeps for the others' accumulators
__host__ __device__ constexpr int most_split(int nt) { return nt == 32 ? 4 : nt == 64 ? 2 : 1; }
__host__ __device__ constexpr int parts_bytes(int nt, bool split) { return split ? (most_split(nt) - 1) * kM * nt * 4 : 0; }
__host__ __device__ constexpr int stages_of(int nt, bool split, int mt) {
  const int fit = (kSmemBudget - parts_bytes(nt, split) - kScaleStages * scale_stage_bytes(nt, mt)) / stage_bytes(nt, mt);
  return fit > 10 ? 10 : fit;
}
// Columns of tensor memory for 128 of the contraction of A's scales, and for a stage's of both.  tcgen05.mma wants a scale matrix to begin
// at a multiple of four columns, so narrow tiles leave some of the four unused.
__host__ __device__ constexpr int cols_a(int nt) { return nt <= 128 ? 4 : 8; }
__host__ __device__ constexpr int scale_cols(int nt, int mt) { return 8 * mt + 2 * cols_a(nt); }

// TMA boxes a stage's rows of A come in
__host__ __device__ constexpr int boxes_of(int nt) { return nt >= 128 ? 2 : 1; }

struct MxParams {
  int64_t rows;
  int N, E, tiles_m, blocks, kblocks;                // blocks: of 32 along the contraction; kblocks: stages of 256
  int act, split;                                    // split: CTAs to a tile
  const int32_t* offsets;
  const void* bias; int bias_f32;
  void* c; uint8_t* c_scales; int64_t c_pitch, c_scale_pitch;     // c_pitch in bytes
  int* status;
#ifdef EC_DEBUG
  int silent;                                        // see ec_debug_mx_wait
#endif
};

enum { OUT_F32 = 0, OUT_BF16 = 1, OUT_MX = 2 };

// The TMA and the MMA warp run as whole warps with the same values in every lane, and one lane, chosen once, carries out what must be done
// once: the compiler then keeps descriptors, addresses and loop counters in uniform registers, where these instructions want them.
// (Inside `if (lane == 0)` every operand is moved there before each instruction: 430 cycles to issue four MMAs of 96.)
__device__ __forceinline__ uint32_t elect_one() {
  uint32_t r;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(r));
  return r;
}
// Clears `alive` when the wait runs out or another role has given up; what the caller then does up to its loop's end it does with its
// lead taken away.  Every lane polls, and none goes on before all have seen the barrier: an elected lane that ran ahead could let
// the barrier pass through the phase that a slower lane still waits for.  (32768 rows, 4096 x 16384: 1443 us with and without the
// __syncwarp(), 1451 with votes on what the lanes have seen.)
__device__ __forceinline__ void wait(uint32_t& alive, uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status, int where) {
  if (alive && !mbar_try(bar, parity)) alive = mbar_wait(bar, parity, abort_flag, status, kStatusStays | where);
  __syncwarp();
}
__device__ __forceinline__ void expect_tx_if(uint32_t lead, uint32_t bar, uint32_t bytes) {
  asm volatile("{\n .reg .pred q;\n setp.ne.b32 q, %2, 0;\n @q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n}\n" ::"r"(bar), "r"(bytes), "r"(lead) : "memory");
}
__device__ __forceinline__ void tma_load_2d_if(uint32_t lead, uint32_t dst, const CUtensorMap* tm, uint32_t bar, int c0, int c1) {
  asm volatile("{\n .reg .pred q;\n setp.ne.b32 q, %5, 0;\n"
               " @q cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];\n}\n"
               ::"r"(dst), "l"(tm), "r"(bar), "r"(c0), "r"(c1), "r"(lead) : "memory");
}
__device__ __forceinline__ void tma_load_3d_if(uint32_t lead, uint32_t dst, const CUtensorMap* tm, uint32_t bar, int c0, int c1, int c2) {
  asm volatile("{\n .reg .pred q;\n setp.ne.b32 q, %6, 0;\n"
               " @q cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];\n}\n"
               ::"r"(dst), "l"(tm), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(lead) : "memory");
}
__device__ __forceinline__ void tc_commit_if(uint32_t lead, uint32_t bar) {
  asm volatile("{\n .reg .pred q;\n setp.ne.b32 q, %1, 0;\n @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n"
               ::"r"(bar), "r"(lead) : "memory");
}
// Descriptors by their lower words (address and leading offset); the upper one is that of make_desc(., 16, 1024).
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_low(uint32_t saddr) { return ((saddr & 0x3FFFFu) >> 4) | (1u << 16); }
__device__ __forceinline__ void tc_mma_mx_if(uint32_t lead, uint32_t d, uint32_t alow, uint32_t blow, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
  asm volatile("{\n .reg .pred p, q;\n .reg .b64 a, b;\n mov.b64 a, {%1, %8};\n mov.b64 b, {%2, %8};\n setp.ne.b32 p, %6, 0;\n setp.ne.b32 q, %7, 0;\n"
               " @q tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], a, b, %3, [%4], [%5], p;\n}\n"
               ::"r"(d), "r"(alow), "r"(blow), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate), "r"(lead), "n"(kDescHigh) : "memory");
}
// What another CTA of the cluster wrote before it arrived: acquire at the cluster's scope.  Gives up like mbar_wait.
__device__ __forceinline__ bool cluster_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status, int where, int lane) {
  bool ok = true;
  if (lane == 0) {
    auto done = [&] {
      uint32_t r;
      asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
                   : "=r"(r) : "r"(bar), "r"(parity) : "memory");
      return r != 0;
    };
    if (!done()) {
      const unsigned long long t0 = globaltimer();
      for (uint32_t spin = 1; !done(); ++spin) {
        if ((spin & 63u) != 0) continue;
        if (*abort_flag) { ok = false; break; }
        if (globaltimer() - t0 > kWaitNs) {
          *abort_flag = 1;
          atomicExch(status + 1, kStatusStays | where); atomicExch(status, EC_ERR_TIMEOUT);
          ok = false;
          break;
        }
      }
    }
  }
  ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
  __syncwarp();                                      // what the lane has seen the others see
  return ok;
}
__device__ __forceinline__ void st_cluster4(uint32_t addr, const float* v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]) : "memory");
}
// A warp's wait with an answer: one lane polls.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status, int where, int lane) {
  bool ok = true;
  if (lane == 0) ok = mbar_wait(bar, parity, abort_flag, status, kStatusStays | where);
  ok = __shfl_sync(0xffffffffu, (int)ok, 0) != 0;
  __syncwarp();                                      // what the lane has seen the others see
  return ok;
}
__device__ __forceinline__ void tc_st8(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ void tc_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// GeLU of a pair, z Phi(z).  erf(u) = u Q(t) with t = 2 u^2 / U^2 - 1, U = 3.8 (erf(3.8) = 1 - 8e-8), Q the degree-14 polynomial through the
// Chebyshev nodes in t of erf(u) / u (fitted for this file; coefficients of the powers of t, all below 1/2, so Horner's rule is stable).
// |error| < 2.6e-7 |z| in fp32, a third of the instructions of erff; below -U sqrt 2 z counts as that, NaN stays NaN.  Phi is held in [0, 1]
// (by the instruction that adds its half), so that in the tail, where the error is as large as the value, the sign is still z's.
__device__ __forceinline__ void gelu_erf2(float& z0, float& z1) {
  constexpr float U = 3.8f, Z = -5.374011538f;
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(z0) : "f"(Z)); asm("max.NaN.f32 %0, %0, %1;" : "+f"(z1) : "f"(Z));
  const unsigned long long z = pk2(z0, z1), u = mul2(z, pk2(0.70710678118654752f, 0.70710678118654752f));
  const unsigned long long uc = pk2(fminf(lo2(u), U), fminf(hi2(u), U));
  const unsigned long long t = fma2(mul2(uc, uc), pk2(2.f / (U * U), 2.f / (U * U)), pk2(-1.f, -1.f));
  constexpr float c[15] = {3.721076250e-01f, -1.856413633e-01f, 1.377403885e-01f, -1.111800969e-01f, 9.081587195e-02f,
                           -7.256521285e-02f, 5.517497286e-02f, -3.874899447e-02f, 2.630480193e-02f, -1.868470572e-02f,
                           1.059229579e-02f, -2.991377143e-03f, 1.846335013e-03f, -2.798850415e-03f, 1.186226029e-03f};
  unsigned long long acc = pk2(c[14], c[14]);
#pragma unroll
  for (int i = 13; i >= 0; --i) acc = fma2(acc, t, pk2(c[i], c[i]));
  const unsigned long long erf = mul2(uc, acc);
  const unsigned long long h = mul2(z, pk2(__saturatef(fmaf(lo2(erf), 0.5f, 0.5f)), __saturatef(fmaf(hi2(erf), 0.5f, 0.5f))));
  z0 = lo2(h); z1 = hi2(h);
}

// The experts that have rows, in shared memory.  Tiles run expert by expert, inside one along its row tiles first: those that run at the
// same time share weights.
struct Groups {
  int expert[kMaxE], lo[kMaxE], count[kMaxE];        // their rows
  int first[kMaxE + 1];                              // row tiles before each, and all of them
  int active, total;                                 // experts; tiles in all
};
// Where a tile lies.  A whole warp asks, for tiles in ascending order: it looks at 32 experts at a time (one at a time, a step of 148 tiles over
// 18 experts took 2500 cycles).
template <int NT>
struct Walk {
  const Groups* g; int tiles_m, lane;
  int i;                                             // the expert's number in the list
  int e, m, row0, rows;                              // the tile at hand
  __device__ __forceinline__ Walk(const Groups* groups, int m, int l) : g(groups), tiles_m(m), lane(l), i(0) {}
  __device__ __forceinline__ void to(int tile) {
    for (;;) {
      const int at = i + 1 + lane, past = __popc(__ballot_sync(0xffffffffu, at < g->active && g->first[at] * tiles_m <= tile));
      i += past;
      if (past < 32) break;
    }
    const int before = g->first[i], n = g->first[i + 1] - before, left = tile - before * tiles_m;
    m = (int)((float)left * __frcp_rn((float)n));    // one off at most: a correction either way
    int t = left - m * n;
    if (t < 0) { --m; t += n; } else if (t >= n) { ++m; t -= n; }
    e = g->expert[i]; row0 = g->lo[i] + t * NT; rows = min(NT, g->count[i] - t * NT);
  }
};

template <int NT, int OUT, bool SPLIT, int MT>
__global__ void __launch_bounds__(kThreads, 1)
gemm_mx_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmAs,
               const __grid_constant__ CUtensorMap tmBs, const MxParams p) {
  constexpr int S = stages_of(NT, SPLIT, MT), kStage = stage_bytes(NT, MT), kScaleStage = scale_stage_bytes(NT, MT);
  constexpr int kTileM = MT * kM, kAt = MT * kBBytes, kBuffers = MT == 1 ? 2 : 1;    // A behind B in a stage; accumulators
  constexpr int kBoxes = boxes_of(NT), kBoxBytes = NT / kBoxes * kRowBytes;
  constexpr int kColsA = cols_a(NT), kScaleCols = scale_cols(NT, MT), kScales0 = kBuffers * MT * NT;
  static_assert(kScales0 + S * kScaleCols <= kTmemCols, "tensor memory");
  static_assert(kScales0 % 4 == 0 && kScaleCols % 4 == 0 && kColsA % 4 == 0, "where a scale matrix may begin");
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  // barriers: full[S], empty[S], of the accumulators full[2], empty[2] (MT = 2: of its halves), of the scales in shared memory the same
  // and, of the parts of a split tile, full and empty
  uint64_t* bars = (uint64_t*)(smem + S * kStage + kScaleStages * kScaleStage + parts_bytes(NT, SPLIT));
  uint32_t* tmem_slot = (uint32_t*)(bars + 2 * S + 6 + 2 * kScaleStages);
  volatile int* abort_flag = (volatile int*)(tmem_slot + 1);
  Groups* groups = (Groups*)(tmem_slot + 2);
  const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * S, accf0 = empty0 + 8 * S, acce0 = accf0 + 16;
  const uint32_t ssf0 = acce0 + 16, sse0 = ssf0 + 8 * kScaleStages, partf = sse0 + 8 * kScaleStages, parte = partf + 8;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // a cluster's CTAs take the same tiles, each a stretch of whole scale stages of the contraction
  const int ctas = SPLIT ? p.split : 1, rank = SPLIT ? (int)blockIdx.x % ctas : 0;
  const int first_tile = SPLIT ? blockIdx.x / ctas : blockIdx.x, tile_step = SPLIT ? gridDim.x / ctas : gridDim.x;
  constexpr int kUnit = kScaleStageK / kStageK;
  const int units = (p.kblocks + kUnit - 1) / kUnit;
  const int kb0 = SPLIT ? units * rank / ctas * kUnit : 0, kb1 = SPLIT ? min(units * (rank + 1) / ctas * kUnit, p.kblocks) : p.kblocks;

  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) { mbar_init(full0 + 8 * s, 1 + kScaleWarps); mbar_init(empty0 + 8 * s, 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(accf0 + 8 * b, 1); mbar_init(acce0 + 8 * b, kEpi); }
    for (int b = 0; b < kScaleStages; ++b) { mbar_init(ssf0 + 8 * b, 1); mbar_init(sse0 + 8 * b, kScaleWarps); }
    if constexpr (SPLIT) { mbar_init(partf, (ctas - 1) * kEpi); mbar_init(parte, kEpi); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (threadIdx.x == 32 * 2) { prefetch_map(&tmA); prefetch_map(&tmB); prefetch_map(&tmAs); prefetch_map(&tmBs); }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  if constexpr (SPLIT) cluster_sync_all();           // the others' barriers exist before anything is sent to them
  tc_fence_after();
  chain_enter();
  const uint32_t tmem_base = *tmem_slot, smem_base = smem_u32(smem), scale_base = smem_base + S * kStage;
  // The first CTA clears the status word; another writes it two seconds into a wait at the earliest.
  if (blockIdx.x == 0 && threadIdx.x == 0) begin_status(p.status);
  // The groups: offsets are the caller's memory, whatever they hold becomes rows inside [0, rows) that no two groups share, so there are
  // no more tiles than the host counted and a row has one writer.
  if (warp == 0) {
    const int32_t* offsets = after_enter(p.offsets);
    int from[kMaxE / 32], to[kMaxE / 32], active = 0, total = 0;
#pragma unroll
    for (int i = 0; i < kMaxE / 32; ++i) {           // all of them under way at once: this is before the first load of a tile
      const int e = 32 * i + lane;
      from[i] = e < p.E ? __ldg(offsets + e) : 0;
      to[i] = e < p.E ? __ldg(offsets + e + 1) : 0;
    }
    bool falls = false;
#pragma unroll
    for (int i = 0; i < kMaxE / 32; ++i) {
      from[i] = min(max(from[i], 0), (int)p.rows); to[i] = min(max(to[i], 0), (int)p.rows);
      falls |= to[i] < from[i];
    }
    if (__any_sync(0xffffffffu, falls)) {            // an offset counts as the largest up to it
      int most = 0;
#pragma unroll
      for (int i = 0; i < kMaxE / 32; ++i) {
#pragma unroll
        for (int o = 1; o < 32; o *= 2) { const int v = __shfl_up_sync(0xffffffffu, from[i], o); if (lane >= o) from[i] = max(from[i], v); }
        from[i] = max(from[i], most); to[i] = max(to[i], from[i]);
        most = __shfl_sync(0xffffffffu, to[i], 31);
      }
    }
#pragma unroll
    for (int i = 0; i < kMaxE / 32; ++i) {
      if (32 * i >= p.E) break;
      const int e = 32 * i + lane, lo = from[i], count = to[i] - lo;
      const unsigned some = __ballot_sync(0xffffffffu, count > 0);
      const int tiles = (count + NT - 1) / NT;
      int before = tiles;                            // of the lanes up to this one
#pragma unroll
      for (int o = 1; o < 32; o *= 2) { const int v = __shfl_up_sync(0xffffffffu, before, o); if (lane >= o) before += v; }
      if (count > 0) {
        const int at = active + __popc(some & ((1u << lane) - 1));
        groups->expert[at] = e; groups->lo[at] = lo; groups->count[at] = count; groups->first[at] = total + before - tiles;
      }
      active += __popc(some);
      total += __shfl_sync(0xffffffffu, before, 31);
    }
    if (lane == 0) { groups->active = active; groups->first[active] = total; groups->total = total * p.tiles_m; }
  }
  __syncthreads();
  const int total = __shfl_sync(0xffffffffu, groups->total, 0);
  bool gave_up = tmem_base != 0;                     // cannot happen with all 512 columns taken; refuse rather than corrupt
  if (gave_up && threadIdx.x == 0) { atomicExch(p.status + 1, kStatusStays | 9); atomicExch(p.status, EC_ERR_TIMEOUT); }

  if (gave_up) {
    // nothing: fall through to the exit
  } else if (warp == 0) {
    // ------------------------------------------------------------------ TMA
    const uint32_t elected = elect_one();
    uint32_t stage = 0, phase = 0, scale_stage = 0, scale_phase = 0, alive = 1;
#ifdef EC_DEBUG
    const int last_tile = p.silent && blockIdx.x == 0 ? 0 : total;
#else
    const int last_tile = total;
#endif
    Walk<NT> walk(groups, p.tiles_m, lane);    // of A only the halves of a tile that hold rows are loaded
    for (int tile = first_tile; tile < last_tile; tile += tile_step) {
      walk.to(tile);
      const int e = __shfl_sync(0xffffffffu, walk.e, 0), col0 = __shfl_sync(0xffffffffu, walk.m, 0) * kTileM, row0 = __shfl_sync(0xffffffffu, walk.row0, 0);
      const int boxes = __shfl_sync(0xffffffffu, walk.rows > NT / kBoxes ? kBoxes : 1, 0);
      for (int kb = kb0; kb < kb1; ++kb) {
        if (kb % kUnit == 0) {
          wait(alive, sse0 + 8 * scale_stage, scale_phase ^ 1, abort_flag, p.status, 7);
          const uint32_t lead = elected & alive;
          const uint32_t sc = scale_base + scale_stage * kScaleStage, bar = ssf0 + 8 * scale_stage;
          expect_tx_if(lead, bar, kScaleStage);
          tma_load_3d_if(lead, sc, &tmBs, bar, kb * (kStageK / 32), col0, e);
          tma_load_2d_if(lead, sc + kTileM * kScaleRow, &tmAs, bar, kb * (kStageK / 32), row0);
          if (++scale_stage == kScaleStages) { scale_stage = 0; scale_phase ^= 1; }
        }
        wait(alive, empty0 + 8 * stage, phase ^ 1, abort_flag, p.status, 1);
        const uint32_t lead = elected & alive;
        const uint32_t sb = smem_base + stage * kStage, bar = full0 + 8 * stage;
        expect_tx_if(lead, bar, kAt + boxes * kBoxBytes);
        tma_load_3d_if(lead, sb, &tmB, bar, kb * kRowBytes, col0, e);
        tma_load_2d_if(lead, sb + kAt, &tmA, bar, kb * kRowBytes, row0);
        if constexpr (kBoxes == 2) tma_load_2d_if(boxes == 2 ? lead : 0u, sb + kAt + kBoxBytes, &tmA, bar, kb * kRowBytes, row0 + NT / 2);
        if (++stage == S) { stage = 0; phase ^= 1; }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA
    // e2m1 operands, ue8m0 scales, 128 rows, as many columns as the tile has rows of A, in 32s; bits 4 and 29: which half of a scale column's four bytes (0 or 2)
    constexpr uint32_t idesc0 = (1u << 7) | (1u << 10) | (1u << 23) | ((uint32_t)(kM >> 4) << 24);
    const uint32_t elected = elect_one(), low0 = desc_low(smem_base);
    uint32_t stage = 0, phase = 0, it = 0, alive = 1;
    Walk<NT> walk(groups, p.tiles_m, lane);
    for (int tile = first_tile; tile < total; tile += tile_step, ++it) {
      walk.to(tile);
      const uint32_t idesc = __shfl_sync(0xffffffffu, idesc0 | ((uint32_t)(walk.rows + 31) / 32 << 19), 0);
      const uint32_t buf = kBuffers == 2 ? it & 1 : 0, use = kBuffers == 2 ? it >> 1 : it, d = buf * NT;
      // MMAs of one stage, of the halves h0 .. h1 - 1
      auto issue = [&](int kb, uint32_t st, int h0, int h1) {
        const uint32_t lead = elected & alive;
        const uint32_t scales = kScales0 + st * kScaleCols, blow = low0 + st * (kStage >> 4), alow = blow + (kAt >> 4);
        const int blocks = p.blocks - 8 * kb;        // left of the contraction; an MMA takes two
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t half = 2 * (i & 1);
#pragma unroll
          for (int h = 0; h < MT; ++h)
            if (h0 <= h && h < h1)
              tc_mma_mx_if(blocks > 2 * i ? lead : 0u, d + h * NT, blow + h * (kBBytes >> 4) + 2 * i, alow + 2 * i, idesc | (half << 4) | (half << 29),
                           scales + 8 * h + 4 * (i >> 1), scales + 8 * MT + kColsA * (i >> 1), (kb - kb0 | i) != 0);
        }
      };
      wait(alive, acce0 + 8 * buf, (use & 1) ^ 1, abort_flag, p.status, 2);
      int kb = kb0;
      if constexpr (MT == 2) {
        // The first half of the accumulator is free before the second: the stages at hand are multiplied into it meanwhile.
        const int some = min(kb0 + S, kb1);
        uint32_t st = stage, ph = phase;
        for (; kb < some; ++kb) {
          wait(alive, full0 + 8 * st, ph, abort_flag, p.status, 4);
          tc_fence_after();
          issue(kb, st, 0, 1);
          if (++st == S) { st = 0; ph ^= 1; }
        }
        wait(alive, acce0 + 8, (use & 1) ^ 1, abort_flag, p.status, 2);
        tc_fence_after();
        for (int k = kb0; k < some; ++k) {
          issue(k, stage, 1, 2);
          tc_commit_if(elected & alive, empty0 + 8 * stage);
          if (++stage == S) { stage = 0; phase ^= 1; }
        }
      }
      for (; kb < kb1; ++kb) {
        wait(alive, full0 + 8 * stage, phase, abort_flag, p.status, 4);
        tc_fence_after();
        issue(kb, stage, 0, MT);
        tc_commit_if(elected & alive, empty0 + 8 * stage);
        if (++stage == S) { stage = 0; phase ^= 1; }
      }
      tc_commit_if(elected & alive, accf0 + 8 * buf);
    }
  } else if (warp >= 2 + kEpi) {
    // ------------------------------------------------------------------ scales
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    constexpr int kRows = NT / 32;                   // of A, a lane's share of a tile; four of B
    uint32_t scale_stage = 0, scale_phase = 0, stage = 0, phase = 0;
    for (int tile = first_tile; tile < total && !gave_up; tile += tile_step) {
      for (int kb = kb0; kb < kb1; ++kb) {
        const int part = kb % kUnit;
        if (part == 0 && !warp_wait(ssf0 + 8 * scale_stage, scale_phase, abort_flag, p.status, 8, lane)) { gave_up = true; break; }
        // a row's eight bytes of this stage; the TMA unit's 32-byte swizzle exchanges the 16-byte halves of every other four rows
        const uint32_t from = scale_base + scale_stage * kScaleStage + lane * kScaleRow + (((part >> 1) ^ ((lane >> 2) & 1)) << 4) + 8 * (part & 1);
        uint32_t v[kScaleCols];                      // as they lie in tensor memory: of each 128 columns B's first 128 of the contraction, its second; A's first, its second
#pragma unroll
        for (int i = 0; i < 4 * MT + kRows; ++i) {
          const int at = i < 4 * MT ? 8 * (i / 4) + i % 4 : 4 * MT + i, half = i < 4 * MT ? 4 : kColsA;
          asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v[at]), "=r"(v[at + half]) : "r"(from + 32 * i * kScaleRow) : "memory");
        }
#pragma unroll
        for (int i = kRows; i < kColsA; ++i) v[8 * MT + i] = v[8 * MT + kColsA + i] = 0;
        const int blocks = p.blocks - 8 * kb;
        if (blocks < 8) {                            // behind the contraction's end: whatever lies there becomes 0, 2^-127
          const uint32_t first = blocks >= 4 ? 0xFFFFFFFFu : 0xFFFFFFFFu >> (32 - 8 * blocks), second = blocks > 4 ? 0xFFFFFFFFu >> (64 - 8 * blocks) : 0u;
#pragma unroll
          for (int i = 0; i < 4 * MT; ++i) { v[8 * (i / 4) + i % 4] &= first; v[8 * (i / 4) + 4 + i % 4] &= second; }
#pragma unroll
          for (int i = 0; i < kColsA; ++i) { v[8 * MT + i] &= first; v[8 * MT + kColsA + i] &= second; }
        }
        if (part == kUnit - 1 || kb + 1 == kb1) {     // all of these scales are in registers
          __syncwarp();
          if (lane == 0) mbar_arrive(sse0 + 8 * scale_stage);
          if (++scale_stage == kScaleStages) { scale_stage = 0; scale_phase ^= 1; }
        }
        if (!warp_wait(empty0 + 8 * stage, phase ^ 1, abort_flag, p.status, 5, lane)) { gave_up = true; break; }
        tc_fence_after();
        const uint32_t col = lanes + kScales0 + stage * kScaleCols;
#pragma unroll
        for (int i = 0; i < kScaleCols; i += 8) tc_st8(col + i, v + i);
        tc_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(full0 + 8 * stage);
        if (++stage == S) { stage = 0; phase ^= 1; }
      }
    }
  } else {
    // ------------------------------------------------------------------ epilogue
    const int q = warp & 3, first = kChunk * ((warp - 2) >> 2);      // chunks of rows in turn with the quarter's other warps
    int it = 0;
    Walk<NT> walk(groups, p.tiles_m, lane);
    for (int tile = first_tile; tile < total; tile += tile_step, ++it) {
      walk.to(tile);
      const int buf = kBuffers == 2 ? it & 1 : 0, rows = walk.rows; const uint32_t use = (uint32_t)(kBuffers == 2 ? it >> 1 : it);
      float biases[MT];
#pragma unroll
      for (int h = 0; h < MT; ++h) {
        const int col = walk.m * kTileM + h * kM + q * 32 + lane;
        biases[h] = 0.f;
        if (p.bias != nullptr && col < p.N) {
          const int64_t at = (int64_t)walk.e * p.N + col;
          biases[h] = p.bias_f32 ? __ldg((const float*)after_enter(p.bias) + at) : __bfloat162float(__ldg((const bf16*)after_enter(p.bias) + at));
        }
      }
      if (!warp_wait(accf0 + 8 * buf, use & 1, abort_flag, p.status, 6, lane)) { gave_up = true; break; }
      tc_fence_after();
      const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + buf * NT;
      // a chunk of a part: this warp's 32 columns times kChunk rows, four values of a lane after those of the others
      const uint32_t parts = scale_base + kScaleStages * kScaleStage + q * (32 * kChunk * 4) + lane * 16;
      constexpr uint32_t kPart = kM * NT * 4, kChunkBytes = kM * kChunk * 4;
      if constexpr (SPLIT) {
        if (rank != 0) {
          if (!cluster_wait(parte, (it & 1) ^ 1, abort_flag, p.status, 10, lane)) { gave_up = true; break; }
          const uint32_t to = map_to_cta(parts + (rank - 1) * kPart, 0);
#pragma unroll 1
          for (int c = first; c < rows; c += kChunk * (kEpi / 4)) {
            uint32_t r[kChunk]; tc_ld16(taddr + c, r);
#pragma unroll
            for (int j = 0; j < kChunk; j += 4) st_cluster4(to + c / kChunk * kChunkBytes + j * 128, reinterpret_cast<const float*>(r) + j);
          }
          asm volatile("fence.acq_rel.cluster;" ::: "memory");
          tc_fence_before();
          __syncwarp();
          if (lane == 0) { mbar_arrive_cluster(map_to_cta(partf, 0)); mbar_arrive(acce0 + 8 * buf); }
          continue;
        }
        if (!cluster_wait(partf, it & 1, abort_flag, p.status, 11, lane)) { gave_up = true; break; }
      }
#pragma unroll 1
      for (int c = first, h = 0; h < MT; c += kChunk * (kEpi / 4)) {         // uniform across the warp
        if (c >= rows) {                             // done with this half of the columns
          if constexpr (MT == 2) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(acce0 + 8 * h);
          }
          c = first - kChunk * (kEpi / 4); ++h;
          continue;
        }
        const int col = walk.m * kTileM + h * kM + q * 32 + lane;
        const bool in = col < p.N;
        const float bias = biases[MT == 1 ? 0 : h];
        __syncwarp();                                // the last chunk's stores parted the lanes
        uint32_t r[kChunk]; tc_ld16(taddr + h * NT + c, r);
        float v[kChunk];
#pragma unroll
        for (int j = 0; j < kChunk; ++j) v[j] = __uint_as_float(r[j]);
        if constexpr (SPLIT) {
          for (int other = 1; other < ctas; ++other)
#pragma unroll
            for (int j = 0; j < kChunk; j += 4) {
              float4 o;
              asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(o.x), "=f"(o.y), "=f"(o.z), "=f"(o.w)
                           : "r"(parts + (other - 1) * kPart + c / kChunk * kChunkBytes + j * 128) : "memory");
              v[j] += o.x; v[j + 1] += o.y; v[j + 2] += o.z; v[j + 3] += o.w;
            }
        }
#pragma unroll
        for (int j = 0; j < kChunk; ++j) v[j] += bias;
        if (p.act == EC_MX_GELU_ERF) {
#pragma unroll
          for (int j = 0; j < kChunk; j += 2) gelu_erf2(v[j], v[j + 1]);
        } else if (p.act == EC_MX_GELU_TANH) {
#pragma unroll
          for (int j = 0; j < kChunk; j += 2) gelu_fwd2<1>(v[j], v[j + 1], v[j], v[j + 1]);
        }
        const int left = rows - c;
        const int64_t row = walk.row0 + c;
        if constexpr (OUT == OUT_F32) {
          float* out = (float*)p.c + row * p.N + col;
#pragma unroll
          for (int j = 0; j < kChunk; ++j) if (in && j < left) out[(int64_t)j * p.N] = v[j];
        } else if constexpr (OUT == OUT_BF16) {
          // two rows at a time: even lanes take their column and the next one's of the first row, odd lanes of the second (N is even)
          const int odd = lane & 1;
          bf16* out = (bf16*)p.c + (row + odd) * p.N + (col - odd);
          const unsigned take = odd ? 0x3276u : 0x5410u;           // of (own, other): the lower halves, or (other, own): the upper ones
          auto store = [&](auto whole) {
#pragma unroll
            for (int j = 0; j < kChunk; j += 2) {
              __nv_bfloat162 h = __floats2bfloat162_rn(v[j], v[j + 1]);
              const unsigned own = *reinterpret_cast<unsigned*>(&h), pair = __byte_perm(own, __shfl_xor_sync(0xffffffffu, own, 1), take);
              if (in && (decltype(whole)::value || j + odd < left)) *reinterpret_cast<unsigned*>(out) = pair;
              out += 2 * (int64_t)p.N;
            }
          };
          if (left >= kChunk) store(std::true_type{}); else store(std::false_type{});
        } else {
          // The warp's 32 columns are one block of every row: the largest magnitude by one reduction per row, eight rows' codes turned
          // between the lanes (lane 8 i + j ends with columns 8 i .. 8 i + 7 of row j).  Columns behind the last are zeros: TMA fills their
          // weights with them.
          const int block = (walk.m * MT + h) * 4 + q;
#pragma unroll
          for (int j0 = 0; j0 < kChunk; j0 += 8) {
            float y[8];
            unsigned mine = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const unsigned amax = __reduce_max_sync(0xffffffffu, __float_as_uint(v[j0 + j]) & 0x7FFFFFFFu);
              y[j] = v[j0 + j] * mx_inverse_of(amax);
              if ((lane & 7) == j) mine = amax;
            }
            unsigned w = mx_codes8(y);               // lane: column, nibble: row
            unsigned o = __shfl_xor_sync(0xffffffffu, w, 1);
            w = lane & 1 ? (w & 0xF0F0F0F0u) | ((o >> 4) & 0x0F0F0F0Fu) : (w & 0x0F0F0F0Fu) | ((o << 4) & 0xF0F0F0F0u);
            o = __shfl_xor_sync(0xffffffffu, w, 2);
            w = __byte_perm(w, o, lane & 2 ? 0x3715u : 0x6240u);
            o = __shfl_xor_sync(0xffffffffu, w, 4);
            w = __byte_perm(w, o, lane & 4 ? 0x3276u : 0x5410u);
            const int j = j0 + (lane & 7);
            const unsigned s = mx_scale_of(mine);
            if (j < left && 32 * block < p.N) {
              *reinterpret_cast<unsigned*>((uint8_t*)p.c + (row + j) * p.c_pitch + 16 * block + 4 * (lane >> 3)) = s == kMxNan ? 0u : w;
              if (lane < 8) p.c_scales[(row + j) * p.c_scale_pitch + block] = (uint8_t)s;
            }
          }
        }
      }
      if constexpr (MT == 1) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(acce0 + 8 * buf);
      }
      if constexpr (SPLIT) {                         // the parts have been read
        if (lane == 0) for (int other = 1; other < ctas; ++other) mbar_arrive_cluster(map_to_cta(parte, other));
      }
    }
  }

  if (*abort_flag) {                                 // let copies and MMAs still in flight drain
    const unsigned long long t0 = globaltimer();
    while (globaltimer() - t0 < 200000ull) __nanosleep(1000);
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if constexpr (SPLIT) cluster_sync_all();           // nobody writes to or arrives at a CTA that has gone
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
  }
}

bool byte_map(CUtensorMap* tm, const void* base, int dims, int64_t inner, int64_t rows, int64_t batches, int box_inner, int box_rows,
              CUtensorMapSwizzle swizzle) {
  auto enc = (PFN_cuTensorMapEncodeTiled_v12000)tensor_map_encoder();
  if (!enc) return false;
  cuuint64_t size[3] = {(cuuint64_t)inner, (cuuint64_t)rows, (cuuint64_t)batches};
  cuuint64_t strides[2] = {(cuuint64_t)inner, (cuuint64_t)(inner * rows)};
  cuuint32_t box[3] = {(cuuint32_t)box_inner, (cuuint32_t)box_rows, 1}, step[3] = {1, 1, 1};
  return enc(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, dims, const_cast<void*>(base), size, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
             swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// No more row tiles than these: every expert may add one that is not full
int64_t most_tiles(const MxGemmArgs& g, int nt) { return (g.rows - 1) / nt + (g.E < g.rows ? g.E : g.rows); }

template <int NT, int OUT, bool SPLIT, int MT = 1>
cudaError_t launch_one(const MxGemmArgs& g, MxParams p, int sms, cudaStream_t st) {
  CUtensorMap ta, tb, tas, tbs;
  const int64_t inner = 16 * (int64_t)p.blocks, pitch = 16 * (int64_t)((g.K + 511) / 512);
  if (!byte_map(&ta, g.A, 2, inner, g.rows, 1, kRowBytes, NT / boxes_of(NT), CU_TENSOR_MAP_SWIZZLE_128B) ||
      !byte_map(&tb, g.B, 3, inner, g.N, g.E, kRowBytes, MT * kM, CU_TENSOR_MAP_SWIZZLE_128B) ||
      !byte_map(&tas, g.A_scales, 2, pitch, g.rows, 1, kScaleRow, NT, CU_TENSOR_MAP_SWIZZLE_32B) ||
      !byte_map(&tbs, g.B_scales, 3, pitch, g.N, g.E, kScaleRow, MT * kM, CU_TENSOR_MAP_SWIZZLE_32B)) return cudaErrorInvalidValue;
  constexpr int S = stages_of(NT, SPLIT, MT);
  p.tiles_m = (g.N + MT * kM - 1) / (MT * kM);
  constexpr int smem = S * stage_bytes(NT, MT) + kScaleStages * scale_stage_bytes(NT, MT) + parts_bytes(NT, SPLIT) + 1024 + (2 * S + 7 + 2 * kScaleStages) * 8 +
                       (int)sizeof(Groups);
  static_assert(smem <= 227 * 1024, "shared memory");
  auto kern = gemm_mx_kernel<NT, OUT, SPLIT, MT>;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  const int64_t most = most_tiles(g, NT) * p.tiles_m, at_once = sms / p.split;
  return launch_chained_cluster(p.split, kern, dim3((unsigned)((most < at_once ? most : at_once) * p.split)), dim3(kThreads), smem, st, ta, tb, tas, tbs, p);
}
// CTAs to a tile: more than one where all tiles then run at once and the contraction is long enough to pay for the joining, about 1 us (one CTA,
// two, four: two experts' rows, 16384 x 4096, 28.4, 20.5 and, not all at once, 30.0 us; one expert's 28.0, 18.9, 15.4; two of 8192 x 2048
// 16.1, 12.8, 12.0; two of 2048 x 2048 7.0, 8.0).  Where tiles take several rounds each round joins anew (eight experts, 4096 x 16384: 52 and 70 us).
int pick_split(const MxGemmArgs& g, const MxParams& p, int nt, int sms) {
  const int64_t tiles = most_tiles(g, nt) * p.tiles_m;
  const int units = (p.kblocks + kScaleStageK / kStageK - 1) / (kScaleStageK / kStageK);
  if (most_split(nt) >= 4 && units >= 8 && tiles * 4 <= sms * 7 / 8) return 4;           // clusters of four do not use every SM
  return units >= 6 && tiles * 2 <= sms ? 2 : 1;
}
template <int NT, int OUT>
cudaError_t launch_narrow(const MxGemmArgs& g, MxParams p, int sms, cudaStream_t st) {
  p.split = pick_split(g, p, NT, sms);
  return p.split > 1 ? launch_one<NT, OUT, true>(g, p, sms, st) : launch_one<NT, OUT, false>(g, p, sms, st);
}
// 256 columns of C per tile instead of 128, where one accumulator for both halves leaves the epilogue in the open: a stage then takes 1028
// cycles for two MMAs side by side instead of 775 for one (an SM receives 52 of its 54 bytes a clock with the narrow tiles, 56 KiB instead of
// 80 for the same work here), the epilogue some 2700 per 128 columns, 5200 with GeLU, 7000 with it to 4 bits.  The fewest cycles for the
// number of tiles to expect, an expert's last being half full.  Measured: 32768 rows, 64 experts, 4096 x 16384, at the power cap 1538 -> 1445 us;
// 3062 rows, 16 experts, 4072 x 1096, 23.5 -> 19.2; 8192 x 4096 to 4 bits 175 -> 161; not taken: 2048 x 4096 53 and 66, 768 x 2048 33 and 45.
bool wide(const MxGemmArgs& g, const MxParams& p, int sms) {
  const double tiles = g.rows / 192.0 + 0.5 * g.E, epi = g.out == EC_MX_OUT_MX ? 7000 : g.act != EC_MX_NONE ? 5200 : 2700;
  auto rounds = [&](int cols) { return ceil(tiles * ((g.N + cols - 1) / cols) / sms); };
  return rounds(256) * (p.kblocks * 1028.0 + 2 * epi + 1500) < rounds(128) * fmax(p.kblocks * 775.0 + 700, epi + 1100);
}
template <int OUT>
cudaError_t launch_out(const MxGemmArgs& g, const MxParams& p, int sms, cudaStream_t st) {
  // Rows per tile.  A tile of 64, 128 or 192 rows takes nearly the same time (64 experts of 4096 x 16384: 350, 396 and 434 us per row tile of
  // each, of which 347 are the reading of the weights), so what counts is how many an expert of uneven size needs.  Measured with
  // choices spread by exp(normal / 2), us for 64, 128, 192: a mean of 32 rows 425, 418, 459; 64 rows 543, 469, 503; 128 rows 839, 619, 598;
  // 256 rows 1510, 964, 843; 512 rows 2921, 1623, 1377; sixteen rows, 1024 x 1024: 15.5, 17.3, 19.2.
  const int64_t mean = g.rows / g.E;
  if (mean <= 2) return launch_narrow<32, OUT>(g, p, sms, st);     // eight rows of one token each: 64 us, with tiles of 64 rows 72 (more of the weights on their way)
  if (mean <= 20) return launch_narrow<64, OUT>(g, p, sms, st);
  if (mean <= 90) return launch_one<128, OUT, false>(g, p, sms, st);
  return wide(g, p, sms) ? launch_one<192, OUT, false, 2>(g, p, sms, st) : launch_one<192, OUT, false>(g, p, sms, st);
}

}  // namespace

cudaError_t launch_gemm_mx(const MxGemmArgs& g, cudaStream_t st) {
  int dev = 0, sms = 148;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  const cudaError_t bound = bind_device_context(dev);
  if (bound != cudaSuccess) return bound;
  MxParams p; memset(&p, 0, sizeof(p));
  p.rows = g.rows; p.N = g.N; p.E = g.E; p.tiles_m = (g.N + kM - 1) / kM;
  p.blocks = (g.K + 31) / 32; p.kblocks = (p.blocks + 7) / 8; p.act = g.act; p.offsets = g.offsets;
  p.bias = g.bias; p.bias_f32 = g.bias_dtype == EC_F32; p.c = g.C; p.c_scales = g.C_scales;
  p.c_pitch = 16 * (int64_t)((g.N + 31) / 32); p.c_scale_pitch = 16 * (int64_t)((g.N + 511) / 512);
  p.status = g.status; p.split = 1;
#ifdef EC_DEBUG
  p.silent = g.silent;
#endif
  switch (g.out) {
    case EC_MX_OUT_F32: return launch_out<OUT_F32>(g, p, sms, st);
    case EC_MX_OUT_BF16: return launch_out<OUT_BF16>(g, p, sms, st);
    default: return launch_out<OUT_MX>(g, p, sms, st);
  }
}

}  // namespace ecmoe
