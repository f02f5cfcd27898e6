// Expert products on 4-bit microscaled operands: tcgen05.mma kind::mxf4 with a scale per block of 32, over groups of rows of any length.
//
//   C[r, :] = act(A[r, :] . B[e]^T + bias[e]),  offsets[e] <= r < offsets[e + 1]
//
// The weights' columns (rows of B[e]) are the 128 rows of an MMA and NT rows of A its columns, at every size: a tile of few rows of A is
// then a narrow MMA with nothing computed on fill, and one kernel serves one token and thousands.  A lane of tensor memory is a column
// of C, a column of it a row.
//
// Per CTA (persistent, one per SM):
//   warp 0      TMA: stages of 256 of the contraction, 128 x 128 bytes of B and NT x 128 bytes of A
//   warp 1      one lane issues the MMAs, 64 of the contraction each
//   warps 2-5   epilogue, a quarter of tensor memory's lanes each
//   warps 6-9   scales: 512 of the contraction (16 bytes of a row's scales) at a time, from global memory through registers into
//               tensor memory, where every quarter of the lanes wants its own copy: row 32 c + l of a tile in lane l, column c, four
//               blocks' bytes to a column.  Rows start anywhere, so no prepared layout could serve them.
// Two accumulators of NT columns, two buffers of scales of 16 + 4 * cols_a columns.
#include "../../include/ecmoe.h"
#include "internal.h"
#include "mx.cuh"
#include "tc_ptx.cuh"

#include <cudaTypedefs.h>
#include <string.h>

namespace ecmoe {

namespace {

constexpr int kM = 128;                              // columns of C per tile
constexpr int kStageK = 256, kRowBytes = kStageK / 2;
constexpr int kBBytes = kM * kRowBytes;              // 16 KiB
constexpr int kEpi = 4, kScaleWarps = 4;
constexpr int kThreads = 32 * (2 + kEpi + kScaleWarps);
constexpr int kMaxE = 256;
constexpr int kTmemCols = 512;
constexpr int kSmemBudget = 220 * 1024;

__host__ __device__ constexpr int stages_of(int nt) { const int fit = kSmemBudget / (kBBytes + nt * kRowBytes); return fit > 10 ? 10 : fit; }
// Columns of tensor memory for 128 of the contraction of A's scales.  tcgen05.mma wants a scale matrix to begin at a multiple of four
// columns, so narrow tiles leave some of the four unused.
__host__ __device__ constexpr int cols_a(int nt) { return nt <= 128 ? 4 : 8; }

struct MxParams {
  int64_t rows;
  int N, E, tiles_m, blocks, kblocks;                // blocks: of 32 along the contraction; kblocks: stages of 256
  int act;
  const int32_t* offsets;
  const uint8_t* a_scales; const uint8_t* b_scales; int64_t scale_pitch;
  const void* bias; int bias_f32;
  void* c; uint8_t* c_scales; int64_t c_pitch, c_scale_pitch;     // c_pitch in bytes
  int* status;
};

enum { OUT_F32 = 0, OUT_BF16 = 1, OUT_MX = 2 };

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* tm, uint32_t bar, int c0, int c1) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
               ::"r"(dst), "l"(tm), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void tc_mma_mx(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
  asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
               " tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}\n"
               ::"r"(d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tc_st4(uint32_t taddr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void tc_st2(uint32_t taddr, uint32_t a, uint32_t b) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x2.b32 [%0], {%1, %2};" ::"r"(taddr), "r"(a), "r"(b) : "memory");
}
__device__ __forceinline__ void tc_st1(uint32_t taddr, uint32_t a) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};" ::"r"(taddr), "r"(a) : "memory");
}
__device__ __forceinline__ void tc_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// word g of a row's 16 scale bytes
__device__ __forceinline__ unsigned word(const uint4& v, int g) { return g == 0 ? v.x : g == 1 ? v.y : g == 2 ? v.z : v.w; }

// Where a tile lies.  Tiles run expert by expert, inside one along its row tiles first: those that run at the same time share weights.
struct Tile { int e, m, row0, rows; };
struct Groups {                                      // in shared memory
  int first[kMaxE + 1];                              // row tiles before expert e
  int lo[kMaxE], count[kMaxE];                       // its rows
};
template <int NT>
__device__ __forceinline__ Tile find_tile(const Groups* g, int tiles_m, int tile, int& e) {
  while ((int64_t)g->first[e + 1] * tiles_m <= tile) ++e;          // tiles only grow
  const int idx = tile - g->first[e] * tiles_m, n = g->first[e + 1] - g->first[e], m = idx / n, t = idx - m * n;
  return {e, m, g->lo[e] + t * NT, min(NT, g->count[e] - t * NT)};
}

template <int NT, int OUT>
__global__ void __launch_bounds__(kThreads, 1)
gemm_mx_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const MxParams p) {
  constexpr int S = stages_of(NT), kStage = kBBytes + NT * kRowBytes;
  constexpr int kColsA = cols_a(NT), kScaleCols = 16 + 4 * kColsA, kScales0 = 2 * NT;
  static_assert(kScales0 + 2 * kScaleCols <= kTmemCols, "tensor memory");
  static_assert(kScales0 % 4 == 0 && kScaleCols % 4 == 0 && kColsA % 4 == 0, "where a scale matrix may begin");
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint64_t* bars = (uint64_t*)(smem + S * kStage);   // full[S], empty[S], acc_full[2], acc_empty[2], sc_full[2], sc_empty[2]
  uint32_t* tmem_slot = (uint32_t*)(bars + 2 * S + 8);
  volatile int* abort_flag = (volatile int*)(tmem_slot + 1);
  Groups* groups = (Groups*)(bars + 2 * S + 10);
  const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * S, accf0 = empty0 + 8 * S, acce0 = accf0 + 16, scf0 = acce0 + 16, sce0 = scf0 + 16;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
    for (int b = 0; b < 2; ++b) {
      mbar_init(accf0 + 8 * b, 1); mbar_init(acce0 + 8 * b, kEpi);
      mbar_init(scf0 + 8 * b, kScaleWarps); mbar_init(sce0 + 8 * b, 1);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (threadIdx.x == 32 * 2) { prefetch_map(&tmA); prefetch_map(&tmB); }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  chain_enter();
  const uint32_t tmem_base = *tmem_slot, smem_base = smem_u32(smem);
  // The first CTA clears the status word; another writes it two seconds into a wait at the earliest.
  if (blockIdx.x == 0 && threadIdx.x == 0) { p.status[0] = 0; p.status[1] = 0; }
  // The groups: offsets are the caller's memory, whatever they hold becomes rows inside [0, rows).
  const int32_t* offsets = after_enter(p.offsets);
  if (threadIdx.x < p.E) {
    const int64_t a = __ldg(offsets + threadIdx.x), b = __ldg(offsets + threadIdx.x + 1);
    const int64_t lo = min(max(a, (int64_t)0), p.rows), hi = min(max(b, (int64_t)0), p.rows);
    groups->lo[threadIdx.x] = (int)lo;
    groups->count[threadIdx.x] = (int)max(hi - lo, (int64_t)0);
  }
  __syncthreads();
  if (warp == 0) {
    int tiles[kMaxE / 32], sum = 0;
#pragma unroll
    for (int i = 0; i < kMaxE / 32; ++i) {
      const int e = lane * (kMaxE / 32) + i;
      tiles[i] = e < p.E ? (groups->count[e] + NT - 1) / NT : 0;
      sum += tiles[i];
    }
    int run = sum;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) { const int v = __shfl_up_sync(0xffffffffu, run, o); if (lane >= o) run += v; }
    run -= sum;
    if (lane == 0) groups->first[0] = 0;
#pragma unroll
    for (int i = 0; i < kMaxE / 32; ++i) { run += tiles[i]; const int e = lane * (kMaxE / 32) + i; if (e < p.E) groups->first[e + 1] = run; }
  }
  __syncthreads();
  const int total = groups->first[p.E] * p.tiles_m;
  bool gave_up = false;

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA
    if (lane == 0) {
      int stage = 0, e = 0; uint32_t phase = 0;
      for (int tile = blockIdx.x; tile < total && !gave_up; tile += gridDim.x) {
        const Tile t = find_tile<NT>(groups, p.tiles_m, tile, e);
        for (int kb = 0; kb < p.kblocks; ++kb) {
          if (!mbar_wait(empty0 + 8 * stage, phase ^ 1, abort_flag, p.status, 1)) { gave_up = true; break; }
          const uint32_t sb = smem_base + stage * kStage, bar = full0 + 8 * stage;
          mbar_expect_tx(bar, kStage);
          tma_load_3d(sb, &tmB, bar, kb * kRowBytes, t.m * kM, t.e);
          tma_load_2d(sb + kBBytes, &tmA, bar, kb * kRowBytes, t.row0);
          if (++stage == S) { stage = 0; phase ^= 1; }
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA
    if (lane == 0) {
      // e2m1 operands, ue8m0 scales, NT columns, 128 rows; bits 4 and 29: which half of a scale column's four bytes (0 or 2)
      const uint32_t idesc = (1u << 7) | (1u << 10) | ((uint32_t)(NT >> 3) << 17) | (1u << 23) | ((uint32_t)(kM >> 4) << 24);
      int stage = 0, it = 0; uint32_t phase = 0, chunk = 0;
      for (int tile = blockIdx.x; tile < total && !gave_up; tile += gridDim.x, ++it) {
        const int buf = it & 1; const uint32_t use = (uint32_t)(it >> 1);
        if (!mbar_wait(acce0 + 8 * buf, (use & 1) ^ 1, abort_flag, p.status, 2)) { gave_up = true; break; }
        const uint32_t d = tmem_base + buf * NT;
        for (int kb = 0; kb < p.kblocks; ++kb) {
          const uint32_t sbuf = chunk & 1, scol = tmem_base + kScales0 + sbuf * kScaleCols;
          if ((kb & 1) == 0 && !mbar_wait(scf0 + 8 * sbuf, (chunk >> 1) & 1, abort_flag, p.status, 3)) { gave_up = true; break; }
          if (!mbar_wait(full0 + 8 * stage, phase, abort_flag, p.status, 4)) { gave_up = true; break; }
          tc_fence_after();
          const uint32_t sb = smem_base + stage * kStage, sa = sb + kBBytes;
          const int steps = min(4, (p.blocks - 8 * kb + 1) / 2);     // MMAs that hold any of the contraction
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (i < steps) {
              const uint32_t g = 2 * (kb & 1) + (i >> 1), half = 2 * (i & 1);
              tc_mma_mx(d, make_desc(sb + 32 * i, 16, 1024), make_desc(sa + 32 * i, 16, 1024), idesc | (half << 4) | (half << 29),
                        scol + 4 * g, scol + 16 + kColsA * g, (kb | i) != 0);
            }
          }
          tc_commit(empty0 + 8 * stage);
          if (++stage == S) { stage = 0; phase ^= 1; }
          if ((kb & 1) == 1 || kb + 1 == p.kblocks) { tc_commit(sce0 + 8 * sbuf); ++chunk; }
        }
        if (!gave_up) tc_commit(accf0 + 8 * buf);
      }
    }
  } else if (warp >= 2 + kEpi) {
    // ------------------------------------------------------------------ scales
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint8_t* asc = after_enter(p.a_scales);
    const uint8_t* bsc = after_enter(p.b_scales);
    const int chunks = (p.kblocks + 1) / 2, last = p.blocks - 16 * (chunks - 1);      // blocks of the last chunk
    constexpr int kRowsA = NT / 32;
    auto keep = [&](uint4 v) {                       // blocks behind the contraction's end: whatever lies there becomes 0, 2^-127
      unsigned* w = reinterpret_cast<unsigned*>(&v);
#pragma unroll
      for (int g = 0; g < 4; ++g) { const int n = last - 4 * g; if (n < 4) w[g] = n <= 0 ? 0u : w[g] & (0xFFFFFFFFu >> (32 - 8 * n)); }
      return v;
    };
    auto load = [&](const Tile& t, int c, uint4* b, uint4* a) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int col = t.m * kM + 32 * i + lane;
        b[i] = col < p.N ? __ldg(reinterpret_cast<const uint4*>(bsc + ((int64_t)t.e * p.N + col) * p.scale_pitch + 16 * c)) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < kRowsA; ++i) {
        const int r = 32 * i + lane;
        a[i] = r < t.rows ? __ldg(reinterpret_cast<const uint4*>(asc + (int64_t)(t.row0 + r) * p.scale_pitch + 16 * c)) : make_uint4(0, 0, 0, 0);
      }
      if (c + 1 == chunks) {
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = keep(b[i]);
#pragma unroll
        for (int i = 0; i < kRowsA; ++i) a[i] = keep(a[i]);
      }
    };
    int e = 0, tile = blockIdx.x, c = 0;
    uint32_t chunk = 0;
    uint4 b[4], a[kRowsA];
    Tile t;
    if (tile < total) { t = find_tile<NT>(groups, p.tiles_m, tile, e); load(t, 0, b, a); }
    while (tile < total) {
      const uint32_t sbuf = chunk & 1;
      const bool ok = mbar_wait(sce0 + 8 * sbuf, ((chunk >> 1) & 1) ^ 1, abort_flag, p.status, 5);
      if (!__all_sync(0xffffffffu, ok)) { gave_up = true; break; }
      tc_fence_after();
      const uint32_t col = tmem_base + lanes + kScales0 + sbuf * kScaleCols;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        tc_st4(col + 4 * g, word(b[0], g), word(b[1], g), word(b[2], g), word(b[3], g));
        const uint32_t ca = col + 16 + kColsA * g;
        if constexpr (NT == 32) tc_st1(ca, word(a[0], g));
        else if constexpr (NT == 64) tc_st2(ca, word(a[0], g), word(a[1], g));
        else {
          tc_st4(ca, word(a[0], g), word(a[1], g), word(a[2], g), word(a[3], g));
          if constexpr (NT == 192) tc_st2(ca + 4, word(a[4], g), word(a[5], g));
        }
      }
      if (++c == chunks) { c = 0; tile += gridDim.x; if (tile < total) t = find_tile<NT>(groups, p.tiles_m, tile, e); }
      if (tile < total) load(t, c, b, a);            // the next chunk's, while this one is used
      tc_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(scf0 + 8 * sbuf);
      ++chunk;
    }
  } else {
    // ------------------------------------------------------------------ epilogue
    const int q = warp & 3;
    int it = 0, e = 0;
    for (int tile = blockIdx.x; tile < total; tile += gridDim.x, ++it) {
      const Tile t = find_tile<NT>(groups, p.tiles_m, tile, e);
      const int buf = it & 1; const uint32_t use = (uint32_t)(it >> 1);
      const int col = t.m * kM + q * 32 + lane;
      const bool in = col < p.N;
      float bias = 0.f;
      if (p.bias != nullptr && in) {
        const int64_t at = (int64_t)t.e * p.N + col;
        bias = p.bias_f32 ? __ldg((const float*)after_enter(p.bias) + at) : __bfloat162float(__ldg((const bf16*)after_enter(p.bias) + at));
      }
      const bool ok = mbar_wait(accf0 + 8 * buf, use & 1, abort_flag, p.status, 6);
      if (!__all_sync(0xffffffffu, ok)) { gave_up = true; break; }
      tc_fence_after();
      const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + buf * NT;
#pragma unroll 1
      for (int c = 0; c < t.rows; c += 32) {         // uniform across the warp
        uint32_t r[32]; tc_ld32(taddr + c, r);
        float v[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]) + bias;
        if (p.act == EC_MX_GELU_ERF) {
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = gelu_fwd(v[j], 0);
        } else if (p.act == EC_MX_GELU_TANH) {
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = gelu_fwd(v[j], 1);
        }
        const int left = t.rows - c;
        const int64_t row = t.row0 + c;
        if constexpr (OUT == OUT_F32) {
          float* out = (float*)p.c + row * p.N + col;
#pragma unroll
          for (int j = 0; j < 32; ++j) if (in && j < left) out[(int64_t)j * p.N] = v[j];
        } else if constexpr (OUT == OUT_BF16) {
          bf16* out = (bf16*)p.c + row * p.N + col;
#pragma unroll
          for (int j = 0; j < 32; ++j) if (in && j < left) out[(int64_t)j * p.N] = __float2bfloat16(v[j]);
        } else {
          // The warp's 32 columns are one block of every row: the largest magnitude by one reduction per row, eight rows' codes turned
          // between the lanes (lane 8 i + j ends with columns 8 i .. 8 i + 7 of row j).
#pragma unroll
          for (int j0 = 0; j0 < 32; j0 += 8) {
            float y[8];
            unsigned mine = 0, nan_rows = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float x = in ? v[j0 + j] : 0.f;
              const unsigned s = mx_scale_of(__reduce_max_sync(0xffffffffu, __float_as_uint(x) & 0x7FFFFFFFu));
              y[j] = x * mx_inverse(s);
              if (s == kMxNan) nan_rows |= 0xFu << (4 * j);
              if ((lane & 7) == j) mine = s;
            }
            unsigned w = mx_codes8(y) & ~nan_rows;   // lane: column, nibble: row
            unsigned o = __shfl_xor_sync(0xffffffffu, w, 1);
            w = lane & 1 ? (w & 0xF0F0F0F0u) | ((o >> 4) & 0x0F0F0F0Fu) : (w & 0x0F0F0F0Fu) | ((o << 4) & 0xF0F0F0F0u);
            o = __shfl_xor_sync(0xffffffffu, w, 2);
            w = lane & 2 ? (w & 0xFF00FF00u) | ((o >> 8) & 0x00FF00FFu) : (w & 0x00FF00FFu) | ((o << 8) & 0xFF00FF00u);
            o = __shfl_xor_sync(0xffffffffu, w, 4);
            w = lane & 4 ? (w & 0xFFFF0000u) | (o >> 16) : (w & 0x0000FFFFu) | (o << 16);
            const int j = j0 + (lane & 7), block = t.m * 4 + q;
            if (j < left && 32 * block < p.N) {
              *reinterpret_cast<unsigned*>((uint8_t*)p.c + (row + j) * p.c_pitch + 16 * block + 4 * (lane >> 3)) = w;
              if (lane < 8) p.c_scales[(row + j) * p.c_scale_pitch + block] = (uint8_t)mine;
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(acce0 + 8 * buf);
    }
  }

  if (*abort_flag) {                                 // let copies and MMAs still in flight drain
    const unsigned long long t0 = globaltimer();
    while (globaltimer() - t0 < 200000ull) __nanosleep(1000);
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
  }
}

bool byte_map(CUtensorMap* tm, const void* base, int dims, int64_t inner, int64_t rows, int64_t batches, int box_rows) {
  auto enc = (PFN_cuTensorMapEncodeTiled_v12000)tensor_map_encoder();
  if (!enc) return false;
  cuuint64_t size[3] = {(cuuint64_t)inner, (cuuint64_t)rows, (cuuint64_t)batches};
  cuuint64_t strides[2] = {(cuuint64_t)inner, (cuuint64_t)(inner * rows)};
  cuuint32_t box[3] = {kRowBytes, (cuuint32_t)box_rows, 1}, step[3] = {1, 1, 1};
  return enc(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, dims, const_cast<void*>(base), size, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int NT, int OUT>
cudaError_t launch_one(const MxGemmArgs& g, MxParams p, int sms, cudaStream_t st) {
  CUtensorMap ta, tb;
  const int64_t inner = 16 * (int64_t)p.blocks;
  if (!byte_map(&ta, g.A, 2, inner, g.rows, 1, NT) || !byte_map(&tb, g.B, 3, inner, g.N, g.E, kM)) return cudaErrorInvalidValue;
  constexpr int smem = stages_of(NT) * (kBBytes + NT * kRowBytes) + 1024 + (2 * stages_of(NT) + 10) * 8 + (int)sizeof(Groups);
  auto kern = gemm_mx_kernel<NT, OUT>;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  // no more CTAs than there can be tiles: every expert may add one that is not full
  const int64_t most = ((g.rows + NT - 1) / NT + (g.E < g.rows ? g.E : g.rows)) * p.tiles_m;
  return launch_chained(kern, dim3((unsigned)(most < sms ? most : sms)), dim3(kThreads), smem, st, ta, tb, p);
}
template <int OUT>
cudaError_t launch_out(const MxGemmArgs& g, const MxParams& p, int sms, cudaStream_t st) {
  const int64_t mean = g.rows / g.E;
  if (mean <= 32) return launch_one<32, OUT>(g, p, sms, st);
  if (mean <= 64) return launch_one<64, OUT>(g, p, sms, st);
  if (mean <= 128) return launch_one<128, OUT>(g, p, sms, st);
  return launch_one<192, OUT>(g, p, sms, st);
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
  p.a_scales = g.A_scales; p.b_scales = g.B_scales; p.scale_pitch = 16 * (int64_t)((g.K + 511) / 512);
  p.bias = g.bias; p.bias_f32 = g.bias_dtype == EC_F32; p.c = g.C; p.c_scales = g.C_scales;
  p.c_pitch = 16 * (int64_t)((g.N + 31) / 32); p.c_scale_pitch = 16 * (int64_t)((g.N + 511) / 512);
  p.status = g.status;
  switch (g.out) {
    case EC_MX_OUT_F32: return launch_out<OUT_F32>(g, p, sms, st);
    case EC_MX_OUT_BF16: return launch_out<OUT_BF16>(g, p, sms, st);
    default: return launch_out<OUT_MX>(g, p, sms, st);
  }
}

}  // namespace ecmoe
