// Quantisation to the 4-bit microscaled format and back: rows, transposed matrices, and rows on their way to their experts.  Each
// kernel reads its input once and writes its output once; the floor is those bytes at the copy rate.
#include "internal.h"
#include "mx.cuh"

#include <type_traits>

namespace ecmoe {

namespace {

__device__ __forceinline__ unsigned max3(unsigned a, unsigned b, unsigned c) { return max(a, max(b, c)); }

// 8 neighbouring values of a row as fp32 bits; those at or beyond `cols` are zeros (cols is a multiple of a 16-byte piece)
__device__ __forceinline__ void load8(const bf16* row, int c, int cols, unsigned* x) {
  uint4 v = make_uint4(0, 0, 0, 0);
  if (c < cols) v = __ldg(reinterpret_cast<const uint4*>(row + c));
  const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = w[i] << 16; x[2 * i + 1] = w[i] & 0xFFFF0000u; }
}
__device__ __forceinline__ void load8(const float* row, int c, int cols, unsigned* x) {
  uint4 v[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
  if (c < cols) v[0] = __ldg(reinterpret_cast<const uint4*>(row + c));
  if (c + 4 < cols) v[1] = __ldg(reinterpret_cast<const uint4*>(row + c + 4));
#pragma unroll
  for (int i = 0; i < 2; ++i) { x[4 * i] = v[i].x; x[4 * i + 1] = v[i].y; x[4 * i + 2] = v[i].z; x[4 * i + 3] = v[i].w; }
}

// Four lanes hold a block, eight values each: their codes, and the block's scale byte.
__device__ __forceinline__ unsigned quantize8(const unsigned* x, unsigned& s) {
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < 8; i += 2) m = max3(m, x[i] & 0x7FFFFFFFu, x[i + 1] & 0x7FFFFFFFu);
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
  s = mx_scale_of(m);
  const float inv = mx_inverse(s);
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = __uint_as_float(x[i]) * inv;
  const unsigned codes = mx_codes8(y);
  return s == kMxNan ? 0u : codes;
}
// L lanes hold a row's stretch, four to a block: the scale bytes of four neighbouring blocks (of L / 4 where that is fewer) as a word,
// in all their lanes.
template <int L> __device__ __forceinline__ unsigned gather_scales(unsigned s, int lane) {
  unsigned w = s << (8 * ((lane % L >> 2) & 3));
  if constexpr (L >= 8) w |= __shfl_xor_sync(0xffffffffu, w, 4);
  if constexpr (L >= 16) w |= __shfl_xor_sync(0xffffffffu, w, 8);
  return w;
}

// L = 32: a warp takes H times 256 columns of a row, lane i eight neighbouring values of each, so its loads and its 128 bytes of codes are
// whole lines.  L = 4, 8, 16: rows of at most L / 4 blocks, 32 / L of them to a warp.  PLACED: the row is a token's and goes to every
// row place[t, j] names.
template <typename T, bool PLACED, int L, int H>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const T* X, int64_t rows, int64_t items, int stretches, int cols, uint8_t* codes, uint8_t* scales,
                                                            const int32_t* place, int K, int64_t out_rows) {
  chain_enter();
  const T* x0 = after_enter(X);
  const int32_t* pl = PLACED ? after_enter(place) : nullptr;
  const int lane = threadIdx.x & 31, blocks = (cols + 31) / 32, groups = (cols + 511) / 512;
  const int64_t code_pitch = 16 * (int64_t)blocks, scale_pitch = 16 * (int64_t)groups;
  for (int64_t it = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 5; it < items; it += (int64_t)gridDim.x * 8) {
    const int64_t first = L == 32 ? it / stretches : it * (32 / L);
    const int64_t row = first + lane / L;
    const int c0 = (L == 32 ? (int)(it - first * stretches) * (256 * H) : 0) + 8 * (lane % L);
    const bool live = L == 32 || row < rows;
    unsigned x[H][8], q[H], s[H];
#pragma unroll
    for (int h = 0; h < H; ++h) load8(x0 + row * cols, c0 + 256 * h, live ? cols : 0, x[h]);
#pragma unroll
    for (int h = 0; h < H; ++h) {
      q[h] = quantize8(x[h], s[h]);
      s[h] = gather_scales<L>(s[h], lane);
    }
    auto store = [&](int64_t r) {
#pragma unroll
      for (int h = 0; h < H; ++h) {
        const int c = c0 + 256 * h;
        if (c < 32 * blocks) *reinterpret_cast<unsigned*>(codes + r * code_pitch + c / 2) = q[h];
        if constexpr (L == 32) {
          if ((lane & 15) == 0 && c < 512 * groups) *reinterpret_cast<unsigned*>(scales + r * scale_pitch + c / 32) = s[h];
        } else {
          if (lane % L == 0) *reinterpret_cast<uint4*>(scales + r * scale_pitch) = make_uint4(s[h], 0, 0, 0);
        }
      }
    };
    if (!live) continue;                             // no lane of the warp is waited for below
    if constexpr (!PLACED) {
      store(row);
    } else {
#pragma unroll 4
      for (int j = 0; j < K; ++j) {
        const int r = __ldg(pl + row * K + j);
        if ((unsigned)r < (unsigned)out_rows) store(r);
      }
    }
  }
}

// X [batches][cols][rows], the contraction along its rows: output row r is column r of a matrix.  A CTA takes 256 of the contraction and
// 64 columns; a warp one block of 32 of the contraction, lane i two neighbouring columns, so its 32 loads are 32 lines.  The codes
// turn in shared memory and leave as 128 bytes of an output row at a time.
template <typename T>
__global__ void __launch_bounds__(256) quantize_columns_kernel(const T* X, int rows, int cols, int groups, uint8_t* codes, uint8_t* scales) {
  __shared__ uint4 tile[64][8 + 1];
  __shared__ __align__(8) uint8_t tile_scales[64][8];
  chain_enter();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, blocks = (cols + 31) / 32;
  const int r0 = blockIdx.x * 64, b0 = blockIdx.y * 8, r = r0 + 2 * lane, b = b0 + warp;
  const T* x = after_enter(X) + (int64_t)blockIdx.z * rows * cols;
  // All 32 loads are under way before the first is looked at.
  using Two = typename std::conditional<sizeof(T) == 2, unsigned, uint2>::type;
  Two w[32];
  const T* from = x + 32 * (int64_t)b * rows + r;
  if (r < rows && 32 * b + 32 <= cols) {
#pragma unroll
    for (int i = 0; i < 32; ++i) w[i] = __ldg(reinterpret_cast<const Two*>(from + (int64_t)i * rows));
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i) { w[i] = Two(); if (r < rows && 32 * b + i < cols) w[i] = __ldg(reinterpret_cast<const Two*>(from + (int64_t)i * rows)); }
  }
  unsigned v[2][32], m[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    if constexpr (sizeof(T) == 2) { v[0][i] = w[i] << 16; v[1][i] = w[i] & 0xFFFF0000u; }
    else { v[0][i] = w[i].x; v[1][i] = w[i].y; }
    m[0] = max(m[0], v[0][i] & 0x7FFFFFFFu); m[1] = max(m[1], v[1][i] & 0x7FFFFFFFu);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const unsigned s = mx_scale_of(m[h]);
    const float inv = mx_inverse(s);
    unsigned q[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = __uint_as_float(v[h][8 * w + i]) * inv;
      q[w] = s == kMxNan ? 0u : mx_codes8(y);
    }
    tile[2 * lane + h][warp] = make_uint4(q[0], q[1], q[2], q[3]);
    tile_scales[2 * lane + h][warp] = (uint8_t)s;
  }
  __syncthreads();
  const int64_t out0 = (int64_t)blockIdx.z * rows + r0;
#pragma unroll
  for (int i = threadIdx.x; i < 512; i += 256) {
    const int tr = i >> 3, tb = i & 7;
    if (r0 + tr < rows && b0 + tb < blocks) reinterpret_cast<uint4*>(codes)[(out0 + tr) * blocks + b0 + tb] = tile[tr][tb];
  }
  if (threadIdx.x < 64 && r0 + (int)threadIdx.x < rows)
    *reinterpret_cast<uint2*>(scales + (out0 + threadIdx.x) * (16 * (int64_t)groups) + b0) = *reinterpret_cast<const uint2*>(tile_scales[threadIdx.x]);
}

// A thread turns a word of eight codes into eight values, four words at a time, each a whole line of the warp's.
template <typename T>
__global__ void __launch_bounds__(256) dequantize_kernel(const uint8_t* codes, const uint8_t* scales, int64_t words, int words_per_row, int cols, int blocks,
                                                         int scale_pitch, T* X) {
  chain_enter();
  const unsigned* q = reinterpret_cast<const unsigned*>(after_enter(codes));
  const uint8_t* sc = after_enter(scales);
  constexpr int U = 4;
  for (int64_t i0 = (int64_t)blockIdx.x * (256 * U) + threadIdx.x; i0 < words; i0 += (int64_t)gridDim.x * (256 * U)) {
    unsigned v[U]; unsigned s[U]; int64_t at[U]; int col[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = i0 + 256 * u, row = i / words_per_row;
      const int w = (int)(i - row * words_per_row);
      col[u] = 8 * w; at[u] = row * cols + 8 * w;
      if (i < words) { v[u] = __ldg(q + row * (4 * (int64_t)blocks) + w); s[u] = __ldg(sc + row * scale_pitch + w / 4); }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + 256 * u >= words) break;
      const float p = mx_scale_value(s[u]);
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const unsigned code = v[u] >> (4 * j), e = (code >> 1) & 3, m = code & 1;
        // 1.m x 2^(e - 1), or m / 2 where e is 0, in fp32's fields
        const unsigned bits = (e == 0 ? m * 0x3F000000u : ((126u + e) << 23) | (m << 22)) | ((code & 8) << 28);
        f[j] = __uint_as_float(bits) * p;
      }
      T* out = X + at[u];
      if constexpr (sizeof(T) == 2) {
        uint4 o;
        unsigned* ow = reinterpret_cast<unsigned*>(&o);
#pragma unroll
        for (int j = 0; j < 4; ++j) { __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * j], f[2 * j + 1]); ow[j] = *reinterpret_cast<unsigned*>(&h); }
        *reinterpret_cast<uint4*>(out) = o;
      } else {
        *reinterpret_cast<float4*>(out) = make_float4(f[0], f[1], f[2], f[3]);
        if (col[u] + 4 < cols) *reinterpret_cast<float4*>(out + 4) = make_float4(f[4], f[5], f[6], f[7]);
      }
    }
  }
}

int sm_count() {
  int dev = 0, sms = 148;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return sms;
}
unsigned grid_of(int64_t ctas) {
  const int64_t most = (int64_t)sm_count() * 16;
  return (unsigned)(ctas < most ? ctas : most);
}

template <typename T, bool PLACED, int L, int H>
cudaError_t rows_with(const T* X, int64_t rows, int cols, uint8_t* codes, uint8_t* scales, const int32_t* place, int K, cudaStream_t st) {
  const int stretches = L == 32 ? (cols + 256 * H - 1) / (256 * H) : 1;
  const int64_t items = L == 32 ? rows * stretches : (rows + 32 / L - 1) / (32 / L);
  return launch_chained(quantize_rows_kernel<T, PLACED, L, H>, dim3(grid_of((items + 7) / 8)), dim3(256), 0, st, X, rows, items, stretches, cols, codes, scales,
                        place, K, rows * K);
}
template <typename T, bool PLACED>
cudaError_t rows_of(const T* X, int64_t rows, int cols, uint8_t* codes, uint8_t* scales, const int32_t* place, int K, cudaStream_t st) {
  if (cols <= 32) return rows_with<T, PLACED, 4, 1>(X, rows, cols, codes, scales, place, K, st);
  if (cols <= 64) return rows_with<T, PLACED, 8, 1>(X, rows, cols, codes, scales, place, K, st);
  if (cols <= 128) return rows_with<T, PLACED, 16, 1>(X, rows, cols, codes, scales, place, K, st);
  if (cols <= 512) return rows_with<T, PLACED, 32, 2>(X, rows, cols, codes, scales, place, K, st);
  return rows_with<T, PLACED, 32, 4>(X, rows, cols, codes, scales, place, K, st);
}

template <typename T>
cudaError_t quantize_of(const void* X, int64_t batches, int rows, int cols, int transposed, uint8_t* codes, uint8_t* scales, cudaStream_t st) {
  const int groups = (cols + 511) / 512;
  if (!transposed) return rows_of<T, false>((const T*)X, batches * rows, cols, codes, scales, nullptr, 0, st);
  for (int64_t b = 0; b < batches; b += 65535) {                  // grid.z
    const int64_t some = batches - b < 65535 ? batches - b : 65535;
    const cudaError_t e = launch_chained(quantize_columns_kernel<T>, dim3((rows + 63) / 64, 2 * groups, (unsigned)some), dim3(256), 0, st,
                                         (const T*)X + b * rows * cols, rows, cols, groups, codes + b * rows * (16 * (int64_t)((cols + 31) / 32)),
                                         scales + b * rows * (16 * (int64_t)groups));
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

cudaError_t launch_mx_quantize(int dtype, const void* X, int64_t batches, int rows, int cols, int transposed, uint8_t* codes, uint8_t* scales, cudaStream_t st) {
  return dtype == 0 ? quantize_of<float>(X, batches, rows, cols, transposed, codes, scales, st)
                    : quantize_of<bf16>(X, batches, rows, cols, transposed, codes, scales, st);
}

cudaError_t launch_mx_dispatch(int dtype, const void* X, const int32_t* place, int64_t n, int d, int K, uint8_t* codes, uint8_t* scales, cudaStream_t st) {
  return dtype == 0 ? rows_of<float, true>((const float*)X, n, d, codes, scales, place, K, st) : rows_of<bf16, true>((const bf16*)X, n, d, codes, scales, place, K, st);
}

cudaError_t launch_mx_dequantize(int dtype, const uint8_t* codes, const uint8_t* scales, int64_t rows, int cols, void* X, cudaStream_t st) {
  const int per_row = (cols + 7) / 8, blocks = (cols + 31) / 32, pitch = 16 * ((cols + 511) / 512);
  const int64_t words = rows * per_row;
  const dim3 grid(grid_of((words + 1023) / 1024));
  if (dtype == 0) return launch_chained(dequantize_kernel<float>, grid, dim3(256), 0, st, codes, scales, words, per_row, cols, blocks, pitch, (float*)X);
  return launch_chained(dequantize_kernel<bf16>, grid, dim3(256), 0, st, codes, scales, words, per_row, cols, blocks, pitch, (bf16*)X);
}

}  // namespace ecmoe
