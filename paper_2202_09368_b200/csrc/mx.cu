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
// row place[t, j] names.  Memory bounds the fp32 form (16384 x 4096 45.7 us, the copy rate); in bf16 a byte costs twice the
// instructions: 31.9 us, 5.3 TB/s (H = 2: 37.4).  To two rows per token 39.3 us.  131072 x 64 7.2 us (with a warp per row 34).
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
    unsigned word = 0;                               // L = 32: lane i takes word i of the stretch's 2 H scale words, one store for all (H = 1: the padding too)
    if constexpr (L == 32) {
#pragma unroll
      for (int h = 0; h < H; ++h) { const unsigned w = __shfl_sync(0xffffffffu, s[h], 16 * (lane & 1)); if (lane >> 1 == h) word = w; }
    }
    auto store = [&](int64_t r) {
#pragma unroll
      for (int h = 0; h < H; ++h) if (c0 + 256 * h < 32 * blocks) *reinterpret_cast<unsigned*>(codes + r * code_pitch + (c0 + 256 * h) / 2) = q[h];
      if constexpr (L == 32) {
        const int at = (c0 - 8 * lane) / 32 + 4 * lane;
        if (lane < (H == 1 ? 4 : 2 * H) && at < 16 * groups) *reinterpret_cast<unsigned*>(scales + r * scale_pitch + at) = word;
      } else {
        if (lane % L == 0) *reinterpret_cast<uint4*>(scales + r * scale_pitch) = make_uint4(s[0], 0, 0, 0);
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
// turn in shared memory and leave as 128 bytes of an output row at a time.  Memory bounds it: 4 x 4096 x 8192 bf16 58 us (89 % of the copy
// rate; two CTAs per SM instead of three 70, loads unpacked one by one as they come 270), fp32 88 us.
template <typename T>
__global__ void __launch_bounds__(256, 3) quantize_columns_kernel(const T* X, int rows, int cols, int groups, uint8_t* codes, uint8_t* scales) {
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

// The codes of 16 bytes of values at a time: eight in bf16, four in fp32, so that a warp's stores are whole lines.  The three bits of a
// magnitude, put where fp32 has the end of its exponent and the start of its fraction, are 2^-126 times what they stand for, the
// subnormal ones among them.  Lanes as in the quantisation: L = 32, U times 32 pieces of a row; else 32 / L rows, U times.  Memory bounds it:
// 16384 x 4096 to bf16 28 us (92 % of the copy rate), to fp32 48.5 (95 %).
template <typename T, int L, int U>
__global__ void __launch_bounds__(256) dequantize_kernel(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t items, int stretches, int pieces,
                                                         int code_pitch, int scale_pitch, uint4* X) {
  constexpr int V = 16 / sizeof(T);
  using Codes = typename std::conditional<V == 8, unsigned, unsigned short>::type;
  chain_enter();
  const uint8_t* q = after_enter(codes);
  const uint8_t* sc = after_enter(scales);
  const int lane = threadIdx.x & 31;
  for (int64_t it = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 5; it < items; it += (int64_t)gridDim.x * 8) {
    const int64_t first = L == 32 ? it / stretches : it * (32 / L * U);
    const int w0 = L == 32 ? (int)(it - first * stretches) * (32 * U) : 0;
    unsigned v[U], s[U];
    bool live[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t row = L == 32 ? first : first + u * (32 / L) + lane / L;
      const int w = L == 32 ? w0 + 32 * u + lane : lane % L;
      live[u] = w < pieces && row < rows;
      if (live[u]) { v[u] = __ldg(reinterpret_cast<const Codes*>(q + row * code_pitch) + w); s[u] = __ldg(sc + row * scale_pitch + w * V / 32); }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!live[u]) continue;
      const int64_t row = L == 32 ? first : first + u * (32 / L) + lane / L;
      const int w = L == 32 ? w0 + 32 * u + lane : lane % L;
      const float p = mx_scale_value(s[u]);
      float f[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const unsigned bits = (4 * j <= 22 ? v[u] << ((22 - 4 * j) & 31) : v[u] >> ((4 * j - 22) & 31)) & 0x01C00000u;
        f[j] = __uint_as_float(bits | ((v[u] << (28 - 4 * j)) & 0x80000000u)) * 0x1p126f * p;
      }
      uint4 o;
      unsigned* ow = reinterpret_cast<unsigned*>(&o);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (V == 8) { __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * j], f[2 * j + 1]); ow[j] = *reinterpret_cast<unsigned*>(&h); }
        else ow[j] = __float_as_uint(f[j]);
      }
      X[row * pieces + w] = o;
    }
  }
}

int sm_count() {
  int dev = 0, sms = 148;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return sms;
}
unsigned grid_of(int64_t ctas, int per_sm) {
  const int64_t most = (int64_t)sm_count() * per_sm;
  return (unsigned)(ctas < most ? ctas : most);
}

template <typename T, bool PLACED, int L, int H>
cudaError_t rows_with(const T* X, int64_t rows, int cols, uint8_t* codes, uint8_t* scales, const int32_t* place, int K, cudaStream_t st) {
  const int stretches = L == 32 ? (cols + 256 * H - 1) / (256 * H) : 1;
  const int64_t items = L == 32 ? rows * stretches : (rows + 32 / L - 1) / (32 / L);
  return launch_chained(quantize_rows_kernel<T, PLACED, L, H>, dim3(grid_of((items + 7) / 8, 16)), dim3(256), 0, st, X, rows, items, stretches, cols, codes, scales,
                        place, K, rows * K);
}
template <typename T, bool PLACED>
cudaError_t rows_of(const T* X, int64_t rows, int cols, uint8_t* codes, uint8_t* scales, const int32_t* place, int K, cudaStream_t st) {
  if (cols <= 32) return rows_with<T, PLACED, 4, 1>(X, rows, cols, codes, scales, place, K, st);
  if (cols <= 64) return rows_with<T, PLACED, 8, 1>(X, rows, cols, codes, scales, place, K, st);
  if (cols <= 128) return rows_with<T, PLACED, 16, 1>(X, rows, cols, codes, scales, place, K, st);
  // 65536 x 176 fp32, two places: 18.1 us with 256 columns to a warp, 23.8 with 512 (half of whose loads have nothing to read).
  if (cols <= 256) return rows_with<T, PLACED, 32, 1>(X, rows, cols, codes, scales, place, K, st);
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

namespace {
template <typename T, int L, int U>
cudaError_t dequantize_with(const uint8_t* codes, const uint8_t* scales, int64_t rows, int cols, int pieces, void* X, cudaStream_t st) {
  const int stretches = L == 32 ? (pieces + 32 * U - 1) / (32 * U) : 1;
  const int64_t items = L == 32 ? rows * stretches : (rows + 32 / L * U - 1) / (32 / L * U);
  return launch_chained(dequantize_kernel<T, L, U>, dim3(grid_of((items + 7) / 8, 64)), dim3(256), 0, st, codes, scales, rows, items, stretches, pieces,
                        16 * ((cols + 31) / 32), 16 * ((cols + 511) / 512), (uint4*)X);
}
template <typename T>
cudaError_t dequantize_of(const uint8_t* codes, const uint8_t* scales, int64_t rows, int cols, void* X, cudaStream_t st) {
  const int pieces = cols / (16 / (int)sizeof(T));
  if (pieces <= 4) return dequantize_with<T, 4, 2>(codes, scales, rows, cols, pieces, X, st);
  if (pieces <= 8) return dequantize_with<T, 8, 2>(codes, scales, rows, cols, pieces, X, st);
  if (pieces <= 16) return dequantize_with<T, 16, 2>(codes, scales, rows, cols, pieces, X, st);
  if (pieces <= 32) return dequantize_with<T, 32, 1>(codes, scales, rows, cols, pieces, X, st);
  return pieces <= 64 ? dequantize_with<T, 32, 2>(codes, scales, rows, cols, pieces, X, st) : dequantize_with<T, 32, 4>(codes, scales, rows, cols, pieces, X, st);
}
}  // namespace

cudaError_t launch_mx_dequantize(int dtype, const uint8_t* codes, const uint8_t* scales, int64_t rows, int cols, void* X, cudaStream_t st) {
  return dtype == 0 ? dequantize_of<float>(codes, scales, rows, cols, X, st) : dequantize_of<bf16>(codes, scales, rows, cols, X, st);
}

}  // namespace ecmoe
