// Quantisation to the 4-bit microscaled format and back: rows, transposed matrices, and rows on their way to their experts.  Each
// kernel reads its input once and writes its output once; the floor is those bytes at the copy rate.
#include "internal.h"
#include "mx.cuh"

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
// The scale bytes of a warp's eight blocks as two words, in lanes 0 and 16 (any of a half's lanes)
__device__ __forceinline__ unsigned gather_scales(unsigned s, int lane) {
  unsigned w = s << (8 * ((lane >> 2) & 3));
  w |= __shfl_xor_sync(0xffffffffu, w, 4);
  w |= __shfl_xor_sync(0xffffffffu, w, 8);
  return w;
}

// A warp takes 512 columns of a row (a piece of 16 scale bytes) at a time, lane i eight neighbouring values of each half: its loads
// and its 128 bytes of codes are whole lines.  PLACED: the row is a token's and goes to every row place[t, j] names.
template <typename T, bool PLACED>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const T* X, int64_t items, int groups, int cols, uint8_t* codes, uint8_t* scales,
                                                            const int32_t* place, int K, int64_t out_rows) {
  chain_enter();
  const T* x0 = after_enter(X);
  const int32_t* pl = PLACED ? after_enter(place) : nullptr;
  const int lane = threadIdx.x & 31, blocks = (cols + 31) / 32;
  const int64_t code_pitch = 16 * (int64_t)blocks, scale_pitch = 16 * (int64_t)groups;
  for (int64_t it = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 5; it < items; it += (int64_t)gridDim.x * 8) {
    const int64_t row = it / groups;
    const int c0 = (int)(it - row * groups) * 512;
    unsigned x[2][8], q[2], s[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) load8(x0 + row * cols, c0 + 256 * h + 8 * lane, cols, x[h]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      q[h] = quantize8(x[h], s[h]);
      s[h] = gather_scales(s[h], lane);
    }
    auto store = [&](int64_t r) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int c = c0 + 256 * h + 8 * lane;
        if (c < 32 * blocks) *reinterpret_cast<unsigned*>(codes + r * code_pitch + c / 2) = q[h];
        if ((lane & 15) == 0) *reinterpret_cast<unsigned*>(scales + r * scale_pitch + (c0 + 256 * h) / 32 + lane / 4) = s[h];
      }
    };
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
  unsigned v[2][32], m[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const int c = 32 * b + i;
    unsigned lo = 0, hi = 0;
    if (c < cols && r < rows) {
      if constexpr (sizeof(T) == 2) {
        const unsigned w = __ldg(reinterpret_cast<const unsigned*>(x + (int64_t)c * rows + r));
        lo = w << 16; hi = w & 0xFFFF0000u;
      } else {
        const uint2 w = __ldg(reinterpret_cast<const uint2*>(x + (int64_t)c * rows + r));
        lo = w.x; hi = w.y;
      }
    }
    v[0][i] = lo; v[1][i] = hi;
  }
#pragma unroll
  for (int i = 0; i < 32; ++i) { m[0] = max(m[0], v[0][i] & 0x7FFFFFFFu); m[1] = max(m[1], v[1][i] & 0x7FFFFFFFu); }
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

// A thread turns a word of eight codes into eight values.
template <typename T>
__global__ void __launch_bounds__(256) dequantize_kernel(const uint8_t* codes, const uint8_t* scales, int64_t words, int words_per_row, int cols, int blocks,
                                                         int scale_pitch, T* X) {
  chain_enter();
  const unsigned* q = reinterpret_cast<const unsigned*>(after_enter(codes));
  const uint8_t* sc = after_enter(scales);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < words; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / words_per_row;
    const int w = (int)(i - row * words_per_row), c = 8 * w;
    const unsigned v = __ldg(q + row * (4 * (int64_t)blocks) + w);
    const float p = mx_scale_value(__ldg(sc + row * scale_pitch + w / 4));
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const unsigned code = v >> (4 * j), e = (code >> 1) & 3, m = code & 1;
      // 1.m x 2^(e - 1), or m / 2 where e is 0, in fp32's fields
      const unsigned bits = (e == 0 ? m * 0x3F000000u : ((126u + e) << 23) | (m << 22)) | ((code & 8) << 28);
      f[j] = __uint_as_float(bits) * p;
    }
    T* out = X + row * cols + c;
    if constexpr (sizeof(T) == 2) {
      uint4 o;
      unsigned* ow = reinterpret_cast<unsigned*>(&o);
#pragma unroll
      for (int j = 0; j < 4; ++j) { __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * j], f[2 * j + 1]); ow[j] = *reinterpret_cast<unsigned*>(&h); }
      *reinterpret_cast<uint4*>(out) = o;
    } else {
      *reinterpret_cast<float4*>(out) = make_float4(f[0], f[1], f[2], f[3]);
      if (c + 4 < cols) *reinterpret_cast<float4*>(out + 4) = make_float4(f[4], f[5], f[6], f[7]);
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

template <typename T>
cudaError_t quantize_of(const void* X, int64_t batches, int rows, int cols, int transposed, uint8_t* codes, uint8_t* scales, cudaStream_t st) {
  const int groups = (cols + 511) / 512;
  if (!transposed) {
    const int64_t items = batches * rows * groups;
    return launch_chained(quantize_rows_kernel<T, false>, dim3(grid_of((items + 7) / 8)), dim3(256), 0, st, (const T*)X, items, groups, cols, codes, scales,
                          (const int32_t*)nullptr, 0, (int64_t)0);
  }
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
  const int groups = (d + 511) / 512;
  const int64_t items = n * groups;
  const dim3 grid(grid_of((items + 7) / 8));
  if (dtype == 0) return launch_chained(quantize_rows_kernel<float, true>, grid, dim3(256), 0, st, (const float*)X, items, groups, d, codes, scales, place, K, n * K);
  return launch_chained(quantize_rows_kernel<bf16, true>, grid, dim3(256), 0, st, (const bf16*)X, items, groups, d, codes, scales, place, K, n * K);
}

cudaError_t launch_mx_dequantize(int dtype, const uint8_t* codes, const uint8_t* scales, int64_t rows, int cols, void* X, cudaStream_t st) {
  const int per_row = (cols + 7) / 8, blocks = (cols + 31) / 32, pitch = 16 * ((cols + 511) / 512);
  const int64_t words = rows * per_row;
  const dim3 grid(grid_of((words + 255) / 256));
  if (dtype == 0) return launch_chained(dequantize_kernel<float>, grid, dim3(256), 0, st, codes, scales, words, per_row, cols, blocks, pitch, (float*)X);
  return launch_chained(dequantize_kernel<bf16>, grid, dim3(256), 0, st, codes, scales, words, per_row, cols, blocks, pitch, (bf16*)X);
}

}  // namespace ecmoe
