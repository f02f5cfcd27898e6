// C ABI of the tokens sorted by expert and of the products on 4-bit operands: argument checks and launches.
#include "../../include/ecmoe.h"
#include "internal.h"

using namespace ecmoe;

namespace {

inline bool misaligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }
inline size_t esize(int dtype) { return dtype == EC_F32 ? 4 : 2; }
inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  return na > 0 && nb > 0 && (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}
template <typename... P> bool bad_pointers(P... p) { return ((p == nullptr || misaligned(p, 16)) || ...); }
// choice, offsets, order and place are read and written one by one: a slice of rows, or one layer of a stack, need not begin at 16 bytes
template <typename... P> bool bad_indices(const P*... p) { return ((p == nullptr || misaligned(p, 4)) || ...); }

#define EC_CUDA(x) do { if ((x) != cudaSuccess) return EC_ERR_CUDA; } while (0)

ec_status check_sort(const ec_sort_config* c) {
  if (!c || c->n < 0 || c->d_model < 1 || c->E < 1 || c->per_token < 1) return EC_ERR_INVALID_ARG;
  if ((c->dtype != EC_F32 && c->dtype != EC_BF16) || (c->y_dtype != EC_F32 && c->y_dtype != EC_BF16)) return EC_ERR_INVALID_ARG;
  if (c->dtype == EC_F32 && c->y_dtype != EC_F32) return EC_ERR_INVALID_ARG;
  if (c->E > 256 || c->per_token > 32 || c->n >= ((int64_t)1 << 31) || c->n * c->per_token >= ((int64_t)1 << 31)) return EC_ERR_UNSUPPORTED;
  if (c->d_model > (1 << 22) - 64 || (c->d_model * esize(c->dtype)) % 16 || (c->d_model * esize(c->y_dtype)) % 16) return EC_ERR_UNSUPPORTED;
  return EC_OK;
}

}  // namespace

size_t ec_sort_workspace_bytes(const ec_sort_config* c) {
  return check_sort(c) == EC_OK ? (sort_scratch_bytes(c->E) + 255) / 256 * 256 : 0;
}

ec_status ec_sort_tokens(const ec_sort_config* c, const int32_t* choice, int32_t* offsets, int32_t* order, int32_t* place, void* ws, size_t ws_bytes,
                         void* stream) {
  const ec_status s = check_sort(c);
  if (s != EC_OK) return s;
  if (bad_indices(offsets) || ws == nullptr || misaligned(ws, 256)) return EC_ERR_INVALID_ARG;
  if (c->n > 0 && bad_indices(choice, order, place)) return EC_ERR_INVALID_ARG;
  if (ws_bytes < ec_sort_workspace_bytes(c)) return EC_ERR_WORKSPACE;
  // the kernels index by what they read back of these arrays
  const size_t flat = (size_t)(c->n * c->per_token) * 4;
  const void* at[] = {choice, offsets, order, place, ws};
  const size_t bytes[] = {flat, (size_t)(c->E + 1) * 4, flat, flat, sort_scratch_bytes(c->E)};
  for (int i = 0; i < 5; ++i)
    for (int j = 0; j < i; ++j) if (overlap(at[i], bytes[i], at[j], bytes[j])) return EC_ERR_INVALID_ARG;
  EC_CUDA(launch_sort_tokens(choice, c->n * c->per_token, c->E, offsets, order, place, ws, (cudaStream_t)stream));
  return EC_OK;
}

ec_status ec_dispatch(const ec_sort_config* c, const void* X, const int32_t* place, void* X_s, void* stream) {
  const ec_status s = check_sort(c);
  if (s != EC_OK || c->n == 0) return s;
  if (bad_pointers(X, X_s) || bad_indices(place)) return EC_ERR_INVALID_ARG;
  EC_CUDA(launch_dispatch(X, place, X_s, c->n, c->d_model * (int64_t)esize(c->dtype), c->per_token, (cudaStream_t)stream));
  return EC_OK;
}

ec_status ec_combine(const ec_sort_config* c, const void* Y, const float* weights, const int32_t* place, void* X_out, void* stream) {
  const ec_status s = check_sort(c);
  if (s != EC_OK || c->n == 0) return s;
  if (bad_pointers(Y, X_out) || bad_indices(place) || (weights != nullptr && misaligned(weights, 16))) return EC_ERR_INVALID_ARG;
  EC_CUDA(launch_combine_rows(c->dtype, c->y_dtype, Y, weights, place, X_out, c->n, c->d_model, c->per_token, (cudaStream_t)stream));
  return EC_OK;
}

ec_status ec_combine_backward(const ec_sort_config* c, const void* dX_out, const void* Y, const float* weights, const int32_t* place, void* dY,
                              float* dweights, void* stream) {
  const ec_status s = check_sort(c);
  if (s != EC_OK || c->n == 0) return s;
  if (bad_pointers(dX_out, Y, weights, dY, dweights) || bad_indices(place)) return EC_ERR_INVALID_ARG;
  EC_CUDA(launch_combine_backward(c->dtype, c->y_dtype, dX_out, Y, weights, place, dY, dweights, c->n, c->d_model, c->per_token, (cudaStream_t)stream));
  return EC_OK;
}

// ---- 4-bit operands --------------------------------------------------------------------------------------------
namespace {
constexpr int64_t kMxMost = (1 << 22) - 64;
}

int64_t ec_mx_code_pitch(int64_t cols) { return cols < 1 ? 0 : 16 * ((cols - 1) / 32 + 1); }
int64_t ec_mx_scale_pitch(int64_t cols) { return cols < 1 ? 0 : 16 * ((cols - 1) / 512 + 1); }

ec_status ec_mx_quantize(int dtype, const void* X, int64_t batches, int64_t rows, int64_t cols, int transposed, uint8_t* codes, uint8_t* scales, void* stream) {
  if ((dtype != EC_F32 && dtype != EC_BF16) || (transposed != 0 && transposed != 1) || batches < 0 || rows < 0 || cols < 1) return EC_ERR_INVALID_ARG;
  // a transposed matrix has its rows on the grid and a 32-bit index inside one; rows as they are only add up
  if (cols > kMxMost || (transposed && rows > kMxMost) || batches >= ((int64_t)1 << 31) || rows >= ((int64_t)1 << 31)) return EC_ERR_UNSUPPORTED;
  if (batches * rows >= ((int64_t)1 << 31) || ((transposed ? rows : cols) * esize(dtype)) % 16) return EC_ERR_UNSUPPORTED;
  if (batches == 0 || rows == 0) return EC_OK;
  if (bad_pointers(X, codes, scales)) return EC_ERR_INVALID_ARG;
  EC_CUDA(launch_mx_quantize(dtype, X, batches, (int)rows, (int)cols, transposed, codes, scales, (cudaStream_t)stream));
  return EC_OK;
}

ec_status ec_mx_dequantize(int dtype, const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* X, void* stream) {
  if ((dtype != EC_F32 && dtype != EC_BF16) || rows < 0 || cols < 1) return EC_ERR_INVALID_ARG;
  if (cols > kMxMost || rows >= ((int64_t)1 << 31) || (cols * esize(dtype)) % 16) return EC_ERR_UNSUPPORTED;
  if (rows == 0) return EC_OK;
  if (bad_pointers(codes, scales, X)) return EC_ERR_INVALID_ARG;
  EC_CUDA(launch_mx_dequantize(dtype, codes, scales, rows, (int)cols, X, (cudaStream_t)stream));
  return EC_OK;
}

ec_status ec_mx_dispatch(const ec_sort_config* c, const void* X, const int32_t* place, uint8_t* codes, uint8_t* scales, void* stream) {
  const ec_status s = check_sort(c);
  if (s != EC_OK || c->n == 0) return s;
  if (bad_pointers(X, codes, scales) || bad_indices(place)) return EC_ERR_INVALID_ARG;
  EC_CUDA(launch_mx_dispatch(c->dtype, X, place, c->n, c->d_model, c->per_token, codes, scales, (cudaStream_t)stream));
  return EC_OK;
}

static ec_status mx_expert_gemm(const ec_mx_gemm_config* c, const uint8_t* A, const uint8_t* A_scales, const int32_t* offsets, const uint8_t* B,
                                const uint8_t* B_scales, const void* bias, void* C, uint8_t* C_scales, void* ws, size_t ws_bytes, int silent, void* stream) {
  if (!c || c->rows < 0 || c->N < 1 || c->K < 1 || c->E < 1) return EC_ERR_INVALID_ARG;
  if (c->out < EC_MX_OUT_F32 || c->out > EC_MX_OUT_MX || c->act < EC_MX_NONE || c->act > EC_MX_GELU_TANH) return EC_ERR_INVALID_ARG;
  if (c->bias_dtype != EC_F32 && c->bias_dtype != EC_BF16) return EC_ERR_INVALID_ARG;
  if (c->E > 256 || c->N > kMxMost || c->K > kMxMost || c->rows >= ((int64_t)1 << 31) - 256) return EC_ERR_UNSUPPORTED;
  if ((c->out == EC_MX_OUT_F32 && c->N % 4) || (c->out == EC_MX_OUT_BF16 && c->N % 8)) return EC_ERR_UNSUPPORTED;
  if ((c->rows / 32 + c->E + 1) * ((c->N + 127) / 128) >= ((int64_t)1 << 31)) return EC_ERR_UNSUPPORTED;      // tiles are counted in 32 bits
  if (ws == nullptr || misaligned(ws, 256)) return EC_ERR_INVALID_ARG;
  if (ws_bytes < EC_MX_WORKSPACE_BYTES) return EC_ERR_WORKSPACE;
  if (c->rows == 0) return EC_OK;
  if (bad_pointers(A, A_scales, B, B_scales, C) || bad_indices(offsets) || (bias != nullptr && misaligned(bias, 16))) return EC_ERR_INVALID_ARG;
  if (c->out == EC_MX_OUT_MX ? bad_pointers(C_scales) : C_scales != nullptr) return EC_ERR_INVALID_ARG;
  MxGemmArgs g{c->rows, c->N, c->K, c->E, c->out, c->act, A, A_scales, offsets, B, B_scales, bias, c->bias_dtype, C, C_scales, (int*)ws, silent};
  EC_CUDA(launch_gemm_mx(g, (cudaStream_t)stream));
  return EC_OK;
}

ec_status ec_mx_expert_gemm(const ec_mx_gemm_config* c, const uint8_t* A, const uint8_t* A_scales, const int32_t* offsets, const uint8_t* B,
                            const uint8_t* B_scales, const void* bias, void* C, uint8_t* C_scales, void* ws, size_t ws_bytes, void* stream) {
  return mx_expert_gemm(c, A, A_scales, offsets, B, B_scales, bias, C, C_scales, ws, ws_bytes, 0, stream);
}

#ifdef EC_DEBUG
// ec_mx_expert_gemm in which the first CTA loads nothing, so that its waits run out, and those of its cluster.
extern "C" ec_status ec_debug_mx_wait(const ec_mx_gemm_config* c, const uint8_t* A, const uint8_t* A_scales, const int32_t* offsets, const uint8_t* B,
                                      const uint8_t* B_scales, const void* bias, void* C, uint8_t* C_scales, void* ws, size_t ws_bytes, void* stream) {
  return mx_expert_gemm(c, A, A_scales, offsets, B, B_scales, bias, C, C_scales, ws, ws_bytes, 1, stream);
}
#endif
