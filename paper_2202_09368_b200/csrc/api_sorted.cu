// C ABI of the tokens sorted by expert: argument checks and launches.
#include "../../include/ecmoe.h"
#include "internal.h"

using namespace ecmoe;

namespace {

inline bool misaligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }
inline size_t esize(int dtype) { return dtype == EC_F32 ? 4 : 2; }
template <typename... P> bool bad_pointers(P... p) { return ((p == nullptr || misaligned(p, 16)) || ...); }

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
  if (bad_pointers(offsets) || ws == nullptr || misaligned(ws, 256)) return EC_ERR_INVALID_ARG;
  if (c->n > 0 && bad_pointers(choice, order, place)) return EC_ERR_INVALID_ARG;
  if (ws_bytes < ec_sort_workspace_bytes(c)) return EC_ERR_WORKSPACE;
  EC_CUDA(launch_sort_tokens(choice, c->n * c->per_token, c->E, offsets, order, place, ws, (cudaStream_t)stream));
  return EC_OK;
}

ec_status ec_dispatch(const ec_sort_config* c, const void* X, const int32_t* place, void* X_s, void* stream) {
  const ec_status s = check_sort(c);
  if (s != EC_OK || c->n == 0) return s;
  if (bad_pointers(X, place, X_s)) return EC_ERR_INVALID_ARG;
  EC_CUDA(launch_dispatch(X, place, X_s, c->n, c->d_model * (int64_t)esize(c->dtype), c->per_token, (cudaStream_t)stream));
  return EC_OK;
}

ec_status ec_combine(const ec_sort_config* c, const void* Y, const float* weights, const int32_t* place, void* X_out, void* stream) {
  const ec_status s = check_sort(c);
  if (s != EC_OK || c->n == 0) return s;
  if (bad_pointers(Y, place, X_out) || (weights != nullptr && misaligned(weights, 16))) return EC_ERR_INVALID_ARG;
  EC_CUDA(launch_combine_rows(c->dtype, c->y_dtype, Y, weights, place, X_out, c->n, c->d_model, c->per_token, (cudaStream_t)stream));
  return EC_OK;
}

ec_status ec_combine_backward(const ec_sort_config* c, const void* dX_out, const void* Y, const float* weights, const int32_t* place, void* dY,
                              float* dweights, void* stream) {
  const ec_status s = check_sort(c);
  if (s != EC_OK || c->n == 0) return s;
  if (bad_pointers(dX_out, Y, weights, place, dY, dweights)) return EC_ERR_INVALID_ARG;
  EC_CUDA(launch_combine_backward(c->dtype, c->y_dtype, dX_out, Y, weights, place, dY, dweights, c->n, c->d_model, c->per_token, (cudaStream_t)stream));
  return EC_OK;
}
