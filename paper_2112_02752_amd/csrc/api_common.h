// What the host layers of the C ABI share: checks of matrices, status codes.
#pragma once

#include "seq_common.h"

namespace emb {

inline int dtype_bytes(int32_t dtype) { return dtype == EMB_FP32 ? 4 : (dtype == EMB_BF16 ? 2 : 0); }

inline emb_status hip_status(hipError_t e) {
  return e == hipSuccess ? EMB_OK : (e == hipErrorNotSupported ? EMB_EUNSUPPORTED : EMB_EHIP);
}

// tokens of one call
constexpr int64_t kMaxTokens = ((int64_t)1 << 31) - 64 - 1;

// bytes from a row to the next where offsets within a block's rows are 32 bits
constexpr int64_t kMaxRowBytes = (int64_t)1 << 24;

// a matrix with `cols` columns in use; saved: an 8-bit checkpoint, else fp32 or bf16
inline emb_status check_mat(const emb_mat* m, int32_t cols, bool saved) {
  if (m == nullptr || m->data == nullptr) return EMB_EINVAL;
  if (saved) {
    if (m->dtype != EMB_SAVED8 || m->exps == nullptr) return EMB_EINVAL;
    const int64_t groups = (cols + (int64_t)EMB_SAVED_GROUP - 1) / EMB_SAVED_GROUP;
    if (m->ld < groups * EMB_SAVED_GROUP || m->ld_exps < groups) return EMB_EINVAL;
    if (m->ld % EMB_SAVED_GROUP != 0 || ((uintptr_t)m->data & 31u) != 0) return EMB_EINVAL;
    return EMB_OK;
  }
  const int size = dtype_bytes(m->dtype);
  if (size == 0 || m->ld < cols) return EMB_EINVAL;
  return ((uintptr_t)m->data & (uintptr_t)(size - 1)) != 0 ? EMB_EINVAL : EMB_OK;
}

inline Rows rows_of(const emb_mat& m) {
  return Rows{static_cast<char*>(m.data), m.ld * (m.dtype == EMB_SAVED8 ? 1 : dtype_bytes(m.dtype)), m.exps, m.ld_exps};
}

}  // namespace emb
