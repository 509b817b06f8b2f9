// C ABI of the operators of a model's block: host-side argument checks, kernel
// dispatch.  No allocation, no synchronisation.
#include <math.h>

#include "api_common.h"
#include "block_common.h"

using namespace emb;

namespace {

bool vectors(const Rows& r) { return (((uintptr_t)r.p | (uintptr_t)r.ld) & 15u) == 0; }

// a matrix that a call may do without
emb_status check_opt(const emb_mat* m, int32_t cols, int32_t dtype, Rows* out) {
  if (m == nullptr || m->data == nullptr) return EMB_OK;
  const emb_status st = check_mat(m, cols, false);
  if (st != EMB_OK) return st;
  if (m->dtype != dtype) return EMB_EINVAL;
  *out = rows_of(*m);
  return EMB_OK;
}

emb_status check_drop(float p, uint64_t seed, int64_t first_row, Drop* out) {
  if (!(p >= 0.f && p < 1.f) || first_row < 0) return EMB_EINVAL;
  *out = make_drop(p, seed, first_row);
  return out->below > 0xffffu ? EMB_EINVAL : EMB_OK;
}

// sizes, weights, dropout; the residual stream's type from the first matrix of it that is there
emb_status check_norm(int64_t rows, int32_t dim, const emb_norm* norm, const emb_mat* x, const emb_mat* const stream[3],
                      NormLaunch* p) {
  if (norm == nullptr || rows < 0 || dim < 1) return EMB_EINVAL;
  if (!(norm->eps >= 0.f) || isinf(norm->eps)) return EMB_EINVAL;
  if (((uintptr_t)norm->weight & 3u) != 0) return EMB_EINVAL;
  const emb_status st = check_drop(norm->drop, norm->seed, norm->first_row, &p->drop);
  if (st != EMB_OK) return st;
  if (rows > kMaxTokens || dim > kNormMaxDim) return EMB_EUNSUPPORTED;
  p->N = rows;
  p->D = dim;
  p->eps = norm->eps;
  p->weight = norm->weight;
  p->aligned = ((uintptr_t)norm->weight & 15u) == 0;
  if (rows == 0) return EMB_OK;
  if (x == nullptr || x->data == nullptr) return EMB_EINVAL;
  p->dtype = x->dtype;
  p->stream_dtype = x->dtype;
  for (int i = 0; i < 3; ++i)
    if (stream[i] != nullptr && stream[i]->data != nullptr) {
      p->stream_dtype = stream[i]->dtype;
      break;
    }
  // (a stream of fewer bits than the branch has no use)
  if (p->dtype == EMB_FP32 && p->stream_dtype != EMB_FP32) return EMB_EINVAL;
  return EMB_OK;
}

}  // namespace

extern "C" {

emb_status emb_norm_fwd(int64_t rows, int32_t dim, const emb_norm* norm, const emb_mat* x, const emb_mat* residual,
                        const emb_mat* total, const emb_mat* y, const emb_mat* saved, void* stream) {
  NormLaunch p{};
  const emb_mat* const of[3] = {residual, total, nullptr};
  emb_status st = check_norm(rows, dim, norm, x, of, &p);
  if (st != EMB_OK || rows == 0) return st;
  if ((st = check_opt(x, dim, p.dtype, &p.x)) != EMB_OK) return st;
  if ((st = check_opt(residual, dim, p.stream_dtype, &p.residual)) != EMB_OK) return st;
  if ((st = check_opt(total, dim, p.stream_dtype, &p.total)) != EMB_OK) return st;
  if ((st = check_opt(y, dim, p.dtype, &p.y)) != EMB_OK) return st;
  if (saved != nullptr && saved->data != nullptr) {
    if ((st = check_mat(saved, dim, true)) != EMB_OK) return st;
    p.saved = rows_of(*saved);
  }
  if (p.y.p == nullptr && p.saved.p == nullptr) return EMB_EINVAL;
  p.aligned = p.aligned && vectors(p.x) && vectors(p.residual) && vectors(p.total) && vectors(p.y);
  return hip_status(launch_norm_fwd(p, (hipStream_t)stream));
}

size_t emb_norm_workspace_size(int64_t rows, int32_t dim) {
  if (rows < 0 || rows > kMaxTokens || dim < 1 || dim > kNormMaxDim) return 0;
  return norm_ws_bytes(rows, dim);
}

emb_status emb_norm_bwd(int64_t rows, int32_t dim, const emb_norm* norm, const emb_mat* total, const emb_mat* dy,
                        const emb_mat* arriving, const emb_mat* dtotal, const emb_mat* dbranch, float* dweight,
                        int32_t add, void* ws, size_t ws_bytes, void* stream) {
  NormLaunch p{};
  const emb_mat* const of[3] = {total, arriving, dtotal};
  emb_status st = check_norm(rows, dim, norm, dy, of, &p);
  if (st != EMB_OK) return st;
  if (dweight != nullptr) {
    if (((uintptr_t)dweight & 3u) != 0) return EMB_EINVAL;
    if (rows > 0 && ws == nullptr) return EMB_EINVAL;
    if (rows > 0 && (ws_bytes < norm_ws_bytes(rows, dim) || ((uintptr_t)ws & 255u) != 0)) return EMB_EWORKSPACE;
  }
  if (rows > 0) {
    if (total == nullptr || total->data == nullptr) return EMB_EINVAL;
    if ((st = check_opt(dy, dim, p.dtype, &p.dy)) != EMB_OK) return st;
    if ((st = check_opt(total, dim, p.stream_dtype, &p.total)) != EMB_OK) return st;
    if ((st = check_opt(arriving, dim, p.stream_dtype, &p.arriving)) != EMB_OK) return st;
    if ((st = check_opt(dtotal, dim, p.stream_dtype, &p.dtotal)) != EMB_OK) return st;
    if ((st = check_opt(dbranch, dim, p.dtype, &p.dbranch)) != EMB_OK) return st;
    p.aligned = p.aligned && vectors(p.total) && vectors(p.dy) && vectors(p.arriving) && vectors(p.dtotal) &&
                vectors(p.dbranch);
  }
  if (rows == 0 && dweight == nullptr) return EMB_OK;
  p.dweight = dweight;
  p.add = add != 0;
  p.ws = static_cast<float*>(ws);
  return hip_status(launch_norm_bwd(p, (hipStream_t)stream));
}

emb_status emb_dropout(int64_t rows, int32_t dim, float drop, uint64_t seed, int64_t first_row, const emb_mat* x,
                       const emb_mat* y, void* stream) {
  if (rows < 0 || dim < 1) return EMB_EINVAL;
  DropLaunch p{};
  emb_status st = check_drop(drop, seed, first_row, &p.drop);
  if (st != EMB_OK) return st;
  if (rows > kMaxTokens || rows * (int64_t)dim >= (int64_t)1 << 40) return EMB_EUNSUPPORTED;
  if (rows == 0) return EMB_OK;
  if ((st = check_mat(x, dim, false)) != EMB_OK) return st;
  if ((st = check_mat(y, dim, false)) != EMB_OK) return st;
  if (x->dtype != y->dtype) return EMB_EINVAL;
  p.N = rows;
  p.D = dim;
  p.dtype = x->dtype;
  p.x = rows_of(*x);
  p.y = rows_of(*y);
  p.aligned = vectors(p.x) && vectors(p.y);
  return hip_status(launch_dropout(p, (hipStream_t)stream));
}

}  // extern "C"
