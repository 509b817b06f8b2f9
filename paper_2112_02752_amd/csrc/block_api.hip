// C ABI of the operators of a model's block: host-side argument checks, kernel
// dispatch.  No allocation, no synchronisation.
#include <math.h>

#include <initializer_list>

#include "api_common.h"
#include "block_common.h"

using namespace emb;

namespace {

bool vectors(const Rows& r) { return (((uintptr_t)r.p | (uintptr_t)r.ld) & 15u) == 0; }

// whether an output over an input is not so row by row
bool across(int64_t rows, const Rows& out, std::initializer_list<Rows> in) {
  for (const Rows& r : in)
    if (rows > 1 && out.p != nullptr && out.p == r.p && out.ld != r.ld) return true;
  return false;
}

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

// (offsets within a chunk's rows are 32 bits)
bool long_rows(const Rows& r) { return r.ld > kMaxRowBytes; }

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

emb_status check_shape(int32_t heads, int32_t groups, int32_t dk, int32_t dv) {
  if (heads < 1 || groups < 1 || heads % groups != 0 || dk < 1 || dv < 1) return EMB_EINVAL;
  // (columns of a row are counted in 32 bits)
  if (dk > kLinMaxDim || dv > kLinMaxDim || heads > (1 << 20)) return EMB_EUNSUPPORTED;
  return EMB_OK;
}

emb_status check_heads(const emb_heads* h, LinLaunch* p) {
  if (h == nullptr || h->num_tokens < 0 || h->num_seqs < 0) return EMB_EINVAL;
  emb_status st = check_shape(h->heads, h->groups, h->dk, h->dv);
  if (st != EMB_OK) return st;
  if (h->num_tokens > kMaxTokens) return EMB_EUNSUPPORTED;
  if (h->num_tokens > 0 && h->num_seqs == 0) return EMB_EINVAL;
  if (h->offsets == nullptr || ((uintptr_t)h->offsets & 3u) != 0) return EMB_EINVAL;
  if (h->num_seqs > 0 && (h->decay == nullptr || ((uintptr_t)h->decay & 3u) != 0)) return EMB_EINVAL;
  if (((uintptr_t)h->first & 3u) != 0 || !isfinite(h->scale)) return EMB_EINVAL;
  p->N = h->num_tokens;
  p->M = h->num_seqs;
  p->heads = h->heads;
  p->groups = h->groups;
  p->dk = h->dk;
  p->dv = h->dv;
  p->offsets = h->offsets;
  p->decay = h->decay;
  p->scale = h->scale;
  p->first = h->first;
  if (h->num_tokens == 0) return EMB_OK;
  const emb_mat* all[3] = {&h->q, &h->k, &h->v};
  const int32_t cols[3] = {h->heads * h->dk, h->groups * h->dk, h->groups * h->dv};
  for (int i = 0; i < 3; ++i) {
    if ((st = check_mat(all[i], cols[i], false)) != EMB_OK) return st;
    if (all[i]->dtype != h->q.dtype) return EMB_EINVAL;
  }
  p->dtype = h->q.dtype;
  p->q = rows_of(h->q);
  p->k = rows_of(h->k);
  p->v = rows_of(h->v);
  if (long_rows(p->q) || long_rows(p->k) || long_rows(p->v)) return EMB_EUNSUPPORTED;
  const int size = dtype_bytes(p->dtype);
  p->aligned = vectors(p->q) && vectors(p->k) && vectors(p->v) && h->dk * size % 16 == 0 && h->dv * size % 16 == 0;
  return EMB_OK;
}

// whether a written matrix begins where one that is read does
bool meets(const Rows& out, const LinLaunch& p) {
  return out.p == p.q.p || out.p == p.k.p || out.p == p.v.p || (p.dy.p != nullptr && out.p == p.dy.p);
}

emb_status check_states(const LinLaunch& p, const void* at, size_t bytes) {
  const size_t need = lin_states_bytes(p.N, p.groups, p.dk, p.dv);
  if (need > 0 && at == nullptr) return EMB_EINVAL;
  return bytes < need || ((uintptr_t)at & 255u) != 0 ? EMB_EWORKSPACE : EMB_OK;
}

emb_status check_logits(int64_t rows, int32_t cols, const emb_mat* logits, const void* ids, int32_t id_bytes,
                        float scale, LogpLaunch* p) {
  if (rows < 0 || cols < 1 || !(scale > 0.f) || isinf(scale)) return EMB_EINVAL;
  if (id_bytes != 4 && id_bytes != 8) return EMB_EINVAL;
  if (((uintptr_t)ids & (uintptr_t)(id_bytes - 1)) != 0) return EMB_EINVAL;
  if (rows > kMaxTokens || cols > kLogpMaxCols) return EMB_EUNSUPPORTED;
  p->N = rows;
  p->D = cols;
  p->scale = scale;
  p->ids = ids;
  p->id_bytes = id_bytes;
  if (rows == 0) return EMB_OK;
  const emb_status st = check_mat(logits, cols, false);
  if (st != EMB_OK) return st;
  p->dtype = logits->dtype;
  p->logits = rows_of(*logits);
  return EMB_OK;
}

emb_status check_dlogits(const emb_mat* dlogits, LogpLaunch* p) {
  const emb_status st = check_mat(dlogits, p->D, false);
  if (st != EMB_OK) return st;
  if (dlogits->dtype != p->dtype) return EMB_EINVAL;
  p->dlogits = rows_of(*dlogits);
  // in place: row by row
  return across(p->N, p->dlogits, {p->logits}) ? EMB_EINVAL : EMB_OK;
}

bool words(const void* a, const void* b, const void* c = nullptr) {
  return (((uintptr_t)a | (uintptr_t)b | (uintptr_t)c) & 3u) == 0;
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
  if (across(rows, p.total, {p.x, p.residual}) || across(rows, p.y, {p.x, p.residual})) return EMB_EINVAL;
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
    for (const Rows& out : {p.dtotal, p.dbranch})
      if (across(rows, out, {p.total, p.dy, p.arriving})) return EMB_EINVAL;
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
  if (across(rows, p.y, {p.x})) return EMB_EINVAL;
  return hip_status(launch_dropout(p, (hipStream_t)stream));
}

size_t emb_linear_states_size(int64_t num_tokens, int32_t groups, int32_t dk, int32_t dv) {
  if (num_tokens < 0 || num_tokens > kMaxTokens || check_shape(groups, groups, dk, dv) != EMB_OK) return 0;
  return lin_states_bytes(num_tokens, groups, dk, dv);
}

emb_status emb_linear_fwd(const emb_heads* heads, const emb_mat* y, float* last, void* states, size_t states_bytes,
                          void* stream) {
  LinLaunch p{};
  emb_status st = check_heads(heads, &p);
  if (st != EMB_OK) return st;
  // (a sequence's last state may be written before its first is read)
  if (((uintptr_t)last & 3u) != 0 || (last != nullptr && last == heads->first)) return EMB_EINVAL;
  if (p.N > 0) {
    if ((st = check_mat(y, p.heads * p.dv, false)) != EMB_OK) return st;
    if (y->dtype != p.dtype) return EMB_EINVAL;
    p.y = rows_of(*y);
    if (long_rows(p.y)) return EMB_EUNSUPPORTED;
    if (meets(p.y, p)) return EMB_EINVAL;
    p.aligned = p.aligned && vectors(p.y);
  }
  if ((st = check_states(p, states, states_bytes)) != EMB_OK) return st;
  if (p.M == 0) return EMB_OK;
  p.last = last;
  p.states = static_cast<float*>(states);
  return hip_status(launch_lin_fwd(p, (hipStream_t)stream));
}

emb_status emb_linear_bwd(const emb_heads* heads, const void* states, size_t states_bytes, const emb_mat* dy,
                          const emb_mat* dq, const emb_mat* dk, const emb_mat* dv, const float* dlast, float* dfirst,
                          void* ws, size_t ws_bytes, void* stream) {
  LinLaunch p{};
  emb_status st = check_heads(heads, &p);
  if (st != EMB_OK) return st;
  if ((((uintptr_t)dlast | (uintptr_t)dfirst) & 3u) != 0) return EMB_EINVAL;
  if (dfirst != nullptr && (dfirst == dlast || dfirst == heads->first)) return EMB_EINVAL;
  if (p.N > 0) {
    const emb_mat* all[4] = {dy, dq, dk, dv};
    const int32_t cols[4] = {p.heads * p.dv, p.heads * p.dk, p.groups * p.dk, p.groups * p.dv};
    Rows* const to[4] = {&p.dy, &p.dq, &p.dkey, &p.dval};
    for (int i = 0; i < 4; ++i) {
      if ((st = check_mat(all[i], cols[i], false)) != EMB_OK) return st;
      if (all[i]->dtype != p.dtype) return EMB_EINVAL;
      *to[i] = rows_of(*all[i]);
      if (long_rows(*to[i])) return EMB_EUNSUPPORTED;
      if (i > 0 && meets(*to[i], p)) return EMB_EINVAL;
      p.aligned = p.aligned && vectors(*to[i]);
    }
  }
  if ((st = check_states(p, states, states_bytes)) != EMB_OK) return st;
  if ((st = check_states(p, ws, ws_bytes)) != EMB_OK) return st;
  if (ws != nullptr && ws == states) return EMB_EINVAL;
  if (p.M == 0) return EMB_OK;
  p.dlast = dlast;
  p.dfirst = dfirst;
  p.states = static_cast<float*>(const_cast<void*>(states));
  p.grads = static_cast<float*>(ws);
  return hip_status(launch_lin_bwd(p, (hipStream_t)stream));
}

emb_status emb_linear_step(int64_t num_tokens, int32_t heads, int32_t groups, int32_t dk, int32_t dv, const emb_mat* q,
                           const emb_mat* k, const emb_mat* v, const float* decay, float scale, float* state,
                           int64_t num_slots, const int32_t* slots, const emb_mat* y, void* stream) {
  if (num_tokens < 0 || num_slots < 0 || !isfinite(scale)) return EMB_EINVAL;
  emb_status st = check_shape(heads, groups, dk, dv);
  if (st != EMB_OK) return st;
  if (num_tokens > kMaxTokens) return EMB_EUNSUPPORTED;
  if (num_tokens == 0) return EMB_OK;
  if (decay == nullptr || (num_slots > 0 && state == nullptr)) return EMB_EINVAL;
  if ((((uintptr_t)decay | (uintptr_t)state | (uintptr_t)slots) & 3u) != 0) return EMB_EINVAL;
  const emb_mat* all[4] = {q, k, v, y};
  const int32_t cols[4] = {heads * dk, groups * dk, groups * dv, heads * dv};
  LinStepLaunch p{};
  Rows* const to[4] = {&p.q, &p.k, &p.v, &p.y};
  for (int i = 0; i < 4; ++i) {
    if ((st = check_mat(all[i], cols[i], false)) != EMB_OK) return st;
    if (all[i]->dtype != q->dtype) return EMB_EINVAL;
    *to[i] = rows_of(*all[i]);
  }
  // (blocks of a token's other heads read its rows)
  if (p.y.p == p.q.p || p.y.p == p.k.p || p.y.p == p.v.p) return EMB_EINVAL;
  p.N = num_tokens;
  p.num_slots = num_slots;
  p.heads = heads;
  p.groups = groups;
  p.dk = dk;
  p.dv = dv;
  p.dtype = q->dtype;
  p.scale = scale;
  p.decay = decay;
  p.state = state;
  p.slots = slots;
  return hip_status(launch_lin_step(p, (hipStream_t)stream));
}

emb_status emb_logp_fwd(int64_t rows, int32_t cols, const emb_mat* logits, const void* ids, int32_t id_bytes,
                        float scale, float* logp, float* entropy, int32_t top, int32_t* top_ids, float* top_logp,
                        float* stats, void* stream) {
  LogpLaunch p{};
  const emb_status st = check_logits(rows, cols, logits, ids, id_bytes, scale, &p);
  if (st != EMB_OK) return st;
  if (top < 0 || top > cols) return EMB_EINVAL;
  if (top > EMB_MAX_TOP) return EMB_EUNSUPPORTED;
  if (!words(logp, entropy) || !words(top_ids, top_logp) || ((uintptr_t)stats & 15u) != 0) return EMB_EINVAL;
  if (rows == 0) return EMB_OK;
  if ((ids == nullptr) != (logp == nullptr)) return EMB_EINVAL;
  if (top > 0 && (top_ids == nullptr || top_logp == nullptr)) return EMB_EINVAL;
  p.logp = logp;
  p.entropy = entropy;
  p.top = top;
  p.top_ids = top_ids;
  p.top_logp = top_logp;
  p.stats = stats;
  return hip_status(launch_logp(p, (hipStream_t)stream));
}

emb_status emb_logp_bwd(int64_t rows, int32_t cols, const emb_mat* logits, const void* ids, int32_t id_bytes,
                        float scale, const float* stats, const float* dlogp, const float* dentropy,
                        const emb_mat* dlogits, void* stream) {
  LogpLaunch p{};
  emb_status st = check_logits(rows, cols, logits, ids, id_bytes, scale, &p);
  if (st != EMB_OK) return st;
  if (!words(dlogp, dentropy) || ((uintptr_t)stats & 15u) != 0) return EMB_EINVAL;
  if (rows == 0) return EMB_OK;
  if (stats == nullptr || (ids == nullptr) != (dlogp == nullptr)) return EMB_EINVAL;
  if ((st = check_dlogits(dlogits, &p)) != EMB_OK) return st;
  p.stats = const_cast<float*>(stats);
  p.dlogp = dlogp;
  p.dentropy = dentropy;
  return hip_status(launch_logp_bwd(p, (hipStream_t)stream));
}

emb_status emb_logp_train(int64_t rows, int32_t cols, const emb_mat* logits, const void* ids, int32_t id_bytes,
                          float scale, const float* dlogp, float* logp, float* entropy, const emb_mat* dlogits,
                          void* stream) {
  LogpLaunch p{};
  emb_status st = check_logits(rows, cols, logits, ids, id_bytes, scale, &p);
  if (st != EMB_OK) return st;
  if (!words(dlogp, logp, entropy)) return EMB_EINVAL;
  if (rows == 0) return EMB_OK;
  if (ids == nullptr || dlogp == nullptr || dlogp == logp || dlogp == entropy) return EMB_EINVAL;
  if ((st = check_dlogits(dlogits, &p)) != EMB_OK) return st;
  p.dlogp = dlogp;
  p.logp = logp;
  p.entropy = entropy;
  return hip_status(launch_logp(p, (hipStream_t)stream));
}

}  // extern "C"
