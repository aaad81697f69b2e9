// Host side of the high-precision entry points: argument validation.  As in the rest of the library nothing here allocates, synchronizes or
// keeps state.
#include "hp_common.h"

#include <cmath>

int hp_launch_norm_fwd(const hp_norm* n, int bf16, int64_t M, int64_t D, const void* x, int64_t ldx, const void* block, int64_t ldb, void* h, int64_t ldh,
                       void* y, int64_t ldy, float* r_before, float* r_after, hipStream_t s);
int hp_launch_norm_bwd(const hp_norm* n, int bf16, int64_t M, int64_t D, const void* dy, int64_t ld_dy, const void* dh, int64_t ld_dh, const void* h,
                       int64_t ldh, const void* block, int64_t ldb, const float* r_before, const float* r_after, void* dx, int64_t ld_dx, void* dblock,
                       int64_t ld_db, void* dgate, int64_t ld_dg, float* dw_before, float* dw_after, int accumulate, float* part, hipStream_t s);
size_t hp_norm_bwd_part(int64_t M, int64_t D);
int hp_launch_embed_fwd(const int64_t* ids, int bf16, int64_t M, int64_t D, int64_t V, const void* table, int64_t ldt, float scale, void* y, int64_t ldy,
                        hipStream_t s);
int hp_launch_embed_bwd(const int64_t* ids, int bf16, int64_t M, int64_t D, int64_t V, const void* dy, int64_t ld_dy, float scale, int accumulate,
                        float* table, int64_t ldt, void* workspace, hipStream_t s);
size_t hp_embed_bwd_room(int64_t M, int64_t D);
int hp_launch_head_fwd(const uint16_t* x, const uint16_t* w, const int64_t* targets, int64_t M, int64_t D, int64_t V, int64_t ldx, int64_t ldw, float* loss,
                       float* lse, void* workspace, hipStream_t s);
int hp_launch_head_bwd(const uint16_t* x, const uint16_t* w, const int64_t* targets, const float* lse, const float* dloss, int64_t M, int64_t D, int64_t V,
                       int64_t ldx, int64_t ldw, uint16_t* dx, int64_t ld_dx, void* dw, int dw_bf16, int64_t ld_dw, int accumulate, void* workspace,
                       hipStream_t s);
size_t hp_head_fwd_room(int64_t M, int64_t V);
size_t hp_head_bwd_room(int64_t M, int64_t D, int64_t V);

namespace {

bool dtype_ok(int dt) { return dt == FP4_F32 || dt == FP4_BF16; }
bool dims_ok(int64_t a, int64_t b, int64_t c) { return a >= 0 && b >= 0 && c >= 0; }
bool within(int64_t a, int64_t b, int64_t c) { return a <= HP_MAX_DIM && b <= HP_MAX_DIM && c <= HP_MAX_DIM; }

// A matrix that is there; `wanted`: whether it has to be.
int check_matrix(const void* x, int64_t rows, int64_t cols, int64_t ld, bool wanted) {
  if (!x) return wanted && rows > 0 && cols > 0 ? FP4_ERR_NULL : FP4_OK;
  if (ld < cols) return FP4_ERR_SHAPE;
  return aligned16(x) && ld % 8 == 0 ? FP4_OK : FP4_ERR_ARG;
}
int check_vector(const void* x, bool wanted) {
  if (!x) return wanted ? FP4_ERR_NULL : FP4_OK;
  return aligned16(x) ? FP4_OK : FP4_ERR_ARG;
}

int check_norm(const hp_norm* n, int dt, int64_t M, int64_t D, const void* block) {
  if (!n) return FP4_ERR_NULL;
  if (!dtype_ok(dt)) return FP4_ERR_DTYPE;
  if (!dims_ok(M, D, 0)) return FP4_ERR_SHAPE;
  if (!within(M, 0, 0) || D > HP_NORM_MAX_D) return FP4_ERR_LIMIT;
  if (!(n->eps > 0.0f) || !std::isfinite(n->eps) || !std::isfinite(n->scale)) return FP4_ERR_ARG;
  if (!block && M > 0 && (n->w_after || n->gate)) return FP4_ERR_ARG;
  int rc = check_vector(n->w_before, false);
  if (!rc) rc = check_vector(n->w_after, false);
  if (!rc) rc = n->ld_gate == 0 ? check_vector(n->gate, false) : check_matrix(n->gate, M, D, n->ld_gate, false);
  return rc;
}

}  // namespace

size_t hp_workspace_bytes(int op, int64_t M, int64_t D, int64_t V) {
  if (op == FP4_OP_HP_NORM_BWD) return hp_norm_bwd_part(M, D) + 256;
  if (op == FP4_OP_HP_EMBED_BWD) return hp_embed_bwd_room(M, D);
  return op == FP4_OP_HP_HEAD_FWD ? hp_head_fwd_room(M, V) : hp_head_bwd_room(M, D, V);
}

extern "C" int hp_norm_fwd(const hp_norm* norm, fp4_dtype dt, int64_t M, int64_t D, const void* x, int64_t ldx, const void* block, int64_t ld_block, void* h,
                           int64_t ldh, void* y, int64_t ldy, float* r_before, float* r_after, void* stream) {
  int rc = check_norm(norm, dt, M, D, block);
  if (rc) return rc;
  if (!h && !y && M > 0 && D > 0) return FP4_ERR_NULL;
  if ((y || r_before) && !norm->w_before && D > 0) return FP4_ERR_NULL;
  if (!rc) rc = check_matrix(x, M, D, ldx, true);
  if (!rc) rc = check_matrix(block, M, D, ld_block, false);
  if (!rc) rc = check_matrix(h, M, D, ldh, false);
  if (!rc) rc = check_matrix(y, M, D, ldy, false);
  if (rc || M == 0 || D == 0) return rc;
  return hp_launch_norm_fwd(norm, dt == FP4_BF16, M, D, x, ldx, block, ld_block, h, ldh, y, ldy, r_before, r_after, (hipStream_t)stream);
}

extern "C" int hp_norm_bwd(const hp_norm* norm, fp4_dtype dt, int64_t M, int64_t D, const void* dy, int64_t ld_dy, const void* dh, int64_t ld_dh, const void* h,
                           int64_t ldh, const void* block, int64_t ld_block, const float* r_before, const float* r_after, void* dx, int64_t ld_dx,
                           void* dblock, int64_t ld_dblock, void* dgate, int64_t ld_dgate, float* dw_before, float* dw_after, int accumulate, void* workspace,
                           size_t workspace_bytes, void* stream) {
  int rc = check_norm(norm, dt, M, D, block);
  if (rc) return rc;
  const bool any = M > 0 && D > 0;
  if (any && !dy && !dh) return FP4_ERR_NULL;
  if (any && dy && (!norm->w_before || !h || !r_before)) return FP4_ERR_NULL;
  if (any && dw_before && !dy) return FP4_ERR_NULL;
  if (any && (dblock || dgate || dw_after) && !block) return FP4_ERR_NULL;
  if (dgate && !norm->gate && D > 0) return FP4_ERR_NULL;
  if (dw_after && !norm->w_after && D > 0) return FP4_ERR_NULL;
  if (any && norm->w_after && !r_after) return FP4_ERR_NULL;
  if (!rc) rc = check_matrix(dy, M, D, ld_dy, false);
  if (!rc) rc = check_matrix(dh, M, D, ld_dh, false);
  if (!rc) rc = check_matrix(h, M, D, ldh, false);
  if (!rc) rc = check_matrix(block, M, D, ld_block, false);
  if (!rc) rc = check_matrix(dx, M, D, ld_dx, false);
  if (!rc) rc = check_matrix(dblock, M, D, ld_dblock, false);
  if (!rc && dgate && norm->ld_gate) rc = check_matrix(dgate, M, D, ld_dgate, false);
  if (!rc) rc = check_vector(dw_before, false);
  if (!rc) rc = check_vector(dw_after, false);
  if (!rc && norm->ld_gate == 0) rc = check_vector(dgate, false);
  if (rc || D == 0) return rc;
  if (!workspace || workspace_bytes < hp_workspace_bytes(FP4_OP_HP_NORM_BWD, M, D, 0)) return FP4_ERR_WORKSPACE;
  return hp_launch_norm_bwd(norm, dt == FP4_BF16, M, D, dy, ld_dy, dh, ld_dh, h, ldh, block, ld_block, r_before, r_after, dx, ld_dx, dblock, ld_dblock, dgate,
                            ld_dgate, dw_before, dw_after, accumulate, (float*)align_up((size_t)(uintptr_t)workspace, 256), (hipStream_t)stream);
}

extern "C" int hp_embed_fwd(const int64_t* ids, fp4_dtype dt, int64_t M, int64_t D, int64_t V, const void* table, int64_t ld_table, float scale, void* y,
                            int64_t ldy, void* stream) {
  if (!dtype_ok(dt)) return FP4_ERR_DTYPE;
  if (!dims_ok(M, D, V)) return FP4_ERR_SHAPE;
  if (!within(M, D, V)) return FP4_ERR_LIMIT;
  if (!ids && M > 0 && D > 0) return FP4_ERR_NULL;
  if (!std::isfinite(scale)) return FP4_ERR_ARG;
  int rc = check_matrix(table, V, D, ld_table, M > 0);
  if (!rc) rc = check_matrix(y, M, D, ldy, true);
  if (rc || M == 0 || D == 0) return rc;
  return hp_launch_embed_fwd(ids, dt == FP4_BF16, M, D, V, table, ld_table, scale, y, ldy, (hipStream_t)stream);
}

extern "C" int hp_embed_bwd(const int64_t* ids, fp4_dtype dt, int64_t M, int64_t D, int64_t V, const void* dy, int64_t ld_dy, float scale, int accumulate,
                            float* dtable, int64_t ld_dtable, void* workspace, size_t workspace_bytes, void* stream) {
  if (!dtype_ok(dt)) return FP4_ERR_DTYPE;
  if (!dims_ok(M, D, V)) return FP4_ERR_SHAPE;
  if (!within(M, D, V)) return FP4_ERR_LIMIT;
  if (!ids && M > 0 && D > 0) return FP4_ERR_NULL;
  if (!std::isfinite(scale)) return FP4_ERR_ARG;
  int rc = check_matrix(dy, M, D, ld_dy, true);
  if (!rc) rc = check_matrix(dtable, V, D, ld_dtable, true);
  if (rc || V == 0 || D == 0) return rc;
  if (!workspace || workspace_bytes < hp_workspace_bytes(FP4_OP_HP_EMBED_BWD, M, D, V)) return FP4_ERR_WORKSPACE;
  return hp_launch_embed_bwd(ids, dt == FP4_BF16, M, D, V, dy, ld_dy, scale, accumulate, dtable, ld_dtable, workspace, (hipStream_t)stream);
}

namespace {
int check_head(const void* x, const void* w, const int64_t* targets, int dt, int64_t M, int64_t D, int64_t V, int64_t ldx, int64_t ldw) {
  if (dt != FP4_BF16) return FP4_ERR_DTYPE;
  if (!dims_ok(M, D, V) || V == 0 || D % 8 != 0) return FP4_ERR_SHAPE;
  if (!within(M, D, V) || ldx > HP_MAX_DIM || ldw > HP_MAX_DIM) return FP4_ERR_LIMIT;
  if (!targets && M > 0) return FP4_ERR_NULL;
  const int rc = check_matrix(x, M, D, ldx, true);
  return rc ? rc : check_matrix(w, V, D, ldw, true);
}
}  // namespace

extern "C" int hp_head_fwd(const void* x, const void* w, const int64_t* targets, fp4_dtype dt, int64_t M, int64_t D, int64_t V, int64_t ldx, int64_t ldw,
                           float* loss, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_head(x, w, targets, dt, M, D, V, ldx, ldw);
  if (rc || M == 0) return rc;
  if (!loss && !lse) return FP4_ERR_NULL;
  if (!workspace || workspace_bytes < hp_workspace_bytes(FP4_OP_HP_HEAD_FWD, M, D, V)) return FP4_ERR_WORKSPACE;
  return hp_launch_head_fwd((const uint16_t*)x, (const uint16_t*)w, targets, M, D, V, ldx, ldw, loss, lse, workspace, (hipStream_t)stream);
}

extern "C" int hp_head_bwd(const void* x, const void* w, const int64_t* targets, const float* lse, const float* dloss, fp4_dtype dt, int64_t M, int64_t D,
                           int64_t V, int64_t ldx, int64_t ldw, void* dx, int64_t ld_dx, void* dw, fp4_dtype dw_dt, int64_t ld_dw, int accumulate,
                           void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_head(x, w, targets, dt, M, D, V, ldx, ldw);
  if (rc) return rc;
  if (!dx && !dw && M > 0 && D > 0) return FP4_ERR_NULL;   // what is empty has no address
  if (M > 0 && (!lse || !dloss)) return FP4_ERR_NULL;
  if (!dtype_ok(dw_dt)) return FP4_ERR_DTYPE;
  if (dw && accumulate && dw_dt != FP4_F32) return FP4_ERR_ARG;
  if (!rc) rc = check_matrix(dx, M, D, ld_dx, false);
  if (!rc) rc = check_matrix(dw, V, D, ld_dw, false);
  if (rc || D == 0) return rc;
  if (!workspace || workspace_bytes < hp_workspace_bytes(FP4_OP_HP_HEAD_BWD, M, D, V)) return FP4_ERR_WORKSPACE;
  return hp_launch_head_bwd((const uint16_t*)x, (const uint16_t*)w, targets, lse, dloss, M, D, V, ldx, ldw, (uint16_t*)dx, ld_dx, dw, dw_dt == FP4_BF16, ld_dw,
                            accumulate, workspace, (hipStream_t)stream);
}
