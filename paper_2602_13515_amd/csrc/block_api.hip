// Entry points of the operators around the block-sparse attention: argument checks, then the launches.
#include "block_ops.h"
#include "cross_check.h"

using namespace spa2;

namespace {

bool strides_ok(int64_t sb, int64_t sh, int64_t sn) { return sb >= 0 && sh >= 0 && sn >= 0; }

int check_norm_shape(const spa2_norm_shape* s) {
  if (!s) return SPA2_ERR_NULL;
  if (s->B <= 0 || s->Hq <= 0 || s->Hk <= 0 || s->N <= 0 || s->d <= 0) return SPA2_ERR_SHAPE;
  if (s->d != 64 && s->d != 128) return SPA2_ERR_UNSUPPORTED;
  if (s->dtype != SPA2_DTYPE_BF16 && s->dtype != SPA2_DTYPE_F32) return SPA2_ERR_UNSUPPORTED;
  if (s->rot < 0 || s->rot > s->d || s->rot % 16) return SPA2_ERR_UNSUPPORTED;
  if (s->pos_bits != 0 && s->pos_bits != 32 && s->pos_bits != 64) return SPA2_ERR_UNSUPPORTED;
  // tokens are numbered in 32 bits
  if ((int64_t)s->B * s->N > (int64_t)1 << 30 || s->Hq > 1 << 20 || s->Hk > 1 << 20) return SPA2_ERR_SHAPE;
  if (s->rot && (s->table_rows <= 0 || (s->pos_bits == 0 && s->table_rows < s->N))) return SPA2_ERR_SHAPE;
  if (s->pos_sb < 0 || !strides_ok(s->q_sb, s->q_sh, s->q_sn) || !strides_ok(s->k_sb, s->k_sh, s->k_sn)) return SPA2_ERR_SHAPE;
  if (!strides_ok(s->qo_sb, s->qo_sh, s->qo_sn) || !strides_ok(s->ko_sb, s->ko_sh, s->ko_sn)) return SPA2_ERR_SHAPE;
  const int64_t in = s->dtype == SPA2_DTYPE_BF16 ? 8 : 4;
  if (s->q_sb % in || s->q_sh % in || s->q_sn % in || s->k_sb % in || s->k_sh % in || s->k_sn % in) return SPA2_ERR_ALIGN;
  if (s->qo_sb % 8 || s->qo_sh % 8 || s->qo_sn % 8 || s->ko_sb % 8 || s->ko_sh % 8 || s->ko_sn % 8) return SPA2_ERR_ALIGN;
  return SPA2_OK;
}

int check_norm(const void* q, const void* k, const float* q_weight, const float* k_weight, const float* cos, const float* sin,
               const void* positions, const spa2_norm_shape* s, float eps) {
  const int rc = check_norm_shape(s);
  if (rc != SPA2_OK) return rc;
  if (!q || !k || (s->rot && (!cos || !sin)) || (s->pos_bits && !positions)) return SPA2_ERR_NULL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(q_weight) || !aligned16(k_weight) || !aligned16(cos) || !aligned16(sin))
    return SPA2_ERR_ALIGN;
  if ((uintptr_t)positions % (s->pos_bits == 64 ? 8 : 4)) return SPA2_ERR_ALIGN;
  if (!(eps > 0.f) || !isfinite(eps)) return SPA2_ERR_RANGE;
  return SPA2_OK;
}

bool dtype_ok(int32_t t) { return t == SPA2_DTYPE_BF16 || t == SPA2_DTYPE_F32; }

uint32_t dropout_cut(double p) { return (uint32_t)floor(p * 65536.0 + 0.5); }

size_t cross_fwd_bytes(const CrossDims& m) { return cross_few(m) ? cross_few_ws(m).total : cross_fwd_ws(m).total; }

int check_cross(const void* q, const void* k, const void* v, const int32_t* lengths, const void* o, const void* o_res,
                const float* lse, const spa2_cross_shape* shape, float scale) {
  const int rc = check_cross_shape(shape);
  if (rc != SPA2_OK) return rc;
  if (!q || !k || !v || !o || !lse) return SPA2_ERR_NULL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) || !aligned16(o_res) || (uintptr_t)lengths % 4 ||
      (uintptr_t)lse % 4)
    return SPA2_ERR_ALIGN;
  if (!(scale > 0.f) || !isfinite(scale)) return SPA2_ERR_RANGE;
  return SPA2_OK;
}

}  // namespace

extern "C" {

size_t spa2_cross_fwd_workspace_bytes(const spa2_cross_shape* shape) {
  if (check_cross_shape(shape) != SPA2_OK) return 0;
  return cross_fwd_bytes(cross_dims(*shape));
}

size_t spa2_cross_bwd_workspace_bytes(const spa2_cross_shape* shape) {
  if (check_cross_shape(shape) != SPA2_OK) return 0;
  return cross_bwd_ws(cross_dims(*shape)).total;
}

int spa2_cross_fwd(const void* q, const void* k, const void* v, const int32_t* lengths, const spa2_cross_shape* shape,
                   float scale, void* o, void* o_res, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_cross(q, k, v, lengths, o, o_res, lse, shape, scale);
  if (rc != SPA2_OK) return rc;
  const CrossDims m = cross_dims(*shape);
  const size_t need = cross_fwd_bytes(m);
  if (need && (!workspace || workspace_bytes < need)) return SPA2_ERR_WORKSPACE;
  if (need && !aligned16(workspace)) return SPA2_ERR_ALIGN;
  return (cross_few(m) ? launch_cross_few : launch_cross_fwd)(q, k, v, m, lengths, scale, o, o_res, lse, workspace,
                                                             (hipStream_t)stream) == hipSuccess ? SPA2_OK : SPA2_ERR_LAUNCH;
}

int spa2_cross_bwd(const void* q, const void* k, const void* v, const int32_t* lengths, const void* o, const void* o_res,
                   const void* d_o, const float* lse, const spa2_cross_shape* shape, float scale, void* dq, void* dk, void* dv,
                   void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_cross(q, k, v, lengths, o, o_res, lse, shape, scale);
  if (rc == SPA2_OK) rc = check_strides(shape->d_sb, shape->d_sh, shape->d_sn, 1, shape->d);
  if (rc != SPA2_OK) return rc;
  if (!d_o || !dq || !dk || !dv) return SPA2_ERR_NULL;
  if (!aligned16(d_o) || !aligned16(dq) || !aligned16(dk) || !aligned16(dv)) return SPA2_ERR_ALIGN;
  const CrossDims m = cross_dims(*shape);
  const CrossBwdWs w = cross_bwd_ws(m);
  if (!workspace || workspace_bytes < w.total) return SPA2_ERR_WORKSPACE;
  if (!aligned16(workspace)) return SPA2_ERR_ALIGN;
  char* ws = (char*)workspace;
  float *delta = (float*)ws, *lse_again = (float*)(ws + w.lse);
  hipStream_t st = (hipStream_t)stream;
  const SplitPlan cols = cross_plan(w.dkdv, ws + w.dkdv_counters, ws + w.dkdv_pool, dkdv_slot_bytes(m.q));
  const SplitPlan rows = cross_plan(w.dq, nullptr, ws + w.dq_pool, dq_slot_bytes(m.q));
  if (launch_cross_dq(q, k, v, o, o_res, d_o, lse, m, lengths, scale, delta, lse_again, dq, cols.arrive, w.dkdv.slots, rows,
                      st) != hipSuccess)
    return SPA2_ERR_LAUNCH;
  return launch_cross_dkdv(q, k, v, d_o, lse_again, delta, m, lengths, scale, dk, dv, cols, st) == hipSuccess ? SPA2_OK : SPA2_ERR_LAUNCH;
}

size_t spa2_norm_rotate_bwd_workspace_bytes(const spa2_norm_shape* shape) {
  if (check_norm_shape(shape) != SPA2_OK) return 0;
  return round256(norm_rotate_partials_bytes(*shape));
}

int spa2_norm_rotate(const void* q, const void* k, const float* q_weight, const float* k_weight, const float* cos,
                     const float* sin, const void* positions, const spa2_norm_shape* shape, float eps, void* q_out,
                     void* k_out, void* stream) {
  const int rc = check_norm(q, k, q_weight, k_weight, cos, sin, positions, shape, eps);
  if (rc != SPA2_OK) return rc;
  if (!q_out || !k_out) return SPA2_ERR_NULL;
  if (!aligned16(q_out) || !aligned16(k_out)) return SPA2_ERR_ALIGN;
  const NormTables t = {cos, sin, shape->pos_bits ? positions : nullptr};
  return launch_norm_rotate(q, k, q_weight, k_weight, t, *shape, eps, q_out, k_out, (hipStream_t)stream) == hipSuccess
             ? SPA2_OK : SPA2_ERR_LAUNCH;
}

int spa2_norm_rotate_bwd(const void* q, const void* k, const float* q_weight, const float* k_weight, const float* cos,
                         const float* sin, const void* positions, const void* d_q_out, const void* d_k_out,
                         const spa2_norm_shape* shape, float eps, void* dq, void* dk, float* d_q_weight,
                         float* d_k_weight, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_norm(q, k, q_weight, k_weight, cos, sin, positions, shape, eps);
  if (rc != SPA2_OK) return rc;
  if (!d_q_out || !d_k_out || !dq || !dk) return SPA2_ERR_NULL;
  if (!aligned16(d_q_out) || !aligned16(d_k_out) || !aligned16(dq) || !aligned16(dk)) return SPA2_ERR_ALIGN;
  if (d_q_weight || d_k_weight) {
    if (!workspace || workspace_bytes < norm_rotate_partials_bytes(*shape)) return SPA2_ERR_WORKSPACE;
    if (!aligned16(workspace)) return SPA2_ERR_ALIGN;
  }
  const NormTables t = {cos, sin, shape->pos_bits ? positions : nullptr};
  return launch_norm_rotate_bwd(q, k, q_weight, k_weight, t, d_q_out, d_k_out, *shape, eps, dq, dk, d_q_weight, d_k_weight,
                                workspace, (hipStream_t)stream) == hipSuccess ? SPA2_OK : SPA2_ERR_LAUNCH;
}

int spa2_dropout_add(const void* x, const void* residual, int64_t n, int32_t x_dtype, int32_t residual_dtype, double p,
                     uint64_t seed, uint64_t offset, const int64_t* seed_offset, void* y, void* stream) {
  if (!x || !y) return SPA2_ERR_NULL;
  if (n <= 0) return SPA2_ERR_SHAPE;
  if (!dtype_ok(x_dtype)) return SPA2_ERR_UNSUPPORTED;
  if (residual && residual_dtype != x_dtype && residual_dtype != SPA2_DTYPE_F32) return SPA2_ERR_UNSUPPORTED;
  if (!aligned16(x) || !aligned16(residual) || !aligned16(y) || (uintptr_t)seed_offset % 8) return SPA2_ERR_ALIGN;
  if (!(p >= 0.0) || !(p <= 1.0)) return SPA2_ERR_RANGE;
  return launch_dropout(x, x_dtype, residual, residual_dtype, n, dropout_cut(p), seed, offset, seed_offset, y,
                        residual ? residual_dtype : x_dtype, (hipStream_t)stream) == hipSuccess ? SPA2_OK : SPA2_ERR_LAUNCH;
}

int spa2_dropout_bwd(const void* d_y, int64_t n, int32_t y_dtype, int32_t x_dtype, double p, uint64_t seed, uint64_t offset,
                     const int64_t* seed_offset, void* dx, void* stream) {
  if (!d_y || !dx) return SPA2_ERR_NULL;
  if (n <= 0) return SPA2_ERR_SHAPE;
  if (!dtype_ok(x_dtype) || (y_dtype != x_dtype && y_dtype != SPA2_DTYPE_F32)) return SPA2_ERR_UNSUPPORTED;
  if (!aligned16(d_y) || !aligned16(dx) || (uintptr_t)seed_offset % 8) return SPA2_ERR_ALIGN;
  if (!(p >= 0.0) || !(p <= 1.0)) return SPA2_ERR_RANGE;
  return launch_dropout(d_y, y_dtype, nullptr, 0, n, dropout_cut(p), seed, offset, seed_offset, dx, x_dtype,
                        (hipStream_t)stream) == hipSuccess ? SPA2_OK : SPA2_ERR_LAUNCH;
}

}  // extern "C"
