// C entry points of include/act8.h: checks of the arguments, then the launches.
#include "act8_internal.h"
#include "run_internal.h"

#include <cmath>

using namespace sl;

namespace {

constexpr int64_t LD_MAX = 1LL << 40;

bool act8_ok(const slide_act8* a) {
  return a && a->codes && a->scales && a->rows >= 1 && a->cols >= 1 && a->rows <= A8_MAX_ROWS && a->cols <= A8_MAX_COLS &&
         ((uintptr_t)a->codes & 15) == 0 && a->ldc % A8_GRAIN == 0 && a->ldc >= a->cols && a->ldc <= LD_MAX &&
         a->lds >= (a->cols + A8_BLOCK - 1) / A8_BLOCK && a->lds <= LD_MAX;
}
bool dtype_ok(int dt) { return dt == DT_F32 || dt == DT_BF16; }
// a matrix of dtype dt with rows of `cols` elements
bool matrix_ok(const void* p, int dt, int64_t ld, int64_t cols) {
  return p && ((uintptr_t)p & (elem_size(dt) - 1)) == 0 && ld >= cols && ld <= LD_MAX;
}
// two matrices of `rows` rows that share no memory
bool apart(const void* a, int64_t lda, int64_t ca, const void* b, int64_t ldb, int64_t cb, int64_t rows, size_t es) {
  const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b, a1 = a0 + ((rows - 1) * lda + ca) * es, b1 = b0 + ((rows - 1) * ldb + cb) * es;
  return a1 <= b0 || b1 <= a0;
}
bool floats_ok(const void* p) { return p && ((uintptr_t)p & 3) == 0; }

int work_ok(const void* work, size_t have, size_t need) {
  if (!work || have < need) return SLIDE_EARENA;
  return ((uintptr_t)work & 255) == 0 ? SLIDE_OK : SLIDE_EINVAL;
}

int status(hipError_t e) {
  if (e == hipSuccess) return SLIDE_OK;
  g_last_hip = (int)e;
  return SLIDE_EHIP;
}

bool norm_ok(const slide_group_norm* s) {
  return s && s->n >= 1 && s->hw >= 1 && s->n <= A8_MAX_ROWS && s->hw <= A8_MAX_ROWS && s->n * s->hw <= A8_MAX_ROWS &&
         s->channels >= 1 && s->channels <= 65536 && s->groups >= 1 && s->channels % s->groups == 0 && dtype_ok(s->dtype) &&
         s->act >= SLIDE_ACT_NONE && s->act <= SLIDE_ACT_GELU && s->eps > 0.f && std::isfinite(s->eps) && s->reserved == 0;
}

}  // namespace

extern "C" {

int slide_act8_pack(const void* x, int dtype, int64_t ldx, int transpose, const slide_act8* out, void* stream) {
  if (!act8_ok(out) || !dtype_ok(dtype) || !matrix_ok(x, dtype, ldx, transpose ? out->rows : out->cols)) return SLIDE_EINVAL;
  (void)hipGetLastError();
  return status(launch_act8_pack(x, dtype, ldx, transpose != 0, *out, (hipStream_t)stream));
}

int slide_act8_unpack(const slide_act8* a, void* y, int dtype, int64_t ldy, void* stream) {
  if (!act8_ok(a) || !dtype_ok(dtype) || !matrix_ok(y, dtype, ldy, a->cols)) return SLIDE_EINVAL;
  (void)hipGetLastError();
  return status(launch_act8_unpack(*a, y, dtype, ldy, (hipStream_t)stream));
}

int slide_act8_linear(const void* x, int dtype, int64_t ldx, const slide_act8* x8, const slide_act8* w8, const float* bias,
                      int act, const void* residual, int64_t ldr, void* y, int64_t ldy, void* stream) {
  if (!act8_ok(x8) || !act8_ok(w8) || !dtype_ok(dtype) || x8->cols != w8->cols) return SLIDE_EINVAL;
  if (act < SLIDE_ACT_NONE || act > SLIDE_ACT_GELU) return SLIDE_EINVAL;
  const int64_t out = w8->rows;
  if ((x && !matrix_ok(x, dtype, ldx, x8->cols)) || (bias && !floats_ok(bias)) || !matrix_ok(y, dtype, ldy, out)) return SLIDE_EINVAL;
  if (residual && (!matrix_ok(residual, dtype, ldr, out) || (residual == y && ldr != ldy))) return SLIDE_EINVAL;
  if (out > A8_MAX_COLS) return SLIDE_EUNSUPPORTED;
  (void)hipGetLastError();
  // Packed inside the product, every workgroup reads x for itself: not where y (a residual stream updated in place) lies on it.
  const bool fused = x && apart(x, ldx, x8->cols, y, ldy, out, x8->rows, elem_size(dtype));
  if (x && !fused) {
    const int rc = status(launch_act8_pack(x, dtype, ldx, false, *x8, (hipStream_t)stream));
    if (rc) return rc;
  }
  A8Linear g{};
  if (fused) { g.xin = x; g.ldxin = ldx; }
  g.x = a8_view(*x8); g.w = a8_view(*w8);
  g.M = x8->rows; g.N = (int)out; g.K = (int)x8->cols;
  g.bias = bias; g.act = act; g.dt = dtype; g.resid = residual; g.ldr = ldr; g.y = y; g.ldy = ldy;
  return status(launch_act8_linear(g, (hipStream_t)stream));
}

size_t slide_act8_wgrad_workspace_bytes(int64_t rows, int64_t out, int64_t in) {
  if (rows < 1 || rows > A8_MAX_ROWS || out < 1 || out > A8_MAX_COLS || in < 1 || in > A8_MAX_COLS) return 0;
  if (((out + 127) / 128) * ((in + 127) / 128) > (1 << 22)) return 0;
  return act8_wgrad_bytes(rows, (int)out, (int)in);
}

int slide_act8_wgrad(const void* dy, int dtype, int64_t lddy, int64_t out, const slide_act8* x8, float* dW, int64_t lddw,
                     float* db, int accumulate, void* work, size_t work_bytes, void* stream) {
  if (!act8_ok(x8) || !dtype_ok(dtype) || out < 1 || !matrix_ok(dy, dtype, lddy, out) ||
      !matrix_ok(dW, DT_F32, lddw, x8->cols) || (db && !floats_ok(db)))
    return SLIDE_EINVAL;
  const size_t need = slide_act8_wgrad_workspace_bytes(x8->rows, out, x8->cols);
  if (!need || x8->ldc > (1 << 24) || x8->lds > (1 << 24)) return SLIDE_EUNSUPPORTED;   // 32-bit offsets within 64 rows
  const int rc = work_ok(work, work_bytes, need);
  if (rc) return rc;
  (void)hipGetLastError();
  A8Wgrad g{};
  g.dy = dy; g.dt = dtype; g.lddy = lddy; g.x = a8_view(*x8);
  g.M = x8->rows; g.N = (int)out; g.K = (int)x8->cols;
  g.dW = dW; g.lddw = lddw; g.db = db; g.accumulate = accumulate != 0; g.work = (float*)work;
  return status(launch_act8_wgrad(g, (hipStream_t)stream));
}

size_t slide_group_norm_workspace_bytes(const slide_group_norm* s) { return norm_ok(s) ? group_norm_bytes(*s) : 0; }

int slide_group_norm_fwd(const slide_group_norm* s, const void* x, int64_t ldx, const float* gamma, const float* beta,
                         const void* residual, int64_t ldr, void* y, int64_t ldy, const slide_act8* x8, float* mean,
                         float* rstd, void* work, size_t work_bytes, void* stream) {
  if (!norm_ok(s) || !matrix_ok(x, s->dtype, ldx, s->channels) || !matrix_ok(y, s->dtype, ldy, s->channels)) return SLIDE_EINVAL;
  if (!floats_ok(gamma) || !floats_ok(beta) || !floats_ok(mean) || !floats_ok(rstd)) return SLIDE_EINVAL;
  if (residual && !matrix_ok(residual, s->dtype, ldr, s->channels)) return SLIDE_EINVAL;
  if ((y == x && ldy != ldx) || (residual && y == residual && ldy != ldr)) return SLIDE_EINVAL;
  if (x8 && (!act8_ok(x8) || x8->rows != s->n * s->hw || x8->cols != s->channels)) return SLIDE_EINVAL;
  const int rc = work_ok(work, work_bytes, group_norm_bytes(*s));
  if (rc) return rc;
  (void)hipGetLastError();
  GroupNorm g{};
  g.s = *s; g.x = x; g.ldx = ldx; g.gamma = gamma; g.beta = beta; g.resid = residual; g.ldr = ldr; g.y = y; g.ldy = ldy;
  g.x8 = x8; g.mean = mean; g.rstd = rstd; g.work = (float*)work;
  return status(launch_group_norm_fwd(g, (hipStream_t)stream));
}

int slide_group_norm_bwd(const slide_group_norm* s, const void* dy, int64_t lddy, const void* x, int64_t ldx,
                         const slide_act8* x8, const float* gamma, const float* beta, const void* residual, int64_t ldr,
                         const float* mean, const float* rstd, void* dx, int64_t lddx, void* dresidual, int64_t lddr,
                         float* dgamma, float* dbeta, int accumulate, void* work, size_t work_bytes, void* stream) {
  if (!norm_ok(s) || !matrix_ok(dy, s->dtype, lddy, s->channels) || !matrix_ok(dx, s->dtype, lddx, s->channels)) return SLIDE_EINVAL;
  if ((x != nullptr) == (x8 != nullptr)) return SLIDE_EINVAL;
  if (x && !matrix_ok(x, s->dtype, ldx, s->channels)) return SLIDE_EINVAL;
  if (x8 && (!act8_ok(x8) || x8->rows != s->n * s->hw || x8->cols != s->channels)) return SLIDE_EINVAL;
  if (!floats_ok(gamma) || !floats_ok(beta) || !floats_ok(mean) || !floats_ok(rstd) || !floats_ok(dgamma) || !floats_ok(dbeta))
    return SLIDE_EINVAL;
  if (residual && !matrix_ok(residual, s->dtype, ldr, s->channels)) return SLIDE_EINVAL;
  if (dresidual && !matrix_ok(dresidual, s->dtype, lddr, s->channels)) return SLIDE_EINVAL;
  if (dx == x || dx == residual || dx == dresidual || (dresidual && (dresidual == x || dresidual == residual))) return SLIDE_EINVAL;
  if ((dx == dy && lddx != lddy) || (dresidual == dy && lddr != lddy)) return SLIDE_EINVAL;
  const int rc = work_ok(work, work_bytes, group_norm_bytes(*s));
  if (rc) return rc;
  (void)hipGetLastError();
  GroupNorm g{};
  g.s = *s; g.x = x; g.ldx = ldx; g.gamma = gamma; g.beta = beta; g.resid = residual; g.ldr = ldr; g.y = dx; g.ldy = lddx;
  g.x8 = x8; g.mean = const_cast<float*>(mean); g.rstd = const_cast<float*>(rstd); g.dy = dy; g.lddy = lddy;
  g.dresid = dresidual; g.lddr = lddr; g.dgamma = dgamma; g.dbeta = dbeta; g.accumulate = accumulate != 0; g.work = (float*)work;
  return status(launch_group_norm_bwd(g, (hipStream_t)stream));
}

}  // extern "C"
