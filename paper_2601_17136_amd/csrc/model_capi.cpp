// Host side of the model operators: the C ABI of layer norm, the class head
// and its losses.  Argument checks run before any HIP call; nothing throws.
#include <hip/hip_runtime.h>

#include <cmath>

#include "kkm.h"
#include "model_ops.h"

using namespace kkm;

namespace {

const char* kTypes = "F32(0), F16(1) or BF16(2)";

bool is_type(int32_t t) { return t == KKM_F32 || t == KKM_F16 || t == KKM_BF16; }

int check_norm(kkm_ctx* c, int32_t type, int64_t n, int32_t d, int32_t wtype) {
  if (!is_type(type)) return ctx_fail(c, KKM_ERR_ARG, "type=%d is not %s", type, kTypes);
  if (wtype != KKM_F32 && wtype != type)
    return ctx_fail(c, KKM_ERR_ARG, "wtype=%d must be F32(0) or the rows' type %d", wtype, type);
  if (n < 0 || n > 2147483647LL) return ctx_fail(c, KKM_ERR_ARG, "n=%lld must be in [0, 2^31-1]", (long long)n);
  if (d < 1 || d > KKM_MAX_FEATURES) return ctx_fail(c, KKM_ERR_ARG, "d=%d must be in [1, %d]", d, KKM_MAX_FEATURES);
  return KKM_OK;
}

int check_ld(kkm_ctx* c, const char* name, int64_t ld, int64_t d) {
  if (ld < d || ld > (int64_t)1 << 31)
    return ctx_fail(c, KKM_ERR_ARG, "%s=%lld must be in [%lld, 2^31]", name, (long long)ld, (long long)d);
  return KKM_OK;
}

int check_eps(kkm_ctx* c, float eps) {
  if (!(eps > 0.f && std::isfinite(eps))) return ctx_fail(c, KKM_ERR_ARG, "eps=%g must be finite and > 0", (double)eps);
  return KKM_OK;
}

int check_head(kkm_ctx* c, const kkm_head* h) {
  if (!h) return ctx_fail(c, KKM_ERR_ARG, "head is NULL");
  if (!is_type(h->type)) return ctx_fail(c, KKM_ERR_ARG, "type=%d is not %s", h->type, kTypes);
  if (h->d < 1 || h->d > KKM_MAX_FEATURES)
    return ctx_fail(c, KKM_ERR_ARG, "d=%d must be in [1, %d]", h->d, KKM_MAX_FEATURES);
  if (h->n < 0 || h->n > KKM_MAX_ROWS)
    return ctx_fail(c, KKM_ERR_ARG, "n=%lld must be in [0, %d]", (long long)h->n, KKM_MAX_ROWS);
  if (h->classes < 1 || h->classes > KKM_MAX_ROWS)
    return ctx_fail(c, KKM_ERR_ARG, "classes=%lld must be in [1, %d]", (long long)h->classes, KKM_MAX_ROWS);
  if (!std::isfinite(h->scale)) return ctx_fail(c, KKM_ERR_ARG, "scale=%g must be finite", (double)h->scale);
  if (int rc = check_ld(c, "ldh", h->ldh, h->d)) return rc;
  return check_ld(c, "ldw", h->ldw, h->d);
}

int check_teacher(kkm_ctx* c, const kkm_head* h, const kkm_teacher* t) {
  if (t->m < 1 || t->m > KKM_MAX_TOP) return ctx_fail(c, KKM_ERR_ARG, "m=%d must be in [1, %d]", t->m, KKM_MAX_TOP);
  if (h->n * t->m > 2147483647LL)
    return ctx_fail(c, KKM_ERR_ARG, "n=%lld times m=%d must be below 2^31", (long long)h->n, t->m);
  if (!std::isfinite(t->scale)) return ctx_fail(c, KKM_ERR_ARG, "teacher's scale=%g must be finite", (double)t->scale);
  return KKM_OK;
}

int missing(kkm_ctx* c, const char* name) { return ctx_fail(c, KKM_ERR_ARG, "%s is NULL", name); }

int done(kkm_ctx* c, hipError_t e, const char* what) {
  return e == hipSuccess ? KKM_OK : ctx_fail(c, KKM_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

// Both losses; ids alone stand for one pair per row.
int head_call(kkm_ctx* c, const char* what, const kkm_head* h, const int32_t* ids, const kkm_teacher* t, bool grad,
              const float* dloss, float* loss, float* lse, void* dh, int64_t lddh, void* dw, int64_t lddw) {
  if (!c) return missing(nullptr, "ctx");
  if (int rc = check_head(c, h)) return rc;
  if (t) {
    if (int rc = check_teacher(c, h, t)) return rc;
    ids = t->ids;
  }
  if (h->n > 0) {
    if (!h->h) return missing(c, "h");
    if (!h->w) return missing(c, "w");
    if (!ids) return missing(c, "ids");
    if (t && !t->logits) return missing(c, "logits");
    if (grad && !dloss) return missing(c, "dloss");
    if (!loss) return missing(c, "loss");
    if (!lse) return missing(c, "lse");
  }
  if (dh)
    if (int rc = check_ld(c, "lddh", lddh, h->d)) return rc;
  if (dw)
    if (int rc = check_ld(c, "lddw", lddw, h->d)) return rc;
  HeadArgs a{};
  a.type = h->type;
  a.n = h->n;
  a.d = h->d;
  a.classes = (int)h->classes;
  a.m = t ? t->m : 1;
  a.h = h->h;
  a.w = h->w;
  a.ldh = h->ldh;
  a.ldw = h->ldw;
  a.scale = h->scale;
  a.tscale = t ? t->scale : 1.f;
  a.offset = h->offset;
  a.ids = ids;
  a.tlogits = t ? t->logits : nullptr;
  a.dloss = dloss;
  a.loss = loss;
  a.lse = lse;
  a.dh = dh;
  a.dw = dw;
  a.lddh = lddh;
  a.lddw = lddw;
  grad = grad && (dh || dw);
  void* ws = nullptr;
  if (const size_t bytes = head_scratch(a, grad))
    if (int rc = ctx_workspace(c, bytes, &ws)) return rc;
  return done(c, launch_head(a, grad, ws, ctx_stream(c)), what);
}

}  // namespace

extern "C" {

int kkm_check_norm_args(int32_t type, int64_t n, int32_t d, int64_t ldx, int32_t wtype, float eps) {
  if (int rc = check_norm(nullptr, type, n, d, wtype)) return rc;
  if (int rc = check_ld(nullptr, "ldx", ldx, d)) return rc;
  return check_eps(nullptr, eps);
}

int kkm_check_head_args(const kkm_head* head, const kkm_teacher* teacher) {
  if (int rc = check_head(nullptr, head)) return rc;
  return teacher ? check_teacher(nullptr, head, teacher) : KKM_OK;
}

int kkm_get_stream(kkm_ctx* c, void** out) {
  if (!c) return missing(nullptr, "ctx");
  if (!out) return missing(c, "out");
  *out = ctx_stream(c);
  return KKM_OK;
}

int kkm_layer_norm(kkm_ctx* c, int32_t type, int64_t n, int32_t d, const void* x, int64_t ldx, int32_t wtype,
                   const void* weight, const void* bias, float eps, void* y, int64_t ldy, float* mean, float* rstd) {
  if (!c) return missing(nullptr, "ctx");
  if (int rc = check_norm(c, type, n, d, wtype)) return rc;
  if (int rc = check_ld(c, "ldx", ldx, d)) return rc;
  if (int rc = check_ld(c, "ldy", ldy, d)) return rc;
  if (int rc = check_eps(c, eps)) return rc;
  if (n > 0 && !x) return missing(c, "x");
  if (n > 0 && !y) return missing(c, "y");
  NormArgs a{};
  a.type = type;
  a.wtype = wtype;
  a.n = n;
  a.d = d;
  a.x = x;
  a.ldx = ldx;
  a.w = weight;
  a.b = bias;
  a.eps = eps;
  a.y = y;
  a.ldy = ldy;
  a.mean = mean;
  a.rstd = rstd;
  return done(c, launch_layer_norm(a, ctx_stream(c)), "layer norm");
}

int kkm_layer_norm_grad(kkm_ctx* c, int32_t type, int64_t n, int32_t d, const void* x, int64_t ldx, int32_t wtype,
                        const void* weight, const float* mean, const float* rstd, const void* dy, int64_t lddy,
                        void* dx, int64_t lddx, void* dweight, void* dbias) {
  if (!c) return missing(nullptr, "ctx");
  if (int rc = check_norm(c, type, n, d, wtype)) return rc;
  if (int rc = check_ld(c, "ldx", ldx, d)) return rc;
  if (int rc = check_ld(c, "lddy", lddy, d)) return rc;
  if (dx)
    if (int rc = check_ld(c, "lddx", lddx, d)) return rc;
  if (n > 0) {
    if (!x) return missing(c, "x");
    if (!dy) return missing(c, "dy");
    if (!mean) return missing(c, "mean");
    if (!rstd) return missing(c, "rstd");
  }
  if (!dx && !dweight && !dbias) return KKM_OK;
  NormArgs a{};
  a.type = type;
  a.wtype = wtype;
  a.n = n;
  a.d = d;
  a.x = x;
  a.ldx = ldx;
  a.w = weight;
  a.mean = const_cast<float*>(mean);
  a.rstd = const_cast<float*>(rstd);
  a.dy = dy;
  a.lddy = lddy;
  a.dx = dx;
  a.lddx = lddx;
  a.dw = dweight;
  a.db = dbias;
  void* lines = nullptr;
  if ((dweight || dbias) && n > 0)
    if (int rc = ctx_workspace(c, norm_scratch(n, d), &lines)) return rc;
  return done(c, launch_layer_norm_grad(a, (float*)lines, ctx_stream(c)), "layer norm's gradient");
}

int kkm_head_loss(kkm_ctx* c, const kkm_head* head, const int32_t* ids, float* loss, float* lse) {
  return head_call(c, "head loss", head, ids, nullptr, false, nullptr, loss, lse, nullptr, 0, nullptr, 0);
}

int kkm_head_grad(kkm_ctx* c, const kkm_head* head, const int32_t* ids, const float* dloss, float* loss, float* lse,
                  void* dh, int64_t lddh, void* dw, int64_t lddw) {
  return head_call(c, "head gradient", head, ids, nullptr, true, dloss, loss, lse, dh, lddh, dw, lddw);
}

int kkm_distill_loss(kkm_ctx* c, const kkm_head* head, const kkm_teacher* teacher, float* loss, float* lse) {
  if (c && !teacher) return missing(c, "teacher");
  return head_call(c, "distillation loss", head, nullptr, teacher, false, nullptr, loss, lse, nullptr, 0, nullptr, 0);
}

int kkm_distill_grad(kkm_ctx* c, const kkm_head* head, const kkm_teacher* teacher, const float* dloss, float* loss,
                     float* lse, void* dh, int64_t lddh, void* dw, int64_t lddw) {
  if (c && !teacher) return missing(c, "teacher");
  return head_call(c, "distillation gradient", head, nullptr, teacher, true, dloss, loss, lse, dh, lddh, dw, lddw);
}

}  // extern "C"
