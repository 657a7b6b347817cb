// Host side of the model operators: the C ABI of layer norm, the class head and
// its losses, adapted projections, orthogonalised updates and answers from logits.
// Argument checks run before any HIP call; nothing throws.
#include <hip/hip_runtime.h>

#include <cmath>
#include <initializer_list>

#include "kkm.h"
#include "model_ops.h"

using namespace kkm;

namespace {

const char* kTypes = "F32(0), F16(1) or BF16(2)";

bool is_type(int32_t t) { return t == KKM_F32 || t == KKM_F16 || t == KKM_BF16; }

int missing(kkm_ctx* c, const char* name) { return ctx_fail(c, KKM_ERR_ARG, "%s is NULL", name); }

int done(kkm_ctx* c, hipError_t e, const char* what) {
  return e == hipSuccess ? KKM_OK : ctx_fail(c, KKM_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

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

int check_adapted(kkm_ctx* c, const kkm_adapted* a) {
  if (!a) return missing(c, "adapted");
  if (!is_type(a->type)) return ctx_fail(c, KKM_ERR_ARG, "type=%d is not %s", a->type, kTypes);
  if (a->d < 1 || a->d > KKM_MAX_FEATURES)
    return ctx_fail(c, KKM_ERR_ARG, "d=%d must be in [1, %d]", a->d, KKM_MAX_FEATURES);
  if (a->n < 0 || a->n > KKM_MAX_ROWS)
    return ctx_fail(c, KKM_ERR_ARG, "n=%lld must be in [0, %d]", (long long)a->n, KKM_MAX_ROWS);
  if (a->m < 1 || a->m > KKM_MAX_FEATURES)
    return ctx_fail(c, KKM_ERR_ARG, "m=%lld must be in [1, %d]", (long long)a->m, KKM_MAX_FEATURES);
  if (a->adapters < 1 || a->adapters > KKM_MAX_ADAPTERS)
    return ctx_fail(c, KKM_ERR_ARG, "adapters=%d must be in [1, %d]", a->adapters, KKM_MAX_ADAPTERS);
  if (a->rank < 1 || a->rank > KKM_MAX_RANK)
    return ctx_fail(c, KKM_ERR_ARG, "rank=%d must be in [1, %d]", a->rank, KKM_MAX_RANK);
  if (int rc = check_ld(c, "ldx", a->ldx, a->d)) return rc;
  return check_ld(c, "ldw", a->ldw, a->d);
}

int adapted_call(kkm_ctx* c, const char* what, const kkm_adapted* q, bool grad, AdaptArgs& a) {
  a.type = q->type;
  a.n = q->n;
  a.d = q->d;
  a.m = (int)q->m;
  a.x = q->x;
  a.ldx = q->ldx;
  a.w = q->w;
  a.ldw = q->ldw;
  a.adapters = q->adapters;
  a.rank = q->rank;
  a.down = q->down;
  a.up = q->up;
  a.ids = q->ids;
  a.factor = q->factor;
  if (a.n > 0) {
    if (!a.x) return missing(c, "x");
    if (!a.w) return missing(c, "w");
    if (!a.down) return missing(c, "down");
    if (!a.up) return missing(c, "up");
    if (!a.ids) return missing(c, "ids");
  }
  void* ws = nullptr;
  if (const size_t bytes = adapt_scratch(a, grad))
    if (int rc = ctx_workspace(c, bytes, &ws)) return rc;
  return done(c, launch_adapt(a, grad, ws, ctx_stream(c)), what);
}

int check_newton(kkm_ctx* c, const kkm_newton* w, int32_t type, int64_t batch, int64_t m, int64_t n, NewtonSteps* out) {
  if (!w) return missing(c, "newton");
  if (!is_type(type)) return ctx_fail(c, KKM_ERR_ARG, "type=%d is not %s", type, kTypes);
  if (batch < 0 || batch > KKM_MAX_ROWS)
    return ctx_fail(c, KKM_ERR_ARG, "batch=%lld must be in [0, %d]", (long long)batch, KKM_MAX_ROWS);
  if (m < 1 || m > KKM_MAX_FEATURES)
    return ctx_fail(c, KKM_ERR_ARG, "m=%lld must be in [1, %d]", (long long)m, KKM_MAX_FEATURES);
  if (n < 1 || n > KKM_MAX_FEATURES)
    return ctx_fail(c, KKM_ERR_ARG, "n=%lld must be in [1, %d]", (long long)n, KKM_MAX_FEATURES);
  if (w->steps < 1 || w->steps > KKM_MAX_STEPS)
    return ctx_fail(c, KKM_ERR_ARG, "steps=%d must be in [1, %d]", w->steps, KKM_MAX_STEPS);
  if (!w->coef) return missing(c, "coef");
  if (!(w->eps > 0 && std::isfinite(w->eps)))
    return ctx_fail(c, KKM_ERR_ARG, "eps=%g must be finite and > 0", w->eps);
  out->steps = w->steps;
  for (int i = 0; i < 3 * w->steps; ++i) {
    if (!std::isfinite(w->coef[i])) return ctx_fail(c, KKM_ERR_ARG, "coef[%d]=%g must be finite", i, w->coef[i]);
    out->coef[i] = w->coef[i];
  }
  if (!newton_in_range(*out))
    return ctx_fail(c, KKM_ERR_ARG, "these %d steps let singular values grow past 2^12", w->steps);
  return KKM_OK;
}

int check_apart(kkm_ctx* c, const char* name, int64_t batch, int64_t m, int64_t n, int64_t ld, int64_t stride) {
  const int64_t least = (m - 1) * ld + n;
  if (batch > 1 && (stride < least || stride > (int64_t)1 << 41))
    return ctx_fail(c, KKM_ERR_ARG, "%s=%lld must be in [%lld, 2^41]", name, (long long)stride, (long long)least);
  return KKM_OK;
}

// A result in its input's place lies as it does.
int check_in_place(kkm_ctx* c, const char* what, bool same) {
  return same ? KKM_OK : ctx_fail(c, KKM_ERR_ARG, "%s of another stride", what);
}

// A result lies apart from what is still read when it is written, and from other results.
struct Named {
  const char* name;
  const void* p;
};
int check_own(kkm_ctx* c, const Named& out, std::initializer_list<Named> others) {
  for (const Named& o : others)
    if (out.p && out.p == o.p) return ctx_fail(c, KKM_ERR_ARG, "%s is %s", out.name, o.name);
  return KKM_OK;
}

int ortho_call(kkm_ctx* c, const char* what, OrthoArgs& a) {
  void* ws = nullptr;
  if (const size_t bytes = ortho_scratch(a))
    if (int rc = ctx_workspace(c, bytes, &ws)) return rc;
  return done(c, launch_ortho(a, ws, ctx_stream(c)), what);
}

int check_choice(kkm_ctx* c, const kkm_choice* q) {
  if (!q) return missing(c, "choice");
  if (!is_type(q->type)) return ctx_fail(c, KKM_ERR_ARG, "type=%d is not %s", q->type, kTypes);
  if (q->n < 0 || q->n > KKM_MAX_ROWS)
    return ctx_fail(c, KKM_ERR_ARG, "n=%lld must be in [0, %d]", (long long)q->n, KKM_MAX_ROWS);
  if (q->classes < 1 || q->classes > KKM_MAX_ROWS)
    return ctx_fail(c, KKM_ERR_ARG, "classes=%d must be in [1, %d]", q->classes, KKM_MAX_ROWS);
  if (int rc = check_ld(c, "ldz", q->ldz, q->classes)) return rc;
  if (!(q->scale > 0.f && std::isfinite(q->scale)))
    return ctx_fail(c, KKM_ERR_ARG, "scale=%g must be finite and > 0", (double)q->scale);
  if (q->ngiven < 0 || q->ngiven > KKM_MAX_GIVEN)
    return ctx_fail(c, KKM_ERR_ARG, "ngiven=%d must be in [0, %d]", q->ngiven, KKM_MAX_GIVEN);
  if (!(q->repeat > 0.f && std::isfinite(q->repeat)))
    return ctx_fail(c, KKM_ERR_ARG, "repeat=%g must be finite and > 0", (double)q->repeat);
  if (!std::isfinite(q->presence) || !std::isfinite(q->frequency))
    return ctx_fail(c, KKM_ERR_ARG, "presence=%g and frequency=%g must be finite", (double)q->presence,
                    (double)q->frequency);
  if (q->nbias < 0 || q->nbias > KKM_MAX_BIASES)
    return ctx_fail(c, KKM_ERR_ARG, "nbias=%d must be in [0, %d]", q->nbias, KKM_MAX_BIASES);
  if (q->nmasks < 0) return ctx_fail(c, KKM_ERR_ARG, "nmasks=%d must not be negative", q->nmasks);
  if (q->masks) {
    if (q->words < (q->classes + 31) / 32)
      return ctx_fail(c, KKM_ERR_ARG, "words=%lld must be at least %d", (long long)q->words, (q->classes + 31) / 32);
    if (!q->mask_ids && q->nmasks < q->n)
      return ctx_fail(c, KKM_ERR_ARG, "nmasks=%d must be at least n=%lld without mask_ids", q->nmasks, (long long)q->n);
  } else if (q->mask_ids) {
    return missing(c, "masks");
  }
  return KKM_OK;
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

int kkm_check_adapted_args(const kkm_adapted* a) { return check_adapted(nullptr, a); }

int kkm_check_newton_args(const kkm_newton* newton, int32_t type, int64_t batch, int64_t m, int64_t n) {
  NewtonSteps steps;
  return check_newton(nullptr, newton, type, batch, m, n, &steps);
}

int kkm_check_choice_args(const kkm_choice* choice) { return check_choice(nullptr, choice); }

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

int kkm_adapted_linear(kkm_ctx* c, const kkm_adapted* q, void* y, int64_t ldy) {
  if (!c) return missing(nullptr, "ctx");
  if (int rc = check_adapted(c, q)) return rc;
  if (int rc = check_ld(c, "ldy", ldy, q->m)) return rc;
  if (q->n == 0) return KKM_OK;
  if (!y) return missing(c, "y");
  if (int rc = check_own(c, {"y", y}, {{"x", q->x}, {"w", q->w}, {"down", q->down}, {"up", q->up}})) return rc;
  AdaptArgs a{};
  a.y = y;
  a.ldy = ldy;
  return adapted_call(c, "adapted projection", q, false, a);
}

int kkm_adapted_linear_grad(kkm_ctx* c, const kkm_adapted* q, const void* dy, int64_t lddy, void* dx, int64_t lddx,
                            void* ddown, void* dup) {
  if (!c) return missing(nullptr, "ctx");
  if (int rc = check_adapted(c, q)) return rc;
  if (int rc = check_ld(c, "lddy", lddy, q->m)) return rc;
  if (dx)
    if (int rc = check_ld(c, "lddx", lddx, q->d)) return rc;
  if (q->n > 0 && !dy) return missing(c, "dy");
  if (!dx && !ddown && !dup) return KKM_OK;
  for (const Named& out : {Named{"dx", dx}, Named{"ddown", ddown}, Named{"dup", dup}})
    if (int rc = check_own(c, out, {{"x", q->x}, {"dy", dy}, {"w", q->w}, {"down", q->down}, {"up", q->up}})) return rc;
  if (int rc = check_own(c, {"dx", dx}, {{"ddown", ddown}, {"dup", dup}})) return rc;
  if (int rc = check_own(c, {"ddown", ddown}, {{"dup", dup}})) return rc;
  AdaptArgs a{};
  a.dy = dy;
  a.lddy = lddy;
  a.dx = dx;
  a.lddx = lddx;
  a.ddown = ddown;
  a.dup = dup;
  return adapted_call(c, "adapted projection's gradient", q, true, a);
}

int kkm_orthogonalize(kkm_ctx* c, const kkm_newton* newton, int32_t type, int64_t batch, int64_t m, int64_t n,
                      const void* x, int64_t ldx, int64_t stride_x, void* y, int64_t ldy, int64_t stride_y) {
  if (!c) return missing(nullptr, "ctx");
  OrthoArgs a{};
  if (int rc = check_newton(c, newton, type, batch, m, n, &a.newton)) return rc;
  if (int rc = check_ld(c, "ldx", ldx, n)) return rc;
  if (int rc = check_ld(c, "ldy", ldy, n)) return rc;
  if (int rc = check_apart(c, "stride_x", batch, m, n, ldx, stride_x)) return rc;
  if (int rc = check_apart(c, "stride_y", batch, m, n, ldy, stride_y)) return rc;
  if (batch > 0 && !x) return missing(c, "x");
  if (batch > 0 && !y) return missing(c, "y");
  if (batch > 0 && x == y)
    if (int rc = check_in_place(c, "y is x", (m == 1 || ldx == ldy) && (batch <= 1 || stride_x == stride_y))) return rc;
  a.type = type;
  a.batch = batch;
  a.m = m;
  a.n = n;
  a.x = x;
  a.ldx = ldx;
  a.stride_x = stride_x;
  a.y = y;
  a.ldy = ldy;
  a.stride_y = stride_y;
  a.eps = newton->eps;
  return ortho_call(c, "orthogonalising", a);
}

int kkm_orthogonal_step(kkm_ctx* c, const kkm_newton* newton, int32_t type, int64_t batch, int64_t m, int64_t n,
                        void* w, int64_t ldw, int64_t stride_w, const void* g, int64_t ldg, int64_t stride_g, float* v,
                        float momentum, int32_t nesterov, float rate, float keep) {
  if (!c) return missing(nullptr, "ctx");
  OrthoArgs a{};
  if (int rc = check_newton(c, newton, type, batch, m, n, &a.newton)) return rc;
  if (int rc = check_ld(c, "ldw", ldw, n)) return rc;
  if (int rc = check_ld(c, "ldg", ldg, n)) return rc;
  if (int rc = check_apart(c, "stride_w", batch, m, n, ldw, stride_w)) return rc;
  if (int rc = check_apart(c, "stride_g", batch, m, n, ldg, stride_g)) return rc;
  if (!std::isfinite(momentum) || !std::isfinite(rate) || !std::isfinite(keep))
    return ctx_fail(c, KKM_ERR_ARG, "momentum=%g, rate=%g and keep=%g must be finite", (double)momentum, (double)rate,
                    (double)keep);
  if (batch > 0 && !w) return missing(c, "w");
  if (batch > 0 && !g) return missing(c, "g");
  if (batch > 0 && !v) return missing(c, "v");
  if (int rc = check_own(c, {"v", v}, {{"w", w}, {"g", g}})) return rc;
  a.type = type;
  a.batch = batch;
  a.m = m;
  a.n = n;
  a.x = g;
  a.ldx = ldg;
  a.stride_x = stride_g;
  a.y = w;
  a.ldy = ldw;
  a.stride_y = stride_w;
  a.v = v;
  a.momentum = momentum;
  a.nesterov = nesterov != 0;
  a.rate = rate;
  a.keep = keep;
  a.eps = newton->eps;
  return ortho_call(c, "orthogonal step", a);
}

int kkm_choose(kkm_ctx* c, const kkm_choice* q, void* out, int64_t ldo, int32_t* ids, float* logp, float* lse) {
  if (!c) return missing(nullptr, "ctx");
  if (int rc = check_choice(c, q)) return rc;
  if (out)
    if (int rc = check_ld(c, "ldo", ldo, q->classes)) return rc;
  if (q->n > 0) {
    if (!q->z) return missing(c, "z");
    if (q->ngiven && !q->given) return missing(c, "given");
    if (q->nbias && !q->bias_ids) return missing(c, "bias_ids");
    if (q->nbias && !q->bias) return missing(c, "bias");
    if (out == q->z)
      if (int rc = check_in_place(c, "out is z", q->n == 1 || ldo == q->ldz)) return rc;
  }
  ChooseArgs a{};
  a.type = q->type;
  a.n = q->n;
  a.classes = q->classes;
  a.z = q->z;
  a.ldz = q->ldz;
  a.scale = q->scale;
  a.offset = q->offset;
  a.given = q->given;
  a.ngiven = q->ngiven;
  a.repeat = q->repeat;
  a.presence = q->presence;
  a.frequency = q->frequency;
  a.bias_ids = q->bias_ids;
  a.bias = q->bias;
  a.nbias = q->nbias;
  a.masks = q->masks;
  a.words = q->words;
  a.nmasks = q->nmasks;
  a.mask_ids = q->mask_ids;
  a.out = out;
  a.ldo = ldo;
  a.ids = ids;
  a.logp = logp;
  a.lse = lse;
  if (const size_t bytes = choose_scratch(a))
    if (int rc = ctx_workspace(c, bytes, &a.parts)) return rc;
  return done(c, launch_choose(a, ctx_stream(c)), "choice");
}

}  // extern "C"
