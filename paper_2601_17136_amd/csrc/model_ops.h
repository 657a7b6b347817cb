// The operators of a model that learns from a clustering: layer norm, and a
// class head with its losses (cross entropy with ids, distillation from a
// teacher's top logits).  Declarations shared by their kernels and their C ABI.
#pragma once
#include "kkm_internal.h"

struct kkm_ctx;

namespace kkm {

enum ElemType { TYPE_F32 = 0, TYPE_F16 = 1, TYPE_BF16 = 2 };
inline size_t elem_bytes(int type) { return type == TYPE_F32 ? 4 : 2; }

// What the C ABI of these operators needs of a context (kkm_capi.cpp).
hipStream_t ctx_stream(const kkm_ctx* c);
int ctx_fail(kkm_ctx* c, int code, const char* fmt, ...);
// At least this many bytes of the context's operator workspace; it grows, and
// goes with the next build or the context.
int ctx_workspace(kkm_ctx* c, size_t bytes, void** out);

struct NormArgs {
  int type, wtype;  // ElemType of x, y, dy, dx and of w, b, dw, db
  int64_t n;
  int d;
  const void *x, *w, *b, *dy;  // w, b may be null (1 and 0)
  int64_t ldx, ldy, lddy, lddx;
  float eps;
  void* y;
  float *mean, *rstd;  // written by the forward pass (may be null), read by the gradient
  void *dx, *dw, *db;  // each may be null
};
size_t norm_scratch(int64_t n, int d);
int norm_lines(int64_t n, int d);
hipError_t launch_layer_norm(const NormArgs& a, hipStream_t s);
hipError_t launch_layer_norm_grad(const NormArgs& a, float* lines, hipStream_t s);

// The head: logits z(i, v) = scale h_i . w_v + offset_v.  A row's target is a
// distribution q over m pairs (class, logit); ids alone are m = 1, q = 1.
struct HeadArgs {
  int type;  // ElemType of h, w, dh, dw
  int64_t n;
  int d, classes, m;
  const void *h, *w;
  int64_t ldh, ldw;
  float scale, tscale;
  const float* offset;   // per class, -inf leaves it out; may be null
  const int32_t* ids;    // n x m; negative: no target
  const float* tlogits;  // n x m teacher logits, or null (m = 1)
  const float* dloss;    // gradient only
  float *loss, *lse;
  void *dh, *dw;  // gradient only; each may be null
  int64_t lddh, lddw;
};
constexpr int kMaxTop = 256;

// How a head runs: FEW, at most kFew classes or rows, and DIRECT, little work on
// more of both, straight from the rows (head_few.hip); TILED, matrix products of
// copies in tiles, at most 256 MB of the logits stored (head.hip).
enum HeadForm { HEAD_FEW, HEAD_DIRECT, HEAD_TILED };
constexpr int kFew = 64;
// n times classes: 64 MB of scores (128 MB with their rows padded to 64, of 65 classes)
constexpr int64_t kDirectScores = (int64_t)16 << 20;
HeadForm head_form(const HeadArgs& a);
size_t head_short_scratch(const HeadArgs& a, bool grad);
hipError_t launch_head_short(const HeadArgs& a, bool grad, void* scratch, hipStream_t s);

size_t head_scratch(const HeadArgs& a, bool grad);
hipError_t launch_head(const HeadArgs& a, bool grad, void* scratch, hipStream_t s);

}  // namespace kkm
