// lm_api.hip -- the C entry points of the language-model operators: checks of
// the arguments on the host, then the launchers of lm.hpp.  A refused call has
// touched nothing.
#include "crossbow_sma.h"
#include "lm.hpp"

#include <algorithm>
#include <cmath>
#include <exception>

using namespace cbk;

namespace {

constexpr int64_t MOST = int64_t(1) << 30;  // rows and words
constexpr int MAX_D = 1 << 20, MAX_K = 65535;

int refuse(const char* who, const char* why, int code = CB_EINVAL) {
  note_error(std::string(who) + ": " + why);
  return code;
}
// A workspace of `given` bytes where `need` are needed (0: more than a launch holds).
int short_of(const char* who, size_t need, size_t given) {
  if (need == 0) return refuse(who, "more workgroups than a launch holds");
  return given < need ? refuse(who, "workspace too small", CB_ENOMEM) : CB_OK;
}
int done(const char* who, hipError_t e) {
  if (e == hipSuccess) return CB_OK;
  note_error(std::string(who) + ": " + hipGetErrorString(e));
  return CB_EDEVICE;
}

// Runs f, and lets no exception (a failed allocation of a message) out.
template <class R, class F>
R shielded(R failed, F f) noexcept {
  try {
    return f();
  } catch (...) {
    return failed;
  }
}

bool type_ok(int type) { return type == LM_F32 || type == LM_F16 || type == LM_BF16; }
bool at(const void* p, int bytes) { return p && (uintptr_t)p % bytes == 0; }
bool at_or_null(const void* p, int bytes) { return (uintptr_t)p % bytes == 0; }

bool rows_ok(int k, int64_t n) {
  return k >= 1 && k <= MAX_K && n >= 1 && (int64_t)k * n <= MOST;
}

// nullptr, or what is wrong.
const char* wrong(const cb_vocab_xent* x) {
  if (!x) return "no description";
  if (!type_ok(x->type)) return "type is none of CB_TYPE_*";
  if (!rows_ok(x->k, x->n)) return "k or n out of range";
  if (x->d < 1 || x->d > MAX_D) return "d out of range";
  if (x->v < 1 || x->v > MOST) return "v out of range";
  // tiles of 32 rows by 256 words, or 128 by 128, are numbered in 31 bits
  if (((int64_t)x->n / 32 + 1) * ((int64_t)x->v / 128 + 1) >= MOST)
    return "n * v out of range";
  const int sz = lm_size(x->type);
  if (!at(x->h, sz) || !at(x->w, sz) || !at(x->labels, 4)) return "h, w or labels NULL or misaligned";
  if (x->ldh < x->d) return "ldh is less than d";
  if (x->k > 1 && x->pstride < (int64_t)x->v * x->d) return "pstride is less than v * d";
  return nullptr;
}

XentArgs xent_args(const cb_vocab_xent* x) {
  XentArgs a{};
  a.type = x->type;
  a.k = x->k;
  a.n = x->n;
  a.d = x->d;
  a.v = x->v;
  a.h = x->h;
  a.ldh = x->ldh;
  a.w = x->w;
  a.pstride = x->pstride;
  a.labels = x->labels;
  a.ignore = x->ignore;
  return a;
}

const char* wrong(const cb_gated_norm* g) {
  if (!g) return "no description";
  if (!type_ok(g->type)) return "type is none of CB_TYPE_*";
  if (!rows_ok(g->k, g->n)) return "k or n out of range";
  if (g->d < 1 || g->d > NORM_MAX_D) return "d out of range";
  if (!std::isfinite(g->res_scale)) return "res_scale is not finite";
  if (!(g->eps > 0.f) || !std::isfinite(g->eps)) return "eps is not positive and finite";
  if (!g->block && (g->gate || g->post)) return "a gate or post without a block";
  if (!g->block && !g->pre) return "neither block nor pre";
  if (g->gate && g->gate_rows < 1) return "gate_rows is less than 1";
  const int sz = lm_size(g->type);
  if (!at_or_null(g->block, sz) || !at_or_null(g->gate, sz) || !at_or_null(g->post, 4) ||
      !at_or_null(g->pre, 4))
    return "a misaligned pointer";
  if (g->k > 1 && ((g->post && g->post_stride < g->d) || (g->pre && g->pre_stride < g->d)))
    return "post_stride or pre_stride is less than d";
  return nullptr;
}

NormArgs norm_args(const cb_gated_norm* g) {
  NormArgs a{};
  a.type = g->type;
  a.k = g->k;
  a.n = g->n;
  a.d = g->d;
  a.block = g->block;
  a.gate = g->gate;
  a.gate_rows = g->gate ? std::min(g->gate_rows, g->n) : g->n;  // more than all is all
  a.res_scale = g->res_scale;
  a.eps = g->eps;
  a.post = g->post;
  a.pre = g->pre;
  a.post_stride = g->post_stride;
  a.pre_stride = g->pre_stride;
  return a;
}

const char* wrong_ckpt(int type, int64_t rows, int d) {
  if (!type_ok(type)) return "type is none of CB_TYPE_*";
  if (rows < 1 || rows > MOST) return "rows out of range";
  if (d < 1 || d > MAX_D) return "d out of range";
  return nullptr;
}
const char* wrong_wgrad(int type, int k, int n, int d, int out) {
  if (!type_ok(type)) return "type is none of CB_TYPE_*";
  if (!rows_ok(k, n)) return "k or n out of range";
  if (d < 1 || d > MAX_D || out < 1 || out > MAX_D) return "d or out out of range";
  return nullptr;
}

KeptGradArgs wgrad_args(int type, int k, int n, int d, int out, const void* dy) {
  KeptGradArgs a{};
  a.type = type;
  a.k = k;
  a.n = n;
  a.d = d;
  a.out = out;
  a.dy = dy;
  return a;
}

}  // namespace

extern "C" {

size_t cb_vocab_xent_workspace_bytes(const cb_vocab_xent* x, int backward) {
  if (wrong(x)) return 0;
  return xent_ws_bytes(xent_args(x), backward != 0);
}

int cb_vocab_xent_fwd(const cb_vocab_xent* x, float* loss, float* lse, void* workspace_dev,
                      size_t ws_bytes, void* stream) {
  return shielded((int)CB_EINVAL, [&]() -> int {
    const char* me = "cb_vocab_xent_fwd";
    if (const char* why = wrong(x)) return refuse(me, why);
    if (!at(loss, 4) || !at(lse, 4)) return refuse(me, "loss or lse NULL or misaligned");
    if (!at(workspace_dev, 256)) return refuse(me, "workspace NULL or not on 256 bytes");
    XentArgs a = xent_args(x);
    if (int rc = short_of(me, xent_ws_bytes(a, false), ws_bytes)) return rc;
    a.loss = loss;
    a.lse = lse;
    a.ws = workspace_dev;
    return done(me, xent_fwd(a, static_cast<hipStream_t>(stream)));
  });
}

int cb_vocab_xent_bwd(const cb_vocab_xent* x, const float* lse, float grad_scale, void* dh,
                      void* dw, int64_t dstride, void* workspace_dev, size_t ws_bytes,
                      void* stream) {
  return shielded((int)CB_EINVAL, [&]() -> int {
    const char* me = "cb_vocab_xent_bwd";
    if (const char* why = wrong(x)) return refuse(me, why);
    const int sz = lm_size(x->type);
    if (!at(lse, 4) || !at(dh, sz) || !at(dw, sz))
      return refuse(me, "lse, dh or dw NULL or misaligned");
    if (!std::isfinite(grad_scale)) return refuse(me, "grad_scale is not finite");
    if (x->k > 1 && dstride < (int64_t)x->v * x->d)
      return refuse(me, "dstride is less than v * d");
    if (!at(workspace_dev, 256)) return refuse(me, "workspace NULL or not on 256 bytes");
    XentArgs a = xent_args(x);
    if (int rc = short_of(me, xent_ws_bytes(a, true), ws_bytes)) return rc;
    a.lse = const_cast<float*>(lse);
    a.grad_scale = grad_scale;
    a.dh = dh;
    a.dw = dw;
    a.dstride = dstride;
    a.ws = workspace_dev;
    return done(me, xent_bwd(a, static_cast<hipStream_t>(stream)));
  });
}

int cb_gated_norm_fwd(const cb_gated_norm* g, const void* x, void* x_out, void* y, void* y_kept,
                      void* stream) {
  return shielded((int)CB_EINVAL, [&]() -> int {
    const char* me = "cb_gated_norm_fwd";
    if (const char* why = wrong(g)) return refuse(me, why);
    const int sz = lm_size(g->type);
    if (!at(x, sz)) return refuse(me, "x NULL or misaligned");
    if (g->block && !at(x_out, sz)) return refuse(me, "x_out NULL or misaligned");
    if (g->pre && !at(y, sz)) return refuse(me, "y NULL or misaligned");
    if (y_kept && (!g->pre || !at(y_kept, 16)))
      return refuse(me, "y_kept without pre, or not on 16 bytes");
    NormArgs a = norm_args(g);
    a.x = x;
    a.x_out = g->block ? x_out : nullptr;
    a.y = g->pre ? y : nullptr;
    a.y_kept = y_kept;
    return done(me, norm_fwd(a, static_cast<hipStream_t>(stream)));
  });
}

size_t cb_gated_norm_workspace_bytes(const cb_gated_norm* g) {
  if (wrong(g)) return 0;
  const NormArgs a = norm_args(g);
  return norm_ws_bytes(a.type, a.k, a.n, a.d, a.gate_rows);
}

int cb_gated_norm_bwd(const cb_gated_norm* g, const void* x_out, const void* dy, const void* dres,
                      void* dx, void* dblock, void* dgate, float* dpost, int64_t dpost_stride,
                      float* dpre, int64_t dpre_stride, void* workspace_dev, size_t ws_bytes,
                      void* stream) {
  return shielded((int)CB_EINVAL, [&]() -> int {
    const char* me = "cb_gated_norm_bwd";
    if (const char* why = wrong(g)) return refuse(me, why);
    const int sz = lm_size(g->type);
    if (g->pre && (!at(x_out, sz) || !at(dy, sz) || !at(dpre, 4)))
      return refuse(me, "x_out, dy or dpre NULL or misaligned");
    if (!g->pre && dy) return refuse(me, "dy without pre");
    if (!g->pre && !dres) return refuse(me, "neither dy nor dres");
    if (!at_or_null(dres, sz) || !at(dx, sz)) return refuse(me, "dres or dx misaligned, or dx NULL");
    if (g->block && !at(dblock, sz)) return refuse(me, "dblock NULL or misaligned");
    if (g->gate && !at(dgate, sz)) return refuse(me, "dgate NULL or misaligned");
    if (g->post && !at(dpost, 4)) return refuse(me, "dpost NULL or misaligned");
    if (g->k > 1 && ((g->post && dpost_stride < g->d) || (g->pre && dpre_stride < g->d)))
      return refuse(me, "dpost_stride or dpre_stride is less than d");
    if (!at(workspace_dev, 256)) return refuse(me, "workspace NULL or not on 256 bytes");
    NormArgs a = norm_args(g);
    const size_t need = norm_ws_bytes(a.type, a.k, a.n, a.d, a.gate_rows);
    if (int rc = short_of(me, need, ws_bytes)) return rc;
    a.x = g->pre ? x_out : nullptr;
    a.dy = dy;
    a.dres = dres;
    a.dx = dx;
    a.dblock = g->block ? dblock : nullptr;
    a.dgate = g->gate ? dgate : nullptr;
    a.dpost = dpost;
    a.dpre = dpre;
    a.dpost_stride = dpost_stride;
    a.dpre_stride = dpre_stride;
    a.ws = workspace_dev;
    return done(me, norm_bwd(a, static_cast<hipStream_t>(stream)));
  });
}

size_t cb_ckpt_bytes(int64_t rows, int d) {
  return wrong_ckpt(LM_F32, rows, d) ? 0 : kept_bytes(rows, d);
}

int cb_ckpt_pack(int type, int64_t rows, int d, const void* x, void* kept, void* stream) {
  return shielded((int)CB_EINVAL, [&]() -> int {
    const char* me = "cb_ckpt_pack";
    if (const char* why = wrong_ckpt(type, rows, d)) return refuse(me, why);
    if (!at(x, lm_size(type)) || !at(kept, 16)) return refuse(me, "x or kept NULL or misaligned");
    return done(me, kept_pack(type, rows, d, x, kept, static_cast<hipStream_t>(stream)));
  });
}

int cb_ckpt_unpack(int type, int64_t rows, int d, const void* kept, void* x, void* stream) {
  return shielded((int)CB_EINVAL, [&]() -> int {
    const char* me = "cb_ckpt_unpack";
    if (const char* why = wrong_ckpt(type, rows, d)) return refuse(me, why);
    if (!at(x, lm_size(type)) || !at(kept, 16)) return refuse(me, "x or kept NULL or misaligned");
    return done(me, kept_unpack(type, rows, d, kept, x, static_cast<hipStream_t>(stream)));
  });
}

size_t cb_ckpt_wgrad_workspace_bytes(int type, int k, int n, int d, int out, const void* dy) {
  return wrong_wgrad(type, k, n, d, out) ? 0
                                         : kept_grad_ws_bytes(wgrad_args(type, k, n, d, out, dy));
}

int cb_ckpt_wgrad(int type, int k, int n, int d, int out, const void* kept, const void* dy,
                  void* dw, int64_t dstride, void* workspace_dev, size_t ws_bytes, void* stream) {
  return shielded((int)CB_EINVAL, [&]() -> int {
    const char* me = "cb_ckpt_wgrad";
    if (const char* why = wrong_wgrad(type, k, n, d, out)) return refuse(me, why);
    const int sz = lm_size(type);
    if (!at(kept, 16) || !at(dy, sz) || !at(dw, sz))
      return refuse(me, "kept, dy or dw NULL or misaligned");
    if (k > 1 && dstride < (int64_t)out * d) return refuse(me, "dstride is less than out * d");
    if (!at(workspace_dev, 256)) return refuse(me, "workspace NULL or not on 256 bytes");
    KeptGradArgs a = wgrad_args(type, k, n, d, out, dy);
    if (int rc = short_of(me, kept_grad_ws_bytes(a), ws_bytes)) return rc;
    a.kept = kept;
    a.dw = dw;
    a.dstride = dstride;
    a.ws = workspace_dev;
    return done(me, kept_grad(a, static_cast<hipStream_t>(stream)));
  });
}

}  // extern "C"
