// Entry points of the operators of token sequence models: their arguments are checked here, on the host, before anything is queued.
// They allocate nothing, wait for nothing and keep nothing but the text of a thread's last error.
#include "../../include/snn.h"
#include "snn_ops.h"

#include <stdarg.h>
#include <stdio.h>

namespace {

thread_local char g_error[512] = "";

snn_status refuse(snn_status s, const char *format, ...) {
  va_list args;
  va_start(args, format);
  vsnprintf(g_error, sizeof g_error, format, args);
  va_end(args);
  return s;
}

snn_status queued(hipError_t e, const char *what) {
  return e == hipSuccess ? SNN_OK : refuse(SNN_E_HIP, "%s: %s", what, hipGetErrorString(e));
}

// The device of a call is current while it lasts.
struct OnDevice {
  int before = -1;
  hipError_t error;
  explicit OnDevice(int device) {
    error = hipGetDevice(&before);
    if (error != hipSuccess || before == device) before = -1;
    else error = hipSetDevice(device);
    if (error != hipSuccess) {
      before = -1;
      (void)hipGetLastError(); // (the call says so; the thread's next one of any kind shall not find it)
    }
  }
  ~OnDevice() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

// One array of a call: what it is called, where it is, how its elements are aligned; `needed`: it may not be NULL.
struct Array { const char *name; const void *p; size_t align; bool needed; };
template <int N> snn_status check(const char *what, const snn_launch *at, const Array (&arrays)[N]) {
  for (const Array &a : arrays) {
    if (!a.p) {
      if (a.needed) return refuse(SNN_E_INVAL, "%s: %s is NULL", what, a.name);
      continue;
    }
    if ((uintptr_t)a.p % a.align) return refuse(SNN_E_INVAL, "%s: %s is not aligned to its elements", what, a.name);
    hipPointerAttribute_t at_;
    if (hipPointerGetAttributes(&at_, a.p) != hipSuccess) {
      (void)hipGetLastError();
      return refuse(SNN_E_INVAL, "%s: %s is not in device memory", what, a.name);
    }
    if (at_.type != hipMemoryTypeDevice || at_.device != at->device)
      return refuse(SNN_E_INVAL, "%s: %s is not in the memory of device %d", what, a.name, at->device);
  }
  return SNN_OK;
}
snn_status check_workspace(const char *what, const snn_launch *at, size_t bytes) {
  if (!bytes) return SNN_OK;
  if (!at->workspace || at->workspace_bytes < bytes)
    return refuse(SNN_E_INVAL, "%s: the workspace has %zu bytes, %zu are needed", what, at->workspace ? at->workspace_bytes : (size_t)0, bytes);
  const Array w[] = {{"the workspace", at->workspace, 256, true}};
  return check(what, at, w);
}

size_t size_of(int dtype) { return dtype == SNN_BF16 ? 2 : 4; }
bool dtype_ok(int dtype) { return dtype == SNN_F32 || dtype == SNN_BF16; }

#define CHECK(call)                    \
  do {                                 \
    const snn_status s_ = (call);      \
    if (s_ != SNN_OK) return s_;       \
  } while (0)

constexpr long long STEP_BYTES = 1 << 27; // of one step of an array, so that offsets inside 16 steps fit 32 bits
snn_status glr_shape(const char *what, const snn_glr *p, GlrShape *g) {
  if (!p) return refuse(SNN_E_INVAL, "%s: no shape", what);
  if (!dtype_ok(p->dtype)) return refuse(SNN_E_INVAL, "%s: unknown type %d", what, p->dtype);
  if (p->T < 0 || p->T > (1 << 30)) return refuse(SNN_E_INVAL, "%s: T = %d", what, p->T);
  if (p->batch < 1 || p->n < 1 || (long long)p->batch * p->n > STEP_BYTES / 4)
    return refuse(SNN_E_INVAL, "%s: batch %d, n %d: 1 .. 2^25 channels in all", what, p->batch, p->n);
  *g = GlrShape{p->T, p->batch, p->n, p->dtype == SNN_BF16, p->ld_z, p->ld_x, p->ld_h, p->ld_dz, p->ld_dx, p->lengths};
  for (long long *ld : {&g->ld_z, &g->ld_x, &g->ld_h, &g->ld_dz, &g->ld_dx}) {
    if (!*ld) *ld = p->n;
    if (*ld < p->n || *ld > STEP_BYTES / p->batch / (long long)size_of(p->dtype))
      return refuse(SNN_E_INVAL, "%s: %lld elements from row to row: n or more, and 2^27 bytes per step at most", what, *ld);
  }
  return SNN_OK;
}
snn_status launch_ok(const char *what, const snn_launch *at) { return at ? SNN_OK : refuse(SNN_E_INVAL, "%s: no device and stream", what); }

snn_status glr_backward(const char *what, const snn_launch *at, const snn_glr *p, GlrInputs in, const float *kept, const void *dh,
                        const float *dh_last, void *dz, void *dx, float *dh0) {
  GlrShape g;
  CHECK(launch_ok(what, at));
  CHECK(glr_shape(what, p, &g));
  const bool some = g.T > 0, packed = in.ze != nullptr || in.xe != nullptr;
  const size_t size = size_of(p->dtype);
  const Array arrays[] = {{packed ? "the codes of z" : "z", in.z, packed ? 1 : size, some}, {packed ? "the codes of x" : "x", in.x, packed ? 1 : size, some},
                          {"the exponents of z", in.ze, 1, packed && some}, {"the exponents of x", in.xe, 1, packed && some},
                          {"kept", kept, 4, some}, {"dh", dh, size, some}, {"dh_last", dh_last, 4, false}, {"dz", dz, size, some},
                          {"dx", dx, size, some}, {"dh0", dh0, 4, false}, {"lengths", g.lengths, 4, false}};
  CHECK(check(what, at, arrays));
  CHECK(check_workspace(what, at, glr_workspace(g)));
  const OnDevice on(at->device);
  if (on.error != hipSuccess) return queued(on.error, what);
  return queued(launch_glr_backward(g, in, kept, dh, dh_last, dz, dx, dh0, at->workspace, (hipStream_t)at->stream), what);
}

snn_status pack_shape(const char *what, const snn_launch *at, int dtype, int64_t rows, int32_t cols, int64_t *ld) {
  CHECK(launch_ok(what, at));
  if (!dtype_ok(dtype)) return refuse(SNN_E_INVAL, "%s: unknown type %d", what, dtype);
  if (rows < 0 || rows > INT32_MAX || cols < 1 || cols > (1 << 30) || (rows && cols > (1ll << 40) / rows))
    return refuse(SNN_E_INVAL, "%s: %lld rows of %d", what, (long long)rows, cols);
  if (!*ld) *ld = cols;
  if (*ld < cols) return refuse(SNN_E_INVAL, "%s: %lld elements from row to row, fewer than a row has", what, (long long)*ld);
  return SNN_OK;
}

snn_status vocab_shape(const char *what, const snn_vocab *p, VocabShape *v) {
  if (!p) return refuse(SNN_E_INVAL, "%s: no shape", what);
  if (!dtype_ok(p->dtype)) return refuse(SNN_E_INVAL, "%s: unknown type %d", what, p->dtype);
  if (p->rows < 0 || p->rows > (1 << 22) || p->d < 1 || p->d > (1 << 16) || p->vocab < 1 || p->vocab > (1 << 24))
    return refuse(SNN_E_INVAL, "%s: rows %d (0 .. 2^22), d %d (1 .. 2^16), vocab %d (1 .. 2^24)", what, p->rows, p->d, p->vocab);
  if ((long long)p->rows * p->d > 1ll << 35) // (what a grid of threads reaches)
    return refuse(SNN_E_INVAL, "%s: %d rows of %d elements: 2^35 in all at most", what, p->rows, p->d);
  *v = VocabShape{p->rows, p->d, p->vocab, p->dtype == SNN_BF16, p->ld_h, p->ld_w};
  for (long long *ld : {&v->ld_h, &v->ld_w}) {
    if (!*ld) *ld = p->d;
    if (*ld < p->d || *ld > (1 << 22)) return refuse(SNN_E_INVAL, "%s: %lld elements from row to row: d .. 2^22", what, *ld);
  }
  return SNN_OK;
}

} // namespace

extern "C" {

const char *snn_launch_error(void) { return g_error; }

size_t snn_glr_workspace(const snn_glr *p) {
  GlrShape g;
  return glr_shape("snn_glr_workspace", p, &g) == SNN_OK ? glr_workspace(g) : 0;
}

snn_status snn_glr_forward(const snn_launch *at, const snn_glr *p, const void *z, const void *x, const float *h0, void *h, float *h_last,
                           float *kept) {
  static const char what[] = "snn_glr_forward";
  GlrShape g;
  CHECK(launch_ok(what, at));
  CHECK(glr_shape(what, p, &g));
  const bool some = g.T > 0;
  const size_t size = size_of(p->dtype);
  const Array arrays[] = {{"z", z, size, some}, {"x", x, size, some}, {"h0", h0, 4, false}, {"h", h, size, some},
                          {"h_last", h_last, 4, false}, {"kept", kept, 4, false}, {"lengths", g.lengths, 4, false}};
  CHECK(check(what, at, arrays));
  CHECK(check_workspace(what, at, glr_workspace(g)));
  const OnDevice on(at->device);
  if (on.error != hipSuccess) return queued(on.error, what);
  return queued(launch_glr_forward(g, z, x, h0, h, h_last, kept, at->workspace, (hipStream_t)at->stream), what);
}

snn_status snn_glr_backward(const snn_launch *at, const snn_glr *p, const void *z, const void *x, const float *kept, const void *dh,
                            const float *dh_last, void *dz, void *dx, float *dh0) {
  return glr_backward("snn_glr_backward", at, p, GlrInputs{z, x, nullptr, nullptr, 0, 0, 0, 0}, kept, dh, dh_last, dz, dx, dh0);
}

snn_status snn_glr_backward_packed(const snn_launch *at, const snn_glr *p, const snn_packed *z, const snn_packed *x, const float *kept,
                                   const void *dh, const float *dh_last, void *dz, void *dx, float *dh0) {
  static const char what[] = "snn_glr_backward_packed";
  if (!p || !z || !x || (p->T > 0 && (!z->codes || !x->codes || !z->exps || !x->exps)))
    return refuse(SNN_E_INVAL, "%s: no shape, or z or x without codes or exponents", what);
  GlrInputs in = {z->codes, x->codes, z->exps, x->exps, z->ld, x->ld, z->ld_exps, x->ld_exps};
  const int64_t bytes = (int64_t)((uint32_t)(p->n > 0 ? p->n : 1) + SNN_PACK_BLOCK - 1) / SNN_PACK_BLOCK;
  for (long long *ld : {&in.ld_z, &in.ld_x, &in.ld_ze, &in.ld_xe}) {
    const int64_t least = ld == &in.ld_z || ld == &in.ld_x ? p->n : bytes;
    if (!*ld) *ld = least;
    if (*ld < least || (p->batch > 0 && *ld > STEP_BYTES / p->batch))
      return refuse(SNN_E_INVAL, "%s: %lld codes or exponents from row to row", what, *ld);
  }
  if (p->T <= 0) in = GlrInputs{};
  return glr_backward(what, at, p, in, kept, dh, dh_last, dz, dx, dh0);
}

snn_status snn_pack(const snn_launch *at, int dtype, int64_t rows, int32_t cols, int64_t ld, const void *x, int8_t *codes, uint8_t *exps) {
  static const char what[] = "snn_pack";
  CHECK(pack_shape(what, at, dtype, rows, cols, &ld));
  if (!rows) return SNN_OK;
  const Array arrays[] = {{"x", x, size_of(dtype), true}, {"the codes", codes, 1, true}, {"the exponents", exps, 1, true}};
  CHECK(check(what, at, arrays));
  const OnDevice on(at->device);
  if (on.error != hipSuccess) return queued(on.error, what);
  return queued(launch_pack(dtype == SNN_BF16, rows, cols, ld, x, codes, exps, (hipStream_t)at->stream), what);
}

snn_status snn_unpack(const snn_launch *at, int dtype, int64_t rows, int32_t cols, int64_t ld, const int8_t *codes, const uint8_t *exps,
                      void *x) {
  static const char what[] = "snn_unpack";
  CHECK(pack_shape(what, at, dtype, rows, cols, &ld));
  if (!rows) return SNN_OK;
  const Array arrays[] = {{"x", x, size_of(dtype), true}, {"the codes", codes, 1, true}, {"the exponents", exps, 1, true}};
  CHECK(check(what, at, arrays));
  const OnDevice on(at->device);
  if (on.error != hipSuccess) return queued(on.error, what);
  return queued(launch_unpack(dtype == SNN_BF16, rows, cols, ld, codes, exps, x, (hipStream_t)at->stream), what);
}

size_t snn_vocab_workspace(const snn_vocab *p, int32_t gradients) {
  VocabShape v;
  return vocab_shape("snn_vocab_workspace", p, &v) == SNN_OK ? vocab_workspace(v, gradients != 0) : 0;
}

snn_status snn_vocab_loss(const snn_launch *at, const snn_vocab *p, const void *h, const void *w, const int32_t *targets, float *loss,
                          float *state) {
  static const char what[] = "snn_vocab_loss";
  VocabShape v;
  CHECK(launch_ok(what, at));
  CHECK(vocab_shape(what, p, &v));
  if (!v.rows) return SNN_OK;
  const size_t size = size_of(p->dtype);
  const Array arrays[] = {{"h", h, size, true}, {"w", w, size, true}, {"targets", targets, 4, true}, {"loss", loss, 4, true}, {"state", state, 4, true}};
  CHECK(check(what, at, arrays));
  CHECK(check_workspace(what, at, vocab_workspace(v, false)));
  const OnDevice on(at->device);
  if (on.error != hipSuccess) return queued(on.error, what);
  return queued(launch_vocab_loss(v, h, w, targets, loss, state, at->workspace, (hipStream_t)at->stream), what);
}

snn_status snn_vocab_loss_grad(const snn_launch *at, const snn_vocab *p, const void *h, const void *w, const int32_t *targets,
                               const float *state, const float *dloss, void *dh, void *dw) {
  static const char what[] = "snn_vocab_loss_grad";
  VocabShape v;
  CHECK(launch_ok(what, at));
  CHECK(vocab_shape(what, p, &v));
  const size_t size = size_of(p->dtype);
  const bool some = v.rows > 0;
  const Array arrays[] = {{"h", h, size, some}, {"w", w, size, some}, {"targets", targets, 4, some}, {"state", state, 4, some},
                          {"dloss", dloss, 4, false}, {"dh", dh, size, some}, {"dw", dw, size, true}};
  CHECK(check(what, at, arrays));
  if (some) CHECK(check_workspace(what, at, vocab_workspace(v, true)));
  const OnDevice on(at->device);
  if (on.error != hipSuccess) return queued(on.error, what);
  return queued(launch_vocab_grad(v, h, w, targets, state, dloss, dh, dw, at->workspace, (hipStream_t)at->stream), what);
}

} // extern "C"
