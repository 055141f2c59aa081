// Entry points of the operators of token sequence models: their arguments are checked here, on the host, before anything is queued.
// They allocate nothing, wait for nothing and keep nothing but the text of a thread's last error.
#include "../../include/snn.h"
#include "snn_ops.h"
#include "snn_share.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <stdarg.h>
#include <stdio.h>
#include <utility>
#include <vector>

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

// An array of a call by the memory that it takes; a result may share none with another one, but that it may take the place of those whose numbers are in `of`.
struct Part { const char *name; Rows at; bool result; unsigned of; };
Rows in_one(const void *p, int64_t elements, size_t size) { return Rows{p, 1, elements * (int64_t)size, elements * (int64_t)size}; }
template <int N> snn_status apart(const char *what, const Part (&parts)[N]) {
  for (int i = 0; i < N; ++i)
    for (int j = 0; j < N && parts[i].result; ++j) {
      if (i == j || (parts[j].result && j < i) || ((parts[i].of >> j & 1) && same_place(parts[i].at, parts[j].at))) continue;
      if (share(parts[i].at, parts[j].at)) return refuse(SNN_E_INVAL, "%s: %s and %s share elements", what, parts[i].name, parts[j].name);
    }
  return SNN_OK;
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

snn_status delta_shape(const char *what, const snn_delta *p, bool back, DeltaShape *d) {
  if (!p) return refuse(SNN_E_INVAL, "%s: no shape", what);
  if (!dtype_ok(p->dtype)) return refuse(SNN_E_INVAL, "%s: unknown type %d", what, p->dtype);
  if (p->T < 0 || p->T > (1 << 30)) return refuse(SNN_E_INVAL, "%s: T = %d", what, p->T);
  if (p->key_heads < 1 || p->heads < 1 || p->heads % p->key_heads)
    return refuse(SNN_E_INVAL, "%s: %d heads, %d of keys: the first must be a multiple of the second", what, p->heads, p->key_heads);
  if (p->dk < 1 || p->dk > 128 || p->dv < 1 || p->dv > 1024) return refuse(SNN_E_INVAL, "%s: dk %d (1 .. 128), dv %d (1 .. 1024)", what, p->dk, p->dv);
  if (p->batch < 1 || (long long)p->batch * p->heads > 1 << 20 || (long long)p->batch * p->heads * p->dv > 1 << 28)
    return refuse(SNN_E_INVAL, "%s: batch %d, %d heads, dv %d: 2^20 heads and 2^28 columns of states in all at most", what, p->batch, p->heads, p->dv);
  if (!std::isfinite(p->scale)) return refuse(SNN_E_INVAL, "%s: scale = %g", what, p->scale);
  *d = DeltaShape{p->T, p->batch, p->heads, p->key_heads, p->dk, p->dv, p->dtype == SNN_BF16, p->scale,
                  p->ld_q, p->ld_k, p->ld_v, p->ld_o, p->ld_dq, p->ld_dk, p->ld_dv, p->lengths};
  const int64_t of_keys = (int64_t)p->key_heads * p->dk, of_values = (int64_t)p->heads * p->dv;
  const std::pair<long long *, int64_t> lds[] = {{&d->ld_q, of_keys}, {&d->ld_k, of_keys}, {&d->ld_v, of_values}, {&d->ld_o, of_values},
                                                 {&d->ld_dq, of_keys}, {&d->ld_dk, of_keys}, {&d->ld_dv, of_values}};
  // places in a chunk of 64 steps fit 32 bits; a step by itself has no chunk
  const long long most = p->T == 1 && !back ? 1ll << 40 : (1 << 25) / p->batch / (long long)size_of(p->dtype);
  for (auto [ld, least] : lds) {
    if (!*ld) *ld = least;
    if (*ld < least || *ld > most)
      return refuse(SNN_E_INVAL, "%s: %lld elements from row to row: those of all heads or more, and 2^25 bytes per step at most (2^40 elements for one step forward)", what, *ld);
  }
  return SNN_OK;
}

struct DeltaParts {
  const DeltaShape &d;
  size_t size;
  Rows rows(const void *p, long long ld, bool keys) const { // of the steps and sequences, with all heads
    return Rows{p, (int64_t)d.T * d.batch, (int64_t)size * (keys ? d.key_heads * d.dk : d.heads * d.dv), ld * (int64_t)size};
  }
  Rows gates(const float *p) const { return in_one(p, (int64_t)d.T * d.batch * d.heads, 4); }
  Rows states(const float *p, int64_t n) const { return in_one(p, n * d.batch * d.heads * d.dk * d.dv, 4); }
  Rows kept(const float *p) const { return states(p, (d.T + SNN_DELTA_INTERVAL - 1) / SNN_DELTA_INTERVAL); }
};

snn_status norm_shape(const char *what, const snn_norm *p, NormShape *n) {
  if (!p) return refuse(SNN_E_INVAL, "%s: no shape", what);
  if (!dtype_ok(p->dtype)) return refuse(SNN_E_INVAL, "%s: unknown type %d", what, p->dtype);
  if (p->n < 1 || p->n > (1 << 15) || p->rows < 0 || p->rows > (1ll << 40) / p->n)
    return refuse(SNN_E_INVAL, "%s: %lld rows of %d: 1 .. 2^15 elements, 2^40 in all at most", what, (long long)p->rows, p->n);
  if (!(p->eps >= 0.f) || !(p->eps < 1e30f)) return refuse(SNN_E_INVAL, "%s: eps = %g", what, p->eps);
  *n = NormShape{p->rows, p->n, p->dtype == SNN_BF16, p->eps, p->ld_x, p->ld_residual, p->ld_total, p->ld_y, p->ld_dtotal, p->ld_dx};
  for (long long *ld : {&n->ld_x, &n->ld_residual, &n->ld_total, &n->ld_y, &n->ld_dtotal, &n->ld_dx}) {
    if (!*ld) *ld = p->n;
    if (*ld < p->n || *ld > (1ll << 40)) return refuse(SNN_E_INVAL, "%s: %lld elements from row to row: n .. 2^40", what, *ld);
  }
  return SNN_OK;
}

snn_status norm_forward(const char *what, const snn_launch *at, const snn_norm *p, const void *x, const void *residual, const void *w, void *total,
                        void *y, int8_t *codes, uint8_t *exps, bool packed) {
  NormShape n;
  CHECK(launch_ok(what, at));
  CHECK(norm_shape(what, p, &n));
  if (!n.rows) return SNN_OK;
  const size_t size = size_of(p->dtype);
  const Array arrays[] = {{"x", x, size, true}, {"residual", residual, size, false}, {"w", w, size, false}, {"total", total, size, false},
                          {"y", y, size, !packed}, {"the codes", codes, 1, packed}, {"the exponents", exps, 1, packed}};
  CHECK(check(what, at, arrays));
  if (total && !residual) return refuse(SNN_E_INVAL, "%s: a total without a residual", what);
  auto rows = [&](const void *q, long long ld) { return Rows{q, n.rows, n.n * (int64_t)size, ld * (int64_t)size}; };
  const Part parts[] = {{"x", rows(x, n.ld_x)}, {"residual", rows(residual, n.ld_residual)}, {"w", in_one(w, n.n, size)}, {"total", rows(total, n.ld_total), true, 1u << 0 | 1u << 1},
                        {"y", rows(y, n.ld_y), true, 1u << 0 | 1u << 1}, {"the codes", in_one(codes, n.rows * n.n, 1), true},
                        {"the exponents", in_one(exps, n.rows * ((n.n + SNN_PACK_BLOCK - 1) / SNN_PACK_BLOCK), 1), true}};
  CHECK(apart(what, parts));
  const OnDevice on(at->device);
  if (on.error != hipSuccess) return queued(on.error, what);
  return queued(launch_norm(n, x, residual, w, total, y, codes, exps, (hipStream_t)at->stream), what);
}

// No two of the arrays that a step writes may share elements: it would change them twice, or at the same time.
struct Written { uintptr_t from, to; };
snn_status adamw_arrays(const char *what, const snn_launch *at, const snn_adamw *how, const snn_adamw_tensor *tensors, int64_t count, std::vector<AdamwTensor> &out) {
  std::vector<Written> written;
  out.reserve(count);
  written.reserve(6 * count + 1);
  if (how->step_on_device) written.push_back({(uintptr_t)how->step_on_device, (uintptr_t)how->step_on_device + 4});
  for (int64_t k = 0; k < count; ++k) {
    const snn_adamw_tensor &x = tensors[k];
    if (!dtype_ok(x.dtype_p) || !dtype_ok(x.dtype_g)) return refuse(SNN_E_INVAL, "%s: tensor %lld: unknown type", what, (long long)k);
    if (x.n < 0 || x.n > (1ll << 40)) return refuse(SNN_E_INVAL, "%s: tensor %lld: %lld elements: 0 .. 2^40", what, (long long)k, (long long)x.n);
    if (!x.m_exps != !x.v_exps) return refuse(SNN_E_INVAL, "%s: tensor %lld: one moment with exponents, one without", what, (long long)k);
    if (x.copy && x.dtype_p != SNN_F32) return refuse(SNN_E_INVAL, "%s: tensor %lld: a copy in bf16 of what is in bf16", what, (long long)k);
    if (!x.n) continue;
    const bool eight = x.m_exps != nullptr;
    const size_t size_p = size_of(x.dtype_p), size_m = eight ? 1 : 4;
    const Array arrays[] = {{"p", x.p, size_p, true}, {"g", x.g, size_of(x.dtype_g), true}, {"m", x.m, size_m, true}, {"v", x.v, size_m, true},
                            {"the exponents of m", x.m_exps, 1, eight}, {"the exponents of v", x.v_exps, 1, eight}, {"the copy", x.copy, 2, false}};
    CHECK(check(what, at, arrays));
    const size_t exps = (x.n + SNN_PACK_BLOCK - 1) / SNN_PACK_BLOCK;
    const std::pair<const void *, size_t> to[] = {{x.p, x.n * size_p}, {x.m, x.n * size_m}, {x.v, x.n * size_m}, {x.m_exps, exps}, {x.v_exps, exps}, {x.copy, 2 * x.n}};
    for (auto [p, bytes] : to)
      if (p) written.push_back({(uintptr_t)p, (uintptr_t)p + bytes});
    out.push_back(AdamwTensor{x.p, x.g, x.m, x.v, x.m_exps, x.v_exps, x.copy, x.n, x.dtype_p == SNN_BF16, x.dtype_g == SNN_BF16});
  }
  std::sort(written.begin(), written.end(), [](const Written &a, const Written &b) { return a.from < b.from; });
  for (size_t i = 1; i < written.size(); ++i)
    if (written[i].from < written[i - 1].to) return refuse(SNN_E_INVAL, "%s: two of the arrays that the step writes share elements", what);
  auto writes = [&](const void *p, int64_t bytes) { // any of these
    const auto next = std::upper_bound(written.begin(), written.end(), (uintptr_t)p, [](uintptr_t v, const Written &w) { return v < w.to; });
    return next != written.end() && next->from < (uintptr_t)p + bytes;
  };
  for (const AdamwTensor &x : out) // a gradient may be anywhere but in what is written
    if (writes(x.g, x.n * (x.g16 ? 2 : 4))) return refuse(SNN_E_INVAL, "%s: a gradient shares elements with an array that the step writes", what);
  if (how->grad_scale && writes(how->grad_scale, 4)) return refuse(SNN_E_INVAL, "%s: the gradients' scale shares elements with an array that the step writes", what);
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

size_t snn_delta_workspace(const snn_delta *p, int32_t gradients) {
  DeltaShape d;
  return delta_shape("snn_delta_workspace", p, gradients != 0, &d) == SNN_OK ? delta_workspace(d, gradients != 0) : 0;
}

snn_status snn_delta_forward(const snn_launch *at, const snn_delta *p, const void *q, const void *k, const void *v, const float *g, const float *beta,
                             const float *s0, void *o, float *s_last, float *kept) {
  static const char what[] = "snn_delta_forward";
  DeltaShape d;
  CHECK(launch_ok(what, at));
  CHECK(delta_shape(what, p, false, &d));
  const bool some = d.T > 0;
  const size_t size = size_of(p->dtype);
  const Array arrays[] = {{"q", q, size, some}, {"k", k, size, some}, {"v", v, size, some}, {"g", g, 4, some}, {"beta", beta, 4, some}, {"s0", s0, 4, false},
                          {"o", o, size, some}, {"s_last", s_last, 4, false}, {"kept", kept, 4, false}, {"lengths", d.lengths, 4, false}};
  CHECK(check(what, at, arrays));
  CHECK(check_workspace(what, at, delta_workspace(d, false)));
  const DeltaParts part{d, size};
  const Part parts[] = {{"q", part.rows(q, d.ld_q, true)}, {"k", part.rows(k, d.ld_k, true)}, {"v", part.rows(v, d.ld_v, false)}, {"g", part.gates(g)},
                        {"beta", part.gates(beta)}, {"s0", part.states(s0, 1)}, {"lengths", in_one(d.lengths, d.batch, 4)},
                        {"o", part.rows(o, d.ld_o, false), true, 1u << 2}, {"s_last", part.states(s_last, 1), true, 1u << 5}, {"kept", part.kept(kept), true}};
  CHECK(apart(what, parts));
  const OnDevice on(at->device);
  if (on.error != hipSuccess) return queued(on.error, what);
  return queued(launch_delta_forward(d, q, k, v, g, beta, s0, o, s_last, kept, at->workspace, (hipStream_t)at->stream), what);
}

snn_status snn_delta_backward(const snn_launch *at, const snn_delta *p, const void *q, const void *k, const void *v, const float *g, const float *beta,
                              const float *kept, const void *dout, const float *ds_last, void *dq, void *dk, void *dv, float *dg, float *dbeta, float *ds0) {
  static const char what[] = "snn_delta_backward";
  DeltaShape d;
  CHECK(launch_ok(what, at));
  CHECK(delta_shape(what, p, true, &d));
  const bool some = d.T > 0;
  const size_t size = size_of(p->dtype);
  const Array arrays[] = {{"q", q, size, some}, {"k", k, size, some}, {"v", v, size, some}, {"g", g, 4, some}, {"beta", beta, 4, some}, {"kept", kept, 4, some},
                          {"do", dout, size, some}, {"ds_last", ds_last, 4, false}, {"dq", dq, size, some}, {"dk", dk, size, some}, {"dv", dv, size, some},
                          {"dg", dg, 4, some}, {"dbeta", dbeta, 4, some}, {"ds0", ds0, 4, false}, {"lengths", d.lengths, 4, false}};
  CHECK(check(what, at, arrays));
  CHECK(check_workspace(what, at, delta_workspace(d, true)));
  const DeltaParts part{d, size};
  const Part parts[] = {{"q", part.rows(q, d.ld_q, true)}, {"k", part.rows(k, d.ld_k, true)}, {"v", part.rows(v, d.ld_v, false)}, {"g", part.gates(g)},
                        {"beta", part.gates(beta)}, {"kept", part.kept(kept)}, {"do", part.rows(dout, d.ld_o, false)}, {"ds_last", part.states(ds_last, 1)},
                        {"lengths", in_one(d.lengths, d.batch, 4)}, {"dq", part.rows(dq, d.ld_dq, true), true, 1u << 0},
                        {"dk", part.rows(dk, d.ld_dk, true), true, 1u << 1}, {"dv", part.rows(dv, d.ld_dv, false), true, 1u << 2},
                        {"dg", part.gates(dg), true, 1u << 3}, {"dbeta", part.gates(dbeta), true, 1u << 4}, {"ds0", part.states(ds0, 1), true, 1u << 7}};
  CHECK(apart(what, parts));
  const OnDevice on(at->device);
  if (on.error != hipSuccess) return queued(on.error, what);
  return queued(launch_delta_backward(d, q, k, v, g, beta, kept, dout, ds_last, dq, dk, dv, dg, dbeta, ds0, at->workspace, (hipStream_t)at->stream), what);
}

size_t snn_norm_workspace(const snn_norm *p) {
  NormShape n;
  return norm_shape("snn_norm_workspace", p, &n) == SNN_OK ? norm_workspace(n) : 0;
}

snn_status snn_norm_forward(const snn_launch *at, const snn_norm *p, const void *x, const void *residual, const void *w, void *total, void *y) {
  return norm_forward("snn_norm_forward", at, p, x, residual, w, total, y, nullptr, nullptr, false);
}

snn_status snn_norm_forward_packed(const snn_launch *at, const snn_norm *p, const void *x, const void *residual, const void *w, void *total,
                                   int8_t *codes, uint8_t *exps) {
  return norm_forward("snn_norm_forward_packed", at, p, x, residual, w, total, nullptr, codes, exps, true);
}

snn_status snn_norm_backward(const snn_launch *at, const snn_norm *p, const void *total, const void *w, const void *dy, const void *dtotal, void *dx,
                             void *dw) {
  static const char what[] = "snn_norm_backward";
  NormShape n;
  CHECK(launch_ok(what, at));
  CHECK(norm_shape(what, p, &n));
  const size_t size = size_of(p->dtype);
  const bool some = n.rows > 0;
  if (!some && !dw) return SNN_OK;
  const Array arrays[] = {{"total", total, size, some}, {"w", w, size, dw != nullptr}, {"dy", dy, size, some}, {"dtotal", dtotal, size, false},
                          {"dx", dx, size, some}, {"dw", dw, size, false}};
  CHECK(check(what, at, arrays));
  if (dw) CHECK(check_workspace(what, at, norm_workspace(n)));
  auto rows = [&](const void *q, long long ld) { return Rows{q, n.rows, n.n * (int64_t)size, ld * (int64_t)size}; };
  const Part parts[] = {{"total", rows(total, n.ld_total)}, {"dy", rows(dy, n.ld_y)}, {"dtotal", rows(dtotal, n.ld_dtotal)}, {"w", in_one(w, n.n, size)},
                        {"dx", rows(dx, n.ld_dx), true, 1u << 0 | 1u << 1 | 1u << 2}, {"dw", in_one(dw, n.n, size), true}};
  CHECK(apart(what, parts));
  const OnDevice on(at->device);
  if (on.error != hipSuccess) return queued(on.error, what);
  return queued(launch_norm_backward(n, total, w, dy, dtotal, dx, dw, (float *)at->workspace, (hipStream_t)at->stream), what);
}

size_t snn_adamw_workspace(const snn_adamw *how) { return how && how->step_on_device ? adamw_workspace() : 0; }

snn_status snn_adamw_step(const snn_launch *at, const snn_adamw *how, const snn_adamw_tensor *tensors, int64_t count) {
  static const char what[] = "snn_adamw_step";
  CHECK(launch_ok(what, at));
  if (!how || count < 0 || count > (1 << 24) || (count && !tensors)) return refuse(SNN_E_INVAL, "%s: no step, or no tensors", what);
  if (!std::isfinite(how->lr) || !std::isfinite(how->weight_decay) || !(how->beta1 >= 0 && how->beta1 < 1) || !(how->beta2 >= 0 && how->beta2 < 1) ||
      !(how->eps >= 0 && how->eps < 1e30))
    return refuse(SNN_E_INVAL, "%s: lr %g, betas %g and %g (0 .. 1, less than 1), eps %g, weight decay %g", what, how->lr, how->beta1, how->beta2,
                  how->eps, how->weight_decay);
  if (!how->step_on_device && how->step < 1) return refuse(SNN_E_INVAL, "%s: step %lld: the first one is 1", what, (long long)how->step);
  const Array arrays[] = {{"the step", how->step_on_device, 4, false}, {"the gradients' scale", how->grad_scale, 4, false}};
  CHECK(check(what, at, arrays));
  CHECK(check_workspace(what, at, snn_adamw_workspace(how)));
  try {
    std::vector<AdamwTensor> all;
    CHECK(adamw_arrays(what, at, how, tensors, count, all));
    const OnDevice on(at->device);
    if (on.error != hipSuccess) return queued(on.error, what);
    const AdamwStep step = {how->lr, how->beta1, how->beta2, how->eps, how->weight_decay, how->step, how->step_on_device, how->grad_scale};
    return queued(launch_adamw(step, all.data(), (long long)all.size(), at->workspace, (hipStream_t)at->stream), what);
  } catch (const std::bad_alloc &) {
    return refuse(SNN_E_HOSTMEM, "%s: no memory for the descriptions of %lld tensors", what, (long long)count);
  }
}

} // extern "C"
