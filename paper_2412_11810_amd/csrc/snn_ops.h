// Internal declarations of the operators of token sequence models: what the entry points (snn_ops.cpp) hand to the kernels'
// launchers.  Everything is checked by then.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

// ---- gated linear recurrence (snn_glr.hip) ------------------------------------------------
#define SNN_GLR_INTERVAL 128 // steps between the states that the forward pass keeps
#define SNN_PACK_BLOCK 32    // consecutive elements of a row that share a step in 8 bits

struct GlrShape {
  int T, batch, n;
  bool bf16;
  long long ld_z, ld_x, ld_h, ld_dz, ld_dx; // elements between the rows (t, b) of an array (ld_h: of h and dh)
  const int *lengths;         // NULL: T steps each
};
// z and x of a backward pass: arrays of the shape's type, or 8-bit codes with an exponent byte for each block (ze, xe != NULL)
struct GlrInputs {
  const void *z, *x;
  const uint8_t *ze, *xe;
  long long ld_z, ld_x, ld_ze, ld_xe; // of the codes and bytes
};
size_t glr_workspace(const GlrShape &p);
hipError_t launch_glr_forward(const GlrShape &p, const void *z, const void *x, const float *h0, void *h, float *h_last, float *kept,
                              void *work, hipStream_t s);
hipError_t launch_glr_backward(const GlrShape &p, const GlrInputs &in, const float *kept, const void *dh, const float *dh_last,
                               void *dz, void *dx, float *dh0, void *work, hipStream_t s);

// ---- activations in 8 bits (snn_pack.hip) ---------------------------------------------------
hipError_t launch_pack(bool bf16, long long rows, int cols, long long ld, const void *x, int8_t *codes, uint8_t *exps, hipStream_t s);
hipError_t launch_unpack(bool bf16, long long rows, int cols, long long ld, const int8_t *codes, const uint8_t *exps, void *x,
                         hipStream_t s);

// ---- softmax cross entropy over a vocabulary (snn_vocab.hip) --------------------------------
struct VocabShape {
  int rows, d, vocab;
  bool bf16;
  long long ld_h, ld_w; // elements between rows of h, w
};
size_t vocab_workspace(const VocabShape &p, bool grad);
hipError_t launch_vocab_loss(const VocabShape &p, const void *h, const void *w, const int *targets, float *loss, float *state,
                             void *work, hipStream_t s);
hipError_t launch_vocab_grad(const VocabShape &p, const void *h, const void *w, const int *targets, const float *state,
                             const float *dloss, void *dh, void *dw, void *work, hipStream_t s);

// ---- root-mean-square norm (snn_norm.hip) ---------------------------------------------------
struct NormShape {
  long long rows;
  int n;
  bool bf16;
  float eps;
  long long ld_x, ld_residual, ld_total, ld_y, ld_dtotal, ld_dx; // elements between rows (ld_y: of y and dy)
};
size_t norm_workspace(const NormShape &p); // of the backward pass
// y, or codes and exps, of x + residual (NULL: of x), which goes to total (NULL: nowhere); w may be NULL
hipError_t launch_norm(const NormShape &p, const void *x, const void *residual, const void *w, void *total, void *y, int8_t *codes, uint8_t *exps,
                       hipStream_t s);
// dtotal, dw may be NULL
hipError_t launch_norm_backward(const NormShape &p, const void *total, const void *w, const void *dy, const void *dtotal, void *dx, void *dw,
                                float *sums, hipStream_t s);

// ---- AdamW (snn_adamw.hip) ------------------------------------------------------------------
struct AdamwStep {
  double lr, beta1, beta2, eps, decay;
  long long t;  // the step's number, or
  int *count;   // where it is, less one, on the device
  const float *scale; // of the gradients; NULL: 1
};
struct AdamwTensor {
  void *p;
  const void *g;
  void *m, *v;                 // 32 bits, or codes where there are
  uint8_t *m_exps, *v_exps;
  void *copy;                  // bf16 or NULL
  long long n;
  bool p16, g16;
};
size_t adamw_workspace(); // where the count is on the device
hipError_t launch_adamw(const AdamwStep &how, const AdamwTensor *tensors, long long count, void *work, hipStream_t s);

// ---- gated delta rule (snn_delta.hip) -------------------------------------------------------
#define SNN_DELTA_INTERVAL 256 // steps between the states that the forward pass keeps

struct DeltaShape {
  int T, batch, heads, key_heads, dk, dv;
  bool bf16;
  float scale;
  long long ld_q, ld_k, ld_v, ld_o, ld_dq, ld_dk, ld_dv; // elements between the rows (t, b) of an array (ld_o: of o and its gradient)
  const int *lengths;                                    // NULL: T steps each
};
size_t delta_workspace(const DeltaShape &p, bool back);
hipError_t launch_delta_forward(const DeltaShape &p, const void *q, const void *k, const void *v, const float *g, const float *beta, const float *s0,
                                void *o, float *s_last, float *kept, void *work, hipStream_t s);
hipError_t launch_delta_backward(const DeltaShape &p, const void *q, const void *k, const void *v, const float *g, const float *beta, const float *kept,
                                 const void *dout, const float *ds_last, void *dq, void *dk, void *dv, float *dg, float *dbeta, float *ds0, void *work,
                                 hipStream_t s);
