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
