// The operators' entry points (snn_ops.cpp) over a stand-in for the HIP runtime and for their kernels: all memory is device 0's, a launch only counts.  A shared
// library, whose calls are made by tests/test_host_ops.py.
#include "snn_ops.cpp"

static int g_launches = 0;
extern "C" int launches() { return g_launches; }

#define HIP(name, ...) extern "C" hipError_t name(__VA_ARGS__)
HIP(hipGetDevice, int *device) { *device = 0; return hipSuccess; }
HIP(hipSetDevice, int) { return hipSuccess; }
HIP(hipGetLastError) { return hipSuccess; }
extern "C" const char *hipGetErrorString(hipError_t) { return "error"; }
HIP(hipPointerGetAttributes, hipPointerAttribute_t *to, const void *) {
  to->type = hipMemoryTypeDevice;
  to->device = 0;
  return hipSuccess;
}

static hipError_t launched() { ++g_launches; return hipSuccess; }
size_t glr_workspace(const GlrShape &) { return 0; }
hipError_t launch_glr_forward(const GlrShape &, const void *, const void *, const float *, void *, float *, float *, void *, hipStream_t) { return launched(); }
hipError_t launch_glr_backward(const GlrShape &, const GlrInputs &, const float *, const void *, const float *, void *, void *, float *, void *, hipStream_t) { return launched(); }
hipError_t launch_pack(bool, long long, int, long long, const void *, int8_t *, uint8_t *, hipStream_t) { return launched(); }
hipError_t launch_unpack(bool, long long, int, long long, const int8_t *, const uint8_t *, void *, hipStream_t) { return launched(); }
size_t vocab_workspace(const VocabShape &, bool) { return 0; }
hipError_t launch_vocab_loss(const VocabShape &, const void *, const void *, const int *, float *, float *, void *, hipStream_t) { return launched(); }
hipError_t launch_vocab_grad(const VocabShape &, const void *, const void *, const int *, const float *, const float *, void *, void *, void *, hipStream_t) { return launched(); }
size_t norm_workspace(const NormShape &) { return 0; }
hipError_t launch_norm(const NormShape &, const void *, const void *, const void *, void *, void *, int8_t *, uint8_t *, hipStream_t) { return launched(); }
hipError_t launch_norm_backward(const NormShape &, const void *, const void *, const void *, const void *, void *, void *, float *, hipStream_t) { return launched(); }
size_t adamw_workspace() { return 0; }
hipError_t launch_adamw(const AdamwStep &, const AdamwTensor *, long long, void *, hipStream_t) { return launched(); }
size_t delta_workspace(const DeltaShape &, bool) { return 0; }
hipError_t launch_delta_forward(const DeltaShape &, const void *, const void *, const void *, const float *, const float *, const float *, void *, float *, float *, void *, hipStream_t) { return launched(); }
hipError_t launch_delta_backward(const DeltaShape &, const void *, const void *, const void *, const float *, const float *, const float *, const void *, const float *, void *, void *, void *, float *, float *, float *, void *, hipStream_t) { return launched(); }
