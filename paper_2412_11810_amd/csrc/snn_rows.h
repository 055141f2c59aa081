// What kernels over rows of elements share: 8 elements of a lane between memory and registers, and blocks of 32 in 8 bits (four lanes).
#pragma once
#include "snn_ops.h"
#include <type_traits>

namespace {

constexpr int LANE = 8; // elements of a lane

// Rows need not begin on whole words: these loads and stores may be at any address
typedef float two __attribute__((ext_vector_type(2)));
typedef __bf16 two_bf16 __attribute__((ext_vector_type(2)));
typedef uint32_t words4 __attribute__((ext_vector_type(4)));
typedef words4 words4_any __attribute__((aligned(2)));
typedef uint32_t words2 __attribute__((ext_vector_type(2)));
typedef words2 words2_any __attribute__((aligned(1)));

template <typename T> __device__ __forceinline__ void read(const T *p, int count, float (&v)[LANE]) {
  if (count >= LANE) {
    if constexpr (sizeof(T) == 2) {
      const words4 r = *(const words4_any *)p;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[2 * j] = __uint_as_float(r[j] << 16);
        v[2 * j + 1] = __uint_as_float(r[j] & 0xffff0000u);
      }
    } else {
      const words4 r[2] = {*(const words4_any *)p, *(const words4_any *)(p + 4)};
#pragma unroll
      for (int j = 0; j < LANE; ++j) v[j] = __uint_as_float(r[j / 4][j % 4]);
    }
  } else
#pragma unroll
    for (int j = 0; j < LANE; ++j) v[j] = j < count ? (float)p[j] : 0.f;
}
template <typename T> __device__ __forceinline__ void write(T *p, int count, const float (&v)[LANE]) {
  if (count >= LANE) {
    if constexpr (sizeof(T) == 2) {
      words4 r;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        r[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(two{v[2 * j], v[2 * j + 1]}, two_bf16));
      *(words4_any *)p = r;
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        words4 r;
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = __float_as_uint(v[4 * i + j]);
        *(words4_any *)(p + 4 * i) = r;
      }
    }
  } else
#pragma unroll
    for (int j = 0; j < LANE; ++j)
      if (j < count) p[j] = (T)v[j];
}

// The step that a block's elements share, from the largest of a lane's as bits (an infinity or NaN is above every number)
struct Step { uint8_t byte; float per_step; bool bad; };
__device__ __forceinline__ uint32_t most_of_block(uint32_t top) {
  top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xb1, 0xf, 0xf, false)); // quad lanes 1 0 3 2
  return max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x4e, 0xf, 0xf, false)); // quad lanes 2 3 0 1
}
// `past`: mantissa from which the largest element is more than 127 steps of the smaller power of two
__device__ __forceinline__ Step step_of(uint32_t top, uint32_t past) {
  // (2^121 is the largest step whose multiples are all floats)
  const int e = min(max((int)(top >> 23) - 6 + ((top & 0x7fffffu) >= past), 1), 248);
  const bool none = top == 0, bad = top >= 0x7f800000u;
  return Step{(uint8_t)(bad ? 255 : none ? 0 : e), __uint_as_float((uint32_t)(254 - e) << 23), bad};
}
// (127.5 steps would round to 128)
__device__ __forceinline__ Step block_step(uint32_t top) { return step_of(most_of_block(top), 0x7f0000u); }
__device__ __forceinline__ void write_bytes(int8_t *to, int count, const int (&k)[LANE]) {
  uint32_t c[2] = {};
#pragma unroll
  for (int j = 0; j < LANE; ++j) c[j / 4] |= (uint32_t)(k[j] & 0xff) << (8 * (j % 4));
  if (count >= LANE) {
    words2 r;
    r[0] = c[0];
    r[1] = c[1];
    *(words2_any *)to = r;
  } else
#pragma unroll
    for (int j = 0; j < LANE; ++j)
      if (j < count) to[j] = (int8_t)(c[j / 4] >> (8 * (j % 4)));
}
__device__ __forceinline__ void write_codes(int8_t *to, int count, const float (&v)[LANE], const Step &step) {
  int k[LANE];
#pragma unroll
  for (int j = 0; j < LANE; ++j) k[j] = step.bad ? 0 : (int)fminf(fmaxf(rintf(v[j] * step.per_step), -127.f), 127.f);
  write_bytes(to, count, k);
}
__device__ __forceinline__ void read_codes(const int8_t *from, int count, float step, float (&v)[LANE]) {
  if (count >= LANE) {
    const words2 r = *(const words2_any *)from;
#pragma unroll
    for (int j = 0; j < LANE; ++j) v[j] = (float)(int8_t)(r[j / 4] >> (8 * (j % 4))) * step;
  } else
#pragma unroll
    for (int j = 0; j < LANE; ++j) v[j] = j < count ? (float)from[j] * step : 0.f;
}

} // namespace
