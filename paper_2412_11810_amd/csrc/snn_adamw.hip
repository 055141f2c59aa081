// A step of AdamW over many tensors:
//
//   m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g^2
//   p = p (1 - lr decay) - lr m / (1 - beta1^t) / (sqrt(v / (1 - beta2^t)) + eps)
//
// in 32 bits, from the moments before they are rounded.  The factors that depend on t are found in 64 bits, on the host or, where the number of
// steps is on the device (a step in a graph), by a kernel of one thread.
//
// Moments in 8 bits are m and the root of v, in blocks of 32 elements with a power of two as their step (the format of snn_pack).  In them a
// change of less than half a step would never take place if codes were rounded to nearest (v changes by 1/1000 at a time), so an
// element is rounded up or down by a threshold u: code = floor(x / step + u).  u = frac(i c1 + t c2) for element i and step t, c1 and c2 the powers 1 and
// 2 of the reciprocal of the root of r^3 = r + 1, whose multiples fill the square evenly: over the steps, and over the elements of a
// block, roundings cancel.  The root of a v that is not 0 has a code of 1 at least, as a divisor of 0 would make a step of any size.
//
// One launch for 40 tensors: their descriptions go as its arguments, so that nothing needs to be kept or copied.  A workgroup takes 8192 elements of one, a
// lane 8 at a time.  What bounds it: memory.  363 million elements in bf16 with moments of 32 bits take 1942 us, 5.2 TB/s; 152 million with moments of 8 bits 494,
// 4.9 TB/s; 17 tensors of 0.2 million in all are bound by the call, 22 us, 8.4 of them in the kernel, whose 34 workgroups take up to four rounds one after the other.
#include "snn_rows.h"
#include <math.h>

namespace {

constexpr int TENSORS = 40, ROUNDS = 4, THREADS = 256, PER_GROUP = THREADS * LANE * ROUNDS;

struct Factors {
  float beta1, rest1, beta2, rest2, keep, lr, root, eps; // rest = 1 - beta; keep = 1 - lr decay; lr / (1 - beta1^t); 1 / sqrt(1 - beta2^t)
  uint32_t t;
};
struct Tensor {
  void *p;
  const void *g;
  void *m, *v;
  uint8_t *m_exps, *v_exps;
  __bf16 *copy;
  long long n;
  uint32_t base;  // the first element's number in its tensor, modulo 2^32
  uint32_t types; // 1: p is bf16, 2: g is
};
// (No array of bytes in here: beside one, this compiler has read `first` by a scalar load from an address that is no multiple of 4.)
struct Args {
  Tensor tensors[TENSORS];
  uint32_t first[TENSORS]; // the tensor's first workgroup
  int count;
  const float *scale;
  const Factors *on_device;
  Factors factors;
};
static_assert(sizeof(Args) <= 3584, "the arguments of a launch");

__host__ __device__ inline Factors factors_of(const AdamwStep &a, long long t) {
  Factors f;
  f.beta1 = (float)a.beta1, f.rest1 = (float)(1 - a.beta1), f.beta2 = (float)a.beta2, f.rest2 = (float)(1 - a.beta2);
  f.keep = (float)(1 - a.lr * a.decay), f.lr = (float)(a.lr / (1 - pow(a.beta1, (double)t))), f.root = (float)(1 / sqrt(1 - pow(a.beta2, (double)t)));
  f.eps = (float)a.eps;
  f.t = (uint32_t)t;
  return f;
}
__global__ void k_adamw_count(AdamwStep a, Factors *to) { *to = factors_of(a, ++*a.count); }

__device__ __forceinline__ float threshold(uint32_t i, uint32_t t, uint32_t c1, uint32_t c2) { return (float)((i * c1 + t * c2) >> 16) * 0x1p-16f; }

// A moment's 8 elements back into codes
__device__ __forceinline__ void to_codes(int8_t *codes, uint8_t *exps, long long i, uint32_t base, int count, const float (&x)[LANE], uint32_t t, uint32_t c1, uint32_t c2, int least) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < LANE; ++j) top = max(top, j < count ? __float_as_uint(x[j]) & 0x7fffffffu : 0u);
  const Step step = step_of(most_of_block(top), 0x7e0001u); // (127 steps are floor(127 + u))
  if (count <= 0) return;
  int k[LANE];
#pragma unroll
  for (int j = 0; j < LANE; ++j) {
    const int c = (int)floorf(x[j] * step.per_step + threshold(base + (uint32_t)i + j, t, c1, c2));
    k[j] = step.bad ? 0 : min(max(c, x[j] > 0.f ? least : -127), 127); // (beyond 127 * 2^121 there is no step)
  }
  write_bytes(codes + i, count, k);
  if (i % SNN_PACK_BLOCK == 0) exps[i / SNN_PACK_BLOCK] = step.byte;
}

__global__ __launch_bounds__(THREADS) void k_adamw(Args a) {
  int at = 0;
  for (int half = 32; half; half /= 2)
    if (at + half < a.count && blockIdx.x >= a.first[at + half]) at += half;
  const Tensor x = a.tensors[at];
  const bool p16 = x.types & 1, g16 = x.types & 2, eight = x.m_exps != nullptr;
  const Factors f = a.on_device ? *a.on_device : a.factors;
  const float scale = a.scale ? *a.scale : 1.f;
  long long i = (long long)(blockIdx.x - a.first[at]) * PER_GROUP + threadIdx.x * LANE;
#pragma unroll 1
  for (int round = 0; round < ROUNDS; ++round, i += THREADS * LANE) {
    if (i - (long long)threadIdx.x * LANE >= x.n) return; // (the whole workgroup)
    const int count = (int)min((long long)LANE, max(x.n - i, 0ll));
    float p[LANE], g[LANE], m[LANE], v[LANE];
    if (p16) read((const __bf16 *)x.p + i, count, p);
    else read((const float *)x.p + i, count, p);
    if (g16) read((const __bf16 *)x.g + i, count, g);
    else read((const float *)x.g + i, count, g);
    if (eight) {
      const float step_m = count > 0 ? __uint_as_float((uint32_t)x.m_exps[i / SNN_PACK_BLOCK] << 23) : 0.f;
      const float step_v = count > 0 ? __uint_as_float((uint32_t)x.v_exps[i / SNN_PACK_BLOCK] << 23) : 0.f;
      read_codes((const int8_t *)x.m + i, count, step_m, m);
      read_codes((const int8_t *)x.v + i, count, step_v, v);
#pragma unroll
      for (int j = 0; j < LANE; ++j) v[j] *= v[j];
    } else {
      read((const float *)x.m + i, count, m);
      read((const float *)x.v + i, count, v);
    }
    float root[LANE];
#pragma unroll
    for (int j = 0; j < LANE; ++j) {
      const float d = g[j] * scale;
      m[j] = fmaf(f.beta1, m[j], f.rest1 * d);
      v[j] = fmaf(f.beta2, v[j], f.rest2 * d * d);
      root[j] = sqrtf(v[j]);
      p[j] = fmaf(p[j], f.keep, -(f.lr * m[j] / fmaf(root[j], f.root, f.eps)));
    }
    if (p16) write((__bf16 *)x.p + i, count, p);
    else write((float *)x.p + i, count, p);
    if (x.copy) write(x.copy + i, count, p);
    if (eight) {
      to_codes((int8_t *)x.m, x.m_exps, i, x.base, count, m, f.t, 0xC13FA9A9u, 0x91E10DA5u, -127);
      to_codes((int8_t *)x.v, x.v_exps, i, x.base, count, root, f.t, 0x91E10DA5u, 0xC13FA9A9u, 1);
    } else {
      write((float *)x.m + i, count, m);
      write((float *)x.v + i, count, v);
    }
  }
}

} // namespace

size_t adamw_workspace() { return sizeof(Factors); }

hipError_t launch_adamw(const AdamwStep &how, const AdamwTensor *tensors, long long count, void *work, hipStream_t s) {
  Args a = {};
  a.scale = how.scale;
  if (how.count) {
    k_adamw_count<<<1, 1, 0, s>>>(how, (Factors *)work);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    a.on_device = (const Factors *)work;
  } else a.factors = factors_of(how, how.t);
  // up to 2^22 workgroups to a launch: a grid has fewer than 2^32 threads
  constexpr long long MOST = 1ll << 22;
  long long groups = 0;
  auto queue = [&]() {
    if (!a.count) return hipSuccess;
    k_adamw<<<(unsigned)groups, THREADS, 0, s>>>(a);
    a.count = 0;
    groups = 0;
    return hipGetLastError();
  };
  for (long long k = 0; k < count; ++k) {
    const AdamwTensor &x = tensors[k];
    for (long long done = 0; done < x.n;) { // (parts begin at whole blocks)
      if (a.count == TENSORS || groups == MOST)
        if (const hipError_t e = queue(); e != hipSuccess) return e;
      const long long part = x.n - done < (MOST - groups) * PER_GROUP ? x.n - done : (MOST - groups) * PER_GROUP;
      const int i = a.count++;
      a.tensors[i] = Tensor{(char *)x.p + done * (x.p16 ? 2 : 4), (const char *)x.g + done * (x.g16 ? 2 : 4),
                            (char *)x.m + done * (x.m_exps ? 1 : 4), (char *)x.v + done * (x.m_exps ? 1 : 4),
                            x.m_exps ? x.m_exps + done / SNN_PACK_BLOCK : nullptr, x.m_exps ? x.v_exps + done / SNN_PACK_BLOCK : nullptr,
                            x.copy ? (__bf16 *)x.copy + done : nullptr, part, (uint32_t)done, (x.p16 ? 1u : 0u) | (x.g16 ? 2u : 0u)};
      a.first[i] = (uint32_t)groups;
      groups += (part + PER_GROUP - 1) / PER_GROUP;
      done += part;
    }
  }
  return queue();
}
