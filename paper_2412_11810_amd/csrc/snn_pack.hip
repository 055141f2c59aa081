// Activations in 8 bits: blocks of 32 consecutive elements of a row share a step 2^k, and each element is the multiple of it
// (-127..127) that is nearest.  k is the smallest from -126 to 121 with which the largest element does not round past 127.  Powers of two
// make both directions exact but for the one rounding to a multiple (half a step at most: 2^-7 of the block's largest element),
// whatever type the values come from or go to.  The byte of a block is the exponent field of its step as a float: 0 decodes to zeros; a
// block with an infinity or NaN has 255 and zero codes, which decodes to 0 * infinity, NaN throughout.
//
// A lane takes 8 elements, the four lanes of a block share their largest element by two permutations inside the quad.  Both
// directions are bound by memory: 32768 x 4096 in bf16 takes 84 us there and 87 back, 4.8 TB/s (a copy reaches 5.1).  Rows of odd widths go the same
// way, with loads and stores at any address: 4329 x 1501 in fp32 takes 8 and 10 us.
#include "snn_ops.h"

namespace {

constexpr int LANE = 8; // elements of a lane
constexpr int THREADS = 256;

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

// The place of a thread: a row and the first of its 8 columns.  `across` threads (a power of two, whole blocks) lie side by side in a row.
// A grid has fewer than 2^32 threads along x: the workgroups of more rows than that go on along y.
constexpr unsigned GRID_X = 1u << 22;
struct Place {
  long long row;
  int col;
  __device__ __forceinline__ Place(int across, int col_groups) {
    const int down = THREADS / across;
    const unsigned block = blockIdx.y * GRID_X + blockIdx.x, group = block % (unsigned)col_groups;
    row = (long long)(block / (unsigned)col_groups) * down + threadIdx.x / across;
    col = (int)(group * across + threadIdx.x % across) * LANE;
  }
};

template <typename T> __global__ __launch_bounds__(THREADS) void k_pack(long long rows, int cols, long long ld, const T *x, int8_t *codes,
                                                                        uint8_t *exps, int across, int col_groups) {
  const Place at(across, col_groups);
  const int count = at.row < rows ? cols - at.col : 0; // elements that are left of the row here
  float v[LANE];
  read(x + at.row * ld + at.col, max(count, 0), v);
  uint32_t top = 0; // as bits: an infinity or NaN is above every number
#pragma unroll
  for (int j = 0; j < LANE; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
  top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xb1, 0xf, 0xf, false)); // quad lanes 1 0 3 2
  top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x4e, 0xf, 0xf, false)); // quad lanes 2 3 0 1
  if (count <= 0) return;
  // (127.5 steps would round to 128; 2^121 is the largest step whose multiples are all floats)
  const int e = min(max((int)(top >> 23) - 6 + ((top & 0x7fffffu) >= 0x7f0000u), 1), 248);
  const bool none = top == 0, bad = top >= 0x7f800000u;
  const float per_step = __uint_as_float((uint32_t)(254 - e) << 23);
  uint32_t c[2] = {};
#pragma unroll
  for (int j = 0; j < LANE; ++j) {
    const int k = bad ? 0 : (int)fminf(fmaxf(rintf(v[j] * per_step), -127.f), 127.f);
    c[j / 4] |= (uint32_t)(k & 0xff) << (8 * (j % 4));
  }
  int8_t *to = codes + at.row * cols + at.col;
  if (count >= LANE) {
    words2 r;
    r[0] = c[0];
    r[1] = c[1];
    *(words2_any *)to = r;
  } else
#pragma unroll
    for (int j = 0; j < LANE; ++j)
      if (j < count) to[j] = (int8_t)(c[j / 4] >> (8 * (j % 4)));
  if (at.col % SNN_PACK_BLOCK == 0)
    exps[at.row * ((cols + SNN_PACK_BLOCK - 1) / SNN_PACK_BLOCK) + at.col / SNN_PACK_BLOCK] = bad ? 255 : none ? 0 : (uint8_t)e;
}

template <typename T> __global__ __launch_bounds__(THREADS) void k_unpack(long long rows, int cols, long long ld, const int8_t *codes,
                                                                          const uint8_t *exps, T *x, int across, int col_groups) {
  const Place at(across, col_groups);
  const int count = at.row < rows ? cols - at.col : 0;
  if (count <= 0) return;
  const float step =
      __uint_as_float((uint32_t)exps[at.row * ((cols + SNN_PACK_BLOCK - 1) / SNN_PACK_BLOCK) + at.col / SNN_PACK_BLOCK] << 23);
  const int8_t *from = codes + at.row * cols + at.col;
  float v[LANE];
  if (count >= LANE) {
    const words2 r = *(const words2_any *)from;
#pragma unroll
    for (int j = 0; j < LANE; ++j) v[j] = (float)(int8_t)(r[j / 4] >> (8 * (j % 4))) * step;
  } else
#pragma unroll
    for (int j = 0; j < LANE; ++j) v[j] = j < count ? (float)from[j] * step : 0.f;
  write(x + at.row * ld + at.col, count, v);
}

struct Grid {
  int across, col_groups;
  dim3 blocks;
  Grid(long long rows, int cols) {
    const int lanes = (cols + SNN_PACK_BLOCK - 1) / SNN_PACK_BLOCK * (SNN_PACK_BLOCK / LANE);
    across = SNN_PACK_BLOCK / LANE;
    while (across < lanes && across < THREADS) across *= 2;
    col_groups = (lanes + across - 1) / across;
    const int down = THREADS / across;
    const unsigned all = (unsigned)((rows + down - 1) / down * col_groups); // (2^31 at most, of 2^40 elements)
    blocks = all < GRID_X ? dim3(all) : dim3(GRID_X, (all + GRID_X - 1) / GRID_X);
  }
};

} // namespace

hipError_t launch_pack(bool bf16, long long rows, int cols, long long ld, const void *x, int8_t *codes, uint8_t *exps, hipStream_t s) {
  const Grid g(rows, cols);
  if (bf16) k_pack<__bf16><<<g.blocks, THREADS, 0, s>>>(rows, cols, ld, (const __bf16 *)x, codes, exps, g.across, g.col_groups);
  else k_pack<float><<<g.blocks, THREADS, 0, s>>>(rows, cols, ld, (const float *)x, codes, exps, g.across, g.col_groups);
  return hipGetLastError();
}

hipError_t launch_unpack(bool bf16, long long rows, int cols, long long ld, const int8_t *codes, const uint8_t *exps, void *x,
                         hipStream_t s) {
  const Grid g(rows, cols);
  if (bf16) k_unpack<__bf16><<<g.blocks, THREADS, 0, s>>>(rows, cols, ld, codes, exps, (__bf16 *)x, g.across, g.col_groups);
  else k_unpack<float><<<g.blocks, THREADS, 0, s>>>(rows, cols, ld, codes, exps, (float *)x, g.across, g.col_groups);
  return hipGetLastError();
}
