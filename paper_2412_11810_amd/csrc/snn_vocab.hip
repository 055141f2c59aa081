// Softmax cross entropy of rows h [rows][d] against a vocabulary w [vocab][d], and its gradients, without a matrix of logits.
//
//   l_rv = h_r . w_v log2(e);  M_r = max_v ceil(l_rv);  S_r = sum_v 2^(l_rv - M_r);  miss_r = sum_{v != y} 2^(l_rv - M_r) / S_r = 1 - p_ry
//   loss_r = -log1p(-miss_r), or (log2 S_r - (l_ry - M_r)) log(2) where miss_r is not small
//   G_rv = dloss_r / c 2^(l_rv - M_r) / S_r;  G_ry = -dloss_r / c miss_r;  dh = c G w;  dw = c G^T h
//
// c is what the rows' dloss have in common (their largest magnitude, 1 / number of rows for a mean): rounded into G, a factor like 1 / 300
// would be off by up to 2^-8 for all rows alike.
// G itself is found in 32 bits and, where h and w are bf16, rounded to bf16 on its way into its two products: the matrix cores take both operands in
// one type, and two parts of G would cost 7 ms beside the 15 of 8192 x 2048 x 128000.  Each element is off by 2^-8 of itself at most, each in its
// own way; that adds 0 to 14 % to what dh and dw are off by for their own rounding (1.66e-3 of their norm; 33 x 512 x 1000 to 2000 x 512 x 5000,
// logits spread over +-1 to +-12).  Sums of few terms would show more of it (one row of 512 with 1000 entries: 57 %): up to 32 rows, which leave half
// of a tile empty, what the rounding leaves goes through the products as further rows.
//
// miss_r is summed without the target, never formed as 1 - p: a target that the model is sure of keeps its loss and gradient.
// The subtrahends are whole numbers: l - M is one fused multiply-add, rounded once to its own size, and sums over different M are brought
// together exactly.
//
// All four products are one kernel, C = A B^T with the sums along the rows of both operands, on the bf16 matrix cores with fp32
// accumulators; what differs is what happens to the accumulators.  Operands of 32 bits go in as three bf16 parts of 8 bits
// each, which hold all 24 bits of a float; of the nine products of parts the six whose weight is above 2^-24 are made, the one of the
// first parts in accumulators of its own.
// The logits are computed twice, for the loss (kept: an exponent and a sum for 32 to 128 of them) and for G, one piece of the vocabulary
// after the other, whose G is all that is ever in memory.
//
// What bounds it: the matrix cores, at the clock that they leave.  8192 x 2048 x 128000 in bf16 takes 15.2 ms, four products of 4.3 TFLOP at
// 1.13 PFLOP/s (a library product with sums of 2048: 1.18 to 1.20); the loss of 4096 x 2048 x 50021 720 us, 1.16 PFLOP/s, matrix instructions in 69 % of
// the cycles at 1.9 GHz.  (Machines differ: on another one 15.8 ms and 747 us.)  Few rows are bound by w: 12 x 768 x 99960 in fp32, 307 MB, takes 93 us.
#include "snn_ops.h"

namespace {

typedef __bf16 frag __attribute__((ext_vector_type(8)));
typedef float tile32 __attribute__((ext_vector_type(16)));

constexpr float LOG2E = 1.44269504f;

// Rows of operands lie in blocks of 32 elements, a block's parts one after the other; the products take KS elements of a row at a time, STEP
// bytes.
template <int PARTS> constexpr int KS = PARTS == 1 ? 64 : 32;
template <int PARTS> constexpr int STEP = KS<PARTS> * PARTS * 2;
template <int PARTS> __device__ __forceinline__ size_t place_of(size_t row, int c, int part, int padded) {
  return (row * padded + (c & ~31)) * PARTS + part * 32 + (c & 31);
}
// Tiles: 256 rows of A by 256 of B, or, in parts, by 128; 64 by 256 where a side has no more than 64 rows (products that make logits: that of B
// only); 128 by 128 where 256 compute units are through with those sooner.  By the rounds that the units take, an element of a small tile takes
// 1.2 to 1.45 times as long in bf16 (loss of 8192 x 1024 x 16384, 8 rounds of large tiles and 32 quarter ones: 284 and 355 us; of 1500 x 768 x
// 12000, 2 rounds and 5 quarters: 58 and 53 us), in parts 1.01 to 1.12 times (2000 x 1024 x 20011: 435 and 446 us; 1500 x 768 x 12000: 193 and
// 174 us).  The rule takes the upper end: at the lower one 2000 x 1024 x 20011 in bf16 would get small tiles, 117 us instead of 106.  Few
// large tiles leave units without work (2048 x 1024 x 4096 in bf16: 39 and 31 us, with gradients 132 and 98; 300 x 512 x 1000: 27 and 17, 66 and 34).
enum Tile { BIG, SMALL, FEW_A, FEW_B };
int rows_of_a(Tile t) { return t == FEW_A ? 64 : t == SMALL ? 128 : 256; }
int rows_of_b(Tile t, int parts) { return t == FEW_B ? 64 : t == FEW_A ? 256 : t == SMALL || parts > 1 ? 128 : 256; }
long long tiles(Tile t, int rows_a, int rows_b, int parts) {
  const int a = rows_of_a(t), b = rows_of_b(t, parts);
  return (long long)((rows_a + a - 1) / a) * ((rows_b + b - 1) / b);
}
Tile tile_for(int rows_a, int rows_b, int parts, bool logits) {
  if (rows_a <= 64 && !logits) return FEW_A;
  if (rows_b <= 64) return FEW_B;
  auto time = [&](Tile t, float each) { return (float)((tiles(t, rows_a, rows_b, parts) + 255) / 256) * rows_of_a(t) * rows_of_b(t, parts) * each; };
  return time(SMALL, parts == 1 ? 1.45f : 1.12f) < time(BIG, 1.f) ? SMALL : BIG;
}

// ---- C = A B^T ----------------------------------------------------------------------------
// Operands: rows of ksteps * STEP bytes.  Rows past the last one are the last one again (not used by the epilogues).  The bytes from a
// tile's first row to the end of its last one fit 32 bits (vocab_shape() and Slices see to it).
struct Product {
  const __bf16 *a, *b;
  long long lda, ldb; // elements from row to row, of all parts
  int rows_a, rows_b, ksteps;
  int tiles_a, tiles_b, slices, slice_steps; // slices along the sums: blockIdx.y, slice_steps each
};

__device__ __forceinline__ void load_lds(const char *base, unsigned off, char *lds) {
  // one wavefront: 64 * 16 bytes, lane after lane, to lds
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, (int)0xffffffff, 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)lds, 16, (int)off, 0, 0, 0);
}

// What an epilogue has of LDS for its wavefront, to turn accumulators into rows that leave in whole lines.  A wavefront's accesses to LDS are
// in order, so that turn() only has to keep the compiler from changing that.
struct Stage {
  char *first, *second; // 4 KB each
  int lane, r, half;
  static __device__ __forceinline__ void turn() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
  }
};

// One tile of BM rows of A by BN rows of B by eight wavefronts, WA along A and WB along B.  LDS holds two steps of 64 elements (128 bytes of
// a row), or of 32 in three parts (192 bytes); its 16-byte chunks are exchanged in a way that depends on the row, so that 16
// lanes of a fragment, which read one chunk of as many rows, use all 64 banks.  Loads go past the registers, a step ahead.  The fragments of
// the next 16 elements are on their way while those of these are multiplied, also across the barrier between two steps: matrix instructions
// wait for nothing but loads that take longer than a step.  (Smaller tiles, of which there are few and which are soon multiplied, hold
// four steps where LDS has room for them: their loads are three ahead.)
// WHOLE: the rows of A are floats as the caller has them (a multiple of 32 each, 128 bytes per step), whose parts are made in registers.
template <int BM, int BN, int WA, int WB, int PARTS, bool WHOLE, class Epilogue>
__global__ __launch_bounds__(512) void k_product(Product p, Epilogue ep) {
  constexpr int ROW = STEP<PARTS>, CHUNKS = ROW / 16, TIMES = KS<PARTS> / 16, ROW_A = WHOLE ? 128 : ROW, CHUNKS_A = ROW_A / 16;
  constexpr int MI = BM / WA / 32, NI = BN / WB / 32, LA = (BM * CHUNKS_A + 511) / 512, LB = (BN * CHUNKS + 511) / 512;
  constexpr int HELD = PARTS == 1 && BM * BN < 256 * 256 ? 4 : 2;
  __shared__ __align__(16) char a0[BM * ROW_A], b0[BN * ROW], a1[BM * ROW_A], b1[BN * ROW];
  __shared__ __align__(16) char a2[HELD > 2 ? BM * ROW_A : 16], b2[HELD > 2 ? BN * ROW : 16], a3[HELD > 2 ? BM * ROW_A : 16], b3[HELD > 2 ? BN * ROW : 16];
  // where chunk c of a row is, and which one is at place c
  auto exchanged = [](int row, int c) { return PARTS == 1 ? c ^ ((row >> 1) & 7) : c ^ ((row >> 2) & 3); };
  auto exchanged_a = [&](int row, int c) { return WHOLE ? c ^ ((row >> 1) & 7) : exchanged(row, c); };
  // tiles in the order of the dies: consecutive workgroups are on different ones, each die takes a run of tiles, in groups of eight
  // along A that share the rows of B
  const unsigned n = p.tiles_a * p.tiles_b, per = n / 8, rest = n % 8;
  const unsigned die = blockIdx.x % 8, at = blockIdx.x / 8;
  const unsigned id = n < 8 ? blockIdx.x : die * per + min(die, rest) + at;
  const unsigned group = id / (8 * p.tiles_b), first = group * 8, wide = min(8u, p.tiles_a - first), in = id - group * 8 * p.tiles_b;
  const int ta = first + in % wide, tb = in / wide;

  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wa = w / WB, wb = w % WB;
  const char *base_a = (const char *)(p.a + (long long)ta * BM * p.lda), *base_b = (const char *)(p.b + (long long)tb * BN * p.ldb);
  // load i of a wavefront: 64 chunks of the tile from number (8 i + w) * 64 on, from the beginning again where it has no more
  unsigned off_a[LA], off_b[LB];
#pragma unroll
  for (int i = 0; i < LA; ++i) {
    const int q = ((8 * i + w) * 64) % (BM * CHUNKS_A) + lane, row = q / CHUNKS_A;
    off_a[i] = (unsigned)min(row, p.rows_a - 1 - ta * BM) * (unsigned)(p.lda * 2) + exchanged_a(row, q % CHUNKS_A) * 16;
  }
#pragma unroll
  for (int i = 0; i < LB; ++i) {
    const int q = ((8 * i + w) * 64) % (BN * CHUNKS) + lane, row = q / CHUNKS;
    off_b[i] = (unsigned)min(row, p.rows_b - 1 - tb * BN) * (unsigned)(p.ldb * 2) + exchanged(row, q % CHUNKS) * 16;
  }

  const int slice = blockIdx.y, k_first = slice * p.slice_steps, k_end = min(k_first + p.slice_steps, p.ksteps);
  base_a += (long long)k_first * ROW_A;
  base_b += (long long)k_first * ROW;
  auto fetch = [&](char *la, char *lb) {
#pragma unroll
    for (int i = 0; i < LA; ++i) load_lds(base_a, off_a[i], la + ((8 * i + w) * 64) % (BM * CHUNKS_A) * 16);
#pragma unroll
    for (int i = 0; i < LB; ++i) load_lds(base_b, off_b[i], lb + ((8 * i + w) * 64) % (BN * CHUNKS) * 16);
    base_a += ROW_A;
    base_b += ROW;
  };
  tile32 acc[MI][NI] = {}, low[PARTS == 1 ? 1 : MI][PARTS == 1 ? 1 : NI] = {};
  frag fa[2][WHOLE ? 1 : PARTS][MI], fb[2][PARTS][NI];
  float4 whole[WHOLE ? 2 : 1][MI][2]; // 8 elements of A, not yet in parts
  const int r = lane & 31, half = lane >> 5;
  auto read = [&](int s, const char *la, const char *lb) {
#pragma unroll
    for (int k = 0; k < PARTS; ++k) {
      const int place = exchanged(r, 4 * k + 2 * s + half) * 16; // (tiles of 32 rows begin at multiples of 32)
      if constexpr (!WHOLE)
#pragma unroll
        for (int i = 0; i < MI; ++i) fa[s & 1][k][i] = *(const frag *)(la + (wa * (BM / WA) + i * 32 + r) * ROW + place);
#pragma unroll
      for (int i = 0; i < NI; ++i) fb[s & 1][k][i] = *(const frag *)(lb + (wb * (BN / WB) + i * 32 + r) * ROW + place);
    }
    if constexpr (WHOLE)
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c)
          whole[s & 1][i][c] = *(const float4 *)(la + (wa * (BM / WA) + i * 32 + r) * 128 + exchanged_a(r, 4 * s + 2 * half + c) * 16);
    __builtin_amdgcn_sched_barrier(0); // (left alone the compiler reads right before it multiplies, into the same registers)
  };
  auto multiply = [&](int s) {
    frag a[PARTS][MI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
      if constexpr (WHOLE) {
        float x[8] = {whole[s & 1][i][0].x, whole[s & 1][i][0].y, whole[s & 1][i][0].z, whole[s & 1][i][0].w,
                      whole[s & 1][i][1].x, whole[s & 1][i][1].y, whole[s & 1][i][1].z, whole[s & 1][i][1].w};
#pragma unroll
        for (int k = 0; k < PARTS; ++k) {
          uint32_t two[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) two[e] = __builtin_amdgcn_perm(__float_as_uint(x[2 * e + 1]), __float_as_uint(x[2 * e]), 0x07060302u); // upper halves
          a[k][i] = __builtin_bit_cast(frag, *(const uint4 *)two);
          if (k < PARTS - 1)
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] -= __uint_as_float(__float_as_uint(x[e]) & 0xffff0000u);
        }
      } else
#pragma unroll
        for (int k = 0; k < PARTS; ++k) a[k][i] = fa[s & 1][k][i];
#pragma unroll
    for (int k = PARTS - 1; k > 0; --k) // parts of A and of B whose numbers add up to k
#pragma unroll
      for (int n = 0; n <= k; ++n)
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int j = 0; j < NI; ++j) low[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[n][i], fb[s & 1][k - n][j], low[i][j], 0, 0, 0);
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0][i], fb[s & 1][0][j], acc[i][j], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  // the next step is in LDS for every wavefront, and every wavefront has what it read before; `later`: the steps behind it may be under way
  auto arrived = [&](bool later) {
    constexpr int LATER = (HELD - 2) * (LA + LB);
    static_assert(LATER < 16, "the count of loads under way");
    if (later) __builtin_amdgcn_s_waitcnt(0x0070 | LATER);
    else __builtin_amdgcn_s_waitcnt(0x0070);
    asm volatile("" ::: "memory"); // (the compiler knows of no store to LDS here)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  int left = k_end - k_first;
  auto step = [&](char *la, char *lb, const char *na, const char *nb, bool more) {
#pragma unroll
    for (int s = 0; s < TIMES - 1; ++s) {
      read(s + 1, la, lb);
      multiply(s);
    }
    if (more || left > 1) {
      arrived(more || left >= HELD);
      if (more || left > HELD) fetch(la, lb);
      read(0, na, nb);
    }
    multiply(TIMES - 1);
    --left;
  };
  fetch(a0, b0);
  if (left > 1) fetch(a1, b1);
  if constexpr (HELD > 2) {
    if (left > 2) fetch(a2, b2);
    if (left > 3) fetch(a3, b3);
  }
  arrived(false);
  read(0, a0, b0);
  if constexpr (HELD > 2) {
    while (left > 7) {
      step(a0, b0, a1, b1, true);
      step(a1, b1, a2, b2, true);
      step(a2, b2, a3, b3, true);
      step(a3, b3, a0, b0, true);
    }
    for (;;) {
      step(a0, b0, a1, b1, false);
      if (!left) break;
      step(a1, b1, a2, b2, false);
      if (!left) break;
      step(a2, b2, a3, b3, false);
      if (!left) break;
      step(a3, b3, a0, b0, false);
      if (!left) break;
    }
  } else {
    while (left > 3) {
      step(a0, b0, a1, b1, true);
      step(a1, b1, a0, b0, true);
    }
    step(a0, b0, a1, b1, false);
    if (left) step(a1, b1, a0, b0, false);
    if (left) step(a0, b0, a1, b1, false);
  }
  __syncthreads();
  if constexpr (PARTS > 1)
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NI; ++j) acc[i][j] += low[i][j];
  // element e of a tile: row 8 (e / 4) + 4 half + e % 4 of A, row r of B.  Every wavefront is through with the tiles in LDS
  constexpr bool HALVES = BM * ROW_A < 8 * 4096 && BN * ROW < 8 * 4096; // four wavefronts in each array
  char *const first0 = HALVES ? (w < 4 ? a0 : b0) + w % 4 * 4096 : (BM * ROW_A >= 8 * 4096 ? a0 : b0) + w * 4096;
  char *const second0 = HALVES ? (w < 4 ? a1 : b1) + w % 4 * 4096 : (BM * ROW_A >= 8 * 4096 ? a1 : b1) + w * 4096;
  const Stage stage = {first0, second0, lane, r, half};
  ep.template finish<MI, NI>(acc, ta * BM + wa * (BM / WA), tb * BN + wb * (BN / WB), slice, stage);
}

__device__ __forceinline__ bool has_target(const int *targets, int m, bool on, int vocab) { return on && targets[m] >= 0 && targets[m] < vocab; }
// Row m's target, counted from entry v0 on; -1: none, or one before v0
__device__ __forceinline__ int entry(const int *targets, int m, bool on, int vocab, int v0) {
  const int y = on ? targets[m] : -1;
  return y >= v0 && y < vocab ? y - v0 : -1;
}

// Logits, A = vocabulary (a piece of it from `first` on), B = rows of h.  A lane has the logits of one row with 16 MI entries of the
// vocabulary: the exponent M of the largest and the sum of the powers above it, the target left out, and the target's logit go to memory.
struct LossEpilogue {
  static constexpr bool LOGITS = true, FEW_ROWS = false;
  const int *targets;
  float2 *part;  // [blocks of 32 MI entries][rows]
  float *picked; // [rows]: the target's logit
  int first, vocab, rows;
  template <int MI, int NI> __device__ __forceinline__ void finish(tile32 (&acc)[MI][NI], int v0, int m0, int, const Stage &st) const {
    const int r = st.r, half = st.half, block = (first + v0) / (32 * MI);
    v0 += first + 4 * half;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int m = m0 + j * 32 + r;
      const bool on = m < rows;
      const int y = entry(targets, m, on, vocab, v0); // the target's entry, counted as below
      if (__any(((unsigned)y < 32u * MI && !(y & 4)) || v0 + 32 * MI > vocab)) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int v = 32 * i + 8 * (e >> 2) + (e & 3);
            if (v == y) picked[m] = acc[i][j][e];
            if (v == y || v0 + v >= vocab) acc[i][j][e] = -INFINITY;
          }
      }
      float most[2] = {-INFINITY, -INFINITY}, sum[2] = {};
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int e = 0; e < 16; e += 2) most[e >> 1 & 1] = fmaxf(fmaxf(most[e >> 1 & 1], acc[i][j][e]), acc[i][j][e + 1]);
      float top = fmaxf(most[0], most[1]);
      top = ceilf(fmaxf(top, __shfl_xor(top, 32)) * LOG2E);
      const float from = top == -INFINITY ? 0.f : top; // nothing here: all terms are 0
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) sum[e & 1] += __builtin_amdgcn_exp2f(fmaf(acc[i][j][e], LOG2E, -from));
      sum[0] += sum[1];
      sum[0] += __shfl_xor(sum[0], 32);
      if (half == 0 && on) part[(size_t)block * rows + m] = make_float2(top, sum[0]);
    }
  }
};

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  typedef float two __attribute__((ext_vector_type(2)));
  typedef __bf16 two_bf16 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(two{a, b}, two_bf16));
}

// The same logits again, turned into G: as rows of h by entries of the vocabulary (gm) and the other way round (gt), in parts.  TWICE (bf16, FEW
// rows or fewer): rounded, and what the rounding left as G of as many rows more, from `rows` on in gm, from FEW on in gt, which have room for
// them (in tiles of 64 rows, in sums of 64 terms).
constexpr int FEW = 32;
template <int PARTS, bool TWICE> struct GradEpilogue {
  static constexpr bool LOGITS = true, FEW_ROWS = TWICE; // (of h: no other tile than FEW_B)
  const int *targets;
  const float *state, *dloss, *common; // dloss [rows] is taken as multiples of common[0]; NULL: 1 for each row with a target
  __bf16 *gm, *gt;                    // [rows padded][width], [width][rows padded], in parts
  int first, vocab, rows, width, padded;
  template <int MI, int NI> __device__ __forceinline__ void finish(tile32 (&acc)[MI][NI], int v0, int m0, int, const Stage &st) const {
    static_assert(NI == 2, "a wavefront has 64 rows of h");
    const int r = st.r, half = st.half, lane = st.lane;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int m = m0 + j * 32 + r;
      const bool on = m < rows;
      const int y = entry(targets, m, on, vocab, first + v0 + 4 * half), left = vocab - first - v0 - 4 * half;
      const float given = !has_target(targets, m, on, vocab) ? 0.f : dloss ? dloss[m] : 1.f;
      const bool none = given == 0.f; // no part in the gradients, whatever its logits
      const float g = dloss ? given / *common : given, top = on ? state[3 * m] : 0.f, per = on ? state[3 * m + 1] * g : 0.f;
      const float miss = on ? state[3 * m + 2] : 0.f;
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float x = __builtin_amdgcn_exp2f(fmaf(acc[i][j][e], LOG2E, -top)) * per;
          acc[i][j][e] = none ? 0.f : x;
        }
      if (__any(((unsigned)y < 32u * MI && !(y & 4)) || left < 32 * MI)) { // targets here, or the vocabulary's end
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int v = 32 * i + 8 * (e >> 2) + (e & 3);
            if (v == y) acc[i][j][e] = none ? 0.f : -miss * g;
            if (v >= left) acc[i][j][e] = 0.f;
          }
      }
    }
    // 32 entries by 64 rows at a time.  first: [64 rows][32 entries], second: [32 entries][64 rows] (16-byte chunks at places that are
    // exchanged by the row, so that a wavefront's writes use all banks).  Two neighbouring lanes exchange one of two entries each, so that a
    // lane writes an entry for two rows at once: an even one entries 0 and 2 of four, an odd one entries 1 and 3.
    const uint32_t pair = lane & 1 ? 0x03020706u : 0x05040100u;
    const int odd = lane & 1;
#pragma unroll
    for (int k = 0; k < (TWICE ? 2 : PARTS); ++k)
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        Stage::turn();
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            uint2 four;
            if constexpr (PARTS == 1) {
              four.x = bf16_pair(acc[i][j][4 * q], acc[i][j][4 * q + 1]);
              four.y = bf16_pair(acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
              if (TWICE && k == 0)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const uint32_t pair_of = e < 2 ? four.x : four.y;
                  acc[i][j][4 * q + e] -= __uint_as_float(e & 1 ? pair_of & 0xffff0000u : pair_of << 16);
                }
            } else {
              uint32_t b[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                b[e] = __float_as_uint(acc[i][j][4 * q + e]) & 0xffff0000u;
                acc[i][j][4 * q + e] -= __uint_as_float(b[e]);
              }
              four.x = b[0] >> 16 | b[1];
              four.y = b[2] >> 16 | b[3];
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t mine = e ? four.y : four.x, other = (uint32_t)__builtin_amdgcn_mov_dpp((int)mine, 0xb1, 0xf, 0xf, false);
              const int v = 8 * q + 4 * half + 2 * e + odd;
              *(uint32_t *)(st.second + v * 128 + (((j * 4 + (r >> 3)) ^ (v & 7)) * 16) + (r & 6) * 2) = __builtin_amdgcn_perm(other, mine, pair);
            }
            *(uint2 *)(st.first + (j * 32 + r) * 64 + ((q ^ ((r >> 1) & 3)) * 16) + half * 8) = four;
          }
        Stage::turn();
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const int m = n * 16 + (lane >> 2), v = n * 8 + (lane >> 3);
          const uint4 of_m = *(const uint4 *)(st.first + m * 64 + (((lane & 3) ^ ((m >> 1) & 3)) * 16));
          const uint4 of_v = *(const uint4 *)(st.second + v * 128 + (((lane & 7) ^ (v & 7)) * 16));
          if constexpr (TWICE) {
            if (m < rows) *(uint4 *)(gm + place_of<1>(k * rows + m, v0 + 32 * i + (lane & 3) * 8, 0, width)) = of_m;
            if ((lane & 7) * 8 < FEW) *(uint4 *)(gt + place_of<1>(v0 + 32 * i + v, k * FEW + (lane & 7) * 8, 0, padded)) = of_v;
          } else {
            *(uint4 *)(gm + place_of<PARTS>(m0 + m, v0 + 32 * i + (lane & 3) * 8, k, width)) = of_m;
            *(uint4 *)(gt + place_of<PARTS>(v0 + 32 * i + v, m0 + (lane & 7) * 8, k, padded)) = of_v;
          }
        }
      }
  }
};

// C as T, times *factor, [rows_a][rows_b] with ld elements per row; or (factor NULL) in 32 bits, a slice each, added to what is there (add: it
// is not the first).  Rows may begin at any element.
typedef uint32_t words4 __attribute__((ext_vector_type(4)));
typedef words4 words4_any __attribute__((aligned(4)));
typedef uint32_t words2 __attribute__((ext_vector_type(2)));
typedef words2 words2_any __attribute__((aligned(2)));
template <typename T> struct StoreEpilogue {
  static constexpr bool LOGITS = false, FEW_ROWS = false;
  T *out;
  const float *factor;
  long long ld, per_slice;
  int rows_a, rows_b;
  bool add;
  template <int MI, int NI> __device__ __forceinline__ void finish(tile32 (&acc)[MI][NI], int ra, int rb, int slice, const Stage &st) const {
    constexpr int COLS = 32 * NI, LANES = COLS / 4, ROWS = 64 / LANES; // four columns per lane, ROWS rows at once
    T *const to = out + slice * per_slice;
    const float by = factor ? *factor : 1.f;
    const int c = rb + st.lane % LANES * 4;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int part = 0; part < 2; ++part) { // 16 rows
        Stage::turn();
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            *(float *)(st.first + ((8 * (e >> 2) + 4 * st.half + (e & 3)) * COLS + j * 32 + st.r) * 4) = acc[i][j][8 * part + e];
        Stage::turn();
#pragma unroll
        for (int n = 0; n < 16 / ROWS; ++n) {
          const int row = n * ROWS + st.lane / LANES, a = ra + 32 * i + 16 * part + row;
          float4 v = *(const float4 *)(st.first + row * COLS * 4 + st.lane % LANES * 16);
          if (a >= rows_a) continue;
          v.x *= by;
          v.y *= by;
          v.z *= by;
          v.w *= by;
          T *const at = to + a * ld + c;
          if (c + 4 <= rows_b) {
            if constexpr (sizeof(T) == 4) {
              if (add) {
                const words4 was = *(const words4_any *)at;
                v.x += __uint_as_float(was[0]);
                v.y += __uint_as_float(was[1]);
                v.z += __uint_as_float(was[2]);
                v.w += __uint_as_float(was[3]);
              }
              *(words4_any *)at = words4{__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w)};
            } else
              *(words2_any *)at = words2{bf16_pair(v.x, v.y), bf16_pair(v.z, v.w)};
          } else {
            const float u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int x = 0; x < 4; ++x)
              if (c + x < rows_b) {
                if (sizeof(T) == 4 && add) at[x] = (T)((float)at[x] + u[x]);
                else at[x] = (T)u[x];
              }
          }
        }
      }
  }
};

template <int PARTS, bool WHOLE, class Epilogue> hipError_t product(Tile t, Product p, const Epilogue &ep, hipStream_t s) {
  constexpr int BN = PARTS == 1 ? 256 : 128, WA = PARTS == 1 ? 2 : 4, WB = 8 / WA; // 64 rows of B to a wavefront
  const int a = rows_of_a(t), b = rows_of_b(t, PARTS);
  p.tiles_a = (p.rows_a + a - 1) / a;
  p.tiles_b = (p.rows_b + b - 1) / b;
  if (!p.slices) {
    p.slices = 1;
    p.slice_steps = p.ksteps;
  }
  const dim3 grid(p.tiles_a * p.tiles_b, p.slices);
  if (Epilogue::FEW_ROWS || t == FEW_B) k_product<256, 64, 8, 1, PARTS, WHOLE, Epilogue><<<grid, 512, 0, s>>>(p, ep);
  else if constexpr (Epilogue::FEW_ROWS) return hipErrorInvalidValue;
  else if (t == SMALL) k_product<128, 128, 4, 2, PARTS, WHOLE, Epilogue><<<grid, 512, 0, s>>>(p, ep);
  else if (t == BIG) k_product<256, BN, WA, WB, PARTS, WHOLE, Epilogue><<<grid, 512, 0, s>>>(p, ep);
  else if constexpr (!Epilogue::LOGITS) k_product<64, 256, 1, 8, PARTS, WHOLE, Epilogue><<<grid, 512, 0, s>>>(p, ep);
  return hipGetLastError();
}

// A product with fewer tiles than half the compute units is cut along its sums, eight steps (in parts: four) or more each; the slices are
// added up afterwards, in order.  A tile's rows are reached by 32-bit offsets from its first one: where 256 of them would lie further apart
// (dw in fp32, from 2.8 million rows of h on) a tile has 128, which do not at 2^22 rows of three parts either.
struct Slices {
  Tile tile;
  int count, steps;
  Slices(int rows_a, int rows_b, int ksteps, int parts, int at_most = 256) {
    const unsigned long long row = (unsigned long long)ksteps * (parts == 1 ? STEP<1> : STEP<3>); // bytes (of dw's operands: of all rows of h)
    tile = 256 * row <= UINT32_MAX ? tile_for(rows_a, rows_b, parts, false) : SMALL;
    const int most = (int)(256 / tiles(tile, rows_a, rows_b, parts)), fit = ksteps / (parts == 1 ? 8 : 4), n = most < fit ? most : fit;
    count = n < 1 ? 1 : n < at_most ? n : at_most;
    steps = (ksteps + count - 1) / count;
    count = (ksteps + steps - 1) / steps;
  }
};

// ---- operands -------------------------------------------------------------------------------
// x in parts of 8 bits each, cut off and not rounded: what is left is exact, and the third part has the last bits of 24
template <int PARTS> __device__ __forceinline__ void split(float x, uint16_t (&part)[PARTS]) {
#pragma unroll
  for (int k = 0; k < PARTS; ++k) {
    const uint32_t bits = __float_as_uint(x) & 0xffff0000u;
    part[k] = (uint16_t)(bits >> 16);
    x -= __uint_as_float(bits);
  }
}
// One matrix on its way into products: its rows [rows][padded cols] in parts, zeros behind their ends, and its columns [cols][padded
// rows] in parts, zeros behind the last row (either may be NULL).  With targets, rows that have none or whose dloss is 0 are
// zeros in the columns: what they hold (padding: anything) would else meet the zeros of G as 0 * NaN.
struct Operand {
  const void *from;
  long long ld;
  int rows, cols, padded_cols, padded_rows;
  __bf16 *to_rows, *to_cols;
  const int *targets;
  const float *dloss;
  int vocab, tiles_c;
  unsigned tiles;
  int again; // from here on the columns have the rows from the first one on again; 0: nowhere
};
// 64 by 64 elements per workgroup, four in a row per thread, through LDS for the columns.  The last workgroup finds what the rows' dloss have in
// common, where that is asked for: their largest finite magnitude, or, without any, 1 / number of rows with a target.
template <typename T, int PARTS> __global__ __launch_bounds__(256) void k_operands(Operand x, Operand y, const int *targets, const float *dloss, int rows, int vocab, float *common) {
  __shared__ float tile[64][65];
  unsigned id = blockIdx.x;
  if (id >= x.tiles + y.tiles) {
    float all = 0.f; // (numbers of rows are exact)
    for (int m = threadIdx.x; m < rows; m += 256)
      if (has_target(targets, m, true, vocab)) {
        const float g = dloss ? fabsf(dloss[m]) : 1.f;
        all = !dloss ? all + g : g < INFINITY ? fmaxf(all, g) : all;
      }
#pragma unroll
    for (int k = 32; k; k >>= 1) {
      const float o = __shfl_xor(all, k);
      all = dloss ? fmaxf(all, o) : all + o;
    }
    if ((threadIdx.x & 63) == 0) tile[0][threadIdx.x >> 6] = all;
    __syncthreads();
    if (threadIdx.x == 0) {
      const float count = tile[0][0] + tile[0][1] + tile[0][2] + tile[0][3];
      *common = dloss ? fmaxf(fmaxf(tile[0][0], tile[0][1]), fmaxf(tile[0][2], tile[0][3])) : count > 0.f ? 1.f / count : 0.f;
    }
    return;
  }
  const bool second = id >= x.tiles;
  if (second) id -= x.tiles;
  const Operand &m = second ? y : x;
  const int c0 = (int)(id % (unsigned)m.tiles_c) * 64, r0 = (int)(id / (unsigned)m.tiles_c) * 64, four = (threadIdx.x & 15) * 4, line = threadIdx.x >> 4;
  const T *const from = (const T *)m.from;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = r0 + i * 16 + line, c = c0 + four;
    float v[4] = {};
    const int of = m.again && r >= m.again ? r - m.again : r;
    if (of < m.rows) {
      const T *const at = from + of * m.ld + c;
      if (c + 4 <= m.cols) {
        if constexpr (sizeof(T) == 4) {
          const words4 q = *(const words4_any *)at;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(q[e]);
        } else {
          const words2 q = *(const words2_any *)at;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(e & 1 ? q[e >> 1] & 0xffff0000u : q[e >> 1] << 16);
        }
      } else
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (c + e < m.cols) v[e] = (float)at[e];
    }
    if (m.to_rows && r < m.rows && c < m.padded_cols) {
      uint16_t part[4][PARTS];
#pragma unroll
      for (int e = 0; e < 4; ++e) split(v[e], part[e]);
#pragma unroll
      for (int k = 0; k < PARTS; ++k)
        *(uint2 *)(m.to_rows + place_of<PARTS>(r, c, k, m.padded_cols)) = make_uint2(part[0][k] | (uint32_t)part[1][k] << 16, part[2][k] | (uint32_t)part[3][k] << 16);
    }
    const bool none = m.targets && of < m.rows && (!has_target(m.targets, of, true, m.vocab) || (m.dloss && m.dloss[of] == 0.f));
#pragma unroll
    for (int e = 0; e < 4; ++e) tile[i * 16 + line][four + e] = none ? 0.f : v[e];
  }
  if (!m.to_cols) return;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = c0 + i * 16 + line, r = r0 + four;
    if (c >= m.cols || r >= m.padded_rows) continue;
    uint16_t part[4][PARTS];
#pragma unroll
    for (int e = 0; e < 4; ++e) split(tile[four + e][i * 16 + line], part[e]);
#pragma unroll
    for (int k = 0; k < PARTS; ++k)
      *(uint2 *)(m.to_cols + place_of<PARTS>(c, r, k, m.padded_rows)) = make_uint2(part[0][k] | (uint32_t)part[1][k] << 16, part[2][k] | (uint32_t)part[3][k] << 16);
  }
}

// The blocks' exponents and sums joined, 16 rows per workgroup (whole lines of `part`), 64 threads each, in an order that depends on
// nothing but the number of blocks.  A block without a logit has no terms: its sum is 0, or NaN where a logit was.
struct Terms {
  float top, sum;
  __device__ __forceinline__ float at(float t) const { return top == t ? sum : sum * exp2f(top - t); }
  __device__ __forceinline__ void join(Terms o) {
    const float t = fmaxf(top, o.top);
    sum = at(t) + o.at(t);
    top = t;
  }
};
__global__ __launch_bounds__(1024) void k_join(const float2 *part, const float *picked, const int *targets, int blocks, int rows, int vocab,
                                               float *loss, float *state) {
  __shared__ Terms all[64][16];
  const int r = threadIdx.x & 15, at = threadIdx.x >> 4, m = blockIdx.x * 16 + r;
  Terms t = {-INFINITY, 0.f};
  if (m < rows)
#pragma unroll 4
    for (int b = at; b < blocks; b += 64) {
      const float2 q = part[(size_t)b * rows + m];
      t.join(Terms{q.x, q.y});
    }
  all[at][r] = t;
#pragma unroll
  for (int n = 32; n; n >>= 1) {
    __syncthreads();
    if (at < n) {
      t.join(all[at + n][r]);
      all[at][r] = t;
    }
  }
  if (at || m >= rows) return;
  const int y = targets[m];
  const bool has = y >= 0 && y < vocab;
  const float own = has ? picked[m] : -INFINITY;
  float top = fmaxf(ceilf(own * LOG2E), t.top);
  // (M is off by half its last place: 64 for a logit of 2^30, which sums bear; some way beyond, terms would be infinite or all be 0)
  if (fabsf(top) >= 0x1p30f * LOG2E && top != -INFINITY) top = __builtin_nanf("");
  const float others = t.at(top), mine = fmaf(own, LOG2E, -top);
  const float total = others + (has ? exp2f(mine) : 0.f), miss = others / total;
  loss[m] = !has ? 0.f : miss < 0.5f ? -log1pf(-miss) : (log2f(total) - mine) * 0.693147181f;
  state[3 * m] = top;
  state[3 * m + 1] = 1.f / total;
  state[3 * m + 2] = miss;
}

// to = *factor times the sum of the slices, each n elements
template <typename T> __global__ __launch_bounds__(256) void k_sum(const float *from, int slices, size_t n, const float *factor, T *to) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) {
    float sum = from[i];
#pragma unroll 8
    for (int k = 1; k < slices; ++k) sum += from[k * n + i];
    to[i] = (T)(sum * *factor);
  }
}
__global__ __launch_bounds__(256) void k_clear(uint16_t *to, size_t n) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) to[i] = 0;
}

// Workgroups of 256 threads for n elements; a grid has fewer than 2^32 threads, the kernels go round
unsigned groups_for(size_t n) { return n < (1u << 28) ? (unsigned)((n + 255) / 256) : 1u << 20; }

// ---- workspace ------------------------------------------------------------------------------
struct Space {
  Tile logits; // of the products that make logits
  int parts, dp, padded, width, block; // width: entries of a piece of the vocabulary; block: those of a wavefront
  bool twice;                          // G is rounded, and has what that left as more rows
  int rows_g;                          // of G with those
  int at_once;                         // entries whose logits one launch makes at most
  size_t h, w, part, picked, common, ht, wt, gm, gt, sum_h, sum_w, bytes;
  Space(const VocabShape &p, bool grad) {
    parts = p.bf16 ? 1 : 3;
    logits = tile_for(p.vocab, p.rows, parts, true);
    block = logits == BIG ? (parts == 1 ? 128 : 64) : 32;
    const int ks = parts == 1 ? KS<1> : KS<3>, rows = rows_of_b(logits, parts);
    dp = (p.d + ks - 1) / ks * ks;
    padded = (p.rows + rows - 1) / rows * rows;
    twice = p.bf16 && p.rows <= FEW;
    rows_g = twice ? 2 * p.rows : p.rows;
    // 2^22 tiles of 512 threads (a grid has fewer than 2^32)
    const int tile_a = rows_of_a(logits), tiles_b = padded / rows, fit_grid = (1 << 22) / (tiles_b > 0 ? tiles_b : 1);
    at_once = fit_grid < (1 << 20) / tile_a ? fit_grid * tile_a : 1 << 20;
    // G of a piece has about 2^27 elements, and a piece of w no more
    const long long all = ((long long)p.vocab + tile_a - 1) / tile_a * tile_a, most = grad ? (padded > dp ? padded : dp) : dp;
    long long fit = (1ll << 27) / (most > 0 ? most : 1) / 256 * 256;
    if (fit < 2048) fit = 2048;
    if (fit > at_once) fit = at_once;
    width = (int)(fit < all ? fit : all);
    size_t at = 0;
    auto take = [&](size_t n) { const size_t was = at; at += (n + 255) / 256 * 256; return was; };
    h = take((size_t)2 * parts * p.rows * dp);
    w = take((size_t)2 * parts * width * dp);
    if (!grad) {
      part = take(sizeof(float2) * (size_t)(all / block) * p.rows);
      picked = take(sizeof(float) * (size_t)p.rows);
    } else {
      common = take(sizeof(float));
      ht = take((size_t)2 * parts * p.d * padded);
      wt = take((size_t)2 * parts * p.d * width);
      gm = take((size_t)2 * parts * padded * width);
      gt = take((size_t)2 * parts * padded * width);
      const Slices sh(rows_g, p.d, width / ks, parts), sw(width < p.vocab ? width : p.vocab, p.d, padded / ks, parts);
      sum_h = take(twice || width < p.vocab || sh.count > 1 ? sizeof(float) * (size_t)sh.count * rows_g * p.d : 0);
      // (the last piece may be so much narrower that it is cut further: no more than 256 tiles in all)
      sum_w = take(sw.count > 1 || width < p.vocab ? sizeof(float) * 256 * (size_t)256 * 256 : 0);
    }
    bytes = at;
  }
};

#define TRY(call)                                 \
  do {                                            \
    const hipError_t e_ = (call);                 \
    if (e_ != hipSuccess) return e_;              \
  } while (0)

// Whether rows can go into products from where they are: whole steps, on 16 bytes.  (Floats as A of the products that make logits only.)
template <typename T> bool direct(const T *from, long long ld, int cols) {
  return cols % (sizeof(T) == 2 ? 64 : 32) == 0 && ld * sizeof(T) % 16 == 0 && (uintptr_t)from % 16 == 0;
}
template <int PARTS, class Epilogue> hipError_t logits(Tile t, bool w_direct, const Product &p, const Epilogue &ep, hipStream_t s) {
  if constexpr (PARTS > 1)
    if (w_direct) return product<PARTS, true>(t, p, ep, s);
  return product<PARTS, false>(t, p, ep, s);
}

template <typename T> Operand operand(const T *from, long long ld, int rows, int cols, int padded_cols, __bf16 *to_rows, int padded_rows, __bf16 *to_cols) {
  Operand m = {from, ld, rows, cols, padded_cols, padded_rows, to_rows, to_cols, nullptr, nullptr, 0, 0, 0, 0};
  m.tiles_c = (padded_cols + 63) / 64;
  m.tiles = to_rows || to_cols ? (unsigned)m.tiles_c * ((unsigned)((to_cols ? padded_rows : rows) + 63) / 64u) : 0;
  return m;
}
template <typename T, int PARTS> hipError_t lay_out(const Operand &x, const Operand &y, const int *targets, const float *dloss, int rows, int vocab, float *common, hipStream_t s) {
  const unsigned blocks = x.tiles + y.tiles + (common != nullptr);
  if (!blocks) return hipSuccess;
  k_operands<T, PARTS><<<blocks, 256, 0, s>>>(x, y, targets, dloss, rows, vocab, common);
  return hipGetLastError();
}

template <typename T, int PARTS>
hipError_t loss(const VocabShape &p, const T *h, const T *w, const int *targets, float *loss, float *state, char *work, hipStream_t s) {
  const Space sp(p, false);
  __bf16 *const hr = (__bf16 *)(work + sp.h), *const wr = (__bf16 *)(work + sp.w);
  const bool h_direct = PARTS == 1 && direct(h, p.ld_h, p.d), w_direct = direct(w, p.ld_w, p.d);
  Product q = {};
  q.rows_b = p.rows;
  q.ksteps = sp.dp / KS<PARTS>;
  q.b = h_direct ? (const __bf16 *)h : hr;
  q.ldb = h_direct ? p.ld_h : sp.dp * PARTS;
  q.lda = w_direct ? p.ld_w * (sizeof(T) / 2) : sp.dp * PARTS;
  const int width = !w_direct ? sp.width : p.vocab < sp.at_once ? p.vocab : sp.at_once;
  LossEpilogue ep = {targets, (float2 *)(work + sp.part), (float *)(work + sp.picked), 0, p.vocab, p.rows};
  for (long long v = 0; v < p.vocab; v += width) {
    const int entries = (int)(p.vocab - v < width ? p.vocab - v : width);
    const T *const piece = w + v * p.ld_w;
    TRY((lay_out<T, PARTS>(operand(h, p.ld_h, p.rows, p.d, sp.dp, h_direct || v ? nullptr : hr, 0, nullptr),
                           operand(piece, p.ld_w, entries, p.d, sp.dp, w_direct ? nullptr : wr, 0, nullptr), nullptr, nullptr, 0, 0, nullptr, s)));
    ep.first = (int)v;
    q.rows_a = entries;
    q.a = w_direct ? (const __bf16 *)piece : wr;
    TRY((logits<PARTS>(sp.logits, w_direct, q, ep, s)));
  }
  const int tile_a = rows_of_a(sp.logits), blocks = (p.vocab + tile_a - 1) / tile_a * (tile_a / sp.block);
  k_join<<<(p.rows + 15) / 16, 1024, 0, s>>>(ep.part, ep.picked, targets, blocks, p.rows, p.vocab, loss, state);
  return hipGetLastError();
}

template <typename T, int PARTS>
hipError_t gradients(const VocabShape &p, const T *h, const T *w, const int *targets, const float *state, const float *dloss, T *dh, T *dw,
                     char *work, hipStream_t s) {
  const Space sp(p, true);
  float *const common = (float *)(work + sp.common), *const sum_h = (float *)(work + sp.sum_h), *const sum_w = (float *)(work + sp.sum_w);
  __bf16 *const hr = (__bf16 *)(work + sp.h), *const wr = (__bf16 *)(work + sp.w), *const ht = (__bf16 *)(work + sp.ht), *const wt = (__bf16 *)(work + sp.wt);
  __bf16 *const gm = (__bf16 *)(work + sp.gm), *const gt = (__bf16 *)(work + sp.gt);
  const bool h_direct = PARTS == 1 && direct(h, p.ld_h, p.d), w_direct = direct(w, p.ld_w, p.d);
  const int tile_a = rows_of_a(sp.logits);
  const bool summed = sp.twice || sp.width < p.vocab || Slices(p.rows, p.d, sp.width / KS<PARTS>, PARTS).count > 1;
  int slices_h = 1;
  for (long long v = 0; v < p.vocab; v += sp.width) {
    const int entries = (int)(p.vocab - v < sp.width ? p.vocab - v : sp.width), width = (entries + tile_a - 1) / tile_a * tile_a;
    const T *const piece = w + v * p.ld_w;
    Operand oh = operand(h, p.ld_h, p.rows, p.d, sp.dp, h_direct || v ? nullptr : hr, sp.padded, v ? nullptr : ht);
    oh.targets = targets;
    oh.dloss = dloss;
    oh.vocab = p.vocab;
    oh.again = sp.twice ? FEW : 0;
    TRY((lay_out<T, PARTS>(oh, operand(piece, p.ld_w, entries, p.d, sp.dp, w_direct ? nullptr : wr, width, wt), targets, dloss, p.rows, p.vocab, v ? nullptr : common, s)));
    Product q = {w_direct ? (const __bf16 *)piece : wr, h_direct ? (const __bf16 *)h : hr, w_direct ? p.ld_w * (long long)(sizeof(T) / 2) : sp.dp * PARTS,
                 h_direct ? p.ld_h : sp.dp * PARTS, entries, p.rows, sp.dp / KS<PARTS>, 0, 0, 0, 0};
    auto g = [&](auto ep) {
      ep = {targets, state, dloss, common, gm, gt, (int)v, p.vocab, p.rows, width, sp.padded};
      return logits<PARTS>(sp.logits, w_direct, q, ep, s);
    };
    if constexpr (PARTS == 1) {
      if (sp.twice) TRY(g(GradEpilogue<1, true>()));
      else TRY(g(GradEpilogue<1, false>()));
    } else TRY(g(GradEpilogue<PARTS, false>()));
    const Slices sh(sp.rows_g, p.d, width / KS<PARTS>, PARTS, v ? slices_h : 256), sw(entries, p.d, sp.padded / KS<PARTS>, PARTS);
    if (!v) slices_h = sh.count;
    Product dhq = {gm, wt, (long long)width * PARTS, (long long)width * PARTS, sp.rows_g, p.d, width / KS<PARTS>, 0, 0, sh.count, sh.steps};
    if (!summed) TRY((product<PARTS, false>(sh.tile, dhq, StoreEpilogue<T>{dh, common, p.d, 0, p.rows, p.d, false}, s)));
    else TRY((product<PARTS, false>(sh.tile, dhq, StoreEpilogue<float>{sum_h, nullptr, p.d, (long long)sp.rows_g * p.d, sp.rows_g, p.d, v > 0}, s)));
    Product dwq = {gt, ht, (long long)sp.padded * PARTS, (long long)sp.padded * PARTS, entries, p.d, sp.padded / KS<PARTS>, 0, 0, sw.count, sw.steps};
    T *const to = dw + v * p.d;
    if (sw.count == 1) TRY((product<PARTS, false>(sw.tile, dwq, StoreEpilogue<T>{to, common, p.d, 0, entries, p.d, false}, s)));
    else {
      const size_t n = (size_t)entries * p.d;
      TRY((product<PARTS, false>(sw.tile, dwq, StoreEpilogue<float>{sum_w, nullptr, p.d, (long long)n, entries, p.d, false}, s)));
      k_sum<T><<<groups_for(n), 256, 0, s>>>(sum_w, sw.count, n, common, to);
      TRY(hipGetLastError());
    }
  }
  if (summed) {
    const size_t n = (size_t)p.rows * p.d;
    k_sum<T><<<groups_for(n), 256, 0, s>>>(sum_h, sp.twice ? 2 * slices_h : slices_h, n, common, dh);
  }
  return hipGetLastError();
}

} // namespace

size_t vocab_workspace(const VocabShape &p, bool grad) { return p.rows ? Space(p, grad).bytes : 0; }

hipError_t launch_vocab_loss(const VocabShape &p, const void *h, const void *w, const int *targets, float *loss_, float *state,
                             void *work, hipStream_t s) {
  if (!p.rows) return hipSuccess;
  return p.bf16 ? loss<__bf16, 1>(p, (const __bf16 *)h, (const __bf16 *)w, targets, loss_, state, (char *)work, s)
                : loss<float, 3>(p, (const float *)h, (const float *)w, targets, loss_, state, (char *)work, s);
}

hipError_t launch_vocab_grad(const VocabShape &p, const void *h, const void *w, const int *targets, const float *state,
                             const float *dloss, void *dh, void *dw, void *work, hipStream_t s) {
  if (!p.rows) {
    const size_t n = (size_t)p.vocab * p.d * (p.bf16 ? 1 : 2);
    k_clear<<<groups_for(n), 256, 0, s>>>((uint16_t *)dw, n);
    return hipGetLastError();
  }
  return p.bf16 ? gradients<__bf16, 1>(p, (const __bf16 *)h, (const __bf16 *)w, targets, state, dloss, (__bf16 *)dh, (__bf16 *)dw, (char *)work, s)
                : gradients<float, 3>(p, (const float *)h, (const float *)w, targets, state, dloss, (float *)dh, (float *)dw, (char *)work, s);
}
