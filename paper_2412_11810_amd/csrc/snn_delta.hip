// Gated delta rule over [T][batch][heads]: a state S [dk][dv] per head, read and corrected by each step.
//
//   S_t = a_t S_{t-1} + k_t u_t^T,  u_t = beta_t (v_t - a_t S_{t-1}^T k_t),  o_t = scale S_t^T q_t,  a_t = exp(g_t)
//
// 64 steps are taken at once.  With G the sum of g from the chunk's first step on, gam = exp(G), D_tj = exp(G_t - G_j) for j <= t, S the state before
// the chunk and L' = (K K^T D) strictly below the diagonal, its steps are
//   E = V - gam K S,  w = A E with A = (1 + L' diag(beta))^-1,  u = beta w,  O = scale gam Q S + P u with P = scale Q K^T D,
//   S' = gam_end S + K^T (gam_end / gam u)
// With A1 = diag(gam_end / gam beta) A and B = P diag(beta) A, found for all chunks beforehand, that is O = scale gam Q S + B E, S' = gam_end S + K^T A1 E;
// and back, from dO and the gradient dS' of S':
//   dV = dE = B^T dO + A1^T K dS',  dS = gam_end dS' + Q^T (scale gam dO) - K^T (gam dE)
//   dP = (dO u^T) D scale,  M = -(dE u^T) D below the diagonal
//   dQ = scale gam dO S^T + dP K,  dK = gam_end / gam u dS'^T - gam dE S^T + dP^T Q + (M + M^T) K
//   dbeta_j = sum_t (P_tj dO_t . w_j - L'_tj dE_t . w_j) + gam_end / gam_j k_j . dS' w_j
//   dg_t = gam_end <S, dS'> + sum_{j<t} k_j . (of dK_j the first part) + sum_{i>=t} (q_i, k_i . the parts of dQ_i, dK_i from S) + sum_{i>=t>j} Z_ij,
//   Z = Q K^T dP + K K^T M: what was written before a decay and read after it.  (Sums of what belongs to a decay: nothing large is taken away again.)
//
// G and its differences are of 64 bits: behind a decay that forgets everything the next steps' ratios keep their digits.  A is found by substitution in
// blocks of 16, in 32 bits, and by products of blocks, so that equal keys do no harm.
// States and sums are of 32 bits.  Products go through the bf16 matrix cores: arrays of bf16 as they are, those of 32 bits in three bf16 parts, and what is
// computed on the way (S, E, u, dE, A, B) in three too, 24 bits of it: six products of two such operands, three of one beside a bf16 array.
// (Two parts would leave 16 bits.  With those, forward 4096 x 8 x 16 x 128 x 128 took 407 us instead of 508 and backward 1638 instead of 1820, but states
// were off by up to 7e-6 of their norm and gradients of gates by 2e-5.  Where nothing but a result in bf16 comes of a product they are not enough either
// (486 us forward): o is the difference of what the state held and what is written in its place, each of which may be thousands of times as large.)
//
// The kernels: what is of a chunk alone (k_chunk: A, B, and the operands in the order in which a wavefront loads them); the walk over the chunks
// with S in registers, its columns dealt to workgroups (k_walk; for the backward pass it starts at each kept state, every 4 chunks); the walk back
// with dS (k_walk_back); and what needs S, dS', w and dE of a chunk (k_grads).  Where there are few heads the walks take segments of a long sequence side by side, from
// states found by the segments' maps, S' = M S + c (k_join).  They go through the sequence in pieces of 2 GB of
// intermediate arrays.  Few steps are taken one after the other, by a kernel whose workgroup holds the whole state of a head (k_steps).
//
// At 4096 x 8 x 16 x 128 x 128 in bf16 forward takes 508 us and backward 1820; the arrays of the call alone would take 135 and 214.  What bounds them is mostly what the kernels
// leave for each other: 2.8 GB between memory and caches forward, 7.2 GB backward, where the call's arrays have 0.7 and 1.1.  Forward that is 5.5 TB/s, a
// copy's 5.2 and what the caches give; backward 4.0, as the walks and the gradients also wait for products that need one another.  Short sequences are bound by the chain
// of a chunk's steps and of the chunks.
#include "snn_rows.h"

namespace {

typedef __bf16 frag __attribute__((ext_vector_type(8)));
typedef __bf16 four __attribute__((ext_vector_type(4)));
typedef float tile __attribute__((ext_vector_type(4)));

constexpr int C = 64;      // steps of a chunk
constexpr int KEPT = SNN_DELTA_INTERVAL / C;
constexpr int FLINE = C + 4; // floats from row to row of a matrix of a chunk's steps in LDS
constexpr float LOG2E = 1.44269504f;

template <class T> constexpr int GIVEN = sizeof(T) == 2 ? 1 : 3; // parts of what the caller's arrays hold
constexpr int MADE = 3;                                    // of what is computed

struct Args {
  const void *q, *k, *v, *dout;
  const float *g, *beta, *from; // from: s0, kept (k_walk in the backward pass), ds_last, or the segments' states; NULL: zeros
  void *o, *dq, *dk_, *dv_;
  float *to, *kept, *dg, *dbeta; // to: s_last, ds0
  const int *lengths;
  // a piece's intermediate arrays, by (chunk, batch, key head) or (chunk, batch, head)
  __bf16 *kf, *qf, *ktf, *qtf; // operands: rows of steps, rows of channels
  __bf16 *af, *bf, *at, *bt;   // A1 (in the backward pass A) and B; A1 and B transposed
  float *gates;                // [3][64]: gam, gam_end / gam, beta
  double *sums;                // [64]: G, as exponents of two
  float *before, *after;       // S and dS' [dk padded][dvp]
  float *w, *de;               // [64][dvp]
  float *maps, *bounds;        // of segments: [dk padded][dvp + dk padded], c and M; the states that they begin with
  long long ld_q, ld_k, ld_v, ld_o, ld_dq, ld_dk, ld_dv;
  int T, batch, heads, key_heads, dk, dv, dvp, blocks;
  int first, chunks; // the piece's first chunk, its chunks
  int length, segments; // those of a segment of the piece
  float scale;
};

__device__ __forceinline__ int length_of(const Args &a, int b) { return a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T; }
// The chunks behind a sequence's end change nothing: they are left out, but for zeros in what they should give. Of c0..c1, those before that
__device__ __forceinline__ int before_end(const Args &a, int len, int c0, int c1) { return min(c1, max(c0, (len + C - 1) / C - a.first)); }

// ---- products ------------------------------------------------------------------------------
// Matrix instructions of 16 x 16 with sums over 32.  Lane l has row (of B: column) l % 16 and sums 8 (l / 16) on of both operands, and elements 4 (l / 16) on of
// the result's column l % 16.
template <int P> struct Operand { frag p[P]; };

template <int PA, int PB> __device__ __forceinline__ void multiply(tile &acc, const Operand<PA> &a, const Operand<PB> &b) {
  constexpr int MOST = PA > PB ? PA : PB;
#pragma unroll
  for (int s = MOST - 1; s >= 0; --s) // parts whose numbers add up to s, the small ones first
#pragma unroll
    for (int i = 0; i <= s; ++i)
      if (i < PA && s - i < PB) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[i], b.p[s - i], acc, 0, 0, 0);
}
// Several columns' products in turn: none waits for the one before
template <int PA, int PB, int N> __device__ __forceinline__ void multiply(tile (&acc)[N], const Operand<PA> &a, const Operand<PB> (&b)[N]) {
  constexpr int MOST = PA > PB ? PA : PB;
#pragma unroll
  for (int s = MOST - 1; s >= 0; --s)
#pragma unroll
    for (int i = 0; i <= s; ++i)
      if (i < PA && s - i < PB)
#pragma unroll
        for (int n = 0; n < N; ++n) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[i], b[n].p[s - i], acc[n], 0, 0, 0);
}
template <int P, int N> __device__ __forceinline__ void split(const float (&x)[N], __bf16 (&to)[P][N]) {
#pragma unroll
  for (int j = 0; j < N; ++j) {
    float left = x[j];
#pragma unroll
    for (int i = 0; i < P; ++i) {
      to[i][j] = (__bf16)left;
      left -= (float)to[i][j];
    }
  }
}
template <int P> __device__ __forceinline__ Operand<P> operand(const float (&x)[LANE]) {
  __bf16 parts[P][LANE];
  split<P, LANE>(x, parts);
  Operand<P> r;
#pragma unroll
  for (int i = 0; i < P; ++i)
#pragma unroll
    for (int j = 0; j < LANE; ++j) r.p[i][j] = parts[i][j];
  return r;
}
// Operands in memory: one after the other, each its parts, each the lanes' 16 bytes
template <int P> __device__ __forceinline__ Operand<P> fetch(const __bf16 *p, int number, int lane) {
  Operand<P> r;
#pragma unroll
  for (int i = 0; i < P; ++i) r.p[i] = *(const frag *)(p + ((number * P + i) * 64 + lane) * LANE);
  return r;
}
template <int P> __device__ __forceinline__ void leave(__bf16 *p, int number, int lane, const Operand<P> &x) {
#pragma unroll
  for (int i = 0; i < P; ++i) __builtin_nontemporal_store(x.p[i], (frag *)(p + ((number * P + i) * 64 + lane) * LANE)); // (more than the caches hold)
}
// and in LDS: planes of rows, whose 16-byte chunks are exchanged in a way that depends on the row.  A read of 16 bytes a lane takes the lanes in fours of
// four, 0-3, 12-15, 20-23 and 24-27 the first, that is rows 0-3 and 12-15 of one chunk and 4-11 of the next: each of the four has all 64 banks to
// itself then (4.3 cycles for a wavefront's; rows with 16 bytes between them 8, whole rows 24).
template <int P, int ROWS, int COLS> struct Planes {
  static_assert(COLS == 128 || COLS == 64 || COLS == 32, "rows of 256, 128 or 64 bytes");
  __bf16 e[P][ROWS * COLS];
  static __device__ __forceinline__ int place(int row, int col) {
    const int chunk = col >> 3, other = COLS == 128 ? row & 15 : COLS == 64 ? row >> 1 & 7 : -(row >> 2) & 3;
    return row * COLS + ((chunk ^ other) << 3) + (col & 7);
  }
  __device__ __forceinline__ Operand<P> get(int row, int col) const {
    Operand<P> r;
#pragma unroll
    for (int i = 0; i < P; ++i) r.p[i] = *(const frag *)(e[i] + place(row, col));
    return r;
  }
  template <int N> __device__ __forceinline__ void get(int row, int col, Operand<P> (&r)[N]) const { // of every 16th row
#pragma unroll
    for (int n = 0; n < N; ++n) r[n] = get(row + 16 * n, col);
  }
  __device__ __forceinline__ tile four_of(int row, int col) const {
    tile r = {};
#pragma unroll
    for (int i = P - 1; i >= 0; --i) {
      const four f = *(const four *)(e[i] + place(row, col));
#pragma unroll
      for (int j = 0; j < 4; ++j) r[j] += (float)f[j];
    }
    return r;
  }
  __device__ __forceinline__ void put(int row, int col, const Operand<P> &x) {
#pragma unroll
    for (int i = 0; i < P; ++i) *(frag *)(e[i] + place(row, col)) = x.p[i];
  }
  // four elements of a row
  __device__ __forceinline__ void put(int row, int col, const tile &x) {
    const float v[4] = {x[0], x[1], x[2], x[3]};
    __bf16 parts[P][4];
    split<P, 4>(v, parts);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      four f;
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = parts[i][j];
      *(four *)(e[i] + place(row, col)) = f;
    }
  }
};

__device__ __forceinline__ void lds_barrier() { // of the LDS alone: loads from memory stay in flight
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// What a lane some lanes on, some lanes back or some lanes round in the same 16 has (0: there is none)
constexpr int NEXT = 0x100, BEFORE = 0x110, ROUND = 0x120;
template <int FROM, class X> __device__ __forceinline__ X in_row(X x) {
  uint32_t word[sizeof(X) / 4];
  __builtin_memcpy(word, &x, sizeof x);
#pragma unroll
  for (uint32_t &v : word) v = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, FROM, 0xf, 0xf, true);
  __builtin_memcpy(&x, word, sizeof x);
  return x;
}
__device__ __forceinline__ double of_lane(double x, int lane) {
  uint32_t word[2];
  __builtin_memcpy(word, &x, sizeof x);
#pragma unroll
  for (uint32_t &v : word) v = (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
  __builtin_memcpy(&x, word, sizeof x);
  return x;
}

template <class T> __device__ __forceinline__ float element(const T *p, bool on) { return on ? (float)*p : 0.f; }
// Elements as they are in memory, asked for ahead of their use
template <class T> struct Octet { // 8 of a row
  words4 raw[sizeof(T) / 2];
  __device__ __forceinline__ void ask(const T *p, int count) {
    if (count >= LANE) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) raw[i] = *(const words4_any *)((const char *)p + 16 * i);
    } else {
      T x[LANE];
#pragma unroll
      for (int j = 0; j < LANE; ++j) x[j] = j < count ? p[j] : (T)0.f;
      __builtin_memcpy(raw, x, sizeof x);
    }
  }
  __device__ __forceinline__ void get(float (&v)[LANE]) const {
    T x[LANE];
    __builtin_memcpy(x, raw, sizeof x);
#pragma unroll
    for (int j = 0; j < LANE; ++j) v[j] = (float)x[j];
  }
  __device__ __forceinline__ Operand<GIVEN<T>> get() const {
    if constexpr (sizeof(T) == 2) return Operand<1>{__builtin_bit_cast(frag, raw[0])};
    else {
      float v[LANE];
      get(v);
      return operand<3>(v);
    }
  }
};
template <class T> struct Quad { // 4 of a row
  T x[4];
  typedef T any __attribute__((ext_vector_type(4), aligned(sizeof(T))));
  __device__ __forceinline__ void ask(const T *p, int count) {
    if (count >= 4) {
      const any y = *(const any *)p;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = y[j];
    } else
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = j < count ? p[j] : (T)0.f;
  }
  static __device__ __forceinline__ void put(T *p, int count, const tile &v) {
    if (count >= 4) {
      any y;
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = (T)v[j];
      *(any *)p = y;
    } else
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j < count) p[j] = (T)v[j];
  }
};

// A wavefront's 16 rows of a tile of BV columns between memory, 16 bytes a lane, and registers, four rows and every 16th column a lane, by way of LDS of its
// own.  (Asked for element by element they are half of all requests to memory, and what the walks wait for.)  Rows are as far apart in LDS as the
// lanes' four rows need to be in banks of their own.
struct Place { int rows, live, cols; }; // from the tile's first row and column on: rows in the array, those before the sequence's end, columns
template <class T, int BV> struct Strip {
  static constexpr int STRIDE = BV * sizeof(T) + 16, BYTES = 16 * STRIDE, OF_ROW = BV / 8, N = (16 * OF_ROW + 63) / 64;
  static __device__ __forceinline__ bool mine(int at) { return 16 * OF_ROW >= 64 || at < 16 * OF_ROW; } // (16 columns are 32 lanes')
  static __device__ __forceinline__ void turn() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
  }
  Octet<T> raw[N];
  // row0: the wavefront's first row of the tile
  __device__ __forceinline__ void ask(const T *head, unsigned step, int row0, int lane, const Place &p) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = 64 * i + lane, row = min(row0 + at / OF_ROW, p.rows - 1), col = at % OF_ROW * 8;
      if (mine(at)) raw[i].ask(head + ((unsigned)row * step + col), p.cols - col);
    }
  }
  template <int NT> __device__ __forceinline__ void get(char *lds, int row0, int lane, const Place &p, bool whole, tile (&v)[NT]) const {
    turn(); // (what was here before has been read)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = 64 * i + lane;
      if (mine(at)) __builtin_memcpy(lds + at / OF_ROW * STRIDE + at % OF_ROW * (8 * sizeof(T)), raw[i].raw, sizeof raw[i].raw);
    }
    turn();
    const int r = lane & 15, q4 = lane >> 4;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = (float)*(const T *)(lds + (4 * q4 + e) * STRIDE + (16 * n + r) * sizeof(T));
        v[n][e] = whole || (row0 + 4 * q4 + e < p.live && 16 * n + r < p.cols) ? x : 0.f;
      }
  }
  template <int NT> static __device__ __forceinline__ void put(char *lds, T *head, unsigned step, int row0, int lane, const Place &p, bool whole, const tile (&v)[NT]) {
    const int r = lane & 15, q4 = lane >> 4;
    turn();
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) *(T *)(lds + (4 * q4 + e) * STRIDE + (16 * n + r) * sizeof(T)) = (T)(whole || row0 + 4 * q4 + e < p.live ? v[n][e] : 0.f);
    turn();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = 64 * i + lane, row = row0 + at / OF_ROW, col = at % OF_ROW * 8;
      if (!mine(at)) continue;
      const char *from = lds + at / OF_ROW * STRIDE + at % OF_ROW * (8 * sizeof(T));
      T *to = head + ((unsigned)row * step + col);
      if (whole || (row < p.rows && col + 8 <= p.cols)) {
#pragma unroll
        for (int k = 0; k < (int)sizeof(T) / 2; ++k) *(words4_any *)((char *)to + 16 * k) = *(const words4 *)(from + 16 * k);
      } else if (row < p.rows)
        for (int j = 0; j < p.cols - col; ++j) to[j] = ((const T *)from)[j];
    }
  }
};
// Waits for all loads, where the compiler would else wait for what comes from before a loop in each of its turns, and for all that was asked for since
__device__ __forceinline__ void loaded() { __builtin_amdgcn_s_waitcnt(0x0f70); }
// Tiles of a state between registers and memory: rows of the lane's wavefront from `row` on, RT tiles of them, every 16th column from col on
template <int RT, int NT> __device__ __forceinline__ void state_from(const float *from, int row, int col, int rows, int cols, tile (&s)[RT][NT]) {
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        s[i][n][e] = element(from + (long long)(row + 16 * i + e) * cols + col + 16 * n, row + 16 * i + e < rows && col + 16 * n < cols);
}
template <int RT, int NT> __device__ __forceinline__ void state_to(float *to, int row, int col, int rows, int cols, bool whole, const tile (&s)[RT][NT]) {
  const unsigned off = (unsigned)row * cols + col;
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int n = 0; n < NT; ++n)
        if (whole || (row + 16 * i + e < rows && col + 16 * n < cols)) (to + (16 * i + e) * cols + 16 * n)[off] = s[i][n][e];
}

// ---- a chunk by itself ------------------------------------------------------------------------
// A workgroup has one head; heads that share queries and keys find the products of those each for itself: a workgroup for all of them, its registers full of
// them, took longer at every size (333 x 5 x 6 of 2 x 48 x 75 in fp32 forward 49 us instead of 35, 2048 x 4 x 6 of 2 x 128 x 128 in bf16 90 instead of 81).
// What bounds it: memory, where there are many chunks: 192 us for 8192 of 128 channels in bf16, 0.71 GB of operands written and 0.30 read, 5.3 TB/s; 131 us for 4096 in the
// backward pass, 0.65 GB, 5.0 TB/s.  Four workgroups to a compute unit, so that registers count, cover the substitution's chain of sums and the barriers between its
// parts; these are what 180 chunks of 64 channels in fp32, less than one to a compute unit, take 16 us for.
template <class T, int DK, bool BACK> __global__ __launch_bounds__(256, sizeof(T) == 2 || DK == 64 ? 4 : 3) void k_chunk(Args a) {
  constexpr int PI = GIVEN<T>, PC = MADE, KK = DK / 32;
  typedef Planes<PI, C, DK> Rows;
  struct Squares { float m[C][FLINE], x[C][FLINE]; };
  __shared__ __align__(16) char space[sizeof(Rows) > sizeof(Squares) ? sizeof(Rows) : sizeof(Squares)];
  __shared__ double sum[C];
  __shared__ float rate[C], left[C]; // beta; gam_end / gam beta
  Rows &rows = *(Rows *)space;
  auto &m = ((Squares *)space)->m, &x = ((Squares *)space)->x;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q4 = lane >> 4;
  const int h = blockIdx.x % a.heads, b = blockIdx.x / a.heads % a.batch, c = blockIdx.x / a.heads / a.batch, sharing = a.heads / a.key_heads, kh = h / sharing;
  const long long unit = ((long long)c * a.batch + b) * a.key_heads + kh, of = ((long long)c * a.batch + b) * a.heads + h;
  const bool lays = h % sharing == 0; // the operands, for all heads that share them
  const int t0 = (a.first + c) * C, len = length_of(a, b);
  if (t0 >= len) return;
  const int t = t0 + 16 * w + r;
  constexpr int SIZE = DK * C * PI; // elements of one operand array of a unit
  Octet<T> kr[KK], qr[KK];
  auto ask = [&](const void *p, long long ld, Octet<T> (&o)[KK]) {
    const T *row = (const T *)p + ((long long)t * a.batch + b) * ld + kh * a.dk;
#pragma unroll
    for (int i = 0; i < KK; ++i) o[i].ask(row + 32 * i + 8 * q4, t < len ? a.dk - 32 * i - 8 * q4 : 0);
  };
  // a head's gates, in the first wavefront, whose lanes are the chunk's steps
  const bool on = t0 + lane < len;
  auto gate = [&](const float *p) { return on ? p[((long long)(t0 + lane) * a.batch + b) * a.heads + h] : 0.f; };
  const float g = w == 0 ? gate(a.g) : 0.f, beta = w == 0 ? gate(a.beta) : 0.f;
  ask(a.k, a.ld_k, kr);
  ask(a.q, a.ld_q, qr);
  if (w == 0) {
    double G = (double)(g < -1e4f ? -1e4f : g) * 1.4426950408889634; // (minus infinity: forgotten all the same)
#pragma unroll
    for (int s = 1; s < C; s *= 2) {
      const double o = __shfl_up(G, s);
      if (lane >= s) G += o;
    }
    sum[lane] = G;
    rate[lane] = beta;
    const double end = __shfl(G, C - 1);
    float *to = a.gates + of * (3 * C);
    to[lane] = __builtin_amdgcn_exp2f((float)G);
    const float tail = __builtin_amdgcn_exp2f((float)(end - G));
    left[lane] = tail * beta;
    to[C + lane] = tail;
    to[2 * C + lane] = beta;
    if constexpr (BACK) a.sums[of * C + lane] = G;
  }
  // rows of steps: to memory as operands, and those of k to LDS
  auto give = [&](const Octet<T> (&o)[KK], Operand<PI> (&f)[KK], __bf16 *to) {
#pragma unroll
    for (int i = 0; i < KK; ++i) {
      f[i] = o[i].get();
      if (lays) leave<PI>(to + unit * SIZE, w * KK + i, lane, f[i]);
    }
  };
  auto to_lds = [&](const Operand<PI> (&f)[KK]) {
#pragma unroll
    for (int i = 0; i < KK; ++i) rows.put(16 * w + r, 32 * i + 8 * q4, f[i]);
  };
  auto turned = [&](__bf16 *to) { // rows of channels
#pragma unroll 1
    for (int f = w; f < DK / 16 * 2; f += 4) {
      Operand<PI> y;
#pragma unroll
      for (int p = 0; p < PI; ++p)
#pragma unroll
        for (int j = 0; j < LANE; ++j) y.p[p][j] = rows.e[p][Rows::place(32 * (f & 1) + 8 * q4 + j, 16 * (f >> 1) + r)];
      leave<PI>(to + unit * SIZE, f, lane, y);
    }
  };
  Operand<PI> kf[KK], qf[KK];
  give(kr, kf, a.kf);
  to_lds(kf);
  give(qr, qf, a.qf);
  __syncthreads();
  tile kk[4] = {}, qk[4] = {};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (j <= w)
#pragma unroll
      for (int i = 0; i < KK; ++i) {
        const Operand<PI> y = rows.get(16 * j + r, 32 * i + 8 * q4);
        multiply(kk[j], kf[i], y);
        multiply(qk[j], qf[i], y);
      }
    __builtin_amdgcn_sched_barrier(0);
  }
  if (lays) turned(a.ktf);
  if (BACK && lays) {
    __syncthreads();
    to_lds(qf);
    __syncthreads();
    turned(a.qtf);
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int row = 16 * w + 4 * q4 + e, col = 16 * j + r;
      float d = 0.f;
      if (j <= w && col <= row) d = __builtin_amdgcn_exp2f((float)(sum[row] - sum[col]));
      m[row][col] = col < row ? kk[j][e] * d * rate[col] : 0.f;
      x[row][col] = col <= row ? qk[j][e] * d * a.scale : 0.f;
    }
  __syncthreads();
  // P diag(beta): its rows of this wavefront's steps
  Operand<PC> pm[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    float e[LANE];
#pragma unroll
    for (int j = 0; j < LANE; ++j) e[j] = x[16 * w + r][32 * s + 8 * q4 + j] * rate[32 * s + 8 * q4 + j];
    pm[s] = operand<PC>(e);
  }
  // column r of the inverse of the diagonal's block w: a row of it after the other, the next row of m on its way
  float y[16];
  tile now[4] = {}, then[4];
#pragma unroll
  for (int n = 0; n < 16; ++n) {
    if (n < 15)
#pragma unroll
      for (int j = 0; j <= n / 4; ++j) then[j] = *(const tile *)&m[16 * w + n + 1][16 * w + 4 * j];
    float s[4] = {n == r ? 1.f : 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < n; ++j) s[j % 4] = fmaf(-now[j / 4][j % 4], y[j], s[j % 4]);
    y[n] = (s[0] + s[1]) + (s[2] + s[3]);
#pragma unroll
    for (int j = 0; j <= n / 4; ++j) now[j] = then[j];
    __builtin_amdgcn_sched_barrier(0);
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (j > w) x[16 * w + 4 * q4 + e][16 * j + r] = 0.f;
#pragma unroll
  for (int n = 0; n < 16; ++n)
    if (n / 4 == q4) x[16 * w + n][16 * w + r] = y[n];
  __syncthreads();
  // column w of blocks, from the diagonal down: X_nw = -X_nn sum_j M_nj X_jw.  Four instructions of 16 x 16 with sums over 4 make a product; their sums
  // are taken over elements e, 4 + e, .. of both operands, so that a result's registers are the next one's operand.
  tile inv[4] = {};
#pragma unroll
  for (int n = 0; n < 4; ++n) {
    if (n == w)
#pragma unroll
      for (int e = 0; e < 4; ++e) inv[n][e] = x[16 * n + 4 * q4 + e][16 * w + r];
    if (n > w) {
      tile s = {}, z = {};
#pragma unroll
      for (int j = 0; j < n; ++j)
        if (j >= w) {
          const tile f = *(const tile *)&m[16 * n + r][16 * j + 4 * q4];
#pragma unroll
          for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(f[e], inv[j][e], s, 0, 0, 0);
        }
      const tile f = *(const tile *)&x[16 * n + r][16 * n + 4 * q4];
#pragma unroll
      for (int e = 0; e < 4; ++e) z = __builtin_amdgcn_mfma_f32_16x16x4f32(-f[e], s[e], z, 0, 0, 0);
      inv[n] = z;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[16 * n + 4 * q4 + e][16 * w + r] = z[e];
    }
  }
  __syncthreads();
  // A lower triangular matrix in x, or its transpose, times a factor of its rows; blocks of zeros, which nothing reads, are left out
  auto emit = [&](__bf16 *to, bool over, bool scaled) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (over ? 2 * s + 1 < w : 2 * s > w) continue;
      float e[LANE];
#pragma unroll
      for (int j = 0; j < LANE; ++j) {
        const int k = 32 * s + 8 * q4 + j;
        e[j] = (over ? x[k][16 * w + r] : x[16 * w + r][k]) * (scaled ? left[over ? k : 16 * w + r] : 1.f);
      }
      leave<PC>(to + of * (C * C * PC), 2 * w + s, lane, operand<PC>(e));
    }
  };
  emit(a.af, false, !BACK);
  if constexpr (BACK) emit(a.at, true, true);
  tile product[4] = {};
#pragma unroll
  for (int n = 0; n < 4; ++n)
#pragma unroll
    for (int s = 0; s < 2; ++s)
      if (n <= w && 2 * s <= w && 2 * s + 1 >= n) {
        float e[LANE];
#pragma unroll
        for (int j = 0; j < LANE; ++j) e[j] = x[32 * s + 8 * q4 + j][16 * n + r];
        multiply(product[n], pm[s], operand<PC>(e));
      }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < 4; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) x[16 * w + 4 * q4 + e][16 * n + r] = product[n][e];
  __syncthreads();
  if constexpr (BACK) emit(a.bt, true, false);
  else emit(a.bf, false, false);
}

// ---- the walk over the chunks -------------------------------------------------------------------
// Workgroups of one head are on one die: they share what k_chunk left.
struct Unit { int of, block; };
__device__ __forceinline__ Unit unit_of(unsigned id, int units, int blocks) {
  if (units % 8 == 0) return {(int)(id / 8 / blocks * 8 + id % 8), (int)(id / 8 % blocks)};
  return {(int)(id / blocks), (int)(id % blocks)};
}

// AGAIN: of the backward pass, from a kept state to the next; leaves S and w of each chunk.  MAPS: leaves what a segment makes of the state before it, M S + c:
// c from no state, and M's columns from those of the identity, without values.
// What bounds it: a chunk's three products after one another, with an exchange through LDS and a barrier after each, 5 us for 32 columns of 128 channels with two
// workgroups in a compute unit, and what these load meanwhile.  337 us for 64 chunks of 128 heads in bf16: 0.69 PFLOP/s, and 1.49 GB read and 0.29 written, 5.3 TB/s.  (0.85 GB
// of it are different ones: a head's workgroups meet in their L2 only in part.)  AGAIN: 179 us for half of the chunks, 0.75 GB, 4.2 TB/s.  Operands as k_chunk laid them out
// go from memory to registers a chunk ahead; made here of rows of q and k they took a quarter longer.
enum Walk { WALK, AGAIN, MAPS };
template <int RT, int NT> __device__ __forceinline__ void identity(int row, int col, tile (&s)[RT][NT]) {
#pragma unroll
  for (int i = 0; i < RT; ++i)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[i][n][e] = row + 16 * i + e == col + 16 * n ? 1.f : 0.f;
}
template <class T, int DK, int BV, Walk HOW> __global__ __launch_bounds__(256, sizeof(T) == 2 || DK == 64 ? 2 : 1) void k_walk(Args a) {
  constexpr bool REC = HOW == AGAIN, OUT = HOW == WALK;
  constexpr int PI = GIVEN<T>, PC = MADE, KK = DK / 32, RT = DK / 64, NT = BV / 16;
  __shared__ __align__(16) Planes<PC, BV, DK> st;
  __shared__ __align__(16) Planes<PC, BV, C> et, wt;
  __shared__ __align__(16) char strips[4][REC && Strip<float, BV>::BYTES > Strip<T, BV>::BYTES ? Strip<float, BV>::BYTES : Strip<T, BV>::BYTES];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q4 = lane >> 4;
  const int per = a.batch * a.heads, blocks = a.blocks + (HOW == MAPS ? DK / BV : 0);
  const Unit u = unit_of(blockIdx.x % (per * blocks), per, blocks);
  const int segment = blockIdx.x / (per * blocks);
  const bool of_map = HOW == MAPS && u.block >= a.blocks;
  const int h = u.of % a.heads, b = u.of / a.heads, kh = h / (a.heads / a.key_heads), v0 = (of_map ? u.block - a.blocks : u.block) * BV;
  const int len = length_of(a, b);
  const int srow = 16 * w * RT + 4 * q4, col = v0 + r;
  const bool cols = !of_map && v0 + BV <= a.dv, all = cols && a.dk == DK; // the columns, the state are there
  tile s[RT][NT] = {};
  if (HOW != MAPS && a.from) state_from(a.from + ((long long)((REC ? a.first / KEPT : 0) + segment) * per + u.of) * a.dk * a.dv, srow, col, a.dk, a.dv, s);
  if (of_map) identity(srow, col, s);
  loaded();
  const int c0 = segment * a.length, chunks = min(c0 + a.length, a.chunks), c1 = before_end(a, len, c0, chunks);
  const int row0 = 16 * w + 4 * q4;
  // What the next chunk needs is on its way while this one is worked on: each part is asked for as soon as this chunk's has been used.
  Operand<PI> k[KK], q[OUT ? KK : 1], kt[RT][2];
  Operand<PC> am[2], bm[2];
  Strip<T, BV> v;
  char *const strip = strips[w];
  tile gam, left; // left: gam_end / gam beta
  float end;
  auto of_keys = [&](int c) { return (((long long)c * a.batch + b) * a.key_heads + kh) * (DK * C * PI); };
  auto of_head = [&](int c) { return ((long long)c * a.batch + b) * a.heads + h; };
  auto ask_rows = [&](int c) {
#pragma unroll
    for (int i = 0; i < KK; ++i) {
      k[i] = fetch<PI>(a.kf + of_keys(c), w * KK + i, lane);
      if constexpr (OUT) q[i] = fetch<PI>(a.qf + of_keys(c), w * KK + i, lane);
    }
  };
  const unsigned step_v = (unsigned)(a.batch * a.ld_v), step_o = (unsigned)(a.batch * a.ld_o);
  auto place_of = [&](int t0) { return Place{a.T - t0, len - t0, of_map ? 0 : a.dv - v0}; };
  auto ask_values = [&](int c) {
    const int t0 = (a.first + c) * C;
    v.ask((const T *)a.v + ((long long)t0 * a.batch + b) * a.ld_v + h * a.dv + v0, step_v, 16 * w, lane, place_of(t0));
  };
  auto ask_squares = [&](const __bf16 *p, int c, Operand<PC> (&m)[2]) { // (lower triangular: the first two rows of blocks have zeros behind)
    m[0] = fetch<PC>(p + of_head(c) * (C * C * PC), 2 * w, lane);
    if (w > 1) m[1] = fetch<PC>(p + of_head(c) * (C * C * PC), 2 * w + 1, lane);
  };
  auto ask_columns = [&](int c) {
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) kt[i][j] = fetch<PI>(a.ktf + of_keys(c), 2 * (w * RT + i) + j, lane);
  };
  auto ask_gates = [&](int c) {
    const float *gates = a.gates + of_head(c) * (3 * C);
    gam = *(const tile *)(gates + row0);
    if constexpr (REC) left = *(const tile *)(gates + C + row0) * *(const tile *)(gates + 2 * C + row0);
    end = gates[C - 1];
  };
  if (c0 < c1) {
    ask_rows(c0);
    ask_values(c0);
    ask_squares(a.af, c0, am);
    if constexpr (OUT) ask_squares(a.bf, c0, bm);
    ask_columns(c0);
    ask_gates(c0);
  }
  for (int c = c0; c < c1; ++c) {
    const int t0 = (a.first + c) * C, next = min(c + 1, c1 - 1);
    const bool whole = cols && t0 + C <= len;
    if constexpr (OUT) {
      if (a.kept && (a.first + c) % KEPT == 0)
        state_to(a.kept + ((long long)((a.first + c) / KEPT) * per + u.of) * a.dk * a.dv, srow, col, a.dk, a.dv, all, s);
    }
    if constexpr (REC)
#pragma unroll
      for (int i = 0; i < RT; ++i) // (dvp is a multiple of the 32 columns of a workgroup)
        Strip<float, BV>::put(strip, a.before + of_head(c) * DK * a.dvp + v0, a.dvp, 16 * (w * RT + i), lane, Place{}, true, s[i]);
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int n = 0; n < NT; ++n) st.put(16 * n + r, 16 * (w * RT + i) + 4 * q4, s[i][n]);
    lds_barrier();
    tile e[NT] = {}, o[NT] = {};
#pragma unroll
    for (int i = 0; i < KK; ++i) {
      Operand<PC> y[NT];
      st.get(r, 32 * i + 8 * q4, y);
      multiply(e, k[i], y);
      if constexpr (OUT) multiply(o, q[i], y);
    }
    ask_rows(next);
    const Place place = place_of(t0);
    tile vn[NT];
    v.get(strip, 16 * w, lane, place, whole, vn);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int i = 0; i < 4; ++i) e[n][i] = fmaf(-gam[i], e[n][i], vn[n][i]);
      et.put(16 * n + r, row0, e[n]);
    }
    ask_values(next);
    lds_barrier();
    tile x[NT] = {};
    if constexpr (OUT)
#pragma unroll
      for (int n = 0; n < NT; ++n) o[n] *= gam * a.scale;
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (2 * j <= w) { // (A and B are lower triangular)
        Operand<PC> y[NT];
        et.get(r, 32 * j + 8 * q4, y);
        multiply(x, am[j], y);
        if constexpr (OUT) multiply(o, bm[j], y);
      }
    ask_squares(a.af, next, am);
    if constexpr (OUT) ask_squares(a.bf, next, bm);
    if constexpr (REC) Strip<float, BV>::put(strip, a.w + of_head(c) * C * a.dvp + v0, a.dvp, 16 * w, lane, Place{}, true, x);
#pragma unroll
    for (int n = 0; n < NT; ++n) wt.put(16 * n + r, row0, REC ? x[n] * left : x[n]);
    if constexpr (OUT) v.put(strip, (T *)a.o + ((long long)t0 * a.batch + b) * a.ld_o + h * a.dv + v0, step_o, 16 * w, lane, place, whole, o);
    lds_barrier();
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int n = 0; n < NT; ++n) s[i][n] *= end;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      Operand<PC> y[NT];
      wt.get(r, 32 * j + 8 * q4, y);
#pragma unroll
      for (int i = 0; i < RT; ++i) multiply(s[i], kt[i][j], y);
    }
    ask_columns(next);
    ask_gates(next);
  }
  if constexpr (HOW == MAPS)
    state_to(a.maps + ((long long)segment * per + u.of) * DK * (a.dvp + DK) + (of_map ? a.dvp : 0), srow, col, DK, a.dvp + DK, true, s);
  if constexpr (OUT) {
    for (int c = c1; c < chunks; ++c) {
      const int t0 = (a.first + c) * C;
      if (a.kept && (a.first + c) % KEPT == 0)
        state_to(a.kept + ((long long)((a.first + c) / KEPT) * per + u.of) * a.dk * a.dv, srow, col, a.dk, a.dv, all, s);
      const tile none[NT] = {};
      v.put(strip, (T *)a.o + ((long long)t0 * a.batch + b) * a.ld_o + h * a.dv + v0, step_o, 16 * w, lane, place_of(t0), false, none);
    }
    if (a.to && segment == a.segments - 1) state_to(a.to + (long long)u.of * a.dk * a.dv, srow, col, a.dk, a.dv, all, s);
  }
}

// ---- the walk back --------------------------------------------------------------------------------
// As the walk, with four products, two of them after one another: 226 us for 32 chunks of 128 heads of 128 channels in bf16, 0.91 GB, 4.0 TB/s.
template <class T, int DK, int BV, Walk HOW> __global__ __launch_bounds__(256, sizeof(T) == 2 || DK == 64 ? 2 : 1) void k_walk_back(Args a) {
  constexpr bool OUT = HOW == WALK;
  constexpr int PI = GIVEN<T>, PC = MADE, KK = DK / 32, RT = DK / 64, NT = BV / 16;
  __shared__ __align__(16) Planes<PC, BV, DK> st;
  __shared__ __align__(16) Planes<PI, BV, C> ot;
  __shared__ __align__(16) Planes<PC, BV, C> got, ut, et; // scale gam dO, K dS', -gam dE
  __shared__ __align__(16) char strips[4][Strip<float, BV>::BYTES];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q4 = lane >> 4;
  const int per = a.batch * a.heads, blocks = a.blocks + (HOW == MAPS ? DK / BV : 0);
  const Unit u = unit_of(blockIdx.x % (per * blocks), per, blocks);
  const int segment = blockIdx.x / (per * blocks) + (HOW == MAPS); // (nothing comes before the first)
  const bool of_map = HOW == MAPS && u.block >= a.blocks;
  const int h = u.of % a.heads, b = u.of / a.heads, kh = h / (a.heads / a.key_heads), v0 = (of_map ? u.block - a.blocks : u.block) * BV;
  const int len = length_of(a, b);
  const int srow = 16 * w * RT + 4 * q4, col = v0 + r;
  const bool cols = !of_map && v0 + BV <= a.dv, all = cols && a.dk == DK;
  tile s[RT][NT] = {};
  if (HOW != MAPS && a.from) state_from(a.from + ((long long)segment * per + u.of) * a.dk * a.dv, srow, col, a.dk, a.dv, s);
  if (of_map) identity(srow, col, s);
  loaded();
  const int row0 = 16 * w + 4 * q4;
  // (as in k_walk)
  Operand<PI> k[KK], kt[RT][2], qt[RT][2];
  Operand<PC> am[2], bm[2];
  Strip<T, BV> raw; // of dO
  char *const strip = strips[w];
  tile gam;
  float end;
  auto of_keys = [&](int c) { return (((long long)c * a.batch + b) * a.key_heads + kh) * (DK * C * PI); };
  auto of_head = [&](int c) { return ((long long)c * a.batch + b) * a.heads + h; };
  auto ask_rows = [&](int c) {
#pragma unroll
    for (int i = 0; i < KK; ++i) k[i] = fetch<PI>(a.kf + of_keys(c), w * KK + i, lane);
  };
  const unsigned step_o = (unsigned)(a.batch * a.ld_o), step_v = (unsigned)(a.batch * a.ld_dv);
  auto place_of = [&](int t0) { return Place{a.T - t0, len - t0, of_map ? 0 : a.dv - v0}; };
  auto ask_values = [&](int c) {
    const int t0 = (a.first + c) * C;
    raw.ask((const T *)a.dout + ((long long)t0 * a.batch + b) * a.ld_o + h * a.dv + v0, step_o, 16 * w, lane, place_of(t0));
  };
  auto ask_squares = [&](const __bf16 *p, int c, Operand<PC> (&m)[2]) { // (upper triangular: the last two rows of blocks begin with zeros)
    if (w < 2) m[0] = fetch<PC>(p + of_head(c) * (C * C * PC), 2 * w, lane);
    m[1] = fetch<PC>(p + of_head(c) * (C * C * PC), 2 * w + 1, lane);
  };
  auto ask_columns = [&](int c) {
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        qt[i][j] = fetch<PI>(a.qtf + of_keys(c), 2 * (w * RT + i) + j, lane);
        kt[i][j] = fetch<PI>(a.ktf + of_keys(c), 2 * (w * RT + i) + j, lane);
      }
  };
  auto ask_gates = [&](int c) {
    const float *gates = a.gates + of_head(c) * (3 * C);
    gam = *(const tile *)(gates + row0);
    end = gates[C - 1];
  };
  const int c0 = segment * a.length, chunks = min(c0 + a.length, a.chunks), c1 = before_end(a, len, c0, chunks);
  if constexpr (OUT)
    for (int c = c1; c < chunks; ++c) {
      const int t0 = (a.first + c) * C;
      const tile none[NT] = {};
      raw.put(strip, (T *)a.dv_ + ((long long)t0 * a.batch + b) * a.ld_dv + h * a.dv + v0, step_v, 16 * w, lane, place_of(t0), false, none);
    }
  if (c0 < c1) {
    const int c = c1 - 1;
    ask_values(c);
    ask_rows(c);
    ask_squares(a.bt, c, bm);
    ask_squares(a.at, c, am);
    ask_columns(c);
    ask_gates(c);
  }
  for (int c = c1 - 1; c >= c0; --c) {
    const int t0 = (a.first + c) * C, next = max(c - 1, c0);
    const long long of = of_head(c);
    const bool whole = cols && t0 + C <= len;
    const Place place = place_of(t0);
    if constexpr (OUT)
#pragma unroll
      for (int i = 0; i < RT; ++i) Strip<float, BV>::put(strip, a.after + of * DK * a.dvp + v0, a.dvp, 16 * (w * RT + i), lane, place, true, s[i]);
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int n = 0; n < NT; ++n) st.put(16 * n + r, srow + 16 * i, s[i][n]);
    tile given[NT];
    raw.get(strip, 16 * w, lane, place, whole, given);
#pragma unroll
    for (int n = 0; n < NT; ++n) ot.put(16 * n + r, row0, given[n]);
    lds_barrier(); // (and every wavefront is through with the last chunk)
#pragma unroll
    for (int n = 0; n < NT; ++n) got.put(16 * n + r, row0, given[n] * (gam * a.scale));
    ask_values(next);
    tile d[NT] = {};
#pragma unroll
    for (int i = 0; i < KK; ++i) {
      Operand<PC> y[NT];
      st.get(r, 32 * i + 8 * q4, y);
      multiply(d, k[i], y);
    }
    ask_rows(next);
#pragma unroll
    for (int n = 0; n < NT; ++n) ut.put(16 * n + r, row0, d[n]);
    tile x[NT] = {};
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (2 * j + 1 >= w) { // (transposed, A1 and B are upper triangular)
        Operand<PI> y[NT];
        ot.get(r, 32 * j + 8 * q4, y);
        multiply(x, bm[j], y);
      }
    ask_squares(a.bt, next, bm);
    lds_barrier();
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (2 * j + 1 >= w) {
        Operand<PC> y[NT];
        ut.get(r, 32 * j + 8 * q4, y);
        multiply(x, am[j], y);
      }
    ask_squares(a.at, next, am);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (!whole)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[n][e] = t0 + row0 + e < len ? x[n][e] : 0.f;
      et.put(16 * n + r, row0, x[n] * -gam);
    }
    if constexpr (OUT) Strip<float, BV>::put(strip, a.de + of * C * a.dvp + v0, a.dvp, 16 * w, lane, place, true, x);
    if constexpr (OUT) raw.put(strip, (T *)a.dv_ + ((long long)t0 * a.batch + b) * a.ld_dv + h * a.dv + v0, step_v, 16 * w, lane, place, whole, x);
    lds_barrier();
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int n = 0; n < NT; ++n) s[i][n] *= end;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      Operand<PC> y[NT], z[NT];
      got.get(r, 32 * j + 8 * q4, y);
      et.get(r, 32 * j + 8 * q4, z);
#pragma unroll
      for (int i = 0; i < RT; ++i) multiply(s[i], qt[i][j], y);
#pragma unroll
      for (int i = 0; i < RT; ++i) multiply(s[i], kt[i][j], z);
    }
    ask_columns(next);
    ask_gates(next);
  }
  if constexpr (HOW == MAPS)
    state_to(a.maps + ((long long)segment * per + u.of) * DK * (a.dvp + DK) + (of_map ? a.dvp : 0), srow, col, DK, a.dvp + DK, true, s);
  else if (a.to && !segment) state_to(a.to + (long long)u.of * a.dk * a.dv, srow, col, a.dk, a.dv, all, s);
}

// ---- the states between segments ------------------------------------------------------------------
// S' = M S + c, a segment after the other, by instructions of 32 bits; a workgroup has 16 columns.
template <int DK, bool BACK> __global__ __launch_bounds__(256) void k_join(Args a) {
  constexpr int RT = DK / 64, KT = DK / 16;
  __shared__ __align__(16) float st[2][16][DK + 4];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q4 = lane >> 4;
  const int per = a.batch * a.heads, blocks = a.dvp / 16, of = blockIdx.x / blocks, col = blockIdx.x % blocks * 16 + r, row0 = 16 * w * RT + 4 * q4, ld = a.dvp + DK;
  tile s[RT][1] = {};
  if (a.from) state_from(a.from + (long long)of * a.dk * a.dv, row0, col, a.dk, a.dv, s);
  tile m[RT][KT], c[RT];
  auto ask = [&](int segment) {
    const float *from = a.maps + ((long long)segment * per + of) * DK * ld;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
#pragma unroll
      for (int j = 0; j < KT; ++j) m[i][j] = *(const tile *)(from + (16 * (w * RT + i) + r) * ld + a.dvp + 16 * j + 4 * q4);
#pragma unroll
      for (int e = 0; e < 4; ++e) c[i][e] = from[(row0 + 16 * i + e) * ld + col];
    }
  };
  if (a.segments > 1) ask(BACK ? a.segments - 1 : 0);
  for (int n = 0; n < a.segments; ++n) {
    const int segment = BACK ? a.segments - 1 - n : n;
    state_to(a.bounds + ((long long)segment * per + of) * a.dk * a.dv, row0, col, a.dk, a.dv, false, s);
    if (n == a.segments - 1) break;
#pragma unroll
    for (int i = 0; i < RT; ++i) *(tile *)&st[n & 1][r][row0 + 16 * i] = s[i][0];
    lds_barrier();
#pragma unroll
    for (int i = 0; i < RT; ++i) s[i][0] = c[i];
#pragma unroll
    for (int j = 0; j < KT; ++j) {
      const tile f = *(const tile *)&st[n & 1][r][16 * j + 4 * q4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < RT; ++i) s[i][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(m[i][j][e], f[e], s[i][0], 0, 0, 0);
    }
    if (n + 2 < a.segments) ask(BACK ? segment - 1 : segment + 1);
  }
}

// ---- gradients of a chunk's queries, keys and gates -----------------------------------------------
// Sums over the state's columns go through LDS 32 at a time, in two places in turn, the next ones on their way; results are [dk][t], so that a lane has four elements of one step's
// row.  Eight wavefronts: four take 16 steps each, with one half of the channels, and of the chunk's steps before theirs, four with the other.
// What bounds it: 46 MFLOP a chunk of 128 x 128, six instructions to a product of what is computed on the way, at 0.50 PFLOP/s, and 1.3 GB for 4096 chunks, 3.5 TB/s: one workgroup
// to a compute unit, so that few wavefronts cover the times from memory and LDS.  373 us for 4096 chunks in bf16, own keys, 211 registers; with 128 registers and two
// workgroups values spill, and it is slower.  Where heads share queries and keys, gq and gk live across the loop over the heads: at 128 channels 256 registers are not enough
// then and 41 spill in bf16, 124 in fp32 (at 64 channels none and 2): 4096 x 8 x 6 heads of 128 x 128 in bf16 take 820 us backward in all with two of keys, 785 with six.
template <class T, int DK, bool ONE> __global__ __launch_bounds__(512, 2) void k_grads(Args a) {
  constexpr int PI = GIVEN<T>, PC = MADE, KK = DK / 32, NT = DK / 32; // NT: tiles of a half of the channels
  struct Sums { Planes<PC, DK, 32> before, after; Planes<PC, C, 32> w; };
  struct Rows { Planes<PI, C, DK> q, k; };
  struct Squares { float dp[C][FLINE], m[C][FLINE]; };
  constexpr size_t FIRST = 2 * sizeof(Sums) > sizeof(Squares) ? 2 * sizeof(Sums) : sizeof(Squares);
  __shared__ __align__(16) char space[sizeof(Rows) > FIRST ? sizeof(Rows) : FIRST];
  __shared__ float of_col[4][C], of_row[3][2][C], of_all[8], gates[3][C];
  __shared__ double G[C];
  Sums *const sums = (Sums *)space; // two, one of which is read while the other is written
  Rows &rows = *(Rows *)space;
  Squares &squares = *(Squares *)space;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = wave & 3, half = wave >> 2, r = lane & 15, q4 = lane >> 4;
  const int unit = blockIdx.x, kh = unit % a.key_heads, b = unit / a.key_heads % a.batch, c = unit / a.key_heads / a.batch;
  const int t0 = (a.first + c) * C, len = length_of(a, b), group = ONE ? 1 : a.heads / a.key_heads, row0 = 16 * w + 4 * q4;
  const int mine = 16 * w + r, t = t0 + mine; // a lane's step
  tile gq[NT] = {}, gk[NT] = {};
  if (t0 >= len && wave == 0 && t0 + lane < a.T)
    for (int i = 0; i < group; ++i) {
      const long long at = ((long long)(t0 + lane) * a.batch + b) * a.heads + kh * group + i;
      a.dg[at] = a.dbeta[at] = 0.f;
    }
  for (int i = 0; i < group && t0 < len; ++i) {
    const int h = kh * group + i;
    const long long of = ((long long)c * a.batch + b) * a.heads + h;
    long long of_k = (long long)unit * (DK * C * PI);
    if constexpr (!ONE) asm volatile("" : "+s"(of_k)); // (what is the same for all heads is read again for each: there are no registers to keep it)
    const float *before = a.before + of * DK * a.dvp, *after = a.after + of * DK * a.dvp, *wp = a.w + of * C * a.dvp, *ep = a.de + of * C * a.dvp;
    const T *dp = (const T *)a.dout + ((long long)t0 * a.batch + b) * a.ld_o + h * a.dv;
    const int srow = threadIdx.x / 4, scol = threadIdx.x % 4 * 8; // of what a thread takes to LDS
    Octet<float> rb, ra, rw, re;
    Octet<T> rd;
    const unsigned off_s = srow * a.dvp + scol, off_e = mine * a.dvp + 8 * q4, off_d = (unsigned)mine * (unsigned)(a.batch * a.ld_o) + 8 * q4;
    auto ask = [&](int v) {
      if (threadIdx.x < 4 * DK) {
        rb.ask((before + v) + off_s, LANE);
        ra.ask((after + v) + off_s, LANE);
      }
      if (threadIdx.x < 4 * C) rw.ask((wp + v) + off_s, LANE);
      re.ask((ep + v) + off_e, LANE);
      rd.ask((dp + v) + off_d, t < len ? a.dv - v - 8 * q4 : 0);
    };
    const float gate = threadIdx.x < 3 * C ? a.gates[of * (3 * C) + threadIdx.x] : 0.f;
    const double sum = threadIdx.x < C ? a.sums[of * C + threadIdx.x] : 0.;
    ask(0);
    tile sq[NT] = {}, se[NT] = {}, su[NT] = {}, p[2] = {}, x[2] = {};
    float both = 0.f; // <S, dS'>
    Operand<PI> d;
    Operand<PC> e;
    auto stage = [&](Sums &to) {
      float y[LANE], z[LANE];
      if (threadIdx.x < 4 * DK) {
        rb.get(y);
        ra.get(z);
#pragma unroll
        for (int j = 0; j < LANE; ++j) both = fmaf(y[j], z[j], both);
        to.before.put(srow, scol, operand<PC>(y));
        to.after.put(srow, scol, operand<PC>(z));
      }
      if (threadIdx.x < 4 * C) {
        rw.get(y);
        to.w.put(srow, scol, operand<PC>(y));
      }
      rd.get(y);
      d = operand<PI>(y);
      re.get(y);
      e = operand<PC>(y);
    };
    lds_barrier(); // (every wavefront is through with the last head)
    if (threadIdx.x < 3 * C) gates[threadIdx.x / C][threadIdx.x % C] = gate;
    if (threadIdx.x < C) G[threadIdx.x] = sum;
    stage(sums[0]);
    if (32 < a.dvp) ask(32);
    for (int v = 0, turn = 0; v < a.dvp; v += 32, turn ^= 1) {
      lds_barrier();
      const Sums &now = sums[turn];
      const Operand<PC> wm = now.w.get(mine, 8 * q4);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int row = 16 * (half * NT + n) + r;
        const Operand<PC> s = now.before.get(row, 8 * q4), s2 = now.after.get(row, 8 * q4);
        multiply(sq[n], s, d);
        multiply(se[n], s, e);
        multiply(su[n], s2, wm);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (2 * half + j <= w) {
          const Operand<PC> y = now.w.get(16 * (2 * half + j) + r, 8 * q4);
          multiply(p[j], d, y);
          multiply(x[j], e, y);
        }
      if (v + 32 < a.dvp) {
        stage(sums[turn ^ 1]);
        if (v + 64 < a.dvp) ask(v + 64);
      }
    }
    // queries and keys of the chunk: what its steps are to each other, and each step's with what came from the states
    {
      Operand<PI> q[KK / 2], k[KK / 2];
#pragma unroll
      for (int n = 0; n < KK / 2; ++n) {
        q[n] = fetch<PI>(a.qf + of_k, w * KK + half * (KK / 2) + n, lane);
        k[n] = fetch<PI>(a.kf + of_k, w * KK + half * (KK / 2) + n, lane);
      }
      lds_barrier();
#pragma unroll
      for (int n = 0; n < KK / 2; ++n) {
        const int col = 32 * (half * (KK / 2) + n) + 8 * q4;
        rows.q.put(mine, col, q[n]);
        rows.k.put(mine, col, k[n]);
      }
      lds_barrier();
    }
    const float gam = gates[0][mine], tail = gates[1][mine], beta = gates[2][mine], end = gates[0][C - 1];
    float read_by = 0.f, wrote = 0.f; // what a step reads of what was before, and what is left of its own at the end, but for beta
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int col = 16 * (half * NT + n) + 4 * q4;
      const tile q = rows.q.four_of(mine, col), k = rows.k.four_of(mine, col);
      sq[n] *= gam * a.scale;
      se[n] *= gam;
      su[n] *= tail;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        read_by += fmaf(q[e], sq[n][e], -(k[e] * se[n][e]));
        wrote = fmaf(k[e], su[n][e], wrote);
      }
      gq[n] += sq[n];
      gk[n] += su[n] * beta - se[n];
    }
    __builtin_amdgcn_sched_barrier(0);
    // (the columns that come last are asked for ahead, as many at a time as there are registers for)
    Operand<PI> kt[2][NT], qt[2][NT];
    auto columns = [&](int s) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        kt[s][n] = fetch<PI>(a.ktf + of_k, 2 * (half * NT + n) + s, lane);
        if (2 * s + 1 >= w) qt[s][n] = fetch<PI>(a.qtf + of_k, 2 * (half * NT + n) + s, lane);
      }
    };
    if constexpr (PI == 1) columns(0);
    tile qk[2] = {}, kk[2] = {};
#pragma unroll
    for (int n = 0; n < KK; ++n) {
      const Operand<PI> q = rows.q.get(mine, 32 * n + 8 * q4), k = rows.k.get(mine, 32 * n + 8 * q4);
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (2 * half + j <= w) {
          const Operand<PI> y = rows.k.get(16 * (2 * half + j) + r, 32 * n + 8 * q4);
          multiply(qk[j], q, y);
          multiply(kk[j], k, y);
        }
    }
    lds_barrier();
    tile of_z = {};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int at = 2 * half + j, col = 16 * at + r;
      const float beta_col = gates[2][col];
      float z_col = 0.f;
      tile z_on;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = row0 + e;
        const bool low = at <= w && col <= row, below = at <= w && col < row;
        const float d = low ? __builtin_amdgcn_exp2f((float)(G[row] - G[col])) : 0.f;
        const float dps = low ? p[j][e] * d * a.scale : 0.f, me = below ? x[j][e] * d : 0.f; // beta of the column is left out
        const float zq = low ? qk[j][e] * dps : 0.f, zk = below ? kk[j][e] * me : 0.f;
        const float z = zq - zk; // of both w . dU less that of what it was taken from; times beta, of what decays lie between
        z_on[e] = z * beta_col;
        z_col += z;
        squares.dp[row][col] = dps * beta_col;
        if (below) squares.m[row][col] = squares.m[col][row] = -me * beta_col;
        if (at == w && col == row) squares.m[row][col] = 0.f;
      }
#pragma unroll
      for (int s = 16; s < 64; s *= 2) z_col += __shfl_xor(z_col, s);
      if (q4 == 0) of_col[w][col] = z_col;
      // Between column and row lies the decay of every step behind the column's up to the row's.  So far that of the row itself: the column's sums from it to the end of these 16
#pragma unroll
      for (int e = 2; e >= 0; --e) z_on[e] += z_on[e + 1];
      float next = __shfl_down(z_on[0], 16);
      if (q4 == 3) next = 0.f;
      const float two_on = __shfl_down(z_on[0] + next, 32);
      if (q4 < 2) next += two_on;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col < row0 + e) of_z[e] += z_on[e] + next;
    }
#pragma unroll
    for (int s = 16; s < 64; s *= 2) {
      read_by += __shfl_xor(read_by, s);
      wrote += __shfl_xor(wrote, s);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      of_z[e] += in_row<ROUND + 8>(of_z[e]);
      of_z[e] += in_row<ROUND + 4>(of_z[e]);
      of_z[e] += in_row<ROUND + 2>(of_z[e]);
      of_z[e] += in_row<ROUND + 1>(of_z[e]);
    }
    if (r == 0) *(tile *)(of_row[0][half] + row0) = of_z;
    if (q4 == 0) {
      of_row[1][half][mine] = read_by;
      of_row[2][half][mine] = wrote;
    }
#pragma unroll
    for (int s = 1; s < 64; s *= 2) both += __shfl_xor(both, s);
    if (lane == 0) of_all[wave] = both;
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (PI == 1) columns(1);
    lds_barrier();
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if constexpr (PI > 1) columns(s);
      // (where heads share keys, a matrix after the other: there are no registers for all three)
      auto apart = [] {
        if constexpr (!ONE) __builtin_amdgcn_sched_barrier(0);
      };
      auto matrix = [&](auto at) {
        float y[LANE];
#pragma unroll
        for (int j = 0; j < LANE; ++j) y[j] = at(32 * s + 8 * q4 + j);
        return operand<PC>(y);
      };
      if (2 * s <= w) {
        const Operand<PC> f = matrix([&](int j) { return squares.dp[mine][j]; });
#pragma unroll
        for (int n = 0; n < NT; ++n) multiply(gq[n], kt[s][n], f);
      }
      apart();
      {
        const Operand<PC> f = matrix([&](int j) { return squares.m[mine][j]; });
#pragma unroll
        for (int n = 0; n < NT; ++n) multiply(gk[n], kt[s][n], f);
      }
      apart();
      if (2 * s + 1 >= w) {
        const Operand<PC> f = matrix([&](int j) { return squares.dp[j][mine]; });
#pragma unroll
        for (int n = 0; n < NT; ++n) multiply(gk[n], qt[s][n], f);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    // A wavefront has the decays of its 16 steps, each a sum of what goes past it alone: behind strong decays that is all there is of it, and much less than
    // what lies on either side
    if (half == 0) {
      const float beta = gates[2][lane], of_w = (of_col[0][lane] + of_col[1][lane]) + (of_col[2][lane] + of_col[3][lane]), left = of_row[2][0][lane] + of_row[2][1][lane];
      float further = 0.f; // read behind these 16 steps
#pragma unroll
      for (int x = 1; x < 4; ++x)
        if (x > w) further += of_col[x][lane];
      // sums from a step on, and of those before it
      double on = (double)of_row[1][0][lane] + of_row[1][1][lane], up = ((double)left + further) * beta;
      on += in_row<NEXT + 1>(on), up += in_row<BEFORE + 1>(up);
      on += in_row<NEXT + 2>(on), up += in_row<BEFORE + 2>(up);
      on += in_row<NEXT + 4>(on), up += in_row<BEFORE + 4>(up);
      on += in_row<NEXT + 8>(on), up += in_row<BEFORE + 8>(up);
      double rest = 0.;
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (x != w) rest += x > w ? of_lane(on, 16 * x) : of_lane(up, 16 * x + 15);
      up = in_row<BEFORE + 1>(up) + rest;
      const float all = end * (((of_all[0] + of_all[1]) + (of_all[2] + of_all[3])) + ((of_all[4] + of_all[5]) + (of_all[6] + of_all[7])));
      if (lane >> 4 == w && t0 + lane < a.T) {
        const long long at = ((long long)(t0 + lane) * a.batch + b) * a.heads + h;
        a.dg[at] = t0 + lane < len ? (float)(all + on + up + ((double)of_row[0][0][lane] + of_row[0][1][lane])) : 0.f;
        a.dbeta[at] = t0 + lane < len ? of_w + left : 0.f;
      }
    }
  }
  if (t >= a.T) return;
  T *dq = (T *)a.dq + ((long long)t * a.batch + b) * a.ld_dq + kh * a.dk, *dk = (T *)a.dk_ + ((long long)t * a.batch + b) * a.ld_dk + kh * a.dk;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int col = 16 * (half * NT + n) + 4 * q4;
    Quad<T>::put(dq + col, a.dk - col, t < len ? gq[n] : tile{});
    Quad<T>::put(dk + col, a.dk - col, t < len ? gk[n] : tile{});
  }
}

// ---- step after step ------------------------------------------------------------------------------
// A workgroup has all of a head's rows and 4 LV columns, four of them and every (256 / LV)-th row a lane.  o_t = scale (q . a S + (q . k) u): both sums over the
// rows are taken of the state as it was, at once.  What bounds it: memory, the state read and written: 36 us for 1024 heads of 128 x 128, 5.7 TB/s, part of it from
// the caches.
template <class T, int DK, int LV> __global__ __launch_bounds__(256) void k_steps(Args a) {
  constexpr int GROUPS = 256 / LV, ROWS = DK / GROUPS;
  __shared__ float qs[2][DK], ks[2][DK], sums[2][4][2][LV * 4], dots[2][4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = threadIdx.x % LV, first = threadIdx.x / LV;
  const Unit u = unit_of(blockIdx.x, a.batch * a.heads, a.blocks);
  const int h = u.of % a.heads, b = u.of / a.heads, kh = h / (a.heads / a.key_heads), col = u.block * (4 * LV) + 4 * at;
  const int len = length_of(a, b), cols = min(4, a.dv - col);
  typedef tile tile_any __attribute__((aligned(4)));
  tile s[ROWS];
  const long long base = (long long)u.of * a.dk * a.dv + col;
#pragma unroll
  for (int i = 0; i < ROWS; ++i) {
    const int row = first + GROUPS * i;
    s[i] = tile{};
    if (a.from && row < a.dk) {
      const float *p = a.from + base + (long long)row * a.dv;
      if (cols == 4) s[i] = *(const tile_any *)p;
      else
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][e] = e < cols ? p[e] : 0.f;
    }
  }
  auto state_to = [&](float *to) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const int row = first + GROUPS * i;
      if (row >= a.dk) continue;
      float *p = to + base + (long long)row * a.dv;
      // (past the caches, which the next call's states need: to another place 35.6 us instead of 50.8 for 1024 heads, in place the same)
      if (cols == 4) __builtin_nontemporal_store(s[i], (tile_any *)p);
      else
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < cols) p[e] = s[i][e];
    }
  };
  if (a.kept && a.T) state_to(a.kept);
  // a step's inputs, asked for while the one before is worked on
  T q = (T)0.f, k = (T)0.f;
  T v[4];
  float g = 0.f, beta = 0.f;
  auto ask = [&](int t) {
    const long long row = (long long)t * a.batch + b;
    if ((int)threadIdx.x < a.dk) {
      q = ((const T *)a.q)[row * a.ld_q + kh * a.dk + threadIdx.x];
      k = ((const T *)a.k)[row * a.ld_k + kh * a.dk + threadIdx.x];
    }
    Quad<T> f;
    f.ask((const T *)a.v + row * a.ld_v + h * a.dv + col, cols);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = f.x[e];
    g = a.g[row * a.heads + h];
    beta = a.beta[row * a.heads + h];
  };
  if (len) ask(0);
  for (int t = 0; t < a.T; ++t) {
    T *op = (T *)a.o + ((long long)t * a.batch + b) * a.ld_o + h * a.dv + col;
    if (t >= len) {
      if (first == 0) Quad<T>::put(op, cols, tile{});
      continue;
    }
    const int turn = t & 1; // (LDS of one step is read while that of the next is written)
    if ((int)threadIdx.x < DK) {
      qs[turn][threadIdx.x] = (float)q;
      ks[turn][threadIdx.x] = (float)k;
    }
    const tile vn = {(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
    const float hold = __builtin_amdgcn_exp2f(g * LOG2E), rate = beta;
    if (t + 1 < len) ask(t + 1);
    lds_barrier();
    tile of_k = {}, of_q = {};
    float qk = 0.f;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const float k = ks[turn][first + GROUPS * i], q = qs[turn][first + GROUPS * i];
      s[i] *= hold;
      qk = fmaf(q, k, qk);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        of_k[e] = fmaf(s[i][e], k, of_k[e]);
        of_q[e] = fmaf(s[i][e], q, of_q[e]);
      }
    }
#pragma unroll
    for (int x = LV; x < 64; x *= 2) {
      qk += __shfl_xor(qk, x);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        of_k[e] += __shfl_xor(of_k[e], x);
        of_q[e] += __shfl_xor(of_q[e], x);
      }
    }
    if (lane == 0) dots[turn][wave] = qk;
    if (lane < LV) {
      *(tile *)(sums[turn][wave][0] + 4 * at) = of_k;
      *(tile *)(sums[turn][wave][1] + 4 * at) = of_q;
    }
    lds_barrier();
    of_k = of_q = tile{};
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      of_k += *(const tile *)(sums[turn][x][0] + 4 * at);
      of_q += *(const tile *)(sums[turn][x][1] + 4 * at);
    }
    qk = (dots[turn][0] + dots[turn][1]) + (dots[turn][2] + dots[turn][3]);
    const tile un = (vn - of_k) * rate;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
      const float k = ks[turn][first + GROUPS * i];
#pragma unroll
      for (int e = 0; e < 4; ++e) s[i][e] = fmaf(k, un[e], s[i][e]);
    }
    if (first == 0) Quad<T>::put(op, cols, (of_q + un * qk) * a.scale);
  }
  if (a.to) state_to(a.to);
}

// ---- launches -------------------------------------------------------------------------------------
constexpr size_t PIECE = (size_t)2 << 30; // bytes of a piece's intermediate arrays, at least 4 chunks

size_t rounded(size_t bytes) { return (bytes + 255) / 256 * 256; }

// Columns of the state that a workgroup walks with: fewer where there would be few workgroups, as a chunk then takes a shorter time.  4096 steps in one segment, 128 x 128, in us,
// with 16 and with 32 columns: forward in fp32 4 heads 260 and 314, 32 heads 363 and 410, 64 heads 710 and 519; in bf16 141 and 192, 191 and 237, 332 and 287;
// backward in fp32 4 heads 351 and 413, 16 heads 587 and 627, 32 heads 907 and 904, 64 heads 1799 and 1434; in bf16 218 and 265, 382 and 408, 595 and 591, 1114
// and 946.  Other sizes change sides at the same number of workgroups: 64 x 64 in bf16 forward 64 heads 199 and 226, 128 heads 346 and 298, backward 32 heads 353 and 366,
// 64 heads 548 and 536; 128 x 256 forward 16 heads 163 and 206, 32 heads 275 and 243.  64 columns to a workgroup are no faster than 32.
int columns(const DeltaShape &p, bool back) {
  const long long heads = (long long)p.batch * p.heads;
  return heads * ((p.dv + 31) / 32) > (back ? 64 : 128) ? 32 : 16;
}

// Whether steps are taken one after the other.  dk and dv 128, in us, so and in chunks: 16 heads, 8 steps 19.8 and 23.6 in fp32, 20.3 and 21.2 in bf16, 12 steps
// 25.3 and 23.6, 25.9 and 21.3; 128 heads, fp32 16 steps 31.9 and 36.2, 32 steps 53.3 and 36.8, bf16 8 steps 21.1 and 24.3, 12 steps 26.6 and
// 24.5; 1024 heads, fp32 32 steps 121 and 224, bf16 12 steps 58 and 100, 16 steps 69 and 101 (from no state; with one, 94.7 and 89.4).  The numbers are those of 128 channels:
// with 64 steps one after the other would pay somewhat longer (16 heads, 12 steps 17.3 and 21.6 in fp32), which the rule does not use.
bool one_by_one(const DeltaShape &p) {
  const long long heads = (long long)p.batch * p.heads;
  return p.T <= (heads < 128 ? 8 : heads < 512 ? p.bf16 ? 8 : 16 : p.bf16 ? 12 : 32);
}

// Segments of a piece, walked side by side: one walk leaves their maps, k_join the states between them, and another walk the results.  That is 2.5 times the work, for
// walks that would leave most of the chip idle, 512 workgroups in all, and at least 8 chunks for each of 3 segments.  In one segment and so, us, forward and backward:
// 16384 steps, 8 heads of 64 x 128 in bf16 450 and 198, 848 and 521, in fp32 648 and 314, 1155 and 768; 4096 steps, 4 heads of 128 x 128 in bf16 140 and 90, 218 and
// 154, in fp32 260 and 144, 351 and 257; 2048 steps, 2 heads of 64 x 64 in bf16 63 and 47, 98 and 78.  It does not pay with fewer chunks (1024 steps, 4 heads, 4 chunks
// each: 47 and 57).  With more workgroups it goes both ways, and the rule leaves it: 96 of them, 12 heads of 128 x 128, 4096 steps in bf16 159 and 186, 363 and 364,
// 16384 steps 620 and 703, 1433 and 1338, in fp32 1179 and 1305, 2341 and 2463; 128 of them, 16 heads, 16384 steps in bf16 602 and 507, 1485 and 1433, in fp32 1165 and 1069, 2302 and 2540.
int segments_of(int bv, long long walks, int chunks) {
  if (bv != 16 || walks > 64) return 1;
  const int n = (int)(512 / walks < chunks / 8 ? 512 / walks : chunks / 8);
  return n > 2 ? n : 1;
}

struct Plan {
  int dk, bv, blocks, dvp, all, chunks, per, units; // units: of key heads
  size_t bytes;
  float *last = nullptr; // where the caller wants the last state, or ds0
  Args a = {};
  Plan(const DeltaShape &p, bool back, char *work) {
    dk = p.dk <= 64 ? 64 : 128;
    per = p.batch * p.heads, units = p.batch * p.key_heads;
    dvp = (p.dv + 31) / 32 * 32;
    bv = columns(p, back);
    blocks = (dvp + bv - 1) / bv;
    all = (p.T + C - 1) / C;
    const size_t pi = p.bf16 ? 1 : 3, pc = MADE;
    auto lay = [&](int n, int segments) {
      size_t at = 0;
      auto take = [&](auto *&to, size_t count) {
        to = (std::remove_reference_t<decltype(to)>)(work ? work + at : nullptr);
        at += rounded(count * sizeof *to);
      };
      const size_t nk = (size_t)n * units, nh = (size_t)n * per;
      float *carry;
      take(carry, (size_t)per * p.dk * p.dv);
      a.to = carry;
      take(a.maps, segments > 1 ? (size_t)segments * per * dk * (dvp + dk) : 0);
      take(a.bounds, segments > 1 ? (size_t)segments * per * p.dk * p.dv : 0);
      for (__bf16 **x : {&a.kf, &a.qf, &a.ktf}) take(*x, nk * dk * C * pi);
      take(a.af, nh * C * C * pc);
      take(a.gates, nh * 3 * C);
      if (!back) take(a.bf, nh * C * C * pc);
      else {
        take(a.qtf, nk * dk * C * pi);
        take(a.bt, nh * C * C * pc);
        take(a.at, nh * C * C * pc);
        take(a.sums, nh * C);
        take(a.before, nh * dk * dvp);
        take(a.after, nh * dk * dvp);
        take(a.w, nh * C * dvp);
        take(a.de, nh * C * dvp);
      }
      return at;
    };
    const size_t one = lay(KEPT, 1) - lay(0, 1);
    const long long most = (long long)(PIECE / one) * KEPT;
    chunks = (int)(most < KEPT ? KEPT : most > all ? all : most);
    if (chunks < all) chunks = (all + (all + chunks - 1) / chunks - 1) / ((all + chunks - 1) / chunks); // as many pieces as it takes, of one length
    chunks = (chunks + KEPT - 1) / KEPT * KEPT;
    if (chunks > all) chunks = all;
    bytes = lay(chunks, segments_of(bv, (long long)per * blocks, chunks));
    a.lengths = p.lengths;
    a.ld_q = p.ld_q, a.ld_k = p.ld_k, a.ld_v = p.ld_v, a.ld_o = p.ld_o, a.ld_dq = p.ld_dq, a.ld_dk = p.ld_dk, a.ld_dv = p.ld_dv;
    a.T = p.T, a.batch = p.batch, a.heads = p.heads, a.key_heads = p.key_heads, a.dk = p.dk, a.dv = p.dv, a.dvp = dvp, a.blocks = blocks;
    a.scale = p.scale;
  }
};

// Cuts a piece into segments.  The last one may be shorter than the others
void cut(Args &a, const Plan &p) {
  a.segments = segments_of(p.bv, (long long)p.per * p.blocks, a.chunks);
  a.length = (a.chunks + a.segments - 1) / a.segments;
  if (a.length) a.segments = (a.chunks + a.length - 1) / a.length;
}

template <class T, int DK> hipError_t forward(Plan &p, hipStream_t s) {
  Args a = p.a;
  float *const carry = a.to;
  const float *from = a.from;
  for (int first = 0; first < p.all; first += p.chunks) {
    a.first = first;
    a.chunks = p.all - first < p.chunks ? p.all - first : p.chunks;
    a.from = from;
    a.to = first + a.chunks < p.all ? carry : p.last;
    k_chunk<T, DK, false><<<a.chunks * p.per, 256, 0, s>>>(a);
    cut(a, p);
    if (a.segments > 1) {
      k_walk<T, DK, 16, MAPS><<<(a.segments - 1) * p.per * (p.blocks + DK / 16), 256, 0, s>>>(a);
      k_join<DK, false><<<p.per * (p.dvp / 16), 256, 0, s>>>(a);
      a.from = a.bounds;
    }
    if (p.bv == 32) k_walk<T, DK, 32, WALK><<<a.segments * p.per * p.blocks, 256, 0, s>>>(a);
    else k_walk<T, DK, 16, WALK><<<a.segments * p.per * p.blocks, 256, 0, s>>>(a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    from = carry;
  }
  return hipSuccess;
}
template <class T, int DK> hipError_t backward(Plan &p, const float *kept, const float *ds_last, hipStream_t s) {
  Args a = p.a;
  float *const carry = a.to;
  const float *from = ds_last;
  if (!p.all) {
    a.from = ds_last;
    a.to = p.last;
    if (p.bv == 32) k_walk_back<T, DK, 32, WALK><<<p.per * p.blocks, 256, 0, s>>>(a);
    else k_walk_back<T, DK, 16, WALK><<<p.per * p.blocks, 256, 0, s>>>(a);
    return hipGetLastError();
  }
  // pieces of whole kept intervals, from the last one on
  for (int first = (p.all - 1) / p.chunks * p.chunks; first >= 0; first -= p.chunks) {
    a.first = first;
    a.chunks = p.all - first < p.chunks ? p.all - first : p.chunks;
    k_chunk<T, DK, true><<<a.chunks * p.per, 256, 0, s>>>(a);
    a.from = kept;
    a.to = nullptr;
    a.length = KEPT;
    a.segments = (a.chunks + KEPT - 1) / KEPT;
    const unsigned walks = p.per * p.blocks;
    if (p.bv == 32) k_walk<T, DK, 32, AGAIN><<<a.segments * walks, 256, 0, s>>>(a);
    else k_walk<T, DK, 16, AGAIN><<<a.segments * walks, 256, 0, s>>>(a);
    a.from = from;
    a.to = first ? carry : p.last;
    cut(a, p);
    if (a.segments > 1) {
      k_walk_back<T, DK, 16, MAPS><<<(a.segments - 1) * p.per * (p.blocks + DK / 16), 256, 0, s>>>(a);
      k_join<DK, true><<<p.per * (p.dvp / 16), 256, 0, s>>>(a);
      a.from = a.bounds;
    }
    if (p.bv == 32) k_walk_back<T, DK, 32, WALK><<<a.segments * walks, 256, 0, s>>>(a);
    else k_walk_back<T, DK, 16, WALK><<<a.segments * walks, 256, 0, s>>>(a);
    if (a.heads == a.key_heads) k_grads<T, DK, true><<<a.chunks * p.units, 512, 0, s>>>(a);
    else k_grads<T, DK, false><<<a.chunks * p.units, 512, 0, s>>>(a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    from = carry;
  }
  return hipSuccess;
}
template <class T> hipError_t steps(Plan &p, hipStream_t s) {
  Args a = p.a;
  a.to = p.last;
  const bool wide = a.dv > 64;
  a.blocks = (a.dv + (wide ? 127 : 63)) / (wide ? 128 : 64);
  const unsigned grid = (unsigned)p.per * a.blocks;
  if (p.dk == 64) {
    if (wide) k_steps<T, 64, 32><<<grid, 256, 0, s>>>(a);
    else k_steps<T, 64, 16><<<grid, 256, 0, s>>>(a);
  } else {
    if (wide) k_steps<T, 128, 32><<<grid, 256, 0, s>>>(a);
    else k_steps<T, 128, 16><<<grid, 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

} // namespace

size_t delta_workspace(const DeltaShape &p, bool back) {
  if (!p.T || (!back && one_by_one(p))) return 0;
  return Plan(p, back, nullptr).bytes;
}

hipError_t launch_delta_forward(const DeltaShape &p, const void *q, const void *k, const void *v, const float *g, const float *beta, const float *s0,
                                void *o, float *s_last, float *kept, void *work, hipStream_t s) {
  Plan plan(p, false, (char *)work);
  Args &a = plan.a;
  a.q = q, a.k = k, a.v = v, a.g = g, a.beta = beta, a.from = s0, a.o = o, a.kept = kept;
  plan.last = s_last;
  if (one_by_one(p)) return p.bf16 ? steps<__bf16>(plan, s) : steps<float>(plan, s);
  if (plan.dk == 64) return p.bf16 ? forward<__bf16, 64>(plan, s) : forward<float, 64>(plan, s);
  return p.bf16 ? forward<__bf16, 128>(plan, s) : forward<float, 128>(plan, s);
}

hipError_t launch_delta_backward(const DeltaShape &p, const void *q, const void *k, const void *v, const float *g, const float *beta, const float *kept,
                                 const void *dout, const float *ds_last, void *dq, void *dk, void *dv, float *dg, float *dbeta, float *ds0, void *work,
                                 hipStream_t s) {
  Plan plan(p, true, (char *)work);
  Args &a = plan.a;
  a.q = q, a.k = k, a.v = v, a.g = g, a.beta = beta, a.dout = dout, a.dq = dq, a.dk_ = dk, a.dv_ = dv, a.dg = dg, a.dbeta = dbeta;
  plan.last = ds0;
  if (plan.dk == 64) return p.bf16 ? backward<__bf16, 64>(plan, kept, ds_last, s) : backward<float, 64>(plan, kept, ds_last, s);
  return p.bf16 ? backward<__bf16, 128>(plan, kept, ds_last, s) : backward<float, 128>(plan, kept, ds_last, s);
}
