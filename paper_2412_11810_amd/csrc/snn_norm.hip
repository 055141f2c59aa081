// Root-mean-square norm of rows, with the addition of what went past the layers before it, and its backward pass.
//
//   s = x + residual (or x);  i = 1 / sqrt(mean(s^2) + eps);  y = w s i
//   c = mean(w dy s i);  dx = i (w dy - s i c) + dtotal;  dw = sum over rows of dy s i
//
// A row is read once and stays in registers: lanes take 8 elements at a time, rows of up to 256 elements share a wavefront with others, longer ones
// have one of their own or a workgroup of 4 or 16.  s is rounded to the arrays' type where it is written; y comes from the sum before that.
// Into 8 bits y goes without a rounding to bf16 first: its blocks are those of snn_pack (four lanes).
// Sums of squares are of 32 bits; where one is too large or too small for that, the row is multiplied by a power of two first.
// dw: a workgroup sums over its rows in registers and leaves one row of sums; a second kernel adds those up.  No atomics, so the same bits each time.
//
// What bounds it: memory.  32768 rows of 4096 in bf16: backward 202 us, 5.3 TB/s, and 11 us for dw's rows of sums; forward with residual and total into 8 bits
// 181 us, 5.2 TB/s.  Few rows are bound by the call: 64 of 2048 take 11 us, 3 of them in the kernel.  Backward in bf16 two things are not at memory's rate.  Up to 1024 rows of sums
// are read again by few workgroups (one for 32 columns): 11 of 27 us for 4329 rows of 2048, whose arrays take 10.  And rows of odd widths begin between words, and none is asked for
// before the last one's sums: 161 us for 32768 of 1501, whose arrays take 57.
#include "snn_rows.h"

namespace {

struct Args {
  const void *x, *residual, *w, *dy;
  void *total, *y, *dx;
  int8_t *codes;
  uint8_t *exps;
  float *sums; // [workgroups][n]
  long long rows, ld_x, ld_r, ld_total, ld_y, ld_dx;
  int n, lanes; // lanes of a row, where a wavefront has several
  float eps, per_n;
};

// Sums over the lanes of a row: of a part of a wavefront (`lanes`), or of WAVES wavefronts
template <int WAVES, int N, bool MOST = false> __device__ __forceinline__ void over_row(float (&v)[N], int lanes, float *lds) {
  for (int m = 1; m < (WAVES == 1 ? lanes : 64); m *= 2)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float o = __shfl_xor(v[i], m);
      v[i] = MOST ? fmaxf(v[i], o) : v[i] + o;
    }
  if constexpr (WAVES > 1) {
    const int wave = threadIdx.x >> 6;
    __syncthreads(); // (what the last sums left here has been read)
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) lds[wave * N + i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float all = lds[i];
#pragma unroll
      for (int k = 1; k < WAVES; ++k) all = MOST ? fmaxf(all, lds[k * N + i]) : all + lds[k * N + i];
      v[i] = all;
    }
  }
}

// w at a lane's place; ones where there are none.  Up to two vectors of it are held from row to row, more are read again (2 MB of L2 hold any row of w).
template <class T> __device__ __forceinline__ void weights(const Args &a, int col, float (&w)[LANE]) {
  if (a.w) read((const T *)a.w + col, a.n - col, w);
  else
#pragma unroll
    for (int j = 0; j < LANE; ++j) w[j] = 1.f;
}
template <int V> constexpr int HELD = V <= 2 ? V : 1;

// s i for a row is (s * scale) * inv: scale is 1 but for rows whose squares leave the range of 32 bits
struct Size { float scale, inv; };
template <int WAVES, int V> __device__ __forceinline__ Size size_of_row(const float (&s)[V][LANE], float squares, const Args &a, float *lds) {
  Size r = {1.f, rsqrtf(squares * a.per_n + a.eps)};
  if (__any(!(squares < 1e37f) || squares < 1e-30f)) { // (in a workgroup per row all wavefronts have the same sum)
    float top[1] = {0.f};
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int j = 0; j < LANE; ++j) top[0] = fmaxf(top[0], fabsf(s[v][j]));
    over_row<WAVES, 1, true>(top, a.lanes, lds);
    float again[1] = {0.f};
    const int e = (int)(__float_as_uint(top[0]) >> 23);
    const float scale = __uint_as_float((uint32_t)min(max(254 - e, 1), 253) << 23);
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int j = 0; j < LANE; ++j) {
        const float t = s[v][j] * scale;
        again[0] = fmaf(t, t, again[0]);
      }
    over_row<WAVES, 1>(again, a.lanes, lds);
    // (a row with an infinity or NaN stays as it is, and so does one of zeros)
    const float eps = a.eps * scale * scale; // (where that is huge, the row is nothing beside eps)
    if ((!(squares < 1e37f) || squares < 1e-30f) && top[0] > 0.f && again[0] < 1e37f && eps < 1e30f) r = Size{scale, rsqrtf(again[0] * a.per_n + eps)};
  }
  return r;
}

// Rows of a workgroup of 256 threads (WAVES 1, 4) or 1024 (16)
template <int WAVES> __device__ __forceinline__ int rows_at_once(int lanes) { return WAVES == 1 ? 256 / lanes : 1; }

template <class T, int WAVES, int V, bool PACKED> __global__ __launch_bounds__(WAVES == 16 ? 1024 : 256) void k_norm(Args a) {
  __shared__ float lds[WAVES > 1 ? WAVES : 1];
  const int lanes = WAVES == 1 ? a.lanes : 64 * WAVES, lane = threadIdx.x % lanes;
  const int at_once = rows_at_once<WAVES>(lanes);
  float w[HELD<V>][LANE];
  if constexpr (V <= 2)
#pragma unroll
    for (int v = 0; v < V; ++v) weights<T>(a, (v * lanes + lane) * LANE, w[v]);
  for (long long first = (long long)blockIdx.x * at_once; first < a.rows; first += (long long)gridDim.x * at_once) {
    const long long row = first + threadIdx.x / lanes;
    const bool on = row < a.rows;
    float s[V][LANE], sum[1] = {0.f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = (v * lanes + lane) * LANE;
      read((const T *)a.x + row * a.ld_x + col, on ? a.n - col : 0, s[v]);
    }
    if (a.residual)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int col = (v * lanes + lane) * LANE;
        float r[LANE];
        read((const T *)a.residual + row * a.ld_r + col, on ? a.n - col : 0, r);
#pragma unroll
        for (int j = 0; j < LANE; ++j) s[v][j] += r[j];
        if (a.total && on) write((T *)a.total + row * a.ld_total + col, a.n - col, s[v]);
      }
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int j = 0; j < LANE; ++j) sum[0] = fmaf(s[v][j], s[v][j], sum[0]);
    over_row<WAVES, 1>(sum, a.lanes, lds);
    const Size size = size_of_row<WAVES>(s, sum[0], a, lds);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = (v * lanes + lane) * LANE;
      constexpr bool AGAIN = V > 2;
      float y[LANE];
      if constexpr (AGAIN) weights<T>(a, col, w[0]);
#pragma unroll
      for (int j = 0; j < LANE; ++j) y[j] = s[v][j] * size.scale * size.inv * w[AGAIN ? 0 : v][j];
      if constexpr (PACKED) {
        const int count = on ? a.n - col : 0;
        if (count < LANE)
#pragma unroll
          for (int j = 0; j < LANE; ++j) y[j] = j < count ? y[j] : 0.f; // (zeros of rows that are not there may have become NaN)
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < LANE; ++j) top = max(top, __float_as_uint(y[j]) & 0x7fffffffu);
        const Step step = block_step(top);
        if (count > 0) {
          write_codes(a.codes + row * a.n + col, count, y, step);
          if (col % SNN_PACK_BLOCK == 0) a.exps[row * ((a.n + SNN_PACK_BLOCK - 1) / SNN_PACK_BLOCK) + col / SNN_PACK_BLOCK] = step.byte;
        }
      } else if (on) write((T *)a.y + row * a.ld_y + col, a.n - col, y);
    }
  }
}

template <class T, int WAVES, int V> __global__ __launch_bounds__(WAVES == 16 ? 1024 : 256) void k_norm_back(Args a) {
  __shared__ float lds[WAVES > 1 ? 2 * WAVES : 4 * 64 * LANE];
  const int lanes = WAVES == 1 ? a.lanes : 64 * WAVES, lane = threadIdx.x % lanes;
  const int at_once = rows_at_once<WAVES>(lanes);
  constexpr bool AGAIN = V > 2;
  float w[HELD<V>][LANE], dw[V][LANE] = {};
  if constexpr (!AGAIN)
#pragma unroll
    for (int v = 0; v < V; ++v) weights<T>(a, (v * lanes + lane) * LANE, w[v]);
  for (long long first = (long long)blockIdx.x * at_once; first < a.rows; first += (long long)gridDim.x * at_once) {
    const long long row = first + threadIdx.x / lanes;
    const bool on = row < a.rows;
    float s[V][LANE], dy[V][LANE], sum[2] = {0.f, 0.f};
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = (v * lanes + lane) * LANE;
      read((const T *)a.x + row * a.ld_x + col, on ? a.n - col : 0, s[v]);
      read((const T *)a.dy + row * a.ld_y + col, on ? a.n - col : 0, dy[v]);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if constexpr (AGAIN) weights<T>(a, (v * lanes + lane) * LANE, w[0]);
#pragma unroll
      for (int j = 0; j < LANE; ++j) {
        sum[0] = fmaf(s[v][j], s[v][j], sum[0]);
        sum[1] = fmaf(s[v][j], dy[v][j] * w[AGAIN ? 0 : v][j], sum[1]);
      }
    }
    over_row<WAVES, 2>(sum, a.lanes, lds);
    const Size size = size_of_row<WAVES>(s, sum[0], a, lds);
    if (__any(size.scale != 1.f)) {
      float again[1] = {0.f};
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if constexpr (AGAIN) weights<T>(a, (v * lanes + lane) * LANE, w[0]);
#pragma unroll
        for (int j = 0; j < LANE; ++j) again[0] = fmaf(s[v][j] * size.scale, dy[v][j] * w[AGAIN ? 0 : v][j], again[0]);
      }
      over_row<WAVES, 1>(again, a.lanes, lds);
      sum[1] = again[0];
    }
    const float c = sum[1] * size.inv * a.per_n;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int col = (v * lanes + lane) * LANE;
      float dx[LANE];
      if constexpr (AGAIN) weights<T>(a, col, w[0]);
#pragma unroll
      for (int j = 0; j < LANE; ++j) {
        const float hat = s[v][j] * size.scale * size.inv;
        dx[j] = (dy[v][j] * w[AGAIN ? 0 : v][j] - hat * c) * size.inv * size.scale;
        if (on) dw[v][j] = fmaf(dy[v][j], hat, dw[v][j]);
      }
      if (on) {
        if (a.residual) {
          float r[LANE];
          read((const T *)a.residual + row * a.ld_r + col, a.n - col, r);
#pragma unroll
          for (int j = 0; j < LANE; ++j) dx[j] += r[j];
        }
        write((T *)a.dx + row * a.ld_dx + col, a.n - col, dx);
      }
    }
  }
  if (!a.sums) return;
  float *to = a.sums + (long long)blockIdx.x * a.n;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int col = (v * lanes + lane) * LANE;
    if constexpr (WAVES == 1) {
      // the rows of a wavefront, then those of the four
      for (int m = lanes; m < 64; m *= 2)
#pragma unroll
        for (int j = 0; j < LANE; ++j) dw[v][j] += __shfl_xor(dw[v][j], m);
      __syncthreads();
#pragma unroll
      for (int j = 0; j < LANE; ++j) lds[j * 256 + threadIdx.x] = dw[v][j];
      __syncthreads();
      if ((int)threadIdx.x >= lanes) continue;
#pragma unroll
      for (int j = 0; j < LANE; ++j) dw[v][j] = (lds[j * 256 + lane] + lds[j * 256 + lane + 64]) + (lds[j * 256 + lane + 128] + lds[j * 256 + lane + 192]);
    }
    write(to + col, a.n - col, dw[v]);
  }
}

// Rows of sums into one: a workgroup takes 32 columns, 8 rows at a time
template <class T> __global__ __launch_bounds__(256) void k_norm_dw(int count, int n, const float *sums, T *dw) {
  __shared__ float lds[8][32];
  const int col = blockIdx.x * 32 + threadIdx.x % 32, part = threadIdx.x / 32;
  float v[4] = {};
  if (col < n) {
    int i = part;
    for (; i + 24 < count; i += 32)
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] += sums[(long long)(i + 8 * k) * n + col];
    for (; i < count; i += 8) v[0] += sums[(long long)i * n + col];
  }
  lds[part][threadIdx.x % 32] = (v[0] + v[1]) + (v[2] + v[3]);
  __syncthreads();
  if (part || col >= n) return;
  float all = 0.f;
#pragma unroll
  for (int k = 0; k < 8; ++k) all += lds[k][threadIdx.x];
  dw[col] = (T)all;
}

// How rows of n elements are dealt to lanes
constexpr long long MOST_FORWARD = 1 << 20, MOST_BACK = 1024; // workgroups
struct Plan {
  int waves, vectors, lanes;
  unsigned groups; // workgroups
  Plan(long long rows, int n, bool bf16, bool back) {
    const int need = (n + LANE - 1) / LANE;
    // A workgroup has a row of more than 2048 elements (n is 2^15 at most: four vectors of a lane), and a shorter one where a wavefront would need four vectors, which
    // takes registers, or two and rows are few.  A wavefront and a workgroup to a row, us in a graph: 64 rows of 2048 in bf16 forward 5.1 and 2.8, 16384 rows
    // 53 and 47, backward 87 and 53; 4329 rows of 1501 in fp32 19.6 and 18.3, 33.4 and 28.6; but many rows in bf16 that leave lanes without elements or
    // begin between words, forward, 16384 of 1500 45 and 68, of 1930 53 and 62 (whole words: 16384 of 1536 31.4 and 30.6, of 1920 37.8 and 38.0).  Of 1024 in bf16 64 rows forward 3.6 and 2.8, 4329 rows 8.3 and 9.7; backward
    // 64 rows 6.4 and 5.1, 256 rows 6.6 and 7.4.
    const bool wide = need > 128 ? back || !bf16 || rows <= 2048 || (need > 240 && n % LANE == 0) : need > 64 && rows <= (back ? 128 : 1024);
    waves = need <= 256 && !wide ? 1 : need <= 1024 ? 4 : 16;
    lanes = 4;
    while (lanes < need && lanes < 64) lanes *= 2;
    const int of_row = waves == 1 ? lanes : 64 * waves;
    vectors = 1;
    while (vectors * of_row < need) vectors *= 2;
    const int at_once = waves == 1 ? 256 / lanes : 1;
    // (Backward a workgroup has four rows at least, where that leaves one for each compute unit: dw's rows of sums are fewer.  1024 rows of 2048 in bf16 13 us instead
    // of 20, of 4096 18 instead of 24)
    const long long all = (rows + at_once - 1) / at_once, four = waves == 1 ? all : rows / 4 > 256 ? rows / 4 : 256;
    const long long most = !back ? MOST_FORWARD : four < MOST_BACK ? four : MOST_BACK;
    groups = (unsigned)(all < most ? all : most);
    if (!groups) groups = 1;
  }
};

// MOST: vectors of a lane where a row has a wavefront
template <int MOST, class F> hipError_t with_plan(const Plan &p, F f) {
  auto v = [&](auto waves) {
    constexpr int W = decltype(waves)::value;
    if constexpr (W < 16)
      if (p.vectors == 1) return f(waves, std::integral_constant<int, 1>());
    if constexpr (W > 1 || MOST > 2)
      if (p.vectors == 4) return f(waves, std::integral_constant<int, 4>());
    f(waves, std::integral_constant<int, 2>());
  };
  if (p.waves == 1) v(std::integral_constant<int, 1>());
  else if (p.waves == 4) v(std::integral_constant<int, 4>());
  else v(std::integral_constant<int, 16>());
  return hipGetLastError();
}

template <class T> hipError_t forward(const Args &a, hipStream_t s) {
  const Plan p(a.rows, a.n, sizeof(T) == 2, false);
  Args b = a;
  b.lanes = p.lanes;
  return with_plan<sizeof(T) == 2 ? 4 : 2>(p, [&](auto waves, auto v) {
    constexpr int W = decltype(waves)::value, V = decltype(v)::value;
    if (b.codes) k_norm<T, W, V, true><<<p.groups, W == 16 ? 1024 : 256, 0, s>>>(b);
    else k_norm<T, W, V, false><<<p.groups, W == 16 ? 1024 : 256, 0, s>>>(b);
  });
}
template <class T> hipError_t backward(const Args &a, void *dw, hipStream_t s) {
  const Plan p(a.rows, a.n, sizeof(T) == 2, true);
  Args b = a;
  b.lanes = p.lanes;
  const hipError_t e = with_plan<2>(p, [&](auto waves, auto v) {
    constexpr int W = decltype(waves)::value, V = decltype(v)::value;
    k_norm_back<T, W, V><<<p.groups, W == 16 ? 1024 : 256, 0, s>>>(b);
  });
  if (e != hipSuccess || !dw) return e;
  k_norm_dw<T><<<(a.n + 31) / 32, 256, 0, s>>>((int)p.groups, a.n, a.sums, (T *)dw);
  return hipGetLastError();
}

} // namespace

size_t norm_workspace(const NormShape &p) { return sizeof(float) * Plan(p.rows, p.n, p.bf16, true).groups * p.n; }

hipError_t launch_norm(const NormShape &p, const void *x, const void *residual, const void *w, void *total, void *y, int8_t *codes, uint8_t *exps,
                       hipStream_t s) {
  Args a = {};
  a.x = x, a.residual = residual, a.w = w, a.total = total, a.y = y, a.codes = codes, a.exps = exps;
  a.rows = p.rows, a.ld_x = p.ld_x, a.ld_r = p.ld_residual, a.ld_total = p.ld_total, a.ld_y = p.ld_y;
  a.n = p.n, a.eps = p.eps, a.per_n = 1.f / p.n;
  return p.bf16 ? forward<__bf16>(a, s) : forward<float>(a, s);
}

hipError_t launch_norm_backward(const NormShape &p, const void *total, const void *w, const void *dy, const void *dtotal, void *dx, void *dw,
                                float *sums, hipStream_t s) {
  Args a = {};
  a.x = total, a.residual = dtotal, a.w = w, a.dy = dy, a.dx = dx, a.sums = dw ? sums : nullptr;
  a.rows = p.rows, a.ld_x = p.ld_total, a.ld_r = p.ld_dtotal, a.ld_y = p.ld_y, a.ld_dx = p.ld_dx;
  a.n = p.n, a.eps = p.eps, a.per_n = 1.f / p.n;
  return p.bf16 ? backward<__bf16>(a, dw, s) : backward<float>(a, dw, s);
}
