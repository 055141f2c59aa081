// Gated linear recurrence over [T][batch][n] and its backward pass.
//
//   a_t = sigmoid(z_t), b_t = sigmoid(-z_t);  h_t = a_t h_{t-1} + b_t x_t
//   g_t = dh_t + G_{t+1};  G_t = a_t g_t;  dx_t = b_t g_t;  dz_t = a_t b_t g_t (h_{t-1} - x_t)
//
// Every channel (b, i) is a recurrence of its own.  16 steps of one channel are a map h -> P h + B, P their product of a, and two maps in a
// row are one again: P = P1 P2, B = P2 B1 + B2.
// Digits: a and b are both computed, accurate relative to themselves, neither as 1 less the other, so that what a closed gate
// (a of 1e-4 and less) lets through of a large state or gradient keeps its digits, and so does the drive of an open one (b of 1e-4 and less).  A P next to one
// would lose those of its drive in its rounding, and over many steps that adds up: where P is the larger one a map holds Q = 1 - P
// instead, found by itself (Q = P2 Q1 + Q2), and is h -> h - Q h + B.
// A wavefront holds 16 steps of 64 lanes in registers, the eight wavefronts of a workgroup hold 128 steps in a row, exchange their maps through LDS and then know the state that each of them starts from: one read of z and x, one write of h.
// The state before every 128 steps is what the forward pass keeps; the backward pass gets h_{t-1} from there by
// the same exchange, beside that of the gradient, which runs the other way.
//
// What bounds it: memory, where there are channels or steps enough.  Forward, 4096 x 8 x 2048 in bf16: 80 us, 5.1 TB/s of z, x and h (a copy reaches
// 5.1); backward, 1000 x 32 x 1024 in fp32: 122 us, 5.4 TB/s; 32768 x 1 x 1024 in bf16: 99 us, of which 26 for the maps of its
// segments; from 8 bits, 4096 x 8 x 2048: 147 us, 3.7 TB/s, bound by the number of 1- and 2-byte loads.  One token of 64 x 2048: 2.8 us.
// Short sequences are bound by the latency of a tile, some 5 us.  Outputs that lie behind a sequence's end are zeros; its steps are read all the same.
#include "snn_ops.h"

namespace {

constexpr int STEPS = 16; // steps of a wavefront
constexpr int WAVES = SNN_GLR_INTERVAL / STEPS;

// VEC consecutive elements of a row as they are in memory
template <typename T, int VEC> struct Raw;
template <> struct Raw<float, 1> { typedef uint32_t type; };
template <> struct Raw<__bf16, 1> { typedef uint16_t type; };
template <> struct Raw<__bf16, 2> { typedef uint32_t type; };
template <> struct Raw<int8_t, 1> { typedef uint8_t type; };
template <> struct Raw<int8_t, 2> { typedef uint16_t type; };

template <typename T, int VEC> __device__ __forceinline__ void widen(typename Raw<T, VEC>::type r, float (&v)[VEC]) {
  if constexpr (sizeof(T) == 4) v[0] = __uint_as_float(r);
  else if constexpr (sizeof(T) == 2) {
    v[0] = __uint_as_float((uint32_t)r << 16);
    if constexpr (VEC == 2) v[1] = __uint_as_float(r & 0xffff0000u);
  } else {
    v[0] = (float)(int8_t)(r & 0xff);
    if constexpr (VEC == 2) v[1] = (float)((int16_t)r >> 8);
  }
}
template <typename T, int VEC> __device__ __forceinline__ typename Raw<T, VEC>::type narrow(const float (&v)[VEC]) {
  if constexpr (sizeof(T) == 4) return __float_as_uint(v[0]);
  else {
    uint32_t r = __builtin_bit_cast(uint16_t, (__bf16)v[0]); // to nearest, ties to even
    if constexpr (VEC == 2) r |= (uint32_t) __builtin_bit_cast(uint16_t, (__bf16)v[1]) << 16;
    return (typename Raw<T, VEC>::type)r;
  }
}

// sigmoid(z) and sigmoid(-z) from z / log(2), which is LARGEST at most (the reciprocal gives no numbers below 2^-126) or, EVERY, taken to be: there
// sigmoid(-z) is 2^-126.  sigmoid(z) below 2^-126 is 0.
constexpr float LOG2E = 1.44269504f, LARGEST = 126.f;
template <bool EVERY> __device__ __forceinline__ void gate(float z, float &a, float &b) {
  const float e = __builtin_amdgcn_exp2f(EVERY && z > LARGEST ? LARGEST : z); // (NaN stays)
  b = __builtin_amdgcn_rcpf(1.f + e);
  a = e * b;
}
__device__ __forceinline__ float nan_if_infinite(float x) { return fmaf(x, 0.f, x); }
// What a map retains: the smaller of P and Q, P as a negative number (its sign bit, as it may be 0)
__device__ __forceinline__ float share(float p, float q) { return p <= 0.5f ? -p : q; }
__device__ __forceinline__ bool is_p(float s) { return __float_as_int(s) < 0; }
// The map applied to h
__device__ __forceinline__ float mapped(float s, float h, float b) { return (is_p(s) ? 0.f : h) + fmaf(-s, h, b); }
// and two of them as one
__device__ __forceinline__ float both(float s, float r) {
  return share((is_p(s) ? -s : 1.f - s) * (is_p(r) ? -r : 1.f - r), fmaf(s, 1.f - r, r));
}

// f(whole) for a wavefront's steps, `whole` known to the compiler: whether every lane's sequence has all of them, as nearly always
template <bool B> struct Known { static constexpr bool value = B; };
template <class F> __device__ __forceinline__ void either(bool whole, F f) {
  if (whole) f(Known<true>());
  else f(Known<false>());
}
// f(ordinary) as if all steps were there and every value an ordinary one, and once more where steps are missing, or `found` has found values
// that are not (32768 x 1 x 1024 backwards: 99 us; with their tests in every step 106).  The second time begins from the elements as
// they were read: `again` makes them values that the compiler knows nothing of, as it would else keep in registers what the first time made of them.
template <class F, class G, class H> __device__ __forceinline__ void ordinarily(bool whole, F f, G found, H again) {
  if (whole) {
    f(Known<true>());
    whole = !__any(found());
  }
  if (!whole) {
    again();
    f(Known<false>());
  }
}
template <class R, int N> __device__ __forceinline__ void unknown(R (&r)[N]) {
#pragma unroll
  for (int j = 0; j < N; ++j) {
    uint32_t was = r[j];
    asm volatile("" : "+v"(was));
    r[j] = (R)was;
  }
}

__device__ __forceinline__ void lds_barrier() { // of the LDS alone: loads from memory stay in flight
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

struct Args {
  const void *z, *x, *dh;
  void *h, *dz, *dx;
  const uint8_t *ze, *xe;
  const int *lengths;
  const float *from;  // forward: h0, backward: dh_last (NULL: zeros)
  float *to;          // forward: h_last, backward: dh0 (NULL: not wanted)
  float *kept;        // [tiles][channels]
  float2 *maps;       // [segments + 1][channels], entry 0: `from`
  long long ld_z, ld_x, ld_h, ld_ze, ld_xe, ld_dz, ld_dx; // elements from one row (t, b) to the next
  int T, batch, n, channels, tiles, seg_tiles, segments;
};

// What a lane works on: VEC channels from c on
template <int VEC> struct Lane {
  int c, b, i, len;
  bool on;
  __device__ __forceinline__ Lane(const Args &a) {
    c = (blockIdx.x * 64 + threadIdx.x) * VEC;
    on = c < a.channels;
    if (!on) c = a.channels - VEC;
    b = c / a.n;
    i = c - b * a.n;
    len = a.T;
    if (a.lengths) len = min(max(a.lengths[b], 0), a.T);
  }
};

// An array [T][batch][ld] of elements of `size` bytes as a lane sees it.  Sixteen steps are reached from a 64-bit scalar address, a
// 32-bit scalar offset for the step (a step has 2^27 bytes at most) and a 32-bit one for the lane: no vector arithmetic for
// addresses.
struct Rows {
  char *base;
  unsigned step, at;
  __device__ __forceinline__ Rows(const void *p, int size, long long ld, int batch, int b, int i)
      : base((char *)p), step((unsigned)(size * ld * batch)), at((unsigned)(size * (b * ld + i))) {}
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t from(int t) const {
    return __builtin_amdgcn_make_buffer_rsrc(base + (unsigned long long)t * step, 0, (int)0xffffffff, 0x00020000);
  }
  // N steps from t0 on.  Steps at and past T are those of the last one again (and not used).
  template <typename R, int N> __device__ __forceinline__ void load(R (&r)[N], int t0, int T) const {
    const int first = min(t0, T - 1), last = T - 1 - first;
    const __amdgpu_buffer_rsrc_t from_first = from(first);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int at_step = (int)(min(j, last) * step);
      if constexpr (sizeof(R) == 4) r[j] = __builtin_amdgcn_raw_buffer_load_b32(from_first, (int)at, at_step, 0);
      else if constexpr (sizeof(R) == 2) r[j] = __builtin_amdgcn_raw_buffer_load_b16(from_first, (int)at, at_step, 0);
      else r[j] = __builtin_amdgcn_raw_buffer_load_b8(from_first, (int)at, at_step, 0);
    }
  }
  // Step j of those, not to be kept in the caches (results are not read again here, z and x are)
  template <typename R> __device__ __forceinline__ void store(const __amdgpu_buffer_rsrc_t &from_first, int j, R r) const {
    constexpr int NT = 2;
    if constexpr (sizeof(R) == 4) __builtin_amdgcn_raw_buffer_store_b32(r, from_first, (int)at, (int)(j * step), NT);
    else __builtin_amdgcn_raw_buffer_store_b16(r, from_first, (int)at, (int)(j * step), NT);
  }
};

// The state behind the first `count` segments (in the backward pass: G, from the end): their maps applied one after the other, their loads
// ahead of that.
template <int VEC> __device__ __forceinline__ void through(const Args &a, int c, int count, float (&h)[VEC]) {
#pragma unroll
  for (int v = 0; v < VEC; ++v) h[v] = a.maps[c + v].y;
#pragma unroll 16
  for (int k = 1; k <= count; ++k)
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      const float2 m = a.maps[(size_t)k * a.channels + c + v];
      h[v] = mapped(m.x, h[v], m.y);
    }
}

// The exponent bytes of a wavefront's 16 steps where its channels lie in four blocks at most: one load, lane l has step l / 4 and the
// block of number l % 4, and the lanes get theirs from there (512 x 64 x 2048: 118 us; a load for each step: 135 us).
struct Exponents {
  unsigned at; // of the block that the lane loads
  int slot;    // of the four, the one that the lane's channels are in
  __device__ __forceinline__ Exponents(const Rows &rows, int block) {
    const int lane = threadIdx.x;
    const int before = __shfl_up(block, 1); // (by every lane: none reads from one that takes no part)
    const uint64_t firsts = __ballot(lane == 0 || before != block); // (blocks of neighbouring lanes are the same or the next)
    slot = __popcll(firsts & (~0ull >> (63 - lane))) - 1;
    uint64_t m = firsts;
    const int want = min(lane & 3, __popcll(firsts) - 1);
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (i < want) m &= m - 1;
    at = (unsigned)__shfl((int)rows.at, __ffsll((unsigned long long)m) - 1);
  }
  __device__ __forceinline__ uint32_t load(const Rows &rows, int t0, int T) const {
    const int first = min(t0, T - 1), last = T - 1 - first;
    return __builtin_amdgcn_raw_buffer_load_b8(rows.from(first), (int)(at + (unsigned)min((int)threadIdx.x >> 2, last) * rows.step), 0, 0);
  }
  // the lane's own value of step j, from what the lanes that loaded the bytes made of them
  __device__ __forceinline__ float of(float loaded, int j) const {
    return __int_as_float(__builtin_amdgcn_ds_bpermute((4 * j + slot) * 4, __float_as_int(loaded)));
  }
};

// LDS of a workgroup: the maps of its wavefronts, for even and odd tiles (a tile's are read while the next one's are written)
template <int VEC, int N> struct Maps { float v[2][N][WAVES][VEC][64]; };

// Forward pass of one segment (blockIdx.y) of tiles.  MAPS: only the segment's map into maps[segment + 1], nothing stored; else the
// state at its beginning comes from the maps before it.  NW = 1: sequences of up to
// S steps, one wavefront each.
template <typename T, int VEC, int NW, int S, bool MAPS>
__global__ __launch_bounds__(64 * NW) void k_glr_forward(Args a) {
  __shared__ Maps<VEC, 2> maps;
  typedef typename Raw<T, VEC>::type R;
  const Lane<VEC> me(a);
  const Rows pz(a.z, sizeof(T), a.ld_z, a.batch, me.b, me.i), px(a.x, sizeof(T), a.ld_x, a.batch, me.b, me.i);
  const Rows ph(a.h, sizeof(T), a.ld_h, a.batch, me.b, me.i);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.y), seg = blockIdx.y;
  const int k0 = seg * a.seg_tiles, k1 = min(k0 + a.seg_tiles, a.tiles);
  float h[VEC], p[VEC]; // the state (MAPS: from zero), and the share that the segment so far retains
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    h[v] = 0.f;
    p[v] = 0.f;
    if (MAPS || a.segments == 1) {
      const float f = a.from && me.on ? a.from[me.c + v] : 0.f;
      if (!MAPS) h[v] = f;
      else if (seg == 0 && w == 0 && me.on) a.maps[me.c + v] = make_float2(0.f, f);
    }
  }
  if (!MAPS && a.segments > 1) through<VEC>(a, me.c, seg, h);
  // (a state that `to` may take the place of is read by every wavefront before the first one may write it)
#pragma unroll
  for (int v = 0; v < VEC; ++v) asm volatile("" ::"v"(h[v]));
  // (the map of a segment is put together from its end, its states are found from its beginning: what was read last is read first again)
  R rz[S], rx[S];
  constexpr int STRIDE = MAPS ? -NW * S : NW * S;
  int t0 = ((MAPS ? k1 - 1 : k0) * NW + w) * S;
  if (k0 < k1) {
    pz.load(rz, t0, a.T);
    px.load(rx, t0, a.T);
  }
  int n = k1 - k0, k = MAPS ? k1 - 1 : k0;
  for (; n > 0; --n, MAPS ? --k : ++k, t0 += STRIDE) {
    // Each step's state as P h + B of the one that these start from.  NW = 1: the smaller of a and b, a as a negative number, and the drive;
    // a state that goes from call to call is moved by h + b (x - h) where a is next to one.
    float P[S][VEC], B[S][VEC], Q[VEC], top = 0.f;
    const int live = me.len - t0; // steps of these 16 that the sequence has
    const bool whole = __all(live >= S);
    ordinarily(
        NW > 1 && whole,
        [&](auto known) {
          constexpr bool ORDINARY = decltype(known)::value;
#pragma unroll
          for (int j = 0; j < S; ++j) {
            float z[VEC], x[VEC];
            widen<T, VEC>(rz[j], z);
            widen<T, VEC>(rx[j], x);
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
              float keep, move;
              z[v] *= LOG2E;
              top = fmaxf(top, z[v]);
              gate<!ORDINARY>(z[v], keep, move);
              if (!ORDINARY) {
                x[v] = nan_if_infinite(x[v]);
                if (j >= live) keep = 1.f, move = x[v] = 0.f;
              }
              if (NW == 1) {
                P[j][v] = keep < move ? -keep : move;
                B[j][v] = x[v];
              } else {
                P[j][v] = j ? P[j - 1][v] * keep : keep;
                Q[v] = j ? fmaf(keep, Q[v], move) : move;
                B[j][v] = j ? fmaf(keep, B[j - 1][v], move * x[v]) : move * x[v];
              }
            }
          }
        },
        [&] {
          bool bad = top > LARGEST;
#pragma unroll
          for (int v = 0; v < VEC; ++v) bad |= !(P[S - 1][v] + fabsf(B[S - 1][v]) < INFINITY); // (once so, so to the end)
          return bad;
        },
        [&] {
          unknown(rz);
          unknown(rx);
        });
    if (n > 1) { // (ahead of the arithmetic above: 104 us instead of 84 for 4096 x 8 x 2048 in bf16)
      pz.load(rz, t0 + STRIDE, a.T);
      px.load(rx, t0 + STRIDE, a.T);
    }
    float start[VEC];
    if (NW > 1) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        maps.v[k & 1][0][w][v][threadIdx.x] = share(P[S - 1][v], Q[v]);
        maps.v[k & 1][1][w][v][threadIdx.x] = B[S - 1][v];
      }
      lds_barrier();
      if (!MAPS && w == 0 && a.kept && me.on)
#pragma unroll
        for (int v = 0; v < VEC; ++v) a.kept[(size_t)k * a.channels + me.c + v] = h[v];
#pragma unroll
      for (int v = 0; v < VEC; ++v) h[v] = nan_if_infinite(h[v]);
#pragma unroll
      for (int i = 0; i < WAVES; ++i)
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          const int wave = MAPS ? WAVES - 1 - i : i;
          const float Pi = maps.v[k & 1][0][wave][v][threadIdx.x], Bi = maps.v[k & 1][1][wave][v][threadIdx.x];
          if (MAPS) { // an earlier map, then the one so far
            h[v] = mapped(p[v], Bi, h[v]);
            p[v] = both(p[v], Pi);
          } else {
            if (i == w) start[v] = h[v];
            h[v] = mapped(Pi, h[v], Bi);
          }
        }
    } else {
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        start[v] = h[v];
        if (a.kept && me.on) a.kept[me.c + v] = h[v];
      }
    }
    if (!MAPS && me.on) {
      const __amdgpu_buffer_rsrc_t to = ph.from(t0);
      either(whole, [&](auto known) {
        constexpr bool ALL = decltype(known)::value;
#pragma unroll
        for (int j = 0; j < S; ++j) {
          float out[VEC];
#pragma unroll
          for (int v = 0; v < VEC; ++v) {
            const float state = NW > 1 ? fmaf(P[j][v], start[v], B[j][v]) : fmaf(P[j][v], B[j][v] - start[v], is_p(P[j][v]) ? B[j][v] : start[v]);
            if (NW == 1) start[v] = state;
            out[v] = ALL || j < live ? state : 0.f;
          }
          if (ALL || t0 + j < a.T) ph.store(to, j, narrow<T, VEC>(out));
        }
      });
      if (NW == 1)
#pragma unroll
        for (int v = 0; v < VEC; ++v) h[v] = start[v];
    }
  }
  if (w == 0 && me.on)
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      if (MAPS) a.maps[(size_t)(seg + 1) * a.channels + me.c + v] = make_float2(p[v], h[v]);
      else if (a.to && seg == a.segments - 1) a.to[me.c + v] = h[v];
    }
}

// Backward pass of one segment, last tile first.  P: the type of z and x in memory (int8_t: codes of blocks, with their exponent
// bytes; SHARED: a wavefront's channels lie in four blocks at most).  MAPS: only the map of the segment's gradient, G at its end -> G at its beginning, which takes no x and no state; segment s
// writes maps[segments - s].
template <typename T, typename P, int VEC, bool SHARED, bool MAPS>
__global__ __launch_bounds__(64 * WAVES) void k_glr_backward(Args a) {
  constexpr bool PACKED = sizeof(P) == 1;
  // dh is not loaded a tile ahead where registers would go to memory instead (512 x 64 x 2080: 149 us, 180 with the loads ahead)
  constexpr bool LATE = PACKED && VEC == 2 && !SHARED;
  __shared__ Maps<VEC, 3> maps;
  typedef typename Raw<T, VEC>::type R;
  const Lane<VEC> me(a);
  const Rows pz(a.z, sizeof(P), a.ld_z, a.batch, me.b, me.i), px(a.x, sizeof(P), a.ld_x, a.batch, me.b, me.i);
  const Rows pze(a.ze, 1, a.ld_ze, a.batch, me.b, me.i / SNN_PACK_BLOCK), pxe(a.xe, 1, a.ld_xe, a.batch, me.b, me.i / SNN_PACK_BLOCK);
  const Rows pd(a.dh, sizeof(T), a.ld_h, a.batch, me.b, me.i);
  const Rows pdz(a.dz, sizeof(T), a.ld_dz, a.batch, me.b, me.i), pdx(a.dx, sizeof(T), a.ld_dx, a.batch, me.b, me.i);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.y), seg = blockIdx.y + (MAPS ? 1 : 0);
  const int k0 = seg * a.seg_tiles, k1 = min(k0 + a.seg_tiles, a.tiles);
  float g[VEC], p[VEC]; // G (MAPS: from zero), and the share that the segment so far retains
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    g[v] = 0.f;
    p[v] = 0.f;
    if (MAPS || a.segments == 1) {
      const float f = a.from && me.on ? a.from[me.c + v] : 0.f;
      if (!MAPS) g[v] = f;
      else if (seg == 1 && w == 0 && me.on) a.maps[me.c + v] = make_float2(0.f, f);
    }
  }
  if (!MAPS && a.segments > 1) through<VEC>(a, me.c, a.segments - 1 - seg, g);
#pragma unroll
  for (int v = 0; v < VEC; ++v) asm volatile("" ::"v"(g[v])); // (as in the forward pass)
  typename Raw<P, VEC>::type rz[STEPS], rx[STEPS];
  R rd[STEPS];
  const int block = me.b * ((a.n + SNN_PACK_BLOCK - 1) / SNN_PACK_BLOCK) + me.i / SNN_PACK_BLOCK;
  const Exponents of_z(pze, SHARED ? block : 0), of_x(pxe, SHARED ? block : 0);
  uint32_t shared_z = 0, shared_x = 0;
  uint8_t ez[STEPS], ex[STEPS];
  float kept[VEC];
  auto fetch = [&](int k) {
    const int t = (k * WAVES + w) * STEPS;
    pz.load(rz, t, a.T);
    if (!LATE) pd.load(rd, t, a.T);
    if (!MAPS) px.load(rx, t, a.T);
    if (SHARED) {
      shared_z = of_z.load(pze, t, a.T);
      if (!MAPS) shared_x = of_x.load(pxe, t, a.T);
    } else if (PACKED) {
      pze.load(ez, t, a.T);
      if (!MAPS) pxe.load(ex, t, a.T);
    }
    if (!MAPS)
#pragma unroll
      for (int v = 0; v < VEC; ++v) kept[v] = a.kept[(size_t)k * a.channels + me.c + v];
  };
  // (as in the forward pass: the map of a segment is put together from its beginning)
  if (k0 < k1) fetch(MAPS ? k0 : k1 - 1);
  int n = k1 - k0, k = MAPS ? k0 : k1 - 1;
  for (; n > 0; --n, MAPS ? ++k : --k) {
    const int t0 = (k * WAVES + w) * STEPS;
    float keep[STEPS][VEC], move[STEPS][VEC], x[STEPS][VEC]; // a, b and b x
    R d[STEPS]; // (as it is in memory: half the registers)
    const int live = me.len - t0;
    const bool whole = __all(live >= STEPS);
    float product[VEC], Q[VEC], top = 0.f;
    if (LATE) pd.load(d, t0, a.T);
    // (a step is a power of two: its product with log2(e) is exact)
    float steps_z = __uint_as_float(shared_z << 23) * LOG2E, steps_x = __uint_as_float(shared_x << 23);
    ordinarily(
        whole,
        [&](auto known) {
          constexpr bool ORDINARY = decltype(known)::value;
#pragma unroll
          for (int j = 0; j < STEPS; ++j) {
            float z[VEC];
            widen<P, VEC>(rz[j], z);
            if (!MAPS) widen<P, VEC>(rx[j], x[j]);
            if (!LATE) d[j] = ORDINARY || j < live ? rd[j] : (R)0;
            const float step_z = SHARED ? of_z.of(steps_z, j) : PACKED ? __uint_as_float((uint32_t)ez[j] << 23) * LOG2E : LOG2E;
            const float step_x = MAPS ? 1.f : SHARED ? of_x.of(steps_x, j) : PACKED ? __uint_as_float((uint32_t)ex[j] << 23) : 1.f;
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
              z[v] *= step_z;
              top = fmaxf(top, z[v]);
              gate<!ORDINARY>(z[v], keep[j][v], move[j][v]);
              if (PACKED && !MAPS) x[j][v] *= step_x;
              if (!MAPS) x[j][v] *= move[j][v];
              if (!ORDINARY && j >= live) keep[j][v] = 1.f, move[j][v] = x[j][v] = 0.f;
              product[v] = j ? product[v] * keep[j][v] : keep[j][v];
              Q[v] = j ? fmaf(keep[j][v], Q[v], move[j][v]) : move[j][v];
            }
          }
        },
        [&] {
          bool bad = top > LARGEST;
#pragma unroll
          for (int v = 0; v < VEC; ++v) bad |= product[v] != product[v];
          return bad;
        },
        [&] {
          unknown(rz);
          if (!MAPS) unknown(rx);
          if (SHARED) asm volatile("" : "+v"(steps_z), "+v"(steps_x));
          else if (PACKED) {
            unknown(ez);
            if (!MAPS) unknown(ex);
          }
        });
    float B[VEC] = {}, G[VEC] = {}, h[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) h[v] = kept[v];
    if (LATE && !whole)
#pragma unroll
      for (int j = 0; j < STEPS; ++j) d[j] = j < live ? d[j] : (R)0;
    if (!MAPS)
#pragma unroll
      for (int j = 0; j < STEPS; ++j)
#pragma unroll
        for (int v = 0; v < VEC; ++v) B[v] = fmaf(keep[j][v], B[v], x[j][v]);
#pragma unroll
    for (int j = STEPS - 1; j >= 0; --j) {
      float dh[VEC];
      widen<T, VEC>(d[j], dh);
#pragma unroll
      for (int v = 0; v < VEC; ++v) G[v] = keep[j][v] * (dh[v] + G[v]);
    }
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      maps.v[k & 1][0][w][v][threadIdx.x] = share(product[v], Q[v]);
      maps.v[k & 1][1][w][v][threadIdx.x] = G[v];
      if (!MAPS) maps.v[k & 1][2][w][v][threadIdx.x] = B[v];
    }
    if (n > 1) fetch(MAPS ? k + 1 : k - 1); // (4096 x 8 x 2048 in bf16: 136 us; before the loops above 148)
    lds_barrier();
    float from[VEC];
#pragma unroll
    for (int i = 0; i < WAVES; ++i)
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const int wave = MAPS ? i : WAVES - 1 - i;
        const float Pi = maps.v[k & 1][0][wave][v][threadIdx.x], Gi = maps.v[k & 1][1][wave][v][threadIdx.x];
        if (MAPS) { // the map of later steps comes first
          g[v] = mapped(p[v], Gi, g[v]);
          p[v] = both(p[v], Pi);
        } else {
          if (wave == w) from[v] = g[v];
          g[v] = mapped(Pi, g[v], Gi);
        }
      }
    if (MAPS) continue;
#pragma unroll
    for (int i = 0; i < WAVES - 1; ++i)
#pragma unroll
      for (int v = 0; v < VEC; ++v)
        if (i < w) h[v] = mapped(maps.v[k & 1][0][i][v][threadIdx.x], h[v], maps.v[k & 1][2][i][v][threadIdx.x]);
#pragma unroll
    for (int j = 0; j < STEPS; ++j)
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const float off = fmaf(move[j][v], h[v], -x[j][v]); // b (h - x)
        h[v] = fmaf(keep[j][v], h[v], x[j][v]);
        x[j][v] = off;
      }
    if (me.on) {
      const __amdgpu_buffer_rsrc_t to_dz = pdz.from(t0), to_dx = pdx.from(t0);
      either(whole, [&](auto known) {
        constexpr bool ALL = decltype(known)::value;
#pragma unroll
        for (int j = STEPS - 1; j >= 0; --j) {
          float dh[VEC], dz[VEC], dx[VEC];
          widen<T, VEC>(d[j], dh);
#pragma unroll
          for (int v = 0; v < VEC; ++v) {
            const float g = dh[v] + from[v];
            dx[v] = move[j][v] * g;
            from[v] = keep[j][v] * g;
            dz[v] = from[v] * x[j][v];
            if (!ALL && j >= live) dz[v] = dx[v] = 0.f; // (whatever the state and its gradient)
          }
          if (ALL || t0 + j < a.T) {
            pdz.store(to_dz, j, narrow<T, VEC>(dz));
            pdx.store(to_dx, j, narrow<T, VEC>(dx));
          }
        }
      });
    }
  }
  if (w == 0 && me.on)
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      if (MAPS) a.maps[(size_t)(a.segments - seg) * a.channels + me.c + v] = make_float2(p[v], g[v]);
      else if (a.to && seg == 0) a.to[me.c + v] = g[v];
    }
}

// From WHOLE groups of channels on, one workgroup per group walks the whole sequence: z and x are read once.  Fewer would leave too many
// compute units without work: the sequence is then cut into segments so that there are WORKGROUPS in all, at the price of a launch before
// that finds the segments' maps (z and x, or dh, are read twice).  Forward passes of 4096 steps in bf16, one channel per lane, whole and cut:
// 128 groups 66 and 60 us, 160 groups 66 and 74 us, 192 groups 67 and 93 us (backward 106 and 86, 106 and 111, 124 and 149); in fp32 128 groups
// 77 and 104 us (backward 166 and 158).  16384 steps of 32 groups in bf16: 244 and 63 us.  A call of few steps is as long as its launches:
// 4 us more where it is cut (333 x 13 x 75 in fp32: 14 and 18 us), which whole sequences of more than five tiles cost as well.
constexpr int WHOLE = 160, WORKGROUPS = 512;
int groups_of(int channels, int vec) { return (channels + 64 * vec - 1) / (64 * vec); }
void cut(Args *a, int vec) {
  const int groups = groups_of(a->channels, vec);
  const int want = groups >= WHOLE ? 1 : (WORKGROUPS + groups - 1) / groups;
  a->tiles = (a->T + SNN_GLR_INTERVAL - 1) / SNN_GLR_INTERVAL;
  a->seg_tiles = a->tiles ? (a->tiles + want - 1) / want : 1;
  a->segments = a->tiles ? (a->tiles + a->seg_tiles - 1) / a->seg_tiles : 1;
}
// Two channels per lane in bf16, unless one per lane makes enough groups to walk the sequence whole and two do not.  4096 steps, one per lane and
// two: 16384 channels (whole, cut) 74 and 112 us, backward 135 and 179; 24576 channels (whole both) 146 and 138 us, backward 245 and 256; 8192
// channels (cut both) 60 and 60 us, backward 86 and 85.
bool two_per_lane(const GlrShape &p) {
  const int channels = p.batch * p.n;
  return p.bf16 && p.n % 2 == 0 && (groups_of(channels, 2) >= WHOLE || groups_of(channels, 1) < WHOLE);
}

Args shape_args(const GlrShape &p) {
  Args a = {};
  a.lengths = p.lengths;
  a.T = p.T;
  a.batch = p.batch;
  a.n = p.n;
  a.channels = p.batch * p.n;
  a.ld_z = p.ld_z;
  a.ld_x = p.ld_x;
  a.ld_dz = p.ld_dz;
  a.ld_dx = p.ld_dx;
  a.ld_h = p.ld_h;
  return a;
}

bool pairs(const void *p, size_t size, long long ld) { return (ld & 1) == 0 && (uintptr_t)p % (2 * size) == 0; }

template <typename T, int VEC> hipError_t forward(Args a, hipStream_t s) {
  const dim3 groups((a.channels + 64 * VEC - 1) / (64 * VEC));
  if (a.T <= STEPS) {
    a.tiles = a.T > 0;
    a.seg_tiles = a.segments = 1;
    if (a.T == 1) k_glr_forward<T, VEC, 1, 1, false><<<groups, 64, 0, s>>>(a);
    else k_glr_forward<T, VEC, 1, STEPS, false><<<groups, 64, 0, s>>>(a);
    return hipGetLastError();
  }
  cut(&a, VEC);
  if (a.segments > 1) {
    k_glr_forward<T, VEC, WAVES, STEPS, true><<<dim3(groups.x, a.segments - 1), dim3(64, WAVES), 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  k_glr_forward<T, VEC, WAVES, STEPS, false><<<dim3(groups.x, a.segments), dim3(64, WAVES), 0, s>>>(a);
  return hipGetLastError();
}

template <typename T, typename P, int VEC, bool SHARED = false> hipError_t backward(Args a, hipStream_t s) {
  const dim3 groups((a.channels + 64 * VEC - 1) / (64 * VEC));
  cut(&a, VEC);
  if (a.segments > 1) {
    k_glr_backward<T, P, VEC, SHARED, true><<<dim3(groups.x, a.segments - 1), dim3(64, WAVES), 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  k_glr_backward<T, P, VEC, SHARED, false><<<dim3(groups.x, a.segments), dim3(64, WAVES), 0, s>>>(a);
  return hipGetLastError();
}

} // namespace

size_t glr_workspace(const GlrShape &p) {
  Args a = shape_args(p);
  cut(&a, two_per_lane(p) ? 2 : 1); // (arrays not aligned to pairs take one per lane all the same: no more segments than with two)
  return a.segments > 1 ? (size_t)(a.segments + 1) * a.channels * sizeof(float2) : 0;
}

hipError_t launch_glr_forward(const GlrShape &p, const void *z, const void *x, const float *h0, void *h, float *h_last, float *kept,
                              void *work, hipStream_t s) {
  Args a = shape_args(p);
  a.z = z;
  a.x = x;
  a.from = h0;
  a.h = h;
  a.to = h_last;
  a.kept = kept;
  a.maps = (float2 *)work;
  if (!p.bf16) return forward<float, 1>(a, s);
  const bool two = two_per_lane(p) && pairs(z, 2, p.ld_z) && pairs(x, 2, p.ld_x) && pairs(h, 2, p.ld_h);
  return two ? forward<__bf16, 2>(a, s) : forward<__bf16, 1>(a, s);
}

hipError_t launch_glr_backward(const GlrShape &p, const GlrInputs &in, const float *kept, const void *dh, const float *dh_last,
                               void *dz, void *dx, float *dh0, void *work, hipStream_t s) {
  Args a = shape_args(p);
  a.z = in.z;
  a.x = in.x;
  a.kept = const_cast<float *>(kept);
  a.dh = dh;
  a.from = dh_last;
  a.dz = dz;
  a.dx = dx;
  a.to = dh0;
  a.maps = (float2 *)work;
  const bool packed = in.ze != nullptr;
  if (packed) {
    a.ze = in.ze;
    a.xe = in.xe;
    a.ld_z = in.ld_z;
    a.ld_x = in.ld_x;
    a.ld_ze = in.ld_ze;
    a.ld_xe = in.ld_xe;
  }
  // 64 channels in a row begin in four blocks at most if there is no more than one row's end among them, 128 if rows are multiples of that
  // (other even rows load a step's exponents one by one: 512 x 64 x 2080 takes 143 us, x 2048 136)
  const bool shared = p.n >= 64;
  if (!p.bf16) return !packed ? backward<float, float, 1>(a, s) : shared ? backward<float, int8_t, 1, true>(a, s) : backward<float, int8_t, 1>(a, s);
  const size_t size = packed ? 1 : 2;
  const bool two = two_per_lane(p) && pairs(in.z, size, a.ld_z) && pairs(in.x, size, a.ld_x) && pairs(dh, 2, p.ld_h) &&
                   pairs(dz, 2, p.ld_dz) && pairs(dx, 2, p.ld_dx);
  if (packed && two) return p.n % 128 == 0 ? backward<__bf16, int8_t, 2, true>(a, s) : backward<__bf16, int8_t, 2>(a, s);
  if (packed) return shared ? backward<__bf16, int8_t, 1, true>(a, s) : backward<__bf16, int8_t, 1>(a, s);
  return two ? backward<__bf16, __bf16, 2>(a, s) : backward<__bf16, __bf16, 1>(a, s);
}
