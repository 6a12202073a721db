// Gated linear recurrence over packed sequences, per channel:
//   L_t = c softplus(lam) sigm(r_t),  a_t = e^-L_t,  q_t = sqrt(1 - a_t^2),
//   h_t = a_t h_{t-1} + q_t sigm(i_t) x_t,
// and its gradient.  The recurrence is linear in h, so a stretch of frames acts
// on the state it starts from as h -> A h + S (A the product of its a_t, S its
// end from a zero state), and stretches compose:
//   (A1, S1) then (A2, S2)  =  (A1 A2, A2 S1 + S2).
// The gradient's carry g_t = a_t (dh_t + g_{t+1}) composes backwards in time with
// the same A.
//
// A workgroup holds 64 groups of V neighbouring channels (a lane each) and W
// consecutive stretches of TC frames (a wave each): a wave evaluates its
// stretch's a_t and inputs once, in registers, leaves (A, S) in LDS, composes
// those of the waves before it, and walks its stretch from the state so found;
// then the workgroup goes on to the next tile of W stretches.  Where the channels
// are too few to fill the chip, time is cut into spans of tiles, a workgroup
// each: one launch leaves every span's (A, S), the next one composes those of the
// spans before its own and runs.
#include "am_device.h"
#include "am_internal.h"

namespace am {
namespace {

constexpr int TC = GR_STRETCH, W = GR_WAVES;  // a tile is W stretches of TC frames
static_assert(TC * W == GR_TILE, "a tile of the saved states");

// V elements of a row as they lie in memory; they stay packed until they are used.
// Accesses go through a buffer descriptor of the frame (a scalar base) at a 32-bit
// offset of the lane; at the offset NONE, which lies past the descriptor's end,
// the hardware loads zeros and drops stores.
typedef __amdgpu_buffer_rsrc_t Frame;
constexpr uint32_t NONE = 0xffffffffu;
__device__ __forceinline__ Frame frame(const void* base, int64_t at) {
  char* p = const_cast<char*>(static_cast<const char*>(base)) + at;
  return __builtin_amdgcn_make_buffer_rsrc(p, 0, (int)0xfffffff0u, 0x00020000);  // raw, 32-bit elements
}

template <typename T, int V> struct Vec;
template <> struct Vec<float, 1> {
  uint32_t raw;
  __device__ __forceinline__ float at(int) const { return __uint_as_float(raw); }
  __device__ __forceinline__ void load(Frame f, uint32_t o) { raw = __builtin_amdgcn_raw_buffer_load_b32(f, o, 0, 0); }
  __device__ __forceinline__ static void store(Frame f, uint32_t o, const float (&v)[1]) {
    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v[0]), f, o, 0, 0);
  }
};
template <> struct Vec<bf16_t, 1> {
  uint16_t raw;
  __device__ __forceinline__ float at(int) const { return bf16_to_f32(raw); }
  __device__ __forceinline__ void load(Frame f, uint32_t o) { raw = __builtin_amdgcn_raw_buffer_load_b16(f, o, 0, 0); }
  __device__ __forceinline__ static void store(Frame f, uint32_t o, const float (&v)[1]) {
    __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, (__bf16)v[0]), f, o, 0, 0);
  }
};
template <> struct Vec<bf16_t, 2> {
  uint32_t raw;
  __device__ __forceinline__ float at(int k) const { return __uint_as_float(k ? raw & 0xffff0000u : raw << 16); }
  __device__ __forceinline__ void load(Frame f, uint32_t o) { raw = __builtin_amdgcn_raw_buffer_load_b32(f, o, 0, 0); }
  __device__ __forceinline__ static void store(Frame f, uint32_t o, const float (&v)[2]) {
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    // (one instruction, to nearest even)
    const bf16x2_t w = __builtin_convertvector((f32x2_t{v[0], v[1]}), bf16x2_t);
    __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, w), f, o, 0, 0);
  }
};

// What a frame's gates come to.  1 - a^2 is 1 - e^-y of y = 2L, from its series
// where the difference would cancel (five terms leave 4e-8 of it at 0.125, where
// the difference keeps 5e-7).  With L = 0 (a shut gate, or a frame past the
// sequence's end) the state passes unchanged, and L / q takes its limit 0.
struct Gates {
  float sr, a, q, Lq;  // sigm(r) (0 past the end), a, q and L / q
};
__device__ __forceinline__ Gates gates(float r, float rate, bool live) {
  Gates g;
  g.sr = live ? sigm(r) : 0.f;
  const float L = rate * g.sr, y = 2.f * L;
  g.a = __builtin_amdgcn_exp2f(-1.44269504f * L);
  float p = 1.f / 120.f;
  p = fmaf(p, -y, 1.f / 24.f);
  p = fmaf(p, -y, 1.f / 6.f);
  p = fmaf(p, -y, 0.5f);
  p = fmaf(p, -y, 1.f);
  const float q2 = y < 0.125f ? p * y : fmaf(-g.a, g.a, 1.f);
  const float rq = __builtin_amdgcn_rsqf(fmaxf(q2, 1.17549435e-38f));
  g.q = q2 * rq;
  g.Lq = L * rq;
  return g;
}

// max(v, 0) + log(1 + e), e = e^-|v|, the logarithm as 2 artanh(e / (2 + e)), whose
// series ends below 2^-24 of it (e / (2 + e) is at most 1 / 3).
__device__ __forceinline__ float softplus(float v) {
  const float e = __expf(-fabsf(v)), s = e / (2.f + e), z = s * s;
  float p = 1.f / 13.f;
  p = fmaf(p, z, 1.f / 11.f);
  p = fmaf(p, z, 1.f / 9.f);
  p = fmaf(p, z, 1.f / 7.f);
  p = fmaf(p, z, 1.f / 5.f);
  p = fmaf(p, z, 1.f / 3.f);
  return fmaxf(v, 0.f) + 2.f * fmaf(p * z, s, s);
}

// The schedule's tables, written by an earlier launch, for scalar loads.
typedef const __attribute__((address_space(4))) int32_t* Table;
__device__ __forceinline__ Table table(const int32_t* p) { return (Table)(uintptr_t)p; }

// This lane's channels and sequence, and the tiles of its workgroup.  A lane
// without channels has a sequence of no frames.
template <int V, bool RAGGED> struct Columns {
  int b, d, len;
  bool on;
  int tiles;     // of the workgroup's longest sequence (its first: they are sorted)
  int64_t st;    // place in a [B][H] matrix
  __device__ Columns(const GatedRecurrence& a, int lane) {
    const uint32_t per_row = (uint32_t)a.H / V, groups = a.B * per_row, g0 = blockIdx.x * 64;
    on = g0 + lane < groups;
    const uint32_t g = on ? g0 + lane : groups - 1;
    b = (int)(g / per_row);
    d = (int)(g - b * per_row) * V;
    st = (int64_t)b * a.H + d;
    len = on ? RAGGED ? a.lens[b] : a.T : 0;
    const int most = RAGGED ? table(a.lens)[g0 / per_row] : a.T;
    tiles = (most + GR_TILE - 1) / GR_TILE;
  }
};

// The first row of frame t (wave-uniform).
template <bool RAGGED>
__device__ __forceinline__ int64_t first_row(const GatedRecurrence& a, int t) {
  return RAGGED ? (int64_t)table(a.offs)[t < a.T ? t : a.T] : (int64_t)t * a.B;
}
// A lane's offset in the frames of a matrix of rows `ld` apart.
template <typename T, int V, bool RAGGED>
__device__ __forceinline__ uint32_t lane_offset(const Columns<V, RAGGED>& c, int64_t ld) {
  return (uint32_t)((c.b * ld + c.d) * (int)sizeof(T));
}

// A stretch's elements of K matrices of one row stride: frames t0 .. of the lane's
// sequence, zeros past its end.
template <bool RAGGED, typename T, int V, int N, int K>
__device__ __forceinline__ void fetch(const GatedRecurrence& a, const void* const (&m)[K], int64_t ld, int t0,
                                      const Columns<V, RAGGED>& c, Vec<T, V> (*const (&out)[K])[N]) {
  const uint32_t mine = lane_offset<T>(c, ld);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int64_t at = first_row<RAGGED>(a, t0 + j) * ld * (int)sizeof(T);
    const uint32_t o = t0 + j < c.len ? mine : NONE;
#pragma unroll
    for (int k = 0; k < K; ++k) (*out[k])[j].load(frame(m[k], at), o);
  }
}

// The state that a span starts from: `from` (or zero) through the stretches
// (A, S) of the spans first, first + step, ... before it.
template <int V, bool RAGGED>
__device__ __forceinline__ void span_start(const GatedRecurrence& a, const Columns<V, RAGGED>& c, const float* from,
                                           int first, int step, int count, float (&carry)[V]) {
  const int64_t BH = (int64_t)a.B * a.H;
#pragma unroll
  for (int v = 0; v < V; ++v) carry[v] = from ? from[c.st + v] : 0.f;
#pragma unroll 8
  for (int n = 0; n < count; ++n) {
    const float* p = a.spans_a + (first + n * step) * BH + c.st;
    const float* q = a.spans_s + (first + n * step) * BH + c.st;
#pragma unroll
    for (int v = 0; v < V; ++v) carry[v] = fmaf(p[v], carry[v], q[v]);
  }
}

// The composition of the stretches (A, S) of waves from, from + by, ... (count of
// them, wave-uniform) applied to a state.
template <int V, int N>
__device__ __forceinline__ void pass(const float (&A)[N][64][V], const float (&S)[N][64][V], int from, int by,
                                     int count, int lane, float (&state)[V]) {
#pragma unroll
  for (int n = 0; n < N - 1; ++n) {
    if (n >= count) break;
    const int s = from + n * by;
#pragma unroll
    for (int v = 0; v < V; ++v) state[v] = fmaf(A[s][lane][v], state[v], S[s][lane][v]);
    if (n & 1) asm volatile("" ::: "memory");  // (the later reads stay behind: registers)
  }
}

// AHEAD: several tiles, the next one's loads under the end of this one.
template <typename T, int V, bool RAGGED, bool AHEAD, int STRETCH, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 4) void gr_forward_kernel(GatedRecurrence a) {
  __shared__ float agg[2][2][WAVES][64][V];  // of tiles taken in turn: A, S of each stretch
  __shared__ float end[2][64][V];            // and the state at the tile's end
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Columns<V, RAGGED> c(a, lane);
  const int first = blockIdx.y * a.span_tiles;
  const int last = first + a.span_tiles < c.tiles ? first + a.span_tiles : c.tiles;
  if (first >= c.tiles && first > 0) return;
  Vec<T, V> x[STRETCH], r[STRETCH], i[STRETCH];
  auto take = [&](int k) {
    fetch<RAGGED, T, V, STRETCH, 3>(a, {a.r, a.i, a.x}, a.ld, k * GR_TILE + w * STRETCH, c, {&r, &i, &x});
  };
  if (first < last) take(first);
  float rate[V], h[V];
#pragma unroll
  for (int v = 0; v < V; ++v) rate[v] = a.c * softplus(a.lam[c.d + v]);
  span_start(a, c, a.h0, 0, 1, (int)blockIdx.y, h);
  const uint32_t mine = lane_offset<T>(c, a.H);
  for (int k = first; k < last; ++k) {
    const int t0 = k * GR_TILE + w * STRETCH;
    float av[STRETCH][V], u[STRETCH][V], A[V], S[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      A[v] = 1.f;
      S[v] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < STRETCH; ++j)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Gates g = gates(r[j].at(v), rate[v], t0 + j < c.len);
        av[j][v] = g.a;
        u[j][v] = g.q * sigm(i[j].at(v)) * x[j].at(v);
        A[v] *= g.a;
        S[v] = fmaf(g.a, S[v], u[j][v]);
      }
    if (AHEAD && k + 1 < last) take(k + 1);
    if constexpr (WAVES > 1) {
      float (&g)[2][WAVES][64][V] = agg[k & 1];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        g[0][w][lane][v] = A[v];
        g[1][w][lane][v] = S[v];
      }
      lds_barrier();
      if (AHEAD && k > first)
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = end[(k & 1) ^ 1][lane][v];
      if (a.saved && c.on && w == 0)
#pragma unroll
        for (int v = 0; v < V; ++v) a.saved[(int64_t)k * a.B * a.H + c.st + v] = h[v];
      pass<V, WAVES>(g[0], g[1], 0, 1, w, lane, h);
    }
#pragma unroll
    for (int j = 0; j < STRETCH; ++j) {
#pragma unroll
      for (int v = 0; v < V; ++v) h[v] = fmaf(av[j][v], h[v], u[j][v]);
      Vec<T, V>::store(frame(a.h, first_row<RAGGED>(a, t0 + j) * a.H * (int)sizeof(T)),
                       t0 + j < c.len ? mine : NONE, h);
    }
    if (AHEAD && w == WAVES - 1)
#pragma unroll
      for (int v = 0; v < V; ++v) end[k & 1][lane][v] = h[v];
  }
  if (a.hT && c.on && w == WAVES - 1 && last == c.tiles)
#pragma unroll
    for (int v = 0; v < V; ++v) a.hT[c.st + v] = h[v];
}

template <typename T, int V, bool RAGGED>
__global__ __launch_bounds__(64 * W, 4) void gr_backward_kernel(GatedRecurrence a) {
  __shared__ float agg[2][3][W][64][V];  // A, S and the carry's end from zero
  __shared__ float end[2][64][V];        // the carry at the tile's start
  __shared__ float lsum[W][64][V];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Columns<V, RAGGED> c(a, lane);
  const int64_t BH = (int64_t)a.B * a.H;
  const int first = blockIdx.y * a.span_tiles;
  const int last = first + a.span_tiles < c.tiles ? first + a.span_tiles : c.tiles;
  float rate[V], carry[V], dlam[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    rate[v] = a.c * softplus(a.lam[c.d + v]);
    dlam[v] = 0.f;
  }
  const int spans = (c.tiles + a.span_tiles - 1) / a.span_tiles;
  span_start(a, c, a.dhT, spans - 1, -1, spans - 1 - (int)blockIdx.y, carry);
  for (int k = last - 1; k >= first; --k) {
    const int t0 = k * GR_TILE + w * TC;
    Vec<T, V> x[TC], r[TC], i[TC], dh[TC];
    fetch<RAGGED, T, V, TC, 3>(a, {a.r, a.i, a.x}, a.ld, t0, c, {&r, &i, &x});
    fetch<RAGGED, T, V, TC, 1>(a, {a.dh}, a.lddh, t0, c, {&dh});
    float h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = a.saved[(int64_t)k * BH + c.st + v];
    // Of a frame: a, sigm(r), q sigm(i) (dx of its dv), x (1 - sigm(i)) (di of its
    // dx), and what its carry is multiplied by in the gradient of log a times log
    // a: v a L / q - L h_{t-1}, at first with the h of a stretch that starts from
    // zero.  (Past the end a = 1 and the rest is 0.)
    float av[TC][V], sr[TC][V], qs[TC][V], xs[TC][V], m[TC][V], A[V], S[V], D[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      A[v] = 1.f;
      S[v] = D[v] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < TC; ++j) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Gates g = gates(r[j].at(v), rate[v], t0 + j < c.len);
        const float si = sigm(i[j].at(v)), xv = x[j].at(v);
        av[j][v] = g.a;
        sr[j][v] = g.sr;
        qs[j][v] = g.q * si;
        xs[j][v] = fmaf(-xv, si, xv);
        m[j][v] = fmaf(si * xv, g.a * g.Lq, -rate[v] * g.sr * S[v]);
        // the carry's end: D + (product of the a before) times the rest
        A[v] *= g.a;
        D[v] = fmaf(A[v], dh[j].at(v), D[v]);
        S[v] = fmaf(g.a, S[v], qs[j][v] * xv);
      }
    }
    // (these and no others pass the barrier: what else would be kept, or moved
    // behind it, does not fit the registers)
#pragma unroll
    for (int j = 0; j < TC; ++j) {
      asm volatile("" : "+v"(dh[j].raw));
#pragma unroll
      for (int v = 0; v < V; ++v)
        asm volatile("" : "+v"(av[j][v]), "+v"(sr[j][v]), "+v"(qs[j][v]), "+v"(xs[j][v]), "+v"(m[j][v]));
    }
    float (&g)[3][W][64][V] = agg[k & 1];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      g[0][w][lane][v] = A[v];
      g[1][w][lane][v] = S[v];
      g[2][w][lane][v] = D[v];
    }
    lds_barrier();
    if (k + 1 < last)
#pragma unroll
      for (int v = 0; v < V; ++v) carry[v] = end[(k & 1) ^ 1][lane][v];
    pass<V, W>(g[0], g[1], 0, 1, w, lane, h);
    pass<V, W>(g[0], g[2], W - 1, -1, W - 1 - w, lane, carry);
#pragma unroll
    for (int j = 0; j < TC; ++j)  // (h: what the state at the stretch's start has come to)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        m[j][v] = fmaf(-rate[v] * sr[j][v], h[v], m[j][v]);
        h[v] *= av[j][v];
      }
    const uint32_t out = lane_offset<T>(c, a.ldd);
#pragma unroll
    for (int j = TC - 1; j >= 0; --j) {
      float dx[V], dr[V], di[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float d = dh[j].at(v) + carry[v];
        carry[v] = av[j][v] * d;
        const float e = carry[v] * m[j][v];
        dlam[v] += e;
        dr[v] = fmaf(-e, sr[j][v], e);
        dx[v] = d * qs[j][v];
        di[v] = dx[v] * xs[j][v];
      }
      const uint32_t o = t0 + j < c.len ? out : NONE;
      const int64_t at = first_row<RAGGED>(a, t0 + j) * a.ldd * (int)sizeof(T);
      Vec<T, V>::store(frame(a.dx, at), o, dx);
      Vec<T, V>::store(frame(a.dr, at), o, dr);
      Vec<T, V>::store(frame(a.di, at), o, di);
    }
    if (w == 0)
#pragma unroll
      for (int v = 0; v < V; ++v) end[k & 1][lane][v] = carry[v];
  }
  if (a.dh0 && c.on && w == 0 && first == 0)
#pragma unroll
    for (int v = 0; v < V; ++v) a.dh0[c.st + v] = carry[v];
#pragma unroll
  for (int v = 0; v < V; ++v) lsum[w][lane][v] = dlam[v];
  __syncthreads();
  if (c.on && w == 0)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float s = lsum[0][lane][v];
#pragma unroll
      for (int k = 1; k < W; ++k) s += lsum[k][lane][v];
      a.parts[blockIdx.y * BH + c.st + v] = s;
    }
}

// What a span does to the state that it starts from: (A, S) forward, (A, the
// carry's end) backward (BACK).  Each wave composes stretches that follow one
// another, then the waves' in order.
template <typename T, int V, bool RAGGED, bool BACK>
__global__ __launch_bounds__(64 * W) void gr_span_kernel(GatedRecurrence a) {
  __shared__ float agg[2][W][64][V];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Columns<V, RAGGED> c(a, lane);
  // what all spans start from, where no span's end (which may go to its place)
  // overwrites it before the others have read it
  const float* from = BACK ? a.dhT : a.h0;
  if (from && blockIdx.y == 0 && c.on && w == 0)
#pragma unroll
    for (int v = 0; v < V; ++v) a.start[c.st + v] = from[c.st + v];
  const int span = blockIdx.y + (BACK ? 1 : 0);  // (the first one's backward is not needed)
  const int first = span * a.span_tiles;
  const int last = first + a.span_tiles < c.tiles ? first + a.span_tiles : c.tiles;
  if (first >= last) return;
  const int mine = last - first;  // stretches a wave
  float rate[V], A[V], S[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    rate[v] = a.c * softplus(a.lam[c.d + v]);
    A[v] = 1.f;
    S[v] = 0.f;
  }
  const int begin = first * GR_TILE + w * mine * TC;
  for (int k = 0; k < mine; ++k) {
    const int t0 = begin + k * TC;
    Vec<T, V> x[TC], r[TC], i[TC], dh[TC];
    if constexpr (BACK) {
      fetch<RAGGED, T, V, TC, 1>(a, {a.r}, a.ld, t0, c, {&r});
      fetch<RAGGED, T, V, TC, 1>(a, {a.dh}, a.lddh, t0, c, {&dh});
    } else {
      fetch<RAGGED, T, V, TC, 3>(a, {a.r, a.i, a.x}, a.ld, t0, c, {&r, &i, &x});
    }
#pragma unroll
    for (int j = 0; j < TC; ++j)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Gates g = gates(r[j].at(v), rate[v], t0 + j < c.len);
        if constexpr (BACK) S[v] = fmaf(A[v] * g.a, dh[j].at(v), S[v]);
        else S[v] = fmaf(g.a, S[v], g.q * sigm(i[j].at(v)) * x[j].at(v));
        A[v] *= g.a;
      }
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    agg[0][w][lane][v] = A[v];
    agg[1][w][lane][v] = S[v];
  }
  __syncthreads();
  if (w != 0 || !c.on) return;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    float at = 1.f, st = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const int s = BACK ? W - 1 - k : k;
      st = fmaf(agg[0][s][lane][v], st, agg[1][s][lane][v]);
      at *= agg[0][s][lane][v];
    }
    const int64_t o = (int64_t)span * a.B * a.H + c.st + v;
    a.spans_a[o] = at;
    a.spans_s[o] = st;
  }
}

// dlam[d] = sigm(lam) / softplus(lam) times the sum of the rows of parts; their
// quotient tends to 1 where both vanish.
__global__ __launch_bounds__(1024) void gr_dlam_kernel(const float* __restrict__ parts, int64_t rows, int H,
                                                       const float* __restrict__ lam,
                                                       float* __restrict__ dlam) {
  __shared__ float sum[32][33];
  const float s = column_sum(parts, rows, H, sum);
  const int d = blockIdx.x * 32 + threadIdx.x;
  if (threadIdx.x >= 32 || d >= H) return;
  const float l = lam[d];
  dlam[d] = l < -20.f ? s : s * (1.f / (1.f + expf(-l))) / softplus(l);
}

// The packed offset of every frame, off_t = B_t t + (the sum of the lengths from
// sequence B_t on), and the lengths, where the kernels read them.
__global__ __launch_bounds__(256) void gr_schedule_kernel(GatedSchedule a) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t <= a.T && a.last) {
    int lo = 0, hi = a.B;  // B_t: the first sequence of at most t frames
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      const int len = mid < a.first ? a.lens[mid] : a.len[mid - a.first];
      if (len > t) lo = mid + 1; else hi = mid;
    }
    const int tail = lo == a.B ? 0 : lo < a.first ? a.tails[lo] : a.tail[lo - a.first];
    a.offs[t] = lo * t + tail;
  }
  if (t < a.count) {
    a.lens[a.first + t] = a.len[t];
    a.tails[a.first + t] = a.tail[t];
  }
}

// Workgroups that fill the chip: three of 8 waves a CU.
constexpr int64_t FULL = 768;

template <typename T, int V, bool RAGGED>
hipError_t launch(GatedRecurrence a, bool forward, hipStream_t s) {
  const int64_t groups = ((int64_t)a.B * (a.H / V) + 63) / 64;
  const int tiles = (a.T + GR_TILE - 1) / GR_TILE;
  // one frame and nothing to keep of it: a wave does without a tile
  if (forward && a.T == 1 && !a.saved) {
    a.span_tiles = 1;
    hipLaunchKernelGGL((gr_forward_kernel<T, V, RAGGED, false, 1, 1>), dim3((unsigned)groups), dim3(64), 0, s, a);
    return hipGetLastError();
  }
  const int spans = gated_spans(a.T, groups);
  a.span_tiles = tiles > 0 ? (tiles + spans - 1) / spans : 1;
  const dim3 grid((unsigned)groups, (unsigned)(tiles > 0 ? (tiles + a.span_tiles - 1) / a.span_tiles : 1));
  if (grid.y > 1) {
    const dim3 most(grid.x, grid.y - 1);
    if (forward) hipLaunchKernelGGL((gr_span_kernel<T, V, RAGGED, false>), most, dim3(64 * W), 0, s, a);
    else hipLaunchKernelGGL((gr_span_kernel<T, V, RAGGED, true>), most, dim3(64 * W), 0, s, a);
    if (a.h0) a.h0 = a.start;
    if (a.dhT) a.dhT = a.start;
  }
  if (forward) {
    if (a.span_tiles > 1) hipLaunchKernelGGL((gr_forward_kernel<T, V, RAGGED, true, TC, W>), grid, dim3(64 * W), 0, s, a);
    else hipLaunchKernelGGL((gr_forward_kernel<T, V, RAGGED, false, TC, W>), grid, dim3(64 * W), 0, s, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((gr_backward_kernel<T, V, RAGGED>), grid, dim3(64 * W), 0, s, a);
  hipLaunchKernelGGL(gr_dlam_kernel, dim3((unsigned)((a.H + 31) / 32)), dim3(1024), 0, s, a.parts,
                     (int64_t)a.B * grid.y, a.H, a.lam, a.dlam);
  return hipGetLastError();
}

// Two bf16 channels a lane where every row starts on a multiple of 4 bytes.
bool paired(const GatedRecurrence& a) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.r) |
                       reinterpret_cast<uintptr_t>(a.i) | reinterpret_cast<uintptr_t>(a.h) |
                       reinterpret_cast<uintptr_t>(a.dh) | reinterpret_cast<uintptr_t>(a.dx) |
                       reinterpret_cast<uintptr_t>(a.dr) | reinterpret_cast<uintptr_t>(a.di);
  return at % 4 == 0 && (a.H | a.ld | a.lddh | a.ldd) % 2 == 0;
}

template <typename T, int V>
hipError_t shaped(const GatedRecurrence& a, bool forward, hipStream_t s) {
  return a.lens ? launch<T, V, true>(a, forward, s) : launch<T, V, false>(a, forward, s);
}

hipError_t route(const GatedRecurrence& a, bool bf16, bool forward, hipStream_t s) {
  if (!bf16) return shaped<float, 1>(a, forward, s);
  return paired(a) ? shaped<bf16_t, 2>(a, forward, s) : shaped<bf16_t, 1>(a, forward, s);
}

}  // namespace

hipError_t gated_schedule(GatedSchedule a, const int32_t* lengths, hipStream_t s) {
  int64_t after = 0;  // frames of the sequences from a place on
  for (int b = 0; b < a.B; ++b) after += lengths[b];
  for (a.first = 0; a.first < a.B; a.first += a.count) {
    a.count = a.B - a.first < GatedSchedule::MAX ? a.B - a.first : GatedSchedule::MAX;
    for (int k = 0; k < a.count; ++k) {
      a.len[k] = lengths[a.first + k];
      a.tail[k] = (int32_t)after;
      after -= lengths[a.first + k];
    }
    a.last = a.first + a.count == a.B;
    const int n = a.last && a.T + 1 > a.count ? a.T + 1 : a.count;
    hipLaunchKernelGGL(gr_schedule_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

hipError_t gated_forward(const GatedRecurrence& a, bool bf16, hipStream_t s) {
  return route(a, bf16, true, s);
}

hipError_t gated_backward(const GatedRecurrence& a, bool bf16, hipStream_t s) {
  return route(a, bf16, false, s);
}

int gated_spans(int T, int64_t groups) {
  const int tiles = (T + GR_TILE - 1) / GR_TILE;
  const int64_t want = groups * 2 > FULL ? 1 : FULL / groups;
  return (int)(want < tiles ? want : tiles > 0 ? tiles : 1);
}

}  // namespace am
