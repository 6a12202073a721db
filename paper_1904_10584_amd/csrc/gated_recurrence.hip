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
// are too few to fill the chip, every tile is a workgroup of its own and they are
// linked through memory (see LINK).
//
// Bounds, bf16: 8 bytes an element forward and 14 backward against 42 and 63 vector
// instructions (three exponentials, two reciprocals and a root among them: 48 and 69
// issue slots counted), which take less time than the bytes and overlap them in part.
// 16384 frames x 768 (64 a sequence): forward 26 us (3.9 TB/s, 15 us of vector
// instructions), backward 41 us (4.3 TB/s, 22 us).  128 utterances of 200 to 1500
// frames x 768: 170 us (4.0 TB/s, 97 us of vector instructions) and 266 us (4.5 TB/s,
// 140 us).  Stores past the caches make these 5 % faster by themselves and what reads
// their results next slower by more (forward with the norm after it: 58 -> 60 us): not
// taken.
#include "am_device.h"
#include "am_internal.h"
#include "poll_budget.h"

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
  __device__ Columns(const GatedRecurrence& a, int lane, uint32_t group, int tile) {
    const uint32_t per_row = (uint32_t)a.H / V, groups = a.B * per_row, g0 = group * 64;
    on = g0 + lane < groups;
    const uint32_t g = on ? g0 + lane : groups - 1;
    b = (int)(g / per_row);
    d = (int)(g - b * per_row) * V;
    st = (int64_t)b * a.H + d;
    len = on ? RAGGED ? a.lens[b] : a.T : 0;
    const int most = RAGGED ? table(a.lens)[g0 / per_row] : a.T;
    tiles = (most + tile - 1) / tile;
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

// V neighbouring fp32 values.
template <int V> __device__ __forceinline__ void fetch_state(Frame f, uint32_t o, float (&out)[V]) {
  static_assert(V == 1 || V == 2, "a word or two");
  if constexpr (V == 1) {
    out[0] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(f, o, 0, 0));
  } else {
    const auto w = __builtin_amdgcn_raw_buffer_load_b64(f, o, 0, 0);
    out[0] = __uint_as_float(w[0]);
    out[1] = __uint_as_float(w[1]);
  }
}

// Tiles as workgroups of their own.  A workgroup draws the next tile of its
// channels from a counter, so it only ever waits for tiles that others have drawn
// before, whose workgroups run already: no wait depends on what is resident or in
// which order it was launched.  LINK tiles make a block.  A tile publishes its
// (A, S) as soon as it is evaluated and composes those of the tiles before it in
// its block; the block's last tile publishes the state that the next block starts
// from.  So the chain through memory has a link for LINK tiles, and what is
// composed with what does not depend on who comes first: the same bits each time.
// All of it is stored and loaded past the caches that XCDs do not share
// (agent-scope atomics).  A tile's (A, S) are followed by its flag; a state carries
// its flag in its upper half.  Polls are bounded; one that runs out (a stalled
// device) sets the workspace's time-out flag and goes on with NaN.
// (One sequence of 40001 frames x 1536, forward: LINK = 4, 8, 12: 134, 135, 136 us.
// Without the links it would take 102, the time of its bytes: the tiles of a group
// wait for one another at the same time, with nothing left to load.)
constexpr int LINK = 8;
constexpr unsigned POLLS = 1u << 22;
constexpr int TICKET_LINE = 64;  // words: a counter to itself

__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  return (uint64_t)__float_as_uint(lo) | ((uint64_t)__float_as_uint(hi) << 32);
}
template <typename U> __device__ __forceinline__ U peek(const U* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <typename U> __device__ __forceinline__ void post(U* p, U v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The state that tile n (of `tiles`, in the order of the recurrence) starts from.
// (A, S): its stretches', `start` what tile 0 starts from, pre and first LDS.  The
// waves share the work, so that its round trips to memory run side by side: the
// last one publishes, the one before it waits for the block's start, and each of
// the first ones composes two of the block's tiles before this one.
template <bool BACK, int V, bool RAGGED>
__device__ __forceinline__ void linked(const GatedRecurrence& a, const Columns<V, RAGGED>& c, int lane, int w,
                                       int n, int tiles, const float (&A)[W][64][V], const float (&S)[W][64][V],
                                       const float (&start)[V], float (&pre)[2][W][64][V], float (&first)[64][V],
                                       float (&state)[V]) {
  static_assert(LINK <= 2 * (W - 2), "two tiles a wave");
  constexpr int PUBLISHES = W - 1, WAITS = W - 2;
  const int64_t BH = (int64_t)a.B * a.H;
  const int block = n / LINK, place = n % LINK;
  const bool more = n + 1 < tiles;
  uint32_t* flags = a.flags + (int64_t)blockIdx.x * a.most_tiles + (n - place);
  uint64_t* parts = a.stretches + (int64_t)(n - place) * BH + c.st;
  float ta[V], ts[V];
  if (w == PUBLISHES && more) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      ta[v] = 1.f;
      ts[v] = 0.f;
    }
#pragma unroll
    for (int q = 0; q < W; ++q)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int s = BACK ? W - 1 - q : q;
        ts[v] = fmaf(A[s][lane][v], ts[v], S[s][lane][v]);
        ta[v] *= A[s][lane][v];
        if (v + 1 == V && (q & 1)) asm volatile("" ::: "memory");
      }
    if (place + 1 < LINK) {
      if (c.on)
#pragma unroll
        for (int v = 0; v < V; ++v) post(parts + place * BH + v, pair(ta[v], ts[v]));
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");  // (the stores have arrived)
      __builtin_amdgcn_s_waitcnt(0);
      if (lane == 0) post(flags + place, 1u);
    }
  }
  float pa[V], ps[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    pa[v] = 1.f;
    ps[v] = 0.f;
  }
  PollBudget<POLLS> budget;
  const int j0 = 2 * w, j1 = 2 * w + 1 < place ? 2 * w + 1 : 2 * w;
  if (j0 < place && w < WAITS) {
    bool lost = false;
    while (!__all(peek(flags + (lane & 1 ? j1 : j0)) != 0)) {
      if (budget.spent()) {
        lost = true;
        *a.err = 1;
        break;
      }
      __builtin_amdgcn_s_sleep(1);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
    uint64_t p0[V], p1[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      p0[v] = peek(parts + j0 * BH + v);
      p1[v] = peek(parts + j1 * BH + v);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      pa[v] = lost ? __builtin_nanf("") : __uint_as_float((uint32_t)p0[v]);
      ps[v] = __uint_as_float((uint32_t)(p0[v] >> 32));
      if (j1 > j0) {
        const float a1 = __uint_as_float((uint32_t)p1[v]), s1 = __uint_as_float((uint32_t)(p1[v] >> 32));
        ps[v] = fmaf(a1, ps[v], s1);
        pa[v] *= a1;
      }
    }
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    pre[0][w][lane][v] = pa[v];
    pre[1][w][lane][v] = ps[v];
  }
  if (w == WAITS) {
    float from[V];
#pragma unroll
    for (int v = 0; v < V; ++v) from[v] = start[v];
    if (block > 0) {
      const uint64_t* at = a.states + (int64_t)block * BH + c.st;
      budget.begin();
      for (;;) {
        bool here = true;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const uint64_t p = peek(at + v);
          from[v] = __uint_as_float((uint32_t)p);
          here = here && (p >> 32) != 0;
        }
        if (__all(here)) break;
        if (budget.spent()) {
          *a.err = 1;
#pragma unroll
          for (int v = 0; v < V; ++v) from[v] = __builtin_nanf("");
          break;
        }
        __builtin_amdgcn_s_sleep(1);
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) first[lane][v] = from[v];
  }
  lds_barrier();
#pragma unroll
  for (int v = 0; v < V; ++v) state[v] = first[lane][v];
#pragma unroll
  for (int s = 0; s < LINK / 2; ++s) {
    if (2 * s >= place) break;
#pragma unroll
    for (int v = 0; v < V; ++v) state[v] = fmaf(pre[0][s][lane][v], state[v], pre[1][s][lane][v]);
    if (s & 1) asm volatile("" ::: "memory");
  }
  if (w == PUBLISHES && more && place + 1 == LINK && c.on)
#pragma unroll
    for (int v = 0; v < V; ++v)
      post(a.states + (int64_t)(block + 1) * BH + c.st + v,
           (uint64_t)__float_as_uint(fmaf(ta[v], state[v], ts[v])) | ((uint64_t)1 << 32));
}

// The tile that this workgroup draws (every wave calls this).
__device__ __forceinline__ int draw_tile(const GatedRecurrence& a) {
  __shared__ int drawn;
  if (threadIdx.x == 0)
    drawn = (int)__hip_atomic_fetch_add(a.tickets + (int64_t)blockIdx.x * TICKET_LINE, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(drawn);
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

// The 64 groups of channels of a workgroup.  Sequences are sorted by length, and
// workgroups 256 apart tend to share a CU: every second 256 are taken from their
// end, so that long and short ones meet (128 utterances of 200 to 1500 frames x 768:
// forward 180 -> 170 us).
template <bool RAGGED> __device__ __forceinline__ uint32_t group_of(uint32_t block, uint32_t blocks) {
  if (!RAGGED || !(block >> 8 & 1)) return block;
  const uint32_t first = block & ~255u, last = first + 255 < blocks ? first + 255 : blocks - 1;
  return first + (last - block);
}

// How a workgroup takes tiles: the one there is, all of its channels' in turn (the
// next one's loads under the end of this one), or one that it draws.
enum Tiles { ONE, IN_TURN, LINKED };

template <typename T, int V, bool RAGGED, Tiles MODE, int STRETCH, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 4) void gr_forward_kernel(GatedRecurrence a) {
  constexpr int TILE = STRETCH * WAVES;
  __shared__ float agg[2][2][WAVES][64][V];  // of tiles taken in turn: A, S of each stretch
  __shared__ float end[2][64][V];            // and the state at the tile's end, or its block's start (LINKED)
  __shared__ float pre[MODE == LINKED ? 2 : 1][MODE == LINKED ? W : 1][64][V];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Columns<V, RAGGED> c(a, lane, group_of<RAGGED && MODE == IN_TURN>(blockIdx.x, gridDim.x), TILE);
  if (MODE != LINKED && a.err && blockIdx.x == 0 && threadIdx.x == 0) *a.err = 0;
  const int first = MODE == LINKED ? draw_tile(a) : 0;
  if (MODE == LINKED && first >= c.tiles && first > 0) return;
  const int last = MODE == IN_TURN ? c.tiles : c.tiles > first ? first + 1 : first;
  Vec<T, V> x[STRETCH], r[STRETCH], i[STRETCH];
  auto take = [&](int k) {
    fetch<RAGGED, T, V, STRETCH, 3>(a, {a.r, a.i, a.x}, a.ld, k * TILE + w * STRETCH, c, {&r, &i, &x});
  };
  if (first < last) take(first);
  float rate[V], h[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    rate[v] = a.c * softplus(a.lam[c.d + v]);
    h[v] = a.h0 && (MODE != LINKED || first < LINK) ? a.h0[c.st + v] : 0.f;
  }
  const uint32_t mine = lane_offset<T>(c, a.H);
  auto tile = [&](int k) {
    const int t0 = k * TILE + w * STRETCH;
    float av[STRETCH][V], u[STRETCH][V], A[V], S[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      A[v] = 1.f;
      S[v] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < STRETCH; ++j) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Gates g = gates(r[j].at(v), rate[v], t0 + j < c.len);
        av[j][v] = g.a;
        u[j][v] = g.q * sigm(i[j].at(v)) * x[j].at(v);
        A[v] *= g.a;
        S[v] = fmaf(g.a, S[v], u[j][v]);
      }
    }
    if (MODE == IN_TURN && k + 1 < last) take(k + 1);
    if constexpr (WAVES > 1) {
      float (&g)[2][WAVES][64][V] = agg[k & 1];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        g[0][w][lane][v] = A[v];
        g[1][w][lane][v] = S[v];
      }
      // (hT may be h0: every wave has read its start before any wave of the workgroup,
      // or one that waits for this tile, can be done.  The barrier itself waits for LDS
      // alone; using the register here waits for the load.)
#pragma unroll
      for (int v = 0; v < V; ++v) asm volatile("" ::"v"(h[v]));
      lds_barrier();
      if constexpr (MODE == LINKED) {
        float start[V];
#pragma unroll
        for (int v = 0; v < V; ++v) start[v] = h[v];
        linked<false>(a, c, lane, w, k, c.tiles, g[0], g[1], start, pre, end[0], h);
      } else if (MODE == IN_TURN && k > first) {
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = end[(k & 1) ^ 1][lane][v];
      }
      pass<V, WAVES>(g[0], g[1], 0, 1, w, lane, h);
      if (a.saved && c.on && t0 % GR_TILE == 0 && t0 < a.T)
#pragma unroll
        for (int v = 0; v < V; ++v) a.saved[(int64_t)(t0 / GR_TILE) * a.B * a.H + c.st + v] = h[v];
    }
#pragma unroll
    for (int j = 0; j < STRETCH; ++j) {
#pragma unroll
      for (int v = 0; v < V; ++v) h[v] = fmaf(av[j][v], h[v], u[j][v]);
      Vec<T, V>::store(frame(a.h, first_row<RAGGED>(a, t0 + j) * a.H * (int)sizeof(T)),
                       t0 + j < c.len ? mine : NONE, h);
    }
    if (MODE == IN_TURN && w == WAVES - 1)
#pragma unroll
      for (int v = 0; v < V; ++v) end[k & 1][lane][v] = h[v];
  };
  if constexpr (MODE == IN_TURN)
    for (int k = first; k < last; ++k) tile(k);
  else if (first < last)
    tile(first);
  if (a.hT && c.on && w == WAVES - 1 && last == c.tiles)
#pragma unroll
    for (int v = 0; v < V; ++v) a.hT[c.st + v] = h[v];
}

template <typename T, int V, bool RAGGED, Tiles MODE>
__global__ __launch_bounds__(64 * W, 4) void gr_backward_kernel(GatedRecurrence a) {
  __shared__ float agg[2][3][W][64][V];  // A, S and the carry's end from zero
  __shared__ float end[2][64][V];        // the carry at the tile's start, or at its block's end (LINKED)
  __shared__ float pre[MODE == LINKED ? 2 : 1][MODE == LINKED ? W : 1][64][V];
  __shared__ float lsum[W][64][V];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Columns<V, RAGGED> c(a, lane, group_of<RAGGED && MODE == IN_TURN>(blockIdx.x, gridDim.x), GR_TILE);
  const int64_t BH = (int64_t)a.B * a.H;
  const int drawn = MODE == LINKED ? draw_tile(a) : 0;  // (from the last tile down)
  const int last = MODE == LINKED ? (drawn < c.tiles ? c.tiles - drawn : 0) : c.tiles;
  const int first = MODE == LINKED ? (last > 0 ? last - 1 : 0) : 0;
  float rate[V], carry[V], dlam[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    rate[v] = a.c * softplus(a.lam[c.d + v]);
    carry[v] = a.dhT && (MODE != LINKED || drawn < LINK) ? a.dhT[c.st + v] : 0.f;
    dlam[v] = 0.f;
  }
  auto tile = [&](int k) {
    const int t0 = k * GR_TILE + w * TC;
    Vec<T, V> x[TC], r[TC], i[TC], dh[TC];
    fetch<RAGGED, T, V, TC, 3>(a, {a.r, a.i, a.x}, a.ld, t0, c, {&r, &i, &x});
    fetch<RAGGED, T, V, TC, 1>(a, {a.dh}, a.lddh, t0, c, {&dh});
    // (zeros for tiles that the lane's sequence does not have: the forward pass may
    // have grouped channels otherwise and saved nothing there.  Sequences of one length
    // have the same tiles.)
    float h[V];
    if constexpr (RAGGED) {
      fetch_state<V>(frame(a.saved, k * BH * 4), k * GR_TILE < c.len ? (uint32_t)c.st * 4 : NONE, h);
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) h[v] = a.saved[(int64_t)k * BH + c.st + v];
    }
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
    // (dh0 may be dhT: as for h0 in the forward pass)
#pragma unroll
    for (int v = 0; v < V; ++v) asm volatile("" ::"v"(carry[v]));
    lds_barrier();
    if constexpr (MODE == LINKED) {
      float start[V];
#pragma unroll
      for (int v = 0; v < V; ++v) start[v] = carry[v];
      linked<true>(a, c, lane, w, drawn, c.tiles, g[0], g[2], start, pre, end[0], carry);
    } else if (k + 1 < last) {
#pragma unroll
      for (int v = 0; v < V; ++v) carry[v] = end[(k & 1) ^ 1][lane][v];
    }
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
    if (MODE != LINKED && w == 0)
#pragma unroll
      for (int v = 0; v < V; ++v) end[k & 1][lane][v] = carry[v];
  };
  if constexpr (MODE != LINKED)
    for (int k = last - 1; k >= first; --k) tile(k);
  else if (first < last)
    tile(first);
  // (every drawn number has its row of parts, and number c.tiles - 1, or 0 where
  // there are none, ends at the first frame)
  if (a.dh0 && c.on && w == 0 && first == 0 && (MODE != LINKED || drawn + 1 == c.tiles || (c.tiles == 0 && drawn == 0)))
#pragma unroll
    for (int v = 0; v < V; ++v) a.dh0[c.st + v] = carry[v];
#pragma unroll
  for (int v = 0; v < V; ++v) lsum[w][lane][v] = dlam[v];
  __syncthreads();
  // (a sequence without frames adds nothing, whatever its dhT: 0 times an infinity
  // is none)
  if (c.on && w == 0)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float s = lsum[0][lane][v];
#pragma unroll
      for (int k = 1; k < W; ++k) s += lsum[k][lane][v];
      a.parts[drawn * BH + c.st + v] = c.len > 0 ? s : 0.f;
    }
}

// Zeros in place of the gradients of a pass whose wait ran out (every thread of the
// grid calls this).
template <typename T> __device__ void discard_gradients(const GatedRecurrence& a) {
  const int64_t i0 = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, step = (int64_t)gridDim.x * blockDim.x;
  for (int64_t i = i0; i < a.N * a.H; i += step) {
    const int64_t row = i / a.H, at = row * a.ldd + (i - row * a.H);
    static_cast<T*>(a.dx)[at] = static_cast<T*>(a.dr)[at] = static_cast<T*>(a.di)[at] = (T)0;
  }
  if (a.dh0)
    for (int64_t i = i0; i < (int64_t)a.B * a.H; i += step) a.dh0[i] = 0.f;
}

// dlam[d] = sigm(lam) / softplus(lam) times the sum of the rows of parts; their
// quotient tends to 1 where both vanish.  (256 rows of 768: 4.9 us, the latency of
// eight rows in turn, a barrier and a launch.)  The last launch of a backward call:
// where a wait of it or of its forward call ran out, it leaves zeros.
template <typename T>
__global__ __launch_bounds__(1024) void gr_dlam_kernel(GatedRecurrence a, int64_t rows) {
  __shared__ float sum[32][33];
  const bool lost = *a.err != 0;
  if (lost) discard_gradients<T>(a);
  const float s = column_sum(a.parts, rows, a.H, sum);
  const int d = blockIdx.x * 32 + threadIdx.x;
  if (threadIdx.x >= 32 || d >= a.H) return;
  const float l = a.lam[d];
  const float g = l < -20.f ? s : s * (1.f / (1.f + expf(-l))) / softplus(l);
  a.dlam[d] = lost ? 0.f : g;
}

// The packed offset of every frame, off_t = B_t t + (the sum of the lengths from
// sequence B_t on), and the lengths, where the kernels read them; and the words that
// linked tiles start from as zeros.  (1500 frames of 128 sequences: 5.2 us, the
// latency of the search.)
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
  if (a.last)
    for (int64_t k = t; k < a.words + a.states; k += (int64_t)gridDim.x * 256) {
      if (k < a.words) a.clear_words[k] = 0;
      else a.clear_states[k - a.words] = 0;
    }
}

hipError_t schedule(GatedSchedule a, const int32_t* lengths, hipStream_t s) {
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
    int64_t n = a.count;
    if (a.last) {
      if (a.T + 1 > n) n = a.T + 1;
      const int64_t clear = a.words + a.states < 65536 ? a.words + a.states : 65536;
      if (clear > n) n = clear;
    }
    hipLaunchKernelGGL(gr_schedule_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

template <typename T, int V, bool RAGGED>
hipError_t launch(GatedRecurrence a, const int32_t* lengths, bool forward, hipStream_t s) {
  const unsigned groups = (unsigned)(((int64_t)a.B * (a.H / V) + 63) / 64);
  a.most_tiles = (a.T + GR_TILE - 1) / GR_TILE;
  const bool link = gated_linked(a.T, groups);
  int64_t words = 0, states = 0;  // (tickets, flags and states start from zero, and the time-out flag)
  if (link) {
    a.flags = a.tickets + (int64_t)groups * TICKET_LINE;
    words = (int64_t)(TICKET_LINE + a.most_tiles) * groups;
    states = (int64_t)((a.most_tiles - 1) / LINK + 1) * a.B * a.H;
  }
  if (RAGGED && forward) {
    GatedSchedule g;
    g.offs = const_cast<int32_t*>(a.offs);
    g.lens = const_cast<int32_t*>(a.lens);
    g.tails = a.tails;
    g.T = a.T;
    g.B = a.B;
    g.clear_words = reinterpret_cast<uint32_t*>(a.err);
    g.clear_states = a.states;
    g.words = link ? words + 1 : 0;
    g.states = states;
    const hipError_t e = schedule(g, lengths, s);
    if (e != hipSuccess) return e;
  } else if (link) {
    // (a backward pass leaves the time-out flag as its forward pass did)
    float* const from = forward ? reinterpret_cast<float*>(a.err) : reinterpret_cast<float*>(a.tickets);
    const hipError_t e = fill_zero2(from, forward ? words + 1 : words, reinterpret_cast<float*>(a.states), 2 * states, s);
    if (e != hipSuccess) return e;
  }
  // one frame and nothing to keep of it: a wave does without a tile
  if (forward && a.T == 1 && !a.saved) {
    hipLaunchKernelGGL((gr_forward_kernel<T, V, RAGGED, ONE, 1, 1>), dim3(groups), dim3(64), 0, s, a);
    return hipGetLastError();
  }
  const dim3 grid(groups, link ? a.most_tiles : 1), block(64 * W);
  if (forward) {
    // (linked stretches of 16 frames, half as many links: the recording of the
    // comment at LINK took 163 us with 8; the backward pass has no registers left)
    constexpr int LONG = 16;
    const dim3 linked(groups, (unsigned)((a.T + LONG * W - 1) / (LONG * W)));
    if (link) hipLaunchKernelGGL((gr_forward_kernel<T, V, RAGGED, LINKED, LONG, W>), linked, block, 0, s, a);
    else if (a.most_tiles > 1) hipLaunchKernelGGL((gr_forward_kernel<T, V, RAGGED, IN_TURN, TC, W>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((gr_forward_kernel<T, V, RAGGED, ONE, TC, W>), grid, block, 0, s, a);
    return hipGetLastError();
  }
  if (link) hipLaunchKernelGGL((gr_backward_kernel<T, V, RAGGED, LINKED>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((gr_backward_kernel<T, V, RAGGED, IN_TURN>), grid, block, 0, s, a);
  hipLaunchKernelGGL(gr_dlam_kernel<T>, dim3((unsigned)((a.H + 31) / 32)), dim3(1024), 0, s, a,
                     (int64_t)a.B * grid.y);
  return hipGetLastError();
}

// Two bf16 channels a lane where every row starts on a multiple of 4 bytes (two / one:
// forward and backward of 256 sequences of 64 x 768, 70 / 74 us; of 128 of 200 to 1500,
// 418 / 486; one of 40001 x 1536, forward, 135 / 149).
bool paired(const GatedRecurrence& a) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.r) |
                       reinterpret_cast<uintptr_t>(a.i) | reinterpret_cast<uintptr_t>(a.h) |
                       reinterpret_cast<uintptr_t>(a.dh) | reinterpret_cast<uintptr_t>(a.dx) |
                       reinterpret_cast<uintptr_t>(a.dr) | reinterpret_cast<uintptr_t>(a.di);
  return at % 4 == 0 && (a.H | a.ld | a.lddh | a.ldd) % 2 == 0;
}

template <typename T, int V>
hipError_t shaped(const GatedRecurrence& a, const int32_t* lengths, bool forward, hipStream_t s) {
  return a.lens ? launch<T, V, true>(a, lengths, forward, s) : launch<T, V, false>(a, lengths, forward, s);
}

hipError_t route(const GatedRecurrence& a, const int32_t* lengths, bool bf16, bool forward, hipStream_t s) {
  if (!bf16) return shaped<float, 1>(a, lengths, forward, s);
  return paired(a) ? shaped<bf16_t, 2>(a, lengths, forward, s) : shaped<bf16_t, 1>(a, lengths, forward, s);
}

}  // namespace

hipError_t gated_schedule(const GatedSchedule& a, const int32_t* lengths, hipStream_t s) {
  return schedule(a, lengths, s);
}

hipError_t gated_forward(const GatedRecurrence& a, const int32_t* lengths, bool bf16, hipStream_t s) {
  return route(a, lengths, bf16, true, s);
}
hipError_t gated_backward(const GatedRecurrence& a, bool bf16, hipStream_t s) {
  return route(a, nullptr, bf16, false, s);
}

// Where at most 400 workgroups' worth of channels leave CUs (or the second workgroup
// of some) without work, from five tiles on, or seven where the first wave of
// workgroups is nearly enough.  Linked / in turn, us, forward and backward, bf16: 6
// groups x 320 frames 12 13 / 17 25, x 2000 14 18 / 95 139; 192 x 320 25 30 / 21 31, x
// 2000 94 176 / 108 222; 256 x 320 28 35 / 22 33, x 500 35 48 / 30 47 (lengths that
// differ 29 40 / 34 46); 384 x 500 46 91 / 46 89, x 2000 172 348 / 201 340; 480 x 2000
// 216 435 / 209 374.  One rule serves both passes and all lengths: a forward call near
// its edge (192 x 320, 256 x 500 of equal lengths) is 4 to 5 us slower for it.
bool gated_linked(int T, int64_t groups) {
  return groups <= 400 && T > (groups <= 192 ? 4 : 6) * GR_TILE;
}
GatedLinks gated_links(int64_t T, int64_t B, int64_t H) {
  GatedLinks l{0, 0, 0};
  const int64_t tiles = (T + GR_TILE - 1) / GR_TILE;
  // two channels a lane make the fewest groups, one a lane the most
  const int64_t fewest = (B * (H / 2) + 63) / 64, most = (B * H + 63) / 64;
  if (!gated_linked((int)T, fewest)) return l;
  l.words = (TICKET_LINE + tiles) * most;
  l.stretches = tiles * B * H;
  l.states = ((tiles - 1) / LINK + 1) * B * H;
  return l;
}

}  // namespace am
