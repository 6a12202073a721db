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
// those of the waves before it, and walks its stretch from the state so found.
#include "am_device.h"
#include "am_internal.h"

namespace am {
namespace {

constexpr int TC = GR_STRETCH, W = GR_WAVES;  // a tile is W stretches of TC frames
static_assert(TC * W == GR_TILE, "a tile of the saved states");

// V elements of a row as loaded, and the access itself.
template <typename T, int V> struct Vec { T e[V]; };
template <> struct alignas(4) Vec<bf16_t, 2> { bf16_t e[2]; };

template <typename T, int V>
__device__ __forceinline__ Vec<T, V> load(const void* base, int64_t at) {
  return *reinterpret_cast<const Vec<T, V>*>(static_cast<const T*>(base) + at);
}
template <typename T, int V>
__device__ __forceinline__ void store(void* base, int64_t at, const float (&v)[V]) {
  Vec<T, V> o;
#pragma unroll
  for (int k = 0; k < V; ++k) o.e[k] = from_f32<T>(v[k]);
  *reinterpret_cast<Vec<T, V>*>(static_cast<T*>(base) + at) = o;
}

// What a frame's gates come to.  1 - a^2 is 1 - e^-y of y = 2L, from its series
// where the difference would cancel (the seven terms leave 2e-8 of it at 0.35).
// With L = 0 (a shut gate, or a frame past the sequence's end) the state passes
// unchanged, and L / q takes its limit 0; so it does where 1 - a^2 is subnormal
// (the reciprocal root takes those for zero).
struct Gates {
  float sr, L, a, q, Lq;  // sigm(r), L, a, q and L / q
};
__device__ __forceinline__ Gates gates(float r, float rate, bool live) {
  Gates g;
  g.sr = sigm(r);
  g.L = live ? rate * g.sr : 0.f;
  g.a = __expf(-g.L);
  const float y = 2.f * g.L;
  float p = 1.f / 5040.f;
  p = fmaf(p, -y, 1.f / 720.f);
  p = fmaf(p, -y, 1.f / 120.f);
  p = fmaf(p, -y, 1.f / 24.f);
  p = fmaf(p, -y, 1.f / 6.f);
  p = fmaf(p, -y, 0.5f);
  p = fmaf(p, -y, 1.f);
  const float q2 = y < 0.35f ? p * y : fmaf(-g.a, g.a, 1.f);
  const float rq = q2 >= 1.17549435e-38f ? __builtin_amdgcn_rsqf(q2) : 0.f;
  g.q = q2 * rq;
  g.Lq = g.L * rq;
  return g;
}

__device__ __forceinline__ float softplus(float v) { return fmaxf(v, 0.f) + log1pf(expf(-fabsf(v))); }

// This lane's channels and sequence.
template <int V> struct Columns {
  int b, d, len;
  bool on;
  __device__ Columns(const GatedRecurrence& a, int lane) {
    const int per_row = a.H / V;
    const int64_t groups = (int64_t)a.B * per_row;
    int64_t g = (int64_t)blockIdx.x * 64 + lane;
    on = g < groups;
    if (!on) g = groups - 1;
    b = (int)(g / per_row);
    d = (int)(g % per_row) * V;
    len = a.lens ? a.lens[b] : a.T;
  }
};

// The packed row of frame t of sequence b (any row that exists if t is not one
// of its frames, for loads whose values are not used).
__device__ __forceinline__ int64_t row_of(const GatedRecurrence& a, int t, int b) {
  const int64_t tt = t < a.T ? t : a.T - 1;
  const int64_t row = (a.offs ? (int64_t)a.offs[tt] : tt * a.B) + b;
  return row < a.N ? row : a.N - 1;
}

template <typename T, int V>
__global__ __launch_bounds__(64 * W) void gr_forward_kernel(GatedRecurrence a) {
  __shared__ float agg[2][2][W][64][V];  // of tiles taken in turn: A, S of each stretch
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const Columns<V> c(a, lane);
  const int64_t st = (int64_t)c.b * a.H + c.d;
  float rate[V], carry[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    rate[v] = a.c * softplus(a.lam[c.d + v]);
    carry[v] = a.h0 ? a.h0[st + v] : 0.f;
  }
  const int tiles = (a.T + GR_TILE - 1) / GR_TILE;
  for (int k = 0; k < tiles; ++k) {
    const int t0 = k * GR_TILE + w * TC;
    Vec<T, V> x[TC], r[TC], i[TC];
    int64_t row[TC];
#pragma unroll
    for (int j = 0; j < TC; ++j) {
      row[j] = row_of(a, t0 + j, c.b);
      x[j] = load<T, V>(a.x, row[j] * a.ldx + c.d);
      r[j] = load<T, V>(a.r, row[j] * a.ldr + c.d);
      i[j] = load<T, V>(a.i, row[j] * a.ldi + c.d);
    }
    if (a.saved && c.on && w == 0)
#pragma unroll
      for (int v = 0; v < V; ++v) a.saved[(int64_t)k * a.B * a.H + st + v] = carry[v];
    float av[TC][V], u[TC][V], A[V], S[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      A[v] = 1.f;
      S[v] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < TC; ++j)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const bool live = t0 + j < c.len;
        const Gates g = gates(to_f32<T>(r[j].e[v]), rate[v], live);
        av[j][v] = g.a;
        u[j][v] = live ? g.q * sigm(to_f32<T>(i[j].e[v])) * to_f32<T>(x[j].e[v]) : 0.f;
        A[v] *= g.a;
        S[v] = fmaf(g.a, S[v], u[j][v]);
      }
    float (&g)[2][W][64][V] = agg[k & 1];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      g[0][w][lane][v] = A[v];
      g[1][w][lane][v] = S[v];
    }
    __syncthreads();
    float h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = carry[v];
#pragma unroll
    for (int s = 0; s < W; ++s)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        carry[v] = fmaf(g[0][s][lane][v], carry[v], g[1][s][lane][v]);
        if (s + 1 == w) h[v] = carry[v];
      }
#pragma unroll
    for (int j = 0; j < TC; ++j) {
#pragma unroll
      for (int v = 0; v < V; ++v) h[v] = fmaf(av[j][v], h[v], u[j][v]);
      if (c.on && t0 + j < c.len) store<T, V>(a.h, row[j] * a.H + c.d, h);
    }
  }
  if (a.hT && c.on && w == 0)
#pragma unroll
    for (int v = 0; v < V; ++v) a.hT[st + v] = carry[v];
}

template <typename T, int V>
__global__ __launch_bounds__(64 * W) void gr_backward_kernel(GatedRecurrence a) {
  __shared__ float agg[2][3][W][64][V];  // A, S and the carry's end from zero
  __shared__ float lsum[W][64][V];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const Columns<V> c(a, lane);
  const int64_t st = (int64_t)c.b * a.H + c.d;
  float rate[V], carry[V], dlam[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    rate[v] = a.c * softplus(a.lam[c.d + v]);
    carry[v] = a.dhT ? a.dhT[st + v] : 0.f;
    dlam[v] = 0.f;
  }
  const int tiles = (a.T + GR_TILE - 1) / GR_TILE;
  for (int k = tiles - 1; k >= 0; --k) {
    const int t0 = k * GR_TILE + w * TC;
    Vec<T, V> x[TC], r[TC], i[TC], dh[TC];
    int64_t row[TC];
#pragma unroll
    for (int j = 0; j < TC; ++j) {
      row[j] = row_of(a, t0 + j, c.b);
      x[j] = load<T, V>(a.x, row[j] * a.ldx + c.d);
      r[j] = load<T, V>(a.r, row[j] * a.ldr + c.d);
      i[j] = load<T, V>(a.i, row[j] * a.ldi + c.d);
      dh[j] = load<T, V>(a.dh, row[j] * a.lddh + c.d);
    }
    float h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = a.saved[(int64_t)k * a.B * a.H + st + v];
    Gates gt[TC][V];
    float si[TC][V], A[V], S[V], D[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      A[v] = 1.f;
      S[v] = D[v] = 0.f;
    }
    // (a frame past the end has a = 1 and q = 0, so only its dh needs a mask: its
    // x and dh may hold anything)
#pragma unroll
    for (int j = 0; j < TC; ++j)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const bool live = t0 + j < c.len;
        gt[j][v] = gates(to_f32<T>(r[j].e[v]), rate[v], live);
        si[j][v] = sigm(to_f32<T>(i[j].e[v]));
        if (!live) x[j].e[v] = dh[j].e[v] = 0;
        const float u = gt[j][v].q * (si[j][v] * to_f32<T>(x[j].e[v]));
        // the carry's end: D + (product of the a before) times the rest
        D[v] = fmaf(A[v] * gt[j][v].a, to_f32<T>(dh[j].e[v]), D[v]);
        A[v] *= gt[j][v].a;
        S[v] = fmaf(gt[j][v].a, S[v], u);
      }
    float (&g)[3][W][64][V] = agg[k & 1];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      g[0][w][lane][v] = A[v];
      g[1][w][lane][v] = S[v];
      g[2][w][lane][v] = D[v];
    }
    __syncthreads();
    float mine[V];
#pragma unroll
    for (int s = 0; s < W; ++s)
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (s < w) h[v] = fmaf(g[0][s][lane][v], h[v], g[1][s][lane][v]);
#pragma unroll
    for (int v = 0; v < V; ++v) mine[v] = carry[v];
#pragma unroll
    for (int s = W - 1; s >= 0; --s)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        carry[v] = fmaf(g[0][s][lane][v], carry[v], g[2][s][lane][v]);
        if (s - 1 == w) mine[v] = carry[v];
      }
    float before[TC][V];
#pragma unroll
    for (int j = 0; j < TC; ++j)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        before[j][v] = h[v];
        h[v] = fmaf(gt[j][v].a, h[v], gt[j][v].q * (si[j][v] * to_f32<T>(x[j].e[v])));
      }
#pragma unroll
    for (int j = TC - 1; j >= 0; --j) {
      float dx[V], dr[V], di[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Gates& q = gt[j][v];
        const float xv = to_f32<T>(x[j].e[v]);
        const float d = to_f32<T>(dh[j].e[v]) + mine[v];
        mine[v] = q.a * d;
        const float e = mine[v] * (si[j][v] * xv * q.a * q.Lq - q.L * before[j][v]);
        dlam[v] += e;
        dr[v] = e * (1.f - q.sr);
        const float dv = d * q.q;
        dx[v] = dv * si[j][v];
        di[v] = dx[v] * xv * (1.f - si[j][v]);
      }
      if (c.on && t0 + j < c.len) {
        store<T, V>(a.dx, row[j] * a.lddx + c.d, dx);
        store<T, V>(a.dr, row[j] * a.lddr + c.d, dr);
        store<T, V>(a.di, row[j] * a.lddi + c.d, di);
      }
    }
  }
  if (a.dh0 && c.on && w == 0)
#pragma unroll
    for (int v = 0; v < V; ++v) a.dh0[st + v] = carry[v];
#pragma unroll
  for (int v = 0; v < V; ++v) lsum[w][lane][v] = dlam[v];
  __syncthreads();
  if (c.on && w == 0)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float s = lsum[0][lane][v];
#pragma unroll
      for (int k = 1; k < W; ++k) s += lsum[k][lane][v];
      a.parts[st + v] = s;
    }
}

// dlam[d] = sigm(lam) / softplus(lam) times the sum of the rows of parts; their
// quotient tends to 1 where both vanish.  A workgroup takes 16 channels, 16
// threads each.
__global__ __launch_bounds__(256) void gr_dlam_kernel(const float* __restrict__ parts, int rows, int H,
                                                      const float* __restrict__ lam,
                                                      float* __restrict__ dlam) {
  __shared__ float sum[16][17];
  const int d = blockIdx.x * 16 + (threadIdx.x & 15), p = threadIdx.x >> 4;
  float s = 0.f;
  if (d < H)
    for (int k = p; k < rows; k += 16) s += parts[(int64_t)k * H + d];
  sum[p][threadIdx.x & 15] = s;
  __syncthreads();
  if (p != 0 || d >= H) return;
  for (int k = 1; k < 16; ++k) s += sum[k][threadIdx.x & 15];
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

template <typename T, int V>
hipError_t launch(const GatedRecurrence& a, bool forward, hipStream_t s) {
  const int64_t groups = (int64_t)a.B * (a.H / V);
  const dim3 grid((unsigned)((groups + 63) / 64));
  if (forward) hipLaunchKernelGGL((gr_forward_kernel<T, V>), grid, dim3(64 * W), 0, s, a);
  else hipLaunchKernelGGL((gr_backward_kernel<T, V>), grid, dim3(64 * W), 0, s, a);
  return hipGetLastError();
}

// Two bf16 channels a lane where every row starts on a multiple of 4 bytes.
bool paired(const GatedRecurrence& a) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.r) |
                       reinterpret_cast<uintptr_t>(a.i) | reinterpret_cast<uintptr_t>(a.h) |
                       reinterpret_cast<uintptr_t>(a.dh) | reinterpret_cast<uintptr_t>(a.dx) |
                       reinterpret_cast<uintptr_t>(a.dr) | reinterpret_cast<uintptr_t>(a.di);
  return at % 4 == 0 && (a.H | a.ldx | a.ldr | a.ldi | a.lddh | a.lddx | a.lddr | a.lddi) % 2 == 0;
}

hipError_t route(const GatedRecurrence& a, bool bf16, bool forward, hipStream_t s) {
  if (!bf16) return launch<float, 1>(a, forward, s);
  return paired(a) ? launch<bf16_t, 2>(a, forward, s) : launch<bf16_t, 1>(a, forward, s);
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
  const hipError_t e = route(a, bf16, false, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(gr_dlam_kernel, dim3((unsigned)((a.H + 15) / 16)), dim3(256), 0, s, a.parts, a.B,
                     a.H, a.lam, a.dlam);
  return hipGetLastError();
}

}  // namespace am
