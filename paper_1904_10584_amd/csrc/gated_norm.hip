// What stands between two blocks of a residual stack, a row (frame) at a time:
//   u = o silu(gate)            the block's output under its gate
//   p = u / rms(u)              normed,
//   R = res + scale w_post p    scaled and added to the residual stream, and
//   y = R / rms(R) w_next       the norm that the next block reads,
// rms(z) = sqrt(mean z^2 + eps), and the gradient of it all.  HBM bounds it:
// every input is read once and every output written once, so a row stays in the
// registers of its wave (of its two or four waves if it is long) across both norms.
// 16384 x 768 with an fp32 stream: forward 35 us (5.0 TB/s), backward 52 us (5.3
// TB/s) and 5 us for the factors' gradients; 32768 x 1536 in bf16: 91 us (5.5 TB/s)
// and 162 us (5.0 TB/s).  64 x 768 forward: 3.6 us, a launch and one row's latency.
#include "am_device.h"
#include "am_internal.h"

namespace am {
namespace {

typedef f32x4_t f32x4_u __attribute__((aligned(4)));
typedef uint16_t u16x4_t __attribute__((ext_vector_type(4)));
typedef u16x4_t u16x4_u __attribute__((aligned(2)));

__device__ __forceinline__ f32x4_t wide(f32x4_t v) { return v; }
__device__ __forceinline__ f32x4_t wide(u16x4_t v) {
  f32x4_t o;
#pragma unroll
  for (int k = 0; k < 4; ++k) o[k] = bf16_to_f32(v[k]);
  return o;
}
template <typename T> struct Four;
template <> struct Four<float> { typedef f32x4_t type; typedef f32x4_u at; };
template <> struct Four<bf16_t> { typedef u16x4_t type; typedef u16x4_u at; };

__device__ __forceinline__ f32x4_t narrow(f32x4_t v, f32x4_t*) { return v; }
__device__ __forceinline__ u16x4_t narrow(f32x4_t v, u16x4_t*) {  // (to nearest even)
  typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(u16x4_t, __builtin_convertvector(v, bf16x4_t));
}

// v moved down by `past` elements (0 to 3; more: all zeros), zeros moving in.
__device__ __forceinline__ f32x4_t moved_down(f32x4_t v, int past) {
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = past & 1 ? (k < 3 ? v[k < 3 ? k + 1 : 3] : 0.f) : v[k];
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = past & 2 ? (k < 2 ? v[k < 2 ? k + 2 : 3] : 0.f) : v[k];
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = past > 3 ? 0.f : v[k];
  return v;
}
// Four bf16 in two words: constant shifts of words.  (Picked one by one, the elements
// became 64-bit shifts by a register.  Where that was the last register of a wave's
// allocation, 40 of 40 in the forward kernel of rows up to 256 in bf16, the results were
// wrong wherever waves shared a SIMD.)
__device__ __forceinline__ u16x4_t moved_down(u16x4_t v, int past) {
  typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
  const u32x2_t w = __builtin_bit_cast(u32x2_t, v);
  uint32_t lo = past & 2 ? w[1] : w[0], hi = past & 2 ? 0u : w[1];
  lo = past & 1 ? __builtin_amdgcn_alignbit(hi, lo, 16) : lo;
  hi = past & 1 ? hi >> 16 : hi;
  return __builtin_bit_cast(u16x4_t, u32x2_t{past > 3 ? 0u : lo, past > 3 ? 0u : hi});
}

// Four elements from place e of a row of H, those past its end as zeros; rows of
// odd lengths start at any element, which the memory instructions take.  `inside`
// (a constant where it is called): none are past it.  Else the load is the same for
// every lane (a branch for each would keep the loads of a row apart): where fewer
// than four are left, the row's last four, moved down.
template <typename T>
__device__ __forceinline__ typename Four<T>::type load4(const T* row, int e, int H, bool inside) {
  typedef typename Four<T>::at At;
  if (inside) return *reinterpret_cast<const At*>(row + e);
  typename Four<T>::type v = {0, 0, 0, 0};
  if (H < 4) {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (e + k < H) v[k] = row[e + k];
    return v;
  }
  const int from = e < H - 4 ? e : H - 4;
  v = *reinterpret_cast<const At*>(row + from);
  return moved_down(v, e - from);
}
template <typename T>
__device__ __forceinline__ void store4(T* row, int e, int H, bool inside, f32x4_t v) {
  typedef typename Four<T>::type Type;
  const Type o = narrow(v, (Type*)nullptr);
  if (inside || e + 4 <= H) {
    *reinterpret_cast<typename Four<T>::at*>(row + e) = o;
  } else {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (e + k < H) row[e + k] = o[k];
  }
}

constexpr int WAVES = 4;  // waves of a workgroup

// Place of this thread's elements: WPR waves have a row, NV times four elements a
// lane; WAVES / WPR rows of a workgroup side by side.
template <int WPR> struct Place {
  static constexpr int ROWS = WAVES / WPR, STEP = 256 * WPR;
  int row, e0;  // row of the workgroup's, first element
  __device__ Place() {
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    row = w / WPR;
    e0 = 4 * ((w % WPR) * 64 + (threadIdx.x & 63));
  }
};

// The sum over the row's WPR waves, in each of them; red: LDS, of sums taken in
// turn (`turn` alternates, so that one barrier a sum is enough).
template <int WPR>
__device__ __forceinline__ float row_sum(float v, float (&red)[2][WAVES], int& turn) {
  v = wave_sum_uniform(v);
  if constexpr (WPR == 1) return v;
  const int w = threadIdx.x >> 6, w0 = w / WPR * WPR;
  if ((threadIdx.x & 63) == 0) red[turn][w] = v;
  __syncthreads();
  float s = red[turn][w0];
#pragma unroll
  for (int k = 1; k < WPR; ++k) s += red[turn][w0 + k];
  turn ^= 1;
  return s;
}

// Of a lane's NV fours those that lie in every row of the lengths that NV stands
// for (see `sized`).
constexpr int whole_fours(int nv) { return nv <= 4 ? nv - 1 : 4; }

// Q8: y as 8-bit codes too (or only), in units of a power of two for each 128 elements
// of a row: 32 lanes have those, so their largest costs five moves between lanes.  16384
// x 768 with codes and y take 30 us (189 MB, 6.3 TB/s: HBM bounds it); 64 x 768 with
// codes alone 4.1, a launch.
template <typename T, typename R, int NV, int WPR, bool EXACT, bool Q8>
__global__ __launch_bounds__(256) void norm_forward_kernel(GatedNorm a) {
  __shared__ float red[2][WAVES];
  int turn = 0;
  const Place<WPR> at;
  auto inside = [](int k) { return EXACT || k < whole_fours(NV); };
  const int H = a.H;
  const float inv = 1.f / (float)H;
  f32x4_t add[NV], next[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int e = at.e0 + k * at.STEP;
    const f32x4_t one = {1.f, 1.f, 1.f, 1.f};
    add[k] = (a.w_post ? load4(a.w_post, e, H, inside(k)) : one) * (a.scale ? load4(a.scale, e, H, inside(k)) : one);
    next[k] = a.w_next ? load4(a.w_next, e, H, inside(k)) : one;
  }
  // (every wave takes as many turns: the sums of several waves have barriers; a row
  // past the last is the last one again, and not stored)
  for (int64_t first = (int64_t)blockIdx.x * at.ROWS; first < a.N; first += (int64_t)gridDim.x * at.ROWS) {
    const bool on = first + at.row < a.N;
    const int64_t row = on ? first + at.row : a.N - 1;
    f32x4_t u[NV], t[NV];
    const R* res = static_cast<const R*>(a.res) + row * H;
#pragma unroll
    for (int k = 0; k < NV; ++k) t[k] = wide(load4(res, at.e0 + k * at.STEP, H, inside(k)));
    float rstd_u = 1.f;
    if (a.o) {
      const T* o = static_cast<const T*>(a.o) + row * a.ldo;
#pragma unroll
      for (int k = 0; k < NV; ++k) u[k] = wide(load4(o, at.e0 + k * at.STEP, H, inside(k)));
      if (a.gate) {
        const T* gate = static_cast<const T*>(a.gate) + row * a.ldg;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const f32x4_t g = wide(load4(gate, at.e0 + k * at.STEP, H, inside(k)));
#pragma unroll
          for (int j = 0; j < 4; ++j) u[k][j] *= g[j] * sigm(g[j]);
        }
      }
      if (a.w_post) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int j = 0; j < 4; ++j) s = fmaf(u[k][j], u[k][j], s);
        rstd_u = rsqrtf(row_sum<WPR>(s, red, turn) * inv + a.eps);
      }
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) t[k][j] = fmaf(u[k][j] * rstd_u, add[k][j], t[k][j]);
      if (on) {
        R* out = static_cast<R*>(a.res_out) + row * H;
#pragma unroll
        for (int k = 0; k < NV; ++k) store4(out, at.e0 + k * at.STEP, H, inside(k), t[k]);
      }
    }
    float rstd_n = 1.f;
    if (a.w_next) {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) s = fmaf(t[k][j], t[k][j], s);
      rstd_n = rsqrtf(row_sum<WPR>(s, red, turn) * inv + a.eps);
      if (on && (!Q8 || a.y)) {
        T* y = static_cast<T*>(a.y) + row * H;
#pragma unroll
        for (int k = 0; k < NV; ++k) store4(y, at.e0 + k * at.STEP, H, inside(k), t[k] * rstd_n * next[k]);
      }
      if constexpr (Q8) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const int e = at.e0 + k * at.STEP;
          f32x4_t v = t[k] * rstd_n * next[k];
          uint32_t top = 0;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (!inside(k) && e + j >= H) v[j] = 0.f;  // (rstd_n may not be finite)
            const uint32_t m = __float_as_uint(v[j]) & 0x7fffffffu;
            top = m < 0x7f800000u && m > top ? m : top;
          }
          top = lanes16_max(top);
          const uint32_t other = (uint32_t)__shfl_xor((int)top, 16, 64);
          const uint32_t ex = q8_exponent(top > other ? top : other);
          if (on && e < ((H + 15) & ~15)) {  // (zeros behind the row's end)
            *reinterpret_cast<uint32_t*>(a.codes + row * a.ldc + e) = q8_codes4(v[0], v[1], v[2], v[3], q8_inverse(ex));
            if ((threadIdx.x & 31) == 0) a.scales[row * a.lds + (e >> 7)] = (uint8_t)ex;
          }
        }
      }
    }
    if (a.rstd && on && at.e0 == 0) {
      a.rstd[2 * row] = rstd_u;
      a.rstd[2 * row + 1] = rstd_n;
    }
  }
}

// Wavefronts a SIMD that the backward pass's registers leave room for: as many
// workgroups a CU make the grid, which then has no last round half empty (32768 x
// 1536 in bf16: 207 us with 1024 workgroups, 162 with 768; 16384 x 768 with an fp32
// stream: 63 and 52).
constexpr int backward_waves(int nv) { return nv <= 3 ? 3 : nv <= 4 ? 2 : 1; }

// With n = R / rms(R), dn = dy w_next:  dR = dres_out + (dn - n mean(dn n)) / rms(R),
// the gradient of res; dp = dR scale w_post;  du = (dp - p mean(dp p)) / rms(u), and
// from it those of o and gate.  R and p are evaluated again from the forward
// pass's inputs (in 32 bits, whatever the stream holds) with its 1 / rms.  The
// gradients of w_post and scale are scale and w_post times the same column sum
// of dR p; the sums run down a wave's rows in its registers and leave as one row
// per workgroup.
template <typename T, typename R, int NV, int WPR, bool EXACT>
__global__ __launch_bounds__(256, backward_waves(NV)) void norm_backward_kernel(GatedNorm a) {
  __shared__ float red[2][WAVES];
  __shared__ f32x4_t sums[2][WPR < WAVES ? NV * 64 * WPR : 1];
  int turn = 0;
  const Place<WPR> at;
  auto inside = [](int k) { return EXACT || k < whole_fours(NV); };
  const int H = a.H;
  const float inv = 1.f / (float)H;
  f32x4_t add[NV], next[NV], along[NV], ndy[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int e = at.e0 + k * at.STEP;
    const f32x4_t one = {1.f, 1.f, 1.f, 1.f};
    add[k] = (a.w_post ? load4(a.w_post, e, H, inside(k)) : one) * (a.scale ? load4(a.scale, e, H, inside(k)) : one);
    next[k] = a.w_next ? load4(a.w_next, e, H, inside(k)) : one;
    along[k] = ndy[k] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  for (int64_t first = (int64_t)blockIdx.x * at.ROWS; first < a.N; first += (int64_t)gridDim.x * at.ROWS) {
    const bool on = first + at.row < a.N;
    const int64_t row = on ? first + at.row : a.N - 1;
    f32x4_t p[NV], t[NV], d[NV];
    typename Four<T>::type o[NV], g[NV];
    const float rstd_u = a.rstd[2 * row], rstd_n = a.rstd[2 * row + 1];
    const R* res = static_cast<const R*>(a.res) + row * H;
#pragma unroll
    for (int k = 0; k < NV; ++k) t[k] = wide(load4(res, at.e0 + k * at.STEP, H, inside(k)));
#pragma unroll
    for (int k = 0; k < NV; ++k)
      d[k] = a.dres_out ? wide(load4(static_cast<const R*>(a.dres_out) + row * H, at.e0 + k * at.STEP, H, inside(k)))
                        : f32x4_t{0.f, 0.f, 0.f, 0.f};
    if (a.o) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        o[k] = load4(static_cast<const T*>(a.o) + row * a.ldo, at.e0 + k * at.STEP, H, inside(k));
        if (a.gate) g[k] = load4(static_cast<const T*>(a.gate) + row * a.ldg, at.e0 + k * at.STEP, H, inside(k));
      }
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        p[k] = wide(o[k]) * rstd_u;
        if (a.gate) {
          const f32x4_t gv = wide(g[k]);
#pragma unroll
          for (int j = 0; j < 4; ++j) p[k][j] *= gv[j] * sigm(gv[j]);
        }
        t[k] += p[k] * add[k];
      }
    }
    if (a.w_next) {
      f32x4_t dy[NV];
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        dy[k] = wide(load4(static_cast<const T*>(a.dy) + row * H, at.e0 + k * at.STEP, H, inside(k)));
        t[k] *= rstd_n;
        if (on) ndy[k] += dy[k] * t[k];
        dy[k] *= next[k];
#pragma unroll
        for (int j = 0; j < 4; ++j) s = fmaf(dy[k][j], t[k][j], s);
      }
      s = row_sum<WPR>(s, red, turn) * inv;
#pragma unroll
      for (int k = 0; k < NV; ++k) d[k] += (dy[k] - t[k] * s) * rstd_n;
    }
    if (on)
#pragma unroll
      for (int k = 0; k < NV; ++k)
        store4(static_cast<R*>(a.dres) + row * H, at.e0 + k * at.STEP, H, inside(k), d[k]);
    if (a.o) {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        if (on) along[k] += d[k] * p[k];
        d[k] *= add[k];
#pragma unroll
        for (int j = 0; j < 4; ++j) s = fmaf(d[k][j], p[k][j], s);
      }
      if (a.w_post) s = row_sum<WPR>(s, red, turn) * inv;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const f32x4_t ov = wide(o[k]);
        f32x4_t du = d[k];
        if (a.w_post) du = (du - p[k] * s) * rstd_u;
        f32x4_t dov = du;
        if (a.gate) {
          const f32x4_t gv = wide(g[k]);
          f32x4_t dg;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float sg = sigm(gv[j]);
            dov[j] = du[j] * gv[j] * sg;
            dg[j] = du[j] * ov[j] * sg * (1.f + gv[j] * (1.f - sg));
          }
          if (on) store4(static_cast<T*>(a.dgate) + row * a.lddg, at.e0 + k * at.STEP, H, inside(k), dg);
        }
        if (on) store4(static_cast<T*>(a.d_o) + row * a.lddo, at.e0 + k * at.STEP, H, inside(k), dov);
      }
    }
  }
  // the column sums of this workgroup's rows, one of them after another
  if constexpr (WPR < WAVES) {
    const int place = at.e0 / 4;
    for (int s = 0; s < at.ROWS; ++s) {
      if (at.row == s)
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          if (s > 0) {
            along[k] += sums[0][k * 64 * WPR + place];
            ndy[k] += sums[1][k * 64 * WPR + place];
          }
          sums[0][k * 64 * WPR + place] = along[k];
          sums[1][k * 64 * WPR + place] = ndy[k];
        }
      __syncthreads();
    }
    if (at.row != at.ROWS - 1) return;
  }
  float* parts = a.parts + (int64_t)blockIdx.x * 2 * H;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    store4(parts, at.e0 + k * at.STEP, H, inside(k), along[k]);
    store4(parts + H, at.e0 + k * at.STEP, H, inside(k), ndy[k]);
  }
}

// The factors' gradients from the column sums of parts [rows][2][H].
__global__ __launch_bounds__(1024) void norm_weights_kernel(const float* __restrict__ parts, int rows,
                                                            GatedNorm a) {
  __shared__ float sum[32][33];
  const float s = column_sum(parts, rows, 2 * a.H, sum);
  const int c = blockIdx.x * 32 + threadIdx.x;
  if (threadIdx.x >= 32 || c >= 2 * a.H) return;
  if (c >= a.H) {
    if (a.dw_next) a.dw_next[c - a.H] = s;
  } else {
    if (a.dw_post) a.dw_post[c] = s * (a.scale ? a.scale[c] : 1.f);
    if (a.dscale) a.dscale[c] = s * (a.w_post ? a.w_post[c] : 1.f);
  }
}

template <typename T, typename R, int NV, int WPR, bool EXACT>
hipError_t launch(const GatedNorm& a, bool forward, hipStream_t s) {
  const int64_t blocks = (a.N * WPR + WAVES - 1) / WAVES, most = forward ? 1024 : 256 * backward_waves(NV);
  const unsigned grid = (unsigned)(blocks < most ? blocks : most);
  if (forward) {
    if (a.codes) hipLaunchKernelGGL((norm_forward_kernel<T, R, NV, WPR, EXACT, true>), dim3(grid), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((norm_forward_kernel<T, R, NV, WPR, EXACT, false>), dim3(grid), dim3(256), 0, s, a);
  } else {
    if (grid > 0) hipLaunchKernelGGL((norm_backward_kernel<T, R, NV, WPR, EXACT>), dim3(grid), dim3(256), 0, s, a);
    hipLaunchKernelGGL(norm_weights_kernel, dim3((unsigned)((2 * a.H + 31) / 32)), dim3(1024), 0, s, a.parts,
                       (int)grid, a);
  }
  return hipGetLastError();
}

template <typename T, typename R, int NV, int WPR>
hipError_t filled(const GatedNorm& a, bool forward, hipStream_t s) {
  return a.H == NV * 256 * WPR ? launch<T, R, NV, WPR, true>(a, forward, s) : launch<T, R, NV, WPR, false>(a, forward, s);
}

// Two waves for rows beyond 1024: as many registers of one wave would leave one or
// two waves a SIMD (32768 x 1536 in bf16, forward and backward: one wave a row 428
// us, two 249).  No more of them where rows are few: the barriers cost what the
// shorter rows save (512 x 768 in bf16, forward and backward: one wave 3.6 and 9.0 us,
// two 4.5 and 9.1, four 4.5 and 9.7; 1237 x 1001 in fp32: 7.3 and 15.9, 6.7 and 16.6,
// 7.9 and 17.2).
template <typename T, typename R>
hipError_t sized(const GatedNorm& a, bool forward, hipStream_t s) {
  if (a.H <= 256) return filled<T, R, 1, 1>(a, forward, s);
  if (a.H <= 512) return filled<T, R, 2, 1>(a, forward, s);
  if (a.H <= 768) return filled<T, R, 3, 1>(a, forward, s);
  if (a.H <= 1024) return filled<T, R, 4, 1>(a, forward, s);
  if (a.H <= 1536) return filled<T, R, 3, 2>(a, forward, s);
  if (a.H <= 2048) return filled<T, R, 4, 2>(a, forward, s);
  if (a.H <= 3 * 1024) return filled<T, R, 3, 4>(a, forward, s);
  if (a.H <= 4096) return filled<T, R, 4, 4>(a, forward, s);
  return filled<T, R, 8, 4>(a, forward, s);
}

hipError_t route(const GatedNorm& a, bool bf16, bool stream_bf16, bool forward, hipStream_t s) {
  if (bf16) return stream_bf16 ? sized<bf16_t, bf16_t>(a, forward, s) : sized<bf16_t, float>(a, forward, s);
  return stream_bf16 ? sized<float, bf16_t>(a, forward, s) : sized<float, float>(a, forward, s);
}

}  // namespace

hipError_t gated_norm_forward(const GatedNorm& a, bool bf16, bool stream_bf16, hipStream_t s) {
  return a.N == 0 ? hipSuccess : route(a, bf16, stream_bf16, true, s);
}
hipError_t gated_norm_backward(const GatedNorm& a, bool bf16, bool stream_bf16, hipStream_t s) {
  return route(a, bf16, stream_bf16, false, s);
}

}  // namespace am
