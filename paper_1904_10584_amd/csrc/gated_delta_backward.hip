// The gated delta rule's backward pass (the chunk's notation: gated_delta.h).  With
// dS' the gradient of a chunk's last state, and everything of the forward pass made
// again from the state it starts from:
//   dU = P^T dO + diag(M_end) K dS',   (I + L)^T dR = dU,   dV = diag(beta) dR,
//   dS = g_end dS' + Q^T diag(g) dO - K^T diag(g beta) dR.
// Those go column by column as the forward pass does, backwards in time
// (gd_backward_kernel), and so do the gates: with  . the product of two rows,
//   dbeta_i beta_i = dR_i . U_i,   dc_i = dO_i . O_i - dV_i . V_i,  and <dS', S'> at
// the chunk's end: every sum over pairs of frames has been put together from sums over
// columns, since P's and L's entries scale with e^c.  What sums over columns, the
// gradients of q and k, is left to a second kernel, which has no order in time
// (gd_keys_kernel):
//   dQ = diag(g) dO S^T + (M o dO U^T) K,
//   dK = -diag(g beta) dR S^T + diag(M_end) U dS'^T + (M o dO U^T)^T Q + (B + B^T) K,
//   B_ij = -beta_i M_ij (dR_i . U_j), j < i.
#include "gated_delta.h"

namespace am {
namespace {

using namespace gd;

// The state that chunk n of a head starts from, and the gradient of the one it ends in.
__device__ __forceinline__ const float* state_before(const GatedDelta& a, int n, int64_t bh) {
  const int64_t state = (int64_t)a.dk * a.dv;
  if (n == 0) return a.s0 ? a.s0 + bh * state : nullptr;
  return a.saved + ((int64_t)(n - 1) * a.B * a.H + bh) * state;
}
__device__ __forceinline__ float* gradient_after(const GatedDelta& a, int n, int64_t bh) {
  return a.dsaved + ((int64_t)n * a.B * a.H + bh) * ((int64_t)a.dk * a.dv);
}

template <typename T, int DKP> struct Backward {
  Chunk<T, DKP, Terms<T>::X> s;
  float rows[2][WAVES][C];  // dO . O - dV . V and dR . U, of a wave's columns
  float end[WAVES];         // <dS', S'>
};

template <typename T, int DKP, int NT>
__global__ __launch_bounds__(THREADS) void gd_backward_kernel(GatedDelta a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  Backward<T, DKP>& all = *reinterpret_cast<Backward<T, DKP>*>(lds);
  Chunk<T, DKP, Terms<T>::X>& s = all.s;
  constexpr int TI = Terms<T>::IN, TX = Terms<T>::X, KT = DKP / 16;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g4 = lane >> 4;
  const int64_t bh = blockIdx.x;
  const Head hd(a, blockIdx.x);
  const Columns<NT> cols(a.dv);
  const float rate = a.c * softplus(a.lam[hd.h]);
  const int64_t state = (int64_t)a.dk * a.dv, ldu = (int64_t)a.H * a.dv;
  const int chunks = (hd.len + C - 1) / C;
  const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
  f32x4_t dS[KT][NT];
  load_state<DKP, NT>(a.dsT ? a.dsT + bh * state : nullptr, a, cols, lane, dS);
  float dlam = 0.f;  // (of frame `lane` of every chunk, in the first wave)
  for (int n = chunks - 1; n >= 0; --n) {
    const int t0 = n * C;
    Fetched<T, DKP> f;
    f.from(a, hd, t0);
    f32x4_t v[NB][NT], u[NB][NT], dO[NB][NT];
    load_rows<T, NT>(a.v, a.ldv, a, hd, t0, cols, lane, v);
    load_rows<T, NT>(a.d_o, a.lddo, a, hd, t0, cols, lane, dO);
    if (n < chunks - 1 || a.keep_end) store_state<DKP, NT>(gradient_after(a, n, bh), a, cols, lane, dS);
    stage<T, DKP>(s, f, a.eps, rate, hd.len - t0);
    __syncthreads();
    triangles(s);

    f32x4_t ks[NB][NT], o[NB][NT], kd[NB][NT];
#pragma unroll
    for (int I = 0; I < NB; ++I)
#pragma unroll
      for (int m = 0; m < NT; ++m) ks[I][m] = o[I][m] = kd[I][m] = zero;
    const float* const before = state_before(a, n, bh);
    float end = 0.f;
    {
      f32x4_t S[KT][NT];
      load_state<DKP, NT>(before, a, cols, lane, S);
#pragma unroll
      for (int t = 0; t < DKP / 32; ++t) {
        Piece<TX> s0[NT], s1[NT], d0[NT], d1[NT];
#pragma unroll
        for (int m = 0; m < NT; ++m) {
          s0[m] = split<TX>(S[2 * t][m]);
          s1[m] = split<TX>(S[2 * t + 1][m]);
          d0[m] = split<TX>(dS[2 * t][m]);
          d1[m] = split<TX>(dS[2 * t + 1][m]);
#pragma unroll
          for (int r = 0; r < 4; ++r) end = fmaf(S[2 * t][m][r], dS[2 * t][m][r], fmaf(S[2 * t + 1][m][r], dS[2 * t + 1][m][r], end));
        }
#pragma unroll
        for (int I = 0; I < NB; ++I) {
          Piece<TI> a0, a1;
          rows_of<T, DKP>(s.k, I, t, lane, a0, a1);
#pragma unroll
          for (int m = 0; m < NT; ++m) {
            mma<TI, TX>(ks[I][m], a0, a1, s0[m], s1[m]);
            mma<TI, TX>(kd[I][m], a0, a1, d0[m], d1[m]);
          }
          rows_of<T, DKP>(s.q, I, t, lane, a0, a1);
#pragma unroll
          for (int m = 0; m < NT; ++m) mma<TI, TX>(o[I][m], a0, a1, s0[m], s1[m]);
        }
      }
    }
    const float g_end = s.g[C - 1];
    end *= g_end;
#pragma unroll
    for (int I = 0; I < NB; ++I) {
      const f32x4_t beta = rows4(s.beta, I, lane), bgk = rows4(s.bgk, I, lane), gq = rows4(s.gq, I, lane), gk = rows4(s.gk, I, lane);
#pragma unroll
      for (int m = 0; m < NT; ++m) {
        u[I][m] = v[I][m] * beta - ks[I][m] * bgk;
        o[I][m] *= gq;
        kd[I][m] *= gk;
      }
    }
    {
      Piece<TX> up[NB][NT];
      solve(s, lane, u, up);
#pragma unroll
      for (int I = 0; I < NB; ++I) {
#pragma unroll
        for (int J = 0; J + 1 <= I; J += 2) {
          const Piece<TX> a0 = block_of(s.p[lower(I, J)], lane), a1 = block_of(s.p[lower(I, J + 1)], lane);
#pragma unroll
          for (int m = 0; m < NT; ++m) mma<TX, TX>(o[I][m], a0, a1, up[J][m], up[J + 1][m]);
        }
        if (I % 2 == 0) {
          const Piece<TX> a0 = block_of(s.p[lower(I, I)], lane);
#pragma unroll
          for (int m = 0; m < NT; ++m) mma<TX, TX>(o[I][m], a0, up[I][m]);
        }
      }
    }
    f32x4_t y1[NB], y2[NB];
#pragma unroll
    for (int I = 0; I < NB; ++I) {
      y1[I] = zero;
#pragma unroll
      for (int m = 0; m < NT; ++m) {
        y1[I] += dO[I][m] * o[I][m];
#pragma unroll
        for (int r = 0; r < 4; ++r) end = fmaf(u[I][m][r], kd[I][m][r], end);
      }
    }
    // dU (in kd), then dR (there too)
    {
      Piece<TI> dop[NB][NT];
#pragma unroll
      for (int I = 0; I < NB; ++I)
#pragma unroll
        for (int m = 0; m < NT; ++m) dop[I][m] = split<TI>(dO[I][m]);
#pragma unroll
      for (int J = 0; J < NB; ++J)
#pragma unroll
        for (int I = J; I < NB; ++I) {
          const Piece<TX> p = block_turned(s.p[lower(I, J)], lane);
#pragma unroll
          for (int m = 0; m < NT; ++m) mma<TX, TI>(kd[J][m], p, dop[I][m]);
        }
    }
    {
      Piece<TX> dp[NB][NT];
#pragma unroll
      for (int I = NB - 1; I >= 0; --I) {
#pragma unroll
        for (int J = NB - 1; J > I; --J) {
          const Piece<TX> p = block_turned(s.l[below(J, I)], lane);
#pragma unroll
          for (int m = 0; m < NT; ++m) mma<TX, TX>(kd[I][m], p, dp[J][m]);
        }
        const Piece<TX> d = block_turned(s.d[I], lane);
#pragma unroll
        for (int m = 0; m < NT; ++m) {
          const Piece<TX> w = split<TX>(kd[I][m]);
          kd[I][m] = zero;
          mma<TX, TX>(kd[I][m], d, w);
          dp[I][m] = split<TX>(kd[I][m]);
        }
      }
    }
    store_rows<float, NT>(a.u, ldu, a, hd, t0, cols, lane, u);
    store_rows<float, NT>(a.dr_rows, ldu, a, hd, t0, cols, lane, kd);
    Piece<TX> w1[NB][NT], w2[NB][NT];
#pragma unroll
    for (int I = 0; I < NB; ++I) {
      const f32x4_t beta = rows4(s.beta, I, lane), bgk = rows4(s.bgk, I, lane), gq = rows4(s.gq, I, lane);
      y2[I] = zero;
#pragma unroll
      for (int m = 0; m < NT; ++m) {
        y2[I] += kd[I][m] * u[I][m];
        const f32x4_t dv = kd[I][m] * beta;
        y1[I] -= dv * v[I][m];
        u[I][m] = dv;
        w1[I][m] = split<TX>(dO[I][m] * gq);
        w2[I][m] = split<TX>(-kd[I][m] * bgk);
      }
    }
    store_rows<T, NT>(a.dv_, a.lddv, a, hd, t0, cols, lane, u);
#pragma unroll
    for (int t = 0; t < KT; ++t) {
#pragma unroll
      for (int m = 0; m < NT; ++m) dS[t][m] *= g_end;
#pragma unroll
      for (int I = 0; I < NB; I += 2) {
        const Piece<TI> q0 = columns_of<T, DKP>(s.q, t, I, lane), q1 = columns_of<T, DKP>(s.q, t, I + 1, lane);
        const Piece<TI> k0 = columns_of<T, DKP>(s.k, t, I, lane), k1 = columns_of<T, DKP>(s.k, t, I + 1, lane);
#pragma unroll
        for (int m = 0; m < NT; ++m) {
          mma<TI, TX>(dS[t][m], q0, q1, w1[I][m], w1[I + 1][m]);
          mma<TI, TX>(dS[t][m], k0, k1, w2[I][m], w2[I + 1][m]);
        }
      }
    }
#pragma unroll
    for (int I = 0; I < NB; ++I)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float s1 = lanes_sum<16>(y1[I][r]), s2 = lanes_sum<16>(y2[I][r]);
        if (l16 == 0) {
          all.rows[0][wave][16 * I + 4 * g4 + r] = s1;
          all.rows[1][wave][16 * I + 4 * g4 + r] = s2;
        }
      }
    end = wave_sum_uniform(end);
    if (lane == 0) all.end[wave] = end;
    __syncthreads();
    if (wave == 0) {  // a frame a lane: the gates' gradients
      float d = (all.rows[0][0][lane] + all.rows[0][1][lane]) + (all.rows[0][2][lane] + all.rows[0][3][lane]);
      const float e = (all.rows[1][0][lane] + all.rows[1][1][lane]) + (all.rows[1][2][lane] + all.rows[1][3][lane]);
#pragma unroll
      for (int k = 1; k < C; k <<= 1) {  // from this frame to the chunk's last
        const float above = __shfl_down(d, k, 64);
        if (lane + k < C) d += above;
      }
      d += (all.end[0] + all.end[1]) + (all.end[2] + all.end[3]);
      const int t = t0 + lane;
      if (t < hd.len) {
        const float sr = sigm(f.r);
        const int64_t row = hd.row(t);
        static_cast<T*>(a.dr)[row * a.lddr + hd.h] = from_f32<T>(-rate * d * sr * (1.f - sr));
        static_cast<T*>(a.db)[row * a.lddb + hd.h] = from_f32<T>(e * (1.f - s.beta[lane]));
        dlam -= d * sr;
      }
    }
    __syncthreads();
  }
  if (a.ds0) store_state<DKP, NT>(a.ds0 + bh * state, a, cols, lane, dS);
  if (wave == 0) {
    dlam = wave_sum_uniform(dlam);
    if (lane == 0) a.parts[bh] = a.c * dlam;
  }
}

// The gradients of q and k of a chunk of a key head, summed over its heads: a wave has
// rows of them (16 columns of q and k at a time), a lane a frame of each block, so that
// what scales with a frame is a factor of a lane.
template <typename T, int DKP> struct Keys {
  static constexpr int TI = Terms<T>::IN, TO = Terms<T>::OUT;
  static constexpr int PITCH = 32 * 2 + 16;  // bytes of a row of a slice of 32 columns of v
  Staged<T, DKP> s;
  union {
    struct { uint8_t dO[TI][C * PITCH], u[TO][C * PITCH], dR[TO][C * PITCH]; } rows;
    struct { uint8_t qk[10][TO][512], kk[10][TO][512]; } blocks;
  };
  float dots[2][WAVES][C];
};

template <int N, int PITCH>
__device__ __forceinline__ void slice_row(const uint8_t (&m)[N][C * PITCH], int I, int lane, Piece<N>& a0, Piece<N>& a1) {
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const uint4 w = *reinterpret_cast<const uint4*>(m[e] + (16 * I + (lane & 15)) * PITCH + (lane >> 4) * 16);
    a0.t[e] = make_uint2(w.x, w.y);
    a1.t[e] = make_uint2(w.z, w.w);
  }
}
template <int N, int PITCH>
__device__ __forceinline__ void slice_store(uint8_t (&m)[N][C * PITCH], int row, int u, const float (&v)[8]) {
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int p = 2 * u + half, slot = (p & 3) * 2 + (p >> 2);
    const Piece<N> w = split<N>(f32x4_t{v[4 * half], v[4 * half + 1], v[4 * half + 2], v[4 * half + 3]});
#pragma unroll
    for (int e = 0; e < N; ++e) *reinterpret_cast<uint2*>(m[e] + row * PITCH + slot * 8) = w.t[e];
  }
}
// Four elements of a state's row from column c on, zeros past its end.
__device__ __forceinline__ f32x4_t state4(const float* m, int row, int c, const GatedDelta& a) {
  f32x4_t v = {0.f, 0.f, 0.f, 0.f};
  if (!m || row >= a.dk) return v;
  const float* p = m + (int64_t)row * a.dv + c;
  if (c + 4 <= a.dv) return *reinterpret_cast<const f32x4_a*>(p);
#pragma unroll
  for (int j = 0; j < 3; ++j)
    if (c + j < a.dv) v[j] = p[j];
  return v;
}

template <typename T, int DKP>
__global__ __launch_bounds__(THREADS) void gd_keys_kernel(GatedDelta a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  Keys<T, DKP>& all = *reinterpret_cast<Keys<T, DKP>*>(lds);
  Staged<T, DKP>& s = all.s;
  constexpr int TI = Terms<T>::IN, TO = Terms<T>::OUT, KM = DKP / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, g4 = lane >> 4;
  const int group = a.H / a.G, n = blockIdx.x / (a.B * a.G), bg = blockIdx.x % (a.B * a.G), t0 = n * C;
  const int b = bg / a.G, kh = bg % a.G;
  const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
  const int64_t ldu = (int64_t)a.H * a.dv;
  f32x4_t dq[KM][NB], dk[KM][NB];
#pragma unroll
  for (int m = 0; m < KM; ++m)
#pragma unroll
    for (int I = 0; I < NB; ++I) dq[m][I] = dk[m][I] = zero;
  for (int member = 0; member < group; ++member) {
    const int64_t bh = (int64_t)b * a.H + kh * group + member;
    const Head hd(a, (int)bh);
    if (t0 >= hd.len) return;  // (all heads of a sequence alike)
    const bool last = t0 + C >= hd.len;
    const float* const S = state_before(a, n, bh);
    const float* const dS = !last || a.keep_end ? gradient_after(a, n, bh)
                            : a.dsT ? a.dsT + bh * ((int64_t)a.dk * a.dv) : nullptr;
    {
      Fetched<T, DKP> f;
      f.from(a, hd, t0);
      stage<T, DKP>(s, f, a.eps, a.c * softplus(a.lam[hd.h]), hd.len - t0);
    }
    f32x4_t pair[5], sq[KM][NB], sk[KM][NB], su[KM][NB];
#pragma unroll
    for (int k = 0; k < 5; ++k) pair[k] = zero;
#pragma unroll
    for (int m = 0; m < KM; ++m)
#pragma unroll
      for (int I = 0; I < NB; ++I) sq[m][I] = sk[m][I] = su[m][I] = zero;
    for (int c0 = 0; c0 < a.dv; c0 += 32) {
      {
        const int row = threadIdx.x >> 2, piece = threadIdx.x & 3, col = c0 + 8 * piece, left = a.dv - col, t = t0 + row;
        float x[3][8];
        if (t < hd.len && left > 0) {
          const int64_t at = hd.row(t), h = (int64_t)hd.h * a.dv + col;
          load8(static_cast<const T*>(a.d_o) + at * a.lddo + h, left, x[0]);
          load8(a.u + at * ldu + h, left, x[1]);
          load8(a.dr_rows + at * ldu + h, left, x[2]);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) x[0][j] = x[1][j] = x[2][j] = 0.f;
        }
        slice_store<TI, Keys<T, DKP>::PITCH>(all.rows.dO, row, piece, x[0]);
        slice_store<TO, Keys<T, DKP>::PITCH>(all.rows.u, row, piece, x[1]);
        slice_store<TO, Keys<T, DKP>::PITCH>(all.rows.dR, row, piece, x[2]);
      }
      __syncthreads();
      if (c0 == 0 && wave == 1) {
        s.bgk[lane] = s.beta[lane] * s.g[lane] * s.rk[lane];
        s.gq[lane] = s.g[lane] * s.rq[lane];
        s.gk[lane] = s.end[lane] * s.rk[lane];
      }
#pragma unroll
      for (int k = 0; k < 5; ++k) {  // ten tiles of U dO^T, ten of U dR^T
        const int job = wave + WAVES * k, at = job < 10 ? job : job - 10;
        const int I = at >= 6 ? 3 : at >= 3 ? 2 : at >= 1 ? 1 : 0, J = at - lower(I, 0);
        Piece<TO> u0, u1;
        slice_row<TO, Keys<T, DKP>::PITCH>(all.rows.u, J, lane, u0, u1);
        if (job < 10) {
          Piece<TI> x0, x1;
          slice_row<TI, Keys<T, DKP>::PITCH>(all.rows.dO, I, lane, x0, x1);
          mma<TO, TI>(pair[k], u0, u1, x0, x1);
        } else {
          Piece<TO> x0, x1;
          slice_row<TO, Keys<T, DKP>::PITCH>(all.rows.dR, I, lane, x0, x1);
          mma<TO, TO>(pair[k], u0, u1, x0, x1);
        }
      }
#pragma unroll
      for (int m = 0; m < KM; ++m) {
        const int row = 16 * (wave + WAVES * m) + l16, c = c0 + 4 * g4;
        const Piece<TO> s0 = split<TO>(state4(S, row, c, a)), s1 = split<TO>(state4(S, row, c + 16, a));
        const Piece<TO> d0 = split<TO>(state4(dS, row, c, a)), d1 = split<TO>(state4(dS, row, c + 16, a));
#pragma unroll
        for (int I = 0; I < NB; ++I) {
          Piece<TI> o0, o1;
          Piece<TO> x0, x1;
          slice_row<TI, Keys<T, DKP>::PITCH>(all.rows.dO, I, lane, o0, o1);
          mma<TO, TI>(sq[m][I], s0, s1, o0, o1);
          slice_row<TO, Keys<T, DKP>::PITCH>(all.rows.dR, I, lane, x0, x1);
          mma<TO, TO>(sk[m][I], s0, s1, x0, x1);
          slice_row<TO, Keys<T, DKP>::PITCH>(all.rows.u, I, lane, x0, x1);
          mma<TO, TO>(su[m][I], d0, d1, x0, x1);
        }
      }
      __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < 5; ++k) {
      const int job = wave + WAVES * k, at = job < 10 ? job : job - 10;
      const int I = at >= 6 ? 3 : at >= 3 ? 2 : at >= 1 ? 1 : 0, J = at - lower(I, 0), i = 16 * I + l16;
      const f32x4_t ch = rows4(s.ch, J, lane), cl = rows4(s.cl, J, lane), rk = rows4(s.rk, J, lane);
      const float hi = s.ch[i], lo = s.cl[i], f = job < 10 ? s.rq[i] : -s.beta[i] * s.rk[i];
      f32x4_t v;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int j = 16 * J + 4 * g4 + r;
        const bool on = job < 10 ? j <= i : j < i;
        v[r] = on ? f * rk[r] * pair[k][r] * expf((hi - ch[r]) + (lo - cl[r])) : 0.f;
      }
      const Piece<TO> p = split<TO>(v);
#pragma unroll
      for (int e = 0; e < TO; ++e)
        *reinterpret_cast<uint2*>((job < 10 ? all.blocks.qk[at][e] : all.blocks.kk[at][e]) + l16 * 32 + g4 * 8) = p.t[e];
    }
    __syncthreads();
#pragma unroll
    for (int m = 0; m < KM; ++m) {
      const int tile = wave + WAVES * m;
#pragma unroll
      for (int I = 0; I < NB; ++I) {
        const float gq = s.gq[16 * I + l16], bgk = s.bgk[16 * I + l16], gk = s.gk[16 * I + l16];
        dq[m][I] += sq[m][I] * gq;
        dk[m][I] += su[m][I] * gk - sk[m][I] * bgk;
      }
#pragma unroll
      for (int I = 0; I < NB; ++I) {
        const Piece<TI> kI = columns_of<T, DKP>(s.k, tile, I, lane), qI = columns_of<T, DKP>(s.q, tile, I, lane);
#pragma unroll
        for (int J = 0; J < NB; ++J) {
          if (J >= I) mma<TI, TO>(dq[m][J], kI, block_of(all.blocks.qk[lower(J, I)], lane));
          if (J <= I) mma<TI, TO>(dk[m][J], qI, block_turned(all.blocks.qk[lower(I, J)], lane));
          if (J >= I) mma<TI, TO>(dk[m][J], kI, block_of(all.blocks.kk[lower(J, I)], lane));
          if (J <= I) mma<TI, TO>(dk[m][J], kI, block_turned(all.blocks.kk[lower(I, J)], lane));
        }
      }
    }
    if (member + 1 < group) __syncthreads();
  }
  // through the lengths: dq = t - q rq^2 (q . t), t what has been summed
  const Head hd(a, (int)((int64_t)b * a.H + kh * group));
  auto elements = [&](const uint8_t (&m)[TI][C * Staged<T, DKP>::PITCH], int tile, int I) {
    f32x4_t v = zero;
    const int at = (16 * I + l16) * Staged<T, DKP>::PITCH + (tile >> 1) * 64 + (g4 * 2 + (tile & 1)) * 8;
#pragma unroll
    for (int e = TI - 1; e >= 0; --e) {
      const uint2 w = *reinterpret_cast<const uint2*>(m[e] + at);
      v += f32x4_t{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                   __uint_as_float(w.y & 0xffff0000u)};
    }
    return v;
  };
#pragma unroll
  for (int I = 0; I < NB; ++I) {
    float x = 0.f, y = 0.f;
#pragma unroll
    for (int m = 0; m < KM; ++m) {
      const f32x4_t q = elements(s.q, wave + WAVES * m, I), k = elements(s.k, wave + WAVES * m, I);
#pragma unroll
      for (int r = 0; r < 4; ++r) x = fmaf(q[r], dq[m][I][r], x), y = fmaf(k[r], dk[m][I][r], y);
    }
    x += __shfl_xor(x, 16, 64);
    y += __shfl_xor(y, 16, 64);
    x += __shfl_xor(x, 32, 64);
    y += __shfl_xor(y, 32, 64);
    if (g4 == 0) {
      all.dots[0][wave][16 * I + l16] = x;
      all.dots[1][wave][16 * I + l16] = y;
    }
  }
  __syncthreads();
#pragma unroll
  for (int I = 0; I < NB; ++I) {
    const int i = 16 * I + l16, t = t0 + i;
    const float x = (all.dots[0][0][i] + all.dots[0][1][i]) + (all.dots[0][2][i] + all.dots[0][3][i]);
    const float y = (all.dots[1][0][i] + all.dots[1][1][i]) + (all.dots[1][2][i] + all.dots[1][3][i]);
    const float fq = s.rq[i] * s.rq[i] * x, fk = s.rk[i] * s.rk[i] * y;
    if (t >= hd.len) continue;
    const int64_t row = hd.row(t);
#pragma unroll
    for (int m = 0; m < KM; ++m) {
      const int tile = wave + WAVES * m, c = 16 * tile + 4 * g4;
      const f32x4_t vq = dq[m][I] - elements(s.q, tile, I) * fq, vk = dk[m][I] - elements(s.k, tile, I) * fk;
      T* const pq = static_cast<T*>(a.dq) + row * a.lddq + (int64_t)kh * a.dk + c;
      T* const pk = static_cast<T*>(a.dk_) + row * a.lddk + (int64_t)kh * a.dk + c;
      if (c + 4 <= a.dk) {
        if constexpr (sizeof(T) == 2) {
          typedef uint32_t u32x2_u __attribute__((ext_vector_type(2), aligned(2)));
          *reinterpret_cast<u32x2_u*>(pq) = u32x2_u{pair_bf16(vq[0], vq[1]), pair_bf16(vq[2], vq[3])};
          *reinterpret_cast<u32x2_u*>(pk) = u32x2_u{pair_bf16(vk[0], vk[1]), pair_bf16(vk[2], vk[3])};
        } else {
          *reinterpret_cast<f32x4_a*>(pq) = vq;
          *reinterpret_cast<f32x4_a*>(pk) = vk;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 3; ++j)
          if (c + j < a.dk) {
            pq[j] = from_f32<T>(vq[j]);
            pk[j] = from_f32<T>(vk[j]);
          }
      }
    }
  }
}

// dlam = sigm(lam) times the sum over sequences of parts [B][H].
__global__ __launch_bounds__(1024) void gd_dlam_kernel(GatedDelta a) {
  __shared__ float sum[32][33];
  const float s = column_sum(a.parts, a.B, a.H, sum);
  const int h = blockIdx.x * 32 + threadIdx.x;
  if (threadIdx.x < 32 && h < a.H) a.dlam[h] = s / (1.f + expf(-a.lam[h]));
}

template <typename T, int DKP, int NT> hipError_t backward(const GatedDelta& a, hipStream_t s) {
  constexpr int LDS = sizeof(Backward<T, DKP>), KEYS = sizeof(Keys<T, DKP>);
  static_assert(LDS <= 160 * 1024 && KEYS <= 160 * 1024, "a workgroup's LDS");
  static PerDevice ready, ready_keys;
  hipError_t e = allow_lds<LDS>(reinterpret_cast<const void*>(&gd_backward_kernel<T, DKP, NT>), ready);
  if (e == hipSuccess) e = allow_lds<KEYS>(reinterpret_cast<const void*>(&gd_keys_kernel<T, DKP>), ready_keys);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((gd_backward_kernel<T, DKP, NT>), dim3((unsigned)(a.B * a.H)), dim3(THREADS), LDS, s, a);
  const unsigned chunks = (unsigned)((a.T + C - 1) / C) * a.B * a.G;
  if (chunks) hipLaunchKernelGGL((gd_keys_kernel<T, DKP>), dim3(chunks), dim3(THREADS), KEYS, s, a);
  hipLaunchKernelGGL(gd_dlam_kernel, dim3((unsigned)((a.H + 31) / 32)), dim3(1024), 0, s, a);
  return hipGetLastError();
}

template <typename T> hipError_t sized(const GatedDelta& a, hipStream_t s) {
  if (a.dk <= 64) return a.dv <= 64 ? backward<T, 64, 1>(a, s) : backward<T, 64, 2>(a, s);
  return a.dv <= 64 ? backward<T, 128, 1>(a, s) : backward<T, 128, 2>(a, s);
}

}  // namespace

hipError_t gated_delta_backward(GatedDelta a, bool bf16, hipStream_t s) {
  return bf16 ? sized<bf16_t>(a, s) : sized<float>(a, s);
}

}  // namespace am
