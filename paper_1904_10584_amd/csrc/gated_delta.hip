// The gated delta rule's forward pass (its mathematics: gated_delta.h): chunks of 64
// frames one after another, a workgroup a head of a sequence; and one frame of many
// sequences, a pass over their states.
#include "gated_delta.h"

namespace am {
namespace {

using namespace gd;

template <typename T, int DKP, int NT>
__global__ __launch_bounds__(THREADS) void gd_forward_kernel(GatedDelta a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  constexpr int TI = Terms<T>::IN, TX = Terms<T>::X, TO = Terms<T>::OUT, KT = DKP / 16;
  Chunk<T, DKP, TO>& s = *reinterpret_cast<Chunk<T, DKP, TO>*>(lds);
  const int lane = threadIdx.x & 63;
  const Head hd(a, blockIdx.x);
  const Columns<NT> cols(a.dv);
  const float rate = a.c * softplus(a.lam[hd.h]);
  const int64_t state = (int64_t)a.dk * a.dv, mine = blockIdx.x * state;
  f32x4_t S[KT][NT];
  load_state<DKP, NT>(a.s0 ? a.s0 + mine : nullptr, a, cols, lane, S);
  for (int t0 = 0; t0 < hd.len; t0 += C) {
    Fetched<T, DKP> f;
    f.from(a, hd, t0);
    f32x4_t u[NB][NT];
    load_rows<T, NT>(a.v, a.ldv, a, hd, t0, cols, lane, u);
    if (a.train && t0 > 0) store_state<DKP, NT>(a.saved + (int64_t)(t0 / C - 1) * gridDim.x * state + mine, a, cols, lane, S);
    stage<T, DKP>(s, f, a.eps, rate, hd.len - t0);
    __syncthreads();
    triangles(s);

    f32x4_t ks[NB][NT], o[NB][NT];
#pragma unroll
    for (int I = 0; I < NB; ++I)
#pragma unroll
      for (int n = 0; n < NT; ++n) ks[I][n] = o[I][n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < DKP / 32; ++t) {
      Piece<TX> s0[NT], s1[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) s0[n] = split<TX>(S[2 * t][n]), s1[n] = split<TX>(S[2 * t + 1][n]);
#pragma unroll
      for (int I = 0; I < NB; ++I) {
        Piece<TI> a0, a1;
        rows_of<T, DKP>(s.k, I, t, lane, a0, a1);
#pragma unroll
        for (int n = 0; n < NT; ++n) mma<TI, TX>(ks[I][n], a0, a1, s0[n], s1[n]);
        rows_of<T, DKP>(s.q, I, t, lane, a0, a1);
#pragma unroll
        for (int n = 0; n < NT; ++n) mma<TI, TO>(o[I][n], a0, a1, first<TO>(s0[n]), first<TO>(s1[n]));
      }
    }
#pragma unroll
    for (int I = 0; I < NB; ++I) {
      const f32x4_t beta = rows4(s.beta, I, lane), bgk = rows4(s.bgk, I, lane), gq = rows4(s.gq, I, lane);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        u[I][n] = u[I][n] * beta - ks[I][n] * bgk;
        o[I][n] *= gq;
      }
    }
    Piece<TX> up[NB][NT];
    solve(s, lane, u, up);
#pragma unroll
    for (int I = 0; I < NB; ++I) {
#pragma unroll
      for (int J = 0; J + 1 <= I; J += 2) {
        const Piece<TO> a0 = block_of(s.p[lower(I, J)], lane), a1 = block_of(s.p[lower(I, J + 1)], lane);
#pragma unroll
        for (int n = 0; n < NT; ++n) mma<TO, TO>(o[I][n], a0, a1, first<TO>(up[J][n]), first<TO>(up[J + 1][n]));
      }
      if (I % 2 == 0) {
        const Piece<TO> a0 = block_of(s.p[lower(I, I)], lane);
#pragma unroll
        for (int n = 0; n < NT; ++n) mma<TO, TO>(o[I][n], a0, first<TO>(up[I][n]));
      }
    }
    store_rows<T, NT>(a.o, a.ldo, a, hd, t0, cols, lane, o);
#pragma unroll
    for (int I = 0; I < NB; ++I) {
      const f32x4_t gk = rows4(s.gk, I, lane);
#pragma unroll
      for (int n = 0; n < NT; ++n) up[I][n] = split<TX>(u[I][n] * gk);
    }
    const float g_end = s.g[C - 1];
#pragma unroll
    for (int t = 0; t < KT; ++t) {
#pragma unroll
      for (int n = 0; n < NT; ++n) S[t][n] *= g_end;
#pragma unroll
      for (int I = 0; I < NB; I += 2) {
        const Piece<TI> a0 = columns_of<T, DKP>(s.k, t, I, lane), a1 = columns_of<T, DKP>(s.k, t, I + 1, lane);
#pragma unroll
        for (int n = 0; n < NT; ++n) mma<TI, TX>(S[t][n], a0, a1, up[I][n], up[I + 1][n]);
      }
    }
    __syncthreads();
  }
  if (a.sT) store_state<DKP, NT>(a.sT + mine, a, cols, lane, S);
}

// One frame of each sequence: a state is read once, kept in registers, and written
// once.  A thread has four columns (CG threads a row) of every RG-th row.
template <typename T, int CG, int RPT>
__global__ __launch_bounds__(THREADS) void gd_token_kernel(GatedDelta a) {
  constexpr int RG = THREADS / CG;
  __shared__ float kq[2][GD_MAX_DIM];
  __shared__ f32x4_t sums[WAVES][CG];
  const Head hd(a, blockIdx.x);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, cg = threadIdx.x % CG, rg = threadIdx.x / CG;
  const int64_t mine = (int64_t)blockIdx.x * a.dk * a.dv;
  const int c0 = 4 * cg, left = a.dv - c0;
  f32x4_t S[RPT];
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const int row = rg + i * RG;
    S[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if (a.s0 && row < a.dk) {
      const float* p = a.s0 + mine + (int64_t)row * a.dv + c0;
      if (left >= 4) S[i] = *reinterpret_cast<const f32x4_a*>(p);
      else
#pragma unroll
        for (int j = 0; j < 3; ++j)
          if (j < left) S[i][j] = p[j];
    }
  }
  if (hd.len == 0) {  // (a sequence without a frame keeps its state)
    if (a.sT)
#pragma unroll
      for (int i = 0; i < RPT; ++i)
        if (rg + i * RG < a.dk)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (j < left) a.sT[mine + (int64_t)(rg + i * RG) * a.dv + c0 + j] = S[i][j];
    return;
  }
  const int64_t row0 = hd.row(0);
  if (wave < 2) {  // k, then q: its elements and 1 / its length
    const T* p = wave == 0 ? static_cast<const T*>(a.k) + row0 * a.ldk : static_cast<const T*>(a.q) + row0 * a.ldq;
    float x[2], sum = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int at = lane + 64 * i;
      x[i] = at < a.dk ? to_f32(p[(int64_t)hd.kh * a.dk + at]) : 0.f;
      sum = fmaf(x[i], x[i], sum);
    }
    const float r = 1.f / sqrtf(wave_sum_uniform(sum) + a.eps);
#pragma unroll
    for (int i = 0; i < 2; ++i) kq[wave][lane + 64 * i] = x[i] * r;
  }
  const float decay = expf(-a.c * softplus(a.lam[hd.h]) * sigm(to_f32(static_cast<const T*>(a.r)[row0 * a.ldr + hd.h])));
  const float beta = sigm(to_f32(static_cast<const T*>(a.b)[row0 * a.ldb + hd.h]));
  f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (j < left) v[j] = to_f32(static_cast<const T*>(a.v)[row0 * a.ldv + (int64_t)hd.h * a.dv + c0 + j]);
  __syncthreads();
  // the sum over the rows of x_row S[row], in every thread
  auto along = [&](const float (&x)[GD_MAX_DIM]) {
    f32x4_t y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < RPT; ++i) y += S[i] * x[min(rg + i * RG, GD_MAX_DIM - 1)];
#pragma unroll
    for (int o = CG; o < 64; o <<= 1)
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] += __shfl_xor(y[j], o, 64);
    if (lane < CG) sums[wave][lane] = y;
    __syncthreads();
    return (sums[0][cg] + sums[1][cg]) + (sums[2][cg] + sums[3][cg]);
  };
#pragma unroll
  for (int i = 0; i < RPT; ++i) S[i] *= decay;
  const f32x4_t u = (v - along(kq[0])) * beta;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < RPT; ++i) S[i] += u * kq[0][min(rg + i * RG, GD_MAX_DIM - 1)];
  const f32x4_t o = along(kq[1]);
  if (rg == 0)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < left) static_cast<T*>(a.o)[row0 * a.ldo + (int64_t)hd.h * a.dv + c0 + j] = from_f32<T>(o[j]);
  if (a.sT)
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
      const int row = rg + i * RG;
      if (row < a.dk) {
        float* p = a.sT + mine + (int64_t)row * a.dv + c0;
        if (left >= 4) *reinterpret_cast<f32x4_a*>(p) = S[i];
        else
#pragma unroll
          for (int j = 0; j < 3; ++j)
            if (j < left) p[j] = S[i][j];
      }
    }
}

template <typename T, int DKP, int NT> hipError_t chunks(const GatedDelta& a, hipStream_t s) {
  constexpr int LDS = sizeof(Chunk<T, DKP, Terms<T>::OUT>);
  static_assert(LDS <= 160 * 1024, "a workgroup's LDS");
  static PerDevice ready;
  const hipError_t e = allow_lds<LDS>(reinterpret_cast<const void*>(&gd_forward_kernel<T, DKP, NT>), ready);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((gd_forward_kernel<T, DKP, NT>), dim3((unsigned)(a.B * a.H)), dim3(THREADS), LDS, s, a);
  return hipGetLastError();
}

template <typename T, int CG> hipError_t token(const GatedDelta& a, hipStream_t s) {
  constexpr int RG = THREADS / CG;
  const dim3 grid((unsigned)(a.B * a.H));
  if (a.dk <= 64) hipLaunchKernelGGL((gd_token_kernel<T, CG, (64 + RG - 1) / RG>), grid, dim3(THREADS), 0, s, a);
  else hipLaunchKernelGGL((gd_token_kernel<T, CG, (128 + RG - 1) / RG>), grid, dim3(THREADS), 0, s, a);
  return hipGetLastError();
}

template <typename T> hipError_t forward(const GatedDelta& a, hipStream_t s) {
  if (a.T == 1 && !a.train) {
    if (a.dv <= 32) return token<T, 8>(a, s);
    if (a.dv <= 64) return token<T, 16>(a, s);
    return token<T, 32>(a, s);
  }
  if (a.dk <= 64) return a.dv <= 64 ? chunks<T, 64, 1>(a, s) : chunks<T, 64, 2>(a, s);
  return a.dv <= 64 ? chunks<T, 128, 1>(a, s) : chunks<T, 128, 2>(a, s);
}

}  // namespace

hipError_t gated_delta_forward(GatedDelta a, bool bf16, hipStream_t s) {
  return bf16 ? forward<bf16_t>(a, s) : forward<float>(a, s);
}

}  // namespace am
