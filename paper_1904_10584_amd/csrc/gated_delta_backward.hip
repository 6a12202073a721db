// The gated delta rule's backward pass (the chunk's notation: gated_delta.h).  With
// dS' the gradient of a chunk's last state, and everything of the forward pass made
// again from the state it starts from:
//   dU = P^T dO + diag(M_end) K dS',   (I + L)^T dR = dU,   dV = diag(beta) dR,
//   dS = g_end dS' + Q^T diag(g) dO - K^T diag(g beta) dR.
// Those go column by column as the forward pass does, backwards in time
// (gd_backward_kernel), and with  . the product of two rows so does
//   dbeta_i beta_i = dR_i . U_i.
// What sums over columns is left to a second kernel, which has no order in time
// (gd_keys_kernel): the gradients of q and k,
//   dQ = diag(g) dO S^T + (M o dO U^T) K,
//   dK = -diag(g beta) dR S^T + diag(M_end) U dS'^T + (M o dO U^T)^T Q + (B + B^T) K,
//   B_ij = -beta_i M_ij (dR_i . U_j), j < i,
// and that of each frame's log a, the sum of what crosses it from before to after,
//   sum_{j < i <= l} X_lj + sum_{l >= i} y_l + sum_{j < i} z_j + g_end <S, dS'>,
//   X_lj = P_lj (dO_l . U_j) - L_lj (dR_l . U_j),
//   y_l = g_l q_l . (S dO_l) - beta_l g_l k_l . (S dR_l),   z_j = M_end,j k_j . (dS' U_j):
// every term has a_i as a factor, however small that is.  (As a difference of sums over
// columns, dO_l . O_l - dV_l . V_l from i on, its rounding is that of the terms that do
// not cross: 2 % of dlam where a_i was e^-5, all of it at e^-12.)
#include "gated_delta.h"

namespace am {
namespace {

using namespace gd;

template <typename T, int DKP, int W> struct Backward {
  Chunk<T, DKP, W, Terms<T>::X, 2> c;
  float rows[W][C];  // dR . U, of a wave's columns
  float end[W];      // <S, dS'>
};

// In order of time within a head, as the forward pass, and bound as it is: 256 x 64
// frames, 12 heads of 64 x 64: 217 us (485 MB, 2.2 TB/s; two workgroups a CU for their
// registers); utterances of 200 to 1500 frames, 64 of 6 heads of 128 x 128: 645 us, in
// which the longest ones have 24 chunks.
//
// ENDS: only what each segment makes of a gradient of zero behind it, at its first state.
template <typename T, int DKP, int W, bool ENDS>
__global__ __launch_bounds__(threads_of<W>, 2) void gd_backward_kernel(GatedDelta a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  constexpr int TI = Terms<T>::IN, TX = Terms<T>::X, TO = Terms<T>::OUT, KT = DKP / 16;
  Backward<T, DKP, W>& all = *reinterpret_cast<Backward<T, DKP, W>*>(lds);
  auto& c = all.c;
  Gates& s = c.s;
  const int seg = blockIdx.y + (ENDS ? 1 : 0);
  const int64_t bh = blockIdx.x, state = (int64_t)a.dk * a.dv;
  const Head hd(a, blockIdx.x);
  const float rate = rate_of(a, hd.h);
  const int all_chunks = (hd.len + C - 1) / C, begin = seg * a.per, chunks = min(all_chunks, begin + a.per);
  if (seg > 0 && begin >= all_chunks) return;
  const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
  f32x4_t dS[KT];
  if (!ENDS && a.segs > 1)  // (dsT itself may be ds0, which the first segment writes)
    load_kept<DKP>(segment<DKP, W>(a.seg_d, a, chunks < all_chunks ? seg : a.segs - 1, bh), column_of(threadIdx.x), threadIdx.x & 63, dS);
  else
    load_state<DKP>(!ENDS && a.dsT ? a.dsT + bh * state : nullptr, a, column_of(threadIdx.x), threadIdx.x & 63, dS);
  Rows<T, DKP, W> fk, fq;
  Values<T, W> fv, fo;
  GateRows<T, W> fg;
  auto fetch = [&](const int32_t (&rows)[C], int next0, int tid) {
    fk.from(a.k, a.ldk, hd.kh, a.dk, rows, tid);
    fq.from(a.q, a.ldq, hd.kh, a.dk, rows, tid);
    if constexpr (!ENDS) fv.from(a.v, a.ldv, hd, a.dv, rows, tid);
    fo.from(a.d_o, a.lddo, hd, a.dv, rows, tid);
    fg.from(a, hd, rows, next0, tid);
  };
  if (begin < chunks) {
    if (threadIdx.x < C) s.row[0][threadIdx.x] = hd.row(a, (chunks - 1) * C + threadIdx.x);
    __syncthreads();
    if (ENDS) fetch(s.row[0], max(chunks - 2, 0) * C, threadIdx.x);
  }
  int turn = 0;
  for (int n = chunks - 1; n >= begin; --n, turn ^= 1) {
    const int left = hd.len - n * C, tid = this_thread(), lane = tid & 63, l16 = lane & 15, g4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = 16 * wave + l16;
    // (A chunk's inputs arrive during the one before where only the gradient of the
    // state goes on.  With everything else in registers that gave nothing, 217 and 645 us
    // either way, and spilled where dk is 128 and dv at most 64.)
    if (!ENDS) fetch(s.row[turn], max(n - 1, 0) * C, tid);
    const T b_now = fg.b;
    fk.lengths(s.rk, a.eps, left, tid);
    fq.lengths(s.rq, a.eps, left, tid);
    fk.store(c.k, tid);
    fq.store(c.q, tid);
    if constexpr (!ENDS) fv.store(&c.v[0], s.row[turn], tid);
    fo.store(&c.v[1], s.row[turn], tid);
    fg.store(s, rate, left, turn, tid);
    __syncthreads();
    if (ENDS && n > begin) fetch(s.row[turn ^ 1], max(n - 2, 0) * C, tid);
    f32x4_t S[KT];
    if constexpr (!ENDS) {
      if (n > 0) load_kept<DKP>(kept_before<DKP, W>(a, n, bh), col, lane, S);
      else load_state<DKP>(a.s0 ? a.s0 + bh * state : nullptr, a, col, lane, S);
    }
    if constexpr (!ENDS) store_kept<DKP>(kept_after<DKP, W>(a, n, bh), col, lane, dS);
    triangles<true>(c, tid);

    f32x4_t u[NB], kd[NB];
#pragma unroll
    for (int I = 0; I < NB; ++I) u[I] = kd[I] = zero;
    float end = 0.f;
#pragma unroll
    for (int t = 0; t < DKP / 32; ++t) {
      const Piece<TX> d0 = split<TX>(dS[2 * t]), d1 = split<TX>(dS[2 * t + 1]);
      Piece<TX> s0, s1;
      if constexpr (!ENDS) {
        s0 = split<TX>(S[2 * t]);
        s1 = split<TX>(S[2 * t + 1]);
#pragma unroll
        for (int r = 0; r < 4; ++r) end = fmaf(S[2 * t][r], dS[2 * t][r], fmaf(S[2 * t + 1][r], dS[2 * t + 1][r], end));
      }
#pragma unroll
      for (int I = 0; I < NB; ++I) {
        Piece<TI> a0, a1;
        rows_of(c.k, I, t, lane, a0, a1);
        mma<TI, TX>(kd[I], a0, a1, d0, d1);
        if constexpr (!ENDS) mma<TI, TX>(u[I], a0, a1, s0, s1);
      }
    }
    const float g_end = s.g[C - 1];
#pragma unroll
    for (int I = 0; I < NB; ++I) {
      if constexpr (!ENDS) u[I] = fv.column_values(wave, I, lane) * rows4(s.beta, I, lane) - u[I] * rows4(s.bgk, I, lane);
      kd[I] *= rows4(s.gk, I, lane);
    }
    // U; transposed, a frame a lane, it is wanted for dR . U
    f32x4_t ut[NB];
    if constexpr (!ENDS) {
      Piece<TX> r[NB], up[NB];
      solve(c, lane, u, r, up);
#pragma unroll
      for (int I = 0; I < NB; ++I) {
        ut[I] = zero;
        mma<TX, TX>(ut[I], r[I], block_of(c.d[I], lane));
      }
      uint16_t* const keep = kept_columns<TX, W>(a.u, a, n, bh);
#pragma unroll
      for (int e = 0; e < TX; ++e)
#pragma unroll
        for (int I = 0; I < NB; ++I)
          *reinterpret_cast<u32x2_t*>(keep + (e * 16 * W + col) * C + 16 * I + 4 * g4) = up[I].t[e];
    }
    float drive[NB];
    // dU in kd, then dR, block after block from the last
#pragma unroll
    for (int J = 0; J < NB; ++J)
#pragma unroll
      for (int I = J; I < NB; ++I) mma<TX, TI>(kd[J], block_turned(c.p[lower(I, J)], lane), fo.column(wave, I, lane));
    {
      Piece<TX> dp[NB];
#pragma unroll
      for (int I = NB - 1; I >= 0; --I) {
        const Piece<TX> d = block_turned(c.d[I], lane), w = split<TX>(kd[I]);
        f32x4_t dr = zero;  // (transposed)
        if constexpr (!ENDS) mma<TX, TX>(dr, w, d);
        kd[I] = zero;
        mma<TX, TX>(kd[I], d, w);
        dp[I] = split<TX>(kd[I]);
#pragma unroll
        for (int J = I - 1; J >= 0; --J) mma<TX, TX>(kd[J], block_turned(c.l[below(I, J)], lane), dp[I]);
        if constexpr (ENDS) continue;
        const f32x4_t dv = dr * s.beta[16 * I + l16], y = dr * ut[I];
        drive[I] = (y[0] + y[1]) + (y[2] + y[3]);
        if (16 * I + l16 < left)
          put4(static_cast<T*>(a.dv_) + s.row[turn][16 * I + l16] * a.lddv + (int64_t)hd.h * a.dv + 16 * wave + 4 * g4,
               a.dv - 16 * wave - 4 * g4, dv);
      }
      uint16_t* const keep = kept_columns<TX, W>(a.dr_rows, a, n, bh);
      if constexpr (!ENDS)
#pragma unroll
      for (int e = 0; e < TX; ++e)
#pragma unroll
        for (int I = 0; I < NB; ++I)
          *reinterpret_cast<u32x2_t*>(keep + (e * 16 * W + col) * C + 16 * I + 4 * g4) = dp[I].t[e];
    }
    {
      Piece<TX> w1[NB], w2[NB];
#pragma unroll
      for (int I = 0; I < NB; ++I) {
        w1[I] = split<TX>(fo.column_values(wave, I, lane) * rows4(s.gq, I, lane));
        w2[I] = split<TX>(-kd[I] * rows4(s.bgk, I, lane));
      }
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        dS[t] *= g_end;
#pragma unroll
        for (int I = 0; I < NB; I += 2) {
          mma<TI, TX>(dS[t], columns_of(c.q, t, I, lane), columns_of(c.q, t, I + 1, lane), w1[I], w1[I + 1]);
          mma<TI, TX>(dS[t], columns_of(c.k, t, I, lane), columns_of(c.k, t, I + 1, lane), w2[I], w2[I + 1]);
        }
      }
    }
    if constexpr (!ENDS) {
#pragma unroll
    for (int I = 0; I < NB; ++I) {
      drive[I] += __shfl_xor(drive[I], 16, 64);
      drive[I] += __shfl_xor(drive[I], 32, 64);
      if (g4 == 0) all.rows[wave][16 * I + l16] = drive[I];
    }
    end = wave_sum_uniform(end);
    if (lane == 0) all.end[wave] = end;
    __syncthreads();
    if (wave == W - 1) {  // a frame a lane
      float e = 0.f, ends = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) e += all.rows[w][lane], ends += all.end[w];
      if (lane < left)
        static_cast<T*>(a.db)[s.row[turn][lane] * a.lddb + hd.h] = from_f32<T>(e * sigm(-to_f32(b_now)));  // (1 - beta, which may be far below 1)
      if (lane == 0) a.parts[n * (int64_t)gridDim.x + bh] = ends;  // (for gd_keys_kernel)
    }
    }
    __syncthreads();
  }
  if constexpr (ENDS) {
    store_kept<DKP>(segment<DKP, W>(a.seg_d, a, seg - 1, bh), column_of(threadIdx.x), threadIdx.x & 63, dS);
    return;
  }
  if (a.ds0 && seg == 0) store_state<DKP>(a.ds0 + bh * state, a, column_of(threadIdx.x), threadIdx.x & 63, dS);
}

// The gradients of the states that segments end in, from the last one on; the last
// one's own is kept behind the others.
template <int DKP, int W> __global__ __launch_bounds__(64) void gd_join_back_kernel(GatedDelta a) {
  const int lane = threadIdx.x, col = 16 * blockIdx.y + (lane & 15), len = a.lens ? a.lens[blockIdx.x / a.H] : a.T;
  f32x4_t dS[DKP / 16];
  load_state<DKP>(a.dsT ? a.dsT + (int64_t)blockIdx.x * a.dk * a.dv : nullptr, a, col, lane, dS);
  auto ends = [&](int seg) { return segment<DKP, W>(a.seg_d, a, seg - 1, blockIdx.x); };
  auto map = [&](int seg) { return segment<DKP, DKP / 16>(a.seg_mt, a, seg, blockIdx.x); };
  store_kept<DKP>(segment<DKP, W>(a.seg_d, a, a.segs - 1, blockIdx.x), col, lane, dS);
  const int frames = a.per * C, last = len > 0 ? (len - 1) / frames : 0;
  Segment<DKP> now, next;
  constexpr bool AHEAD = DKP == 64;
  if (AHEAD && last > 0) now.from(ends(last), map(last), col, lane);
  for (int seg = last; seg > 0; --seg) {
    if (!AHEAD) now.from(ends(seg), map(seg), col, lane);
    else if (seg > 1) next.from(ends(seg - 1), map(seg - 1), col, lane);
    now.apply(dS);
    store_kept<DKP>(ends(seg), col, lane, dS);
    if (AHEAD) now = next;
  }
}

// Sums over the lanes up to each of them: within rows of 16, and over the wave.
template <int CTRL, int ROWS> __device__ __forceinline__ float lanes_up(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float row_sums(float v) {
  v += lanes_up<0x111, 0xf>(v);
  v += lanes_up<0x112, 0xf>(v);
  v += lanes_up<0x114, 0xf>(v);
  return v + lanes_up<0x118, 0xf>(v);
}
__device__ __forceinline__ float wave_sums(float v) {
  v = row_sums(v);
  v += lanes_up<0x142, 0xa>(v);
  return v + lanes_up<0x143, 0xc>(v);
}

// What a tile (I, J) of X gives to the sums over pairs (l, j) with j < i <= l: a lane has
// row l = lane % 16 and columns j = 4 (lane / 16) to + 3.  On the diagonal sums[0][i] is
// what crosses frame i within the tile; below it, sums[0][l] are sums of rows and
// sums[1][j] of columns.
__device__ __forceinline__ void crossing(f32x4_t x, bool diagonal, float (&sums)[2][16], int lane) {
  const int l16 = lane & 15, g4 = lane >> 4;
  float all = (x[0] + x[1]) + (x[2] + x[3]);
  f32x4_t out;
  if (diagonal) {
    float up = __shfl_up(all, 16, 64);
    all += g4 >= 1 ? up : 0.f;
    up = __shfl_up(all, 32, 64);
    all += g4 >= 2 ? up : 0.f;
    up = __shfl_up(all, 16, 64);
    float before = g4 >= 1 ? up : 0.f;  // the row's sum before each column
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      out[r] = lanes_sum<16>(l16 >= 4 * g4 + r ? before : 0.f);
      before += x[r];
    }
    if (l16 == 0) *reinterpret_cast<f32x4_t*>(&sums[0][4 * g4]) = out;
  } else {
    all += __shfl_xor(all, 16, 64);
    all += __shfl_xor(all, 32, 64);
    if (g4 == 0) sums[0][l16] = all;
#pragma unroll
    for (int r = 0; r < 4; ++r) out[r] = lanes_sum<16>(x[r]);
    if (l16 == 0) *reinterpret_cast<f32x4_t*>(&sums[1][4 * g4]) = out;
  }
}
// The sum of X over the pairs that cross frame `lane`, y from it on, and z before it, from
// the tiles' sums and the waves' parts of y and z.  A suffix is a prefix of the lanes in
// reverse.
template <int W>
__device__ __forceinline__ float crossed(const float (&sums)[10][2][16], const float (&yz)[2][W][C], int lane) {
  const int b = lane >> 4, i = lane & 15, back = C - 1 - lane, bb = back >> 4, bi = back & 15;
  float y = 0.f, z = 0.f, rows = 0.f, cols = 0.f, both = 0.f;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    y += yz[0][w][back];
    z += lane > 0 ? yz[1][w][max(lane - 1, 0)] : 0.f;
  }
#pragma unroll
  for (int J = 0; J + 1 < NB; ++J) rows += J < bb ? sums[lower(bb, min(J, bb))][0][bi] : 0.f;
#pragma unroll
  for (int I = 1; I < NB; ++I) cols += I > b && i > 0 ? sums[lower(max(I, b), b)][1][max(i - 1, 0)] : 0.f;
#pragma unroll
  for (int I = 2; I < NB; ++I)
#pragma unroll
    for (int J = 0; J + 1 < I; ++J) both += J < b && b < I ? sums[lower(I, J)][0][i] : 0.f;
  const float from = __shfl(wave_sums(y) + row_sums(rows), back, 64);
  return (from + wave_sums(z)) + (row_sums(cols) + lanes_sum<16>(both)) + sums[lower(b, b)][0][i];
}

// The gradients of q and k of a chunk of a key head, summed over its heads: a wave has
// 16 columns of them, a lane a frame of each block, so that what scales with a frame is
// a factor of a lane; and those of its heads' decays.  It goes through v's columns 32 at
// a time, then takes the sums over pairs of frames to K and Q, which have the same LDS by
// then.  S, dS', U and dR enter in three terms, since dlam is a sum of what they make in
// 32 bits: with two, dlam of 256 x 64 frames in bf16 was off by 4.1e-6 and not 2.9e-7, for
// 484 and not 517 us of a training pass.  Chunks are all independent here; 202 us for
// those frames, 12 heads of 64 x 64 (375 MB, 1.9 TB/s), 594 for the utterances: the LDS
// pipeline, vector and matrix instructions, one after another between barriers.
template <typename T, int DKP> struct Keys {
  static constexpr int TI = Terms<T>::IN, TX = Terms<T>::X, TO = Terms<T>::OUT;
  static constexpr int FRAMES = C * 2 + 16, KEYS = DKP * 2 + 16;  // bytes of a row of columns, of states
  union {
    struct {
      Matrix<TI, 32> dO;
      uint8_t u[TX][32 * FRAMES], dR[TX][32 * FRAMES];  // 32 columns over frames
      uint8_t S[TX][32 * KEYS], dS[TX][32 * KEYS];      // and over keys
    } slice;
    struct {
      Matrix<TI, DKP> k, q;
      uint8_t qk[10][TO][512], kk[10][TO][512];
    } pairs;
  };
  float dots[2][DKP / 16][C];
  float yz[2][DKP / 16][C], cross[10][2][16];  // of a head's decays
  Gates s;
};

template <typename T, int DKP, int VP>
__global__ __launch_bounds__(DKP * 4, 2) void gd_keys_kernel(GatedDelta a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  Keys<T, DKP>& all = *reinterpret_cast<Keys<T, DKP>*>(lds);
  Gates& s = all.s;
  constexpr int TI = Terms<T>::IN, TX = Terms<T>::X, TO = Terms<T>::OUT, W = DKP / 16, TH = threads_of<W>, VW = VP / 16;
  constexpr int FRAMES = Keys<T, DKP>::FRAMES, KEYS = Keys<T, DKP>::KEYS;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, g4 = lane >> 4;
  const int group = a.H / a.G, n = blockIdx.x / (a.B * a.G), bg = blockIdx.x % (a.B * a.G), t0 = n * C;
  const int b = bg / a.G, kh = bg % a.G;
  const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
  f32x4_t dq[NB], dk[NB];
#pragma unroll
  for (int I = 0; I < NB; ++I) dq[I] = dk[I] = zero;
  Rows<T, DKP, W> fk, fq;
  GateRows<T, W> fg;
  for (int member = 0; member < group; ++member) {
    const int64_t bh = (int64_t)b * a.H + kh * group + member;
    const Head hd(a, (int)bh);
    const int left = hd.len - t0;
    if (left <= 0) {  // (all heads of a sequence alike)
      for (int m = threadIdx.x; m < group; m += TH) a.parts[(int64_t)n * a.B * a.H + bh + m] = 0.f;
      return;
    }
    if (member == 0) {
      if (threadIdx.x < C) s.row[0][threadIdx.x] = hd.row(a, t0 + threadIdx.x);
      __syncthreads();
    }
    const int tid = this_thread();
    fk.from(a.k, a.ldk, kh, a.dk, s.row[0], tid);
    fq.from(a.q, a.ldq, kh, a.dk, s.row[0], tid);
    fg.from(a, hd, s.row[0], t0, tid);
    const float* const S = n > 0 ? kept_before<DKP, VW>(a, n, bh) : nullptr;
    const float* const S0 = a.s0 ? a.s0 + bh * ((int64_t)a.dk * a.dv) : nullptr;
    const float* const dS = kept_after<DKP, VW>(a, n, bh);
    const uint16_t *const U = kept_columns<TX, VW>(a.u, a, n, bh), *const dR = kept_columns<TX, VW>(a.dr_rows, a, n, bh);
    const T* const d_o = static_cast<const T*>(a.d_o) + (int64_t)hd.h * a.dv;
    f32x4_t pair_q[(10 + W - 1) / W], pair_k[(10 + W - 1) / W], sq[NB], sk[NB], su[NB];
#pragma unroll
    for (int k = 0; k < (10 + W - 1) / W; ++k) pair_q[k] = pair_k[k] = zero;
#pragma unroll
    for (int I = 0; I < NB; ++I) sq[I] = sk[I] = su[I] = zero;
    // a slice on its way: pieces of eight columns of dO, of eight frames of U and dR, of
    // four keys of S and dS
    constexpr int NC = (TX * 256 + TH - 1) / TH, NS = 8 * DKP / TH;
    Eight<T> so;
    u32x4_t su4[NC], sr4[NC];
    f32x4_t ss[NS], sd[NS];
    auto arrive = [&](int c0) {
      {
        const int row = (tid >> 2) & 63, u = tid & 3, more = a.dv - c0 - 8 * u;
        const T* const p = d_o + s.row[0][row] * a.lddo + c0 + 8 * u;
        if (a.dv % 8 == 0) {
          so.load(p + min(more - 8, 0));
          if (more < 8) so.zero();
        } else {
          so.load(p, more);
        }
      }
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int at = min(i * TH + tid, TX * 256 - 1), e = at >> 8, row = (at >> 3) & 31, u = at & 7;
        const int from = (e * VP + c0 + row) * C + 8 * u;
        su4[i] = *reinterpret_cast<const u32x4_t*>(U + from);
        sr4[i] = *reinterpret_cast<const u32x4_t*>(dR + from);
      }
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        const int at = i * TH + tid, row = at / (DKP / 4), u = at % (DKP / 4);
        sd[i] = *reinterpret_cast<const f32x4_t*>(dS + (c0 + row) * DKP + 4 * u);
        ss[i] = zero;
        if (S) {
          ss[i] = *reinterpret_cast<const f32x4_t*>(S + (c0 + row) * DKP + 4 * u);
        } else if (S0) {  // (as it lies in memory: columns side by side)
          const int col = c0 + at % 32, key = 4 * (at / 32);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float x = S0[min(key + r, a.dk - 1) * a.dv + min(col, a.dv - 1)];
            ss[i][r] = key + r < a.dk && col < a.dv ? x : 0.f;
          }
        }
      }
    };
    arrive(0);
    for (int c0 = 0; c0 < a.dv; c0 += 32) {
      if (tid < 256) {
        const int row = tid >> 2, u = tid & 3;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int w = 2 * u + half, slot = (w & 3) * 2 + (w >> 2);
          const Piece<TI> v = so.piece(half);
#pragma unroll
          for (int e = 0; e < TI; ++e) *reinterpret_cast<u32x2_t*>(all.slice.dO.at[e] + place<32>(row, slot >> 1) + (slot & 1) * 8) = v.t[e];
        }
      }
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int at = i * TH + tid, e = at >> 8, row = (at >> 3) & 31, u = at & 7;
        if (at < TX * 256) {
          *reinterpret_cast<u32x4_t*>(all.slice.u[e] + row * FRAMES + 16 * u) = su4[i];
          *reinterpret_cast<u32x4_t*>(all.slice.dR[e] + row * FRAMES + 16 * u) = sr4[i];
        }
      }
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        const int at = i * TH + tid, row = at / (DKP / 4), u = at % (DKP / 4);
        const int mine = S ? row * KEYS + 8 * u : at % 32 * KEYS + 8 * (at / 32);
        const Piece<TX> x = split<TX>(ss[i]), y = split<TX>(sd[i]);
#pragma unroll
        for (int e = 0; e < TX; ++e) {
          *reinterpret_cast<u32x2_t*>(all.slice.S[e] + mine) = x.t[e];
          *reinterpret_cast<u32x2_t*>(all.slice.dS[e] + row * KEYS + 8 * u) = y.t[e];
        }
      }
      __syncthreads();
      if (c0 + 32 < a.dv) arrive(c0 + 32);
      // column 16 j + lane % 16 of those over rows 4 (lane / 16) and on, of both halves of the 32
      auto over = [&](const auto& m, int pitch, int j, Piece<TX>& x0, Piece<TX>& x1) {
        const int at = (4 * g4 + (l16 >> 2)) * pitch + (16 * j + 4 * (lane & 3)) * 2;
#pragma unroll
        for (int e = 0; e < TX; ++e) {
          x0.t[e] = turned(m[e] + at);
          x1.t[e] = turned(m[e] + at + 16 * pitch);
        }
      };
      Piece<TX> s0, s1, d0, d1;
      over(all.slice.S, KEYS, wave, s0, s1);
      over(all.slice.dS, KEYS, wave, d0, d1);
#pragma unroll
      for (int I = 0; I < NB; ++I) {
        Piece<TI> o0, o1;
        Piece<TX> x0, x1;
        rows_of(all.slice.dO, I, 0, lane, o0, o1);
        mma<TX, TI>(sq[I], s0, s1, o0, o1);
        over(all.slice.dR, FRAMES, I, x0, x1);
        mma<TX, TX>(sk[I], s0, s1, x0, x1);
        over(all.slice.u, FRAMES, I, x0, x1);
        mma<TX, TX>(su[I], d0, d1, x0, x1);
      }
#pragma unroll
      for (int k = 0; k < (10 + W - 1) / W; ++k) {  // ten tiles of U dO^T and of U dR^T
        const int at = wave + W * k;
        if (at >= 10) break;
        const int I = block_row(at), J = at - lower(I, 0);
        Piece<TI> o0, o1;
        Piece<TX> u0, u1, x0, x1;
        over(all.slice.u, FRAMES, J, u0, u1);
        rows_of(all.slice.dO, I, 0, lane, o0, o1);
        mma<TX, TI>(pair_q[k], u0, u1, o0, o1);
        over(all.slice.dR, FRAMES, I, x0, x1);
        mma<TX, TX>(pair_k[k], u0, u1, x0, x1);
      }
      __syncthreads();
    }
    {  // (places in LDS are made again here: kept through the slices, they were spilled)
      const int tid = this_thread(), lane = tid & 63, l16 = lane & 15, g4 = lane >> 4;
      fk.lengths(s.rk, a.eps, left, tid);
      fq.lengths(s.rq, a.eps, left, tid);
      fk.store(all.pairs.k, tid);
      fq.store(all.pairs.q, tid);
      fg.store(s, rate_of(a, hd.h), left, 0, tid);
      __syncthreads();
      if (wave == W - 1) combine(s, lane);
#pragma unroll
      for (int I = 0; I < NB; ++I) {
        const int i = 16 * I + l16;
        const f32x4_t q = values(row4_of(all.pairs.q, I, wave, lane)), k = values(row4_of(all.pairs.k, I, wave, lane));
        float qs = 0.f, ks = 0.f, ku = 0.f;
#pragma unroll
        for (int r = 0; r < 4; ++r) qs = fmaf(q[r], sq[I][r], qs), ks = fmaf(k[r], sk[I][r], ks), ku = fmaf(k[r], su[I][r], ku);
        float y = s.g[i] * (s.rq[i] * qs - s.beta[i] * s.rk[i] * ks), z = s.end[i] * s.rk[i] * ku;
        y += __shfl_xor(y, 16, 64);
        z += __shfl_xor(z, 16, 64);
        y += __shfl_xor(y, 32, 64);
        z += __shfl_xor(z, 32, 64);
        if (g4 == 0) {
          all.yz[0][wave][i] = y;
          all.yz[1][wave][i] = z;
        }
      }
#pragma unroll
      for (int k = 0; k < (10 + W - 1) / W; ++k) {
        const int at = wave + W * k;
        if (at >= 10) break;
        const int I = block_row(at), J = at - lower(I, 0), i = 16 * I + l16;
        f32x4_t qk = zero, kk = zero;
#pragma unroll
        for (int t = 0; t < DKP / 32; ++t) {
          Piece<TI> a0, a1, b0, b1;
          rows_of(all.pairs.k, J, t, lane, a0, a1);
          rows_of(all.pairs.k, I, t, lane, b0, b1);
          mma<TI, TI>(kk, a0, a1, b0, b1);
          rows_of(all.pairs.q, I, t, lane, b0, b1);
          mma<TI, TI>(qk, a0, a1, b0, b1);
        }
        const f32x4_t ch = rows4(s.ch, J, lane), cl = rows4(s.cl, J, lane), rk = rows4(s.rk, J, lane);
        const float hi = s.ch[i], lo = s.cl[i], f = s.rq[i], h = -s.beta[i] * s.rk[i];
        f32x4_t x, y;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int j = 16 * J + 4 * g4 + r;
          const float m = rk[r] * __builtin_amdgcn_exp2f((hi - ch[r]) + (lo - cl[r]));
          x[r] = j <= i ? f * m * pair_q[k][r] : 0.f;
          y[r] = j < i ? h * m * pair_k[k][r] : 0.f;
        }
        const Piece<TO> p = split<TO>(x), q = split<TO>(y);
#pragma unroll
        for (int e = 0; e < TO; ++e) {
          *reinterpret_cast<u32x2_t*>(all.pairs.qk[at][e] + spot(l16, g4)) = p.t[e];
          *reinterpret_cast<u32x2_t*>(all.pairs.kk[at][e] + spot(l16, g4)) = q.t[e];
        }
        crossing(x * qk + y * kk, I == J, all.cross[at], lane);
      }
      __syncthreads();
      if (wave == W - 1) {  // a frame a lane: the gradient of log a
        float* const part = a.parts + (int64_t)n * a.B * a.H + bh;
        const float e = crossed<W>(all.cross, all.yz, lane) + s.g[C - 1] * *part;
        const float rate = rate_of(a, hd.h), r = to_f32(fg.r), sr = sigm(r);
        if (lane < left) static_cast<T*>(a.dr)[s.row[0][lane] * a.lddr + hd.h] = from_f32<T>(-rate * sr * (sigm(-r) * e));
        const float sum = wave_sum_uniform(lane < left ? -e * sr : 0.f);
        if (lane == 0) *part = a.c * sum;
      }
#pragma unroll
      for (int I = 0; I < NB; ++I) {
        const int i = 16 * I + l16;
        dq[I] += sq[I] * s.gq[i];
        dk[I] += su[I] * s.gk[i] - sk[I] * s.bgk[i];
      }
#pragma unroll
      for (int I = 0; I < NB; ++I) {
        const Piece<TI> kI = columns_of(all.pairs.k, wave, I, lane), qI = columns_of(all.pairs.q, wave, I, lane);
#pragma unroll
        for (int J = 0; J < NB; ++J) {
          if (J >= I) mma<TI, TO>(dq[J], kI, block_of(all.pairs.qk[lower(J, I)], lane));
          if (J <= I) mma<TI, TO>(dk[J], qI, block_turned(all.pairs.qk[lower(I, J)], lane));
          if (J >= I) mma<TI, TO>(dk[J], kI, block_of(all.pairs.kk[lower(J, I)], lane));
          if (J <= I) mma<TI, TO>(dk[J], kI, block_turned(all.pairs.kk[lower(I, J)], lane));
        }
      }
    }
    if (member + 1 < group) __syncthreads();
  }
  // through the lengths: dq = t - q rq^2 (q . t), t what has been summed
  const int left = (a.lens ? a.lens[b] : a.T) - t0;
#pragma unroll
  for (int I = 0; I < NB; ++I) {
    const f32x4_t q = values(row4_of(all.pairs.q, I, wave, lane)) * dq[I], k = values(row4_of(all.pairs.k, I, wave, lane)) * dk[I];
    float x = (q[0] + q[1]) + (q[2] + q[3]), y = (k[0] + k[1]) + (k[2] + k[3]);
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
    const int i = 16 * I + l16, cols = a.dk - 16 * wave - 4 * g4;
    float x = 0.f, y = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) x += all.dots[0][w][i], y += all.dots[1][w][i];
    const f32x4_t vq = dq[I] - values(row4_of(all.pairs.q, I, wave, lane)) * (s.rq[i] * s.rq[i] * x);
    const f32x4_t vk = dk[I] - values(row4_of(all.pairs.k, I, wave, lane)) * (s.rk[i] * s.rk[i] * y);
    if (i >= left) continue;
    const int64_t row = s.row[0][i], at = (int64_t)kh * a.dk + 16 * wave + 4 * g4;
    put4(static_cast<T*>(a.dq) + row * a.lddq + at, cols, vq);
    put4(static_cast<T*>(a.dk_) + row * a.lddk + at, cols, vk);
  }
}

// dlam = sigm(lam) times the sum over chunks and sequences of parts.
__global__ __launch_bounds__(1024) void gd_dlam_kernel(GatedDelta a) {
  __shared__ float sum[32][33];
  const float s = column_sum(a.parts, (int64_t)((a.T + C - 1) / C) * a.B, a.H, sum);
  const int h = blockIdx.x * 32 + threadIdx.x;
  if (threadIdx.x < 32 && h < a.H) a.dlam[h] = s / (1.f + expf(-a.lam[h]));
}

template <typename T, int DKP, int W, bool ENDS> hipError_t pass(const GatedDelta& a, int segs, hipStream_t s) {
  constexpr int LDS = sizeof(Backward<T, DKP, W>);
  static_assert(LDS <= 160 * 1024, "a workgroup's LDS");
  static PerDevice ready;
  const hipError_t e = allow_lds<LDS>(reinterpret_cast<const void*>(&gd_backward_kernel<T, DKP, W, ENDS>), ready);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((gd_backward_kernel<T, DKP, W, ENDS>), dim3((unsigned)(a.B * a.H), segs), dim3(threads_of<W>), LDS, s, a);
  return hipGetLastError();
}
template <typename T, int DKP, int W> hipError_t backward(const GatedDelta& a, hipStream_t s) {
  constexpr int KEYS = sizeof(Keys<T, DKP>);
  static_assert(KEYS <= 160 * 1024, "a workgroup's LDS");
  static PerDevice ready;
  hipError_t e = allow_lds<KEYS>(reinterpret_cast<const void*>(&gd_keys_kernel<T, DKP, 16 * W>), ready);
  if (e == hipSuccess && a.segs > 1) {
    e = pass<T, DKP, W, true>(a, a.segs - 1, s);
    if (e == hipSuccess)
      hipLaunchKernelGGL((gd_join_back_kernel<DKP, W>), dim3((unsigned)(a.B * a.H), W), dim3(64), 0, s, a);
  }
  if (e == hipSuccess) e = pass<T, DKP, W, false>(a, a.segs, s);
  if (e != hipSuccess) return e;
  const unsigned chunks = (unsigned)((a.T + C - 1) / C) * a.B * a.G;
  if (chunks) hipLaunchKernelGGL((gd_keys_kernel<T, DKP, 16 * W>), dim3(chunks), dim3(DKP * 4), KEYS, s, a);
  hipLaunchKernelGGL(gd_dlam_kernel, dim3((unsigned)((a.H + 31) / 32)), dim3(1024), 0, s, a);
  return hipGetLastError();
}

template <typename T> hipError_t sized(const GatedDelta& a, hipStream_t s) {
  if (a.dk <= 64) return a.dv <= 64 ? backward<T, 64, 4>(a, s) : backward<T, 64, 8>(a, s);
  return a.dv <= 64 ? backward<T, 128, 4>(a, s) : backward<T, 128, 8>(a, s);
}

}  // namespace

hipError_t gated_delta_backward(GatedDelta a, bool bf16, hipStream_t s) {
  return bf16 ? sized<bf16_t>(a, s) : sized<float>(a, s);
}

}  // namespace am
