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

template <typename T, int DKP, int W> struct Backward {
  Chunk<T, DKP, W, Terms<T>::X, 2> c;
  float rows[2][W][C];  // dO . O - dV . V and dR . U, of a wave's columns
  float end[W];         // <dS', S'>
};

// In order of time within a head, as the forward pass, and bound as it is: 256 x 64
// frames, 12 heads of 64 x 64: 222 us (435 MB, 2 TB/s; two workgroups a CU for their
// registers); utterances of 200 to 1500 frames, 64 of 6 heads of 128 x 128: 700 us, in
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
  if (seg > 0 && begin >= all_chunks) {
    if (!ENDS && threadIdx.x == 0) a.parts[seg * (int64_t)gridDim.x + bh] = 0.f;
    return;
  }
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
  float dlam = 0.f;  // (of a frame a lane of every chunk, in the last wave)
  int turn = 0;
  for (int n = chunks - 1; n >= begin; --n, turn ^= 1) {
    const int left = hd.len - n * C, tid = this_thread(), lane = tid & 63, l16 = lane & 15, g4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = 16 * wave + l16;
    // (A chunk's inputs arrive during the one before where only the gradient of the
    // state goes on.  With everything else in registers that would not fit: the compiler
    // then kept them in scratch memory, whose waits cost 10 % of the whole.)
    if (!ENDS) fetch(s.row[turn], max(n - 1, 0) * C, tid);
    const T r_now = fg.r;
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

    f32x4_t u[NB], o[NB], kd[NB];
#pragma unroll
    for (int I = 0; I < NB; ++I) u[I] = o[I] = kd[I] = zero;
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
        if constexpr (!ENDS) {
          mma<TI, TX>(u[I], a0, a1, s0, s1);
          rows_of(c.q, I, t, lane, a0, a1);
          mma<TX, TI>(o[I], s0, s1, a0, a1);
        }
      }
    }
    const float g_end = s.g[C - 1];
    end *= g_end;
#pragma unroll
    for (int I = 0; I < NB; ++I) {
      if constexpr (!ENDS) {
        u[I] = fv.column_values(wave, I, lane) * rows4(s.beta, I, lane) - u[I] * rows4(s.bgk, I, lane);
        o[I] *= s.gq[16 * I + l16];
      }
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
#pragma unroll
        for (int r4 = 0; r4 < 4; ++r4) end = fmaf(u[I][r4], kd[I][r4], end);
#pragma unroll
        for (int J = 0; J + 1 <= I; J += 2)
          mma<TX, TX>(o[I], up[J], up[J + 1], block_of(c.p[lower(I, J)], lane), block_of(c.p[lower(I, J + 1)], lane));
        if (I % 2 == 0) mma<TX, TX>(o[I], up[I], block_of(c.p[lower(I, I)], lane));
      }
      uint16_t* const keep = kept_columns<TO, W>(a.u, a, n, bh);
#pragma unroll
      for (int e = 0; e < TO; ++e)
#pragma unroll
        for (int I = 0; I < NB; ++I)
          *reinterpret_cast<u32x2_t*>(keep + (e * 16 * W + col) * C + 16 * I + 4 * g4) = up[I].t[e];
    }
    float y1[NB], y2[NB];
#pragma unroll
    for (int I = 0; I < NB; ++I) {
      if constexpr (ENDS) break;
      const f32x4_t x = fo.row_values(I, wave, lane) * o[I];
      y1[I] = (x[0] + x[1]) + (x[2] + x[3]);
    }
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
        const f32x4_t dv = dr * s.beta[16 * I + l16], x = dv * fv.row_values(I, wave, lane), y = dr * ut[I];
        y1[I] -= (x[0] + x[1]) + (x[2] + x[3]);
        y2[I] = (y[0] + y[1]) + (y[2] + y[3]);
        if (16 * I + l16 < left)
          put4(static_cast<T*>(a.dv_) + s.row[turn][16 * I + l16] * a.lddv + (int64_t)hd.h * a.dv + 16 * wave + 4 * g4,
               a.dv - 16 * wave - 4 * g4, dv);
      }
      uint16_t* const keep = kept_columns<TO, W>(a.dr_rows, a, n, bh);
      if constexpr (!ENDS)
#pragma unroll
      for (int e = 0; e < TO; ++e)
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
      y1[I] += __shfl_xor(y1[I], 16, 64);
      y2[I] += __shfl_xor(y2[I], 16, 64);
      y1[I] += __shfl_xor(y1[I], 32, 64);
      y2[I] += __shfl_xor(y2[I], 32, 64);
      if (g4 == 0) {
        all.rows[0][wave][16 * I + l16] = y1[I];
        all.rows[1][wave][16 * I + l16] = y2[I];
      }
    }
    end = wave_sum_uniform(end);
    if (lane == 0) all.end[wave] = end;
    __syncthreads();
    if (wave == W - 1) {  // a frame a lane: the gates' gradients
      float d = 0.f, e = 0.f, ends = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) d += all.rows[0][w][lane], e += all.rows[1][w][lane], ends += all.end[w];
#pragma unroll
      for (int k = 1; k < C; k <<= 1) {  // from this frame to the chunk's last
        const float above = __shfl_down(d, k, 64);
        if (lane + k < C) d += above;
      }
      d += ends;
      if (lane < left) {
        // Its gradient is a difference of sums that is as small as the decay itself; of one
        // below e^-69 only their rounding would be left, times any rate.
        const float sr = sigm(to_f32(r_now));
        const bool lost = rate * sr > 69.f;
        const int64_t row = s.row[turn][lane];
        if (lost) d = 0.f;
        static_cast<T*>(a.dr)[row * a.lddr + hd.h] = from_f32<T>(lost ? 0.f : -rate * sr * ((1.f - sr) * d));
        static_cast<T*>(a.db)[row * a.lddb + hd.h] = from_f32<T>(e * (1.f - s.beta[lane]));
        dlam -= d * sr;
      }
    }
    }
    __syncthreads();
  }
  if constexpr (ENDS) {
    store_kept<DKP>(segment<DKP, W>(a.seg_d, a, seg - 1, bh), column_of(threadIdx.x), threadIdx.x & 63, dS);
    return;
  }
  if (a.ds0 && seg == 0) store_state<DKP>(a.ds0 + bh * state, a, column_of(threadIdx.x), threadIdx.x & 63, dS);
  if (threadIdx.x >= threads_of<W> - 64) {
    dlam = wave_sum_uniform(dlam);
    if (threadIdx.x == threads_of<W> - 64) a.parts[seg * (int64_t)gridDim.x + bh] = a.c * dlam;
  }
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

// The gradients of q and k of a chunk of a key head, summed over its heads: a wave has
// 16 columns of them, a lane a frame of each block, so that what scales with a frame is
// a factor of a lane.  It goes through v's columns 32 at a time, then takes the sums
// over pairs of frames to K and Q, which have the same LDS by then.  Chunks are all
// independent here; 162 us for 256 x 64 frames, 12 heads of 64 x 64 (325 MB, 2 TB/s),
// 427 for the utterances: the LDS pipeline, vector and matrix instructions take about a
// third of it each, one after another between barriers.
template <typename T, int DKP> struct Keys {
  static constexpr int TI = Terms<T>::IN, TO = Terms<T>::OUT;
  static constexpr int FRAMES = C * 2 + 16, KEYS = DKP * 2 + 16;  // bytes of a row of columns, of states
  union {
    struct {
      Matrix<TI, 32> dO;
      uint8_t u[TO][32 * FRAMES], dR[TO][32 * FRAMES];  // 32 columns over frames
      uint8_t S[TO][32 * KEYS], dS[TO][32 * KEYS];      // and over keys
    } slice;
    struct {
      Matrix<TI, DKP> k, q;
      uint8_t qk[10][TO][512], kk[10][TO][512];
    } pairs;
  };
  float dots[2][DKP / 16][C];
  Gates s;
};

template <typename T, int DKP, int VP>
__global__ __launch_bounds__(DKP * 4, 2) void gd_keys_kernel(GatedDelta a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  Keys<T, DKP>& all = *reinterpret_cast<Keys<T, DKP>*>(lds);
  Gates& s = all.s;
  constexpr int TI = Terms<T>::IN, TO = Terms<T>::OUT, W = DKP / 16, TH = threads_of<W>, VW = VP / 16;
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
    if (left <= 0) return;  // (all heads of a sequence alike)
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
    const uint16_t *const U = kept_columns<TO, VW>(a.u, a, n, bh), *const dR = kept_columns<TO, VW>(a.dr_rows, a, n, bh);
    const T* const d_o = static_cast<const T*>(a.d_o) + (int64_t)hd.h * a.dv;
    f32x4_t pair_q[(10 + W - 1) / W], pair_k[(10 + W - 1) / W], sq[NB], sk[NB], su[NB];
#pragma unroll
    for (int k = 0; k < (10 + W - 1) / W; ++k) pair_q[k] = pair_k[k] = zero;
#pragma unroll
    for (int I = 0; I < NB; ++I) sq[I] = sk[I] = su[I] = zero;
    // a slice on its way: pieces of eight columns of dO, of eight frames of U and dR, of
    // four keys of S and dS
    constexpr int NC = (TO * 256 + TH - 1) / TH, NS = 8 * DKP / TH;
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
        const int at = min(i * TH + tid, TO * 256 - 1), e = at >> 8, row = (at >> 3) & 31, u = at & 7;
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
        if (at < TO * 256) {
          *reinterpret_cast<u32x4_t*>(all.slice.u[e] + row * FRAMES + 16 * u) = su4[i];
          *reinterpret_cast<u32x4_t*>(all.slice.dR[e] + row * FRAMES + 16 * u) = sr4[i];
        }
      }
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        const int at = i * TH + tid, row = at / (DKP / 4), u = at % (DKP / 4);
        const int mine = S ? row * KEYS + 8 * u : at % 32 * KEYS + 8 * (at / 32);
        const Piece<TO> x = split<TO>(ss[i]), y = split<TO>(sd[i]);
#pragma unroll
        for (int e = 0; e < TO; ++e) {
          *reinterpret_cast<u32x2_t*>(all.slice.S[e] + mine) = x.t[e];
          *reinterpret_cast<u32x2_t*>(all.slice.dS[e] + row * KEYS + 8 * u) = y.t[e];
        }
      }
      __syncthreads();
      if (c0 + 32 < a.dv) arrive(c0 + 32);
      // column 16 j + lane % 16 of those over rows 4 (lane / 16) and on, of both halves of the 32
      auto over = [&](const auto& m, int pitch, int j, Piece<TO>& x0, Piece<TO>& x1) {
        const int at = (4 * g4 + (l16 >> 2)) * pitch + (16 * j + 4 * (lane & 3)) * 2;
#pragma unroll
        for (int e = 0; e < TO; ++e) {
          x0.t[e] = turned(m[e] + at);
          x1.t[e] = turned(m[e] + at + 16 * pitch);
        }
      };
      Piece<TO> s0, s1, d0, d1;
      over(all.slice.S, KEYS, wave, s0, s1);
      over(all.slice.dS, KEYS, wave, d0, d1);
#pragma unroll
      for (int I = 0; I < NB; ++I) {
        Piece<TI> o0, o1;
        Piece<TO> x0, x1;
        rows_of(all.slice.dO, I, 0, lane, o0, o1);
        mma<TO, TI>(sq[I], s0, s1, o0, o1);
        over(all.slice.dR, FRAMES, I, x0, x1);
        mma<TO, TO>(sk[I], s0, s1, x0, x1);
        over(all.slice.u, FRAMES, I, x0, x1);
        mma<TO, TO>(su[I], d0, d1, x0, x1);
      }
#pragma unroll
      for (int k = 0; k < (10 + W - 1) / W; ++k) {  // ten tiles of U dO^T and of U dR^T
        const int at = wave + W * k;
        if (at >= 10) break;
        const int I = block_row(at), J = at - lower(I, 0);
        Piece<TI> o0, o1;
        Piece<TO> u0, u1, x0, x1;
        over(all.slice.u, FRAMES, J, u0, u1);
        rows_of(all.slice.dO, I, 0, lane, o0, o1);
        mma<TO, TI>(pair_q[k], u0, u1, o0, o1);
        over(all.slice.dR, FRAMES, I, x0, x1);
        mma<TO, TO>(pair_k[k], u0, u1, x0, x1);
      }
      __syncthreads();
    }
    fk.lengths(s.rk, a.eps, left, tid);
    fq.lengths(s.rq, a.eps, left, tid);
    fk.store(all.pairs.k, tid);
    fq.store(all.pairs.q, tid);
    fg.store(s, rate_of(a, hd.h), left, 0, tid);
    __syncthreads();
    if (wave == W - 1) combine(s, lane);
#pragma unroll
    for (int k = 0; k < (10 + W - 1) / W; ++k) {
      const int at = wave + W * k;
      if (at >= 10) break;
      const int I = block_row(at), J = at - lower(I, 0), i = 16 * I + l16;
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
    }
    __syncthreads();
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

// dlam = sigm(lam) times the sum over segments and sequences of parts.
__global__ __launch_bounds__(1024) void gd_dlam_kernel(GatedDelta a) {
  __shared__ float sum[32][33];
  const float s = column_sum(a.parts, (int64_t)a.segs * a.B, a.H, sum);
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
