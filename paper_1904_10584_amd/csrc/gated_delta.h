// What the passes of the gated delta rule share: a chunk of 64 frames of one head in
// LDS, and products of its matrices with columns that stay in registers.
//
// Per head, S [dk][dv] over frames t (k and q of unit length):
//   S_t = a_t S_{t-1} + beta_t k_t (v_t - a_t S_{t-1}^T k_t)^T,   o_t = S_t^T q_t.
// Over a chunk that starts from S, with c_i the sum of log a up to frame i, g_i =
// e^c_i and M_ij = e^(c_i - c_j) for j <= i:
//   R = diag(beta) (V - diag(g) K S)          what each frame would add by itself,
//   (I + L) U = R,  L_ij = beta_i M_ij (k_i k_j), j < i,
//   O = diag(g) Q S + P U,  P_ij = M_ij (q_i k_j), j <= i,
//   S' = g_end S + K^T diag(M_end) U.
// Every column of S, R, U and O goes its way alone, so a wave keeps its columns of
// them in registers from one product to the next: what a 16 x 16 product leaves in a
// lane (column lane % 16, rows 4 (lane / 16) + 0..3) is, as it is, the right operand of
// the next one.  The left operands (K, Q, their transposes, L, P) are the same for all
// columns and lie in LDS.  (I + L) U = R is solved block after block of 16 rows with
// the inverses of I + L's diagonal blocks, which come from substitution: frames that
// repeat a key make the powers of L grow, but not its inverse.
//
// Inputs in bf16 enter the matrix cores as they are; their lengths and decays are
// factors of rows.  What is held in 32 bits (states, U, L, P, inputs in fp32) enters as
// three terms of 8 bits each, which leave nothing of its 24 bits; products of terms
// below the last place are left out.  (Two terms left states, 4e-6, and the gradient of
// lam, up to 3e-5, further off than 32 bits do.)  Two terms, off by 2^-18, serve where a
// sum is only rounded to bf16: O, and the gradients of q and k.
#pragma once

#include "am_device.h"
#include "am_internal.h"
#include "per_device.h"

namespace am {
namespace gd {

// Dynamic LDS of more than 64 KiB for a kernel, set once a device.
template <int BYTES> hipError_t allow_lds(const void* kernel, PerDevice& ready) {
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e == hipSuccess)
    e = ready.once(device, [&] { return hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, BYTES); });
  return e;
}

constexpr int C = GD_CHUNK, NB = C / 16;  // frames of a chunk, blocks of 16
constexpr int THREADS = 256, WAVES = 4;

typedef short s16x4_t __attribute__((ext_vector_type(4)));

template <typename T> struct Terms;
template <> struct Terms<bf16_t> { static constexpr int IN = 1, X = 3, OUT = 2; };
template <> struct Terms<float> { static constexpr int IN = 3, X = 3, OUT = 3; };

template <int N> struct Piece { uint2 t[N]; };  // four elements in N terms
template <int M, int N> __device__ __forceinline__ Piece<M> first(const Piece<N>& p) {
  Piece<M> q;
#pragma unroll
  for (int i = 0; i < M; ++i) q.t[i] = p.t[i];
  return q;
}

// Two elements rounded to nearest even, in one word.  (The empty statement keeps the word
// whole: taken apart again, each half became a conversion of its own.  The conversion
// itself is the compiler's, which keeps the distance that it needs from a product whose
// result it reads.)
__device__ __forceinline__ uint32_t pair_bf16(float a, float b) {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  typedef float f2 __attribute__((ext_vector_type(2)));
  uint32_t r = __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{a, b}, b2));
  asm("" : "+v"(r));
  return r;
}
template <int N> __device__ __forceinline__ Piece<N> split(f32x4_t v) {
  Piece<N> p;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    p.t[i] = make_uint2(pair_bf16(v[0], v[1]), pair_bf16(v[2], v[3]));
    if (i + 1 < N) {
      v[0] -= __uint_as_float(p.t[i].x << 16);
      v[1] -= __uint_as_float(p.t[i].x & 0xffff0000u);
      v[2] -= __uint_as_float(p.t[i].y << 16);
      v[3] -= __uint_as_float(p.t[i].y & 0xffff0000u);
    }
  }
  return p;
}

__device__ __forceinline__ bf16x8_t join(uint2 a, uint2 b) {
  return __builtin_bit_cast(bf16x8_t, make_uint4(a.x, a.y, b.x, b.y));
}
// acc += A B over 16, or over two blocks of 16, of the inner axis; small terms first.
// Over 16, an instruction of 32 takes two products of terms.  (Instructions of 16 are
// not used: one that added to what an instruction of 32 had just written gave wrong
// sums, since the compiler left too little room between the two.)
template <int TA, int TB>
__device__ __forceinline__ void mma(f32x4_t& acc, const Piece<TA>& a, const Piece<TB>& b) {
  constexpr int N = TA > TB ? TA : TB;
  uint2 wa = make_uint2(0, 0), wb = wa;
  int held = 0;
#pragma unroll
  for (int s = N - 1; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < TA; ++i)
      if (s - i >= 0 && s - i < TB) {
        if (held) {
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(join(wa, a.t[i]), join(wb, b.t[s - i]), acc, 0, 0, 0);
          held = 0;
        } else {
          wa = a.t[i];
          wb = b.t[s - i];
          held = 1;
        }
      }
  if (held) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(join(wa, make_uint2(0, 0)), join(wb, make_uint2(0, 0)), acc, 0, 0, 0);
}
template <int TA, int TB>
__device__ __forceinline__ void mma(f32x4_t& acc, const Piece<TA>& a0, const Piece<TA>& a1, const Piece<TB>& b0,
                                    const Piece<TB>& b1) {
  constexpr int N = TA > TB ? TA : TB;
#pragma unroll
  for (int s = N - 1; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < TA; ++i)
      if (s - i >= 0 && s - i < TB)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(join(a0.t[i], a1.t[i]), join(b0.t[s - i], b1.t[s - i]), acc, 0, 0, 0);
}

// Rows of any element alignment, in pieces.
typedef uint32_t u32x4_u __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_a __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x2_a __attribute__((ext_vector_type(2), aligned(4)));
typedef uint32_t u32_u __attribute__((aligned(2)));

// A chunk of a head in LDS.  A row of K or Q has its pieces of four columns, of each 32,
// in the order 0 4 1 5 2 6 3 7: the two that a lane takes for a step of 32 lie together.
template <typename T, int DKP> struct Staged {
  static constexpr int TI = Terms<T>::IN, TX = Terms<T>::X;
  static constexpr int PITCH = DKP * 2 + 16;  // bytes of a row
  uint8_t k[TI][C * PITCH], q[TI][C * PITCH];
  float ch[C], cl[C];          // c, and what is left of it behind 24 bits
  float g[C], end[C], beta[C], rk[C], rq[C];  // e^c, e^(c_end - c), gates, 1 / lengths
  float bgk[C], gq[C], gk[C];  // beta g rk, g rq, end rk
};
// PT: terms of P.
template <typename T, int DKP, int PT> struct Chunk : Staged<T, DKP> {
  static constexpr int TX = Terms<T>::X;
  uint8_t l[6][TX][512], d[NB][TX][512], p[10][PT][512];  // blocks of 16 x 16: -L below the diagonal,
                                                          // (I + L)^-1 on it, P
  float n[NB][260];            // L on the diagonal, transposed
};

// Eight columns of a row, zeros past `cols`.
__device__ __forceinline__ void load8(const bf16_t* p, int left, float (&v)[8]) {
  if (left >= 8) {
    const u32x4_u u = *reinterpret_cast<const u32x4_u*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(u[i] << 16);
      v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? bf16_to_f32(p[i]) : 0.f;
  }
}
__device__ __forceinline__ void load8(const float* p, int left, float (&v)[8]) {
  if (left >= 8) {
    const f32x4_a a = *reinterpret_cast<const f32x4_a*>(p), b = *reinterpret_cast<const f32x4_a*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : 0.f;
  }
}

// The sequence and head of a workgroup, and where its frames' rows are.
struct Head {
  int b, h, kh, len;  // sequence, head, key head, frames
  const int32_t* offs;
  int B;
  __device__ Head(const GatedDelta& a, int bh) {
    b = bh / a.H;
    h = bh % a.H;
    kh = h / (a.H / a.G);
    len = a.lens ? a.lens[b] : a.T;
    offs = a.offs;
    B = a.B;
  }
  __device__ int64_t row(int t) const { return offs ? (int64_t)offs[t] + b : (int64_t)t * B + b; }
};

// The sum over each group of 8 or 16 lanes, in every one of them.
template <int LANES> __device__ __forceinline__ float lanes_sum(float v) {
  v += lanes_moved<0xB1>(v);
  v += lanes_moved<0x4E>(v);
  v += lanes_moved<0x141>(v);
  if constexpr (LANES == 16) v += lanes_moved<0x140>(v);
  return v;
}

// K, Q and the gates of a chunk on their way from memory.
template <typename T, int DKP> struct Fetched {
  static constexpr int PER_ROW = DKP / 8, PIECES = C * PER_ROW / THREADS;
  float k[PIECES][8], q[PIECES][8];
  float r, b;
  __device__ __forceinline__ void from(const GatedDelta& a, const Head& hd, int t0) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int at = threadIdx.x + i * THREADS, t = t0 + at / PER_ROW, u = at % PER_ROW, left = a.dk - 8 * u;
      if (t < hd.len && left > 0) {
        const int64_t row = hd.row(t), col = (int64_t)hd.kh * a.dk + 8 * u;
        load8(static_cast<const T*>(a.k) + row * a.ldk + col, left, k[i]);
        load8(static_cast<const T*>(a.q) + row * a.ldq + col, left, q[i]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) k[i][j] = q[i][j] = 0.f;
      }
    }
    if (threadIdx.x < C) {
      const int t = t0 + threadIdx.x;
      if (t < hd.len) {
        const int64_t row = hd.row(t);
        r = to_f32(static_cast<const T*>(a.r)[row * a.ldr + hd.h]);
        b = to_f32(static_cast<const T*>(a.b)[row * a.ldb + hd.h]);
      }
    }
  }
};

// Writes a chunk's K, Q, lengths and gates.  (Ends without a barrier.)
template <typename T, int DKP>
__device__ __forceinline__ void stage(Staged<T, DKP>& s, const Fetched<T, DKP>& f, float eps, float rate, int left) {
  typedef Fetched<T, DKP> F;
  constexpr int TI = Terms<T>::IN;
#pragma unroll
  for (int i = 0; i < F::PIECES; ++i) {
    const int at = threadIdx.x + i * THREADS, row = at / F::PER_ROW, u = at % F::PER_ROW;
    float sk = 0.f, sq = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) sk = fmaf(f.k[i][j], f.k[i][j], sk), sq = fmaf(f.q[i][j], f.q[i][j], sq);
    sk = lanes_sum<F::PER_ROW>(sk);
    sq = lanes_sum<F::PER_ROW>(sq);
    if (u == 0) {
      s.rk[row] = 1.f / sqrtf(sk + eps);
      s.rq[row] = 1.f / sqrtf(sq + eps);
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int p = 2 * (u & 3) + half, slot = (p & 3) * 2 + (p >> 2);  // of the eight pieces of 32 columns
      const int to = row * Staged<T, DKP>::PITCH + (u >> 2) * 64 + slot * 8;
      const f32x4_t kv = {f.k[i][4 * half], f.k[i][4 * half + 1], f.k[i][4 * half + 2], f.k[i][4 * half + 3]};
      const f32x4_t qv = {f.q[i][4 * half], f.q[i][4 * half + 1], f.q[i][4 * half + 2], f.q[i][4 * half + 3]};
      const Piece<TI> kp = split<TI>(kv), qp = split<TI>(qv);
#pragma unroll
      for (int e = 0; e < TI; ++e) {
        *reinterpret_cast<uint2*>(s.k[e] + to) = kp.t[e];
        *reinterpret_cast<uint2*>(s.q[e] + to) = qp.t[e];
      }
    }
  }
  if (threadIdx.x < C) {  // one wave: the decays' sums in 64 bits
    const int t = threadIdx.x;
    const bool live = t < left;
    double c = live ? (double)(-rate * sigm(f.r)) : 0.0;
#pragma unroll
    for (int o = 1; o < C; o <<= 1) {
      const double below = __shfl_up(c, o, 64);
      if (t >= o) c += below;
    }
    const double last = __shfl(c, C - 1, 64);
    const float hi = (float)c;
    s.ch[t] = hi;
    s.cl[t] = (float)(c - (double)hi);
    s.g[t] = expf(hi);
    s.end[t] = expf((float)(last - c));
    s.beta[t] = live ? sigm(f.b) : 0.f;
  }
}

// Left operands: rows 16 I + lane % 16 of K or Q over columns 32 t and on ...
template <typename T, int DKP>
__device__ __forceinline__ void rows_of(const uint8_t (&m)[Terms<T>::IN][C * Staged<T, DKP>::PITCH], int I, int t, int lane,
                                        Piece<Terms<T>::IN>& a0, Piece<Terms<T>::IN>& a1) {
#pragma unroll
  for (int e = 0; e < Terms<T>::IN; ++e) {
    const uint4 u = *reinterpret_cast<const uint4*>(m[e] + (16 * I + (lane & 15)) * Staged<T, DKP>::PITCH + t * 64 + (lane >> 4) * 16);
    a0.t[e] = make_uint2(u.x, u.y);
    a1.t[e] = make_uint2(u.z, u.w);
  }
}
// ... and of their transposes: columns 16 t + lane % 16 over frames of block I.  A
// group of 16 lanes reads 4 rows of 16 columns, and each lane gets a column's four.
__device__ __forceinline__ uint2 turned(const uint8_t* p) {
  typedef __attribute__((address_space(3))) s16x4_t* At;
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(p)));
}
template <typename T, int DKP>
__device__ __forceinline__ Piece<Terms<T>::IN> columns_of(const uint8_t (&m)[Terms<T>::IN][C * Staged<T, DKP>::PITCH], int t, int I,
                                                          int lane) {
  Piece<Terms<T>::IN> a;
  const int row = 16 * I + (lane >> 4) * 4 + ((lane & 15) >> 2), slot = (lane & 3) * 2 + (t & 1);
#pragma unroll
  for (int e = 0; e < Terms<T>::IN; ++e) a.t[e] = turned(m[e] + row * Staged<T, DKP>::PITCH + (t >> 1) * 64 + slot * 8);
  return a;
}
// A block of 16 x 16, and its transpose.
template <int TX> __device__ __forceinline__ Piece<TX> block_of(const uint8_t (&m)[TX][512], int lane) {
  Piece<TX> a;
#pragma unroll
  for (int e = 0; e < TX; ++e) a.t[e] = *reinterpret_cast<const uint2*>(m[e] + (lane & 15) * 32 + (lane >> 4) * 8);
  return a;
}
template <int TX> __device__ __forceinline__ Piece<TX> block_turned(const uint8_t (&m)[TX][512], int lane) {
  Piece<TX> a;
#pragma unroll
  for (int e = 0; e < TX; ++e) a.t[e] = turned(m[e] + ((lane >> 4) * 4 + ((lane & 15) >> 2)) * 32 + (lane & 3) * 8);
  return a;
}
__device__ __forceinline__ f32x4_t rows4(const float (&v)[C], int I, int lane) {  // of block I, this lane's
  return *reinterpret_cast<const f32x4_t*>(v + 16 * I + 4 * (lane >> 4));
}
constexpr int below(int I, int J) { return I * (I - 1) / 2 + J; }   // block of l
constexpr int lower(int I, int J) { return I * (I + 1) / 2 + J; }   // block of p

// L, P and the inverses of I + L's diagonal blocks from a staged chunk (behind a
// barrier; ends with one).
template <typename T, int DKP, int PT> __device__ __forceinline__ void triangles(Chunk<T, DKP, PT>& s) {
  constexpr int TI = Terms<T>::IN, TX = Terms<T>::X;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, g4 = lane >> 4;
  if (wave == 1) {
    const int t = lane;
    s.bgk[t] = s.beta[t] * s.g[t] * s.rk[t];
    s.gq[t] = s.g[t] * s.rq[t];
    s.gk[t] = s.end[t] * s.rk[t];
  }
#pragma unroll
  for (int m = 0; m < 5; ++m) {  // ten tiles of K K^T, ten of Q K^T
    const int job = wave + WAVES * m, at = job < 10 ? job : job - 10;
    const int I = at >= 6 ? 3 : at >= 3 ? 2 : at >= 1 ? 1 : 0, J = at - lower(I, 0);
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < DKP / 32; ++t) {
      Piece<TI> a0, a1, b0, b1;
      rows_of<T, DKP>(s.k, J, t, lane, a0, a1);
      if (job < 10) rows_of<T, DKP>(s.k, I, t, lane, b0, b1);
      else rows_of<T, DKP>(s.q, I, t, lane, b0, b1);
      mma<TI, TI>(acc, a0, a1, b0, b1);
    }
    // a lane has row i and columns j, j + 1, ... of the tile
    const int i = 16 * I + l16;
    const f32x4_t ch = rows4(s.ch, J, lane), cl = rows4(s.cl, J, lane), rk = rows4(s.rk, J, lane);
    const float hi = s.ch[i], lo = s.cl[i], f = job < 10 ? s.beta[i] * s.rk[i] : s.rq[i];
    f32x4_t v;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int j = 16 * J + 4 * g4 + r;
      const bool on = job < 10 ? j < i : j <= i;
      v[r] = on ? f * rk[r] * acc[r] * expf((hi - ch[r]) + (lo - cl[r])) : 0.f;
    }
    if (job >= 10) {
      const Piece<PT> p = split<PT>(v);
#pragma unroll
      for (int e = 0; e < PT; ++e) *reinterpret_cast<uint2*>(s.p[at][e] + l16 * 32 + g4 * 8) = p.t[e];
    } else if (I == J) {
#pragma unroll
      for (int r = 0; r < 4; ++r) s.n[I][(4 * g4 + r) * 16 + l16] = v[r];
    } else {
      const Piece<TX> p = split<TX>(-v);
#pragma unroll
      for (int e = 0; e < TX; ++e) *reinterpret_cast<uint2*>(s.l[at - I][e] + l16 * 32 + g4 * 8) = p.t[e];
    }
  }
  __syncthreads();
  if (wave == 0) {  // 16 lanes a block, a column each: substitution
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = i == l16 ? 1.f : 0.f;
#pragma unroll
    for (int j = 0; j < 15; ++j) {
#pragma unroll
      for (int i4 = (j + 1) / 4; i4 < 4; ++i4) {
        const f32x4_t v = *reinterpret_cast<const f32x4_t*>(&s.n[g4][j * 16 + 4 * i4]);
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (4 * i4 + r > j) x[4 * i4 + r] = fmaf(-v[r], x[j], x[4 * i4 + r]);
      }
    }
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      const Piece<TX> p = split<TX>(f32x4_t{x[4 * i4], x[4 * i4 + 1], x[4 * i4 + 2], x[4 * i4 + 3]});
#pragma unroll
      for (int e = 0; e < TX; ++e) {
        uint16_t* to = reinterpret_cast<uint16_t*>(s.d[g4][e]) + 4 * i4 * 16 + l16;
        to[0] = (uint16_t)p.t[e].x;
        to[16] = (uint16_t)(p.t[e].x >> 16);
        to[32] = (uint16_t)p.t[e].y;
        to[48] = (uint16_t)(p.t[e].y >> 16);
      }
    }
  }
  __syncthreads();
}

// U from R, in place, and U's terms: (I + L) U = R, block after block.
template <typename T, int DKP, int PT, int NT>
__device__ __forceinline__ void solve(const Chunk<T, DKP, PT>& s, int lane, f32x4_t (&u)[NB][NT], Piece<Terms<T>::X> (&up)[NB][NT]) {
  constexpr int TX = Terms<T>::X;
#pragma unroll
  for (int I = 0; I < NB; ++I) {
    if (I >= 2) {
      const Piece<TX> a0 = block_of(s.l[below(I, 0)], lane), a1 = block_of(s.l[below(I, 1)], lane);
#pragma unroll
      for (int n = 0; n < NT; ++n) mma<TX, TX>(u[I][n], a0, a1, up[0][n], up[1][n]);
    }
    if (I == 1 || I == 3) {
      const Piece<TX> a = block_of(s.l[below(I, I - 1)], lane);
#pragma unroll
      for (int n = 0; n < NT; ++n) mma<TX, TX>(u[I][n], a, up[I - 1][n]);
    }
    const Piece<TX> d = block_of(s.d[I], lane);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const Piece<TX> r = split<TX>(u[I][n]);
      u[I][n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      mma<TX, TX>(u[I][n], d, r);
      up[I][n] = split<TX>(u[I][n]);
    }
  }
}

// The columns of v (or of a matrix like it) that a wave has: NT a lane, side by side.
template <int NT> struct Columns {
  int first;  // this lane's first column
  int count;  // how many of its columns there are
  __device__ Columns(int dv) {
    first = NT * ((threadIdx.x >> 6) * 16 + (threadIdx.x & 15));
    count = dv - first < 0 ? 0 : dv - first < NT ? dv - first : NT;
  }
  __device__ __forceinline__ void load(const bf16_t* p, float (&v)[NT]) const {
    if (NT == 2 && count == 2) {
      const uint32_t u = *reinterpret_cast<const u32_u*>(p);
      v[0] = __uint_as_float(u << 16);
      v[NT - 1] = __uint_as_float(u & 0xffff0000u);
    } else {
#pragma unroll
      for (int n = 0; n < NT; ++n) v[n] = n < count ? bf16_to_f32(p[n]) : 0.f;
    }
  }
  __device__ __forceinline__ void load(const float* p, float (&v)[NT]) const {
    if (NT == 2 && count == 2) {
      const f32x2_a u = *reinterpret_cast<const f32x2_a*>(p);
      v[0] = u[0];
      v[NT - 1] = u[1];
    } else {
#pragma unroll
      for (int n = 0; n < NT; ++n) v[n] = n < count ? p[n] : 0.f;
    }
  }
  __device__ __forceinline__ void store(bf16_t* p, const float (&v)[NT]) const {
    if (NT == 2 && count == 2) {
      *reinterpret_cast<u32_u*>(p) = pair_bf16(v[0], v[NT - 1]);
    } else {
#pragma unroll
      for (int n = 0; n < NT; ++n)
        if (n < count) p[n] = f32_to_bf16(v[n]);
    }
  }
  __device__ __forceinline__ void store(float* p, const float (&v)[NT]) const {
    if (NT == 2 && count == 2) {
      *reinterpret_cast<f32x2_a*>(p) = f32x2_a{v[0], v[NT - 1]};
    } else {
#pragma unroll
      for (int n = 0; n < NT; ++n)
        if (n < count) p[n] = v[n];
    }
  }
};

// A state's columns from memory [dk][dv] (null: zero), and to it.
template <int DKP, int NT>
__device__ __forceinline__ void load_state(const float* m, const GatedDelta& a, const Columns<NT>& cols, int lane,
                                           f32x4_t (&S)[DKP / 16][NT]) {
#pragma unroll
  for (int t = 0; t < DKP / 16; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * t + 4 * (lane >> 4) + r;
      float v[NT];
      if (m && row < a.dk) {
        cols.load(m + (int64_t)row * a.dv + cols.first, v);
      } else {
#pragma unroll
        for (int n = 0; n < NT; ++n) v[n] = 0.f;
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) S[t][n][r] = v[n];
    }
}
template <int DKP, int NT>
__device__ __forceinline__ void store_state(float* m, const GatedDelta& a, const Columns<NT>& cols, int lane,
                                            const f32x4_t (&S)[DKP / 16][NT]) {
#pragma unroll
  for (int t = 0; t < DKP / 16; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * t + 4 * (lane >> 4) + r;
      float v[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) v[n] = S[t][n][r];
      if (row < a.dk) cols.store(m + (int64_t)row * a.dv + cols.first, v);
    }
}
// Rows of v, frames t0 and on: this lane's of each block of 16, zeros past the end.
template <typename T, int NT>
__device__ __forceinline__ void load_rows(const void* m, int64_t ld, const GatedDelta& a, const Head& hd, int t0,
                                          const Columns<NT>& cols, int lane, f32x4_t (&v)[NB][NT]) {
#pragma unroll
  for (int I = 0; I < NB; ++I)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int t = t0 + 16 * I + 4 * (lane >> 4) + r;
      float x[NT];
      if (t < hd.len) {
        cols.load(static_cast<const T*>(m) + hd.row(t) * ld + (int64_t)hd.h * a.dv + cols.first, x);
      } else {
#pragma unroll
        for (int n = 0; n < NT; ++n) x[n] = 0.f;
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) v[I][n][r] = x[n];
    }
}
template <typename T, int NT>
__device__ __forceinline__ void store_rows(void* m, int64_t ld, const GatedDelta& a, const Head& hd, int t0,
                                           const Columns<NT>& cols, int lane, const f32x4_t (&v)[NB][NT]) {
#pragma unroll
  for (int I = 0; I < NB; ++I)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int t = t0 + 16 * I + 4 * (lane >> 4) + r;
      float x[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) x[n] = v[I][n][r];
      if (t < hd.len) cols.store(static_cast<T*>(m) + hd.row(t) * ld + (int64_t)hd.h * a.dv + cols.first, x);
    }
}

}  // namespace gd
}  // namespace am
