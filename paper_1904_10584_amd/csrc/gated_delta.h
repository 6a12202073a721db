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
// Every column of S, R, U and O goes its way alone, so a wave keeps 16 columns of them in
// registers from one product to the next: what a 16 x 16 product leaves in a lane
// (column lane % 16, rows 4 (lane / 16) + 0..3) is, as it is, an operand of the next
// one.  As its right operand the columns stay with their lanes; as its left one they
// come out transposed, a frame a lane and four columns side by side, which is how rows
// leave for memory.  The other operands (K, Q, their transposes, L, P) are the same for
// all columns and lie in LDS.  (I + L) U = R is solved block after block of 16 rows with
// the inverses of I + L's diagonal blocks, which come from substitution: frames that
// repeat a key make the powers of L grow, but not its inverse.
//
// Inputs in bf16 enter the matrix cores as they are; their lengths and decays are
// factors of rows.  What is held in 32 bits (states, U, L, P, inputs in fp32) enters as
// three terms of 8 bits each, which leave nothing of its 24 bits; products of terms
// below the last place are left out.  (Two terms left states, 4e-6, and the gradient of
// lam, up to 3e-5, further off than 32 bits do.)  Two terms, off by 2^-18, serve where a
// sum is only rounded to bf16: in O, and in what pairs of frames give the gradients of q
// and k.
//
// What bounds it: neither HBM nor the matrix cores, but a chunk's chain of dependent
// steps (staging, the triangles, the solve, the state), with two or three workgroups of
// a CU to fill the waits.  A chunk of 64 x 64 keeps the vector units busy for 25 to 37 %
// of its time, half of that splitting into terms, and the matrix cores for 8 to 10 %.
// Blocks of 16 rows in the order of `spot` and rows in that of `place` brought LDS bank
// conflicts from 12.2 M to 3.5 M cycles (256 sequences of one chunk, 12 heads).
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

typedef short s16x4_t __attribute__((ext_vector_type(4)));

template <typename T> struct Terms;
template <> struct Terms<bf16_t> { static constexpr int IN = 1, X = 3, OUT = 2; };
template <> struct Terms<float> { static constexpr int IN = 3, X = 3, OUT = 3; };

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
template <int N> struct Piece { u32x2_t t[N]; };  // four elements in N terms
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
    p.t[i] = u32x2_t{pair_bf16(v[0], v[1]), pair_bf16(v[2], v[3])};
    if (i + 1 < N) {
      v[0] -= __uint_as_float(p.t[i].x << 16);
      v[1] -= __uint_as_float(p.t[i].x & 0xffff0000u);
      v[2] -= __uint_as_float(p.t[i].y << 16);
      v[3] -= __uint_as_float(p.t[i].y & 0xffff0000u);
    }
  }
  return p;
}

__device__ __forceinline__ bf16x8_t join(u32x2_t a, u32x2_t b) {
  return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(a, b, 0, 1, 2, 3));
}
// acc += A B over 16, or over two blocks of 16, of the inner axis; small terms first.
// Over 16, an instruction of 32 takes two products of terms.  (Instructions of 16 are
// not used: one that added to what an instruction of 32 had just written gave wrong
// sums.  Why is not known.)
template <int TA, int TB>
__device__ __forceinline__ void mma(f32x4_t& acc, const Piece<TA>& a, const Piece<TB>& b) {
  constexpr int N = TA > TB ? TA : TB;
  u32x2_t wa = u32x2_t{0, 0}, wb = wa;
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
  if (held) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(join(wa, u32x2_t{0, 0}), join(wb, u32x2_t{0, 0}), acc, 0, 0, 0);
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
typedef uint32_t u32x2_u __attribute__((ext_vector_type(2), aligned(2)));
typedef float f32x4_a __attribute__((ext_vector_type(4), aligned(4)));

// A workgroup of W waves has 16 W columns of v: 64 or 128, as the padded heads have.
template <int W> constexpr int threads_of = 64 * W;
// Where 16 bytes of a row lie in LDS: rows that are read together, 8 next to one another
// (b128) or 4 by 4 (transposing), then meet in no bank, or in two.
template <int COLS> constexpr int pitch_of = COLS * 2;  // bytes of a row
template <int COLS> __device__ __forceinline__ int place(int row, int sixteen) {
  const int key = COLS == 32 ? (row >> 1) & 3 : (row & 1) << 2 | ((row >> 1) & 3);
  return row * pitch_of<COLS> + (sixteen ^ key) * 16;
}

// A chunk of a head in LDS.  A row has its pieces of four columns, of each 32, in the
// order 0 4 1 5 2 6 3 7: the two that a lane takes for a step of 32 are 16 bytes.
// Frames past a sequence's end are its last one again, whose row can be read, with
// beta, rk and rq 0: everything that they touch is multiplied by one of those.
struct Gates {
  float ch[C], cl[C];          // c log2(e), and what is left of it behind 24 bits
  float g[C], end[C], beta[C], rk[C], rq[C];  // e^c, e^(c_end - c), gates, 1 / lengths
  float bgk[C], gq[C], gk[C];  // beta g rk, g rq, end rk
  int32_t row[2][C];           // the frames' rows, of this chunk and of the next one
};
template <int N, int COLS> struct Matrix { uint8_t at[N][C * pitch_of<COLS>]; };  // in N terms
// PT: terms of P; R: matrices like v (v, and in the backward pass dO).  (Inputs in fp32
// would not leave room for those: they stay in memory.)  In the forward pass v has been
// read when L is written, and everywhere n when d is: with 46 instead of 60 KiB three
// workgroups with heads of 64 x 64 share a CU.
template <int TI, int TX, int W, int R> struct Below {
  Matrix<1, 16 * W> v[TI == 1 ? R : 0];
  uint8_t l[6][TX][512];                     // blocks of 16 x 16 of -L below the diagonal
};
template <int TX, int W> struct Below<1, TX, W, 1> {
  union {
    Matrix<1, 16 * W> v[1];
    uint8_t l[6][TX][512];
  };
};
template <typename T, int DKP, int W, int PT, int R> struct Chunk : Below<Terms<T>::IN, Terms<T>::X, W, R> {
  static constexpr int TI = Terms<T>::IN, TX = Terms<T>::X;
  Matrix<TI, DKP> k, q;
  union {
    float n[NB][16][20];                     // -L on the diagonal, transposed
    uint8_t d[NB][TX][528];                  // (I + L)^-1 there
  };
  uint8_t p[10][PT][512];                    // blocks of P
  Gates s;
};

// Eight columns of a row as they lie in memory.  load(p, left): `left` of them are there,
// which may be none; what lies before the row's end is read in their place, so that
// lanes without them need no branch.
template <typename T> struct Eight;
template <> struct Eight<bf16_t> {
  uint32_t w[4];
  __device__ __forceinline__ float at(int i) const { return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16); }
  __device__ __forceinline__ Piece<1> piece(int half) const { return {{u32x2_t{w[2 * half], w[2 * half + 1]}}}; }
  __device__ __forceinline__ void zero() { w[0] = w[1] = w[2] = w[3] = 0; }
  __device__ __forceinline__ void load(const bf16_t* p) {
    const u32x4_u u = *reinterpret_cast<const u32x4_u*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = u[i];
  }
  __device__ __forceinline__ void load(const bf16_t* p, int left) {
    uint32_t x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = p[min(i, left - 1)];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (2 * i < left ? x[2 * i] : 0u) | (2 * i + 1 < left ? x[2 * i + 1] << 16 : 0u);
  }
};
template <> struct Eight<float> {
  f32x4_t v[2];
  __device__ __forceinline__ float at(int i) const { return v[i >> 2][i & 3]; }
  __device__ __forceinline__ Piece<3> piece(int half) const { return split<3>(v[half]); }
  __device__ __forceinline__ void zero() { v[0] = v[1] = f32x4_t{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ void load(const float* p) {
    v[0] = *reinterpret_cast<const f32x4_a*>(p);
    v[1] = *reinterpret_cast<const f32x4_a*>(p + 4);
  }
  __device__ __forceinline__ void load(const float* p, int left) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = p[min(i, left - 1)];
      v[i >> 2][i & 3] = i < left ? x : 0.f;
    }
  }
};
// What terms stand for.
template <int N> __device__ __forceinline__ f32x4_t values(const Piece<N>& p) {
  f32x4_t v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int e = N - 1; e >= 0; --e)
    v += f32x4_t{__uint_as_float(p.t[e].x << 16), __uint_as_float(p.t[e].x & 0xffff0000u),
                 __uint_as_float(p.t[e].y << 16), __uint_as_float(p.t[e].y & 0xffff0000u)};
  return v;
}
// Four columns of a row to memory, `left` of them where that is less.
__device__ __forceinline__ void put4(bf16_t* p, int left, f32x4_t v) {
  const uint32_t lo = pair_bf16(v[0], v[1]), hi = pair_bf16(v[2], v[3]);
  if (left >= 4) {
    *reinterpret_cast<u32x2_u*>(p) = u32x2_u{lo, hi};
  } else {
    if (left > 0) p[0] = (uint16_t)lo;
    if (left > 1) p[1] = (uint16_t)(lo >> 16);
    if (left > 2) p[2] = (uint16_t)hi;
  }
}
__device__ __forceinline__ void put4(float* p, int left, f32x4_t v) {
  if (left >= 4) {
    *reinterpret_cast<f32x4_a*>(p) = v;
  } else {
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if (j < left) p[j] = v[j];
  }
}

// The column of v that a thread's lane has.
__device__ __forceinline__ int column_of(int tid) { return (tid >> 6) * 16 + (tid & 15); }

// A head's rate of decay.  What would pass 32 bits is their largest: with a gate that is
// shut, whose sigmoid is 0, it makes 0 and not a NaN.
__device__ __forceinline__ float rate_of(const GatedDelta& a, int h) {
  const float rate = a.c * softplus(a.lam[h]);
  return rate > 3.402823466e38f ? 3.402823466e38f : rate;
}

// The sequence and head of a workgroup.
struct Head {
  int b, h, kh, len;  // sequence, head, key head, frames
  __device__ Head(const GatedDelta& a, int bh) {
    b = bh / a.H;
    h = bh % a.H;
    kh = h / (a.H / a.G);
    len = a.lens ? a.lens[b] : a.T;
  }
  // the row of frame t, or of the last one
  __device__ __forceinline__ int row(const GatedDelta& a, int t) const {
    t = min(t, len - 1);
    return (a.offs ? a.offs[t] : t * a.B) + b;
  }
};

// The sum over each group of 8 or 16 lanes, in every one of them.
template <int LANES> __device__ __forceinline__ float lanes_sum(float v) {
  v += lanes_moved<0xB1>(v);
  v += lanes_moved<0x4E>(v);
  v += lanes_moved<0x141>(v);
  if constexpr (LANES == 16) v += lanes_moved<0x140>(v);
  return v;
}
// The sums of a wave's lanes up to each of them, in 64 bits: lane moves by 1, 2, 4 and 8
// within rows of 16, then the ends of rows (of two rows) to those behind them.
template <int CTRL, int ROWS> __device__ __forceinline__ double lanes_before(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, ROWS, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double sums_before(double c) {
  c += lanes_before<0x111, 0xf>(c);
  c += lanes_before<0x112, 0xf>(c);
  c += lanes_before<0x114, 0xf>(c);
  c += lanes_before<0x118, 0xf>(c);
  c += lanes_before<0x142, 0xa>(c);
  c += lanes_before<0x143, 0xc>(c);
  return c;
}

// Rows of COLS columns (`dim` of them there) of a chunk on their way from memory to LDS.
template <typename T, int COLS, int W> struct Rows {
  static constexpr int PER_ROW = COLS / 8, PIECES = C * PER_ROW / threads_of<W>;
  static_assert(PIECES >= 1, "every thread has a piece");
  Eight<T> v[PIECES];
  __device__ __forceinline__ void from(const void* m, int64_t ld, int head, int dim, const int32_t (&rows)[C], int tid) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int at = tid + i * threads_of<W>, u = at % PER_ROW, left = dim - 8 * u;
      const T* p = static_cast<const T*>(m) + rows[at / PER_ROW] * ld + (int64_t)head * dim + 8 * u;
      if (dim % 8 == 0) {
        v[i].load(p + min(left - 8, 0));
        if (dim < COLS && left < 8) v[i].zero();
      } else {
        v[i].load(p, left);
      }
    }
  }
  __device__ __forceinline__ void store(Matrix<Terms<T>::IN, COLS>& m, int tid) const {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int at = tid + i * threads_of<W>, u = at % PER_ROW;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int p = 2 * (u & 3) + half, slot = (p & 3) * 2 + (p >> 2);  // of the eight pieces of 32 columns
        const Piece<Terms<T>::IN> w = v[i].piece(half);
#pragma unroll
        for (int e = 0; e < Terms<T>::IN; ++e)
          *reinterpret_cast<u32x2_t*>(m.at[e] + place<COLS>(at / PER_ROW, (u >> 2) * 4 + (slot >> 1)) + (slot & 1) * 8) = w.t[e];
      }
    }
  }
  // 1 / sqrt(sum of squares + eps) of each row; 0 from row `left` on
  __device__ __forceinline__ void lengths(float (&out)[C], float eps, int left, int tid) const {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int at = tid + i * threads_of<W>, row = at / PER_ROW;
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) s = fmaf(v[i].at(j), v[i].at(j), s);
      s = lanes_sum<PER_ROW>(s);
      if (at % PER_ROW == 0) out[row] = row < left ? rsqrtf(s + eps) : 0.f;
    }
  }
};
// Rows of a matrix like v, 16 W columns of it: in LDS if they are bf16, which arrive
// while the chunk before is in hand; in memory if they are fp32.
template <typename T, int W> struct Values;
template <int W> struct Values<bf16_t, W> {
  Rows<bf16_t, 16 * W, W> v;
  const Matrix<1, 16 * W>* m;
  __device__ __forceinline__ void from(const void* p, int64_t ld, const Head& hd, int dv, const int32_t (&rows)[C], int tid) {
    v.from(p, ld, hd.h, dv, rows, tid);
  }
  __device__ __forceinline__ void store(Matrix<1, 16 * W>* to, const int32_t (&)[C], int tid) {
    v.store(*to, tid);
    m = to;
  }
  // columns 16 t + lane % 16 over frames of block I
  __device__ __forceinline__ Piece<1> column(int t, int I, int lane) const;
  __device__ __forceinline__ f32x4_t column_values(int t, int I, int lane) const;
};
template <int W> struct Values<float, W> {
  const float* p;
  int64_t ld;
  int dv;
  const int32_t* rows;
  __device__ __forceinline__ void from(const void* m, int64_t stride, const Head& hd, int cols, const int32_t (&)[C], int) {
    p = static_cast<const float*>(m) + (int64_t)hd.h * cols;
    ld = stride;
    dv = cols;
  }
  __device__ __forceinline__ void store(Matrix<1, 16 * W>*, const int32_t (&at)[C], int) { rows = at; }
  __device__ __forceinline__ f32x4_t column_values(int t, int I, int lane) const {
    const int col = 16 * t + (lane & 15);
    f32x4_t v;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float x = p[rows[16 * I + 4 * (lane >> 4) + r] * ld + min(col, dv - 1)];
      v[r] = col < dv ? x : 0.f;
    }
    return v;
  }
  __device__ __forceinline__ Piece<3> column(int t, int I, int lane) const { return split<3>(column_values(t, I, lane)); }
};
// The gates of a chunk and the rows of another one; the last wave's.
template <typename T, int W> struct GateRows {
  T r, b;
  int next;
  __device__ __forceinline__ static bool mine(int tid) { return tid >= threads_of<W> - C; }
  __device__ __forceinline__ void from(const GatedDelta& a, const Head& hd, const int32_t (&rows)[C], int next0, int tid) {
    if (!mine(tid)) return;
    const int t = tid & 63;
    const int64_t row = rows[t];
    r = static_cast<const T*>(a.r)[row * a.ldr + hd.h];
    b = static_cast<const T*>(a.b)[row * a.ldb + hd.h];
    next = hd.row(a, next0 + t);
  }
  // `left`: frames that the sequence has from here on
  __device__ __forceinline__ void store(Gates& s, float rate, int left, int turn, int tid) const {
    if (!mine(tid)) return;
    const int t = tid & 63;
    const bool live = t < left;
    // (2^-256 is a decay to nothing; a greater one would only cost the sums their places)
    const double step = (double)(-rate * sigm(to_f32(r))) * 1.4426950408889634;
    const double c = sums_before(live ? step < -256.0 ? -256.0 : step : 0.0);
    const double last = __shfl(c, C - 1, 64);
    const float hi = (float)c;
    s.ch[t] = hi;
    s.cl[t] = (float)(c - (double)hi);
    s.g[t] = __builtin_amdgcn_exp2f(hi);
    s.end[t] = __builtin_amdgcn_exp2f((float)(last - c));
    s.beta[t] = live ? sigm(to_f32(b)) : 0.f;
    s.row[turn ^ 1][t] = next;
  }
};

// Operands from LDS: rows 16 I + lane % 16 over columns 32 t and on ...
template <int N, int COLS>
__device__ __forceinline__ void rows_of(const Matrix<N, COLS>& m, int I, int t, int lane, Piece<N>& a0, Piece<N>& a1) {
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const u32x4_t u = *reinterpret_cast<const u32x4_t*>(m.at[e] + place<COLS>(lane & 15, t * 4 + (lane >> 4)) + 16 * I * pitch_of<COLS>);
    a0.t[e] = u.xy;
    a1.t[e] = u.zw;
  }
}
// (four of them: columns 16 t + 4 (lane / 16) and on)
template <int N, int COLS> __device__ __forceinline__ Piece<N> row4_of(const Matrix<N, COLS>& m, int I, int t, int lane) {
  Piece<N> a;
#pragma unroll
  for (int e = 0; e < N; ++e)
    a.t[e] = *reinterpret_cast<const u32x2_t*>(m.at[e] + place<COLS>(lane & 15, (t >> 1) * 4 + (lane >> 4)) +
                                               16 * I * pitch_of<COLS> + (t & 1) * 8);
  return a;
}
// ... and columns 16 t + lane % 16 over frames of block I.  A group of 16 lanes reads 4
// rows of 16 columns, and each lane gets a column's four.
__device__ __forceinline__ u32x2_t turned(const uint8_t* p) {
  typedef __attribute__((address_space(3))) s16x4_t* At;
  return __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((At)(p)));
}
template <int N, int COLS> __device__ __forceinline__ Piece<N> columns_of(const Matrix<N, COLS>& m, int t, int I, int lane) {
  Piece<N> a;
  const int row = (lane >> 4) * 4 + ((lane & 15) >> 2);  // (of a block: its key is that of every block's)
#pragma unroll
  for (int e = 0; e < N; ++e)
    a.t[e] = turned(m.at[e] + place<COLS>(row, (t >> 1) * 4 + (lane & 3)) + 16 * I * pitch_of<COLS> + (t & 1) * 8);
  return a;
}
template <int W> __device__ __forceinline__ Piece<1> Values<bf16_t, W>::column(int t, int I, int lane) const {
  return columns_of(*m, t, I, lane);
}
template <int W> __device__ __forceinline__ f32x4_t Values<bf16_t, W>::column_values(int t, int I, int lane) const {
  return values(columns_of(*m, t, I, lane));
}
// A block of 16 x 16 has columns 4 g to 4 g + 3 of all rows in 128 bytes, in an order in
// which neither the 16 lanes that read a column group nor those that read four rows of
// all of them (transposing) meet in a bank.
__device__ __forceinline__ int spot(int row, int g) { return g * 128 + (row ^ (4 * g)) * 8; }
// Such a block, and its transpose.
template <int TX, int S> __device__ __forceinline__ Piece<TX> block_of(const uint8_t (&m)[TX][S], int lane) {
  Piece<TX> a;
#pragma unroll
  for (int e = 0; e < TX; ++e) a.t[e] = *reinterpret_cast<const u32x2_t*>(m[e] + spot(lane & 15, lane >> 4));
  return a;
}
template <int TX, int S> __device__ __forceinline__ Piece<TX> block_turned(const uint8_t (&m)[TX][S], int lane) {
  Piece<TX> a;
#pragma unroll
  for (int e = 0; e < TX; ++e) a.t[e] = turned(m[e] + spot((lane >> 4) * 4 + ((lane & 15) >> 2), lane & 3));
  return a;
}
__device__ __forceinline__ f32x4_t rows4(const float (&v)[C], int I, int lane) {  // of block I, this lane's
  return *reinterpret_cast<const f32x4_t*>(v + 16 * I + 4 * (lane >> 4));
}
constexpr int below(int I, int J) { return I * (I - 1) / 2 + J; }   // block of l
constexpr int lower(int I, int J) { return I * (I + 1) / 2 + J; }   // block of p
__device__ __forceinline__ int block_row(int at) { return at >= 6 ? 3 : at >= 3 ? 2 : at >= 1 ? 1 : 0; }

__device__ __forceinline__ void combine(Gates& s, int t) {
  s.bgk[t] = s.beta[t] * s.g[t] * s.rk[t];
  s.gq[t] = s.g[t] * s.rq[t];
  s.gk[t] = s.end[t] * s.rk[t];
}

// x_i += n_i of lane J, x_J, for every i below J; and so on from column J + 1.
template <int J> __device__ __forceinline__ void substitute(float (&x)[16], const float (&n)[16]) {
  if constexpr (J < 15) {
#pragma unroll
    for (int i = J + 1; i < 16; ++i) x[i] = fmaf(lanes_moved<0x150 + J>(n[i]), x[J], x[i]);
    substitute<J + 1>(x, n);
  }
}

// Tile (I, J) of -L and, with OUT, of P from K K^T and Q K^T.
template <bool OUT, typename T, int DKP, int W, int PT, int R>
__device__ __forceinline__ void tile(Chunk<T, DKP, W, PT, R>& c, int I, int J, int lane) {
  constexpr int TI = Terms<T>::IN, TX = Terms<T>::X;
  const int l16 = lane & 15, g4 = lane >> 4, at = lower(I, J);
  const Gates& s = c.s;
  f32x4_t kk = {0.f, 0.f, 0.f, 0.f}, qk = kk;
#pragma unroll
  for (int t = 0; t < DKP / 32; ++t) {
    Piece<TI> a0, a1, b0, b1;
    rows_of(c.k, J, t, lane, a0, a1);
    rows_of(c.k, I, t, lane, b0, b1);
    mma<TI, TI>(kk, a0, a1, b0, b1);
    if constexpr (OUT) {
      rows_of(c.q, I, t, lane, b0, b1);
      mma<TI, TI>(qk, a0, a1, b0, b1);
    }
  }
  // a lane has row i and columns j, j + 1, ... of the tile
  const int i = 16 * I + l16;
  const f32x4_t ch = rows4(s.ch, J, lane), cl = rows4(s.cl, J, lane), rk = rows4(s.rk, J, lane);
  const float hi = s.ch[i], lo = s.cl[i], fk = -s.beta[i] * s.rk[i], fq = s.rq[i];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int j = 16 * J + 4 * g4 + r;
    const float m = rk[r] * __builtin_amdgcn_exp2f((hi - ch[r]) + (lo - cl[r]));
    kk[r] = j < i ? fk * kk[r] * m : 0.f;
    qk[r] = j <= i ? fq * qk[r] * m : 0.f;
  }
  if constexpr (OUT) {
    const Piece<PT> p = split<PT>(qk);
#pragma unroll
    for (int e = 0; e < PT; ++e) *reinterpret_cast<u32x2_t*>(c.p[at][e] + spot(l16, g4)) = p.t[e];
  }
  if (I == J) {
#pragma unroll
    for (int r = 0; r < 4; ++r) c.n[I][4 * g4 + r][l16] = kk[r];
  } else {
    const Piece<TX> w = split<TX>(kk);
#pragma unroll
    for (int e = 0; e < TX; ++e) *reinterpret_cast<u32x2_t*>(c.l[at - I][e] + spot(l16, g4)) = w.t[e];
  }
}

// L, P and the inverses of I + L's diagonal blocks from a staged chunk (behind a
// barrier; ends with one).  The first four waves make the tiles on the diagonal; then
// one wave inverts, and the others make the six tiles below.
template <bool OUT, typename T, int DKP, int W, int PT, int R> __device__ __forceinline__ void triangles(Chunk<T, DKP, W, PT, R>& c, int tid) {
  constexpr int TX = Terms<T>::X;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g4 = lane >> 4;
  if (wave < NB) tile<OUT>(c, wave, wave, lane);
  if (wave == W - 1) combine(c.s, lane);
  __syncthreads();
  if (wave > 0) {
    constexpr int EACH = (6 + W - 2) / (W - 1);
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int at = min(wave - 1 + (W - 1) * k, 5), I = at >= 3 ? 3 : at >= 1 ? 2 : 1;
      tile<OUT>(c, I, at - below(I, 0), lane);
    }
  } else {  // 16 lanes a block, a column each: substitution
    // (lane j of the 16 has column j of -L, and gives its elements to the others)
    float x[16], n[16];
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      const f32x4_t v = *reinterpret_cast<const f32x4_t*>(&c.n[g4][l16][4 * i4]);
#pragma unroll
      for (int r = 0; r < 4; ++r) n[4 * i4 + r] = v[r], x[4 * i4 + r] = 4 * i4 + r == l16 ? 1.f : 0.f;
    }
    substitute<0>(x, n);
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
      const Piece<TX> p = split<TX>(f32x4_t{x[4 * i4], x[4 * i4 + 1], x[4 * i4 + 2], x[4 * i4 + 3]});
#pragma unroll
      for (int e = 0; e < TX; ++e) {
        uint16_t* to = reinterpret_cast<uint16_t*>(c.d[g4][e] + spot(4 * i4, l16 >> 2)) + (l16 & 3);
        to[0] = (uint16_t)p.t[e].x;
        to[4] = (uint16_t)(p.t[e].x >> 16);
        to[8] = (uint16_t)p.t[e].y;
        to[12] = (uint16_t)(p.t[e].y >> 16);
      }
    }
  }
  __syncthreads();
}

// U's terms from R, block after block: (I + L) U = R; a block of U is taken from those
// below it as soon as it is there.  What U_I is made from stays in r, as terms.
template <typename Ch, int TX>
__device__ __forceinline__ void solve(const Ch& c, int lane, f32x4_t (&u)[NB], Piece<TX> (&r)[NB], Piece<TX> (&up)[NB]) {
#pragma unroll
  for (int I = 0; I < NB; ++I) {
    r[I] = split<TX>(u[I]);
    u[I] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    mma<TX, TX>(u[I], block_of(c.d[I], lane), r[I]);
    up[I] = split<TX>(u[I]);
#pragma unroll
    for (int J = I + 1; J < NB; ++J) mma<TX, TX>(u[J], block_of(c.l[below(J, I)], lane), up[I]);
  }
}

// A state's 16 columns of a wave: from memory [dk][dv] (null: zero), and to it ...
template <int DKP>
__device__ __forceinline__ void load_state(const float* m, const GatedDelta& a, int col, int lane, f32x4_t (&S)[DKP / 16]) {
#pragma unroll
  for (int t = 0; t < DKP / 16; ++t) S[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  if (!m) return;
#pragma unroll
  for (int t = 0; t < DKP / 16; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * t + 4 * (lane >> 4) + r;
      const float x = m[min(row, a.dk - 1) * a.dv + min(col, a.dv - 1)];
      S[t][r] = row < a.dk && col < a.dv ? x : 0.f;
    }
}
template <int DKP>
__device__ __forceinline__ void store_state(float* m, const GatedDelta& a, int col, int lane, const f32x4_t (&S)[DKP / 16]) {
  if (col >= a.dv) return;
#pragma unroll
  for (int t = 0; t < DKP / 16; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int row = 16 * t + 4 * (lane >> 4) + r;
      if (a.dk == DKP || row < a.dk) m[row * a.dv + col] = S[t][r];
    }
}
// ... and where the passes keep it, a padded column after another.
template <int DKP> __device__ __forceinline__ void load_kept(const float* m, int col, int lane, f32x4_t (&S)[DKP / 16]) {
#pragma unroll
  for (int t = 0; t < DKP / 16; ++t) S[t] = *reinterpret_cast<const f32x4_t*>(m + col * DKP + 16 * t + 4 * (lane >> 4));
}
template <int DKP> __device__ __forceinline__ void store_kept(float* m, int col, int lane, const f32x4_t (&S)[DKP / 16]) {
#pragma unroll
  for (int t = 0; t < DKP / 16; ++t) *reinterpret_cast<f32x4_t*>(m + col * DKP + 16 * t + 4 * (lane >> 4)) = S[t];
}
// Long sequences of few heads are cut in segments.  A chunk, and so a segment, acts on
// the state it starts from as S -> M S + N; N is what it makes of a zero state, and M
// what it makes of the identity without v.  Those are found for all segments at once,
// then put together in order (join), then each segment runs from its own state.  So
// does the gradient, backwards, with M^T.  Segment `seg` of a head keeps a padded state.
template <int DKP, int W> __device__ __forceinline__ float* segment(float* m, const GatedDelta& a, int seg, int64_t bh) {
  return m + ((int64_t)seg * a.B * a.H + bh) * (DKP * 16 * W);
}

// A segment's N and M on their way from memory: a wave's 16 columns of N; of M, whose
// rows are DKP apart, four elements of a row side by side.
template <int DKP> struct Segment {
  static constexpr int KT = DKP / 16;
  f32x4_t n[KT], m[KT][KT];
  __device__ __forceinline__ void from(const float* ends, const float* map, int col, int lane) {
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      n[t] = *reinterpret_cast<const f32x4_t*>(ends + col * DKP + 16 * t + 4 * (lane >> 4));
#pragma unroll
      for (int k = 0; k < KT; ++k) m[t][k] = *reinterpret_cast<const f32x4_t*>(map + (16 * t + (lane & 15)) * DKP + 16 * k + 4 * (lane >> 4));
    }
  }
  // N + M X
  __device__ __forceinline__ void apply(f32x4_t (&X)[KT]) const {
    Piece<3> x[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) x[t] = split<3>(X[t]), X[t] = n[t];
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int k = 0; k < KT; k += 2) mma<3, 3>(X[t], split<3>(m[t][k]), split<3>(m[t][k + 1]), x[k], x[k + 1]);
  }
};

// Where chunk n of a head keeps what: the state that it starts from (n >= 1) ...
template <int DKP, int W> __device__ __forceinline__ float* kept_before(const GatedDelta& a, int n, int64_t bh) {
  return a.saved + ((int64_t)(n - 1) * a.B * a.H + bh) * (DKP * 16 * W);
}
// ... the gradient of the one that it ends in, and columns of U and dR, 64 frames each.
template <int DKP, int W> __device__ __forceinline__ float* kept_after(const GatedDelta& a, int n, int64_t bh) {
  return a.dsaved + ((int64_t)n * a.B * a.H + bh) * (DKP * 16 * W);
}
template <int N, int W> __device__ __forceinline__ uint16_t* kept_columns(uint16_t* m, const GatedDelta& a, int n, int64_t bh) {
  return m + ((int64_t)n * a.B * a.H + bh) * (N * 16 * W * C);
}

}  // namespace gd
}  // namespace am
