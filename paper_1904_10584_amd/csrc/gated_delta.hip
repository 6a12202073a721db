// The gated delta rule's forward pass (its mathematics: gated_delta.h): chunks of 64
// frames one after another, a workgroup a head of a sequence; and one frame of many
// sequences, a pass over their states.
#include "gated_delta.h"

#include <algorithm>
#include <cmath>

namespace am {
namespace {

using namespace gd;

constexpr int THREADS = 256, WAVES = 4;  // of a frame's kernel

// What a workgroup makes: the outputs, or of a segment what it makes of a zero state
// (ENDS), or of the identity without v (MAPS).
enum Pass { OUTPUTS, ENDS, MAPS };

// All columns of a head are one workgroup's: with 128 of them on two of 64, which share
// nothing but repeat the triangles, 64 utterances of 200 to 1500 frames and 6 heads of
// 128 x 128 took 357 us and not 335.  The next chunk's rows arrive in registers while one
// is in hand.  256 x 64 frames, 12 heads of 64 x 64: 92 us (202 MB with both states, 2.2
// TB/s); 40001 frames of 12 heads in segments 384 us, 4.4 ms without.
template <typename T, int DKP, int W, Pass PASS> __device__ __forceinline__ void forward_pass(const GatedDelta& a, uint8_t* lds) {
  constexpr int TI = Terms<T>::IN, TX = Terms<T>::X, TO = Terms<T>::OUT, KT = DKP / 16;
  constexpr bool OUT = PASS == OUTPUTS;
  Chunk<T, DKP, W, TO, 1>& c = *reinterpret_cast<Chunk<T, DKP, W, TO, 1>*>(lds);
  Gates& s = c.s;
  const Head hd(a, blockIdx.x);
  const int seg = blockIdx.y, begin = seg * a.per * C, end = min(hd.len, begin + a.per * C);
  if (seg > 0 && begin >= hd.len) return;
  const float rate = rate_of(a, hd.h);
  const int64_t mine = (int64_t)blockIdx.x * a.dk * a.dv;
  const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
  f32x4_t S[KT];
  {
    const int lane = threadIdx.x & 63, col = column_of(threadIdx.x);
    if (PASS == MAPS) {
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[t][r] = 16 * t + 4 * (lane >> 4) + r == col ? 1.f : 0.f;
    } else if (OUT && a.segs > 1) {  // (s0 itself may be sT, which the last segment writes)
      load_kept<DKP>(segment<DKP, W>(a.seg_n, a, seg > 0 ? seg - 1 : a.segs - 1, blockIdx.x), col, lane, S);
    } else {
      load_state<DKP>(OUT && a.s0 ? a.s0 + mine : nullptr, a, col, lane, S);
    }
  }
  Rows<T, DKP, W> fk, fq;
  Values<T, W> fv;
  GateRows<T, W> fg;
  auto fetch = [&](const int32_t (&rows)[C], int next0, int tid) {
    fk.from(a.k, a.ldk, hd.kh, a.dk, rows, tid);
    if constexpr (OUT) fq.from(a.q, a.ldq, hd.kh, a.dk, rows, tid);
    if constexpr (PASS != MAPS) fv.from(a.v, a.ldv, hd, a.dv, rows, tid);
    fg.from(a, hd, rows, next0, tid);
  };
  if (begin < end) {
    if (threadIdx.x < C) s.row[0][threadIdx.x] = hd.row(a, begin + threadIdx.x);
    __syncthreads();
    fetch(s.row[0], begin + C, threadIdx.x);
  }
  int turn = 0;
  for (int t0 = begin; t0 < end; t0 += C, turn ^= 1) {
    const int left = hd.len - t0, tid = this_thread(), lane = tid & 63, l16 = lane & 15, g4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = 16 * wave + l16;
    if (OUT && a.train && t0 > 0) store_kept<DKP>(kept_before<DKP, W>(a, t0 / C, blockIdx.x), col, lane, S);
    fk.lengths(s.rk, a.eps, left, tid);
    fk.store(c.k, tid);
    if constexpr (OUT) {
      fq.lengths(s.rq, a.eps, left, tid);
      fq.store(c.q, tid);
    }
    if constexpr (PASS != MAPS) fv.store(&c.v[0], s.row[turn], tid);
    fg.store(s, rate, left, turn, tid);
    __syncthreads();
    f32x4_t v[NB];
#pragma unroll
    for (int I = 0; I < NB; ++I) {
      if constexpr (PASS != MAPS) v[I] = fv.column_values(wave, I, lane);
      else v[I] = zero;
    }
    if (t0 + C < end) fetch(s.row[turn ^ 1], t0 + 2 * C, tid);  // the next chunk's, which arrive during this one
    triangles<OUT>(c, tid);

    f32x4_t u[NB], o[NB];
#pragma unroll
    for (int I = 0; I < NB; ++I) u[I] = o[I] = zero;
#pragma unroll
    for (int t = 0; t < DKP / 32; ++t) {
      const Piece<TX> s0 = split<TX>(S[2 * t]), s1 = split<TX>(S[2 * t + 1]);
#pragma unroll
      for (int I = 0; I < NB; ++I) {
        Piece<TI> a0, a1;
        rows_of(c.k, I, t, lane, a0, a1);
        mma<TI, TX>(u[I], a0, a1, s0, s1);
        if constexpr (OUT) {
          rows_of(c.q, I, t, lane, a0, a1);
          mma<TO, TI>(o[I], first<TO>(s0), first<TO>(s1), a0, a1);
        }
      }
    }
#pragma unroll
    for (int I = 0; I < NB; ++I) {
      u[I] = v[I] * rows4(s.beta, I, lane) - u[I] * rows4(s.bgk, I, lane);
      if constexpr (OUT) o[I] *= s.gq[16 * I + l16];
    }
    Piece<TX> r[NB], up[NB];
    solve(c, lane, u, r, up);
    if constexpr (OUT) {
#pragma unroll
      for (int I = 0; I < NB; ++I) {
#pragma unroll
        for (int J = 0; J + 1 <= I; J += 2)
          mma<TO, TO>(o[I], first<TO>(up[J]), first<TO>(up[J + 1]), block_of(c.p[lower(I, J)], lane), block_of(c.p[lower(I, J + 1)], lane));
        if (I % 2 == 0) mma<TO, TO>(o[I], first<TO>(up[I]), block_of(c.p[lower(I, I)], lane));
      }
#pragma unroll
      for (int I = 0; I < NB; ++I)
        if (16 * I + l16 < left)
          put4(static_cast<T*>(a.o) + s.row[turn][16 * I + l16] * a.ldo + (int64_t)hd.h * a.dv + 16 * wave + 4 * g4,
               a.dv - 16 * wave - 4 * g4, o[I]);
    }
#pragma unroll
    for (int I = 0; I < NB; ++I) up[I] = split<TX>(u[I] * rows4(s.gk, I, lane));
    const float g_end = s.g[C - 1];
#pragma unroll
    for (int t = 0; t < KT; ++t) {
      S[t] *= g_end;
#pragma unroll
      for (int I = 0; I < NB; I += 2) mma<TI, TX>(S[t], columns_of(c.k, t, I, lane), columns_of(c.k, t, I + 1, lane), up[I], up[I + 1]);
    }
    __syncthreads();
  }
  const int lane = threadIdx.x & 63, col = column_of(threadIdx.x);
  if (PASS == ENDS) {
    store_kept<DKP>(segment<DKP, W>(a.seg_n, a, seg, blockIdx.x), col, lane, S);
  } else if (PASS == MAPS) {  // by columns, for the backward pass, and by rows
    store_kept<DKP>(segment<DKP, W>(a.seg_mt, a, seg, blockIdx.x), col, lane, S);
    float* const m = segment<DKP, W>(a.seg_m, a, seg, blockIdx.x);
#pragma unroll
    for (int t = 0; t < KT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) m[(16 * t + 4 * (lane >> 4) + r) * DKP + col] = S[t][r];
  } else if (a.sT && hd.len <= begin + a.per * C) {
    store_state<DKP>(a.sT + mine, a, col, lane, S);
  }
}

template <typename T, int DKP, int W>
__global__ __launch_bounds__(threads_of<W>, sizeof(T) == 2 && DKP == 64 ? 3 : 2) void gd_forward_kernel(GatedDelta a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  forward_pass<T, DKP, W, OUTPUTS>(a, lds);
}

// Both parts of what segments do to a state, in one launch: neither fills the chip.
// (2000 frames of 12 heads, forward, 70 us and not 79; 8 such of 16 heads 165, 203.)  A
// training pass needs the last segments' maps too, for the gradient.  (The waves that a
// part has no columns for end; barriers are the others'.)
template <int DKP, int W> constexpr int segment_threads = threads_of<(W > DKP / 16 ? W : DKP / 16)>;
template <typename T, int DKP, int W>
__global__ __launch_bounds__((segment_threads<DKP, W>), sizeof(T) == 2 && DKP == 64 ? 3 : 2) void gd_segments_kernel(GatedDelta a) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  const bool last = (int)blockIdx.y == a.segs - 1;
  if (blockIdx.z == 0) {
    if (threadIdx.x < threads_of<DKP / 16> && (!last || a.train)) forward_pass<T, DKP, DKP / 16, MAPS>(a, lds);
  } else {
    if (threadIdx.x < threads_of<W> && !last) forward_pass<T, DKP, W, ENDS>(a, lds);
  }
}

// The states that segments start from, one after another: the products of a head's
// columns wait for the ones before them, so nothing else may (the next segment's maps
// arrive meanwhile).  The first one's is kept in the last one's place.
template <int DKP, int W> __global__ __launch_bounds__(64) void gd_join_kernel(GatedDelta a) {
  const int lane = threadIdx.x, col = 16 * blockIdx.y + (lane & 15), len = a.lens ? a.lens[blockIdx.x / a.H] : a.T;
  f32x4_t S[DKP / 16];
  load_state<DKP>(a.s0 ? a.s0 + (int64_t)blockIdx.x * a.dk * a.dv : nullptr, a, col, lane, S);
  auto go = [&](int seg) { return seg + 1 < a.segs && (seg + 1) * a.per * C < len; };
  auto ends = [&](int seg) { return segment<DKP, W>(a.seg_n, a, seg, blockIdx.x); };
  auto map = [&](int seg) { return segment<DKP, DKP / 16>(a.seg_m, a, seg, blockIdx.x); };
  store_kept<DKP>(ends(a.segs - 1), col, lane, S);
  Segment<DKP> now, next;
  constexpr bool AHEAD = DKP == 64;  // (of 128 x 128, one map fills the registers)
  if (AHEAD && go(0)) now.from(ends(0), map(0), col, lane);
  for (int seg = 0; go(seg); ++seg) {
    if (!AHEAD) now.from(ends(seg), map(seg), col, lane);
    else if (go(seg + 1)) next.from(ends(seg + 1), map(seg + 1), col, lane);
    now.apply(S);
    store_kept<DKP>(ends(seg), col, lane, S);
    if (AHEAD) now = next;
  }
}

// One frame of each sequence: a state is read once, kept in registers, and written
// once, in fp32 throughout, with no matrix instruction: 8 operations for 8 bytes.  A
// thread has four columns (CG threads a row) of every RG-th row.  64 sequences, 12 heads
// of 64 x 64: 6.8 us for 25.6 MB (3.8 TB/s, with the launch); as a chunk of one frame 19.
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
  const int64_t row0 = hd.row(a, 0);
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
  const float decay = expf(-rate_of(a, hd.h) * sigm(to_f32(static_cast<const T*>(a.r)[row0 * a.ldr + hd.h])));
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

template <typename T, int DKP, int W> hipError_t chunks(const GatedDelta& a, hipStream_t s) {
  constexpr int LDS = sizeof(Chunk<T, DKP, W, Terms<T>::OUT, 1>), MAPS_LDS = sizeof(Chunk<T, DKP, DKP / 16, Terms<T>::OUT, 1>);
  constexpr int BOTH = LDS > MAPS_LDS ? LDS : MAPS_LDS;
  static_assert(BOTH <= 160 * 1024, "a workgroup's LDS");
  static PerDevice ready, segments_ready;
  hipError_t e = allow_lds<LDS>(reinterpret_cast<const void*>(&gd_forward_kernel<T, DKP, W>), ready);
  if (e == hipSuccess && a.segs > 1)
    e = allow_lds<BOTH>(reinterpret_cast<const void*>(&gd_segments_kernel<T, DKP, W>), segments_ready);
  if (e != hipSuccess) return e;
  const unsigned heads = (unsigned)(a.B * a.H);
  if (a.segs > 1) {
    hipLaunchKernelGGL((gd_segments_kernel<T, DKP, W>), dim3(heads, a.segs, 2), dim3(segment_threads<DKP, W>), BOTH, s, a);
    hipLaunchKernelGGL((gd_join_kernel<DKP, W>), dim3(heads, W), dim3(64), 0, s, a);
  }
  hipLaunchKernelGGL((gd_forward_kernel<T, DKP, W>), dim3(heads, a.segs), dim3(threads_of<W>), LDS, s, a);
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
  if (a.dk <= 64) return a.dv <= 64 ? chunks<T, 64, 4>(a, s) : chunks<T, 64, 8>(a, s);
  return a.dv <= 64 ? chunks<T, 128, 4>(a, s) : chunks<T, 128, 8>(a, s);
}

}  // namespace

// A forward pass goes through its chunks three times where it is cut (MAPS and ENDS at
// once, then OUTPUTS, over all segments at once), a backward pass twice, and the joins
// take the segments one after another: about 2 us each, a third of a chunk.  n chunks of few
// heads are so best in segments of about sqrt(n / 8), and heads that fill the chip
// between them are not cut: two workgroups of 64 columns a CU, one of 128.  Measured, us:
//   short segments or longer ones (12 heads of 64 x 64, a training pass): 500 frames in
//   segments of 1, 2 and 8 chunks (uncut) 108, 119 and 178; 2000 frames of 1, 2, 3, 4 and
//   8 212, 181, 187, 205 and 302, uncut 622; 8000 of 3, 4 and 6 388, 371 and 377;
//   workgroups of all segments: 40001 frames of 12 heads, forward, 276, 384, 504, 756 and
//   948 491, 381, 380, 376 and 425; 1500 frames of 24 heads of 128 x 128 96, 144, 192 and
//   288 443, 443, 399 and 504 in training (forward 134 and 121 with 96 and 144, 142 with
//   192, which the rule takes);
//   least segments: three in training (2000 frames of 160 heads 761, uncut 845; 190 of
//   12 86, uncut 93), four in a forward pass alone (2000 of 128 161, uncut 221; in three,
//   190 of 12 30 and 28, 1500 of 84 of 128 x 128 231 and 219, but 2000 of 160 199 and 224).
DeltaSegments delta_segments(int64_t T, int64_t heads, int dv, bool train) {
  const int64_t chunks = (T + GD_CHUNK - 1) / GD_CHUNK, room = (dv <= 64 ? 512 : 256) / heads, least = train ? 3 : 4;
  if (room < least) return {1, (int)chunks};
  const int64_t per = std::max({(chunks + room - 1) / room, (int64_t)std::sqrt(chunks / 8.0), (int64_t)1});
  const int64_t segs = (chunks + per - 1) / per;
  if (segs < least) return {1, (int)chunks};
  return {(int)segs, (int)per};
}

hipError_t gated_delta_forward(GatedDelta a, bool bf16, hipStream_t s) {
  return bf16 ? forward<bf16_t>(a, s) : forward<float>(a, s);
}

}  // namespace am
