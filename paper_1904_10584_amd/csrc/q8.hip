// Matrices as 8-bit floats and their products.
//
// A matrix is held as codes (4 bits of exponent of bias 7, 3 of fraction) with a
// power of two for each 128 elements of a row, or for each tile of 128 x 128, that
// puts the largest of them into [128, 256).  Powers of two make the scaling exact,
// and the matrix cores apply them inside the product: an instruction of 128 elements
// of the sum takes one exponent byte for each row of either operand.
#include "am_device.h"
#include "am_internal.h"
#include "per_device.h"

namespace am {
namespace {

// ------------------------------------------------------------- quantising --
//
// One workgroup takes a tile of 128 x 128: a thread has 8 x 8 elements of it, so its
// rows leave as words and its columns, through LDS, as 16-byte pieces.  The matrix is
// read once for both layouts: 16384 x 2304 in bf16, both layouts, takes 38 us for 151 MB
// (4.0 TB/s; a copy of its size reaches 5.1 to 7).  Nothing is busy throughout: the vector
// units for 19 us of it, LDS for 9 (8 of them conflicts of the transposed tile's rows),
// HBM for 21 to 29; a workgroup loads, computes and stores one after another, three of
// them a CU.  Loads and stores without branches, so that all are in flight, brought it
// there from 57.

constexpr int QT = 128;           // rows and columns of a tile, elements of a scale
constexpr int QPITCH = QT + 16;   // bytes between the transposed tile's rows in LDS

// The bits of |v|, or 0 where v is not finite: what is not a number sets no scale.
__device__ __forceinline__ uint32_t magnitude(float v) {
  const uint32_t u = __float_as_uint(v) & 0x7fffffffu;
  return u < 0x7f800000u ? u : 0u;
}
__device__ __forceinline__ uint32_t umax32(uint32_t a, uint32_t b) { return a > b ? a : b; }

// Eight elements of a row as they lie in memory: the first `left` of those at p, which
// may be none, then zeros.  Lanes that have fewer read what lies before the row's end in
// their place, and need no branch.
template <typename T> struct Eight;
template <> struct Eight<bf16_t> {
  typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
  u32x4_t w;
  __device__ __forceinline__ float at(int k) const { return __uint_as_float(k & 1 ? w[k >> 1] & 0xffff0000u : w[k >> 1] << 16); }
  __device__ __forceinline__ void load(const bf16_t* p, int left, bool wide) {
    if (wide) {  // (uniform: whole pieces on 16 bytes)
      w = *reinterpret_cast<const u32x4_t*>(p + min(left - 8, 0));
      w = left > 0 ? w : u32x4_t{0, 0, 0, 0};
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t lo = p[min(2 * k, left - 1)], hi = p[min(2 * k + 1, left - 1)];
        w[k] = (2 * k < left ? lo : 0u) | (2 * k + 1 < left ? hi << 16 : 0u);
      }
    }
  }
};
template <> struct Eight<float> {
  f32x4_t w[2];
  __device__ __forceinline__ float at(int k) const { return w[k >> 2][k & 3]; }
  __device__ __forceinline__ void load(const float* p, int left, bool wide) {
    if (wide) {
      p += min(left - 8, 0);
      w[0] = *reinterpret_cast<const f32x4_t*>(p);
      w[1] = *reinterpret_cast<const f32x4_t*>(p + 4);
      if (left <= 0) w[0] = w[1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float x = p[min(k, left - 1)];
        w[k >> 2][k & 3] = k < left ? x : 0.f;
      }
    }
  }
};

template <typename T>
__global__ __launch_bounds__(256, 3) void q8_quantise_kernel(Q8Quantise a) {
  __shared__ __attribute__((aligned(16))) uint8_t turned[QT * QPITCH];
  __shared__ uint32_t tops[16][QT + 4];
  const int t = threadIdx.x, cx = t & 15, ry = t >> 4;
  const uint32_t tile = a.first + blockIdx.x;
  const int64_t ty = tile / a.across, tx = tile % a.across, r0 = ty * QT, c0 = tx * QT;
  const int64_t rows = a.rows, cols = a.cols, c = c0 + 8 * cx;
  Eight<T> v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {  // (of a row past the last nothing is kept: it is the last one again, without elements)
    const int64_t r = r0 + 8 * ry + i;
    v[i].load(static_cast<const T*>(a.x) + min(r, rows - 1) * a.ld + c, (int)(cols - c), a.wide);
  }
  const int here = (int)min((int64_t)8, rows - r0 - 8 * ry);  // of this thread's rows
  uint32_t row_top[8], col_top[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) row_top[i] = col_top[i] = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t m = i < here ? magnitude(v[i].at(k)) : 0u;
      row_top[i] = umax32(row_top[i], m);
      col_top[k] = umax32(col_top[k], m);
    }
  // along a row: the 16 threads of it are 16 lanes
#pragma unroll
  for (int i = 0; i < 8; ++i) row_top[i] = lanes16_max(row_top[i]);
  if (a.tiles) {
    uint32_t top = row_top[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = umax32(top, row_top[i]);
    if (cx == 0) tops[ry][0] = top;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k) top = umax32(top, tops[k][0]);
#pragma unroll
    for (int i = 0; i < 8; ++i) row_top[i] = col_top[i] = top;
  } else if (a.codes_t) {
#pragma unroll
    for (int k = 0; k < 8; ++k) tops[ry][8 * cx + k] = col_top[k];
    __syncthreads();
    if (t < QT) {  // a column a thread
      uint32_t top = tops[0][t];
#pragma unroll
      for (int q = 1; q < 16; ++q) top = umax32(top, tops[q][t]);
      tops[0][t] = top;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 8; ++k) col_top[k] = tops[0][8 * cx + k];
  }
  if (a.codes) {
    const int64_t pad = (cols + 15) & ~(int64_t)15;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t r = r0 + 8 * ry + i;
      const uint32_t e = q8_exponent(row_top[i]);
      const float inv = q8_inverse(e);
      if (r < rows) {
        if (c < pad)
          *reinterpret_cast<uint2*>(a.codes + r * a.ldc + c) =
              make_uint2(q8_codes4(v[i].at(0), v[i].at(1), v[i].at(2), v[i].at(3), inv),
                         q8_codes4(v[i].at(4), v[i].at(5), v[i].at(6), v[i].at(7), inv));
        if (!a.tiles && cx == 0) a.scales[r * a.lds + tx] = (uint8_t)e;
      }
    }
    if (a.tiles && t == 0) a.scales[ty * a.lds + tx] = (uint8_t)q8_exponent(row_top[0]);
  }
  if (!a.codes_t) return;
  const uint32_t k_lo = here >= 4 ? ~0u : here > 0 ? (1u << 8 * here) - 1 : 0u;
  const uint32_t k_hi = here >= 8 ? ~0u : here > 4 ? (1u << 8 * (here - 4)) - 1 : 0u;
  const uint64_t keep = (uint64_t)k_hi << 32 | k_lo;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const uint32_t e = q8_exponent(col_top[k]);
    const float inv = q8_inverse(e);
    // (rows past the last have zeros: the codes of as many as there are are kept)
    const uint64_t w = (uint64_t)q8_codes4(v[4].at(k), v[5].at(k), v[6].at(k), v[7].at(k), inv) << 32 |
                       q8_codes4(v[0].at(k), v[1].at(k), v[2].at(k), v[3].at(k), inv);
    *reinterpret_cast<uint64_t*>(turned + (8 * cx + k) * QPITCH + 8 * ry) = w & keep;
    if (!a.tiles && ry == 0 && c + k < cols) a.scales_t[(c + k) * a.ldst + ty] = (uint8_t)e;
  }
  if (a.tiles && t == 0) a.scales_t[tx * a.ldst + ty] = (uint8_t)q8_exponent(col_top[0]);
  __syncthreads();
  const int64_t pad = (rows + 15) & ~(int64_t)15;
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const int col = p * 32 + (t >> 3), piece = 16 * (t & 7);
    if (c0 + col < cols && r0 + piece < pad)
      *reinterpret_cast<uint4*>(a.codes_t + (c0 + col) * a.ldct + r0 + piece) =
          *reinterpret_cast<const uint4*>(turned + col * QPITCH + piece);
  }
}

// --------------------------------------------------------------- products --
//
// out = a b^T over k.  The matrix instruction forms 16 columns of out (rows of b) by
// 16 rows (of a): a lane then has columns of one row, and with the rows of b dealt to
// the instructions in fours it has 4 FN of them side by side, which leave as 16-byte
// stores.  Operand tiles of 128 elements of the sum go from global memory straight to
// LDS, NS stages deep, with their scales: a word of a row's scales serves four of
// them, and an instruction picks its byte.
//
// Sums of 128 products are the matrix cores': of products of like size they leave the
// rounding to bf16 as it is (1.66e-3 of the outputs' size in the root mean square), of
// products over the codes' whole range they were off by 2^-12.6 of the sum of magnitudes
// at most.  So out is bf16, and no fp32 output is offered.
//
// 32768 x 4608 x 1536 in Large tiles: 254 us, 1.82 PFLOP/s; a library's product of the
// same codes with one scale a matrix takes 234.  Each 128 more of K take 11.8 us (2.45
// PFLOP/s); about 70 us are the output's way to memory (302 MB), beside which no tile of
// the same CU runs.  Slower there: two waves that take turns at a SIMD 334, stages of 64
// 310; 128 x 256 and 256 x 128 tiles 373, four by four waves 477 (of 315 then); runs of
// 8 columns of tiles for ACROSS 308 (4: 305; whole rows of tiles 315).

__device__ uint4 g_none[1];  // zeros: what lies outside an operand

constexpr int BK = 128;     // elements of the sum a stage
constexpr int XCDS = 8;
constexpr int ACROSS = 4;  // tiles side by side that a run goes through together

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));

// Four bytes a lane from global memory to LDS at lds_base + 4 * lane; and 16 from a
// base that is the wave's, and an offset below 4 GiB that is the lane's.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void dma16_at(const void* base, uint32_t offset, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               ::"v"(offset), "s"(base), "s"(lds_base) : "memory", "m0");
}
__device__ __forceinline__ void dma4(const void* src, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(src), "s"(lds_base) : "memory", "m0");
}
#pragma clang diagnostic pop

template <int OP>
__device__ __forceinline__ void mma8(f32x4_t& acc, const i32x8_t& a, const i32x8_t& b, int sa, int sb) {
  acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 0, 0, OP, sa, OP, sb);
}

template <int BM_, int BN_, int WM_, int WN_, int NS_> struct Shape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, NS = NS_;
  static constexpr int WAVES = WM * WN, THREADS = 64 * WAVES;
  static constexpr int TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16;
  static constexpr int A_BYTES = BM * BK, B_BYTES = BN * BK, STAGE = A_BYTES + B_BYTES;
  static constexpr int LOADS = (BM + BN) / 8 / WAVES;             // 16-byte loads a stage of each wave
  static constexpr int SCALE_ROWS = BM + BN, SCALE_WAVES = SCALE_ROWS / 64;
  static constexpr bool SPLIT = BM < 256;                         // (the largest tiles come by the hundred)
  static constexpr int SETS = (NS + 6) / 4;                       // sets of scales alive at once
  static constexpr int LDS = NS * STAGE + SETS * SCALE_ROWS * 4;
  static_assert(BM % 64 == 0 && BN % 64 == 0 && (BM + BN) % (8 * WAVES) == 0, "whole loads");
  static_assert(SCALE_WAVES <= WAVES, "one load of scales a wave");
  static_assert(4 % NS == 0, "a stage's place is known where it is used");
  static_assert(FN == 2 || FN == 4, "columns of a lane in 16-byte pieces");
};

// Which 16-byte piece of a row of 128 bytes lies in which slot: lanes that are served
// together read rows whose keys differ.
__device__ __forceinline__ int key_a(int row) { return row & 7; }
template <int FN> __device__ __forceinline__ int key_b(int row) { return (row & 3) | ((row / (4 * FN)) & 1) << 2; }

// The bias of a lane's 4 FN columns.
template <int FN> __device__ __forceinline__ void bias_of(const Q8Matmul& a, int64_t col, f32x4_t (&v)[FN]) {
#pragma unroll
  for (int j = 0; j < FN; ++j) v[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  if (a.bias)
#pragma unroll
    for (int j = 0; j < 4 * FN; ++j) v[j / 4][j % 4] = a.bias[min(col + j, a.N - 1)];
}
// One row's columns: + bias, + what out holds, rounded once.
template <int FN>
__device__ __forceinline__ void q8_store(const Q8Matmul& a, int64_t row, int64_t col, const f32x4_t (&bias)[FN],
                                         const f32x4_t (&v)[FN]) {
  typedef __bf16 b8 __attribute__((ext_vector_type(8)));
  typedef float f8 __attribute__((ext_vector_type(8)));
  if (row >= a.M || col >= a.N) return;
  bf16_t* p = a.out + row * a.ldo + col;
#pragma unroll
  for (int h = 0; h < FN / 2; ++h) {
    f8 w = __builtin_shufflevector(v[2 * h] + bias[2 * h], v[2 * h + 1] + bias[2 * h + 1], 0, 1, 2, 3, 4, 5, 6, 7);
    if (a.wide && col + 8 * h + 8 <= a.N) {
      if (a.accumulate) w += __builtin_convertvector(reinterpret_cast<const b8*>(p)[h], f8);
      reinterpret_cast<b8*>(p)[h] = __builtin_convertvector(w, b8);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (col + 8 * h + j < a.N) p[8 * h + j] = f32_to_bf16(a.accumulate ? w[j] + bf16_to_f32(p[8 * h + j]) : w[j]);
    }
  }
}

// The tile that a workgroup of a launch takes: each XCD has a run of them, so that
// tiles with the same rows of a share its L2.
struct Tile { int m, n; };
__device__ __forceinline__ Tile tile_at(int T, int tiles_m, int tiles_n) {
  const int whole = ACROSS * tiles_m, group = T / whole, in = T - group * whole;
  const int wide = min(ACROSS, tiles_n - group * ACROSS);
  return {in / wide, group * ACROSS + in % wide};
}
__device__ __forceinline__ int tile_of(int b, int tiles) {
  const int x = b % XCDS, q = tiles / XCDS, rem = tiles % XCDS;
  return x * q + min(x, rem) + b / XCDS;
}

template <typename S>
__global__ __launch_bounds__(S::THREADS) void q8_matmul_kernel(Q8Matmul a) {
  extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
  constexpr int FM = S::FM, FN = S::FN;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tile = tile_of(blockIdx.x, a.tiles_m * a.tiles_n);
  const Tile place = tile_at(tile, a.tiles_m, a.tiles_n);
  const int64_t m0 = (int64_t)place.m * S::BM, n0 = (int64_t)place.n * S::BN;
  const int split = blockIdx.y, k0 = split * a.steps, nk = min(a.blocks - k0, a.steps);  // (blocks of BK)
  const uint32_t base = lds_address(lds), scales = base + S::NS * S::STAGE;
  const uint8_t* scale_lds = lds + S::NS * S::STAGE;

  // where this lane's loads come from: offsets from the tile's first rows.  (Rows past an
  // operand's last are that one again: nothing that they make is stored.)
  const uint8_t* const base_a = a.a + m0 * a.lda;
  const uint8_t* const base_b = a.b + n0 * a.ldb;
  uint32_t offset[S::LOADS];
#pragma unroll
  for (int i = 0; i < S::LOADS; ++i) {
    const int row = (wave * S::LOADS + i) * 8 + (lane >> 3);  // of both operands' tiles
    const bool is_a = (wave * S::LOADS + i) * 8 < S::BM;
    const int r = is_a ? row : row - S::BM;
    const int64_t last = (is_a ? a.M - m0 : a.N - n0) - 1;
    offset[i] = (uint32_t)min((int64_t)r, last) * (uint32_t)(is_a ? a.lda : a.ldb) +
                16 * ((lane & 7) ^ (is_a ? key_a(r) : key_b<FN>(r)));
  }
  // and one row's scales
  const uint8_t* scale_src = nullptr;
  if (wave < S::SCALE_WAVES) {
    const int row = wave * 64 + lane;
    if (row < S::BM) {
      scale_src = a.a_scale + min(m0 + row, a.M - 1) * a.ldas;
    } else {
      const int64_t g = min(n0 + row - S::BM, a.N - 1);
      scale_src = a.b_scale + (a.b_tiles ? g / QT : g) * a.ldbs;
    }
  }
  auto load = [&](int t, int slot) {  // stage t of this workgroup's, t % NS = slot
    const int64_t at = (int64_t)(k0 + t) * BK;
    const uint32_t to = base + slot * S::STAGE + wave * S::LOADS * 1024;
    if (t % 4 == 0 && wave < S::SCALE_WAVES)
      dma4(scale_src + at / BK, scales + (t / 4 % S::SETS) * S::SCALE_ROWS * 4 + wave * 256);
    if (at + BK <= a.K) {
#pragma unroll
      for (int i = 0; i < S::LOADS; ++i)
        dma16_at(((wave * S::LOADS + i) * 8 < S::BM ? base_a : base_b) + at, offset[i], to + i * 1024);
    } else {  // pieces past the rows' ends come from zeros
      const int ln = this_thread() & 63;
#pragma unroll
      for (int i = 0; i < S::LOADS; ++i) {
        const bool is_a = (wave * S::LOADS + i) * 8 < S::BM;
        const int row = (wave * S::LOADS + i) * 8 - (is_a ? 0 : S::BM) + (ln >> 3);
        const int piece = 16 * ((ln & 7) ^ (is_a ? key_a(row) : key_b<FN>(row)));
        dma16(at + piece < a.K ? (const void*)((is_a ? base_a : base_b) + at + offset[i]) : (const void*)g_none, to + i * 1024);
      }
    }
  };
#pragma unroll
  for (int t = 0; t < S::NS - 1; ++t)
    if (t < nk) load(t, t);

  const int wm = wave / S::WN, wn = wave % S::WN;
  f32x4_t acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  int sa[FM], sb[FN];

  auto step = [&](int t, auto op) {
    constexpr int OP = decltype(op)::value;
    // stage t is here once at most the later stages' loads are in flight
    const int later = min(nk - 1 - t, S::NS - 2);
    wait_vm_n<S::LOADS * (S::NS - 2)>(later * S::LOADS);
    lds_barrier();
    if (t + S::NS - 1 < nk) load(t + S::NS - 1, (OP + S::NS - 1) % S::NS);  // (into the stage read before the barrier)
    const uint8_t* st = lds + OP % S::NS * S::STAGE;
    const int ln = this_thread() & 63, i16 = ln & 15, g4 = ln >> 4;
    if constexpr (OP == 0) {
      const uint8_t* sc = scale_lds + (t / 4 % S::SETS) * S::SCALE_ROWS * 4;
#pragma unroll
      for (int i = 0; i < FM; ++i) sa[i] = *reinterpret_cast<const int*>(sc + 4 * (wm * S::TM + 16 * i + i16));
#pragma unroll
      for (int j = 0; j < FN; ++j)
        sb[j] = *reinterpret_cast<const int*>(sc + 4 * (S::BM + wn * S::TN + (i16 >> 2) * 4 * FN + 4 * j + (i16 & 3)));
    }
    auto fragment = [&](const uint8_t* row, int key) {
      return (i32x8_t)__builtin_shufflevector(*reinterpret_cast<const i32x4_t*>(row + 16 * ((2 * g4) ^ key)),
                                              *reinterpret_cast<const i32x4_t*>(row + 16 * ((2 * g4 + 1) ^ key)), 0, 1,
                                              2, 3, 4, 5, 6, 7);
    };
    i32x8_t fb[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int r = wn * S::TN + (i16 >> 2) * 4 * FN + 4 * j + (i16 & 3);
      fb[j] = fragment(st + S::A_BYTES + r * BK, key_b<FN>(r));
    }
    const uint8_t* const rows = st + (wm * S::TM + i16) * BK;
    i32x8_t fa[2];
    fa[0] = fragment(rows, key_a(i16));
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      if (i + 1 < FM) fa[(i + 1) & 1] = fragment(rows + 16 * (i + 1) * BK, key_a(i16));
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int j = 0; j < FN; ++j) mma8<OP>(acc[i][j], fb[j], fa[i & 1], sb[j], sa[i]);
      __builtin_amdgcn_s_setprio(0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  for (int t = 0; t < nk; t += 4) {
    step(t, std::integral_constant<int, 0>());
    if (t + 1 < nk) step(t + 1, std::integral_constant<int, 1>());
    if (t + 2 < nk) step(t + 2, std::integral_constant<int, 2>());
    if (t + 3 < nk) step(t + 3, std::integral_constant<int, 3>());
  }

  if (S::SPLIT && a.parts) {  // one of several sums: in the order of the registers
    float4* p = reinterpret_cast<float4*>(a.parts) +
                (((int64_t)split * a.tiles_m * a.tiles_n + tile) * FM * FN) * S::THREADS + threadIdx.x;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
        p[(int64_t)(i * FN + j) * S::THREADS] = make_float4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]);
    return;
  }
  const int i16 = lane & 15, g4 = lane >> 4;
  f32x4_t bias[FN];
  bias_of<FN>(a, n0 + wn * S::TN + g4 * 4 * FN, bias);
#pragma unroll
  for (int i = 0; i < FM; ++i)
    q8_store<FN>(a, m0 + wm * S::TM + 16 * i + i16, n0 + wn * S::TN + g4 * 4 * FN, bias, acc[i]);
}

// The sums of a split product, added in the order of the splits.
template <typename S>
__global__ __launch_bounds__(S::THREADS) void q8_join_kernel(Q8Matmul a) {
  constexpr int FM = S::FM, FN = S::FN;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int tile = blockIdx.x / FM, i = blockIdx.x % FM;
  const int64_t tiles = (int64_t)a.tiles_m * a.tiles_n;
  const float4* p = reinterpret_cast<const float4*>(a.parts) + ((int64_t)tile * FM + i) * FN * S::THREADS + threadIdx.x;
  f32x4_t v[FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) v[j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < a.splits; ++s, p += tiles * FM * FN * S::THREADS)
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const float4 u = p[j * S::THREADS];
      v[j] += f32x4_t{u.x, u.y, u.z, u.w};
    }
  const Tile place = tile_at(tile, a.tiles_m, a.tiles_n);
  const int64_t m0 = (int64_t)place.m * S::BM, n0 = (int64_t)place.n * S::BN;
  const int64_t col = n0 + wave % S::WN * S::TN + (lane >> 4) * 4 * FN;
  f32x4_t bias[FN];
  bias_of<FN>(a, col, bias);
  q8_store<FN>(a, m0 + wave / S::WN * S::TM + 16 * i + (lane & 15), col, bias, v);
}

typedef Shape<256, 256, 2, 4, 2> Large;
typedef Shape<128, 128, 2, 2, 2> Medium;
typedef Shape<64, 64, 2, 2, 4> Small;

template <typename S> void plan_of(Q8Plan& p, int64_t M, int64_t N, int64_t K) {
  const int64_t tiles = ((M + S::BM - 1) / S::BM) * ((N + S::BN - 1) / S::BN), blocks = (K + BK - 1) / BK;
  // Split where the tiles leave CUs idle and the sum is long, two workgroups a CU: each
  // part has eight steps at least, in whole words of scales.  (64 x 2304 with K = 4096
  // takes 9.5 us so, 15.1 in one; 768 x 768 with 16384 26 and 92; but with K = 2048 the
  // sums' way through memory costs what it saves: 768 x 768 11.0 and 9.5.)
  int64_t splits = 1;
  const int64_t room = 512 / tiles;
  if (S::SPLIT && room >= 2 && blocks >= 32) splits = std::min<int64_t>(room, blocks / 8);
  const int64_t steps = ((blocks + splits - 1) / splits + 3) / 4 * 4;
  splits = blocks ? (blocks + steps - 1) / steps : 1;
  p.steps = (int)steps;
  p.splits = (int)splits;
  p.bytes = splits > 1 ? splits * tiles * S::BM * S::BN * 4 : 0;
}

template <typename S> hipError_t run(Q8Matmul a, const Q8Plan& p, hipStream_t s) {
  static PerDevice ready;
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e == hipSuccess)
    e = ready.once(device, [] {
      return hipFuncSetAttribute(reinterpret_cast<const void*>(&q8_matmul_kernel<S>),
                                 hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS);
    });
  if (e != hipSuccess) return e;
  a.tiles_m = (int)((a.M + S::BM - 1) / S::BM);
  a.tiles_n = (int)((a.N + S::BN - 1) / S::BN);
  a.blocks = (int)((a.K + BK - 1) / BK);
  a.steps = p.steps;
  a.splits = p.splits;
  if (p.splits == 1) a.parts = nullptr;
  const unsigned tiles = (unsigned)((int64_t)a.tiles_m * a.tiles_n);
  hipLaunchKernelGGL((q8_matmul_kernel<S>), dim3(tiles, p.splits), dim3(S::THREADS), S::LDS, s, a);
  if constexpr (S::SPLIT)
    if (p.splits > 1) hipLaunchKernelGGL((q8_join_kernel<S>), dim3(tiles * S::FM), dim3(S::THREADS), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t q8_quantise(Q8Quantise a, bool bf16, hipStream_t s) {
  a.across = (unsigned)((a.cols + QT - 1) / QT);
  const int64_t tiles = a.across * ((a.rows + QT - 1) / QT), most = (1 << 24) - 1;  // (a launch has less than 2^32 threads)
  hipError_t e = hipSuccess;
  for (int64_t first = 0; first < tiles && e == hipSuccess; first += most) {
    const dim3 grid((unsigned)std::min(most, tiles - first));
    a.first = (uint32_t)first;
    if (bf16) hipLaunchKernelGGL((q8_quantise_kernel<bf16_t>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((q8_quantise_kernel<float>), grid, dim3(256), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

Q8Plan q8_plan(int64_t M, int64_t N, int64_t K) {
  Q8Plan p{};
  const int64_t large = ((M + 255) / 256) * ((N + 255) / 256), small = ((M + 63) / 64) * ((N + 63) / 64);
  // What was measured, us (K = 768 where no other is named):
  //   Large from about three tiles a CU on: 24576 x 4608 120 (Medium 128), 12288 x 4608
  //   with K = 1536 103.5 (106); with 576 tiles 80.1 (75.7).
  //   Small while all of its tiles run at once, two a CU: 1024 x 2048 6.5 (Medium 9.2),
  //   2048 x 1024 with K = 1536 9.0 (13.1); 1100 x 2048 9.6 (9.3).
  //   A long sum over tiles that cannot be split further favours Medium's fewer bytes a
  //   product: 2304 x 768 with K = 4096 21.6 (Small 16.9), with K = 16384 47 (62.7).
  // (Of 64 rows or columns Medium's tiles would be half empty.)
  p.kind = large >= 832 ? 2 : M > 64 && N > 64 && (small > 512 || (small > 256 && K >= 8192)) ? 1 : 0;
  if (p.kind == 2) plan_of<Large>(p, M, N, K);
  else if (p.kind == 1) plan_of<Medium>(p, M, N, K);
  else plan_of<Small>(p, M, N, K);
  return p;
}

hipError_t q8_matmul(const Q8Matmul& a, hipStream_t s) {
  const Q8Plan p = q8_plan(a.M, a.N, a.K);
  return p.kind == 2 ? run<Large>(a, p, s) : p.kind == 1 ? run<Medium>(a, p, s) : run<Small>(a, p, s);
}

}  // namespace am
