// AdamW over many tensors in one launch (several beyond AdamwBatch::MAX), in
// this order and without fused multiply-adds, each operation rounded to fp32, so
// that the result is the element-wise definition's bit for bit:
//   g = grad * grad_scale;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) (g g);
//   w = w keep - step (m / (sqrt(v) root + eps)).
// HBM bounds it: 30 bytes an element with 32-bit moments, fp32 gradients and the
// bf16 copy, 18 with 8-bit moments (16 with bf16 gradients).  24.1 M elements with
// 32-bit moments: 120 us (6.0 TB/s); 95.4 M with 8-bit moments and bf16 gradients: 277 us (5.5
// TB/s), where 111 vector instruction slots an element are as long (269 us counted).
// A launch has up to 48 tensors, a workgroup 2048 elements of one: every load of a
// wave's two blocks comes before the first use.
//
// 8-bit moments: blocks of 256 elements of a tensor share a scale, the power of
// two that puts the block's largest magnitude into [128, 256); m and sqrt(v) are
// held in units of it as 8-bit floats of 4 exponent and 3 fraction bits (down to
// 2^-9).  A wave has a block, four elements a lane.  An average that moves by a
// thousandth a step would never leave its code if codes were rounded to nearest,
// so they are rounded up with the probability of what is cut off (16 bits of a
// hash of the element's index, its tensor's number and the caller's seed).  A
// nonzero sqrt(v) keeps the smallest code at least: with code 0 under an m that
// has one, an element without a gradient would step by m / eps.
#include <type_traits>

#include "am_device.h"
#include "am_internal.h"

namespace am {
namespace {

typedef f32x4_t f32x4_u __attribute__((aligned(4)));
typedef uint16_t u16x4_t __attribute__((ext_vector_type(4)));
typedef u16x4_t u16x4_u __attribute__((aligned(2)));
typedef uint32_t u32_u __attribute__((aligned(1)));

// Four elements from place e of a tensor's n, at any alignment.  WHOLE: all four
// are there; else those past the end are zeros, or not stored.  STREAM: past the
// caches.
template <bool WHOLE, bool STREAM> struct Access {
  __device__ __forceinline__ static f32x4_t load(const float* p, int64_t e, int64_t n) {
    if (WHOLE || e + 4 <= n) {
      const f32x4_u* at = reinterpret_cast<const f32x4_u*>(p + e);
      if constexpr (STREAM) return __builtin_nontemporal_load(at);
      else return *at;
    }
    f32x4_t v = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < 3; ++k)
      if (e + k < n) v[k] = p[e + k];
    return v;
  }
  __device__ __forceinline__ static u16x4_t load(const bf16_t* p, int64_t e, int64_t n) {
    if (WHOLE || e + 4 <= n) {
      const u16x4_u* at = reinterpret_cast<const u16x4_u*>(p + e);
      if constexpr (STREAM) return __builtin_nontemporal_load(at);
      else return *at;
    }
    u16x4_t v = {0, 0, 0, 0};
    for (int k = 0; k < 3; ++k)
      if (e + k < n) v[k] = p[e + k];
    return v;
  }
  // codes: a byte each, element e's the lowest
  __device__ __forceinline__ static uint32_t load(const uint8_t* p, int64_t e, int64_t n) {
    if (WHOLE || e + 4 <= n) {
      const u32_u* at = reinterpret_cast<const u32_u*>(p + e);
      if constexpr (STREAM) return __builtin_nontemporal_load(at);
      else return *at;
    }
    uint32_t c = 0;
    for (int k = 0; k < 3; ++k)
      if (e + k < n) c |= (uint32_t)p[e + k] << (8 * k);
    return c;
  }
  __device__ __forceinline__ static void store(float* p, int64_t e, int64_t n, f32x4_t v) {
    if (WHOLE || e + 4 <= n) {
      f32x4_u* at = reinterpret_cast<f32x4_u*>(p + e);
      if constexpr (STREAM) __builtin_nontemporal_store(v, at);
      else *at = v;
    } else {
      for (int k = 0; k < 3; ++k)
        if (e + k < n) p[e + k] = v[k];
    }
  }
  __device__ __forceinline__ static void store(bf16_t* p, int64_t e, int64_t n, f32x4_t v) {
    typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = v[k] == v[k] ? v[k] : __builtin_nanf("");  // (0x7FC0)
    const u16x4_t h = __builtin_bit_cast(u16x4_t, __builtin_convertvector(v, bf16x4_t));  // (to nearest even)
    if (WHOLE || e + 4 <= n) {
      u16x4_u* at = reinterpret_cast<u16x4_u*>(p + e);
      if constexpr (STREAM) __builtin_nontemporal_store(h, at);
      else *at = h;
    } else {
      for (int k = 0; k < 3; ++k)
        if (e + k < n) p[e + k] = h[k];
    }
  }
  __device__ __forceinline__ static void store(uint8_t* p, int64_t e, int64_t n, uint32_t c) {
    if (WHOLE || e + 4 <= n) {
      u32_u* at = reinterpret_cast<u32_u*>(p + e);
      if constexpr (STREAM) __builtin_nontemporal_store(c, at);
      else *at = c;
    } else {
      for (int k = 0; k < 3; ++k)
        if (e + k < n) p[e + k] = (uint8_t)(c >> (8 * k));
    }
  }
};

__device__ __forceinline__ f32x4_t wide(f32x4_t v) { return v; }
__device__ __forceinline__ f32x4_t wide(u16x4_t v) {
  f32x4_t o;
#pragma unroll
  for (int k = 0; k < 4; ++k) o[k] = bf16_to_f32(v[k]);
  return o;
}

__device__ __forceinline__ f32x4_t decode(uint32_t c, float scale) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
  return f32x4_t{lo[0] * scale, lo[1] * scale, hi[0] * scale, hi[1] * scale};
}

// (Two multipliers and shifts of 15: published constants, from a search for hashes of
// 32 bits of little bias, hash-prospector.)
__device__ __forceinline__ uint32_t hash(uint32_t i, uint32_t key) {
  uint32_t x = i * 0x85EBCA6Bu + key;
  x = (x ^ (x >> 15)) * 0xD168AAADu;
  x = (x ^ (x >> 15)) * 0xAF723597u;
  return x ^ (x >> 15);
}

// |x| < 256 on the codes' grid, up with probability (what is cut off), `bits` of
// 65536 the draw.  Adding the draw below the code's last bit carries into it
// exactly when the two exceed one unit; below 2^-6 the unit is 2^-9 throughout.
// LEAST: the smallest code of what is not zero.
template <bool LEAST> __device__ __forceinline__ uint32_t encode(float x, uint32_t bits) {
  const uint32_t u = __float_as_uint(x), mag = u & 0x7fffffffu;
  const uint32_t normal = ((mag + (bits << 4)) >> 20) - (120u << 3);
  const uint32_t small = ((uint32_t)(__uint_as_float(mag) * 33554432.f) + bits) >> 16;
  uint32_t c = mag < (121u << 23) ? small : normal;
  if (LEAST) c = max(c, min(mag, 1u));  // (a root has no sign)
  else c |= (u >> 31) << 7;
  return c;
}

// The block's codes and scale from four values a lane.
template <bool LEAST>
__device__ __forceinline__ uint32_t encode4(f32x4_t v, const uint32_t (&bits)[4], float* scale) {
#pragma clang fp contract(off)
  float top = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) top = fmaxf(top, fabsf(v[k]));
  // (a sum with something in it that is not finite is not; nor is one that
  // overflows, which the loop below finds out)
  const float all = (fabsf(v[0]) + fabsf(v[1])) + (fabsf(v[2]) + fabsf(v[3]));
  const bool odd = __any(!(all < __builtin_inff()));
  uint32_t lost = 0;  // codes of what is not finite
  if (odd) {
    top = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (!(fabsf(v[k]) < __builtin_inff())) {
        lost |= 0x7fu << (8 * k);
        v[k] = 0.f;
      }
      top = fmaxf(top, fabsf(v[k]));
    }
  }
  top = wave_max_uniform(top);
  const int e = (int)(__float_as_uint(top) >> 23) - 7;
  const uint32_t ex = e < 1 ? 1u : (uint32_t)e;
  *scale = __uint_as_float(ex << 23);
  const float inv = __uint_as_float((254u - ex) << 23);
  uint32_t c = lost;
#pragma unroll
  for (int k = 0; k < 4; ++k) c |= encode<LEAST>(v[k] * inv, bits[k]) << (8 * k);
  return c;
}

struct Moments {
  f32x4_t w, m, r;  // r: sqrt(v)
  f32x4_t v;
};
__device__ __forceinline__ Moments step4(const AdamwBatch& a, f32x4_t w, f32x4_t g, f32x4_t m, f32x4_t v,
                                         float keep) {
#pragma clang fp contract(off)
  Moments o;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    o.m[k] = m[k] * a.b1 + g[k] * a.c1;
    o.v[k] = v[k] * a.b2 + g[k] * g[k] * a.c2;
    o.r[k] = sqrtf(o.v[k]);
    o.w[k] = w[k] * keep - o.m[k] / (o.r[k] * a.root + a.eps) * a.step;
  }
  return o;
}

// N blocks of 256 elements of one tensor, 1024 elements apart: every load first.
template <typename G, bool CODES, bool STREAM, bool WHOLE, int N>
__device__ __forceinline__ void blocks(const AdamwBatch& a, const AdamwOne& t, float gs, int64_t start, int lane) {
#pragma clang fp contract(off)
  typedef Access<WHOLE, STREAM> At;
  typedef typename std::conditional<CODES, uint8_t, float>::type S;  // a moment's element
  S *tm = static_cast<S*>(t.m), *tv = static_cast<S*>(t.v);
  decltype(At::load(tm, 0, 0)) m[N], v[N];
  decltype(At::load(static_cast<const G*>(t.g), 0, 0)) g[N];
  f32x4_t w[N];
  float ms[N], vs[N];
#pragma unroll
  for (int q = 0; q < N; ++q) {
    const int64_t e = start + q * 1024 + lane * 4;
    w[q] = At::load(t.w, e, t.n);
    g[q] = At::load(static_cast<const G*>(t.g), e, t.n);
    m[q] = At::load(tm, e, t.n);
    v[q] = At::load(tv, e, t.n);
    if constexpr (CODES) {
      ms[q] = t.m_scale[(start >> 8) + 4 * q];
      vs[q] = t.v_scale[(start >> 8) + 4 * q];
    }
  }
#pragma unroll
  for (int q = 0; q < N; ++q) {
    const int64_t e = start + q * 1024 + lane * 4;
    f32x4_t gq = wide(g[q]);
    if (a.grad_scale) gq *= gs;
    if constexpr (CODES) {
      const f32x4_t r = decode(v[q], vs[q]);
      const Moments o = step4(a, w[q], gq, decode(m[q], ms[q]), r * r, t.keep);
      uint32_t for_m[4], for_v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t h = hash((uint32_t)(e + k), t.key);
        for_m[k] = h & 0xFFFFu;
        for_v[k] = h >> 16;
      }
      const uint32_t mo = encode4<false>(o.m, for_m, &ms[q]), vo = encode4<true>(o.r, for_v, &vs[q]);
      At::store(t.w, e, t.n, o.w);
      if (t.w16) At::store(t.w16, e, t.n, o.w);
      At::store(tm, e, t.n, mo);
      At::store(tv, e, t.n, vo);
      if (lane == 0) {
        t.m_scale[(start >> 8) + 4 * q] = ms[q];
        t.v_scale[(start >> 8) + 4 * q] = vs[q];
      }
    } else {
      const Moments o = step4(a, w[q], gq, m[q], v[q], t.keep);
      At::store(t.w, e, t.n, o.w);
      if (t.w16) At::store(t.w16, e, t.n, o.w);
      At::store(tm, e, t.n, o.m);
      At::store(tv, e, t.n, o.v);
    }
  }
}

template <typename G, bool CODES, bool STREAM>
__global__ __launch_bounds__(256) void adamw_kernel(AdamwBatch a) {
  float gs = 1.f;
  if (a.grad_scale) {
    gs = *a.grad_scale;
    if (!(fabsf(gs) < __builtin_inff())) return;
  }
  int lo = 0, hi = a.count - 1;  // the tensor of this workgroup's elements
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.first[mid] <= blockIdx.x) lo = mid; else hi = mid - 1;
  }
  const AdamwOne& t = a.t[lo];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t start = (int64_t)(blockIdx.x - a.first[lo]) * ADAMW_CHUNK + w * 256;
  constexpr int N = ADAMW_CHUNK / 1024;
  if (start + (N - 1) * 1024 + 256 <= t.n) {
    blocks<G, CODES, STREAM, true, N>(a, t, gs, start, lane);
    return;
  }
  for (int q = 0; q < N; ++q)
    if (start + q * 1024 < t.n) blocks<G, CODES, STREAM, false, 1>(a, t, gs, start + q * 1024, lane);
}

}  // namespace

hipError_t adamw_launch(const AdamwBatch& a, bool grad_bf16, bool codes, int64_t bytes, hipStream_t s) {
  const unsigned grid = a.first[a.count];
  if (grid == 0) return hipSuccess;
  // Past the caches where the memory-side one (256 MB) keeps nothing that the next
  // step reads.  Through them / past them, us, steps one after another: 31 MB 7.4 /
  // 7.7, 126 MB 20 / 22, 252 MB 37 / 44, 377 MB 55 / 65 (8-bit, 386 MB: 67 / 77),
  // 676 MB 121 / 116, 724 MB 134 / 124, 2.99 GB 551 / 506 (8-bit, 1.59 GB: 306 /
  // 291).
  const bool stream = bytes > ((int64_t)512 << 20);
  auto kernel = grad_bf16 ? (codes ? (stream ? adamw_kernel<bf16_t, true, true> : adamw_kernel<bf16_t, true, false>)
                                   : (stream ? adamw_kernel<bf16_t, false, true> : adamw_kernel<bf16_t, false, false>))
                          : (codes ? (stream ? adamw_kernel<float, true, true> : adamw_kernel<float, true, false>)
                                   : (stream ? adamw_kernel<float, false, true> : adamw_kernel<float, false, false>));
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace am
