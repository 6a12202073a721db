// AdamW over many tensors in one launch (several beyond AdamwBatch::MAX), in
// this order and without fused multiply-adds, each operation rounded to fp32, so
// that the result is the element-wise definition's bit for bit:
//   g = grad * grad_scale;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) (g g);
//   w = w keep - step (m / (sqrt(v) root + eps)).
// HBM bounds it: 30 bytes an element with 32-bit moments, fp32 gradients and the
// bf16 copy, 18 with 8-bit moments.
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
#include "am_device.h"
#include "am_internal.h"

namespace am {
namespace {

typedef f32x4_t f32x4_u __attribute__((aligned(4)));
typedef uint16_t u16x4_t __attribute__((ext_vector_type(4)));
typedef u16x4_t u16x4_u __attribute__((aligned(2)));
typedef uint32_t u32_u __attribute__((aligned(1)));

// Four elements from place e of a tensor's n (any alignment), zeros past them.
__device__ __forceinline__ f32x4_t load4(const float* p, int64_t e, int64_t n) {
  f32x4_t v = {0.f, 0.f, 0.f, 0.f};
  if (e + 4 <= n) v = *reinterpret_cast<const f32x4_u*>(p + e);
  else
    for (int k = 0; k < 3; ++k)
      if (e + k < n) v[k] = p[e + k];
  return v;
}
__device__ __forceinline__ f32x4_t load4(const bf16_t* p, int64_t e, int64_t n) {
  u16x4_t h = {0, 0, 0, 0};
  if (e + 4 <= n) h = *reinterpret_cast<const u16x4_u*>(p + e);
  else
    for (int k = 0; k < 3; ++k)
      if (e + k < n) h[k] = p[e + k];
  f32x4_t v;
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = bf16_to_f32(h[k]);
  return v;
}
__device__ __forceinline__ void store4(float* p, int64_t e, int64_t n, f32x4_t v) {
  if (e + 4 <= n) *reinterpret_cast<f32x4_u*>(p + e) = v;
  else
    for (int k = 0; k < 3; ++k)
      if (e + k < n) p[e + k] = v[k];
}
__device__ __forceinline__ void store4(bf16_t* p, int64_t e, int64_t n, f32x4_t v) {
  u16x4_t h;
#pragma unroll
  for (int k = 0; k < 4; ++k) h[k] = f32_to_bf16(v[k]);
  if (e + 4 <= n) *reinterpret_cast<u16x4_u*>(p + e) = h;
  else
    for (int k = 0; k < 3; ++k)
      if (e + k < n) p[e + k] = h[k];
}

// Four codes (a byte each, element e's the lowest) and what they stand for.
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int64_t e, int64_t n) {
  if (e + 4 <= n) return *reinterpret_cast<const u32_u*>(p + e);
  uint32_t c = 0;
  for (int k = 0; k < 3; ++k)
    if (e + k < n) c |= (uint32_t)p[e + k] << (8 * k);
  return c;
}
__device__ __forceinline__ void store_codes(uint8_t* p, int64_t e, int64_t n, uint32_t c) {
  if (e + 4 <= n) *reinterpret_cast<u32_u*>(p + e) = c;
  else
    for (int k = 0; k < 3; ++k)
      if (e + k < n) p[e + k] = (uint8_t)(c >> (8 * k));
}
__device__ __forceinline__ f32x4_t decode(uint32_t c, float scale) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
  return f32x4_t{lo[0] * scale, lo[1] * scale, hi[0] * scale, hi[1] * scale};
}

__device__ __forceinline__ uint32_t hash(uint32_t i, uint32_t key) {
  uint32_t x = i * 0x85EBCA6Bu + key;
  x = (x ^ (x >> 15)) * 0xD168AAADu;
  x = (x ^ (x >> 15)) * 0xAF723597u;
  return x ^ (x >> 15);
}

// |x| < 256 on the codes' grid, up with probability (what is cut off), `bits` of
// 65536 the draw.  Adding the draw below the code's last bit carries into it
// exactly when the two exceed one unit; below 2^-6 the unit is 2^-9 throughout.
__device__ __forceinline__ uint32_t encode(float x, uint32_t bits, uint32_t least) {
  const uint32_t u = __float_as_uint(x), mag = u & 0x7fffffffu;
  const uint32_t normal = ((mag + (bits << 4)) >> 20) - (120u << 3);
  const uint32_t small = ((uint32_t)(__uint_as_float(mag) * 33554432.f) + bits) >> 16;
  uint32_t c = mag < (121u << 23) ? small : normal;
  if (mag != 0 && c < least) c = least;
  if (mag >= 0x7f800000u) c = 0x7f;
  return c | ((u >> 31) << 7);
}

// The block's codes and scale from four values a lane.
__device__ __forceinline__ uint32_t encode4(f32x4_t v, const uint32_t (&bits)[4], uint32_t least,
                                            float* scale) {
#pragma clang fp contract(off)
  float top = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float m = fabsf(v[k]);
    top = fmaxf(top, m < __builtin_inff() ? m : 0.f);
  }
  top = wave_max_uniform(top);
  const int e = (int)(__float_as_uint(top) >> 23) - 7;
  const uint32_t ex = e < 1 ? 1u : (uint32_t)e;
  *scale = __uint_as_float(ex << 23);
  const float inv = __uint_as_float((254u - ex) << 23);
  uint32_t c = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) c |= encode(v[k] * inv, bits[k], least) << (8 * k);
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

template <typename G, bool CODES>
__global__ __launch_bounds__(256) void adamw_kernel(AdamwBatch a) {
#pragma clang fp contract(off)
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
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int64_t n = t.n, base = (int64_t)(blockIdx.x - a.first[lo]) * ADAMW_CHUNK;
#pragma unroll
  for (int q = 0; q < ADAMW_CHUNK / 1024; ++q) {
    const int64_t start = base + (q * 4 + w) * 256, e = start + lane * 4;
    if (start >= n) return;
    const f32x4_t wv = load4(t.w, e, n);
    f32x4_t g = load4(static_cast<const G*>(t.g), e, n);
    if (a.grad_scale) g *= gs;
    if constexpr (CODES) {
      const int64_t blk = start >> 8;
      const uint32_t mc = load_codes(static_cast<const uint8_t*>(t.m), e, n);
      const uint32_t vc = load_codes(static_cast<const uint8_t*>(t.v), e, n);
      const f32x4_t r = decode(vc, t.v_scale[blk]);
      const Moments o = step4(a, wv, g, decode(mc, t.m_scale[blk]), r * r, t.keep);
      uint32_t for_m[4], for_v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t h = hash((uint32_t)(e + k), t.key);
        for_m[k] = h & 0xFFFFu;
        for_v[k] = h >> 16;
      }
      float ms, vs;
      const uint32_t mo = encode4(o.m, for_m, 0, &ms), vo = encode4(o.r, for_v, 1, &vs);
      store4(t.w, e, n, o.w);
      if (t.w16) store4(t.w16, e, n, o.w);
      store_codes(static_cast<uint8_t*>(t.m), e, n, mo);
      store_codes(static_cast<uint8_t*>(t.v), e, n, vo);
      if (lane == 0) {
        t.m_scale[blk] = ms;
        t.v_scale[blk] = vs;
      }
    } else {
      const Moments o = step4(a, wv, g, load4(static_cast<const float*>(t.m), e, n),
                              load4(static_cast<const float*>(t.v), e, n), t.keep);
      store4(t.w, e, n, o.w);
      if (t.w16) store4(t.w16, e, n, o.w);
      store4(static_cast<float*>(t.m), e, n, o.m);
      store4(static_cast<float*>(t.v), e, n, o.v);
    }
  }
}

}  // namespace

hipError_t adamw_launch(const AdamwBatch& a, bool grad_bf16, bool codes, hipStream_t s) {
  const unsigned grid = a.first[a.count];
  if (grid == 0) return hipSuccess;
  if (grad_bf16) {
    if (codes) hipLaunchKernelGGL((adamw_kernel<bf16_t, true>), dim3(grid), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((adamw_kernel<bf16_t, false>), dim3(grid), dim3(256), 0, s, a);
  } else {
    if (codes) hipLaunchKernelGGL((adamw_kernel<float, true>), dim3(grid), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((adamw_kernel<float, false>), dim3(grid), dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace am
