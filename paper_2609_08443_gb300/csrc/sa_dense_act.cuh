// Activations of the linear layer and their slopes, in fp32.
#pragma once
#include "sa_dense.cuh"
#include "sa_ptx.cuh"

namespace sa {
namespace dense {

// Eight neighbours, 16-byte aligned.
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float* v) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = __uint_as_float(w[j] << 16);
    v[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float* v) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float* v) {
  *reinterpret_cast<uint4*>(p) = make_uint4(ptx::pack_bf16(v[0], v[1]), ptx::pack_bf16(v[2], v[3]),
                                            ptx::pack_bf16(v[4], v[5]), ptx::pack_bf16(v[6], v[7]));
}
__device__ __forceinline__ void store8(float* p, const float* v) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

// 16 bytes on their way from memory to this thread's place in shared memory.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// ... through L1, where the neighbour's half of the same 32 bytes is found again
__device__ __forceinline__ void copy16_l1(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// 16 bytes of neighbours: eight bf16 or four fp32.  Loads of what the kernel does not write, so that they may go ahead of
// stores.
__device__ __forceinline__ void load16(const __nv_bfloat16* p, float* v) {
  const uint4 u = __ldg(reinterpret_cast<const uint4*>(p));
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = __uint_as_float(w[j] << 16);
    v[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load16(const float* p, float* v) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(p));
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
}
__device__ __forceinline__ float ld_nc(const float* p) { return __ldg(p); }
__device__ __forceinline__ float ld_nc(const __nv_bfloat16* p) {
  return __uint_as_float(uint32_t(__ldg(reinterpret_cast<const unsigned short*>(p))) << 16);
}
__device__ __forceinline__ void store16(__nv_bfloat16* p, const float* v) { store8(p, v); }
__device__ __forceinline__ void store16(float* p, const float* v) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
}
// 16 bytes of neighbours, or four bf16
template <int N>
__device__ __forceinline__ void load_n(const float* p, float* v) { load16(p, v); }
template <int N>
__device__ __forceinline__ void load_n(const __nv_bfloat16* p, float* v) {
  if (N == 8) {
    load16(p, v);
  } else {
    const uint2 u = __ldg(reinterpret_cast<const uint2*>(p));
    v[0] = __uint_as_float(u.x << 16), v[1] = __uint_as_float(u.x & 0xFFFF0000u);
    v[2] = __uint_as_float(u.y << 16), v[3] = __uint_as_float(u.y & 0xFFFF0000u);
  }
}
template <int N>
__device__ __forceinline__ void store_n(float* p, const float* v) { store16(p, v); }
template <int N>
__device__ __forceinline__ void store_n(__nv_bfloat16* p, const float* v) {
  if (N == 8)
    store16(p, v);
  else
    *reinterpret_cast<uint2*>(p) = make_uint2(ptx::pack_bf16(v[0], v[1]), ptx::pack_bf16(v[2], v[3]));
}

// Term k of an fp32 value of which `left` is left: that rounded to nearest, but bf16's largest where a finite value would round
// to an infinity, whose remainder would be a NaN.
__device__ __forceinline__ __nv_bfloat16 term_of(float left, int k) {
  const __nv_bfloat16 t = __float2bfloat16_rn(left);
  if (k == 0 && fabsf(left) >= 3.3961775e38f && fabsf(left) <= 3.4028235e38f)
    return __float2bfloat16_rz(left);
  return t;
}

// Eight fp32 values as three terms of bf16 each, in planes `plane` elements apart: nothing is left after the third for sizes
// from 2^-110 on; below, what lies under half of bf16's smallest subnormal, 2^-134, is lost.
__device__ __forceinline__ void store_terms(__nv_bfloat16* p, int64_t plane, const float* v) {
  float left[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) left[j] = v[j];
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    float t[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      t[j] = __bfloat162float(term_of(left[j], k));
      left[j] -= t[j];
    }
    store8(p + k * plane, t);
  }
}

// 1 / (1 + e^-z), from the hardware's 2^x and 1/x (a few 2^-23).  FULL, for fp32 results: -z log2 e is kept in two
// parts, since its rounding, times |z|, would be the largest error by far, and 1/x gets a Newton step.
template <bool FULL>
__device__ __forceinline__ float sigmoid(float z) {
  if (!FULL) return ptx::rcp_approx(1.f + ptx::ex2(-1.4426950409f * z));
  const float t = -1.4426950409f * z;
  // what the product and the constant were rounded by: log2 e = 1.44269502... + 1.92596e-8
  const float low = fmaf(-1.4426950409f, z, -t) - 1.92596302e-8f * z;
  float e = ptx::ex2(t);
  e = isinf(e) || t < -126.f ? e : fmaf(e, 0.69314718f * low, e);
  const float d = 1.f + e, r = ptx::rcp_approx(d);
  return isinf(d) ? r : fmaf(r, fmaf(-d, r, 1.f), r);
}

// z sigmoid<false>(z) of two neighbours; the products and sums go in pairs
__device__ __forceinline__ void silu_pair(float* v) {
  const float2 z = make_float2(v[0], v[1]);
  const float2 t = __fmul2_rn(z, make_float2(-1.4426950409f, -1.4426950409f));
  const float2 d = __fadd2_rn(make_float2(ptx::ex2(t.x), ptx::ex2(t.y)), make_float2(1.f, 1.f));
  const float2 y = __fmul2_rn(z, make_float2(ptx::rcp_approx(d.x), ptx::rcp_approx(d.y)));
  v[0] = y.x, v[1] = y.y;
}

// Phi(z) and e^(-z^2/2), Phi the normal distribution function.
// FULL: from CUDA's erfc.  Else Phi(-x) = e^(-x^2/2) R(1 / (1 + 0.31 x)) for x >= 0, R of degree 6 without a constant
// term: a least-squares fit with weights that level the relative error over 0 <= x <= 20 (Lawson's
// iteration), 7.5e-6 at most; bf16's half step is 2e-3 to 4e-3.
template <bool FULL>
__device__ __forceinline__ float normal_cdf(float z, float* density) {
  const float e = FULL ? expf(-0.5f * z * z) : ptx::ex2(-0.72134752f * z * z);
  if (density) *density = e;
  if (FULL) return 0.5f * erfcf(-0.70710678f * z);
  const float t = ptx::rcp_approx(fmaf(0.31f, fabsf(z), 1.f));
  float r = fmaf(-0.07230377f, t, 0.17592333f);
  r = fmaf(r, t, 0.020491485f);
  r = fmaf(r, t, 0.13110992f);
  r = fmaf(r, t, 0.120964423f);
  r = fmaf(r, t, 0.12381754f) * t * e;
  return z < 0.f ? r : 1.f - r;
}

// z normal_cdf<false>(z) of two neighbours
__device__ __forceinline__ void gelu_pair(float* v) {
  auto two = [](float c) { return make_float2(c, c); };
  const float2 z = make_float2(v[0], v[1]);
  const float2 q = __fmul2_rn(__fmul2_rn(two(-0.72134752f), z), z);
  const float2 d = __ffma2_rn(two(0.31f), make_float2(fabsf(z.x), fabsf(z.y)), two(1.f));
  const float2 t = make_float2(ptx::rcp_approx(d.x), ptx::rcp_approx(d.y));
  float2 r = __ffma2_rn(two(-0.07230377f), t, two(0.17592333f));
  r = __ffma2_rn(r, t, two(0.020491485f));
  r = __ffma2_rn(r, t, two(0.13110992f));
  r = __ffma2_rn(r, t, two(0.120964423f));
  r = __ffma2_rn(r, t, two(0.12381754f));
  r = __fmul2_rn(__fmul2_rn(r, t), make_float2(ptx::ex2(q.x), ptx::ex2(q.y)));
  const float2 u = __ffma2_rn(two(-1.f), r, two(1.f));
  const float2 y = __fmul2_rn(z, make_float2(z.x < 0.f ? r.x : u.x, z.y < 0.f ? r.y : u.y));
  v[0] = y.x, v[1] = y.y;
}

// act(z) of one value (SA_ACT_SWIGLU: of the gate's half)
template <bool FULL>
__device__ __forceinline__ float activate(int act, float z) {
  switch (act) {
    case SA_ACT_RELU: return z < 0.f ? 0.f : z;  // a NaN stays one
    case SA_ACT_GELU: return z * normal_cdf<FULL>(z, nullptr);
    case SA_ACT_SILU:
    case SA_ACT_SWIGLU: return z * sigmoid<FULL>(z);
    default: return z;
  }
}

// act'(z)
template <bool FULL>
__device__ __forceinline__ float slope(int act, float z) {
  switch (act) {
    case SA_ACT_RELU: return z > 0.f ? 1.f : 0.f;
    case SA_ACT_GELU: {
      float e;
      const float p = normal_cdf<FULL>(z, &e);
      return fmaf(z * 0.39894228f, e, p);  // Phi + z phi, phi = e^(-z^2/2) / sqrt(2 pi)
    }
    case SA_ACT_SILU:
    case SA_ACT_SWIGLU: {
      const float p = sigmoid<FULL>(z);
      return p * fmaf(z, 1.f - p, 1.f);
    }
    default: return 1.f;
  }
}

}  // namespace dense
}  // namespace sa
