// The 4-bit cache: page geometry, the format's arithmetic on the device, and the
// interface between the host API (sa_cache_api.cu) and the kernel files.
#pragma once
#include <cuda_fp16.h>

#include "../../include/sa_cache.h"
#include "sa_common.cuh"

namespace sa {
namespace cache {

constexpr int kGroup = 16;        // features per scale
constexpr uint32_t kCodeMin = 8;  // 2^-14: the smallest normal float16, so every scale has four significant bits
constexpr uint32_t kCodeMax = 225;  // 9216: 7 x 9216 is the largest multiple that float16 holds

// Where the cached rows are.
struct Pages {
  const uint8_t* pool;
  int64_t n_pages;
  const int32_t* table;  // [B, max_pages]
  int max_pages;
  int page, log2page;
  int H, d;
  int rec;  // bytes of one record (keys or values of one page and head)

  // Byte offset of the key record of (page p, head h); the value record follows it.
  SA_HD int64_t record(int64_t p, int h) const { return (p * H + h) * 2 * int64_t(rec); }
};

struct RowArgs {
  Pages c;
  const void *K, *V;  // write: sources
  void *Ko, *Vo;      // read: destinations [N, H, d]
  int64_t user_stride, row_stride, head_stride;
  const int32_t* cu;  // NULL: `per_user` rows each
  int64_t per_user;
  int B;
  int64_t N;
  const int32_t* start;
  sa_dtype dt;
  void* ws;
};

struct AttnArgs {
  Pages c;
  const void* q;
  int64_t q_row, q_head;  // strides in elements
  const int32_t* cu_q;
  int B;
  int64_t T;
  int Hq, G;  // query heads, query heads per cached head
  const int32_t *lens, *begin, *end;
  float scale;
  sa_dtype dt;
  void* out;        // forward: destination; backward: the forward's result
  float* lse;       // forward: destination or NULL; backward: the forward's result
  const void* dout;
  void* dq;
  int workers;      // contiguous shares of the work
  void* ws;         // header
  WsHeader* slots;  // [CTAs] error word and wait limit of each CTA
  int ctas;
  void* piece;      // [workers] what each worker's first segment is
  float* partial;   // [workers][2] unfinished sums of cut segments
  uint64_t wait_limit_ns;
};

cudaError_t launch_write(const RowArgs& a, cudaStream_t st);
cudaError_t launch_read(const RowArgs& a, cudaStream_t st);

// Warp-level kernels (sa_cache_mma.cu)
struct AttnPlan {
  int ctas, workers;
  size_t piece_bytes, partial_floats;  // per worker; per worker and slot
};
AttnPlan mma_plan(int sms, int B, int64_t T, int G, int d, sa_dtype dt, bool bwd);
cudaError_t launch_mma(const AttnArgs& a, bool bwd, cudaStream_t st);

// tcgen05 kernels (sa_cache_tc.cu, sa_cache_tc_bwd.cu)
bool tc_supported(int B, int64_t T, int G, int d, sa_dtype dt, float scale, bool bwd);
AttnPlan tc_plan(int sms, int d, bool bwd);
cudaError_t launch_tc_bwd(const AttnArgs& a, cudaStream_t st);
cudaError_t launch_tc(const AttnArgs& a, bool bwd, cudaStream_t st);

// ------------------------------------------------------------------ arithmetic
#ifdef __CUDACC__
// The fp32 value of a scale code: the float16 with bits code << 7.
__device__ __forceinline__ float scale_value(uint32_t code) {
  return __uint_as_float((code << 20) + ((127u - 15u) << 23));
}

// Code of the smallest scale with 7.5 s >= big, within [kCodeMin, kCodeMax].  The
// first guess truncates 2/15 big to the scale's four bits; both corrections compare
// exact products (15 (8 + m) / 2 has eight significant bits).
__device__ __forceinline__ uint32_t scale_code(float big) {
  const int guess = int(__float_as_uint(big * (2.f / 15.f)) >> 20) - ((127 - 15) << 3);
  uint32_t c = uint32_t(min(max(guess, int(kCodeMin)), int(kCodeMax)));
  if (c < kCodeMax && 7.5f * scale_value(c) < big) ++c;
  if (c > kCodeMin && 7.5f * scale_value(c - 1) >= big) --c;
  return c;
}

__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t fma_f16x2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ uint32_t add_f16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("add.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t and_or(uint32_t a, uint32_t m, uint32_t o) {
  uint32_t d;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(a), "r"(m), "r"(o));  // (a & m) | o
  return d;
}

// bf16 scales of the codes in the two halves of `cc`, as (s / 8, -24 s): a level field
// u at mantissa bits 3..6 of 128.0 reads 128 + 8 u, and (128 + 8 u) s/8 - 24 s =
// (u - 8) s in one rounding, which is exact (24 s has six significant bits).
struct ScaleB {
  uint32_t s8, c;
};
__device__ __forceinline__ ScaleB scale_bf16(uint32_t cc) {
  ScaleB r;
  r.s8 = cc * 16u + 0x36803680u;
  r.c = mul_bf16x2(r.s8, 0xC340C340u);  // -192
  return r;
}
// word of codes -> four bf16 pairs
__device__ __forceinline__ void values_bf16(uint32_t w, ScaleB s, uint32_t* r) {
  r[0] = fma_bf16x2(and_or(w << 3, 0x00780078u, 0x43004300u), s.s8, s.c);
  r[1] = fma_bf16x2(and_or(w >> 1, 0x00780078u, 0x43004300u), s.s8, s.c);
  r[2] = fma_bf16x2(and_or(w >> 5, 0x00780078u, 0x43004300u), s.s8, s.c);
  r[3] = fma_bf16x2(and_or(w >> 9, 0x00780078u, 0x43004300u), s.s8, s.c);
}
// word of codes -> four float16 pairs, times the float16 scales s2.  The level comes
// first and alone (72 s would pass float16's range), then one exact product.
__device__ __forceinline__ void values_f16(uint32_t w, uint32_t s2, uint32_t* r) {
  const uint32_t v = w >> 8;
  r[0] = mul_f16x2(add_f16x2(and_or(w, 0x000F000Fu, 0x64006400u), 0xE408E408u), s2);               // 1024 + u - 1032
  r[1] = mul_f16x2(fma_f16x2(and_or(w, 0x00F000F0u, 0x64006400u), 0x2C002C00u, 0xD480D480u), s2);  // (1024 + 16 u) / 16 - 72
  r[2] = mul_f16x2(add_f16x2(and_or(v, 0x000F000Fu, 0x64006400u), 0xE408E408u), s2);
  r[3] = mul_f16x2(fma_f16x2(and_or(v, 0x00F000F0u, 0x64006400u), 0x2C002C00u, 0xD480D480u), s2);
}

// What no written row has, but bytes that nobody wrote can: a code above kCodeMax, which
// float16 reads as an infinity, a NaN or a value past the format's range, and level -8
// with one of the two scales (codes 224, 225) whose eighth multiple float16 does not hold.
// A hidden position's weight is 0, and 0 x inf is not 0, so such codes count as 0 and
// such levels as -7; written rows come out as they are.
constexpr uint32_t kCodeSafe = 223;  // up to it 8 x scale is finite
__device__ __forceinline__ uint32_t level_min7(uint32_t w) {
  uint32_t any = w | w >> 1;
  any |= any >> 2;  // the lowest bit of each nibble: whether it has one set
  return w | (~any & 0x11111111u);
}
#endif

}  // namespace cache
}  // namespace sa
