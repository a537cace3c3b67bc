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
int mma_workers(int sms, int d, sa_dtype dt, bool bwd, int* ctas);
size_t mma_piece_bytes();
size_t mma_partial_floats(int d);
cudaError_t launch_mma(const AttnArgs& a, bool bwd, cudaStream_t st);

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

// |x| / s to the nearest whole number, halves down, at most 7.  The quotient by the
// rounded reciprocal may sit on the wrong side of a half; the remainder x - q s is
// exact there (both are within a factor of two of each other), so it decides.
__device__ __forceinline__ uint32_t level_of(float ax, float s, float inv_s) {
  float q = fminf(rintf(ax * inv_s), 8.f);
  const float r = fmaf(-q, s, ax);
  if (r > 0.5f * s) q += 1.f;
  if (r <= -0.5f * s) q -= 1.f;
  return uint32_t(fminf(q, 7.f));
}
#endif

}  // namespace cache
}  // namespace sa
