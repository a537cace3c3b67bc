// Rows into the 4-bit cache and back (sa_cache_write, sa_cache_read).
//
// One thread handles one group of 16 features of one key or value row: writing, it
// takes the largest magnitude, picks the scale, rounds to levels and stores 8 code
// bytes and a scale byte; reading, it does the reverse.  Both are bound by memory
// (per feature 2 or 4 bytes of the row and 9/16 of the cache).  A block takes a run
// of tokens of one head, so that what it touches in a page is contiguous, and keys
// and values side by side (blockIdx.z).
#include "sa_cache.cuh"
#include "sa_kernels.cuh"
#include "sa_simt_util.cuh"

namespace sa {
namespace cache {

constexpr int kThreads = 256;

// Where row `row` of the call lives: its user, the offset of the source row and the
// cache position.  `ok` is false for offsets that lead outside the batch.
struct RowRef {
  bool ok;
  int b;
  int64_t i;    // row within the user
  int64_t pos;  // cache position
};

__device__ __forceinline__ RowRef find_row(const RowArgs& a, int64_t row) {
  RowRef r;
  if (a.cu) {
    r.b = user_of_token(a.cu, a.B, row);
    r.i = row - a.cu[r.b];
    r.ok = r.i >= 0 && row < a.cu[r.b + 1];
  } else {
    r.b = int(row / a.per_user);
    r.i = row - r.b * a.per_user;
    r.ok = true;
  }
  const int64_t s = a.start ? a.start[r.b] : 0;
  r.pos = s + r.i;
  r.ok = r.ok && s >= 0 && (r.pos >> a.c.log2page) < a.c.max_pages;
  return r;
}

// Byte offset of the row's record (K or V: kv), or -1 where there is no page.
__device__ __forceinline__ int64_t find_record(const RowArgs& a, const RowRef& r, int h, int kv) {
  const int p = a.c.table[int64_t(r.b) * a.c.max_pages + (r.pos >> a.c.log2page)];
  if (p < 0 || p >= a.c.n_pages) return -1;
  return a.c.record(p, h) + int64_t(kv) * a.c.rec;
}

// Checks of what the host cannot see, by one more block: writes the call's status.
__device__ void check_rows(const RowArgs& a) {
  __shared__ int bad;
  if (threadIdx.x == 0) bad = 0;
  __syncthreads();
  int mine = 0;
  for (int b = threadIdx.x; b < a.B; b += blockDim.x) {
    const int64_t c0 = a.cu ? int64_t(a.cu[b]) : b * a.per_user;
    const int64_t c1 = a.cu ? int64_t(a.cu[b + 1]) : (b + 1) * a.per_user;
    const int64_t s = a.start ? a.start[b] : 0;
    if ((b == 0 && c0 != 0) || (b == a.B - 1 && c1 != a.N) || c0 > c1 || s < 0 ||
        s + (c1 - c0) > (int64_t(a.c.max_pages) << a.c.log2page))
      mine = max(mine, int(SA_ERR_BAD_SEQLENS));
  }
  if (mine) atomicMax(&bad, mine);
  __syncthreads();
  if (bad == 0) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int b = warp; b < a.B; b += blockDim.x >> 5) {
      const int64_t n = a.cu ? a.cu[b + 1] - a.cu[b] : a.per_user;
      if (n == 0) continue;
      const int64_t s = a.start ? a.start[b] : 0;
      const int p0 = int(s >> a.c.log2page), p1 = int((s + n - 1) >> a.c.log2page);
      for (int p = p0 + lane; p <= p1; p += 32) {
        const int e = a.c.table[int64_t(b) * a.c.max_pages + p];
        if (e < 0 || e >= a.c.n_pages) mine = int(SA_ERR_BAD_PAGE);
      }
    }
    if (mine) atomicMax(&bad, mine);
    __syncthreads();
  }
  if (threadIdx.x == 0) ws_header(a.ws)->err = uint32_t(bad);
}

// Any offset out of order makes every block leave: the whole call writes nothing.
__device__ __forceinline__ bool offsets_ok(const RowArgs& a) {
  if (!a.cu) return true;
  int bad = 0;
  for (int b = threadIdx.x; b < a.B; b += blockDim.x)
    bad |= (b == 0 && a.cu[0] != 0) || (b == a.B - 1 && int64_t(a.cu[a.B]) != a.N) || a.cu[b] > a.cu[b + 1];
  return !__syncthreads_or(bad);
}

// grid: x = runs of tokens (+ 1 for the checks), y = heads, z = keys / values
template <typename T>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(RowArgs a, int rows_per_block) {
  if (blockIdx.x == gridDim.x - 1) {
    if (blockIdx.y == 0 && blockIdx.z == 0) check_rows(a);
    return;
  }
  if (!offsets_ok(a)) return;
  const int ng = a.c.d / kGroup, h = blockIdx.y, kv = blockIdx.z;
  const int64_t row0 = int64_t(blockIdx.x) * rows_per_block;
  const T* src = static_cast<const T*>(kv ? a.V : a.K) + int64_t(h) * a.head_stride;
  uint8_t* pool = const_cast<uint8_t*>(a.c.pool);
  for (int e = threadIdx.x; e < rows_per_block * ng; e += kThreads) {
    const int64_t row = row0 + e / ng;
    const int g = e % ng;
    if (row >= a.N) break;
    const RowRef r = find_row(a, row);
    if (!r.ok) continue;
    const int64_t rec = find_record(a, r, h, kv);
    if (rec < 0) continue;
    const T* p = src + (a.cu ? row : int64_t(0)) * a.row_stride +
                 (a.cu ? int64_t(0) : r.b * a.user_stride + r.i * a.row_stride) + g * kGroup;
    float x[kGroup];
#pragma unroll
    for (int k = 0; k < kGroup; k += Vec<T>::n) Vec<T>::load(p + k, x + k);
    float big = 0.f;
#pragma unroll
    for (int k = 0; k < kGroup; ++k) {
      if (isnan(x[k])) x[k] = 0.f;
      big = fmaxf(big, fabsf(x[k]));
    }
    const uint32_t code = scale_code(big);
    const float s = scale_value(code), inv = 1.f / s;
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int k = 0; k < kGroup; ++k) {
      const uint32_t l = level_of(fabsf(x[k]), s, inv);
      const uint32_t u = x[k] < 0.f ? 8u - l : 8u + l;
      w[k >> 3] |= u << (4 * (((k & 7) >> 1) + 4 * (k & 1)));
    }
    const int slot = int(r.pos & (a.c.page - 1));
    *reinterpret_cast<uint2*>(pool + rec + int64_t(slot) * (a.c.d / 2) + g * 8) = make_uint2(w[0], w[1]);
    pool[rec + int64_t(a.c.page) * (a.c.d / 2) + slot * ng + g] = uint8_t(code);
  }
}

template <typename T> __device__ __forceinline__ void store16(T* p, const float* x);
template <> __device__ __forceinline__ void store16<float>(float* p, const float* x) {
#pragma unroll
  for (int k = 0; k < 16; k += 4) *reinterpret_cast<float4*>(p + k) = make_float4(x[k], x[k + 1], x[k + 2], x[k + 3]);
}
template <> __device__ __forceinline__ void store16<__nv_bfloat16>(__nv_bfloat16* p, const float* x) {
#pragma unroll
  for (int k = 0; k < 16; k += 8) {
    __nv_bfloat162 v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = __floats2bfloat162_rn(x[k + 2 * j], x[k + 2 * j + 1]);
    *reinterpret_cast<uint4*>(p + k) = *reinterpret_cast<const uint4*>(v);
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(RowArgs a, int rows_per_block) {
  if (blockIdx.x == gridDim.x - 1) {
    if (blockIdx.y == 0 && blockIdx.z == 0) check_rows(a);
    return;
  }
  if (!offsets_ok(a)) return;
  const int ng = a.c.d / kGroup, h = blockIdx.y, kv = blockIdx.z;
  const int64_t row0 = int64_t(blockIdx.x) * rows_per_block;
  T* dst = static_cast<T*>(kv ? a.Vo : a.Ko) + int64_t(h) * a.c.d;
  for (int e = threadIdx.x; e < rows_per_block * ng; e += kThreads) {
    const int64_t row = row0 + e / ng;
    const int g = e % ng;
    if (row >= a.N) break;
    const RowRef r = find_row(a, row);
    if (!r.ok) continue;
    const int64_t rec = find_record(a, r, h, kv);
    if (rec < 0) continue;
    const int slot = int(r.pos & (a.c.page - 1));
    const uint2 w2 = *reinterpret_cast<const uint2*>(a.c.pool + rec + int64_t(slot) * (a.c.d / 2) + g * 8);
    const float s = scale_value(a.c.pool[rec + int64_t(a.c.page) * (a.c.d / 2) + slot * ng + g]);
    float x[kGroup];
#pragma unroll
    for (int k = 0; k < kGroup; ++k) {
      const uint32_t w = k < 8 ? w2.x : w2.y;
      x[k] = s * float(int((w >> (4 * (((k & 7) >> 1) + 4 * (k & 1)))) & 15u) - 8);
    }
    store16(dst + row * a.c.H * a.c.d + g * kGroup, x);
  }
}

// Rows a block takes: enough groups for its threads.
static int rows_per_block(const RowArgs& a) { return kThreads / (a.c.d / kGroup) > 0 ? kThreads / (a.c.d / kGroup) : 1; }

static dim3 row_grid(const RowArgs& a, int rpb) {
  return dim3(unsigned((a.N + rpb - 1) / rpb + 1), unsigned(a.c.H), 2);
}

cudaError_t launch_write(const RowArgs& a, cudaStream_t st) {
  const int rpb = rows_per_block(a);
  if (a.dt == SA_BF16)
    cache_write_kernel<__nv_bfloat16><<<row_grid(a, rpb), kThreads, 0, st>>>(a, rpb);
  else
    cache_write_kernel<float><<<row_grid(a, rpb), kThreads, 0, st>>>(a, rpb);
  return cudaGetLastError();
}

cudaError_t launch_read(const RowArgs& a, cudaStream_t st) {
  const int rpb = rows_per_block(a);
  if (a.dt == SA_BF16)
    cache_read_kernel<__nv_bfloat16><<<row_grid(a, rpb), kThreads, 0, st>>>(a, rpb);
  else
    cache_read_kernel<float><<<row_grid(a, rpb), kThreads, 0, st>>>(a, rpb);
  return cudaGetLastError();
}

}  // namespace cache
}  // namespace sa
