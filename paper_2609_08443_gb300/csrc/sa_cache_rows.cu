// Rows into the 4-bit cache and back (sa_cache_write, sa_cache_read).
//
// One thread handles one group of 16 features of one key or value row: writing, it
// takes the largest magnitude, picks the scale, rounds to levels and stores 8 code
// bytes and a scale byte; reading, it does the reverse.  Both are bound by memory
// (per feature 2 or 4 bytes of the row and 9/16 of the cache), so a thread has several
// groups' loads in flight and the arithmetic is kept to a few instructions a feature.
// A block takes up to 64 consecutive rows, looks up their pages once, and goes through
// them head by head with the groups of a row, then the rows, over its threads: what a
// warp touches is contiguous in the page and in runs of a row on the other side.
//
// Measured (GB300, bytes that have to move over time): ragged bf16 histories written and
// read back (2.0 GB) 339 us, fp32 sketches written and read back (1.2 GB) 238 us, 64 x 1024
// rows of 8 x 128 read as bf16 (0.34 GB) 66 us: 5.9, 5.1 and 5.2 TB/s of a measured copy's
// 6.8.  Two groups a thread in flight beat four (histories 343 against 358 us: 40 registers
// a thread instead of 77).
#include "sa_cache.cuh"
#include "sa_kernels.cuh"
#include "sa_ptx.cuh"
#include "sa_simt_util.cuh"

namespace sa {
namespace cache {

constexpr int kThreads = 256;
constexpr int kAtOnce = 2;  // groups in flight per thread

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

// Whether this thread's part of the users' offsets and starts is out of order or leads past
// the table: any such makes every block leave, and the whole call writes nothing.
__device__ __forceinline__ int offsets_bad(const RowArgs& a) {
  const int64_t most = int64_t(a.c.max_pages) << a.c.log2page;
  int bad = 0;
  if (a.cu || a.start) {
    for (int b = threadIdx.x; b < a.B; b += blockDim.x) {
      const int64_t c0 = a.cu ? int64_t(a.cu[b]) : b * a.per_user;
      const int64_t c1 = a.cu ? int64_t(a.cu[b + 1]) : c0 + a.per_user;
      const int64_t s = a.start ? a.start[b] : 0;
      bad |= (b == 0 && c0 != 0) || (b == a.B - 1 && c1 != a.N) || c0 > c1 || s < 0 || s + (c1 - c0) > most;
    }
  } else {
    bad = a.per_user > most;
  }
  return bad;
}

// Checks of what the host cannot see, by one more block: writes the call's status.
__device__ void check_rows(const RowArgs& a) {
  int status = __syncthreads_or(offsets_bad(a)) ? int(SA_ERR_BAD_SEQLENS) : 0;
  if (!status) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int bad = 0;
    for (int b = warp; b < a.B; b += blockDim.x >> 5) {
      const int64_t n = a.cu ? a.cu[b + 1] - a.cu[b] : a.per_user;
      if (n == 0) continue;
      const int64_t s = a.start ? a.start[b] : 0;
      const int p0 = int(s >> a.c.log2page), p1 = int((s + n - 1) >> a.c.log2page);
      for (int p = p0 + lane; p <= p1; p += 32) {
        const int e = a.c.table[int64_t(b) * a.c.max_pages + p];
        bad |= e < 0 || e >= a.c.n_pages;
      }
    }
    if (__syncthreads_or(bad)) status = int(SA_ERR_BAD_PAGE);
  }
  if (threadIdx.x == 0) ws_header(a.ws)->err = uint32_t(status);
}

// ------------------------------------------------------------------ a block's rows
constexpr int kLog2Rows = 6, kRows = 1 << kLog2Rows;

struct Rows {
  int64_t rec[kRows];  // byte offset of head 0's key record, or -1: nothing to do
  int64_t at[kRows];   // element offset of head 0 on the other side
  int slot[kRows];     // token within the page
};

// Rows [row0, row0 + n) of the call, looked up by the first threads.  The last block
// only checks; false: leave.
template <bool WRITE>
__device__ __forceinline__ bool find_rows(const RowArgs& a, int n, Rows& s) {
  if (blockIdx.x == gridDim.x - 1) {
    check_rows(a);
    return false;
  }
  const int bad = offsets_bad(a);
  if (threadIdx.x < n) {
    const int64_t row = int64_t(blockIdx.x) * n + threadIdx.x;
    int64_t rec = -1;
    if (row < a.N) {
      const RowRef r = find_row(a, row);
      if (r.ok) {
        const int p = a.c.table[int64_t(r.b) * a.c.max_pages + (r.pos >> a.c.log2page)];
        if (p >= 0 && p < a.c.n_pages) rec = a.c.record(p, 0);
        s.slot[threadIdx.x] = int(r.pos & (a.c.page - 1));
        if (!WRITE)
          s.at[threadIdx.x] = row * a.c.H * a.c.d;
        else if (a.cu)
          s.at[threadIdx.x] = row * a.row_stride;
        else
          s.at[threadIdx.x] = r.b * a.user_stride + r.i * a.row_stride;
      }
    }
    s.rec[threadIdx.x] = rec;
  }
  return !__syncthreads_or(bad);
}

// Group e of the block: its group of features, row, head and side (0 keys, 1 values).
// Groups run fastest, then rows (a power of two), then heads.
struct Groups {
  int ng, log2n, H;
  uint32_t inv;  // 2^32 / ng rounded up: e * inv >> 32 is e / ng exactly for e < 2^29
};
static Groups groups_of(const RowArgs& a, int log2n) {
  const int ng = a.c.d / kGroup;
  return {ng, log2n, a.c.H, ng > 1 ? 0xFFFFFFFFu / uint32_t(ng) + 1u : 0u};
}
struct GroupRef {
  int g, r, h, kv;
};
__device__ __forceinline__ GroupRef group_of(int e, const Groups& s) {
  GroupRef x;
  const int u = s.ng > 1 ? int(__umulhi(uint32_t(e), s.inv)) : e, hk = u >> s.log2n;
  x.g = e - u * s.ng;
  x.r = u - (hk << s.log2n);
  x.kv = hk >= s.H;
  x.h = x.kv ? hk - s.H : hk;
  return x;
}

// ------------------------------------------------------------------- quantising
// 16 features as they came.
template <typename T> struct Raw;
template <> struct Raw<__nv_bfloat16> {
  uint4 v[2];
  __device__ __forceinline__ void load(const __nv_bfloat16* p) {
    v[0] = __ldcs(reinterpret_cast<const uint4*>(p));
    v[1] = __ldcs(reinterpret_cast<const uint4*>(p) + 1);
  }
  __device__ __forceinline__ uint32_t word(int i) const {
    const uint4& q = v[i >> 2];
    return (i & 3) == 0 ? q.x : (i & 3) == 1 ? q.y : (i & 3) == 2 ? q.z : q.w;
  }
  // bits of the largest magnitude as fp32 (a NaN is larger than infinity)
  __device__ __forceinline__ uint32_t largest() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = __vmaxu2(m, word(i) & 0x7FFF7FFFu);
    return max(m & 0xFFFF0000u, m << 16);
  }
  __device__ __forceinline__ float get(int k) const {
    const uint32_t w = word(k >> 1);
    return __uint_as_float(k & 1 ? w & 0xFFFF0000u : w << 16);
  }
};
template <> struct Raw<float> {
  float4 v[4];
  __device__ __forceinline__ void load(const float* p) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __ldcs(reinterpret_cast<const float4*>(p) + i);
  }
  __device__ __forceinline__ float get(int k) const {
    const float4& q = v[k >> 2];
    return (k & 3) == 0 ? q.x : (k & 3) == 1 ? q.y : (k & 3) == 2 ? q.z : q.w;
  }
  __device__ __forceinline__ uint32_t largest() const {
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 16; ++k) m = max(m, __float_as_uint(get(k)) & 0x7FFFFFFFu);
    return m;
  }
};

// 1.5 x 2^23 + 8: adding it leaves level + 8 in the low bits of the sum
constexpr float kRound = 12582920.f;
constexpr uint32_t kRoundBits = 0x4B400000u;
__host__ __device__ constexpr int shift_of(int k) { return 4 * (((k & 7) >> 1) + 4 * (k & 1)); }
__host__ __device__ constexpr uint32_t round_bits_sum() {
  uint32_t s = 0;
  for (int k = 0; k < 8; ++k) s += kRoundBits << shift_of(k);
  return s;
}

// Levels of a group.  The quotient by a reciprocal made smaller by 2^-20 (the
// approximation and the product's rounding are under 2^-21) lies below the true one, so a
// half always rounds towards zero.  It can come out a level too low only for a quotient within
// 2^-19 above a half: impossible for bf16 (eight significant bits against the scale's
// four), and seen for fp32 from the remainder x - q s, which is exact there.
template <bool ODD, typename T>
__device__ __forceinline__ uint2 levels(const Raw<T>& x, uint32_t code) {
  const float s = scale_value(code), inv = ptx::rcp_approx(s) * (1.f - 0x1p-20f);
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int k = 0; k < kGroup; ++k) {
    float v = x.get(k);
    if constexpr (ODD) {  // NaN to zero, beyond the largest scale saturates
      if (isnan(v)) v = 0.f;
      v = fminf(fmaxf(v, -7.f * s), 7.f * s);
    }
    float u = fmaf(v, inv, kRound);
    if constexpr (sizeof(T) == 4) {
      const float r = fmaf(kRound - u, s, v);
      if (fabsf(r) > 0.5f * s) u += copysignf(1.f, v);
    }
    w[k >> 3] += __float_as_uint(u) << shift_of(k);
  }
  return make_uint2(w[0] - round_bits_sum(), w[1] - round_bits_sum());
}

template <typename T>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(const __grid_constant__ RowArgs a, const __grid_constant__ Groups geo) {
  __shared__ Rows rows;
  const int n = 1 << geo.log2n;
  if (!find_rows<true>(a, n, rows)) return;
  constexpr int U = kAtOnce;
  const int ng = geo.ng, count = ng * n * a.c.H * 2;
  const T* src[2] = {static_cast<const T*>(a.K), static_cast<const T*>(a.V)};
  uint8_t* pool = const_cast<uint8_t*>(a.c.pool);
  for (int e0 = threadIdx.x; e0 < count; e0 += U * kThreads) {
    Raw<T> x[U];
    GroupRef ref[U];
    bool on[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int e = e0 + i * kThreads;
      ref[i] = group_of(e, geo);
      on[i] = e < count && rows.rec[ref[i].r] >= 0;
      if (on[i]) x[i].load((ref[i].kv ? src[1] : src[0]) + rows.at[ref[i].r] + ref[i].h * a.head_stride + ref[i].g * kGroup);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (!on[i]) continue;
      uint32_t big = x[i].largest();
      if (big > 0x7F800000u) {  // a NaN: the largest of the others
        big = 0;
#pragma unroll
        for (int k = 0; k < kGroup; ++k) {
          const float v = x[i].get(k);
          if (!isnan(v)) big = max(big, __float_as_uint(v) & 0x7FFFFFFFu);
        }
        big |= 1u << 31;
      }
      const uint32_t code = scale_code(__uint_as_float(big & 0x7FFFFFFFu));
      const uint2 w = code == kCodeMax || (big >> 31) ? levels<true>(x[i], code) : levels<false>(x[i], code);
      const int64_t rec = rows.rec[ref[i].r] + int64_t(2 * ref[i].h + ref[i].kv) * a.c.rec;
      const int slot = rows.slot[ref[i].r];
      *reinterpret_cast<uint2*>(pool + rec + slot * (a.c.d / 2) + ref[i].g * 8) = w;
      pool[rec + a.c.page * (a.c.d / 2) + slot * ng + ref[i].g] = uint8_t(code);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(const __grid_constant__ RowArgs a, const __grid_constant__ Groups geo) {
  __shared__ Rows rows;
  const int n = 1 << geo.log2n;
  if (!find_rows<false>(a, n, rows)) return;
  constexpr int U = kAtOnce;
  const int ng = geo.ng, count = ng * n * a.c.H * 2;
  T* dst[2] = {static_cast<T*>(a.Ko), static_cast<T*>(a.Vo)};
  for (int e0 = threadIdx.x; e0 < count; e0 += U * kThreads) {
    uint2 w[U];
    uint32_t code[U];
    GroupRef ref[U];
    bool on[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int e = e0 + i * kThreads;
      ref[i] = group_of(e, geo);
      on[i] = e < count && rows.rec[ref[i].r] >= 0;
      if (!on[i]) continue;
      const uint8_t* rec = a.c.pool + rows.rec[ref[i].r] + int64_t(2 * ref[i].h + ref[i].kv) * a.c.rec;
      const int slot = rows.slot[ref[i].r];
      w[i] = __ldcs(reinterpret_cast<const uint2*>(rec + slot * (a.c.d / 2) + ref[i].g * 8));
      code[i] = __ldcs(rec + a.c.page * (a.c.d / 2) + slot * ng + ref[i].g);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (!on[i]) continue;
      uint32_t v[8];
      const ScaleB s = scale_bf16(code[i] * 0x00010001u);
      values_bf16(w[i].x, s, v);
      values_bf16(w[i].y, s, v + 4);
      T* p = (ref[i].kv ? dst[1] : dst[0]) + rows.at[ref[i].r] + ref[i].h * a.c.d + ref[i].g * kGroup;
      if constexpr (sizeof(T) == 2) {
        reinterpret_cast<uint4*>(p)[0] = make_uint4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<uint4*>(p)[1] = make_uint4(v[4], v[5], v[6], v[7]);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          reinterpret_cast<float4*>(p)[k] =
              make_float4(__uint_as_float(v[2 * k] << 16), __uint_as_float(v[2 * k] & 0xFFFF0000u),
                          __uint_as_float(v[2 * k + 1] << 16), __uint_as_float(v[2 * k + 1] & 0xFFFF0000u));
      }
    }
  }
}

// log2 of the rows a block takes: the most, up to 64, whose source (writing) or result
// (reading) is no more than `most` bytes and that leave every SM four blocks.  More rows
// spread the look-up of users and pages over more work; too many and the tail grows.
static int log2_rows(const RowArgs& a, int64_t most) {
  const int64_t bytes = int64_t(2) * a.c.H * a.c.d * (a.dt == SA_BF16 ? 2 : 4);  // a row's, keys and values
  int log2n = kLog2Rows;
  while (log2n > 0 && ((a.N >> log2n) < 608 || (bytes << log2n) > most)) --log2n;
  return log2n;
}

static cudaError_t launch_rows(void (*kernel)(RowArgs, Groups), const RowArgs& a, int64_t most, cudaStream_t st) {
  const int log2n = log2_rows(a, most), n = 1 << log2n;
  kernel<<<unsigned((a.N + n - 1) / n + 1), kThreads, 0, st>>>(a, groups_of(a, log2n));
  return cudaGetLastError();
}

// Measured on a GB300, written and read back: 64 users' up to 20,011 bf16 rows (8 heads of
// 64) and 128 users' 512 fp32 rows (8 heads of 128) take 347 and 247 us at 64 KiB a block,
// 343 and 237 at 128 KiB, 349 and 262 at 32 rows always.  Reading 64 users' 1024 rows (8 heads
// of 128) as bf16 takes 66 us at 64 KiB, 71 at 128 KiB.
constexpr int64_t kWriteBytes = 128 << 10, kReadBytes = 64 << 10;

cudaError_t launch_write(const RowArgs& a, cudaStream_t st) {
  return a.dt == SA_BF16 ? launch_rows(cache_write_kernel<__nv_bfloat16>, a, kWriteBytes, st)
                         : launch_rows(cache_write_kernel<float>, a, kWriteBytes, st);
}

cudaError_t launch_read(const RowArgs& a, cudaStream_t st) {
  return a.dt == SA_BF16 ? launch_rows(cache_read_kernel<__nv_bfloat16>, a, kReadBytes, st)
                         : launch_rows(cache_read_kernel<float>, a, kReadBytes, st);
}

}  // namespace cache
}  // namespace sa
