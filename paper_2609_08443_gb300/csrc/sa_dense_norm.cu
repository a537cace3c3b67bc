// Layer norm of x + r and its gradient (include/sa_dense.h).
//
//   y = (h - mean) rstd w + b,   dh = rstd (g - mean(g) - xh mean(g xh)),  g = dy w,
//   dw = sum_rows dy xh,  db = sum_rows dy
//
// Bound by memory: each element is read once and written once, the row stays in registers
// between the mean, the variance (of the differences from that mean, so a mean far from zero
// costs it no digits; the mean's own rounding, 2^-24 of it, stays in y) and the result.  T threads hold a row, C chunks of 8 elements each: 4 to 32
// lanes of a warp up to 512 features (1024), a block above.  A block walks rows with the parameters,
// and in the backward pass the columns' running sums, in registers (shared memory above 8192
// features, whose sums would not fit); its sums leave as one partial row, and a second kernel
// adds the partial rows in block order, so results do not depend on timing.
//
// A row's loads, sums and stores wait for one another, so the next two rows are on their way meanwhile, by cp.async
// into a ring in shared memory (8192 x 4096 in bf16, gradient: 134 us without, 46 with; 43 with the row's statistics
// asked for a row ahead too): each thread's own 16-byte pieces (nobody else reads them, so nothing but the
// thread's own copies is waited for), or, where rows are not 16-byte aligned, the 16-byte pieces that the row touches,
// from which the row's threads pick their elements.  524288 x 128, fp32 plus a bf16 residual: 81 us, 6.6 TB/s.
#include "sa_dense_act.cuh"
#include "sa_tc_common.cuh"

namespace sa {
namespace dense {

int sm_count() { return tcc::device_sm_count(); }

namespace {

constexpr int kThreads = 256;  // of a block that holds several rows at once
// Rows of a thread's ring: the one in work and two on their way (2 to 8 measured the same; the widest rows have room for 2).
template <int T>
constexpr int ring_rows() { return T >= 512 ? 2 : 3; }

template <int T>
constexpr int block_threads() { return T <= 32 ? kThreads : T; }
template <int T>
constexpr int rows_at_once() { return T <= 32 ? kThreads / T : 1; }

// Column of element j of this thread's chunk c: eight neighbours where rows are 16-byte aligned
// (VEC), else one of T neighbouring threads' elements, so that single-element accesses coalesce.
template <int T, bool VEC>
__device__ __forceinline__ int column(int t, int c, int j) {
  return VEC ? (c * T + t) * 8 + j : (c * 8 + j) * T + t;
}

template <int T, int C, bool VEC>
__device__ __forceinline__ void load_row(const void* p, sa_dtype dt, int64_t at, int t, int n, float* v) {
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (VEC) {
      const int k = column<T, true>(t, c, 0);
      if (k >= n) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[8 * c + j] = 0.f;
      } else if (dt == SA_BF16) {
        load8(static_cast<const __nv_bfloat16*>(p) + at + k, v + 8 * c);
      } else {
        load8(static_cast<const float*>(p) + at + k, v + 8 * c);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int k = column<T, false>(t, c, j);
        v[8 * c + j] = k >= n ? 0.f : dt == SA_BF16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[at + k])
                                                    : static_cast<const float*>(p)[at + k];
      }
    }
  }
}

// bytes of the 16-byte pieces that a row of n elements can touch
__host__ __device__ __forceinline__ uint32_t row_span(const Mat& m, int n) {
  return !m.p ? 0 : ((uint32_t(n) * (m.dt == SA_BF16 ? 2 : 4) + 15) / 16 + 1) * 16;
}

// 16-byte pieces that a chunk of 8 elements takes
__device__ __forceinline__ int pieces(const Mat& m) { return !m.p ? 0 : m.dt == SA_BF16 ? 1 : 2; }

// One matrix along a walk: where the next row to be fetched is (aligned rows: this thread's first element of it), and how
// far the row after it is away.
struct Track {
  const char* p;
  int64_t step;
  bool half;       // bf16
  uint32_t shift;  // of the row in work from its 16-byte boundary
  __device__ __forceinline__ Track(const Mat& m, int64_t row, int64_t rows, int first)
      : p(static_cast<const char*>(m.p)), half(m.dt == SA_BF16) {
    p += (row * m.stride + first) << (half ? 1 : 2);
    step = (rows * m.stride) << (half ? 1 : 2);
    shift = uint32_t(reinterpret_cast<uintptr_t>(p)) & 15;
  }
};

// The rows that a block walks, with the next ones on their way.  NEXT: false where the ring has no room.
template <int T, int C, bool VEC, bool NEXT, bool GRAD>
struct Walk {
  const int t, n;
  const uint32_t rows, step;
  uint32_t row, ahead;  // this thread's row, and the next that it fetches
  const bool sum;       // there is a second summand
  bool in[VEC ? C : 1];
  Track x, r, dy;
  const char* ring;
  uint32_t put, get;  // byte offsets of the rows to fetch and to take
  uint32_t per_row, off_r, off_dy;

  static constexpr uint32_t kApart = block_threads<T>() * 16;
  static constexpr int kRing = ring_rows<T>();

  __device__ Walk(const NormArgs& a, char* mem)
      : t(threadIdx.x % T), n(a.n), rows(uint32_t(a.rows)), step(gridDim.x * rows_at_once<T>()),
        row(blockIdx.x * rows_at_once<T>() + threadIdx.x / T), ahead(row), sum(a.r.p != nullptr),
        x(a.x, row, step, VEC ? t * 8 : 0), r(a.r, row, step, VEC ? t * 8 : 0), dy(a.dy, row, step, VEC ? t * 8 : 0) {
    put = get = 0;
    if (VEC) {
#pragma unroll
      for (int c = 0; c < C; ++c) in[c] = column<T, true>(t, c, 0) < n;
      ring = mem + threadIdx.x * 16;
      off_r = C * kApart * pieces(a.x);
      off_dy = off_r + C * kApart * pieces(a.r);
      per_row = off_dy + (GRAD ? C * kApart * pieces(a.dy) : 0);
    } else {
      off_r = row_span(a.x, n);
      off_dy = off_r + row_span(a.r, n);
      per_row = off_dy + (GRAD ? row_span(a.dy, n) : 0);
      ring = mem + (threadIdx.x / T) * (kRing * per_row);
    }
    if (NEXT) {
#pragma unroll
      for (int i = 0; i < kRing - 1; ++i) fetch();
    }
  }
  __device__ __forceinline__ void copy(const Track& m, uint32_t to) const {
    if (VEC) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        if (!in[VEC ? c : 0]) continue;
        if (m.half) {
          copy16(to + c * kApart, m.p + c * T * 16);
        } else {
          copy16_l1(to + 2 * c * kApart, m.p + c * T * 32);
          copy16_l1(to + (2 * c + 1) * kApart, m.p + c * T * 32 + 16);
        }
      }
    } else {
      // the pieces that hold a byte of the row (the ends of the first and the last may belong to other rows)
      const int shift = int(reinterpret_cast<uintptr_t>(m.p) & 15), bytes = shift + (n << (m.half ? 1 : 2));
      const char* from = m.p - shift;
      for (int at = t * 16; at < bytes; at += T * 16) copy16(to + at, from + at);
    }
  }
  // the next row's elements on their way
  __device__ __forceinline__ void fetch() {
    if (ahead < rows) {
      const uint32_t to = ptx::smem_u32(ring) + put;
      copy(x, to);
      if (sum) copy(r, to + off_r);
      if (GRAD) copy(dy, to + off_dy);
    }
    ahead += step;
    x.p += x.step;
    if (sum) r.p += r.step;
    if (GRAD) dy.p += dy.step;
    asm volatile("cp.async.commit_group;" ::: "memory");
    put = put == (kRing - 1) * per_row ? 0 : put + per_row;
  }
  // the block's rows are not all done (the same for all of its threads)
  __device__ __forceinline__ bool more() const { return row - threadIdx.x / T < rows; }
  __device__ __forceinline__ bool here() const { return T > 32 || row < rows; }

  template <bool ADD>
  __device__ __forceinline__ void unpack(bool half, const char* from, float* v) const {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float q[8];
      if (half) {
        load8(reinterpret_cast<const __nv_bfloat16*>(from + c * kApart), q);
      } else {
        const float4 a = *reinterpret_cast<const float4*>(from + 2 * c * kApart);
        const float4 b = *reinterpret_cast<const float4*>(from + (2 * c + 1) * kApart);
        q[0] = a.x, q[1] = a.y, q[2] = a.z, q[3] = a.w, q[4] = b.x, q[5] = b.y, q[6] = b.z, q[7] = b.w;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) v[8 * c + j] = ADD ? v[8 * c + j] + q[j] : q[j];
    }
  }
  // one element each T columns of an unaligned row
  template <bool ADD>
  __device__ __forceinline__ void pick(Track& m, const char* from, float* v) const {
    from += m.shift;
    m.shift = (m.shift + uint32_t(m.step)) & 15;
#pragma unroll
    for (int i = 0; i < 8 * C; ++i) {
      const int k = i * T + t;
      float q = 0.f;
      if (k < n)
        q = m.half ? __uint_as_float(uint32_t(reinterpret_cast<const uint16_t*>(from)[k]) << 16)
                   : reinterpret_cast<const float*>(from)[k];
      v[i] = ADD ? v[i] + q : q;
    }
  }
  // x + r (and dy) of this thread's row; zeros behind the row's end and, in dy, behind the last row
  __device__ __forceinline__ void take(const NormArgs& a, float* h, float* g) {
    if (NEXT && VEC) {
      fetch();
      asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
      const char* from = ring + get;
      unpack<false>(x.half, from, h);
      if (sum) unpack<true>(r.half, from + off_r, h);
      if (GRAD) unpack<false>(dy.half, from + off_dy, g);
      get = get == (kRing - 1) * per_row ? 0 : get + per_row;
      if (!in[C - 1] || !here()) {  // slots that nothing was copied to hold whatever was there
#pragma unroll
        for (int c = 0; c < C; ++c)
          if (!in[c] || !here())
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              h[8 * c + j] = 0.f;
              if (GRAD) g[8 * c + j] = 0.f;
            }
      }
    } else if (NEXT) {
      // the slot that is filled here was read before the last row's sums, which the row's threads made together
      fetch();
      asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
      if (T <= 32)
        __syncwarp();
      else
        __syncthreads();
      const char* from = ring + get;
      pick<false>(x, from, h);
      if (sum) pick<true>(r, from + off_r, h);
      if (GRAD) pick<false>(dy, from + off_dy, g);
      get = get == (kRing - 1) * per_row ? 0 : get + per_row;
      if (!here())  // the slots hold whatever was there
#pragma unroll
        for (int i = 0; i < 8 * C; ++i) {
          h[i] = 0.f;
          if (GRAD) g[i] = 0.f;
        }
    } else {
      const int end = here() ? n : 0;
      load_row<T, C, VEC>(a.x.p, a.x.dt, int64_t(row) * a.x.stride, t, end, h);
      if (GRAD) load_row<T, C, VEC>(a.dy.p, a.dy.dt, int64_t(row) * a.dy.stride, t, end, g);
      if (sum) {
        float v[8 * C];
        load_row<T, C, VEC>(a.r.p, a.r.dt, int64_t(row) * a.r.stride, t, end, v);
#pragma unroll
        for (int i = 0; i < 8 * C; ++i) h[i] += v[i];
      }
    }
  }
};

template <int T, int C, bool VEC>
__device__ __forceinline__ void store_row(void* p, sa_dtype dt, int64_t at, int t, int n, const float* v) {
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (VEC) {
      const int k = column<T, true>(t, c, 0);
      if (k >= n) continue;
      if (dt == SA_BF16)
        store8(static_cast<__nv_bfloat16*>(p) + at + k, v + 8 * c);
      else
        store8(static_cast<float*>(p) + at + k, v + 8 * c);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int k = column<T, false>(t, c, j);
        if (k >= n) continue;
        if (dt == SA_BF16)
          static_cast<__nv_bfloat16*>(p)[at + k] = __float2bfloat16_rn(v[8 * c + j]);
        else
          static_cast<float*>(p)[at + k] = v[8 * c + j];
      }
    }
  }
}

// The factors w, 1 where there are none.
template <int T, int C, bool VEC>
__device__ __forceinline__ void load_factors(const NormArgs& a, int t, int n, float* w) {
  if (a.w) {
    load_row<T, C, VEC>(a.w, a.w_dt, 0, t, n, w);
  } else {
#pragma unroll
    for (int i = 0; i < 8 * C; ++i) w[i] = 1.f;
  }
}

// Whether a thread holds its parameters from row to row: the widest rows leave it no registers for
// them, and read them again for each row, from L1 or L2.
template <int T, int C>
constexpr bool keep_parameters() { return T * C < 2048; }

// Two sums over the T threads of a row.  Within a warp by shuffles; over a block through `red`, whose
// two halves take turns, so one barrier a sum is enough.
template <int T>
__device__ __forceinline__ void row_sum(float (&v)[2], float* red, int& turn) {
  if constexpr (T <= 32) {
#pragma unroll
    for (int o = T / 2; o > 0; o >>= 1)
#pragma unroll
      for (int k = 0; k < 2; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
  } else {
    // the first exchange leaves each half of the warp with one of the two sums
    const bool high = threadIdx.x & 16;
    float x = (high ? v[1] : v[0]) + __shfl_xor_sync(0xFFFFFFFFu, high ? v[0] : v[1], 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    constexpr int W = T / 32;
    float* s = red + turn * W * 2;
    turn ^= 1;
    const int lane = threadIdx.x & 31;
    if ((lane & 15) == 0) s[(lane >> 4) * W + (threadIdx.x >> 5)] = x;
    __syncthreads();
    if constexpr (W <= 16) {  // likewise: the lower half of the warp adds one sum's parts, the upper the other's
      x = (lane & 15) < W ? s[(lane >> 4) * W + (lane & 15)] : 0.f;
#pragma unroll
      for (int o = W / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
      v[0] = __shfl_sync(0xFFFFFFFFu, x, 0);
      v[1] = __shfl_sync(0xFFFFFFFFu, x, 16);
    } else {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        v[k] = s[k * W + lane];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
      }
    }
  }
}

// Mean of a row's n elements and the sum of the squared differences from it, of the warps' own (sum, sum of
// squared differences from the warp's mean, elements): M = sum M_w + sum n_w (mean_w - mean)^2, one barrier in all.
template <int T>
__device__ __forceinline__ float2 row_moments(float sum, float m2, float count, float inv_n, float* red, int& turn) {
  constexpr int W = T / 32;
  float* s = red + turn * W * 3;
  turn ^= 1;
  const int lane = threadIdx.x & 31;
  if (lane == 0) {
    s[(threadIdx.x >> 5)] = sum;
    s[W + (threadIdx.x >> 5)] = m2;
    s[2 * W + (threadIdx.x >> 5)] = count;
  }
  __syncthreads();
  const float sw = lane < W ? s[lane] : 0.f, mw = lane < W ? s[W + lane] : 0.f, cw = lane < W ? s[2 * W + lane] : 0.f;
  float all = sw;
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) all += __shfl_xor_sync(0xFFFFFFFFu, all, o);
  if (W < 32) all = __shfl_sync(0xFFFFFFFFu, all, 0);
  const float mean = all * inv_n;
  const float d = cw > 0.f ? sw / cw - mean : 0.f;
  float m = fmaf(cw * d, d, mw);
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) m += __shfl_xor_sync(0xFFFFFFFFu, m, o);
  if (W < 32) m = __shfl_sync(0xFFFFFFFFu, m, 0);
  return make_float2(mean, m);
}

__device__ __forceinline__ float2 pair(const float* v, int i) { return make_float2(v[2 * i], v[2 * i + 1]); }
__device__ __forceinline__ void unpair(float* v, int i, float2 x) { v[2 * i] = x.x, v[2 * i + 1] = x.y; }
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// Blocks an SM that the register budget is made for: 64 to 128 a thread, by what it holds.
template <int T, int C, bool VEC, bool GRAD>
constexpr int blocks_at_once() {
  return T == 1024 ? 1 : 512 / block_threads<T>();
}

template <int T, int C, bool VEC, bool NEXT>
__global__ void __launch_bounds__(block_threads<T>(), blocks_at_once<T, C, VEC, false>()) norm_fwd_kernel(const NormArgs a) {
  extern __shared__ __align__(16) char ring[];
  __shared__ float red[T > 32 ? 6 * T / 32 : 1];
  constexpr int P = 4 * C;  // pairs of elements, whose arithmetic goes two at a time
  const int t = threadIdx.x % T, n = a.n;
  const float inv_n = 1.f / float(n);
  int turn = 0;
  float w[8 * C], b[8 * C];
  Walk<T, C, VEC, NEXT, false> at(a, ring);
  if (keep_parameters<T, C>()) {
    load_factors<T, C, VEC>(a, t, n, w);
    load_row<T, C, VEC>(a.b, a.w_dt, 0, t, a.b ? n : 0, b);
  }
  auto inside = [&](int i) { return VEC ? at.in[VEC ? i / 8 : 0] : column<T, false>(t, i / 8, i % 8) < n; };
  float count = 0.f;  // elements of this warp, in a row that is spread over several
  if (T > 32) {
#pragma unroll
    for (int i = 0; i < 8 * C; ++i) count += inside(i) ? 1.f : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) count += __shfl_xor_sync(0xFFFFFFFFu, count, o);
  }
  const float inv_count = T <= 32 ? inv_n : count > 0.f ? 1.f / count : 0.f;
  constexpr int lanes = T < 32 ? T : 32;
  for (; at.more(); at.row += at.step) {
    float h[8 * C];
    at.take(a, h, nullptr);
    float2 s2 = both(0.f);
#pragma unroll
    for (int i = 0; i < P; ++i) s2 = __fadd2_rn(s2, pair(h, i));
    float sum = s2.x + s2.y;
#pragma unroll
    for (int o = lanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    // squared differences from the mean of what the warp holds: the row's, or the warp's own
    float mean = sum * inv_count;
    float2 m2 = both(0.f);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const float2 d = __fadd2_rn(pair(h, i), both(-mean));
      if (T <= 32) unpair(h, i, d);
      if (VEC) {
        if (inside(2 * i)) m2 = __ffma2_rn(d, d, m2);
      } else {
        if (inside(2 * i)) m2.x = fmaf(d.x, d.x, m2.x);
        if (inside(2 * i + 1)) m2.y = fmaf(d.y, d.y, m2.y);
      }
    }
    float m = m2.x + m2.y;
#pragma unroll
    for (int o = lanes / 2; o > 0; o >>= 1) m += __shfl_xor_sync(0xFFFFFFFFu, m, o);
    if constexpr (T > 32) {
      const float2 all = row_moments<T>(sum, m, count, inv_n, red, turn);
      mean = all.x;
      m = all.y;
#pragma unroll
      for (int i = 0; i < P; ++i) unpair(h, i, __fadd2_rn(pair(h, i), both(-mean)));
    }
    const float rstd = rsqrtf(fmaf(m, inv_n, a.eps));  // off by 2^-22 at most, of which a correct root would save a step of y's fp32
    if (at.here()) {  // a warp's last rows may lie behind the end
      if (!keep_parameters<T, C>()) {
        load_factors<T, C, VEC>(a, t, n, w);
        load_row<T, C, VEC>(a.b, a.w_dt, 0, t, a.b ? n : 0, b);
      }
#pragma unroll
      for (int i = 0; i < P; ++i)
        unpair(h, i, __ffma2_rn(__fmul2_rn(pair(h, i), both(rstd)), pair(w, i), pair(b, i)));
      store_row<T, C, VEC>(a.y, a.y_dt, int64_t(at.row) * n, t, n, h);
      if (a.stats && t == 0) *reinterpret_cast<float2*>(a.stats + 2 * int64_t(at.row)) = make_float2(mean, rstd);
    }
  }
}

// Adds to the shared sums of pair i's columns ([2][n]; each thread has its own columns).
template <int T, int C, bool VEC>
__device__ __forceinline__ void add_to_sums(float* sums, int n, int t, int i, float2 w, float2 b) {
  const int k = column<T, VEC>(t, i / 4, 2 * i % 8);
  if (VEC) {
    if (k >= n) return;
    float2* p = reinterpret_cast<float2*>(sums + k);
    *p = __fadd2_rn(*p, w);
    p = reinterpret_cast<float2*>(sums + n + k);
    *p = __fadd2_rn(*p, b);
  } else {
    const int l = column<T, VEC>(t, i / 4, 2 * i % 8 + 1);
    if (k < n) sums[k] += w.x, sums[n + k] += b.x;
    if (l < n) sums[l] += w.y, sums[n + l] += b.y;
  }
}

// SUMS: where the columns' running sums are: 0 nowhere, 1 registers, 2 shared memory.
template <int T, int C, bool VEC, bool NEXT, int SUMS>
__global__ void __launch_bounds__(block_threads<T>(), blocks_at_once<T, C, VEC, true>()) norm_bwd_kernel(const NormArgs a) {
  // SUMS = 2: [2][n] sums; SUMS = 1 and T <= 32: at the end [warps][2][8 C T]; NEXT: the ring
  extern __shared__ __align__(16) float sums[];
  __shared__ float red[T > 32 ? 4 * T / 32 : 1];
  constexpr int P = 4 * C;
  const int t = threadIdx.x % T, n = a.n;
  const float inv_n = 1.f / float(n);
  int turn = 0;
  float w[8 * C];
  Walk<T, C, VEC, NEXT, true> at(a, reinterpret_cast<char*>(sums));
  if (keep_parameters<T, C>()) load_factors<T, C, VEC>(a, t, n, w);
  float sw[SUMS == 1 ? 8 * C : 1], sb[SUMS == 1 ? 8 * C : 1];
  if (SUMS == 1)
#pragma unroll
    for (int i = 0; i < 8 * C; ++i) sw[i] = sb[i] = 0.f;
  if (SUMS == 2)
#pragma unroll
    for (int i = 0; i < 8 * C; ++i) {  // each thread's own columns: no barrier needed
      const int k = column<T, VEC>(t, i / 8, i % 8);
      if (k < n) sums[k] = sums[n + k] = 0.f;
    }
  // a row's mean and 1 / sqrt(var), asked for a row ahead
  auto stats_of = [&](uint32_t row) {
    return row < at.rows ? __ldg(reinterpret_cast<const float2*>(a.stats) + row) : make_float2(0.f, 0.f);
  };
  float2 next = stats_of(at.row);
  for (; at.more(); at.row += at.step) {
    const bool here = at.here();
    float h[8 * C], g[8 * C], s[2] = {0.f, 0.f};
    const float2 st = next;
    next = stats_of(at.row + at.step);
    at.take(a, h, g);
    if (!keep_parameters<T, C>()) load_factors<T, C, VEC>(a, t, n, w);
    float2 g2 = both(0.f), x2 = both(0.f);
#pragma unroll
    for (int i = 0; i < P; ++i) {
      // xh; behind the row's end dy is 0, which keeps it out of all sums
      const float2 xh = __fmul2_rn(__fadd2_rn(pair(h, i), both(-st.x)), both(st.y)), d = pair(g, i);
      unpair(h, i, xh);
      if (SUMS == 1) {
        unpair(sw, SUMS == 1 ? i : 0, __ffma2_rn(d, xh, pair(sw, SUMS == 1 ? i : 0)));
        unpair(sb, SUMS == 1 ? i : 0, __fadd2_rn(pair(sb, SUMS == 1 ? i : 0), d));
      }
      const float2 gw = __fmul2_rn(d, pair(w, i));
      if (SUMS == 2) add_to_sums<T, C, VEC>(sums, n, t, i, __fmul2_rn(d, xh), d);
      unpair(g, i, gw);
      g2 = __fadd2_rn(g2, gw);
      x2 = __ffma2_rn(gw, xh, x2);
    }
    s[0] = g2.x + g2.y;
    s[1] = x2.x + x2.y;
    row_sum<T>(s, red, turn);
    if (here) {
      const float2 mg = both(-s[0] * inv_n * st.y), mx = both(-s[1] * inv_n * st.y), rs = both(st.y);
#pragma unroll
      for (int i = 0; i < P; ++i)
        unpair(g, i, __ffma2_rn(pair(g, i), rs, __ffma2_rn(pair(h, i), mx, mg)));
      if (a.dx) store_row<T, C, VEC>(a.dx, a.x.dt, int64_t(at.row) * n, t, n, g);
      if (a.dr) store_row<T, C, VEC>(a.dr, a.r.dt, int64_t(at.row) * n, t, n, g);
    }
  }
  if (SUMS == 0) return;
  float* out = a.partial + int64_t(blockIdx.x) * 2 * n;
  if constexpr (SUMS == 2) {
#pragma unroll
    for (int i = 0; i < 8 * C; ++i) {
      const int k = column<T, VEC>(t, i / 8, i % 8);
      if (k < n) {
        out[k] = sums[k];
        out[n + k] = sums[n + k];
      }
    }
  } else if constexpr (T > 32 && VEC) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int k = column<T, true>(t, c, 0);
      if (k >= n) continue;
      store8(out + k, sw + 8 * c);
      store8(out + n + k, sb + 8 * c);
    }
  } else if constexpr (T > 32) {
#pragma unroll
    for (int i = 0; i < 8 * C; ++i) {
      const int k = column<T, VEC>(t, i / 8, i % 8);
      if (k < n) {
        out[k] = sw[i];
        out[n + k] = sb[i];
      }
    }
  } else {
    // the warp's rows, then the warps in order
#pragma unroll
    for (int o = T; o < 32; o <<= 1)
#pragma unroll
      for (int i = 0; i < 8 * C; ++i) {
        sw[i] += __shfl_xor_sync(0xFFFFFFFFu, sw[i], o);
        sb[i] += __shfl_xor_sync(0xFFFFFFFFu, sb[i], o);
      }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __syncthreads();  // the ring is read out (no copy is in flight: the last rows' were waited for)
    if (lane < T)
#pragma unroll
      for (int i = 0; i < 8 * C; ++i) {
        const int k = column<T, VEC>(t, i / 8, i % 8);
        sums[(warp * 2) * 8 * C * T + k] = sw[i];
        sums[(warp * 2 + 1) * 8 * C * T + k] = sb[i];
      }
    __syncthreads();
    for (int e = threadIdx.x; e < 2 * n; e += kThreads) {
      const int which = e >= n, k = e - which * n;
      float s = 0.f;
#pragma unroll
      for (int v = 0; v < kThreads / 32; ++v) s += sums[(v * 2 + which) * 8 * C * T + k];
      out[e] = s;
    }
  }
}

// Column sums of one or two sets of partial rows (the first takes `blocks0` blocks).
__global__ void __launch_bounds__(1024)
    join_columns_kernel(const float* __restrict__ p0, int G, int64_t pitch, int64_t n0, void* d0,
                        const float* __restrict__ p1, int64_t n1, void* d1, unsigned blocks0, sa_dtype dt) {
  // 32 columns a block, 32 threads a column that take every 32nd partial row, then their sums in order
  __shared__ float part[32][33];
  const int lane = threadIdx.x & 31, part_id = threadIdx.x >> 5;
  const bool second = blockIdx.x >= blocks0;
  const float* partial = second ? p1 : p0;
  const int64_t n = second ? n1 : n0, c = int64_t(blockIdx.x - (second ? blocks0 : 0)) * 32 + lane;
  float s = 0.f;
  if (c < n) {
    int g = part_id;
    for (; g + 96 < G; g += 128) {  // four rows in flight
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = partial[int64_t(g + 32 * i) * pitch + c];
#pragma unroll
      for (int i = 0; i < 4; ++i) s += v[i];
    }
    for (; g < G; g += 32) s += partial[int64_t(g) * pitch + c];
  }
  part[part_id][lane] = s;
  __syncthreads();
  if (part_id == 0 && c < n) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) sum += part[i][lane];
    void* dst = second ? d1 : d0;
    if (dt == SA_BF16)
      static_cast<__nv_bfloat16*>(dst)[c] = __float2bfloat16_rn(sum);
    else
      static_cast<float*>(dst)[c] = sum;
  }
}

bool aligned_rows(const Mat& m) {
  if (!m.p) return true;
  const int e = m.dt == SA_BF16 ? 8 : 4;
  return reinterpret_cast<uintptr_t>(m.p) % 16 == 0 && m.stride % e == 0;
}
bool aligned_base(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

bool vec_ok(const NormArgs& a) {
  return a.n % 8 == 0 && aligned_rows(a.x) && aligned_rows(a.r) && aligned_rows(a.dy) && aligned_base(a.w) &&
         aligned_base(a.b) && aligned_base(a.y) && aligned_base(a.dx) && aligned_base(a.dr);
}

// Calls f with the layout for n features: (threads a row, chunks of 8 a thread).  More chunks spread what a thread spends
// on a row's sums over more elements: two (8192 x 4096 in bf16, forward and gradient 30 and 43 us; one chunk 37 and 58),
// four in the forward of wide rows that are read in bf16 alone (26 us; but 62 with fp32 rows and a residual, for 43
// with two).  Unaligned rows: two (10007 x 1001 in bf16 18 us, one 20, four 22), above 4096 features four (8000 x 8191:
// 88 us, two 98).
template <bool GRAD, class F>
auto with_layout(int n, bool vec, bool narrow, F f) {
  using std::integral_constant;
#define SA_LAYOUT(T, C, V) f(integral_constant<int, T>{}, integral_constant<int, C>{}, integral_constant<bool, V>{})
  if constexpr (!GRAD) {
    if (vec && narrow && n > 512) {
      if (n <= 1024) return SA_LAYOUT(32, 4, true);
      if (n <= 2048) return SA_LAYOUT(64, 4, true);
      if (n <= 4096) return SA_LAYOUT(128, 4, true);
      if (n <= 8192) return SA_LAYOUT(256, 4, true);
      return SA_LAYOUT(512, 4, true);
    }
    if (!vec && n > 4096 && n <= 8192) return SA_LAYOUT(256, 4, false);
  }
  if (vec) {
    if (n <= 64) return SA_LAYOUT(4, 2, true);
    if (n <= 128) return SA_LAYOUT(8, 2, true);
    if (n <= 256) return SA_LAYOUT(16, 2, true);
    if (n <= 512) return SA_LAYOUT(32, 2, true);
    if (n <= 1024) return SA_LAYOUT(64, 2, true);
    if (n <= 2048) return SA_LAYOUT(128, 2, true);
    if (n <= 4096) return SA_LAYOUT(256, 2, true);
    if (n <= 8192) return SA_LAYOUT(512, 2, true);
    return SA_LAYOUT(1024, 2, true);
  }
  if (n <= 64) return SA_LAYOUT(4, 2, false);
  if (n <= 128) return SA_LAYOUT(8, 2, false);
  if (n <= 256) return SA_LAYOUT(16, 2, false);
  if (n <= 512) return SA_LAYOUT(32, 2, false);
  if (n <= 1024) return SA_LAYOUT(64, 2, false);
  if (n <= 2048) return SA_LAYOUT(128, 2, false);
  if (n <= 4096) return SA_LAYOUT(256, 2, false);
  if (n <= 8192) return SA_LAYOUT(512, 2, false);
  return SA_LAYOUT(1024, 2, false);
#undef SA_LAYOUT
}

template <int T>
int64_t blocks_for(int64_t rows) { return (rows + rows_at_once<T>() - 1) / rows_at_once<T>(); }

// A walk's grid and the bytes of a block's ring: the blocks that are resident together, fewer where their rings need the
// room (an SM has 227 KB, of which a little is left to the sums' exchange).
constexpr size_t kRoom = 220 * 1024;
struct Walkers {
  int blocks;
  size_t ring;
};
template <int T, int C, bool VEC, bool NEXT, bool GRAD>
Walkers walkers(const NormArgs& a) {
  Walkers w{blocks_at_once<T, C, VEC, GRAD>(), 0};
  if (NEXT) {
    auto pieces_of = [](const Mat& m) { return !m.p ? 0 : m.dt == SA_BF16 ? 1 : 2; };
    const size_t row = VEC ? size_t(C) * (pieces_of(a.x) + pieces_of(a.r) + (GRAD ? pieces_of(a.dy) : 0)) * block_threads<T>() * 16
                           : size_t(row_span(a.x, a.n) + row_span(a.r, a.n) + (GRAD ? row_span(a.dy, a.n) : 0)) * rows_at_once<T>();
    w.ring = ring_rows<T>() * row;
    const int fit = int(kRoom / (w.ring + 2048));
    if (w.blocks > fit) w.blocks = fit;
  }
  const int64_t most = int64_t(sm_count()) * w.blocks, need = blocks_for<T>(a.rows);
  w.blocks = int(need < most ? need : most);
  return w;
}

template <auto Kernel>
cudaError_t launch_walk(const Walkers& w, int threads, size_t smem, const NormArgs& a, cudaStream_t st) {
  if (smem > 40 * 1024) {  // with the sums' exchange above what a launch may take unasked
    const cudaError_t e = allow_smem<Kernel>(kRoom);
    if (e != cudaSuccess) return e;
  }
  Kernel<<<w.blocks, threads, smem, st>>>(a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_norm_fwd(const NormArgs& a, cudaStream_t st) {
  const bool narrow = a.x.dt == SA_BF16 && (!a.r.p || a.r.dt == SA_BF16);
  return with_layout<false>(a.n, vec_ok(a), narrow, [&](auto T, auto C, auto V) {
    constexpr bool NEXT = T() < 1024 || V();
    const Walkers w = walkers<T(), C(), V(), NEXT, false>(a);
    if constexpr (T() == 1024 && NEXT) {
      if (w.blocks == 0) {  // no room for two rows of fp32
        const Walkers plain = walkers<T(), C(), V(), false, false>(a);
        return launch_walk<norm_fwd_kernel<T(), C(), V(), false>>(plain, block_threads<T()>(), 0, a, st);
      }
    }
    return launch_walk<norm_fwd_kernel<T(), C(), V(), NEXT>>(w, block_threads<T()>(), w.ring, a, st);
  });
}

int norm_bwd_blocks(int64_t rows, int n) {
  int most = 0;
  for (const bool vec : {false, true}) {
    const int g = with_layout<true>(n, vec, false, [&](auto T, auto C, auto V) {
      const int64_t all = int64_t(sm_count()) * blocks_at_once<T(), C(), V(), true>(), need = blocks_for<T()>(rows);
      return int(need < all ? need : all);
    });
    most = g > most ? g : most;
  }
  return most;
}

cudaError_t launch_norm_bwd(const NormArgs& a, cudaStream_t st, int* launches) {
  int G = 0;
  cudaError_t e = cudaSuccess;
  if (a.rows > 0)
    e = with_layout<true>(a.n, vec_ok(a), false, [&](auto T, auto C, auto V) {
      constexpr bool NEXT = T() < 1024;
      constexpr int threads = block_threads<T()>();
      const Walkers w = walkers<T(), C(), V(), NEXT, true>(a);
      G = w.blocks;
      ++*launches;
      if (!a.partial) return launch_walk<norm_bwd_kernel<T(), C(), V(), NEXT, 0>>(w, threads, w.ring, a, st);
      constexpr int SUMS = T() == 1024 ? 2 : 1;
      const size_t sums = SUMS == 2 ? size_t(2) * a.n * 4 : T() <= 32 ? size_t(kThreads / 32) * 2 * 8 * C() * T() * 4 : 0;
      return launch_walk<norm_bwd_kernel<T(), C(), V(), NEXT, SUMS>>(w, threads, sums > w.ring ? sums : w.ring, a, st);
    });
  if (e != cudaSuccess) return e;
  if (a.dw || a.db) {
    e = launch_join_columns2(a.partial, G, 2 * int64_t(a.n), a.n, a.dw, a.partial + a.n, a.n, a.db, a.w_dt, st);
    ++*launches;
  }
  return e;
}

cudaError_t launch_join_columns2(const float* p0, int G, int64_t pitch, int64_t n0, void* d0, const float* p1, int64_t n1,
                                 void* d1, sa_dtype dt, cudaStream_t st) {
  if (!d0) n0 = 0;
  if (!d1) n1 = 0;
  const unsigned b0 = unsigned((n0 + 31) / 32), b1 = unsigned((n1 + 31) / 32);
  if (b0 + b1 == 0) return cudaSuccess;
  join_columns_kernel<<<b0 + b1, 1024, 0, st>>>(p0, G, pitch, n0, d0, p1, n1, d1, b0, dt);
  return cudaGetLastError();
}

cudaError_t launch_join_columns(const float* partial, int G, int64_t pitch, int64_t n, void* dst, sa_dtype dt,
                                cudaStream_t st) {
  return launch_join_columns2(partial, G, pitch, n, dst, nullptr, 0, nullptr, dt, st);
}

}  // namespace dense
}  // namespace sa
