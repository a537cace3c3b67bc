// Layer norm of x + r and its gradient (include/sa_dense.h).
//
//   y = (h - mean) rstd w + b,   dh = rstd (g - mean(g) - xh mean(g xh)),  g = dy w,
//   dw = sum_rows dy xh,  db = sum_rows dy
//
// Bound by memory: each element is read once and written once, the row stays in registers
// between the mean, the variance (of the differences from that mean, so a mean far from zero
// costs no digits) and the result.  T threads hold a row, C chunks of 8 elements each: 8 to 32
// lanes of a warp up to 512 features, a block above.  A block walks rows with the parameters,
// and in the backward pass the columns' running sums, in registers (shared memory above 4096
// features, whose sums would not fit); its sums leave as one partial row, and a second kernel
// adds the partial rows in block order, so results do not depend on timing.
#include "sa_dense.cuh"
#include "sa_tc_common.cuh"

namespace sa {
namespace dense {

int sm_count() { return tcc::device_sm_count(); }

namespace {

constexpr int kThreads = 256;  // of a block that holds several rows at once

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
  if (dt == SA_BF16) {
    const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(p) + at;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (VEC) {
        uint4 u = make_uint4(0, 0, 0, 0);
        if (column<T, true>(t, c, 0) < n) u = *reinterpret_cast<const uint4*>(q + column<T, true>(t, c, 0));
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[8 * c + 2 * j] = __uint_as_float(w[j] << 16);
          v[8 * c + 2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int k = column<T, false>(t, c, j);
          v[8 * c + j] = k < n ? __bfloat162float(q[k]) : 0.f;
        }
      }
    }
  } else {
    const float* q = static_cast<const float*>(p) + at;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (VEC) {
        float4 a = make_float4(0, 0, 0, 0), b = a;
        if (column<T, true>(t, c, 0) < n) {
          const float4* s = reinterpret_cast<const float4*>(q + column<T, true>(t, c, 0));
          a = s[0];
          b = s[1];
        }
        const float w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) v[8 * c + j] = w[j];
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int k = column<T, false>(t, c, j);
          v[8 * c + j] = k < n ? q[k] : 0.f;
        }
      }
    }
  }
}

template <int T, int C, bool VEC>
__device__ __forceinline__ void store_row(void* p, sa_dtype dt, int64_t at, int t, int n, const float* v) {
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (VEC) {
      const int k = column<T, true>(t, c, 0);
      if (k >= n) continue;
      if (dt == SA_BF16) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = ptx::pack_bf16(v[8 * c + 2 * j], v[8 * c + 2 * j + 1]);
        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p) + at + k) = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
        float4* s = reinterpret_cast<float4*>(static_cast<float*>(p) + at + k);
        s[0] = make_float4(v[8 * c], v[8 * c + 1], v[8 * c + 2], v[8 * c + 3]);
        s[1] = make_float4(v[8 * c + 4], v[8 * c + 5], v[8 * c + 6], v[8 * c + 7]);
      }
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

// Sums over the T threads of a row.  Within a warp by shuffles; over a block through `red`, whose
// two halves take turns, so one barrier a sum is enough.
template <int T, int K>
__device__ __forceinline__ void row_sum(float (&v)[K], float* red, int& turn) {
  constexpr int lanes = T < 32 ? T : 32;
#pragma unroll
  for (int o = lanes / 2; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
  if constexpr (T > 32) {
    constexpr int W = T / 32;
    float* s = red + turn * W * K;
    turn ^= 1;
    const int lane = threadIdx.x & 31;
    if (lane == 0)
#pragma unroll
      for (int k = 0; k < K; ++k) s[(threadIdx.x >> 5) * K + k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      v[k] = lane < W ? s[lane * K + k] : 0.f;
#pragma unroll
      for (int o = W / 2; o > 0; o >>= 1) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
      if (W < 32) v[k] = __shfl_sync(0xFFFFFFFFu, v[k], 0);
    }
  }
}

template <int T, int C, bool VEC>
__global__ void __launch_bounds__(block_threads<T>()) norm_fwd_kernel(const NormArgs a) {
  __shared__ float red[T > 32 ? 2 * T / 32 : 1];
  const int t = threadIdx.x % T, n = a.n;
  const float inv_n = 1.f / float(n);
  int turn = 0;
  float w[8 * C], b[8 * C];
  if (keep_parameters<T, C>()) {
    load_factors<T, C, VEC>(a, t, n, w);
    load_row<T, C, VEC>(a.b, a.w_dt, 0, t, a.b ? n : 0, b);
  }
  const int64_t step = int64_t(gridDim.x) * rows_at_once<T>();
  for (int64_t base = int64_t(blockIdx.x) * rows_at_once<T>(); base < a.rows; base += step) {
    const int64_t row = base + threadIdx.x / T;
    const int here = row < a.rows ? n : 0;  // a warp's last rows may lie behind the end
    float h[8 * C], s[1] = {0.f};
    load_row<T, C, VEC>(a.x.p, a.x.dt, row * a.x.stride, t, here, h);
    if (a.r.p) {
      float r[8 * C];
      load_row<T, C, VEC>(a.r.p, a.r.dt, row * a.r.stride, t, here, r);
#pragma unroll
      for (int i = 0; i < 8 * C; ++i) h[i] += r[i];
    }
#pragma unroll
    for (int i = 0; i < 8 * C; ++i) s[0] += h[i];
    row_sum<T>(s, red, turn);
    const float mean = s[0] * inv_n;
    s[0] = 0.f;
#pragma unroll
    for (int i = 0; i < 8 * C; ++i) {
      h[i] -= mean;
      if (column<T, VEC>(t, i / 8, i % 8) < n) s[0] = fmaf(h[i], h[i], s[0]);
    }
    row_sum<T>(s, red, turn);
    const float rstd = rsqrtf(fmaf(s[0], inv_n, a.eps));
    if (here) {
      if (!keep_parameters<T, C>()) {
        load_factors<T, C, VEC>(a, t, n, w);
        load_row<T, C, VEC>(a.b, a.w_dt, 0, t, a.b ? n : 0, b);
      }
#pragma unroll
      for (int i = 0; i < 8 * C; ++i) h[i] = fmaf(h[i] * rstd, w[i], b[i]);
      store_row<T, C, VEC>(a.y, a.y_dt, row * n, t, n, h);
      if (a.stats && t == 0) *reinterpret_cast<float2*>(a.stats + 2 * row) = make_float2(mean, rstd);
    }
  }
}

// SUMS: where the columns' running sums are: 0 nowhere, 1 registers, 2 shared memory.
template <int T, int C, bool VEC, int SUMS>
__global__ void __launch_bounds__(block_threads<T>()) norm_bwd_kernel(const NormArgs a) {
  extern __shared__ float sums[];  // SUMS = 2: [2][n]; SUMS = 1 and T <= 32: [warps][2][8 C lanes]
  __shared__ float red[T > 32 ? 4 * T / 32 : 1];
  const int t = threadIdx.x % T, n = a.n;
  const float inv_n = 1.f / float(n);
  int turn = 0;
  float w[8 * C];
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
  const int64_t step = int64_t(gridDim.x) * rows_at_once<T>();
  for (int64_t base = int64_t(blockIdx.x) * rows_at_once<T>(); base < a.rows; base += step) {
    const int64_t row = base + threadIdx.x / T;
    const int here = row < a.rows ? n : 0;
    float h[8 * C], g[8 * C], s[2] = {0.f, 0.f};
    load_row<T, C, VEC>(a.dy.p, a.dy.dt, row * a.dy.stride, t, here, g);
    load_row<T, C, VEC>(a.x.p, a.x.dt, row * a.x.stride, t, here, h);
    if (a.r.p) {
      float r[8 * C];
      load_row<T, C, VEC>(a.r.p, a.r.dt, row * a.r.stride, t, here, r);
#pragma unroll
      for (int i = 0; i < 8 * C; ++i) h[i] += r[i];
    }
    if (!keep_parameters<T, C>()) load_factors<T, C, VEC>(a, t, n, w);
    const float2 st = here ? *reinterpret_cast<const float2*>(a.stats + 2 * row) : make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < 8 * C; ++i) {
      h[i] = (h[i] - st.x) * st.y;  // xh; behind the row's end g is 0, which keeps it out of both sums
      const int k = column<T, VEC>(t, i / 8, i % 8);
      if (k >= here) h[i] = 0.f;
      if (SUMS == 1) {
        sw[i] = fmaf(g[i], h[i], sw[i]);
        sb[i] += g[i];
      } else if (SUMS == 2) {
        if (k < n) {
          sums[k] = fmaf(g[i], h[i], sums[k]);
          sums[n + k] += g[i];
        }
      }
      g[i] *= w[i];
      s[0] += g[i];
      s[1] = fmaf(g[i], h[i], s[1]);
    }
    row_sum<T>(s, red, turn);
    if (here) {
      const float mg = s[0] * inv_n, mx = s[1] * inv_n;
#pragma unroll
      for (int i = 0; i < 8 * C; ++i) g[i] = st.y * (g[i] - fmaf(h[i], mx, mg));
      if (a.dx) store_row<T, C, VEC>(a.dx, a.x.dt, row * n, t, n, g);
      if (a.dr) store_row<T, C, VEC>(a.dr, a.r.dt, row * n, t, n, g);
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

__global__ void __launch_bounds__(1024) join_columns_kernel(const float* __restrict__ partial, int G, int64_t pitch,
                                                            int64_t n, void* dst, sa_dtype dt) {
  // 32 columns a block, 32 threads a column that take every 32nd partial row, then their sums in order
  __shared__ float part[32][33];
  const int lane = threadIdx.x & 31, part_id = threadIdx.x >> 5;
  const int64_t c = int64_t(blockIdx.x) * 32 + lane;
  float s = 0.f;
  if (c < n)
    for (int g = part_id; g < G; g += 32) s += partial[int64_t(g) * pitch + c];
  part[part_id][lane] = s;
  __syncthreads();
  if (part_id == 0 && c < n) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) sum += part[i][lane];
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

// Calls f with the layout for n features: (threads a row, chunks of 8 a thread, where the sums are).
template <class F>
auto with_layout(int n, F f) {
  using std::integral_constant;
#define SA_LAYOUT(T, C, S) f(integral_constant<int, T>{}, integral_constant<int, C>{}, integral_constant<int, S>{})
  if (n <= 64) return SA_LAYOUT(8, 1, 1);
  if (n <= 128) return SA_LAYOUT(16, 1, 1);
  if (n <= 256) return SA_LAYOUT(32, 1, 1);
  if (n <= 512) return SA_LAYOUT(32, 2, 1);
  if (n <= 1024) return SA_LAYOUT(128, 1, 1);
  if (n <= 2048) return SA_LAYOUT(256, 1, 1);
  if (n <= 4096) return SA_LAYOUT(512, 1, 1);
  if (n <= 8192) return SA_LAYOUT(1024, 1, 2);
  return SA_LAYOUT(1024, 2, 2);
#undef SA_LAYOUT
}

template <int T>
int64_t blocks_for(int64_t rows) { return (rows + rows_at_once<T>() - 1) / rows_at_once<T>(); }

}  // namespace

cudaError_t launch_norm_fwd(const NormArgs& a, cudaStream_t st) {
  const bool vec = vec_ok(a);
  return with_layout(a.n, [&](auto T, auto C, auto) {
    constexpr int threads = block_threads<T()>();
    const int64_t most = int64_t(sm_count()) * (2048 / threads);
    const int64_t need = blocks_for<T()>(a.rows);
    const unsigned grid = unsigned(need < most ? need : most);
    if (vec)
      norm_fwd_kernel<T(), C(), true><<<grid, threads, 0, st>>>(a);
    else
      norm_fwd_kernel<T(), C(), false><<<grid, threads, 0, st>>>(a);
    return cudaGetLastError();
  });
}

int norm_bwd_blocks(int64_t rows, int n) {
  return with_layout(n, [&](auto T, auto, auto) {
    const int64_t most = int64_t(sm_count()) * (1024 / block_threads<T()>());
    const int64_t need = blocks_for<T()>(rows);
    return int(need < most ? need : most);
  });
}

cudaError_t launch_norm_bwd(const NormArgs& a, cudaStream_t st, int* launches) {
  const bool vec = vec_ok(a);
  const int G = norm_bwd_blocks(a.rows, a.n);
  cudaError_t e = cudaSuccess;
  if (G > 0)
    e = with_layout(a.n, [&](auto T, auto C, auto S) {
      auto go = [&](auto kernel, size_t smem) {
        if (smem > 48 * 1024) {
          const cudaError_t s = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem));
          if (s != cudaSuccess) return s;
        }
        kernel<<<G, block_threads<T()>(), smem, st>>>(a);
        ++*launches;
        return cudaGetLastError();
      };
      if (!a.partial) return vec ? go(norm_bwd_kernel<T(), C(), true, 0>, 0) : go(norm_bwd_kernel<T(), C(), false, 0>, 0);
      const size_t smem = S() == 2 ? size_t(2) * a.n * 4 : T() <= 32 ? size_t(kThreads / 32) * 2 * 8 * C() * T() * 4 : 0;
      return vec ? go(norm_bwd_kernel<T(), C(), true, S()>, smem) : go(norm_bwd_kernel<T(), C(), false, S()>, smem);
    });
  if (e != cudaSuccess) return e;
  if (a.dw) {
    e = launch_join_columns(a.partial, G, 2 * int64_t(a.n), a.n, a.dw, a.w_dt, st);
    ++*launches;
  }
  if (e == cudaSuccess && a.db) {
    e = launch_join_columns(a.partial + a.n, G, 2 * int64_t(a.n), a.n, a.db, a.w_dt, st);
    ++*launches;
  }
  return e;
}

cudaError_t launch_join_columns(const float* partial, int G, int64_t pitch, int64_t n, void* dst, sa_dtype dt,
                                cudaStream_t st) {
  join_columns_kernel<<<unsigned((n + 31) / 32), 1024, 0, st>>>(partial, G, pitch, n, dst, dt);
  return cudaGetLastError();
}

}  // namespace dense
}  // namespace sa
