// Linear layers for at most 16 rows of x (single tokens, a small request): y = act(x W^T + b) + r.
//
// Bound by reading W once, so W goes from memory straight into registers: a block makes a few columns of y for
// all rows of x, its eight warps each take an eighth of k (64 or 128 elements in turn), and their sums meet in
// shared memory, in order.
//   bf16: 16 rows of W against 8 or 16 rows of x with warp-level products (m16n8k16).  Which k an element of a fragment
//         stands for does not matter as long as both operands agree, so a thread takes 8 neighbours of a row
//         of W and the same 8 of a row of x, and uses them in two products.
//   fp32: 4 (2) rows of W against 8 (16) rows of x with multiply-adds.
// 1 x 4096 -> 8192 gated in bf16: 23 us (5.9 TB/s), 16 rows 26 us (x comes from L1 and L2 as well as W from memory); 1 x 1024
// -> 4096: 2.9 us, a launch.
//
// Their gradients, where the tensor cores would want a copy of W first (fp32, whose terms are three times its reading, and
// up to four rows where TMA cannot read W):
//   dx = dz W    bound by reading W once: a thread holds a few columns of dx for all rows and walks down its block's share of
//                W's rows; the shares' sums are added in order by a second kernel.
//   dW = dz^T x  bound by writing dW: a thread holds a few columns of x and walks down rows of dW.
// Both for 4 x 5954 -> 5312 in fp32: 87 us of a floor of 38 (copies for the tensor cores: 212).
#include "sa_dense_act.cuh"

namespace sa {
namespace dense {
namespace {

constexpr int kWarps = 8;
constexpr int kRowsRun = 65536;  // features of a run: 512 additions a warp

// 16 bytes of W, which nobody reads again soon
__device__ __forceinline__ uint4 stream16(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

// Eight bf16 from k on (zeros behind K)
template <bool VEC, bool ONCE>
__device__ __forceinline__ uint4 take8(const __nv_bfloat16* row, int k, int K) {
  if (VEC) {
    if (k >= K) return make_uint4(0, 0, 0, 0);
    return ONCE ? stream16(row + k) : __ldg(reinterpret_cast<const uint4*>(row + k));
  }
  const unsigned short* p = reinterpret_cast<const unsigned short*>(row) + k;
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t lo = k + 2 * j < K ? __ldg(p + 2 * j) : 0, hi = k + 2 * j + 1 < K ? __ldg(p + 2 * j + 1) : 0;
    w[j] = lo | hi << 16;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

template <bool VEC, bool ONCE>
__device__ __forceinline__ float4 take4(const float* row, int k, int K) {
  if (VEC) {
    if (k >= K) return make_float4(0, 0, 0, 0);
    if (!ONCE) return __ldg(reinterpret_cast<const float4*>(row + k));
    const uint4 u = stream16(row + k);
    return make_float4(__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w));
  }
  float4 v;
  v.x = k < K ? __ldg(row + k) : 0.f;
  v.y = k + 1 < K ? __ldg(row + k + 1) : 0.f;
  v.z = k + 2 < K ? __ldg(row + k + 2) : 0.f;
  v.w = k + 3 < K ? __ldg(row + k + 3) : 0.f;
  return v;
}

__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The end of y[m, n] (z: the sums of both halves for SwiGLU)
template <typename T, bool GATED>
__device__ __forceinline__ void end_one(const GemmArgs& a, int64_t m, int n, float z0, float z1) {
  constexpr bool FULL = sizeof(T) == 4;
  const int64_t Z = GATED ? 2 * int64_t(a.N) : a.N;
  if (a.bias) {
    z0 += ld_f32(static_cast<const T*>(a.bias) + n);
    if (GATED) z1 += ld_f32(static_cast<const T*>(a.bias) + a.N + n);
  }
  if (a.z) {
    st_from_f32(static_cast<T*>(a.z) + m * Z + n, z0);
    if (GATED) st_from_f32(static_cast<T*>(a.z) + m * Z + a.N + n, z1);
  }
  float y = activate<FULL>(a.act, z0);
  if (GATED) y *= z1;
  if (a.r.p) y += ld_f32(static_cast<const T*>(a.r.p) + m * a.r.stride + n);
  st_from_f32(static_cast<T*>(a.y) + m * a.N + n, y);
}

__device__ __forceinline__ void clear_status(const GemmArgs& a) {
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    ws_header(a.ws)->err = 0;
    ws_header(a.ws)->timeout_site = 0;
  }
}

// MT: tiles of 8 rows of x
template <int MT, bool GATED, bool VEC>
__global__ void __launch_bounds__(256, 2) rows_bf16_kernel(const GemmArgs a) {
  constexpr int S = GATED ? 2 : 1, U = 2;  // U: steps in flight
  __shared__ float sums[kWarps][S][MT][16][8];
  clear_status(a);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int n0 = blockIdx.x * 16, K = int(a.K), M = int(a.M);
  const __nv_bfloat16* W = static_cast<const __nv_bfloat16*>(a.B);
  const __nv_bfloat16* X = static_cast<const __nv_bfloat16*>(a.A);
  // rows behind the last are read as the last, and not written
  const __nv_bfloat16 *w[S][2], *x[MT];
#pragma unroll
  for (int s = 0; s < S; ++s)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int n = n0 + g + 8 * i < a.N ? n0 + g + 8 * i : a.N - 1;
      w[s][i] = W + (int64_t(s) * a.N + n) * a.b_n;
    }
#pragma unroll
  for (int i = 0; i < MT; ++i) x[i] = X + int64_t(i * 8 + g < M ? i * 8 + g : M - 1) * a.a_m;
  float acc[S][MT][4] = {};
  auto add = [&](bool to) {  // this thread's cells of `sums`
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const float* c = acc[s][i];
        float2* lo = reinterpret_cast<float2*>(&sums[warp][s][i][g][2 * t]);
        float2* hi = reinterpret_cast<float2*>(&sums[warp][s][i][g + 8][2 * t]);
        *lo = to ? make_float2(lo->x + c[0], lo->y + c[1]) : make_float2(c[0], c[1]);
        *hi = to ? make_float2(hi->x + c[2], hi->y + c[3]) : make_float2(c[2], c[3]);
      }
  };
  add(false);
  for (int k0 = warp * 64; k0 < K; k0 += U * kWarps * 64) {
    uint4 wv[U][2][S][2], xv[U][2][MT];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int k = k0 + u * kWarps * 64 + c * 32 + 8 * t;
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
          for (int i = 0; i < 2; ++i) wv[u][c][s][i] = take8<VEC, true>(w[s][i], k, K);
#pragma unroll
        for (int i = 0; i < MT; ++i) xv[u][c][i] = take8<VEC, false>(x[i], k, K);
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            const uint4 p = wv[u][c][s][0], q = wv[u][c][s][1], b = xv[u][c][i];
            mma16816(acc[s][i], p.x, q.x, p.y, q.y, b.x, b.y);
            mma16816(acc[s][i], p.z, q.z, p.w, q.w, b.z, b.w);
          }
    // The products' sums lose about a step of fp32 an addition, towards zero; sums of runs round to nearest (2^20 features of
    // one sign were 7.9e-4 off in one go).
    if (k0 % kRowsRun >= kRowsRun - U * kWarps * 64) {
      add(true);
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[s][i][0] = acc[s][i][1] = acc[s][i][2] = acc[s][i][3] = 0.f;
    }
  }
  add(true);
  __syncthreads();
  const int e = threadIdx.x, n = e % 16, m = e / 16;  // 16 columns of up to 16 rows
  if (m < M && m < 8 * MT && n0 + n < a.N) {
    float z[2] = {0.f, 0.f};
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int v = 0; v < kWarps; ++v) z[s] += sums[v][s][m / 8][n][m % 8];
    end_one<__nv_bfloat16, GATED>(a, m, n0 + n, z[0], z[1]);
  }
}

// R rows of W (of each half) against MT rows of x
template <int R, int MT, bool GATED, bool VEC>
__global__ void __launch_bounds__(256, 2) rows_f32_kernel(const GemmArgs a) {
  constexpr int S = GATED ? 2 : 1, RS = R / S;  // columns of y
  __shared__ float sums[kWarps][R][MT];
  clear_status(a);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n0 = blockIdx.x * RS, K = int(a.K), M = int(a.M);
  const float *w[R], *x[MT];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int n = n0 + i % RS < a.N ? n0 + i % RS : a.N - 1;
    w[i] = static_cast<const float*>(a.B) + (int64_t(i / RS) * a.N + n) * a.b_n;
  }
#pragma unroll
  for (int i = 0; i < MT; ++i) x[i] = static_cast<const float*>(a.A) + int64_t(i < M ? i : M - 1) * a.a_m;
  float acc[R][MT] = {};
  for (int k = warp * 128 + 4 * lane; k - 4 * lane < K; k += kWarps * 128) {
    float4 wv[R];
#pragma unroll
    for (int i = 0; i < R; ++i) wv[i] = take4<VEC, true>(w[i], k, K);
#pragma unroll
    for (int j = 0; j < MT; ++j) {
      const float4 xv = take4<VEC, false>(x[j], k, K);
#pragma unroll
      for (int i = 0; i < R; ++i)
        acc[i][j] = fmaf(wv[i].w, xv.w, fmaf(wv[i].z, xv.z, fmaf(wv[i].y, xv.y, fmaf(wv[i].x, xv.x, acc[i][j]))));
    }
  }
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) acc[i][j] += __shfl_xor_sync(0xFFFFFFFFu, acc[i][j], o);
      if (lane == 0) sums[warp][i][j] = acc[i][j];
    }
  __syncthreads();
  const int e = threadIdx.x, n = e % RS, m = e / RS;
  if (m < M && m < MT && n0 + n < a.N) {
    float z[2] = {0.f, 0.f};
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int v = 0; v < kWarps; ++v) z[s] += sums[v][s * RS + n][m];
    end_one<float, GATED>(a, m, n0 + n, z[0], z[1]);
  }
}

constexpr int kCols = 4;            // columns of a thread
constexpr int kStrip = 256 * kCols;  // and of a block

// Column j of this thread in strip c0: neighbours where rows allow them to be accessed together, else one of 256 threads'.
template <bool VEC>
__device__ __forceinline__ int strip_column(int c0, int j) {
  return c0 + (VEC ? int(threadIdx.x) * kCols + j : j * 256 + int(threadIdx.x));
}
template <bool VEC>
__device__ __forceinline__ void load_columns(const float* row, int c0, int K, float* v) {
  if (VEC) {
    const int k = strip_column<VEC>(c0, 0);
    const float4 f = k < K ? __ldg(reinterpret_cast<const float4*>(row + k)) : make_float4(0, 0, 0, 0);
    v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w;
  } else {
#pragma unroll
    for (int j = 0; j < kCols; ++j) v[j] = strip_column<VEC>(c0, j) < K ? __ldg(row + strip_column<VEC>(c0, j)) : 0.f;
  }
}
template <bool VEC>
__device__ __forceinline__ void load_columns(const __nv_bfloat16* row, int c0, int K, float* v) {
  if (VEC) {
    const int k = strip_column<VEC>(c0, 0);
    const uint2 u = k < K ? __ldg(reinterpret_cast<const uint2*>(row + k)) : make_uint2(0, 0);
    v[0] = __uint_as_float(u.x << 16), v[1] = __uint_as_float(u.x & 0xFFFF0000u);
    v[2] = __uint_as_float(u.y << 16), v[3] = __uint_as_float(u.y & 0xFFFF0000u);
  } else {
#pragma unroll
    for (int j = 0; j < kCols; ++j) v[j] = strip_column<VEC>(c0, j) < K ? ld_nc(row + strip_column<VEC>(c0, j)) : 0.f;
  }
}

// dz of `count` rows of W from z0 on into shared memory, [row][MT], zeros behind M.
template <int MT, typename T>
__device__ __forceinline__ void load_dz(const RowsGradArgs& a, int64_t z0, int count, float (*s)[MT]) {
  for (int e = threadIdx.x; e < count * MT; e += 256) {
    const int i = e % count, m = e / count;
    s[i][m] = m < a.M ? ld_f32(static_cast<const T*>(a.dz) + int64_t(m) * a.pitch + z0 + i) : 0.f;
  }
}

constexpr int kDzRows = 64;  // rows of W whose dz a block holds at a time

// partial[blockIdx.y][m][k] = sum of dz[m, z] W[z, k] over the block's share of z
template <typename T, int MT, bool VEC>
__global__ void __launch_bounds__(256) rows_dx_kernel(const RowsGradArgs a) {
  __shared__ __align__(16) float dz[kDzRows][MT];
  const int c0 = blockIdx.x * kStrip;
  const int64_t begin = range_begin(a.Z, gridDim.y, blockIdx.y), stop = range_begin(a.Z, gridDim.y, blockIdx.y + 1);
  float acc[MT][kCols] = {};
  for (int64_t z0 = begin; z0 < stop; z0 += kDzRows) {
    const int count = stop - z0 < kDzRows ? int(stop - z0) : kDzRows;
    __syncthreads();
    load_dz<MT, T>(a, z0, count, dz);
    __syncthreads();
    const T* w = static_cast<const T*>(a.w) + z0 * a.w_stride;
    for (int i = 0; i < count; i += 4) {  // four rows of W on their way
      float v[4][kCols];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (i + k < count) {
          load_columns<VEC>(w + (i + k) * a.w_stride, c0, a.K, v[k]);
        } else {
#pragma unroll
          for (int j = 0; j < kCols; ++j) v[k][j] = 0.f;
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (i + k >= count) break;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const float d = dz[i + k][m];
#pragma unroll
          for (int j = 0; j < kCols; ++j) acc[m][j] = fmaf(d, v[k][j], acc[m][j]);
        }
      }
    }
  }
  float* out = a.partial + int64_t(blockIdx.y) * a.M * a.K;
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int j = 0; j < kCols; ++j)
      if (m < a.M && strip_column<VEC>(c0, j) < a.K) out[int64_t(m) * a.K + strip_column<VEC>(c0, j)] = acc[m][j];
}

template <typename T, int MT, bool VEC>
__global__ void __launch_bounds__(256) rows_dw_kernel(const RowsGradArgs a) {
  __shared__ __align__(16) float dz[kDzRows][MT];
  const int c0 = blockIdx.x * kStrip;
  const int64_t z0 = int64_t(blockIdx.y) * kDzRows;
  const int count = a.Z - z0 < kDzRows ? int(a.Z - z0) : kDzRows;
  load_dz<MT, T>(a, z0, count, dz);
  float x[MT][kCols];
#pragma unroll
  for (int m = 0; m < MT; ++m)  // behind M dz is 0: the last row again, which is there
    load_columns<VEC>(static_cast<const T*>(a.x) + int64_t(m < a.M ? m : a.M - 1) * a.x_stride, c0, a.K, x[m]);
  __syncthreads();
  T* out = static_cast<T*>(a.dw) + z0 * a.K;
#pragma unroll 2
  for (int i = 0; i < count; ++i, out += a.K) {
    float v[kCols] = {};
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      if (m >= a.M) break;
      const float d = dz[i][m];
#pragma unroll
      for (int j = 0; j < kCols; ++j) v[j] = fmaf(d, x[m][j], v[j]);
    }
    if (VEC) {
      if (strip_column<VEC>(c0, 0) < a.K) store_n<4>(out + strip_column<VEC>(c0, 0), v);
    } else {
#pragma unroll
      for (int j = 0; j < kCols; ++j)
        if (strip_column<VEC>(c0, j) < a.K) st_from_f32(out + strip_column<VEC>(c0, j), v[j]);
    }
  }
}

}  // namespace

int rows_dx_shares(int64_t Z, int64_t K) {
  const int64_t strips = (K + kStrip - 1) / kStrip, most = (Z + 31) / 32;
  const int64_t want = (int64_t(sm_count()) * 4 + strips - 1) / strips;
  return int(want < most ? want : most);
}

cudaError_t launch_rows_grads(const RowsGradArgs& a, cudaStream_t st, int* launches) {
  const size_t es = a.dt == SA_BF16 ? 2 : 4;
  auto ok = [&](const void* p, int64_t stride) {  // rows of four neighbours
    return reinterpret_cast<uintptr_t>(p) % (4 * es) == 0 && stride % 4 == 0;
  };
  const unsigned strips = unsigned((a.K + kStrip - 1) / kStrip);
  cudaError_t e = cudaSuccess;
  auto go = [&](auto kernel, unsigned y) {
    kernel<<<dim3(strips, y), 256, 0, st>>>(a);
    ++*launches;
    e = cudaGetLastError();
  };
#define SA_PICK(KERNEL, VEC, Y)                                                                                   \
  (a.dt == SA_BF16 ? (VEC ? go(KERNEL<__nv_bfloat16, 4, true>, Y) : go(KERNEL<__nv_bfloat16, 4, false>, Y))     \
                   : (a.M <= 4 ? (VEC ? go(KERNEL<float, 4, true>, Y) : go(KERNEL<float, 4, false>, Y))           \
                               : (VEC ? go(KERNEL<float, 16, true>, Y) : go(KERNEL<float, 16, false>, Y))))
  if (a.dx) {
    const int G = rows_dx_shares(a.Z, a.K);
    SA_PICK(rows_dx_kernel, a.K % 4 == 0 && ok(a.w, a.w_stride), unsigned(G));
    const int64_t n = int64_t(a.M) * a.K;
    if (e == cudaSuccess) e = launch_join_columns(a.partial, G, n, n, a.dx, a.dt, st);
    ++*launches;
  }
  if (e == cudaSuccess && a.dw)
    SA_PICK(rows_dw_kernel, a.K % 4 == 0 && ok(a.x, a.x_stride) && ok(a.dw, a.K), unsigned((a.Z + kDzRows - 1) / kDzRows));
#undef SA_PICK
  return e;
}

cudaError_t launch_rows(const GemmArgs& a, cudaStream_t st) {
  const bool gated = a.act == SA_ACT_SWIGLU;
  const int each = a.dt == SA_BF16 ? 8 : 4;
  auto row_ok = [&](const void* p, int64_t stride) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % each == 0;
  };
  const bool vec = a.K % each == 0 && row_ok(a.A, a.a_m) && row_ok(a.B, a.b_n);
  auto go = [&](auto kernel, int columns) {
    kernel<<<unsigned((a.N + columns - 1) / columns), 256, 0, st>>>(a);
    return cudaGetLastError();
  };
#define SA_PICK(K, COLS, ...)                                                                          \
  (gated ? (vec ? go(K<__VA_ARGS__, true, true>, COLS) : go(K<__VA_ARGS__, true, false>, COLS))         \
         : (vec ? go(K<__VA_ARGS__, false, true>, COLS) : go(K<__VA_ARGS__, false, false>, COLS)))
  if (a.dt == SA_BF16) return a.M <= 8 ? SA_PICK(rows_bf16_kernel, 16, 1) : SA_PICK(rows_bf16_kernel, 16, 2);
  if (a.M <= 8) return SA_PICK(rows_f32_kernel, (gated ? 2 : 4), 4, 8);
  return SA_PICK(rows_f32_kernel, (gated ? 1 : 2), 2, 16);
#undef SA_PICK
}

}  // namespace dense
}  // namespace sa
