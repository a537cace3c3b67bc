// Linear layers on the CUDA cores, for every size, stride and type, and the activation's slope in
// the gradient.
//
//   gemm      C[m, n] = sum_k A(m, k) B(n, k) for any strides of m, n and k, then bias, activation
//             and residual.  One block makes 64 x 64 results, each thread 4 x 4, from 16-deep slices
//             in shared memory; sums in fp32 in order of k.
//   act_grad  dz = dy act'(z) and the column sums of dz, one pass over dy and z: bound by memory.
#include "sa_dense_act.cuh"

namespace sa {
namespace dense {
namespace {

constexpr int TM = 64, TN = 64, TK = 16;

template <typename T, bool GATED>
__global__ void __launch_bounds__(256) simt_gemm_kernel(const GemmArgs g) {
  constexpr int S = GATED ? 2 : 1;
  __shared__ float sa[TK][TM + 4];
  __shared__ float sb[S][TK][TN + 4];
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  const int64_t m0 = int64_t(blockIdx.x) * TM;
  const int n0 = blockIdx.y * TN;
  const T* A = static_cast<const T*>(g.A);
  const T* B = static_cast<const T*>(g.B);
  float acc[S][4][4] = {};
  // neighbouring threads read along the contiguous axis
  const bool a_along_k = g.a_k == 1, b_along_k = g.b_k == 1;
  for (int64_t k0 = 0; k0 < g.K; k0 += TK) {
#pragma unroll
    for (int i = 0; i < TM * TK / 256; ++i) {
      const int e = threadIdx.x + i * 256;
      const int m = a_along_k ? e / TK : e % TM, k = a_along_k ? e % TK : e / TM;
      sa[k][m] = m0 + m < g.M && k0 + k < g.K ? ld_f32(A + (m0 + m) * g.a_m + (k0 + k) * g.a_k) : 0.f;
    }
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int i = 0; i < TN * TK / 256; ++i) {
        const int e = threadIdx.x + i * 256;
        const int n = b_along_k ? e / TK : e % TN, k = b_along_k ? e % TK : e / TN;
        sb[s][k][n] = n0 + n < g.N && k0 + k < g.K
                          ? ld_f32(B + (int64_t(s) * g.N + n0 + n) * g.b_n + (k0 + k) * g.b_k)
                          : 0.f;
      }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < TK; ++k) {
      float a[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] = sa[k][ty + 16 * i];
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float b = sb[s][k][tx + 16 * j];
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[s][i][j] = fmaf(a[i], b, acc[s][i][j]);
        }
    }
    __syncthreads();
  }
  constexpr bool FULL = sizeof(T) == 4;
  const int64_t Z = int64_t(S) * g.N;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t m = m0 + ty + 16 * i;
      const int n = n0 + tx + 16 * j;
      if (m >= g.M || n >= g.N) continue;
      float z[S];
#pragma unroll
      for (int s = 0; s < S; ++s) {
        z[s] = acc[s][i][j];
        if (g.bias) z[s] += ld_f32(static_cast<const T*>(g.bias) + int64_t(s) * g.N + n);
        if (g.z) st_from_f32(static_cast<T*>(g.z) + m * Z + int64_t(s) * g.N + n, z[s]);
      }
      float y = activate<FULL>(g.act, z[0]);
      if (GATED) y *= z[S - 1];
      if (g.r.p) y += ld_f32(static_cast<const T*>(g.r.p) + m * g.r.stride + n);
      st_from_f32(static_cast<T*>(g.y) + m * g.N + n, y);
    }
}

// Columns are spread over 32 lanes x 8 (fewer lanes where there are fewer columns, and the rest of the
// warp takes other rows); a block's eight warps and its share of the rows leave one partial row of sums.

// Aligned rows (VEC) come through a ring of three rows a thread in shared memory, filled by the thread's own cp.async: a
// row's loads and its arithmetic would wait for each other (the columns' sums of 16384 x 8192 gated: 107 us with two rows
// in registers, 70 so, 5.7 TB/s).
constexpr int kRing = 3;

template <typename T, bool VEC, bool GATED>
__global__ void __launch_bounds__(256, GATED && sizeof(T) == 4 ? 2 : 3) act_grad_kernel(const ActGradArgs a, int lanes) {
  constexpr int S = GATED ? 2 : 1;
  constexpr bool FULL = sizeof(T) == 4;
  constexpr int P = int(sizeof(T)) / 2;  // 16-byte pieces of 8 values
  extern __shared__ __align__(16) char mem[];  // VEC: the ring; at the end the warps' sums [8][S][256]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int t = lane % lanes, per_warp = 32 / lanes;
  const int c0 = blockIdx.x * 256;
  const T* dy = static_cast<const T*>(a.dy.p);
  const T* z = static_cast<const T*>(a.z);
  float sum[S][8] = {};
  const int64_t step = int64_t(gridDim.y) * 8 * per_warp;
  auto col = [&](int j) { return c0 + (VEC ? t * 8 + j : j * lanes + t); };
  int64_t row = (int64_t(blockIdx.y) * 8 + warp) * per_warp + lane / lanes;

  constexpr int kApart = 256 * 16, kRow = (S + 1) * P * kApart;  // bytes between a thread's pieces, and between rows
  char* own = mem + threadIdx.x * 16;
  const bool in = col(0) < a.N;
  int64_t ahead = row;
  int put = 0, get = 0;
  auto copy8 = [&](int slot, const T* p) {
    const uint32_t to = ptx::smem_u32(own) + slot;
    if (P == 1) {
      copy16(to, p);
    } else {
      copy16_l1(to, p);
      copy16_l1(to + kApart, p + 4);
    }
  };
  auto fetch = [&] {
    if (ahead < a.M && in) {
      copy8(put, dy + ahead * a.dy.stride + col(0));
      if (a.act != SA_ACT_NONE)
#pragma unroll
        for (int s = 0; s < S; ++s) copy8(put + (s + 1) * P * kApart, z + ahead * a.Z + int64_t(s) * a.N + col(0));
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    ahead += step;
    put = put == (kRing - 1) * kRow ? 0 : put + kRow;
  };
  auto take8 = [&](int slot, float* v) {
    if (P == 1) {
      load8(reinterpret_cast<const __nv_bfloat16*>(own + slot), v);
    } else {
      const float4 x = *reinterpret_cast<const float4*>(own + slot), y = *reinterpret_cast<const float4*>(own + slot + kApart);
      v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w, v[4] = y.x, v[5] = y.y, v[6] = y.z, v[7] = y.w;
    }
  };
  if (VEC)
#pragma unroll
    for (int i = 0; i < kRing - 1; ++i) fetch();

  for (; row < a.M; row += step) {
    float g[8], zz[S][8];
    if (VEC) {
      fetch();
      asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
      if (in) {
        take8(get, g);
        if (a.act != SA_ACT_NONE)
#pragma unroll
          for (int s = 0; s < S; ++s) take8(get + (s + 1) * P * kApart, zz[s]);
      }
      get = get == (kRing - 1) * kRow ? 0 : get + kRow;
      if (!in) continue;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool inside = col(j) < a.N;
        g[j] = inside ? ld_f32(dy + row * a.dy.stride + col(j)) : 0.f;
#pragma unroll
        for (int s = 0; s < S; ++s)
          zz[s][j] = inside && a.act != SA_ACT_NONE ? ld_f32(z + row * a.Z + int64_t(s) * a.N + col(j)) : 0.f;
      }
    }
    float d[S][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (GATED) {
        const float p = sigmoid<FULL>(zz[0][j]);
        d[0][j] = g[j] * zz[S - 1][j] * (p * fmaf(zz[0][j], 1.f - p, 1.f));
        d[S - 1][j] = g[j] * (zz[0][j] * p);
      } else {
        d[0][j] = a.act == SA_ACT_NONE   ? g[j]
                  : a.act == SA_ACT_RELU ? (zz[0][j] > 0.f ? g[j] : 0.f)
                                         : g[j] * slope<FULL>(a.act, zz[0][j]);
      }
    }
#pragma unroll
    for (int s = 0; s < S; ++s) {
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[s][j] += d[s][j];
      if (!a.dz) continue;
      const int64_t at = row * a.pitch + int64_t(s) * a.N;
      if (sizeof(T) == 4 && a.terms) {  // never of bf16
        __nv_bfloat16* o = static_cast<__nv_bfloat16*>(a.dz) + at;
        const int64_t plane = a.M * a.pitch;
        if (VEC) {
          store_terms(o + col(0), plane, d[s]);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (col(j) < a.N) {
              float left = d[s][j];
#pragma unroll
              for (int k = 0; k < 3; ++k) {
                const __nv_bfloat16 term = term_of(left, k);
                o[k * plane + col(j)] = term;
                left -= __bfloat162float(term);
              }
            }
        }
      } else {
        T* o = static_cast<T*>(a.dz) + at;
        if (VEC) {
          store8(o + col(0), d[s]);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (col(j) < a.N) st_from_f32(o + col(j), d[s][j]);
        }
      }
    }
  }
  if (!a.partial) return;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    if (o >= lanes)
#pragma unroll
      for (int s = 0; s < S; ++s)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[s][j] += __shfl_xor_sync(0xFFFFFFFFu, sum[s][j], o);
  float(*part)[S][256] = reinterpret_cast<float(*)[S][256]>(mem);
  __syncthreads();  // the ring is read out (no copy is in flight: the last rows' were waited for)
  if (lane < lanes)
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j) part[warp][s][col(j) - c0] = sum[s][j];
  __syncthreads();
  const int c = c0 + threadIdx.x;
  if (c < a.N && threadIdx.x < lanes * 8)
#pragma unroll
    for (int s = 0; s < S; ++s) {
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < 8; ++w) v += part[w][s][threadIdx.x];
      a.partial[int64_t(blockIdx.y) * a.Z + int64_t(s) * a.N + c] = v;
    }
}

int lanes_for(int N) {
  int lanes = 1;
  while (lanes < 32 && lanes * 8 < N) lanes *= 2;
  return lanes;
}

}  // namespace

int act_grad_blocks(int64_t M, int N) {
  const int strips = (N + 255) / 256, rows = 8 * (32 / lanes_for(N));
  const int64_t most = (int64_t(sm_count()) * 8 + strips - 1) / strips;
  const int64_t need = (M + rows - 1) / rows;
  const int64_t g = need < most ? need : most;
  return int(g < 65535 ? g : 65535);
}

cudaError_t launch_act_grad(const ActGradArgs& a, cudaStream_t st) {
  const int G = act_grad_blocks(a.M, a.N);
  if (G == 0) return cudaSuccess;
  const int lanes = lanes_for(a.N), e = a.dy.dt == SA_BF16 ? 8 : 4;
  const dim3 grid((a.N + 255) / 256, G);
  const bool gated = a.act == SA_ACT_SWIGLU;
  auto base_ok = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; };
  const bool vec = a.N % 8 == 0 && base_ok(a.dy.p) && a.dy.stride % e == 0 && base_ok(a.z) && base_ok(a.dz) &&
                   a.pitch % 8 == 0;
  const size_t sums = size_t(8) * (gated ? 2 : 1) * 256 * sizeof(float);
  const size_t ring = vec ? size_t(kRing) * (gated ? 3 : 2) * (a.dy.dt == SA_BF16 ? 1 : 2) * 256 * 16 : 0;
  const size_t smem = ring > sums ? ring : sums;
  // the same size for a kernel at all times
  auto go = [&](auto type, auto aligned, auto halves) {
    using T = decltype(type);
    constexpr auto kernel = act_grad_kernel<T, aligned(), halves()>;
    if (smem > 48 * 1024) {
      const cudaError_t s = allow_smem<kernel>(smem);
      if (s != cudaSuccess) return s;
    }
    kernel<<<grid, 256, smem, st>>>(a, lanes);
    return cudaGetLastError();
  };
  auto pick = [&](auto type) {
    using std::true_type;
    using std::false_type;
    if (vec) return gated ? go(type, true_type{}, true_type{}) : go(type, true_type{}, false_type{});
    return gated ? go(type, false_type{}, true_type{}) : go(type, false_type{}, false_type{});
  };
  return a.dy.dt == SA_BF16 ? pick(__nv_bfloat16{}) : pick(float{});
}

cudaError_t launch_simt_gemm(const GemmArgs& g, cudaStream_t st) {
  const dim3 grid(unsigned((g.M + TM - 1) / TM), unsigned((g.N + TN - 1) / TN));
  const bool gated = g.act == SA_ACT_SWIGLU;
  if (g.dt == SA_BF16) {
    if (gated)
      simt_gemm_kernel<__nv_bfloat16, true><<<grid, 256, 0, st>>>(g);
    else
      simt_gemm_kernel<__nv_bfloat16, false><<<grid, 256, 0, st>>>(g);
  } else if (gated) {
    simt_gemm_kernel<float, true><<<grid, 256, 0, st>>>(g);
  } else {
    simt_gemm_kernel<float, false><<<grid, 256, 0, st>>>(g);
  }
  return cudaGetLastError();
}

}  // namespace dense
}  // namespace sa
