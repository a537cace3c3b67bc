// Linear layers' products on tcgen05: arguments, the share of the work each CTA (or pair) takes, and
// the end of a tile (bias, activation, residual, stores), which the product kernel and the join of cut
// tiles have in common.
#pragma once
#include "sa_dense_act.cuh"

namespace sa {
namespace dense {

// C[m, n] = sum over k of A[m, k] B[n, k], in tiles of 128 rows a CTA.
struct TcArgs {
  int64_t M;       // rows of C
  int N;           // columns of y
  int KB;          // blocks of 64 along k
  int mt, nt;      // tiles along m (of 128 rows, of 256 for a pair) and along y's columns
  int W;           // workers: CTAs or pairs
  int64_t whole;   // tiles [0, whole) go to workers in turn, the rest in equal shares of blocks
  int64_t cut;     // the rest's tiles
  int cutters;     // workers that take a share of them (at most one a block)
  int64_t half;    // SwiGLU: rows of B before the second half
  const void* bias;
  const void* r;
  int64_t r_stride;
  int act;
  void* y;
  void* z;
  int64_t Z;       // columns of z
  int vec;         // rows allow 16-byte access: 1 y and z, 2 r
  float* piece;    // [W][2][CTAs of a worker][BN / 4][128][4]
  void* ws;
  int clear;       // this launch clears the call's status
};

// Tile t's place: groups of eight tiles along m, within a group m first, so that tiles in flight
// together share rows of A and of B in L2.
__device__ __forceinline__ void tile_place(const TcArgs& a, int64_t t, int* mb, int* nb) {
  const int64_t per = int64_t(8) * a.nt, g = t / per;
  const int first = int(g) * 8, rows = a.mt - first < 8 ? a.mt - first : 8;
  const int in = int(t - g * per);
  *mb = first + in % rows;
  *nb = in / rows;
}

// A worker's segments in order: (tile, blocks [k0, k1)).
struct Segments {
  const TcArgs& a;
  int64_t t, u, u1;
  int64_t tile;
  int k0, k1;
  __device__ Segments(const TcArgs& a_, int w) : a(a_), t(w) {
    const int64_t total = a.cut * a.KB;
    u = u1 = 0;
    if (w < a.cutters) {
      u = range_begin(total, a.cutters, w);
      u1 = range_begin(total, a.cutters, w + 1);
    }
  }
  __device__ bool next() {
    if (t < a.whole) {
      tile = t;
      k0 = 0;
      k1 = a.KB;
      t += a.W;
      return true;
    }
    if (u >= u1) return false;
    const int64_t i = u / a.KB;
    tile = a.whole + i;
    k0 = int(u - i * a.KB);
    const int64_t left = u1 - u;
    k1 = left < a.KB - k0 ? k0 + int(left) : a.KB;
    u += k1 - k0;
    return true;
  }
  __device__ bool complete() const { return k0 == 0 && k1 == a.KB; }
};

enum { EPI_PLAIN = 0, EPI_FULL = 1, EPI_GATED = 2 };

template <int CTAS>
struct TileShape {
  static constexpr int BN = CTAS == 2 ? 256 : 128;           // accumulator columns
  template <int EPI>
  static constexpr int YN = EPI == EPI_GATED ? BN / 2 : BN;  // columns of y
  // chunks of 32 columns of y that an epilogue warp (of two for a row) makes, and where they begin
  template <int EPI>
  static constexpr int CHUNKS = YN<EPI> / 64;
};

// Rows' 32 columns as the warp stores them: 16-byte pieces in an order that keeps both the row-wise
// and the column-wise access free of bank conflicts.
template <typename T>
struct Stage;
template <>
struct Stage<__nv_bfloat16> {
  static constexpr int BYTES = 2048, PIECES = 4, EACH = 8;  // 16-byte pieces of a row, elements of a piece
  __device__ static uint32_t at(int row, int p) { return row * 64 + ((p ^ ((row >> 1) & 3)) << 4); }
};
template <>
struct Stage<float> {
  static constexpr int BYTES = 4096, PIECES = 8, EACH = 4;
  __device__ static uint32_t at(int row, int p) { return row * 128 + ((p ^ (row & 7)) << 4); }
};

// 32 values of this lane's row into the stage
__device__ __forceinline__ void stage_put(__nv_bfloat16*, char* s, int lane, const float* v) {
#pragma unroll
  for (int p = 0; p < 4; ++p)
    *reinterpret_cast<uint4*>(s + Stage<__nv_bfloat16>::at(lane, p)) =
        make_uint4(ptx::pack_bf16(v[8 * p], v[8 * p + 1]), ptx::pack_bf16(v[8 * p + 2], v[8 * p + 3]),
                   ptx::pack_bf16(v[8 * p + 4], v[8 * p + 5]), ptx::pack_bf16(v[8 * p + 6], v[8 * p + 7]));
}
__device__ __forceinline__ void stage_put(float*, char* s, int lane, const float* v) {
#pragma unroll
  for (int p = 0; p < 8; ++p)
    *reinterpret_cast<float4*>(s + Stage<float>::at(lane, p)) =
        make_float4(v[4 * p], v[4 * p + 1], v[4 * p + 2], v[4 * p + 3]);
}
// v += this lane's row of the stage
__device__ __forceinline__ void stage_add(__nv_bfloat16*, const char* s, int lane, float* v) {
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const uint4 q = *reinterpret_cast<const uint4*>(s + Stage<__nv_bfloat16>::at(lane, p));
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[8 * p + 2 * j] += __uint_as_float(w[j] << 16);
      v[8 * p + 2 * j + 1] += __uint_as_float(w[j] & 0xFFFF0000u);
    }
  }
}
__device__ __forceinline__ void stage_add(float*, const char* s, int lane, float* v) {
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const float4 q = *reinterpret_cast<const float4*>(s + Stage<float>::at(lane, p));
    v[4 * p] += q.x, v[4 * p + 1] += q.y, v[4 * p + 2] += q.z, v[4 * p + 3] += q.w;
  }
}

// The stage's 32 x 32 values to rows m0.. and columns n0.. of a matrix of M rows and n_end columns.
template <typename T>
__device__ __forceinline__ void stage_store(const char* s, int lane, void* dst, int64_t pitch, int64_t m0, int64_t M,
                                            int64_t n0, int64_t n_end, bool vec) {
  using S = Stage<T>;
  T* d = static_cast<T*>(dst);
  if (vec) {
    constexpr int ROWS = 32 / S::PIECES;
    const int p = lane % S::PIECES;
    const int64_t n = n0 + p * S::EACH;
#pragma unroll
    for (int i = 0; i < S::PIECES; ++i) {
      const int row = i * ROWS + lane / S::PIECES;
      const uint4 q = *reinterpret_cast<const uint4*>(s + S::at(row, p));
      if (m0 + row < M && n < n_end) *reinterpret_cast<uint4*>(d + (m0 + row) * pitch + n) = q;
    }
  } else {
#pragma unroll 4
    for (int row = 0; row < 32; ++row) {
      const T v = *reinterpret_cast<const T*>(s + S::at(row, lane / S::EACH) + (lane % S::EACH) * sizeof(T));
      if (m0 + row < M && n0 + lane < n_end) d[(m0 + row) * pitch + n0 + lane] = v;
    }
  }
}

// A chunk's residual, read ahead: 16-byte pieces in the order in which they are stored.
template <typename T>
struct Residual {
  uint4 q[Stage<T>::PIECES];
  __device__ __forceinline__ void load(const TcArgs& a, int lane, int64_t m0, int n0) {
    using S = Stage<T>;
    if (!(a.vec & 2)) return;
    const T* r = static_cast<const T*>(a.r);
    constexpr int ROWS = 32 / S::PIECES;
    const int n = n0 + (lane % S::PIECES) * S::EACH;
#pragma unroll
    for (int i = 0; i < S::PIECES; ++i) {
      const int64_t m = m0 + i * ROWS + lane / S::PIECES;
      q[i] = make_uint4(0, 0, 0, 0);
      if (m < a.M && n < a.N) q[i] = *reinterpret_cast<const uint4*>(r + m * a.r_stride + n);
    }
  }
  __device__ __forceinline__ void put(const TcArgs& a, char* s, int lane, int64_t m0, int n0) const {
    using S = Stage<T>;
    if (a.vec & 2) {
      constexpr int ROWS = 32 / S::PIECES;
#pragma unroll
      for (int i = 0; i < S::PIECES; ++i)
        *reinterpret_cast<uint4*>(s + S::at(i * ROWS + lane / S::PIECES, lane % S::PIECES)) = q[i];
    } else {
      const T* r = static_cast<const T*>(a.r);
#pragma unroll 16
      for (int row = 0; row < 32; ++row) {
        T v = T(0.f);
        if (m0 + row < a.M && n0 + lane < a.N) v = r[(m0 + row) * a.r_stride + n0 + lane];
        *reinterpret_cast<T*>(s + S::at(row, lane / S::EACH) + (lane % S::EACH) * sizeof(T)) = v;
      }
    }
  }
};

// The end of 32 rows (m0 + lane) x 32 columns (n0 ..) of y: v holds the sums (SwiGLU: of the gate's half, u of
// the other's), bv and bu the biases of these columns (in shared memory), s the warp's stage.
template <typename T, int EPI>
__device__ __forceinline__ void finish_chunk(const TcArgs& a, float* v, float* u, const float* bv, const float* bu,
                                             const Residual<T>& res, char* s, int lane, int64_t m0, int n0) {
  constexpr bool FULL = sizeof(T) == 4;
  T* tag = nullptr;
  const bool vec = (a.vec & 1) != 0;
  if (EPI != EPI_PLAIN) {
#pragma unroll
    for (int j = 0; j < 32; j += 4) {
      const float4 b = *reinterpret_cast<const float4*>(bv + j);
      v[j] += b.x, v[j + 1] += b.y, v[j + 2] += b.z, v[j + 3] += b.w;
      if (EPI == EPI_GATED) {
        const float4 c = *reinterpret_cast<const float4*>(bu + j);
        u[j] += c.x, u[j + 1] += c.y, u[j + 2] += c.z, u[j + 3] += c.w;
      }
    }
    if (a.z) {
      stage_put(tag, s, lane, v);
      __syncwarp();
      stage_store<T>(s, lane, a.z, a.Z, m0, a.M, n0, a.N, vec);
      __syncwarp();
      if (EPI == EPI_GATED) {
        stage_put(tag, s, lane, u);
        __syncwarp();
        stage_store<T>(s, lane, a.z, a.Z, m0, a.M, a.half + n0, a.half + a.N, vec);
        __syncwarp();
      }
    }
    if (EPI == EPI_GATED) {
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = v[j] * sigmoid<FULL>(v[j]) * u[j];
    } else if (a.act == SA_ACT_RELU) {
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = activate<FULL>(SA_ACT_RELU, v[j]);
    } else if (a.act == SA_ACT_GELU) {
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = activate<FULL>(SA_ACT_GELU, v[j]);
    } else if (a.act == SA_ACT_SILU) {
#pragma unroll
      for (int j = 0; j < 32; ++j) v[j] = activate<FULL>(SA_ACT_SILU, v[j]);
    }
    if (a.r) {
      res.put(a, s, lane, m0, n0);
      __syncwarp();
      stage_add(tag, s, lane, v);
      __syncwarp();
    }
  }
  stage_put(tag, s, lane, v);
  __syncwarp();
  stage_store<T>(s, lane, a.y, a.N, m0, a.M, n0, a.N, vec);
  __syncwarp();
}

}  // namespace dense
}  // namespace sa
