// Linear layers' products on tcgen05: arguments, the share of the work each CTA (or pair) takes, and
// the end of a tile (bias, activation, residual, stores), which the product kernel and the join of cut
// tiles have in common.
#pragma once
#include "sa_dense_act.cuh"

namespace sa {
namespace dense {

// n / d of n < 2^31 by a product: with 2^(s-1) < d <= 2^s and m = floor(2^32 (2^s - d) / d) + 1, it is
// (floor(n m / 2^32) + n) / 2^s rounded down.
struct Divisor {
  uint32_t m;
  int s;
  Divisor() = default;
  explicit Divisor(uint32_t d) : s(0) {
    while ((uint64_t(1) << s) < d) ++s;
    m = uint32_t((((uint64_t(1) << s) - d) << 32) / d) + 1;
  }
  __device__ __forceinline__ uint32_t quotient(uint32_t n) const { return (__umulhi(n, m) + n) >> s; }
};

// Blocks of bf16 products that accumulate in TMEM in one go (sa_dense_tc.cu): 16384 terms a sum.
constexpr int kRun = 256;

// C[m, n] = sum over k of A[m, k] B[n, k], in tiles of 128 rows a CTA.
struct TcArgs {
  int64_t M;       // rows of C
  int N;           // columns of y
  int KB;          // blocks of 64 along k
  int mt, nt;      // tiles along m (of 128 rows, of 256 for a pair) and along y's columns
  Divisor by_group, by_last;  // by the tiles of eight along m, and of the last ones' along m
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
  float* piece;    // [cutters][2][CTAs of a worker][BN / 4][128][4]
  float* sums;     // bf16 and more than kRun blocks: [W][CTAs of a worker][BN / 4][128][4]
  void* ws;
  int clear;       // this launch clears the call's status
  uint32_t wait_ns;  // limit of every wait
};

// Tile t's place: groups of eight tiles along m, within a group m first, so that tiles in flight
// together share rows of A and of B in L2.  (64-bit divisions here cost 0.1 us a tile.)
__device__ __forceinline__ void tile_place(const TcArgs& a, int64_t t, int* mb, int* nb) {
  const uint32_t n = uint32_t(t), per = 8u * uint32_t(a.nt), g = a.by_group.quotient(n), in = n - g * per;
  const int first = int(g) * 8;
  const bool last = a.mt - first < 8;
  const uint32_t column = last ? a.by_last.quotient(in) : in >> 3;
  *mb = first + int(in - column * (last ? uint32_t(a.mt - first) : 8u));
  *nb = int(column);
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

template <int CTAS>
struct TileShape {
  static constexpr int BN = CTAS == 2 ? 256 : 128;           // accumulator columns
  static constexpr int GROUPS = 2;                            // epilogue warps of a row
  template <int EPI>
  static constexpr int YN = EPI == EPI_GATED ? BN / 2 : BN;  // columns of y
  // chunks of 32 columns of y that an epilogue warp makes
  template <int EPI>
  static constexpr int CHUNKS = YN<EPI> / (32 * GROUPS);
};

// A chunk's sums on their way from one row a lane to whole rows a few lanes: 32 rows of 128 bytes, 16-byte pieces in
// an order that keeps both directions free of bank conflicts.
constexpr int kStageBytes = 4096;
__device__ __forceinline__ uint32_t stage_at(int row, int p) { return row * 128 + ((p ^ (row & 7)) << 4); }

// COLS values of this lane's row into the stage, from 16-byte piece `first` on
template <int COLS>
__device__ __forceinline__ void stage_put(char* s, int lane, const float* v, int first = 0) {
#pragma unroll
  for (int p = 0; p < COLS / 4; ++p)
    *reinterpret_cast<float4*>(s + stage_at(lane, first + p)) = make_float4(v[4 * p], v[4 * p + 1], v[4 * p + 2], v[4 * p + 3]);
}

// How a chunk ends: EACH neighbouring values a lane of a row's COLS columns.  SwiGLU's chunks have 16 columns, so that the
// gate's and the other half's share the stage.
template <typename T, int EPI>
struct ChunkEnd {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int COLS = EPI == EPI_GATED ? 16 : 32;
  static constexpr int EACH = F32 || EPI == EPI_GATED ? 4 : 8;
  static constexpr int LANES = COLS / EACH;   // lanes of a row
  static constexpr int ROWS = 32 / LANES;     // rows at a time
  static constexpr int U = COLS / 4;          // the other half's first 16-byte piece of the stage

  float bv[EACH], bu[EACH];  // biases of this lane's columns

  // the biases of columns n0 ..; on their way while the products are awaited
  __device__ __forceinline__ void load_bias(const TcArgs& a, int lane, int n0) {
    if (EPI == EPI_PLAIN) return;
    const T* b = static_cast<const T*>(a.bias);
#pragma unroll
    for (int j = 0; j < EACH; ++j) bv[j] = bu[j] = 0.f;
    if (!b) return;
    if (a.vec & 1) {
      const int n = n0 + (lane % LANES) * EACH;
      if (n >= a.N) return;
#pragma unroll
      for (int j = 0; j < EACH; ++j) {
        bv[j] = ld_f32(b + n + j);
        if (EPI == EPI_GATED) bu[j] = ld_f32(b + a.half + n + j);
      }
    } else {
      const int n = n0 + lane % COLS;
      if (n >= a.N) return;
      bv[0] = ld_f32(b + n);
      if (EPI == EPI_GATED) bu[0] = ld_f32(b + a.half + n);
    }
  }

  __device__ __forceinline__ static void activate_all(int act, float* v, const float* u) {
    if (EPI == EPI_GATED) {
#pragma unroll
      for (int j = 0; j < EACH; ++j) v[j] = v[j] * sigmoid<F32>(v[j]) * u[j];
    } else if (act == SA_ACT_RELU) {
#pragma unroll
      for (int j = 0; j < EACH; ++j) v[j] = activate<F32>(SA_ACT_RELU, v[j]);
    } else if (act == SA_ACT_GELU) {
#pragma unroll
      for (int j = 0; j < EACH; ++j) v[j] = activate<F32>(SA_ACT_GELU, v[j]);
    } else if (act == SA_ACT_SILU) {
#pragma unroll
      for (int j = 0; j < EACH; ++j) v[j] = activate<F32>(SA_ACT_SILU, v[j]);
    }
  }

  __device__ __forceinline__ static void read(const char* s, int row, int first, float* v) {
#pragma unroll
    for (int p = 0; p < EACH / 4; ++p) {
      const float4 f = *reinterpret_cast<const float4*>(s + stage_at(row, first + p));
      v[4 * p] = f.x, v[4 * p + 1] = f.y, v[4 * p + 2] = f.z, v[4 * p + 3] = f.w;
    }
  }

  // Rows m0 .. m0 + 31, columns n0 .. n0 + COLS - 1 of y, of the sums in the stage; of PARTS, the rows of `part` only.
  template <int PARTS>
  __device__ __forceinline__ void finish(const TcArgs& a, const char* s, int lane, int64_t m0, int n0, int part) const {
    if (a.vec & 1) {
      const int p = lane % LANES, n = n0 + p * EACH;
      const bool res = EPI != EPI_PLAIN && a.r, res_vec = (a.vec & 2) != 0;
      const int first = part * (LANES / PARTS);
      int64_t m = m0 + first * ROWS + lane / LANES;
      T* y = static_cast<T*>(a.y) + m * a.N + n;
      T* z = static_cast<T*>(a.z) + m * a.Z + n;
      const T* r = static_cast<const T*>(a.r) + m * a.r_stride + n;
      // rows by fours (fewer where there are fewer): their residuals are on their way together, and a long activation has
      // four copies and not more, which the instruction cache holds
      constexpr int COUNT = LANES / PARTS, FOUR = COUNT < 4 ? COUNT : 4;
#pragma unroll 1
      for (int i0 = 0; i0 < COUNT; i0 += FOUR) {
        float rv[FOUR][EACH];
        if (EPI != EPI_PLAIN && res) {
#pragma unroll
          for (int k = 0; k < FOUR; ++k) {
            if (m + k * ROWS >= a.M || n >= a.N) continue;
            const T* from = r + int64_t(k * ROWS) * a.r_stride;
            if (res_vec) {
              load_n<EACH>(from, rv[k]);
            } else {
#pragma unroll
              for (int j = 0; j < EACH; ++j) rv[k][j] = ld_nc(from + j);
            }
          }
          r += int64_t(FOUR * ROWS) * a.r_stride;
        }
#pragma unroll
        for (int k = 0; k < FOUR; ++k) {
          const int row = (first + i0 + k) * ROWS + lane / LANES;
          const bool here = m < a.M && n < a.N;
          float v[EACH], u[EACH];
          read(s, row, p * (EACH / 4), v);
          if (EPI == EPI_GATED) read(s, row, U + p * (EACH / 4), u);
          if (EPI != EPI_PLAIN) {
#pragma unroll
            for (int j = 0; j < EACH; ++j) {
              v[j] += bv[j];
              if (EPI == EPI_GATED) u[j] += bu[j];
            }
            if (a.z && here) {
              store_n<EACH>(z, v);
              if (EPI == EPI_GATED) store_n<EACH>(z + a.half, u);
            }
            activate_all(a.act, v, u);
            if (res) {
#pragma unroll
              for (int j = 0; j < EACH; ++j) v[j] += rv[k][j];
            }
            z += int64_t(ROWS) * a.Z;
          }
          if (here) store_n<EACH>(y, v);
          m += ROWS;
          y += int64_t(ROWS) * a.N;
        }
      }
    } else {  // one value a lane, so that single-element accesses coalesce; four rows at a time
      const int c = lane % COLS, n = n0 + c;
      constexpr int AT_ONCE = 32 / COLS;
      const bool res = EPI != EPI_PLAIN && a.r;
      float next[4];
      auto fetch = [&](int i) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int64_t m = m0 + (i + k) * AT_ONCE + lane / COLS;
          next[k] = m < a.M && n < a.N ? ld_nc(static_cast<const T*>(a.r) + m * a.r_stride + n) : 0.f;
        }
      };
      const int begin = part * (COLS / PARTS), stop = begin + COLS / PARTS;
      if (res) fetch(begin);
#pragma unroll 1
      for (int i = begin; i < stop; i += 4) {
        float rv[4] = {0.f, 0.f, 0.f, 0.f};
        if (res) {
#pragma unroll
          for (int k = 0; k < 4; ++k) rv[k] = next[k];
          if (i + 4 < stop) fetch(i + 4);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int row = (i + k) * AT_ONCE + lane / COLS;
          const int64_t m = m0 + row;
          const bool here = m < a.M && n < a.N;
          float v = *reinterpret_cast<const float*>(s + stage_at(row, c / 4) + c % 4 * 4), u = 0.f;
          if (EPI == EPI_GATED) u = *reinterpret_cast<const float*>(s + stage_at(row, U + c / 4) + c % 4 * 4);
          if (EPI != EPI_PLAIN) {
            v += bv[0];
            if (EPI == EPI_GATED) u += bu[0];
            if (a.z && here) {
              st_from_f32(static_cast<T*>(a.z) + m * a.Z + n, v);
              if (EPI == EPI_GATED) st_from_f32(static_cast<T*>(a.z) + m * a.Z + a.half + n, u);
            }
            v = activate<F32>(EPI == EPI_GATED ? SA_ACT_SWIGLU : a.act, v);
            if (EPI == EPI_GATED) v *= u;
            v += rv[k];
          }
          if (here) st_from_f32(static_cast<T*>(a.y) + m * a.N + n, v);
        }
      }
    }
  }
};

// 16 columns of 32 lanes' accumulators (see ptx::tmem_ld32)
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float* v) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, "
      "[%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}

// The end of bf16 chunks whose rows TMA can write: each lane keeps its row's 32 columns in registers to the end, and
// a chunk's 32 x 32 results (z, SwiGLU's other half of z, y) leave together from the warp's buffers (64-byte rows, TMA's
// 64-byte swizzle).  That takes a third of the shared-memory traffic of the way above.
constexpr int kOutBytes = 2048;
template <int EPI, int SETS>
struct TmaOut {
  static constexpr int SET = EPI == EPI_GATED ? 3 : EPI == EPI_FULL ? 2 : 1;  // results of a chunk
  static constexpr int BUFFERS = SETS * SET;  // sets in turn (unaligned rows' stage is as long as two buffers)
  char* ring;
  int lane, turn;
  float b0, b1;

  __device__ __forceinline__ TmaOut(char* ring_, int lane_) : ring(ring_), lane(lane_), turn(0) {}

  __device__ __forceinline__ void load_bias(const TcArgs& a, int n0) {
    b0 = b1 = 0.f;
    if (EPI == EPI_PLAIN || !a.bias || n0 + lane >= a.N) return;
    const __nv_bfloat16* b = static_cast<const __nv_bfloat16*>(a.bias) + n0 + lane;
    b0 = ld_nc(b);
    if (EPI == EPI_GATED) b1 = ld_nc(b + a.half);
  }
  __device__ __forceinline__ static uint32_t at(int row, int p) { return row * 64 + ((p ^ ((row >> 1) & 3)) << 4); }
  __device__ __forceinline__ void put(char* s, const float* v) const {
#pragma unroll
    for (int p = 0; p < 4; ++p) store8(reinterpret_cast<__nv_bfloat16*>(s + at(lane, p)), v + 8 * p);
  }

  // `acc`: this lane's accumulators of the chunk, SwiGLU's other half at `other`; read() is called once they are read.
  template <class F>
  __device__ __forceinline__ void finish(const TcArgs& a, const CUtensorMap& ty, const CUtensorMap& tz, uint32_t acc,
                                         uint32_t other, int64_t m0, int n0, F read) {
    float v[32];
    ptx::tmem_ld32(acc, v);
    // this set, once the stores of its last chunk have read it
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(SETS - 1) : "memory");
    char* s = ring + (SETS == 2 ? turn ^= 1 : 0) * SET * kOutBytes;  // y, then z's halves
    uint4 res[EPI == EPI_FULL ? 4 : 1];
    const bool direct = EPI != EPI_PLAIN && a.r && (a.vec & 2);
    auto load_residual = [&](uint4* q) {  // whole rows a few lanes
      const int n = n0 + lane % 4 * 8;
      const __nv_bfloat16* r = static_cast<const __nv_bfloat16*>(a.r) + n;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t m = m0 + i * 8 + lane / 4;
        q[i] = make_uint4(0, 0, 0, 0);
        if (m < a.M && n < a.N) q[i] = __ldg(reinterpret_cast<const uint4*>(r + m * a.r_stride));
      }
    };
    if constexpr (EPI == EPI_FULL) {
      if (direct) load_residual(res);  // on its way meanwhile
    }
    __syncwarp();
    // y's buffer holds the biases until y itself
    float* bias = reinterpret_cast<float*>(s);
    auto add_bias = [&](const float* from, float* to, int count) {
#pragma unroll
      for (int j = 0; j < count; j += 4) {
        const float4 b = *reinterpret_cast<const float4*>(from + j);
        const float2 p = __fadd2_rn(make_float2(to[j], to[j + 1]), make_float2(b.x, b.y));
        const float2 q = __fadd2_rn(make_float2(to[j + 2], to[j + 3]), make_float2(b.z, b.w));
        to[j] = p.x, to[j + 1] = p.y, to[j + 2] = q.x, to[j + 3] = q.y;
      }
    };
    if (EPI != EPI_PLAIN && a.bias) {
      bias[lane] = b0;
      if (EPI == EPI_GATED) bias[32 + lane] = b1;
      __syncwarp();
    }
    ptx::tmem_ld_wait();
    if (EPI != EPI_GATED) read();
    float u[EPI == EPI_GATED ? 32 : 1];
    if constexpr (EPI == EPI_GATED) ptx::tmem_ld32(other, u);  // the other half, on its way meanwhile
    if (EPI != EPI_PLAIN) {
      if (a.bias) add_bias(bias, v, 32);
      if (a.z) put(s + kOutBytes, v);
    }
    if constexpr (EPI == EPI_GATED) {
#pragma unroll
      for (int j = 0; j < 32; j += 2) silu_pair(v + j);
      ptx::tmem_ld_wait();
      read();
      if (a.bias) add_bias(bias + 32, u, 32);
      if (a.z) put(s + 2 * kOutBytes, u);
#pragma unroll
      for (int j = 0; j < 32; j += 2) {
        const float2 p = __fmul2_rn(make_float2(v[j], v[j + 1]), make_float2(u[j], u[j + 1]));
        v[j] = p.x, v[j + 1] = p.y;
      }
    }
    if constexpr (EPI == EPI_FULL) {
      if (a.act == SA_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = activate<false>(SA_ACT_RELU, v[j]);
      } else if (a.act == SA_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < 32; j += 2) gelu_pair(v + j);
      } else if (a.act == SA_ACT_SILU) {
#pragma unroll
        for (int j = 0; j < 32; j += 2) silu_pair(v + j);
      }
    }
    if (EPI != EPI_PLAIN) {
      if (a.bias) __syncwarp();  // the biases are read
      if (a.r) {
        if (direct) {
          uint4 late[4];
          if constexpr (EPI == EPI_GATED) load_residual(late);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *reinterpret_cast<uint4*>(s + at(i * 8 + lane / 4, lane % 4)) = EPI == EPI_FULL ? res[EPI == EPI_FULL ? i : 0] : late[i];
        } else {
          const __nv_bfloat16* r = static_cast<const __nv_bfloat16*>(a.r) + n0 + lane;
#pragma unroll 8
          for (int i = 0; i < 32; ++i)
            *reinterpret_cast<__nv_bfloat16*>(s + at(i, lane / 8) + lane % 8 * 2) =
                __float2bfloat16_rn(m0 + i < a.M && n0 + lane < a.N ? ld_nc(r + (m0 + i) * a.r_stride) : 0.f);
        }
        __syncwarp();
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          float w[8];
          load8(reinterpret_cast<const __nv_bfloat16*>(s + at(lane, p)), w);
#pragma unroll
          for (int j = 0; j < 8; ++j) v[8 * p + j] += w[j];
        }
      }
    }
    put(s, v);  // over the residual: each lane its own row
    ptx::fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      if (m0 < a.M && n0 < a.N) {
        if (EPI != EPI_PLAIN && a.z) {
          ptx::tma_store_3d(&tz, ptx::smem_u32(s + kOutBytes), n0, 0, int(m0));
          if (EPI == EPI_GATED) ptx::tma_store_3d(&tz, ptx::smem_u32(s + 2 * kOutBytes), n0, 1, int(m0));
        }
        ptx::tma_store_3d(&ty, ptx::smem_u32(s), n0, 0, int(m0));
      }
      ptx::bulk_commit_group();  // an empty group counts too
    }
  }
  __device__ __forceinline__ void done() const {
    if (lane == 0) ptx::bulk_wait_all();
  }
};

}  // namespace dense
}  // namespace sa
