// Products of the linear layers on tcgen05 (include/sa_dense.h): y = act(x W^T + b) + r, dx = dz W,
// dW = dz^T x, one kernel for the three with operands in either order (K-major or MN-major tiles, so
// nothing is transposed in memory).
//
// A tile is 256 x 256 for a pair of CTAs (cta_group::2: each holds 128 rows of A, half of B's rows and
// 128 rows of the result) or 128 x 128 for one CTA.  One warp loads (TMA, 64 deep blocks, up to five stages), one issues the
// products, and the others end tiles, 32 x 32 results at a time, while the next tile's products go to another set of
// accumulators in TMEM.  A pair's CTA has eight of them, each with its part of every tile, and two sets.  A single CTA,
// whose tiles have few products an element, has twelve with 152 registers, in three groups that take the chunks of all tiles
// in turn, and three sets (65536 x 128 -> 512, eight warps and twelve: gated 44 and 40 us, silu 42 and 36, none 31 and 26;
// without more registers for them 45, from spills).  SwiGLU's tile takes the same columns of both halves of W, so gate
// and value meet in one warp.
//
// 8192 x 4096 -> 4096 with a residual: 159 us alone, 1.73 PFLOP/s, tensor pipe 82 % busy (six and three quarters waves of
// pairs); 16384 x 4096 gated, dx and dW: 297 us, 1.85 PFLOP/s.  65536 x 128 -> 512 gated with z: 38 us (5.7 TB/s), of which
// loads and products alone would take 28 and barriers alone 20.
//
// Work: tiles go to the workers (one CTA or pair an SM or two) in turn.  Where the last turn would leave many idle, its
// tiles are dealt out in equal shares of blocks instead; a tile cut by shares leaves fp32 pieces that a second
// kernel adds in worker order and ends, so results do not depend on timing.
//
// fp32 operands come as three bf16 terms each, and six of the nine products of terms are made.  The tensor
// core's sums lose about a step of fp32 an addition, always towards zero (1024 x 1024 sums of 1024 products were
// 6.5e-6 off with eight blocks in a row), so each block starts with its small products, and its
// accumulators are added to sums in registers, which round to nearest.
// bf16 sums lose as much: 200,003 products of one sign came out 7.3e-4 too small.  So a tile's blocks go in runs of at most
// kRun, and the runs' sums are added in memory, in fp32 (a worker's own cells, which L2 holds): a run loses 6e-5, a sixtieth of
// the largest rounding of a result, and its 68 us of products hide the 256 KB each way.
#include "sa_dense_tc.cuh"

#include <cmath>
#include <mutex>

#include "sa_tc_common.cuh"

namespace sa {
namespace dense {
namespace {

using namespace ptx;

constexpr int kBlockBytes = 16384;  // 128 rows x 64 bf16
// What a worker that gave up allows its own copies and products in flight, each.
constexpr uint64_t kDrainNs = 200000000ull;

template <int CTAS, bool F32, int EPI>
struct TcCfg {
  using T = typename std::conditional<F32, float, __nv_bfloat16>::type;
  using End = ChunkEnd<T, EPI>;
  // three groups of epilogue warps take the chunks in turn (else two, each with its half of a tile's columns)
  static constexpr bool POOL = CTAS == 1 && !F32;
  static constexpr int GROUPS = POOL ? 3 : TileShape<CTAS>::GROUPS;
  static constexpr int SETS = POOL ? 3 : 2;      // of accumulators
  static constexpr int EPI0 = POOL ? 0 : 4;      // the first epilogue warp
  static constexpr int LOAD = POOL ? 12 : 0;     // the warp that loads, before the one that issues the products
  static constexpr int ALLOC = POOL ? 12 : 2;
  static constexpr int PLANES = F32 ? 3 : 1;
  static constexpr int STAGE = 2 * PLANES * kBlockBytes;
  static constexpr int OUT_SETS = POOL && EPI != EPI_PLAIN ? 1 : 2;
  static constexpr int OUT = F32 ? kStageBytes : TmaOut<EPI, OUT_SETS>::BUFFERS * kOutBytes;  // of an epilogue warp
  static constexpr int STAGES = F32 ? 2 : EPI == EPI_GATED || (POOL && EPI == EPI_FULL) ? 4 : 5;  // (five measured the same there)
  static constexpr int BN = TileShape<CTAS>::BN;
  static constexpr int WARPS = 4 * GROUPS;  // that end tiles
  static constexpr int THREADS = 32 * WARPS + 128;
  static constexpr int TMEM = POOL ? 512 : 2 * BN;  // a power of two
  static constexpr int OFF_OUT = STAGES * STAGE;
  static constexpr int OFF_BAR = OFF_OUT + WARPS * OUT;
  static constexpr int SMEM = OFF_BAR + 256;
};
static_assert(TcCfg<2, false, EPI_GATED>::SMEM <= 232448 && TcCfg<2, false, EPI_FULL>::SMEM <= 232448 &&
                  TcCfg<1, true, EPI_GATED>::SMEM <= 232448 && TcCfg<1, false, EPI_GATED>::SMEM <= 232448 &&
                  TcCfg<1, false, EPI_FULL>::SMEM <= 232448 && TcCfg<1, false, EPI_PLAIN>::SMEM <= 232448,
              "shared memory of a CTA");

// ------------------------------------------------------ cta_group::2 forms
template <int CTAS>
__device__ __forceinline__ void tc_alloc(uint32_t dst, uint32_t cols) {
  if (CTAS == 1) {
    tmem_alloc(dst, cols);
  } else {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
}
template <int CTAS>
__device__ __forceinline__ void tc_dealloc(uint32_t t, uint32_t cols) {
  if (CTAS == 1)
    tmem_dealloc(t, cols);
  else
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(t), "r"(cols) : "memory");
}
template <int CTAS>
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if (CTAS == 1)
    umma_ss(d, a, b, idesc, accumulate);
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate));
}
// arrives on the barrier at this offset in every CTA of the worker
template <int CTAS>
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  if (CTAS == 1)
    umma_commit(bar);
  else
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
        "h"(uint16_t(3))
        : "memory");
}
// a word of the first CTA's or the other CTA's shared memory (a shared::cluster address)
__device__ __forceinline__ void st_cluster_u32(uint32_t addr_cl, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr_cl), "r"(v) : "memory");
}
// takes `bytes` off what a barrier of this CTA still expects
__device__ __forceinline__ void mbar_complete_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// `bar` is the first CTA's barrier (a shared::cluster address)
template <int CTAS>
__device__ __forceinline__ void tc_load(uint32_t dst, const void* map, uint32_t bar, int c0, int c1, int c2) {
  if (CTAS == 1)
    tma_load_3d(dst, map, bar, c0, c1, c2);
  else
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2)
        : "memory");
}

// The work of one CTA.  Maps: K-major operands [planes][rows][k], boxes of 64 x (A: 128, B: 64) rows; MN-major ones
// [planes][k][mn], boxes of 64 x 64.
// LONG: a tile may take several runs.
template <int CTAS, bool A_MN, bool B_MN, bool F32, int EPI, bool LONG>
__device__ __forceinline__ void tc_linear_work(const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& ty,
                                               const CUtensorMap& tz, const TcArgs& a, const int worker,
                                               const bool clear) {
  using C = TcCfg<CTAS, F32, EPI>;
  using End = typename C::End;
  using Shape = TileShape<CTAS>;
  constexpr int YN = Shape::template YN<EPI>;
  extern __shared__ __align__(1024) char smem[];
  const uint32_t base = smem_u32(smem);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CTAS == 2 ? cluster_rank() : 0;

  auto full = [&](int s) { return base + C::OFF_BAR + 8 * s; };
  auto empty = [&](int s) { return base + C::OFF_BAR + 64 + 8 * s; };
  auto acc_full = [&](int s) { return base + C::OFF_BAR + 128 + 8 * s; };
  auto acc_empty = [&](int s) { return base + C::OFF_BAR + 192 + 8 * s; };
  const uint32_t drain = base + C::OFF_BAR + 216, never = base + C::OFF_BAR + 224;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::OFF_BAR + 160);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::OFF_BAR + 176);  // three words
  // in the first CTA: blocks that each CTA of the worker has asked for, once its loads are done
  volatile uint32_t* loads = reinterpret_cast<volatile uint32_t*>(smem + C::OFF_BAR + 232);

  if (threadIdx.x == 0) {
    if (clear) {
      ws_header(a.ws)->err = 0;
      ws_header(a.ws)->timeout_site = 0;
    }
    for (int s = 0; s < C::STAGES; ++s) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), 1);
    }
    for (int s = 0; s < C::SETS; ++s) {
      mbar_init(acc_full(s), 1);
      mbar_init(acc_empty(s), C::WARPS * CTAS);
    }
    mbar_init(drain, 1);
    mbar_init(never, 1);
    abort_flag[0] = 0;
    reinterpret_cast<volatile uint32_t*>(abort_flag)[2] = a.wait_ns;
    fence_mbar_init();
    tma_prefetch_desc(&ta);
    tma_prefetch_desc(&tb);
  }
  if (warp == C::ALLOC) tc_alloc<CTAS>(smem_u32(tmem_slot), C::TMEM);
  tc_fence_before();
  if (CTAS == 2)
    cluster_sync_all();
  else
    __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  // a role that gave up: the pair's other CTA stops too
  auto gave_up = [&] {
    if (CTAS == 2) st_cluster_u32(mapa_shared(smem_u32(const_cast<int*>(abort_flag)), rank ^ 1u), 1u);
  };
  if (warp >= C::EPI0 && warp < C::EPI0 + C::WARPS) {
    // of the launch's 512 x 128 registers: 384 x 152 here, 128 x 56 there
    if constexpr (C::POOL) setmaxnreg_inc<152>();
    // -------------------------------------------------------- tiles' ends
    const int e = warp - C::EPI0, q = e & 3, h = e >> 2;
    char* out = smem + C::OFF_OUT + e * C::OUT;
    const uint32_t lanes = uint32_t(q * 32) << 16;
    const uint32_t lead_empty = CTAS == 2 ? mapa_shared(acc_empty(0), 0) : acc_empty(0);
    constexpr int CH = C::POOL ? YN / 32 : Shape::template CHUNKS<EPI>;
    TmaOut<EPI, C::OUT_SETS> outs(out, lane);
    Segments seg(a, worker);
    uint32_t g = 0, tiles = 0;  // sets of accumulators used, tiles
    bool ok = true;
    auto release = [&](uint32_t set) {
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        // relaxed: only the accumulators' reads come before it, and a release would wait for this warp's stores
        if (CTAS == 2)
          mbar_arrive_relaxed_cluster(lead_empty + 8 * set);
        else
          mbar_arrive(acc_empty(set));
      }
    };
    for (; ok && seg.next(); ++tiles) {
      // this warp's chunks: of a pool every third of all tiles' chunks, else half of each tile's
      constexpr int STEP = C::POOL ? 3 : 1;
      const int first = C::POOL ? (h + int(tiles % 3) * (3 - CH % 3)) % 3 : h * CH, stop = C::POOL ? CH : first + CH;
      int mb, nb;
      tile_place(a, seg.tile, &mb, &nb);
      const int64_t m0 = int64_t(mb * CTAS + int(rank)) * 128 + q * 32;
      const bool complete = seg.complete();
      float* piece = nullptr;
      if (!complete) {
        const int64_t total = a.cut * a.KB, first = (seg.tile - a.whole) * a.KB;
        const int slot = partial_slot(total, a.cutters, worker, first);
        piece = a.piece + (int64_t(worker * 2 + slot) * CTAS + rank) * (128 * C::BN) + (q * 32 + lane) * 4;
      }
      auto col = [&](int i, int half) {  // accumulator column of chunk i (SwiGLU: of either half)
        return half * YN + i * 32;
      };
      auto put_piece = [&](int c, const float* v) {
        if (m0 + lane < a.M)
#pragma unroll
          for (int j = 0; j < 8; ++j)
            *reinterpret_cast<float4*>(piece + int64_t(c / 4 + j) * 512) =
                make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
      };
      End end;
      const int y0 = nb * YN;
      if constexpr (F32) {
        constexpr int HALVES = EPI == EPI_GATED ? 2 : 1;
        float sum[CH][HALVES][32];
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
          for (int k = 0; k < HALVES; ++k)
#pragma unroll
            for (int j = 0; j < 32; ++j) sum[i][k][j] = 0.f;
        for (int kb = seg.k0; kb < seg.k1; ++kb) {
          const uint32_t set = g & 1u;
          ok = __all_sync(0xFFFFFFFFu, mbar_wait(acc_full(set), (g >> 1) & 1u, abort_flag, a.ws, 0x404));
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int k = 0; k < HALVES; ++k) {
              float v[32];
              tmem_ld32(tmem + lanes + set * C::BN + col(first + i, k), v);
              tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 32; ++j) sum[i][k][j] += v[j];
            }
          release(set);
          ++g;
        }
        if (!ok) break;
        if (complete) {
          // all chunks pass through one copy of their end, so the registers they are in are chosen by selects
#pragma unroll 1
          for (int i = 0; i < CH * 32 / End::COLS; ++i) {
            const int n0 = y0 + first * 32 + i * End::COLS;
            if (n0 >= a.N || m0 >= a.M) break;
            end.load_bias(a, lane, n0);
#pragma unroll
            for (int k = 0; k < CH * 32 / End::COLS; ++k)
              if (k == i) {
                stage_put<End::COLS>(out, lane, &sum[k * End::COLS / 32][0][k * End::COLS % 32]);
                if (EPI == EPI_GATED)
                  stage_put<End::COLS>(out, lane, &sum[k * End::COLS / 32][HALVES - 1][k * End::COLS % 32], End::U);
              }
            __syncwarp();
            end.template finish<1>(a, out, lane, m0, n0, 0);
            __syncwarp();
          }
        } else {
#pragma unroll
          for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int k = 0; k < HALVES; ++k) put_piece(col(first + i, k), sum[i][k]);
        }
      } else {
        // the sums of the runs so far: this thread's cells of chunk i
        auto sums_of = [&](int i, int k) {
          return a.sums + (int64_t(worker) * CTAS + rank) * (128 * C::BN) + (q * 32 + lane) * 4 + int64_t(col(i, k) / 4) * 512;
        };
        auto add_sums = [&](const float* p, float* v) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float4 f = *reinterpret_cast<const float4*>(p + j * 512);
            v[4 * j] += f.x, v[4 * j + 1] += f.y, v[4 * j + 2] += f.z, v[4 * j + 3] += f.w;
          }
        };
        constexpr int HALVES = EPI == EPI_GATED ? 2 : 1;
        int kb = seg.k0;
        for (; LONG && seg.k1 - kb > kRun; kb += kRun, ++g) {  // runs before a tile's last
          const uint32_t set = g % C::SETS, acc = tmem + lanes + set * C::BN;
          ok = __all_sync(0xFFFFFFFFu, mbar_wait(acc_full(set), g / C::SETS & 1u, abort_flag, a.ws, 0x405));
          if (!ok) break;
          tc_fence_after();
#pragma unroll 1
          for (int i = first; i < stop; i += STEP)
#pragma unroll 1
            for (int k = 0; k < HALVES; ++k) {
              float v[32];
              float* p = sums_of(i, k);
              tmem_ld32(acc + col(i, k), v);
              tmem_ld_wait();
              if (kb != seg.k0) add_sums(p, v);
#pragma unroll
              for (int j = 0; j < 8; ++j)
                *reinterpret_cast<float4*>(p + j * 512) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
            }
          release(set);
        }
        if (!ok) break;
        const bool tma = (a.vec & 1) != 0;
        if (complete && tma && first < stop) outs.load_bias(a, y0 + first * 32);
        const uint32_t set = g % C::SETS, acc = tmem + lanes + set * C::BN;
        ok = __all_sync(0xFFFFFFFFu, mbar_wait(acc_full(set), g / C::SETS & 1u, abort_flag, a.ws, 0x404));
        if (!ok) break;
        tc_fence_after();
        if (LONG && kb != seg.k0) {  // the last run's accumulators become the tile's sums
#pragma unroll 1
          for (int i = first; i < stop; i += STEP)
#pragma unroll 1
            for (int k = 0; k < HALVES; ++k) {
              float v[32];
              tmem_ld32(acc + col(i, k), v);
              tmem_ld_wait();
              add_sums(sums_of(i, k), v);
              tmem_st16(acc + col(i, k), reinterpret_cast<const uint32_t*>(v));
              tmem_st16(acc + col(i, k) + 16, reinterpret_cast<const uint32_t*>(v) + 16);
            }
          tmem_st_wait();
        }
        if (C::POOL && first >= stop) release(set);
#pragma unroll 1
        for (int i = first; i < stop; i += STEP) {
          auto read = [&] {
            if (i + STEP >= stop) release(set);
          };
          if (y0 + i * 32 >= a.N || m0 >= a.M) {  // nothing of it is in y
            read();
          } else if (complete && tma) {
            outs.finish(a, ty, tz, acc + col(i, 0), acc + col(i, 1), m0, y0 + i * 32, read);
            if (i + STEP < stop) outs.load_bias(a, y0 + (i + STEP) * 32);
          } else if (complete) {
#pragma unroll 1
            for (int k = 0; k < 2; ++k) {  // by 16 columns
              float v[16];
              const int n0 = y0 + i * 32 + k * 16;
              tmem_ld16(acc + col(i, 0) + k * 16, v);
              tmem_ld_wait();
              stage_put<16>(out, lane, v, End::COLS == 32 ? 4 * k : 0);
              if (EPI == EPI_GATED) {
                tmem_ld16(acc + col(i, 1) + k * 16, v);
                tmem_ld_wait();
                stage_put<16>(out, lane, v, End::U);
              }
              if (k == 1) read();
              if (End::COLS == 32 && k == 0) continue;
              __syncwarp();
              end.load_bias(a, lane, End::COLS == 32 ? y0 + i * 32 : n0);
              end.template finish<1>(a, out, lane, m0, End::COLS == 32 ? y0 + i * 32 : n0, 0);
              __syncwarp();
            }
          } else {
#pragma unroll 1
            for (int k = 0; k < (EPI == EPI_GATED ? 2 : 1); ++k) {
              float v[32];
              tmem_ld32(acc + col(i, k), v);
              tmem_ld_wait();
              put_piece(col(i, k), v);
            }
            read();
          }
        }
        ++g;
      }
    }
    if (!F32) outs.done();
    if (!ok && lane == 0) gave_up();
  } else {
    if constexpr (C::POOL) setmaxnreg_dec<56>();
    if (warp == C::LOAD && lane == 0) {
      // ------------------------------------------------------------- loads
      const uint32_t lead = CTAS == 2 ? mapa_shared(base, 0) : base;
      Segments seg(a, worker);
      uint32_t n = 0;  // blocks loaded
      bool ok = true;
      while (ok && seg.next()) {
        int mb, nb;
        tile_place(a, seg.tile, &mb, &nb);
        const int m0 = (mb * CTAS + int(rank)) * 128;
        // this CTA's 128 rows of B: SwiGLU's halves are the pair's CTAs, or 64 rows each
        int b0, b1;
        if (EPI == EPI_GATED) {
          b0 = CTAS == 2 ? int(rank * a.half) + nb * YN : nb * YN;
          b1 = CTAS == 2 ? b0 + 64 : int(a.half) + nb * YN;
        } else {
          b0 = nb * YN + (CTAS == 2 ? int(rank) * 128 : 0);
          b1 = b0 + 64;
        }
        for (int kb = seg.k0; kb < seg.k1; ++kb, ++n) {
          const uint32_t s = n % C::STAGES, ph = (n / C::STAGES) & 1u;
          ok = mbar_wait(empty(s), ph ^ 1u, abort_flag, a.ws, 0x401);
          if (!ok) break;
          if (rank == 0) mbar_arrive_expect_tx(full(s), CTAS * C::STAGE);
          const uint32_t bar = lead + C::OFF_BAR + 8 * s, dst = base + s * C::STAGE;
          const int k = kb * 64;
  #pragma unroll
          for (int p = 0; p < C::PLANES; ++p) {
            const uint32_t da = dst + p * kBlockBytes, db = dst + (C::PLANES + p) * kBlockBytes;
            if (A_MN) {
              tc_load<CTAS>(da, &ta, bar, m0, k, p);
              tc_load<CTAS>(da + 8192, &ta, bar, m0 + 64, k, p);
            } else {
              tc_load<CTAS>(da, &ta, bar, k, m0, p);
            }
            if (B_MN) {
              tc_load<CTAS>(db, &tb, bar, b0, k, p);
              tc_load<CTAS>(db + 8192, &tb, bar, b1, k, p);
            } else {
              tc_load<CTAS>(db, &tb, bar, k, b0, p);
              tc_load<CTAS>(db + 8192, &tb, bar, k, b1, p);
            }
          }
        }
      }
      if (CTAS == 2)
        st_cluster_u32(lead + C::OFF_BAR + 232 + 4 * rank, n);
      else
        loads[0] = n;
      if (!ok) gave_up();
    } else if (warp == C::LOAD + 1 && lane == 0 && rank == 0) {
      // ---------------------------------------------------------- products
      constexpr uint32_t idesc = idesc_bf16(128 * CTAS, C::BN, A_MN, B_MN);
      constexpr uint32_t step_a = A_MN ? 2048 : 32, step_b = B_MN ? 2048 : 32;
      const uint64_t d_a = sdesc(base, A_MN ? 8192 : 16, 1024);
      const uint64_t d_b = sdesc(base + C::PLANES * kBlockBytes, B_MN ? 8192 : 16, 1024);
      Segments seg(a, worker);
      uint32_t n = 0, g = 0;  // blocks, sets of accumulators used
      // under a test limit (sa_set_wait_limit_ns) the first wait is for a barrier that nothing completes
      bool ok = a.wait_ns >= kPollLimitNs || mbar_wait(never, 0, abort_flag, a.ws, 0x400);
      while (ok && seg.next()) {
        for (int kb = seg.k0; ok && kb < seg.k1;) {
          const int end = F32 ? kb + 1 : LONG && seg.k1 - kb > kRun ? kb + kRun : seg.k1;
          const uint32_t set = g % C::SETS, d = tmem + set * C::BN;
          ok = mbar_wait(acc_empty(set), (g / C::SETS & 1u) ^ 1u, abort_flag, a.ws, 0x402);
          if (!ok) break;
          tc_fence_after();
          uint32_t accumulate = 0;
          for (; kb < end; ++kb, ++n) {
            const uint32_t s = n % C::STAGES;
            ok = mbar_wait(full(s), (n / C::STAGES) & 1u, abort_flag, a.ws, 0x403);
            if (!ok) break;
            tc_fence_after();
            const uint64_t sa = sdesc_add(d_a, s * C::STAGE), sb = sdesc_add(d_b, s * C::STAGE);
            constexpr int pa[6] = {2, 1, 0, 1, 0, 0}, pb[6] = {0, 1, 2, 0, 1, 0};
  #pragma unroll
            for (int i = F32 ? 0 : 5; i < 6; ++i)
  #pragma unroll
              for (int k = 0; k < 4; ++k) {
                tc_mma<CTAS>(d, sdesc_add(sa, pa[i] * kBlockBytes + k * step_a),
                             sdesc_add(sb, pb[i] * kBlockBytes + k * step_b), idesc, accumulate);
                accumulate = 1;
              }
            tc_commit<CTAS>(empty(s));
          }
          if (!ok) break;
          tc_commit<CTAS>(acc_full(set));
          ++g;
        }
      }
      if (!ok) gave_up();
    }
  }
  __syncwarp();
  auto meet = [&] {
    if (CTAS == 2)
      cluster_sync_all();
    else
      __syncthreads();
  };
  meet();  // nothing of the worker's is still read or written, unless a role gave up
  if (abort_flag[0]) {  // the same for all of the worker's threads: no role is left to set it
    // whichever role gave up, copies and products may be in flight: they end before the CTA and its TMEM do
    if (warp == C::LOAD + 1 && lane == 0) {
      if (rank == 0) tc_commit<CTAS>(drain);  // the thread that issued the products
      tcc::mbar_wait_bounded(drain, 0, kDrainNs);
    }
    if (warp == C::LOAD && lane == 0 && rank == 0) {
      const uint32_t n0 = loads[0], n1 = CTAS == 2 ? loads[1] : n0, n = n0 > n1 ? n0 : n1;
      for (uint32_t i = n > C::STAGES ? n - C::STAGES : 0; i < n; ++i) {
        const uint32_t bar = full(i % C::STAGES);
        if (i >= n0)
          mbar_arrive_expect_tx(bar, C::STAGE);  // the second CTA's copies alone
        else if (i >= n1)
          mbar_complete_tx(bar, C::STAGE);  // the first CTA's alone: the others were expected, and do not come
        tcc::mbar_wait_bounded(bar, (i / C::STAGES) & 1u, kDrainNs);
      }
    }
    __syncwarp();
    meet();
  }
  if (warp == C::ALLOC) {
    tc_fence_after();
    tc_dealloc<CTAS>(tmem, C::TMEM);
  }
  if (CTAS == 2) cluster_sync_all();
}

template <int CTAS, bool A_MN, bool B_MN, bool F32, int EPI, bool LONG>
__global__ void __launch_bounds__(TcCfg<CTAS, F32, EPI>::THREADS, 1)
    tc_linear_kernel(const __grid_constant__ CUtensorMap ta, const __grid_constant__ CUtensorMap tb,
                     const __grid_constant__ CUtensorMap ty, const __grid_constant__ CUtensorMap tz, const TcArgs a) {
  tc_linear_work<CTAS, A_MN, B_MN, F32, EPI, LONG>(ta, tb, ty, tz, a, int(blockIdx.x) / CTAS, a.clear && blockIdx.x == 0);
}

// dx and dW side by side, for gradients that would leave most of the GPU idle one after the other: the first
// x.W CTAs (or pairs) make dx.
template <int CTAS, bool F32, bool LONG>
__global__ void __launch_bounds__(TcCfg<CTAS, F32, EPI_PLAIN>::THREADS, 1)
    tc_linear_grads_kernel(const __grid_constant__ CUtensorMap xa, const __grid_constant__ CUtensorMap xb,
                           const __grid_constant__ CUtensorMap wa, const __grid_constant__ CUtensorMap wb,
                           const __grid_constant__ CUtensorMap xy, const __grid_constant__ CUtensorMap wy, const TcArgs x,
                           const TcArgs w) {
  const int worker = int(blockIdx.x) / CTAS;
  if (worker < x.W)
    tc_linear_work<CTAS, false, true, F32, EPI_PLAIN, LONG>(xa, xb, xy, xy, x, worker, blockIdx.x == 0);
  else
    tc_linear_work<CTAS, true, true, F32, EPI_PLAIN, LONG>(wa, wb, wy, wy, w, worker - x.W, false);
}

// Cut tiles: a block of 16 warps ends 128 rows x 32 columns of y.  Warp (q, part) adds the pieces of the rows of q and eight
// columns (SwiGLU: of both halves), in worker order, and after they have met in shared memory ends eight rows of q.
constexpr int kJoinThreads = 512;
template <int CTAS, bool F32, int EPI>
__device__ __forceinline__ void tc_join_work(const TcArgs& a, const int block) {
  using C = TcCfg<CTAS, F32, EPI>;
  using End = typename C::End;
  using Shape = TileShape<CTAS>;
  constexpr int YN = Shape::template YN<EPI>, CH = YN / 32;
  constexpr int HALVES = EPI == EPI_GATED ? 2 : 1;
  extern __shared__ __align__(128) char stages[];  // [4][32 / COLS][kStageBytes]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, q = warp & 3, part = warp >> 2;
  const int i = block % CH, rank = block / CH % CTAS;
  const int64_t rest = block / (CH * CTAS);
  const int64_t total = a.cut * a.KB, first = rest * a.KB, last = first + a.KB - 1;
  const int w0 = owner_of(total, a.cutters, first), w1 = owner_of(total, a.cutters, last);
  if (w0 == w1) return;  // its worker ended it
  if (ws_failed(a.ws)) return;  // a worker gave up: its pieces are not there (asked later, it cost a register and 1 us)
  int mb, nb;
  tile_place(a, a.whole + rest, &mb, &nb);
  const int64_t m0 = int64_t(mb * CTAS + rank) * 128 + q * 32;
  const int n0 = nb * YN + i * 32;
  if (m0 - q * 32 >= a.M || n0 >= a.N) return;
  End end;
  end.load_bias(a, lane, n0);
  const int64_t piece = int64_t(CTAS) * 128 * C::BN;
  // every worker between has a piece (none has an empty share), in its first slot but for the first, whose share may
  // begin before the tile
  const float* p0 = a.piece + int64_t(rank) * 128 * C::BN + (q * 32 + lane) * 4;
  char* out = stages + q * HALVES * kStageBytes;
#pragma unroll
  for (int k = 0; k < HALVES; ++k) {
    const int c = (EPI == EPI_GATED ? k * YN : 0) + i * 32 + part * 8;
    float4 x[2] = {make_float4(0, 0, 0, 0), make_float4(0, 0, 0, 0)};
    if (m0 + lane < a.M) {
      auto add = [&](const float4* f) {
#pragma unroll
        for (int j = 0; j < 2; ++j) x[j].x += f[j].x, x[j].y += f[j].y, x[j].z += f[j].z, x[j].w += f[j].w;
      };
      auto read = [&](int w, float4* f) {
        const int slot = w == w0 ? partial_slot(total, a.cutters, w0, first) : 0;
        const float* p = p0 + (int64_t(w) * 2 + slot) * piece + int64_t(c / 4) * 512;
        f[0] = *reinterpret_cast<const float4*>(p);
        f[1] = *reinterpret_cast<const float4*>(p + 512);
      };
      int w = w0;
      for (; w + 3 <= w1; w += 4) {  // four pieces in flight
        float4 f[4][2];
#pragma unroll
        for (int l = 0; l < 4; ++l) read(w + l, f[l]);
#pragma unroll
        for (int l = 0; l < 4; ++l) add(f[l]);
      }
      float4 f[3][2];
#pragma unroll
      for (int l = 0; l < 3; ++l)
        if (w + l <= w1) read(w + l, f[l]);
#pragma unroll
      for (int l = 0; l < 3; ++l)
        if (w + l <= w1) add(f[l]);
    }
    const float v[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
    if constexpr (End::COLS == 32)
      stage_put<8>(out, lane, v, part * 2);
    else  // columns 0-15 of both halves in one stage, 16-31 in the next
      stage_put<8>(out + (part >> 1) * kStageBytes, lane, v, k * End::U + (part & 1) * 2);
  }
  __syncthreads();
#pragma unroll 1
  for (int k = 0; k < 32 / End::COLS; ++k) {
    if (k) end.load_bias(a, lane, n0 + k * End::COLS);
    end.template finish<4>(a, out + k * kStageBytes, lane, m0, n0 + k * End::COLS, part);
  }
}

template <int CTAS, bool F32, int EPI>
__global__ void __launch_bounds__(kJoinThreads, EPI == EPI_GATED ? 1 : 2) tc_join_kernel(const TcArgs a) {
  tc_join_work<CTAS, F32, EPI>(a, blockIdx.x);
}

// dx's cut tiles in the first `split` blocks, dW's in the rest
template <int CTAS, bool F32>
__global__ void __launch_bounds__(kJoinThreads, 2) tc_join_grads_kernel(const TcArgs x, const TcArgs w, const int split) {
  const bool second = int(blockIdx.x) >= split;
  tc_join_work<CTAS, F32, EPI_PLAIN>(second ? w : x, int(blockIdx.x) - (second ? split : 0));
}

// Rows into rows of bf16, `pitch` elements apart: as they are, or as three terms in three planes whose sum is the value.
// One or two matrices (the first takes `blocks0` blocks).
template <typename T>
__global__ void __launch_bounds__(256) repack_kernel(const Repack r0, const Repack r1, unsigned blocks0) {
  const bool second = blockIdx.x >= blocks0;
  const Repack& r = second ? r1 : r0;
  const T* src = static_cast<const T*>(r.src.p);
  __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(r.dst);
  const int64_t plane = r.rows * r.pitch, all = r.rows * (r.pitch / 8);
  const int per_row = int(r.pitch / 8);
  const unsigned block = blockIdx.x - (second ? blocks0 : 0), blocks = second ? gridDim.x - blocks0 : blocks0;
  for (int64_t e = block * int64_t(blockDim.x) + threadIdx.x; e < all; e += int64_t(blocks) * blockDim.x) {
    const int64_t row = e / per_row;
    const int c = int(e - row * per_row) * 8;
    float v[8];
    const T* s = src + row * r.src.stride + c;
    if (r.vec) {
      load8(s, v);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = c + j < r.cols ? ld_f32(s + j) : 0.f;
    }
    __nv_bfloat16* d = dst + row * r.pitch + c;
    if (sizeof(T) == 2)
      store8(d, v);
    else
      store_terms(d, plane, v);
  }
}

// ------------------------------------------------------------------ launch

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                             const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                             CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encode_fn() {
  static EncodeFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeFn>(p);
  });
  return fn;
}

// rows of `cols` bf16, `pitch` elements apart, `planes` times
bool make_map(CUtensorMap* m, const TcOperand& o, bool f32, int box_rows) {
  EncodeFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {cuuint64_t(o.cols), cuuint64_t(o.rows), cuuint64_t(f32 ? 3 : 1)};
  const cuuint64_t strides[2] = {cuuint64_t(o.pitch) * 2, cuuint64_t(o.pitch) * o.rows * 2};
  const cuuint32_t box[3] = {64, cuuint32_t(box_rows), 1};
  const cuuint32_t es[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(o.p), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A launch of `ctas` CTAs in clusters of CTAS.
template <int CTAS, auto Kernel, class... A>
cudaError_t launch_cluster(int ctas, int threads, size_t smem, cudaStream_t st, const A&... args) {
  const cudaError_t e = allow_smem<Kernel>(smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(ctas), 1, 1);
  cfg.blockDim = dim3(unsigned(threads), 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = CTAS;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = CTAS > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, Kernel, args...);
}

// `halves` matrices of N bf16 columns side by side in rows of halves * N: boxes of 32 x 32 to be written.
bool make_out_map(CUtensorMap* m, const void* p, int64_t M, int N, int halves) {
  EncodeFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[3] = {cuuint64_t(N), cuuint64_t(halves), cuuint64_t(M)};
  const cuuint64_t strides[2] = {cuuint64_t(N) * 2, cuuint64_t(N) * halves * 2};
  const cuuint32_t box[3] = {32, 1, 32};
  const cuuint32_t es[3] = {1, 1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(p), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// f(LONG).  The code of several runs costs a single CTA's tiles, whose products are short, 0.3 us of 41 where it is not used
// (65536 x 128 -> 512 gated), so they have kernels without it; pairs none.
template <int CTAS, bool F32, class F>
cudaError_t with_runs(bool several, F f) {
  if constexpr (F32)
    return f(std::false_type{});
  else if constexpr (CTAS == 2)
    return f(std::true_type{});
  else
    return several ? f(std::true_type{}) : f(std::false_type{});
}

template <int CTAS, bool A_MN, bool B_MN, bool F32, int EPI>
cudaError_t launch_one(const TcGemm& g, const TcPlan& p, const TcArgs& a, cudaStream_t st, int* launches) {
  using C = TcCfg<CTAS, F32, EPI>;
  CUtensorMap ta, tb;
  if (!make_map(&ta, g.A, F32, A_MN ? 64 : 128) || !make_map(&tb, g.B, F32, 64)) return cudaErrorInvalidValue;
  CUtensorMap ty = ta, tz = ta;
  if (!F32 && (a.vec & 1)) {
    if (!make_out_map(&ty, a.y, a.M, a.N, 1) || (a.z && !make_out_map(&tz, a.z, a.M, a.N, EPI == EPI_GATED ? 2 : 1)))
      return cudaErrorInvalidValue;
  }
  auto go = [&](auto runs) {
    return launch_cluster<CTAS, tc_linear_kernel<CTAS, A_MN, B_MN, F32, EPI, runs()>>(p.W * CTAS, C::THREADS, C::SMEM, st, ta,
                                                                                      tb, ty, tz, a);
  };
  const cudaError_t e = with_runs<CTAS, F32>(a.KB > kRun, go);
  ++*launches;
  if (e != cudaSuccess || p.cut == 0) return e;
  constexpr int CH = TileShape<CTAS>::template YN<EPI> / 32;
  tc_join_kernel<CTAS, F32, EPI>
      <<<unsigned(p.cut * CTAS * CH), kJoinThreads, 4 * (EPI == EPI_GATED ? 2 : 1) * kStageBytes, st>>>(a);
  ++*launches;
  return cudaGetLastError();
}

template <int CTAS, bool F32>
cudaError_t launch_grads(const TcGemm& gx, const TcPlan& px, const TcArgs& x, const TcGemm& gw, const TcPlan& pw,
                         const TcArgs& w, cudaStream_t st, int* launches) {
  using C = TcCfg<CTAS, F32, EPI_PLAIN>;
  CUtensorMap xa, xb, wa, wb;
  if (!make_map(&xa, gx.A, F32, 128) || !make_map(&xb, gx.B, F32, 64) || !make_map(&wa, gw.A, F32, 64) ||
      !make_map(&wb, gw.B, F32, 64))
    return cudaErrorInvalidValue;
  CUtensorMap xy = xa, wy = wa;
  if (!F32 && ((x.vec & 1) && !make_out_map(&xy, x.y, x.M, x.N, 1))) return cudaErrorInvalidValue;
  if (!F32 && ((w.vec & 1) && !make_out_map(&wy, w.y, w.M, w.N, 1))) return cudaErrorInvalidValue;
  auto go = [&](auto runs) {
    return launch_cluster<CTAS, tc_linear_grads_kernel<CTAS, F32, runs()>>((px.W + pw.W) * CTAS, C::THREADS, C::SMEM, st, xa, xb,
                                                                           wa, wb, xy, wy, x, w);
  };
  const cudaError_t e = with_runs<CTAS, F32>(x.KB > kRun || w.KB > kRun, go);
  ++*launches;
  if (e != cudaSuccess || px.cut + pw.cut == 0) return e;
  constexpr int CH = TileShape<CTAS>::template YN<EPI_PLAIN> / 32;
  tc_join_grads_kernel<CTAS, F32>
      <<<unsigned((px.cut + pw.cut) * CTAS * CH), kJoinThreads, 4 * kStageBytes, st>>>(x, w, int(px.cut * CTAS * CH));
  ++*launches;
  return cudaGetLastError();
}

template <int CTAS, bool F32>
cudaError_t launch_kind(const TcGemm& g, const TcPlan& p, const TcArgs& a, cudaStream_t st, int* launches) {
  if (g.a_mn) return launch_one<CTAS, true, true, F32, EPI_PLAIN>(g, p, a, st, launches);
  if (g.b_mn) return launch_one<CTAS, false, true, F32, EPI_PLAIN>(g, p, a, st, launches);
  if (g.act == SA_ACT_SWIGLU) return launch_one<CTAS, false, false, F32, EPI_GATED>(g, p, a, st, launches);
  return launch_one<CTAS, false, false, F32, EPI_FULL>(g, p, a, st, launches);
}

}  // namespace

// What a product of these sizes runs on, by the time that its blocks would take, in units of a 64-deep block of a pair's
// tile: 512 cycles of products.  Measured beside that: a single CTA's block, a quarter of the products for the same
// 32 KB a CTA, 1.4 units; of fp32 terms 4.5 (24 products read 8 KB each and 96 KB are written beside them: 2304 cycles of
// shared memory; pairs of 256 x 128 and half-deep stages measured the same or worse).  A tile takes
// no less than its end, which the next tile's products only hide (of a single CTA's tile 1.2 to 2.8 us, by the activation);
// the last end is not hidden.  Cut tiles cost a second
// kernel, 25 units, and their pieces' way to L2 and back (2048 x 1024 -> 1024: 9 us whole, 19 cut; 128 x 4096 -> 8192: 23
// and 20; dx of 16384 x 8192 -> 1024: 168 and 158).  And memory moves 6.6 TB/s, 1.8 MB a unit.  `ctas_only` 0: either kind.
TcPlan tc_plan(int64_t M, int64_t N, int64_t K, int act, bool f32, int sms, int ctas_only) {
  TcPlan best{};
  if (sms <= 0) sms = sm_count();
  const int64_t KB = (K + 63) / 64;
  const bool gated = act == SA_ACT_SWIGLU, plain = act == kPlain;
  // the end of a tile: rows that 16-byte pieces do not fit go element by element; fp32 has CUDA's erfc in gelu
  const double slow = N % (f32 ? 4 : 8) == 0 ? 1.0 : f32 ? 1.5 : 3.0;
  const double full = act == SA_ACT_GELU ? 10.4 : act == SA_ACT_SILU ? 8.0 : act == SA_ACT_RELU ? 6.5 : 5.4;
  const double end1 = slow * (!f32 ? (plain ? 6.0 : gated ? 5.5 : full)
                                   : act == SA_ACT_GELU ? 36.0 : gated ? 20.0 : plain ? 8.0 : 12.0);
  best.KB = KB;
  best.bytes = double(f32 ? 4 : 2) * (double(M) * K + double(N) * K * (gated ? 2 : 1) + double(M) * N * (gated ? 2 : 1));
  for (int ctas = 1; ctas <= (f32 || sms < 2 ? 1 : 2); ++ctas) {
    if (ctas_only && ctas != ctas_only) continue;
    const int bn = ctas == 2 ? 256 : 128, yn = gated ? bn / 2 : bn;
    const int64_t mt = (M + 128 * ctas - 1) / (128 * ctas), nt = (N + yn - 1) / yn, tiles = mt * nt;
    const int workers = sms / ctas;
    const int64_t waves = tiles / workers, rest = tiles % workers;
    const double block = f32 ? 4.5 : ctas == 2 ? 1.0 : 1.4;
    // a pair's CTAs have twice the columns and eight warps for twelve
    const double end = end1 * (ctas == 1 ? 1.0 : plain ? 1.8 : gated ? 1.9 : 2.2);
    const double tile = KB * block > end ? KB * block : end;
    for (int cut = 0; cut <= (rest && KB > 1 ? 1 : 0); ++cut) {
      int cutters = 0;
      if (cut) {
        // n shares of a tile take KB / n blocks each and half a unit each to be joined: least at sqrt(2 KB) (and never more
        // than its blocks)
        const int64_t each = int64_t(std::sqrt(2.0 * block * double(KB))) + 1, most = rest * (KB < each ? KB : each);
        cutters = int(most < workers ? most : workers);
      }
      const double rows = M < 128 * ctas ? double(M) : 128.0 * ctas;  // of a piece
      const double join = 25 + 0.5 * cutters / (rest ? rest : 1) + 2.0 * (cutters + rest) * rows * bn * 4 / 1.8e6;
      const double c = double(waves) * tile + (cut ? double((rest * KB + cutters - 1) / cutters) * block + join
                                                   : (rest ? tile : 0.0) + end) +
                       (ctas == 2 ? 8.0 : 0.0);  // a pair's launch and its two meetings
      if (best.ctas == 0 || c < best.cost) {
        best.cost = c;
        best.ctas = ctas;
        best.W = int(waves ? workers : cut ? cutters : rest);
        best.mt = mt;
        best.nt = nt;
        best.whole = cut ? waves * workers : tiles;
        best.cut = cut ? rest : 0;
        best.cutters = cutters;
      }
    }
  }
  if (best.cost < best.bytes / 1.8e6) best.cost = best.bytes / 1.8e6;
  const size_t cells = size_t(best.ctas) * 128 * (best.ctas == 2 ? 256 : 128) * sizeof(float);  // a worker's tile
  best.sums_at = best.cut ? size_t(best.cutters) * 2 * cells : 0;
  best.piece_bytes = best.sums_at + (!f32 && KB > kRun ? size_t(best.W) * cells : 0);
  return best;
}

// Both gradients' products side by side, each on a share of the SMs, where that is better than one after the other on all of
// them with a launch or two more (about ten units).
bool tc_plan_grads(int64_t M, int64_t Z, int64_t K, bool f32, double apart, TcPlan* x, TcPlan* w) {
  const int sms = sm_count();
  if (sms < 8 || apart > 1500) return false;  // large products fill the GPU by themselves
  double best = apart + 10;
  bool found = false;
  for (int ctas = 1; ctas <= (f32 ? 1 : 2); ++ctas)
    for (int eighths = 2; eighths <= 6; ++eighths) {
      const int sx = sms * eighths / 8 / ctas * ctas;
      const TcPlan px = tc_plan(M, K, Z, kPlain, f32, sx, ctas), pw = tc_plan(Z, K, M, kPlain, f32, sms - sx, ctas);
      double c = px.cost > pw.cost ? px.cost : pw.cost;
      if (c < (px.bytes + pw.bytes) / 1.8e6) c = (px.bytes + pw.bytes) / 1.8e6;
      if (c < best) {
        best = c;
        *x = px;
        *w = pw;
        found = true;
      }
    }
  return found;
}

namespace {

TcArgs tc_args(const TcGemm& g, const TcPlan& p) {
  TcArgs a{};
  a.M = g.M;
  a.N = g.N;
  a.KB = int(p.KB);
  a.mt = int(p.mt);
  a.nt = int(p.nt);
  a.by_group = Divisor(uint32_t(8 * p.nt));
  a.by_last = Divisor(uint32_t(p.mt % 8 ? p.mt % 8 : 8));
  a.W = p.W;
  a.whole = p.whole;
  a.cut = p.cut;
  a.cutters = p.cutters;
  a.half = g.N;
  a.bias = g.bias;
  a.r = g.r.p;
  a.r_stride = g.r.stride;
  a.act = g.act;
  a.y = g.y;
  a.z = g.z;
  a.Z = g.act == SA_ACT_SWIGLU ? 2 * int64_t(g.N) : g.N;
  const int each = g.dt == SA_BF16 ? 8 : 4;
  auto base_ok = [](const void* q) { return reinterpret_cast<uintptr_t>(q) % 16 == 0; };
  a.vec = (g.N % each == 0 && base_ok(g.y) && base_ok(g.z) ? 1 : 0) |
          (g.N % each == 0 && g.r.stride % each == 0 && base_ok(g.r.p) ? 2 : 0);
  a.piece = g.piece;
  a.sums = g.piece + p.sums_at / sizeof(float);
  a.ws = g.ws;
  a.clear = g.clear;
  const uint64_t ns = wait_limit_ns();
  a.wait_ns = ns > 0xFFFFFFFFull ? 0xFFFFFFFFu : uint32_t(ns);
  return a;
}

}  // namespace

cudaError_t launch_tc_gemm(const TcGemm& g, const TcPlan& p, cudaStream_t st, int* launches) {
  const TcArgs a = tc_args(g, p);
  if (g.dt == SA_F32) return launch_kind<1, true>(g, p, a, st, launches);
  return p.ctas == 2 ? launch_kind<2, false>(g, p, a, st, launches) : launch_kind<1, false>(g, p, a, st, launches);
}

cudaError_t launch_tc_grads(const TcGemm& gx, const TcPlan& px, const TcGemm& gw, const TcPlan& pw, cudaStream_t st,
                            int* launches) {
  const TcArgs x = tc_args(gx, px), w = tc_args(gw, pw);
  if (gx.dt == SA_F32) return launch_grads<1, true>(gx, px, x, gw, pw, w, st, launches);
  return px.ctas == 2 ? launch_grads<2, false>(gx, px, x, gw, pw, w, st, launches)
                      : launch_grads<1, false>(gx, px, x, gw, pw, w, st, launches);
}

cudaError_t launch_repack(Repack r0, Repack r1, cudaStream_t st) {
  auto blocks = [](Repack& r) {
    r.vec = r.cols % 8 == 0 && reinterpret_cast<uintptr_t>(r.src.p) % 16 == 0 &&
            r.src.stride % (r.src.dt == SA_BF16 ? 8 : 4) == 0;
    const int64_t all = r.dst ? r.rows * (r.pitch / 8) : 0, need = (all + 255) / 256, most = int64_t(sm_count()) * 16;
    return unsigned(need < most ? need : most);
  };
  const unsigned b0 = blocks(r0), b1 = blocks(r1);
  if (b0 + b1 == 0) return cudaSuccess;
  if ((b0 ? r0 : r1).src.dt == SA_BF16)
    repack_kernel<__nv_bfloat16><<<b0 + b1, 256, 0, st>>>(r0, r1, b0);
  else
    repack_kernel<float><<<b0 + b1, 256, 0, st>>>(r0, r1, b0);
  return cudaGetLastError();
}

}  // namespace dense
}  // namespace sa
