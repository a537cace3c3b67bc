// Attention over the 4-bit cache with warp-level tensor-core products: the form for
// few queries (serving's single tokens), for fp32 and for every width.
//
// One warp is one worker.  It owns 8 NR query rows (a user's queries times the query
// heads that share a cached head) and walks KB cached positions at a time, everything
// transposed so that the cache is the 16-row operand and a few queries the 8-column one:
//     S^T = K Q^T  (m16n8k16)  ->  online softmax in registers  ->  O^T += V^T P^T
// The 4-bit words go from shared memory straight into the A operands' registers:
//   - for K Q^T lane (g, t) = (lane / 4, lane % 4) takes keys g and g + 8 and features
//     [D/4 t, D/4 (t+1)): the contraction order is free, so Q's fragments are laid out
//     the same way once per segment;
//   - for V^T P^T it takes four keys' features of column group g; a byte permute puts
//     two keys' words side by side and the same masks give the pairs (k, k+1) that the
//     operand wants.  S^T's accumulators become P^T's operand by a transpose of 8 x 8
//     tiles between registers.
// So nothing is stored dequantised, and a cached byte costs one bulk copy and one
// shared-memory read per product.  With one query per user the call is bound by
// reading the cache, 144 bytes a key and head at d = 128, and next by issuing about
// 20 instructions a key and head and warp, four fifths of them dequantisation.
//
// Measured (GB300): one query of 16 users over up to 100,000 positions, 8 heads of 128
// (0.82 GB of cache), 204 us: 4.0 TB/s of a measured copy's 6.8, DRAM busy 53 %, the integer
// pipe 48 %, issue slots 64 %.  A lone query over 512 positions takes 11 us, two launches and
// a walk of one block a warp.  Four tiles of 8 rows a warp for the bf16 gradient
// spilled and were slower, plain asynchronous copies instead of bulk copies the same.
//
// Work is the list of (user, cached head, row tile, block of positions), cut into
// equal contiguous shares; a segment cut by share borders leaves unfinished
// (O, max, sum) pieces that the join kernel adds in order.  Every CTA scans the
// users' lengths itself, so a call is two launches.
#include <type_traits>

#include "sa_cache.cuh"
#include "sa_cache_walk.cuh"
#include "sa_kernels.cuh"
#include "sa_ptx.cuh"
#include "sa_simt_util.cuh"

namespace sa {
namespace cache {

template <int D_, bool F32_, bool BWD_, int NR_>
struct Cfg {
  static constexpr int D = D_;
  static constexpr bool F32 = F32_, BWD = BWD_;
  static constexpr int NR = NR_;           // column tiles of 8 query rows
  static constexpr int ROWS = 8 * NR;
  static constexpr int KB = 64;            // positions per block
  static constexpr int HALF = ROWS;        // every block of work costs the same
  // bf16 terms of a query element, of dO's and of dS's.  One for bf16 calls: q and dO are bf16,
  // and dS takes the rounding that the tcgen05 gradient's dS takes, for the same reason.
  static constexpr int NS = F32 ? 3 : 1;
  static constexpr int NP = F32 ? 2 : 1;   // float16 terms of a weight
  static constexpr int LW = D / 32;        // words of 8 features a lane holds of a key
  static constexpr int MT = D / 16;        // row tiles of the transposed output
  static constexpr int FRAG = LW * 32 * 16 * NR;
  static constexpr int FRAGS = FRAG * NS * (BWD ? 2 : 1);
  static constexpr int STAGE = KB * 2 * (D / 2 + D / 16);
  static constexpr int WARP_SMEM = FRAGS + 2 * STAGE;
  static constexpr int FIT = (232448 - 8192) / WARP_SMEM;  // warps that shared memory holds
  static constexpr int WANT = D == 128 ? (BWD || F32 || NR > 1 ? 8 : 10) : (F32 && NR > 1 ? 8 : BWD || F32 || NR > 1 ? 12 : 14);
  static constexpr int NWARP = FIT < WANT ? FIT : WANT;
  static constexpr int THREADS = NWARP * 32;
  static constexpr int OFF_BAR = NWARP * WARP_SMEM + 128;  // the last lanes of a narrow row may read past a stage
  static constexpr int OFF_SCAN = OFF_BAR + NWARP * 16;
  static constexpr int OFF_CTL = OFF_SCAN + (THREADS + 2) * 8;
  static constexpr int SMEM = OFF_CTL + 16;
  static_assert(SMEM <= 232448, "shared memory budget");
};

// ------------------------------------------------------------- small pieces
__device__ __forceinline__ void mma_bf16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// 8 x 8 tile of 16-bit values: lane (g, t) gives row g, columns 2t and 2t + 1, and gets
// column g, rows 2t and 2t + 1.
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 unpack_f16(uint32_t v) { return __half22float2(*reinterpret_cast<__half2*>(&v)); }
__device__ __forceinline__ float2 unpack_bf16(uint32_t v) {
  return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
               "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}

// Row c of an 8-key tile is this key of the tile: pairs differ in parity and the
// even rows hold two even and two odd keys, so the reads of K (two keys a phase)
// and of V (four keys a phase) spread over the shared-memory banks.
__device__ __forceinline__ int key_of(int c) { return c ^ ((c >> 1) & 1); }

// --------------------------------------------------------------- the kernel
template <class C, bool FULL>
struct Warp {
  const AttnArgs& a;
  const int lane, g, t4;
  uint8_t* const frag;       // Q (and dout) fragments
  uint8_t* const ring;       // two stages
  const uint32_t bar;        // two barriers
  volatile int* const ctl;
  WsHeader* const slot;
  static constexpr int KB = C::KB;
  uint32_t issued = 0, used = 0;
  bool ok = true;

  // A stage holds the block's key codes, key scales, value codes and value scales, each
  // contiguous over the positions whatever the page size.  Lane 4 p + i copies part i of
  // the block's p-th page (all of it, or KB positions of a larger one).
  __device__ __forceinline__ int width() const { return FULL ? C::D : a.c.d; }
  __device__ __forceinline__ bool wanted(const Walk& w, int kb) const {
    const int n = min(a.c.page, KB), off = (lane >> 2) * n, p0 = kb * KB + off;
    return off < KB && p0 < w.vis1 && p0 + n > w.vis0;
  }
  __device__ __forceinline__ int page_id(const Walk& w, int kb) const {
    if (!wanted(w, kb)) return 0;
    const int p0 = kb * KB + (lane >> 2) * min(a.c.page, KB);
    return a.c.table[int64_t(w.b) * a.c.max_pages + (p0 >> a.c.log2page)];
  }
  __device__ __forceinline__ void issue(const Walk& w, int kb, int pid) {
    const uint32_t s = issued & 1u;
    const uint32_t b = bar + 8u * s;
    const uint32_t dst = smem_u32(ring) + s * C::STAGE;
    bool want = wanted(w, kb);
    if (want && (pid < 0 || pid >= a.c.n_pages)) {
      const int n = min(a.c.page, KB), p0 = kb * KB + (lane >> 2) * n;
      if (tile_sees<C>(a, w, p0, p0 + n, 0, 1)) atomicCAS(&slot->err, 0u, uint32_t(SA_ERR_BAD_PAGE));
      want = false;
    }
    if (a.c.page == KB) {  // a block is a page, and a page's records lie as the stage does
      if (lane == 0) {
        const uint32_t bytes = want ? 2u * a.c.rec : 0u;
        mbar_arrive_expect_tx(b, bytes);
        if (want) bulk_load(dst, a.c.pool + a.c.record(pid, w.h), bytes, b);
      }
    } else {
      const int n = min(a.c.page, KB), off = (lane >> 2) * n, first = (kb * KB + off) & (a.c.page - 1);
      const int kv = (lane >> 1) & 1, rb = lane & 1 ? a.c.d / 16 : a.c.d / 2;  // bytes of a row of this part
      const uint32_t bytes = want ? uint32_t(n * rb) : 0u;
      const uint32_t total = __reduce_add_sync(0xffffffffu, bytes);
      if (lane == 0) mbar_arrive_expect_tx(b, total);
      __syncwarp();
      if (want) {
        const uint8_t* src = a.c.pool + a.c.record(pid, w.h) + kv * a.c.rec + (lane & 1 ? a.c.page * (a.c.d / 2) : 0) + first * rb;
        bulk_load(dst + (kv * (KB * (a.c.d / 2 + a.c.d / 16))) + (lane & 1 ? KB * (a.c.d / 2) : 0) + off * rb, src, bytes, b);
      }
    }
    ++issued;
  }

  // Code row and scales of key k (kv = 0) or value k (kv = 1) within the stage.
  __device__ __forceinline__ const uint8_t* row(const uint8_t* st, int k, int kv) const {
    return st + kv * (KB * (width() / 2 + width() / 16)) + k * (width() / 2);
  }
  __device__ __forceinline__ const uint8_t* scales(const uint8_t* st, int k, int kv) const {
    return st + kv * (KB * (width() / 2 + width() / 16)) + KB * (width() / 2) + k * (width() / 16);
  }
  // This lane's words of key row k in the contraction layout, and its scale codes.
  __device__ __forceinline__ void load_words(const uint8_t* st, int k, int kv, uint32_t* w, uint32_t& codes) const {
    const uint8_t* p = row(st, k, kv) + t4 * (C::LW * 4);
    const uint8_t* sp = scales(st, k, kv) + t4 * (C::LW / 2);
    if constexpr (C::LW == 4) {
      if constexpr (FULL) {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
        codes = *reinterpret_cast<const uint16_t*>(sp);
      } else {
        const uint2 v = *reinterpret_cast<const uint2*>(p), u = *reinterpret_cast<const uint2*>(p + 8);
        w[0] = v.x, w[1] = v.y, w[2] = u.x, w[3] = u.y;
        codes = uint32_t(sp[0]) | uint32_t(sp[1]) << 8;
      }
    } else {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      w[0] = v.x, w[1] = v.y;
      codes = sp[0];
    }
  }
  // acc[m][n] = key tile m (16 keys from 16 (m0 + m)) x query rows 8 n ..; `fr` their fragments
  template <int NM>
  __device__ __forceinline__ void contract(const uint8_t* st, int m0, int kv, const uint8_t* fr,
                                           float (*acc)[C::NR][4]) const {
    uint32_t w[NM][2][C::LW], codes[NM][2];
#pragma unroll
    for (int m = 0; m < NM; ++m) {
      load_words(st, 16 * (m0 + m) + key_of(g), kv, w[m][0], codes[m][0]);
      load_words(st, 16 * (m0 + m) + 8 + key_of(g), kv, w[m][1], codes[m][1]);
#pragma unroll
      for (int n = 0; n < C::NR; ++n) acc[m][n][0] = acc[m][n][1] = acc[m][n][2] = acc[m][n][3] = 0.f;
    }
    ScaleB sc[NM][2];
#pragma unroll
    for (int i = 0; i < C::LW; ++i) {
      uint4 q[C::NS][C::NR];
#pragma unroll
      for (int s = 0; s < C::NS; ++s)
#pragma unroll
        for (int n = 0; n < C::NR; ++n)
          q[s][n] = *reinterpret_cast<const uint4*>(fr + s * C::FRAG + ((n * C::LW + i) * 32 + lane) * 16);
#pragma unroll
      for (int m = 0; m < NM; ++m) {
        if (i % 2 == 0) {  // two words share a scale
          sc[m][0] = scale_bf16(((codes[m][0] >> (8 * (i / 2))) & 255u) * 0x00010001u);
          sc[m][1] = scale_bf16(((codes[m][1] >> (8 * (i / 2))) & 255u) * 0x00010001u);
        }
        uint32_t lo[4], hi[4];
        values_bf16(w[m][0][i], sc[m][0], lo);
        values_bf16(w[m][1][i], sc[m][1], hi);
        const uint32_t A0[4] = {lo[0], hi[0], lo[1], hi[1]}, A1[4] = {lo[2], hi[2], lo[3], hi[3]};
#pragma unroll
        for (int s = C::NS - 1; s >= 0; --s)  // the smallest terms first
#pragma unroll
          for (int n = 0; n < C::NR; ++n) {
            mma_bf16(acc[m][n], A0, q[s][n].x, q[s][n].y);
            mma_bf16(acc[m][n], A1, q[s][n].z, q[s][n].w);
          }
      }
    }
  }
  // A block that some row does not see whole may hold bytes that nobody wrote (see
  // level_min7): seen to in the stage, before its values are read as float16.
  __device__ __forceinline__ uint8_t* value_codes(uint8_t* st) const { return st + KB * (width() / 2 + width() / 16); }
  __device__ __forceinline__ uint8_t* value_scales(uint8_t* st) const { return value_codes(st) + KB * (width() / 2); }
  // Not 0 where this lane's part of the scales has a code above kCodeSafe.
  __device__ __forceinline__ uint32_t high_scales(uint8_t* st) const {
    static_assert(kCodeSafe == 0xDF, "the codes above it are those with their upper three bits set");
    uint32_t high = 0;
#pragma unroll
    for (int i = lane; i < C::D; i += 32) {  // four scales a word
      const uint32_t v = i < width() ? reinterpret_cast<const uint32_t*>(value_scales(st))[i] : 0u;
      high |= v & v << 1 & v << 2;
    }
    return high & 0x80808080u;
  }
  __device__ __forceinline__ void make_finite(uint8_t* st) const {
    uint8_t* sc = value_scales(st);
#pragma unroll 1
    for (int i = lane; i < 4 * width(); i += 32) {  // groups, 8 bytes of codes each
      if (sc[i] <= kCodeSafe) continue;
      uint2* w = reinterpret_cast<uint2*>(value_codes(st) + 8 * i);
      *w = make_uint2(level_min7(w->x), level_min7(w->y));
      if (sc[i] > kCodeMax) sc[i] = 0;
    }
    fence_proxy_async_smem();  // before the next copy into the stage
    __syncwarp();
  }
  // acc += (rows of 16 keys from 16 jj, transposed) x weights B, WT terms each; F16 or bf16
  // values.
  template <bool F16, int WT>
  __device__ __forceinline__ void combine(const uint8_t* st, int jj, int kv, const uint32_t (*B)[WT][2],
                                          float (*acc)[C::NR][4]) const {
    int k[4];
    k[0] = 16 * jj + key_of(2 * t4);
    k[1] = 16 * jj + key_of(2 * t4 + 1);
    k[2] = k[0] + 8;
    k[3] = k[1] + 8;
    constexpr int NW = C::D / 64;  // words of column group g
    uint32_t w[4][NW], code[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint8_t* p = row(st, k[i], kv) + g * (4 * NW);
      if constexpr (NW == 2) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        w[i][0] = v.x, w[i][1] = v.y;
        code[i] = scales(st, k[i], kv)[g];
      } else {
        w[i][0] = *reinterpret_cast<const uint32_t*>(p);
        code[i] = scales(st, k[i], kv)[g >> 1];
      }
    }
    const uint32_t c01 = code[0] | code[1] << 16, c23 = code[2] | code[3] << 16;
    const ScaleB sb01 = scale_bf16(c01), sb23 = scale_bf16(c23);
    auto values = [&](uint32_t x, bool second, uint32_t* r) {
      if constexpr (F16)
        values_f16(x, (second ? c23 : c01) << 7, r);
      else
        values_bf16(x, second ? sb23 : sb01, r);
    };
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      uint32_t e01[4], e23[4], o01[4], o23[4];  // even and odd features, keys 0 1 and 2 3
      values(__byte_perm(w[0][i], w[1][i], 0x5410u), false, e01);
      values(__byte_perm(w[0][i], w[1][i], 0x7632u), false, o01);
      values(__byte_perm(w[2][i], w[3][i], 0x5410u), true, e23);
      values(__byte_perm(w[2][i], w[3][i], 0x7632u), true, o23);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t A[4] = {e01[e], o01[e], e23[e], o23[e]};
#pragma unroll
        for (int n = 0; n < C::NR; ++n)
#pragma unroll
          for (int s = WT - 1; s >= 0; --s) {
            if constexpr (F16)
              mma_f16(acc[4 * i + e][n], A, B[n][s][0], B[n][s][1]);
            else
              mma_bf16(acc[4 * i + e][n], A, B[n][s][0], B[n][s][1]);
          }
      }
    }
  }

  // Rows g of src (element offsets r[n]; negative: no row) as fragments.
  template <typename T>
  __device__ __forceinline__ void load_frags(const T* src, const int64_t* r, uint8_t* fr) const {
    const int base = (C::D / 4) * t4, d = FULL ? C::D : a.c.d;
#pragma unroll
    for (int n = 0; n < C::NR; ++n)
#pragma unroll
      for (int i = 0; i < C::LW; ++i) {
        const int c = base + 8 * i;
        uint32_t p[C::NS][4] = {};
        if (r[n] >= 0 && c < d) {
          if constexpr (C::F32) {
            float x[8];
            *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(src + r[n] + c);
            *reinterpret_cast<float4*>(x + 4) = *reinterpret_cast<const float4*>(src + r[n] + c + 4);
#pragma unroll
            for (int s = 0; s < C::NS; ++s)
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                p[s][k] = pack_bf16(x[2 * k], x[2 * k + 1]);
                const float2 f = unpack_bf16(p[s][k]);
                x[2 * k] -= f.x;
                x[2 * k + 1] -= f.y;
              }
          } else {
            *reinterpret_cast<uint4*>(p[0]) = *reinterpret_cast<const uint4*>(src + r[n] + c);
          }
        }
#pragma unroll
        for (int s = 0; s < C::NS; ++s)
          *reinterpret_cast<uint4*>(fr + s * C::FRAG + ((n * C::LW + i) * 32 + lane) * 16) =
              *reinterpret_cast<const uint4*>(p[s]);
      }
  }
};

template <class C, bool FULL>
__global__ void __launch_bounds__(C::THREADS, 1) cache_mma_kernel(const __grid_constant__ AttnArgs a) {
  using T = typename std::conditional<C::F32, float, __nv_bfloat16>::type;
  extern __shared__ __align__(128) uint8_t smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  WsHeader* slot = a.slots + blockIdx.x;
  volatile int* ctl = reinterpret_cast<volatile int*>(smem + C::OFF_CTL);
  const uint32_t bar = smem_u32(smem) + C::OFF_BAR + warp * 16;
  if (lane == 0) {
    mbar_init(bar, 1);
    mbar_init(bar + 8, 1);
  }
  if (threadIdx.x == 0) {
    slot->err = 0;
    slot->timeout_site = 0;
    slot->wait_limit_ns = a.wait_limit_ns;
    wait_ctl_init(ctl, slot);
  }
  fence_mbar_init();
  int64_t* pre = reinterpret_cast<int64_t*>(smem + C::OFF_SCAN);
  const int chunk = (a.B + C::THREADS - 1) / C::THREADS;
  const int64_t total = scan_users<C>(a, pre, chunk);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    ws_header(a.ws)->tiles_per_head = total;
    if (total < 0) slot->err = uint32_t(SA_ERR_BAD_SEQLENS);
  }
  asm volatile("griddepcontrol.launch_dependents;");
  if (total <= 0) return;

  // Worker order runs over the CTAs first, so that little work still spreads over the SMs.
  const int wk = int(blockIdx.x) + warp * int(gridDim.x), W = shares(a, total);
  if (wk >= W) return;
  const int64_t tb = range_begin(total, W, wk), te = range_begin(total, W, wk + 1);

  uint8_t* mine = smem + warp * C::WARP_SMEM;
  Warp<C, FULL> x{a, lane, lane >> 2, lane & 3, mine, mine + C::FRAGS, bar, ctl, slot};
  constexpr int KB = C::KB, NR = C::NR;
  const int g = x.g, t4 = x.t4, d = FULL ? C::D : a.c.d;
  const float c2 = a.scale * kLog2e;

  Walk cur, ahead;  // `ahead` runs up to two blocks in front and issues the copies
  cur.t = tb;
  cur.te = te;
  {
    int64_t rem;
    find_tile<C>(a, pre, chunk, tb, lane, cur.b, rem);
    set_piece<C>(a, cur, user_sizes<C>(a, cur.b), rem, lane);
  }
  if (lane == 0) {
    Piece p{cur.seg0, cur.seg1, cur.b, cur.h, cur.rt, 0};
    static_cast<Piece*>(a.piece)[wk] = p;
  }
  ahead = cur;
  int akb = ahead.kb0;
  bool more = true;
  auto settle = [&]() {  // move `ahead` to a block that exists
    while (more && akb >= ahead.kb1) {
      more = next_piece<C>(a, ahead, lane);
      akb = ahead.kb0;
    }
  };
  settle();
  int pid = more ? x.page_id(ahead, akb) : 0;
  auto produce = [&]() {
    if (!more) return;
    x.issue(ahead, akb, pid);
    ++akb;
    settle();
    pid = more ? x.page_id(ahead, akb) : 0;
  };
  produce();
  produce();

  const T* q = static_cast<const T*>(a.q);
  for (bool have = true; have && x.ok;) {
    // Row g of each column tile feeds the products; rows 2t and 2t + 1 are this lane's in
    // the accumulators (their windows, statistics and sums).
    int64_t q_at[NR];
    int lo[NR][2], hi[NR][2];
    float D_[NR][2], L[NR][2];
    int lo_most = 0, hi_least = 0x7fffffff;
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int r = cur.rt * C::ROWS + 8 * n + g;
      q_at[n] = r < cur.s.rows ? (cur.s.q0 + r / a.G) * a.q_row + (cur.h * a.G + r % a.G) * a.q_head : -1;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int s = cur.rt * C::ROWS + 8 * n + 2 * t4 + e;
        lo[n][e] = 0, hi[n][e] = 0x7fffffff;
        if (s < cur.s.rows) row_window(a, cur.s.q0 + s / a.G, cur.s.len, lo[n][e], hi[n][e]);
        lo_most = max(lo_most, lo[n][e]);
        hi_least = min(hi_least, hi[n][e]);
        D_[n][e] = L[n][e] = 0.f;
      }
    }
    lo_most = __reduce_max_sync(0xffffffffu, lo_most);
    hi_least = __reduce_min_sync(0xffffffffu, hi_least);
    // row i of this lane's: element offset in the dense tensors / d, or -1
    auto dense = [&](int i) {
      const int r = cur.rt * C::ROWS + i;
      return r < cur.s.rows ? (cur.s.q0 + r / a.G) * a.Hq + cur.h * a.G + r % a.G : int64_t(-1);
    };
    if (cur.kb0 < cur.kb1) {
      x.load_frags(q, q_at, x.frag);
      if constexpr (C::BWD) {
        const T* dout = static_cast<const T*>(a.dout);
        const T* out = static_cast<const T*>(a.out);
        int64_t o_at[NR];
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          const int64_t o = dense(8 * n + g);
          o_at[n] = o < 0 ? -1 : o * d;
          float s = 0.f;
          if (o >= 0)
            for (int c = (C::D / 4) * t4; c < (C::D / 4) * (t4 + 1) && c < d; c += Vec<T>::n) {
              float u[Vec<T>::n], v[Vec<T>::n];
              Vec<T>::load(dout + o * d + c, u);
              Vec<T>::load(out + o * d + c, v);
#pragma unroll
              for (int k = 0; k < Vec<T>::n; ++k) s = fmaf(u[k], v[k], s);
            }
          s += __shfl_xor_sync(0xffffffffu, s, 1);
          s += __shfl_xor_sync(0xffffffffu, s, 2);  // row g's sum in its four lanes
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            D_[n][e] = __shfl_sync(0xffffffffu, s, 4 * (2 * t4 + e));
            const int64_t oe = dense(8 * n + 2 * t4 + e);
            if (oe >= 0) L[n][e] = a.lse[oe] * kLog2e;
          }
        }
        x.load_frags(dout, o_at, x.frag + C::NS * C::FRAG);
      }
    }

    float acc[C::MT][NR][4], m[NR][2], l[NR][2];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
#pragma unroll
      for (int i = 0; i < C::MT; ++i) acc[i][n][0] = acc[i][n][1] = acc[i][n][2] = acc[i][n][3] = 0.f;
      m[n][0] = m[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.f;
    }

    for (int kb = cur.kb0; kb < cur.kb1; ++kb) {
      const uint32_t s = x.used & 1u;
      x.ok = __all_sync(0xffffffffu, mbar_wait(bar + 8 * s, (x.used >> 1) & 1u, ctl, slot, 0xC01u));
      if (!x.ok) break;
      uint8_t* st = x.ring + s * C::STAGE;
      const int k0 = kb * KB;
      const bool inside = k0 >= lo_most && k0 + KB <= hi_least;
      // accumulator element e of key tile i: key 16 i + 8 (e / 2) + key_of(g), row 2t + e % 2
      auto key = [&](int i, int e) { return k0 + 16 * i + 8 * (e >> 1) + key_of(g); };
      if constexpr (!C::BWD) {
        float S[KB / 16][NR][4];
        const uint32_t high = inside ? 0u : x.high_scales(st);
        x.template contract<KB / 16>(st, 0, 0, x.frag, S);
        if (!inside && __any_sync(0xffffffffu, high != 0)) x.make_finite(st);
        bool moved = false;
        float nm[NR][2], z[NR][2];
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          float b[2] = {-INFINITY, -INFINITY};
#pragma unroll
          for (int i = 0; i < KB / 16; ++i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              S[i][n][e] *= c2;
              if (!inside && (key(i, e) < lo[n][e & 1] || key(i, e) >= hi[n][e & 1])) S[i][n][e] = -INFINITY;
            }
            b[0] = fmax3(b[0], S[i][n][0], S[i][n][2]);
            b[1] = fmax3(b[1], S[i][n][1], S[i][n][3]);
          }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int o = 4; o <= 16; o <<= 1) b[e] = fmaxf(b[e], __shfl_xor_sync(0xffffffffu, b[e], o));
            nm[n][e] = fmaxf(m[n][e], b[e]);
            // nothing seen yet: shift by zero, so that 2^(-inf) = 0 and no inf - inf appears
            z[n][e] = nm[n][e] == -INFINITY ? 0.f : nm[n][e];
            moved = moved || nm[n][e] != m[n][e];
          }
        }
        if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
          for (int n = 0; n < NR; ++n) {
            const float f0 = ex2(m[n][0] - z[n][0]), f1 = ex2(m[n][1] - z[n][1]);
            l[n][0] *= f0;
            l[n][1] *= f1;
#pragma unroll
            for (int i = 0; i < C::MT; ++i) {
              acc[i][n][0] *= f0, acc[i][n][1] *= f1;
              acc[i][n][2] *= f0, acc[i][n][3] *= f1;
            }
            m[n][0] = nm[n][0];
            m[n][1] = nm[n][1];
          }
        }
#pragma unroll
        for (int i = 0; i < KB / 16; ++i) {
          uint32_t B[NR][C::NP][2];
#pragma unroll
          for (int n = 0; n < NR; ++n) {
            float* p = S[i][n];
            const float sh0 = z[n][0] - kLift, sh1 = z[n][1] - kLift;
            p[0] = ex2(p[0] - sh0), p[1] = ex2(p[1] - sh1);
            p[2] = ex2(p[2] - sh0), p[3] = ex2(p[3] - sh1);
            l[n][0] += p[0] + p[2];
            l[n][1] += p[1] + p[3];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const uint32_t h = pack_f16(p[2 * u], p[2 * u + 1]);
              B[n][0][u] = transpose8x8(h);
              if constexpr (C::NP == 2) {
                const float2 f = unpack_f16(h);
                B[n][1][u] = transpose8x8(pack_f16(p[2 * u] - f.x, p[2 * u + 1] - f.y));
              }
            }
          }
          x.template combine<true, C::NP>(st, i, 1, B, acc);
        }
      } else {
        constexpr int HM = KB / 32;  // half a block at a time: two products' scores are live
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
          float S[HM][NR][4], P[HM][NR][4];
          x.template contract<HM>(st, HM * half, 0, x.frag, S);
          x.template contract<HM>(st, HM * half, 1, x.frag + C::NS * C::FRAG, P);
#pragma unroll
          for (int i = 0; i < HM; ++i) {
            uint32_t B[NR][C::NS][2];
#pragma unroll
            for (int n = 0; n < NR; ++n) {
              float p[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int k = key(HM * half + i, e);
                const float w = ex2(fmaf(S[i][n][e], c2, -L[n][e & 1])) * (P[i][n][e] - D_[n][e & 1]);
                p[e] = inside || (k >= lo[n][e & 1] && k < hi[n][e & 1]) ? w : 0.f;
              }
#pragma unroll
              for (int s2 = 0; s2 < C::NS; ++s2)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                  const uint32_t h = pack_bf16(p[2 * u], p[2 * u + 1]);
                  B[n][s2][u] = transpose8x8(h);
                  const float2 f = unpack_bf16(h);
                  p[2 * u] -= f.x, p[2 * u + 1] -= f.y;
                }
            }
            x.template combine<false, C::NS>(st, HM * half + i, 0, B, acc);
          }
        }
      }
      ++x.used;
      __syncwarp();  // every lane is done with the stage
      produce();
    }
    if (!x.ok) break;

    // the piece's end: this lane has features [per g, per (g + 1)) of rows 2t and 2t + 1
    const bool whole = cur.seg0 >= tb && cur.seg1 <= te;
    constexpr int PER = C::D / 8;
    float* part = a.partial + (int64_t(wk) * 2 + (tb >= cur.seg0 ? 0 : 1)) * partial_floats(C::ROWS, C::D);
    T* dst = static_cast<T*>(C::BWD ? a.dq : a.out);
#pragma unroll
    for (int n = 0; n < NR; ++n) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float sum = l[n][e];
        if constexpr (!C::BWD) {
#pragma unroll
          for (int o = 4; o <= 16; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        }
        const int i = 8 * n + 2 * t4 + e;
        const int64_t o = dense(i);
        if (o < 0) continue;
        const float f = !whole ? 1.f : C::BWD ? a.scale : sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int w = 0; w < PER / 8; ++w) {
          float y[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) y[k] = acc[4 * w + k / 2][n][2 * (k & 1) + e] * f;
          const int c = PER * g + 8 * w;
          if (c >= d) continue;
          if (whole)
            store8(dst + o * d + c, y);
          else
            store8(part + i * C::D + c, y);
        }
        if constexpr (!C::BWD) {
          if (g == 0) {
            if (!whole)
              *reinterpret_cast<float2*>(part + C::ROWS * C::D + 2 * i) = make_float2(m[n][e], sum);
            else if (a.lse)
              a.lse[o] = sum == 0.f ? -INFINITY : (m[n][e] + log2f(sum) - kLift) * kLn2;
          }
        }
      }
    }
    have = next_piece<C>(a, cur, lane);
  }
  if (!x.ok) {  // no copy may still be in flight when the CTA's shared memory goes
    for (; x.used != x.issued; ++x.used) {
      const uint64_t t0 = globaltimer();
      while (!mbar_try_wait(bar + 8 * (x.used & 1u), (x.used >> 1) & 1u) && globaltimer() - t0 < 200000000ull) {
      }
    }
  }
}

// ---------------------------------------------------------------- launching
template <class C, bool FULL>
static cudaError_t run_main(const AttnArgs& a, cudaStream_t st) {
  cudaError_t e = cudaFuncSetAttribute(cache_mma_kernel<C, FULL>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
  if (e != cudaSuccess) return e;
  cache_mma_kernel<C, FULL><<<a.ctas, C::THREADS, C::SMEM, st>>>(a);
  return cudaGetLastError();
}

template <class C>
static cudaError_t run(const AttnArgs& a, cudaStream_t st) {
  const cudaError_t e = a.c.d == C::D ? run_main<C, true>(a, st) : run_main<C, false>(a, st);
  if (e != cudaSuccess) return e;
  return launch_join<C>(a, st);
}

// Rows of a tile: 8 where a user's rows fit (the average over the call decides: half the
// products and registers of 16), else 16, which dequantises half as often; always 8 for the
// fp32 gradient, whose 16 rows spill (their times: when they existed).  Measured on a GB300,
// us (8 | 16 a tile), 16 users x 8 heads x 10,000 positions:
//                          8 rows        16 rows
//     forward, bf16        63 | 71      103 |  76    (d = 128; 64: 42 | 48 and 66 | 51)
//     forward, fp32        71 | 104     115 | 111    (d = 64: 43 | 61 and 70 | 66)
//     gradient, bf16       76 | 93      126 | 101    (d = 64: 45 | 56 and 73 | 61)
//     gradient, fp32      109 | 223     192 | 230    (d = 64: 60 | 95 and 102 | 104)
static bool two_tiles(int B, int64_t T, int G, sa_dtype dt, bool bwd) {
  return T * G > int64_t(8) * B && !(bwd && dt == SA_F32);
}

// f(configuration) for a call's sizes
template <class F>
static auto with_config(int d, sa_dtype dt, bool bwd, bool two, F&& f) {
  auto rows = [&](auto D, auto f32, auto back) {
    constexpr int W = decltype(D)::value;
    constexpr bool X = decltype(f32)::value, Y = decltype(back)::value;
    if constexpr (!(X && Y)) {
      if (two) return f(Cfg<W, X, Y, 2>{});
    }
    return f(Cfg<W, X, Y, 1>{});
  };
  auto dir = [&](auto D, auto f32) { return bwd ? rows(D, f32, std::true_type{}) : rows(D, f32, std::false_type{}); };
  auto type = [&](auto D) { return dt == SA_F32 ? dir(D, std::true_type{}) : dir(D, std::false_type{}); };
  return d > 64 ? type(std::integral_constant<int, 128>{}) : type(std::integral_constant<int, 64>{});
}

AttnPlan mma_plan(int sms, int B, int64_t T, int G, int d, sa_dtype dt, bool bwd) {
  AttnPlan p;
  p.ctas = sms;
  p.workers = sms * with_config(d, dt, bwd, two_tiles(B, T, G, dt, bwd), [](auto c) { return decltype(c)::NWARP; });
  p.piece_bytes = sizeof(Piece);
  p.partial_floats =
      with_config(d, dt, bwd, two_tiles(B, T, G, dt, bwd), [](auto c) { return partial_floats(decltype(c)::ROWS, decltype(c)::D); });
  return p;
}

cudaError_t launch_mma(const AttnArgs& a, bool bwd, cudaStream_t st) {
  return with_config(a.c.d, a.dt, bwd, two_tiles(a.B, a.T, a.G, a.dt, bwd), [&](auto c) { return run<decltype(c)>(a, st); });
}

}  // namespace cache
}  // namespace sa
