// Gradient of the queries over the 4-bit cache on tcgen05, for many queries of a user:
// bf16, d in {64, 128}.
//
// A CTA holds 128 query rows with their gradients dO and walks 64 cached positions at a
// time.  Eight warps turn a block's 4-bit keys and values into bf16 operands in shared
// memory, once for all the rows:
//     S  = Q K^T,  dP = dO V^T      (M = 128, N = 64, K = d)       accumulated in TMEM
//     dS = 2^(S c - lse) (dP - D)   in registers, bf16, back over S in TMEM
//     dQ += dS K                    (M = 128, N = d, K = 64; dS read from TMEM, K as it lies
//                                   for S, now with the positions as the contraction)
// dS is rounded to bf16 once, as the third product's operand: the result is then 2.4e-3 from
// 64 bits (relative, 2-norm) where its own rounding to bf16 alone leaves 1.7e-3.  A second
// term would be a fourth product and as many instructions again for the warps that make dS,
// which bound the kernel with the others.
//
// lse and D = dO . out are known beforehand, so blocks are independent: two softmax
// warpgroups take them in turn, each with its own S and dP, and the products of one run
// under the other's exponentials.
//
// Warp roles: 0 walks the share, publishes its pieces to the other roles and copies the
// pages' codes and scales into a ring (bulk copies), 1 issues the products, 2 and 3
// load the rows of Q and dO, 4..7 dequantise keys, 8..11 values, 12..19 dS and results.  Every
// wait is bounded: past the limit the CTA's roles leave, its copies and products drain
// and the error is reported.
//
// Measured (GB300): 40 queries x 16 heads of 64 users over one shared head of 1024 x 128,
// 74 us (435 TFLOP/s of a library product's 1894; the warp-level kernel 171); up to 300 windowed
// queries of 16 users over up to 10,000 positions, 8 heads of 128, 264 us (warp-level 585;
// windows hide two thirds of the products that the blocks make).  Bound like the forward, by
// the roles' own instructions: without exponentials 250, with an eighth of the products
// 240, with a quarter of the dequantisation 248, with a quarter of the copies' code 262.
#include "sa_cache_tc.cuh"
#include "sa_simt_util.cuh"

namespace sa {
namespace cache {

template <int D_>
struct TcBwd {
  static constexpr int D = D_;
  static constexpr bool F32 = false, BWD = true;
  static constexpr int ROWS = 128, HALF = 128, KB = 64;
  static constexpr int NWARP = 20, THREADS = 640;
  static constexpr int QT = 128 * D * 2;   // query rows, [D / 64][128][128 bytes]
  static constexpr int TILE = KB * D * 2;  // a block's keys or values, [D / 64][64][128 bytes]
  static constexpr int NB = 3;             // blocks in the ring: keys in places 2 b, values in 2 b + 1
  static constexpr int NSLOT = 2 * NB;
  static constexpr int NR = D == 128 ? 3 : 6, NRAW = 2 * NR;  // blocks as they are stored
  static constexpr int RAW = KB * (D / 2 + D / 16);
  static constexpr int OFF_Q = 0, OFF_DO = QT;
  static constexpr int OFF_RING = 2 * QT;
  static constexpr int OFF_SCAN = OFF_RING;  // used before anything is dequantised
  static constexpr int OFF_RAW = OFF_RING + NSLOT * TILE;
  static constexpr int OFF_BAR = OFF_RAW + NRAW * RAW;
  static constexpr int NPIECE = 4;    // pieces published ahead
  static constexpr int NREADER = 19;  // warps that read them
  static constexpr int NBAR = 2 * NSLOT + 2 * NRAW + 9 + 2 * NPIECE;
  static constexpr int OFF_PIECE = (OFF_BAR + NBAR * 8 + 15) / 16 * 16;
  static constexpr int OFF_CTL = OFF_PIECE + NPIECE * 64;
  static constexpr int OFF_TMEM = OFF_CTL + 16;
  static constexpr int SMEM = OFF_TMEM + 16;
  static_assert(SMEM <= 232448, "shared memory budget");
  static constexpr int S_COL = 0, Q_COL = 256, COLS = 512;  // (S, dP) of each warpgroup, then dQ
};

// A piece as the roles see it (64 bytes of shared memory).
struct Part {
  int n;         // blocks; -1: the share is done
  int kb0;       // first block
  int vis0, vis1;
  int rows;      // of the tile
  int row0;      // of the tile within the user's rows of this head
  int h, len;
  int whole;     // the segment lies within this share
  int second;    // which of the worker's two unfinished pieces it is, if not whole
  int64_t q0;    // the user's first query
};
static_assert(sizeof(Part) <= 64, "one slot of the piece ring");

template <int D>
__global__ void __launch_bounds__(640, 1) cache_tc_bwd_kernel(const __grid_constant__ AttnArgs a) {
  using C = TcBwd<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  WsHeader* slot = a.slots + blockIdx.x;
  Ctl* ctl = reinterpret_cast<Ctl*>(smem + C::OFF_CTL);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::OFF_TMEM);
  const uint32_t sb = smem_u32(smem), bar0 = sb + C::OFF_BAR;
  auto slot_full = [&](uint32_t s) { return bar0 + 8u * s; };
  auto slot_empty = [&](uint32_t s) { return bar0 + 8u * (C::NSLOT + s); };
  auto raw_full = [&](uint32_t s) { return bar0 + 8u * (2 * C::NSLOT + s); };
  auto raw_empty = [&](uint32_t s) { return bar0 + 8u * (2 * C::NSLOT + C::NRAW + s); };
  const uint32_t per = bar0 + 8u * (2 * C::NSLOT + 2 * C::NRAW);
  auto s_full = [&](uint32_t g) { return per + 8u * g; };  // per warpgroup
  auto p_full = [&](uint32_t g) { return per + 8u * (2 + g); };
  const uint32_t o_full = per + 32, o_empty = per + 40, q_full = per + 48, q_empty = per + 56, drain = per + 64;
  auto piece_full = [&](uint32_t s) { return per + 8u * (9 + s); };
  auto piece_empty = [&](uint32_t s) { return per + 8u * (9 + C::NPIECE + s); };

  if (threadIdx.x == 0) {
    for (int i = 0; i < C::NBAR; ++i) {
      const int p = i - 2 * C::NSLOT - 2 * C::NRAW;
      uint32_t n = 1;
      if (i < C::NSLOT || (p < 0 && p >= -C::NRAW)) n = 4;  // slot_full, raw_empty: the dequantising warps
      if (p == 2 || p == 3) n = 4;                          // p_full: a warpgroup
      if (p == 6) n = 2;                                    // q_full: both loaders
      if (p == 5) n = 8;                                    // o_empty: both
      if (p >= 9 + C::NPIECE) n = C::NREADER;               // piece_empty
      mbar_init(bar0 + 8u * i, n);
    }
    slot->err = 0;
    slot->timeout_site = 0;
    ctl->abort = 0;
    fence_mbar_init();
  }
  int64_t* pre = reinterpret_cast<int64_t*>(smem + C::OFF_SCAN);
  const int chunk = (a.B + C::THREADS - 1) / C::THREADS;
  const int64_t total = scan_users<C>(a, pre, chunk);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    ws_header(a.ws)->tiles_per_head = total;
    if (total < 0) slot->err = uint32_t(SA_ERR_BAD_SEQLENS);
  }
  asm volatile("griddepcontrol.launch_dependents;");
  if (total <= 0) return;
  const int W = shares(a, total), wk = int(blockIdx.x);
  if (wk >= W) return;
  if (sb & 1023u) {  // the swizzled operands need 1024-byte alignment
    if (threadIdx.x == 0) slot->err = uint32_t(SA_ERR_CUDA);
    return;
  }
  const int64_t tb = range_begin(total, W, wk), te = range_begin(total, W, wk + 1);
  Walk cur;  // warp 0 walks
  if (warp == 0) {
    cur.t = tb;
    cur.te = te;
    int64_t rem;
    find_tile<C>(a, pre, chunk, tb, lane, cur.b, rem);
    set_piece<C>(a, cur, user_sizes<C>(a, cur.b), rem, lane);
    if (lane == 0) {
      Piece p{cur.seg0, cur.seg1, cur.b, cur.h, cur.rt, 0};
      static_cast<Piece*>(a.piece)[wk] = p;
    }
  }
  if (warp == 2) tmem_alloc(smem_u32(tmem_slot), C::COLS);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const uint32_t limit = wait_limit(a);
  bool ok = true;
  auto wait = [&](uint32_t bar, uint32_t parity, uint32_t site) {
    ok = ok && warp_wait(bar, parity, ctl, limit, site);
    return ok;
  };

  Part* ring = reinterpret_cast<Part*>(smem + C::OFF_PIECE);
  uint32_t np = 0;  // pieces read (or published) so far
  // the next piece; done() gives its place back
  auto next = [&](Part& u) {
    if (!wait(piece_full(np % C::NPIECE), np / C::NPIECE, 0xD51u)) return false;
    u = *reinterpret_cast<const Part*>(reinterpret_cast<const uint8_t*>(ring) + 64 * (np % C::NPIECE));
    return u.n >= 0;
  };
  auto done = [&]() {
    __syncwarp();
    if (lane == 0) mbar_arrive(piece_empty(np % C::NPIECE));
    ++np;
  };

  if (warp < 4) {
    setmaxnreg_dec<80>();
    if (warp == 0) {
      // ------------------------------------------------------------- copies
      // A block is one page, part of one, or several; a page of its size comes in one
      // piece, codes and scales together, as they lie in the ring.
      uint32_t c = 0;  // blocks copied
      const uint32_t e = elect_one();
      const int n = min(a.c.page, C::KB), pages = C::KB / n;
      const int per_page = n * (D / 2 + D / 16);
      // Page numbers come 32 at a time, one a lane, and the next 32 are always on their
      // way: a lookup per block would hold the copies up by its latency.
      int base = 0, ids0 = 0, ids1 = 0;
      auto ids_from = [&](int first) {
        const int i = first + lane;
        return i < a.c.max_pages && (int64_t(i) << a.c.log2page) < cur.vis1 ? a.c.table[int64_t(cur.b) * a.c.max_pages + i] : -1;
      };
      auto page_of = [&](int p0) {  // of position p0; -2: nobody sees these positions
        const int i = (p0 >> a.c.log2page) - base;
        const int x = __shfl_sync(0xffffffffu, ids0, i & 31), y = __shfl_sync(0xffffffffu, ids1, i & 31);
        return p0 >= cur.vis1 || p0 + n <= cur.vis0 ? -2 : max(i < 32 ? x : y, -1);
      };
      auto usable = [&](int id) { return id >= 0 && id < a.c.n_pages; };
      auto publish = [&](bool end) {
        const uint32_t s = np % C::NPIECE;
        if (np >= C::NPIECE && !wait(piece_empty(s), np / C::NPIECE + 1, 0xD52u)) return;
        if (lane == 0) {
          Part u;
          u.n = end ? -1 : max(cur.kb1 - cur.kb0, 0);
          u.kb0 = cur.kb0;
          u.vis0 = cur.vis0;
          u.vis1 = cur.vis1;
          u.row0 = cur.rt * C::ROWS;
          u.rows = min(cur.s.rows - u.row0, C::ROWS);
          u.h = cur.h;
          u.len = cur.s.len;
          u.whole = cur.seg0 >= tb && cur.seg1 <= te;
          u.second = tb >= cur.seg0 ? 0 : 1;
          u.q0 = cur.s.q0;
          *reinterpret_cast<Part*>(reinterpret_cast<uint8_t*>(ring) + 64 * s) = u;
          mbar_arrive(piece_full(s));
        }
        __syncwarp();
        ++np;
      };
      for (bool have = true; have && ok;) {
        publish(false);
        base = (cur.kb0 * C::KB) >> a.c.log2page;
        ids0 = ids_from(base);
        ids1 = ids_from(base + 32);
        for (int kb = cur.kb0; kb < cur.kb1 && ok; ++kb) {
          if (((kb * C::KB) >> a.c.log2page) >= base + 32) {
            base += 32;
            ids0 = ids1;
            ids1 = ids_from(base + 32);
          }
          const int p0 = kb * C::KB, in = p0 & (a.c.page - 1);  // position, and its place in a larger page
          uint32_t sum = 0;
          for (int i = 0; i < pages; ++i) {
            const int id = page_of(p0 + i * n);
            if (id != -2 && !usable(id) && __any_sync(0xffffffffu, tile_sees<C>(a, cur, p0 + i * n, p0 + (i + 1) * n, lane, 32)) && e)
              atomicCAS(&slot->err, 0u, uint32_t(SA_ERR_BAD_PAGE));
            if (usable(id)) sum += per_page;
            const int ahead = kb + 4 < cur.kb1 ? page_of(p0 + 4 * C::KB + i * n) : -2;
            if (usable(ahead)) {
              const uint8_t* p = a.c.pool + a.c.record(ahead, cur.h);
              if (a.c.page <= C::KB) {
                l2_prefetch_if(e, p, 2 * a.c.rec);
              } else {
                const int at = (p0 + 4 * C::KB) & (a.c.page - 1);
                l2_prefetch_if(e, p + at * (D / 2), n * (D / 2));
                l2_prefetch_if(e, p + a.c.rec + at * (D / 2), n * (D / 2));
              }
            }
          }
#pragma unroll 1
          for (int kv = 0; kv < 2; ++kv) {
            const uint32_t s = c % C::NR + (kv ? C::NR : 0), dst = sb + C::OFF_RAW + s * C::RAW;
            if (c >= C::NR && !wait(raw_empty(s), c / C::NR + 1, 0xD01u)) break;
            if (e) mbar_arrive_expect_tx(raw_full(s), sum);
            __syncwarp();
            for (int i = 0; i < pages; ++i) {
              const int id = page_of(p0 + i * n);
              if (!usable(id)) continue;
              const uint8_t* rec = a.c.pool + a.c.record(id, cur.h) + kv * a.c.rec;
              if (a.c.page == C::KB) {
                bulk_copy_if(e, dst, rec, per_page, raw_full(s));
              } else {
                bulk_copy_if(e, dst + i * n * (D / 2), rec + in * (D / 2), n * (D / 2), raw_full(s));
                bulk_copy_if(e, dst + C::KB * (D / 2) + i * n * (D / 16), rec + a.c.page * (D / 2) + in * (D / 16), n * (D / 16),
                          raw_full(s));
              }
            }
          }
          ++c;
        }
        have = next_piece<C>(a, cur, lane);
      }
      if (ok) publish(true);
      if (!ok)  // no copy may be in flight when the CTA's shared memory goes
        for (uint32_t s = 0; s < C::NRAW; ++s)  // one phase or the other of each place is the last copy's
          for (uint32_t ph = 0; ph < 2; ++ph) tcc::mbar_wait_bounded(raw_full(s), ph, 1000000ull);
    } else if (warp == 1) {
      // ----------------------------------------------------------- products
      // In order: S and dP of the first two blocks, then, as dS come, dQ and at once S and
      // dP of the block two on, which overwrite them.
      constexpr uint32_t idS = idesc_bf16(128, C::KB, 0, 0);  // Q, dO (K-major) x K^T, V^T (K-major)
      constexpr uint32_t idQ = idesc_bf16(128, D, 0, 1);      // dS (TMEM) x K (MN-major)
      constexpr uint32_t kPart = C::KB * 128;                 // bytes of 64 features of a block
      const uint32_t e = elect_one();
      const uint32_t dq = desc_lo(sb + C::OFF_Q, 16), dd = desc_lo(sb + C::OFF_DO, 16);
      const uint32_t lo_s = desc_lo(sb + C::OFF_RING, 16), lo_q = desc_lo(sb + C::OFF_RING, kPart);
      uint32_t kt = 0, pt = 0, pieces = 0;  // blocks whose scores, and whose dS, are issued
      for (Part un; next(un); done()) {
        const int n = un.n;
        if (n > 0 && !wait(q_full, pieces, 0xD12u)) break;
#pragma unroll 1
        for (int b = 0; b < n + 2 && n > 0; ++b) {
          if (b >= 2) {  // dQ of block b - 2
            const uint32_t g = pt & 1u, s = 2 * (pt % C::NB);
            if (b == 2 && pieces > 0 && !wait(o_empty, pieces - 1, 0xD15u)) break;
            if (!wait(p_full(g), pt >> 1, 0xD13u)) break;
            tc_fence_after();
            const uint32_t dk = lo_q + s * (C::TILE >> 4), more = b > 2;
#pragma unroll
            for (int k = 0; k < C::KB / 16; ++k)
              mma_ts(e, tmem + C::Q_COL, tmem + C::S_COL + 128 * g + 8 * k, dk + ((k * 2048) >> 4), idQ, k == 0 ? more : 1u);
            commit_if(e, slot_empty(s));
            if (b == n + 1) commit_if(e, o_full);
            ++pt;
          }
          if (b < n) {  // S and dP of block b
            const uint32_t g = kt & 1u, s = 2 * (kt % C::NB), tS = tmem + C::S_COL + 128 * g;
            if (!wait(slot_full(s), kt / C::NB, 0xD11u)) break;
            if (!wait(slot_full(s + 1), kt / C::NB, 0xD14u)) break;
            tc_fence_after();
            const uint32_t dk = lo_s + s * (C::TILE >> 4), dv = dk + (C::TILE >> 4);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
              const uint32_t qo = ((k >> 2) * 16384 + (k & 3) * 32) >> 4, ko = ((k >> 2) * kPart + (k & 3) * 32) >> 4;
              mma_ss(e, tS, dq + qo, dk + ko, idS, k > 0 ? 1u : 0u);
              mma_ss(e, tS + 64, dd + qo, dv + ko, idS, k > 0 ? 1u : 0u);
            }
            commit_if(e, s_full(g));
            commit_if(e, slot_empty(s + 1));
            if (b + 1 == n) commit_if(e, q_empty);
            ++kt;
          }
        }
        if (!ok) break;
        pieces += n > 0;
      }
      commit_if(e, drain);  // no product may still run when TMEM is released
      if (e) tcc::mbar_wait_bounded(drain, 0, 200000000ull);
      __syncwarp();
    } else {
      // ---------------------------------------- query rows (2), their gradients (3)
      uint32_t loads = 0;
      for (Part un; next(un); done()) {
        if (un.n == 0) continue;
        if (loads > 0 && !wait(q_empty, loads - 1, 0xD21u)) break;
        ++loads;
        load_rows<D>(warp == 2 ? a.q : a.dout, sb + (warp == 2 ? C::OFF_Q : C::OFF_DO), lane, [&](int r) {
          const int row = un.row0 + r;
          const int64_t t = un.q0 + row / a.G, h = un.h * a.G + row % a.G;
          return r >= un.rows ? int64_t(-1) : warp == 2 ? t * a.q_row + h * a.q_head : (t * a.Hq + h) * D;
        });
        if (lane == 0) mbar_arrive(q_full);
      }
    }
  } else if (warp < 12) {
    setmaxnreg_dec<72>();
    // ------------------------------------------------------- dequantisation
    // Lane (r, q) = (lane / 4, lane % 4) takes a quarter of row 8 w + r: two or four
    // words.  With 128 features the quarters of the two 64-feature halves go in
    // swapped order, so that a store's eight lanes hit eight different banks.
    const int kv = warp >= 8, w = warp & 3, q4 = lane & 3;
    uint32_t c = 0;  // blocks
    for (Part un; next(un); done()) {
#pragma unroll 1
      for (int kb = un.kb0; kb < un.kb0 + un.n; ++kb, ++c) {
        const uint32_t s = 2 * (c % C::NB) + kv, rs = c % C::NR + (kv ? C::NR : 0);
        if (!wait(raw_full(rs), c / C::NR, 0xD31u)) break;
        if (c >= C::NB && !wait(slot_empty(s), c / C::NB + 1, 0xD32u)) break;
        uint8_t* out = smem + C::OFF_RING + s * C::TILE;
        const uint8_t* raw = smem + C::OFF_RAW + rs * C::RAW;
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            const int r = 32 * p + 8 * w + (lane >> 2);
            constexpr int NW = D / 32;
            uint32_t x[NW], code;
            if constexpr (D == 128) {
              const uint4 v = *reinterpret_cast<const uint4*>(raw + r * (D / 2) + q4 * 16);
              x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
              code = *reinterpret_cast<const uint16_t*>(raw + C::KB * (D / 2) + r * (D / 16) + 2 * q4);
              if (q4 & 2) {
                x[0] = v.z, x[1] = v.w, x[2] = v.x, x[3] = v.y;
                code = __byte_perm(code, 0, 0x4401);
              }
            } else {
              const uint2 v = *reinterpret_cast<const uint2*>(raw + r * (D / 2) + q4 * 8);
              x[0] = v.x, x[1] = v.y;
              code = raw[C::KB * (D / 2) + r * (D / 16) + q4];
            }
#pragma unroll
            for (int i = 0; i < NW; ++i) {
              const int word = D == 128 ? (i ^ (q4 & 2)) : i;  // of the lane's quarter
              const int chunk = q4 * NW + word;                // of the row: 8 features, 16 bytes
              uint32_t y[4];
              values_bf16(x[i], scale_bf16(__byte_perm(code, 0, i < 2 ? 0x4040 : 0x4141)), y);
              *reinterpret_cast<uint4*>(out + (chunk >> 3) * (C::KB * 128) + r * 128 + (((chunk & 7) ^ (r & 7)) << 4)) =
                  make_uint4(y[0], y[1], y[2], y[3]);
            }
          }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(slot_full(s));
          mbar_arrive(raw_empty(rs));
        }
      }
    }
  } else {
    setmaxnreg_inc<128>();
    // ----------------------------------------------------- softmax and results
    const int g = (warp - 12) >> 2, quad = warp & 3, i = 32 * quad + lane;  // the row
    const uint32_t lane_off = uint32_t(32 * quad) << 16;
    const uint32_t tS = tmem + lane_off + C::S_COL + 128 * g, tQ = tmem + lane_off + C::Q_COL;
    const float c2 = a.scale * kLog2e;
    const __nv_bfloat16* dout = static_cast<const __nv_bfloat16*>(a.dout);
    const __nv_bfloat16* res = static_cast<const __nv_bfloat16*>(a.out);
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.dq);
    uint32_t t0 = 0, sn = 0, pieces = 0;  // first block of the piece; blocks of this warpgroup
    for (Part un; next(un); done()) {
      const bool whole = un.whole;
      float* part = a.partial + (int64_t(wk) * 2 + un.second) * partial_floats(C::ROWS, D);
      const int r = un.row0 + i;
      // the row's index among the (query, head) pairs, or -1
      const int64_t o = i < un.rows ? (un.q0 + r / a.G) * a.Hq + un.h * a.G + r % a.G : -1;
      // each warpgroup stores half of the columns
      auto put = [&](int col, const float* y, float f) {
        if (o < 0) return;
#pragma unroll
        for (int k = 0; k < 32; k += 8) {
          float z[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) z[e] = y[k + e] * f;
          if (whole)
            store8(out + o * D + col + k, z);
          else
            store8(part + i * D + col + k, z);
        }
      };
      if (un.n == 0) {  // nobody sees anything
        float zero[32] = {};
#pragma unroll 1
        for (int c = g * (D / 2); c < (g + 1) * (D / 2); c += 32) put(c, zero, 0.f);
        continue;
      }
      int lo = 0, hi = 0x7fffffff;
      float L = 0.f, Dr = 0.f;
      if (o >= 0) {
        row_window(a, un.q0 + r / a.G, un.len, lo, hi);
        L = a.lse[o] * kLog2e;
#pragma unroll 1
        for (int c = 0; c < D; c += 8) {
          float x[8], y[8];
          Vec<__nv_bfloat16>::load(dout + o * D + c, x);
          Vec<__nv_bfloat16>::load(res + o * D + c, y);
#pragma unroll
          for (int k = 0; k < 8; ++k) Dr = fmaf(x[k], y[k], Dr);
        }
      }
#pragma unroll 1
      for (int b = int((t0 & 1u) ^ uint32_t(g)); b < un.n; b += 2) {
        const int k0 = (un.kb0 + b) * C::KB;
        if (!wait(s_full(g), sn++, 0xD41u)) break;
        tc_fence_after();
        const bool masked = __any_sync(0xffffffffu, k0 < lo || k0 + C::KB > hi);
#pragma unroll 1
        for (int c = 0; c < C::KB; c += 32) {
          float s[32], p[32];
          tmem_ld32(tS + c, s);
          tmem_ld32(tS + 64 + c, p);
          tmem_ld_wait();
          exp2_shift<32>(s, c2, L);
          uint32_t d[16];
#pragma unroll
          for (int k = 0; k < 32; k += 2) {
            float2 x = __fmul2_rn(make_float2(s[k], s[k + 1]), __fadd2_rn(make_float2(p[k], p[k + 1]), make_float2(-Dr, -Dr)));
            if (masked) {
              if (k0 + c + k < lo || k0 + c + k >= hi) x.x = 0.f;
              if (k0 + c + k + 1 < lo || k0 + c + k + 1 >= hi) x.y = 0.f;
            }
            d[k / 2] = pack_bf16(x.x, x.y);
          }
          tmem_st16(tS + c / 2, d);  // over scores that have been read
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full(g));
      }
      t0 += un.n;
      if (!ok || !wait(o_full, pieces, 0xD42u)) break;
      ++pieces;
      tc_fence_after();
#pragma unroll 1
      for (int c = g * (D / 2); c < (g + 1) * (D / 2); c += 32) {
        float y[32];
        tmem_ld32(tQ + c, y);
        tmem_ld_wait();
        put(c, y, whole ? a.scale : 1.f);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(o_empty);
    }
  }
  __syncthreads();
  if (threadIdx.x == 0 && ctl->abort) {
    slot->err = uint32_t(SA_ERR_TIMEOUT);
    slot->timeout_site = ctl->site;
  }
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc(tmem, C::COLS);
  }
}

template <int D>
static cudaError_t run_bwd(const AttnArgs& a, cudaStream_t st) {
  using C = TcBwd<D>;
  const cudaError_t e =
      cudaFuncSetAttribute(cache_tc_bwd_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
  if (e != cudaSuccess) return e;
  cache_tc_bwd_kernel<D><<<a.ctas, C::THREADS, C::SMEM, st>>>(a);
  const cudaError_t e2 = cudaGetLastError();
  return e2 != cudaSuccess ? e2 : launch_join<C>(a, st);
}

cudaError_t launch_tc_bwd(const AttnArgs& a, cudaStream_t st) { return a.c.d == 128 ? run_bwd<128>(a, st) : run_bwd<64>(a, st); }

}  // namespace cache
}  // namespace sa
