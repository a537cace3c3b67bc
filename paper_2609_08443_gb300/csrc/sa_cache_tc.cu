// Attention over the 4-bit cache on tcgen05, for many queries of a user (the candidates
// of a request, the requests of a training group times the query heads of a cached
// head): bf16, d in {64, 128}, a positive scale.
//
// A CTA holds up to 256 query rows as two halves of 128 and walks 128 cached positions
// at a time.  The products need 16-bit operands in shared memory, so eight warps turn a
// block's 4-bit words into them once for all the rows:
//     S = Q K^T   (M = 128 rows, N = 128 positions, bf16)       accumulated in TMEM
//     P = 2^(S - shift) in registers, float16, back over S in TMEM (its 11 bits leave the
//         result's error where the result's own rounding to bf16 puts it, at 1.7e-3)
//     O += P V    (M = 128, N = d, K = 128 positions, float16; P read from TMEM)
// Dequantising costs about 16 instructions a word of 8 features; spread over 256 rows it
// stays below the products.  The two warpgroups of the softmax take the units (block,
// half) in turn, so that one's exponentials run under the other's products.  A row tile
// of at most 128 rows has one half only: its blocks alternate between the warpgroups,
// each with its own O and shift, and the two are added at the end.
//
// The shift of a row is changed lazily, when a block's maximum passes the shift in use
// by more than 3 (log2 units), and only then is the row of O rescaled in TMEM; S of a
// block is issued after the product that read the warpgroup's last weights, so when it
// arrives O is at rest.
//
// Warp roles: 0 walks the share, publishes its pieces to the other roles and copies the
// pages' codes and scales into a ring (bulk copies), 1 issues the products, 2 and 3 load
// the halves' query rows, 4..11 dequantise, 12..19 softmax and results.  Every wait is
// bounded: past the limit the CTA's roles leave, its copies and products drain and the
// error is reported.
//
// Measured (GB300): 300 queries of 16 users over 10,000 positions, 8 heads of 128, 274 us, 718
// TFLOP/s of a library product's 1894; the warp-level kernel takes 944.  No resource is
// full (tensor pipe 44 %, integer pipe 41 %): a block of 128 positions x 256 rows takes about 2,700
// cycles, and dequantising, exponentials and issue each fill most of them with one
// warp's instructions in a row.  Two issuers, 64 positions with twice the score buffers,
// two CTAs an SM, and loads straight from the pages into registers were all slower.
#include "sa_cache_tc.cuh"

namespace sa {
namespace cache {

constexpr float kLazy = 3.f;  // with kLift = 12 a weight stays below 2^15, inside float16

template <int D_>
struct TcFwd {
  static constexpr int D = D_;
  static constexpr bool F32 = false, BWD = false;
  static constexpr int ROWS = 256, HALF = 128, KB = 128;
  static constexpr int NWARP = 20, THREADS = 640;
  static constexpr int TILE = 128 * D * 2;  // 128 rows of 16-bit values, [D / 64][128][128 bytes]
  // Keys of block t are in place 2 (t % 2) of the ring, its values in the next: a lone
  // half runs two blocks of scores ahead of its weights.
  static constexpr int NSLOT = 4, NRAW = D == 128 ? 3 : 8;
  static constexpr int RAW = KB * (D / 2 + D / 16);
  static constexpr int OFF_Q = 0;
  static constexpr int OFF_RING = OFF_Q + 2 * TILE;
  static constexpr int OFF_SCAN = OFF_RING;  // used before anything is dequantised
  static constexpr int OFF_RAW = OFF_RING + NSLOT * TILE;
  static constexpr int OFF_X = OFF_RAW + NRAW * RAW;  // a warpgroup's shifts and sums for the other
  static constexpr int X_BYTES = 128 * 8;
  static constexpr int OFF_BAR = OFF_X + X_BYTES;
  static constexpr int NPIECE = 4;    // pieces published ahead
  static constexpr int NREADER = 19;  // warps that read them
  static constexpr int NBAR = 2 * NSLOT + 2 * NRAW + 2 * 6 + 2 + 2 * NPIECE;
  static constexpr int OFF_PIECE = (OFF_BAR + NBAR * 8 + 15) / 16 * 16;
  static constexpr int OFF_CTL = OFF_PIECE + NPIECE * 64;
  static constexpr int OFF_TMEM = OFF_CTL + 16;
  static constexpr int SMEM = OFF_TMEM + 16;
  static_assert(SMEM <= 232448, "shared memory budget");
  static constexpr int S_COL = 0, O_COL = 256;  // two halves each
};

// A piece as the roles see it (64 bytes of shared memory).  Units, (block, half) pairs,
// alternate between the warpgroups over the whole share; `parity` is the first one's.
struct Units {
  int n;         // blocks; -1: the share is done
  int halves;    // 1 or 2
  int parity;
  int kb0;       // first block
  int rows;      // of the tile
  int row0;      // of the tile within the user's rows of this head
  int h, len;
  int whole;     // the segment lies within this share
  int second;    // which of the worker's two unfinished pieces it is, if not whole
  int64_t q0;    // the user's first query
  __device__ __forceinline__ int count() const { return n * halves; }
  // warpgroup wg's blocks: first, first + step, ...
  __device__ __forceinline__ int first(int wg) const { return halves == 2 ? 0 : wg ^ parity; }
  __device__ __forceinline__ int step() const { return halves == 2 ? 1 : 2; }
  __device__ __forceinline__ int mine(int wg) const { return n > first(wg) ? (n - first(wg) + step() - 1) / step() : 0; }
  // the half of the rows that warpgroup wg has
  __device__ __forceinline__ int half(int wg) const { return halves == 2 ? wg ^ parity : 0; }
};
static_assert(sizeof(Units) <= 64, "one slot of the piece ring");

template <int D>
__global__ void __launch_bounds__(640, 1) cache_tc_fwd_kernel(const __grid_constant__ AttnArgs a) {
  using C = TcFwd<D>;
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
  auto s_full = [&](int g) { return per + 8u * g; };
  auto p_full = [&](int g) { return per + 8u * (2 + g); };
  auto o_full = [&](int g) { return per + 8u * (4 + g); };
  auto o_empty = [&](int g) { return per + 8u * (6 + g); };
  auto q_full = [&](int g) { return per + 8u * (8 + g); };
  auto q_empty = [&](int g) { return per + 8u * (10 + g); };
  const uint32_t x_full = per + 8u * 12, drain = per + 8u * 13;
  auto piece_full = [&](uint32_t s) { return per + 8u * (14 + s); };
  auto piece_empty = [&](uint32_t s) { return per + 8u * (14 + C::NPIECE + s); };

  if (threadIdx.x == 0) {
    for (int i = 0; i < C::NBAR; ++i) {
      const int p = i - 2 * C::NSLOT - 2 * C::NRAW;  // barriers of the halves
      uint32_t n = 1;
      if (i < C::NSLOT) n = 8;                                                       // slot_full: the dequantising warps
      if (i >= 2 * C::NSLOT + C::NRAW && i < 2 * C::NSLOT + 2 * C::NRAW) n = 8;      // raw_empty
      if (p == 2 || p == 3 || p == 6 || p == 7 || p == 12) n = 4;         // a softmax warpgroup's warps
      if (p >= 14 + C::NPIECE) n = C::NREADER;                                       // piece_empty
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
  if (warp == 2) tmem_alloc(smem_u32(tmem_slot), 512);
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

  Units* ring = reinterpret_cast<Units*>(smem + C::OFF_PIECE);
  uint32_t np = 0;  // pieces read (or published) so far
  // the next piece; done() gives its place back
  auto next = [&](Units& u) {
    if (!wait(piece_full(np % C::NPIECE), np / C::NPIECE, 0xD51u)) return false;
    u = *reinterpret_cast<const Units*>(reinterpret_cast<const uint8_t*>(ring) + 64 * (np % C::NPIECE));
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
      // lane 2 p + i copies the codes (i = 0) or scales of the block's p-th page
      uint32_t c = 0;  // keys and values of block after block
      const int n = min(a.c.page, C::KB), part = lane & 1, off = (lane >> 1) * n;
      const int rb = part ? D / 16 : D / 2;
      auto holds = [&](const Walk& w, int kb) {  // whether the lane's page of the block has positions that may be seen
        const int p0 = kb * C::KB + off;
        return off < C::KB && kb < w.kb1 && p0 < w.vis1 && p0 + n > w.vis0;
      };
      auto page_of = [&](const Walk& w, int kb) {
        return holds(w, kb) ? a.c.table[int64_t(w.b) * a.c.max_pages + ((kb * C::KB + off) >> a.c.log2page)] : -1;
      };
      int parity = 0;
      auto publish = [&](bool end) {
        const uint32_t s = np % C::NPIECE;
        if (np >= C::NPIECE && !wait(piece_empty(s), np / C::NPIECE + 1, 0xD52u)) return;
        if (lane == 0) {
          Units u;
          u.n = end ? -1 : max(cur.kb1 - cur.kb0, 0);
          u.halves = cur.weight;
          u.parity = parity;
          u.kb0 = cur.kb0;
          u.row0 = cur.rt * C::ROWS;
          u.rows = min(cur.s.rows - u.row0, C::ROWS);
          u.h = cur.h;
          u.len = cur.s.len;
          u.whole = cur.seg0 >= tb && cur.seg1 <= te;
          u.second = tb >= cur.seg0 ? 0 : 1;
          u.q0 = cur.s.q0;
          *reinterpret_cast<Units*>(reinterpret_cast<uint8_t*>(ring) + 64 * s) = u;
          mbar_arrive(piece_full(s));
        }
        __syncwarp();
        ++np;
        if (!end) parity = (parity + max(cur.kb1 - cur.kb0, 0) * cur.weight) & 1;
      };
      for (bool have = true; have && ok;) {
        publish(false);
        // the pages of this block and the next two; two blocks ahead go to L2
        int pid = page_of(cur, cur.kb0), pid1 = page_of(cur, cur.kb0 + 1), pid2 = page_of(cur, cur.kb0 + 2);
        for (int kb = cur.kb0; kb < cur.kb1 && ok; ++kb) {
          const bool want = pid >= 0 && pid < a.c.n_pages;
          const int64_t rec = want ? a.c.record(pid, cur.h) : 0;
          const int first = (kb * C::KB + off) & (a.c.page - 1);
          const uint32_t bytes = want ? uint32_t(n * rb) : 0u;
          // the block's bytes, and above them how many of its pages are missing
          const bool missing = !want && !part && holds(cur, kb);
          uint32_t sum = __reduce_add_sync(0xffffffffu, bytes | uint32_t(missing) << 24);
          if (sum >> 24) {
            for (uint32_t m = __ballot_sync(0xffffffffu, missing); m; m &= m - 1) {
              const int p0 = kb * C::KB + ((__ffs(m) - 1) >> 1) * n;
              if (__any_sync(0xffffffffu, tile_sees<C>(a, cur, p0, p0 + n, lane, 32)) && lane == 0)
                atomicCAS(&slot->err, 0u, uint32_t(SA_ERR_BAD_PAGE));
            }
            sum &= 0xFFFFFFu;
          }
          if (pid2 >= 0 && pid2 < a.c.n_pages) {
            const uint8_t* p = a.c.pool + a.c.record(pid2, cur.h) + (part ? a.c.page * (D / 2) : 0) +
                               (((kb + 2) * C::KB + off) & (a.c.page - 1)) * rb;
            l2_prefetch(p, n * rb);
            l2_prefetch(p + a.c.rec, n * rb);
          }
          pid = pid1;
          pid1 = pid2;
          pid2 = page_of(cur, kb + 3);
          for (int kv = 0; kv < 2; ++kv, ++c) {
            const uint32_t s = c % C::NRAW;
            if (c >= C::NRAW && !wait(raw_empty(s), c / C::NRAW + 1, 0xD01u)) break;
            if (lane == 0) mbar_arrive_expect_tx(raw_full(s), sum);
            __syncwarp();
            if (want)
              bulk_copy(sb + C::OFF_RAW + s * C::RAW + (part ? C::KB * (D / 2) : 0) + off * rb,
                        a.c.pool + rec + kv * a.c.rec + (part ? a.c.page * (D / 2) : 0) + first * rb, bytes, raw_full(s));
          }
        }
        have = next_piece<C>(a, cur, lane);
      }
      if (ok) publish(true);
      if (!ok)  // no copy may be in flight when the CTA's shared memory goes
        for (uint32_t k = c > C::NRAW ? c - C::NRAW : 0; k < c; ++k)
          tcc::mbar_wait_bounded(raw_full(k % C::NRAW), (k / C::NRAW) & 1u, 200000000ull);
    } else if (warp == 1) {
      // ----------------------------------------------------------- products
      constexpr uint32_t idS = idesc_bf16(128, C::KB, 0, 0);  // Q (K-major) x K^T (K-major)
      constexpr uint32_t idO = idesc_f16(128, D, 0, 1);       // P (TMEM) x V (MN-major)
      const uint32_t e = elect_one();
      const uint32_t lo_q = desc_lo(sb + C::OFF_Q, 16), lo_k = desc_lo(sb + C::OFF_RING, 16);
      const uint32_t lo_v = desc_lo(sb + C::OFF_RING, 16384);
      uint32_t kt = 0, vt = 0;            // blocks whose scores, and whose weights, are issued
      uint32_t qph = 0, pph = 0, oph = 3; // phases, bit g for warpgroup g
      uint32_t seen = 0;                  // warpgroups that have had a piece: the first does not wait for O
      for (Units un; next(un); done()) {
        // Units alternate between the warpgroups; S runs two units ahead of O, and the last
        // two units' products are issued before the next piece is looked at: the walk may
        // be waiting for what they release.
        const int total = un.count(), two = un.halves == 2;
#pragma unroll 1
        for (int i = 0; i < total + 2 && total > 0; ++i) {
          const uint32_t g = uint32_t(un.parity + i) & 1u;  // also of unit i - 2
          if (i >= 2) {  // O of unit i - 2
            const int j = i - 2;
            const uint32_t vs = 2 * (vt & 1u) + 1;
            if (!wait(slot_full(vs), vt >> 1, 0xD14u)) break;
            if (j < 2) {  // the warpgroup's first of the piece
              if (((seen >> g) & 1u) && !wait(o_empty(g), oph >> g, 0xD15u)) break;
              seen |= 1u << g;
              oph ^= 1u << g;
            }
            if (!wait(p_full(g), pph >> g, 0xD13u)) break;
            pph ^= 1u << g;
            tc_fence_after();
            const uint32_t dv = lo_v + vs * (C::TILE >> 4), dst = tmem + C::O_COL + g * 128, src = tmem + C::S_COL + g * 128;
#pragma unroll
            for (int s = 0; s < C::KB / 16; ++s)
              mma_ts(e, dst, src + 8 * s, dv + ((s * 2048) >> 4), idO, s == 0 ? uint32_t(j >= 2) : 1u);
            if (!two || (j & 1)) {
              commit_if(e, slot_empty(vs));
              ++vt;
            }
            if (j + 2 >= total) commit_if(e, o_full(g));
          }
          if (i < total) {  // S of unit i
            const uint32_t ks = 2 * (kt & 1u);
            if ((!two || !(i & 1)) && !wait(slot_full(ks), kt >> 1, 0xD11u)) break;
            if (i < 2) {
              if (!wait(q_full(g), qph >> g, 0xD12u)) break;
              qph ^= 1u << g;
            }
            tc_fence_after();
            const uint32_t dq = lo_q + g * (C::TILE >> 4), dk = lo_k + ks * (C::TILE >> 4), dst = tmem + C::S_COL + g * 128;
#pragma unroll
            for (int s = 0; s < D / 16; ++s) {
              const uint32_t at = ((s >> 2) * 16384 + (s & 3) * 32) >> 4;
              mma_ss(e, dst, dq + at, dk + at, idS, s > 0 ? 1u : 0u);
            }
            commit_if(e, s_full(g));
            if (i + 2 >= total) commit_if(e, q_empty(g));
            if (!two || (i & 1)) {
              commit_if(e, slot_empty(ks));
              ++kt;
            }
          }
        }
        if (!ok) break;
      }
      commit_if(e, drain);  // no product may still run when TMEM is released
      if (e) tcc::mbar_wait_bounded(drain, 0, 200000000ull);
      __syncwarp();
    } else {
      // ------------------------------------------------- query rows of half `g`
      const int g = warp - 2;
      uint32_t loads = 0;
      for (Units un; next(un); done()) {
        if (un.mine(g) == 0) continue;
        if (loads > 0 && !wait(q_empty(g), loads - 1, 0xD21u)) break;
        const int r0 = un.half(g) * 128;
        load_rows<D>(a.q, sb + C::OFF_Q + g * C::TILE, lane, [&](int r) {
          const int row = un.row0 + r0 + r;
          return r0 + r < un.rows ? (un.q0 + row / a.G) * a.q_row + (un.h * a.G + row % a.G) * a.q_head : int64_t(-1);
        });
        if (lane == 0) mbar_arrive(q_full(g));
        ++loads;
      }
    }
  } else if (warp < 12) {
    setmaxnreg_dec<64>();
    // ------------------------------------------------------- dequantisation
    // Lane (r, q) = (lane / 4, lane % 4) takes a quarter of rows 8 w + r, 64 on: two or four
    // words.  With 128 features the quarters of the two 64-feature halves go in
    // swapped order, so that a store's eight lanes hit eight different banks.
    // All eight warps take each place of the ring in turn, keys, then values: the places
    // are shared, and a warpgroup that left every other one to its neighbour could take a
    // place's last phase but one for the one it waits for.
    const int w = warp - 4, q4 = lane & 3;
    uint32_t c = 0;
    for (Units un; next(un); done()) {
#pragma unroll 1
      for (int i = 0; i < 2 * un.n; ++i, ++c) {
        const int kv = i & 1;
        const uint32_t rs = c % C::NRAW, s = c % C::NSLOT;
        if (!wait(raw_full(rs), c / C::NRAW, 0xD31u)) break;
        if (c >= C::NSLOT && !wait(slot_empty(s), c / C::NSLOT + 1, 0xD32u)) break;
        const uint8_t* raw = smem + C::OFF_RAW + rs * C::RAW;
        uint8_t* out = smem + C::OFF_RING + s * C::TILE;
        // hidden positions' bytes may be nobody's, which float16 may read as infinities
        auto rows = [&](auto f16, auto values) {
#pragma unroll 1
          for (int p = 0; p < 2; ++p) {
            const int r = 64 * p + 8 * w + (lane >> 2);
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
            if (f16 && ((code & 255u) > kCodeSafe || (code >> 8) > kCodeSafe)) {
              code = ((code & 255u) > kCodeMax ? 0u : code & 255u) | ((code >> 8) > kCodeMax ? 0u : code & 0xFF00u);
#pragma unroll
              for (int i = 0; i < NW; ++i) x[i] = level_min7(x[i]);
            }
#pragma unroll
            for (int i = 0; i < NW; ++i) {
              const int word = D == 128 ? (i ^ (q4 & 2)) : i;  // of the lane's quarter
              const int chunk = q4 * NW + word;                // of the row: 8 features, 16 bytes
              uint32_t y[4];
              values(x[i], __byte_perm(code, 0, i < 2 ? 0x4040 : 0x4141), y);
              *reinterpret_cast<uint4*>(out + (chunk >> 3) * 16384 + r * 128 + (((chunk & 7) ^ (r & 7)) << 4)) =
                  make_uint4(y[0], y[1], y[2], y[3]);
            }
          }
        };
        if (kv)
          rows(std::true_type{}, [](uint32_t x, uint32_t cc, uint32_t* y) { values_f16(x, cc << 7, y); });
        else
          rows(std::false_type{}, [](uint32_t x, uint32_t cc, uint32_t* y) { values_bf16(x, scale_bf16(cc), y); });
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(slot_full(s));
          mbar_arrive(raw_empty(rs));
        }
      }
    }
  } else {
    setmaxnreg_inc<136>();
    // ----------------------------------------------------- softmax and results
    const int g = (warp - 12) >> 2, quad = warp & 3, rr = 32 * quad + lane;
    const uint32_t lane_off = uint32_t(32 * quad) << 16;
    const uint32_t tS = tmem + lane_off + C::S_COL + g * 128, tO = tmem + lane_off + C::O_COL + g * 128;
    const float c2 = a.scale * kLog2e;
    float2* X = reinterpret_cast<float2*>(smem + C::OFF_X);
    uint32_t sn = 0, pieces = 0, xn = 0;
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out);
    for (Units un; next(un); done()) {
      const int mine = un.mine(g);
      const bool whole = un.whole;
      float* part = a.partial + (int64_t(wk) * 2 + un.second) * partial_floats(C::ROWS, D);
      // row i of the tile: its index among the (query, head) pairs, or -1
      auto dense = [&](int i) {
        const int r = un.row0 + i;
        return i < un.rows ? (un.q0 + r / a.G) * a.Hq + un.h * a.G + r % a.G : int64_t(-1);
      };
      // 32 columns of one row, unnormalised or final
      auto put = [&](int i, int64_t o, int col, const float* y, float f) {
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
      auto put_stat = [&](int i, int64_t o, float m, float l) {
        if (o < 0) return;
        if (!whole)
          *reinterpret_cast<float2*>(part + C::ROWS * D + 2 * i) = make_float2(m, l);
        else if (a.lse)
          a.lse[o] = l == 0.f ? -INFINITY : (m + log2f(l) - kLift) * kLn2;
      };
      if (un.n == 0 && g == 0) {  // nobody sees anything
        float zero[32] = {};
#pragma unroll 1
        for (int hf = 0; hf < un.halves; ++hf) {
          const int i = 128 * hf + rr;
          const int64_t o = dense(i);
#pragma unroll 1
          for (int col = 0; col < D; col += 32) put(i, o, col, zero, 0.f);
          put_stat(i, o, -INFINITY, 0.f);
        }
      }
      if (mine > 0) {
        const int i = 128 * un.half(g) + rr;
        int lo = 0, hi = 0x7fffffff;
        const int64_t o = dense(i);
        if (o >= 0) row_window(a, un.q0 + (un.row0 + i) / a.G, un.len, lo, hi);
        float msh = -INFINITY, l = 0.f;
        for (int b = 0; b < mine; ++b) {
          const int k0 = (un.kb0 + un.first(g) + b * un.step()) * C::KB;
          if (!wait(s_full(g), sn++, 0xD41u)) break;
          tc_fence_after();
          const bool masked = __any_sync(0xffffffffu, k0 < lo || k0 + C::KB > hi);
          // 32 columns at a time, twice: for the maximum and for the weights (a second
          // read of TMEM costs less than the registers and the code of a whole row)
          float v[32];
          auto load = [&](int c) {
            tmem_ld32(tS + c, v);
            tmem_ld_wait();
            if (masked) {
              const int from = lo - k0 - c, to = hi - k0 - c;
#pragma unroll
              for (int k = 0; k < 32; ++k)
                if (k < from || k >= to) v[k] = -INFINITY;
            }
          };
          float mt = -INFINITY;
#pragma unroll 1
          for (int c = 0; c < C::KB; c += 32) {
            load(c);
            mt = fmaxf(mt, row_max<32>(v));
          }
          mt *= c2;
          float alpha = 1.f;
          if (msh == -INFINITY) {
            msh = mt;  // O and l are zero so far
          } else if (mt > msh + kLazy) {
            alpha = ex2(msh - mt);
            msh = mt;
          }
          // nothing seen yet: any shift gives zeros
          const float sh = msh == -INFINITY ? 0.f : msh - kLift;
          l *= alpha;
#pragma unroll 1
          for (int c = 0; c < C::KB; c += 32) {
            load(c);
            l += exp2_shift_sum<32>(v, c2, sh);
            uint32_t p[16];
#pragma unroll
            for (int k = 0; k < 16; ++k)
              asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(p[k]) : "f"(v[2 * k + 1]), "f"(v[2 * k]));
            tmem_st16(tS + c / 2, p);  // over columns that have been read
          }
          if (b > 0 && __any_sync(0xffffffffu, alpha != 1.f)) {
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
              float y[32];
              tmem_ld32(tO + c, y);
              tmem_ld_wait();
#pragma unroll
              for (int k = 0; k < 32; ++k) y[k] *= alpha;
              tmem_st16(tO + c, reinterpret_cast<const uint32_t*>(y));
              tmem_st16(tO + c + 16, reinterpret_cast<const uint32_t*>(y) + 16);
            }
          }
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(p_full(g));
        }
        if (!ok || !wait(o_full(g), pieces, 0xD42u)) break;
        ++pieces;
        tc_fence_after();
        // The other warpgroup has the other blocks' share of these rows: one of the two
        // leaves its shifts and sums in X, and the other, whose warps read the same lanes
        // of TMEM, adds and stores.
        const bool both = un.halves == 1 && un.n > 1;
        if (both && un.first(g) == 1) {
          X[rr] = make_float2(msh, l);
          ++xn;
          __syncwarp();
          if (lane == 0) mbar_arrive(x_full);
          continue;  // the other warpgroup gives O back
        }
        float m = msh, f0 = 1.f, f1 = 0.f;
        if (both) {
          if (!wait(x_full, xn++, 0xD44u)) break;
          tc_fence_after();
          const float2 s = X[rr];
          m = fmaxf(msh, s.x);
          f0 = msh == -INFINITY ? 0.f : ex2(msh - m);
          f1 = s.x == -INFINITY ? 0.f : ex2(s.x - m);
          l = l * f0 + s.y * f1;
        }
        const float f = !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
        f0 *= f;
        f1 *= f;
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          float y[32];
          tmem_ld32(tO + c, y);
          tmem_ld_wait();
          if (both) {
            float z[32];
            tmem_ld32(tmem + lane_off + C::O_COL + (g ^ 1) * 128 + c, z);
            tmem_ld_wait();
#pragma unroll
            for (int k = 0; k < 32; ++k) y[k] = y[k] * f0 + z[k] * f1;
          }
          put(i, o, c, y, both ? 1.f : f0);
        }
        put_stat(i, o, m, l);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(o_empty(g));
          if (both) mbar_arrive(o_empty(g ^ 1));
        }
      }
    }
  }
  __syncthreads();
  if (threadIdx.x == 0 && ctl->abort) {
    slot->err = uint32_t(SA_ERR_TIMEOUT);
    slot->timeout_site = ctl->site;
  }
  if (warp == 2) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <int D>
static cudaError_t run_fwd(const AttnArgs& a, cudaStream_t st) {
  using C = TcFwd<D>;
  const cudaError_t e =
      cudaFuncSetAttribute(cache_tc_fwd_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
  if (e != cudaSuccess) return e;
  cache_tc_fwd_kernel<D><<<a.ctas, C::THREADS, C::SMEM, st>>>(a);
  const cudaError_t e2 = cudaGetLastError();
  return e2 != cudaSuccess ? e2 : launch_join<C>(a, st);
}

// Taken from so many rows (queries times query heads) of an average user for a cached
// head: the tcgen05 kernels take about the same time up to 128 rows, the warp-level ones go up by
// 16.  Measured on a GB300, us (tcgen05 | warp-level), 16 users x 8 heads x 10,000 positions:
//     rows                 16          32          48          64          128
//     forward, d = 128     112 |  76   113 | 122   115 | 173   116 | 224   123 | 423
//     forward, d = 64      104 |  51   104 |  82   105 | 113   106 | 144   111 | 269
//     gradient, d = 128    177 | 101   178 | 164   180 | 233   182 | 302   188 | 571
//     gradient, d = 64     169 |  60   169 |  99   169 | 139   170 | 177   174 | 333
// and the same order at 64 users x 4 heads x 1024 (forward, d = 128: 42 | 46 at 32 rows; gradient: 52
// | 55).  The forward takes its maximum on the raw scores, so its scale is positive.
bool tc_supported(int B, int64_t T, int G, int d, sa_dtype dt, float scale, bool bwd) {
  if (dt != SA_BF16 || (d != 64 && d != 128) || (!bwd && !(scale > 0.f))) return false;
  const int64_t rows = d == 128 ? (bwd ? 40 : 32) : (bwd ? 56 : 40);
  return T * G >= rows * B && tcc::device_is_sm103();
}

AttnPlan tc_plan(int sms, int d, bool bwd) {
  AttnPlan p;
  p.ctas = p.workers = sms;
  p.piece_bytes = sizeof(Piece);
  p.partial_floats = partial_floats(bwd ? 128 : 256, d);
  return p;
}

cudaError_t launch_tc(const AttnArgs& a, bool bwd, cudaStream_t st) {
  if (bwd) return launch_tc_bwd(a, st);
  return a.c.d == 128 ? run_fwd<128>(a, st) : run_fwd<64>(a, st);
}

}  // namespace cache
}  // namespace sa
