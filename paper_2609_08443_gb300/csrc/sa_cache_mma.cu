// Attention over the 4-bit cache with warp-level tensor-core products: the form for
// few queries (serving's single tokens), for fp32 and for every width.
//
// One warp is one worker.  It owns 16 query rows (a user's queries times the query
// heads that share a cached head) and walks 64 cached positions at a time:
//     S = Q K^T  (m16n8k16)  ->  online softmax in registers  ->  O += P V  (m16n8k16)
// The 4-bit words go from shared memory straight into the B operands' registers:
//   - for Q K^T lane (g, t) = (lane / 4, lane % 4) takes key g's features
//     [D/4 t, D/4 (t+1)): the contraction order is free, so Q's fragments are laid
//     out the same way once per segment;
//   - for P V it takes four keys' features of column group g; a byte permute puts
//     two keys' words side by side and the same masks give the pairs (k, k+1) that
//     the operand wants.  S's accumulators are P's A operand as they stand.
// So nothing is stored dequantised, and a cached byte costs one bulk copy and one
// shared-memory read per product.  With one query per user the call is bound by
// reading the cache: 144 bytes a key and head at d = 128.
//
// Work is the list of (user, cached head, 16-row tile, 64-position block), cut into
// equal contiguous shares; a segment cut by share borders leaves unfinished
// (O, max, sum) pieces that the join kernel adds in order.  Every CTA scans the
// users' lengths itself, so a call is two launches.
#include <type_traits>

#include "sa_cache.cuh"
#include "sa_kernels.cuh"
#include "sa_ptx.cuh"

namespace sa {
namespace cache {

using namespace ptx;

constexpr int KB = 64;       // positions per block
constexpr int ROWS = 16;     // query rows per tile
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// Weights are kept as 2^12 exp(S - max): float16 then holds weights down to 2^-26 of
// the largest in full precision.
constexpr float kLift = 12.f;

template <int D_, bool F32_, bool BWD_>
struct Cfg {
  static constexpr int D = D_;
  static constexpr bool F32 = F32_, BWD = BWD_;
  static constexpr int NS = F32 ? 3 : 1;   // bf16 terms of a query or gradient element
  static constexpr int NP = F32 ? 2 : 1;   // float16 terms of a weight
  static constexpr int LW = D / 32;        // words of 8 features a lane holds of a key
  static constexpr int KS = D / 16;        // contraction steps
  static constexpr int NT = D / 8;         // column tiles of the output
  static constexpr int FRAG = KS * 32 * 16;
  static constexpr int FRAGS = FRAG * NS * (BWD ? 2 : 1);
  static constexpr int STAGE = KB * 2 * (D / 2 + D / 16);
  static constexpr int WARP_SMEM = FRAGS + 2 * STAGE;
  static constexpr int NWARP = BWD ? (F32 ? (D == 128 ? 4 : 8) : (D == 128 ? 8 : 12))
                                   : (F32 ? (D == 128 ? 6 : 8) : (D == 128 ? 8 : 12));
  static constexpr int THREADS = NWARP * 32;
  static constexpr int OFF_BAR = NWARP * WARP_SMEM + 128;  // the last lanes of a narrow row may read past a stage
  static constexpr int OFF_SCAN = OFF_BAR + NWARP * 16;
  static constexpr int OFF_CTL = OFF_SCAN + (THREADS + 2) * 8;
  static constexpr int SMEM = OFF_CTL + 16;
  static_assert(SMEM <= 232448, "shared memory budget");
};

// Partial of one piece: 16 rows of D sums, then 16 (max, sum) pairs.
__host__ __device__ constexpr int partial_floats(int D) { return ROWS * D + ROWS * 2; }

// Shares of a call with `total` tiles: none is empty.
__device__ __forceinline__ int shares(const AttnArgs& a, int64_t total) { return int(total < a.workers ? total : a.workers); }

struct Piece {  // what a worker's first segment is, for the join
  int64_t seg0, seg1;
  int b, h, rt, pad;
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

// Column c of an 8-key tile is this key of the tile: pairs differ in parity and the
// even columns hold two even and two odd keys, so the reads of K (two keys a phase)
// and of V (four keys a phase) spread over the shared-memory banks.
__device__ __forceinline__ int key_of(int c) { return c ^ ((c >> 1) & 1); }

// ------------------------------------------------------------------ the walk
// One worker's share of one segment.  Uniform over the warp.
struct Walk {
  int64_t t, te;          // next tile, end of the share
  int64_t seg0, seg1;     // tiles of the segment
  int b, h, rt;
  int nrt, nkb, rows, len;
  int64_t q0;             // first query of the user
  int vis0, vis1;         // positions that some row of the tile sees
  int kb0, kb1;           // blocks of this piece (empty: kb0 >= kb1)
};

struct Sizes {
  int64_t tiles;
  int nrt, nkb, rows, len;
  int64_t q0;
};
__device__ __forceinline__ Sizes user_sizes(const AttnArgs& a, int b) {
  Sizes s;
  const int c0 = a.cu_q[b], c1 = a.cu_q[b + 1];
  s.q0 = c0;
  s.len = a.lens[b];
  s.rows = (c1 - c0) * a.G;
  s.nrt = (s.rows + ROWS - 1) / ROWS;
  s.nkb = s.len > 0 ? (s.len + KB - 1) / KB : 1;  // a user with nothing cached still gets its zeros
  s.tiles = int64_t(s.nrt) * s.nkb * a.c.H;
  return s;
}

__device__ __forceinline__ void row_window(const AttnArgs& a, int64_t t, int len, int& lo, int& hi) {
  lo = a.begin ? max(a.begin[t], 0) : 0;
  hi = a.end ? min(a.end[t], len) : len;
}

// The piece that starts at tile w.t of user w.b (sizes in s).
__device__ __forceinline__ void set_piece(const AttnArgs& a, Walk& w, const Sizes& s, int64_t rem, int lane) {
  w.nrt = s.nrt;
  w.nkb = s.nkb;
  w.rows = s.rows;
  w.len = s.len;
  w.q0 = s.q0;
  const int64_t per_head = int64_t(s.nrt) * s.nkb;
  w.h = int(rem / per_head);
  const int64_t r2 = rem - w.h * per_head;
  w.rt = int(r2 / s.nkb);
  const int kb = int(r2 - int64_t(w.rt) * s.nkb);
  w.seg0 = w.t - kb;
  w.seg1 = w.seg0 + s.nkb;
  w.vis0 = 0;
  w.vis1 = w.len;
  if (a.begin || a.end) {
    int lo = 0x7fffffff, hi = 0;
    const int r = w.rt * ROWS + (lane & (ROWS - 1));
    if (r < w.rows) {
      int l, e;
      row_window(a, w.q0 + r / a.G, w.len, l, e);
      if (l < e) {
        lo = l;
        hi = e;
      }
    }
    w.vis0 = __reduce_min_sync(0xffffffffu, lo);
    w.vis1 = __reduce_max_sync(0xffffffffu, hi);
  }
  const int64_t last = w.te < w.seg1 ? w.te : w.seg1;
  w.kb0 = max(kb, w.vis0 / KB);
  w.kb1 = min(int(last - w.seg0), (w.vis1 + KB - 1) / KB);
  if (w.vis0 >= w.vis1) w.kb1 = w.kb0;
}

// Move to the next piece of the share; false at its end.
__device__ __forceinline__ bool next_piece(const AttnArgs& a, Walk& w, int lane) {
  w.t = w.te < w.seg1 ? w.te : w.seg1;
  if (w.t >= w.te) return false;
  Sizes s;
  int64_t rem;
  if (w.rt + 1 < w.nrt || w.h + 1 < a.c.H) {
    s.nrt = w.nrt;
    s.nkb = w.nkb;
    s.rows = w.rows;
    s.len = w.len;
    s.q0 = w.q0;
    rem = (int64_t(w.h) * w.nrt + w.rt + 1) * w.nkb;
  } else {
    int b = w.b + 1;
    for (;;) {  // the next user with queries (one exists: tiles are left)
      const int u = b + lane;
      const bool has = u < a.B && a.cu_q[u + 1] > a.cu_q[u];
      const uint32_t m = __ballot_sync(0xffffffffu, has);
      if (m) {
        b += __ffs(m) - 1;
        break;
      }
      b += 32;
      if (b >= a.B) return false;
    }
    w.b = b;
    s = user_sizes(a, b);
    rem = 0;
  }
  set_piece(a, w, s, rem, lane);
  return true;
}

// Exclusive scan of the users' tiles over the CTA's threads (each takes `chunk`
// consecutive users) into pre[0..THREADS]; returns the total, or -1 where offsets or
// lengths are out of order.
template <int THREADS>
__device__ int64_t scan_users(const AttnArgs& a, int64_t* pre, int chunk) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int b0 = tid * chunk, b1 = min(a.B, b0 + chunk);
  int64_t sum = 0;
  int bad = 0;
  const int64_t most = int64_t(a.c.max_pages) << a.c.log2page;
  for (int b = b0; b < b1; ++b) {
    const int c0 = a.cu_q[b], c1 = a.cu_q[b + 1], len = a.lens[b];
    if (c0 > c1 || (b == 0 && c0 != 0) || (b == a.B - 1 && int64_t(c1) != a.T) || len < 0 || len > most) bad = 1;
    sum += user_sizes(a, b).tiles;
  }
  int64_t inc = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t v = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += v;
  }
  __shared__ int64_t warp_sum[32];
  if (lane == 31) warp_sum[warp] = inc;
  bad = __syncthreads_or(bad);
  int64_t before = 0, total = 0;
  for (int i = 0; i < THREADS / 32; ++i) {
    if (i < warp) before += warp_sum[i];
    total += warp_sum[i];
  }
  pre[tid] = before + inc - sum;
  if (tid == 0) pre[THREADS] = total;
  __syncthreads();
  return bad ? -1 : total;
}

// The user of tile t and the tile's rank among the user's.
template <int THREADS>
__device__ void find_tile(const AttnArgs& a, const int64_t* pre, int chunk, int64_t t, int lane, int& b, int64_t& rem) {
  int lo = 0, hi = THREADS - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (pre[mid] <= t) lo = mid; else hi = mid - 1;
  }
  int64_t at = pre[lo];
  for (int b0 = lo * chunk;; b0 += 32) {
    const int u = b0 + lane;
    const int64_t mine = u < a.B && u < (lo + 1) * chunk ? user_sizes(a, u).tiles : 0;
    int64_t inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += v;
    }
    const uint32_t m = __ballot_sync(0xffffffffu, at + inc > t);
    if (m) {
      const int l = __ffs(m) - 1;
      b = b0 + l;
      rem = t - at - __shfl_sync(0xffffffffu, inc - mine, l);
      return;
    }
    at += __shfl_sync(0xffffffffu, inc, 31);
    if (b0 >= a.B) {  // cannot happen for t < total
      b = a.B - 1;
      rem = 0;
      return;
    }
  }
}

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
  int pe, log2pe, recS;      // positions and bytes of a record in shared memory
  uint32_t issued = 0, used = 0;
  bool ok = true;

  // What lane `lane` copies of block kb of the piece, and the page it comes from.
  __device__ __forceinline__ int copies() const { return a.c.page <= KB ? KB / a.c.page : 4; }
  __device__ __forceinline__ bool wanted(const Walk& w, int kb) const {
    if (lane >= copies()) return false;
    const int p0 = kb * KB + (a.c.page <= KB ? lane * a.c.page : 0);
    return p0 < w.vis1 && p0 + pe > w.vis0;
  }
  __device__ __forceinline__ int page_id(const Walk& w, int kb) const {
    if (!wanted(w, kb)) return 0;
    const int p0 = kb * KB + (a.c.page <= KB ? lane * a.c.page : 0);
    return a.c.table[int64_t(w.b) * a.c.max_pages + (p0 >> a.c.log2page)];
  }
  __device__ __forceinline__ void issue(const Walk& w, int kb, int pid) {
    const uint32_t s = issued & 1u;
    const uint32_t dst = smem_u32(ring) + s * C::STAGE, b = bar + 8u * s;
    bool want = wanted(w, kb);
    if (want && (pid < 0 || pid >= a.c.n_pages)) {
      atomicCAS(&slot->err, 0u, uint32_t(SA_ERR_BAD_PAGE));
      want = false;
    }
    uint32_t bytes = 0, off = 0;
    int64_t src = 0;
    if (want) {
      src = a.c.record(pid, w.h);
      if (a.c.page <= KB) {
        bytes = 2u * a.c.rec;
        off = lane * bytes;
      } else {
        const int sub = (kb * KB) & (a.c.page - 1), kv = lane >> 1;
        src += int64_t(kv) * a.c.rec;
        off = kv * recS;
        if (lane & 1) {
          src += int64_t(a.c.page) * (a.c.d / 2) + sub * (a.c.d / 16);
          off += KB * (a.c.d / 2);
          bytes = KB * (a.c.d / 16);
        } else {
          src += int64_t(sub) * (a.c.d / 2);
          bytes = KB * (a.c.d / 2);
        }
      }
    }
    const uint32_t total = __reduce_add_sync(0xffffffffu, bytes);
    if (lane == 0) mbar_arrive_expect_tx(b, total);
    __syncwarp();
    if (want) bulk_load(dst + off, a.c.pool + src, bytes, b);
    ++issued;
  }

  // Address of key k's code row (kv = 0) or value row (kv = 1) within the stage.
  __device__ __forceinline__ const uint8_t* row(const uint8_t* st, int k, int kv) const {
    return st + ((k >> log2pe) * 2 + kv) * recS + (k & (pe - 1)) * (FULL ? C::D / 2 : a.c.d / 2);
  }
  __device__ __forceinline__ const uint8_t* scales(const uint8_t* st, int k, int kv) const {
    const int d = FULL ? C::D : a.c.d;
    return st + ((k >> log2pe) * 2 + kv) * recS + pe * (d / 2) + (k & (pe - 1)) * (d / 16);
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
  // acc[j] += rows x key tile j, j < NJ, keys 8 (j0 + j) + key_of(c); `fr` the rows' fragments
  template <int NJ>
  __device__ __forceinline__ void contract(const uint8_t* st, int j0, int kv, const uint8_t* fr, float (*acc)[4]) const {
    uint32_t w[NJ][C::LW], codes[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      load_words(st, 8 * (j0 + j) + key_of(g), kv, w[j], codes[j]);
      acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < C::LW; ++i) {
      uint32_t A[C::NS][2][4];
#pragma unroll
      for (int s = 0; s < C::NS; ++s)
#pragma unroll
        for (int k = 0; k < 2; ++k)
          *reinterpret_cast<uint4*>(A[s][k]) =
              *reinterpret_cast<const uint4*>(fr + s * C::FRAG + ((2 * i + k) * 32 + lane) * 16);
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        uint32_t v[4];
        values_bf16(w[j][i], scale_bf16(((codes[j] >> (8 * (i / 2))) & 255u) * 0x00010001u), v);
#pragma unroll
        for (int s = C::NS - 1; s >= 0; --s) {  // the smallest terms first
          mma_bf16(acc[j], A[s][0], v[0], v[1]);
          mma_bf16(acc[j], A[s][1], v[2], v[3]);
        }
      }
    }
  }
  // acc += weights x rows of 16 keys 16 jj ..: WT terms of A operands; F16 or bf16 values.
  // Keys outside [first, last) of the block count as zero: what nobody wrote can read as
  // an infinity in float16, and 0 x inf is not 0.
  template <bool F16, int WT>
  __device__ __forceinline__ void combine(const uint8_t* st, int jj, int kv, const uint32_t (*A)[4], float (*acc)[4],
                                          bool inside, int first, int last) const {
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
      if (!inside && (k[i] < first || k[i] >= last)) code[i] = 0;
    }
    const uint32_t c01 = code[0] | code[1] << 16, c23 = code[2] | code[3] << 16;
    const ScaleB sb01 = scale_bf16(c01), sb23 = scale_bf16(c23);
#pragma unroll
    for (int n = 0; n < NW; ++n) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {  // even, then odd features
        const uint32_t sel = half ? 0x7632u : 0x5410u;
        const uint32_t x = __byte_perm(w[0][n], w[1][n], sel), y = __byte_perm(w[2][n], w[3][n], sel);
        uint32_t b0[4], b1[4];
        if constexpr (F16) {
          values_f16(x, c01 << 7, b0);
          values_f16(y, c23 << 7, b1);
        } else {
          values_bf16(x, sb01, b0);
          values_bf16(y, sb23, b1);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int s = WT - 1; s >= 0; --s) {
            if constexpr (F16)
              mma_f16(acc[8 * n + 2 * e + half], A[s], b0[e], b1[e]);
            else
              mma_bf16(acc[8 * n + 2 * e + half], A[s], b0[e], b1[e]);
          }
      }
    }
  }

  // Rows g and g + 8 of src (element offsets r0, r1; negative: no row) as fragments.
  template <typename T>
  __device__ __forceinline__ void load_frags(const T* src, int64_t r0, int64_t r1, uint8_t* fr) const {
    const int base = (C::D / 4) * t4, d = FULL ? C::D : a.c.d;
#pragma unroll
    for (int i = 0; i < C::LW; ++i) {
      const int c = base + 8 * i;
      uint32_t A[C::NS][2][4];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int64_t r = half ? r1 : r0;
        uint32_t p[C::NS][4] = {};
        if (r >= 0 && c < d) {
          if constexpr (C::F32) {
            float x[8];
            *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(src + r + c);
            *reinterpret_cast<float4*>(x + 4) = *reinterpret_cast<const float4*>(src + r + c + 4);
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
            *reinterpret_cast<uint4*>(p[0]) = *reinterpret_cast<const uint4*>(src + r + c);
          }
        }
#pragma unroll
        for (int s = 0; s < C::NS; ++s)
#pragma unroll
          for (int k = 0; k < 4; ++k) A[s][k >> 1][half + 2 * (k & 1)] = p[s][k];
      }
#pragma unroll
      for (int s = 0; s < C::NS; ++s)
#pragma unroll
        for (int k = 0; k < 2; ++k)
          *reinterpret_cast<uint4*>(fr + s * C::FRAG + ((2 * i + k) * 32 + lane) * 16) =
              *reinterpret_cast<const uint4*>(A[s][k]);
    }
  }
};

// 8 consecutive results of one row
__device__ __forceinline__ void store8(float* p, const float* x) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float* x) {
  uint4 v;
  v.x = pack_bf16(x[0], x[1]), v.y = pack_bf16(x[2], x[3]), v.z = pack_bf16(x[4], x[5]), v.w = pack_bf16(x[6], x[7]);
  *reinterpret_cast<uint4*>(p) = v;
}

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
  const int64_t total = scan_users<C::THREADS>(a, pre, chunk);
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
  x.pe = min(a.c.page, KB);
  x.log2pe = min(a.c.log2page, 6);
  x.recS = x.pe * (a.c.d / 2 + a.c.d / 16);
  const int g = x.g, t4 = x.t4, d = FULL ? C::D : a.c.d;
  const float c2 = a.scale * kLog2e;

  Walk cur, ahead;  // `ahead` runs up to two blocks in front and issues the copies
  cur.t = tb;
  cur.te = te;
  {
    int64_t rem;
    find_tile<C::THREADS>(a, pre, chunk, tb, lane, cur.b, rem);
    set_piece(a, cur, user_sizes(a, cur.b), rem, lane);
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
      more = next_piece(a, ahead, lane);
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

  for (bool have = true; have && x.ok;) {
    // rows of this piece
    const int r0 = cur.rt * ROWS + g, r1 = r0 + 8;
    const int64_t q_t0 = cur.q0 + r0 / a.G, q_t1 = cur.q0 + r1 / a.G;
    const int hd0 = cur.h * a.G + r0 % a.G, hd1 = cur.h * a.G + r1 % a.G;
    const bool v0 = r0 < cur.rows, v1 = r1 < cur.rows;
    int lo0 = 0, hi0 = 0x7fffffff, lo1 = 0, hi1 = 0x7fffffff;
    if (v0) row_window(a, q_t0, cur.len, lo0, hi0);
    if (v1) row_window(a, q_t1, cur.len, lo1, hi1);
    const int lo_most = __reduce_max_sync(0xffffffffu, max(lo0, lo1));
    const int hi_least = __reduce_min_sync(0xffffffffu, min(hi0, hi1));
    __syncwarp();
    if (cur.kb0 < cur.kb1) {
      const T* q = static_cast<const T*>(a.q);
      x.load_frags(q, v0 ? q_t0 * a.q_row + hd0 * a.q_head : -1, v1 ? q_t1 * a.q_row + hd1 * a.q_head : -1, x.frag);
    }
    const int64_t o0 = (q_t0 * a.Hq + hd0) * d, o1 = (q_t1 * a.Hq + hd1) * d;  // rows of the dense tensors
    float D0 = 0.f, D1 = 0.f, L0 = 0.f, L1 = 0.f;
    if constexpr (C::BWD) {
      const T* dout = static_cast<const T*>(a.dout);
      const T* out = static_cast<const T*>(a.out);
      if (cur.kb0 < cur.kb1) x.load_frags(dout, v0 ? o0 : -1, v1 ? o1 : -1, x.frag + C::NS * C::FRAG);
      for (int c = (C::D / 4) * t4; c < (C::D / 4) * (t4 + 1) && c < d; ++c) {
        if (v0) D0 = fmaf(ld_f32(dout + o0 + c), ld_f32(out + o0 + c), D0);
        if (v1) D1 = fmaf(ld_f32(dout + o1 + c), ld_f32(out + o1 + c), D1);
      }
      D0 += __shfl_xor_sync(0xffffffffu, D0, 1);
      D0 += __shfl_xor_sync(0xffffffffu, D0, 2);
      D1 += __shfl_xor_sync(0xffffffffu, D1, 1);
      D1 += __shfl_xor_sync(0xffffffffu, D1, 2);
      if (v0) L0 = a.lse[q_t0 * a.Hq + hd0] * kLog2e;
      if (v1) L1 = a.lse[q_t1 * a.Hq + hd1] * kLog2e;
    }
    __syncwarp();

    float acc[C::NT][4];
#pragma unroll
    for (int i = 0; i < C::NT; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;

    for (int kb = cur.kb0; kb < cur.kb1; ++kb) {
      const uint32_t s = x.used & 1u;
      x.ok = __all_sync(0xffffffffu, mbar_wait(bar + 8 * s, (x.used >> 1) & 1u, ctl, slot, 0xC01u));
      if (!x.ok) break;
      const uint8_t* st = x.ring + s * C::STAGE;
      const int k0 = kb * KB;
      const bool inside = k0 >= lo_most && k0 + KB <= hi_least;
      if constexpr (!C::BWD) {
        float S[KB / 8][4];
        x.template contract<KB / 8>(st, 0, 0, x.frag, S);
        float b0 = -INFINITY, b1 = -INFINITY;
#pragma unroll
        for (int j = 0; j < KB / 8; ++j) {
#pragma unroll
          for (int e = 0; e < 4; ++e) S[j][e] *= c2;
          if (!inside) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int k = k0 + 8 * j + key_of(2 * t4 + e);
              if (k < lo0 || k >= hi0) S[j][e] = -INFINITY;
              if (k < lo1 || k >= hi1) S[j][2 + e] = -INFINITY;
            }
          }
          b0 = fmax3(b0, S[j][0], S[j][1]);
          b1 = fmax3(b1, S[j][2], S[j][3]);
        }
        b0 = fmaxf(b0, __shfl_xor_sync(0xffffffffu, b0, 1));
        b0 = fmaxf(b0, __shfl_xor_sync(0xffffffffu, b0, 2));
        b1 = fmaxf(b1, __shfl_xor_sync(0xffffffffu, b1, 1));
        b1 = fmaxf(b1, __shfl_xor_sync(0xffffffffu, b1, 2));
        const float n0 = fmaxf(m0, b0), n1 = fmaxf(m1, b1);
        // nothing seen yet: shift by zero, so that 2^(-inf) = 0 and no inf - inf appears
        const float z0 = n0 == -INFINITY ? 0.f : n0, z1 = n1 == -INFINITY ? 0.f : n1;
        if (__any_sync(0xffffffffu, n0 != m0 || n1 != m1)) {
          const float f0 = ex2(m0 - z0), f1 = ex2(m1 - z1);
          l0 *= f0;
          l1 *= f1;
#pragma unroll
          for (int i = 0; i < C::NT; ++i) {
            acc[i][0] *= f0, acc[i][1] *= f0;
            acc[i][2] *= f1, acc[i][3] *= f1;
          }
          m0 = n0;
          m1 = n1;
        }
        const float sh0 = z0 - kLift, sh1 = z1 - kLift;
#pragma unroll
        for (int jj = 0; jj < KB / 16; ++jj) {
          uint32_t A[C::NP][4];
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            float* p = S[2 * jj + u];
            p[0] = ex2(p[0] - sh0), p[1] = ex2(p[1] - sh0);
            p[2] = ex2(p[2] - sh1), p[3] = ex2(p[3] - sh1);
            l0 += p[0] + p[1];
            l1 += p[2] + p[3];
            A[0][2 * u] = pack_f16(p[0], p[1]);
            A[0][2 * u + 1] = pack_f16(p[2], p[3]);
            if constexpr (C::NP == 2) {
              const float2 f = unpack_f16(A[0][2 * u]), e = unpack_f16(A[0][2 * u + 1]);
              A[1][2 * u] = pack_f16(p[0] - f.x, p[1] - f.y);
              A[1][2 * u + 1] = pack_f16(p[2] - e.x, p[3] - e.y);
            }
          }
          x.template combine<true, C::NP>(st, jj, 1, A, acc, inside, cur.vis0 - k0, cur.vis1 - k0);
        }
      } else {
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
          float S[4][4], P[4][4];
          x.template contract<4>(st, 4 * half, 0, x.frag, S);
          x.template contract<4>(st, 4 * half, 1, x.frag + C::NS * C::FRAG, P);
#pragma unroll
          for (int jj = 0; jj < 2; ++jj) {
            uint32_t A[C::NS][4];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const int j = 2 * jj + u;
              float p[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int k = k0 + 32 * half + 8 * j + key_of(2 * t4 + (e & 1));
                const bool see = inside || (e < 2 ? k >= lo0 && k < hi0 : k >= lo1 && k < hi1);
                const float w = ex2(fmaf(S[j][e], c2, e < 2 ? -L0 : -L1));
                p[e] = see ? w * (P[j][e] - (e < 2 ? D0 : D1)) : 0.f;
              }
#pragma unroll
              for (int s2 = 0; s2 < C::NS; ++s2) {
                A[s2][2 * u] = pack_bf16(p[0], p[1]);
                A[s2][2 * u + 1] = pack_bf16(p[2], p[3]);
                if (s2 + 1 < C::NS) {
                  const float2 f = unpack_bf16(A[s2][2 * u]), e = unpack_bf16(A[s2][2 * u + 1]);
                  p[0] -= f.x, p[1] -= f.y, p[2] -= e.x, p[3] -= e.y;
                }
              }
            }
            x.template combine<false, C::NS>(st, 2 * half + jj, 0, A, acc, true, 0, KB);
          }
        }
      }
      ++x.used;
      __syncwarp();  // every lane is done with the stage
      produce();
    }
    if (!x.ok) break;

    // the piece's end
    const bool whole = cur.seg0 >= tb && cur.seg1 <= te;
    if constexpr (!C::BWD) {
      l0 += __shfl_xor_sync(0xffffffffu, l0, 1);
      l0 += __shfl_xor_sync(0xffffffffu, l0, 2);
      l1 += __shfl_xor_sync(0xffffffffu, l1, 1);
      l1 += __shfl_xor_sync(0xffffffffu, l1, 2);
    }
    float* part = a.partial + (int64_t(wk) * 2 + (tb >= cur.seg0 ? 0 : 1)) * partial_floats(C::D);
    const float f0 = C::BWD ? a.scale : (l0 > 0.f ? 1.f / l0 : 0.f), f1 = C::BWD ? a.scale : (l1 > 0.f ? 1.f / l1 : 0.f);
    T* dst = static_cast<T*>(C::BWD ? a.dq : a.out);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (!(half ? v1 : v0)) continue;
#pragma unroll
      for (int i = 0; i < C::LW; ++i) {
        // columns 2 t4 (the first half of the lane's features) and 2 t4 + 1 (the second)
        float y[8];
        constexpr int PER = C::NT / 8;  // words per column
        const int col = i / PER, n = i % PER;
        const float f = whole ? (half ? f1 : f0) : 1.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = acc[8 * n + e][2 * half + col] * f;
        const int c = (C::D / 4) * t4 + 8 * i;
        if (c >= d) continue;
        if (whole)
          store8(dst + (half ? o1 : o0) + c, y);
        else
          store8(part + (g + 8 * half) * C::D + c, y);
      }
      if constexpr (!C::BWD) {
        const float m = half ? m1 : m0, l = half ? l1 : l0;
        if (t4 == 0) {
          if (!whole)
            *reinterpret_cast<float2*>(part + ROWS * C::D + 2 * (g + 8 * half)) = make_float2(m, l);
          else if (a.lse)
            a.lse[half ? q_t1 * a.Hq + hd1 : q_t0 * a.Hq + hd0] = l > 0.f ? (m + log2f(l) - kLift) * kLn2 : -INFINITY;
        }
      }
    }
    have = next_piece(a, cur, lane);
  }
  if (!x.ok) {  // no copy may still be in flight when the CTA's shared memory goes
    for (; x.used != x.issued; ++x.used) {
      const uint64_t t0 = globaltimer();
      while (!mbar_try_wait(bar + 8 * (x.used & 1u), (x.used >> 1) & 1u) && globaltimer() - t0 < 200000000ull) {
      }
    }
  }
}

// Adds the pieces of segments that share borders cut, in worker order, and gathers
// the CTAs' status.  Block w handles the segment whose first cut is where worker w
// starts.  Eight warps take rp rows at a time and split each row's pieces 8 / rp
// ways: with one row (a single token over a long history) a segment has many pieces,
// with sixteen it has few.
constexpr int kJoinWarps = 8;

template <class C>
__global__ void __launch_bounds__(32 * kJoinWarps) cache_join_kernel(const __grid_constant__ AttnArgs a) {
  using T = typename std::conditional<C::F32, float, __nv_bfloat16>::type;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, w = blockIdx.x;
  if (w == 0) {
    __shared__ int all;
    if (threadIdx.x == 0) all = 0;
    __syncthreads();
    int e = 0;
    for (int i = threadIdx.x; i < a.ctas; i += blockDim.x) e = max(e, int(a.slots[i].err));
    if (e) atomicMax(&all, e);
    __syncthreads();
    if (threadIdx.x == 0) ws_header(a.ws)->err = uint32_t(all);
    return;
  }
  const int64_t total = ws_header(a.ws)->tiles_per_head;
  if (total <= 0) return;
  const int W = shares(a, total);
  if (w >= W) return;
  const int64_t tb = range_begin(total, W, w);
  const Piece p = static_cast<const Piece*>(a.piece)[w];
  if (p.seg0 >= tb) return;
  if (range_begin(total, W, w - 1) > p.seg0) return;  // an earlier border already cut this segment
  const int first = w - 1, n = owner_of(total, W, p.seg1 - 1) - first + 1;
  constexpr int PF = partial_floats(C::D);
  // the first worker's piece is its second one unless its share begins with the segment
  const float* base = a.partial + int64_t(first) * 2 * PF;
  const int first_off = range_begin(total, W, first) >= p.seg0 ? 0 : PF;
  const int64_t q0 = a.cu_q[p.b];
  const int rows = min(ROWS, int((a.cu_q[p.b + 1] - q0) * a.G - p.rt * ROWS));
  const int rp = rows <= 1 ? 1 : rows <= 2 ? 2 : rows <= 4 ? 4 : 8, ns = kJoinWarps / rp;
  const int split = warp / rp, d = a.c.d;
  constexpr int V = C::D / 32;
  __shared__ float part[kJoinWarps][C::D];
  __shared__ float2 stat[kJoinWarps];
  for (int r0 = 0; r0 < rows; r0 += rp) {
    const int r = r0 + warp % rp;
    float m = -INFINITY, l = 0.f, y[V] = {};
    if (r < rows) {
      for (int k0 = split * 32; k0 < n; k0 += ns * 32) {  // 32 pieces at a time, one lane each for the weights
        const int k = k0 + lane;
        float f = 1.f;
        if constexpr (!C::BWD) {
          float2 ml = make_float2(-INFINITY, 0.f);
          if (k < n)
            ml = *reinterpret_cast<const float2*>(base + int64_t(k) * 2 * PF + (k == 0 ? first_off : 0) + ROWS * C::D + 2 * r);
          float bm = ml.x;
#pragma unroll
          for (int o = 16; o; o >>= 1) bm = fmaxf(bm, __shfl_xor_sync(0xffffffffu, bm, o));
          const float nm = fmaxf(m, bm), z = nm == -INFINITY ? 0.f : nm, back = ex2(m - z);
          f = ex2(ml.x - z);
          float bl = ml.y * f;
#pragma unroll
          for (int o = 16; o; o >>= 1) bl += __shfl_xor_sync(0xffffffffu, bl, o);
          l = fmaf(l, back, bl);
#pragma unroll
          for (int i = 0; i < V; ++i) y[i] *= back;
          m = nm;
        }
        const int cnt = min(32, n - k0);
#pragma unroll 4
        for (int j = 0; j < cnt; ++j) {
          const float* s = base + int64_t(k0 + j) * 2 * PF + (k0 + j == 0 ? first_off : 0) + r * C::D + lane;
          const float fj = __shfl_sync(0xffffffffu, f, j);
#pragma unroll
          for (int i = 0; i < V; ++i) y[i] = fmaf(s[32 * i], fj, y[i]);
        }
      }
    }
    if (ns > 1) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < V; ++i) part[warp][32 * i + lane] = y[i];
      if (lane == 0) stat[warp] = make_float2(m, l);
      __syncthreads();
      if (split == 0)
        for (int s = 1; s < ns; ++s) {
          const int o = warp + s * rp;
          float f = 1.f, back = 1.f;
          if constexpr (!C::BWD) {
            const float2 ml = stat[o];
            const float nm = fmaxf(m, ml.x), z = nm == -INFINITY ? 0.f : nm;
            back = ex2(m - z);
            f = ex2(ml.x - z);
            l = fmaf(l, back, ml.y * f);
            m = nm;
          }
#pragma unroll
          for (int i = 0; i < V; ++i) y[i] = fmaf(part[o][32 * i + lane], f, y[i] * back);
        }
    }
    if (split == 0 && r < rows) {
      const int row = p.rt * ROWS + r;
      const int64_t o = (q0 + row / a.G) * a.Hq + p.h * a.G + row % a.G;
      const float f = C::BWD ? a.scale : (l > 0.f ? 1.f / l : 0.f);
      T* dst = static_cast<T*>(C::BWD ? a.dq : a.out) + o * d;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (32 * i + lane < d) st_from_f32(dst + 32 * i + lane, y[i] * f);
      if (!C::BWD && a.lse && lane == 0) a.lse[o] = l > 0.f ? (m + log2f(l) - kLift) * kLn2 : -INFINITY;
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
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(a.workers));
  cfg.blockDim = dim3(32 * kJoinWarps);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, cache_join_kernel<C>, a);
}

template <int D>
static cudaError_t run_d(const AttnArgs& a, bool bwd, cudaStream_t st) {
  if (a.dt == SA_F32) return bwd ? run<Cfg<D, true, true>>(a, st) : run<Cfg<D, true, false>>(a, st);
  return bwd ? run<Cfg<D, false, true>>(a, st) : run<Cfg<D, false, false>>(a, st);
}

template <int D>
static int warps(bool f32, bool bwd) {
  if (f32) return bwd ? Cfg<D, true, true>::NWARP : Cfg<D, true, false>::NWARP;
  return bwd ? Cfg<D, false, true>::NWARP : Cfg<D, false, false>::NWARP;
}

static bool wide(int d) { return d > 64; }

int mma_workers(int sms, int d, sa_dtype dt, bool bwd, int* ctas) {
  *ctas = sms;
  return sms * (wide(d) ? warps<128>(dt == SA_F32, bwd) : warps<64>(dt == SA_F32, bwd));
}
size_t mma_piece_bytes() { return sizeof(Piece); }
size_t mma_partial_floats(int d) { return size_t(partial_floats(wide(d) ? 128 : 64)); }

cudaError_t launch_mma(const AttnArgs& a, bool bwd, cudaStream_t st) {
  return wide(a.c.d) ? run_d<128>(a, bwd, st) : run_d<64>(a, bwd, st);
}

}  // namespace cache
}  // namespace sa
