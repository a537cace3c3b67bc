// Shares of an attention call's work, and the sum of what shares leave unfinished.
// Used by the cache's kernels, which differ in the rows and positions of a tile.
//
// The unit of work is one block of C::KB positions for C::HALF query rows of one user
// and cached head; the list is ordered (user, head, row tile, block), and worker w of W
// owns the contiguous range [range_begin(w), range_begin(w + 1)) of it.  A segment, all
// blocks of one row tile, that lies within one range is finished by its worker; of a
// segment that borders cut every worker leaves a piece (unnormalised sums and, forward,
// each row's shift and sum), and cache_join_kernel adds the pieces in worker order: the
// result is bitwise reproducible for a given W.
#pragma once
#include <type_traits>

#include "sa_cache.cuh"
#include "sa_ptx.cuh"

namespace sa {
namespace cache {

using namespace ptx;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// Weights are kept as 2^12 exp(S - max): float16 then holds weights down to 2^-26 of
// the largest in full precision.
constexpr float kLift = 12.f;

// Partial of one piece: its rows' D sums, then their (max, sum) pairs.
__host__ __device__ constexpr int partial_floats(int rows, int D) { return rows * D + rows * 2; }

// Shares of a call with `total` tiles: none is empty.
__device__ __forceinline__ int shares(const AttnArgs& a, int64_t total) { return int(total < a.workers ? total : a.workers); }

struct Piece {  // what a worker's first segment is, for the join
  int64_t seg0, seg1;
  int b, h, rt, pad;
};

// ------------------------------------------------------------------ the walk
struct Sizes {
  int64_t units;  // of the user, all heads
  int nrt, nkb, rows, len;
  int64_t q0;
  // Units of one block of row tile rt: 2 where it has more than HALF rows, if the
  // kernel's row tile has two halves, else 1.
  template <class C>
  __device__ __forceinline__ int weight(int rt) const {
    return C::HALF < C::ROWS && rows - rt * C::ROWS > C::HALF ? 2 : 1;
  }
  template <class C>
  __device__ __forceinline__ int64_t per_head() const {
    return nrt ? int64_t(nkb) * ((nrt - 1) * (C::HALF < C::ROWS ? 2 : 1) + weight<C>(nrt - 1)) : 0;
  }
};
// One worker's share of one segment.  Uniform over the warp.
struct Walk {
  int64_t t, te;          // next unit of work, end of the share
  int64_t seg0, seg1;     // units of the segment
  int b, h, rt;
  int weight;             // units of one block
  Sizes s;                // of the user
  int vis0, vis1;         // positions that some row of the tile sees
  int kb0, kb1;           // blocks of this piece (empty: kb0 >= kb1)
};

template <class C>
__device__ __forceinline__ Sizes user_sizes(const AttnArgs& a, int b) {
  Sizes s;
  const int c0 = a.cu_q[b], c1 = a.cu_q[b + 1];
  s.q0 = c0;
  s.len = a.lens[b];
  s.rows = (c1 - c0) * a.G;
  s.nrt = (s.rows + C::ROWS - 1) / C::ROWS;
  s.nkb = s.len > 0 ? (s.len + C::KB - 1) / C::KB : 1;  // a user with nothing cached still gets its zeros
  s.units = s.per_head<C>() * a.c.H;
  return s;
}

// Query t's positions; neither end is negative, so that differences with positions stay in range.
__device__ __forceinline__ void row_window(const AttnArgs& a, int64_t t, int len, int& lo, int& hi) {
  lo = a.begin ? max(a.begin[t], 0) : 0;
  hi = a.end ? max(min(a.end[t], len), 0) : len;
}

// The piece that starts at unit w.t of user w.b (sizes in s).
template <class C>
__device__ __forceinline__ void set_piece(const AttnArgs& a, Walk& w, const Sizes& s, int64_t rem, int lane) {
  w.s = s;
  const int64_t per_head = s.per_head<C>();
  w.h = int(rem / per_head);
  const int64_t r2 = rem - w.h * per_head;
  constexpr int most = C::HALF < C::ROWS ? 2 : 1;
  w.rt = min(int(r2 / (int64_t(s.nkb) * most)), s.nrt - 1);
  const int64_t in = r2 - int64_t(w.rt) * s.nkb * most;
  const int wt = s.weight<C>(w.rt);
  w.weight = wt;
  w.seg0 = w.t - in;
  w.seg1 = w.seg0 + int64_t(s.nkb) * wt;
  // a border inside a block gives the block to the share that has its first unit
  const int kb = int((in + wt - 1) / wt);
  w.vis0 = 0;
  w.vis1 = s.len;
  if (a.begin || a.end) {
    int lo = 0x7fffffff, hi = 0;
    for (int i = lane; i < C::ROWS; i += 32) {
      const int r = w.rt * C::ROWS + i;
      if (r >= s.rows) break;
      int l, e;
      row_window(a, s.q0 + r / a.G, s.len, l, e);
      if (l < e) {
        lo = min(lo, l);
        hi = max(hi, e);
      }
    }
    w.vis0 = __reduce_min_sync(0xffffffffu, lo);
    w.vis1 = __reduce_max_sync(0xffffffffu, hi);
  }
  const int64_t last = w.te < w.seg1 ? w.te : w.seg1;
  w.kb0 = max(kb, w.vis0 / C::KB);
  w.kb1 = min(int((last - w.seg0 + wt - 1) / wt), (w.vis1 + C::KB - 1) / C::KB);
  if (w.vis0 >= w.vis1) w.kb1 = w.kb0;
}

// Whether one of rows r, r + step, ... below `end` of a user sees one of positions [p0, p1), p0
// within the user's length.  Asked only where a page is missing: between the windows of a
// tile's rows a page may be nobody's, and is then no error.  Out of line, for the loops that
// ask are bound by the code they run through (inlined, 300 queries over 10,000 positions
// take 276 us instead of 273).
static __device__ __noinline__ bool rows_see(const AttnArgs& a, int64_t q0, int len, int r, int end, int step, int p0,
                                             int p1) {
  if (!a.begin && !a.end) return true;
  for (; r < end; r += step) {
    int l, e;
    row_window(a, q0 + r / a.G, len, l, e);
    if (max(l, p0) < min(e, p1)) return true;
  }
  return false;
}
// The same of rows first, first + step, ... of the walk's tile.
template <class C>
__device__ __forceinline__ bool tile_sees(const AttnArgs& a, const Walk& w, int p0, int p1, int first, int step) {
  return rows_see(a, w.s.q0, w.s.len, w.rt * C::ROWS + first, min(w.s.rows, (w.rt + 1) * C::ROWS), step, p0, p1);
}

// Move to the next piece of the share; false at its end.
template <class C>
__device__ __forceinline__ bool next_piece(const AttnArgs& a, Walk& w, int lane) {
  w.t = w.te < w.seg1 ? w.te : w.seg1;
  if (w.t >= w.te) return false;
  Sizes s;
  int64_t rem;
  if (w.rt + 1 < w.s.nrt || w.h + 1 < a.c.H) {
    s = w.s;
    constexpr int most = C::HALF < C::ROWS ? 2 : 1;
    rem = w.h * s.per_head<C>() + int64_t(w.rt) * s.nkb * most + int64_t(s.nkb) * w.weight;
  } else {
    int b = w.b + 1;
    for (;;) {  // the next user with queries (one exists: units are left)
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
    s = user_sizes<C>(a, b);
    rem = 0;
  }
  set_piece<C>(a, w, s, rem, lane);
  return true;
}

// Exclusive scan of the users' units over the CTA's threads (each takes `chunk`
// consecutive users) into pre[0..C::THREADS]; returns the total, or -1 where offsets or
// lengths are out of order.
template <class C>
__device__ int64_t scan_users(const AttnArgs& a, int64_t* pre, int chunk) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int b0 = tid * chunk, b1 = min(a.B, b0 + chunk);
  int64_t sum = 0;
  int bad = 0;
  const int64_t most = int64_t(a.c.max_pages) << a.c.log2page;
  for (int b = b0; b < b1; ++b) {
    const int c0 = a.cu_q[b], c1 = a.cu_q[b + 1], len = a.lens[b];
    if (c0 > c1 || (b == 0 && c0 != 0) || (b == a.B - 1 && int64_t(c1) != a.T) || len < 0 || len > most) bad = 1;
    sum += user_sizes<C>(a, b).units;
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
  for (int i = 0; i < C::NWARP; ++i) {
    if (i < warp) before += warp_sum[i];
    total += warp_sum[i];
  }
  pre[tid] = before + inc - sum;
  if (tid == 0) pre[C::THREADS] = total;
  __syncthreads();
  return bad ? -1 : total;
}

// The user of unit t and the unit's rank among the user's.
template <class C>
__device__ void find_tile(const AttnArgs& a, const int64_t* pre, int chunk, int64_t t, int lane, int& b, int64_t& rem) {
  int lo = 0, hi = C::THREADS - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (pre[mid] <= t) lo = mid; else hi = mid - 1;
  }
  int64_t at = pre[lo];
  for (int b0 = lo * chunk;; b0 += 32) {
    const int u = b0 + lane;
    const int64_t mine = u < a.B && u < (lo + 1) * chunk ? user_sizes<C>(a, u).units : 0;
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

// Adds the pieces of segments that share borders cut, in worker order, and gathers
// the CTAs' status.  Block w handles the segment whose first cut is where worker w
// starts, and the blocks beside it (y) its other rows.  Eight warps take rp rows at a
// time and split each row's pieces 8 / rp ways: with one row (a single token over a long
// history) a segment has many pieces, with sixteen it has few.  Its launch overlaps the main
// kernel's tail; what it adds is latency: one query of 16 users over up to 100,000 positions
// takes 204 us, the main kernel alone 199 (GB300).
constexpr int kJoinWarps = 8;

template <class C>
__global__ void __launch_bounds__(32 * kJoinWarps) cache_join_kernel(const __grid_constant__ AttnArgs a) {
  using T = typename std::conditional<C::F32, float, __nv_bfloat16>::type;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, w = blockIdx.x;
  if (w == 0) {
    if (blockIdx.y) return;
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
  // one unit a share in a small call: no divisions (each costs about as much as a load)
  auto begin = [&](int x) { return W == total ? int64_t(x) : range_begin(total, W, x); };
  const Piece p = static_cast<const Piece*>(a.piece)[w];
  if (p.seg0 >= begin(w)) return;
  if (begin(w - 1) > p.seg0) return;  // an earlier border already cut this segment
  const int first = w - 1;
  const int n = (W == total ? int(p.seg1 - 1) : owner_of(total, W, p.seg1 - 1)) - first + 1;
  constexpr int ROWS = C::ROWS, PF = partial_floats(ROWS, C::D);
  // the first worker's piece is its second one unless its share begins with the segment
  const float* base = a.partial + int64_t(first) * 2 * PF;
  const int first_off = begin(first) >= p.seg0 ? 0 : PF;
  const int64_t q0 = a.cu_q[p.b];
  const int rows = min(ROWS, int((a.cu_q[p.b + 1] - q0) * a.G - p.rt * ROWS));
  const int rp = rows <= 1 ? 1 : rows <= 2 ? 2 : rows <= 4 ? 4 : 8, ns = kJoinWarps / rp;
  const int split = warp / rp, d = a.c.d;
  // Pieces whose loads are in flight: they come from L2, and their latency is the time.  A
  // tall tile's segments are cut into few (300 queries over 10,000 positions: the call takes
  // 274 us with two, 277 with four, 281 with eight; up to 7 windowed queries over 3001: 20 us
  // with eight, 27 with four).
  constexpr int V = C::D / 32, AT = ROWS > 16 ? 2 : 8;
  __shared__ float part[kJoinWarps][C::D];
  __shared__ float2 stat[kJoinWarps];
  for (int r0 = blockIdx.y * rp; r0 < rows; r0 += gridDim.y * rp) {
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
        for (int j0 = 0; j0 < cnt; j0 += AT) {
          float s[AT][V];
#pragma unroll
          for (int j = 0; j < AT; ++j) {
            const int k = k0 + j0 + j;
            const float* src = base + int64_t(k) * 2 * PF + (k == 0 ? first_off : 0) + r * C::D + lane;
#pragma unroll
            for (int i = 0; i < V; ++i) s[j][i] = k < n ? src[32 * i] : 0.f;
          }
#pragma unroll
          for (int j = 0; j < AT; ++j) {
            const float fj = __shfl_sync(0xffffffffu, f, j0 + j);
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = fmaf(s[j][i], fj, y[i]);
          }
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
      const float f = C::BWD ? a.scale : (l == 0.f ? 0.f : 1.f / l);
      T* dst = static_cast<T*>(C::BWD ? a.dq : a.out) + o * d;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (32 * i + lane < d) st_from_f32(dst + 32 * i + lane, y[i] * f);
      if (!C::BWD && a.lse && lane == 0) a.lse[o] = l == 0.f ? -INFINITY : (m + log2f(l) - kLift) * kLn2;
    }
  }
}

template <class C>
static cudaError_t launch_join(const AttnArgs& a, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(a.workers), C::ROWS > 16 ? C::ROWS / 16 : 1);
  cfg.blockDim = dim3(32 * kJoinWarps);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, cache_join_kernel<C>, a);
}

}  // namespace cache
}  // namespace sa
