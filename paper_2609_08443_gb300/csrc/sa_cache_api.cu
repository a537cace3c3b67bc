// Host side of the 4-bit cache: argument checks, workspace layout, the choice of
// kernels and launches on the caller's stream.  Declarations and the meaning of
// every argument: include/sa_cache.h.
#include <cmath>

#include "sa_cache.cuh"
#include "sa_kernels.cuh"
#include "sa_tc_common.cuh"

namespace {

using sa::cache::AttnArgs;
using sa::cache::Pages;
using sa::cache::RowArgs;

#define SA_TRY(x)               \
  do {                          \
    const sa_status s_ = (x);   \
    if (s_ != SA_OK) return s_; \
  } while (0)

constexpr int64_t kMost = int64_t(1) << 31;
// A user's positions, and its rows for a cached head, are counted in int32 and rounded up to
// tiles of at most 256.
constexpr int64_t kMostTiled = kMost - 256;

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

bool page_ok(int page) { return page >= 16 && page <= 256 && (page & (page - 1)) == 0; }
bool width_ok(int d) { return d >= 16 && d <= sa::kMaxD && d % 16 == 0; }

sa_status set_pages(Pages* c, const void* pool, int64_t n_pages, int page, const int32_t* table, int max_pages, int H,
                    int d) {
  if (!pool || !table || !aligned(pool, 16)) return SA_ERR_INVALID_ARG;
  if (n_pages < 1 || max_pages < 1 || H < 1 || d < 1 || page < 1) return SA_ERR_INVALID_ARG;
  if (!page_ok(page) || !width_ok(d) || H > sa::kMaxH || n_pages >= kMost || int64_t(max_pages) * page > kMostTiled)
    return SA_ERR_UNSUPPORTED;
  c->pool = static_cast<const uint8_t*>(pool);
  c->n_pages = n_pages;
  c->table = table;
  c->max_pages = max_pages;
  c->page = page;
  c->log2page = 0;
  while ((1 << c->log2page) < page) ++c->log2page;
  c->H = H;
  c->d = d;
  c->rec = page * (d / 2 + d / 16);
  return SA_OK;
}

sa_status check_workspace(const void* ws, size_t bytes, size_t need) {
  if (!ws || !aligned(ws, 256)) return SA_ERR_INVALID_ARG;
  return bytes < need ? SA_ERR_WORKSPACE : SA_OK;
}

sa_status check_rows(const RowArgs& a) {
  if (a.B < 1 || a.N < 0) return SA_ERR_INVALID_ARG;
  if (a.N >= kMost || (a.dt != SA_F32 && a.dt != SA_BF16)) return SA_ERR_UNSUPPORTED;
  return SA_OK;
}

// 16-byte aligned rows for strides in elements of type dt
bool stride_ok(int64_t s, sa_dtype dt) { return s >= 0 && s % (dt == SA_BF16 ? 8 : 4) == 0; }

// Sections of an attention call's workspace.
struct Layout {
  size_t slots, piece, partial, total;
  int workers, ctas;
};

Layout attn_layout(int B, int64_t T, int G, int d, sa_dtype dt, bool bwd, bool tc) {
  Layout l{};
  const int sms = sa::tcc::device_sm_count();
  const sa::cache::AttnPlan p = tc ? sa::cache::tc_plan(sms, d, bwd) : sa::cache::mma_plan(sms, B, T, G, d, dt, bwd);
  l.ctas = p.ctas;
  l.workers = p.workers;
  size_t off = sizeof(sa::WsHeader);
  l.slots = off;
  off += size_t(l.ctas) * sizeof(sa::WsHeader);
  l.piece = off;
  off = sa::align256(off + size_t(l.workers) * p.piece_bytes);
  l.partial = off;
  off = sa::align256(off + size_t(l.workers) * 2 * p.partial_floats * sizeof(float));
  l.total = off;
  return l;
}

// The kernel of a call: tcgen05 where its sizes are worth it (tc_supported) and sa_select_path
// leaves it.  A workspace's size asks for the sizes alone: it serves either kernel.
bool takes_tc(int B, int64_t T, int G, int d, sa_dtype dt, float scale, bool bwd) {
  return sa::tc_path_enabled() && sa::cache::tc_supported(B, T, G, d, dt, scale, bwd);
}

bool attn_sizes_ok(int B, int64_t T, int Hq, int H, int d, sa_dtype dt) {
  return B >= 1 && T >= 0 && H >= 1 && H <= sa::kMaxH && Hq >= H && Hq % H == 0 && width_ok(d) &&
         (dt == SA_F32 || dt == SA_BF16) && T <= kMostTiled / (Hq / H) && Hq < 65536;
}

sa_status attn(AttnArgs& a, const void* q, int64_t q_row, int64_t q_head, const int32_t* cu_q, int B, int64_t T, int Hq,
               const void* pool, int64_t n_pages, int page, const int32_t* table, int max_pages, const int32_t* lens,
               int H, int d, const int32_t* begin, const int32_t* end, float scale, sa_dtype dt, void* ws,
               size_t ws_bytes, void* stream, bool bwd) {
  SA_TRY(set_pages(&a.c, pool, n_pages, page, table, max_pages, H, d));
  if (!cu_q || !lens || !std::isfinite(scale) || B < 1 || T < 0 || Hq < 1) return SA_ERR_INVALID_ARG;
  if (!attn_sizes_ok(B, T, Hq, H, d, dt)) return SA_ERR_UNSUPPORTED;
  if (T > 0 && (!q || !aligned(q, 16))) return SA_ERR_INVALID_ARG;
  if (!stride_ok(q_row, dt) || !stride_ok(q_head, dt)) return SA_ERR_INVALID_ARG;
  const bool tc = takes_tc(B, T, Hq / H, d, dt, scale, bwd);
  const Layout l = attn_layout(B, T, Hq / H, d, dt, bwd, tc);
  SA_TRY(check_workspace(ws, ws_bytes, l.total));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  char* base = static_cast<char*>(ws);
  if (T == 0) return cudaMemsetAsync(ws, 0, sizeof(sa::WsHeader), st) == cudaSuccess ? SA_OK : SA_ERR_CUDA;
  a.q = q;
  a.q_row = q_row;
  a.q_head = q_head;
  a.cu_q = cu_q;
  a.B = B;
  a.T = T;
  a.Hq = Hq;
  a.G = Hq / H;
  a.lens = lens;
  a.begin = begin;
  a.end = end;
  a.scale = scale;
  a.dt = dt;
  a.ws = ws;
  a.slots = reinterpret_cast<sa::WsHeader*>(base + l.slots);
  a.ctas = l.ctas;
  a.workers = l.workers;
  a.piece = base + l.piece;
  a.partial = reinterpret_cast<float*>(base + l.partial);
  a.wait_limit_ns = sa::wait_limit_ns();
  const cudaError_t e = tc ? sa::cache::launch_tc(a, bwd, st) : sa::cache::launch_mma(a, bwd, st);
  sa::count_launches(2);
  return e == cudaSuccess ? SA_OK : SA_ERR_CUDA;
}

}  // namespace

extern "C" {

size_t sa_cache_page_bytes(int H, int d, int page) {
  if (H < 1 || H > sa::kMaxH || !width_ok(d) || !page_ok(page)) return 0;
  return size_t(H) * 2 * size_t(page) * size_t(d / 2 + d / 16);
}

sa_status sa_cache_write(const void* K, const void* V, int64_t user_stride, int64_t row_stride, int64_t head_stride,
                         const int32_t* cu_seqlens, int B, int64_t N, const int32_t* start, int H, int d, sa_dtype dt,
                         void* pool, int64_t n_pages, int page, const int32_t* block_table, int max_pages,
                         void* workspace, size_t ws_bytes, void* stream) {
  RowArgs a{};
  SA_TRY(set_pages(&a.c, pool, n_pages, page, block_table, max_pages, H, d));
  a.cu = cu_seqlens;
  a.B = B;
  a.N = N;
  a.dt = dt;
  SA_TRY(check_rows(a));
  if (!cu_seqlens && N % B != 0) return SA_ERR_INVALID_ARG;
  if (N > 0 && (!K || !V || !aligned(K, 16) || !aligned(V, 16))) return SA_ERR_INVALID_ARG;
  if (!stride_ok(row_stride, dt) || !stride_ok(head_stride, dt) || !stride_ok(user_stride, dt))
    return SA_ERR_INVALID_ARG;
  SA_TRY(check_workspace(workspace, ws_bytes, sizeof(sa::WsHeader)));
  a.K = K;
  a.V = V;
  a.user_stride = user_stride;
  a.row_stride = row_stride;
  a.head_stride = head_stride;
  a.per_user = N / B;
  a.start = start;
  a.ws = workspace;
  const cudaError_t e = sa::cache::launch_write(a, static_cast<cudaStream_t>(stream));
  sa::count_launches(1);
  return e == cudaSuccess ? SA_OK : SA_ERR_CUDA;
}

sa_status sa_cache_read(const void* pool, int64_t n_pages, int page, const int32_t* block_table, int max_pages,
                        const int32_t* cu_seqlens, int B, int64_t N, const int32_t* start, int H, int d, sa_dtype dt,
                        void* K, void* V, void* workspace, size_t ws_bytes, void* stream) {
  RowArgs a{};
  SA_TRY(set_pages(&a.c, pool, n_pages, page, block_table, max_pages, H, d));
  a.cu = cu_seqlens;
  a.B = B;
  a.N = N;
  a.dt = dt;
  if (!cu_seqlens) return SA_ERR_INVALID_ARG;
  SA_TRY(check_rows(a));
  if (N > 0 && (!K || !V || !aligned(K, 16) || !aligned(V, 16))) return SA_ERR_INVALID_ARG;
  SA_TRY(check_workspace(workspace, ws_bytes, sizeof(sa::WsHeader)));
  a.Ko = K;
  a.Vo = V;
  a.start = start;
  a.ws = workspace;
  const cudaError_t e = sa::cache::launch_read(a, static_cast<cudaStream_t>(stream));
  sa::count_launches(1);
  return e == cudaSuccess ? SA_OK : SA_ERR_CUDA;
}

size_t sa_cache_attn_workspace_size(int B, int64_t T, int Hq, int H, int d, sa_dtype dt, int64_t max_tokens, int bwd) {
  if (!attn_sizes_ok(B, T, Hq, H, d, dt) || max_tokens < 0) return 0;
  // enough for either kernel: the scale and the path, which may change, have a say
  const size_t x = attn_layout(B, T, Hq / H, d, dt, bwd != 0, false).total;
  if (!sa::cache::tc_supported(B, T, Hq / H, d, dt, 1.f, bwd != 0)) return x;
  const size_t y = attn_layout(B, T, Hq / H, d, dt, bwd != 0, true).total;
  return x > y ? x : y;
}

sa_status sa_cache_attn_fwd(const void* q, int64_t q_row_stride, int64_t q_head_stride, const int32_t* cu_q, int B,
                            int64_t T, int Hq, const void* pool, int64_t n_pages, int page, const int32_t* block_table,
                            int max_pages, const int32_t* cache_lens, int H, int d, const int32_t* kv_begin,
                            const int32_t* kv_end, float scale, sa_dtype dt, void* out, float* lse, void* workspace,
                            size_t ws_bytes, void* stream) {
  if (T > 0 && (!out || !aligned(out, 16))) return SA_ERR_INVALID_ARG;
  AttnArgs a{};
  a.out = out;
  a.lse = lse;
  return attn(a, q, q_row_stride, q_head_stride, cu_q, B, T, Hq, pool, n_pages, page, block_table, max_pages,
              cache_lens, H, d, kv_begin, kv_end, scale, dt, workspace, ws_bytes, stream, false);
}

sa_status sa_cache_attn_bwd(const void* q, int64_t q_row_stride, int64_t q_head_stride, const int32_t* cu_q, int B,
                            int64_t T, int Hq, const void* pool, int64_t n_pages, int page, const int32_t* block_table,
                            int max_pages, const int32_t* cache_lens, int H, int d, const int32_t* kv_begin,
                            const int32_t* kv_end, float scale, sa_dtype dt, const void* out, const float* lse,
                            const void* dout, void* dq, void* workspace, size_t ws_bytes, void* stream) {
  if (T > 0 && (!out || !lse || !dout || !dq || !aligned(out, 16) || !aligned(dout, 16) || !aligned(dq, 16)))
    return SA_ERR_INVALID_ARG;
  AttnArgs a{};
  a.out = const_cast<void*>(out);
  a.lse = const_cast<float*>(lse);
  a.dout = dout;
  a.dq = dq;
  return attn(a, q, q_row_stride, q_head_stride, cu_q, B, T, Hq, pool, n_pages, page, block_table, max_pages,
              cache_lens, H, d, kv_begin, kv_end, scale, dt, workspace, ws_bytes, stream, true);
}

const char* sa_cache_attn_kernel_name(int B, int64_t T, int Hq, int H, int d, float scale, sa_dtype dt, int bwd) {
  if (!attn_sizes_ok(B, T, Hq, H, d, dt) || !std::isfinite(scale)) return "unsupported";
  if (takes_tc(B, T, Hq / H, d, dt, scale, bwd != 0)) return bwd ? "tc5_cache_attn_bwd" : "tc5_cache_attn_fwd";
  return bwd ? "mma_cache_attn_bwd" : "mma_cache_attn_fwd";
}

}  // extern "C"
