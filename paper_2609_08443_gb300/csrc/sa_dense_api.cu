// Host side of the dense operators: argument checks, workspace layout, the choice of kernels and
// launches on the caller's stream.  Declarations and the meaning of every argument: include/sa_dense.h.
#include <cmath>

#include "sa_dense.cuh"
#include "sa_kernels.cuh"
#include "sa_tc_common.cuh"

namespace {

using sa::dense::Mat;

constexpr int64_t kMostRows = (int64_t(1) << 31) - 256;

#define SA_TRY(x)               \
  do {                          \
    const sa_status s_ = (x);   \
    if (s_ != SA_OK) return s_; \
  } while (0)

bool type_ok(sa_dtype dt) { return dt == SA_F32 || dt == SA_BF16; }
size_t size_of(sa_dtype dt) { return dt == SA_BF16 ? 2 : 4; }
bool to_element(const void* p, sa_dtype dt) { return reinterpret_cast<uintptr_t>(p) % size_of(dt) == 0; }

sa_status check_mat(const Mat& m, bool needed) {
  if (!type_ok(m.dt)) return SA_ERR_UNSUPPORTED;
  if ((needed && !m.p) || !to_element(m.p, m.dt) || m.stride < 0) return SA_ERR_INVALID_ARG;
  return SA_OK;
}

sa_status check_workspace(const void* ws, size_t bytes, size_t need) {
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 256 != 0) return SA_ERR_INVALID_ARG;
  return bytes < need ? SA_ERR_WORKSPACE : SA_OK;
}

sa_status status(cudaError_t e) { return e == cudaSuccess ? SA_OK : SA_ERR_CUDA; }

// ------------------------------------------------------------- layer norm

sa_status check_norm(const sa::dense::NormArgs& a) {
  if (a.rows < 0 || a.n < 1) return SA_ERR_INVALID_ARG;
  if (a.rows > kMostRows || a.n > sa::dense::kMaxNorm || !type_ok(a.w_dt) || !type_ok(a.y_dt)) return SA_ERR_UNSUPPORTED;
  SA_TRY(check_mat(a.x, a.rows > 0));
  SA_TRY(check_mat(a.r, false));
  if (!to_element(a.w, a.w_dt) || !to_element(a.b, a.w_dt)) return SA_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(a.stats) % 8 != 0) return SA_ERR_INVALID_ARG;
  return SA_OK;
}

// ----------------------------------------------------------------- linear

struct Linear {
  int64_t M;
  int N, K, Z;
  int act;
  sa_dtype dt;
};

bool linear_sizes_ok(int64_t M, int N, int K, int act, sa_dtype dt) {
  return M >= 0 && N >= 1 && K >= 1 && M <= kMostRows && act >= SA_ACT_NONE && act <= SA_ACT_SWIGLU && type_ok(dt) &&
         K <= sa::dense::kMaxWidth && N <= sa::dense::kMaxWidth / (act == SA_ACT_SWIGLU ? 2 : 1);
}

sa_status make_linear(Linear* l, int64_t M, int N, int K, sa_act act, sa_dtype dt) {
  if (M < 0 || N < 1 || K < 1 || act < SA_ACT_NONE || act > SA_ACT_SWIGLU) return SA_ERR_INVALID_ARG;
  if (!linear_sizes_ok(M, N, K, act, dt)) return SA_ERR_UNSUPPORTED;
  *l = Linear{M, N, K, act == SA_ACT_SWIGLU ? 2 * N : N, act, dt};
  return SA_OK;
}

// Which matrices TMA cannot read as they are (include/sa_dense.h): copied into aligned rows first.
enum { COPY_X = 1, COPY_W = 2, COPY_DY = 4 };

// Sections of a linear call's workspace: the operands' copies (fp32: their terms), dz, the pieces of cut tiles (of
// one product at a time) and the partial column sums.
struct Layout {
  size_t x, w, dz, dz_terms, piece, partial, dx_partial, total;
  sa::dense::TcPlan plan, dx, dw, side_dx, side_dw;  // of y; of either gradient alone; of both side by side
  bool side;
};

// A product of this many rows of x is a matter of reading W (sa_dense_rows.cu), and takes no workspace on any path.  us, rows
// kernel | tensor cores: bf16 1024 -> 1024, 1 row 2.6 | 8.8, 16 rows 3.1 | 8.9, 32 rows (in two calls) 5.6 | 9.2; 4096 -> 8192
// gated, 16 rows 26 | 34, 17 rows 48 | 34; 8192 -> 1024, 16 rows 11.3 | 13.3, 17 rows 17.5 | 13.3.  fp32 4096 -> 8192 gated,
// 16 rows 161 | 189, 17 rows 236 | 190; 8192 -> 1024, 16 rows 22 | 30, 17 rows 31 | 31.  The other way round: fp32 of unaligned
// rows (4095 -> 4096), 8 rows 38 | 56, 16 rows 87 | 56.
bool few_rows(const Linear& l) { return l.M <= sa::dense::kMostFewRows; }

int64_t pitch_of(int64_t cols) { return (cols + 7) / 8 * 8; }

// Few rows' gradients go without the tensor cores where these would want a copy of W: in bf16 up to 4 rows of an unaligned W
// (us, rows kernels | tensor cores: 4095 -> 4096, 4 rows 51 | 63, 8 rows 111 | 62; aligned, 1024 -> 4096, 4 rows 27 | 18), in fp32
// up to 16, which also keep infinite factors (1024 -> 4096, 4 rows 25 | 33, 16 rows 42 | 32; 4096 -> 8192 gated, 4 rows 111 |
// 247, 16 rows 187 | 248; 8192 -> 1024, 4 rows 33 | 43, 16 rows 61 | 44).
bool few_rows_grads(const Linear& l, int repack) {
  return l.M > 0 && l.M <= sa::dense::most_few_grads(l.dt) && (l.dt == SA_F32 || (repack & COPY_W));
}

Layout linear_layout(const Linear& l, bool bwd, int repack) {
  Layout s{};
  const bool f32 = l.dt == SA_F32;
  // few rows' gradients in fp32, or with a W that needs a copy, never reach the tensor cores
  const bool few_f32 = bwd && f32 && few_rows(l);
  if (f32) repack = few_f32 ? 0 : COPY_X | COPY_W | COPY_DY;
  if (bwd && l.M <= sa::dense::most_few_grads(l.dt)) repack &= ~COPY_W;
  size_t off = sizeof(sa::WsHeader);
  auto section = [&](bool there, size_t bytes) {
    const size_t at = off;
    if (there) off = sa::align256(off + bytes);
    return at;
  };
  const size_t each = f32 ? 6 : 2;  // bytes of an element's terms
  if (!bwd && few_rows(l)) repack = 0;
  s.x = section(repack & COPY_X, size_t(l.M) * pitch_of(l.K) * each);
  s.w = section(repack & COPY_W, size_t(l.Z) * pitch_of(l.K) * each);
  size_t piece = 0;
  if (!bwd && few_rows(l)) {
    // no workspace but the status
  } else if (!bwd) {
    s.plan = sa::dense::tc_plan(l.M, l.N, l.K, l.act, f32);
    piece = s.plan.piece_bytes;
  } else {
    const bool act = l.act != SA_ACT_NONE;
    // dz, or dy's copy, or fp32's terms of either: in one place, since only the CUDA-core path has an fp32 dz and no terms
    const bool terms = f32 && !few_f32;
    s.dz = s.dz_terms = section(act || terms || (repack & COPY_DY), size_t(l.M) * pitch_of(l.Z) * (terms ? each : size_of(l.dt)));
    s.dx = sa::dense::tc_plan(l.M, l.K, l.Z, sa::dense::kPlain, f32);
    s.dw = sa::dense::tc_plan(l.Z, l.K, l.M, sa::dense::kPlain, f32);
    s.side = sa::dense::tc_plan_grads(l.M, l.Z, l.K, f32, s.dx.cost + s.dw.cost, &s.side_dx, &s.side_dw);
    piece = few_f32 ? 0 : s.dx.piece_bytes > s.dw.piece_bytes ? s.dx.piece_bytes : s.dw.piece_bytes;
    if (s.side && !few_f32 && s.side_dx.piece_bytes + s.side_dw.piece_bytes > piece)
      piece = s.side_dx.piece_bytes + s.side_dw.piece_bytes;
  }
  s.piece = section(piece > 0, piece);
  s.partial = section(bwd, size_t(sa::dense::act_grad_blocks(l.M, l.N)) * size_t(l.Z) * sizeof(float));
  // whichever way few rows go, which an operand's alignment has a say in, the size is enough
  s.dx_partial = section(bwd && l.M <= sa::dense::most_few_grads(l.dt), size_t(sa::dense::rows_dx_shares(l.Z, l.K)) * size_t(l.M) * size_t(l.K) * sizeof(float));
  s.total = off;
  return s;
}


bool on_tensor_cores() {
  static std::atomic<int> known[64];  // 0: not asked yet, 1: yes, 2: no
  if (!sa::tc_path_enabled()) return false;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  if (dev >= 64) return sa::tcc::device_is_sm103();
  int k = known[dev].load(std::memory_order_relaxed);
  if (k == 0) {
    k = sa::tcc::device_is_sm103() ? 1 : 2;
    known[dev].store(k, std::memory_order_relaxed);
  }
  return k == 1;
}

int repack_bits(const Mat& x, const Mat& w, const Mat& dy, const Linear& l) {
  auto need = [&](const Mat& m, int64_t len) {
    return reinterpret_cast<uintptr_t>(m.p) % 16 != 0 || m.stride * int64_t(size_of(m.dt)) % 16 != 0 || m.stride < len;
  };
  return (need(x, l.K) ? COPY_X : 0) | (need(w, l.K) ? COPY_W : 0) | (dy.p && need(dy, l.N) ? COPY_DY : 0);
}

// A product's operand: the rows as they are, or their copy at `at`, which is made by the launch of `r`.
sa::dense::TcOperand operand(const Mat& m, int64_t rows, int64_t cols, bool copy, void* at, sa::dense::Repack* r) {
  sa::dense::TcOperand o{m.p, rows, cols, m.stride};
  if (!copy && m.dt == SA_BF16) return o;
  o.p = at;
  o.pitch = pitch_of(cols);
  *r = sa::dense::Repack{m, rows, int(cols), at, o.pitch, 0};
  return o;
}

cudaError_t repack(const sa::dense::Repack& r0, const sa::dense::Repack& r1, cudaStream_t st, int* launches) {
  if (!r0.dst && !r1.dst) return cudaSuccess;
  ++*launches;
  return sa::dense::launch_repack(r0, r1, st);
}

}  // namespace

extern "C" {

size_t sa_layer_norm_workspace_size(int64_t rows, int n) {
  if (rows < 0 || rows > kMostRows || n < 1 || n > sa::dense::kMaxNorm) return 0;
  return sizeof(sa::WsHeader) +
         sa::align256(size_t(sa::dense::norm_bwd_blocks(rows, n)) * 2 * size_t(n) * sizeof(float));
}

sa_status sa_layer_norm_fwd(const void* x, int64_t x_stride, sa_dtype x_dt, const void* r, int64_t r_stride,
                            sa_dtype r_dt, const void* w, const void* b, sa_dtype w_dt, int64_t rows, int n, float eps,
                            void* y, sa_dtype y_dt, float* stats, void* stream) {
  sa::dense::NormArgs a{};
  a.x = Mat{x, x_stride, x_dt};
  a.r = Mat{r, r_stride, r ? r_dt : SA_F32};
  a.dy = Mat{nullptr, 0, SA_F32};
  a.w = w;
  a.b = b;
  a.w_dt = w_dt;
  a.rows = rows;
  a.n = n;
  a.eps = eps;
  a.y = y;
  a.y_dt = y_dt;
  a.stats = stats;
  SA_TRY(check_norm(a));
  if (!(eps > 0.f) || !std::isfinite(eps)) return SA_ERR_INVALID_ARG;
  if (!to_element(y, y_dt) || (rows > 0 && !y)) return SA_ERR_INVALID_ARG;
  if (rows == 0) return SA_OK;
  const cudaError_t e = sa::dense::launch_norm_fwd(a, static_cast<cudaStream_t>(stream));
  sa::count_launches(1);
  return status(e);
}

sa_status sa_layer_norm_bwd(const void* dy, int64_t dy_stride, sa_dtype y_dt, const void* x, int64_t x_stride,
                            sa_dtype x_dt, const void* r, int64_t r_stride, sa_dtype r_dt, const void* w,
                            sa_dtype w_dt, const float* stats, int64_t rows, int n, void* dx, void* dr, void* dw,
                            void* db, void* workspace, size_t ws_bytes, void* stream) {
  sa::dense::NormArgs a{};
  a.x = Mat{x, x_stride, x_dt};
  a.r = Mat{r, r_stride, r ? r_dt : SA_F32};
  a.dy = Mat{dy, dy_stride, y_dt};
  a.w = w;
  a.w_dt = w_dt;
  a.rows = rows;
  a.n = n;
  a.y_dt = y_dt;
  a.stats = const_cast<float*>(stats);
  a.dx = dx;
  a.dr = dr;
  a.dw = dw;
  a.db = db;
  SA_TRY(check_norm(a));
  SA_TRY(check_mat(a.dy, rows > 0));
  if (rows > 0 && !stats) return SA_ERR_INVALID_ARG;
  if ((dr && !r) || !to_element(dx, x_dt) || !to_element(dr, a.r.dt) || !to_element(dw, w_dt) || !to_element(db, w_dt))
    return SA_ERR_INVALID_ARG;
  if (dw || db) {
    SA_TRY(check_workspace(workspace, ws_bytes, sa_layer_norm_workspace_size(rows, n)));
    a.partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + sizeof(sa::WsHeader));
  } else if (rows == 0 || (!dx && !dr)) {
    return SA_OK;
  }
  int launches = 0;
  const cudaError_t e = sa::dense::launch_norm_bwd(a, static_cast<cudaStream_t>(stream), &launches);
  sa::count_launches(launches);
  return status(e);
}

size_t sa_linear_workspace_size(int64_t M, int N, int K, sa_act act, sa_dtype dt, int bwd, int repack) {
  Linear l;
  if (make_linear(&l, M, N, K, act, dt) != SA_OK) return 0;
  return linear_layout(l, bwd != 0, repack).total;
}

sa_status sa_linear_fwd(const void* x, int64_t x_stride, const void* w, int64_t w_stride, const void* b,
                        const void* r, int64_t r_stride, int64_t M, int N, int K, sa_act act, sa_dtype dt, void* y,
                        void* z, void* workspace, size_t ws_bytes, void* stream) {
  Linear l;
  SA_TRY(make_linear(&l, M, N, K, act, dt));
  const Mat mx{x, x_stride, dt}, mw{w, w_stride, dt}, mr{r, r_stride, dt};
  SA_TRY(check_mat(mx, M > 0));
  SA_TRY(check_mat(mw, true));
  SA_TRY(check_mat(mr, false));
  if ((M > 0 && !y) || !to_element(y, dt) || !to_element(z, dt) || !to_element(b, dt)) return SA_ERR_INVALID_ARG;
  const int copies = repack_bits(mx, mw, Mat{nullptr, 0, dt}, l);
  const Layout lay = linear_layout(l, false, copies);
  SA_TRY(check_workspace(workspace, ws_bytes, lay.total));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  char* base = static_cast<char*>(workspace);
  const bool few = few_rows(l);
  if (M == 0 || few || !on_tensor_cores()) {
    const bool rows = few && sa::tc_path_enabled();
    if ((M == 0 || !rows) && cudaMemsetAsync(workspace, 0, sizeof(sa::WsHeader), st) != cudaSuccess) return SA_ERR_CUDA;
    if (M == 0) return SA_OK;
    sa::dense::GemmArgs g{};
    g.A = x;
    g.a_m = x_stride;
    g.a_k = 1;
    g.B = w;
    g.b_n = w_stride;
    g.b_k = 1;
    g.M = M;
    g.N = N;
    g.K = K;
    g.bias = b;
    g.r = mr;
    g.act = act;
    g.dt = dt;
    g.y = y;
    g.z = z;
    g.ws = workspace;
    sa::count_launches(1);
    return status(rows ? sa::dense::launch_rows(g, st) : sa::dense::launch_simt_gemm(g, st));
  }
  int launches = 0;
  sa::dense::TcGemm g{};
  sa::dense::Repack rx{}, rw{};
  g.A = operand(mx, M, K, copies & COPY_X, base + lay.x, &rx);
  g.B = operand(mw, l.Z, K, copies & COPY_W, base + lay.w, &rw);
  cudaError_t e = repack(rx, rw, st, &launches);
  g.M = M;
  g.N = N;
  g.bias = b;
  g.r = mr;
  g.act = act;
  g.dt = dt;
  g.y = y;
  g.z = z;
  g.piece = reinterpret_cast<float*>(base + lay.piece);
  g.ws = workspace;
  g.clear = 1;
  if (e == cudaSuccess)
    e = sa::dense::launch_tc_gemm(g, lay.plan, st, &launches);
  sa::count_launches(launches);
  return status(e);
}

sa_status sa_linear_bwd(const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, const void* w,
                        int64_t w_stride, const void* z, int64_t M, int N, int K, sa_act act, sa_dtype dt, void* dx,
                        void* dw, void* db, void* workspace, size_t ws_bytes, void* stream) {
  Linear l;
  SA_TRY(make_linear(&l, M, N, K, act, dt));
  const Mat mx{x, x_stride, dt}, mw{w, w_stride, dt}, mdy{dy, dy_stride, dt};
  SA_TRY(check_mat(mx, M > 0));
  SA_TRY(check_mat(mw, true));
  SA_TRY(check_mat(mdy, M > 0));
  if ((M > 0 && act != SA_ACT_NONE && !z) || !to_element(z, dt) || !to_element(dx, dt) || !to_element(dw, dt) ||
      !to_element(db, dt))
    return SA_ERR_INVALID_ARG;
  const int copies = repack_bits(mx, mw, mdy, l);
  const Layout lay = linear_layout(l, true, copies);
  SA_TRY(check_workspace(workspace, ws_bytes, lay.total));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  char* base = static_cast<char*>(workspace);
  const bool few = few_rows_grads(l, copies) && sa::tc_path_enabled();
  const bool tc = !few && on_tensor_cores() && M > 0 && (dx || dw);
  if (!tc && cudaMemsetAsync(workspace, 0, sizeof(sa::WsHeader), st) != cudaSuccess) return SA_ERR_CUDA;

  // dz and the columns' sums
  sa::dense::ActGradArgs a{};
  a.dy = mdy;
  a.z = act == SA_ACT_NONE ? nullptr : z;
  a.M = M;
  a.N = N;
  a.Z = l.Z;
  a.act = act;
  const bool terms = tc && dt == SA_F32;  // dz goes straight into the products' terms
  a.dz = act == SA_ACT_NONE || (!dx && !dw) ? nullptr : base + (terms ? lay.dz_terms : lay.dz);
  a.terms = terms;
  a.pitch = pitch_of(l.Z);
  a.partial = db ? reinterpret_cast<float*>(base + lay.partial) : nullptr;
  int launches = 0;
  cudaError_t e = cudaSuccess;
  if (M > 0 && (a.dz || a.partial)) {
    e = sa::dense::launch_act_grad(a, st);
    ++launches;
  }
  if (e == cudaSuccess && db) {
    e = sa::dense::launch_join_columns(a.partial, sa::dense::act_grad_blocks(M, N), l.Z, l.Z, db, dt, st);
    ++launches;
  }
  const Mat dz = a.dz ? Mat{a.dz, a.pitch, dt} : mdy;
  if (few) {
    sa::dense::RowsGradArgs r{};
    r.dz = dz.p;
    r.w = w;
    r.x = x;
    r.pitch = dz.stride;
    r.w_stride = w_stride;
    r.x_stride = x_stride;
    r.M = int(M);
    r.Z = l.Z;
    r.K = K;
    r.dt = dt;
    r.partial = reinterpret_cast<float*>(base + lay.dx_partial);
    r.dx = dx;
    r.dw = dw;
    if (e == cudaSuccess) e = sa::dense::launch_rows_grads(r, st, &launches);
  } else if (tc) {
    sa::dense::Repack rz{}, rx{}, rw{};
    sa::dense::TcOperand oz{a.dz, M, l.Z, a.pitch};
    if (!a.dz) oz = operand(dz, M, l.Z, copies & COPY_DY, base + lay.dz_terms, &rz);
    const sa::dense::TcOperand ox = dw ? operand(mx, M, K, copies & COPY_X, base + lay.x, &rx) : sa::dense::TcOperand{};
    const sa::dense::TcOperand ow = dx ? operand(mw, l.Z, K, copies & COPY_W, base + lay.w, &rw) : sa::dense::TcOperand{};
    if (e == cudaSuccess) e = repack(rx, rw, st, &launches);
    if (e == cudaSuccess) e = repack(rz, sa::dense::Repack{}, st, &launches);
    sa::dense::TcGemm gx{}, gw{};
    gx.dt = gw.dt = dt;
    gx.piece = gw.piece = reinterpret_cast<float*>(base + lay.piece);
    gx.ws = gw.ws = workspace;
    gx.A = gw.A = oz;
    gx.clear = 1;
    gw.clear = !dx;
    gx.B = ow;  // dx = dz W
    gx.b_mn = 1;
    gx.M = M;
    gx.y = dx;
    gw.B = ox;  // dW = dz^T x
    gw.a_mn = gw.b_mn = 1;
    gw.M = l.Z;
    gw.y = dw;
    gx.N = gw.N = K;
    if (dx && dw && lay.side) {
      gw.piece += lay.side_dx.piece_bytes / sizeof(float);
      if (e == cudaSuccess) e = sa::dense::launch_tc_grads(gx, lay.side_dx, gw, lay.side_dw, st, &launches);
    } else {
      if (e == cudaSuccess && dx) e = sa::dense::launch_tc_gemm(gx, lay.dx, st, &launches);
      if (e == cudaSuccess && dw) e = sa::dense::launch_tc_gemm(gw, lay.dw, st, &launches);
    }
  } else {
    sa::dense::GemmArgs g{};
    g.A = dz.p;
    g.dt = dt;
    if (e == cudaSuccess && dx && M > 0) {
      g.a_m = dz.stride;
      g.a_k = 1;
      g.B = w;
      g.b_n = 1;
      g.b_k = w_stride;
      g.M = M;
      g.N = K;
      g.K = l.Z;
      g.y = dx;
      e = sa::dense::launch_simt_gemm(g, st);
      ++launches;
    }
    if (e == cudaSuccess && dw) {
      g.a_m = 1;
      g.a_k = dz.stride;
      g.B = x;
      g.b_n = 1;
      g.b_k = x_stride;
      g.M = l.Z;
      g.N = K;
      g.K = M;
      g.y = dw;
      e = sa::dense::launch_simt_gemm(g, st);
      ++launches;
    }
  }
  sa::count_launches(launches);
  return status(e);
}

const char* sa_linear_kernel_name(int64_t M, int N, int K, sa_act act, sa_dtype dt, int pass) {
  if (!linear_sizes_ok(M, N, K, act, dt) || pass < 0 || pass > 2) return "unsupported";
  if (M <= sa::dense::kMostFewRows && sa::tc_path_enabled() && (pass == 0 || (dt == SA_F32 && M > 0)))
    return pass == 0 && dt == SA_BF16 ? "mma_linear_rows" : "linear_rows";
  if (!on_tensor_cores()) return "simt_linear";
  const int64_t Z = act == SA_ACT_SWIGLU ? 2 * int64_t(N) : N;
  const bool f32 = dt == SA_F32;
  const sa::dense::TcPlan p = pass == 0   ? sa::dense::tc_plan(M, N, K, act, f32)
                              : pass == 1 ? sa::dense::tc_plan(M, K, Z, sa::dense::kPlain, f32)
                                          : sa::dense::tc_plan(Z, K, M, sa::dense::kPlain, f32);
  return f32 ? "tc5_linear_f32" : p.ctas == 2 ? "tc5_linear_pair" : "tc5_linear";
}

}  // extern "C"
