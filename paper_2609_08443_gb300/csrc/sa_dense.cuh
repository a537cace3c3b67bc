// Interface of the dense operators' kernels (include/sa_dense.h): layer norm and linear layers.
#pragma once
#include <atomic>

#include "sa_common.cuh"

#include "../../include/sa_dense.h"

namespace sa {
namespace dense {

constexpr int kMaxNorm = 16384;  // features of a normalised row
constexpr int kMaxWidth = 1 << 20;  // K and Z of a linear layer

// A matrix of contiguous rows.
struct Mat {
  const void* p;
  int64_t stride;  // elements between rows
  sa_dtype dt;
};

struct NormArgs {
  Mat x, r, dy;  // r.p NULL: no second summand
  const void* w;
  const void* b;
  sa_dtype w_dt;
  int64_t rows;
  int n;
  float eps;
  void* y;
  sa_dtype y_dt;
  float* stats;
  void *dx, *dr, *dw, *db;
  float* partial;  // [blocks][2][n]: column sums of the blocks (backward)
};

cudaError_t launch_norm_fwd(const NormArgs& a, cudaStream_t st);
cudaError_t launch_norm_bwd(const NormArgs& a, cudaStream_t st, int* launches);
int norm_bwd_blocks(int64_t rows, int n);  // blocks that leave partial column sums

// dst[c] = sum over g < G of partial[g * pitch + c], c < n, in order of g, rounded to dt.
cudaError_t launch_join_columns(const float* partial, int G, int64_t pitch, int64_t n, void* dst, sa_dtype dt,
                                cudaStream_t st);

// The same for two sets in one launch (d NULL: none).
cudaError_t launch_join_columns2(const float* p0, int G, int64_t pitch, int64_t n0, void* d0, const float* p1, int64_t n1,
                                 void* d1, sa_dtype dt, cudaStream_t st);

// C[m, n] = sum_k A(m, k) B(n, k) and what follows it.
struct GemmArgs {
  const void* A;
  const void* B;
  int64_t a_m, a_k, b_n, b_k;  // element strides
  int64_t M;
  int N;  // columns of y (SwiGLU: B has 2 N rows)
  int64_t K;
  const void* bias;
  Mat r;
  int act;
  sa_dtype dt;
  void* y;
  void* z;
  void* ws;  // launch_rows: the call's status, cleared
};

cudaError_t launch_simt_gemm(const GemmArgs& g, cudaStream_t st);
constexpr int kMostFewRows = 16;
// y for at most kMostFewRows rows of x
cudaError_t launch_rows(const GemmArgs& g, cudaStream_t st);

// Gradients for at most so many rows, without the tensor cores: dx [M, K] from shares of W's rows
// (partial: [rows_dx_shares][M][K]), dW [Z, K]; NULL where not wanted.
constexpr int most_few_grads(sa_dtype dt) { return dt == SA_BF16 ? 4 : kMostFewRows; }
struct RowsGradArgs {
  const void *dz, *w, *x;  // dz [M, Z], w [Z, K], x [M, K]
  int64_t pitch, w_stride, x_stride;
  int M, Z, K;
  sa_dtype dt;
  float* partial;
  void *dx, *dw;
};
int rows_dx_shares(int64_t Z, int64_t K);
cudaError_t launch_rows_grads(const RowsGradArgs& a, cudaStream_t st, int* launches);

// dz = dy act'(z) as [M, Z] rows of type dt, `pitch` elements apart (dz NULL: not stored), and
// column sums of the unrounded dz into partial[g * Z + c] (NULL: none).
struct ActGradArgs {
  Mat dy;
  const void* z;
  int64_t M;
  int N, Z;
  int act;
  void* dz;        // type dt; fp32: as three planes of bf16 terms where `terms` is set
  int64_t pitch;
  int terms;
  float* partial;
};
cudaError_t launch_act_grad(const ActGradArgs& a, cudaStream_t st);
int act_grad_blocks(int64_t M, int N);

// A matrix of bf16 rows `pitch` elements apart, 16-byte aligned, as TMA reads it; of fp32 values three planes of
// terms, one behind the other.
struct TcOperand {
  const void* p;
  int64_t rows, cols, pitch;
};

// How a product's tiles are dealt out (sa_dense_tc.cu).
struct TcPlan {
  int ctas, W;  // CTAs of a worker, workers
  int64_t mt, nt, KB, whole, cut;
  int cutters;  // workers that share the cut tiles
  size_t piece_bytes, sums_at;  // of cut tiles' pieces and, from sums_at on, of the sums of tiles in several runs
  double cost, bytes;  // estimated time (sa_dense_tc.cu has the unit), what has to move
};

// C[m, n] = sum_k A(m, k) B(n, k) on tcgen05.  K-major operands have k along their rows (a_mn, b_mn 0).
struct TcGemm {
  TcOperand A, B;
  int a_mn, b_mn;
  int64_t M;
  int N;
  const void* bias;
  Mat r;
  int act;
  sa_dtype dt;
  void* y;
  void* z;
  float* piece;
  void* ws;
  int clear;
};

// How a product ends: as it is, with bias, activation and residual, or as SwiGLU.
enum { EPI_PLAIN = 0, EPI_FULL = 1, EPI_GATED = 2 };
// `act`: kPlain for a product that ends as it is.
constexpr int kPlain = -1;
TcPlan tc_plan(int64_t M, int64_t N, int64_t K, int act, bool f32, int sms = 0, int ctas_only = 0);
cudaError_t launch_tc_gemm(const TcGemm& g, const TcPlan& p, cudaStream_t st, int* launches);
// Plans of dx = dz W and dW = dz^T x (dz [M, Z], W [Z, K]) side by side (launch_tc_grads), where that is better than one
// after the other at a cost of `apart`.
bool tc_plan_grads(int64_t M, int64_t Z, int64_t K, bool f32, double apart, TcPlan* x, TcPlan* w);
cudaError_t launch_tc_grads(const TcGemm& gx, const TcPlan& px, const TcGemm& gw, const TcPlan& pw, cudaStream_t st,
                            int* launches);

// A copy of rows in bf16 (fp32: three planes of terms), `pitch` elements apart, filled up with zeros.
struct Repack {
  Mat src;
  int64_t rows;
  int cols;
  void* dst;  // NULL: nothing to copy
  int64_t pitch;
  int vec;
};
cudaError_t launch_repack(Repack r0, Repack r1, cudaStream_t st);

int sm_count();

// Lets a kernel take `bytes` of dynamic shared memory on the current device; asked of the runtime once a device.  A kernel
// asks for the same number at all times: threads' calls may come in any order.
template <auto Kernel>
cudaError_t allow_smem(size_t bytes) {
  static std::atomic<bool> allowed[64];
  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 64 && allowed[dev].load(std::memory_order_relaxed)) return cudaSuccess;
  const cudaError_t s = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(bytes));
  if (s == cudaSuccess && dev < 64) allowed[dev].store(true, std::memory_order_relaxed);
  return s;
}

}  // namespace dense
}  // namespace sa
