/*
 * sa_dense.h -- C ABI of libsa_sketch.so's dense operators: layer norm (of a sum)
 * and linear layers with bias, activation and residual, each with its gradient.
 *
 * They are what surrounds the sketching step in the stacked refinement (paper Sec. 3.3):
 *     X1 = LN(X~ + A X),   X~' = LN(X1 + FFN(X1)),   queries X~' W_Q, keys X W_K,
 * with FFN the SwiGLU layer of App. G.2, and in front of the targets (width adapter and
 * target map, Sec. 3.4).
 *
 * Conventions (otherwise those of sa_sketch.h: device pointers, the caller's stream and
 * memory, no synchronisation, bitwise reproducible results)
 *   - Matrices are rows of contiguous elements; `*_stride` is the distance of two rows in
 *     elements (any value >= 0 for inputs: rows may repeat or overlap).  Outputs are
 *     contiguous.  Base pointers are aligned to their element.
 *   - Outputs may not overlap inputs or one another, except where a call says so.
 *   - Where a norm's rows of x, r or dy do not start on 16 bytes, the 16-byte pieces that a row begins and ends in are read
 *     whole: up to 15 bytes beside the matrix, in the same piece as its first or last element. What they hold has no effect.
 *   - An output pointer that may be NULL is not computed then.
 *   - All arithmetic is in fp32 or better; each output is rounded to its type once.
 *   - `workspace` is 256-byte aligned and need not be cleared.  A linear call's first 256 bytes hold its status
 *     (sa_get_device_error): SA_ERR_TIMEOUT where a wait reached sa_set_wait_limit_ns's limit, and the outputs are undefined.
 */
#ifndef SA_DENSE_H
#define SA_DENSE_H

#include "sa_sketch.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------- layer norm
 * For each of `rows` rows, h = x + r (r NULL: h = x), over n features (1..16384):
 *     mean = sum h / n,  rstd = 1 / sqrt(sum (h - mean)^2 / n + eps),
 *     y = (h - mean) rstd w + b            (w NULL: 1, b NULL: 0)
 * x, r, y and the parameters have types of their own (SA_F32 or SA_BF16).  h is not
 * rounded before it is normalised.  eps > 0.  The squares are summed in fp32: a row whose sum of them exceeds 3.4e38
 * has rstd 0.
 *     x, r  : [rows, n] with strides      w, b : [n] of type w_dt
 *     y     : [rows, n] of type y_dt      stats: fp32 [rows, 2] = (mean, rstd), 8-byte aligned, or NULL
 * y may be x or r where type and layout are the same. */
sa_status sa_layer_norm_fwd(const void* x, int64_t x_stride, sa_dtype x_dt, const void* r, int64_t r_stride,
                            sa_dtype r_dt, const void* w, const void* b, sa_dtype w_dt, int64_t rows, int n, float eps,
                            void* y, sa_dtype y_dt, float* stats, void* stream);

/* Gradient: with xh = (h - mean) rstd and g = dy w,
 *     dh = rstd (g - sum g / n - xh sum(g xh) / n),   dw = sum_rows dy xh,   db = sum_rows dy
 * dx is dh in x's type and dr is dh in r's (either may be NULL; with r of x's type the
 * two are the same numbers).  dw, db : [n] of type w_dt (w NULL: of that type all the
 * same), NULL where not wanted.  stats are the forward's.  The rows are summed in fp32 in a
 * fixed order.  `workspace` has sa_layer_norm_workspace_size bytes; its first 256 are left
 * alone.  It may be NULL where neither dw nor db is asked for.
 *     dy : [rows, n] of type y_dt with strides;   dx : [rows, n] of x_dt;   dr : [rows, n] of r_dt */
size_t sa_layer_norm_workspace_size(int64_t rows, int n);
sa_status sa_layer_norm_bwd(const void* dy, int64_t dy_stride, sa_dtype y_dt, const void* x, int64_t x_stride,
                            sa_dtype x_dt, const void* r, int64_t r_stride, sa_dtype r_dt, const void* w,
                            sa_dtype w_dt, const float* stats, int64_t rows, int n, void* dx, void* dr, void* dw,
                            void* db, void* workspace, size_t ws_bytes, void* stream);

/* ----------------------------------------------------------------- linear
 * z = x W^T + b,   y = act(z) + r          (b NULL: 0, r NULL: 0)
 *     SA_ACT_NONE  z            SA_ACT_RELU  max(z, 0)
 *     SA_ACT_GELU  z Phi(z), Phi the normal distribution function
 *     SA_ACT_SILU  z / (1 + e^-z)
 *     SA_ACT_SWIGLU  W has 2 N rows, z = [a, u], y = a / (1 + e^-a) u + r
 * With Z = 2 N for SwiGLU and Z = N otherwise, all of type dt:
 *     x : [M, K] with strides    w : [Z, K] with strides    b : [Z]
 *     r : [M, N] with strides    y : [M, N]                 z : [M, Z], or NULL
 * The activation takes z before its rounding.  K >= 1, N >= 1, Z and K at most 2^20, M < 2^31 - 256.
 * bf16 products accumulate in fp32 on the tensor cores, whose additions round towards zero: a sum of terms of one sign
 * comes out less than 2^-13 too small, however long it is (6e-5 measured).  fp32 factors are split into three
 * bf16 terms each (exactly for sizes from 2^-110 on; of smaller ones, what lies below 2^-134 is lost), of which the six
 * largest products are taken (the rest is below 2^-23 of a product's size) and summed in fp32; with more than 16 rows an
 * infinite factor there gives a NaN.  y may not be r. */
typedef enum { SA_ACT_NONE = 0, SA_ACT_RELU = 1, SA_ACT_GELU = 2, SA_ACT_SILU = 3, SA_ACT_SWIGLU = 4 } sa_act;

/* `repack` says which operands need a copy in aligned rows, because their address or row
 * stride is not a multiple of 16 bytes or the stride is below the row's length: 1 for x, 2 for w,
 * 4 for dy.  Bits that need not be set do no harm. */
size_t sa_linear_workspace_size(int64_t M, int N, int K, sa_act act, sa_dtype dt, int bwd, int repack);
sa_status sa_linear_fwd(const void* x, int64_t x_stride, const void* w, int64_t w_stride, const void* b,
                        const void* r, int64_t r_stride, int64_t M, int N, int K, sa_act act, sa_dtype dt, void* y,
                        void* z, void* workspace, size_t ws_bytes, void* stream);

/* Gradient: dz = dy act'(z) (the forward's z; not looked at for SA_ACT_NONE),
 *     dx = dz W,   dW = dz^T x,   db = sum_rows dz          (each NULL where not wanted)
 * relu's slope at 0 is 0.  dz is rounded to dt where it enters the products (bf16: by up to 2^-8 relative, as any operand
 * there: dx and dW are 2.3e-3 from 64 bits, norm-wise, of which their own rounding is 1.7e-3; fp32: not), db sums it unrounded.
 *     dy : [M, N] with strides   z : [M, Z]   dx : [M, K]   dw : [Z, K]   db : [Z] */
sa_status sa_linear_bwd(const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, const void* w,
                        int64_t w_stride, const void* z, int64_t M, int N, int K, sa_act act, sa_dtype dt, void* dx,
                        void* dw, void* db, void* workspace, size_t ws_bytes, void* stream);

/* Name of the kernel that makes the products of a call with these sizes and aligned operands (pass: 0 y, 1 dx alone,
 * 2 dW alone).  sa_select_path(1) takes plain CUDA-core kernels for every call (a cross-check). */
const char* sa_linear_kernel_name(int64_t M, int N, int K, sa_act act, sa_dtype dt, int pass);

#ifdef __cplusplus
}
#endif
#endif /* SA_DENSE_H */
