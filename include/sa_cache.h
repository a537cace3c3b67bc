/*
 * sa_cache.h -- C ABI of libsa_sketch.so's 4-bit cache: writing rows of keys and
 * values into pages, reading them back, and attention over the pages.
 *
 * The paper keeps each user's sketch in a cache (Sec. 4.1) and lets the ranked
 * targets attend over it and over the recent history (Sec. 3.4); it fixes no
 * storage format.  Here a cached row takes 4 bits a feature and 8 bits a group
 * of 16 features, 28 % of its bf16 size.
 *
 * Format.  A group is 16 consecutive features of one row (token, head).
 *   - Its scale is the smallest s = (8 + m) 2^(e - 18), code 8 e + m in 8..225,
 *     with 7.5 s >= max |x|: the float16 whose upper eight bits, sign dropped, are
 *     the code (2^-14 .. 9216).  Larger values saturate at 7 x 9216 = 64512.
 *   - Its 16 levels are the whole numbers nearest to x / s, halves towards zero,
 *     at most 7 in size, each stored as level + 8 in four bits.
 *   - level x s has at most 7 significant bits, so it is exact in bf16 and float16.
 *   - The format holds no infinity (saturates) and no NaN (stored as zero).
 *   A page holds `page` tokens (a power of two, 16..256) of all H heads:
 *     pool   : uint8 [n_pages, H, 2, page * (d/2 + d/16)], keys first, then values;
 *     record : page rows of d/2 code bytes, then page rows of d/16 scale bytes.
 *     Each 32-bit word of codes holds 8 features, from the lowest four bits up
 *     0 2 4 6 1 3 5 7 (so that a mask leaves the pair 2i, 2i + 1 in the two halves).
 *   Position i of user b is token i % page of page block_table[b][i / page].
 *
 * Conventions (otherwise those of sa_sketch.h: device pointers, the caller's
 * stream and memory, no synchronisation, bitwise reproducible results)
 *   - d is a multiple of 16, 16..128; 1 <= H <= 64 cached heads.  max_pages * page and
 *     T * Hq / H are at most 2^31 - 256.
 *   - block_table : int32 [B, max_pages].  Entries outside a user's positions are
 *     not looked at.  A used entry outside [0, n_pages) is skipped and reported
 *     (SA_ERR_BAD_PAGE); the results of that call are then undefined.  Attention
 *     uses an entry where a query sees one of the page's positions.
 *   - `workspace` is 256-byte aligned and need not be cleared.  Its error word is
 *     read by sa_get_device_error(); bad offsets or starts give SA_ERR_BAD_SEQLENS and the
 *     call writes nothing.
 *   - The pool and every base pointer are 16-byte aligned; row and head strides
 *     are in elements and keep rows 16-byte aligned.
 */
#ifndef SA_CACHE_H
#define SA_CACHE_H

#include "sa_sketch.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A device-detected status of the calls below, besides those of sa_sketch.h. */
#define SA_ERR_BAD_PAGE ((sa_status)7)

/* Bytes of one page: 2 * H * page * (d/2 + d/16); 0 for unsupported sizes. */
size_t sa_cache_page_bytes(int H, int d, int page);

/* Write rows of keys and values into the cache.  User b's row i goes to position
 * start[b] + i (start NULL: 0).
 *   Packed rows (cu_seqlens given, N = cu_seqlens[B]): row i of user b, head h is
 *     at K + (cu_seqlens[b] + i) * row_stride + h * head_stride.
 *   Equal counts (cu_seqlens NULL, N = B * n for some n): it is at
 *     K + b * user_stride + i * row_stride + h * head_stride -- a batch of
 *     sketches [B, H, P, d] is written in place with head_stride P*d.
 * V has the same strides.  dt: SA_F32 or SA_BF16.  `workspace` is 256 bytes. */
sa_status sa_cache_write(const void* K, const void* V, int64_t user_stride, int64_t row_stride,
                         int64_t head_stride, const int32_t* cu_seqlens, int B, int64_t N,
                         const int32_t* start, int H, int d, sa_dtype dt, void* pool, int64_t n_pages,
                         int page, const int32_t* block_table, int max_pages, void* workspace,
                         size_t ws_bytes, void* stream);

/* Read positions start[b] .. start[b] + cu_seqlens[b+1] - cu_seqlens[b] - 1 of
 * every user back into packed rows K, V [N, H, d] of type dt (the stored values,
 * exact in either type).  `workspace` is 256 bytes. */
sa_status sa_cache_read(const void* pool, int64_t n_pages, int page, const int32_t* block_table, int max_pages,
                        const int32_t* cu_seqlens, int B, int64_t N, const int32_t* start, int H, int d,
                        sa_dtype dt, void* K, void* V, void* workspace, size_t ws_bytes, void* stream);

/* Attention of packed queries over the cache.  Query t of user b (cu_q[b] <= t <
 * cu_q[b+1]) and query head j reads cached head j / (Hq / H):
 *     S_i = scale q . k_i,   out = sum_i softmax(S)_i v_i,   lse = log sum_i exp S_i
 * over the positions max(0, kv_begin[t]) <= i < min(cache_lens[b], kv_end[t])
 * (NULL: 0 and cache_lens[b]).  A query that sees nothing gets out = 0 and
 * lse = -inf; what it does not see never reaches it, written or not.
 *     q, out : [T, Hq, d] of type dt; q has strides, out is contiguous
 *     lse    : [T, Hq] fp32, or NULL
 *     cu_q   : int32 [B + 1], cache_lens : int32 [B], kv_begin, kv_end : int32 [T]
 * Hq is a multiple of H.  Any finite scale.  Products take the cached values and
 * bf16 queries exactly (fp32 queries as three bf16 terms) and accumulate in fp32;
 * the weights are rounded to float16 before they meet the values (two float16
 * terms for fp32; a weight below 2^-37 of the largest counts as nothing), their
 * sum is kept in fp32.
 * The workspace is a few MB to tens of MB of unfinished pieces, one or two per worker; its
 * size depends on neither the lengths nor max_tokens, the most cached positions of a
 * user, which may not be negative. */
size_t sa_cache_attn_workspace_size(int B, int64_t T, int Hq, int H, int d, sa_dtype dt, int64_t max_tokens, int bwd);
sa_status sa_cache_attn_fwd(const void* q, int64_t q_row_stride, int64_t q_head_stride, const int32_t* cu_q, int B,
                            int64_t T, int Hq, const void* pool, int64_t n_pages, int page,
                            const int32_t* block_table, int max_pages, const int32_t* cache_lens, int H, int d,
                            const int32_t* kv_begin, const int32_t* kv_end, float scale, sa_dtype dt, void* out,
                            float* lse, void* workspace, size_t ws_bytes, void* stream);

/* Gradient of the queries (the cached rows are constants): with P_i =
 * exp(S_i - lse) and D = dout . out,
 *     dq = scale sum_i P_i (dout . v_i - D) k_i.
 * out and lse are the forward's; out, dout and dq are contiguous [T, Hq, d] of
 * type dt.  P (dout . v - D) is rounded to bf16 (three bf16 terms for fp32). */
sa_status sa_cache_attn_bwd(const void* q, int64_t q_row_stride, int64_t q_head_stride, const int32_t* cu_q, int B,
                            int64_t T, int Hq, const void* pool, int64_t n_pages, int page,
                            const int32_t* block_table, int max_pages, const int32_t* cache_lens, int H, int d,
                            const int32_t* kv_begin, const int32_t* kv_end, float scale, sa_dtype dt,
                            const void* out, const float* lse, const void* dout, void* dq, void* workspace,
                            size_t ws_bytes, void* stream);

/* Name of the kernel a call with these sizes runs on ("tc5..." = tcgen05, "mma..."
 * = warp-level tensor-core products, the cached rows dequantised in registers).
 * sa_select_path(1) takes the warp-level kernels for every call (a cross-check: there
 * are no CUDA-core ones); workspaces do not depend on it. */
const char* sa_cache_attn_kernel_name(int B, int64_t T, int Hq, int H, int d, float scale, sa_dtype dt, int bwd);

#ifdef __cplusplus
}
#endif
#endif /* SA_CACHE_H */
