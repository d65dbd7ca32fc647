/*
 * attn.h - C ABI of the MI355X (gfx950) attention product, its gradient and its cache, with a
 * caller-given device-memory limit.  Part of the same shared library as knn.h, kmv.h and sgpr.h and
 * sharing their conventions (row-major matrices with leading dimensions in elements, DEVICE / HOST
 * pointers, decimal size units, no ownership taken, knn_status return codes, knn_last_hip_error()).
 *
 * Operation.  kmv_apply multiplies an n x m matrix of exponentials by a vector without the matrix
 * ever existing.  Attention is that product with rows that add up to one and values that are rows:
 *     O_i = sum_j P_ij V_j,   P_ij = exp(s_ij - lse_i),   lse_i = log sum_j exp(s_ij),
 *     s_ij = w_ij - slope |p_i - j|,   w_ij = cap tanh(u_ij / cap)  (u_ij without a cap),
 *     u_ij = scale <Q_i, K_j>,
 * the sums over the keys j that row i sees.  The n x m matrices s and P are the big intermediates of
 * paper section 4.3: they are made tile by tile in registers on the matrix cores, reduced at once
 * (a running maximum and sum per row) and dropped.
 *
 * Which keys a row sees.  Rows and keys are cut into `docs` documents by starts and k_starts; a row
 * sees keys of its own document only.  Row t (from 0) of a document with nq rows and nk keys stands
 * at p = t + nk - nq among the keys j = 0 .. nk - 1 of the document (the last row at the last key).
 * Without `causal` it sees all of them, with it those with j <= p and those with j < prefix.  A row
 * that sees none has O = 0, lse = -infinity and gradients 0.
 *
 * Heads.  Q and O have hq heads, K and V hkv; hkv divides hq, and head h reads K and V of head
 * h / (hq / hkv).  Gradients of K and V are sums over the heads that read them.
 */
#ifndef ATTN_MI355X_H
#define ATTN_MI355X_H

#include <stdint.h>

#include "knn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ATTN_MAX_D 128 /* entries of a row */

/* types of Q, K, V, O and of the gradients, all the same */
typedef enum { ATTN_BF16 = 0, ATTN_F16 = 1 } attn_dtype;

/*
 * A DEVICE tensor [rows][heads][d]: entry t of row i of head h is at data + i * ld + h * hs + t
 * (elements).  ld, hs >= 0; an output's entries must not overlap each other or an input.
 * Rows are read 16 bytes at a time where data is 16-byte aligned and d, ld and hs are multiples
 * of 8; otherwise entry by entry, which is slower and gives the same results.
 */
typedef struct {
    void *data;
    int64_t ld, hs;
} attn_rows_t;

typedef struct {
    int32_t dtype;            /* attn_dtype */
    int32_t causal;           /* 0 or 1 */
    double scale;             /* > 0, finite */
    double cap;               /* 0: none; else > 0, finite */
    const float *slopes;      /* DEVICE [hq], finite; NULL: none.  Not differentiated */
    int64_t docs;             /* >= 1 with starts; without starts there is one document */
    const int32_t *starts;    /* DEVICE [docs + 1], ascending, within 0 .. n; NULL: 0, n */
    const int32_t *k_starts;  /* DEVICE [docs + 1], ascending, within 0 .. m; NULL together with starts */
    const int32_t *prefix;    /* DEVICE [docs]; NULL: none.  Only looked at with causal */
} attn_options_t;

/*
 * The plan.  One workgroup owns tile_rows rows of one head and walks the keys; where that leaves
 * compute units idle and the limit has room, the keys are cut into n_splits ranges walked
 * concurrently, whose unnormalised sums, maxima and totals (fp32) lie in the workspace until a last
 * kernel joins them in ascending range order.  The gradient keeps one fp32 number per row and head
 * (the row sums of dO * O), and cuts the heads that share a K and V into n_splits parts likewise.
 * Results differ between limits that give different n_splits by the rounding of those sums.
 */
typedef struct {
    int64_t n, m;
    int32_t hq, hkv, d;
    int32_t tile_rows;
    int32_t n_splits;
    int32_t reserved;
    uint64_t workspace_bytes; /* <= limit */
    uint64_t min_limit_bytes; /* smallest limit that can run this shape */
} attn_plan_t;

/*
 * HOST.  n >= 0 rows, m >= 0 keys, hq >= hkv >= 1 with hq % hkv == 0, 1 <= d.  KNN_OK,
 * KNN_ERR_INVALID_ARG, KNN_ERR_UNSUPPORTED (d > ATTN_MAX_D, n or m above 2^30, hq above 65535) or
 * KNN_ERR_MEM_LIMIT_TOO_SMALL (then *out still carries min_limit_bytes).
 */
knn_status attn_plan(int64_t n, int64_t m, int32_t hq, int32_t hkv, int32_t d, uint64_t mem_limit_bytes,
                     attn_plan_t *out /* HOST */);
knn_status attn_grad_plan(int64_t n, int64_t m, int32_t hq, int32_t hkv, int32_t d, uint64_t mem_limit_bytes,
                          attn_plan_t *out /* HOST */);

/*
 * attn_apply - O and lse.
 *   Q [n][hq][d], K, V [m][hkv][d]   DEVICE in
 *   options     HOST; what it points to is DEVICE
 *   workspace   DEVICE, 256-byte aligned, workspace_bytes >= plan.workspace_bytes (NULL where that is 0)
 *   O [n][hq][d]                     DEVICE out
 *   lse [hq][n]                      DEVICE out, fp32, contiguous (natural logarithm); NULL: not wanted
 *   hip_stream  hipStream_t (NULL: default stream); the call only enqueues work and allocates nothing.
 * Rows before the first document or behind the last are neither read nor written, keys there are not
 * read.  Scores, maxima, totals and sums are fp32; a tile's probabilities are rounded to the type of V
 * for their product with it, and O is rounded once.  Every sum has a fixed order.
 * An entry that is not finite (NaN in Q; infinite or NaN in K or V) reaches the rows that see it and
 * no others.  A row whose scores are all -infinity counts as one that sees no key.
 */
knn_status attn_apply(const attn_rows_t *Q, const attn_rows_t *K, const attn_rows_t *V, int64_t n, int64_t m,
                      int32_t hq, int32_t hkv, int32_t d, const attn_options_t *options, uint64_t mem_limit_bytes,
                      void *workspace, uint64_t workspace_bytes, const attn_rows_t *O, float *lse, void *hip_stream);

/*
 * attn_grad - the gradients of sum(dO * O) by Q, K and V:
 *     dV_j = sum_i P_ij dO_i,  ds_ij = P_ij (<dO_i, V_j> - <dO_i, O_i>),  du_ij = ds_ij (1 - tanh^2(u_ij / cap)),
 *     dQ_i = scale sum_j du_ij K_j,  dK_j = scale sum_i du_ij Q_i,
 * P made again from Q, K and lse.  Arguments as attn_apply, with
 *   O, lse      DEVICE in, as attn_apply left them (same Q, K, V and options)
 *   dO [n][hq][d]                            DEVICE in
 *   dQ [n][hq][d], dK, dV [m][hkv][d]        DEVICE out, in the type of Q, overwritten
 *   workspace_bytes >= attn_grad_plan(...).workspace_bytes
 * Rows and keys outside the documents are left as they were.  P and ds are rounded to the type of Q for
 * the products, whose sums are fp32 in a fixed order: no atomics, the same bits on every call.
 * An entry that is not finite makes the gradients not finite of the rows and keys that it meets, and no others.
 */
knn_status attn_grad(const attn_rows_t *Q, const attn_rows_t *K, const attn_rows_t *V, const attn_rows_t *O,
                     const float *lse, const attn_rows_t *dO, int64_t n, int64_t m, int32_t hq, int32_t hkv,
                     int32_t d, const attn_options_t *options, uint64_t mem_limit_bytes, void *workspace,
                     uint64_t workspace_bytes, const attn_rows_t *dQ, const attn_rows_t *dK, const attn_rows_t *dV,
                     void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* ATTN_MI355X_H */
