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
 * (elements).  ld, hs >= 0, of an output >= d where there are several rows (heads); an output's entries must not
 * overlap each other or an input.
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
    double scale;             /* 2^-60 .. 2^60 */
    double cap;               /* 0: none; else 2^-60 .. 2^60.  Scores are off by 2^-23 of a cap up to 64, beyond by steps of 2^-24 of themselves */
    const float *slopes;      /* DEVICE [hq], finite; NULL: none.  Not differentiated */
    int64_t docs;             /* >= 1 with starts; without starts there is one document */
    const int32_t *starts;    /* DEVICE [docs + 1], ascending, within 0 .. n; NULL: 0, n */
    const int32_t *k_starts;  /* DEVICE [docs + 1], ascending, within 0 .. m; NULL together with starts */
    const int32_t *prefix;    /* DEVICE [docs]; NULL: none.  Only looked at with causal */
} attn_options_t;

/*
 * The plan.  One workgroup owns tile_rows rows (of all heads that share a K and V, side by side) and walks
 * the keys; where that leaves compute units idle and the limit has room, the keys are cut into n_splits
 * ranges walked concurrently, whose unnormalised sums, maxima and totals (fp32) lie in the workspace until a
 * last kernel joins them in ascending range order.  The gradient keeps two fp32 numbers per row and head (the row
 * sums of dO * O, the log-sums), and for dK and dV cuts the rows of all heads that read them into n_splits parts likewise,
 * for dQ the keys into row_splits ranges.
 * Results differ between limits that give different n_splits by the rounding of those sums.
 */
typedef struct {
    int64_t n, m;
    int32_t hq, hkv, d;
    int32_t tile_rows;
    int32_t n_splits;
    int32_t row_splits; /* gradient: ranges of keys for dQ; 0 elsewhere */
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
 * Rows before the first document or behind the last are not written; what they and keys there hold has no
 * influence.  Scores, maxima, totals and sums are fp32; a tile's probabilities are rounded to the type of V
 * for their product with it, and O is rounded once.  Every sum has a fixed order.
 * An entry that is not finite (NaN in Q; infinite or NaN in K or V) reaches the rows that see it, one of V however
 * small its weight, and no others.  A row whose scores are all -infinity counts as one that sees no key.
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
 * the products (in f16, where they lie below what it holds for many keys or a small dO, P times 2^14 and ds times a power of two for
 * every row and key), whose sums are fp32 in a fixed order: no atomics, the same bits on every call.
 * Entries that are not finite.  One in a row's Q or dO (or O) makes its dQ, and dK and dV of the keys that it sees, not finite, one in K
 * the dQ of the rows that see it, and so on by the formulas where a score is NaN or +infinity (the row's log-sum is NaN); no others.
 * A row that sees no key, or whose scores are all -infinity, has dQ = 0 and adds nothing to the others.
 * How exact: P is made from lse, which holds a score to 2^-24 of itself; <dO, O> takes the O that attn_apply rounded, so
 * where one key has nearly all of a row's weight its ds, a small difference, is off by that rounding.
 */
knn_status attn_grad(const attn_rows_t *Q, const attn_rows_t *K, const attn_rows_t *V, const attn_rows_t *O,
                     const float *lse, const attn_rows_t *dO, int64_t n, int64_t m, int32_t hq, int32_t hkv,
                     int32_t d, const attn_options_t *options, uint64_t mem_limit_bytes, void *workspace,
                     uint64_t workspace_bytes, const attn_rows_t *dQ, const attn_rows_t *dK, const attn_rows_t *dV,
                     void *hip_stream);

/* ---- a cache of keys and values in 8 bits ------------------------------------------------------
 *
 * What answers one row at a time keeps the K and V of the rows before it.  Here they lie as 8-bit codes
 * in blocks of `block` rows ("tokens"), in any order; a table gives each request its blocks, and every
 * block has a scale for each head: a value is code * scale.  With rows of 64 or 128 entries half the bytes of 16-bit rows, and
 * less than a hundredth on top for the scales: with a limit on device memory, twice the history.  (Rows are kept
 * 64 or 128 wide, so others gain less: one of 96 takes two thirds of its 16-bit bytes, one below 32 more than those.)
 *
 *   k  [blocks][hkv][block][row]   codes, a token's entries together
 *   v  [blocks][hkv][row][block]   codes, an entry's tokens together: the product with V sums over tokens
 *   k_scale, v_scale  [blocks][hkv]  fp32, >= 0
 * all DEVICE and contiguous, k and v 16-byte aligned.  row = attn_cache_row(d) entries, those behind d
 * zero.  The slot of token t of block b is b * block + t.
 */
typedef enum { ATTN_INT8 = 0, ATTN_E4M3 = 1 } attn_code; /* -127 .. 127; OCP e4m3, up to 448 */

typedef struct {
    void *k, *v;
    float *k_scale, *v_scale;
    int64_t blocks;
    int32_t hkv, d;
    int32_t block; /* 16, 32, 64, 128 or 256 */
    int32_t code;  /* attn_code */
} attn_cache_t;

/* HOST.  Entries of a row in the cache: 64 or 128; 0 where d < 1 or d > ATTN_MAX_D. */
int32_t attn_cache_row(int32_t d);

/*
 * attn_cache_map - a step's block tables and slots, from the requests' lengths.
 *   lengths [batch], news [batch]   DEVICE in, int32: tokens of each request after the step, and how many
 *               of them are new (0 <= news <= lengths)
 *   table [batch][width]   DEVICE in/out, int32: entries 0 .. ceil(before / block) - 1 of a request, before =
 *               lengths - news, are its blocks already; those up to ceil(lengths / block) - 1 are written, with
 *               the next entries of `free` for the requests in order.  The others are left as they were.
 *   free [n_free]          DEVICE in, int32: blocks that no request has.  Where they run out -1 is written.
 *   starts [batch + 1]     DEVICE out, int32: the new tokens of request i are rows starts[i] .. starts[i + 1] - 1
 *   slots [n_slots]        DEVICE out, int64: where each goes; -1 where it has no block, and behind the last
 *   used [1]               DEVICE out, int32: how many entries of `free` the step needs (more than n_free: too few)
 * Lengths beyond width * block, and negative ones, are taken as the nearest that fits; news likewise.  Calling
 * again with the same inputs writes the same.  batch <= 16384.  Errors: KNN_ERR_INVALID_ARG, KNN_ERR_UNSUPPORTED
 * (batch, or width * block above 2^30), KNN_ERR_HIP.  (Sums of lengths beyond 2^31 - 1 are taken as that.)
 */
knn_status attn_cache_map(const int32_t *lengths, const int32_t *news, int64_t batch, int32_t *table, int64_t width,
                          int32_t block, const int32_t *free, int64_t n_free, int32_t *starts, int64_t *slots,
                          int64_t n_slots, int32_t *used, void *hip_stream);

/*
 * attn_cache_append - rows K [count][hkv][d], V [count][hkv][d] (DEVICE, of `dtype`) into the cache at
 * slots [count] (DEVICE, int64).  Slots outside the cache (-1) are passed over.
 * For each block and head with new tokens, K and V apart: a block that gets its token 0 is begun anew, all its
 * codes zero and its scale 0.  scale' = max(scale, fl(a / most)), a the largest magnitude of the new rows,
 * most = 127 or 448, fl to fp32.  If scale' > scale the codes there become the nearest to code * scale / scale'.
 * A new code is the nearest to x / scale' (of two as near the even one; quotients of real numbers).
 * NaN becomes 0 and an infinity the largest code; neither counts for a.  (Of a scale of 0 every code is 0.)
 * The slots of one block must stand together in `slots`, in any order, with any that are passed over among them; of a slot given
 * twice the last counts.  Where one block's slots stand apart, with another block's between them, what becomes of that
 * block is not defined.  At most 2^27 rows times heads, and 65535 heads.
 */
knn_status attn_cache_append(const attn_cache_t *cache, int32_t dtype, const attn_rows_t *K, const attn_rows_t *V,
                             int64_t count, const int64_t *slots, void *hip_stream);

/*
 * The plan of attn_cache_apply: the tokens of a request are cut into ranges of range_tokens that
 * workgroups walk concurrently; with more than one range in width * block tokens their sums (fp32) lie
 * in the workspace until a last kernel joins them in ascending order.
 */
typedef struct {
    int64_t batch, longest; /* longest: width * block */
    int32_t nq, hq, hkv, d;
    int32_t range_tokens;
    int32_t n_ranges;
    uint64_t workspace_bytes; /* <= limit */
    uint64_t min_limit_bytes; /* 0 */
} attn_cache_plan_t;

/* HOST.  batch, longest >= 0, nq >= 1, heads and d as attn_plan. */
knn_status attn_cache_plan(int64_t batch, int32_t nq, int32_t hq, int32_t hkv, int32_t d, int64_t longest,
                           uint64_t mem_limit_bytes, attn_cache_plan_t *out /* HOST */);

/*
 * attn_cache_apply - attention of the last nq rows of each request over the cache.
 *   Q, O [batch * nq][hq][d]   DEVICE in / out, of `dtype`: row i * nq + t is the t-th of request i's last nq,
 *                  at p = lengths[i] - nq + t; it sees the tokens j <= p (none where p < 0: O = 0)
 *   table [batch][width], lengths [batch]   DEVICE in, int32.  Tokens whose table entry is no block of the cache
 *                  are not seen; a length is at most width * block.
 *   scale, cap, slopes   as in attn_options_t
 * Scores, maxima, totals and sums are fp32 (values times their number of tokens below 2^127).  A code is exact in 16 bits;
 * probabilities are rounded to f16, times the ratio of their block's scale to the largest of 64 tokens' scales, times 2^14.
 */
knn_status attn_cache_apply(const attn_cache_t *cache, int32_t dtype, const attn_rows_t *Q, int64_t batch, int32_t nq,
                            int32_t hq, const int32_t *table, int64_t width, const int32_t *lengths, double scale,
                            double cap, const float *slopes, uint64_t mem_limit_bytes, void *workspace,
                            uint64_t workspace_bytes, const attn_rows_t *O, void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* ATTN_MI355X_H */
