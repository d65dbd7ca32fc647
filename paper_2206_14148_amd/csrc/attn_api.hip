// C ABI of the attention product, its gradient and its cache (see include/attn.h for the contract).
#include <hip/hip_runtime.h>

#include <cstring>

#include "../../include/attn.h"
#include "attn_kernels.h"
#include "knn_config.h"

namespace knn {  // api.hip
void set_last_hip_error(hipError_t e, const char* what);
hipEvent_t profile_mark(hipStream_t stream);
void profile_close(hipEvent_t begin, hipStream_t stream, int kind);
void profile_drop(hipEvent_t begin);
}  // namespace knn

namespace {

constexpr int64_t kMostRows = (int64_t)1 << 30;

// Into how many parts a walk is cut.  What a part costs, measured for bf16 rows of 80 and 128, one to 50021 of them: a step (64
// keys, or 32 rows by keys) takes 1.15 us where a compute unit has one workgroup and 1.7 times that where two share it; parts have
// to be written and read at 4 TB/s, and their join is a launch of 5 us.  A workgroup's walk ends no earlier than its
// own steps, all workgroups' no earlier than 2 to a compute unit allow; `share` is the part of the steps that the mean
// workgroup has (by keys half, as with a causal mask, where the first keys' workgroups have all).
// 3 rows of 16 heads against 50021 keys: 854 us in one part, 25 in 128; 1201 rows of 8 heads: 27 in one, 22 in 4, 27 in 8;
// the gradient of 4096 rows of 32 heads: 1000 in one, 575 in 4.
int best_parts(int64_t workgroups, int64_t steps, double share, double bytes_a_part, uint64_t room, uint64_t (*bytes)(const int64_t*, int64_t),
               const int64_t* shape) {
    int best = 1;
    double least = 0;
    for (int64_t s = 1; s <= attn::kMaxSplits && (s == 1 || (steps >= 2 * s && bytes(shape, s) <= room)); s *= 2) {
        const double each = (double)((steps + s - 1) / s) * 1.15, all = (double)workgroups * s;
        const double own = each * (all > knn::kNumCU ? 1.7 : 1.0), total = all * each * share * 1.7 / (2 * knn::kNumCU);
        const double t = (own > total ? own : total) + (s > 1 ? 5.0 + s * bytes_a_part / 4e6 : 0.0);
        if (s == 1 || t < 0.95 * least) {
            best = (int)s;
            least = t;
        }
    }
    return best;
}

uint64_t row_parts(const int64_t* rows_d, int64_t parts) {  // rows times heads, d
    return parts > 1 ? knn::align_up((uint64_t)parts * rows_d[0] * (rows_d[1] + 2) * 4) : 0;
}
uint64_t grad_row_parts(const int64_t* rows_d, int64_t parts) {  // rows times heads, d: dQ
    return parts > 1 ? knn::align_up((uint64_t)parts * rows_d[0] * rows_d[1] * 4) : 0;
}
uint64_t key_parts(const int64_t* keys_d, int64_t parts) {  // keys times heads, d: dK and dV
    return parts > 1 ? knn::align_up((uint64_t)parts * 2 * keys_d[0] * keys_d[1] * 4) : 0;
}

knn_status check_shape(int64_t n, int64_t m, int32_t hq, int32_t hkv, int32_t d, attn_plan_t* out) {
    if (!out) return KNN_ERR_INVALID_ARG;
    std::memset(out, 0, sizeof(*out));
    if (n < 0 || m < 0 || hkv < 1 || hq < hkv || hq % hkv != 0 || d < 1) return KNN_ERR_INVALID_ARG;
    if (d > ATTN_MAX_D || n > kMostRows || m > kMostRows || hq > 65535) return KNN_ERR_UNSUPPORTED;
    // rows times heads in 32 bits, and work items of a launch: one workgroup of 256 for each tile and head (parts only where there are few)
    if ((n / attn::kTileRows + 1) * hq >= (1 << 24) || (m / attn::kTileRows + 1) * hq >= (1 << 24)) return KNN_ERR_UNSUPPORTED;
    out->n = n;
    out->m = m;
    out->hq = hq;
    out->hkv = hkv;
    out->d = d;
    out->tile_rows = attn::kTileRows;
    out->n_splits = 1;
    return KNN_OK;
}

knn_status hip_fail(hipError_t e, const char* what) {
    knn::set_last_hip_error(e, what);
    return KNN_ERR_HIP;
}

bool usable(const attn_rows_t* t, int64_t rows) {
    if (!t || t->ld < 0 || t->hs < 0) return false;
    return rows == 0 || t->data;
}

// An output: no two of its entries may be one.  Rows or heads closer than d would be, wherever there are two ...
bool writable(const attn_rows_t* t, int64_t rows, int32_t heads, int32_t d) {
    return usable(t, rows) && (rows <= 1 || t->ld >= d) && (heads == 1 || t->hs >= d);
}

// ... and so would row i of one head and row 0 of the h-th behind it that are closer than d: workgroups would race for them.
bool apart(const attn_rows_t* t, int64_t rows, int32_t heads, int32_t d) {
    if (rows <= 1 || heads <= 1) return true;
    const __int128 ld = t->ld, hs = t->hs;
    if (ld >= (heads - 1) * hs + d || hs >= (rows - 1) * ld + d) return true;
    for (int32_t h = 1; h < heads; ++h)
        for (__int128 i = h * hs / ld; i <= h * hs / ld + 1; ++i) {
            const __int128 off = i * ld - h * hs;
            if (i >= 1 && i < rows && off < d && off > -d) return false;
        }
    return true;
}

// 0 (a cap: none) or a number that 32 bits, its inverse and its quotients with another one hold with room to spare
bool ordinary(double x) { return x >= 0x1p-60 && x <= 0x1p60; }

attn::Rows rows_of(const attn_rows_t* t, int32_t d) {
    attn::Rows r;
    r.data = static_cast<unsigned short*>(t->data);
    r.ld = t->ld;
    r.hs = t->hs;
    r.wide = reinterpret_cast<uintptr_t>(t->data) % 16 == 0 && d % 8 == 0 && t->ld % 8 == 0 && t->hs % 8 == 0 &&
             t->ld < (1 << 22);  // 64 rows are 2^29 bytes at most: offsets in 32 bits
    return r;
}

knn_status fill_problem(const attn_options_t* o, int64_t n, int64_t m, int32_t hq, int32_t hkv, int32_t d, attn::Problem* p) {
    if (!o || (o->dtype != ATTN_BF16 && o->dtype != ATTN_F16) || (o->causal != 0 && o->causal != 1)) return KNN_ERR_INVALID_ARG;
    if (!ordinary(o->scale) || (o->cap != 0.0 && !ordinary(o->cap))) return KNN_ERR_INVALID_ARG;
    if ((o->starts == nullptr) != (o->k_starts == nullptr)) return KNN_ERR_INVALID_ARG;
    if (o->starts ? o->docs < 1 || o->docs >= ((int64_t)1 << 31) - 1 : o->docs != 0 && o->docs != 1) return KNN_ERR_INVALID_ARG;
    std::memset(p, 0, sizeof(*p));
    p->mask.starts = o->starts;
    p->mask.k_starts = o->k_starts;
    p->mask.prefix = o->causal ? o->prefix : nullptr;
    p->mask.docs = o->starts ? (int)o->docs : 1;
    p->mask.causal = o->causal;
    p->mask.n = (int)n;
    p->mask.m = (int)m;
    p->hq = hq;
    p->hkv = hkv;
    p->d = d;
    p->f16 = o->dtype == ATTN_F16;
    p->scale = (float)o->scale;
    p->cap = (float)o->cap;
    p->slopes = o->slopes;
    return KNN_OK;
}

knn_status check_workspace(const attn_plan_t& plan, const void* workspace, uint64_t workspace_bytes) {
    if (plan.workspace_bytes == 0) return KNN_OK;
    if (!workspace || reinterpret_cast<uintptr_t>(workspace) % knn::kAlign != 0) return KNN_ERR_INVALID_ARG;
    return workspace_bytes < plan.workspace_bytes ? KNN_ERR_WORKSPACE_TOO_SMALL : KNN_OK;
}

}  // namespace

extern "C" knn_status attn_plan(int64_t n, int64_t m, int32_t hq, int32_t hkv, int32_t d, uint64_t mem_limit_bytes,
                                attn_plan_t* out) {
    const knn_status st = check_shape(n, m, hq, hkv, d, out);
    if (st != KNN_OK) return st;
    const int64_t tiles = (n * (hq / hkv) + attn::kTileRows - 1) / attn::kTileRows * hkv;
    const int64_t shape[2] = {n * hq, d};
    out->n_splits = n == 0 ? 1 : best_parts(tiles, (m + attn::kTileKeys - 1) / attn::kTileKeys, 1.0, 8.0 * n * hq * (d + 2), mem_limit_bytes,
                                            row_parts, shape);
    out->workspace_bytes = row_parts(shape, out->n_splits);
    return KNN_OK;
}

extern "C" knn_status attn_grad_plan(int64_t n, int64_t m, int32_t hq, int32_t hkv, int32_t d, uint64_t mem_limit_bytes,
                                     attn_plan_t* out) {
    const knn_status st = check_shape(n, m, hq, hkv, d, out);
    if (st != KNN_OK) return st;
    const uint64_t sums = knn::align_up((uint64_t)n * hq * 8);
    out->min_limit_bytes = sums;
    if (mem_limit_bytes < sums) return KNN_ERR_MEM_LIMIT_TOO_SMALL;
    const int64_t tiles = (m + attn::kTileRows - 1) / attn::kTileRows * hkv;
    const int64_t steps = (n + attn::kStepRows - 1) / attn::kStepRows * (hq / hkv);
    const int64_t shape[2] = {m * hkv, d};
    out->n_splits = m == 0 ? 1 : best_parts(tiles, steps, 0.5, 16.0 * m * hkv * d, mem_limit_bytes - sums, key_parts, shape);
    const uint64_t of_keys = key_parts(shape, out->n_splits);
    // dQ likewise, with the room that those leave (the gradient of 3 rows of 16 heads against 50021
    // keys: 1354 us without, 107 with 128 parts; 1000 rows against 4000 keys, 8 heads: 181 and 116)
    const int64_t row_tiles = (n * (hq / hkv) + attn::kTileRows - 1) / attn::kTileRows * hkv;
    const int64_t row_shape[2] = {n * hq, d};
    out->row_splits = n == 0 ? 1 : best_parts(row_tiles, (m + attn::kTileKeys - 1) / attn::kTileKeys, 1.0, 8.0 * n * hq * d,
                                              mem_limit_bytes - sums - of_keys, grad_row_parts, row_shape);
    out->workspace_bytes = sums + of_keys + grad_row_parts(row_shape, out->row_splits);
    return KNN_OK;
}

extern "C" knn_status attn_apply(const attn_rows_t* Q, const attn_rows_t* K, const attn_rows_t* V, int64_t n, int64_t m,
                                 int32_t hq, int32_t hkv, int32_t d, const attn_options_t* options,
                                 uint64_t mem_limit_bytes, void* workspace, uint64_t workspace_bytes,
                                 const attn_rows_t* O, float* lse, void* hip_stream) {
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    attn_plan_t plan;
    knn_status st = attn_plan(n, m, hq, hkv, d, mem_limit_bytes, &plan);
    if (st != KNN_OK) return st;
    attn::Problem p;
    st = fill_problem(options, n, m, hq, hkv, d, &p);
    if (st != KNN_OK) return st;
    if (!usable(Q, n) || !usable(K, m) || !usable(V, m) || !writable(O, n, hq, d)) return KNN_ERR_INVALID_ARG;
    if (n == 0) return KNN_OK;
    st = check_workspace(plan, workspace, workspace_bytes);
    if (st != KNN_OK) return st;
    if (!apart(O, n, hq, d)) return KNN_ERR_INVALID_ARG;
    p.q = rows_of(Q, d);
    p.k = rows_of(K, d);
    p.v = rows_of(V, d);
    p.o = rows_of(O, d);
    p.lse = lse;
    p.splits = plan.n_splits;
    p.partial = static_cast<float*>(workspace);
    hipEvent_t t = knn::profile_mark(stream);
    const hipError_t e = attn::launch_forward(p, stream);
    if (e != hipSuccess) {
        knn::profile_drop(t);
        return hip_fail(e, "attention kernel");
    }
    knn::profile_close(t, stream, 1);
    return KNN_OK;
}

extern "C" knn_status attn_grad(const attn_rows_t* Q, const attn_rows_t* K, const attn_rows_t* V, const attn_rows_t* O,
                                const float* lse, const attn_rows_t* dO, int64_t n, int64_t m, int32_t hq,
                                int32_t hkv, int32_t d, const attn_options_t* options, uint64_t mem_limit_bytes,
                                void* workspace, uint64_t workspace_bytes, const attn_rows_t* dQ,
                                const attn_rows_t* dK, const attn_rows_t* dV, void* hip_stream) {
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    attn_plan_t plan;
    knn_status st = attn_grad_plan(n, m, hq, hkv, d, mem_limit_bytes, &plan);
    if (st != KNN_OK) return st;
    attn::Problem p;
    st = fill_problem(options, n, m, hq, hkv, d, &p);
    if (st != KNN_OK) return st;
    if (!usable(Q, n) || !usable(K, m) || !usable(V, m) || !usable(O, n) || !usable(dO, n) ||
        !writable(dQ, n, hq, d) || !writable(dK, m, hkv, d) || !writable(dV, m, hkv, d) || (n > 0 && !lse))
        return KNN_ERR_INVALID_ARG;
    if (n == 0 && m == 0) return KNN_OK;
    st = check_workspace(plan, workspace, workspace_bytes);
    if (st != KNN_OK) return st;
    if (!apart(dQ, n, hq, d) || !apart(dK, m, hkv, d) || !apart(dV, m, hkv, d)) return KNN_ERR_INVALID_ARG;
    p.q = rows_of(Q, d);
    p.k = rows_of(K, d);
    p.v = rows_of(V, d);
    p.o = rows_of(O, d);
    p.dO = rows_of(dO, d);
    p.dq = rows_of(dQ, d);
    p.dk = rows_of(dK, d);
    p.dv = rows_of(dV, d);
    p.lse = const_cast<float*>(lse);
    p.splits = plan.n_splits;
    p.row_splits = plan.row_splits;
    p.rowsums = static_cast<float*>(workspace);
    p.partial = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + knn::align_up((uint64_t)n * hq * 8));
    const int64_t keys_d[2] = {m * hkv, d};
    p.row_partial = p.partial + key_parts(keys_d, p.splits) / 4;
    hipEvent_t t = knn::profile_mark(stream);
    const hipError_t e = attn::launch_grad(p, stream);
    if (e != hipSuccess) {
        knn::profile_drop(t);
        return hip_fail(e, "attention gradient kernels");
    }
    knn::profile_close(t, stream, 1);
    return KNN_OK;
}

// ---- the cache --------------------------------------------------------------------------------

namespace {

bool cache_of(const attn_cache_t* c, attn::Cache* out) {
    if (!c || c->hkv < 1 || c->blocks < 0 || c->blocks > kMostRows || attn_cache_row(c->d) == 0) return false;
    if (c->block < 16 || c->block > 256 || (c->block & (c->block - 1)) != 0) return false;
    if (c->code != ATTN_INT8 && c->code != ATTN_E4M3) return false;
    if (c->blocks > 0 && (!c->k || !c->v || !c->k_scale || !c->v_scale)) return false;
    if (reinterpret_cast<uintptr_t>(c->k) % 16 != 0 || reinterpret_cast<uintptr_t>(c->v) % 16 != 0) return false;
    out->k = static_cast<unsigned char*>(c->k);
    out->v = static_cast<unsigned char*>(c->v);
    out->k_scale = c->k_scale;
    out->v_scale = c->v_scale;
    out->blocks = c->blocks;
    out->hkv = c->hkv;
    out->d = c->d;
    out->row = attn_cache_row(c->d);
    out->block = c->block;
    out->e4m3 = c->code == ATTN_E4M3;
    return true;
}

// Tokens that one workgroup walks: so many ranges that the longest request alone, and the batch at about half
// of its length, occupy the GPU.  Below 512 tokens a range the join, a launch of its own, costs more than the walk.
constexpr int64_t kWantCache = 8 * knn::kNumCU;
constexpr int64_t kLeastTokens = 512;
constexpr int64_t kMostRanges = 64;
constexpr int64_t kStepTokens = 256;  // that its four waves take at once

}  // namespace

extern "C" int32_t attn_cache_row(int32_t d) { return d < 1 || d > ATTN_MAX_D ? 0 : d <= 64 ? 64 : 128; }

extern "C" knn_status attn_cache_map(const int32_t* lengths, const int32_t* news, int64_t batch, int32_t* table,
                                     int64_t width, int32_t block, const int32_t* free, int64_t n_free,
                                     int32_t* starts, int64_t* slots, int64_t n_slots, int32_t* used, void* hip_stream) {
    if (batch < 0 || width < 0 || n_free < 0 || n_slots < 0 || block < 16 || block > 256 || (block & (block - 1)) != 0)
        return KNN_ERR_INVALID_ARG;
    if (batch > attn::kMostBatch || width > kMostRows / block) return KNN_ERR_UNSUPPORTED;
    if (!starts || !used || (batch > 0 && (!lengths || !news)) || (batch > 0 && width > 0 && !table) ||
        (n_free > 0 && !free) || (n_slots > 0 && !slots))
        return KNN_ERR_INVALID_ARG;
    attn::MapProblem p;
    p.lengths = lengths;
    p.news = news;
    p.free = free;
    p.table = table;
    p.starts = starts;
    p.used = used;
    p.slots = slots;
    p.n_slots = n_slots;
    p.n_free = n_free;
    p.batch = (int)batch;
    p.width = (int)width;
    p.block = block;
    const hipError_t e = attn::launch_map(p, static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? KNN_OK : hip_fail(e, "attention cache map kernel");
}

extern "C" knn_status attn_cache_append(const attn_cache_t* cache, int32_t dtype, const attn_rows_t* K, const attn_rows_t* V,
                                        int64_t count, const int64_t* slots, void* hip_stream) {
    attn::AppendProblem p;
    if (!cache_of(cache, &p.cache) || (dtype != ATTN_BF16 && dtype != ATTN_F16) || count < 0) return KNN_ERR_INVALID_ARG;
    if (!usable(K, count) || !usable(V, count) || (count > 0 && !slots)) return KNN_ERR_INVALID_ARG;
    if (count > kMostRows || cache->hkv > 65535 || count * cache->hkv > ((int64_t)1 << 27)) return KNN_ERR_UNSUPPORTED;
    if (count == 0 || cache->blocks == 0) return KNN_OK;
    p.k = rows_of(K, cache->d);
    p.v = rows_of(V, cache->d);
    p.slots = slots;
    p.count = count;
    p.f16 = dtype == ATTN_F16;
    const hipError_t e = attn::launch_append(p, static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? KNN_OK : hip_fail(e, "attention cache append kernel");
}

extern "C" knn_status attn_cache_plan(int64_t batch, int32_t nq, int32_t hq, int32_t hkv, int32_t d, int64_t longest,
                                      uint64_t mem_limit_bytes, attn_cache_plan_t* out) {
    if (!out) return KNN_ERR_INVALID_ARG;
    std::memset(out, 0, sizeof(*out));
    if (batch < 0 || longest < 0 || nq < 1 || hkv < 1 || hq < hkv || hq % hkv != 0 || d < 1) return KNN_ERR_INVALID_ARG;
    if (d > ATTN_MAX_D || longest > kMostRows || batch > kMostRows || hq > 65535 || nq > 65535) return KNN_ERR_UNSUPPORTED;
    const int64_t rows = (int64_t)nq * (hq / hkv), per = rows > 16 ? 32 : 16;
    if ((double)batch * hkv * ((rows + per - 1) / per) >= (1 << 24)) return KNN_ERR_UNSUPPORTED;
    const int64_t sets = batch * hkv * ((rows + per - 1) / per);
    auto bytes = [&](int64_t ranges) {
        return ranges > 1 ? knn::align_up((uint64_t)ranges * batch * nq * hq * (d + 2) * 4) : 0;
    };
    int64_t ranges = 1;
    while (sets > 0 && sets * ranges < kWantCache && ranges < kMostRanges && longest / (2 * ranges) >= kLeastTokens &&
           bytes(2 * ranges) <= mem_limit_bytes)
        ranges *= 2;
    const int64_t tokens = ((longest + ranges - 1) / ranges + kStepTokens - 1) / kStepTokens * kStepTokens;
    out->batch = batch;
    out->longest = longest;
    out->nq = nq;
    out->hq = hq;
    out->hkv = hkv;
    out->d = d;
    out->range_tokens = (int32_t)(tokens ? tokens : kStepTokens);
    out->n_ranges = tokens ? (int32_t)((longest + tokens - 1) / tokens) : 1;
    out->workspace_bytes = bytes(out->n_ranges);
    return KNN_OK;
}

extern "C" knn_status attn_cache_apply(const attn_cache_t* cache, int32_t dtype, const attn_rows_t* Q, int64_t batch,
                                       int32_t nq, int32_t hq, const int32_t* table, int64_t width,
                                       const int32_t* lengths, double scale, double cap, const float* slopes,
                                       uint64_t mem_limit_bytes, void* workspace, uint64_t workspace_bytes,
                                       const attn_rows_t* O, void* hip_stream) {
    attn::CacheProblem p;
    if (!cache_of(cache, &p.cache) || (dtype != ATTN_BF16 && dtype != ATTN_F16) || width < 0) return KNN_ERR_INVALID_ARG;
    if (!ordinary(scale) || (cap != 0.0 && !ordinary(cap))) return KNN_ERR_INVALID_ARG;
    if (width > kMostRows / cache->block) return KNN_ERR_UNSUPPORTED;
    attn_cache_plan_t plan;
    const knn_status st = attn_cache_plan(batch, nq, hq, cache->hkv, cache->d, width * cache->block, mem_limit_bytes, &plan);
    if (st != KNN_OK) return st;
    if (!usable(Q, batch) || !writable(O, batch * nq, hq, cache->d) || (batch > 0 && !lengths) || (batch > 0 && width > 0 && !table))
        return KNN_ERR_INVALID_ARG;
    if (batch == 0) return KNN_OK;
    if (plan.workspace_bytes > 0) {
        if (!workspace || reinterpret_cast<uintptr_t>(workspace) % knn::kAlign != 0) return KNN_ERR_INVALID_ARG;
        if (workspace_bytes < plan.workspace_bytes) return KNN_ERR_WORKSPACE_TOO_SMALL;
    }
    if (!apart(O, batch * nq, hq, cache->d)) return KNN_ERR_INVALID_ARG;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    p.q = rows_of(Q, cache->d);
    p.o = rows_of(O, cache->d);
    p.table = table;
    p.lengths = lengths;
    p.slopes = slopes;
    p.partial = static_cast<float*>(workspace);
    p.batch = (int)batch;
    p.nq = nq;
    p.hq = hq;
    p.width = (int)width;
    p.f16 = dtype == ATTN_F16;
    p.ranges = plan.n_ranges;
    p.range_tokens = plan.range_tokens;
    p.scale = (float)scale;
    p.cap = (float)cap;
    hipEvent_t t = knn::profile_mark(stream);
    const hipError_t e = attn::launch_cache(p, stream);
    if (e != hipSuccess) {
        knn::profile_drop(t);
        return hip_fail(e, "attention cache kernel");
    }
    knn::profile_close(t, stream, 1);
    return KNN_OK;
}
