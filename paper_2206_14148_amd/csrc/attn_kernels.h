// Internal launcher interface between the attention C ABI (attn_api.hip) and its gfx950 kernels.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace attn {

constexpr int kTileRows = 128;  // rows of Q (forward, dQ) or keys (dK, dV) per workgroup: 4 waves x 32
constexpr int kTileKeys = 64;   // keys, or rows, per step of the walk
constexpr int kStepRows = 32;    // rows per step of the gradient by keys
constexpr int kMaxSplits = 256;

struct Rows {  // one tensor [rows][heads][d], see attn_rows_t
    unsigned short* data;
    int64_t ld, hs;
    int wide;  // 16 bytes at a time
};

struct Mask {
    const int *starts, *k_starts, *prefix;
    int docs, causal, n, m;
};

struct Problem {
    Rows q, k, v, o, dO, dq, dk, dv;
    Mask mask;
    int hq, hkv, d, f16;
    float scale, cap;
    const float* slopes;
    float* lse;      // [hq][n] or null
    float* rowsums;  // gradient: [2][hq][n], what a row takes off its products: -log-sum / scale, -sum of dO * O
    float* partial;  // n_splits > 1
    int splits;
    int row_splits;      // gradient: parts of dQ,
    float* row_partial;  // row_splits > 1: [row_splits][hq][n][d]
};

hipError_t launch_forward(const Problem& p, hipStream_t stream);
hipError_t launch_grad(const Problem& p, hipStream_t stream);

// ---- the cache (attn_cache.hip) ---------------------------------------------------------------

struct Cache {
    unsigned char *k, *v;
    float *k_scale, *v_scale;
    int64_t blocks;
    int hkv, d, row, block, e4m3;
};

constexpr int kMostBatch = 16384;  // of a map: their new blocks and tokens are summed up in LDS

struct MapProblem {
    const int *lengths, *news, *free;
    int *table, *starts, *used;
    int64_t* slots;
    int64_t n_slots, n_free;
    int batch, width, block;
};
hipError_t launch_map(const MapProblem& p, hipStream_t stream);

struct AppendProblem {
    Cache cache;
    Rows k, v;
    const int64_t* slots;
    int64_t count;
    int f16;
};
hipError_t launch_append(const AppendProblem& p, hipStream_t stream);

struct CacheProblem {
    Cache cache;
    Rows q, o;
    const int *table, *lengths;
    const float* slopes;
    float* partial;
    int batch, nq, hq, width, f16, ranges, range_tokens;
    float scale, cap;
};
hipError_t launch_cache(const CacheProblem& p, hipStream_t stream);

}  // namespace attn
