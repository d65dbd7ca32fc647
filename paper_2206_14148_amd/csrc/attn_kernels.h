// Internal launcher interface between the attention C ABI (attn_api.hip) and its gfx950 kernels.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace attn {

constexpr int kTileRows = 128;  // rows of Q (forward, dQ) or keys (dK, dV) per workgroup: 4 waves x 32
constexpr int kTileKeys = 64;   // keys, or rows, per step of the walk
constexpr int kMaxSplits = 64;

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
    float* rowsums;  // gradient: [hq][n]
    float* partial;  // n_splits > 1
    int splits;
};

hipError_t launch_forward(const Problem& p, hipStream_t stream);
hipError_t launch_grad(const Problem& p, hipStream_t stream);

}  // namespace attn
