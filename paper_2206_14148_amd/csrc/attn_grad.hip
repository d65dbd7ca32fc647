// The gradient of O = softmax(scores) V.  P is made again from Q, K and the rows' log-sums, tile by tile, in two
// walks: by rows for dQ (which also makes the row sums of dO * O), by keys for dK and dV.  Two walks cost two of
// seven products more than one walk would, and in return every sum has its place and its order: with one, dQ
// would have to be added to memory by whichever workgroup comes first.
#include "attn_device.h"

namespace attn {

namespace {

// Scores of a tile to P (given the rows' or the row's log-sum, in powers of two) and, where they are capped, to
// the slope of the cap.
struct Scores {
    float factor, to_cap, from_cap, slope;
    bool capped, general;
    __device__ __forceinline__ Scores(const Problem& p, int head) {
        capped = p.cap > 0.f;
        general = capped || p.slopes;
        slope = p.slopes ? p.slopes[head] * kLog2e : 0.f;
        factor = p.scale * kLog2e;
        to_cap = capped ? 2.f * kLog2e * p.scale / p.cap : 0.f;
        from_cap = p.cap * kLog2e;
    }
    // u -> score in powers of two; `steep`: 1 - tanh^2
    __device__ __forceinline__ float score(float u, float away, float& steep) const {
        float s = u * factor;
        if (capped) {
            const float t = __builtin_fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(to_cap * u)), 1.f);
            s = from_cap * t;
            steep = __builtin_fmaf(-t, t, 1.f);
        }
        return __builtin_fmaf(-slope, fabsf(away), s);
    }
};

__device__ __forceinline__ float in_twos(float lse) { return lse == -kInf ? kInf : lse * kLog2e; }  // no keys: P = 0

template <typename T, int DP>
__global__ __launch_bounds__(256, DP == 96 ? 1 : 2) void attn_grad_rows_kernel(Problem p) {
    typedef Tile<DP> L;
    constexpr int kBlocks = DP / 32, kSteps = DP / 16;
    __shared__ __attribute__((aligned(16))) unsigned char lds[4 * L::kBytes];
    __shared__ int ends[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    const int tiles = (p.mask.n + kTileRows - 1) / kTileRows;
    const int w = work_of(blockIdx.x, gridDim.x);
    const int tile = tiles - 1 - w % tiles, head = w / tiles, kv = head / (p.hq / p.hkv);
    const int row = tile * kTileRows + wave * 32 + (lane & 31);
    const Span see = keys_of_row(p.mask, row);
    const bool some = see.lo < see.hi;
    const int low = wave_least(some ? see.lo : INT_MAX), high = wave_most(some ? see.hi : INT_MIN);
    const int all_low = wave_most(see.inside ? see.lo : INT_MIN), all_high = wave_least(see.inside ? see.hi : INT_MAX);
    if (tid < 2) ends[tid] = tid ? INT_MIN : INT_MAX;
    __syncthreads();
    if (lane == 0) {
        atomicMin(&ends[0], low);
        atomicMax(&ends[1], high);
    }
    __syncthreads();
    int first = ends[0], last = ends[1];
    if (first >= last) first = last = 0;

    const int64_t at = (int64_t)head * p.mask.n + row;
    s16x8 q[kSteps], g[kSteps];
    float rowsum = 0.f;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        u32x4 a = {0, 0, 0, 0}, b = a, c = a;
        const int column = 16 * s + 8 * half;
        if (see.inside) {
            a = entries8(p.q.data + row * p.q.ld + head * p.q.hs, column, p.d, p.q.wide);
            b = entries8(p.dO.data + row * p.dO.ld + head * p.dO.hs, column, p.d, p.dO.wide);
            c = entries8(p.o.data + row * p.o.ld + head * p.o.hs, column, p.d, p.o.wide);
        }
        q[s] = __builtin_bit_cast(s16x8, a);
        g[s] = __builtin_bit_cast(s16x8, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            rowsum = __builtin_fmaf(T::low(b[e]), T::low(c[e]), rowsum);
            rowsum = __builtin_fmaf(T::high(b[e]), T::high(c[e]), rowsum);
        }
    }
    rowsum = sum_of_halves(rowsum);
    const float lse = see.inside ? in_twos(p.lse[at]) : kInf;
    if (see.inside && half == 0) {  // for the walk by keys, whose entries of Q and dO may stand in as zeros
        p.rowsums[at] = rowsum;
        p.rowsums[(int64_t)p.hq * p.mask.n + at] = fabsf(rowsum) < kInf ? lse : __builtin_nanf("");
    }
    const Scores to(p, head);

    f32x16 sum[kBlocks];
    // An entry of K that is not finite meets the zero weights of rows that do not see it as well.  If a sum comes
    // out not finite the workgroup walks once more with those entries as zeros: the rows that see one have a
    // log-sum that is NaN, and with it P.
    for (int entries = kAsTheyAre;; ++entries) {
        for (int b = 0; b < kBlocks; ++b) sum[b] = f32x16{};
        const bool direct = p.k.wide && p.v.wide && entries == kAsTheyAre;
        const Direct<DP, 256> from_k(p.k, kv, p.d, tid), from_v(p.v, kv, p.d, tid);
        Lane<DP> at_lane(lane);
        int buffer = 0;
        auto fetch = [&](int j0, int to) {
            from_k.fetch(lds + to, j0, first, last, tid);
            from_v.fetch(lds + to + L::kBytes, j0, first, last, tid);
        };
        arrive_and_wait();
        if (direct && first < last) fetch(first, 0);
        for (int j0 = first; j0 < last; j0 += kTileKeys, buffer ^= 2 * L::kBytes, at_lane.other(2 * L::kBytes)) {
            if (!direct) {
                stage<T, DP, 256>(lds + buffer, p.k, kv, j0, first, last, p.d, tid, entries);
                stage<T, DP, 256>(lds + buffer + L::kBytes, p.v, kv, j0, first, last, p.d, tid, kAsTheyAre);
            }
            arrive_and_wait();
            if (direct && j0 + kTileKeys < last) fetch(j0 + kTileKeys, buffer ^ 2 * L::kBytes);
            if (j0 >= high || j0 + kTileKeys <= low) continue;
            const bool edge = j0 < all_low || j0 + kTileKeys > all_high;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                f32x16 x{}, y{};
#pragma unroll
                for (int k = 0; k < kSteps; ++k) {
                    x = T::mfma(at_lane.row(lds, t, k), q[k], x);
                    y = T::mfma(at_lane.row(lds + L::kBytes, t, k), g[k], y);
                }
                const float away = (float)(see.at - j0 - 4 * half - 32 * t);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    float steep = 1.f;
                    const int j = 8 * (e >> 2) + (e & 3);
                    const float s = to.score(x[e], away - (float)j, steep);
                    float weight = __builtin_amdgcn_exp2f(s - lse) * (y[e] - rowsum) * steep;
                    if (edge && (unsigned)(j0 + 4 * half + 32 * t + j - see.lo) >= (unsigned)(see.hi - see.lo)) weight = 0.f;
                    x[e] = weight;
                }
                const s16x8 w0 = rounded_operand<T>(x, 0), w1 = rounded_operand<T>(x, 1);
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) {
                    sum[b] = T::mfma(at_lane.column(lds, b, 2 * t), w0, sum[b]);
                    sum[b] = T::mfma(at_lane.column(lds, b, 2 * t + 1), w1, sum[b]);
                }
            }
        }
        if (entries != kAsTheyAre) break;
        float zero = 0.f;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) zero = __builtin_fmaf(sum[b][e], 0.f, zero);
        if (!__syncthreads_or(zero != 0.f)) break;
    }
    if (!see.inside) return;
    unsigned short* const o = p.dq.data + row * p.dq.ld + head * p.dq.hs;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = sum[b][4 * a + e] * p.scale;
            put4<T>(o, 32 * b + 8 * a + 4 * half, p.d, p.dq.wide, x);
        }
}

template <typename T, int DP>
__global__ __launch_bounds__(256, 1) void attn_grad_keys_kernel(Problem p) {
    typedef Tile<DP> L;
    constexpr int kBlocks = DP / 32, kSteps = DP / 16;
    __shared__ __attribute__((aligned(16))) unsigned char lds[4 * L::kBytes];
    __shared__ __attribute__((aligned(16))) float of_rows[2][2][kTileKeys];  // log-sums, row sums
    __shared__ int ends[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    const int tiles = (p.mask.m + kTileRows - 1) / kTileRows, group = p.hq / p.hkv;
    const int w = work_of(blockIdx.x, gridDim.x);
    // the first keys first: with a causal mask most rows see them
    const int part = w % p.splits, tile = w / p.splits % tiles, kv = w / p.splits / tiles;
    const int key = tile * kTileRows + wave * 32 + (lane & 31);
    const Span see = rows_of_key(p.mask, key);
    const bool some = see.lo < see.hi;
    const int low = wave_least(some ? see.lo : INT_MAX), high = wave_most(some ? see.hi : INT_MIN);
    const int all_low = wave_most(see.inside ? see.lo : INT_MIN), all_high = wave_least(see.inside ? see.hi : INT_MAX);
    if (tid < 2) ends[tid] = tid ? INT_MIN : INT_MAX;
    __syncthreads();
    if (lane == 0) {
        atomicMin(&ends[0], low);
        atomicMax(&ends[1], high);
    }
    __syncthreads();
    int first = ends[0], last = ends[1];
    if (first >= last) first = last = 0;

    s16x8 k[kSteps], v[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        u32x4 a = {0, 0, 0, 0}, b = a;
        const int column = 16 * s + 8 * half;
        if (see.inside) {
            a = entries8(p.k.data + key * p.k.ld + kv * p.k.hs, column, p.d, p.k.wide);
            b = entries8(p.v.data + key * p.v.ld + kv * p.v.hs, column, p.d, p.v.wide);
        }
        k[s] = __builtin_bit_cast(s16x8, a);
        v[s] = __builtin_bit_cast(s16x8, b);
    }

    f32x16 dk[kBlocks], dv[kBlocks];
    const int64_t all = (int64_t)p.hq * p.mask.n;
    const int head0 = kv * group + group * part / p.splits, head1 = kv * group + group * (part + 1) / p.splits;
    // As by rows: entries of Q and dO that are not finite as zeros in a second walk.  Their rows have a log-sum or a
    // row sum, and with it P, that is NaN.
    for (int entries = kAsTheyAre;; ++entries) {
        for (int b = 0; b < kBlocks; ++b) dk[b] = dv[b] = f32x16{};
        const bool direct = p.q.wide && p.dO.wide && entries == kAsTheyAre;
        Lane<DP> at_lane(lane);
        int buffer = 0;
        auto fetch = [&](int head, int i0, int to) {
            const Direct<DP, 256> from_q(p.q, head, p.d, tid), from_g(p.dO, head, p.d, tid);
            from_q.fetch(lds + to * 2 * L::kBytes, i0, first, last, tid);
            from_g.fetch(lds + to * 2 * L::kBytes + L::kBytes, i0, first, last, tid);
            if (wave < 2) {
                const float* const from = p.rowsums + (wave ? 0 : all) + (int64_t)head * p.mask.n + i0;
                fetch_words(of_rows[to][wave], from, lane, last - i0);
            }
        };
        arrive_and_wait();
        if (direct && first < last) fetch(head0, first, 0);
        for (int head = head0; head < head1; ++head) {
            const Scores to(p, head);
            for (int i0 = first; i0 < last; i0 += kTileKeys, buffer ^= 1, at_lane.other(2 * L::kBytes)) {
                if (!direct) {
                    unsigned char* const to = lds + buffer * 2 * L::kBytes;
                    stage<T, DP, 256>(to, p.q, head, i0, first, last, p.d, tid, entries);
                    stage<T, DP, 256>(to + L::kBytes, p.dO, head, i0, first, last, p.d, tid, entries);
                    if (tid < 2 * kTileKeys) {
                        const float* const from = p.rowsums + (wave ? 0 : all) + (int64_t)head * p.mask.n + i0;
                        of_rows[buffer][wave][lane] = i0 + lane < last ? from[lane] : 0.f;
                    }
                }
                arrive_and_wait();
                if (direct) {
                    if (i0 + kTileKeys < last)
                        fetch(head, i0 + kTileKeys, buffer ^ 1);
                    else if (head + 1 < head1)
                        fetch(head + 1, first, buffer ^ 1);
                }
                if (i0 >= high || i0 + kTileKeys <= low) continue;
                const bool edge = i0 < all_low || i0 + kTileKeys > all_high;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    f32x16 x{}, y{};
#pragma unroll
                    for (int c = 0; c < kSteps; ++c) {
                        x = T::mfma(at_lane.row(lds, t, c), k[c], x);
                        y = T::mfma(at_lane.row(lds + L::kBytes, t, c), v[c], y);
                    }
                    const float away = (float)(i0 + see.at - key + 4 * half + 32 * t);
#pragma unroll
                    for (int a = 0; a < 4; ++a) {
                        const f32x4 lse = *reinterpret_cast<const f32x4*>(&of_rows[buffer][0][32 * t + 8 * a + 4 * half]);
                        const f32x4 rowsum = *reinterpret_cast<const f32x4*>(&of_rows[buffer][1][32 * t + 8 * a + 4 * half]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float steep = 1.f;
                            const int i = 8 * a + e;
                            const float s = to.score(x[4 * a + e], away + (float)i, steep);
                            float weight = __builtin_amdgcn_exp2f(s - lse[e]);
                            float slope = weight * (y[4 * a + e] - rowsum[e]) * steep;
                            if (edge && (unsigned)(i0 + 4 * half + 32 * t + i - see.lo) >= (unsigned)(see.hi - see.lo))
                                weight = slope = 0.f;
                            x[4 * a + e] = weight;
                            y[4 * a + e] = slope;
                        }
                    }
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const s16x8 weights = rounded_operand<T>(x, c), slopes = rounded_operand<T>(y, c);
#pragma unroll
                        for (int b = 0; b < kBlocks; ++b) {
                            dv[b] = T::mfma(at_lane.column(lds + L::kBytes, b, 2 * t + c), weights, dv[b]);
                            dk[b] = T::mfma(at_lane.column(lds, b, 2 * t + c), slopes, dk[b]);
                        }
                    }
                }
            }
        }
        if (entries != kAsTheyAre) break;
        float zero = 0.f;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) zero = __builtin_fmaf(dk[b][e], 0.f, __builtin_fmaf(dv[b][e], 0.f, zero));
        if (!__syncthreads_or(zero != 0.f)) break;
    }
    if (!see.inside) return;
    if (p.splits > 1) {
        const int64_t keys = (int64_t)p.mask.m * p.hkv;
        float* const o = p.partial + (2 * part * keys + (int64_t)key * p.hkv + kv) * p.d;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int c = 32 * b + 8 * (e >> 2) + 4 * half + (e & 3);
                if (c >= p.d) continue;
                o[c] = dk[b][e] * p.scale;
                o[keys * p.d + c] = dv[b][e];
            }
        return;
    }
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            float x[4], y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[e] = dk[b][4 * a + e] * p.scale;
                y[e] = dv[b][4 * a + e];
            }
            put4<T>(p.dk.data + key * p.dk.ld + kv * p.dk.hs, 32 * b + 8 * a + 4 * half, p.d, p.dk.wide, x);
            put4<T>(p.dv.data + key * p.dv.ld + kv * p.dv.hs, 32 * b + 8 * a + 4 * half, p.d, p.dv.wide, y);
        }
}

// dK and dV of one key and head from the parts, in ascending order: a wave for each.
template <typename T>
__global__ __launch_bounds__(256) void attn_grad_join_kernel(Problem p) {
    const int lane = threadIdx.x & 63;
    const int64_t keys = (int64_t)p.mask.m * p.hkv, at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (at >= keys) return;
    const int key = (int)(at / p.hkv), kv = (int)(at % p.hkv);
    if (!rows_of_key(p.mask, key).inside) return;
    for (int c = lane; c < p.d; c += 64) {
        float a = 0.f, b = 0.f;
        for (int s = 0; s < p.splits; ++s) {
            const float* o = p.partial + (2 * s * keys + at) * p.d + c;
            a += o[0];
            b += o[keys * p.d];
        }
        p.dk.data[key * p.dk.ld + kv * p.dk.hs + c] = (unsigned short)T::pack(a, 0.f);
        p.dv.data[key * p.dv.ld + kv * p.dv.hs + c] = (unsigned short)T::pack(b, 0.f);
    }
}

template <typename T, int DP>
hipError_t launch_kernels(const Problem& p, hipStream_t stream) {
    const int64_t row_tiles = (p.mask.n + kTileRows - 1) / kTileRows, key_tiles = (p.mask.m + kTileRows - 1) / kTileRows;
    const dim3 block(256);
    if (row_tiles) attn_grad_rows_kernel<T, DP><<<dim3((unsigned)(row_tiles * p.hq)), block, 0, stream>>>(p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !key_tiles) return e;
    attn_grad_keys_kernel<T, DP><<<dim3((unsigned)(key_tiles * p.hkv * p.splits)), block, 0, stream>>>(p);
    e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    attn_grad_join_kernel<T><<<dim3((unsigned)(((int64_t)p.mask.m * p.hkv + 3) / 4)), block, 0, stream>>>(p);
    return hipGetLastError();
}

template <typename T>
hipError_t launch(const Problem& p, hipStream_t stream) {
    return p.d <= 64 ? launch_kernels<T, 64>(p, stream) : p.d <= 96 ? launch_kernels<T, 96>(p, stream) : launch_kernels<T, 128>(p, stream);
}

}  // namespace

hipError_t launch_grad(const Problem& p, hipStream_t stream) {
    return p.f16 ? launch<F16>(p, stream) : launch<Bf16>(p, stream);
}

}  // namespace attn
