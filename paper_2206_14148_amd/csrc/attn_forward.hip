// O = softmax(scores) V with a running maximum and sum: one pass over the keys, no n x m matrix.
#include "attn_device.h"

namespace attn {

namespace {

// A row's weights are powers of two of its scores less `top`, which goes up so that the largest is 2^kPower when it is over 2^kSlack.
// bf16: that is, sums are scaled down for a score that grows by 8.  f16: its largest powers of two are used, so that a weight of 2^-21 of
// the row's largest keeps all its bits (many small ones beside a large one add up: with kPower = 0 60000 weights of
// 2^-24.5 came to 1.4 times their sum).
template <typename T>
constexpr float kPower = T::kOne == F16::kOne ? 7.f : 0.f;
template <typename T>
constexpr float kSlack = 8.f + kPower<T>;

// A lane's sums of its row to memory, or to the workspace as they are.  entries: see the walk below.
template <typename T, int BLOCKS>
__device__ __forceinline__ void write_rows(const Problem& p, const Span& see, int head, int row, int split, int half, int entries,
                                           const f32x16* sum, float top, float total) {
    const int64_t at = (int64_t)head * p.mask.n + row;
    const float inverse = p.splits > 1 ? 1.f : total == 0.f ? 0.f : 1.f / total;
    const int64_t rows = (int64_t)p.hq * p.mask.n;
    float* const parts = p.partial + ((int64_t)split * rows + at) * p.d;
    unsigned short* const o = p.o.data + row * p.o.ld + head * p.o.hs;
    if (entries >= kUp) {
        const float mark = entries == kUp ? kInf : -kInf;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int c = 32 * b + 8 * (e >> 2) + 4 * half + (e & 3);
                if (c >= p.d || !(sum[b][e] > 0.f)) continue;
                if (p.splits > 1)
                    parts[c] += mark;
                else
                    o[c] = (unsigned short)T::pack(T::low(o[c]) + mark, 0.f);
            }
        return;
    }
    if (p.splits > 1) {
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int a = 0; a < 4; ++a) put4(parts, 32 * b + 8 * a + 4 * half, p.d, sum[b], 4 * a);
        if (half == 0) {
            float* ends_of = p.partial + (int64_t)p.splits * rows * p.d + 2 * ((int64_t)split * rows + at);
            ends_of[0] = top;
            ends_of[1] = total;
        }
        return;
    }
    if (p.lse && half == 0) p.lse[at] = total == 0.f ? -kInf : (top + __builtin_amdgcn_logf(total)) * kLn2;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = total == 0.f ? 0.f : sum[b][4 * a + e] * inverse;
            put4<T>(o, 32 * b + 8 * a + 4 * half, p.d, p.o.wide, x);
        }
}

// Four waves of 32 rows; a step takes 64 keys, whose K and V go straight to LDS while the last step's are worked on (64 KiB, two
// workgroups on a compute unit, one's exponentials beside the other's products).  8192 rows, causal, 32 heads on 8, d = 128,
// bf16: 541 us, 1020 TFLOP/s (a large matrix product reaches 1390 here).  Matrix cores are busy for 53 % of the cycles.  A wave has one
// set of rows, so every MFMA reads 1 KB of its own from LDS: at 128 bytes a cycle another 53 %, with the tiles' writes and
// conflicts four fifths.  The vector unit (a maximum, a product, an exponential, a sum and half a conversion for each score)
// is busy for about half as well, and the clock falls to 1.8 GHz: an order of instructions that kept the matrix cores
// 14 % busier took the same time.  Which of them binds was not separated.
// With a cap another exponential and a reciprocal come to each score, and the vector unit alone bounds it.
template <typename T, int DP, bool LARGE_CAP>  // cap > kLargeCap
__global__ __launch_bounds__(256, 2) void attn_forward_kernel(Problem p) {
    typedef Tile<DP> L;
    constexpr int kBlocks = DP / 32, kSteps = DP / 16;
    __shared__ __attribute__((aligned(16))) unsigned char lds[4 * L::kBytes];
    __shared__ int ends[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
    // The heads that share a K and V stand side by side: "rows" of the tile are rows and, within a row, its heads.
    const int group = p.hq / p.hkv, tiles = (int)(((int64_t)p.mask.n * group + kTileRows - 1) / kTileRows);
    const Work work = work_of(blockIdx.x, p.hkv, tiles * p.splits);
    // the last rows first: with a causal mask they see the most keys
    const int split = work.piece % p.splits, tile = tiles - 1 - work.piece / p.splits, kv = work.kv;
    const int line = tile * kTileRows + wave * 32 + (lane & 31), row = line / group, head = kv * group + line % group;
    __shared__ LocalDocs local;
    const Span see = keys_of_row(with_local(p.mask, local, tid), row);
    const bool some = see.lo < see.hi;
    const int low = wave_least(some ? see.lo : INT_MAX), high = wave_most(some ? see.hi : INT_MIN);
    // keys that all rows of the wave see (rows that are not written do not count)
    const int all_low = wave_most(see.inside ? see.lo : INT_MIN), all_high = wave_least(see.inside ? see.hi : INT_MAX);
    if (tid < 2) ends[tid] = tid ? INT_MIN : INT_MAX;
    __syncthreads();
    if (lane == 0) {
        atomicMin(&ends[0], low);
        atomicMax(&ends[1], high);
    }
    __syncthreads();
    int first = __builtin_amdgcn_readfirstlane(ends[0]), last = __builtin_amdgcn_readfirstlane(ends[1]);
    if (first >= last) first = last = 0;
    const int steps = (last - first + kTileKeys - 1) / kTileKeys;
    const int s0 = (int)((int64_t)steps * split / p.splits), s1 = (int)((int64_t)steps * (split + 1) / p.splits);

    s16x8 q[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        u32x4 v = {0, 0, 0, 0};
        if (see.inside) v = entries8(p.q.data + row * p.q.ld + head * p.q.hs, 16 * s + 8 * half, p.d, p.q.wide);
        q[s] = __builtin_bit_cast(s16x8, v);
    }
    // What the walk calls a score is u / scale: the product itself, and a cap and slopes divided by the scale.
    const float factor = p.scale * kLog2e;  // of a score, to powers of two
    const bool capped = LARGE_CAP || p.cap > 0.f;
    const float to_cap = LARGE_CAP ? p.scale / p.cap : capped ? 2.f * factor / p.cap : 0.f, from_cap = p.cap / p.scale;
    const float slope = p.slopes && see.inside ? p.slopes[head] / p.scale : 0.f;
    float slack = kSlack<T> / factor, lift = kPower<T> / factor;

    f32x16 sum[kBlocks];
    float top, total;  // of a lane's row: what its scores are taken less of, the sum of its weights (of half the keys)
    float most_over;   // how far a score may be over top: slack, and for a row that has seen no key nothing at all
    Lane<DP> at(lane);
    unsigned char* const keys = lds;
    unsigned char* const values = lds + 2 * L::kBytes;
    auto begin = [&]() {
        for (int b = 0; b < kBlocks; ++b) sum[b] = f32x16{};
        top = total = 0.f;
        most_over = -kInf;
    };
    auto products = [&](f32x16* x) {
        const float less = capped ? 0.f : -top;  // top comes off as the product's first summand
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[t][e] = less;
#pragma unroll
            for (int k = 0; k < kSteps; ++k) x[t] = T::mfma(at.row(keys, t, k), q[k], x[t]);
        }
    };
    // A tile's products x to what the weights are the exponentials of.
    auto scores = [&](f32x16* x, int j0, bool marks) {
        if (LARGE_CAP) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) x[t][e] = __builtin_fmaf(from_cap, tanh_of(to_cap * x[t][e]), -top);
        } else if (capped) {
            const float one = from_cap - top, two = -2.f * from_cap;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    x[t][e] = __builtin_fmaf(two, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(to_cap * x[t][e])), one);
        }
        if (p.slopes) {
            const float away = (float)(see.at - j0 - 4 * half);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    x[t][e] = __builtin_fmaf(-slope, fabsf(away - (float)(32 * t + 8 * (e >> 2) + (e & 3))), x[t][e]);
        }
        if (j0 < all_low || j0 + kTileKeys > all_high) {
            const unsigned width = (unsigned)(see.hi - see.lo);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if ((unsigned)(j0 + 4 * half + 32 * t + 8 * (e >> 2) + (e & 3) - see.lo) >= width) x[t][e] = -kInf;
        }
        float most = x[0][0];
#pragma unroll
        for (int e = 1; e < 16; ++e) most = fmaxf(most, x[0][e]);
#pragma unroll
        for (int e = 0; e < 16; ++e) most = fmaxf(most, x[1][e]);
        most = max_of_halves(most);
        if (__any(most > most_over)) {
            const bool none = most_over != slack;
            const float up = none ? (most == -kInf ? 0.f : most - lift) : fmaxf(most - lift, 0.f);
            const float shrink = none || marks ? 1.f : __builtin_amdgcn_exp2f(-up * factor);
            if (most > -kInf) most_over = slack;
            top += up;
            total *= shrink;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) sum[b] *= shrink;
#pragma unroll
            for (int t = 0; t < 2; ++t) x[t] -= up;
        }
    };
    // One tile that lies in LDS.  marks: with a weight of one for every key that is seen (and has a score
    // above -infinity), whatever comes behind it.
    auto tile_of = [&](int j0, bool marks) {
        if (j0 >= high || j0 + kTileKeys <= low) return;
        f32x16 x[2];
        products(x);
        scores(x, j0, marks);
        if (marks) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) x[t][e] = x[t][e] > -kInf ? 0.f : -kInf;
        }
        s16x8 weights[4];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float part = 0.f;  // (16 are added up before they meet what may be much larger)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                x[t][e] = __builtin_amdgcn_exp2f(x[t][e] * factor);
                part = e ? part + x[t][e] : x[t][e];
            }
            weights[2 * t] = rounded_operand<T>(x[t], 0);
            weights[2 * t + 1] = rounded_operand<T>(x[t], 1);
            total += part;
        }
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int k = 0; k < 4; ++k) sum[b] = T::mfma(at.column(values, b, k), weights[k], sum[b]);
    };
    auto write = [&](int entries) {
        if (see.inside)
            write_rows<T, kBlocks>(p, see, head, row, split, half, entries, sum, most_over == slack ? top * factor : -kInf,
                                   sum_of_halves(total));
    };

    int entries = kAsTheyAre;
    float zero;  // NaN where a lane's sums are not finite
    auto all_finite = [&]() {
        zero = 0.f;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) zero = __builtin_fmaf(sum[b][e], 0.f, zero);
        return !__syncthreads_or(zero != 0.f);
    };
    if (p.k.wide && p.v.wide) {
        // one pair of buffers is worked on while the other is filled
        const Direct<DP, 256> from_k(p.k, kv, p.d, tid), from_v(p.v, kv, p.d, tid);
        auto bring = [&](int s) {
            from_k.fetch(keys + (s - s0 & 1) * L::kBytes, first + s * kTileKeys, first, last, tid);
            from_v.fetch(values + (s - s0 & 1) * L::kBytes, first + s * kTileKeys, first, last, tid);
        };
        begin();
        if (s0 < s1) bring(s0);
        for (int s = s0; s < s1; ++s, at.other(L::kBytes)) {
            arrive_and_wait();
            if (s + 1 < s1) bring(s + 1);
            tile_of(first + s * kTileKeys, false);
        }
        if (all_finite()) {
            write(entries);
            return;
        }
        at = Lane<DP>(lane);
        entries = kFinite;
    }
    // Without 16-byte reads; and where a sum came out not finite.  An infinity or a NaN in V meets the zero weights of
    // rows that do not see it as well, and 0 * infinity is NaN.  Then the workgroup walks three times more: with those
    // entries as zeros, and with ones for what raises a sum to +infinity and to -infinity, whose sums are not zero
    // for the rows that see one (all weights are one there: a small one may round to zero, and still carries an infinity).
    // In bf16 values near the largest number may add up past it though their mean is finite.  Rows whose sums are not finite without
    // such entries either are made again with weights of 2^-32 at most, of which the 2^30 keys there can be add up to 1 / 4.
    for (bool low = false, mine = true;;) {
        begin();
        for (int s = s0; s < s1; ++s) {
            const int j0 = first + s * kTileKeys;
            arrive_and_wait();
            stage<T, DP, 256>(keys, p.k, kv, j0, first, last, p.d, tid, kAsTheyAre);
            stage<T, DP, 256>(values, p.v, kv, j0, first, last, p.d, tid, entries);
            arrive_and_wait();
            tile_of(j0, entries >= kUp);
        }
        const bool fine = entries >= kUp || all_finite();
        if (entries == kAsTheyAre && !fine) {
            entries = kFinite;
            continue;
        }
        if (mine) write(entries);
        if (entries == kAsTheyAre || entries == kDown) return;
        if (entries == kFinite && !fine && !low && kPower<T> == 0.f) {  // (f16 has no such values)
            low = true;
            slack = (kSlack<T> - 40.f) / factor;
            lift = -40.f / factor;
            mine = sum_of_halves(zero) != 0.f;
            continue;
        }
        mine = true;
        ++entries;
    }
}

// The ranges' sums of one row, in ascending order: WAVES waves for each row and head.
static_assert(kMaxSplits <= 4 * 64, "");
template <typename T, int WAVES>
__global__ __launch_bounds__(256) void attn_join_kernel(Problem p) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t rows = (int64_t)p.hq * p.mask.n, at = WAVES == 1 ? (int64_t)blockIdx.x * 4 + wave : (int64_t)blockIdx.x;
    if (at >= rows) return;
    const int head = (int)(at / p.mask.n), row = (int)(at % p.mask.n);
    if (!keys_of_row(p.mask, row).inside) return;
    const Joined r = join_ranges<WAVES>(p.partial, p.splits, p.splits, rows, at, p.d, lane, wave);
    if (WAVES > 1 && wave > 0) return;
    const float inverse = r.total == 0.f ? 0.f : 1.f / r.total;
    for (int e = 0; e < 2; ++e)
        if (64 * e + lane < p.d)
            p.o.data[row * p.o.ld + head * p.o.hs + 64 * e + lane] =
                (unsigned short)T::pack(r.total == 0.f ? 0.f : r.x[e] * inverse, 0.f);
    if (p.lse && lane == 0) p.lse[at] = r.total == 0.f ? -kInf : (r.top + __builtin_amdgcn_logf(r.total)) * kLn2;
}

template <typename T, bool LARGE_CAP>
void launch_walk(const Problem& p, dim3 grid, hipStream_t stream) {
    if (p.d <= 64)
        attn_forward_kernel<T, 64, LARGE_CAP><<<grid, dim3(256), 0, stream>>>(p);
    else if (p.d <= 96)
        attn_forward_kernel<T, 96, LARGE_CAP><<<grid, dim3(256), 0, stream>>>(p);
    else
        attn_forward_kernel<T, 128, LARGE_CAP><<<grid, dim3(256), 0, stream>>>(p);
}

template <typename T>
hipError_t launch(const Problem& p, hipStream_t stream) {
    const int64_t tiles = ((int64_t)p.mask.n * (p.hq / p.hkv) + kTileRows - 1) / kTileRows;
    const dim3 grid((unsigned)(tiles * p.hkv * p.splits)), block(256);
    // (a kernel of its own: as a branch the series of large caps cost the walks without it 2 %)
    if (p.cap > kLargeCap)
        launch_walk<T, true>(p, grid, stream);
    else
        launch_walk<T, false>(p, grid, stream);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    const int64_t rows = (int64_t)p.hq * p.mask.n;
    if (p.splits <= 64)
        attn_join_kernel<T, 1><<<dim3((unsigned)((rows + 3) / 4)), block, 0, stream>>>(p);
    else
        attn_join_kernel<T, 4><<<dim3((unsigned)rows), block, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_forward(const Problem& p, hipStream_t stream) {
    return p.f16 ? launch<F16>(p, stream) : launch<Bf16>(p, stream);
}

}  // namespace attn
