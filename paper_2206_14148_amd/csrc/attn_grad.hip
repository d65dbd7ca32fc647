// The gradient of O = softmax(scores) V.  P is made again from Q, K and the rows' log-sums, tile by tile, in two
// walks: by rows for dQ (which also makes the row sums of dO * O), by keys for dK and dV.  Two walks cost two of
// seven products more than one walk would, and in return every sum has its place and its order: with one, dQ
// would have to be added to memory by whichever workgroup comes first.
#include "attn_device.h"

namespace attn {

namespace {

// 16 products x = <Q, K>, less lse / scale, and y = <dO, V>, less the row sum, to P and P y (1 - tanh^2).  Both come with what
// is taken off as their products' first summand; with a cap x comes without.  Scores are in units of the product: a cap, slopes and
// the log-sum are divided by the scale.  `lse` gives number e's log-sum and `far` how far its row stands from its key.
template <bool LARGE_CAP, bool POWERS>  // cap > kLargeCap
struct Scores {
    float factor, to_cap, from_cap, slope, per_scale;
    bool capped, sloped;
    __device__ __forceinline__ explicit Scores(const Problem& p) {
        capped = LARGE_CAP || p.cap > 0.f;
        sloped = p.slopes;
        slope = 0.f;
        per_scale = 1.f / p.scale;
        factor = p.scale * kLog2e;
        to_cap = LARGE_CAP ? p.scale / p.cap : capped ? 2.f * factor / p.cap : 0.f;
        from_cap = p.cap / p.scale;
    }
    __device__ __forceinline__ void of_head(const Problem& p, int head) {
        if (sloped) slope = p.slopes[head] * per_scale;
    }
    // `power`: of two, that both come times (0: none)
    template <typename Lse, typename Far>
    __device__ __forceinline__ void weights(f32x16& x, f32x16& y, Lse lse, Far far, float power) const {
        if (capped) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float t = LARGE_CAP ? tanh_of(to_cap * x[e])
                                          : __builtin_fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(to_cap * x[e])), 1.f);
                y[e] *= __builtin_fmaf(-t, t, 1.f);
                x[e] = __builtin_fmaf(from_cap, t, -lse(e));
            }
        }
        if (sloped) {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = __builtin_fmaf(-slope, fabsf(far(e)), x[e]);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            x[e] = __builtin_amdgcn_exp2f(POWERS ? __builtin_fmaf(x[e], factor, power) : x[e] * factor);
            y[e] *= x[e];
        }
    }
};

// The power of two that ds of a lane's row (dQ) or key (dK) is taken times as an operand in f16, and that comes off the sums at the end: ds is
// some size of <dO, V> / m, mostly below f16's normal numbers (6e-5), and with a large dO beyond its largest.  The largest
// |<dO, V> - <dO, O>| that is seen of the first tile with one, by which P <= 1 is multiplied yet, goes to 2^8 for a row, to 2^4 for a key
// (or <dO, O>: of a row that sees one key the difference is nothing but rounding): ds of a P of 2^-22 and 2^-18 keeps all its bits, and a later
// one has room for 2^7, and 2^11 by keys, whose rows' dO may be of many magnitudes.  Should one be larger, the sums are not finite, and the walk that follows first looks for
// the largest |ds|, which goes to 2^14 (scaling the sums down as it comes, as a softmax does, would not fit the registers: 550 to 700 us at
// 4096 rows, 32 heads on 8, d = 128, f16).  bf16 has the powers of two of 32 bits.
template <typename T>
struct Fitted {
    static constexpr bool kFits = T::kOne == F16::kOne;
    static constexpr unsigned kNone = 8u << 23;
    unsigned inverse;  // as bits of a float
    __device__ __forceinline__ explicit Fitted(bool sees) { inverse = sees ? kNone : 127u << 23; }  // (else nothing would ever come)
    // Whether a lane has none yet of those that see something of 32 keys (rows) of a tile; `from`: how far the lane's first of them, which is the
    // tile's first or fourth, is behind the first that it sees of `seen`.
    __device__ __forceinline__ bool wanted(int from, unsigned seen) const {
        return kFits && __any(inverse == kNone && (unsigned)(from + 31) < seen + 35u);
    }
    __device__ __forceinline__ void put(float most, int power) {
        most = max_of_halves(most);
        if (inverse == kNone && most > 0.f && most < kInf) inverse = min(max((int)(__float_as_uint(most) >> 23) - power, 9), 246) << 23;
    }
    // (a power that was not too much stays, and with it the bits of the results that did not need this walk)
    __device__ __forceinline__ void put_again(float most) {
        if (max_of_halves(most) > 0x1p15f * __uint_as_float(inverse)) inverse = kNone;
        put(most, 14);
    }
    __device__ __forceinline__ float power() const { return (float)(127 - (int)(inverse >> 23)); }
    __device__ __forceinline__ float back() const { return kFits ? __uint_as_float(inverse) : 1.f; }
    __device__ __forceinline__ s16x8 operand(const f32x16& y, int step, bool look) const {
        if constexpr (!kFits) return rounded_operand<T>(y, step);
        const float times = look ? 0.f : __uint_as_float((254u << 23) - inverse);
        u32x4 r;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            F16::v2 w;  // (one instruction each with its rounding: the product with a power of two is exact)
            w[0] = (_Float16)__builtin_fmaf(y[8 * step + 2 * e], times, 0.f);
            w[1] = (_Float16)__builtin_fmaf(y[8 * step + 2 * e + 1], times, 0.f);
            r[e] = __builtin_bit_cast(unsigned, w);
        }
        return __builtin_bit_cast(s16x8, r);
    }
};
template <typename Size>
__device__ __forceinline__ float largest(Size size) {  // of 16
    float most = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) most = fmaxf(most, size(e));
    return most;
}

// Which of a tile's 64 rows hold an entry that is not finite: a bit for each, the same in all lanes.
template <typename T, typename L>
__device__ __forceinline__ uint64_t not_finite(const unsigned char* lds, int lane) {
    constexpr unsigned kExp = T::kExponents & 0xffffu;
    bool bad = false;
#pragma unroll 1
    for (int piece = 0; piece < L::kPieces; ++piece) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(lds + lane * L::kRowBytes + 16 * piece);
#pragma unroll
        for (int e = 0; e < 4; ++e) bad = bad || (w[e] & kExp) == kExp || (w[e] >> 16 & kExp) == kExp;
    }
    return __ballot(bad);
}
// Bits low .. high - 1 of 64.
__device__ __forceinline__ uint64_t bits_between(int low, int high) {
    auto below = [](int x) { return x <= 0 ? (uint64_t)0 : x >= 64 ? ~(uint64_t)0 : ((uint64_t)1 << x) - 1; };
    return below(high) & ~below(low);
}

template <typename T, int DP, bool LARGE_CAP>
__global__ __launch_bounds__(256, 2) void attn_grad_rows_kernel(Problem p) {
    typedef Tile<DP> L;
    constexpr int kBlocks = DP / 32, kSteps = DP / 16;
    __shared__ __attribute__((aligned(16))) unsigned char lds[4 * L::kBytes];
    __shared__ int ends[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
    // (rows and, within a row, the heads that share a K and V, as in the forward pass)
    const int group = p.hq / p.hkv, tiles = (int)(((int64_t)p.mask.n * group + kTileRows - 1) / kTileRows);
    const Work work = work_of(blockIdx.x, p.hkv, tiles * p.row_splits);
    const int split = work.piece % p.row_splits, tile = tiles - 1 - work.piece / p.row_splits, kv = work.kv;
    const int line = tile * kTileRows + wave * 32 + (lane & 31), row = line / group, head = kv * group + line % group;
    __shared__ LocalDocs local;
    const Span see = keys_of_row(with_local(p.mask, local, tid), row);
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
    int first = __builtin_amdgcn_readfirstlane(ends[0]), last = __builtin_amdgcn_readfirstlane(ends[1]);
    if (first >= last) first = last = 0;
    if (p.row_splits > 1) {  // this part's steps
        const int64_t steps = (last - first + kTileKeys - 1) / kTileKeys;
        const int s0 = (int)(steps * split / p.row_splits), s1 = (int)(steps * (split + 1) / p.row_splits);
        last = min(last, first + s1 * kTileKeys);
        first += s0 * kTileKeys;
    }

    const int64_t at = (int64_t)head * p.mask.n + row;
    s16x8 q[kSteps], g[kSteps];
    float rowsum = 0.f, zero = 0.f;  // zero: NaN if an entry of Q is not finite
    unsigned bits = 0;               // of dO: none in a row that has no part in a loss
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
            bits |= b[e] & 0x7fff7fffu;
            zero = __builtin_fmaf(T::low(a[e]), 0.f, __builtin_fmaf(T::high(a[e]), 0.f, zero));
        }
    }
    rowsum = sum_of_halves(rowsum);
    const float log_sum = see.inside ? p.lse[at] : 0.f;
    const bool none = log_sum == -kInf;  // no keys: P = 0
    const float lse = none ? kInf : log_sum / p.scale;
    // An entry of Q, dO or O that is not finite (those of dO and O reach the row sum): the row's gradients and those of the keys
    // that it sees are NaN, whatever its scores come to (an infinity behind a cap gives finite ones).
    bool lost = sum_of_halves(zero) != 0.f || !(fabsf(rowsum) < kInf);
    if (see.inside && half == 0 && split == 0) {  // for the walk by keys, whose entries of Q and dO may stand in as zeros
        p.rowsums[at] = none || !lost ? -lse : __builtin_nanf("");
        p.rowsums[(int64_t)p.hq * p.mask.n + at] = none ? 0.f : -rowsum;
    }
    Scores<LARGE_CAP, Fitted<T>::kFits> to(p);
    if (see.inside) to.of_head(p, head);

    f32x16 sum[kBlocks];
    Fitted<T> fitted(some && sum_of_halves(bits ? 1.f : 0.f) > 0.f);
    float most = 0.f;  // |ds|, where a walk looks for it
    Lane<DP> at_lane(lane);
    unsigned char* const keys = lds;
    unsigned char* const values = lds + 2 * L::kBytes;
    auto begin = [&]() {
        for (int b = 0; b < kBlocks; ++b) sum[b] = f32x16{};
    };
    // One tile that lies in LDS, its rows as the last product takes them at `last_keys`.
    auto tile_of = [&](int j0, const unsigned char* last_keys, bool look) {
        if (j0 >= high || j0 + kTileKeys <= low) return;
        const bool edge = j0 < all_low || j0 + kTileKeys > all_high;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x16 x, y;
            float x_less = to.capped ? 0.f : -lse, y_less = -rowsum;
            asm("" : "+v"(x_less), "+v"(y_less));  // (or 32 registers hold them sixteen times all along)
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = x_less, y[e] = y_less;
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                x = T::mfma(at_lane.row(keys, t, k), q[k], x);
                y = T::mfma(at_lane.row(values, t, k), g[k], y);
            }
            auto seen = [&](int from, int e) { return (unsigned)(from + 8 * (e >> 2) + (e & 3)) < (unsigned)(see.hi - see.lo); };
            const int from_lo = j0 + 4 * half + 32 * t - see.lo;
            if (!look && fitted.wanted(from_lo, see.hi - see.lo)) {
                int from = from_lo;
                asm("" : "+v"(from));  // (or what this rarely needs is kept for the mask: registers)
                fitted.put(largest([&](int e) { return seen(from, e) ? fmaxf(fabsf(y[e]), fabsf(rowsum)) : 0.f; }), 8);
            }
            const float away = (float)(see.at - j0 - 4 * half - 32 * t);
            to.weights(x, y, [&](int) { return lse; }, [&](int e) { return away - (float)(8 * (e >> 2) + (e & 3)); },
                       look ? 0.f : fitted.power());
            if (edge) {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (!seen(from_lo, e)) y[e] = 0.f;
            }
            if (look) {
                most = fmaxf(most, largest([&](int e) { return fabsf(y[e]); }));
                y *= 0.f;
            }
            const s16x8 w0 = rounded_operand<T>(y, 0), w1 = rounded_operand<T>(y, 1);
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                sum[b] = T::mfma(at_lane.column(last_keys, b, 2 * t), w0, sum[b]);
                sum[b] = T::mfma(at_lane.column(last_keys, b, 2 * t + 1), w1, sum[b]);
            }
            __builtin_amdgcn_sched_barrier(0);  // (the halves do not mix: registers)
        }
    };
    auto all_finite = [&]() {
        float zero = 0.f;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) zero = __builtin_fmaf(sum[b][e], 0.f, zero);
        return !__syncthreads_or(zero != 0.f);  // (NaN)
    };
    int entries = kAsTheyAre;
    bool done = false;
    if (p.k.wide && p.v.wide) {
        const Direct<DP, 256> from_k(p.k, kv, p.d, tid), from_v(p.v, kv, p.d, tid);
        int buffer = 0;
        auto bring = [&](int j0, int to) {
            from_k.fetch(keys + to, j0, first, last, tid);
            from_v.fetch(values + to, j0, first, last, tid);
        };
        begin();
        if (first < last) bring(first, 0);
        for (int j0 = first; j0 < last; j0 += kTileKeys, buffer ^= L::kBytes, at_lane.other(L::kBytes)) {
            arrive_and_wait();
            if (j0 + kTileKeys < last) bring(j0 + kTileKeys, buffer ^ L::kBytes);
            tile_of(j0, keys, false);
        }
        done = all_finite();
        at_lane = Lane<DP>(lane_again());
        entries = kFinite;
    }
    // Without 16-byte reads; and where a sum came out not finite.  An entry of K that is not finite meets the zero weights
    // of rows that do not see it as well.  Then the workgroup walks once more, with zeros in the place of those entries
    // for the product with ds alone (the scores are made of what K holds), and keeps in mind which rows see one: of
    // those, and of no others, the gradient is NaN, as 0 * infinity is.
    for (; !done; ++entries) {
        for (int look = Fitted<T>::kFits && entries == kFinite; look >= 0; --look) {
            begin();
            for (int j0 = first; j0 < last; j0 += kTileKeys) {
                const int own_tid = 64 * wave + lane_again();
                arrive_and_wait();
                stage<T, DP, 256>(keys, p.k, kv, j0, first, last, p.d, own_tid, kAsTheyAre);
                stage<T, DP, 256>(values, p.v, kv, j0, first, last, p.d, own_tid, kAsTheyAre);
                if (entries == kFinite) stage<T, DP, 256>(keys + L::kBytes, p.k, kv, j0, first, last, p.d, own_tid, kFinite);
                arrive_and_wait();
                if (entries == kFinite) {
                    const uint64_t bad = not_finite<T, L>(keys, own_tid & 63);
                    lost = lost || (bad & bits_between(see.lo - j0, see.hi - j0));
                }
                tile_of(j0, entries == kFinite ? keys + L::kBytes : keys, look);
            }
            if (look) fitted.put_again(most);
        }
        done = entries == kFinite || all_finite();
    }
    if (!see.inside) return;
    const float times = lost ? __builtin_nanf("") : p.scale * fitted.back();
    // (made again here rather than kept from where it was first needed)
    const int own_lane = lane_again(), own_half = own_lane >> 5, own_line = tile * kTileRows + wave * 32 + (own_lane & 31);
    const int own_row = own_line / group, own_head = kv * group + own_line % group;
    if (p.row_splits > 1) {
        float* const parts = p.row_partial + ((split * (int64_t)p.hq + own_head) * p.mask.n + own_row) * p.d;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int a = 0; a < 4; ++a) put4(parts, 32 * b + 8 * a + 4 * own_half, p.d, none ? f32x16{} : sum[b] * times, 4 * a);
        return;
    }
    unsigned short* const o = p.dq.data + own_row * p.dq.ld + own_head * p.dq.hs;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = none ? 0.f : sum[b][4 * a + e] * times;
            put4<T>(o, 32 * b + 8 * a + 4 * own_half, p.d, p.dq.wide, x);
        }
}

// By keys a step takes 32 rows, and V, the second operand of only one product, stays in LDS: so two workgroups share a
// compute unit, one's exponentials beside the other's products.  4096 rows and keys, causal, 32 heads on 8, d = 128, bf16: 345 us
// or 800 TFLOP/s of its four products (with V in registers and 64 rows a step one workgroup, and 444 us); the walk by rows
// takes 247 us for its three, 830 TFLOP/s.  Matrix cores are busy for 44 and 48 % of the cycles; their operands from LDS, 1 KB for
// an MFMA (by keys a quarter more, V's), take 55 and 48 % of them at 128 bytes a cycle, the tiles' writes and conflicts 17 and 16 %;
// the vector instructions of the exponentials (some 10 for a score) hide behind the other workgroup's products only in part.
template <typename T, int DP, bool LARGE_CAP>
__global__ __launch_bounds__(256, 2) void attn_grad_keys_kernel(Problem p) {
    typedef Tile<DP, kStepRows> L;
    constexpr int kBlocks = DP / 32, kSteps = DP / 16;
    __shared__ __attribute__((aligned(16))) unsigned char lds[4 * L::kBytes + 2 * Tile<DP>::kBytes];
    __shared__ __attribute__((aligned(16))) float of_rows[2][2][kStepRows];  // see Problem::rowsums
    __shared__ int ends[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
    const int tiles = (p.mask.m + kTileRows - 1) / kTileRows, group = p.hq / p.hkv;
    const Work work = work_of(blockIdx.x, p.hkv, tiles * p.splits);
    // the first keys first: with a causal mask most rows see them
    const int part = work.piece % p.splits, tile = work.piece / p.splits, kv = work.kv;
    const int key = tile * kTileRows + wave * 32 + (lane & 31);
    __shared__ LocalDocs local;
    const Span see = rows_of_key(with_local(p.mask, local, tid), key);
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
    int first = __builtin_amdgcn_readfirstlane(ends[0]), last = __builtin_amdgcn_readfirstlane(ends[1]);
    if (first >= last) first = last = 0;

    unsigned char* const queries = lds;
    unsigned char* const grads = lds + 2 * L::kBytes;
    unsigned char* const values = lds + 4 * L::kBytes;  // rows of 128 keys
    unsigned char* const own_values = values + wave * 32 * L::kRowBytes;
    for (int x = 0; x < 2; ++x)
        stage<T, DP, 256>(values + x * Tile<DP>::kBytes, p.v, kv, tile * kTileRows + x * kTileKeys, 0, p.mask.m, p.d, tid, kAsTheyAre);
    s16x8 k[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        u32x4 a = {0, 0, 0, 0};
        if (see.inside) a = entries8(p.k.data + key * p.k.ld + kv * p.k.hs, 16 * s + 8 * half, p.d, p.k.wide);
        k[s] = __builtin_bit_cast(s16x8, a);
    }

    f32x16 dk[kBlocks], dv[kBlocks];
    Fitted<T> fitted(some);  // of dk
    float most = 0.f;
    Lane<DP> at_lane(lane);
    // This part's steps, of those through all rows of all heads that read K and V: from row0 of head0 to before row1 of the
    // last head.
    const int through = (last - first + kStepRows - 1) / kStepRows;
    const int step0 = (int)((int64_t)through * group * part / p.splits), step1 = (int)((int64_t)through * group * (part + 1) / p.splits);
    int head0 = 0, head1 = 0, row0 = 0, row1 = 0;
    if (step0 < step1) {
        head0 = kv * group + step0 / through;
        head1 = kv * group + (step1 - 1) / through + 1;
        row0 = first + step0 % through * kStepRows;
        row1 = first + ((step1 - 1) % through + 1) * kStepRows;
    }
    auto begin = [&]() {
        for (int b = 0; b < kBlocks; ++b) dk[b] = dv[b] = f32x16{};
    };
    // of a lane's first row of a tile: how far past the key it stands, and past the first row that sees the key
    int from_key = see.at - key + 4 * half;
    asm("" : "+v"(from_key));  // (or what it is made of is kept as well)
    const int from_first = 4 * half - see.lo;
    const unsigned seen = see.hi - see.lo;
    // 32 rows that lie in LDS.
    Scores<LARGE_CAP, Fitted<T>::kFits> to(p);
    // P of f16 (of many keys some 1 / m, below its normal numbers from 16000 on) as an operand times 2^14, and ds with it.
    constexpr int kPower = Fitted<T>::kFits ? 14 : 0;
    constexpr float kBack = kPower ? 0x1p-14f : 1.f;
    auto tile_of = [&](int i0, int buffer, bool look) {
        if (i0 >= high || i0 + kStepRows <= low) return;
        const unsigned own = at_lane.rows ^ (buffer ? L::kBytes : 0);
        auto own_at = [&](int c) { return *reinterpret_cast<const s16x8*>(own_values + (own ^ (32 * c))); };
        f32x16 x, y;
        auto of_all = [&](f32x16& to_x, int which) {
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                const f32x4 four = *reinterpret_cast<const f32x4*>(&of_rows[buffer][which][8 * a + 4 * half]);
#pragma unroll
                for (int e = 0; e < 4; ++e) to_x[4 * a + e] = four[e];
            }
        };
        if (to.capped)
            x = f32x16{};
        else
            of_all(x, 0);
        of_all(y, 1);
#pragma unroll
        for (int c = 0; c < kSteps; ++c) {
            x = T::mfma(at_lane.row(queries, 0, c), k[c], x);
            y = T::mfma(at_lane.row(grads, 0, c), own_at(c), y);
            if (c % 2 == 1) __builtin_amdgcn_sched_barrier(0);
        }
        auto sees = [&](int from, int e) { return (unsigned)(from + 8 * (e >> 2) + (e & 3)) < seen; };
        if (!look && fitted.wanted(i0 + from_first, seen)) {
            int from = i0 + from_first;
            asm("" : "+v"(from));
            float most = 0.f;
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                const f32x4 rowsum = *reinterpret_cast<const f32x4*>(&of_rows[buffer][1][8 * a + 4 * half]);
#pragma unroll
                for (int e = 0; e < 4; ++e) most = fmaxf(most, sees(from, 4 * a + e) ? fmaxf(fabsf(y[4 * a + e]), fabsf(rowsum[e])) : 0.f);
            }
            fitted.put(most, 4 - kPower);
        }
        const float away = (float)(i0 + from_key);
        to.weights(x, y, [&](int e) { return -of_rows[buffer][0][8 * (e >> 2) + 4 * half + (e & 3)]; },
                   [&](int e) { return away + (float)(8 * (e >> 2) + (e & 3)); }, (float)kPower);
        if (i0 < all_low || i0 + kStepRows > all_high) {
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (!sees(i0 + from_first, e)) x[e] = y[e] = 0.f;
        }
        if (look) most = fmaxf(most, largest([&](int e) { return fabsf(y[e]); }));
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const s16x8 weights = rounded_operand<T>(x, c), slopes = fitted.operand(y, c, look);
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                dv[b] = T::mfma(at_lane.column(grads, b, c), weights, dv[b]);
                dk[b] = T::mfma(at_lane.column(queries, b, c), slopes, dk[b]);
                if (b % 2 == 1) __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    auto all_finite = [&]() {
        float zero = 0.f;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) zero = __builtin_fmaf(dk[b][e], 0.f, __builtin_fmaf(dv[b][e], 0.f, zero));
        return !__syncthreads_or(zero != 0.f);
    };
    auto sums_of = [&](int which, int head, int i0) {
        return p.rowsums + ((int64_t)which * p.hq + head) * p.mask.n + i0;
    };
    int entries = kAsTheyAre;
    bool done = false;
    if (p.q.wide && p.dO.wide) {
        int buffer = 0;
        auto bring = [&](int head, int i0, int to) {
            const Direct<DP, 256, kStepRows> from_q(p.q, head, p.d, tid), from_g(p.dO, head, p.d, tid);
            from_q.fetch(queries + to * L::kBytes, i0, first, last, tid);
            from_g.fetch(grads + to * L::kBytes, i0, first, last, tid);
            if (wave < 2 && lane < kStepRows) fetch_words(of_rows[to][wave], sums_of(wave, head, i0), lane, last - i0);
        };
        begin();
        if (head0 < head1) bring(head0, row0, 0);
        for (int head = head0; head < head1; ++head) {
            to.of_head(p, head);
            const int end = head + 1 < head1 ? last : row1;
            for (int i0 = head == head0 ? row0 : first; i0 < end; i0 += kStepRows, buffer ^= 1, at_lane.other(L::kBytes)) {
                arrive_and_wait();
                if (i0 + kStepRows < end)
                    bring(head, i0 + kStepRows, buffer ^ 1);
                else if (head + 1 < head1)
                    bring(head + 1, first, buffer ^ 1);
                tile_of(i0, buffer, false);
            }
        }
        done = all_finite();
        at_lane = Lane<DP>(lane_again());
        entries = kFinite;
    }
    // Entries of Q and dO that are not finite as zeros in a second walk.  Their rows have a log-sum that the walk by rows
    // has made NaN, and with it P (or minus infinity, and P = 0).
    for (; !done; ++entries) {
        for (int look = Fitted<T>::kFits && entries == kFinite; look >= 0; --look) {
            begin();
            for (int head = head0; head < head1; ++head) {
                to.of_head(p, head);
                const int end = head + 1 < head1 ? last : row1;
                for (int i0 = head == head0 ? row0 : first; i0 < end; i0 += kStepRows) {
                    const int own_lane = lane_again(), own_tid = 64 * wave + own_lane;
                    arrive_and_wait();
                    stage<T, DP, 256, kStepRows>(queries, p.q, head, i0, first, last, p.d, own_tid, entries);
                    stage<T, DP, 256, kStepRows>(grads, p.dO, head, i0, first, last, p.d, own_tid, entries);
                    if (wave < 2 && own_lane < kStepRows) of_rows[0][wave][own_lane] = i0 + own_lane < last ? sums_of(wave, head, i0)[own_lane] : 0.f;
                    arrive_and_wait();
                    tile_of(i0, 0, look);
                }
            }
            if (look) fitted.put_again(most);
        }
        done = entries == kFinite || all_finite();
    }
    if (!see.inside) return;
    // (made again here rather than kept, in registers or beside them, from where it was first needed)
    const int lane_here = lane_again(), half_again = lane_here >> 5;
    const int64_t row = tile * kTileRows + wave * 32 + (lane_here & 31);
    const float times = p.scale * kBack * fitted.back();
    if (p.splits > 1) {
        const int64_t keys = (int64_t)p.mask.m * p.hkv;
        float* const o = p.partial + (2 * part * keys + row * p.hkv + kv) * p.d;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                put4(o, 32 * b + 8 * a + 4 * half_again, p.d, dk[b] * times, 4 * a);
                put4(o + keys * p.d, 32 * b + 8 * a + 4 * half_again, p.d, dv[b] * kBack, 4 * a);
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
                x[e] = dk[b][4 * a + e] * times;
                y[e] = dv[b][4 * a + e] * kBack;
            }
            put4<T>(p.dk.data + row * p.dk.ld + kv * p.dk.hs, 32 * b + 8 * a + 4 * half_again, p.d, p.dk.wide, x);
            put4<T>(p.dv.data + row * p.dv.ld + kv * p.dv.hs, 32 * b + 8 * a + 4 * half_again, p.d, p.dv.wide, y);
        }
}

// dQ of one row and head, or dK and dV of one key and head, from the parts, in ascending order: a wave for each.  One launch for
// both, as it costs 5 us.
template <typename T>
__global__ __launch_bounds__(256) void attn_grad_join_kernel(Problem p, int64_t row_blocks) {
    const int lane = threadIdx.x & 63;
    if (blockIdx.x >= row_blocks) {
        const int64_t keys = (int64_t)p.mask.m * p.hkv, at = ((int64_t)blockIdx.x - row_blocks) * 4 + (threadIdx.x >> 6);
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
        return;
    }
    const int64_t rows = (int64_t)p.hq * p.mask.n, at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (at >= rows) return;
    const int head = (int)(at / p.mask.n), row = (int)(at % p.mask.n);
    if (!keys_of_row(p.mask, row).inside) return;
    for (int c = lane; c < p.d; c += 64) {
        float a = 0.f;
#pragma unroll 8
        for (int s = 0; s < p.row_splits; ++s) a += p.row_partial[(s * rows + at) * p.d + c];
        p.dq.data[row * p.dq.ld + head * p.dq.hs + c] = (unsigned short)T::pack(a, 0.f);
    }
}

template <typename T, int DP, bool LARGE_CAP>
hipError_t launch_kernels(const Problem& p, hipStream_t stream) {
    const int64_t row_tiles = ((int64_t)p.mask.n * (p.hq / p.hkv) + kTileRows - 1) / kTileRows, key_tiles = (p.mask.m + kTileRows - 1) / kTileRows;
    const dim3 block(256);
    if (row_tiles) attn_grad_rows_kernel<T, DP, LARGE_CAP><<<dim3((unsigned)(row_tiles * p.hkv * p.row_splits)), block, 0, stream>>>(p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (key_tiles) attn_grad_keys_kernel<T, DP, LARGE_CAP><<<dim3((unsigned)(key_tiles * p.hkv * p.splits)), block, 0, stream>>>(p);
    e = hipGetLastError();
    const int64_t row_blocks = p.row_splits > 1 ? ((int64_t)p.mask.n * p.hq + 3) / 4 : 0, key_blocks = p.splits > 1 ? ((int64_t)p.mask.m * p.hkv + 3) / 4 : 0;
    if (e != hipSuccess || row_blocks + key_blocks == 0) return e;
    attn_grad_join_kernel<T><<<dim3((unsigned)(row_blocks + key_blocks)), block, 0, stream>>>(p, row_blocks);
    return hipGetLastError();
}

template <typename T, bool LARGE_CAP>
hipError_t launch(const Problem& p, hipStream_t stream) {
    return p.d <= 64   ? launch_kernels<T, 64, LARGE_CAP>(p, stream)
           : p.d <= 96 ? launch_kernels<T, 96, LARGE_CAP>(p, stream)
                       : launch_kernels<T, 128, LARGE_CAP>(p, stream);
}
template <typename T>
hipError_t launch(const Problem& p, hipStream_t stream) {  // (both forms in one kernel would not fit its registers)
    return p.cap > kLargeCap ? launch<T, true>(p, stream) : launch<T, false>(p, stream);
}

}  // namespace

hipError_t launch_grad(const Problem& p, hipStream_t stream) {
    return p.f16 ? launch<F16>(p, stream) : launch<Bf16>(p, stream);
}

}  // namespace attn
