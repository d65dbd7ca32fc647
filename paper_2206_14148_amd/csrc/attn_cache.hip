// Attention over a cache of 8-bit blocks, what writes the cache, and what finds its places.
#include "attn_device.h"

namespace attn {

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// ---- block tables and slots -------------------------------------------------------------------

// Every workgroup sums up the whole batch by itself (a few words a request, from the L2) and then writes its own
// part of the tables and slots: one launch, nothing to wait for.  New blocks are looked up in `free` and not in the
// table, which another workgroup may be writing.
constexpr int kMapThreads = 512;
__global__ __launch_bounds__(kMapThreads) void attn_map_kernel(MapProblem p) {
    extern __shared__ int sums[];  // [batch + 1] new tokens before a request, [batch + 1] new blocks
    int* const tokens = sums;
    int* const blocks = sums + p.batch + 1;
    __shared__ int of_wave[2][kMapThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int most = p.width * p.block;
    auto request = [&](int i, int& before, int& after) {
        after = min(max(p.lengths[i], 0), most);
        before = after - min(max(p.news[i], 0), after);
    };
    // sums of lengths are cut at 2^31 - 1: they only ever grow along the batch, and no place is past its request
    auto plus = [](int a, int b) { return (int)min((unsigned)a + (unsigned)b, (unsigned)INT_MAX); };
    int base_t = 0, base_b = 0;
    for (int i0 = 0; i0 < p.batch; i0 += kMapThreads) {
        const int i = i0 + tid;
        int before = 0, after = 0;
        if (i < p.batch) request(i, before, after);
        int t = after - before, b = (after + p.block - 1) / p.block - (before + p.block - 1) / p.block;
        for (int s = 1; s < 64; s <<= 1) {
            const int x = __shfl_up(t, s), y = __shfl_up(b, s);
            if (lane >= s) {
                t = plus(t, x);
                b = plus(b, y);
            }
        }
        __syncthreads();
        if (lane == 63) {
            of_wave[0][wave] = t;
            of_wave[1][wave] = b;
        }
        __syncthreads();
        // those before this request: of the batch so far, of the waves before, of the lanes before
        t = __shfl_up(t, 1);
        b = __shfl_up(b, 1);
        if (lane == 0) t = b = 0;
        int all_t = base_t, all_b = base_b;
        for (int w = 0; w < kMapThreads / 64; ++w) {
            if (w == wave && i < p.batch) {
                tokens[i] = plus(all_t, t);
                blocks[i] = plus(all_b, b);
            }
            all_t = plus(all_t, of_wave[0][w]);
            all_b = plus(all_b, of_wave[1][w]);
        }
        base_t = all_t;
        base_b = all_b;
    }
    if (tid == 0) {
        tokens[p.batch] = base_t;
        blocks[p.batch] = base_b;
    }
    __syncthreads();
    const int64_t at = (int64_t)blockIdx.x * kMapThreads + tid, step = (int64_t)gridDim.x * kMapThreads;
    for (int64_t i = at; i <= p.batch; i += step) p.starts[i] = tokens[i];
    if (at == 0) *p.used = base_b;
    auto free_block = [&](int64_t i) { return i < p.n_free ? p.free[i] : -1; };
    // new blocks, each by the request whose sum it falls into
    auto owner = [&](const int* of, int64_t x) {  // the last request with of[i] <= x
        int low = 0, high = p.batch;
        while (high - low > 1) {
            const int mid = (low + high) >> 1;
            if (of[mid] <= x)
                low = mid;
            else
                high = mid;
        }
        return low;
    };
    for (int64_t x = at; x < base_b; x += step) {
        const int i = owner(blocks, x);
        int before, after;
        request(i, before, after);
        p.table[(int64_t)i * p.width + (before + p.block - 1) / p.block + (x - blocks[i])] = free_block(x);
    }
    for (int64_t x = at; x < p.n_slots; x += step) {
        int64_t slot = -1;
        if (x < base_t) {
            const int i = owner(tokens, x);
            int before, after;
            request(i, before, after);
            const int j = before + (int)(x - tokens[i]), held = (before + p.block - 1) / p.block, b = j / p.block;
            const int block = b < held ? p.table[(int64_t)i * p.width + b] : free_block(blocks[i] + (int64_t)(b - held));
            if (block >= 0) slot = (int64_t)block * p.block + j % p.block;
        }
        p.slots[x] = slot;
    }
}

// ---- new rows ---------------------------------------------------------------------------------

template <bool E4M3>
__device__ __forceinline__ float value_of(unsigned code) {
    if constexpr (E4M3) return __builtin_amdgcn_cvt_f32_fp8(code, 0);
    return (float)(signed char)code;
}

// The code nearest to y; y is exact or rounded to odd (its last bit says that something was cut off), so that the
// one rounding here is that of the real number.
template <bool E4M3>
__device__ __forceinline__ unsigned code_of(float y) {
    constexpr float kMost = E4M3 ? 448.f : 127.f;
    y = y == y ? fminf(fmaxf(y, -kMost), kMost) : 0.f;
    if constexpr (E4M3) return __builtin_amdgcn_cvt_pk_fp8_f32(y, 0.f, 0, false) & 0xffu;
    return (unsigned)(int)__builtin_rintf(y) & 0xffu;
}

// x / s rounded to odd, by s and 1 / s (a division for each would be three times the instructions).  Both are taken times
// 2^100 where s is so small that 1 / s may be infinite; of s = 0 every quotient is 0.
struct Divisor {
    float s, inverse, times;
    __device__ __forceinline__ explicit Divisor(float s_) {
        times = s_ == 0.f ? 0.f : s_ < 0x1p-100f ? 0x1p100f : 1.f;
        s = s_ == 0.f ? 1.f : s_ * times;
        inverse = 1.f / s;
    }
    __device__ __forceinline__ float operator()(float x) const {
        x *= times;
        float y = x * inverse;
        y = __builtin_fmaf(__builtin_fmaf(-y, s, x), inverse, y);
        const unsigned bits = __float_as_uint(y);
        const float rest = __builtin_fmaf(-y, s, x);  // exact: its sign says on which side of y the quotient lies
        const unsigned odd = (rest < 0.f) == (y < 0.f) ? bits | 1 : bits - 1;
        y = (bits & 1) || rest == 0.f ? y : __uint_as_float(odd);
        return fabsf(x) < kInf ? y : x;
    }
};

// code * from / to likewise
__device__ __forceinline__ float quotient_of(float code, float from, float to) {
    const double y = (double)code * from / to;
    float f = (float)y;
    if (fabs((double)f) > fabs(y)) f = __uint_as_float(__float_as_uint(f) - 1);
    if ((double)f != y) f = __uint_as_float(__float_as_uint(f) | 1);
    return f;
}

// A workgroup looks at `tokens` new rows for one head; where the first row of a run of rows that go to one block is among
// them it does the run.  What bounds it for a step's few rows is one memory access waiting for another: slots, then rows and
// scales, then the codes go out (8 us for one row, 12 for 64 rows and 8 heads, of which a launch is 3).  Blocks of up to 32
// tokens take a wave, whose lanes need not wait for each other (9216 rows of 128, 8 heads, blocks of 16: 34 us, with four
// waves 69), larger ones four (64 rows, blocks of 64: 13 us, with one wave 40; 9216 rows 92).  Rows are kept in registers from the
// search of the largest magnitude to the codes where they fit, else read again.  A block's codes of V lie across its rows, so
// they are put together in LDS and written a word of four tokens at a time; a word that the run fills in part, and that is not
// begun anew, is written byte by byte.
// e4m3 needs few enough registers for a fifth wave on a SIMD (append of 8 prompts of up to 2048 rows, blocks of 64: 135 us with the
// values that are looked at, 144 with four).
constexpr int kAppendPasses = 4;
constexpr int kAhead = 8;  // loads of slots under way together where rows without a place are passed over
template <typename T, bool E4M3, int THREADS>
__global__ __launch_bounds__(THREADS, E4M3 ? 5 : 4) void attn_append_kernel(AppendProblem p, int tokens) {
    const Cache& c = p.cache;
    extern __shared__ __attribute__((aligned(16))) unsigned char turned[];  // [row][block + 4]
    __shared__ int last_of[256];               // the last row of the run that goes to each token, -1: none
    __shared__ int token_of[THREADS];   // of the run's first rows
    __shared__ unsigned covered[8];            // tokens of the block that the run writes
    __shared__ unsigned char moved_to[2][256];  // what becomes of each code that the block holds
    __shared__ float of_wave[2][THREADS / 64];
    __shared__ int run_end, run_last, run_hole;
    const int thread = threadIdx.x;
    const int head = blockIdx.x % c.hkv, shift = __builtin_ctz(c.block), pitch = c.block + 4;
    const int64_t group = (int64_t)(blockIdx.x / c.hkv) * tokens, slots = c.blocks << shift;
    auto block_of = [&](int64_t t) {  // -1: none
        const int64_t s = t >= 0 && t < p.count ? p.slots[t] : -1;
        return s >= 0 && s < slots ? (int)(s >> shift) : -1;
    };
    // lane l of each wave: whether a run begins at row group + l
    const int lane = thread & 63;
    const int mine = lane < tokens ? block_of(group + lane) : -1;
    int before_mine = lane < tokens ? block_of(group + lane - 1) : -1;
    if (__any(mine >= 0 && before_mine < 0 && group + lane > 0)) {
        // Rows without a place are passed over, however many: what counts is the last one before that has one, of this group or of those before.
        const unsigned long long placed = __ballot(mine >= 0);
        int before = -1;
        unsigned long long found = 0;
        for (int64_t t = group - 1; !found && t >= 0; t -= kAhead * 64) {
            int b[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) b[k] = block_of(t - 64 * k - lane);
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (!found) {
                    before = b[k];
                    found = __ballot(before >= 0);
                }
        }
        before = found ? __shfl(before, __builtin_ctzll(found)) : -1;
        const unsigned long long below = placed & ((1ull << lane) - 1);
        before_mine = __shfl(mine, below ? 63 - __builtin_clzll(below) : 0);
        if (!below) before_mine = before;
    }
    unsigned long long firsts = __ballot(mine >= 0 && mine != before_mine);
    const int pieces = c.row / 8, per_pass = THREADS / pieces, piece = thread % pieces, line = thread / pieces;
    while (firsts) {
        int tid = thread;
        asm volatile("" : "+v"(tid));  // (or addresses made of it are kept from run to run: registers)
        const int64_t first = group + __builtin_ctzll(firsts);
        const int block = block_of(first);
        const int64_t at = (int64_t)block * c.hkv + head;
        firsts &= firsts - 1;
        __syncthreads();
        if (tid < 8) covered[tid] = 0;
        if (tid == 0) run_end = run_hole = INT_MAX, run_last = 0;
        for (int i = tid; i < c.block; i += THREADS) last_of[i] = -1;
        const float scales[2] = {c.k_scale[at], c.v_scale[at]};
        __syncthreads();
        // The run goes on to before the first row that has another place; `count` to behind its last row, `hole` is the first row
        // without a place in between.  (Slots may be given twice: it can be longer than a block.)
        int count = 1, hole = INT_MAX;
        bool ended = false;
        for (int from = 0; !ended; from += from ? kAhead * THREADS : THREADS) {
            int b[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) b[k] = k == 0 || from ? block_of(first + from + k * THREADS + tid) : -1;
            if (from == 0) token_of[tid] = b[0] == block ? (int)(p.slots[first + tid] & (c.block - 1)) : -1;
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                if (ended || (k && !from)) continue;
                const int wave_from = from + k * THREADS + (tid & ~63);
                const unsigned long long ends = __ballot(b[k] != block && (b[k] >= 0 || first + wave_from + lane >= p.count));
                int end = ends ? wave_from + __builtin_ctzll(ends) : INT_MAX;
                if constexpr (THREADS > 64) {
                    if (lane == 0 && ends) atomicMin(&run_end, end);
                    __syncthreads();
                    end = run_end;
                }
                const unsigned long long inside = end >= wave_from + 64 ? ~0ull : end <= wave_from ? 0 : (1ull << (end - wave_from)) - 1;
                const unsigned long long own = __ballot(b[k] == block) & inside, none = __ballot(b[k] < 0) & inside;
                if constexpr (THREADS > 64) {
                    if (lane == 0 && own) atomicMax(&run_last, wave_from + 63 - __builtin_clzll(own));
                    if (lane == 0 && none) atomicMin(&run_hole, wave_from + __builtin_ctzll(none));
                    __syncthreads();  // (and before anyone lowers the end again)
                } else {
                    if (own) count = wave_from + 64 - __builtin_clzll(own);
                    if (none && hole == INT_MAX) hole = wave_from + __builtin_ctzll(none);
                }
                ended = end != INT_MAX;
            }
        }
        if constexpr (THREADS > 64) {
            count = run_last + 1;
            hole = run_hole;
        }
        const bool holes = hole < count;
        __syncthreads();
        auto token = [&](int i) {  // -1: none
            return i < THREADS ? token_of[i] : block_of(first + i) == block ? (int)(p.slots[first + i] & (c.block - 1)) : -1;
        };
        u32x4 rows[2][kAppendPasses];
        auto read = [&](int i0) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int n = 0; n < kAppendPasses; ++n) {
                    const int i = i0 + line * kAppendPasses + n;
                    const Rows& r = x ? p.v : p.k;
                    rows[x][n] = u32x4{0, 0, 0, 0};
                    if (i < count) rows[x][n] = entries8(r.data + (first + i) * r.ld + head * r.hs, 8 * piece, c.d, r.wide);
                }
        };
        float a[2] = {0.f, 0.f};
        const int round = kAppendPasses * per_pass;
        for (int i0 = 0; i0 < count; i0 += round) {
            read(i0);
            for (int i = i0 + tid; i < min(i0 + round, count); i += THREADS) {
                const int to = token(i);
                if (to < 0) continue;
                atomicOr(&covered[to >> 5], 1u << (to & 31));
                atomicMax(&last_of[to], i);
            }
            if (holes) {
#pragma unroll
                for (int n = 0; n < kAppendPasses; ++n) {
                    const int i = i0 + line * kAppendPasses + n;
                    if (i < count && token(i) < 0) rows[0][n] = rows[1][n] = u32x4{0, 0, 0, 0};
                }
            }
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int n = 0; n < kAppendPasses; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float low = fabsf(T::low(rows[x][n][e])), high = fabsf(T::high(rows[x][n][e]));
                        a[x] = fmaxf(a[x], fmaxf(low < kInf ? low : 0.f, high < kInf ? high : 0.f));
                    }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            for (int s = 32; s; s >>= 1) a[x] = fmaxf(a[x], __shfl_xor(a[x], s));
            if (tid % 64 == 0) of_wave[x][tid / 64] = a[x];
        }
        __syncthreads();
#pragma unroll
        for (int x = 0; x < 2; ++x)
            for (int w = 0; w < THREADS / 64; ++w) a[x] = fmaxf(a[x], of_wave[x][w]);
        const bool fresh = covered[0] & 1;  // token 0: begun anew
        float after[2];
        bool moves[2];
        for (int x = 0; x < 2; ++x) {
            const float before = fresh ? 0.f : scales[x];
            after[x] = fmaxf(before, a[x] / (E4M3 ? 448.f : 127.f));
            if (tid == 0) (x ? c.v_scale : c.k_scale)[at] = after[x];
            moves[x] = !fresh && after[x] > before;  // codes that the block holds follow its scale
            if (moves[x])
                for (int i = tid; i < 256; i += THREADS)
                    moved_to[x][i] = before > 0.f ? (unsigned char)code_of<E4M3>(quotient_of(value_of<E4M3>(i), before, after[x])) : 0;
        }
        if (moves[0] || moves[1]) {
            __syncthreads();
            for (int x = 0; x < 2; ++x) {
                if (!moves[x]) continue;
                unsigned* const codes = reinterpret_cast<unsigned*>((x ? c.v : c.k) + at * (int64_t)c.block * c.row);
                for (int i = tid; i < c.block * c.row / 4; i += THREADS) {
                    const unsigned w = codes[i];
                    codes[i] = moved_to[x][w & 255] | moved_to[x][w >> 8 & 255] << 8 | moved_to[x][w >> 16 & 255] << 16 |
                               (unsigned)moved_to[x][w >> 24] << 24;
                }
            }
            // other lanes write the new codes into those words: the stores have to be done, not only begun (a fence for
            // the whole device would write the L2 back, 40 us)
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(0);
            __syncthreads();
        }
        const Divisor by[2] = {Divisor(after[0]), Divisor(after[1])};
        unsigned char* const k_codes = c.k + at * (int64_t)c.block * c.row;
        unsigned* const v_codes = reinterpret_cast<unsigned*>(c.v + at * (int64_t)c.block * c.row);
        for (int i0 = 0; i0 < count; i0 += round) {
            if (count > round) read(i0);
            // a thread's four rows mostly go to four tokens in a row
            if (i0 + line * kAppendPasses >= count) continue;
            int to[kAppendPasses];
            u32x2 w[kAppendPasses];
            bool together = true;
#pragma unroll
            for (int n = 0; n < kAppendPasses; ++n) {
                const int i = i0 + line * kAppendPasses + n;
                to[n] = i < count ? token(i) : -1;
                if (to[n] >= 0 && last_of[to[n]] != i) to[n] = -1;  // a slot given twice
                together = together && to[n] >= 0 && to[n] == to[0] + n;
                w[n] = u32x2{0, 0};
                if (to[n] < 0) continue;
                u32x2 k = {0, 0};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const unsigned a = rows[0][n][e / 2], b = rows[1][n][e / 2];
                    k[e / 4] |= code_of<E4M3>(by[0](e & 1 ? T::high(a) : T::low(a))) << (8 * (e % 4));
                    w[n][e / 4] |= code_of<E4M3>(by[1](e & 1 ? T::high(b) : T::low(b))) << (8 * (e % 4));
                }
                *reinterpret_cast<u32x2*>(k_codes + to[n] * c.row + 8 * piece) = k;
            }
            static_assert(kAppendPasses == 4, "");
            if (together && to[0] % 4 == 0) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    unsigned v = 0;
#pragma unroll
                    for (int n = 0; n < 4; ++n) v |= (w[n][e / 4] >> (8 * (e % 4)) & 0xffu) << (8 * n);
                    *reinterpret_cast<unsigned*>(turned + (8 * piece + e) * pitch + to[0]) = v;
                }
            } else {
#pragma unroll
                for (int n = 0; n < 4; ++n)
                    if (to[n] >= 0)
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            turned[(8 * piece + e) * pitch + to[n]] = (unsigned char)(w[n][e / 4] >> (8 * (e % 4)));
            }
        }
        __syncthreads();
        for (int i = tid; i < c.block * c.row / 4; i += THREADS) {
            if (fresh) {
                const int to = 4 * i >> (c.row == 64 ? 6 : 7);
                if (!(covered[to >> 5] >> (to & 31) & 1)) reinterpret_cast<unsigned*>(k_codes)[i] = 0;
            }
            const int to = 4 * i & (c.block - 1), column = 4 * i >> shift;
            const unsigned have = covered[to >> 5] >> (to & 31) & 15u;
            if (!have && !fresh) continue;
            const unsigned word = have ? *reinterpret_cast<const unsigned*>(turned + column * pitch + to) : 0;
            const unsigned mask = (have & 1 ? 0xffu : 0) | (have & 2 ? 0xff00u : 0) | (have & 4 ? 0xff0000u : 0) | (have & 8 ? 0xff000000u : 0);
            if (fresh || have == 15u) {
                v_codes[i] = word & mask;
            } else {
                unsigned char* const bytes = reinterpret_cast<unsigned char*>(v_codes + i);
                for (int b = 0; b < 4; ++b)
                    if (have >> b & 1) bytes[b] = (unsigned char)(word >> (8 * b));
            }
        }
    }
}

// ---- attention over the cache -----------------------------------------------------------------

// Eight codes to an operand of 16-bit numbers; every code is exact in either type.
template <bool E4M3>
__device__ __forceinline__ f16x8 halves_of(u32x2 w) {
    f16x8 r;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        if constexpr (E4M3) {
            const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[e], 1.f, false);
            const f16x2 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[e], 1.f, true);
            r[4 * e] = a[0], r[4 * e + 1] = a[1], r[4 * e + 2] = b[0], r[4 * e + 3] = b[1];
        } else {
            // c + 128 below the byte 0x64 is 1024 + 128 + c in f16, exactly
            const unsigned u = w[e] ^ 0x80808080u;
            const f16x2 less = {(_Float16)-1152.f, (_Float16)-1152.f};
            const f16x2 a = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x07010700u)) + less;
            const f16x2 b = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, u, 0x07030702u)) + less;
            r[4 * e] = a[0], r[4 * e + 1] = a[1], r[4 * e + 2] = b[0], r[4 * e + 3] = b[1];
        }
    }
    return r;
}
template <typename T, bool E4M3>
__device__ __forceinline__ f32x4 codes_mfma(u32x2 w, s16x8 q, f32x4 c) {
    if constexpr (T::kOne == F16::kOne) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(halves_of<E4M3>(w), __builtin_bit_cast(f16x8, q), c, 0, 0, 0);
    } else {
        bf16x8 r;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            if constexpr (E4M3) {
                const Bf16::v2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[e], 1.f, false);
                const Bf16::v2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[e], 1.f, true);
                r[4 * e] = a[0], r[4 * e + 1] = a[1], r[4 * e + 2] = b[0], r[4 * e + 3] = b[1];
            } else {
#pragma unroll
                for (int b = 0; b < 4; ++b) r[4 * e + b] = (__bf16)(float)(signed char)(w[e] >> (8 * b));
            }
        }
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(r, __builtin_bit_cast(bf16x8, q), c, 0, 0, 0);
    }
}

// A wave takes 64 tokens at a time, and 16 SETS rows: those of the heads that share a K and V, and of the nq rows.
// Codes go from memory to registers in the order in which v_mfma_f32_16x16x32 takes them: lane l of a product has
// column l % 16 (a row) and rows 4 (l / 16) + r.  K: operand row i of product t is token 16 (i / 4) + 4 t + i % 4, so
// that the lanes of group g = l / 16 get the scores of tokens 16 g .. 16 g + 15, which lie in one block; a lane reads
// its quarter of a token's row.  V: a lane reads one entry's tokens 16 g .. 16 g + 15, 16 bytes, and its scores,
// rounded, are the other operand as they are.  Nothing goes through LDS until the four waves' sums meet.  Bound by reading the
// codes: 200003 tokens of 8 heads of 128 in 87 us, 4.7 TB/s with the join, as fast as a large copy here; 64 requests of 512 to
// 8192 tokens in 134 us, 4.2 TB/s: the last workgroups end one after the other.
template <typename T, bool E4M3, int ROW, int SETS>
__global__ __launch_bounds__(256) void attn_cache_kernel(CacheProblem p) {
    constexpr int kSteps = ROW / 32, kTiles = ROW / 16;
    __shared__ float of_waves[4][16 * SETS][ROW + 4];
    __shared__ float ends[4][16 * SETS][2];
    const Cache& c = p.cache;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, g = lane >> 4, col = lane & 15;
    const int group = p.hq / c.hkv, rows = p.nq * group, row_sets = (rows + 16 * SETS - 1) / (16 * SETS);
    // Heads go round first: the eight XCDs take workgroups in turn, so each gets its share of every request (in runs of
    // requests the longest ones made some XCDs work half as long again as others).
    const int w = blockIdx.x, head = w % c.hkv, set = w / c.hkv % row_sets, b = w / c.hkv / row_sets % p.batch;
    const int range = w / c.hkv / row_sets / p.batch;
    const int length = min(max(p.lengths[b], 0), p.width * c.block);
    const int begin = range * p.range_tokens, end = min(length, begin + p.range_tokens);
    // (of an empty request the first range writes the rows)
    if (begin >= length && range > 0) return;
    const int* const table = p.table + (int64_t)b * p.width;

    s16x8 q[SETS][kSteps];
    int hi[SETS];       // a row sees tokens below this
    float slope[SETS];
#pragma unroll
    for (int s = 0; s < SETS; ++s) {
        const int r = (set * SETS + s) * 16 + col, t = r / group, h = head * group + r % group;
        hi[s] = r < rows ? length - p.nq + t + 1 : 0;
        slope[s] = p.slopes && r < rows ? p.slopes[h] * kLog2e : 0.f;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            u32x4 v = {0, 0, 0, 0};
            if (r < rows)
                v = entries8(p.q.data + ((int64_t)b * p.nq + t) * p.q.ld + h * p.q.hs, g * (ROW / 4) + 8 * k, c.d, p.q.wide);
            q[s][k] = __builtin_bit_cast(s16x8, v);
        }
    }
    const float to_cap = p.cap > 0.f ? (p.cap > kLargeCap ? 1.f : 2.f * kLog2e) * p.scale / p.cap : 0.f, from_cap = p.cap * kLog2e;
    const int seen_by_all = length - p.nq + 1;  // tokens below this are seen by every row

    f32x4 sum[SETS][kTiles];
    float top[SETS], total[SETS];
#pragma unroll
    for (int s = 0; s < SETS; ++s) {
        top[s] = -kInf;
        total[s] = 0.f;
#pragma unroll
        for (int t = 0; t < kTiles; ++t) sum[s][t] = f32x4{};
    }
    const int64_t block_bytes = (int64_t)c.block * ROW;
    auto block_at = [&](int j) {  // the block that holds token j, or -1
        const int x = j < end ? table[j / c.block] : -1;
        return x >= 0 && x < c.blocks ? x : -1;
    };
    for (int j0 = begin + 64 * wave; j0 < end; j0 += 256) {
        // this lane's token of K: 16 (col / 4) + 4 t + col % 4; of V and of the scores: 16 g + ...
        const int jk = j0 + 16 * (col >> 2), jv = j0 + 16 * g;
        const int bk = block_at(jk), bv = block_at(jv);
        const bool whole = j0 + 64 <= seen_by_all && j0 + 64 <= end && !__any(bv < 0);
        u32x4 kc[4][ROW / 64], vc[kTiles];
        const unsigned char* kp = c.k + (bk * (int64_t)c.hkv + head) * block_bytes + ((jk + (col & 3)) % c.block) * ROW + g * (ROW / 4);
        const unsigned char* vp = c.v + (bv * (int64_t)c.hkv + head) * block_bytes + col * c.block + jv % c.block;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < ROW / 64; ++e)
                kc[t][e] = bk >= 0 ? *reinterpret_cast<const u32x4*>(kp + 4 * t * ROW + 16 * e) : u32x4{0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
            vc[t] = bv >= 0 ? *reinterpret_cast<const u32x4*>(vp + 16 * t * c.block) : u32x4{0, 0, 0, 0};
        const float ks = bv >= 0 ? c.k_scale[bv * (int64_t)c.hkv + head] : 0.f;
        const float vs = bv >= 0 ? c.v_scale[bv * (int64_t)c.hkv + head] : 0.f;
        if (!whole && jv + 16 > end) {
            // codes behind the last token may be anything, NaN among it
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int left = end - jv - 4 * e;  // tokens of this word
                    vc[t][e] &= left >= 4 ? ~0u : left <= 0 ? 0u : ~0u >> (8 * (4 - left));
                }
        }
        float vmost = fmaxf(vs, __shfl_xor(vs, 16));
        vmost = fmaxf(vmost, __shfl_xor(vmost, 32));
        // A weight is at most one.  As an operand it comes times its block's scale over the largest of these tokens', and times 2^14:
        // down to 2^-28 of weight and scales together an f16 keeps all its bits.
        const float share = vmost > 0.f ? vs / vmost * 0x1p14f : 0.f;
#pragma unroll
        for (int s = 0; s < SETS; ++s) {
            f32x4 x[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                x[t] = f32x4{};
#pragma unroll
                for (int k = 0; k < kSteps; ++k)
                    x[t] = codes_mfma<T, E4M3>(u32x2{kc[t][k / 2][2 * (k % 2)], kc[t][k / 2][2 * (k % 2) + 1]}, q[s][k], x[t]);
            }
            const float factor = p.scale * kLog2e * ks;
            if (p.cap > kLargeCap) {
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[t][e] = from_cap * tanh_of(to_cap * ks * x[t][e]);
            } else if (p.cap > 0.f) {
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        x[t][e] = from_cap * __builtin_fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(to_cap * ks * x[t][e])), 1.f);
            } else {
#pragma unroll
                for (int t = 0; t < 4; ++t) x[t] *= factor;
            }
            if (p.slopes) {
                const float away = (float)(hi[s] - 1 - jv);
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[t][e] = __builtin_fmaf(-slope[s], away - (float)(4 * t + e), x[t][e]);
            }
            if (!whole) {
                const int left = bv >= 0 ? min(hi[s], end) - jv : 0;
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (4 * t + e >= left) x[t][e] = -kInf;
            }
            float most = x[0][0];
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) most = fmaxf(most, x[t][e]);
            most = fmaxf(most, __shfl_xor(most, 16));
            most = fmaxf(most, __shfl_xor(most, 32));
            if (__any(most > top[s])) {
                const float now = fmaxf(top[s], most), shrink = top[s] == now ? 1.f : __builtin_amdgcn_exp2f(top[s] - now);
                top[s] = now;
                total[s] *= shrink;
#pragma unroll
                for (int t = 0; t < kTiles; ++t) sum[s][t] *= shrink;
            }
            const float base = top[s] == -kInf ? 0.f : top[s];
            float part;  // (16 are added up before they meet what may be much larger)
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[t][e] = __builtin_amdgcn_exp2f(x[t][e] - base);
                    part = t + e ? part + x[t][e] : x[t][e];
                }
            total[s] += part;
            f16x8 weights[2];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 8; ++e) weights[u][e] = (_Float16)(x[2 * u + e / 4][e % 4] * share);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                f32x4 y{};
                y = __builtin_amdgcn_mfma_f32_16x16x32_f16(halves_of<E4M3>(u32x2{vc[t][0], vc[t][1]}), weights[0], y, 0, 0, 0);
                y = __builtin_amdgcn_mfma_f32_16x16x32_f16(halves_of<E4M3>(u32x2{vc[t][2], vc[t][3]}), weights[1], y, 0, 0, 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[s][t][e] = __builtin_fmaf(y[e] * 0x1p-14f, vmost, sum[s][t][e]);
            }
        }
    }
    // the four waves' sums, in their order
#pragma unroll
    for (int s = 0; s < SETS; ++s) {
        total[s] += __shfl_xor(total[s], 16);
        total[s] += __shfl_xor(total[s], 32);
        if (g == 0) {
            ends[wave][16 * s + col][0] = top[s];
            ends[wave][16 * s + col][1] = total[s];
        }
#pragma unroll
        for (int t = 0; t < kTiles; ++t) *reinterpret_cast<f32x4*>(&of_waves[wave][16 * s + col][16 * t + 4 * g]) = sum[s][t];
    }
    __syncthreads();
    const int64_t all = (int64_t)p.batch * c.hkv * rows;
    for (int i = tid; i < 16 * SETS * ROW; i += 256) {
        const int r = i / ROW, d = i % ROW, row = set * 16 * SETS + r;
        if (row >= rows || d >= c.d) continue;
        float most = -kInf, whole = 0.f, y = 0.f;
        for (int x = 0; x < 4; ++x) most = fmaxf(most, ends[x][r][0]);
        const float base = most == -kInf ? 0.f : most;
        for (int x = 0; x < 4; ++x) {
            const float f = __builtin_amdgcn_exp2f(ends[x][r][0] - base);
            whole = __builtin_fmaf(ends[x][r][1], f, whole);
            y = __builtin_fmaf(of_waves[x][r][d], f, y);
        }
        if (p.ranges > 1) {
            const int64_t at = ((int64_t)b * c.hkv + head) * rows + row;
            p.partial[(range * all + at) * c.d + d] = y;
            if (d == 0) {
                float* const e = p.partial + p.ranges * all * c.d + 2 * (range * all + at);
                e[0] = most;
                e[1] = whole;
            }
        } else {
            unsigned short* const o = p.o.data + ((int64_t)b * p.nq + row / group) * p.o.ld + (head * group + row % group) * p.o.hs;
            o[d] = (unsigned short)T::pack(whole == 0.f ? 0.f : y / whole, 0.f);
        }
    }
}

// The ranges' sums of one row in ascending order: a wave for each.
template <typename T>
__global__ __launch_bounds__(256) void attn_cache_join_kernel(CacheProblem p) {
    const Cache& c = p.cache;
    const int lane = threadIdx.x & 63, group = p.hq / c.hkv, rows = p.nq * group;
    const int64_t all = (int64_t)p.batch * c.hkv * rows, at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (at >= all) return;
    const int row = (int)(at % rows), head = (int)(at / rows % c.hkv), b = (int)(at / rows / c.hkv);
    const int length = min(max(p.lengths[b], 0), p.width * c.block);
    const int ranges = max(1, (length + p.range_tokens - 1) / p.range_tokens);
    const Joined r = join_ranges<1>(p.partial, p.ranges, ranges, all, at, c.d, lane, 0);
    unsigned short* const o = p.o.data + ((int64_t)b * p.nq + row / group) * p.o.ld + (head * group + row % group) * p.o.hs;
    for (int e = 0; e < 2; ++e)
        if (64 * e + lane < c.d) o[64 * e + lane] = (unsigned short)T::pack(r.total == 0.f ? 0.f : r.x[e] / r.total, 0.f);
}

template <typename T, bool E4M3, int ROW>
hipError_t launch(const CacheProblem& p, hipStream_t stream) {
    const int group = p.hq / p.cache.hkv, rows = p.nq * group;
    const int sets = rows > 16 ? 2 : 1;
    const int64_t workgroups = (int64_t)p.batch * p.cache.hkv * ((rows + 16 * sets - 1) / (16 * sets)) * p.ranges;
    if (sets == 1)
        attn_cache_kernel<T, E4M3, ROW, 1><<<dim3((unsigned)workgroups), dim3(256), 0, stream>>>(p);
    else
        attn_cache_kernel<T, E4M3, ROW, 2><<<dim3((unsigned)workgroups), dim3(256), 0, stream>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.ranges == 1) return e;
    const int64_t all = (int64_t)p.batch * p.cache.hkv * rows;
    attn_cache_join_kernel<T><<<dim3((unsigned)((all + 3) / 4)), dim3(256), 0, stream>>>(p);
    return hipGetLastError();
}
template <typename T>
hipError_t launch(const CacheProblem& p, hipStream_t stream) {
    if (p.cache.row == 64) return p.cache.e4m3 ? launch<T, true, 64>(p, stream) : launch<T, false, 64>(p, stream);
    return p.cache.e4m3 ? launch<T, true, 128>(p, stream) : launch<T, false, 128>(p, stream);
}

}  // namespace

hipError_t launch_map(const MapProblem& p, hipStream_t stream) {
    const size_t lds = 2 * ((size_t)p.batch + 1) * 4;
    if (lds > 48 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(attn_map_kernel),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    const int64_t work = p.n_slots > p.batch + 1 ? p.n_slots : p.batch + 1;
    int64_t grid = (work + kMapThreads - 1) / kMapThreads;
    if (grid > 256) grid = 256;
    attn_map_kernel<<<dim3((unsigned)grid), dim3(kMapThreads), lds, stream>>>(p);
    return hipGetLastError();
}

namespace {
template <int THREADS>
hipError_t append_in(const AppendProblem& p, int tokens, hipStream_t stream) {
    const dim3 grid((unsigned)((p.count + tokens - 1) / tokens * p.cache.hkv)), block(THREADS);
    const size_t lds = (size_t)p.cache.row * (p.cache.block + 4);
    auto kernel = p.f16 ? (p.cache.e4m3 ? attn_append_kernel<F16, true, THREADS> : attn_append_kernel<F16, false, THREADS>)
                        : (p.cache.e4m3 ? attn_append_kernel<Bf16, true, THREADS> : attn_append_kernel<Bf16, false, THREADS>);
    kernel<<<grid, block, lds, stream>>>(p, tokens);
    return hipGetLastError();
}
}  // namespace

hipError_t launch_append(const AppendProblem& p, hipStream_t stream) {
    // A step's few rows each go to a block of their own: a workgroup for each row and head.  Of many rows most go where the row
    // before went, and a workgroup looks at up to as many as the smallest block holds: fewer that find nothing to do.
    const int64_t all = p.count * p.cache.hkv;
    const int tokens = all <= 4096 ? 1 : all <= 32768 ? 4 : 16;
    return p.cache.block <= 32 ? append_in<64>(p, tokens, stream) : append_in<256>(p, tokens, stream);
}

hipError_t launch_cache(const CacheProblem& p, hipStream_t stream) {
    return p.f16 ? launch<F16>(p, stream) : launch<Bf16>(p, stream);
}

}  // namespace attn
