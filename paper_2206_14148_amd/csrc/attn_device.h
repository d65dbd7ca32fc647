// Device-side helpers shared by the gfx950 attention kernels: matrix-core operands, tiles of 64 rows in
// LDS, and the interval of keys (or rows) that a row (or key) sees.  Unnamed namespace: each translation
// unit has its own copy.
//
// The layouts all follow from one choice.  v_mfma_f32_32x32x16 gives lane l of a 32 x 32 product the column
// l % 32 and the rows 8 a + 4 (l / 32) + b (a, b = 0 .. 3, register 4 a + b), and takes from it, of its
// second operand, column l % 32 and eight of sixteen values of k.  Which eight is free as long as both
// operands agree.  So the transposed scores (keys x rows) are made, a lane holds sixteen scores of ONE row
// (the softmax is within a lane, and one exchange with lane ^ 32), and its registers 8 s .. 8 s + 7 are,
// rounded, the second operand of the next product over keys 16 s + 8 e + 4 (l / 32) + b, without any move.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "attn_kernels.h"

// Products and sums are fused only where it is written: a score that is rounded once for the maximum and left
// unrounded for the exponential is off by 2^-24 of itself there, however large it is.
#pragma clang fp contract(off)

namespace attn {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_huge_valf();

struct Bf16 {
    typedef __bf16 v8 __attribute__((ext_vector_type(8)));
    typedef __bf16 v2 __attribute__((ext_vector_type(2)));
    static constexpr unsigned kExponents = 0x7f807f80u, kOne = 0x3f80u;
    static __device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ unsigned pack(float x, float y) {  // to nearest even
        v2 r;
        r[0] = (__bf16)x;
        r[1] = (__bf16)y;
        return __builtin_bit_cast(unsigned, r);
    }
    static __device__ __forceinline__ float low(unsigned w) { return __uint_as_float(w << 16); }
    static __device__ __forceinline__ float high(unsigned w) { return __uint_as_float(w & 0xffff0000u); }
};

struct F16 {
    typedef _Float16 v8 __attribute__((ext_vector_type(8)));
    typedef _Float16 v2 __attribute__((ext_vector_type(2)));
    static constexpr unsigned kExponents = 0x7c007c00u, kOne = 0x3c00u;
    static __device__ __forceinline__ f32x16 mfma(s16x8 a, s16x8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ unsigned pack(float x, float y) {
        v2 r;
        r[0] = (_Float16)x;
        r[1] = (_Float16)y;
        return __builtin_bit_cast(unsigned, r);
    }
    static __device__ __forceinline__ float low(unsigned w) { return (float)__builtin_bit_cast(v2, w)[0]; }
    static __device__ __forceinline__ float high(unsigned w) { return (float)__builtin_bit_cast(v2, w)[1]; }
};

// Caps.  1 - 2 / (1 + exp(2 z)) is off by some 2^-23 however small its tanh(z) is, so a score by 2^-23 of the cap: up to kLargeCap
// that is less than 1e-5.  Beyond it a z below 1/2 has its series instead, which is off by steps of 2^-24 of the score itself
// (tanh z = z - z^3 / 3 + 2 z^5 / 15 - ...; what is left out behind z^15 is below 2^-26 of it).  Both are made for every
// score, twelve instructions more.  8000 rows, 16 heads, d = 64, f16: 210 us without a cap, 316 with 50, 488 with 65; gradient of
// 4096 rows, 32 heads on 8, d = 128, bf16, causal: 542, 652, 756; the cache's 200003 tokens, 32 heads on 8: 88, 87, 88.
constexpr float kLargeCap = 64.f;
__device__ __forceinline__ float tanh_of(float z) {
    constexpr float c[] = {1.f, -1.f / 3.f, 2.f / 15.f, -17.f / 315.f, 62.f / 2835.f, -1382.f / 155925.f, 21844.f / 6081075.f,
                           -929569.f / 638512875.f};
    const float w = z * z;
    float series = c[7];
#pragma unroll
    for (int i = 6; i >= 0; --i) series = __builtin_fmaf(series, w, c[i]);
    const float far = __builtin_fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(2.f * kLog2e * z)), 1.f);
    return fabsf(z) < 0.5f ? z * series : far;
}

// what lane ^ 32 holds, combined with one's own
__device__ __forceinline__ u32x2 both_halves(float v) {
    return __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
}
__device__ __forceinline__ float max_of_halves(float v) {
    const u32x2 r = both_halves(v);
    return fmaxf(__uint_as_float(r.x), __uint_as_float(r.y));
}
__device__ __forceinline__ float sum_of_halves(float v) {
    const u32x2 r = both_halves(v);
    return __uint_as_float(r.x) + __uint_as_float(r.y);
}

// smallest or largest over the wave of a value that is the same in lane l and lane l ^ 32
__device__ __forceinline__ int wave_least(int v) {
    for (int s = 16; s; s >>= 1) v = min(v, __shfl_xor(v, s));
    return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int wave_most(int v) {
    for (int s = 16; s; s >>= 1) v = max(v, __shfl_xor(v, s));
    return __builtin_amdgcn_readfirstlane(v);
}

// The lane's number made anew, for what comes behind a walk: no register keeps it, or threadIdx, meanwhile.
__device__ __forceinline__ int lane_again() {
    int lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    asm volatile("" : "+v"(lane));
    return lane;
}

// ---- documents --------------------------------------------------------------------------------

// The document that holds x, by its starts: the last one that begins at or before x; -1 if x lies outside all.
__device__ __forceinline__ int document_of(const int* starts, int docs, int x) {
    if (x < starts[0] || x >= starts[docs]) return -1;
    int low = 0, high = docs;  // starts[low] <= x < starts[high]
    while (high - low > 1) {
        const int mid = (low + high) >> 1;
        if (starts[mid] <= x)
            low = mid;
        else
            high = mid;
    }
    return low;
}

// The arrays in LDS where there are few documents, so that the searches, every step of which waits for the one before,
// do not go to memory (some 4 us a kernel).  All threads of the workgroup, which wait for each other here.
constexpr int kLocalDocs = 127;
struct LocalDocs {
    int starts[kLocalDocs + 1], k_starts[kLocalDocs + 1], prefix[kLocalDocs + 1];
};
__device__ __forceinline__ Mask with_local(const Mask& k, LocalDocs& local, int tid) {
    Mask m = k;
    if (k.docs > kLocalDocs || !(k.starts || k.prefix)) return m;
    if (tid <= k.docs) {
        if (k.starts) {
            local.starts[tid] = k.starts[tid];
            local.k_starts[tid] = k.k_starts[tid];
        }
        if (k.prefix && tid < k.docs) local.prefix[tid] = k.prefix[tid];
    }
    __syncthreads();
    if (k.starts) {
        m.starts = local.starts;
        m.k_starts = local.k_starts;
    }
    if (k.prefix) m.prefix = local.prefix;
    return m;
}

__device__ __forceinline__ int clamp_to(int64_t x, int low, int high) {
    return x < low ? low : x > high ? high : (int)x;
}

struct Document {
    int qs, qe, ks, ke, prefix;
    int64_t shift;  // row i stands at key i + shift
};
// (clamped: whatever the arrays hold, rows stay within 0 .. n and keys within 0 .. m)
__device__ __forceinline__ Document document(const Mask& k, int c) {
    Document e{0, k.n, 0, k.m, 0, 0};
    int64_t last = k.n;
    int64_t first = 0;
    if (k.starts) {
        first = k.starts[c];
        last = k.starts[c + 1];
        e.qs = clamp_to(first, 0, k.n);
        e.qe = clamp_to(last, e.qs, k.n);
        e.ks = clamp_to(k.k_starts[c], 0, k.m);
        e.ke = clamp_to(k.k_starts[c + 1], e.ks, k.m);
    }
    if (k.prefix) e.prefix = max(k.prefix[c], 0);
    e.shift = (int64_t)e.ke - last;
    return e;
}

// What a row sees: keys lo .. hi - 1; it stands at key `at`.
struct Span {
    int lo, hi, at, inside;
};
__device__ __forceinline__ Span keys_of_row(const Mask& k, int i) {
    Span s{0, 0, 0, 0};
    if (i >= k.n) return s;
    const int c = k.starts ? document_of(k.starts, k.docs, i) : 0;
    if (c < 0) return s;
    const Document e = document(k, c);
    const int64_t at = i + e.shift;
    s.inside = 1;
    s.at = (int)at;
    s.lo = e.ks;
    s.hi = k.causal ? clamp_to(max(at + 1, (int64_t)e.ks + e.prefix), e.ks, e.ke) : e.ke;
    return s;
}
// Which rows see a key: lo .. hi - 1; row i stands at key i + at.
__device__ __forceinline__ Span rows_of_key(const Mask& k, int j) {
    Span s{0, 0, 0, 0};
    if (j >= k.m) return s;
    const int c = k.starts ? document_of(k.k_starts, k.docs, j) : 0;
    if (c < 0) return s;
    const Document e = document(k, c);
    s.inside = 1;
    s.at = (int)e.shift;
    s.hi = e.qe;
    s.lo = k.causal && (int64_t)j >= (int64_t)e.ks + e.prefix ? clamp_to(j - e.shift, e.qs, e.qe) : e.qs;
    return s;
}

// ---- tiles in LDS -----------------------------------------------------------------------------

// ROWS rows of DP entries (d rounded up; zeros behind d), row-major, a row 128 or 256 bytes.  Two readers: a
// lane reads 16 bytes of row l % 32 (32 rows apart by whole rows: all in the same banks), and 16 lanes read
// 32 bytes of each of 4 consecutive rows.  The 16-byte pieces of a row are therefore permuted by an exclusive-or
// with bits of the row's number, (r1 r0 r2) below and r3 above: any eight rows in a run have different pieces, and
// any four different pairs of pieces.
template <int DP, int ROWS = kTileKeys>
struct Tile {
    static constexpr int kPieces = DP <= 64 ? 8 : 16;  // of 16 bytes, in a row
    static constexpr int kRowBytes = 16 * kPieces;
    static constexpr int kBytes = ROWS * kRowBytes;
    static __device__ __forceinline__ int turn(int row) {
        const int t = ((row & 3) << 1) | ((row >> 2) & 1);
        return kPieces == 16 ? t | (row & 8) : t;
    }
};

// Eight entries from column c on, those at or behind d zero.
__device__ __forceinline__ u32x4 entries8(const unsigned short* p, int c, int d, int wide) {
    u32x4 r = {0, 0, 0, 0};
    if (wide) {
        if (c < d) r = *reinterpret_cast<const u32x4*>(p + c);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < d) r[e >> 1] |= (unsigned)p[c + e] << (16 * (e & 1));
    }
    return r;
}

// What a pass makes of entries that are not finite, before they meet weights that may be zero (see the kernels).
enum Entries { kAsTheyAre = 0, kFinite = 1, kUp = 2, kDown = 3 };  // kUp, kDown: 1 for +infinity (-infinity) or NaN, else 0

template <typename T>
__device__ __forceinline__ unsigned chosen(unsigned w, int entries) {
    constexpr unsigned kExp = T::kExponents & 0xffffu;
    unsigned r = 0;
#pragma unroll
    for (int s = 0; s < 32; s += 16) {
        const unsigned v = (w >> s) & 0xffffu;
        const bool finite = (v & kExp) != kExp, none = !finite && (v & 0x7fffu) != kExp;
        if (entries == kFinite)
            r |= finite ? v << s : 0;
        else if (!finite && (none || (v >> 15) == (entries == kDown)))
            r |= T::kOne << s;
    }
    return r;
}

// Rows first .. first + ROWS - 1 of one head into LDS; those outside lo .. hi - 1 become zeros.
template <typename T, int DP, int THREADS, int ROWS = kTileKeys>
__device__ __forceinline__ void stage(unsigned char* lds, const Rows& t, int head, int first, int lo, int hi, int d, int tid,
                                      int entries) {
    typedef Tile<DP> L;
    const unsigned short* base = t.data + head * t.hs;
#pragma unroll 1  // (registers)
    for (int it = 0; it < ROWS * L::kPieces / THREADS; ++it) {
        const int at = it * THREADS + tid, r = at / L::kPieces, piece = (at % L::kPieces) ^ L::turn(r);
        const int row = first + r;
        u32x4 v = {0, 0, 0, 0};
        if (row >= lo && row < hi) v = entries8(base + row * t.ld, 8 * piece, d, t.wide);
        if (entries != kAsTheyAre)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = chosen<T>(v[e], entries);
        *reinterpret_cast<u32x4*>(lds + at * 16) = v;
    }
}

// The same without registers in between (t.wide only): 16 bytes a lane, counted by vmcnt; the caller waits with
// arrive_and_wait.  A lane whose piece lies outside rows or entries reads beyond the descriptor's end, which gives zeros.
// A thread's piece is the same in every round (THREADS / kPieces is a multiple of the rows that the turn goes by).
template <int DP, int THREADS, int ROWS = kTileKeys>
struct Direct {
    typedef Tile<DP> L;
    static constexpr int kRows = THREADS / L::kPieces, kRounds = ROWS / kRows;
    static_assert(kRows % L::kPieces == 0 && ROWS % kRows == 0, "");
    uint64_t base;
    unsigned offset;  // of this thread's piece; behind d: beyond the end
    int stride;       // of a row, bytes
    __device__ __forceinline__ Direct(const Rows& t, int head, int d, int tid) {
        const int r = tid / L::kPieces, piece = (tid % L::kPieces) ^ L::turn(r);
        base = reinterpret_cast<uint64_t>(t.data + head * t.hs);
        stride = (int)t.ld * 2;
        offset = 8 * piece < d ? r * stride + 16 * piece : 0x80000000u;
    }
    __device__ __forceinline__ void fetch(const unsigned char* lds, int first, int lo, int hi, int tid) const {
        const uint64_t from = base + (uint64_t)first * stride;
        i32x4 words;
        words[0] = __builtin_amdgcn_readfirstlane((int)from);
        words[1] = __builtin_amdgcn_readfirstlane((int)(from >> 32) & 0xffff);
        words[2] = 0x7fffffff;
        words[3] = 0x00027000;
        const unsigned at = (unsigned)(uintptr_t)(__attribute__((address_space(3))) const unsigned char*)lds;
        const int row = first + tid / L::kPieces;
#pragma unroll
        for (int it = 0; it < kRounds; ++it) {
            const bool in = row + it * kRows >= lo && row + it * kRows < hi;
            const unsigned m = __builtin_amdgcn_readfirstlane(at + (it * THREADS + (tid & ~63)) * 16);
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(m),
                         "v"(in ? offset : 0x80000000u), "s"(words), "s"(it * kRows * stride)
                         : "memory", "m0");
        }
    }
};
// A word for each lane that calls likewise; zeros from `count` on.
__device__ __forceinline__ void fetch_words(const float* lds, const float* from, int lane, int count) {
    const uint64_t base = reinterpret_cast<uint64_t>(from);
    i32x4 words;
    words[0] = __builtin_amdgcn_readfirstlane((int)base);
    words[1] = __builtin_amdgcn_readfirstlane((int)(base >> 32) & 0xffff);
    words[2] = 0x7fffffff;
    words[3] = 0x00027000;
    const unsigned m =
        __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) const float*)lds);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(m),
                 "v"(lane < count ? 4u * lane : 0x80000000u), "s"(words)
                 : "memory", "m0");
}
// This wave's loads are in and its reads of LDS done, then all waves'.  (Built-ins, so that the compiler knows what
// has arrived: it would wait for the loads of the rows again in every round, and with them for the tiles under way.)
__device__ __forceinline__ void arrive_and_wait() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Where a lane reads its operands, from the tile's start.  (A power of two's worth of pieces a row: the piece's
// number and the turn meet in an exclusive-or, which takes what is the same for all lanes last.)
template <int DP>
struct Lane {
    typedef Tile<DP> L;
    unsigned rows, columns;
    __device__ __forceinline__ explicit Lane(int lane) {
        const int half = lane >> 5, r = lane & 31;
        rows = r * L::kRowBytes + (half ^ L::turn(r)) * 16;
        const int b = (lane >> 2) & 3, c = 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
        columns = (4 * half + b) * L::kRowBytes + (c ^ L::turn(4 * half + b)) * 16 + (lane & 1) * 8;
    }
    __device__ __forceinline__ void other(unsigned bytes) {  // the tile that many bytes away, a power of two, in either direction
        rows ^= bytes;
        columns ^= bytes;
    }
    // First operand, rows as they are: row 32 part + l % 32 of the tile, entries 16 step + 8 (l / 32) ...
    __device__ __forceinline__ s16x8 row(const unsigned char* lds, int part, int step) const {
        return *reinterpret_cast<const s16x8*>(lds + (rows ^ (32 * step)) + 32 * part * L::kRowBytes);
    }
    // First operand, turned: column 32 block + l % 32 of the tile, rows 16 step + 8 e + 4 (l / 32) + b.  The
    // transposing read gives lane i of 16 the i-th of the 16 entries that lanes 4 b .. 4 b + 3 hold, b = 0 .. 3.
    __device__ __forceinline__ s16x8 column(const unsigned char* lds, int block, int step) const {
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        s16x4 part[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const unsigned char* p = lds + (columns ^ (64 * block ^ (L::turn(8 * e) * 16))) + (16 * step + 8 * e) * L::kRowBytes;
            part[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
        }
        return __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

// Second operand from 16 numbers of a 32 x 32 product: registers 8 step .. 8 step + 7.
template <typename T>
__device__ __forceinline__ s16x8 rounded_operand(const f32x16& x, int step) {
    u32x4 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = T::pack(x[8 * step + 2 * e], x[8 * step + 2 * e + 1]);
    return __builtin_bit_cast(s16x8, r);
}

// Which K and V head a workgroup has, and which of the `each` pieces of its work, of `heads` * `each` workgroups.  They go round the
// eight XCDs.  As many heads as that gives every XCD the same number of go to one XCD each, and its L2; those left over are dealt out
// piece by piece, so that every XCD has long and short walks of them.  Causal, bf16, 16384 rows of 8 heads on 2, d = 128, forward and
// gradient: 610 and 1851 us (in runs, where two XCDs have all the long walks, 873 and 2860); 5000 rows of 20 heads, d = 96:
// 133 and 425 us (159 and 526); without a mask, and with 8 heads, as fast as in runs.
struct Work {
    int kv, piece;
};
__device__ __forceinline__ Work work_of(int id, int heads, int each) {
    const int left = heads % 8;
    if (id < left * each) return {heads - left + id % left, id / left};
    id -= left * each;
    return {id % 8 * (heads / 8) + id / 8 / each, id / 8 % each};
}

// Four entries c .. c + 3 of a row to memory.
template <typename T>
__device__ __forceinline__ void put4(unsigned short* p, int c, int d, int wide, const float* x) {
    const unsigned a = T::pack(x[0], x[1]), b = T::pack(x[2], x[3]);
    if (wide) {
        if (c < d) *reinterpret_cast<u32x2*>(p + c) = u32x2{a, b};
    } else {
        if (c < d) p[c] = (unsigned short)a;
        if (c + 1 < d) p[c + 1] = (unsigned short)(a >> 16);
        if (c + 2 < d) p[c + 2] = (unsigned short)b;
        if (c + 3 < d) p[c + 3] = (unsigned short)(b >> 16);
    }
}

// Numbers e .. e + 3 of x as entries c .. c + 3 of a row of d, 16 bytes at a time where rows are.
__device__ __forceinline__ void put4(float* p, int c, int d, const f32x16& x, int e) {
    if (d % 4 == 0) {
        if (c < d) *reinterpret_cast<f32x4*>(p + c) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + i < d) p[c + i] = x[e + i];
    }
}

// The sums of one row over ranges of its keys: partial [ranges][rows][d], behind it [ranges][rows] maximum (in powers of two)
// and total.  A wave for up to 64 ranges, lane s looking after one; WAVES waves for a row, whose sums meet in LDS.
struct Joined {
    float top, total;  // top: 0 if there is no key
    float x[2];        // entries lane and 64 + lane
};
template <int WAVES>
__device__ __forceinline__ Joined join_ranges(const float* partial, int ranges, int used, int64_t rows, int64_t at, int d, int lane,
                                              int wave) {
    const float* const ends = partial + ranges * rows * d;
    const int first = WAVES == 1 ? 0 : 64 * wave;
    used -= first;
    float top = -kInf, total = 0.f;
    if (lane < used) {
        const float* const e = ends + 2 * ((first + lane) * rows + at);  // (4-byte aligned: ranges, rows and d may all be odd)
        top = e[0];
        total = e[1];
    }
    float most = top;
#pragma unroll
    for (int s = 32; s; s >>= 1) most = fmaxf(most, __shfl_xor(most, s));
    // (parts that are finite each may add up past the largest number: 256 of them do not where each comes times 2^-8)
    if (most > -kInf) most += 8.f;
    const float base = most == -kInf ? 0.f : most;
    const float f = __builtin_amdgcn_exp2f(top - base);
    total *= f;
    Joined r{base, 0.f, {0.f, 0.f}};
    // eight at a time, so that their loads are under way together
    const float* o = partial + (first * rows + at) * d + lane;
    const bool in0 = lane < d, in1 = 64 + lane < d;
    for (int s0 = 0; s0 < min(used, 64); s0 += 8) {
        float a[8], b[8];
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const float* const from = o + (s0 + s) * rows * d;
            a[s] = s0 + s < used && in0 ? from[0] : 0.f;
            b[s] = s0 + s < used && in1 ? from[64] : 0.f;
        }
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const float fs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), s0 + s));
            r.total += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(total), s0 + s));
            // (an infinity of a range whose weights have vanished against another's is one all the same)
            r.x[0] = __builtin_fmaf(a[s], fabsf(a[s]) < kInf ? fs : 1.f, r.x[0]);
            r.x[1] = __builtin_fmaf(b[s], fabsf(b[s]) < kInf ? fs : 1.f, r.x[1]);
        }
    }
    if constexpr (WAVES > 1) {
        __shared__ float of_wave[WAVES][130];
        of_wave[wave][lane] = r.x[0];
        of_wave[wave][64 + lane] = r.x[1];
        if (lane == 0) {
            of_wave[wave][128] = most;
            of_wave[wave][129] = r.total;
        }
        __syncthreads();
        most = of_wave[0][128];
        for (int w = 1; w < WAVES; ++w) most = fmaxf(most, of_wave[w][128]);
        r.top = most == -kInf ? 0.f : most;
        r.total = r.x[0] = r.x[1] = 0.f;
        for (int w = 0; w < WAVES; ++w) {
            const float fw = __builtin_amdgcn_exp2f(of_wave[w][128] - r.top);
            r.total = __builtin_fmaf(of_wave[w][129], fw, r.total);
            const float a = of_wave[w][lane], b = of_wave[w][64 + lane];
            r.x[0] = __builtin_fmaf(a, fabsf(a) < kInf ? fw : 1.f, r.x[0]);
            r.x[1] = __builtin_fmaf(b, fabsf(b) < kInf ? fw : 1.f, r.x[1]);
        }
    }
    return r;
}

}  // namespace

}  // namespace attn
