// What the attention kernels share: element types, tiles in LDS, fragments of the matrix
// instructions, scores.
//
// Every product goes through v_mfma_f32_32x32x16 (float: eight v_mfma_f32_32x32x2 in its place): a wavefront multiplies
// A (32 rows x 16) with B (16 x 32 columns); lane l holds 8 elements of A's row l % 32 and 8 of B's column l % 32, at the
// places 8 (l / 32) + j of the 16; of the result it holds column l % 32 and rows
// 8 (i / 4) + 4 (l / 32) + i % 4, i = 0..15.  The order of the 16 is free as long as A and B agree.
//
// The operand that stays (queries forward, keys in the gradient of the keys) is B, held in registers for the whole
// kernel; what streams past it is A, read from LDS.  So a product of scores S^T = K Q^T leaves each lane
// the scores of ONE query with half of the tile's keys: the softmax needs no exchange but with
// lane ^ 32, and the probabilities are already the B fragments of O^T = V^T P^T, with the keys
// {4 h + 0..3, 8 + 4 h + 0..3} of every 16 in lane half h.  V^T's A fragments in that order are two
// transposing LDS reads (ds_read_b64_tr_b16) of the row-major tile.
#pragma once

#include <type_traits>

#include "bload_common.hpp"

namespace bload {

typedef _Float16 att_half;
typedef __bf16 att_bf16;
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
template <typename T> using frag8 = T __attribute__((ext_vector_type(8)));
template <typename T> using frag4 = T __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// [B, T, heads, D]: elements of a head side by side, any distance (in elements) between the rest.
struct AttTensor {
    const void* p;
    int64_t sb, st, sh;
};

struct AttArgs {
    AttTensor q, k, v, out, rest, dout, dq, dk, dv;
    float *lse, *delta;              // [B, Hq, T]
    const int4* mask;                // [B, T]: key_lo, key_hi, query_lo, query_hi
    const float* slopes;             // [Hq] or null
    float scale, cap;
    int32_t B, T, Hq, Hkv, G, D, tiles;
};

template <typename T>
__device__ __forceinline__ T* att_at(const AttTensor& t, int64_t b, int64_t slot, int64_t head)
{
    return reinterpret_cast<T*>(const_cast<void*>(t.p)) + b * t.sb + slot * t.st + head * t.sh;
}

__device__ __forceinline__ f32x16 mma(frag8<att_half> a, frag8<att_half> b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(frag8<att_bf16> a, frag8<att_bf16> b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(frag8<float> a, frag8<float> b, f32x16 c)
{
    // eight products of depth 2: lane half h supplies place h of the j-th
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
}

// N elements from or to memory that is aligned to an element only (one access of the full width).
template <typename T, int N>
__device__ __forceinline__ void load_any(const T* p, T (&x)[N]) { __builtin_memcpy(&x, p, sizeof(x)); }

// 16 bytes of a row of D elements from element d on; zeros beyond the row (which, unless ODD, is a whole number of them long).
template <typename T, bool ODD>
__device__ __forceinline__ vec16 load_chunk(const T* row, int d, int D)
{
    constexpr int N = 16 / sizeof(T);
    vec16 r = {0, 0, 0, 0};
    if (d + N <= D) {
        __builtin_memcpy(&r, row + d, 16);
    } else if (ODD && d < D) {
        T x[N];
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = d + j < D ? row[d + j] : (T)0.0f;
        __builtin_memcpy(&r, &x, 16);
    }
    return r;
}

// A B fragment straight from memory: elements d .. d + 7 of a row; zeros beyond the row.
template <typename T, bool ODD>
__device__ __forceinline__ frag8<T> load_frag(const T* row, int d, int D)
{
    frag8<T> f;
    vec16 c[sizeof(T) / 2];
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) c[i] = load_chunk<T, ODD>(row, d + i * (16 / (int)sizeof(T)), D);
    __builtin_memcpy(&f, &c, sizeof(f));
    return f;
}

// Four results side by side, d .. d + 3 of a row of D.
template <typename T>
__device__ __forceinline__ void store4(T* row, int d, int D, f32x4 x)
{
    T y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = (T)x[j];
    if (d + 4 <= D) {
        __builtin_memcpy(row + d, &y, sizeof(y));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (d + j < D) row[d + j] = y[j];
    }
}

// Rows of DP elements in LDS, in chunks of 16 bytes.  A chunk's place in its row is XORed with a
// number of the row, such that neither the rows of 16 lanes at one chunk (row_frag; of 16-bit types, whose rows are read most) nor
// four rows at four chunks (col_frag) meet in one bank.  The number is linear: that of a XOR b is that of a XOR that of b.
template <typename T, int DP>
struct Tile {
    static constexpr int kElems = 16 / (int)sizeof(T);
    static constexpr int kChunks = DP / kElems;
    static constexpr bool kByEight = sizeof(T) == 2 && (kChunks == 16 || kChunks == 8);      // rows 8 apart lie differently

    __device__ static __forceinline__ int swizzle(int row)
    {
        if constexpr (kByEight && kChunks == 16) return ((row & 3) << 2) | ((row & 4) >> 1) | ((row & 8) >> 3);
        else if constexpr (kByEight) return ((row & 2) << 1) | ((row & 4) >> 1) | ((row & 8) >> 3);
        else if constexpr (kChunks == 16) return ((row & 1) << 2) | ((row & 2) << 2) | ((row >> 1) & 1) | ((row >> 1) & 2);
        else if constexpr (kChunks == 8) return ((row & 1) << 2) | ((row >> 1) & 3);
        else if constexpr (kChunks == 24 || kChunks == 32) return row & 7;
        else return (row >> 1) & 3;
    }
    __device__ static __forceinline__ int at(int row, int chunk)       // in elements
    {
        return (row * kChunks + (chunk ^ swizzle(row))) * kElems;
    }
    // Where a lane reads, in bytes: `off` and, XORed with what is the same for all lanes, `place`.  Both are the
    // same for all tiles of a kernel; `renew` keeps the compiler from holding every XOR of theirs in a register.
    struct Reader {
        int off, place;
        __device__ __forceinline__ void renew() { asm volatile("" : "+v"(off), "+v"(place)); }
    };
    __device__ static __forceinline__ Reader rows()
    {
        const int row = lane_id() & 31, h = lane_id() >> 5;
        return {row * kChunks * 16, ((h * (8 / kElems)) ^ swizzle(row)) * 16};
    }
    // elements 16 s + 8 (lane / 32) .. + 7 of row r0 + lane % 32; r0: a multiple of 32
    __device__ static __forceinline__ frag8<T> row_frag(const T* tile, Reader r, int r0, int s)
    {
        frag8<T> f;
        vec16 x[8 / kElems];
#pragma unroll
        for (int i = 0; i < 8 / kElems; ++i)
            __builtin_memcpy(&x[i], reinterpret_cast<const char*>(tile) + r.off + (((s * (16 / kElems) + i) * 16) ^ r.place) + r0 * kChunks * 16, 16);
        __builtin_memcpy(&f, &x, sizeof(f));
        return f;
    }
    __device__ static __forceinline__ Reader columns()
    {
        const int lane = lane_id();
        if constexpr (sizeof(T) == 2) {
            // 16 lanes read four rows of 16 elements, 4 elements a lane, and get a column of four each
            const int r = 4 * (lane >> 5) + ((lane & 15) >> 2);
            return {r * kChunks * 16 + (lane & 1) * 8, ((((lane & 16) >> 3) | ((lane & 3) >> 1)) ^ swizzle(r)) * 16};
        } else {
            const int d = lane & 31, r = 4 * (lane >> 5);
            return {r * kChunks * 16 + (d & 3) * 4, ((d >> 2) ^ swizzle(r)) * 16};
        }
    }
    // element d0 + lane % 32 of the rows r0 + {4 h + 0..3, 8 + 4 h + 0..3}, h = lane / 32; r0: a multiple of 16, d0 of 32
    __device__ static __forceinline__ frag8<T> col_frag(const T* tile, Reader r, int r0, int d0)
    {
        if constexpr (sizeof(T) == 2) {
            typedef __attribute__((address_space(3))) s16x4* lds_ptr;
            s16x4 x[2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
                x[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_ptr)(reinterpret_cast<const char*>(tile) + r.off + (((d0 / kElems + (kByEight ? i : 0)) * 16) ^ r.place) + (r0 + 8 * i) * kChunks * 16));
            frag8<T> f;
            __builtin_memcpy(&f, &x, sizeof(f));
            return f;
        } else {
            // (the swizzle is linear: that of row 4 h + j is that of 4 h XOR that of j)
            frag8<T> f;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                f[j] = *reinterpret_cast<const T*>(reinterpret_cast<const char*>(tile) + r.off + (((d0 / 4) ^ swizzle(j & 3)) * 16 ^ r.place) +
                                                   (r0 + (j & 3) + 8 * (j >> 2)) * kChunks * 16);
            return f;
        }
    }
};

// R rows of D elements on their way from memory to LDS through the registers of `THREADS` threads (a workgroup, or each
// of its wavefronts for itself).  A thread keeps one place of a row and goes down the rows with it.  Nothing beyond a row
// is read, and nothing depends on the alignment of rows: where D is no whole number of chunks (ODD), the 16 bytes that hold a
// row's end are taken from D - 16 / sizeof(T) on and shifted down.
template <typename T, int DP, int R, bool ODD, int THREADS = kThreads>
struct Stage {
    using L = Tile<T, DP>;
    static constexpr int N = L::kElems, kWide = L::kChunks <= 4 ? 4 : L::kChunks <= 8 ? 8 : L::kChunks <= 16 ? 16 : 32;
    static constexpr int kRows = THREADS / kWide, kEach = R > kRows ? R / kRows : 1;
    vec16 x[kEach];
    int64_t st;                      // in elements: of two rows
    const T* at;                     // this thread's place of the next rows
    int row, place, from, D;

    __device__ __forceinline__ Stage(int64_t st_, int D_) : st(st_), D(D_)
    {
        const int t = (int)threadIdx.x % THREADS;
        row = min(t / kWide, R - 1);
        place = t % kWide;
        from = ODD && D < N ? 0 : min(place * N, D - N);
    }
    __device__ __forceinline__ void begin(const T* base, int row0) { at = base + (row0 + row) * st + from; }
    __device__ __forceinline__ void skip(int rows) { at += rows * st; }
    __device__ __forceinline__ vec16 get(const T* p) const
    {
        vec16 r;
        if (!ODD || D >= N) {
            __builtin_memcpy(&r, p, 16);
        } else {                                           // a row is shorter than 16 bytes
            T y[N];
#pragma unroll
            for (int j = 0; j < N; ++j) y[j] = p[min(j, D - 1)];
            __builtin_memcpy(&r, &y, 16);
        }
        return r;
    }
    // the R rows from row0 on, where begin() or the last load() left off; in the place of rows from `limit` on, the last one in
    // front of it
    __device__ __forceinline__ void load(int row0, int limit)
    {
        if (row0 + R <= limit) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) x[i] = get(at + i * kRows * st);
        } else {
#pragma unroll
            for (int i = 0; i < kEach; ++i) x[i] = get(at + (i * kRows - max(row0 + row + i * kRows - (limit - 1), 0)) * st);
        }
        at += R * st;
    }
    __device__ __forceinline__ vec16 whole(vec16 v) const
    {
        const int d = place * N;
        if (!ODD) return d < D ? v : vec16{0, 0, 0, 0};
        const int over = D < N ? d : d - from;             // elements in front of this place
        uint64_t y[2];
        __builtin_memcpy(&y, &v, 16);
        if (D < N) {                                       // (repeats of the last element behind the row)
            const int bits = D * (int)sizeof(T) * 8;
            y[1] = bits <= 64 ? 0 : y[1] & ((1ull << (bits - 64)) - 1);
            y[0] = bits >= 64 ? y[0] : y[0] & ((1ull << bits) - 1);
        }
        const int bits = min(over * (int)sizeof(T) * 8, 127);
        const uint64_t lo = bits >= 64 ? y[1] >> (bits & 63) : (y[0] >> bits) | (y[1] << 1 << (63 - (bits & 63)));
        const uint64_t hi = bits >= 64 ? 0 : y[1] >> bits;
        y[0] = d < D ? lo : 0;
        y[1] = d < D ? hi : 0;
        __builtin_memcpy(&v, &y, 16);
        return v;
    }
    __device__ __forceinline__ void put(T* tile, int i, vec16 y) const { __builtin_memcpy(tile + L::at(row + i * kRows, place), &y, 16); }
    // `left`: rows in front of the limit; zeros behind them, as 0 times what they hold has to be 0
    __device__ __forceinline__ void store(T* tile, int left) const
    {
        if (kWide != L::kChunks && place >= L::kChunks) return;
        if (kRows > R && (int)threadIdx.x % THREADS / kWide >= R) return;
        if (left < R) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) put(tile, i, row + i * kRows < left ? whole(x[i]) : vec16{0, 0, 0, 0});
        } else if (D == DP) {
            asm volatile("");                              // (a branch: by selection instead it costs every 16 bytes four of them)
#pragma unroll
            for (int i = 0; i < kEach; ++i) put(tile, i, x[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kEach; ++i) put(tile, i, whole(x[i]));
        }
    }
};

// Sums over a loop of matrix products stay in accumulation registers: said at the top of every step, or the compiler keeps
// them in others and copies them there and back around the products.  For kernels of one wave a SIMD, which
// have accumulation registers apart from the 256 others.
template <int N>
__device__ __forceinline__ void keep_sums(f32x16 (&x)[N])
{
#pragma unroll
    for (int d = 0; d < N; ++d) asm volatile("" : "+a"(x[d]));
}

// Nothing moves across: what stands in front is issued in front.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_sched_barrier(0); }

// use(n, get(n)) for n = 0 .. N - 1 with `AHEAD` fragments on their way from LDS in front of the one that is used.
template <int N, int AHEAD, typename Get, typename Use>
__device__ __forceinline__ void ahead(Get get, Use use)
{
    constexpr int kRing = AHEAD + 1;
    decltype(get(0)) f[kRing];
#pragma unroll
    for (int n = 0; n < AHEAD && n < N; ++n) f[n] = get(n);
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (n + AHEAD < N) f[(n + AHEAD) % kRing] = get(n + AHEAD);
        in_order();
        use(n, f[n % kRing]);
    }
}

// Operands that were loaded in front of a loop have arrived: without this the compiler waits for them inside the loop,
// and there for everything that is on its way from memory, at every step.
template <typename F, int N>
__device__ __forceinline__ void arrived(F (&x)[N])
{
#pragma unroll
    for (int s = 0; s < N; ++s) asm volatile("" : "+v"(x[s]));
}

// Eight probabilities, or gradients of scores, in 32 bits to a B fragment.  16-bit types: rounded to nearest, half a step of the type
// on each, because the matrix instructions take no wider operand beside 16-bit keys and values.  These are the roundings between the
// inputs and the output: one forward, two on the way to dq and dk; sums and states stay in 32 bits.
template <typename T>
__device__ __forceinline__ frag8<T> pack8(const f32x16& x, int from)
{
    f32x8 y;
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = x[from + j];
    return __builtin_convertvector(y, frag8<T>);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// What a kernel does to the products of queries and keys, compiled in: the bias by distance costs two instructions a score, the cap
// six and two transcendental ones, and a branch on either in the loop would keep the compiler from laying scores among products.
// With a cap there is the bias too, of slope 0 where there is none.  kCapFar: for 16-bit types and caps beyond kNearCap, seven
// instructions more a score.
enum { kPlain = 0, kBias = 1, kCap = 2, kCapFar = 3 };

// tanh x = 1 - 2 / (1 + e^2x) has an absolute error of up to 2e-7, which a cap multiplies: 1.3e-5 of a score at 64, less than a
// thirtieth of what rounding a probability to half takes, and the whole of it at 1e7.  Beyond this cap, below x = 1/8, the odd series
// x - x^3/3 + 2 x^5/15 takes its place: within 2^-19 of the score whatever the cap.  The series for all caps measured 269 us on a
// pass over 24 blocks of 777 with 6 heads of 37 bfloat16, which takes 225 without.
constexpr float kNearCap = 64.0f;

// A raw product q.k as a score in units of ln 2: cap tanh(scale q.k / cap) - slope |i - j|.
struct Score {
    float scale, inner, outer, slope;                      // all but `inner` in units of ln 2; outer: 0 without a cap
    __device__ __forceinline__ Score(const AttArgs& a, int head)
        : scale(a.scale * kLog2e), inner(a.cap > 0.0f ? fminf(a.scale / a.cap, 1e37f) : 0.0f), outer(a.cap * kLog2e),
          slope(a.slopes ? a.slopes[head] * kLog2e : 0.0f) {}
    // `keep`: the derivative of the capped score by the scaled one
    template <typename T, int MOD>
    __device__ __forceinline__ float of(float qk, float distance, float& keep) const
    {
        keep = 1.0f;
        if constexpr (MOD == kPlain) return qk * scale;
        if constexpr (MOD == kBias) return fmaf(-slope, fabsf(distance), qk * scale);
        float t;
        if constexpr (sizeof(T) == 2) t = 1.0f - 2.0f * __builtin_amdgcn_rcpf(1.0f + exp2_fast(qk * (inner * (2.0f * kLog2e))));
        else t = tanhf(qk * inner);
        if constexpr (sizeof(T) == 2 && MOD == kCapFar) {
            const float x = qk * inner, y = x * x;
            t = fabsf(x) < 0.125f ? fmaf(x * y, fmaf(y, 2.0f / 15, -1.0f / 3), x) : t;
        }
        keep = 1.0f - t * t;
        return fmaf(-slope, fabsf(distance), outer * t);
    }
    // as the arguments say
    template <typename T>
    __device__ __forceinline__ float any(float qk, int distance, float& keep) const
    {
        return outer > 0.0f ? of<T, kCapFar>(qk, (float)distance, keep) : of<T, kBias>(qk, (float)distance, keep);
    }
};

// Row n (0 .. 15) of a result, beside the lane's first.
__device__ __forceinline__ constexpr int result_row(int n) { return 8 * (n / 4) + n % 4; }

// Sum and maximum over a lane and lane ^ 32: one instruction hands each half of the wavefront the other's.
struct Halves {
    float low, high;
    __device__ __forceinline__ Halves(float x)
    {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        low = __uint_as_float(r[0]);
        high = __uint_as_float(r[1]);
    }
};
__device__ __forceinline__ float halves_sum(float x)
{
    const Halves h(x);
    return h.low + h.high;
}
__device__ __forceinline__ float halves_max(float x)
{
    const Halves h(x);
    return fmaxf(h.low, h.high);
}

// The running maximum of a softmax, in units of ln 2.  It follows the scores only where one passes it by more than kSlack: until
// then probabilities may be up to 2^kSlack, which costs no accuracy (they are floating point, and the sum that
// divides them has the same factor), and the sums need not be scaled.
constexpr float kSlack = 8.0f;

struct Maximum {
    float m = -INFINITY;
    __device__ __forceinline__ float base() const { return m == -INFINITY ? 0.0f : m; }
    // `top`: the largest of the new scores.  Whether some lane's maximum moved; then `f` is what each lane's sums shrink by.
    __device__ __forceinline__ bool moves(float top, float& f)
    {
        if (!__any(top > m + kSlack)) return false;
        const float up = fmaxf(m, top);
        f = up == -INFINITY ? 1.0f : exp2_fast(m - up);
        m = up;
        return true;
    }
};

// Gradients of scores, p (dp - delta), may lie anywhere in the range of dout, and far below it where a row sees many: float16 would
// lose them among its subnormals, or overflow.  They are packed as a multiple `by` of themselves, a power of two for each row of results:
// the first ones that are not 0 bring the largest of its tile between 2^6 and 2^7, and one that passes 2^15 does so again; the
// row's sums shrink along.  Measured: 16 blocks of 3000 short recordings, 16 heads of 128: dq 411 -> 424 us, dk and dv 533 -> 562 (20
// more from 2^12 on: more rows whose sums have to shrink).
struct Reach {
    enum { kNone = 0, kFirst, kSums };
    float by = 1.0f, limit = 0.0f;
    // `top`: the largest of the new ones, times `by`.  Whether some lane's multiple changed, and that of sums which are not all 0; then
    // `f` is what each lane's change by.
    __device__ __forceinline__ int moves(float top, float& f)
    {
        if (!__any(top > limit)) return kNone;
        f = 1.0f;
        bool held = false;
        if (top > limit) {
            held = limit > 0.0f;
            f = ldexpf(1.0f, min(7 - __builtin_amdgcn_frexp_expf(top), 64));     // (times any dp, below 2^41: far inside float32)
            by *= f;
            limit = 0x1p15f;
        }
        return __any(held) ? kSums : kFirst;
    }
};

__device__ __forceinline__ float wave_sum(float x)
{
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) x += __shfl_xor(x, d);
    return x;
}
__device__ __forceinline__ int wave_min(int x)
{
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) x = min(x, __shfl_xor(x, d));
    return __builtin_amdgcn_readfirstlane(x);
}
__device__ __forceinline__ int wave_max(int x)
{
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) x = max(x, __shfl_xor(x, d));
    return __builtin_amdgcn_readfirstlane(x);
}

// What one lane's row may look at, inside [0, T); an empty interval is [0, 0).
struct Span {
    int lo, hi;
    __device__ __forceinline__ bool has(int at) const { return (uint32_t)(at - lo) < (uint32_t)(hi - lo); }
};
__device__ __forceinline__ Span clamp_span(int lo, int hi, int T)
{
    Span s = {max(lo, 0), min(hi, T)};
    if (s.lo >= s.hi) s = {0, 0};
    return s;
}

// Intervals of all rows of a wavefront together: the hull, and the part that every row sees.
struct SpanRange {
    int lo, hi, in_lo, in_hi;
    __device__ __forceinline__ void of_wave(Span s)
    {
        lo = wave_min(s.hi > s.lo ? s.lo : 0x7fffffff);
        hi = wave_max(s.hi);
        in_lo = wave_max(s.lo);
        in_hi = wave_min(s.hi);
    }
    __device__ __forceinline__ bool meets(int k, int n) const { return k < hi && k + n > lo; }
    __device__ __forceinline__ bool full(int k, int n) const { return k >= in_lo && k + n <= in_hi; }
};

// Row D elements of a tensor in a wavefront's lanes, lane l holding elements l and l + 64 (D <= 128).
template <typename T>
__device__ __forceinline__ void load_row2(const T* row, int D, float (&x)[2])
{
    const int l = lane_id();
    x[0] = l < D ? (float)row[l] : 0.0f;
    x[1] = l + 64 < D ? (float)row[l + 64] : 0.0f;
}
template <typename T>
__device__ __forceinline__ void store_row2(T* row, int D, float x0, float x1)
{
    const int l = lane_id();
    if (l < D) row[l] = (T)x0;
    if (l + 64 < D) row[l + 64] = (T)x1;
}

__device__ __forceinline__ bool not_finite(float x) { return !(fabsf(x) <= 3.402823466e38f); }

// ---- rows that come out not finite ---------------------------------------------------
//
// What the mask hides has probability 0 in a matrix product, and 0 times an infinite or NaN element is NaN.  Such rows are computed
// again by their wavefront, in plain 32-bit arithmetic and from what they see alone, but only where something hidden is not finite:
// a row that sees such an element itself is what the matrix product made of it.

// The kernel's arguments read anew, so that those which only the rows below use are not held in registers up to there.
__device__ __forceinline__ AttArgs args_again()
{
    auto p = __builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    AttArgs a;
    __builtin_memcpy(&a, (const void*)p, sizeof(a));
    return a;
}

template <typename T>
__device__ __forceinline__ bool row_not_finite(const T* row, int D)
{
    constexpr int N = 16 / (int)sizeof(T);
    bool bad = false;
    for (int d = 0; d < D; d += 4 * N) {
        vec16 c[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = load_chunk<T, true>(row, d + i * N, D);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            T x[N];
            __builtin_memcpy(&x, &c[i], 16);
#pragma unroll
            for (int n = 0; n < N; ++n) bad |= not_finite((float)x[n]);
        }
    }
    return bad;
}

// Rows of operands that are not finite, as each lane's row meets them: hidden from it, or seen.
struct Met {
    bool hidden = false, seen = false;
    // bad(r): row r of the operands has an element that is not finite; lanes ask for 64 rows at a time
    template <typename Bad>
    __device__ __forceinline__ void look(Span span, int lo, int hi, Bad bad)
    {
        for (int r0 = lo; r0 < hi; r0 += kWave) {
            const int r = r0 + lane_id();
            for (uint64_t rows = __ballot(r < hi && bad(r)); rows; rows &= rows - 1) {
                const bool has = span.has(r0 + __ffsll((unsigned long long)rows) - 1);
                hidden |= !has;
                seen |= has;
            }
        }
    }
    // of the rows that its wavefront's tiles can have held: those that some lane does not see, or all
    template <typename Bad>
    __device__ __forceinline__ void look_around(Span span, int T, bool all, Bad bad)
    {
        const bool any = span.hi > span.lo;
        const int from = max(0, wave_min(any ? span.lo : T) - 64), to = min(T, wave_max(span.hi) + 64);
        const int in_lo = wave_max(any ? span.lo : 0), in_hi = wave_min(any ? span.hi : T);
        if (all || in_lo >= in_hi) return look(span, from, to, bad);
        look(span, from, in_lo, bad);
        look(span, in_hi, to, bad);
    }
};

// x.y over N pairs of rows of a lane's own; elements beyond D count as 0
template <typename T, int N>
__device__ __forceinline__ void row_dots(const T* const (&x)[N], const T* const (&y)[N], int D, float (&dot)[N])
{
    constexpr int kElems = 16 / (int)sizeof(T);
#pragma unroll
    for (int n = 0; n < N; ++n) dot[n] = 0.0f;
    for (int d = 0; d < D; d += 4 * kElems) {
        vec16 a[N][4], b[N][4];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                a[n][i] = load_chunk<T, true>(x[n], d + i * kElems, D);
                b[n][i] = load_chunk<T, true>(y[n], d + i * kElems, D);
            }
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                T u[kElems], w[kElems];
                __builtin_memcpy(&u, &a[n][i], 16);
                __builtin_memcpy(&w, &b[n][i], 16);
#pragma unroll
                for (int e = 0; e < kElems; ++e) dot[n] = fmaf((float)u[e], (float)w[e], dot[n]);
            }
    }
}

// acc += the sum over n < count of lane n's `weight` times row n, two elements of the rows to a lane (as load_row2 has them)
template <typename T>
__device__ __forceinline__ void add_rows(const T* rows, int64_t stride, int count, int D, float weight, float (&acc)[2])
{
    constexpr int kRows = sizeof(T) == 2 ? 16 : 8;         // on their way at a time
    const int d0 = min(lane_id(), D - 1), d1 = min(lane_id() + 64, D - 1);     // (what is beyond a row is stored nowhere)
    for (int n0 = 0; n0 < count; n0 += kRows) {
        T x[kRows][2];
#pragma unroll
        for (int n = 0; n < kRows; ++n) {
            const T* row = rows + min(n0 + n, count - 1) * stride;
            x[n][0] = row[d0];
            x[n][1] = row[d1];
        }
#pragma unroll
        for (int n = 0; n < kRows; ++n) {
            if (n0 + n >= count) break;
            const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight), n0 + n));
            acc[0] = fmaf(w, (float)x[n][0], acc[0]);
            acc[1] = fmaf(w, (float)x[n][1], acc[1]);
        }
    }
}

// Whether any element of a row that lies in the lanes as load_row2 has it is finite.
__device__ __forceinline__ bool any_finite(const float (&x)[2], int D)
{
    return __any((lane_id() < D && !not_finite(x[0])) || (lane_id() + 64 < D && !not_finite(x[1])));
}

// One query, at slot `at` of its block, over the keys [lo, hi), by one wavefront: lanes take a key each for the scores, then two
// elements of the values each.  The result is a mean all along (a sum could leave float32 where the mean does not), NaN where no
// key has a probability.  m and l as in the kernels: the maximum in units of ln 2, the sum of 2^(s - m).
template <typename T>
__device__ __forceinline__ void plain_row(const T* q, const T* k, const T* v, int64_t k_stride, int64_t v_stride, int D, const Score& score, int at, int lo, int hi,
                          float (&o)[2], float& m, float& l)
{
    o[0] = o[1] = l = 0.0f;
    m = -INFINITY;
    for (int j0 = lo; j0 < hi; j0 += kWave) {
        const int j = j0 + lane_id();
        float s = -INFINITY, keep, qk[1];
        if (j < hi) {
            row_dots<T, 1>({q}, {k + j * k_stride}, D, qk);
            s = score.any<T>(qk[0], at - j, keep);
        }
        float top = s;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
        const float up = fmaxf(m, top), base = up == -INFINITY ? 0.0f : up;
        const float p = exp2_fast(s - base), part = l * exp2_fast(m - base);
        m = up;
        l = part + wave_sum(p);
        if (l != l) break;                                 // a score that is no number: nor is anything else
        const float inv = l > 0.0f ? 1.0f / l : 0.0f;
        o[0] *= part * inv;
        o[1] *= part * inv;
        if (any_finite(o, D)) add_rows(v + j0 * v_stride, v_stride, min(hi - j0, kWave), D, p * inv, o);
    }
    if (!(l > 0.0f)) o[0] = o[1] = NAN;
}

}  // namespace bload
