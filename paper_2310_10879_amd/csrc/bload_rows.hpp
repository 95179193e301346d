// What the kernels that go through rows of features share: pieces of 16 bytes at any alignment, division by sizes, slot flags.
#pragma once

#include "bload_attention_host.hpp"

namespace bload {

// V elements side by side, as they lie in memory; any alignment.  They stay the words that were loaded until they are used: taken
// apart behind the load, each load is waited for before the next is sent.
template <typename T, int V>
struct RowPiece {
    static constexpr int kWords = V * sizeof(T) >= 4 ? V * (int)sizeof(T) / 4 : 1;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const T* p) { __builtin_memcpy(&w, p, V * sizeof(T)); }
    // Read once: the caches need not keep it.
    __device__ __forceinline__ void load_once(const T* p)
    {
        typedef uint32_t words __attribute__((ext_vector_type(kWords), aligned(sizeof(T))));
        if constexpr (V * sizeof(T) >= 4) {
            const words v = __builtin_nontemporal_load(reinterpret_cast<const words*>(p));
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = v[i];
        } else {
            load(p);
        }
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
    }
    // From here on the words count as new ones: what was made of them is made again, where holding it would take more registers.
    __device__ __forceinline__ void renew()
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) asm volatile("" : "+v"(w[i]));
    }
    __device__ __forceinline__ float operator[](int v) const
    {
        if constexpr (sizeof(T) == 4) {
            return __uint_as_float(w[v]);
        } else if constexpr (std::is_same<T, att_bf16>::value) {
            return __uint_as_float(v % 2 ? w[v / 2] & 0xffff0000u : w[v / 2] << 16);
        } else {
            const uint16_t half = (uint16_t)(v % 2 ? w[v / 2] >> 16 : w[v / 2]);
            T t;
            __builtin_memcpy(&t, &half, 2);
            return (float)t;
        }
    }
};

// Elements from `skip` on: those in front belong to the neighbouring lane.  A row that is no whole number of pieces ends with
// a piece that overlaps the one in front of it, so that every load and nearly every store is whole.
template <typename T, int V>
__device__ __forceinline__ void store_row(T* p, const float (&x)[V], int skip)
{
    if (skip == 0) {
        T t[V];
#pragma unroll
        for (int v = 0; v < V; ++v) t[v] = (T)x[v];
        __builtin_memcpy(p, &t, sizeof(t));
    } else {
#pragma unroll
        for (int v = 1; v < V; ++v)
            if (v >= skip) p[v] = (T)x[v];
    }
}

// The same past the caches, for what nothing reads soon.
template <typename T, int V>
__device__ __forceinline__ void store_row_once(T* p, const float (&x)[V], int skip)
{
    if constexpr (V * sizeof(T) < 4) {
        store_row<T, V>(p, x, skip);
    } else {
        constexpr int kWords = V * (int)sizeof(T) / 4;
        typedef uint32_t words __attribute__((ext_vector_type(kWords), aligned(sizeof(T))));
        if (skip == 0) {
            T t[V];
#pragma unroll
            for (int v = 0; v < V; ++v) t[v] = (T)x[v];
            words w;
            __builtin_memcpy(&w, &t, sizeof(t));
            __builtin_nontemporal_store(w, reinterpret_cast<words*>(p));
        } else {
            store_row<T, V>(p, x, skip);
        }
    }
}

template <int V>
__device__ __forceinline__ void load_floats(const float* p, float (&x)[V])
{
    __builtin_memcpy(&x, p, sizeof(x));
}

// Elements of a lane's piece: 16 bytes.
template <typename T> constexpr int kRowPiece = 16 / (int)sizeof(T);

// n / d for 0 <= n < 2^31: m = 2^(31 + s) / d rounded up, s = the bits of d - 1, is off by less than 1, so n m is off by less
// than 2^31 of 2^(31 + s), which is below the 1 / d that separates two quotients.
struct Divisor {
    uint32_t d, m, s;
};
inline Divisor divisor(int64_t d)
{
    Divisor r = {(uint32_t)d, 0, 0};
    while (((int64_t)1 << r.s) < d) ++r.s;
    if (r.s) r.m = (uint32_t)((((uint64_t)1 << (31 + r.s)) + (uint64_t)d - 1) / (uint64_t)d);
    return r;
}
__device__ __forceinline__ uint32_t over(uint32_t n, const Divisor& d) { return d.s ? __umulhi(n, d.m) >> (d.s - 1) : n; }

// The sum of two values over the lanes of an aligned group of L (a power of two up to 64), in every lane of it.
template <int L>
__device__ __forceinline__ void lanes_sum(float& a, float& b)
{
#pragma unroll
    for (int d = 1; d < L; d <<= 1) {
        a += __shfl_xor(a, d);
        b += __shfl_xor(b, d);
    }
}
template <int L>
__device__ __forceinline__ float lanes_sum(float a)
{
#pragma unroll
    for (int d = 1; d < L; d <<= 1) a += __shfl_xor(a, d);
    return a;
}

// What a slot does: 0 padding, 1 starts a sequence, 2 goes on from the slot in front of it (the first one from a state).
__device__ __forceinline__ int slot_does(const uint8_t* reset, const uint8_t* valid, int t, bool has_state)
{
    if (!valid[t]) return 0;
    if (reset[t]) return 1;
    return (t == 0 ? has_state : valid[t - 1] != 0) ? 2 : 1;
}

// Sums over what workgroups left, [n_parts][columns] float32 -> [columns], the parts in a fixed order (bload_norm.hip).
// The columns up to end[0] go to dst[0], those from there to end[1] to dst[1] and so on; where it is null, nowhere.
struct ColumnSums {
    const float* parts;
    int64_t n_parts, columns;
    float* dst[4];
    int64_t end[4];
};
bload_status column_sums(const ColumnSums& a, hipStream_t stream);

// 64 columns to a workgroup, 16 lanes of four columns and 16 shares of the parts, whose sums are added in their order.
__device__ __forceinline__ void column_sums_of_64(const ColumnSums& a, int64_t group)
{
    constexpr int kShares = 16;
    __shared__ float sums[kShares][64];
    const int c = ((int)threadIdx.x % 16) * 4, share = (int)threadIdx.x / 16;
    const int64_t first = group * 64 + c, each = (a.n_parts + kShares - 1) / kShares;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (first + 4 <= a.columns) {
#pragma unroll 4
        for (int64_t p = share * each; p < min((share + 1) * each, a.n_parts); ++p) {
            float x[4];
            load_floats<4>(a.parts + p * a.columns + first, x);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] += x[i];
        }
    } else {
        for (int64_t p = share * each; p < min((share + 1) * each, a.n_parts); ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (first + i < a.columns) s[i] += a.parts[p * a.columns + first + i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[share][c + i] = s[i];
    __syncthreads();
    const int64_t column = group * 64 + threadIdx.x;
    if (threadIdx.x >= 64 || column >= a.columns) return;
    float y = 0.0f;
#pragma unroll
    for (int i = 0; i < kShares; ++i) y += sums[i][threadIdx.x];
    int64_t from = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (column >= from && column < a.end[i] && a.dst[i]) a.dst[i][column - from] = y;
        from = a.end[i];
    }
}

template <typename F>
inline void by_dtype(bload_dtype dtype, F f)
{
    if (dtype == BLOAD_F16) f(type_is<att_half>());
    else if (dtype == BLOAD_BF16) f(type_is<att_bf16>());
    else f(type_is<float>());
}

}  // namespace bload
