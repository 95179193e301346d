// What both passes of the selective scan share: arguments, staging of tiles, the lanes' states.
#pragma once

#include <algorithm>

#include "bload_rows.hpp"

namespace bload {

constexpr int kTile = 16;            // slots that are staged together, and after which the forward pass saves a state
constexpr int kLanesC = 16;          // channels of a wavefront: lane l has channel l % 16
constexpr int kGroupC = 64;          // channels of a workgroup

struct ScanArgs {
    AttTensor x, dt, z, b, c, out;
    AttTensor dout, dx, ddt, dz, db, dc;
    const float *rate, *skip, *dt_bias;      // [D, N], [D] or null, [D] or null
    const uint8_t *reset, *valid;
    const float* in;                 // [B, D, N] or null: the state in front; backward: that of the forward pass
    float* last;                     // [B, D, N] or null: the state behind; backward: the gradient by `in`
    const float* dlast;              // backward: the gradient by `last`
    float* saved;                    // [B, tiles, D, N] or null: the state in front of every tile
    float* maps;                     // [B, chunks, D, N]: a chunk's own part of the state behind it, then the state in front of it
    float* spans;                    // [B, chunks, D]: the sum of its steps
    uint8_t* cut;                    // [B, chunks]: some slot of it does not go on
    float* shares;                   // backward: [slices][B][T][G][2][N], the slices' shares of dB and dC
    float* parts;                    // backward: [parts][D N + 2 D]
    int64_t B;
    int32_t T, D, N, G, per;         // per: channels of a group
    int32_t slices, chunks, chunk, tiles, blocks;      // chunk in slots; blocks: of a workgroup at a time, backward
    int32_t softplus;
};

// log(1 + e^x): max(x, 0) + log1p(w), w = e^-|x|, and log1p(w) = 2 atanh(w / (2 + w)) by its series, whose argument is at
// most 1/3: what is left out is below 2^-25 of it.  (log2 of 1 + w would lose the small ones, which are the ordinary steps.)
__device__ __forceinline__ float softplus(float x)
{
    const float w = __builtin_amdgcn_exp2f(-kLog2e * fabsf(x)), s = w * __builtin_amdgcn_rcpf(2.0f + w), t = s * s;
    float p = 1.0f / 13.0f;
    p = fmaf(p, t, 1.0f / 11.0f);
    p = fmaf(p, t, 1.0f / 9.0f);
    p = fmaf(p, t, 1.0f / 7.0f);
    p = fmaf(p, t, 1.0f / 5.0f);
    p = fmaf(p, t, 1.0f / 3.0f);
    p = fmaf(p, t, 1.0f);
    return fmaf(2.0f * s, p, fmaxf(x, 0.0f));
}
__device__ __forceinline__ float logistic(float x) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * x)); }

// Four channels of one slot, as a thread stages them.
template <typename T> using Four = RowPiece<T, 4>;

// Where a workgroup and its threads are.  States: lane l of a wavefront has channel 16 wave + l % 16 and, of every part of
// 4 NS states, the NS from NS (l / 16) on.  Staging: thread t has slot t / 16 of a tile and channels 4 (t % 16) on, zeros where
// there are none.
struct ScanPlace {
    int64_t b;
    int group, chunk, d0, d1;        // channels of the workgroup
    int d, q;                        // the lane's
    bool mine;
    int slot, four, n_four;          // the thread's, staging: its slot, first channel, and how many there are
    __device__ __forceinline__ ScanPlace(const ScanArgs& a, int64_t n)
    {
        const int slice = (int)(n % a.slices);
        n /= a.slices;
        group = (int)(n % a.G);
        n /= a.G;
        chunk = (int)(n % a.chunks);
        b = n / a.chunks;
        d0 = group * a.per + slice * kGroupC;
        d1 = min(d0 + kGroupC, (group + 1) * a.per);
        const int tid = (int)threadIdx.x;
        d = d0 + wave_id() * kLanesC + tid % kLanesC;
        q = lane_id() / kLanesC;
        mine = d < d1;
        slot = tid / 16;
        four = d0 + 4 * (tid % 16);
        n_four = min(max(d1 - four, 0), 4);
    }
};

// The thread's four channels of its slot, a tile further on with every load or store; BACK: a tile back.
template <typename T, bool BACK = false>
struct Stream {
    T* p;
    int64_t tile;
    int n;
    __device__ __forceinline__ Stream(const AttTensor& x, const ScanPlace& at, int t0)
        : p(att_at<T>(x, at.b, t0 + at.slot, 0) + at.four), tile((BACK ? -kTile : kTile) * x.st), n(at.n_four)
    {
    }
    __device__ __forceinline__ void load(Four<T>& x, bool here)
    {
        x.zero();
        if (here && n == 4) x.load(p);
        if (here && n && n < 4) {
            T t[4] = {};
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < n) t[i] = p[i];
            __builtin_memcpy(&x.w, &t, sizeof(t));
        }
        p += tile;
    }
    __device__ __forceinline__ void store(const float (&x)[4])
    {
        if (n == 4) {
            T t[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) t[i] = (T)x[i];
            __builtin_memcpy(p, &t, sizeof(t));
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < n) p[i] = (T)x[i];
        }
        p += tile;
    }
    __device__ __forceinline__ void pass() { p += tile; }
};
// The same for B and C: elements threadIdx % 16 and every 16th behind it of the thread's slot.
template <typename T, int NP, bool BACK = false>
struct PairStream {
    static constexpr int kEach = (NP + 15) / 16;
    const T* p;
    int64_t tile;
    int n, N;
    T v[kEach];
    __device__ __forceinline__ PairStream(const AttTensor& x, const ScanArgs& a, const ScanPlace& at, int t0)
        : p(att_at<T>(x, at.b, t0 + at.slot, at.group) + threadIdx.x % 16), tile((BACK ? -kTile : kTile) * x.st), n((int)threadIdx.x % 16), N(a.N)
    {
    }
    __device__ __forceinline__ void load(bool here)
    {
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            v[k] = (T)0.0f;
            if (here && n + 16 * k < N) v[k] = p[16 * k];
        }
        p += tile;
    }
    __device__ __forceinline__ void stage(float* row, bool live) const
    {
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            if (NP % 16 == 0 || n + 16 * k < NP) row[n + 16 * k] = live ? (float)v[k] : 0.0f;
    }
};

// The lane's states of all parts; nothing (0) beyond N or beyond the workgroup's channels.
template <int NS, int PARTS>
__device__ __forceinline__ void load_states(const float* base, int64_t row, const ScanArgs& a, const ScanPlace& at, float (&x)[PARTS][NS])
{
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
        const int n = (p * 4 + at.q) * NS;
        const float* from = base + (row * a.D + at.d) * a.N + n;
        if (base && at.mine && n + NS <= a.N) {
            __builtin_memcpy(&x[p], from, sizeof(x[p]));
        } else {
#pragma unroll
            for (int i = 0; i < NS; ++i) x[p][i] = base && at.mine && n + i < a.N ? from[i] : 0.0f;
        }
    }
}
template <int NS, int PARTS>
__device__ __forceinline__ void store_states(float* base, int64_t row, const ScanArgs& a, const ScanPlace& at, const float (&x)[PARTS][NS])
{
    if (!at.mine) return;
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
        const int n = (p * 4 + at.q) * NS;
        float* to = base + (row * a.D + at.d) * a.N + n;
        if (n + NS <= a.N) {
            __builtin_memcpy(to, &x[p], sizeof(x[p]));
        } else {
#pragma unroll
            for (int i = 0; i < NS; ++i)
                if (n + i < a.N) to[i] = x[p][i];
        }
    }
}

// Four columns of a row in LDS, 16 bytes aligned.
__device__ __forceinline__ void get_four(float (&x)[4], const float* p) { __builtin_memcpy(&x, __builtin_assume_aligned(p, 16), 16); }
__device__ __forceinline__ void put_four(float* p, const float (&x)[4]) { __builtin_memcpy(__builtin_assume_aligned(p, 16), &x, 16); }
__device__ __forceinline__ void get_steps(float2 (&s)[4], const float2* p) { __builtin_memcpy(&s, __builtin_assume_aligned(p, 16), 32); }
__device__ __forceinline__ void put_steps(float2* p, const float2 (&s)[4]) { __builtin_memcpy(__builtin_assume_aligned(p, 16), &s, 32); }

// Of four values for four slots in every lane, the sum over the four lanes of a channel (l % 16): lane q = l / 16
// gets that of slot q.  Each exchange leaves half of the values, whole where the other half went.
__device__ __forceinline__ float sum_states(float y0, float y1, float y2, float y3)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(y0), __float_as_uint(y2), false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(y1), __float_as_uint(y3), false, false);
    const float s = __uint_as_float(a[0]) + __uint_as_float(a[1]), t = __uint_as_float(b[0]) + __uint_as_float(b[1]);
    const auto c = __builtin_amdgcn_permlane16_swap(__float_as_uint(s), __float_as_uint(t), false, false);
    return __uint_as_float(c[0]) + __uint_as_float(c[1]);
}

// What the slots of a tile do, one bit each, the same in every lane of a wavefront: whether they are valid, and whether the state
// in front of them is dropped.  Slots from `end` on do nothing: neither.  The flags are sent for with the tile's other inputs, long
// before they are looked at.
struct TileFlags {
    uint32_t live, cut;
};
// Whose flags are looked at for slot t of a block of T: its own and those of the one in front, both inside the block whatever t is.
// (What is read for a first slot's front, and for slots behind the block, is not used.)
struct LookSlots {
    int own, front;
};
__host__ __device__ constexpr LookSlots look_slots(int t, int T)
{
    const int own = t < T ? t : T - 1;
    return {own, own > 0 ? own - 1 : 0};
}
struct TileLook {
    uint8_t reset, valid, before;
    __device__ __forceinline__ void load(const ScanArgs& a, int64_t b, int t0)
    {
        const LookSlots look = look_slots(t0 + lane_id() % kTile, a.T);
        const int64_t first = b * a.T;
        reset = a.reset[first + look.own];
        valid = a.valid[first + look.own];
        before = a.valid[first + look.front];
    }
    __device__ __forceinline__ TileFlags flags(int t0, int end, bool has_state) const
    {
        const int t = t0 + lane_id() % kTile;
        const bool there = t < end, live = there && valid, on = live && !reset && (t > 0 ? before != 0 : has_state);
        return {(uint32_t)__ballot(live) & 0xffffu, (uint32_t)__ballot(there && !on) & 0xffffu};
    }
};

// f(NS, PARTS)
template <typename F>
inline void scan_by_states(int32_t N, F f)
{
    using std::integral_constant;
    if (N <= 4) f(integral_constant<int, 1>(), integral_constant<int, 1>());
    else if (N <= 8) f(integral_constant<int, 2>(), integral_constant<int, 1>());
    else if (N <= 16) f(integral_constant<int, 4>(), integral_constant<int, 1>());
    else if (N <= 32) f(integral_constant<int, 4>(), integral_constant<int, 2>());
    else if (N <= 48) f(integral_constant<int, 4>(), integral_constant<int, 3>());
    else f(integral_constant<int, 4>(), integral_constant<int, 4>());
}

// Sizes and the choice of chunks, for both passes.
inline bload_status scan_sizes(ScanArgs& a, int64_t B, int32_t T, int32_t D, int32_t N, int32_t G, bload_dtype dtype)
{
    if (B < 0 || T < 1 || D < 1 || N < 1 || N > BLOAD_SELECTIVE_MAX_STATES || G < 1 || D % G != 0 || !att_dtype(dtype)) return BLOAD_EINVAL;
    if (T > (1 << 30) || D > (1 << 24) || B >= ((int64_t)1 << 40) / T || B > ((int64_t)1 << 48) / D / N ||
        B * T > ((int64_t)1 << 56) / D / N)
        return BLOAD_EOVERFLOW;
    a.B = B;
    a.T = T;
    a.D = D;
    a.N = N;
    a.G = G;
    a.per = D / G;
    a.slices = (int32_t)ceil_div(a.per, kGroupC);
    a.tiles = (int32_t)ceil_div(T, kTile);
    const int64_t alone = B * G * a.slices;
    // Cut, the states are gone through twice (and the results of all chunks wait for that); whole, a compute unit has at most one
    // workgroup.  4096 slots of 16 states, bfloat16, forward alone / with gradients: 64 workgroups cut 160 / 532 us, whole 542 / 2426; 192
    // cut 436 / 1668, whole 543 / 2453; 256 cut 539 / 2001, whole 544 / 2467; 448 cut 992 / 3798, whole 718 / 3140.  One bound
    // for both passes: whole, the forward pass loses nothing from 240 on; with gradients 256 would be faster cut.
    a.chunks = 1;
    if (alone > 0 && alone < 240) a.chunks = (int32_t)std::max<int64_t>(1, std::min<int64_t>({ceil_div(1024, alone), a.tiles / 4, 64}));
    const int64_t each = ceil_div(a.tiles, a.chunks);
    a.chunk = (int32_t)each * kTile;
    a.chunks = (int32_t)ceil_div(a.tiles, each);
    if (alone > kMaxGroups / a.chunks || B * D > kMaxGroups * 16 || ceil_div(B * (int64_t)D * N, kThreads) > kMaxGroups) return BLOAD_EOVERFLOW;
    return BLOAD_OK;
}

inline bool states_meet(const float* in, const float* out, const ScanArgs& a, bool same_is_fine)
{
    if (!in || !out || (in == out && same_is_fine)) return false;
    const uintptr_t p = reinterpret_cast<uintptr_t>(in), q = reinterpret_cast<uintptr_t>(out);
    return (p < q ? q - p : p - q) < (uintptr_t)a.B * a.D * a.N * sizeof(float);
}

// bload_selective.hip
bload_status scan_args(ScanArgs& a, const bload_selective* s);
// The states in front of every chunk from the chunks' own parts (or backward, the gradients behind them), in their place.
void scan_join(const ScanArgs& a, const float* first, bool back, hipStream_t stream);

}  // namespace bload
