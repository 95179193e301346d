// bload_segment_conv: a short causal convolution per feature inside the sequences of packed blocks, forward and backward.
//
//     p_t = bias + sum_j w[K-1-j] x_{t-j}   over the taps j < K that reach no further back than slot t's sequence does,
//     y = p or p sigmoid(p);  0 on padding
// Backward, with dp = dout (or dout s (1 + p (1 - s)), s = sigmoid(p)):
//     dx_t = sum_j w[K-1-j] dp_{t+j} over the slots t+j that reach back to t;  dw[K-1-j] = sum dp_t x_{t-j};  dbias = sum dp
// A block may go on from the K - 1 inputs in front of it, and leaves those that the next one goes on from.
//
// HBM bound: x is read and y written once; backward x and dout are read and dx is written, p formed again.  A lane takes V
// features (16 bytes) and a run of slots, holds the last K - 1 inputs in registers, and a slot's age (how many slots of its
// sequence lie in front of it, up to K - 1) says which of them to forget.  Ages of a run lie in LDS.  Runs begin with the K - 1 inputs in
// front of them, which their neighbour reads as well (from L2); backward a run also forms dp of the K - 1 slots
// behind it.  The weights' gradients stay in registers over all runs of a lane, are added inside the workgroup
// and left in the workspace, and column_sums adds the workgroups' in a fixed order.
// Backward a step is four slots, whose inputs are loaded while the four in front of them are computed, and a step whose slots all look back
// over all taps and lie inside the run has no branch in it.  Half of the forward pass's 16 bytes to a lane there: with all of them,
// or with more slots to a step, the registers spill (343 -> 822 us); with a quarter there are four wavefronts a SIMD in place of two, and
// four taps take 458 us both ways in place of 467, three 418 in place of 404.
// Measured, averages among other kernels: 48000 slots of 4096 bfloat16, 4 taps, sequences of some 24 slots: forward 154 us for 0.79 GB,
// 5.1 TB/s; backward 322 us for 1.18 GB, 3.7 TB/s (runs of 128 slots; when that was chosen 310 us, with 64 343, with 32 372): 36 vector
// instructions an element, 28 of them the formulas', and memory that waits for them.  In float16 the forward kernel takes 227
// registers for bfloat16's 164, two wavefronts a SIMD for three: 293 us.
#include <algorithm>

#include "bload_rows.hpp"

namespace bload {
namespace {

struct ConvArgs {
    AttTensor x, out, dout;          // out: y, backward dx
    const uint8_t *reset, *valid;
    const float *weight, *bias;      // [D, K], [D] or null
    const void* in;                  // [B, K - 1, D] or null
    void* last;                      // the same, or null; backward: din
    const void* dlast;
    float* parts;                    // [groups of items][D K + D]
    int64_t items, groups;           // items: runs of all blocks; groups: of items, one to a workgroup at a time
    int32_t T, D, F, slices, runs, run;        // runs of a block, slots of a run
    int32_t silu;
};

// 1 + the slots of its sequence in front of slot t, up to most; 0 on padding.
__device__ __forceinline__ int slot_age(const uint8_t* reset, const uint8_t* valid, int t, bool has_state, int most)
{
    int what = slot_does(reset, valid, t, has_state), age = 0;
    if (what == 0) return 0;
    while (what == 2 && age < most) {
        ++age;
        if (--t < 0) return 1 + most;
        what = slot_does(reset, valid, t, has_state);
    }
    return 1 + age;
}

__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * x)); }

// Elements of a lane's piece, of the sizes and for the pass that the kernel is built or planned for.
constexpr int conv_piece(int elem_bytes, int taps, bool back) { return 16 / elem_bytes / (taps <= 4 ? 1 : 2) / (back ? 2 : 1); }

// Where a WIDE instance is built: the numbers of taps in use.
template <int V, int K> constexpr bool kWideTaps = V > 1 && K >= 2 && K <= 4;

template <bool WIDE>
__device__ __forceinline__ int slot_value(int x)
{
    return WIDE ? __builtin_amdgcn_readfirstlane(x) : x;
}

// What both passes set up: a lane's features and its weights.
template <int V, int K>
struct ConvLane {
    int d, skip;
    bool mine;
    float w[K][V], bias[V];
    __device__ __forceinline__ ConvLane(const ConvArgs& a, int f, int slice)
    {
        const int d0 = (slice * a.F + f) * V;
        mine = d0 < a.D;
        d = min(d0, a.D - V);
        skip = min(d0 - d, V);
        float rows[V * K];
        load_floats<V * K>(a.weight + (int64_t)d * K, rows);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            bias[v] = a.bias ? a.bias[d + v] : 0.0f;
#pragma unroll
            for (int k = 0; k < K; ++k) w[k][v] = rows[v * K + k];
        }
    }
};

template <typename T, int V, int K>
__device__ __forceinline__ void load_slot(RowPiece<T, V>& piece, const ConvArgs& a, int64_t b, int t, int d)
{
    piece.zero();
    if (t >= 0) {
        if (t < a.T) piece.load(att_at<T>(a.x, b, t, 0) + d);
    } else if (a.in) {
        piece.load(reinterpret_cast<const T*>(a.in) + (b * (K - 1) + K - 1 + t) * a.D + d);
    }
}

// R: slots of a run.  WIDE: a wavefront has one run (F is 64), so that ages are the same in all its lanes, and rows are whole pieces.
template <typename T, int V, int K, int R, bool WIDE>
__global__ __launch_bounds__(kThreads) void conv_kernel(ConvArgs a)
{
    __shared__ uint8_t ages[kThreads * R];
    const int f = (int)threadIdx.x & (a.F - 1), lane_item = (int)threadIdx.x / a.F, each = kThreads / a.F;
    const int slice = (int)(blockIdx.x % a.slices);
    const int64_t item0 = (int64_t)(blockIdx.x / a.slices) * each, item = item0 + lane_item;
    for (int n = (int)threadIdx.x; n < each * R; n += kThreads) {
        const int64_t i = item0 + n / R, b = i / a.runs;
        const int t = (int)(i - b * a.runs) * R + n % R;
        ages[n] = i < a.items && t < a.T ? (uint8_t)slot_age(a.reset + b * a.T, a.valid + b * a.T, t, a.in != nullptr, K - 1) : 0;
    }
    __syncthreads();
    const ConvLane<V, K> lane(a, f, slice);
    if (item >= a.items || !lane.mine) return;
    const int64_t b = item / a.runs;
    const int t0 = (int)(item - b * a.runs) * R;
    RowPiece<T, V> x[K - 1 + R];
#pragma unroll
    for (int i = 0; i < K - 1 + R; ++i) load_slot<T, V, K>(x[i], a, b, t0 - (K - 1) + i, lane.d);
    const bool last = a.last && t0 + R >= a.T;
    float seen[K][V];                // seen[j]: the input of j slots before
#pragma unroll
    for (int j = 1; j < K; ++j)
#pragma unroll
        for (int v = 0; v < V; ++v) seen[j][v] = x[K - 1 - j][v];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (t0 + i >= a.T) break;
        const int age = slot_value<WIDE>(ages[lane_item * R + i]);
        float p[V];
#pragma unroll
        for (int v = 0; v < V; ++v) seen[0][v] = x[K - 1 + i][v];
        if (age < K)
#pragma unroll
            for (int j = 0; j < K; ++j)
                if (j >= age)
#pragma unroll
                    for (int v = 0; v < V; ++v) seen[j][v] = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            p[v] = lane.bias[v];
#pragma unroll
            for (int j = K - 1; j >= 0; --j) p[v] = fmaf(lane.w[K - 1 - j][v], seen[j][v], p[v]);
            if (a.silu) p[v] *= sigmoid(p[v]);
            if (age == 0) p[v] = 0.0f;
        }
        store_row_once<T, V>(att_at<T>(a.out, b, t0 + i, 0) + lane.d, p, WIDE ? 0 : lane.skip);
        if (last && t0 + i == a.T - 1)
#pragma unroll
            for (int j = 0; j < K - 1; ++j)
                store_row<T, V>(reinterpret_cast<T*>(a.last) + (b * (K - 1) + K - 2 - j) * a.D + lane.d, seen[j], lane.skip);
#pragma unroll
        for (int j = K - 1; j > 0; --j)
#pragma unroll
            for (int v = 0; v < V; ++v) seen[j][v] = seen[j - 1][v];
    }
}

// Backward: slots whose loads are on their way together, most slots of a run, and slots behind it that its steps may look at.
constexpr int kConvStep = 4, kConvRun = 128, kConvHalo = 8;
static_assert(kConvHalo % kConvStep == 0 && kConvHalo >= BLOAD_CONV_MAX_TAPS - 1, "the last step's slots have ages");

// SILU: 1 or 0, or -1 where the call says which.
template <typename T, int V, int K, bool WIDE, int SILU>
__global__ __launch_bounds__(kThreads) void conv_backward_kernel(ConvArgs a)
{
    constexpr int S = kConvStep;
    const bool silu = SILU < 0 ? a.silu : SILU;
    extern __shared__ float shared[];
    const int f = (int)threadIdx.x & (a.F - 1), lane_item = slot_value<WIDE>((int)threadIdx.x / a.F), each = kThreads / a.F;
    const int reach = a.run + kConvHalo;                   // slots whose ages a run needs, in whole steps
    const int slice = (int)(blockIdx.x % a.slices);
    uint8_t* ages = reinterpret_cast<uint8_t*>(shared);    // [each][reach], and the last slot's of each run's block
    uint8_t* last_age = ages + each * reach;
    const ConvLane<V, K> lane(a, f, slice);
    float dw[K][V], db[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        db[v] = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) dw[k][v] = 0.0f;
    }
    for (int64_t group = blockIdx.x / a.slices; group < a.groups; group += gridDim.x / a.slices) {
        const int64_t item0 = group * each, item = item0 + lane_item;
        __syncthreads();
        for (int n = (int)threadIdx.x; n < each * (reach + 1); n += kThreads) {
            const bool final = n >= each * reach;
            const int64_t i = item0 + (final ? n - each * reach : n / reach), b = i / a.runs;
            const int t = final ? a.T - 1 : (int)(i - b * a.runs) * a.run + n % reach;
            ages[n] = i < a.items && t < a.T ? (uint8_t)slot_age(a.reset + b * a.T, a.valid + b * a.T, t, a.in != nullptr, K - 1) : 0;
        }
        __syncthreads();
        if (item >= a.items || !lane.mine) continue;
        const int64_t b = item / a.runs;
        const int t0 = (int)(item - b * a.runs) * a.run, t1 = min(t0 + a.run, a.T), end = t1 + K - 1;
        const int kept = slot_value<WIDE>(a.dlast ? last_age[lane_item] : 0);
        float seen[K][V], acc[K][V];                       // acc[j]: of dx of the slot j before, from the slots up to here
#pragma unroll
        for (int j = 1; j < K; ++j) {
            RowPiece<T, V> x;
            load_slot<T, V, K>(x, a, b, t0 - j, lane.d);
#pragma unroll
            for (int v = 0; v < V; ++v) seen[j][v] = x[v], acc[j][v] = 0.0f;
        }
        const T *px = att_at<T>(a.x, b, t0, 0), *pd = att_at<T>(a.dout, b, t0, 0);
        T* to = att_at<T>(a.out, b, t0, 0);
        RowPiece<T, V> x_next[S], dy_next[S];              // the next step's, on their way while one is computed
        auto load = [&](int s0) {
            const int n = min(end, a.T) - s0;
#pragma unroll
            for (int i = 0; i < S; ++i) {
                x_next[i].zero();
                dy_next[i].zero();
                if (i < n) {
                    x_next[i].load(px + (s0 - t0 + i) * a.x.st + lane.d);
                    dy_next[i].load(pd + (s0 - t0 + i) * a.dout.st + lane.d);
                }
            }
        };
        load(t0);
        for (int s0 = t0; s0 < end; s0 += S) {
            RowPiece<T, V> x[S], dy[S];
#pragma unroll
            for (int i = 0; i < S; ++i) x[i] = x_next[i], dy[i] = dy_next[i];
            load(s0 + S);
            // Inner steps: the slots are the run's own, and so are those that they complete, none of which a gradient of the state
            // reaches; and every slot looks back over all taps.
            auto step = [&](auto all_inner) {
                constexpr bool kInner = decltype(all_inner)::value;
#pragma unroll
                for (int i = 0; i < S; ++i) {
                    const int s = s0 + i;
                    if (!kInner && s >= end) break;
                    const int age = kInner ? K : slot_value<WIDE>(ages[lane_item * reach + s - t0]);
                    float dp[V];
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        seen[0][v] = x[i][v];
                        acc[0][v] = 0.0f;
                        dp[v] = age ? dy[i][v] : 0.0f;
                    }
                    if (!kInner && age < K)
#pragma unroll
                        for (int j = 0; j < K; ++j)
                            if (j >= age)
#pragma unroll
                                for (int v = 0; v < V; ++v) seen[j][v] = 0.0f;
                    if (silu) {
#pragma unroll
                        for (int v = 0; v < V; ++v) {
                            float p = lane.bias[v];
#pragma unroll
                            for (int j = K - 1; j >= 0; --j) p = fmaf(lane.w[K - 1 - j][v], seen[j][v], p);
                            const float sg = sigmoid(p);
                            // (padding: dp stays 0 whatever the slope of the bias)
                            dp[v] *= sg * fmaf(p, 1.0f - sg, 1.0f);
                        }
                    }
                    if (kInner || s < t1)
#pragma unroll
                        for (int v = 0; v < V; ++v) {
                            db[v] += dp[v];
#pragma unroll
                            for (int j = 0; j < K; ++j)
                                if (kInner || j < age) dw[K - 1 - j][v] = fmaf(dp[v], seen[j][v], dw[K - 1 - j][v]);
                        }
#pragma unroll
                    for (int j = 0; j < K; ++j)
                        if (kInner || j < age)
#pragma unroll
                            for (int v = 0; v < V; ++v) acc[j][v] = fmaf(lane.w[K - 1 - j][v], dp[v], acc[j][v]);
                    // slot u has heard from all that look back to it
                    const int u = s - (K - 1);
                    if constexpr (kInner) {
                        store_row_once<T, V>(to + (u - t0) * a.out.st + lane.d, acc[K - 1], WIDE ? 0 : lane.skip);
                    } else if (u >= t0 || (t0 == 0 && a.last)) {
                        const int row = u - (a.T - (K - 1));
                        if (row >= 0 && row < K - 1 && kept >= K - 1 - row) {
                            const T* p = reinterpret_cast<const T*>(a.dlast) + (b * (K - 1) + row) * a.D + lane.d;
#pragma unroll
                            for (int v = 0; v < V; ++v) acc[K - 1][v] += (float)p[v];
                        }
                        T* p = u >= 0 ? to + (u - t0) * a.out.st : reinterpret_cast<T*>(a.last) + (b * (K - 1) + K - 1 + u) * a.D;
                        store_row_once<T, V>(p + lane.d, acc[K - 1], WIDE ? 0 : lane.skip);
                    }
#pragma unroll
                    for (int j = K - 1; j > 0; --j)
#pragma unroll
                        for (int v = 0; v < V; ++v) {
                            seen[j][v] = seen[j - 1][v];
                            acc[j][v] = acc[j - 1][v];
                        }
                }
            };
            uint32_t words[S / 4];
            __builtin_memcpy(&words, ages + lane_item * reach + s0 - t0, S);
            bool full = true;
#pragma unroll
            for (int i = 0; i < S / 4; ++i) full = full && words[i] == 0x01010101u * K;
            const bool inner = s0 + S <= t1 && s0 >= t0 + K - 1 && (!a.dlast || s0 + S - 1 < a.T);
            if (__all(inner && full)) step(std::true_type());
            else step(std::false_type());
        }
    }
    if (!a.parts) return;
    // runs of a wavefront, then the wavefronts one after another
    __syncthreads();
    float sums[K + 1][V];
#pragma unroll
    for (int k = 0; k <= K; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            sums[k][v] = k < K ? dw[k < K ? k : 0][v] : db[v];
            for (int dist = a.F; dist < kWave; dist <<= 1) sums[k][v] += __shfl_xor(sums[k][v], dist);
        }
    const int at = f * V;                                  // [K + 1][F * V]
    for (int turn = 0; turn < kThreads / kWave; ++turn) {
        if (wave_id() == turn && lane_id() < a.F)
#pragma unroll
            for (int k = 0; k <= K; ++k)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    float* p = shared + k * a.F * V + at + v;
                    *p = sums[k][v] + (turn ? *p : 0.0f);
                }
        __syncthreads();
    }
    if ((int)threadIdx.x >= a.F || !lane.mine) return;
    float* part = a.parts + (int64_t)(blockIdx.x / a.slices) * a.D * (K + 1);
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (v >= lane.skip) {
#pragma unroll
            for (int k = 0; k < K; ++k) part[(int64_t)(lane.d + v) * K + k] = shared[k * a.F * V + at + v];
            part[(int64_t)a.D * K + lane.d + v] = shared[K * a.F * V + at + v];
        }
}

// ---------------------------------------------------------------- host

struct ConvPlan {
    int32_t V, F, slices, runs, run;
    int64_t items, groups, workgroups;       // workgroups: along the items
    bool wide;
};

inline ConvPlan conv_plan(int64_t B, int32_t T, int32_t D, int32_t K, bload_dtype dtype, bool back)
{
    ConvPlan p = {};
    p.V = conv_piece((int)att_elem_bytes(dtype), K, back);
    if (D < p.V) p.V = 1;
    const int64_t lanes = ceil_div(D, p.V);
    p.F = 1;
    while (p.F < kWave && p.F < lanes) p.F *= 2;
    p.slices = (int32_t)ceil_div(lanes, p.F);
    p.wide = p.F == kWave && D % p.V == 0;
    const int64_t each = kThreads / p.F;
    if (!back) {
        p.run = T == 1 ? 1 : 16;
    } else {
        // long runs read little twice; short ones where long ones would leave the card empty
        p.run = std::min(kConvRun, 16 * p.F);              // (ages of 4096 slots of a workgroup, at most)
        while (p.run > 16 && ceil_div(B * ceil_div(T, p.run), each) * p.slices < 1024) p.run /= 2;
    }
    p.runs = (int32_t)ceil_div(T, p.run);
    p.items = B * p.runs;
    p.groups = ceil_div(p.items, each);
    p.workgroups = back ? std::min<int64_t>(p.groups, 1024) : p.groups;
    return p;
}

// f(type, V, K)
template <typename T, bool BACK, typename F>
inline void conv_dispatch_taps(int32_t D, int32_t K, F f)
{
    using std::integral_constant;
    auto by_taps = [&](auto k) {
        constexpr int V = conv_piece(sizeof(T), k, BACK);
        if (D < V) f(type_is<T>(), integral_constant<int, 1>(), k);
        else f(type_is<T>(), integral_constant<int, V>(), k);
    };
    if (K == 1) by_taps(integral_constant<int, 1>());
    else if (K == 2) by_taps(integral_constant<int, 2>());
    else if (K == 3) by_taps(integral_constant<int, 3>());
    else if (K == 4) by_taps(integral_constant<int, 4>());
    else if (K == 5) by_taps(integral_constant<int, 5>());
    else if (K == 6) by_taps(integral_constant<int, 6>());
    else if (K == 7) by_taps(integral_constant<int, 7>());
    else by_taps(integral_constant<int, 8>());
}

inline bload_status conv_check(int64_t num_blocks, int32_t t_blk, int32_t feat_dim, int32_t taps, bload_dtype dtype)
{
    if (num_blocks < 0 || t_blk < 1 || feat_dim < 1 || taps < 1 || taps > BLOAD_CONV_MAX_TAPS || !att_dtype(dtype)) return BLOAD_EINVAL;
    if (t_blk > (1 << 30) || feat_dim > (1 << 26) || num_blocks >= ((int64_t)1 << 40) / t_blk) return BLOAD_EOVERFLOW;
    return BLOAD_OK;
}

inline bool conv_states_apart(const void* in, const void* out, int64_t bytes, int32_t t_blk)
{
    if (!in || !out || (in == out && t_blk <= 8)) return true;
    const uintptr_t p = reinterpret_cast<uintptr_t>(in), q = reinterpret_cast<uintptr_t>(out);
    return (p < q ? q - p : p - q) >= (uintptr_t)bytes;
}

inline ConvArgs conv_args(const ConvPlan& p, int32_t T, int32_t D, int32_t silu)
{
    ConvArgs a = {};
    a.items = p.items;
    a.groups = p.groups;
    a.T = T;
    a.D = D;
    a.F = p.F;
    a.slices = p.slices;
    a.runs = p.runs;
    a.run = p.run;
    a.silu = silu;
    return a;
}

}  // namespace
}  // namespace bload

using namespace bload;

extern "C" bload_status bload_segment_conv(const bload_heads* x, const float* d_weight, const float* d_bias, const uint8_t* d_reset,
                                           const uint8_t* d_valid, int64_t num_blocks, int32_t t_blk, int32_t feat_dim, int32_t taps,
                                           bload_dtype dtype, int32_t silu, const void* d_state_in, const bload_heads* out,
                                           void* d_state_out, void* hip_stream)
{
    bload_status st = conv_check(num_blocks, t_blk, feat_dim, taps, dtype);
    if (st != BLOAD_OK) return st;
    if (silu < 0 || silu > 1) return BLOAD_EINVAL;
    if (num_blocks == 0) return BLOAD_OK;
    const ConvPlan p = conv_plan(num_blocks, t_blk, feat_dim, taps, dtype, false);
    if (p.workgroups > kMaxGroups / p.slices) return BLOAD_EOVERFLOW;
    ConvArgs a = conv_args(p, t_blk, feat_dim, silu);
    if ((st = att_tensor(a.x, x, dtype)) != BLOAD_OK || (st = att_tensor(a.out, out, dtype)) != BLOAD_OK) return st;
    if (!d_weight || !d_reset || !d_valid) return BLOAD_EINVAL;
    const size_t e = att_elem_bytes(dtype);
    if (!aligned_to(d_weight, 4) || !aligned_to(d_bias, 4) || !aligned_to(d_state_in, e) || !aligned_to(d_state_out, e)) return BLOAD_EALIGN;
    if (!conv_states_apart(d_state_in, d_state_out, num_blocks * (taps - 1) * feat_dim * (int64_t)e, t_blk)) return BLOAD_EINVAL;
    a.reset = d_reset;
    a.valid = d_valid;
    a.weight = d_weight;
    a.bias = d_bias;
    a.in = d_state_in;
    a.last = d_state_out;
    const dim3 grid((unsigned)(p.workgroups * p.slices)), block(kThreads);
    by_dtype(dtype, [&](auto type) {
        conv_dispatch_taps<typename decltype(type)::type, false>(feat_dim, taps, [&](auto t, auto v, auto k) {
            using T = typename decltype(t)::type;
            if (p.run == 1) conv_kernel<T, v, k, 1, false><<<grid, block, 0, (hipStream_t)hip_stream>>>(a);
            else if (kWideTaps<v, k> && p.wide) conv_kernel<T, v, k, 16, kWideTaps<v, k>><<<grid, block, 0, (hipStream_t)hip_stream>>>(a);
            else conv_kernel<T, v, k, 16, false><<<grid, block, 0, (hipStream_t)hip_stream>>>(a);
        });
    });
    return launch_status();
}

extern "C" size_t bload_segment_conv_backward_workspace_bytes(int64_t num_blocks, int32_t t_blk, int32_t feat_dim, int32_t taps, bload_dtype dtype)
{
    if (num_blocks <= 0 || conv_check(num_blocks, t_blk, feat_dim, taps, dtype) != BLOAD_OK) return 0;
    return round_up((size_t)conv_plan(num_blocks, t_blk, feat_dim, taps, dtype, true).workgroups * feat_dim * (taps + 1) * sizeof(float), 16);
}

extern "C" bload_status bload_segment_conv_backward(const bload_heads* dout, const bload_heads* x, const float* d_weight, const float* d_bias,
                                                    const uint8_t* d_reset, const uint8_t* d_valid, int64_t num_blocks, int32_t t_blk,
                                                    int32_t feat_dim, int32_t taps, bload_dtype dtype, int32_t silu, const void* d_state_in,
                                                    const void* d_dstate_out, const bload_heads* dx, float* d_dweight, float* d_dbias,
                                                    void* d_dstate_in, void* d_workspace, size_t workspace_bytes, void* hip_stream)
{
    bload_status st = conv_check(num_blocks, t_blk, feat_dim, taps, dtype);
    if (st != BLOAD_OK) return st;
    if (silu < 0 || silu > 1) return BLOAD_EINVAL;
    if (!aligned_to(d_dweight, 4) || !aligned_to(d_dbias, 4)) return BLOAD_EALIGN;
    const bool sums = d_dweight || d_dbias;
    ColumnSums c = {};
    c.dst[0] = d_dweight;
    c.dst[1] = d_dbias;
    c.end[0] = (int64_t)feat_dim * taps;
    c.end[1] = c.columns = (int64_t)feat_dim * (taps + 1);
    const hipStream_t stream = (hipStream_t)hip_stream;
    if (num_blocks > 0) {
        const ConvPlan p = conv_plan(num_blocks, t_blk, feat_dim, taps, dtype, true);
        if (p.workgroups > kMaxGroups / p.slices) return BLOAD_EOVERFLOW;
        ConvArgs a = conv_args(p, t_blk, feat_dim, silu);
        if ((st = att_tensor(a.x, x, dtype)) != BLOAD_OK || (st = att_tensor(a.dout, dout, dtype)) != BLOAD_OK ||
            (st = att_tensor(a.out, dx, dtype)) != BLOAD_OK)
            return st;
        if (!d_weight || !d_reset || !d_valid) return BLOAD_EINVAL;
        const size_t e = att_elem_bytes(dtype);
        if (!aligned_to(d_weight, 4) || !aligned_to(d_bias, 4) || !aligned_to(d_state_in, e) || !aligned_to(d_dstate_out, e) ||
            !aligned_to(d_dstate_in, e))
            return BLOAD_EALIGN;
        const int64_t state = num_blocks * (taps - 1) * feat_dim * (int64_t)e;
        if (!conv_states_apart(d_dstate_out, d_dstate_in, state, 9) || !conv_states_apart(d_state_in, d_dstate_in, state, 9)) return BLOAD_EINVAL;
        if (sums) {
            if (!d_workspace) return BLOAD_EINVAL;
            if (!aligned_to(d_workspace, 16)) return BLOAD_EALIGN;
            if (workspace_bytes < (size_t)p.workgroups * c.columns * sizeof(float)) return BLOAD_EWORKSPACE;
            a.parts = static_cast<float*>(d_workspace);
        }
        a.reset = d_reset;
        a.valid = d_valid;
        a.weight = d_weight;
        a.bias = d_bias;
        a.in = d_state_in;
        a.dlast = d_dstate_out;
        a.last = d_dstate_in;
        const dim3 grid((unsigned)(p.workgroups * p.slices)), block(kThreads);
        const int64_t each = kThreads / p.F;
        const size_t lds = std::max<size_t>(each * (p.run + kConvHalo + 1), (size_t)p.F * p.V * (taps + 1) * sizeof(float));
        by_dtype(dtype, [&](auto type) {
            conv_dispatch_taps<typename decltype(type)::type, true>(feat_dim, taps, [&](auto t, auto v, auto k) {
                using T = typename decltype(t)::type;
                constexpr bool kWide = kWideTaps<v, k>;
                if (kWide && p.wide && silu) conv_backward_kernel<T, v, k, kWide, kWide ? 1 : -1><<<grid, block, lds, stream>>>(a);
                else if (kWide && p.wide) conv_backward_kernel<T, v, k, kWide, kWide ? 0 : -1><<<grid, block, lds, stream>>>(a);
                else conv_backward_kernel<T, v, k, false, -1><<<grid, block, lds, stream>>>(a);
            });
        });
        if ((st = launch_status()) != BLOAD_OK) return st;
        c.parts = a.parts;
        c.n_parts = p.workgroups;
    }
    return sums ? column_sums(c, stream) : BLOAD_OK;
}
