// The gradients of keys and values (the formulas and the other kernel: bload_attention_backward.hip).
#include "bload_attention.hpp"
#include "bload_attention_host.hpp"

namespace bload {
namespace {

// One row of dk and dv again, from the queries that see it alone.
template <typename T>
__device__ __forceinline__ void dkv_row(const AttArgs& a, int b, int kv, int j, Span span)
{
    const int D = a.D;
    float dk[2] = {0.0f, 0.0f}, dv[2] = {0.0f, 0.0f};
    const T *k = att_at<T>(a.k, b, j, kv), *v = att_at<T>(a.v, b, j, kv);
    // a probability that is no number: no element of the rows is one; a gradient of a score: none of dk
    bool lost = false, lost_dk = false;
    for (int g = 0; g < a.G && !lost; ++g) {
        const int head = kv * a.G + g;
        const Score score(a, head);
        const int64_t at = ((int64_t)b * a.Hq + head) * a.T;
        const T *q = att_at<T>(a.q, b, 0, head), *go = att_at<T>(a.dout, b, 0, head);
        for (int i0 = span.lo; i0 < span.hi && !lost; i0 += kWave) {
            const int i = i0 + lane_id();
            float p = 0.0f, ds = 0.0f, keep, dot[2];
            if (i < span.hi) {
                row_dots<T, 2>({k, v}, {q + i * a.q.st, go + i * a.dout.st}, D, dot);
                p = exp2_fast(score.any<T>(dot[0], i - j, keep) - a.lse[at + i] * kLog2e);
                ds = p * (dot[1] - a.delta[at + i]) * keep;
            }
            lost = __any(p != p);
            lost_dk |= __any(ds != ds);
            const int count = min(span.hi - i0, kWave);
            add_rows(go + i0 * a.dout.st, a.dout.st, count, D, p, dv);
            if (!lost_dk) add_rows(q + i0 * a.q.st, a.q.st, count, D, ds, dk);
            else if (!any_finite(dv, D)) break;            // (what is lost stays lost)
        }
    }
    if (lost) dv[0] = dv[1] = NAN;
    if (lost || lost_dk) dk[0] = dk[1] = NAN;
    store_row2(att_at<T>(a.dk, b, j, kv), D, dk[0] * a.scale, dk[1] * a.scale);
    store_row2(att_at<T>(a.dv, b, j, kv), D, dv[0], dv[1]);
}

// A workgroup takes 128 keys of one head of keys, a wavefront 32: k and v stay in registers as B fragments, dk^T and
// dv^T as results; tiles of 64 queries (float: 32) with their do stream through LDS, head after head of those that
// share the keys, and are read by rows for the scores and by columns for dk and dv.  128 sums, 64 registers of operands and
// the scores leave room for one wave a SIMD, which has to overlap its own work: the order of its instructions is written out.
// Measured: 8 blocks of 4096 bfloat16, 32 heads of 128 over 8, causal: 2.92 ms, 750 TFLOP/s over its four products; matrix units are
// busy for 39 % of the cycles, vector units for 31, LDS for 30: the one wave waits for each in turn where the order leaves a gap.  16 blocks of
// 3000 short recordings, 16 heads, float16: 0.56 ms, 2.0 TB/s: one workgroup a CU waits out each latency of its few tiles.
template <typename T, int DP, int MOD, bool ODD>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 && DP <= 64 ? 2 : 1) void attention_dkv_kernel(AttArgs a)
{
    using L = Tile<T, DP>;
    constexpr int kSteps = DP / 16, kParts = DP / 32, kQueries = sizeof(T) == 2 ? 64 : 32;
    __shared__ T tiles[2][2][kQueries * DP];               // of queries and of do: one array, so that one address serves both
    __shared__ float sums[2][2][kQueries];                 // lse (in units of ln 2, less what probabilities carry) and delta of the tile's queries
    __shared__ int hull[2][kThreads / kWave];
    const int lane = lane_id(), wave = wave_id(), tid = (int)threadIdx.x;

    const uint32_t item = xcd_contiguous(blockIdx.x, gridDim.x);
    const int kv = (int)(item % a.Hkv);
    const int tile = (int)((item / a.Hkv) % a.tiles), b = (int)(item / a.Hkv / a.tiles);
    const int D = a.D, T_ = a.T;
    const int row = tile * 128 + wave * 32 + (lane & 31);

    Span span = {0, 0};
    if (row < T_) {
        const int4 r = a.mask[(int64_t)b * T_ + row];
        span = clamp_span(r.z, r.w, T_);
    }
    frag8<T> k[kSteps], v[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) k[s] = v[s] = frag8<T>{};
    if (row < T_) {
        const T* pk = att_at<T>(a.k, b, row, kv);
        const T* pv = att_at<T>(a.v, b, row, kv);
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            k[s] = load_frag<T, ODD>(pk, 16 * s + 8 * (lane >> 5), D);
            v[s] = load_frag<T, ODD>(pv, 16 * s + 8 * (lane >> 5), D);
        }
    }
    SpanRange range;
    range.of_wave(span);
    if (lane == 0) {
        hull[0][wave] = range.lo;
        hull[1][wave] = range.hi;
    }
    __syncthreads();
    const int lo = min(min(hull[0][0], hull[0][1]), min(hull[0][2], hull[0][3]));
    const int hi = max(max(hull[1][0], hull[1][1]), max(hull[1][2], hull[1][3]));

    f32x16 dk[kParts], dv[kParts];
#pragma unroll
    for (int d = 0; d < kParts; ++d) dk[d] = dv[d] = f32x16{};

    Stage<T, DP, kQueries, ODD> next_q(a.q.st, D), next_g(a.dout.st, D);
    typename L::Reader by_row = L::rows(), by_col = L::columns();
    float next_sum = 0.0f;
    const float* next_at = nullptr;                        // (of the first 64 threads: lse, delta of a query each)
    // A tile of keys begins with a head of its own: rows of one head lie in few
    // of the cache's channels.
    int turn = tile % a.G;
    auto begin = [&]() {
        const int head = kv * a.G + turn;
        next_q.begin(att_at<T>(a.q, b, 0, head), lo);
        next_g.begin(att_at<T>(a.dout, b, 0, head), lo);
        next_at = (tid < kQueries ? a.lse : a.delta) + ((int64_t)b * a.Hq + head) * T_ + lo + (tid & (kQueries - 1));
    };
    auto load = [&](int q0) {
        next_q.load(q0, hi);
        next_g.load(q0, hi);
        if (tid < 2 * kQueries) next_sum = next_at[-max(q0 + (tid & (kQueries - 1)) - (hi - 1), 0)];
        next_at += kQueries;
    };
    const float c = a.scale * kLog2e;
    // float16: probabilities carry 2^12, so that those of long sequences stay above its subnormals
    constexpr bool kHalf = std::is_same<T, att_half>::value;
    constexpr int kMore = kHalf ? 12 : 0;
    constexpr bool kAccumulators = !(sizeof(T) == 2 && DP <= 64);
    Reach reach;

    int left = lo < hi ? a.G : 0, q0 = lo;                 // heads
    if (left > 0) {
        begin();
        load(q0);
    }
    arrived(k);
    arrived(v);
    for (int buf = 0; left > 0; buf ^= 1) {
        if constexpr (kAccumulators) {
            keep_sums(dk);
            keep_sums(dv);
        }
        next_q.store(tiles[buf][0], hi - q0);
        next_g.store(tiles[buf][1], hi - q0);
        if (tid < 2 * kQueries) {
            // (a query that sees nothing has lse -infinity: no part of it may get a probability)
            float z = next_sum;
            if (tid < kQueries) z = z == -INFINITY ? INFINITY : z * kLog2e - kMore;
            sums[buf][tid / kQueries][tid & (kQueries - 1)] = z;
        }
        __syncthreads();
        const int now_head = kv * a.G + turn, now_q = q0;
        q0 += kQueries;
        if (q0 >= hi) {
            q0 = lo;
            turn = turn + 1 == a.G ? 0 : turn + 1;
            if (--left > 0) begin();
        }
        if (left > 0) load(q0);
#pragma unroll 1
        for (int t = 0; t < kQueries / 32; ++t) {
            const int q32 = now_q + 32 * t;
            if (!range.meets(q32, 32)) continue;
            const T *tq = tiles[buf][0] + 32 * t * DP, *tg = tq + kQueries * DP;
            if constexpr (!(sizeof(T) == 2 && DP > 64)) {  // (where there are registers to hold places, they are held)
                by_row.renew();
                by_col.renew();
            }
            const Score score(a, now_head);

            // Products stand between the arithmetic on the ones in front of them: scores; dp beside the exponentials; the
            // products of half of the tile beside ds of the other half.  The order is as written: in_order() ends each
            // step of it.
            constexpr int kAhead = kSteps < 4 ? kSteps : 4;    // fragments
            frag8<T> f[kAhead];
            f32x16 x = {}, y = {};
            f32x4 lse[4], delta[4];
#pragma unroll
            for (int n = 0; n < kAhead; ++n) f[n] = L::row_frag(tq, by_row, 0, n);
            in_order();
#pragma unroll
            for (int n = 0; n < kSteps; ++n) {
                x = mma(f[n % kAhead], k[n], x);
                f[n % kAhead] = n + kAhead < kSteps ? L::row_frag(tq, by_row, 0, n + kAhead) : L::row_frag(tg, by_row, 0, n + kAhead - kSteps);
                in_order();
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                __builtin_memcpy(&lse[i], &sums[buf][0][32 * t + 8 * i + 4 * (lane >> 5)], 16);
                __builtin_memcpy(&delta[i], &sums[buf][1][32 * t + 8 * i + 4 * (lane >> 5)], 16);
            }
            const int query0 = q32 + 4 * (lane >> 5);
            if (MOD == kPlain && !range.full(q32, 32)) {       // what does not see the key gets probability 0
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = span.has(query0 + result_row(i)) ? x[i] : -INFINITY;
            }
            in_order();
            frag8<T> cq[2][kParts], cg[2][kParts];
            auto column = [&](int u, int d) {
                if (d < kParts) cg[u][d] = L::col_frag(tg, by_col, 16 * u, 32 * d);
                else cq[u][d - kParts] = L::col_frag(tq, by_col, 16 * u, 32 * (d - kParts));
            };
            float keep[16];
            const float away = (float)(query0 - row);
            auto probability = [&](int i) {
                if constexpr (MOD != kPlain) {                 // (a cap makes a finite score of -infinity: hidden here, in any tile)
                    const float s = score.of<T, MOD>(x[i], away + result_row(i), keep[i]) - lse[i / 4][i % 4];
                    x[i] = exp2_fast(span.has(query0 + result_row(i)) ? s : -INFINITY);
                } else {
                    x[i] = exp2_fast(fmaf(x[i], c, -lse[i / 4][i % 4]));
                }
            };
            auto slope = [&](int i) {                          // ds / scale
                y[i] = x[i] * (y[i] - delta[i / 4][i % 4]);
                if constexpr (MOD >= kCap) y[i] *= keep[i];
            };
#pragma unroll
            for (int n = 0; n < kSteps; ++n) {
                y = mma(f[(n + kSteps) % kAhead], v[n], y);
                if (n + kAhead < kSteps) f[(n + kSteps) % kAhead] = L::row_frag(tg, by_row, 0, n + kAhead);
                else column(0, n + kAhead - kSteps);
#pragma unroll
                for (int i = n * 16 / kSteps; i < (n + 1) * 16 / kSteps; ++i) probability(i);
                in_order();
            }
#pragma unroll
            for (int d = kAhead; d < 2 * kParts; ++d) column(0, d);
            frag8<T> p = pack8<T>(x, 0), ds;
            if constexpr (kHalf) {
                // (both halves' products with p first, beside the search for the largest ds, on which the multiple depends)
                float top = 0.0f, f;
#pragma unroll
                for (int d = 0; d < kParts; ++d) {
                    dv[d] = mma(cg[0][d], p, dv[d]);
                    column(1, d);
#pragma unroll
                    for (int i = 16 * d / kParts; i < 16 * (d + 1) / kParts; ++i) {
                        slope(i);
                        top = fmaxf(top, fabsf(y[i]));
                    }
                    in_order();
                }
                if (reach.moves(halves_max(top) * reach.by, f) == Reach::kSums) {
                    if constexpr (kAccumulators) keep_sums(dk);        // (they leave their registers here, not at every step)
#pragma unroll
                    for (int d = 0; d < kParts; ++d) dk[d] *= f;
                    if constexpr (kAccumulators) keep_sums(dk);
                }
                p = pack8<T>(x, 8);
                in_order();
#pragma unroll
                for (int d = 0; d < kParts; ++d) {
                    dv[d] = mma(cg[1][d], p, dv[d]);
#pragma unroll
                    for (int i = 8 * d / kParts; i < 8 * (d + 1) / kParts; ++i) y[i] *= reach.by;
                    in_order();
                }
                ds = pack8<T>(y, 0);
#pragma unroll
                for (int d = 0; d < kParts; ++d) {
                    dk[d] = mma(cq[0][d], ds, dk[d]);
                    column(1, kParts + d);
#pragma unroll
                    for (int i = 8 + 8 * d / kParts; i < 8 + 8 * (d + 1) / kParts; ++i) y[i] *= reach.by;
                    in_order();
                }
                ds = pack8<T>(y, 8);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) slope(i);
                in_order();
                ds = pack8<T>(y, 0);
#pragma unroll
                for (int d = 0; d < 2 * kParts; ++d) {
                    if (d < kParts) dv[d] = mma(cg[0][d], p, dv[d]);
                    else dk[d - kParts] = mma(cq[0][d - kParts], ds, dk[d - kParts]);
                    column(1, d);
#pragma unroll
                    for (int i = 8 + 4 * d / kParts; i < 8 + 4 * (d + 1) / kParts; ++i) slope(i);
                    in_order();
                }
                p = pack8<T>(x, 8);
                ds = pack8<T>(y, 8);
#pragma unroll
                for (int d = 0; d < kParts; ++d) dv[d] = mma(cg[1][d], p, dv[d]);
            }
#pragma unroll
            for (int d = 0; d < kParts; ++d) dk[d] = mma(cq[1][d], ds, dk[d]);
        }
    }
    bool bad = false;
#pragma unroll
    for (int d = 0; d < kParts; ++d) {
        dk[d] *= kHalf ? a.scale / (reach.by * (1 << kMore)) : a.scale;
        if constexpr (kHalf) dv[d] *= 1.0f / (1 << kMore);
#pragma unroll
        for (int i = 0; i < 16; ++i) bad |= not_finite(dk[d][i]) || not_finite(dv[d][i]);
        if (span.hi <= span.lo) dk[d] = dv[d] = f32x16{};
    }
    if (row < T_) {
        T* pk = att_at<T>(a.dk, b, row, kv);
        T* pv = att_at<T>(a.dv, b, row, kv);
#pragma unroll
        for (int d = 0; d < kParts; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = 32 * d + 8 * i + 4 * (lane >> 5);
                const f32x4 y = {dk[d][4 * i], dk[d][4 * i + 1], dk[d][4 * i + 2], dk[d][4 * i + 3]};
                const f32x4 z = {dv[d][4 * i], dv[d][4 * i + 1], dv[d][4 * i + 2], dv[d][4 * i + 3]};
                store4(pk, at, D, y);
                store4(pv, at, D, z);
            }
    }
    if (!__any(bad && span.hi > span.lo)) return;
    const AttArgs late = args_again();
    Met met;
    for (int g = 0; g < late.G; ++g) {
        const int head = kv * late.G + g;
        const int64_t at = ((int64_t)b * late.Hq + head) * late.T;
        met.look_around(span, late.T, false, [&](int r) {
            return not_finite(late.delta[at + r]) || !(late.lse[at + r] < INFINITY) || row_not_finite(att_at<T>(late.q, b, r, head), late.D) ||
                   row_not_finite(att_at<T>(late.dout, b, r, head), late.D);
        });
    }
    uint64_t again = __ballot(bad && span.hi > span.lo && met.hidden);
    again = (again | (again >> 32)) & 0xffffffffu;
    while (again) {
        const int r = __ffsll((unsigned long long)again) - 1;
        again &= again - 1;
        dkv_row<T>(late, b, kv, __builtin_amdgcn_readlane(row, r), {__builtin_amdgcn_readlane(span.lo, r), __builtin_amdgcn_readlane(span.hi, r)});
    }
}

template <typename T, int DP>
void launch_dkv(const AttArgs& a, hipStream_t stream)
{
    const dim3 grid((unsigned)((int64_t)a.B * a.Hkv * a.tiles)), block(kThreads);
    att_variant<T>(a, [&](auto mod, auto odd) { attention_dkv_kernel<T, DP, mod.value, odd.value><<<grid, block, 0, stream>>>(a); });
}

}  // namespace

bload_status attention_dkv(const AttArgs& a, bload_dtype dtype, hipStream_t stream)
{
    att_dispatch(dtype, a.D, [&](auto type, auto dim) { launch_dkv<typename decltype(type)::type, decltype(dim)::value>(a, stream); });
    return launch_status();
}

}  // namespace bload
