// bload_segment_attention: attention inside the sequences of packed blocks, forward.
//
// For query i of head h, over the keys j of the interval that the mask gives it:
//     s_j = cap tanh(scale q.k_j / cap) - slope_h |i - j|,  p = softmax(s),  out = sum p_j v_j,
//     lse = ln sum e^s_j
// in one pass over the keys with a running maximum m and sum l: a tile of keys with scores s takes
// m' = max(m, s), O = O 2^(m - m') + 2^(s - m') V, l likewise; O / l in the end.
#include "bload_attention.hpp"
#include "bload_attention_host.hpp"

namespace bload {
namespace {

// Keys of a tile: 64, of float 32, so that two workgroups share a CU (LDS and registers) and one multiplies while the other
// waits at its barrier or forms probabilities.
template <typename T> constexpr int kTileKeys = sizeof(T) == 2 ? 64 : 32;

// One query again, from visible keys alone.
template <typename T>
__device__ __forceinline__ void forward_row(const AttArgs& a, int b, int head, int i, Span span)
{
    const int D = a.D, kv = head / a.G;
    float o[2], m, l;
    plain_row<T>(att_at<T>(a.q, b, i, head), att_at<T>(a.k, b, 0, kv), att_at<T>(a.v, b, 0, kv), a.k.st, a.v.st, D, Score(a, head), i, span.lo,
                 span.hi, o, m, l);
    store_row2(att_at<T>(a.out, b, i, head), D, o[0], o[1]);
    if (a.rest.p) store_row2(att_at<T>(a.rest, b, i, head), D, o[0] - (float)(T)o[0], o[1] - (float)(T)o[1]);
    if (a.lse && lane_id() == 0) a.lse[((int64_t)b * a.Hq + head) * a.T + i] = (m + log2f(l)) * kLn2;
}

// A workgroup takes 128 queries of one head, a wavefront 32 of them (they stay in its registers, as does O^T);
// tiles of keys and values go through LDS, two tiles deep, the next one on its way from memory
// while the present one is multiplied.
// Measured: 8 blocks of 4096 bfloat16, 32 heads of 128 over 8, causal: 1.45 ms, 760 TFLOP/s (a product of 8192 x 8192 matrices reaches
// 1200 on that card).  Matrix units are busy for 41 % of the cycles, vector units for 45 (exponentials), LDS for 31, at 1.8 GHz: the
// two kinds of work of the two waves of a SIMD hardly overlap.  Units of 32 keys whose exponentials stood between the products of
// their neighbours took 1.53 ms, a higher priority around products changed nothing.  16 blocks of 3000, 16 heads of 128, some 65 keys to
// a query: 0.32 ms, 3.0 TB/s, bound by the latencies of few tiles.
template <typename T, int DP, int MOD, bool ODD>
__global__ __launch_bounds__(kThreads, 2) void attention_forward_kernel(AttArgs a)
{
    using L = Tile<T, DP>;
    constexpr int kKeys = kTileKeys<T>, kHalves = kKeys / 32;
    constexpr int kSteps = DP / 16, kParts = DP / 32, kAhead = sizeof(T) == 2 ? 3 : 1;      // fragments on their way from LDS
    __shared__ T ks[2][kKeys * DP], vs[2][kKeys * DP];
    __shared__ int hull[2][kThreads / kWave];
    const int lane = lane_id(), wave = wave_id();

    // heads that share keys side by side, the latest queries (causally the longest) first
    const uint32_t item = xcd_contiguous(blockIdx.x, gridDim.x);
    const int g = (int)(item % a.G), kv = (int)((item / a.G) % a.Hkv);
    const int tile = a.tiles - 1 - (int)((item / a.Hq) % a.tiles), b = (int)(item / a.Hq / a.tiles);
    const int head = kv * a.G + g, D = a.D, T_ = a.T;
    const int row = tile * 128 + wave * 32 + (lane & 31);

    Span span = {0, 0};
    if (row < T_) {
        const int4 r = a.mask[(int64_t)b * T_ + row];
        span = clamp_span(r.x, r.y, T_);
    }
    frag8<T> q[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) q[s] = frag8<T>{};
    if (row < T_) {
        const T* p = att_at<T>(a.q, b, row, head);
#pragma unroll
        for (int s = 0; s < kSteps; ++s) q[s] = load_frag<T, ODD>(p, 16 * s + 8 * (lane >> 5), D);
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

    Stage<T, DP, kKeys, ODD> next_k(a.k.st, D), next_v(a.v.st, D);
    if (lo < hi) {
        next_k.begin(att_at<T>(a.k, b, 0, kv), lo);
        next_v.begin(att_at<T>(a.v, b, 0, kv), lo);
        next_k.load(lo, hi);
        next_v.load(lo, hi);
    }
    arrived(q);
    const Score score(a, head);
    const float c = MOD != kPlain ? 1.0f : a.scale * kLog2e;

    f32x16 o[kParts];
#pragma unroll
    for (int d = 0; d < kParts; ++d) o[d] = f32x16{};
    Maximum max;
    float l = 0.0f;

    typename L::Reader by_row = L::rows(), by_col = L::columns();
    int buf = 0;
    for (int k0 = lo; k0 < hi; k0 += kKeys, buf ^= 1) {
        next_k.store(ks[buf], hi - k0);
        next_v.store(vs[buf], hi - k0);
        __syncthreads();
        if (k0 + kKeys < hi) {
            next_k.load(k0 + kKeys, hi);
            next_v.load(k0 + kKeys, hi);
        }
        by_row.renew();
        by_col.renew();
        if (!range.meets(k0, kKeys)) continue;
        f32x16 x[kHalves] = {};
        ahead<kHalves * kSteps, kAhead>([&](int n) { return L::row_frag(ks[buf], by_row, 32 * (n / kSteps), n % kSteps); },
                                  [&](int n, frag8<T> f) { x[n / kSteps] = mma(f, q[n % kSteps], x[n / kSteps]); });
        const int key0 = k0 + 4 * (lane >> 5);
        if constexpr (MOD != kPlain) {
            const float away = (float)(row - key0);
            float keep;
#pragma unroll
            for (int t = 0; t < kHalves; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) x[t][i] = score.of<T, MOD>(x[t][i], away - (32 * t + result_row(i)), keep);
        }
        if (!range.full(k0, kKeys)) {
#pragma unroll
            for (int t = 0; t < kHalves; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) x[t][i] = span.has(key0 + 32 * t + result_row(i)) ? x[t][i] : -INFINITY;
        }
        float top = x[0][0];
#pragma unroll
        for (int t = 0; t < kHalves; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, x[t][i]);
        float f, sum = 0.0f;
        if (max.moves(halves_max(top) * c, f)) {
            l *= f;
#pragma unroll
            for (int d = 0; d < kParts; ++d) o[d] *= f;
        }
        const float base = max.base();
        auto probability = [&](int t, int i) {
            x[t][i] = exp2_fast(fmaf(x[t][i], c, -base));
            sum += x[t][i];
        };
#pragma unroll
        for (int i = 0; i < 16; ++i) probability(0, i);
        // the second half's probabilities between the products of the first
        ahead<2 * kHalves * kParts, kAhead>([&](int n) { return L::col_frag(vs[buf], by_col, 16 * (n / kParts), 32 * (n % kParts)); },
                                  [&](int n, frag8<T> f) {
                                      const int t = n / kParts, d = n % kParts;
                                      o[d] = mma(f, pack8<T>(x[t >> 1], 8 * (t & 1)), o[d]);
                                      if (kHalves == 2 && n < 2 * kParts)
#pragma unroll
                                          for (int i = 8 * n / kParts; i < 8 * (n + 1) / kParts; ++i) probability(kHalves - 1, i);
                                  });
        l += sum;
    }
    l = halves_sum(l);
    const float inv = span.hi > span.lo ? 1.0f / l : 0.0f;
    bool bad = false;
#pragma unroll
    for (int d = 0; d < kParts; ++d) {
        o[d] *= inv;
#pragma unroll
        for (int i = 0; i < 16; ++i) bad |= not_finite(o[d][i]);
        if (span.hi <= span.lo) o[d] = f32x16{};           // a row that sees nothing is 0, whatever lies around it
    }
    if (row < T_) {
        T* p = att_at<T>(a.out, b, row, head);
#pragma unroll
        for (int d = 0; d < kParts; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 y = {o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
                store4(p, 32 * d + 8 * i + 4 * (lane >> 5), D, y);
            }
        if (a.rest.p) {
            T* p = att_at<T>(a.rest, b, row, head);
#pragma unroll
            for (int d = 0; d < kParts; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    f32x4 y;
                    for (int j = 0; j < 4; ++j) y[j] = o[d][4 * i + j] - (float)(T)o[d][4 * i + j];
                    store4(p, 32 * d + 8 * i + 4 * (lane >> 5), D, y);
                }
        }
        if (a.lse && lane < 32)
            a.lse[((int64_t)b * a.Hq + head) * T_ + row] = span.hi > span.lo ? (max.m + log2f(l)) * kLn2 : -INFINITY;
    }
    if (!__any(bad && span.hi > span.lo)) return;
    const AttArgs late = args_again();
    // spoiled by what is hidden; or by sums that left float32, which those of halfs cannot: then nothing seen is at fault
    Met met;
    auto keys = [&](int r) { return row_not_finite(att_at<T>(late.k, b, r, kv), late.D) || row_not_finite(att_at<T>(late.v, b, r, kv), late.D); };
    constexpr bool kHalf = std::is_same<T, att_half>::value;
    met.look_around(span, late.T, !kHalf, keys);
    uint64_t again = __ballot(bad && span.hi > span.lo && (met.hidden || (!kHalf && !met.seen)));
    again = (again | (again >> 32)) & 0xffffffffu;
    while (again) {
        const int r = __ffsll((unsigned long long)again) - 1;
        again &= again - 1;
        forward_row<T>(late, b, head, __builtin_amdgcn_readlane(row, r), {__builtin_amdgcn_readlane(span.lo, r), __builtin_amdgcn_readlane(span.hi, r)});
    }
}

template <typename T, int DP>
void launch(const AttArgs& a, hipStream_t stream)
{
    const dim3 grid((unsigned)((int64_t)a.B * a.Hq * a.tiles)), block(kThreads);
    att_variant<T>(a, [&](auto mod, auto odd) { attention_forward_kernel<T, DP, mod.value, odd.value><<<grid, block, 0, stream>>>(a); });
}

}  // namespace
}  // namespace bload

using namespace bload;

extern "C" bload_status bload_segment_attention(const bload_heads* q, const bload_heads* k, const bload_heads* v, const int32_t* d_mask,
                                                int64_t num_blocks, int32_t t_blk, int32_t heads_q, int32_t heads_kv, int32_t head_dim,
                                                bload_dtype dtype, float scale, float cap, const float* d_slopes, const bload_heads* out,
                                                float* d_lse, const bload_heads* out_rest, void* hip_stream)
{
    AttArgs a = {};
    bload_status st = att_args(a, num_blocks, t_blk, heads_q, heads_kv, head_dim, dtype, scale, cap, d_slopes, d_mask, 128);
    if (st != BLOAD_OK) return st;
    if (num_blocks == 0) return BLOAD_OK;
    if ((st = att_tensor(a.q, q, dtype)) || (st = att_tensor(a.k, k, dtype)) || (st = att_tensor(a.v, v, dtype)) ||
        (st = att_tensor(a.out, out, dtype)))
        return st;
    if (out_rest && (st = att_tensor(a.rest, out_rest, dtype))) return st;
    if (!aligned_to(d_lse, 4)) return BLOAD_EALIGN;
    a.lse = d_lse;
    att_dispatch(dtype, head_dim, [&](auto type, auto dim) { launch<typename decltype(type)::type, decltype(dim)::value>(a, (hipStream_t)hip_stream); });
    return launch_status();
}
