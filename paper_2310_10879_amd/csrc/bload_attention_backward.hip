// bload_segment_attention_backward: the gradients of attention inside the sequences of packed blocks.
//
// With p_ij = e^(s_ij - lse_i), dp_ij = do_i . v_j, delta_i = do_i . out_i and t = tanh(scale q.k / cap):
//     ds_ij = p_ij (dp_ij - delta_i) (1 - t_ij^2) scale
//     dq_i = sum_j ds_ij k_j      dk_j = sum_i ds_ij q_i      dv_j = sum_i p_ij do_i
// Two kernels: one walks the keys of 128 queries and leaves dq and delta, the other walks the queries of
// 128 keys, over all heads that share them, and leaves dk and dv.  Both recompute the scores: 7 products of
// the size of q.k where one kernel would do with 5, but every sum is formed in one place and in
// one order, without atomic additions, so that the same inputs give the same bits.
#include "bload_attention.hpp"
#include "bload_attention_host.hpp"

namespace bload {
namespace {

constexpr int kKeys = 64;

// One row of dq again, from visible keys alone.
template <typename T>
__device__ __forceinline__ void dq_row(const AttArgs& a, int b, int head, int i, Span span)
{
    const int D = a.D, kv = head / a.G;
    const Score score(a, head);
    const int64_t at = ((int64_t)b * a.Hq + head) * a.T + i;
    const float lse = a.lse[at] * kLog2e, delta = a.delta[at];
    const T *q = att_at<T>(a.q, b, i, head), *g = att_at<T>(a.dout, b, i, head);
    const T *k = att_at<T>(a.k, b, 0, kv), *v = att_at<T>(a.v, b, 0, kv);
    float acc[2] = {0.0f, 0.0f};
    for (int j0 = span.lo; j0 < span.hi; j0 += kWave) {
        const int j = j0 + lane_id();
        float ds = 0.0f, keep, dot[2];
        if (j < span.hi) {
            row_dots<T, 2>({q, g}, {k + j * a.k.st, v + j * a.v.st}, D, dot);
            const float s = score.any<T>(dot[0], i - j, keep);
            ds = exp2_fast(s - lse) * (dot[1] - delta) * keep;
        }
        if (__any(ds != ds)) {                             // no element of the row is a number
            acc[0] = acc[1] = NAN;
            break;
        }
        add_rows(k + j0 * a.k.st, a.k.st, min(span.hi - j0, kWave), D, ds, acc);
    }
    store_row2(att_at<T>(a.dq, b, i, head), D, acc[0] * a.scale, acc[1] * a.scale);
}

// A workgroup takes 128 queries of one head, a wavefront 32: q and do stay in registers as B fragments, dq^T as
// the result; keys and values stream through LDS as in the forward kernel, the keys read by rows
// (for the scores) and by columns (for dq).
// Measured: 8 blocks of 4096 bfloat16, 32 heads of 128 over 8, causal: 1.83 ms, 900 TFLOP/s over its three products (a product of
// 8192 x 8192 matrices: 1200); matrix units busy for 47 % of the cycles, vector units for 43, LDS for 32.  16 blocks of 3000 short recordings,
// 16 heads, float16: 0.42 ms, 3.3 TB/s.
template <typename T, int DP, int MOD, bool ODD>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) void attention_dq_kernel(AttArgs a)
{
    using L = Tile<T, DP>;
    constexpr int kSteps = DP / 16, kParts = DP / 32, kAhead = 1;      // fragments on their way from LDS
    __shared__ T ks[2][kKeys * DP], vs[2][kKeys * DP];
    __shared__ int hull[2][kThreads / kWave];
    const int lane = lane_id(), wave = wave_id();

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
    frag8<T> q[kSteps], go[kSteps], y[kSteps], z[kSteps];
    float lse = 0.0f;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) q[s] = go[s] = y[s] = z[s] = frag8<T>{};
    if (row < T_) {
        const T* pq = att_at<T>(a.q, b, row, head);
        const T* pg = att_at<T>(a.dout, b, row, head);
        const T* po = att_at<T>(a.out, b, row, head);
        const T* pr = a.rest.p ? att_at<T>(a.rest, b, row, head) : nullptr;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int d = 16 * s + 8 * (lane >> 5);
            q[s] = load_frag<T, ODD>(pq, d, D);
            go[s] = load_frag<T, ODD>(pg, d, D);
            y[s] = load_frag<T, ODD>(po, d, D);
            if (pr) z[s] = load_frag<T, ODD>(pr, d, D);
        }
        lse = a.lse[((int64_t)b * a.Hq + head) * T_ + row] * kLog2e;
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
    float delta = 0.0f;
#pragma unroll
    for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int j = 0; j < 8; ++j) delta += (float)go[s][j] * ((float)y[s][j] + (float)z[s][j]);
    delta = halves_sum(delta);
    if (row < T_ && lane < 32) a.delta[((int64_t)b * a.Hq + head) * T_ + row] = delta;
    arrived(q);
    arrived(go);
    const Score score(a, head);
    const float c = a.scale * kLog2e;

    f32x16 o[kParts];
#pragma unroll
    for (int d = 0; d < kParts; ++d) o[d] = f32x16{};
    constexpr bool kHalf = std::is_same<T, att_half>::value;
    Reach reach;
    typename L::Reader by_row = L::rows(), by_col = L::columns();
    int buf = 0;
    for (int k0 = lo; k0 < hi; k0 += kKeys, buf ^= 1) {
        if constexpr (sizeof(T) == 4) keep_sums(o);
        next_k.store(ks[buf], hi - k0);
        next_v.store(vs[buf], hi - k0);
        __syncthreads();
        if (k0 + kKeys < hi) {
            next_k.load(k0 + kKeys, hi);
            next_v.load(k0 + kKeys, hi);
        }
        by_row.renew();
        by_col.renew();
#pragma unroll
        for (int t = 0; t < kKeys / 32; ++t) {
            if (!range.meets(k0 + 32 * t, 32)) continue;
            f32x16 x = {}, y = {};
            ahead<2 * kSteps, kAhead>([&](int n) { return n < kSteps ? L::row_frag(ks[buf], by_row, 32 * t, n) : L::row_frag(vs[buf], by_row, 32 * t, n - kSteps); },
                                      [&](int n, frag8<T> f) {
                                          if (n < kSteps) x = mma(f, q[n], x);
                                          else y = mma(f, go[n - kSteps], y);
                                      });
            const int key0 = k0 + 32 * t + 4 * (lane >> 5);
            if (MOD == kPlain && !range.full(k0 + 32 * t, 32)) {       // what is hidden gets probability 0
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] = span.has(key0 + result_row(i)) ? x[i] : -INFINITY;
            }
            const float away = (float)(row - key0);
            const float less = kHalf ? delta * reach.by : delta;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                y[i] = kHalf ? fmaf(y[i], reach.by, -less) : y[i] - less;
                if constexpr (MOD != kPlain) {                 // (a cap makes a finite score of -infinity: hidden here, in any tile)
                    float keep;
                    const float s = score.of<T, MOD>(x[i], away - result_row(i), keep) - lse;
                    x[i] = exp2_fast(span.has(key0 + result_row(i)) ? s : -INFINITY);
                    if constexpr (MOD >= kCap) y[i] *= keep;
                } else {
                    x[i] = exp2_fast(fmaf(x[i], c, -lse));
                }
                x[i] *= y[i];
            }
            if constexpr (kHalf) {
                in_order();                                    // (with what follows among it some instances need more registers than there are)
                float top = 0.0f, f;
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(x[i]));
                if (const int moved = reach.moves(halves_max(top), f)) {
                    x *= f;
                    if (moved == Reach::kSums) {
#pragma unroll
                        for (int d = 0; d < kParts; ++d) o[d] *= f;
                    }
                }
            }
            ahead<2 * kParts, kAhead>([&](int n) { return L::col_frag(ks[buf], by_col, 32 * t + 16 * (n / kParts), 32 * (n % kParts)); },
                                      [&](int n, frag8<T> f) { o[n % kParts] = mma(f, pack8<T>(x, 8 * (n / kParts)), o[n % kParts]); });
        }
    }
    bool bad = false;
#pragma unroll
    for (int d = 0; d < kParts; ++d) {
        o[d] *= kHalf ? a.scale / reach.by : a.scale;
#pragma unroll
        for (int i = 0; i < 16; ++i) bad |= not_finite(o[d][i]);
        if (span.hi <= span.lo) o[d] = f32x16{};
    }
    if (row < T_) {
        T* p = att_at<T>(a.dq, b, row, head);
#pragma unroll
        for (int d = 0; d < kParts; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 y = {o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
                store4(p, 32 * d + 8 * i + 4 * (lane >> 5), D, y);
            }
    }
    if (!__any(bad && span.hi > span.lo)) return;
    const AttArgs late = args_again();
    Met met;
    met.look_around(span, late.T, false, [&](int r) { return row_not_finite(att_at<T>(late.k, b, r, kv), late.D) || row_not_finite(att_at<T>(late.v, b, r, kv), late.D); });
    uint64_t again = __ballot(bad && span.hi > span.lo && met.hidden);
    again = (again | (again >> 32)) & 0xffffffffu;
    while (again) {
        const int r = __ffsll((unsigned long long)again) - 1;
        again &= again - 1;
        dq_row<T>(late, b, head, __builtin_amdgcn_readlane(row, r), {__builtin_amdgcn_readlane(span.lo, r), __builtin_amdgcn_readlane(span.hi, r)});
    }
}

template <typename T, int DP>
void launch_dq(const AttArgs& a, hipStream_t stream)
{
    const dim3 grid((unsigned)((int64_t)a.B * a.Hq * a.tiles)), block(kThreads);
    att_variant<T>(a, [&](auto mod, auto odd) { attention_dq_kernel<T, DP, mod.value, odd.value><<<grid, block, 0, stream>>>(a); });
}

}  // namespace
}  // namespace bload

using namespace bload;

extern "C" size_t bload_segment_attention_backward_workspace_bytes(int64_t num_blocks, int32_t t_blk, int32_t heads_q)
{
    if (num_blocks <= 0 || t_blk < 1 || heads_q < 1 || t_blk > (1 << 30) || num_blocks >= ((int64_t)1 << 40) / t_blk) return 0;
    return round_up((size_t)num_blocks * t_blk * heads_q * sizeof(float), 16);
}

extern "C" bload_status bload_segment_attention_backward(const bload_heads* dout, const bload_heads* q, const bload_heads* k,
                                                         const bload_heads* v, const bload_heads* out, const float* d_lse,
                                                         const bload_heads* out_rest, const int32_t* d_mask, int64_t num_blocks,
                                                         int32_t t_blk, int32_t heads_q, int32_t heads_kv, int32_t head_dim,
                                                         bload_dtype dtype, float scale, float cap, const float* d_slopes,
                                                         const bload_heads* dq, const bload_heads* dk, const bload_heads* dv,
                                                         void* d_workspace, size_t workspace_bytes, void* hip_stream)
{
    AttArgs a = {};
    bload_status st = att_args(a, num_blocks, t_blk, heads_q, heads_kv, head_dim, dtype, scale, cap, d_slopes, d_mask, 128);
    if (st != BLOAD_OK) return st;
    if (num_blocks == 0) return BLOAD_OK;
    if ((st = att_tensor(a.dout, dout, dtype)) || (st = att_tensor(a.q, q, dtype)) || (st = att_tensor(a.k, k, dtype)) ||
        (st = att_tensor(a.v, v, dtype)) || (st = att_tensor(a.out, out, dtype)) || (st = att_tensor(a.dq, dq, dtype)) ||
        (st = att_tensor(a.dk, dk, dtype)) || (st = att_tensor(a.dv, dv, dtype)))
        return st;
    if (out_rest && (st = att_tensor(a.rest, out_rest, dtype))) return st;
    if (!d_lse || !d_workspace) return BLOAD_EINVAL;
    if (!aligned_to(d_lse, 4) || !aligned_to(d_workspace, 16)) return BLOAD_EALIGN;
    if (workspace_bytes < bload_segment_attention_backward_workspace_bytes(num_blocks, t_blk, heads_q)) return BLOAD_EWORKSPACE;
    a.lse = const_cast<float*>(d_lse);
    a.delta = static_cast<float*>(d_workspace);
    att_dispatch(dtype, head_dim, [&](auto type, auto dim) { launch_dq<typename decltype(type)::type, decltype(dim)::value>(a, (hipStream_t)hip_stream); });
    if ((st = launch_status()) != BLOAD_OK) return st;
    return attention_dkv(a, dtype, (hipStream_t)hip_stream);
}
