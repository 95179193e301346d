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

// ------------------------------------------------------------------ dq

constexpr int kKeys = 64;

// One row of dq from visible keys alone (see forward_row in bload_attention.hip): for rows that come
// out not finite from the matrix products.
template <typename T>
__device__ void dq_row(const AttArgs& a, int b, int head, int i, Span span)
{
    const int D = a.D, kv = head / a.G;
    const Score score(a, head);
    const int64_t at = ((int64_t)b * a.Hq + head) * a.T + i;
    const float lse = a.lse[at] * kLog2e, delta = a.delta[at];
    float q[2], g[2], acc[2] = {0.0f, 0.0f};
    load_row2(att_at<T>(a.q, b, i, head), D, q);
    load_row2(att_at<T>(a.dout, b, i, head), D, g);
    for (int j = span.lo; j < span.hi; ++j) {
        float k[2], v[2], keep;
        load_row2(att_at<T>(a.k, b, j, kv), D, k);
        load_row2(att_at<T>(a.v, b, j, kv), D, v);
        const float s = score.of<T>(wave_sum(q[0] * k[0] + q[1] * k[1]), i - j, &keep);
        const float ds = exp2_fast(s - lse) * (wave_sum(g[0] * v[0] + g[1] * v[1]) - delta) * keep;
        acc[0] += ds * k[0];
        acc[1] += ds * k[1];
    }
    store_row2(att_at<T>(a.dq, b, i, head), D, acc[0] * a.scale, acc[1] * a.scale);
}

// A workgroup takes 128 queries of one head, a wavefront 32: q and do stay in registers as B fragments, dq^T as
// the result; keys and values stream through LDS as in the forward kernel, the keys read by rows
// (for the scores) and by columns (for dq).
template <typename T, int DP, bool MOD>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) void attention_dq_kernel(AttArgs a)
{
    using L = Tile<T, DP>;
    constexpr int kSteps = DP / 16, kParts = DP / 32;
    __shared__ T ks[2][kKeys * DP], vs[2][kKeys * DP];
    __shared__ int hull[2][kThreads / kWave];
    const int lane = lane_id(), wave = wave_id();

    const uint32_t item = xcd_contiguous(blockIdx.x, gridDim.x);
    const int g = (int)(item % a.G), tile = a.tiles - 1 - (int)((item / a.G) % a.tiles);
    const int kv = (int)((item / a.G / a.tiles) % a.Hkv), b = (int)(item / a.G / a.tiles / a.Hkv);
    const int head = kv * a.G + g, D = a.D, T_ = a.T;
    const int row = tile * 128 + wave * 32 + (lane & 31);

    Span span = {0, 0};
    if (row < T_) {
        const int4 r = a.mask[(int64_t)b * T_ + row];
        span = clamp_span(r.x, r.y, T_);
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

    frag8<T> q[kSteps], go[kSteps];
    float delta = 0.0f, lse = 0.0f;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) q[s] = go[s] = frag8<T>{};
    if (row < T_) {
        const T* pq = att_at<T>(a.q, b, row, head);
        const T* pg = att_at<T>(a.dout, b, row, head);
        const T* po = att_at<T>(a.out, b, row, head);
        const T* pr = a.rest.p ? att_at<T>(a.rest, b, row, head) : nullptr;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int d = 16 * s + 8 * (lane >> 5);
            q[s] = load_frag(pq, d, D);
            go[s] = load_frag(pg, d, D);
            const frag8<T> y = load_frag(po, d, D);
            if (pr) {
                const frag8<T> z = load_frag(pr, d, D);
#pragma unroll
                for (int j = 0; j < 8; ++j) delta += (float)go[s][j] * ((float)y[j] + (float)z[j]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) delta += (float)go[s][j] * (float)y[j];
            }
        }
        lse = a.lse[((int64_t)b * a.Hq + head) * T_ + row] * kLog2e;
    }
    delta += other_half(delta);
    if (row < T_ && lane < 32) a.delta[((int64_t)b * a.Hq + head) * T_ + row] = delta;
    const Score score(a, head);
    const float c = MOD ? 1.0f : a.scale * kLog2e;

    f32x16 o[kParts];
#pragma unroll
    for (int d = 0; d < kParts; ++d) o[d] = f32x16{};
    const T* kp = att_at<T>(a.k, b, 0, kv);
    const T* vp = att_at<T>(a.v, b, 0, kv);
    Stage<T, DP, kKeys> next_k, next_v;
    if (lo < hi) {
        next_k.load(kp, a.k.st, lo, hi, D);
        next_v.load(vp, a.v.st, lo, hi, D);
    }
    int buf = 0;
    for (int k0 = lo; k0 < hi; k0 += kKeys, buf ^= 1) {
        next_k.store(ks[buf]);
        next_v.store(vs[buf]);
        __syncthreads();
        if (k0 + kKeys < hi) {
            next_k.load(kp, a.k.st, k0 + kKeys, hi, D);
            next_v.load(vp, a.v.st, k0 + kKeys, hi, D);
        }
#pragma unroll
        for (int t = 0; t < kKeys / 32; ++t) {
            if (!range.meets(k0 + 32 * t, 32)) continue;
            f32x16 x = {}, y = {};
#pragma unroll
            for (int s = 0; s < kSteps; ++s) x = mma(L::row_frag(ks[buf], 32 * t + (lane & 31), s), q[s], x);
#pragma unroll
            for (int s = 0; s < kSteps; ++s) y = mma(L::row_frag(vs[buf], 32 * t + (lane & 31), s), go[s], y);
            const int key0 = k0 + 32 * t + 4 * (lane >> 5);
            const bool full = range.full(k0 + 32 * t, 32);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int key = key0 + 8 * (i / 4) + i % 4;
                float keep = 1.0f;
                const float s = MOD ? score.of<T>(x[i], row - key, &keep) : x[i];
                const float ds = exp2_fast(fmaf(s, c, -lse)) * (y[i] - delta) * keep;
                x[i] = full || (key >= span.lo && key < span.hi) ? ds : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const frag8<T> p = pack8<T>(x, 8 * u);
#pragma unroll
                for (int d = 0; d < kParts; ++d) o[d] = mma(L::col_frag(ks[buf], 32 * t + 16 * u, 32 * d), p, o[d]);
            }
        }
    }
    bool bad = false;
#pragma unroll
    for (int d = 0; d < kParts; ++d) {
        o[d] *= a.scale;
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
    uint64_t again = __ballot(bad && span.hi > span.lo);
    again = (again | (again >> 32)) & 0xffffffffu;
    while (again) {
        const int r = __ffsll((unsigned long long)again) - 1;
        again &= again - 1;
        dq_row<T>(a, b, head, tile * 128 + wave * 32 + r, {__shfl(span.lo, r), __shfl(span.hi, r)});
    }
}

// ------------------------------------------------------------------ dk, dv

// One row of dk and dv from the queries that see it alone.
template <typename T>
__device__ void dkv_row(const AttArgs& a, int b, int kv, int j, Span span)
{
    const int D = a.D;
    float k[2], v[2], dk[2] = {0.0f, 0.0f}, dv[2] = {0.0f, 0.0f};
    load_row2(att_at<T>(a.k, b, j, kv), D, k);
    load_row2(att_at<T>(a.v, b, j, kv), D, v);
    for (int g = 0; g < a.G; ++g) {
        const int head = kv * a.G + g;
        const Score score(a, head);
        const int64_t at = ((int64_t)b * a.Hq + head) * a.T;
        for (int i = span.lo; i < span.hi; ++i) {
            float q[2], go[2], keep;
            load_row2(att_at<T>(a.q, b, i, head), D, q);
            load_row2(att_at<T>(a.dout, b, i, head), D, go);
            const float s = score.of<T>(wave_sum(q[0] * k[0] + q[1] * k[1]), i - j, &keep);
            const float p = exp2_fast(s - a.lse[at + i] * kLog2e);
            const float ds = p * (wave_sum(go[0] * v[0] + go[1] * v[1]) - a.delta[at + i]) * keep;
            for (int n = 0; n < 2; ++n) {
                dv[n] += p * go[n];
                dk[n] += ds * q[n];
            }
        }
    }
    store_row2(att_at<T>(a.dk, b, j, kv), D, dk[0] * a.scale, dk[1] * a.scale);
    store_row2(att_at<T>(a.dv, b, j, kv), D, dv[0], dv[1]);
}

constexpr int kQueries = 32;           // queries of a tile

// A workgroup takes 128 keys of one head of keys, a wavefront 32: k and v stay in registers as B fragments, dk^T and
// dv^T as results; tiles of 32 queries with their do stream through LDS, head after head of those that
// share the keys, read by rows for the scores and by columns for dk and dv.
template <typename T, int DP, bool MOD>
__global__ __launch_bounds__(kThreads, 1) void attention_dkv_kernel(AttArgs a)
{
    using L = Tile<T, DP>;
    constexpr int kSteps = DP / 16, kParts = DP / 32;
    __shared__ T qs[2][kQueries * DP], gs[2][kQueries * DP];
    __shared__ float sums[2][2][kQueries];                 // lse (in units of ln 2) and delta of the tile's queries
    __shared__ int hull[2][kThreads / kWave];
    const int lane = lane_id(), wave = wave_id(), tid = (int)threadIdx.x;

    const uint32_t item = xcd_contiguous(blockIdx.x, gridDim.x);
    const int tile = (int)(item % a.tiles);
    const int kv = (int)((item / a.tiles) % a.Hkv), b = (int)(item / a.tiles / a.Hkv);
    const int D = a.D, T_ = a.T;
    const int row = tile * 128 + wave * 32 + (lane & 31);

    Span span = {0, 0};
    if (row < T_) {
        const int4 r = a.mask[(int64_t)b * T_ + row];
        span = clamp_span(r.z, r.w, T_);
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
    const int steps = lo < hi ? (hi - lo + kQueries - 1) / kQueries : 0;

    frag8<T> k[kSteps], v[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) k[s] = v[s] = frag8<T>{};
    if (row < T_) {
        const T* pk = att_at<T>(a.k, b, row, kv);
        const T* pv = att_at<T>(a.v, b, row, kv);
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            k[s] = load_frag(pk, 16 * s + 8 * (lane >> 5), D);
            v[s] = load_frag(pv, 16 * s + 8 * (lane >> 5), D);
        }
    }
    f32x16 dk[kParts], dv[kParts];
#pragma unroll
    for (int d = 0; d < kParts; ++d) dk[d] = dv[d] = f32x16{};

    Stage<T, DP, kQueries> next_q, next_g;
    float next_sum = 0.0f;
    auto load = [&](int n) {
        const int head = kv * a.G + n / steps, q0 = lo + (n % steps) * kQueries;
        next_q.load(att_at<T>(a.q, b, 0, head), a.q.st, q0, hi, D);
        next_g.load(att_at<T>(a.dout, b, 0, head), a.dout.st, q0, hi, D);
        if (tid < 2 * kQueries) {
            const int i = q0 + (tid & (kQueries - 1));
            const int64_t at = ((int64_t)b * a.Hq + head) * T_ + i;
            next_sum = i < hi ? (tid < kQueries ? a.lse[at] * kLog2e : a.delta[at]) : 0.0f;
        }
    };
    const int all = steps * a.G;
    if (all > 0) load(0);
    int buf = 0;
    for (int n = 0; n < all; ++n, buf ^= 1) {
        next_q.store(qs[buf]);
        next_g.store(gs[buf]);
        if (tid < 2 * kQueries) sums[buf][tid / kQueries][tid & (kQueries - 1)] = next_sum;
        __syncthreads();
        if (n + 1 < all) load(n + 1);
        const int q0 = lo + (n % steps) * kQueries;
        if (!range.meets(q0, kQueries)) continue;
        const Score score(a, kv * a.G + n / steps);
        const float c = MOD ? 1.0f : a.scale * kLog2e;
        f32x16 x = {}, y = {};
#pragma unroll
        for (int s = 0; s < kSteps; ++s) x = mma(L::row_frag(qs[buf], lane & 31, s), k[s], x);
#pragma unroll
        for (int s = 0; s < kSteps; ++s) y = mma(L::row_frag(gs[buf], lane & 31, s), v[s], y);
        const bool full = range.full(q0, kQueries);
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
            const int at = 8 * i4 + 4 * (lane >> 5);
            f32x4 lse, delta;
            __builtin_memcpy(&lse, &sums[buf][0][at], 16);
            __builtin_memcpy(&delta, &sums[buf][1][at], 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int i = 4 * i4 + j, query = q0 + at + j;
                float keep = 1.0f;
                const float s = MOD ? score.of<T>(x[i], query - row, &keep) : x[i];
                const bool sees = full || (query >= span.lo && query < span.hi);
                const float p = exp2_fast(fmaf(s, c, -lse[j]));
                x[i] = sees ? p : 0.0f;
                y[i] = sees ? p * (y[i] - delta[j]) * keep : 0.0f;
            }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const frag8<T> p = pack8<T>(x, 8 * u), ds = pack8<T>(y, 8 * u);
#pragma unroll
            for (int d = 0; d < kParts; ++d) {
                dv[d] = mma(L::col_frag(gs[buf], 16 * u, 32 * d), p, dv[d]);
                dk[d] = mma(L::col_frag(qs[buf], 16 * u, 32 * d), ds, dk[d]);
            }
        }
    }
    bool bad = false;
#pragma unroll
    for (int d = 0; d < kParts; ++d) {
        dk[d] *= a.scale;
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
    uint64_t again = __ballot(bad && span.hi > span.lo);
    again = (again | (again >> 32)) & 0xffffffffu;
    while (again) {
        const int r = __ffsll((unsigned long long)again) - 1;
        again &= again - 1;
        dkv_row<T>(a, b, kv, tile * 128 + wave * 32 + r, {__shfl(span.lo, r), __shfl(span.hi, r)});
    }
}

template <typename T, int DP>
void launch(const AttArgs& a, hipStream_t stream)
{
    const dim3 block(kThreads), by_query((unsigned)((int64_t)a.B * a.Hq * a.tiles)), by_key((unsigned)((int64_t)a.B * a.Hkv * a.tiles));
    if (a.cap > 0.0f || a.slopes) {
        attention_dq_kernel<T, DP, true><<<by_query, block, 0, stream>>>(a);
        attention_dkv_kernel<T, DP, true><<<by_key, block, 0, stream>>>(a);
    } else {
        attention_dq_kernel<T, DP, false><<<by_query, block, 0, stream>>>(a);
        attention_dkv_kernel<T, DP, false><<<by_key, block, 0, stream>>>(a);
    }
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
    att_dispatch(dtype, head_dim, [&](auto type, auto dim) { launch<typename decltype(type)::type, decltype(dim)::value>(a, (hipStream_t)hip_stream); });
    return launch_status();
}
