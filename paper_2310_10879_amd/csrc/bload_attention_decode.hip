// bload_segment_attention_decode: one query per sequence over the packed blocks as a cache.
//
// The formulas are those of bload_attention.hip with one query; its heads that share keys are the 32
// columns of the matrix products (fewer heads leave columns idle: the products are a tenth of the time that
// the keys and values take from memory, which bounds this kernel).  A sequence's keys are cut
// into `splits` shares, a workgroup to each, and a share into tiles of 32 keys that the four wavefronts take
// in turn, each through its own part of LDS and without a barrier.  Two parts of the keys
// with (m1, l1, O1) and (m2, l2, O2) join to m = max(m1, m2), l = l1 2^(m1 - m) + l2 2^(m2 - m), O likewise: in LDS
// over the wavefronts, in a second launch over the shares.
#include <algorithm>

#include "bload_attention.hpp"
#include "bload_attention_host.hpp"

namespace bload {
namespace {

constexpr int kTileKeys = 32;

struct DecodeArgs {
    AttArgs a;
    const int32_t *block, *offset, *length;
    float* part;                     // [n_seq, Hq, splits, D + 2]: m, l and O of a share
    int64_t n_seq, blocks;
    int32_t splits, column_groups;
};

__device__ __forceinline__ int decode_length(const DecodeArgs& p, int64_t seq, int64_t& block, int& offset)
{
    block = p.block[seq];
    offset = p.offset[seq];
    const int n = p.length[seq];
    return block >= 0 && block < p.blocks && offset >= 0 && n > 0 && n <= p.a.T - offset ? n : 0;
}

// One sequence and head again, where the result is not finite: a value that is seen and infinite meets the zeros of a tile's missing
// keys, and sums of values near the largest float leave float32 (see plain_row).
template <typename T>
__device__ __forceinline__ void decode_row(const AttArgs& a, int64_t seq, int head, int64_t b, int offset, int n)
{
    const int kv = head / a.G;
    float o[2], m, l;
    plain_row<T>(att_at<T>(a.q, seq, 0, head), att_at<T>(a.k, b, offset, kv), att_at<T>(a.v, b, offset, kv), a.k.st, a.v.st, a.D, Score(a, head), n - 1,
                 0, n, o, m, l);
    store_row2(att_at<T>(a.out, seq, 0, head), a.D, o[0], o[1]);
}

// One share of one sequence for up to 32 heads of queries.  Measured: 32 blocks of 32768 slots, 8 heads of 128 bfloat16 read by 32: 0.57 ms,
// 5.7 TB/s of keys and values (tiles are read at 6.8 where nothing else is done).
template <typename T, int DP, int MOD, bool ODD>
__global__ __launch_bounds__(kThreads) void attention_decode_kernel(DecodeArgs p)
{
    using L = Tile<T, DP>;
    constexpr int kSteps = DP / 16, kParts = DP / 32, kWaves = kThreads / kWave;
    constexpr int kTile = kTileKeys * DP;
    // tiles of keys and values, later the wavefronts' results
    __shared__ __attribute__((aligned(16))) char raw[std::max<size_t>(2 * kWaves * kTile * sizeof(T), kWaves * 32 * DP * sizeof(float))];
    __shared__ float tops[kWaves][32], sums[kWaves][32];
    __shared__ int again[32], any_again;                   // heads whose result is not finite
    const AttArgs& a = p.a;
    const int lane = lane_id(), wave = wave_id(), D = a.D;
    T* ks = reinterpret_cast<T*>(raw) + wave * 2 * kTile;
    T* vs = ks + kTile;

    uint32_t item = xcd_contiguous(blockIdx.x, gridDim.x);
    const int cg = (int)(item % p.column_groups);
    item /= p.column_groups;
    const int split = (int)(item % p.splits);
    item /= p.splits;
    const int kv = (int)(item % a.Hkv);
    const int64_t seq = item / a.Hkv;
    int64_t b;
    int off;
    const int n = decode_length(p, seq, b, off);
    const int share = ((n + p.splits - 1) / p.splits + kTileKeys - 1) & ~(kTileKeys - 1);
    const int lo = min(split * share, n), hi = min(lo + share, n);

    const int column = cg * 32 + (lane & 31), head = kv * a.G + min(column, a.G - 1);
    frag8<T> q[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) q[s] = frag8<T>{};
    if (column < a.G && n > 0) {
        const T* pq = att_at<T>(a.q, seq, 0, head);
#pragma unroll
        for (int s = 0; s < kSteps; ++s) q[s] = load_frag<T, ODD>(pq, 16 * s + 8 * (lane >> 5), D);
    }
    arrived(q);
    const Score score(a, head);
    const float c = MOD != kPlain ? 1.0f : a.scale * kLog2e;
    f32x16 o[kParts];
#pragma unroll
    for (int d = 0; d < kParts; ++d) o[d] = f32x16{};
    Maximum max;
    float l = 0.0f;

    Stage<T, DP, kTileKeys, ODD, kWave> next_k(a.k.st, D), next_v(a.v.st, D);
    typename L::Reader by_row = L::rows(), by_col = L::columns();
    int k0 = lo + wave * kTileKeys;
    if (k0 < hi) {
        next_k.begin(att_at<T>(a.k, b, off, kv), k0);
        next_v.begin(att_at<T>(a.v, b, off, kv), k0);
        next_k.load(k0, hi);
        next_v.load(k0, hi);
    }
    for (; k0 < hi; k0 += kWaves * kTileKeys) {
        next_k.store(ks, kTileKeys);                       // (rows beyond hi as they are: decode_row takes care of what they spoil)
        next_v.store(vs, kTileKeys);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        const int k1 = k0 + kWaves * kTileKeys;
        if (k1 < hi) {
            next_k.skip((kWaves - 1) * kTileKeys);
            next_v.skip((kWaves - 1) * kTileKeys);
            next_k.load(k1, hi);
            next_v.load(k1, hi);
        }
        by_row.renew();
        by_col.renew();
        f32x16 x = {};
        ahead<kSteps, 1>([&](int n) { return L::row_frag(ks, by_row, 0, n); }, [&](int n, frag8<T> f) { x = mma(f, q[n], x); });
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int key = k0 + 4 * (lane >> 5) + result_row(i);
            float keep;
            if constexpr (MOD != kPlain) x[i] = score.of<T, MOD>(x[i], (float)(n - 1 - key), keep);
            x[i] = key < hi ? x[i] : -INFINITY;
            top = fmaxf(top, x[i]);
        }
        float f, sum = 0.0f;
        if (max.moves(halves_max(top) * c, f)) {
            l *= f;
#pragma unroll
            for (int d = 0; d < kParts; ++d) o[d] *= f;
        }
        const float base = max.base();
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            x[i] = exp2_fast(fmaf(x[i], c, -base));
            sum += x[i];
        }
        l += sum;
        ahead<2 * kParts, 1>([&](int n) { return L::col_frag(vs, by_col, 16 * (n / kParts), 32 * (n % kParts)); },
                             [&](int n, frag8<T> f) { o[n % kParts] = mma(f, pack8<T>(x, 8 * (n / kParts)), o[n % kParts]); });
        __builtin_amdgcn_wave_barrier();
    }
    l = halves_sum(l);

    // the wavefronts' parts to one
    __syncthreads();
    float (*acc)[32][DP] = reinterpret_cast<float (*)[32][DP]>(raw);
    if (column < a.G) {
#pragma unroll
        for (int d = 0; d < kParts; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 y = {o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
                __builtin_memcpy(&acc[wave][lane & 31][32 * d + 8 * i + 4 * (lane >> 5)], &y, 16);
            }
    }
    if (lane < 32) {
        tops[wave][lane] = max.m;
        sums[wave][lane] = l;
        if (wave == 0) again[lane] = any_again = 0;
    }
    __syncthreads();
    const int columns = min(a.G - cg * 32, 32);
    for (int e = (int)threadIdx.x; e < columns * D; e += kThreads) {
        const int col = e / D, d = e - col * D, h = kv * a.G + cg * 32 + col;
        float up = tops[0][col];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) up = fmaxf(up, tops[w][col]);
        const float base = up == -INFINITY ? 0.0f : up;
        float y = 0.0f, z = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = exp2_fast(tops[w][col] - base);
            y += f * acc[w][col][d];
            z += f * sums[w][col];
        }
        if (p.splits == 1) {
            const float r = n > 0 ? y / z : 0.0f;
            att_at<T>(a.out, seq, 0, h)[d] = (T)r;
            if (not_finite(r)) again[col] = any_again = 1;
        } else {
            float* to = p.part + ((seq * a.Hq + h) * p.splits + split) * (D + 2);
            to[2 + d] = y;
            if (d == 0) {
                to[0] = up;
                to[1] = z;
            }
        }
    }
    if (p.splits > 1) return;
    __syncthreads();
    if (!any_again) return;
    for (int col = wave; col < columns; col += kWaves)
        if (again[col]) decode_row<T>(a, seq, kv * a.G + cg * 32 + col, b, off, n);
}

// The shares of one sequence and head to one: a wavefront each.
template <typename T>
__global__ __launch_bounds__(kThreads) void attention_join_kernel(DecodeArgs p)
{
    const AttArgs& a = p.a;
    const int64_t at = (int64_t)blockIdx.x * (kThreads / kWave) + wave_id();
    if (at >= p.n_seq * a.Hq) return;
    const int64_t seq = at / a.Hq;
    const int head = (int)(at - seq * a.Hq), lane = lane_id(), D = a.D;
    int64_t b;
    int off;
    const int n = decode_length(p, seq, b, off);
    const float* part = p.part + at * p.splits * (D + 2);
    float up = -INFINITY;
    for (int s = lane; s < p.splits; s += kWave) up = fmaxf(up, part[(int64_t)s * (D + 2)]);
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) up = fmaxf(up, __shfl_xor(up, d));
    const float base = up == -INFINITY ? 0.0f : up;
    float y[2] = {0.0f, 0.0f}, z = 0.0f;
    for (int s = 0; s < p.splits; ++s) {
        const float* q = part + (int64_t)s * (D + 2);
        const float f = exp2_fast(q[0] - base);
        z += f * q[1];
        if (lane < D) y[0] += f * q[2 + lane];
        if (lane + kWave < D) y[1] += f * q[2 + lane + kWave];
    }
    const float inv = n > 0 ? 1.0f / z : 0.0f;
    if (n == 0) y[0] = y[1] = 0.0f;
    y[0] *= inv;
    y[1] *= inv;
    if (__any(not_finite(y[0]) || not_finite(y[1]))) decode_row<T>(a, seq, head, b, off, n);
    else store_row2(att_at<T>(a.out, seq, 0, head), D, y[0], y[1]);
}

// Shares: as many as make 2048 workgroups, of at least 256 keys of the longest sequence that a block can hold; eight rounds of them on the
// card for heads of 128, of which one workgroup is resident a CU, fewer for smaller ones.  The lengths are on the device, so the
// number goes by the blocks' size: many sequences (2048 with all their heads of keys) get one share however long one of them is.
inline int decode_splits(int64_t n_seq, int32_t t_blk, int32_t heads_kv, int32_t groups)
{
    const int64_t alone = n_seq * heads_kv * groups;
    return (int)std::max<int64_t>(1, std::min<int64_t>({ceil_div(2048, alone), ceil_div(t_blk, 256), 128}));
}

template <typename T, int DP>
void launch(const DecodeArgs& p, hipStream_t stream)
{
    const dim3 grid((unsigned)(p.n_seq * p.a.Hkv * p.splits * p.column_groups)), block(kThreads);
    att_variant<T>(p.a, [&](auto mod, auto odd) { attention_decode_kernel<T, DP, mod.value, odd.value><<<grid, block, 0, stream>>>(p); });
    if (p.splits > 1)
        attention_join_kernel<T><<<dim3((unsigned)ceil_div(p.n_seq * p.a.Hq, kThreads / kWave)), block, 0, stream>>>(p);
}

}  // namespace
}  // namespace bload

using namespace bload;

extern "C" size_t bload_segment_attention_decode_workspace_bytes(int64_t n_seq, int32_t t_blk, int32_t heads_q, int32_t heads_kv,
                                                                 int32_t head_dim)
{
    if (n_seq <= 0 || n_seq > BLOAD_MAX_SEQ || t_blk < 1 || heads_q < 1 || heads_kv < 1 || heads_q % heads_kv || head_dim < 1 ||
        head_dim > BLOAD_ATTENTION_MAX_HEAD_DIM)
        return 0;
    const int splits = decode_splits(n_seq, t_blk, heads_kv, (int)ceil_div(heads_q / heads_kv, 32));
    return splits == 1 ? 0 : round_up((size_t)n_seq * heads_q * splits * (head_dim + 2) * sizeof(float), 16);
}

extern "C" bload_status bload_segment_attention_decode(const bload_heads* q, const bload_heads* k, const bload_heads* v,
                                                       const int32_t* d_block_of_seq, const int32_t* d_offset_of_seq,
                                                       const int32_t* d_lengths, int64_t n_seq, int64_t num_blocks, int32_t t_blk,
                                                       int32_t heads_q, int32_t heads_kv, int32_t head_dim, bload_dtype dtype, float scale,
                                                       float cap, const float* d_slopes, const bload_heads* out, void* d_workspace,
                                                       size_t workspace_bytes, void* hip_stream)
{
    DecodeArgs p = {};
    bload_status st = att_args(p.a, 0, t_blk, heads_q, heads_kv, head_dim, dtype, scale, cap, d_slopes, nullptr, t_blk);
    if (st != BLOAD_OK) return st;
    if (n_seq < 0 || num_blocks < 0) return BLOAD_EINVAL;
    if (n_seq > BLOAD_MAX_SEQ || num_blocks >= ((int64_t)1 << 40) / t_blk) return BLOAD_EOVERFLOW;
    if (n_seq == 0) return BLOAD_OK;
    if ((st = att_tensor(p.a.q, q, dtype)) || (st = att_tensor(p.a.out, out, dtype))) return st;
    if (num_blocks > 0 && ((st = att_tensor(p.a.k, k, dtype)) || (st = att_tensor(p.a.v, v, dtype)))) return st;
    if (!d_block_of_seq || !d_offset_of_seq || !d_lengths) return BLOAD_EINVAL;
    if (!aligned_to(d_block_of_seq, 4) || !aligned_to(d_offset_of_seq, 4) || !aligned_to(d_lengths, 4)) return BLOAD_EALIGN;
    p.column_groups = (int32_t)ceil_div(p.a.G, 32);
    p.splits = decode_splits(n_seq, t_blk, heads_kv, p.column_groups);
    if (n_seq > kMaxGroups / heads_kv / p.splits / p.column_groups || (p.splits > 1 && ceil_div(n_seq * heads_q, kThreads / kWave) > kMaxGroups))
        return BLOAD_EOVERFLOW;
    const size_t need = bload_segment_attention_decode_workspace_bytes(n_seq, t_blk, heads_q, heads_kv, head_dim);
    if (need) {
        if (!d_workspace) return BLOAD_EINVAL;
        if (!aligned_to(d_workspace, 16)) return BLOAD_EALIGN;
        if (workspace_bytes < need) return BLOAD_EWORKSPACE;
    }
    p.block = d_block_of_seq;
    p.offset = d_offset_of_seq;
    p.length = d_lengths;
    p.part = static_cast<float*>(d_workspace);
    p.n_seq = n_seq;
    p.blocks = num_blocks;
    att_dispatch(dtype, head_dim, [&](auto type, auto dim) { launch<typename decltype(type)::type, decltype(dim)::value>(p, (hipStream_t)hip_stream); });
    return launch_status();
}
