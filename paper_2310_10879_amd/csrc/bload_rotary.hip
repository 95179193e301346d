// bload_rotary: rotary positions from the frame numbers of packed blocks.
//
// A pair (x, y) of a head's elements is turned by the angle position * frequency:
//     (x cos - y sin, y cos + x sin),
// pairs being elements i and i + rot / 2 ("half") or 2 i and 2 i + 1 ("interleaved"); the turn back,
// with the sine negated, is also the gradient.  The angle is formed in 64 bits, in turns, and reduced
// to half a turn before it is rounded to 32: position 2^24 at one radian a frame has an error of
// 2^-24 turns that way and not of a whole one.
//
// HBM bound: every element is read and written once.  A lane keeps one place of a slot (16 bytes of a
// head, or twice 16 where the pairs lie apart) and goes through the heads with it, so that an angle costs its some
// 60 instructions once per slot and not once per head.
#include "bload_attention_host.hpp"

namespace bload {
namespace {

struct RotaryArgs {
    AttTensor x, out;
    const int32_t* positions;        // [B, T]
    const float* freq;               // [rot / 2]
    int64_t slots;
    int32_t T, H, D, rot, places, heads_each, inverse;
    float scale;
};

template <typename T, bool HALF>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a)
{
    constexpr int N = 16 / (int)sizeof(T);                 // elements of 16 bytes
    const int64_t n = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t slot = n / a.places;
    if (slot >= a.slots) return;
    const int place = (int)(n - slot * a.places);
    const int64_t b = slot / a.T;
    const int t = (int)(slot - b * a.T);
    const int32_t pos = a.positions[slot];
    const int h0 = (int)blockIdx.y * a.heads_each, h1 = min(h0 + a.heads_each, a.H);

    // the turned places first, then those that are handed through; at most N elements from `d` on
    const int pairs = a.rot / 2;
    const int turned = HALF ? (pairs + N - 1) / N : (a.rot + N - 1) / N;
    const bool turn = place < turned;
    const int d = turn ? place * N : a.rot + (place - turned) * N;
    const int end = turn ? (HALF ? pairs : a.rot) : a.D;

    float cs[HALF ? N : N / 2], sn[HALF ? N : N / 2];
    if (turn && pos >= 0) {
#pragma unroll
        for (int j = 0; j < (HALF ? N : N / 2); ++j) {
            const int i = (HALF ? d : d / 2) + j;
            const double turns = (double)pos * ((double)a.freq[min(i, pairs - 1)] * 0.15915494309189533577);
            sincospif(2.0f * (float)(turns - rint(turns)), &sn[j], &cs[j]);
            cs[j] *= a.scale;
            sn[j] *= a.inverse ? -a.scale : a.scale;
        }
    }
    const bool whole = d + N <= end;
    auto load = [&](const T* p, int at, T (&v)[N]) {
        if (whole) {
            load_any(p + at, v);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) v[j] = d + j < end ? p[at + j] : (T)0.0f;
        }
    };
    auto store = [&](T* p, int at, const T (&v)[N]) {
        if (whole) {
            __builtin_memcpy(p + at, &v, 16);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (d + j < end) p[at + j] = v[j];
        }
    };
#pragma unroll 4
    for (int h = h0; h < h1; ++h) {
        const T* px = att_at<T>(a.x, b, t, h);
        T* py = att_at<T>(a.out, b, t, h);
        T u[N], w[N];
        if (pos < 0) {                                     // padding: zeros, whatever lies there
#pragma unroll
            for (int j = 0; j < N; ++j) u[j] = w[j] = (T)0.0f;
        } else {
            load(px, d, u);
            if (HALF && turn) load(px, d + pairs, w);
            if (turn) {
#pragma unroll
                for (int j = 0; j < (HALF ? N : N / 2); ++j) {
                    const float p = (float)(HALF ? u[j] : u[2 * j]), q = (float)(HALF ? w[j] : u[2 * j + 1]);
                    const T r = (T)(p * cs[j] - q * sn[j]), s = (T)(q * cs[j] + p * sn[j]);
                    if constexpr (HALF) {
                        u[j] = r;
                        w[j] = s;
                    } else {
                        u[2 * j] = r;
                        u[2 * j + 1] = s;
                    }
                }
            }
        }
        store(py, d, u);
        if (HALF && turn) store(py, d + pairs, w);
    }
}

template <typename T>
void rotary_launch(const RotaryArgs& a, dim3 grid, bool half, hipStream_t stream)
{
    if (half) rotary_kernel<T, true><<<grid, dim3(kThreads), 0, stream>>>(a);
    else rotary_kernel<T, false><<<grid, dim3(kThreads), 0, stream>>>(a);
}

}  // namespace
}  // namespace bload

using namespace bload;

extern "C" bload_status bload_rotary_frequencies(int32_t rot_dim, double base, double factor, int64_t trained, double slow, double fast,
                                                 float* h_freq)
{
    if (rot_dim < 2 || rot_dim % 2 || !(base > 0.0) || !(factor > 0.0) || trained < 0 || !std::isfinite(base) || !std::isfinite(factor) || !h_freq)
        return BLOAD_EINVAL;
    if (trained > 0 && !(slow < fast && std::isfinite(slow) && std::isfinite(fast))) return BLOAD_EINVAL;
    for (int32_t i = 0; i < rot_dim / 2; ++i) {
        const double f = std::pow(base, -2.0 * i / rot_dim);
        double keep = 0.0;
        if (trained > 0) {
            const double turns = (double)trained * f * 0.15915494309189533577;
            keep = std::fmin(std::fmax((turns - slow) / (fast - slow), 0.0), 1.0);
        }
        h_freq[i] = (float)(f * (keep + (1.0 - keep) / factor));
    }
    return BLOAD_OK;
}

extern "C" bload_status bload_rotary(const bload_heads* x, const int32_t* d_positions, int64_t num_blocks, int32_t t_blk, int32_t heads,
                                     int32_t head_dim, bload_dtype dtype, const float* d_freq, int32_t rot_dim, bload_rotary_layout layout,
                                     float scale, int32_t inverse, const bload_heads* out, void* hip_stream)
{
    if (num_blocks < 0 || t_blk < 1 || heads < 1 || head_dim < 1 || !att_dtype(dtype) || rot_dim < 2 || rot_dim % 2 || rot_dim > head_dim ||
        ((int)layout != BLOAD_ROTARY_HALF && (int)layout != BLOAD_ROTARY_INTERLEAVED) || !std::isfinite(scale) || (inverse != 0 && inverse != 1))
        return BLOAD_EINVAL;
    if (num_blocks >= ((int64_t)1 << 40) / t_blk) return BLOAD_EOVERFLOW;
    if (num_blocks == 0) return BLOAD_OK;
    RotaryArgs a = {};
    bload_status st;
    if ((st = att_tensor(a.x, x, dtype)) || (st = att_tensor(a.out, out, dtype))) return st;
    if (!d_positions || !d_freq) return BLOAD_EINVAL;
    if (!aligned_to(d_positions, 4) || !aligned_to(d_freq, 4)) return BLOAD_EALIGN;
    const int N = 16 / (int)att_elem_bytes(dtype);
    const bool half = layout == BLOAD_ROTARY_HALF;
    a.positions = d_positions;
    a.freq = d_freq;
    a.slots = num_blocks * t_blk;
    a.T = t_blk;
    a.H = heads;
    a.D = head_dim;
    a.rot = rot_dim;
    a.places = (int32_t)(ceil_div(half ? rot_dim / 2 : rot_dim, N) + ceil_div(head_dim - rot_dim, N));
    a.inverse = inverse;
    a.scale = scale;
    if (a.slots > (int64_t)0x7fffffff * kThreads / a.places) return BLOAD_EOVERFLOW;
    const int64_t groups = ceil_div(a.slots * a.places, kThreads);
    // all heads in one lane, unless that leaves CUs without work: then as many to a lane as give each CU four workgroups
    int64_t split = groups < 1024 ? std::min<int64_t>(heads, ceil_div(1024, groups)) : 1;
    a.heads_each = (int32_t)ceil_div(heads, split);
    split = ceil_div(heads, a.heads_each);
    const dim3 grid((unsigned)groups, (unsigned)split);
    if (dtype == BLOAD_F16) rotary_launch<att_half>(a, grid, half, (hipStream_t)hip_stream);
    else if (dtype == BLOAD_BF16) rotary_launch<att_bf16>(a, grid, half, (hipStream_t)hip_stream);
    else rotary_launch<float>(a, grid, half, (hipStream_t)hip_stream);
    return launch_status();
}
