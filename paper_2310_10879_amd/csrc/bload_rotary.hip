// bload_rotary: rotary positions from the frame numbers of packed blocks.
//
// A pair (x, y) of a head's elements is turned by the angle position * frequency:
//     (x cos - y sin, y cos + x sin),
// pairs being elements i and i + rot / 2 ("half") or 2 i and 2 i + 1 ("interleaved"); the turn back,
// with the sine negated, is also the gradient.  The angle is formed in 64 bits, in turns, and reduced
// to half a turn before it is rounded to 32: position 2^24 at one radian a frame has an error of
// 2^-24 turns that way and not of a whole one.
//
// HBM bound: every element is read and written once.  A workgroup takes a few slots with all their heads.  Its threads first make
// the cosines and sines of those slots, each of them once (some 60 instructions), and leave them in LDS; then they go
// through the slots' memory from end to end, 16 bytes a lane (twice 16 where pairs lie apart), so that neighbouring lanes
// read and write side by side.  (A lane that kept its angles in registers and walked the heads with them reached 3.4 TB/s on
// 65536 slots of 40 heads of 128 bfloat16 in rows of 48: strides of a row between eight lanes and the next eight.)
#include "bload_attention_host.hpp"

namespace bload {
namespace {

constexpr int kPairs = BLOAD_ROTARY_MAX_DIM / 2;           // of a workgroup's table

struct RotaryArgs {
    AttTensor x, out;
    const int32_t* positions;        // [B, T]
    const float* freq;               // [rot / 2]
    int64_t slots;
    int32_t T, H, D, rot, places, slots_each, heads_each, inverse;
    uint32_t by_places, by_heads, by_pairs;               // 2^32 / n, rounded up: n / places = by_places * n >> 32 for small n
    float scale;
};

__device__ __forceinline__ int over(int n, uint32_t magic) { return magic ? (int)__umulhi((uint32_t)n, magic) : n; }

template <typename T, bool HALF>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a)
{
    constexpr int N = 16 / (int)sizeof(T);                 // elements of 16 bytes
    __shared__ float2 table[kPairs];                       // cosine and sine, by slot and pair
    const int64_t slot0 = (int64_t)blockIdx.x * a.slots_each;
    const int slots = (int)min((int64_t)a.slots_each, a.slots - slot0), tid = (int)threadIdx.x, pairs = a.rot / 2;
    const int h0 = (int)blockIdx.y * a.heads_each, heads = min(a.heads_each, a.H - h0);
    const int64_t b0 = slot0 / a.T;
    const int t0 = (int)(slot0 - b0 * a.T);

    for (int n = tid; n < slots * pairs; n += kThreads) {
        const int s = over(n, a.by_pairs), pos = a.positions[slot0 + s];
        const double turns = (double)pos * ((double)a.freq[n - s * pairs] * 0.15915494309189533577);
        float2 y;
        sincospif(2.0f * (float)(turns - rint(turns)), &y.y, &y.x);
        y.x *= a.scale;
        y.y *= a.inverse ? -a.scale : a.scale;
        table[n] = y;
    }
    __syncthreads();

    // the turned places first, then those that are handed through; at most N elements from `d` on
    const int turned = HALF ? (pairs + N - 1) / N : (a.rot + N - 1) / N, all = slots * a.heads_each * a.places;
    for (int n = tid; n < all; n += kThreads) {
        const int sh = over(n, a.by_places), place = n - sh * a.places, s = over(sh, a.by_heads), h = sh - s * a.heads_each;
        if (h >= heads) continue;
        int64_t b = b0;
        int t = t0 + s;
        for (; t >= a.T; t -= a.T) ++b;
        const bool turn = place < turned, live = a.positions[slot0 + s] >= 0;         // padding: zeros, whatever lies there
        const int d = turn ? place * N : a.rot + (place - turned) * N;
        const int count = min(N, (turn ? (HALF ? pairs : a.rot) : a.D) - d);
        const T* px = att_at<T>(a.x, b, t, h0 + h) + d;
        T* py = att_at<T>(a.out, b, t, h0 + h) + d;
        T u[N], w[N];
#pragma unroll
        for (int j = 0; j < N; ++j) u[j] = w[j] = (T)0.0f;
        if (live && count == N) {
            load_any(px, u);
            if (HALF && turn) load_any(px + pairs, w);
        } else if (live) {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (j < count) {
                    u[j] = px[j];
                    if (HALF && turn) w[j] = px[pairs + j];
                }
        }
        if (turn && live) {
            const float2* cs = table + s * pairs + (HALF ? d : d / 2);
#pragma unroll
            for (int j = 0; j < (HALF ? N : N / 2); ++j) {
                const float2 c = cs[min(j, (HALF ? count : count / 2) - 1)];
                const float p = (float)(HALF ? u[j] : u[2 * j]), q = (float)(HALF ? w[j] : u[2 * j + 1]);
                const T r = (T)(p * c.x - q * c.y), z = (T)(q * c.x + p * c.y);
                if constexpr (HALF) {
                    u[j] = r;
                    w[j] = z;
                } else {
                    u[2 * j] = r;
                    u[2 * j + 1] = z;
                }
            }
        }
        if (count == N) {
            __builtin_memcpy(py, &u, 16);
            if (HALF && turn) __builtin_memcpy(py + pairs, &w, 16);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (j < count) {
                    py[j] = u[j];
                    if (HALF && turn) py[pairs + j] = w[j];
                }
        }
    }
}

template <typename T>
void rotary_launch(const RotaryArgs& a, dim3 grid, bool half, hipStream_t stream)
{
    if (half) rotary_kernel<T, true><<<grid, dim3(kThreads), 0, stream>>>(a);
    else rotary_kernel<T, false><<<grid, dim3(kThreads), 0, stream>>>(a);
}

// 0 for 1, which needs no division; exact for n below 2^32 / d
inline uint32_t magic(int64_t d) { return d == 1 ? 0u : (uint32_t)(((uint64_t)1 << 32) / (uint64_t)d + 1); }

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
    if (num_blocks < 0 || t_blk < 1 || heads < 1 || head_dim < 1 || !att_dtype(dtype) || rot_dim < 2 || rot_dim % 2 || rot_dim > head_dim || rot_dim > BLOAD_ROTARY_MAX_DIM ||
        head_dim > 65536 || ((int)layout != BLOAD_ROTARY_HALF && (int)layout != BLOAD_ROTARY_INTERLEAVED) || !std::isfinite(scale) || (inverse != 0 && inverse != 1))
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
    // A place or two to a thread, as many slots as that makes, fewer where that leaves a CU less than four workgroups; where one
    // slot alone is more, its heads are shared out.
    const int64_t most = 2 * kThreads;
    const int64_t each = std::max<int64_t>(1, std::min<int64_t>({most / ((int64_t)heads * a.places), ceil_div(a.slots, 1024), kPairs / (rot_dim / 2)}));
    int64_t heads_each = each == 1 ? std::max<int64_t>(1, std::min<int64_t>(heads, most / a.places)) : heads;
    if (a.slots * ceil_div(heads, heads_each) < 1024) heads_each = std::max<int64_t>(1, ceil_div(heads * a.slots, 1024));
    a.slots_each = (int32_t)each;
    a.heads_each = (int32_t)heads_each;
    a.by_places = magic(a.places);
    a.by_heads = magic(heads_each);
    a.by_pairs = magic(rot_dim / 2);
    const int64_t groups = ceil_div(a.slots, each), parts = ceil_div(heads, heads_each);
    if (groups > kMaxGroups || parts > 65535) return BLOAD_EOVERFLOW;
    const dim3 grid((unsigned)groups, (unsigned)parts);
    if (dtype == BLOAD_F16) rotary_launch<att_half>(a, grid, half, (hipStream_t)hip_stream);
    else if (dtype == BLOAD_BF16) rotary_launch<att_bf16>(a, grid, half, (hipStream_t)hip_stream);
    else rotary_launch<float>(a, grid, half, (hipStream_t)hip_stream);
    return launch_status();
}
