// bload_selective_scan: a state space whose steps, inputs and outputs go by the frame, over packed blocks.
//
// Per channel d with N states, along the slots of a block:
//     step = softplus(dt + bias) (or dt + bias),   a_n = exp(step A[d, n])
//     h_n = a_n h_n + step B_n x   where the slot goes on;   h_n = step B_n x   where it starts a sequence;   0 on padding
//     y = sum_n C_n h_n + skip x;   out = y z sigmoid(z), or y
//
// The vector units bound it: an element (d, n) of a slot costs a product, an exponential (two issue slots), a product and two
// fused ones, 6 slots, and there are N of them for 8 bytes of x, step, z and out in 16 bits.  So a lane holds up to 4 states of a channel (times
// the parts of more than 16) in registers from end to end, 16 channels to a wavefront and four lanes to a channel, which share
// what is per channel and slot: a workgroup stages 16 slots of 64 channels in LDS as (step, step x), once per slot and channel, and B and C as
// floats, and its threads take the sums over states back in the same layout for skip, z and the store.  The sum over a channel's
// four lanes is three exchanges for four slots, after which each lane has one slot's.
// Blocks are walked from end to end where that fills the card; else they are cut into chunks: one launch finds each chunk's
// own part of the state behind it and the sum of its steps (the product of its a_n is exp(A_n sum)), a second joins them, a third
// computes the results from the joined states.  No workgroup waits for another one.
// States, steps, exponentials and sums are in 32 bits (a decay below 2^-126 is 0); only results are rounded to the type.
// Measured, averages among other kernels: 8 blocks of 4096 slots, 4096 channels of 16 states, bfloat16: 0.72 ms, with states saved for
// the backward pass 0.78; the vector units are busy for 0.55 of it with 35 instructions a slot and wavefront (of 16 channels), 20 of
// them the states', the rest softplus, gates and staging.  512 workgroups, two a
// compute unit: what is left are waits that two wavefronts a SIMD do not hide.  2 blocks of 4096, 2048 channels, cut into 16 chunks:
// 63 + 5 + 95 us.  One slot of 256 streams, 4096 channels: 30 us for 143 MB, 4.8 TB/s.
#include <algorithm>

#include "bload_selective.hpp"

namespace bload {
namespace {

// LDS holds two tiles: while one is computed the next is staged and the results of the one in front go out, with one barrier a tile.
// What a lane reads of LDS for four slots it reads while it computes the four in front of them.  With 16 states in 16 bits the registers
// leave room for three wavefronts a SIMD, which cut blocks use (prompt below); in float32 for two: held to three it spills 20 of them
// (8 blocks below in float32 727 -> 825 us, the prompt 158 -> 175).
template <typename T, int NS, int PARTS, bool MAPS>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 4))) void scan_kernel(ScanArgs a)
{
    constexpr int NP = 4 * NS * PARTS;
    __shared__ __attribute__((aligned(16))) float2 steps[2][kTile][kGroupC];           // step, step x
    __shared__ __attribute__((aligned(16))) float bs[2][kTile][NP], cs[2][MAPS ? 1 : kTile][NP];
    __shared__ __attribute__((aligned(16))) float ys[2][MAPS ? 1 : kTile][kGroupC];
    const ScanPlace at(a, blockIdx.x);
    const int first = at.chunk * a.chunk, end = min(first + a.chunk, a.T), col = wave_id() * kLanesC + lane_id() % kLanesC;
    const int four = at.four - at.d0;
    const bool has_state = a.in != nullptr;

    float h[PARTS][NS], rate[PARTS][NS];
    load_states<NS, PARTS>(a.rate, 0, a, at, rate);
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
        for (int i = 0; i < NS; ++i) rate[p][i] *= kLog2e, h[p][i] = 0.0f;
    if (!MAPS) {
        if (a.chunks > 1) load_states<NS, PARTS>(a.maps, at.b * a.chunks + at.chunk, a, at, h);
        else load_states<NS, PARTS>(a.in, at.b, a, at, h);
    }
    float skip[4], bias[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        skip[i] = a.skip && i < at.n_four ? a.skip[at.four + i] : 0.0f;
        bias[i] = a.dt_bias && i < at.n_four ? a.dt_bias[at.four + i] : 0.0f;
    }
    float span = 0.0f;                                     // MAPS: the lane's channel's steps so far
    bool any_cut = false;

    Stream<T> px(a.x, at, first), pdt(a.dt, at, first), pz(a.z, at, first), pout(a.out, at, first);
    PairStream<T, NP> pb(a.b, a, at, first), pc(a.c, a, at, first);
    Four<T> x, dt, z;                                      // of the tile that is staged next
    TileLook look;
    auto load = [&](int t0) {
        const bool here = t0 + at.slot < end;
        px.load(x, here);
        pdt.load(dt, here);
        if (!MAPS) pz.load(z, here && a.z.p);
        pb.load(here);
        if (!MAPS) pc.load(here);
        look.load(a, at.b, t0);
    };
    auto stage = [&](int buf, const TileFlags& flags) {
        const bool live = flags.live >> at.slot & 1;
        float2 s[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float v = dt[i] + bias[i], step = a.softplus ? softplus(v) : v;
            s[i] = live ? make_float2(step, step * x[i]) : make_float2(0.0f, 0.0f);
        }
        put_steps(&steps[buf][at.slot][four], s);
        pb.stage(bs[buf][at.slot], live);
        if (!MAPS) pc.stage(cs[buf][MAPS ? 0 : at.slot], live);
    };
    // results of a tile: the thread's four channels of its slot
    auto finish = [&](int buf, bool here, bool live, const Four<T>& x, const Four<T>& z) {
        if (!here) return;
        float y[4];
        get_four(y, &ys[buf][MAPS ? 0 : at.slot][four]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            y[i] = fmaf(skip[i], x[i], y[i]);
            if (a.z.p) y[i] *= z[i] * logistic(z[i]);
            if (!live) y[i] = 0.0f;
        }
        pout.store(y);
    };

    load(first);
    TileFlags flags = look.flags(first, end, has_state);
    stage(0, flags);
    Four<T> x_now = x, z_now = z, x_before = x, z_before = z;
    bool live_before = false;
    int buf = 0;
    for (int t0 = first; t0 < end; t0 += kTile, buf ^= 1) {
        __syncthreads();                                   // this tile is staged, the results of the one in front are there
        const bool more = t0 + kTile < end;
        if (more) load(t0 + kTile);
        if (!MAPS && a.saved) store_states<NS, PARTS>(a.saved, at.b * a.tiles + t0 / kTile, a, at, h);

        float2 s[2][4];
        float bb[2][4][NS], cc[2][4][NS], y[4];
        auto read = [&](int e) {                           // four slots of one part
            const int g = e / PARTS, p = e % PARTS, n0 = (p * 4 + at.q) * NS;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (p == 0) s[g & 1][i] = steps[buf][4 * g + i][col];
                __builtin_memcpy(&bb[e & 1][i], &bs[buf][4 * g + i][n0], sizeof(bb[0][0]));
                if (!MAPS) __builtin_memcpy(&cc[e & 1][i], &cs[buf][MAPS ? 0 : 4 * g + i][n0], sizeof(cc[0][0]));
            }
        };
        read(0);
#pragma unroll
        for (int e = 0; e < 4 * PARTS; ++e) {
            const int g = e / PARTS, p = e % PARTS;
            if (e + 1 < 4 * PARTS) read(e + 1);
            __builtin_amdgcn_sched_barrier(0);
            if (p == 0)
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = 0.0f;
            auto slot = [&](int i) {
                const float2 v = s[g & 1][i];
#pragma unroll
                for (int k = 0; k < NS; ++k) {
                    h[p][k] = fmaf(__builtin_amdgcn_exp2f(v.x * rate[p][k]), h[p][k], v.y * bb[e & 1][i][k]);
                    if constexpr (!MAPS) y[i] = fmaf(cc[e & 1][i][k], h[p][k], y[i]);
                }
                if (MAPS && p == 0) span += v.x;
            };
            if ((flags.cut >> (4 * g) & 15) == 0) {
#pragma unroll
                for (int i = 0; i < 4; ++i) slot(i);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (flags.cut >> (4 * g + i) & 1) {    // (no product with a state of 0: a decay that overflows would make it NaN)
                        const float2 v = s[g & 1][i];
#pragma unroll
                        for (int k = 0; k < NS; ++k) {
                            h[p][k] = v.y * bb[e & 1][i][k];
                            if constexpr (!MAPS) y[i] = fmaf(cc[e & 1][i][k], h[p][k], y[i]);
                        }
                        if (MAPS && p == 0) span += v.x;
                    } else {
                        slot(i);
                    }
                }
            }
            if (!MAPS && p == PARTS - 1) ys[buf][MAPS ? 0 : 4 * g + at.q][col] = sum_states(y[0], y[1], y[2], y[3]);
        }
        any_cut |= flags.cut != 0;
        if (!MAPS && t0 > first) finish(buf ^ 1, at.n_four > 0, live_before, x_before, z_before);
        live_before = flags.live >> at.slot & 1;
        x_before = x_now, z_before = z_now;
        if (more) {
            flags = look.flags(t0 + kTile, end, has_state);
            stage(buf ^ 1, flags);
            x_now = x, z_now = z;
        }
    }
    if (MAPS) {
        const int64_t row = at.b * a.chunks + at.chunk;
        store_states<NS, PARTS>(a.maps, row, a, at, h);
        if (at.mine && at.q == 0) a.spans[row * a.D + at.d] = span;
        if (threadIdx.x == 0 && at.d0 == 0) a.cut[row] = any_cut;
    } else {
        __syncthreads();
        finish(buf ^ 1, at.n_four > 0 && (end - 1) / kTile * kTile + at.slot < end, live_before, x_before, z_before);
        if (a.last && end == a.T) store_states<NS, PARTS>(a.last, at.b, a, at, h);
    }
}

// A lane takes one state of a channel through the chunks.
__global__ __launch_bounds__(kThreads) void scan_join_kernel(ScanArgs a, const float* first, int back)
{
    const int64_t each = (int64_t)a.D * a.N, n = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (n >= a.B * each) return;
    const int64_t b = n / each, dn = n - b * each, d = dn / a.N;
    const float rate = a.rate[dn] * kLog2e;
    float h = first ? first[n] : 0.0f;
    for (int c0 = 0; c0 < a.chunks; c0 += 4) {
        float own[4], span[4];
        uint8_t cut[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = min(c0 + i, a.chunks - 1);
            const int64_t row = b * a.chunks + (back ? a.chunks - 1 - c : c);
            own[i] = a.maps[row * each + dn];
            span[i] = a.spans[row * a.D + d];
            cut[i] = a.cut[row];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (c0 + i >= a.chunks) break;
            const int64_t row = b * a.chunks + (back ? a.chunks - 1 - (c0 + i) : c0 + i);
            a.maps[row * each + dn] = h;
            h = cut[i] ? own[i] : fmaf(__builtin_amdgcn_exp2f(rate * span[i]), h, own[i]);
        }
    }
    if (back && a.last) a.last[n] = h;
}

// Blocks of a few slots (one, when streams are served): bound by the states, which are read and written once.  A lane takes 4
// states of a channel, L lanes (a power of two) a channel, next to each other as they lie in memory; every state has one lane, so
// it may be advanced in place.
constexpr int kScanShort = 8;

template <typename T, int L, bool WHOLE>
__global__ __launch_bounds__(kThreads) void scan_short_kernel(ScanArgs a)
{
    const int64_t n = (int64_t)blockIdx.x * (kThreads / L) + (int)threadIdx.x / L;
    const int lane = (int)threadIdx.x % L;
    if (n >= a.B * a.D) return;
    const int64_t b = n / a.D;
    const int d = (int)(n - b * a.D), group = d / a.per, n0 = 4 * lane;
    const bool has_state = a.in != nullptr;
    float h[4], rate[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = rate[i] = 0.0f;
    auto states = [&](const float* p, float (&x)[4]) {
        if (WHOLE) {
            load_floats<4>(p + n0, x);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n0 + i < a.N) x[i] = p[n0 + i];
        }
    };
    states(a.rate + (int64_t)d * a.N, rate);
    if (a.in) states(a.in + n * a.N, h);
    const float bias = a.dt_bias ? a.dt_bias[d] : 0.0f, skip = a.skip ? a.skip[d] : 0.0f;
    for (int t = 0; t < a.T; ++t) {
        // (all loads are sent before the first is waited for; what padding holds is dropped below)
        const T x_raw = att_at<T>(a.x, b, t, 0)[d], dt_raw = att_at<T>(a.dt, b, t, 0)[d], z_raw = a.z.p ? att_at<T>(a.z, b, t, 0)[d] : (T)0.0f;
        const T *pb = att_at<T>(a.b, b, t, group) + n0, *pc = att_at<T>(a.c, b, t, group) + n0;
        RowPiece<T, 4> bb, cc;
        if (WHOLE) {
            bb.load(pb);
            cc.load(pc);
        } else {
            T some[4] = {}, more[4] = {};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n0 + i < a.N) some[i] = pb[i], more[i] = pc[i];
            __builtin_memcpy(&bb.w, &some, sizeof(some));
            __builtin_memcpy(&cc.w, &more, sizeof(more));
        }
        const int what = slot_does(a.reset + b * a.T, a.valid + b * a.T, t, has_state);
        float y = 0.0f;
        if (!what)
#pragma unroll
            for (int i = 0; i < 4; ++i) h[i] = 0.0f;
        if (what) {
            const float x = (float)x_raw, v = (float)dt_raw + bias, step = a.softplus ? softplus(v) : v;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float own = step * x * bb[i], on = fmaf(__builtin_amdgcn_exp2f(step * (rate[i] * kLog2e)), h[i], own);
                h[i] = what == 2 ? on : own;
                y = fmaf(cc[i], h[i], y);
            }
            y = fmaf(skip, x, lanes_sum<L>(y));
            if (a.z.p) y *= (float)z_raw * logistic((float)z_raw);
        }
        if (lane == 0) att_at<T>(a.out, b, t, 0)[d] = (T)y;
    }
    if (a.last) {
        float* p = a.last + n * a.N + n0;
        if (WHOLE) {
            __builtin_memcpy(p, &h, sizeof(h));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n0 + i < a.N) p[i] = h[i];
        }
    }
}

}  // namespace

struct ScanRoom {
    size_t maps, spans, cut, bytes;
};
inline ScanRoom scan_room(const ScanArgs& a)
{
    ScanRoom r = {};
    if (a.chunks > 1) {
        r.maps = round_up((size_t)a.B * a.chunks * a.D * a.N * sizeof(float), 16);
        r.spans = round_up((size_t)a.B * a.chunks * a.D * sizeof(float), 16);
        r.cut = round_up((size_t)a.B * a.chunks, 16);
    }
    r.bytes = r.maps + r.spans + r.cut;
    return r;
}
inline void scan_place_room(ScanArgs& a, void* workspace)
{
    const ScanRoom r = scan_room(a);
    if (a.chunks == 1) return;
    char* p = static_cast<char*>(workspace);
    a.maps = reinterpret_cast<float*>(p);
    a.spans = reinterpret_cast<float*>(p + r.maps);
    a.cut = reinterpret_cast<uint8_t*>(p + r.maps + r.spans);
}

bload_status scan_args(ScanArgs& a, const bload_selective* s)
{
    if (!s) return BLOAD_EINVAL;
    a = {};
    bload_status st = scan_sizes(a, s->num_blocks, s->t_blk, s->feat_dim, s->states, s->groups, s->dtype);
    if (st != BLOAD_OK) return st;
    if (s->softplus < 0 || s->softplus > 1) return BLOAD_EINVAL;
    if (s->num_blocks == 0) return BLOAD_OK;
    if ((st = att_tensor(a.x, &s->x, s->dtype)) != BLOAD_OK || (st = att_tensor(a.dt, &s->dt, s->dtype)) != BLOAD_OK ||
        (st = att_tensor(a.b, &s->b, s->dtype)) != BLOAD_OK || (st = att_tensor(a.c, &s->c, s->dtype)) != BLOAD_OK)
        return st;
    if (s->z.d_data && (st = att_tensor(a.z, &s->z, s->dtype)) != BLOAD_OK) return st;
    if (!s->d_rate || !s->d_reset || !s->d_valid) return BLOAD_EINVAL;
    if (!aligned_to(s->d_rate, 4) || !aligned_to(s->d_skip, 4) || !aligned_to(s->d_dt_bias, 4) || !aligned_to(s->d_state_in, 4))
        return BLOAD_EALIGN;
    a.rate = s->d_rate;
    a.skip = s->d_skip;
    a.dt_bias = s->d_dt_bias;
    a.reset = s->d_reset;
    a.valid = s->d_valid;
    a.in = s->d_state_in;
    a.softplus = s->softplus;
    return BLOAD_OK;
}

void scan_join(const ScanArgs& a, const float* first, bool back, hipStream_t stream)
{
    scan_join_kernel<<<dim3((unsigned)ceil_div(a.B * (int64_t)a.D * a.N, kThreads)), dim3(kThreads), 0, stream>>>(a, first, back);
}

}  // namespace bload

using namespace bload;

extern "C" size_t bload_selective_scan_workspace_bytes(int64_t num_blocks, int32_t t_blk, int32_t feat_dim, int32_t states, int32_t groups)
{
    ScanArgs a = {};
    if (num_blocks <= 0 || scan_sizes(a, num_blocks, t_blk, feat_dim, states, groups, BLOAD_F32) != BLOAD_OK || t_blk <= kScanShort) return 0;
    return scan_room(a).bytes;
}

extern "C" size_t bload_selective_scan_saved_bytes(int64_t num_blocks, int32_t t_blk, int32_t feat_dim, int32_t states, int32_t groups)
{
    ScanArgs a = {};
    if (num_blocks <= 0 || scan_sizes(a, num_blocks, t_blk, feat_dim, states, groups, BLOAD_F32) != BLOAD_OK) return 0;
    return (size_t)num_blocks * a.tiles * feat_dim * states * sizeof(float);
}

extern "C" bload_status bload_selective_scan(const bload_selective* s, const bload_heads* out, float* d_state_out, float* d_saved,
                                             void* d_workspace, size_t workspace_bytes, void* hip_stream)
{
    ScanArgs a;
    bload_status st = scan_args(a, s);
    if (st != BLOAD_OK || a.B == 0) return st;
    if ((st = att_tensor(a.out, out, s->dtype)) != BLOAD_OK) return st;
    if (!aligned_to(d_state_out, 4) || !aligned_to(d_saved, 4)) return BLOAD_EALIGN;
    if (states_meet(a.in, d_state_out, a, a.T <= kScanShort)) return BLOAD_EINVAL;
    a.last = d_state_out;
    a.saved = d_saved;
    const hipStream_t stream = (hipStream_t)hip_stream;
    const dim3 block(kThreads);
    if (a.T <= kScanShort && !d_saved) {
        by_dtype(s->dtype, [&](auto type) {
            using T = typename decltype(type)::type;
            auto go = [&](auto l, auto whole) {
                scan_short_kernel<T, l, whole><<<dim3((unsigned)ceil_div(a.B * a.D, kThreads / l)), block, 0, stream>>>(a);
            };
            auto by_lanes = [&](auto l) {
                if (a.N == 4 * l) go(l, std::true_type());
                else go(l, std::false_type());
            };
            using std::integral_constant;
            if (a.N <= 4) by_lanes(integral_constant<int, 1>());
            else if (a.N <= 8) by_lanes(integral_constant<int, 2>());
            else if (a.N <= 16) by_lanes(integral_constant<int, 4>());
            else if (a.N <= 32) by_lanes(integral_constant<int, 8>());
            else by_lanes(integral_constant<int, 16>());
        });
        return launch_status();
    }
    const ScanRoom room = scan_room(a);
    if (room.bytes) {
        if (!d_workspace) return BLOAD_EINVAL;
        if (!aligned_to(d_workspace, 16)) return BLOAD_EALIGN;
        if (workspace_bytes < room.bytes) return BLOAD_EWORKSPACE;
        scan_place_room(a, d_workspace);
    }
    const dim3 grid((unsigned)(a.B * a.G * a.slices * a.chunks));
    by_dtype(s->dtype, [&](auto type) {
        scan_by_states(a.N, [&](auto ns, auto parts) {
            using T = typename decltype(type)::type;
            if (a.chunks > 1) {
                scan_kernel<T, ns, parts, true><<<grid, block, 0, stream>>>(a);
                scan_join(a, a.in, false, stream);
            }
            scan_kernel<T, ns, parts, false><<<grid, block, 0, stream>>>(a);
        });
    });
    return launch_status();
}
