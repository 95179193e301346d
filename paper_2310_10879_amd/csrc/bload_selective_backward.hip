// bload_selective_scan_backward: the gradients of bload_selective_scan.
//
// With dy = dout z sigmoid(z) (or dout), and from the last slot to the first
//     g_n = C_n dy + u_n,   u_n = a_n g_n for the slot in front (0 where this one does not go on),   p_n = u_n h_n(front)
//     dC_n = sum_d dy h_n,   dB_n = sum_d step x g_n,   q = sum_n g_n B_n,   w = sum_n p_n A_n
//     dx = step q + skip dy,   dstep = w + x q,   ddt = dstep sigmoid(dt + bias),   dA_n = sum p_n step,
//     dskip = sum dy x,   dbias = sum ddt,   dz = dout y sigmoid(z) (1 + z (1 - sigmoid(z)))
//
// Lanes, tiles and chunks are those of the forward pass, whose state in front of every tile of 16 slots is read
// back: from it a lane forms the tile's states again and keeps them, and the decays, in registers on the way back.  Sums over states
// are exchanges between the four lanes of a channel; sums over channels (dB, dC) halve 2 NS values four times between 16 lanes,
// then the workgroup's wavefronts through LDS, and leave a share for each slice of 64 channels, which a
// last kernel adds in a fixed order.  The gradients of A, skip and bias stay in registers and are added by column_sums.
//
// States and decays of 16 slots at once do not fit beside two wavefronts a SIMD (5.0 ms in the case below, one wavefront): a lane holds
// 8, the second half of a tile first, for which the first half's states are formed once more in front (3 of some 23
// issue slots of an element).  A state saved for every 8 slots in place of 16 would save those and cost as much in bytes.
// Measured, average among other kernels: 8 blocks of 4096 slots, 4096 channels of 16 states, bfloat16, with z: 2.43 ms, the vector units
// busy for 1.7 of them: 114
// instructions a slot and wavefront of 16 channels, 8 for the first half again, 22 for states, decays and y, 32 on the
// way back, 30 for dB and dC, the rest staging, gates and sums.
#include <algorithm>

#include "bload_selective.hpp"

namespace bload {
namespace {

// One halving: of n values in every lane, n / 2, each with the partner's; lanes with `upper` keep the upper half.
template <int CTRL, int N>
__device__ __forceinline__ void halve(float (&v)[N], int n, bool upper)
{
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        if (i >= n / 2) break;
        const float keep = upper ? v[i + n / 2] : v[i], send = upper ? v[i] : v[i + n / 2];
        v[i] = keep + dpp_move<CTRL>(send, 0.0f);
    }
}
constexpr int kMirror = 0x140, kHalfMirror = 0x141, kQuadSwap2 = 0x4e, kQuadSwap1 = 0xb1;

// Of N (2, 4 or 8) values of one slot in every lane the sums over the 16 lanes of a row, but for the last step, from lane to
// neighbour: the lane has that of value `channel_value`.  The last step is for two slots together: even lanes get the first one's.
template <int N>
__device__ __forceinline__ float sum_channels(float (&v)[N])
{
    const int lane = lane_id();
    halve<kMirror, N>(v, N, lane & 8);
    if constexpr (N >= 4) halve<kHalfMirror, N>(v, N / 2, lane & 4);
    else v[0] += dpp_move<kHalfMirror>(v[0], 0.0f);
    if constexpr (N >= 8) halve<kQuadSwap2, N>(v, N / 4, lane & 2);
    else v[0] += dpp_move<kQuadSwap2>(v[0], 0.0f);
    return v[0];
}
__device__ __forceinline__ float sum_pairs(float even, float odd)
{
    const bool upper = lane_id() & 1;
    const float keep = upper ? odd : even, send = upper ? even : odd;
    return keep + dpp_move<kQuadSwap1>(send, 0.0f);
}
template <int N>
__device__ __forceinline__ int channel_value(int lane)
{
    return N == 8 ? lane >> 1 & 7 : (N == 4 ? lane >> 2 & 3 : lane >> 3 & 1);
}

// A chunk's own part of the gradient in front of it, from its end to its start.
template <typename T, int NS, int PARTS>
__global__ __launch_bounds__(kThreads) void scan_backward_maps_kernel(ScanArgs a)
{
    constexpr int NP = 4 * NS * PARTS;
    __shared__ __attribute__((aligned(16))) float2 steps[2][kTile][kGroupC];           // step, dy
    __shared__ __attribute__((aligned(16))) float cs[2][kTile][NP];
    const ScanPlace at(a, blockIdx.x);
    const int first = at.chunk * a.chunk, end = min(first + a.chunk, a.T), col = wave_id() * kLanesC + lane_id() % kLanesC;
    const int four = at.four - at.d0, last_tile = first + (end - first - 1) / kTile * kTile;
    float u[PARTS][NS], rate[PARTS][NS], bias[4];
    load_states<NS, PARTS>(a.rate, 0, a, at, rate);
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
        for (int i = 0; i < NS; ++i) rate[p][i] *= kLog2e, u[p][i] = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) bias[i] = a.dt_bias && i < at.n_four ? a.dt_bias[at.four + i] : 0.0f;
    float span = 0.0f;
    bool any_cut = false;
    Stream<T, true> pdt(a.dt, at, last_tile), pz(a.z, at, last_tile), pdo(a.dout, at, last_tile);
    PairStream<T, NP, true> pc(a.c, a, at, last_tile);
    Four<T> dt, z, dout;
    TileLook look;
    auto load = [&](int t0) {
        const bool here = t0 + at.slot < end;
        pdt.load(dt, here);
        pdo.load(dout, here);
        pz.load(z, here && a.z.p);
        pc.load(here);
        look.load(a, at.b, t0);
    };
    auto stage = [&](int buf, const TileFlags& flags) {
        const bool live = flags.live >> at.slot & 1;
        float2 s[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float v = dt[i] + bias[i], step = a.softplus ? softplus(v) : v;
            float dy = dout[i];
            if (a.z.p) dy *= z[i] * logistic(z[i]);
            s[i] = live ? make_float2(step, dy) : make_float2(0.0f, 0.0f);
        }
        put_steps(&steps[buf][at.slot][four], s);
        pc.stage(cs[buf][at.slot], live);
    };
    load(last_tile);
    TileFlags flags = look.flags(last_tile, end, a.in != nullptr);
    stage(0, flags);
    int buf = 0;
    for (int t0 = last_tile; t0 >= first; t0 -= kTile, buf ^= 1) {
        __syncthreads();
        const bool more = t0 > first;
        if (more) load(t0 - kTile);
#pragma unroll
        for (int t = kTile - 1; t >= 0; --t) {
            const float2 s = steps[buf][t][col];
            span += s.x;
            if (flags.live >> t & 1)
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    float cc[NS];
                    __builtin_memcpy(&cc, &cs[buf][t][(p * 4 + at.q) * NS], sizeof(cc));
#pragma unroll
                    for (int i = 0; i < NS; ++i) u[p][i] = __builtin_amdgcn_exp2f(s.x * rate[p][i]) * fmaf(cc[i], s.y, u[p][i]);
                }
            if (flags.cut >> t & 1)
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
#pragma unroll
                    for (int i = 0; i < NS; ++i) u[p][i] = 0.0f;
        }
        any_cut |= flags.cut != 0;
        if (more) {
            flags = look.flags(t0 - kTile, end, a.in != nullptr);
            stage(buf ^ 1, flags);
        }
    }
    const int64_t row = at.b * a.chunks + at.chunk;
    store_states<NS, PARTS>(a.maps, row, a, at, u);
    if (at.mine && at.q == 0) a.spans[row * a.D + at.d] = span;
    if (threadIdx.x == 0 && at.d0 == 0) a.cut[row] = any_cut;
}

template <typename T, int NS, int PARTS>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(PARTS == 1 ? 2 : 1, 2))) void scan_backward_kernel(ScanArgs a)
{
    constexpr int NP = 4 * NS * PARTS, kWaves = kThreads / kWave, kRun = 8;
    __shared__ __attribute__((aligned(16))) float2 steps[kTile][kGroupC];              // step, step x
    __shared__ __attribute__((aligned(16))) float dys[kTile][kGroupC], ys[kTile][kGroupC], qs[kTile][kGroupC], ws[kTile][kGroupC];
    __shared__ __attribute__((aligned(16))) float bs[kTile][NP], cs[kTile][NP];
    __shared__ float sums[kWaves][kTile][2][NP];           // dB and dC of a wavefront's channels
    __shared__ __attribute__((aligned(16))) float drates[PARTS][kThreads][NS], losts[PARTS][kThreads][NS];       // a lane's sums of dA so far
    __shared__ Four<T> kept[4][kThreads];                  // a thread's x, dt, z and dout until the tile's results go out
    __shared__ __attribute__((aligned(16))) float skips[kGroupC], biases[kGroupC], dskips[kTile][kGroupC], dbiases[kTile][kGroupC];
    ScanPlace at(a, blockIdx.x);
    const int first = at.chunk * a.chunk, end = min(first + a.chunk, a.T), col = wave_id() * kLanesC + lane_id() % kLanesC;
    const int four = at.four - at.d0, last_tile = first + (end - first - 1) / kTile * kTile;
    const int64_t part = at.b * a.chunks + at.chunk;
    const bool has_state = a.in != nullptr, gated = a.z.p != nullptr;
    const int lane = lane_id() % 16, value = channel_value<2 * NS>(lane);              // whose sums over channels the lane gets
    float* my_sums = &sums[wave_id()][lane & 1][value / NS][at.q * NS + value % NS];    // of even slots or odd ones

    float rate[PARTS][NS];
    load_states<NS, PARTS>(a.rate, 0, a, at, rate);
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            rate[p][i] *= kLog2e;
            drates[p][threadIdx.x][i] = losts[p][threadIdx.x][i] = 0.0f;
        }
    if ((int)threadIdx.x < kGroupC) {
        const int d = at.d0 + (int)threadIdx.x;
        skips[threadIdx.x] = a.skip && d < at.d1 ? a.skip[d] : 0.0f;
        biases[threadIdx.x] = a.dt_bias && d < at.d1 ? a.dt_bias[d] : 0.0f;
    }
    {
        const float none[4] = {};
        put_four(&dskips[at.slot][four], none);
        put_four(&dbiases[at.slot][four], none);
    }
    __syncthreads();
    for (; at.b < a.B; at.b += a.blocks) {
        float u[PARTS][NS];
        if (a.chunks > 1) load_states<NS, PARTS>(a.maps, at.b * a.chunks + at.chunk, a, at, u);
        else load_states<NS, PARTS>(a.dlast, at.b, a, at, u);
        Stream<T, true> px(a.x, at, last_tile), pdt(a.dt, at, last_tile), pz(a.z, at, last_tile), pdo(a.dout, at, last_tile);
        Stream<T, true> pdx(a.dx, at, last_tile), pddt(a.ddt, at, last_tile), pdz(a.dz, at, last_tile);
        PairStream<T, NP, true> pb(a.b, a, at, last_tile), pc(a.c, a, at, last_tile);
        Four<T> x, dt, z, dout;
        TileLook look;
        float h0[PARTS][NS];
        auto load = [&](int t0) {
            const bool here = t0 + at.slot < end;
            px.load(x, here);
            pdt.load(dt, here);
            pdo.load(dout, here);
            pz.load(z, here && gated);
            pb.load(here);
            pc.load(here);
            look.load(a, at.b, t0);
        };
        auto load_front = [&](int t0) { load_states<NS, PARTS>(a.saved, at.b * a.tiles + t0 / kTile, a, at, h0); };
        load(last_tile);
        load_front(last_tile);
        for (int t0 = last_tile; t0 >= first; t0 -= kTile) {
            const TileFlags flags = look.flags(t0, end, has_state);
            const bool live = flags.live >> at.slot & 1;
            {
                float2 s[4];
                float dy[4], bias[4];
                get_four(bias, &biases[four]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float v = dt[i] + bias[i], step = a.softplus ? softplus(v) : v;
                    dy[i] = dout[i];
                    if (gated) dy[i] *= z[i] * logistic(z[i]);
                    s[i] = live ? make_float2(step, step * x[i]) : make_float2(0.0f, 0.0f);
                    dy[i] = live ? dy[i] : 0.0f;
                }
                put_steps(&steps[at.slot][four], s);
                put_four(&dys[at.slot][four], dy);
                pb.stage(bs[at.slot], live);
                pc.stage(cs[at.slot], live);
            }
            kept[0][threadIdx.x] = x;
            kept[1][threadIdx.x] = dt;
            kept[2][threadIdx.x] = z;
            kept[3][threadIdx.x] = dout;
            __syncthreads();
            if (t0 > first) load(t0 - kTile);

            // A lane keeps the states and decays of kRun slots in registers: the tile's runs from the last to the first, their states
            // from that in front of the tile.
            auto tile = [&](auto all_go_on) {
                constexpr bool kAll = decltype(all_go_on)::value;
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    const int n0 = (p * 4 + at.q) * NS;
                    float start[kTile / kRun][NS], dr[NS];
#pragma unroll
                    for (int i = 0; i < NS; ++i) start[0][i] = h0[p][i], dr[i] = 0.0f;
#pragma unroll
                    for (int r = 1; r < kTile / kRun; ++r) {
#pragma unroll
                        for (int i = 0; i < NS; ++i) start[r][i] = start[r - 1][i];
#pragma unroll
                        for (int t = (r - 1) * kRun; t < r * kRun; ++t) {
                            const float2 s = steps[t][col];
                            float bb[NS];
                            __builtin_memcpy(&bb, &bs[t][n0], sizeof(bb));
                            const bool cut = !kAll && (flags.cut >> t & 1);        // (selects: 0 times a decay that overflows is NaN)
#pragma unroll
                            for (int i = 0; i < NS; ++i) {
                                const float own = s.y * bb[i], on = fmaf(__builtin_amdgcn_exp2f(s.x * rate[p][i]), start[r][i], own);
                                start[r][i] = cut ? own : on;
                            }
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int r = kTile / kRun - 1; r >= 0; --r) {
                        float h[kRun + 1][NS], decay[kRun][NS];
#pragma unroll
                        for (int i = 0; i < NS; ++i) h[0][i] = start[r][i];
#pragma unroll
                        for (int k0 = 0; k0 < kRun; k0 += 4) {
                            float y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                            for (int k = k0; k < k0 + 4; ++k) {
                                const int t = r * kRun + k;
                                const float2 s = steps[t][col];
                                float bb[NS];
                                __builtin_memcpy(&bb, &bs[t][n0], sizeof(bb));
                                const bool cut = !kAll && (flags.cut >> t & 1);
#pragma unroll
                                for (int i = 0; i < NS; ++i) {
                                    decay[k][i] = __builtin_amdgcn_exp2f(s.x * rate[p][i]);
                                    const float own = s.y * bb[i], on = fmaf(decay[k][i], h[k][i], own);
                                    h[k + 1][i] = cut ? own : on;
                                }
                                if (gated) {
                                    float cc[NS];
                                    __builtin_memcpy(&cc, &cs[t][n0], sizeof(cc));
#pragma unroll
                                    for (int i = 0; i < NS; ++i) y[k - k0] = fmaf(cc[i], h[k + 1][i], y[k - k0]);
                                }
                            }
                            if (gated) {
                                const float sum = sum_states(y[0], y[1], y[2], y[3]);
                                float& to = ys[r * kRun + k0 + at.q][col];
                                to = p ? to + sum : sum;
                            }
                            __builtin_amdgcn_sched_barrier(0);
                        }
#pragma unroll
                        for (int k0 = kRun - 4; k0 >= 0; k0 -= 4) {
                            float q[4] = {0.0f, 0.0f, 0.0f, 0.0f}, w[4] = {0.0f, 0.0f, 0.0f, 0.0f}, odd = 0.0f;
#pragma unroll
                            for (int k = k0 + 3; k >= k0; --k) {
                                float sum = 0.0f;
                                const int t = r * kRun + k;
                                if (kAll || (flags.live >> t & 1)) {
                                    const float2 s = steps[t][col];
                                    const float dy = dys[t][col];
                                    const bool cut = !kAll && (flags.cut >> t & 1);
                                    float bb[NS], cc[NS], v[2 * NS];
                                    __builtin_memcpy(&bb, &bs[t][n0], sizeof(bb));
                                    __builtin_memcpy(&cc, &cs[t][n0], sizeof(cc));
#pragma unroll
                                    for (int i = 0; i < NS; ++i) {
                                        const float grad = fmaf(cc[i], dy, u[p][i]);
                                        v[i] = s.y * grad;
                                        v[NS + i] = dy * h[k + 1][i];
                                        q[k - k0] = fmaf(grad, bb[i], q[k - k0]);
                                        u[p][i] = cut ? 0.0f : decay[k][i] * grad;
                                        const float m = u[p][i] * (cut ? 0.0f : h[k][i]);
                                        w[k - k0] = fmaf(m, rate[p][i], w[k - k0]);
                                        dr[i] = fmaf(m, s.x, dr[i]);
                                    }
                                    sum = sum_channels<2 * NS>(v);
                                } else if (flags.cut >> t & 1) {
#pragma unroll
                                    for (int i = 0; i < NS; ++i) u[p][i] = 0.0f;
                                }
                                if (k % 2) odd = sum;
                                else my_sums[t * 2 * NP + p * 4 * NS] = sum_pairs(sum, odd);
                            }
                            const float sq = sum_states(q[0], q[1], q[2], q[3]), sw = sum_states(w[0], w[1], w[2], w[3]);
                            float &to_q = qs[r * kRun + k0 + at.q][col], &to_w = ws[r * kRun + k0 + at.q][col];
                            to_q = p ? to_q + sq : sq;
                            to_w = p ? to_w + sw : sw;
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                    // tiles are added with what the additions round off kept beside: there may be thousands
#pragma unroll
                    for (int i = 0; i < NS; ++i) {
                        const float had = drates[p][threadIdx.x][i], more = dr[i] - losts[p][threadIdx.x][i], sum = had + more;
                        losts[p][threadIdx.x][i] = (sum - had) - more;
                        drates[p][threadIdx.x][i] = sum;
                    }
                }
            };
            if (flags.live == 0xffffu && flags.cut == 0) tile(std::true_type());
            else tile(std::false_type());
            if (t0 > first) load_front(t0 - kTile);
            __syncthreads();
            if (t0 + at.slot < end && at.n_four) {
                float dx[4], ddt[4], dz[4], dy[4], q[4], w[4], y[4], skip[4], bias[4];
                float2 s[4];
                const Four<T> x_now = kept[0][threadIdx.x], dt_now = kept[1][threadIdx.x], z_now = kept[2][threadIdx.x], dout_now = kept[3][threadIdx.x];
                get_four(dy, &dys[at.slot][four]);
                get_four(q, &qs[at.slot][four]);
                get_four(w, &ws[at.slot][four]);
                if (gated) get_four(y, &ys[at.slot][four]);
                get_four(skip, &skips[four]);
                get_four(bias, &biases[four]);
                get_steps(s, &steps[at.slot][four]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = x_now[i];
                    dx[i] = fmaf(s[i].x, q[i], skip[i] * dy[i]);
                    ddt[i] = fmaf(x, q[i], w[i] * kLn2);
                    if (a.softplus) ddt[i] *= logistic(dt_now[i] + bias[i]);
                    dz[i] = 0.0f;
                    if (gated) {
                        const float z = z_now[i], sg = logistic(z);
                        dz[i] = dout_now[i] * fmaf(skip[i], x, y[i]) * sg * fmaf(z, 1.0f - sg, 1.0f);
                    }
                    if (!live) dx[i] = ddt[i] = dz[i] = 0.0f;
                }
                if (live) {                                // (the slot's sums over all tiles are its threads' own)
                    get_four(skip, &dskips[at.slot][four]);
                    get_four(bias, &dbiases[at.slot][four]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) skip[i] = fmaf(dy[i], x_now[i], skip[i]), bias[i] += ddt[i];
                    put_four(&dskips[at.slot][four], skip);
                    put_four(&dbiases[at.slot][four], bias);
                }
                pdx.store(dx);
                pddt.store(ddt);
                if (gated) pdz.store(dz);
            } else {
                pdx.pass(), pddt.pass(), pdz.pass();
            }
            // this slice's share of dB and dC
            const int64_t slice = (at.d0 - at.group * a.per) / kGroupC;
            float* share = a.shares + (((slice * a.B + at.b) * a.T + t0) * a.G + at.group) * 2 * a.N;
            for (int n = (int)threadIdx.x; n < kTile * 2 * NP; n += kThreads) {
                const int t = n / (2 * NP), which = n / NP % 2, k = n % NP;
                if (k >= a.N || t0 + t >= end) continue;
                float s = 0.0f;
                if (flags.live >> t & 1)
#pragma unroll
                    for (int wave = 0; wave < kWaves; ++wave) s += sums[wave][t][which][k];
                share[(int64_t)t * a.G * 2 * a.N + which * a.N + k] = s;
            }
            __syncthreads();
        }
        if (a.last && a.chunks == 1) store_states<NS, PARTS>(a.last, at.b, a, at, u);
    }
    float* to = a.parts + part * a.D * (a.N + 2);
    float drate[PARTS][NS];
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
        for (int i = 0; i < NS; ++i) drate[p][i] = drates[p][threadIdx.x][i];
    store_states<NS, PARTS>(to, 0, a, at, drate);
    // dskip and dbias of the 16 slots of a tile, one after another
    to += (int64_t)a.D * a.N;
    if ((int)threadIdx.x < at.d1 - at.d0) {
        float s = 0.0f, b = 0.0f;
#pragma unroll
        for (int t = 0; t < kTile; ++t) s += dskips[t][threadIdx.x], b += dbiases[t][threadIdx.x];
        to[at.d0 + threadIdx.x] = s;
        to[a.D + at.d0 + threadIdx.x] = b;
    }
}

// dB and dC: the slices' shares, added in their order; and in the workgroups behind them, the sums of the other gradients.
template <typename T>
__global__ __launch_bounds__(kThreads) void scan_finish_kernel(ScanArgs a, int64_t all, int64_t groups, ColumnSums c)
{
    if ((int64_t)blockIdx.x >= groups) {
        column_sums_of_64(c, (int64_t)blockIdx.x - groups);
        return;
    }
    const int64_t n = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (n >= all) return;
    float s = 0.0f;
#pragma unroll 8
    for (int slice = 0; slice < a.slices; ++slice) s += a.shares[slice * all + n];
    const int64_t row = n / a.N, pair = row / 2, slot = pair / a.G, b = slot / a.T;
    att_at<T>(row % 2 ? a.dc : a.db, b, slot - b * a.T, pair - slot * a.G)[n - row * a.N] = (T)s;
}

struct BackRoom {
    size_t maps, spans, cut, shares, parts, bytes;
    int64_t n_parts;
};
inline BackRoom back_room(ScanArgs& a)
{
    BackRoom r = {};
    const int64_t each = (int64_t)a.chunks * a.G * a.slices;
    a.blocks = (int32_t)std::max<int64_t>(1, std::min<int64_t>(a.B, ceil_div(4096, each)));
    r.n_parts = (int64_t)a.blocks * a.chunks;
    if (a.chunks > 1) {
        r.maps = round_up((size_t)a.B * a.chunks * a.D * a.N * sizeof(float), 16);
        r.spans = round_up((size_t)a.B * a.chunks * a.D * sizeof(float), 16);
        r.cut = round_up((size_t)a.B * a.chunks, 16);
    }
    r.shares = round_up((size_t)a.slices * a.B * a.T * a.G * 2 * a.N * sizeof(float), 16);
    r.parts = round_up((size_t)r.n_parts * a.D * (a.N + 2) * sizeof(float), 16);
    r.bytes = r.maps + r.spans + r.cut + r.shares + r.parts;
    return r;
}

}  // namespace
}  // namespace bload

using namespace bload;

extern "C" size_t bload_selective_scan_backward_workspace_bytes(int64_t num_blocks, int32_t t_blk, int32_t feat_dim, int32_t states, int32_t groups)
{
    ScanArgs a = {};
    if (num_blocks <= 0 || scan_sizes(a, num_blocks, t_blk, feat_dim, states, groups, BLOAD_F32) != BLOAD_OK) return 0;
    return back_room(a).bytes;
}

extern "C" bload_status bload_selective_scan_backward(const bload_selective* s, const bload_heads* dout, const float* d_saved,
                                                      const float* d_dstate_out, const bload_heads* dx, const bload_heads* ddt,
                                                      float* d_drate, const bload_heads* db, const bload_heads* dc, float* d_dskip,
                                                      const bload_heads* dz, float* d_ddt_bias, float* d_dstate_in, void* d_workspace,
                                                      size_t workspace_bytes, void* hip_stream)
{
    ScanArgs a;
    bload_status st = scan_args(a, s);
    if (st != BLOAD_OK) return st;
    if (!aligned_to(d_drate, 4) || !aligned_to(d_dskip, 4) || !aligned_to(d_ddt_bias, 4)) return BLOAD_EALIGN;
    ColumnSums c = {};
    c.dst[0] = d_drate;
    c.dst[1] = d_dskip;
    c.dst[2] = d_ddt_bias;
    c.end[0] = (int64_t)s->feat_dim * s->states;
    c.end[1] = c.end[0] + s->feat_dim;
    c.end[2] = c.columns = c.end[1] + s->feat_dim;
    const hipStream_t stream = (hipStream_t)hip_stream;
    if (a.B > 0) {
        const bload_dtype dtype = s->dtype;
        if ((st = att_tensor(a.dout, dout, dtype)) != BLOAD_OK || (st = att_tensor(a.dx, dx, dtype)) != BLOAD_OK ||
            (st = att_tensor(a.ddt, ddt, dtype)) != BLOAD_OK || (st = att_tensor(a.db, db, dtype)) != BLOAD_OK ||
            (st = att_tensor(a.dc, dc, dtype)) != BLOAD_OK)
            return st;
        if (a.z.p && (st = att_tensor(a.dz, dz, dtype)) != BLOAD_OK) return st;
        if (!d_saved) return BLOAD_EINVAL;
        if (!aligned_to(d_saved, 4) || !aligned_to(d_dstate_out, 4) || !aligned_to(d_dstate_in, 4)) return BLOAD_EALIGN;
        if (states_meet(d_dstate_out, d_dstate_in, a, false) || states_meet(a.in, d_dstate_in, a, false)) return BLOAD_EINVAL;
        const BackRoom room = back_room(a);
        if (!d_workspace) return BLOAD_EINVAL;
        if (!aligned_to(d_workspace, 16)) return BLOAD_EALIGN;
        if (workspace_bytes < room.bytes) return BLOAD_EWORKSPACE;
        const int64_t all = a.B * (int64_t)a.T * a.G * 2 * a.N, groups = ceil_div(all, kThreads);
        const int64_t sums = d_drate || d_dskip || d_ddt_bias ? ceil_div(c.columns, 64) : 0;
        if (groups > kMaxGroups - sums) return BLOAD_EOVERFLOW;
        char* p = static_cast<char*>(d_workspace);
        a.maps = reinterpret_cast<float*>(p);
        a.spans = reinterpret_cast<float*>(p += room.maps);
        a.cut = reinterpret_cast<uint8_t*>(p += room.spans);
        a.shares = reinterpret_cast<float*>(p += room.cut);
        a.parts = reinterpret_cast<float*>(p += room.shares);
        a.saved = const_cast<float*>(d_saved);
        a.dlast = d_dstate_out;
        a.last = d_dstate_in;
        c.parts = a.parts;
        c.n_parts = room.n_parts;
        const dim3 block(kThreads);
        const int64_t each = (int64_t)a.chunks * a.G * a.slices;
        by_dtype(dtype, [&](auto type) {
            scan_by_states(a.N, [&](auto ns, auto parts) {
                using T = typename decltype(type)::type;
                if (a.chunks > 1) {
                    scan_backward_maps_kernel<T, ns, parts><<<dim3((unsigned)(a.B * each)), block, 0, stream>>>(a);
                    scan_join(a, a.dlast, true, stream);
                }
                scan_backward_kernel<T, ns, parts><<<dim3((unsigned)(a.blocks * each)), block, 0, stream>>>(a);
                scan_finish_kernel<T><<<dim3((unsigned)(groups + sums)), block, 0, stream>>>(a, all, groups, c);
            });
        });
        return launch_status();
    }
    return d_drate || d_dskip || d_ddt_bias ? column_sums(c, stream) : BLOAD_OK;
}
