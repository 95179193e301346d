// bload_layer_norm: layer norm and root mean square norm of rows of features, forward and backward.
//
// A row is one slot's head (or all of a slot's features); with s = x, or the rounded sum of x and a residual,
//     m = mean(s) (0 where it is not centred),  r = 1 / sqrt(mean((s - m)^2) + eps),  y = (s - m) r w + b
// Backward, with g = dy w and u = (s - m) r:
//     ds = r (g - mean(g) - u mean(g u)) + dsum  (no mean(g) where it is not centred),  dw = sum dy u,  db = sum dy
//
// HBM bound: a row is read once into registers and everything else is done there, the variance from the differences to
// the mean, not from the squares.  A team of L lanes takes a row, P pieces of 16 bytes to a lane: 4 to 64 lanes of a wavefront, or a
// workgroup of 256 or 512.  The gradients of weights are a sum over all rows: every team keeps that of the rows it takes in registers,
// workgroups leave theirs in the workspace, and a second kernel adds those in a fixed order, so the
// same inputs give the same bits.  Rows too long for registers (more than 2048 pieces) are read again from the cache.  Loads and
// stores go past the caches (documents below: 475 -> 437 us for both passes; 97 -> 80 us for rows of 1537 floats).
// Measured, averages among other kernels: 32768 rows of 4096 bfloat16 with a residual: forward 185 us for 1.07 GB, 5.8 TB/s; backward 214 us
// for as much, 5.0 TB/s (which needs workgroups in whole rounds of what the registers let be at work), its sums 7 us.  480000
// heads of 128: 53 and 76 us, 4.7 and 4.9 TB/s.
#include <algorithm>

#include "bload_rows.hpp"

namespace bload {
namespace {

struct NormArgs {
    AttTensor x, res, out, sum;              // backward: x the rows that were normalised, res dsum, out dx
    AttTensor dout;
    const uint8_t* valid;                    // [B, T] or null
    const float *weight, *bias;
    float2* stats;                           // [rows]: mean, 1 / deviation
    float* parts;                            // backward: [groups][2][D] or null
    uint32_t rows;
    Divisor H, T;
    int32_t D, center;
    float eps, inv;                          // inv: 1 / D
};

struct RowAt {
    int64_t b, t, h;
    __device__ __forceinline__ RowAt(const NormArgs& a, uint32_t row)
    {
        const uint32_t slot = over(row, a.H), block = over(slot, a.T);
        h = row - slot * a.H.d;
        t = slot - block * a.T.d;
        b = block;
    }
    __device__ __forceinline__ bool live(const NormArgs& a) const { return !a.valid || a.valid[b * a.T.d + t]; }
};

// Threads of a workgroup whose teams have L lanes.
template <int L> constexpr int kNormThreads = L > kThreads ? L : kThreads;

// Sums over a team of R rows' values; a workgroup's go through LDS, in one of two buffers in turn.
template <int L, int R>
struct Team {
    float (*room)[R][2][kNormThreads<L> / kWave];
    int turn = 0;
    __device__ __forceinline__ void sum(float (&a)[R], float (&b)[R])
    {
#pragma unroll
        for (int r = 0; r < R; ++r) lanes_sum<(L < kWave ? L : kWave)>(a[r], b[r]);
        if constexpr (L > kWave) {
            if (lane_id() == 0)
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    room[turn][r][0][wave_id()] = a[r];
                    room[turn][r][1][wave_id()] = b[r];
                }
            __syncthreads();
#pragma unroll
            for (int r = 0; r < R; ++r) {
                a[r] = b[r] = 0.0f;
#pragma unroll
                for (int w = 0; w < L / kWave; ++w) a[r] += room[turn][r][0][w], b[r] += room[turn][r][1][w];
            }
            turn ^= 1;
        }
    }
    __device__ __forceinline__ void sum(float (&a)[R])
    {
        if constexpr (L <= kWave) {
#pragma unroll
            for (int r = 0; r < R; ++r) a[r] = lanes_sum<L>(a[r]);
        } else {
            float none[R];
#pragma unroll
            for (int r = 0; r < R; ++r) none[r] = 0.0f;
            sum(a, none);
        }
    }
};

// A lane's pieces of a row: where they begin, and how many elements in front of each are a neighbour's (all: V, none of it).
template <int V, int P, int L>
struct Places {
    int at[P], skip[P];
    __device__ __forceinline__ Places(int D, int lane)
    {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int d = (p * L + lane) * V;
            at[p] = min(d, D - V);
            skip[p] = min(d - at[p], V);
        }
    }
};

template <int V>
__device__ __forceinline__ void blank(float (&x)[V], int skip)
{
    if (skip)
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = v < skip ? 0.0f : x[v];
}

// A team takes R rows at a time, whose loads are on their way together.  Teams of lanes of a wavefront take theirs alike; a
// lane without a row of its own takes part in the sums.
template <typename T, int V, int P, int L, int R>
__global__ __launch_bounds__(kNormThreads<L>) void norm_kernel(NormArgs a)
{
    __shared__ float room[2][R][2][kNormThreads<L> / kWave];
    constexpr int kTeams = kNormThreads<L> / L;
    constexpr bool kHold = P * V <= 16;      // weights stay in registers from row to row
    const int lane = (int)threadIdx.x % L;
    const Places<V, P, L> places(a.D, lane);
    Team<L, R> team{room};
    float w[kHold ? P : 1][V], bias[kHold ? P : 1][V];
    auto weights = [&](int p, float (&w)[V], float (&b)[V]) {
#pragma unroll
        for (int v = 0; v < V; ++v) w[v] = 1.0f, b[v] = 0.0f;
        if (a.weight) load_floats<V>(a.weight + places.at[p], w);
        if (a.bias) load_floats<V>(a.bias + places.at[p], b);
    };
    if constexpr (kHold)
#pragma unroll
        for (int p = 0; p < P; ++p) weights(p, w[p], bias[p]);

    const uint32_t step = gridDim.x * kTeams * R;
    for (uint32_t row0 = blockIdx.x * kTeams * R; row0 < a.rows; row0 += step) {
        RowPiece<T, V> piece[R][P], more[R][P];
        bool here[R], live[R];
        float x[R][P][V];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint32_t row = row0 + r * kTeams + (int)threadIdx.x / L;
            here[r] = row < a.rows;
            const RowAt at(a, here[r] ? row : 0);
            live[r] = here[r] && at.live(a);
            const T *px = att_at<T>(a.x, at.b, at.t, at.h), *pr = att_at<T>(a.res, at.b, at.t, at.h);
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const bool mine = live[r] && places.skip[p] < V;
                piece[r][p].zero();
                more[r][p].zero();
                if (mine) piece[r][p].load_once(px + places.at[p]);
                if (mine && a.res.p) more[r][p].load_once(pr + places.at[p]);
            }
        }
        float mean[R], square[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            mean[r] = square[r] = 0.0f;
#pragma unroll
            for (int p = 0; p < P; ++p) {
#pragma unroll
                for (int v = 0; v < V; ++v) x[r][p][v] = piece[r][p][v];
                if (a.res.p)
#pragma unroll
                    for (int v = 0; v < V; ++v) x[r][p][v] = (float)(T)(x[r][p][v] + more[r][p][v]);
                if (a.sum.p && here[r] && places.skip[p] < V) {
                    const RowAt at(a, row0 + r * kTeams + (int)threadIdx.x / L);
                    store_row_once<T, V>(att_at<T>(a.sum, at.b, at.t, at.h) + places.at[p], x[r][p], places.skip[p]);
                }
                blank<V>(x[r][p], places.skip[p]);
#pragma unroll
                for (int v = 0; v < V; ++v) mean[r] += x[r][p][v];
            }
        }
        if (a.center) team.sum(mean);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            mean[r] = a.center ? mean[r] * a.inv : 0.0f;
#pragma unroll
            for (int p = 0; p < P; ++p) {
#pragma unroll
                for (int v = 0; v < V; ++v) x[r][p][v] -= mean[r];
                blank<V>(x[r][p], places.skip[p]);
#pragma unroll
                for (int v = 0; v < V; ++v) square[r] = fmaf(x[r][p][v], x[r][p][v], square[r]);
            }
        }
        team.sum(square);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (!here[r]) continue;
            const uint32_t row = row0 + r * kTeams + (int)threadIdx.x / L;
            const RowAt at(a, row);
            const float inv = rsqrtf(fmaf(square[r], a.inv, a.eps));
            if (lane == 0 && a.stats) a.stats[row] = live[r] ? make_float2(mean[r], inv) : make_float2(0.0f, 0.0f);
            T* po = att_at<T>(a.out, at.b, at.t, at.h);
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if (places.skip[p] >= V) continue;
                float ww[V], bb[V], y[V];
                if constexpr (!kHold) weights(p, ww, bb);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    if constexpr (kHold) ww[v] = w[p][v], bb[v] = bias[p][v];
                    y[v] = live[r] ? fmaf(x[r][p][v] * inv, ww[v], bb[v]) : 0.0f;
                }
                store_row_once<T, V>(po + places.at[p], y, places.skip[p]);
            }
        }
    }
}

// One row's pieces on their way while the row in front of it is computed.
template <typename T, int V, int P>
struct BackRow {
    RowPiece<T, V> x[P], dy[P], more[P];
    float2 stat;
    bool here, live;
    template <int L>
    __device__ __forceinline__ void load(const NormArgs& a, const Places<V, P, L>& places, uint32_t row)
    {
        here = row < a.rows;
        const RowAt at(a, here ? row : 0);
        live = here && at.live(a);
        const T *px = att_at<T>(a.x, at.b, at.t, at.h), *pd = att_at<T>(a.dout, at.b, at.t, at.h), *pr = att_at<T>(a.res, at.b, at.t, at.h);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const bool mine = live && places.skip[p] < V;
            x[p].zero();
            dy[p].zero();
            more[p].zero();
            if (mine) x[p].load_once(px + places.at[p]);
            if (mine) dy[p].load_once(pd + places.at[p]);
            if (mine && a.res.p) more[p].load_once(pr + places.at[p]);
        }
        stat = live ? a.stats[row] : make_float2(0.0f, 0.0f);
    }
};

template <typename T, int V, int P, int L>
__global__ __launch_bounds__(kNormThreads<L>) void norm_backward_kernel(NormArgs a)
{
    __shared__ float room[2][1][2][kNormThreads<L> / kWave];
    constexpr int kTeams = kNormThreads<L> / L;
    constexpr bool kHold = P * V <= 16;
    const int lane = (int)threadIdx.x % L;
    const Places<V, P, L> places(a.D, lane);
    Team<L, 1> team{room};
    float w[kHold ? P : 1][V], dw[P][V], db[P][V];
    auto weights = [&](int p, float (&w)[V]) {
#pragma unroll
        for (int v = 0; v < V; ++v) w[v] = 1.0f;
        if (a.weight) load_floats<V>(a.weight + places.at[p], w);
    };
#pragma unroll
    for (int p = 0; p < P; ++p) {
        if constexpr (kHold) weights(p, w[p]);
#pragma unroll
        for (int v = 0; v < V; ++v) dw[p][v] = db[p][v] = 0.0f;
    }
    const uint32_t step = gridDim.x * kTeams, mine = (int)threadIdx.x / L;
    constexpr bool kAhead = P * V < 32;      // (more pieces leave no registers for the next row's)
    BackRow<T, V, P> now, next;
    if (kAhead) next.load(a, places, blockIdx.x * kTeams + mine);
    for (uint32_t row0 = blockIdx.x * kTeams; row0 < a.rows; row0 += step) {
        if constexpr (kAhead) {
            now = next;
            next.load(a, places, row0 + step + mine);
        } else {
            now.load(a, places, row0 + mine);
        }
        const float mean = a.center ? now.stat.x : 0.0f, inv = now.stat.y;
        float sum_g[1] = {0.0f}, sum_gu[1] = {0.0f};
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float ww[V], d[V], u[V];
            if constexpr (!kHold) weights(p, ww);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if constexpr (kHold) ww[v] = w[p][v];
                d[v] = now.dy[p][v];
                u[v] = (now.x[p][v] - mean) * inv;
            }
            blank<V>(d, places.skip[p]);
            blank<V>(u, places.skip[p]);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float g = d[v] * ww[v];
                dw[p][v] = fmaf(d[v], u[v], dw[p][v]);
                db[p][v] += d[v];
                sum_g[0] += g;
                sum_gu[0] = fmaf(g, u[v], sum_gu[0]);
            }
        }
        team.sum(sum_g, sum_gu);
        if (!now.here) continue;
        const RowAt at(a, row0 + mine);
        const float c1 = a.center ? sum_g[0] * a.inv : 0.0f, c2 = sum_gu[0] * a.inv;
        T* po = att_at<T>(a.out, at.b, at.t, at.h);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            now.x[p].renew();
            now.dy[p].renew();
            if (places.skip[p] >= V) continue;
            float ww[V], y[V];
            if constexpr (!kHold) weights(p, ww);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if constexpr (kHold) ww[v] = w[p][v];
                const float u = (now.x[p][v] - mean) * inv;
                y[v] = now.live ? fmaf(inv, fmaf(-u, c2, fmaf(now.dy[p][v], ww[v], -c1)), now.more[p][v]) : 0.0f;
            }
            store_row_once<T, V>(po + places.at[p], y, places.skip[p]);
        }
    }
    if (!a.parts) return;
    float* part = a.parts + (int64_t)blockIdx.x * 2 * a.D;
    if constexpr (L <= kWave) {
        // the teams of a wavefront, then the wavefronts one after another
        __shared__ float whole[2][P * L * V];
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int d = L; d < kWave; d <<= 1) {
                    dw[p][v] += __shfl_xor(dw[p][v], d);
                    db[p][v] += __shfl_xor(db[p][v], d);
                }
        for (int turn = 0; turn < kThreads / kWave; ++turn) {
            if (wave_id() == turn && lane_id() < L)
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        const int n = (p * L + lane) * V + v;
                        whole[0][n] = dw[p][v] + (turn ? whole[0][n] : 0.0f);
                        whole[1][n] = db[p][v] + (turn ? whole[1][n] : 0.0f);
                    }
            __syncthreads();
        }
        // (element v of a piece is its row's element at + v; the last piece of a row lies `skip` further on in here)
        if ((int)threadIdx.x < L)
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (v >= places.skip[p]) {
                        const int n = (p * L + lane) * V + v;
                        part[places.at[p] + v] = whole[0][n];
                        part[a.D + places.at[p] + v] = whole[1][n];
                    }
    } else {
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (v >= places.skip[p]) {
                    part[places.at[p] + v] = dw[p][v];
                    part[a.D + places.at[p] + v] = db[p][v];
                }
    }
}

// Rows that no workgroup holds in its registers: one element a lane at a time, the row three times over, from the cache.
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_long_kernel(NormArgs a)
{
    __shared__ float room[2][1][2][kThreads / kWave];
    Team<kThreads, 1> team{room};
    for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const RowAt at(a, row);
        const bool live = at.live(a);
        const T *px = att_at<T>(a.x, at.b, at.t, at.h), *pr = att_at<T>(a.res, at.b, at.t, at.h);
        T *po = att_at<T>(a.out, at.b, at.t, at.h), *ps = att_at<T>(a.sum, at.b, at.t, at.h);
        if (!live) {
            for (int d = (int)threadIdx.x; d < a.D; d += kThreads) {
                po[d] = (T)0.0f;
                if (a.sum.p) ps[d] = (T)0.0f;
            }
            if (threadIdx.x == 0 && a.stats) a.stats[row] = make_float2(0.0f, 0.0f);
            continue;
        }
        auto value = [&](int d) { return a.res.p ? (float)(T)((float)px[d] + (float)pr[d]) : (float)px[d]; };
        float sum[1] = {0.0f}, square[1] = {0.0f};
        if (a.center) {
            for (int d = (int)threadIdx.x; d < a.D; d += kThreads) sum[0] += value(d);
            team.sum(sum);
        }
        const float mean = sum[0] * a.inv;
        for (int d = (int)threadIdx.x; d < a.D; d += kThreads) {
            const float x = value(d) - mean;
            square[0] = fmaf(x, x, square[0]);
        }
        team.sum(square);
        const float r = rsqrtf(fmaf(square[0], a.inv, a.eps));
        if (threadIdx.x == 0 && a.stats) a.stats[row] = make_float2(mean, r);
        for (int d = (int)threadIdx.x; d < a.D; d += kThreads) {
            const float s = value(d);
            if (a.sum.p) ps[d] = (T)s;
            po[d] = (T)fmaf((s - mean) * r, a.weight ? a.weight[d] : 1.0f, a.bias ? a.bias[d] : 0.0f);
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void norm_long_backward_kernel(NormArgs a)
{
    __shared__ float room[2][1][2][kThreads / kWave];
    Team<kThreads, 1> team{room};
    for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const RowAt at(a, row);
        T* po = att_at<T>(a.out, at.b, at.t, at.h);
        if (!at.live(a)) {
            for (int d = (int)threadIdx.x; d < a.D; d += kThreads) po[d] = (T)0.0f;
            continue;
        }
        const T *px = att_at<T>(a.x, at.b, at.t, at.h), *pd = att_at<T>(a.dout, at.b, at.t, at.h), *pr = att_at<T>(a.res, at.b, at.t, at.h);
        const float2 stat = a.stats[row];
        const float mean = a.center ? stat.x : 0.0f, r = stat.y;
        float sum_g[1] = {0.0f}, sum_gu[1] = {0.0f};
        for (int d = (int)threadIdx.x; d < a.D; d += kThreads) {
            const float g = (float)pd[d] * (a.weight ? a.weight[d] : 1.0f);
            sum_g[0] += g;
            sum_gu[0] = fmaf(g, ((float)px[d] - mean) * r, sum_gu[0]);
        }
        team.sum(sum_g, sum_gu);
        const float c1 = a.center ? sum_g[0] * a.inv : 0.0f, c2 = sum_gu[0] * a.inv;
        for (int d = (int)threadIdx.x; d < a.D; d += kThreads) {
            const float g = (float)pd[d] * (a.weight ? a.weight[d] : 1.0f), u = ((float)px[d] - mean) * r;
            po[d] = (T)fmaf(r, fmaf(-u, c2, g - c1), a.res.p ? (float)pr[d] : 0.0f);
        }
    }
}

// Its gradients of weights: a lane takes a column, a workgroup some of the rows.
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_long_columns_kernel(NormArgs a, uint32_t each)
{
    const int d = (int)(blockIdx.y * kThreads + threadIdx.x);
    if (d >= a.D) return;
    float dw = 0.0f, db = 0.0f;
    const uint32_t first = blockIdx.x * each;
    for (uint32_t row = first; row < min(first + each, a.rows); ++row) {
        const RowAt at(a, row);
        if (!at.live(a)) continue;
        const float2 stat = a.stats[row];
        const float dy = (float)att_at<T>(a.dout, at.b, at.t, at.h)[d];
        dw = fmaf(dy, ((float)att_at<T>(a.x, at.b, at.t, at.h)[d] - (a.center ? stat.x : 0.0f)) * stat.y, dw);
        db += dy;
    }
    a.parts[(int64_t)blockIdx.x * 2 * a.D + d] = dw;
    a.parts[((int64_t)blockIdx.x * 2 + 1) * a.D + d] = db;
}

__global__ __launch_bounds__(kThreads) void column_sums_kernel(ColumnSums a) { column_sums_of_64(a, blockIdx.x); }

// ---------------------------------------------------------------- host

constexpr int64_t kLongGroups = 1024;        // of rows that no team holds
static_assert(kLongGroups * ((int64_t)BLOAD_LAYER_NORM_MAX_DIM / kThreads) <= kMaxGroups && BLOAD_LAYER_NORM_MAX_DIM / kThreads < 65536, "a launch holds them");
// Workgroups of the backward pass, each of which leaves a part of the weights' gradients: as many as are at work at once, by the registers
// of a row's pieces (4096 bfloat16: 768 180 us, 512 203, 1024 208; 4096 floats, of four pieces: 512 275, 768 319, 1024 281; heads of
// 128 bfloat16: 1024 75, 768 81, 1280 96).
constexpr int64_t norm_groups_most(int elements, int pieces, int lanes)
{
    return elements < 16 ? 1024 : (lanes > kThreads || pieces >= 4 ? 512 : 768);
}

// f(pieces' elements, pieces, lanes of a team, rows at a time); false for rows that no team holds.  Several rows at a time, for more
// loads on their way, where there are enough of them to fill the card all the same.
template <typename T, bool BACK, typename F>
inline bool norm_dispatch(int64_t rows, int32_t D, F f)
{
    constexpr int V = kRowPiece<T>;
    auto by_rows = [&](auto v, auto p, auto l) {
        using std::integral_constant;
        constexpr int kRows = p * v >= 32 ? 1 : (p * v >= 16 ? 2 : 4);
        if (rows >= 2048 * (kNormThreads<l> / l) * kRows) f(v, p, l, integral_constant<int, kRows>());
        else f(v, p, l, integral_constant<int, 1>());
    };
#define BLOAD_NORM_CASE(v, p, l) by_rows(std::integral_constant<int, v>(), std::integral_constant<int, p>(), std::integral_constant<int, l>())
    const int64_t n = ceil_div(D, V);
    if (D < V) BLOAD_NORM_CASE(1, 1, 8);
    else if (n <= 4) BLOAD_NORM_CASE(V, 1, 4);
    else if (n <= 8) BLOAD_NORM_CASE(V, 1, 8);
    else if (n <= 16) BLOAD_NORM_CASE(V, 1, 16);
    else if (n <= 32) BLOAD_NORM_CASE(V, 1, 32);
    else if (n <= 64) BLOAD_NORM_CASE(V, 1, 64);
    else if (n <= 128) BLOAD_NORM_CASE(V, 2, 64);
    else if (n > 2048) return false;
    else if constexpr (V == 4) {             // (floats: half the elements to a piece)
        if (n <= 512) BLOAD_NORM_CASE(V, BACK ? 2 : 8, BACK ? 256 : 64);
        else if (n <= 1024) BLOAD_NORM_CASE(V, 4, 256);
        else BLOAD_NORM_CASE(V, 4, 512);
    } else {
        if (n <= 256) BLOAD_NORM_CASE(V, 1, 256);
        else if (n <= 512) BLOAD_NORM_CASE(V, 2, 256);
        else if (n <= 1024) BLOAD_NORM_CASE(V, 2, 512);
        else BLOAD_NORM_CASE(V, 4, 512);
    }
#undef BLOAD_NORM_CASE
    return true;
}

inline bload_status norm_check(int64_t num_blocks, int32_t t_blk, int32_t heads, int32_t dim, bload_dtype dtype)
{
    if (num_blocks < 0 || t_blk < 1 || heads < 1 || dim < 1 || !att_dtype(dtype)) return BLOAD_EINVAL;
    // (dim: what a launch holds of workgroups over the rows' shares and the columns of norm_long_columns_kernel)
    if (t_blk > (1 << 30) || dim > BLOAD_LAYER_NORM_MAX_DIM || num_blocks > 0x7fffffffLL / t_blk / heads) return BLOAD_EOVERFLOW;
    return BLOAD_OK;
}

// Workgroups of the backward pass and with that the parts that are added behind it.
inline int64_t norm_groups(int64_t rows, int32_t dim, bload_dtype dtype)
{
    int64_t groups = 0;
    auto by_type = [&](auto type) {
        if (!norm_dispatch<typename decltype(type)::type, true>(rows, dim, [&](auto v, auto p, auto l, auto) {
                groups = std::min<int64_t>(norm_groups_most(p * v, p, l), ceil_div(rows, kNormThreads<l> / l));
            }))
            groups = std::min<int64_t>(kLongGroups, rows);
    };
    if (dtype == BLOAD_F32) by_type(type_is<float>());
    else by_type(type_is<att_half>());
    return groups;
}

inline NormArgs norm_args(int64_t rows, int32_t t_blk, int32_t heads, int32_t dim, int32_t center)
{
    NormArgs a = {};
    a.rows = (uint32_t)rows;
    a.H = divisor(heads);
    a.T = divisor(t_blk);
    a.D = dim;
    a.center = center;
    a.inv = 1.0f / (float)dim;
    return a;
}

// Where the blocks of all tensors follow one another as their slots do, slots are counted through: one division less a row.
inline void merge_blocks(NormArgs& a)
{
    AttTensor* all[] = {&a.x, &a.res, &a.out, &a.sum, &a.dout};
    for (AttTensor* t : all)
        if (t->p && t->sb != t->st * (int64_t)a.T.d) return;
    for (AttTensor* t : all) t->sb = t->st;
    a.T = divisor(1);
}

}  // namespace

bload_status column_sums(const ColumnSums& a, hipStream_t stream)
{
    const int64_t groups = ceil_div(a.columns, 64);
    if (groups > kMaxGroups) return BLOAD_EOVERFLOW;
    if (groups > 0) column_sums_kernel<<<dim3((unsigned)groups), dim3(kThreads), 0, stream>>>(a);
    return launch_status();
}

}  // namespace bload

using namespace bload;

extern "C" bload_status bload_layer_norm(const bload_heads* x, const bload_heads* residual, const uint8_t* d_valid, int64_t num_blocks,
                                         int32_t t_blk, int32_t heads, int32_t dim, bload_dtype dtype, int32_t center, float eps,
                                         const float* d_weight, const float* d_bias, const bload_heads* out, const bload_heads* sum,
                                         float* d_stats, void* hip_stream)
{
    bload_status st = norm_check(num_blocks, t_blk, heads, dim, dtype);
    if (st != BLOAD_OK) return st;
    if (center < 0 || center > 1 || !(eps >= 0.0f) || !std::isfinite(eps)) return BLOAD_EINVAL;
    if (num_blocks == 0) return BLOAD_OK;
    const int64_t rows = num_blocks * t_blk * heads;
    NormArgs a = norm_args(rows, t_blk, heads, dim, center);
    a.eps = eps;
    if ((st = att_tensor(a.x, x, dtype)) != BLOAD_OK || (st = att_tensor(a.out, out, dtype)) != BLOAD_OK) return st;
    if (residual && (st = att_tensor(a.res, residual, dtype)) != BLOAD_OK) return st;
    if (sum && (st = att_tensor(a.sum, sum, dtype)) != BLOAD_OK) return st;
    if (!aligned_to(d_weight, 4) || !aligned_to(d_bias, 4) || !aligned_to(d_stats, 8)) return BLOAD_EALIGN;
    a.valid = d_valid;
    a.weight = d_weight;
    a.bias = d_bias;
    a.stats = reinterpret_cast<float2*>(d_stats);
    merge_blocks(a);
    const hipStream_t stream = (hipStream_t)hip_stream;
    by_dtype(dtype, [&](auto type) {
        using T = typename decltype(type)::type;
        const bool held = norm_dispatch<T, false>(rows, dim, [&](auto v, auto p, auto l, auto r) {
            const int64_t groups = std::min<int64_t>(4096, ceil_div(rows, kNormThreads<l> / l * r));
            norm_kernel<T, v, p, l, r><<<dim3((unsigned)groups), dim3(kNormThreads<l>), 0, stream>>>(a);
        });
        if (!held) norm_long_kernel<T><<<dim3((unsigned)std::min<int64_t>(4096, rows)), dim3(kThreads), 0, stream>>>(a);
    });
    return launch_status();
}

extern "C" size_t bload_layer_norm_backward_workspace_bytes(int64_t num_blocks, int32_t t_blk, int32_t heads, int32_t dim, bload_dtype dtype)
{
    if (num_blocks <= 0 || norm_check(num_blocks, t_blk, heads, dim, dtype) != BLOAD_OK) return 0;
    return round_up((size_t)norm_groups(num_blocks * t_blk * heads, dim, dtype) * 2 * dim * sizeof(float), 16);
}

extern "C" bload_status bload_layer_norm_backward(const bload_heads* dout, const bload_heads* x, const float* d_stats, const uint8_t* d_valid,
                                                  int64_t num_blocks, int32_t t_blk, int32_t heads, int32_t dim, bload_dtype dtype,
                                                  int32_t center, const float* d_weight, const bload_heads* dsum, const bload_heads* dx,
                                                  float* d_dweight, float* d_dbias, void* d_workspace, size_t workspace_bytes,
                                                  void* hip_stream)
{
    bload_status st = norm_check(num_blocks, t_blk, heads, dim, dtype);
    if (st != BLOAD_OK) return st;
    if (center < 0 || center > 1) return BLOAD_EINVAL;
    if (!aligned_to(d_dweight, 4) || !aligned_to(d_dbias, 4)) return BLOAD_EALIGN;
    const hipStream_t stream = (hipStream_t)hip_stream;
    const int64_t rows = num_blocks * t_blk * heads;
    const bool sums = d_dweight || d_dbias;
    ColumnSums c = {};
    c.dst[0] = d_dweight;
    c.dst[1] = d_dbias;
    c.end[0] = dim;
    c.end[1] = c.columns = 2 * (int64_t)dim;
    if (rows > 0) {
        NormArgs a = norm_args(rows, t_blk, heads, dim, center);
        if ((st = att_tensor(a.x, x, dtype)) != BLOAD_OK || (st = att_tensor(a.dout, dout, dtype)) != BLOAD_OK ||
            (st = att_tensor(a.out, dx, dtype)) != BLOAD_OK)
            return st;
        if (dsum && (st = att_tensor(a.res, dsum, dtype)) != BLOAD_OK) return st;
        if (!d_stats) return BLOAD_EINVAL;
        if (!aligned_to(d_stats, 8) || !aligned_to(d_weight, 4)) return BLOAD_EALIGN;
        const int64_t groups = norm_groups(rows, dim, dtype);
        if (sums) {
            if (!d_workspace) return BLOAD_EINVAL;
            if (!aligned_to(d_workspace, 16)) return BLOAD_EALIGN;
            if (workspace_bytes < (size_t)groups * 2 * dim * sizeof(float)) return BLOAD_EWORKSPACE;
            a.parts = static_cast<float*>(d_workspace);
        }
        a.valid = d_valid;
        a.weight = d_weight;
        a.stats = reinterpret_cast<float2*>(const_cast<float*>(d_stats));
        merge_blocks(a);
        by_dtype(dtype, [&](auto type) {
            using T = typename decltype(type)::type;
            const bool held = norm_dispatch<T, true>(rows, dim, [&](auto v, auto p, auto l, auto) {
                norm_backward_kernel<T, v, p, l><<<dim3((unsigned)groups), dim3(kNormThreads<l>), 0, stream>>>(a);
            });
            if (held) return;
            // (the columns first: dx may lie where dout does)
            const uint32_t each = (uint32_t)ceil_div(rows, groups);
            if (sums)
                norm_long_columns_kernel<T><<<dim3((unsigned)groups, (unsigned)ceil_div(dim, kThreads)), dim3(kThreads), 0, stream>>>(a, each);
            norm_long_backward_kernel<T><<<dim3((unsigned)std::min<int64_t>(4096, rows)), dim3(kThreads), 0, stream>>>(a);
        });
        if ((st = launch_status()) != BLOAD_OK) return st;
        c.parts = a.parts;
        c.n_parts = groups;
    }
    return sums ? column_sums(c, stream) : BLOAD_OK;
}
