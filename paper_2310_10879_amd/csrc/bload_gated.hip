// bload_gated_scan: the recurrence h_t = gate_t h_{t-1} + x_t per feature over packed blocks, forward and
// backward.
//
// Forward, over the slots of a block in order (a slot "goes on" when it is valid, carries no start flag and the
// slot in front of it is valid; the block's first slot goes on from a state that was handed in):
//     h = gate h_prev + x   where the slot goes on;   h = x   where it starts a sequence;   0 on padding
// Backward, against the order, u being what comes back to a slot from the one behind it:
//     g = dh + u  (0 on padding);   dx = g;   dgate = g h_prev, u' = gate g  where the slot goes on, else 0
//
// A stretch of slots is an affine map of what enters it: out = A in + H, A the product of its gates, or
// out = H where some slot of it does not go on (by selection: A in may be NaN then).  Two stretches
// make one: (A2 A1, A2 H1 + H2).  A workgroup takes F lanes across features, four elements each, and
// 256 / F stretches of K slots: every lane keeps its K slots in registers, forms the map, the maps are
// scanned across lanes and waves, and the slots are gone through again from what really enters.  So the data is read
// once and written once; HBM bound.  Blocks are walked from end to end by one workgroup, or where that
// leaves the card empty, cut into chunks: a first launch forms the maps of all chunks, the second starts each
// chunk from the maps in front of it (the data is read twice, which matters little: it is
// small, or it would not leave the card empty).  No workgroup waits for another one.
// All of h, g, A, H and u is in 32 bits; only results are rounded to the type.  Backward, h_prev is the forward pass's rounded
// result: dgate is off by half a step of the type from that, beside its own rounding, where x would have to be read for
// more.
// Measured: 48 blocks of 3000 x 2048 half: forward 0.46 ms for 1.77 GB, 3.8 TB/s, backward 0.61 ms for 2.95 GB, 4.8 TB/s (a copy in tiles:
// 6.4).  Forward, a step loads, exchanges, and stores with nothing on its way meanwhile: latency more than HBM.
#include <algorithm>

#include "bload_attention_host.hpp"

namespace bload {
namespace {

struct GatedArgs {
    const void *gate, *x;            // forward: x; backward: dh
    const void* h;                   // backward: the forward pass's result
    const uint8_t *reset, *valid;
    const float* in;                 // [B, D] or null: h0, backward dstate
    const float* h0;                 // backward: [B, D] or null
    void *y, *dgate;                 // h, backward dx;  backward dgate
    float* last;                     // [B, D] or null: the state behind the last slot, backward dh0
    float* maps;                     // [B, chunks, 2, D]: A and H of every chunk
    uint8_t* cut;                    // [B, chunks]: some slot of the chunk does not go on
    int32_t T, D, slices, chunks, chunk, F;
};

enum { kApply = 0, kMaps = 1 };

// What a slot does: 0 padding, 1 starts a sequence, 2 goes on.
__device__ __forceinline__ int slot_code(const GatedArgs& a, const uint8_t* reset, const uint8_t* valid, int t, bool has_state)
{
    if (!valid[t]) return 0;
    if (reset[t]) return 1;
    return (t == 0 ? has_state : valid[t - 1] != 0) ? 2 : 1;
}

// V elements side by side, as they lie in memory; any alignment.  A lane whose V elements would pass the end of a row takes the
// row's last V instead.  Some of them are its neighbour's too, which in gated_kernel computes and stores the same.
template <typename T, int V>
struct Piece {
    static constexpr int kWords = V * sizeof(T) >= 4 ? V * (int)sizeof(T) / 4 : 1;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const void* base, int64_t row, int D, int d)
    {
        __builtin_memcpy(&w, reinterpret_cast<const T*>(base) + row * D + d, V * sizeof(T));
    }
    __device__ __forceinline__ void widen(float (&x)[V]) const
    {
        T t[V];
        __builtin_memcpy(&t, &w, sizeof(t));
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = (float)t[v];
    }
};

template <typename T, int V>
__device__ __forceinline__ void store_piece(void* base, int64_t row, int D, int d, const float (&x)[V])
{
    T t[V];
#pragma unroll
    for (int v = 0; v < V; ++v) t[v] = (T)x[v];
    __builtin_memcpy(reinterpret_cast<T*>(base) + row * D + d, &t, sizeof(t));
}

// Elements from `skip` on alone; the others are 0, or are not stored.
template <int V>
__device__ __forceinline__ void load_state(const float* base, int64_t b, int D, int d, float (&x)[V], int skip = 0)
{
#pragma unroll
    for (int v = 0; v < V; ++v) x[v] = base && v >= skip ? base[b * D + d + v] : 0.0f;
}
template <typename T, int V>
__device__ __forceinline__ void store_behind(void* base, int64_t row, int D, int d, const float (&x)[V], int skip)
{
    if (skip == 0) {
        store_piece<T, V>(base, row, D, d, x);
    } else {
#pragma unroll
        for (int v = 1; v < V; ++v)
            if (v >= skip) reinterpret_cast<T*>(base)[row * D + d + v] = (T)x[v];
    }
}

// K slots of one lane in the order of the recurrence: slot i is row first + i forward, first - i backward, and the chunk's last
// one, `end`, in the place of those behind it (nothing becomes of them).
template <typename T, int V, int K, bool BACK>
struct Run {
    Piece<T, V> gate[K], x[K], h[BACK ? K : 1];

    __device__ __forceinline__ void load(const GatedArgs& a, int64_t b, int first, int end, int d, bool want_h)
    {
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const int t = BACK ? max(first - i, end) : min(first + i, end);
            const int64_t row = b * a.T + t;
            gate[i].load(a.gate, row, a.D, d);
            x[i].load(a.x, row, a.D, d);
            if constexpr (BACK)
                if (want_h) h[i].load(a.h, t > 0 ? row - 1 : row, a.D, d);
        }
    }
};

// A map of the state that enters a stretch: out = A in + H, or H alone where `cut`.
template <int V>
struct Map {
    float A[V], H[V];
    int cut;
    __device__ __forceinline__ void one()
    {
#pragma unroll
        for (int v = 0; v < V; ++v) A[v] = 1.0f, H[v] = 0.0f;
        cut = 0;
    }
    // this map after `f`
    __device__ __forceinline__ void after(const Map& f)
    {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            H[v] = cut ? H[v] : fmaf(A[v], f.H[v], H[v]);
            A[v] = A[v] * f.A[v];
        }
        cut |= f.cut;
    }
    __device__ __forceinline__ void apply(float (&in)[V]) const
    {
#pragma unroll
        for (int v = 0; v < V; ++v) in[v] = cut ? H[v] : fmaf(A[v], in[v], H[v]);
    }
};

template <typename T, int V, int K, bool BACK, int MODE>
__global__ __launch_bounds__(kThreads) void gated_kernel(GatedArgs a)
{
    constexpr int kWaves = kThreads / kWave;
    __shared__ uint8_t code[2][kThreads * K];
    __shared__ float total[2][kWaves][2][kWave * V];       // of a wave's lanes together, by feature
    __shared__ int cuts[2][kWaves], folded[8];

    const int lane = lane_id(), wave = wave_id(), tid = (int)threadIdx.x;
    const int F = a.F, runs = kThreads / F, f = tid & (F - 1), run = tid / F;
    const int slice = (int)(blockIdx.x % a.slices), chunk = (int)((blockIdx.x / a.slices) % a.chunks);
    const int64_t b = blockIdx.x / a.slices / a.chunks;
    const bool mine = (slice * F + f) * V < a.D;
    const int d = min((slice * F + f) * V, a.D - V);
    // chunk c holds the slots c * chunk .. of the block in the order of the recurrence
    const int c0 = chunk * a.chunk, c1 = min(c0 + a.chunk, a.T);
    const uint8_t* reset = a.reset + b * a.T;
    const uint8_t* valid = a.valid + b * a.T;
    const bool has_state = (BACK ? a.h0 : a.in) != nullptr;

    // what enters the chunk
    float in[V];
    load_state<V>(a.in, b, a.D, d, in);
    if (MODE == kApply && chunk > 0) {
        // the maps of the chunks in front, an eighth of them to each of eight runs (four loads on their way at a time), then
        // those eight one after another
        const int folds = min(runs, 8), each = (chunk + folds - 1) / folds;
        float (*fold)[2][kWave * V / 2] = reinterpret_cast<float (*)[2][kWave * V / 2]>(&total[0][0][0][0]);
        if (run < folds) {
            Map<V> all;
            all.one();
            for (int c = run * each; c < min((run + 1) * each, chunk); c += 4) {
                Map<V> m[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int64_t at = b * a.chunks + min(c + i, chunk - 1);
                    m[i].cut = a.cut[at];
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        m[i].A[v] = a.maps[at * 2 * a.D + d + v];
                        m[i].H[v] = a.maps[(at * 2 + 1) * a.D + d + v];
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (c + i < min((run + 1) * each, chunk)) {
                        m[i].after(all);
                        all = m[i];
                    }
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                fold[run][0][f * V + v] = all.A[v];
                fold[run][1][f * V + v] = all.H[v];
            }
            if (f == 0) folded[run] = all.cut;
        }
        __syncthreads();
        for (int r = 0; r < folds; ++r) {
            Map<V> m;
            m.cut = folded[r];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                m.A[v] = fold[r][0][f * V + v];
                m.H[v] = fold[r][1][f * V + v];
            }
            m.apply(in);
        }
    }
    Map<V> sum;                                            // kMaps: of the chunk so far
    sum.one();

    const int span = runs * K;                             // slots of a step
    auto load_code = [&](int s, int buf) {
        for (int n = tid; n < span; n += kThreads) {
            const int i = s + n;
            code[buf][n] = i < c1 ? (uint8_t)slot_code(a, reset, valid, BACK ? a.T - 1 - i : i, has_state) : 3;
        }
    };
    auto slots_left = [&](int s) { return min(max(c1 - (s + run * K), 0), K); };
    auto first_slot = [&](int s) { return BACK ? a.T - 1 - (s + run * K) : s + run * K; };

    Run<T, V, K, BACK> now;
    load_code(c0, 0);
    int buf = 0;
    for (int s = c0; s < c1; s += span, buf ^= 1) {
        now.load(a, b, first_slot(s), BACK ? a.T - c1 : c1 - 1, d, MODE == kApply);
        __syncthreads();                                   // code[buf] is there
        if (s + span < c1) load_code(s + span, buf ^ 1);
        int what[K];
#pragma unroll
        for (int i = 0; i < K; ++i) what[i] = code[buf][run * K + i];        // 3 behind the chunk's end: nothing happens
        Map<V> m;
        m.one();
#pragma unroll
        for (int i = 0; i < K; ++i) {
            float g[V], x[V];
            now.gate[i].widen(g);
            now.x[i].widen(x);
            if (what[i] == 3) continue;
            if constexpr (!BACK) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    m.H[v] = what[i] == 2 ? fmaf(g[v], m.H[v], x[v]) : (what[i] == 1 ? x[v] : 0.0f);
                    m.A[v] *= g[v];
                }
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    m.H[v] = what[i] == 2 ? g[v] * (x[v] + m.H[v]) : 0.0f;
                    m.A[v] *= g[v];
                }
            }
            m.cut |= what[i] != 2;
        }
        // inclusive over the wave's stretches (lanes F apart)
        for (int dist = F; dist < kWave; dist <<= 1) {
            Map<V> o;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                o.A[v] = __shfl_up(m.A[v], dist);
                o.H[v] = __shfl_up(m.H[v], dist);
            }
            o.cut = __shfl_up(m.cut, dist);
            if (lane >= dist) m.after(o);
        }
        if (lane >= kWave - F) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                total[buf][wave][0][f * V + v] = m.A[v];
                total[buf][wave][1][f * V + v] = m.H[v];
            }
            if (lane == kWave - 1) cuts[buf][wave] = m.cut;
        }
        // what lies in front of this lane's stretch in its wave
        Map<V> o;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            o.A[v] = __shfl_up(m.A[v], F & (kWave - 1));
            o.H[v] = __shfl_up(m.H[v], F & (kWave - 1));
        }
        o.cut = __shfl_up(m.cut, F & (kWave - 1));
        if (lane < F) o.one();
        __syncthreads();
        float at[V];                                       // what enters this lane's stretch
#pragma unroll
        for (int v = 0; v < V; ++v) at[v] = in[v];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            Map<V> q;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                q.A[v] = total[buf][w][0][f * V + v];
                q.H[v] = total[buf][w][1][f * V + v];
            }
            q.cut = cuts[buf][w];
            if (MODE == kApply) {
                if (w == wave)
#pragma unroll
                    for (int v = 0; v < V; ++v) at[v] = in[v];
                q.apply(in);
            } else {
                q.after(sum);
                sum = q;
            }
        }
        if (MODE != kApply) continue;
        o.apply(at);
        const int n = slots_left(s), first = first_slot(s);
#pragma unroll
        for (int i = 0; i < K; ++i) {
            if (i >= n || !mine) continue;
            const int64_t row = b * a.T + (BACK ? first - i : first + i);
            float g[V], x[V];
            now.gate[i].widen(g);
            now.x[i].widen(x);
            if constexpr (!BACK) {
#pragma unroll
                for (int v = 0; v < V; ++v) at[v] = what[i] == 2 ? fmaf(g[v], at[v], x[v]) : (what[i] == 1 ? x[v] : 0.0f);
                store_piece<T, V>(a.y, row, a.D, d, at);
            } else {
                float h[V], dg[V];
                if (first - i > 0) now.h[i].widen(h);
                else load_state<V>(a.h0, b, a.D, d, h);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    x[v] = what[i] ? x[v] + at[v] : 0.0f;
                    dg[v] = what[i] == 2 ? x[v] * h[v] : 0.0f;
                    at[v] = what[i] == 2 ? g[v] * x[v] : 0.0f;
                }
                store_piece<T, V>(a.y, row, a.D, d, x);
                store_piece<T, V>(a.dgate, row, a.D, d, dg);
            }
        }
    }
    if (!mine || run != 0) return;
    if (MODE == kMaps) {
        float* p = a.maps + (b * a.chunks + chunk) * 2 * a.D;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            p[d + v] = sum.A[v];
            p[a.D + d + v] = sum.H[v];
        }
        if (d == 0) a.cut[b * a.chunks + chunk] = (uint8_t)(sum.cut != 0);
    } else if (chunk == a.chunks - 1 && a.last) {
#pragma unroll
        for (int v = 0; v < V; ++v) a.last[b * a.D + d + v] = in[v];
    }
}

// Blocks of a few slots (one, when streams are served): a lane takes V elements of a block from its first slot
// to its last.  The state may be advanced in place, and nothing orders one wavefront's loads and another's stores: every element
// has one lane that reads its state and stores its results.  The last lane of a row leaves `skip` elements to its neighbour.
constexpr int kShort = 8;

template <typename T, int V, bool BACK>
__global__ __launch_bounds__(kThreads) void gated_short_kernel(GatedArgs a, int64_t lanes)
{
    const int64_t n = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (n >= lanes) return;
    const int64_t b = n / a.slices;
    const int d0 = (int)(n - b * a.slices) * V, d = min(d0, a.D - V), skip = d0 - d;
    const bool has_state = (BACK ? a.h0 : a.in) != nullptr;
    const uint8_t* reset = a.reset + b * a.T;
    const uint8_t* valid = a.valid + b * a.T;
    float at[V];
    load_state<V>(a.in, b, a.D, d, at, skip);
    for (int i = 0; i < a.T; ++i) {
        const int t = BACK ? a.T - 1 - i : i;
        const int64_t row = b * a.T + t;
        const int what = slot_code(a, reset, valid, t, has_state);
        float g[V], x[V];
        Piece<T, V> piece;
        piece.load(a.gate, row, a.D, d);
        piece.widen(g);
        piece.load(a.x, row, a.D, d);
        piece.widen(x);
        if constexpr (!BACK) {
#pragma unroll
            for (int v = 0; v < V; ++v) at[v] = what == 2 ? fmaf(g[v], at[v], x[v]) : (what == 1 ? x[v] : 0.0f);
            store_behind<T, V>(a.y, row, a.D, d, at, skip);
        } else {
            float h[V], dg[V];
            if (t > 0) {
                piece.load(a.h, row - 1, a.D, d);
                piece.widen(h);
            } else {
                load_state<V>(a.h0, b, a.D, d, h, skip);
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                x[v] = what ? x[v] + at[v] : 0.0f;
                dg[v] = what == 2 ? x[v] * h[v] : 0.0f;
                at[v] = what == 2 ? g[v] * x[v] : 0.0f;
            }
            store_behind<T, V>(a.y, row, a.D, d, x, skip);
            store_behind<T, V>(a.dgate, row, a.D, d, dg, skip);
        }
    }
    if (a.last)
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (v >= skip) a.last[b * a.D + d + v] = at[v];
}

struct GatedPlan {
    int32_t F, slices, chunks, chunk;
    int64_t groups;
    size_t maps, bytes;              // of the chunks' maps alone, of the workspace
};

// Elements and slots of a lane at a time.  What the lanes exchange goes by the elements, so few elements and many slots cost
// least of it.
constexpr int kPiece = 4;                                  // (1 where a row has fewer than 4)
constexpr int kSlots = 8;

// Features across 32 lanes, fewer where a row is shorter; a block to a workgroup, or where that
// makes fewer workgroups than there are CUs, chunks of whole steps.
inline GatedPlan gated_plan(int64_t B, int32_t T, int64_t D)
{
    GatedPlan p = {};
    const int64_t lanes = D < kPiece ? D : ceil_div(D, kPiece);
    p.F = 1;
    while (p.F < 32 && p.F < lanes) p.F *= 2;
    p.slices = (int32_t)ceil_div(lanes, p.F);
    const int64_t step = (int64_t)(kThreads / p.F) * kSlots;
    const int64_t steps = ceil_div(T, step), alone = B * p.slices;
    int64_t chunks = alone < 256 ? std::min<int64_t>({ceil_div(1024, alone), steps, 64}) : 1;
    p.chunk = (int32_t)(ceil_div(steps, chunks) * step);
    p.chunks = (int32_t)ceil_div(T, p.chunk);
    p.groups = alone * p.chunks;
    if (p.chunks > 1) {
        p.maps = round_up((size_t)B * p.chunks * 2 * D * sizeof(float), 16);
        p.bytes = p.maps + round_up((size_t)B * p.chunks, 16);
    }
    return p;
}

inline bload_status gated_check(int64_t num_blocks, int32_t t_blk, int64_t feat_dim, bload_dtype dtype)
{
    if (num_blocks < 0 || t_blk < 1 || feat_dim < 1 || !att_dtype(dtype)) return BLOAD_EINVAL;
    if (t_blk > (1 << 30) || feat_dim > (1 << 30) || num_blocks >= ((int64_t)1 << 40) / t_blk ||
        num_blocks > ((int64_t)1 << 50) / feat_dim / t_blk)
        return BLOAD_EOVERFLOW;
    return BLOAD_OK;
}

// A state may be handed in and out in one buffer where every element has one lane (gated_short_kernel); elsewhere a workgroup
// could read what another one has advanced already.
inline bool states_apart(const float* in, const float* out, int64_t num_blocks, int32_t t_blk, int64_t feat_dim)
{
    if (!in || !out || (in == out && t_blk <= kShort)) return true;
    const uintptr_t p = reinterpret_cast<uintptr_t>(in), q = reinterpret_cast<uintptr_t>(out);
    return (p < q ? q - p : p - q) >= (uintptr_t)num_blocks * (uintptr_t)feat_dim * sizeof(float);
}

template <typename T, int V, bool BACK>
void gated_launch(const GatedArgs& a, const GatedPlan& p, hipStream_t stream)
{
    const dim3 grid((unsigned)p.groups), block(kThreads);
    if (p.chunks > 1) gated_kernel<T, V, kSlots, BACK, kMaps><<<grid, block, 0, stream>>>(a);
    gated_kernel<T, V, kSlots, BACK, kApply><<<grid, block, 0, stream>>>(a);
}

template <typename T, bool BACK>
bload_status gated_run(GatedArgs a, int64_t B, void* workspace, size_t room, hipStream_t stream)
{
    if (a.T <= kShort) {
        const int V = a.D < kPiece ? 1 : kPiece;
        a.slices = (int32_t)ceil_div(a.D, V);
        const int64_t lanes = B * a.slices, groups = ceil_div(lanes, kThreads);
        if (groups > kMaxGroups) return BLOAD_EOVERFLOW;
        const dim3 grid((unsigned)groups), block(kThreads);
        if (V == 1) gated_short_kernel<T, 1, BACK><<<grid, block, 0, stream>>>(a, lanes);
        else gated_short_kernel<T, kPiece, BACK><<<grid, block, 0, stream>>>(a, lanes);
        return launch_status();
    }
    const GatedPlan p = gated_plan(B, a.T, a.D);
    if (p.groups > kMaxGroups) return BLOAD_EOVERFLOW;
    if (p.bytes) {
        if (!workspace) return BLOAD_EINVAL;
        if (!aligned_to(workspace, 16)) return BLOAD_EALIGN;
        if (room < p.bytes) return BLOAD_EWORKSPACE;
        a.maps = static_cast<float*>(workspace);
        a.cut = static_cast<uint8_t*>(workspace) + p.maps;
    }
    a.F = p.F;
    a.slices = p.slices;
    a.chunks = p.chunks;
    a.chunk = p.chunk;
    if (a.D < kPiece) gated_launch<T, 1, BACK>(a, p, stream);
    else gated_launch<T, kPiece, BACK>(a, p, stream);
    return launch_status();
}

template <bool BACK>
bload_status gated_by_type(const GatedArgs& a, int64_t B, bload_dtype dtype, void* workspace, size_t room, hipStream_t stream)
{
    if (dtype == BLOAD_F16) return gated_run<att_half, BACK>(a, B, workspace, room, stream);
    if (dtype == BLOAD_BF16) return gated_run<att_bf16, BACK>(a, B, workspace, room, stream);
    return gated_run<float, BACK>(a, B, workspace, room, stream);
}

}  // namespace
}  // namespace bload

using namespace bload;

extern "C" size_t bload_gated_scan_workspace_bytes(int64_t num_blocks, int32_t t_blk, int64_t feat_dim, bload_dtype dtype)
{
    if (num_blocks <= 0 || gated_check(num_blocks, t_blk, feat_dim, dtype) != BLOAD_OK || t_blk <= kShort) return 0;
    return gated_plan(num_blocks, t_blk, feat_dim).bytes;
}

extern "C" bload_status bload_gated_scan(const void* d_gate, const void* d_x, const uint8_t* d_reset, const uint8_t* d_valid,
                                         int64_t num_blocks, int32_t t_blk, int64_t feat_dim, bload_dtype dtype, const float* d_state_in,
                                         void* d_out, float* d_state_out, void* d_workspace, size_t workspace_bytes, void* hip_stream)
{
    const bload_status st = gated_check(num_blocks, t_blk, feat_dim, dtype);
    if (st != BLOAD_OK) return st;
    if (num_blocks == 0) return BLOAD_OK;
    if (!d_gate || !d_x || !d_reset || !d_valid || !d_out) return BLOAD_EINVAL;
    const size_t e = att_elem_bytes(dtype);
    if (!aligned_to(d_gate, e) || !aligned_to(d_x, e) || !aligned_to(d_out, e) || !aligned_to(d_state_in, 4) || !aligned_to(d_state_out, 4))
        return BLOAD_EALIGN;
    if (!states_apart(d_state_in, d_state_out, num_blocks, t_blk, feat_dim)) return BLOAD_EINVAL;
    GatedArgs a = {};
    a.gate = d_gate;
    a.x = d_x;
    a.reset = d_reset;
    a.valid = d_valid;
    a.in = d_state_in;
    a.y = d_out;
    a.last = d_state_out;
    a.T = t_blk;
    a.D = (int32_t)feat_dim;
    return gated_by_type<false>(a, num_blocks, dtype, d_workspace, workspace_bytes, (hipStream_t)hip_stream);
}

extern "C" bload_status bload_gated_scan_backward(const void* d_dout, const void* d_gate, const void* d_out, const uint8_t* d_reset,
                                                  const uint8_t* d_valid, int64_t num_blocks, int32_t t_blk, int64_t feat_dim,
                                                  bload_dtype dtype, const float* d_state_in, const float* d_dstate_out, void* d_dgate,
                                                  void* d_dx, float* d_dstate_in, void* d_workspace, size_t workspace_bytes, void* hip_stream)
{
    const bload_status st = gated_check(num_blocks, t_blk, feat_dim, dtype);
    if (st != BLOAD_OK) return st;
    if (num_blocks == 0) return BLOAD_OK;
    if (!d_dout || !d_gate || !d_out || !d_reset || !d_valid || !d_dgate || !d_dx) return BLOAD_EINVAL;
    const size_t e = att_elem_bytes(dtype);
    if (!aligned_to(d_dout, e) || !aligned_to(d_gate, e) || !aligned_to(d_out, e) || !aligned_to(d_dgate, e) || !aligned_to(d_dx, e) ||
        !aligned_to(d_state_in, 4) || !aligned_to(d_dstate_out, 4) || !aligned_to(d_dstate_in, 4))
        return BLOAD_EALIGN;
    if (!states_apart(d_dstate_out, d_dstate_in, num_blocks, t_blk, feat_dim) || !states_apart(d_state_in, d_dstate_in, num_blocks, t_blk, feat_dim))
        return BLOAD_EINVAL;
    GatedArgs a = {};
    a.gate = d_gate;
    a.x = d_dout;
    a.h = d_out;
    a.reset = d_reset;
    a.valid = d_valid;
    a.in = d_dstate_out;
    a.h0 = d_state_in;
    a.y = d_dx;
    a.dgate = d_dgate;
    a.last = d_dstate_in;
    a.T = t_blk;
    a.D = (int32_t)feat_dim;
    return gated_by_type<true>(a, num_blocks, dtype, d_workspace, workspace_bytes, (hipStream_t)hip_stream);
}
