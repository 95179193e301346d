// bload_segment_mask: for every slot of the packed blocks the interval of slots whose keys its query
// may look at, and the interval of slots whose queries look at its key.
//
// A sequence lies in consecutive slots [f, e) of one block.  Without order every slot t of it sees
// [f, e); causally it sees [f, t + 1), and with a prefix of p frames [f, max(t + 1, min(f + p, e))):
// in every case an interval, and so is what sees a key (the transposed relation): [f, e), or causally
// [t, e) beyond the prefix and [f, e) inside it.  The attention kernels need no other mask.
#include "bload_common.hpp"

namespace bload {
namespace {

constexpr int kSlotsPerThread = 4;
constexpr int kMaskTile = kThreads * kSlotsPerThread;

struct MaskArgs {
    const uint8_t *reset, *valid;
    const int32_t *seq_id, *prefix;      // both or neither
    int4* out;
    int64_t n_seq;
    int32_t t_blk, tiles, causal;
};

// What a slot is: bit 0 a sequence starts here, bit 1 a sequence that lay in front of it has ended.
__device__ __forceinline__ int slot_kind(const uint8_t* reset, const uint8_t* valid, int32_t t)
{
    if (!valid[t]) return 2;
    return (t == 0 || reset[t] || !valid[t - 1]) ? 3 : 0;
}

// A workgroup takes 1024 consecutive slots of a block.  Where the sequence of its first slot began and
// where that of its last one ends it looks up itself, 1024 flags a step: 32768 slots without a start are
// 32 steps.  Latency bound (two passes of a scan over 256 lanes); the writes are 16 bytes a slot:
// 1.5 MB for 24 blocks of 4096 slots.
__global__ __launch_bounds__(kThreads) void segment_mask_kernel(MaskArgs a)
{
    __shared__ int32_t lasts[kThreads / kWave], firsts[kThreads / kWave];
    const int64_t b = blockIdx.x / a.tiles;
    const int32_t t0 = (int32_t)(blockIdx.x % a.tiles) * kMaskTile, T = a.t_blk;
    const uint8_t* reset = a.reset + b * T;
    const uint8_t* valid = a.valid + b * T;
    const int lane = lane_id(), wave = wave_id(), tid = (int)threadIdx.x;

    // kinds of this thread's slots, its last start and its first end
    int kind[kSlotsPerThread];
    int32_t last = -1, first = T;
    const int32_t mine = t0 + tid * kSlotsPerThread;
#pragma unroll
    for (int j = 0; j < kSlotsPerThread; ++j) {
        kind[j] = mine + j < T ? slot_kind(reset, valid, mine + j) : 2;
        if (kind[j] & 1) last = mine + j;
    }
#pragma unroll
    for (int j = kSlotsPerThread - 1; j >= 0; --j)
        if (mine + j < T && (kind[j] & 2)) first = mine + j;
    // inclusive maximum over the threads in front, inclusive minimum over those behind
    int32_t inc_last = last, inc_first = first;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const int32_t u = __shfl_up(inc_last, d), v = __shfl_down(inc_first, d);
        if (lane >= d) inc_last = max(inc_last, u);
        if (lane + d < kWave) inc_first = min(inc_first, v);
    }
    if (lane == kWave - 1) lasts[wave] = inc_last;
    if (lane == 0) firsts[wave] = inc_first;
    // the sequence that reaches into the tile from the left, and where the one that leaves it ends
    int32_t from = -1, to = T;
    const int32_t end = min(t0 + kMaskTile, T);
    if (t0 > 0 && valid[t0] && slot_kind(reset, valid, t0) == 0) {
        for (int32_t hi = t0; hi > 0 && from < 0; hi -= kMaskTile) {
            int32_t at = -1;
            for (int j = 0; j < kSlotsPerThread; ++j) {
                const int32_t t = hi - 1 - (tid * kSlotsPerThread + j);
                if (t >= 0 && at < 0 && (slot_kind(reset, valid, t) & 1)) at = t;
            }
            for (int d = 1; d < kWave; d <<= 1) at = max(at, __shfl_xor(at, d));
            __shared__ int32_t found[kThreads / kWave];
            if (lane == 0) found[wave] = at;
            __syncthreads();
            from = max(max(found[0], found[1]), max(found[2], found[3]));
            __syncthreads();
        }
    }
    for (int32_t lo = end; lo < T && to == T; lo += kMaskTile) {
        int32_t at = T;
        for (int j = kSlotsPerThread - 1; j >= 0; --j) {
            const int32_t t = lo + tid * kSlotsPerThread + j;
            if (t < T && (slot_kind(reset, valid, t) & 2)) at = t;
        }
        for (int d = 1; d < kWave; d <<= 1) at = min(at, __shfl_xor(at, d));
        __shared__ int32_t found[kThreads / kWave];
        if (lane == 0) found[wave] = at;
        __syncthreads();
        to = min(min(found[0], found[1]), min(found[2], found[3]));
        __syncthreads();
    }
    __syncthreads();
    int32_t before = from, behind = to;                  // of this thread's first slot, of its last one
    for (int w = 0; w < wave; ++w) before = max(before, lasts[w]);
    for (int w = kThreads / kWave - 1; w > wave; --w) behind = min(behind, firsts[w]);
    const int32_t up = __shfl_up(inc_last, 1), down = __shfl_down(inc_first, 1);
    if (lane > 0) before = max(before, up);
    if (lane < kWave - 1) behind = min(behind, down);

    int32_t ends[kSlotsPerThread];
    int32_t e = behind;
#pragma unroll
    for (int j = kSlotsPerThread - 1; j >= 0; --j) {
        ends[j] = e;
        if (kind[j] & 2) e = mine + j;
    }
    int32_t f = before;
#pragma unroll
    for (int j = 0; j < kSlotsPerThread; ++j) {
        const int32_t t = mine + j;
        if (t >= T) break;
        if (kind[j] & 1) f = t;
        int4 r = make_int4(0, 0, 0, 0);
        if (kind[j] != 2) {
            int32_t head = 0;
            if (a.prefix) {
                const int64_t id = a.seq_id[b * T + t];
                if (id >= 0 && id < a.n_seq) head = min(max(a.prefix[id], 0), ends[j] - f);
            }
            r.x = f;
            r.y = a.causal ? max(t + 1, f + head) : ends[j];
            r.z = a.causal && t >= f + head ? t : f;
            r.w = ends[j];
        }
        a.out[b * T + t] = r;
    }
}

}  // namespace
}  // namespace bload

using namespace bload;

extern "C" bload_status bload_segment_mask(const uint8_t* d_reset, const uint8_t* d_valid, const int32_t* d_seq_id,
                                           int64_t num_blocks, int32_t t_blk, int32_t causal, const int32_t* d_prefix,
                                           int64_t n_seq, int32_t* d_mask, void* hip_stream)
{
    if (num_blocks < 0 || t_blk < 1 || n_seq < 0 || (causal != 0 && causal != 1)) return BLOAD_EINVAL;
    if (d_prefix && !d_seq_id) return BLOAD_EINVAL;
    if (t_blk > (1 << 30) || num_blocks >= ((int64_t)1 << 40) / t_blk || n_seq > BLOAD_MAX_SEQ) return BLOAD_EOVERFLOW;
    if (num_blocks == 0) return BLOAD_OK;
    if (!d_reset || !d_valid || !d_mask) return BLOAD_EINVAL;
    if (!aligned_to(d_mask, 16) || !aligned_to(d_seq_id, 4) || !aligned_to(d_prefix, 4)) return BLOAD_EALIGN;
    const int64_t tiles = ceil_div(t_blk, kMaskTile), groups = num_blocks * tiles;
    if (groups > kMaxGroups) return BLOAD_EOVERFLOW;
    const MaskArgs a = {d_reset, d_valid, d_seq_id, d_prefix, reinterpret_cast<int4*>(d_mask), n_seq, t_blk, (int32_t)tiles, causal};
    segment_mask_kernel<<<dim3((unsigned)groups), dim3(kThreads), 0, (hipStream_t)hip_stream>>>(a);
    return launch_status();
}
