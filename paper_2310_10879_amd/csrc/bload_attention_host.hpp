// Host side of the attention entry points: argument checks, and the choice of a kernel's instance.
#pragma once

#include <cmath>

#include "bload_attention.hpp"

namespace bload {

template <typename T> struct type_is { using type = T; };

inline size_t att_elem_bytes(bload_dtype dtype) { return dtype == BLOAD_F32 ? 4 : 2; }

inline bool att_dtype(bload_dtype dtype) { return dtype == BLOAD_F16 || dtype == BLOAD_BF16 || dtype == BLOAD_F32; }

// bload_attention_dkv.hip: dk and dv, behind the kernel that leaves delta.
bload_status attention_dkv(const AttArgs& a, bload_dtype dtype, hipStream_t stream);

// Everything but the tensors.  `rows`: slots of a workgroup's tile.
inline bload_status att_args(AttArgs& a, int64_t num_blocks, int32_t t_blk, int32_t heads_q, int32_t heads_kv, int32_t head_dim,
                             bload_dtype dtype, float scale, float cap, const float* d_slopes, const int32_t* d_mask, int rows)
{
    if (num_blocks < 0 || t_blk < 1 || heads_q < 1 || heads_kv < 1 || heads_q % heads_kv != 0 || head_dim < 1 ||
        head_dim > BLOAD_ATTENTION_MAX_HEAD_DIM || !att_dtype(dtype) || !(scale > 0.0f) || !std::isfinite(scale) || !(cap >= 0.0f) ||
        !std::isfinite(cap))
        return BLOAD_EINVAL;
    if (t_blk > (1 << 30) || num_blocks >= ((int64_t)1 << 40) / t_blk) return BLOAD_EOVERFLOW;
    const int64_t tiles = ceil_div(t_blk, rows);
    // one workgroup per tile and head (by division: heads * blocks alone may not fit)
    if (num_blocks > 0 && tiles > kMaxGroups / heads_q / num_blocks) return BLOAD_EOVERFLOW;
    if (num_blocks > 0 && !d_mask) return BLOAD_EINVAL;
    if (!aligned_to(d_mask, 16) || !aligned_to(d_slopes, 4)) return BLOAD_EALIGN;
    a.mask = reinterpret_cast<const int4*>(d_mask);
    a.slopes = d_slopes;
    a.scale = scale;
    a.cap = std::fmin(cap, 0x1p100f);      // what float32 keeps of scores that such a cap moves (2^88 and more) has steps of 2^64
    a.B = (int32_t)num_blocks;
    a.T = t_blk;
    a.Hq = heads_q;
    a.Hkv = heads_kv;
    a.G = heads_q / heads_kv;
    a.D = head_dim;
    a.tiles = (int32_t)tiles;
    return BLOAD_OK;
}

inline bload_status att_tensor(AttTensor& t, const bload_heads* h, bload_dtype dtype)
{
    if (!h || !h->d_data) return BLOAD_EINVAL;
    if (!aligned_to(h->d_data, att_elem_bytes(dtype))) return BLOAD_EALIGN;
    t = {h->d_data, h->block_stride, h->slot_stride, h->head_stride};
    return BLOAD_OK;
}

// Heads are padded with zeros to 32, 64, 96 or 128 elements.
template <typename T, typename F>
inline void att_dispatch_dim(int32_t D, F f)
{
    if (D <= 32) f(type_is<T>(), std::integral_constant<int, 32>());
    else if (D <= 64) f(type_is<T>(), std::integral_constant<int, 64>());
    else if (D <= 96) f(type_is<T>(), std::integral_constant<int, 96>());
    else f(type_is<T>(), std::integral_constant<int, 128>());
}
template <typename F>
inline void att_dispatch(bload_dtype dtype, int32_t D, F f)
{
    if (dtype == BLOAD_F16) att_dispatch_dim<att_half>(D, f);
    else if (dtype == BLOAD_BF16) att_dispatch_dim<att_bf16>(D, f);
    else att_dispatch_dim<float>(D, f);
}

// A kernel's variant: what it does to scores, and for heads that are no whole number of 16 bytes (which come with a bias at least,
// of slope 0 if need be: fewer instances of what loads slowly anyway).
template <typename T, typename F>
inline void att_variant(const AttArgs& a, F f)
{
    using bias = std::integral_constant<int, kBias>;
    using cap = std::integral_constant<int, kCap>;
    using cap_far = std::integral_constant<int, sizeof(T) == 2 ? kCapFar : kCap>;
    if (a.D % (16 / (int)sizeof(T))) {
        if (a.cap > kNearCap) f(cap_far(), std::true_type());
        else if (a.cap > 0.0f) f(cap(), std::true_type());
        else f(bias(), std::true_type());
    } else if (a.cap > kNearCap) {
        f(cap_far(), std::false_type());
    } else if (a.cap > 0.0f) {
        f(cap(), std::false_type());
    } else if (a.slopes) {
        f(bias(), std::false_type());
    } else {
        f(std::integral_constant<int, kPlain>(), std::false_type());
    }
}

}  // namespace bload
