// Sums over neighbouring lanes and the statistics of a norm, shared by the kernels that go once over their rows (rotary.hip,
// residual_norm.hip).  No trips to LDS: permutations of four lanes, mirrors of eight and sixteen, and the swaps of rows of sixteen and of
// half-waves.  All lanes of a wave take part.
#pragma once
#include "s3r_attn_device.h"

namespace s3r {

template <int CTRL> __device__ __forceinline__ float lane_moved(float x)
{
    return __uint_as_float(static_cast<unsigned>(__builtin_amdgcn_mov_dpp(static_cast<int>(__float_as_uint(x)), CTRL, 0xf, 0xf, true)));
}

// The sum over each run of L lanes (8, 16, 32 or 64), to all of them.
template <int L> __device__ __forceinline__ float sum_over_lanes(float x)
{
    static_assert(L == 8 || L == 16 || L == 32 || L == 64, "");
    x += lane_moved<0xb1>(x);   // lanes 1 apart
    x += lane_moved<0x4e>(x);   // 2 apart
    x += lane_moved<0x141>(x);  // the mirror of eight
    if constexpr (L >= 16) x += lane_moved<0x140>(x);  // of sixteen
    if constexpr (L >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if constexpr (L == 64) x = sum_with_other_half(x);
    return x;
}

// 1 / sqrt(x) for normal x: the hardware's estimate (off by up to 2^-23 of it) and a step of Newton's method, off by 2^-24 and a little.
__device__ __forceinline__ float inverse_root(float x)
{
    const float y = __builtin_amdgcn_rsqf(x);
    return fmaf(0.5f * y, fmaf(-x * y, y, 1.f), y);
}

// Eight weights of a norm, or of a channel scale, from a tensor of fp32 or bf16 (null: `none` in their place).
__device__ __forceinline__ void load_weights(const void *from, bool is_bf16, int at, bool ok, float none, float (&w)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = none;
    if (from == nullptr || !ok) return;
    if (is_bf16) {
        Io8<bf16_t> v;
        v.load(static_cast<const bf16_t *>(from) + at);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = v.get(j);
    } else {
        Io8<float> v;
        v.load(static_cast<const float *>(from) + at);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = v.get(j);
    }
}

__device__ __forceinline__ void store_weight(void *to, bool is_bf16, int64_t at, float x)
{
    if (is_bf16)
        static_cast<bf16_t *>(to)[at] = static_cast<bf16_t>(x);
    else
        static_cast<float *>(to)[at] = x;
}

}  // namespace s3r
