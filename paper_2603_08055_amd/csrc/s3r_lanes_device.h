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

// Sums of N tensors' rows (fp32 or 64 bits) `stride` apart, `count` of them, the tensors `gap` apart, of 16 channels, by a workgroup of 1024 threads: a thread
// takes four channels (from: the first of its own, 4 (thread mod 4); ok: they are there) of every 256th row, AT_ONCE of them requested together.  In
// 64 bits, which cost nothing here, in a fixed order.  To threads 0 .. 15, a channel each.
template <int N> struct PartSums { double rows[N][128][16], groups[N][16][16]; };
template <int N, int AT_ONCE, typename P> __device__ __forceinline__ void sum_parts(const P *from, int64_t count, int64_t stride, int64_t gap, bool ok, PartSums<N> &lds, double (&s)[N])
{
    typedef P P4 __attribute__((ext_vector_type(4)));
    const int t = threadIdx.x, lane = t & 63;
    double own[N][4] = {};
    if (ok)
        for (int64_t i = t >> 2; i < count; i += 256 * AT_ONCE) {
            P4 x[N][AT_ONCE];
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k)
                    x[n][k] = i + 256 * k < count ? *reinterpret_cast<const P4 *>(from + n * gap + (i + 256 * k) * stride) : P4{};
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k)
#pragma unroll
                    for (int e = 0; e < 4; ++e) own[n][e] += x[n][k][e];
        }
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            own[n][e] += __shfl_xor(own[n][e], 32, 64);
            if (lane < 32) lds.rows[n][(t >> 6) * 8 + (lane >> 2)][4 * (t & 3) + e] = own[n][e];
        }
    __syncthreads();
    if (t < 256 * N) {
        double x = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) x += lds.rows[t >> 8][8 * ((t >> 4) & 15) + i][t & 15];
        lds.groups[t >> 8][(t >> 4) & 15][t & 15] = x;
    }
    __syncthreads();
    if (t >= 16) return;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        s[n] = 0.0;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[n] += lds.groups[n][i][t];
    }
}

}  // namespace s3r
