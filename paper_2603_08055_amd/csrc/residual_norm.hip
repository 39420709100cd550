// The residual stream of a block with the norms around it, for rows of `width` channels, and the gradient.
//   u = post(f) (or f),  r = x + s u,  s = residual_scale * scale[channel] * gate[sequence][channel],  y = norm(r),
//   norm(z) = n weight + bias,  n = (z - [layer] mean z) / sigma.
//   Gradient, from x and f once more and not from stored statistics (r as it is before its rounding):
//   g = dy weight,  dr' = dr + (g - [layer] mean g - n mean(g n)) / sigma,  dx = dr',  du = s dr',
//   g' = du post_weight,  df = (g' - [layer] mean g' - n' mean(g' n')) / sigma',
//   and over the rows: d weight = sum dy n, d bias = sum dy, d post_weight = sum du n', d post_bias = sum du,
//   d scale = residual_scale sum gate dr' u,  d gate[b] = residual_scale scale (sum over sequence b) dr' u.
//
// Bound by HBM: every row is read once and written once.  A row is in the registers of L lanes of one wave, or of W waves, CH
// chunks of eight channels in each; sums over a row are lane moves, and a trip through LDS where waves share one.  Sums over rows stay in
// registers for the rows of a workgroup, which follow one another; what the workgroups have is added up by another launch in a
// fixed order.
#include "s3r_lanes_device.h"

namespace s3r {

namespace {

constexpr int threads_of(int w) { return w > 4 ? 64 * w : 256; }

// A thread's part of a row, and sums over rows of channels.
template <int L, int W, int CH> struct RowPart {
    static constexpr int kRows = W == 1 ? 4 * (64 / L) : threads_of(W) / (64 * W);  // of a workgroup at a time
    int sub, chunk0;
    bool has[CH];
    float *lds;   // [2][waves][2]
    int turn;
    __device__ __forceinline__ RowPart(int width, float *lds_) : lds(lds_), turn(0)
    {
        const int t = threadIdx.x;
        sub = t / (L * W);
        chunk0 = t % (L * W);
#pragma unroll
        for (int i = 0; i < CH; ++i) has[i] = at(i) < width;
    }
    __device__ __forceinline__ int at(int i) const { return 8 * (chunk0 + L * W * i); }
    // Sums of a and b over the row, to all of its threads.  One barrier: a wave writes a buffer again only two sums on.
    __device__ __forceinline__ void sum2(float &a, float &b)
    {
        a = sum_over_lanes<L>(a);
        b = sum_over_lanes<L>(b);
        if constexpr (W > 1) {
            const int wave = threadIdx.x >> 6, mine = wave / W * W;
            float *to = lds + turn * (2 * (threads_of(W) / 64));
            if ((threadIdx.x & 63) == 0) { to[2 * wave] = a; to[2 * wave + 1] = b; }
            lds_barrier();
            a = b = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) { a += to[2 * (mine + w)]; b += to[2 * (mine + w) + 1]; }
            turn ^= 1;
        }
    }
};

template <typename T, int CH> struct Raw {
    Io8<T> v[CH];
    template <typename Part> __device__ __forceinline__ void load(const T *row, const Part &part, bool ok)
    {
#pragma unroll
        for (int i = 0; i < CH; ++i)
            if (ok && part.has[i]) v[i].load(row + part.at(i));
    }
    template <typename Part> __device__ __forceinline__ void get(float (&x)[CH][8], const Part &part) const
    {
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) x[i][j] = part.has[i] ? v[i].get(j) : 0.f;
    }
};

template <typename T, int CH, typename Part> __device__ __forceinline__ void store_row(T *row, const float (&x)[CH][8], const Part &part, bool ok)
{
#pragma unroll
    for (int i = 0; i < CH; ++i)
        if (ok && part.has[i]) Io8<T>::store(row + part.at(i), x[i]);
}

template <int CH, typename Part> __device__ __forceinline__ void channel_weights(const void *from, bool is_bf16, const Part &part, float none, float (&w)[CH][8])
{
#pragma unroll
    for (int i = 0; i < CH; ++i) load_weights(from, is_bf16, part.at(i), part.has[i], none, w[i]);
}

// z -> n, and 1 / sigma.  The mean is taken twice, of z and of what is left, so that one much larger than the spread costs no bits.
template <int CH, typename Part> __device__ __forceinline__ float row_norm(int kind, float eps, float of_width, Part &part, float (&z)[CH][8])
{
    if (kind == kNormLayer) {
        float s = 0.f, none = 0.f;
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) s += z[i][j];
        part.sum2(s, none);
        const float mean = s * of_width;
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) z[i][j] = part.has[i] ? z[i][j] - mean : 0.f;
    }
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            s1 += z[i][j];
            s2 = fmaf(z[i][j], z[i][j], s2);
        }
    part.sum2(s1, s2);
    s1 = kind == kNormLayer ? s1 * of_width : 0.f;
    s2 *= of_width;
    const float inv = inverse_root(fmaxf(fmaf(-s1, s1, s2), 0.f) + 0.f * s2 + eps);  // (a NaN stays one)
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) z[i][j] = part.has[i] ? (z[i][j] - s1) * inv : 0.f;
    return inv;
}

// g, the gradient of n, becomes that of z (0 in chunks behind the row's end, which count in later sums).
template <int CH, typename Part>
__device__ __forceinline__ void row_norm_back(int kind, float of_width, float inv, const float (&n)[CH][8], Part &part, float (&g)[CH][8])
{
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            s1 += g[i][j];
            s2 = fmaf(g[i][j], n[i][j], s2);
        }
    part.sum2(s1, s2);
    s1 = kind == kNormLayer ? s1 * of_width : 0.f;
    s2 *= of_width;
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) g[i][j] = part.has[i] ? inv * (g[i][j] - s1 - n[i][j] * s2) : 0.f;
}

// The sequence that has this row (the last that starts at or before it): 64 starts looked at together.  The same row in all lanes.
__device__ __forceinline__ int find_sequence(const Spans &spans, int64_t row)
{
    if (spans.start == nullptr) return 0;
    const int lane = threadIdx.x & 63;
    int lo = 0, count = spans.batch;
    while (count > 1) {
        const int step = (count + 63) / 64, mine = lo + lane * step;
        const bool before = lane * step < count && spans.start[mine] <= row;
        const int n = __popcll(__ballot(before));
        lo += (n < 1 ? 0 : n - 1) * step;
        count = min(step, spans.batch - lo);
    }
    return lo;
}

// FULL: with a post-norm or gates.
template <typename TX, typename T, int L, int W, int CH, bool FULL> __global__ __launch_bounds__(threads_of(W)) void residual_kernel(ResidualArgs a)
{
    __shared__ float lds[2 * 2 * (threads_of(W) / 64)];
    RowPart<L, W, CH> part(a.width, lds);
    const float of_width = 1.f / static_cast<float>(a.width);
    const int64_t r0 = static_cast<int64_t>(blockIdx.x) * a.rows_per_block, r1 = min(r0 + a.rows_per_block, a.n);
    const TX *x_at = static_cast<const TX *>(a.x);
    const T *f_at = static_cast<const T *>(a.f), *gate_at = static_cast<const T *>(a.gate);
    float w[CH][8], b[CH][8], scale[CH][8], pw[CH][8], pb[CH][8];
    int seq = 0;
    int64_t lo = 0, hi = a.n;
    Raw<TX, CH> x;
    Raw<T, CH> f, gate;
    auto request = [&](int64_t row, bool ok) {
        x.load(x_at + row * a.x_row, part, ok);
        if (f_at != nullptr) f.load(f_at + row * a.f_row, part, ok);
        if constexpr (FULL)
            if (gate_at != nullptr) {
                if (a.spans.start != nullptr)
                    while (ok && seq + 1 < a.spans.batch && a.spans.start[seq + 1] <= row) ++seq;
                gate.load(gate_at + seq * a.gate_row, part, ok);
            }
    };
    if constexpr (FULL)
        if (a.spans.start != nullptr) {
            seq = find_sequence(a.spans, r0);
            lo = a.spans.start[0];
            hi = a.spans.start[a.spans.batch];
        }
    auto counts = [&](int64_t row) { return row < r1 && row >= lo && row < hi; };
    request(r0 + part.sub, counts(r0 + part.sub));
    channel_weights<CH>(a.weight, a.w_bf16, part, 1.f, w);
    channel_weights<CH>(a.bias, a.w_bf16, part, 0.f, b);
    channel_weights<CH>(a.scale, a.w_bf16, part, 1.f, scale);
    if constexpr (FULL) {
        channel_weights<CH>(a.post_weight, a.w_bf16, part, 1.f, pw);
        channel_weights<CH>(a.post_bias, a.w_bf16, part, 0.f, pb);
    }
    for (int64_t first = r0; first < r1; first += part.kRows) {
        const int64_t row = first + part.sub;
        const bool ok = counts(row);
        float z[CH][8], u[CH][8];
        x.get(z, part);
        if (f_at != nullptr) {
            f.get(u, part);
            float g[CH][8];
            if constexpr (FULL)
                if (gate_at != nullptr) gate.get(g, part);
            request(row + part.kRows, counts(row + part.kRows));
            if constexpr (FULL)
                if (a.post != kNormNone) {
                    row_norm<CH>(a.post, a.eps, of_width, part, u);
#pragma unroll
                    for (int i = 0; i < CH; ++i)
#pragma unroll
                        for (int j = 0; j < 8; ++j) u[i][j] = fmaf(u[i][j], pw[i][j], pb[i][j]);
                }
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float s = a.residual_scale * scale[i][j];
                    if constexpr (FULL)
                        if (gate_at != nullptr) s *= g[i][j];
                    z[i][j] = fmaf(s, u[i][j], z[i][j]);
                }
        } else {
            request(row + part.kRows, counts(row + part.kRows));
        }
        if (a.r != nullptr) store_row<TX, CH>(static_cast<TX *>(a.r) + row * a.width, z, part, ok);
        if (a.y == nullptr) continue;
        row_norm<CH>(a.norm, a.eps, of_width, part, z);
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) z[i][j] = fmaf(z[i][j], w[i][j], b[i][j]);
        store_row<T, CH>(static_cast<T *>(a.y) + row * a.width, z, part, ok);
    }
}

// A workgroup's sums over rows, of each of its threads' channels, to `to` [width].  Rows of a workgroup side by side are added up in LDS.
template <int L, int W, int CH, typename Part> __device__ __forceinline__ void store_sums(const float (&s)[CH][8], float *to, int width, const Part &part, float *lds)
{
    constexpr int kRows = Part::kRows;
    if constexpr (kRows == 1) {
#pragma unroll
        for (int i = 0; i < CH; ++i)
            if (part.has[i]) Io8<float>::store(to + part.at(i), s[i]);
        return;
    } else {
        constexpr int kWidth = 8 * L * W;   // channels of one chunk of all threads of a row
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) lds[part.sub * kWidth + j * (L * W) + part.chunk0] = s[i][j];
            __syncthreads();
            for (int c = threadIdx.x; c < kWidth; c += threads_of(W)) {
                const int channel = kWidth * i + 8 * (c % (L * W)) + c / (L * W);
                if (channel >= width) continue;
                float sum = 0.f;
#pragma unroll
                for (int r = 0; r < kRows; ++r) sum += lds[r * kWidth + c];
                to[channel] = sum;
            }
        }
    }
}

template <typename TX, typename T, int L, int W, int CH, bool FULL> __global__ __launch_bounds__(threads_of(W)) void residual_grad_kernel(ResidualArgs a)
{
    using Part = RowPart<L, W, CH>;
    __shared__ float lds[2 * 2 * (threads_of(W) / 64)];
    __shared__ float join[Part::kRows > 1 ? Part::kRows * 8 * L * W : 1];
    Part part(a.width, lds);
    const float of_width = 1.f / static_cast<float>(a.width);
    const int64_t r0 = static_cast<int64_t>(blockIdx.x) * a.rows_per_block, r1 = min(r0 + a.rows_per_block, a.n);
    float w[CH][8], scale[CH][8], pw[CH][8], pb[CH][8], gate[CH][8];
    channel_weights<CH>(a.weight, a.w_bf16, part, 1.f, w);
    channel_weights<CH>(a.scale, a.w_bf16, part, 1.f, scale);
    if constexpr (FULL) {
        channel_weights<CH>(a.post_weight, a.w_bf16, part, 1.f, pw);
        channel_weights<CH>(a.post_bias, a.w_bf16, part, 0.f, pb);
    }
    float dw[CH][8], db[CH][8], ds[CH][8], dpw[CH][8], dpb[CH][8], dg[CH][8];
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[i][j] = db[i][j] = ds[i][j] = dpw[i][j] = dpb[i][j] = dg[i][j] = 0.f, gate[i][j] = 1.f;
    const TX *x_at = static_cast<const TX *>(a.x), *dr_at = static_cast<const TX *>(a.d_r);
    const T *f_at = static_cast<const T *>(a.f), *dy_at = static_cast<const T *>(a.d_y);
    auto rows_of = [&](int64_t from, int64_t to) {
        Raw<TX, CH> x, dr;
        Raw<T, CH> f, dy;
        auto request = [&](int64_t row) {
            const bool ok = row < to;
            x.load(x_at + row * a.x_row, part, ok);
            if (f_at != nullptr) f.load(f_at + row * a.f_row, part, ok);
            if (dy_at != nullptr) dy.load(dy_at + row * a.width, part, ok);
            if (dr_at != nullptr) dr.load(dr_at + row * a.width, part, ok);
        };
        request(from + part.sub);
        for (int64_t first = from; first < to; first += Part::kRows) {
            const int64_t row = first + part.sub;
            const bool ok = row < to;
            float z[CH][8], u[CH][8], g[CH][8], d[CH][8];
            x.get(z, part);
            if (f_at != nullptr) f.get(u, part);
            if (dy_at != nullptr) dy.get(g, part);
            if (dr_at != nullptr) dr.get(d, part);
            request(row + Part::kRows);
            float post_inv = 0.f;
            if constexpr (FULL)
                if (a.post != kNormNone) post_inv = row_norm<CH>(a.post, a.eps, of_width, part, u);
            auto branch = [&](int i, int j) {  // u of the formulas
                if constexpr (FULL) return fmaf(u[i][j], pw[i][j], pb[i][j]);
                return u[i][j];
            };
            auto factor = [&](int i, int j) {
                float s = a.residual_scale * scale[i][j];
                if constexpr (FULL) s *= gate[i][j];
                return s;
            };
            if (dr_at == nullptr)
#pragma unroll
                for (int i = 0; i < CH; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[i][j] = 0.f;
            if (dy_at != nullptr) {
                if (f_at != nullptr)
#pragma unroll
                    for (int i = 0; i < CH; ++i)
#pragma unroll
                        for (int j = 0; j < 8; ++j) z[i][j] = fmaf(factor(i, j), branch(i, j), z[i][j]);
                const float inv = row_norm<CH>(a.norm, a.eps, of_width, part, z);
#pragma unroll
                for (int i = 0; i < CH; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if (ok) {
                            dw[i][j] = fmaf(g[i][j], z[i][j], dw[i][j]);
                            db[i][j] += g[i][j];
                        }
                        g[i][j] *= w[i][j];
                    }
                row_norm_back<CH>(a.norm, of_width, inv, z, part, g);
#pragma unroll
                for (int i = 0; i < CH; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[i][j] += g[i][j];
            }
            store_row<TX, CH>(static_cast<TX *>(a.dx) + row * a.width, d, part, ok);
            if (f_at == nullptr) continue;
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float t = d[i][j] * branch(i, j);
                    d[i][j] *= factor(i, j);
                    if (!ok) continue;
                    if constexpr (FULL) {
                        ds[i][j] = fmaf(gate[i][j], t, ds[i][j]);
                        dg[i][j] += t;
                        dpw[i][j] = fmaf(d[i][j], u[i][j], dpw[i][j]);
                        dpb[i][j] += d[i][j];
                    } else {
                        ds[i][j] += t;
                    }
                }
            if constexpr (FULL)
                if (a.post != kNormNone) {
#pragma unroll
                    for (int i = 0; i < CH; ++i)
#pragma unroll
                        for (int j = 0; j < 8; ++j) d[i][j] *= pw[i][j];
                    row_norm_back<CH>(a.post, of_width, post_inv, u, part, d);
                }
            store_row<T, CH>(static_cast<T *>(a.df) + row * a.width, d, part, ok);
        }
    };
    if (FULL && a.gate != nullptr) {
        // sequence by sequence; what a workgroup's rows of sequence b give goes to place blockIdx.x + b, which no other pair has
        int seq = find_sequence(a.spans, r0);
        for (; seq < a.spans.batch; ++seq) {
            int first, len;
            a.spans.of(seq, first, len);
            if (first >= r1) break;
            const int64_t from = max(r0, static_cast<int64_t>(first)), to = min(r1, static_cast<int64_t>(first) + len);
            if (from >= to) continue;
            Raw<T, CH> raw;
            raw.load(static_cast<const T *>(a.gate) + seq * a.gate_row, part, true);
            raw.get(gate, part);
            rows_of(from, to);
            if (a.part_gate != nullptr)
                store_sums<L, W, CH>(dg, a.part_gate + (static_cast<int64_t>(blockIdx.x) + seq) * a.width, a.width, part, join);
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) dg[i][j] = 0.f;
        }
    } else {
        rows_of(r0, r1);
    }
    const int64_t share = static_cast<int64_t>(gridDim.x) * a.width;
    float *to = a.part + blockIdx.x * static_cast<int64_t>(a.width);
    if (a.part == nullptr) return;
    if (a.d_weight != nullptr) store_sums<L, W, CH>(dw, to, a.width, part, join);
    if (a.d_bias != nullptr) store_sums<L, W, CH>(db, to + share, a.width, part, join);
    if (a.d_scale != nullptr) store_sums<L, W, CH>(ds, to + 2 * share, a.width, part, join);
    if constexpr (FULL) {
        if (a.d_post_weight != nullptr) store_sums<L, W, CH>(dpw, to + 3 * share, a.width, part, join);
        if (a.d_post_bias != nullptr) store_sums<L, W, CH>(dpb, to + 4 * share, a.width, part, join);
    }
}

// Sums over the workgroups, 32 channels of one tensor (blockIdx.y) for a workgroup of eight groups.
__global__ __launch_bounds__(256) void residual_sums_kernel(ResidualArgs a, int blocks)
{
    const int which = blockIdx.y, c = threadIdx.x & 31, group = threadIdx.x >> 5, channel = blockIdx.x * 32 + c;
    void *to = which == 0 ? a.d_weight : (which == 1 ? a.d_bias : (which == 2 ? a.d_scale : (which == 3 ? a.d_post_weight : a.d_post_bias)));
    if (to == nullptr) return;
    __shared__ float sums[8][32];
    float s = 0.f;
    if (channel < a.width)
        for (int i = group; i < blocks; i += 8) s += a.part[(static_cast<int64_t>(which) * blocks + i) * a.width + channel];
    sums[group][c] = s;
    __syncthreads();
    if (group != 0 || channel >= a.width) return;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += sums[i][c];
    store_weight(to, a.w_bf16, channel, which == 2 ? s * a.residual_scale : s);
}

// The gradient of a sequence's gate: the sum over the workgroups that had rows of it.
template <typename T> __global__ __launch_bounds__(256) void residual_gate_kernel(ResidualArgs a)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int64_t seq = i / a.width;
    if (seq >= a.spans.batch) return;
    const int c = static_cast<int>(i - seq * a.width);
    int first, len;
    a.spans.of(static_cast<int>(seq), first, len);
    float s = 0.f;
    if (len > 0)
        for (int64_t g = first / a.rows_per_block; g <= (static_cast<int64_t>(first) + len - 1) / a.rows_per_block; ++g)
            s += a.part_gate[(g + seq) * a.width + c];
    s *= a.residual_scale;
    if (a.scale != nullptr) s *= a.w_bf16 ? static_cast<float>(static_cast<const bf16_t *>(a.scale)[c]) : static_cast<const float *>(a.scale)[c];
    static_cast<T *>(a.d_gate)[i] = from_float<T>(s);
}

// Rows of up to 128, 512, 1024, 4096 and 8192 channels.
template <typename TX, typename T, bool FULL, typename Launch> hipError_t by_width(int width, Launch &&launch)
{
    if (width <= 128) return launch(&residual_kernel<TX, T, 16, 1, 1, FULL>, &residual_grad_kernel<TX, T, 16, 1, 1, FULL>, 256);
    if (width <= 512) return launch(&residual_kernel<TX, T, 64, 1, 1, FULL>, &residual_grad_kernel<TX, T, 64, 1, 1, FULL>, 256);
    if (width <= 1024) return launch(&residual_kernel<TX, T, 64, 1, 2, FULL>, &residual_grad_kernel<TX, T, 64, 1, 2, FULL>, 256);
    if (width <= 4096) return launch(&residual_kernel<TX, T, 64, 4, 2, FULL>, &residual_grad_kernel<TX, T, 64, 4, 2, FULL>, 256);
    return launch(&residual_kernel<TX, T, 64, 8, 2, FULL>, &residual_grad_kernel<TX, T, 64, 8, 2, FULL>, 512);
}

template <typename Launch> hipError_t by_type(const ResidualArgs &a, bool x_bf16, bool is_bf16, Launch &&launch)
{
    const bool full = a.post != kNormNone || a.gate != nullptr;
    if (!is_bf16) return full ? by_width<float, float, true>(a.width, launch) : by_width<float, float, false>(a.width, launch);
    if (x_bf16) return full ? by_width<bf16_t, bf16_t, true>(a.width, launch) : by_width<bf16_t, bf16_t, false>(a.width, launch);
    return full ? by_width<float, bf16_t, true>(a.width, launch) : by_width<float, bf16_t, false>(a.width, launch);
}

}  // namespace

hipError_t launch_residual(const ResidualArgs &a, bool x_bf16, bool is_bf16, hipStream_t stream)
{
    const int64_t blocks = (a.n + a.rows_per_block - 1) / a.rows_per_block;
    return by_type(a, x_bf16, is_bf16, [&](auto kernel, auto, int threads) {
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks)), dim3(threads), 0, stream, a);
        return hipGetLastError();
    });
}

hipError_t launch_residual_grad(const ResidualArgs &a, bool x_bf16, bool is_bf16, hipStream_t stream)
{
    const int64_t blocks = (a.n + a.rows_per_block - 1) / a.rows_per_block;
    if (blocks > 0) {
        const hipError_t e = by_type(a, x_bf16, is_bf16, [&](auto, auto kernel, int threads) {
            hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks)), dim3(threads), 0, stream, a);
            return hipGetLastError();
        });
        if (e != hipSuccess) return e;
    }
    if (a.d_weight != nullptr || a.d_bias != nullptr || a.d_scale != nullptr || a.d_post_weight != nullptr || a.d_post_bias != nullptr) {
        hipLaunchKernelGGL(residual_sums_kernel, dim3((a.width + 31) / 32, 5), dim3(256), 0, stream, a, static_cast<int>(blocks));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.d_gate == nullptr) return hipSuccess;
    const int64_t gates = (static_cast<int64_t>(a.spans.batch) * a.width + 255) / 256;
    if (is_bf16)
        hipLaunchKernelGGL(residual_gate_kernel<bf16_t>, dim3(static_cast<unsigned>(gates)), dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL(residual_gate_kernel<float>, dim3(static_cast<unsigned>(gates)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace s3r
