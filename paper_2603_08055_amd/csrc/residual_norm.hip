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
// fixed order.  256 terms and fewer are added in fp32 by a thread, then those of the workgroup's rows side by side; the rest in 64 bits.
// Rows of 1024: 137400 with an fp32 stream beside bf16, channel scale and LayerNorm, 337 us, 5.0 TB/s, the rate of a copy of as much (4.97);
// 41220 all in bf16 60 us, 5.6 TB/s, their gradient 109 us, 4.65 TB/s (six tensors at once), and 6 us for the sums.  3001 rows of 1000 in
// fp32 with a post-norm and gates: 13 us (3.7 TB/s) and 25 + 6 (2.8 TB/s): four sums over a row, one after the other, and six rows for a workgroup, two at a time.
#include "s3r_lanes_device.h"

#include <type_traits>

namespace s3r {

namespace {

constexpr int threads_of(int w) { return w > 4 ? 64 * w : 256; }
// The sums of a gradient over the rows of a workgroup, in the workspace: of dy n, of dy, and (see residual_grad_kernel) C, A and B.
enum { kPartWeight, kPartBias, kPartC, kPartA, kPartB };
static_assert(kPartB + 1 == kResidualParts, "");

// A thread's part of a row, and sums over rows of channels.
template <int L, int W, int CH> struct RowPart {
    static constexpr int kRows = threads_of(W) / (L * W);  // of a workgroup at a time
    int sub, chunk0;
    bool has[CH];
    float *lds;   // [2][waves][2]
    int turn;
    __device__ __forceinline__ RowPart(int width, float *lds_) : lds(lds_), turn(0)
    {
        const int t = threadIdx.x;
        sub = t / (L * W);
        if constexpr (L == 64) sub = __builtin_amdgcn_readfirstlane(sub);  // rows and their addresses are scalars then
        chunk0 = t % (L * W);
#pragma unroll
        for (int i = 0; i < CH; ++i) has[i] = at(i) < width;
    }
    __device__ __forceinline__ int at(int i) const { return 8 * (chunk0 + L * W * i); }
    // The thread's i-th chunk of a row (`anyway`: the first chunk where there is none): the row's address, a scalar where a wave has one row, and
    // an offset of 32 bits.
    template <typename T> __device__ __forceinline__ T *chunk(T *row, int i, bool anyway) const
    {
        const unsigned offset = anyway && !has[i] ? 0u : static_cast<unsigned>(at(i)) * static_cast<unsigned>(sizeof(T));
        return reinterpret_cast<T *>(reinterpret_cast<uintptr_t>(row) + offset);
    }
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

// A thread's chunks of a row as they come from memory; those behind the row's end are the row's first (no lane is left out of a load).
template <typename T, int CH> struct Raw {
    Io8<T> v[CH];
    template <typename Part> __device__ __forceinline__ void load(const T *row, const Part &part)
    {
#pragma unroll
        for (int i = 0; i < CH; ++i) v[i].load(part.chunk(row, i, true));
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
        if (ok && part.has[i]) Io8<T>::store(part.chunk(row, i, false), x[i]);
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
    // (rows that there are not: the last)
    auto request = [&](int64_t row) {
        row = min(row, r1 - 1);
        x.load(x_at + row * a.x_row, part);
        if (f_at != nullptr) f.load(f_at + row * a.f_row, part);
        if constexpr (FULL)
            if (gate_at != nullptr) {
                if (a.spans.start != nullptr)
                    while (seq + 1 < a.spans.batch && a.spans.start[seq + 1] <= row) ++seq;
                gate.load(gate_at + seq * a.gate_row, part);
            }
    };
    if constexpr (FULL)
        if (a.spans.start != nullptr) {
            seq = find_sequence(a.spans, r0);
            lo = a.spans.start[0];
            hi = a.spans.start[a.spans.batch];
        }
    auto counts = [&](int64_t row) { return row < r1 && row >= lo && row < hi; };
    request(r0 + part.sub);
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
            request(row + part.kRows);
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
            request(row + part.kRows);
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

// A place [width] for a workgroup's sums: fp32, or (WIDE) 64 bits, where they come in shares (see ResidualArgs::turns), which all but the first are added to it.
template <bool WIDE> struct Place {
    std::conditional_t<WIDE, double, float> *at;
    bool add;
    __device__ __forceinline__ Place(void *base, int64_t offset, bool add_) : at(static_cast<decltype(at)>(base) + offset), add(add_) {}
    __device__ __forceinline__ void put(int channel, float x) const
    {
        if constexpr (WIDE)
            at[channel] = (add ? at[channel] : 0.0) + static_cast<double>(x);
        else
            at[channel] = x;
    }
};

// A workgroup's sums over rows, of each of its threads' channels.  Rows of a workgroup side by side are added up in LDS.
template <int L, int W, int CH, bool WIDE, typename Part> __device__ __forceinline__ void store_sums(const float (&s)[CH][8], const Place<WIDE> &to, int width, const Part &part, float *lds)
{
    constexpr int kRows = Part::kRows;
    if constexpr (kRows == 1) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            if (!part.has[i]) continue;
            if constexpr (WIDE) {
#pragma unroll
                for (int j = 0; j < 8; ++j) to.put(part.at(i) + j, s[i][j]);
            } else {
                Io8<float>::store(to.at + part.at(i), s[i]);
            }
        }
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
                to.put(channel, sum);
            }
        }
    }
}

// A thread's channels of a sum, or of a weight, in places of its own in LDS.
template <int THREADS, int CH> struct OwnSum {
    floatx4 *at;  // [2 CH][THREADS]
    __device__ __forceinline__ OwnSum(float *lds, int which) : at(reinterpret_cast<floatx4 *>(lds) + which * (2 * CH * THREADS) + threadIdx.x)
    {
        clear();
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < 2 * CH; ++i) at[i * THREADS] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ void add(const float (&x)[CH][8])
    {
#pragma unroll
        for (int i = 0; i < 2 * CH; ++i) {
            floatx4 t = at[i * THREADS];
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] += x[i / 2][4 * (i & 1) + e];
            at[i * THREADS] = t;
        }
    }
    __device__ __forceinline__ void add(const float (&x)[CH][8], const float (&w)[CH][8])
    {
#pragma unroll
        for (int i = 0; i < 2 * CH; ++i) {
            floatx4 t = at[i * THREADS];
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] = fmaf(x[i / 2][4 * (i & 1) + e], w[i / 2][4 * (i & 1) + e], t[e]);
            at[i * THREADS] = t;
        }
    }
    __device__ __forceinline__ void set(const float (&x)[CH][8])
    {
#pragma unroll
        for (int i = 0; i < 2 * CH; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) at[i * THREADS][e] = x[i / 2][4 * (i & 1) + e];
    }
    __device__ __forceinline__ void get(float (&x)[CH][8]) const
    {
#pragma unroll
        for (int i = 0; i < 2 * CH; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[i / 2][4 * (i & 1) + e] = at[i * THREADS][e];
    }
};

// Rows over 4096 channels with a post-norm or gates: registers run out, and the sums of dy n and dy and the post weights and biases are in LDS, the sums over
// sequences in the workgroup's place of the workspace, which is for its threads alone.
template <int W, int CH, bool FULL> constexpr bool kWidest = FULL && W * CH >= 16;
// LDS of a gradient: GA, GB and GC, or those four.
template <int W, int CH, bool FULL> constexpr size_t kGradLds = !FULL ? 0 : (kWidest<W, CH, FULL> ? 4 : 3) * 8 * CH * threads_of(W) * sizeof(float);

// A thread's part of the rows of a gradient.
template <typename TX, typename T, int CH> struct GradRows {
    Raw<TX, CH> x, dr;
    Raw<T, CH> f, dy;
    template <typename Part> __device__ __forceinline__ void load(const ResidualArgs &a, int64_t row, int64_t end, const Part &part)
    {
        row = min(row, end - 1);  // (rows that there are not: the last)
        x.load(static_cast<const TX *>(a.x) + row * a.x_row, part);
        if (a.f != nullptr) f.load(static_cast<const T *>(a.f) + row * a.f_row, part);
        if (a.d_y != nullptr) dy.load(static_cast<const T *>(a.d_y) + row * a.width, part);
        if (a.d_r != nullptr) dr.load(static_cast<const TX *>(a.d_r) + row * a.width, part);
    }
};

// FULL: with a post-norm or gates.  What scale, gate and post weights multiply is the same for all rows of a sequence, so that their
// gradients are made of sums over these, A = sum dr' n' (n': f normed, or f), B = sum dr' and C = sum dr' u:
//   d gate = residual_scale scale C,  and with GA, GB and GC the sums of gate A, gate B and gate C over the sequences,
//   d scale = residual_scale GC,  d post_weight = residual_scale scale GA,  d post_bias = residual_scale scale GB.
// (C is post_weight A + post_bias B, but u may be far smaller than these parts, and then that loses what a sum of its own keeps.)
// WIDE: in shares (a.wide), of which each starts with sums of 0.
template <typename TX, typename T, int L, int W, int CH, bool FULL, bool WIDE> __global__ __launch_bounds__(threads_of(W)) void residual_grad_kernel(ResidualArgs a)
{
    using Part = RowPart<L, W, CH>;
    constexpr int kThreads = threads_of(W);
    constexpr bool kWide = kWidest<W, CH, FULL>;
    __shared__ float lds[2 * 2 * (kThreads / 64)];
    __shared__ float join[Part::kRows > 1 ? Part::kRows * 8 * L * W : 1];
    extern __shared__ __align__(16) float own_sums[];  // FULL: see kGradLds
    Part part(a.width, lds);
    const float of_width = 1.f / static_cast<float>(a.width);
    const int64_t r0 = static_cast<int64_t>(blockIdx.x) * a.rows_per_block, r1 = min(r0 + a.rows_per_block, a.n);
    const int64_t share = static_cast<int64_t>(gridDim.x) * a.width;
    float w[CH][8], factor[CH][8], pw[CH][8], pb[CH][8], dw[CH][8], db[CH][8], sa[CH][8], sb[CH][8], sc[CH][8];  // (not FULL: A is C)
    channel_weights<CH>(a.weight, a.w_bf16, part, 1.f, w);
    constexpr int kOwn = FULL && !kWide ? CH : 0, kAside = kWide ? CH : 0;
    OwnSum<kThreads, kOwn> ga(own_sums, 0), gb(own_sums, 1), gc(own_sums, 2);
    OwnSum<kThreads, kAside> own_dw(own_sums, 0), own_db(own_sums, 1), own_pw(own_sums, 2), own_pb(own_sums, 3);
    if constexpr (FULL) {
        channel_weights<CH>(a.post_weight, a.w_bf16, part, 1.f, pw);
        channel_weights<CH>(a.post_bias, a.w_bf16, part, 0.f, pb);
        if constexpr (kWide) {
            own_pw.set(pw);
            own_pb.set(pb);
        }
    }
    auto get_post = [&]() {
        if constexpr (kWide) {
            own_pw.get(pw);
            own_pb.get(pb);
        }
    };
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[i][j] = db[i][j] = sa[i][j] = sb[i][j] = sc[i][j] = 0.f;
    const bool gated = FULL && a.gate != nullptr, with_f = a.f != nullptr;
    const bool of_scale = a.part != nullptr && a.d_scale != nullptr, of_post_weight = a.part != nullptr && a.d_post_weight != nullptr,
               of_post_bias = a.part != nullptr && a.d_post_bias != nullptr;
    auto place = [&](int which, bool add) { return Place<WIDE>(a.part, which * share + blockIdx.x * static_cast<int64_t>(a.width), add); };
    auto clear = [&](float (&x)[CH][8]) {
#pragma unroll
        for (int i = 0; i < CH; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) x[i][j] = 0.f;
    };
    bool fresh = true;  // nothing in the places of the sums over sequences yet
    // In shares of `turns` rows of a thread (and sequences), as many as are added up in fp32; sequence by sequence (without gates: all rows at once).
    int seq = gated ? find_sequence(a.spans, r0) : 0;
    int64_t next = r0;  // of a sequence that a share ended in
    bool more = true;
    for (bool first_share = true; more; first_share = false) {
        more = false;
        int turns = a.turns;
        for (; seq < a.spans.batch; ++seq) {
            int first_row = 0, len = 0;
            if (gated) a.spans.of(seq, first_row, len);
            if (first_row >= r1) break;
            const int64_t begin = gated ? max(r0, static_cast<int64_t>(first_row)) : r0, end = gated ? min(r1, static_cast<int64_t>(first_row) + len) : r1;
            const int64_t from = WIDE ? max(begin, next) : begin, to = WIDE ? min(end, from + static_cast<int64_t>(turns) * Part::kRows) : end;
            if (from >= end) continue;
            if constexpr (WIDE) {
                more = turns <= 0;
                if (more) break;
                turns -= static_cast<int>((to - from + Part::kRows - 1) / Part::kRows);
            }
            GradRows<TX, T, CH> ahead;
            constexpr bool kAhead = W * CH < 16 || (!FULL && sizeof(TX) == 2);  // (the widest rows leave no registers for the next one)
            if (kAhead) ahead.load(a, from + part.sub, to, part);
            auto get_gate = [&](float (&gate)[CH][8]) {
                Raw<T, CH> raw;
                raw.load(static_cast<const T *>(a.gate) + seq * a.gate_row, part);
                raw.get(gate, part);
            };
            channel_weights<CH>(a.scale, a.w_bf16, part, 1.f, factor);
            {
                float gate[CH][8];
                if (gated) get_gate(gate);
#pragma unroll
                for (int i = 0; i < CH; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        factor[i][j] *= a.residual_scale;
                        if (gated) factor[i][j] *= gate[i][j];
                    }
            }
            for (int64_t first = from; first < to; first += Part::kRows) {
                const int64_t row = first + part.sub;
                const bool ok = Part::kRows == 1 || row < to;
                float z[CH][8], n[CH][8], g[CH][8], d[CH][8];
                GradRows<TX, T, CH> here;
                if (kAhead) here = ahead; else here.load(a, row, to, part);
                here.x.get(z, part);
                if (with_f) here.f.get(n, part);
                if (a.d_y != nullptr) here.dy.get(g, part);
                if (a.d_r != nullptr) here.dr.get(d, part);
                if (kAhead) ahead.load(a, row + Part::kRows, to, part);
                float post_inv = 0.f;
                if constexpr (FULL)
                    if (a.post != kNormNone) post_inv = row_norm<CH>(a.post, a.eps, of_width, part, n);
                if (a.d_r == nullptr)
#pragma unroll
                    for (int i = 0; i < CH; ++i)
#pragma unroll
                        for (int j = 0; j < 8; ++j) d[i][j] = 0.f;
                if (a.d_y != nullptr) {
                    if (with_f) {
                        get_post();
#pragma unroll
                        for (int i = 0; i < CH; ++i)
#pragma unroll
                            for (int j = 0; j < 8; ++j) z[i][j] = fmaf(factor[i][j], FULL ? fmaf(n[i][j], pw[i][j], pb[i][j]) : n[i][j], z[i][j]);
                    }
                    const float inv = row_norm<CH>(a.norm, a.eps, of_width, part, z);
                    if constexpr (kWide) {  // (one row at a time)
                        own_dw.add(g, z);
                        own_db.add(g);
                    }
#pragma unroll
                    for (int i = 0; i < CH; ++i)
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            if (!kWide && ok) {
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
                if (!with_f) continue;
                if constexpr (FULL) get_post();
#pragma unroll
                for (int i = 0; i < CH; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if (ok) {
                            if constexpr (FULL) {
                                sa[i][j] = fmaf(d[i][j], n[i][j], sa[i][j]);
                                sb[i][j] += d[i][j];
                            }
                            sc[i][j] = fmaf(d[i][j], FULL ? fmaf(n[i][j], pw[i][j], pb[i][j]) : n[i][j], sc[i][j]);
                        }
                        d[i][j] *= FULL ? factor[i][j] * pw[i][j] : factor[i][j];
                    }
                if constexpr (FULL)
                    if (a.post != kNormNone) row_norm_back<CH>(a.post, of_width, post_inv, n, part, d);
                store_row<T, CH>(static_cast<T *>(a.df) + row * a.width, d, part, ok);
            }
            if constexpr (FULL)
                if (gated) {
                    float gate[CH][8];
                    get_gate(gate);
                    if (a.part_gate != nullptr)  // at place blockIdx.x + seq, which no other pair has
                        store_sums<L, W, CH>(sc, Place<WIDE>(a.part_gate, (static_cast<int64_t>(blockIdx.x) + seq) * a.width, from > begin), a.width, part, join);
                    // times the gate to the sums over sequences
                    auto add = [&](float (&sums)[CH][8], int which, OwnSum<kThreads, kOwn> &own) {
                        if constexpr (kWide) {
                            const Place<WIDE> to = place(which, !fresh);
#pragma unroll
                            for (int i = 0; i < CH; ++i) {
                                if (!part.has[i]) continue;
#pragma unroll
                                for (int j = 0; j < 8; ++j) sums[i][j] *= gate[i][j];
                                if constexpr (!WIDE)
                                    if (!fresh) {
                                        Io8<float> x;
                                        x.load(to.at + part.at(i));
#pragma unroll
                                        for (int j = 0; j < 8; ++j) sums[i][j] += x.get(j);
                                    }
                            }
                            store_sums<L, W, CH>(sums, to, a.width, part, join);
                        } else {
                            own.add(sums, gate);
                        }
                    };
                    if (of_scale || !kWide) add(sc, kPartC, gc);
                    if (of_post_weight || !kWide) add(sa, kPartA, ga);
                    if (of_post_bias || !kWide) add(sb, kPartB, gb);
                    clear(sa);
                    clear(sb);
                    clear(sc);
                    fresh = false;
                }
            if constexpr (WIDE) {
                next = to < end ? to : r0;
                more = to < end;
                if (more) break;
            }
            if (!gated) break;
        }
        if (a.part == nullptr) {
            if constexpr (WIDE) continue;
            return;
        }
        if (a.d_weight != nullptr || a.d_bias != nullptr) {
            if constexpr (kWide) {
                own_dw.get(dw);
                own_db.get(db);
                if constexpr (WIDE) {
                    own_dw.clear();
                    own_db.clear();
                }
            }
            store_sums<L, W, CH>(dw, place(kPartWeight, !first_share), a.width, part, join);
            store_sums<L, W, CH>(db, place(kPartBias, !first_share), a.width, part, join);
            if constexpr (WIDE) {
                clear(dw);
                clear(db);
            }
        }
        if (kWide && gated && !fresh) {
            if constexpr (WIDE) continue;
            return;
        }
        if constexpr (kOwn > 0)
            if (gated) {
                ga.get(sa);
                gb.get(sb);
                gc.get(sc);
                if constexpr (WIDE) {
                    ga.clear();
                    gb.clear();
                    gc.clear();
                }
            }
        if (of_scale) store_sums<L, W, CH>(sc, place(kPartC, !first_share), a.width, part, join);
        if (of_post_weight) store_sums<L, W, CH>(sa, place(kPartA, !first_share), a.width, part, join);
        if (of_post_bias) store_sums<L, W, CH>(sb, place(kPartB, !first_share), a.width, part, join);
        if constexpr (!WIDE) return;
        clear(sa);
        clear(sb);
        clear(sc);
    }
}

__device__ __forceinline__ float weight_at(const void *w, bool is_bf16, int c, float none)
{
    if (w == nullptr) return none;
    return is_bf16 ? static_cast<float>(static_cast<const bf16_t *>(w)[c]) : static_cast<const float *>(w)[c];
}

// What is made of the workgroups' sums, 16 channels for a workgroup; blockIdx.y: d weight and d bias (of_norm), then d scale (of_scale), then d post
// weight and d post bias (of_post), then the gates, sequence by sequence.
template <typename P> __global__ __launch_bounds__(1024) void residual_sums_kernel(ResidualArgs a, int blocks, bool of_norm, bool of_scale, bool of_post, bool is_bf16)
{
    __shared__ union { PartSums<2> two; PartSums<1> one; } lds;
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), four = blockIdx.x * 16 + 4 * (threadIdx.x & 3);
    const int y = static_cast<int>(blockIdx.y), seq = y - (of_norm + of_scale + of_post);
    const bool ok = four < a.width, mine = threadIdx.x < 16 && c < a.width;
    const double scale = a.residual_scale * static_cast<double>(mine ? weight_at(a.scale, a.w_bf16, c, 1.f) : 0.f);
    const int64_t gap = static_cast<int64_t>(blocks) * a.width;
    const bool first = of_norm && y == 0;
    const P *part = static_cast<const P *>(a.part);
    double s[2];
    if (seq >= 0) {
        int row, len;
        a.spans.of(seq, row, len);
        const int64_t from = row / a.rows_per_block, count = len > 0 ? (static_cast<int64_t>(row) + len - 1) / a.rows_per_block - from + 1 : 0;
        sum_parts<1, 2>(static_cast<const P *>(a.part_gate) + (from + seq) * a.width + four, count, a.width, 0, ok, lds.one, reinterpret_cast<double(&)[1]>(s));
        if (mine) store_weight(a.d_gate, is_bf16, static_cast<int64_t>(seq) * a.width + c, static_cast<float>(scale * s[0]));
    } else if (of_scale && y == of_norm) {
        sum_parts<1, 2>(part + kPartC * gap + four, blocks, a.width, 0, ok, lds.one, reinterpret_cast<double(&)[1]>(s));
        if (mine) store_weight(a.d_scale, a.w_bf16, c, static_cast<float>(a.residual_scale * s[0]));
    } else {
        // (a sum that is not asked for may not be there: the other one in its place)
        const int at = first ? kPartWeight : (a.d_post_weight != nullptr ? kPartA : kPartB);
        sum_parts<2, 2>(part + at * gap + four, blocks, a.width, first || (a.d_post_weight != nullptr && a.d_post_bias != nullptr) ? gap : 0, ok, lds.two, s);
        void *const one = first ? a.d_weight : a.d_post_weight, *const two = first ? a.d_bias : a.d_post_bias;
        if (mine && one != nullptr) store_weight(one, a.w_bf16, c, static_cast<float>(first ? s[0] : scale * s[0]));
        if (mine && two != nullptr) store_weight(two, a.w_bf16, c, static_cast<float>(first ? s[1] : scale * s[1]));
    }
}

// The gates of sequences that few workgroups had rows of each: a thread for a channel.
template <typename P> __global__ __launch_bounds__(256) void residual_gate_kernel(ResidualArgs a, bool is_bf16)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int seq = static_cast<int>(i / a.width), c = static_cast<int>(i % a.width);
    if (seq >= a.spans.batch) return;
    int row, len;
    a.spans.of(seq, row, len);
    const int64_t from = row / a.rows_per_block, count = len > 0 ? (static_cast<int64_t>(row) + len - 1) / a.rows_per_block - from + 1 : 0;
    const P *part = static_cast<const P *>(a.part_gate) + (from + seq) * a.width + c;
    double s = 0.0;
    for (int64_t g = 0; g < count; ++g) s += part[g * a.width];
    store_weight(a.d_gate, is_bf16, i, static_cast<float>(s * a.residual_scale * weight_at(a.scale, a.w_bf16, c, 1.f)));
}

// Kernels for rows of up to 64, 128, 256 .. channels: lanes, waves and chunks of a row.
template <typename TX, typename T, bool FULL> struct Kernels {
    struct { void (*kernel)(ResidualArgs); int threads; size_t lds; } forward, grad;
    bool wide;
    template <int L, int W, int CH> void set_forward() { forward = {&residual_kernel<TX, T, L, W, CH, FULL>, threads_of(W), 0}; }
    template <int L, int W, int CH> void set_grad()
    {
        grad = {wide ? &residual_grad_kernel<TX, T, L, W, CH, FULL, true> : &residual_grad_kernel<TX, T, L, W, CH, FULL, false>, threads_of(W), kGradLds<W, CH, FULL>};
    }
    template <int L, int W, int CH> void set() { set_forward<L, W, CH>(); set_grad<L, W, CH>(); }
    Kernels(int width, bool wide_) : wide(wide_)
    {
        if (width <= 64) set<8, 1, 1>();
        else if (width <= 128) set<16, 1, 1>();
        else if (width <= 256) set<32, 1, 1>();
        else if (width <= 512) set<64, 1, 1>();
        else if constexpr (FULL) {
            if (width <= 1024) set<64, 2, 1>();
            else if (width <= 2048) set<64, 4, 1>();
            else if (width <= 4096) set<64, 8, 1>();
            else { set_forward<64, 16, 1>(); set_grad<64, 8, 2>(); }
        } else {
            if (width <= 1024) set<64, 1, 2>();
            else if (width <= 2048) set<64, 2, 2>();
            else if (width <= 4096) set<64, 4, 2>();
            else set<64, 8, 2>();
        }
    }
};

template <typename Launch> hipError_t by_type(const ResidualArgs &a, bool x_bf16, bool is_bf16, Launch &&launch)
{
    const bool full = a.post != kNormNone || a.gate != nullptr;
    if (!is_bf16) return full ? launch(Kernels<float, float, true>(a.width, a.wide)) : launch(Kernels<float, float, false>(a.width, a.wide));
    if (x_bf16) return full ? launch(Kernels<bf16_t, bf16_t, true>(a.width, a.wide)) : launch(Kernels<bf16_t, bf16_t, false>(a.width, a.wide));
    return full ? launch(Kernels<float, bf16_t, true>(a.width, a.wide)) : launch(Kernels<float, bf16_t, false>(a.width, a.wide));
}

}  // namespace

hipError_t launch_residual(const ResidualArgs &a, bool x_bf16, bool is_bf16, hipStream_t stream)
{
    const int64_t blocks = (a.n + a.rows_per_block - 1) / a.rows_per_block;
    return by_type(a, x_bf16, is_bf16, [&](auto kernels) {
        hipLaunchKernelGGL(kernels.forward.kernel, dim3(static_cast<unsigned>(blocks)), dim3(kernels.forward.threads), 0, stream, a);
        return hipGetLastError();
    });
}

hipError_t launch_residual_grad(const ResidualArgs &a, bool x_bf16, bool is_bf16, hipStream_t stream)
{
    const int64_t blocks = (a.n + a.rows_per_block - 1) / a.rows_per_block;
    if (blocks > 0) {
        const hipError_t e = by_type(a, x_bf16, is_bf16, [&](auto kernels) {
            const hipError_t allowed = allow_lds(kernels.grad.kernel, kernels.grad.lds);
            if (allowed != hipSuccess) return allowed;
            hipLaunchKernelGGL(kernels.grad.kernel, dim3(static_cast<unsigned>(blocks)), dim3(kernels.grad.threads), kernels.grad.lds, stream, a);
            return hipGetLastError();
        });
        if (e != hipSuccess) return e;
    }
    const bool of_norm = a.d_weight != nullptr || a.d_bias != nullptr, of_scale = a.d_scale != nullptr, of_post = a.d_post_weight != nullptr || a.d_post_bias != nullptr;
    // (more than eight workgroups for a sequence: a workgroup adds them up; 40 us where a thread does, for 6 sequences of 501 workgroups, 4 so)
    const bool spread = a.d_gate != nullptr && blocks > 8 * static_cast<int64_t>(a.spans.batch);
    const unsigned rows = of_norm + of_scale + of_post + (spread ? a.spans.batch : 0);
    if (rows > 0) {
        hipLaunchKernelGGL(a.wide ? &residual_sums_kernel<double> : &residual_sums_kernel<float>, dim3((a.width + 15) / 16, rows), dim3(1024), 0, stream, a, static_cast<int>(blocks), of_norm, of_scale, of_post, is_bf16);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.d_gate == nullptr || spread) return hipSuccess;
    const int64_t gates = (static_cast<int64_t>(a.spans.batch) * a.width + 255) / 256;
    hipLaunchKernelGGL(a.wide ? &residual_gate_kernel<double> : &residual_gate_kernel<float>, dim3(static_cast<unsigned>(gates)), dim3(256), 0, stream, a, is_bf16);
    return hipGetLastError();
}

}  // namespace s3r
