// Rotary positions of several axes for rows of q and k, with the norm of a head before them, and the gradient.
//   n = norm(x) over the head's 64 channels (or x),  m = n weight + bias,
//   a pair (a, b) of channels with the cosine c and sine s of its axis' position:  y_a = m_a c - m_b s,  y_b = m_b c + m_a s.
//   Gradient:  dm_a = dy_a c + dy_b s,  dm_b = dy_b c - dy_a s (the rotation by -s),  d weight = sum dm n,  d bias = sum dm,
//   dn = dm weight,  dx = (dn - [layer] mean(dn) - n mean(dn n)) / sigma, from x once more and not from stored statistics.
//
// Bound by HBM: a row of a head is read and written once.  Eight lanes have a head's 64 channels, a wave eight rows and a run of
// heads, so that a row's cosines and sines stay in registers for the heads in turn, and the sums over a head are three lane moves.
#include "s3r_lanes_device.h"

namespace s3r {

namespace {

// Where a channel's partner is: in the same lane (neighbours, axes of multiples of four pairs), at the same place of another of the
// eight lanes (axes of multiples of eight pairs), or anywhere: then through LDS.
enum Mode { kInLane, kAcross, kAnywhere };

struct Channel { int pair, partner, axis; bool turned, second; };
__device__ __forceinline__ Channel channel_of(const RotaryArgs &a, int c)
{
    Channel r;
    const int p0 = a.axis_pairs[0], p1 = a.axis_pairs[1], total = a.n_pairs;
    r.turned = c < 2 * total;
    if (a.pairing == kPairsNeighbours) {
        r.pair = c >> 1;
        r.partner = c ^ 1;
        r.second = (c & 1) != 0;
    } else if (a.pairing == kPairsWhole) {
        r.second = c >= total;
        r.pair = r.second ? c - total : c;
        r.partner = r.second ? c - total : c + total;
    } else {
        const int off = c >= 2 * (p0 + p1) ? p0 + p1 : (c >= 2 * p0 ? p0 : 0), p = c >= 2 * (p0 + p1) ? a.axis_pairs[2] : (c >= 2 * p0 ? p1 : p0);
        r.second = c - 2 * off >= p;
        r.pair = c - off - (r.second ? p : 0);
        r.partner = r.second ? c - p : c + p;
    }
    r.axis = (r.pair >= p0 ? 1 : 0) + (r.pair >= p0 + p1 ? 1 : 0);
    return r;
}

// Cosines and sines of a lane's eight channels of a row, the sines with the sign that the channel's half of the pair takes (times
// `sign`), and where its partners are.
template <Mode MODE> struct Turn {
    float co[8], si[8];
    int from;            // kAcross: lane of the partners, times 4
    int at[8];           // kAnywhere: of the partners in LDS; -1: not turned
    bool turned;

    __device__ __forceinline__ void place(const RotaryArgs &a, int lane)
    {
        const int c = lane & 7;
        if constexpr (MODE == kAnywhere) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const Channel ch = channel_of(a, 8 * c + j);
                at[j] = ch.turned ? (ch.partner & 7) * 64 + (lane & 56) + (ch.partner >> 3) : -1;
            }
        } else if constexpr (MODE == kAcross) {
            from = 4 * ((lane & 56) + (channel_of(a, 8 * c).partner >> 3));
        }
    }
    __device__ __forceinline__ void load(const RotaryArgs &a, int64_t row, int lane)
    {
        const int c = lane & 7;
        int64_t where[3];
#pragma unroll
        for (int x = 0; x < 3; ++x) {
            int64_t p = 0;
            if (x < a.axes) p = a.positions != nullptr ? a.positions[row * a.axes + x] : row;
            where[x] = (p < 0 ? 0 : (p >= a.places ? a.places - 1 : p)) * a.n_pairs;
        }
        const Channel first = channel_of(a, 8 * c);
        turned = first.turned;
        if constexpr (MODE == kAnywhere) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const Channel ch = channel_of(a, 8 * c + j);
                co[j] = 1.f;
                si[j] = 0.f;
                if (!ch.turned) continue;
                const int64_t i = (ch.axis == 0 ? where[0] : (ch.axis == 1 ? where[1] : where[2])) + ch.pair;
                co[j] = a.cos[i];
                si[j] = ch.second ? a.sin[i] : -a.sin[i];
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) { co[j] = 1.f; si[j] = 0.f; }
            if (!turned) return;
            const int64_t i = (first.axis == 0 ? where[0] : (first.axis == 1 ? where[1] : where[2])) + first.pair;
            if constexpr (MODE == kInLane) {
                const floatx4 x = *reinterpret_cast<const floatx4 *>(a.cos + i), y = *reinterpret_cast<const floatx4 *>(a.sin + i);
#pragma unroll
                for (int j = 0; j < 8; ++j) { co[j] = x[j >> 1]; si[j] = (j & 1) != 0 ? y[j >> 1] : -y[j >> 1]; }
            } else {
                Io8<float> x, y;
                x.load(a.cos + i);
                y.load(a.sin + i);
#pragma unroll
                for (int j = 0; j < 8; ++j) { co[j] = x.get(j); si[j] = first.second ? y.get(j) : -y.get(j); }
            }
        }
    }
    // x cos + (partner) sin, with the rounding of the second product made up for (a sum of products that cancel keeps its bits; where an
    // infinity makes that NaN, the sum as it is).  sign: 1, or -1 to turn back.  lds: 512 floats of the wave's own.
    __device__ __forceinline__ void apply(const float (&x)[8], float (&y)[8], float sign, float *lds, int lane) const
    {
        float other[8];
        if constexpr (MODE == kInLane) {
#pragma unroll
            for (int j = 0; j < 8; ++j) other[j] = x[j ^ 1];
        } else if constexpr (MODE == kAcross) {
#pragma unroll
            for (int j = 0; j < 8; ++j) other[j] = __uint_as_float(static_cast<unsigned>(__builtin_amdgcn_ds_bpermute(from, static_cast<int>(__float_as_uint(x[j])))));
        } else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int j = 0; j < 8; ++j) lds[64 * j + lane] = x[j];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int j = 0; j < 8; ++j) other[j] = lds[at[j] < 0 ? 0 : at[j]];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float s = sign * si[j], p = other[j] * s, rest = fmaf(other[j], s, -p), sum = fmaf(x[j], co[j], p), whole = sum + rest;
            const bool is_turned = MODE == kAnywhere ? at[j] >= 0 : turned;
            y[j] = !is_turned ? x[j] : (whole == whole ? whole : sum);
        }
    }
};

// A head's norm: n and 1 / sigma of its 64 channels, eight in each of eight lanes.  The mean is taken twice, of x and of what is left, so
// that a mean much larger than the spread costs no bits.
__device__ __forceinline__ float head_norm(const RotaryArgs &a, const float (&x)[8], float (&n)[8])
{
    float mean = 0.f;
    if (a.norm == kNormLayer) {
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) s += x[j];
        mean = sum_over_lanes<8>(s) * (1.f / 64);
    }
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        n[j] = x[j] - mean;
        s1 += n[j];
        s2 = fmaf(n[j], n[j], s2);
    }
    s2 = sum_over_lanes<8>(s2) * (1.f / 64);
    if (a.norm == kNormLayer) {
        s1 = sum_over_lanes<8>(s1) * (1.f / 64);
        s2 = fmaxf(fmaf(-s1, s1, s2), 0.f) + 0.f * s2;  // (a NaN stays one)
#pragma unroll
        for (int j = 0; j < 8; ++j) n[j] -= s1;
    }
    const float inv = inverse_root(s2 + a.eps);
#pragma unroll
    for (int j = 0; j < 8; ++j) n[j] *= inv;
    return inv;
}

// A wave's rows and heads: eight rows, heads h0 .. h1 - 1 of one side (q or k).
struct HeadRun { int side, h0, h1; int64_t row; bool ok; };
__device__ __forceinline__ HeadRun head_run(const RotaryArgs &a, int64_t item, int side, int run, int lane)
{
    HeadRun r;
    const int heads = a.side[side].heads, runs = (heads + run - 1) / run;
    const int64_t octet = item / runs;
    r.side = side;
    r.h0 = static_cast<int>(item - octet * runs) * run;
    r.h1 = min(r.h0 + run, heads);
    r.row = octet * 8 + (lane >> 3);
    r.ok = r.row < a.n_rows;
    return r;
}

template <typename T> constexpr int kAhead = sizeof(T) == 4 ? 2 : 4;  // heads whose rows are requested at once: 64 bytes of a lane

template <typename T, Mode MODE, bool NORM> __global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a, int run)
{
    __shared__ float exchange[MODE == kAnywhere ? 4 * 512 : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    float *lds = exchange + (MODE == kAnywhere ? wave * 512 : 0);
    const int64_t octets = (a.n_rows + 7) / 8;
    int64_t item = static_cast<int64_t>(blockIdx.x) * 4 + wave;
    const int64_t of_q = octets * ((a.side[0].heads + run - 1) / run);
    const int side = item >= of_q ? 1 : 0;
    if (side == 1) item -= of_q;
    if (item >= octets * ((a.side[side].heads + run - 1) / run)) return;
    const HeadRun r = head_run(a, item, side, run, lane);
    const RotarySide s = side == 0 ? a.side[0] : a.side[1];
    const int c = lane & 7;
    const int64_t row = r.ok ? r.row : 0;
    Turn<MODE> turn;
    const bool turns = a.cos != nullptr;
    turn.place(a, lane);
    if (turns) turn.load(a, row, lane);
    float w[8], b[8];
    if constexpr (NORM) {
        load_weights(s.weight, a.w_bf16, 8 * c, true, 1.f, w);
        load_weights(s.bias, a.w_bf16, 8 * c, true, 0.f, b);
    }
    const T *in = static_cast<const T *>(s.in) + row * s.in_row + 8 * c;
    T *out = static_cast<T *>(s.out) + row * s.out_row + 8 * c;
    for (int h0 = r.h0; h0 < r.h1; h0 += kAhead<T>) {
        Io8<T> raw[kAhead<T>];
#pragma unroll
        for (int i = 0; i < kAhead<T>; ++i)
            if (h0 + i < r.h1) raw[i].load(in + (h0 + i) * s.in_head);
#pragma unroll
        for (int i = 0; i < kAhead<T>; ++i) {
            if (h0 + i >= r.h1) break;
            float x[8], y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = raw[i].get(j);
            if constexpr (NORM) {
                head_norm(a, x, y);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = fmaf(y[j], w[j], b[j]);
            }
            if (turns) {
                turn.apply(x, y, a.sign, lds, lane);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = x[j];
            }
            if (r.ok) Io8<T>::store(out + (h0 + i) * s.out_head, y);
        }
    }
}

// Gradient through a norm.  A workgroup stays with q or with k and adds up what its rows give to the gradients of weight and bias;
// another launch adds up the workgroups.
template <typename T, Mode MODE> __global__ __launch_bounds__(256) void rotary_norm_grad_kernel(RotaryArgs a, int run, int wgs_q)
{
    __shared__ float exchange[4 * 512];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    float *lds = exchange + wave * 512;
    const int side = static_cast<int>(blockIdx.x) >= wgs_q ? 1 : 0, first = side == 0 ? 0 : wgs_q, wgs = side == 0 ? wgs_q : static_cast<int>(gridDim.x) - wgs_q;
    const RotarySide s = side == 0 ? a.side[0] : a.side[1];
    const int64_t items = (a.n_rows + 7) / 8 * ((s.heads + run - 1) / run);
    const int c = lane & 7;
    Turn<MODE> turn;
    const bool turns = a.cos != nullptr;
    turn.place(a, lane);
    float w[8], dw[8], db[8];
    load_weights(s.weight, a.w_bf16, 8 * c, true, 1.f, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[j] = db[j] = 0.f;
    for (int64_t item = (static_cast<int64_t>(blockIdx.x) - first) * 4 + wave; item < items; item += 4 * wgs) {
        const HeadRun r = head_run(a, item, side, run, lane);
        const int64_t row = r.ok ? r.row : 0;
        if (turns) turn.load(a, row, lane);
        const T *in = static_cast<const T *>(s.in) + row * s.in_row + 8 * c, *grad = static_cast<const T *>(s.grad) + row * s.heads * 64 + 8 * c;
        T *out = static_cast<T *>(s.out) + row * s.out_row + 8 * c;
        for (int h0 = r.h0; h0 < r.h1; h0 += kAhead<T>) {
            Io8<T> raw[kAhead<T>], raw_g[kAhead<T>];
#pragma unroll
            for (int i = 0; i < kAhead<T>; ++i)
                if (h0 + i < r.h1) {
                    raw[i].load(in + (h0 + i) * s.in_head);
                    raw_g[i].load(grad + (h0 + i) * 64);
                }
#pragma unroll
            for (int i = 0; i < kAhead<T>; ++i) {
                if (h0 + i >= r.h1) break;
                float x[8], n[8], g[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) { x[j] = raw[i].get(j); n[j] = raw_g[i].get(j); }
                if (turns) {
                    turn.apply(n, g, -1.f, lds, lane);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) g[j] = n[j];
                }
                const float inv = head_norm(a, x, n);
                float s1 = 0.f, s2 = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (r.ok) {
                        dw[j] = fmaf(g[j], n[j], dw[j]);
                        db[j] += g[j];
                    }
                    g[j] *= w[j];
                    s1 += g[j];
                    s2 = fmaf(g[j], n[j], s2);
                }
                s1 = a.norm == kNormLayer ? sum_over_lanes<8>(s1) * (1.f / 64) : 0.f;
                s2 = sum_over_lanes<8>(s2) * (1.f / 64);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = inv * (g[j] - s1 - n[j] * s2);
                if (r.ok) Io8<T>::store(out + (h0 + i) * s.out_head, x);
            }
        }
    }
    if (a.part == nullptr) return;
    // the wave's eight rows, then the workgroup's waves
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        for (int m = 8; m < 64; m <<= 1) {
            dw[j] += __shfl_xor(dw[j], m, 64);
            db[j] += __shfl_xor(db[j], m, 64);
        }
        if (lane < 8) {
            lds[8 * c + j] = dw[j];
            lds[64 + 8 * c + j] = db[j];
        }
    }
    __syncthreads();
    if (threadIdx.x < 128)
        a.part[static_cast<int64_t>(blockIdx.x) * 128 + threadIdx.x] =
            (exchange[threadIdx.x] + exchange[512 + threadIdx.x]) + (exchange[1024 + threadIdx.x] + exchange[1536 + threadIdx.x]);
}

// The gradients of weight and bias of q and of k as sums over the workgroups, in 64 bits: 16 of the 64 channels of one of the four for a
// workgroup, whose 64 groups take every 64th.
__global__ __launch_bounds__(1024) void rotary_weight_grad_kernel(RotaryArgs a, int wgs_q, int wgs)
{
    const int side = blockIdx.x >> 3, which = (blockIdx.x >> 2) & 1, c = threadIdx.x & 15, group = threadIdx.x >> 4, channel = (blockIdx.x & 3) * 16 + c;
    const int first = side == 0 ? 0 : wgs_q, end = side == 0 ? wgs_q : wgs;
    void *to = which == 0 ? a.side[side].d_weight : a.side[side].d_bias;
    if (to == nullptr) return;
    __shared__ double sums[64][16];
    constexpr int kMost = kRotaryGradGroups / 64;
    float x[kMost];
#pragma unroll
    for (int i = 0; i < kMost; ++i) x[i] = first + group + 64 * i < end ? a.part[static_cast<int64_t>(first + group + 64 * i) * 128 + which * 64 + channel] : 0.f;
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < kMost; ++i) s += x[i];
    sums[group][c] = s;
    __syncthreads();
    if (group != 0) return;
    s = 0.0;
#pragma unroll
    for (int i = 0; i < 64; ++i) s += sums[i][c];
    store_weight(to, a.w_bf16, channel, static_cast<float>(s));
}

// Whether a position is outside the table.  One workgroup.
__global__ __launch_bounds__(1024) void rotary_status_kernel(RotaryArgs a, int *status)
{
    bool bad = false;
    if (a.positions == nullptr)
        bad = a.n_rows > a.places;
    else
        for (int64_t i = threadIdx.x; i < a.n_rows * a.axes; i += 1024) bad |= a.positions[i] < 0 || a.positions[i] >= a.places;
    const int any = __syncthreads_or(bad);
    if (threadIdx.x == 0) *status = any ? kDiagPosition : 0;
}

Mode mode_of(const RotaryArgs &a)
{
    int common = 8;
    for (int x = 0; x < a.axes; ++x)
        while (a.axis_pairs[x] % common != 0) common /= 2;
    if (a.axes == 0) return kInLane;
    if (a.pairing == kPairsNeighbours) return common >= 4 ? kInLane : kAnywhere;
    return common == 8 ? kAcross : kAnywhere;
}

// Heads that a wave takes in a row: as many, up to 16, as leave the card 8192 waves (eight for each of 1024 SIMDs).
int run_of_heads(const RotaryArgs &a)
{
    int run = 1;
    while (run < 16 && (a.n_rows + 7) / 8 * ((a.side[0].heads + a.side[1].heads + 2 * run - 1) / (2 * run)) >= 8192) run *= 2;
    return run;
}

int64_t items_of(const RotaryArgs &a, int side, int run) { return (a.n_rows + 7) / 8 * ((a.side[side].heads + run - 1) / run); }

template <typename T> hipError_t launch_rotary_t(const RotaryArgs &a, hipStream_t stream)
{
    const int run = run_of_heads(a);
    const int64_t blocks = (items_of(a, 0, run) + items_of(a, 1, run) + 3) / 4;
    if (blocks <= 0 || blocks > 0xffffff) return hipErrorInvalidValue;
    const Mode mode = mode_of(a);
    const bool norm = a.norm != kNormNone;
    auto kernel = mode == kInLane ? (norm ? &rotary_kernel<T, kInLane, true> : &rotary_kernel<T, kInLane, false>)
                : mode == kAcross ? (norm ? &rotary_kernel<T, kAcross, true> : &rotary_kernel<T, kAcross, false>)
                                  : (norm ? &rotary_kernel<T, kAnywhere, true> : &rotary_kernel<T, kAnywhere, false>);
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, a, run);
    return hipGetLastError();
}

template <typename T> hipError_t launch_norm_grad_t(const RotaryArgs &a, int run, int wgs_q, int wgs, hipStream_t stream)
{
    const Mode mode = mode_of(a);
    auto kernel = mode == kInLane ? &rotary_norm_grad_kernel<T, kInLane>
                : mode == kAcross ? &rotary_norm_grad_kernel<T, kAcross> : &rotary_norm_grad_kernel<T, kAnywhere>;
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(wgs)), dim3(256), 0, stream, a, run, wgs_q);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs &a, bool is_bf16, hipStream_t stream)
{
    return is_bf16 ? launch_rotary_t<bf16_t>(a, stream) : launch_rotary_t<float>(a, stream);
}

hipError_t launch_rotary_norm_grad(const RotaryArgs &a, bool is_bf16, hipStream_t stream)
{
    const int run = run_of_heads(a);
    const int64_t of_q = items_of(a, 0, run), of_k = items_of(a, 1, run);
    // workgroups of q and of k by their share of the work, at least one for either that has any
    const int64_t most_q = (of_q + 3) / 4, most_k = (of_k + 3) / 4;
    int64_t q = of_q + of_k > 0 ? kRotaryGradGroups * of_q / (of_q + of_k) : 0, k = kRotaryGradGroups - q;
    if (of_q > 0 && q == 0) { q = 1; k -= 1; }
    if (of_k > 0 && k == 0) { k = 1; q -= 1; }
    const int wgs_q = static_cast<int>(q < most_q ? q : most_q), wgs = wgs_q + static_cast<int>(k < most_k ? k : most_k);
    hipError_t e = hipSuccess;
    if (wgs > 0) e = is_bf16 ? launch_norm_grad_t<bf16_t>(a, run, wgs_q, wgs, stream) : launch_norm_grad_t<float>(a, run, wgs_q, wgs, stream);
    if (e != hipSuccess || a.part == nullptr) return e;
    hipLaunchKernelGGL(rotary_weight_grad_kernel, dim3(16), dim3(1024), 0, stream, a, wgs_q, wgs);
    return hipGetLastError();
}

hipError_t launch_rotary_status(const RotaryArgs &a, int *status, hipStream_t stream)
{
    hipLaunchKernelGGL(rotary_status_kernel, dim3(1), dim3(1024), 0, stream, a, status);
    return hipGetLastError();
}

}  // namespace s3r
