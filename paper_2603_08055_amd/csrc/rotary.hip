// Rotary positions of several axes for rows of q and k, with the norm of a head before them, and the gradient.
//   n = norm(x) over the head's 64 channels (or x),  m = n weight + bias,
//   a pair (a, b) of channels with the cosine c and sine s of its axis' position:  y_a = m_a c - m_b s,  y_b = m_b c + m_a s.
//   Gradient:  dm_a = dy_a c + dy_b s,  dm_b = dy_b c - dy_a s (the rotation by -s),  d weight = sum dm n,  d bias = sum dm,
//   dn = dm weight,  dx = (dn - [layer] mean(dn) - n mean(dn n)) / sigma, from x once more and not from stored statistics.
//
// Bound by HBM: a row of a head is read and written once.  Eight lanes have a head's 64 channels, a wave eight rows and a run of
// heads, so that a row's cosines and sines stay in registers for the heads in turn, and the sums over a head are three lane moves.
// 27480 rows of 16 + 16 heads in bf16, LayerNorm and two axes of 16 pairs, by rocprofv3 in turn, the inputs changing: 45 us, 5.0 TB/s of what is read and written (a
// copy of as much: 5.2 to 5.4; one call after the other on the same inputs 37 us by events, part of them from the caches); the gradient, which reads q and k again beside the
// gradients, 69 us, 4.9 TB/s, and 5 us for adding up those of the weights.  3001 rows of 15 + 5 heads in fp32, axes of 10, 11 and 11 pairs: 10.5 us (2.9 TB/s) and 15.3 + 3.9.
#include "s3r_lanes_device.h"

namespace s3r {

namespace {

// Where a channel's partner is: in the same lane (neighbours, axes of multiples of four pairs); at the same place of the lane whose number
// differs by 2 or 4 (all axes of 16 pairs, or one of 32, or, paired as halves of the whole, 32 pairs whatever their axes: the angles of a lane's channels then lie apart),
// or of another of the eight (axes of multiples of eight); or anywhere: then through LDS.
enum Mode { kInLane, kAcross2, kAcross4, kAcross4Apart, kAcross, kAnywhere };
constexpr bool angles_apart(Mode mode) { return mode == kAcross4Apart || mode == kAnywhere; }

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

// The value of the lane whose number differs by BIT (2 or 4), without a trip to LDS.
template <int BIT> __device__ __forceinline__ float other_lane(float x)
{
    if constexpr (BIT == 2) return lane_moved<0x4e>(x);
    return lane_moved<0x1b>(lane_moved<0x141>(x));  // the mirror of eight lanes, and that of four
}

// Cosines and sines of a lane's eight channels of a row, the sines with the sign that the channel's half of the pair takes times
// that of the rotation, and where its partners are.
template <typename T, Mode MODE> struct Turn {
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
    __device__ __forceinline__ void load(const RotaryArgs &a, int64_t row, int lane, float sign)
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
        if constexpr (angles_apart(MODE)) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const Channel ch = channel_of(a, 8 * c + j);
                // (channels that are not turned take another's angle, which goes unused)
                const int64_t i = (ch.axis == 0 ? where[0] : (ch.axis == 1 ? where[1] : where[2])) + ch.pair;
                co[j] = a.cos[ch.turned ? i : where[0]];
                si[j] = a.sin[ch.turned ? i : where[0]] * (ch.second ? sign : -sign);
            }
        } else {
            const int64_t i = turned ? (first.axis == 0 ? where[0] : (first.axis == 1 ? where[1] : where[2])) + first.pair : where[0];
            if constexpr (MODE == kInLane) {
                const floatx4 x = *reinterpret_cast<const floatx4 *>(a.cos + i), y = *reinterpret_cast<const floatx4 *>(a.sin + i);
#pragma unroll
                for (int j = 0; j < 8; ++j) { co[j] = x[j >> 1]; si[j] = y[j >> 1] * ((j & 1) != 0 ? sign : -sign); }
            } else {
                Io8<float> x, y;
                x.load(a.cos + i);
                y.load(a.sin + i);
#pragma unroll
                for (int j = 0; j < 8; ++j) { co[j] = x.get(j); si[j] = y.get(j) * (first.second ? sign : -sign); }
            }
        }
    }
    // x cos + (partner) sin, with the rounding of the second product made up for: a sum of products that cancel keeps its bits, in bf16 as well, where
    // equal products would else leave their rounding in place of 0 (27480 rows, 16 + 16 heads in bf16 with a norm, one call after the other, 36.2 us without, 36.9 so).
    // What is made up for is below 2^104; held to that, it leaves an infinity as it is.  lds: 512 floats of the wave's own.
    __device__ __forceinline__ void apply(const RotaryArgs &a, const float (&x)[8], float (&y)[8], float *lds, int lane) const
    {
        float other[8];
        if constexpr (MODE == kAnywhere) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int j = 0; j < 8; ++j) lds[64 * j + lane] = x[j];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (MODE == kInLane) other[j] = x[j ^ 1];
            if constexpr (MODE == kAcross2) other[j] = other_lane<2>(x[j]);
            if constexpr (MODE == kAcross4 || MODE == kAcross4Apart) other[j] = other_lane<4>(x[j]);
            if constexpr (MODE == kAcross)
                other[j] = __uint_as_float(static_cast<unsigned>(__builtin_amdgcn_ds_bpermute(from, static_cast<int>(__float_as_uint(x[j])))));
            if constexpr (MODE == kAnywhere) other[j] = lds[at[j] < 0 ? 0 : at[j]];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float p = other[j] * si[j];
            y[j] = fmaf(x[j], co[j], p);
            y[j] += __builtin_amdgcn_fmed3f(fmaf(other[j], si[j], -p), -0x1p104f, 0x1p104f);  // (the lower bound where it is NaN)
        }
        if (a.n_pairs < 32)
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = (MODE == kAnywhere ? at[j] >= 0 : turned) ? y[j] : x[j];
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
    s1 = a.norm == kNormLayer ? sum_over_lanes<8>(s1) * (1.f / 64) : 0.f;
    const float inv = inverse_root(fmaxf(fmaf(-s1, s1, s2), 0.f) + 0.f * s2 + a.eps);  // (a NaN stays one)
    s1 *= -inv;
#pragma unroll
    for (int j = 0; j < 8; ++j) n[j] = fmaf(n[j], inv, s1);
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

typedef double doublex2 __attribute__((ext_vector_type(2)));

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
    Turn<T, MODE> turn;
    const bool turns = a.cos != nullptr;
    turn.place(a, lane);
    if (turns) turn.load(a, row, lane, a.sign);
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
                turn.apply(a, x, y, lds, lane);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = x[j];
            }
            if (r.ok) Io8<T>::store(out + (h0 + i) * s.out_head, y);
        }
    }
}

// Gradient through a norm.  A workgroup stays with q or with k and adds up what its rows give to the gradients of weight and bias, a run of heads in
// fp32 and runs, of which a lane may have thousands, in 64 bits; another launch adds up the workgroups.  (Those totals are in LDS: 32 registers more
// cost a wave on a SIMD where a lane's angles lie apart, 27480 rows, forward and gradient 114 -> 121 us; from LDS 115.)
template <typename T, Mode MODE> __global__ __launch_bounds__(256) void rotary_norm_grad_kernel(RotaryArgs a, int run, int wgs_q)
{
    __shared__ float exchange[4 * 512];
    __shared__ doublex2 totals[8][256];  // of each thread's channels: dw, db
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    float *lds = exchange + wave * 512;
    const int side = static_cast<int>(blockIdx.x) >= wgs_q ? 1 : 0, first = side == 0 ? 0 : wgs_q, wgs = side == 0 ? wgs_q : static_cast<int>(gridDim.x) - wgs_q;
    const RotarySide s = side == 0 ? a.side[0] : a.side[1];
    const int64_t items = (a.n_rows + 7) / 8 * ((s.heads + run - 1) / run);
    const int c = lane & 7;
    Turn<T, MODE> turn;
    const bool turns = a.cos != nullptr;
    turn.place(a, lane);
    float w[8];
    load_weights(s.weight, a.w_bf16, 8 * c, true, 1.f, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) totals[j][threadIdx.x] = doublex2{0.0, 0.0};
    for (int64_t item = (static_cast<int64_t>(blockIdx.x) - first) * 4 + wave; item < items; item += 4 * wgs) {
        const HeadRun r = head_run(a, item, side, run, lane);
        const int64_t row = r.ok ? r.row : 0;
        if (turns) turn.load(a, row, lane, -1.f);
        const T *in = static_cast<const T *>(s.in) + row * s.in_row + 8 * c, *grad = static_cast<const T *>(s.grad) + row * s.heads * 64 + 8 * c;
        T *out = static_cast<T *>(s.out) + row * s.out_row + 8 * c;
        float dw[8] = {}, db[8] = {};
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
                    turn.apply(a, n, g, lds, lane);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) g[j] = n[j];
                }
                const float inv = head_norm(a, x, n);
                float s1 = 0.f, s2 = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    dw[j] = fmaf(g[j], n[j], dw[j]);
                    db[j] += g[j];
                    g[j] *= w[j];
                    s1 += g[j];
                    s2 = fmaf(g[j], n[j], s2);
                }
                s1 = a.norm == kNormLayer ? sum_over_lanes<8>(s1) * (-inv / 64) : 0.f;
                s2 = sum_over_lanes<8>(s2) * (-inv / 64);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = fmaf(n[j], s2, fmaf(g[j], inv, s1));
                if (r.ok) Io8<T>::store(out + (h0 + i) * s.out_head, x);
            }
        }
        if (r.ok)
#pragma unroll
            for (int j = 0; j < 8; ++j) totals[j][threadIdx.x] += doublex2{static_cast<double>(dw[j]), static_cast<double>(db[j])};
    }
    if (a.part == nullptr) return;
    // the wave's eight rows, then the workgroup's waves
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        double dw = totals[j][threadIdx.x][0], db = totals[j][threadIdx.x][1];
        for (int m = 8; m < 64; m <<= 1) {
            dw += __shfl_xor(dw, m, 64);
            db += __shfl_xor(db, m, 64);
        }
        if (lane < 8) {
            lds[8 * c + j] = static_cast<float>(dw);
            lds[64 + 8 * c + j] = static_cast<float>(db);
        }
    }
    __syncthreads();
    if (threadIdx.x < 128)
        a.part[static_cast<int64_t>(blockIdx.x) * 128 + threadIdx.x] =
            (exchange[threadIdx.x] + exchange[512 + threadIdx.x]) + (exchange[1024 + threadIdx.x] + exchange[1536 + threadIdx.x]);
}

// The gradients of weight and bias of q and of k as sums over the workgroups: 16 of the 64 channels of one of the four for a workgroup.
__global__ __launch_bounds__(1024) void rotary_weight_grad_kernel(RotaryArgs a, int wgs_q, int wgs)
{
    __shared__ PartSums<1> lds;
    const int side = blockIdx.x >> 3, which = (blockIdx.x >> 2) & 1, channels = (blockIdx.x & 3) * 16;
    const int first = side == 0 ? 0 : wgs_q, end = side == 0 ? wgs_q : wgs;
    void *to = which == 0 ? a.side[side].d_weight : a.side[side].d_bias;
    if (to == nullptr) return;
    double s[1];
    sum_parts<1, kRotaryGradGroups / 256>(a.part + static_cast<int64_t>(first) * 128 + which * 64 + channels + 4 * (threadIdx.x & 3), end - first, 128, 0, true, lds, s);
    if (threadIdx.x < 16) store_weight(to, a.w_bf16, channels + threadIdx.x, static_cast<float>(s[0]));
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
    if (a.pairing == kPairsWhole && a.n_pairs == 32 && common < 8) return kAcross4Apart;
    if (common < 8) return kAnywhere;
    const int half = a.pairing == kPairsWhole ? a.n_pairs : a.axis_pairs[0];  // channels from one of a pair to the other
    for (int x = 1; x < a.axes; ++x)
        if (a.pairing == kPairsHalves && a.axis_pairs[x] != half) return kAcross;
    return half == 16 ? kAcross2 : (half == 32 ? kAcross4 : kAcross);
}

// Heads that a wave takes in a row: as many as leave the card 2048 waves, up to 4, 8 through a norm's gradient (more to be read for the
// same angles), twice as many where a lane's angles lie apart, 16 where partners are looked up (whose places take longest to find).  us by events, one call after
// the other, 1 / 2 / 4 / 8 / 16 of them: 27480 rows of 16 + 16 heads, norm and rotation 67 / 41 / 36 / 37 / 38, with the gradient 209 / 139 / 118 / 114 / 114; axes of
// 10, 11 and 11 pairs 100 / 58 / 40 / 38 / 40, with the gradient 280 / 178 / 134 / 119 / 115, with partners looked up 370 / 229 / 168 / - / 133.
int run_of_heads(const RotaryArgs &a, Mode mode, bool grad)
{
    const int most = mode == kAnywhere || (mode == kAcross4Apart && grad) ? 16 : (mode == kAcross4Apart || grad ? 8 : 4);
    int run = 1;
    auto waves = [&](int r) { return (a.n_rows + 7) / 8 * ((a.side[0].heads + r - 1) / r + (a.side[1].heads + r - 1) / r); };
    while (run < most && waves(2 * run) >= 2048) run *= 2;
    return run;
}

int64_t items_of(const RotaryArgs &a, int side, int run) { return (a.n_rows + 7) / 8 * ((a.side[side].heads + run - 1) / run); }

template <typename T, Mode MODE> auto rotary_kernel_of(bool norm) { return norm ? &rotary_kernel<T, MODE, true> : &rotary_kernel<T, MODE, false>; }

template <typename T> hipError_t launch_rotary_t(const RotaryArgs &a, hipStream_t stream)
{
    const Mode mode = mode_of(a);
    const int run = run_of_heads(a, mode, false);
    const int64_t blocks = (items_of(a, 0, run) + items_of(a, 1, run) + 3) / 4;
    if (blocks <= 0 || blocks > 0xffffff) return hipErrorInvalidValue;
    const bool norm = a.norm != kNormNone;
    auto kernel = rotary_kernel_of<T, kAnywhere>(norm);
    switch (mode) {
    case kInLane: kernel = rotary_kernel_of<T, kInLane>(norm); break;
    case kAcross2: kernel = rotary_kernel_of<T, kAcross2>(norm); break;
    case kAcross4: kernel = rotary_kernel_of<T, kAcross4>(norm); break;
    case kAcross4Apart: kernel = rotary_kernel_of<T, kAcross4Apart>(norm); break;
    case kAcross: kernel = rotary_kernel_of<T, kAcross>(norm); break;
    case kAnywhere: break;
    }
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, a, run);
    return hipGetLastError();
}

template <typename T> hipError_t launch_norm_grad_t(const RotaryArgs &a, Mode mode, int run, int wgs_q, int wgs, hipStream_t stream)
{
    auto kernel = &rotary_norm_grad_kernel<T, kAnywhere>;
    switch (mode) {
    case kInLane: kernel = &rotary_norm_grad_kernel<T, kInLane>; break;
    case kAcross2: kernel = &rotary_norm_grad_kernel<T, kAcross2>; break;
    case kAcross4: kernel = &rotary_norm_grad_kernel<T, kAcross4>; break;
    case kAcross4Apart: kernel = &rotary_norm_grad_kernel<T, kAcross4Apart>; break;
    case kAcross: kernel = &rotary_norm_grad_kernel<T, kAcross>; break;
    case kAnywhere: break;
    }
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
    const Mode mode = mode_of(a);
    const int run = run_of_heads(a, mode, true);
    const int64_t of_q = items_of(a, 0, run), of_k = items_of(a, 1, run);
    // the same number of items for every wave, or one less, in as many workgroups as there is room for (27480 rows of 16 + 16 heads 114 us, in
    // 1024 122; axes of 10, 11 and 11 pairs 133, in 512 127)
    int64_t each = 1;
    const int most = mode == kAnywhere ? 512 : kRotaryGradGroups;
    while ((of_q + 4 * each - 1) / (4 * each) + (of_k + 4 * each - 1) / (4 * each) > most) ++each;
    const int wgs_q = static_cast<int>((of_q + 4 * each - 1) / (4 * each)), wgs = wgs_q + static_cast<int>((of_k + 4 * each - 1) / (4 * each));
    hipError_t e = hipSuccess;
    if (wgs > 0) e = is_bf16 ? launch_norm_grad_t<bf16_t>(a, mode, run, wgs_q, wgs, stream) : launch_norm_grad_t<float>(a, mode, run, wgs_q, wgs, stream);
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
