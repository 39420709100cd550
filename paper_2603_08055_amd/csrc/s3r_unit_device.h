// Device-side parts shared by cross attention, its gradient and attention over a 4-bit cache (cross_attn.hip, cache.hip).
//
// All of them walk units of 64 rows ("streamed" rows: keys, or queries in the gradient of keys) past 32 rows per wave
// ("held" rows).  A unit of a tensor lies in LDS as bf16 [64 rows][64 channels]; the held rows are B operands in registers.
// With 32x32x16 MFMAs and A from LDS, a product of streamed by held rows leaves every lane one held row (column lane % 32)
// and 16 streamed rows of a half unit, 8 (r / 4) + 4 (lane / 32) + r % 4 for register r: softmax sums run inside a lane, and the
// registers are, eight at a time, the B operand of the next product, whose contraction is over the streamed rows.  That
// product's A operand is the transposed unit: gfx950 reads it from the same LDS rows with ds_read_b64_tr_b16.
//
// fp32 tensors are held in three bf16 parts, the upper 8, the middle 8 and the lower 8 bits of the significand, each cut and
// not rounded, so that they add up to the value exactly.  Of the nine products of two such operands the six
// largest are computed; the others are below 2^-23 of the product of the magnitudes.
#pragma once
#include "s3r_attn_device.h"

namespace s3r {

typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) shortx4 LdsShort4;

constexpr int kUnitRows = 64;
constexpr int kPlane = kUnitRows * 64;  // bf16 elements of a unit of one tensor (of one part of it): 8 KiB

// Element offset of 8-channel chunk c of row `row` in a unit.  The chunks of a row are permuted so that neither
// sixteen rows of one chunk (the A operand) nor four rows of four chunks (the transposed one) meet in an LDS bank.
__device__ __forceinline__ int unit_chunk(int row, int c)
{
    return row * 64 + ((c ^ (((row & 2) << 1) | ((row >> 2) & 3))) << 3);
}

// A operand: rows 32 half .. + 31 of a unit, channels 16 s .. + 15.
__device__ __forceinline__ bf16x8 unit_rows(const bf16_t *unit, int half, int s, int lane)
{
    return *reinterpret_cast<const bf16x8 *>(unit + unit_chunk(32 * half + (lane & 31), 2 * s + (lane >> 5)));
}

// A operand of the transposed unit: channels 32 dt .. + 31, rows 32 half + 16 u + 8 (j / 4) + 4 (lane / 32) + j % 4, j = 0 .. 7.
// Sixteen lanes fetch four rows of sixteen channels and get one channel of the four rows each.
__device__ __forceinline__ bf16x8 unit_channels(const bf16_t *unit, int half, int u, int dt, int lane)
{
    const int i = lane & 15, row = 32 * half + 16 * u + 4 * (lane >> 5) + (i >> 2);
    const int chunk = 4 * dt + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1), in_chunk = 4 * (i & 1);
    typedef short shortx8 __attribute__((ext_vector_type(8)));
    const shortx4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4 *)(unit + unit_chunk(row, chunk) + in_chunk));
    const shortx4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4 *)(unit + unit_chunk(row + 8, chunk) + in_chunk));
    const shortx8 ab = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8, ab);
}

// The part of x that its upper 16 bits hold (a NaN stays one).
__device__ __forceinline__ float upper_part(float x)
{
    return __uint_as_float((__float_as_uint(x) & 0xffff0000u) | (x != x ? 0x00400000u : 0u));
}

// x = p[0] + p[1] + p[2] (parts 3), or p[0] = x rounded to bf16 (parts 1).
template <int PARTS> __device__ __forceinline__ void split_parts(const float (&x)[8], bf16x8 (&p)[PARTS])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if constexpr (PARTS == 1) {
            p[0][j] = static_cast<bf16_t>(x[j]);
        } else {
            const float h = upper_part(x[j]), rest = __builtin_isfinite(x[j]) ? x[j] - h : 0.f;
            const float m = __uint_as_float(__float_as_uint(rest) & 0xffff0000u), l = rest - m;
            p[0][j] = __builtin_bit_cast(bf16_t, static_cast<unsigned short>(__float_as_uint(h) >> 16));
            p[1][j] = __builtin_bit_cast(bf16_t, static_cast<unsigned short>(__float_as_uint(m) >> 16));
            p[2][j] = __builtin_bit_cast(bf16_t, static_cast<unsigned short>(__float_as_uint(l) >> 16));
        }
    }
}

// acc += a b for an A operand that `fetch(part)` reads and a held operand of PB parts; A has PA.
template <int PA, int PB, typename Fetch>
__device__ __forceinline__ void multiply(floatx16 &acc, const bf16x8 (&b)[PB], Fetch &&fetch)
{
#pragma unroll
    for (int i = 0; i < PA; ++i) {
        const bf16x8 a = fetch(i);
#pragma unroll
        for (int j = 0; j < PB; ++j)
            if (i + j < 3) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b[j], acc, 0, 0, 0);
    }
}

// ---- sequences and tiles -----------------------------------------------------------------------------

// Tile `t` of the sequences' tiles of `tile` items in turn, a sequence having len * per_row items: its sequence and number
// in it; false when there are fewer tiles.  All lanes of a wave call it.
__device__ __forceinline__ bool find_tile(const Spans &spans, int per_row, int tile, int64_t t, int &b, int &in_seq)
{
    if (spans.batch == 1) {
        int first, len;
        spans.of(0, first, len);
        b = 0;
        in_seq = static_cast<int>(t);
        return t * tile < static_cast<int64_t>(len) * per_row;
    }
    const int lane = threadIdx.x & 63;
    int64_t before = 0;
    for (int b0 = 0; b0 < spans.batch; b0 += 64) {
        int tiles = 0;
        if (b0 + lane < spans.batch) {
            int first, len;
            spans.of(b0 + lane, first, len);
            tiles = static_cast<int>((static_cast<int64_t>(len) * per_row + tile - 1) / tile);
        }
        int upto = tiles;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int v = __shfl_up(upto, d, 64);
            if (lane >= d) upto += v;
        }
        const unsigned long long past = __ballot(before + upto > t);
        if (past != 0) {
            const int l = __ffsll(past) - 1;
            b = b0 + l;
            in_seq = static_cast<int>(t - before - (__shfl(upto, l, 64) - __shfl(tiles, l, 64)));
            b = __builtin_amdgcn_readfirstlane(b);
            in_seq = __builtin_amdgcn_readfirstlane(in_seq);
            return true;
        }
        before += __shfl(upto, 63, 64);
    }
    return false;
}

// Workgroup id -> item: neighbouring items (tiles of one head, which read the same keys) go to one XCD and its L2.
__device__ __forceinline__ int64_t xcd_neighbours(int64_t bid, int64_t n) { return (bid & 7) * ((n + 7) / 8) + (bid >> 3); }
inline int64_t xcd_padded(int64_t n) { return (n + 7) / 8 * 8; }

// A workgroup's share of the grid: a tile of the held rows, a head of keys, one of n_split pieces of the streamed units.
struct Share { int seq, tile, kv_head, split; };

__device__ __forceinline__ bool find_share(const Spans &spans, int per_row, int tile, int64_t tiles, int n_split, int kv_heads, Share &s)
{
    const int64_t item = xcd_neighbours(blockIdx.x, tiles * n_split * kv_heads);
    const int64_t rest = item / tiles;
    s.split = static_cast<int>(rest % n_split);
    s.kv_head = static_cast<int>(rest / n_split);
    return s.kv_head < kv_heads && find_tile(spans, per_row, tile, item - rest * tiles, s.seq, s.tile);
}

__device__ __forceinline__ void piece(int units, int n_split, int split, int &u0, int &u1)
{
    const int per = (units + n_split - 1) / n_split;
    u0 = min(split * per, units);
    u1 = min(u0 + per, units);
}

// ---- streamed rows -------------------------------------------------------------------------------------

// Eight channels as they come from memory.
template <typename T> __device__ __forceinline__ void load8(const T *p, float (&x)[8])
{
    Io8<T> v;
    v.load(p);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = v.get(j);
}

// Units of two tensors with the same rows (keys and values, or queries and output gradients), brought in by THREADS threads: item r of
// a sequence is head r % per_row of its row r / per_row.  fetch() requests a unit's rows, put() writes them to LDS, with zeros in the
// place of rows that do not count (behind the end, or masked: what stands there may be no number), and gives the 64 bits of those that do.
template <typename T, int THREADS> struct RowUnits {
    static constexpr int kParts = sizeof(T) == 4 ? 3 : 1;
    static constexpr int kChunks = 512 / THREADS;
    const T *a, *b;                  // of item 0
    int64_t a_row, a_head, b_row, b_head;
    const uint8_t *mask;             // of row 0, or null
    int items, per_row;
    Io8<T> ra[kChunks], rb[kChunks];
    int seen;                        // of the lane's row of the unit

    __device__ __forceinline__ void fetch(int unit, int t)
    {
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int id = t + c * THREADS, r = unit * kUnitRows + (id >> 3);
            if (r < items) {
                const int row = per_row == 1 ? r : static_cast<int>(static_cast<unsigned>(r) / static_cast<unsigned>(per_row));
                const int head = r - row * per_row;
                ra[c].load(a + row * a_row + head * a_head + (id & 7) * 8);
                rb[c].load(b + row * b_row + head * b_head + (id & 7) * 8);
            }
        }
        const int r = unit * kUnitRows + (t & 63);
        seen = r < items;
        if (mask != nullptr && seen) seen = mask[r];
    }
    // lds: kParts planes of a, then kParts planes of b
    __device__ __forceinline__ unsigned long long put(bf16_t *lds, int t)
    {
        const unsigned long long valid = __ballot(seen != 0);
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int id = t + c * THREADS, row = id >> 3;
            const bool ok = (valid >> row) & 1;
            const int at = unit_chunk(row, id & 7);
            put8(lds + at, ra[c], ok);
            put8(lds + kParts * kPlane + at, rb[c], ok);
        }
        return valid;
    }
    static __device__ __forceinline__ void put8(bf16_t *to, const Io8<T> &r, bool ok)
    {
        if constexpr (kParts == 1) {
            bf16x8 x = {};
            if (ok) x = r.x;
            *reinterpret_cast<bf16x8 *>(to) = x;
        } else {
            float x[8];
            bf16x8 p[kParts];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = ok ? r.get(j) : 0.f;
            split_parts<kParts>(x, p);
#pragma unroll
            for (int i = 0; i < kParts; ++i) *reinterpret_cast<bf16x8 *>(to + i * kPlane) = p[i];
        }
    }
};

// ---- softmax over units -----------------------------------------------------------------------------------

// Which of a half unit's 32 streamed rows a lane's 16 registers have, as bits 8 (r / 4) + r % 4.
__device__ __forceinline__ uint32_t lane_bits(unsigned long long seen, int half, int lane)
{
    return static_cast<uint32_t>(seen >> (32 * half)) >> (4 * (lane >> 5));
}
__device__ __forceinline__ bool lane_bit(uint32_t bits, int r) { return (bits >> (8 * (r >> 2) + (r & 3))) & 1; }

// The lowest `n` of 64 bits.
__device__ __forceinline__ unsigned long long low_bits(int n)
{
    return n >= 64 ? ~0ull : (n <= 0 ? 0ull : (1ull << n) - 1);
}

// A held row's part of a softmax over keys: the product with v so far (transposed: channels 32 dt + acc_row(lane, r) of the lane's row),
// the largest score and the sum of exponentials of this lane's keys (the other half-wave has the others).
template <int PQ> struct SoftRow {
    bf16x8 q[4][PQ];
    floatx16 o[2];
    float top, sum;

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int r = 0; r < 16; ++r) o[0][r] = o[1][r] = 0.f;
        top = -INFINITY;
        sum = 0.f;
    }
    template <typename T> __device__ __forceinline__ void load(const T *row, bool ok, int lane)
    {
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            float x[8] = {};
            if (ok) load8(row + 16 * s + 8 * (lane >> 5), x);
            split_parts<PQ>(x, q[s]);
            // A lower part of 0 would make NaN of an infinite key, whose score is -inf and counts for nothing: the smallest
            // normal number with the sign of x stands in, below every product's rounding.
            if constexpr (PQ == 3) {
#pragma unroll
                for (int i = 1; i < 3; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        if (static_cast<float>(q[s][i][j]) == 0.f && x[j] != 0.f) q[s][i][j] = static_cast<bf16_t>(copysignf(0x1p-126f, x[j]));
            }
        }
    }
    // One unit of keys (PS planes) and values (PS planes); seen: the keys that count for the lane's row; factor: scale * log2(e).
    template <int PS>
    __device__ __forceinline__ void unit(const bf16_t *k, const bf16_t *v, unsigned long long seen, float factor, int lane)
    {
        floatx16 s[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[half][r] = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                multiply<PS>(s[half], q[i], [&](int part) { return unit_rows(k + part * kPlane, half, i, lane); });
        }
        if (!__all(seen == ~0ull)) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const uint32_t bits = lane_bits(seen, half, lane);
#pragma unroll
                for (int r = 0; r < 16; ++r) s[half][r] = lane_bit(bits, r) ? s[half][r] : -INFINITY;
            }
        }
        float most = s[0][0];
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, s[half][r]);
        most = max_with_other_half(most);
        if (__any(most > top)) {
            const float next = fmaxf(top, most);
            const float w = next == -INFINITY ? 1.f : fast_exp2((top - next) * factor);
            top = next;
            sum *= w;
#pragma unroll
            for (int r = 0; r < 16; ++r) { o[0][r] *= w; o[1][r] *= w; }
        }
        const float base = top == -INFINITY ? 0.f : top * factor;
        float unit_sum = 0.f;  // the unit's own sum first: a long row's chain of additions is a 32nd as long
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    x[j] = fast_exp2(fmaf(s[half][8 * u + j], factor, -base));
                    unit_sum += x[j];
                }
                bf16x8 p[PQ];
                split_parts<PQ>(x, p);
#pragma unroll
                for (int dt = 0; dt < 2; ++dt)
                    multiply<PS>(o[dt], p, [&](int part) { return unit_channels(v + part * kPlane, half, u, dt, lane); });
            }
        sum += unit_sum;
    }
    // The sum of exponentials over both half-waves, and its log2 (-inf: no keys).
    __device__ __forceinline__ void totals(float factor, float &total, float &log2_total) const
    {
        total = sum_with_other_half(sum);
        log2_total = total == 0.f ? -INFINITY : fmaf(top, factor, log2f(total));
    }
};

// A lane's 32 channels of its row (transposed accumulators) times w, as T, at `to` = the row's first channel.
template <typename T> __device__ __forceinline__ void store_row(const floatx16 (&o)[2], float w, T *to, bool ok, int lane)
{
#pragma unroll
    for (int dt = 0; dt < 2; ++dt)
#pragma unroll
        for (int b = 0; b < 4; b += 2) {
            float x[4], y[4], z[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[e] = o[dt][4 * b + e] * w; y[e] = o[dt][4 * b + 4 + e] * w; }
            join_runs_32(x, y, z);
            if (ok) Io8<T>::store(to + 32 * dt + 8 * (b + (lane >> 5)), z);
        }
}

template <typename T, int PQ>
__device__ __forceinline__ void store_soft(const SoftRow<PQ> &soft, float factor, const SoftOut &to, int split, int64_t row,
                                           int head, bool ok, int lane)
{
    float total, l2;
    soft.totals(factor, total, l2);
    const float w = total == 0.f ? 0.f : 1.f / total;
    const int64_t at = row * to.heads + head;
    if (to.part_o != nullptr) {
        const int64_t part = split * to.rows * to.heads + at;
        store_row(soft.o, w, to.part_o + part * 64, ok, lane);
        if (ok && lane < 32) to.part_lse[part] = l2;
    } else {
        store_row(soft.o, w, static_cast<T *>(to.out) + at * 64, ok, lane);
        if (ok && lane < 32 && to.lse != nullptr) to.lse[head * to.rows + row] = l2 * kLn2;
    }
}

// The joint result of WAVES waves that had a share of the keys each, for the same 32 rows.  lds: WAVES * kJoinFloats floats.
constexpr int kJoinFloats = 2048 + 64;
template <int WAVES, int PQ> __device__ __forceinline__ void join_waves(SoftRow<PQ> &soft, float factor, float *lds, int wave, int lane)
{
    float *mine = lds + wave * kJoinFloats;
#pragma unroll
    for (int dt = 0; dt < 2; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) mine[(dt * 16 + r) * 64 + lane] = soft.o[dt][r];
    const float both = sum_with_other_half(soft.sum);
    if (lane < 32) { mine[2048 + lane] = soft.top; mine[2080 + lane] = both; }
    __syncthreads();
    if (wave != 0) return;
    float top = -INFINITY, sum = 0.f, w[WAVES];
#pragma unroll
    for (int j = 0; j < WAVES; ++j) top = fmaxf(top, lds[j * kJoinFloats + 2048 + (lane & 31)]);
#pragma unroll
    for (int j = 0; j < WAVES; ++j) {
        const float t = lds[j * kJoinFloats + 2048 + (lane & 31)];
        w[j] = t == top ? 1.f : (t == -INFINITY ? 0.f : fast_exp2((t - top) * factor));
        sum += lds[j * kJoinFloats + 2080 + (lane & 31)] * w[j];
    }
#pragma unroll
    for (int dt = 0; dt < 2; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            float x = 0.f;
#pragma unroll
            for (int j = 0; j < WAVES; ++j) x += lds[j * kJoinFloats + (dt * 16 + r) * 64 + lane] * w[j];
            soft.o[dt][r] = x;
        }
    soft.top = top;
    soft.sum = lane < 32 ? sum : 0.f;
}

// A thread of 1024's finding whether a list of spans is out of range or out of order.
__device__ __forceinline__ bool spans_bad(const Spans &s)
{
    bool bad = false;
    if (s.start != nullptr)
        for (int b = threadIdx.x; b <= s.batch; b += 1024) {
            const int64_t x = s.start[b];
            bad |= x < 0 || x > s.n || (b < s.batch && s.start[b + 1] < x);
        }
    return bad;
}

// A launch's threads must stay below 2^32.
inline bool grid_ok(int64_t blocks_of_256) { return blocks_of_256 > 0 && blocks_of_256 <= 0xffffff; }

// More than 64 KiB of LDS have to be allowed to a kernel first.
template <typename Kernel> hipError_t allow_lds(Kernel kernel, size_t bytes)
{
    if (bytes <= size_t(64) << 10) return hipSuccess;
    return hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
}

}  // namespace s3r
