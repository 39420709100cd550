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
// not rounded, so that they add up to the value exactly.  Of the nine products of two such operands the six largest are computed.  The
// three others are below 2^-22, 2^-22 and 2^-30 of the product of the magnitudes and have its sign, so that each product comes out too
// small by up to 2^-21 of it; by 0.32 * 2^-23 on average over random significands.
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

// The same value, of which the compiler knows nothing: what is computed from it stays where it is written and holds no registers
// through a loop that seldom comes by.
__device__ __forceinline__ int opaque(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}

// Where a lane's pieces of the two kinds of A operand lie in a unit.  Rows 16, 32 and 48 further the chunks are permuted alike, so that
// these few offsets serve a whole unit with constants added.
struct UnitLanes {
    int rows[4];   // channels 16 s + 8 (lane / 32) .. of row lane % 32
    int tr[2][2];  // four channels of row 4 (lane / 32) + (lane % 16) / 4, of channels 32 dt + 16 ((lane / 16) % 2) .. + 15; row 8 further
    __device__ __forceinline__ explicit UnitLanes(int lane)
    {
        const int i = lane & 15, row = 4 * (lane >> 5) + (i >> 2), in_chunk = 4 * (i & 1);
#pragma unroll
        for (int s = 0; s < 4; ++s) rows[s] = unit_chunk(lane & 31, 2 * s + (lane >> 5));
#pragma unroll
        for (int dt = 0; dt < 2; ++dt) {
            const int chunk = 4 * dt + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
            tr[dt][0] = unit_chunk(row, chunk) + in_chunk;
            tr[dt][1] = unit_chunk(row + 8, chunk) + in_chunk;
        }
    }
};

// A operand: rows 32 half .. + 31 of a unit, channels 16 s .. + 15.
__device__ __forceinline__ bf16x8 unit_rows(const bf16_t *unit, int half, int s, const UnitLanes &at)
{
    return *reinterpret_cast<const bf16x8 *>(unit + at.rows[s] + half * 2048);
}

// A operand of the transposed unit: channels 32 dt .. + 31, rows 32 half + 16 u + 8 (j / 4) + 4 (lane / 32) + j % 4, j = 0 .. 7.
// Sixteen lanes fetch four rows of sixteen channels and get one channel of the four rows each.
__device__ __forceinline__ bf16x8 unit_channels(const bf16_t *unit, int half, int u, int dt, const UnitLanes &at)
{
    typedef short shortx8 __attribute__((ext_vector_type(8)));
    const bf16_t *from = unit + (32 * half + 16 * u) * 64;
    const shortx4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4 *)(from + at.tr[dt][0]));
    const shortx4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4 *)(from + at.tr[dt][1]));
    const shortx8 ab = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8, ab);
}

// All A operands of half a unit, sent for together.
template <int PS> struct RowOperands {
    bf16x8 x[4][PS];
    __device__ __forceinline__ void read(const bf16_t *unit, int half, const UnitLanes &at)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int part = 0; part < PS; ++part) x[i][part] = unit_rows(unit + part * kPlane, half, i, at);
    }
};

template <int PS> struct ChannelOperands {
    bf16x8 x[2][2][PS];
    __device__ __forceinline__ void read(const bf16_t *unit, int half, const UnitLanes &at)
    {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int dt = 0; dt < 2; ++dt)
#pragma unroll
                for (int part = 0; part < PS; ++part) x[u][dt][part] = unit_channels(unit + part * kPlane, half, u, dt, at);
    }
};

// The part of x that its upper 16 bits hold (a NaN stays one).
__device__ __forceinline__ float upper_part(float x)
{
    return __uint_as_float((__float_as_uint(x) & 0xffff0000u) | (x != x ? 0x00400000u : 0u));
}

// x = p[0] + p[1] + p[2] (parts 3), p[0] = x rounded to bf16 (parts 1), or p[0] = x cut to bf16 and p[1] what is left, rounded (parts 2: off by
// 2^-16 of x at most).  Of two parts both have the sign of x, and neither is 0 unless x is (2^-24 of x goes to the second): their products
// with an infinity are that of x, where a part of 0 or of the other sign would make NaN of it.
template <int PARTS> __device__ __forceinline__ void split_parts(const float (&x)[8], bf16x8 (&p)[PARTS])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if constexpr (PARTS == 1) {
            p[0][j] = static_cast<bf16_t>(x[j]);
        } else if constexpr (PARTS == 2) {
            const float h = __uint_as_float(__float_as_uint(x[j]) & 0xffff0000u);  // (of a NaN: p[1] is one)
            p[0][j] = __builtin_bit_cast(bf16_t, static_cast<unsigned short>(__float_as_uint(x[j]) >> 16));
            p[1][j] = static_cast<bf16_t>(fmaf(x[j], 0x1p-24f, x[j] - h));
        } else {
            const float h = upper_part(x[j]), rest = __builtin_isfinite(x[j]) ? x[j] - h : 0.f;
            const float m = __uint_as_float(__float_as_uint(rest) & 0xffff0000u), l = rest - m;
            p[0][j] = __builtin_bit_cast(bf16_t, static_cast<unsigned short>(__float_as_uint(h) >> 16));
            p[1][j] = __builtin_bit_cast(bf16_t, static_cast<unsigned short>(__float_as_uint(m) >> 16));
            p[2][j] = __builtin_bit_cast(bf16_t, static_cast<unsigned short>(__float_as_uint(l) >> 16));
        }
    }
}

// The same for held rows.  A lower part of 0 would make NaN of an infinite key, whose score is -inf and counts for nothing: the
// smallest normal number with the sign of x stands in, for x of 2^-102 and more below every product's rounding.  (Rows of 2^-108 over keys
// of 2^108: out off by 1.2e-5, at 2^-100 by 2e-7 as ever.)
template <int PARTS> __device__ __forceinline__ void split_held(const float (&x)[8], bf16x8 (&p)[PARTS])
{
    split_parts<PARTS>(x, p);
#pragma unroll
    for (int i = 1; i < PARTS; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (static_cast<float>(p[i][j]) == 0.f && x[j] != 0.f) p[i][j] = static_cast<bf16_t>(copysignf(0x1p-126f, x[j]));
}

__device__ __forceinline__ floatx16 mfma(const bf16x8 &a, const bf16x8 &b, const floatx16 &acc)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0);
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
            if (i + j < 3) acc = mfma(a, b[j], acc);
    }
}

// A product over STEPS steps of the channels, begun anew: product(step, i, j) for the parts i of A (PA) and j of the held operand (PB), the
// smallest parts first, so that only the last STEPS additions are rounded at the size of the sum (fp32 gradients of short sequences,
// against 64 bits: part by part for each step 1.3e-6 and 1.1e-6 in dq and dv, so 7.7e-7 and 5.3e-7).
template <int PA, int PB, int STEPS, typename Product> __device__ __forceinline__ void each_part(Product &&product)
{
#pragma unroll
    for (int both = (PA + PB > 4 ? 2 : PA + PB - 2); both >= 0; --both)
#pragma unroll
        for (int i = 0; i < PA; ++i) {
            const int j = both - i;
            if (j < 0 || j >= PB) continue;
#pragma unroll
            for (int step = 0; step < STEPS; ++step) product(step, i, j);
        }
}

// ---- sequences and tiles -----------------------------------------------------------------------------

// A workgroup's sequence: its number, its rows, and its entry of another list (or 0).
struct Sequence { int seq, first, len, entry; };

// The sum over the lanes up to this one.  Shifts by 1, 2, 4 and 8 within sixteen lanes, then the last of each sixteen to the next, and of
// the lower half to the upper: vector instructions, no trips to LDS.
__device__ __forceinline__ int sum_up_to(int x)
{
    constexpr int kShift = 0x110, kLastOf16 = 0x142, kLastOf32 = 0x143;
    x += __builtin_amdgcn_update_dpp(0, x, kShift + 1, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, kShift + 2, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, kShift + 4, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, kShift + 8, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, kLastOf16, 0xa, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, kLastOf32, 0xc, 0xf, false);
    return x;
}

// Tile `t` of the sequences' tiles of `tile` items in turn, a sequence having len * per_row items: its sequence and number
// in it; false when there are fewer tiles.  All lanes of a wave call it.  What is needed of a sequence is read for 64 of them at once,
// and not when the number is known: one wait less before a short launch's first key.
__device__ __forceinline__ bool find_tile(const Spans &spans, const int32_t *list, int per_row, int tile, int64_t t, Sequence &q, int &in_seq)
{
    if (spans.batch == 1) {
        q.seq = 0;
        q.entry = list != nullptr ? list[0] : 0;
        spans.of(0, q.first, q.len);
        in_seq = static_cast<int>(t);
        return t * tile < static_cast<int64_t>(q.len) * per_row;
    }
    const int lane = threadIdx.x & 63;
    int64_t before = 0;
    for (int b0 = 0; b0 < spans.batch; b0 += 64) {
        int tiles = 0, first = 0, len = 0, entry = 0;
        if (b0 + lane < spans.batch) {
            if (list != nullptr) entry = list[b0 + lane];
            spans.of(b0 + lane, first, len);
            tiles = static_cast<int>((static_cast<int64_t>(len) * per_row + tile - 1) / tile);
        }
        const int upto = sum_up_to(tiles);
        const unsigned long long past = __ballot(before + upto > t);
        if (past != 0) {
            const int l = __ffsll(past) - 1;
            q.seq = b0 + l;
            q.first = __builtin_amdgcn_readlane(first, l);
            q.len = __builtin_amdgcn_readlane(len, l);
            q.entry = __builtin_amdgcn_readlane(entry, l);
            in_seq = static_cast<int>(t - before) - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(tiles, l));
            return true;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// Workgroup id -> item: neighbouring items (tiles of one head, which read the same keys) go to one XCD and its L2.
__device__ __forceinline__ int64_t xcd_neighbours(int64_t bid, int64_t n) { return (bid & 7) * ((n + 7) / 8) + (bid >> 3); }
inline int64_t xcd_padded(int64_t n) { return (n + 7) / 8 * 8; }

// A workgroup's share of the grid: a tile of the held rows, a head of keys, one of n_split pieces of the streamed units.
struct Share { Sequence of; int tile, kv_head, split; };

// Two orders of the workgroups.  together: neighbouring tiles, which read the same keys, on one XCD and its L2, the heads and pieces one
// after the other.  Else tile by tile, each with its heads and pieces side by side over the XCDs, the last tile first (causal rows:
// those that see most begin) or, `first_first`, the last one last: with sequences of several lengths, or causal rows, the later pieces
// are short or empty, and an XCD with several heads' later pieces would have less to do than its neighbours.  Tiles that `tiles` counts
// and the sequences do not have are found here as well.
__device__ __forceinline__ bool find_share(const Spans &spans, const int32_t *list, int per_row, int tile, int64_t tiles, int n_split, int kv_heads,
                                           bool together, bool first_first, Share &s)
{
    int64_t t;
    if (together) {
        const int64_t item = xcd_neighbours(blockIdx.x, tiles * n_split * kv_heads), rest = item / tiles;
        s.split = static_cast<int>(rest % n_split);
        s.kv_head = static_cast<int>(rest / n_split);
        t = item - rest * tiles;
    } else {
        const unsigned each = static_cast<unsigned>(n_split) * static_cast<unsigned>(kv_heads), u = blockIdx.x / each, rest = blockIdx.x - u * each;
        s.split = static_cast<int>(rest / static_cast<unsigned>(kv_heads));
        s.kv_head = static_cast<int>(rest) - s.split * kv_heads;
        t = first_first ? u : tiles - 1 - u;
    }
    return t >= 0 && t < tiles && s.kv_head < kv_heads && find_tile(spans, list, per_row, tile, t, s.of, s.tile);
}

// Units of a piece: the same for all pieces of a tile but the last ones, which may be shorter or empty; short sequences have fewer pieces.
__device__ __forceinline__ int piece_units(int units, int n_split, int least) { return max((units + n_split - 1) / n_split, least); }
__device__ __forceinline__ void piece(int units, int n_split, int least, int split, int &u0, int &u1)
{
    const int per = piece_units(units, n_split, least);
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

// Units of one tensor, brought in by THREADS threads.  Item r of a sequence is its row r, or (GROUPED) head r % per_row of its row
// r / per_row.  fetch() requests a unit's rows, put() writes them to LDS (`kParts` planes), with zeros in the place of rows that do not
// count (behind the end, or masked: what stands there may be no number).
template <typename T, int THREADS, bool GROUPED = false> struct RowUnits {
    static constexpr int kParts = sizeof(T) == 4 ? 3 : 1;
    static constexpr int kChunks = 512 / THREADS;
    const T *base;  // item 0
    int64_t row_stride, head_stride;
    int items, per_row;
    int64_t mine;   // of the thread's first chunk in a unit
    Io8<T> r[kChunks];

    __device__ __forceinline__ RowUnits(const T *base_, int items_, int64_t row_stride_, int64_t head_stride_, int per_row_, int t)
        : base(base_), row_stride(row_stride_), head_stride(head_stride_), items(items_), per_row(per_row_), mine((t >> 3) * row_stride_ + (t & 7) * 8)
    {
    }
    __device__ __forceinline__ void fetch(int unit, int t)
    {
        const T *from = base + unit * (kUnitRows * row_stride);
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int id = t + c * THREADS, at = unit * kUnitRows + (id >> 3);
            if (at >= items) continue;
            if constexpr (GROUPED) {
                const int row = static_cast<int>(static_cast<unsigned>(at) / static_cast<unsigned>(per_row));
                r[c].load(base + row * row_stride + (at - row * per_row) * head_stride + (id & 7) * 8);
            } else {
                r[c].load(from + c * (THREADS / 8 * row_stride) + mine);
            }
        }
    }
    __device__ __forceinline__ void put(bf16_t *lds, unsigned long long counts, int t) const
    {
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int id = t + c * THREADS, row = id >> 3;
            put8(lds + unit_chunk(row, id & 7), r[c], (counts >> row) & 1);
        }
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

// Which of a unit's 64 rows count, lane by lane: those before `items` that a mask (or null: all) does not leave out.
struct CountedRows {
    const uint8_t *mask;
    int items, mine;
    __device__ __forceinline__ void fetch(int unit, int lane)
    {
        const int r = unit * kUnitRows + lane;
        mine = r < items;
        if (mask != nullptr && mine) mine = mask[r];
    }
    __device__ __forceinline__ unsigned long long counts() const { return __ballot(mine != 0); }
};

// The same rows of a bf16 tensor brought to LDS without passing registers (256 threads): a wave requests two KiB of every unit, eight rows
// each, lane by lane from where the chunk that belongs at its place of the unit lies.  Rows behind the end are the last one's, and made
// zeros afterwards, as masked ones are (blank_rows): what stands there may be no number.
template <bool GROUPED> struct DirectUnits {
    const bf16_t *base;  // item 0
    int64_t row_stride, head_stride;
    int items, per_row;
    unsigned off[2];     // bytes from the unit's first row; not GROUPED, and rows near enough for 32 bits
    bool near;

    __device__ __forceinline__ DirectUnits(const bf16_t *base_, int items_, int64_t row_stride_, int64_t head_stride_, int per_row_, int wave, int lane)
        : base(base_), row_stride(row_stride_), head_stride(head_stride_), items(items_), per_row(per_row_)
    {
        near = row_stride < (int64_t(1) << 23);
#pragma unroll
        for (int i = 0; i < 2; ++i) off[i] = 2 * (row_in_unit(wave, i, lane) * static_cast<unsigned>(row_stride) + 8 * chunk(wave, i, lane));
    }
    static __device__ __forceinline__ int row_in_unit(int wave, int i, int lane) { return 8 * (2 * wave + i) + (lane >> 3); }
    static __device__ __forceinline__ int chunk(int wave, int i, int lane)
    {
        const int row = row_in_unit(wave, i, lane);
        return (unit_chunk(row, lane & 7) - row * 64) >> 3;
    }
    // `lds`: byte address of the unit's place; wave and unit are the same for all lanes
    __device__ __forceinline__ void request(int unit, unsigned lds, int wave, int lane) const
    {
        if (!GROUPED && near && (unit + 1) * kUnitRows <= items) {
            const bf16_t *from = base + unit * (kUnitRows * row_stride);
#pragma unroll
            for (int i = 0; i < 2; ++i) lds_dma_16_x1(from, off[i], lds + (2 * wave + i) * 1024);
            return;
        }
        lane = opaque(lane);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int at = min(unit * kUnitRows + row_in_unit(wave, i, lane), items - 1);
            const int row = GROUPED && per_row != 1 ? static_cast<int>(static_cast<unsigned>(at) / static_cast<unsigned>(per_row)) : at;
            lds_dma_16(base + row * row_stride + (at - row * (GROUPED ? per_row : 1)) * head_stride + 8 * chunk(wave, i, lane), lds + (2 * wave + i) * 1024);
        }
    }
};

__device__ __forceinline__ void blank_rows(bf16_t *unit, unsigned long long counts, int t)
{
    t = opaque(t);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const int id = t + c * 256;
        if (((counts >> (id >> 3)) & 1) == 0) *reinterpret_cast<bf16x8 *>(unit + id * 8) = bf16x8{};
    }
}

// Two tensors with the same rows, unit by unit, for 256 threads.  step(u) gives unit u's place in LDS, tensor a's planes and then b's, once
// all of it is there, and sends for unit u + 1.
//   bf16: straight to LDS, two stages, one barrier per unit (another where rows do not count);
//   fp32: through registers, where values are cut into parts; one stage, two barriers.
template <typename T, bool GROUPED = false> struct UnitPairs {
    static constexpr int kParts = 3, kStages = 1, kStage = 2 * kParts * kPlane;  // bf16 elements
    RowUnits<T, 256, GROUPED> a, b;
    bf16_t *lds;
    int end, t;
    __device__ __forceinline__ UnitPairs(const T *a_, const T *b_, int items, int64_t a_row, int64_t a_head, int64_t b_row, int64_t b_head, int per_row,
                                         bf16_t *lds_)
        : a(a_, items, a_row, a_head, per_row, threadIdx.x), b(b_, items, b_row, b_head, per_row, threadIdx.x), lds(lds_), end(0), t(threadIdx.x)
    {
    }
    template <typename More> __device__ __forceinline__ void begin(int u0, int u1, More &&more)
    {
        end = u1;
        if (u0 < u1) { a.fetch(u0, t); b.fetch(u0, t); more(u0); }
    }
    // counts(): which of the unit's rows count, from what more(u) fetched; put(): what else goes to LDS for the unit
    template <typename More, typename Counts, typename Put>
    __device__ __forceinline__ bf16_t *step(int u, bool first, More &&more, Counts &&counts, Put &&put)
    {
        if (!first) __syncthreads();
        const unsigned long long c = counts();
        a.put(lds, c, t);
        b.put(lds + kParts * kPlane, c, t);
        put(0);
        __syncthreads();
        if (u + 1 < end) { a.fetch(u + 1, t); b.fetch(u + 1, t); more(u + 1); }
        return lds;
    }
};

template <bool GROUPED> struct UnitPairs<bf16_t, GROUPED> {
    static constexpr int kParts = 1, kStages = 2, kStage = 2 * kPlane;
    DirectUnits<GROUPED> a, b;
    bf16_t *lds;
    int end, wave, lane, stage;
    __device__ __forceinline__ UnitPairs(const bf16_t *a_, const bf16_t *b_, int items, int64_t a_row, int64_t a_head, int64_t b_row, int64_t b_head,
                                         int per_row, bf16_t *lds_)
        : a(a_, items, a_row, a_head, per_row, threadIdx.x >> 6, threadIdx.x & 63),
          b(b_, items, b_row, b_head, per_row, threadIdx.x >> 6, threadIdx.x & 63), lds(lds_), end(0),
          wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), lane(threadIdx.x & 63), stage(0)
    {
    }
    __device__ __forceinline__ void send(int u, int to) const
    {
        const unsigned at = static_cast<unsigned>(reinterpret_cast<size_t>(lds)) + to * (kStage * 2);
        a.request(u, at, wave, lane);
        b.request(u, at + kPlane * 2, wave, lane);
    }
    template <typename More> __device__ __forceinline__ void begin(int u0, int u1, More &&more)
    {
        end = u1;
        if (u0 < u1) { more(u0); send(u0, 0); }
    }
    template <typename More, typename Counts, typename Put>
    __device__ __forceinline__ bf16_t *step(int u, bool first, More &&more, Counts &&counts, Put &&put)
    {
        wait_vmcnt<0>();
        const unsigned long long c = counts();
        bf16_t *here = lds + stage * kStage;
        put(stage);
        lds_barrier();
        if (c != ~0ull) {
            blank_rows(here, c, threadIdx.x);
            blank_rows(here + kPlane, c, threadIdx.x);
            lds_barrier();
        }
        stage ^= 1;
        if (u + 1 < end) { more(u + 1); send(u + 1, stage); }
        return here;
    }
};

// ---- softmax over units -----------------------------------------------------------------------------------

// Which of a half unit's 32 streamed rows, of those in a lane's 16 registers, do not count: bits 8 (r / 4) + r % 4.  Opaque to the
// compiler, which would else make the masks of all registers ahead, for units that need none as well.
__device__ __forceinline__ uint32_t left_out(unsigned long long seen, int half, int lane)
{
    return static_cast<uint32_t>(opaque(static_cast<int>(static_cast<uint32_t>(~seen >> (32 * half)) >> (4 * (lane >> 5)))));
}
__device__ __forceinline__ uint32_t left_out_mask(uint32_t bits, int r)  // all ones: left out
{
    return static_cast<uint32_t>(__builtin_amdgcn_sbfe(static_cast<int>(bits), 8 * (r >> 2) + (r & 3), 1));
}
__device__ __forceinline__ float replace(float x, float by, uint32_t mask)  // bit by bit: x may be NaN
{
    return __uint_as_float((__float_as_uint(x) & ~mask) | (__float_as_uint(by) & mask));
}

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
            split_held<PQ>(x, q[s]);
        }
        // they are waited for here: a wait in the loop would be one for the units on their way, too
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int i = 0; i < PQ; ++i) asm volatile("" : "+v"(q[s][i]));
    }
    // One unit of keys (PS planes) and values (PS planes); seen: the keys that count for the lane's row; factor: scale * log2(e).
    // `top` need not be the largest score so far: it is raised only where a row's exponentials of a unit add up to more than 255, that is
    // where one is above 2^8 times its like at `top`; the scores are then computed again.  That spares almost all units the search.
    // All LDS reads of a product are sent for before its first MFMA.
    // bf16: probabilities enter the product with v rounded to bf16, as in the library's dense attention.  Two parts would leave of the error of
    // out its own rounding alone (2.2e-3 -> 1.66e-3 against 64 bits, 2748 rows over 10992 keys) and take 24 matrix instructions for a unit in place of 16: us,
    // one part / two, 1374 rows over 27480 keys of 16 heads 203 / 297, 8192 over 8192 317 / 469, over cached tokens of 4 bits 402 / 517.
    template <int PS>
    __device__ __forceinline__ void unit(const bf16_t *k, const bf16_t *v, unsigned long long seen, float factor, const UnitLanes &at, int lane)
    {
        const bool all = __all(seen == ~0ull);
        floatx16 s[2];
        auto scores = [&]() {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                RowOperands<PS> a;
                a.read(k, half, at);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int r = 0; r < 16; ++r) s[half][r] = 0.f;
                each_part<PS, PQ, 4>([&](int step, int i, int j) { s[half] = mfma(a.x[step][i], q[step][j], s[half]); });
            }
            if (!all) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint32_t out = left_out(seen, half, lane);
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[half][r] = replace(s[half][r], -INFINITY, left_out_mask(out, r));
                }
            }
        };
        auto raise = [&]() {
            float most = s[0][0];
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int r = 0; r < 16; ++r) most = fmaxf(most, s[half][r]);
            most = max_with_other_half(most);
            const float next = fmaxf(top, most);
            const float w = next == -INFINITY ? 1.f : fast_exp2((top - next) * factor);
            top = next;
            sum *= w;
#pragma unroll
            for (int r = 0; r < 16; ++r) { o[0][r] *= w; o[1][r] *= w; }
        };
        float unit_sum;  // the unit's own sum first: a long row's chain of additions is a 32nd as long
        auto exponentials = [&]() {
            const float base = top == -INFINITY ? 0.f : top * factor;
            float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[half][r] = fast_exp2(fmaf(s[half][r], factor, -base));
                    part[r & 3] += s[half][r];
                }
            unit_sum = (part[0] + part[1]) + (part[2] + part[3]);
        };
        for (bool look = !__all(top > -INFINITY);; look = true) {
            scores();
            if (look) raise();
            exponentials();
            if (look || __all(unit_sum <= kMaxUnitSum)) break;
        }
        sum += unit_sum;
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                bf16x8 a[2][PS];
#pragma unroll
                for (int dt = 0; dt < 2; ++dt)
#pragma unroll
                    for (int part = 0; part < PS; ++part) a[dt][part] = unit_channels(v + part * kPlane, half, u, dt, at);
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = s[half][8 * u + j];
                bf16x8 p[PQ];
                split_parts<PQ>(x, p);
#pragma unroll
                for (int dt = 0; dt < 2; ++dt) multiply<PS>(o[dt], p, [&](int part) { return a[dt][part]; });
            }
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

// A piece without keys leaves its rows' log-sums only, by which it is known.
__device__ __forceinline__ void store_no_keys(const SoftOut &to, int split, int64_t row, int head, bool ok)
{
    if (ok) to.part_lse[split * to.rows * to.heads + row * to.heads + head] = -INFINITY;
}

// A row without a weight above 0 is 0, also where its product with v is not: 0 times an infinity or NaN.
template <typename T, int PQ>
__device__ __forceinline__ void store_soft(SoftRow<PQ> &soft, float factor, const SoftOut &to, int split, int64_t row,
                                           int head, bool ok, int lane)
{
    float total, l2;
    soft.totals(factor, total, l2);
    const float w = total == 0.f ? 0.f : 1.f / total;
    if (total == 0.f)
#pragma unroll
        for (int r = 0; r < 16; ++r) soft.o[0][r] = soft.o[1][r] = 0.f;
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

// ---- few rows -----------------------------------------------------------------------------------------------
// Up to 16 held rows, the same for all waves of a workgroup, each of which takes its own units (16x16x32 MFMAs; bound by the memory that
// keys and values come from).  Keys go from memory to the A operand as they are: lane (key l % 16, channels 16 (l / 16) .. + 15) of each
// 16-key tile; only values pass through LDS, to be transposed.  A lane has row l % 16 and, of every tile of 16 keys (or channels),
// 4 (l / 16) + r.
constexpr int kFewRows = 16;

// A operand of the transposed unit: channels 16 ct .. + 15; keys 32 ks + 4 (lane / 16) + j, then 16 further.
__device__ __forceinline__ bf16x8 few_channels(const bf16_t *unit, int ks, int ct, int lane)
{
    const int i = lane & 15, row = 32 * ks + 4 * (lane >> 4) + (i >> 2);
    const int chunk = 2 * ct + ((i & 3) >> 1), in_chunk = 4 * (i & 1);
    typedef short shortx8 __attribute__((ext_vector_type(8)));
    const shortx4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4 *)(unit + unit_chunk(row, chunk) + in_chunk));
    const shortx4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4 *)(unit + unit_chunk(row + 16, chunk) + in_chunk));
    const shortx8 ab = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8, ab);
}

__device__ __forceinline__ float max_over_groups(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return max_with_other_half(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}

__device__ __forceinline__ float sum_over_groups(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return sum_with_other_half(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

template <int PQ> struct FewRows {
    bf16x8 q[2][PQ];  // B operands: row l % 16, channels 16 (l / 16) + 8 s ..
    floatx4 o[4];     // channels 16 ct + 4 (l / 16) + r
    float top, sum;

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int ct = 0; ct < 4; ++ct) o[ct] = floatx4{0.f, 0.f, 0.f, 0.f};
        top = -INFINITY;
        sum = 0.f;
    }
    template <typename T> __device__ __forceinline__ void load(const T *row, bool ok, int lane)
    {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            float x[8] = {};
            if (ok) load8(row + 16 * (lane >> 4) + 8 * s, x);
            split_held<PQ>(x, q[s]);
        }
    }
    // key(t, s, parts): the A operand of key tile t, its PS parts; v: PS planes in LDS; PP: parts in which probabilities enter the product
    template <int PS, int PP, typename Key>
    __device__ __forceinline__ void unit(Key &&key, const bf16_t *v, unsigned long long seen, float factor, int lane)
    {
        floatx4 s[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            s[t] = floatx4{0.f, 0.f, 0.f, 0.f};
            bf16x8 k[2][PS];
#pragma unroll
            for (int i = 0; i < 2; ++i) key(t, i, k[i]);
            each_part<PS, PQ, 2>([&](int step, int a, int b) {
                s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[step][a], q[step][b], s[t], 0, 0, 0);
            });
        }
        if (!__all(seen == ~0ull)) {
            const unsigned long long mine = seen >> (4 * (lane >> 4));
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[t][r] = (mine >> (16 * t + r)) & 1 ? s[t][r] : -INFINITY;
        }
        float most = s[0][0];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) most = fmaxf(most, s[t][r]);
        most = max_over_groups(most);
        if (__any(most > top)) {
            const float next = fmaxf(top, most);
            const float w = next == -INFINITY ? 1.f : fast_exp2((top - next) * factor);
            top = next;
            sum *= w;
#pragma unroll
            for (int ct = 0; ct < 4; ++ct) o[ct] *= w;
        }
        const float base = top == -INFINITY ? 0.f : top * factor;
        float unit_sum = 0.f;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[j] = fast_exp2(fmaf(s[2 * ks + (j >> 2)][j & 3], factor, -base));
                unit_sum += x[j];
            }
            bf16x8 p[PP];
            split_parts<PP>(x, p);
#pragma unroll
            for (int ct = 0; ct < 4; ++ct)
#pragma unroll
                for (int a = 0; a < PS; ++a) {
                    const bf16x8 vt = few_channels(v + a * kPlane, ks, ct, lane);
#pragma unroll
                    for (int b = 0; b < PP; ++b)
                        if (a + b < 3) o[ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, p[b], o[ct], 0, 0, 0);
                }
        }
        sum += unit_sum;
    }
};

// The joint result of WAVES waves that had a share of the keys each, and its store: wave w < 4 takes channels 16 w .. + 15.
// lds: WAVES * kFewJoin floats.
constexpr int kFewJoin = 1024 + 32;
template <typename T, int WAVES, int PQ>
__device__ __forceinline__ void store_few(const FewRows<PQ> &few, float factor, const SoftOut &to, int split, int64_t row, int head, bool ok,
                                          float *lds, int wave, int lane)
{
    float *mine = lds + wave * kFewJoin;
#pragma unroll
    for (int ct = 0; ct < 4; ++ct)
#pragma unroll
        for (int r = 0; r < 4; ++r) mine[(ct * 4 + r) * 64 + lane] = few.o[ct][r];
    const float all = sum_over_groups(few.sum);
    if (lane < 16) { mine[1024 + lane] = few.top; mine[1040 + lane] = all; }
    __syncthreads();
    if (wave >= 4) return;
    const int q = lane & 15;
    float top = -INFINITY, sum = 0.f;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < WAVES; ++j) top = fmaxf(top, lds[j * kFewJoin + 1024 + q]);
#pragma unroll
    for (int j = 0; j < WAVES; ++j) {
        const float t = lds[j * kFewJoin + 1024 + q];
        const float w = t == top ? 1.f : (t == -INFINITY ? 0.f : fast_exp2((t - top) * factor));
        sum += lds[j * kFewJoin + 1040 + q] * w;
#pragma unroll
        for (int r = 0; r < 4; ++r) o[r] += lds[j * kFewJoin + (wave * 4 + r) * 64 + lane] * w;
    }
    if (!ok) return;
    const float inv = 1.f / sum, l2 = sum == 0.f ? -INFINITY : fmaf(top, factor, log2f(sum));
#pragma unroll
    for (int r = 0; r < 4; ++r) o[r] = sum == 0.f ? 0.f : o[r] * inv;  // (see store_soft)
    const int64_t at = row * to.heads + head, part = split * to.rows * to.heads + at;
    const int c = 16 * wave + 4 * (lane >> 4);
    if (to.part_o != nullptr) {
        *reinterpret_cast<floatx4 *>(to.part_o + part * 64 + c) = o;
        if (wave == 0 && lane < 16) to.part_lse[part] = l2;
    } else {
        T *dst = static_cast<T *>(to.out) + at * 64 + c;
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<floatx4 *>(dst) = o;
        } else {
            bf16x4 x;
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = static_cast<bf16_t>(o[r]);
            *reinterpret_cast<bf16x4 *>(dst) = x;
        }
        if (wave == 0 && lane < 16 && to.lse != nullptr) to.lse[head * to.rows + row] = l2 * kLn2;
    }
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
