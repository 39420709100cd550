// A cache of keys and values in 4 bits: appending to its pages with the position rotation on the way, reading rows back, and
// attention over it.
//
// The form is that of the OCP microscaling formats, which gfx950 converts in hardware: 32 channels share a power of two 2^e and
// are e2m1 numbers (+-0, 0.5, 1, 1.5, 2, 3, 4, 6) in its units.  e is the smallest with max |x| < 7 * 2^e, so that the largest
// channel, too, is off by half a step at most (where e is cut to the largest exponent below max |x|, up to a quarter of it is lost).
// A block with a NaN or an infinity gets the exponent byte 255 and reads as NaN.
#include "s3r_unit_device.h"

namespace s3r {

namespace {

// x with its last bit set if it is not y exactly (round to odd): rounding it once more to fewer bits, or comparing it with a number of
// fewer bits, gives what y itself would.
__device__ __forceinline__ float round_to_odd(double y)
{
    const float x = static_cast<float>(y);
    const double off = y - static_cast<double>(x);
    unsigned bits = __float_as_uint(x);
    if (off != 0.0 && (bits & 1) == 0 && __builtin_isfinite(y)) bits += (off > 0.0) == (y > 0.0) ? 1 : -1;
    return __uint_as_float(bits);
}

// The value of the lane whose number differs by BIT (1, 2 or 4), without a trip to LDS: within four lanes as a permutation of them; four
// further as the mirror of eight lanes and that of four.  All lanes of the wave take part.
template <int BIT> __device__ __forceinline__ unsigned other_lane(unsigned x)
{
    constexpr int kSwap1 = 0xb1, kSwap2 = 0x4e, kMirror4 = 0x1b, kMirror8 = 0x141;
    int y = static_cast<int>(x);
    if constexpr (BIT == 4) y = __builtin_amdgcn_mov_dpp(y, kMirror8, 0xf, 0xf, true);
    return static_cast<unsigned>(__builtin_amdgcn_mov_dpp(y, BIT == 1 ? kSwap1 : (BIT == 2 ? kSwap2 : kMirror4), 0xf, 0xf, true));
}

// ---- append and read ----------------------------------------------------------------------------------
// Bound by HBM: 256 bytes of bf16 for 68 in the cache, of every token and head.  A wave takes eight rows, eight lanes each with eight
// channels, and a run of heads: what a row needs (its sequence, its place, the angles) is found once for them, and the 32 bytes of
// codes of neighbouring tokens, which lie side by side in a page, are written together.  The products of the rotation are exact in 64
// bits and their sum is rounded once, so that the codes are those of the exact values.
// 100 views of 1374 tokens, 16 heads: append 166 us, without rotation 135, read 138; a plain copy of as many bytes 140 (each on end; append and
// read in turn 180 and 124).  The rotation is
// what memory does not hide: 101 registers, four waves on a SIMD; held to 96 they spill (200 us).

// The rows of a wave and its heads: `octets` of rows, and for each heads h0 .. h1 - 1 of `heads`, `run` at a time.
struct HeadRun { int64_t row; int h0, h1; };
__device__ __forceinline__ bool head_run(int64_t rows, int heads, int run, HeadRun &r)
{
    const unsigned wave = blockIdx.x * 4u + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), runs = (heads + run - 1) / run, octet = wave / runs;
    r.row = static_cast<int64_t>(octet) * 8 + ((threadIdx.x & 63) >> 3);
    r.h0 = static_cast<int>(wave - octet * runs) * run;
    r.h1 = min(r.h0 + run, heads);
    return static_cast<int64_t>(octet) * 8 < rows;
}

// A row's token in its sequence and the place of head 0's 64 channels in the cache, in tokens; -1: none.
__device__ __forceinline__ int64_t place(const CacheArgs &a, int64_t row, bool covered, int &token)
{
    token = 0;
    if (!covered) return -1;
    const int b = a.spans.find(row);
    int first, len;
    a.spans.of(b, first, len);
    const int n = a.cache.length(b);
    token = n - len + static_cast<int>(row) - first;
    return token < 0 || token >= n ? -1 : a.cache.slot(b, token);
}

// Cosines and sines for channels 8 c .. 8 c + 7 of a row (halves: of the eight pairs they belong to; neighbours: of four), the sines with
// the sign that the channel's own half takes.
struct Angles {
    float co[8], si[8];
    __device__ __forceinline__ void load(const Rotation &rot, int64_t row, int token, int c)
    {
        const int pairs = 32 / rot.axes, axis = rot.axes == 2 ? c >> 2 : 0;
        int64_t at = rot.positions != nullptr ? rot.positions[row * rot.axes + axis] : token;
        at = at < 0 ? 0 : (at >= rot.places ? rot.places - 1 : at);
        const int index = rot.neighbours ? (4 * c) % pairs : (8 * c) % pairs;
        const float *cs = rot.cos + at * pairs + index, *sn = rot.sin + at * pairs + index;
        if (rot.neighbours) {
            const floatx4 x = *reinterpret_cast<const floatx4 *>(cs), y = *reinterpret_cast<const floatx4 *>(sn);
#pragma unroll
            for (int j = 0; j < 8; ++j) { co[j] = x[j >> 1]; si[j] = (j & 1) != 0 ? y[j >> 1] : -y[j >> 1]; }
        } else {
            load8(cs, co);
            load8(sn, si);
            const bool second = (c & (rot.axes == 2 ? 2 : 4)) != 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) si[j] = second ? si[j] : -si[j];
        }
    }
    // A channel a of a pair becomes a cos - b sin, its partner b cos + a sin: rounded to odd (the last bit is set where the value is not
    // exact), so that rounding to fewer bits, or comparing with numbers of fewer bits, gives what the exact value would.  Only values whose
    // lower bits are all the same as those of such a number can tell the difference: 15 zero bits, or 20 for the codes.
    // odd = false: rounded to fp32, to be kept as that.
    __device__ __forceinline__ void turn(const Rotation &rot, const float (&x)[8], float (&y)[8], bool odd) const
    {
        float other[8];
        if (rot.neighbours) {
#pragma unroll
            for (int j = 0; j < 8; ++j) other[j] = x[j ^ 1];
        } else if (rot.axes == 2) {
#pragma unroll
            for (int j = 0; j < 8; ++j) other[j] = __uint_as_float(other_lane<2>(__float_as_uint(x[j])));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) other[j] = __uint_as_float(other_lane<4>(__float_as_uint(x[j])));
        }
        auto exact = [&](int j) {
            return fma(static_cast<double>(x[j]), static_cast<double>(co[j]), static_cast<double>(other[j]) * static_cast<double>(si[j]));
        };
        unsigned lowest = 0x7fffu;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            y[j] = static_cast<float>(exact(j));
            lowest = min(lowest, __float_as_uint(y[j]) & 0x7fffu);
        }
        if (odd && lowest == 0)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if ((__float_as_uint(y[j]) & 0x7fffu) == 0) y[j] = round_to_odd(exact(j));
    }
};

// Heads whose rows are requested at once: 64 bytes of a lane.
template <typename T> constexpr int kAhead = sizeof(T) == 4 ? 2 : 4;

template <typename T> __global__ __launch_bounds__(256) void cache_append_kernel(CacheArgs a, int run)
{
    const int kv_heads = a.cache.kv_heads, turned = a.q != nullptr ? a.heads : 0;  // the heads in turn: q, k, v
    HeadRun r;
    if (!head_run(a.n_rows, turned + 2 * kv_heads, run, r)) return;
    const int c = threadIdx.x & 7;
    const bool covered = r.row < a.n_rows && a.spans.covers(r.row);
    int token;
    const int64_t slot = place(a, r.row, covered, token);
    Angles angles;
    const bool turns = a.rot.cos != nullptr;
    if (turns && r.h0 < turned + kv_heads && covered) angles.load(a.rot, r.row, token, c);
    for (int h0 = r.h0; h0 < r.h1; h0 += kAhead<T>) {
        Io8<T> in[kAhead<T>];
#pragma unroll
        for (int i = 0; i < kAhead<T>; ++i) {
            const int h = h0 + i;
            if (h >= r.h1 || !covered) continue;
            if (h < turned)
                in[i].load(static_cast<const T *>(a.q) + r.row * a.q_row + h * a.q_head + 8 * c);
            else if (h < turned + kv_heads)
                in[i].load(static_cast<const T *>(a.k) + r.row * a.kv_row + (h - turned) * a.kv_head + 8 * c);
            else
                in[i].load(static_cast<const T *>(a.v) + r.row * a.kv_row + (h - turned - kv_heads) * a.kv_head + 8 * c);
        }
#pragma unroll
        for (int i = 0; i < kAhead<T>; ++i) {
            const int h = h0 + i;
            if (h >= r.h1) continue;
            float x[8], y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = in[i].get(j);
            if (turns && h < turned + kv_heads) {
                angles.turn(a.rot, x, y, sizeof(T) == 2 || h >= turned);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = x[j];
            }
            if (h < turned) {
                if (covered) Io8<T>::store(static_cast<T *>(a.to.out) + (r.row * a.heads + h) * 64 + 8 * c, y);
                continue;
            }
            const bool is_v = h >= turned + kv_heads;
            unsigned most = 0;  // magnitudes compare as integers; infinities and NaNs are the largest
#pragma unroll
            for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(y[j]) & 0x7fffffffu);
            most = max(most, other_lane<1>(most));
            most = max(most, other_lane<2>(most));
            int e = static_cast<int>(most >> 23) - 129 + ((most & 0x7fffffu) >= 0x600000u ? 1 : 0);
            e = e < -100 ? -100 : (e > 125 ? 125 : e);
            const bool none = most >= 0x7f800000u;
            const unsigned scale = none ? 255u : static_cast<unsigned>(e + 127);
            const float unit = __uint_as_float(static_cast<unsigned>(e + 127) << 23);
            unsigned codes = 0;
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[0], y[1], unit, 0);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[2], y[3], unit, 1);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[4], y[5], unit, 2);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, y[6], y[7], unit, 3);
            const unsigned second = other_lane<4>(scale);
            if (slot < 0) continue;
            const int64_t at = slot + (static_cast<int64_t>(h - turned - (is_v ? kv_heads : 0)) << a.cache.page_shift);
            *reinterpret_cast<unsigned *>((is_v ? a.cache.v_codes : a.cache.k_codes) + at * 32 + 4 * c) = none ? 0u : codes;
            if (c == 0)
                *reinterpret_cast<unsigned short *>((is_v ? a.cache.v_scales : a.cache.k_scales) + at * 2) = static_cast<unsigned short>(scale | second << 8);
        }
    }
}

// Two codes at a time -> bf16, exactly; `scale`: the exponent byte.
__device__ __forceinline__ bf16x8 values8(unsigned codes, unsigned scale)
{
    const float unit = __uint_as_float(scale << 23);
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 1);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 3);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

template <typename T> __global__ __launch_bounds__(256) void cache_read_kernel(CacheArgs a, int run)
{
    const int kv_heads = a.cache.kv_heads;  // the heads in turn: k, v
    HeadRun r;
    if (!head_run(a.n_rows, 2 * kv_heads, run, r)) return;
    if (r.row >= a.n_rows || !a.spans.covers(r.row)) return;
    const int c = threadIdx.x & 7;
    int token;
    const int64_t slot = place(a, r.row, true, token);
    for (int h0 = r.h0; h0 < r.h1; h0 += 4) {
        unsigned codes[4], scale[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int h = h0 + i;
            if (h >= r.h1 || slot < 0) continue;
            const bool is_v = h >= kv_heads;
            const int64_t at = slot + (static_cast<int64_t>(h - (is_v ? kv_heads : 0)) << a.cache.page_shift);
            codes[i] = *reinterpret_cast<const unsigned *>((is_v ? a.cache.v_codes : a.cache.k_codes) + at * 32 + 4 * c);
            scale[i] = (is_v ? a.cache.v_scales : a.cache.k_scales)[at * 2 + (c >> 2)];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int h = h0 + i;
            if (h >= r.h1) continue;
            bf16x8 x = {};
            if (slot >= 0) x = values8(codes[i], scale[i]);
            T *to = (h >= kv_heads ? static_cast<T *>(a.v) + (h - kv_heads) * a.kv_head : static_cast<T *>(a.k) + h * a.kv_head) + r.row * a.kv_row + 8 * c;
            if constexpr (sizeof(T) == 2) {
                *reinterpret_cast<bf16x8 *>(to) = x;
            } else {
                float f[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = static_cast<float>(x[j]);
                Io8<T>::store(to, f);
            }
        }
    }
}

// ---- attention -------------------------------------------------------------------------------------------

// Units of 64 cached tokens, a token for a lane.  In LDS they are bf16, which holds the values exactly.  Blocks of values that read as
// NaN are put as zeros and told apart by a word per 32 channels, because only rows that see their token may become NaN.
constexpr int kCacheStage = 2 * kPlane + 32;  // bf16 elements: keys, values, two 64-bit words and room to stay aligned

// A page of 64 tokens and more (WIDE) holds whole units: its number and all addresses but a constant per lane are then scalars (one
// token over 137400 cached 34.2 -> 32.3 us; with many rows, where the matrix and vector units bind, no difference).
template <bool WIDE> struct PageUnits {
    Cache cache;
    int seq, kv_head, len;
    int64_t next;  // of the unit to be fetched next: the lane's place in the cache, head 0's; WIDE: the unit's.  -1: nowhere
    bool there;    // the lane's token of the unit that was fetched
    __device__ __forceinline__ void find(int unit, int lane)
    {
        const int t = unit * kUnitRows + (WIDE ? 0 : lane);
        next = t < len ? cache.slot(seq, t) : -1;
    }
    // Byte offset of the unit's codes in the arrays of codes: from here a lane's are lane * 32 further (WIDE), or here.
    __device__ __forceinline__ int64_t fetch(int unit, int lane)
    {
        there = next >= 0 && (!WIDE || unit * kUnitRows + lane < len);
        return (next + (static_cast<int64_t>(kv_head) << cache.page_shift)) * 32;
    }
    // The same of 16 tokens, which lie on one page; a tile that is nowhere reads the first page instead, and counts for nothing.
    __device__ __forceinline__ int64_t tile(int t) const
    {
        int64_t at = next;
        if constexpr (WIDE) {
            at = (at < 0 ? 0 : at) + 16 * t;
        } else {
            const unsigned lo = __builtin_amdgcn_readlane(static_cast<unsigned>(at), 16 * t), hi = __builtin_amdgcn_readlane(static_cast<unsigned>(at >> 32), 16 * t);
            at = static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
            at = at < 0 ? 0 : at;
        }
        return (at + (static_cast<int64_t>(kv_head) << cache.page_shift)) * 32;
    }
    static __device__ __forceinline__ int lane_bytes(int lane) { return WIDE ? lane * 32 : 0; }
};

// 32 channels of a lane's token, as bf16 to a unit in LDS; not `ok`: zeros.
__device__ __forceinline__ void put_block(bf16_t *unit, int row, int half, uint4 codes, unsigned scale, bool ok)
{
    if (!ok) { codes = uint4{0, 0, 0, 0}; scale = 127; }
    *reinterpret_cast<bf16x8 *>(unit + unit_chunk(row, 4 * half + 0)) = values8(codes.x, scale);
    *reinterpret_cast<bf16x8 *>(unit + unit_chunk(row, 4 * half + 1)) = values8(codes.y, scale);
    *reinterpret_cast<bf16x8 *>(unit + unit_chunk(row, 4 * half + 2)) = values8(codes.z, scale);
    *reinterpret_cast<bf16x8 *>(unit + unit_chunk(row, 4 * half + 3)) = values8(codes.w, scale);
}

// What a workgroup's rows of a sequence see.
struct Sight {
    int first, rows, len, sees, most;  // sees: tokens that the lane's row sees; most: that the last row of the tile sees
    int64_t row;
    int head;
    bool ok;
    __device__ __forceinline__ void find(const CacheArgs &a, const Share &sh, int tile, int item_in_tile)
    {
        first = sh.of.first;
        rows = sh.of.len;
        len = a.cache.held_length(sh.of.entry);
        const int64_t items = static_cast<int64_t>(rows) * a.per_row, item0 = static_cast<int64_t>(sh.tile) * tile, item = item0 + item_in_tile;
        ok = item < items;
        const int in_seq = static_cast<int>(item / a.per_row);
        row = first + in_seq;
        head = sh.kv_head * a.per_row + static_cast<int>(item - static_cast<int64_t>(in_seq) * a.per_row);
        sees = most = len;
        if (a.causal) {
            sees = min(len, len - rows + in_seq + 1);
            const int64_t last = (item0 + tile < items ? item0 + tile : items) - 1;
            most = max(0, min(len, len - rows + static_cast<int>(last / a.per_row) + 1));
            if (!ok) sees = most;
        }
    }
};

// Many rows: four waves hold 32 rows each and share every unit; a wave brings 32 channels of its keys (waves 0, 1) or values (2, 3).
template <typename T> __global__ __launch_bounds__(256, 2) void cache_attn_kernel(CacheArgs a)
{
    constexpr int P = sizeof(T) == 4 ? 3 : 1;
    extern __shared__ __align__(16) unsigned char smem[];
    bf16_t *lds = reinterpret_cast<bf16_t *>(smem);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = wave & 1;
    const bool is_v = wave >= 2;
    Share sh;
    if (!find_share(a.spans, a.cache.kv_len, a.per_row, 128, a.tiles, a.n_split, a.cache.kv_heads, !a.uneven, false, sh)) return;
    Sight sight;
    sight.find(a, sh, 128, 32 * wave + (lane & 31));
    int u0, u1;
    piece((sight.most + kUnitRows - 1) / kUnitRows, a.n_split, a.least, sh.split, u0, u1);
    if (a.to.part_o != nullptr && u0 == u1) return store_no_keys(a.to, sh.split, sight.row, sight.head, sight.ok && lane < 32);
    SoftRow<P> soft;
    soft.clear();
    soft.load(static_cast<const T *>(a.q) + sight.row * a.q_row + sight.head * a.q_head, sight.ok, lane);
    PageUnits<false> units{a.cache, sh.of.seq, sh.kv_head, sight.len, -1, false};
    const uint8_t *codes = is_v ? a.cache.v_codes : a.cache.k_codes, *scales = is_v ? a.cache.v_scales : a.cache.k_scales;
    uint4 code = {};
    unsigned scale = 0;
    auto fetch = [&](int u) {
        const int64_t from = units.fetch(u, lane);
        if (!units.there) return;
        code = *reinterpret_cast<const uint4 *>(codes + from + (units.lane_bytes(lane) + 16 * half));
        scale = (scales + from / 16)[units.lane_bytes(lane) / 16 + half];
    };
    const UnitLanes at(lane);
    if (u0 < u1) { units.find(u0, lane); fetch(u0); units.find(u0 + 1, lane); }
    for (int u = u0; u < u1; ++u) {
        bf16_t *stage = lds + ((u - u0) & 1) * kCacheStage;
        unsigned long long *words = reinterpret_cast<unsigned long long *>(stage + 2 * kPlane);
        const bool none = is_v && units.there && scale == 255u;
        put_block(stage + (is_v ? kPlane : 0), lane, half, code, scale, units.there && !none);
        const unsigned long long w = __ballot(none);
        if (is_v && lane == 0) words[half] = w;
        const unsigned long long seen = __ballot(units.there) & low_bits(sight.sees - u * kUnitRows);
        __syncthreads();
        if (u + 1 < u1) { fetch(u + 1); units.find(u + 2, lane); }
        soft.template unit<1>(stage, stage + kPlane, seen, a.factor, at, lane);
#pragma unroll
        for (int dt = 0; dt < 2; ++dt) {
            const unsigned long long nan = words[dt];
            if (nan != 0 && (nan & seen) != 0)
#pragma unroll
                for (int r = 0; r < 16; ++r) soft.o[dt][r] = NAN;
        }
    }
    store_soft<T>(soft, a.factor, a.to, sh.split, sight.row, sight.head, sight.ok, lane);
}

// Few rows: WAVES waves with the same 16 rows take the units in turn.  Probabilities of bf16 rows enter in one part: a second one costs up to
// a tenth (one row over 137400 tokens 37.9 us -> 41.6) and spares an error of 1e-3 beside that of the 4 bits.
template <typename T, int WAVES, bool WIDE> __global__ __launch_bounds__(64 * WAVES, WAVES == 4 ? 2 : 1) void cache_few_kernel(CacheArgs a)
{
    constexpr int P = sizeof(T) == 4 ? 3 : 1;
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    bf16_t *mine = reinterpret_cast<bf16_t *>(smem) + wave * kPlane;
    Share sh;
    if (!find_share(a.spans, a.cache.kv_len, a.per_row, kFewRows, a.tiles, a.n_split, a.cache.kv_heads, false, true, sh)) return;
    Sight sight;
    sight.find(a, sh, kFewRows, lane & 15);
    int u0, u1;
    piece((sight.most + kUnitRows - 1) / kUnitRows, a.n_split, a.least, sh.split, u0, u1);
    if (a.to.part_o != nullptr && u0 == u1) return store_no_keys(a.to, sh.split, sight.row, sight.head, sight.ok && threadIdx.x < 16);
    FewRows<P> few;
    few.clear();
    few.load(static_cast<const T *>(a.q) + sight.row * a.q_row + sight.head * a.q_head, sight.ok, lane);
    PageUnits<WIDE> units{a.cache, sh.of.seq, sh.kv_head, sight.len, -1, false};
    uint2 k[4] = {};
    uint4 v[2] = {};
    unsigned ks[4] = {}, vs = 0;
    auto fetch = [&](int u) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int64_t from = units.tile(t);
            k[t] = *reinterpret_cast<const uint2 *>(a.cache.k_codes + from + ((lane & 15) * 32 + (lane >> 4) * 8));
            ks[t] = (a.cache.k_scales + from / 16)[(lane & 15) * 2 + (lane >> 5)];
        }
        const int64_t from = units.fetch(u, lane);
        if (!units.there) return;
        const uint8_t *codes = a.cache.v_codes + from + units.lane_bytes(lane);
        v[0] = *reinterpret_cast<const uint4 *>(codes);
        v[1] = *reinterpret_cast<const uint4 *>(codes + 16);
        vs = *reinterpret_cast<const unsigned short *>(a.cache.v_scales + from / 16 + units.lane_bytes(lane) / 16);
    };
    int u = u0 + wave;
    if (u < u1) { units.find(u, lane); fetch(u); units.find(u + WAVES, lane); }
    for (; u < u1; u += WAVES) {
        unsigned long long nan[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const unsigned scale = (vs >> (8 * half)) & 255u;
            const bool none = units.there && scale == 255u;
            put_block(mine, lane, half, v[half], scale, units.there && !none);
            nan[half] = __ballot(none);
        }
        const unsigned long long seen = __ballot(units.there) & low_bits(sight.sees - u * kUnitRows);
        bf16x8 kk[4][2];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            kk[t][0] = values8(k[t].x, ks[t]);
            kk[t][1] = values8(k[t].y, ks[t]);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (u + WAVES < u1) { fetch(u + WAVES); units.find(u + 2 * WAVES, lane); }
        few.template unit<1, P>([&](int t, int s, bf16x8(&to)[1]) { to[0] = kk[t][s]; }, mine, seen, a.factor, lane);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int half = 0; half < 2; ++half)
            if (nan[half] != 0 && (nan[half] & seen) != 0)
#pragma unroll
                for (int r = 0; r < 4; ++r) few.o[2 * half][r] = few.o[2 * half + 1][r] = NAN;
    }
    __syncthreads();
    store_few<T, WAVES>(few, a.factor, a.to, sh.split, sight.row, sight.head, sight.ok, reinterpret_cast<float *>(smem), wave, lane);
}

// ---- faults of what a call was given ---------------------------------------------------------------------
__global__ __launch_bounds__(1024) void cache_status_kernel(CacheArgs a, bool appends, int *status)
{
    int bad = spans_bad(a.spans) ? kDiagSpans : 0;
    for (int b = 0; b < a.spans.batch; ++b) {
        const int n = a.cache.length(b);
        int first, len;
        a.spans.of(b, first, len);
        if (a.cache.kv_len[b] != n || (appends && len > n)) bad |= kDiagLength;
        const int pages = (n + (1 << a.cache.page_shift) - 1) >> a.cache.page_shift;
        for (int p = threadIdx.x; p < pages; p += 1024)
            if (a.cache.slot(b, p << a.cache.page_shift) < 0) bad |= kDiagPage;
        if (appends && a.rot.cos != nullptr && a.rot.positions == nullptr && len > 0 && n > a.rot.places) bad |= kDiagPosition;
    }
    if (appends && a.rot.cos != nullptr && a.rot.positions != nullptr)
        for (int64_t i = threadIdx.x; i < a.n_rows * a.rot.axes; i += 1024)
            if (a.spans.covers(i / a.rot.axes) && (a.rot.positions[i] < 0 || a.rot.positions[i] >= a.rot.places)) bad |= kDiagPosition;
    __shared__ int all;
    if (threadIdx.x == 0) all = 0;
    __syncthreads();
    if (bad != 0) atomicOr(&all, bad);
    __syncthreads();
    if (threadIdx.x == 0) *status = all;
}

template <typename T, int WAVES, bool WIDE> hipError_t launch_few(const CacheArgs &a, int64_t n, hipStream_t stream)
{
    constexpr size_t kLds = WAVES * kPlane * sizeof(bf16_t);
    const hipError_t e = allow_lds(&cache_few_kernel<T, WAVES, WIDE>, kLds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((cache_few_kernel<T, WAVES, WIDE>), dim3(static_cast<unsigned>(n)), dim3(64 * WAVES), kLds, stream, a);
    return hipGetLastError();
}

template <typename T> hipError_t launch_cache_attn_t(const CacheArgs &a, bool few_rows, hipStream_t stream)
{
    const int64_t shares = a.tiles * a.n_split * a.cache.kv_heads, n = few_rows ? shares : xcd_padded(shares);
    if (!grid_ok(few_rows ? 4 * n : n)) return hipErrorInvalidValue;  // (up to 1024 threads)
    if (few_rows) {
        constexpr int kMany = sizeof(T) == 4 ? 8 : 16;
        if (a.cache.page_shift >= 6)
            return a.n_split > 1 ? launch_few<T, 4, true>(a, n, stream) : launch_few<T, kMany, true>(a, n, stream);
        return a.n_split > 1 ? launch_few<T, 4, false>(a, n, stream) : launch_few<T, kMany, false>(a, n, stream);
    }
    hipLaunchKernelGGL(cache_attn_kernel<T>, dim3(static_cast<unsigned>(n)), dim3(256), 2 * kCacheStage * sizeof(bf16_t), stream, a);
    return hipGetLastError();
}

// Heads that a wave takes in a row: as many, up to 16, as leave the card 8192 waves (eight for each of 1024 SIMDs).
int run_of_heads(int64_t rows, int heads)
{
    int run = 1;
    while (run < 16 && (rows + 7) / 8 * ((heads + 2 * run - 1) / (2 * run)) >= 8192) run *= 2;
    return run;
}

}  // namespace

hipError_t launch_cache_append(const CacheArgs &a, bool is_bf16, hipStream_t stream)
{
    const int heads = 2 * a.cache.kv_heads + (a.q != nullptr ? a.heads : 0), run = run_of_heads(a.n_rows, heads);
    const int64_t blocks = ((a.n_rows + 7) / 8 * ((heads + run - 1) / run) + 3) / 4;
    if (!grid_ok(blocks)) return hipErrorInvalidValue;
    if (is_bf16)
        hipLaunchKernelGGL(cache_append_kernel<bf16_t>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, a, run);
    else
        hipLaunchKernelGGL(cache_append_kernel<float>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, a, run);
    return hipGetLastError();
}

hipError_t launch_cache_read(const CacheArgs &a, bool is_bf16, hipStream_t stream)
{
    const int heads = 2 * a.cache.kv_heads, run = run_of_heads(a.n_rows, heads);
    const int64_t blocks = ((a.n_rows + 7) / 8 * ((heads + run - 1) / run) + 3) / 4;
    if (!grid_ok(blocks)) return hipErrorInvalidValue;
    if (is_bf16)
        hipLaunchKernelGGL(cache_read_kernel<bf16_t>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, a, run);
    else
        hipLaunchKernelGGL(cache_read_kernel<float>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, a, run);
    return hipGetLastError();
}

hipError_t launch_cache_attn(const CacheArgs &a, bool few_rows, bool is_bf16, hipStream_t stream)
{
    return is_bf16 ? launch_cache_attn_t<bf16_t>(a, few_rows, stream) : launch_cache_attn_t<float>(a, few_rows, stream);
}

hipError_t launch_cache_status(const CacheArgs &a, bool appends, int *status, hipStream_t stream)
{
    hipLaunchKernelGGL(cache_status_kernel, dim3(1), dim3(1024), 0, stream, a, appends, status);
    return hipGetLastError();
}

}  // namespace s3r
