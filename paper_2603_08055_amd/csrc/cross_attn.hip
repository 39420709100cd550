// Cross attention, out[i] = sum_j softmax_j(scale q_i . k_j) v_j, with keys of another length than the queries, and its gradient
//   P = exp(scale q k^T - lse),  D_i = out_i . d_out_i,  dS = scale P (d_out v^T - D),
//   dq = dS k,  dk = dS^T q,  dv = P^T d_out.
// Batches of ragged sequences lie one behind the other; several query heads may share a head of keys: their rows are then
// items of one tile, and the gradient of the shared head is one sum over all of them.  No atomics: a sum that is split over workgroups
// goes through partial results in the workspace, which another launch adds up in a fixed order.
//
// CAUSAL: the rows of a sequence are its last tokens, and see those of their own view and of earlier ones; units that no row of a tile (of a
// wave) sees are not walked, and the tiles, which now differ in length, are dealt out the longest first (of up to 64 sequences; of more, one sequence after the other).  What bounds a unit of keys is what bounds it
// without (matrix pipe and vector ALU, which hardly overlap): 10992 rows in views of 1374, 16 heads in bf16, 344 to 367 us, 760 to 810 TFLOP/s of the
// pairs that count; 8192 rows in three prompts, 16 heads that share 4: 87 us forward, 119 + 144 + 12 (joining) for the gradients.
#include "s3r_unit_device.h"

namespace s3r {

namespace {

constexpr int kTile = 128;  // held rows of a workgroup: 32 for each of four waves

// Keys and values of a sequence, for a head of theirs.
template <typename T>
__device__ __forceinline__ UnitPairs<T> key_units(const CrossArgs &a, int kv_head, int first, int len, bf16_t *lds)
{
    const int64_t at = first * a.kv_row + kv_head * a.kv_head;
    return UnitPairs<T>(static_cast<const T *>(a.k) + at, static_cast<const T *>(a.v) + at, len, a.kv_row, 0, a.kv_row, 0, 1, lds);
}

__device__ __forceinline__ CountedRows counted(const CrossArgs &a, int first, int len)
{
    return CountedRows{a.key_mask != nullptr ? a.key_mask + first : nullptr, len, 0};
}

// Causal rows: the n rows of a sequence are its last tokens of m, and each sees the tokens of its own view of `view` tokens and of those
// before (view 1: the tokens up to itself).  Keys that row i sees, and the first row that sees a key.
__device__ __forceinline__ int keys_seen(int i, int n, int m, int view)
{
    const int t = m - n + i;
    return t < 0 ? 0 : (view == 1 ? t + 1 : min(m, (t / view + 1) * view));
}
__device__ __forceinline__ int first_seer(int key, int n, int m, int view) { return max(0, (view == 1 ? key : key / view * view) - (m - n)); }

// Keys that the last of a tile's items sees; `items`: of the sequence.
__device__ __forceinline__ int tile_sees(int64_t end, int64_t items, int per_row, int n, int m, int view)
{
    return keys_seen(static_cast<int>((end < items ? end : items) - 1) / per_row, n, m, view);
}

// Pieces of causal tiles, n_split of them or fewer, by the lengths of up to 64 sequences, of which the host knows the sums alone: a lane for a
// sequence, then one for a number of pieces, by the host's model of the launch (causal_us).  The kernels of a call have to find the same: sums
// are those of integers, and no product of floats is added to anything, which the compiler might round once or twice.
// bf16, forward and gradients, us with the number that the host guesses / so: 17 sequences of up to 220 rows, one over 4075 keys 142 / 73, 17 of up to 203
// over up to 1160 100 / 72, 64 of up to 64 rows, one over 2026 keys 87 / 65; what it costs where it finds no use: 17 of 60 rows over 500 keys 59 / 68.
template <bool OF_KEYS> __device__ __forceinline__ int causal_split(const CrossArgs &a)
{
    if (a.resident == 0) return a.n_split;
    const int lane = threadIdx.x & 63;
    int tiles = 0, work = 0, longest = 0;  // work: twice the units of all tiles
    if (lane < a.q_spans.batch) {
        int at, n, m;
        a.q_spans.of(lane, at, n);
        a.kv_spans.of(lane, at, m);
        if (n > 0 && m > 0) {
            const int items = n * a.per_row, before = max(m - n, 0), last = OF_KEYS ? items : m;
            const int first = OF_KEYS ? static_cast<int>(static_cast<float>(items) * (static_cast<float>(before) / static_cast<float>(m))) : min(before + a.view, m);
            tiles = ((OF_KEYS ? m : items) + kTile - 1) / kTile;
            work = static_cast<int>(min(static_cast<int64_t>(tiles) * (first / kUnitRows + last / kUnitRows + 1), int64_t(1) << 24));
            longest = (last + kUnitRows - 1) / kUnitRows;
        }
    }
    for (int x = 1; x < 64; x <<= 1) {
        tiles += __shfl_xor(tiles, x, 64);
        work += __shfl_xor(work, x, 64);
        longest = max(longest, __shfl_xor(longest, x, 64));
    }
    tiles = min(tiles, 1 << 10) * a.kv_heads;
    const int n = lane + 1, others = a.resident - 1, on_cus = min(max(tiles * n, 256), 256 * a.resident);
    const float alone = others > 1 ? 2000.f : (others > 0 ? 1600.f : 1100.f);
    const float pace = others > 0 ? static_cast<float>(3 * 256 * others - (on_cus - 256)) / static_cast<float>(2 * 256 * others) : 1.f;
    const float all = static_cast<float>(work) * static_cast<float>(a.kv_heads) * a.unit_us * pace * (1000.f / 512), piece = static_cast<float>(longest) * a.unit_us * alone / static_cast<float>(n);
    int ns = static_cast<int>(fminf(fmaxf(all, piece), 1e9f)) + (lane == 0 ? 0 : a.join_ns + tiles * n * a.tile_ns);
    if (lane >= a.n_split || (lane > 0 && longest < a.least * n)) ns = 0x7fffffff;
    int least = ns;
    for (int x = 1; x < 64; x <<= 1) least = min(least, __shfl_xor(least, x, 64));
    return __builtin_amdgcn_readfirstlane(static_cast<int>(__ffsll(__ballot(ns - least <= least / 100))));
}

// Pieces of a causal tile: n_split alike of `least` units or more, or fewer (so that they differ in length as the tiles do, and the CUs that are
// done first find short ones), none of them empty where there are units; a tile of one piece goes straight to the results.
// (Pieces of one length for all tiles, by the longest: 4096 rows of 16 heads that share 4 with gradients 273 us so, 330 by length; 8192 in three
// sequences 370 and 364.)
__device__ __forceinline__ int causal_pieces(int units, int n_split, int least)
{
    const int per = max(1, piece_units(units, n_split, least));
    return max(1, (units + per - 1) / per);
}
__device__ __forceinline__ bool causal_piece(int units, int n_split, int least, int split, int &u0, int &u1, bool &whole)
{
    const int n = causal_pieces(units, n_split, least);
    piece(units, n_split, least, split, u0, u1);
    whole = n == 1;
    return split < n;
}

// Units of a tile of keys: those from the first that sees its first key.
__device__ __forceinline__ void seeing_units(const CrossArgs &a, int tile, int q_len, int k_len, int &from, int &end)
{
    end = (q_len * a.per_row + kUnitRows - 1) / kUnitRows;
    from = min(end, first_seer(tile * kTile, q_len, k_len, a.view) * a.per_row / kUnitRows);
}

// Tiles of a sequence of n rows and m keys that walk `units` units or more (1 or more), which are the last ones of the rows (OF_KEYS: of
// the keys, the first ones).
template <bool OF_KEYS> __device__ __forceinline__ int tiles_of_units(const CrossArgs &a, int n, int m, int tiles, int units)
{
    if constexpr (!OF_KEYS) {
        const int key = (units - 1) * kUnitRows;
        const int row = first_seer(key, n, m, a.view);
        return key >= m || row >= n ? 0 : tiles - row * a.per_row / kTile;
    } else {
        const int end = (n * a.per_row + kUnitRows - 1) / kUnitRows;
        if (units > end) return 0;
        const int last = ((end - units + 1) * kUnitRows - 1) / a.per_row + m - n;  // its first key's view begins here at the latest
        if (last < 0) return 0;
        const int keys = a.view == 1 ? last + 1 : (last / a.view + 1) * a.view;
        return min(tiles, (keys - 1) / kTile + 1);
    }
}

// A workgroup's share of causal work.  The tiles are taken by the number of units they walk, the most first, so that the CUs that are done
// first take short ones last; of up to 64 sequences, a lane for each: the number of units by bisection, then the tile among those that walk as
// many.  (More sequences: one after the other, the longest tile of each first, and pieces by their mean length: a long one among them that comes early is started late, and
// in as many pieces as the mean asks for.)  8192 rows in three sequences, 16 heads that share 4, sequence by
// sequence / so: forward 108 / 90 us, query gradient 157 / 131.
template <bool OF_KEYS> __device__ __forceinline__ bool find_causal_share(const CrossArgs &a, int n_split, Share &s)
{
    const int each = n_split * a.kv_heads, u = static_cast<int>(blockIdx.x) / each, rest = static_cast<int>(blockIdx.x) - u * each;
    s.split = rest / a.kv_heads;
    s.kv_head = rest - s.split * a.kv_heads;
    const Spans &held = OF_KEYS ? a.kv_spans : a.q_spans, &other = OF_KEYS ? a.q_spans : a.kv_spans;
    const int per_row = OF_KEYS ? 1 : a.per_row;
    if (held.batch == 1 || held.batch > 64) {
        const int64_t t = OF_KEYS ? u : a.tiles - 1 - u;
        if (t < 0 || t >= a.tiles) return false;
        return find_tile(held, nullptr, per_row, kTile, t, s.of, s.tile);
    }
    const int lane = threadIdx.x & 63;
    int first = 0, len = 0, other_first = 0, other_len = 0;
    if (lane < held.batch) {
        held.of(lane, first, len);
        other.of(lane, other_first, other_len);
    }
    const int n = OF_KEYS ? other_len : len, m = OF_KEYS ? len : other_len;
    const int tiles = static_cast<int>((static_cast<int64_t>(len) * per_row + kTile - 1) / kTile);
    auto total = [](int x) { return __builtin_amdgcn_readlane(sum_up_to(x), 63); };
    if (u >= total(tiles)) return false;
    int most = OF_KEYS ? (n * a.per_row + kUnitRows - 1) / kUnitRows : (m + kUnitRows - 1) / kUnitRows;
    if (tiles == 0) most = 0;
    for (int d = 1; d < 64; d <<= 1) most = max(most, __shfl_xor(most, d, 64));
    int lo = 0, hi = __builtin_amdgcn_readfirstlane(most) + 1;  // more than u tiles walk lo units or more, and not so many walk hi
    int lo_tiles = tiles, hi_tiles = 0;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2, c = tiles_of_units<OF_KEYS>(a, n, m, tiles, mid);
        if (total(c) > u) { lo = mid; lo_tiles = c; } else { hi = mid; hi_tiles = c; }
    }
    const int here = lo_tiles - hi_tiles, upto = sum_up_to(here), rank = u - total(hi_tiles);
    const int l = __ffsll(__ballot(upto > rank)) - 1;
    const int k = rank - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(here, l)), above = __builtin_amdgcn_readlane(hi_tiles, l);
    s.of.seq = l;
    s.of.first = __builtin_amdgcn_readlane(first, l);
    s.of.len = __builtin_amdgcn_readlane(len, l);
    s.tile = OF_KEYS ? above + k : __builtin_amdgcn_readlane(tiles, l) - above - 1 - k;
    return true;
}

// What a tile of kTile items, a wave of it and the lane's row see; `tile` keys are walked.  Without CAUSAL: all.
template <bool CAUSAL> struct CausalTile {
    int tile, mine, wave, all;  // all: keys that all of the tile's rows see
    __device__ __forceinline__ CausalTile(const CrossArgs &a, int t, int n, int m, int64_t item, bool ok, int w) : tile(m), mine(m), wave(m), all(m)
    {
        if constexpr (CAUSAL) {
            const int64_t items = static_cast<int64_t>(n) * a.per_row, item0 = static_cast<int64_t>(t) * kTile + 32 * w;
            tile = tile_sees(static_cast<int64_t>(t + 1) * kTile, items, a.per_row, n, m, a.view);
            wave = __builtin_amdgcn_readfirstlane(item0 < items ? tile_sees(item0 + 32, items, a.per_row, n, m, a.view) : 0);
            mine = ok ? keys_seen(static_cast<int>(item) / a.per_row, n, m, a.view) : wave;
            all = keys_seen(t * kTile / a.per_row, n, m, a.view);
        }
    }
    __device__ __forceinline__ bool sees(int unit) const { return !CAUSAL || unit * kUnitRows < wave; }
    __device__ __forceinline__ unsigned long long of(unsigned long long seen, int unit) const
    {
        return CAUSAL ? seen & low_bits(mine - unit * kUnitRows) : seen;
    }
};

// Many rows: four waves hold 32 rows each and share every unit.  PP: parts of their probabilities.
template <typename T, int PP, bool CAUSAL> __global__ __launch_bounds__(256, sizeof(T) == 4 ? 2 : 4) void cross_kernel(CrossArgs a)
{
    constexpr int P = UnitPairs<T>::kParts;
    extern __shared__ __align__(16) unsigned char smem[];
    bf16_t *lds = reinterpret_cast<bf16_t *>(smem);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Share sh;
    int pieces;  // causal: of a tile, at most
    if constexpr (CAUSAL) {
        pieces = causal_split<false>(a);
        if (!find_causal_share<false>(a, pieces, sh)) return;
    } else {
        if (!find_share(a.q_spans, nullptr, a.per_row, kTile, a.tiles, a.n_split, a.kv_heads, !a.uneven, true, sh)) return;
    }
    const int q0 = sh.of.first, q_len = sh.of.len;
    int k0, k_len;
    a.kv_spans.of(sh.of.seq, k0, k_len);
    const int64_t item = static_cast<int64_t>(sh.tile) * kTile + 32 * wave + (lane & 31);
    const bool ok = item < static_cast<int64_t>(q_len) * a.per_row;
    const int64_t row = q0 + item / a.per_row;
    const int head = sh.kv_head * a.per_row + static_cast<int>(item % a.per_row);
    const CausalTile<CAUSAL> sight(a, sh.tile, q_len, k_len, item, ok, wave);
    int u0, u1;
    SoftOut to = a.to;
    if constexpr (CAUSAL) {
        bool whole;
        if (!causal_piece((sight.tile + kUnitRows - 1) / kUnitRows, pieces, a.least, sh.split, u0, u1, whole)) return;
        if (whole) to.part_o = nullptr;
    } else {
        piece((sight.tile + kUnitRows - 1) / kUnitRows, a.n_split, a.least, sh.split, u0, u1);
    }
    if (to.part_o != nullptr && u0 == u1) return store_no_keys(to, sh.split, row, head, ok && lane < 32);
    SoftRow<P> soft;
    soft.clear();
    soft.load(static_cast<const T *>(a.q) + row * a.q_row + head * a.q_head, ok, lane);
    auto units = key_units<T>(a, sh.kv_head, k0, k_len, lds);
    auto rows = counted(a, k0, k_len);
    unsigned long long seen = 0;
    auto more = [&](int u) { rows.fetch(u, lane); };
    const UnitLanes at(lane);
    units.begin(u0, u1, more);
    for (int u = u0; u < u1; ++u) {
        bf16_t *k = units.step(u, u == u0, more, [&]() { return seen = rows.counts(); }, [](int) {});
        if constexpr (CAUSAL)
            if ((u + 1) * kUnitRows > sight.all && unit_is_wild(k + P * kPlane, lane)) {  // (all waves find the same)
                add_wild(soft.o, k + P * kPlane, sight.of(seen, u), lane);
                lds_barrier();
                tame_unit(k + P * kPlane, threadIdx.x);
                lds_barrier();
            }
        if (sight.sees(u)) soft.template unit<P, PP, CAUSAL>(k, k + P * kPlane, sight.of(seen, u), a.factor, at, lane);
    }
    store_soft<T>(soft, a.factor, to, sh.split, row, head, ok, lane);
}

// Probabilities of few bf16 rows enter in two parts, which the memory that binds hides (16 rows over 10992 keys of 16 heads 15.4 us with one,
// 16.0 with two): the error of out is the rounding of its store, also where few keys count (rows over 17 keys, up to 2.4e-3 with one).
template <typename T> constexpr int kFewParts = sizeof(T) == 4 ? 3 : 2;

// Few rows: WAVES waves with the same 16 rows take the units in turn, values through an LDS stage of their own (8 or 24 KiB).
template <typename T, int WAVES, bool CAUSAL> __global__ __launch_bounds__(64 * WAVES, sizeof(T) == 4 || WAVES > 4 ? 1 : 2) void cross_few_kernel(CrossArgs a)
{
    constexpr int P = UnitPairs<T>::kParts;
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    bf16_t *mine = reinterpret_cast<bf16_t *>(smem) + wave * P * kPlane;
    Share sh;
    if (!find_share(a.q_spans, nullptr, a.per_row, kFewRows, a.tiles, a.n_split, a.kv_heads, false, true, sh)) return;
    const int q0 = sh.of.first, q_len = sh.of.len;
    int k0, k_len;
    a.kv_spans.of(sh.of.seq, k0, k_len);
    const int64_t item = static_cast<int64_t>(sh.tile) * kFewRows + (lane & 15);
    const bool ok = item < static_cast<int64_t>(q_len) * a.per_row;
    const int64_t row = q0 + item / a.per_row;
    const int head = sh.kv_head * a.per_row + static_cast<int>(item % a.per_row);
    int sees = k_len, walked = k_len;
    if constexpr (CAUSAL) {
        walked = tile_sees(static_cast<int64_t>(sh.tile + 1) * kFewRows, static_cast<int64_t>(q_len) * a.per_row, a.per_row, q_len, k_len, a.view);
        sees = ok ? keys_seen(static_cast<int>(item) / a.per_row, q_len, k_len, a.view) : walked;
    }
    int u0, u1;
    piece((walked + kUnitRows - 1) / kUnitRows, a.n_split, a.least, sh.split, u0, u1);
    if (a.to.part_o != nullptr && u0 == u1) return store_no_keys(a.to, sh.split, row, head, ok && threadIdx.x < 16);
    FewRows<P> few;
    few.clear();
    few.load(static_cast<const T *>(a.q) + row * a.q_row + head * a.q_head, ok, lane);
    const T *keys = static_cast<const T *>(a.k) + k0 * a.kv_row + sh.kv_head * a.kv_head + 16 * (lane >> 4);
    RowUnits<T, 64> values(static_cast<const T *>(a.v) + k0 * a.kv_row + sh.kv_head * a.kv_head, k_len, a.kv_row, 0, 1, lane);
    auto rows = counted(a, k0, k_len);
    Io8<T> k[4][2];
    auto fetch = [&](int u) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int r = u * kUnitRows + 16 * t + (lane & 15);
            if (r < k_len) {
                k[t][0].load(keys + r * a.kv_row);
                k[t][1].load(keys + r * a.kv_row + 8);
            }
        }
        values.fetch(u, lane);
        rows.fetch(u, lane);
    };
    int u = u0 + wave;
    if (u < u1) fetch(u);
    for (; u < u1; u += WAVES) {
        const unsigned long long seen = rows.counts();
        values.put(mine, seen, lane);
        bf16x8 kk[4][2][P];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = k[t][s].get(j);
                split_parts<P>(x, kk[t][s]);
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (u + WAVES < u1) fetch(u + WAVES);
        few.template unit<P, kFewParts<T>, CAUSAL>([&](int t, int s, bf16x8(&to)[P]) {
#pragma unroll
            for (int i = 0; i < P; ++i) to[i] = kk[t][s][i];
        }, mine, CAUSAL ? seen & low_bits(sees - u * kUnitRows) : seen, a.factor, lane);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    __syncthreads();
    store_few<T, WAVES, CAUSAL>(few, a.factor, a.to, sh.split, row, head, ok, reinterpret_cast<float *>(smem), wave, lane);
}

// One result from the splits' normalised ones: weights 2^(lse_j - lse).  GROUPS x 16 threads for a row of a head: 16 take four
// channels each, the groups every GROUPS-th split.  With one group, the splits follow one another; with four (a wave for a row of a
// head), the log-sums of 64 splits are one load, and 64 splits' partial results are requested at once.  64 splits of 16 rows: 22.4 us
// with one group, 4.6 with four; 13 splits of 22 thousand rows 16 with one, 19 with four.
constexpr int kSplitChunks = kMostSplits / 64;
constexpr int kJoinAtOnce = 4;  // pieces whose loads are under way together where a thread goes through them
template <typename T, int GROUPS, bool CAUSAL> __device__ __forceinline__ void soft_combine(const SoftOut &to, int64_t row, int64_t at, int n_split)
{
    const int64_t share = to.rows * to.heads;
    const int c = static_cast<int>(threadIdx.x & 15) * 4, group = static_cast<int>(threadIdx.x >> 4) % GROUPS, lane = threadIdx.x & 63;
    float top = -INFINITY, total = 0.f;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    auto weight = [&](float l) { return l == -INFINITY ? 0.f : (l == top ? 1.f : (CAUSAL ? held_weight(l - top) : fast_exp2(l - top))); };  // -inf: no keys in the piece
    auto add = [&](float l, const floatx4 &o) {
        const float w = weight(l);
        total += w;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += l == -INFINITY ? 0.f : w * o[e];  // a piece without keys left no result
    };
    if constexpr (GROUPS == 4) {
        float l[kSplitChunks];
#pragma unroll
        for (int k = 0; k < kSplitChunks; ++k) l[k] = 64 * k + lane < n_split ? to.part_lse[(64 * k + lane) * share + at] : -INFINITY;
#pragma unroll
        for (int k = 0; k < kSplitChunks; ++k) top = fmaxf(top, l[k]);
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m, 64));
#pragma unroll
        for (int k = 0; k < kSplitChunks; ++k) {
            if (64 * k >= n_split) break;
            floatx4 o[16];
#pragma unroll
            for (int s = 0; s < 16; ++s) {
                const int j = 64 * k + 4 * s + group;
                if (64 * k + 4 * s < n_split) o[s] = *reinterpret_cast<const floatx4 *>(to.part_o + ((j < n_split ? j : 0) * share + at) * 64 + c);
            }
#pragma unroll
            for (int s = 0; s < 16; ++s)
                if (64 * k + 4 * s < n_split) add(__shfl(l[k], 4 * s + group, 64), o[s]);
        }
#pragma unroll
        for (int m = 16; m < 64; m <<= 1) {
            total += __shfl_xor(total, m, 64);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], m, 64);
        }
        if (group != 0) return;
    } else {
        for (int j0 = 0; j0 < n_split; j0 += kJoinAtOnce) {
            float l[kJoinAtOnce];
#pragma unroll
            for (int k = 0; k < kJoinAtOnce; ++k) l[k] = to.part_lse[min(j0 + k, n_split - 1) * share + at];
#pragma unroll
            for (int k = 0; k < kJoinAtOnce; ++k) top = fmaxf(top, l[k]);
        }
        for (int j0 = 0; j0 < n_split; j0 += kJoinAtOnce) {
            float l[kJoinAtOnce];
            floatx4 o[kJoinAtOnce];
#pragma unroll
            for (int k = 0; k < kJoinAtOnce; ++k) {
                const int64_t from = min(j0 + k, n_split - 1) * share + at;
                l[k] = to.part_lse[from];
                o[k] = *reinterpret_cast<const floatx4 *>(to.part_o + from * 64 + c);
            }
#pragma unroll
            for (int k = 0; k < kJoinAtOnce; ++k)
                if (j0 + k < n_split && l[k] != -INFINITY) add(l[k], o[k]);
        }
    }
    const float w = total == 0.f ? 0.f : 1.f / total;
    T *dst = static_cast<T *>(to.out) + at * 64 + c;
#pragma unroll
    for (int e = 0; e < 4; ++e) dst[e] = from_float<T>(acc[e] * w);
    if (c == 0 && to.lse != nullptr)
        to.lse[(at - row * to.heads) * to.rows + row] = total == 0.f ? -INFINITY : (top + log2f(total)) * kLn2;
}

template <typename T, int GROUPS, bool CAUSAL> __global__ __launch_bounds__(256) void soft_combine_kernel(SoftOut to, Spans spans, int n_split)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, at = i / (16 * GROUPS);
    if (at >= to.rows * to.heads) return;
    const int64_t row = at / to.heads;
    if (spans.covers(row)) soft_combine<T, GROUPS, CAUSAL>(to, row, at, n_split);
}

// What causal tiles left in pieces is joined tile by tile: kItems items of a tile of kTile for a workgroup, which is done at once where the
// tile had one piece.  (A thread that looks for its row's sequence by itself takes 15 us for 8192 rows of 16 heads that have nothing to join.)
struct TileItems { Share of; int item0; };
__device__ __forceinline__ bool find_items(const Spans &spans, int per_row, int kv_heads, int items, TileItems &t)
{
    const unsigned chunks = kTile / items, th = blockIdx.x / chunks;
    t.item0 = static_cast<int>(blockIdx.x - th * chunks) * items;
    t.of.kv_head = static_cast<int>(th % static_cast<unsigned>(kv_heads));
    return find_tile(spans, nullptr, per_row, kTile, th / static_cast<unsigned>(kv_heads), t.of.of, t.of.tile);
}

template <int GROUPS> constexpr int kJoinItems = GROUPS == 4 ? 4 : 32;
template <typename T, int GROUPS> __global__ __launch_bounds__(256) void causal_combine_kernel(CrossArgs a)
{
    constexpr int kItems = kJoinItems<GROUPS>;
    TileItems t;
    if (!find_items(a.q_spans, a.per_row, a.kv_heads, kItems, t)) return;
    int k0, k_len;
    a.kv_spans.of(t.of.of.seq, k0, k_len);
    const int64_t items = static_cast<int64_t>(t.of.of.len) * a.per_row, tile0 = static_cast<int64_t>(t.of.tile) * kTile;
    const int n = causal_pieces((tile_sees(tile0 + kTile, items, a.per_row, t.of.of.len, k_len, a.view) + kUnitRows - 1) / kUnitRows, causal_split<false>(a), a.least);
    if (n == 1) return;
    for (int i = threadIdx.x / (16 * GROUPS); i < kItems; i += 256 / (16 * GROUPS)) {
        const int64_t item = tile0 + t.item0 + i, in_seq = item / a.per_row, row = t.of.of.first + in_seq;
        if (item < items) soft_combine<T, GROUPS, true>(a.to, row, row * a.heads + t.of.kv_head * a.per_row + (item - in_seq * a.per_row), n);
    }
}

// ---- gradient --------------------------------------------------------------------------------------------

// D from the stored out: in bf16 it is off by the rounding of out, the same amount for all keys of a row, and that would be most of the
// error of dq and dk.  The dS of a row add up to 0 over all keys: what they do add up to in fp32 is what D lacks, and goes into D for the
// gradient of keys.  What they add up to as they enter the product, rounded, has the roundings in it as well; the query gradient takes that
// out of its own result, dS k - sum(dS) * P k.  One product more of four.  Against 64 bits, 2748 rows over 10992 keys of which a few channels
// are large: dq 4.0e-3 without, 2.2e-3 so, dk 2.7e-3 and 2.3e-3; 300 normal rows over 700 keys dq 2.8e-3 and 2.2e-3, dk 2.5e-3 and 2.3e-3.  The
// kernel of 2748 rows, 16 heads: 208 us without, 281 so.
template <typename T> constexpr bool kMendD = sizeof(T) == 2;

__device__ __forceinline__ float sum8(const bf16x8 &x)
{
    const bf16x2 one = {static_cast<bf16_t>(1.f), static_cast<bf16_t>(1.f)};
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; i += 2) s = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{x[i], x[i + 1]}, one, s, false);
    return s;
}

// PX: bf16 parts in which dS enters its product.
template <typename T, int PX, bool CAUSAL> __global__ __launch_bounds__(256, sizeof(T) == 4 ? 1 : 2) void grad_q_kernel(CrossArgs a)
{
    constexpr int P = UnitPairs<T>::kParts;
    extern __shared__ __align__(16) unsigned char smem[];
    bf16_t *lds = reinterpret_cast<bf16_t *>(smem);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Share sh;
    int pieces;  // causal: of a tile, at most
    if constexpr (CAUSAL) {
        pieces = causal_split<false>(a);
        if (!find_causal_share<false>(a, pieces, sh)) return;
    } else {
        if (!find_share(a.q_spans, nullptr, a.per_row, kTile, a.tiles, a.n_split, a.kv_heads, !a.uneven, true, sh)) return;
    }
    const int q0 = sh.of.first, q_len = sh.of.len;
    int k0, k_len;
    a.kv_spans.of(sh.of.seq, k0, k_len);
    const int64_t item = static_cast<int64_t>(sh.tile) * kTile + 32 * wave + (lane & 31);
    const bool ok = item < static_cast<int64_t>(q_len) * a.per_row;
    const int64_t row = q0 + item / a.per_row;
    const int head = sh.kv_head * a.per_row + static_cast<int>(item % a.per_row);
    const CausalTile<CAUSAL> sight(a, sh.tile, q_len, k_len, item, ok, wave);
    int u0, u1;
    float *part_q = a.part_q;
    if constexpr (CAUSAL) {
        bool whole;
        if (!causal_piece((sight.tile + kUnitRows - 1) / kUnitRows, pieces, a.least, sh.split, u0, u1, whole)) return;
        if (whole) part_q = nullptr;
    } else {
        piece((sight.tile + kUnitRows - 1) / kUnitRows, a.n_split, a.least, sh.split, u0, u1);
    }
    if (sh.split > 0 && u0 == u1) return;
    SoftRow<P> held, grad;  // q, and d_out; held.o: P k, grad.o: the gradient
    held.clear();
    held.load(static_cast<const T *>(a.q) + row * a.q_row + head * a.q_head, ok, lane);
    grad.clear();
    grad.load(static_cast<const T *>(a.d_out) + (row * a.heads + head) * 64, ok, lane);
    // What the gradient of keys needs of the row as well: its log-sum, in log2 (+inf where it saw no keys, so that every probability is
    // 0), and -D, D = out . d_out.
    float l2 = INFINITY, d = 0.f, sum = 0.f, entered = 0.f;  // d: -D
    float *stats = a.stats + 2 * (head * a.n_q + row);
    if (ok) {
        const T *o = static_cast<const T *>(a.to.out) + (row * a.heads + head) * 64, *g = static_cast<const T *>(a.d_out) + (row * a.heads + head) * 64;
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            float x[8], y[8];
            load8(o + 16 * s + 8 * (lane >> 5), x);
            load8(g + 16 * s + 8 * (lane >> 5), y);
#pragma unroll
            for (int j = 0; j < 8; ++j) d = fmaf(-x[j], y[j], d);
        }
        const float l = a.to.lse[head * a.n_q + row];
        l2 = l == -INFINITY ? INFINITY : l * kLog2e;
    }
    d = sum_with_other_half(d);
    if (ok && lane < 32 && sh.split == 0) { stats[0] = l2; stats[1] = d; }
    auto units = key_units<T>(a, sh.kv_head, k0, k_len, lds);
    auto rows = counted(a, k0, k_len);
    unsigned long long seen = 0;
    auto more = [&](int u) { rows.fetch(u, lane); };
    const UnitLanes at(lane);
    floatx16 minus_d;
#pragma unroll
    for (int r = 0; r < 16; ++r) minus_d[r] = d;
    asm volatile("" : "+v"(minus_d));  // sixteen registers to start from, and not a move for each of them in every product
    units.begin(u0, u1, more);
    for (int u = u0; u < u1; ++u) {
        const bf16_t *k = units.step(u, u == u0, more, [&]() { return seen = rows.counts(); }, [](int) {}), *v = k + P * kPlane;
        if (!sight.sees(u)) continue;
        seen = sight.of(seen, u);
        const bool some = CAUSAL ? __any(seen != ~0ull) : seen != ~0ull, wild = CAUSAL && some && unit_is_wild(k, lane);
        // dP - D comes out of the product itself where it starts at -D
        RowOperands<P> kr, vr;
        kr.read(k, 0, at);
        vr.read(v, 0, at);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            floatx16 s = {}, dp = minus_d;
            each_part<P, P, 4>([&](int step, int i, int j) {
                s = mfma(kr.x[step][i], held.q[step][j], s);
                dp = mfma(vr.x[step][i], grad.q[step][j], dp);
            });
            if (half == 0) {
                kr.read(k, 1, at);
                vr.read(v, 1, at);
            }
            ChannelOperands<P> kt;
            kt.read(k, half, at);
            if (CAUSAL && wild) kt.tame_all();
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[r] = fast_exp2(fmaf(s[r], a.factor, -l2));
                dp[r] *= s[r];
            }
            if (some) {
                const uint32_t out = left_out(seen, half, lane);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[r] = replace(s[r], 0.f, left_out_mask(out, r));
                    dp[r] = replace(dp[r], 0.f, left_out_mask(out, r));
                }
            }
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                float x[8], y[8], add[2] = {0.f, 0.f};
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    y[j] = s[8 * w + j];
                    x[j] = dp[8 * w + j];
                    if constexpr (kMendD<T>) add[j & 1] += x[j];
                }
                bf16x8 ds[PX], p[P];
                split_parts<PX>(x, ds);
                if constexpr (kMendD<T>) {
                    split_parts<P>(y, p);
                    sum += add[0] + add[1];
                    entered += sum8(ds[0]);
                    if constexpr (PX == 2) entered += sum8(ds[1]);
                }
#pragma unroll
                for (int dt = 0; dt < 2; ++dt) {
                    multiply<P>(grad.o[dt], ds, [&](int part) { return kt.x[w][dt][part]; });
                    if constexpr (kMendD<T>) multiply<P>(held.o[dt], p, [&](int part) { return kt.x[w][dt][part]; });
                }
            }
        }
        if (CAUSAL && wild) add_wild(grad.o, k, seen, lane);
    }
    const int64_t to = row * a.heads + head, part = sh.split * a.n_q * a.heads + to;
    if constexpr (kMendD<T>) {
        sum = sum_with_other_half(sum);
        entered = sum_with_other_half(entered);
        if (part_q == nullptr) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                grad.o[0][r] -= entered * held.o[0][r];
                grad.o[1][r] -= entered * held.o[1][r];
            }
            if (ok && lane < 32) stats[1] = d - sum;
        } else {
            store_row(held.o, 1.f, a.part_pk + part * 64, ok, lane);
            if (ok && lane < 32) { a.part_sum[2 * part] = sum; a.part_sum[2 * part + 1] = entered; }
        }
    }
    if (part_q != nullptr)
        store_row(grad.o, 1.f, part_q + part * 64, ok, lane);
    else
        store_row(grad.o, a.scale, static_cast<T *>(a.dq) + to * 64, ok, lane);
}

// Pieces that a sequence's streamed rows (items: rows * per_row) were divided into.
__device__ __forceinline__ int pieces_of(const Spans &streamed, int seq, int per_row, const CrossArgs &a)
{
    int first, len;
    streamed.of(seq, first, len);
    const int units = (len * per_row + kUnitRows - 1) / kUnitRows, per = piece_units(units, a.n_split, a.least);
    return (units + per - 1) / per;
}

// The query gradient from its pieces over keys.  16 threads for a row of a head.
template <typename T> __device__ __forceinline__ void grad_q_combine(const CrossArgs &a, int64_t row, int64_t at, int n)
{
    const int64_t share = a.n_q * a.heads;
    const int c = static_cast<int>(threadIdx.x & 15) * 4;
    floatx4 g = {0.f, 0.f, 0.f, 0.f}, pk = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f, entered = 0.f;
    for (int j0 = 0; j0 < n; j0 += kJoinAtOnce) {
        floatx4 q[kJoinAtOnce], p[kJoinAtOnce];
        float s[kJoinAtOnce][2];
#pragma unroll
        for (int k = 0; k < kJoinAtOnce; ++k) {
            const int64_t from = min(j0 + k, n - 1) * share + at;
            q[k] = *reinterpret_cast<const floatx4 *>(a.part_q + from * 64 + c);
            if constexpr (kMendD<T>) {
                p[k] = *reinterpret_cast<const floatx4 *>(a.part_pk + from * 64 + c);
                s[k][0] = a.part_sum[2 * from];
                s[k][1] = a.part_sum[2 * from + 1];
            }
        }
#pragma unroll
        for (int k = 0; k < kJoinAtOnce; ++k) {
            if (j0 + k >= n) break;
            g += q[k];
            if constexpr (kMendD<T>) {
                pk += p[k];
                sum += s[k][0];
                entered += s[k][1];
            }
        }
    }
    T *dst = static_cast<T *>(a.dq) + at * 64 + c;
#pragma unroll
    for (int e = 0; e < 4; ++e) dst[e] = from_float<T>(a.scale * (g[e] - entered * pk[e]));
    if (kMendD<T> && c == 0) a.stats[2 * ((at - row * a.heads) * a.n_q + row) + 1] -= sum;
}
template <typename T> __global__ __launch_bounds__(256) void grad_q_combine_kernel(CrossArgs a)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, at = i >> 4;
    if (at >= a.n_q * a.heads) return;
    const int64_t row = at / a.heads;
    if (a.q_spans.covers(row)) grad_q_combine<T>(a, row, at, pieces_of(a.kv_spans, a.q_spans.find(row), 1, a));
}
template <typename T> __global__ __launch_bounds__(256) void causal_grad_q_combine_kernel(CrossArgs a)
{
    TileItems t;
    if (!find_items(a.q_spans, a.per_row, a.kv_heads, kJoinItems<1>, t)) return;
    int k0, k_len;
    a.kv_spans.of(t.of.of.seq, k0, k_len);
    const int64_t items = static_cast<int64_t>(t.of.of.len) * a.per_row, tile0 = static_cast<int64_t>(t.of.tile) * kTile;
    const int n = causal_pieces((tile_sees(tile0 + kTile, items, a.per_row, t.of.of.len, k_len, a.view) + kUnitRows - 1) / kUnitRows, causal_split<false>(a), a.least);
    if (n == 1) return;
    for (int i = threadIdx.x / 16; i < kJoinItems<1>; i += 16) {
        const int64_t item = tile0 + t.item0 + i, in_seq = item / a.per_row, row = t.of.of.first + in_seq;
        if (item < items) grad_q_combine<T>(a, row, row * a.heads + t.of.kv_head * a.per_row + (item - in_seq * a.per_row), n);
    }
}

// Few rows: probabilities and dS rounded to bf16 would be most of the error of dk and dv, whose sums have few terms, and now and then of
// dq, where a few dS count (2.4e-3 to 2.9e-3, against 1.66e-3 by the rounding of the results themselves, which is what two parts leave).
// With many rows the errors are 2.35e-3 and 2.3e-3 and no memory hides the products.  Gradient of 16 heads in bf16, us, one part / two: 1 row over 10992
// keys 55 / 60, 64 over 2000 24.8 / 26.6, 2748 over 10992 588 / 795, 8192 over 8192 1129 / 1554; dk and dv alone: 128 over 10992 71 / 80, 512 over
// 10992 137 / 163.
// CAUSAL: of many rows, too, the last keys are seen by few, and so the last tile of a sequence takes its last kFewItems items in two parts (errors of the last 16 keys
// of 2048 2.9e-3 with one, 1.7e-3 so; forward and gradients, 17 sequences of 60 rows over 500 keys 66.7 / 68.7 us, 8192 rows in three 364 / 365).
// All rows in two parts where the caller asks for it: causal, 10992 rows in views of 1374 1136 / 1527, 8192 by token 585 / 788, in three prompts 278 / 351.
constexpr int kFewItems = kUnitRows;
template <int N> struct Parts { static constexpr int value = N; };

// PX: bf16 parts in which probabilities and dS enter the products.
template <typename T, int PX, bool CAUSAL> __global__ __launch_bounds__(256, sizeof(T) == 4 ? 1 : 2) void grad_kv_kernel(CrossArgs a)
{
    constexpr int P = UnitPairs<T>::kParts;
    extern __shared__ __align__(16) unsigned char smem[];
    bf16_t *lds = reinterpret_cast<bf16_t *>(smem);
    float *row_stats = reinterpret_cast<float *>(smem + sizeof(bf16_t) * UnitPairs<T>::kStages * UnitPairs<T>::kStage);  // [stages][2][64]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Share sh;
    int pieces;  // causal: of a tile, at most
    if constexpr (CAUSAL) {
        pieces = causal_split<true>(a);
        if (!find_causal_share<true>(a, pieces, sh)) return;
    } else {
        if (!find_share(a.kv_spans, nullptr, 1, kTile, a.tiles, a.n_split, a.kv_heads, !a.uneven, true, sh)) return;
    }
    const int k0 = sh.of.first, k_len = sh.of.len;
    int q0, q_len;
    a.q_spans.of(sh.of.seq, q0, q_len);
    const int key = sh.tile * kTile + 32 * wave + (lane & 31);
    const bool ok = key < k_len, seen = ok && (a.key_mask == nullptr || a.key_mask[k0 + key] != 0);
    const int64_t row = k0 + key;
    const int items = q_len * a.per_row, head0 = sh.kv_head * a.per_row;
    float *part_k = a.part_k;
    int u0, u1, from = 0, wave_from = 0;  // causal: the first item that sees the lane's key, and the wave's first
    int two_from = 0x7fffffff;            // units from here on enter in two parts
    if constexpr (CAUSAL) {
        int begin, end;
        seeing_units(a, sh.tile, q_len, k_len, begin, end);
        bool whole;
        if (!causal_piece(end - begin, pieces, a.least, sh.split, u0, u1, whole)) return;
        if (whole) part_k = nullptr;
        u0 += begin;
        u1 += begin;
        from = first_seer(key, q_len, k_len, a.view) * a.per_row;
        wave_from = __builtin_amdgcn_readfirstlane(from);
        const int few = max(0, items - kFewItems);
        if (PX == 1 && first_seer(min(k_len, (sh.tile + 1) * kTile) - 1, q_len, k_len, a.view) * a.per_row >= few) two_from = few / kUnitRows;
    } else {
        piece((items + kUnitRows - 1) / kUnitRows, a.n_split, a.least, sh.split, u0, u1);
    }
    if (sh.split > 0 && u0 == u1) return;
    SoftRow<P> kk, vv;  // k and v; .o: their gradients
    kk.clear();
    vv.clear();
    kk.load(static_cast<const T *>(a.k) + row * a.kv_row + sh.kv_head * a.kv_head, seen, lane);
    vv.load(static_cast<const T *>(a.v) + row * a.kv_row + sh.kv_head * a.kv_head, seen, lane);

    UnitPairs<T, true> units(static_cast<const T *>(a.q) + q0 * a.q_row + head0 * a.q_head,
                             static_cast<const T *>(a.d_out) + (static_cast<int64_t>(q0) * a.heads + head0) * 64, items, a.q_row, a.q_head,
                             static_cast<int64_t>(a.heads) * 64, 64, a.per_row, lds);
    float st = 0.f;
    const int which = threadIdx.x >> 6;  // threads 0 .. 63 bring the rows' log-sums, 64 .. 127 their D
    auto more = [&](int u) {
        const int r = u * kUnitRows + lane;
        st = which == 0 ? INFINITY : 0.f;
        if (which < 2 && r < items) {
            const int i = r / a.per_row;
            st = a.stats[2 * ((head0 + r - i * a.per_row) * a.n_q + q0 + i) + which];
        }
    };
    const UnitLanes at(lane);
    units.begin(u0, u1, more);
    const float *stats = row_stats;
    auto walk = [&](auto parts, int u) {
        constexpr int kParts = parts.value;
        const bf16_t *q = units.step(u, u == u0, more, [&]() { return low_bits(items - u * kUnitRows); }, [&](int stage) {
            float *to = row_stats + stage * 128;
            if (which < 2) to[which * 64 + lane] = st;
            stats = to;
        }), *g = q + P * kPlane;
        unsigned long long items_seen = ~0ull;
        bool some = false, wild = false;
        if constexpr (CAUSAL) {
            if ((u + 1) * kUnitRows <= wave_from) return;
            items_seen = ~low_bits(from - u * kUnitRows);
            some = __any(items_seen != ~0ull);
            wild = some && (unit_is_wild(q, lane) || unit_is_wild(g, lane));
        }
        RowOperands<P> qr, gr;
        qr.read(q, 0, at);
        gr.read(g, 0, at);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            floatx16 s = {}, dp;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const floatx4 d = *reinterpret_cast<const floatx4 *>(stats + 64 + 32 * half + 8 * b + 4 * (lane >> 5));
#pragma unroll
                for (int e = 0; e < 4; ++e) dp[4 * b + e] = d[e];
            }
            each_part<P, P, 4>([&](int step, int i, int j) {
                s = mfma(qr.x[step][i], kk.q[step][j], s);
                dp = mfma(gr.x[step][i], vv.q[step][j], dp);
            });
            if (half == 0) {
                qr.read(q, 1, at);
                gr.read(g, 1, at);
            }
            ChannelOperands<P> qt, gt;
            gt.read(g, half, at);
            qt.read(q, half, at);
            if (CAUSAL && wild) {
                gt.tame_all();
                qt.tame_all();
            }
            const uint32_t out = CAUSAL && some ? left_out(items_seen, half, lane) : 0u;
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                float x[8], y[8];
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int r0 = 32 * half + 16 * w + 8 * b + 4 * (lane >> 5);
                    const floatx4 l2 = *reinterpret_cast<const floatx4 *>(stats + r0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int r = 8 * w + 4 * b + e;
                        x[4 * b + e] = fast_exp2(fmaf(s[r], a.factor, -l2[e]));
                        y[4 * b + e] = x[4 * b + e] * dp[r];
                    }
                }
                if (CAUSAL && some)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        x[j] = replace(x[j], 0.f, left_out_mask(out, 8 * w + j));
                        y[j] = replace(y[j], 0.f, left_out_mask(out, 8 * w + j));
                    }
                bf16x8 p[kParts], ds[kParts];
                split_parts<kParts>(x, p);
                split_parts<kParts>(y, ds);
#pragma unroll
                for (int dt = 0; dt < 2; ++dt) {
                    multiply<P>(vv.o[dt], p, [&](int part) { return gt.x[w][dt][part]; });
                    multiply<P>(kk.o[dt], ds, [&](int part) { return qt.x[w][dt][part]; });
                }
            }
        }
        if (CAUSAL && wild) {
            add_wild(vv.o, g, items_seen, lane);
            add_wild(kk.o, q, items_seen, lane);
            add_wild(kk.o, g, items_seen, lane);
        }
    };
    int u = u0;
    for (const int to = min(u1, two_from); u < to; ++u) walk(Parts<PX>(), u);
    if constexpr (CAUSAL && PX == 1)
        for (; u < u1; ++u) walk(Parts<2>(), u);
    if (!seen)  // a masked key gets no gradient, whatever its lanes added up
#pragma unroll
        for (int r = 0; r < 16; ++r) kk.o[0][r] = kk.o[1][r] = vv.o[0][r] = vv.o[1][r] = 0.f;
    const int64_t to = (row * a.kv_heads + sh.kv_head) * 64, share = a.n_kv * a.kv_heads * 64;
    if (part_k != nullptr) {
        store_row(kk.o, a.scale, part_k + sh.split * share + to, ok, lane);
        store_row(vv.o, 1.f, a.part_v + sh.split * share + to, ok, lane);
    } else {
        store_row(kk.o, a.scale, static_cast<T *>(a.dk) + to, ok, lane);
        store_row(vv.o, 1.f, static_cast<T *>(a.dv) + to, ok, lane);
    }
}

// dk and dv as the sums of their pieces over queries.  16 threads for a row of a head; blockIdx.y: dk or dv.
template <typename T> __device__ __forceinline__ void grad_kv_combine(const CrossArgs &a, int64_t i, int pieces)
{
    const int64_t n = a.n_kv * a.kv_heads * 16;
    const float *part = blockIdx.y == 0 ? a.part_k : a.part_v;
    T *out = static_cast<T *>(blockIdx.y == 0 ? a.dk : a.dv);
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int j0 = 0; j0 < pieces; j0 += kJoinAtOnce) {
        floatx4 x[kJoinAtOnce];
#pragma unroll
        for (int k = 0; k < kJoinAtOnce; ++k) x[k] = *reinterpret_cast<const floatx4 *>(part + (min(j0 + k, pieces - 1) * n + i) * 4);
#pragma unroll
        for (int k = 0; k < kJoinAtOnce; ++k)
            if (j0 + k < pieces) acc += x[k];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) out[i * 4 + e] = from_float<T>(acc[e]);
}
template <typename T> __global__ __launch_bounds__(256) void grad_kv_combine_kernel(CrossArgs a)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, n = a.n_kv * a.kv_heads * 16;
    if (i >= n || !a.kv_spans.covers(i / (a.kv_heads * 16))) return;
    grad_kv_combine<T>(a, i, pieces_of(a.q_spans, a.kv_spans.find(i / (a.kv_heads * 16)), a.per_row, a));
}
template <typename T> __global__ __launch_bounds__(256) void causal_grad_kv_combine_kernel(CrossArgs a)
{
    TileItems t;
    if (!find_items(a.kv_spans, 1, a.kv_heads, kJoinItems<1>, t)) return;
    int q0, q_len, from, end;
    a.q_spans.of(t.of.of.seq, q0, q_len);
    seeing_units(a, t.of.tile, q_len, t.of.of.len, from, end);
    const int n = causal_pieces(end - from, causal_split<true>(a), a.least);
    if (n == 1) return;
    for (int i = threadIdx.x / 16; i < kJoinItems<1>; i += 16) {
        const int key = t.of.tile * kTile + t.item0 + i;
        if (key < t.of.of.len) grad_kv_combine<T>(a, ((static_cast<int64_t>(t.of.of.first) + key) * a.kv_heads + t.of.kv_head) * 16 + (threadIdx.x & 15), n);
    }
}

// Faults of the lists a call was given, as bits of *status.  One workgroup.
__global__ __launch_bounds__(1024) void span_status_kernel(Spans q, Spans kv, int *status)
{
    const int bad = __syncthreads_or(spans_bad(q) || spans_bad(kv));
    if (threadIdx.x == 0) *status = bad ? kDiagSpans : 0;
}

template <typename T, int WAVES> hipError_t launch_few(const CrossArgs &a, int64_t n, hipStream_t stream)
{
    constexpr size_t kLds = WAVES * UnitPairs<T>::kParts * kPlane * sizeof(bf16_t);
    auto kernel = a.view > 0 ? &cross_few_kernel<T, WAVES, true> : &cross_few_kernel<T, WAVES, false>;
    const hipError_t e = allow_lds(kernel, kLds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(n)), dim3(64 * WAVES), kLds, stream, a);
    return hipGetLastError();
}

template <typename T, int PP> auto cross_kernel_of(bool causal) { return causal ? &cross_kernel<T, PP, true> : &cross_kernel<T, PP, false>; }

template <typename T> hipError_t launch_cross_t(const CrossArgs &a, bool few_rows, hipStream_t stream)
{
    const int64_t shares = a.tiles * a.n_split * a.kv_heads, n = few_rows ? shares : xcd_padded(shares);
    if (!grid_ok(few_rows ? 2 * n : n)) return hipErrorInvalidValue;  // (up to 512 threads)
    if (few_rows) {
        if constexpr (sizeof(T) == 2)
            if (a.n_split == 1) return launch_few<T, 8>(a, n, stream);
        return launch_few<T, 4>(a, n, stream);
    } else {
        constexpr size_t kLds = UnitPairs<T>::kStages * UnitPairs<T>::kStage * sizeof(bf16_t);
        auto kernel = cross_kernel_of<T, UnitPairs<T>::kParts>(a.view > 0);
        if constexpr (sizeof(T) == 2)
            if (a.accurate) kernel = cross_kernel_of<T, 2>(a.view > 0);
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(n)), dim3(256), kLds, stream, a);
    }
    return hipGetLastError();
}

template <typename T, int PX> auto grad_kernel(bool of_keys, bool causal)
{
    return of_keys ? (causal ? &grad_kv_kernel<T, PX, true> : &grad_kv_kernel<T, PX, false>)
                   : (causal ? &grad_q_kernel<T, PX, true> : &grad_q_kernel<T, PX, false>);
}
template <typename T> hipError_t launch_grad_t(const CrossArgs &a, bool of_keys, hipStream_t stream)
{
    const int64_t n = xcd_padded(a.tiles * a.n_split * a.kv_heads);
    if (!grid_ok(n)) return hipErrorInvalidValue;
    const size_t lds = UnitPairs<T>::kStages * (UnitPairs<T>::kStage * sizeof(bf16_t) + (of_keys ? 128 * sizeof(float) : 0));
    auto kernel = grad_kernel<T, UnitPairs<T>::kParts>(of_keys, a.view > 0);
    if constexpr (sizeof(T) == 2)
        if (a.accurate || a.n_q * a.per_row <= kFewItems * a.q_spans.batch) kernel = grad_kernel<T, 2>(of_keys, a.view > 0);
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(n)), dim3(256), lds, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cross(const CrossArgs &a, bool few_rows, bool is_bf16, hipStream_t stream)
{
    return is_bf16 ? launch_cross_t<bf16_t>(a, few_rows, stream) : launch_cross_t<float>(a, few_rows, stream);
}

hipError_t launch_grad_q(const CrossArgs &a, bool is_bf16, hipStream_t stream)
{
    return is_bf16 ? launch_grad_t<bf16_t>(a, false, stream) : launch_grad_t<float>(a, false, stream);
}

// Workgroups that join what causal tiles left in pieces.
int64_t join_blocks(const CrossArgs &a, int items) { return a.tiles * a.kv_heads * (kTile / items); }

hipError_t launch_grad_q_combine(const CrossArgs &a, bool is_bf16, hipStream_t stream)
{
    const bool causal = a.view > 0;
    const int64_t blocks = causal ? join_blocks(a, kJoinItems<1>) : (a.n_q * a.heads * 16 + 255) / 256;
    if (!grid_ok(blocks)) return hipErrorInvalidValue;
    auto kernel = is_bf16 ? (causal ? &causal_grad_q_combine_kernel<bf16_t> : &grad_q_combine_kernel<bf16_t>)
                          : (causal ? &causal_grad_q_combine_kernel<float> : &grad_q_combine_kernel<float>);
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_grad_kv(const CrossArgs &a, bool is_bf16, hipStream_t stream)
{
    return is_bf16 ? launch_grad_t<bf16_t>(a, true, stream) : launch_grad_t<float>(a, true, stream);
}

template <int GROUPS, bool CAUSAL> auto soft_combine_of(bool is_bf16) { return is_bf16 ? &soft_combine_kernel<bf16_t, GROUPS, CAUSAL> : &soft_combine_kernel<float, GROUPS, CAUSAL>; }

hipError_t launch_soft_combine(const SoftOut &to, const Spans &spans, int n_split, bool causal, bool is_bf16, hipStream_t stream)
{
    // (us, wide or not: 5 splits of 4800 rows 17.7 / 19.2 with the attention, 4 of 8192 23.5 / 21.6, 10 of 2048 15.7 / 20.0, 6 of 256 9.8 / 12.8,
    // 2 of 16 9.0 / 8.5)
    const int64_t share = to.rows * to.heads;
    const bool wide = n_split >= 3 && share <= 1024 * (n_split < 8 ? n_split : 8);
    const int64_t blocks = (share * (wide ? 64 : 16) + 255) / 256;
    if (!grid_ok(blocks) || n_split > kMostSplits) return hipErrorInvalidValue;
    auto kernel = causal ? (wide ? soft_combine_of<4, true>(is_bf16) : soft_combine_of<1, true>(is_bf16))
                         : (wide ? soft_combine_of<4, false>(is_bf16) : soft_combine_of<1, false>(is_bf16));
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, to, spans, n_split);
    return hipGetLastError();
}

hipError_t launch_causal_combine(const CrossArgs &a, bool is_bf16, hipStream_t stream)
{
    const int64_t share = a.to.rows * a.to.heads;
    const bool wide = a.n_split >= 3 && share <= 1024 * (a.n_split < 8 ? a.n_split : 8);  // as above
    const int64_t blocks = join_blocks(a, wide ? kJoinItems<4> : kJoinItems<1>);
    if (!grid_ok(blocks) || a.n_split > kMostSplits) return hipErrorInvalidValue;
    auto kernel = is_bf16 ? (wide ? &causal_combine_kernel<bf16_t, 4> : &causal_combine_kernel<bf16_t, 1>)
                          : (wide ? &causal_combine_kernel<float, 4> : &causal_combine_kernel<float, 1>);
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_grad_kv_combine(const CrossArgs &a, bool is_bf16, hipStream_t stream)
{
    const bool causal = a.view > 0;
    const int64_t blocks = causal ? join_blocks(a, kJoinItems<1>) : (a.n_kv * a.kv_heads * 16 + 255) / 256;
    if (!grid_ok(2 * blocks)) return hipErrorInvalidValue;
    auto kernel = is_bf16 ? (causal ? &causal_grad_kv_combine_kernel<bf16_t> : &grad_kv_combine_kernel<bf16_t>)
                          : (causal ? &causal_grad_kv_combine_kernel<float> : &grad_kv_combine_kernel<float>);
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks), 2), dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_span_status(const Spans &q, const Spans &kv, int *status, hipStream_t stream)
{
    hipLaunchKernelGGL(span_status_kernel, dim3(1), dim3(1024), 0, stream, q, kv, status);
    return hipGetLastError();
}

}  // namespace s3r
