// Cross attention, out[i] = sum_j softmax_j(scale q_i . k_j) v_j, with keys of another length than the queries, and its gradient
//   P = exp(scale q k^T - lse),  D_i = out_i . d_out_i,  dS = scale P (d_out v^T - D),
//   dq = dS k,  dk = dS^T q,  dv = P^T d_out.
// Batches of ragged sequences lie one behind the other; several query heads may share a head of keys: their rows are then
// items of one tile, and the gradient of the shared head is one sum over all of them.  No atomics: a sum that is split over workgroups
// goes through partial results in the workspace, which another launch adds up in a fixed order.
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

// Many rows: four waves hold 32 rows each and share every unit.
template <typename T> __global__ __launch_bounds__(256, sizeof(T) == 4 ? 2 : 4) void cross_kernel(CrossArgs a)
{
    constexpr int P = UnitPairs<T>::kParts;
    extern __shared__ __align__(16) unsigned char smem[];
    bf16_t *lds = reinterpret_cast<bf16_t *>(smem);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Share sh;
    if (!find_share(a.q_spans, nullptr, a.per_row, kTile, a.tiles, a.n_split, a.kv_heads, !a.uneven, true, sh)) return;
    const int q0 = sh.of.first, q_len = sh.of.len;
    int k0, k_len;
    a.kv_spans.of(sh.of.seq, k0, k_len);
    const int64_t item = static_cast<int64_t>(sh.tile) * kTile + 32 * wave + (lane & 31);
    const bool ok = item < static_cast<int64_t>(q_len) * a.per_row;
    const int64_t row = q0 + item / a.per_row;
    const int head = sh.kv_head * a.per_row + static_cast<int>(item % a.per_row);
    int u0, u1;
    piece((k_len + kUnitRows - 1) / kUnitRows, a.n_split, a.least, sh.split, u0, u1);
    if (a.to.part_o != nullptr && u0 == u1) return store_no_keys(a.to, sh.split, row, head, ok && lane < 32);
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
        const bf16_t *k = units.step(u, u == u0, more, [&]() { return seen = rows.counts(); }, [](int) {});
        soft.template unit<P>(k, k + P * kPlane, seen, a.factor, at, lane);
    }
    store_soft<T>(soft, a.factor, a.to, sh.split, row, head, ok, lane);
}

// Probabilities of few bf16 rows enter in two parts, which the memory that binds hides (16 rows over 10992 keys of 16 heads 15.4 us with one,
// 16.0 with two): the error of out is the rounding of its store, also where few keys count (rows over 17 keys, up to 2.4e-3 with one).
template <typename T> constexpr int kFewParts = sizeof(T) == 4 ? 3 : 2;

// Few rows: WAVES waves with the same 16 rows take the units in turn, values through an LDS stage of their own (8 or 24 KiB).
template <typename T, int WAVES> __global__ __launch_bounds__(64 * WAVES, sizeof(T) == 4 || WAVES > 4 ? 1 : 2) void cross_few_kernel(CrossArgs a)
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
    int u0, u1;
    piece((k_len + kUnitRows - 1) / kUnitRows, a.n_split, a.least, sh.split, u0, u1);
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
        few.template unit<P, kFewParts<T>>([&](int t, int s, bf16x8(&to)[P]) {
#pragma unroll
            for (int i = 0; i < P; ++i) to[i] = kk[t][s][i];
        }, mine, seen, a.factor, lane);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    __syncthreads();
    store_few<T, WAVES>(few, a.factor, a.to, sh.split, row, head, ok, reinterpret_cast<float *>(smem), wave, lane);
}

// One result from the splits' normalised ones: weights 2^(lse_j - lse).  GROUPS x 16 threads for a row of a head: 16 take four
// channels each, the groups every GROUPS-th split.  With one group, the splits follow one another; with four (a wave for a row of a
// head), the log-sums of 64 splits are one load, and 64 splits' partial results are requested at once.  64 splits of 16 rows: 22.4 us
// with one group, 4.6 with four; 13 splits of 22 thousand rows 16 with one, 19 with four.
constexpr int kSplitChunks = kMostSplits / 64;
template <typename T, int GROUPS> __global__ __launch_bounds__(256) void soft_combine_kernel(SoftOut to, Spans spans, int n_split)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, at = i / (16 * GROUPS), share = to.rows * to.heads;
    if (at >= share) return;
    const int64_t row = at / to.heads;
    if (!spans.covers(row)) return;
    const int c = static_cast<int>(i & 15) * 4, group = static_cast<int>(i >> 4) % GROUPS, lane = threadIdx.x & 63;
    float top = -INFINITY, total = 0.f;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    auto weight = [&](float l) { return l == -INFINITY ? 0.f : (l == top ? 1.f : fast_exp2(l - top)); };  // -inf: no keys in the piece
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
        for (int j = 0; j < n_split; ++j) top = fmaxf(top, to.part_lse[j * share + at]);
        for (int j = 0; j < n_split; ++j) {
            const float l = to.part_lse[j * share + at];
            if (l != -INFINITY) add(l, *reinterpret_cast<const floatx4 *>(to.part_o + (j * share + at) * 64 + c));
        }
    }
    const float w = total == 0.f ? 0.f : 1.f / total;
    T *dst = static_cast<T *>(to.out) + at * 64 + c;
#pragma unroll
    for (int e = 0; e < 4; ++e) dst[e] = from_float<T>(acc[e] * w);
    if (c == 0 && to.lse != nullptr)
        to.lse[(at - row * to.heads) * to.rows + row] = total == 0.f ? -INFINITY : (top + log2f(total)) * kLn2;
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
template <typename T, int PX> __global__ __launch_bounds__(256, sizeof(T) == 4 ? 1 : 2) void grad_q_kernel(CrossArgs a)
{
    constexpr int P = UnitPairs<T>::kParts;
    extern __shared__ __align__(16) unsigned char smem[];
    bf16_t *lds = reinterpret_cast<bf16_t *>(smem);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Share sh;
    if (!find_share(a.q_spans, nullptr, a.per_row, kTile, a.tiles, a.n_split, a.kv_heads, !a.uneven, true, sh)) return;
    const int q0 = sh.of.first, q_len = sh.of.len;
    int k0, k_len;
    a.kv_spans.of(sh.of.seq, k0, k_len);
    const int64_t item = static_cast<int64_t>(sh.tile) * kTile + 32 * wave + (lane & 31);
    const bool ok = item < static_cast<int64_t>(q_len) * a.per_row;
    const int64_t row = q0 + item / a.per_row;
    const int head = sh.kv_head * a.per_row + static_cast<int>(item % a.per_row);
    int u0, u1;
    piece((k_len + kUnitRows - 1) / kUnitRows, a.n_split, a.least, sh.split, u0, u1);
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
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[r] = fast_exp2(fmaf(s[r], a.factor, -l2));
                dp[r] *= s[r];
            }
            if (seen != ~0ull) {
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
    }
    const int64_t to = row * a.heads + head, part = sh.split * a.n_q * a.heads + to;
    if constexpr (kMendD<T>) {
        sum = sum_with_other_half(sum);
        entered = sum_with_other_half(entered);
        if (a.part_q == nullptr) {
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
    if (a.part_q != nullptr)
        store_row(grad.o, 1.f, a.part_q + part * 64, ok, lane);
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
template <typename T> __global__ __launch_bounds__(256) void grad_q_combine_kernel(CrossArgs a)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, at = i >> 4, share = a.n_q * a.heads;
    if (at >= share) return;
    const int64_t row = at / a.heads;
    if (!a.q_spans.covers(row)) return;
    const int c = static_cast<int>(i & 15) * 4;
    floatx4 g = {0.f, 0.f, 0.f, 0.f}, pk = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f, entered = 0.f;
    const int n = pieces_of(a.kv_spans, a.q_spans.find(row), 1, a);
    for (int j = 0; j < n; ++j) {
        g += *reinterpret_cast<const floatx4 *>(a.part_q + (j * share + at) * 64 + c);
        if constexpr (kMendD<T>) {
            pk += *reinterpret_cast<const floatx4 *>(a.part_pk + (j * share + at) * 64 + c);
            sum += a.part_sum[2 * (j * share + at)];
            entered += a.part_sum[2 * (j * share + at) + 1];
        }
    }
    T *dst = static_cast<T *>(a.dq) + at * 64 + c;
#pragma unroll
    for (int e = 0; e < 4; ++e) dst[e] = from_float<T>(a.scale * (g[e] - entered * pk[e]));
    if (kMendD<T> && c == 0) a.stats[2 * ((at - row * a.heads) * a.n_q + row) + 1] -= sum;
}

// PX: bf16 parts in which probabilities and dS enter the products.
template <typename T, int PX> __global__ __launch_bounds__(256, sizeof(T) == 4 ? 1 : 2) void grad_kv_kernel(CrossArgs a)
{
    constexpr int P = UnitPairs<T>::kParts;
    extern __shared__ __align__(16) unsigned char smem[];
    bf16_t *lds = reinterpret_cast<bf16_t *>(smem);
    float *row_stats = reinterpret_cast<float *>(smem + sizeof(bf16_t) * UnitPairs<T>::kStages * UnitPairs<T>::kStage);  // [stages][2][64]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Share sh;
    if (!find_share(a.kv_spans, nullptr, 1, kTile, a.tiles, a.n_split, a.kv_heads, !a.uneven, true, sh)) return;
    const int k0 = sh.of.first, k_len = sh.of.len;
    int q0, q_len;
    a.q_spans.of(sh.of.seq, q0, q_len);
    const int key = sh.tile * kTile + 32 * wave + (lane & 31);
    const bool ok = key < k_len, seen = ok && (a.key_mask == nullptr || a.key_mask[k0 + key] != 0);
    const int64_t row = k0 + key;
    const int items = q_len * a.per_row, head0 = sh.kv_head * a.per_row;
    int u0, u1;
    piece((items + kUnitRows - 1) / kUnitRows, a.n_split, a.least, sh.split, u0, u1);
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
    for (int u = u0; u < u1; ++u) {
        const bf16_t *q = units.step(u, u == u0, more, [&]() { return low_bits(items - u * kUnitRows); }, [&](int stage) {
            float *to = row_stats + stage * 128;
            if (which < 2) to[which * 64 + lane] = st;
            stats = to;
        }), *g = q + P * kPlane;
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
                bf16x8 p[PX], ds[PX];
                split_parts<PX>(x, p);
                split_parts<PX>(y, ds);
#pragma unroll
                for (int dt = 0; dt < 2; ++dt) {
                    multiply<P>(vv.o[dt], p, [&](int part) { return gt.x[w][dt][part]; });
                    multiply<P>(kk.o[dt], ds, [&](int part) { return qt.x[w][dt][part]; });
                }
            }
        }
    }
    if (!seen)  // a masked key gets no gradient, whatever its lanes added up
#pragma unroll
        for (int r = 0; r < 16; ++r) kk.o[0][r] = kk.o[1][r] = vv.o[0][r] = vv.o[1][r] = 0.f;
    const int64_t to = (row * a.kv_heads + sh.kv_head) * 64, share = a.n_kv * a.kv_heads * 64;
    if (a.part_k != nullptr) {
        store_row(kk.o, a.scale, a.part_k + sh.split * share + to, ok, lane);
        store_row(vv.o, 1.f, a.part_v + sh.split * share + to, ok, lane);
    } else {
        store_row(kk.o, a.scale, static_cast<T *>(a.dk) + to, ok, lane);
        store_row(vv.o, 1.f, static_cast<T *>(a.dv) + to, ok, lane);
    }
}

// dk and dv as the sums of their pieces over queries.  16 threads for a row of a head; blockIdx.y: dk or dv.
template <typename T> __global__ __launch_bounds__(256) void grad_kv_combine_kernel(CrossArgs a)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, n = a.n_kv * a.kv_heads * 16;
    if (i >= n || !a.kv_spans.covers(i / (a.kv_heads * 16))) return;
    const float *part = blockIdx.y == 0 ? a.part_k : a.part_v;
    T *out = static_cast<T *>(blockIdx.y == 0 ? a.dk : a.dv);
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    const int pieces = pieces_of(a.q_spans, a.kv_spans.find(i / (a.kv_heads * 16)), a.per_row, a);
    for (int j = 0; j < pieces; ++j) acc += *reinterpret_cast<const floatx4 *>(part + (j * n + i) * 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) out[i * 4 + e] = from_float<T>(acc[e]);
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
    const hipError_t e = allow_lds(&cross_few_kernel<T, WAVES>, kLds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((cross_few_kernel<T, WAVES>), dim3(static_cast<unsigned>(n)), dim3(64 * WAVES), kLds, stream, a);
    return hipGetLastError();
}

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
        hipLaunchKernelGGL(cross_kernel<T>, dim3(static_cast<unsigned>(n)), dim3(256), kLds, stream, a);
    }
    return hipGetLastError();
}

// Few rows: probabilities and dS rounded to bf16 would be most of the error of dk and dv, whose sums have few terms, and now and then of
// dq, where a few dS count (2.4e-3 to 2.9e-3, against 1.66e-3 by the rounding of the results themselves, which is what two parts leave).
// With many rows the errors are 2.35e-3 and 2.3e-3 and no memory hides the products.  Gradient of 16 heads in bf16, us, one part / two: 1 row over 10992
// keys 55 / 60, 64 over 2000 24.8 / 26.6, 2748 over 10992 588 / 795, 8192 over 8192 1129 / 1554; dk and dv alone: 128 over 10992 71 / 80, 512 over
// 10992 137 / 163.
constexpr int kFewItems = kUnitRows;
template <typename T> hipError_t launch_grad_t(const CrossArgs &a, bool of_keys, hipStream_t stream)
{
    const int64_t n = xcd_padded(a.tiles * a.n_split * a.kv_heads);
    if (!grid_ok(n)) return hipErrorInvalidValue;
    const size_t lds = UnitPairs<T>::kStages * (UnitPairs<T>::kStage * sizeof(bf16_t) + (of_keys ? 128 * sizeof(float) : 0));
    auto kernel = of_keys ? &grad_kv_kernel<T, UnitPairs<T>::kParts> : &grad_q_kernel<T, UnitPairs<T>::kParts>;
    if constexpr (sizeof(T) == 2)
        if (a.n_q * a.per_row <= kFewItems * a.q_spans.batch) kernel = of_keys ? &grad_kv_kernel<T, 2> : &grad_q_kernel<T, 2>;
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

hipError_t launch_grad_q_combine(const CrossArgs &a, bool is_bf16, hipStream_t stream)
{
    const int64_t blocks = (a.n_q * a.heads * 16 + 255) / 256;
    if (!grid_ok(blocks)) return hipErrorInvalidValue;
    if (is_bf16)
        hipLaunchKernelGGL(grad_q_combine_kernel<bf16_t>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL(grad_q_combine_kernel<float>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_grad_kv(const CrossArgs &a, bool is_bf16, hipStream_t stream)
{
    return is_bf16 ? launch_grad_t<bf16_t>(a, true, stream) : launch_grad_t<float>(a, true, stream);
}

hipError_t launch_soft_combine(const SoftOut &to, const Spans &spans, int n_split, bool is_bf16, hipStream_t stream)
{
    // (us, wide or not: 5 splits of 4800 rows 17.7 / 19.2 with the attention, 4 of 8192 23.5 / 21.6, 10 of 2048 15.7 / 20.0, 6 of 256 9.8 / 12.8,
    // 2 of 16 9.0 / 8.5)
    const int64_t share = to.rows * to.heads;
    const bool wide = n_split >= 3 && share <= 1024 * (n_split < 8 ? n_split : 8);
    const int64_t blocks = (share * (wide ? 64 : 16) + 255) / 256;
    if (!grid_ok(blocks) || n_split > kMostSplits) return hipErrorInvalidValue;
    auto kernel = is_bf16 ? (wide ? &soft_combine_kernel<bf16_t, 4> : &soft_combine_kernel<bf16_t, 1>)
                          : (wide ? &soft_combine_kernel<float, 4> : &soft_combine_kernel<float, 1>);
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream, to, spans, n_split);
    return hipGetLastError();
}

hipError_t launch_grad_kv_combine(const CrossArgs &a, bool is_bf16, hipStream_t stream)
{
    const int64_t blocks = (a.n_kv * a.kv_heads * 16 + 255) / 256;
    if (!grid_ok(2 * blocks)) return hipErrorInvalidValue;
    const dim3 grid(static_cast<unsigned>(blocks), 2);
    if (is_bf16)
        hipLaunchKernelGGL(grad_kv_combine_kernel<bf16_t>, grid, dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL(grad_kv_combine_kernel<float>, grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}

hipError_t launch_span_status(const Spans &q, const Spans &kv, int *status, hipStream_t stream)
{
    hipLaunchKernelGGL(span_status_kernel, dim3(1), dim3(1024), 0, stream, q, kv, status);
    return hipGetLastError();
}

}  // namespace s3r
