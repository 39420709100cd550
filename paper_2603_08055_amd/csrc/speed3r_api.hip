// C ABI of the library (see include/speed3r.h): argument checks, workspace carving, launch
// sequencing, optional per-stage event timing.  No kernel code here.
#include "../../include/speed3r.h"
#include "s3r_kernels.h"

#include <climits>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <algorithm>
#include <initializer_list>
#include <mutex>
#include <tuple>
#include <utility>
#include <vector>

// Scratch of speed3r_sparse_global_attn_noalloc: device memory that exists from the moment the code object
// is loaded, one copy per GPU, so that entry point never allocates.  In host code this name only stands for
// the symbol; the device address comes from hipGetSymbolAddress (static_scratch below).
constexpr size_t kStaticScratchBytes = S3R_STATIC_SCRATCH_BYTES;
static __device__ __align__(256) unsigned char scratch[kStaticScratchBytes];

namespace {

thread_local char g_err[512] = "no error";
thread_local bool t_no_events = false;  // set while an entry point that must not create HIP events runs

s3r_status fail(s3r_status st, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
    return st;
}

s3r_status hip_fail(hipError_t e, const char *what)
{
    return fail(S3R_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

#define S3R_HIP(call, what)                                  \
    do {                                                     \
        hipError_t e_ = (call);                              \
        if (e_ != hipSuccess) return hip_fail(e_, what);     \
    } while (0)

constexpr size_t kAlign = 256;
constexpr size_t kScoreBytesCap = size_t(8) << 30;  // S_guide is processed in head chunks of at most this size

size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int g_kernel_choice = 0;  // 0 auto, 1 generic attention kernels only, 2 TopK from scores written to memory

// every supported block size, bf16 and fp32 (the latter with K/V in bf16 operand parts)
bool mfma_ok(s3r_dtype dtype, int block) { (void)dtype; (void)block; return g_kernel_choice != 1; }
// copies of a K (or V) tile array the MFMA kernels read: fp32 problems keep bf16 parts hi, lo and (K) lo2
size_t tile_parts(s3r_dtype dtype) { return dtype == S3R_BF16 ? 1 : 3; }

// Dense attention of few query rows (the special tokens) in key splits: the number of splits with the shortest time
// by a model of the launch, in microseconds on MI355X (256 CUs; three workgroups fill a CU).  A CU works through
// n = ceil(workgroups * s / 256) of them:
//   * each is reckoned at 0.68 us per key unit (1.1 over small blocks, which take 0.7: see below) and 4 us at its start
//     and end;
//   * the bf16 kernel needs two to three workgroups on a CU to fill it: one left over in the last round costs as
//     much as 1.75, two as 2.3;
//   * the workgroups of later rounds no longer walk the keys in step and share less of them in the L2s: 2.5 % per
//     round, 30 % at most;
//   * the combine kernel reads s partial rows one after the other (0.6 us each) and moves them at 4 TB/s.
// Measured, 16 heads, 5 special rows per view, dense kernel and combine (ms for the number of splits, * = chosen):
//   bf16, blocks of 64, 20 views    1: 0.340   8: 0.060  16: 0.046*  24: 0.051  32: 0.053
//                       100 views   4: 0.481   8: 0.359  12: 0.354*  24: 0.407  32: 0.431
//                       300 views   2: 3.75    3: 3.87    4: 3.01*   6: 3.38    8: 3.03   12: 3.32
//                       1000 views  1: 36.1    2: 32.1*   3: 33.6    4: 32.5    6: 33.8
//   bf16, blocks of 16, 20 views    8: 0.076  16: 0.056   24: 0.059  32: 0.061*
//                       100 views   8: 0.447  12: 0.413*  16: 0.440  32: 0.493
//   fp32, blocks of 64, 20 views    8: 0.120  16: 0.082*  24: 0.092  32: 0.098
//                       60 views    8: 0.589  10: 0.503   16: 0.512* 20: 0.536   32: 0.548   (2.12 with a ring of
//                       120 KiB, one workgroup per CU and the operand array of a chunk looked up in scratch memory)
// In fp32 the error of a row against 64 bits grows with the units in one chain of sums (200 views: 1.0e-5 in one split,
// 7.6e-6 in 2, 5.7e-6 in 6, 5.4e-6 in 8, 5.0e-6 in 16).  A unit is therefore weighed at four times the 1.95 us it takes
// (small blocks: twice), against the start and the combine kernel: in fp32 this is a rule for exactness more than a model
// of the time.  There are at least 8 splits although fewer can be faster, and with up to 48 workgroups, which 8 leave at one
// or two to a CU where two run at once, at least 16.
// In bf16 it is the rounding of P, which gains from the splits, every split's largest probability being exact (outlier keys,
// against 64 bits: 30 views in 4 x 4 windows, 8 heads 1.80e-3 in one split, 1.69e-3 in 32, 1.67e-3 in 48; 20 views, 4 heads
// 1.680e-3 in 28 splits, 1.668e-3 in 36; blocks of 32, 40 views, 16 heads 1.705e-3 in 16, 1.689e-3 in 24).  So the units of
// small blocks stay weighed at what they took with another kernel: as many splits as then, 10 % of this launch at 20 views.
// lean: the counts that the time alone would give (bf16), or at least 8 (fp32), for workspaces that hold no more.
constexpr int kMaxDenseSplit = 64;
int dense_splits(int64_t n_rows, int heads, int64_t n_units, s3r_dtype dtype, int block, bool lean)
{
    const bool bf16 = dtype == S3R_BF16;
    const int64_t wgs = (n_rows + 127) / 128 * heads;
    if (wgs >= 3072) return 1;  // 12 workgroups and more per CU: even enough
    const double unit_us = bf16 ? (block >= 64 ? (lean ? 0.64 : 0.68) : (lean ? 0.7 : 1.1)) : (block >= 64 ? 8.0 : 3.8);
    const int64_t at_once = bf16 ? 3 : 1;
    const double left_over[3] = {0.0, bf16 ? 0.75 : 0.0, bf16 ? 0.3 : 0.0};
    auto time_us = [&](int s) {
        const int64_t n = (wgs * s + 255) / 256, rounds = (n + at_once - 1) / at_once;
        const double drift = 0.025 * static_cast<double>(rounds - 1);
        const double walk = (static_cast<double>(n) + left_over[n % at_once]) * (static_cast<double>((n_units + s - 1) / s) * unit_us + 4.0) *
                            (1.0 + (drift < 0.3 ? drift : 0.3));
        return s == 1 ? walk : walk + s * (0.6 + 1.3e-4 * static_cast<double>(n_rows * heads));
    };
    int most = static_cast<int>(n_units / 4 < kMaxDenseSplit ? n_units / 4 : kMaxDenseSplit);  // at least 4 units each
    if (most < 1) most = 1;
    const int least32 = wgs <= 48 && !lean ? 16 : 8;
    const int least = bf16 ? 1 : (most < least32 ? most : least32);
    double us[kMaxDenseSplit + 1], shortest = INFINITY;
    for (int s = least; s <= most; ++s) {
        us[s] = time_us(s);
        if (us[s] < shortest) shortest = us[s];
    }
    int s = least;
    while (us[s] > 1.01 * shortest) ++s;  // the fewest that come within 1 %: their partial results take workspace
    return s;
}

constexpr int kCandCap = 256;  // candidate slots per list of the TopK-in-the-sweep path (two lists per row)

s3r_status check_shape(int64_t n_tok, int heads, int head_dim, int block, int topk, int dtype)
{
    if (n_tok <= 0 || heads <= 0 || topk <= 0)
        return fail(S3R_ERR_INVALID_ARG, "n_tok (%lld), heads (%d) and topk (%d) must be positive",
                    static_cast<long long>(n_tok), heads, topk);
    if (dtype != S3R_F32 && dtype != S3R_BF16) return fail(S3R_ERR_UNSUPPORTED, "unknown dtype %d", dtype);
    if (head_dim != 64) return fail(S3R_ERR_UNSUPPORTED, "head_dim %d unsupported (must be 64)", head_dim);
    if (block != 16 && block != 32 && block != 64 && block != 128)
        return fail(S3R_ERR_UNSUPPORTED, "block %d unsupported (must be 16, 32, 64 or 128)", block);
    if (heads > 65535) return fail(S3R_ERR_UNSUPPORTED, "heads %d unsupported (max 65535)", heads);
    const int64_t n_blk = (n_tok + block - 1) / block;
    if (n_blk * heads > 0x7fffffffLL) return fail(S3R_ERR_UNSUPPORTED, "n_blk * heads exceeds 2^31 - 1");
    return S3R_OK;
}

// ---- workspace layout of the full path -------------------------------------------------------
struct Layout {
    int64_t n_blk, tiles, ld_s;
    int kk;      // blocks TopK picks per row (among the non-forced ones)
    int width;   // blocks attended per row: kk + n_forced
    int head_chunk;
    size_t qc, kc, vc, oc, tile[8], idx, idx_merged, forced_clean, forced_words, s, kb, vb, kb_spec, vb_spec;
    size_t stat_slots, head_stats, thr, cand, cand_count, overflow, blk_len, oc_tok, spec_part_o, spec_part_lse, total;
    int spec_split;  // key splits of the special rows' dense attention (1: none)
};

// n_tok: tokens on the sparse path (the image tokens); n_spec: special tokens (dense rows).  have: bytes there are; special
// rows that would not fit with the number of key splits they should have take fewer.
Layout make_layout(int64_t n_tok, int heads, int block, int topk, int n_forced, s3r_dtype dtype,
                   int64_t n_spec = 0, bool token_queries = false, size_t have = SIZE_MAX)
{
    Layout L{};
    L.n_blk = (n_tok + block - 1) / block;
    const int64_t free_blk = L.n_blk - n_forced;
    L.kk = static_cast<int>(topk < free_blk ? topk : free_blk);
    L.width = L.kk + n_forced;
    L.tiles = s3r::pooled_tiles_padded(L.n_blk);
    L.ld_s = (L.n_blk + 63) / 64 * 64;
    const size_t per_head_s = static_cast<size_t>(L.n_blk) * L.ld_s * sizeof(float);
    int64_t hc = static_cast<int64_t>(kScoreBytesCap / per_head_s);
    if (hc < 1) hc = 1;
    if (hc > heads) hc = heads;
    L.head_chunk = static_cast<int>(hc);
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t o = off; off += align_up(bytes); return o; };
    const size_t pooled = static_cast<size_t>(heads) * L.n_blk * 64 * sizeof(float);
    L.qc = take(pooled);
    L.kc = take(pooled);
    L.vc = take(pooled);
    L.oc = take(pooled);
    for (int a = 0; a < 8; ++a) L.tile[a] = take(static_cast<size_t>(heads) * L.tiles * 32 * 64 * 2);
    L.idx = take(static_cast<size_t>(heads) * L.n_blk * L.kk * sizeof(int32_t));
    L.idx_merged = take(n_forced > 0 ? static_cast<size_t>(heads) * L.n_blk * L.width * sizeof(int32_t) : 0);
    L.forced_clean = take(static_cast<size_t>(n_forced) * sizeof(int32_t));
    L.forced_words = take(n_forced > 0 ? static_cast<size_t>((L.n_blk + 63) / 64) * sizeof(unsigned long long) : 0);
    L.s = take(per_head_s * L.head_chunk);
    const size_t blocked = mfma_ok(dtype, block) ? static_cast<size_t>(heads) * L.n_blk * block * 64 * 2 * tile_parts(dtype) : 0;
    L.kb = take(blocked);
    L.vb = take(blocked);
    const size_t spec_tiles = mfma_ok(dtype, block) ? static_cast<size_t>(heads) * ((n_spec + 63) / 64) * 64 * 64 * 2 * tile_parts(dtype) : 0;
    L.kb_spec = take(spec_tiles);
    L.vb_spec = take(spec_tiles);
    // TopK-in-the-sweep buffers, for all heads at once (the sweeps are not chunked)
    const size_t chunk_rows = static_cast<size_t>(heads) * L.n_blk;
    L.stat_slots = take(static_cast<size_t>(heads) * 3 * s3r::kStatSlots * sizeof(unsigned));
    L.head_stats = take(static_cast<size_t>(heads) * sizeof(s3r::HeadStats));
    L.thr = take(chunk_rows * sizeof(float));
    L.cand = take(chunk_rows * 2 * kCandCap * sizeof(int32_t));
    L.cand_count = take(chunk_rows * 2 * sizeof(int));
    L.overflow = take(sizeof(int));
    L.blk_len = take(static_cast<size_t>(L.n_blk) * sizeof(int32_t));
    // compression branch with unpooled queries: fp32 compressed output per query slot
    L.oc_tok = take(token_queries ? static_cast<size_t>(L.n_blk) * block * heads * 64 * sizeof(float) : 0);
    // special rows in key splits: normalised partial results and their log-sums
    const size_t before = off;
    for (const bool lean : {false, true}) {
        off = before;
        L.spec_split = 1;
        if (n_spec > 0 && mfma_ok(dtype, block))
            L.spec_split = dense_splits(n_spec, heads, (L.n_blk * block + 63) / 64 + (n_spec + 63) / 64, dtype, block, lean);
        const size_t part_rows = L.spec_split > 1 ? static_cast<size_t>(L.spec_split) * n_spec * heads : 0;
        L.spec_part_o = take(part_rows * 64 * sizeof(float));
        L.spec_part_lse = take(part_rows * sizeof(float));
        L.total = off;
        if (L.total <= have) break;
    }
    return L;
}

// ---- library-held scratch --------------------------------------------------------------------
std::mutex g_mu;
constexpr int kMaxDevices = 64;
void *g_scratch[kMaxDevices] = {};
size_t g_scratch_bytes[kMaxDevices] = {};

s3r_status scratch_get(size_t bytes, void **out)
{
    int dev = 0;
    S3R_HIP(hipGetDevice(&dev), "hipGetDevice");
    if (dev < 0 || dev >= kMaxDevices) return fail(S3R_ERR_UNSUPPORTED, "device ordinal %d unsupported", dev);
    std::lock_guard<std::mutex> lock(g_mu);
    if (bytes > g_scratch_bytes[dev]) {
        S3R_HIP(hipDeviceSynchronize(), "hipDeviceSynchronize before growing scratch");
        if (g_scratch[dev]) {
            S3R_HIP(hipFree(g_scratch[dev]), "hipFree(scratch)");
            g_scratch[dev] = nullptr;
            g_scratch_bytes[dev] = 0;
        }
        void *p = nullptr;
        hipError_t e = hipMalloc(&p, bytes);
        if (e != hipSuccess) return fail(S3R_ERR_WORKSPACE, "hipMalloc of %zu scratch bytes failed: %s", bytes, hipGetErrorString(e));
        g_scratch[dev] = p;
        g_scratch_bytes[dev] = bytes;
    }
    *out = g_scratch[dev];
    return S3R_OK;
}

// Device address of this GPU's copy of `scratch`, looked up once per device with that device current.
void *g_static_ptr[kMaxDevices] = {};

s3r_status static_scratch(void **out)
{
    int dev = 0;
    S3R_HIP(hipGetDevice(&dev), "hipGetDevice");
    if (dev < 0 || dev >= kMaxDevices) return fail(S3R_ERR_UNSUPPORTED, "device ordinal %d unsupported", dev);
    std::lock_guard<std::mutex> lock(g_mu);
    if (g_static_ptr[dev] == nullptr) {
        void *ptr = nullptr;
        S3R_HIP(hipGetSymbolAddress(&ptr, HIP_SYMBOL(scratch)), "hipGetSymbolAddress(scratch)");
        if (ptr == nullptr || (reinterpret_cast<uintptr_t>(ptr) & (kAlign - 1)) != 0)
            return fail(S3R_ERR_HIP, "static scratch has no usable device address (%p)", ptr);
        g_static_ptr[dev] = ptr;
    }
    *out = g_static_ptr[dev];
    return S3R_OK;
}

// ---- per-stage event timing ------------------------------------------------------------------
bool g_profiling = false;
struct Span { int stage; hipEvent_t start, stop; };
std::vector<Span> g_spans;        // spans recorded since the last speed3r_get_stage_ms
std::vector<hipEvent_t> g_pool;   // recycled events

hipEvent_t event_take()
{
    if (!g_pool.empty()) { hipEvent_t e = g_pool.back(); g_pool.pop_back(); return e; }
    hipEvent_t e = nullptr;
    if (hipEventCreate(&e) != hipSuccess) return nullptr;
    return e;
}

struct StageTimer {
    hipStream_t stream;
    Span span{};
    bool on = false;
    StageTimer(int stage, hipStream_t st) : stream(st)
    {
        if (!g_profiling || t_no_events) return;
        std::lock_guard<std::mutex> lock(g_mu);
        span.stage = stage;
        span.start = event_take();
        span.stop = event_take();
        on = span.start && span.stop;
        if (on) on = hipEventRecord(span.start, stream) == hipSuccess;
    }
    ~StageTimer()
    {
        if (!on) return;
        if (hipEventRecord(span.stop, stream) != hipSuccess) return;
        std::lock_guard<std::mutex> lock(g_mu);
        g_spans.push_back(span);
    }
};

char *at(void *base, size_t off) { return static_cast<char *>(base) + off; }

// Buffers of the TopK-in-the-sweep path (all null: TopK from scores written to s_buf).
struct FusedBufs {
    void *stat_slots = nullptr;             // scratch of launch_pooled_stats
    s3r::HeadStats *head_stats = nullptr;   // [heads]
    float *thr = nullptr;
    int32_t *cand = nullptr;
    int *cand_count = nullptr;
    int *overflow = nullptr;
};

// pooled fp32 -> operand tiles -> S_guide / Oc' -> TopK, in head chunks bounded by the S buffer
s3r_status run_compress_topk(const float *qc, const float *kc, const float *vc, void *const tile[8],
                             float *s_buf, int64_t ld_s, int head_chunk, float *o_comp, int32_t *idx,
                             int64_t n_blk, int64_t tiles, int heads, int kk, float scale,
                             bool accurate_pv, bool want_topk, const unsigned long long *forced_words,
                             const FusedBufs &fb, bool keep_tiles, hipStream_t stream)
{
    // Short sequences: one launch on the pooled means themselves (keep_tiles: the caller reads the operand tiles).
    if (want_topk && g_kernel_choice != 2 && s3r::compress_small_takes(n_blk, heads, kk)) {
        StageTimer tm(S3R_STAGE_COMPRESS, stream);
        S3R_HIP(s3r::launch_compress_small(qc, kc, vc, o_comp, idx, n_blk, heads, kk, scale, forced_words, stream),
                "compress (short sequence) kernel launch");
        if (keep_tiles)
            S3R_HIP(s3r::launch_split(qc, kc, vc, tile[0], tile[1], tile[2], tile[3], tile[4], nullptr, nullptr, nullptr,
                                      nullptr, nullptr, n_blk, heads, stream),
                    "split kernel launch");
        return S3R_OK;
    }
    // Without S_guide in memory when k allows it.  Should a candidate list run over (long runs of
    // equal scores), the overflow word makes the two plain launches that follow redo the chunk;
    // otherwise they return at once.  A row's two lists divide its keys evenly, 16 of every 32 each, so up
    // to 2 kCandCap blocks no list can run over and the two launches are left out (4 us of a call).
    const bool fused = want_topk && fb.thr != nullptr && kk >= 1 && kk <= s3r::kFusedTopkMaxK && g_kernel_choice != 2;
    {
        StageTimer tm(S3R_STAGE_SPLIT, stream);
        if (fused)
            S3R_HIP(s3r::launch_pooled_stats(qc, kc, n_blk, heads, fb.stat_slots, stream),
                    "pooled statistics kernel launch");
        S3R_HIP(s3r::launch_split(qc, kc, vc, tile[0], tile[1], tile[2], tile[3], tile[4],
                                  accurate_pv ? tile[5] : nullptr, fused ? tile[6] : nullptr, fused ? tile[7] : nullptr,
                                  fused ? fb.stat_slots : nullptr, fused ? fb.head_stats : nullptr, n_blk, heads, stream),
                "split kernel launch");
    }
    const size_t tile_head = static_cast<size_t>(tiles) * 32 * 64 * 2;  // bytes per head per array
    if (fused) {
        // all heads in one launch each: nothing here is as large as S
        {
            StageTimer tm(S3R_STAGE_COMPRESS, stream);
            S3R_HIP(s3r::launch_compress_threshold(tile[0], tile[1], tile[2], tile[3], tile[4],
                                                   accurate_pv ? tile[5] : nullptr, tile[6], tile[7], o_comp, n_blk, heads, scale,
                                                   forced_words, kk, fb.head_stats, fb.thr, fb.overflow, stream),
                    "compress (threshold) kernel launch");
        }
        StageTimer tm(S3R_STAGE_TOPK, stream);
        S3R_HIP(s3r::launch_compress_filter(tile[6], tile[7], n_blk, heads, forced_words, fb.thr,
                                            fb.cand, fb.cand_count, kCandCap, fb.overflow, stream),
                "compress (filter) kernel launch");
        S3R_HIP(s3r::launch_topk_candidates(qc, kc, fb.cand, fb.cand_count, kCandCap, idx, n_blk, heads, kk, stream),
                "candidate topk kernel launch");
    }
    if (fused && n_blk <= 2 * kCandCap) return S3R_OK;
    const int *run_flag = fused ? fb.overflow : nullptr;
    for (int h0 = 0; h0 < heads; h0 += head_chunk) {
        const int hc = (heads - h0 < head_chunk) ? heads - h0 : head_chunk;
        {
            StageTimer tm(S3R_STAGE_COMPRESS, stream);
            S3R_HIP(s3r::launch_compress(at(tile[0], h0 * tile_head), at(tile[1], h0 * tile_head),
                                         at(tile[2], h0 * tile_head), at(tile[3], h0 * tile_head),
                                         at(tile[4], h0 * tile_head),
                                         accurate_pv ? at(tile[5], h0 * tile_head) : nullptr, s_buf, ld_s,
                                         o_comp + static_cast<size_t>(h0) * n_blk * 64, n_blk, hc, scale,
                                         forced_words, run_flag, stream),
                    "compress kernel launch");
        }
        if (want_topk && kk > 0) {
            StageTimer tm(S3R_STAGE_TOPK, stream);
            S3R_HIP(s3r::launch_topk(s_buf, ld_s, idx + static_cast<size_t>(h0) * n_blk * kk, n_blk,
                                     static_cast<int64_t>(hc) * n_blk, kk, run_flag, stream),
                    "topk kernel launch");
        }
    }
    return S3R_OK;
}

// Special / image token split of a sequence of `n_tok` rows in views of `period` rows whose first
// `special` rows are special tokens (0, 0: no special tokens).
struct Split {
    int64_t n_img;   // slots of the sequence the sparse path works on (with windows: n_blk * block, edge
                     // windows leaving slots empty)
    int64_t n_spec;
    bool windows;
    s3r::TokenMap img, spec;
};

s3r_status make_split(int64_t n_tok, int period, int special, int grid_h, int grid_w, int window, int block,
                      Split *out)
{
    Split sp{};
    sp.n_img = n_tok;
    sp.n_spec = 0;
    sp.windows = false;
    if (window != 0 || grid_h != 0 || grid_w != 0) {
        if (window <= 0 || grid_h <= 0 || grid_w <= 0)
            return fail(S3R_ERR_INVALID_ARG, "window (%d), grid_h (%d) and grid_w (%d) must all be positive or all 0",
                        window, grid_h, grid_w);
        if (window * window != block)
            return fail(S3R_ERR_INVALID_ARG, "block (%d) must equal window * window (%d)", block, window * window);
        if (period <= 0 || special < 0 || period - special != grid_h * grid_w)
            return fail(S3R_ERR_INVALID_ARG, "tokens_per_view (%d) must equal special_per_view (%d) + grid_h * grid_w (%d)",
                        period, special, grid_h * grid_w);
    }
    if (period == 0 && special == 0) { *out = sp; return S3R_OK; }
    if (period <= 0 || special < 0 || special >= period)
        return fail(S3R_ERR_INVALID_ARG, "special_per_view (%d) must lie in [0, tokens_per_view = %d)", special, period);
    if (n_tok % period != 0)
        return fail(S3R_ERR_INVALID_ARG, "n_tok (%lld) is not a multiple of tokens_per_view (%d)",
                    static_cast<long long>(n_tok), period);
    if (n_tok > 0x7fffffffLL) return fail(S3R_ERR_UNSUPPORTED, "n_tok exceeds 2^31 - 1 with special tokens");
    if (special == 0 && window == 0) { *out = sp; return S3R_OK; }
    const int64_t views = n_tok / period;
    sp.n_spec = views * special;
    sp.n_img = n_tok - sp.n_spec;
    sp.img.period = period; sp.img.first = special; sp.img.count = period - special;
    sp.spec.period = period; sp.spec.first = 0; sp.spec.count = special;
    if (window != 0) {
        sp.windows = true;
        sp.img.win = window; sp.img.grid_h = grid_h; sp.img.grid_w = grid_w;
        sp.img.nwx = (grid_w + window - 1) / window;
        sp.img.nw = sp.img.nwx * ((grid_h + window - 1) / window);
        sp.n_img = views * sp.img.nw * block;
        if (sp.n_img > 0x7fffffffLL) return fail(S3R_ERR_UNSUPPORTED, "windowed sequence exceeds 2^31 - 1 slots");
    }
    *out = sp;
    return S3R_OK;
}

float resolve_scale(float s, int head_dim) { return s > 0.f ? s : 1.f / std::sqrt(static_cast<float>(head_dim)); }

}  // namespace

extern "C" {

const char *speed3r_last_error(void) { return g_err; }

s3r_status speed3r_set_profiling(int enable)
{
    std::lock_guard<std::mutex> lock(g_mu);
    g_profiling = enable != 0;
    return S3R_OK;
}

s3r_status speed3r_set_kernel_choice(int choice)
{
    if (choice < 0 || choice > 2) return fail(S3R_ERR_INVALID_ARG, "kernel choice %d unknown", choice);
    g_kernel_choice = choice;
    return S3R_OK;
}

s3r_status speed3r_get_stage_ms(float *ms, int *launches)
{
    if (!ms || !launches) return fail(S3R_ERR_INVALID_ARG, "ms and launches must be non-null host arrays");
    std::lock_guard<std::mutex> lock(g_mu);
    for (int i = 0; i < S3R_N_STAGES; ++i) { ms[i] = 0.f; launches[i] = 0; }
    for (auto &s : g_spans) {
        S3R_HIP(hipEventSynchronize(s.stop), "hipEventSynchronize");
        float t = 0.f;
        S3R_HIP(hipEventElapsedTime(&t, s.start, s.stop), "hipEventElapsedTime");
        ms[s.stage] += t;
        launches[s.stage] += 1;
    }
    for (auto &s : g_spans) { g_pool.push_back(s.start); g_pool.push_back(s.stop); }
    g_spans.clear();
    return S3R_OK;
}

s3r_status speed3r_release_scratch(void)
{
    int dev = 0;
    S3R_HIP(hipGetDevice(&dev), "hipGetDevice");
    if (dev < 0 || dev >= kMaxDevices) return S3R_OK;
    std::lock_guard<std::mutex> lock(g_mu);
    if (g_scratch[dev]) {
        S3R_HIP(hipDeviceSynchronize(), "hipDeviceSynchronize");
        S3R_HIP(hipFree(g_scratch[dev]), "hipFree(scratch)");
        g_scratch[dev] = nullptr;
        g_scratch_bytes[dev] = 0;
    }
    return S3R_OK;
}

size_t speed3r_workspace_bytes(int64_t n_tok, int heads, int head_dim, int block, int topk, int n_forced,
                               s3r_dtype dtype)
{
    if (check_shape(n_tok, heads, head_dim, block, topk, dtype) != S3R_OK) return 0;
    if (n_forced < 0 || n_forced > (n_tok + block - 1) / block) {
        fail(S3R_ERR_INVALID_ARG, "n_forced (%d) must lie in [0, n_blk]", n_forced);
        return 0;
    }
    return make_layout(n_tok, heads, block, topk, n_forced, dtype).total;
}

size_t speed3r_workspace_bytes_ex(const s3r_params *p)
{
    if (!p) { fail(S3R_ERR_INVALID_ARG, "params is null"); return 0; }
    if (check_shape(p->n_tok, p->heads, p->head_dim, p->block, p->topk, p->dtype) != S3R_OK) return 0;
    Split sp{};
    if (make_split(p->n_tok, p->tokens_per_view, p->special_per_view, p->grid_h, p->grid_w, p->window, p->block,
                   &sp) != S3R_OK)
        return 0;
    if (p->n_forced < 0 || p->n_forced > (sp.n_img + p->block - 1) / p->block) {
        fail(S3R_ERR_INVALID_ARG, "n_forced (%d) must lie in [0, n_blk]", p->n_forced);
        return 0;
    }
    if (p->compress_queries != 0 && p->compress_queries != 1) {
        fail(S3R_ERR_INVALID_ARG, "compress_queries (%d) must be 0 or 1", p->compress_queries);
        return 0;
    }
    return make_layout(sp.n_img, p->heads, p->block, p->topk, p->n_forced, p->dtype, sp.n_spec, p->compress_queries == 1).total;
}

int64_t speed3r_num_blocks(const s3r_params *p)
{
    if (!p) { fail(S3R_ERR_INVALID_ARG, "params is null"); return -1; }
    if (check_shape(p->n_tok, p->heads, p->head_dim, p->block, p->topk, p->dtype) != S3R_OK) return -1;
    Split sp{};
    if (make_split(p->n_tok, p->tokens_per_view, p->special_per_view, p->grid_h, p->grid_w, p->window, p->block,
                   &sp) != S3R_OK)
        return -1;
    return (sp.n_img + p->block - 1) / p->block;
}

int speed3r_selected_per_row(int64_t n_tok, int block, int topk, int n_forced)
{
    if (n_tok <= 0 || block <= 0 || topk <= 0 || n_forced < 0) return -1;
    const int64_t n_blk = (n_tok + block - 1) / block;
    if (n_forced > n_blk) return -1;
    const int64_t free_blk = n_blk - n_forced;
    return static_cast<int>(n_forced + (topk < free_blk ? topk : free_blk));
}

s3r_status speed3r_sparse_global_attn_ex(const s3r_params *p)
{
    if (!p) return fail(S3R_ERR_INVALID_ARG, "params is null");
    s3r_status st = check_shape(p->n_tok, p->heads, p->head_dim, p->block, p->topk, p->dtype);
    if (st != S3R_OK) return st;
    if (!p->q || !p->k || !p->v || !p->out) return fail(S3R_ERR_INVALID_ARG, "q, k, v and out must be non-null");
    if (!aligned16(p->q) || !aligned16(p->k) || !aligned16(p->v) || !aligned16(p->out) ||
        !aligned16(p->gate_logits) || !aligned16(p->o_sel) || !aligned16(p->o_comp) ||
        !aligned16(p->topk_idx) || !aligned16(p->lse_sel) || (reinterpret_cast<uintptr_t>(p->status) & 3u) != 0)
        return fail(S3R_ERR_INVALID_ARG, "device pointers must be 16-byte aligned");
    if (p->out == p->q || p->out == p->k || p->out == p->v) return fail(S3R_ERR_INVALID_ARG, "out must not alias an input");
    // 16-byte vector loads: rows and heads of q, k, v must start on 16-byte boundaries
    if (p->stride_tok < 0 || p->stride_head < 0 || p->stride_tok % 8 != 0 || p->stride_head % 8 != 0)
        return fail(S3R_ERR_INVALID_ARG, "stride_tok (%lld) and stride_head (%lld) must be non-negative multiples of 8 elements",
                    static_cast<long long>(p->stride_tok), static_cast<long long>(p->stride_head));
    s3r::InStride in{};  // {0, 0} = packed
    if (p->stride_tok != 0 || p->stride_head != 0) {
        in.tok = p->stride_tok != 0 ? p->stride_tok : static_cast<int64_t>(p->heads) * 64;
        in.head = p->stride_head != 0 ? p->stride_head : 64;
    }
    const int n_forced = p->forced_blocks ? p->n_forced : 0;
    if (p->n_forced < 0 || (p->n_forced > 0 && !p->forced_blocks) || (p->forced_blocks && p->n_forced == 0))
        return fail(S3R_ERR_INVALID_ARG, "forced_blocks and n_forced (%d) must be given together", p->n_forced);
    Split sp{};
    st = make_split(p->n_tok, p->tokens_per_view, p->special_per_view, p->grid_h, p->grid_w, p->window, p->block, &sp);
    if (st != S3R_OK) return st;
    if (n_forced > (sp.n_img + p->block - 1) / p->block)
        return fail(S3R_ERR_INVALID_ARG, "n_forced (%d) exceeds the number of blocks", n_forced);
    if (p->compress_queries != 0 && p->compress_queries != 1)
        return fail(S3R_ERR_INVALID_ARG, "compress_queries (%d) must be 0 or 1", p->compress_queries);
    const bool token_queries = p->compress_queries == 1;
    if (token_queries && p->dtype == S3R_BF16 && !mfma_ok(p->dtype, p->block))
        return fail(S3R_ERR_UNSUPPORTED, "compress_queries = 1 on bf16 data needs the MFMA kernels (kernel choice 1 is set)");
    const Layout L = make_layout(sp.n_img, p->heads, p->block, p->topk, n_forced, p->dtype, sp.n_spec, token_queries,
                                 p->workspace_bytes);
    if (!p->workspace) return fail(S3R_ERR_WORKSPACE, "workspace is null (%zu bytes needed)", L.total);
    if ((reinterpret_cast<uintptr_t>(p->workspace) & (kAlign - 1)) != 0)
        return fail(S3R_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    if (p->workspace_bytes < L.total)
        return fail(S3R_ERR_WORKSPACE, "workspace too small: %zu bytes given, %zu needed", p->workspace_bytes, L.total);

    hipStream_t stream = static_cast<hipStream_t>(p->stream);
    const bool is_bf16 = p->dtype == S3R_BF16;
    const bool mfma = mfma_ok(p->dtype, p->block);
    const float scale = resolve_scale(p->softmax_scale, p->head_dim);
    void *ws = p->workspace;
    float *qc = reinterpret_cast<float *>(at(ws, L.qc));
    float *kc = reinterpret_cast<float *>(at(ws, L.kc));
    float *vc = reinterpret_cast<float *>(at(ws, L.vc));
    float *oc = p->o_comp ? p->o_comp : reinterpret_cast<float *>(at(ws, L.oc));
    // idx_sel: what the selection kernel reads ([heads][n_blk][width]); idx_dyn: what TopK writes.
    int32_t *idx_sel = p->topk_idx ? p->topk_idx
                                   : reinterpret_cast<int32_t *>(at(ws, n_forced > 0 ? L.idx_merged : L.idx));
    int32_t *idx_dyn = n_forced > 0 ? reinterpret_cast<int32_t *>(at(ws, L.idx)) : idx_sel;
    int32_t *forced_clean = reinterpret_cast<int32_t *>(at(ws, L.forced_clean));
    unsigned long long *forced_words =
        n_forced > 0 ? reinterpret_cast<unsigned long long *>(at(ws, L.forced_words)) : nullptr;
    void *tile[8];
    for (int a = 0; a < 8; ++a) tile[a] = at(ws, L.tile[a]);
    void *kb = mfma ? at(ws, L.kb) : nullptr;
    void *vb = mfma ? at(ws, L.vb) : nullptr;

    int32_t *blk_len = nullptr;
    {
        StageTimer tm(S3R_STAGE_POOL, stream);
        if (sp.windows) {
            blk_len = reinterpret_cast<int32_t *>(at(ws, L.blk_len));
            S3R_HIP(s3r::launch_block_lens(sp.img, p->block, sp.n_img, L.n_blk, blk_len, stream), "block length kernel launch");
        }
        S3R_HIP(s3r::launch_pool(p->q, p->k, p->v, qc, kc, vc, kb, vb, sp.n_img, p->heads, p->block, is_bf16,
                                 sp.img, in, stream),
                "pool kernel launch");
    }
    FusedBufs fb;
    fb.stat_slots = at(ws, L.stat_slots);
    fb.head_stats = reinterpret_cast<s3r::HeadStats *>(at(ws, L.head_stats));
    fb.thr = reinterpret_cast<float *>(at(ws, L.thr));
    fb.cand = reinterpret_cast<int32_t *>(at(ws, L.cand));
    fb.cand_count = reinterpret_cast<int *>(at(ws, L.cand_count));
    fb.overflow = reinterpret_cast<int *>(at(ws, L.overflow));
    if (n_forced > 0 || p->status != nullptr) {
        StageTimer tm(S3R_STAGE_TOPK, stream);
        S3R_HIP(s3r::launch_forced_prepare(p->forced_blocks, n_forced, L.n_blk, forced_clean, forced_words, p->status, stream),
                "forced-block prepare kernel launch");
    }
    st = run_compress_topk(qc, kc, vc, tile, reinterpret_cast<float *>(at(ws, L.s)), L.ld_s, L.head_chunk, oc,
                           idx_dyn, L.n_blk, L.tiles, p->heads, L.kk, scale, !is_bf16, true, forced_words, fb,
                           token_queries && mfma && is_bf16, stream);
    if (st != S3R_OK) return st;
    if (n_forced > 0) {
        StageTimer tm(S3R_STAGE_TOPK, stream);
        S3R_HIP(s3r::launch_merge_forced(idx_dyn, L.kk, forced_clean, n_forced, idx_sel,
                                         static_cast<int64_t>(p->heads) * L.n_blk, stream),
                "forced-block merge kernel launch");
    }

    float *oc_tok = nullptr;
    if (token_queries) {
        // Compression branch with unpooled queries: every image row's own query against the pooled keys,
        // i.e. dense attention over the pooled tensors (n_blk keys per head), result in fp32 per query
        // slot.  bf16 problems: the bf16 hi tiles of Kc, Vc written by the split kernel are already in
        // the unit layout of the MFMA kernel; fp32 problems: the generic kernel on Kc, Vc themselves.
        oc_tok = reinterpret_cast<float *>(at(ws, L.oc_tok));
        s3r::SelectArgs c{};
        c.q = p->q; c.qmap = sp.img; c.n_tok = sp.n_img; c.lse_stride = p->n_tok;
        c.n_keys = L.n_blk; c.n_blk = (L.n_blk + 63) / 64; c.block = 64; c.heads = p->heads;
        c.scale = scale; c.is_bf16 = is_bf16;
        c.x.out_f32 = oc_tok; c.x.q_blk_len = blk_len; c.x.q_block = p->block; c.x.in = in;
        StageTimer tm(S3R_STAGE_COMPRESS, stream);
        if (mfma && is_bf16) {
            c.kb = tile[2]; c.vb = tile[4];
            c.x.kv_head_stride = L.tiles * 32 * 64;
            S3R_HIP(s3r::launch_select_mfma(c, stream), "compression branch (unpooled queries) kernel launch");
        } else {
            c.k = kc; c.v = vc;
            c.x.k_row_stride = 64; c.x.k_head_stride = L.n_blk * 64;
            S3R_HIP(s3r::launch_select_generic(c, stream), "compression branch (unpooled queries) kernel launch");
        }
    }

    s3r::SelectArgs a{};
    a.x.o_comp_tok = oc_tok; a.x.in = in;
    a.n_common = n_forced;
    a.q = p->q; a.k = p->k; a.v = p->v; a.kb = kb; a.vb = vb; a.idx = idx_sel; a.o_comp = oc;
    a.gate = p->gate_logits; a.out = p->out; a.o_sel = p->o_sel; a.lse = p->lse_sel;
    a.n_tok = sp.n_img; a.n_keys = sp.n_img; a.n_blk = L.n_blk; a.lse_stride = p->n_tok;
    a.qmap = sp.img; a.kmap = sp.img; a.blk_len = blk_len;
    a.heads = p->heads; a.block = p->block; a.kk = L.width;
    a.scale = scale; a.is_bf16 = is_bf16;
    a.lo_off = (mfma && !is_bf16) ? static_cast<int64_t>(p->heads) * L.n_blk * p->block * 64 : 0;
    {
        StageTimer tm(S3R_STAGE_SELECT, stream);
        S3R_HIP(mfma ? s3r::launch_select_mfma(a, stream) : s3r::launch_select_generic(a, stream),
                "select kernel launch");
    }
    if (sp.n_spec > 0) {
        // Special tokens (Sec. 3.2 eq. 2): plain attention of those rows over every token.
        s3r::SelectArgs d{};
        d.q = p->q; d.k = p->k; d.v = p->v; d.idx = nullptr; d.o_comp = nullptr; d.gate = nullptr;
        d.out = p->out; d.o_sel = nullptr; d.lse = nullptr;
        d.n_tok = sp.n_spec; d.qmap = sp.spec; d.lse_stride = p->n_tok;
        d.heads = p->heads; d.block = p->block; d.kk = 0; d.scale = scale; d.is_bf16 = is_bf16;
        d.x.in = in;
        if (mfma) {
            void *kb_s = at(ws, L.kb_spec), *vb_s = at(ws, L.vb_spec);
            {
                StageTimer tm(S3R_STAGE_POOL, stream);
                S3R_HIP(s3r::launch_pool(p->q, p->k, p->v, nullptr, nullptr, nullptr, kb_s, vb_s, sp.n_spec, p->heads,
                                         64, is_bf16, sp.spec, in, stream),
                        "pool kernel launch (special tokens)");
            }
            d.kb = kb; d.vb = vb; d.n_keys = sp.n_img; d.n_blk = L.n_blk;      // image keys, then special keys
            d.blk_len = blk_len;
            d.kb2 = kb_s; d.vb2 = vb_s; d.n_keys2 = sp.n_spec;
            if (!is_bf16) {
                d.lo_off = a.lo_off;
                d.lo_off2 = static_cast<int64_t>(p->heads) * ((sp.n_spec + 63) / 64) * 64 * 64;
            }
            if (L.spec_split > 1) {
                d.x.n_split = L.spec_split;
                d.x.out_f32 = reinterpret_cast<float *>(at(ws, L.spec_part_o));
                d.x.part_lse = reinterpret_cast<float *>(at(ws, L.spec_part_lse));
            }
        } else {
            d.n_keys = p->n_tok; d.n_blk = (p->n_tok + p->block - 1) / p->block;  // every row, in place
        }
        StageTimer tm(S3R_STAGE_DENSE, stream);
        S3R_HIP(mfma ? s3r::launch_select_mfma(d, stream) : s3r::launch_select_generic(d, stream),
                "dense kernel launch (special tokens)");
        if (d.x.n_split > 1)
            S3R_HIP(s3r::launch_dense_combine(d.x.out_f32, d.x.part_lse, d.x.n_split, sp.n_spec, p->heads, sp.spec,
                                              p->out, is_bf16, stream),
                    "dense combine kernel launch (special tokens)");
    }
    return S3R_OK;
}

int speed3r_sparse_global_attn(const void *q, const void *k, const void *v, void *out, int64_t n_tok,
                               int heads, int head_dim, int block, int topk, void *stream)
{
    s3r_status st = check_shape(n_tok, heads, head_dim, block, topk, S3R_BF16);
    if (st != S3R_OK) return st;
    s3r_params p{};
    p.q = q; p.k = k; p.v = v; p.out = out;
    p.n_tok = n_tok; p.heads = heads; p.head_dim = head_dim; p.block = block; p.topk = topk;
    p.dtype = S3R_BF16; p.softmax_scale = 0.f; p.stream = stream;
    p.workspace_bytes = speed3r_workspace_bytes(n_tok, heads, head_dim, block, topk, 0, S3R_BF16);
    st = scratch_get(p.workspace_bytes, &p.workspace);
    if (st != S3R_OK) return st;
    return speed3r_sparse_global_attn_ex(&p);
}

int speed3r_sparse_global_attn_noalloc(const void *q, const void *k, const void *v, void *out, int64_t n_tok,
                                       int heads, int head_dim, int block, int topk, void *stream)
{
    s3r_status st = check_shape(n_tok, heads, head_dim, block, topk, S3R_BF16);
    if (st != S3R_OK) return st;
    const size_t need = speed3r_workspace_bytes(n_tok, heads, head_dim, block, topk, 0, S3R_BF16);
    if (need == 0 || need > kStaticScratchBytes)
        return fail(S3R_ERR_WORKSPACE,
                    "problem needs %zu bytes of scratch, the static scratch of this entry point holds %zu: "
                    "use speed3r_sparse_global_attn_ex with a caller workspace",
                    need, kStaticScratchBytes);
    s3r_params p{};
    p.q = q; p.k = k; p.v = v; p.out = out;
    p.n_tok = n_tok; p.heads = heads; p.head_dim = head_dim; p.block = block; p.topk = topk;
    p.dtype = S3R_BF16; p.softmax_scale = 0.f; p.stream = stream;
    p.workspace_bytes = kStaticScratchBytes;
    st = static_scratch(&p.workspace);
    if (st != S3R_OK) return st;
    // nothing of the previous call's scratch contents is relied on: every flag and counter the kernels
    // read is cleared by a kernel of this call
    t_no_events = true;
    st = speed3r_sparse_global_attn_ex(&p);
    t_no_events = false;
    return st;
}

s3r_status speed3r_pool_blocks(const void *q, const void *k, const void *v, float *qc, float *kc, float *vc,
                               int64_t n_tok, int heads, int head_dim, int block, s3r_dtype dtype, void *stream)
{
    s3r_status st = check_shape(n_tok, heads, head_dim, block, 1, dtype);
    if (st != S3R_OK) return st;
    if (!q || !k || !v || !qc || !kc || !vc) return fail(S3R_ERR_INVALID_ARG, "all six tensors must be non-null");
    if (!aligned16(q) || !aligned16(k) || !aligned16(v)) return fail(S3R_ERR_INVALID_ARG, "device pointers must be 16-byte aligned");
    StageTimer tm(S3R_STAGE_POOL, static_cast<hipStream_t>(stream));
    S3R_HIP(s3r::launch_pool(q, k, v, qc, kc, vc, nullptr, nullptr, n_tok, heads, block, dtype == S3R_BF16,
                             s3r::TokenMap{}, s3r::InStride{}, static_cast<hipStream_t>(stream)),
            "pool kernel launch");
    return S3R_OK;
}

s3r_status speed3r_compress_attn_scores(const float *qc, const float *kc, const float *vc, float *s_guide,
                                        int64_t ld_s, float *o_comp, int64_t n_blk, int heads, int head_dim,
                                        float softmax_scale, int accurate_pv, void *stream)
{
    if (n_blk <= 0 || heads <= 0 || heads > 65535) return fail(S3R_ERR_INVALID_ARG, "n_blk and heads must be positive");
    if (head_dim != 64) return fail(S3R_ERR_UNSUPPORTED, "head_dim %d unsupported (must be 64)", head_dim);
    if (!qc || !kc || !vc || !s_guide || !o_comp) return fail(S3R_ERR_INVALID_ARG, "all five tensors must be non-null");
    if (ld_s < n_blk || ld_s % 4 != 0) return fail(S3R_ERR_INVALID_ARG, "ld_s must be >= n_blk and a multiple of 4");
    if (!aligned16(s_guide) || !aligned16(o_comp)) return fail(S3R_ERR_INVALID_ARG, "s_guide and o_comp must be 16-byte aligned");
    const int64_t tiles = s3r::pooled_tiles_padded(n_blk);
    const size_t arr = align_up(static_cast<size_t>(heads) * tiles * 32 * 64 * 2);
    void *ws = nullptr;
    s3r_status st = scratch_get(8 * arr, &ws);
    if (st != S3R_OK) return st;
    void *tile[8];
    for (int a = 0; a < 8; ++a) tile[a] = at(ws, a * arr);
    return run_compress_topk(qc, kc, vc, tile, s_guide, ld_s, heads, o_comp, nullptr, n_blk, tiles, heads, 0,
                             resolve_scale(softmax_scale, head_dim), accurate_pv != 0, false, nullptr, FusedBufs{}, false,
                             static_cast<hipStream_t>(stream));
}

s3r_status speed3r_compress_attn_topk(const float *qc, const float *kc, const float *vc, float *o_comp, int32_t *idx,
                                      int64_t n_blk, int heads, int head_dim, int topk, float softmax_scale,
                                      int accurate_pv, void *stream)
{
    if (n_blk <= 0 || heads <= 0 || heads > 65535 || topk <= 0)
        return fail(S3R_ERR_INVALID_ARG, "n_blk, heads and topk must be positive");
    if (head_dim != 64) return fail(S3R_ERR_UNSUPPORTED, "head_dim %d unsupported (must be 64)", head_dim);
    if (!qc || !kc || !vc || !o_comp || !idx) return fail(S3R_ERR_INVALID_ARG, "all five tensors must be non-null");
    if (!aligned16(qc) || !aligned16(kc) || !aligned16(o_comp))
        return fail(S3R_ERR_INVALID_ARG, "qc, kc and o_comp must be 16-byte aligned");
    if (n_blk * heads > 0x7fffffffLL) return fail(S3R_ERR_UNSUPPORTED, "n_blk * heads exceeds 2^31 - 1");
    const int kk = static_cast<int>(topk < n_blk ? topk : n_blk);
    if (kk > s3r::kFusedTopkMaxK) return fail(S3R_ERR_UNSUPPORTED, "k = %d exceeds %d", kk, s3r::kFusedTopkMaxK);
    if (g_kernel_choice == 2) return fail(S3R_ERR_UNSUPPORTED, "TopK inside the sweep is switched off (kernel choice 2)");
    // scratch: six operand tile arrays, bounds, candidate lists and counts, overflow word, and S for the
    // fallback in head chunks
    const int64_t tiles = s3r::pooled_tiles_padded(n_blk);
    const size_t arr = align_up(static_cast<size_t>(heads) * tiles * 32 * 64 * 2);
    const size_t rows = static_cast<size_t>(heads) * n_blk;
    const int64_t ld_s = (n_blk + 63) / 64 * 64;
    const size_t per_head_s = static_cast<size_t>(n_blk) * ld_s * sizeof(float);
    int64_t hc = static_cast<int64_t>(kScoreBytesCap / per_head_s);
    if (hc < 1) hc = 1;
    if (hc > heads) hc = heads;
    size_t off = 8 * arr;
    auto take = [&](size_t bytes) { const size_t o = off; off += align_up(bytes); return o; };
    const size_t o_slots = take(static_cast<size_t>(heads) * 3 * s3r::kStatSlots * sizeof(unsigned));
    const size_t o_stats = take(static_cast<size_t>(heads) * sizeof(s3r::HeadStats));
    const size_t o_thr = take(rows * sizeof(float));
    const size_t o_cand = take(rows * 2 * kCandCap * sizeof(int32_t));
    const size_t o_cnt = take(rows * 2 * sizeof(int));
    const size_t o_ovf = take(sizeof(int));
    const size_t o_s = take(per_head_s * hc);
    void *ws = nullptr;
    s3r_status st = scratch_get(off, &ws);
    if (st != S3R_OK) return st;
    void *tile[8];
    for (int a = 0; a < 8; ++a) tile[a] = at(ws, a * arr);
    FusedBufs fb;
    fb.stat_slots = at(ws, o_slots);
    fb.head_stats = reinterpret_cast<s3r::HeadStats *>(at(ws, o_stats));
    fb.thr = reinterpret_cast<float *>(at(ws, o_thr));
    fb.cand = reinterpret_cast<int32_t *>(at(ws, o_cand));
    fb.cand_count = reinterpret_cast<int *>(at(ws, o_cnt));
    fb.overflow = reinterpret_cast<int *>(at(ws, o_ovf));
    return run_compress_topk(qc, kc, vc, tile, reinterpret_cast<float *>(at(ws, o_s)), ld_s, static_cast<int>(hc), o_comp,
                             idx, n_blk, tiles, heads, kk, resolve_scale(softmax_scale, head_dim), accurate_pv != 0, true,
                             nullptr, fb, false, static_cast<hipStream_t>(stream));
}

s3r_status speed3r_topk_blocks(const float *s_guide, int64_t ld_s, int32_t *idx, int64_t n_blk, int heads,
                               int topk, void *stream)
{
    if (n_blk <= 0 || heads <= 0 || topk <= 0) return fail(S3R_ERR_INVALID_ARG, "n_blk, heads and topk must be positive");
    if (!s_guide || !idx) return fail(S3R_ERR_INVALID_ARG, "s_guide and idx must be non-null");
    if (ld_s < n_blk) return fail(S3R_ERR_INVALID_ARG, "ld_s must be >= n_blk");
    if (n_blk * heads > 0x7fffffffLL) return fail(S3R_ERR_UNSUPPORTED, "n_blk * heads exceeds 2^31 - 1");
    const int kk = static_cast<int>(topk < n_blk ? topk : n_blk);
    StageTimer tm(S3R_STAGE_TOPK, static_cast<hipStream_t>(stream));
    S3R_HIP(s3r::launch_topk(s_guide, ld_s, idx, n_blk, n_blk * heads, kk, nullptr, static_cast<hipStream_t>(stream)),
            "topk kernel launch");
    return S3R_OK;
}

s3r_status speed3r_select_attn(const void *q, const void *k, const void *v, const int32_t *idx,
                               const float *o_comp, const void *gate_logits, void *out, void *o_sel,
                               float *lse, int64_t n_tok, int heads, int head_dim, int block, int kk,
                               s3r_dtype dtype, float softmax_scale, void *stream)
{
    s3r_status st = check_shape(n_tok, heads, head_dim, block, kk, dtype);
    if (st != S3R_OK) return st;
    if (!q || !k || !v || !idx || !out) return fail(S3R_ERR_INVALID_ARG, "q, k, v, idx and out must be non-null");
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(gate_logits) ||
        !aligned16(o_sel) || !aligned16(o_comp))
        return fail(S3R_ERR_INVALID_ARG, "device pointers must be 16-byte aligned");
    const int64_t n_blk = (n_tok + block - 1) / block;
    if (kk > n_blk) return fail(S3R_ERR_INVALID_ARG, "k (%d) exceeds the number of blocks (%lld)", kk, static_cast<long long>(n_blk));
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool mfma = mfma_ok(dtype, block);
    s3r::SelectArgs a{};
    if (mfma) {
        const size_t blocked = align_up(static_cast<size_t>(heads) * n_blk * block * 64 * 2 * tile_parts(dtype));
        void *ws = nullptr;
        st = scratch_get(2 * blocked, &ws);
        if (st != S3R_OK) return st;
        a.kb = ws;
        a.vb = at(ws, blocked);
        a.lo_off = dtype == S3R_BF16 ? 0 : static_cast<int64_t>(heads) * n_blk * block * 64;
        StageTimer tm(S3R_STAGE_POOL, s);
        S3R_HIP(s3r::launch_pool(q, k, v, nullptr, nullptr, nullptr, const_cast<void *>(a.kb),
                                 const_cast<void *>(a.vb), n_tok, heads, block, dtype == S3R_BF16, s3r::TokenMap{},
                                 s3r::InStride{}, s),
                "pool kernel launch");
    }
    a.q = q; a.k = k; a.v = v; a.idx = idx; a.o_comp = o_comp; a.gate = gate_logits; a.out = out;
    a.o_sel = o_sel; a.lse = lse; a.n_tok = n_tok; a.n_keys = n_tok; a.lse_stride = n_tok; a.n_blk = n_blk;
    a.heads = heads; a.block = block;
    a.kk = kk; a.scale = resolve_scale(softmax_scale, head_dim); a.is_bf16 = dtype == S3R_BF16;
    StageTimer tm(S3R_STAGE_SELECT, s);
    S3R_HIP(mfma ? s3r::launch_select_mfma(a, s) : s3r::launch_select_generic(a, s), "select kernel launch");
    return S3R_OK;
}

s3r_status speed3r_probe_select_loads(const void *q, const void *k, const void *v, const int32_t *idx, void *out,
                                      int64_t n_tok, int heads, int head_dim, int block, int kk, int ring_stages,
                                      int wg_per_cu, void *stream)
{
    s3r_status st = check_shape(n_tok, heads, head_dim, block, kk, S3R_BF16);
    if (st != S3R_OK) return st;
    if (block != 64 && block != 128) return fail(S3R_ERR_UNSUPPORTED, "the load probe covers blocks of 64 and 128 tokens");
    if (ring_stages != 0 && (ring_stages < 2 || ring_stages > 4))
        return fail(S3R_ERR_INVALID_ARG, "ring_stages (%d) must be 0 or 2..4", ring_stages);
    if (wg_per_cu < 0 || wg_per_cu > 5 || (wg_per_cu > 0 && 160 / wg_per_cu < 16 * (ring_stages ? ring_stages : 2)))
        return fail(S3R_ERR_INVALID_ARG, "wg_per_cu (%d) must be 0 or 1..5 and leave each workgroup room for a ring of %d stages of 16 KiB",
                    wg_per_cu, ring_stages ? ring_stages : 2);
    if (!q || !k || !v || !idx || !out) return fail(S3R_ERR_INVALID_ARG, "q, k, v, idx and out must be non-null");
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out))
        return fail(S3R_ERR_INVALID_ARG, "device pointers must be 16-byte aligned");
    const int64_t n_blk = (n_tok + block - 1) / block;
    if (kk > n_blk) return fail(S3R_ERR_INVALID_ARG, "k (%d) exceeds the number of blocks (%lld)", kk, static_cast<long long>(n_blk));
    hipStream_t s = static_cast<hipStream_t>(stream);
    const size_t blocked = align_up(static_cast<size_t>(heads) * n_blk * block * 64 * 2);
    void *ws = nullptr;
    st = scratch_get(2 * blocked, &ws);
    if (st != S3R_OK) return st;
    s3r::SelectArgs a{};
    a.kb = ws;
    a.vb = at(ws, blocked);
    {
        StageTimer tm(S3R_STAGE_POOL, s);
        S3R_HIP(s3r::launch_pool(q, k, v, nullptr, nullptr, nullptr, const_cast<void *>(a.kb), const_cast<void *>(a.vb),
                                 n_tok, heads, block, true, s3r::TokenMap{}, s3r::InStride{}, s),
                "pool kernel launch");
    }
    a.q = q; a.k = k; a.v = v; a.idx = idx; a.out = out;
    a.n_tok = n_tok; a.n_keys = n_tok; a.lse_stride = n_tok; a.n_blk = n_blk;
    a.heads = heads; a.block = block; a.kk = kk; a.scale = 1.f; a.is_bf16 = true; a.loads_only = true;
    a.probe_stages = ring_stages; a.probe_wg_per_cu = wg_per_cu;
    StageTimer tm(S3R_STAGE_SELECT, s);
    S3R_HIP(s3r::launch_select_mfma(a, s), "select (loads only) kernel launch");
    return S3R_OK;
}

s3r_status speed3r_dense_attn(const void *q, const void *k, const void *v, void *out, float *lse, int64_t n_tok,
                              int heads, int head_dim, s3r_dtype dtype, float softmax_scale, void *stream)
{
    const int block = 64;
    s3r_status st = check_shape(n_tok, heads, head_dim, block, 1, dtype);
    if (st != S3R_OK) return st;
    if (!q || !k || !v || !out) return fail(S3R_ERR_INVALID_ARG, "q, k, v and out must be non-null");
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out))
        return fail(S3R_ERR_INVALID_ARG, "device pointers must be 16-byte aligned");
    const int64_t n_blk = (n_tok + block - 1) / block;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool mfma = mfma_ok(dtype, block);
    s3r::SelectArgs a{};
    if (mfma) {
        const size_t blocked = align_up(static_cast<size_t>(heads) * n_blk * block * 64 * 2 * tile_parts(dtype));
        void *ws = nullptr;
        st = scratch_get(2 * blocked, &ws);
        if (st != S3R_OK) return st;
        a.kb = ws;
        a.vb = at(ws, blocked);
        a.lo_off = dtype == S3R_BF16 ? 0 : static_cast<int64_t>(heads) * n_blk * block * 64;
        StageTimer tm(S3R_STAGE_POOL, s);
        S3R_HIP(s3r::launch_pool(q, k, v, nullptr, nullptr, nullptr, const_cast<void *>(a.kb),
                                 const_cast<void *>(a.vb), n_tok, heads, block, dtype == S3R_BF16, s3r::TokenMap{},
                                 s3r::InStride{}, s),
                "pool kernel launch");
    }
    a.q = q; a.k = k; a.v = v; a.idx = nullptr; a.o_comp = nullptr; a.gate = nullptr; a.out = out;
    a.o_sel = nullptr; a.lse = lse; a.n_tok = n_tok; a.n_keys = n_tok; a.lse_stride = n_tok; a.n_blk = n_blk;
    a.heads = heads; a.block = block;
    a.kk = 0; a.scale = resolve_scale(softmax_scale, head_dim); a.is_bf16 = dtype == S3R_BF16;
    StageTimer tm(S3R_STAGE_DENSE, s);
    S3R_HIP(mfma ? s3r::launch_select_mfma(a, s) : s3r::launch_select_generic(a, s), "dense kernel launch");
    return S3R_OK;
}

// ---- cross attention ---------------------------------------------------------------------------------
namespace {

constexpr int64_t kMaxRowHeads = int64_t(1) << 28;  // rows * heads: 16 threads each stay below the 2^32 of a launch

bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

s3r_status check_heads(int heads, int kv_heads, int head_dim, int dtype)
{
    if (heads <= 0 || kv_heads <= 0 || heads % kv_heads != 0)
        return fail(S3R_ERR_INVALID_ARG, "heads (%d) must be a positive multiple of kv_heads (%d)", heads, kv_heads);
    if (heads > 65535) return fail(S3R_ERR_UNSUPPORTED, "heads %d unsupported (max 65535)", heads);
    if (head_dim != 64) return fail(S3R_ERR_UNSUPPORTED, "head_dim %d unsupported (must be 64)", head_dim);
    if (dtype != S3R_F32 && dtype != S3R_BF16) return fail(S3R_ERR_UNSUPPORTED, "unknown dtype %d", dtype);
    return S3R_OK;
}

// A workgroup looks for its sequence 64 at a time, and a launch of few rows has up to four workgroups of 1024 threads for a sequence
// and head.
s3r_status check_batch(int batch, int kv_heads)
{
    if (batch > 65536 || batch > (1 << 19) / kv_heads)
        return fail(S3R_ERR_UNSUPPORTED, "batch (%d) exceeds 65536, or batch * kv_heads 2^19", batch);
    return S3R_OK;
}

s3r_status check_strides(const char *what, int64_t tok, int64_t head)
{
    if (tok < 0 || head < 0 || tok % 8 != 0 || head % 8 != 0)
        return fail(S3R_ERR_INVALID_ARG, "the strides of %s (%lld, %lld) must be non-negative multiples of 8 elements", what,
                    static_cast<long long>(tok), static_cast<long long>(head));
    return S3R_OK;
}

// Pieces that the streamed units are divided into, a workgroup for each, by a model of the launch in microseconds.  A CU works through
// n = ceil(workgroups * pieces / 256) of them, `resident` at a time; one alone on a CU takes half as long again as its share
// of a full one.  A workgroup takes `unit_us` for each unit and two units' time to start and end; more than one piece costs a launch that
// joins them (3.5 us, and `part_bytes` of partial results for a piece at 5 TB/s; their way out is under the work).  A piece has
// `least` units or more.
// Measured, 16 heads: 1374 rows over 27480 keys (176 workgroups) in 3 pieces 300 us, in 10 215-238 and 13 to join them; gradient of q,
// 2748 rows over 10992 keys (352), in 2 pieces 335, in 4 255 and 16.
struct Pace { double unit_us; int resident, least, uneven; };
constexpr Pace kCrossPace[2] = {{2.2, 2, 3, 256}, {0.67, 4, 4, 512}};  // [bf16]
constexpr Pace kGradQPace[2] = {{5.5, 1, 3, 256}, {1.1, 2, 4, 512}};
constexpr Pace kGradKvPace[2] = {{7.3, 1, 3, 256}, {1.3, 2, 4, 512}};
constexpr Pace kCachePace[2] = {{2.0, 2, 3, 256}, {0.85, 3, 4, 512}};
constexpr int kFewLeast = 4;
int pieces(int64_t workgroups, int64_t units, const Pace &pace, double part_bytes)
{
    auto time_us = [&](int s) {
        const int64_t n = (workgroups * s + 255) / 256, rest = n % pace.resident;
        const double share = static_cast<double>(n) + (rest == 0 ? 0.0 : 0.5 - 0.5 * static_cast<double>(rest - 1) / pace.resident);
        return share * static_cast<double>((units + s - 1) / s + 2) * pace.unit_us + (s == 1 ? 0.0 : 3.5 + s * part_bytes / 5e6);
    };
    int most = 1;
    double shortest = time_us(1);
    while (most < s3r::kMostSplits && units >= static_cast<int64_t>(pace.least) * (most + 1)) {
        const double us = time_us(++most);
        if (us < shortest) shortest = us;
    }
    for (int s = 1; s < most; ++s)
        if (time_us(s) <= 1.01 * shortest) return s;  // the fewest that come within 1 %: their partial results take workspace
    return most;
}

// The same for sequences of several lengths, or causal rows, of which only the mean (or the longest) is known here: the longer they are, the
// further apart they can be, and the more workgroups level that out.  16 of them for every unit, up to five for each CU, and at least
// `uneven`; short ones are left whole where most CUs have a workgroup.  `most`: units of the longest.  Measured, us, forward / gradient
// (workgroups, units): bf16, 16 times 200 rows over 500 keys (256, 8) in 1 14 / 36, in 2 24 / 51; 17 rows over 28 to 4329 keys (119, 16) gradient
// in 3 72, in 5 65; 2000, 700 and 100 rows over 4000, 1000 and 9000 keys (360, 73) in 2 109 / 285, 4 95 / 268; 4 times 1374 over 2748 (704, 43)
// in 1 91 / 291, 2 103 / 319; 5000 and 300 over 9000 and 700 (672, 76) in 1 249 / 848, 2 231 / 810; fp32 300, 20, 900 and 64 over 3000, 8000,
// 100 and 600 (48, 47) in 9 61 / 235, 16 49 / 188; 500, 1 and 129 over 1369, 700 and 64 (42, 11) in 6 29 / 83, 12 33 / 93.
int pieces_uneven(int64_t workgroups, int64_t units, int64_t most, const Pace &pace)
{
    const int64_t least = workgroups >= 192 ? 256 : pace.uneven, all = 16 * units < least ? least : (units >= 80 ? 1280 : 16 * units);
    int64_t s = (all + workgroups - 1) / workgroups;
    if (s > most / pace.least) s = most / pace.least;
    return s < 1 ? 1 : (s > s3r::kMostSplits ? s3r::kMostSplits : static_cast<int>(s));
}

// The same where a workgroup holds few rows and its waves take the units in turn.  Undivided, it has `waves` of them, takes `whole_us` for
// a round and `start` rounds' time to start and end; divided, it has four, and takes `unit_us` for a round as one of `resident` on a
// CU, half as long again as its share alone, and up to 40 % less where few CUs are busy, a round and a quarter to start and end; joining
// takes `join_us` and 0.03 for a piece.  Only as many pieces are looked at as fill the CUs once, twice .. and 64 and 128, with a unit at
// least for each wave.  `workgroups`: were the sequences all as long as their mean.
// Measured / by this model, us, one row for a head (workgroups, units): cross bf16 (16, 172) in 43 pieces 17.0, 16 15.2 / 15.5; (64, 94) 16
// 26, 4 23 / 23; (1, 2147) 256 21.4, 128 19.8 / 21; (16, 10) 2 9.5 / 9.6, 1 7.4 / 7.5; fp32 (64, 94) 16 80, 4 55 / 53; (128, 24) 2 35 / 33, 1
// 48 / 49; cache bf16 (128, 94) 8 20 / 20, 2 27, 1 23 / 22; (16, 2147) 64 38 / 42, 16 58; (64, 24) 6 9.8 / 9.7, 1 9.7 / 9.3; fp32 (128, 94) 6
// 25 / 26, 1 36 / 34.
struct FewPace { double unit_us; int resident; double join_us, whole_us, start; int waves; };
constexpr FewPace kCrossFew[2] = {{6.7, 1, 4.0, 6.7, 1.25, 4}, {2.6, 1, 4.0, 3.0, 1.25, 8}};  // [bf16]
constexpr FewPace kCacheFew[2] = {{1.33, 3, 5.0, 2.45, 2.1, 8}, {0.85, 4, 5.0, 3.0, 1.6, 16}};
int pieces_few(int64_t workgroups, int64_t units, const FewPace &pace)
{
    int best = 1;
    double shortest = static_cast<double>((workgroups + 255) / 256) * (static_cast<double>(units) / pace.waves + pace.start) * pace.whole_us;
    auto look = [&](int64_t s) {
        if (s > units / 4) s = units / 4;
        if (s > s3r::kMostSplits) s = s3r::kMostSplits;
        if (s < 2) return;
        const int64_t all = workgroups * s, n = (all + 255) / 256, rest = n % pace.resident, rounds = ((units + s - 1) / s + 3) / 4;
        const double share = static_cast<double>(n) + (rest == 0 ? 0.0 : 0.5 - 0.5 * static_cast<double>(rest - 1) / pace.resident);
        const double busy = all < 256 ? 0.6 + 0.4 * static_cast<double>(all) / 256 : 1.0;
        const double us = share * busy * (static_cast<double>(rounds) + 1.25) * pace.unit_us + pace.join_us + 0.03 * static_cast<double>(s);
        if (us < shortest) {
            shortest = us;
            best = static_cast<int>(s);
        }
    };
    for (int n = 1; n <= pace.resident; ++n) look(256 * n / workgroups);
    look(64);
    look(128);
    return best;
}
// Tiles, were the sequences all as long as their mean.
int64_t mean_tiles(int64_t n, int per_row, int tile, int batch)
{
    const int64_t some = n < batch ? (n < 1 ? 1 : n) : batch, each = (n * per_row + some - 1) / some;
    return some * (each < 1 ? 1 : (each + tile - 1) / tile);
}

// The same for causal rows: `tiles` (heads counted) walk `units` units on average, the longest of them `longest`, and all are divided alike.  They
// are taken the longest first, so that the short ones fill the CUs up.  The work takes its time at the pace of as many workgroups as a CU
// has (alone half as long again), and the longest piece twice its share at the pace of a full CU, or 1.6 times where two fill it; joining
// 9 us and `tile_us` for each tile's piece, out and in again.
// Measured (1, 2, 3, 4 .. pieces), us: forward, bf16, 4096 rows of 16 heads that share 4 87 / 75 / 79 / 87, 1374 of 16 38 / 31 / 32 / 33, 512 over
// 16384 285 / 156 / 112 / 93, 8 69, 12 67, 16 66, 32 75, 8192 in three sequences 93 / 108 / 119 / 134; the whole step with gradients of keys
// in these: 8192 in three sequences 599 / 437 / 398 / 385, 6 391, 8 420; 4096 568 / 388 / 337 / 310, 6 293, 8 302.
double causal_us(int n, double tiles, double units, double longest, const Pace &pace, double join_us, double tile_us)
{
    const double all = tiles * units / 256 * pace.unit_us, alone = pace.resident > 2 ? 2.0 : (pace.resident > 1 ? 1.6 : 1.1);
    const double on_a_cu = tiles * n / 256, k = on_a_cu < 1 ? 1 : (on_a_cu > pace.resident ? pace.resident : on_a_cu);
    const double work = all * (pace.resident > 1 ? 1.5 - 0.5 * (k - 1) / (pace.resident - 1) : 1.0), piece = alone * longest / n * pace.unit_us;
    return (work > piece ? work : piece) + (n == 1 ? 0.0 : join_us + tiles * n * tile_us);
}
constexpr double kJoinUs = 9.0;
int causal_pieces(double tiles, double units, double longest, const Pace &pace, double tile_bytes)
{
    int best = 1;
    double least_us = causal_us(1, tiles, units, longest, pace, kJoinUs, tile_bytes * 2 / 5e6);
    for (int n = 2; n <= s3r::kMostSplits && longest >= static_cast<double>(pace.least) * n; ++n) {
        const double us = causal_us(n, tiles, units, longest, pace, kJoinUs, tile_bytes * 2 / 5e6);
        if (us < 0.99 * least_us) {
            least_us = us;
            best = n;
        }
    }
    return best;
}
// Of 2 to 64 sequences: the most pieces that their lengths may ask for, where one of them may have all the `longest` units.  What is left over of the
// grid, and a launch that may find nothing to join, cost some us for each kernel: as many as make 1024 workgroups, 8 at most, and
// only where that promises half the time.  (The kernels find the number that the lengths do ask for, causal_split.)
int causal_most_pieces(int guess, double tiles, double units, double longest, const Pace &pace, double tile_bytes)
{
    const int n = std::min({causal_pieces(tiles, units, longest, pace, tile_bytes), 8, static_cast<int>(1024 / tiles)});
    auto us = [&](int k) { return causal_us(k, tiles, units, longest, pace, kJoinUs, tile_bytes * 2 / 5e6); };
    return n > guess && us(guess) > 2 * us(n) ? n : guess;
}

struct CrossPlan {
    bool few_rows, adapts, adapts_q, adapts_kv;  // causal: kernels take fewer pieces by the sequences' lengths
    int batch, per_row, split, least, split_q, split_kv;
    int64_t tiles, q_tiles, kv_tiles;
    size_t part_o, part_lse, forward;                   // workspace of the forward call
    size_t stats, part_q, part_pk, part_sum, part_k, part_v, backward;     // of the gradient
};

// view: tokens of a view whose rows see those of their own and of earlier ones, 0: all rows see all keys.
s3r_status plan_cross(const s3r_cross_params *p, int view, CrossPlan *out)
{
    if (!p) return fail(S3R_ERR_INVALID_ARG, "params is null");
    s3r_status st = check_heads(p->heads, p->kv_heads, p->head_dim, p->dtype);
    if (st != S3R_OK) return st;
    if (p->n_q < 0 || p->n_kv < 0) return fail(S3R_ERR_INVALID_ARG, "n_q and n_kv must not be negative");
    if (p->batch < 0 || (p->batch > 1 && !p->q_start))
        return fail(S3R_ERR_INVALID_ARG, "batch (%d) must be 1 without q_start and kv_start, and never negative", p->batch);
    if ((p->q_start != nullptr) != (p->kv_start != nullptr)) return fail(S3R_ERR_INVALID_ARG, "q_start and kv_start must be given together");
    if (p->q_start && p->batch == 0) return fail(S3R_ERR_INVALID_ARG, "batch must be positive with q_start and kv_start");
    CrossPlan c{};
    c.batch = p->batch == 0 ? 1 : p->batch;
    c.per_row = p->heads / p->kv_heads;
    if (p->n_q > kMaxRowHeads / p->heads || p->n_kv > kMaxRowHeads / p->kv_heads) return fail(S3R_ERR_UNSUPPORTED, "rows * heads exceeds 2^28");
    st = check_batch(c.batch, p->kv_heads);
    if (st != S3R_OK) return st;
    const int bf16 = p->dtype == S3R_BF16;
    const bool uneven = c.batch > 1 || view > 0;
    // (the longest of several sequences counts, and only their sum is known: four times their mean, if there is that much)
    auto units_of = [&](int64_t rows) { return ((uneven ? (4 * rows / c.batch < rows ? 4 * rows / c.batch : rows) : rows) + 63) / 64; };
    auto split_of = [&](int64_t tiles, int64_t held, int per_row, int64_t streamed, const Pace &pace, double part_bytes) {
        if (!uneven) return pieces(tiles * p->kv_heads, units_of(streamed), pace, part_bytes);
        return pieces_uneven(mean_tiles(held, per_row, 128, c.batch) * p->kv_heads, streamed / c.batch / 64 + 1, units_of(streamed), pace);
    };
    const int64_t items = p->n_q * c.per_row, units = units_of(p->n_kv);
    const double q_bytes = 256.0 * static_cast<double>(p->n_q) * p->heads, kv_bytes = 512.0 * static_cast<double>(p->n_kv) * p->kv_heads;
    // Few rows for a sequence: tiles of 16, which bring the keys in once each, in place of one of 128, whose waves are mostly idle: more of
    // them the smaller keys and values are beside the L2s (us, one of 128 / tiles of 16: 64 rows over 2000 keys of 16 heads 12.6 / 10.6, 48
    // over 20000 of 4 heads 15.1 / 16.0; 32 over 10992 of 16 heads (45 MB) 19.9 / 19.0, over 137400 of 16 122 / 168; fp32 64 over 2000
    // 23.7 / 22.5, 32 over 10992 (90 MB) 43.8 / 50.5).
    const int64_t kv_tensors = p->n_kv * p->kv_heads * (bf16 ? 256 : 512);
    c.few_rows = items <= int64_t(kv_tensors <= (16 << 20) ? 64 : (kv_tensors <= (48 << 20) ? 32 : 16)) * c.batch;
    c.tiles = s3r::most_tiles(p->n_q, c.per_row, c.few_rows ? 16 : 128, c.batch);
    c.split = c.few_rows ? pieces_few(mean_tiles(p->n_q, c.per_row, 16, c.batch) * p->kv_heads, units, kCrossFew[bf16])
                         : split_of(c.tiles, p->n_q, c.per_row, p->n_kv, kCrossPace[bf16], q_bytes);
    c.least = c.few_rows ? kFewLeast : kCrossPace[bf16].least;
    c.q_tiles = s3r::most_tiles(p->n_q, c.per_row, 128, c.batch);
    c.split_q = split_of(c.q_tiles, p->n_q, c.per_row, p->n_kv, kGradQPace[bf16], bf16 ? 2 * q_bytes : q_bytes);
    c.kv_tiles = s3r::most_tiles(p->n_kv, 1, 128, c.batch);
    c.split_kv = split_of(c.kv_tiles, p->n_kv, 1, items, kGradKvPace[bf16], kv_bytes);
    if (view > 0) {
        // Of several sequences only the sums of their lengths are known: the longest is taken to be 1.75 times their mean.  (Where there are few
        // tiles, and it may be far longer, the kernels are given room for more pieces, and find how many by themselves.)
        const double n = static_cast<double>(p->n_q) / c.batch, m = static_cast<double>(p->n_kv) / c.batch, v = view < m ? view : m;
        const double spread = c.batch > 1 ? 1.75 : 1.0, first = m > n ? m - n + v : v;
        const double most = m * spread / 64 + 0.5, least = first < m ? first / 64 + 0.5 : most;
        const double q_tiles = static_cast<double>(mean_tiles(p->n_q, c.per_row, 128, c.batch)) * p->kv_heads, tile_bytes = 128.0 * 256;
        // Keys: the first ones are seen by all rows, the last ones by a view's, or by all where there are earlier tokens.
        const double rows = n * c.per_row / 64, kv_tiles = static_cast<double>(mean_tiles(p->n_kv, 1, 128, c.batch)) * p->kv_heads, few = (m > n ? rows * (m - n) / m : 0.0) + 0.5;
        const double mean_q = ((first < m ? first : m) + m) / 128 + 0.5, mean_k = (rows + few) / 2 + 0.5;
        auto split = [&](double tiles, double shortest, double longest, double mean, double total, const Pace &pace, double bytes, bool *adapts) {
            const int guess = causal_pieces(tiles, (shortest + longest) / 2, longest, pace, bytes);
            const int n = c.batch > 1 && c.batch <= 64 ? causal_most_pieces(guess, tiles, mean, total, pace, bytes) : guess;
            *adapts = n > guess;
            return n;
        };
        if (!c.few_rows) c.split = split(q_tiles, least, most, mean_q, m * c.batch / 64 + 0.5, kCrossPace[bf16], tile_bytes, &c.adapts);
        c.split_q = split(q_tiles, least, most, mean_q, m * c.batch / 64 + 0.5, kGradQPace[bf16], bf16 ? 2 * tile_bytes : tile_bytes, &c.adapts_q);
        c.split_kv = split(kv_tiles, few, rows * spread + 0.5, mean_k, rows * c.batch + 0.5, kGradKvPace[bf16], 2 * tile_bytes, &c.adapts_kv);
    }
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t o = off; off += align_up(bytes); return o; };
    const size_t rows = static_cast<size_t>(p->n_q) * p->heads, keys = static_cast<size_t>(p->n_kv) * p->kv_heads;
    c.part_o = take(c.split > 1 ? c.split * rows * 64 * sizeof(float) : 0);
    c.part_lse = take(c.split > 1 ? c.split * rows * sizeof(float) : 0);
    c.forward = off;
    off = 0;
    c.stats = take(rows * 2 * sizeof(float));
    c.part_q = take(c.split_q > 1 ? c.split_q * rows * 64 * sizeof(float) : 0);
    const bool mend = c.split_q > 1 && bf16;
    c.part_pk = take(mend ? c.split_q * rows * 64 * sizeof(float) : 0);
    c.part_sum = take(mend ? c.split_q * rows * 2 * sizeof(float) : 0);
    c.part_k = take(c.split_kv > 1 ? c.split_kv * keys * 64 * sizeof(float) : 0);
    c.part_v = take(c.split_kv > 1 ? c.split_kv * keys * 64 * sizeof(float) : 0);
    c.backward = off;
    *out = c;
    return S3R_OK;
}

s3r_status check_workspace(const void *ws, size_t have, size_t need)
{
    if (need == 0) return S3R_OK;
    if (!ws || have < need) return fail(S3R_ERR_WORKSPACE, "workspace of %zu bytes given, %zu needed", ws ? have : size_t(0), need);
    if (!aligned(ws, kAlign)) return fail(S3R_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    return S3R_OK;
}

// Checks and arguments that the forward call and the gradient have in common.
s3r_status cross_args(const s3r_cross_params *p, const CrossPlan &c, int view, s3r::CrossArgs *out)
{
    if (p->n_q > 0 && (!p->q || !p->out)) return fail(S3R_ERR_INVALID_ARG, "q and out must be non-null");
    if (p->n_kv > 0 && (!p->k || !p->v)) return fail(S3R_ERR_INVALID_ARG, "k and v must be non-null");
    if (!aligned16(p->q) || !aligned16(p->k) || !aligned16(p->v) || !aligned16(p->out) || !aligned(p->lse, 4) ||
        !aligned(p->q_start, 4) || !aligned(p->kv_start, 4) || !aligned(p->status, 4))
        return fail(S3R_ERR_INVALID_ARG, "device pointers must be 16-byte aligned (lse, starts and status: 4)");
    if (p->n_q > 0 && (p->out == p->q || p->out == p->k || p->out == p->v)) return fail(S3R_ERR_INVALID_ARG, "out must not alias an input");
    s3r_status st = check_strides("q", p->q_stride_tok, p->q_stride_head);
    if (st != S3R_OK) return st;
    st = check_strides("k and v", p->kv_stride_tok, p->kv_stride_head);
    if (st != S3R_OK) return st;
    s3r::CrossArgs a{};
    a.q = p->q; a.k = p->k; a.v = p->v;
    a.q_row = p->q_stride_tok ? p->q_stride_tok : int64_t(p->heads) * 64;
    a.q_head = p->q_stride_head ? p->q_stride_head : 64;
    a.kv_row = p->kv_stride_tok ? p->kv_stride_tok : int64_t(p->kv_heads) * 64;
    a.kv_head = p->kv_stride_head ? p->kv_stride_head : 64;
    a.key_mask = p->key_mask;
    a.q_spans = s3r::Spans{p->q_start, c.batch, p->n_q};
    a.kv_spans = s3r::Spans{p->kv_start, c.batch, p->n_kv};
    a.n_q = p->n_q; a.n_kv = p->n_kv;
    a.heads = p->heads; a.kv_heads = p->kv_heads; a.per_row = c.per_row; a.uneven = c.batch > 1 || view > 0;
    a.accurate = p->accurate_pv != 0;
    a.view = view;
    a.scale = resolve_scale(p->softmax_scale, 64);
    a.factor = a.scale * 1.4426950408889634f;
    a.to.out = p->out; a.to.lse = p->lse; a.to.rows = p->n_q; a.to.heads = p->heads;
    *out = a;
    return S3R_OK;
}

float *floats_at(void *base, size_t off) { return reinterpret_cast<float *>(at(base, off)); }

// What the kernels divide tiles by.  (A launch that joins is there in any case: 2 us of it remain.)
void set_pace(s3r::CrossArgs *a, bool adapts, const Pace &pace, double tile_bytes)
{
    a->resident = adapts ? pace.resident : 0;
    a->unit_us = static_cast<float>(pace.unit_us);
    a->join_ns = 2000;
    a->tile_ns = static_cast<int>(tile_bytes * 2 / 5e3);
}

s3r_status cross_forward(const s3r_cross_params *p, int view)
{
    CrossPlan c;
    s3r_status st = plan_cross(p, view, &c);
    if (st != S3R_OK) return st;
    s3r::CrossArgs a;
    st = cross_args(p, c, view, &a);
    if (st != S3R_OK) return st;
    st = check_workspace(p->workspace, p->workspace_bytes, c.forward);
    if (st != S3R_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(p->stream);
    const bool bf16 = p->dtype == S3R_BF16;
    if (p->status) S3R_HIP(s3r::launch_span_status(a.q_spans, a.kv_spans, p->status, s), "status kernel launch");
    if (p->n_q == 0) return S3R_OK;
    a.tiles = c.tiles;
    a.n_split = c.split;
    a.least = c.least;
    if (!c.few_rows) set_pace(&a, c.adapts, kCrossPace[bf16], 128.0 * 256);
    if (c.split > 1) {
        a.to.part_o = floats_at(p->workspace, c.part_o);
        a.to.part_lse = floats_at(p->workspace, c.part_lse);
    }
    StageTimer tm(S3R_STAGE_DENSE, s);
    S3R_HIP(s3r::launch_cross(a, c.few_rows, bf16, s), "cross attention kernel launch");
    if (c.split > 1)
        S3R_HIP(view > 0 && !c.few_rows ? s3r::launch_causal_combine(a, bf16, s) : s3r::launch_soft_combine(a.to, a.q_spans, c.split, view > 0, bf16, s),
                "cross attention combine kernel launch");
    return S3R_OK;
}

s3r_status cross_backward(const s3r_cross_params *p, int view)
{
    CrossPlan c;
    s3r_status st = plan_cross(p, view, &c);
    if (st != S3R_OK) return st;
    s3r::CrossArgs a;
    st = cross_args(p, c, view, &a);
    if (st != S3R_OK) return st;
    if (p->n_q > 0 && (!p->lse || !p->d_out || !p->dq)) return fail(S3R_ERR_INVALID_ARG, "lse, d_out and dq must be non-null");
    if (p->n_kv > 0 && (!p->dk || !p->dv)) return fail(S3R_ERR_INVALID_ARG, "dk and dv must be non-null");
    if (!aligned16(p->d_out) || !aligned16(p->dq) || !aligned16(p->dk) || !aligned16(p->dv))
        return fail(S3R_ERR_INVALID_ARG, "device pointers must be 16-byte aligned");
    for (const void *g : {p->dq, p->dk, p->dv})
        if (g && (g == p->q || g == p->k || g == p->v || g == p->out || g == p->d_out))
            return fail(S3R_ERR_INVALID_ARG, "gradients must not alias inputs");
    if ((p->dk && (p->dk == p->dv || p->dk == p->dq)) || (p->dq && p->dq == p->dv))
        return fail(S3R_ERR_INVALID_ARG, "gradients must not alias each other");
    st = check_workspace(p->workspace, p->workspace_bytes, c.backward);
    if (st != S3R_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(p->stream);
    const bool bf16 = p->dtype == S3R_BF16;
    if (p->status) S3R_HIP(s3r::launch_span_status(a.q_spans, a.kv_spans, p->status, s), "status kernel launch");
    float *stats = p->n_q > 0 ? floats_at(p->workspace, c.stats) : nullptr;
    a.d_out = p->d_out; a.stats = stats;
    a.dq = p->dq; a.dk = p->dk; a.dv = p->dv;
    StageTimer tm(S3R_STAGE_DENSE, s);
    if (p->n_q > 0) {
        a.tiles = c.q_tiles;
        a.n_split = c.split_q;
        a.least = kGradQPace[bf16].least;
        set_pace(&a, c.adapts_q, kGradQPace[bf16], bf16 ? 2 * 128.0 * 256 : 128.0 * 256);
        if (c.split_q > 1) {
            a.part_q = floats_at(p->workspace, c.part_q);
            a.part_pk = floats_at(p->workspace, c.part_pk);
            a.part_sum = floats_at(p->workspace, c.part_sum);
        }
        S3R_HIP(s3r::launch_grad_q(a, bf16, s), "query gradient kernel launch");
        if (c.split_q > 1) S3R_HIP(s3r::launch_grad_q_combine(a, bf16, s), "query gradient combine kernel launch");
    }
    if (p->n_kv > 0) {
        a.tiles = c.kv_tiles;
        a.n_split = c.split_kv;
        a.least = kGradKvPace[bf16].least;
        set_pace(&a, c.adapts_kv, kGradKvPace[bf16], 2 * 128.0 * 256);
        if (c.split_kv > 1) {
            a.part_k = floats_at(p->workspace, c.part_k);
            a.part_v = floats_at(p->workspace, c.part_v);
        }
        S3R_HIP(s3r::launch_grad_kv(a, bf16, s), "key gradient kernel launch");
        if (c.split_kv > 1) S3R_HIP(s3r::launch_grad_kv_combine(a, bf16, s), "key gradient combine kernel launch");
    }
    return S3R_OK;
}

// Tokens of a view that a causal call is given, held to the keys there are (a larger view sees all of them).
s3r_status causal_view(const s3r_cross_params *p, int tokens_per_view, int *view)
{
    if (!p) return fail(S3R_ERR_INVALID_ARG, "params is null");
    if (tokens_per_view <= 0) return fail(S3R_ERR_INVALID_ARG, "tokens_per_view (%d) must be positive", tokens_per_view);
    const int64_t most = p->n_kv < 1 ? 1 : (p->n_kv > kMaxRowHeads ? kMaxRowHeads : p->n_kv);
    *view = tokens_per_view < most ? tokens_per_view : static_cast<int>(most);
    return S3R_OK;
}

}  // namespace

size_t speed3r_cross_workspace_bytes(const s3r_cross_params *p, int backward)
{
    CrossPlan c;
    if (plan_cross(p, 0, &c) != S3R_OK) return SIZE_MAX;
    return backward ? c.backward : c.forward;
}

s3r_status speed3r_cross_attn(const s3r_cross_params *p) { return cross_forward(p, 0); }
s3r_status speed3r_cross_attn_backward(const s3r_cross_params *p) { return cross_backward(p, 0); }

size_t speed3r_causal_workspace_bytes(const s3r_cross_params *p, int tokens_per_view, int backward)
{
    CrossPlan c;
    int view;
    if (causal_view(p, tokens_per_view, &view) != S3R_OK || plan_cross(p, view, &c) != S3R_OK) return SIZE_MAX;
    return backward ? c.backward : c.forward;
}

s3r_status speed3r_causal_attn(const s3r_cross_params *p, int tokens_per_view)
{
    int view;
    const s3r_status st = causal_view(p, tokens_per_view, &view);
    return st != S3R_OK ? st : cross_forward(p, view);
}

s3r_status speed3r_causal_attn_backward(const s3r_cross_params *p, int tokens_per_view)
{
    int view;
    const s3r_status st = causal_view(p, tokens_per_view, &view);
    return st != S3R_OK ? st : cross_backward(p, view);
}

// ---- a cache in 4 bits ---------------------------------------------------------------------------------
namespace {

struct CachePlan {
    bool few_rows;
    int split, least;
    int64_t tiles;
    size_t part_o, part_lse, need, total;
};

// attends: the attention's pieces as well.  Either order of its rows, causal or not, has room in the workspace of the larger.
s3r_status plan_cache(const s3r_cache_params *p, bool attends, CachePlan *out)
{
    if (!p) return fail(S3R_ERR_INVALID_ARG, "params is null");
    s3r_status st = check_heads(p->heads, p->kv_heads, p->head_dim, p->dtype);
    if (st != S3R_OK) return st;
    if (p->page != 16 && p->page != 32 && p->page != 64 && p->page != 128)
        return fail(S3R_ERR_UNSUPPORTED, "page %d unsupported (must be 16, 32, 64 or 128)", p->page);
    if (p->n_pages <= 0 || p->max_pages <= 0 || p->batch <= 0 || p->n_rows < 0)
        return fail(S3R_ERR_INVALID_ARG, "n_pages (%lld), max_pages (%d) and batch (%d) must be positive, n_rows (%lld) not negative",
                    static_cast<long long>(p->n_pages), p->max_pages, p->batch, static_cast<long long>(p->n_rows));
    if (p->batch > 1 && !p->row_start) return fail(S3R_ERR_INVALID_ARG, "batch (%d) must be 1 without row_start", p->batch);
    if (int64_t(p->max_pages) * p->page > 0x7fffffffLL - 4096 || p->n_pages > 0x7fffffffLL)
        return fail(S3R_ERR_UNSUPPORTED, "max_pages * page exceeds 2^31 - 4097 tokens, or n_pages 2^31 - 1");
    if (p->n_rows > kMaxRowHeads / (p->heads + 2 * p->kv_heads)) return fail(S3R_ERR_UNSUPPORTED, "rows * (heads + 2 kv_heads) exceeds 2^28");
    st = check_batch(p->batch, p->kv_heads);
    if (st != S3R_OK) return st;
    CachePlan c{};
    const int per_row = p->heads / p->kv_heads;
    const int64_t units = (int64_t(p->max_pages) * p->page + 63) / 64;
    // Few rows for a sequence: tiles of 16 in place of one of 128.  Codes are a quarter of bf16 keys, and three tiles still take less than
    // one mostly idle one; five where there are too few of those for the card (us, one of 128 / tiles of 16: 80 rows over 10992 tokens of 16
    // heads 26.1 / 21.1, over 137400 131 / 133, 16 sequences of 1500 tokens and 4 heads 20.3 / 17.5; 64 of these, 48 rows 31 / 31, 64 rows 36 / 40).
    c.few_rows = p->n_rows * per_row <= int64_t(p->batch * p->kv_heads <= 64 ? 80 : 48) * p->batch;
    c.tiles = s3r::most_tiles(p->n_rows, per_row, c.few_rows ? 16 : 128, p->batch);
    if (attends) {
        const Pace &pace = kCachePace[p->dtype == S3R_BF16];
        const size_t rows = static_cast<size_t>(p->n_rows) * p->heads;
        auto layout = [&](bool uneven) {
            if (c.few_rows)
                c.split = pieces_few(mean_tiles(p->n_rows, per_row, 16, p->batch) * p->kv_heads, units, kCacheFew[p->dtype == S3R_BF16]);
            else if (uneven) {
                // Only the longest is known, and counts.  A sequence alone is uneven by what its own rows do not see: two workgroups on a CU (us,
                // 600 causal rows over 5000 in 7 pieces 46, 16 51; 2748 over 10992 in 1 287, 2 198).
                const int64_t mean = p->batch > 1 || units < 32 ? units : 32;
                c.split = pieces_uneven(mean_tiles(p->n_rows, per_row, 128, p->batch) * p->kv_heads, mean, units, pace);
            }
            else
                c.split = pieces(c.tiles * p->kv_heads, units, pace, 256.0 * static_cast<double>(rows));
            const size_t parts = c.split > 1 ? c.split * rows : 0;
            c.part_o = 0;
            c.part_lse = align_up(parts * 64 * sizeof(float));
            return c.part_lse + align_up(parts * sizeof(float));
        };
        c.least = c.few_rows ? kFewLeast : pace.least;
        const bool uneven = p->batch > 1 || p->causal;
        const size_t other = c.few_rows ? 0 : layout(!uneven), need = layout(uneven);
        c.need = need;
        c.total = need > other ? need : other;
    }
    *out = c;
    return S3R_OK;
}

s3r_status cache_args(const s3r_cache_params *p, s3r::CacheArgs *out)
{
    if (!p->k_codes || !p->v_codes || !p->k_scales || !p->v_scales || !p->page_table || !p->kv_len)
        return fail(S3R_ERR_INVALID_ARG, "the cache's four arrays, page_table and kv_len must be non-null");
    if (!aligned16(p->k_codes) || !aligned16(p->v_codes) || !aligned(p->k_scales, 4) || !aligned(p->v_scales, 4) || !aligned(p->page_table, 4) ||
        !aligned(p->kv_len, 4) || !aligned(p->row_start, 4) || !aligned(p->status, 4) || !aligned(p->lse, 4) || !aligned(p->positions, 4) ||
        !aligned16(p->q) || !aligned16(p->k) || !aligned16(p->v) || !aligned16(p->out) || !aligned16(p->cos) || !aligned16(p->sin))
        return fail(S3R_ERR_INVALID_ARG, "device pointers must be 16-byte aligned (scales, lists, lse and status: 4)");
    s3r_status st = check_strides("q", p->q_stride_tok, p->q_stride_head);
    if (st != S3R_OK) return st;
    st = check_strides("k and v", p->kv_stride_tok, p->kv_stride_head);
    if (st != S3R_OK) return st;
    s3r::CacheArgs a{};
    int shift = 4;
    while ((1 << shift) < p->page) ++shift;
    a.cache = s3r::Cache{p->k_codes, p->v_codes, p->k_scales, p->v_scales, p->page_table, p->kv_len, p->n_pages, p->max_pages, shift, p->kv_heads};
    a.spans = s3r::Spans{p->row_start, p->batch, p->n_rows};
    a.q = p->q; a.k = p->k; a.v = p->v;
    a.q_row = p->q_stride_tok ? p->q_stride_tok : int64_t(p->heads) * 64;
    a.q_head = p->q_stride_head ? p->q_stride_head : 64;
    a.kv_row = p->kv_stride_tok ? p->kv_stride_tok : int64_t(p->kv_heads) * 64;
    a.kv_head = p->kv_stride_head ? p->kv_stride_head : 64;
    a.n_rows = p->n_rows; a.heads = p->heads; a.per_row = p->heads / p->kv_heads;
    a.causal = p->causal != 0;
    a.uneven = p->batch > 1 || a.causal;
    a.factor = resolve_scale(p->softmax_scale, 64) * 1.4426950408889634f;
    a.to.out = p->out; a.to.lse = p->lse; a.to.rows = p->n_rows; a.to.heads = p->heads;
    *out = a;
    return S3R_OK;
}

}  // namespace

size_t speed3r_cache_workspace_bytes(const s3r_cache_params *p)
{
    CachePlan c;
    return plan_cache(p, true, &c) == S3R_OK ? c.total : SIZE_MAX;
}

s3r_status speed3r_cache_append(const s3r_cache_params *p)
{
    CachePlan c;
    s3r_status st = plan_cache(p, false, &c);
    if (st != S3R_OK) return st;
    s3r::CacheArgs a;
    st = cache_args(p, &a);
    if (st != S3R_OK) return st;
    if (p->n_rows > 0 && (!p->k || !p->v)) return fail(S3R_ERR_INVALID_ARG, "k and v must be non-null");
    if (p->k_codes == p->v_codes || p->k_scales == p->v_scales) return fail(S3R_ERR_INVALID_ARG, "keys and values must not share an array");
    if ((p->cos != nullptr) != (p->sin != nullptr)) return fail(S3R_ERR_INVALID_ARG, "cos and sin must be given together");
    if (p->n_rows > 0 && (p->q != nullptr) != (p->out != nullptr)) return fail(S3R_ERR_INVALID_ARG, "q and out must be given together");
    if (p->q && !p->cos) return fail(S3R_ERR_INVALID_ARG, "q is given to be rotated: cos and sin are needed");
    // (waves have rows' queries, keys and values apart: one may write over what another is still to read)
    if (p->q && (p->out == p->q || p->out == p->k || p->out == p->v)) return fail(S3R_ERR_INVALID_ARG, "out must not alias an input");
    if (p->cos) {
        if (p->rot_axes != 1 && p->rot_axes != 2) return fail(S3R_ERR_INVALID_ARG, "rot_axes (%d) must be 1 or 2", p->rot_axes);
        if (p->rot_axes == 2 && !p->positions) return fail(S3R_ERR_INVALID_ARG, "two axes need positions");
        if (p->rot_neighbours != 0 && p->rot_neighbours != 1) return fail(S3R_ERR_INVALID_ARG, "rot_neighbours (%d) must be 0 or 1", p->rot_neighbours);
        if (p->n_positions <= 0) return fail(S3R_ERR_INVALID_ARG, "n_positions must be positive");
        a.rot = s3r::Rotation{p->cos, p->sin, p->positions, p->n_positions, p->rot_axes, p->rot_neighbours != 0};
    }
    hipStream_t s = static_cast<hipStream_t>(p->stream);
    if (p->status) S3R_HIP(s3r::launch_cache_status(a, true, p->status, s), "status kernel launch");
    if (p->n_rows == 0) return S3R_OK;
    StageTimer tm(S3R_STAGE_POOL, s);
    S3R_HIP(s3r::launch_cache_append(a, p->dtype == S3R_BF16, s), "cache append kernel launch");
    return S3R_OK;
}

s3r_status speed3r_cache_read(const s3r_cache_params *p)
{
    CachePlan c;
    s3r_status st = plan_cache(p, false, &c);
    if (st != S3R_OK) return st;
    s3r::CacheArgs a;
    st = cache_args(p, &a);
    if (st != S3R_OK) return st;
    if (p->n_rows > 0 && (!p->k || !p->v || p->k == p->v)) return fail(S3R_ERR_INVALID_ARG, "k and v must be non-null and apart");
    hipStream_t s = static_cast<hipStream_t>(p->stream);
    if (p->status) S3R_HIP(s3r::launch_cache_status(a, true, p->status, s), "status kernel launch");
    if (p->n_rows == 0) return S3R_OK;
    StageTimer tm(S3R_STAGE_POOL, s);
    S3R_HIP(s3r::launch_cache_read(a, p->dtype == S3R_BF16, s), "cache read kernel launch");
    return S3R_OK;
}

s3r_status speed3r_cache_attn(const s3r_cache_params *p)
{
    CachePlan c;
    s3r_status st = plan_cache(p, true, &c);
    if (st != S3R_OK) return st;
    s3r::CacheArgs a;
    st = cache_args(p, &a);
    if (st != S3R_OK) return st;
    if (p->n_rows > 0 && (!p->q || !p->out)) return fail(S3R_ERR_INVALID_ARG, "q and out must be non-null");
    if (p->n_rows > 0 && p->q == p->out) return fail(S3R_ERR_INVALID_ARG, "out must not alias an input");
    if (p->causal != 0 && p->causal != 1) return fail(S3R_ERR_INVALID_ARG, "causal (%d) must be 0 or 1", p->causal);
    st = check_workspace(p->workspace, p->workspace_bytes, c.need);
    if (st != S3R_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(p->stream);
    const bool bf16 = p->dtype == S3R_BF16;
    if (p->status) S3R_HIP(s3r::launch_cache_status(a, false, p->status, s), "status kernel launch");
    if (p->n_rows == 0) return S3R_OK;
    a.tiles = c.tiles;
    a.n_split = c.split;
    a.least = c.least;
    if (c.split > 1) {
        a.to.part_o = floats_at(p->workspace, c.part_o);
        a.to.part_lse = floats_at(p->workspace, c.part_lse);
    }
    StageTimer tm(S3R_STAGE_DENSE, s);
    S3R_HIP(s3r::launch_cache_attn(a, c.few_rows, bf16, s), "cache attention kernel launch");
    if (c.split > 1) S3R_HIP(s3r::launch_soft_combine(a.to, a.spans, c.split, false, bf16, s), "cache attention combine kernel launch");
    return S3R_OK;
}

// ---- rotary positions with the norm of a head ------------------------------------------------------------
namespace {

s3r_status check_eps(float eps)
{
    if (!(eps >= 1.17549435e-38f) || !std::isfinite(eps)) return fail(S3R_ERR_INVALID_ARG, "eps (%g) must be positive and finite", static_cast<double>(eps));
    return S3R_OK;
}

s3r_status check_norm(const char *what, int norm)
{
    if (norm < S3R_NORM_NONE || norm > S3R_NORM_LAYER) return fail(S3R_ERR_INVALID_ARG, "%s (%d) must be one of S3R_NORM_*", what, norm);
    return S3R_OK;
}

// Checks of what the shape fields hold.
s3r_status check_rotary(const s3r_rotary_params *p)
{
    if (!p) return fail(S3R_ERR_INVALID_ARG, "params is null");
    if (p->heads < 0 || p->kv_heads < 0 || p->heads + static_cast<int64_t>(p->kv_heads) == 0)
        return fail(S3R_ERR_INVALID_ARG, "heads (%d) and kv_heads (%d) must not be negative, nor both 0", p->heads, p->kv_heads);
    if (p->heads > 65535 || p->kv_heads > 65535) return fail(S3R_ERR_UNSUPPORTED, "heads %d, %d unsupported (max 65535)", p->heads, p->kv_heads);
    if (p->head_dim != 64) return fail(S3R_ERR_UNSUPPORTED, "head_dim %d unsupported (must be 64)", p->head_dim);
    if (p->dtype != S3R_F32 && p->dtype != S3R_BF16) return fail(S3R_ERR_UNSUPPORTED, "unknown dtype %d", p->dtype);
    if (p->weight_dtype != S3R_F32 && p->weight_dtype != S3R_BF16) return fail(S3R_ERR_UNSUPPORTED, "unknown weight_dtype %d", p->weight_dtype);
    if (p->n_rows < 0) return fail(S3R_ERR_INVALID_ARG, "n_rows must not be negative");
    if (p->n_rows > kMaxRowHeads / (p->heads + p->kv_heads)) return fail(S3R_ERR_UNSUPPORTED, "rows * heads exceeds 2^28");
    s3r_status st = check_norm("norm", p->norm);
    if (st != S3R_OK) return st;
    if (p->axes < 0 || p->axes > 3) return fail(S3R_ERR_INVALID_ARG, "axes (%d) must be 0 to 3", p->axes);
    if (p->axes == 0 && p->norm == S3R_NORM_NONE) return fail(S3R_ERR_INVALID_ARG, "neither axes nor a norm: nothing to do");
    int pairs = 0;
    for (int x = 0; x < p->axes; ++x) {
        if (p->axis_pairs[x] < 1 || p->axis_pairs[x] > 32) return fail(S3R_ERR_INVALID_ARG, "axis_pairs[%d] (%d) must be 1 to 32", x, p->axis_pairs[x]);
        pairs += p->axis_pairs[x];
    }
    if (pairs > 32) return fail(S3R_ERR_INVALID_ARG, "axis_pairs add up to %d, more than the 32 pairs of a head", pairs);
    if (p->pairs < S3R_PAIRS_HALVES || p->pairs > S3R_PAIRS_WHOLE) return fail(S3R_ERR_INVALID_ARG, "pairs (%d) must be one of S3R_PAIRS_*", p->pairs);
    if (p->norm != S3R_NORM_NONE) return check_eps(p->eps);
    if (p->q_weight || p->q_bias || p->k_weight || p->k_bias || p->dq_weight || p->dq_bias || p->dk_weight || p->dk_bias)
        return fail(S3R_ERR_INVALID_ARG, "weights and biases need a norm");
    return S3R_OK;
}

// What the two calls have in common; the tensors' pointers and strides are theirs.
s3r_status rotary_args(const s3r_rotary_params *p, s3r::RotaryArgs *out)
{
    s3r_status st = check_rotary(p);
    if (st != S3R_OK) return st;
    if ((p->axes > 0) != (p->cos != nullptr) || (p->axes > 0) != (p->sin != nullptr))
        return fail(S3R_ERR_INVALID_ARG, "cos, sin and axes must be given together");
    if (!aligned16(p->cos) || !aligned16(p->sin) || !aligned(p->positions, 4) || !aligned(p->status, 4))
        return fail(S3R_ERR_INVALID_ARG, "cos and sin must be 16-byte aligned, positions and status 4-byte");
    if (p->axes > 0 && p->n_positions <= 0) return fail(S3R_ERR_INVALID_ARG, "n_positions must be positive");
    if (p->axes > 1 && !p->positions && p->n_rows > 0) return fail(S3R_ERR_INVALID_ARG, "positions must be given for %d axes", p->axes);
    if (p->axes == 0 && p->positions) return fail(S3R_ERR_INVALID_ARG, "positions need axes");
    for (const void *t : {p->q, p->k, static_cast<const void *>(p->q_out), static_cast<const void *>(p->k_out), p->d_q_out, p->d_k_out,
                          static_cast<const void *>(p->dq), static_cast<const void *>(p->dk), p->q_weight, p->q_bias, p->k_weight, p->k_bias,
                          static_cast<const void *>(p->dq_weight), static_cast<const void *>(p->dq_bias), static_cast<const void *>(p->dk_weight),
                          static_cast<const void *>(p->dk_bias)})
        if (!aligned16(t)) return fail(S3R_ERR_INVALID_ARG, "device pointers must be 16-byte aligned");
    for (auto [what, tok, head] : {std::make_tuple("q", p->q_stride_tok, p->q_stride_head), std::make_tuple("k", p->k_stride_tok, p->k_stride_head),
                                   std::make_tuple("dq", p->dq_stride_tok, p->dq_stride_head), std::make_tuple("dk", p->dk_stride_tok, p->dk_stride_head)}) {
        st = check_strides(what, tok, head);
        if (st != S3R_OK) return st;
    }
    s3r::RotaryArgs a{};
    a.cos = p->cos; a.sin = p->sin; a.positions = p->positions;
    a.n_rows = p->n_rows; a.places = p->n_positions;
    a.axes = p->axes; a.pairing = p->pairs; a.norm = p->norm;
    for (int x = 0; x < p->axes; ++x) {
        a.axis_pairs[x] = p->axis_pairs[x];
        a.n_pairs += p->axis_pairs[x];
    }
    a.w_bf16 = p->weight_dtype == S3R_BF16;
    a.eps = p->eps;
    a.sign = 1.f;
    a.side[0].heads = p->heads; a.side[0].weight = p->q_weight; a.side[0].bias = p->q_bias;
    a.side[1].heads = p->kv_heads; a.side[1].weight = p->k_weight; a.side[1].bias = p->k_bias;
    *out = a;
    return S3R_OK;
}

int64_t or_else(int64_t given, int64_t packed) { return given ? given : packed; }

bool same_as_any(const void *t, std::initializer_list<const void *> others)
{
    for (const void *o : others)
        if (t && t == o) return true;
    return false;
}

}  // namespace

size_t speed3r_rotary_workspace_bytes(const s3r_rotary_params *p)
{
    if (check_rotary(p) != S3R_OK) return SIZE_MAX;
    return p->norm != S3R_NORM_NONE && (p->dq_weight || p->dq_bias || p->dk_weight || p->dk_bias)
               ? align_up(static_cast<size_t>(s3r::kRotaryGradGroups) * 128 * sizeof(float)) : 0;
}

s3r_status speed3r_rotary(const s3r_rotary_params *p)
{
    s3r::RotaryArgs a;
    s3r_status st = rotary_args(p, &a);
    if (st != S3R_OK) return st;
    if (p->n_rows > 0 && ((p->heads > 0 && (!p->q || !p->q_out)) || (p->kv_heads > 0 && (!p->k || !p->k_out))))
        return fail(S3R_ERR_INVALID_ARG, "q, k, q_out and k_out must be non-null");
    if (same_as_any(p->q_out, {p->q, p->k, p->k_out}) || same_as_any(p->k_out, {p->q, p->k}))
        return fail(S3R_ERR_INVALID_ARG, "q_out and k_out must not alias inputs or each other");
    const int64_t q_row = int64_t(p->heads) * 64, k_row = int64_t(p->kv_heads) * 64;
    s3r::RotarySide &q = a.side[0], &k = a.side[1];
    q.in = p->q; q.out = p->q_out; q.in_row = or_else(p->q_stride_tok, q_row); q.in_head = or_else(p->q_stride_head, 64); q.out_row = q_row; q.out_head = 64;
    k.in = p->k; k.out = p->k_out; k.in_row = or_else(p->k_stride_tok, k_row); k.in_head = or_else(p->k_stride_head, 64); k.out_row = k_row; k.out_head = 64;
    hipStream_t s = static_cast<hipStream_t>(p->stream);
    if (p->status) S3R_HIP(s3r::launch_rotary_status(a, p->status, s), "status kernel launch");
    if (p->n_rows == 0) return S3R_OK;
    StageTimer tm(S3R_STAGE_POOL, s);
    S3R_HIP(s3r::launch_rotary(a, p->dtype == S3R_BF16, s), "rotary kernel launch");
    return S3R_OK;
}

s3r_status speed3r_rotary_backward(const s3r_rotary_params *p)
{
    s3r::RotaryArgs a;
    s3r_status st = rotary_args(p, &a);
    if (st != S3R_OK) return st;
    const bool norm = p->norm != S3R_NORM_NONE;
    if (p->n_rows > 0 && ((p->heads > 0 && (!p->d_q_out || !p->dq || (norm && !p->q))) || (p->kv_heads > 0 && (!p->d_k_out || !p->dk || (norm && !p->k)))))
        return fail(S3R_ERR_INVALID_ARG, "d_q_out, d_k_out, dq and dk (and, with a norm, q and k) must be non-null");
    if (same_as_any(p->dq, {p->q, p->k, p->d_q_out, p->d_k_out, p->dk}) || same_as_any(p->dk, {p->q, p->k, p->d_q_out, p->d_k_out}))
        return fail(S3R_ERR_INVALID_ARG, "gradients must not alias inputs or each other");
    const size_t need = speed3r_rotary_workspace_bytes(p);
    st = check_workspace(p->workspace, p->workspace_bytes, need);
    if (st != S3R_OK) return st;
    const int64_t q_row = int64_t(p->heads) * 64, k_row = int64_t(p->kv_heads) * 64;
    s3r::RotarySide &q = a.side[0], &k = a.side[1];
    q.out = p->dq; q.out_row = or_else(p->dq_stride_tok, q_row); q.out_head = or_else(p->dq_stride_head, 64);
    k.out = p->dk; k.out_row = or_else(p->dk_stride_tok, k_row); k.out_head = or_else(p->dk_stride_head, 64);
    q.in = norm ? p->q : p->d_q_out; q.in_row = norm ? or_else(p->q_stride_tok, q_row) : q_row; q.in_head = norm ? or_else(p->q_stride_head, 64) : 64;
    k.in = norm ? p->k : p->d_k_out; k.in_row = norm ? or_else(p->k_stride_tok, k_row) : k_row; k.in_head = norm ? or_else(p->k_stride_head, 64) : 64;
    q.grad = p->d_q_out; q.d_weight = p->dq_weight; q.d_bias = p->dq_bias;
    k.grad = p->d_k_out; k.d_weight = p->dk_weight; k.d_bias = p->dk_bias;
    a.part = need > 0 ? static_cast<float *>(p->workspace) : nullptr;
    hipStream_t s = static_cast<hipStream_t>(p->stream);
    if (p->status) S3R_HIP(s3r::launch_rotary_status(a, p->status, s), "status kernel launch");
    if (p->n_rows == 0 && a.part == nullptr) return S3R_OK;
    StageTimer tm(S3R_STAGE_POOL, s);
    if (norm) {
        S3R_HIP(s3r::launch_rotary_norm_grad(a, p->dtype == S3R_BF16, s), "rotary gradient kernel launch");
    } else {
        a.sign = -1.f;
        S3R_HIP(s3r::launch_rotary(a, p->dtype == S3R_BF16, s), "rotary gradient kernel launch");
    }
    return S3R_OK;
}

// ---- the residual stream with the norms around a block -----------------------------------------------------
namespace {

struct ResidualPlan {
    int batch, rows_per_block;
    int64_t blocks;
    bool wide;                     // sums of the gradient in 64 bits between shares of kResidualTurns
    size_t part, part_gate, need;  // workspace of the gradient
};

// Workgroups: as many as the card holds at once, or fewer; their rows follow one another, a multiple of what they have at a time.
constexpr int kResidualBlocks = 2048, kResidualGradBlocks = 512;
// Terms of a gradient that a thread adds up in fp32, one after the other: off by up to 2^-16 of the sum of their magnitudes.  (512 workgroups reach it at
// 131072 rows of 2048 channels and more, four million of 64.)
constexpr int kResidualTurns = 256;

s3r_status plan_residual(const s3r_residual_params *p, bool backward, ResidualPlan *out)
{
    if (!p) return fail(S3R_ERR_INVALID_ARG, "params is null");
    if (p->width < 8 || p->width > 8192 || p->width % 8 != 0) return fail(S3R_ERR_UNSUPPORTED, "width %d unsupported (must be a multiple of 8 up to 8192)", p->width);
    if (p->n_rows < 0) return fail(S3R_ERR_INVALID_ARG, "n_rows must not be negative");
    if (p->n_rows > kMaxRowHeads) return fail(S3R_ERR_UNSUPPORTED, "n_rows exceeds 2^28");
    if (p->dtype != S3R_F32 && p->dtype != S3R_BF16) return fail(S3R_ERR_UNSUPPORTED, "unknown dtype %d", p->dtype);
    if (p->x_dtype != S3R_F32 && p->x_dtype != p->dtype) return fail(S3R_ERR_UNSUPPORTED, "x_dtype must be dtype or fp32");
    if (p->weight_dtype != S3R_F32 && p->weight_dtype != S3R_BF16) return fail(S3R_ERR_UNSUPPORTED, "unknown weight_dtype %d", p->weight_dtype);
    if (p->batch < 0 || (p->batch > 1 && !p->row_start)) return fail(S3R_ERR_INVALID_ARG, "batch (%d) must be 1 without row_start, and never negative", p->batch);
    if (p->row_start && (p->batch == 0 || !p->gate)) return fail(S3R_ERR_INVALID_ARG, "row_start needs gates and a positive batch");
    if (p->batch > 65536) return fail(S3R_ERR_UNSUPPORTED, "batch (%d) exceeds 65536", p->batch);
    s3r_status st = check_norm("norm", p->norm);
    if (st != S3R_OK) return st;
    st = check_norm("post_norm", p->post_norm);
    if (st != S3R_OK) return st;
    if (p->norm != S3R_NORM_NONE || p->post_norm != S3R_NORM_NONE) {
        st = check_eps(p->eps);
        if (st != S3R_OK) return st;
    }
    if (!std::isfinite(p->residual_scale)) return fail(S3R_ERR_INVALID_ARG, "residual_scale must be finite");
    if (p->norm == S3R_NORM_NONE && (p->weight || p->bias || p->d_weight || p->d_bias)) return fail(S3R_ERR_INVALID_ARG, "weight and bias need a norm");
    if (p->post_norm == S3R_NORM_NONE && (p->post_weight || p->post_bias || p->d_post_weight || p->d_post_bias))
        return fail(S3R_ERR_INVALID_ARG, "post_weight and post_bias need a post_norm");
    if (p->n_rows > 0 && !p->f && (p->post_norm != S3R_NORM_NONE || p->scale || p->gate || p->d_scale || p->d_gate))
        return fail(S3R_ERR_INVALID_ARG, "a post_norm, scale and gate need f");
    if (p->d_gate && !p->gate) return fail(S3R_ERR_INVALID_ARG, "d_gate needs a gate");
    ResidualPlan c{};
    c.batch = p->batch == 0 ? 1 : p->batch;
    const int64_t at_once = s3r::residual_rows(p->width, p->gate || p->post_norm != S3R_NORM_NONE), most = backward ? kResidualGradBlocks : kResidualBlocks;
    const int64_t rows = ((p->n_rows + most - 1) / most + at_once - 1) / at_once * at_once;
    c.rows_per_block = static_cast<int>(rows < at_once ? at_once : rows);
    c.blocks = (p->n_rows + c.rows_per_block - 1) / c.rows_per_block;
    c.wide = c.rows_per_block / at_once + (p->gate ? std::min<int64_t>(c.batch, c.rows_per_block) : 0) > kResidualTurns;
    const size_t row = static_cast<size_t>(p->width) * (c.wide ? sizeof(double) : sizeof(float));
    size_t off = 0;
    c.part = off;
    if (p->d_weight || p->d_bias || p->d_scale || p->d_post_weight || p->d_post_bias) off += align_up(s3r::kResidualParts * static_cast<size_t>(c.blocks) * row);
    c.part_gate = off;
    if (p->d_gate) off += align_up((static_cast<size_t>(c.blocks) + c.batch) * row);
    c.need = off;
    *out = c;
    return S3R_OK;
}

s3r_status residual_args(const s3r_residual_params *p, const ResidualPlan &c, s3r::ResidualArgs *out)
{
    if (p->n_rows > 0 && !p->x) return fail(S3R_ERR_INVALID_ARG, "x must be non-null");
    for (const void *t : {p->x, p->f, static_cast<const void *>(p->r), static_cast<const void *>(p->y), p->weight, p->bias, p->post_weight, p->post_bias,
                          p->scale, p->gate, p->d_r, p->d_y, static_cast<const void *>(p->dx), static_cast<const void *>(p->df),
                          static_cast<const void *>(p->d_weight), static_cast<const void *>(p->d_bias), static_cast<const void *>(p->d_post_weight),
                          static_cast<const void *>(p->d_post_bias), static_cast<const void *>(p->d_scale), static_cast<const void *>(p->d_gate)})
        if (!aligned16(t)) return fail(S3R_ERR_INVALID_ARG, "device pointers must be 16-byte aligned");
    if (!aligned(p->row_start, 4) || !aligned(p->status, 4)) return fail(S3R_ERR_INVALID_ARG, "row_start and status must be 4-byte aligned");
    for (auto [what, stride] : {std::make_pair("x", p->x_stride), std::make_pair("f", p->f_stride), std::make_pair("gate", p->gate_stride)}) {
        s3r_status st = check_strides(what, stride, 0);
        if (st != S3R_OK) return st;
    }
    s3r::ResidualArgs a{};
    a.x = p->x; a.f = p->f; a.gate = p->gate;
    a.x_row = or_else(p->x_stride, p->width); a.f_row = or_else(p->f_stride, p->width); a.gate_row = or_else(p->gate_stride, p->width);
    a.weight = p->weight; a.bias = p->bias; a.post_weight = p->post_weight; a.post_bias = p->post_bias; a.scale = p->scale;
    a.spans = s3r::Spans{p->row_start, c.batch, p->n_rows};
    a.n = p->n_rows; a.width = p->width; a.norm = p->norm; a.post = p->post_norm; a.rows_per_block = c.rows_per_block;
    a.w_bf16 = p->weight_dtype == S3R_BF16;
    a.eps = p->eps;
    a.residual_scale = p->residual_scale == 0.f ? 1.f : p->residual_scale;
    *out = a;
    return S3R_OK;
}

}  // namespace

size_t speed3r_residual_workspace_bytes(const s3r_residual_params *p)
{
    ResidualPlan c;
    if (plan_residual(p, true, &c) != S3R_OK) return SIZE_MAX;
    return c.need;
}

s3r_status speed3r_residual_norm(const s3r_residual_params *p)
{
    ResidualPlan c;
    s3r_status st = plan_residual(p, false, &c);
    if (st != S3R_OK) return st;
    s3r::ResidualArgs a;
    st = residual_args(p, c, &a);
    if (st != S3R_OK) return st;
    if (p->n_rows > 0 && !p->r && !p->y) return fail(S3R_ERR_INVALID_ARG, "r and y must not both be null");
    if (p->y && p->norm == S3R_NORM_NONE) return fail(S3R_ERR_INVALID_ARG, "y needs a norm");
    if (same_as_any(p->y, {p->x, p->f, p->r, p->gate}) || same_as_any(p->r, {p->f, p->gate}) || (p->r && p->r == p->x && a.x_row != p->width))
        return fail(S3R_ERR_INVALID_ARG, "outputs must not alias inputs or each other (but r may be a packed x)");
    a.r = p->r; a.y = p->y;
    hipStream_t s = static_cast<hipStream_t>(p->stream);
    if (p->status) S3R_HIP(s3r::launch_span_status(a.spans, a.spans, p->status, s), "status kernel launch");
    if (p->n_rows == 0) return S3R_OK;
    StageTimer tm(S3R_STAGE_POOL, s);
    S3R_HIP(s3r::launch_residual(a, p->x_dtype == S3R_BF16, p->dtype == S3R_BF16, s), "residual norm kernel launch");
    return S3R_OK;
}

s3r_status speed3r_residual_norm_backward(const s3r_residual_params *p)
{
    ResidualPlan c;
    s3r_status st = plan_residual(p, true, &c);
    if (st != S3R_OK) return st;
    s3r::ResidualArgs a;
    st = residual_args(p, c, &a);
    if (st != S3R_OK) return st;
    if (p->n_rows > 0 && !p->dx) return fail(S3R_ERR_INVALID_ARG, "dx must be non-null");
    if (p->n_rows > 0 && (p->f != nullptr) != (p->df != nullptr)) return fail(S3R_ERR_INVALID_ARG, "f and df must be given together");
    if (p->n_rows > 0 && !p->d_r && !p->d_y) return fail(S3R_ERR_INVALID_ARG, "d_r and d_y must not both be null");
    if (p->d_y && p->norm == S3R_NORM_NONE) return fail(S3R_ERR_INVALID_ARG, "d_y needs a norm");
    if (same_as_any(p->dx, {p->x, p->f, p->d_r, p->d_y, p->df, p->gate}) || same_as_any(p->df, {p->x, p->f, p->d_r, p->d_y, p->gate}))
        return fail(S3R_ERR_INVALID_ARG, "gradients must not alias inputs or each other");
    st = check_workspace(p->workspace, p->workspace_bytes, c.need);
    if (st != S3R_OK) return st;
    a.d_r = p->d_r; a.d_y = p->d_y; a.dx = p->dx; a.df = p->df;
    a.d_weight = p->d_weight; a.d_bias = p->d_bias; a.d_post_weight = p->d_post_weight; a.d_post_bias = p->d_post_bias;
    a.d_scale = p->d_scale; a.d_gate = p->d_gate;
    a.wide = c.wide;
    a.turns = c.wide ? kResidualTurns : INT_MAX;
    if (c.part_gate > c.part) a.part = at(p->workspace, c.part);
    if (p->d_gate) a.part_gate = at(p->workspace, c.part_gate);
    hipStream_t s = static_cast<hipStream_t>(p->stream);
    if (p->status) S3R_HIP(s3r::launch_span_status(a.spans, a.spans, p->status, s), "status kernel launch");
    StageTimer tm(S3R_STAGE_POOL, s);
    S3R_HIP(s3r::launch_residual_grad(a, p->x_dtype == S3R_BF16, p->dtype == S3R_BF16, s), "residual norm gradient kernel launch");
    return S3R_OK;
}

}  // extern "C"
