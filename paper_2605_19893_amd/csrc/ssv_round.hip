// Host side of the C ABI declared in include/ssv_round.h: argument checks, launch planning and launches of the operators
// around a verification round.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>

#include "../../include/ssv_round.h"
#include "k_accept.hpp"
#include "k_prefix.hpp"
#include "k_sample.hpp"

namespace {

using namespace ssv;

constexpr int kMaxDevices = 64;   // per-device one-time set-up flags

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }
size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
bool misaligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }
bool launchable(int64_t workgroups, int threads) { return workgroups * threads < (1ll << 32); }      // threads of a launch are counted in 32 bits
// Strides of something written in place: distinct indices are distinct places.
bool repeats(int64_t extent, int64_t stride) { return extent > 1 && stride == 0; }

// ---- shared-prefix attention
constexpr int kPrefixMaxSlices = kPrefixMaxSlots / 2;      // per part (prefix, own rows)
constexpr int kPrefixWgs = 256;            // one round of workgroups: one per CU
constexpr int64_t kPrefixMaxGroups = 1 << 19;      // (cache, KV head, row group) per part: with a slice each, both parts fit a launch

struct PartPlan {
    int caches, per, rows, path, n_rg;
    int units, slots, min_tiles;       // slices of all caches together (0: no such part), slots per row, tiles per slice at least
    bool by_length;
};

struct PrefixLayout {
    int H_g, es;
    PartPlan part[2];            // prefix, own rows
    int n_slots;
    int64_t rows_total;
    int64_t q_s[3], out_s[3];    // bytes
    size_t off_stats, off_acc, total;
};

// Path and row groups of a part.  Up to 16 rows the keys path, with more the rows path (fp32: 32 rows of the keys path).  16
// sequences of 8192 own rows, 4 KV heads of 128 + 128, keys against rows path: 8 rows 37.9 and 40.1 us, 16 rows 39.2 and
// 40.9 us, 24 and 32 rows (two groups, every key read twice) 61.6 and 41.1 us.  fp32, 4 rows behind 4097: 14.7 us with 16
// rows in a workgroup, 17.0 us with 32; with 32 rows 20.2 us.
int plan_rows(PartPlan* pt, bool bf16, int H_kv) {
    pt->by_length = pt->caches > 1 && pt->caches <= kPrefixMaxDealt;
    pt->path = pt->rows <= 16 ? 1 : (bf16 ? 0 : 2);
    pt->n_rg = ceil_div(pt->rows, pt->path ? 16 * pt->path : 256);
    return (int64_t)pt->caches * H_kv * pt->n_rg <= kPrefixMaxGroups ? SSV_OK : SSV_EUNSUPPORTED;
}

// What a part would cost in a number of slices: workgroups, and microseconds of the longest and of an average one.  A rough model
// from in-kernel clocks: a tile takes a workgroup of the rows path 2.1 us at 192 + 128 and 1.1 us at 64 + 64 (with at most one
// wavefront per SIMD 1.1 and 0.8), one of the keys path what its bytes take at 60 GB/s; 7 us pass from the first instruction to the
// first tile and from the last one to the end.
struct SliceCost { int units, slots, min_tiles, wgs; float us, mean; };
struct PartCost {
    float tile_us, mean;
    int tiles, groups, caches;
    bool by_length;
    PartCost(const PartPlan& pt, const ssv_prefix_params* p, int64_t max_keys, float mean_share) : mean(mean_share), caches(pt.caches), by_length(pt.by_length) {
        const float mma = (p->d_k + p->d_v) / 8.f, bytes = 64.f * (p->d_k + p->d_v) * 2;
        tile_us = p->dtype == SSV_F32 ? 0.6f * pt.path
                  : pt.path            ? bytes / 60e3f
                                       : (pt.rows > 128 ? 0.35f + 0.044f * mma : 0.6f + 0.0135f * mma);
        tiles = (int)((max_keys + kTile - 1) / kTile);
        groups = p->H_kv * pt.n_rg;
    }
    // slices per cache in eighths (8 and more)
    SliceCost at(int eighths) const {
        SliceCost c;
        if (by_length) {
            c.units = caches * eighths / 8;
            c.slots = std::min(kPrefixMaxSlices, 2 * ((eighths + 7) / 8) + 1);
            c.min_tiles = std::max(kPrefixMinTiles, (tiles + c.slots - 1) / c.slots);
            // lengths of which the slices are cut: the mean of the caches; a cache's last slice is half empty
            const float all = tiles * mean * caches, longest = std::max((float)c.min_tiles, all / std::max(1.f, c.units - (mean < 1.f ? 0.5f * caches : 0.f)));
            c.us = 7.f + std::min((float)tiles, longest) * tile_us;
            c.mean = 7.f + all / c.units * tile_us;
        } else {
            const int chunk = std::max(kPrefixMinTiles, (tiles + eighths / 8 - 1) / (eighths / 8));
            c.slots = (tiles + chunk - 1) / chunk;
            c.units = caches * c.slots;
            c.min_tiles = kPrefixMinTiles;
            c.us = 7.f + chunk * tile_us;
            c.mean = 7.f + chunk * tile_us * mean;
        }
        c.wgs = groups * c.units;
        return c;
    }
};
// n workgroups of mixed lengths on `cus` compute units, in any order
float spread_us(const SliceCost& c, float n, float cus) { return n <= 0 ? 0.f : n <= cus ? c.us : n * c.mean / cus + c.us / 2; }

// Slices of both parts: the pair with the least estimated time for one launch (the prefix's workgroups in rounds of 256, the own
// ones in the places they leave) and for the partial states, which are written and read back at 4 TB/s.
void plan_slices(PrefixLayout* lo, const ssv_prefix_params* p) {
    static constexpr int eighths[] = {8, 10, 12, 16, 20, 24, 32, 40, 48, 56, 64, 72, 80, 96, 112, 128, 144, 160, 192, 224, 256, 320, 384, 512};
    constexpr int N = sizeof(eighths) / sizeof(eighths[0]);
    const bool shared = p->max_prefix_len > 0;
    SliceCost own[N], first = {0, 0, 0, 0, 0.f, 0.f};
    const PartCost oc(lo->part[1], p, (int64_t)p->max_seq_len + p->T, p->B > 1 ? 0.5f : 1.f);       // (sequences of mixed lengths, the bound is the longest's)
    int n_own = 0;
    for (int n : eighths) {
        const SliceCost c = oc.at(n);
        if (!n_own || c.units > own[n_own - 1].units) own[n_own++] = c;
    }
    const float state_us = (float)(p->d_v * 4 + 8) * 2 / 4e6f;       // of a partial state
    auto put = [](PartPlan* pt, const SliceCost& c) {
        pt->units = c.units;
        pt->slots = c.slots;
        pt->min_tiles = c.min_tiles;
    };
    float best = 1e30f;
    int last = -1;
    for (int i = 0; i < (shared ? N : 1); ++i) {
        if (shared) first = PartCost(lo->part[0], p, p->max_prefix_len, 1.f).at(eighths[i]);
        if (first.units == last) continue;
        last = first.units;
        const int full = first.wgs / kPrefixWgs, rest = first.wgs % kPrefixWgs;
        const float idle = rest ? kPrefixWgs - rest : 0, done = (full + (rest ? 1 : 0)) * first.us;
        for (int j = 0; j < n_own; ++j) {
            const SliceCost& c = own[j];
            if (!launchable((int64_t)first.wgs + c.wgs + 16, kPrefixThreads)) break;      // (more slices of these are more still; one each always fits)
            float us = done + spread_us(c, c.wgs, kPrefixWgs);       // behind the prefix's workgroups, or in the idle places of their last round
            if (idle > 0) us = std::min(us, std::max(done, full * first.us + spread_us(c, c.wgs, idle)));
            us += ((float)first.units * lo->part[0].rows + (float)c.units * lo->part[1].rows) * p->H_kv * state_us;
            if (us < best) {
                best = us;
                if (shared) put(&lo->part[0], first);
                put(&lo->part[1], c);
            }
        }
    }
}

int prefix_layout(const ssv_prefix_params* p, PrefixLayout* lo) {
    if (!p) return SSV_EINVAL;
    if (p->B < 1 || p->T < 1 || p->H < 1 || p->H_kv < 1 || p->d_k < 1 || p->d_v < 1) return SSV_EINVAL;
    if (p->H % p->H_kv || p->n_prefix < 1 || p->B % p->n_prefix) return SSV_EINVAL;
    if (p->dtype != SSV_F32 && p->dtype != SSV_BF16) return SSV_EINVAL;
    if (p->max_prefix_len < 0 || p->max_seq_len < 0 || !(p->scale >= 0.f) || std::isinf(p->scale)) return SSV_EINVAL;
    const int H_g = p->H / p->H_kv;
    if (p->T > SSV_MAX_T || (p->scale > 0.f && !(p->scale >= 0x1p-100f && p->scale <= 0x1p100f))) return SSV_EUNSUPPORTED;      // (scale * log2(e) stays normal)
    if (H_g != 1 && H_g != 2 && H_g != 4 && H_g != 8 && H_g != 16) return SSV_EUNSUPPORTED;
    if (!ssv_nsa_supported(p->dtype, p->d_k, p->d_v)) return SSV_EUNSUPPORTED;
    if (p->max_seq_len > INT32_MAX - SSV_MAX_T - 64 || p->max_prefix_len > INT32_MAX - 64) return SSV_EUNSUPPORTED;
    const int es = p->dtype == SSV_BF16 ? 2 : 4;
    const int64_t* strides[4] = {p->kp_stride, p->vp_stride, p->k_stride, p->v_stride};
    for (int s = p->max_prefix_len ? 0 : 2; s < 4; ++s)
        for (int j = 0; j < 3; ++j) {
            if (strides[s][j] < 0 || strides[s][j] * es % 16) return SSV_EINVAL;
            if (j == 2 && strides[s][j] < (s % 2 ? p->d_v : p->d_k)) return SSV_EINVAL;
            // a tile's rows are addressed by 31-bit offsets from its first one
            if (j == 2 && strides[s][j] * es >= (1 << 25)) return SSV_EUNSUPPORTED;
        }
    std::memset(lo, 0, sizeof(*lo));
    const int64_t* given[2] = {p->q_stride, p->out_stride};
    int64_t* bytes[2] = {lo->q_s, lo->out_s};
    const int dd[2] = {p->d_k, p->d_v};
    for (int s = 0; s < 2; ++s) {
        const bool dense = !given[s][0] && !given[s][1] && !given[s][2];
        const int64_t st[3] = {dense ? (int64_t)p->T * p->H * dd[s] : given[s][0], dense ? (int64_t)p->H * dd[s] : given[s][1],
                               dense ? dd[s] : given[s][2]};
        for (int j = 0; j < 3; ++j) {
            if (st[j] < 0 || st[j] * es % 16) return SSV_EINVAL;
            bytes[s][j] = st[j] * es;
        }
        if (!dense && st[2] < dd[s] && p->H > 1) return SSV_EINVAL;
    }
    if (repeats(p->B, lo->out_s[0]) || repeats(p->T, lo->out_s[1])) return SSV_EINVAL;
    lo->H_g = H_g;
    lo->es = es;
    lo->rows_total = (int64_t)p->B * p->T * p->H;
    if (!launchable(lo->rows_total + kThreads, p->d_v / 4)) return SSV_EUNSUPPORTED;      // (k_prefix_combine; sizes fit 31 bits)
    const bool bf16 = p->dtype == SSV_BF16;
    PartPlan& shared = lo->part[0];
    if (p->max_prefix_len) {
        shared.caches = p->n_prefix;
        shared.per = p->B / p->n_prefix;
        shared.rows = shared.per * p->T * H_g;
        if (const int rc = plan_rows(&shared, bf16, p->H_kv)) return rc;
    }
    PartPlan& own = lo->part[1];
    own.caches = p->B;
    own.per = 1;
    own.rows = p->T * H_g;
    if (const int rc = plan_rows(&own, bf16, p->H_kv)) return rc;
    plan_slices(lo, p);
    lo->n_slots = shared.slots + own.slots;
    lo->off_stats = 0;
    lo->off_acc = align_up((size_t)lo->n_slots * lo->rows_total * 8, 256);
    lo->total = align_up(lo->off_acc + (size_t)lo->n_slots * lo->rows_total * p->d_v * 4, 256);
    return SSV_OK;
}

template <bool BF16, int DK, int DV, int PREFIX, int OWN>
int prefix_enqueue(const PrefixArgs& a, hipStream_t stream) {
    constexpr int rows = PREFIX == 0 || OWN == 0 ? PrefixRowsCfg<DK, DV>::LDS : 0;
    constexpr int keys = PREFIX != 0 || OWN != 0 ? PrefixKeysCfg<DV>::LDS : 0;
    constexpr int lds = rows > keys ? rows : keys;
    const auto fn = k_prefix<BF16, DK, DV, PREFIX, OWN>;
    if (lds > 64 * 1024) {      // once per device and kernel
        static std::atomic<bool> raised[kMaxDevices];
        int dev = 0;
        if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return SSV_ELAUNCH;
        if (!raised[dev].load(std::memory_order_acquire)) {
            if (hipFuncSetAttribute((const void*)fn, hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess) return SSV_ELAUNCH;
            raised[dev].store(true, std::memory_order_release);
        }
    }
    hipLaunchKernelGGL(fn, dim3(a.part[0].n_pad + a.part[1].n_pad), dim3(kPrefixThreads), lds, stream, a);
    return hipGetLastError() == hipSuccess ? SSV_OK : SSV_ELAUNCH;
}

template <bool BF16, int DK, int DV>
int prefix_launch(const void* q, const void* kp, const void* vp, const void* k, const void* v, const int32_t* prefix_lens,
                  const int32_t* seq_lens, const int32_t* n_query, const int32_t* parents, const ssv_prefix_params* p, void* out,
                  char* ws, const PrefixLayout& lo, hipStream_t stream) {
    const float scale = p->scale > 0.f ? p->scale : 1.f / std::sqrt((float)p->d_k);
    PrefixArgs a{};
    a.q = (const char*)q;
    a.n_query = n_query;
    a.parents = parents;
    a.part_stats = (float*)(ws + lo.off_stats);
    a.part_acc = (float*)(ws + lo.off_acc);
    a.T = p->T; a.H = p->H; a.H_kv = p->H_kv; a.H_g = lo.H_g;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.rows_total = lo.rows_total;
    a.div_TH = FastDiv::of(p->T * lo.H_g);
    a.div_Hg = FastDiv::of(lo.H_g);
    for (int j = 0; j < 3; ++j) a.q_s[j] = lo.q_s[j];
    for (int own = 0; own < 2; ++own) {
        const PartPlan& pl = lo.part[own];
        PrefixPart& pt = a.part[own];
        pt.k = (const char*)(own ? k : kp);
        pt.v = (const char*)(own ? v : vp);
        pt.lens = own ? seq_lens : prefix_lens;
        pt.caches = pl.caches; pt.per = pl.per; pt.rows = pl.rows; pt.n_rg = pl.n_rg;
        pt.max_len = own ? p->max_seq_len : p->max_prefix_len;
        pt.units = pl.units; pt.slots = pl.slots; pt.min_tiles = pl.min_tiles;
        pt.slot0 = own ? lo.part[0].slots : 0;
        pt.by_length = pl.by_length;
        pt.div_groups = FastDiv::of(p->H_kv * pl.n_rg);
        pt.div_rg = FastDiv::of(pl.n_rg);
        pt.div_slices = FastDiv::of(pl.slots);
        pt.n_wg = pl.units * p->H_kv * pl.n_rg;
        pt.n_pad = (int)align_up(pt.n_wg, 8);
        for (int j = 0; j < 3; ++j) {
            pt.k_s[j] = (own ? p->k_stride : p->kp_stride)[j] * lo.es;
            pt.v_s[j] = (own ? p->v_stride : p->vp_stride)[j] * lo.es;
        }
    }
    // the prefix's rows are the own ones of one sequence or more: its path is the same or the next one up
    const int own = lo.part[1].path, shared = lo.part[0].units ? lo.part[0].path : own;
    constexpr int MANY = BF16 ? 0 : 2;
    const int rc = own == MANY      ? prefix_enqueue<BF16, DK, DV, MANY, MANY>(a, stream)
                   : shared == MANY ? prefix_enqueue<BF16, DK, DV, MANY, 1>(a, stream)
                                    : prefix_enqueue<BF16, DK, DV, 1, 1>(a, stream);
    if (rc != SSV_OK) return rc;
    PrefixCombineArgs c{};
    c.part_stats = (const float*)(ws + lo.off_stats);
    c.part_acc = (const float*)(ws + lo.off_acc);
    c.n_query = n_query;
    c.out = (char*)out;
    c.T = p->T; c.H = p->H; c.n_slots = lo.n_slots;
    c.rows_total = lo.rows_total;
    c.div_H = FastDiv::of(p->H);
    c.div_T = FastDiv::of(p->T);
    for (int j = 0; j < 3; ++j) c.out_s[j] = lo.out_s[j];
    // Up to two workgroups per CU fetch sums before they know whether they count, more of them only what counts: 4096 rows of 128 5.5
    // and 6.3 us, 8192 rows 9.8 and 9.6, 12800 rows (four slots of eight in use) 10.3 and 6.2, 22848 rows 16 and 9.4.
    const int wgs = ceil_div(lo.rows_total, kThreads / (DV / 4));
    if (wgs <= 2 * kPrefixWgs) hipLaunchKernelGGL((k_prefix_combine<BF16, DV, true>), dim3(wgs), dim3(kThreads), 0, stream, c);
    else hipLaunchKernelGGL((k_prefix_combine<BF16, DV, false>), dim3(wgs), dim3(kThreads), 0, stream, c);
    return hipGetLastError() == hipSuccess ? SSV_OK : SSV_ELAUNCH;
}

// ---- sampling
int sample_check(const ssv_sample_params* p, int64_t s[2]) {
    if (!p || p->B < 1 || p->T < 1 || p->V < 1) return SSV_EINVAL;
    if (p->dtype != SSV_F32 && p->dtype != SSV_BF16) return SSV_EINVAL;
    if (p->logits_stride[0] < 0 || p->logits_stride[1] < 0) return SSV_EINVAL;
    const int64_t rows = (int64_t)p->B * p->T;
    if (p->V > SSV_SAMPLE_MAX_V || !launchable(rows, kSampleThreads) ||
        !launchable(rows * ceil_div(sample_blocks(p->V), kThreads / 64), kThreads)) return SSV_EUNSUPPORTED;
    const int es = p->dtype == SSV_BF16 ? 2 : 4;
    const bool dense = !p->logits_stride[0] && !p->logits_stride[1];
    s[0] = (dense ? (int64_t)p->T * p->V : p->logits_stride[0]) * es;
    s[1] = (dense ? (int64_t)p->V : p->logits_stride[1]) * es;
    return SSV_OK;
}

size_t sample_blocks_bytes(const ssv_sample_params* p) {
    return align_up((size_t)p->B * p->T * sample_blocks(p->V) * sizeof(SampleBlock), 256);
}
size_t sample_maxima_bytes(const ssv_sample_params* p) { return (size_t)p->B * p->T * sample_blocks(p->V) * kSampleChunks * 2; }

}  // namespace

extern "C" {

size_t ssv_prefix_workspace_bytes(const ssv_prefix_params* p) {
    PrefixLayout lo;
    return prefix_layout(p, &lo) == SSV_OK ? lo.total : 0;
}

int ssv_prefix_verify(const void* q, const void* k_prefix, const void* v_prefix, const void* k, const void* v,
                      const int32_t* prefix_lens, const int32_t* seq_lens, const int32_t* n_query, const int32_t* tree_parents,
                      const ssv_prefix_params* p, void* out, void* workspace, size_t workspace_bytes, void* stream) {
    PrefixLayout lo;
    const int rc = prefix_layout(p, &lo);
    if (rc != SSV_OK) return rc;
    if (!q || !k || !v || !seq_lens || !out) return SSV_EINVAL;
    if (p->max_prefix_len && (!k_prefix || !v_prefix || !prefix_lens)) return SSV_EINVAL;
    const void* rows[] = {q, k, v, out, p->max_prefix_len ? k_prefix : nullptr, p->max_prefix_len ? v_prefix : nullptr};
    for (const void* r : rows)
        if (misaligned(r, 16)) return SSV_EINVAL;
    const void* words[] = {p->max_prefix_len ? prefix_lens : nullptr, seq_lens, n_query, tree_parents};
    for (const void* w : words)
        if (misaligned(w, 4)) return SSV_EINVAL;
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < lo.total) return SSV_EWORKSPACE;
#define SSV_DISPATCH(BF, DK, DV)                                                                                          \
    if (p->dtype == ((BF) ? SSV_BF16 : SSV_F32) && p->d_k == (DK) && p->d_v == (DV))                                      \
        return prefix_launch<BF, DK, DV>(q, k_prefix, v_prefix, k, v, prefix_lens, seq_lens, n_query, tree_parents, p, out, \
                                         (char*)workspace, lo, (hipStream_t)stream);
    SSV_DISPATCH(true, 192, 128)
    SSV_DISPATCH(true, 128, 128)
    SSV_DISPATCH(true, 64, 64)
    SSV_DISPATCH(false, 64, 64)
#undef SSV_DISPATCH
    return SSV_EUNSUPPORTED;
}

size_t ssv_sample_workspace_bytes(const ssv_sample_params* p) {
    int64_t s[2];
    return sample_check(p, s) == SSV_OK ? sample_blocks_bytes(p) + sample_maxima_bytes(p) : 0;
}

int ssv_sample(const void* logits, const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
               const float* u, const int32_t* n_query, const ssv_sample_params* p, int32_t* tokens, float* probs,
               void* workspace, size_t workspace_bytes, void* stream) {
    SampleArgs a{};
    const int rc = sample_check(p, a.s);
    if (rc != SSV_OK) return rc;
    if (!logits || !u || !tokens) return SSV_EINVAL;
    if (misaligned(logits, p->dtype == SSV_BF16 ? 2 : 4)) return SSV_EINVAL;
    const void* words[] = {temperature, top_k, top_p, min_p, u, n_query, tokens, probs};
    for (const void* w : words)
        if (misaligned(w, 4)) return SSV_EINVAL;
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < sample_blocks_bytes(p) + sample_maxima_bytes(p)) return SSV_EWORKSPACE;
    a.logits = (const char*)logits;
    a.temperature = temperature; a.top_p = top_p; a.min_p = min_p; a.u = u; a.top_k = top_k; a.n_query = n_query;
    a.tokens = tokens; a.probs = probs;
    a.blocks = (SampleBlock*)workspace;
    a.maxima = (uint16_t*)((char*)workspace + sample_blocks_bytes(p));
    a.T = p->T; a.V = p->V;
    a.n_blocks = sample_blocks(p->V);
    a.wg_per_row = ceil_div(a.n_blocks, kThreads / 64);
    a.div_wg = FastDiv::of(a.wg_per_row);
    a.div_T = FastDiv::of(p->T);
    const dim3 grid(p->B * p->T * a.wg_per_row), rows(p->B * p->T);
    if (p->dtype == SSV_BF16) {
        hipLaunchKernelGGL(k_sample_blocks<true>, grid, dim3(kThreads), 0, (hipStream_t)stream, a);
        if (hipGetLastError() != hipSuccess) return SSV_ELAUNCH;
        hipLaunchKernelGGL(k_sample_pick<true>, rows, dim3(kSampleThreads), 0, (hipStream_t)stream, a);
    } else {
        hipLaunchKernelGGL(k_sample_blocks<false>, grid, dim3(kThreads), 0, (hipStream_t)stream, a);
        if (hipGetLastError() != hipSuccess) return SSV_ELAUNCH;
        hipLaunchKernelGGL(k_sample_pick<false>, rows, dim3(kSampleThreads), 0, (hipStream_t)stream, a);
    }
    return hipGetLastError() == hipSuccess ? SSV_OK : SSV_ELAUNCH;
}

int ssv_accept(const int32_t* draft_tokens, const int32_t* root_tokens, const int32_t* sampled, const int32_t* seq_lens,
               const int32_t* n_query, const int32_t* tree_parents, int32_t B, int32_t T, int32_t* path, int32_t* n_accepted,
               int32_t* next_tokens, int32_t* committed, void* stream) {
    if (B < 1 || T < 1) return SSV_EINVAL;
    if (T > SSV_MAX_T || !launchable(ceil_div(B, kThreads / 64), kThreads)) return SSV_EUNSUPPORTED;
    if (!draft_tokens || !root_tokens || !sampled || !seq_lens || !path || !n_accepted || !next_tokens || !committed) return SSV_EINVAL;
    const void* words[] = {draft_tokens, root_tokens, sampled, seq_lens, n_query, tree_parents, path, n_accepted, next_tokens, committed};
    for (const void* w : words)
        if (misaligned(w, 4)) return SSV_EINVAL;
    const AcceptArgs a{draft_tokens, root_tokens, sampled, seq_lens, n_query, tree_parents, path, n_accepted, next_tokens, committed, B, T};
    hipLaunchKernelGGL(k_accept, dim3(ceil_div(B, kThreads / 64)), dim3(kThreads), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? SSV_OK : SSV_ELAUNCH;
}

int ssv_commit(void* k, void* v, const int32_t* path, const int32_t* n_accepted, const int32_t* seq_lens,
               const ssv_commit_params* p, void* stream) {
    if (!p || p->layers < 1 || p->B < 1 || p->T < 1 || p->H_kv < 1 || p->d_k < 1 || p->d_v < 1 || p->kv_capacity < 0) return SSV_EINVAL;
    if (p->dtype != SSV_F32 && p->dtype != SSV_BF16) return SSV_EINVAL;
    if (p->T > SSV_MAX_T) return SSV_EUNSUPPORTED;
    const int es = p->dtype == SSV_BF16 ? 2 : 4;
    if ((int64_t)p->d_k * es % 16 || (int64_t)p->d_v * es % 16) return SSV_EINVAL;
    const int64_t* strides[2] = {p->k_stride, p->v_stride};
    for (int s = 0; s < 2; ++s)
        for (int j = 0; j < 4; ++j) {
            if (strides[s][j] < 0 || strides[s][j] * es % 16) return SSV_EINVAL;
            if (j == 3 && strides[s][j] < (s ? p->d_v : p->d_k)) return SSV_EINVAL;
            const int extents[4] = {p->layers, p->B, p->H_kv, 1};
            if (repeats(extents[j], strides[s][j])) return SSV_EINVAL;
        }
    if (!k || !v || !path || !n_accepted || !seq_lens || misaligned(k, 16) || misaligned(v, 16)) return SSV_EINVAL;
    if (misaligned(path, 4) || misaligned(n_accepted, 4) || misaligned(seq_lens, 4)) return SSV_EINVAL;
    CommitArgs a{};
    a.k = (char*)k; a.v = (char*)v;
    a.path = path; a.n_accepted = n_accepted; a.seq_lens = seq_lens;
    a.B = p->B; a.T = p->T; a.H_kv = p->H_kv; a.cap = p->kv_capacity;
    a.k_chunks = p->d_k * es / 16;
    a.chunks = a.k_chunks + p->d_v * es / 16;
    const int64_t pairs = (int64_t)p->layers * p->B * p->H_kv;
    if (pairs >= (1ll << 31) || !launchable(pairs, a.chunks) || !launchable(ceil_div(pairs * a.chunks, kThreads), kThreads)) return SSV_EUNSUPPORTED;
    a.total = pairs * a.chunks;
    for (int j = 0; j < 4; ++j) {
        a.k_s[j] = p->k_stride[j] * es;
        a.v_s[j] = p->v_stride[j] * es;
    }
    hipLaunchKernelGGL(k_commit, dim3(ceil_div(a.total, kThreads)), dim3(kThreads), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? SSV_OK : SSV_ELAUNCH;
}

}  // extern "C"
