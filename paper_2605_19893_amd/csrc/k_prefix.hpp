// Dense verification attention over a shared prefix and each sequence's own rows.
//
//   out = sum_s p_s v_s,  p = softmax_s(scale q . k_s),  s over the prefix and over the sequence's visible slots
//
// is split over slices of keys; every slice leaves a partial softmax state (m, Z = sum 2^(x - m), sum 2^(x - m) v) per row and
// k_prefix_combine joins them.  The rows that meet a prefix are those of all its sequences, stacked: row r of a (prefix, KV
// head) pair is (sequence, node, head of the group) = (r / (T H_g), r / H_g % T, r % H_g), so a prefix row is read once for
// all rows of a workgroup.  The rows that meet a sequence's own keys are the same with one sequence.
//
// One launch holds the workgroups of both parts, each on the path that its row count asks for:
//   rows path (prefix_rows, bf16, more than 16 rows): up to 256 rows share every key tile through LDS, one block of 32 rows per
//     wavefront on the 32x32x16 matrix instruction: bound by the matrix cores when the rows are many;
//   keys path (prefix_keys): 16 rows (fp32: up to 32); the wavefronts divide the keys instead, nothing is shared: bound by memory.
//
// Measured (kernel alone, MI355X): chains of 16 in 32 sequences of 64 heads behind 32768 shared and 2048 own rows, 192 + 128:
// 582 to 592 us apart from each other, 1.20 to 1.22 PFLOP/s, where a large matrix product of the library reaches 1.25 on the same
// card (up to 684 us in some dozen launches one behind the other); one token each in 32 sequences behind 16411 + 1024: 36.8 us
// for 92 MB and 22 GFLOP (18 us of either): 160 workgroups have 13 prefix tiles each, 27 us on the matrix cores, 96 of the 128 that
// stream own keys run beside them on the other CUs and the last 32 behind, and 7 us pass before the first tile and after the last; four
// sequences behind 2048 + 128: 9.4 us, all of it latency; fp32 chains of five behind 4097 + 300: 17.2 us.
#pragma once
#include <type_traits>

#include "device_common.hpp"
#include "wave_ops.hpp"

namespace ssv {

struct PrefixPart {
    const char *k, *v;                 // the prefixes, or the sequences' own caches
    const int32_t* lens;               // rows of each prefix, or committed tokens of each sequence
    int caches, per;                   // per: sequences that share a cache (1: the sequences' own)
    int rows, n_rg;                    // rows per (cache, KV head); groups of them, one per workgroup
    int max_len;
    int units;                         // slices of all caches together; each is taken by H_kv * n_rg workgroups
    int slots, slot0;                  // partial-state slots per row (slices a cache can have), and the first one
    int min_tiles;                     // tiles of 64 keys that a slice holds at least
    int by_length;                     // 1: the slices are dealt out by the lengths; 0: units / caches to every cache
    FastDiv div_groups, div_rg, div_slices;
    int n_wg, n_pad;                   // workgroups, and the same rounded up to a multiple of 8
    int64_t k_s[3], v_s[3];            // bytes: cache, KV head, row
};

struct PrefixArgs {
    PrefixPart part[2];                // prefix, own
    const char* q;
    const int32_t *n_query, *parents;
    float *part_stats, *part_acc;
    int T, H, H_kv, H_g;
    float scale_log2;
    int64_t rows_total;
    FastDiv div_TH, div_Hg;
    int64_t q_s[3];                    // bytes: sequence, node, head
};

constexpr int kPrefixThreads = 512;
constexpr int kPrefixWaves = kPrefixThreads / 64;
constexpr int kPrefixStep = 32;        // keys per step of a wavefront on the keys path
constexpr int kPrefixMaxSlots = 128;   // partial states per row
constexpr int kPrefixMinTiles = 2;     // tiles of 64 keys that a slice holds at least
constexpr int kPrefixMaxDealt = 64;    // caches whose slices are dealt out by length: a lane each
constexpr float kPrefixRaiseLog2 = 8.f;   // the reference maximum follows the running one at a distance of up to 2^8

struct PrefixTree {                    // LDS: the draft tree of one sequence
    AncSet anc[kMaxT];
    int par[kMaxT];
};

// Ancestors-or-self of every node of one sequence (the set bits of s_anc[i]), from the parent indices; null: a chain.
__device__ __forceinline__ void build_ancestors(int tid, int b, int T, int Tq, const int32_t* parents, int* s_par, AncSet* s_anc) {
    if (parents) {
        if (tid < kMaxT) {
            int par = tid < Tq ? parents[(int64_t)b * T + tid] : -1;
            s_par[tid] = (par >= tid || par < -1) ? -1 : par;
        }
        __syncthreads();
    }
    if (tid < kMaxT) {
        AncSet anc = {0ull, 0ull};
        if (!parents) {
            anc.lo = (tid >= 63) ? ~0ull : ((2ull << tid) - 1ull);
            anc.hi = (tid < 64) ? 0ull : ((tid == 127) ? ~0ull : ((2ull << (tid - 64)) - 1ull));
        } else {
            for (int t = tid; t >= 0; t = s_par[t]) {      // strictly decreasing
                if (t < 64) anc.lo |= 1ull << t; else anc.hi |= 1ull << (t - 64);
            }
        }
        s_anc[tid] = anc;
    }
    __syncthreads();
}

// Bits of the 32 keys from slot0 on that a row sees: the slots below `len`, and draft slot len + t for every t in anc.
__device__ __forceinline__ uint32_t visible_word(AncSet anc, int len, int slot0) {
    const int off = slot0 - len;
    if (off >= 128) return 0u;
    if (off >= 64) return (uint32_t)(anc.hi >> (off - 64));
    if (off > 0) return (uint32_t)((anc.lo >> off) | (anc.hi << (64 - off)));
    if (off > -32) return (uint32_t)((anc.lo << -off) | ((1ull << -off) - 1ull));
    return ~0u;
}

// sum + the two bf16 values of a register.
__device__ __forceinline__ float add_bf16_pair(uint32_t pair, float sum) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3f803f80u), sum, false);
}

// What a workgroup of either path works on.
//
// The host deals out workgroups without knowing the lengths.  With up to 64 caches every wavefront reads them all, a lane each,
// and finds the least slice length L (nearly) for which the slices of all caches are no more than the units there are:
//   sum_c max(1, ceil(tiles_c / L)) <= units;
// slices are then equally long whatever the lengths are.  (Two prompts of 12K and 6K rows with equal counts: the shorter one's
// workgroups are done in half the time.)  With one cache, or more than 64, every cache has the same number of slices.
struct PrefixWork {
    int rg, slice, cache, g;
    int len, Tq, n_keys;               // Tq: nodes of the sequence (own caches only)
    int t0, t1;                        // tiles of 64 keys
    bool any, last;                    // there is a slice for this workgroup; it is its cache's last one
};
template <bool OWN>
__device__ __forceinline__ PrefixWork prefix_work(const PrefixArgs& a, int wg) {
    const PrefixPart& pt = a.part[OWN];
    PrefixWork w;
    const int unit = pt.div_groups.div(wg), in = wg - unit * (a.H_kv * pt.n_rg);
    w.g = pt.div_rg.div(in);
    w.rg = in - w.g * pt.n_rg;                             // neighbours read the same keys
    if (pt.by_length) {                                    // (uniform)
        const int c = threadIdx.x & 63, cc = min(c, pt.caches - 1);
        const int len = min(max(pt.lens[cc], 0), pt.max_len);
        const int Tq = OWN ? (a.n_query ? min(max(a.n_query[cc], 0), a.T) : a.T) : 0;
        const bool there = c < pt.caches && (!OWN || Tq > 0);      // (a sequence without nodes has no rows)
        const int tiles = there ? (len + Tq + kTile - 1) / kTile : 0;
        int L = max(pt.min_tiles, (wave_sum(tiles) + pt.units - 1) / pt.units), n, end;
        for (;;) {                     // ends: with L at the longest cache's tiles there is one slice per cache
            n = there ? max(1, (tiles + L - 1) / L) : 0;
            end = wave_incl_scan(n);
            if (last_lane(end) <= pt.units) break;
            L += max(1, L >> 4);
        }
        const uint64_t m = __builtin_amdgcn_ballot_w64(n > 0 && end - n <= unit);
        w.any = unit < last_lane(end);
        w.cache = m ? 63 - __builtin_clzll(m) : 0;
        w.slice = unit - __builtin_amdgcn_readlane(end - n, w.cache);
        w.last = w.slice + 1 == __builtin_amdgcn_readlane(n, w.cache);
        w.len = __builtin_amdgcn_readlane(len, w.cache);
        w.Tq = __builtin_amdgcn_readlane(Tq, w.cache);
        w.n_keys = w.len + w.Tq;
        const int n_tiles = (w.n_keys + kTile - 1) / kTile;
        w.t0 = min(n_tiles, w.slice * L);
        w.t1 = min(n_tiles, w.t0 + L);
    } else {
        w.cache = pt.div_slices.div(unit);
        w.slice = unit - w.cache * pt.slots;
        w.any = true;
        w.last = w.slice + 1 == pt.slots;
        w.len = min(max(pt.lens[w.cache], 0), pt.max_len);
        w.Tq = OWN ? (a.n_query ? min(max(a.n_query[w.cache], 0), a.T) : a.T) : 0;
        w.n_keys = w.len + w.Tq;
        const int n_tiles = (w.n_keys + kTile - 1) / kTile;
        const int L = max(pt.div_slices.div(n_tiles + pt.slots - 1), pt.min_tiles);
        w.t0 = min(n_tiles, w.slice * L);
        w.t1 = min(n_tiles, w.t0 + L);
    }
    return w;
}

// Row r of a (cache, KV head): its sequence, node and head; and whether it exists.
struct PrefixRow { int b, i, h; };
template <bool OWN>
__device__ __forceinline__ PrefixRow prefix_row(const PrefixArgs& a, const PrefixWork& w, int r) {
    const int rc = min(r, a.part[OWN].rows - 1);
    const int bl = OWN ? 0 : a.div_TH.div(rc), in = rc - bl * a.T * a.H_g;
    PrefixRow x;
    x.i = a.div_Hg.div(in);
    x.h = w.g * a.H_g + in - x.i * a.H_g;
    x.b = w.cache * a.part[OWN].per + bl;
    return x;
}
template <bool OWN>
__device__ __forceinline__ bool prefix_row_exists(const PrefixArgs& a, const PrefixWork& w, const PrefixRow& x, int r) {
    return r < a.part[OWN].rows && x.i < (OWN ? w.Tq : (a.n_query ? a.n_query[x.b] : a.T));
}
__device__ __forceinline__ int64_t prefix_state_row(const PrefixArgs& a, const PrefixRow& x) { return ((int64_t)x.b * a.T + x.i) * a.H + x.h; }

// (m, Z) of a row's slice; the cache's last slice marks the slots behind its own as empty.
__device__ __forceinline__ void put_statistics(const PrefixArgs& a, const PrefixPart& pt, const PrefixWork& w, int64_t row, float m, float Z) {
    float* at = a.part_stats + ((int64_t)(pt.slot0 + w.slice) * a.rows_total + row) * 2;
    *reinterpret_cast<float2*>(at) = make_float2(m, Z);
    if (w.last)
        for (int s = w.slice + 1; s < pt.slots; ++s) *reinterpret_cast<float2*>(at += a.rows_total * 2) = make_float2(0.f, 0.f);
}

// ---- keys path --------------------------------------------------------------------------------------------------------
// One workgroup = 16 RB rows of one (cache, KV head) x one slice of its keys.  Its wavefronts hold the same rows and take
// the slice's steps of 32 keys in turn, each with a softmax state of its own, merged in LDS at the end: no barrier while keys
// are streamed.  K fragments are loaded as the matrix instruction wants them (lane: one key, 16 bytes); V rows are loaded as
// they lie, a lane holding DV / 16 neighbouring columns of the eight keys whose probabilities it holds after S^T = K Q^T
// (four of each block of 16), and a byte permutation per register turns them into the operand of O^T = V^T P^T: matrix
// instruction j then sums column DV / 16 * m + j of every lane group m.  Nothing passes through LDS on the way.
template <int DV>
struct PrefixKeysCfg {
    static constexpr int PITCH = DV + 4;
    static constexpr int LDS = kPrefixWaves * 16 * PITCH * 4;
};

template <bool BF16, int DK, int DV, int RB, bool OWN>
__device__ __forceinline__ void prefix_keys(const PrefixArgs& a, int wg, char* smem, PrefixTree& tree) {
    constexpr int ES = BF16 ? 2 : 4;
    constexpr int KC = DK * ES / 64;             // 64-byte chunks of a K row
    constexpr int CW = DV / 16;                  // V columns per lane
    constexpr int VW = CW * ES / 4;              // 32-bit words of them
    constexpr int PITCH = PrefixKeysCfg<DV>::PITCH;
    __shared__ float s_m[kPrefixWaves][16 * RB], s_z[kPrefixWaves][16 * RB];
    float* s_acc = reinterpret_cast<float*>(smem);

    const PrefixPart& pt = a.part[OWN];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = lane & 15, G = lane >> 4;
    // ---- rows
    const PrefixWork w = prefix_work<OWN>(a, wg);
    if (!w.any) return;
    PrefixRow row[RB];
    u32x4 qf[RB][KC];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        row[rb] = prefix_row<OWN>(a, w, (w.rg * RB + rb) * 16 + n);
        const char* qp = a.q + row[rb].b * a.q_s[0] + row[rb].i * a.q_s[1] + row[rb].h * a.q_s[2] + G * 16;
#pragma unroll
        for (int c = 0; c < KC; ++c) qf[rb][c] = *reinterpret_cast<const u32x4*>(qp + c * 64);
    }

    // ---- this slice's steps
    const int t0 = w.t0 * (kTile / kPrefixStep), t1 = min(w.t1 * (kTile / kPrefixStep), (w.n_keys + kPrefixStep - 1) / kPrefixStep);
    const char* kbase = pt.k + w.cache * pt.k_s[0] + w.g * pt.k_s[1] + G * 16;
    const char* vbase = pt.v + w.cache * pt.v_s[0] + w.g * pt.v_s[1] + n * (CW * ES);
    const uint32_t krow = (uint32_t)pt.k_s[2], vrow = (uint32_t)pt.v_s[2];

    u32x4 kf[2][KC];
    uint32_t vf[2][4][VW];
    auto load_k = [&](int t) {
        const char* p = kbase + (int64_t)t * kPrefixStep * pt.k_s[2];
        const int last = w.n_keys - 1 - t * kPrefixStep;       // rows behind the last one repeat it; their scores are masked
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const char* r = p + (uint32_t)min(kb * 16 + n, last) * krow;
#pragma unroll
            for (int c = 0; c < KC; ++c) kf[kb][c] = *reinterpret_cast<const u32x4*>(r + c * 64);
        }
    };
    auto load_v = [&](int t) {
        const char* p = vbase + (int64_t)t * kPrefixStep * pt.v_s[2];
        const int last = w.n_keys - 1 - t * kPrefixStep;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const char* at = p + (uint32_t)min(kb * 16 + 4 * G + r, last) * vrow;
                if constexpr (VW == 4) {
                    const u32x4 x = *reinterpret_cast<const u32x4*>(at);
#pragma unroll
                    for (int e = 0; e < 4; ++e) vf[kb][r][e] = x[e];
                } else {
                    const u32x2 x = *reinterpret_cast<const u32x2*>(at);
                    vf[kb][r][0] = x[0];
                    vf[kb][r][1] = x[1];
                }
            }
    };

    f32x4 acc[RB][CW];
    float mref[RB], z[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        mref[rb] = -INFINITY;
        z[rb] = 0.f;
#pragma unroll
        for (int j = 0; j < CW; ++j) acc[rb][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const float raise = fminf(kPrefixRaiseLog2 / a.scale_log2, 3e38f);      // (finite: -inf + raise stays below every score)
    const int full = OWN ? w.len : w.n_keys;       // keys that every row sees

    int t = t0 + wave;
    if (t < t1) {
        load_k(t);
        load_v(t);
    }
    bool valid[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        valid[rb] = prefix_row_exists<OWN>(a, w, row[rb], (w.rg * RB + rb) * 16 + n);
        if (!valid[rb]) {
#pragma unroll
            for (int c = 0; c < KC; ++c) qf[rb][c] = u32x4{0, 0, 0, 0};
        }
    }
    if constexpr (OWN) build_ancestors(tid, w.cache, a.T, w.Tq, a.parents, tree.par, tree.anc);
    for (; t < t1; t += kPrefixWaves) {
        const int next = t + kPrefixWaves;
        f32x4 s[RB][2];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                s[rb][kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < KC; ++c) s[rb][kb] = mma_frag<BF16>(kf[kb][c], qf[rb][c], s[rb][kb]);
            }
        if (next < t1) load_k(next);
        u32x4 pk[RB][BF16 ? 1 : 2];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            if ((t + 1) * kPrefixStep > full) {      // (uniform)
                const uint32_t word = OWN ? visible_word(tree.anc[row[rb].i], w.len, t * kPrefixStep) : (1u << (w.n_keys - t * kPrefixStep)) - 1u;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (!((word >> (kb * 16 + 4 * G + r)) & 1u)) s[rb][kb][r] = -INFINITY;
            }
            float mx = max_nan(max_nan(max_nan(s[rb][0][0], s[rb][0][1]), max_nan(s[rb][0][2], s[rb][0][3])),
                               max_nan(max_nan(s[rb][1][0], s[rb][1][1]), max_nan(s[rb][1][2], s[rb][1][3])));
            if (__builtin_amdgcn_ballot_w64(mx > mref[rb] + raise) != 0ull) {        // (uniform; rare after the first steps)
                mx = xor32_max(xor16_max(mx));
                const bool up = mx > mref[rb] + raise;
                const float alpha = up ? fast_exp2((mref[rb] - mx) * a.scale_log2) : 1.f;
                mref[rb] = up ? mx : mref[rb];
                z[rb] *= alpha;
#pragma unroll
                for (int j = 0; j < CW; ++j) acc[rb][j] *= alpha;
            }
            const float neg = mref[rb] == -INFINITY ? 0.f : -mref[rb] * a.scale_log2;
            float p[2][4];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 4; ++r) p[kb][r] = fast_exp2(__builtin_fmaf(s[rb][kb][r], a.scale_log2, neg));
            if constexpr (BF16) {      // (rounded for the matrix instruction; Z sums them as rounded, so that their errors cancel in the quotient)
                bf16x8 v;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = (__bf16)p[e >> 2][e & 3];
                pk[rb][0] = __builtin_bit_cast(u32x4, v);
#pragma unroll
                for (int e = 0; e < 4; ++e) z[rb] = add_bf16_pair(pk[rb][0][e], z[rb]);
            } else {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) z[rb] += p[kb][r];
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
                    pk[rb][kb] = u32x4{__float_as_uint(p[kb][0]), __float_as_uint(p[kb][1]), __float_as_uint(p[kb][2]), __float_as_uint(p[kb][3])};
            }
        }
#pragma unroll
        for (int j = 0; j < CW; ++j) {
            if constexpr (BF16) {
                const uint32_t sel = (j & 1) ? 0x07060302u : 0x05040100u;      // the upper or the lower halves of two keys
                const int e = j >> 1;
                const u32x4 vt = {__builtin_amdgcn_perm(vf[0][1][e], vf[0][0][e], sel), __builtin_amdgcn_perm(vf[0][3][e], vf[0][2][e], sel),
                                  __builtin_amdgcn_perm(vf[1][1][e], vf[1][0][e], sel), __builtin_amdgcn_perm(vf[1][3][e], vf[1][2][e], sel)};
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) acc[rb][j] = mma_frag<true>(vt, pk[rb][0], acc[rb][j]);
            } else {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    const u32x4 vt = {vf[kb][0][j], vf[kb][1][j], vf[kb][2][j], vf[kb][3][j]};
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) acc[rb][j] = mma_frag<false>(vt, pk[rb][kb], acc[rb][j]);
                }
            }
        }
        if (next < t1) load_v(next);
    }

    // ---- the wavefronts' states become one
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        z[rb] = xor32_add(xor16_add(z[rb]));
        if (G == 0) {
            s_m[wave][rb * 16 + n] = mref[rb] * a.scale_log2;      // statistics leave the kernel in the log2 domain
            s_z[wave][rb * 16 + n] = z[rb];
        }
    }
    __syncthreads();
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        float M = -INFINITY, Z = 0.f;
#pragma unroll
        for (int o = 0; o < kPrefixWaves; ++o)
            if (!(s_z[o][rb * 16 + n] == 0.f)) M = max_nan(M, s_m[o][rb * 16 + n]);
#pragma unroll
        for (int o = 0; o < kPrefixWaves; ++o)
            if (!(s_z[o][rb * 16 + n] == 0.f)) Z += s_z[o][rb * 16 + n] * fast_exp2(s_m[o][rb * 16 + n] - M);
        // (the maximum as it was rounded for Z: the product taken again would go into one instruction with the difference, unrounded)
        const float f = z[rb] == 0.f ? 0.f : fast_exp2(s_m[wave][rb * 16 + n] - M);
        const int64_t slot = (int64_t)(pt.slot0 + w.slice) * a.rows_total;
        if (wave == 0 && G == 0 && valid[rb]) put_statistics(a, pt, w, prefix_state_row(a, row[rb]), M, Z);
        if (t0 >= t1) continue;                      // (uniform) an empty slice leaves Z = 0 and no sums
        if (rb > 0) __syncthreads();
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < CW; j += 4)
                *reinterpret_cast<f32x4*>(s_acc + (wave * 16 + n) * PITCH + CW * (4 * G + r) + j) =
                    f32x4{acc[rb][j][r] * f, acc[rb][j + 1][r] * f, acc[rb][j + 2][r] * f, acc[rb][j + 3][r] * f};
        __syncthreads();
        for (int e = tid; e < 16 * DV / 4; e += kPrefixThreads) {
            const int rr = e / (DV / 4), c = e % (DV / 4) * 4;
            f32x4 sum = *reinterpret_cast<const f32x4*>(s_acc + rr * PITCH + c);
#pragma unroll
            for (int o = 1; o < kPrefixWaves; ++o) sum += *reinterpret_cast<const f32x4*>(s_acc + (o * 16 + rr) * PITCH + c);
            const int r = (w.rg * RB + rb) * 16 + rr;
            const PrefixRow x = prefix_row<OWN>(a, w, r);
            if (prefix_row_exists<OWN>(a, w, x, r)) *reinterpret_cast<f32x4*>(a.part_acc + (slot + prefix_state_row(a, x)) * DV + c) = sum;
        }
    }
}

// ---- rows path --------------------------------------------------------------------------------------------------------
// One workgroup = 256 rows of one (cache, KV head) x one slice of its keys, one per CU.  K and V tiles of 64 rows go from
// global memory straight into a ring of three LDS stages, two tiles ahead of the one in use; every wavefront multiplies its
// 32 rows with them on the 32x32x16 matrix instruction:
//   S^T = K Q^T in 32-key x 32-row blocks, K rows as the M dimension: a lane holds 16 keys of one row, so row maxima and sums
//   stay in the lane except for one exchange between the lane halves, and P^T (bf16) is directly the B operand of
//   O^T = V^T P^T, whose A operand the transposing LDS read brings.
// A tile is a matrix phase (O of the tile before, S of this one) and a vector phase (softmax, and the loads of a later tile).
// The eight wavefronts run in two halves one phase apart, with a barrier after every phase, so that of the two wavefronts of a
// SIMD one feeds the matrix pipe while the other computes exponentials.  Wavefronts without a row only load.
template <int DK, int DV>
struct PrefixRowsCfg {
    static constexpr int KROW = DK * 2, VROW = DV * 2;      // bytes per row
    static constexpr int STEPS = DK / 16;                   // 16-element contraction steps of S^T = K Q^T
    static constexpr int MB = DV / 32;                      // 32-column blocks of O^T
    static constexpr int KT = kTile * KROW, VT = kTile * VROW;
    static constexpr int STAGE = KT + VT;                   // one stage of the ring: K(t), then V(t)
    static constexpr int LDS = 3 * STAGE;
    static constexpr int ROWS = 32 * kPrefixWaves;
};

template <int DK, int DV, bool OWN>
__device__ __forceinline__ void prefix_rows(const PrefixArgs& a, int wg, char* smem, PrefixTree& tree) {
    using Cfg = PrefixRowsCfg<DK, DV>;
    constexpr int KQ = Cfg::KROW == 256 ? 8 : 4;      // contraction steps after which the swizzle of a K row repeats
    using KLoader = DirectRowTile<Cfg::KROW, KQ == 8 ? 3 : 1, kPrefixThreads>;
    using VLoader = DirectRowTile<Cfg::VROW, 2, kPrefixThreads>;
    constexpr int STEPS = Cfg::STEPS, MB = Cfg::MB, KT = Cfg::KT, KROW = Cfg::KROW, VROW = Cfg::VROW, STAGE = Cfg::STAGE;
    constexpr int KI = KLoader::ITERS, VI = VLoader::ITERS;     // load instructions per wavefront and tile

    const PrefixPart& pt = a.part[OWN];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, hb = lane >> 5;

    // ---- rows: B operands of S^T = K Q^T, row n of this wavefront's block, all contraction steps
    const PrefixWork w = prefix_work<OWN>(a, wg);
    if (!w.any) return;
    const int t0 = w.t0, t1 = w.t1;
    const int r0 = w.rg * Cfg::ROWS + wave * 32;
    const bool live = r0 < pt.rows;                               // (uniform) the wavefront has rows
    const PrefixRow row = prefix_row<OWN>(a, w, r0 + n);
    u32x4 qf[STEPS];
    {
        const char* qp = a.q + row.b * a.q_s[0] + row.i * a.q_s[1] + row.h * a.q_s[2] + hb * 16;
#pragma unroll
        for (int st = 0; st < STEPS; ++st) qf[st] = *reinterpret_cast<const u32x4*>(qp + st * 32);
    }

    // ---- tile loads: K(t), then V(t), in one of three stages of the ring that take turns.  A load moves its pointer on, so that
    //      offsets stay within a tile however long the cache is; past the slice's last tile it is the same instructions with
    //      an empty buffer, which fetch nothing (the counted waits below need no cases).
    const uint32_t krow = (uint32_t)pt.k_s[2], vrow = (uint32_t)pt.v_s[2];
    const int64_t kstep = pt.k_s[2] * kTile, vstep = pt.v_s[2] * kTile;
    const char* knext = pt.k + w.cache * pt.k_s[0] + w.g * pt.k_s[1] + t0 * kstep;      // of the next tile to load
    const char* vnext = pt.v + w.cache * pt.v_s[0] + w.g * pt.v_s[1] + t0 * vstep;
    int kleft = w.n_keys - t0 * kTile, vleft = kleft;             // rows from there on
    int kt_left = t1 - t0, vt_left = t1 - t0;                     // tiles of the slice from there on
    KLoader kld;
    VLoader vld;
    kld.init(krow, tid);
    vld.init(vrow, tid);
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_addr(smem));
    const uint32_t kdst = lds0 + wave * (KI * 1024), vdst = lds0 + KT + wave * (VI * 1024);
    uint32_t kstage = 0, vstage = 0;                              // offsets of the stages that the next loads fill
    auto load = [&](auto& loader, const char*& next, int64_t step, uint32_t row, int& left, int& tiles, uint32_t dst, uint32_t& stage) {
        using Loader = std::remove_reference_t<decltype(loader)>;
        if (tiles > 0 && left < kTile) loader.clamp(row, left, tid);      // (uniform; the last tile: rows behind the last one repeat it)
        const uint64_t at = (uint64_t)next;
        const u32x4 rsrc = {(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, tiles > 0 ? (uint32_t)step : 0u, 0x00020000u};
#pragma unroll
        for (int j = 0; j < Loader::ITERS; ++j) buffer_load_lds16(rsrc, dst + stage + j * 1024, loader.off[j], 0u);
        next += step;
        left -= kTile;
        --tiles;
        stage = stage == 2 * STAGE ? 0u : stage + STAGE;
    };
    auto load_k = [&] { load(kld, knext, kstep, krow, kleft, kt_left, kdst, kstage); };
    auto load_v = [&] { load(vld, vnext, vstep, vrow, vleft, vt_left, vdst, vstage); };
    if (t0 < t1) load_k();

    const bool valid = prefix_row_exists<OWN>(a, w, row, r0 + n);
    if constexpr (OWN) build_ancestors(tid, w.cache, a.T, w.Tq, a.parents, tree.par, tree.anc);
    const AncSet anc = OWN ? tree.anc[row.i] : AncSet{0ull, 0ull};
    arrived(qf);
    if (!valid) {
#pragma unroll
        for (int st = 0; st < STEPS; ++st) qf[st] = u32x4{0, 0, 0, 0};
    }

    // this lane's byte offsets into a K tile for the contraction steps of a 128- or 256-byte group (key row n of a 32-key block,
    // granule 2 q + hb), and into a V tile for the transposing reads of column block mb (key row 4 hb + (p >> 2) of a run of 16
    // keys, 8-byte chunk p & 3 of the 16 columns 32 mb + 16 mh .., p = lane % 16, mh = bit 4 of the lane)
    int koff[KQ], voff[MB];
#pragma unroll
    for (int q = 0; q < KQ; ++q) koff[q] = n * KROW + KLoader::swizzled(n, 2 * q + hb) * 16;
    {
        const int p = lane & 15, mh = (lane >> 4) & 1, r = 4 * hb + (p >> 2);
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) voff[mb] = r * VROW + VLoader::swizzled(r, 4 * mb + 2 * mh) * 16 + (p & 3) * 8;
    }
    const bool late = wave >= kPrefixWaves / 2;      // the half that runs one phase behind
    const int full = (OWN ? w.len : w.n_keys) / kTile;      // tiles below it need no mask

    f32x16 acc[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[mb][i] = 0.f;
    float mref = -INFINITY, neg = 0.f, zrun = 0.f;      // reference maximum, - mref * scale, this lane's part of Z
    float limit = -1.f;     // of a tile's sum in this lane; below 0: the row has no reference yet
    f32x16 s[2];            // scores of a tile, between its matrix phase and its vector phase
    u32x4 pk[2][2];         // its probabilities, between the vector phase and the next matrix phase

    // Between two phases.  Into the even phase of tile t: K(t) and V(t - 1) have landed (issued two tiles ago; loads complete in
    // issue order, and only K(t + 1) and V(t) were issued since), and every wavefront has left K(t - 1) and V(t - 2), whose
    // places K(t + 2) and V(t + 1) take.
    auto boundary = [&](bool into_even) {
        if (into_even) wait_vmcnt<KI + VI>();
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
    };
    auto issue_ahead = [&] {
        load_k();
        load_v();
        __builtin_amdgcn_sched_barrier(0);
    };
    // Matrix phase: O^T += V(tile - 1)^T P^T (not for the first tile), then S^T = K(tile) Q^T (not behind the last one), one
    // stream of fragments with LEAD reads ahead of their matrix instructions.
    //   accumulation, fragment i: 32 columns of V (block i % MB) against keys 16 (i / MB) .. + 15
    //   products, fragment i: contraction step i / 2 of key block i % 2; lane layout of s[kb]: row n, key 32 kb + 8 j + 4 hb + r
    //     at vector index 4 j + r
    const char* kt = smem;              // stage of the tile whose products come next
    const char* vt = smem + KT;         // of the tile before it
    auto matrix_phase = [&](auto first, int tile) {
        constexpr int N_V = decltype(first)::value ? 0 : 4 * MB, N = N_V + 2 * STEPS, LEAD = 6;
        auto frag = [&](int i) {
            if (i < N_V) {
                const int kh = i / MB, mb = i % MB;
                const u32x2 v0 = lds_read_tr16(vt + voff[mb] + (16 * kh) * VROW);
                const u32x2 v1 = lds_read_tr16(vt + voff[mb] + (16 * kh + 8) * VROW);
                return u32x4{v0[0], v0[1], v1[0], v1[1]};
            }
            const int st = (i - N_V) >> 1, kb = (i - N_V) & 1;
            return lds_read16(kt + kb * 32 * KROW + koff[st % KQ] + st / KQ * (KQ * 32));
        };
        __builtin_amdgcn_s_setprio(1);      // above the other half's vector phase, or the first LDS reads would wait for it
        u32x4 fb[LEAD];
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < LEAD; ++i) fb[i] = frag(i);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[kb][i] = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            if (N_V && i == N_V && tile >= t1) break;      // (uniform)
            if (i < N_V) {
                const int kh = i / MB, mb = i % MB;
                acc[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fb[i % LEAD]), __builtin_bit_cast(bf16x8, pk[kh >> 1][kh & 1]),
                                                                  acc[mb], 0, 0, 0);
            } else {
                const int st = (i - N_V) >> 1, kb = (i - N_V) & 1;
                s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fb[i % LEAD]), __builtin_bit_cast(bf16x8, qf[st]), s[kb], 0, 0, 0);
            }
            if (i + LEAD < N) fb[i % LEAD] = frag(i + LEAD);
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(0);
        vt = kt + KT;
        kt = kt == smem + 2 * STAGE ? smem : kt + STAGE;
    };
    // Vector phase, in the log2 domain: scores -> bf16 probabilities (pk[kb][h] = keys 32 kb + 16 h .. + 15 in the order the products
    // delivered them).  Taken against the reference of the tiles before, without looking for a maximum: scores that exceed it show
    // in the sum (a sum above 2^9, infinite or not a number), and only then the reference is raised and the tile taken again.
    // Z sums the probabilities as they are rounded, so that their errors cancel in the quotient.
    auto softmax = [&](int tile) {
        issue_ahead();
        if (!live) return;
        if (tile >= full) {       // (uniform)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                const int slot0 = tile * kTile + 32 * kb;
                uint32_t word;
                if constexpr (OWN) word = visible_word(anc, w.len, slot0);
                else word = w.n_keys >= slot0 + 32 ? ~0u : (w.n_keys <= slot0 ? 0u : (1u << (w.n_keys - slot0)) - 1u);
                word >>= 4 * hb;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!((word >> (8 * (i >> 2) + (i & 3))) & 1u)) s[kb][i] = -INFINITY;
            }
        }
        float rs4[4];
        auto probabilities = [&] {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    bf16x8 v;
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = (__bf16)fast_exp2(__builtin_fmaf(s[kb][8 * h + e], a.scale_log2, neg));
                    pk[kb][h] = __builtin_bit_cast(u32x4, v);
                    float sum = 0.f;
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum = add_bf16_pair(pk[kb][h][e], sum);
                    rs4[2 * kb + h] = sum;
                }
        };
        probabilities();
        float rs = (rs4[0] + rs4[1]) + (rs4[2] + rs4[3]);
        if (__builtin_amdgcn_ballot_w64(!(rs <= limit)) != 0ull) {       // (uniform; the first tile, rare after it)
            float mx = s[0][0];
#pragma unroll
            for (int i = 1; i < 32; ++i) mx = max_nan(mx, s[i >> 4][i & 15]);
            mx = xor32_max(mx);
            const bool up = !(mx <= mref);
            const float alpha = up && mref != -INFINITY ? fast_exp2((mref - mx) * a.scale_log2) : 1.f;
            mref = up ? mx : mref;
            neg = mref == -INFINITY ? 0.f : -mref * a.scale_log2;
            limit = mref == -INFINITY ? -1.f : 512.f;
            zrun *= alpha;
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[mb][i] *= alpha;
            probabilities();
            rs = (rs4[0] + rs4[1]) + (rs4[2] + rs4[3]);
        }
        zrun += rs;
        asm volatile("" : "+v"(pk[0][0]), "+v"(pk[0][1]), "+v"(pk[1][0]), "+v"(pk[1][1]));     // (the conversions belong to this phase)
        __builtin_amdgcn_sched_barrier(0);
    };

    if (t0 < t1) {
        wait_vmcnt<0>();
        __syncthreads();
        load_k();
        load_v();
        __builtin_amdgcn_sched_barrier(0);
        if (late) {
            issue_ahead();
            boundary(false);
        }
        if (live) matrix_phase(std::true_type{}, t0);
        for (int tile = t0;; ++tile) {
            boundary(late);
            softmax(tile);
            boundary(!late);
            if (live) matrix_phase(std::false_type{}, tile + 1);
            if (tile + 1 == t1) break;
        }
        if (!late) boundary(false);
        wait_vmcnt<0>();        // (the empty loads count too)
    }
    zrun = xor32_add(zrun);

    // ---- partial state of this slice: (reference maximum, Z) per row and the un-normalised accumulator; lane layout of
    //      acc[mb]: row n of the block, columns 32 mb + 8 j + 4 hb + r at vector index 4 j + r
    if (valid) {
        const int64_t pr = (int64_t)(pt.slot0 + w.slice) * a.rows_total + prefix_state_row(a, row);
        if (hb == 0) put_statistics(a, pt, w, prefix_state_row(a, row), mref * a.scale_log2, zrun);
        if (!(zrun == 0.f)) {
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<f32x4*>(a.part_acc + pr * DV + 32 * mb + 8 * j + 4 * hb) =
                        f32x4{acc[mb][4 * j], acc[mb][4 * j + 1], acc[mb][4 * j + 2], acc[mb][4 * j + 3]};
        }
    }
}

// Path of a part: 0 the rows path, 1 and 2 the keys path with 16 and 32 rows.
template <bool BF16, int DK, int DV, int PATH, bool OWN>
__device__ __forceinline__ void prefix_path(const PrefixArgs& a, int wg, char* smem, PrefixTree& tree) {
    if constexpr (PATH == 0) prefix_rows<DK, DV, OWN>(a, wg, smem, tree);
    else prefix_keys<BF16, DK, DV, PATH, OWN>(a, wg, smem, tree);
}

// The prefix's workgroups first (they are the longer ones), then those of the sequences' own keys; within each part every XCD
// gets a contiguous range.
template <bool BF16, int DK, int DV, int PREFIX, int OWN>
__global__ void __launch_bounds__(kPrefixThreads, 1) __attribute__((amdgpu_waves_per_eu(2, 2))) k_prefix(const PrefixArgs a) {
    extern __shared__ __align__(16) char smem[];
    __shared__ PrefixTree tree;
    touch_args<PrefixArgs>();
    const int n0 = a.part[0].n_pad;
    if ((int)blockIdx.x < n0) {
        const int wg = (blockIdx.x & 7) * (n0 >> 3) + (blockIdx.x >> 3);
        if (wg < a.part[0].n_wg) prefix_path<BF16, DK, DV, PREFIX, false>(a, wg, smem, tree);
    } else {
        const int id = blockIdx.x - n0, wg = (id & 7) * (a.part[1].n_pad >> 3) + (id >> 3);
        if (wg < a.part[1].n_wg) prefix_path<BF16, DK, DV, OWN, true>(a, wg, smem, tree);
    }
}

struct PrefixCombineArgs {
    const float *part_stats, *part_acc;
    const int32_t* n_query;
    char* out;
    int T, H, n_slots;
    int64_t rows_total;
    FastDiv div_H, div_T;
    int64_t out_s[3];     // bytes: sequence, node, head
};

// out = sum_s 2^(m_s - M) acc_s / sum_s 2^(m_s - M) Z_s over the slices that saw a key; DV / 4 threads per row.  The small calls
// are bound by latency: a lane of the row's group fetches the statistics of its own slots while (EARLY) the first eight slots' sums
// are on their way, the maximum and the total go through lane exchanges, and every later batch of eight is fetched at once.
// Measured: 3.9 us for 256 rows, 5.5 us for 2048 (22 MB of partial states), 14.5 us for 32768 (70 MB, 4.8 TB/s).
// EARLY: the first eight slots' sums are fetched before it is known which of them count; else (many rows, which hide the second
// round trip) only those that do.
template <bool BF16, int DV, bool EARLY>
__global__ void __launch_bounds__(kThreads) k_prefix_combine(const PrefixCombineArgs a) {
    touch_args<PrefixCombineArgs>();
    constexpr int TPR = DV / 4, RPW = kThreads / TPR, PER = kPrefixMaxSlots / TPR, BATCH = 8;
    const int64_t row = (int64_t)blockIdx.x * RPW + threadIdx.x / TPR;
    if (row >= a.rows_total) return;
    const int l = threadIdx.x % TPR, c = l;
    const int bi = a.div_H.div((int)row), b = a.div_T.div(bi), i = bi - b * a.T, h = (int)row - bi * a.H;
    const int Tq = a.n_query ? a.n_query[b] : a.T;
    float2 st[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        st[k] = make_float2(0.f, 0.f);
        if (l + k * TPR < a.n_slots) st[k] = *reinterpret_cast<const float2*>(a.part_stats + ((int64_t)(l + k * TPR) * a.rows_total + row) * 2);
    }
    const float* at = a.part_acc + row * DV + c * 4;
    const int64_t step = a.rows_total * DV;
    f32x4 v[BATCH];
#pragma unroll
    for (int s = 0; s < BATCH; ++s) v[s] = EARLY ? *reinterpret_cast<const f32x4*>(at + min(s, a.n_slots - 1) * step) : f32x4{0.f, 0.f, 0.f, 0.f};
    float M = -INFINITY, Z = 0.f;
#pragma unroll
    for (int k = 0; k < PER; ++k)
        if (!(st[k].y == 0.f)) M = max_nan(M, st[k].x);
#pragma unroll
    for (int off = 1; off < TPR; off <<= 1) M = max_nan(M, __shfl_xor(M, off, TPR));
    float w[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        w[k] = st[k].y == 0.f ? 0.f : fast_exp2(st[k].x - M);
        Z += w[k] == 0.f ? 0.f : w[k] * st[k].y;
    }
#pragma unroll
    for (int off = 1; off < TPR; off <<= 1) Z += __shfl_xor(Z, off, TPR);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < PER; ++k)
        for (int s0 = k * TPR; s0 < (k + 1) * TPR && s0 < a.n_slots; s0 += BATCH) {
            // slots that saw no key, or that do not exist, hold anything: their weight is 0, and but for an early first batch they are not fetched
            float ws[BATCH];
#pragma unroll
            for (int s = 0; s < BATCH; ++s) {
                ws[s] = __shfl(w[k], s0 - k * TPR + s, TPR);
                if ((s0 || !EARLY) && ws[s] != 0.f) v[s] = *reinterpret_cast<const f32x4*>(at + (s0 + s) * step);
            }
#pragma unroll
            for (int s = 0; s < BATCH; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] += ws[s] == 0.f ? 0.f : ws[s] * v[s][e];
        }
    acc *= 1.f / Z;
    if (i >= Tq) acc = f32x4{0.f, 0.f, 0.f, 0.f};       // (a node that exists sees itself: Z > 0)
    char* o = a.out + b * a.out_s[0] + i * a.out_s[1] + h * a.out_s[2];
    if constexpr (BF16) {
        __bf16 r[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = (__bf16)acc[e];
        *reinterpret_cast<u32x2*>(o + c * 8) = *reinterpret_cast<u32x2*>(r);
    } else {
        *reinterpret_cast<f32x4*>(o + c * 16) = acc;
    }
}

}  // namespace ssv
