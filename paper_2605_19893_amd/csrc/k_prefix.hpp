// Dense verification attention over a shared prefix and each sequence's own rows.
//
//   out = sum_s p_s v_s,  p = softmax_s(scale q . k_s),  s over the prefix and over the sequence's visible slots
//
// is split over slices of keys; every slice leaves a partial softmax state (m, Z = sum 2^(x - m), sum 2^(x - m) v) per row and
// k_prefix_combine joins them.  The rows that meet a prefix are those of all its sequences, stacked: row r of a (prefix, KV
// head) pair is (sequence, node, head of the group) = (r / (T H_g), r / H_g % T, r % H_g), so a prefix row is read once for
// up to 16 RB rows of the batch.  The rows that meet a sequence's own keys are the same with one sequence.
#pragma once
#include "device_common.hpp"

namespace ssv {

struct PrefixArgs {
    const char *q, *k, *v;             // k, v: the prefixes or the sequences' own caches
    const int32_t *lens;               // rows of each prefix, or committed tokens of each sequence
    const int32_t *n_query, *parents;
    float *part_stats, *part_acc;
    int T, H, H_kv, H_g;
    int per;                           // sequences that share a cache (1: the sequences' own)
    int rows, n_rg;                    // rows per (cache, KV head); groups of 16 RB of them
    int own;                           // 1: own caches: draft rows behind the committed ones, visible by ancestry
    int max_len;
    int n_slices, slot0;               // slices per pair, and the first one's partial-state slot
    int min_steps;                     // key steps a slice holds at least
    int n_wg;                          // workgroups (the grid is padded to a multiple of 8)
    float scale_log2;
    int64_t rows_total;
    FastDiv div_TH, div_Hg;
    int64_t k_s[3], v_s[3];            // bytes: cache, KV head, row
    int64_t q_s[3];                    // bytes: sequence, node, head
};

constexpr int kPrefixStep = 32;        // keys per step of a wavefront
constexpr int kPrefixWaves = kThreads / 64;

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

// One workgroup = 16 RB rows of one (cache, KV head) x one slice of its keys.  Its four wavefronts hold the same rows and take
// the slice's steps of 32 keys in turn, each with a softmax state of its own, merged in LDS at the end: no barrier while keys
// are streamed.  K fragments are loaded as the matrix instruction wants them (lane: one key, 16 bytes); V rows are loaded as
// they lie, a lane holding DV / 16 neighbouring columns of the eight keys whose probabilities it holds after S^T = K Q^T
// (four of each block of 16), and a byte permutation per register turns them into the operand of O^T = V^T P^T: matrix
// instruction j then sums column DV / 16 * m + j of every lane group m.  Nothing passes through LDS on the way.
template <bool BF16, int DK, int DV, int RB>
__global__ void __launch_bounds__(kThreads, RB == 4 ? 1 : 2) k_prefix_stream(const PrefixArgs a) {
    constexpr int ES = BF16 ? 2 : 4;
    constexpr int KC = DK * ES / 64;             // 64-byte chunks of a K row
    constexpr int CW = DV / 16;                  // V columns per lane
    constexpr int VW = CW * ES / 4;              // 32-bit words of them
    constexpr int ACC_PITCH = DV + 4;
    __shared__ AncSet s_anc[kMaxT];
    __shared__ int s_par[kMaxT];
    __shared__ float s_m[kPrefixWaves][16 * RB], s_z[kPrefixWaves][16 * RB];
    __shared__ __align__(16) float s_acc[kPrefixWaves][16][ACC_PITCH];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = lane & 15, G = lane >> 4;
    const int wg = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);   // every XCD gets a contiguous range of work
    if (wg >= a.n_wg) return;
    const int rg = wg % a.n_rg, ps = wg / a.n_rg;                              // neighbours read the same keys
    const int slice = ps % a.n_slices, pair = ps / a.n_slices;
    const int cache = pair / a.H_kv, g = pair - cache * a.H_kv;

    const int len = min(max(a.lens[cache], 0), a.max_len);
    const int Tq0 = a.n_query ? min(max(a.n_query[cache * a.per], 0), a.T) : a.T;     // (own caches: this sequence's)
    const int n_keys = a.own ? len + Tq0 : len;

    // ---- rows
    bool valid[RB];
    int node[RB];
    int64_t grow[RB];
    u32x4 qf[RB][KC];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int r = (rg * RB + rb) * 16 + n;
        const int rc = min(r, a.rows - 1);
        const int bl = a.div_TH.div(rc), in = rc - bl * a.T * a.H_g;
        const int i = a.div_Hg.div(in), h = in - i * a.H_g;
        const int b = cache * a.per + bl;
        const int Tq = a.own ? Tq0 : (a.n_query ? a.n_query[b] : a.T);
        valid[rb] = r < a.rows && i < Tq;
        node[rb] = i;
        grow[rb] = ((int64_t)b * a.T + i) * a.H + g * a.H_g + h;
        const char* qp = a.q + b * a.q_s[0] + i * a.q_s[1] + (g * a.H_g + h) * a.q_s[2] + G * 16;
#pragma unroll
        for (int c = 0; c < KC; ++c) qf[rb][c] = *reinterpret_cast<const u32x4*>(qp + c * 64);
        if (!valid[rb]) {
#pragma unroll
            for (int c = 0; c < KC; ++c) qf[rb][c] = u32x4{0, 0, 0, 0};
        }
    }
    if (a.own) build_ancestors(tid, cache, a.T, Tq0, a.parents, s_par, s_anc);

    // ---- this slice's steps
    const int n_steps = (n_keys + kPrefixStep - 1) / kPrefixStep;
    const int chunk = max((n_steps + a.n_slices - 1) / a.n_slices, a.min_steps);
    const int t0 = slice * chunk, t1 = min(n_steps, t0 + chunk);
    const char* kbase = a.k + cache * a.k_s[0] + g * a.k_s[1] + G * 16;
    const char* vbase = a.v + cache * a.v_s[0] + g * a.v_s[1] + n * (CW * ES);
    const uint32_t krow = (uint32_t)a.k_s[2], vrow = (uint32_t)a.v_s[2];

    u32x4 kf[2][KC];
    uint32_t vf[2][4][VW];
    auto load_k = [&](int t) {
        const char* p = kbase + (int64_t)t * kPrefixStep * a.k_s[2];
        const int last = n_keys - 1 - t * kPrefixStep;       // rows behind the last one repeat it; their scores are masked
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const char* row = p + (uint32_t)min(kb * 16 + n, last) * krow;
#pragma unroll
            for (int c = 0; c < KC; ++c) kf[kb][c] = *reinterpret_cast<const u32x4*>(row + c * 64);
        }
    };
    auto load_v = [&](int t) {
        const char* p = vbase + (int64_t)t * kPrefixStep * a.v_s[2];
        const int last = n_keys - 1 - t * kPrefixStep;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const char* row = p + (uint32_t)min(kb * 16 + 4 * G + r, last) * vrow;
                if constexpr (VW == 4) {
                    const u32x4 x = *reinterpret_cast<const u32x4*>(row);
#pragma unroll
                    for (int w = 0; w < 4; ++w) vf[kb][r][w] = x[w];
                } else {
                    const u32x2 x = *reinterpret_cast<const u32x2*>(row);
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
    const float raise = 8.f / a.scale_log2;      // the reference maximum follows the running one at a distance of up to 2^8
    const int full = a.own ? len : n_keys;       // keys that every row sees

    int t = t0 + wave;
    if (t < t1) {
        load_k(t);
        load_v(t);
    }
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
                uint32_t word;
                if (a.own) {
                    word = visible_word(s_anc[node[rb]], len, t * kPrefixStep);
                } else {
                    word = (1u << (n_keys - t * kPrefixStep)) - 1u;
                }
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
                for (int r = 0; r < 4; ++r) {
                    p[kb][r] = fast_exp2(__builtin_fmaf(s[rb][kb][r], a.scale_log2, neg));
                    z[rb] += p[kb][r];
                }
            if constexpr (BF16) {
                bf16x8 v;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = (__bf16)p[e >> 2][e & 3];
                pk[rb][0] = __builtin_bit_cast(u32x4, v);
            } else {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
                    pk[rb][kb] = u32x4{__float_as_uint(p[kb][0]), __float_as_uint(p[kb][1]), __float_as_uint(p[kb][2]), __float_as_uint(p[kb][3])};
            }
        }
#pragma unroll
        for (int j = 0; j < CW; ++j) {
            if constexpr (BF16) {
                const uint32_t sel = (j & 1) ? 0x07060302u : 0x05040100u;      // the upper or the lower halves of two keys
                const int w = j >> 1;
                const u32x4 vt = {__builtin_amdgcn_perm(vf[0][1][w], vf[0][0][w], sel), __builtin_amdgcn_perm(vf[0][3][w], vf[0][2][w], sel),
                                  __builtin_amdgcn_perm(vf[1][1][w], vf[1][0][w], sel), __builtin_amdgcn_perm(vf[1][3][w], vf[1][2][w], sel)};
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

    // ---- the four wavefronts' states become one
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        z[rb] = xor32_add(xor16_add(z[rb]));
        if (G == 0) {
            s_m[wave][rb * 16 + n] = mref[rb] * a.scale_log2;
            s_z[wave][rb * 16 + n] = z[rb];
        }
    }
    __syncthreads();
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        float M = -INFINITY, Z = 0.f;
#pragma unroll
        for (int w = 0; w < kPrefixWaves; ++w)
            if (!(s_z[w][rb * 16 + n] == 0.f)) M = max_nan(M, s_m[w][rb * 16 + n]);
#pragma unroll
        for (int w = 0; w < kPrefixWaves; ++w)
            if (!(s_z[w][rb * 16 + n] == 0.f)) Z += s_z[w][rb * 16 + n] * fast_exp2(s_m[w][rb * 16 + n] - M);
        const float f = z[rb] == 0.f ? 0.f : fast_exp2(mref[rb] * a.scale_log2 - M);
        const int64_t pr = (int64_t)(a.slot0 + slice) * a.rows_total + grow[rb];
        if (wave == 0 && G == 0 && valid[rb]) *reinterpret_cast<float2*>(a.part_stats + pr * 2) = make_float2(M, Z);
        if (t0 >= t1) continue;                      // (uniform) an empty slice leaves Z = 0 and no sums
        if (rb > 0) __syncthreads();
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < CW; j += 4)
                *reinterpret_cast<f32x4*>(&s_acc[wave][n][CW * (4 * G + r) + j]) =
                    f32x4{acc[rb][j][r] * f, acc[rb][j + 1][r] * f, acc[rb][j + 2][r] * f, acc[rb][j + 3][r] * f};
        __syncthreads();
        for (int e = tid; e < 16 * DV / 4; e += kThreads) {
            const int row = e / (DV / 4), c = e % (DV / 4) * 4;
            f32x4 sum = *reinterpret_cast<const f32x4*>(&s_acc[0][row][c]);
#pragma unroll
            for (int w = 1; w < kPrefixWaves; ++w) sum += *reinterpret_cast<const f32x4*>(&s_acc[w][row][c]);
            const int rr = (rg * RB + rb) * 16 + row;
            if (rr < a.rows) {                       // (rows of nodes that do not exist have places too; nothing reads them)
                const int bl = a.div_TH.div(rr), in = rr - bl * a.T * a.H_g;
                const int i = a.div_Hg.div(in), h = in - i * a.H_g;
                const int64_t gr = ((int64_t)(cache * a.per + bl) * a.T + i) * a.H + g * a.H_g + h;
                *reinterpret_cast<f32x4*>(a.part_acc + ((int64_t)(a.slot0 + slice) * a.rows_total + gr) * DV + c) = sum;
            }
        }
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

// out = sum_s 2^(m_s - M) acc_s / sum_s 2^(m_s - M) Z_s over the slices that saw a key; DV / 4 threads per row.
template <bool BF16, int DV>
__global__ void __launch_bounds__(kThreads) k_prefix_combine(const PrefixCombineArgs a) {
    constexpr int TPR = DV / 4, RPW = kThreads / TPR;
    const int64_t row = (int64_t)blockIdx.x * RPW + threadIdx.x / TPR;
    if (row >= a.rows_total) return;
    const int c = threadIdx.x % TPR;
    const int bi = a.div_H.div((int)row), b = a.div_T.div(bi), i = bi - b * a.T, h = (int)row - bi * a.H;
    const int Tq = a.n_query ? a.n_query[b] : a.T;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (i < Tq) {
        float M = -INFINITY, Z = 0.f;
        for (int s = 0; s < a.n_slots; ++s) {
            const float2 st = *reinterpret_cast<const float2*>(a.part_stats + ((int64_t)s * a.rows_total + row) * 2);
            if (!(st.y == 0.f)) M = max_nan(M, st.x);
        }
        for (int s = 0; s < a.n_slots; ++s) {
            const int64_t pr = (int64_t)s * a.rows_total + row;
            const float2 st = *reinterpret_cast<const float2*>(a.part_stats + pr * 2);
            if (st.y == 0.f) continue;
            const float w = fast_exp2(st.x - M);
            Z += st.y * w;
            acc += w * *reinterpret_cast<const f32x4*>(a.part_acc + pr * DV + c * 4);
        }
        acc *= 1.f / Z;        // (a node sees itself: Z > 0)
    }
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
