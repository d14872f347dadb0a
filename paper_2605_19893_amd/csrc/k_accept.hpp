// What a verification round does with its samples: the walk through the draft tree, and the accepted rows moved to the
// front of the draft slots.
#pragma once
#include "device_common.hpp"

namespace ssv {

struct AcceptArgs {
    const int32_t *draft, *root, *sampled, *seq_lens, *n_query, *parents;
    int32_t *path, *n_accepted, *next, *committed;
    int B, T;
};

// One wavefront per sequence, two nodes per lane.  A step of the walk is a ballot over the nodes that are a child of the
// current one and carry the wanted token; the lowest set bit is the child, and its sample is the next wanted token.  Node
// indices ascend along a path, so the walk ends after at most T steps.  Bound by its launch and three dependent reads: 2.1 us for
// one sequence of 8 nodes, 3.0 us for 256 of 40 (4 KB to 200 KB).
__global__ void __launch_bounds__(kThreads) k_accept(const AcceptArgs a) {
    const int lane = threadIdx.x & 63;
    const int b = blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    if (b >= a.B) return;
    const int Tq = a.n_query ? min(max(a.n_query[b], 0), a.T) : a.T;
    int parent[2], draft[2], says[2], line[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = lane + 64 * k;
        parent[k] = -2;              // a node that does not exist is nobody's child
        draft[k] = says[k] = line[k] = -1;
        if (i < Tq) {
            const int64_t at = (int64_t)b * a.T + i;
            parent[k] = a.parents ? a.parents[at] : i - 1;
            if (parent[k] >= i || parent[k] < -1) parent[k] = -1;
            draft[k] = a.draft[at];
            says[k] = a.sampled[at];
        }
    }
    const int len = a.seq_lens[b];
    int at = -1, want = a.root[b], count = 0;
    while (want >= 0) {
        const uint64_t lo = __builtin_amdgcn_ballot_w64(parent[0] == at && draft[0] == want);
        const uint64_t hi = __builtin_amdgcn_ballot_w64(parent[1] == at && draft[1] == want);
        if (!(lo | hi)) break;
        at = lo ? __builtin_ctzll(lo) : 64 + __builtin_ctzll(hi);
        want = __builtin_amdgcn_readlane(lo ? says[0] : says[1], at & 63);
        if (count < 64) {
            if (lane == count) line[0] = at;
        } else {
            if (lane == count - 64) line[1] = at;
        }
        ++count;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (lane + 64 * k < a.T) a.path[(int64_t)b * a.T + lane + 64 * k] = line[k];
    if (lane == 0) {
        a.n_accepted[b] = count;
        a.next[b] = want;
        a.committed[b] = len + count;
    }
}

struct CommitArgs {
    char *k, *v;
    const int32_t *path, *n_accepted, *seq_lens;
    int B, T, H_kv, cap;
    int k_chunks, chunks;              // 16-byte chunks of a K row, of a K and a V row
    int64_t total;                     // layers x B x H_kv x chunks
    int64_t k_s[4], v_s[4];            // bytes: layer, sequence, KV head, row
};

// One thread per 16-byte column of a (layer, sequence, KV head), which walks the path in order.  Paths ascend, so a row is
// written only after every thread's own column of it has been read, and the rows that later entries read lie behind it: eight rows are
// in flight at a time and no thread waits for another.  Bound by its launch and four dependent reads (length, path, row, and the
// store): 3.5 us for four trees in one layer, 4.8 us for 16 in 32 layers (1.6 MB each way).
__global__ void __launch_bounds__(kThreads) k_commit(const CommitArgs a) {
    const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (at >= a.total) return;
    const int64_t pair = at / a.chunks;
    const int c = (int)(at - pair * a.chunks);
    const int64_t lb = pair / a.H_kv;
    const int g = (int)(pair - lb * a.H_kv), b = (int)(lb % a.B);
    const int64_t layer = lb / a.B;
    const int len = a.seq_lens[b];
    const int32_t* path = a.path + (int64_t)b * a.T;
    const int n = min(a.n_accepted[b], a.T);
    if (len < 0) return;
    const bool is_v = c >= a.k_chunks;
    const int64_t row = is_v ? a.v_s[3] : a.k_s[3];
    char* base = is_v ? a.v + layer * a.v_s[0] + b * a.v_s[1] + g * a.v_s[2] + (int64_t)(c - a.k_chunks) * 16
                      : a.k + layer * a.k_s[0] + b * a.k_s[1] + g * a.k_s[2] + (int64_t)c * 16;
    int before = -1;
    for (int j0 = 0; j0 < n; j0 += 8) {
        u32x4 x[8];
        int from[8];
        bool fine = true;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            from[j] = j0 + j < n ? path[j0 + j] : -1;
            fine = fine && from[j] > before && from[j] < a.T && (int64_t)len + from[j] < a.cap;
            if (!fine) from[j] = -1;
            before = from[j];
            if (fine && from[j] != j0 + j) x[j] = *reinterpret_cast<const u32x4*>(base + ((int64_t)len + from[j]) * row);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (from[j] >= 0 && from[j] != j0 + j) *reinterpret_cast<u32x4*>(base + ((int64_t)len + j0 + j) * row) = x[j];
        if (!fine) break;
    }
}

}  // namespace ssv
