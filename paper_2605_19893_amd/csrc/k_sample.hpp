// One token per row of logits from a given random number: temperature, top-k, top-p and min-p as a threshold, then the inverse
// of the cumulative weights in index order.
//
// All three filters keep a head of the order (logit descending, index ascending), so what they keep together is
//   { key > tau } and the first `quota` indices (ascending) of { key == tau },
// key being the logit's bits in an order-preserving integer form.  tau of top-k is a radix selection by counts, tau of top-p
// one by mass; masses are summed as 64-bit fixed point, so the sums do not depend on the order of the atomics.
#pragma once
#include "device_common.hpp"

namespace ssv {

struct SampleArgs {
    const char* logits;
    const float *temperature, *top_p, *min_p, *u;
    const int32_t *top_k, *n_query;
    int32_t* tokens;
    float* probs;
    int T, V;
    int64_t s[2];          // bytes: sequence, node
    double mass_scale;     // fixed-point units of a weight of 1: V times it stays below 2^63
};

constexpr int kSampleThreads = 1024, kSampleWaves = kSampleThreads / 64;
constexpr int kSampleMaxV = 1 << 20;
constexpr int kSampleMaxIters = kSampleMaxV / (8 * kSampleThreads) + 1;     // (an unaligned row starts inside its first chunk)

__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t b = __float_as_uint(x);
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu)); }

// Weight of a logit; 1 at the maximum, whatever that is.
struct SampleWeight {
    double M, inv_t;
    float Mf;
    __device__ __forceinline__ double operator()(float x) const {
        if (x == Mf) return 1.0;
        if (x == -INFINITY) return 0.0;
        return exp(((double)x - M) * inv_t);
    }
};

template <typename V>
__device__ __forceinline__ V wave_sum(V x) {
#pragma unroll
    for (int off = 32; off; off >>= 1) x += __shfl_xor(x, off);
    return x;
}
template <typename V>
__device__ __forceinline__ V wave_incl_scan(V x, int lane) {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const V up = __shfl_up(x, off);
        if (lane >= off) x += up;
    }
    return x;
}

// Over part[0, n) in LDS (entries >= 0), by one whole wavefront: the first positive entry whose inclusive prefix sum exceeds
// target(total), and the sum before it; where none does, the last positive entry, with the total as the sum before it.
template <typename V>
struct Found { int at; V before, total; };
template <typename V, typename Target>
__device__ __forceinline__ Found<V> find_prefix(const V* part, int n, int lane, Target target_of) {
    const int per = (n + 63) / 64, lo = min(n, lane * per), hi = min(n, lo + per);
    V sum = 0;
    int last = -1;
    for (int i = lo; i < hi; ++i) {
        sum += part[i];
        if (part[i] > 0) last = i;
    }
    const V incl = wave_incl_scan(sum, lane);
    Found<V> f;
    f.total = __shfl(incl, 63);
    const V target = target_of(f.total);
    const uint64_t over = __builtin_amdgcn_ballot_w64(incl > target && last >= 0);
    if (over) {
        V run = incl - sum, before = run;
        int at = last;
        for (int i = lo; i < hi; ++i) {
            if (!(part[i] > 0)) continue;
            before = run;
            run += part[i];
            at = i;
            if (run > target) break;
        }
        const int who = __builtin_ctzll(over);
        f.at = __shfl(at, who);
        f.before = __shfl(before, who);
    } else {
#pragma unroll
        for (int off = 32; off; off >>= 1) last = max(last, __shfl_xor(last, off));
        f.at = max(last, 0);
        f.before = f.total;
    }
    return f;
}

template <bool BF16>
__global__ void __launch_bounds__(kSampleThreads) k_sample(const SampleArgs a) {
    constexpr int ES = BF16 ? 2 : 4;
    __shared__ float s_f[kSampleWaves];
    __shared__ int s_i[kSampleWaves];
    __shared__ unsigned long long s_hist[256];
    __shared__ double s_sum[kSampleMaxIters * kSampleWaves];
    __shared__ uint32_t s_cnt[kSampleMaxIters * kSampleWaves];
    __shared__ uint32_t s_digit;
    __shared__ unsigned long long s_above;

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row = blockIdx.x, b = row / a.T, i = row - b * a.T;
    if (a.n_query && i >= a.n_query[b]) {
        if (tid == 0) {
            a.tokens[row] = -1;
            if (a.probs) a.probs[row] = 0.f;
        }
        return;
    }
    const char* base = a.logits + b * a.s[0] + i * a.s[1];
    const int shift = (int)((uintptr_t)base & 15) / ES;        // elements of the first chunk that lie before the row
    const int n_chunks = (a.V + shift + 7) / 8, iters = (n_chunks + kSampleThreads - 1) / kSampleThreads;

    // chunk c: elements 8 c - shift .. + 7; elements outside the row read as -inf, NaN counts as -inf, -0 as 0
    auto load8 = [&](int c, float (&x)[8]) {
        const int e0 = 8 * c - shift;
        if (e0 >= 0 && e0 + 8 <= a.V) {
            const u32x4* p = reinterpret_cast<const u32x4*>(base + (int64_t)e0 * ES);
            if constexpr (BF16) {
                const u32x4 v = *p;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[2 * j] = __uint_as_float(v[j] << 16);
                    x[2 * j + 1] = __uint_as_float(v[j] & 0xffff0000u);
                }
            } else {
                const u32x4 v = p[0], w = p[1];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[j] = __uint_as_float(v[j]);
                    x[4 + j] = __uint_as_float(w[j]);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[j] = -INFINITY;
                if (c < n_chunks && e0 + j >= 0 && e0 + j < a.V) {
                    if constexpr (BF16) x[j] = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(base)[e0 + j] << 16);
                    else x[j] = reinterpret_cast<const float*>(base)[e0 + j];
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = x[j] != x[j] ? -INFINITY : x[j] + 0.f;
    };
    auto each = [&](auto&& body) {       // body(iteration, first element of the chunk, its eight values)
        for (int it = 0; it < iters; ++it) {
            const int c = it * kSampleThreads + tid;
            float x[8];
            load8(c, x);
            body(it, 8 * c - shift, x);
        }
    };

    // ---- the maximum
    float mx = -INFINITY;
    each([&](int, int, const float (&x)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) mx = fmaxf(mx, x[j]);
    });
#pragma unroll
    for (int off = 32; off; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off));
    if (lane == 0) s_f[wave] = mx;
    __syncthreads();
    mx = s_f[0];
#pragma unroll
    for (int w = 1; w < kSampleWaves; ++w) mx = fmaxf(mx, s_f[w]);
    if (mx == -INFINITY) {
        if (tid == 0) {
            a.tokens[row] = -1;
            if (a.probs) a.probs[row] = 0.f;
        }
        return;
    }
    const float t = a.temperature ? a.temperature[b] : 1.f;
    const bool greedy = !(t > 0.f);
    const SampleWeight weight{(double)mx, greedy ? 1.0 : 1.0 / (double)t, mx};
    int top_k = a.top_k ? a.top_k[b] : 0;
    float top_p = a.top_p ? a.top_p[b] : 1.f;
    const float min_p = a.min_p ? a.min_p[b] : 0.f;
    if (greedy || top_p <= 0.f) top_k = 1;
    if (top_k <= 0 || top_k > a.V) top_k = a.V;
    const bool by_k = top_k < a.V, by_p = top_k > 1 && top_p > 0.f && top_p < 1.f;

    uint32_t tau = 0, quota = 0xffffffffu;
    // ---- radix selection, eight bits at a time: the digit in which the sum from the top reaches `target`
    auto pick_digit = [&](double target, unsigned long long above) {      // s_hist -> s_digit, s_above
        __syncthreads();
        if (wave == 0) {
            unsigned long long h[4], sum = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                h[j] = s_hist[255 - (4 * lane + j)];
                sum += h[j];
            }
            const unsigned long long incl = wave_incl_scan(sum, lane) + above;
            const uint64_t reached = __builtin_amdgcn_ballot_w64((double)incl >= target && sum > 0);
            // rounding of the target can leave nothing that reaches it: then the lowest digit that holds something
            const uint64_t any = __builtin_amdgcn_ballot_w64(sum > 0);
            const int who = reached ? __builtin_ctzll(reached) : 63 - __builtin_clzll(any | 1ull);
            if (lane == who) {
                unsigned long long run = incl - sum;
                int d = 0, held = 0;
                unsigned long long before = run;
                for (; d < 4; ++d) {
                    if (h[d] == 0) continue;
                    before = run;
                    held = d;
                    run += h[d];
                    if ((double)run >= target) break;
                }
                s_digit = 255 - (4 * lane + held);
                s_above = before;
            }
        }
        __syncthreads();
    };
    if (by_k) {
        unsigned long long above = 0;
        uint32_t prefix = 0;
        for (int sh = 24; sh >= 0; sh -= 8) {
            if (tid < 256) s_hist[tid] = 0;
            __syncthreads();
            each([&](int, int e0, const float (&x)[8]) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t k = order_key(x[j]);
                    const bool in = e0 + j >= 0 && e0 + j < a.V && (sh == 24 || (k >> (sh + 8)) == prefix);
                    if (in) atomicAdd(&s_hist[(k >> sh) & 255], 1ull);
                }
            });
            pick_digit((double)top_k, above);
            prefix = (prefix << 8) | s_digit;
            above = s_above;
        }
        tau = prefix;
        quota = (uint32_t)(top_k - (int)above);
    }
    if (by_p) {
        const uint32_t tau_k = tau, quota_k = quota;
        auto mass = [&](uint32_t k) { return (unsigned long long)(weight(key_value(k)) * a.mass_scale + 0.5); };
        unsigned long long above = 0;
        uint32_t prefix = 0;
        double target = 0.0;
        for (int sh = 24; sh >= 0; sh -= 8) {
            if (tid < 256) s_hist[tid] = 0;
            __syncthreads();
            each([&](int, int e0, const float (&x)[8]) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t k = order_key(x[j]);
                    if (k < tau_k || (by_k && k == tau_k) || x[j] == -INFINITY || (sh != 24 && (k >> (sh + 8)) != prefix)) continue;
                    const unsigned long long m = mass(k);
                    if (m) atomicAdd(&s_hist[(k >> sh) & 255], m);
                }
            });
            if (by_k && tid == 0 && (sh == 24 || (tau_k >> (sh + 8)) == prefix)) atomicAdd(&s_hist[(tau_k >> sh) & 255], quota_k * mass(tau_k));
            if (sh == 24) {
                __syncthreads();
                unsigned long long h = 0;
                for (int d = lane; d < 256; d += 64) h += s_hist[d];
                target = (double)top_p * (double)wave_sum(h);
            }
            pick_digit(target, above);
            prefix = (prefix << 8) | s_digit;
            above = s_above;
            __syncthreads();
        }
        const unsigned long long each_m = mass(prefix);
        const uint32_t ties = (by_k && prefix == tau_k) ? quota_k : 0xffffffffu;
        double m = ceil((target - (double)above) / (double)each_m);
        m = fmin(fmax(m, 1.0), (double)ties);
        tau = prefix;
        quota = (uint32_t)m;
    }
    if (min_p >= 1.f) {
        if (tau != order_key(mx)) quota = 0xffffffffu;
        tau = order_key(mx);
    } else if (min_p > 0.f && !(weight(key_value(tau)) >= (double)min_p)) {     // (tau = 0, no threshold yet, reads as NaN)
        // the lowest key of weight min_p or more: within a few units of the key of M + t ln(min_p)
        const float near = (float)((double)mx + log((double)min_p) * (double)t);
        const uint32_t k0 = order_key(near);
        const uint32_t k = k0 + (uint32_t)lane - 32u;
        const uint64_t reach = __builtin_amdgcn_ballot_w64(weight(key_value(k)) >= (double)min_p);
        tau = reach ? k0 + (uint32_t)__builtin_ctzll(reach) - 32u : order_key(mx);
        quota = 0xffffffffu;
    }

    // ---- ties at the threshold: the last index that is kept
    int cut = a.V;
    const int n_parts = iters * kSampleWaves;
    if (quota != 0xffffffffu) {
        each([&](int it, int, const float (&x)[8]) {
            int c = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) c += order_key(x[j]) == tau ? 1 : 0;
            c = wave_sum(c);
            if (lane == 0) s_cnt[it * kSampleWaves + wave] = (uint32_t)c;
        });
        __syncthreads();
        const Found<uint32_t> f = find_prefix(s_cnt, n_parts, lane, [&](uint32_t) { return quota - 1; });
        if (f.total > quota) {
            float x[8];
            const int c = f.at * 64 + lane;
            load8(c, x);
            uint32_t mine = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) mine += order_key(x[j]) == tau ? 1u : 0u;
            uint32_t run = f.before + wave_incl_scan(mine, lane) - mine;
            int found = -1;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (order_key(x[j]) == tau && ++run == quota) found = 8 * c - shift + j;
            }
            const uint64_t who = __builtin_amdgcn_ballot_w64(found >= 0);
            cut = __shfl(found, (int)__builtin_ctzll(who));
        }
    }
    auto kept = [&](float x, int e) {
        const uint32_t k = order_key(x);
        return k > tau || (k == tau && e <= cut);
    };

    // ---- sums of the kept weights by blocks of 512 consecutive elements, then the block, lane and element of u
    each([&](int it, int e0, const float (&x)[8]) {
        double sum = 0.0;
        bool any = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) any = any || kept(x[j], e0 + j);
        if (__builtin_amdgcn_ballot_w64(any)) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (kept(x[j], e0 + j)) sum += weight(x[j]);
            sum = wave_sum(sum);
        }
        if (lane == 0) s_sum[it * kSampleWaves + wave] = sum;
    });
    __syncthreads();
    if (wave != 0) return;
    float u = a.u[row];
    u = u >= 0.f ? fminf(u, 1.f) : 0.f;
    const Found<double> f = find_prefix(s_sum, n_parts, lane, [&](double total) { return (double)u * total; });
    const double target = (double)u * f.total;
    const int c = f.at * 64 + lane;
    float x[8];
    load8(c, x);
    double w[8], sum = 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        w[j] = kept(x[j], 8 * c - shift + j) ? weight(x[j]) : 0.0;
        sum += w[j];
    }
    double run = f.before + wave_incl_scan(sum, lane) - sum;
    const bool past = f.before >= f.total;          // nothing exceeds the target: the last positive weight
    int found = -1, last = -1;
    double wf = 0.0, wl = 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        run += w[j];
        if (w[j] > 0.0) {
            last = 8 * c - shift + j;
            wl = w[j];
            if (found < 0 && run > target) {
                found = last;
                wf = w[j];
            }
        }
    }
    const uint64_t hit = past ? 0ull : __builtin_amdgcn_ballot_w64(found >= 0);
    const uint64_t pos = __builtin_amdgcn_ballot_w64(last >= 0);
    const int who = hit ? (int)__builtin_ctzll(hit) : 63 - (int)__builtin_clzll(pos);
    if (lane == who) {
        a.tokens[row] = hit ? found : last;
        if (a.probs) a.probs[row] = (float)((hit ? wf : wl) / f.total);
    }
}

}  // namespace ssv
