// One token per row of logits from a given random number: temperature, top-k, top-p and min-p as a threshold, then the inverse
// of the cumulative weights in index order.
//
// All three filters keep a head of the order (logit descending, index ascending), so what they keep together is
//   { key > tau } and, of { key == tau }, the indices up to `cut`,
// key being the logit's bits in an order-preserving integer form.
//
// Two launches.  k_sample_blocks reads the logits once, 2048 per wavefront over the whole chip, and leaves per block of 2048 the
// maximum and (where the whole vocabulary counts) the sum of weights against it, and per chunk of 8 the upper half of the
// maximum's key.  k_sample_pick, one workgroup per row, finds the token from these: without filters by the block in which the
// running sum passes u, of which alone the logits are read again; with filters from a list of candidates in LDS, the logits above
// a bound that no kept entry can lie below (from histograms of the chunks' maxima), and only the histogram bin in which the
// threshold falls is ordered.  Rows with more candidates than the list holds take the general way, radix selections that read the row again for
// every digit: rows whose filters keep more than that, rows with more in the threshold's bin than is sorted, and rows whose top-k
// is above the number of chunks that hold a finite logit (every logit is a candidate there: 1000 of 6000, say).
//
// Measured (kernels alone, MI355X; blocks + pick): 512 rows of 100003 fp32 logits without filters 51 + 8.8 us, 4.0 TB/s where
// 5.1 is a copy's: fifteen 64-bit instructions per logit take more than half as long as the bytes, and the pick holds its eight logits per
// thread in scratch memory (8.4 MB written); 128 rows of 131071 bf16 logits with
// mixed settings 13 + 20 us, the second for the rows that keep about a thousand (3.5 us the bound, 2.2 the chunks, 3.5 their
// logits, 7 the thresholds: some fifteen barriers, LDS round trips and code that runs once); 8 rows of 32000 4.5 + 8 us, all of it latency.
#pragma once
#include <type_traits>

#include "device_common.hpp"
#include "wave_ops.hpp"

namespace ssv {

struct SampleBlock { double sum, max; };     // of 2048 logits: sum of 2^((x - max) c), c = log2(e) / t; maximum

struct SampleArgs {
    const char* logits;
    const float *temperature, *top_p, *min_p, *u;
    const int32_t *top_k, *n_query;
    int32_t* tokens;
    float* probs;
    SampleBlock* blocks;   // [row][n_blocks]
    uint16_t* maxima;      // [row][n_blocks * 256]: upper half of the order key of each chunk's maximum
    int T, V, n_blocks;
    int wg_per_row;        // k_sample_blocks
    FastDiv div_wg, div_T;
    int64_t s[2];          // bytes: sequence, node
};

constexpr int kSampleThreads = 512, kSampleWaves = kSampleThreads / 64;     // of k_sample_pick
constexpr int kSampleMaxV = 1 << 20;
constexpr int kSampleBlock = 2048, kSampleChunks = kSampleBlock / 8;
constexpr int kSampleMaxBlocks = kSampleMaxV / kSampleBlock + 1;            // (an unaligned row starts inside its first chunk)
constexpr int kSampleMaxIters = kSampleMaxV / (8 * kSampleThreads) + 1;
constexpr int kSampleList = 4096;                                           // candidates that k_sample_pick holds ...
constexpr int kSampleSort = 2048;                                           // ... and sorts, of one bin
constexpr int kSampleBins = 256;
static_assert(kSampleThreads >= kSampleChunks && kSampleThreads >= kSampleBins, "a thread per chunk of a block, and per bin");

__host__ __device__ __forceinline__ int sample_blocks(int V) { return (V + 7 + kSampleBlock - 1) / kSampleBlock; }

__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t b = __float_as_uint(x);
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu)); }

// 2^f, f in [-1/2, 1/2]: the polynomial of degree 10 that takes the values of 2^f at the eleven Chebyshev points, off by at most 4e-16.
__device__ __forceinline__ double exp2_near_0(double f) {
    double p = 7.072585949269223e-09;
    p = __builtin_fma(p, f, 1.0208690299958306e-07);
    p = __builtin_fma(p, f, 1.321544258792169e-06);
    p = __builtin_fma(p, f, 1.5252657260200837e-05);
    p = __builtin_fma(p, f, 0.0001540353044173605);
    p = __builtin_fma(p, f, 0.0013333558230164974);
    p = __builtin_fma(p, f, 0.009618129107606888);
    p = __builtin_fma(p, f, 0.05550410866444772);
    p = __builtin_fma(p, f, 0.24022650695910097);
    p = __builtin_fma(p, f, 0.69314718055995);
    return __builtin_fma(p, f, 1.0);
}

// 2^y for y <= 0 (lower than -1100, -inf and NaN count as -1100, which gives 0).  Eighteen instructions at the rate of 32-bit ones.
__device__ __forceinline__ double exp2_64(double y) {
    y = fmax(y, -1100.0);
    const double n = __builtin_rint(y);
    return __builtin_ldexp(exp2_near_0(y - n), (int)n);
}

// 2^(d c) for d c in [-1000, 0], 1 for d = 0, for sums over blocks, without slow conversions: adding 1.5 * 2^52 rounds to a whole
// number and leaves it in the low bits, from where it goes into the exponent.
__device__ __forceinline__ double exp2_64_short(double d, double c) {
    constexpr double MAGIC = 6755399441055744.0;
    const double t = __builtin_fma(d, c, MAGIC);
    const uint64_t bits = __builtin_bit_cast(uint64_t, exp2_near_0(__builtin_fma(d, c, MAGIC - t)));
    const uint32_t n = (uint32_t)__builtin_bit_cast(uint64_t, t);
    return __builtin_bit_cast(double, (uint64_t)((uint32_t)(bits >> 32) + (n << 20)) << 32 | (uint32_t)bits);
}

// Weight of a logit against a maximum; 1 at the maximum, whatever that is.
struct SampleWeight {
    double M, c;       // c = log2(e) / temperature
    float Mf;
    __device__ __forceinline__ double operator()(float x) const { return exp2_64(x == Mf ? 0.0 : ((double)x - M) * c); }
};

// The settings of a sequence as the header reads them.
struct SampleRule {
    float t, top_p, min_p;
    int top_k;
    double c;
    bool first;            // the first entry alone
    bool by_k, by_p, by_m;
    __device__ __forceinline__ bool sums() const { return !first && (by_p ? !by_k : !(by_k || by_m)); }      // the whole vocabulary's sum counts
    __device__ __forceinline__ bool filters() const { return !first && (by_k || by_p || by_m); }
};
__device__ __forceinline__ SampleRule sample_rule(const SampleArgs& a, int b) {
    SampleRule r;
    r.t = a.temperature ? a.temperature[b] : 1.f;
    r.top_k = a.top_k ? a.top_k[b] : 0;
    r.top_p = a.top_p ? a.top_p[b] : 1.f;
    r.min_p = a.min_p ? a.min_p[b] : 0.f;
    r.first = !(r.t > 0.f) || r.top_p <= 0.f || r.top_k == 1;
    r.by_k = r.top_k > 0 && r.top_k < a.V;
    r.by_p = r.top_p < 1.f;
    r.by_m = r.min_p > 0.f;
    r.c = fmax(1.4426950408889634 / (double)r.t, 1e-300);      // (infinite temperature: every finite logit weighs the same, -inf nothing)
    return r;
}

// A row of logits in chunks of 8 from a 16-byte boundary on: chunk c holds elements 8 c - shift .. + 7.  Elements outside the
// row read as -inf, NaN counts as -inf, -0 as 0.  A chunk comes in two steps, so that several fetches are in flight before the
// first is looked at: every chunk that lies in the row as a whole is fetched without a condition, the first and the last one are
// read by elements where they do not.
template <bool BF16>
struct SampleRow {
    static constexpr int ES = BF16 ? 2 : 4;
    struct Raw { u32x4 v[BF16 ? 1 : 2]; };
    const char* base;
    int V, shift, n_chunks;
    int lo, hi;            // chunks that lie in the row as a whole: [lo, hi)
    __device__ __forceinline__ SampleRow(const SampleArgs& a, int b, int i) : base(a.logits + b * a.s[0] + i * a.s[1]), V(a.V) {
        shift = (int)((uintptr_t)base & 15) / ES;
        n_chunks = (V + shift + 7) / 8;
        lo = shift ? 1 : 0;
        hi = (V + shift) / 8;
    }
    __device__ __forceinline__ int first(int c) const { return 8 * c - shift; }
    __device__ __forceinline__ static float clean(float x) { return fmaxf(x + 0.f, -INFINITY); }
    __device__ __forceinline__ Raw fetch(int c) const {
        Raw r{};
        if (lo < hi) {     // (uniform)
            const u32x4* p = reinterpret_cast<const u32x4*>(base + (int64_t)first(min(max(c, lo), hi - 1)) * ES);
#pragma unroll
            for (int k = 0; k < (BF16 ? 1 : 2); ++k) r.v[k] = p[k];
        }
        return r;
    }
    // The chunks at the ends of the row and beyond, by elements (in a loop of its own: the code is fetched more often than it runs).
    __device__ __forceinline__ void ends(int c, Raw& r) const {
        if (c >= lo && c < hi) return;
        uint32_t w[8 * ES / 4];
#pragma unroll
        for (int k = 0; k < 8 * ES / 4; ++k) w[k] = 0;
#pragma unroll 1
        for (int j = 0; j < 8; ++j) {
            const int e = first(c) + j;
            const bool in = e >= 0 && e < V;
#pragma unroll
            for (int k = 0; k + 1 < 8 * ES / 4; ++k) w[k] = BF16 ? __builtin_amdgcn_alignbit(w[k + 1], w[k], 16) : w[k + 1];
            uint32_t& last = w[8 * ES / 4 - 1];
            if constexpr (BF16) last = last >> 16 | (uint32_t)(in ? reinterpret_cast<const uint16_t*>(base)[e] : 0xff80u) << 16;
            else last = in ? reinterpret_cast<const uint32_t*>(base)[e] : 0xff800000u;
        }
#pragma unroll
        for (int k = 0; k < 8 * ES / 4; ++k) r.v[k >> 2][k & 3] = w[k];
    }
    template <bool CLEAN = true>
    __device__ __forceinline__ void unpack(const Raw& r, float (&x)[8]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (BF16) x[j] = __uint_as_float(j & 1 ? r.v[0][j >> 1] & 0xffff0000u : r.v[0][j >> 1] << 16);
            else x[j] = __uint_as_float(r.v[j >> 2][j & 3]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = CLEAN ? clean(x[j]) : x[j] + 0.f;      // (either way no signalling NaN)
    }
    __device__ __forceinline__ void load(int c, float (&x)[8]) const {
        Raw r = fetch(c);
        ends(c, r);
        unpack(r, x);
    }
    template <bool CLEAN = true, int N>
    __device__ __forceinline__ void load_each(int c, int step, float (&x)[N][8]) const {      // chunks c, c + step, ...
        Raw r[N];
#pragma unroll
        for (int k = 0; k < N; ++k) r[k] = fetch(c + k * step);
        if (__builtin_amdgcn_ballot_w64(c < lo || c + (N - 1) * step >= hi)) {
#pragma unroll
            for (int k = 0; k < N; ++k) ends(c + k * step, r[k]);
        }
#pragma unroll
        for (int k = 0; k < N; ++k) unpack<CLEAN>(r[k], x[k]);
    }
};

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
    const V incl = wave_incl_scan(sum);
    Found<V> f;
    f.total = last_lane(incl);
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
        f.at = max(wave_max(last), 0);
        f.before = f.total;
    }
    return f;
}

// One wavefront per block of 2048 logits, four blocks per workgroup.  Seven wavefronts to a SIMD (72 registers) hide the reads behind the
// exponentials: 512 rows of 100003 fp32 logits take 51 us; 53.3 with three, 35.5 without the exponentials, 40 a copy's time.
template <bool BF16>
__global__ void __launch_bounds__(kThreads, 7) k_sample_blocks(const SampleArgs a) {
    touch_args<SampleArgs>();
    const int lane = threadIdx.x & 63;
    const int row = a.div_wg.div((int)blockIdx.x);
    const int blk = ((int)blockIdx.x - row * a.wg_per_row) * (kThreads / 64) + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int b = a.div_T.div(row), i = row - b * a.T;
    if (blk >= a.n_blocks || (a.n_query && i >= a.n_query[b])) return;
    const SampleRow<BF16> logits(a, b, i);
    float x[4][8];
    logits.template load_each<false>(blk * kSampleChunks + lane, 64, x);       // (a maximum passes over NaN)
    const SampleRule rule = sample_rule(a, b);
    float m[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        m[k] = -INFINITY;
#pragma unroll
        for (int j = 0; j < 8; ++j) m[k] = fmaxf(m[k], x[k][j]);
        m[k] += 0.f;
    }
    const float M = wave_max(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])));
    if (rule.filters()) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            a.maxima[(int64_t)row * a.n_blocks * kSampleChunks + blk * kSampleChunks + k * 64 + lane] = (uint16_t)(order_key(m[k]) >> 16);
    }
    double sum = 0.0;
    if (rule.sums() && M != -INFINITY) {
        const double Md = (double)M;
        double part[4] = {0.0, 0.0, 0.0, 0.0};
        if (M == INFINITY) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) part[k] += x[k][j] == M ? 1.0 : 0.0;
        } else {
            // logits below M - 1000 / c, and NaN, count as that: they weigh 2^-1000, and a sum of 1 or more does not notice
            const double low = fmax(-693.1471805599453 * (double)rule.t, -1e303);
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) part[k] += exp2_64_short(fmax((double)x[k][j] - Md, low), rule.c);
        }
        sum = wave_sum((part[0] + part[1]) + (part[2] + part[3]));
    }
    if (lane == 0) a.blocks[(int64_t)row * a.n_blocks + blk] = SampleBlock{sum, (double)M};
}

// Exclusive prefix sums and maxima over the threads of a workgroup, with one barrier each: calls alternate between two arrays, so
// that what a call writes was last read before the barrier of the call in between.  Every thread makes the same calls.
struct SampleBlockOps {
    uint64_t (*part)[kSampleWaves];      // LDS, two of them
    int lane, wave, turn;
    template <typename V>
    __device__ __forceinline__ V scan(V x, V& total) {
        V* p = reinterpret_cast<V*>(part[turn]);
        turn ^= 1;
        const V incl = wave_incl_scan(x);
        if (lane == 63) p[wave] = incl;
        __syncthreads();
        V before = 0;
        total = 0;
#pragma unroll
        for (int w = 0; w < kSampleWaves; ++w) {
            if (w == wave) before = total;
            total += p[w];
        }
        return before + incl - x;
    }
    __device__ __forceinline__ int max(int x) {
        int* p = reinterpret_cast<int*>(part[turn]);
        turn ^= 1;
        x = wave_max(x);
        if (lane == 0) p[wave] = x;
        __syncthreads();
        x = p[0];
#pragma unroll
        for (int w = 1; w < kSampleWaves; ++w) x = p[w] > x ? p[w] : x;
        return x;
    }
};

// body(k, load(k)) for k in [0, n), n <= n_max (n_max uniform, n - 1 >= 0 or nothing), four loads on their way at a time.
template <typename Load, typename Body>
__device__ __forceinline__ void each_of(int n, int n_max, Load load, Body body) {
#pragma unroll 1
    for (int k0 = 0; k0 < n_max; k0 += 4) {
        decltype(load(0)) x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = load(max(0, min(k0 + k, n - 1)));
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k0 + k < n) body(k0 + k, x[k]);
    }
}

__device__ __forceinline__ uint64_t read_lane(uint64_t x, int lane) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane);
}

// The n <= 64 entries of a list in LDS (all different), in descending order over the lanes (0 behind the last one), by one wavefront: an
// entry's place is the number of larger ones.  `sorted` is LDS for 64 entries; wavefronts may share it if they order the same list.
__device__ __forceinline__ uint64_t wave_order(const uint64_t* list, int n, uint64_t* sorted, int lane) {
    const uint64_t x = lane < n ? list[lane] : ~0ull;
    int rank = lane < n ? 0 : lane;
    int j = 0;
    for (; j + 8 <= n; j += 8) {
        uint64_t y[8];                   // (all on their way before the first is looked at)
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = list[j + k];
#pragma unroll
        for (int k = 0; k < 8; ++k) rank += y[k] > x ? 1 : 0;
    }
    for (; j < n; ++j) rank += list[j] > x ? 1 : 0;
    sorted[rank] = lane < n ? x : 0ull;
    __builtin_amdgcn_wave_barrier();
    return sorted[lane];
}

// A list entry: larger is earlier in the order (logit descending, index ascending).
__device__ __forceinline__ uint64_t list_entry(uint32_t key, int e) { return (uint64_t)key << 32 | (0xffffffffu - (uint32_t)e); }
__device__ __forceinline__ float entry_value(uint64_t x) { return key_value((uint32_t)(x >> 32)); }
__device__ __forceinline__ int entry_index(uint64_t x) { return (int)(0xffffffffu - (uint32_t)x); }

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u16x2 halves(uint32_t x) { return __builtin_bit_cast(u16x2, x); }

struct BinFound { int bin, reached; uint32_t before; uint64_t mass; };      // before, mass: of the bins ahead of it

template <bool BF16>
__global__ void __launch_bounds__(kSampleThreads) k_sample_pick(const SampleArgs a) {
    __shared__ __align__(16) char s_mem[kSampleList * 8];
    __shared__ uint64_t s_sorted[kSampleSort];
    __shared__ unsigned long long s_mass[kSampleBins], s_above;
    __shared__ uint64_t s_part[2][kSampleWaves];
    __shared__ uint32_t s_count[kSampleBins], s_digit;
    static_assert(kSampleMaxIters * kSampleWaves * 12 + 256 * 8 <= sizeof(s_mem) && kSampleMaxBlocks * 8 <= sizeof(s_mem), "one array for every way");
    static_assert(sizeof(s_sorted) == kSampleList * 4, "the chunks of the candidates lie where a bin is sorted later");

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    SampleBlockOps block{s_part, lane, wave, 0};
    touch_args<SampleArgs>();
    const int row = blockIdx.x, b = a.div_T.div(row), i = row - b * a.T;
    int32_t* const token = a.tokens + row;
    float* const prob = a.probs ? a.probs + row : nullptr;
    if (a.n_query && i >= a.n_query[b]) {
        if (tid == 0) {
            *token = -1;
            if (prob) *prob = 0.f;
        }
        return;
    }
    const SampleBlock* blocks = a.blocks + (int64_t)row * a.n_blocks;
    const SampleRow<BF16> logits(a, b, i);
    const SampleRule rule = sample_rule(a, b);
    float u = a.u[row];
    u = u >= 0.f ? fminf(u, 1.f) : 0.f;

    // (every wavefront for itself: a barrier takes longer than the blocks of a row)
    float mx = -INFINITY;
    for (int k = lane; k < a.n_blocks; k += 64) mx = fmaxf(mx, (float)blocks[k].max);
    mx = wave_max(mx);
    if (mx == -INFINITY) {
        if (tid == 0) {
            *token = -1;
            if (prob) *prob = 0.f;
        }
        return;
    }
    if (rule.first) {
        if (wave) return;
        int at = -0x7fffffff;      // minus the first block that holds the maximum
        for (int k = lane; k < a.n_blocks; k += 64)
            if ((float)blocks[k].max == mx) at = max(at, -k);
        const int c = -wave_max(at) * kSampleChunks + lane * (kSampleChunks / 64);
        float x[kSampleChunks / 64][8];
        logits.load_each(c, 1, x);
        int e = -0x7fffffff;
#pragma unroll
        for (int k = 8 * (kSampleChunks / 64) - 1; k >= 0; --k)
            if (x[k >> 3][k & 7] == mx) e = -(logits.first(c) + k);
        e = -wave_max(e);
        if (lane == 0) {
            *token = e;
            if (prob) *prob = 1.f;
        }
        return;
    }
    const SampleWeight weight{(double)mx, rule.c, mx};

    // ---- sums of the blocks against the row's maximum
    double* s_sum = reinterpret_cast<double*>(s_mem);
    double total = 0.0;
    if (rule.sums()) {
        for (int k = lane; k < a.n_blocks; k += 64) {
            const SampleBlock x = blocks[k];
            const double v = x.sum == 0.0 ? 0.0 : x.sum * weight((float)x.max);
            s_sum[k] = v;              // (every wavefront writes what it reads below: the same values)
            total += v;
        }
        total = wave_sum(total);
    }
    if (!rule.filters()) {
        __builtin_amdgcn_wave_barrier();
        const Found<double> f = find_prefix(s_sum, a.n_blocks, lane, [&](double all) { return (double)u * all; });
        const double target = (double)u * f.total;
        const bool past = u >= 1.f || f.before >= f.total;      // nothing exceeds the target: the last positive weight
        constexpr int PER = kSampleBlock / kSampleThreads;      // logits of a thread
        static_assert(PER == 4);
        float x[8];
        const int c = f.at * kSampleChunks + tid / 2, e0 = logits.first(c) + PER * (tid & 1);
        logits.load(c, x);
        double w[PER], sum = 0.0, all;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            w[j] = weight(tid & 1 ? x[PER + j] : x[j]);
            sum += w[j];
        }
        double run = f.before + block.scan(sum, all), wf = 0.0;
        int found = -1, last = -1;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            run += w[j];
            if (w[j] > 0.0 && found < 0) {
                wf = w[j];
                last = e0 + j;
                if (!past && run > target) found = last;
            }
        }
        // the first thread with an element beyond the target, or else the last one with a weight
        const int claim = found >= 0 ? 0x40000000 - tid : (last >= 0 ? tid - 0x40000000 : -0x7fffffff);
        if (block.max(claim) != claim || last < 0) return;
        *token = last;
        if (prob) *prob = (float)(wf / f.total);
        return;
    }

    // ---- lo: a value that no kept entry lies below
    const uint16_t* maxima = a.maxima + (int64_t)row * a.n_blocks * kSampleChunks;
    const int n_groups8 = a.n_blocks * (kSampleChunks / 8);
    const int n_it = (n_groups8 + kSampleThreads - 1) / kSampleThreads;
    // A thread has n_it consecutive groups of eight chunks, in order; N groups at a time: body(first chunk, four pairs of halves each).  N
    // is 8, so that the groups of a vocabulary of up to 262144 are fetched at once, or 2 where a thread has no more (up to 65536: a
    // chain of eight over 32000 takes 13.8 us, 14.5 with the code of eight; mixed settings over 131071 33.4 us, 35.0 with that of two).
    auto fetch_max = [&](int it) { return *reinterpret_cast<const u32x4*>(maxima + 8 * min(tid * n_it + it, n_groups8 - 1)); };
    auto each_max = [&](auto&& body) {
        auto run = [&](auto groups) {
            constexpr int N = decltype(groups)::value;
#pragma unroll 1
            for (int it0 = 0; it0 < n_it; it0 += N) {
                u32x4 x[N];
#pragma unroll
                for (int k = 0; k < N; ++k) x[k] = it0 + k < n_it ? fetch_max(it0 + k) : u32x4{0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < N; ++k)
                    if (it0 + k >= n_it || tid * n_it + it0 + k >= n_groups8) x[k] = u32x4{0, 0, 0, 0};
                body(8 * (tid * n_it + it0), x);
            }
        };
        if (n_it <= 2) run(std::integral_constant<int, 2>{});
        else run(std::integral_constant<int, 8>{});
    };
    auto each_half = [&](auto&& body) {      // one by one (where the code's length counts more)
#pragma unroll 1
        for (int it = 0; it < n_it; ++it) {
            u32x4 x = tid * n_it + it < n_groups8 ? fetch_max(it) : u32x4{0, 0, 0, 0};
#pragma unroll 1
            for (int j = 0; j < 8; ++j) {
                body(x[0] & 0xffffu);
                x = u32x4{__builtin_amdgcn_alignbit(x[1], x[0], 16), __builtin_amdgcn_alignbit(x[2], x[1], 16), __builtin_amdgcn_alignbit(x[3], x[2], 16), x[3] >> 16};
            }
        }
    };
    // A weight in fixed point: sums of these do not depend on the order of the atomics.  The unit is the power of two that brings the sum of
    // what is added up to 2^62 .. 2^63, so that V roundings to it are at most V 2^-63 of that sum, however peaked the row is.  (A unit
    // made for V weights of 1 leaves the tail of a peaked row a few bits: of 2^20 entries behind a peak, of which top-p 0.9999999 keeps
    // 214736, it kept 320161.)  Without top-k the sum is the row's, known from its blocks.
    auto mass_scale_of = [](double sum) { return __builtin_ldexp(1.0, 63 - __builtin_amdgcn_frexp_exp(sum)); };      // sum below 2^exp
    double mass_scale = rule.by_p && !rule.by_k ? mass_scale_of(total) : 0.0;
    auto mass = [&](uint32_t k) { return (uint64_t)(weight(key_value(k)) * mass_scale + 0.5); };
    auto clear_bins = [&] {              // (a barrier follows before they are used)
        if (tid < kSampleBins) {
            s_mass[tid] = 0;
            s_count[tid] = 0;
        }
    };
    clear_bins();
    // The first bin up to which the entries number `n` or more, or weigh `m` or more (the last one that holds any, if none does).  By every
    // wavefront for itself.
    auto find_bin = [&](bool by_mass, uint32_t n, double m) {
        constexpr int PER = kSampleBins / 64;
        uint32_t c[PER], cs = 0;
        uint64_t w[PER], ws = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            c[j] = s_count[PER * lane + j];
            w[j] = s_mass[PER * lane + j];
            cs += c[j];
            ws += w[j];
        }
        const uint32_t ci = wave_incl_scan(cs);
        const uint64_t wi = wave_incl_scan(ws);
        const uint64_t reached = __builtin_amdgcn_ballot_w64(cs > 0 && (by_mass ? (double)wi >= m : ci >= n));
        const uint64_t some = __builtin_amdgcn_ballot_w64(cs > 0);
        const int who = reached ? (int)__builtin_ctzll(reached) : 63 - (int)__builtin_clzll(some | 1ull);
        BinFound f{0, 0, 0u, 0ull};      // (of this lane's bins; that of lane `who` counts)
        uint32_t run = ci - cs;
        uint64_t weigh = wi - ws;
        bool done = false;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            if (c[j] == 0 || done) continue;
            f.bin = PER * lane + j;
            f.before = run;
            f.mass = weigh;
            run += c[j];
            weigh += w[j];
            done = by_mass ? (double)weigh >= m : run >= n;
        }
        return BinFound{__builtin_amdgcn_readlane(f.bin, who), reached != 0, (uint32_t)__builtin_amdgcn_readlane((int)f.before, who), read_lane(f.mass, who)};
    };
    uint32_t tau_m = 0;                      // min-p's threshold
    if (rule.by_m) {
        if (rule.min_p >= 1.f) {
            tau_m = order_key(mx);
        } else {
            // The lowest key of weight min_p or more, 64 keys looked at at once.  It lies within a few units of the key of M + t ln(min_p), but
            // where M and t ln(min_p) cancel: what is left may be off by thousands of units, and the border is looked for between
            // -inf, which weighs nothing, and the maximum, in six steps at most.
            const uint32_t k0 = order_key((float)((double)mx + log((double)rule.min_p) * (double)rule.t));
            uint64_t reach = __builtin_amdgcn_ballot_w64(weight(key_value(k0 + (uint32_t)lane - 32u)) >= (double)rule.min_p);
            tau_m = k0 + (uint32_t)__builtin_ctzll(reach | 1ull << 63) - 32u;
            if (!reach || (reach & 1u)) {                      // (uniform)
                uint32_t below = order_key(-INFINITY);
                tau_m = order_key(mx);
                while (tau_m - below > 1u) {                   // (each step leaves a 64th of what lies between)
                    const uint32_t step = (tau_m - below + 63u) / 64u, k = min(below + step * (uint32_t)(lane + 1), tau_m);
                    reach = __builtin_amdgcn_ballot_w64(k == tau_m || weight(key_value(k)) >= (double)rule.min_p);
                    const uint32_t first = (uint32_t)__builtin_ctzll(reach);      // (the last lane's key is tau_m)
                    tau_m = min(below + step * (first + 1u), tau_m);
                    below += step * first;
                }
            }
        }
    }
    const uint32_t lowest = order_key(-3.4028235e38f);      // (entries of -inf are never kept)
    const uint32_t top_half = order_key(mx) >> 16;
    // bins of equal width in halves, from the maximum's down over a range: 2^shift halves each; the lowest half of the bins up to f's
    auto bin_shift = [](uint32_t range) { return range < (uint32_t)kSampleBins ? 0 : 32 - __builtin_clz(range) - __builtin_ctz(kSampleBins); };
    auto bin_edge = [&](const BinFound& f, int shift) {
        const uint32_t reach = (uint32_t)(f.bin + 1) << shift;
        return f.reached && reach <= top_half ? top_half + 1 - reach : 0u;
    };
    uint32_t lo = lowest;
    if (rule.by_k) {
        // the k-th largest of the maxima of groups of chunks, four per thread (the lower edge of its bin): as many logits are as large.  With
        // fewer groups the least of the maxima of all chunks, if there are k.
        u16x2 v2[4] = {};
        each_max([&](int, const auto& x) {
#pragma unroll
            for (int k = 0; k < (int)(sizeof(x) / 16); ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) v2[j] = __builtin_elementwise_max(v2[j], halves(x[k][j]));
        });
        uint32_t v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = max((uint32_t)v2[j][0], (uint32_t)v2[j][1]);
        int count = 0, n_held;
        uint32_t least = 0xffffu;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (v[j] >= lowest >> 16) {
                ++count;
                least = min(least, v[j]);
            }
        block.scan(count, n_held);
        const bool by_groups = n_held >= rule.top_k;
        if (!by_groups) {
            count = 0;
            least = 0xffffu;
            each_half([&](uint32_t half) {
                count += half >= lowest >> 16 ? 1 : 0;
                least = half >= lowest >> 16 ? min(least, half) : least;
            });
            block.scan(count, n_held);
        }
        if (n_held >= rule.top_k) {
            uint32_t edge = (uint32_t)(0xffff - block.max((int)(0xffffu - least)));
            if (by_groups) {
                const int shift = bin_shift(top_half - edge);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (v[j] >= edge) atomicAdd(&s_count[(top_half - v[j]) >> shift], 1u);
                __syncthreads();
                edge = max(edge, bin_edge(find_bin(false, (uint32_t)rule.top_k, 0.0), shift));
            }
            lo = edge << 16;
        }
    } else if (rule.by_p) {
        // entries of weight below (1 - p) Z / V hold less than (1 - p) Z together
        const double least = (1.0 - (double)rule.top_p) * (1.0 - 1e-9) * total / (double)a.V;
        // (a logarithm of 24 bits with 1e-5 to spare: least lies between 2^-45 and 1)
        const float log2_least = __builtin_amdgcn_logf((float)least) * 1.00001f - 1e-5f;
        const uint32_t k = order_key(mx == INFINITY ? mx : (float)((double)mx + (double)log2_least * 0.6931471805599453 * (double)rule.t));
        lo = max(lo, k > 2 ? k - 2 : 0);
    }
    if (rule.by_m && !rule.by_p) lo = max(lo, tau_m);
    lo = max(lo, lowest);

    // ---- the candidates, in index order.  First chunks whose maximum (its upper half's upper end) reaches a bound, then their logits.
    uint64_t* s_list = reinterpret_cast<uint64_t*>(s_mem);
    uint32_t* s_chunk = reinterpret_cast<uint32_t*>(s_sorted);
    // how many chunks' halves reach `half`; the chunks to `list` if they fit
    auto list_chunks = [&](uint32_t half, uint32_t* list) {
        const uint32_t less = half - 1;          // (half is 0x80 or more: that of the lowest finite key)
        auto hits_of = [&](const auto& x) {
            uint64_t hits = 0;                   // bit 8 k + j: chunk j of group k
#pragma unroll
            for (int k = 0; k < (int)(sizeof(x) / 16); ++k) {
                uint32_t two = 0;                // bits 0, 2, 4, 6: the lower halves, 16, 18, ..: the upper ones
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const u16x2 over = __builtin_elementwise_sub_sat(halves(x[k][j]), u16x2{(uint16_t)less, (uint16_t)less});
                    two |= __builtin_bit_cast(uint32_t, __builtin_elementwise_min(over, u16x2{1, 1})) << (2 * j);
                }
                hits |= (uint64_t)((two | two >> 15) & 0xffu) << (8 * k);
            }
            return hits;
        };
        int mine = 0, n_hit;
        uint64_t hits;
        each_max([&](int, const auto& x) { mine += __builtin_popcountll(hits = hits_of(x)); });
        int to = block.scan(mine, n_hit);
        clear_bins();
        if (n_hit <= kSampleList) {
            auto put = [&](int c) {
                for (; hits; hits &= hits - 1) list[to++] = (uint32_t)(c + __builtin_ctzll(hits));
            };
            if (n_it <= 8) {
                put(8 * tid * n_it);
            } else {
                each_max([&](int c, const auto& x) {
                    hits = hits_of(x);
                    put(c);
                });
            }
        }
        __syncthreads();
        return n_hit;
    };
    // Of these, by bins of equal width in halves: where the chunks' maxima alone (their lower ends) suffice, nothing beyond that bin is
    // kept.  (By count the bound is as good already, unless the list is too long.)
    uint32_t half = lo >> 16;
    const bool by_mass = rule.by_p && !rule.by_k;
    uint32_t* s_first = by_mass ? reinterpret_cast<uint32_t*>(s_mem) : s_chunk;
    uint16_t* s_half = reinterpret_cast<uint16_t*>(s_mem + kSampleList * 4);
    int n_hit = list_chunks(half, s_first);
    if (by_mass || (rule.by_k && n_hit > kSampleList)) {
        const int shift = bin_shift(top_half - half);
        auto count = [&](uint32_t h) {
            if (h << 16 < lo) return;
            const uint32_t at = (top_half - h) >> shift;
            atomicAdd(&s_count[at], 1u);
            if (by_mass) atomicAdd(&s_mass[at], mass(h << 16));
        };
        const bool fits = n_hit <= kSampleList;
        const int q = (n_hit + kSampleThreads - 1) / kSampleThreads, h0 = min(n_hit, tid * q), h1 = min(n_hit, h0 + q);
        if (fits) {
            each_of(h1 - h0, q, [&](int k) { return maxima[s_first[min(h0 + k, n_hit - 1)]]; },
                    [&](int k, uint16_t h) {
                        s_half[h0 + k] = h;
                        count(h);
                    });
        } else {
            each_half(count);
        }
        __syncthreads();
        half = max(half, bin_edge(find_bin(by_mass, (uint32_t)rule.top_k, (double)rule.top_p * (1.0 + 1e-9) * total * mass_scale), shift));
        lo = max(lo, half << 16);
        if (fits) {
            int mine = 0;
            for (int h = h0; h < h1; ++h) mine += s_half[h] >= half ? 1 : 0;
            int at = block.scan(mine, n_hit);
            clear_bins();
            for (int h = h0; h < h1; ++h)
                if (s_half[h] >= half) s_chunk[at++] = s_first[h];
            __syncthreads();
        } else {
            n_hit = list_chunks(half, s_chunk);
        }
    }
    bool listed = n_hit <= kSampleList;
    int n = 0;
    if (listed) {
        // their logits, a chunk per thread at a time
        typename SampleRow<BF16>::Raw raw = {};
        int c = -1;
        auto fetch = [&](int h) {
            c = h < n_hit ? (int)s_chunk[h] : -1;
            raw = logits.fetch(c);
        };
        fetch(tid);
#pragma unroll 1
        for (int h = tid; h - tid < n_hit; h += kSampleThreads) {
            float x[8];
            const int e0 = logits.first(c);
            uint32_t hits = 0;
            if (c >= 0) {
                logits.ends(c, raw);
                logits.unpack(raw, x);
#pragma unroll
                for (int j = 0; j < 8; ++j) hits |= (order_key(x[j]) >= lo ? 1u : 0u) << j;
            }
            fetch(h + kSampleThreads);
            int all, at = n + block.scan(__builtin_popcount(hits), all);
            n += all;
            if (n > kSampleList) break;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (hits >> j & 1u) s_list[at++] = list_entry(order_key(x[j]), e0 + j);
        }
        listed = n <= kSampleList;
        __syncthreads();
    }

    // ---- bins of equal width from the maximum down to lo, which the candidates reach
    const float width = mx - key_value(lo);
    const float inv = width > 0.f && width < INFINITY ? (float)kSampleBins / width : 0.f;
    auto bin_of = [&](float x) { return x == mx ? 0 : min(kSampleBins - 1, (int)((mx - x) * inv)); };
    if (listed && n <= 64) {
        // ---- one wavefront, an entry per lane, no barriers
        if (wave) return;
        const uint64_t entry = lane < n ? s_list[lane] : 0ull;
        uint64_t last_kept = 0;
        if (rule.by_k || rule.by_p) {
            const uint64_t x = wave_order(s_list, n, s_sorted, lane);
            int kept = rule.by_k ? min(rule.top_k, n) : n;
            if (rule.by_p) {
                const double cum = wave_incl_scan(lane < n ? weight(entry_value(x)) : 0.0);
                const double target = (double)rule.top_p * (rule.by_k ? __shfl(cum, kept - 1) : total);
                kept = min(kept, 1 + __builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < kept && cum < target)));
            }
            last_kept = __shfl(x, kept - 1);
        }
        const double w = lane < n && entry >= last_kept && (uint32_t)(entry >> 32) >= tau_m ? weight(entry_value(entry)) : 0.0;
        const double cum = wave_incl_scan(w), all = last_lane(cum);
        const uint64_t over = u < 1.f ? __builtin_amdgcn_ballot_w64(w > 0.0 && cum > (double)u * all) : 0ull;
        const uint64_t some = __builtin_amdgcn_ballot_w64(w > 0.0);
        if (lane == (over ? __builtin_ctzll(over) : 63 - __builtin_clzll(some | 1ull))) {
            *token = entry_index(entry);
            if (prob) *prob = (float)(w / all);
        }
        return;
    }
    const int q = (n + kSampleThreads - 1) / kSampleThreads, l0 = min(n, tid * q), l1 = min(n, l0 + q);     // this thread's entries
    auto entry = [&](int k) { return s_list[l0 + k]; };
    uint64_t last_kept = 0;             // the last entry that is kept
    if (listed && (rule.by_k || rule.by_p)) {
        if (rule.by_k) mass_scale = 2.0 * mass_scale_of((double)n);      // (n weights of at most 1, sums below 2^64; off by n^2 2^-64 of the kept sum, 1 or more, at most)
        // ---- the exact threshold: a histogram of the list, and the entries of the bin in which it falls in order
        each_of(l1 - l0, q, entry, [&](int, uint64_t x) {
            const int at = bin_of(entry_value(x));
            atomicAdd(&s_count[at], 1u);
            if (rule.by_p) atomicAdd(&s_mass[at], mass((uint32_t)(x >> 32)));
        });
        __syncthreads();
        // The entries of a bin in order, and how many there are: up to 64 (as a rule there are ten to forty) with the lanes of every wavefront, and
        // their running mass; more in LDS.
        uint64_t x = 0, x_run = 0;
        auto order_bin = [&](int bin) {
            uint32_t mine = 0;                   // which of this thread's entries (at most eight)
            each_of(l1 - l0, q, entry, [&](int k, uint64_t x) { mine |= (bin_of(entry_value(x)) == bin ? 1u : 0u) << k; });
            int m, at = block.scan(__builtin_popcount(mine), m);
            if (m > kSampleSort) return m;
            for (; mine; mine &= mine - 1) s_sorted[at++] = s_list[l0 + __builtin_ctz(mine)];
            if (m <= 64) {
                __syncthreads();
                x = wave_order(s_sorted, m, s_sorted + 64, lane);
                x_run = rule.by_p ? wave_incl_scan(lane < m ? mass((uint32_t)(x >> 32)) : 0ull) : 0ull;
                return m;
            }
            int size = 128;
            while (size < m) size *= 2;
            for (int k = m + tid; k < size; k += kSampleThreads) s_sorted[k] = 0ull;
            __syncthreads();
            for (int run = 2; run <= size; run *= 2)
                for (int gap = run / 2; gap; gap /= 2) {
                    for (int k = tid; k < size / 2; k += kSampleThreads) {
                        const int p = (k & ~(gap - 1)) * 2 + (k & (gap - 1));
                        const uint64_t x = s_sorted[p], y = s_sorted[p + gap];
                        if ((x < y) == !(p & run)) {
                            s_sorted[p] = y;
                            s_sorted[p + gap] = x;
                        }
                    }
                    __syncthreads();
                }
            return m;
        };
        auto nth = [&](int m, int n) { return m <= 64 ? read_lane(x, n) : s_sorted[n]; };
        // of the first r of m ordered entries: their mass; how many come before the running mass from `base` reaches the target
        auto sum_of = [&](int k0, int k1) {
            uint64_t sum = 0;
            for (int k = k0; k < k1; ++k) sum += mass((uint32_t)(s_sorted[k] >> 32));
            return sum;
        };
        auto mass_of_first = [&](int m, int r) {
            if (m <= 64) return read_lane(x_run, r - 1);
            const int s = (r + kSampleThreads - 1) / kSampleThreads;
            uint64_t all;
            block.scan(sum_of(min(r, tid * s), min(r, (tid + 1) * s)), all);
            return all;
        };
        auto reach_mass = [&](int m, int r, uint64_t base, double target) {
            if (m <= 64) return (int)__builtin_popcountll(__builtin_amdgcn_ballot_w64(lane < r && (double)(base + x_run) < target));
            const int s = (r + kSampleThreads - 1) / kSampleThreads, k0 = min(r, tid * s), k1 = min(r, k0 + s);
            uint64_t all, run = base + block.scan(sum_of(k0, k1), all);
            int below = 0, n_below;
            for (int k = k0; k < k1; ++k) {
                run += mass((uint32_t)(s_sorted[k] >> 32));
                below += (double)run < target ? 1 : 0;
            }
            block.scan(below, n_below);
            return n_below;
        };
        // by count, then by mass if that ends in another bin, or by mass alone
        double target = (double)rule.top_p * total * mass_scale;
        bool of_mass = !rule.by_k;
#pragma unroll 1
        for (;;) {
            const BinFound f = find_bin(of_mass, (uint32_t)rule.top_k, target);
            const int m = order_bin(f.bin);
            listed = m <= kSampleSort;
            if (!listed) break;
            int r = m;
            if (!of_mass) {
                r = max(1, min(m, rule.top_k - (int)f.before));       // the k-th entry is the r-th of the bin (all, if there are fewer than k)
                last_kept = nth(m, r - 1);
                if (!rule.by_p) break;
                target = (double)rule.top_p * (double)(f.mass + mass_of_first(m, r));
                of_mass = (double)f.mass >= target;
                if (of_mass) continue;
            }
            last_kept = nth(m, max(0, min(reach_mass(m, r, f.mass, target), r - 1)));
            break;
        }
    }
    if (listed) {
        // ---- the kept entries in index order: the one whose running sum passes u
        auto kept_weight = [&](uint64_t x) { return x >= last_kept && (uint32_t)(x >> 32) >= tau_m ? weight(entry_value(x)) : 0.0; };
        double sum = 0.0, all;
        each_of(l1 - l0, q, entry, [&](int, uint64_t x) { sum += kept_weight(x); });
        const double before = block.scan(sum, all);
        const double target = (double)u * all;
        // the first thread that passes the target, or else the last one with a weight
        const bool over = sum > 0.0 && before + sum > target && u < 1.f;
        const int claim = over ? 0x40000000 - tid : (sum > 0.0 ? tid - 0x40000000 : -0x7fffffff);
        if (block.max(claim) != claim || !(sum > 0.0)) return;
        double run = before, wf = 0.0;
        int at = 0;
        for (int l = l0; l < l1; ++l) {
            const double w = kept_weight(s_list[l]);
            if (!(w > 0.0)) continue;
            run += w;
            at = entry_index(s_list[l]);
            wf = w;
            if (over && run > target) break;
        }
        *token = at;
        if (prob) *prob = (float)(wf / all);
        return;
    }

    // ---- the general way: radix selections over the row, re-read for every digit.  tau of top-k is selected by counts, tau of top-p by
    //      mass.
    __syncthreads();
    double* s_sums = reinterpret_cast<double*>(s_mem);
    uint32_t* s_cnt = reinterpret_cast<uint32_t*>(s_mem + kSampleMaxIters * kSampleWaves * 8);
    unsigned long long* s_hist = reinterpret_cast<unsigned long long*>(s_mem + kSampleMaxIters * kSampleWaves * 12);
    const int iters = (logits.n_chunks + kSampleThreads - 1) / kSampleThreads;
    auto each = [&](auto&& body) {       // body(iteration, first element of the chunk, its eight values)
        for (int it = 0; it < iters; it += 4) {
            float x[4][8];
            logits.load_each(it * kSampleThreads + tid, kSampleThreads, x);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (it + k < iters) body(it + k, logits.first((it + k) * kSampleThreads + tid), x[k]);
        }
    };
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
            const unsigned long long incl = wave_incl_scan(sum) + above;
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
    if (rule.by_k) {
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
            pick_digit((double)rule.top_k, above);
            prefix = (prefix << 8) | s_digit;
            above = s_above;
        }
        tau = prefix;
        quota = (uint32_t)(rule.top_k - (int)above);
    }
    if (rule.by_p) {
        const uint32_t tau_k = tau, quota_k = quota;
        if (rule.by_k) {                 // the sum over the first top_k entries, for the unit
            double sum = 0.0, all;
            each([&](int, int, const float (&x)[8]) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (order_key(x[j]) > tau_k) sum += weight(x[j]);
            });
            block.scan(sum, all);
            mass_scale = mass_scale_of(all + (double)quota_k * weight(key_value(tau_k)));
        }
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
                    if (k < tau_k || (rule.by_k && k == tau_k) || x[j] == -INFINITY || (sh != 24 && (k >> (sh + 8)) != prefix)) continue;
                    const unsigned long long m = mass(k);
                    if (m) atomicAdd(&s_hist[(k >> sh) & 255], m);
                }
            });
            if (rule.by_k && tid == 0 && (sh == 24 || (tau_k >> (sh + 8)) == prefix)) atomicAdd(&s_hist[(tau_k >> sh) & 255], quota_k * mass(tau_k));
            if (sh == 24) {
                __syncthreads();
                unsigned long long h = 0;
                for (int d = lane; d < 256; d += 64) h += s_hist[d];
                target = (double)rule.top_p * (double)wave_sum(h);
            }
            pick_digit(target, above);
            prefix = (prefix << 8) | s_digit;
            above = s_above;
            __syncthreads();
        }
        const unsigned long long each_m = mass(prefix);
        const uint32_t ties = (rule.by_k && prefix == tau_k) ? quota_k : 0xffffffffu;
        double m = ceil((target - (double)above) / (double)each_m);
        m = fmin(fmax(m, 1.0), (double)ties);
        tau = prefix;
        quota = (uint32_t)m;
    }
    if (rule.by_m && tau < tau_m) {
        tau = tau_m;
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
            logits.load(c, x);
            uint32_t mine = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) mine += order_key(x[j]) == tau ? 1u : 0u;
            uint32_t run = f.before + wave_incl_scan(mine) - mine;
            int found = -1;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (order_key(x[j]) == tau && ++run == quota) found = 8 * c - logits.shift + j;
            }
            const uint64_t who = __builtin_amdgcn_ballot_w64(found >= 0);
            cut = __shfl(found, (int)__builtin_ctzll(who));
        }
    }
    auto kept = [&](float x, int e) {
        const uint32_t k = order_key(x);
        return k > tau || (k == tau && e <= cut);
    };

    // ---- sums of the kept weights by blocks of 512 consecutive elements, then the block and the element of u
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
        if (lane == 0) s_sums[it * kSampleWaves + wave] = sum;
    });
    __syncthreads();
    const Found<double> f = find_prefix(s_sums, n_parts, lane, [&](double sum) { return (double)u * sum; });
    if (wave) return;
    const double target = (double)u * f.total;
    const int c = f.at * 64 + lane;
    float x[8];
    logits.load(c, x);
    double w[8], sum = 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        w[j] = kept(x[j], 8 * c - logits.shift + j) ? weight(x[j]) : 0.0;
        sum += w[j];
    }
    double run = f.before + wave_incl_scan(sum) - sum;
    const bool past = u >= 1.f || f.before >= f.total;          // nothing exceeds the target: the last positive weight
    int found = -1, last = -1;
    double wf = 0.0, wl = 0.0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        run += w[j];
        if (w[j] > 0.0) {
            last = 8 * c - logits.shift + j;
            wl = w[j];
            if (found < 0 && run > target) {
                found = last;
                wf = w[j];
            }
        }
    }
    const uint64_t hit = past ? 0ull : __builtin_amdgcn_ballot_w64(found >= 0);
    const uint64_t pos = __builtin_amdgcn_ballot_w64(last >= 0);
    const int who = hit ? (int)__builtin_ctzll(hit) : 63 - (int)__builtin_clzll(pos | 1ull);
    if (lane == who) {
        *token = hit ? found : last;
        if (prob) *prob = (float)((hit ? wf : wl) / f.total);
    }
}

}  // namespace ssv
