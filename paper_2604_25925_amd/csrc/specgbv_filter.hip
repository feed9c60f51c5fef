// Truncated distributions and draws from them (specgbv_sample_filtered): one workgroup per row.
//
// With the entries of a row in the order "largest logit first, ties by the lowest index", each of top-k, min-p and top-p keeps the
// front of the order, and the draw looks for the entry at which the running weight passes a goal.  So everything asked for is a place in
// that order, by rank or by running weight, and the row needs no sorting: a histogram says in which bin the place lies, and only that
// bin's entries are put in order.
//
// What bounds it.  One row is a chain of passes and searches in one workgroup, and a workgroup's waits are covered only where two share a
// compute unit.  bfloat16 (k_filter_counts): 256 rows of 128256 entries, tokens, 33.3 us (loads and counts 9, weights of the values that occur 5, places 3,
// indices 4, launch and the spread of the loads over the card the rest; the bytes alone 13.6); 1152 rows of 32000, truncated rows, 56 us (30.5; 76 with one workgroup
// a compute unit); one row of 32000 13.3.  float32 (k_filter): 287 rows of 32003, tokens and rows, 53 us (15.2): a row is read from memory for its
// largest value (7), for the histogram (9, the additions in LDS), for each place that is looked for (4 - 5) and for the output.
//
// Weights decide which entry is drawn, and every entry counts, so they are held to more than float32: the histogram's sums are sums of
// integers, which do not hang on the order of the additions, and running sums are float64 in a fixed order.
#include "specgbv_internal.hpp"

namespace specgbv {
namespace {

constexpr int kFilterThreads = 1024, kFilterWaves = kFilterThreads / 64;
constexpr int kBins = 4096;                   // of the row's histogram: 1/64 of an octave of the weight each, the last one all below 2^-64
constexpr int kList = 1024;                   // entries that are put in order at once; bins of a closer histogram

typedef unsigned long long u64;

// Order of logits as order of integers; both zeros are one value, and what is no number comes last, as -inf does.
__device__ __forceinline__ uint32_t key_of(float z)
{
    const uint32_t b = __float_as_uint(z == z ? z + 0.0f : -INFINITY);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
constexpr uint32_t kNothing = 0x007FFFFFu;    // key of -inf
// The value of a key that bounds others from above: -0 has a key of its own, which no entry has, and equals the 0 above it.
__device__ __forceinline__ float bound_of(uint32_t k) { return value_of(k == 0x7FFFFFFFu ? k - 1 : k); }

// e^x for x <= 1 in float64: 2^n times the Taylor sum of e^r, |r| <= ln(2) / 2, to r^12 / 12!, whose remainder is 2 10^-16 of it.
__device__ __forceinline__ double exp_of(double x)
{
    x = fmax(x, -800.0);                                     // (below 2^-1074: 0)
    const double n = rint(x * 1.44269504088896340736);
    double r = fma(n, -0x1.62e42fefa2000p-1, x);            // ln 2 to 40 bits behind the point, whose products with n are exact, then the rest
    r = fma(n, -0x1.9ef35793c7673p-41, r);
    double s = 1.0 / 479001600.0;
    s = fma(s, r, 1.0 / 39916800.0);
    s = fma(s, r, 1.0 / 3628800.0);
    s = fma(s, r, 1.0 / 362880.0);
    s = fma(s, r, 1.0 / 40320.0);
    s = fma(s, r, 1.0 / 5040.0);
    s = fma(s, r, 1.0 / 720.0);
    s = fma(s, r, 1.0 / 120.0);
    s = fma(s, r, 1.0 / 24.0);
    s = fma(s, r, 1.0 / 6.0);
    s = fma(s, r, 0.5);
    s = fma(s, r, 1.0);
    s = fma(s, r, 1.0);
    return ldexp(s, static_cast<int>(n));
}

// The same with 2^(j / 64), j < 64, at hand: the Taylor sum of what is left, at most ln(2) / 128, to r^5 / 5!, whose remainder is 4 10^-17 of it.
__device__ __forceinline__ double exp_from(const double *of_octave, double x)
{
    x = fmax(x, -800.0);
    const double n = rint(x * 92.33248261689366);
    double r = fma(n, -0x1.62e42fefa0000p-7, x);            // ln(2) / 64 to 42 bits behind the point, whose products with n are exact, then the rest
    r = fma(n, -0x1.cf79abc9e3b3ap-46, r);
    double s = 1.0 / 120.0;
    s = fma(s, r, 1.0 / 24.0);
    s = fma(s, r, 1.0 / 6.0);
    s = fma(s, r, 0.5);
    s = fma(s, r, 1.0);
    s = fma(s, r, 1.0);
    const int k = static_cast<int>(n);
    return ldexp(of_octave[k & 63] * s, k >> 6);
}

// How the entries of a row are weighed and binned.  With y = 64 log2(e) (z - top) / T, a weight is 2^(y / 64) = 2^(-bin / 64) (1 + d), bin the
// nearest integer to -y and |d| < 2^-7.  A bin's sum is 2^(-bin / 64) (n (1 - 2^-7) + sum of (d + 2^-7)), and n and that sum of
// non-negative numbers share one 64-bit integer: the count in the bits from `shift` on, the sum in units of 2^-(bits + 6) below it.  So an
// entry costs one addition in LDS.  V takes c bits, the sum of V numbers below 2^bits takes bits + c, which leaves bits = 64 - 2 c: 34 at
// V = 32003, 28 at 152064 (a weight is then rounded to 2^-35 of itself).
struct RowRule {
    float top;                                // the row's largest logit
    float least;                              // smaller entries do not take part
    double inv_t, per;                        // 1 / T; y per unit of the logit
    int shift, bits;

    __device__ __forceinline__ double weight(float z) const
    {
        if (z == top) return 1.0;
        return exp_of((static_cast<double>(z) - static_cast<double>(top)) * inv_t);
    }
    __device__ __forceinline__ double scaled(float z) const
    {
        return z == top ? 0.0 : fmax((static_cast<double>(z) - static_cast<double>(top)) * per, -static_cast<double>(kBins - 1));
    }
    __device__ __forceinline__ int bin(float z) const { return -static_cast<int>(rint(scaled(z))); }
    // one entry as its bin adds it up: the count of 1 and its part of the sum
    __device__ __forceinline__ u64 packed(float z, int &bin) const
    {
        constexpr double a = 0.69314718055994530942 / 64.0;
        const double y = scaled(z), k = rint(y), f = y - k;
        bin = -static_cast<int>(k);
        double d = a * a * a * a * a / 120.0;                // Taylor sum of 2^(f / 64) - 1; the remainder is below 2^-54
        d = fma(d, f, a * a * a * a / 24.0);
        d = fma(d, f, a * a * a / 6.0);
        d = fma(d, f, a * a / 2.0);
        d = fma(d, f, a);
        d *= f;
        // added to 2^52, the sum leaves its integer in the low bits
        const u64 low = static_cast<u64>(__double_as_longlong(fma(d, ldexp(1.0, bits + 6), 4503599627370496.0 + ldexp(1.0, bits - 1)))) & 0xFFFFFFFFFFFFFull;
        return (1ull << shift) + low;
    }
    __device__ __forceinline__ uint32_t count_of(u64 sums) const { return static_cast<uint32_t>(sums >> shift); }
    // the weight of what `sums` adds up, over 2^(-bin / 64)
    __device__ __forceinline__ double weight_of(u64 sums) const
    {
        return static_cast<double>(sums >> shift) * (1.0 - 0.0078125) + ldexp(static_cast<double>(sums & ((1ull << shift) - 1)), -(bits + 6));
    }
    // 2^(-bin / 64); what the last bin holds weighs nothing.  2^(-8 group / 64) times 2^(-i / 64), so that a thread with bins next to each
    // other forms one exponential.
    static __device__ __forceinline__ double weight_of_group(int group) { return exp_of(group * (-0.69314718055994530942 / 8.0)); }
    static __device__ __forceinline__ double weight_in_group(int i)
    {
        constexpr double step[8] = {1.0, 0.9892280131939755, 0.9785720620877001, 0.9680308967461472, 0.9576032806985737,
                                    0.9472879907934828, 0.93708381705515, 0.9269895625416927};
        return step[i];
    }
    __device__ __forceinline__ double weight_of_bin(int bin) const
    {
        return bin == kBins - 1 ? 0.0 : weight_of_group(bin >> 3) * weight_in_group(bin & 7);
    }
    // The smallest value whose bin is at most `bin`: it lies within a step or two of where its weight says.  By a whole wave.
    __device__ __forceinline__ float least_of(int bin) const
    {
        if (bin >= kBins - 1) return least;
        const uint32_t top_key = key_of(top), low_key = key_of(least);
        const float about = static_cast<float>(static_cast<double>(top) - (bin + 0.5) / per);
        const uint32_t at = key_of(about == about ? about : top), from = max(at, low_key + 31u) - 31u;
        const uint32_t mine = min(from + (threadIdx.x & 63), top_key);
        const u64 passed = __ballot(this->bin(value_of(mine)) <= bin);
        return value_of(min(from + (passed ? __ffsll(static_cast<long long>(passed)) - 1 : 63), top_key));
    }
};

// f(logit, index) for every entry of the row, by all TH threads of the workgroup: whole 16-byte vectors where the row allows, AHEAD of
// them on their way at once.
template <int TH, int AHEAD, typename T, typename F>
__device__ __forceinline__ void for_entries(const T *row, int V, F f)
{
    constexpr int PV = Elem<T>::kPerVec;
    const int tid = threadIdx.x;
    const int head = min(V, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / static_cast<int>(sizeof(T)));
    const int vectors = (V - head) / PV, tail = head + vectors * PV;
    if (tid < head) f(Elem<T>::scalar(row + tid), tid);
    const U4 *vec = reinterpret_cast<const U4 *>(row + head);
    for (int v = tid; v < vectors; v += TH * AHEAD) {
        U4 x[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) x[i] = vec[min(v + i * TH, vectors - 1)];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (v + i * TH >= vectors) break;
            float z[PV];
            Elem<T>::unpack(x[i], z);
#pragma unroll
            for (int j = 0; j < PV; ++j) f(z[j], head + (v + i * TH) * PV + j);
        }
    }
    if (tid < V - tail) f(Elem<T>::scalar(row + tail + tid), tail + tid);
}

struct Found {                                // a place in the order
    uint32_t key;
    int index;
    double weight;                            // of the entries up to and including it
};

struct alignas(16) Listed { u64 order, sums; };       // larger `order` stands in front

struct FilterShared {
    u64 sums[kBins];
    union {
        Listed list[kList];                   // entries in question, as their bin adds them up
        u64 closer[kList];                    // a closer histogram
    };
    double thread_weight[kFilterThreads];     // running sums over the threads of a wave, each with its bins
    uint32_t thread_count[kFilterThreads];
    double wave_weight[kFilterWaves];         // running sums over the waves
    u64 wave_sums[kFilterWaves];
    uint32_t wave_count[kFilterWaves];
    uint32_t n, lo, hi, count0;
    double weight0;
    float from, to;
    int bin;
    Found found;
};

// What is looked for: the first place whose count (0) or weight (1) reaches the goal, or whose weight exceeds it (2).
struct Goal {
    int how;
    double goal;
    __device__ __forceinline__ bool reached(uint32_t count, double weight) const
    {
        return how == 0 ? count >= goal : (how == 1 ? weight >= goal : weight > goal);
    }
};

// The first place of the row that reaches the goal, which the whole row does.
template <int TH, typename T>
__device__ Found find_place(FilterShared &sh, const T *row, int V, const RowRule &rule, Goal goal)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    constexpr int kPer = kBins / TH;
    // One wave goes down from waves' bins to threads' bins to bins, to the first that holds entries and reaches the goal (where rounding
    // leaves none: the last that holds some); the others would only take its issue slots.
    if (wave == 0) {
        auto first = [&](bool holds, uint32_t c, double w) {
            const u64 hit = __ballot(holds && goal.reached(c, w)), some = __ballot(holds);
            return hit ? __ffsll(static_cast<long long>(hit)) - 1 : 63 - __clzll(static_cast<long long>(some | 1));
        };
        const int l = lane & (TH / 64 - 1);
        const double ww = sh.wave_weight[l];
        const uint32_t wc = sh.wave_count[l], wb = l ? sh.wave_count[l - 1] : 0u;
        const int block = first(lane < TH / 64 && wc != wb, wc, ww);
        double w0 = block ? lane_value(ww, block - 1) : 0.0;
        uint32_t c0 = block ? __builtin_amdgcn_readlane(wc, block - 1) : 0u;
        const double tw = sh.thread_weight[block * 64 + lane];
        const uint32_t tc = sh.thread_count[block * 64 + lane], tb = lane ? sh.thread_count[block * 64 + lane - 1] : 0u;
        const int t = first(tc != tb, c0 + tc, w0 + tw);
        if (t) { w0 += lane_value(tw, t - 1); c0 += __builtin_amdgcn_readlane(tc, t - 1); }
        const int b0 = (block * 64 + t) * kPer, b = b0 + (lane & (kPer - 1));
        const u64 sums = lane < kPer ? sh.sums[b] : 0ull;
        const uint32_t c = rule.count_of(sums);
        const double w = c ? rule.weight_of_bin(b) * rule.weight_of(sums) : 0.0;
        const double iw = wave_inclusive_sum(w);
        const uint32_t ic = wave_inclusive_count(c);
        const int i = first(c != 0, c0 + ic, w0 + iw);
        const uint32_t n = __builtin_amdgcn_readlane(c, i);
        if (i) { w0 += lane_value(iw, i - 1); c0 += __builtin_amdgcn_readlane(ic, i) - n; }
        const float from = rule.least_of(b0 + i);
        const float to = b0 + i == 0 ? rule.top : bound_of(key_of(rule.least_of(b0 + i - 1)) - 1);
        if (lane == 0) { sh.bin = b0 + i; sh.n = n; sh.count0 = c0; sh.weight0 = w0; sh.from = from; sh.to = to; }
    }
    __syncthreads();
    const uint32_t count0 = sh.count0;
    const double weight0 = sh.weight0, factor = rule.weight_of_bin(sh.bin);
    uint32_t n = sh.n;
    u64 front = 0;                                          // of the bin's entries in front of those in question
    float from_z = sh.from, to_z = sh.to;                   // the entries in question
    auto inside = [&](float z) { return z >= from_z && z <= to_z; };
    auto weight_at = [&](u64 sums) { return weight0 + factor * rule.weight_of(sums); };
    auto reached = [&](u64 sums) { return goal.reached(count0 + rule.count_of(sums), weight_at(sums)); };

    while (n > kList) {
        // keys of the entries in question, and a closer histogram over them
        __syncthreads();
        if (tid == 0) { sh.lo = 0xFFFFFFFFu; sh.hi = 0; sh.bin = -1; }
        __syncthreads();
        uint32_t least = 0xFFFFFFFFu, most = 0;
        for_entries<TH, 4>(row, V, [&](float z, int) {
            const uint32_t key = key_of(z);
            if (inside(z)) { least = min(least, key); most = max(most, key); }
        });
        atomicMin(&sh.lo, least);
        atomicMax(&sh.hi, most);
        for (int i = tid; i < kList; i += TH) sh.closer[i] = 0;
        __syncthreads();
        const uint32_t from = sh.lo, to = sh.hi;
        if (from == to) { from_z = to_z = value_of(from); break; }                  // ties alone
        int shift = 0;
        while (((to - from) >> shift) >= kList) ++shift;
        for_entries<TH, 1>(row, V, [&](float z, int) {
            const uint32_t key = key_of(z);
            if (inside(z)) {
                int b;
                atomicAdd(&sh.closer[(to - key) >> shift], rule.packed(z, b));
            }
        });
        __syncthreads();
        // running sums
        u64 own[kList / TH], run = 0;
#pragma unroll
        for (int i = 0; i < kList / TH; ++i) own[i] = run += sh.closer[tid * (kList / TH) + i];
        u64 incl = run;
        for (int d = 1; d < 64; d <<= 1) {
            const u64 o = __shfl_up(incl, d, 64);
            if (lane >= d) incl += o;
        }
        if (lane == 63) sh.wave_sums[wave] = incl;
        __syncthreads();
        u64 before = front + incl - run;
        for (int i = 0; i < wave; ++i) before += sh.wave_sums[i];
#pragma unroll
        for (int i = 0; i < kList / TH; ++i) sh.closer[tid * (kList / TH) + i] = before + own[i];
        __syncthreads();
        for (int i = tid; i < kList; i += TH) {
            const u64 before_i = i ? sh.closer[i - 1] : front;
            if (sh.closer[i] != before_i && reached(sh.closer[i]) && (before_i == front || !reached(before_i))) sh.bin = i;
        }
        __syncthreads();
        int b = sh.bin;
        if (b < 0) b = static_cast<int>((to - from) >> shift);                     // (rounding: the last one)
        const u64 upto = sh.closer[b];
        if (b) front = sh.closer[b - 1];
        n = rule.count_of(upto - front);
        const uint32_t top = to - (static_cast<uint32_t>(b) << shift), width = (1u << shift) - 1;
        to_z = bound_of(top); from_z = value_of(top - from >= width ? top - width : from);
    }
    __syncthreads();

    if (n > kList) {                                        // more ties than the list holds: by index, a stretch of the row per wave
        int b;
        const u64 one = rule.packed(to_z, b);
        const double each = factor * rule.weight_of(one), gone = weight_at(front);
        double nth = goal.how == 0 ? goal.goal - (count0 + rule.count_of(front)) : (goal.goal - gone) / each;
        nth = goal.how == 0 ? nth : (goal.how == 1 ? ceil(nth) : floor(nth) + 1.0);
        nth = nth >= 1.0 ? nth : 1.0;
        const uint32_t place = nth < n ? static_cast<uint32_t>(nth) : n;
        const int stretch = (V + TH / 64 - 1) / (TH / 64), from = min(V, wave * stretch), to = min(V, from + stretch);
        uint32_t mine = 0;
        for (int i = from; i < to; i += 64) {
            const bool is = i + lane < to && Elem<T>::scalar(row + min(i + lane, V - 1)) == to_z;
            mine += __popcll(__ballot(is));
        }
        if (lane == 0) sh.wave_sums[wave] = mine;
        __syncthreads();
        uint32_t before = 0;
        for (int i = 0; i < wave; ++i) before += static_cast<uint32_t>(sh.wave_sums[i]);
        if (before < place && place <= before + mine) {     // one wave
            for (int i = from; i < to; i += 64) {
                const bool is = i + lane < to && Elem<T>::scalar(row + min(i + lane, V - 1)) == to_z;
                const u64 all = __ballot(is);
                const uint32_t here = __popcll(all);
                if (place <= before + here) {
                    if (is && before + __popcll(all & ((2ull << lane) - 1)) == place) sh.found = Found{key_of(to_z), i + lane, weight_at(front + place * one)};
                    break;
                }
                before += here;
            }
        }
        __syncthreads();
        return sh.found;
    }

    // the entries in question in order: each thread counts what stands in front of its own
    if (tid == 0) sh.n = 0;
    __syncthreads();
    for_entries<TH, 8>(row, V, [&](float z, int i) {
        if (inside(z)) {
            const uint32_t at = atomicAdd(&sh.n, 1u);
            if (at < kList) sh.list[at].order = static_cast<u64>(key_of(z)) << 32 | ~static_cast<uint32_t>(i);
        }
    });
    __syncthreads();
    for (uint32_t e = tid; e < n; e += TH) {
        int b;
        sh.list[e].sums = rule.packed(value_of(static_cast<uint32_t>(sh.list[e].order >> 32)), b);
    }
    __syncthreads();
    for (uint32_t e = tid; e < n; e += TH) {
        const Listed own = sh.list[e];
        u64 sums = front;
#pragma unroll 4
        for (uint32_t i = 0; i < n; ++i) {
            const Listed x = sh.list[i];
            sums += x.order > own.order ? x.sums : 0ull;
        }
        const u64 incl = sums + own.sums;
        const bool last = rule.count_of(incl - front) == n;                        // (where rounding leaves none)
        if ((reached(incl) || last) && (sums == front || !reached(sums)))
            sh.found = Found{static_cast<uint32_t>(own.order >> 32), static_cast<int>(~static_cast<uint32_t>(own.order)), weight_at(incl)};
    }
    __syncthreads();
    return sh.found;
}

// Parameters of a row.
struct RowAsked {
    float temperature, top_p, min_p;
    int k;                                    // INT32_MAX: no limit

    __device__ __forceinline__ RowAsked(const FilterProblem &p, int r)
    {
        temperature = p.temperature ? p.temperature[r] : 1.0f;
        top_p = p.top_p ? p.top_p[r] : 1.0f;
        min_p = p.min_p && p.min_p[r] > 0.0f ? fminf(p.min_p[r], 1.0f) : 0.0f;          // (what is no number: off)
        const int asked = p.top_k ? p.top_k[r] : 0;
        k = asked > 0 ? asked : INT32_MAX;
        if (!(temperature > 0.0f)) { temperature = 1.0f; k = 1; }
    }
    // 1 / temperature.  min_p = 1 leaves the entries that equal the largest, and of these no temperature changes the weight: a factor that
    // takes every other weight to 0 keeps out those that would round to 1.
    __device__ __forceinline__ double per_temperature() const
    {
        return min_p == 1.0f && temperature < INFINITY ? 1e300 : 1.0 / static_cast<double>(temperature);
    }
};

// A row of any length and type, read from memory in every step.
template <int TH, typename T>
__device__ __forceinline__ void filter_row(const FilterProblem &p, int r, FilterShared &sh)
{
    const int tid = threadIdx.x;
    const T *row = static_cast<const T *>(p.logits) + r * p.row_stride;
    const int V = p.V;
    const RowAsked asked(p, r);
    const float temperature = asked.temperature, top_p = asked.top_p, min_p = asked.min_p;
    const int k = asked.k;

    for (int b = tid; b < kBins; b += TH) sh.sums[b] = 0;
    if (tid == 0) sh.hi = kNothing;
    __syncthreads();
    float highest = -INFINITY;
    for_entries<TH, 8>(row, V, [&](float z, int) { highest = fmaxf(highest, z); });          // (what is no number is passed over)
    uint32_t most = key_of(highest);
    for (int m = 32; m > 0; m >>= 1) most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), m, 64)));
    if ((tid & 63) == 0) atomicMax(&sh.hi, most);
    __syncthreads();
    most = sh.hi;

    uint32_t cut_key = kNothing + 1;                        // what is kept: higher keys, and this one up to an index
    int cut_index = INT32_MAX;
    int token = -1;
    if (most != kNothing) {                                 // uniform
        RowRule rule;
        rule.top = value_of(most);
        rule.inv_t = asked.per_temperature();
        rule.per = rule.inv_t * (64.0 * 1.44269504088896340736);
        const int length = 32 - __clz(V);                   // bits of V
        rule.shift = 64 - length;
        rule.bits = min(44, 64 - 2 * length);
        rule.least = -3.402823466e38f;
        if (min_p > 0.0f) {
            // the lowest key whose weight is at least min_p, among the keys around top + temperature ln min_p
            const float about = static_cast<float>(static_cast<double>(rule.top) + static_cast<double>(temperature) * log(static_cast<double>(min_p)));
            const uint32_t centre = max(key_of(about), kNothing + 32u);
            const uint32_t mine = min(centre - 31u + (tid & 63), most);
            const u64 passed = __ballot(rule.weight(value_of(mine)) >= static_cast<double>(min_p));
            const int first = passed ? __ffsll(static_cast<long long>(passed)) - 1 : 63;
            rule.least = value_of(min(centre - 31u + first, most));
        }
        cut_key = key_of(rule.least);
        for_entries<TH, 2>(row, V, [&](float z, int) {
            if (z >= rule.least) {
                int b;
                const u64 one = rule.packed(z, b);
                atomicAdd(&sh.sums[b], one);
            }
        });
        __syncthreads();
        // ---- running counts and weights over the threads' bins
        constexpr int kPer = kBins / TH;
        static_assert(8 % kPer == 0, "a thread's bins lie in one group");
        const int lane = tid & 63, wave = tid >> 6;
        const double group = RowRule::weight_of_group(tid * kPer >> 3);
        uint32_t run_c = 0;
        double run_w = 0.0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const u64 sums = sh.sums[tid * kPer + i];
            run_c += rule.count_of(sums);
            if (tid * kPer + i < kBins - 1) run_w += group * (kPer == 8 ? RowRule::weight_in_group(i) : (tid & 1 ? RowRule::weight_in_group(4 + i % 4) : RowRule::weight_in_group(i % 4))) * rule.weight_of(sums);
        }
        const double iw = wave_inclusive_sum(run_w);
        const uint32_t ic = wave_inclusive_count(run_c);
        sh.thread_weight[tid] = iw;
        sh.thread_count[tid] = ic;
        if (lane == 63) { sh.wave_weight[wave] = iw; sh.wave_count[wave] = ic; }
        __syncthreads();
        if (wave == 0) {
            const double ww = wave_inclusive_sum(lane < TH / 64 ? sh.wave_weight[lane & (TH / 64 - 1)] : 0.0);
            const uint32_t wc = wave_inclusive_count(lane < TH / 64 ? sh.wave_count[lane & (TH / 64 - 1)] : 0u);
            if (lane < TH / 64) { sh.wave_weight[lane] = ww; sh.wave_count[lane] = wc; }
        }
        __syncthreads();
        const uint32_t all = sh.wave_count[TH / 64 - 1];
        double total = sh.wave_weight[TH / 64 - 1];
        bool cut = false;
        Found last{};
#pragma unroll 1
        for (int mode = 0; mode < 3; ++mode) {              // top_k, top_p, the draw
            Goal goal{mode, 0.0};
            if (mode == 0) {
                if (static_cast<uint32_t>(k) >= all) continue;
                goal.goal = k;
            } else if (mode == 1) {
                if (!(top_p < 1.0f)) continue;
                goal.goal = fmin(fmax(static_cast<double>(top_p) * total, 1e-300), total);
            } else {
                if (!p.out_tokens) continue;
                goal.goal = fmax(static_cast<double>(p.u[r]) * total, 0.0);
                if (!(goal.goal < total)) {                 // the last place
                    if (cut) { token = last.index; continue; }
                    goal = Goal{0, static_cast<double>(all)};
                }
            }
            const Found f = find_place<TH>(sh, row, V, rule, goal);
            if (mode == 2) token = f.index;
            else { last = f; cut = true; total = f.weight; cut_key = f.key; cut_index = f.index; }
        }
    }
    if (p.out_tokens && tid == 0) p.out_tokens[r] = token;
    if (!p.kept) return;
    T *kept = static_cast<T *>(p.kept) + r * p.kept_stride;
    constexpr int PV = Elem<T>::kPerVec;
    const float cut_z = value_of(cut_key);                  // (where the row is empty: the lowest finite value)
    auto stays = [&](float z, int i) { return z > cut_z || (z == cut_z && i <= cut_index); };
    const T gone = sizeof(T) == 2 ? static_cast<T>(0xFF80u) : __builtin_bit_cast(float, 0xFF800000u);
    const int head = min(V, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / static_cast<int>(sizeof(T)));
    const bool wide = ((reinterpret_cast<uintptr_t>(row) ^ reinterpret_cast<uintptr_t>(kept)) & 15) == 0;
    const int vectors = wide ? (V - head) / PV : 0;
    constexpr int kAtOnce = 4;
    for (int v0 = tid; v0 < vectors; v0 += TH * kAtOnce) {
        U4 raw[kAtOnce];
#pragma unroll
        for (int n = 0; n < kAtOnce; ++n) raw[n] = *reinterpret_cast<const U4 *>(row + head + min(v0 + n * TH, vectors - 1) * PV);
#pragma unroll
        for (int n = 0; n < kAtOnce; ++n) {
            const int i = head + (v0 + n * TH) * PV;
            if (v0 + n * TH >= vectors) break;
            float z[PV];
            T e[PV];
            Elem<T>::unpack(raw[n], z);
            __builtin_memcpy(e, &raw[n], 16);
#pragma unroll
            for (int j = 0; j < PV; ++j) e[j] = stays(z[j], i + j) ? e[j] : gone;
            U4 out;
            __builtin_memcpy(&out, e, 16);
            *reinterpret_cast<U4 *>(kept + i) = out;
        }
    }
    const int done = vectors * PV;                          // entries in front of and behind the vectors
    for (int j = tid; j < V - done; j += TH) {
        const int i = j < head || !wide ? j : j + done;
        const T e = row[i];
        kept[i] = stays(Elem<T>::scalar(row + i), i) ? e : gone;
    }
}

template <int TH, typename T>
__global__ void __launch_bounds__(TH, 4) k_filter(FilterProblem p)
{
    __shared__ FilterShared sh;
    filter_row<TH, T>(p, blockIdx.x, sh);
}

// bfloat16 rows of up to NV 8 TH - 7 entries, and 65521 where the halves of the counters are not looked after.
//
// A bfloat16 has 2^15 magnitudes: the row is counted into one 32-bit counter each, entries in the low half and those below zero in the high
// half, and everything about the order follows from the counts.  So an entry costs one addition in LDS, an exponential in
// float64 is formed for each value that occurs and not for each entry, and sums of weights are products and sums in float64 in a fixed
// order.  The row stays in registers, where the index of the n-th entry of a value is looked up and from where the kept entries are
// written.  A half overflows if a magnitude occurs 65536 times or more; the entries counted and the sum of the low halves disagree then
// (each overflow takes 65535 or 65536 from it), and the row is done by filter_row.
typedef uint16_t U2x16 __attribute__((ext_vector_type(2)));
constexpr uint32_t kNegInf2 = 0xFF80FF80u;
constexpr int kMaxTurns = 8192;               // rows of a workgroup at most

// TH threads count 32 TH magnitudes: 1024 all of them, 512 those from 2^-63 (which stands for 0) up to 2^65 (the last one stands for -inf).
// A row with other entries than these (and 0 and -inf) is done by filter_row.
template <int TH> struct CountShared {
    uint32_t count[32 * TH];
    double of_octave[64];                     // 2^(j / 64)
    // of the segments of 64 values: TH / 2 of magnitudes from the top down, then TH / 2 below zero from 0 down
    double seg_weight[TH];                    // running sums within blocks of 64 segments
    uint32_t seg_count[TH];
    double wave_weight[TH / 64];
    uint32_t wave_count[TH / 64];
    uint32_t chunk[TH / 64];                  // entries of a value
    uint32_t place[2], nth[2];                // the cut's value (nth 0: all its entries stay) and the token's
    u64 occurs[TH / 64], above[TH / 64];
    uint32_t counted, summed, outside;
    int index;
};

struct Value {                                // the n-th of `all` entries of one value in a row
    uint32_t bits;                            // as in memory; zero: both
    uint32_t nth, all;
    double weight;                            // of the entries up to and including it
};

__device__ __forceinline__ u64 lane_bits_of(u64 v, int src)
{
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(v), src), hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(v >> 32), src);
    return static_cast<u64>(hi) << 32 | lo;
}

template <int NV, int TH>
__global__ void __launch_bounds__(TH, 4) k_filter_counts(FilterProblem p)
{
    constexpr int kWaves = TH / 64;
    constexpr uint32_t kMagnitudes = 32 * TH, kLowest = TH == 1024 ? 0u : 0x2000u;     // counter c is of magnitude kLowest + c
    __shared__ union { CountShared<TH> c; FilterShared f; } shared;
    __shared__ uint32_t again[kMaxTurns / 32];                     // rows of this workgroup that are to be done over
    CountShared<TH> &sh = shared.c;
    constexpr bool kAhead = NV == 8 && TH == 1024;                 // the next row is loaded while this one is worked on
    constexpr bool kMayOverflow = NV * TH > 8 * 1024;              // fewer vectors than 2^13 hold fewer than 2^16 entries
    int tid = threadIdx.x;
    const int V = p.V;
    const uint16_t *logits = static_cast<const uint16_t *>(p.logits);

    // vector j of a row: entries 8 j - lead to 8 j - lead + 7, from the 16-byte boundary in front of it on
    auto lead_of = [&](int r) { return static_cast<int>((reinterpret_cast<uintptr_t>(logits + r * p.row_stride) & 15) / 2); };
    // (a wave's vectors are adjacent, so that entries of lower indices are in lower waves)
    auto per_thread = [&](int lead) { return (lead + V + 8 * TH - 1) / (8 * TH); };
    auto load = [&](int r, U4 (&x)[NV]) {
        const int lead = lead_of(r), last = (lead + V - 1) / 8, j0 = (tid >> 6) * per_thread(lead) * 64 + (tid & 63);
        const U4 *vec = reinterpret_cast<const U4 *>(logits + r * p.row_stride - lead);
#pragma unroll
        for (int v = 0; v < NV; ++v) x[v] = vec[min(j0 + v * 64, last)];
    };
    auto clear = [&]() {
        U4 *c = reinterpret_cast<U4 *>(sh.count);
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i * TH + tid] = U4{0, 0, 0, 0};
    };
    // two entries' counters
    auto counters = [&](uint32_t w) {
        w &= 0x7FFF7FFFu;
        if constexpr (TH == 1024) return w;
        constexpr uint16_t last = kMagnitudes - 1;
        const U2x16 x = __builtin_elementwise_sub_sat(__builtin_bit_cast(U2x16, w), U2x16{kLowest, kLowest});
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(x, U2x16{last, last}));
    };

    U4 row[NV], next[kAhead ? NV : 1];
    int r = blockIdx.x, nth_row = 0;
    if (r >= p.rows) return;
    if (tid < kMaxTurns / 32) again[tid] = 0;
    load(r, row);
    clear();
    if (tid == 0) { sh.counted = 0; sh.summed = 0; sh.outside = 0; }
    sh.seg_weight[tid] = 0.0;
    sh.seg_count[tid] = 0;
    if (tid >= TH - 64) sh.of_octave[tid - (TH - 64)] = exp_of((tid - (TH - 64)) * 0.010830424696249145);      // ln(2) / 64
    __syncthreads();
    for (;;) {
        if constexpr (kAhead) asm volatile("" : "+v"(tid));        // (what follows from it is made anew: kept over rows it would cost the registers)
        const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const RowAsked asked(p, r);
        const float u = p.out_tokens ? p.u[r] : 0.0f;
        const int lead = lead_of(r), vectors = (lead + V + 7) / 8, after = r + gridDim.x;
        const int turns = per_thread(lead), j0 = wave * turns * 64 + lane;       // of its vectors: v < turns, number j0 + 64 v
        if constexpr (kAhead) if (after < p.rows) load(after, next);

        // ---- counts
        uint32_t counted = 0;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            __builtin_amdgcn_sched_barrier(0);                     // (one vector at a time: registers)
            if (v >= turns) continue;                              // uniform
            const int i0 = 8 * (j0 + 64 * v) - lead;
            if (i0 < 0 || i0 + 8 > V) {                            // entries that are not the row's (a call in place may be writing them) are -inf
                uint32_t *w = &row[v].x;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (i0 + 2 * i < 0 || i0 + 2 * i >= V) w[i] = (w[i] & 0xFFFF0000u) | 0xFF80u;
                    if (i0 + 2 * i + 1 < 0 || i0 + 2 * i + 1 >= V) w[i] = (w[i] & 0xFFFFu) | 0xFF800000u;
                }
            }
            const U4 x = row[v];
            const bool some = j0 + 64 * v < vectors &&
                              ((x.x ^ kNegInf2) | (x.y ^ kNegInf2) | (x.z ^ kNegInf2) | (x.w ^ kNegInf2)) != 0;
            counted += __popcll(__ballot(some));
            if (some) {
                const uint32_t *w = &x.x;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t c = counters(w[i]);
                    atomicAdd(&sh.count[c & 0xFFFFu], (w[i] << 1 & 0x10000u) + 1u);
                    atomicAdd(&sh.count[c >> 16], (w[i] >> 15 & 0x10000u) + 1u);
                }
            }
        }
        if (lane == 0) atomicAdd(&sh.counted, 8 * counted);
        __syncthreads();
        if constexpr (TH < 1024) {
            if ((sh.count[0] | sh.count[kMagnitudes - 1]) != 0) {  // uniform: of the row's entries, are these 0 and -inf?
                uint32_t found = 0;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    __builtin_amdgcn_sched_barrier(0);
                    if (v >= turns || j0 + 64 * v >= vectors) continue;
                    const uint32_t *w = &row[v].x;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t e = w[i / 2] >> (i & 1) * 16 & 0xFFFFu, m = e & 0x7FFFu;
                        found |= m - kLowest - 1 >= kMagnitudes - 2 && m != 0 && e != 0xFF80u ? 1u : 0u;
                    }
                }
                if (__any(found != 0) && lane == 0) sh.outside = 1;
            }
        }

        // ---- which magnitudes occur: 32 a thread, its eight vectors in an order in which neighbours meet no bank twice
        auto split = [&](int m, uint32_t &pos, uint32_t &neg) {
            const uint32_t d = sh.count[m];
            if constexpr (TH == 1024) {
                neg = m == 0 || m >= 0x7F80 ? 0u : d >> 16;        // (both zeros are one value; -inf and what is no number do not take part)
                pos = m > 0x7F80 ? 0u : (m == 0x7F80 ? (d & 0xFFFFu) - (d >> 16) : (d & 0xFFFFu) - neg);
            } else {
                neg = m == 0 || m == kMagnitudes - 1 ? 0u : d >> 16;
                pos = m == kMagnitudes - 1 ? 0u : (d & 0xFFFFu) - neg;
            }
        };
        {
            uint32_t any = 0, twice_above = 0, both = 0;
            const U4 *mine = reinterpret_cast<const U4 *>(sh.count) + tid * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const U4 d = mine[(i + tid) & 7];
                const uint32_t *w = &d.x;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    any |= w[e];
                    twice_above = __builtin_amdgcn_sad_u16(w[e], __builtin_amdgcn_alignbit(w[e], w[e], 16), twice_above);   // 2 (low - high)
                    if (kMayOverflow) both = __builtin_amdgcn_sad_u16(w[e], 0u, both);                                      // low + high
                }
            }
            const u64 occurs = __ballot(any != 0), above = __ballot(twice_above != 0);
            if (lane == 0) {                                       // segments of 64 are pairs of threads: the even bits
                sh.occurs[wave] = (occurs | occurs >> 1) & 0x5555555555555555ull;
                sh.above[wave] = (above | above >> 1) & 0x5555555555555555ull;
            }
            if (kMayOverflow) {
                // low = (low + high + |low - high|) / 2; where a half overflowed this is less than what was counted
                uint32_t low = (both + twice_above / 2) / 2;
                low = wave_inclusive_count(low);
                if (lane == 63) atomicAdd(&sh.summed, low);
            }
        }
        __syncthreads();
        const u64 occurs = lane < kWaves ? sh.occurs[lane] : 0ull;
        // the largest value: the highest segment with one above zero, else the first below; 0x8000 + counter, or 0x7FFF - counter
        uint32_t top = 0;
        {
            u64 above = lane < kWaves ? sh.above[lane] : 0ull;
            if (lane == 0) above |= 1;                             // (zeros below zero alone do not show)
            while (top == 0) {
                const u64 words = __ballot(above != 0);
                if (words == 0) break;
                const int word = 63 - __clzll(static_cast<long long>(words));
                const u64 bits = lane_bits_of(above, word);
                const int bit = 63 - __clzll(static_cast<long long>(bits)), base = (word * 32 + bit / 2) * 64;
                uint32_t pos, neg;
                split(base + lane, pos, neg);
                const u64 hit = __ballot(pos != 0);
                if (hit) top = 0x8000u + base + 63 - __clzll(static_cast<long long>(hit));
                if (lane == word) above &= ~(1ull << bit);
            }
            u64 left = occurs;
            while (top == 0) {
                const u64 words = __ballot(left != 0);
                if (words == 0) break;
                const int word = __ffsll(static_cast<long long>(words)) - 1;
                const u64 bits = lane_bits_of(left, word);
                const int bit = __ffsll(static_cast<long long>(bits)) - 1, base = (word * 32 + bit / 2) * 64;
                uint32_t pos, neg;
                split(base + lane, pos, neg);
                const u64 hit = __ballot(neg != 0);
                if (hit) top = 0x7FFFu - base - (__ffsll(static_cast<long long>(hit)) - 1);
                if (lane == word) left &= ~(1ull << bit);
            }
        }
        const bool overflow = TH < 1024 ? sh.outside != 0 : kMayOverflow && sh.summed != sh.counted;       // uniform
        uint32_t cut_bits = 0xFF7Fu;                               // what is kept: larger values, and this one up to an index
        int cut_index = INT32_MAX, token = -1;
        if (overflow || top == 0) {                                // to be done over at the end, or no entries
            __syncthreads();
            clear();
            if (overflow && tid == 0) again[nth_row / 32] |= 1u << nth_row % 32;
        } else {
            // bits of the value of a counter
            auto value_bits = [&](uint32_t c) { return TH == 1024 || c == 0 ? c : kLowest + c; };
            const float top_z = __uint_as_float((top >= 0x8000u ? value_bits(top - 0x8000u) : 0x8000u | value_bits(0x7FFFu - top)) << 16);
            const double inv_t = asked.per_temperature(), min_w = asked.min_p > 0.0f ? static_cast<double>(asked.min_p) : 0.0;
            auto weight = [&](uint32_t bits) {
                const float z = __uint_as_float(bits << 16);
                return z == top_z ? 1.0 : exp_from(sh.of_octave, (static_cast<double>(z) - static_cast<double>(top_z)) * inv_t);
            };
            // ---- counts and weights of the segments that hold something: segment n is wave n % kWaves's
#pragma unroll 1
            for (int set = 0; set < 32; set += kWaves) {
                u64 words = __ballot((occurs >> (2 * (wave + set)) & 1) != 0);
#pragma unroll 1
                while (words) {
                    const int word = __ffsll(static_cast<long long>(words)) - 1, at = word * 32 + wave + set;
                    words &= words - 1;
                    uint32_t pos, neg;
                    split(at * 64 + lane, pos, neg);
                    const double wp = weight(value_bits(at * 64 + lane)), wn = weight(0x8000u | value_bits(at * 64 + lane));
                    if (!(wp >= min_w)) pos = 0;
                    if (!(wn >= min_w)) neg = 0;
                    const uint32_t cp = wave_inclusive_count(pos), cn = wave_inclusive_count(neg);
                    const double sp = wave_inclusive_sum(pos ? pos * wp : 0.0), sn = wave_inclusive_sum(neg ? neg * wn : 0.0);
                    if (lane == 63) {
                        sh.seg_count[TH / 2 - 1 - at] = cp; sh.seg_weight[TH / 2 - 1 - at] = sp;
                        sh.seg_count[TH / 2 + at] = cn; sh.seg_weight[TH / 2 + at] = sn;
                    }
                }
            }
            __syncthreads();
            // ---- running sums over the segments, within blocks of 64
            const double run_w = wave_inclusive_sum(sh.seg_weight[tid]);
            const uint32_t run_c = wave_inclusive_count(sh.seg_count[tid]);
            sh.seg_weight[tid] = run_w;
            sh.seg_count[tid] = run_c;
            if (lane == 63) { sh.wave_weight[wave] = run_w; sh.wave_count[wave] = run_c; }
            __syncthreads();

            // ---- places in the order: by count (top_k; or all, where what min_p leaves is asked for), by weight (top_p), and the draw.
            // One wave goes down from blocks to segments to values, 64 at a time; the others would only take its issue slots.
            if (wave == 0) {
                const double block_w = wave_inclusive_sum(lane < kWaves ? sh.wave_weight[lane & (kWaves - 1)] : 0.0);
                const uint32_t block_c = wave_inclusive_count(lane < kWaves ? sh.wave_count[lane & (kWaves - 1)] : 0u);
                const uint32_t all = __builtin_amdgcn_readlane(block_c, 63);
                double total = lane_value(block_w, 63);

                // the first place whose count (how 0) or weight (1) reaches the goal, or whose weight exceeds it (2)
                auto locate = [&](int how, double goal) {
                    // the first of 64 running sums to reach it; where rounding leaves none, the last that holds something
                    auto first = [&](uint32_t c, double w, bool holds) {
                        const u64 hit = __ballot(holds && (how == 0 ? c >= goal : (how == 1 ? w >= goal : w > goal))), some = __ballot(holds);
                        return hit ? __ffsll(static_cast<long long>(hit)) - 1 : 63 - __clzll(static_cast<long long>(some | 1));
                    };
                    const int block = first(block_c, block_w, lane < kWaves && sh.wave_count[lane & (kWaves - 1)] != 0);
                    double w0 = block ? lane_value(block_w, block - 1) : 0.0;
                    uint32_t c0 = block ? __builtin_amdgcn_readlane(block_c, block - 1) : 0u;
                    const double seg_w = sh.seg_weight[block * 64 + lane];
                    const uint32_t seg_c = sh.seg_count[block * 64 + lane], seg_before = lane ? sh.seg_count[block * 64 + lane - 1] : 0u;
                    const int seg = first(c0 + seg_c, w0 + seg_w, seg_c != seg_before), o = block * 64 + seg;
                    if (seg) { w0 += lane_value(seg_w, seg - 1); c0 += __builtin_amdgcn_readlane(seg_c, seg - 1); }
                    const bool minus = o >= TH / 2;
                    const int at = minus ? o - TH / 2 : TH / 2 - 1 - o, m = at * 64 + (minus ? lane : 63 - lane);
                    uint32_t pos, neg;
                    split(m, pos, neg);
                    uint32_t n = minus ? neg : pos;
                    const uint32_t bits = (minus ? 0x8000u : 0u) | value_bits(m);
                    const double w = weight(bits);
                    if (!(w >= min_w)) n = 0;
                    const double iw = w0 + wave_inclusive_sum(n ? n * w : 0.0);
                    const uint32_t ic = c0 + wave_inclusive_count(n);
                    const int l = first(ic, iw, n != 0);
                    Value f;
                    f.bits = __builtin_amdgcn_readlane(bits, l);
                    f.all = __builtin_amdgcn_readlane(n, l);
                    const double each = lane_value(w, l), front_w = lane_value(iw, l) - f.all * each;
                    const uint32_t front_c = __builtin_amdgcn_readlane(ic, l) - f.all;
                    double nth = how == 0 ? goal - front_c : (goal - front_w) / each;
                    nth = how == 0 ? nth : (how == 1 ? ceil(nth) : floor(nth) + 1.0);
                    nth = nth >= 1.0 ? nth : 1.0;                  // (each may be 0: then the first)
                    f.nth = nth < f.all ? static_cast<uint32_t>(nth) : f.all;
                    f.weight = front_w + f.nth * each;
                    return f;
                };
                bool cut = false;
                Value last{}, drawn{};
#pragma unroll 1
                for (int mode = 0; mode < 3; ++mode) {
                    double goal;
                    int how = mode;
                    if (mode == 0) {
                        if (static_cast<uint32_t>(asked.k) >= all && !(min_w > 0.0 && p.kept)) continue;
                        goal = static_cast<uint32_t>(asked.k) < all ? asked.k : all;
                    } else if (mode == 1) {
                        if (!(asked.top_p < 1.0f)) continue;
                        goal = fmax(static_cast<double>(asked.top_p) * total, 1e-300);
                    } else {
                        if (!p.out_tokens) continue;
                        goal = fmax(static_cast<double>(u) * total, 0.0);
                        if (!(goal < total)) {                     // the last place
                            if (cut) { drawn = last; continue; }
                            how = 0; goal = all;
                        }
                    }
                    const Value f = locate(how, goal);
                    if (mode == 2) drawn = f;
                    else { last = f; cut = true; total = f.weight; }
                }
                if (lane == 0) {
                    sh.place[0] = cut ? last.bits : 0xFF7Fu;       // (without a cut: the lowest value there is, all of it)
                    sh.nth[0] = cut && last.nth < last.all ? last.nth : 0u;
                    sh.place[1] = drawn.bits; sh.nth[1] = drawn.nth;
                }
            }
            __syncthreads();
            clear();
            sh.seg_weight[tid] = 0.0;
            sh.seg_count[tid] = 0;

            // ---- their indices in the row, from the registers: how many entries of the value each wave holds, then the wave in question
            cut_bits = sh.place[0];
#pragma unroll 1
            for (int which = 0; which < 2; ++which) {
                const uint32_t bits = sh.place[which], nth = sh.nth[which];
                if (which == 0 ? !p.kept || nth == 0 : !p.out_tokens) continue;          // uniform
                const uint32_t pair = bits | bits << 16, care = bits == 0 ? 0x7FFF7FFFu : 0xFFFFFFFFu;
                int j1 = j0;
                asm volatile("" : "+v"(j1));                       // (what follows from it is not made for every vector in front of the loops)
                auto some_match = [&](const U4 &x) {
                    const uint32_t *w = &x.x;
                    U2x16 least = __builtin_bit_cast(U2x16, (w[0] ^ pair) & care);
#pragma unroll
                    for (int i = 1; i < 4; ++i) least = __builtin_elementwise_min(least, __builtin_bit_cast(U2x16, (w[i] ^ pair) & care));
                    return least.x == 0 || least.y == 0;
                };
                auto matches = [&](const U4 &x, int v) {           // bits: which of a vector's entries are the row's and of the value
                    const uint32_t *w = &x.x;
                    uint32_t m = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t d = (w[i] ^ pair) & care;
                        m |= ((d & 0xFFFFu) == 0 ? 1u : 0u) << (2 * i) | (d >> 16 == 0 ? 2u : 0u) << (2 * i);
                    }
                    return j1 + 64 * v < vectors ? m : 0u;         // (behind the row: its last vector again)
                };
                uint32_t mine = 0;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    __builtin_amdgcn_sched_barrier(0);
                    if (v >= turns) continue;
                    if (some_match(row[v])) mine += __popc(matches(row[v], v));
                }
                const uint32_t run = wave_inclusive_count(mine);
                if (lane == 63) sh.chunk[wave] = run;
                __syncthreads();
                const uint32_t before = wave_inclusive_count(lane < wave ? sh.chunk[lane & (kWaves - 1)] : 0u), here = sh.chunk[wave];
                const uint32_t front = __builtin_amdgcn_readlane(before, 63);
                if (front < nth && nth <= front + here) {          // one wave
                    uint32_t left = nth - front;
#pragma unroll
                    for (int v = 0; v < NV; ++v) {
                        __builtin_amdgcn_sched_barrier(0);
                        if (v >= turns) continue;
                        if (!__any(some_match(row[v]))) continue;
                        uint32_t m = matches(row[v], v);
                        const uint32_t c = __popc(m), ic = wave_inclusive_count(c), n = __builtin_amdgcn_readlane(ic, 63);
                        if (left >= 1 && left <= n && ic >= left && ic - c < left) {
                            for (uint32_t skip = left - (ic - c); skip > 1; --skip) m &= m - 1;
                            sh.index = 8 * (j1 + 64 * v) - lead + __ffs(static_cast<int>(m)) - 1;
                        }
                        left -= n;                                 // (at or past the place: 0 or a huge number, and no lane is left)
                    }
                }
                __syncthreads();
                if (which == 0) cut_index = sh.index;
                else token = sh.index;
            }
        }
        if (!overflow) {
            if (p.out_tokens && tid == 0) p.out_tokens[r] = token;
            if (p.kept) {
                uint16_t *kept = static_cast<uint16_t *>(p.kept) + r * p.kept_stride;
                const bool wide = static_cast<int>((reinterpret_cast<uintptr_t>(kept) & 15) / 2) == lead;
                const float least = __uint_as_float(cut_bits << 16);
                // larger than `under` is at least `least`
                const float under = least == 0.0f ? -__uint_as_float(1u) : __uint_as_float(least > 0.0f ? __float_as_uint(least) - 1 : __float_as_uint(least) + 1);
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    __builtin_amdgcn_sched_barrier(0);
                    const int j = j0 + 64 * v, i0 = 8 * j - lead;
                    if (v >= turns || j >= vectors) continue;
                    const uint32_t *w = &row[v].x;
                    const float whole = i0 > cut_index ? least : under;
                    U4 x;
                    uint32_t *o = &x.x;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float lo = bf16_lo(w[e]), hi = bf16_hi(w[e]);
                        bool a = lo > whole, b = hi > whole;
                        if (i0 <= cut_index && i0 + 7 > cut_index) {               // one vector of the row at most
                            a = lo > least || (lo == least && i0 + 2 * e <= cut_index);
                            b = hi > least || (hi == least && i0 + 2 * e + 1 <= cut_index);
                        }
                        o[e] = (a ? w[e] & 0xFFFFu : 0xFF80u) | (b ? w[e] & 0xFFFF0000u : 0xFF800000u);
                    }
                    if (wide && i0 >= 0 && i0 + 8 <= V) *reinterpret_cast<U4 *>(kept + i0) = x;
                    else
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (i0 + e >= 0 && i0 + e < V) kept[i0 + e] = static_cast<uint16_t>(o[e / 2] >> (e & 1) * 16);
                }
            }
        }
        if (!kAhead || after >= p.rows) break;
        r = after;
        ++nth_row;
        if (tid == 0) { sh.counted = 0; sh.summed = 0; sh.outside = 0; }
        if constexpr (kAhead) {
#pragma unroll
            for (int v = 0; v < NV; ++v) row[v] = next[v];
        }
        __syncthreads();
    }
    if constexpr (!kMayOverflow && TH == 1024) return;
    __syncthreads();
    for (int i = 0; i <= nth_row; ++i)
        if (again[i / 32] >> i % 32 & 1) {                         // uniform
            filter_row<TH, uint16_t>(p, blockIdx.x + i * gridDim.x, shared.f);
            __syncthreads();
        }
}

template <int NV, int TH>
hipError_t launch_counts(const FilterProblem &p, hipStream_t stream)
{
    const int units = NV == 8 && TH == 1024 ? compute_units() : p.rows, least = (p.rows + kMaxTurns - 1) / kMaxTurns, most = units > least ? units : least;
    hipLaunchKernelGGL((k_filter_counts<NV, TH>), dim3(p.rows < most ? p.rows : most), dim3(TH), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_filter(const FilterProblem &p, int dtype, hipStream_t stream)
{
    const int64_t span = static_cast<int64_t>(p.V) + 7;            // entries with those in front of the row's first vector
    const bool few = p.rows <= compute_units();
    // 16 / 8 waves, us, rows of 32000: 200 of them 15.7 / 16.1, 270 28 / 21, 1152 70 / 48.  Longer rows do not fit into the registers of two workgroups.
    if (dtype == 1 && span <= 8 * 4096 && !few) return launch_counts<8, 512>(p, stream);
    // The fewest vectors a lane that hold the row (more cost registers and turns).  With these / the next ones, 100 rows, us: 32000 entries 15.6 / 17.6, 64000
    // 20.5 / 21.5 (600 rows, which load ahead, 60 / 63), 128256 28 / 32, 152064 36 / 77 (k_filter).
    if (dtype == 1 && span <= 4 * 8192) return launch_counts<4, 1024>(p, stream);
    if (dtype == 1 && span <= 8 * 8191) return launch_counts<8, 1024>(p, stream);          // (one vector less: its counters must not overflow)
    if (dtype == 1 && span <= 16 * 8192) return launch_counts<16, 1024>(p, stream);
    if (dtype == 1 && span <= 20 * 8192) return launch_counts<20, 1024>(p, stream);
    // A row a compute unit: 16 waves each; more: 8, so that two rows share a unit and one's waits are the other's work.  16 / 8 waves, us:
    // float32 rows of 32003 entries, 64 of them 26 / 30, 256 33 / 38, 287 53 / 45, 1200 133 / 122; bfloat16 of 200000, 64 of them 90 / 119, 300 182 / 174.
    const dim3 grid(p.rows);
    if (dtype == 1 && few) hipLaunchKernelGGL((k_filter<1024, uint16_t>), grid, dim3(1024), 0, stream, p);
    else if (dtype == 1) hipLaunchKernelGGL((k_filter<512, uint16_t>), grid, dim3(512), 0, stream, p);
    else if (few) hipLaunchKernelGGL((k_filter<1024, float>), grid, dim3(1024), 0, stream, p);
    else hipLaunchKernelGGL((k_filter<512, float>), grid, dim3(512), 0, stream, p);
    return hipGetLastError();
}

}  // namespace specgbv
