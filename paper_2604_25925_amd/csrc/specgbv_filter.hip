// Truncated distributions and draws from them (specgbv_sample_filtered): one workgroup per row.
//
// With the entries of a row in the order "largest logit first, ties by the lowest index", each of top-k, min-p and top-p keeps the
// front of the order, and the draw looks for the entry at which the running weight passes a goal.  So everything asked for is a place in
// that order, by rank or by running weight, and the row needs no sorting: a histogram by value (counts and sums of weights) says in which
// bin the place lies, and only that bin's entries are put in order.
//
// Weights decide which entry is drawn, and every entry counts: they are exponentials in float64, summed as integers of 43 fractional bits,
// so that neither the order of the additions nor their rounding can move a border (2^20 entries of at most 1 stay below 2^64; what the
// rounding of each leaves out is 2^-44 of the largest entry).
#include "specgbv_internal.hpp"

namespace specgbv {
namespace {

constexpr int kFilterThreads = 1024, kFilterWaves = kFilterThreads / 64;
constexpr int kBins = 4096;                   // of the row's histogram, equally wide in the logit
constexpr int kList = 1024;                   // entries that are put in order at once; bins of a closer histogram
constexpr float kSpan = 48.0f;                // the histogram's width in temperatures: e^-48 of the largest weight is less than 2^-44
constexpr double kOne = 8796093022208.0;      // 2^43

typedef unsigned long long u64;

// Order of logits as order of integers; both zeros are one value, and what is no number comes last, as -inf does.
__device__ __forceinline__ uint32_t key_of(float z)
{
    const uint32_t b = __float_as_uint(z == z ? z + 0.0f : -INFINITY);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
constexpr uint32_t kNothing = 0x007FFFFFu;    // key of -inf

// e^x for x <= 0 in float64: 2^n times the Taylor sum of e^r, |r| <= ln(2) / 2, to r^12 / 12!, whose remainder is 2 10^-16 of it.
__device__ __forceinline__ double exp_of(double x)
{
    x = fmax(x, -800.0);                                     // (below 2^-1074: 0)
    const double n = rint(x * 1.44269504088896340736);
    double r = fma(n, -6.93147180369123816490e-01, x);       // the high bits of ln 2, then the rest
    r = fma(n, -1.90821492927058770002e-10, r);
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

struct RowRule {                              // how a row's entries are weighed and binned
    float top;                                // its largest logit
    double inv_t;
    float bins;                               // bins per unit of the logit
    uint32_t least;                           // entries of lower keys do not take part

    __device__ __forceinline__ double weight(float z) const
    {
        if (z == top) return 1.0;
        return exp_of((static_cast<double>(z) - static_cast<double>(top)) * inv_t);
    }
    __device__ __forceinline__ u64 fixed(float z) const { return static_cast<u64>(weight(z) * kOne + 0.5); }
    __device__ __forceinline__ int bin(float z) const
    {
        return z == top ? 0 : static_cast<int>(fminf((top - z) * bins, static_cast<float>(kBins - 1)));
    }
};

// f(logit, index) for every entry of the row, by all threads of the workgroup: whole 16-byte vectors where the row allows.
template <typename T, typename F>
__device__ __forceinline__ void for_entries(const T *row, int V, F f)
{
    constexpr int PV = Elem<T>::kPerVec;
    const int head = min(V, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / static_cast<int>(sizeof(T)));
    const int vectors = (V - head) / PV, tail = head + vectors * PV;
    if (static_cast<int>(threadIdx.x) < head) f(Elem<T>::scalar(row + threadIdx.x), static_cast<int>(threadIdx.x));
    const U4 *vec = reinterpret_cast<const U4 *>(row + head);
    for (int v = threadIdx.x; v < vectors; v += kFilterThreads) {
        float z[PV];
        Elem<T>::unpack(vec[v], z);
#pragma unroll
        for (int j = 0; j < PV; ++j) f(z[j], head + v * PV + j);
    }
    if (static_cast<int>(threadIdx.x) < V - tail) f(Elem<T>::scalar(row + tail + threadIdx.x), tail + static_cast<int>(threadIdx.x));
}

struct Found {                                // a place in the order
    uint32_t key;
    int index;
    u64 count, weight;                        // of the entries up to and including it
};

struct FilterShared {
    u64 weight[kBins];                        // after the scan: up to and including the bin
    uint32_t count[kBins];
    u64 list_weight[kList];                   // of the list, or of the closer histogram
    uint32_t list_key[kList];
    uint32_t list_index[kList];
    u64 wave_weight[kFilterWaves];
    uint32_t wave_count[kFilterWaves];
    uint32_t n, lo, hi;
    int bin;
    Found found;
};

// Running sums over n = kFilterThreads * PER bins in place.
template <int PER>
__device__ void scan_bins(FilterShared &sh, u64 *weight, uint32_t *count)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    u64 w = 0;
    uint32_t c = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) { w += weight[tid * PER + i]; c += count[tid * PER + i]; }
    u64 iw = w;
    uint32_t ic = c;
    for (int d = 1; d < 64; d <<= 1) {
        const u64 ow = __shfl_up(iw, d, 64);
        const uint32_t oc = __shfl_up(ic, d, 64);
        if (lane >= d) { iw += ow; ic += oc; }
    }
    if (lane == 63) { sh.wave_weight[wave] = iw; sh.wave_count[wave] = ic; }
    __syncthreads();
    for (int i = 0; i < wave; ++i) { iw += sh.wave_weight[i]; ic += sh.wave_count[i]; }
    iw -= w; ic -= c;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        iw += weight[tid * PER + i]; ic += count[tid * PER + i];
        weight[tid * PER + i] = iw; count[tid * PER + i] = ic;
    }
    __syncthreads();
}

// The first place whose count (by_count) or weight reaches `goal` (at least 1 and at most the row's).
template <typename T>
__device__ Found find_place(FilterShared &sh, const T *row, int V, const RowRule &rule, bool by_count, u64 goal)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    auto reached = [&](u64 count, u64 weight) { return (by_count ? count : weight) >= goal; };
    for (int b = tid; b < kBins; b += kFilterThreads)
        if (reached(sh.count[b], sh.weight[b]) && (b == 0 || !reached(sh.count[b - 1], sh.weight[b - 1]))) sh.bin = b;
    __syncthreads();
    const int bin = sh.bin;
    u64 count0 = bin ? sh.count[bin - 1] : 0, weight0 = bin ? sh.weight[bin - 1] : 0;
    uint32_t n = sh.count[bin] - static_cast<uint32_t>(count0);
    uint32_t lo = 0, hi = 0xFFFFFFFFu;
    bool closer = false;                                    // the keys in question are [lo, hi], else the bin
    auto inside = [&](float z, uint32_t key) { return key >= rule.least && (closer ? key >= lo && key <= hi : rule.bin(z) == bin); };

    while (n > kList) {
        // keys of the entries in question, and a closer histogram over them
        __syncthreads();
        if (tid == 0) { sh.lo = 0xFFFFFFFFu; sh.hi = 0; }
        __syncthreads();
        uint32_t least = 0xFFFFFFFFu, most = 0;
        for_entries(row, V, [&](float z, int) {
            const uint32_t key = key_of(z);
            if (inside(z, key)) { least = min(least, key); most = max(most, key); }
        });
        atomicMin(&sh.lo, least);
        atomicMax(&sh.hi, most);
        sh.list_weight[tid] = 0; sh.list_key[tid] = 0;
        __syncthreads();
        const uint32_t from = sh.lo, to = sh.hi;
        if (from == to) { lo = hi = from; closer = true; break; }                  // ties alone
        int shift = 0;
        while (((to - from) >> shift) >= kList) ++shift;
        for_entries(row, V, [&](float z, int) {
            const uint32_t key = key_of(z);
            if (inside(z, key)) {
                atomicAdd(&sh.list_key[(to - key) >> shift], 1u);
                atomicAdd(&sh.list_weight[(to - key) >> shift], rule.fixed(z));
            }
        });
        __syncthreads();
        scan_bins<1>(sh, sh.list_weight, sh.list_key);
        if (reached(count0 + sh.list_key[tid], weight0 + sh.list_weight[tid]) &&
            (tid == 0 || !reached(count0 + sh.list_key[tid - 1], weight0 + sh.list_weight[tid - 1]))) sh.bin = tid;
        __syncthreads();
        const int b = sh.bin;
        n = sh.list_key[b] - (b ? sh.list_key[b - 1] : 0u);
        if (b) { count0 += sh.list_key[b - 1]; weight0 += sh.list_weight[b - 1]; }
        const uint32_t top = to - (static_cast<uint32_t>(b) << shift), width = (1u << shift) - 1;
        hi = top; lo = top - from >= width ? top - width : from;
        closer = true;
    }
    __syncthreads();

    if (n > kList) {                                        // more ties than the list holds: by index, a stretch of the row per wave
        const u64 each = rule.fixed(value_of(lo));
        const u64 nth = by_count ? goal - count0 : (goal - weight0 + each - 1) / each;         // from 1 on
        const int stretch = (V + kFilterWaves - 1) / kFilterWaves, from = min(V, wave * stretch), to = min(V, from + stretch);
        uint32_t mine = 0;
        for (int i = from; i < to; i += 64) {
            const bool is = i + lane < to && key_of(Elem<T>::scalar(row + min(i + lane, V - 1))) == lo;
            mine += __popcll(__ballot(is));
        }
        if (lane == 0) sh.wave_count[wave] = mine;
        __syncthreads();
        u64 before = 0;
        for (int i = 0; i < wave; ++i) before += sh.wave_count[i];
        if (before < nth && nth <= before + mine) {         // one wave
            for (int i = from; i < to; i += 64) {
                const bool is = i + lane < to && key_of(Elem<T>::scalar(row + min(i + lane, V - 1))) == lo;
                const u64 all = __ballot(is);
                const uint32_t here = __popcll(all);
                if (nth <= before + here) {
                    if (is && before + __popcll(all & ((2ull << lane) - 1)) == nth)
                        sh.found = Found{lo, i + lane, count0 + nth, weight0 + nth * each};
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
    for_entries(row, V, [&](float z, int i) {
        const uint32_t key = key_of(z);
        if (inside(z, key)) {
            const uint32_t at = atomicAdd(&sh.n, 1u);
            if (at < kList) { sh.list_key[at] = key; sh.list_index[at] = i; sh.list_weight[at] = rule.fixed(z); }
        }
    });
    __syncthreads();
    if (tid < static_cast<int>(n)) {
        const uint32_t key = sh.list_key[tid], index = sh.list_index[tid];
        const u64 own = sh.list_weight[tid];
        u64 count = count0, weight = weight0;
        for (uint32_t i = 0; i < n; ++i) {
            const uint32_t k = sh.list_key[i];
            if (k > key || (k == key && sh.list_index[i] < index)) { ++count; weight += sh.list_weight[i]; }
        }
        if (reached(count + 1, weight + own) && !reached(count, weight)) sh.found = Found{key, static_cast<int>(index), count + 1, weight + own};
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
        min_p = p.min_p ? fminf(p.min_p[r], 1.0f) : 0.0f;
        const int asked = p.top_k ? p.top_k[r] : 0;
        k = asked > 0 ? asked : INT32_MAX;
        if (!(temperature > 0.0f)) { temperature = 1.0f; k = 1; }
    }
};

// A row of any length and type, read from memory in every step.
template <typename T>
__device__ __forceinline__ void filter_row(const FilterProblem &p, int r, FilterShared &sh)
{
    const int tid = threadIdx.x;
    const T *row = static_cast<const T *>(p.logits) + r * p.row_stride;
    const int V = p.V;
    const RowAsked asked(p, r);
    const float temperature = asked.temperature, top_p = asked.top_p, min_p = asked.min_p;
    const int k = asked.k;

    for (int b = tid; b < kBins; b += kFilterThreads) { sh.count[b] = 0; sh.weight[b] = 0; }
    if (tid == 0) sh.hi = kNothing;
    __syncthreads();
    uint32_t most = kNothing;
    for_entries(row, V, [&](float z, int) { most = max(most, key_of(z)); });
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
        rule.inv_t = 1.0 / static_cast<double>(temperature);
        rule.bins = fminf((kBins - 1) / (kSpan * temperature), 3.0e38f);
        rule.least = kNothing + 1;
        if (min_p > 0.0f) {
            // the lowest key whose weight is at least min_p, among the keys around top + temperature ln min_p
            const float about = static_cast<float>(static_cast<double>(rule.top) + static_cast<double>(temperature) * log(static_cast<double>(min_p)));
            const uint32_t centre = max(key_of(about), kNothing + 32u);
            const uint32_t mine = min(centre - 31u + (tid & 63), most);
            const u64 passed = __ballot(rule.weight(value_of(mine)) >= static_cast<double>(min_p));
            const int first = passed ? __ffsll(static_cast<long long>(passed)) - 1 : 63;
            rule.least = min(centre - 31u + first, most);
        }
        for_entries(row, V, [&](float z, int) {
            if (key_of(z) >= rule.least) {
                const int b = rule.bin(z);
                atomicAdd(&sh.count[b], 1u);
                atomicAdd(&sh.weight[b], rule.fixed(z));
            }
        });
        __syncthreads();
        scan_bins<kBins / kFilterThreads>(sh, sh.weight, sh.count);
        u64 total = sh.weight[kBins - 1];
        cut_key = rule.least;
        if (static_cast<uint32_t>(k) < sh.count[kBins - 1]) {
            const Found f = find_place(sh, row, V, rule, true, static_cast<u64>(k));
            cut_key = f.key; cut_index = f.index; total = f.weight;
        }
        if (top_p < 1.0f) {
            const double goal = ceil(static_cast<double>(top_p) * static_cast<double>(total));
            const Found f = find_place(sh, row, V, rule, false, goal < 1.0 ? 1 : min(static_cast<u64>(goal), total));
            cut_key = f.key; cut_index = f.index; total = f.weight;
        }
        if (p.out_tokens) {
            const double goal = static_cast<double>(p.u[r]) * static_cast<double>(total);
            token = find_place(sh, row, V, rule, false, goal >= 0.0 ? (goal < static_cast<double>(total) ? min(static_cast<u64>(goal) + 1, total) : total) : 1).index;
        }
    }
    if (p.out_tokens && tid == 0) p.out_tokens[r] = token;
    if (!p.kept) return;
    T *kept = static_cast<T *>(p.kept) + r * p.kept_stride;
    constexpr int PV = Elem<T>::kPerVec;
    auto stays = [&](float z, int i) {
        const uint32_t key = key_of(z);
        return key > cut_key || (key == cut_key && i <= cut_index);
    };
    const T gone = sizeof(T) == 2 ? static_cast<T>(0xFF80u) : __builtin_bit_cast(float, 0xFF800000u);
    const int head = min(V, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / static_cast<int>(sizeof(T)));
    const bool wide = ((reinterpret_cast<uintptr_t>(row) ^ reinterpret_cast<uintptr_t>(kept)) & 15) == 0;
    const int vectors = wide ? (V - head) / PV : 0;
    for (int v = tid; v < vectors; v += kFilterThreads) {
        const int i = head + v * PV;
        const U4 raw = *reinterpret_cast<const U4 *>(row + i);
        float z[PV];
        T e[PV];
        Elem<T>::unpack(raw, z);
        __builtin_memcpy(e, &raw, 16);
#pragma unroll
        for (int j = 0; j < PV; ++j) e[j] = stays(z[j], i + j) ? e[j] : gone;
        U4 out;
        __builtin_memcpy(&out, e, 16);
        *reinterpret_cast<U4 *>(kept + i) = out;
    }
    const int done = vectors * PV;                          // entries in front of and behind the vectors
    for (int j = tid; j < V - done; j += kFilterThreads) {
        const int i = j < head || !wide ? j : j + done;
        const T e = row[i];
        kept[i] = stays(Elem<T>::scalar(row + i), i) ? e : gone;
    }
}

template <typename T>
__global__ void __launch_bounds__(kFilterThreads) k_filter(FilterProblem p)
{
    __shared__ FilterShared sh;
    filter_row<T>(p, blockIdx.x, sh);
}

// bfloat16 rows of up to NV 8192 - 8 entries.
//
// A bfloat16 has 2^15 magnitudes: the row is counted into one 32-bit counter each, entries in the low half and those below zero in the high
// half, and everything about the order follows from the counts.  So an entry costs one addition in LDS, an exponential in
// float64 is formed for each value that occurs and not for each entry, and sums of weights are products and sums in float64 in a fixed
// order.  The row stays in registers, where the index of the n-th entry of a value is looked up and from where the kept entries are
// written.  A half overflows if a magnitude occurs 65536 times or more; the entries counted and the sum of the low halves disagree then
// (each overflow takes 65535 or 65536 from it), and the row is done by filter_row.
typedef uint16_t U2x16 __attribute__((ext_vector_type(2)));
constexpr uint32_t kNegInf2 = 0xFF80FF80u;
constexpr int kSegments = 1024;               // of 64 values each: 512 of magnitudes from the top down, then 512 below zero from 0 down
constexpr int kMaxTurns = 8192;               // rows of a workgroup at most

struct CountShared {
    uint32_t count[1 << 15];
    double seg_weight[kSegments];             // running sums within blocks of 64 segments
    uint32_t seg_count[kSegments];
    double wave_weight[kFilterWaves];
    uint32_t wave_count[kFilterWaves];
    uint32_t chunk[kFilterWaves];             // entries of a value
    uint32_t place[2], nth[2];                // the cut's value (nth 0: all its entries stay) and the token's
    u64 occurs[kFilterWaves], above[kFilterWaves];
    uint32_t counted, summed;
    int index;
};

struct Value {                                // the n-th of `all` entries of one value in a row
    uint32_t bits;                            // as in memory; zero: both
    uint32_t nth, all;
    double weight;                            // of the entries up to and including it
};

// Running sum over the wave by moves between lanes, as wave_inclusive_sum.
__device__ __forceinline__ uint32_t wave_inclusive_count(uint32_t v)
{
#define SPECGBV_COUNT_STEP(CTRL, ROW_MASK) \
    v += static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, ROW_MASK, 0xf, false))
    SPECGBV_COUNT_STEP(0x111, 0xf);
    SPECGBV_COUNT_STEP(0x112, 0xf);
    SPECGBV_COUNT_STEP(0x114, 0xf);
    SPECGBV_COUNT_STEP(0x118, 0xf);
    SPECGBV_COUNT_STEP(0x142, 0xa);
    SPECGBV_COUNT_STEP(0x143, 0xc);
#undef SPECGBV_COUNT_STEP
    return v;
}

__device__ __forceinline__ u64 lane_bits_of(u64 v, int src)
{
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(v), src), hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(v >> 32), src);
    return static_cast<u64>(hi) << 32 | lo;
}

template <int NV>
__global__ void __launch_bounds__(kFilterThreads) k_filter_counts(FilterProblem p)
{
    __shared__ union { CountShared c; FilterShared f; } shared;
    __shared__ uint32_t again[kMaxTurns / 32];                     // rows of this workgroup whose counts overflowed
    CountShared &sh = shared.c;
    constexpr bool kAhead = NV <= 8;          // the next row is loaded while this one is worked on
    constexpr bool kMayOverflow = NV > 8;     // shorter rows hold fewer than 2^16 entries
    int tid = threadIdx.x;
    const int V = p.V;
    const uint16_t *logits = static_cast<const uint16_t *>(p.logits);

    // vector j of a row: entries 8 j - lead to 8 j - lead + 7, from the 16-byte boundary in front of it on
    auto lead_of = [&](int r) { return static_cast<int>((reinterpret_cast<uintptr_t>(logits + r * p.row_stride) & 15) / 2); };
    // (a wave's vectors are adjacent, so that entries of lower indices are in lower waves)
    auto per_thread = [&](int lead) { return (lead + V + 8 * kFilterThreads - 1) / (8 * kFilterThreads); };
    auto load = [&](int r, U4 (&x)[NV]) {
        const int lead = lead_of(r), last = (lead + V - 1) / 8, j0 = (tid >> 6) * per_thread(lead) * 64 + (tid & 63);
        const U4 *vec = reinterpret_cast<const U4 *>(logits + r * p.row_stride - lead);
#pragma unroll
        for (int v = 0; v < NV; ++v) x[v] = vec[min(j0 + v * 64, last)];
    };
    auto clear = [&]() {
        U4 *c = reinterpret_cast<U4 *>(sh.count);
#pragma unroll
        for (int i = 0; i < (1 << 13) / kFilterThreads; ++i) c[i * kFilterThreads + tid] = U4{0, 0, 0, 0};
    };

    U4 row[NV], next[kAhead ? NV : 1];
    int r = blockIdx.x, nth_row = 0;
    if (r >= p.rows) return;
    if (tid < kMaxTurns / 32) again[tid] = 0;
    load(r, row);
    clear();
    if (tid == 0) { sh.counted = 0; sh.summed = 0; }
    sh.seg_weight[tid] = 0.0;
    sh.seg_count[tid] = 0;
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
            const U4 x = row[v];
            const bool some = j0 + 64 * v < vectors &&
                              ((x.x ^ kNegInf2) | (x.y ^ kNegInf2) | (x.z ^ kNegInf2) | (x.w ^ kNegInf2)) != 0;
            counted += __popcll(__ballot(some));
            if (some) {
                const uint32_t *w = &x.x;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    atomicAdd(&sh.count[w[i] & 0x7FFFu], (w[i] << 1 & 0x10000u) + 1u);
                    atomicAdd(&sh.count[w[i] >> 16 & 0x7FFFu], (w[i] >> 15 & 0x10000u) + 1u);
                }
            }
        }
        if (lane == 0) atomicAdd(&sh.counted, 8 * counted);
        if (wave == 0) {                                           // entries in front of the row and behind it are taken out again
            const int i = lane < 8 ? lane - lead : V + lane - 8;   // (those of a vector of eight times -inf were not counted)
            if (lane < 16 && (lane < 8 ? i < 0 : i < 8 * vectors - lead)) {
                const U4 x = reinterpret_cast<const U4 *>(logits + r * p.row_stride - lead)[lane < 8 ? 0 : vectors - 1];
                const uint32_t e = logits[r * p.row_stride + i];
                if (((x.x ^ kNegInf2) | (x.y ^ kNegInf2) | (x.z ^ kNegInf2) | (x.w ^ kNegInf2)) != 0) {
                    atomicSub(&sh.count[e & 0x7FFFu], (e << 1 & 0x10000u) + 1u);
                    atomicSub(&sh.counted, 1u);
                }
            }
        }
        __syncthreads();

        // ---- which magnitudes occur: 32 a thread, its eight vectors in an order in which neighbours meet no bank twice
        auto split = [&](int m, uint32_t &pos, uint32_t &neg) {
            const uint32_t d = sh.count[m];
            neg = m == 0 || m >= 0x7F80 ? 0u : d >> 16;            // (both zeros are one value; -inf and what is no number do not take part)
            pos = m > 0x7F80 ? 0u : (m == 0x7F80 ? (d & 0xFFFFu) - (d >> 16) : (d & 0xFFFFu) - neg);
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
        const u64 occurs = lane < kFilterWaves ? sh.occurs[lane] : 0ull;
        // the largest value: the highest segment with one above zero, else the first below; 0x8000 + magnitude, or 0x7FFF - magnitude
        uint32_t top = 0;
        {
            u64 above = lane < kFilterWaves ? sh.above[lane] : 0ull;
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
        const bool overflow = kMayOverflow && sh.summed != sh.counted;       // uniform
        uint32_t cut_bits = 0xFF7Fu;                               // what is kept: larger values, and this one up to an index
        int cut_index = INT32_MAX, token = -1;
        if (overflow || top == 0) {                                // to be done over at the end, or no entries
            __syncthreads();
            clear();
            if (overflow && tid == 0) again[nth_row / 32] |= 1u << nth_row % 32;
        } else {
            const float top_z = __uint_as_float((top >= 0x8000u ? top - 0x8000u : 0x8000u | (0x7FFFu - top)) << 16);
            const double inv_t = 1.0 / static_cast<double>(asked.temperature), min_w = asked.min_p > 0.0f ? static_cast<double>(asked.min_p) : 0.0;
            auto weight = [&](uint32_t bits) {
                const float z = __uint_as_float(bits << 16);
                return z == top_z ? 1.0 : exp_of((static_cast<double>(z) - static_cast<double>(top_z)) * inv_t);
            };
            // ---- counts and weights of the segments that hold something: segment n is wave n % 16's
#pragma unroll 1
            for (int half = 0; half < 2; ++half) {
                u64 words = __ballot((occurs >> (2 * wave + 32 * half) & 1) != 0);
#pragma unroll 1
                while (words) {
                    const int word = __ffsll(static_cast<long long>(words)) - 1, at = word * 32 + wave + 16 * half;
                    words &= words - 1;
                    uint32_t pos, neg;
                    split(at * 64 + lane, pos, neg);
                    const double wp = weight(at * 64 + lane), wn = weight(0x8000u | (at * 64 + lane));
                    if (!(wp >= min_w)) pos = 0;
                    if (!(wn >= min_w)) neg = 0;
                    const uint32_t cp = wave_inclusive_count(pos), cn = wave_inclusive_count(neg);
                    const double sp = wave_inclusive_sum(pos ? pos * wp : 0.0), sn = wave_inclusive_sum(neg ? neg * wn : 0.0);
                    if (lane == 63) {
                        sh.seg_count[511 - at] = cp; sh.seg_weight[511 - at] = sp;
                        sh.seg_count[512 + at] = cn; sh.seg_weight[512 + at] = sn;
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
                const double block_w = wave_inclusive_sum(lane < kFilterWaves ? sh.wave_weight[lane & 15] : 0.0);
                const uint32_t block_c = wave_inclusive_count(lane < kFilterWaves ? sh.wave_count[lane & 15] : 0u);
                const uint32_t all = __builtin_amdgcn_readlane(block_c, 63);
                double total = lane_value(block_w, 63);

                // the first place whose count (how 0) or weight (1) reaches the goal, or whose weight exceeds it (2)
                auto locate = [&](int how, double goal) {
                    // the first of 64 running sums to reach it; where rounding leaves none, the last that holds something
                    auto first = [&](uint32_t c, double w, bool holds) {
                        const u64 hit = __ballot(holds && (how == 0 ? c >= goal : (how == 1 ? w >= goal : w > goal))), some = __ballot(holds);
                        return hit ? __ffsll(static_cast<long long>(hit)) - 1 : 63 - __clzll(static_cast<long long>(some | 1));
                    };
                    const int block = first(block_c, block_w, lane < kFilterWaves && sh.wave_count[lane & 15] != 0);
                    double w0 = block ? lane_value(block_w, block - 1) : 0.0;
                    uint32_t c0 = block ? __builtin_amdgcn_readlane(block_c, block - 1) : 0u;
                    const double seg_w = sh.seg_weight[block * 64 + lane];
                    const uint32_t seg_c = sh.seg_count[block * 64 + lane], seg_before = lane ? sh.seg_count[block * 64 + lane - 1] : 0u;
                    const int seg = first(c0 + seg_c, w0 + seg_w, seg_c != seg_before), o = block * 64 + seg;
                    if (seg) { w0 += lane_value(seg_w, seg - 1); c0 += __builtin_amdgcn_readlane(seg_c, seg - 1); }
                    const bool minus = o >= 512;
                    const int at = minus ? o - 512 : 511 - o, m = at * 64 + (minus ? lane : 63 - lane);
                    uint32_t pos, neg;
                    split(m, pos, neg);
                    uint32_t n = minus ? neg : pos;
                    const uint32_t bits = (minus ? 0x8000u : 0u) | m;
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
                    const int i0 = 8 * (j1 + 64 * v) - lead;
                    if (i0 < 0) m &= 0xFFu << -i0;
                    if (i0 + 8 > V) m &= i0 < V ? 0xFFu >> (i0 + 8 - V) : 0u;
                    return m;
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
                const uint32_t before = wave_inclusive_count(lane < wave ? sh.chunk[lane & 15] : 0u), here = sh.chunk[wave];
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
        if (tid == 0) { sh.counted = 0; sh.summed = 0; }
        if constexpr (kAhead) {
#pragma unroll
            for (int v = 0; v < NV; ++v) row[v] = next[v];
        }
        __syncthreads();
    }
    __syncthreads();
    for (int i = 0; i <= nth_row; ++i)
        if (again[i / 32] >> i % 32 & 1) {                         // uniform
            filter_row<uint16_t>(p, blockIdx.x + i * gridDim.x, shared.f);
            __syncthreads();
        }
}

template <int NV>
hipError_t launch_counts(const FilterProblem &p, hipStream_t stream)
{
    const int units = NV <= 8 ? compute_units() : p.rows, least = (p.rows + kMaxTurns - 1) / kMaxTurns, most = units > least ? units : least;
    hipLaunchKernelGGL((k_filter_counts<NV>), dim3(p.rows < most ? p.rows : most), dim3(kFilterThreads), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_filter(const FilterProblem &p, int dtype, hipStream_t stream)
{
    const int64_t span = static_cast<int64_t>(p.V) + 7;            // entries with those in front of the row's first vector
    if (dtype == 1 && span <= 8192) return launch_counts<1>(p, stream);
    if (dtype == 1 && span <= 4 * 8192) return launch_counts<4>(p, stream);
    if (dtype == 1 && span <= 8 * 8192) return launch_counts<8>(p, stream);
    if (dtype == 1 && span <= 16 * 8192) return launch_counts<16>(p, stream);
    if (dtype == 1 && span <= 20 * 8192) return launch_counts<20>(p, stream);
    if (dtype == 1) hipLaunchKernelGGL((k_filter<uint16_t>), dim3(p.rows), dim3(kFilterThreads), 0, stream, p);
    else hipLaunchKernelGGL((k_filter<float>), dim3(p.rows), dim3(kFilterThreads), 0, stream, p);
    return hipGetLastError();
}

}  // namespace specgbv
