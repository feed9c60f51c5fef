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

struct RowRule {                              // how a row's entries are weighed and binned
    float top;                                // its largest logit
    double inv_t;
    float bins;                               // bins per unit of the logit
    uint32_t least;                           // entries of lower keys do not take part

    __device__ __forceinline__ double weight(float z) const
    {
        if (z == top) return 1.0;
        return exp((static_cast<double>(z) - static_cast<double>(top)) * inv_t);
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

template <typename T>
__global__ void __launch_bounds__(kFilterThreads) k_filter(FilterProblem p)
{
    __shared__ FilterShared sh;
    const int tid = threadIdx.x;
    const T *row = static_cast<const T *>(p.logits) + blockIdx.x * p.row_stride;
    const int V = p.V;

    float temperature = p.temperature ? p.temperature[blockIdx.x] : 1.0f;
    int64_t k = p.top_k && p.top_k[blockIdx.x] > 0 ? p.top_k[blockIdx.x] : INT64_MAX;
    const float top_p = p.top_p ? p.top_p[blockIdx.x] : 1.0f;
    const float min_p = p.min_p ? fminf(p.min_p[blockIdx.x], 1.0f) : 0.0f;
    if (!(temperature > 0.0f)) { temperature = 1.0f; k = 1; }

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
        if (k < static_cast<int64_t>(sh.count[kBins - 1])) {
            const Found f = find_place(sh, row, V, rule, true, static_cast<u64>(k));
            cut_key = f.key; cut_index = f.index; total = f.weight;
        }
        if (top_p < 1.0f) {
            const double goal = ceil(static_cast<double>(top_p) * static_cast<double>(total));
            const Found f = find_place(sh, row, V, rule, false, goal < 1.0 ? 1 : min(static_cast<u64>(goal), total));
            cut_key = f.key; cut_index = f.index; total = f.weight;
        }
        if (p.out_tokens) {
            const double goal = static_cast<double>(p.u[blockIdx.x]) * static_cast<double>(total);
            token = find_place(sh, row, V, rule, false, goal >= 0.0 ? (goal < static_cast<double>(total) ? min(static_cast<u64>(goal) + 1, total) : total) : 1).index;
        }
    }
    if (p.out_tokens && tid == 0) p.out_tokens[blockIdx.x] = token;
    if (!p.kept) return;
    T *kept = static_cast<T *>(p.kept) + blockIdx.x * p.kept_stride;
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

}  // namespace

hipError_t launch_filter(const FilterProblem &p, int dtype, hipStream_t stream)
{
    if (dtype == 1) hipLaunchKernelGGL((k_filter<uint16_t>), dim3(p.rows), dim3(kFilterThreads), 0, stream, p);
    else hipLaunchKernelGGL((k_filter<float>), dim3(p.rows), dim3(kFilterThreads), 0, stream, p);
    return hipGetLastError();
}

}  // namespace specgbv
