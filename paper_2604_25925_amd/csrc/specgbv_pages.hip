// Block tables on the GPU: pages given back, taken and handed on as the texts of a batch of requests grow, end and begin; and where new tokens lie.
//
// The free pages stand in a ring: `count` of them from `head` on.  A request (a prefix with K drafts) has the pages of its whole part once, for all
// its drafts, and behind them pages of each draft's own.  Per request, with (w, h) pages so far (w shared, h in all) and (w', h') wanted, the chosen draft
// has [0, h) and wants [0, h'), another one has [w, h) and wants [w', h'); what it has and does not want is given back, what it wants and
// has not is taken, and the entries [w, w') of the others become the chosen draft's.  Pages given back go behind the ring's last in a set order, then
// pages are taken from its front in the same order (requests, in each the chosen draft first, then by page), so a call's result does not hang on
// which workgroup comes first: every page's place follows from sums over the requests in front.
//
// A request that needs more pages than it gives back is served if there are enough for it and those in front of it; a request that is not served
// keeps what it has.  All numbers are whole and of 32 bits (rows x width is at most 2^30).
//
// Latency bounds it: sums over the requests, then a read and a write of a few entries each.  Small tables: one workgroup does all of it, with
// the sums in LDS and its threads dealt out over all entries that change (32 requests of 8 drafts, 130 pages wide: 8.0 us, of which its arithmetic takes 0.6 for each 1024 entries
// that change).  Larger ones: a launch for the sums (5.6 us for 1000 requests of 4 drafts) and one each for giving and taking (3.3 and 3.7).
#include "specgbv_internal.hpp"

namespace specgbv {
namespace {

constexpr int kPlanThreads = 1024, kMoveThreads = 256;
constexpr int kSmallRows = 1024;              // and so at most as many requests, one a thread

// What a request has and gets; gives / takes: in front of it in the batch.
struct alignas(16) Request {
    int32_t whole0, held0, whole1, held1;
    int32_t chosen, served;                   // served: 1, 0 (not enough pages) or -1 (longer than the table)
    int32_t gives, takes;
};
struct Totals { int32_t head, count, gives, takes; };

__device__ __forceinline__ int least(int a, int b) { return a < b ? a : b; }
__device__ __forceinline__ int over0(int x) { return x > 0 ? x : 0; }

// Two ranges of entries one after the other, of a row of a request.
struct Ranges {
    int a0, an, b0, bn;
    __device__ __forceinline__ int size() const { return an + bn; }
    __device__ __forceinline__ int entry(int i) const { return i < an ? a0 + i : b0 + (i - an); }
};
__device__ __forceinline__ Ranges given_by_chosen(const Request &q) { return {q.held1, over0(q.held0 - q.held1), 0, 0}; }
__device__ __forceinline__ Ranges given_by_other(const Request &q)
{
    const int from = max(q.whole0, q.held1);
    return {q.whole0, over0(least(q.held0, q.whole1) - q.whole0), from, over0(q.held0 - from)};
}
__device__ __forceinline__ Ranges taken_by_chosen(const Request &q) { return {q.held0, over0(q.held1 - q.held0), 0, 0}; }
__device__ __forceinline__ Ranges taken_by_other(const Request &q)
{
    const int from = max(q.whole1, q.held0);
    return {q.whole1, over0(least(q.held1, q.whole0) - q.whole1), from, over0(q.held1 - from)};
}
// Entries that become empty without being given back: shared ones, in the rows of the drafts that were not chosen.
__device__ __forceinline__ Ranges cleared(const Request &q) { return {q.held1, over0(q.whole0 - q.held1), 0, 0}; }
// Entries that become the chosen draft's.
__device__ __forceinline__ Ranges adopted(const Request &q) { return {q.whole0, over0(q.whole1 - q.whole0), 0, 0}; }

__device__ __forceinline__ int clamped(int x, int lo, int hi) { return max(lo, min(x, hi)); }

__device__ __forceinline__ Request request_of(const PagesProblem &p, int b)
{
    Request q{};
    q.held0 = clamped(p.held[2 * b + 1], 0, p.width);
    q.whole0 = clamped(p.held[2 * b], 0, q.held0);
    q.chosen = p.chosen ? clamped(p.chosen[b], 0, p.drafts - 1) : 0;
    const int length = p.length[b];
    q.served = 1;
    if (length > 0) {
        const int64_t held = (static_cast<int64_t>(length) + p.room + p.by_page.d - 1) / p.by_page.d;
        if (held > p.width) q.served = -1;
        else { q.held1 = static_cast<int>(held); q.whole1 = p.by_page.div(length); }
    }
    if (q.served < 0) { q.whole1 = q.whole0; q.held1 = q.held0; }
    return q;
}
__device__ __forceinline__ int gives_of(const Request &q, int drafts) { return given_by_chosen(q).size() + (drafts - 1) * given_by_other(q).size(); }
__device__ __forceinline__ int takes_of(const Request &q, int drafts) { return taken_by_chosen(q).size() + (drafts - 1) * taken_by_other(q).size(); }

// Sum over the threads in front of this one, itself included; `total`: over all.  (Two barriers.)
__device__ __forceinline__ int sum_in_front(int x, int *sh, int &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    int run = static_cast<int>(wave_inclusive_count(static_cast<uint32_t>(x)));
    if (lane == 63) sh[wave] = run;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < waves; ++w) {
        const int v = sh[w];
        before += w < wave ? v : 0;
        all += v;
    }
    __syncthreads();
    total = all;
    return run + before;
}

__device__ __forceinline__ int at_ring(int i, int pages) { return i % pages; }

// The requests of a batch in their order, kPlanThreads at a time: `put` gets each.
template <typename Put>
__device__ __forceinline__ Totals plan_all(const PagesProblem &p, Put &&put)
{
    __shared__ int sh[kPlanThreads / 64];
    Totals t;
    t.head = clamped(p.ends[0], 0, p.pages - 1);
    t.count = clamped(p.ends[1], 0, p.pages);
    t.gives = t.takes = 0;
    int64_t free_pages = t.count;
    for (int b0 = 0; b0 < p.prefixes; b0 += blockDim.x) {              // what those give back that need no more than that
        const int b = b0 + threadIdx.x;
        int back = 0, all;
        if (b < p.prefixes) {
            const Request q = request_of(p, b);
            back = over0(gives_of(q, p.drafts) - takes_of(q, p.drafts));
        }
        sum_in_front(back, sh, all);
        free_pages += all;
    }
    int64_t needed = 0;
    for (int b0 = 0; b0 < p.prefixes; b0 += blockDim.x) {
        const int b = b0 + threadIdx.x;
        Request q{};
        int more = 0, all, gives = 0, takes = 0;
        if (b < p.prefixes) {
            q = request_of(p, b);
            gives = gives_of(q, p.drafts); takes = takes_of(q, p.drafts);
            more = over0(takes - gives);
        }
        const int run = sum_in_front(more, sh, all);
        if (more > 0 && needed + run > free_pages) {
            q.served = 0; q.whole1 = q.whole0; q.held1 = q.held0;
            gives = takes = 0;
        }
        needed += all;
        int all_gives, all_takes;
        const int g = sum_in_front(gives, sh, all_gives), k = sum_in_front(takes, sh, all_takes);
        q.gives = t.gives + g - gives; q.takes = t.takes + k - takes;
        if (b < p.prefixes) put(b, q);
        t.gives += all_gives; t.takes += all_takes;
    }
    return t;
}

// The row of a request's i-th draft: the chosen one first.
__device__ __forceinline__ int draft_at(const Request &q, int i) { return i == 0 ? q.chosen : (i <= q.chosen ? i - 1 : i); }

__device__ __forceinline__ int32_t *row_of(const PagesProblem &p, int b, int draft) { return p.table + (static_cast<int64_t>(b) * p.drafts + draft) * p.table_stride; }

// Entries of a request that are given back or cleared, and that are taken or adopted: how many, and what becomes of the i-th.
__device__ __forceinline__ int clearing_of(const Request &q, int drafts) { return given_by_chosen(q).size() + (drafts - 1) * (given_by_other(q).size() + cleared(q).size()); }
__device__ __forceinline__ int filling_of(const Request &q, int drafts) { return taken_by_chosen(q).size() + (drafts - 1) * (taken_by_other(q).size() + adopted(q).size()); }

__device__ __forceinline__ void clear_entry(const PagesProblem &p, const Totals &t, int b, const Request &q, int i)
{
    const Ranges first = given_by_chosen(q), other = given_by_other(q), empty = cleared(q);
    int draft = 0, n = i, place = 0;
    bool back = true;
    Ranges r = first;
    if (n >= first.size()) {
        n -= first.size();
        const int each = other.size() + empty.size();
        draft = 1 + n / each;
        n -= (draft - 1) * each;
        back = n < other.size();
        place = first.size() + (draft - 1) * other.size() + n;
        if (back) r = other;
        else { r = empty; n -= other.size(); }
    } else place = n;
    const int e = r.entry(n);
    int32_t *at = row_of(p, b, draft_at(q, draft)) + e;
    if (back) p.ring[at_ring(at_ring(t.head + t.count, p.pages) + at_ring(q.gives + place, p.pages), p.pages)] = *at;
    if (e >= q.held1) *at = -1;
}

__device__ __forceinline__ void fill_entry(const PagesProblem &p, const Totals &t, int b, const Request &q, int i)
{
    const Ranges first = taken_by_chosen(q), other = taken_by_other(q), handed = adopted(q);
    int draft = 0, n = i, place = i;
    bool take = true;
    Ranges r = first;
    if (n >= first.size()) {
        n -= first.size();
        const int each = other.size() + handed.size();
        draft = 1 + n / each;
        n -= (draft - 1) * each;
        take = n < other.size();
        place = first.size() + (draft - 1) * other.size() + n;
        if (take) r = other;
        else { r = handed; n -= other.size(); }
    }
    const int e = r.entry(n);
    if (!take) place = e - q.held0;                                    // among those that the chosen draft takes, where it had none
    int page;
    if (take || e >= q.held0) page = p.ring[at_ring(t.head + at_ring(q.takes + place, p.pages), p.pages)];
    else page = row_of(p, b, q.chosen)[e];
    row_of(p, b, draft_at(q, draft))[e] = page;
}

__device__ __forceinline__ void finish(const PagesProblem &p, int b, const Request &q)
{
    p.served[b] = q.served;
    p.shared_len[b] = q.whole1 * static_cast<int>(p.by_page.d);
    if (q.served > 0) { p.held[2 * b] = q.whole1; p.held[2 * b + 1] = q.held1; }
}
__device__ __forceinline__ void finish_ends(const PagesProblem &p, const Totals &t)
{
    p.ends[0] = at_ring(t.head + at_ring(t.takes, p.pages), p.pages);
    p.ends[1] = clamped(t.count + t.gives - t.takes, 0, p.pages);
}

// The last request whose entries begin at i or in front of it.
__device__ __forceinline__ int request_at(const int *begins, int n, int i)
{
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (begins[mid] <= i) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// All of it by one workgroup, for up to kSmallRows requests.
__global__ void __launch_bounds__(kPlanThreads) k_pages_small(PagesProblem p)
{
    __shared__ Request sh_request[kSmallRows];
    __shared__ int sh_clear[kSmallRows], sh_fill[kSmallRows], sh_sum[kPlanThreads / 64];
    const int tid = threadIdx.x;
    const Totals t = plan_all(p, [&](int b, const Request &q) { sh_request[b] = q; });
    __syncthreads();
    int clearing = 0, filling = 0, all_clearing, all_filling;
    if (tid < p.prefixes) {
        clearing = clearing_of(sh_request[tid], p.drafts);
        filling = filling_of(sh_request[tid], p.drafts);
    }
    const int c = sum_in_front(clearing, sh_sum, all_clearing), f = sum_in_front(filling, sh_sum, all_filling);
    if (tid < p.prefixes) { sh_clear[tid] = c - clearing; sh_fill[tid] = f - filling; }
    __syncthreads();
    for (int i = tid; i < all_clearing; i += kPlanThreads) {
        const int b = request_at(sh_clear, p.prefixes, i);
        clear_entry(p, t, b, sh_request[b], i - sh_clear[b]);
    }
    __syncthreads();                                                   // (what was given back is there for the workgroup)
    for (int i = tid; i < all_filling; i += kPlanThreads) {
        const int b = request_at(sh_fill, p.prefixes, i);
        fill_entry(p, t, b, sh_request[b], i - sh_fill[b]);
    }
    if (tid < p.prefixes) finish(p, tid, sh_request[tid]);
    if (tid == 0) finish_ends(p, t);
}

__global__ void __launch_bounds__(kPlanThreads) k_pages_plan(PagesProblem p)
{
    Request *requests = reinterpret_cast<Request *>(static_cast<char *>(p.plan) + 256);
    const Totals t = plan_all(p, [&](int b, const Request &q) { requests[b] = q; });
    if (threadIdx.x == 0) *static_cast<Totals *>(p.plan) = t;
}

template <bool FILL>
__global__ void __launch_bounds__(kMoveThreads) k_pages_move(PagesProblem p)
{
    const int b = blockIdx.x, step = gridDim.y * kMoveThreads;
    const Request q = reinterpret_cast<const Request *>(static_cast<const char *>(p.plan) + 256)[b];
    const Totals t = *static_cast<const Totals *>(p.plan);
    const int n = FILL ? filling_of(q, p.drafts) : clearing_of(q, p.drafts);
    for (int i = blockIdx.y * kMoveThreads + threadIdx.x; i < n; i += step) {
        if (FILL) fill_entry(p, t, b, q, i);
        else clear_entry(p, t, b, q, i);
    }
    if (FILL && blockIdx.y == 0 && threadIdx.x == 0) {
        finish(p, b, q);
        if (b == 0) finish_ends(p, t);
    }
}

// Positions and places of new tokens, a thread each; 4 + 8 bytes are written a token, and latency bounds it (2.8 us for 256 rows of 24 tokens and 3.1 for 64 of 4001).
__global__ void __launch_bounds__(kMoveThreads) k_slots(SlotsProblem p)
{
    const int64_t all = static_cast<int64_t>(blockIdx.x) * kMoveThreads + threadIdx.x;
    if (all >= static_cast<int64_t>(p.sequences) * p.tokens) return;
    const int item = static_cast<int>(all), s = p.by_tokens.div(item), t = p.by_tokens.mod(item, s), b = p.by_drafts.div(s);
    const int count = clamped(p.count[b], 0, p.tokens), i = p.right ? t - (p.tokens - count) : t;
    int64_t pos = -1;
    if (i >= 0 && i < count) pos = static_cast<int64_t>(p.start[b]) + i;
    if (pos < 0 || pos > INT32_MAX) pos = -1;
    p.positions[s * p.positions_stride + t] = static_cast<int32_t>(pos);
    if (!p.slots) return;
    Place at{-1, 0};
    if (pos >= 0) at = place_of(p.map, s, static_cast<int32_t>(pos));
    p.slots[s * p.slots_stride + t] = at.page < 0 ? -1 : static_cast<int64_t>(at.page) * p.map.page.d + at.slot;
}

// One workgroup's turns over the entries against two more launches.  One / three launches, us, in a graph: where few entries change, as between steps, 6.9 / 7.7 for a request of 8 drafts,
// 8.1 / 8.7 for 32, 8.7 / 8.9 for 128, but 11.5 / 9.9 for 512 and 15.5 / 11.0 for 1024; 8.7 / 9.9 for 1024 without drafts; called one by one, where the host's launches count,
// 11 / 17 for 32.  Where all entries change, as when a batch begins, 8.6 / 8.4 at 4096 of them, 22 / 9.2 at 33280 and 40 / 10 at 65536: which a batch's later steps bring back.
bool small_table(int prefixes, int drafts, int width)
{
    const int64_t rows = static_cast<int64_t>(prefixes) * drafts;
    return rows <= kSmallRows && rows * width <= (1 << 16);
}

}  // namespace

size_t pages_bytes(int prefixes, int drafts, int width)
{
    return small_table(prefixes, drafts, width) ? 0 : 256 + static_cast<size_t>(prefixes) * sizeof(Request);
}

hipError_t launch_pages(const PagesProblem &p, hipStream_t stream)
{
    if (small_table(p.prefixes, p.drafts, p.width)) {
        hipLaunchKernelGGL(k_pages_small, dim3(1), dim3(kPlanThreads), 0, stream, p);
        return hipGetLastError();
    }
    const int64_t entries = static_cast<int64_t>(p.drafts) * p.width;
    int64_t slices = entries / 4096 + 1;
    if (slices > 64) slices = 64;
    if (p.prefixes * slices >= kLaunchGroups) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(k_pages_plan, dim3(1), dim3(kPlanThreads), 0, stream, p);
    hipLaunchKernelGGL((k_pages_move<false>), dim3(p.prefixes, static_cast<unsigned>(slices)), dim3(kMoveThreads), 0, stream, p);
    hipLaunchKernelGGL((k_pages_move<true>), dim3(p.prefixes, static_cast<unsigned>(slices)), dim3(kMoveThreads), 0, stream, p);
    return hipGetLastError();
}

hipError_t launch_slots(const SlotsProblem &p, hipStream_t stream)
{
    const int64_t grid = (static_cast<int64_t>(p.sequences) * p.tokens + kMoveThreads - 1) / kMoveThreads;
    if (grid >= kLaunchGroups) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(k_slots, dim3(static_cast<unsigned>(grid)), dim3(kMoveThreads), 0, stream, p);
    return hipGetLastError();
}

}  // namespace specgbv
