// What the kernels of attention over a paged cache have in common: the division of units into parts, stores of results, and the join of parts.
#pragma once

#include "specgbv_internal.hpp"

namespace specgbv {
namespace {

typedef float F4 __attribute__((ext_vector_type(4)));
typedef __bf16 B8 __attribute__((ext_vector_type(8)));
typedef __bf16 B2 __attribute__((ext_vector_type(2)));

constexpr int kAttendThreads = 256, kWavesPerGroup = 4;

constexpr float kRaise = 8.0f;                // a reference is raised where a score is this far above it
constexpr int kMaxParts = 256;                // partial sums of a row at most: a workgroup's threads

template <typename T> __device__ __forceinline__ T rounded(float x);
template <> __device__ __forceinline__ float rounded<float>(float x) { return x; }
template <> __device__ __forceinline__ uint16_t rounded<uint16_t>(float x) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x)); }

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }      // (2^-126 and below: 0)

// Over the 16 rows of a wave, which its four quarters hold alike: by moves between the lanes of a quarter.
__device__ __forceinline__ int rows_least(int x)
{
    x = min(x, __builtin_amdgcn_update_dpp(x, x, 0x111, 0xf, 0xf, false));
    x = min(x, __builtin_amdgcn_update_dpp(x, x, 0x112, 0xf, 0xf, false));
    x = min(x, __builtin_amdgcn_update_dpp(x, x, 0x114, 0xf, 0xf, false));
    x = min(x, __builtin_amdgcn_update_dpp(x, x, 0x118, 0xf, 0xf, false));
    return __builtin_amdgcn_readlane(x, 15);
}
__device__ __forceinline__ int rows_most(int x) { return ~rows_least(~x); }

// Largest and sum over the four lanes of a row (l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float row_largest(float x) { x = fmaxf(x, __shfl_xor(x, 16, 64)); return fmaxf(x, __shfl_xor(x, 32, 64)); }
__device__ __forceinline__ float row_total(float x) { x += __shfl_xor(x, 16, 64); return x + __shfl_xor(x, 32, 64); }

// A sequence's row of the table through scalar loads: it is read by whole waves, and nothing in the kernel writes it.
typedef const int32_t __attribute__((address_space(4))) *ConstTable;

// Which part of which unit (a sequence, or a prefix with its drafts) a workgroup has, and how many parts the unit is in.
struct Share { int unit, part, parts, at, length; };          // at: place of the unit's first part among all; length: keys of a part

// Units differ in length, and a launch lasts as long as its last workgroup.  So every workgroup looks at all units' lengths (one a lane)
// and takes its part of a division into equal lengths, the shortest for which all workgroups fit onto the card at once.  With more units
// than lanes each is cut into the same number of parts.
__device__ __forceinline__ Share share_of(const AttendProblem &p, int index, int held, int lane)
{
    if (!p.balanced) {
        const int unit = p.by_chunks.div(index);
        if (unit >= p.units) return Share{-1, 0, 0, 0, 0};
        return Share{unit, p.by_chunks.mod(index, unit), p.chunks, unit * p.chunks, p.chunk_keys};
    }
    int length = 0;
    if (lane < p.units) {
        if (p.shared_len) length = max(0, min(p.shared_len[lane], held));
        else
            for (int t = 0; t < p.tokens; ++t) length = max(length, min(p.positions[lane * p.positions_stride + t], held - 1) + 1);
        if (p.window > 0) length = min(length, min(p.window, held) + p.tokens);
        length = max(length + p.own_keys, 1);
    }
    // (in two halves, as whole numbers: exact, and by moves between lanes where a sum of float64 goes through LDS)
    const uint32_t low = __builtin_amdgcn_readlane(wave_inclusive_count(length & 0xFFFF), 63), high = __builtin_amdgcn_readlane(wave_inclusive_count(length >> 16), 63);
    const double all = high * 65536.0 + low;
    int part = static_cast<int>(all / p.most_parts) / p.grain * p.grain + p.grain;            // at most most_parts + units parts
    part = max(part, p.chunk_keys);
    uint32_t n = 0, run = 0;
    for (int i = 0; i < 8; ++i) {
        n = (static_cast<uint32_t>(length) + static_cast<uint32_t>(part) - 1u) / static_cast<uint32_t>(part);
        run = wave_inclusive_count(n);
        if (__builtin_amdgcn_readlane(run, 63) <= static_cast<uint32_t>(p.most_parts)) break;
        part += (part / 8 + p.grain - 1) / p.grain * p.grain;
    }
    const unsigned long long above = __ballot(run > static_cast<uint32_t>(index));
    if (above == 0) return Share{-1, 0, 0, 0, 0};
    const int unit = __ffsll(static_cast<long long>(above)) - 1;
    const int parts = __builtin_amdgcn_readlane(n, unit), at = __builtin_amdgcn_readlane(run, unit) - parts;
    return Share{unit, index - at, parts, at, part};
}

// Four entries of a result, over the sum of weights (inv 0: there is none, and the result is 0).
template <typename T> __device__ __forceinline__ void store_entries(T *dst, F4 v, float inv, int wide)
{
    struct alignas(4 * sizeof(T)) Vec { T e[4]; } o;
#pragma unroll
    for (int j = 0; j < 4; ++j) o.e[j] = rounded<T>(inv == 0.0f ? 0.0f : v[j] * inv);
    if (wide) *reinterpret_cast<Vec *>(dst) = o;
    else
#pragma unroll
        for (int j = 0; j < 4; ++j) dst[j] = o.e[j];
}

// The place of a row of the result and of its parts.
struct JoinRow {
    int draft, s, t, h, parts;
    int64_t part0, between;

    __device__ __forceinline__ JoinRow(const AttendProblem &p, int at)
    {
        const int rows = p.tokens * p.group * p.drafts, pair = p.by_rows.div(at), row = p.by_rows.mod(at, pair);
        const int unit = p.by_kv_heads.div(pair), head0 = p.by_kv_heads.mod(pair, unit);
        draft = p.by_in_draft.div(row);
        const int in = p.by_in_draft.mod(row, draft);
        s = unit * p.drafts + draft; t = p.by_group.div(in); h = head0 * p.group + p.by_group.mod(in, t);
        const int2 where = p.balanced ? p.places[unit] : make_int2(unit * p.chunks, p.chunks);
        parts = where.y;
        part0 = (static_cast<int64_t>(where.x) * p.kv_heads + head0) * rows + row;
        between = static_cast<int64_t>(p.kv_heads) * rows;
    }
};

// Entry of a row that vector `vec` of its partial sums starts with; VEC: adjacent entries of a value that a lane took.
template <int VEC> __device__ __forceinline__ int entry_at(const AttendProblem &p, int vec)
{
    const int quad = vec & 3, piece = vec >> 2, n = piece % (VEC / 4), gi = piece / (VEC / 4), i = gi & 3, g = gi >> 2;
    return p.in_order ? 4 * vec : (16 * g + 4 * quad + i) * VEC + 4 * n;
}

// The parts of a row joined by DP / 4 lanes, each with a vector of its entries: several rows per wave, so that all are on their way at once.
template <typename T, int DP, int VEC>
__global__ void __launch_bounds__(kAttendThreads) k_attend_join(AttendProblem p)
{
    constexpr int kLanes = DP / 4, kAhead = 4;
    const int vec = threadIdx.x % kLanes;
    const int at = blockIdx.x * (kAttendThreads / kLanes) + threadIdx.x / kLanes;     // (fewer than 2^30 rows)
    if (at >= p.sequences * p.heads * p.tokens) return;                               // whole groups of lanes
    const JoinRow row(p, at);
    const int pos = p.positions[row.s * p.positions_stride + row.t];
    const F4 *acc_of = reinterpret_cast<const F4 *>(p.acc) + vec;

    // the first parts' sums are on their way while the references of all parts are looked at
    F4 v[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) v[i] = acc_of[(row.part0 + min(i, row.parts - 1) * row.between) * (DP / 4)];
    float most = -INFINITY;
    for (int c = vec; c < row.parts; c += kLanes) {
        const float2 ml = p.ml[row.part0 + c * row.between];
        if (ml.y != 0.0f) most = fmaxf(most, ml.x);                                    // (a sum that is no number goes on)
    }
#pragma unroll
    for (int m = kLanes / 2; m > 0; m >>= 1) most = fmaxf(most, __shfl_xor(most, m, 64));
    F4 acc{0, 0, 0, 0};
    float total = 0.0f;
    for (int c0 = 0; c0 < row.parts; c0 += kAhead) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int c = c0 + i;
            if (c >= row.parts) break;
            const float2 ml = p.ml[row.part0 + c * row.between];
            if (ml.y != 0.0f) {                                                        // else there is nothing to read
                const float f = ml.x == most ? 1.0f : exp2_of(ml.x - most);
                total += ml.y * f;
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] += v[i][e] * f;
            }
            if (c + kAhead < row.parts) v[i] = acc_of[(row.part0 + (c + kAhead) * row.between) * (DP / 4)];
        }
    }
    const int d = entry_at<VEC>(p, vec);
    if (d >= p.head_dim) return;
    const float inv = pos >= 0 && total != 0.0f ? 1.0f / total : 0.0f;
    store_entries(static_cast<T *>(p.out) + row.s * p.out_stride[0] + row.t * p.out_stride[1] + row.h * p.out_stride[2] + d, acc, inv, p.out_wide);
}

// The same by a workgroup per row, for many parts: 4096 / DP of them at once.
template <typename T, int DP, int VEC>
__global__ void __launch_bounds__(kAttendThreads) k_attend_join_many(AttendProblem p)
{
    constexpr int kLanes = DP / 4, kSets = kAttendThreads / kLanes, kAhead = 4;
    __shared__ float sh_f[kMaxParts];
    __shared__ float sh_most[kWavesPerGroup], sh_total[kWavesPerGroup];
    __shared__ F4 sh_acc[kWavesPerGroup * kLanes];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, vec = tid % kLanes, set = tid / kLanes;
    const JoinRow row(p, blockIdx.x);
    const F4 *acc_of = reinterpret_cast<const F4 *>(p.acc) + vec;

    F4 v[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) v[i] = acc_of[(row.part0 + min(set + i * kSets, row.parts - 1) * row.between) * (DP / 4)];
    float2 ml{-INFINITY, 0.0f};
    if (tid < row.parts) ml = p.ml[row.part0 + tid * row.between];                     // (parts are at most the threads)
    const int pos = p.positions[row.s * p.positions_stride + row.t];
    const bool some = ml.y != 0.0f;
    float most = some ? ml.x : -INFINITY;
    for (int m = 32; m > 0; m >>= 1) most = fmaxf(most, __shfl_xor(most, m, 64));
    if (lane == 0) sh_most[wave] = most;
    __syncthreads();
    most = fmaxf(fmaxf(sh_most[0], sh_most[1]), fmaxf(sh_most[2], sh_most[3]));
    const float f = !some ? 0.0f : (ml.x == most ? 1.0f : exp2_of(ml.x - most));
    float total = some ? ml.y * f : 0.0f;
    for (int m = 32; m > 0; m >>= 1) total += __shfl_xor(total, m, 64);
    if (lane == 0) sh_total[wave] = total;
    sh_f[tid] = some ? f : -1.0f;                                                      // (-1: there is nothing to read)
    __syncthreads();
    total = (sh_total[0] + sh_total[1]) + (sh_total[2] + sh_total[3]);
    F4 acc{0, 0, 0, 0};
    for (int c0 = set; c0 - set < row.parts; c0 += kAhead * kSets) {                   // the same count for all
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int c = c0 + i * kSets, n = c + kAhead * kSets;
            const float w = c >= row.parts ? -1.0f : sh_f[c];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] += w < 0.0f ? 0.0f : v[i][e] * w;
            if (n < row.parts) v[i] = acc_of[(row.part0 + n * row.between) * (DP / 4)];
        }
    }
#pragma unroll
    for (int m = 32; m >= kLanes; m >>= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], m, 64);
    if (lane < kLanes) sh_acc[wave * kLanes + vec] = acc;
    __syncthreads();
    if (tid >= kLanes) return;
    acc = (sh_acc[vec] + sh_acc[kLanes + vec]) + (sh_acc[2 * kLanes + vec] + sh_acc[3 * kLanes + vec]);
    const int d = entry_at<VEC>(p, vec);
    if (d >= p.head_dim) return;
    const float inv = pos >= 0 && total != 0.0f ? 1.0f / total : 0.0f;
    store_entries(static_cast<T *>(p.out) + row.s * p.out_stride[0] + row.t * p.out_stride[1] + row.h * p.out_stride[2] + d, acc, inv, p.out_wide);
}

// Few parts (8 a unit on average): several rows per wave, so that all rows are on their way at once; many: a workgroup per row, so that
// a row's parts are.
template <int DP> int64_t join_grid(const AttendProblem &p)
{
    const int64_t rows = static_cast<int64_t>(p.sequences) * p.heads * p.tokens, per = p.all_parts <= 8 * p.units ? kAttendThreads / (DP / 4) : 1;
    return (rows + per - 1) / per;
}

template <typename T, int DP, int VEC> hipError_t launch_join(const AttendProblem &p, hipStream_t stream)
{
    const dim3 grid(static_cast<unsigned>(join_grid<DP>(p)));
    if (p.all_parts <= 8 * p.units) hipLaunchKernelGGL((k_attend_join<T, DP, VEC>), grid, dim3(kAttendThreads), 0, stream, p);
    else hipLaunchKernelGGL((k_attend_join_many<T, DP, VEC>), grid, dim3(kAttendThreads), 0, stream, p);
    return hipGetLastError();
}

}  // namespace
}  // namespace specgbv
