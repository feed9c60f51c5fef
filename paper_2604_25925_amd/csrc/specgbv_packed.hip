// Appending new tokens to a paged cache whose entries are held in 4 bits, and reading tokens back.
//
// Norm of each head of q and k, rotation by the position (as for the cache of 16 and 32 bits), then keys and values in blocks of 32 entries:
// with A the block's largest magnitude the power 2^e is the least with A <= 7 2^e, e in [-120, 125], and an entry becomes the nearest of
// 0, 1/2, 1, 3/2, 2, 3, 4, 6 times 2^e, of two as near the one of even code, 6 above 5.  (A between 6 and 7 costs its entry no more than the
// half step of 1 that entries between 4 and 6 are off by; a power more for all the others would cost each of them a bit.)  A block that holds
// what is not finite has the byte 255, and all of it is no number.
//
// Keys are normalised and rotated in float64 and only what decides the code is kept of it: a float32 cut off behind its last bit, with that
// bit set where anything was cut (no border lies there, so the conversion, which rounds once, decides as it would for the float64).  So a code
// differs from the definition's only where the float64 lies within its own error of a border, 2^-50 of the entry instead of 2^-20.
//
// A lane has 8 adjacent entries, which are one word of the cache, and four lanes a block; the entry that another one turns with is read a second
// time (from the cache) instead of exchanged.  Every entry is read from memory once, so memory bounds it.
#include "specgbv_internal.hpp"

namespace specgbv {
namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 2;                    // tokens of a workgroup at most
constexpr int kMaxPairs = 128;
constexpr int kLane = 8;                      // entries of a lane

__device__ __forceinline__ float widen(uint16_t x) { return __uint_as_float(static_cast<uint32_t>(x) << 16); }
__device__ __forceinline__ float widen(float x) { return x; }
template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ float narrow<float>(float x) { return x; }
template <> __device__ __forceinline__ uint16_t narrow<uint16_t>(float x) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x)); }

template <typename T> struct alignas(16) Vec { T e[16 / sizeof(T)]; };

template <typename T, bool WIDE> __device__ __forceinline__ void load8(const T *src, float (&x)[kLane])
{
    constexpr int W = 16 / sizeof(T);
    if constexpr (WIDE) {
#pragma unroll
        for (int i = 0; i < kLane / W; ++i) {
            const Vec<T> v = reinterpret_cast<const Vec<T> *>(src)[i];
#pragma unroll
            for (int j = 0; j < W; ++j) x[i * W + j] = widen(v.e[j]);
        }
    } else
#pragma unroll
        for (int j = 0; j < kLane; ++j) x[j] = widen(src[j]);
}

template <typename T, bool WIDE> __device__ __forceinline__ void store8(T *dst, const float (&x)[kLane])
{
    constexpr int W = 16 / sizeof(T);
    if constexpr (WIDE) {
#pragma unroll
        for (int i = 0; i < kLane / W; ++i) {
            Vec<T> v;
#pragma unroll
            for (int j = 0; j < W; ++j) v.e[j] = narrow<T>(x[i * W + j]);
            reinterpret_cast<Vec<T> *>(dst)[i] = v;
        }
    } else
#pragma unroll
        for (int j = 0; j < kLane; ++j) dst[j] = narrow<T>(x[j]);
}

// A lane's entries of a head, normalised and rotated, in F (float or double).  x: its entries, b: those they turn with.
template <typename T, bool WIDE, typename F>
__device__ __forceinline__ void turned(const PackedAppendProblem &p, const T *src, const T *weight, const double2 *turn, int e0, bool there, int lanes, F (&y)[kLane])
{
    float x[kLane], b[kLane], w[kLane], wb[kLane];
    const bool turning = there && e0 < 2 * p.pairs;
    const bool split = turning && !p.interleaved;
#pragma unroll
    for (int j = 0; j < kLane; ++j) { x[j] = b[j] = 0.0f; w[j] = wb[j] = 1.0f; }
    int other[WIDE ? 1 : kLane];                              // where the entries that turn with these begin, or each of them
    if constexpr (WIDE) other[0] = e0 < p.pairs ? e0 + p.pairs : e0 - p.pairs;
    else
#pragma unroll
        for (int j = 0; j < kLane; ++j) other[j] = e0 + j >= 2 * p.pairs ? e0 + j : (e0 + j < p.pairs ? e0 + j + p.pairs : e0 + j - p.pairs);
    if (there) load8<T, WIDE>(src + e0, x);
    if (split) {
        if constexpr (WIDE) load8<T, true>(src + other[0], b);
        else
#pragma unroll
            for (int j = 0; j < kLane; ++j) b[j] = widen(src[other[j]]);
    }
    F inv = 1;
    if (weight) {                                             // the same for the head's lanes
        if (there) load8<T, WIDE>(weight + e0, w);
        if (split) {
            if constexpr (WIDE) load8<T, true>(weight + other[0], wb);
            else
#pragma unroll
                for (int j = 0; j < kLane; ++j) wb[j] = widen(weight[other[j]]);
        }
        F sum = 0;
#pragma unroll
        for (int j = 0; j < kLane; ++j) sum += static_cast<F>(x[j]) * static_cast<F>(x[j]);
        for (int m = lanes >> 1; m > 0; m >>= 1) sum += __shfl_xor(sum, m, 64);
        if constexpr (sizeof(F) == 8) inv = 1.0 / sqrt(sum / p.head_dim + p.eps);
        else inv = 1.0f / sqrtf(sum / static_cast<float>(p.head_dim) + static_cast<float>(p.eps));
    }
#pragma unroll
    for (int j = 0; j < kLane; ++j) y[j] = weight ? static_cast<F>(x[j]) * inv * static_cast<F>(w[j]) : static_cast<F>(x[j]);
    if (!turning) return;
    if (p.interleaved) {
#pragma unroll
        for (int j = 0; j < kLane; j += 2)
            if (e0 + j < 2 * p.pairs) {
                const double2 cs = turn[(e0 + j) / 2];
                const F a = y[j], c = y[j + 1];
                y[j] = a * static_cast<F>(cs.x) - c * static_cast<F>(cs.y);
                y[j + 1] = c * static_cast<F>(cs.x) + a * static_cast<F>(cs.y);
            }
        return;
    }
#pragma unroll
    for (int j = 0; j < kLane; ++j) {
        const int e = e0 + j;
        if (!WIDE && e >= 2 * p.pairs) continue;
        const bool lower = e < p.pairs;
        const double2 cs = turn[lower ? e : e - p.pairs];
        const F o = weight ? static_cast<F>(b[j]) * inv * static_cast<F>(wb[j]) : static_cast<F>(b[j]);
        const F side = o * static_cast<F>(cs.y);
        y[j] = lower ? y[j] * static_cast<F>(cs.x) - side : y[j] * static_cast<F>(cs.x) + side;
    }
}

// A float32 that lies on the same side of every border between codes as x.
__device__ __forceinline__ float decisive(double x)
{
    const float r = static_cast<float>(x);
    const double back = r;
    uint32_t bits = __float_as_uint(r);
    if (back != x) bits = (fabs(back) > fabs(x) ? bits - 1 : bits) | 1u;
    return __uint_as_float(bits);
}

// The word of a lane's 8 entries; `byte`: its block's power of two (four lanes have a block).
__device__ __forceinline__ uint32_t packed(const double (&y)[kLane], uint32_t &byte)
{
    double most = 0.0;
#pragma unroll
    for (int j = 0; j < kLane; ++j) most = fabs(y[j]) < INFINITY ? fmax(most, fabs(y[j])) : INFINITY;
    most = fmax(most, __shfl_xor(most, 1, 64));
    most = fmax(most, __shfl_xor(most, 2, 64));
    const uint64_t bits = static_cast<uint64_t>(__double_as_longlong(most));
    int e = static_cast<int>(bits >> 52) - 1023 - 2 + ((bits & 0xFFFFFFFFFFFFFull) > 0xC000000000000ull ? 1 : 0);      // 1.75 2^n = 7 2^(n - 2)
    e = max(-120, min(e, 125));
    byte = static_cast<uint32_t>(e + 127);
    const double up = __longlong_as_double(static_cast<long long>(1023 - e) << 52);
    uint32_t word = 0;
    const float one = 1.0f;
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, decisive(y[0] * up), decisive(y[1] * up), one, 0);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, decisive(y[2] * up), decisive(y[3] * up), one, 1);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, decisive(y[4] * up), decisive(y[5] * up), one, 2);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, decisive(y[6] * up), decisive(y[7] * up), one, 3);
    if (most == INFINITY) { byte = 255u; word = 0u; }
    return word;
}

template <typename T, bool WIDE>
__global__ void __launch_bounds__(kThreads) k_packed_append(PackedAppendProblem p)
{
    __shared__ double2 sh_turn[kTokens][kMaxPairs];
    __shared__ int sh_pos[kTokens], sh_page[kTokens], sh_slot[kTokens];
    const int tid = threadIdx.x;
    const int heads_all = p.heads + 2 * p.kv_heads;
    const int n0 = blockIdx.x * p.block_tokens;
    const int nt = min(p.block_tokens, p.tokens_all - n0);

    if (tid < nt) {
        const int s = p.by_tokens.div(n0 + tid), t = p.by_tokens.mod(n0 + tid, s);
        const int pos = p.positions[s * p.positions_stride + t];
        Place at{-1, 0};
        if (pos >= 0) at = place_of(p.map, s, pos);
        sh_pos[tid] = pos; sh_page[tid] = at.page; sh_slot[tid] = at.slot;
    }
    for (int i = tid; i < nt * p.pairs; i += kThreads) {
        const int k = i / p.pairs, r = i - k * p.pairs;
        const int s = p.by_tokens.div(n0 + k), t = p.by_tokens.mod(n0 + k, s);
        // a turn in float64: whole turns are taken off before the sine and cosine
        const double turns = static_cast<double>(p.positions[s * p.positions_stride + t]) * p.inv_freq[r] * 0.15915494309189533577;
        double sn, cs;
        sincospi(2.0 * (turns - rint(turns)), &sn, &cs);
        sh_turn[k][r] = make_double2(cs, sn);
    }
    __syncthreads();

    const int lanes = 1 << p.lane_bits, u = tid & (lanes - 1), e0 = u * kLane;
    const int slots = kThreads >> p.lane_bits;
    const int todo = nt * heads_all;
    for (int base = 0; base < todo; base += slots) {                   // uniform
        const int item = base + (tid >> p.lane_bits);
        if (item >= todo) continue;                                    // whole groups of lanes
        const int k = p.by_heads.div(item), h = p.by_heads.mod(item, k);
        const int s = p.by_tokens.div(n0 + k), t = p.by_tokens.mod(n0 + k, s);
        const bool mine = e0 < p.head_dim;
        if (h < p.heads) {
            const bool there = mine && sh_pos[k] >= 0;
            float y[kLane];
            turned<T, WIDE, float>(p, static_cast<const T *>(p.q) + s * p.q_stride[0] + t * p.q_stride[1] + h * p.q_stride[2],
                                   static_cast<const T *>(p.q_weight), sh_turn[k], e0, there, lanes, y);
            if (!there)
#pragma unroll
                for (int j = 0; j < kLane; ++j) y[j] = 0.0f;
            if (mine) store8<T, WIDE>(static_cast<T *>(p.q_out) + s * p.q_out_stride[0] + t * p.q_out_stride[1] + h * p.q_out_stride[2] + e0, y);
            continue;
        }
        if (sh_pos[k] < 0 || sh_page[k] < 0) continue;                 // the same for the token's lanes
        const bool value = h >= p.heads + p.kv_heads;
        const int hd = value ? h - p.heads - p.kv_heads : h - p.heads;
        double y[kLane];
        if (value) {
            float x[kLane];
#pragma unroll
            for (int j = 0; j < kLane; ++j) x[j] = 0.0f;
            if (mine) load8<T, WIDE>(static_cast<const T *>(p.v) + s * p.v_stride[0] + t * p.v_stride[1] + hd * p.v_stride[2] + e0, x);
#pragma unroll
            for (int j = 0; j < kLane; ++j) y[j] = x[j];
        } else
            turned<T, WIDE, double>(p, static_cast<const T *>(p.k) + s * p.k_stride[0] + t * p.k_stride[1] + hd * p.k_stride[2],
                                    static_cast<const T *>(p.k_weight), sh_turn[k], e0, mine, lanes, y);
        uint32_t byte;
        const uint32_t word = packed(y, byte);
        if (!mine) continue;
        const int64_t page = sh_page[k], slot = sh_slot[k];
        const int64_t *cs = value ? p.v_cache_stride : p.k_cache_stride, *ss = value ? p.v_scale_stride : p.k_scale_stride;
        *reinterpret_cast<uint32_t *>((value ? p.v_cache : p.k_cache) + page * cs[0] + hd * cs[1] + slot * cs[2] + e0 / 2) = word;
        if (u % 4 == 0) (value ? p.v_scale : p.k_scale)[page * ss[0] + hd * ss[1] + u / 4 * ss[2] + slot] = static_cast<uint8_t>(byte);
    }
}

template <typename T, bool WIDE>
__global__ void __launch_bounds__(kThreads) k_packed_read(PackedReadProblem p)
{
    const int lanes = 1 << p.lane_bits, u = threadIdx.x & (lanes - 1), e0 = u * kLane;
    const int64_t all = static_cast<int64_t>(blockIdx.x) * (kThreads >> p.lane_bits) + (threadIdx.x >> p.lane_bits);
    if (all >= static_cast<int64_t>(p.tokens_all) * 2 * p.kv_heads || e0 >= p.head_dim) return;
    const int item = static_cast<int>(all);                            // (fewer than 2^31)
    const int n = p.by_heads.div(item), h = p.by_heads.mod(item, n);
    const int s = p.by_tokens.div(n), t = p.by_tokens.mod(n, s);
    const int pos = p.positions[s * p.positions_stride + t];
    Place at{-1, 0};
    if (pos >= 0) at = place_of(p.map, s, pos);
    const bool value = h >= p.kv_heads;
    const int hd = value ? h - p.kv_heads : h;
    float x[kLane];
#pragma unroll
    for (int j = 0; j < kLane; ++j) x[j] = 0.0f;
    if (at.page >= 0) {
        const int64_t *cs = value ? p.v_cache_stride : p.k_cache_stride, *ss = value ? p.v_scale_stride : p.k_scale_stride;
        const uint32_t word = *reinterpret_cast<const uint32_t *>((value ? p.v_cache : p.k_cache) + at.page * cs[0] + hd * cs[1] + at.slot * cs[2] + e0 / 2);
        const float power = __uint_as_float(static_cast<uint32_t>((value ? p.v_scale : p.k_scale)[at.page * ss[0] + hd * ss[1] + u / 4 * ss[2] + at.slot]) << 23);
        uint32_t two[4];
        two[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, power, 0));
        two[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, power, 1));
        two[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, power, 2));
        two[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, power, 3));
#pragma unroll
        for (int j = 0; j < kLane; ++j) x[j] = __uint_as_float(j % 2 ? two[j / 2] & 0xFFFF0000u : two[j / 2] << 16);
    }
    T *dst = value ? static_cast<T *>(p.v) + s * p.v_stride[0] + t * p.v_stride[1] + hd * p.v_stride[2]
                   : static_cast<T *>(p.k) + s * p.k_stride[0] + t * p.k_stride[1] + hd * p.k_stride[2];
    store8<T, WIDE>(dst + e0, x);
}

int lane_bits_of(int head_dim)
{
    int bits = 2;                                                      // a block's four lanes at least
    while ((kLane << bits) < head_dim) ++bits;
    return bits;
}

}  // namespace

hipError_t launch_packed_append(const PackedAppendProblem &given, int dtype, bool wide, hipStream_t stream)
{
    PackedAppendProblem p = given;
    p.lane_bits = lane_bits_of(p.head_dim);
    p.block_tokens = p.tokens_all >= 8 * compute_units() ? kTokens : 1;
    const int64_t grid = (static_cast<int64_t>(p.tokens_all) + p.block_tokens - 1) / p.block_tokens;
    if (grid >= kLaunchGroups) return hipErrorInvalidConfiguration;
    const dim3 groups(static_cast<unsigned>(grid)), threads(kThreads);
    if (dtype == 1) {
        if (wide) hipLaunchKernelGGL((k_packed_append<uint16_t, true>), groups, threads, 0, stream, p);
        else hipLaunchKernelGGL((k_packed_append<uint16_t, false>), groups, threads, 0, stream, p);
    } else {
        if (wide) hipLaunchKernelGGL((k_packed_append<float, true>), groups, threads, 0, stream, p);
        else hipLaunchKernelGGL((k_packed_append<float, false>), groups, threads, 0, stream, p);
    }
    return hipGetLastError();
}

hipError_t launch_packed_read(const PackedReadProblem &given, int dtype, bool wide, hipStream_t stream)
{
    PackedReadProblem p = given;
    p.lane_bits = lane_bits_of(p.head_dim);
    const int64_t per = kThreads >> p.lane_bits, grid = (static_cast<int64_t>(p.tokens_all) * 2 * p.kv_heads + per - 1) / per;
    if (grid >= kLaunchGroups) return hipErrorInvalidConfiguration;
    const dim3 groups(static_cast<unsigned>(grid)), threads(kThreads);
    if (dtype == 1) {
        if (wide) hipLaunchKernelGGL((k_packed_read<uint16_t, true>), groups, threads, 0, stream, p);
        else hipLaunchKernelGGL((k_packed_read<uint16_t, false>), groups, threads, 0, stream, p);
    } else {
        if (wide) hipLaunchKernelGGL((k_packed_read<float, true>), groups, threads, 0, stream, p);
        else hipLaunchKernelGGL((k_packed_read<float, false>), groups, threads, 0, stream, p);
    }
    return hipGetLastError();
}

}  // namespace specgbv
