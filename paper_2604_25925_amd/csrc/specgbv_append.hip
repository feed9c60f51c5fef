// Appending new tokens to a paged cache: norm of each head of q and k, rotation by the position, keys and values to their pages.
//
// For a head x of D entries at position p:  y = x (sum x^2 / D + eps)^(-1/2) w;  (y_a, y_b) turned by the angle p f_i for every pair
// i < R, (a, b) = (i, i + R) or (2 i, 2 i + 1).  Every entry is read once and written once, so memory bounds it; the angles
// (one product, a reduction to a quarter turn in float64 and a sine and cosine per token and pair) are formed once per token and kept
// in LDS for all its heads.
//
// A lane takes a "unit": the two vectors whose entries turn into each other (W entries at i and W at i + R, or 2 W adjacent ones),
// so the rotation stays within a lane, and a head is a power of two of lanes, so its norm is a few exchanges in a wave.  W is 16
// bytes where pairs, strides and addresses allow it.
//
// 5 prompts of up to 4001 tokens, 32 heads and 8 kv heads of 128, bfloat16: 330 MB in 73 us, 4.5 TB/s (a copy 4.8).  256 tokens with norms: 6.0 us;
// one token: 2.9; both the latency of position, table, input and store in a row.
#include "specgbv_internal.hpp"

namespace specgbv {
namespace {

constexpr int kAppendThreads = 256;
constexpr int kAppendTokens = 2;              // tokens of a workgroup at most
constexpr int kAppendMaxPairs = 128;

template <typename T, int W> struct alignas(sizeof(T) * W) Pack { T e[W]; };

__device__ __forceinline__ float widen(uint16_t x) { return __uint_as_float(static_cast<uint32_t>(x) << 16); }
__device__ __forceinline__ float widen(float x) { return x; }
template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ float narrow<float>(float x) { return x; }
template <> __device__ __forceinline__ uint16_t narrow<uint16_t>(float x)
{
    return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));       // to nearest, ties to even
}

// sin and cos of 2 pi turns: the nearest quarter turn is taken off in float64, so that what is rounded to float32 is at most an
// eighth of a turn and its rounding is relative to the small angle.
__device__ __forceinline__ float2 turn_of(double turns)
{
    const double quarters = rint(turns * 4.0);
    const float r = static_cast<float>((turns * 4.0 - quarters) * 0.5);        // in half turns, |r| <= 1/4
    float s, c;
    sincospif(r, &s, &c);
    // (quarters is beyond 2^31 only for angles whose float64 no longer holds the turn; the remainder mod 4 is exact below 2^53)
    const int q = static_cast<int>(quarters - 4.0 * floor(quarters * 0.25));
    const float c1 = (q & 1) ? -s : c, s1 = (q & 1) ? c : s;
    return (q & 2) ? make_float2(-c1, -s1) : make_float2(c1, s1);
}

template <typename T, int W, int NU>
__global__ void __launch_bounds__(kAppendThreads) k_append(AppendProblem p)
{
    __shared__ float2 sh_turn[kAppendTokens][kAppendMaxPairs];
    __shared__ int sh_pos[kAppendTokens];
    __shared__ int64_t sh_k[kAppendTokens], sh_v[kAppendTokens];       // where the token's heads go in the cache, < 0: nowhere
    const int tid = threadIdx.x;
    const int heads_all = p.heads + 2 * p.kv_heads;
    const int n0 = blockIdx.x * p.block_tokens;
    const int nt = min(p.block_tokens, p.tokens_all - n0);

    if (tid < nt) {
        const int s = p.by_tokens.div(n0 + tid), t = p.by_tokens.mod(n0 + tid, s);
        const int pos = p.positions[s * p.positions_stride + t];
        Place at{-1, 0};
        if (pos >= 0) at = place_of(p.map, s, pos);
        sh_pos[tid] = pos;
        sh_k[tid] = at.page < 0 ? -1 : at.page * p.k_cache_stride[0] + at.slot * p.k_cache_stride[2];
        sh_v[tid] = at.page < 0 ? -1 : at.page * p.v_cache_stride[0] + at.slot * p.v_cache_stride[2];
    }
    for (int i = tid; i < nt * p.pairs; i += kAppendThreads) {
        const int k = i / p.pairs, r = i - k * p.pairs;
        const int s = p.by_tokens.div(n0 + k), t = p.by_tokens.mod(n0 + k, s);
        const int pos = p.positions[s * p.positions_stride + t];
        sh_turn[k][r] = turn_of(static_cast<double>(pos) * p.inv_freq[r] * 0.15915494309189533577);
    }
    __syncthreads();

    const int lanes = 1 << p.lane_bits, u0 = tid & (lanes - 1);
    const int slots = kAppendThreads >> p.lane_bits;
    const int units = p.head_dim / (2 * W), turning = p.pairs / W;
    const int todo = nt * heads_all;
    for (int base = 0; base < todo; base += slots) {                   // uniform
        const int item = base + (tid >> p.lane_bits);
        if (item >= todo) continue;                                    // whole groups of lanes
        const int k = p.by_heads.div(item), h = p.by_heads.mod(item, k);
        const int s = p.by_tokens.div(n0 + k), t = p.by_tokens.mod(n0 + k, s);
        const int kind = h < p.heads ? 0 : (h < p.heads + p.kv_heads ? 1 : 2);
        const int hd = kind == 0 ? h : (kind == 1 ? h - p.heads : h - p.heads - p.kv_heads);
        const T *src = kind == 0 ? static_cast<const T *>(p.q) + s * p.q_stride[0] + t * p.q_stride[1] + hd * p.q_stride[2]
                     : kind == 1 ? static_cast<const T *>(p.k) + s * p.k_stride[0] + t * p.k_stride[1] + hd * p.k_stride[2]
                                 : static_cast<const T *>(p.v) + s * p.v_stride[0] + t * p.v_stride[1] + hd * p.v_stride[2];
        const T *weight = static_cast<const T *>(kind == 0 ? p.q_weight : (kind == 1 ? p.k_weight : nullptr));
        const int64_t place = kind == 1 ? sh_k[k] : (kind == 2 ? sh_v[k] : 0);
        const bool there = sh_pos[k] >= 0 && place >= 0;
        T *dst = kind == 0 ? static_cast<T *>(p.q_out) + s * p.q_out_stride[0] + t * p.q_out_stride[1] + hd * p.q_out_stride[2]
               : kind == 1 ? static_cast<T *>(p.k_cache) + place + hd * p.k_cache_stride[1]
                           : static_cast<T *>(p.v_cache) + place + hd * p.v_cache_stride[1];
        float x[NU][2][W];
        int at[NU][2];
        float sum = 0.0f;
#pragma unroll
        for (int n = 0; n < NU; ++n) {
            const int u = u0 + n * lanes;
            const bool split = !p.interleaved && u < turning;
            at[n][0] = split ? u * W : u * 2 * W;
            at[n][1] = split ? u * W + p.pairs : u * 2 * W + W;
            if (u >= units || !there) {
#pragma unroll
                for (int j = 0; j < W; ++j) x[n][0][j] = x[n][1][j] = 0.0f;
                continue;
            }
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                const Pack<T, W> v = *reinterpret_cast<const Pack<T, W> *>(src + at[n][d]);
#pragma unroll
                for (int j = 0; j < W; ++j) { x[n][d][j] = widen(v.e[j]); sum = fmaf(x[n][d][j], x[n][d][j], sum); }
            }
        }
        if (weight) {                                                  // uniform within the head's lanes
            for (int m = lanes >> 1; m > 0; m >>= 1) sum += __shfl_xor(sum, m, 64);
            const float inv = 1.0f / sqrtf(sum * p.inv_dim + p.eps);
#pragma unroll
            for (int n = 0; n < NU; ++n)
                if (u0 + n * lanes < units)
#pragma unroll
                    for (int d = 0; d < 2; ++d) {
                        const Pack<T, W> w = *reinterpret_cast<const Pack<T, W> *>(weight + at[n][d]);
#pragma unroll
                        for (int j = 0; j < W; ++j) x[n][d][j] = x[n][d][j] * inv * widen(w.e[j]);
                    }
        }
        if (kind != 2) {
#pragma unroll
            for (int n = 0; n < NU; ++n) {
                const int u = u0 + n * lanes;
                if (u >= turning) continue;
                if (!p.interleaved || W == 1) {
#pragma unroll
                    for (int j = 0; j < W; ++j) {
                        const float2 cs = sh_turn[k][u * W + j];
                        const float a = x[n][0][j], b = x[n][1][j];
                        x[n][0][j] = a * cs.x - b * cs.y;
                        x[n][1][j] = b * cs.x + a * cs.y;
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < W; ++j) {
                        const float2 cs = sh_turn[k][u * W + j];
                        float *pair = &x[n][2 * j / W][2 * j % W];
                        const float a = pair[0], b = pair[1];
                        pair[0] = a * cs.x - b * cs.y;
                        pair[1] = b * cs.x + a * cs.y;
                    }
                }
            }
        }
        if (kind != 0 && !there) continue;
#pragma unroll
        for (int n = 0; n < NU; ++n) {
            if (u0 + n * lanes >= units) continue;
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                Pack<T, W> v;
#pragma unroll
                for (int j = 0; j < W; ++j) v.e[j] = there ? narrow<T>(x[n][d][j]) : narrow<T>(0.0f);
                *reinterpret_cast<Pack<T, W> *>(dst + at[n][d]) = v;
            }
        }
    }
}

template <typename T, int W>
hipError_t launch_width(const AppendProblem &p, hipStream_t stream)
{
    const int grid = (p.tokens_all + p.block_tokens - 1) / p.block_tokens;      // (fewer than 2^30 tokens)
    hipLaunchKernelGGL((k_append<T, W, W == 1 ? 2 : 1>), dim3(grid), dim3(kAppendThreads), 0, stream, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_append(const AppendProblem &given, int dtype, int width, hipStream_t stream)
{
    AppendProblem p = given;
    const int units = p.head_dim / (2 * width);
    p.lane_bits = 0;
    while (p.lane_bits < 6 && (1 << p.lane_bits) < units) ++p.lane_bits;
    // tokens of a workgroup, 1 / 2 / 4, us (32 heads, 8 kv heads of 128, bfloat16): 5.5 / 6.8 / 10.5 for 256 tokens, 8.2 / 9.0 / 12.2 for 1024,
    // 13.2 / 12.9 / 16.0 for 2304, 82 / 77 / 79 for 20005
    p.block_tokens = p.tokens_all >= 8 * compute_units() ? kAppendTokens : 1;
    if ((static_cast<int64_t>(p.tokens_all) + p.block_tokens - 1) / p.block_tokens >= kLaunchGroups) return hipErrorInvalidConfiguration;
    if (dtype == 1) switch (width) {
        case 8: return launch_width<uint16_t, 8>(p, stream);
        case 4: return launch_width<uint16_t, 4>(p, stream);
        case 2: return launch_width<uint16_t, 2>(p, stream);
        default: return launch_width<uint16_t, 1>(p, stream);
    }
    switch (width) {
    case 4: return launch_width<float, 4>(p, stream);
    case 2: return launch_width<float, 2>(p, stream);
    default: return launch_width<float, 1>(p, stream);
    }
}

}  // namespace specgbv
