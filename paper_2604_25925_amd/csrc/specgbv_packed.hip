// Appending new tokens to a paged cache whose entries are held in 4 bits, and reading tokens back.
//
// Norm of each head of q and k, rotation by the position (as for the cache of 16 and 32 bits), then keys and values in blocks of 32 entries:
// with A the block's largest magnitude the power 2^e is the least with A <= 7 2^e, e in [-120, 125], and an entry becomes the nearest of
// 0, 1/2, 1, 3/2, 2, 3, 4, 6 times 2^e, of two as near the one of even code, 6 above 5.  (A between 6 and 7 costs its entry no more than the
// half step of 1 that entries between 4 and 6 are off by; a power more for all the others would cost each of them a bit.)  A block that holds
// what is not finite has the byte 255, and all of it is no number.
//
// Keys are normalised and rotated in float64, and what decides the code is kept of it: 20 bits of its mantissa, as a float32 with a last bit that is set
// where anything was cut (no border lies there, so the conversion, which rounds once, decides as it would for the float64).  So a code differs from the
// definition's only where the entry lies within the float64's own error of a border: 2^-50 (|a| + |b|) for a pair (a, b) that turns, whatever the position, since the product
// of position and frequency and 1 / (2 pi) have tails, and 2^-49 more of it for a norm (a sum of D squares, a root, a quotient and two products).
//
// A lane has 8 adjacent entries, which are one word of the cache, and four lanes a block; the entry that another one turns with is read a second
// time (from the cache) instead of exchanged.  Every entry is read from memory once.
//
// What bounds it.  Memory, where tokens are many and their heads fill a wave: 5 prompts of up to 4001 tokens (32 heads, 8 kv heads of 128, bfloat16; 13622 tokens and padding), appending 82 us for 346 MB that
// have to move (167 read, 179 written: 164 are queries, those of padding too, which become zeros), 367 by the counters (scales are bytes by themselves), 4.5 TB/s or 95 % of what a copy reaches.
// Inputs one pass ahead spill (87 us), 4 and 6 waves a SIMD 87 us.  Keys in float32 first, and in float64 only near borders: 22 us more, nearly every wave has one that lies near.  Reading back 19 us for
// 97 MB, 5.2 TB/s.  256 tokens of drafts 6.3 and 3.5 us, one token 3.1 and 2.3: the chain from the position over the table to the inputs, once.  Few small heads leave lanes idle, since a wave has one
// token: of 2 heads of 32 on 2 kv heads 8 lanes of 64 work in each pass, and each token costs a whole wave's start (30 sequences of 983 tokens, with the reading back, 46 us where the bytes need 4).
#include "specgbv_internal.hpp"

namespace specgbv {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kMaxPairs = 128;
constexpr int kLane = 8;                      // entries of a lane

__device__ __forceinline__ float widen(uint16_t x) { return __uint_as_float(static_cast<uint32_t>(x) << 16); }
__device__ __forceinline__ float widen(float x) { return x; }
template <typename T> __device__ __forceinline__ T narrow(float x);
template <> __device__ __forceinline__ float narrow<float>(float x) { return x; }
template <> __device__ __forceinline__ uint16_t narrow<uint16_t>(float x) { return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x)); }

template <typename T> struct alignas(16) Vec { T e[16 / sizeof(T)]; };

// Eight adjacent entries as they come from memory: words of two (bfloat16) or one.
template <typename T> struct Entries {
    static constexpr int kWords = kLane * sizeof(T) / 4;
    uint32_t w[kWords];
    __device__ __forceinline__ float operator[](int j) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[j]);
        else return __uint_as_float(j % 2 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
    }
    __device__ __forceinline__ void put(int j, T x)
    {
        if constexpr (sizeof(T) == 4) w[j] = __float_as_uint(x);
        else w[j / 2] = j % 2 ? (w[j / 2] & 0xFFFFu) | static_cast<uint32_t>(x) << 16 : x;
    }
};

template <typename T, bool WIDE> __device__ __forceinline__ void load8(const T *src, Entries<T> &x)
{
    if constexpr (WIDE) {
#pragma unroll
        for (int i = 0; i < Entries<T>::kWords / 4; ++i) {
            const U4 v = reinterpret_cast<const U4 *>(src)[i];
            x.w[4 * i] = v.x; x.w[4 * i + 1] = v.y; x.w[4 * i + 2] = v.z; x.w[4 * i + 3] = v.w;
        }
    } else
#pragma unroll
        for (int j = 0; j < kLane; ++j) x.put(j, src[j]);
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

// The entries that a lane's entries e0.. of a head turn with; 0 for those that do not turn.  (WIDE: pairs are whole vectors, or lie in one.)
template <typename T, bool WIDE> __device__ __forceinline__ void load_partners(const T *head, int e0, int pairs, int interleaved, Entries<T> &b)
{
    if (WIDE && !interleaved) load8<T, true>(head + (e0 < pairs ? e0 + pairs : e0 - pairs), b);
    else
#pragma unroll
        for (int j = 0; j < kLane; ++j) {
            const int e = e0 + j;
            if (e < 2 * pairs) b.put(j, head[interleaved ? e ^ 1 : (e < pairs ? e + pairs : e - pairs)]);
        }
}

// The pair that entry e belongs to, where it turns; and whether it is the pair's first.
__device__ __forceinline__ int pair_of(const PackedAppendProblem &p, int e) { return p.interleaved ? e >> 1 : (e < p.pairs ? e : e - p.pairs); }
__device__ __forceinline__ bool first_of_pair(const PackedAppendProblem &p, int e) { return p.interleaved ? e % 2 == 0 : e < p.pairs; }

// pos * f in turns, without the whole ones.  Both products and 1 / (2 pi) have tails: half a step of a product alone is up to 2^-23 of an angle at the last positions; what is left, half a turn at most, is
// off by half a step.
__device__ __forceinline__ double turns_left(double pos, double f)
{
#pragma clang fp contract(off)                                         // (a product taken into the subtraction would count its tail twice)
    constexpr double kTurn = 0.15915494309189533577, kTurnTail = -9.839338337591243e-18;      // 1 / (2 pi) is their sum
    const double angle = pos * f, angle_tail = fma(pos, f, -angle), turns = angle * kTurn;
    const double tail = fma(angle, kTurn, -turns) + fma(angle, kTurnTail, angle_tail * kTurn);
    return (turns - rint(turns)) + tail;
}

// A lane's entries x of a key's head, normalised and rotated in float64; b: those they turn with (0 where they do not turn).
template <typename T, bool WIDE>
__device__ __forceinline__ void turned(const PackedAppendProblem &p, const Entries<T> &x, const Entries<T> &b, const double2 *turn, int e0, bool there, int lanes, double (&y)[kLane])
{
    const T *weight = static_cast<const T *>(p.k_weight);
    const bool turning = there && e0 < 2 * p.pairs;
    double o[kLane];
#pragma unroll
    for (int j = 0; j < kLane; ++j) { y[j] = x[j]; o[j] = b[j]; }
    if (weight) {                                             // the same for the head's lanes
        Entries<T> w{}, wb{};
        if (there) load8<T, WIDE>(weight + e0, w);
        if (turning) load_partners<T, WIDE>(weight, e0, p.pairs, p.interleaved, wb);
        double sum = 0;
#pragma unroll
        for (int j = 0; j < kLane; ++j) sum += y[j] * y[j];
        for (int m = lanes >> 1; m > 0; m >>= 1) sum += __shfl_xor(sum, m, 64);
        const double inv = 1.0 / sqrt(sum / p.head_dim + p.eps);
#pragma unroll
        for (int j = 0; j < kLane; ++j) {
            y[j] *= inv * static_cast<double>(w[j]);
            o[j] *= inv * static_cast<double>(wb[j]);
        }
    }
    if (!turning) return;
    if (WIDE && !p.interleaved) {                             // all of a lane's entries are first ones, or none
        const double2 *mine = turn + (e0 < p.pairs ? e0 : e0 - p.pairs);
        const double sign = e0 < p.pairs ? -1.0 : 1.0;
#pragma unroll
        for (int j = 0; j < kLane; ++j) y[j] = y[j] * mine[j].x + o[j] * (mine[j].y * sign);
        return;
    }
#pragma unroll
    for (int j = 0; j < kLane; ++j)
        if (e0 + j < 2 * p.pairs) {
            const double2 cs = turn[pair_of(p, e0 + j)];
            y[j] = y[j] * cs.x + o[j] * (first_of_pair(p, e0 + j) ? -cs.y : cs.y);
        }
}

// A float64's bits as those of a float32 that lies on the same side of every border between codes: the first 20 of the mantissa, and the last bit set where any behind the first 20 were.
// Beyond float32's range it is the largest or a smallest one, whose codes are the same; what is not finite is looked at elsewhere.
__device__ __forceinline__ uint32_t decisive(double x)
{
    const uint64_t bits = static_cast<uint64_t>(__double_as_longlong(x));
    const uint32_t hi = static_cast<uint32_t>(bits >> 32), size = hi & 0x7FFFFFFFu;
    const uint32_t in_range = min(max(size, 0x38000000u), 0x47EFFFFFu);                  // 2^-127 and the last below 2^128
    return (in_range - 0x38000000u) << 3 | min(static_cast<uint32_t>(bits), 1u) | (hi & 0x80000000u);
}

// The word of a lane's 8 entries, given by a float32's bits each; `odd`: the lane has one that is not finite.  `byte`: its block's power of two (four lanes have a block).
__device__ __forceinline__ uint32_t packed(const uint32_t (&y)[kLane], bool odd, uint32_t &byte)
{
    uint32_t most = odd ? 0x7FFFFFFFu : 0u;                            // as bits: in order
#pragma unroll
    for (int j = 0; j < kLane; ++j) most = max(most, y[j] & 0x7FFFFFFFu);
    most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 1, 64)));
    most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), 2, 64)));
    // the least e with most <= 7 2^e = 7/4 2^(e + 2)
    const int e = max(-120, min(static_cast<int>(most >> 23) - 127 - 2 + ((most & 0x7FFFFFu) > 0x600000u ? 1 : 0), 125));
    byte = static_cast<uint32_t>(e + 127);
    const float power = __uint_as_float(byte << 23);
    uint32_t word = 0;
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, __uint_as_float(y[0]), __uint_as_float(y[1]), power, 0);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, __uint_as_float(y[2]), __uint_as_float(y[3]), power, 1);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, __uint_as_float(y[4]), __uint_as_float(y[5]), power, 2);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, __uint_as_float(y[6]), __uint_as_float(y[7]), power, 3);
    if (most >= 0x7F800000u) { byte = 255u; word = 0u; }
    return word;
}

// What does not change in a kernel, by scalar loads.
typedef const int32_t __attribute__((address_space(4))) *ConstInts;
__device__ __forceinline__ int scalar_at(const int32_t *p, int64_t i) { return reinterpret_cast<ConstInts>(reinterpret_cast<uintptr_t>(p))[i]; }

// A token of a wave: its sequence, its place among the sequence's tokens and its position; all scalar.
struct Token { int s, t, pos; };
__device__ __forceinline__ Token token_of(const Divider &by_tokens, const int32_t *positions, int64_t stride, int n)
{
    const int s = by_tokens.div(n), t = by_tokens.mod(n, s);
    return {s, t, scalar_at(positions, s * stride + t)};
}
__device__ __forceinline__ Place scalar_place(const PageMap &m, int sequence, int pos)
{
    const int n = m.page.div(pos);
    if (pos < 0 || n >= m.width) return {-1, 0};
    const int page = scalar_at(m.table, sequence * m.table_stride + n);
    return {static_cast<uint32_t>(page) < static_cast<uint32_t>(m.pages) ? page : -1, m.page.mod(pos, n)};
}

// A wave has one token, and of its heads' passes (as many heads at once as 64 lanes hold; of q, then k, then v) a slice, so that all that belongs to the
// token is scalar arithmetic; no barrier stands anywhere.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(kThreads, WIDE ? (sizeof(T) == 2 ? 5 : 4) : 3) k_packed_append(PackedAppendProblem p)
{
    __shared__ double2 sh_turn[kWaves][kMaxPairs];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int at_all = static_cast<int>(blockIdx.x) * kWaves + wave;
    const int n = p.by_slices.div(at_all), slice = p.by_slices.mod(at_all, n);
    if (n >= p.tokens_all) return;
    const int first = slice * p.slice, last = min(p.passes, first + p.slice);
    const int k_pass = p.q_passes, v_pass = p.q_passes + p.k_passes;
    const Token tk = token_of(p.by_tokens, p.positions, p.positions_stride, n);
    const int lanes = 1 << p.lane_bits, u = lane & (lanes - 1), e0 = u * kLane, head = lane >> p.lane_bits, heads = 64 >> p.lane_bits;
    const bool mine = e0 < p.head_dim;

    Place at{-1, 0};
    if (last > k_pass && tk.pos >= 0) at = scalar_place(p.map, tk.s, tk.pos);
    const int64_t page = at.page, slot = at.slot;

    auto load = [&](const T *src, bool there, Entries<T> &x, Entries<T> &b) {
        x = b = Entries<T>{};
        if (!there) return;
        load8<T, WIDE>(src + e0, x);
        if (e0 < 2 * p.pairs) load_partners<T, WIDE>(src, e0, p.pairs, p.interleaved, b);
    };
    auto store = [&](uint8_t *data, int32_t data_head, uint8_t *scale, int32_t scale_head, int32_t scale_block, int hd, uint32_t word, uint32_t byte) {
        *reinterpret_cast<uint32_t *>(data + (static_cast<int64_t>(hd) * data_head + e0 / 2)) = word;
        if (u % 4 == 0) scale[static_cast<int64_t>(hd) * scale_head + static_cast<int64_t>(u / 4) * scale_block] = static_cast<uint8_t>(byte);
    };

    // ---- values: as they are
    if (at.page >= 0) {
        const T *base = static_cast<const T *>(p.v) + (tk.s * p.v_stride[0] + tk.t * p.v_stride[1]);
        uint8_t *data = p.v_cache + (page * p.v_cache_stride[0] + slot * p.v_cache_stride[1]), *scale = p.v_scale + (page * p.v_scale_page + slot);
#pragma unroll 2
        for (int pass = max(first, v_pass); pass < last; ++pass) {
            const int hd = (pass - v_pass) * heads + head;
            const bool there = mine && hd < p.kv_heads;
            Entries<T> x{};
            if (there) load8<T, WIDE>(base + static_cast<int64_t>(hd) * p.v_head + e0, x);
            uint32_t bits[kLane], byte;
#pragma unroll
            for (int j = 0; j < kLane; ++j) bits[j] = __float_as_uint(x[j]);
            const uint32_t word = packed(bits, false, byte);
            if (there) store(data, p.v_cache_head, scale, p.v_scale_head, p.v_scale_block, hd, word, byte);
        }
    }
    if (first >= v_pass) return;

    // ---- what q and k turn by
    if (tk.pos >= 0)
        for (int i = lane; i < p.pairs; i += 64) {
            double sn, cs;
            sincospi(2.0 * turns_left(tk.pos, p.inv_freq[i]), &sn, &cs);
            sh_turn[wave][i] = make_double2(cs, sn);
        }
    __builtin_amdgcn_wave_barrier();                                   // (a wave's accesses to LDS are done in their order)

    if (at.page >= 0) {
        const T *base = static_cast<const T *>(p.k) + (tk.s * p.k_stride[0] + tk.t * p.k_stride[1]);
        uint8_t *data = p.k_cache + (page * p.k_cache_stride[0] + slot * p.k_cache_stride[1]), *scale = p.k_scale + (page * p.k_scale_page + slot);
#pragma unroll 1
        for (int pass = max(first, k_pass); pass < min(last, v_pass); ++pass) {
            const int hd = (pass - k_pass) * heads + head;
            const bool there = mine && hd < p.kv_heads;
            Entries<T> x, b;
            load(base + static_cast<int64_t>(hd) * p.k_head, there, x, b);
            double y[kLane];
            turned<T, WIDE>(p, x, b, sh_turn[wave], e0, there, lanes, y);
            uint32_t bits[kLane], byte, top = 0;
#pragma unroll
            for (int j = 0; j < kLane; ++j) {
                bits[j] = decisive(y[j]);
                top = max(top, static_cast<uint32_t>(__double2hiint(y[j])) & 0x7FFFFFFFu);
            }
            const uint32_t word = packed(bits, top >= 0x7FF00000u, byte);
            if (there) store(data, p.k_cache_head, scale, p.k_scale_head, p.k_scale_block, hd, word, byte);
        }
    }

    // ---- queries, in float32: what a lane's entries are multiplied by is the same for all heads
    if (first >= min(last, k_pass)) return;
    const T *base = static_cast<const T *>(p.q) + (tk.s * p.q_stride[0] + tk.t * p.q_stride[1]), *weight = static_cast<const T *>(p.q_weight);
    T *out = static_cast<T *>(p.q_out) + (tk.s * p.q_out_stride[0] + tk.t * p.q_out_stride[1]);
    float cs[kLane], sn[kLane];
    Entries<T> w{}, wb{};
    if (weight && mine) {
        load8<T, WIDE>(weight + e0, w);
        if (e0 < 2 * p.pairs) load_partners<T, WIDE>(weight, e0, p.pairs, p.interleaved, wb);
    }
#pragma unroll
    for (int j = 0; j < kLane; ++j) {
        cs[j] = 1.0f; sn[j] = 0.0f;
        if (e0 + j < 2 * p.pairs) {
            const double2 t = sh_turn[wave][pair_of(p, e0 + j)];
            cs[j] = static_cast<float>(t.x);
            sn[j] = static_cast<float>(first_of_pair(p, e0 + j) ? -t.y : t.y);
        }
    }
#pragma unroll 2
    for (int pass = first; pass < min(last, k_pass); ++pass) {
        const int hd = pass * heads + head;
        const bool there = mine && hd < p.heads && tk.pos >= 0;
        Entries<T> x, b;
        load(base + static_cast<int64_t>(hd) * p.q_head, there, x, b);
        float y[kLane];
        if (weight) {
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < kLane; ++j) sum = fmaf(x[j], x[j], sum);
            for (int m = lanes >> 1; m > 0; m >>= 1) sum += __shfl_xor(sum, m, 64);
            const float inv = 1.0f / sqrtf(sum * p.inv_dim + static_cast<float>(p.eps));
#pragma unroll
            for (int j = 0; j < kLane; ++j) y[j] = x[j] * inv * w[j] * cs[j] + b[j] * inv * wb[j] * sn[j];
        } else
#pragma unroll
            for (int j = 0; j < kLane; ++j) y[j] = x[j] * cs[j] + b[j] * sn[j];
        if (!there)
#pragma unroll
            for (int j = 0; j < kLane; ++j) y[j] = 0.0f;
        if (mine && hd < p.heads) store8<T, WIDE>(out + static_cast<int64_t>(hd) * p.q_out_head + e0, y);
    }
}

// A wave has a token and a slice of its passes, of k and then of v, as above.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(kThreads) k_packed_read(PackedReadProblem p)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int at_all = static_cast<int>(blockIdx.x) * kWaves + wave;
    const int n = p.by_slices.div(at_all), slice = p.by_slices.mod(at_all, n);
    if (n >= p.tokens_all) return;
    const int first = slice * p.slice, last = min(2 * p.k_passes, first + p.slice);
    const Token tk = token_of(p.by_tokens, p.positions, p.positions_stride, n);
    const Place at = scalar_place(p.map, tk.s, tk.pos);
    const int lanes = 1 << p.lane_bits, u = lane & (lanes - 1), e0 = u * kLane, heads = 64 >> p.lane_bits;
    if (e0 >= p.head_dim) return;
    const int64_t page = at.page, slot = at.slot;
    const uint8_t *data[2] = {p.k_cache + (page * p.k_cache_stride[0] + slot * p.k_cache_stride[1]), p.v_cache + (page * p.v_cache_stride[0] + slot * p.v_cache_stride[1])};
    const uint8_t *scale[2] = {p.k_scale + (page * p.k_scale_page + slot), p.v_scale + (page * p.v_scale_page + slot)};
    T *out[2] = {static_cast<T *>(p.k) + (tk.s * p.k_stride[0] + tk.t * p.k_stride[1]), static_cast<T *>(p.v) + (tk.s * p.v_stride[0] + tk.t * p.v_stride[1])};
#pragma unroll 4
    for (int pass = first; pass < last; ++pass) {
        const bool value = pass >= p.k_passes;
        const int hd = (value ? pass - p.k_passes : pass) * heads + (lane >> p.lane_bits);
        if (hd >= p.kv_heads) continue;
        const int64_t h = hd;
        float x[kLane];
#pragma unroll
        for (int j = 0; j < kLane; ++j) x[j] = 0.0f;
        if (at.page >= 0) {
            const uint32_t word = *reinterpret_cast<const uint32_t *>(data[value] + (h * (value ? p.v_cache_head : p.k_cache_head) + e0 / 2));
            const uint32_t byte = scale[value][h * (value ? p.v_scale_head : p.k_scale_head) + static_cast<int64_t>(u / 4) * (value ? p.v_scale_block : p.k_scale_block)];
            const float power = __uint_as_float(byte << 23);
            uint32_t two[4];
            two[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, power, 0));
            two[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, power, 1));
            two[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, power, 2));
            two[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, power, 3));
#pragma unroll
            for (int j = 0; j < kLane; ++j) x[j] = __uint_as_float(j % 2 ? two[j / 2] & 0xFFFF0000u : two[j / 2] << 16);
        }
        store8<T, WIDE>(out[value] + h * (value ? p.v_head : p.k_head) + e0, x);
    }
}

int lane_bits_of(int head_dim)
{
    int bits = 2;                                                      // a block's four lanes at least
    while ((kLane << bits) < head_dim) ++bits;
    return bits;
}

}  // namespace

static int passes_of(int heads, int lane_bits) { return (heads + (64 >> lane_bits) - 1) / (64 >> lane_bits); }

hipError_t launch_packed_append(const PackedAppendProblem &given, int dtype, bool wide, hipStream_t stream)
{
    PackedAppendProblem p = given;
    p.lane_bits = lane_bits_of(p.head_dim);
    p.q_passes = passes_of(p.heads, p.lane_bits);
    p.k_passes = passes_of(p.kv_heads, p.lane_bits);
    p.passes = p.q_passes + 2 * p.k_passes;
    // Few tokens: a wave takes one pass.  Many: all of a token's, which then needs its sines and cosines once.  All / 4 / 2 / 1 of 12 passes a wave, 5 prompts of up to 4001
    // tokens: 83 / 89 / 107 / 157 us.
    p.slice = p.tokens_all >= 8 * compute_units() ? p.passes : 1;
    const int slices = (p.passes + p.slice - 1) / p.slice;
    p.by_slices = Divider::of(slices);
    const int64_t grid = (static_cast<int64_t>(p.tokens_all) * slices + kWaves - 1) / kWaves;
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
    p.k_passes = passes_of(p.kv_heads, p.lane_bits);
    p.slice = p.tokens_all >= 8 * compute_units() ? 2 * p.k_passes : 1;
    const int slices = (2 * p.k_passes + p.slice - 1) / p.slice;
    p.by_slices = Divider::of(slices);
    const int64_t grid = (static_cast<int64_t>(p.tokens_all) * slices + kWaves - 1) / kWaves;
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
