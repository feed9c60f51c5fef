// Attention of new queries over a paged cache whose entries are held in 4 bits.
//
//   out = sum_j w_j v_j / sum_j w_j,   w_j = 2^(c <q, k_j> - m),   c = scale log2(e),
// in one pass over the keys with a running reference m per query, as over a cache of 16 or 32 bits (see there): units, rows, parts and the
// join of parts are the same.
//
// A block of 32 entries is 16 bytes and one power of two.  One instruction makes two bfloat16 values of two codes and the power, exactly, so
// keys and values reach the matrix instructions as bfloat16 without a rounding.  A float32 query is the sum of three bfloat16 values (8 bits
// each, cut off and not rounded, so that nothing is lost and nothing overflows), and so is a float32 weight: three products have 24 bits.
//
// A wave takes tiles of 32 keys straight into registers: 16 neighbouring lanes hold one block of 16 keys each, the other lanes the keys' other
// blocks, so a load instruction covers 16 whole keys, and what a lane decodes is what it multiplies.  The product is formed as keys x rows: a
// lane then has scores of one row (lane % 16) and 8 adjacent keys (run lane / 16), the layout in which the second product (values^T x weights)
// takes its right operand.  Of the values a lane takes 8 adjacent entries (4 for heads of 64 and less) of the 8 keys of its run, one word a key, and the 8
// keys' powers in one load (they lie next to each other).
//
// SHARED: the waves of a workgroup have the same rows, take the tiles in turn and join at the end through LDS: four of them, or as many as a compute unit holds where there is
// about one workgroup for each.  Else every wave has rows of its own and walks all tiles by itself; no barrier anywhere, and the waves of a workgroup find each other's tiles in the cache.
//
// What bounds it (heads of 128, 32 on 8 kv heads, bfloat16, unless said).  4 sequences of 131072 tokens: the reads, 570 MB in 104 + 5 us, 5.5 TB/s.  32 prefixes of up to 2048 tokens with 8
// drafts, a query each: 26 us for 43 MB; the start (positions, rows, queries, table, 3.5 us) and the join in LDS (2 us) stand beside 4 to 8 tiles a wave, each of which
// waits for its loads.  8 prefixes of up to 4096 tokens, 8 drafts, 9 queries each (32 rows at once): 47 + 8 us for 19 GFLOP.  Their 72 stretches of rows a prefix fill the card's 512 places, so each prefix is
// one part: nothing is split, the longest prefix's workgroups end the launch (1.3 waves a SIMD on average where 2 have room, the matrix unit busy for 13 % of the time, vector issue for 38 %), and the
// form of parts only costs: 9.4 MB of partial sums and the join that copies them, 8 us.  With 64 rows at once a tile takes
// a wave 4000 cycles, of which 1024 are the matrix unit's: scores 1270, weights 1310, values 1110 follow each other, and two waves a SIMD (the sums are 128 registers) cover little of it.
// 24 float32 sequences, 5 queries of 14 heads on 2 kv heads of 64, window 1000: 13 us for 2 tiles a wave; what the start, the tiles (three products an operand) and the join of 16 waves take of it was not
// measured apart.  One query of 200 tokens: 5.5 us, all latency.  Heads of 32 run as heads of 64, half of whose products are of zeros.
#pragma once

#include "specgbv_attend.hpp"

namespace specgbv {
namespace {

template <int DP> struct Packed {
    static constexpr int kSteps = DP / 32;                   // products of 32 entries, 8 a lane
    static constexpr int kPieces = DP == 256 ? 2 : 1;        // blocks of a key that a lane takes (heads of 64 and less: half a block)
    static constexpr int kWords = kSteps / kPieces;          // 8 entries each
    static constexpr int kVec = DP >= 128 ? 8 : 4;           // adjacent entries of a value that a lane takes
    static constexpr int kGroups = DP / (16 * kVec);         // such runs of entries
    static constexpr int kCols = kGroups * kVec;             // result tiles of 16 entries

    // First entry of a lane's step, the byte its piece starts at, and the piece's block.
    __device__ static constexpr int entry(int i, int quad) { return DP == 64 ? 16 * quad + 8 * i : 32 * (quad + 4 * (i >> 2)) + 8 * (i & 3); }
    __device__ static constexpr int byte(int n, int quad) { return DP == 64 ? 8 * quad : 16 * (quad + 4 * n); }
    __device__ static constexpr int block(int n, int quad) { return DP == 64 ? quad >> 1 : quad + 4 * n; }
};
constexpr int kTile = 32, kRunKeys = 8;
constexpr float kVast = 1048576.0f;           // references beyond it: c <q, k> is rounded as the reference was, before the difference

// Whether a workgroup's queries stand in LDS and not in registers: where so many rows or operands would leave few waves.  (Waves with rows of their own hold theirs.)  Registers / LDS, us: float32 heads of 256
// (2 waves a SIMD instead of 1), 64 sequences of 72 rows 75 / 59 at 1024 tokens, 190 / 149 at 4096, 32 of 8 rows 25 / 23 and, at 3000, 39 / 36, one query of 8 sequences 17.0 / 16.8; not so bfloat16 heads of 256 (3
// instead of 2), 64 of 72 rows 43 / 39 and 109 / 94, but 32 of 8 rows 16.4 / 17.0 and, at 3000, 28.5 / 31.9, one query of 8 sequences 12.6 / 13.3; nor float32 heads of 128 (4 instead of 3), 32 of 85
// rows 32 / 31 and 84 / 88, 64 of 4 22 / 22 and 71 / 75.
constexpr bool queries_in_lds(int element_bytes, int DP, int RT) { return RT == 4 || (element_bytes == 4 && DP == 256); }

// Waves per SIMD that the registers of rows, sums and a tile leave room for; alone: of waves with rows of their own.
constexpr int packed_waves(int element_bytes, int DP, int RT, bool alone = false)
{
    if (element_bytes == 4) return DP == 64 ? 4 : (DP == 128 ? 3 : (alone ? 1 : 2));
    return DP == 256 ? 2 : (RT == 1 ? 4 : RT == 2 && DP == 64 ? 3 : 2);
}

// Waves of a workgroup that has a compute unit for itself (4: there is none but the usual one).
constexpr int packed_wide(int element_bytes, int DP, int RT)
{
    const int waves = packed_waves(element_bytes, DP, RT);
    return RT == 4 || waves == 1 ? 4 : (waves >= 4 ? 16 : 8);
}

// Most tiles of 16 rows that a wave takes: more pay for bfloat16 heads of up to 128 only.  Two for one, us: float32, 200 sequences of 36 rows, heads of 64, 73 / 54 at 1024 tokens, 199 / 152 at 4096; 32 of 85
// rows, heads of 128, 57 / 34 and 150 / 89 (one wave a SIMD); bfloat16 heads of 256, 64 of 72 rows 53 / 43 and 130 / 109, 128 of 68 79 / 66 and 214 / 195.
constexpr int rows_tall(int element_bytes, int DP) { return element_bytes == 4 || DP == 256 ? 1 : 4; }

// Two entries of a word (byte SEL) at a power of two, whose exponent stands in bits 23 to 30; the other bits are of no matter, an exponent of
// all ones gives NaN.
template <int SEL> __device__ __forceinline__ uint32_t decoded(uint32_t word, uint32_t power)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, __uint_as_float(power), SEL));
}
__device__ __forceinline__ U4 decoded8(uint32_t word, uint32_t power)
{
    return U4{decoded<0>(word, power), decoded<1>(word, power), decoded<2>(word, power), decoded<3>(word, power)};
}
__device__ __forceinline__ uint32_t decoded_at(uint32_t word, uint32_t power, int sel)      // (sel is a constant where this is unrolled)
{
    return sel == 0 ? decoded<0>(word, power) : sel == 1 ? decoded<1>(word, power) : sel == 2 ? decoded<2>(word, power) : decoded<3>(word, power);
}

__device__ __forceinline__ F4 product(U4 a, U4 b, F4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(B8, a), __builtin_bit_cast(B8, b), c, 0, 0, 0);
}

// The upper halves of two floats in one word, the first in the low bits.
__device__ __forceinline__ uint32_t upper_halves(float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); }
__device__ __forceinline__ float cut_to_bf16(float x) { return __uint_as_float(__float_as_uint(x) & 0xFFFF0000u); }

// Eight floats as N bfloat16 operands whose sum they are (N = 3), or rounded (N = 1).
template <int N> __device__ __forceinline__ void operands(const float (&x)[8], U4 (&o)[N])
{
    if constexpr (N == 1) {
        B8 b;
#pragma unroll
        for (int k = 0; k < 8; ++k) b[k] = static_cast<__bf16>(x[k]);
        o[0] = __builtin_bit_cast(U4, b);
    } else {
        float rest[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) rest[k] = x[k];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = upper_halves(rest[2 * j], rest[2 * j + 1]);
            o[n] = U4{w[0], w[1], w[2], w[3]};
#pragma unroll
            for (int k = 0; k < 8; ++k) rest[k] -= cut_to_bf16(rest[k]);
        }
    }
}

// WAVES: of a workgroup that share its rows; 0: each of four by itself.
template <typename T, int DP, int RT, int WAVES, bool PARTS, int PAGES, typename Off>
__global__ void __launch_bounds__(WAVES > 0 ? WAVES * 64 : kAttendThreads, (packed_waves(sizeof(T), DP, RT, WAVES == 0))) k_packed_attend(PackedProblem pk)
{
    constexpr bool SHARED = WAVES > 0, kOwn = PARTS || WAVES > kWavesPerGroup;      // kOwn: drafts may share keys and have keys of their own
    using S = Packed<DP>;
    constexpr int kSteps = S::kSteps, kPieces = S::kPieces, kWords = S::kWords, kVec = S::kVec, kGroups = S::kGroups, kCols = S::kCols,
                  N = sizeof(T) == 2 ? 1 : 3;
    constexpr bool kQueriesInLds = WAVES > 0 && queries_in_lds(sizeof(T), DP, RT);
    const AttendProblem &p = pk.a;
    __shared__ F4 sh_acc[SHARED ? WAVES * RT * kGroups * 4 * 64 : 1];
    __shared__ float sh_m[SHARED ? WAVES : 1][RT * 16], sh_l[SHARED ? WAVES : 1][RT * 16];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, quad = lane >> 4;

    // ---- which rows, which keys.  Workgroups that read the same keys are 8 apart: on one XCD, by strips of pk.by_strip of them.
    const int set = pk.by_strip.div(static_cast<int>(blockIdx.x >> 3));
    const int group_at = (set * 8 + static_cast<int>(blockIdx.x & 7)) * static_cast<int>(pk.by_strip.d) + pk.by_strip.mod(static_cast<int>(blockIdx.x >> 3), set);
    const int at_all = SHARED ? group_at : group_at * kWavesPerGroup + wave;
    const int item = p.by_blocks.div(at_all), block = p.by_blocks.mod(at_all, item);
    if (item >= p.items) return;                              // (SHARED: the same for the whole workgroup)
    const int rest = p.by_kv_heads.div(item), head0 = p.by_kv_heads.mod(item, rest);
    const int held = static_cast<int>(capacity_of(p.map));
    Share share{rest, 0, 1, rest, 0};
    if (PARTS) {
        share = share_of(p, rest, held, lane);
        if (share.unit < 0) return;                           // (the same)
        if (p.balanced && share.part == 0 && head0 == 0 && block == 0 && lane == 0 && (!SHARED || wave == 0)) p.places[share.unit] = make_int2(share.at, share.parts);
    }
    const int unit = share.unit, part = share.part;
    const int first = unit * p.drafts;                        // its first sequence
    const int in_draft = p.tokens * p.group, rows = in_draft * p.drafts;
    const int row0 = block * 16 * RT, row_end = min(rows, row0 + 16 * RT);
    const int shared = p.shared_len ? max(0, min(p.shared_len[unit], held)) : held;

    // Rows behind the last one take its place (their loads are those of the last row) and are nowhere stored.
    int64_t q_at[RT];
    int pos[RT], draft[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row = min(row0 + r * 16 + col, row_end - 1);
        draft[r] = p.by_in_draft.div(row);
        const int in = p.by_in_draft.mod(row, draft[r]), t = p.by_group.div(in), head = head0 * p.group + p.by_group.mod(in, t), s = first + draft[r];
        pos[r] = p.positions[s * p.positions_stride + t];
        q_at[r] = s * p.q_stride[0] + t * p.q_stride[1] + head * p.q_stride[2];
    }

    // ---- queries
    static_assert(!kQueriesInLds || RT <= WAVES, "a wave brings one tile of 16 rows to LDS");
    U4 qf[kQueriesInLds ? 1 : RT][kQueriesInLds ? 1 : kSteps][N];
    U4 *q_lds = reinterpret_cast<U4 *>(sh_acc) + lane;
    const T *q = static_cast<const T *>(p.q);
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        if (kQueriesInLds && r != wave) continue;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            const int e = S::entry(i, quad);
            const bool there = e < p.head_dim;
            const T *src = q + q_at[r] + (there ? e : 0);
            U4 (&mine_q)[N] = qf[kQueriesInLds ? 0 : r][kQueriesInLds ? 0 : i];
            if constexpr (N == 1) {
                U4 w;
                if (p.q_wide) w = *reinterpret_cast<const U4 *>(src);
                else w = U4{src[0] | static_cast<uint32_t>(src[1]) << 16, src[2] | static_cast<uint32_t>(src[3]) << 16,
                            src[4] | static_cast<uint32_t>(src[5]) << 16, src[6] | static_cast<uint32_t>(src[7]) << 16};
                if (!there) w = U4{0, 0, 0, 0};
                mine_q[0] = w;
            } else {
                float x[8];
                if (p.q_wide) {
                    const F4 lo = *reinterpret_cast<const F4 *>(src), hi = *reinterpret_cast<const F4 *>(src + 4);
#pragma unroll
                    for (int k = 0; k < 4; ++k) { x[k] = lo[k]; x[4 + k] = hi[k]; }
                } else
#pragma unroll
                    for (int k = 0; k < 8; ++k) x[k] = src[k];
#pragma unroll
                for (int k = 0; k < 8; ++k) if (!there) x[k] = 0.0f;
                operands<N>(x, mine_q);
                // (what is not finite is in the first operand alone, as a whole; the others would make NaN of an infinity)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t bits = __float_as_uint(x[2 * j + h]), mine = h ? 0xFFFF0000u : 0x0000FFFFu;
                        if ((bits & 0x7F800000u) == 0x7F800000u) {
                            uint32_t *o0 = &mine_q[0].x + j, *o1 = &mine_q[1].x + j, *o2 = &mine_q[2].x + j;
                            if (bits & 0x007FFFFFu) *o0 |= 0x00400040u & mine;
                            *o1 &= ~mine; *o2 &= ~mine;
                        }
                    }
            }
            if constexpr (kQueriesInLds)
#pragma unroll
                for (int n = 0; n < N; ++n) q_lds[((r * kSteps + i) * N + n) * 64] = mine_q[n];
        }
    }
    if constexpr (kQueriesInLds) __syncthreads();
#pragma unroll
    for (int r = 0; r < RT; ++r)
        if (row0 + r * 16 + col >= row_end) pos[r] = -1;

    F4 acc[RT][kCols];
    float ref[RT], sum[RT];                                   // sum: over the lane's own keys
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        ref[r] = -INFINITY; sum[r] = 0.0f;
#pragma unroll
        for (int c = 0; c < kCols; ++c) acc[r][c] = F4{0, 0, 0, 0};
    }

    // ---- the keys: one stretch of the unit's, or each draft's own ones in turn
    const uint8_t *kb = static_cast<const uint8_t *>(p.k) + head0 * static_cast<int64_t>(p.k_head_stride);
    const uint8_t *vb = static_cast<const uint8_t *>(p.v) + head0 * static_cast<int64_t>(p.v_head_stride);
    const uint8_t *ksb = pk.k_scale + head0 * static_cast<int64_t>(pk.k_scale_head_stride);
    const uint8_t *vsb = pk.v_scale + head0 * static_cast<int64_t>(pk.v_scale_head_stride);
    const int run_k = col >> 2, in_run = col & 3;             // row m of the product is key 8 (m / 4) + 4 h + m % 4 of the tile
    const int blocks = p.head_dim / 32;
    // A tile's keys lie in PAGES pages at most (page_size a multiple of the keys between, a chunk).  What differs between the lanes of a chunk stays
    // the same for all tiles.
    constexpr int kChunk = kTile / PAGES, kRuns = kChunk / kRunKeys;
    uint32_t k_byte[kPieces], v_byte[kGroups], ks_at[kPieces], vs_at[kGroups];
#pragma unroll
    for (int n = 0; n < kPieces; ++n) {
        const bool there = S::block(n, quad) < blocks;
        const uint32_t key = run_k % kRuns * kRunKeys + in_run;
        k_byte[n] = key * p.k_token_stride + (there ? S::byte(n, quad) : 0);
        ks_at[n] = static_cast<uint32_t>(there ? S::block(n, quad) : 0) * pk.k_scale_block_stride + key;
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        const int e = (g * 16 + col) * kVec;
        const uint32_t key = quad % kRuns * kRunKeys;
        v_byte[g] = key * p.v_token_stride + (e < p.head_dim ? e / 2 : 0);
        vs_at[g] = static_cast<uint32_t>(e < p.head_dim ? e / 32 : 0) * pk.v_scale_block_stride + key;
    }

    // the drafts' own keys, behind the shared ones: the unit's parts take the drafts in turn, and so do the waves of a workgroup that share its rows
    const int draft0 = p.by_in_draft.div(row0), draft1 = p.by_in_draft.div(row_end - 1) + 1;       // drafts with rows here
    const int own_to = !kOwn || !p.shared_len ? 0 : draft1;
    const int own_from = draft0 + WAVES * part + wave, own_step = WAVES * share.parts;
    bool any = draft0 + WAVES * part < own_to;        // something may have been summed (the same for waves that share their rows)
    bool vast = false;                                        // a row of this wave has, or had, a reference beyond kVast
#pragma unroll 1
    for (int seg = -1; seg < own_to; seg = seg < 0 ? own_from : seg + own_step) {
    const bool own = seg >= 0;                                // -1: what the unit's sequences share
    const bool turns = SHARED && !own;                        // the waves take the tiles in turn
    const int step = turns ? WAVES * kTile : kTile;
    const int sequence = first + max(seg, 0);
    int row_low[RT], row_high[RT];
    int lo_all = INT32_MAX, lo_most = -1, hi_all = 0, hi_least = INT32_MAX;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        row_low[r] = row_high[r] = 0;
        if (pos[r] >= 0 && (!own || draft[r] == seg)) {
            row_low[r] = max(own ? shared : 0, p.window > 0 ? pos[r] - (p.window - 1) : 0);
            row_high[r] = min(own ? held : shared, pos[r] < INT32_MAX ? pos[r] + 1 : pos[r]);
            if (row_high[r] <= row_low[r]) row_low[r] = row_high[r] = hi_least = 0;       // sees nothing here: no tile is whole
            else {
                lo_all = min(lo_all, row_low[r]); lo_most = max(lo_most, row_low[r]);
                hi_all = max(hi_all, row_high[r]); hi_least = min(hi_least, row_high[r]);
            }
        } else if (pos[r] >= 0) hi_least = 0;
    }
    lo_all = rows_least(lo_all); hi_least = rows_least(hi_least);
    lo_most = rows_most(lo_most); hi_all = rows_most(hi_all);
    int start = lo_all >= hi_all ? 0 : lo_all / kTile * kTile, end = lo_all >= hi_all ? 0 : hi_all;
    if (PARTS && !own) {
        // parts of the planned length, or longer ones where the sequence is longer than was planned for; with drafts' own keys, which come
        // on top, of one length
        const int span = end - start, least = (span + share.parts - 1) / share.parts;
        const int length = max(p.shared_len ? 0 : share.length, (least + step - 1) / step * step);
        const int64_t at = start + static_cast<int64_t>(part) * length;
        start = static_cast<int>(min(at, static_cast<int64_t>(end)));
        end = static_cast<int>(min(at + length, static_cast<int64_t>(end)));
    }
    any = any || start < end;
    int tile = start + (turns ? wave * kTile : 0);

    // The places of a tile's chunks: page_size is a multiple of a chunk, and so is where a tile starts.  Chunks behind the last key take the last one's
    // place, so that nothing is read outside pages that hold keys; their scores are masked.  All of it is the same for the whole wave: scalar loads and arithmetic.
    struct Pages { int page[PAGES]; };
    const ConstTable row_table = reinterpret_cast<ConstTable>(reinterpret_cast<uintptr_t>(p.map.table + sequence * p.map.table_stride));
    auto chunk_key = [&](int t, int r) { return min(t + r * kChunk, (end - 1) / kChunk * kChunk); };
    auto pages_of = [&](int t) {                              // as they stand in the table: nothing waits for them here
        Pages at;
#pragma unroll
        for (int r = 0; r < PAGES; ++r) at.page[r] = row_table[p.map.page.div(chunk_key(t, r))];
        return at;
    };
    struct Where { Off k[PAGES], ks[PAGES], v[PAGES], vs[PAGES]; uint32_t lost; };        // where the chunks begin; lost: a bit for each that has no page
    auto where = [&](const Pages &at, int t, bool there) {
        Where o;
        o.lost = 0;
#pragma unroll
        for (int r = 0; r < PAGES; ++r) {
            const int key = chunk_key(t, r);
            const bool held_page = static_cast<uint32_t>(at.page[r]) < static_cast<uint32_t>(p.map.pages);
            const Off page = held_page && there ? at.page[r] : 0, slot = there ? p.map.page.mod(key, p.map.page.div(key)) : 0;
            o.k[r] = page * static_cast<uint32_t>(p.k_page_stride) + slot * static_cast<uint32_t>(p.k_token_stride);
            o.v[r] = page * static_cast<uint32_t>(p.v_page_stride) + slot * static_cast<uint32_t>(p.v_token_stride);
            o.ks[r] = page * static_cast<uint32_t>(pk.k_scale_page_stride) + slot;
            o.vs[r] = page * static_cast<uint32_t>(pk.v_scale_page_stride) + slot;
            o.lost |= held_page ? 0u : 1u << r;
        }
        return o;
    };
    auto of_run = [&](const Off (&x)[PAGES], int run) {       // of the chunk that a run lies in
        if constexpr (PAGES == 1) return x[0];
        else if constexpr (PAGES == 2) {
            const bool upper = run & 2;
            const Off lo = x[0], hi = x[1];
            return upper ? hi : lo;
        }
        else {
            const bool odd = run & 1, upper = run & 2;
            const Off lo = odd ? x[1] : x[0], hi = odd ? x[3] : x[2];
            return upper ? hi : lo;
        }
    };
    // (PAGES = 1: the chunk's place is scalar, and the lanes' offsets never change)
    auto at_lane = [&](const uint8_t *base, Off chunk, uint32_t mine) {
        if constexpr (PAGES == 1) return base + chunk + mine;
        else return base + static_cast<Off>(chunk + mine);
    };
    uint32_t kw[2][kSteps], ks[2][kPieces];                   // words of the lane's two keys, and their blocks' powers
    uint32_t vw[kRunKeys][kGroups];                           // of the lane's run of keys
    uint2 vs[kGroups];
    // (`there` false: the loads go to one place and nobody uses them.  They are issued all the same, or the waits for what was loaded
    // before them would have to allow for their absence and wait for everything.)
    auto load_keys = [&](const Where &at) {
        const Off data = of_run(at.k, run_k), scale = of_run(at.ks, run_k);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint8_t *keys = kb + 4 * h * static_cast<int64_t>(p.k_token_stride), *powers = ksb + 4 * h;
#pragma unroll
            for (int n = 0; n < kPieces; ++n) {
                struct alignas(4 * kWords) Words { uint32_t w[kWords]; };
                const Words v = *reinterpret_cast<const Words *>(at_lane(keys, data, k_byte[n]));
#pragma unroll
                for (int i = 0; i < kWords; ++i) kw[h][n * kWords + i] = v.w[i];
                ks[h][n] = *at_lane(powers, scale, ks_at[n]);
            }
        }
    };
    auto load_values = [&](Off data, Off scale) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
#pragma unroll
            for (int k = 0; k < kRunKeys; ++k) {
                const uint8_t *src = at_lane(vb + k * static_cast<int64_t>(p.v_token_stride), data, v_byte[g]);
                if constexpr (kVec == 8) vw[k][g] = *reinterpret_cast<const uint32_t *>(src);
                else vw[k][g] = *reinterpret_cast<const uint16_t *>(src);
            }
            vs[g] = *reinterpret_cast<const uint2 *>(at_lane(vsb, scale, vs_at[g]));
        }
    };

    Pages next{};
    uint32_t lost_runs = 0;
    if (tile < end) {
        const Where at = where(pages_of(tile), tile, true);
        load_keys(at);
        load_values(of_run(at.v, quad), of_run(at.vs, quad));
        lost_runs = at.lost;
        next = pages_of(tile + step);                         // (behind the end: the last run's page)
    }
#pragma unroll 1
    for (; tile < end; tile += step) {
        const bool more = tile + step < end;
        // scores: keys x rows
        F4 s[RT][2];
#pragma unroll
        for (int r = 0; r < RT; ++r) s[r][0] = s[r][1] = F4{0, 0, 0, 0};
        if (p.head_dim != DP) {
#pragma unroll
            for (int n = 0; n < kPieces; ++n)
                if (S::block(n, quad) >= blocks)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        ks[h][n] = 127;
#pragma unroll
                        for (int i = 0; i < kWords; ++i) kw[h][n * kWords + i] = 0;
                    }
        }
        int again = 0;
        if constexpr (kQueriesInLds) asm volatile("" : "+v"(again));        // (read in every tile: kept over the loop they would be registers)
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            U4 a[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) a[h] = decoded8(kw[h][i], ks[h][i / kWords] << 23);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                U4 b[N];
#pragma unroll
                for (int n = 0; n < N; ++n) {
                    if constexpr (kQueriesInLds) b[n] = q_lds[again + ((r * kSteps + i) * N + n) * 64];
                    else b[n] = qf[r][i][n];
                }
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int n = 0; n < N; ++n) s[r][h] = product(a[h], b[n], s[r][h]);
            }
        }
        const uint32_t lost_here = lost_runs;
        __builtin_amdgcn_sched_barrier(0);
        const Where to_come = where(next, tile + step, more);
        load_keys(to_come);
        const Off v_data = of_run(to_come.v, quad), v_scale = of_run(to_come.vs, quad);
        lost_runs = to_come.lost;
        next = pages_of(tile + 2 * step);
        __builtin_amdgcn_sched_barrier(0);

        // weights
        const bool lost = lost_here >> quad / kRuns & 1;
        const bool partial = tile < lo_most || tile + kTile > hi_least || tile + kTile > end || lost_here != 0;
        if (partial) {
            const int base = tile + quad * kRunKeys;
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const int from = max(row_low[r] - base, 0), to = lost ? 0 : min(max(row_high[r] - base, 0), kRunKeys);
#pragma unroll
                for (int k = 0; k < kRunKeys; ++k) s[r][k / 4][k % 4] = k >= from && k < to ? s[r][k / 4][k % 4] : -INFINITY;
            }
        }
        // (all rows' maxima first, and one branch for all: the rows' exponentials then stand side by side)
        float top[RT];
        bool raise = false;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            top[r] = s[r][0][0];
#pragma unroll
            for (int k = 1; k < kRunKeys; ++k) top[r] = fmaxf(top[r], s[r][k / 4][k % 4]);
            top[r] *= p.c;
            raise = raise || top[r] > ref[r] + kRaise;
        }
        if (__any(raise)) {
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                // (row by row: what a row gets does not hang on the rows next to it)
                const float most = row_largest(top[r]);
                const float now = most > ref[r] + kRaise ? most : ref[r];
                const float f = now == ref[r] ? 1.0f : exp2_of(ref[r] - now);        // (-inf to -inf: nothing summed yet)
                vast = vast || __any(fabsf(now) > kVast && now != -INFINITY);
                ref[r] = now;
                sum[r] *= f;
#pragma unroll
                for (int c = 0; c < kCols; ++c) acc[r][c] *= f;
            }
        }
        if (vast) {
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const float m = ref[r] == -INFINITY ? 0.0f : ref[r];
                const bool mine = fabsf(m) > kVast;            // (a row at a time: what the others get is what they get without it)
#pragma unroll
                for (int k = 0; k < kRunKeys; ++k) {
                    float x = s[r][k / 4][k % 4] * p.c;
                    asm volatile("" : "+v"(x));                // (rounded by itself)
                    s[r][k / 4][k % 4] = exp2_of(mine ? x - m : fmaf(s[r][k / 4][k % 4], p.c, -m));
                }
            }
        } else {
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const float m = ref[r] == -INFINITY ? 0.0f : ref[r];
#pragma unroll
                for (int k = 0; k < kRunKeys; ++k) s[r][k / 4][k % 4] = exp2_of(fmaf(s[r][k / 4][k % 4], p.c, -m));
            }
        }
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int k = 0; k < kRunKeys; ++k) sum[r] += s[r][k / 4][k % 4];

        // A value is not finite only where its block's power says so (bytes above 252), and a weight of 0 does not take it out.  In tiles that some rows
        // do not see whole, keys that no row sees are cleared, blocks of the others that are not finite as well, and the rows that do see one get NaN:
        // a product of marks says which.
        if (partial) {
            const int base = tile + quad * kRunKeys;
            const int from = min(max(lo_all - base, 0), kRunKeys), to = lost ? 0 : min(max(hi_all - base, 0), kRunKeys);
            uint32_t seen = to > from ? ((1u << to) - 1u) & ~((1u << from) - 1u) : 0u;
            uint32_t bad[kGroups], some = 0;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                bad[g] = 0;
#pragma unroll
                for (int k = 0; k < kRunKeys; ++k) {
                    uint32_t &word = k < 4 ? vs[g].x : vs[g].y;
                    const uint32_t over = (word >> 8 * (k % 4) & 255u) > 252u ? 1u : 0u;
                    if (over || !(seen >> k & 1)) {
                        word = (word & ~(255u << 8 * (k % 4))) | 127u << 8 * (k % 4);
                        vw[k][g] = 0;
                    }
                    bad[g] |= (over & (seen >> k)) << k;
                }
                some |= bad[g];
            }
            if (__any(some != 0)) {
#pragma unroll 1
                for (int g = 0; g < kGroups; ++g) {
                    const uint32_t mine = kGroups == 1 ? bad[0] : (g == 0 ? bad[0] : bad[kGroups - 1]);
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        const int lo = max(row_low[r] - base, 0), hi = lost ? 0 : min(max(row_high[r] - base, 0), kRunKeys);
                        B8 a, b;
#pragma unroll
                        for (int k = 0; k < kRunKeys; ++k) {
                            a[k] = static_cast<__bf16>(mine >> k & 1 ? 1.0f : 0.0f);
                            b[k] = static_cast<__bf16>(k >= lo && k < hi ? 1.0f : 0.0f);
                        }
                        F4 n{0, 0, 0, 0};
                        n = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, n, 0, 0, 0);
#pragma unroll
                        for (int c = 0; c < kCols; ++c)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (c / kVec == g && n[i] > 0.0f) acc[r][c][i] = NAN;
                    }
                }
            }
        }

        // sums of values: entries x rows.  bfloat16 results: weights are rounded to bfloat16, the values' own type here (see the cache of 16 bits for what
        // that costs); float32: three products.
        U4 w[RT][N];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float x[8];
#pragma unroll
            for (int k = 0; k < kRunKeys; ++k) x[k] = s[r][k / 4][k % 4];
            operands<N>(x, w[r]);
        }
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            uint32_t power[kRunKeys];
#pragma unroll
            for (int k = 0; k < kRunKeys; ++k) {
                const uint32_t word = k < 4 ? vs[g].x : vs[g].y;
                power[k] = k % 4 == 3 ? word >> 1 : word << (23 - 8 * (k % 4));
            }
#pragma unroll
            for (int j = 0; j < kVec / 2; ++j) {
                uint32_t two[kRunKeys];                       // entries 2 j and 2 j + 1 of each key
#pragma unroll
                for (int k = 0; k < kRunKeys; ++k) two[k] = decoded_at(vw[k][g], power[k], j);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t e[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) e[k] = __builtin_amdgcn_perm(two[2 * k + 1], two[2 * k], h ? 0x07060302u : 0x05040100u);
                    const U4 a{e[0], e[1], e[2], e[3]};
#pragma unroll
                    for (int r = 0; r < RT; ++r)
#pragma unroll
                        for (int n = 0; n < N; ++n) acc[r][g * kVec + 2 * j + h] = product(a, w[r][n], acc[r][g * kVec + 2 * j + h]);
                }
            }
        }
        load_values(v_data, v_scale);
    }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) sum[r] = row_total(sum[r]);

    // ---- the waves of a workgroup join: each brings its sums to the largest reference, then wave i adds up the entries i of all
    float inv[RT];
    int64_t at[RT];
    if constexpr (SHARED) {
        if (quad == 0)
#pragma unroll
            for (int r = 0; r < RT; ++r) { sh_m[wave][r * 16 + col] = ref[r]; sh_l[wave][r * 16 + col] = sum[r]; }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float most = -INFINITY, total = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) most = fmaxf(most, sh_m[w][r * 16 + col]);
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float m = sh_m[w][r * 16 + col];
                total += sh_l[w][r * 16 + col] * (m == most ? 1.0f : exp2_of(m - most));
            }
            const float f = ref[r] == most ? 1.0f : exp2_of(ref[r] - most);
            ref[r] = most; sum[r] = total;
#pragma unroll
            for (int c = 0; c < kCols; ++c) acc[r][c] *= f;
        }
    }
    // Partial sums are held in the order in which lanes hold them: vector ((g 4 + i) kVec / 4 + n) 4 + quad of a row are entries
    // (16 g + 4 quad + i) kVec + 4 n + 0..3.  Where nothing was summed they are not written: the sum of weights says so.
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        inv[r] = sum[r] != 0.0f && pos[r] >= 0 ? 1.0f / sum[r] : 0.0f;
        at[r] = PARTS ? (static_cast<int64_t>(share.at + part) * p.kv_heads + head0) * rows + row0 + r * 16 + col : 0;
        if (PARTS && row0 + r * 16 + col < row_end && (!SHARED || wave == 0) && quad == 0) p.ml[at[r]] = make_float2(ref[r], sum[r]);
    }
    if (PARTS && !any) return;                                // (the same for waves that share their rows)
    T *out[RT];
    int row1 = row0;
    asm volatile("" : "+s"(row1));                            // (worked out anew: kept over the loop, the rows' places would be registers)
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row = min(row1 + r * 16 + col, row_end - 1), d = p.by_in_draft.div(row), in = p.by_in_draft.mod(row, d), t = p.by_group.div(in);
        out[r] = static_cast<T *>(p.out) + (PARTS ? 0 : (first + d) * p.out_stride[0] + t * p.out_stride[1] + (head0 * p.group + p.by_group.mod(in, t)) * p.out_stride[2]);
    }
    auto emit = [&](int r, int g, int i, int n, F4 v) {
        const int d = (16 * g + 4 * quad + i) * kVec + 4 * n;
        if (row0 + r * 16 + col >= row_end) return;
        if (PARTS) reinterpret_cast<F4 *>(p.acc + at[r] * DP)[((g * 4 + i) * (kVec / 4) + n) * 4 + quad] = v;
        else if (d < p.head_dim) store_entries(out[r] + d, v, inv[r], p.out_wide);
    };
#pragma unroll
    for (int n = 0; n < kVec / 4; ++n) {
        if constexpr (SHARED) {
            if (n > 0) __syncthreads();
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int g = 0; g < kGroups; ++g)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        sh_acc[(((wave * RT + r) * kGroups + g) * 4 + i) * 64 + lane] =
                            F4{acc[r][g * kVec + 4 * n][i], acc[r][g * kVec + 4 * n + 1][i], acc[r][g * kVec + 4 * n + 2][i], acc[r][g * kVec + 4 * n + 3][i]};
            __syncthreads();
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {
                    if (WAVES > kWavesPerGroup && (r * kGroups + g) % (WAVES / kWavesPerGroup) != wave / kWavesPerGroup) continue;
                    const int i = wave % kWavesPerGroup;
                    F4 v{0, 0, 0, 0};
#pragma unroll
                    for (int w = 0; w < WAVES; ++w) v += sh_acc[(((w * RT + r) * kGroups + g) * 4 + i) * 64 + lane];
                    emit(r, g, i, n, v);
                }
        } else {
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int g = 0; g < kGroups; ++g)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        emit(r, g, i, n, F4{acc[r][g * kVec + 4 * n][i], acc[r][g * kVec + 4 * n + 1][i], acc[r][g * kVec + 4 * n + 2][i], acc[r][g * kVec + 4 * n + 3][i]});
        }
    }
}

template <typename T, int DP, int RT, int WAVES, bool PARTS, int PAGES, typename Off>
hipError_t launch_pages(PackedProblem p, hipStream_t stream)
{
    p.a.items = p.a.all_parts * p.a.kv_heads;
    p.a.by_blocks = Divider::of(p.a.row_blocks);
    const int64_t all = static_cast<int64_t>(p.a.items) * p.a.row_blocks, groups = WAVES > 0 ? all : (all + kWavesPerGroup - 1) / kWavesPerGroup;
    // a strip: the row blocks of an item (of four items where waves have rows of their own), shorter where there would be few strips for 8 XCDs
    int64_t strip = groups / 32 < 1 ? 1 : groups / 32;
    if (strip > p.a.row_blocks) strip = p.a.row_blocks;
    p.by_strip = Divider::of(static_cast<int32_t>(strip));
    const int64_t grid = (groups + 8 * strip - 1) / (8 * strip) * (8 * strip);
    if (grid >= kLaunchGroups) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((k_packed_attend<T, DP, RT, WAVES, PARTS, PAGES, Off>), dim3(static_cast<unsigned>(grid)), dim3(WAVES > 0 ? WAVES * 64 : kAttendThreads), 0, stream, p);
    return hipGetLastError();
}

template <typename T, int DP, int RT, int WAVES, bool PARTS>
hipError_t launch_ways(const PackedProblem &p, hipStream_t stream)
{
    const int page = static_cast<int>(p.a.map.page.d);
    if (page % 32 == 0) return launch_pages<T, DP, RT, WAVES, PARTS, 1, uint64_t>(p, stream);
    if (p.near && page % 16 == 0) return launch_pages<T, DP, RT, WAVES, PARTS, 2, uint32_t>(p, stream);
    if constexpr (WAVES > 0) if (!p.near) return launch_pages<T, DP, RT, WAVES, PARTS, 4, uint64_t>(p, stream);
    return launch_pages<T, DP, RT, WAVES, PARTS, 4, uint32_t>(p, stream);
}

template <typename T, int DP, int RT>
hipError_t launch_tall(const PackedProblem &p, hipStream_t stream)
{
    constexpr int kWide = packed_wide(sizeof(T), DP, RT);
    if (p.a.ml) return launch_ways<T, DP, RT, kWavesPerGroup, true>(p, stream);
    if constexpr (RT < 4)                                      // (64 rows: the waves always share them)
        if (!p.a.few && (p.near || p.a.map.page.d % 32 == 0)) return launch_ways<T, DP, RT, 0, false>(p, stream);
    if constexpr (kWide > kWavesPerGroup)
        if (p.a.few == kWide) return launch_ways<T, DP, RT, kWide, false>(p, stream);
    return launch_ways<T, DP, RT, kWavesPerGroup, false>(p, stream);
}

template <typename T, int DP>
hipError_t launch_typed(const PackedProblem &p, hipStream_t stream)
{
    if (p.a.ml && join_grid<DP>(p.a) >= kLaunchGroups) return hipErrorInvalidConfiguration;
    hipError_t e = hipErrorInvalidValue;
    if (p.a.block_rows == 16) e = launch_tall<T, DP, 1>(p, stream);
    if constexpr (rows_tall(sizeof(T), DP) > 1) {
        if (p.a.block_rows == 32) e = launch_tall<T, DP, 2>(p, stream);
        if (p.a.block_rows == 64) e = launch_tall<T, DP, 4>(p, stream);
    }
    return e != hipSuccess || !p.a.ml ? e : launch_join<T, DP, Packed<DP>::kVec>(p.a, stream);
}

}  // namespace
}  // namespace specgbv
